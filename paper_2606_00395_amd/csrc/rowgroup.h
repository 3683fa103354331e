// Rows held in registers by one wavefront or by the wavefronts of a workgroup together, with their
// sums and maxima.
#pragma once

#include "chunk.h"

namespace pr2 {

// A row of up to 64 NW F elements: piece i of lane t is the row's (t + 64 NW i)-th of 16 bytes.  A last
// piece that would end behind the row is moved back over the one before and read and written
// whole; its first `skip` elements are that one's and count there.
template <typename T, int NW, int F> struct RowGroup {
    static constexpr int E = Chunk<T>::E;
    static constexpr int kLanes = 64 * NW;
    static constexpr int kPieces = F / E;
    static_assert(F % E == 0, "whole pieces");

    int d, lane;
    __device__ __forceinline__ RowGroup(int d_, int lane_) : d(d_), lane(lane_) {}
    __device__ __forceinline__ int column(int i) const { return (lane + i * kLanes) * E; }
    __device__ __forceinline__ bool on(int i) const { return column(i) < d; }
    // Whether any lane of the wavefront has a piece i (a scalar branch).  Rows on 16 wavefronts leave many
    // without one (quantising 3600 rows of 9000 36 -> 30 us); on fewer the branch costs more than it saves.
    __device__ __forceinline__ bool any(int i) const {
        return NW < 16 || __builtin_amdgcn_readfirstlane(column(i)) < d;
    }
    __device__ __forceinline__ bool narrow() const { return d < E; }
    __device__ __forceinline__ int start(int i) const { return max(0, min(column(i), d - E)); }
    __device__ __forceinline__ int skip(int i) const { return column(i) - start(i); }

    // piece i of a row; what lies outside is 0
    template <bool NT = false>
    __device__ __forceinline__ u32x4 load(const T* row, int i) const {
        if (!on(i)) return u32x4{0, 0, 0, 0};
        return narrow() ? load_chunk<T, NT>(row, 0, 0, d) : load16<NT>(row + start(i));
    }
    __device__ __forceinline__ void store(T* row, int i, const u32x4& w) const {
        if (!on(i)) return;
        if (narrow()) copy_chunk<T>(row, 0, 0, d, w);
        else store16<false>(row + start(i), w);
    }
    // without the elements that another piece counts
    __device__ __forceinline__ void store_own(T* row, int i, const u32x4& w) const {
        const int n = skip(i);
        if (n <= 0 || !on(i)) return store(row, i, w);
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (j >= n)
                row[start(i) + j] =
                    __builtin_bit_cast(T, (typename Chunk<T>::Bits)(E == 8 ? w[j / 2] >> (16 * (j & 1)) : w[j]));
    }
    // the same of an fp32 row beside it (which starts at any float)
    __device__ __forceinline__ void load_f32(const float* row, int i, float* v) const {
        typedef f32x4 f32x4_any __attribute__((aligned(4)));
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = 0.0f;
        if (!on(i)) return;
        if (narrow()) {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (j < d) v[j] = row[j];
            return;
        }
#pragma unroll
        for (int j = 0; j < E; j += 4) {
            const f32x4 w = *(const f32x4_any*)(row + start(i) + j);
#pragma unroll
            for (int h = 0; h < 4; ++h) v[j + h] = w[h];
        }
    }
    // 0 in the elements that another piece counts
    __device__ __forceinline__ void mask(int i, float* v) const {
        const int n = skip(i);
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = j < n ? 0.0f : v[j];
    }
};

// the value of another lane by DPP: of lane ^ 1 and lane ^ 2, and of a mirrored lane of 8 and of 16,
// which stands for lane ^ 4 and lane ^ 8 once the lanes of 4 and of 8 are alike
enum { XOR1 = 0xb1, XOR2 = 0x4e, MIRROR8 = 0x141, MIRROR16 = 0x140 };
template <int ctrl>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false);
}
template <int ctrl>
__device__ __forceinline__ double from_lane(double v) {
    return __hiloint2double((int)from_lane<ctrl>((uint32_t)__double2hiint(v)),
                            (int)from_lane<ctrl>((uint32_t)__double2loint(v)));
}
__device__ __forceinline__ uint32_t of_lane(uint32_t v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ double of_lane(double v, int lane) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane),
                            __builtin_amdgcn_readlane(__double2loint(v), lane));
}
struct AddF32 {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }
};
struct AddF64 {
    __device__ __forceinline__ double operator()(double a, double b) const { return a + b; }
};
struct MaxU32 {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); }
};
// over 16 lanes, as a tree of neighbours
template <typename V, typename Op>
__device__ __forceinline__ V reduce16(V v, Op op) {
    v = op(v, from_lane<XOR1>(v));
    v = op(v, from_lane<XOR2>(v));
    v = op(v, from_lane<MIRROR8>(v));
    return op(v, from_lane<MIRROR16>(v));
}

// Over a row of NW wavefronts with P pieces in each lane: every piece over its groups of 16 lanes, each
// group's NW P pieces as a tree of neighbours in the row's order, then the four groups.  Pieces behind the
// row's end are zeros, so the result does not depend on how many wavefronts and pieces hold the row: a
// row's norm has the same bits in any batch.  `red` holds 8 NW MOST values (MOST: the most pieces of a
// reduction in the kernel, in values of this one's type); `turn` alternates, so that one barrier is enough: the values
// of a turn are written again only behind the next turn's barrier, which every wavefront reaches after it read them.
template <int NW, int P, int MOST, typename V, typename Op>
__device__ __forceinline__ V row_reduce(V (&v)[P], V* red, int& turn, Op op) {
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = reduce16(v[i], op);
    V w;
    if (NW == 1) {
#pragma unroll
        for (int n = 1; n < P; n *= 2)
#pragma unroll
            for (int i = 0; i < P; i += 2 * n) v[i] = op(v[i], v[i + n]);
        w = v[0];
    } else {
        constexpr int n = NW * P, M = n < 16 ? 1 : n / 16;      // pieces, and those that a lane joins
        V* r = red + turn * (4 * NW * MOST);
        turn ^= 1;
        const int group = (threadIdx.x & 63) >> 4, at = threadIdx.x & 15;
        if (at == 0) {
#pragma unroll
            for (int i = 0; i < P; ++i) r[4 * (i * NW + (threadIdx.x >> 6)) + group] = v[i];
        }
        __syncthreads();
        V u[M];
#pragma unroll
        for (int m = 0; m < M; ++m) u[m] = at * M + m < n ? r[4 * (at * M + m) + group] : V(0);
#pragma unroll
        for (int q = 1; q < M; q *= 2)
#pragma unroll
            for (int m = 0; m < M; m += 2 * q) u[m] = op(u[m], u[m + q]);
        w = reduce16(u[0], op);
    }
    return op(op(of_lane(w, 0), of_lane(w, 16)), op(of_lane(w, 32), of_lane(w, 48)));
}

// the row's largest magnitude (bits), of its pieces'
template <int NW, int P, int MOST>
__device__ __forceinline__ uint32_t row_max(const uint32_t (&m)[P], uint32_t* red, int& turn) {
    uint32_t one[1] = {m[0]};
#pragma unroll
    for (int i = 1; i < P; ++i) one[0] = max(one[0], m[i]);
    return row_reduce<NW, 1, MOST>(one, red, turn, MaxU32());
}

// The row form of 8 bits: q = rint(v / step), step = fp32(max(m, 2^-100) fp32(1 / 127)) with m (its bits)
// the row's largest magnitude.  (Below 2^-100 the inverse would leave fp32's range.)
struct RowStep {
    float step, inverse;
    bool finite;
};
__device__ __forceinline__ RowStep row_step(uint32_t m_bits) {
    const float m = fmaxf(__uint_as_float(m_bits), 0x1p-100f);
    const bool finite = m_bits < 0x7f800000u;
    return RowStep{finite ? m * (1.0f / 127.0f) : __uint_as_float(0x7fc00000u), finite ? 127.0f / m : 0.0f, finite};
}
// v / step rounded to even as exact arithmetic rounds it: the product with the inverse is off by up to
// 127 3 2^-24, so that next to a half it may take the wrong side.  The remainder v - q step
// is one of fp32's numbers (a multiple of both operands' last places, at most about half a step) and
// tells.
__device__ __forceinline__ float row_round(float v, const RowStep& s) {
    const float q = rintf(v * s.inverse);
    const float rest = __builtin_fmaf(-q, s.step, v), half = 0.5f * s.step;
    const bool odd = (int)q & 1;
    const float up = rest > half || (rest == half && odd) ? 1.0f : 0.0f;
    const float down = rest < -half || (rest == -half && odd) ? 1.0f : 0.0f;
    return q + up - down;
}
__device__ __forceinline__ uint32_t byte_of(float q) {
    return (uint32_t)(int)fminf(fmaxf(q, -127.0f), 127.0f) & 255u;
}
// E elements as bytes, in order (zeros where the row is not finite)
template <int E>
__device__ __forceinline__ void quantise_row(const float* v, const RowStep& s, uint32_t (&q)[E / 4]) {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) w |= byte_of(row_round(v[4 * i + j], s)) << (8 * j);
        q[i] = s.finite ? w : 0u;
    }
}
// the packed form's: multiples of a power of two, whose inverse is exact
template <int E>
__device__ __forceinline__ void quantise_group(const float* v, float inverse, uint32_t (&q)[E / 4]) {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) w |= byte_of(rintf(v[4 * i + j] * inverse)) << (8 * j);
        q[i] = w;
    }
}
// E bytes of a row that starts anywhere
template <int E>
__device__ __forceinline__ void store_bytes(int8_t* p, const uint32_t (&q)[E / 4]) {
    typedef uint32_t u32_byte __attribute__((aligned(1)));
    typedef uint64_t u64_byte __attribute__((aligned(1)));
    if (E == 4) *(u32_byte*)p = q[0];
    else *(u64_byte*)p = (uint64_t)q[0] | (uint64_t)q[E / 4 - 1] << 32;
}

}  // namespace pr2
