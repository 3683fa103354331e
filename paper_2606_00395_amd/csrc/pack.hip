// Activations in 8 bits: int8 multiples of a power of two per group of 32 columns.
//
// The power comes from the exponent of the group's largest magnitude alone, so the values are
// exact in bf16, no rounding depends on the order of anything, and an element costs a multiply
// by an exact power, one rounding to an integer and a byte.  All kernels here are bound by
// HBM: each input is read once in 16-byte pieces and each output written once.  A thread takes
// 16 columns (half a group), so that q moves in 16-byte pieces too, and no second unit: with
// four units in turn SwiGLU took 165 and its backward 211 us where workgroups of 512 with one
// each take 142 and 183 (131072 x 768 bf16, 5.7 and 5.5 TB/s; a large copy reaches 5.2).
// Packing 33.5 M bf16 values and taking them back out: 36 us, 5.6 TB/s.
#include "chunk.h"

namespace pr2 {
namespace {

constexpr int kThreads = 512;
constexpr int kUnit = 16;               // columns per thread
constexpr int kUnits = kThreads;        // units per workgroup, about

typedef u32x4 u32x4_byte __attribute__((aligned(1)));    // int8 rows start anywhere

// A workgroup takes `rows` whole rows of `per` units (or, per > kUnits, one row); a unit's
// row is its index over per by a multiply: exact for indexes below 2^16 and per below 2^16.
struct Tiling {
    int64_t R;
    int rows, per;
    uint32_t magic;         // ceil(2^32 / per); 0 with one row per workgroup (and unused at per = 1)
    uint32_t across;        // the grid's first dimension (asked of the grid, 16384 x 2048 take 36.0 us for 35.4)
};

dim3 grid_of(const Tiling& t) { return wide_grid((t.R + t.rows - 1) / t.rows, kThreads); }

Tiling tiling(int64_t R, int64_t per) {
    Tiling t{};
    t.R = R;
    t.per = (int)per;
    t.rows = per >= kUnits ? 1 : (int)(kUnits / per);
    t.magic = t.rows == 1 ? 0 : (uint32_t)(((1ull << 32) + per - 1) / per);
    t.across = grid_of(t).x;
    return t;
}

struct Unit {
    int64_t row;
    int u;
};
__device__ __forceinline__ Unit unit_of(const Tiling& t, int i) {
    const int r = t.per == 1 ? i : (int)__umulhi((uint32_t)i, t.magic);
    return Unit{(int64_t)(blockIdx.x + blockIdx.y * t.across) * t.rows + r, i - r * t.per};
}

// 16 elements at p, the first n of them inside the row (zeros for the others)
template <typename T, bool NT = false>
__device__ __forceinline__ void load_unit(const T* p, int n, float (&v)[kUnit]) {
    constexpr int E = Chunk<T>::E;
    if (n >= kUnit) {
        u32x4 w[kUnit / E];
#pragma unroll
        for (int i = 0; i < kUnit / E; ++i) w[i] = load16<NT>(p + i * E);
#pragma unroll
        for (int i = 0; i < kUnit / E; ++i) Chunk<T>::open(w[i], v + i * E);
    } else {
#pragma unroll
        for (int i = 0; i < kUnit; ++i) v[i] = i < n ? Act<T>::to_f32(p[i]) : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store_unit(T* p, int n, const float (&v)[kUnit]) {
    constexpr int E = Chunk<T>::E;
    if (n >= kUnit) {
#pragma unroll
        for (int i = 0; i < kUnit / E; ++i) store16<false>(p + i * E, Chunk<T>::close(v + i * E));
    } else {
#pragma unroll
        for (int i = 0; i < kUnit; ++i)
            if (i < n) p[i] = Act<T>::from_f32(v[i]);
    }
}

// The scale byte of a group whose two units lie in lanes 2 i and 2 i + 1.  The largest
// magnitude is taken on the bits: a NaN is above every number then, and is seen.
__device__ __forceinline__ uint32_t group_scale(const float (&v)[kUnit]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kUnit; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, false));
    const int e = (int)(m >> 23);
    return e == 255 ? 255u : (uint32_t)max(e - 6, 1);
}

__device__ __forceinline__ float scale_step(uint32_t byte) { return __uint_as_float(byte << 23); }

__device__ __forceinline__ u32x4 quantise(const float (&v)[kUnit], uint32_t byte) {
    u32x4 w = {0, 0, 0, 0};
    if (byte == 255u) return w;
    const float inv = __uint_as_float((254u - byte) << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float q = fminf(fmaxf(rintf(v[4 * i + j] * inv), -127.0f), 127.0f);
            w[i] |= ((uint32_t)(int)q & 255u) << (8 * j);
        }
    }
    return w;
}

__device__ __forceinline__ float byte_value(uint32_t w, int j) {
    return (float)((int)(w << (24 - 8 * j)) >> 24);
}

// q and the values of 16 columns; n as in load_unit
__device__ __forceinline__ u32x4 load_q(const int8_t* p, int n) {
    if (n >= kUnit) return *(const u32x4_byte*)p;
    u32x4 w = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kUnit; ++i)
        if (i < n) w[i / 4] |= (uint32_t)(uint8_t)p[i] << (8 * (i % 4));
    return w;
}

__device__ __forceinline__ void store_q(int8_t* p, int n, const u32x4& w) {
    if (n >= kUnit) {
        *(u32x4_byte*)p = w;
    } else {
#pragma unroll
        for (int i = 0; i < kUnit; ++i)
            if (i < n) p[i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
    }
}

// The values of columns c .. c + 15 of a row whose scales start at e: one group (WITHIN: c is
// a multiple of 16) or two.
template <bool WITHIN>
__device__ __forceinline__ void load_values(const int8_t* q, const uint8_t* e, int c, int n,
                                            float (&v)[kUnit]) {
    const u32x4 w = load_q(q + c, n);
    const float s0 = scale_step(e[c / 32]);
    const float s1 = WITHIN || n <= 0 ? s0 : scale_step(e[(c + min(n, kUnit) - 1) / 32]);
#pragma unroll
    for (int i = 0; i < kUnit; ++i)
        v[i] = byte_value(w[i / 4], i % 4) * (WITHIN || (c + i) / 32 == c / 32 ? s0 : s1);
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
act_pack_kernel(Tiling t, int C, int64_t groups, const T* x, int8_t* q, uint8_t* scale) {
    for (int i = threadIdx.x; i < t.rows * t.per; i += kThreads) {      // (per is even)
        const Unit at = unit_of(t, i);
        if (at.row >= t.R) continue;
        const int c = at.u * kUnit, n = C - c;
        float v[kUnit];
        load_unit<T, true>(x + at.row * C + c, n, v);      // read once
        const uint32_t byte = group_scale(v);
        if (n > 0) store_q(q + at.row * C + c, n, quantise(v, byte));
        if ((at.u & 1) == 0) scale[at.row * groups + at.u / 2] = (uint8_t)byte;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
act_unpack_kernel(Tiling t, int C, int64_t groups, const int8_t* q, const uint8_t* scale, T* x) {
    for (int i = threadIdx.x; i < t.rows * t.per; i += kThreads) {
        const Unit at = unit_of(t, i);
        if (at.row >= t.R) continue;
        const int c = at.u * kUnit, n = C - c;
        float v[kUnit];
        load_values<true>(q + at.row * C, scale + at.row * groups, c, n, v);
        store_unit(x + at.row * C + c, n, v);
    }
}

// As the layer's own silu, also in fp32: within 1e-6 (1 + |a|) relatively, where an exact exponential
// and division reach 2e-7, and 0 below 2^-126.
__device__ __forceinline__ float sigmoid(float a) {
    return __builtin_amdgcn_rcpf(1.0f + __expf(-a));
}

// h = silu(a) u; with PACK (m a multiple of 32) the packed form of a and u as well
template <typename T, bool PACK>
__global__ void __launch_bounds__(kThreads)
swiglu_kernel(Tiling t, int m, int64_t groups, const T* au, T* h, int8_t* q, uint8_t* scale) {
    for (int i = threadIdx.x; i < t.rows * t.per; i += kThreads) {
        const Unit at = unit_of(t, i);
        if (at.row >= t.R) continue;
        const int c = at.u * kUnit, n = m - c;
        const T* p = au + at.row * (2 * (int64_t)m) + c;
        float a[kUnit], u[kUnit];
        load_unit(p, n, a);
        load_unit(p + m, n, u);
        if (PACK) {
            const uint32_t ba = group_scale(a), bu = group_scale(u);
            int8_t* qp = q + at.row * (2 * (int64_t)m) + c;
            store_q(qp, n, quantise(a, ba));
            store_q(qp + m, n, quantise(u, bu));
            if ((at.u & 1) == 0) {
                uint8_t* e = scale + at.row * groups + at.u / 2;
                e[0] = (uint8_t)ba;
                e[m / 32] = (uint8_t)bu;
            }
        }
#pragma unroll
        for (int j = 0; j < kUnit; ++j) a[j] = a[j] * sigmoid(a[j]) * u[j];
        store_unit(h + at.row * m + c, n, a);
    }
}

// WITHIN: m is a multiple of 16
template <typename T, bool WITHIN>
__global__ void __launch_bounds__(kThreads)
swiglu_backward_kernel(Tiling t, int m, int64_t groups, const int8_t* q, const uint8_t* scale,
                       const T* dh, T* dau, T* h) {
    for (int i = threadIdx.x; i < t.rows * t.per; i += kThreads) {
        const Unit at = unit_of(t, i);
        if (at.row >= t.R) continue;
        const int c = at.u * kUnit, n = m - c;
        const int8_t* qr = q + at.row * (2 * (int64_t)m);
        const uint8_t* er = scale + at.row * groups;
        float a[kUnit], u[kUnit], d[kUnit];
        load_values<true>(qr, er, c, n, a);
        load_values<WITHIN>(qr, er, m + c, n, u);
        load_unit(dh + at.row * m + c, n, d);
#pragma unroll
        for (int j = 0; j < kUnit; ++j) {
            const float sig = sigmoid(a[j]);
            const float s = a[j] * sig;
            const float du = d[j] * s;
            const float da = d[j] * u[j] * (sig * (1.0f + a[j] * (1.0f - sig)));
            d[j] = s * u[j];
            a[j] = da;
            u[j] = du;
        }
        T* p = dau + at.row * (2 * (int64_t)m) + c;
        store_unit(p, n, a);
        store_unit(p + m, n, u);
        if (h) store_unit(h + at.row * m + c, n, d);
    }
}

// ------------------------------------------------------------------ host ----
bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

pr2_status check_pack(int64_t R, int64_t C, const char* name, int act_dtype) {
    if (act_dtype != PR2_F32 && act_dtype != PR2_BF16)
        return fail(PR2_ERR_DTYPE, "act_dtype %d is not PR2_F32 or PR2_BF16", act_dtype);
    if (R < 0) return fail(PR2_ERR_SHAPE, "R = %lld < 0", (long long)R);
    if (C < 1) return fail(PR2_ERR_SHAPE, "%s = %lld < 1", name, (long long)C);
    if (C > (1 << 28)) return fail(PR2_ERR_UNSUPPORTED, "%s = %lld > 2^28", name, (long long)C);
    if (R > 0x7fffffff) return fail(PR2_ERR_UNSUPPORTED, "R = %lld rows exceed 2^31 - 1", (long long)R);
    return PR2_OK;
}

pr2_status check_ptrs(std::initializer_list<const void*> need) {
    for (const void* p : need) {
        if (!p) return fail(PR2_ERR_NULL, "a required tensor is NULL");
        if (!aligned16(p)) return fail(PR2_ERR_ALIGN, "a tensor is not 16-byte aligned");
    }
    return PR2_OK;
}

template <typename T>
hipError_t launch_pack(int64_t R, int32_t C, const void* x, int8_t* q, uint8_t* scale, hipStream_t st) {
    const int64_t groups = ((int64_t)C + 31) / 32;
    const Tiling t = tiling(R, 2 * groups);
    LaunchScope scope("act_pack", st);
    hipLaunchKernelGGL(act_pack_kernel<T>, grid_of(t), dim3(kThreads), 0, st, t, C, groups,
                       (const T*)x, q, scale);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_unpack(int64_t R, int32_t C, const int8_t* q, const uint8_t* scale, void* x,
                         hipStream_t st) {
    const Tiling t = tiling(R, ((int64_t)C + kUnit - 1) / kUnit);
    LaunchScope scope("act_unpack", st);
    hipLaunchKernelGGL(act_unpack_kernel<T>, grid_of(t), dim3(kThreads), 0, st, t, C,
                       ((int64_t)C + 31) / 32, q, scale, (T*)x);
    return hipGetLastError();
}

// m not a multiple of 32: u's groups straddle a's end and the units' own, so the
// packing is a launch of its own that reads au again
template <typename T>
hipError_t launch_swiglu(int64_t R, int32_t m, const void* au, void* h, int8_t* q, uint8_t* scale,
                         hipStream_t st) {
    const bool fused = m % 32 == 0;
    const int64_t groups = (2 * (int64_t)m + 31) / 32;
    const Tiling t = tiling(R, ((int64_t)m + kUnit - 1) / kUnit);
    {
        LaunchScope scope("swiglu_pack", st);
        if (fused)
            hipLaunchKernelGGL((swiglu_kernel<T, true>), grid_of(t), dim3(kThreads), 0, st, t, m,
                               groups, (const T*)au, (T*)h, q, scale);
        else
            hipLaunchKernelGGL((swiglu_kernel<T, false>), grid_of(t), dim3(kThreads), 0, st, t, m,
                               groups, (const T*)au, (T*)h, q, scale);
    }
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || fused ? e : launch_pack<T>(R, 2 * m, au, q, scale, st);
}

template <typename T>
hipError_t launch_swiglu_backward(int64_t R, int32_t m, const int8_t* q, const uint8_t* scale,
                                  const void* dh, void* dau, void* h, hipStream_t st) {
    const int64_t groups = (2 * (int64_t)m + 31) / 32;
    const Tiling t = tiling(R, ((int64_t)m + kUnit - 1) / kUnit);
    LaunchScope scope("swiglu_backward", st);
    if (m % kUnit == 0)
        hipLaunchKernelGGL((swiglu_backward_kernel<T, true>), grid_of(t), dim3(kThreads), 0, st, t,
                           m, groups, q, scale, (const T*)dh, (T*)dau, (T*)h);
    else
        hipLaunchKernelGGL((swiglu_backward_kernel<T, false>), grid_of(t), dim3(kThreads), 0, st, t,
                           m, groups, q, scale, (const T*)dh, (T*)dau, (T*)h);
    return hipGetLastError();
}

}  // namespace
}  // namespace pr2

using namespace pr2;

extern "C" {

pr2_status pr2_act_pack(int64_t R, int32_t C, int act_dtype, const void* x, int8_t* q,
                        uint8_t* scale, pr2_stream_t stream) {
    pr2_status s = check_pack(R, C, "C", act_dtype);
    if (s != PR2_OK) return s;
    if (R == 0) return ok();
    if ((s = check_ptrs({x, q, scale})) != PR2_OK) return s;
    if ((s = device_ready()) != PR2_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = act_dtype == PR2_BF16 ? launch_pack<bf16_t>(R, C, x, q, scale, st)
                                               : launch_pack<float>(R, C, x, q, scale, st);
    if (e != hipSuccess) return hip_fail(e, "act_pack launch");
    return ok();
}

pr2_status pr2_act_unpack(int64_t R, int32_t C, int act_dtype, const int8_t* q,
                          const uint8_t* scale, void* x, pr2_stream_t stream) {
    pr2_status s = check_pack(R, C, "C", act_dtype);
    if (s != PR2_OK) return s;
    if (R == 0) return ok();
    if ((s = check_ptrs({q, scale, x})) != PR2_OK) return s;
    if ((s = device_ready()) != PR2_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = act_dtype == PR2_BF16 ? launch_unpack<bf16_t>(R, C, q, scale, x, st)
                                               : launch_unpack<float>(R, C, q, scale, x, st);
    if (e != hipSuccess) return hip_fail(e, "act_unpack launch");
    return ok();
}

pr2_status pr2_swiglu_pack(int64_t R, int32_t m, int act_dtype, const void* au, void* h,
                           int8_t* q, uint8_t* scale, pr2_stream_t stream) {
    pr2_status s = check_pack(R, m, "m", act_dtype);
    if (s != PR2_OK) return s;
    if (R == 0) return ok();
    if ((s = check_ptrs({au, h, q, scale})) != PR2_OK) return s;
    if ((s = device_ready()) != PR2_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = act_dtype == PR2_BF16 ? launch_swiglu<bf16_t>(R, m, au, h, q, scale, st)
                                               : launch_swiglu<float>(R, m, au, h, q, scale, st);
    if (e != hipSuccess) return hip_fail(e, "swiglu_pack launch");
    return ok();
}

pr2_status pr2_swiglu_backward_packed(int64_t R, int32_t m, int act_dtype, const int8_t* q,
                                      const uint8_t* scale, const void* dh, void* d_au,
                                      void* h_out, pr2_stream_t stream) {
    pr2_status s = check_pack(R, m, "m", act_dtype);
    if (s != PR2_OK) return s;
    if (R == 0) return ok();
    if ((s = check_ptrs({q, scale, dh, d_au})) != PR2_OK) return s;
    if (!aligned16(h_out)) return fail(PR2_ERR_ALIGN, "h_out is not 16-byte aligned");
    if ((s = device_ready()) != PR2_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e =
        act_dtype == PR2_BF16 ? launch_swiglu_backward<bf16_t>(R, m, q, scale, dh, d_au, h_out, st)
                              : launch_swiglu_backward<float>(R, m, q, scale, dh, d_au, h_out, st);
    if (e != hipSuccess) return hip_fail(e, "swiglu_backward_packed launch");
    return ok();
}

}  // extern "C"
