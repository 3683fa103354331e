// Products of rows sorted by expert with their experts' weights W [N, n_out, n_in]:
//
//   out[r, :] = x[src(r), :] W[e]^T           src(r) the token of row r's route, or r itself
//   dx[r, :]  = dy[r, :] W[e]                  the gradient of the row
//   out[r, o] = s_src(r) w[e, o] sum_c q[src(r), c] Wq[e, o, c]     both in 8 bits
//
// A row without a source and the rows behind the last expert's are zeros.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "chunk.h"
#include "copies.h"
#include "rowtiles.h"

namespace pr2 {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef u32x4 u32x4_byte __attribute__((aligned(1)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;

struct MmArgs {
    const void* x;              // [Rx, K] rows read (dy, q)
    const void* W;              // [N, n_out, n_in]
    const int* offsets;         // [N + 1] or null (one weight, all rows)
    const int* route;           // [R] or null
    void* out;                  // [R, C]
    const float* row_scale;     // [Rx] (8 bits)
    const float* w_scale;       // [N, n_out] (8 bits)
    int R, Rx;
    int K, C;                   // length of the sums, columns of out
    int N, k;
};

// Outputs of at least this much are written past the caches, half the size of the last-level cache: the
// tiles that run meanwhile find more of their weights and rows there (16384 tokens, 8 of 64 or 128 experts, bf16
// 1 to 4 % of the product, 8 bits 3 to 9 %).
constexpr int64_t kStreamBytes = 128 << 20;

// the row of x behind row r of the product, -1 if it has none
__device__ __forceinline__ int source(const MmArgs& a, int r) {
    if (!a.route) return r;
    const int q = a.route[r];
    const int t = q / a.k;
    return q >= 0 && t < a.Rx ? t : -1;
}

// ------------------------------------------------------------------- fp32 rows --
// 64 x 64 outputs per workgroup, four wavefronts of 32 x 32 on v_mfma_f32_32x32x2_f32, 32 K at a time
// staged in LDS, the next 32 in flight meanwhile.  An operand whose rows run along K is read four K at a time; the
// weights of dy W, whose rows run along the columns, one K at a time.  A step's four K of either half
// wavefront are the same in both operands, so that any order of them gives the sum.  (2000 x 2000 x 2000
// in 149 us, 4096 x 4096 x 4096 in 1211, 114 TFLOP/s, their row gradients 151 and 1094; the library's products 140
// and 919.)
constexpr int kTile = 64;
constexpr int kStep = 32;
constexpr int kRowPitch = kStep + 4;        // 16-byte reads of 32 rows: every bank equally often
constexpr int kColPitch = kTile + 8;        // K rows 4 apart (the two half wavefronts) 32 banks apart

// 8 elements of a row from element c on, the ones past the row's n (or all, if !on) as 0
__device__ __forceinline__ void load8(const float* row, int c, int n, bool on, f32x4 (&w)[2]) {
    typedef f32x4 f32x4_any __attribute__((aligned(4)));
    if (on && c + 8 <= n) {
        w[0] = *(const f32x4_any*)(row + c);
        w[1] = *(const f32x4_any*)(row + c + 4);
        return;
    }
    w[0] = w[1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (!on) return;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < n) w[i / 4][i % 4] = row[c + i];
}

// BACK: out = x W (W [K, C] an expert), else out = x W^T (W [C, K])
template <bool BACK>
__global__ void __launch_bounds__(256) mm_tile_kernel(MmArgs a) {
    __shared__ __attribute__((aligned(16))) float A[kTile * kRowPitch];
    __shared__ __attribute__((aligned(16))) float B[BACK ? kStep * kColPitch : kTile * kRowPitch];
    __shared__ int s_src[kTile];
    RowTile t;
    if (!find_tile(a.offsets, a.N, a.R, kTile, (a.C + kTile - 1) / kTile, block_number(), &t)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int c0 = t.panel * kTile;
    if (tid < kTile) s_src[tid] = tid < t.rows && t.expert < a.N ? source(a, t.row0 + tid) : -1;
    __syncthreads();
    const int len = t.expert < a.N ? a.K : 0;
    const float* W = (const float*)a.W + (int64_t)(len ? t.expert : 0) * a.K * a.C;

    const int ar = tid / 4, ak = (tid % 4) * 8;             // what this thread stages of x
    const int br = BACK ? tid / 8 : ar, bk = BACK ? (tid % 8) * 8 : ak;
    const int src = s_src[ar];
    const float* x = (const float*)a.x + (int64_t)max(src, 0) * a.K;
    f32x4 wa[2], wb[2];
    auto fetch = [&](int k0) __attribute__((always_inline)) {
        load8(x, k0 + ak, a.K, src >= 0, wa);
        if (BACK) load8(W + (int64_t)min(k0 + br, a.K - 1) * a.C, c0 + bk, a.C, k0 + br < a.K, wb);
        else load8(W + (int64_t)min(c0 + br, a.C - 1) * a.K, k0 + bk, a.K, c0 + br < a.C, wb);
    };
    const int half = lane >> 5, l32 = lane & 31;
    const int ao = 32 * (wave >> 1) + l32, bo = 32 * (wave & 1) + l32;
    f32x16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.0f;
    if (len) fetch(0);
    for (int k0 = 0; k0 < len; k0 += kStep) {
        __syncthreads();
        float* const to_a = A + ar * kRowPitch + ak;
        float* const to_b = B + (BACK ? br * kColPitch : br * kRowPitch) + bk;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            *(f32x4*)(to_a + 4 * i) = wa[i];
            *(f32x4*)(to_b + 4 * i) = wb[i];
        }
        __syncthreads();
        if (k0 + kStep < len) fetch(k0 + kStep);
#pragma unroll
        for (int k = 0; k < kStep; k += 8) {
            const f32x4 fa = *(const f32x4*)(A + ao * kRowPitch + k + 4 * half);
            f32x4 fb;
            if (BACK) {
#pragma unroll
                for (int j = 0; j < 4; ++j) fb[j] = B[(k + 4 * half + j) * kColPitch + bo];
            } else {
                fb = *(const f32x4*)(B + bo * kRowPitch + k + 4 * half);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[j], fb[j], acc, 0, 0, 0);
        }
    }
    // lane l holds column l % 32 and rows 8 (v / 4) + 4 (l / 32) + v % 4
    const int c = c0 + bo;
    if (c >= a.C) return;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int r = 32 * (wave >> 1) + 8 * (v / 4) + 4 * half + v % 4;
        // (a row without a source is 0 even where the weights are not finite)
        if (r < t.rows) ((float*)a.out)[(int64_t)(t.row0 + r) * a.C + c] = s_src[r] >= 0 ? acc[v] : 0.0f;
    }
}

// ------------------------------------------------- bf16 and 8-bit rows of any length --
constexpr int kStepB = 128;
constexpr int kPitchB = kStepB + 16;

// 16 bytes from any address, by loads of whole words, put together where they are used: a load that is
// not 4-byte aligned takes several times as long (517 x 1001 outputs of 999 int8 in 32 x 32 tiles: 13.5 us,
// of 1000 6.5; this way 10.4 and 7.7 in a row of calls).  No word is read that holds none of the bytes.  ANY false: the address is 4-byte aligned.
template <bool ANY> struct Piece {
    u32x4 w;
    uint32_t next;
    __device__ __forceinline__ void load(const unsigned char* p) {
        typedef u32x4 u32x4_word __attribute__((aligned(4)));
        const uint32_t drop = ANY ? (uint32_t)(uintptr_t)p & 3 : 0;
        const uint32_t* words = (const uint32_t*)(p - drop);
        w = *(const u32x4_word*)words;
        if (ANY) next = words[drop ? 4 : 3];
    }
    // drop: how far behind a word's start p was
    __device__ __forceinline__ u32x4 bytes(uint32_t drop) const {
        if (!ANY) return w;
        return u32x4{__builtin_amdgcn_alignbyte(w[1], w[0], drop), __builtin_amdgcn_alignbyte(w[2], w[1], drop),
                     __builtin_amdgcn_alignbyte(w[3], w[2], drop), drop ? __builtin_amdgcn_alignbyte(next, w[3], drop) : w[3]};
    }
};

// --------------------------------------------------------- matrix instructions --
// bf16 rows of a multiple of 16 bytes on v_mfma_f32_16x16x32_bf16, 8-bit ones on
// v_mfma_i32_16x16x64_i8: a lane's fragment is 16 consecutive bytes of a row in both, so one kernel
// in bytes serves both.
template <typename E> struct Mma;
template <> struct Mma<bf16_t> {
    using Frag = bf16x8;
    using Acc = f32x4;
    static constexpr int kSteps = 1;
    __device__ __forceinline__ static Acc mul(Frag a, Frag b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    __device__ __forceinline__ static Acc step(Frag a, Frag b, int, Acc c) { return mul(a, b, c); }
};
template <> struct Mma<int8_t> {
    using Frag = i32x4;
    using Acc = i32x4;
    static constexpr int kSteps = 1;
    __device__ __forceinline__ static Acc mul(Frag a, Frag b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
    }
    __device__ __forceinline__ static Acc step(Frag a, Frag b, int, Acc c) { return mul(a, b, c); }
};

// fp32: four K values of a row, one a step of v_mfma_f32_16x16x4_f32
template <> struct Mma<float> {
    using Frag = f32x4;
    using Acc = f32x4;
    static constexpr int kSteps = 4;
    __device__ __forceinline__ static Acc step(const Frag& a, const Frag& b, int k, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x4f32(a[k], b[k], c, 0, 0, 0);
    }
};

// 16 bytes of a row from byte c on, those past the row's n as 0
__device__ __forceinline__ u32x4 load16_bytes(const unsigned char* row, int c, int n) {
    if (c + 16 <= n) return *(const u32x4_byte*)(row + c);
    u32x4 w = {0, 0, 0, 0};
    if (c >= n) return w;
    if (n >= 16) {
        // the row's last 16 bytes, moved down
        const u32x4 v = *(const u32x4_byte*)(row + n - 16);
        const int drop = c + 16 - n;            // 1 .. 15
        uint64_t lo = (uint64_t)v[0] | (uint64_t)v[1] << 32, hi = (uint64_t)v[2] | (uint64_t)v[3] << 32;
        if (drop >= 8) {
            lo = hi;
            hi = 0;
        }
        const int bits = 8 * (drop & 7);
        if (bits) {
            lo = lo >> bits | hi << (64 - bits);
            hi >>= bits;
        }
        return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (c + i < n) w[i / 4] |= (uint32_t)(uint8_t)row[c + i] << (8 * (i % 4));
    return w;
}

// the same two types on blocks of 32 x 32
template <typename E> struct Wide;
template <> struct Wide<bf16_t> {
    using Acc = f32x16;
    __device__ __forceinline__ static Acc mul(const u32x4& a, const u32x4& b, Acc c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Wide<int8_t> {
    using Acc = i32x16;
    __device__ __forceinline__ static Acc mul(const u32x4& a, const u32x4& b, Acc c) {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    }
};

// Rows off 16 bytes: 64 x 64 outputs, 128 bytes of K at a time through registers (unaligned 16-byte
// loads) into LDS, two steps in flight.  BACK: out = x W, bf16, the weights' 64 K rows of 64 columns read as
// fragments by the transposing LDS read.  (bf16, 128 experts of 1024 rows, 1535 x 2047 2.42 ms, int8 1.49, 2000 x 2001
// x 2001 55 us; in 32 x 32 tiles 7.77 ms and 162 us.  The row gradients of one row of
// 1001 20 us, of 128 x 1024 rows 2.57 ms; in tiles of 16 to 32 rows straight from memory 24 us and 9.3 ms.)
template <typename E, typename O, bool BACK>
__global__ void __launch_bounds__(256) mm_any_kernel(MmArgs a) {
    __shared__ __attribute__((aligned(16))) unsigned char A[kTile * kPitchB], B[kTile * kPitchB];
    __shared__ int s_src[kTile];
    RowTile t;
    if (!find_tile(a.offsets, a.N, a.R, kTile, (a.C + kTile - 1) / kTile, block_number(), &t)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int c0 = t.panel * kTile;
    if (tid < kTile) s_src[tid] = tid < t.rows && t.expert < a.N ? source(a, t.row0 + tid) : -1;
    __syncthreads();
    const bool real = t.expert < a.N;
    const int kb = a.K * (int)sizeof(E), len = real ? kb : 0;
    const int expert = real ? t.expert : 0;
    const unsigned char* W = (const unsigned char*)a.W + (int64_t)expert * a.C * kb;
    struct Set {
        u32x4 a[2], b[2];
    };
    const int wb = BACK ? a.C * (int)sizeof(E) : kb;        // bytes of a row of the weights
    const unsigned char *xr[2], *wr[2];             // rows tid / 8 and + 32 (BACK: of the step's weights)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = tid / 8 + 32 * i;
        xr[i] = (const unsigned char*)a.x + (int64_t)max(s_src[r], 0) * kb;
        wr[i] = BACK ? W + (int64_t)r * wb : W + (int64_t)min(c0 + r, a.C - 1) * wb;
    }
    auto fetch = [&](Set& s, int k0) __attribute__((always_inline)) {
        const int c = k0 + (tid % 8) * 16;
        if (BACK) {
            const int first = k0 / (int)sizeof(E), col = c0 * (int)sizeof(E) + (tid % 8) * 16;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                s.a[i] = load16_bytes(xr[i], c, kb);
                s.b[i] = load16_bytes(wr[i] + (int64_t)first * wb, first + tid / 8 + 32 * i < a.K ? col : wb, wb);
            }
        } else if (k0 + kStepB <= kb) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                s.a[i] = *(const u32x4_byte*)(xr[i] + c);
                s.b[i] = *(const u32x4_byte*)(wr[i] + c);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                s.a[i] = load16_bytes(xr[i], c, kb);
                s.b[i] = load16_bytes(wr[i], c, kb);
            }
        }
    };
    const int half = lane >> 5, l32 = lane & 31;
    const int ao = 32 * (wave >> 1) + l32, bo = 32 * (wave & 1) + l32;
    typename Wide<E>::Acc acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0;
    // (BACK) 8 K values of column bo from K row k + 8 half on, four of them a read
    const int s16 = lane & 15, nl = 16 * ((lane >> 4) & 1) + 4 * (s16 & 3), kl = 8 * half + (s16 >> 2);
    auto columns = [&](int k) __attribute__((always_inline)) {
        const unsigned char* p = B + (k + kl) * kPitchB + (32 * (wave & 1) + nl) * 2;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)p);
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p + 4 * kPitchB));
        return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // two steps in flight behind the one that is multiplied
    auto step = [&](Set& s, int k0) __attribute__((always_inline)) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = (tid / 8 + 32 * i) * kPitchB + (tid % 8) * 16;
            *(u32x4*)(A + at) = s.a[i];
            *(u32x4*)(B + at) = s.b[i];
        }
        __syncthreads();
        if (k0 + 2 * kStepB < len) fetch(s, k0 + 2 * kStepB);
#pragma unroll
        for (int k = 0; k < kStepB; k += 32) {
            const u32x4 fa = *(const u32x4*)(A + ao * kPitchB + k + 16 * half);
            const u32x4 fb = BACK ? columns(k / 2) : *(const u32x4*)(B + bo * kPitchB + k + 16 * half);
            acc = Wide<E>::mul(fa, fb, acc);
        }
    };
    Set s0, s1;
    if (len) fetch(s0, 0);
    if (kStepB < len) fetch(s1, kStepB);
    for (int k0 = 0; k0 < len; k0 += 2 * kStepB) {
        step(s0, k0);
        if (k0 + kStepB < len) step(s1, k0 + kStepB);
    }
    const int c = c0 + bo;
    if (c >= a.C) return;
    const float sw = sizeof(E) == 1 ? a.w_scale[(int64_t)expert * a.C + c] : 1.0f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int r = 32 * (wave >> 1) + 8 * (v / 4) + 4 * half + v % 4;
        if (r >= t.rows) continue;
        const int src = s_src[r];
        float y = 0.0f;         // (without a source, also where the weights are not finite)
        if (src >= 0) y = sizeof(E) == 1 ? (float)acc[v] * a.row_scale[src] * sw : (float)acc[v];
        ((O*)a.out)[(int64_t)(t.row0 + r) * a.C + c] = Act<O>::from_f32(y);
    }
}

constexpr int kRowB = 128;                  // bytes of a row per K slice
constexpr int MT = 16;
__device__ __attribute__((aligned(16))) const unsigned char kZeros[16] = {};

// 16-byte chunk c of LDS row r lies at c ^ swz(r): 8 or 16 consecutive rows read at the same chunk
// hit disjoint banks
__device__ __forceinline__ int swz(int r) { return (r & 7) ^ ((r >> 3) & 1); }

// wait until at most n of this wavefront's copies are outstanding
template <int n>
__device__ __forceinline__ void wait_vmcnt() {
    static_assert(n >= 0 && n < 16, "vmcnt field");
    __builtin_amdgcn_s_waitcnt(0x0f70 | n);
}
// a barrier that leaves the copies in flight
__device__ __forceinline__ void plain_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
}

// Four consecutive columns of a row's sums as outputs; `on` false: a row without a source.
template <typename E>
__device__ __forceinline__ f32x4 finish(const typename Mma<E>::Acc& acc, bool on, float sr, const f32x4& sw) {
    f32x4 y;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        if (sizeof(E) == 1) y[v] = (float)acc[v] * sr * sw[v];
        else y[v] = (float)acc[v];
        y[v] = on ? y[v] : 0.0f;
    }
    return y;
}
// the channels' scales of columns c .. c + 3 of C (zeros past them)
__device__ __forceinline__ f32x4 four_scales(const float* w, int c, int C) {
    typedef f32x4 f32x4_any __attribute__((aligned(4)));
    if (c + 4 <= C) return *(const f32x4_any*)(w + c);
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (c + v < C) s[v] = w[c + v];
    return s;
}
// four columns from c on of a row of C, wherever the row starts
template <typename O>
__device__ __forceinline__ void store_four(O* row, int c, int C, const f32x4& y) {
    typedef f32x4 f32x4_any __attribute__((aligned(4)));
    typedef uint64_t u64_any __attribute__((aligned(2)));
    if (c + 4 <= C) {
        if (sizeof(O) == 4) {
            *(f32x4_any*)(row + c) = y;
        } else {
            const uint32_t lo = (uint32_t)f32_to_bf16(y[0]) | (uint32_t)f32_to_bf16(y[1]) << 16;
            const uint32_t hi = (uint32_t)f32_to_bf16(y[2]) | (uint32_t)f32_to_bf16(y[3]) << 16;
            *(u64_any*)(row + c) = (uint64_t)hi << 32 | lo;
        }
        return;
    }
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (c + v < C) row[c + v] = Act<O>::from_f32(y[v]);
}
// zeros in the columns of a panel of the rows that belong to no expert
template <typename O>
__device__ __forceinline__ void zero_tile(const MmArgs& a, const RowTile& t, int width, int threads) {
    const int c0 = t.panel * width, n = min(width, a.C - c0);
    for (int i = threadIdx.x; i < t.rows * width; i += threads) {
        const int r = i / width, c = i % width;
        if (c < n) ((O*)a.out)[(int64_t)(t.row0 + r) * a.C + c0 + c] = Act<O>::from_f32(0.0f);
    }
}

// 256 rows x 256 columns per workgroup, eight wavefronts of 64 x 128 (two per SIMD).  K advances in
// slices of 128 bytes a row, copied into LDS directly; the slice's only barrier sits between its two
// sub-steps, so that the fragments of the next sub-step are always read among the MFMAs of the one
// before.  Three stages of rows and two of weights: rows are copied among a slice's first sub-step and
// weights among its second, one copy for 8 MFMAs and no branch at any (with two stages of both all
// copies fall into the second sub-step: zeros, where power does not limit, 131072 x 1536 x 2048 17 % longer, random
// numbers 3 %).  Chunks past a row's end are copied from zeros, in both operands.  The
// MFMAs take (weights, rows), so that a lane holds four consecutive columns of one row.
// (bf16 131072 x 1536 x 2048 in 128 experts 709 us, 1163 TFLOP/s, the library's product with one weight 623;
// int8 131072 x 2048 x 2048 in 64 experts 537 us, 2.05 POP/s, with one weight 519, the library's 603.)
constexpr int BM = 256, BP = 256;
constexpr int WM = 64, WN = 128;
constexpr int NJ = WN / MT;
constexpr int kThreads = 512;
constexpr int kCopy = 4;                    // copies of 8 rows of either operand per wavefront and slice
constexpr int kOperandB = 256 * kRowB;      // a stage of one operand

template <typename E, typename O, bool STREAM>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
mm_wide_kernel(MmArgs a) {
    using M = Mma<E>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[5 * kOperandB];     // three of rows, two of weights
    RowTile t;
    if (!find_tile(a.offsets, a.N, a.R, BM, (a.C + BP - 1) / BP, block_number(), &t)) return;
    if (t.expert >= a.N) {
        zero_tile<O>(a, t, BP, kThreads);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave >> 1, wc = wave & 1;
    const int c0 = t.panel * BP;
    // wavefronts past the tile's rows or the matrix only help copy
    const bool active = wr * MT < t.rows && c0 + wc * WN < a.C;
    const int kb = a.K * (int)sizeof(E);

    // wavefront w copies rows 32 w + 8 i + lane / 8 of both operands (past their ends the last one)
    const int wrow0 = wave * 8 * kCopy;
    const int chunk0 = (lane & 7) ^ swz(lane >> 3);         // of copies 0, 2, ..; the others ^ 1
    const unsigned char* const xb = (const unsigned char*)a.x + (a.route ? 0 : (int64_t)t.row0 * kb);
    const unsigned char* const wb = (const unsigned char*)a.W + ((int64_t)t.expert * a.C + c0) * kb;
    uint32_t xo[kCopy], wo[kCopy];
    int src[kCopy];
#pragma unroll
    for (int i = 0; i < kCopy; ++i) {
        const int r = min(wrow0 + 8 * i + lane / 8, t.rows - 1);
        src[i] = a.route ? a.route[t.row0 + r] : r;
    }
#pragma unroll
    for (int i = 0; i < kCopy; ++i) {
        const int row = a.route ? min(max(src[i], 0) / a.k, a.Rx - 1) : src[i];
        const int ch = (chunk0 ^ (i & 1)) << 4;
        xo[i] = (uint32_t)row * (uint32_t)kb + ch;
        wo[i] = (uint32_t)min(wrow0 + 8 * i + lane / 8, a.C - 1 - c0) * (uint32_t)kb + ch;
    }
    const int whole = kb / kRowB;                           // slices inside every row
    const int nk = max(2, (kb + kRowB - 1) / kRowB);
    const uint32_t lds0 = lds_address(lds) + wave * (kCopy * 1024);
    using C0 = std::integral_constant<int, 0>;
    using C1 = std::integral_constant<int, 1>;
    // copy i of slice kt; PART: the slice may pass the rows' end
    auto issue = [&](auto PART, const unsigned char* from, const uint32_t* off, int kt, uint32_t to, int i)
                     __attribute__((always_inline)) {
        from += kt * kRowB;
        if (!decltype(PART)::value) dma16_to(from, off[i], to + i * 1024);
        else dma16_to((chunk0 ^ (i & 1)) * 16 < kb - kt * kRowB ? from + off[i] : kZeros, to + i * 1024);
    };
    const bool has_x = wrow0 < t.rows;      // (asked where the tile has up to 128 rows)
    auto issue_x = [&](auto PART, int kt, int stage, int i) __attribute__((always_inline)) {
        issue(PART, xb, xo, kt, lds0 + stage * kOperandB, i);
    };
    auto issue_w = [&](auto PART, int kt, int i) __attribute__((always_inline)) {
        issue(PART, wb, wo, kt, lds0 + (3 + (kt & 1)) * kOperandB, i);
    };

    // The tile's rows in BLOCKS times 64: block i of a wavefront is rows 64 i + 16 wr on, so that a tile of fewer rows
    // takes fewer MFMAs of all (16384 tokens, 8 of 128 experts unevenly, 1536 x 2048: 797 -> 783 us; a tile of up to 64
    // rows still costs half of a full one, for the latency of its slices' copies).
    auto run = [&](auto BLOCKS) __attribute__((always_inline)) {
        constexpr int MB = decltype(BLOCKS)::value;
        constexpr bool kFewRows = MB <= 2;
        typename M::Acc acc[MB][NJ];
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][j][v] = 0;
        // fragments: lane l reads row l % 16 of a block, chunk 4 ks + (0, 2, 1, 3)[l / 16] (both operands
        // alike, and so that the two halves of a read cycle hit disjoint banks)
        const int lrow = lane & 15, grp = lane >> 4;
        const int cperm = ((grp & 1) << 1) | (grp >> 1);
        int kpos[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) kpos[ks] = lrow * kRowB + (((4 * ks + cperm) ^ swz(lrow)) << 4);
        const int a0 = wr * MT * kRowB, b0 = (3 * BM + wc * WN) * kRowB;
        typename M::Frag fa[2][MB], fb[2][NJ];
        auto frag = [&](int at) __attribute__((always_inline)) {
            return __builtin_bit_cast(typename M::Frag, *(const u32x4*)(lds + at));
        };
        // the slice before that of the last n copies has arrived, and this wavefront's LDS reads have ended
        auto sync = [&](auto N) __attribute__((always_inline)) {
            if (!kFewRows || has_x) wait_vmcnt<decltype(N)::value>();
            else wait_vmcnt<0>();
            __builtin_amdgcn_s_waitcnt(0xc07f);
            plain_barrier();
        };
        // MFMAs of a sub-step on fragment set S, among them the reads of the next one's (sub-step ks of the rows'
        // stage xs and the weights' ws) and copy(0 .. 3)
        auto phase = [&](auto S_, auto READ, int xs, int ws, int ks, auto copy) __attribute__((always_inline)) {
            constexpr int S = decltype(S_)::value;
            const int xa = xs * kOperandB + kpos[ks] + a0, wa = ws * kOperandB + kpos[ks] + b0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                copy(q);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 2 * q; j < 2 * q + 2; ++j)
#pragma unroll
                    for (int i = 0; i < MB; ++i) acc[i][j] = M::mul(fb[S][j], fa[S][i], acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
                if (decltype(READ)::value && q < 3) {
                    if (q < 2) {
#pragma unroll
                        for (int h = 2 * q; h < 2 * q + 2; ++h) {
                            if (h < MB) fa[S ^ 1][h < MB ? h : 0] = frag(xa + h * 4 * MT * kRowB);
                            fb[S ^ 1][h] = frag(wa + h * MT * kRowB);
                        }
                    } else {
#pragma unroll
                        for (int h = 4; h < NJ; ++h) fb[S ^ 1][h] = frag(wa + h * MT * kRowB);
                    }
                }
            }
        };
        auto no_copy = [](int) {};
        using Behind = std::integral_constant<int, kCopy>;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < kCopy; ++i) {
                if (!kFewRows || has_x) issue_x(C1{}, kt, kt, i);
                issue_w(C1{}, kt, i);
            }
        if (!kFewRows || has_x) wait_vmcnt<2 * kCopy>();
        else wait_vmcnt<kCopy>();
        plain_barrier();
        int kt = 0, xs = 0;         // the slice and its rows' stage
        auto next = [](int s) __attribute__((always_inline)) { return s == 2 ? 0 : s + 1; };
        if (active) {
#pragma unroll
            for (int i = 0; i < MB; ++i) fa[0][i] = frag(kpos[0] + a0 + i * 4 * MT * kRowB);
#pragma unroll
            for (int j = 0; j < NJ; ++j) fb[0][j] = frag(kpos[0] + b0 + j * MT * kRowB);
            // slice kt with the copies of slice kt + 2
            auto slice = [&](auto PART) __attribute__((always_inline)) {
                const int x1 = next(xs), x2 = next(x1);
                phase(C0{}, C1{}, xs, kt & 1, 1, [&](int q) __attribute__((always_inline)) {
                    if (!kFewRows || has_x) issue_x(PART, kt + 2, x2, q);
                });
                sync(Behind{});
                phase(C1{}, C1{}, x1, (kt + 1) & 1, 0, [&](int q) __attribute__((always_inline)) { issue_w(PART, kt + 2, q); });
                xs = x1;
            };
            for (; kt + 2 < whole; ++kt) slice(C0{});
            for (; kt + 2 < nk; ++kt) slice(C1{});
            phase(C0{}, C1{}, xs, kt & 1, 1, no_copy);
            sync(C0{});
            xs = next(xs);
            phase(C1{}, C1{}, xs, (kt + 1) & 1, 0, no_copy);
            phase(C0{}, C1{}, xs, (kt + 1) & 1, 1, no_copy);
            phase(C1{}, C0{}, 0, 0, 0, no_copy);
        } else {
            for (; kt + 2 < nk; ++kt) {
#pragma unroll
                for (int i = 0; i < kCopy; ++i)
                    if (!kFewRows || has_x) issue_x(C1{}, kt + 2, next(next(xs)), i);
                sync(Behind{});
#pragma unroll
                for (int i = 0; i < kCopy; ++i) issue_w(C1{}, kt + 2, i);
                xs = next(xs);
            }
            sync(C0{});
        }

        // a lane's rows: lane % 16 of the wavefront's blocks
        auto row_of = [&](int i) __attribute__((always_inline)) { return 4 * MT * i + wr * MT + lrow; };
        const int col0 = c0 + wc * WN + 4 * grp;
        bool on[MB];
        float sr[MB];
        if (active) {
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const int src = source(a, t.row0 + min(row_of(i), t.rows - 1));
                on[i] = src >= 0;
                sr[i] = sizeof(E) == 1 ? a.row_scale[max(src, 0)] : 0.0f;
            }
        }
        const float* sw = sizeof(E) == 1 ? a.w_scale + (int64_t)t.expert * a.C : nullptr;
        const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
        if (sizeof(O) == 4) {
            // 64 bytes of a row per store and 16 lanes, straight from the registers
            if (!active) return;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const f32x4 s4 = sizeof(E) == 1 ? four_scales(sw, col0 + j * MT, a.C) : none;
#pragma unroll
                for (int i = 0; i < MB; ++i) {
                    const int r = row_of(i);
                    if (r < t.rows)
                        store_four((O*)a.out + (int64_t)(t.row0 + r) * a.C, col0 + j * MT, a.C,
                                   finish<E>(acc[i][j], on[i], sr[i], s4));
                }
            }
            return;
        }
        // bf16: through this wavefront's share of the freed stages (16-byte chunks XOR-swizzled by row, the
        // halves of a chunk swapped in rows with bit 3 set: every write cycle's rows in other banks), so
        // that a store covers whole 256-byte row segments
        __syncthreads();
        if (!active) return;
        constexpr int RB = WN * 2, NCH = RB / 16;
        unsigned char* stage_w = lds + wave * (WM * RB);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const f32x4 s4 = sizeof(E) == 1 ? four_scales(sw, col0 + j * MT, a.C) : none;
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const int row = i * MT + lrow, col = j * MT + 4 * grp;
                const f32x4 y = finish<E>(acc[i][j], on[i], sr[i], s4);
                const uint32_t lo = (uint32_t)f32_to_bf16(y[0]) | (uint32_t)f32_to_bf16(y[1]) << 16;
                const uint32_t hi = (uint32_t)f32_to_bf16(y[2]) | (uint32_t)f32_to_bf16(y[3]) << 16;
                *(uint2*)(stage_w + row * RB + (((col >> 3) ^ (row & (NCH - 1))) << 4) + (((col & 4) << 1) ^ (row & 8))) =
                    make_uint2(lo, hi);
            }
        }
        // (one wavefront's own region: its LDS operations complete in order)
        __builtin_amdgcn_s_waitcnt(0xc07f);
        __builtin_amdgcn_wave_barrier();
        const int ch = lane % NCH;
        const int col = c0 + wc * WN + ch * 8, left = a.C - col;
#pragma unroll
        for (int p = 0; p < MB * MT / (64 / NCH); ++p) {
            const int row = p * (64 / NCH) + lane / NCH;
            const int r = 4 * MT * (row / MT) + wr * MT + row % MT;
            u32x4 v = *(const u32x4*)(stage_w + row * RB + ((ch ^ (row & (NCH - 1))) << 4));
            if (row & 8) v = u32x4{v[2], v[3], v[0], v[1]};
            if (r >= t.rows) continue;
            bf16_t* to = (bf16_t*)a.out + (int64_t)(t.row0 + r) * a.C + col;
            if (left >= 8) {
                store16<STREAM>(to, v);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < left) to[e] = (bf16_t)(v[e / 2] >> (16 * (e & 1)));
            }
        }
    };
    const int blocks = (t.rows + 4 * MT - 1) / (4 * MT);
    if (blocks == 4) run(std::integral_constant<int, 4>{});
    else if (blocks == 3) run(std::integral_constant<int, 3>{});
    else if (blocks == 2) run(std::integral_constant<int, 2>{});
    else run(std::integral_constant<int, 1>{});
}

// Few rows per expert: the weights' bytes in flight are what matters.  64 rows x 128 columns per
// workgroup of four wavefronts, slices of 128 bytes a row through a ring of three stages, two
// workgroups on a CU.
constexpr int kFewM = 64, kFewP = 128;
constexpr int kFewStageB = (kFewM + kFewP) * kRowB;
constexpr int kFewStages = 3;

template <typename E, typename O>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
mm_few_kernel(MmArgs a) {
    using M = Mma<E>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kFewStages * kFewStageB];
    RowTile t;
    if (!find_tile<true>(a.offsets, a.N, a.R, kFewM, (a.C + kFewP - 1) / kFewP, block_number(), &t)) return;
    if (t.expert >= a.N) {
        zero_tile<O>(a, t, kFewP, 256);
        return;
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c0 = t.panel * kFewP;
    const int kb = a.K * (int)sizeof(E);
    // copies: weight rows 32 wave .. + 31 (four of 8), rows 16 wave .. + 15 (two, fewer past the end)
    const int chunk0 = (lane & 7) ^ swz(lane >> 3);
    const unsigned char* wb = (const unsigned char*)a.W + ((int64_t)t.expert * a.C + c0) * kb;
    const unsigned char* xb = (const unsigned char*)a.x + (a.route ? 0 : (int64_t)t.row0 * kb);
    uint32_t woff[4], xoff[2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        woff[i] = (uint32_t)min(32 * wave + 8 * i + lane / 8, a.C - 1 - c0) * (uint32_t)kb + ((chunk0 ^ (i & 1)) << 4);
    const int nx = max(0, min(2, (t.rows - 16 * wave + 7) / 8));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = min(16 * wave + 8 * i + lane / 8, t.rows - 1);
        const int row = a.route ? min(max(a.route[t.row0 + r], 0) / a.k, a.Rx - 1) : r;
        xoff[i] = (uint32_t)row * (uint32_t)kb + ((chunk0 ^ i) << 4);
    }
    const int whole = kb / kRowB;
    const int nk = max(2, (kb + kRowB - 1) / kRowB);
    const uint32_t lds0 = lds_address(lds), lds_w = lds0 + (kFewM + 32 * wave) * kRowB, lds_x = lds0 + 16 * wave * kRowB;
    const int turn = (5 * t.panel + 3 * t.expert) % nk;
    auto issue = [&](int step) __attribute__((always_inline)) {
        const int kt = step + turn < nk ? step + turn : step + turn - nk;
        const uint32_t st = (step % kFewStages) * kFewStageB;
        const unsigned char* const w = wb + kt * kRowB;
        const unsigned char* const x = xb + kt * kRowB;
        if (kt < whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) dma16_to(w, woff[i], lds_w + st + i * 1024);
            if (nx > 0) dma16_to(x, xoff[0], lds_x + st);
            if (nx > 1) dma16_to(x, xoff[1], lds_x + st + 1024);
        } else {
            const int left = kb - kt * kRowB;
            auto part = [&](const unsigned char* p, int i) __attribute__((always_inline)) {
                return (chunk0 ^ (i & 1)) * 16 < left ? p : kZeros;
            };
#pragma unroll
            for (int i = 0; i < 4; ++i) dma16_to(part(w + woff[i], i), lds_w + st + i * 1024);
            if (nx > 0) dma16_to(part(x + xoff[0], 0), lds_x + st);
            if (nx > 1) dma16_to(part(x + xoff[1], 1), lds_x + st + 1024);
        }
    };
    // a slice has landed, the one after it may still be in flight
    auto wait_one = [&]() __attribute__((always_inline)) {
        if (nx == 2) wait_vmcnt<6>();
        else if (nx == 1) wait_vmcnt<5>();
        else wait_vmcnt<4>();
    };
    const int lrow = lane & 15, grp = lane >> 4;
    const int cperm = ((grp & 1) << 1) | (grp >> 1);
    int kpos[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) kpos[ks] = lrow * kRowB + (((4 * ks + cperm) ^ swz(lrow)) << 4);
    const int b0 = (kFewM + 32 * wave) * kRowB, b1 = b0 + 16 * kRowB;
    typename M::Acc acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[i][j][v] = 0;
    const int mi = (t.rows + 15) / 16;
    issue(0);
    issue(1);
    for (int kt = 0; kt < nk; ++kt) {
        if (kt + 1 < nk) wait_one();
        else wait_vmcnt<0>();
        __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0)
        plain_barrier();
        if (kt + 2 < nk) issue(kt + 2);
        const unsigned char* st = lds + (kt % kFewStages) * kFewStageB;
        auto frag = [&](int at) __attribute__((always_inline)) {
            return __builtin_bit_cast(typename M::Frag, *(const u32x4*)(st + at));
        };
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const typename M::Frag w0 = frag(b0 + kpos[ks]), w1 = frag(b1 + kpos[ks]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= mi) continue;
                const typename M::Frag x = frag(16 * i * kRowB + kpos[ks]);
                acc[i][0] = M::mul(w0, x, acc[i][0]);
                acc[i][1] = M::mul(w1, x, acc[i][1]);
            }
        }
    }
    // lane l holds columns 4 (l / 16) .. + 3 of row l % 16
    const float* sw = sizeof(E) == 1 ? a.w_scale + (int64_t)t.expert * a.C : nullptr;
    f32x4 s4[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
    const int col = c0 + 32 * wave + 4 * grp;
    if (sizeof(E) == 1) {
        s4[0] = four_scales(sw, col, a.C);
        s4[1] = four_scales(sw, col + 16, a.C);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 16 * i + lrow;
        if (r >= t.rows) continue;
        const int src = source(a, t.row0 + r);
        const float sr = sizeof(E) == 1 ? a.row_scale[max(src, 0)] : 0.0f;
        O* row = (O*)a.out + (int64_t)(t.row0 + r) * a.C;
#pragma unroll
        for (int j = 0; j < 2; ++j) store_four(row, col + 16 * j, a.C, finish<E>(acc[i][j], src >= 0, sr, s4[j]));
    }
}

constexpr int kMidM = 128, kMidP = 128, kMidStages = 2;
constexpr int kMidStageB = (kMidM + kMidP) * kRowB;

template <typename E, typename O>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
mm_mid_kernel(MmArgs a) {
    using M = Mma<E>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kMidStages * kMidStageB];
    RowTile t;
    if (!find_tile<true>(a.offsets, a.N, a.R, kMidM, (a.C + kMidP - 1) / kMidP, block_number(), &t)) return;
    if (t.expert >= a.N) {
        zero_tile<O>(a, t, kMidP, 256);
        return;
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c0 = t.panel * kMidP;
    const int kb = a.K * (int)sizeof(E);
    // copies: weight rows 32 wave .. + 31 (four of 8), rows 32 wave .. + 31 (four, fewer past the end)
    const int chunk0 = (lane & 7) ^ swz(lane >> 3);
    const unsigned char* wb = (const unsigned char*)a.W + ((int64_t)t.expert * a.C + c0) * kb;
    const unsigned char* xb = (const unsigned char*)a.x + (a.route ? 0 : (int64_t)t.row0 * kb);
    uint32_t woff[4], xoff[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        woff[i] = (uint32_t)min(32 * wave + 8 * i + lane / 8, a.C - 1 - c0) * (uint32_t)kb + ((chunk0 ^ (i & 1)) << 4);
    const int nx = max(0, min(4, (t.rows - 32 * wave + 7) / 8));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = min(32 * wave + 8 * i + lane / 8, t.rows - 1);
        const int row = a.route ? min(max(a.route[t.row0 + r], 0) / a.k, a.Rx - 1) : r;
        xoff[i] = (uint32_t)row * (uint32_t)kb + ((chunk0 ^ (i & 1)) << 4);
    }
    const int whole = kb / kRowB;
    const int nk = max(2, (kb + kRowB - 1) / kRowB);
    const uint32_t lds0 = lds_address(lds) + 32 * wave * kRowB;
    const int turn = (5 * t.panel + 3 * t.expert) % nk;
    auto issue = [&](int step) __attribute__((always_inline)) {
        const int kt = step + turn < nk ? step + turn : step + turn - nk;
        const uint32_t st = lds0 + (step % kMidStages) * kMidStageB;
        const unsigned char* const w = wb + kt * kRowB;
        const unsigned char* const x = xb + kt * kRowB;
        if (kt < whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) dma16_to(w, woff[i], st + kMidM * kRowB + i * 1024);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < nx) dma16_to(x, xoff[i], st + i * 1024);
        } else {
            const int left = kb - kt * kRowB;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool on = (chunk0 ^ (i & 1)) * 16 < left;
                dma16_to(on ? w + woff[i] : kZeros, st + kMidM * kRowB + i * 1024);
                if (i < nx) dma16_to(on ? x + xoff[i] : kZeros, st + i * 1024);
            }
        }
    };
    const int lrow = lane & 15, grp = lane >> 4;
    const int cperm = ((grp & 1) << 1) | (grp >> 1);
    int kpos[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) kpos[ks] = lrow * kRowB + (((4 * ks + cperm) ^ swz(lrow)) << 4);
    const int wr = wave >> 1, wc = wave & 1;
    const int a0 = wr * 64 * kRowB, b0 = (kMidM + 64 * wc) * kRowB;
    typename M::Acc acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[i][j][v] = 0;
    const int mi = (t.rows - 64 * wr + 15) / 16;
    issue(0);
    for (int kt = 0; kt < nk; ++kt) {
        wait_vmcnt<0>();
        __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0)
        plain_barrier();
        if (kt + 1 < nk) issue(kt + 1);
        const unsigned char* st = lds + (kt % kMidStages) * kMidStageB;
        auto frag = [&](int at) __attribute__((always_inline)) {
            return __builtin_bit_cast(typename M::Frag, *(const u32x4*)(st + at));
        };
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            typename M::Frag w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = frag(b0 + 16 * j * kRowB + kpos[ks]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= mi) continue;
                const typename M::Frag x = frag(a0 + 16 * i * kRowB + kpos[ks]);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = M::mul(w[j], x, acc[i][j]);
            }
        }
    }
    // lane l holds columns 4 (l / 16) .. + 3 of row l % 16
    const float* sw = sizeof(E) == 1 ? a.w_scale + (int64_t)t.expert * a.C : nullptr;
    f32x4 s4[4];
    const int col = c0 + 64 * wc + 4 * grp;
#pragma unroll
    for (int j = 0; j < 4; ++j) s4[j] = sizeof(E) == 1 ? four_scales(sw, col + 16 * j, a.C) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 64 * wr + 16 * i + lrow;
        if (r >= t.rows) continue;
        const int src = source(a, t.row0 + r);
        const float sr = sizeof(E) == 1 ? a.row_scale[max(src, 0)] : 0.0f;
        O* row = (O*)a.out + (int64_t)(t.row0 + r) * a.C;
#pragma unroll
        for (int j = 0; j < 4; ++j) store_four(row, col + 16 * j, a.C, finish<E>(acc[i][j], src >= 0, sr, s4[j]));
    }
}

// Few rows or few outputs: what counts is how many workgroups there are and how long each one's chain of
// loads is.  32 rows x 32 columns, the four wavefronts of a workgroup take every fourth 128 bytes
// of K, straight from memory into the MFMAs' layout (a fragment is 16 bytes of a row, from any
// address), two pairs of 64 bytes in flight; their sums meet in LDS, in order.
template <typename E, typename O, bool ANY>
__global__ void __launch_bounds__(256) mm_thin_kernel(MmArgs a) {
    using M = Mma<E>;
    using Acc = typename M::Acc;
    constexpr int RB = 2, CB = 2, kRows = 16 * RB, kCols = 16 * CB;
    __shared__ __attribute__((aligned(16))) Acc sums[4][RB * CB][64];
    RowTile t;
    if (!find_tile(a.offsets, a.N, a.R, kRows, (a.C + kCols - 1) / kCols, block_number(), &t)) return;
    if (t.expert >= a.N) {
        zero_tile<O>(a, t, kCols, 256);
        return;
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lrow = lane & 15, grp = lane >> 4;
    const int c0 = t.panel * kCols;
    const int kb = a.K * (int)sizeof(E);
    const unsigned char *x[RB], *w[CB];
    uint32_t xd[RB], wd[CB];
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        const int src = source(a, t.row0 + min(16 * i + lrow, t.rows - 1));
        x[i] = (const unsigned char*)a.x + (int64_t)max(src, 0) * kb;
        xd[i] = (uint32_t)(uintptr_t)x[i] & 3;
    }
#pragma unroll
    for (int j = 0; j < CB; ++j) {
        w[j] = (const unsigned char*)a.W + ((int64_t)t.expert * a.C + min(c0 + 16 * j + lrow, a.C - 1)) * kb;
        wd[j] = (uint32_t)(uintptr_t)w[j] & 3;
    }
    Acc acc[RB][CB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[i][j][v] = 0;
    struct Set {
        Piece<ANY> x[2][RB], w[2][CB];
    };
    auto mul = [&](const Set& s) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            typename M::Frag fx[RB], fw[CB];
#pragma unroll
            for (int i = 0; i < RB; ++i) fx[i] = __builtin_bit_cast(typename M::Frag, s.x[h][i].bytes(xd[i]));
#pragma unroll
            for (int j = 0; j < CB; ++j) fw[j] = __builtin_bit_cast(typename M::Frag, s.w[h][j].bytes(wd[j]));
#pragma unroll
            for (int k = 0; k < M::kSteps; ++k)     // (a step of every block before the next: none waits for its own sum)
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int j = 0; j < CB; ++j) acc[i][j] = M::step(fw[j], fx[i], k, acc[i][j]);
        }
    };
    auto load = [&](Set& s, int at) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < CB; ++j) s.w[h][j].load(w[j] + at + 64 * h + 16 * grp);
#pragma unroll
            for (int i = 0; i < RB; ++i) s.x[h][i].load(x[i] + at + 64 * h + 16 * grp);
        }
    };
    int at = 128 * wave;
    Set s0, s1;
    const int whole = kb - 128;             // last place with 128 bytes behind it
    if (at <= whole) load(s0, at);
    for (; at <= whole; at += 1024) {
        const bool two = at + 512 <= whole;
        if (two) load(s1, at + 512);
        mul(s0);
        if (at + 1024 <= whole) load(s0, at + 1024);
        if (two) mul(s1);
    }
    // the row's last bytes, fewer than 128: of one wavefront, zeros behind them
    const int rest = kb / 128 * 128;
    if (rest < kb && (kb / 128) % 4 == wave) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < CB; ++j) {
                s0.w[h][j].w = load16_bytes(w[j], rest + 64 * h + 16 * grp, kb);
                wd[j] = 0;
            }
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                s0.x[h][i].w = load16_bytes(x[i], rest + 64 * h + 16 * grp, kb);
                xd[i] = 0;
            }
        }
        mul(s0);
    }
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) sums[wave][i * CB + j][lane] = acc[i][j];
    __syncthreads();
    // block b: wavefront b % 4; lane l holds columns 4 (l / 16) .. + 3 of row l % 16
    const float* sw = sizeof(E) == 1 ? a.w_scale + (int64_t)t.expert * a.C : nullptr;
#pragma unroll
    for (int b0 = 0; b0 < RB * CB; b0 += 4) {
        const int b = b0 + wave;
        if (b >= RB * CB) continue;
        Acc v = sums[0][b][lane];
#pragma unroll
        for (int q = 1; q < 4; ++q) v += sums[q][b][lane];
        const int r = 16 * (b / CB) + lrow, c = c0 + 16 * (b % CB) + 4 * grp;
        if (r >= t.rows || c >= a.C) continue;
        const int src = source(a, t.row0 + r);
        f32x4 s4 = {0.0f, 0.0f, 0.0f, 0.0f};
        if (sizeof(E) == 1) s4 = four_scales(sw, c, a.C);
        const float sr = sizeof(E) == 1 ? a.row_scale[max(src, 0)] : 0.0f;
        store_four((O*)a.out + (int64_t)(t.row0 + r) * a.C, c, a.C, finish<E>(v, src >= 0, sr, s4));
    }
}

// The same of dx = dy W: a wavefront takes every fourth K (n_out) step of 32 (fp32: 16), a lane E columns of
// E K rows (16 bytes each, 256 bytes of a row by 16 lanes).  MFMA j has the j-th of every lane's columns, so
// that the lane's own pieces hold its fragments, transposed in registers for bf16 (for fp32 an
// element is a fragment).
template <typename T> struct BackMma;
template <> struct BackMma<bf16_t> {
    // column j of 8 K rows of 8 columns
    __device__ __forceinline__ static bf16x8 column(const u32x4 (&w)[8], int j) {
        u32x4 f;
        const uint32_t pick = j & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_perm(w[2 * i + 1][j / 2], w[2 * i][j / 2], pick);
        return __builtin_bit_cast(bf16x8, f);
    }
    __device__ __forceinline__ static f32x4 mul(const u32x4 (&w)[8], int j, const u32x4& x, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(column(w, j), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
    }
};
template <> struct BackMma<float> {
    __device__ __forceinline__ static f32x4 mul(const u32x4 (&w)[4], int j, const u32x4& x, f32x4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i][j]), __uint_as_float(x[i]), c, 0, 0, 0);
        return c;
    }
};

template <typename T, int RB>
__global__ void __launch_bounds__(256) mm_back_thin_kernel(MmArgs a) {
    constexpr int E = Chunk<T>::E;              // columns and K rows of a lane
    constexpr int kRows = 16 * RB, kCols = 16 * E, kK = 4 * E;
    __shared__ __attribute__((aligned(16))) f32x4 sums[4][RB * E][64];
    RowTile t;
    if (!find_tile(a.offsets, a.N, a.R, kRows, (a.C + kCols - 1) / kCols, block_number(), &t)) return;
    if (t.expert >= a.N) {
        zero_tile<T>(a, t, kCols, 256);
        return;
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lrow = lane & 15, grp = lane >> 4;
    const int c = t.panel * kCols + E * lrow;
    const T* x[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i) x[i] = (const T*)a.x + (int64_t)(t.row0 + min(16 * i + lrow, t.rows - 1)) * a.K;
    const T* w = (const T*)a.W + (int64_t)t.expert * a.K * a.C;
    f32x4 acc[RB][E];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int full = a.C / E, rem = a.C % E;
    struct Set {
        u32x4 x[RB], w[E];
    };
    auto load = [&](Set& s, int k0) __attribute__((always_inline)) {
        const int k = k0 + E * grp;
#pragma unroll
        for (int i = 0; i < RB; ++i) s.x[i] = load_chunk(x[i], k / E, a.K / E, a.K % E);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            s.w[i] = load_chunk(w + (int64_t)min(k + i, a.K - 1) * a.C, c / E, full, rem);
            if (k + i >= a.K) s.w[i] = u32x4{0, 0, 0, 0};
        }
    };
    auto mul = [&](const Set& s) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < E; ++j)
#pragma unroll
            for (int i = 0; i < RB; ++i) acc[i][j] = BackMma<T>::mul(s.w, j, s.x[i], acc[i][j]);
    };
    Set s0, s1;
    int k0 = kK * wave;
    if (k0 < a.K) load(s0, k0);
    for (; k0 < a.K; k0 += 8 * kK) {
        const bool two = k0 + 4 * kK < a.K;
        if (two) load(s1, k0 + 4 * kK);
        mul(s0);
        if (k0 + 8 * kK < a.K) load(s0, k0 + 8 * kK);
        if (two) mul(s1);
    }
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) sums[wave][i * E + j][lane] = acc[i][j];
    __syncthreads();
    // Lane l of MFMA j holds row l % 16 and of columns E m + j those with m = 4 (l / 16) + v: wavefront q
    // takes v = q, whose E columns are consecutive.
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        const int r = 16 * i + lrow;
        if (r >= t.rows) continue;
        float y[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            float v = 0.0f;
#pragma unroll
            for (int q = 0; q < 4; ++q) v += ((const float*)&sums[q][i * E + j][lane])[wave];
            y[j] = v;
        }
        store_chunk((T*)a.out + (int64_t)(t.row0 + r) * a.C, t.panel * 16 + 4 * grp + wave, full, rem, y);
    }
}

// dx = dy W on v_mfma_f32_32x32x16_bf16 (n_out and n_in multiples of 8): 256 x 256 outputs, K = n_out in
// steps of 32 through a ring of four stages.  The rows of dy run along K (64 bytes of each a
// step); the weights lie along their columns, 32 K rows of 512 bytes, and are read as fragments by the
// transposing LDS read.
constexpr int kBK = 32;
constexpr int kBStages = 4, kCopies = 4;
constexpr int kOpB = kBK * 512;
constexpr int kBStageB = 2 * kOpB;
constexpr int BI = WM / 32, BJ = WN / 32;

// chunk c of a 64-byte LDS row r lies at c ^ rswz(r)
__device__ __forceinline__ int rswz(int r) { return (r >> 2) & 3; }

__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
mm_back_wide_kernel(MmArgs a) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kBStages * kBStageB];
    RowTile t;
    if (!find_tile(a.offsets, a.N, a.R, BM, (a.C + BP - 1) / BP, block_number(), &t)) return;
    if (t.expert >= a.N) {
        zero_tile<bf16_t>(a, t, BP, kThreads);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave >> 1, wc = wave & 1;
    const int half = wave >> 2, wq = wave & 3;      // copies: 0 the rows of dy, 1 the weights
    const int c0 = t.panel * BP;
    const bool active = wr * WM < t.rows && c0 + wc * WN < a.C;
    const int hi = lane >> 5;
    const bf16_t* const xb = (const bf16_t*)a.x + (int64_t)t.row0 * a.K;
    const bf16_t* const wb = (const bf16_t*)a.W + (int64_t)t.expert * a.K * a.C + c0;
    uint32_t off[kCopies];
    int xk = 0;                                     // first K of this lane's chunk of a step, copies 0 and 2
    if (half == 0) {
        // copy i: rows 64 wq + 16 i + lane / 4
        xk = 8 * ((lane & 3) ^ rswz(lane / 4));
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int r = 64 * wq + 16 * i + lane / 4;
            off[i] = 2u * ((uint32_t)min(r, t.rows - 1) * (uint32_t)a.K + xk);
        }
    } else {
        // copy i: K rows 8 wq + 2 i (lanes 0-31) and + 1, chunk c of K row kr at c ^ 4 (kr & 3).  (Columns
        // past the matrix read the panel's first: they reach only outputs that are not stored.)
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int c = 8 * ((lane & 31) ^ (4 * (hi + 2 * (i & 1))));
            off[i] = 2u * ((uint32_t)hi * (uint32_t)a.C + (c0 + c < a.C ? c : 0));
        }
    }
    const int whole = a.K / kBK;
    const int nh = max(kBStages, (a.K + kBK - 1) / kBK);
    const uint32_t lds0 = lds_address(lds) + half * kOpB + wq * 4096;
    const bf16_t* const from0 = half == 0 ? xb : wb + (int64_t)(8 * wq) * a.C;
    const int64_t of_step = half == 0 ? kBK : (int64_t)kBK * a.C, of_copy = half == 0 ? 0 : 2 * (int64_t)a.C;
    // copy i of step h; PART: the step may pass the last K
    auto issue = [&](auto PART, int h, int i) __attribute__((always_inline)) {
        const uint32_t to = lds0 + (h % kBStages) * kBStageB + i * 1024;
        const bf16_t* const from = from0 + h * of_step + i * of_copy;
        if (!decltype(PART)::value) {
            dma16_to(from, off[i], to);
        } else {
            const int k = h * kBK + (half == 0 ? xk : 8 * wq + 2 * i + hi);
            dma16_to(k < a.K ? (const unsigned char*)from + off[i] : kZeros, to);
        }
    };
    auto issue_all = [&](auto PART, int h) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) issue(PART, h, i);
    };

    f32x16 acc[BI][BJ];
#pragma unroll
    for (int i = 0; i < BI; ++i)
#pragma unroll
        for (int j = 0; j < BJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
    const int lrow = lane & 31;
    int kpos[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) kpos[ks] = lrow * 64 + (((2 * ks + hi) ^ rswz(lrow)) << 4);
    // weights: two transposing reads a fragment, each of four K values of a column
    const int s16 = lane & 15, g4 = lane >> 4;
    const int nl = 16 * (g4 & 1) + 4 * (s16 & 3);
    const int kl = 8 * (g4 >> 1) + (s16 >> 2);
    const int tsw = (nl >> 3) ^ (4 * (kl & 3));
    int a_pos[BI], b_pos[BJ];
#pragma unroll
    for (int i = 0; i < BI; ++i) a_pos[i] = (wr * WM + i * 32) * 64;
#pragma unroll
    for (int j = 0; j < BJ; ++j)
        b_pos[j] = kOpB + kl * 512 + (((wc * WN + j * 32) >> 3 ^ tsw) << 4) + ((nl & 4) << 1);
    auto wait_steps = [&](int n) __attribute__((always_inline)) {
        if (n >= 2) wait_vmcnt<2 * kCopies>();
        else if (n == 1) wait_vmcnt<kCopies>();
        else wait_vmcnt<0>();
    };
    auto barrier = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0)
        plain_barrier();
    };
    bf16x8 fa[2][BI], fb[2][BJ];
    auto tr_frag = [&](const unsigned char* p) __attribute__((always_inline)) {
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)p);
        const v4s hi4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p + 4 * 512));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi4, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto row_frag = [&](const unsigned char* p) __attribute__((always_inline)) {
        return __builtin_bit_cast(bf16x8, *(const u32x4*)p);
    };
    // MFMAs on fragment set S, among them the reads of sub-step ks of a stage into the other set and copy(0 .. 3)
    auto phase = [&](auto S_, int stage, int ks, auto copy) __attribute__((always_inline)) {
        constexpr int S = decltype(S_)::value;
        const unsigned char* st = lds + stage * kBStageB;
#pragma unroll
        for (int j = 0; j < BJ; ++j) {
            copy(j);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < BI; ++i)
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[S][j], fa[S][i], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (j == 0) {
                fa[S ^ 1][0] = row_frag(st + a_pos[0] + kpos[ks]);
                fa[S ^ 1][1] = row_frag(st + a_pos[1] + kpos[ks]);
                fb[S ^ 1][0] = tr_frag(st + b_pos[0] + ks * 8192);
            } else if (j == 1) {
                fb[S ^ 1][1] = tr_frag(st + b_pos[1] + ks * 8192);
                fb[S ^ 1][2] = tr_frag(st + b_pos[2] + ks * 8192);
                fb[S ^ 1][3] = tr_frag(st + b_pos[3] + ks * 8192);
            }
        }
    };
    using C0 = std::integral_constant<int, 0>;
    using C1 = std::integral_constant<int, 1>;
#pragma unroll
    for (int h = 0; h < kBStages; ++h) issue_all(C1{}, h);
    wait_vmcnt<3 * kCopies>();
    barrier();
    int h = 0;
    if (active) {
#pragma unroll
        for (int i = 0; i < BI; ++i) fa[0][i] = row_frag(lds + a_pos[i] + kpos[0]);
#pragma unroll
        for (int j = 0; j < BJ; ++j) fb[0][j] = tr_frag(lds + b_pos[j]);
        auto no_copy = [](int) {};
        // step h with the copies of step h + kBStages
        auto step = [&](auto PART) __attribute__((always_inline)) {
            phase(C0{}, h % kBStages, 1, no_copy);
            wait_vmcnt<2 * kCopies>();
            barrier();
            phase(C1{}, (h + 1) % kBStages, 0, [&](int j) __attribute__((always_inline)) { issue(PART, h + kBStages, j); });
        };
        for (; h + kBStages < whole; ++h) step(C0{});
        for (; h + kBStages < nh; ++h) step(C1{});
        for (; h < nh; ++h) {
            phase(C0{}, h % kBStages, 1, no_copy);
            wait_steps(nh - 2 - h);
            barrier();
            // (past the last step the reads fetch an old stage; unused)
            phase(C1{}, (h + 1) % kBStages, 0, no_copy);
        }
    } else {
        for (; h < nh; ++h) {
            wait_steps(min(nh - 1, h + kBStages - 1) - (h + 1));
            barrier();
            if (h + kBStages < nh) issue_all(C1{}, h + kBStages);
        }
    }
    // Lane l holds row l % 32 of each 32-row block, columns 8 (v / 4) + 4 (l / 32) + v % 4 of each
    // 32-column block; staged as the product's outputs are.
    __syncthreads();
    if (!active) return;
    constexpr int RB = WN * 2, NCH = RB / 16;
    unsigned char* sw = lds + wave * (WM * RB);
#pragma unroll
    for (int i = 0; i < BI; ++i) {
        const int row = i * 32 + lrow;
#pragma unroll
        for (int j = 0; j < BJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; v += 4) {
                const int col = j * 32 + 2 * v + 4 * hi;
                const uint32_t w0 = (uint32_t)f32_to_bf16(acc[i][j][v]) | (uint32_t)f32_to_bf16(acc[i][j][v + 1]) << 16;
                const uint32_t w1 = (uint32_t)f32_to_bf16(acc[i][j][v + 2]) | (uint32_t)f32_to_bf16(acc[i][j][v + 3]) << 16;
                *(uint2*)(sw + row * RB + (((col >> 3) ^ (row & (NCH - 1))) << 4) + (((col & 4) << 1) ^ (row & 8))) =
                    make_uint2(w0, w1);
            }
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);
    __builtin_amdgcn_wave_barrier();
    const int ch = lane % NCH;
    const int col = c0 + wc * WN + ch * 8;
#pragma unroll
    for (int p = 0; p < WM / (64 / NCH); ++p) {
        const int row = p * (64 / NCH) + lane / NCH;
        const int r = wr * WM + row;
        u32x4 v = *(const u32x4*)(sw + row * RB + ((ch ^ (row & (NCH - 1))) << 4));
        if (row & 8) v = u32x4{v[2], v[3], v[0], v[1]};
        if (r < t.rows && col < a.C) *(u32x4*)((bf16_t*)a.out + (int64_t)(t.row0 + r) * a.C + col) = v;
    }
}

// out = 0 (no row has a source)
__global__ void __launch_bounds__(256) mm_zero_kernel(uint32_t* p, int64_t words, uint16_t* last) {
    const int64_t i = (int64_t)block_number() * 256 + threadIdx.x;
    if (i < words) p[i] = 0;
    if (i == 0 && last) *last = 0;
}

// ------------------------------------------------------------------ host ----
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, uintptr_t n) { return (uintptr_t)p % n == 0; }

pr2_status check_mm(const pr2_wgrad_desc* desc, bool source_rows) {
    if (!desc) return fail(PR2_ERR_NULL, "desc is NULL");
    const pr2_wgrad_desc& d = *desc;
    if (d.act_dtype != PR2_F32 && d.act_dtype != PR2_BF16)
        return fail(PR2_ERR_DTYPE, "act_dtype %d is not PR2_F32 or PR2_BF16", d.act_dtype);
    if (d.R < 0) return fail(PR2_ERR_SHAPE, "R = %lld < 0", (long long)d.R);
    if (source_rows && d.Rx < 0) return fail(PR2_ERR_SHAPE, "Rx = %lld < 0", (long long)d.Rx);
    if (d.n_out < 1 || d.n_in < 1) return fail(PR2_ERR_SHAPE, "n_out = %d or n_in = %d < 1", d.n_out, d.n_in);
    if (d.N < 1) return fail(PR2_ERR_SHAPE, "N = %d < 1", d.N);
    if (source_rows && d.k < 1) return fail(PR2_ERR_SHAPE, "k = %d < 1", d.k);
    if (d.N > kMaxExperts) return fail(PR2_ERR_UNSUPPORTED, "N = %d > %d", d.N, kMaxExperts);
    if (d.R > 0x7fffffff - 1024 || (source_rows && d.Rx > 0x7fffffff - 1024))
        return fail(PR2_ERR_UNSUPPORTED, "R = %lld or Rx = %lld rows exceed 2^31 - 1025", (long long)d.R,
                    (long long)d.Rx);
    if (d.n_out > (1 << 20) || d.n_in > (1 << 20))
        return fail(PR2_ERR_UNSUPPORTED, "n_out = %d or n_in = %d > 2^20", d.n_out, d.n_in);
    if ((int64_t)d.N * d.n_out * d.n_in > (int64_t)1 << 36)
        return fail(PR2_ERR_UNSUPPORTED, "N n_out n_in > 2^36");
    const int64_t groups = tile_groups(d.R, d.N, 16, ceil_div(std::max(d.n_out, d.n_in), 32));     // no kernel has more
    if (groups > 0x7fffffff) return fail(PR2_ERR_UNSUPPORTED, "R rows of these widths are more than 2^31 tiles");
    return PR2_OK;
}

// rows, their weights and the plan; the caller has checked desc and that R > 0
pr2_status check_mm_args(const pr2_wgrad_desc& d, const void* x, const char* x_name, const void* W,
                         const int32_t* offsets, const int32_t* route, bool gathers, const void* out,
                         const char* out_name, size_t x_bytes, size_t w_bytes, size_t out_bytes) {
    if ((!x && !(gathers && d.Rx == 0)) || !W || !out) return fail(PR2_ERR_NULL, "%s, W and %s are required", x_name, out_name);
    if (!offsets && d.N != 1) return fail(PR2_ERR_NULL, "offsets is NULL with N = %d > 1", d.N);
    if (!aligned(x, 16) || !aligned(W, 16) || !aligned(out, 16))
        return fail(PR2_ERR_ALIGN, "%s, W or %s is not 16-byte aligned", x_name, out_name);
    if (!aligned(offsets, 4) || !aligned(route, 4))
        return fail(PR2_ERR_ALIGN, "offsets or route_of_row is not 4-byte aligned");
    if (gathers && !route && d.R > d.Rx)
        return fail(PR2_ERR_SHAPE, "R = %lld > Rx = %lld without route_of_row", (long long)d.R, (long long)d.Rx);
    if (share_memory(out, out_bytes, x, x_bytes) || share_memory(out, out_bytes, W, w_bytes))
        return fail(PR2_ERR_SHAPE, "%s overlaps %s or W", out_name, x_name);
    return PR2_OK;
}

size_t act_bytes(const pr2_wgrad_desc& d) { return d.act_dtype == PR2_BF16 ? 2 : 4; }
size_t weights_of(const pr2_wgrad_desc& d) { return (size_t)d.N * d.n_out * d.n_in; }

hipError_t launch_zero(void* out, int64_t bytes, hipStream_t st) {
    LaunchScope scope("mm_zero", st);
    const int64_t words = bytes / 4;
    hipLaunchKernelGGL(mm_zero_kernel, wide_grid(std::max<int64_t>(1, ceil_div(words, 256)), 256), dim3(256), 0, st,
                       (uint32_t*)out, words, bytes % 4 ? (uint16_t*)out + bytes / 2 - 1 : nullptr);
    return hipGetLastError();
}

template <typename K>
hipError_t launch_tiles(const char* name, K kernel, const MmArgs& a, int rows, int columns, int threads,
                        hipStream_t st) {
    LaunchScope scope(name, st);
    hipLaunchKernelGGL(kernel, wide_grid(tile_groups(a.R, a.N, rows, ceil_div(a.C, columns)), threads), dim3(threads),
                       0, st, a);
    return hipGetLastError();
}

// Whether the copies reach every row: whole 16-byte chunks, and 32-bit offsets into gathered rows (into
// sorted ones they start at the tile).  Gathered rows past 4 GiB go through registers: 1052672 of 2048 to 1536 outputs in 128
// experts 13.2 ms, sorted 5.3, and 1044480 through the plan 5.2.
bool mfma_ok(const MmArgs& a, int64_t element) {
    return a.K * element % 16 == 0 && (!a.route || (int64_t)a.Rx * a.K * element < (int64_t)1 << 32);
}

// Which tile: the one that is expected to take the least time.  In us, fitted to products of 1, 8 and 64
// experts of 1 to 1024 rows, 256 to 2048 columns, 512 to 4096 bytes of K, bf16 and int8, every kernel
// at each of the 190 sizes (378 for both types): alone on its CU a tile takes start + chain a slice of 128
// bytes of K, and where all CUs are busy a CU takes 1 + busy a slice for each of its tiles (wide
// tiles, one on a CU, in whole rounds).
// By this rule the products take 0.9 % more than by the best kernel at each of 147 sizes, 35 % (7.1 us for
// 5.2) at most; with the 256-row tile alone 2.4 times as long at the sizes of one expert.  (Fitted before that tile took its
// rows in turns, which made one that is not full cheaper than "half full" below says; not fitted again since.)
struct TileCost {
    int rows, columns;
    float start, chain, busy;
    bool rounds;            // one tile fills a CU
};
constexpr TileCost kThinCost{32, 32, 1.8f, 0.11f, 0.16f, false};
constexpr TileCost kThinAnyCost{32, 32, 1.8f, 0.2f, 0.33f, false};     // rows off 4 bytes
constexpr TileCost kThinF32Cost{32, 32, 1.8f, 0.11f, 0.2f, false};
constexpr TileCost kFewCost{kFewM, kFewP, 0.95f, 0.645f, 0.535f, false};
constexpr TileCost kMidCost{kMidM, kMidP, 1.4f, 0.68f, 0.74f, false};
constexpr TileCost kWideCost{BM, BP, 3.5f, 0.75f, 2.0f, true};
constexpr TileCost kTileF32Cost{kTile, kTile, 1.5f, 0.72f, 0.55f, false};
constexpr TileCost kTileAnyCost{kTile, kTile, 1.5f, 0.7f, 0.45f, false};
constexpr TileCost kBackThin1Cost{16, 128, 1.4f, 0.5f, 0.286f, false};
constexpr TileCost kBackThin2Cost{32, 128, 1.0f, 0.62f, 0.477f, false};
constexpr TileCost kBackThin1F32Cost{16, 64, 1.4f, 0.25f, 0.2f, false};
constexpr TileCost kBackWideCost{BM, BP, 2.6f, 1.16f, 1.6f, true};

float tile_time(const MmArgs& a, int element, const TileCost& t) {
    constexpr float kCus = 256.0f;
    // experts with rows, of routes that fall evenly, and their tiles, the last one of each half full
    const float N = (float)a.N, R = (float)a.R;
    const float experts = N * (1.0f - expf(-R / N));
    const float tiles = std::max(experts, R / (float)t.rows + 0.5f * experts);
    const float items = std::ceil(tiles) * (float)ceil_div(a.C, t.columns);
    const float slices = (float)a.K * (float)element / 128.0f;
    const float one = t.start + t.chain * slices, loaded = 1.0f + t.busy * slices;
    float time = std::max(one, items / kCus * loaded);
    if (t.rounds) {
        const float full = std::floor(items / kCus);
        const float last = items / kCus - full;
        time = full * std::max(loaded, one) + (last > 0.0f ? one + last * std::max(loaded - one, 0.0f) : 0.0f);
    }
    return time;
}

template <typename E, typename O>
hipError_t launch_product(const MmArgs& a, hipStream_t st) {
    constexpr bool f32 = sizeof(E) == 4, i8 = sizeof(E) == 1;
    constexpr float kNever = 3e38f;
    const bool words = a.K * (int)sizeof(E) % 4 == 0;
    const float thin = tile_time(a, sizeof(E), f32 ? kThinF32Cost : words ? kThinCost : kThinAnyCost);
    float few = kNever, mid = kNever, wide = kNever, tile = kNever;
    if (!f32 && mfma_ok(a, sizeof(E))) {
        few = tile_time(a, sizeof(E), kFewCost);
        mid = tile_time(a, sizeof(E), kMidCost);
        wide = tile_time(a, sizeof(E), kWideCost);
    } else {
        tile = tile_time(a, sizeof(E), f32 ? kTileF32Cost : kTileAnyCost);
    }
    const float least = std::min({thin, few, mid, wide, tile});
    if constexpr (!f32) {
        if (few == least) return launch_tiles("mm_few", mm_few_kernel<E, O>, a, kFewM, kFewP, 256, st);
        if (mid == least) return launch_tiles("mm_mid", mm_mid_kernel<E, O>, a, kMidM, kMidP, 256, st);
        if constexpr (sizeof(O) == 2)
            if (wide == least && (int64_t)a.R * a.C * 2 >= kStreamBytes)
                return launch_tiles("mm_wide", mm_wide_kernel<E, O, true>, a, BM, BP, kThreads, st);
        if (wide == least) return launch_tiles("mm_wide", mm_wide_kernel<E, O, false>, a, BM, BP, kThreads, st);
        if (thin == least && !words) return launch_tiles("mm_thin", mm_thin_kernel<E, O, true>, a, 32, 32, 256, st);
    }
    if (thin == least) return launch_tiles("mm_thin", mm_thin_kernel<E, O, false>, a, 32, 32, 256, st);
    if constexpr (f32) return launch_tiles("mm_tile", mm_tile_kernel<false>, a, kTile, kTile, 256, st);
    else return launch_tiles("mm_tile", mm_any_kernel<E, O, false>, a, kTile, kTile, 256, st);
}

hipError_t launch_back_f32(const MmArgs& a, hipStream_t st) {
    if (tile_time(a, 4, kBackThin1F32Cost) <= tile_time(a, 4, kTileF32Cost))
        return launch_tiles("mm_back_thin", mm_back_thin_kernel<float, 1>, a, 16, 64, 256, st);
    return launch_tiles("mm_back_tile", mm_tile_kernel<true>, a, kTile, kTile, 256, st);
}

hipError_t launch_back_bf16(const MmArgs& a, hipStream_t st) {
    if (a.K % 8 || a.C % 8)
        return launch_tiles("mm_back_tile", mm_any_kernel<bf16_t, bf16_t, true>, a, kTile, kTile, 256, st);
    const float one = tile_time(a, 2, kBackThin1Cost), two = tile_time(a, 2, kBackThin2Cost);
    if (tile_time(a, 2, kBackWideCost) < std::min(one, two))
        return launch_tiles("mm_back_wide", mm_back_wide_kernel, a, BM, BP, kThreads, st);
    if (one <= two) return launch_tiles("mm_back_thin", mm_back_thin_kernel<bf16_t, 1>, a, 16, 128, 256, st);
    return launch_tiles("mm_back_thin2", mm_back_thin_kernel<bf16_t, 2>, a, 32, 128, 256, st);
}

}  // namespace
}  // namespace pr2

using namespace pr2;

extern "C" {

pr2_status pr2_grouped_mm(const pr2_wgrad_desc* desc, const void* x, const void* W, const int32_t* offsets,
                          const int32_t* route_of_row, void* out, pr2_stream_t stream) {
    pr2_status s = check_mm(desc, true);
    if (s != PR2_OK) return s;
    const pr2_wgrad_desc& d = *desc;
    if (d.R == 0) return ok();
    const size_t a1 = act_bytes(d);
    if ((s = check_mm_args(d, x, "x", W, offsets, route_of_row, true, out, "out", a1 * d.Rx * d.n_in,
                           a1 * weights_of(d), a1 * d.R * d.n_out)) != PR2_OK)
        return s;
    if ((s = device_ready()) != PR2_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    const MmArgs a{x, W, offsets, route_of_row, out, nullptr, nullptr, (int)d.R, (int)d.Rx, d.n_in, d.n_out, d.N, d.k};
    const hipError_t e = d.Rx == 0 ? launch_zero(out, d.R * d.n_out * act_bytes(d), st)
                        : d.act_dtype == PR2_BF16 ? launch_product<bf16_t, bf16_t>(a, st)
                                                  : launch_product<float, float>(a, st);
    if (e != hipSuccess) return hip_fail(e, "grouped_mm launch");
    return ok();
}

pr2_status pr2_grouped_mm_backward(const pr2_wgrad_desc* desc, const void* dy, const void* W,
                                   const int32_t* offsets, void* dx, pr2_stream_t stream) {
    pr2_status s = check_mm(desc, false);
    if (s != PR2_OK) return s;
    const pr2_wgrad_desc& d = *desc;
    if (d.R == 0) return ok();
    const size_t a1 = act_bytes(d);
    if ((s = check_mm_args(d, dy, "dy", W, offsets, nullptr, false, dx, "dx", a1 * d.R * d.n_out,
                           a1 * weights_of(d), a1 * d.R * d.n_in)) != PR2_OK)
        return s;
    if ((s = device_ready()) != PR2_OK) return s;
    const MmArgs a{dy, W, offsets, nullptr, dx, nullptr, nullptr, (int)d.R, (int)d.R, d.n_out, d.n_in, d.N, 1};
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = d.act_dtype == PR2_BF16 ? launch_back_bf16(a, st) : launch_back_f32(a, st);
    if (e != hipSuccess) return hip_fail(e, "grouped_mm_backward launch");
    return ok();
}

pr2_status pr2_grouped_mm_quant(const pr2_wgrad_desc* desc, const int8_t* q, const float* row_scale,
                                const int8_t* Wq, const float* w_scale, const int32_t* offsets,
                                const int32_t* route_of_row, void* out, pr2_stream_t stream) {
    pr2_status s = check_mm(desc, true);
    if (s != PR2_OK) return s;
    const pr2_wgrad_desc& d = *desc;
    if (d.n_in >= 1 << 17) return fail(PR2_ERR_UNSUPPORTED, "n_in = %d: sums of 2^17 or more products", d.n_in);
    if (d.R == 0) return ok();
    if ((!row_scale && d.Rx > 0) || !w_scale) return fail(PR2_ERR_NULL, "row_scale and w_scale are required");
    if ((s = check_mm_args(d, q, "q", Wq, offsets, route_of_row, true, out, "out", (size_t)d.Rx * d.n_in,
                           weights_of(d), act_bytes(d) * d.R * d.n_out)) != PR2_OK)
        return s;
    if (!aligned(row_scale, 4) || !aligned(w_scale, 4))
        return fail(PR2_ERR_ALIGN, "row_scale or w_scale is not 4-byte aligned");
    if ((s = device_ready()) != PR2_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    const MmArgs a{q, Wq, offsets, route_of_row, out, row_scale, w_scale, (int)d.R, (int)d.Rx, d.n_in, d.n_out,
                   d.N, d.k};
    const hipError_t e = d.Rx == 0 ? launch_zero(out, d.R * d.n_out * act_bytes(d), st)
                                   : d.act_dtype == PR2_BF16 ? launch_product<int8_t, bf16_t>(a, st)
                                                  : launch_product<int8_t, float>(a, st);
    if (e != hipSuccess) return hip_fail(e, "grouped_mm_quant launch");
    return ok();
}

}  // extern "C"
