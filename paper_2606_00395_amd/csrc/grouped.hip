// Products of rows sorted by expert with their experts' weights W [N, n_out, n_in]:
//
//   out[r, :] = x[src(r), :] W[e]^T           src(r) the token of row r's route, or r itself
//   dx[r, :]  = dy[r, :] W[e]                  the gradient of the row
//   out[r, o] = s_src(r) w[e, o] sum_c q[src(r), c] Wq[e, o, c]     both in 8 bits
//
// A row without a source and the rows behind the last expert's are zeros.
#include <algorithm>
#include <type_traits>

#include "chunk.h"
#include "rowtiles.h"

namespace pr2 {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef u32x4 u32x4_byte __attribute__((aligned(1)));

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

// the row of x behind row r of the product, -1 if it has none
__device__ __forceinline__ int source(const MmArgs& a, int r) {
    if (!a.route) return r;
    const int q = a.route[r];
    const int t = q / a.k;
    return q >= 0 && t < a.Rx ? t : -1;
}

// ------------------------------------------------ any type, width and row count --
// 64 x 64 outputs per workgroup, four wavefronts of 32 x 32 on v_mfma_f32_32x32x2_f32 (fp32
// products and sums), 32 K at a time staged in LDS as fp32, the next 32 in flight meanwhile.  An
// operand whose rows run along K lies in LDS as it comes and is read four K at a time; the weights of
// dy W, whose rows run along the columns, are read one K at a time.  A step's four K of either half
// wavefront are the same in both operands, so that any order of them gives the sum.
constexpr int kTile = 64;
constexpr int kStep = 32;
constexpr int kRowPitch = kStep + 4;        // 16-byte reads of 32 rows: every bank equally often
constexpr int kColPitch = kTile + 8;        // K rows 4 apart (the two half wavefronts) 32 banks apart

// 8 elements of a row from element c on, the ones past the row's n (or all, if !on) as 0
template <typename T>
__device__ __forceinline__ void load8(const T* row, int c, int n, bool on, u32x4 (&w)[8 / Chunk<T>::E]) {
    constexpr int E = Chunk<T>::E;
    if (on && c + 8 <= n) {
#pragma unroll
        for (int i = 0; i < 8 / E; ++i) w[i] = load16<false>(row + c + i * E);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8 / E; ++i) w[i] = u32x4{0, 0, 0, 0};
    if (!on) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (c + i >= n) continue;
        const uint32_t b = __builtin_bit_cast(typename Chunk<T>::Bits, row[c + i]);
        if (E == 4) w[i / 4][i % 4] = b;
        else w[0][i / 2] |= i & 1 ? b << 16 : b;
    }
}

// BACK: out = x W (W [K, C] an expert), else out = x W^T (W [C, K])
template <typename T, bool BACK>
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
    const T* W = (const T*)a.W + (int64_t)(len ? t.expert : 0) * a.K * a.C;

    const int ar = tid / 4, ak = (tid % 4) * 8;             // what this thread stages of x
    const int br = BACK ? tid / 8 : ar, bk = BACK ? (tid % 8) * 8 : ak;
    const int src = s_src[ar];
    const T* x = (const T*)a.x + (int64_t)max(src, 0) * a.K;
    constexpr int E = Chunk<T>::E;
    u32x4 wa[8 / E], wb[8 / E];
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
        float va[8], vb[8];
#pragma unroll
        for (int i = 0; i < 8 / E; ++i) {
            Chunk<T>::open(wa[i], va + i * E);
            Chunk<T>::open(wb[i], vb + i * E);
        }
        __syncthreads();
        float* const to = B + (BACK ? br * kColPitch : br * kRowPitch) + bk;
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            *(f32x4*)(A + ar * kRowPitch + ak + i) = f32x4{va[i], va[i + 1], va[i + 2], va[i + 3]};
            *(f32x4*)(to + i) = f32x4{vb[i], vb[i + 1], vb[i + 2], vb[i + 3]};
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
        if (r < t.rows)
            ((T*)a.out)[(int64_t)(t.row0 + r) * a.C + c] = Act<T>::from_f32(s_src[r] >= 0 ? acc[v] : 0.0f);
    }
}

// The same in 8 bits: 128 K at a time as bytes, v_mfma_i32_32x32x32_i8.
constexpr int kStep8 = 128;
constexpr int kPitch8 = kStep8 + 16;

// 16 bytes of a row from byte c on, those past the row's n as 0
__device__ __forceinline__ u32x4 load16_bytes(const int8_t* row, int c, int n) {
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

template <typename O>
__global__ void __launch_bounds__(256) mm8_tile_kernel(MmArgs a) {
    __shared__ __attribute__((aligned(16))) unsigned char A[kTile * kPitch8], B[kTile * kPitch8];
    __shared__ int s_src[kTile];
    RowTile t;
    if (!find_tile(a.offsets, a.N, a.R, kTile, (a.C + kTile - 1) / kTile, block_number(), &t)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int c0 = t.panel * kTile;
    if (tid < kTile) s_src[tid] = tid < t.rows && t.expert < a.N ? source(a, t.row0 + tid) : -1;
    __syncthreads();
    const bool real = t.expert < a.N;
    const int len = real ? a.K : 0;
    const int expert = real ? t.expert : 0;
    const int8_t* W = (const int8_t*)a.W + (int64_t)expert * a.K * a.C;
    u32x4 wa[2], wb[2];
    auto fetch = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = tid / 8 + 32 * i, c = k0 + (tid % 8) * 16;
            wa[i] = load16_bytes((const int8_t*)a.x + (int64_t)max(s_src[r], 0) * a.K, c, a.K);
            wb[i] = load16_bytes(W + (int64_t)min(c0 + r, a.C - 1) * a.K, c, a.K);
        }
    };
    const int half = lane >> 5, l32 = lane & 31;
    const int ao = 32 * (wave >> 1) + l32, bo = 32 * (wave & 1) + l32;
    i32x16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0;
    if (len) fetch(0);
    for (int k0 = 0; k0 < len; k0 += kStep8) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = (tid / 8 + 32 * i) * kPitch8 + (tid % 8) * 16;
            *(u32x4*)(A + at) = wa[i];
            *(u32x4*)(B + at) = wb[i];
        }
        __syncthreads();
        if (k0 + kStep8 < len) fetch(k0 + kStep8);
#pragma unroll
        for (int k = 0; k < kStep8; k += 32) {
            const i32x4 fa = *(const i32x4*)(A + ao * kPitch8 + k + 16 * half);
            const i32x4 fb = *(const i32x4*)(B + bo * kPitch8 + k + 16 * half);
            acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa, fb, acc, 0, 0, 0);
        }
    }
    const int c = c0 + bo;
    if (c >= a.C) return;
    const float sw = a.w_scale[(int64_t)expert * a.C + c];
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int r = 32 * (wave >> 1) + 8 * (v / 4) + 4 * half + v % 4;
        if (r >= t.rows) continue;
        const int src = s_src[r];
        const float y = src >= 0 ? (float)acc[v] * a.row_scale[src] * sw : 0.0f;
        ((O*)a.out)[(int64_t)(t.row0 + r) * a.C + c] = Act<O>::from_f32(y);
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
    const int64_t groups = tile_groups(d.R, d.N, kTile, ceil_div(std::max(d.n_out, d.n_in), kTile));
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

hipError_t launch_mm(const pr2_wgrad_desc& d, const MmArgs& a, hipStream_t st) {
    if (d.act_dtype == PR2_BF16) return launch_tiles("mm_tile", mm_tile_kernel<bf16_t, false>, a, kTile, kTile, 256, st);
    return launch_tiles("mm_tile", mm_tile_kernel<float, false>, a, kTile, kTile, 256, st);
}

hipError_t launch_mm_back(const pr2_wgrad_desc& d, const MmArgs& a, hipStream_t st) {
    if (d.act_dtype == PR2_BF16)
        return launch_tiles("mm_back_tile", mm_tile_kernel<bf16_t, true>, a, kTile, kTile, 256, st);
    return launch_tiles("mm_back_tile", mm_tile_kernel<float, true>, a, kTile, kTile, 256, st);
}

hipError_t launch_mm8(const pr2_wgrad_desc& d, const MmArgs& a, hipStream_t st) {
    if (d.act_dtype == PR2_BF16) return launch_tiles("mm8_tile", mm8_tile_kernel<bf16_t>, a, kTile, kTile, 256, st);
    return launch_tiles("mm8_tile", mm8_tile_kernel<float>, a, kTile, kTile, 256, st);
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
                                   : launch_mm(d, a, st);
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
    const hipError_t e = launch_mm_back(d, a, (hipStream_t)stream);
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
                                   : launch_mm8(d, a, st);
    if (e != hipSuccess) return hip_fail(e, "grouped_mm_quant launch");
    return ok();
}

}  // extern "C"
