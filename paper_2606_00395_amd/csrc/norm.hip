// Root-mean-square norm of rows with the residual's addition, its output also in 8 bits, and the
// backward pass.
//
//   h = round(x + residual),  r = (mean h^2 + eps)^-1/2,  y = h r w
//   g = dy w,  dx = dh + r (g - h r^2 mean(g h)),  dw = sum over the rows of dy h r
//
// A row is read once, held in registers (a wavefront's up to 2048 elements, a workgroup's above)
// while its sum is formed, and written once.  dw is summed per workgroup over its rows in registers,
// then in LDS, and the workgroups' sums are joined in order by a second launch.  HBM is the bound where
// there are many rows of up to 16384 elements (gradients: bf16 of 8192, fp32 of 1024): 16384 x 2048 bf16 with
// residual and h in 53 us, their gradients in 55, fp32 99 and 118 (floors of a copy 52 and 105).  Longer rows pass the
// registers and spill: 2000 bf16 rows of 20000 in 79 us, their gradients in 257 (floor 62), and fp32 rows of 1025 to 2048 do so
// in the gradients.  What sixteen wavefronts on one row wait for adds to that (3600 of 9000, gradients 65 us for 51).
#include <algorithm>
#include <initializer_list>

#include "rowgroup.h"

namespace pr2 {
namespace {

constexpr int kMaxWidth = 32768;
constexpr int kCus = 256;
// Rows of at least this much are read past the caches, half the size of the last-level cache, which
// then holds what is written (16384 x 2048 fp32 with the residual: h and y 104 -> 99 us, y alone 77 -> 73; in
// smaller tensors what the caller wrote last may still lie there).
constexpr size_t kStreamBytes = 128 << 20;

struct NormArgs {
    const void* x;
    const void* residual;       // or null
    const float* w;
    void* h;                    // or null
    void* y;                    // or null
    float* rstd;                // or null
    int8_t* q;                  // or null
    uint8_t* scale;             // the packed form's; null: the row form
    float* row_scale;
    int64_t T;
    int d;
    float eps;
};

// the scale byte of the packed form for a group's largest magnitude (its bits)
__device__ __forceinline__ uint32_t pack_scale(uint32_t m) {
    const int e = (int)(m >> 23);
    return e == 255 ? 255u : (uint32_t)max(e - 6, 1);
}

// Rounded to fp32, and never to bf16 in the same step (which a compiler that may contract makes of the two): bf16
// results are rounded through fp32, as torch rounds a 64-bit value to bf16.
__device__ __forceinline__ float to_f32(double v) {
#pragma clang fp contract(off)
    return (float)v;
}
// The same number, to be widened where it is used: the compiler else widens h and w ahead and holds them in twice the
// registers (32 elements a lane with the next row's: 217 for 168).
__device__ __forceinline__ float own_copy(float v) {
    asm volatile("" : "+v"(v));
    return v;
}

// STREAM: the rows are read past the caches.  AHEAD: a wavefront's next row is loaded one ahead.
template <typename T, int NW, int F, bool STREAM, bool AHEAD>
__global__ void __launch_bounds__(NW == 16 ? 1024 : 256) norm_kernel(NormArgs a) {
    using G = RowGroup<T, NW, F>;
    constexpr int E = G::E, P = G::kPieces;
    constexpr int kRows = NW == 1 ? 4 : 1;          // rows of a workgroup at a time
    __shared__ double red[8 * NW * P];
    int turn = 0;
    const int sub = NW == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const G g(a.d, NW == 1 ? threadIdx.x & 63 : threadIdx.x);
    float w[F];
#pragma unroll
    for (int i = 0; i < P; ++i) g.load_f32(a.w, i, w + i * E);
    const double inv_d = 1.0 / (double)a.d;
    struct Row {
        u32x4 x[P], res[P];
    };
    auto load = [&](Row& r, int64_t row) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < P; ++i) r.x[i] = g.template load<STREAM>((const T*)a.x + row * a.d, i);
        if (!a.residual) return;
#pragma unroll
        for (int i = 0; i < P; ++i) r.res[i] = g.template load<STREAM>((const T*)a.residual + row * a.d, i);
    };
    const int64_t first = (int64_t)blockIdx.x * kRows + sub, stride = (int64_t)gridDim.x * kRows;
    Row cur, next;
    if (AHEAD && first < a.T) load(next, first);
    for (int64_t row = first; row < a.T; row += stride) {
        if (!AHEAD) {
            load(cur, row);
        } else {
            cur = next;
            if (row + stride < a.T) load(next, row + stride);
        }
        u32x4 (&raw)[P] = cur.x, (&add)[P] = cur.res;
        float h[F];
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                if (!g.any(i)) continue;
                float v[E];
                Chunk<T>::open(raw[i], h + i * E);
                Chunk<T>::open(add[i], v);
#pragma unroll
                for (int j = 0; j < E; ++j) h[i * E + j] += v[j];
                raw[i] = Chunk<T>::close(h + i * E);        // the norm is taken of what h_out holds
            }
        }
        // The squares (exact), their sum, the root and h r w in fp64, so that y is the definition's value with one fp32
        // rounding before its own: from an fp32 sum a fifth of the fp32 y are a last place off, and a y that is
        // rounded to the other side is a whole step of act_dtype off and may move a packed value by its step.
        // Squares and r w may lie anywhere, too.
        double square[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            Chunk<T>::open(raw[i], h + i * E);
            float v[E];
            double s = 0.0;
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = h[i * E + j];
            g.mask(i, v);
#pragma unroll
            for (int j = 0; j < E; ++j) s = __builtin_fma((double)v[j], (double)v[j], s);
            square[i] = s;
        }
        const double root = rsqrt(row_reduce<NW, P, P>(square, red, turn, AddF64()) * inv_d + (double)a.eps);
        const float r = (float)root;
        // (behind the reduction: every element has been read, h may lie where x or the residual does)
        if (a.h) {
#pragma unroll
            for (int i = 0; i < P; ++i) g.store((T*)a.h + row * a.d, i, raw[i]);
        }
        if (a.rstd && g.lane == 0) a.rstd[row] = r;
        if (a.q && !a.scale) {
            // the row form: of h w, the row's r goes into its scale
            uint32_t part[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                part[i] = 0;
#pragma unroll
                for (int j = 0; j < E; ++j)
                    part[i] = max(part[i], __float_as_uint(h[i * E + j] * w[i * E + j]) & 0x7fffffffu);
            }
            const RowStep s = row_step(row_max<NW, P, 2 * P>(part, (uint32_t*)red, turn));
            if (g.lane == 0) a.row_scale[row] = r * s.step;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                if (!g.on(i)) continue;
                float v[E];
                uint32_t q[E / 4];
#pragma unroll
                for (int j = 0; j < E; ++j) v[j] = h[i * E + j] * w[i * E + j];
                quantise_row<E>(v, s, q);
                int8_t* to = a.q + row * a.d + g.start(i);
                if (!g.narrow()) {
                    store_bytes<E>(to, q);
                } else {
#pragma unroll
                    for (int j = 0; j < E; ++j)
                        if (j < a.d) to[j] = (int8_t)(q[j / 4] >> (8 * (j % 4)));
                }
            }
        }
        if (!a.y && !a.scale) continue;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (!g.any(i)) continue;
            float v[E];
#pragma unroll
            for (int j = 0; j < E; ++j) {
                v[j] = to_f32((double)own_copy(h[i * E + j]) * root * (double)own_copy(w[i * E + j]));
            }
            const u32x4 out = Chunk<T>::close(v);
            if (a.y) g.store((T*)a.y + row * a.d, i, out);
            if (!a.scale) continue;
            // the packed form of the rounded y; a group of 32 columns is 32 / E lanes' pieces
            Chunk<T>::open(out, v);
            g.mask(i, v);
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
            m = max(m, from_lane<XOR1>(m));
            m = max(m, from_lane<XOR2>(m));
            if (E == 4) m = max(m, from_lane<MIRROR8>(m));
            if (!g.on(i)) continue;
            const uint32_t byte = pack_scale(m);
            const float inverse = byte == 255u ? 0.0f : __uint_as_float((254u - byte) << 23);
            const int skip = g.skip(i);
            uint32_t q[E / 4];
            quantise_group<E>(v, inverse, q);
            if (byte == 255u) {
#pragma unroll
                for (int j = 0; j < E / 4; ++j) q[j] = 0;
            }
            int8_t* to = a.q + row * a.d + g.start(i);
            if (skip == 0 && !g.narrow()) {
                store_bytes<E>(to, q);
            } else {
                // (the skipped elements may belong to the group before)
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (j >= skip && g.start(i) + j < a.d) to[j] = (int8_t)(q[j / 4] >> (8 * (j % 4)));
            }
            if (g.column(i) % 32 == 0)
                a.scale[row * (int64_t)((a.d + 31) / 32) + g.column(i) / 32] = (uint8_t)byte;
        }
    }
}

struct NormBackArgs {
    const void* dy;
    const void* dh;             // or null
    const void* h;
    const float* rstd;
    const float* w;
    void* dx;
    float* part;                // [gridDim.x, d] sums of dw, or null
    int64_t T;
    int d;
};

// Wavefronts of a workgroup: eight rows at a time, or one row.
template <int NW> constexpr int back_threads() { return NW == 1 ? 512 : 64 * NW; }

template <typename T, int NW, int F>
__global__ void __launch_bounds__(back_threads<NW>()) norm_backward_kernel(NormBackArgs a) {
    using G = RowGroup<T, NW, F>;
    constexpr int E = G::E, P = G::kPieces;
    constexpr int kRows = NW == 1 ? 8 : 1;
    __shared__ uint32_t red[8 * NW * P];
    __shared__ float sums[NW == 1 ? 64 * F * kRows : 1];
    int turn = 0;
    const int sub = NW == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const G g(a.d, NW == 1 ? threadIdx.x & 63 : threadIdx.x);
    float w[F], dw[F];
#pragma unroll
    for (int i = 0; i < P; ++i) g.load_f32(a.w, i, w + i * E);
#pragma unroll
    for (int f = 0; f < F; ++f) dw[f] = 0.0f;
    const float inv_d = 1.0f / (float)a.d;
    const int64_t first = (int64_t)blockIdx.x * kRows + sub, stride = (int64_t)gridDim.x * kRows;
    struct Row {
        u32x4 h[P], y[P], e[P];
        float r;
    };
    auto load = [&](Row& w, int64_t row) __attribute__((always_inline)) {
        const int64_t at = row * a.d;
#pragma unroll
        for (int i = 0; i < P; ++i) w.h[i] = g.load((const T*)a.h + at, i);
#pragma unroll
        for (int i = 0; i < P; ++i) w.y[i] = g.load((const T*)a.dy + at, i);
        if (a.dh) {
#pragma unroll
            for (int i = 0; i < P; ++i) w.e[i] = g.load((const T*)a.dh + at, i);
        }
        w.r = a.rstd[row];
    };
    // (The next row's loads ahead hold twice the registers: on sixteen wavefronts they spill, 3600 rows of 9000 in 96 us
    // for 65, 2000 fp32 rows of 12000 in 161 for 90, and on four it was slower, too.)
    Row cur;
    for (int64_t row = first; row < a.T; row += stride) {
        load(cur, row);
        const float r = cur.r;
        uint32_t part[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            part[i] = 0;
            if (!g.any(i)) continue;
            float h[E], y[E], v[E], s = 0.0f;
            Chunk<T>::open(cur.h[i], h);
            Chunk<T>::open(cur.y[i], y);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float n = h[j] * r;
                dw[i * E + j] += y[j] * n;
                v[j] = y[j] * w[i * E + j] * n;
            }
            g.mask(i, v);
#pragma unroll
            for (int j = 0; j < E; ++j) s += v[j];
            part[i] = __float_as_uint(s);
        }
        const float mean = __uint_as_float(row_reduce<NW, P, P>(part, red, turn, AddF32())) * inv_d;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (!g.any(i)) continue;
            float h[E], y[E], e[E];
            Chunk<T>::open(cur.h[i], h);
            Chunk<T>::open(cur.y[i], y);
            if (a.dh) Chunk<T>::open(cur.e[i], e);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float v = r * (y[j] * w[i * E + j] - h[j] * r * mean);
                y[j] = a.dh ? v + e[j] : v;
            }
            // (dx may lie on dh, of which another wavefront may not yet hold what a moved-back piece shares
            // with it: h and dy have been summed before the barrier)
            if (NW > 1) g.store_own((T*)a.dx + row * a.d, i, Chunk<T>::close(y));
            else g.store((T*)a.dx + row * a.d, i, Chunk<T>::close(y));
        }
    }
    if (!a.part) return;
    float* out = a.part + (int64_t)blockIdx.x * a.d;
    if (NW > 1) {
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (g.on(i) && j >= g.skip(i) && g.start(i) + j < a.d) out[g.start(i) + j] = dw[i * E + j];
        return;
    }
    // the wavefronts' sums, in order: element f of lane l is word 64 f + l of its wavefront's
#pragma unroll
    for (int f = 0; f < F; ++f) sums[(sub * F + f) * 64 + g.lane] = dw[f];
    __syncthreads();
    for (int f = sub; f < F; f += kRows) {
        float v = sums[f * 64 + g.lane];
#pragma unroll
        for (int q = 1; q < kRows; ++q) v += sums[(q * F + f) * 64 + g.lane];
        const int i = f / E, c = g.start(i) + f % E;
        if (g.on(i) && f % E >= g.skip(i) && c < a.d) out[c] = v;
    }
}

// dw = the n workgroups' sums: 64 columns per workgroup, 16 wavefronts of consecutive parts each,
// joined in order
__global__ void __launch_bounds__(1024) norm_join_kernel(const float* part, int n, int d, float* dw) {
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    const int each = (n + 15) / 16;
    float v = 0.0f;
    if (c < d) {
        const int last = min(n, (wave + 1) * each);
#pragma unroll 8
        for (int p = wave * each; p < last; ++p) v += part[(int64_t)p * d + c];
    }
    s[wave][lane] = v;
    __syncthreads();
    if (wave != 0 || c >= d) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) v += s[w][lane];
    dw[c] = v;
}

__global__ void __launch_bounds__(256) norm_zero_kernel(float* p, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i] = 0.0f;
}

// ------------------------------------------------------------------ host ----
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups of the backward: each CU two of eight wavefronts (or of four, or one of sixteen), so
// that the sums of dw to be joined stay few.
int back_groups(int64_t T, int d) {
    const int64_t rows = d <= 2048 ? 8 : 1;
    const int64_t most = d <= 2048 ? kCus : d <= 8192 ? 2 * kCus : kCus;
    return (int)std::min<int64_t>(ceil_div(T, rows), most);
}

size_t norm_ws_bytes(int64_t T, int32_t d) {
    return sizeof(float) * (size_t)back_groups(T, d) * d + 16;
}

pr2_status check_norm(int64_t T, int32_t d, int act_dtype) {
    if (act_dtype != PR2_F32 && act_dtype != PR2_BF16)
        return fail(PR2_ERR_DTYPE, "act_dtype %d is not PR2_F32 or PR2_BF16", act_dtype);
    if (T < 0) return fail(PR2_ERR_SHAPE, "T = %lld < 0", (long long)T);
    if (d < 1) return fail(PR2_ERR_SHAPE, "d = %d < 1", d);
    if (d > kMaxWidth) return fail(PR2_ERR_UNSUPPORTED, "d = %d > %d", d, kMaxWidth);
    if (T > 0x7fffffff) return fail(PR2_ERR_UNSUPPORTED, "T = %lld rows exceed 2^31 - 1", (long long)T);
    return PR2_OK;
}

bool aligned(const void* p, uintptr_t n) { return (uintptr_t)p % n == 0; }

template <typename T, int NW, int F, bool STREAM, bool AHEAD = false>
void norm_launch(const NormArgs& a, hipStream_t st) {
    const int64_t groups = ceil_div(a.T, NW == 1 ? 4 : 1);
    const int64_t most = NW == 16 || AHEAD ? 2 * kCus : 8 * kCus;
    hipLaunchKernelGGL((norm_kernel<T, NW, F, STREAM, AHEAD>), dim3((unsigned)std::min(groups, most)),
                       dim3(NW == 16 ? 1024 : 256), 0, st, a);
}

template <typename T>
hipError_t launch_norm(const NormArgs& a, hipStream_t st) {
    LaunchScope scope("rms_norm", st);
    // A wavefront works through a lane's elements one after the other (four clocks an instruction): few
    // rows go to more lanes each (8 rows of 2048 bf16 in the row form 7.0 -> 4.9 us, 1024 rows 8.2 -> 6.3).
    const bool few = a.T <= 8 * kCus;
    const bool stream = (size_t)a.T * a.d * sizeof(T) >= kStreamBytes;
    // Several rows of 32 elements a lane for each wavefront: with a quarter of the wavefronts and the next row's
    // loads ahead 16384 x 2048 bf16 with the residual 55.5 -> 53.4 us, 8192 x 2048 packed 40.0 -> 37.7 (2500 x 2048 12.6
    // -> 13.0, 65536 x 2048 past the caches 232 -> 240; rows of 16 elements a lane gain nothing).
    const bool ahead = a.T >= 16 * kCus;
    if (stream) {
        if (a.d <= 512) norm_launch<T, 1, 8, true>(a, st);
        else if (a.d <= 1024) norm_launch<T, 1, 16, true>(a, st);
        else if (a.d <= 2048) norm_launch<T, 1, 32, true>(a, st);
        else if (a.d <= 4096) norm_launch<T, 4, 16, true>(a, st);
        else if (a.d <= 8192) norm_launch<T, 4, 32, true>(a, st);
        else if (a.d <= 16384) norm_launch<T, 16, 16, true>(a, st);
        else norm_launch<T, 16, 32, true>(a, st);
    } else if (few) {
        if (a.d <= 512) norm_launch<T, 1, 8, false>(a, st);
        else if (a.d <= 2048) norm_launch<T, 4, 8, false>(a, st);
        else if (a.d <= 8192) norm_launch<T, 16, 8, false>(a, st);
        else if (a.d <= 16384) norm_launch<T, 16, 16, false>(a, st);
        else norm_launch<T, 16, 32, false>(a, st);
    } else {
        if (a.d <= 512) norm_launch<T, 1, 8, false>(a, st);
        else if (a.d <= 1024) norm_launch<T, 1, 16, false>(a, st);
        else if (a.d <= 2048 && ahead) norm_launch<T, 1, 32, false, true>(a, st);
        else if (a.d <= 2048) norm_launch<T, 1, 32, false>(a, st);
        else if (a.d <= 4096) norm_launch<T, 4, 16, false>(a, st);
        else if (a.d <= 8192) norm_launch<T, 4, 32, false>(a, st);
        else if (a.d <= 16384) norm_launch<T, 16, 16, false>(a, st);
        else norm_launch<T, 16, 32, false>(a, st);
    }
    return hipGetLastError();
}

template <typename T, int NW, int F>
void back_launch(const NormBackArgs& a, int groups, hipStream_t st) {
    hipLaunchKernelGGL((norm_backward_kernel<T, NW, F>), dim3(groups), dim3(back_threads<NW>()), 0, st, a);
}

template <typename T>
hipError_t launch_norm_backward(const NormBackArgs& a, float* dw, hipStream_t st) {
    const int groups = back_groups(a.T, a.d);
    {
        LaunchScope scope("rms_norm_backward", st);
        if (a.d <= 512) back_launch<T, 1, 8>(a, groups, st);
        else if (a.d <= 1024) back_launch<T, 1, 16>(a, groups, st);
        else if (a.d <= 2048) back_launch<T, 1, 32>(a, groups, st);
        else if (a.d <= 4096) back_launch<T, 4, 16>(a, groups, st);
        else if (a.d <= 8192) back_launch<T, 4, 32>(a, groups, st);
        else if (a.d <= 16384) back_launch<T, 16, 16>(a, groups, st);
        else back_launch<T, 16, 32>(a, groups, st);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !dw) return e;
    LaunchScope scope("rms_norm_join", st);
    hipLaunchKernelGGL(norm_join_kernel, dim3((a.d + 63) / 64), dim3(1024), 0, st, a.part, groups, a.d, dw);
    return hipGetLastError();
}

}  // namespace
}  // namespace pr2

using namespace pr2;

extern "C" {

pr2_status pr2_rms_norm(int64_t T, int32_t d, int act_dtype, float eps, const void* x, const void* residual,
                        const float* weight, void* h_out, void* y, float* rstd_out, int8_t* q, uint8_t* scale,
                        float* row_scale, pr2_stream_t stream) {
    pr2_status s = check_norm(T, d, act_dtype);
    if (s != PR2_OK) return s;
    if (!(eps >= 0.0f) || eps > 3e38f) return fail(PR2_ERR_SHAPE, "eps = %g is not finite and >= 0", eps);
    if (T == 0) return ok();
    if (!x || !weight) return fail(PR2_ERR_NULL, "x and weight are required");
    if (!y && !q && !h_out && !rstd_out) return fail(PR2_ERR_NULL, "no output is given");
    if (!q != !(scale || row_scale)) return fail(PR2_ERR_NULL, "q goes with scale or row_scale");
    if (scale && row_scale) return fail(PR2_ERR_SHAPE, "scale and row_scale are both given");
    if (!aligned(x, 16) || !aligned(residual, 16) || !aligned(h_out, 16) || !aligned(y, 16) ||
        !aligned(q, 16) || !aligned(scale, 16))
        return fail(PR2_ERR_ALIGN, "x, residual, h_out, y, q or scale is not 16-byte aligned");
    if (!aligned(weight, 4) || !aligned(rstd_out, 4) || !aligned(row_scale, 4))
        return fail(PR2_ERR_ALIGN, "weight, rstd_out or row_scale is not 4-byte aligned");
    const size_t n = (size_t)T * d, bytes = n * (act_dtype == PR2_BF16 ? 2 : 4);
    const size_t groups = (size_t)T * ((d + 31) / 32);
    for (const void* in : {x, residual}) {
        if (share_memory(h_out, bytes, in, bytes, true) || share_memory(y, bytes, in, bytes, true))
            return fail(PR2_ERR_SHAPE, "h_out or y overlaps x or residual without being it");
        if (share_memory(q, n, in, bytes) || share_memory(scale, groups, in, bytes))
            return fail(PR2_ERR_SHAPE, "q or scale overlaps x or residual");
    }
    if (share_memory(y, bytes, h_out, bytes)) return fail(PR2_ERR_SHAPE, "y overlaps h_out");
    if ((s = device_ready()) != PR2_OK) return s;
    const NormArgs a{x, residual, weight, h_out, y, rstd_out, q, scale, row_scale, T, d, eps};
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = act_dtype == PR2_BF16 ? launch_norm<bf16_t>(a, st) : launch_norm<float>(a, st);
    if (e != hipSuccess) return hip_fail(e, "rms_norm launch");
    return ok();
}

size_t pr2_rms_norm_workspace_bytes(int64_t T, int32_t d) {
    if (T < 0 || T > 0x7fffffff || d < 1 || d > kMaxWidth) return 0;
    return norm_ws_bytes(T, d);
}

pr2_status pr2_rms_norm_backward(int64_t T, int32_t d, int act_dtype, const void* dy, const void* dh,
                                 const void* h, const float* rstd, const float* weight, void* dx, float* dweight,
                                 void* ws, size_t ws_bytes, pr2_stream_t stream) {
    pr2_status s = check_norm(T, d, act_dtype);
    if (s != PR2_OK) return s;
    if (!aligned(dweight, 4)) return fail(PR2_ERR_ALIGN, "dweight is not 4-byte aligned");
    const hipStream_t st = (hipStream_t)stream;
    if (T == 0) {
        if (!dweight) return ok();
        if ((s = device_ready()) != PR2_OK) return s;
        LaunchScope scope("rms_norm_zero", st);
        hipLaunchKernelGGL(norm_zero_kernel, dim3((d + 255) / 256), dim3(256), 0, st, dweight, d);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "rms_norm_backward zero fill");
        return ok();
    }
    if (!dy || !h || !rstd || !weight || !dx) return fail(PR2_ERR_NULL, "dy, h, rstd, weight and dx are required");
    if (!aligned(dy, 16) || !aligned(dh, 16) || !aligned(h, 16) || !aligned(dx, 16))
        return fail(PR2_ERR_ALIGN, "dy, dh, h or dx is not 16-byte aligned");
    if (!aligned(rstd, 4) || !aligned(weight, 4)) return fail(PR2_ERR_ALIGN, "rstd or weight is not 4-byte aligned");
    const size_t bytes = (size_t)T * d * (act_dtype == PR2_BF16 ? 2 : 4);
    for (const void* in : {dy, dh, h})
        if (share_memory(dx, bytes, in, bytes, true))
            return fail(PR2_ERR_SHAPE, "dx overlaps dy, dh or h without being it");
    if (dweight) {
        const size_t need = norm_ws_bytes(T, d);
        if (!ws) return fail(PR2_ERR_NULL, "ws is NULL (need %zu bytes)", need);
        if (ws_bytes < need) return fail(PR2_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, need);
    }
    if ((s = device_ready()) != PR2_OK) return s;
    float* part = nullptr;
    if (dweight) {
        drop_split_records(ws, ws_bytes);
        part = (float*)(((uintptr_t)ws + 15) & ~(uintptr_t)15);
    }
    const NormBackArgs a{dy, dh, h, rstd, weight, dx, part, T, d};
    const hipError_t e = act_dtype == PR2_BF16 ? launch_norm_backward<bf16_t>(a, dweight, st)
                                               : launch_norm_backward<float>(a, dweight, st);
    if (e != hipSuccess) return hip_fail(e, "rms_norm_backward launch");
    return ok();
}

}  // extern "C"
