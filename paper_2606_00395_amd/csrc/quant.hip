// Rows in 8 bits with one scale each, what the products with 8-bit weights read: of a tensor, or of
// silu(a) u.
//
//   m = the row's largest magnitude,  scale = max(m, 2^-100) (1 / 127),  q = rint(v / scale)
//
// Bound by HBM (silu(a) u of many bf16 rows: by its exponential and quotient): a row is read once and held in registers
// while its maximum is formed (rows above 32768 elements are read again).  16384 x 2048 bf16 in 24 us, as much as a copy of
// its bytes; silu(a) u of 131072 rows of 768 in 176, where a copy takes 98.
#include <algorithm>

#include "rowgroup.h"

namespace pr2 {
namespace {

constexpr int kCus = 256;
constexpr int kHeld = 32768;            // elements of a row that a workgroup's registers hold

struct QuantArgs {
    const void* x;          // [R, C], or a | u [R, 2 C]
    int8_t* q;
    float* scale;
    int64_t R;
    int C;
};

// The values of a piece: x, or silu(a) u to a few last places of fp32.  Of bf16 rows too: what follows is no rounding to
// bf16 but one to 8 bits, which an error takes to the other side of a half as often as it is large, and the row's
// step shows it as it is.  (The short exponential and reciprocal, off by 1e-6 (1 + |a|), take 256 rows of 1024 from bf16
// in 4.2 us for 4.3, 16384 in 17.4 for 24.6, where the arithmetic is the bound.)
template <typename T, bool SWIGLU, int E>
__device__ __forceinline__ void open_piece(const u32x4& x, const u32x4& second, float* v) {
    Chunk<T>::open(x, v);
    if (!SWIGLU) return;
    float u[E];
    Chunk<T>::open(second, u);
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = v[j] / (1.0f + expf(-v[j])) * u[j];
}

template <typename G>
__device__ __forceinline__ void store_row_piece(const G& g, int8_t* row, int i, const float* v, const RowStep& s) {
    if (!g.any(i)) return;
    uint32_t q[G::E / 4];
    quantise_row<G::E>(v, s, q);
    if (!g.on(i)) return;
    int8_t* to = row + g.start(i);
    if (!g.narrow()) {
        store_bytes<G::E>(to, q);
    } else {
#pragma unroll
        for (int j = 0; j < G::E; ++j)
            if (j < g.d) to[j] = (int8_t)(q[j / 4] >> (8 * (j % 4)));
    }
}

template <int E>
__device__ __forceinline__ uint32_t largest(const float* v) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < E; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
    return m;
}

// (a moved-back last piece holds some elements twice: neither the maximum nor what is written
// is different for it)
template <typename T, bool SWIGLU, int NW, int F>
__global__ void __launch_bounds__(NW == 16 ? 1024 : 256) quant_kernel(QuantArgs a) {
    using G = RowGroup<T, NW, F>;
    constexpr int E = G::E, P = G::kPieces;
    constexpr int kRows = NW == 1 ? 4 : 1;
    __shared__ uint32_t red[8 * NW];
    int turn = 0;
    const int sub = NW == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const G g(a.C, NW == 1 ? threadIdx.x & 63 : threadIdx.x);
    for (int64_t row = (int64_t)blockIdx.x * kRows + sub; row < a.R; row += (int64_t)gridDim.x * kRows) {
        const T* x = (const T*)a.x + row * (SWIGLU ? 2 : 1) * a.C;
        u32x4 raw[P], second[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            raw[i] = g.load(x, i);
            if (SWIGLU) second[i] = g.load(x + a.C, i);
        }
        float v[F];
        uint32_t m[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            m[i] = 0;
            if (!g.any(i)) continue;
            open_piece<T, SWIGLU, E>(raw[i], second[i], v + i * E);
            m[i] = largest<E>(v + i * E);
        }
        const RowStep s = row_step(row_max<NW, P, 1>(m, red, turn));
        if (g.lane == 0) a.scale[row] = s.step;
#pragma unroll
        for (int i = 0; i < P; ++i) store_row_piece(g, a.q + row * a.C, i, v + i * E, s);
    }
}

// rows of any width, read twice
template <typename T, bool SWIGLU>
__global__ void __launch_bounds__(1024) quant_wide_kernel(QuantArgs a) {
    using G = RowGroup<T, 16, Chunk<T>::E>;
    constexpr int E = G::E;
    __shared__ uint32_t red[8 * 16];
    int turn = 0;
    const G all(a.C, threadIdx.x);
    const int pieces = (a.C + E * G::kLanes - 1) / (E * G::kLanes);
    for (int64_t row = blockIdx.x; row < a.R; row += gridDim.x) {
        const T* x = (const T*)a.x + row * (SWIGLU ? 2 : 1) * a.C;
        uint32_t m[1] = {0};
        float v[E];
        for (int i = 0; i < pieces; ++i) {
            open_piece<T, SWIGLU, E>(all.load(x, i), SWIGLU ? all.load(x + a.C, i) : u32x4{0, 0, 0, 0}, v);
            m[0] = max(m[0], largest<E>(v));
        }
        const RowStep s = row_step(row_max<16, 1, 1>(m, red, turn));
        if (threadIdx.x == 0) a.scale[row] = s.step;
        for (int i = 0; i < pieces; ++i) {
            open_piece<T, SWIGLU, E>(all.load(x, i), SWIGLU ? all.load(x + a.C, i) : u32x4{0, 0, 0, 0}, v);
            store_row_piece(all, a.q + row * a.C, i, v, s);
        }
    }
}

// ------------------------------------------------------------------ host ----
template <typename T, bool SWIGLU, int NW, int F>
void quant_launch(const QuantArgs& a, hipStream_t st) {
    const int64_t groups = (a.R + (NW == 1 ? 3 : 0)) / (NW == 1 ? 4 : 1);
    const int64_t most = NW == 16 ? 2 * kCus : 8 * kCus;
    hipLaunchKernelGGL((quant_kernel<T, SWIGLU, NW, F>), dim3((unsigned)std::min(groups, most)),
                       dim3(NW == 16 ? 1024 : 256), 0, st, a);
}

template <typename T, bool SWIGLU>
hipError_t launch_quant(const QuantArgs& a, hipStream_t st) {
    LaunchScope scope(SWIGLU ? "swiglu_quant" : "act_quant", st);
    const bool few = a.R <= 8 * kCus;           // (more lanes a row, as for the norm)
    if (a.C <= 512) quant_launch<T, SWIGLU, 1, 8>(a, st);
    else if (a.C <= 2048 && few) quant_launch<T, SWIGLU, 4, 8>(a, st);
    else if (a.C <= 1024) quant_launch<T, SWIGLU, 1, 16>(a, st);
    else if (a.C <= 2048) quant_launch<T, SWIGLU, 1, 32>(a, st);
    else if (a.C <= 4096) quant_launch<T, SWIGLU, 4, 16>(a, st);
    else if (a.C <= 8192 && few) quant_launch<T, SWIGLU, 16, 8>(a, st);
    else if (a.C <= 8192) quant_launch<T, SWIGLU, 4, 32>(a, st);
    else if (a.C <= 16384) quant_launch<T, SWIGLU, 16, 16>(a, st);
    else if (a.C <= kHeld) quant_launch<T, SWIGLU, 16, 32>(a, st);
    else
        hipLaunchKernelGGL((quant_wide_kernel<T, SWIGLU>), dim3((unsigned)std::min<int64_t>(a.R, 2 * kCus)),
                           dim3(1024), 0, st, a);
    return hipGetLastError();
}

template <bool SWIGLU>
pr2_status quant(int64_t R, int32_t C, const char* width, int act_dtype, const void* x, int8_t* q, float* row_scale,
                 pr2_stream_t stream) {
    if (act_dtype != PR2_F32 && act_dtype != PR2_BF16)
        return fail(PR2_ERR_DTYPE, "act_dtype %d is not PR2_F32 or PR2_BF16", act_dtype);
    if (R < 0) return fail(PR2_ERR_SHAPE, "R = %lld < 0", (long long)R);
    if (C < 1) return fail(PR2_ERR_SHAPE, "%s = %d < 1", width, C);
    if (C > (1 << 28)) return fail(PR2_ERR_UNSUPPORTED, "%s = %d > 2^28", width, C);
    if (R > 0x7fffffff) return fail(PR2_ERR_UNSUPPORTED, "R = %lld rows exceed 2^31 - 1", (long long)R);
    if (R == 0) return ok();
    if (!x || !q || !row_scale) return fail(PR2_ERR_NULL, "a required tensor is NULL");
    if ((uintptr_t)x % 16 || (uintptr_t)q % 16)
        return fail(PR2_ERR_ALIGN, "the input or q is not 16-byte aligned");
    if ((uintptr_t)row_scale % 4) return fail(PR2_ERR_ALIGN, "row_scale is not 4-byte aligned");
    if (share_memory(q, (size_t)R * C, x, (size_t)R * C * (SWIGLU ? 2 : 1) * (act_dtype == PR2_BF16 ? 2 : 4)))
        return fail(PR2_ERR_SHAPE, "q overlaps the input");
    const pr2_status s = device_ready();
    if (s != PR2_OK) return s;
    const QuantArgs a{x, q, row_scale, R, C};
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = act_dtype == PR2_BF16 ? launch_quant<bf16_t, SWIGLU>(a, st)
                                               : launch_quant<float, SWIGLU>(a, st);
    if (e != hipSuccess) return hip_fail(e, SWIGLU ? "swiglu_quant launch" : "act_quant launch");
    return ok();
}

}  // namespace
}  // namespace pr2

using namespace pr2;

extern "C" {

pr2_status pr2_act_quant(int64_t R, int32_t C, int act_dtype, const void* x, int8_t* q, float* row_scale,
                         pr2_stream_t stream) {
    return quant<false>(R, C, "C", act_dtype, x, q, row_scale, stream);
}

pr2_status pr2_swiglu_quant(int64_t R, int32_t m, int act_dtype, const void* au, int8_t* q, float* row_scale,
                            pr2_stream_t stream) {
    return quant<true>(R, m, "m", act_dtype, au, q, row_scale, stream);
}

}  // extern "C"
