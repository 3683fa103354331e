// Weight gradients whose input operand is an 8-bit checkpoint:
//   dW[e] [n_out, n_in] = sum over expert e's rows r of dy[r]^T value(x)[src(r)],
// src(r) the token of row r's route, or r itself.
//
// A packed value is an int8 times a power of two, exact in bf16 and fp32, so nothing is
// rounded on the way into the products.
#include "chunk.h"

namespace pr2 {
namespace {

struct WgradArgs {
    const void* dy;             // [R, n_out]
    const int8_t* q;            // [Rx, n_in]
    const uint8_t* scale;       // [Rx, groups]
    const int* offsets;         // [N + 1] or null (one weight over all rows)
    const int* route;           // [R] or null
    float* dW;                  // [N, n_out, n_in]
    int64_t R, Rx;
    int n_out, n_in, N, k;
    int groups;
};

// rows of expert e, clamped to the R that there are
__device__ __forceinline__ void expert_rows(const WgradArgs& a, int e, int* first, int* last) {
    const int R = (int)a.R;
    *first = a.offsets ? min(max(a.offsets[e], 0), R) : 0;
    *last = a.offsets ? max(min(a.offsets[e + 1], R), *first) : R;
}

// packed row of dy's row r, -1 if it has none
__device__ __forceinline__ int source_row(const WgradArgs& a, int r) {
    if (!a.route) return r;
    const int q = a.route[r];
    const int t = q / a.k;
    return q >= 0 && t < a.Rx ? t : -1;
}

// Any type, width and row count: 64 x 64 outputs per workgroup, 4 x 4 per thread, 16 rows of
// both operands staged in LDS as fp32.  Bound by its vector FMAs and LDS reads.
constexpr int kTile = 64;
constexpr int kStep = 16;

template <typename T>
__global__ void __launch_bounds__(256) wgrad_tile_kernel(WgradArgs a) {
    __shared__ float A[kStep][kTile + 4], B[kStep][kTile + 4];
    const int tid = threadIdx.x;
    const int nct = (a.n_in + kTile - 1) / kTile;
    const int o0 = (int)(blockIdx.x / nct) * kTile, c0 = (int)(blockIdx.x % nct) * kTile;
    const int e = blockIdx.y;
    int first, last;
    expert_rows(a, e, &first, &last);
    const int sr = tid / 16, sc = (tid % 16) * 4;       // row and columns this thread stages
    const int tr = (tid / 16) * 4, tc = (tid % 16) * 4; // outputs it owns
    float acc[4][4] = {};
    for (int r0 = first; r0 < last; r0 += kStep) {
        const int r = r0 + sr;
        const bool in = r < last;
        const int x = in ? source_row(a, r) : -1;
        const T* dy = (const T*)a.dy + (int64_t)(in ? r : 0) * a.n_out;
        const int8_t* q = a.q + (int64_t)max(x, 0) * a.n_in;
        const uint8_t* s = a.scale + (int64_t)max(x, 0) * a.groups;
        float va[4], vb[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int o = o0 + sc + j, c = c0 + sc + j;
            // a row without a source is zeros in both operands: nothing of it multiplies
            va[j] = x >= 0 && o < a.n_out ? Act<T>::to_f32(dy[o]) : 0.0f;
            vb[j] = x >= 0 && c < a.n_in ? (float)q[c] * __uint_as_float((uint32_t)s[c / 32] << 23) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            A[sr][sc + j] = va[j];
            B[sr][sc + j] = vb[j];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
            const float4 p = *(const float4*)&A[i][tr], w = *(const float4*)&B[i][tc];
            const float pa[4] = {p.x, p.y, p.z, p.w}, wb[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[u][v] = fmaf(pa[u], wb[v], acc[u][v]);
        }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int o = o0 + tr + u, c = c0 + tc + v;
            if (o < a.n_out && c < a.n_in)
                a.dW[((int64_t)e * a.n_out + o) * a.n_in + c] = acc[u][v];
        }
}

// ------------------------------------------------------------------ host ----
pr2_status check_wgrad(const pr2_wgrad_desc* desc) {
    if (!desc) return fail(PR2_ERR_NULL, "desc is NULL");
    const pr2_wgrad_desc& d = *desc;
    if (d.act_dtype != PR2_F32 && d.act_dtype != PR2_BF16)
        return fail(PR2_ERR_DTYPE, "act_dtype %d is not PR2_F32 or PR2_BF16", d.act_dtype);
    if (d.R < 0 || d.Rx < 0)
        return fail(PR2_ERR_SHAPE, "R = %lld or Rx = %lld < 0", (long long)d.R, (long long)d.Rx);
    if (d.n_out < 1 || d.n_in < 1)
        return fail(PR2_ERR_SHAPE, "n_out = %d or n_in = %d < 1", d.n_out, d.n_in);
    if (d.N < 1) return fail(PR2_ERR_SHAPE, "N = %d < 1", d.N);
    if (d.k < 1) return fail(PR2_ERR_SHAPE, "k = %d < 1", d.k);
    if (d.N > kMaxExperts) return fail(PR2_ERR_UNSUPPORTED, "N = %d > %d", d.N, kMaxExperts);
    if (d.R > 0x7fffffff - 1024 || d.Rx > 0x7fffffff - 1024)
        return fail(PR2_ERR_UNSUPPORTED, "R = %lld or Rx = %lld rows exceed 2^31 - 1025",
                    (long long)d.R, (long long)d.Rx);
    if (d.n_out > (1 << 20) || d.n_in > (1 << 20))
        return fail(PR2_ERR_UNSUPPORTED, "n_out = %d or n_in = %d > 2^20", d.n_out, d.n_in);
    return PR2_OK;
}

}  // namespace
}  // namespace pr2

using namespace pr2;

extern "C" {

size_t pr2_weight_grad_workspace_bytes(const pr2_wgrad_desc* desc) {
    (void)desc;
    return 0;
}

pr2_status pr2_weight_grad_packed(const pr2_wgrad_desc* desc, const void* dy, const int8_t* q,
                                  const uint8_t* scale, const int32_t* offsets,
                                  const int32_t* route_of_row, float* dW, void* ws,
                                  size_t ws_bytes, pr2_stream_t stream) {
    pr2_status s = check_wgrad(desc);
    if (s != PR2_OK) return s;
    const pr2_wgrad_desc& d = *desc;
    if (!dW) return fail(PR2_ERR_NULL, "dW is NULL");
    if ((uintptr_t)dW % 16) return fail(PR2_ERR_ALIGN, "dW is not 16-byte aligned");
    if (d.R > 0) {
        if (!dy || !q || !scale) return fail(PR2_ERR_NULL, "dy, q and scale are required");
        if ((uintptr_t)dy % 16 || (uintptr_t)q % 16 || (uintptr_t)scale % 16)
            return fail(PR2_ERR_ALIGN, "dy, q and scale must be 16-byte aligned");
        if (!offsets && d.N != 1) return fail(PR2_ERR_NULL, "offsets is NULL with N = %d > 1", d.N);
        if (!route_of_row && d.R > d.Rx)
            return fail(PR2_ERR_SHAPE, "R = %lld > Rx = %lld without route_of_row", (long long)d.R,
                        (long long)d.Rx);
        if ((uintptr_t)offsets % 4 || (uintptr_t)route_of_row % 4)
            return fail(PR2_ERR_ALIGN, "offsets or route_of_row is not 4-byte aligned");
        const size_t need = pr2_weight_grad_workspace_bytes(desc);
        if (need && !ws) return fail(PR2_ERR_NULL, "ws is NULL (need %zu bytes)", need);
        if (ws_bytes < need)
            return fail(PR2_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, need);
    }
    s = device_ready();
    if (s != PR2_OK) return s;
    drop_split_records(ws, ws_bytes);
    const hipStream_t st = (hipStream_t)stream;
    WgradArgs a{dy, q, scale, d.R ? offsets : nullptr, route_of_row, dW, d.R, d.Rx, d.n_out, d.n_in,
                d.N, d.k, (d.n_in + 31) / 32};
    const unsigned tiles = (unsigned)((d.n_out + kTile - 1) / kTile) * ((d.n_in + kTile - 1) / kTile);
    {
        LaunchScope scope("wgrad_tile", st);
        if (d.act_dtype == PR2_BF16)
            hipLaunchKernelGGL(wgrad_tile_kernel<bf16_t>, dim3(tiles, d.N), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL(wgrad_tile_kernel<float>, dim3(tiles, d.N), dim3(256), 0, st, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "weight_grad_packed launch");
    return ok();
}

}  // extern "C"
