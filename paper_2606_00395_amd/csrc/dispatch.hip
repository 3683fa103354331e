// Tokens sorted by expert and back, for experts of the caller's own, with both gradients.
//
//   dispatch           xs[row(t, s)] = x[t]
//   dispatch backward  dx[t] = sum_s dxs[row(t, s)]
//   combine            y[t] = sum_s g_ts o[row(t, s)]
//   combine backward   do[row(t, s)] = g_ts dy[t],  dg_ts = <dy[t], o[row(t, s)]>
//
// Every one is bound by HBM and goes token by token: the token's row is read (or written)
// once and its k sorted rows, each contiguous, are written or read as whole segments; no
// row is read for a route that was dropped.  The sums over the slots run in slot order in
// fp32, so no atomics and the same bits every time.  16384 tokens of 2048 bf16, k 8: dispatch
// 111 us (5.5 TB/s), combine 111 (5.4), combine backward 218 (5.3), dispatch backward 105 (5.8);
// a large copy reaches 5.2.  A token's row indexes are read together, before its pieces go out
// (dispatch and combine with their plan 244.6 -> 240.5 us).
#include <algorithm>

#include "chunk.h"

namespace pr2 {
namespace {

constexpr int kThreads = 256;
constexpr int kSlots = 8;           // route slots whose rows are in flight together
// Sorted rows of more than this are written past the caches, half the size of the last-level
// cache: their reader would not find them there, and they push out what it would find.  537 MB
// of rows: dispatch and combine 274 -> 246 us (with the reads), combine backward and
// dispatch backward 351 -> 328.
constexpr int64_t kStreamBytes = 128 << 20;

struct RowArgs {
    const void* tok;        // [T, d] x or dy
    const void* rows;       // [T k, d] sorted rows read
    const int* offsets;     // [N + 1]
    const int* row;         // [T, k]
    const float* gate;      // [T, k]
    void* tok_out;          // [T, d]
    void* rows_out;         // [T k, d]
    float* dgate;           // [T, k]
    int64_t T;
    int64_t Tk;
    int d, k, N;
};

// sorted rows from `filled` on belong to no route: zeros; workgroup b of `wgs` takes every wgs-th
template <typename T, bool NT>
__device__ __forceinline__ void zero_rest(const RowArgs& a, int filled, int lanes, int lane, int64_t b,
                                          int64_t wgs) {
    const int full = a.d / Chunk<T>::E, rem = a.d % Chunk<T>::E;
    const int n = full + (rem != 0);
    const float v[Chunk<T>::E] = {};
    for (int64_t r = max(filled, 0) + b; r < a.Tk; r += wgs)
        for (int c = lane; c < n; c += lanes)
            store_chunk<T, NT>((T*)a.rows_out + r * a.d, c, full, rem, v);
}

// First element of piece c of a row of d >= E elements.  A last piece that would end outside the
// row is moved back over its neighbour, so that all are read and written whole (element by
// element in one lane it took up to as long as the rest: 1349 tokens of 1639, k 8, the backward
// 68.6 -> 35.3 us; 3979 of 2263, k 7, both directions 259 -> 187).
template <typename T>
__device__ __forceinline__ int piece_start(int c, int d) {
    return min(c * Chunk<T>::E, d - Chunk<T>::E);
}

// blockDim = (lanes per token, tokens per workgroup); lanes is a multiple of 64.  With few tokens a
// token's pieces past the first lanes go to workgroups of their own (gridDim.y), in gather_sum
// too.
template <typename T, bool NT>
__global__ void __launch_bounds__(kThreads) dispatch_kernel(RowArgs a) {
    const int full = a.d / Chunk<T>::E, rem = a.d % Chunk<T>::E;
    const int n = full + (rem != 0);
    const bool narrow = a.d < Chunk<T>::E;
    const int y = __builtin_amdgcn_readfirstlane(threadIdx.y);
    const int64_t b = (int64_t)blockIdx.x * blockDim.y + y;
    const int64_t wgs = (int64_t)gridDim.x * blockDim.y;
    const int filled = a.offsets[a.N];
    for (int64_t t = b; t < a.T; t += wgs) {
        const T* x = (const T*)a.tok + t * a.d;
        for (int c = blockIdx.y * blockDim.x + threadIdx.x; c < n; c += gridDim.y * blockDim.x) {
            const int at = piece_start<T>(c, a.d);
            const u32x4 w = narrow ? load_chunk<T, true>(x, c, full, rem) : load16<true>(x + at);
            for (int s0 = 0; s0 < a.k; s0 += kSlots) {
                int r[kSlots];
#pragma unroll
                for (int j = 0; j < kSlots; ++j) r[j] = s0 + j < a.k ? a.row[t * a.k + s0 + j] : -1;
#pragma unroll
                for (int j = 0; j < kSlots; ++j) {
                    if ((uint32_t)r[j] >= (uint64_t)a.Tk) continue;
                    T* row = (T*)a.rows_out + (int64_t)r[j] * a.d;
                    if (narrow) copy_chunk<T, NT>(row, c, full, rem, w);
                    else store16<NT>(row + at, w);
                }
            }
        }
    }
    if (blockIdx.y == 0) zero_rest<T, NT>(a, filled, blockDim.x, threadIdx.x, b, wgs);
}

// y[t] = sum_s [gate] row: combine (GATED) and the gradient of dispatch.  (Two tokens at a
// time, twice the loads in flight: no faster.)
template <typename T, bool GATED>
__global__ void __launch_bounds__(kThreads) gather_sum_kernel(RowArgs a) {
    constexpr int E = Chunk<T>::E;
    const int full = a.d / E, rem = a.d % E;
    const int n = full + (rem != 0);
    const bool narrow = a.d < E;
    const int y = __builtin_amdgcn_readfirstlane(threadIdx.y);
    const int64_t wgs = (int64_t)gridDim.x * blockDim.y;
    for (int64_t t = (int64_t)blockIdx.x * blockDim.y + y; t < a.T; t += wgs) {
        for (int c = blockIdx.y * blockDim.x + threadIdx.x; c < n; c += gridDim.y * blockDim.x) {
            const int at = piece_start<T>(c, a.d);
            float acc[E] = {};
            for (int s0 = 0; s0 < a.k; s0 += kSlots) {
                u32x4 w[kSlots];
                int r[kSlots];
#pragma unroll
                for (int j = 0; j < kSlots; ++j) {
                    r[j] = s0 + j < a.k ? a.row[t * a.k + s0 + j] : -1;
                    if ((uint32_t)r[j] >= (uint64_t)a.Tk) r[j] = -1;
                }
#pragma unroll
                for (int j = 0; j < kSlots; ++j) {
                    if (r[j] < 0) continue;
                    const T* row = (const T*)a.rows + (int64_t)r[j] * a.d;
                    w[j] = narrow ? load_chunk<T, true>(row, c, full, rem) : load16<true>(row + at);
                }
#pragma unroll
                for (int j = 0; j < kSlots; ++j) {
                    if (r[j] < 0) continue;
                    float v[E];
                    Chunk<T>::open(w[j], v);
                    const float g = GATED ? a.gate[t * a.k + s0 + j] : 1.0f;
#pragma unroll
                    for (int i = 0; i < E; ++i) acc[i] = GATED ? fmaf(g, v[i], acc[i]) : acc[i] + v[i];
                }
            }
            T* to = (T*)a.tok_out + t * a.d;
            if (narrow) store_chunk(to, c, full, rem, acc);
            else store16<false>(to + at, Chunk<T>::close(acc));
        }
    }
}

// Sums of eight values over a wavefront, each halving of the lanes halving the values a lane
// carries: slot (4 b5 + 2 b4 + b3) of the lane's bits ends in that lane.
__device__ __forceinline__ float sum_slots(const float (&v)[kSlots], int lane) {
    static_assert(kSlots == 8, "three halvings");
    float a[4], b[2];
    const bool h5 = lane & 32, h4 = lane & 16, h3 = lane & 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float other = __shfl_xor(h5 ? v[i] : v[i + 4], 32, 64);
        a[i] = (h5 ? v[i + 4] : v[i]) + other;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float other = __shfl_xor(h4 ? a[i] : a[i + 2], 16, 64);
        b[i] = (h4 ? a[i + 2] : a[i]) + other;
    }
    float r = (h3 ? b[1] : b[0]) + __shfl_xor(h3 ? b[0] : b[1], 8, 64);
#pragma unroll
    for (int off = 4; off >= 1; off >>= 1) r += __shfl_xor(r, off, 64);
    return r;
}

// d_o may be o: a thread reads its piece of a row before it writes it.  With few tokens a
// token's groups of slots go to workgroups of their own (gridDim.y).
template <typename T, bool NT>
__global__ void __launch_bounds__(kThreads) combine_backward_kernel(RowArgs a) {
    constexpr int E = Chunk<T>::E;
    __shared__ float part[kThreads / 64][kSlots];
    const int full = a.d / E, rem = a.d % E;
    const int n = full + (rem != 0);
    const bool narrow = a.d < E;
    const int y = __builtin_amdgcn_readfirstlane(threadIdx.y);
    const int lane = threadIdx.x & 63;
    const int waves = blockDim.x / 64;                  // wavefronts of one token
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) + y * waves;
    const int64_t b = (int64_t)blockIdx.x * blockDim.y + y;
    const int64_t wgs = (int64_t)gridDim.x * blockDim.y;
    const int filled = a.offsets[a.N];
    const int64_t turns = (a.T + wgs - 1) / wgs;        // the same for all: barriers inside
    for (int64_t turn = 0; turn < turns; ++turn) {
        const int64_t t = turn * wgs + b;
        const bool in = t < a.T;
        for (int s0 = blockIdx.y * kSlots; s0 < a.k; s0 += gridDim.y * kSlots) {
            int r[kSlots];
            float g[kSlots];
            float dot[kSlots] = {};
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                const bool has = in && s0 + j < a.k;
                r[j] = has ? a.row[t * a.k + s0 + j] : -1;
                if ((uint32_t)r[j] >= (uint64_t)a.Tk) r[j] = -1;
                g[j] = has ? a.gate[t * a.k + s0 + j] : 0.0f;
            }
            if (in) {
                for (int c = threadIdx.x; c < n; c += blockDim.x) {
                    u32x4 w[kSlots];
                    // (a last piece that was moved back: its first elements are another lane's,
                    // read but not used, and not written, since d_o may be o)
                    const int at = piece_start<T>(c, a.d);
                    const int skip = narrow ? 0 : c * E - at;
                    const T* tok = (const T*)a.tok + t * a.d;
                    const u32x4 dw = narrow ? load_chunk<T, true>(tok, c, full, rem) : load16<true>(tok + at);
#pragma unroll
                    for (int j = 0; j < kSlots; ++j) {
                        if (r[j] < 0) continue;
                        const T* row = (const T*)a.rows + (int64_t)r[j] * a.d;
                        w[j] = narrow ? load_chunk<T, true>(row, c, full, rem) : load16<true>(row + at);
                    }
                    float dy[E];
                    Chunk<T>::open(dw, dy);
#pragma unroll
                    for (int j = 0; j < kSlots; ++j) {
                        if (r[j] < 0) continue;
                        float v[E];
                        Chunk<T>::open(w[j], v);
#pragma unroll
                        for (int i = 0; i < E; ++i) {
                            if (i >= skip) dot[j] = fmaf(dy[i], v[i], dot[j]);
                            v[i] = g[j] * dy[i];
                        }
                        T* row = (T*)a.rows_out + (int64_t)r[j] * a.d;
                        if (skip == 0) {
                            store_chunk<T, NT>(row, c, full, rem, v);
                        } else {
#pragma unroll
                            for (int i = 1; i < E; ++i)
                                if (i >= skip) row[at + i] = Act<T>::from_f32(v[i]);
                        }
                    }
                }
            }
            const float sum = sum_slots(dot, lane);
            if (waves > 1) {
                __syncthreads();
                if ((lane & 7) == 0) part[wave][lane >> 3] = sum;
                __syncthreads();
                if (in && threadIdx.x < kSlots && s0 + (int)threadIdx.x < a.k) {
                    float v = 0.0f;
                    for (int w = 0; w < waves; ++w) v += part[y * waves + w][threadIdx.x];
                    a.dgate[t * a.k + s0 + threadIdx.x] = v;
                }
            } else if (in && (lane & 7) == 0 && s0 + (lane >> 3) < a.k) {
                a.dgate[t * a.k + s0 + (lane >> 3)] = sum;
            }
        }
    }
    if (blockIdx.y == 0) zero_rest<T, NT>(a, filled, blockDim.x, threadIdx.x, b, wgs);
}

// ------------------------------------------------------------------ host ----
bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

// lanes per token: a wavefront for each 64 pieces of a row, at most four
dim3 row_block(const RowArgs& a, int elem) {
    const int64_t n = ((int64_t)a.d * elem + 15) / 16;
    const unsigned lanes = n <= 64 ? 64 : n <= 128 ? 128 : 256;
    return dim3(lanes, kThreads / lanes);
}

dim3 row_grid(const RowArgs& a, dim3 block) {
    const int64_t want = (a.T + block.y - 1) / block.y;
    return dim3((unsigned)(want < 16384 ? want : 16384));
}

// Whether the sorted rows that a call writes pass the caches by.
bool stream_rows(const RowArgs& a, int elem) { return a.Tk * a.d * elem > kStreamBytes; }

// Up to a few thousand tokens, where the tokens alone do not fill the chip, more workgroups per token: for each eight slots in
// combine backward, for each 256 pieces of a row in the others (9 tokens of 4058, k 11, both
// directions 42.9 -> 32.1 us; 1500 of 2988, k 10, the backward 105.5 -> 89.7, 4000 of 1000, k 12,
// 64.5 -> 61.9; 300 and 3000 of 4096, k 8, plan, dispatch and combine 21.7 -> 19.1 and 108.9 ->
// 105.0).
constexpr int64_t kFewTokens = 4096;
unsigned slot_groups(const RowArgs& a) { return a.T <= kFewTokens ? (a.k + kSlots - 1) / kSlots : 1; }
unsigned piece_groups(const RowArgs& a, int elem) {
    const int64_t n = ((int64_t)a.d * elem + 15) / 16;
    return a.T <= kFewTokens ? (unsigned)std::min<int64_t>((n + kThreads - 1) / kThreads, 16) : 1;
}

template <typename K>
pr2_status launch_rows(K kernel, const RowArgs& a, int elem, const char* name, hipStream_t st,
                       unsigned groups = 1) {
    const dim3 block = row_block(a, elem);
    {
        LaunchScope scope(name, st);
        dim3 grid = row_grid(a, block);
        grid.y = groups;
        hipLaunchKernelGGL(kernel, grid, block, 0, st, a);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ok() : hip_fail(e, name);
}

RowArgs row_args(const pr2_moe_desc& d, const int32_t* offsets, const int32_t* row) {
    RowArgs a{};
    a.offsets = offsets;
    a.row = row;
    a.T = d.T;
    a.Tk = d.T * (int64_t)d.k;
    a.d = d.d;
    a.k = d.k;
    a.N = d.N;
    return a;
}

// the checks that the four row calls share; sets *done for T == 0
pr2_status check_rows(const pr2_moe_desc* desc, const int32_t* row, bool* done) {
    *done = false;
    const pr2_status s = check_desc(desc, false, false);
    if (s != PR2_OK) return s;
    if (desc->T == 0) {
        *done = true;
        return PR2_OK;
    }
    if (!row) return fail(PR2_ERR_NULL, "row_of_route is NULL");
    if ((uintptr_t)row % 4) return fail(PR2_ERR_ALIGN, "row_of_route is not 4-byte aligned");
    return PR2_OK;
}

bool overlap(const void* p, size_t n, const void* q, size_t m) {
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
    return a < b + m && b < a + n;
}

struct PlanWs {
    ReplayWs w;
    size_t bytes;
};

PlanWs plan_ws(const pr2_moe_desc& d, void* base) {
    PlanWs p{};
    const int tb = perm_tokens_per_block(d.k);
    p.w.nblk = (d.T + tb - 1) / tb;
    p.w.max_tiles = (d.T * (int64_t)d.k + kTileM - 1) / kTileM + d.N;
    char* q = base ? (char*)(((uintptr_t)base + 255) & ~(uintptr_t)255) : nullptr;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char* r = q ? q + off : nullptr;
        off += (bytes + 255) & ~(size_t)255;
        return r;
    };
    p.w.err = (int*)take(sizeof(int) * ERR_WORDS);
    p.w.tile_count = (int*)take(sizeof(int));
    p.w.bcount = (int*)take(sizeof(int) * (size_t)d.N * p.w.nblk);
    p.w.tiles = (int*)take(sizeof(int) * 3 * (size_t)p.w.max_tiles);
    p.bytes = off + 256;
    return p;
}

}  // namespace

size_t dispatch_plan_bytes(const pr2_moe_desc& d) { return plan_ws(d, nullptr).bytes; }

}  // namespace pr2

using namespace pr2;

extern "C" {

pr2_status pr2_dispatch_plan(const pr2_moe_desc* desc, const void* idx, int64_t ldi,
                             int32_t* offsets, int32_t* row_of_route, int32_t* route_of_row,
                             void* ws, size_t ws_bytes, pr2_stream_t stream) {
    pr2_status s = check_desc(desc, false, true);
    if (s != PR2_OK) return s;
    const pr2_moe_desc& d = *desc;
    const hipStream_t st = (hipStream_t)stream;
    if (!offsets) return fail(PR2_ERR_NULL, "offsets is NULL");
    if ((uintptr_t)offsets % 4) return fail(PR2_ERR_ALIGN, "offsets is not 4-byte aligned");
    if (ldi < d.k) return fail(PR2_ERR_SHAPE, "ldi = %lld < k = %d", (long long)ldi, d.k);
    if (d.T > 0) {
        if (!idx) return fail(PR2_ERR_NULL, "idx is NULL");
        if ((uintptr_t)idx % (d.idx_dtype == PR2_I16 ? 2 : 4))
            return fail(PR2_ERR_ALIGN, "idx is not aligned to its element size");
        if (!row_of_route || !route_of_row)
            return fail(PR2_ERR_NULL, "row_of_route and route_of_row are required");
        if ((uintptr_t)row_of_route % 4 || (uintptr_t)route_of_row % 4)
            return fail(PR2_ERR_ALIGN, "row_of_route or route_of_row is not 4-byte aligned");
        const size_t need = dispatch_plan_bytes(d);
        if (!ws) return fail(PR2_ERR_NULL, "ws is NULL (need %zu bytes)", need);
        if (ws_bytes < need)
            return fail(PR2_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, need);
    }
    s = device_ready();
    if (s != PR2_OK) return s;
    hipError_t e;
    if (d.T == 0) {
        e = launch_zero_i32(offsets, d.N + 1, st);
    } else {
        drop_split_records(ws, ws_bytes);
        PlanWs p = plan_ws(d, ws);
        p.w.offsets = offsets;
        p.w.perm_src = route_of_row;
        p.w.inv = row_of_route;
        e = launch_permute(d, idx, ldi, p.w, st);
    }
    if (e != hipSuccess) return hip_fail(e, "dispatch_plan launch");
    return ok();
}

pr2_status pr2_dispatch(const pr2_moe_desc* desc, const void* x, const int32_t* offsets,
                        const int32_t* row_of_route, void* xs, pr2_stream_t stream) {
    bool done;
    pr2_status s = check_rows(desc, row_of_route, &done);
    if (s != PR2_OK) return s;
    if (done) return ok();
    const pr2_moe_desc& d = *desc;
    if (!x || !xs || !offsets) return fail(PR2_ERR_NULL, "x, offsets and xs are required");
    if (!aligned16(x) || !aligned16(xs)) return fail(PR2_ERR_ALIGN, "x and xs must be 16-byte aligned");
    if ((uintptr_t)offsets % 4) return fail(PR2_ERR_ALIGN, "offsets is not 4-byte aligned");
    const size_t row = (size_t)d.d * (d.act_dtype == PR2_BF16 ? 2 : 4);
    if (overlap(x, d.T * row, xs, d.T * d.k * row)) return fail(PR2_ERR_SHAPE, "xs overlaps x");
    s = device_ready();
    if (s != PR2_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    RowArgs a = row_args(d, offsets, row_of_route);
    a.tok = x;
    a.rows_out = xs;
    if (d.act_dtype == PR2_F32)
        return launch_rows(stream_rows(a, 4) ? dispatch_kernel<float, true> : dispatch_kernel<float, false>,
                           a, 4, "dispatch", st, piece_groups(a, 4));
    return launch_rows(stream_rows(a, 2) ? dispatch_kernel<bf16_t, true> : dispatch_kernel<bf16_t, false>,
                       a, 2, "dispatch", st, piece_groups(a, 2));
}

pr2_status pr2_dispatch_backward(const pr2_moe_desc* desc, const void* dxs,
                                 const int32_t* row_of_route, void* dx, pr2_stream_t stream) {
    bool done;
    pr2_status s = check_rows(desc, row_of_route, &done);
    if (s != PR2_OK) return s;
    if (done) return ok();
    const pr2_moe_desc& d = *desc;
    if (!dxs || !dx) return fail(PR2_ERR_NULL, "dxs and dx are required");
    if (!aligned16(dxs) || !aligned16(dx))
        return fail(PR2_ERR_ALIGN, "dxs and dx must be 16-byte aligned");
    const size_t row = (size_t)d.d * (d.act_dtype == PR2_BF16 ? 2 : 4);
    if (overlap(dx, d.T * row, dxs, d.T * d.k * row)) return fail(PR2_ERR_SHAPE, "dx overlaps dxs");
    s = device_ready();
    if (s != PR2_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    RowArgs a = row_args(d, nullptr, row_of_route);
    a.rows = dxs;
    a.tok_out = dx;
    if (d.act_dtype == PR2_F32)
        return launch_rows(gather_sum_kernel<float, false>, a, 4, "dispatch_backward", st, piece_groups(a, 4));
    return launch_rows(gather_sum_kernel<bf16_t, false>, a, 2, "dispatch_backward", st, piece_groups(a, 2));
}

pr2_status pr2_combine(const pr2_moe_desc* desc, const void* o, const int32_t* row_of_route,
                       const float* gate, void* y, pr2_stream_t stream) {
    bool done;
    pr2_status s = check_rows(desc, row_of_route, &done);
    if (s != PR2_OK) return s;
    if (done) return ok();
    const pr2_moe_desc& d = *desc;
    if (!o || !gate || !y) return fail(PR2_ERR_NULL, "o, gate and y are required");
    if (!aligned16(o) || !aligned16(y)) return fail(PR2_ERR_ALIGN, "o and y must be 16-byte aligned");
    if ((uintptr_t)gate % 4) return fail(PR2_ERR_ALIGN, "gate is not 4-byte aligned");
    const size_t row = (size_t)d.d * (d.act_dtype == PR2_BF16 ? 2 : 4);
    if (overlap(y, d.T * row, o, d.T * d.k * row)) return fail(PR2_ERR_SHAPE, "y overlaps o");
    s = device_ready();
    if (s != PR2_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    RowArgs a = row_args(d, nullptr, row_of_route);
    a.rows = o;
    a.gate = gate;
    a.tok_out = y;
    if (d.act_dtype == PR2_F32)
        return launch_rows(gather_sum_kernel<float, true>, a, 4, "combine_rows", st, piece_groups(a, 4));
    return launch_rows(gather_sum_kernel<bf16_t, true>, a, 2, "combine_rows", st, piece_groups(a, 2));
}

pr2_status pr2_combine_backward(const pr2_moe_desc* desc, const void* dy, const void* o,
                                const int32_t* offsets, const int32_t* row_of_route,
                                const float* gate, void* d_o, float* dgate, pr2_stream_t stream) {
    bool done;
    pr2_status s = check_rows(desc, row_of_route, &done);
    if (s != PR2_OK) return s;
    if (done) return ok();
    const pr2_moe_desc& d = *desc;
    if (!dy || !o || !offsets || !gate || !d_o || !dgate)
        return fail(PR2_ERR_NULL, "dy, o, offsets, gate, d_o and dgate are required");
    if (!aligned16(dy) || !aligned16(o) || !aligned16(d_o))
        return fail(PR2_ERR_ALIGN, "dy, o and d_o must be 16-byte aligned");
    if ((uintptr_t)offsets % 4 || (uintptr_t)gate % 4 || (uintptr_t)dgate % 4)
        return fail(PR2_ERR_ALIGN, "offsets, gate or dgate is not 4-byte aligned");
    const size_t row = (size_t)d.d * (d.act_dtype == PR2_BF16 ? 2 : 4);
    const size_t rows = (size_t)d.T * d.k * row;
    if (overlap(d_o, rows, dy, d.T * row)) return fail(PR2_ERR_SHAPE, "d_o overlaps dy");
    if (d_o != o && overlap(d_o, rows, o, rows))
        return fail(PR2_ERR_SHAPE, "d_o overlaps o without being it");
    s = device_ready();
    if (s != PR2_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    RowArgs a = row_args(d, offsets, row_of_route);
    a.tok = dy;
    a.rows = o;
    a.gate = gate;
    a.rows_out = d_o;
    a.dgate = dgate;
    if (d.act_dtype == PR2_F32)
        return launch_rows(stream_rows(a, 4) ? combine_backward_kernel<float, true>
                                             : combine_backward_kernel<float, false>,
                           a, 4, "combine_backward", st, slot_groups(a));
    return launch_rows(stream_rows(a, 2) ? combine_backward_kernel<bf16_t, true>
                                         : combine_backward_kernel<bf16_t, false>,
                       a, 2, "combine_backward", st, slot_groups(a));
}

}  // extern "C"
