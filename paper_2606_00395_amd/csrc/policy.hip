// The policy's loss on the sampled tokens and its gradient.
//
// For each row of V logits z with target y and s = 1 / temperature: the running
// maximum M and, relative to it, S = sum 2^(k (z - M)) and E = sum of the same terms
// times their exponents, k = s log2(e), give in one pass
//   logp = s (z_y - M) - ln S,  lse = s M + ln S,  entropy = ln S - ln2 E / S,
// and with the gradient's coefficient c = d loss / d logp, which depends on logp alone,
//   dlogits_v = c s ([v = y] - 2^(k (z_v - M)) / S).
// Bound by HBM: V elements read per row, and V written where the gradient is wanted;
// two exponentials per element (a quarter-rate instruction each) come next.  Loss and gradient
// of 4096 x 151936 bf16 logits take 484 us, 5.15 TB/s (a large copy reaches 5.2); of 517 x
// 50257 fp32 in two calls 59 us, 5.3 TB/s; log-probabilities of 8 rows 10 us, two launches.
#include <type_traits>

#include "chunk.h"

namespace pr2 {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.4028234663852886e38f;
constexpr float kNegInf = -__builtin_huge_valf();

// Running statistics of part of a row.  m starts at the lowest finite number, so that a row
// of -infinity alone keeps s = 0 and no term ever subtracts -infinity from itself.
struct Stat {
    float m, s, e;
};

// One instruction, a relative error of 2^-22 or so; powers below 2^-126 are 0: a probability that is
// subnormal in fp32 has a gradient of 0.
__device__ __forceinline__ float exp2_native(float x) { return __builtin_amdgcn_exp2f(x); }

// moves the terms to the maximum m (>= a.m); exponents are cut off where their power is 0
__device__ __forceinline__ void rebase(Stat& a, float m, float k) {
    const float t = (a.m - m) * k;
    const float f = exp2_native(t);
    a.e = f * (a.e + fmaxf(t, -1e4f) * a.s);
    a.s *= f;
    a.m = m;
}

template <int n>
__device__ __forceinline__ void add_terms(Stat& a, const float* v, float k) {
    float m = v[0];
#pragma unroll
    for (int i = 1; i < n; ++i) m = fmaxf(m, v[i]);
    if (m > a.m) rebase(a, m, k);
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const float t = (v[i] - a.m) * k;
        const float p = exp2_native(t);
        a.s += p;
        a.e += p * fmaxf(t, -1e4f);      // a term of 0 adds 0, also at -infinity
    }
}

__device__ __forceinline__ void join_lanes(Stat& a, float k) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        Stat b{__shfl_xor(a.m, off, 64), __shfl_xor(a.s, off, 64), __shfl_xor(a.e, off, 64)};
        const float m = fmaxf(a.m, b.m);
        rebase(a, m, k);
        rebase(b, m, k);
        a.s += b.s;
        a.e += b.e;
    }
}

// What the wavefronts of a workgroup exchange.
template <int W>
struct Exchange {
    float m[W], s[W], e[W];
};

// all threads get the workgroup's statistics, joined in the same order every time
template <int W>
__device__ __forceinline__ void join_block(Stat& a, float k, Exchange<W>& x) {
    join_lanes(a, k);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) {
        x.m[wave] = a.m;
        x.s[wave] = a.s;
        x.e[wave] = a.e;
    }
    __syncthreads();
    Stat r{x.m[0], x.s[0], x.e[0]};
    float m = r.m;
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, x.m[w]);
    rebase(r, m, k);
#pragma unroll
    for (int w = 1; w < W; ++w) {
        Stat b{x.m[w], x.s[w], x.e[w]};
        rebase(b, m, k);
        r.s += b.s;
        r.e += b.e;
    }
    a = r;
}

struct PolicyArgs {
    const void* z;
    const void* y;
    const float* old;       // the loss's inputs; null for log-probabilities alone
    const float* ref;       // may be null
    const float* adv;
    const float* w;         // may be null: 1
    float* logp;            // outputs, each may be null
    float* lse;
    float* ent;
    float* coef;
    float4* rowsum;         // [T] the row's terms of the four sums (null without a loss)
    float4* part;           // [T, S] statistics of the parts of split rows
    float4* kept;           // [T] maximum, sum, coef and logp for the gradient's launch (may be null)
    void* dz;               // may be null, may be z
    const float* grad;      // backward: one number or null
    int64_t T, ldl, ldd;
    int V, S, y64;
    float it, k, lo, hi, beta;
};

// everything about row t that does not depend on its logits
struct Row {
    int64_t y;
    float w;
    bool on;
};

__device__ __forceinline__ Row open_row(const PolicyArgs& a, int64_t t) {
    Row r;
    r.y = a.y64 ? ((const int64_t*)a.y)[t] : (int64_t)((const int32_t*)a.y)[t];
    r.w = a.w ? a.w[t] : 1.0f;
    r.on = r.y >= 0 && r.y < a.V && r.w != 0.0f;
    return r;
}

struct Result {
    float coef;     // d loss / d logp
    float logp;
};

// From a row's statistics to its results; `write` for the thread that stores them.
__device__ __forceinline__ Result close_row(const PolicyArgs& a, int64_t t, const Row& r, float zy,
                                            const Stat& st, bool write) {
    const bool on = r.on && st.s != 0.0f;      // (NaN counts: it has to be seen)
    float logp = 0.0f, lse = kNegInf, ent = 0.0f, coef = 0.0f;
    float4 sums = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (on) {
        const float ls = logf(st.s);
        logp = (zy - st.m) * a.it - ls;
        lse = st.m * a.it + ls;
        ent = ls - kLn2 * (st.e / st.s);
        if (a.old) {
            const float A = a.adv[t];
            const float ratio = expf(logp - a.old[t]);
            const bool clipped = (A > 0.0f && ratio > a.hi) || (A < 0.0f && ratio < a.lo);
            float surr = 0.0f, dl = 0.0f;
            if (A != 0.0f) {
                surr = clipped ? (A > 0.0f ? a.hi : a.lo) * A : ratio * A;
                dl = clipped ? 0.0f : -A * ratio;
            }
            float kl = 0.0f, loss = -surr;
            if (a.ref) {
                const float d = a.ref[t] - logp;
                const float x = expm1f(d);
                kl = x - d;
                if (a.beta != 0.0f) {
                    loss += a.beta * kl;
                    dl -= a.beta * x;
                }
            }
            coef = r.w * dl;
            sums = make_float4(r.w * loss, r.w * kl, clipped ? r.w : 0.0f, r.w * ent);
        }
    }
    if (write) {
        if (a.logp) a.logp[t] = logp;
        if (a.lse) a.lse[t] = lse;
        if (a.ent) a.ent[t] = ent;
        if (a.coef) a.coef[t] = coef;
        if (a.rowsum) a.rowsum[t] = sums;
        if (a.kept) a.kept[t] = make_float4(st.m, st.s, coef, logp);
    }
    return Result{coef, logp};
}

template <typename T>
__device__ __forceinline__ void zero_chunks(T* row, int c0, int c1, int step, int full, int rem) {
    float v[Chunk<T>::E] = {};
    for (int c = c0; c < c1; c += step) store_chunk(row, c, full, rem, v);
}

// Statistics of row b / S, part b % S for workgroup b (whole rows finish here).
constexpr int kStatThreads = 256;
constexpr int kStatDeep = 4;        // chunks in flight per thread

template <typename T>
__global__ void __launch_bounds__(kStatThreads) policy_stats_kernel(PolicyArgs a) {
    constexpr int E = Chunk<T>::E;
    const uint32_t b = block_number();
    const int64_t t = b / (uint32_t)a.S;
    const int part = (int)(b - t * a.S);
    if (t >= a.T) return;
    __shared__ Exchange<kStatThreads / 64> x;
    const Row r = open_row(a, t);
    Stat st{kLowest, 0.0f, 0.0f};
    const T* z = (const T*)a.z + t * a.ldl;
    float zy = 0.0f;
    if (r.on) {
        zy = Act<T>::to_f32(z[r.y]);
        const int full = a.V / E, rem = a.V % E;
        const int n = full + (rem != 0);
        const int per = (n + a.S - 1) / a.S;
        const int c0 = part * per, c1 = min(n, c0 + per);
        int c = c0 + (int)threadIdx.x;
        for (; c + (kStatDeep - 1) * kStatThreads < min(c1, full); c += kStatDeep * kStatThreads) {
            u32x4 w[kStatDeep];
#pragma unroll
            for (int i = 0; i < kStatDeep; ++i)
                w[i] = *(const u32x4_any*)(z + (int64_t)(c + i * kStatThreads) * E);
#pragma unroll
            for (int i = 0; i < kStatDeep; ++i) {
                float v[E];
                Chunk<T>::open(w[i], v);
                add_terms<E>(st, v, a.k);
            }
        }
        for (; c < c1; c += kStatThreads) {
            float v[E];
            Chunk<T>::open(load_chunk(z, c, full, rem, Chunk<T>::kNegInf), v);
            add_terms<E>(st, v, a.k);
        }
        join_block(st, a.k, x);
    }
    if (a.S > 1) {
        if (threadIdx.x == 0) a.part[b] = make_float4(st.m, st.s, st.e, 0.0f);
    } else {
        close_row(a, t, r, zy, st, threadIdx.x == 0);
    }
}

// the four sums over the tokens, in fp64 and a fixed order, by one workgroup
constexpr int kSumThreads = 1024;
__device__ __forceinline__ void sum_rows(const float4* rows, int64_t T, float* out) {
    __shared__ double sh[4][kSumThreads / 64];
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    for (int64_t t = threadIdx.x; t < T; t += kSumThreads) {
        const float4 r = rows[t];
        v[0] += r.x;
        v[1] += r.y;
        v[2] += r.z;
        v[3] += r.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) v[i] += __shfl_xor(v[i], off, 64);
        if ((threadIdx.x & 63) == 0) sh[i][threadIdx.x >> 6] = v[i];
    }
    __syncthreads();
    if (threadIdx.x < 4) {
        double s = 0.0;
        for (int w = 0; w < kSumThreads / 64; ++w) s += sh[threadIdx.x][w];
        out[threadIdx.x] = (float)s;
    }
}

// Rows whose statistics came in S <= 64 parts: one wavefront per row.  With SUMS one workgroup
// takes all rows and the sums as well.
template <typename T, bool SUMS>
__global__ void __launch_bounds__(SUMS ? kSumThreads : 256) policy_finish_kernel(PolicyArgs a, float* sums) {
    constexpr int kWaves = (SUMS ? kSumThreads : 256) / 64;
    const int lane = threadIdx.x & 63;
    for (int64_t t = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); t < a.T;
         t += (int64_t)gridDim.x * kWaves) {
        const Row r = open_row(a, t);
        Stat st{kLowest, 0.0f, 0.0f};
        if (lane < a.S) {
            const float4 p = a.part[t * a.S + lane];
            st = Stat{p.x, p.y, p.z};
        }
        join_lanes(st, a.k);
        const float zy = r.on ? Act<T>::to_f32(((const T*)a.z)[t * a.ldl + r.y]) : 0.0f;
        close_row(a, t, r, zy, st, lane == 0);
    }
    if (SUMS) {
        __syncthreads();
        sum_rows(a.rowsum, a.T, sums);
    }
}

// dlogits of row b / S, part b % S for workgroup b.  KEPT: from what the statistics of the same
// call left, p = 2^(k (z - M)) / S as the fused form has it; otherwise from the caller's lse
// and coef, where log p has the rounding of lse (half a last place of a number that grows with
// the level of the logits).  NT: the gradient passes the caches by.
template <typename T, bool KEPT, bool NT>
__global__ void __launch_bounds__(256) policy_grad_kernel(PolicyArgs a) {
    constexpr int E = Chunk<T>::E;
    const uint32_t b = block_number();
    const int64_t t = b / (uint32_t)a.S;
    const int part = (int)(b - t * a.S);
    if (t >= a.T) return;
    const T* z = (const T*)a.z + t * a.ldl;
    T* dz = (T*)a.dz + t * a.ldd;
    const int full = a.V / E, rem = a.V % E;
    const int n = full + (rem != 0);
    const int per = (n + a.S - 1) / a.S;
    const int c0 = part * per, c1 = min(n, c0 + per);
    const int64_t y = a.y64 ? ((const int64_t*)a.y)[t] : (int64_t)((const int32_t*)a.y)[t];
    float4 kept = make_float4(0.0f, 1.0f, 0.0f, 0.0f);
    if (KEPT) kept = a.kept[t];
    const float coef = KEPT ? kept.z : a.coef[t];
    if (coef == 0.0f || y < 0 || y >= a.V) {
        zero_chunks(dz, c0 + (int)threadIdx.x, c1, 256, full, rem);
        return;
    }
    const float lse = KEPT ? 0.0f : a.lse[t];
    const float g = coef * a.it * (a.grad ? *a.grad : 1.0f);
    const float gs = KEPT ? -g / kept.y : -g;
    const int yc = (int)(y / E), ye = (int)(y % E);
    constexpr int D = 4;
    for (int c = c0 + (int)threadIdx.x; c < c1; c += D * 256) {
        u32x4 w[D];
#pragma unroll
        for (int i = 0; i < D; ++i)
            if (c + i * 256 < c1)
                w[i] = load_chunk(z, c + i * 256, full, rem, Chunk<T>::kNegInf);
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const int ci = c + i * 256;
            if (ci >= c1) continue;
            float v[E];
            Chunk<T>::open(w[i], v);
            float ly = kept.w;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (KEPT) {
                    v[j] = gs * exp2_native((v[j] - kept.x) * a.k);
                } else {        // log p first, in one rounding, then its power
                    v[j] = fmaf(v[j], a.it, -lse);
                    if (j == ye) ly = v[j];
                    v[j] = gs * exp2_native(v[j] * kLog2e);
                }
            }
            if (ci == yc) {
                const float gy = -g * expm1f(ly);       // c s (1 - p_y)
#pragma unroll
                for (int j = 0; j < E; ++j) v[j] = j == ye ? gy : v[j];
            }
            store_chunk<T, NT>(dz, ci, full, rem, v);
        }
    }
}

// Loss and gradient, one row at a time per workgroup.  The row's first NT * NCH chunks stay in
// registers between the two passes (a CU's register file is 512 KiB, a row of 151936 bf16
// logits 297 KiB), the rest is read again; the elements after its last whole chunk go one to
// a thread.  A workgroup that fills a CU (NEXT) takes rows from a counter until they are used
// up, and loads each piece of the next row into the registers that the piece of this one
// has just left, so that the memory does not wait for a row's statistics; the others take
// one row, and hide behind each other.
template <typename T, int NT, int NCH, bool NEXT>
__global__ void __launch_bounds__(NT) policy_fused_kernel(PolicyArgs a, int* counter) {
    constexpr int E = Chunk<T>::E;
    __shared__ Exchange<NT / 64> x[2];
    __shared__ int s_next[2];
    int tid = threadIdx.x;
    const int full = a.V / E, rem = a.V % E;
    int64_t t = block_number();
    if (t >= a.T) return;
    Row r = open_row(a, t);
    u32x4 w[NCH];
    auto load_piece = [&](const T* z, int i) __attribute__((always_inline)) {
        const int c = i * NT + tid;
        constexpr uint32_t p = Chunk<T>::kNegInf;
        w[i] = c < full ? load16<false>(z + (int64_t)c * E) : u32x4{p, p, p, p};
    };
    if (r.on) {
#pragma unroll
        for (int i = 0; i < NCH; ++i) load_piece((const T*)a.z + t * a.ldl, i);
    }
    for (int turn = 0;; turn ^= 1) {
        // (a new number each time: kept over the turns, the pieces' addresses fill the registers)
        if (NEXT) asm volatile("" : "+v"(tid));
        const T* z = (const T*)a.z + t * a.ldl;
        T* dz = (T*)a.dz + t * a.ldd;
        if (NEXT && tid == 0) s_next[turn] = gridDim.x + atomicAdd(counter, 1);
        Stat st{kLowest, 0.0f, 0.0f};
        float zy = 0.0f, zt = 0.0f;
        if (r.on) {
            zy = Act<T>::to_f32(z[r.y]);
            if (tid < rem) {
                zt = Act<T>::to_f32(z[(int64_t)full * E + tid]);
                add_terms<1>(st, &zt, a.k);
            }
#pragma unroll
            for (int i = 0; i < NCH; ++i) {
                float v[E];
                Chunk<T>::open(w[i], v);
                add_terms<E>(st, v, a.k);
            }
            for (int c = NCH * NT + tid; c < full; c += NT) {
                float v[E];
                Chunk<T>::open(load16<false>(z + (int64_t)c * E), v);
                add_terms<E>(st, v, a.k);
            }
            // every thread holds z_y before the barrier behind which it may be overwritten
            asm volatile("" ::"v"(zy));
            join_block(st, a.k, x[turn]);
        } else if (NEXT) {
            __syncthreads();
        }
        const int64_t t1 = NEXT ? s_next[turn] : a.T;
        const Row r1 = NEXT && t1 < a.T ? open_row(a, t1) : Row{0, 0.0f, false};
        const T* z1 = (const T*)a.z + (NEXT && t1 < a.T ? t1 * a.ldl : 0);
        const Result res = close_row(a, t, r, zy, st, tid == 0);
        const float g = res.coef * a.it;
        const float gy = -g * expm1f(res.logp);       // c s (1 - p_y) without the cancellation
        const int yc = (int)(r.y / E), ye = (int)(r.y % E);
        const bool some = res.coef != 0.0f;
        const float gs = some ? -g / st.s : 0.0f;
        auto open_piece = [&](const u32x4& raw, int c, float (&v)[E]) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = 0.0f;
            if (!some) return;
            Chunk<T>::open(raw, v);
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = gs * exp2_native((v[j] - st.m) * a.k);
            if (c == yc) {
#pragma unroll
                for (int j = 0; j < E; ++j) v[j] = j == ye ? gy : v[j];
            }
        };
        auto pieces = [&](auto more) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NCH; ++i) {
                const int c = i * NT + tid;
                float v[E];
                open_piece(w[i], c, v);
                const u32x4 o = Chunk<T>::close(v);
                if (decltype(more)::value) load_piece(z1, i);
                if (c < full) store16<false>(dz + (int64_t)c * E, o);
                if (NEXT) __builtin_amdgcn_sched_barrier(0);    // one piece's values at a time
            }
        };
        if (NEXT && r1.on) pieces(std::true_type{});
        else pieces(std::false_type{});
        for (int c = NCH * NT + tid; c < full; c += NT) {
            u32x4 raw = {};
            float v[E];
            if (some) raw = load16<false>(z + (int64_t)c * E);
            open_piece(raw, c, v);
            store16<false>(dz + (int64_t)c * E, Chunk<T>::close(v));
        }
        if (tid < rem) {
            float v = some ? gs * exp2_native((zt - st.m) * a.k) : 0.0f;
            if (some && full == yc && tid == ye) v = gy;
            dz[(int64_t)full * E + tid] = Act<T>::from_f32(v);
        }
        if (t1 >= a.T) return;
        t = t1;
        r = r1;
    }
}

__global__ void __launch_bounds__(kSumThreads)
policy_sums_kernel(const float4* rows, int64_t T, float* out) {
    sum_rows(rows, T, out);
}

// ------------------------------------------------------------------ host ----
constexpr int kCus = 256;
constexpr int kMaxParts = 64;
constexpr int64_t kMaxRows = 0x7fffffff / kMaxParts;    // T x parts are numbered in 32 bits
constexpr int64_t kMaxStride = (int64_t)1 << 35;        // T x stride in bytes stays below 2^63
constexpr int64_t kFillWgs = 2048;      // workgroups of 256 that fill the chip
constexpr size_t kPartBytes = sizeof(float4) * 2 * kFillWgs;

// Rows of up to this many chunks fit the registers of 512 threads.
constexpr int kShortRow = 512 * 18;

// Chunks per thread that 1024 threads hold of a longer one.
constexpr int kLongHeld = 19;

int row_chunks(const pr2_policy_desc& d) {
    const int e = d.act_dtype == PR2_BF16 ? 8 : 4;
    return (int)(((int64_t)d.V + e - 1) / e);
}

// Parts per row: enough workgroups to fill the chip, each with two chunks a thread at least.
int row_parts(const pr2_policy_desc& d) {
    const int64_t fill = (kFillWgs + d.T - 1) / d.T;
    const int64_t most = row_chunks(d) / (2 * kStatThreads);
    int64_t s = fill < most ? fill : most;
    if (s > kMaxParts) s = kMaxParts;
    return s < 1 ? 1 : (int)s;
}

// Gradients above this are written past the caches, so that the logits that the pass before
// read are still there (104 MB of each: both passes 68 -> 57 us).  The eight L2s hold 32 MiB.
constexpr int64_t kStreamBytes = 32 << 20;

// Long rows, a whole CU each in the fused form, are better read twice by many workgroups while
// they are few.  Read twice and fused, us, loss and gradient of
//              32 rows      64          128         192         256         512
//   151936 bf16  18.8 28.3    23.2 29.6   29.6 31.6   38.5 32.9   44.8 35.0   75.7 74.7
//    80000 bf16  16.2 26.1    18.3 26.9   22.6 28.5   28.1 29.7   29.5 30.8   47.1 54.8
//   151936 fp32  20.8 31.1    26.4 37.4   42.9 40.1   57.7 47.8   70.6 65.5   157 160
//    76000 fp32  17.4 18.5    22.0 20.0   26.6 22.1   35.9 26.0   43.0 30.6   69.9 68.5
//    50257 fp32  16.0 17.7    18.4 18.7   23.5 20.5   27.2 22.8   33.3 25.2   52.0 43.6
// so they are even near 140, above 512, 115, 45 and 75 rows.  One limit stands for all, which gives
// away up to 10 us just below it in fp32 and 8 us at 512 rows of 80000.  Shorter rows are faster
// fused at any count (32000 logits: 13 against 16 us for one row, 63 against 77 for 2048).
constexpr int64_t kFewRows = 192;
bool fuse_rows(const pr2_policy_desc& d) { return d.T >= kFewRows || row_chunks(d) <= kShortRow; }

struct PolicyWs {
    int* counter;
    float4* rowsum;
    float4* part;
    float4* kept;
    size_t bytes;
};

PolicyWs policy_ws(const pr2_policy_desc& d, void* base) {
    char* p = base ? (char*)(((uintptr_t)base + 255) & ~(uintptr_t)255) : nullptr;
    PolicyWs w{};
    w.part = (float4*)p;            // (split rows and the counter exclude each other)
    w.counter = (int*)p;
    const size_t stats = (sizeof(float4) * (size_t)d.T + 255) & ~(size_t)255;
    w.rowsum = (float4*)(p ? p + kPartBytes : nullptr);
    w.kept = (float4*)(p ? p + kPartBytes + stats : nullptr);
    w.bytes = kPartBytes + 2 * stats + 256;
    return w;
}

bool finite_nonneg(float v) { return v >= 0.0f && v <= 3.4028234663852886e38f; }
bool aligned_to(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

pr2_status check_policy(const pr2_policy_desc* desc, bool loss, bool grad) {
    if (!desc) return fail(PR2_ERR_NULL, "desc is NULL");
    const pr2_policy_desc& d = *desc;
    if (d.act_dtype != PR2_F32 && d.act_dtype != PR2_BF16)
        return fail(PR2_ERR_DTYPE, "act_dtype %d is not PR2_F32 or PR2_BF16", d.act_dtype);
    if (d.token_dtype != PR2_I32 && d.token_dtype != PR2_I64)
        return fail(PR2_ERR_DTYPE, "token_dtype %d is not PR2_I32 or PR2_I64", d.token_dtype);
    if (d.T < 0) return fail(PR2_ERR_SHAPE, "T = %lld < 0", (long long)d.T);
    if (d.V < 1) return fail(PR2_ERR_SHAPE, "V = %d < 1", d.V);
    if (d.ldl < d.V) return fail(PR2_ERR_SHAPE, "ldl = %lld < V = %d", (long long)d.ldl, d.V);
    if (grad && d.ldd < d.V)
        return fail(PR2_ERR_SHAPE, "ldd = %lld < V = %d", (long long)d.ldd, d.V);
    if (!(d.inv_temp > 0.0f) || !finite_nonneg(d.inv_temp))
        return fail(PR2_ERR_SHAPE, "inv_temp = %g is not positive and finite", (double)d.inv_temp);
    if (loss && !(finite_nonneg(d.clip_low) && finite_nonneg(d.clip_high) && finite_nonneg(d.kl_coef)))
        return fail(PR2_ERR_SHAPE, "clip_low, clip_high and kl_coef must be finite and >= 0");
    if (d.T > kMaxRows)
        return fail(PR2_ERR_UNSUPPORTED, "T = %lld rows exceed %lld", (long long)d.T,
                    (long long)kMaxRows);
    if (d.V > 0x7fffffff - 65536)
        return fail(PR2_ERR_UNSUPPORTED, "V = %d is too large", d.V);
    if (d.ldl > kMaxStride || (grad && d.ldd > kMaxStride))
        return fail(PR2_ERR_UNSUPPORTED, "ldl = %lld or ldd = %lld exceeds %lld", (long long)d.ldl,
                    (long long)d.ldd, (long long)kMaxStride);
    return PR2_OK;
}

pr2_status check_logits(const pr2_policy_desc& d, const void* logits, const void* token,
                        const void* dlogits, bool grad) {
    const size_t e = d.act_dtype == PR2_BF16 ? 2 : 4;
    if (!logits) return fail(PR2_ERR_NULL, "logits is NULL");
    if (!token) return fail(PR2_ERR_NULL, "token is NULL");
    if (grad && !dlogits) return fail(PR2_ERR_NULL, "dlogits is NULL");
    if (!aligned_to(logits, e) || (grad && !aligned_to(dlogits, e)))
        return fail(PR2_ERR_ALIGN, "logits or dlogits is not aligned to its element size");
    if (!aligned_to(token, d.token_dtype == PR2_I64 ? 8 : 4))
        return fail(PR2_ERR_ALIGN, "token is not aligned to its element size");
    if (grad) {
        const uintptr_t z0 = (uintptr_t)logits, z1 = z0 + e * ((size_t)(d.T - 1) * d.ldl + d.V);
        const uintptr_t g0 = (uintptr_t)dlogits, g1 = g0 + e * ((size_t)(d.T - 1) * d.ldd + d.V);
        // rows of the same stride can lie between each other: the gradient's start is then `off`
        // bytes into a row's period, past its logits and with room before the next one's
        const size_t period = e * (size_t)d.ldl, row = e * (size_t)d.V;
        const size_t off = g0 >= z0 ? (g0 - z0) % period : (period - (z0 - g0) % period) % period;
        const bool between = d.ldl == d.ldd && off >= row && off + row <= period;
        if (z0 < g1 && g0 < z1 && !between && !(z0 == g0 && d.ldl == d.ldd))
            return fail(PR2_ERR_SHAPE, "dlogits overlaps logits without being the same rows");
    }
    return PR2_OK;
}

PolicyArgs policy_args(const pr2_policy_desc& d, const void* logits, const void* token) {
    PolicyArgs a{};
    a.z = logits;
    a.y = token;
    a.T = d.T;
    a.ldl = d.ldl;
    a.ldd = d.ldd;
    a.V = d.V;
    a.S = 1;
    a.y64 = d.token_dtype == PR2_I64;
    a.it = d.inv_temp;
    a.k = d.inv_temp * kLog2e;
    a.lo = 1.0f - d.clip_low;
    a.hi = 1.0f + d.clip_high;
    a.beta = d.kl_coef;
    return a;
}

hipError_t launch_sums(const float4* rows, int64_t T, float* sums, hipStream_t s) {
    LaunchScope scope("policy_sums", s);
    hipLaunchKernelGGL(policy_sums_kernel, dim3(1), dim3(kSumThreads), 0, s, rows, T, sums);
    return hipGetLastError();
}

// One workgroup finishes split rows and their sums in one launch where each of its wavefronts has
// one row (loss and gradient of one row of 151936 logits 18.3 -> 15.7 us; 32 rows, two each,
// 19.8 and 20.0, 64 rows 23.7 and 28.2).
constexpr int64_t kOneFinish = kSumThreads / 64;

// statistics and per-row results; with sums the four sums too
template <typename T>
hipError_t launch_stats(const pr2_policy_desc& d, PolicyArgs a, float* sums, hipStream_t s) {
    a.S = row_parts(d);
    {
        LaunchScope scope("policy_stats", s);
        hipLaunchKernelGGL(policy_stats_kernel<T>, wide_grid(d.T * a.S, kStatThreads), dim3(kStatThreads),
                           0, s, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.S > 1 && sums && d.T <= kOneFinish) {
        LaunchScope scope("policy_finish", s);
        hipLaunchKernelGGL((policy_finish_kernel<T, true>), dim3(1), dim3(kSumThreads), 0, s, a, sums);
        return hipGetLastError();
    }
    if (a.S > 1) {
        LaunchScope scope("policy_finish", s);
        hipLaunchKernelGGL((policy_finish_kernel<T, false>), dim3((unsigned)((d.T + 3) / 4)), dim3(256),
                           0, s, a, nullptr);
        e = hipGetLastError();
    }
    return e == hipSuccess && sums ? launch_sums(a.rowsum, d.T, sums, s) : e;
}

template <typename T>
hipError_t launch_grad(const pr2_policy_desc& d, PolicyArgs a, hipStream_t s) {
    a.S = row_parts(d);
    LaunchScope scope("policy_grad", s);
    const dim3 grid = wide_grid(d.T * a.S, 256);
    const bool stream = d.T * d.V * (int64_t)sizeof(T) > kStreamBytes;
    if (a.kept && stream)
        hipLaunchKernelGGL((policy_grad_kernel<T, true, true>), grid, dim3(256), 0, s, a);
    else if (a.kept)
        hipLaunchKernelGGL((policy_grad_kernel<T, true, false>), grid, dim3(256), 0, s, a);
    else if (stream)
        hipLaunchKernelGGL((policy_grad_kernel<T, false, true>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((policy_grad_kernel<T, false, false>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_fused(const pr2_policy_desc& d, const PolicyArgs& a, int* counter, hipStream_t s) {
    const int n = row_chunks(d);
    const dim3 grid = wide_grid(d.T, 1024);
    // Rows that are held whole, eight a CU or more: the counter's turns (4096 rows of 151936
    // bf16 logits, a tenth of them without weight, 519 -> 484 us; without it 2048 rows took
    // 266 and 1024 rows 148 us, with it 267 and 149; 2048 fp32 rows, half of each read
    // again, 529 and 559).
    if (n > kShortRow && n <= 1024 * kLongHeld && d.T >= 8 * kCus) {
        const hipError_t e = launch_zero_i32(counter, 1, s);
        if (e != hipSuccess) return e;
        LaunchScope scope("policy_fused", s);
        hipLaunchKernelGGL((policy_fused_kernel<T, 1024, kLongHeld, true>), dim3(kCus), dim3(1024), 0, s, a, counter);
        return hipGetLastError();
    }
    LaunchScope scope("policy_fused", s);
    // (short rows to one wavefront each, no barrier: 16384 rows of 1609 bf16 logits 82 -> 36 us,
    // of 4000 85 -> 53; of 8000 104 with four wavefronts, 117 with one)
    if (n <= 64 * 4)
        hipLaunchKernelGGL((policy_fused_kernel<T, 64, 4, false>), grid, dim3(64), 0, s, a, nullptr);
    else if (n <= 64 * 8)
        hipLaunchKernelGGL((policy_fused_kernel<T, 64, 8, false>), grid, dim3(64), 0, s, a, nullptr);
    else if (n <= 256 * 4)
        hipLaunchKernelGGL((policy_fused_kernel<T, 256, 4, false>), grid, dim3(256), 0, s, a, nullptr);
    else if (n <= 256 * 16)
        hipLaunchKernelGGL((policy_fused_kernel<T, 256, 16, false>), grid, dim3(256), 0, s, a, nullptr);
    else if (n <= kShortRow)
        hipLaunchKernelGGL((policy_fused_kernel<T, 512, 18, false>), grid, dim3(512), 0, s, a, nullptr);
    else
        hipLaunchKernelGGL((policy_fused_kernel<T, 1024, kLongHeld, false>), grid, dim3(1024), 0, s, a, nullptr);
    return hipGetLastError();
}

}  // namespace
}  // namespace pr2

using namespace pr2;

extern "C" {

size_t pr2_policy_workspace_bytes(const pr2_policy_desc* desc) {
    if (!desc || desc->T < 0 || desc->T > kMaxRows || desc->V < 1) return 0;
    return policy_ws(*desc, nullptr).bytes;
}

pr2_status pr2_token_logprob(const pr2_policy_desc* desc, const void* logits, const void* token,
                             float* logp_out, float* lse_out, float* entropy_out, void* ws,
                             size_t ws_bytes, pr2_stream_t stream) {
    pr2_status s = check_policy(desc, false, false);
    if (s != PR2_OK) return s;
    const pr2_policy_desc& d = *desc;
    if (d.T == 0) return ok();
    s = check_logits(d, logits, token, nullptr, false);
    if (s != PR2_OK) return s;
    if (!logp_out) return fail(PR2_ERR_NULL, "logp_out is NULL");
    if (!aligned_to(logp_out, 4) || !aligned_to(lse_out, 4) || !aligned_to(entropy_out, 4))
        return fail(PR2_ERR_ALIGN, "a per-token output is not 4-byte aligned");
    const size_t need = policy_ws(d, nullptr).bytes;
    if (!ws) return fail(PR2_ERR_NULL, "ws is NULL (need %zu bytes)", need);
    if (ws_bytes < need)
        return fail(PR2_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, need);
    s = device_ready();
    if (s != PR2_OK) return s;
    drop_split_records(ws, ws_bytes);
    PolicyArgs a = policy_args(d, logits, token);
    a.logp = logp_out;
    a.lse = lse_out;
    a.ent = entropy_out;
    a.part = policy_ws(d, ws).part;
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = d.act_dtype == PR2_BF16 ? launch_stats<bf16_t>(d, a, nullptr, st)
                                                 : launch_stats<float>(d, a, nullptr, st);
    if (e != hipSuccess) return hip_fail(e, "token_logprob launch");
    return ok();
}

pr2_status pr2_policy_loss(const pr2_policy_desc* desc, const void* logits, const void* token,
                           const float* logp_old, const float* logp_ref, const float* adv,
                           const float* weight, float* sums_out, float* logp_out, float* lse_out,
                           float* entropy_out, float* coef_out, void* dlogits, void* ws,
                           size_t ws_bytes, pr2_stream_t stream) {
    const bool grad = dlogits != nullptr;
    pr2_status s = check_policy(desc, true, grad);
    if (s != PR2_OK) return s;
    const pr2_policy_desc& d = *desc;
    if (!sums_out) return fail(PR2_ERR_NULL, "sums_out is NULL");
    for (const void* p : {(const void*)logp_old, (const void*)logp_ref, (const void*)adv,
                          (const void*)weight, (const void*)sums_out, (const void*)logp_out,
                          (const void*)lse_out, (const void*)entropy_out, (const void*)coef_out})
        if (!aligned_to(p, 4)) return fail(PR2_ERR_ALIGN, "a per-token tensor is not 4-byte aligned");
    const hipStream_t st = (hipStream_t)stream;
    if (d.T > 0) {
        s = check_logits(d, logits, token, dlogits, grad);
        if (s != PR2_OK) return s;
        if (!logp_old || !adv) return fail(PR2_ERR_NULL, "logp_old and adv are required");
        const size_t need = policy_ws(d, nullptr).bytes;
        if (!ws) return fail(PR2_ERR_NULL, "ws is NULL (need %zu bytes)", need);
        if (ws_bytes < need)
            return fail(PR2_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, need);
    }
    s = device_ready();
    if (s != PR2_OK) return s;
    const PolicyWs w = policy_ws(d, ws);
    hipError_t e;
    if (d.T == 0) {
        e = launch_sums(nullptr, 0, sums_out, st);
    } else {
        drop_split_records(ws, ws_bytes);
        PolicyArgs a = policy_args(d, logits, token);
        a.old = logp_old;
        a.ref = logp_ref;
        a.adv = adv;
        a.w = weight;
        a.logp = logp_out;
        a.lse = lse_out;
        a.ent = entropy_out;
        a.coef = coef_out;
        a.rowsum = w.rowsum;
        a.part = w.part;
        a.dz = dlogits;
        const bool bf = d.act_dtype == PR2_BF16;
        if (grad && fuse_rows(d)) {
            e = bf ? launch_fused<bf16_t>(d, a, w.counter, st) : launch_fused<float>(d, a, w.counter, st);
            if (e == hipSuccess) e = launch_sums(w.rowsum, d.T, sums_out, st);
        } else {
            if (grad) a.kept = w.kept;
            e = bf ? launch_stats<bf16_t>(d, a, sums_out, st) : launch_stats<float>(d, a, sums_out, st);
            if (e == hipSuccess && grad)
                e = bf ? launch_grad<bf16_t>(d, a, st) : launch_grad<float>(d, a, st);
        }
    }
    if (e != hipSuccess) return hip_fail(e, "policy_loss launch");
    return ok();
}

pr2_status pr2_policy_loss_backward(const pr2_policy_desc* desc, const void* logits,
                                    const void* token, const float* lse, const float* coef,
                                    const float* grad_loss, void* dlogits, pr2_stream_t stream) {
    pr2_status s = check_policy(desc, false, true);
    if (s != PR2_OK) return s;
    const pr2_policy_desc& d = *desc;
    if (d.T == 0) return ok();
    s = check_logits(d, logits, token, dlogits, true);
    if (s != PR2_OK) return s;
    if (!lse || !coef) return fail(PR2_ERR_NULL, "lse and coef are required");
    if (!aligned_to(lse, 4) || !aligned_to(coef, 4) || !aligned_to(grad_loss, 4))
        return fail(PR2_ERR_ALIGN, "lse, coef or grad_loss is not 4-byte aligned");
    s = device_ready();
    if (s != PR2_OK) return s;
    PolicyArgs a = policy_args(d, logits, token);
    a.lse = const_cast<float*>(lse);
    a.coef = const_cast<float*>(coef);
    a.grad = grad_loss;
    a.dz = dlogits;
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = d.act_dtype == PR2_BF16 ? launch_grad<bf16_t>(d, a, st)
                                                 : launch_grad<float>(d, a, st);
    if (e != hipSuccess) return hip_fail(e, "policy_loss_backward launch");
    return ok();
}

}  // extern "C"
