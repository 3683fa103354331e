// Weight gradients of linear layers, their input rows as they are or as an 8-bit checkpoint:
//   dW[e] [n_out, n_in] = sum over expert e's rows r of dy[r]^T x[src(r)],
// src(r) the token of row r's route, or r itself.
//
// A packed value is an int8 times a power of two, exact in bf16 and fp32, so nothing is
// rounded on the way into the products.
#include <algorithm>
#include <type_traits>

#include "chunk.h"
#include "copies.h"

namespace pr2 {
namespace {

typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;

struct WgradArgs {
    const void* dy;             // [R, n_out]
    const int8_t* q;            // [Rx, n_in]; null: x is not packed
    const uint8_t* scale;       // [Rx, groups]
    const void* x;              // [Rx, n_in] as dy, where it is not packed
    const int* offsets;         // [N + 1] or null (one weight over all rows)
    const int* route;           // [R] or null
    float* dW;                  // [N, n_out, n_in]
    int64_t R, Rx;
    int n_out, n_in, N, k;
    int groups;
    const int* order;           // [N] experts by decreasing row count; null: as they come
    float* part;                // [S, N, n_out, n_in] partial sums of S > 1 slices of the rows
    int S;
    int G;                      // 256 x 256 tiles: column tiles per workgroup
    bool split;                 // each expert's tiles on all XCDs
};

// rows of expert e, clamped to the R that there are
__device__ __forceinline__ void expert_rows(const WgradArgs& a, int e, int* first, int* last) {
    const int R = (int)a.R;
    *first = a.offsets ? min(max(a.offsets[e], 0), R) : 0;
    *last = a.offsets ? max(min(a.offsets[e + 1], R), *first) : R;
}

// slice s of a.S of them, whole steps of 32
__device__ __forceinline__ void slice_rows(const WgradArgs& a, int s, int* first, int* last) {
    const int len = ((*last - *first + a.S - 1) / a.S + 31) / 32 * 32;
    *first = (int)min((int64_t)*last, *first + (int64_t)s * len);
    *last = (int)min((int64_t)*last, (int64_t)*first + len);
}

// packed row of dy's row r, -1 if it has none
__device__ __forceinline__ int source_row(const WgradArgs& a, int r) {
    if (!a.route) return r;
    const int q = a.route[r];
    const int t = q / a.k;
    return q >= 0 && t < a.Rx ? t : -1;
}

// Any type, width and row count: 64 x 64 outputs per workgroup, four wavefronts of 32 x 32 on
// v_mfma_f32_32x32x2_f32 (fp32 products and sums), 32 rows of both operands staged in LDS as
// fp32 at a time, the next 32 in flight meanwhile.  Small layers are bound by the latency of
// that chain (with the packing 15.5 us at 1226 rows, 7 experts of 135 x 203; 17.7 where the
// operands were opened on arrival), large ones by the fp32 MFMA and the LDS (112 TFLOP/s at
// 4096 x 4096 over 32768 rows, where the library's fp32 product reaches 154).  dy and rows of x in bf16
// stay so: v_mfma_f32_32x32x16_bf16 with the transposing LDS read (4096 x 1001 x 999 in 90 us, opened to
// fp32 119).
constexpr int kTile = 64;
constexpr int kStep = 32;
constexpr int kTilePitch = kTile + 32;      // the two halves of a wavefront read other banks

// 8 elements of a row from column c on, their bits as they lie there; those past the row's n
// stand in for others of it (WHOLE: there are none)
template <typename T, bool WHOLE>
__device__ __forceinline__ void load8(const T* row, int c, int n, u32x4 (&w)[8 / Chunk<T>::E]) {
    constexpr int E = Chunk<T>::E;
    if (WHOLE) {
#pragma unroll
        for (int i = 0; i < 8 / E; ++i) w[i] = load16<false>(row + c + i * E);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __builtin_bit_cast(typename Chunk<T>::Bits, row[min(c + i, n - 1)]);
        if (E == 4) w[i / 4][i % 4] = b;
        else w[0][i / 2] = i & 1 ? w[0][i / 2] | b << 16 : b;
    }
}

// the same of a packed row, 8 bytes (shifted into place: the ones past the row's end are 0)
__device__ __forceinline__ uint64_t load8_packed(const int8_t* row, int c, int n) {
    typedef uint64_t u64_byte __attribute__((aligned(1)));
    if (n >= 8) {
        const int at = min(c, n - 8);
        return *(const u64_byte*)(row + at) >> min(8 * (c - at), 63);
    }
    uint64_t w = 0;
    for (int i = 0; i < n - c; ++i) w |= (uint64_t)(uint8_t)row[c + i] << (8 * i);
    return w;
}

template <typename T, bool PACKED>
__global__ void __launch_bounds__(256) wgrad_tile_kernel(WgradArgs a) {
    __shared__ __attribute__((aligned(16))) float A[kStep * kTilePitch], B[kStep * kTilePitch];
    const int tid = threadIdx.x;
    const int lane = tid & 63, wave = tid >> 6;
    const int o0 = (int)blockIdx.y * kTile, c0 = (int)blockIdx.x * kTile;
    const int slice = a.S == 1 ? 0 : (int)blockIdx.z / a.N;
    const int e = (int)blockIdx.z - slice * a.N;
    int first, last;
    expert_rows(a, e, &first, &last);
    slice_rows(a, slice, &first, &last);
    const int sr = tid / 8, sc = (tid % 8) * 8;         // row and columns this thread stages
    f32x16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.0f;
    // A step's operands as they come: nothing is computed from them before the products of the
    // step before.  Columns past the matrix hold anything, they reach only outputs that are
    // not stored.
    constexpr int E = Chunk<T>::E;
    const bool whole = o0 + kTile <= a.n_out, whole_x = c0 + kTile <= a.n_in;
    u32x4 wa[8 / E], wx[8 / E];
    uint64_t wb = 0;
    uint32_t byte = 0;
    bool on;
    auto fetch = [&](int r0) __attribute__((always_inline)) {
        const int r = min(r0 + sr, last - 1);
        const int x = source_row(a, r);
        on = r0 + sr < last && x >= 0;
        const int64_t xr = max(x, 0);
        const T* row = (const T*)a.dy + (int64_t)r * a.n_out;
        if (whole) load8<T, true>(row, o0 + sc, a.n_out, wa);
        else load8<T, false>(row, o0 + sc, a.n_out, wa);
        if (PACKED) {
            wb = load8_packed(a.q + xr * a.n_in, c0 + sc, a.n_in);
            byte = a.scale[xr * a.groups + min(c0 + sc, a.n_in - 1) / 32];
        } else {
            const T* from = (const T*)a.x + xr * a.n_in;
            if (whole_x) load8<T, true>(from, c0 + sc, a.n_in, wx);
            else load8<T, false>(from, c0 + sc, a.n_in, wx);
        }
    };
    const int ao = 32 * (wave >> 1) + (lane & 31), bo = 32 * (wave & 1) + (lane & 31), k2 = lane >> 5;
    // bf16: 8 rows' values of a wavefront's column, from row k + 8 (lane / 32) on, four of them a read
    constexpr bool kBf16 = !PACKED && sizeof(T) == 2;
    constexpr int kPitch16 = 2 * kTile + 16;
    unsigned char* const A16 = (unsigned char*)A;
    unsigned char* const B16 = (unsigned char*)B;
    const int s16 = lane & 15, nl = 16 * ((lane >> 4) & 1) + 4 * (s16 & 3), kl = 8 * k2 + (s16 >> 2);
    auto columns = [&](const unsigned char* from, int k, int col) __attribute__((always_inline)) {
        const unsigned char* p = from + (k + kl) * kPitch16 + (col + nl) * 2;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)p);
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p + 4 * kPitch16));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    if (a.Rx == 0) last = first;        // no row has a source
    if (first < last) fetch(first);
    for (int r0 = first; r0 < last; r0 += kStep) {
        // a row without a source is zeros in both operands: nothing of it multiplies
        if constexpr (kBf16) {
            const u32x4 none = {0, 0, 0, 0};
            __syncthreads();
            *(u32x4*)(A16 + sr * kPitch16 + sc * 2) = on ? wa[0] : none;
            *(u32x4*)(B16 + sr * kPitch16 + sc * 2) = on ? wx[0] : none;
            __syncthreads();
            if (r0 + kStep < last) fetch(r0 + kStep);
#pragma unroll
            for (int k = 0; k < kStep; k += 16)
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(columns(A16, k, 32 * (wave >> 1)),
                                                              columns(B16, k, 32 * (wave & 1)), acc, 0, 0, 0);
            continue;
        }
        float va[8], vb[8];
#pragma unroll
        for (int i = 0; i < 8 / E; ++i) {
            Chunk<T>::open(wa[i], va + i * E);
            if (!PACKED) Chunk<T>::open(wx[i], vb + i * E);
        }
        const float step = on ? __uint_as_float(byte << 23) : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            va[i] = on ? va[i] : 0.0f;
            if (PACKED) vb[i] = (float)(int8_t)(wb >> (8 * i)) * step;
            else vb[i] = on ? vb[i] : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            *(f32x4*)(A + sr * kTilePitch + sc + i) = f32x4{va[i], va[i + 1], va[i + 2], va[i + 3]};
            *(f32x4*)(B + sr * kTilePitch + sc + i) = f32x4{vb[i], vb[i + 1], vb[i + 2], vb[i + 3]};
        }
        __syncthreads();
        if (r0 + kStep < last) fetch(r0 + kStep);
#pragma unroll
        for (int k = 0; k < kStep; k += 2)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(A[(k + k2) * kTilePitch + ao], B[(k + k2) * kTilePitch + bo],
                                                       acc, 0, 0, 0);
    }
    // lane l holds column l % 32 and rows 8 (v / 4) + 4 (l / 32) + v % 4
    const int c = c0 + bo;
    if (c >= a.n_in) return;
    const int o = o0 + 32 * (wave >> 1) + 4 * k2;
    float* to = (a.S > 1 ? a.part : a.dW) + ((int64_t)blockIdx.z * a.n_out + o) * a.n_in + c;
#pragma unroll
    for (int v = 0; v < 16; ++v)
        if (o + 8 * (v / 4) + v % 4 < a.n_out) to[(int64_t)(8 * (v / 4) + v % 4) * a.n_in] = acc[v];
}

// Few outputs from rows that are not packed: 32 x 32 per workgroup, each of its four wavefronts takes every
// fourth 16 rows on v_mfma_f32_16x16x4_f32, straight from memory (a lane loads two columns of a row; MFMA
// (i, j) has the i-th of the lanes' columns of dy and the j-th of x's), the next 16 rows in flight, and their
// sums meet in LDS, in order.  The chain of a row step is short then and there are four times as many
// workgroups (the rule that takes it says what it gains).
constexpr int kThin = 32;
template <typename T>
__global__ void __launch_bounds__(256) wgrad_thin_kernel(WgradArgs a) {
    typedef typename Chunk<T>::Bits Bits;
    __shared__ f32x4 sums[4][4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int at = lane & 15, grp = lane >> 4;
    const int o0 = (int)blockIdx.y * kThin, c0 = (int)blockIdx.x * kThin, e = (int)blockIdx.z;
    int first, last;
    expert_rows(a, e, &first, &last);
    if (a.Rx == 0) last = first;
    // this lane's columns 2 at and 2 at + 1; those past the matrix read its last one and are not stored
    int oc[2], cc[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        oc[j] = min(o0 + 2 * at + j, a.n_out - 1);
        cc[j] = min(c0 + 2 * at + j, a.n_in - 1);
    }
    struct Set {
        Bits y[4][2], x[4][2];      // of rows 4 grp + 0 .. 3
        bool on[4];
    };
    auto load = [&](Set& s, int r0) __attribute__((always_inline)) {
        int src[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + 4 * grp + i;
            src[i] = r < last ? source_row(a, r) : -1;
            s.on[i] = src[i] >= 0;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Bits* y = (const Bits*)a.dy + (int64_t)min(r0 + 4 * grp + i, last - 1) * a.n_out;
            const Bits* x = (const Bits*)a.x + (int64_t)max(src[i], 0) * a.n_in;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                s.y[i][j] = y[oc[j]];
                s.x[i][j] = x[cc[j]];
            }
        }
    };
    f32x4 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto mul = [&](const Set& s) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float y[2], x[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // (a row without a source is zeros in both operands: nothing of it multiplies)
                y[j] = s.on[q] ? Act<T>::to_f32(__builtin_bit_cast(T, s.y[q][j])) : 0.0f;
                x[j] = s.on[q] ? Act<T>::to_f32(__builtin_bit_cast(T, s.x[q][j])) : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[i], x[j], acc[i][j], 0, 0, 0);
        }
    };
    Set s0, s1;
    int r = first + 16 * wave;
    if (r < last) load(s0, r);
    for (; r < last; r += 128) {
        const bool two = r + 64 < last;
        if (two) load(s1, r + 64);
        mul(s0);
        if (r + 128 < last) load(s0, r + 128);
        if (two) mul(s1);
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) sums[wave][b][lane] = acc[b / 2][b % 2];
    __syncthreads();
    // block b = (i, j) of wavefront b: lane l holds outputs 2 (4 (l / 16) + v) + i of column 2 (l % 16) + j
    f32x4 v = sums[0][wave][lane];
#pragma unroll
    for (int q = 1; q < 4; ++q) v += sums[q][wave][lane];
    const int c = c0 + 2 * at + wave % 2;
    if (c >= a.n_in) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int o = o0 + 2 * (4 * grp + q) + wave / 2;
        if (o < a.n_out) a.dW[((int64_t)e * a.n_out + o) * a.n_in + c] = v[q];
    }
}

// bf16 dy on MFMA (n_out a multiple of 8, n_in of 16, or of 8 where x is not packed): 256 x 256 outputs
// at a time, eight
// wavefronts of 64 x 128 on v_mfma_f32_32x32x16_bf16, K (the rows) in steps of 32 through a
// ring of four LDS stages.  Both operands lie along K rows of 512 bytes (the tile's columns
// as bf16) and are read as fragments by the transposing LDS read.  dy is copied into LDS
// directly by four of the wavefronts; the other four load the packed rows (half of dy's
// bytes), turn them into bf16 in registers, among their MFMAs, and write them, or copy the rows of
// x as the first four copy dy's.
// Row indexes go to LDS a few thousand at a time; a row past the last one or without a source
// is zeros in both operands, since a zero of one would turn an infinity of the other into NaN.
// A workgroup goes through several tiles of the same rows of dy: the row indexes stay, and
// the next tile's first steps are fetched before this one's outputs are stored.
// 128 experts of 1536 x 2048 over 131072 rows take 955-990 us (833-863 TFLOP/s; the library's
// product of that size and layout, with one shared output, reaches 822): 775 in the steps, the
// MFMA units 42-48 % busy at the clock that the power limit leaves, and 8 us per tile for its
// 256 KB of outputs.  Two workgroups a CU with tiles of 256 x 128, so that one stores while
// the other multiplies, took 1120.
constexpr int BM = 256, BN = 256;
constexpr int kBK = 32;
constexpr int WM = 64, WN = 128;
constexpr int MI = WM / 32, NJ = WN / 32;
constexpr int kMfmaThreads = 512;
constexpr int kPitch = 512;                 // bytes of a K row
constexpr int kOpB = kBK * kPitch;
constexpr int kStageB = 2 * kOpB;
constexpr int kStages = 4;
constexpr int kCopies = 4;                  // per dy wavefront and step
constexpr int kRowsHeld = 8128;             // row indexes held in LDS
constexpr int kNumXcd = 8;
constexpr uint32_t kNoRow = 0xffffffffu;

__device__ __attribute__((aligned(16))) const bf16_t kZeros[8] = {};

template <int n>
__device__ __forceinline__ void wait_vmcnt() {
    static_assert(n >= 0 && n < 64, "vmcnt field");
    __builtin_amdgcn_s_waitcnt(0x0f70 | (n & 15) | ((n >> 4) << 14));
}

// Byte j of q as a signed number, in one instruction.  (A cast is left as shifts, bit-field
// extracts and conversions, and the kernel below spills 320 registers; with the sign carried as
// 128 and taken off again it takes 1006 us where this, run in turn, takes 960: 128 experts of 1536 x
// 2048.)
template <int j>
__device__ __forceinline__ float signed_byte(uint32_t q) {
    float f;
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_%2"
        : "=v"(f) : "v"(q), "n"(j));
    return f;
}

// 8 packed values as bf16 (exact).  The sign comes in before the step does: 128 of the largest
// step, 2^121, are no number any more.
__device__ __forceinline__ u32x4 open_packed(uint32_t q0, uint32_t q1, float step) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t q = i ? q1 : q0;
        const uint32_t w0 = __float_as_uint(signed_byte<0>(q) * step);
        const uint32_t w1 = __float_as_uint(signed_byte<1>(q) * step);
        const uint32_t w2 = __float_as_uint(signed_byte<2>(q) * step);
        const uint32_t w3 = __float_as_uint(signed_byte<3>(q) * step);
        // the upper halves of the fp32 values, which have no lower bits
        r[2 * i] = __builtin_amdgcn_perm(w1, w0, 0x07060302u);
        r[2 * i + 1] = __builtin_amdgcn_perm(w3, w2, 0x07060302u);
    }
    return r;
}

// The tiles of one work item, for the wavefronts that load packed rows, dy or the rows of x:
// instances, so that what the one kind keeps in flight is no merge of both kinds' registers.
enum { LOAD_DY = 0, LOAD_PACKED = 1, LOAD_X = 2 };
template <int LOADS>
__device__ __forceinline__ void wgrad_tiles(const WgradArgs& a, unsigned char* lds, uint32_t* src,
                                            int* s_bad) {
    constexpr bool PACKS = LOADS == LOAD_PACKED;
    // Work items (expert, slice, row tile, group of column tiles).  Many experts are dealt to the
    // XCDs round-robin and an expert's items run on one XCD, whose L2 then holds its rows; of
    // few experts (split) each XCD takes an eighth of each one's items, a contiguous range,
    // every expert's ranges beginning at another XCD.
    const int nct = (a.n_in + BN - 1) / BN;
    const int ngr = (nct + a.G - 1) / a.G;
    const int nrt = (a.n_out + BM - 1) / BM;
    const int per_e = nrt * ngr * a.S;
    const int xcd = blockIdx.x % kNumXcd, local = blockIdx.x / kNumXcd;
    int slot, item;
    if (a.split) {
        const int each = (per_e + kNumXcd - 1) / kNumXcd;
        slot = local / each;
        item = (xcd + slot) % kNumXcd * each + local % each;
    } else {
        slot = xcd + kNumXcd * (local / per_e);
        item = local % per_e;
    }
    if (slot >= a.N || item >= per_e) return;
    const int expert = __builtin_amdgcn_readfirstlane(a.order ? a.order[slot] : slot);
    const int slice = item / (nrt * ngr);
    const int rt = item % (nrt * ngr) / ngr;
    const int ct0 = item % ngr * a.G;
    const int ct1 = min(nct, ct0 + a.G);
    int row0, last;
    expert_rows(a, expert, &row0, &last);
    slice_rows(a, slice, &row0, &last);
    row0 = __builtin_amdgcn_readfirstlane(row0);
    const int klen = __builtin_amdgcn_readfirstlane(last) - row0;

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave >> 1, wc = wave & 1;    // 64-row and 128-column block of the tile
    const int krow = 8 * (wave & 3);            // first K row of a step that it loads

    // dy: copy i moves K rows krow + 2 i (lanes 0-31) and + 1 (lanes 32-63); chunk c of K row
    // kr is stored at c ^ 4 (kr & 3).  (Columns past the matrix read its first: they reach
    // only outputs that are not stored.)
    const int hi = lane >> 5;
    uint32_t doff[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = 8 * ((lane & 31) ^ (4 * (hi + 2 * i)));
        doff[i] = 2u * (uint32_t)(hi * a.n_out + (rt * BM + c < a.n_out ? c : 0));
    }
    const bf16_t* const dy = (const bf16_t*)a.dy + (int64_t)(row0 + krow) * a.n_out + rt * BM;
    // packed rows: piece p of a lane is 16 columns of K row krow + 4 p + lane / 16, stored as
    // chunks pchunk and pchunk ^ 1
    const int prow = lane >> 4;
    const int pchunk = (2 * (lane & 15)) ^ (4 * prow);

    // MFMA fragments by two transposing reads each
    const int s16 = lane & 15, g4 = lane >> 4;
    const int nl = 16 * (g4 & 1) + 4 * (s16 & 3);
    const int kl = 8 * (g4 >> 1) + (s16 >> 2);
    const int tsw = (nl >> 3) ^ (4 * (kl & 3));
    auto tr_pos = [&](int cb) { return kl * kPitch + ((((cb >> 3) ^ tsw)) << 4) + ((nl & 4) << 1); };
    int a_pos[MI], b_pos[NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i) a_pos[i] = tr_pos(wr * WM + i * 32);
#pragma unroll
    for (int j = 0; j < NJ; ++j) b_pos[j] = kOpB + tr_pos(wc * WN + j * 32);

    auto barrier = [&]() __attribute__((always_inline)) {
        // a plain barrier: __syncthreads() would wait for every load in flight
        __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    };
    using C0 = std::integral_constant<int, 0>;
    using C1 = std::integral_constant<int, 1>;

    int kc = 0, nh = 0, whole = 0;      // the rows whose indexes are in LDS: first, steps, whole steps
    auto hold_rows = [&](int first) __attribute__((always_inline)) {
        kc = first;
        const int clen = min(kRowsHeld, klen - kc);
        nh = (clen + kBK - 1) / kBK;
        bool none = false;
        for (int i = tid; i < nh * kBK; i += kMfmaThreads) {
            const uint32_t r = i < clen ? (uint32_t)source_row(a, row0 + kc + i) : kNoRow;
            none |= i < clen && r == kNoRow;
            src[i] = r;
        }
        const int bad = __ballot(none) != 0;
        if (lane == 0) s_bad[wave] = bad;
        barrier();
        int any = 0;
#pragma unroll
        for (int w = 0; w < kMfmaThreads / 64; ++w) any |= s_bad[w];
        // steps before this one have a source for every row
        whole = __builtin_amdgcn_readfirstlane(any) ? 0 : clen / kBK;
    };
    auto stage_of = [&](int h) __attribute__((always_inline)) { return lds + (h % kStages) * kStageB; };
    // Copy i of a step, dy's or rows of x to the same places of the other operand, each half wavefront's row
    // by its index.  WHOLE: every row of the step has a source.
    const uint32_t lds0 = lds_address(lds) + (LOADS == LOAD_X ? kOpB : 0) + krow * kPitch;
    auto row_of = [&](int h, int i) __attribute__((always_inline)) { return src[h * kBK + krow + 2 * i + hi]; };
    auto copy_row = [&](auto WHOLE, int ct, int h, int i, uint32_t row) __attribute__((always_inline)) {
        const uint32_t to = lds0 + (h % kStages) * kStageB + i * 1024;
        if (LOADS == LOAD_X) {
            const int c = ct * BN + 8 * ((lane & 31) ^ (4 * (hi + 2 * (i & 1))));
            const bf16_t* p = (const bf16_t*)a.x + (uint64_t)row * (uint32_t)a.n_in + (c < a.n_in ? c : 0);
            dma16_to(decltype(WHOLE)::value || row != kNoRow ? p : (const bf16_t*)kZeros, to);
        } else {
            const bf16_t* p = dy + (int64_t)(kc + h * kBK + 2 * i) * a.n_out;
            if (decltype(WHOLE)::value) dma16_to(p, doff[i & 1], to);
            else dma16_to(row != kNoRow ? (const unsigned char*)p + doff[i & 1] : (const unsigned char*)kZeros, to);
        }
    };
    // Packed pieces in flight: two steps' worth.  Nothing is computed from them on arrival
    // (a row that is none reads row 0, and its scale is masked when it is opened) and a step past
    // the end reads the last one again, so that the wait for a piece leaves the later ones
    // in flight.
    u32x4 q[2][2];
    uint32_t sb[2][2], mask[2][2];
    auto load_packed = [&](auto S_, int ct, int h) __attribute__((always_inline)) {
        constexpr int S = decltype(S_)::value;
        int c = ct * BN + 16 * (lane & 15);
        c = c < a.n_in ? c : 0;             // (as dy's columns)
        const int k0 = min(h, nh - 1) * kBK + krow + prow;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const uint32_t t = src[k0 + 4 * p];
            const uint32_t row = t == kNoRow ? 0u : t;
            mask[S][p] = t == kNoRow ? 0u : 255u << 23;
            q[S][p] = *(const u32x4*)(a.q + (uint64_t)row * (uint32_t)a.n_in + c);
            sb[S][p] = a.scale[(uint64_t)row * (uint32_t)a.groups + c / 32];
        }
    };
    // quarter i of a step's packed values
    auto write_packed = [&](auto S_, int h, int i) __attribute__((always_inline)) {
        constexpr int S = decltype(S_)::value;
        const int p = i >> 1;
        unsigned char* dst = stage_of(h) + kOpB + (krow + 4 * p + prow) * kPitch;
        const float step = __uint_as_float((sb[S][p] << 23) & mask[S][p]);
        if (i & 1) *(u32x4*)(dst + (pchunk ^ 1) * 16) = open_packed(q[S][p][2], q[S][p][3], step);
        else *(u32x4*)(dst + pchunk * 16) = open_packed(q[S][p][0], q[S][p][1], step);
    };
    // at most n steps' copies may still be in flight
    auto wait_steps = [&](int n) __attribute__((always_inline)) {
        if (n >= 3) wait_vmcnt<3 * kCopies>();
        else if (n == 2) wait_vmcnt<2 * kCopies>();
        else if (n == 1) wait_vmcnt<kCopies>();
        else wait_vmcnt<0>();
    };
    // The first steps, in two parts, with the stores of the tile before in between: dy's steps
    // 0..3 into the stages, the packed steps 0 and 1 into registers; then these are written and
    // 2 and 3 fetched.
    auto fetch = [&](int ct) __attribute__((always_inline)) {
        if (PACKS) {
            load_packed(C0{}, ct, 0);
            load_packed(C1{}, ct, 1);
        } else {
            for (int h = 0; h < min(nh, kStages); ++h) {
#pragma unroll
                for (int i = 0; i < kCopies; ++i) copy_row(C0{}, ct, h, i, row_of(h, i));
            }
        }
    };
    auto start = [&](int ct) __attribute__((always_inline)) {
        if (PACKS) {
#pragma unroll
            for (int i = 0; i < 4; ++i) write_packed(C0{}, 0, i);
            if (nh > 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) write_packed(C1{}, 1, i);
            }
            load_packed(C0{}, ct, 2);
            load_packed(C1{}, ct, 3);
        } else {
            wait_steps(min(nh, kStages) - 1);
        }
        barrier();
    };

    if (klen > 0) {
        hold_rows(0);
        fetch(ct0);
    }
    for (int ct = ct0; ct < ct1; ++ct) {
        // blocks past the matrix: their wavefronts only load
        const bool active = rt * BM + wr * WM < a.n_out && ct * BN + wc * WN < a.n_in;
        f32x16 acc[MI][NJ];
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

        for (int k = 0; k < klen; k += kRowsHeld) {
            if (klen > kRowsHeld && (k > 0 || ct > ct0)) {
                barrier();           // the last readers of src and of the stages are done
                hold_rows(k);
                fetch(ct);
            }
            start(ct);

            bf16x8 fa[2][MI], fb[2][NJ];
            auto tr_frag = [&](const unsigned char* p) __attribute__((always_inline)) {
                const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)p);
                const v4s hi4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p + 4 * kPitch));
                return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi4, 0, 1, 2, 3, 4, 5, 6, 7));
            };
            // MFMAs on fragment set S, among them the reads of sub-step ks of a stage into the
            // other set, and part(0..3)
            auto phase = [&](auto S_, int stage, int ks, auto part) __attribute__((always_inline)) {
                constexpr int S = decltype(S_)::value;
                const unsigned char* base = lds + stage * kStageB + ks * (16 * kPitch);
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < MI; ++i)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[S][i], fb[S][j], acc[i][j], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if (j == 0) {
                        fa[S ^ 1][0] = tr_frag(base + a_pos[0]);
                        fa[S ^ 1][1] = tr_frag(base + a_pos[1]);
                    } else if (j < 3) {
                        fb[S ^ 1][2 * j - 2] = tr_frag(base + b_pos[2 * j - 2]);
                        fb[S ^ 1][2 * j - 1] = tr_frag(base + b_pos[2 * j - 1]);
                    }
                    part(j);
                }
            };
            // Step h.  Behind the barrier between its sub-steps every wavefront holds the step's
            // last fragments, so its stage takes dy's step h + kStages; the packed step h + 2 goes
            // into a stage whose last reader was a step earlier at least, and h + 4 is fetched.
            // (Past the last step the reads fetch an old stage; unused.)
            auto step = [&](auto S_, int h) __attribute__((always_inline)) {
                uint32_t rows[kCopies];
                if (!PACKS && h + kStages < nh) {
#pragma unroll
                    for (int i = 0; i < kCopies; ++i) rows[i] = row_of(h + kStages, i);
                }
                if (active) phase(C0{}, h % kStages, 1, [](int) __attribute__((always_inline)) {});
                if (!PACKS) wait_steps(min(nh - 1, h + kStages - 1) - (h + 1));
                barrier();
                auto part = [&](int j) __attribute__((always_inline)) {
                    if (PACKS) {
                        write_packed(S_, h + 2, j);     // (past the end into a stage nobody reads)
                        if (j == 3) load_packed(S_, ct, h + 4);
                    } else if (h + kStages < nh) {
                        copy_row(C0{}, ct, h + kStages, j, rows[j]);
                    }
                };
                if (active) {
                    phase(C1{}, (h + 1) % kStages, 0, part);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) part(j);
                }
            };
            if (active) {
#pragma unroll
                for (int i = 0; i < MI; ++i) fa[0][i] = tr_frag(lds + a_pos[i]);
#pragma unroll
                for (int j = 0; j < NJ; ++j) fb[0][j] = tr_frag(lds + b_pos[j]);
            }
            int h = 0;
            if (!PACKS) {
                // Steps whose copies are of whole steps: no test per copy, and the rows' indexes are read a sub-step
                // ahead (rows of x, 128 experts of 1024 rows, 2048 x 768: 543 -> 480 us, 1536 x 2048: 1007 -> 907).
                if (active) {
                    for (; h + kStages < whole; ++h) {
                        uint32_t rows[kCopies];
#pragma unroll
                        for (int i = 0; i < kCopies; ++i) rows[i] = LOADS == LOAD_X ? row_of(h + kStages, i) : 0u;
                        phase(C0{}, h % kStages, 1, [](int) __attribute__((always_inline)) {});
                        wait_vmcnt<2 * kCopies>();
                        barrier();
                        phase(C1{}, (h + 1) % kStages, 0, [&](int j) __attribute__((always_inline)) {
                            copy_row(C1{}, ct, h + kStages, j, rows[j]);
                        });
                    }
                }
                for (; h < nh; ++h) step(C0{}, h);
            } else {
                for (; h + 1 < nh; h += 2) {
                    step(C0{}, h);
                    step(C1{}, h + 1);
                }
                if (h < nh) step(C0{}, h);
            }
        }
        barrier();          // (no wavefront reads a stage any more: all hold the last step's fragments)
        if (ct + 1 < ct1 && klen > 0 && klen <= kRowsHeld) fetch(ct + 1);

        // Lane l holds column l % 32 of each 32-column block and rows 8 (v / 4) + 4 (l / 32) + v % 4
        // of each 32-row block: a store writes whole 128-byte pieces of two rows, straight from
        // the accumulators (128 experts of 1536 x 2048: 1002 -> 973 us against rows of 256 bytes
        // put together in LDS; past the caches 976).
        if (active) {
            const int rows_left = a.n_out - rt * BM - wr * WM;      // multiples of 8 and 16
            const int cols_left = a.n_in - ct * BN - wc * WN;
            float* const out = (a.S > 1 ? a.part : a.dW) + ct * BN + wc * WN + (lane & 31) +
                ((int64_t)(slice * a.N + expert) * a.n_out + rt * BM + wr * WM + 4 * hi) * a.n_in;
            if (rows_left >= WM && cols_left >= WN) {
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        float* to = out + (int64_t)(i * 32 + 8 * (v / 4) + v % 4) * a.n_in;
#pragma unroll
                        for (int j = 0; j < NJ; ++j) to[j * 32] = acc[i][j][v];
                    }
            } else {
                // (one condition per lane and column block, one for all lanes per 8 rows)
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    if (j * 32 + (lane & 31) >= cols_left) continue;
#pragma unroll
                    for (int i = 0; i < MI; ++i)
#pragma unroll
                        for (int v0 = 0; v0 < 16; v0 += 4) {
                            if (i * 32 + 2 * v0 >= rows_left) continue;
#pragma unroll
                            for (int v = v0; v < v0 + 4; ++v)
                                out[(int64_t)(i * 32 + 2 * v0 + v - v0) * a.n_in + j * 32] = acc[i][j][v];
                        }
                }
            }
        }
    }
}

template <bool PACKED>
__global__ void __launch_bounds__(kMfmaThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
wgrad_mfma_kernel(WgradArgs a) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kStages * kStageB];
    __shared__ __attribute__((aligned(16))) uint32_t src[kRowsHeld];
    __shared__ int s_bad[kMfmaThreads / 64];
    if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) >= 4)
        wgrad_tiles<PACKED ? LOAD_PACKED : LOAD_X>(a, lds, src, s_bad);
    else
        wgrad_tiles<LOAD_DY>(a, lds, src, s_bad);
}

// dW = the slices' partial sums in slice order, four elements per thread
__global__ void __launch_bounds__(256) wgrad_join_kernel(const float* part, int64_t n, int S, float* dW) {
    typedef f32x4 f32x4_any __attribute__((aligned(4)));        // a slice starts at any float
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i + 4 <= n) {
        f32x4 v = *(const f32x4_any*)(part + i);
#pragma unroll 8
        for (int s = 1; s < S; ++s) v += *(const f32x4_any*)(part + s * n + i);
        *(f32x4*)(dW + i) = v;
    } else {
        for (int64_t j = i; j < n; ++j) {
            float v = part[j];
            for (int s = 1; s < S; ++s) v += part[s * n + j];
            dW[j] = v;
        }
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
    if ((int64_t)d.N * d.n_out * d.n_in > (int64_t)1 << 36)
        return fail(PR2_ERR_UNSUPPORTED, "N n_out n_in > 2^36");
    return PR2_OK;
}

bool mfma_ok(const pr2_wgrad_desc& d, bool packed) {
    return d.act_dtype == PR2_BF16 && d.n_out % 8 == 0 && d.n_in % (packed ? 16 : 8) == 0;
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Output tiles over all experts.
int64_t wgrad_tile_count(const pr2_wgrad_desc& d, int tile) {
    return ceil_div(d.n_out, tile) * ceil_div(d.n_in, tile) * d.N;
}

// Slices of the rows: where the output tiles leave the chip idle, as many as are expected to
// take the least time, up to what fills it once (one 256 x 256 tile per CU, or four of 64 x 64).
// More slices take fewer steps of 32 rows each, but write and read partial sums and need the
// join.  In us, as measured: a step of a chip full of tiles 0.9 and 1.2, the join's launch 6, its
// traffic and the slices' writes at 6.5 TB/s.  Against a fixed 256 and 128 rows a slice at
// least, with the packing: 700 rows of 2048 x 2048 outputs 33.0 -> 30.3, 32768 of 64 x 128
// 48.6 -> 26.1, 8192 of 512 x 512 35.7 -> 31.0, 20 fp32 experts of 33 x 50 25.9 -> 13.6.
constexpr int kCus = 256;
constexpr int kMaxSlices = 64;
struct SliceCost {
    int64_t steps;          // steps of 32 rows of a tile that is not sliced
    float step, join, part; // us: a step, the join's launch, a slice's traffic
    int most;               // slices that can pay; does not decrease with the rows
};
SliceCost slice_cost(const pr2_wgrad_desc& d, bool packed) {
    const bool big = mfma_ok(d, packed);
    const int64_t tiles = wgrad_tile_count(d, big ? BM : kTile);
    SliceCost c{};
    c.steps = ceil_div(d.R / d.N, kBK);
    c.step = big ? 0.9f : 1.2f;
    c.join = 6.0f;
    c.part = 2.0f * sizeof(float) * (float)((int64_t)d.N * d.n_out * d.n_in) / 6.5e6f;
    const int64_t fill = std::min<int64_t>({(big ? kCus : 4 * kCus) / tiles, c.steps, kMaxSlices});
    const float whole = c.step * (float)c.steps;
    c.most = 1;
    while (c.most < fill && c.join + (float)(c.most + 1) * c.part < whole) ++c.most;
    return c;
}
int wgrad_slices(const pr2_wgrad_desc& d, bool packed) {
    const SliceCost c = slice_cost(d, packed);
    int best = 1;
    float least = c.step * (float)c.steps;
    for (int s = 2; s <= c.most; ++s) {
        const float t = c.step * (float)ceil_div(d.R / d.N, (int64_t)s * kBK) + c.join + (float)s * c.part;
        if (t < least) {
            least = t;
            best = s;
        }
    }
    return best;
}

// Column tiles per workgroup: two where that leaves each CU eight workgroups.
int wgrad_group(const pr2_wgrad_desc& d) {
    return wgrad_tile_count(d, BM) >= 16 * kCus ? 2 : 1;
}

// Experts from which on one runs on one XCD: 2, 4, 9, 25 and 33 of them took 53, 135, 107, 174 and
// 400 us that way and 30, 80, 79, 154 and 366 on all XCDs, 64 and 128 took 705 and 975 against 737
// and 1025 (1536 x 2048 outputs, 64: 2816, 2: 2288 x 1376).
constexpr int kManyExperts = 64;

// Whether longest experts first is worth its launch of 5 us: not where all work items run at
// once, and not where the longest expert could take little longer than that (2 experts of 2288 x
// 1376 over 89 rows 16.3 -> 14.2 us without, 25 of 736 x 1600 over 312 32.7 -> 30.2).
bool order_pays(const pr2_wgrad_desc& d, int64_t items) {
    return d.N > 1 && d.N * items > kCus && d.R > 512;
}

// Few rows an expert and few outputs: 7 experts of 135 x 203 over 175 rows each 8.7 -> 6.2 us, one of 32 x 32 over
// 175 9.5 -> 6.2 (over 1226 9.7 -> 15.1), 7 of 400 x 390 over 175 13.3 -> 11.6, of 1001 x 999 41 -> 50.  In bf16,
// whose 64 x 64 tiles are faster, 8.4 -> 7.4 and 8.4 -> 7.5, but 9.4 -> 13.0.
bool thin_ok(const pr2_wgrad_desc& d, bool packed) {
    return !packed && d.R > 0 && !mfma_ok(d, packed) && d.R <= 512 * (int64_t)d.N &&
           wgrad_tile_count(d, kThin) <= (d.act_dtype == PR2_BF16 ? 1 : 5) * kCus;
}

struct WgradWs {
    int* order;
    float* part;
    size_t bytes;
};

WgradWs wgrad_ws(const pr2_wgrad_desc& d, void* base) {
    WgradWs w{};
    char* p = base ? (char*)(((uintptr_t)base + 255) & ~(uintptr_t)255) : nullptr;
    const size_t order = (sizeof(int) * (size_t)d.N + 255) & ~(size_t)255;
    // not the slices of these rows alone: fewer rows can have more (nor of one form of x: they share
    // the size)
    const int S = std::max(slice_cost(d, true).most, slice_cost(d, false).most);
    w.order = (int*)p;
    w.part = (float*)(p ? p + order : nullptr);
    w.bytes = order + (S > 1 ? sizeof(float) * (size_t)S * d.N * d.n_out * d.n_in : 0) + 256;
    return w;
}

hipError_t launch_wgrad(const pr2_wgrad_desc& d, WgradArgs a, const WgradWs& w, hipStream_t st) {
    const bool packed = a.q != nullptr;
    if (thin_ok(d, packed)) {
        LaunchScope scope("wgrad_thin", st);
        const dim3 grid((unsigned)ceil_div(d.n_in, kThin), (unsigned)ceil_div(d.n_out, kThin), d.N);
        if (d.act_dtype == PR2_BF16) hipLaunchKernelGGL(wgrad_thin_kernel<bf16_t>, grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL(wgrad_thin_kernel<float>, grid, dim3(256), 0, st, a);
        return hipGetLastError();
    }
    a.S = d.R > 0 ? wgrad_slices(d, packed) : 1;
    a.part = w.part;
    hipError_t e;
    if (d.R > 0 && d.Rx > 0 && mfma_ok(d, packed)) {
        a.G = wgrad_group(d);
        const int64_t items = ceil_div(d.n_out, BM) * ceil_div(ceil_div(d.n_in, BN), a.G) * a.S;
        a.split = d.N < kManyExperts;
        const int64_t grid = kNumXcd * (a.split ? ceil_div(items, kNumXcd) * d.N : items * ceil_div(d.N, kNumXcd));
        if (order_pays(d, items)) {
            e = launch_expert_order(a.offsets, d.N, w.order, st);
            if (e != hipSuccess) return e;
            a.order = w.order;
        }
        LaunchScope scope("wgrad_mfma", st);
        if (packed) hipLaunchKernelGGL(wgrad_mfma_kernel<true>, dim3((unsigned)grid), dim3(kMfmaThreads), 0, st, a);
        else hipLaunchKernelGGL(wgrad_mfma_kernel<false>, dim3((unsigned)grid), dim3(kMfmaThreads), 0, st, a);
    } else {
        // (column and row tiles apart, at most 2^14 each: together they can be more than a
        // dimension holds; N S <= 1024)
        const dim3 grid((unsigned)ceil_div(d.n_in, kTile), (unsigned)ceil_div(d.n_out, kTile), d.N * a.S);
        LaunchScope scope("wgrad_tile", st);
        const bool bf16 = d.act_dtype == PR2_BF16;
        if (bf16 && packed) hipLaunchKernelGGL((wgrad_tile_kernel<bf16_t, true>), grid, dim3(256), 0, st, a);
        else if (bf16) hipLaunchKernelGGL((wgrad_tile_kernel<bf16_t, false>), grid, dim3(256), 0, st, a);
        else if (packed) hipLaunchKernelGGL((wgrad_tile_kernel<float, true>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((wgrad_tile_kernel<float, false>), grid, dim3(256), 0, st, a);
    }
    e = hipGetLastError();
    if (e != hipSuccess || a.S == 1) return e;
    const int64_t n = (int64_t)d.N * d.n_out * d.n_in;
    LaunchScope scope("wgrad_join", st);
    hipLaunchKernelGGL(wgrad_join_kernel, dim3((unsigned)ceil_div(n, 1024)), dim3(256), 0, st, a.part,
                       n, a.S, a.dW);
    return hipGetLastError();
}

// x, or (packed) its packed form (q, scale)
pr2_status weight_grad(const pr2_wgrad_desc* desc, bool packed, const void* dy, const int8_t* q,
                       const uint8_t* scale, const void* x, const int32_t* offsets, const int32_t* route_of_row, float* dW, void* ws,
                       size_t ws_bytes, pr2_stream_t stream) {
    pr2_status s = check_wgrad(desc);
    if (s != PR2_OK) return s;
    const pr2_wgrad_desc& d = *desc;
    if (!dW) return fail(PR2_ERR_NULL, "dW is NULL");
    if ((uintptr_t)dW % 16) return fail(PR2_ERR_ALIGN, "dW is not 16-byte aligned");
    if (d.R > 0) {
        if (packed && (!dy || !q || !scale)) return fail(PR2_ERR_NULL, "dy, q and scale are required");
        if (!packed && (!dy || (!x && d.Rx > 0))) return fail(PR2_ERR_NULL, "dy and x are required");
        if ((uintptr_t)dy % 16 || (uintptr_t)q % 16 || (uintptr_t)scale % 16)
            return fail(PR2_ERR_ALIGN, "dy, q and scale must be 16-byte aligned");
        if (!offsets && d.N != 1) return fail(PR2_ERR_NULL, "offsets is NULL with N = %d > 1", d.N);
        if (!route_of_row && d.R > d.Rx)
            return fail(PR2_ERR_SHAPE, "R = %lld > Rx = %lld without route_of_row", (long long)d.R,
                        (long long)d.Rx);
        if ((uintptr_t)offsets % 4 || (uintptr_t)route_of_row % 4)
            return fail(PR2_ERR_ALIGN, "offsets or route_of_row is not 4-byte aligned");
        const size_t a1 = d.act_dtype == PR2_BF16 ? 2 : 4, out = sizeof(float) * (size_t)d.N * d.n_out * d.n_in;
        if (!packed && (share_memory(dW, out, dy, a1 * d.R * d.n_out) || share_memory(dW, out, x, a1 * d.Rx * d.n_in)))
            return fail(PR2_ERR_SHAPE, "dW overlaps dy or x");
        const size_t need = wgrad_ws(d, nullptr).bytes;
        if (need && !ws) return fail(PR2_ERR_NULL, "ws is NULL (need %zu bytes)", need);
        if (ws_bytes < need)
            return fail(PR2_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, need);
    }
    s = device_ready();
    if (s != PR2_OK) return s;
    drop_split_records(ws, ws_bytes);
    const hipStream_t st = (hipStream_t)stream;
    WgradArgs a{dy, q, scale, x, d.R ? offsets : nullptr, route_of_row, dW, d.R, d.Rx, d.n_out, d.n_in,
                d.N, d.k, (d.n_in + 31) / 32, nullptr, nullptr, 1, 1, false};
    const hipError_t e = launch_wgrad(d, a, wgrad_ws(d, ws), st);
    if (e != hipSuccess) return hip_fail(e, packed ? "weight_grad_packed launch" : "weight_grad launch");
    return ok();
}

}  // namespace
}  // namespace pr2

using namespace pr2;

extern "C" {

size_t pr2_weight_grad_workspace_bytes(const pr2_wgrad_desc* desc) {
    if (!desc || desc->N < 1 || desc->N > kMaxExperts || desc->R < 0 || desc->n_out < 1 ||
        desc->n_in < 1 || desc->n_out > (1 << 20) || desc->n_in > (1 << 20) || desc->R > 0x7fffffff)
        return 0;
    return wgrad_ws(*desc, nullptr).bytes;
}

pr2_status pr2_weight_grad(const pr2_wgrad_desc* desc, const void* dy, const void* x, const int32_t* offsets,
                           const int32_t* route_of_row, float* dW, void* ws, size_t ws_bytes,
                           pr2_stream_t stream) {
    if ((uintptr_t)x % 16) return fail(PR2_ERR_ALIGN, "x is not 16-byte aligned");
    return weight_grad(desc, false, dy, nullptr, nullptr, x, offsets, route_of_row, dW, ws, ws_bytes, stream);
}

pr2_status pr2_weight_grad_packed(const pr2_wgrad_desc* desc, const void* dy, const int8_t* q,
                                  const uint8_t* scale, const int32_t* offsets,
                                  const int32_t* route_of_row, float* dW, void* ws,
                                  size_t ws_bytes, pr2_stream_t stream) {
    return weight_grad(desc, true, dy, q, scale, nullptr, offsets, route_of_row, dW, ws, ws_bytes, stream);
}

}  // extern "C"
