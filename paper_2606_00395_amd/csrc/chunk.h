// Rows of bf16 or fp32 elements in pieces of 16 bytes, at any element's address, and grids for
// any number of rows.
#pragma once

#include "common.h"

namespace pr2 {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// the same at any element's address: rows start where the caller's strides put them
typedef u32x4 u32x4_any __attribute__((aligned(2)));

// 16 bytes of a row: 8 bf16 or 4 fp32 elements
template <typename T> struct Chunk;
template <> struct Chunk<bf16_t> {
    static constexpr int E = 8;
    using Bits = uint16_t;
    static constexpr uint32_t kNegInf = 0xff80ff80u;
    __device__ __forceinline__ static void open(const u32x4& w, float* v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ static u32x4 close(const float* v) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = (uint32_t)f32_to_bf16(v[2 * i]) | ((uint32_t)f32_to_bf16(v[2 * i + 1]) << 16);
        return w;
    }
};
template <> struct Chunk<float> {
    static constexpr int E = 4;
    using Bits = uint32_t;
    static constexpr uint32_t kNegInf = 0xff800000u;
    __device__ __forceinline__ static void open(const u32x4& w, float* v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
    }
    __device__ __forceinline__ static u32x4 close(const float* v) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[i]);
        return w;
    }
};

// 16 bytes at any element's address; NT: not to be kept in the caches
template <bool NT>
__device__ __forceinline__ u32x4 load16(const void* p) {
    return NT ? __builtin_nontemporal_load((const u32x4_any*)p) : *(const u32x4_any*)p;
}
template <bool NT>
__device__ __forceinline__ void store16(void* p, const u32x4& w) {
    if (NT) __builtin_nontemporal_store(w, (u32x4_any*)p);
    else *(u32x4_any*)p = w;
}

// chunk c of a row of `full` whole chunks and `rem` more elements; past the end `pad`, two
// bf16 or one fp32 value
template <typename T, bool NT = false>
__device__ __forceinline__ u32x4 load_chunk(const T* row, int c, int full, int rem,
                                            uint32_t pad = 0) {
    constexpr int E = Chunk<T>::E;
    if (c < full) return load16<NT>(row + (int64_t)c * E);
    u32x4 w = {pad, pad, pad, pad};
    if (c == full) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (i >= rem) continue;
            const uint32_t b = __builtin_bit_cast(typename Chunk<T>::Bits, row[(int64_t)c * E + i]);
            if (E == 8) w[i / 2] = (i & 1) ? (w[i / 2] & 0xffffu) | (b << 16) : (w[i / 2] & 0xffff0000u) | b;
            else w[i] = b;
        }
    }
    return w;
}

// the bits of a chunk as they are
template <typename T, bool NT = false>
__device__ __forceinline__ void copy_chunk(T* row, int c, int full, int rem, const u32x4& w) {
    constexpr int E = Chunk<T>::E;
    if (c < full) {
        store16<NT>(row + (int64_t)c * E, w);
    } else if (c == full) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < rem)
                row[(int64_t)c * E + i] =
                    __builtin_bit_cast(T, (typename Chunk<T>::Bits)(E == 8 ? w[i / 2] >> (16 * (i & 1)) : w[i]));
    }
}

template <typename T, bool NT = false>
__device__ __forceinline__ void store_chunk(T* row, int c, int full, int rem, const float* v) {
    constexpr int E = Chunk<T>::E;
    if (c < full) {
        store16<NT>(row + (int64_t)c * E, Chunk<T>::close(v));
    } else if (c == full) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < rem) row[(int64_t)c * E + i] = Act<T>::from_f32(v[i]);
    }
}

// Grids of n workgroups (below 2^31) of `threads`, over two dimensions where one does not hold
// them: HIP cuts a dimension of more than 2^32 work-items off without an error.  A kernel asks
// block_number() which workgroup it is and has nothing to do from the n-th on.
inline dim3 wide_grid(int64_t n, int threads) {
    const int64_t most = ((int64_t)1 << 31) / threads;
    const int64_t x = n < most ? n : most;
    return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}
__device__ __forceinline__ uint32_t block_number() { return blockIdx.x + blockIdx.y * gridDim.x; }

}  // namespace pr2
