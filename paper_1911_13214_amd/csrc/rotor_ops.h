// Shared by the operators of a language-model chain's stages (dropout,
// embedding, residual norm, cross entropy): element types, vector accesses
// and wave reductions.  Nothing here is part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rotor.h"

namespace rotor {

// Element types of a call: storage type T, arithmetic in float.
typedef __bf16 bf16;
typedef _Float16 f16;

template <int TYPE> struct ElemOf;
template <> struct ElemOf<ROTOR_F32> { typedef float T; };
template <> struct ElemOf<ROTOR_BF16> { typedef bf16 T; };
template <> struct ElemOf<ROTOR_F16> { typedef f16 T; };

inline int64_t elem_bytes(int32_t type) { return type == ROTOR_F32 ? 4 : 2; }
inline bool type_ok(int32_t type) { return type == ROTOR_F32 || type == ROTOR_BF16 || type == ROTOR_F16; }

// N adjacent elements, aligned to one element only: gfx950 loads and stores
// 16 bytes from any element-aligned address, so odd pitches need no kernel of
// their own.
template <typename T, int N> struct VecOf {
    typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

template <typename T, int N> __device__ inline void load_vec(const T *p, float (&f)[N])
{
    typedef typename VecOf<T, N>::V V;
    const V v = *(const V *)p;
#pragma unroll
    for (int k = 0; k < N; ++k)
        f[k] = (float)v[k];
}

template <typename T, int N> __device__ inline void store_vec(T *p, const float (&f)[N])
{
    typedef typename VecOf<T, N>::V V;
    V v;
#pragma unroll
    for (int k = 0; k < N; ++k)
        v[k] = (T)f[k];
    *(V *)p = v;
}

// The same for the first `n` of N elements (a row's end): the rest reads as 0
// and is not written.
template <typename T, int N> __device__ inline void load_some(const T *p, int n, float (&f)[N])
{
    if (n >= N) {
        load_vec(p, f);
        return;
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
        f[k] = k < n ? (float)p[k] : 0.f;
}

template <typename T, int N> __device__ inline void store_some(T *p, int n, const float (&f)[N])
{
    if (n >= N) {
        store_vec(p, f);
        return;
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (k < n)
            p[k] = (T)f[k];
}

__device__ inline float wave_sum(float v)
{
#pragma unroll
    for (int off = 32; off >= 1; off /= 2)
        v += __shfl_xor(v, off);
    return v;
}

// Calls f with the element type's tag: f(ElemOf<TYPE>{}).
template <typename F> inline void with_type(int32_t type, F f)
{
    if (type == ROTOR_F32)
        f(ElemOf<ROTOR_F32>{});
    else if (type == ROTOR_BF16)
        f(ElemOf<ROTOR_BF16>{});
    else
        f(ElemOf<ROTOR_F16>{});
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A grid of `blocks` workgroups, of up to 1024 threads each.  Along one index it
// holds fewer than 2^32 threads (more of them are not refused: the number
// wraps, and the rest never runs), so workgroups past 2^20 go along a second
// index; block_at is a workgroup's place, past `blocks` for some of the last.
constexpr int64_t kGridX = (int64_t)1 << 20;
inline bool grid_ok(int64_t blocks) { return blocks <= kGridX * 65535; }
inline dim3 grid_of(int64_t blocks)
{
    return blocks <= kGridX ? dim3((uint32_t)blocks) : dim3((uint32_t)kGridX, (uint32_t)ceil_div(blocks, kGridX));
}
__device__ inline int64_t block_at() { return blockIdx.x + (int64_t)blockIdx.y * gridDim.x; }
// The same where y is taken: the second index is z.
inline dim3 grid_of(int64_t blocks, int64_t y)
{
    const dim3 g = grid_of(blocks);
    return dim3(g.x, (uint32_t)y, g.y);
}
__device__ inline int64_t block_at_xz() { return blockIdx.x + (int64_t)blockIdx.z * gridDim.x; }

inline uint64_t round256(uint64_t x) { return (x + 255) / 256 * 256; }

// A matrix operand: pitch >= cols, pointer aligned to its elements, byte
// extent within 63 bits.
inline bool matrix_ok(const void *p, int64_t rows, int64_t cols, int64_t pitch, int64_t bytes)
{
    if (rows < 0 || cols < 1 || pitch < cols)
        return false;
    if (rows == 0)
        return true;
    return p && (uintptr_t)p % (uintptr_t)bytes == 0 &&
           (unsigned __int128)rows * (unsigned __int128)pitch * (unsigned __int128)bytes <
               ((unsigned __int128)1 << 62);
}

}  // namespace rotor
