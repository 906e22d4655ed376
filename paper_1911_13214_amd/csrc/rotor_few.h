// The cross entropy of few tokens (up to 64): W is read as it is, once
// forward and twice backward, straight into the matrix units' operands; what
// bounds it is that reading, and the writing of dW.
//
// A tile of 256 tokens would leave three quarters and more of its work
// unused here, and copies of W (transposed, or split into terms) would cost
// several times the reading.
#pragma once

#include "rotor_product.h"

namespace rotor {
namespace {

constexpr int kFew = 64;       // tokens
constexpr int kFewRows = 64;   // rows of W of a workgroup, 16 a wave
constexpr int kFewThreads = 256;
constexpr int kFewCols = 128;  // columns of dH of a workgroup

// Eight adjacent elements of a row from column k, 0 past its end.
template <typename T> __device__ inline typename VecOf<T, 8>::V row_piece(const T *row, int64_t k, int64_t cols)
{
    typedef typename VecOf<T, 8>::V V;
    V v;
    if (k + 8 <= cols) {
        v = *(const V *)(row + k);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = k + e < cols ? row[k + e] : (T)0.f;
    }
    return v;
}

// The terms of eight elements as operands of the matrix units.
template <typename T>
__device__ inline void terms_of(typename VecOf<T, 8>::V v,
                                typename Mfma<typename ProductOf<T>::P>::Frag (&t)[ProductOf<T>::kParts])
{
    if constexpr (ProductOf<T>::kParts == 1) {
        t[0] = v;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bf16 s[kTerms];
            split(v[e], s);
#pragma unroll
            for (int q = 0; q < kTerms; ++q)
                t[q][e] = s[q];
        }
    }
}

// Adds the product of two operands' terms.
template <typename P, int PARTS>
__device__ inline f32x4 multiply_terms(const typename Mfma<P>::Frag (&a)[PARTS],
                                       const typename Mfma<P>::Frag (&b)[PARTS], f32x4 c)
{
    if constexpr (PARTS == 1) {
        return Mfma<P>::run(a[0], b[0], c);
    } else {
#pragma unroll
        for (int s = 0; s < kTermProducts; ++s)
            c = Mfma<P>::run(a[term_a(s)], b[term_b(s)], c);
        return c;
    }
}

template <typename T> struct FewArgs {
    typedef typename ProductOf<T>::P P;
    const T *w;
    int64_t w_pitch, rows, cols;
    Operand<P> h;
    int tokens;
    const int64_t *targets;
    // forward: maximum and sum of exponentials of each 64 rows, [rows / 64][tokens]
    float2 *part;
    float *target_logit;
    // backward
    const float *lse, *grad, *scale;
    P *p;                        // [tokens][terms][p_seg], NULL: not wanted
    int64_t p_seg;
    const P *ht;                 // [cols][terms][32 * KS]: H transposed, 0 past the tokens
    T *dw;                       // NULL: not wanted
    int64_t dw_pitch;
};

// C: 16-token tiles.  A wave multiplies 16 rows of W with all tokens; loads
// of W and H are batched U steps of 32 columns deep.
template <typename T, int C, bool BACK>
__global__ __launch_bounds__(kFewThreads) void few_kernel(FewArgs<T> a)
{
    typedef typename ProductOf<T>::P P;
    typedef typename Mfma<P>::Frag Frag;
    constexpr int kParts = ProductOf<T>::kParts;
    constexpr int U = C == 1 ? 8 : C == 2 ? 4 : 2;
    constexpr int KS = C <= 2 ? 1 : 2;  // steps of 32 tokens
    constexpr int kPitch = 32 * KS + 8;
    __shared__ Soft soft[BACK ? 1 : 4][BACK ? 1 : 16 * C];
    __shared__ __attribute__((aligned(16))) P tile[BACK ? kParts : 1][BACK ? kFewRows : 1][kPitch];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    const int64_t v0 = (int64_t)blockIdx.x * kFewRows + wave * 16;
    const T *const row = a.w + (v0 + low < a.rows ? v0 + low : a.rows - 1) * a.w_pitch;
    const P *hrow[C];
#pragma unroll
    for (int c = 0; c < C; ++c)
        hrow[c] = a.h.p + (16 * c + low < a.tokens ? 16 * c + low : a.tokens - 1) * a.h.pitch;
    f32x4 acc[C];
#pragma unroll
    for (int c = 0; c < C; ++c)
        acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int64_t k0 = high * 8; k0 - high * 8 < a.cols; k0 += 32 * U) {
        typename VecOf<T, 8>::V raw[U];
        Frag hb[U][C][kParts];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t k = k0 + 32 * u;
            raw[u] = row_piece(row, k, a.cols);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int q = 0; q < kParts; ++q) {
                    if (k < a.cols)
                        hb[u][c][q] = *(const Frag *)(hrow[c] + q * a.h.seg + k);
                    else
                        hb[u][c][q] = Frag{};
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Frag t[kParts];
            terms_of<T>(raw[u], t);
#pragma unroll
            for (int c = 0; c < C; ++c)
                acc[c] = multiply_terms<P, kParts>(t, hb[u][c], acc[c]);
        }
    }
    // acc[c][e]: the logit of row v0 + 4 high + e and token 16 c + low
    const int64_t v = v0 + 4 * high;
    if constexpr (!BACK) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int j = 16 * c + low;
            const int64_t t = j < a.tokens ? a.targets[j] : -1;
            float top = -__builtin_inff();
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (v + e >= a.rows)
                    acc[c][e] = -__builtin_inff();
                else if (v + e == t)
                    a.target_logit[j] = acc[c][e];
                top = fmaxf(top, acc[c][e]);
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m = finite_or_0(top);
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum += __expf(acc[c][e] - m);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (high == 0)
                soft[wave][j] = Soft{top, sum};
        }
        __syncthreads();
        const int j = threadIdx.x;
        if (j < 16 * C && j < a.tokens) {
            Soft s = soft[0][j];
#pragma unroll
            for (int w = 1; w < 4; ++w)
                s = join(s, soft[w][j]);
            a.part[(int64_t)blockIdx.x * a.tokens + j] = make_float2(s.top, s.sum);
        }
    } else {
#pragma unroll
        for (int c = 0; c < 2 * KS; ++c) {
            const int j = 16 * c + low;
            const bool in = c < C && j < a.tokens;
            const float g = in ? a.grad[j] : 0.f, l = in ? a.lse[j] : 0.f;
            const int64_t t = in ? a.targets[j] : -1;
            typename VecOf<P, 4>::V out[kParts];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = __expf(acc[c < C ? c : 0][e] - l) - (v + e == t ? 1.f : 0.f);
                // a select: what a token without a target holds may be NaN
                x = g != 0.f && v + e < a.rows ? x * g : 0.f;
                if constexpr (kParts == 1) {
                    out[0][e] = (P)x;
                } else {
                    bf16 s[kTerms];
                    split(x, s);
#pragma unroll
                    for (int q = 0; q < kTerms; ++q)
                        out[q][e] = s[q];
                }
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    tile[q][wave * 16 + 4 * high + e][j] = out[q][e];
            }
            if (a.p && in)
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    *(typename VecOf<P, 4>::V *)(a.p + (j * kParts + q) * a.p_seg + v) = out[q];
        }
        if (!a.dw)
            return;
        __syncthreads();
        // dW of the workgroup's 64 rows: P is held in registers, H^T streams
        // through, a wave every fourth 16 columns
        Frag pb[4][KS][kParts];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    pb[r][s][q] = *(const Frag *)&tile[q][16 * r + low][32 * s + 8 * high];
        const float f = *a.scale;
        for (int64_t d0 = wave * 16; d0 < a.cols; d0 += 64) {
            Frag ha[KS][kParts];
            const P *src = a.ht + (d0 + low < a.cols ? d0 + low : a.cols - 1) * (kParts * 32 * KS) + 8 * high;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    ha[s][q] = *(const Frag *)(src + q * 32 * KS + 32 * s);
            const int64_t d = d0 + 4 * high;
            const int left = a.cols - d < 4 ? (int)(a.cols - d) : 4;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    o = multiply_terms<P, kParts>(ha[s], pb[r][s], o);
                const int64_t vr = (int64_t)blockIdx.x * kFewRows + 16 * r + low;
                const float x[4] = {o[0] * f, o[1] * f, o[2] * f, o[3] * f};
                if (vr < a.rows && left > 0)
                    store_some(a.dw + vr * a.dw_pitch + d, left, x);
            }
        }
    }
}

// Sums over a part of the vocabulary of P W, 128 columns a workgroup: 64 rows
// of W at a time go through LDS, which turns them (a wave reads eight rows of
// one column as an operand); the next 64 are loaded meanwhile.
template <typename T> struct FewSumArgs {
    typedef typename ProductOf<T>::P P;
    const T *w;
    int64_t w_pitch, rows, cols;
    const P *p;
    int64_t p_seg;
    int tokens;
    float *sum;  // [parts][tokens][sum_pitch]
    int64_t sum_pitch, tiles;  // tiles of 64 rows of one part
};

template <typename T, int C>
__global__ __launch_bounds__(kFewThreads) void few_sum_kernel(FewSumArgs<T> a)
{
    typedef typename ProductOf<T>::P P;
    typedef typename Mfma<P>::Frag Frag;
    constexpr int kParts = ProductOf<T>::kParts;
    __shared__ __attribute__((aligned(16))) P tile[kParts][kFewRows][kFewCols + 8];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    const int64_t c0 = (int64_t)blockIdx.x * kFewCols;
    const int64_t all = (a.rows + kFewRows - 1) / kFewRows;
    const int64_t t0 = (int64_t)blockIdx.y * a.tiles, t1 = t0 + a.tiles < all ? t0 + a.tiles : all;
    const int lr = threadIdx.x / 16, lc = threadIdx.x % 16 * 8;
    typename VecOf<T, 8>::V raw[4];
    auto load = [&](int64_t t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // rows past the end meet zeros of P, but have to be numbers
            const int64_t r = t * kFewRows + lr + 16 * i;
            raw[i] = row_piece(a.w + (r < a.rows ? r : a.rows - 1) * a.w_pitch, c0 + lc, r < a.rows ? a.cols : 0);
        }
    };
    f32x4 acc[2][C];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c)
            acc[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (t0 < t1)
        load(t0);
    for (int64_t t = t0; t < t1; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            Frag s[kParts];
            terms_of<T>(raw[i], s);
#pragma unroll
            for (int q = 0; q < kParts; ++q)
                *(Frag *)&tile[q][lr + 16 * i][lc] = s[q];
        }
        __syncthreads();
        if (t + 1 < t1)
            load(t + 1);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            Frag pb[C][kParts];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int j = 16 * c + low < a.tokens ? 16 * c + low : a.tokens - 1;
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    pb[c][q] = *(const Frag *)(a.p + (j * kParts + q) * a.p_seg + t * kFewRows + 32 * s + 8 * high);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                Frag wa[kParts];
#pragma unroll
                for (int q = 0; q < kParts; ++q)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        wa[q][e] = tile[q][32 * s + 8 * high + e][wave * 32 + 16 * i + low];
#pragma unroll
                for (int c = 0; c < C; ++c)
                    acc[i][c] = multiply_terms<P, kParts>(wa, pb[c], acc[i][c]);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t d = c0 + wave * 32 + 16 * i + 4 * high;  // sum_pitch is a multiple of 4
            const int j = 16 * c + low;
            if (j < a.tokens && d < a.sum_pitch)
                *(f32x4 *)(a.sum + ((int64_t)blockIdx.y * a.tokens + j) * a.sum_pitch + d) = acc[i][c];
        }
}

}  // namespace
}  // namespace rotor
