// The cross entropy of few tokens (up to 64; which calls: few_tokens): W is
// read as it is, once forward and twice backward, straight into the matrix
// units' operands; what bounds it is that reading, and the writing of dW.
//
// Tiles would leave most of their work unused here, which only a forward over
// many aligned rows hides, and copies of W (split into terms, or aligned) would
// cost several times the reading.
#pragma once

#include "rotor_product.h"

namespace rotor {
namespace {

constexpr int kFew = 64;       // tokens
constexpr int kFewRows = 64;   // rows of W of a workgroup of the sums
constexpr int kFewThreads = 256;
constexpr int kFewCols = 128;  // columns of dH of a workgroup

// 16-token tiles, and 16-row tiles of W a wave multiplies them with (what it
// reads of H it uses for both).
constexpr int few_tiles(int64_t tokens) { return tokens <= 16 ? 1 : tokens <= 32 ? 2 : 4; }
constexpr int few_row_tiles(int tiles) { return tiles == 1 ? 1 : 2; }

// Rows of W of a workgroup of the logits: its four waves take rows of their
// own, or, if those are fewer than two workgroups for each CU, a quarter of
// the columns of the same rows each.
constexpr int few_rows(int64_t tokens, int64_t rows)
{
    const int own = 16 * few_row_tiles(few_tiles(tokens));
    return (rows + 4 * own - 1) / (4 * own) >= 512 ? 4 * own : own;
}

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
    // forward: maximum and sum of exponentials of each workgroup's rows, [workgroups][tokens]
    float2 *part;
    float *target_logit;
    // backward
    const float *lse, *grad;
    P *p;           // [tokens][terms][p_seg], NULL: not wanted
    P *pt;          // [rows][terms][nk], 0 past the tokens, NULL: not wanted
    int64_t p_seg;
    int nk;
};

// C: tiles of 16 tokens.  KW: waves that share their rows and split the
// columns.  Loads of W and H are batched U steps of 32 columns deep.  Bound by
// reading W: backward, one token, 50000 x 2048 bf16, 40 us (205 MB, 5.1 TB/s);
// 32 tokens 57 us, H then costs half as many loads as W.
// Of 32-bit tensors, the bound on registers keeps the waves that the sums of the
// low products would cost a SIMD (64 tokens x 32000 x 1024, forward, 122 -> 94 us).
template <typename T, int C, int KW, bool BACK>
__global__ __launch_bounds__(kFewThreads, sizeof(T) == 4 ? (C == 2 ? 3 : 2) : 1) void few_kernel(FewArgs<T> a)
{
    typedef typename ProductOf<T>::P P;
    typedef typename Mfma<P>::Frag Frag;
    constexpr int kParts = ProductOf<T>::kParts;
    constexpr int R = few_row_tiles(C);
    constexpr int U = C == 1 ? 8 : kParts > 1 ? 2 : 4;
    __shared__ Soft soft[4][16 * C];
    __shared__ f32x4 other[KW > 1 ? KW - 1 : 1][KW > 1 ? R * C : 1][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    const int64_t v0 = ((int64_t)blockIdx.x * (4 / KW) + wave / KW) * (16 * R);
    const T *row[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
        row[r] = a.w + (v0 + 16 * r + low < a.rows ? v0 + 16 * r + low : a.rows - 1) * a.w_pitch;
    const P *hrow[C];
#pragma unroll
    for (int c = 0; c < C; ++c)
        hrow[c] = a.h.p + (16 * c + low < a.tokens ? 16 * c + low : a.tokens - 1) * a.h.pitch;
    f32x4 acc[R][C];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c)
            acc[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    // of terms: the sums of all products but the last
    [[maybe_unused]] f32x4 low_acc[kParts > 1 ? R : 1][kParts > 1 ? C : 1] = {};
    for (int64_t k0 = (wave % KW) * 32 * U; k0 < a.cols; k0 += 32 * U * KW) {
        typename VecOf<T, 8>::V raw[U][R];
        Frag hb[U][C][kParts];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t k = k0 + 32 * u + 8 * high;
#pragma unroll
            for (int r = 0; r < R; ++r)
                raw[u][r] = row_piece(row[r], k, a.cols);
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
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                Frag t[kParts];
                terms_of<T>(raw[u][r], t);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    if constexpr (kParts > 1) {
                        constexpr int kLast = kTermProducts - 1;
#pragma unroll
                        for (int s = 0; s < kLast; ++s)
                            low_acc[r][c] = Mfma<P>::run(t[term_a(s)], hb[u][c][term_b(s)], low_acc[r][c]);
                        acc[r][c] = Mfma<P>::run(t[term_a(kLast)], hb[u][c][term_b(kLast)], acc[r][c]);
                    } else {
                        acc[r][c] = Mfma<P>::run(t[0], hb[u][c][0], acc[r][c]);
                    }
                }
            }
    }
    if constexpr (kParts > 1) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[r][c][e] += finite_or_0(low_acc[r][c][e]);
    }
    if constexpr (KW > 1) {
        if (wave > 0)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int c = 0; c < C; ++c)
                    other[wave - 1][r * C + c][lane] = acc[r][c];
        __syncthreads();
        if (wave > 0)
            return;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int w = 0; w < KW - 1; ++w)
                    acc[r][c] += other[w][r * C + c][lane];
    }
    // acc[r][c][e]: the logit of row v0 + 16 r + 4 high + e and token 16 c + low
    if constexpr (!BACK) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int j = 16 * c + low;
            const int64_t t = j < a.tokens ? a.targets[j] : -1;
            float top = -__builtin_inff();
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t v = v0 + 16 * r + 4 * high + e;
                    if (v >= a.rows)
                        acc[r][c][e] = -__builtin_inff();
                    else if (v == t)
                        a.target_logit[j] = acc[r][c][e];
                    top = fmaxf(top, acc[r][c][e]);
                }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m = finite_or_0(top);
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sum += __expf(acc[r][c][e] - m);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (high == 0 && KW > 1 && j < a.tokens)
                a.part[(int64_t)blockIdx.x * a.tokens + j] = make_float2(top, sum);
            if (high == 0 && KW == 1)
                soft[wave][j] = Soft{top, sum};
        }
        if (KW > 1)
            return;
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
        constexpr int kTiles = C == 1 ? 2 : C;  // nk / 16
#pragma unroll
        for (int c = 0; c < kTiles; ++c) {
            const int j = 16 * c + low;
            const bool in = c < C && j < a.tokens;
            const float g = in ? a.grad[j] : 0.f, l = in ? a.lse[j] : 0.f;
            const int64_t t = in ? a.targets[j] : -1;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int64_t v = v0 + 16 * r + 4 * high;
                typename VecOf<P, 4>::V out[kParts];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = __expf(acc[r][c < C ? c : 0][e] - l) - (v + e == t ? 1.f : 0.f);
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
                    if (a.pt && v + e < a.rows)
#pragma unroll
                        for (int q = 0; q < kParts; ++q)
                            a.pt[((v + e) * kParts + q) * a.nk + j] = out[q][e];
                }
                if (a.p && in && v < a.p_seg)
#pragma unroll
                    for (int q = 0; q < kParts; ++q)
                        *(typename VecOf<P, 4>::V *)(a.p + (j * kParts + q) * a.p_seg + v) = out[q];
            }
        }
    }
}

// dW = P^T H of few tokens: 64 rows a workgroup, P held in registers, H^T
// streaming through from the L2.  What bounds it is writing dW: a wave's 16 x
// 64 results of a 16-bit type go through LDS, so that a row's 128 bytes are
// written at once.  32 tokens, 50000 x 2048 bf16: 37 us (205 MB, 5.5 TB/s).
template <typename T> struct FewWeightArgs {
    typedef typename ProductOf<T>::P P;
    const P *pt;  // [rows][terms][32 KS]
    const P *ht;  // [cols][terms][32 KS]: H transposed, 0 past the tokens
    const float *scale;
    T *dw;
    int64_t pitch, rows, cols;
};

template <typename T, int KS>
__global__ __launch_bounds__(kFewThreads) void few_weight_kernel(FewWeightArgs<T> a)
{
    typedef typename ProductOf<T>::P P;
    typedef typename Mfma<P>::Frag Frag;
    constexpr int kParts = ProductOf<T>::kParts;
    constexpr int kLine = 32 * KS * kParts;
    __shared__ __attribute__((aligned(16))) T turn[sizeof(T) == 2 ? 4 : 1][16][sizeof(T) == 2 ? 72 : 8];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    const int64_t v0 = (int64_t)blockIdx.x * kFewRows;
    Frag pb[4][KS][kParts];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t v = v0 + 16 * r + low;
        const P *src = a.pt + (v < a.rows ? v : a.rows - 1) * kLine + 8 * high;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int q = 0; q < kParts; ++q)
                pb[r][s][q] = *(const Frag *)(src + q * 32 * KS + 32 * s);
    }
    const float f = *a.scale;
    // 64 columns at a time, a wave's own
    for (int64_t d0 = ((int64_t)blockIdx.y * 4 + wave) * 64; d0 < a.cols; d0 += (int64_t)gridDim.y * 256) {
        Frag ha[4][KS][kParts];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t d = d0 + 16 * i + low;
            const P *src = a.ht + (d < a.cols ? d : a.cols - 1) * kLine + 8 * high;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    ha[i][s][q] = *(const Frag *)(src + q * 32 * KS + 32 * s);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t v = v0 + 16 * r + low;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    o = multiply_terms<P, kParts>(ha[i][s], pb[r][s], o);
                const float x[4] = {o[0] * f, o[1] * f, o[2] * f, o[3] * f};
                if constexpr (sizeof(T) == 2) {
                    typename VecOf<T, 4>::V t;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        t[e] = (T)x[e];
                    *(typename VecOf<T, 4>::V *)&turn[wave][low][16 * i + 4 * high] = t;
                } else {
                    const int64_t d = d0 + 16 * i + 4 * high;
                    const int left = a.cols - d < 4 ? (int)(a.cols - d) : 4;
                    if (v < a.rows && left > 0)
                        store_some(a.dw + v * a.pitch + d, left, x);
                }
            }
            if constexpr (sizeof(T) == 2) {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int line = lane / 8 + 8 * k;
                    const int64_t vr = v0 + 16 * r + line, d = d0 + lane % 8 * 8;
                    const typename VecOf<T, 8>::V t = *(const typename VecOf<T, 8>::V *)&turn[wave][line][lane % 8 * 8];
                    if (vr < a.rows) {
                        T *const at = a.dw + vr * a.pitch + d;
                        if (d + 8 <= a.cols)
                            *(typename VecOf<T, 8>::V *)at = t;
                        else
#pragma unroll
                            for (int e = 0; e < 7; ++e)
                                if (d + e < a.cols)
                                    at[e] = t[e];
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
        }
    }
}

// Sums over a part of the vocabulary of P W, 128 columns a workgroup: 64 rows
// of W at a time go through LDS and are read transposed out of it; the next 64
// are loaded meanwhile.  50000 x 2048 bf16, one token 51 us, 32 tokens 66 us (205
// MB, 3.1 TB/s: each step waits for its loads and two barriers).
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
    // 288 bytes a row: the four rows of a transposing read lie in different banks
    __shared__ __attribute__((aligned(16))) P tile[kParts][kFewRows][kFewCols + 16];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, low = lane % 16, high = lane / 16;
    const int64_t c0 = (int64_t)blockIdx.x * kFewCols;
    const int64_t all = (a.rows + kFewRows - 1) / kFewRows;
    const int64_t t0 = (int64_t)blockIdx.y * a.tiles, t1 = t0 + a.tiles < all ? t0 + a.tiles : all;
    const int lr = threadIdx.x / 16, lc = threadIdx.x % 16 * 8;
    typename VecOf<T, 8>::V raw[4];
    Frag next[2][C][kParts];  // of P
    auto load = [&](int64_t t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // rows past the end meet zeros of P, but have to be numbers
            const int64_t r = t * kFewRows + lr + 16 * i;
            raw[i] = row_piece(a.w + (r < a.rows ? r : a.rows - 1) * a.w_pitch, c0 + lc, r < a.rows ? a.cols : 0);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int j = 16 * c + low < a.tokens ? 16 * c + low : a.tokens - 1;
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    next[s][c][q] = *(const Frag *)(a.p + (j * kParts + q) * a.p_seg + t * kFewRows + 32 * s + 8 * high);
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
        Frag pb[2][C][kParts];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    pb[s][c][q] = next[s][c][q];
        __syncthreads();
        if (t + 1 < t1)
            load(t + 1);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                Frag wa[kParts];
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
                for (int q = 0; q < kParts; ++q) {
                    const P *at = &tile[q][32 * s + 8 * high + low / 4][wave * 32 + 16 * i + low % 4 * 4];
                    wa[q] = __builtin_bit_cast(
                        Frag, __builtin_shufflevector(turned((const char *)at),
                                                      turned((const char *)(at + 4 * (kFewCols + 16))), 0, 1, 2, 3,
                                                      4, 5, 6, 7));
                }
#endif
#pragma unroll
                for (int c = 0; c < C; ++c)
                    acc[i][c] = multiply_terms<P, kParts>(wa, pb[s][c], acc[i][c]);
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
