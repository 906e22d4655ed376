// rotor_xent: projection onto a vocabulary and softmax cross entropy, without
// the logits.
//
// Forward: the product W H^T in tiles; a tile's logits stay in registers, and
// each of its columns (a token) leaves a maximum and a sum of exponentials.
// A second launch joins the tiles' pairs.
// Backward, for pieces of the vocabulary: the same product again, whose
// epilogue turns logits into P = (softmax - target) * gradient and writes
// it in 16 bits; then dH^T += W^T P^T and dW = P^T H.  Both read
// their second operand with k over its rows and turn it on its way out of LDS,
// the one of which a wave reads fewer fragments: that costs nothing, where the
// first one turned would cost a tenth and both a third (8192 x 8192 results at
// k = 8192, without stores: 1458 TF/s with none, 1467 and 1319 with one, 931
// with both).  So dH is summed transposed, and H is transposed once for dW.
#include "rotor_few.h"
#include "rotor_product.h"

namespace rotor {
namespace {

typedef Tile<256, 256, 2, 4> Large;
typedef Tile<128, 128, 2, 2> Small;

// dst[r][c] = src[r][c], 0 for columns up to `cols_to` (a multiple of 8): eight
// columns a thread.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T *src, int64_t rows, int64_t cols, int64_t pitch,
                                                   typename ProductOf<T>::P *dst, int64_t dst_pitch, int64_t dst_seg,
                                                   int64_t cols_to)
{
    typedef typename ProductOf<T>::P P;
    constexpr int kParts = ProductOf<T>::kParts;
    const int64_t at = block_at() * 256 + threadIdx.x, pieces = cols_to / 8;
    const int64_t r = at / pieces, c = at % pieces * 8;
    if (r >= rows)
        return;
    typename Mfma<P>::Frag t[kParts];
    terms_of<T>(row_piece(src + r * pitch, c, cols), t);
#pragma unroll
    for (int q = 0; q < kParts; ++q)
        *(typename Mfma<P>::Frag *)(dst + r * dst_pitch + q * dst_seg + c) = t[q];
}

// The tokens that count, in two layouts as operands: packed[r][c] = row
// order[r] of src, and turned[c][r], which is 0 for r from their number up to
// the next multiple of 8 (NULL: not wanted), and whose columns r are multiplied
// by undo[r] (NULL: 1).  64 x 64 elements a workgroup through LDS, eight adjacent
// ones a load and a store.  8192 x 4096 bf16: 23 us.
template <typename P> struct TurnArgs {
    int64_t cols, pitch;
    const int *order, *live;
    const float *undo;
    P *packed, *turned;
    int64_t packed_pitch, packed_seg, turned_pitch, turned_seg;
};
template <typename T>
__global__ __launch_bounds__(256) void turn_kernel(const T *src, TurnArgs<typename ProductOf<T>::P> a)
{
    typedef typename ProductOf<T>::P P;
    constexpr int kParts = ProductOf<T>::kParts;
    __shared__ float tile[64][65];
    const int64_t r0 = (int64_t)blockIdx.x * 64, c0 = (int64_t)blockIdx.y * 64;
    const int live = *a.live;
    if (r0 >= live)
        return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int row = threadIdx.x / 8 + 32 * k, col = threadIdx.x % 8 * 8;
        const int64_t r = r0 + row;
        const bool some = r < live;
        const typename VecOf<T, 8>::V v =
            row_piece(src + (int64_t)(some ? a.order[r] : 0) * a.pitch, c0 + col, some ? a.cols : 0);
        const float u = some && a.undo ? a.undo[r] : 1.f;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            tile[row][col + e] = (float)v[e] * u;
        if (some && c0 + col < a.cols) {
            typename Mfma<P>::Frag t[kParts];
            terms_of<T>(v, t);
#pragma unroll
            for (int q = 0; q < kParts; ++q)
                *(typename Mfma<P>::Frag *)(a.packed + r * a.packed_pitch + q * a.packed_seg + c0 + col) = t[q];
        }
    }
    if (!a.turned)
        return;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int col = threadIdx.x / 8 + 32 * k, row = threadIdx.x % 8 * 8;
        if (c0 + col >= a.cols || r0 + row >= live)
            continue;
        typename VecOf<T, 8>::V v;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = (T)tile[row + e][col];
        typename Mfma<P>::Frag t[kParts];
        terms_of<T>(v, t);
#pragma unroll
        for (int q = 0; q < kParts; ++q)
            *(typename Mfma<P>::Frag *)(a.turned + (c0 + col) * a.turned_pitch + q * a.turned_seg + r0 + row) = t[q];
    }
}

// ---- epilogues -------------------------------------------------------------------

// Maximum and sum of exponentials of each token over the tile's rows of W,
// and the target's logit.
// Measured (the whole launch): 4096 tokens x 32768 x 2048 bf16 454 us (1211
// TF/s), 8192 x 128000 x 4096 6.4 ms (1340 TF/s); at 2048 columns the
// exponentials are about a tenth of it.  One token, 50021 x 2048: 35 us (205 MB,
// 5.8 TB/s), bound by reading W.
struct StatsEpilogue {
    [[maybe_unused]] static constexpr Live kLive = kLiveNone;
    float2 *part;  // [tiles_i][tokens]
    float *target_logit;
    const int64_t *targets;
    int64_t v0;         // the first row of W
    int vocab, tokens;  // rows, tokens
    template <typename S> __device__ void operator()(Results<S> &r, char *lds) const
    {
        Soft(*other)[S::BJ] = (Soft(*)[S::BJ])lds;
        const int have = vocab - r.tile_i * S::BI;  // rows of W in the tile
        const int j0 = r.tile_j * S::BJ;
        if (have < S::BI) {
#pragma unroll
            for (int ii = 0; ii < S::NI; ++ii)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (r.i + 16 * ii + e >= have)
#pragma unroll
                        for (int jj = 0; jj < S::NJ; ++jj)
                            r.acc[ii][jj][e] = -__builtin_inff();
        }
#pragma unroll
        for (int jj = 0; jj < S::NJ; ++jj) {
            const int j = j0 + r.j + 16 * jj;
            // the target's place among this lane's rows, if it is there
            const int64_t t64 = (j < tokens ? targets[j] : -1) - v0 - r.tile_i * S::BI;
            const int t = t64 >= 0 && t64 < S::BI && t64 < have ? (int)t64 - r.i : -1;
            if (__any(t >= 0 && t < 16 * S::NI)) {  // few tokens have their target in one tile
#pragma unroll
                for (int ii = 0; ii < S::NI; ++ii)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (t == 16 * ii + e)
                            target_logit[j] = r.acc[ii][jj][e];
            }
            float top = -__builtin_inff();
#pragma unroll
            for (int ii = 0; ii < S::NI; ++ii)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    top = fmaxf(top, r.acc[ii][jj][e]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m2 = finite_or_0(top) * kLog2e;
            float sum = 0.f;
#pragma unroll
            for (int ii = 0; ii < S::NI; ++ii)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sum += exp_over(r.acc[ii][jj][e], m2);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (r.lane < 16)
                other[r.wave_i][(r.wave_j * S::NJ + jj) * 16 + r.lane] = Soft{top, sum};
        }
        __syncthreads();
        const int j = threadIdx.x;
        if (j >= S::BJ || j0 + j >= tokens)
            return;
        Soft s = other[0][j];
#pragma unroll
        for (int w = 1; w < S::WI; ++w)
            s = join(s, other[w][j]);
        part[(int64_t)r.tile_i * tokens + j0 + j] = make_float2(s.top, s.sum);
    }
};

// P[j][i] from the logits, rounded once to 16 bits (what the two products
// after it take; in bf16 an error of at most 2^-8 of each term, that of the
// gradients' own rounding), or split into three terms.  8192 tokens x 8000 x
// 4096 bf16: 445 us (1210 TF/s), with 131 MB of P written.
template <typename T> struct ProbEpilogue {
    typedef typename ProductOf<T>::P P;
    static constexpr int kParts = ProductOf<T>::kParts;
    static constexpr Live kLive = kLiveB;
    const int *live;
    P *p;
    int pitch, seg;
    const float *lse, *grad;  // of the tokens that count; grad: scaled gradient of the loss
    const int *targets;
    int v0, rows;  // the piece's first row of W, and its rows
    template <typename S> __device__ void operator()(Results<S> &r, char *) const
    {
        typedef typename VecOf<P, 4>::V V4;
        const int have = rows - r.tile_i * S::BI, tokens = *live;
        const int j0 = r.tile_j * S::BJ;
        // the piece is padded to whole tiles, and so is P's pitch
        P *const tile = p + (int64_t)j0 * pitch + r.tile_i * S::BI;
#pragma unroll
        for (int jj = 0; jj < S::NJ; ++jj) {
            int row = r.j + 16 * jj;
            opaque(row);
            const int j = j0 + row;
            const bool in = j < tokens;
            const float g = in ? grad[j] : 0.f, l2 = in ? lse[j] * kLog2e : 0.f;
            const int at_target = (in ? targets[j] : -1) - v0 - r.tile_i * S::BI;
            const int t = at_target >= 0 && at_target < S::BI ? at_target - r.i : -1;
#pragma unroll
            for (int ii = 0; ii < S::NI; ++ii)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    r.acc[ii][jj][e] = exp_over(r.acc[ii][jj][e], l2) * g;
            if (__any(t >= 0 && t < 16 * S::NI)) {  // few tokens have their target in one tile
#pragma unroll
                for (int ii = 0; ii < S::NI; ++ii)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        r.acc[ii][jj][e] -= t == 16 * ii + e ? g : 0.f;
            }
            if (have < S::BI) {
#pragma unroll
                for (int ii = 0; ii < S::NI; ++ii)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        r.acc[ii][jj][e] = r.i + 16 * ii + e < have ? r.acc[ii][jj][e] : 0.f;
            }
            if constexpr (kParts > 1) {
                if (!in)
                    continue;
#pragma unroll
                for (int ii = 0; ii < S::NI; ++ii) {
                    P *const at = tile + (uint32_t)(row * pitch + r.i + 16 * ii);
                    V4 w[kTerms];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        bf16 s[kTerms];
                        split(r.acc[ii][jj][e], s);
#pragma unroll
                        for (int q = 0; q < kTerms; ++q)
                            w[q][e] = s[q];
                    }
#pragma unroll
                    for (int q = 0; q < kTerms; ++q)
                        *(V4 *)(at + q * seg) = w[q];
                }
            }
        }
        if constexpr (kParts == 1)
            put_rows(r, tile, pitch, tokens - j0, S::BI);
    }
};

// C as 32-bit sums, one part of a split product, added to what is there or not:
// dH, transposed (L is kLiveA), and dW where it has few tiles (kLiveK).  8192 x 4096 from 8000 rows bf16: 452 us (1190 TF/s with 268
// MB of sums read and written; 475 us as C[token][column], for which more
// fragments are read turned).
template <Live L> struct SumEpilogue {
    static constexpr Live kLive = L;
    const int *live;
    float *c;
    int64_t part;  // elements between the parts
    int pitch, cols, rows, add;
    template <typename S> __device__ void operator()(Results<S> &r, char *) const
    {
        float *const tile = c + r.part * part + (int64_t)r.tile_j * S::BJ * pitch + r.tile_i * S::BI;
        const int cols_in = (L == kLiveA ? *live : cols) - r.tile_i * S::BI, rows_in = rows - r.tile_j * S::BJ;
#pragma unroll
        for (int jj = 0; jj < S::NJ; ++jj) {
            int j = r.j + 16 * jj;
            opaque(j);
            if (j >= rows_in)
                continue;
#pragma unroll
            for (int ii = 0; ii < S::NI; ++ii) {
                const int i = r.i + 16 * ii;  // pitch is a multiple of 4
                if (i >= cols_in)
                    continue;
                f32x4 *at = (f32x4 *)(tile + (uint32_t)(j * pitch + i));
                *at = add ? *at + r.acc[ii][jj] : r.acc[ii][jj];
            }
        }
    }
};

// dW: C in the type of the result, times a scale from the device.  8000 x 4096
// from 8192 tokens bf16: 437 us (1230 TF/s; 465 us with H not transposed before).
template <typename T> struct OutEpilogue {
    static constexpr Live kLive = kLiveK;
    const int *live;
    T *c;
    const float *scale;
    int pitch, cols, rows;
    template <typename S> __device__ void operator()(Results<S> &r, char *) const
    {
        const float f = *scale;
        T *const tile = c + (int64_t)r.tile_j * S::BJ * pitch + r.tile_i * S::BI;
        const int cols_in = cols - r.tile_i * S::BI, rows_in = rows - r.tile_j * S::BJ;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int jj = 0; jj < S::NJ; ++jj)
#pragma unroll
                for (int ii = 0; ii < S::NI; ++ii)
                    r.acc[ii][jj] *= f;
            put_rows(r, tile, pitch, rows_in, cols_in);
        } else {
#pragma unroll
            for (int jj = 0; jj < S::NJ; ++jj) {
                int j = r.j + 16 * jj;
                opaque(j);
                if (j >= rows_in)
                    continue;
#pragma unroll
                for (int ii = 0; ii < S::NI; ++ii) {
                    const int i = r.i + 16 * ii, left = cols_in - i < 4 ? cols_in - i : 4;
                    const float v[4] = {r.acc[ii][jj][0] * f, r.acc[ii][jj][1] * f, r.acc[ii][jj][2] * f,
                                        r.acc[ii][jj][3] * f};
                    if (left > 0)
                        store_some(tile + (uint32_t)(j * pitch + i), left, v);
                }
            }
        }
    }
};

// ---- small launches -----------------------------------------------------------------

// Joins the tiles' maxima and sums: X tokens a workgroup, 256 / X lanes each.
template <int X>
__global__ __launch_bounds__(256) void loss_kernel(const float2 *part, int64_t tiles, const float *target_logit,
                                                   const int64_t *targets, int64_t ignore, int64_t vocab,
                                                   int64_t tokens, float *loss, float *lse)
{
    constexpr int Y = 256 / X;
    __shared__ Soft other[Y][X + 1];
    const int x = threadIdx.x % X, y = threadIdx.x / X;
    const int64_t j = (int64_t)blockIdx.x * X + x;
    Soft s{-__builtin_inff(), 0.f};
    if (j < tokens) {
#pragma unroll 4
        for (int64_t t = y; t < tiles; t += Y) {
            const float2 v = part[t * tokens + j];
            s = join(s, Soft{v.x, v.y});
        }
    }
    other[y][x] = s;
    for (int half = Y / 2; half >= 1; half /= 2) {
        __syncthreads();
        if (y < half)
            other[y][x] = join(other[y][x], other[y + half][x]);
    }
    if (y > 0 || j >= tokens)
        return;
    s = other[0][x];
    const float l = finite_or_0(s.top) + logf(s.sum);
    lse[j] = l;
    const int64_t t = targets[j];
    loss[j] = t == ignore ? 0.f : t >= 0 && t < vocab ? l - target_logit[j] : __builtin_nanf("");
}

// Gradients of the losses, 0 without a target, divided by the largest and
// multiplied by 2^15, so that P fits the range of 16-bit floats whatever the
// loss was divided by; `scale` undoes it.  The gradient of a mean or a sum is
// then 2^15 for every token, and what P holds at the targets, by far the largest
// of its terms, is 2^15 (p - 1): rounded to 16 bits it is off by a third less on
// average than at gradients between two powers of two, and by p at most for a
// small p (70 draws in bf16: errors of the gradients up to 1.5 times those of a
// last rounding alone, with a power of two as the divisor up to twice).
//
// Of f16, whose range ends 2^40 below that, the smaller gradients are multiplied
// by up to 2^8 more, a power of two for each token (undo: its inverse), and the
// token's column of H^T is divided by it: the probabilities of a token with
// 2^-20 of the largest gradient would vanish otherwise, and with them their part
// of its row of dH (60000 x 64, off by a quarter).  2^8, since h in 16 bits stays
// within its own rounding down to 2^-6.
struct GradArgs {
    const float *grad_loss;
    const int64_t *targets;
    int64_t ignore, vocab, tokens;
    int lift;  // the most by which a gradient is multiplied, as a power of two
    float *grad, *scale, *undo;  // undo: NULL without lift
};
constexpr int kTop = 15;
__device__ inline float grad_size(const GradArgs &a, int64_t j)
{
    const int64_t t = a.targets[j];
    const float g = fabsf(a.grad_loss[j]);
    return t != a.ignore && g <= 3.4028234e38f ? g : 0.f;
}
__device__ inline float grad_unit(float most) { return fmaxf(most, 0x1p-100f); }
__device__ inline float scaled_grad(const GradArgs &a, int64_t j, float unit)
{
    const int64_t t = a.targets[j];
    const float g = a.grad_loss[j] / unit * 0x1p15f;
    return t == a.ignore ? 0.f : t >= 0 && t < a.vocab ? g : __builtin_nanf("");
}
__device__ inline int lift_of(const GradArgs &a, float scaled)
{
    int e = 0;
    (void)frexpf(scaled, &e);
    return e >= kTop ? 0 : kTop - e < a.lift ? kTop - e : a.lift;
}
__device__ inline float wave_max(float v)
{
#pragma unroll
    for (int off = 32; off >= 1; off /= 2)
        v = fmaxf(v, __shfl_xor(v, off));
    return v;
}

// The tokens that count, those with a gradient other than 0, in order: order
// lists them, and then the others; their number is *live; the gradients, lse and
// targets (-1: none of the rows) of a token that counts lie at its place among
// them.  The others cost the backward's three products nothing: 4096 tokens x
// 32768 x 2048 bf16, 30% of them without a target, forward and backward 1535 us,
// 1855 with all of them in the products.  Every workgroup finds the largest
// gradient, and how many tokens count before its own, for itself: 12 bytes a token
// from the L2 (65536 tokens 36 us, 175 in one workgroup), at most 256 times over
// at the 2^20 tokens that a call takes.
struct TokenArgs {
    GradArgs g;
    const float *lse;
    float *live_lse;
    int *order, *live_target, *live;
};
constexpr int kEach = 4;                   // adjacent tokens of a thread
constexpr int kGradTokens = 1024 * kEach;  // of a workgroup
__global__ __launch_bounds__(1024) void grad_kernel(TokenArgs a)
{
    __shared__ float top[16];
    __shared__ int before[16], count[16];
    const int tokens = (int)a.g.tokens, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    float m = 0.f;
#pragma unroll 8
    for (int j = threadIdx.x; j < tokens; j += 1024)
        m = fmaxf(m, grad_size(a.g, j));
    m = wave_max(m);
    if (lane == 0)
        top[wave] = m;
    __syncthreads();
    for (int w = 0; w < 16; ++w)
        m = fmaxf(m, top[w]);
    const float unit = grad_unit(m);
    const int j0 = blockIdx.x * kGradTokens, j = j0 + (int)threadIdx.x * kEach;
    int sum = 0;  // of the tokens before this workgroup's
#pragma unroll 8
    for (int i = threadIdx.x; i < j0; i += 1024)
        sum += scaled_grad(a.g, i, unit) != 0.f;
    for (int off = 32; off >= 1; off /= 2)
        sum += __shfl_xor(sum, off);
    if (lane == 0)
        before[wave] = sum;
    float g[kEach];
    int at = 0;
    sum = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        g[k] = j + k < tokens ? scaled_grad(a.g, j + k, unit) : 0.f;
        const uint64_t mask = __ballot(g[k] != 0.f);
        at += __popcll(mask & (((uint64_t)1 << lane) - 1));
        sum += __popcll(mask);
    }
    if (lane == 0)
        count[wave] = sum;
    __syncthreads();
    int live = 0;  // tokens that count, up to the workgroup's last
    for (int w = 0; w < 16; ++w) {
        at += before[w] + (w < wave ? count[w] : 0);
        live += before[w] + count[w];
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        if (g[k] != 0.f) {
            const int64_t t = a.g.targets[j + k];
            a.order[at] = j + k;
            const int lift = lift_of(a.g, g[k]);
            a.g.grad[at] = ldexpf(g[k], lift);
            if (a.g.undo)
                a.g.undo[at] = ldexpf(1.f, -lift);
            a.live_lse[at] = a.lse[j + k];
            a.live_target[at] = t >= 0 && t < a.g.vocab ? (int)t : -1;
            ++at;
        } else if (j + k < tokens) {
            a.order[tokens - 1 - (j + k - at)] = j + k;  // of the tokens before it, `at` count
        }
    }
    if (threadIdx.x == 0 && blockIdx.x == 0)
        *a.g.scale = unit * 0x1p-15f;
    if (threadIdx.x == 0 && blockIdx.x == gridDim.x - 1)
        *a.live = live;
}

// The same for few tokens, H transposed (dst[c][r] = src[r][c], 0 for rows up
// to `rows_to` and for those without a target) and, where it is wanted, copied
// as a product's operand, in one launch: 64 columns a workgroup, every one of
// which finds the scale for itself.
template <typename T> struct FewPrepareArgs {
    typedef typename ProductOf<T>::P P;
    GradArgs g;
    const T *h;
    int64_t pitch, cols, cols_to;
    P *turned;  // [cols][terms][rows_to], NULL: not wanted
    P *packed;  // [tokens][terms][cols_to], NULL: not wanted
    int rows_to;
};
template <typename T> __global__ __launch_bounds__(256) void few_prepare_kernel(FewPrepareArgs<T> a)
{
    typedef typename ProductOf<T>::P P;
    constexpr int kParts = ProductOf<T>::kParts;
    __shared__ float tile[kFew][65];
    const int x = threadIdx.x % 64, y = threadIdx.x / 64;
    const int tokens = (int)a.g.tokens;
    const float unit = grad_unit(wave_max(x < tokens ? grad_size(a.g, x) : 0.f));
    const float g = x < tokens ? scaled_grad(a.g, x, unit) : 0.f;
    const int lift = lift_of(a.g, g);
    const float undo = ldexpf(1.f, -lift);
    if (blockIdx.x == 0 && y == 0) {
        if (x < tokens) {
            a.g.grad[x] = ldexpf(g, lift);
            if (a.g.undo)
                a.g.undo[x] = undo;
        }
        if (x == 0)
            *a.g.scale = unit * 0x1p-15f;
    }
    const int64_t c = (int64_t)blockIdx.x * 64 + x;
    for (int k = y; k < kFew; k += 4) {
        const bool some = __shfl(g, k) != 0.f;
        tile[k][x] = k < tokens && c < a.cols && some ? (float)a.h[k * a.pitch + c] : 0.f;
    }
    __syncthreads();
    if (a.turned && x < a.rows_to)
        for (int k = y; k < 64 && blockIdx.x * 64 + k < a.cols; k += 4) {
            P *at = a.turned + ((int64_t)blockIdx.x * 64 + k) * kParts * a.rows_to + x;
            if constexpr (kParts == 1) {
                *at = (P)(tile[x][k] * undo);
            } else {
                bf16 t[kTerms];
                split(tile[x][k], t);
#pragma unroll
                for (int q = 0; q < kTerms; ++q)
                    at[q * a.rows_to] = t[q];
            }
        }
    if (a.packed && c < a.cols_to)
        for (int k = y; k < tokens; k += 4) {
            P *at = a.packed + k * kParts * a.cols_to + c;
            if constexpr (kParts == 1) {
                *at = (P)tile[k][x];
            } else {
                bf16 t[kTerms];
                split(tile[k][x], t);
#pragma unroll
                for (int q = 0; q < kTerms; ++q)
                    at[q * a.cols_to] = t[q];
            }
        }
}

// A gradient from its parts' sums: four columns a thread, Y threads a share of the
// parts each, the shares then in order.  Where rows are tokens (grad is their
// losses' gradients), those without a gradient are 0 whatever their sums hold: 0
// times a row of W that is not finite is NaN.  undo: factors of the rows, or NULL.
template <typename T, int Y>
__global__ __launch_bounds__(256) void finish_kernel(const float *sum, int64_t pitch, int64_t part, int parts,
                                                     int64_t rows, int64_t cols, const float *scale,
                                                     const float *grad, const float *undo, T *out,
                                                     int64_t out_pitch)
{
    constexpr int X = 256 / Y;
    __shared__ f32x4 other[Y][X];
    const int64_t quads = (cols + 3) / 4;
    const int x = threadIdx.x % X, y = threadIdx.x / X;
    const int64_t at = (int64_t)blockIdx.x * X + x;
    const bool in = at < rows * quads;
    const int64_t j = in ? at / quads : 0, i = in ? at % quads * 4 : 0;
    const int each = (parts + Y - 1) / Y, to = (y + 1) * each < parts ? (y + 1) * each : parts;
    f32x4 s{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int q = y * each; q < to; ++q)
        s += *(const f32x4 *)(sum + q * part + j * pitch + i);
    if (Y > 1) {
        other[y][x] = s;
        __syncthreads();
        if (y > 0)
            return;
#pragma unroll
        for (int w = 1; w < Y; ++w)
            s += other[w][x];
    }
    if (!in)
        return;
    if (grad && grad[j] == 0.f)
        s = f32x4{0.f, 0.f, 0.f, 0.f};
    const float f = *scale * (undo ? undo[j] : 1.f);
    const float v[4] = {s[0] * f, s[1] * f, s[2] * f, s[3] * f};
    store_some(out + j * out_pitch + i, cols - i < 4 ? (int)(cols - i) : 4, v);
}

// The same from sums of the tokens that count, which lie transposed,
// [parts][cols][pitch], and 0 for the others: D columns of 64 rows a workgroup,
// through LDS.  64 columns, or 16 where each has four parts or more to add: more
// workgroups then read them (171 x 1088 of 29 parts 8 us,
// with 64 columns 16 us; 512 x 1024 of 32 parts 11 and 14 us).
template <typename T, int D>
__global__ __launch_bounds__(256) void turn_finish_kernel(const float *sum, int64_t pitch, int64_t part, int parts,
                                                          int64_t rows, int64_t cols, const int *order,
                                                          const int *count, const float *scale,
                                                          const float *undo, T *out, int64_t out_pitch)
{
    __shared__ float tile[D][65];
    const int live = *count;
    const int64_t r0 = (int64_t)blockIdx.x * 64, c0 = (int64_t)blockIdx.y * D;
    const int x = threadIdx.x % 16 * 4, y = threadIdx.x / 16;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
        const int64_t c = c0 + y + 16 * k;
        f32x4 s{0.f, 0.f, 0.f, 0.f};
        if (c < cols && r0 + x < live) {  // pitch is a multiple of 4
#pragma unroll 8
            for (int q = 0; q < parts; ++q)
                s += *(const f32x4 *)(sum + q * part + c * pitch + r0 + x);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            tile[y + 16 * k][x + e] = s[e];
    }
    __syncthreads();
    const float f = *scale;
    const int col = threadIdx.x % (D / 4) * 4, row0 = threadIdx.x / (D / 4);
    const int64_t c = c0 + col;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
        const int row = row0 + 1024 / D * k;
        if (r0 + row >= rows || c >= cols)
            continue;
        const float u = undo && r0 + row < live ? f * undo[r0 + row] : f;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = r0 + row < live ? tile[col + e][row] * u : 0.f;
        store_some(out + order[r0 + row] * out_pitch + c, cols - c < 4 ? (int)(cols - c) : 4, v);
    }
}

// Clears a matrix (gradients of nothing).
template <typename T> __global__ __launch_bounds__(256) void clear_kernel(T *out, int64_t rows, int64_t cols,
                                                                          int64_t pitch)
{
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < cols; c += 256)
            out[r * pitch + c] = (T)0.f;
}

// ---- plans --------------------------------------------------------------------------

constexpr int64_t kPad = 256;                        // columns of P in whole tiles
constexpr int64_t kPieceBytes = (int64_t)128 << 20;  // of P, or of a copied piece of W

int64_t pad(int64_t n, int64_t to) { return ceil_div(n, to) * to; }

struct Bump {
    uint64_t at = 0;
    uint64_t take(uint64_t bytes)
    {
        const uint64_t here = at;
        at = round256(at + bytes);
        return here;
    }
};

bool xent_sizes_ok(int32_t type, int64_t n, int64_t d, int64_t v)
{
    return type_ok(type) && n >= 0 && n <= ROTOR_XENT_MAX_TOKENS && d >= 1 && d <= ROTOR_XENT_MAX_COLS && v >= 1 &&
           v <= ROTOR_XENT_MAX_ROWS;
}

// The largest pitch, in elements, with which 256 rows lie within 2^31 bytes.
constexpr int64_t kMostPitch = (int64_t)1 << 22;

// Whether the rows of a matrix can be read where they are.
bool rows_aligned(const void *p, int64_t cols, int64_t pitch)
{
    return (uintptr_t)p % 16 == 0 && cols % 8 == 0 && pitch % 8 == 0;
}

// Whether a call goes the way of few tokens: that of the probabilities as a
// whole, in two layouts, if those are no larger than two pieces.  Operands that
// would have to be copied always do: the small tiles read a copy of W, the few
// tokens' kernels W itself (64 tokens x 32000 x 1024 f32 80 against 192 us forward,
// 245 against 330 backward).  Others where W's rows do not give small tiles to
// three quarters of the CUs (1 x 1000 x 4096 bf16 16 against 47 us), and up to
// 32 tokens backward (1 x 50000 x 2048 139 against 174 us; 64 tokens 228
// against 193); forward the small tiles read W faster (1 x 50021 x 2048 44
// against 38 us, 64 x 128000 x 4096 402 against 180).
bool few_tokens(int32_t type, int64_t n, int64_t v, bool pack, bool backward)
{
    const int64_t parts = type == ROTOR_F32 ? kTerms : 1;
    if (n > kFew || 2 * 2 * parts * kFew * v > 2 * kPieceBytes)
        return false;
    return pack || ceil_div(v, Small::BI) < 192 || (backward && n <= 32);
}

struct ForwardLayout {
    uint64_t part, target, h, w, total;
    int64_t dk, piece;
};

// `pack`: H and W are copied as product operands, W piece by piece.
ForwardLayout forward_layout(int32_t type, int64_t n, int64_t d, int64_t v, bool pack)
{
    ForwardLayout l;
    Bump b;
    const int64_t parts = type == ROTOR_F32 ? kTerms : 1;
    l.dk = pad(d, kStep);
    l.part = b.take(8ull * (uint64_t)ceil_div(v, few_tokens(type, n, v, pack, false) ? few_rows(n, v) : 128) * (uint64_t)n);
    l.target = b.take(4ull * (uint64_t)n);
    l.piece = v;
    l.h = l.w = b.at;
    if (few_tokens(type, n, v, pack, false)) {
        l.h = b.take(pack ? 2ull * (uint64_t)(parts * l.dk * n) : 0);
    } else if (pack) {
        const int64_t most = kPieceBytes / (2 * parts * l.dk) / kPad * kPad;  // at least kPad: see the limits
        l.piece = v < most ? v : most;
        l.h = b.take(2ull * (uint64_t)(parts * l.dk * n));
        l.w = b.take(2ull * (uint64_t)(parts * l.dk * l.piece));
    }
    l.total = b.at;
    return l;
}

// Rows of the library's own operands start 512 bytes further on than their
// lengths ask for: with a power of two between them, the rows of a tile lie in
// few of the memory's channels (a product of 8192 x 8192 results at k = 2048
// 1336 TF/s, 1463 with the 512 bytes).
constexpr int64_t kSkew = 256;
int64_t skewed(int64_t cols) { return cols + kSkew; }

struct BackwardLayout {
    uint64_t grad, scale, undo, order, lse, target, live, h, w, ht, p, pt, sum, w_sum, total;
    int64_t dk, piece, nk, p_pitch, sum_pitch, w_pitch;
    int split, w_split;
};

int64_t tiles(int64_t a, int64_t b, int64_t side) { return ceil_div(a, side) * ceil_div(b, side); }

BackwardLayout backward_layout(int32_t type, int64_t n, int64_t d, int64_t v, bool pack)
{
    BackwardLayout l;
    Bump b;
    const int64_t parts = type == ROTOR_F32 ? kTerms : 1;
    l.dk = pad(d, kStep);
    l.sum_pitch = pad(d, 4);
    l.grad = b.take(4ull * (uint64_t)n);
    l.scale = b.take(4);
    l.undo = b.take(type == ROTOR_F16 ? 4ull * (uint64_t)n : 0);
    if (few_tokens(type, n, v, pack, true)) {
        l.nk = n <= 32 ? 32 : 64;
        l.piece = pad(v, kFewRows);
        l.h = b.take(pack ? 2ull * (uint64_t)(parts * l.dk * n) : 0);
        l.ht = b.take(2ull * (uint64_t)(parts * l.nk * d));
        l.p = b.take(2ull * (uint64_t)(parts * l.piece * n));
        l.pt = b.take(2ull * (uint64_t)(parts * l.nk * v));
        // parts of the vocabulary for three workgroups on every CU, of four
        // tiles at least
        const int64_t t = l.piece / kFewRows, most = ceil_div(t, 4);
        const int64_t want = ceil_div(768, ceil_div(d, kFewCols));
        l.split = (int)(want < most ? want : most);
        l.sum = b.take(4ull * (uint64_t)(l.split * n * l.sum_pitch));
        l.w = l.w_sum = l.order = l.lse = l.target = l.live = 0;
        l.total = b.at;
        return l;
    }
    l.order = b.take(4ull * (uint64_t)n);
    l.lse = b.take(4ull * (uint64_t)n);
    l.target = b.take(4ull * (uint64_t)n);
    l.live = b.take(4);
    l.nk = skewed(pad(n, 8));
    l.piece = pad(v, kPad);
    int64_t most = kPieceBytes / (2 * parts * (pack && l.dk > n ? l.dk : n));
    if (most > kMostPitch / parts - kSkew)
        most = kMostPitch / parts - kSkew;
    most = most < kPad ? kPad : most / kPad * kPad;
    if (l.piece > most) {
        // pieces of equal size
        const int64_t count = ceil_div(l.piece, most);
        l.piece = pad(ceil_div(l.piece, count), kPad);
    }
    l.h = b.take(2ull * (uint64_t)(parts * l.dk * n));
    l.w = b.take(pack ? 2ull * (uint64_t)(parts * l.dk * l.piece) : 0);
    l.p_pitch = skewed(l.piece);
    l.sum_pitch = pad(n, 4);
    l.p = b.take(2ull * (uint64_t)(parts * l.p_pitch * n));
    l.ht = b.take(2ull * (uint64_t)(parts * l.nk * d));
    l.pt = 0;
    // few tiles of dH: its summed index (the piece) in parts, for a large
    // tile on every CU, of eight steps at least
    int64_t split = ceil_div(256, tiles(d, n, 256));
    const int64_t steps = (type == ROTOR_F32 ? kTermProducts : 1) * (l.piece / kStep);
    if (split > steps / 8)
        split = steps / 8 > 0 ? steps / 8 : 1;
    l.split = (int)split;
    l.sum = b.take(4ull * (uint64_t)(l.split * d * l.sum_pitch));
    // and few of dW: the tokens in parts, if there is a whole round of them
    // (65536 tokens x 1000 x 512 bf16, backward, 1267 us without, 519 with; 2048
    // x 5000 x 1024, which has 80 tiles, 118 without, 135 with)
    l.w_split = tiles(d, l.piece, 256) <= 64 ? (int)(256 / tiles(d, l.piece, 256)) : 1;
    const int64_t w_steps = (type == ROTOR_F32 ? kTermProducts : 1) * ceil_div(n, kStep);
    if (l.w_split > w_steps / 8)
        l.w_split = (int)(w_steps / 8);
    if (l.w_split < 2)
        l.w_split = 1;
    l.w_pitch = pad(d, 4);
    l.w_sum = b.take(l.w_split > 1 ? 4ull * (uint64_t)(l.w_split * l.piece * l.w_pitch) : 0);
    l.total = b.at;
    return l;
}

// C of ni x nj results, the summed index in `split` parts.
struct Extent {
    int64_t ni, nj, k;
    int split;
};

template <typename P, typename S, bool KB, bool TERMS, typename E>
void run_tiles(const Operand<P> &a, const Operand<P> &b, const Extent &x, E e, hipStream_t s)
{
    ProductArgs p;
    p.k = x.k;
    p.products = a.seg ? kTermProducts : 1;
    p.tiles_i = (int)ceil_div(x.ni, S::BI);
    p.tiles_j = (int)ceil_div(x.nj, S::BJ);
    p.steps = p.products * (int)ceil_div(x.k, kStep);
    p.split_steps = (int)ceil_div(p.steps, x.split);
    // as many workgroups as the 256 CUs hold at once (by their LDS)
    const int64_t tiles = (int64_t)p.tiles_i * p.tiles_j, most = 256 * ((160 << 10) / (2 * S::kBytes)) / x.split;
    product_kernel<P, S, KB, TERMS, E>
        <<<dim3((uint32_t)(tiles < most || most < 8 ? tiles : most / 8 * 8), (uint32_t)x.split), S::kThreads, 0, s>>>(
            a, b, p, e);
}

// Large tiles if they fill half of the 256 CUs and neither side fits a small
// one.  Measured, forward and backward, large against small: 171 tokens x
// 15156 x 1088 107 against 114 us at 120 large tiles, 2000 x 30000 x 64 205
// against 178 us at under 100; 70 x 50000 x 2048 267 against 239 us, 4096 x
// 50000 x 128 733 against 695 us, where half a large tile's work would go
// unused.
bool large_tiles(int64_t a, int64_t b, int split)
{
    return tiles(a, b, 256) * split >= 128 && a > 128 && b > 128;
}

template <bool KB, bool TERMS = false, typename P, typename E>
void run_product(const Operand<P> &a, const Operand<P> &b, const Extent &x, E e, hipStream_t s)
{
    if (large_tiles(x.ni, x.nj, x.split))
        run_tiles<P, Large, KB, TERMS, E>(a, b, x, e, s);
    else
        run_tiles<P, Small, KB, TERMS, E>(a, b, x, e, s);
}

// The parts' sums joined, into a gradient.
template <typename T>
void finish_rows(const float *sum, int64_t pitch, int64_t part, int parts, int64_t rows, int64_t cols,
                 const float *scale, const float *grad, const float *undo, T *out, int64_t out_pitch, hipStream_t s)
{
    const int share = parts >= 8 ? 16 : 1;
    const auto finish = share > 1 ? finish_kernel<T, 16> : finish_kernel<T, 1>;
    finish<<<dim3((uint32_t)ceil_div(rows * ceil_div(cols, 4), 256 / share)), 256, 0, s>>>(
        sum, pitch, part, parts, rows, cols, scale, grad, undo, out, out_pitch);
}

// H or rows of W as a product's operand, copied into `space` if need be.
template <typename T>
Operand<typename ProductOf<T>::P> operand(const T *src, int64_t rows, int64_t cols, int64_t pitch, bool pack,
                                          void *space, int64_t dk, hipStream_t s)
{
    typedef typename ProductOf<T>::P P;
    constexpr int64_t parts = ProductOf<T>::kParts;
    if (!pack)
        return Operand<P>{(const P *)src, rows, cols, pitch, 0};
    pack_kernel<T><<<grid_of(ceil_div(rows * (dk / 8), 256)), 256, 0, s>>>(
        src, rows, cols, pitch, (P *)space, parts * dk, dk, dk);
    return Operand<P>{(const P *)space, rows, pad(cols, 8), parts * dk, parts > 1 ? dk : 0};
}

// Calls f with the number of 16-token tiles that few tokens take and the
// waves that share the workgroup's rows.
template <int V> struct IntV { static constexpr int v = V; };
template <typename F> void with_few(int64_t tokens, int rows, F f)
{
    const auto split = [&](auto c) {
        if (rows == 64 * few_row_tiles(decltype(c)::v))
            f(c, IntV<1>{});
        else
            f(c, IntV<4>{});
    };
    if (few_tiles(tokens) == 1)
        split(IntV<1>{});
    else if (few_tiles(tokens) == 2)
        split(IntV<2>{});
    else
        split(IntV<4>{});
}

void run_loss(const float2 *part, int64_t tiles, const float *target_logit, const int64_t *targets, int64_t ignore,
              int64_t vocab, int64_t tokens, float *loss, float *lse, hipStream_t s)
{
    // a workgroup a token until those fill the device
    if (tokens <= 1024)
        loss_kernel<1><<<dim3((uint32_t)tokens), 256, 0, s>>>(part, tiles, target_logit, targets, ignore, vocab,
                                                              tokens, loss, lse);
    else
        loss_kernel<16><<<dim3((uint32_t)ceil_div(tokens, 16)), 256, 0, s>>>(part, tiles, target_logit, targets,
                                                                             ignore, vocab, tokens, loss, lse);
}

}  // namespace
}  // namespace rotor

using namespace rotor;

extern "C" {

int32_t rotor_xent_workspace_bytes(int32_t type, int64_t n_tokens, int64_t cols, int64_t n_rows, int32_t aligned,
                                   int32_t backward, uint64_t *bytes)
{
    if (!bytes || !xent_sizes_ok(type, n_tokens, cols, n_rows))
        return ROTOR_EINVAL;
    const bool pack = type == ROTOR_F32 || !aligned;
    *bytes = n_tokens == 0 ? 0
             : backward    ? backward_layout(type, n_tokens, cols, n_rows, pack).total
                           : forward_layout(type, n_tokens, cols, n_rows, pack).total;
    return ROTOR_OK;
}

int32_t rotor_xent(int32_t type, int64_t n_tokens, int64_t cols, int64_t n_rows, const void *d_h, int64_t h_pitch,
                   const void *d_w, int64_t w_pitch, const int64_t *d_targets, int64_t ignore, float *d_loss,
                   float *d_lse, int32_t aligned, void *d_work, uint64_t work_bytes, void *stream)
{
    if (!xent_sizes_ok(type, n_tokens, cols, n_rows))
        return ROTOR_EINVAL;
    const int64_t es = elem_bytes(type);
    const bool pack = type == ROTOR_F32 || !aligned;
    if (!matrix_ok(d_h, n_tokens, cols, h_pitch, es) || !matrix_ok(d_w, n_rows, cols, w_pitch, es) ||
        h_pitch > kMostPitch || w_pitch > kMostPitch)
        return ROTOR_EINVAL;
    if (n_tokens == 0)
        return ROTOR_OK;
    if (!pack && (!rows_aligned(d_h, cols, h_pitch) || !rows_aligned(d_w, cols, w_pitch)))
        return ROTOR_EINVAL;
    const ForwardLayout l = forward_layout(type, n_tokens, cols, n_rows, pack);
    if (!d_targets || (uintptr_t)d_targets % 8 || !d_loss || (uintptr_t)d_loss % 4 || !d_lse ||
        (uintptr_t)d_lse % 4 || !d_work || (uintptr_t)d_work % 16 || work_bytes < l.total)
        return ROTOR_EINVAL;
    char *const work = (char *)d_work;
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();  // an error the caller's earlier calls left behind is not this launch's
    with_type(type, [&](auto e) {
        typedef typename decltype(e)::T T;
        typedef typename ProductOf<T>::P P;
        const T *w = (const T *)d_w;
        const Operand<P> b = operand<T>((const T *)d_h, n_tokens, cols, h_pitch, pack, work + l.h, l.dk, s);
        float2 *part = (float2 *)(work + l.part);
        float *target = (float *)(work + l.target);
        if (few_tokens(type, n_tokens, n_rows, pack, false)) {
            FewArgs<T> f{};
            f.w = w;
            f.w_pitch = w_pitch;
            f.rows = n_rows;
            f.cols = cols;
            f.h = b;
            f.tokens = (int)n_tokens;
            f.targets = d_targets;
            f.part = part;
            f.target_logit = target;
            const int rows = few_rows(n_tokens, n_rows);
            const int64_t blocks = ceil_div(n_rows, rows);
            with_few(n_tokens, rows, [&](auto c, auto kw) {
                few_kernel<T, decltype(c)::v, decltype(kw)::v, false><<<dim3((uint32_t)blocks), kFewThreads, 0, s>>>(f);
            });
            run_loss(part, blocks, target, d_targets, ignore, n_rows, n_tokens, d_loss, d_lse, s);
            return;
        }
        int64_t tiles_done = 0;
        for (int64_t v0 = 0; v0 < n_rows; v0 += l.piece) {
            const int64_t rows = n_rows - v0 < l.piece ? n_rows - v0 : l.piece;
            const Operand<P> a = operand<T>(w + v0 * w_pitch, rows, cols, w_pitch, pack, work + l.w, l.dk, s);
            StatsEpilogue ep;
            ep.part = part + tiles_done * n_tokens;
            ep.target_logit = target;
            ep.targets = d_targets;
            ep.vocab = (int)rows;
            ep.tokens = (int)n_tokens;
            ep.v0 = v0;
            run_product<false, (ProductOf<T>::kParts > 1)>(a, b, Extent{rows, n_tokens, cols, 1}, ep, s);
            tiles_done += ceil_div(rows, large_tiles(rows, n_tokens, 1) ? 256 : 128);
        }
        run_loss(part, tiles_done, target, d_targets, ignore, n_rows, n_tokens, d_loss, d_lse, s);
    });
    return hipGetLastError() == hipSuccess ? ROTOR_OK : ROTOR_EDEVICE;
}

int32_t rotor_xent_backward(int32_t type, int64_t n_tokens, int64_t cols, int64_t n_rows, const void *d_h,
                            int64_t h_pitch, const void *d_w, int64_t w_pitch, const int64_t *d_targets,
                            int64_t ignore, const float *d_lse, const float *d_grad_loss, void *d_dh,
                            int64_t dh_pitch, void *d_dw, int64_t dw_pitch, int32_t aligned, void *d_work,
                            uint64_t work_bytes, void *stream)
{
    if (!xent_sizes_ok(type, n_tokens, cols, n_rows) || (!d_dh && !d_dw))
        return ROTOR_EINVAL;
    const int64_t es = elem_bytes(type);
    const bool pack = type == ROTOR_F32 || !aligned;
    if (!matrix_ok(d_h, n_tokens, cols, h_pitch, es) || !matrix_ok(d_w, n_rows, cols, w_pitch, es) ||
        h_pitch > kMostPitch || w_pitch > kMostPitch || (d_dw && dw_pitch > kMostPitch) ||
        (d_dh && !matrix_ok(d_dh, n_tokens, cols, dh_pitch, es)) ||
        (d_dw && !matrix_ok(d_dw, n_rows, cols, dw_pitch, es)))
        return ROTOR_EINVAL;
    const hipStream_t s = (hipStream_t)stream;
    if (n_tokens == 0) {
        (void)hipGetLastError();
        if (d_dw)
            with_type(type, [&](auto e) {
                typedef typename decltype(e)::T T;
                clear_kernel<T><<<dim3((uint32_t)(n_rows < 4096 ? n_rows : 4096)), 256, 0, s>>>((T *)d_dw, n_rows,
                                                                                               cols, dw_pitch);
            });
        return hipGetLastError() == hipSuccess ? ROTOR_OK : ROTOR_EDEVICE;
    }
    const BackwardLayout l = backward_layout(type, n_tokens, cols, n_rows, pack);
    if (!pack && (!rows_aligned(d_h, cols, h_pitch) || !rows_aligned(d_w, cols, w_pitch)))
        return ROTOR_EINVAL;
    if (!d_targets || (uintptr_t)d_targets % 8 || !d_lse || (uintptr_t)d_lse % 4 || !d_grad_loss ||
        (uintptr_t)d_grad_loss % 4 || !d_work || (uintptr_t)d_work % 16 || work_bytes < l.total)
        return ROTOR_EINVAL;
    char *const work = (char *)d_work;
    (void)hipGetLastError();  // an error the caller's earlier calls left behind is not this launch's
    with_type(type, [&](auto e) {
        typedef typename decltype(e)::T T;
        typedef typename ProductOf<T>::P P;
        constexpr int64_t parts = ProductOf<T>::kParts;
        float *const grad = (float *)(work + l.grad), *const scale = (float *)(work + l.scale);
        float *const sum = (float *)(work + l.sum);
        int *const order = (int *)(work + l.order), *const live = (int *)(work + l.live);
        const T *h = (const T *)d_h, *w = (const T *)d_w;
        float *const undo = type == ROTOR_F16 ? (float *)(work + l.undo) : nullptr;
        const GradArgs ga{d_grad_loss, d_targets, ignore, n_rows, n_tokens, undo ? 8 : 0, grad, scale, undo};
        const bool few = few_tokens(type, n_tokens, n_rows, pack, true);
        Operand<P> hb{(const P *)d_h, n_tokens, cols, h_pitch, 0};
        if (few) {
            FewPrepareArgs<T> f;
            f.g = ga;
            f.h = h;
            f.pitch = h_pitch;
            f.cols = cols;
            f.cols_to = l.dk;
            f.turned = d_dw ? (P *)(work + l.ht) : nullptr;
            f.packed = pack ? (P *)(work + l.h) : nullptr;
            f.rows_to = (int)l.nk;
            few_prepare_kernel<T><<<dim3((uint32_t)(l.dk / 64)), 256, 0, s>>>(f);
            if (pack)
                hb = Operand<P>{f.packed, n_tokens, pad(cols, 8), parts * l.dk, parts > 1 ? l.dk : 0};
        } else {
            const TokenArgs ta{ga, d_lse, (float *)(work + l.lse), order, (int *)(work + l.target), live};
            grad_kernel<<<dim3((uint32_t)ceil_div(n_tokens, kGradTokens)), 1024, 0, s>>>(ta);
            TurnArgs<P> t;
            t.cols = cols;
            t.pitch = h_pitch;
            t.order = order;
            t.live = live;
            t.undo = undo;
            t.packed = (P *)(work + l.h);
            t.packed_pitch = parts * l.dk;
            t.packed_seg = l.dk;
            t.turned = d_dw ? (P *)(work + l.ht) : nullptr;
            t.turned_pitch = parts * l.nk;
            t.turned_seg = l.nk;
            turn_kernel<T>
                <<<dim3((uint32_t)ceil_div(n_tokens, 64), (uint32_t)ceil_div(cols, 64)), 256, 0, s>>>(h, t);
            hb = Operand<P>{t.packed, n_tokens, pad(cols, 8), t.packed_pitch, parts > 1 ? l.dk : 0};
        }
        if (few) {
            FewArgs<T> f{};
            f.w = w;
            f.w_pitch = w_pitch;
            f.rows = n_rows;
            f.cols = cols;
            f.h = hb;
            f.tokens = (int)n_tokens;
            f.targets = d_targets;
            f.lse = d_lse;
            f.grad = grad;
            f.p = d_dh ? (P *)(work + l.p) : nullptr;
            f.p_seg = l.piece;
            f.pt = d_dw ? (P *)(work + l.pt) : nullptr;
            f.nk = (int)l.nk;
            const int rows = few_rows(n_tokens, n_rows);
            with_few(n_tokens, rows, [&](auto c, auto kw) {
                constexpr int C = decltype(c)::v;
                // all of P, past the rows of W too: the sums take 64 at a time
                few_kernel<T, C, decltype(kw)::v, true><<<dim3((uint32_t)ceil_div(l.piece, rows)), kFewThreads, 0, s>>>(
                    f);
            });
            if (d_dw) {
                FewWeightArgs<T> g;
                g.pt = f.pt;
                g.ht = (const P *)(work + l.ht);
                g.scale = scale;
                g.dw = (T *)d_dw;
                g.pitch = dw_pitch;
                g.rows = n_rows;
                g.cols = cols;
                // workgroups side by side over the columns until there are
                // four for each CU
                const int64_t x = ceil_div(n_rows, kFewRows), most = ceil_div(cols, 256), want = ceil_div(1024, x);
                const auto kernel = l.nk == 32 ? few_weight_kernel<T, 1> : few_weight_kernel<T, 2>;
                kernel<<<dim3((uint32_t)x, (uint32_t)(want < most ? want : most)), kFewThreads, 0, s>>>(g);
            }
            if (d_dh) {
                FewSumArgs<T> g;
                g.w = w;
                g.w_pitch = w_pitch;
                g.rows = n_rows;
                g.cols = cols;
                g.p = f.p;
                g.p_seg = l.piece;
                g.tokens = (int)n_tokens;
                g.sum = sum;
                g.sum_pitch = l.sum_pitch;
                g.tiles = ceil_div(ceil_div(n_rows, kFewRows), l.split);
                const auto kernel = few_tiles(n_tokens) == 1   ? few_sum_kernel<T, 1>
                                    : few_tiles(n_tokens) == 2 ? few_sum_kernel<T, 2>
                                                               : few_sum_kernel<T, 4>;
                kernel<<<dim3((uint32_t)ceil_div(cols, kFewCols), (uint32_t)l.split), kFewThreads, 0, s>>>(g);
            }
        }
        for (int64_t v0 = 0; v0 < n_rows && !few; v0 += l.piece) {
            const int64_t rows = n_rows - v0 < l.piece ? n_rows - v0 : l.piece;
            const Operand<P> wa = operand<T>(w + v0 * w_pitch, rows, cols, w_pitch, pack, work + l.w, l.dk, s);
            ProbEpilogue<T> ep;
            ep.p = (P *)(work + l.p);
            ep.pitch = (int)(parts * l.p_pitch);
            ep.seg = (int)l.p_pitch;
            ep.live = live;
            ep.lse = (const float *)(work + l.lse);
            ep.grad = grad;
            ep.targets = (const int *)(work + l.target);
            ep.v0 = (int)v0;
            ep.rows = (int)rows;
            run_product<false, (parts > 1)>(wa, hb, Extent{rows, n_tokens, cols, 1}, ep, s);
            const Operand<P> pb{(const P *)(work + l.p), n_tokens, pad(rows, 8), parts * l.p_pitch,
                                parts > 1 ? l.p_pitch : 0};
            if (d_dh) {
                SumEpilogue<kLiveA> se;
                se.c = sum;
                se.pitch = (int)l.sum_pitch;
                se.part = cols * l.sum_pitch;
                se.live = live;
                se.cols = (int)n_tokens;
                se.rows = (int)cols;
                se.add = v0 > 0;
                run_product<true>(pb, wa, Extent{n_tokens, cols, rows, l.split}, se, s);
            }
            if (d_dw) {
                const Operand<P> ha{(const P *)(work + l.ht), cols, pad(n_tokens, 8), parts * l.nk,
                                    parts > 1 ? l.nk : 0};
                if (l.w_split > 1) {
                    SumEpilogue<kLiveK> we;
                    we.live = live;
                    we.c = (float *)(work + l.w_sum);
                    we.part = rows * l.w_pitch;
                    we.pitch = (int)l.w_pitch;
                    we.cols = (int)cols;
                    we.rows = (int)rows;
                    we.add = 0;
                    run_product<true>(ha, pb, Extent{cols, rows, n_tokens, l.w_split}, we, s);
                    finish_rows(we.c, l.w_pitch, we.part, l.w_split, rows, cols, scale, nullptr, nullptr,
                                (T *)d_dw + v0 * dw_pitch, dw_pitch, s);
                } else {
                    OutEpilogue<T> oe;
                    oe.live = live;
                    oe.c = (T *)d_dw + v0 * dw_pitch;
                    oe.pitch = (int)dw_pitch;
                    oe.cols = (int)cols;
                    oe.rows = (int)rows;
                    oe.scale = scale;
                    run_product<true>(ha, pb, Extent{cols, rows, n_tokens, 1}, oe, s);
                }
            }
        }
        if (d_dh && !few) {
            const int side = l.split >= 4 ? 16 : 64;
            const auto finish = side == 16 ? turn_finish_kernel<T, 16> : turn_finish_kernel<T, 64>;
            finish<<<dim3((uint32_t)ceil_div(n_tokens, 64), (uint32_t)ceil_div(cols, side)), 256, 0, s>>>(
                sum, l.sum_pitch, cols * l.sum_pitch, l.split, n_tokens, cols, order, live, scale, undo, (T *)d_dh,
                dh_pitch);
        } else if (d_dh) {
            finish_rows(sum, l.sum_pitch, n_tokens * l.sum_pitch, l.split, n_tokens, cols, scale, grad, undo,
                        (T *)d_dh, dh_pitch, s);
        }
    });
    return hipGetLastError() == hipSuccess ? ROTOR_OK : ROTOR_EDEVICE;
}

}  // extern "C"
