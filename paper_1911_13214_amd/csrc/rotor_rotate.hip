// rotor_head_norm_rotate: norms of query and key heads and their rotation by
// position, one pass; and the gradients.
//
// A head's columns are width / 2 pairs: those that turn together and, past the
// rotated columns, the rest in pairs of no meaning.  A lane holds V adjacent
// pairs, a team of lanes (a power of two) a head, a wave 64 / team heads at a
// time of one token, whose angles it computes once.
//
// Angles.  A frequency is a 64-bit fraction of a turn, so that position times
// frequency, modulo 2^64, is the angle, exact but for the frequency's own last
// bit; a quarter turn is taken off and the rest, at most pi / 4, goes through
// the Taylor series of sine and cosine (to x^9 and x^10: within 2e-9).
#include "rotor_ops.h"

#include <math.h>

namespace rotor {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxPairs = ROTOR_ROTATE_MAX_WIDTH / 2;
// Workgroups of the gradients; each leaves one row of sums.  (4 x 4096 tokens of
// 32 + 8 heads, 128 wide, bf16: 130 us with 1280, which are all resident at once,
// 108 with 2048, 109 and twice as long a join with 4096.)
constexpr int kBlocks = 2048;

struct HeadRows {
    char *p;
    int64_t batch, token, head;  // bytes
};

struct RotateArgs {
    HeadRows in[2], out[2], grad[2];  // of q and k; gradients of the results
    const void *weight[2];
    const void *positions;
    int64_t position_batch;
    int position_bytes, norm;
    int tokens, heads[2], width, rotary, team;
    int64_t all;      // tokens of all sequences
    int turns, split; // rounds of heads, and into how many waves a token's are split
    int splits[2], blocks_q;  // gradients: the same of q and k, workgroups that take q
    float eps, by_width;  // by_width = 1 / width
    float *sums;      // [block][width]
    uint64_t frequency[kMaxPairs];
};

#if defined(__HIP_DEVICE_COMPILE__)

// Sums over teams of lanes, in registers: within four and eight lanes by their
// neighbours, then by mirrors (the lanes of a half hold the same by then), past
// 16 by swapped rows.
template <int CTRL> __device__ inline float moved(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <typename R> __device__ inline float both(const R &r)
{
    const uint32_t x = r[0], y = r[1];
    return __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
}
template <int N> __device__ inline void team_sum(float (&v)[N], int team)
{
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = f(v[i]);
    };
    if (team >= 2)
        each([](float x) { return x + moved<0xB1>(x); });
    if (team >= 4)
        each([](float x) { return x + moved<0x4E>(x); });
    if (team >= 8)
        each([](float x) { return x + moved<0x141>(x); });
    if (team >= 16)
        each([](float x) { return x + moved<0x140>(x); });
    if (team >= 32)
        each([](float x) {
            const uint32_t b = __builtin_bit_cast(uint32_t, x);
            return both(__builtin_amdgcn_permlane16_swap(b, b, false, false));
        });
    if (team >= 64)
        each([](float x) {
            const uint32_t b = __builtin_bit_cast(uint32_t, x);
            return both(__builtin_amdgcn_permlane32_swap(b, b, false, false));
        });
}

__device__ inline void turn_of(uint64_t phase, float &c, float &s)
{
    const uint64_t quarter = (phase + ((uint64_t)1 << 61)) >> 62;
    const int64_t rest = (int64_t)(phase - (quarter << 62));
    const float x = (float)(int32_t)(rest >> 30) * 3.6572952e-10f;  // 2 pi / 2^34
    const float y = x * x;
    float sn = __builtin_fmaf(y, 2.7557319e-6f, -1.9841270e-4f);
    sn = __builtin_fmaf(y, sn, 8.3333333e-3f);
    sn = __builtin_fmaf(y, sn, -1.6666667e-1f);
    sn = __builtin_fmaf(x * y, sn, x);
    float cs = __builtin_fmaf(y, -2.7557319e-7f, 2.4801587e-5f);
    cs = __builtin_fmaf(y, cs, -1.3888889e-3f);
    cs = __builtin_fmaf(y, cs, 4.1666667e-2f);
    cs = __builtin_fmaf(y, cs, -0.5f);
    cs = __builtin_fmaf(y, cs, 1.f);
    const bool odd = quarter & 1;
    c = odd ? sn : cs;
    s = odd ? cs : sn;
    c = quarter == 1 || quarter == 2 ? -c : c;
    s = quarter == 2 || quarter == 3 ? -s : s;
}

// A lane's pairs of a head.
template <typename T, int V, int N, bool INTER> struct Pairs {
    int first[N], col[N], apart[N];  // first pair; its columns
    bool have[N], turns[N];          // V divides the pairs that turn: all of them or none
    __device__ void init(const RotateArgs &a, int lane)
    {
        const int half = a.rotary / 2;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int s = (n * 64 + lane % a.team) * V;
            first[n] = s;
            have[n] = s < a.width / 2;
            turns[n] = s < half;
            if (INTER) {
                col[n] = 2 * s;
                apart[n] = 0;
            } else {
                col[n] = s < half ? s : s + half;
                apart[n] = s < half ? half : a.width / 2 - half;
            }
        }
    }
    // Loads as they are, and their conversion: what is on its way takes half the
    // registers, and nothing waits for it.
    typedef typename VecOf<T, V>::V Half;
    struct Raw {
        Half x[N][2];
    };
    __device__ void fetch(const T *p, bool row, Raw &r) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            r.x[n][0] = r.x[n][1] = Half{};
            if (row && have[n]) {
                // (interleaved: the second half lies next to the first)
                r.x[n][0] = *(const Half *)(p + col[n]);
                r.x[n][1] = *(const Half *)(p + col[n] + (INTER ? V : apart[n]));
            }
        }
    }
    __device__ void unpack(const Raw &r, float (&x)[N][2][V]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if constexpr (INTER) {
                    x[n][0][e] = (float)(2 * e < V ? r.x[n][0][2 * e % V] : r.x[n][1][2 * e % V]);
                    x[n][1][e] = (float)(2 * e + 1 < V ? r.x[n][0][(2 * e + 1) % V] : r.x[n][1][(2 * e + 1) % V]);
                } else {
                    x[n][0][e] = (float)r.x[n][0][e];
                    x[n][1][e] = (float)r.x[n][1][e];
                }
            }
    }
    __device__ void load(const T *p, bool row, float (&x)[N][2][V]) const
    {
        Raw r;
        fetch(p, row, r);
        unpack(r, x);
    }
    template <typename O> __device__ void store(O *p, bool row, const float (&x)[N][2][V]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (!row || !have[n])
                continue;
            if constexpr (INTER) {
                float f[2 * V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    f[2 * e] = x[n][0][e];
                    f[2 * e + 1] = x[n][1][e];
                }
                store_vec(p + col[n], f);
            } else {
                store_vec(p + col[n], x[n][0]);
                store_vec(p + col[n] + apart[n], x[n][1]);
            }
        }
    }
    // The angles of a position.
    __device__ void angles(const RotateArgs &a, uint64_t position, float (&c)[N][V], float (&s)[N][V]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                c[n][e] = 1.f;
                s[n][e] = 0.f;
                if (turns[n])
                    turn_of(position * a.frequency[first[n] + e], c[n][e], s[n][e]);
            }
    }
    // Rotates; what is not rotated is not touched (0 times infinity).
    __device__ void rotate(float (&x)[N][2][V], const float (&c)[N][V], const float (&s)[N][V], float way) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (turns[n]) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float u = x[n][0][e], v = x[n][1][e], t = s[n][e] * way;
                    x[n][0][e] = u * c[n][e] - v * t;
                    x[n][1][e] = v * c[n][e] + u * t;
                }
            }
    }
};

template <int V, int N, typename F> __device__ inline void each(F f)
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int e = 0; e < V; ++e)
                f(n, z, e);
}

// u less its mean, for layer norms.
template <int V, int N, typename P> __device__ inline void centre(const RotateArgs &a, const P &at, float (&u)[N][2][V])
{
    if (a.norm != ROTOR_NORM_LAYER)
        return;
    float sum[1] = {0.f};
    each<V, N>([&](int n, int z, int e) { sum[0] += u[n][z][e]; });
    team_sum(sum, a.team);
    const float mean = sum[0] * a.by_width;
    each<V, N>([&](int n, int z, int e) { u[n][z][e] = at.have[n] ? u[n][z][e] - mean : 0.f; });
}

__device__ inline uint64_t position_of(const RotateArgs &a, int64_t b, int t)
{
    if (!a.positions)
        return (uint64_t)t;
    const int64_t i = b * a.position_batch + t;
    return a.position_bytes == 8 ? (uint64_t)((const int64_t *)a.positions)[i]
                                 : (uint64_t)(int64_t)((const int32_t *)a.positions)[i];
}
__device__ inline char *token_at(const HeadRows &h, int64_t b, int t) { return h.p + b * h.batch + t * h.token; }
#endif

// A wave takes a token's heads, or where tokens are few a share of them, and
// writes each once it has its sums: bound by memory (4 x 4096 tokens of 32 + 8
// heads, 128 wide, bf16: 336 MB in 63 us, 5.3 TB/s).
template <typename T, int V, int N, bool INTER> __global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const int lane = threadIdx.x % 64;
    const int64_t task = block_at() * kWaves + threadIdx.x / 64, n = task / a.split;
    if (n >= a.all)
        return;
    const int part = (int)(task - n * a.split);
    const int64_t b = n / a.tokens;
    const int t = (int)(n - b * a.tokens), teams = 64 / a.team;
    Pairs<T, V, N, INTER> at;
    at.init(a, lane);
    const char *const in[2] = {token_at(a.in[0], b, t), token_at(a.in[1], b, t)};
    char *const out[2] = {token_at(a.out[0], b, t), token_at(a.out[1], b, t)};
    float c[N][V], s[N][V];
    at.angles(a, position_of(a, b, t), c, s);
    for (int i = part; i < a.turns; i += a.split) {
        int head = i * teams + lane / a.team;
        const bool row = head < a.heads[0] + a.heads[1], z = head >= a.heads[0];
        head -= z ? a.heads[0] : 0;
        const T *const x = (const T *)((z ? in[1] : in[0]) + head * (z ? a.in[1].head : a.in[0].head));
        T *const y = (T *)((z ? out[1] : out[0]) + head * (z ? a.out[1].head : a.out[0].head));
        float u[N][2][V];
        at.load(x, row, u);
        if (a.norm != ROTOR_NORM_NONE) {
            const T *weight = (const T *)(z ? a.weight[1] : a.weight[0]);
            float w[N][2][V];
            each<V, N>([&](int n, int q, int e) { w[n][q][e] = 1.f; });
            if (weight)
                at.load(weight, true, w);
            centre<V, N>(a, at, u);
            float sum[1] = {0.f};
            each<V, N>([&](int n, int q, int e) { sum[0] += u[n][q][e] * u[n][q][e]; });
            team_sum(sum, a.team);
            const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(sum[0], a.by_width, a.eps));
            each<V, N>([&](int n, int q, int e) { u[n][q][e] *= r * w[n][q][e]; });
        }
        at.rotate(u, c, s, 1.f);
        at.store(y, row, u);
    }
#endif
}

// The first `blocks_q` workgroups take the heads of q, the others those of k:
// the sums of one weight's gradient fit the registers.  The next heads' loads are
// under way while one round's sums cross the team (the forward case's sizes: 503
// MB in 108 us, 4.65 TB/s; the weights read anew each round, and workgroups in
// proportion to the heads alone, 137 us).
template <typename T, int V, int N, bool INTER>
__global__ __launch_bounds__(kThreads) void rotate_back_kernel(RotateArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), teams = 64 / a.team;
    const int z = (int)blockIdx.x >= a.blocks_q ? 1 : 0, block = blockIdx.x - (z ? a.blocks_q : 0);
    const int heads = a.heads[z], split = a.splits[z];
    const int64_t stride = (int64_t)(z ? gridDim.x - a.blocks_q : a.blocks_q) * kWaves;
    const T *weight = (const T *)a.weight[z];
    const HeadRows in = a.in[z], out = a.out[z], grad = a.grad[z];
    Pairs<T, V, N, INTER> at;
    at.init(a, lane);
    typename Pairs<T, V, N, INTER>::Raw weights;
    at.fetch(weight, weight != nullptr, weights);
    float sums[N][2][V];
    each<V, N>([&](int p, int q, int e) { sums[p][q][e] = 0.f; });
    for (int64_t task = (int64_t)block * kWaves + wave; task < a.all * split; task += stride) {
        const int64_t n = task / split, b = n / a.tokens;
        const int t = (int)(n - b * a.tokens), part = (int)(task - n * split);
        const char *const grad_at = token_at(grad, b, t), *const in_at = token_at(in, b, t);
        char *const out_at = token_at(out, b, t);
        typename Pairs<T, V, N, INTER>::Raw next_g, next_u;
        auto fetch = [&](int i) {
            const int head = i + lane / a.team;
            at.fetch((const T *)(grad_at + head * grad.head), head < heads, next_g);
            if (a.norm != ROTOR_NORM_NONE)
                at.fetch((const T *)(in_at + head * in.head), head < heads, next_u);
        };
        fetch(part * teams);
        float c[N][V], s[N][V];
        at.angles(a, position_of(a, b, t), c, s);
        for (int i = part * teams; i < heads; i += split * teams) {
            const int head = i + lane / a.team;
            const bool row = head < heads;
            float g[N][2][V], u[N][2][V];
            at.unpack(next_g, g);
            if (a.norm != ROTOR_NORM_NONE)
                at.unpack(next_u, u);
            if (i + split * teams < heads)
                fetch(i + split * teams);
            if (a.norm != ROTOR_NORM_NONE) {
                float w[N][2][V];
                each<V, N>([&](int p, int q, int e) { w[p][q][e] = 1.f; });
                if (weight)
                    at.unpack(weights, w);
                at.rotate(g, c, s, -1.f);
                centre<V, N>(a, at, u);
                // of u^2, of the weighted gradient times u, and of it alone
                float sum[3] = {0.f, 0.f, 0.f};
                each<V, N>([&](int p, int q, int e) {
                    const float y = g[p][q][e] * w[p][q][e];
                    sum[0] += u[p][q][e] * u[p][q][e];
                    sum[1] += y * u[p][q][e];
                    sum[2] += y;
                });
                team_sum(sum, a.team);
                const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(sum[0], a.by_width, a.eps));
                const float dot = sum[1] * r * a.by_width;
                const float mean = a.norm == ROTOR_NORM_LAYER ? sum[2] * a.by_width : 0.f;
                each<V, N>([&](int p, int q, int e) {
                    const float v = u[p][q][e] * r;  // (0 where there is no head)
                    sums[p][q][e] += row ? g[p][q][e] * v : 0.f;
                    g[p][q][e] = r * (g[p][q][e] * w[p][q][e] - mean - v * dot);
                });
            } else {
                at.rotate(g, c, s, -1.f);
            }
            at.store((T *)(out_at + head * out.head), row, g);
        }
    }
    if (!a.sums)
        return;
    // over the teams, then over the waves in order
    __shared__ float lines[kWaves][ROTOR_ROTATE_MAX_WIDTH];
    each<V, N>([&](int p, int q, int e) {
        for (int off = a.team; off < 64; off *= 2)
            sums[p][q][e] += __shfl_xor(sums[p][q][e], off);
    });
    at.store(lines[wave], lane < a.team, sums);
    __syncthreads();
    for (int col = threadIdx.x; col < a.width; col += kThreads) {
        float v = lines[0][col];
#pragma unroll
        for (int k = 1; k < kWaves; ++k)
            v += lines[k][col];
        a.sums[(int64_t)blockIdx.x * a.width + col] = v;
    }
#endif
}

// The blocks' sums joined in their order: 16 columns a workgroup, 64 strips of
// blocks, joined by eights (16 strips: 8 us for 2048 rows of 128, these 5, of which
// the launch is most); blockIdx.y: q, k.
constexpr int kStrips = 64, kEights = kStrips / 8;

template <typename T>
__global__ __launch_bounds__(16 * kStrips) void join_kernel(const float *sums, int blocks_q, int blocks, int width,
                                                            T *dq, T *dk)
{
    __shared__ float strip[kStrips][16], eights[kEights][16];
    const int lane = threadIdx.x % 16, col = blockIdx.x * 16 + lane, k = threadIdx.x / 16, z = blockIdx.y;
    const int end = z ? blocks : blocks_q;
    float v = 0.f;
    if (col < width)
#pragma unroll 8
        for (int i = (z ? blocks_q : 0) + k; i < end; i += kStrips)
            v += sums[(int64_t)i * width + col];
    strip[k][lane] = v;
    __syncthreads();
    if (k < kEights) {
        v = strip[8 * k][lane];
#pragma unroll
        for (int i = 1; i < 8; ++i)
            v += strip[8 * k + i][lane];
        eights[k][lane] = v;
    }
    __syncthreads();
    T *const out = z ? dk : dq;
    if (k == 0 && col < width && out) {
#pragma unroll
        for (int i = 1; i < kEights; ++i)
            v += eights[i][lane];
        out[col] = (T)v;
    }
}

bool rotation_ok(const rotor_head_rotation *n)
{
    return n && type_ok(n->type) && n->norm >= ROTOR_NORM_NONE && n->norm <= ROTOR_NORM_LAYER &&
           (n->interleaved == 0 || n->interleaved == 1) && n->batch >= 0 && n->tokens >= 0 && n->heads >= 1 &&
           n->kv_heads >= 0 && n->heads <= 1 << 20 && n->kv_heads <= 1 << 20 && n->width >= 2 &&
           n->width <= ROTOR_ROTATE_MAX_WIDTH && n->width % 2 == 0 && n->rotary >= 0 && n->rotary <= n->width &&
           n->rotary % 2 == 0 && n->eps >= 0. && n->tokens < ((int64_t)1 << 31) &&
           (unsigned __int128)n->batch * (unsigned __int128)n->tokens < ((uint64_t)1 << 40);
}

bool head_rows_ok(const rotor_heads *h, const rotor_head_rotation *n, int64_t heads, HeadRows &out)
{
    out = HeadRows{nullptr, 0, 0, 0};
    if (heads == 0 || n->batch == 0 || n->tokens == 0)
        return true;
    const int64_t es = elem_bytes(n->type);
    if (!h || !h->p || (uintptr_t)h->p % (uintptr_t)es)
        return false;
    const int64_t count[3] = {n->batch, n->tokens, heads}, s[3] = {h->batch, h->token, h->head};
    int64_t by[3];
    for (int i = 0; i < 3; ++i) {
        by[i] = count[i] == 1 ? 0 : s[i];
        if (by[i] < 0 || (unsigned __int128)by[i] * (unsigned __int128)count[i] >= ((unsigned __int128)1 << 58))
            return false;
        by[i] *= es;
    }
    out = HeadRows{(char *)h->p, by[0], by[1], by[2]};
    return true;
}

template <int N> struct Num {
    static constexpr int v = N;
};

// Adjacent pairs of a lane: four where they divide both parts of a head (with
// eight, whole 16 bytes of 16-bit columns, the registers leave fewer waves: 4 x
// 4096 tokens of 32 + 8 heads, 128 wide, bf16, gradients: 205 us, with four 157).
int pairs_of(const rotor_head_rotation *n)
{
    for (int v = 4; v > 1; v /= 2)
        if (n->width / 2 % v == 0 && n->rotary / 2 % v == 0)
            return v;
    return 1;
}

template <typename F> void with_pairs(const rotor_head_rotation *n, F f)
{
    const int v = pairs_of(n);
    if (n->interleaved) {
        if (v == 4)
            f(Num<4>{}, Num<1>{}, Num<1>{});
        else if (v == 2)
            f(Num<2>{}, Num<1>{}, Num<1>{});
        else
            f(Num<1>{}, Num<2>{}, Num<1>{});
    } else {
        if (v == 4)
            f(Num<4>{}, Num<1>{}, Num<0>{});
        else if (v == 2)
            f(Num<2>{}, Num<1>{}, Num<0>{});
        else
            f(Num<1>{}, Num<2>{}, Num<0>{});
    }
}

bool fill(RotateArgs &a, const rotor_head_rotation *n)
{
    const int64_t es = elem_bytes(n->type);
    if ((n->rotary > 0 && !n->frequencies) || (n->norm == ROTOR_NORM_NONE && (n->q_weight || n->k_weight)) ||
        (uintptr_t)n->q_weight % (uintptr_t)es || (uintptr_t)n->k_weight % (uintptr_t)es || n->position_batch < 0 ||
        (n->positions && ((n->position_bytes != 4 && n->position_bytes != 8) ||
                          (uintptr_t)n->positions % (uintptr_t)n->position_bytes)))
        return false;
    for (int64_t i = 0; i < n->rotary / 2; ++i) {
        const double f = n->frequencies[i];
        if (!isfinite(f))
            return false;
        // as a fraction of a turn; of less than half a turn it is one product
        long double turn = (long double)f * 0.15915494309189533576888376337251436L;
        if (!(fabs(f) < 3.14)) {
            turn -= floorl(turn);
            turn -= turn >= 0.5L ? 1.L : 0.L;
        }
        a.frequency[i] = (uint64_t)(int64_t)(turn * 18446744073709551616.0L);
    }
    a.weight[0] = n->q_weight;
    a.weight[1] = n->k_weight;
    a.positions = n->positions;
    a.position_batch = n->position_batch;
    a.position_bytes = n->position_bytes;
    a.norm = n->norm;
    a.tokens = (int)n->tokens;
    a.heads[0] = (int)n->heads;
    a.heads[1] = (int)n->kv_heads;
    a.width = (int)n->width;
    a.rotary = (int)n->rotary;
    a.all = n->batch * n->tokens;
    a.eps = (float)n->eps;
    a.by_width = 1.f / (float)n->width;
    a.sums = nullptr;
    const int lanes = (int)n->width / 2 / pairs_of(n);
    a.team = 1;
    while (a.team < lanes && a.team < 64)
        a.team *= 2;
    return true;
}

// Waves among which a token's heads are split: all of a token's in one wave
// compute its angles once, but few tokens leave CUs without work.
int split_of(int64_t all, int turns)
{
    const int64_t want = all > 0 ? 8192 / all : 1;
    return (int)(want < 1 || turns < 1 ? 1 : want > turns ? turns : want);
}

}  // namespace
}  // namespace rotor

using namespace rotor;

extern "C" {

int32_t rotor_head_norm_rotate(const rotor_head_rotation *how, const rotor_heads *q, const rotor_heads *k,
                               const rotor_heads *q_out, const rotor_heads *k_out, void *stream)
{
    RotateArgs a;
    if (!rotation_ok(how) || !fill(a, how) || !head_rows_ok(q, how, how->heads, a.in[0]) ||
        !head_rows_ok(k, how, how->kv_heads, a.in[1]) || !head_rows_ok(q_out, how, how->heads, a.out[0]) ||
        !head_rows_ok(k_out, how, how->kv_heads, a.out[1]))
        return ROTOR_EINVAL;
    a.grad[0] = a.grad[1] = HeadRows{nullptr, 0, 0, 0};
    if (a.all == 0)
        return ROTOR_OK;
    a.turns = (int)ceil_div(a.heads[0] + a.heads[1], 64 / a.team);
    a.split = split_of(a.all, a.turns);
    const int64_t blocks = ceil_div(a.all * a.split, kWaves);
    if (!grid_ok(blocks))
        return ROTOR_EINVAL;
    (void)hipGetLastError();  // an error the caller's earlier calls left behind is not this launch's
    with_type(how->type, [&](auto e) {
        typedef typename decltype(e)::T T;
        with_pairs(how, [&](auto v, auto n, auto inter) {
            rotate_kernel<T, decltype(v)::v, decltype(n)::v, decltype(inter)::v == 1>
                <<<grid_of(blocks), kThreads, 0, (hipStream_t)stream>>>(a);
        });
    });
    return hipGetLastError() == hipSuccess ? ROTOR_OK : ROTOR_EDEVICE;
}

int32_t rotor_head_norm_rotate_workspace_bytes(const rotor_head_rotation *how, uint64_t *bytes)
{
    if (!bytes || !rotation_ok(how))
        return ROTOR_EINVAL;
    *bytes = how->norm == ROTOR_NORM_NONE ? 0 : (uint64_t)kBlocks * how->width * 4;
    return ROTOR_OK;
}

int32_t rotor_head_norm_rotate_backward(const rotor_head_rotation *how, const rotor_heads *dq_out,
                                        const rotor_heads *dk_out, const rotor_heads *q, const rotor_heads *k,
                                        const rotor_heads *dq, const rotor_heads *dk, void *d_dq_weight,
                                        void *d_dk_weight, void *d_work, uint64_t work_bytes, void *stream)
{
    RotateArgs a;
    uint64_t need = 0;
    if (!rotation_ok(how) || !fill(a, how) ||
        rotor_head_norm_rotate_workspace_bytes(how, &need) != ROTOR_OK)
        return ROTOR_EINVAL;
    const int64_t es = elem_bytes(how->type);
    a.in[0] = a.in[1] = HeadRows{nullptr, 0, 0, 0};
    if (!head_rows_ok(dq_out, how, how->heads, a.grad[0]) || !head_rows_ok(dk_out, how, how->kv_heads, a.grad[1]) ||
        (how->norm != ROTOR_NORM_NONE &&
         (!head_rows_ok(q, how, how->heads, a.in[0]) || !head_rows_ok(k, how, how->kv_heads, a.in[1]))) ||
        !head_rows_ok(dq, how, how->heads, a.out[0]) || !head_rows_ok(dk, how, how->kv_heads, a.out[1]) ||
        (uintptr_t)d_dq_weight % (uintptr_t)es || (uintptr_t)d_dk_weight % (uintptr_t)es ||
        (how->norm == ROTOR_NORM_NONE && (d_dq_weight || d_dk_weight)))
        return ROTOR_EINVAL;
    const bool sums = d_dq_weight || d_dk_weight;
    if (sums && (!d_work || (uintptr_t)d_work % 16 || work_bytes < need))
        return ROTOR_EINVAL;
    // workgroups by the rounds of heads of each and two more a token, for its
    // angles and the first loads; one at least
    const int teams = 64 / a.team;
    int64_t want[2], cost[2];
    for (int z = 0; z < 2; ++z) {
        const int64_t rounds = ceil_div(a.heads[z], teams);
        a.splits[z] = split_of(a.all, (int)rounds);
        cost[z] = a.heads[z] ? rounds + 2 * a.splits[z] : 0;
        want[z] = ceil_div(a.all * (a.heads[z] ? a.splits[z] : 0), kWaves);
    }
    for (int z = 0; z < 2; ++z) {
        const int64_t most = kBlocks * cost[z] / (cost[0] + cost[1]);
        want[z] = want[z] > 0 && want[z] > most ? (most > 1 ? most : 1) : want[z];
    }
    a.blocks_q = (int)want[0];
    const int blocks = (int)(want[0] + want[1]);
    a.sums = sums ? (float *)d_work : nullptr;
    (void)hipGetLastError();  // an error the caller's earlier calls left behind is not this launch's
    with_type(how->type, [&](auto e) {
        typedef typename decltype(e)::T T;
        if (blocks > 0)
            with_pairs(how, [&](auto v, auto n, auto inter) {
                rotate_back_kernel<T, decltype(v)::v, decltype(n)::v, decltype(inter)::v == 1>
                    <<<dim3((uint32_t)blocks), kThreads, 0, (hipStream_t)stream>>>(a);
            });
        if (sums)
            join_kernel<T><<<dim3((uint32_t)ceil_div(how->width, 16), 2), 16 * kStrips, 0, (hipStream_t)stream>>>(
                a.sums, a.blocks_q, blocks, a.width, (T *)d_dq_weight, (T *)d_dk_weight);
    });
    return hipGetLastError() == hipSuccess ? ROTOR_OK : ROTOR_EDEVICE;
}

}  // extern "C"
