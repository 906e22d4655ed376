// rotor_residual_norm: y = a x + gate * post(z), h = pre(y), and the
// gradients of all it takes.
//
// A row is held in the registers of its threads (64 to 1024 of them, 8
// elements each, 16 past 8192 columns), so each tensor is read once and written
// once in either direction.  Backward, a workgroup walks a strip of rows and
// keeps the sums over rows (weights, biases, gate) in registers; the strips'
// sums are added by a second launch.  Past 4096 columns the registers do not
// hold both: the rows' gradients and the sums over rows are launches of their
// own.
#include "rotor_ops.h"

#include <type_traits>

namespace rotor {
namespace {

constexpr int kVec = 8;

struct NormArgs {
    int64_t rows, cols, x_pitch, z_pitch, y_pitch, h_pitch, gate_pitch;
    int64_t group;  // rows of one gate row
    int post, pre;
    float a, eps;
    const void *post_w, *post_b, *gate, *pre_w, *pre_b;
    float *stats;
};

// The threads of one row: TH of them; rows of one wave four side by side in a
// workgroup.
template <int TH> struct Team {
    static constexpr int kRows = TH > 64 ? 1 : 4;
    static constexpr int kBlock = TH * kRows;
};

// Sums of two values over the threads of a row.  `red` has two halves, used
// in turn, so that one barrier per sum is enough.
template <int TH> __device__ inline void row_sum2(float &u, float &v, float (*red)[16][2], int &half)
{
    u = wave_sum(u);
    v = wave_sum(v);
    if (TH == 64)
        return;
    const int wave = threadIdx.x / 64;
    if (threadIdx.x % 64 == 0) {
        red[half][wave][0] = u;
        red[half][wave][1] = v;
    }
    __syncthreads();
    u = v = 0.f;
#pragma unroll
    for (int w = 0; w < TH / 64; ++w) {
        u += red[half][w][0];
        v += red[half][w][1];
    }
    half ^= 1;
}

template <int TH> __device__ inline float row_sum(float u, float (*red)[16][2], int &half)
{
    float v = 0.f;
    row_sum2<TH>(u, v, red, half);
    return u;
}

// The pieces of a row that a thread holds: N pieces of V columns.  The last
// piece of a row is moved back to end with the row; its first `dup` columns
// are the piece before's, computed twice but counted once in sums.
template <int TH, int V, int N> struct Pieces {
    int col[N], dup[N];
    bool in[N];
    __device__ Pieces(int t, int cols)
    {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int c = (k * TH + t) * V;
            in[k] = c < cols;
            col[k] = in[k] ? (c < cols - V ? c : cols - V) : 0;
            dup[k] = in[k] ? c - col[k] : V;
        }
    }
};

template <typename T, int V, int N> struct Row {
    float f[N][V];
    template <typename P> __device__ void load(const P &p, const T *src)
    {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (p.in[k])
                load_vec(src + p.col[k], f[k]);
            else
#pragma unroll
                for (int j = 0; j < V; ++j)
                    f[k][j] = 0.f;
    }
    template <typename P> __device__ void store(const P &p, T *dst) const
    {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (p.in[k])
                store_vec(dst + p.col[k], f[k]);
    }
};

// A row as it is stored, or a constant where there is none (src is NULL).
template <typename T, int V, int N> struct Param {
    typedef typename VecOf<T, V>::V Vec;
    Vec v[N];
    template <typename P> __device__ void load(const P &p, const T *src, float otherwise)
    {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (src && p.in[k])
                v[k] = *(const Vec *)(src + p.col[k]);
            else
#pragma unroll
                for (int j = 0; j < V; ++j)
                    v[k][j] = (T)otherwise;
        }
    }
    __device__ float at(int k, int j) const { return (float)v[k][j]; }
};

#define FOR_ELEMENTS                                                                                                  \
    _Pragma("unroll") for (int k = 0; k < N; ++k) _Pragma("unroll") for (int j = 0; j < V; ++j)

// Mean and 1 / deviation of a row (kind RMS or LAYER).
template <int TH, int V, int N, typename P>
__device__ inline void row_stats(int kind, const float (&u)[N][V], const P &p, float cols, float eps, float &mean,
                                 float &rstd, float (*red)[16][2], int &half)
{
    mean = 0.f;
    if (kind == ROTOR_NORM_LAYER) {
        float s = 0.f;
        FOR_ELEMENTS
        if (j >= p.dup[k])
            s += u[k][j];
        mean = row_sum<TH>(s, red, half) / cols;
    }
    float q = 0.f;
    FOR_ELEMENTS
    if (j >= p.dup[k])
        q += (u[k][j] - mean) * (u[k][j] - mean);
    rstd = 1.f / sqrtf(row_sum<TH>(q, red, half) / cols + eps);
}

// Bound by memory, with the sums in registers and one barrier each (none in
// rows of a wave): 16384 x 2048 bf16, two norms and a gate, 53 us (268 MB, 5.1
// TB/s); 4096 x 1024 f32, LayerNorm, 14 us (67 MB, 4.7 TB/s).
template <typename T, int TH, int V, int N>
__global__ __launch_bounds__(Team<TH>::kBlock) void norm_kernel(const T *x, const T *z, T *y, T *h, NormArgs a)
{
    __shared__ float red[2][16][2];
    int half = 0;
    const int t = threadIdx.x % TH;
    const int64_t r = block_at() * Team<TH>::kRows + threadIdx.x / TH;
    if (r >= a.rows)
        return;  // whole waves, and no barrier where a workgroup holds several rows
    const Pieces<TH, V, N> p(t, (int)a.cols);
    const float cols = (float)a.cols;
    Row<T, V, N> u, b;
    u.load(p, x + r * a.x_pitch);
    float mean1 = 0.f, rstd1 = 1.f, mean2 = 0.f, rstd2 = 1.f;
    FOR_ELEMENTS u.f[k][j] *= a.a;
    if (z) {
        b.load(p, z + r * a.z_pitch);
        Param<T, V, N> w, c, g;
        w.load(p, (const T *)a.post_w, 1.f);
        c.load(p, (const T *)a.post_b, 0.f);
        g.load(p, a.gate ? (const T *)a.gate + r / a.group * a.gate_pitch : nullptr, 1.f);
        if (a.post != ROTOR_NORM_NONE)
            row_stats<TH, V, N>(a.post, b.f, p, cols, a.eps, mean1, rstd1, red, half);
        FOR_ELEMENTS u.f[k][j] += g.at(k, j) * ((b.f[k][j] - mean1) * rstd1 * w.at(k, j) + c.at(k, j));
    }
    if (y)
        u.store(p, y + r * a.y_pitch);
    if (h) {
        Param<T, V, N> w, c;
        w.load(p, (const T *)a.pre_w, 1.f);
        c.load(p, (const T *)a.pre_b, 0.f);
        row_stats<TH, V, N>(a.pre, u.f, p, cols, a.eps, mean2, rstd2, red, half);
        Row<T, V, N> out;
        FOR_ELEMENTS out.f[k][j] = (u.f[k][j] - mean2) * rstd2 * w.at(k, j) + c.at(k, j);
        out.store(p, h + r * a.h_pitch);
        // The backward takes the normed row from y as it was rounded.  Where
        // that rounding passes 1/64 of the row's deviation (a LayerNorm of a
        // row whose mean is far from 0; its square, 2^-12, would show in the
        // gradient), or the deviation is below sqrt(eps), those values and
        // y's own statistics no longer make a row of mean 0 and deviation 1:
        // the backward then gets the statistics of the rounded values.
        constexpr float kUnit = sizeof(T) == 4 ? 0.f : std::is_same<T, f16>::value ? 0x1p-11f : 0x1p-8f;
        if (a.stats && sizeof(T) == 2 && a.pre == ROTOR_NORM_LAYER &&
            (fabsf(mean2) * rstd2 * kUnit > 0x1p-6f || rstd2 * rstd2 * a.eps > 0.5f)) {
            FOR_ELEMENTS u.f[k][j] = (float)(T)u.f[k][j];
            row_stats<TH, V, N>(a.pre, u.f, p, cols, a.eps, mean2, rstd2, red, half);
        }
    }
    if (a.stats && t == 0)
        *(float4 *)(a.stats + 4 * r) = make_float4(mean1, rstd1, mean2, rstd2);
}

// ---- backward -------------------------------------------------------------------

// Sums over rows.  A group's rows (those of one gate row) are cut into
// `per_group` strips of `strip` rows; a workgroup walks `per_block` strips,
// keeps the sums of the weights and biases over all of them and those of the
// gate over each.
enum { kPostW, kPostB, kPreW, kPreB, kGate, kSums };

struct StripPlan {
    int64_t group, groups, strip, per_group, strips, per_block, blocks;
};

struct BackArgs {
    int64_t rows, cols, dy_pitch, dh_pitch, y_pitch, z_pitch, dx_pitch, dz_pitch, gate_pitch, dgate_pitch;
    int post, pre;
    float a;
    const void *post_w, *post_b, *gate, *pre_w;
    const float *stats;
    float *part[kSums];  // [blocks][cols], gate: [strips][cols]; NULL: not wanted
    void *dgate;         // written here if each group is one strip (part[kGate] is NULL then)
    float2 *row_sums;    // of wide rows: means of d and d n of each row's pre norm
    StripPlan plan;
};

// A strip's sums of all rows of the workgroup, to one row of `dst`: in the
// order of the rows side by side.
template <int TH, int V, int N, typename D>
__device__ inline void put_sums(const float (&s)[N][V], const Pieces<TH, V, N> &p, D *dst, float (*buf)[TH * V * N])
{
    constexpr int R = Team<TH>::kRows;
    const int t = threadIdx.x % TH, row = threadIdx.x / TH;
    float v[N][V];
    FOR_ELEMENTS v[k][j] = s[k][j];
    if (R > 1) {
        __syncthreads();
        FOR_ELEMENTS buf[row][(k * V + j) * TH + t] = s[k][j];
        __syncthreads();
        if (row > 0)
            return;
        FOR_ELEMENTS
        {
            for (int o = 1; o < R; ++o)
                v[k][j] += buf[o][(k * V + j) * TH + t];
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (p.in[k])
            store_vec(dst + p.col[k], v[k]);
}

// Bound by memory: 16384 x 2048 bf16, two norms and a gate for each 2048 rows,
// 86 us (403 MB, 4.7 TB/s; 162 us without the next row's loads under the
// present one's work); 4096 x 1024 f32, LayerNorm, 20 us (101 MB, 5.0 TB/s).
template <typename T, int TH, int V, int N>
__global__ __launch_bounds__(Team<TH>::kBlock) void back_kernel(const T *dy, const T *dh, const T *y, const T *z,
                                                                 T *dx, T *dz, BackArgs a)
{
    constexpr int R = Team<TH>::kRows;
    __shared__ float red[2][16][2];
    __shared__ float buf[R > 1 ? R : 1][R > 1 ? TH * V * N : 1];
    float(*sums_buf)[TH * V * N] = (float(*)[TH * V * N])buf;
    int half = 0;
    const int t = threadIdx.x % TH, row = threadIdx.x / TH;
    const Pieces<TH, V, N> p(t, (int)a.cols);
    const float inv = 1.f / (float)a.cols;
    const bool gate_sums = a.part[kGate] || a.dgate;
    Param<T, V, N> w1, b1, w2, g;
    w1.load(p, (const T *)a.post_w, 1.f);
    b1.load(p, (const T *)a.post_b, 0.f);
    w2.load(p, (const T *)a.pre_w, 1.f);
    float s_post_w[N][V] = {}, s_post_b[N][V] = {}, s_pre_w[N][V] = {}, s_pre_b[N][V] = {}, s_gate[N][V] = {};
    // a row is loaded, as it is stored, while the one before is worked on
    Param<T, V, N> next_d, next_u, next_q, next_v;
    float4 next_st;
    auto fetch = [&](int64_t r) {
        next_d.load(p, dh ? dh + r * a.dh_pitch : nullptr, 0.f);
        next_u.load(p, dh ? y + r * a.y_pitch : nullptr, 0.f);
        next_q.load(p, dy ? dy + r * a.dy_pitch : nullptr, 0.f);
        next_v.load(p, z ? z + r * a.z_pitch : nullptr, 0.f);
        next_st = *(const float4 *)(a.stats + 4 * r);
    };
    const int64_t s0 = (int64_t)blockIdx.x * a.plan.per_block;
    const int64_t s1 = s0 + a.plan.per_block < a.plan.strips ? s0 + a.plan.per_block : a.plan.strips;
    for (int64_t s = s0; s < s1; ++s) {
        const int64_t group = s / a.plan.per_group;
        const int64_t in_group = (s - group * a.plan.per_group) * a.plan.strip;
        const int64_t r0 = group * a.plan.group + in_group;
        const int64_t n = in_group + a.plan.strip < a.plan.group ? a.plan.strip : a.plan.group - in_group;
        g.load(p, a.gate ? (const T *)a.gate + group * a.gate_pitch : nullptr, 1.f);
        if (row < n)
            fetch(r0 + row);
        for (int64_t i = row; i < n; i += R) {
            const int64_t r = r0 + i;
            Row<T, V, N> d, u, q, v;
            FOR_ELEMENTS
            {
                d.f[k][j] = next_d.at(k, j);
                u.f[k][j] = next_u.at(k, j);
                q.f[k][j] = next_q.at(k, j);
                v.f[k][j] = next_v.at(k, j);
            }
            const float4 st = next_st;
            if (i + R < n)
                fetch(r + R);
            if (dh) {
                float c1 = 0.f, c2 = 0.f;
                FOR_ELEMENTS
                {
                    u.f[k][j] = (u.f[k][j] - st.z) * st.w;
                    if (p.in[k]) {
                        s_pre_w[k][j] += d.f[k][j] * u.f[k][j];
                        s_pre_b[k][j] += d.f[k][j];
                    }
                    d.f[k][j] *= w2.at(k, j);
                    if (j >= p.dup[k]) {
                        c1 += d.f[k][j];
                        c2 += d.f[k][j] * u.f[k][j];
                    }
                }
                row_sum2<TH>(c1, c2, red, half);
                c1 = a.pre == ROTOR_NORM_LAYER ? c1 * inv : 0.f;
                c2 *= inv;
                FOR_ELEMENTS q.f[k][j] += st.w * (d.f[k][j] - c1 - u.f[k][j] * c2);
            }
            // q: the gradient of y, complete
            if (z) {
                float c1 = 0.f, c2 = 0.f;
                FOR_ELEMENTS
                {
                    v.f[k][j] = (v.f[k][j] - st.x) * st.y;
                    d.f[k][j] = g.at(k, j) * q.f[k][j];
                    if (p.in[k]) {
                        s_gate[k][j] += q.f[k][j] * (v.f[k][j] * w1.at(k, j) + b1.at(k, j));
                        s_post_w[k][j] += d.f[k][j] * v.f[k][j];
                        s_post_b[k][j] += d.f[k][j];
                    }
                    d.f[k][j] *= w1.at(k, j);
                    if (j >= p.dup[k]) {
                        c1 += d.f[k][j];
                        c2 += d.f[k][j] * v.f[k][j];
                    }
                }
                if (a.post != ROTOR_NORM_NONE) {
                    row_sum2<TH>(c1, c2, red, half);
                    c1 = a.post == ROTOR_NORM_LAYER ? c1 * inv : 0.f;
                    c2 *= inv;
                    FOR_ELEMENTS d.f[k][j] = st.y * (d.f[k][j] - c1 - v.f[k][j] * c2);
                }
                d.store(p, dz + r * a.dz_pitch);
            }
            FOR_ELEMENTS q.f[k][j] *= a.a;
            q.store(p, dx + r * a.dx_pitch);
        }
        if (gate_sums) {
            if (a.dgate)
                put_sums<TH, V, N>(s_gate, p, (T *)a.dgate + group * a.dgate_pitch, sums_buf);
            else
                put_sums<TH, V, N>(s_gate, p, a.part[kGate] + s * a.cols, sums_buf);
            FOR_ELEMENTS s_gate[k][j] = 0.f;
        }
    }
    const int64_t at = (int64_t)blockIdx.x * a.cols;
    if (a.part[kPostW])
        put_sums<TH, V, N>(s_post_w, p, a.part[kPostW] + at, sums_buf);
    if (a.part[kPostB])
        put_sums<TH, V, N>(s_post_b, p, a.part[kPostB] + at, sums_buf);
    if (a.part[kPreW])
        put_sums<TH, V, N>(s_pre_w, p, a.part[kPreW] + at, sums_buf);
    if (a.part[kPreB])
        put_sums<TH, V, N>(s_pre_b, p, a.part[kPreB] + at, sums_buf);
}

// The gradients of wide rows, a workgroup a row.  With the sums over rows
// beside them in one launch of 512 to 1024 threads with 16 elements each,
// registers spilled: 8192 x 5120 bf16 450 us, 3000 x 12288 2243 us; the two
// launches 183 and 172 us (ten tensors moved instead of six, 4.3 to 4.7 TB/s).
// In one launch with 8 elements a thread (the same two of bf16, then f32, in one
// launch and in two): 8192 x 5120 147 and 183, 585 and 327 us; 4096 x 6144 88 and
// 104, 415 and 203; 4096 x 8192, where every shape spills most, 369 and 138, 1011
// and 263.
template <typename T, int TH, int V, int N>
__global__ __launch_bounds__(TH) void wide_row_kernel(const T *dy, const T *dh, const T *y, const T *z, T *dx, T *dz,
                                                      BackArgs a)
{
    __shared__ float red[2][16][2];
    int half = 0;
    const int64_t r = block_at();
    if (r >= a.rows)
        return;  // the whole workgroup
    const Pieces<TH, V, N> p(threadIdx.x, (int)a.cols);
    const float inv = 1.f / (float)a.cols;
    const float4 st = *(const float4 *)(a.stats + 4 * r);
    Param<T, V, N> in_d, in_u, in_q, in_v;
    in_d.load(p, dh ? dh + r * a.dh_pitch : nullptr, 0.f);
    in_u.load(p, dh ? y + r * a.y_pitch : nullptr, 0.f);
    in_q.load(p, dy ? dy + r * a.dy_pitch : nullptr, 0.f);
    in_v.load(p, z ? z + r * a.z_pitch : nullptr, 0.f);
    Row<T, V, N> d, q;
    FOR_ELEMENTS q.f[k][j] = in_q.at(k, j);
    if (dh) {
        Param<T, V, N> w2;
        w2.load(p, (const T *)a.pre_w, 1.f);
        float c1 = 0.f, c2 = 0.f;
        FOR_ELEMENTS
        {
            d.f[k][j] = in_d.at(k, j) * w2.at(k, j);
            if (j >= p.dup[k]) {
                c1 += d.f[k][j];
                c2 += d.f[k][j] * ((in_u.at(k, j) - st.z) * st.w);
            }
        }
        row_sum2<TH>(c1, c2, red, half);
        c1 = a.pre == ROTOR_NORM_LAYER ? c1 * inv : 0.f;
        c2 *= inv;
        if (threadIdx.x == 0)
            a.row_sums[r] = make_float2(c1, c2);
        FOR_ELEMENTS q.f[k][j] += st.w * (d.f[k][j] - c1 - (in_u.at(k, j) - st.z) * st.w * c2);
    }
    if (z) {
        Param<T, V, N> w1, g;
        w1.load(p, (const T *)a.post_w, 1.f);
        g.load(p, a.gate ? (const T *)a.gate + r / a.plan.group * a.gate_pitch : nullptr, 1.f);
        float c1 = 0.f, c2 = 0.f;
        FOR_ELEMENTS
        {
            d.f[k][j] = g.at(k, j) * q.f[k][j] * w1.at(k, j);
            if (j >= p.dup[k]) {
                c1 += d.f[k][j];
                c2 += d.f[k][j] * ((in_v.at(k, j) - st.x) * st.y);
            }
        }
        if (a.post != ROTOR_NORM_NONE) {
            row_sum2<TH>(c1, c2, red, half);
            c1 = a.post == ROTOR_NORM_LAYER ? c1 * inv : 0.f;
            c2 *= inv;
            FOR_ELEMENTS d.f[k][j] = st.y * (d.f[k][j] - c1 - (in_v.at(k, j) - st.x) * st.y * c2);
        }
        d.store(p, dz + r * a.dz_pitch);
    }
    FOR_ELEMENTS q.f[k][j] *= a.a;
    q.store(p, dx + r * a.dx_pitch);
}

// The sums over the rows of wide ones, the gradient of y once more from the
// row's means: eight columns a thread, a strip of rows a workgroup.
template <typename T> __global__ __launch_bounds__(256) void wide_sum_kernel(const T *dy, const T *dh, const T *y,
                                                                             const T *z, BackArgs a)
{
    constexpr int V = kVec;
    typedef typename VecOf<T, V>::V Vec;
    const int64_t at = ((int64_t)blockIdx.y * 256 + threadIdx.x) * V;
    if (at >= a.cols)
        return;
    const int64_t c = at < a.cols - V ? at : a.cols - V;  // the last piece ends with the row
    const bool gate_sums = a.part[kGate] || a.dgate, after = z && (gate_sums || a.part[kPostW] || a.part[kPostB]);
    float w1[V], b1[V], w2[V], g[V];
    float s_post_w[V] = {}, s_post_b[V] = {}, s_pre_w[V] = {}, s_pre_b[V] = {}, s_gate[V] = {};
    auto param = [&](const void *src, float otherwise, float (&v)[V]) {
        if (src)
            load_vec((const T *)src + c, v);
        else
#pragma unroll
            for (int j = 0; j < V; ++j)
                v[j] = otherwise;
    };
    param(a.post_w, 1.f, w1);
    param(a.post_b, 0.f, b1);
    param(a.pre_w, 1.f, w2);
    auto put = [&](const float (&v)[V], auto *dst) { store_vec(dst + c, v); };
    const int64_t s0 = (int64_t)blockIdx.x * a.plan.per_block;
    const int64_t s1 = s0 + a.plan.per_block < a.plan.strips ? s0 + a.plan.per_block : a.plan.strips;
    for (int64_t s = s0; s < s1; ++s) {
        const int64_t group = s / a.plan.per_group;
        const int64_t in_group = (s - group * a.plan.per_group) * a.plan.strip;
        const int64_t r0 = group * a.plan.group + in_group;
        const int64_t n = in_group + a.plan.strip < a.plan.group ? a.plan.strip : a.plan.group - in_group;
        param(a.gate ? (const T *)a.gate + group * a.gate_pitch : nullptr, 1.f, g);
        constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;  // rows in flight
        for (int64_t i = 0; i < n; i += kAhead) {
            Vec d[kAhead] = {}, u[kAhead] = {}, q[kAhead] = {}, v[kAhead] = {};
            float4 st[kAhead];
            float2 m[kAhead];
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                const int64_t r = r0 + (i + e < n ? i + e : i);
                st[e] = *(const float4 *)(a.stats + 4 * r);
                m[e] = dh ? a.row_sums[r] : make_float2(0.f, 0.f);
                if (dh) {
                    d[e] = *(const Vec *)(dh + r * a.dh_pitch + c);
                    u[e] = *(const Vec *)(y + r * a.y_pitch + c);
                }
                if (after) {
                    if (dy)
                        q[e] = *(const Vec *)(dy + r * a.dy_pitch + c);
                    v[e] = *(const Vec *)(z + r * a.z_pitch + c);
                }
            }
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                if (i + e >= n)
                    break;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float t = (float)q[e][j];
                    if (dh) {
                        const float b = (float)d[e][j], k = ((float)u[e][j] - st[e].z) * st[e].w;
                        s_pre_w[j] += b * k;
                        s_pre_b[j] += b;
                        t += st[e].w * (b * w2[j] - m[e].x - k * m[e].y);
                    }
                    if (after) {
                        const float k = ((float)v[e][j] - st[e].x) * st[e].y, b = g[j] * t;
                        s_gate[j] += t * (k * w1[j] + b1[j]);
                        s_post_w[j] += b * k;
                        s_post_b[j] += b;
                    }
                }
            }
        }
        if (gate_sums) {
            if (a.dgate)
                put(s_gate, (T *)a.dgate + group * a.dgate_pitch);
            else
                put(s_gate, a.part[kGate] + s * a.cols);
#pragma unroll
            for (int j = 0; j < V; ++j)
                s_gate[j] = 0.f;
        }
    }
    const int64_t row = (int64_t)blockIdx.x * a.cols;
    if (a.part[kPostW])
        put(s_post_w, a.part[kPostW] + row);
    if (a.part[kPostB])
        put(s_post_b, a.part[kPostB] + row);
    if (a.part[kPreW])
        put(s_pre_w, a.part[kPreW] + row);
    if (a.part[kPreB])
        put(s_pre_b, a.part[kPreB] + row);
}

// Adds the strips' sums: 64 columns of one output row a workgroup, its 16
// waves a part of the strips each, the parts then in order (5 us for those of
// 16384 x 2048).
struct AddArgs {
    const float *part[kSums];
    void *out[kSums];
    int64_t out_pitch[kSums];
    int64_t count[kSums];   // strips of one output row
    int64_t first[kSums + 1];  // of grid y: a task's output rows
    int64_t cols;
};

constexpr int kAddWaves = 16;
template <typename T> __global__ __launch_bounds__(kAddWaves * 64) void add_kernel(AddArgs a)
{
    __shared__ float other[kAddWaves - 1][64];
    int task = 0;
    while (task + 1 < kSums && (int64_t)blockIdx.y >= a.first[task + 1])
        ++task;
    const int64_t out_row = (int64_t)blockIdx.y - a.first[task];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    const int64_t n = a.count[task], each = (n + kAddWaves - 1) / kAddWaves;
    const int64_t from = wave * each, to = from + each < n ? from + each : n;
    float s = 0.f;
    if (c < a.cols) {
        const float *src = a.part[task] + out_row * n * a.cols + c;
#pragma unroll 8
        for (int64_t k = from; k < to; ++k)
            s += src[k * a.cols];
    }
    if (wave > 0)
        other[wave - 1][lane] = s;
    __syncthreads();
    if (wave > 0 || c >= a.cols)
        return;
#pragma unroll
    for (int w = 0; w < kAddWaves - 1; ++w)
        s += other[w][lane];
    ((T *)a.out[task])[out_row * a.out_pitch[task] + c] = (T)s;
}

// Calls f(team, V, N) with the smallest shape that holds a row (forward, 8192 x
// 5120 bf16: 640 threads of 8 elements 80 us, 1024 88, 512 of 16 102).
template <int V> struct IntV { static constexpr int v = V; };
template <typename F> void with_shape(int64_t cols, F f)
{
    if (cols < kVec)
        f(IntV<64>{}, IntV<1>{}, IntV<1>{});
    else if (cols <= 64 * 8)
        f(IntV<64>{}, IntV<8>{}, IntV<1>{});
    else if (cols <= 128 * 8)
        f(IntV<128>{}, IntV<8>{}, IntV<1>{});
    else if (cols <= 256 * 8)
        f(IntV<256>{}, IntV<8>{}, IntV<1>{});
    else if (cols <= 512 * 8)
        f(IntV<512>{}, IntV<8>{}, IntV<1>{});
    else if (cols <= 640 * 8)
        f(IntV<640>{}, IntV<8>{}, IntV<1>{});
    else if (cols <= 768 * 8)
        f(IntV<768>{}, IntV<8>{}, IntV<1>{});
    else if (cols <= 1024 * 8)
        f(IntV<1024>{}, IntV<8>{}, IntV<1>{});
    else if (cols <= 640 * 16)
        f(IntV<640>{}, IntV<8>{}, IntV<2>{});
    else if (cols <= 768 * 16)
        f(IntV<768>{}, IntV<8>{}, IntV<2>{});
    else
        f(IntV<1024>{}, IntV<8>{}, IntV<2>{});
}

// Columns past which the backward goes its way of wide rows.
constexpr int kNarrow = 512 * kVec;
bool wide(int64_t cols) { return cols > kNarrow; }

// Bytes of the backward's workspace for the rows' means.
uint64_t row_sums_bytes(const rotor_norm *n)
{
    return wide(n->cols) && n->pre != ROTOR_NORM_NONE ? (8ull * (uint64_t)n->rows + 15) / 16 * 16 : 0;
}

// Strips for as many workgroups as the 256 CUs hold at once: 8 waves each.
StripPlan strip_plan(int64_t rows, int64_t cols, int64_t gate_rows)
{
    int64_t blocks_at_once = 256;  // of wide rows, times their slices of columns
    if (!wide(cols))
        with_shape(cols, [&](auto th, auto, auto) { blocks_at_once = 256 * 8 * 64 / Team<decltype(th)::v>::kBlock; });
    StripPlan s;
    s.groups = gate_rows > 0 ? gate_rows : 1;
    s.group = rows / s.groups;
    int64_t per = blocks_at_once / s.groups;
    if (per < 1)
        per = 1;
    s.strip = ceil_div(s.group, per);
    if (s.strip < 1)
        s.strip = 1;
    s.per_group = s.group > 0 ? ceil_div(s.group, s.strip) : 1;  // no rows: one empty strip
    s.strips = s.groups * s.per_group;
    s.per_block = ceil_div(s.strips, blocks_at_once);
    s.blocks = ceil_div(s.strips, s.per_block);
    return s;
}

bool norm_sizes_ok(const rotor_norm *n)
{
    return n && type_ok(n->type) && n->post >= ROTOR_NORM_NONE && n->post <= ROTOR_NORM_LAYER &&
           n->pre >= ROTOR_NORM_NONE && n->pre <= ROTOR_NORM_LAYER && n->rows >= 0 && n->rows < ((int64_t)1 << 31) &&
           n->cols >= 1 && n->cols <= ROTOR_NORM_MAX_COLS && n->gate_rows >= 0 &&
           (n->gate_rows == 0 || n->rows % n->gate_rows == 0) && n->eps >= 0.;
}

bool norm_params_ok(const rotor_norm *n)
{
    const int64_t es = elem_bytes(n->type);
    for (const void *q : {n->post_weight, n->post_bias, n->gate, n->pre_weight, n->pre_bias})
        if ((uintptr_t)q % (uintptr_t)es)
            return false;
    if ((n->post == ROTOR_NORM_NONE && (n->post_weight || n->post_bias)) ||
        (n->pre == ROTOR_NORM_NONE && (n->pre_weight || n->pre_bias)))
        return false;
    return n->gate_rows > 0 ? matrix_ok(n->gate, n->gate_rows, n->cols, n->gate_pitch, es) : !n->gate;
}

}  // namespace
}  // namespace rotor

using namespace rotor;

extern "C" {

int32_t rotor_residual_norm(const rotor_norm *how, const void *d_x, int64_t x_pitch, const void *d_z,
                            int64_t z_pitch, void *d_y, int64_t y_pitch, void *d_h, int64_t h_pitch, float *d_stats,
                            void *stream)
{
    if (!norm_sizes_ok(how) || !norm_params_ok(how))
        return ROTOR_EINVAL;
    const int64_t es = elem_bytes(how->type), rows = how->rows, cols = how->cols;
    const bool pre = how->pre != ROTOR_NORM_NONE;
    if (rows == 0)
        return ROTOR_OK;
    if (!matrix_ok(d_x, rows, cols, x_pitch, es) || (d_z && !matrix_ok(d_z, rows, cols, z_pitch, es)) ||
        (d_y && !matrix_ok(d_y, rows, cols, y_pitch, es)) || (pre && !matrix_ok(d_h, rows, cols, h_pitch, es)) ||
        (!pre && d_h) || (uintptr_t)d_stats % 16)
        return ROTOR_EINVAL;
    if (!d_z && (how->post != ROTOR_NORM_NONE || how->gate_rows))
        return ROTOR_EINVAL;
    if (!d_y && (d_z || how->residual_scale != 1.))
        return ROTOR_EINVAL;
    NormArgs a;
    a.rows = rows;
    a.cols = cols;
    a.x_pitch = x_pitch;
    a.z_pitch = z_pitch;
    a.y_pitch = y_pitch;
    a.h_pitch = h_pitch;
    a.gate_pitch = how->gate_pitch;
    a.group = how->gate_rows > 0 ? rows / how->gate_rows : rows;
    a.post = how->post;
    a.pre = how->pre;
    a.a = (float)how->residual_scale;
    a.eps = (float)how->eps;
    a.post_w = how->post_weight;
    a.post_b = how->post_bias;
    a.gate = how->gate;
    a.pre_w = how->pre_weight;
    a.pre_b = how->pre_bias;
    a.stats = d_stats;
    (void)hipGetLastError();  // an error the caller's earlier calls left behind is not this launch's
    with_type(how->type, [&](auto e) {
        typedef typename decltype(e)::T T;
        with_shape(cols, [&](auto th, auto v, auto n) {
            constexpr int TH = decltype(th)::v;
            norm_kernel<T, TH, decltype(v)::v, decltype(n)::v>
                <<<grid_of(ceil_div(rows, Team<TH>::kRows)), Team<TH>::kBlock, 0, (hipStream_t)stream>>>(
                    (const T *)d_x, (const T *)d_z, (T *)d_y, (T *)d_h, a);
        });
    });
    return hipGetLastError() == hipSuccess ? ROTOR_OK : ROTOR_EDEVICE;
}

int32_t rotor_residual_norm_workspace_bytes(const rotor_norm *how, uint64_t *bytes)
{
    if (!bytes || !norm_sizes_ok(how))
        return ROTOR_EINVAL;
    const StripPlan s = strip_plan(how->rows, how->cols, how->gate_rows);
    *bytes = row_sums_bytes(how) + 4ull * (uint64_t)how->cols * (uint64_t)((kSums - 1) * s.blocks + (s.per_group > 1 ? s.strips : 0));
    if (*bytes < 16)
        *bytes = 16;
    return ROTOR_OK;
}

int32_t rotor_residual_norm_backward(const rotor_norm *how, const void *d_dy, int64_t dy_pitch, const void *d_dh,
                                     int64_t dh_pitch, const void *d_y, int64_t y_pitch, const void *d_z,
                                     int64_t z_pitch, const float *d_stats, void *d_dx, int64_t dx_pitch, void *d_dz,
                                     int64_t dz_pitch, const rotor_norm_grads *grads, void *d_work,
                                     uint64_t work_bytes, void *stream)
{
    uint64_t need = 0;
    if (!grads || !norm_sizes_ok(how) || !norm_params_ok(how) ||
        rotor_residual_norm_workspace_bytes(how, &need) != ROTOR_OK)
        return ROTOR_EINVAL;
    const int64_t es = elem_bytes(how->type), rows = how->rows, cols = how->cols;
    const bool pre = how->pre != ROTOR_NORM_NONE, post = how->post != ROTOR_NORM_NONE;
    if (!matrix_ok(d_dx, rows, cols, dx_pitch, es) || (!d_dy && !pre && rows > 0) ||
        (d_dy && !matrix_ok(d_dy, rows, cols, dy_pitch, es)) ||
        (pre && (!matrix_ok(d_dh, rows, cols, dh_pitch, es) || !matrix_ok(d_y, rows, cols, y_pitch, es))) ||
        (!pre && d_dh) || (d_z && (!matrix_ok(d_z, rows, cols, z_pitch, es) || !matrix_ok(d_dz, rows, cols, dz_pitch, es))) ||
        (!d_z && rows > 0 && (post || how->gate_rows || d_dz)) || (rows > 0 && (!d_stats || (uintptr_t)d_stats % 16)) ||
        !d_work || (uintptr_t)d_work % 16 || work_bytes < need)
        return ROTOR_EINVAL;
    if ((!post && (grads->post_weight || grads->post_bias)) || (!pre && (grads->pre_weight || grads->pre_bias)) ||
        (grads->gate && (how->gate_rows < 1 || !matrix_ok(grads->gate, how->gate_rows, cols, grads->gate_pitch, es))))
        return ROTOR_EINVAL;
    for (const void *q : {grads->post_weight, grads->post_bias, grads->gate, grads->pre_weight, grads->pre_bias})
        if ((uintptr_t)q % (uintptr_t)es)
            return ROTOR_EINVAL;
    const StripPlan plan = strip_plan(rows, cols, how->gate_rows);
    void *const out[kSums] = {grads->post_weight, grads->post_bias, grads->pre_weight, grads->pre_bias, grads->gate};
    const bool gate_here = grads->gate && plan.per_group == 1;
    BackArgs a;
    AddArgs add;
    int64_t tasks = 0;
    int last = -1;
    a.row_sums = (float2 *)d_work;
    float *w = (float *)((char *)d_work + row_sums_bytes(how));
    for (int k = 0; k < kSums; ++k) {
        const bool wanted = out[k] && !(k == kGate && gate_here);
        a.part[k] = wanted ? w : nullptr;
        add.part[k] = w;
        add.out[k] = out[k];
        add.out_pitch[k] = k == kGate ? grads->gate_pitch : cols;
        add.count[k] = k == kGate ? plan.per_group : plan.blocks;
        add.first[k] = tasks;
        if (!wanted)
            continue;
        last = k;
        tasks += k == kGate ? plan.groups : 1;
        w += (k == kGate ? plan.strips : plan.blocks) * cols;
    }
    add.first[kSums] = tasks;
    add.cols = cols;
    if (tasks > 65535)
        return ROTOR_EINVAL;
    a.rows = rows;
    a.cols = cols;
    a.dy_pitch = dy_pitch;
    a.dh_pitch = dh_pitch;
    a.y_pitch = y_pitch;
    a.z_pitch = z_pitch;
    a.dx_pitch = dx_pitch;
    a.dz_pitch = dz_pitch;
    a.gate_pitch = how->gate_pitch;
    a.dgate_pitch = grads->gate_pitch;
    a.post = how->post;
    a.pre = how->pre;
    a.a = (float)how->residual_scale;
    a.post_w = how->post_weight;
    a.post_b = how->post_bias;
    a.gate = how->gate;
    a.pre_w = how->pre_weight;
    a.stats = d_stats;
    a.dgate = gate_here ? grads->gate : nullptr;
    a.plan = plan;
    (void)hipGetLastError();  // an error the caller's earlier calls left behind is not this launch's
    with_type(how->type, [&](auto e) {
        typedef typename decltype(e)::T T;
        // without rows the strips are empty, and the sums 0
        with_shape(cols, [&](auto th, auto v, auto n) {
            constexpr int TH = decltype(th)::v, V = decltype(v)::v, N = decltype(n)::v;
            const hipStream_t st = (hipStream_t)stream;
            const T *const dy = (const T *)d_dy, *const dh = (const T *)d_dh, *const y = (const T *)d_y,
                    *const z = (const T *)d_z;
            if constexpr (TH * V * N <= kNarrow) {
                back_kernel<T, TH, V, N>
                    <<<dim3((uint32_t)plan.blocks), Team<TH>::kBlock, 0, st>>>(dy, dh, y, z, (T *)d_dx, (T *)d_dz, a);
            } else {
                if (rows > 0)
                    wide_row_kernel<T, TH, V, N>
                        <<<grid_of(rows), TH, 0, st>>>(dy, dh, y, z, (T *)d_dx, (T *)d_dz, a);
                if (last >= 0 || gate_here)
                    wide_sum_kernel<T>
                        <<<dim3((uint32_t)plan.blocks, (uint32_t)ceil_div(cols, 256 * kVec)), 256, 0, st>>>(dy, dh, y,
                                                                                                         z, a);
            }
        });
        if (last >= 0)
            add_kernel<T><<<dim3((uint32_t)ceil_div(cols, 64), (uint32_t)tasks), kAddWaves * 64, 0,
                            (hipStream_t)stream>>>(add);
    });
    return hipGetLastError() == hipSuccess ? ROTOR_OK : ROTOR_EDEVICE;
}

}  // extern "C"
