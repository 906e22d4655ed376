// rotor_window_attention and rotor_window_attention_step: softmax attention of
// the keys that a row sees, one pass over them with a running maximum and sum.
#include "rotor_attention.h"

#include <type_traits>

namespace rotor {
namespace {

constexpr int kFewRows = 32;

#if defined(__HIP_DEVICE_COMPILE__)

// The running softmax of a wave's 32 rows (a row is a lane's column): what it
// has summed so far is relative to `top`, which is raised only when a score
// lies more than 2^kSlack above it; `sum` is that of the lane's half.
constexpr float kSlack = 8.f;

template <typename T, int NB> struct Rows {
    typename Frag<T>::F q[Shape<T, NB>::NK];
    f32x16 acc[NB];
    float top, sum;

    __device__ void reset()
    {
        clear(acc);
        top = -kInf;
        sum = 0.f;
    }

    // 32 keys: masked scores to probabilities.  First the maximum: `by` is the
    // factor by which what acc holds falls behind, if any row's is raised.
    __device__ bool raise(const f32x16 &s, float c, float &by)
    {
        float most = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e)
            most = fmaxf(most, s[e]);
        most = halves_max(most);
        const bool any = __any((most - top) * c > kSlack);  // (-inf - -inf is NaN: no)
        if (any) {
            const float next = fmaxf(top, most);
            by = next > top ? exp2_of((top - next) * c) : 1.f;
            sum *= by;
            top = next;
        }
        return any;
    }
    __device__ void soften(f32x16 &s, float c)
    {
        // a row that has seen nothing yet: exp2(-inf - 0) = 0
        const float base = top == -kInf ? 0.f : top * c;
        float add = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = exp2_of(__builtin_fmaf(s[e], c, -base));
            add += s[e];
        }
        sum += add;
    }
    __device__ void scale(float by)
    {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                acc[b][e] *= by;
    }
};

// Where a row's results go: out and lse, or this part's sums.
template <typename T, int NB>
__device__ inline void put_rows(const Attention &a, const Rows<T, NB> &w, int b, int kv, int part, int row, bool seen,
                                int h)
{
    const float sum = halves_sum(w.sum);
    if (row >= a.rows)
        return;
    if (a.parts > 1) {
        const int64_t at = ((int64_t)part * a.batch * a.kv + (int64_t)b * a.kv + kv) * a.rows + row;
        if (h == 0)
            a.part_soft[at] = make_float2(w.top * a.c, sum);
        put_sums(a.part_out + at * a.width, h, a.width, w.acc);
        return;
    }
    const int t = row / a.group, head = kv * a.group + row % a.group;
    put_row<T>(rows_of(a.out, b, head) + t * a.out.token, h, a.width, w.acc, 1.f / sum, seen);
    if (h == 0 && a.lse)
        a.lse[((int64_t)b * a.tokens + t) * ((int64_t)a.kv * a.group) + head] =
            seen ? (w.top * a.c + __builtin_amdgcn_logf(sum)) * kLn2 : -kInf;
}
#endif

// A workgroup takes 128 rows of one key head and goes over the keys that any of
// them sees, 32 a step.  The steps overlap: while the exponentials of one are
// computed, the matrix units work on the scores of the next and on the values
// of the one before, in one stream of independent instructions.  Three places
// in LDS for keys and for values: one is read, two are on their way.
// blockIdx.x: key head and sequence (so that an XCD keeps to few of them),
// y: rows, the last (with the most keys) first, z: part of the keys.
template <typename T, int NB>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 1 : 2) void attention_kernel(Attention a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    typedef Shape<T, NB> S;
    typedef typename Frag<T>::F F;
    constexpr int kBytes = kTileKeys * S::kRow;
    // one array a place: a read waits for the loads into its own array alone
    __shared__ __attribute__((aligned(1024))) char keys0[kBytes], keys1[kBytes], keys2[kBytes];
    __shared__ __attribute__((aligned(1024))) char vals0[kBytes], vals1[kBytes], vals2[kBytes];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 32;
    const int b = blockIdx.x / a.kv, kv = blockIdx.x % a.kv;
    const int r0 = (gridDim.y - 1 - blockIdx.y) * kTileRows, rw = r0 + wave * 32, row = rw + lane % 32;
    const Span span(a, b);
    const int last_row = min(a.rows - 1, r0 + kTileRows - 1);

    const int t = row / a.group, p = span.offset + t;
    const bool seen = row < a.rows && p >= 0 && p < span.length;
    Rows<T, NB> w;
    w.reset();
    int lo, hi;
    if (!span.positions(r0 / a.group, last_row / a.group, lo, hi)) {
        put_rows(a, w, b, kv, blockIdx.z, row, false, h);
        return;
    }
    {
        const char *q = rows_of(a.q, b, kv * a.group + row % a.group) + t * a.q.token;
#pragma unroll
        for (int k = 0; k < S::NK; ++k)
            w.q[k] = global_frag<T>(q, seen, 2 * k + h, a.width);
    }
    const Sight sight{p - a.window + 1, p, a.sinks};
    // what all rows of the wave see, and what any of them does
    int wlo = 0, whi = -1;
    const bool some = rw < a.rows && span.positions(rw / a.group, min(a.rows - 1, rw + 31) / a.group, wlo, whi);

    const Steps<kTileKeys> steps(a, lo, hi);
    const int i0 = (int)((int64_t)steps.n * blockIdx.z / a.parts);
    const int i1 = (int)((int64_t)steps.n * (blockIdx.z + 1) / a.parts);

    typedef Loader<T, NB, kTileKeys, kWaves> Load;
    Load lk, lv;
    lk.init(wave, lane, a.width, a.k.token);
    lv.init(wave, lane, a.width, a.v.token);
    Reader<T, NB> rd;
    rd.init(lane);
    const char *const k0 = rows_of(a.k, b, kv), *const v0 = rows_of(a.v, b, kv);
    const uint32_t k_stride = (uint32_t)a.k.token, v_stride = (uint32_t)a.v.token;
    const int row_bytes = a.width * (int)sizeof(T);
    auto load_keys = [&](char *place, int j) {
        lk.load(place, row_at(k0, j, k_stride), hi + 1 - j, k_stride, row_bytes);
    };
    auto load_values = [&](char *place, int j) {
        lv.load(place, row_at(v0, j, v_stride), hi + 1 - j, v_stride, row_bytes);
    };
    const int all_from = whi - a.window + 1;
    auto mask = [&](f32x16 &s, int j) {
        const int je = j + kTileKeys - 1;
        if (!some || je > wlo || (je >= a.sinks && j < all_from)) {
            asm volatile("");  // a branch: few steps need it
#pragma unroll
            for (int e = 0; e < 16; ++e)
                s[e] = sight(j + row_of(e, h)) ? s[e] : -kInf;
        }
    };

    // keys of this step and of the next three
    int j = steps.key(i0), j1 = steps.next(j), j2 = steps.next(j1);
    load_keys(keys0, j);
    load_keys(keys1, j1);
    load_values(vals2, hi + 1);  // zeros: there is no step before
    load_keys(keys2, j2);
    load_values(vals0, j);
    step_barrier<4 * Load::kLoads>();
    f32x16 s = product<T, NB>(keys0, rd, w.q);
    Packed<T, NB> before{};
    auto step = [&](char *free, char *next_keys, char *next_vals, char *last_vals) {
        step_barrier<2 * Load::kLoads>();
        const int j3 = steps.next(j2);
        F kf[S::NK];
        fetch_rows<T, NB>(next_keys, rd, kf);
        load_keys(free, j3);
        load_values(next_vals, j1);
        mask(s, j);
        float by;
        const bool raised = w.raise(s, a.c, by);
        __builtin_amdgcn_sched_barrier(0);
        f32x16 ahead;
        multiply<T>(ahead, kf, w.q);
        w.soften(s, a.c);
        add_rows<T, NB>(w.acc, last_vals, rd, before);
        before = Packed<T, NB>(s);
        before.pin();
        constexpr int kColumns = S::kGroups * NB, kReads = S::kTurned * kColumns;
        beside<T, S::NK, kReads / S::NK, 32 / S::NK, 0>();
        beside<T, kColumns, 0, 2, 16 / kColumns>();
        __builtin_amdgcn_sched_barrier(0);
        if (raised)
            w.scale(by);
        s = ahead;
        j = j1;
        j1 = j2;
        j2 = j3;
    };
    int left = i1 - i0;
    for (; left >= 3; left -= 3) {
        step(keys0, keys1, vals1, vals2);
        step(keys1, keys2, vals2, vals0);
        step(keys2, keys0, vals0, vals1);
    }
    if (left > 0)
        step(keys0, keys1, vals1, vals2);
    if (left > 1)
        step(keys1, keys2, vals2, vals0);
    tile_barrier();
    if (left == 0)
        add_rows<T, NB>(w.acc, vals2, rd, before);
    else if (left == 1)
        add_rows<T, NB>(w.acc, vals0, rd, before);
    else
        add_rows<T, NB>(w.acc, vals1, rd, before);

    // Infinities or NaN: they may have come from keys that a row does not see,
    // as 0 times their values.
    if (__syncthreads_or(!finite(w.acc))) {
        w.reset();
        j = steps.key(i0);
        for (int i = i0; i < i1; ++i, j = steps.next(j)) {
            load_keys(keys0, j);
            load_values(vals0, j);
            tile_barrier();
            s = product<T, NB>(keys0, rd, w.q);
            mask(s, j);
            float by;
            if (w.raise(s, a.c, by))
                w.scale(by);
            w.soften(s, a.c);
            add_rows_apart<T, NB>(w.acc, vals0, lane, s);
            tile_barrier();
        }
    }
    put_rows(a, w, b, kv, blockIdx.z, row, seen, h);
#endif
}

// Up to 32 rows of a key head: the waves share the rows and split the keys.
// Each has tiles of 32 keys of its own in LDS, the next on its way while one is
// used, and waits for no other before the end, when the waves' sums are joined.
// The keys that any row sees are a list: the first ones, then the window's.
// STEP: one token, whose key and value are new: they are in the place of the
// last key of the list, and go into the cache.
template <typename T, int NB, bool STEP>
__global__ __launch_bounds__(256, 1) void few_kernel(Attention a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    typedef Shape<T, NB> S;
    constexpr int W = sizeof(T) == 4 ? 2 : 4;  // waves that have tiles
    constexpr int kBytes = 32 * S::kRow, kAtOnce = 64 / S::kPieces, kLoads = 32 / kAtOnce;
    __shared__ __attribute__((aligned(1024))) char tiles[W][2][2][kBytes];
    __shared__ float2 soft[W][32];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 32;
    const int b = blockIdx.x / a.kv, kv = blockIdx.x % a.kv;
    const int r0 = blockIdx.y * kFewRows, row = r0 + lane % 32;
    const Span span(a, b);
    const int t = row / a.group, p = span.offset + t;
    const bool seen = row < a.rows && p >= 0 && p < span.length;
    Rows<T, NB> w;
    w.reset();
    {
        const char *q = rows_of(a.q, b, kv * a.group + row % a.group) + t * a.q.token;
#pragma unroll
        for (int k = 0; k < S::NK; ++k)
            w.q[k] = global_frag<T>(q, seen, 2 * k + h, a.width);
    }
    int lo = 0, hi = -1;
    const bool some = span.positions(r0 / a.group, min(a.rows - 1, r0 + kFewRows - 1) / a.group, lo, hi);
    const int from = max(0, lo - a.window + 1), ahead = min(a.sinks, from);
    const int n = some ? ahead + hi - from + 1 : 0;
    const int share = (n + a.parts - 1) / a.parts;
    const int e0 = min(n, (int)blockIdx.z * share), e1 = min(n, e0 + share);
    const Sight sight{p - a.window + 1, p, a.sinks};
    // position of the list's element e
    auto position = [&](int e) { return e < ahead ? e : from + e - ahead; };
    // rounds that the ring has made before the window's first key
    const int turns = a.ring && from > a.sinks ? (from - a.sinks) / a.ring * a.ring : 0;
    auto slot = [&](int j) {
        if (!a.ring || j < a.sinks)
            return j;
        int x = j - a.sinks;
        x -= x >= turns ? turns : 0;
        x -= x >= a.ring ? a.ring : 0;
        return a.sinks + x;
    };
    const char *const k0 = rows_of(a.k, b, kv), *const v0 = rows_of(a.v, b, kv);
    const bool whole = a.width == NB * 32;

    // Rows past the end are the last one again: their probabilities are 0, and
    // what they hold is what the rows see anyway.
    auto load = [&](char (&to)[2][kBytes], int e) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = i * kAtOnce + lane / S::kPieces;
            int c = (lane % S::kPieces) ^ S::turn(r);
            c = c * Frag<T>::N < a.width ? c : 0;
            const int j = slot(position(min(e + r, e1 - 1)));
            __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void *)(k0 + j * a.k.token + c * 16),
                                             (lds_ptr)(to[0] + i * 1024), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void *)(v0 + j * a.v.token + c * 16),
                                             (lds_ptr)(to[1] + i * 1024), 16, 0, 0);
        }
    };
    // the new key and value: a piece a lane
    typedef typename Frag<T>::F F;
    F fresh[2] = {{}, {}};
    const int piece = lane % S::kPieces;
    const bool mine = STEP && e0 < e1 && e1 == n;  // this part has the last key
    if (mine && piece * Frag<T>::N < a.width) {
        fresh[0] = *(const F *)(rows_of(a.k_new, b, kv) + piece * 16);
        fresh[1] = *(const F *)(rows_of(a.v_new, b, kv) + piece * 16);
        if (wave == 0 && lane < S::kPieces && r0 == 0) {
            const int j = slot(hi);
            *(F *)(rows_of(a.k, b, kv) + j * a.k.token + piece * 16) = fresh[0];
            *(F *)(rows_of(a.v, b, kv) + j * a.v.token + piece * 16) = fresh[1];
        }
    }
    Reader<T, NB> rd;
    rd.init(lane);
    auto pass = [&](auto apart) {
        constexpr bool kApart = decltype(apart)::value;
        int e = e0 + wave * 32, which = 0;
        if (wave < W && e < e1)
            load(tiles[wave][0], e);
        for (; wave < W && e < e1; e += 32 * W, which ^= 1) {
            const bool more = e + 32 * W < e1;
            __builtin_amdgcn_sched_barrier(0);
            if (more) {
                // what read this place is done: its results were used
                load(tiles[wave][which ^ 1], e + 32 * W);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kLoads) : "memory");
            } else {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
            __builtin_amdgcn_sched_barrier(0);
            char *keys = tiles[wave][which][0], *vals = tiles[wave][which][1];
            if (mine && e + 32 >= n) {
                // in the place of the last key, and of what follows it there
                for (int r = n - 1 - e + lane / S::kPieces; r < 32; r += kAtOnce) {
                    *(F *)(keys + r * S::kRow + (piece ^ S::turn(r)) * 16) = fresh[0];
                    *(F *)(vals + r * S::kRow + (piece ^ S::turn(r)) * 16) = fresh[1];
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
            f32x16 s;
            if (whole) {
                s = product<T, NB>(keys, rd, w.q);
            } else {
                // columns past the width hold others again: they count as 0
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    s[x] = 0.f;
#pragma unroll
                for (int k = 0; k < S::NK; ++k) {
                    F f = rd.row(keys, k);
                    if ((2 * k + h) * Frag<T>::N >= a.width)
                        f = F{};
                    s = Frag<T>::mma(f, w.q[k], s);
                }
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const int at = e + row_of(x, h);
                s[x] = at < e1 && sight(position(at)) ? s[x] : -kInf;
            }
            float by;
            if (w.raise(s, a.c, by))
                w.scale(by);
            w.soften(s, a.c);
            if constexpr (kApart)
                add_rows_apart<T, NB>(w.acc, vals, lane, s);
            else
                add_rows<T, NB>(w.acc, vals, rd, Packed<T, NB>(s));
        }
    };
    pass(std::false_type{});
    if (__syncthreads_or(!finite(w.acc))) {
        w.reset();
        pass(std::true_type{});
        __syncthreads();
    }

    // the waves' sums: relative to the highest maximum, added in order
    if (wave < W)
        w.sum = halves_sum(w.sum);
    if (wave < W && h == 0)
        soft[wave][lane] = make_float2(w.top, w.sum);
    __syncthreads();
    float top = -kInf, sum = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i)
        top = fmaxf(top, soft[i][lane % 32].x);
    const float base = top == -kInf ? 0.f : top;
#pragma unroll
    for (int i = 0; i < W; ++i)
        sum += soft[i][lane % 32].y * exp2_of((soft[i][lane % 32].x - base) * a.c);
    // a wave's 32 rows of sums, skewed by 16 bytes for the banks' sake
    constexpr int kLine = NB * 32 + 4;
    float *const lines = (float *)tiles;
    static_assert(W * 32 * kLine * 4 <= (int)sizeof(tiles), "all waves' sums");
    if (wave < W) {
        const float by = exp2_of((w.top - base) * a.c);
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *(f32x4 *)(lines + (wave * 32 + lane % 32) * kLine + 32 * i + 8 * r + 4 * h) =
                    f32x4{w.acc[i][4 * r], w.acc[i][4 * r + 1], w.acc[i][4 * r + 2], w.acc[i][4 * r + 3]} * by;
    }
    __shared__ float2 joined[32];
    if (wave == 0 && h == 0)
        joined[lane] = make_float2(top, sum);
    __syncthreads();
    // 8 lanes a row, four columns at a time
    const int line = threadIdx.x / 8, rr = r0 + line;
    if (rr >= a.rows)
        return;
    const float2 j = joined[line];
    const int tt = rr / a.group, head = kv * a.group + rr % a.group, pp = span.offset + tt;
    const bool sees = pp >= 0 && pp < span.length;
    const int64_t part = ((int64_t)blockIdx.z * a.batch * a.kv + (int64_t)b * a.kv + kv) * a.rows + rr;
    // a position past the cache of a single token has no result
    const float none = STEP && span.offset >= 0 ? __builtin_nanf("") : 0.f;
    for (int col = threadIdx.x % 8 * 4; col < a.width; col += 32) {
        f32x4 v = *(const f32x4 *)(lines + line * kLine + col);
#pragma unroll
        for (int i = 1; i < W; ++i)
            v += *(const f32x4 *)(lines + (i * 32 + line) * kLine + col);
        if (a.parts > 1) {
            *(f32x4 *)(a.part_out + part * a.width + col) = v;
        } else {
            typedef T V __attribute__((ext_vector_type(4)));
            V x;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = (T)(sees ? v[e] / j.y : none);
            *(V *)(rows_of(a.out, b, head) + tt * a.out.token + col * sizeof(T)) = x;
        }
    }
    if (threadIdx.x % 8 == 0) {
        if (a.parts > 1)
            a.part_soft[part] = make_float2(j.x * a.c, j.y);
        else if (a.lse)
            a.lse[((int64_t)b * a.tokens + tt) * ((int64_t)a.kv * a.group) + head] =
                sees ? (j.x * a.c + __builtin_amdgcn_logf(j.y)) * kLn2 : -kInf;
    }
#endif
}

// The parts' sums of a row joined, in their order: four columns a thread.
template <typename T, bool STEP> __global__ __launch_bounds__(256) void join_kernel(Attention a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const int per = (a.width + 3) / 4;
    const int64_t heads = (int64_t)a.batch * a.kv, all = heads * a.rows;
    const int64_t i = block_at() * 256 + threadIdx.x, at = i / per;
    if (at >= all)
        return;
    const int col = (int)(i - at * per) * 4, row = (int)(at % a.rows), bk = (int)(at / a.rows);
    const int b = bk / a.kv, kv = bk % a.kv, t = row / a.group, head = kv * a.group + row % a.group;
    const Span span(a, b);
    const int p = span.offset + t;
    const bool seen = p >= 0 && p < span.length;
    float top = -kInf;
    for (int k = 0; k < a.parts; ++k)
        top = fmaxf(top, a.part_soft[k * all + at].x);
    const float base = top == -kInf ? 0.f : top;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll 4
    for (int k = 0; k < a.parts; ++k) {
        const float2 s = a.part_soft[k * all + at];
        const float by = exp2_of(s.x - base);
        sum += s.y * by;
        const f32x4 o = *(const f32x4 *)(a.part_out + (k * all + at) * a.width + col);
        // a part without keys has nothing to scale, whatever its factor
        v += s.y != 0.f || s.x != -kInf ? o * by : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float none = STEP && span.offset >= 0 ? __builtin_nanf("") : 0.f;
    typedef T V __attribute__((ext_vector_type(4)));
    V x;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        x[e] = (T)(seen ? v[e] / sum : none);
    *(V *)(rows_of(a.out, b, head) + t * a.out.token + col * sizeof(T)) = x;
    if (col == 0 && a.lse)
        a.lse[((int64_t)b * a.tokens + t) * ((int64_t)a.kv * a.group) + head] =
            seen ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -kInf;
#endif
}

}  // namespace
}  // namespace rotor

namespace rotor {
namespace {

struct ForwardPlan {
    bool few;
    int parts;
    uint64_t out_bytes, soft_bytes;
};

// Few rows (one token of each sequence, or a few): the keys alone bound the
// call, and are split until the device is full.  Otherwise rows are split
// first, keys only where they leave half of the CUs without work: 64 rows
// against 32768 keys of 128 columns bf16, 8 key heads, take 8 workgroups.
ForwardPlan forward_plan(const rotor_attention *n, bool step)
{
    ForwardPlan p;
    const int64_t group = n->heads / n->kv_heads, rows = n->tokens * group, bk = n->batch * n->kv_heads;
    int64_t most = n->keys;  // keys that a tile of rows sees
    if (n->window && n->window < most)
        most = n->window + n->sinks + (step ? 0 : 128 / group + 1) < most
                   ? n->window + n->sinks + (step ? 0 : 128 / group + 1)
                   : most;
    p.few = step || rows <= kFewRows;
    int64_t parts = 1;
    if (p.few) {
        // workgroups that run at once, by their LDS
        const int64_t at_once = 256 * (n->width <= 64 ? 2 : 1), base = bk * ceil_div(rows, kFewRows);
        const int64_t limit = most / 512;  // 4 tiles of 32 keys for each of 4 waves
        double best = 0.;
        for (int64_t k = 1; base && k <= limit && k <= 256; ++k) {
            const int64_t rounds = ceil_div(base * k, at_once);
            const double full = (double)(base * k) / (double)(rounds * at_once);
            if (full > best + 0.02) {
                best = full;
                parts = k;
            }
            if (rounds > 4 || full > 0.95)
                break;
        }
    } else {
        const int64_t base = bk * ceil_div(rows, kTileRows), tiles = most / 64;
        if (base < 256 && tiles >= 16)
            parts = ceil_div(512, base) < tiles / 8 ? ceil_div(512, base) : tiles / 8;
    }
    p.parts = (int)(parts < 1 ? 1 : parts);
    p.out_bytes = p.soft_bytes = 0;
    if (p.parts > 1) {
        p.out_bytes = round256((uint64_t)p.parts * bk * rows * n->width * 4);
        p.soft_bytes = round256((uint64_t)p.parts * bk * rows * 8);
    }
    return p;
}

int32_t launch_forward(const rotor_attention *n, Attention &a, bool step, void *work, uint64_t work_bytes,
                       void *stream)
{
    const ForwardPlan p = forward_plan(n, step);
    if (p.parts > 1 && (!work || (uintptr_t)work % 16 || work_bytes < p.out_bytes + p.soft_bytes))
        return ROTOR_EINVAL;
    a.parts = p.parts;
    a.part_out = (float *)work;
    a.part_soft = (float2 *)((char *)work + p.out_bytes);
    const hipStream_t s = (hipStream_t)stream;
    const uint32_t bk = (uint32_t)(a.batch * a.kv), z = (uint32_t)a.parts;
    (void)hipGetLastError();  // an error the caller's earlier calls left behind is not this launch's
    with_shape(n->type, n->width, [&](auto e, auto nb) {
        typedef typename decltype(e)::T T;
        constexpr int NB = decltype(nb)::v;
        const dim3 few(bk, (uint32_t)ceil_div(a.rows, kFewRows), z);
        if (step)
            few_kernel<T, NB, true><<<few, 256, 0, s>>>(a);
        else if (p.few)
            few_kernel<T, NB, false><<<few, 256, 0, s>>>(a);
        else
            attention_kernel<T, NB><<<dim3(bk, (uint32_t)ceil_div(a.rows, kTileRows), z), kThreads, 0, s>>>(a);
        if (a.parts > 1) {
            const dim3 grid = grid_of(ceil_div((int64_t)bk * a.rows * (a.width / 4), 256));
            if (step)
                join_kernel<T, true><<<grid, 256, 0, s>>>(a);
            else
                join_kernel<T, false><<<grid, 256, 0, s>>>(a);
        }
    });
    return hipGetLastError() == hipSuccess ? ROTOR_OK : ROTOR_EDEVICE;
}

}  // namespace
}  // namespace rotor

using namespace rotor;

extern "C" {

int32_t rotor_window_attention(const rotor_attention *how, const rotor_heads *q, const rotor_heads *k,
                               const rotor_heads *v, const rotor_heads *out, float *d_lse, void *d_work,
                               uint64_t work_bytes, void *stream)
{
    if (!attention_sizes_ok(how) || !index_ok(how->positions, how->position_bytes) ||
        !index_ok(how->lengths, how->length_bytes))
        return ROTOR_EINVAL;
    const int64_t es = elem_bytes(how->type);
    Attention a;
    fill(a, how);
    if (!heads_ok(q, how->batch, how->tokens, how->heads, es, a.q) ||
        !heads_ok(k, how->batch, how->keys, how->kv_heads, es, a.k) ||
        !heads_ok(v, how->batch, how->keys, how->kv_heads, es, a.v) ||
        !heads_ok(out, how->batch, how->tokens, how->heads, es, a.out) || !tiles_ok(a.k, 1) || !tiles_ok(a.v, 1) ||
        (uintptr_t)d_lse % 4)
        return ROTOR_EINVAL;
    if (how->batch == 0 || how->tokens == 0)
        return ROTOR_OK;
    a.lse = d_lse;
    return launch_forward(how, a, false, d_work, work_bytes, stream);
}

int32_t rotor_window_attention_step(const rotor_attention *how, const rotor_heads *q, const rotor_heads *k,
                                    const rotor_heads *v, const rotor_heads *k_cache, const rotor_heads *v_cache,
                                    int32_t ring, const rotor_heads *out, void *d_work, uint64_t work_bytes,
                                    void *stream)
{
    if (!attention_sizes_ok(how) || how->tokens != 1 || how->keys < 1 || !how->positions || how->lengths ||
        !index_ok(how->positions, how->position_bytes) || (ring != 0 && ring != 1))
        return ROTOR_EINVAL;
    // a ring holds the first keys and then at least a window
    if (ring && (how->window < 1 || how->sinks > how->keys || how->window > how->keys - how->sinks))
        return ROTOR_EINVAL;
    const int64_t es = elem_bytes(how->type);
    Attention a;
    fill(a, how);
    if (ring) {
        a.sinks = (int)how->sinks;
        a.ring = (int)(how->keys - how->sinks);
    }
    if (!heads_ok(q, how->batch, 1, how->heads, es, a.q) || !heads_ok(k, how->batch, 1, how->kv_heads, es, a.k_new) ||
        !heads_ok(v, how->batch, 1, how->kv_heads, es, a.v_new) ||
        !heads_ok(k_cache, how->batch, how->keys, how->kv_heads, es, a.k) ||
        !heads_ok(v_cache, how->batch, how->keys, how->kv_heads, es, a.v) ||
        !heads_ok(out, how->batch, 1, how->heads, es, a.out))
        return ROTOR_EINVAL;
    if (how->batch == 0)
        return ROTOR_OK;
    return launch_forward(how, a, true, d_work, work_bytes, stream);
}

int32_t rotor_window_attention_workspace_bytes(const rotor_attention *how, int32_t step, uint64_t *bytes)
{
    if (!bytes || !attention_sizes_ok(how) || (step != 0 && step != 1) || (step && how->tokens != 1))
        return ROTOR_EINVAL;
    const ForwardPlan p = forward_plan(how, step);
    *bytes = p.out_bytes + p.soft_bytes;
    return ROTOR_OK;
}

}  // extern "C"
