// rotor_embedding: rows of a table by token, scaled; and the table's gradient
// by sorted tokens.
//
// Backward: a stable radix sort of (token, position), one launch per digit of
// up to 9 bits (one in all for up to 2048 tokens; past 32768 tokens one more per
// digit, for its counts), whose few workgroups share the device with others
// that clear the gradient; then one launch in which groups of lanes take 32
// sorted positions each, add the rows of one token in registers and write each
// token that lies within their positions; then one launch that joins the
// tokens that cross the 32-position cuts.  No atomics on the sums: their order
// depends on the tokens alone.
#include "rotor_ops.h"

namespace rotor {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;        // adjacent elements of a lane, V below (1 in rows of fewer)
constexpr int kChunk = 32;     // sorted positions of a group
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kPart = 2048;    // keys that one workgroup of the sort moves
constexpr int kDigits = 512;
constexpr int kFewParts = 16;   // parts whose workgroups count all keys
constexpr int kMostSlabs = 256; // workgroups that sort more parts

// First column of piece k of a row, V columns each.  The last piece is moved
// back to end with the row: what it shares with the one before is computed
// and written twice, with the same bits.
template <int V> __device__ inline int64_t column(int64_t k, int64_t cols)
{
    return k * V < cols - V ? k * V : cols - V;
}

__device__ inline int64_t token_at(const void *tokens, int bytes, int64_t i)
{
    return bytes == 8 ? ((const int64_t *)tokens)[i] : ((const int32_t *)tokens)[i];
}

// ---- forward ------------------------------------------------------------------

// A wave per token (several for few tokens); lanes read V adjacent elements
// each, so 16-bit rows move in pieces of 1 KiB, four of them in flight.  Bound
// by memory: 32768 tokens of a 65536 x 2048 bf16 table 35 us (134 MB written,
// about 35 MB of rows read; 4.8 TB/s).
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const void *tokens, int token_bytes, int64_t n, int64_t rows,
                                                          int64_t cols, const T *table, int64_t pitch, float scale,
                                                          T *y, int64_t y_pitch)
{
    const int64_t i = block_at_xz() * (kThreads / 64) + threadIdx.x / 64;
    if (i >= n)
        return;
    const int64_t t = token_at(tokens, token_bytes, i);
    const bool in = t >= 0 && t < rows;
    const T *src = table + (in ? t : 0) * pitch;
    T *dst = y + i * y_pitch;
    const int64_t pieces = (cols + V - 1) / V;
    constexpr int kAhead = 4;  // loads in flight
    for (int64_t k0 = threadIdx.x % 64 + 64 * blockIdx.y; k0 < pieces; k0 += 64 * kAhead * gridDim.y) {
        float v[kAhead][V];
        int64_t c[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            // past the end the first piece again, which is not written twice
            const int64_t k = k0 + q * 64 * gridDim.y;
            c[q] = column<V>(k < pieces ? k : k0, cols);
            load_vec(src + c[q], v[q]);
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            if (q > 0 && k0 + q * 64 * gridDim.y >= pieces)
                break;
#pragma unroll
            for (int j = 0; j < V; ++j)
                v[q][j] = in ? v[q][j] * scale : __builtin_nanf("");
            store_vec(dst + c[q], v[q]);
        }
    }
}

// ---- sort -----------------------------------------------------------------------

// One pass of a stable radix sort over the digit key >> shift, `bits` wide
// (<= 9).  The first pass reads the tokens and leaves out those without a
// gradient; later ones read the pass before.  Up to kFewParts parts of 2048
// keys, a workgroup takes one part and counts all keys (the digits of the keys
// before its own part and of all), so no pass needs a launch for its counts:
// parts times 4 or 8 bytes a key, from the L2.  The sort of 32768 tokens (16
// parts, two passes) takes less than the clearing beside it (134 MB, 27 us a
// pass, 5.0 TB/s).  That grows with the square of the tokens, so of more parts
// the digits are counted once, in a launch of their own, by at most kMostSlabs
// workgroups, which take several parts in turn and add each other's counts
// (gradient of 65536 x 8 bf16, us without and with that launch: 16384 tokens 34
// and 37, 32768 39 and 36, 65536 48 and 38, 2^20 640 and 142, 2^22 8070 and 388).
struct SortArgs {
    const void *tokens;
    int token_bytes;
    int64_t n, rows, padding;
    const uint32_t *key_in, *pos_in;
    uint32_t *key_out, *pos_out;
    int32_t *count;  // keys that are sorted: written by the first pass, read by the others
    int shift, bits;
    int passes;      // of this launch: all of them if one workgroup sorts, else one
    uint32_t parts;  // workgroups that sort; the others clear rows [clear_from, clear_to) of out
    int64_t slab;    // keys of one of them: a multiple of kPart
    uint32_t *table; // [parts][kDigits] counts of their digits, or NULL: every one counts all keys
    int64_t clear_from, clear_to, cols, out_pitch;
};

// A workgroup's share of the rows to clear, 16 bytes a lane; PAST: past the
// caches, for rows that start 16-byte aligned.  Nobody reads them soon, and
// the sums that follow find the caches clean (32768 tokens of a 65536 x 2048
// bf16 table 146 -> 137 us); of other rows both parts of a line would go to
// memory one by one.
template <typename T, int V, bool PAST> __device__ void clear_rows(T *out, const SortArgs &a)
{
    constexpr int W = V == 1 ? 1 : 16 / (int)sizeof(T);
    typedef typename VecOf<T, W>::V Vec;
    const int64_t blocks = gridDim.x - a.parts, rows = a.clear_to - a.clear_from;
    const int64_t pieces = (a.cols + W - 1) / W;
    // whole waves take rows, adjacent waves adjacent ones
    const int64_t wave = (int64_t)(blockIdx.x - a.parts) * kSortWaves + threadIdx.x / 64;
    for (int64_t r = wave; r < rows; r += blocks * kSortWaves) {
        T *dst = out + (a.clear_from + r) * a.out_pitch;
        for (int64_t k = threadIdx.x % 64; k < pieces; k += 64) {
            Vec *const at = (Vec *)(dst + column<W>(k, a.cols));
            if constexpr (PAST)
                __builtin_nontemporal_store(Vec{}, at);
            else
                *at = Vec{};
        }
    }
}

template <bool FIRST> __device__ inline bool sort_key(const SortArgs &a, int64_t i, uint32_t &key)
{
    if constexpr (FIRST) {
        const int64_t t = token_at(a.tokens, a.token_bytes, i);
        key = (uint32_t)t;
        return t >= 0 && t < a.rows && t != a.padding;
    }
    key = a.key_in[i];
    return true;
}

// Orders LDS accesses of the lanes of one wave, which runs in step.
__device__ inline void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Eight counters a digit, by lane: tokens repeat, and lanes that count at one
// address wait for each other.
constexpr int kCopies = 8;
struct SortShared {
    uint32_t before[kDigits][kCopies], from[kDigits][kCopies];
    uint32_t at[kSortWaves][kDigits];
    uint32_t wave_total[kSortWaves];
};

// The digits of a workgroup's keys, for a sort of many parts.
template <bool FIRST> __global__ __launch_bounds__(kSortThreads) void count_kernel(SortArgs a)
{
    __shared__ uint32_t counts[kDigits][kCopies];
    const int tid = threadIdx.x;
    for (int d = tid; d < kDigits * kCopies; d += kSortThreads)
        (&counts[0][0])[d] = 0;
    __syncthreads();
    const uint32_t mask = (1u << a.bits) - 1;
    const int64_t n = FIRST ? a.n : (int64_t)*a.count;
    const int64_t begin = (int64_t)blockIdx.x * a.slab, end = begin + a.slab < n ? begin + a.slab : n;
    constexpr int kAhead = kPart / kSortThreads;
    for (int64_t i0 = begin + tid; i0 < end; i0 += kPart) {
        uint32_t key[kAhead];
        bool have[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int64_t i = i0 + q * kSortThreads;
            have[q] = sort_key<FIRST>(a, i < end ? i : i0, key[q]) && i < end;
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
            if (have[q])
                atomicAdd(&counts[key[q] >> a.shift & mask][tid % kCopies], 1u);
    }
    __syncthreads();
    if (tid < kDigits) {
        uint32_t all = 0;
#pragma unroll
        for (int c = 0; c < kCopies; ++c)
            all += counts[tid][c];
        a.table[(int64_t)blockIdx.x * kDigits + tid] = all;
    }
}

template <bool FIRST> __device__ void sort_pass(const SortArgs &a, SortShared &sh)
{
    auto &before = sh.before, &from = sh.from;
    auto &at = sh.at;
    auto &wave_total = sh.wave_total;
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const uint32_t mask = (1u << a.bits) - 1;
    const int64_t n = FIRST ? a.n : (int64_t)*a.count;
    const int64_t begin = (int64_t)blockIdx.x * a.slab, end = begin + a.slab < n ? begin + a.slab : n;
    for (int d = tid; d < kDigits; d += kSortThreads) {
#pragma unroll
        for (int c = 0; c < kCopies; ++c)
            before[d][c] = from[d][c] = 0;
        for (int w = 0; w < kSortWaves; ++w)
            at[w][d] = 0;
    }
    __syncthreads();
    if (begin >= n && !(FIRST && blockIdx.x == 0))
        return;  // the whole workgroup
    // digits of the keys before the workgroup's own, and of the rest
    if (a.table) {
        uint32_t b = 0, f = 0;
        const int d = tid % kDigits, first = tid / kDigits;
#pragma unroll 8
        for (uint32_t p = first; p < a.parts; p += kSortThreads / kDigits) {
            const uint32_t c = a.table[(int64_t)p * kDigits + d];
            b += p < blockIdx.x ? c : 0;
            f += p < blockIdx.x ? 0 : c;
        }
        before[d][first] = b;
        from[d][first] = f;
    } else {
        // (loads in batches: one at a time would take its latency for each)
        constexpr int kAhead = 8;
        for (int64_t i0 = tid; i0 < n; i0 += kSortThreads * kAhead) {
            uint32_t key[kAhead];
            bool have[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const int64_t i = i0 + q * kSortThreads;
                have[q] = sort_key<FIRST>(a, i < n ? i : i0, key[q]) && i < n;
            }
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
                if (have[q])
                    atomicAdd(&(i0 + q * kSortThreads < begin ? before
                                                              : from)[key[q] >> a.shift & mask][lane % kCopies],
                              1u);
        }
    }
    uint32_t base = 0;  // place of the next key of digit `tid`
    for (int64_t part = begin;; part += kPart) {
        // each wave's keys of the part, kPart / kSortWaves adjacent ones, and
        // their digits
        constexpr int kOwn = kPart / kSortWaves / 64;
        const int64_t own = part + (int64_t)wave * kOwn * 64 + lane;
        uint32_t key[kOwn], pos[kOwn];
        bool have[kOwn];
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const int64_t i = own + k * 64;
            have[k] = i < n;
            key[k] = pos[k] = 0;
            if (have[k]) {
                have[k] = sort_key<FIRST>(a, i, key[k]);
                pos[k] = FIRST ? (uint32_t)i : a.pos_in[i];
            }
        }
#pragma unroll
        for (int k = 0; k < kOwn; ++k)
            if (have[k])
                atomicAdd(&at[wave][key[k] >> a.shift & mask], 1u);
        __syncthreads();
        if (part == begin) {
            // first place of each digit (threads 0..511, one digit each)
            uint32_t all = 0, earlier = 0;
            if (tid < kDigits)
#pragma unroll
                for (int c = 0; c < kCopies; ++c) {
                    earlier += before[tid][c];
                    all += from[tid][c];
                }
            all += earlier;
            uint32_t upto = all;
#pragma unroll
            for (int off = 1; off < 64; off *= 2) {
                const uint32_t u = __shfl_up(upto, off);
                if (lane >= off)
                    upto += u;
            }
            if (lane == 63)
                wave_total[wave] = upto;
            __syncthreads();
            if (tid < kDigits) {
                base = upto - all;
                for (int w = 0; w < wave; ++w)
                    base += wave_total[w];
                base += earlier;
            }
            if (FIRST && blockIdx.x == 0 && tid == 0) {
                uint32_t total = 0;
                for (int w = 0; w < kDigits / 64; ++w)
                    total += wave_total[w];
                *a.count = (int32_t)total;
            }
        }
        // then of each wave's first key of that digit
        if (tid < kDigits)
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = at[w][tid];
                at[w][tid] = base;
                base += c;
            }
        __syncthreads();
        // 64 keys at a time, in order: a key's place is its digit's next one
        // plus the lanes before it that hold the same digit
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const uint32_t d = key[k] >> a.shift & mask;
            uint64_t same = __ballot(have[k]);
            for (int b = 0; b < a.bits; ++b) {
                const uint64_t set = __ballot(have[k] && (d >> b & 1));
                same &= d >> b & 1 ? set : ~set;
            }
            if (have[k]) {
                const uint32_t place = at[wave][d] + __popcll(same & ((1ull << lane) - 1));
                a.key_out[place] = key[k];
                a.pos_out[place] = pos[k];
            }
            wave_sync();
            if (have[k] && (same >> lane) == 1)  // the last lane of its digit
                at[wave][d] += __popcll(same);
            wave_sync();
        }
        if (part + kPart >= end)
            break;  // the whole workgroup
        __syncthreads();
        for (int d = tid; d < kDigits; d += kSortThreads)
            for (int w = 0; w < kSortWaves; ++w)
                at[w][d] = 0;
        __syncthreads();
    }
}

template <typename T, int V, bool PAST, bool FIRST>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(SortArgs a, T *out)
{
    __shared__ SortShared sh;
    if (blockIdx.x >= a.parts) {
        clear_rows<T, V, PAST>(out, a);
        return;
    }
    sort_pass<FIRST>(a, sh);
    if constexpr (FIRST) {
        // the other passes of a single workgroup, which sees what it wrote
        uint32_t *key = (uint32_t *)a.key_in, *pos = (uint32_t *)a.pos_in;
        for (int p = 1; p < a.passes; ++p) {
            __syncthreads();
            a.key_in = a.key_out;
            a.pos_in = a.pos_out;
            a.key_out = key;
            a.pos_out = pos;
            key = (uint32_t *)a.key_in;
            pos = (uint32_t *)a.pos_in;
            a.shift += a.bits;
            sort_pass<false>(a, sh);
        }
    }
}

// ---- sums -----------------------------------------------------------------------

struct SumArgs {
    int64_t cols, dy_pitch, out_pitch;
    const uint32_t *key, *pos;
    const int32_t *count;
    float *part;        // [chunks][2][part_pitch]: sums of the token that enters, and of the one that leaves
    int64_t part_pitch;
    float scale;
    int lanes;          // lanes of a group: a power of two, 64 at least
    uint32_t slices;    // workgroups side by side over a row's columns
};

// Sums of the rows of each token.  Chunks of 32 positions, whatever the
// tokens, spread one that makes up a tenth of a batch over the device; eight
// rows are in flight a lane.  Bound by memory: 32768 x 2048 bf16 42 us (134 MB
// read, 33 MB written, beside what the clearing left to write).
template <typename T, int V> __global__ __launch_bounds__(kThreads) void sum_kernel(const T *dy, T *out, SumArgs a)
{
    const int64_t n = *a.count;
    const int64_t block = block_at(), strip = block / a.slices;
    const int64_t chunk = strip * (kThreads / a.lanes) + __builtin_amdgcn_readfirstlane(threadIdx.x / a.lanes);
    const int64_t begin = chunk * kChunk;
    if (begin >= n)
        return;
    const int64_t end = begin + kChunk < n ? begin + kChunk : n;
    const int64_t piece = (block - strip * a.slices) * a.lanes + threadIdx.x % a.lanes;
    if ((piece - threadIdx.x % 64) * V >= a.cols)
        return;  // the whole wave
    // lanes past the row's end repeat its last piece
    const int64_t c = column<V>(piece, a.cols);
    // A wave lies within one group, so the chunk's keys and positions, and
    // with them what happens at each of them, are the same in all its lanes:
    // lane k holds those of entry k (63: the entry before the chunk), and the
    // loop reads them as scalars.
    const int lane = threadIdx.x % 64, count = (int)(end - begin);
    const int64_t mine = lane == 63 ? (begin > 0 ? begin - 1 : begin) : begin + lane < n ? begin + lane : n - 1;
    const int keys = (int)a.key[mine], places = (int)a.pos[mine];
    const bool enters = begin > 0 && __builtin_amdgcn_readlane(keys, 63) == __builtin_amdgcn_readlane(keys, 0);
    const bool leaves = end < n && __builtin_amdgcn_readlane(keys, kChunk) ==
                                       __builtin_amdgcn_readlane(keys, kChunk - 1);
    float sum[V] = {};
    bool whole = !enters;  // the present token starts here
    constexpr int kAhead = 8;
    for (int i = 0; i < count; i += kAhead) {
        float v[kAhead][V];
        // past the end the last position again, which is not added
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const uint32_t row = __builtin_amdgcn_readlane(places, i + k < count ? i + k : count - 1);
            load_vec(dy + (int64_t)row * a.dy_pitch + c, v[k]);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i + k >= count)
                break;
#pragma unroll
            for (int j = 0; j < V; ++j)
                sum[j] += v[k][j];
            const bool last = i + k + 1 == count;
            const int key = __builtin_amdgcn_readlane(keys, i + k);
            if (!last && __builtin_amdgcn_readlane(keys, i + k + 1) == key)
                continue;
            if (whole && !(last && leaves)) {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    sum[j] *= a.scale;
                store_vec(out + (int64_t)(uint32_t)key * a.out_pitch + c, sum);
            } else {
                // the first half for a token that enters (whether or not it
                // also leaves), the second for one that starts here
                store_vec(a.part + (chunk * 2 + (whole ? 1 : 0)) * a.part_pitch + c, sum);
            }
#pragma unroll
            for (int j = 0; j < V; ++j)
                sum[j] = 0.f;
            whole = true;
        }
    }
}

// Joins a token that starts in one chunk and leaves it: its sums of that
// chunk and of all it enters, split over the four waves of a workgroup (64 *
// V columns), each in order, the waves' sums then in order.  Few chunks do:
// 5.6 us for 32768 tokens by Zipf's law.
template <typename T, int V> __global__ __launch_bounds__(kThreads) void join_kernel(T *out, SumArgs a)
{
    __shared__ float other[kThreads / 64 - 1][64][V + 1];
    const int64_t n = *a.count;
    const int64_t chunk = block_at_xz();
    const int64_t end = (chunk + 1) * kChunk;
    if (end >= n)
        return;
    const uint32_t key = a.key[end - 1];
    if (a.key[end] != key)
        return;
    const int64_t begin = chunk * kChunk;
    if (begin > 0 && a.key[begin - 1] == key)
        return;  // it started before (sorted: the chunk holds nothing else)
    // the last chunk it enters, 64 chunks a look
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int64_t last = chunk;
    for (uint64_t all = ~0ull; all == ~0ull;) {
        const int64_t first = (last + 1 + lane) * kChunk;
        all = __ballot(first < n && a.key[first] == key);
        last += all == ~0ull ? 64 : __builtin_ctzll(~all);
    }
    const int64_t piece = (int64_t)blockIdx.y * 64 + lane;
    const bool have = piece * V < a.cols;
    const int64_t c = have ? column<V>(piece, a.cols) : 0;
    const int64_t each = (last - chunk + kThreads / 64) / (kThreads / 64);
    const int64_t from = chunk + wave * each, to = from + each < last + 1 ? from + each : last + 1;
    float sum[V] = {};
#pragma unroll 4
    for (int64_t k = from; k < to; ++k) {
        float v[V];
        load_vec(a.part + (k * 2 + (k == chunk ? 1 : 0)) * a.part_pitch + c, v);
#pragma unroll
        for (int j = 0; j < V; ++j)
            sum[j] += v[j];
    }
    if (wave > 0)
#pragma unroll
        for (int j = 0; j < V; ++j)
            other[wave - 1][lane][j] = sum[j];
    __syncthreads();
    if (wave > 0 || !have)
        return;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        for (int w = 0; w < kThreads / 64 - 1; ++w)
            sum[j] += other[w][lane][j];
        sum[j] *= a.scale;
    }
    store_vec(out + (int64_t)key * a.out_pitch + c, sum);
}

// Workspace: key and position arrays of two passes, the count, the digits'
// counts of many parts, the partial sums.
struct EmbedLayout {
    uint64_t key[2], pos[2], count, table, part, total;
    int64_t part_pitch;
};

EmbedLayout embed_layout(int64_t n, int64_t cols)
{
    EmbedLayout l;
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t here = at;
        at = round256(at + bytes);
        return here;
    };
    for (int k = 0; k < 2; ++k) {
        l.key[k] = take(4 * (uint64_t)n);
        l.pos[k] = take(4 * (uint64_t)n);
    }
    l.count = take(4);
    l.table = take(ceil_div(n, kPart) > kFewParts ? 4ull * kMostSlabs * kDigits : 0);
    l.part_pitch = ceil_div(cols, kVec) * kVec;
    l.part = take(8 * (uint64_t)ceil_div(n, kChunk) * (uint64_t)l.part_pitch);
    l.total = at;
    return l;
}

bool embed_sizes_ok(int64_t n, int64_t rows, int64_t cols)
{
    return n >= 0 && n < ((int64_t)1 << 31) && rows >= 1 && rows < ((int64_t)1 << 31) && cols >= 1 &&
           cols < ((int64_t)1 << 31);
}

}  // namespace
}  // namespace rotor

using namespace rotor;

extern "C" {

int32_t rotor_embedding(int32_t type, int64_t n_tokens, int64_t n_rows, int64_t cols, const void *d_tokens,
                        int32_t token_bytes, const void *d_table, int64_t table_pitch, double scale, void *d_y,
                        int64_t y_pitch, void *stream)
{
    if (!type_ok(type) || !embed_sizes_ok(n_tokens, n_rows, cols) || (token_bytes != 4 && token_bytes != 8))
        return ROTOR_EINVAL;
    const int64_t es = elem_bytes(type);
    if (!matrix_ok(d_table, n_rows, cols, table_pitch, es) || !matrix_ok(d_y, n_tokens, cols, y_pitch, es))
        return ROTOR_EINVAL;
    if (n_tokens == 0)
        return ROTOR_OK;
    if (!d_tokens || (uintptr_t)d_tokens % (uintptr_t)token_bytes)
        return ROTOR_EINVAL;
    (void)hipGetLastError();  // an error the caller's earlier calls left behind is not this launch's
    with_type(type, [&](auto e) {
        typedef typename decltype(e)::T T;
        // few tokens: a row's pieces over several waves
        const int64_t pieces = ceil_div(cols, 64 * kVec);
        const int64_t slices = n_tokens >= 1024 ? 1 : pieces < 64 ? pieces : 64;
        const auto kernel = cols >= kVec ? lookup_kernel<T, kVec> : lookup_kernel<T, 1>;
        kernel<<<grid_of(ceil_div(n_tokens, kThreads / 64), slices), kThreads, 0, (hipStream_t)stream>>>(d_tokens, token_bytes, n_tokens, n_rows, cols, (const T *)d_table,
                                        table_pitch, (float)scale, (T *)d_y, y_pitch);
    });
    return hipGetLastError() == hipSuccess ? ROTOR_OK : ROTOR_EDEVICE;
}

int32_t rotor_embedding_workspace_bytes(int64_t n_tokens, int64_t n_rows, int64_t cols, uint64_t *bytes)
{
    if (!bytes || !embed_sizes_ok(n_tokens, n_rows, cols))
        return ROTOR_EINVAL;
    *bytes = embed_layout(n_tokens, cols).total;
    return ROTOR_OK;
}

int32_t rotor_embedding_backward(int32_t type, int64_t n_tokens, int64_t n_rows, int64_t cols, const void *d_tokens,
                                 int32_t token_bytes, const void *d_dy, int64_t dy_pitch, double scale,
                                 int64_t padding, void *d_dtable, int64_t dtable_pitch, void *d_work,
                                 uint64_t work_bytes, void *stream)
{
    if (!type_ok(type) || !embed_sizes_ok(n_tokens, n_rows, cols) || (token_bytes != 4 && token_bytes != 8) ||
        padding < -1 || padding >= n_rows)
        return ROTOR_EINVAL;
    const int64_t es = elem_bytes(type);
    if (!matrix_ok(d_dy, n_tokens, cols, dy_pitch, es) || !matrix_ok(d_dtable, n_rows, cols, dtable_pitch, es))
        return ROTOR_EINVAL;
    if (n_tokens > 0 && (!d_tokens || (uintptr_t)d_tokens % (uintptr_t)token_bytes))
        return ROTOR_EINVAL;
    const EmbedLayout l = embed_layout(n_tokens, cols);
    if (!d_work || (uintptr_t)d_work % 16 || work_bytes < l.total)
        return ROTOR_EINVAL;
    char *const w = (char *)d_work;
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();  // an error the caller's earlier calls left behind is not this launch's

    // as few passes as digits of 9 bits allow, of equal width
    int bits = 0;
    while (((int64_t)1 << bits) < n_rows)
        ++bits;
    const int passes = bits <= 9 ? 1 : (bits + 8) / 9;
    const int width = bits == 0 ? 1 : (bits + passes - 1) / passes;
    SortArgs a{};
    a.tokens = d_tokens;
    a.token_bytes = token_bytes;
    a.n = n_tokens;
    a.rows = n_rows;
    a.padding = padding;
    a.count = (int32_t *)(w + l.count);
    a.bits = width;
    const int64_t parts = n_tokens > 0 ? ceil_div(n_tokens, kPart) : 1;
    const bool many = parts > kFewParts;
    a.slab = kPart * ceil_div(parts, many ? kMostSlabs : parts);
    a.parts = (uint32_t)(many ? ceil_div(n_tokens, a.slab) : parts);
    a.table = many ? (uint32_t *)(w + l.table) : nullptr;
    a.cols = cols;
    a.out_pitch = dtable_pitch;
    SumArgs b;
    b.cols = cols;
    b.dy_pitch = dy_pitch;
    b.out_pitch = dtable_pitch;
    b.key = (const uint32_t *)(w + l.key[(passes + 1) % 2]);
    b.pos = (const uint32_t *)(w + l.pos[(passes + 1) % 2]);
    b.count = a.count;
    b.part = (float *)(w + l.part);
    b.part_pitch = l.part_pitch;
    b.scale = (float)scale;
    b.lanes = 64;
    while (b.lanes < kThreads && b.lanes * kVec < cols)
        b.lanes *= 2;
    const int64_t chunks = ceil_div(n_tokens, kChunk);
    b.slices = (uint32_t)ceil_div(cols, (int64_t)b.lanes * kVec);
    const int64_t sum_blocks = ceil_div(chunks, kThreads / b.lanes) * b.slices;
    const int64_t join_slices = ceil_div(cols, 64 * kVec);
    if (join_slices > 65535 || !grid_ok(sum_blocks))
        return ROTOR_EINVAL;
    with_type(type, [&](auto e) {
        typedef typename decltype(e)::T T;
        T *const out = (T *)d_dtable;
        const int launches = a.parts == 1 ? 1 : passes;
        a.passes = passes / launches;
        for (int p = 0; p < launches; ++p) {
            a.key_in = (const uint32_t *)(w + l.key[(p + 1) % 2]);
            a.pos_in = (const uint32_t *)(w + l.pos[(p + 1) % 2]);
            a.key_out = (uint32_t *)(w + l.key[p % 2]);
            a.pos_out = (uint32_t *)(w + l.pos[p % 2]);
            a.shift = p * width;
            a.clear_from = n_rows * p / launches;
            a.clear_to = n_rows * (p + 1) / launches;
            // a row a wave, up to four workgroups on every CU
            const int64_t clear = ceil_div(a.clear_to - a.clear_from, kSortWaves);
            const dim3 grid(a.parts + (uint32_t)(clear < 1024 ? clear : 1024));
            const bool past = ((uintptr_t)out | (uintptr_t)(dtable_pitch * es)) % 16 == 0;
            const auto sort =
                cols < kVec ? (p == 0 ? sort_kernel<T, 1, false, true> : sort_kernel<T, 1, false, false>)
                : past      ? (p == 0 ? sort_kernel<T, kVec, true, true> : sort_kernel<T, kVec, true, false>)
                            : (p == 0 ? sort_kernel<T, kVec, false, true> : sort_kernel<T, kVec, false, false>);
            if (many)
                (p == 0 ? count_kernel<true> : count_kernel<false>)<<<dim3(a.parts), kSortThreads, 0, s>>>(a);
            sort<<<grid, kSortThreads, 0, s>>>(a, out);
        }
        const auto sum = cols >= kVec ? sum_kernel<T, kVec> : sum_kernel<T, 1>;
        const auto join = cols >= kVec ? join_kernel<T, kVec> : join_kernel<T, 1>;
        if (chunks > 0)
            sum<<<grid_of(sum_blocks), kThreads, 0, s>>>((const T *)d_dy, out, b);
        if (chunks > 1)
            join<<<grid_of(chunks - 1, join_slices), kThreads, 0, s>>>(out, b);
    });
    return hipGetLastError() == hipSuccess ? ROTOR_OK : ROTOR_EDEVICE;
}

}  // extern "C"
