// Matrix products of the cross entropy: C[j][i] = sum over k of A(i, k) B(j, k),
// operands 16-bit, k adjacent in A's memory and k or j in B's, sums in 32
// bits on the matrix units, a tile's results handed to an epilogue while they
// are in registers.
#pragma once

#include "rotor_ops.h"

namespace rotor {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Mfma;
template <> struct Mfma<bf16> {
    typedef bf16 Frag __attribute__((ext_vector_type(8)));
    static __device__ f32x4 run(Frag a, Frag b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mfma<f16> {
    typedef f16 Frag __attribute__((ext_vector_type(8)));
    static __device__ f32x4 run(Frag a, Frag b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};

#if defined(__HIP_DEVICE_COMPILE__)
// The transposing read of four 16-bit elements: of the 16 lanes that address
// four rows of 16 columns, lane i gets column i of the four rows.
typedef short Turned __attribute__((ext_vector_type(4)));
__device__ inline Turned turned(const char *lds)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Turned *)lds);
}
#endif

// An operand: `rows` rows of `cols` elements, `pitch` elements apart, 16-byte
// aligned, cols a multiple of 8.  The summed index k runs along the rows, or,
// for B in a product with KB set, over them.  A 32-bit matrix is held as three
// bf16 terms whose sum has its 24 bits, the terms of a row `seg` elements
// apart.
template <typename T> struct Operand {
    const T *p;
    int64_t rows, cols, pitch, seg;
};

// The products of terms (a, b) whose sum is the product of two 32-bit
// matrices: all that are not below 2^-24 of the largest, the smallest first.
// 16-bit operands take the last one alone.
// An infinity times the other operand's terms is right in the last product
// alone: the others hold 0 or the other sign, and make NaN.  Where a result with
// an infinity among its factors counts (a logit: minus infinity masks a row of
// W), what the first five give is therefore kept only if it is finite; it is
// below 2^-7 of the last, so it is not finite for another reason unless the last
// is not either. (1000 x 10007 x 1024 f32, forward: 147 us so, 143 without.)
constexpr int kTerms = 3;
constexpr int kTermProducts = 6;
__device__ constexpr int term_a(int s) { return 0x124 >> (2 * s) & 3; }  // 0 1 2 0 1 0
__device__ constexpr int term_b(int s) { return 0x046 >> (2 * s) & 3; }  // 2 1 0 1 0 0

// The three bf16 terms of a 32-bit value.  Infinities and NaN stay in the
// first; finite values above the largest bf16 do not become one.
__device__ inline void split(float v, bf16 (&t)[kTerms])
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr float kMost = 3.3895314e38f;  // of bf16
    const bool finite = fabsf(v) <= 3.4028235e38f;
    t[0] = (bf16)(finite ? __builtin_amdgcn_fmed3f(v, -kMost, kMost) : v);
    const float r = finite ? v - (float)t[0] : 0.f;
    t[1] = (bf16)r;
    t[2] = (bf16)(r - (float)t[1]);
#endif
}

// Element type of the products of a call: bf16 terms for 32-bit tensors.
template <typename T> struct ProductOf {
    typedef T P;
    static constexpr int kParts = 1;
};
template <> struct ProductOf<float> {
    typedef bf16 P;
    static constexpr int kParts = kTerms;
};

// exp(x - m), m2 = m log2(e): one multiplication-addition and the hardware's
// power of two.
constexpr float kLog2e = 1.44269504088896341f;
__device__ inline float exp_over(float x, float m2)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2e, -m2));
#else
    return 0.f * (x + m2);
#endif
}

// A maximum and the sum of exponentials above it.
struct Soft {
    float top, sum;
};
__device__ inline float finite_or_0(float v) { return fabsf(v) <= 3.4028234e38f ? v : 0.f; }
__device__ inline Soft join(Soft a, Soft b)
{
    const float top = fmaxf(a.top, b.top), m = finite_or_0(top);
    return Soft{top, a.sum * __expf(a.top - m) + b.sum * __expf(b.top - m)};
}

constexpr int kStep = 64;         // of k in one step
constexpr int kRowBytes = 2 * kStep;

struct ProductArgs {
    int64_t k;
    int products;     // kTermProducts, or 1
    int tiles_i, tiles_j;
    int steps;        // of all products, ceil(k / kStep) each
    int split_steps;  // of one part (grid y)
};

// Which of a product's extents is that of the tokens that count, whose number is
// on the device (an epilogue's `live`): none of them (all tokens count), the
// rows of A, those of B, or the summed index.
enum Live { kLiveNone, kLiveA, kLiveB, kLiveK };

// The shape of a workgroup's tile: BI x BJ results, WI x WJ waves.
template <int BI_, int BJ_, int WI_, int WJ_> struct Tile {
    static constexpr int BI = BI_, BJ = BJ_, WI = WI_, WJ = WJ_;
    static constexpr int kWaves = WI * WJ, kThreads = kWaves * 64;
    static constexpr int NI = BI / WI / 16, NJ = BJ / WJ / 16;  // 16 x 16 results of a wave
    static constexpr int kBytes = (BI + BJ) * kRowBytes;
    static constexpr int kLoadsA = BI / 8 / kWaves, kLoadsB = BJ / 8 / kWaves;  // of a wave in one step
};

// A wave's results: element r of acc[ii][jj] of a lane is row (of A)
// i + 16 ii + r and row (of B) j + 16 jj of the tile that starts at
// (tile_i * BI, tile_j * BJ).
template <typename S> struct Results {
    f32x4 acc[S::NI][S::NJ];
    int tile_i, tile_j;
    int i, j;
    int wave_i, wave_j, lane;
    int part;
    char *lds;  // the wave's own share of LDS
};

// Hides where a value comes from, so that what is computed from it stays
// where it is written: the epilogues' addresses would otherwise be computed
// before the product's loop and spilled.
__device__ inline void opaque(int &v) { asm volatile("" : "+v"(v)); }

// Writes a wave's results, rounded to 16 bits, row by row of j: c is the
// tile's first element, rows and cols what the matrix has from there.  They go
// through the wave's share of LDS, half of them at a time, so that a row's 32
// NI bytes are written at once (straight from the registers it would be 32
// bytes a row and store); a row's 16-byte pieces change places by the row, for
// the banks' sake.
template <typename T, typename S>
__device__ inline void put_rows(const Results<S> &r, T *c, int pitch, int rows, int cols)
{
    typedef T V4 __attribute__((ext_vector_type(4)));
    typedef T V8 __attribute__((ext_vector_type(8)));
    constexpr int kRow = S::NI * 32, kPieces = S::NI * 2, kAtOnce = 64 / kPieces, kHalf = S::NJ / 2;
    static_assert(kHalf * 16 * kRow <= S::kBytes / S::kWaves, "the wave's share of LDS");
    const int low = r.lane % 16, high = r.lane / 16;
    int line = r.lane / kPieces;
    opaque(line);
    const int piece = r.lane % kPieces, i = r.wave_i * S::NI * 16 + piece * 8;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int jj = 0; jj < kHalf; ++jj)
#pragma unroll
            for (int ii = 0; ii < S::NI; ++ii) {
                V4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = (T)r.acc[ii][half * kHalf + jj][e];
                *(V4 *)(r.lds + (16 * jj + low) * kRow + ((2 * ii + high / 2) ^ (low % kPieces)) * 16 +
                        high % 2 * 8) = v;
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int k = 0; k < kHalf * 16 / kAtOnce; ++k) {
            const int row = line + k * kAtOnce, j = (r.wave_j * S::NJ + half * kHalf) * 16 + row;
            const V8 v = *(const V8 *)(r.lds + row * kRow + (piece ^ (row % 16 % kPieces)) * 16);
            if (j < rows) {
                T *const at = c + (uint32_t)(j * pitch + i);
                if (i + 8 <= cols)
                    *(typename VecOf<T, 8>::V *)at = v;
                else
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (i + e < cols)
                            at[e] = v[e];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// Tile order: the eight XCDs (workgroups go to them in turn) take contiguous
// runs, so that what neighbours share stays in one XCD's L2; in a run four
// tiles of j for each tile of i.
__device__ inline void tile_of(int id, int tiles_i, int tiles_j, int &ti, int &tj)
{
    const int n = tiles_i * tiles_j, xcd = id % 8, q = n / 8, r = n % 8;
    id = xcd * q + (xcd < r ? xcd : r) + id / 8;
    constexpr int kGroup = 4;
    const int group = id / (kGroup * tiles_i), first = group * kGroup;
    const int width = tiles_j - first < kGroup ? tiles_j - first : kGroup;
    const int in = id - group * kGroup * tiles_i;
    ti = in / width;
    tj = first + in % width;
}

// Buffer descriptors exist in device code only: the host's pass sees a kernel
// without a body.
#if defined(__HIP_DEVICE_COMPILE__)
template <typename T> __device__ inline __amdgpu_buffer_rsrc_t rsrc_of(const T *p, int64_t elements)
{
    const int64_t bytes = elements * (int64_t)sizeof(T);
    return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)(bytes < 0x7FFFFFFF ? bytes : 0x7FFFFFFF),
                                             0x00020000);
}

typedef __attribute__((address_space(3))) void *lds_ptr;

// One operand's part of a step, global memory to LDS without registers, and
// its fragments out of LDS.  SIDE: rows (columns) of the workgroup's tile;
// LOADS: of a wave in one step; N: fragments of a wave.  What lies outside
// the operand comes as 0 (the buffer's bound).
template <typename T, int SIDE, int LOADS, int N, bool KROWS> struct Loader;

// k along the rows.  A wave's load moves 8 rows of 128 bytes; row r's 16-byte
// piece c lands in place c ^ (r % 8), so that the 16 rows a fragment reads lie
// in different banks.
template <typename T, int SIDE, int LOADS, int N> struct Loader<T, SIDE, LOADS, N, false> {
    __amdgpu_buffer_rsrc_t rsrc;
    uint32_t at[LOADS];
    int limit;  // bytes of k before this lane's piece leaves the row
    int first;  // LDS byte of this wave's first load
    int base, swz[2];
    __device__ void init(const Operand<T> &o, int64_t side0, int wave, int lane, int wave_side)
    {
        const int64_t have = o.rows - side0 < SIDE ? o.rows - side0 : SIDE;
        rsrc = rsrc_of(o.p + side0 * o.pitch, (have - 1) * o.pitch + o.seg * (kTerms - 1) + o.cols);
        const int piece = (lane % 8) ^ (lane / 8);
#pragma unroll
        for (int q = 0; q < LOADS; ++q)
            at[q] = (uint32_t)((wave * LOADS + q) * 8 + lane / 8) * (uint32_t)(o.pitch * sizeof(T)) + piece * 16;
        limit = (int)(o.cols * sizeof(T)) - piece * 16;
        first = wave * LOADS * 1024;
        const int row = lane % 16;
        base = (wave_side * N * 16 + row) * kRowBytes;
        swz[0] = ((lane / 16) ^ (row & 7)) * 16;
        swz[1] = ((4 + lane / 16) ^ (row & 7)) * 16;
    }
    // `term`: elements from a row's start to its term; `step`: of k
    __device__ void load(const Operand<T> &, char *lds, int64_t term, int step, bool live) const
    {
        const int kb = live ? step * kRowBytes : 0x7FFFFF00;
        const uint32_t off = (uint32_t)(term * sizeof(T)) + (uint32_t)kb;
        const bool in = kb < limit;
#pragma unroll
        for (int q = 0; q < LOADS; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)(lds + first + q * 1024), 16,
                                                     in ? at[q] + off : 0x80000000u, 0, 0, 0);
    }
    __device__ void read(const char *lds, int h, typename Mfma<T>::Frag (&f)[N]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
            f[n] = *(const typename Mfma<T>::Frag *)(lds + base + swz[h] + n * 16 * kRowBytes);
    }
};

// k over the rows: LDS holds 64 rows of SIDE elements, and the transposing
// read hands four rows' elements of one column to a lane (its 16 lanes address
// four rows of 16 columns).  The 16 rows that a read touches are spread over
// the banks by the 32-byte slots' places, s ^ (r % 4 + 4 (r / 8 % 2)).
template <typename T, int SIDE, int LOADS, int N> struct Loader<T, SIDE, LOADS, N, true> {
    static constexpr int kRow = SIDE * 2, kLanes = kRow / 16;  // bytes of a row, and lanes that load it
    const T *start;
    int64_t cols;
    uint32_t at[LOADS];
    int first, base;
    static __device__ int turn(int row) { return (row & 3) | (row >> 3 & 1) << 2; }
    __device__ void init(const Operand<T> &o, int64_t side0, int wave, int lane, int wave_side)
    {
        start = o.p + side0;
        cols = o.cols - side0 + o.seg * (kTerms - 1);
#pragma unroll
        for (int q = 0; q < LOADS; ++q) {
            const int row = (wave * LOADS + q) * (64 / kLanes) + lane / kLanes;
            at[q] = (uint32_t)row * (uint32_t)(o.pitch * sizeof(T)) + ((lane % kLanes) ^ (turn(row) << 1)) * 16;
        }
        first = wave * LOADS * 1024;
        const int g = lane / 16, i = lane % 16;
        // bits 5 to 7 hold the place of the wave's first slot of 32 bytes: its
        // n-th is at base ^ (32 n)
        const int slot = wave_side * N;
        base = (g * 8 + i / 4) * kRow + i % 4 * 8 + ((slot & ~7) | ((slot & 7) ^ turn(g * 8 + i / 4))) * 32;
    }
    __device__ void load(const Operand<T> &o, char *lds, int64_t term, int step, bool live) const
    {
        const int64_t row0 = (int64_t)step * kStep, have = o.rows - row0 < kStep ? o.rows - row0 : kStep;
        const auto rsrc = rsrc_of(start + row0 * o.pitch, live && have > 0 ? (have - 1) * o.pitch + cols : 0);
        const uint32_t off = (uint32_t)(term * sizeof(T));
#pragma unroll
        for (int q = 0; q < LOADS; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)(lds + first + q * 1024), 16, at[q] + off, 0, 0,
                                                     0);
    }
    __device__ void read(const char *lds, int h, typename Mfma<T>::Frag (&f)[N]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const char *p = lds + (base ^ (n * 32)) + h * 32 * kRow;
            f[n] = __builtin_bit_cast(typename Mfma<T>::Frag,
                                      __builtin_shufflevector(turned(p), turned(p + 4 * kRow), 0, 1, 2, 3, 4, 5, 6,
                                                              7));
        }
    }
};

// A barrier that waits only for what it names: a workgroup barrier of the
// language would also wait for the loads that the next phases hide.
enum { kWaitNone, kWaitLds, kWaitAll };
template <int WAIT> __device__ inline void phase_barrier()
{
    __builtin_amdgcn_sched_barrier(0);
    if (WAIT == kWaitAll)
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else if (WAIT == kWaitLds)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else
        asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
#endif

// Bound by the matrix units and, close behind, by LDS: for 32 of k a tile of
// 256 x 256 takes 512 cycles of every SIMD's matrix unit for each group, and
// 384 (reads) + 128 (arriving operands) cycles of LDS.  Measured on 8192 x 8192
// results, TF/s at k = 2048, 4096, 8192, 32-bit sums stored: two buffers and
// one barrier a step 944, 966, 1121; with the waves that multiply at a higher
// priority 1073, 1233, 1306; four waves of 128 x 128 each 740, 806, 863; four
// buffers of 32 with counted waits 1066, 1183, 1247; two groups half a phase
// apart (this one) 1101, 1267, 1372, and 1398, 1480, 1514 without the stores.
// The library's product of 8192^3 reaches 1297 here, of 16384^3 1559.
// TERMS: of 32-bit operands, whose results may have infinite factors.
template <typename T, typename S, bool KB, bool TERMS, typename E>
__global__ __launch_bounds__(S::kThreads) void product_kernel(Operand<T> a, Operand<T> b, ProductArgs p, E epilogue)
{
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (E::kLive != kLiveNone) {
        const int n = *epilogue.live;
        if constexpr (E::kLive == kLiveA) {
            a.rows = n;
            p.tiles_i = (n + S::BI - 1) / S::BI;
        } else if constexpr (E::kLive == kLiveB) {
            b.rows = n;
            p.tiles_j = (n + S::BJ - 1) / S::BJ;
        } else {
            a.cols = (n + 7) / 8 * 8;
            b.rows = n;
            p.k = n > 0 ? n : 1;  // for no tokens a step of zeros
            p.steps = p.products * (int)((p.k + kStep - 1) / kStep);
            p.split_steps = (p.steps + (int)gridDim.y - 1) / (int)gridDim.y;
        }
        if ((int)blockIdx.x >= p.tiles_i * p.tiles_j)
            return;
    }
    // two steps: one is multiplied while the other arrives
    __shared__ __attribute__((aligned(1024))) char even[S::kBytes];
    __shared__ __attribute__((aligned(1024))) char odd[S::kBytes];
    typedef typename Mfma<T>::Frag Frag;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wi = wave / S::WJ, wj = wave % S::WJ;
    constexpr int kB = S::BI * kRowBytes;  // LDS byte of B's part
    const int per = (int)((p.k + kStep - 1) / kStep);
    const int t0 = blockIdx.y * p.split_steps;
    const int t1 = t0 + p.split_steps < p.steps ? t0 + p.split_steps : p.steps;
    const int tiles = p.tiles_i * p.tiles_j;

    int ti, tj, s, at;  // the tile; product and step of the next load
    Loader<T, S::BI, S::kLoadsA, S::NI, false> la;
    Loader<T, S::BJ, S::kLoadsB, S::NJ, KB> lb;
    auto load = [&](char *lds, bool live) {
        la.load(a, lds, term_a(s) * a.seg, at, live);
        lb.load(b, lds + kB, term_b(s) * b.seg, at, live);
        if ((!TERMS || live) && ++at == per) {
            at = 0;
            ++s;
        }
    };
    auto begin = [&](int id) {
        tile_of(id, p.tiles_i, p.tiles_j, ti, tj);
        la.init(a, (int64_t)ti * S::BI, wave, lane, wi);
        lb.init(b, (int64_t)tj * S::BJ, wave, lane, wj);
        s = kTermProducts - p.products + t0 / per;
        at = t0 % per;
        if (t0 < t1)
            load(even, true);
    };

    Results<S> res;
    Frag fa[S::NI], fb[S::NJ];
    auto read = [&](const char *lds, int h) {  // half h of a step: 32 of k
        lb.read(lds + kB, h, fb);
        la.read(lds, h, fa);
    };
    auto multiply = [&]() {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int ii = 0; ii < S::NI; ++ii)
#pragma unroll
            for (int jj = 0; jj < S::NJ; ++jj)
                res.acc[ii][jj] = Mfma<T>::run(fa[ii], fb[jj], res.acc[ii][jj]);
        __builtin_amdgcn_s_setprio(0);
    };

    // Where TERMS, the steps are those of all six products, in one part.  The
    // last product starts at an even step: after an odd number of them comes
    // one of zeros.
    const int low = (kTermProducts - 1) * per, dead = TERMS && low % 2 ? low : -1, last = low + low % 2;
    const int end = TERMS ? t1 + low % 2 : t1;
    auto drop_infinite = [&]() {
#pragma unroll
        for (int ii = 0; ii < S::NI; ++ii)
#pragma unroll
            for (int jj = 0; jj < S::NJ; ++jj)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    res.acc[ii][jj][e] = finite_or_0(res.acc[ii][jj][e]);
    };

    // A workgroup takes every gridDim.x-th tile; the next one's first step is
    // loaded while the epilogue works.
    begin(blockIdx.x);
    for (int id = blockIdx.x;;) {
#pragma unroll
        for (int ii = 0; ii < S::NI; ++ii)
#pragma unroll
            for (int jj = 0; jj < S::NJ; ++jj)
                res.acc[ii][jj] = f32x4{0.f, 0.f, 0.f, 0.f};
        // an odd number of steps is followed by one of zeros: one way out of
        // the loop, so that the sums stay where they are
        if constexpr (S::kWaves == 8) {
            // Two groups of four waves, one on each SIMD, half a phase apart:
            // while one multiplies what it holds (32 of k), the other reads
            // its next operands from LDS.  Every phase has two barriers; the
            // second group starts one barrier later and ends one earlier.  A
            // step's place in LDS is written again one barrier after the
            // other group's last read of it, and the loads into it are waited
            // for three phases later, one barrier before its first read.
            const bool late = wave >= 4;
            auto phase = [&](const char *lds, int h, char *next, bool live) {
                read(lds, h);
                __builtin_amdgcn_sched_barrier(0);
                if (next)
                    load(next, live);
                if (h == 1 && late)
                    phase_barrier<kWaitAll>();
                else
                    phase_barrier<kWaitLds>();
                multiply();
                if (h == 1 && !late)
                    phase_barrier<kWaitAll>();
                else
                    phase_barrier<kWaitNone>();
            };
            phase_barrier<kWaitAll>();
            if (late)
                phase_barrier<kWaitNone>();
            for (int t = t0; t < end; t += 2) {
                if (TERMS && t == last)
                    drop_infinite();
                phase(even, 0, odd, t + 1 < end && t + 1 != dead);
                phase(even, 1, nullptr, false);
                phase(odd, 0, even, t + 2 < end);
                phase(odd, 1, nullptr, false);
            }
            if (!late)
                phase_barrier<kWaitNone>();
            __syncthreads();
        } else {
            auto step = [&](const char *lds) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    read(lds, h);
                    multiply();
                }
            };
            __syncthreads();
            // (two loops: inside of one, dropping costs 5 of 57 us in 300 x
            // 8000 x 512 f32; of the large tiles it is the other way round)
            for (int from = t0, to = TERMS ? last : end;; from = to, to = end) {
                for (int t = from; t < to; t += 2) {
                    load(odd, t + 1 < end && t + 1 != dead);
                    step(even);
                    __syncthreads();
                    if (t + 2 < end)
                        load(even, true);
                    step(odd);
                    __syncthreads();
                }
                if (!TERMS || to == end)
                    break;
                drop_infinite();
            }
        }
        res.tile_i = ti;
        res.tile_j = tj;
        res.wave_i = wi;
        res.wave_j = wj;
        res.lane = lane;
        res.i = wi * S::NI * 16 + lane / 16 * 4;
        res.j = wj * S::NJ * 16 + lane % 16;
        res.part = blockIdx.y;
        res.lds = odd + wave * (S::kBytes / S::kWaves);
        id += gridDim.x;
        if (id < tiles)
            begin(id);
        opaque(res.i);
        opaque(res.j);
        epilogue(res, odd);
        if (id >= tiles)
            return;
    }
#endif
}

}  // namespace
}  // namespace rotor
