// rotor_dropout: y = residual + keep * x / (1 - q), the mask recomputed from
// a counter wherever it is needed.
//
// One thread takes groups of 8 elements: one counter of the generator gives
// 4 x 32 bits, 16 for each of the 8, so a mask costs ten rounds of two 32 x
// 32 -> 64 bit products per 8 elements.
#include "rotor_ops.h"

#include <math.h>

namespace rotor {
namespace {

constexpr int kGroup = 8;       // elements of one counter
constexpr int kThreads = 256;

struct DropArgs {
    int64_t rows, cols, x_pitch, r_pitch, y_pitch;
    uint64_t seed, step;
    const int64_t *d_step;
    uint32_t threshold;  // keep 16 bits >= threshold
    float scale;
};

// Philox4x32 with ten rounds: four words from a 128-bit counter under a
// 64-bit key.
__device__ inline void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
        c[0] = (uint32_t)(b >> 32) ^ c[1] ^ k0;
        c[1] = (uint32_t)b;
        c[2] = (uint32_t)(a >> 32) ^ c[3] ^ k1;
        c[3] = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// The 16 bits of element k of a group.
__device__ inline uint32_t bits_of(const uint32_t (&c)[4], int k)
{
    return k % 2 ? c[k / 2] >> 16 : c[k / 2] & 0xFFFFu;
}

// PACKED: all rows are adjacent (pitch == cols), so groups are contiguous.
//
// Bound by memory: the generator's twenty wide products for 8 elements hide
// under the loads of the other waves.  16 bits an element, not 32: p is met to
// 2^-17, and the generator costs half.  8192 x 4096 bf16: 37 us with a residual
// (201 MB, 5.4 TB/s), 23 us without (134 MB, 5.7 TB/s; a copy of 1 GiB reaches
// 5.1).
template <typename T, bool PACKED, bool RESIDUAL>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const T *x, const T *res, T *y, DropArgs a)
{
    const uint64_t g = (uint64_t)block_at() * kThreads + threadIdx.x;
    const uint64_t n = (uint64_t)a.rows * (uint64_t)a.cols;
    const uint64_t i0 = g * kGroup;
    if (i0 >= n)
        return;
    const int left = n - i0 < kGroup ? (int)(n - i0) : kGroup;
    float v[kGroup], r[kGroup];
    uint64_t row = 0, col = i0;
    bool whole = true;  // the group lies in one row
    if (!PACKED) {
        row = n <= 0xFFFFFFFFull ? (uint32_t)i0 / (uint32_t)a.cols : i0 / (uint64_t)a.cols;
        col = i0 - row * (uint64_t)a.cols;
        whole = col + left <= (uint64_t)a.cols;
    }
    if (whole) {
        load_some(x + row * a.x_pitch + col, left, v);
        if (RESIDUAL)
            load_some(res + row * a.r_pitch + col, left, r);
    } else {
        uint64_t rw = row, cl = col;
#pragma unroll
        for (int k = 0; k < kGroup; ++k) {
            v[k] = k < left ? (float)x[rw * a.x_pitch + cl] : 0.f;
            if (RESIDUAL)
                r[k] = k < left ? (float)res[rw * a.r_pitch + cl] : 0.f;
            if (++cl == (uint64_t)a.cols) {
                cl = 0;
                ++rw;
            }
        }
    }
    const uint64_t step = a.step + (a.d_step ? (uint64_t)*a.d_step : 0);
    uint32_t c[4] = {(uint32_t)g, (uint32_t)(g >> 32), (uint32_t)step, (uint32_t)(step >> 32)};
    philox(c, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
        // a select, not a product: what is dropped may be infinite or NaN
        v[k] = bits_of(c, k) >= a.threshold ? v[k] * a.scale : 0.f;
        if (RESIDUAL)
            v[k] += r[k];
    }
    if (whole) {
        store_some(y + row * a.y_pitch + col, left, v);
    } else {
#pragma unroll
        for (int k = 0; k < kGroup; ++k) {
            if (k < left)
                y[row * a.y_pitch + col] = (T)v[k];
            if (++col == (uint64_t)a.cols) {
                col = 0;
                ++row;
            }
        }
    }
}

template <typename T> void launch(const void *x, const void *res, void *y, const DropArgs &a, hipStream_t s)
{
    const dim3 grid = grid_of(ceil_div(a.rows * a.cols, (int64_t)kThreads * kGroup));
    const bool packed = a.x_pitch == a.cols && a.y_pitch == a.cols && (!res || a.r_pitch == a.cols);
    if (packed && res)
        dropout_kernel<T, true, true><<<grid, kThreads, 0, s>>>((const T *)x, (const T *)res, (T *)y, a);
    else if (packed)
        dropout_kernel<T, true, false><<<grid, kThreads, 0, s>>>((const T *)x, nullptr, (T *)y, a);
    else if (res)
        dropout_kernel<T, false, true><<<grid, kThreads, 0, s>>>((const T *)x, (const T *)res, (T *)y, a);
    else
        dropout_kernel<T, false, false><<<grid, kThreads, 0, s>>>((const T *)x, nullptr, (T *)y, a);
}

}  // namespace
}  // namespace rotor

using namespace rotor;

extern "C" int32_t rotor_dropout(int32_t type, int64_t rows, int64_t cols, const void *d_x, int64_t x_pitch,
                                 const void *d_residual, int64_t residual_pitch, void *d_y, int64_t y_pitch,
                                 double p, uint64_t seed, uint64_t step, const int64_t *d_step, void *stream)
{
    if (!type_ok(type) || !(p >= 0. && p <= 1.) || (uintptr_t)d_step % 8)
        return ROTOR_EINVAL;
    const int64_t es = elem_bytes(type);
    if (!matrix_ok(d_x, rows, cols, x_pitch, es) || !matrix_ok(d_y, rows, cols, y_pitch, es) ||
        (d_residual && !matrix_ok(d_residual, rows, cols, residual_pitch, es)))
        return ROTOR_EINVAL;
    if (rows == 0)
        return ROTOR_OK;
    if (!grid_ok(ceil_div(rows * cols, (int64_t)kThreads * kGroup)))
        return ROTOR_EINVAL;
    DropArgs a;
    a.rows = rows;
    a.cols = cols;
    if (x_pitch == cols && y_pitch == cols && (!d_residual || residual_pitch == cols)) {
        a.rows = 1;
        a.cols = x_pitch = y_pitch = residual_pitch = rows * cols;
    }
    a.x_pitch = x_pitch;
    a.r_pitch = residual_pitch;
    a.y_pitch = y_pitch;
    a.seed = seed;
    a.step = step;
    a.d_step = d_step;
    a.threshold = (uint32_t)lrint(p * 65536.);
    a.scale = a.threshold < 65536u ? (float)(65536. / (65536. - a.threshold)) : 0.f;
    (void)hipGetLastError();  // an error the caller's earlier calls left behind is not this launch's
    with_type(type, [&](auto e) {
        launch<typename decltype(e)::T>(d_x, d_residual, d_y, a, (hipStream_t)stream);
    });
    return hipGetLastError() == hipSuccess ? ROTOR_OK : ROTOR_EDEVICE;
}
