// Dropout of a matrix (scar_dropout_apply of scar.h): y = residual + m . x, the mask computed on the way (mask.cuh).  The same
// call with the same rule is its own gradient.
//
// What bounds it: memory (16384 x 8192 bfloat16 with a residual: 117 us back to back, 6.9 TB/s, 134 where inputs and outputs change from
// call to call; without one 99, where the generator's multiplications show); rows anywhere cost two aligned loads for one (4099 x 5003
// float16: 27 us, 3.1 TB/s; float32 rows 31, 5.3).
#include <algorithm>

#include "mask.cuh"
#include "rows.cuh"

using namespace scar;

namespace {

constexpr unsigned kThreads = 256;
// Blocks of a thread: 16384 x 8192 bfloat16 with a residual takes 134 / 117 / 132 us with one, two, four; rows anywhere (4099 x 5003 float16
// with one) 27 / 27 / 30.
constexpr int kEach = 2;

template <typename T> struct DropArgs {
    const T *x, *res;
    T *y;
    unsigned long long x_pitch, res_pitch, y_pitch;
    unsigned rows, cols;
    DropRule rule;
};

// A thread has kEach blocks of eight columns, kThreads apart, all of their loads before the generator's work.
template <typename T, bool RES, bool VEC, int kEach>
__global__ void __launch_bounds__(kThreads) k_dropout_words(const __grid_constant__ DropArgs<T> g) {
    const unsigned blocks = (g.cols + 7) / 8, lane = threadIdx.x & 31;
    const unsigned long long total = (unsigned long long)g.rows * blocks;
    const unsigned long long first = (unsigned long long)blockIdx.x * (kThreads * kEach) + threadIdx.x;
    unsigned row[kEach], block[kEach];
    Pack8<T> x[kEach], r[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const unsigned long long at = first + i * kThreads;
        row[i] = total >> 32 ? (unsigned)(at / blocks) : (unsigned)at / blocks;
        block[i] = (unsigned)(at - (unsigned long long)row[i] * blocks);
        if (at >= total) continue;
        x[i] = row8(g.x + row[i] * g.x_pitch, block[i] * 8, g.cols, VEC);
        if (RES) r[i] = row8(g.res + row[i] * g.res_pitch, block[i] * 8, g.cols, VEC);
    }
    const unsigned long long offset = g.rule.at();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const unsigned long long at = first + i * kThreads;
        float2 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = Two<T>::get(x[i].v + 2 * j);
        if (g.rule.on) mask_apply(g.rule, mask_bits(g.rule, offset, row[i], block[i]), v);
#pragma unroll
        for (int j = 0; j < 4; ++j) Two<T>::put(x[i].v + 2 * j, RES ? add2(Two<T>::get(r[i].v + 2 * j), v[j]) : v[j]);
        put8(g.y + row[i] * g.y_pitch, block[i] * 8, g.cols, VEC, x[i], at < total, lane < 31 && at + 1 < total && block[i] + 1 < blocks, lane > 0 && block[i] > 0);
    }
}

// float32 rows anywhere: a warp has 256 columns of a row.  Each lane computes the mask of eight neighbouring columns and takes every
// 32nd of the warp's columns, so that a load or store is one run of memory wherever it begins.
template <typename T, bool RES>
__global__ void __launch_bounds__(kThreads) k_dropout_lines(const __grid_constant__ DropArgs<T> g) {
    const unsigned spans = (g.cols + 255) / 256, lane = threadIdx.x & 31;
    const unsigned long long at = (unsigned long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const unsigned row = (unsigned)(at / spans), col0 = (unsigned)(at - (unsigned long long)row * spans) * 256;
    if (row >= g.rows) return;
    const T *px = g.x + row * g.x_pitch, *pr = RES ? g.res + row * g.res_pitch : nullptr;
    T *py = g.y + row * g.y_pitch;
    T x[8], r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned col = col0 + i * 32 + lane;
        if (col >= g.cols) continue;
        x[i] = px[col];
        if (RES) r[i] = pr[col];
    }
    const unsigned mask = mask_byte(g.rule, mask_bits(g.rule, g.rule.at(), row, col0 / 8 + lane));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned col = col0 + i * 32 + lane;
        const bool keep = __shfl_sync(0xffffffffu, mask, i * 4 + (lane >> 3)) >> (lane & 7) & 1u;
        if (col >= g.cols) continue;
        const float v = keep ? to_f32(x[i]) * g.rule.scale : 0.f;
        py[col] = from_f32<T>(RES ? to_f32(r[i]) + v : v);
    }
}

template <typename T> int run_dropout(const DropArgs<T> &g, cudaStream_t stream) {
    const auto whole = [](const T *p, unsigned long long pitch) { return (uintptr_t)p % 16 == 0 && pitch * sizeof(T) % 16 == 0; };
    const bool words = whole(g.x, g.x_pitch) && whole(g.y, g.y_pitch) && (!g.res || whole(g.res, g.res_pitch));
    const bool lines = !words && sizeof(T) == 4;
    const uint64_t todo = lines ? (uint64_t)g.rows * ((g.cols + 255) / 256) * 32 : (uint64_t)g.rows * ((g.cols + 7) / 8);
    const uint64_t per = words ? (uint64_t)kEach * kThreads : kThreads, ctas = (todo + per - 1) / per;
    if (ctas >= 1ull << 31) return SCAR_ERR_CAPACITY;
    if (lines) {
        if constexpr (sizeof(T) == 4) (g.res ? k_dropout_lines<T, true> : k_dropout_lines<T, false>)<<<(unsigned)ctas, kThreads, 0, stream>>>(g);
    } else if (words) {
        (g.res ? k_dropout_words<T, true, true, kEach> : k_dropout_words<T, false, true, kEach>)<<<(unsigned)ctas, kThreads, 0, stream>>>(g);
    } else {
        if constexpr (sizeof(T) == 2) (g.res ? k_dropout_words<T, true, false, 1> : k_dropout_words<T, false, false, 1>)<<<(unsigned)ctas, kThreads, 0, stream>>>(g);
    }
    TRAIN_TRY(cudaGetLastError());
    return SCAR_OK;
}

}  // namespace

extern "C" int scar_dropout_apply(const scar_dropout *rule, scar_dtype dtype, const void *d_x, uint64_t x_pitch, const void *d_residual,
                                  uint64_t residual_pitch, void *d_y, uint64_t y_pitch, uint64_t rows, uint64_t cols, void *cuda_stream) {
    DropRule r;
    if (!rule || !is_operand_type(dtype)) return SCAR_ERR_INVALID_ARG;
    int rc = make_rule(rule, &r);
    if (rc != SCAR_OK) return rc;
    if (rows >= 1ull << 31 || cols >= 1ull << 31) return SCAR_ERR_CAPACITY;
    if (rows == 0 || cols == 0) return SCAR_OK;
    const unsigned b = elem_size(dtype);
    if (!d_x || !d_y || (uintptr_t)d_x % b || (uintptr_t)d_y % b || (uintptr_t)d_residual % b) return SCAR_ERR_INVALID_ARG;
    const uint64_t far = 1ull << 40;  // rows times pitch stays below 2^63 bytes
    const auto fits = [&](uint64_t pitch) { return pitch < far && (rows == 1 || pitch >= cols); };
    if (!fits(x_pitch) || !fits(y_pitch) || (d_residual && !fits(residual_pitch))) return SCAR_ERR_INVALID_ARG;
    rc = SCAR_ERR_CUDA;
    dispatch_operand(dtype, [&](auto e) {
        using T = decltype(e);
        rc = run_dropout<T>({static_cast<const T *>(d_x), static_cast<const T *>(d_residual), static_cast<T *>(d_y), x_pitch, residual_pitch, y_pitch,
                             (unsigned)rows, (unsigned)cols, r},
                            static_cast<cudaStream_t>(cuda_stream));
    });
    return rc;
}
