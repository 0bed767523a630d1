// Dropout of a matrix (scar_dropout_apply of scar.h): y = residual + m . x, the mask computed on the way (mask.cuh).  The same
// call with the same rule is its own gradient.
//
// What bounds it: memory, once the generator's multiplications hide under it.
#include <algorithm>

#include "mask.cuh"

using namespace scar;

namespace {

constexpr unsigned kThreads = 256;

template <typename T> struct DropArgs {
    const T *x, *res;
    T *y;
    unsigned long long x_pitch, res_pitch, y_pitch;
    unsigned rows, cols;
    DropRule rule;
};

template <typename T> union Pack8 {
    uint4 u[sizeof(T) / 2];
    T v[8];
};
template <typename T> __device__ __forceinline__ Pack8<T> load8(const T *p) {
    Pack8<T> x;
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i) x.u[i] = reinterpret_cast<const uint4 *>(p)[i];
    return x;
}
template <typename T> __device__ __forceinline__ void store8(T *p, const Pack8<T> &x) {
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = x.u[i];
}

// Rows on 16-byte boundaries: a thread has kEach blocks of eight columns, kThreads apart, all of their loads before the
// generator's work.  The last block of a row may be short: it goes element by element.
template <typename T, bool RES, int kEach>
__global__ void __launch_bounds__(kThreads) k_dropout_words(const __grid_constant__ DropArgs<T> g) {
    const unsigned blocks = (g.cols + 7) / 8;
    const unsigned long long total = (unsigned long long)g.rows * blocks;
    const unsigned long long first = (unsigned long long)blockIdx.x * (kThreads * kEach) + threadIdx.x;
    unsigned row[kEach], block[kEach], left[kEach];
    Pack8<T> x[kEach], r[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const unsigned long long at = first + i * kThreads;
        row[i] = total >> 32 ? (unsigned)(at / blocks) : (unsigned)at / blocks;
        block[i] = (unsigned)(at - (unsigned long long)row[i] * blocks);
        left[i] = at < total ? min(8u, g.cols - block[i] * 8) : 0u;
        const T *px = g.x + row[i] * g.x_pitch + block[i] * 8ull, *pr = RES ? g.res + row[i] * g.res_pitch + block[i] * 8ull : nullptr;
        if (left[i] == 8) {
            x[i] = load8(px);
            if (RES) r[i] = load8(pr);
        } else {
#pragma unroll
            for (unsigned j = 0; j < 8; ++j)
                if (j < left[i]) {
                    x[i].v[j] = px[j];
                    if (RES) r[i].v[j] = pr[j];
                }
        }
    }
    const unsigned long long offset = g.rule.at();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        float2 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = Two<T>::get(x[i].v + 2 * j);
        if (g.rule.on) mask_apply(g.rule, mask_bits(g.rule, offset, row[i], block[i]), v);
#pragma unroll
        for (int j = 0; j < 4; ++j) Two<T>::put(x[i].v + 2 * j, RES ? add2(Two<T>::get(r[i].v + 2 * j), v[j]) : v[j]);
        T *py = g.y + row[i] * g.y_pitch + block[i] * 8ull;
        if (left[i] == 8) {
            store8(py, x[i]);
        } else {
#pragma unroll
            for (unsigned j = 0; j < 8; ++j)
                if (j < left[i]) py[j] = x[i].v[j];
        }
    }
}

// Rows anywhere: a warp has 256 columns of a row.  Each lane computes the mask of eight neighbouring columns and takes every
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
    const uint64_t todo = words ? (uint64_t)g.rows * ((g.cols + 7) / 8) : (uint64_t)g.rows * ((g.cols + 255) / 256) * 32;
    const uint64_t per = words ? 2ull * kThreads : kThreads, ctas = (todo + per - 1) / per;
    if (ctas >= 1ull << 31) return SCAR_ERR_CAPACITY;
    if (words) {
        if (g.res) k_dropout_words<T, true, 2><<<(unsigned)ctas, kThreads, 0, stream>>>(g);
        else k_dropout_words<T, false, 2><<<(unsigned)ctas, kThreads, 0, stream>>>(g);
    } else {
        if (g.res) k_dropout_lines<T, true><<<(unsigned)ctas, kThreads, 0, stream>>>(g);
        else k_dropout_lines<T, false><<<(unsigned)ctas, kThreads, 0, stream>>>(g);
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
