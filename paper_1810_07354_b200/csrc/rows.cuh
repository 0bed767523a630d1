// Rows of a matrix eight values at a time, wherever they begin.
#pragma once
#include "train_common.cuh"

namespace scar {

// 16 bytes that begin `by` bytes (even, below 16) into the 32 bytes a, b.
__device__ __forceinline__ uint4 shifted(const uint4 &a, const uint4 &b, unsigned by) {
    unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (by & 8) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (by & 4) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    if (by & 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T> union Pack8 {
    uint4 u[sizeof(T) / 2];
    T v[8];
};
// Eight values from column c of a row of n that begins anywhere (`vec`: on a 16-byte boundary), zeros behind the last one.
template <typename T> __device__ __forceinline__ Pack8<T> row8(const T *row, unsigned c, unsigned n, bool vec) {
    Pack8<T> x;
    const T *s = row + c;
    if (vec && c + 8 <= n) {
#pragma unroll
        for (unsigned i = 0; i < sizeof(T) / 2; ++i) x.u[i] = reinterpret_cast<const uint4 *>(s)[i];
        return x;
    }
    if constexpr (sizeof(T) == 2) {
        if (!vec && c && c + 16 <= n) {  // the two aligned words that hold it lie within the row
            const unsigned by = (unsigned)(uintptr_t)s & 15u;
            const uint4 *a = reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(s) - by);
            x.u[0] = by ? shifted(a[0], a[1], by) : a[0];
            return x;
        }
    }
#pragma unroll
    for (unsigned j = 0; j < 8; ++j) x.v[j] = c + j < n ? s[j] : from_f32<T>(0.f);
    return x;
}
// The first of eight values that lie within the row, for a whole warp.  A 16-bit row that begins anywhere is written in 4-byte words:
// where it begins between two of them, a lane's last word takes the next lane's first value (`next`: that lane goes on with this
// row; `before`: the lane before this one does, and has written the first).
template <typename T> __device__ __forceinline__ void put8(T *row, unsigned c, unsigned n, bool vec, const Pack8<T> &x, bool has, bool next, bool before) {
    unsigned ahead = 0;
    if constexpr (sizeof(T) == 2) ahead = __shfl_down_sync(0xffffffffu, x.u[0].x, 1);
    if (!has) return;
    T *const o = row + c;
    if (vec && c + 8 <= n) {
#pragma unroll
        for (unsigned i = 0; i < sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(o)[i] = x.u[i];
        return;
    }
    if constexpr (sizeof(T) == 2) {
        if (c + 8 <= n) {
            const unsigned w[4] = {x.u[0].x, x.u[0].y, x.u[0].z, x.u[0].w};
            if (((uintptr_t)o & 2u) == 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j) reinterpret_cast<unsigned *>(o)[j] = w[j];
                return;
            }
#pragma unroll
            for (int j = 0; j < 3; ++j) reinterpret_cast<unsigned *>(o + 1)[j] = __funnelshift_r(w[j], w[j + 1], 16);
            if (next && c + 8 < n) *reinterpret_cast<unsigned *>(o + 7) = __funnelshift_r(w[3], ahead, 16);
            else o[7] = x.v[7];
            if (!before) o[0] = x.v[0];
            return;
        }
    }
#pragma unroll
    for (unsigned j = 0; j < 8; ++j)
        if (c + j < n) o[j] = x.v[j];
}

}  // namespace scar
