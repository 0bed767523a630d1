// The norms before and after a residual block with the block's gate and residual scale (scar_resnorm_* of scar.h):
//
//   u = f or N(f; w_post, b_post)      y = x + scale gate u      n = N(y; w_pre, b_pre)
//   N(v) = (v - mean) r w + b, r = 1 / sqrt(mean of (v - mean)^2 + eps)      (RMS: without mean and b)
//
// and the gradients.  A CTA holds a row in its registers, so x, f and the gate are read once and y and n written once; backward
// reads dy, dn, y, f and the gate once and forms the statistics again from them: storing them would save one of two reductions
// and cost the caller a tensor.  With g = dn w_pre, h = du w_post and hats for normalised rows:
//
//   dY = dy + r_y (g - mean g - y^ mean(g y^))          dx = dY           dw_pre = sum dn y^    db_pre = sum dn
//   du = scale gate dY    dgate = scale sum dY u        df = r_f (h - mean h - f^ mean(h f^))   dw_post = sum du f^   db_post = sum du
//
// The statistics of a row and the two sums over g come out of one reduction: a thread's count, mean and sum of squared deviations
// are merged pair by pair (Chan, Golub, LeVeque 1979), and so is its sum of g (y - its own mean).  No sum of squares is taken far
// from the mean, so rows whose mean is large beside their deviation keep theirs.
//
// Sums over rows: a CTA walks a run of rows and keeps its threads' columns in registers; k_resnorm_join adds the CTAs' sums in
// order.  Gates shared by several rows end inside a CTA's run, or reach over its ends: those leave partial sums too.
#include <algorithm>
#include <initializer_list>
#include <new>
#include <type_traits>

#include "train_common.cuh"

using namespace scar;

namespace {

constexpr unsigned kMostThreads = 512;

template <typename T> struct NormArgs {
    unsigned rows, dim;
    float scale, eps;
    int post, pre;
    const T *gate;
    unsigned long long gate_pitch;
    unsigned per_gate;
    const T *w_post, *b_post, *w_pre, *b_pre;
    const T *x, *f;  // backward: x is dy (may be nullptr)
    unsigned long long x_pitch, f_pitch;
    T *y, *n;        // backward: y is read, n is dx
    unsigned long long y_pitch, n_pitch;
    // backward
    const T *dn;
    T *df, *dgate;
    unsigned long long dn_pitch, df_pitch, dgate_pitch;
    unsigned per_cta;            // rows
    float *part;                 // [4][CTAs][dim]: dw_pre, dw_post, db_pre, db_post
    float *part_gate;            // [CTAs][2][dim]: of a gate that began before the CTA's rows, of one that ends behind them
    T *dw_post, *db_post, *dw_pre, *db_pre;
};

// A thread's values of one row.  Rows on 16-byte boundaries: groups of eight neighbours, a group per thread and round.  Rows
// anywhere: single values, neighbouring threads next to one another, so that a warp's access is one run of memory.
template <typename T, int NC> union Row {
    uint4 u[NC * sizeof(T) / 2];
    T v[8 * NC];
};
template <bool VEC> __device__ __forceinline__ unsigned col_of(int i) {
    return VEC ? (i / 8 * blockDim.x + threadIdx.x) * 8 + i % 8 : i * blockDim.x + threadIdx.x;
}
template <bool VEC, typename T, int NC> __device__ __forceinline__ void load_row(Row<T, NC> &r, const T *p, unsigned dim) {
    if (VEC) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const unsigned col = col_of<true>(c * 8);
            if (col + 8 <= dim) {
#pragma unroll
                for (unsigned k = 0; k < sizeof(T) / 2; ++k) r.u[c * (sizeof(T) / 2) + k] = reinterpret_cast<const uint4 *>(p + col)[k];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) r.v[c * 8 + j] = col + j < dim ? p[col + j] : from_f32<T>(0.f);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8 * NC; ++i) {
            const unsigned col = col_of<false>(i);
            r.v[i] = col < dim ? p[col] : from_f32<T>(0.f);
        }
    }
}
template <bool VEC, typename T, int NC> __device__ __forceinline__ void store_row(T *p, const Row<T, NC> &r, unsigned dim) {
    if (VEC) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const unsigned col = col_of<true>(c * 8);
            if (col + 8 <= dim) {
#pragma unroll
                for (unsigned k = 0; k < sizeof(T) / 2; ++k) reinterpret_cast<uint4 *>(p + col)[k] = r.u[c * (sizeof(T) / 2) + k];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (col + j < dim) p[col + j] = r.v[c * 8 + j];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8 * NC; ++i) {
            const unsigned col = col_of<false>(i);
            if (col < dim) p[col] = r.v[i];
        }
    }
}

// What is known of some values of a row: how many, their mean, their squared deviations from it (RMS: their squares), and for
// backward the sums of g and of g times the deviation (RMS: of g times the value).
struct Stat {
    float n, mean, m2, g, gv;
};
template <bool LAYER, bool GRAD> __device__ __forceinline__ Stat merge(const Stat &a, const Stat &b) {
    Stat s;
    if (!LAYER) {
        s.n = s.mean = s.g = 0.f;
        s.m2 = a.m2 + b.m2;
        s.gv = GRAD ? a.gv + b.gv : 0.f;
        return s;
    }
    s.n = a.n + b.n;
    const float inv = s.n > 0.f ? __frcp_rn(s.n) : 0.f, d = a.mean - b.mean;
    s.mean = (a.n * a.mean + b.n * b.mean) * inv;
    s.m2 = (a.m2 + b.m2) + d * d * (a.n * b.n * inv);
    s.g = GRAD ? a.g + b.g : 0.f;
    // a's deviations are from a's mean: from the common one they are larger by a.mean - s.mean = d b.n / n
    s.gv = GRAD ? (a.gv + b.gv) + (a.g * (d * (b.n * inv)) - b.g * (d * (a.n * inv))) : 0.f;
    return s;
}
template <bool LAYER, bool GRAD> __device__ __forceinline__ Stat other(const Stat &a, int o) {
    Stat s{0.f, 0.f, 0.f, 0.f, 0.f};
    s.m2 = __shfl_xor_sync(0xffffffffu, a.m2, o);
    if (LAYER) {
        s.n = __shfl_xor_sync(0xffffffffu, a.n, o);
        s.mean = __shfl_xor_sync(0xffffffffu, a.mean, o);
    }
    if (GRAD) s.gv = __shfl_xor_sync(0xffffffffu, a.gv, o);
    if (GRAD && LAYER) s.g = __shfl_xor_sync(0xffffffffu, a.g, o);
    return s;
}
// Of N sets over the CTA, the same bits in every thread (merging is symmetric).  `sh` holds two halves of 32 * N that alternate
// from one reduction to the next: a half is written again only behind the barrier of the reduction between.
template <bool LAYER, bool GRAD, int N> __device__ __forceinline__ void cta_stats(Stat (&s)[N], Stat *sh, unsigned &half) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] = merge<LAYER, GRAD>(s[k], other<LAYER, GRAD>(s[k], o));
    }
    if (blockDim.x == 32) return;
    Stat *at = sh + half * 32 * N;
    half ^= 1;
    const unsigned warps = blockDim.x / 32, lane = threadIdx.x & 31;
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) at[k * 32 + threadIdx.x / 32] = s[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = lane < warps ? at[k * 32 + lane] : Stat{0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int o = 16; o; o >>= 1) {  // of 16 warps at most: the first step adds nothing
        if (o >= (int)warps) continue;
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] = merge<LAYER, GRAD>(s[k], other<LAYER, GRAD>(s[k], o));
    }
    // lanes beyond the largest power of two that holds the warps have merged nothing but zeros
#pragma unroll
    for (int k = 0; k < N; ++k) {
        s[k].n = __shfl_sync(0xffffffffu, s[k].n, 0);
        s[k].mean = __shfl_sync(0xffffffffu, s[k].mean, 0);
        s[k].m2 = __shfl_sync(0xffffffffu, s[k].m2, 0);
        s[k].g = __shfl_sync(0xffffffffu, s[k].g, 0);
        s[k].gv = __shfl_sync(0xffffffffu, s[k].gv, 0);
    }
}

// A thread's own values.
template <bool LAYER, bool VEC, int N> __device__ __forceinline__ Stat stat_of(const float (&v)[N], unsigned dim) {
    Stat s{0.f, 0.f, 0.f, 0.f, 0.f};
    if (!LAYER) {
#pragma unroll
        for (int i = 0; i < N; ++i) s.m2 = fmaf(v[i], v[i], s.m2);
        return s;
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {  // what lies behind the row is zero
        s.n += col_of<VEC>(i) < dim ? 1.f : 0.f;
        sum += v[i];
    }
    s.mean = s.n > 0.f ? sum / s.n : 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = col_of<VEC>(i) < dim ? v[i] - s.mean : 0.f;
        s.m2 = fmaf(d, d, s.m2);
    }
    return s;
}
__device__ __forceinline__ float deviation_inv(const Stat &s, float dim, float eps) { return rsqrtf(s.m2 / dim + eps); }

template <typename T, bool LAYER, bool VEC, int NC>
__global__ void __launch_bounds__(kMostThreads) k_resnorm_forward(const __grid_constant__ NormArgs<T> g) {
    constexpr int N = 8 * NC;
    __shared__ Stat sh[64];
    unsigned half = 0;
    for (unsigned row = blockIdx.x; row < g.rows; row += gridDim.x) {
        Row<T, NC> rx, rf, rg, out;
        load_row<VEC>(rx, g.x + row * g.x_pitch, g.dim);
        float y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = to_f32(rx.v[i]);
        if (g.f) {
            load_row<VEC>(rf, g.f + row * g.f_pitch, g.dim);
            if (g.gate) load_row<VEC>(rg, g.gate + row / g.per_gate * g.gate_pitch, g.dim);
            float u[N];
#pragma unroll
            for (int i = 0; i < N; ++i) u[i] = to_f32(rf.v[i]);
            if (g.post) {
                Row<T, NC> w, b;
                if (g.w_post) load_row<VEC>(w, g.w_post, g.dim);
                if (LAYER && g.b_post) load_row<VEC>(b, g.b_post, g.dim);
                Stat s[1] = {stat_of<LAYER, VEC>(u, g.dim)};
                cta_stats<LAYER, false>(s, sh, half);
                const float r = deviation_inv(s[0], (float)g.dim, g.eps);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    u[i] = (u[i] - (LAYER ? s[0].mean : 0.f)) * r;
                    if (g.w_post) u[i] *= to_f32(w.v[i]);
                    if (LAYER && g.b_post) u[i] += to_f32(b.v[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = fmaf(g.gate ? g.scale * to_f32(rg.v[i]) : g.scale, u[i], y[i]);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            out.v[i] = from_f32<T>(y[i]);
            y[i] = to_f32(out.v[i]);  // the norm is that of the values handed on: backward has them and nothing else
        }
        if (g.y) store_row<VEC>(g.y + row * g.y_pitch, out, g.dim);
        if (!g.pre) continue;
        Row<T, NC> w, b;
        if (g.w_pre) load_row<VEC>(w, g.w_pre, g.dim);
        if (LAYER && g.b_pre) load_row<VEC>(b, g.b_pre, g.dim);
        if (LAYER) {
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = col_of<VEC>(i) < g.dim ? y[i] : 0.f;  // b_post stands nowhere behind the row
        }
        Stat s[1] = {stat_of<LAYER, VEC>(y, g.dim)};
        cta_stats<LAYER, false>(s, sh, half);
        const float r = deviation_inv(s[0], (float)g.dim, g.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float v = (y[i] - (LAYER ? s[0].mean : 0.f)) * r;
            if (g.w_pre) v *= to_f32(w.v[i]);
            if (LAYER && g.b_pre) v += to_f32(b.v[i]);
            out.v[i] = from_f32<T>(v);
        }
        store_row<VEC>(g.n + row * g.n_pitch, out, g.dim);
    }
}

// Two plain sums over the CTA.
__device__ __forceinline__ float2 cta_sums(float2 v, float2 *sh, unsigned &half) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if (blockDim.x == 32) return v;
    float2 *at = sh + half * 32;
    half ^= 1;
    const unsigned warps = blockDim.x / 32, lane = threadIdx.x & 31;
    if (lane == 0) at[threadIdx.x / 32] = v;
    __syncthreads();
    v = lane < warps ? at[lane] : make_float2(0.f, 0.f);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    return v;
}

template <bool VEC, int N> __device__ __forceinline__ void put_part(float *p, const float (&v)[N], unsigned dim) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (col_of<VEC>(i) < dim) p[col_of<VEC>(i)] = v[i];
}

template <typename T, bool LAYER, bool VEC, int NC>
__global__ void __launch_bounds__(kMostThreads, 1) k_resnorm_backward(const __grid_constant__ NormArgs<T> g) {
    constexpr int N = 8 * NC;
    __shared__ Stat sh[128];
    __shared__ float2 sh2[64];
    unsigned half = 0, half2 = 0;
    const unsigned r0 = blockIdx.x * g.per_cta, r1 = min(g.rows, r0 + g.per_cta);
    const float dim = (float)g.dim, inv_dim = 1.f / dim;
    const bool shared_gate = g.dgate && g.per_gate > 1;
    float a_wpre[N] = {}, a_wpost[N] = {}, a_bpre[LAYER ? N : 1] = {}, a_bpost[LAYER ? N : 1] = {}, a_gate[N] = {};
    Row<T, NC> w_pre, w_post, b_post;
    if (g.pre && g.w_pre) load_row<VEC>(w_pre, g.w_pre, g.dim);
    if (g.post && g.w_post) load_row<VEC>(w_post, g.w_post, g.dim);
    if (LAYER && g.post && g.b_post) load_row<VEC>(b_post, g.b_post, g.dim);
    for (unsigned row = r0; row < r1; ++row) {
        Row<T, NC> rdy, rdn, ry, rf, rg, out;
        if (g.x) load_row<VEC>(rdy, g.x + row * g.x_pitch, g.dim);
        if (g.pre) {
            load_row<VEC>(rdn, g.dn + row * g.dn_pitch, g.dim);
            load_row<VEC>(ry, static_cast<const T *>(g.y) + row * g.y_pitch, g.dim);
        }
        if (g.f) {
            load_row<VEC>(rf, g.f + row * g.f_pitch, g.dim);
            if (g.gate) load_row<VEC>(rg, g.gate + row / g.per_gate * g.gate_pitch, g.dim);
        }
        Stat s[2] = {{0.f, 0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f, 0.f}};
        if (g.pre) {
            float y[N];
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = to_f32(ry.v[i]);
            s[0] = stat_of<LAYER, VEC>(y, g.dim);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float q = to_f32(rdn.v[i]) * (g.w_pre ? to_f32(w_pre.v[i]) : 1.f);
                if (LAYER) s[0].g += q;
                s[0].gv = fmaf(q, y[i] - (LAYER ? s[0].mean : 0.f), s[0].gv);
            }
        }
        if (g.f && g.post) {
            float f[N];
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = to_f32(rf.v[i]);
            s[1] = stat_of<LAYER, VEC>(f, g.dim);
        }
        if (g.pre || (g.f && g.post)) cta_stats<LAYER, true>(s, sh, half);
        float d[N];  // dY
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] = g.x ? to_f32(rdy.v[i]) : 0.f;
        if (g.pre) {
            const float r = deviation_inv(s[0], dim, g.eps), mg = LAYER ? s[0].g * inv_dim : 0.f, mgy = s[0].gv * r * inv_dim;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float dn = to_f32(rdn.v[i]), hat = (to_f32(ry.v[i]) - (LAYER ? s[0].mean : 0.f)) * r;
                d[i] += r * (dn * (g.w_pre ? to_f32(w_pre.v[i]) : 1.f) - mg - hat * mgy);
                if (LAYER && col_of<VEC>(i) >= g.dim) d[i] = 0.f;
                a_wpre[i] = fmaf(dn, hat, a_wpre[i]);
                if (LAYER) a_bpre[i] += dn;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) out.v[i] = from_f32<T>(d[i]);
        if (g.n) store_row<VEC>(g.n + row * g.n_pitch, out, g.dim);
        if (!g.f) continue;
        float hat[N];  // f, normalised where there is a norm
        const float r = g.post ? deviation_inv(s[1], dim, g.eps) : 1.f, m = g.post && LAYER ? s[1].mean : 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) hat[i] = (to_f32(rf.v[i]) - m) * r;
        if (g.dgate) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float u = hat[i];
                if (g.post && g.w_post) u *= to_f32(w_post.v[i]);
                if (LAYER && g.post && g.b_post) u += to_f32(b_post.v[i]);
                const float e = g.scale * d[i] * u;
                if (shared_gate) a_gate[i] += e;
                else out.v[i] = from_f32<T>(e);
            }
            const unsigned gate = row / g.per_gate;
            if (!shared_gate) {
                store_row<VEC>(g.dgate + row * g.dgate_pitch, out, g.dim);
            } else if (row + 1 == r1 || row + 1 == (gate + 1) * g.per_gate) {
                const unsigned first = gate * g.per_gate, end = g.rows - first > g.per_gate ? first + g.per_gate : g.rows;
                if (first >= r0 && end <= r1) {
#pragma unroll
                    for (int i = 0; i < N; ++i) out.v[i] = from_f32<T>(a_gate[i]);
                    store_row<VEC>(g.dgate + gate * g.dgate_pitch, out, g.dim);
                } else {
                    put_part<VEC>(g.part_gate + (blockIdx.x * 2ull + (first < r0 ? 0 : 1)) * g.dim, a_gate, g.dim);
                }
#pragma unroll
                for (int i = 0; i < N; ++i) a_gate[i] = 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] *= g.gate ? g.scale * to_f32(rg.v[i]) : g.scale;  // du
        if (g.post) {
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                a_wpost[i] = fmaf(d[i], hat[i], a_wpost[i]);
                if (LAYER) a_bpost[i] += d[i];
                if (g.w_post) d[i] *= to_f32(w_post.v[i]);
                // behind the row d is zero, and hat may not be
                if (LAYER) sum.x += d[i];
                sum.y = fmaf(d[i], hat[i], sum.y);
            }
            sum = cta_sums(sum, sh2, half2);
            const float mh = LAYER ? sum.x * inv_dim : 0.f, mhf = sum.y * inv_dim;
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = r * (d[i] - mh - hat[i] * mhf);
        }
        if (g.df) {
#pragma unroll
            for (int i = 0; i < N; ++i) out.v[i] = from_f32<T>(d[i]);
            store_row<VEC>(g.df + row * g.df_pitch, out, g.dim);
        }
    }
    const unsigned long long each = (unsigned long long)gridDim.x * g.dim, mine = (unsigned long long)blockIdx.x * g.dim;
    if (g.dw_pre) put_part<VEC>(g.part + mine, a_wpre, g.dim);
    if (g.dw_post) put_part<VEC>(g.part + each + mine, a_wpost, g.dim);
    if constexpr (LAYER) {
        if (g.db_pre) put_part<VEC>(g.part + 2 * each + mine, a_bpre, g.dim);
        if (g.db_post) put_part<VEC>(g.part + 3 * each + mine, a_bpost, g.dim);
    }
}

// Adds the CTAs' sums, 32 columns a CTA, 32 walkers over the rows of the list, in an order that depends on the sizes alone.
// blockIdx.y 0 .. 3: the vectors; 4 + c: the gate that the last row of CTA c has, where it begins in c and ends behind it.
template <typename T> __global__ void __launch_bounds__(1024) k_resnorm_join(const __grid_constant__ NormArgs<T> g, unsigned ctas) {
    __shared__ float sh[32][33];
    const unsigned col = blockIdx.x * 32 + (threadIdx.x & 31), walker = threadIdx.x >> 5;
    T *out;
    const float *from;
    unsigned long long step = g.dim;
    unsigned n = ctas;
    if (blockIdx.y < 4) {
        T *const to[4] = {g.dw_pre, g.dw_post, g.db_pre, g.db_post};
        out = to[blockIdx.y];
        from = g.part + blockIdx.y * (unsigned long long)ctas * g.dim;
        if (!out) return;
    } else {
        const unsigned c = blockIdx.y - 4, r0 = c * g.per_cta, r1 = min(g.rows, r0 + g.per_cta);
        const unsigned gate = (r1 - 1) / g.per_gate, first = gate * g.per_gate;
        const unsigned end = g.rows - first > g.per_gate ? first + g.per_gate : g.rows;
        if (first < r0 || end <= r1) return;
        out = g.dgate + gate * g.dgate_pitch;
        n = (end - 1) / g.per_cta - c + 1;
        from = g.part_gate + c * 2ull * g.dim;  // the first of its parts is the CTA's second, the others' their first
        step = 2ull * g.dim;
    }
    float v = 0.f;
    if (col < g.dim)
        for (unsigned k = walker; k < n; k += 32) v += from[k * step + (blockIdx.y >= 4 && k == 0 ? g.dim : 0u) + col];
    sh[walker][threadIdx.x & 31] = v;
    __syncthreads();
    if (walker == 0 && col < g.dim) {
        v = 0.f;
#pragma unroll
        for (int k = 0; k < 32; ++k) v += sh[k][threadIdx.x];
        out[col] = from_f32<T>(v);
    }
}

}  // namespace

struct scar_resnorm {
    int device = 0;
    cudaStream_t stream = nullptr;
    scar_resnorm_config cfg{};
    unsigned sms = 148, threads = 32, rounds = 1;  // threads of a row's CTA, groups of eight values each has
    unsigned back_ctas = 1;                        // most CTAs of backward
    float *part = nullptr;
    uint64_t launches = 0;
};

namespace {

// f(std::integral_constant<int, NC>) for the operator's rounds.
template <typename F> void with_rounds(unsigned rounds, F &&f) {
    if (rounds == 1) f(std::integral_constant<int, 1>());
    else if (rounds == 2) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 4>());
}

template <typename T> bool aligned16(const T *p, uint64_t pitch = 0) { return (uintptr_t)p % 16 == 0 && pitch * sizeof(T) % 16 == 0; }

template <typename T> void run_forward(scar_resnorm *op, const NormArgs<T> &g) {
    const bool vec = aligned16(g.x, g.x_pitch) && aligned16(g.f, g.f_pitch) && aligned16(g.y, g.y_pitch) && aligned16(g.n, g.n_pitch) &&
                     aligned16(g.gate, g.gate_pitch) && aligned16(g.w_post) && aligned16(g.b_post) && aligned16(g.w_pre) && aligned16(g.b_pre);
    const bool layer = op->cfg.kind == SCAR_RESNORM_LAYER;
    const unsigned ctas = std::min(g.rows, op->sms * std::max(1u, 2048 / op->threads));
    with_rounds(op->rounds, [&](auto nc) {
        constexpr int NC = decltype(nc)::value;
        auto kernel = layer ? (vec ? k_resnorm_forward<T, true, true, NC> : k_resnorm_forward<T, true, false, NC>)
                            : (vec ? k_resnorm_forward<T, false, true, NC> : k_resnorm_forward<T, false, false, NC>);
        kernel<<<ctas, op->threads, 0, op->stream>>>(g);
    });
    op->launches++;
}

template <typename T> void run_backward(scar_resnorm *op, NormArgs<T> g) {
    const bool vec = aligned16(g.x, g.x_pitch) && aligned16(g.f, g.f_pitch) && aligned16(g.y, g.y_pitch) && aligned16(g.n, g.n_pitch) &&
                     aligned16(g.dn, g.dn_pitch) && aligned16(g.df, g.df_pitch) && aligned16(g.dgate, g.dgate_pitch) &&
                     aligned16(g.gate, g.gate_pitch) && aligned16(g.w_post) && aligned16(g.b_post) && aligned16(g.w_pre);
    const bool layer = op->cfg.kind == SCAR_RESNORM_LAYER;
    unsigned ctas = 0;
    if (g.rows) {
        ctas = std::min(g.rows, op->back_ctas);
        g.per_cta = (g.rows + ctas - 1) / ctas;
        ctas = (g.rows + g.per_cta - 1) / g.per_cta;
        g.part = op->part;
        g.part_gate = op->part + 4ull * op->back_ctas * g.dim;
        with_rounds(op->rounds, [&](auto nc) {
            constexpr int NC = decltype(nc)::value;
            auto kernel = layer ? (vec ? k_resnorm_backward<T, true, true, NC> : k_resnorm_backward<T, true, false, NC>)
                                : (vec ? k_resnorm_backward<T, false, true, NC> : k_resnorm_backward<T, false, false, NC>);
            kernel<<<ctas, op->threads, 0, op->stream>>>(g);
        });
        op->launches++;
    }
    const bool gates = g.dgate && g.per_gate > 1 && ctas > 1;
    if (!g.dw_pre && !g.dw_post && !g.db_pre && !g.db_post && !gates) return;
    k_resnorm_join<T><<<dim3((g.dim + 31) / 32, 4 + (gates ? ctas : 0)), 1024, 0, op->stream>>>(g, ctas);
    op->launches++;
}

constexpr uint64_t kFar = 1ull << 40;  // elements of a pitch: rows times pitch stays below 2^63 bytes

struct Matrix {
    const void *p;
    uint64_t pitch, rows;
    bool wanted;  // a nullptr is an error
};
int check_matrices(const scar_resnorm *op, std::initializer_list<Matrix> all) {
    const unsigned b = elem_size(op->cfg.dtype);
    for (const Matrix &m : all) {
        if (!m.p && m.wanted) return SCAR_ERR_INVALID_ARG;
        if (m.p && ((uintptr_t)m.p % b || m.pitch >= kFar || (m.rows > 1 && m.pitch < op->cfg.dim))) return SCAR_ERR_INVALID_ARG;
    }
    return SCAR_OK;
}
int check_block(const scar_resnorm *op, const scar_resnorm_block *k, const void *f, uint64_t rows) {
    if (!op || !k) return SCAR_ERR_INVALID_ARG;
    if (rows > op->cfg.max_rows) return SCAR_ERR_CAPACITY;
    const unsigned b = elem_size(op->cfg.dtype);
    for (const void *p : {k->d_w_post, k->d_b_post, k->d_w_pre, k->d_b_pre})
        if ((uintptr_t)p % b) return SCAR_ERR_INVALID_ARG;
    if (op->cfg.kind == SCAR_RESNORM_RMS && (k->d_b_post || k->d_b_pre)) return SCAR_ERR_INVALID_ARG;
    if (rows && !f && (k->post || k->d_gate)) return SCAR_ERR_INVALID_ARG;
    if (k->d_gate && !k->rows_per_gate) return SCAR_ERR_INVALID_ARG;
    return check_current_device(op->device);
}
template <typename T> NormArgs<T> block_args(const scar_resnorm *op, const scar_resnorm_block *k, uint64_t rows) {
    NormArgs<T> g{};
    g.rows = (unsigned)rows;
    g.dim = (unsigned)op->cfg.dim;
    g.scale = k->scale;
    g.eps = (float)op->cfg.eps;
    g.post = k->post != 0;
    g.pre = k->pre != 0;
    g.gate = static_cast<const T *>(k->d_gate);
    g.gate_pitch = k->gate_pitch;
    g.per_gate = (unsigned)std::min<uint64_t>(std::max<uint64_t>(k->rows_per_gate, 1), std::max<uint64_t>(rows, 1));
    g.w_post = k->post ? static_cast<const T *>(k->d_w_post) : nullptr;
    g.b_post = k->post ? static_cast<const T *>(k->d_b_post) : nullptr;
    g.w_pre = k->pre ? static_cast<const T *>(k->d_w_pre) : nullptr;
    g.b_pre = k->pre ? static_cast<const T *>(k->d_b_pre) : nullptr;
    return g;
}
uint64_t gates_of(const scar_resnorm_block *k, uint64_t rows) { return k->rows_per_gate ? (rows + k->rows_per_gate - 1) / k->rows_per_gate : 0; }

int done(scar_resnorm *) {
    TRAIN_TRY(cudaGetLastError());
    return SCAR_OK;
}

}  // namespace

extern "C" {

int scar_resnorm_init(scar_resnorm **out, const scar_resnorm_config *cfg, void *cuda_stream) {
    if (!out) return SCAR_ERR_INVALID_ARG;
    *out = nullptr;
    if (!cfg || !is_operand_type(cfg->dtype) || (cfg->kind != SCAR_RESNORM_RMS && cfg->kind != SCAR_RESNORM_LAYER) || !cfg->dim ||
        cfg->max_rows >= 1ull << 31 || !(cfg->eps >= 0. && cfg->eps < 1e30))
        return SCAR_ERR_INVALID_ARG;
    if (cfg->dim > SCAR_RESNORM_MAX_DIM) return SCAR_ERR_CAPACITY;
    scar_resnorm *op = new (std::nothrow) scar_resnorm();
    if (!op) return SCAR_ERR_ALLOC;
    op->cfg = *cfg;
    op->stream = static_cast<cudaStream_t>(cuda_stream);
    auto setup = [&]() -> int {
        TRAIN_TRY(cudaGetDevice(&op->device));
        int sms = 0;
        TRAIN_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, op->device));
        op->sms = std::max(1, sms);
        const unsigned groups = (unsigned)((cfg->dim + 7) / 8);
        op->rounds = groups <= kMostThreads ? 1 : groups <= 2 * kMostThreads ? 2 : 4;
        op->threads = (unsigned)round_up((groups + op->rounds - 1) / op->rounds, 32);
        // CTAs of backward: as many as run at a time (128 registers a thread), and eight rows each where there are many
        op->back_ctas = (unsigned)std::max<uint64_t>(1, std::min<uint64_t>((uint64_t)op->sms * std::max(1u, 512 / op->threads), cfg->max_rows));
        if (!cfg->forward_only) {
            if (cudaMalloc(&op->part, 6ull * op->back_ctas * cfg->dim * sizeof(float)) != cudaSuccess) {
                cudaGetLastError();
                return SCAR_ERR_ALLOC;
            }
        }
        TRAIN_TRY(cudaStreamSynchronize(op->stream));
        return SCAR_OK;
    };
    const int rc = setup();
    if (rc != SCAR_OK) {
        scar_resnorm_destroy(op);
        return rc;
    }
    *out = op;
    return SCAR_OK;
}

int scar_resnorm_forward(scar_resnorm *op, const scar_resnorm_block *block, const void *d_x, uint64_t x_pitch, const void *d_f, uint64_t f_pitch,
                         uint64_t n_rows, void *d_y, uint64_t y_pitch, void *d_n, uint64_t n_pitch) {
    int rc = check_block(op, block, d_f, n_rows);
    if (rc != SCAR_OK) return rc;
    const bool any = n_rows != 0;
    rc = check_matrices(op, {{d_x, x_pitch, n_rows, any}, {d_f, f_pitch, n_rows, false}, {d_y, y_pitch, n_rows, any && d_f != nullptr},
                             {d_n, n_pitch, n_rows, any && block->pre}, {block->d_gate, block->gate_pitch, gates_of(block, n_rows), false}});
    if (rc != SCAR_OK) return rc;
    if (!any) return SCAR_OK;
    dispatch_operand(op->cfg.dtype, [&](auto e) {
        using T = decltype(e);
        NormArgs<T> g = block_args<T>(op, block, n_rows);
        g.x = static_cast<const T *>(d_x); g.x_pitch = x_pitch;
        g.f = static_cast<const T *>(d_f); g.f_pitch = f_pitch;
        g.y = static_cast<T *>(d_y); g.y_pitch = y_pitch;
        g.n = block->pre ? static_cast<T *>(d_n) : nullptr; g.n_pitch = n_pitch;
        run_forward(op, g);
    });
    return done(op);
}

int scar_resnorm_backward(scar_resnorm *op, const scar_resnorm_block *block, const void *d_dy, uint64_t dy_pitch, const void *d_dn, uint64_t dn_pitch,
                          const void *d_y, uint64_t y_pitch, const void *d_f, uint64_t f_pitch, uint64_t n_rows, void *d_dx, uint64_t dx_pitch,
                          void *d_df, uint64_t df_pitch, void *d_dgate, uint64_t dgate_pitch, void *d_dw_post, void *d_db_post, void *d_dw_pre,
                          void *d_db_pre) {
    int rc = check_block(op, block, d_f, n_rows);
    if (rc != SCAR_OK) return rc;
    if (op->cfg.forward_only) return SCAR_ERR_STATE;
    const bool any = n_rows != 0, layer = op->cfg.kind == SCAR_RESNORM_LAYER;
    // a gradient without the input that it is of
    if ((d_dgate && !block->d_gate) || (d_df && !d_f) || ((d_dw_post || d_db_post) && !block->post) || ((d_dw_pre || d_db_pre) && !block->pre) ||
        ((d_db_post || d_db_pre) && !layer))
        return SCAR_ERR_INVALID_ARG;
    rc = check_matrices(op, {{d_dy, dy_pitch, n_rows, any && !block->pre}, {d_dn, dn_pitch, n_rows, any && block->pre}, {d_y, y_pitch, n_rows, any && block->pre},
                             {d_f, f_pitch, n_rows, false}, {d_dx, dx_pitch, n_rows, false}, {d_df, df_pitch, n_rows, false},
                             {block->d_gate, block->gate_pitch, gates_of(block, n_rows), false}, {d_dgate, dgate_pitch, gates_of(block, n_rows), false},
                             {d_dw_post, 0, 1, false}, {d_db_post, 0, 1, false}, {d_dw_pre, 0, 1, false}, {d_db_pre, 0, 1, false}});
    if (rc != SCAR_OK) return rc;
    dispatch_operand(op->cfg.dtype, [&](auto e) {
        using T = decltype(e);
        NormArgs<T> g = block_args<T>(op, block, n_rows);
        g.x = static_cast<const T *>(d_dy); g.x_pitch = dy_pitch;
        g.dn = static_cast<const T *>(d_dn); g.dn_pitch = dn_pitch;
        g.y = const_cast<T *>(static_cast<const T *>(d_y)); g.y_pitch = y_pitch;
        g.f = static_cast<const T *>(d_f); g.f_pitch = f_pitch;
        g.n = static_cast<T *>(d_dx); g.n_pitch = dx_pitch;
        g.df = static_cast<T *>(d_df); g.df_pitch = df_pitch;
        g.dgate = static_cast<T *>(d_dgate); g.dgate_pitch = dgate_pitch;
        g.dw_post = static_cast<T *>(d_dw_post);
        g.db_post = static_cast<T *>(d_db_post);
        g.dw_pre = static_cast<T *>(d_dw_pre);
        g.db_pre = static_cast<T *>(d_db_pre);
        run_backward(op, g);
    });
    return done(op);
}

uint64_t scar_resnorm_launch_count(const scar_resnorm *op) { return op ? op->launches : 0; }

int scar_resnorm_destroy(scar_resnorm *op) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    const bool ok = cudaStreamSynchronize(op->stream) == cudaSuccess;
    if (op->part) cudaFree(op->part);
    delete op;
    if (!ok) cudaGetLastError();
    return ok ? SCAR_OK : SCAR_ERR_CUDA;
}

}  // extern "C"
