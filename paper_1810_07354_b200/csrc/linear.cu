// A hidden layer (scar_linear_* of scar.h): y = residual + m . act(x w^T + b) with its gradients.
//
//   forward    the product's epilogue adds the bias, applies the activation, the mask (computed, mask.cuh) and the residual, and
//              leaves the activation's derivative for backward; where the product's sum is split, and in float32, k_linear_join
//              does the same from the float32 sums
//   backward   k_linear_dz: dz = m . dy . slope, rounded to the operands' type (float32: three bfloat16 planes), and its sums
//              over the rows; dx = dz w and dw = dz^T x in one launch (k_tc_gemm)
//
// The derivative and not z is kept: it lies in [-0.13, 1.13], so float16 holds it to 2^-11 of itself whatever the operands'
// type, and backward needs no activation.  Computing z again instead would be 8 rather than 6 T K N operations.
#include <algorithm>
#include <new>
#include <vector>

#include "tc_host.cuh"

using namespace scar;

namespace {

// Two matrices of d columns copied to the layout the products read: x and w, each where it has rows.
template <typename T>
__global__ void __launch_bounds__(256) k_linear_place(Copy<T> a, Copy<T> b, unsigned d, unsigned dp) {
    griddep_start();
    const unsigned groups = dp / 8;
    const unsigned long long na = (unsigned long long)a.n * groups, total = na + (unsigned long long)b.n * groups;
    for (unsigned long long i = (unsigned long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (unsigned long long)gridDim.x * 256) {
        const bool second = i >= na;
        const unsigned long long k = second ? i - na : i;
        const unsigned r = total >> 32 ? (unsigned)(k / groups) : (unsigned)k / groups;
        copy_eight(second ? b : a, r, r, (unsigned)(k - (unsigned long long)r * groups) * 8, d, dp);
    }
}

template <typename T> union Pack8 {
    uint4 u[sizeof(T) / 2];
    T v[8];
};
// Eight values from column c of a row of n that begins anywhere, zeros behind the last one.
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
// The first of eight values that lie within the row.
template <typename T> __device__ __forceinline__ void put8(T *row, unsigned c, unsigned n, bool vec, const Pack8<T> &x) {
    if (vec && c + 8 <= n) {
#pragma unroll
        for (unsigned i = 0; i < sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(row + c)[i] = x.u[i];
        return;
    }
#pragma unroll
    for (unsigned j = 0; j < 8; ++j)
        if (c + j < n) row[c + j] = x.v[j];
}

// The parts of a product whose sum was split (or its float32 result) to the layer's output: what epi_layer does without a split.
template <typename T, int ACT>
__global__ void __launch_bounds__(128) k_linear_join(const __grid_constant__ TcArgs g) {
    griddep_start();
    const LayerArgs &l = g.layer;
    const unsigned m = rows_of(g), pitch = (g.n + 7) & ~7u, groups = pitch / 8, splits = parts_of(g);
    const unsigned long long stride = (unsigned long long)g.m * pitch, total = (unsigned long long)m * groups;
    const unsigned long long offset = l.drop.on ? l.drop.at() : 0ull;
    for (unsigned long long i = (unsigned long long)blockIdx.x * 128 + threadIdx.x; i < total; i += (unsigned long long)gridDim.x * 128) {
        const unsigned row = total >> 32 ? (unsigned)(i / groups) : (unsigned)i / groups;
        const unsigned col = (unsigned)(i - (unsigned long long)row * groups) * 8;
        const float *p = g.part + (unsigned long long)row * pitch + col;
        float2 z[4] = {}, slope[4];
#pragma unroll 2
        for (unsigned s = 0; s < splits; ++s) {
            const float4 a = *reinterpret_cast<const float4 *>(p + s * stride), b = *reinterpret_cast<const float4 *>(p + s * stride + 4);
            z[0] = add2(z[0], make_float2(a.x, a.y));
            z[1] = add2(z[1], make_float2(a.z, a.w));
            z[2] = add2(z[2], make_float2(b.x, b.y));
            z[3] = add2(z[3], make_float2(b.z, b.w));
        }
        Pack8<T> r;
        if (l.res) r = row8(static_cast<const T *>(l.res) + row * l.res_pitch, col, g.n, l.res_vec);
        layer8<ACT, T>(l, offset, row, col, g.n, z, slope);
        if (l.slope) {
            const unsigned long long at = (unsigned long long)row * pitch + col;
            if constexpr (sizeof(T) == 4) {
                float4 *o = reinterpret_cast<float4 *>(static_cast<float *>(l.slope) + at);
                o[0] = make_float4(slope[0].x, slope[0].y, slope[1].x, slope[1].y);
                o[1] = make_float4(slope[2].x, slope[2].y, slope[3].x, slope[3].y);
            } else {
                *reinterpret_cast<uint4 *>(static_cast<unsigned short *>(l.slope) + at) = pack8<__half>(slope);
            }
        }
        Pack8<T> y;
#pragma unroll
        for (int j = 0; j < 4; ++j) Two<T>::put(y.v + 2 * j, l.res ? add2(Two<T>::get(r.v + 2 * j), z[j]) : z[j]);
        put8(static_cast<T *>(g.out) + row * g.out_pitch, col, g.n, g.out_vec, y);
    }
}

// dz and its sums over the rows.  A CTA has 256 columns, eight per lane, and a run of rows, one per warp at a time.
template <typename T> struct DzArgs {
    const T *dy;
    unsigned long long dy_pitch;
    int vec;
    const void *slope;  // or nullptr: 1
    unsigned rows, n, np, per_cta;
    DropRule drop;
    unsigned short *dz;  // [planes][rows][np], or nullptr: dy is dz
    unsigned long long plane;
    float *part;         // [CTAs of a strip][np]
    T *dbias;            // or nullptr
    unsigned *left;      // per strip: CTAs that are through
};
constexpr int kDzRows = 4;  // of a warp, under way together
template <typename T>
__global__ void __launch_bounds__(256) k_linear_dz(const __grid_constant__ DzArgs<T> g) {
    __shared__ float sums[8][256];
    __shared__ bool last;
    griddep_start();
    const unsigned lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 256 + lane * 8;
    const unsigned r1 = min(g.rows, (blockIdx.y + 1) * g.per_cta);
    const unsigned long long offset = g.drop.on ? g.drop.at() : 0ull;
    using S = typename std::conditional<sizeof(T) == 4, float, __half>::type;
    float2 sum[4] = {};
    if (col < g.n) {
        for (unsigned r0 = blockIdx.y * g.per_cta + warp; r0 < r1; r0 += 8 * kDzRows) {
            Pack8<T> d[kDzRows];
            Pack8<S> s[kDzRows];
#pragma unroll
            for (int k = 0; k < kDzRows; ++k) {
                const unsigned r = r0 + k * 8;
                if (r >= r1) continue;
                d[k] = row8(g.dy + r * g.dy_pitch, col, g.n, g.vec);
                if (g.slope) s[k] = row8(static_cast<const S *>(g.slope) + r * (unsigned long long)g.np, col, g.np, true);
            }
#pragma unroll
            for (int k = 0; k < kDzRows; ++k) {
                const unsigned r = r0 + k * 8;
                if (r >= r1) continue;
                float2 z[4];  // zeros behind the row: row8 fills up with them
#pragma unroll
                for (int j = 0; j < 4; ++j) z[j] = Two<T>::get(d[k].v + 2 * j);
                if (g.slope) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) z[j] = mul2(z[j], Two<S>::get(s[k].v + 2 * j));
                }
                if (g.drop.on) mask_apply(g.drop, mask_bits(g.drop, offset, r, col >> 3), z);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] = add2(sum[j], z[j]);
                if (!g.dz) continue;
                unsigned short *o = g.dz + r * (unsigned long long)g.np + col;
                if constexpr (sizeof(T) == 2) {
                    *reinterpret_cast<uint4 *>(o) = pack8<T>(z);
                } else {
                    Eight p[3];
#pragma unroll
                    for (int j = 0; j < 8; ++j) split3(j & 1 ? z[j / 2].y : z[j / 2].x, p[0].b[j], p[1].b[j], p[2].b[j]);
#pragma unroll
                    for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4 *>(o + q * g.plane) = p[q].u;
                }
            }
        }
    }
    if (!g.dbias) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<float2 *>(&sums[warp][lane * 8 + 2 * j]) = sum[j];
    __syncthreads();
    const unsigned c = blockIdx.x * 256 + threadIdx.x;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += sums[w][threadIdx.x];
    if (gridDim.y > 1) {  // the strip's last CTA adds what its CTAs have left, in order
        if (c < g.n) g.part[blockIdx.y * (unsigned long long)g.np + c] = v;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicInc(g.left + blockIdx.x, gridDim.y - 1) == gridDim.y - 1;
        __syncthreads();
        if (!last) return;
        __threadfence();
        v = 0.f;
        if (c < g.n) {
#pragma unroll 8
            for (unsigned k = 0; k < gridDim.y; ++k) v += __ldcg(g.part + k * (unsigned long long)g.np + c);
        }
    }
    if (c < g.n) g.dbias[c] = from_f32<T>(v);
}

struct LinearRecord {
    unsigned error;   // a wait inside a product gave up; cleared when its report has been read
    unsigned splits;  // parts of the split product that ran last
};

}  // namespace

struct scar_linear : TcHost {
    scar_linear_config cfg{};
    uint64_t kp = 0, np = 0;       // in and out features, rounded up to a multiple of 8
    unsigned dz_ctas = 1;          // most CTAs of a strip of k_linear_dz
    unsigned short *x = nullptr;   // copies for operands whose rows the products cannot read in place, float32's planes
    unsigned short *w = nullptr;
    unsigned short *dz = nullptr;
    float *sums = nullptr;         // [dz_ctas][np]
    unsigned *left = nullptr;
    LinearRecord *rec = nullptr;
    std::vector<void *> owned;
    uint64_t bytes = 0;
    bool arm_error = false;
};

namespace {

template <typename P> int linear_alloc(scar_linear *op, P **p, uint64_t bytes) {
    void *q = nullptr;
    if (cudaMalloc(&q, bytes) != cudaSuccess) {
        cudaGetLastError();
        return SCAR_ERR_ALLOC;
    }
    op->owned.push_back(q);
    op->bytes += bytes;
    *p = static_cast<P *>(q);
    return SCAR_OK;
}

uint64_t slope_size(const scar_linear *op) { return op->cfg.dtype == SCAR_F32 ? 4 : 2; }
bool has_slope(const scar_linear *op) { return op->cfg.activation != SCAR_ACT_IDENTITY; }

// x and w as the products read them: in place, or copied.
struct Operands {
    Operand x, w;
    bool w_copied;
};
template <typename T>
int place(scar_linear *op, const T *x, uint64_t xp, const T *w, uint64_t wp, unsigned rows, bool want_x, bool want_w, Operands *o) {
    constexpr int PL = sizeof(T) == 4 ? 3 : 1;
    const uint64_t K = op->cfg.in_features, N = op->cfg.out_features, x_rows = std::max<uint64_t>(op->cfg.max_rows, 1);
    const bool cx = want_x && (PL == 3 || !rows_aligned(x, xp, 2)), cw = want_w && (PL == 3 || !rows_aligned(w, wp, 2));
    int rc;
    if (cx && !op->x && (rc = linear_alloc(op, &op->x, PL * x_rows * op->kp * 2)) != SCAR_OK) return rc;
    if (cw && !op->w && (rc = linear_alloc(op, &op->w, PL * N * op->kp * 2)) != SCAR_OK) return rc;
    o->x = cx ? Operand{op->x, K, rows, op->kp, PL, x_rows * op->kp} : Operand{x, K, rows, rows > 1 ? xp : op->kp, 1, 0};
    o->w = cw ? Operand{op->w, K, N, op->kp, PL, N * op->kp} : Operand{w, K, N, N > 1 ? wp : op->kp, 1, 0};
    o->w_copied = cw;
    if (!cx && !cw) return SCAR_OK;
    const Copy<T> a{x, xp, cx ? rows : 0u, rows_aligned(x, xp, sizeof(T)), op->x, x_rows * op->kp};
    const Copy<T> b{w, wp, cw ? (unsigned)N : 0u, rows_aligned(w, wp, sizeof(T)), op->w, N * op->kp};
    const uint64_t groups = ((uint64_t)a.n + b.n) * (op->kp / 8);
    launch(op, k_linear_place<T>, (unsigned)std::min<uint64_t>((groups + 255) / 256, 16 * op->pairs), 256, 0, a, b, (unsigned)K, (unsigned)op->kp);
    return SCAR_OK;
}

TcArgs product(const scar_linear *op, unsigned m, unsigned n, unsigned k, int dyn) {
    TcArgs g{};
    g.m = m;
    g.n = n;
    g.k = k;
    g.dyn = dyn;
    g.most = dyn ? k : m;
    g.splits = 1;
    g.chosen = &op->rec->splits;
    g.error = &op->rec->error;
    g.bf16 = op->dtype != SCAR_F16;
    g.part = op->part;
    g.out_type = op->dtype;
    g.scale = 1.f;
    g.n_fast = n < m;
    return g;
}

int finish(scar_linear *op) {
    if (op->failed) {
        op->failed = false;
        cudaGetLastError();
        return SCAR_ERR_CUDA;
    }
    TRAIN_TRY(cudaGetLastError());
    if (op->arm_error) {  // self-test: the report of a wait that gave up
        op->arm_error = false;
        TRAIN_TRY(cudaMemsetAsync(&op->rec->error, 1, 1, op->stream));
    }
    return SCAR_OK;
}

// The join of a layer's parts with its epilogue costs about a launch.
template <typename T>
int run_forward(scar_linear *op, const T *x, uint64_t xp, const T *w, uint64_t wp, const T *bias, const T *res, uint64_t rp, const DropRule &drop,
                unsigned rows, T *y, uint64_t yp, void *slope) {
    constexpr int PL = sizeof(T) == 4 ? 3 : 1;
    const unsigned K = (unsigned)op->cfg.in_features, N = (unsigned)op->cfg.out_features;
    Operands o;
    int rc = place(op, x, xp, w, wp, rows, true, true, &o);
    if (rc != SCAR_OK) return rc;
    TcArgs g = product(op, rows, N, K, 0);
    if ((rc = make_map(op, &g.a, o.x, 128)) != SCAR_OK || (rc = make_map(op, &g.b, o.w, kBN / 2)) != SCAR_OK) return rc;
    g.out = y;
    g.out_pitch = yp;
    g.out_vec = rows_aligned(y, yp, sizeof(T));
    LayerArgs &l = g.layer;
    l.slope = slope;
    l.bias = bias;
    l.bias_vec = (uintptr_t)bias % 16 == 0;
    l.res = res;
    l.res_pitch = rp;
    l.res_vec = rows_aligned(res, rp, sizeof(T));
    l.drop = drop;
    choose_splits(op, g, PL == 3 ? 0.f : kLaunchS);  // float32 has that launch in any case
    dispatch_activation(op->cfg.activation, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        if (PL == 1 && g.splits == 1) {
            // a tensor map's store clips rows to whole 16-byte words only
            g.c_map = g.out_vec && N % 8 == 0;
            if (g.c_map) rc = make_map(op, &g.c, {y, N, rows, rows > 1 ? yp : op->np, 1, 0}, 32, 2, 64);
            if (rc == SCAR_OK && slope) rc = make_map(op, &l.slope_map, {slope, op->np, rows, op->np, 1, 0}, 32, 2, 64);
            if constexpr (PL == 1) {
                if (rc == SCAR_OK) launch_tc<1, false, false, (Epi)((int)Epi::kIdentity + ACT)>(op, g);
            }
            return;
        }
        launch_tc<PL, false, false, Epi::kPart>(op, g);
        const uint64_t todo = (uint64_t)rows * (op->np / 8);
        launch(op, k_linear_join<T, ACT>, (unsigned)std::min<uint64_t>((todo + 127) / 128, 32 * op->pairs), 128, 0, g);
    });
    return rc;
}

template <typename T>
int run_backward(scar_linear *op, const T *dy, uint64_t dyp, const T *x, uint64_t xp, const T *w, uint64_t wp, const void *slope, const DropRule &drop,
                 unsigned rows, T *dx, uint64_t dxp, T *dw, uint64_t dwp, T *dbias) {
    constexpr int PL = sizeof(T) == 4 ? 3 : 1;
    const unsigned K = (unsigned)op->cfg.in_features, N = (unsigned)op->cfg.out_features;
    int rc;
    if (rows == 0) {
        if (dw) TRAIN_TRY(cudaMemset2DAsync(dw, dwp * sizeof(T), 0, K * sizeof(T), N, op->stream));
        if (dbias) TRAIN_TRY(cudaMemsetAsync(dbias, 0, N * sizeof(T), op->stream));
        return SCAR_OK;
    }
    // dy itself where nothing changes it
    const bool direct = PL == 1 && !slope && !drop.on && rows_aligned(dy, dyp, 2);
    const uint64_t dz_rows = std::max<uint64_t>(op->cfg.max_rows, 1);
    if (!direct && !op->dz && (rc = linear_alloc(op, &op->dz, PL * dz_rows * op->np * 2)) != SCAR_OK) return rc;
    if (!direct || dbias) {
        const unsigned strips = (N + 255) / 256;
        const unsigned per = (unsigned)round_up((rows + op->dz_ctas - 1) / op->dz_ctas, 8);
        const DzArgs<T> a{dy, dyp, rows_aligned(dy, dyp, sizeof(T)), slope, rows, N, (unsigned)op->np, per, drop, direct ? nullptr : op->dz, dz_rows * op->np,
                          op->sums, dbias, op->left};
        launch(op, k_linear_dz<T>, dim3(strips, (rows + per - 1) / per), 256, 0, a);
    }
    if (!dx && !dw) return SCAR_OK;
    Operands o;
    if ((rc = place(op, x, xp, w, wp, rows, dw != nullptr, dx != nullptr, &o)) != SCAR_OK) return rc;
    const Operand dz = direct ? Operand{dy, N, rows, rows > 1 ? dyp : op->np, 1, 0} : Operand{op->dz, N, rows, op->np, PL, dz_rows * op->np};
    TcArgs dxg = product(op, rows, K, N, 0), dwg = product(op, N, K, rows, 1);
    if (dx) {
        if ((rc = make_map(op, &dxg.a, dz, 128)) != SCAR_OK || (rc = make_map(op, &dxg.b, o.w, 64)) != SCAR_OK) return rc;
        dxg.out = dx;
        dxg.out_pitch = dxp;
        dxg.out_vec = rows_aligned(dx, dxp, sizeof(T));
        dxg.c_map = dxg.out_vec && K * sizeof(T) % 16 == 0;
        if (dxg.c_map && (rc = make_map(op, &dxg.c, {dx, K, rows, rows > 1 ? dxp : op->kp, 1, 0}, 32, sizeof(T), PL == 1 ? 64 : 128)) != SCAR_OK) return rc;
    }
    // rows of dw that do not lie on 16-byte boundaries go through the room of w's copy, which dx is done with by then
    bool through_w = false;
    if (dw) {
        if ((rc = make_map(op, &dwg.a, dz, 64)) != SCAR_OK || (rc = make_map(op, &dwg.b, o.x, 64)) != SCAR_OK) return rc;
        dwg.out = dw;
        dwg.out_pitch = dwp;
        dwg.out_vec = rows_aligned(dw, dwp, sizeof(T));
        through_w = !dwg.out_vec && op->w;
        if (through_w) {
            dwg.out = op->w;
            dwg.out_pitch = op->kp;
            dwg.out_vec = 1;
        }
        dwg.c_map = through_w || (dwg.out_vec && K * sizeof(T) % 16 == 0);
        if (dwg.c_map && (rc = make_map(op, &dwg.c, {dwg.out, K, N, N > 1 ? dwg.out_pitch : op->kp, 1, 0}, 32, sizeof(T), PL == 1 ? 64 : 128)) != SCAR_OK) return rc;
    }
    if (dx && dw) {
        launch_grads<PL>(op, dxg, dwg, through_w);
    } else if (dx) {
        choose_splits(op, dxg, kLaunchS);
        launch_out<PL, false>(op, dxg);
    } else {
        choose_splits(op, dwg, kLaunchS);
        launch_out<PL, true>(op, dwg);
    }
    if (through_w)
        launch(op, k_unplace<T>, (unsigned)std::min<uint64_t>((N + 7) / 8, 16 * op->pairs), 256, 0, reinterpret_cast<const T *>(op->w), op->kp, N, K, dw, dwp);
    return SCAR_OK;
}

struct Matrix {
    const void *p;
    uint64_t pitch, rows, cols;
    bool wanted;  // a nullptr is an error
};
int check_matrices(const scar_linear *op, std::initializer_list<Matrix> all) {
    const unsigned b = elem_size(op->dtype);
    for (const Matrix &m : all) {
        if (!m.p && m.wanted) return SCAR_ERR_INVALID_ARG;
        if (m.p && ((uintptr_t)m.p % b || m.pitch >= kPitchEnd || (m.rows > 1 && m.pitch < m.cols))) return SCAR_ERR_INVALID_ARG;
    }
    return SCAR_OK;
}

template <typename F> int guarded(scar_linear *op, F &&f) {
    int rc = SCAR_OK;
    try {
        dispatch_operand(op->dtype, [&](auto e) { rc = f(e); });
    } catch (...) {
        rc = SCAR_ERR_ALLOC;
    }
    const int end = finish(op);
    return rc != SCAR_OK ? rc : end;
}

int setup(scar_linear *op) {
    const scar_linear_config &c = op->cfg;
    TRAIN_TRY(cudaGetDevice(&op->device));
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    TRAIN_TRY(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found));
    if (found != cudaDriverEntryPointSuccess || !fn) return SCAR_ERR_CUDA;
    op->encode = reinterpret_cast<EncodeTiled>(fn);
    const bool f32 = c.dtype == SCAR_F32;
    if (f32 ? !allow_smem_all<3>()
            : !(allow_smem_all<1>() && allow_smem(k_tc_gemm<1, false, false, Epi::kIdentity, 1>) && allow_smem(k_tc_gemm<1, false, false, Epi::kRelu, 1>) &&
                allow_smem(k_tc_gemm<1, false, false, Epi::kGelu, 1>) && allow_smem(k_tc_gemm<1, false, false, Epi::kSilu, 1>)))
        return SCAR_ERR_CUDA;
    int sms = 0;
    TRAIN_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, op->device));
    op->pairs = std::max(1, sms / 2);
    op->planes = f32 ? 3 : 1;
    op->kp = round_up(c.in_features, 8);
    op->np = round_up(c.out_features, 8);
    const uint64_t T = std::max<uint64_t>(c.max_rows, 1), strips = (op->np + 255) / 256;
    // about four CTAs of k_linear_dz per SM over all strips
    op->dz_ctas = (unsigned)std::min<uint64_t>((T + 31) / 32, std::max<uint64_t>(1, 8 * op->pairs / strips));
    uint64_t most = T * op->np;
    if (!c.forward_only) most = std::max(most, std::max(T * op->kp, c.out_features * op->kp));
    op->part_bytes = std::min<uint64_t>(64ull << 20, most * 4 * kMostSplits);
    if (f32) op->part_bytes = std::max(op->part_bytes, T * op->np * 4);  // the layer's sums
    const bool copies = f32 || c.in_features % 8;
    struct {
        void **p;
        uint64_t bytes;
    } const want[] = {
        {(void **)&op->rec, sizeof(LinearRecord)}, {(void **)&op->part, op->part_bytes}, {(void **)&op->left, 4 * strips},
        {(void **)&op->sums, c.forward_only ? 0 : 4ull * op->dz_ctas * op->np}, {(void **)&op->dz, c.forward_only || (!f32 && !has_slope(op)) ? 0 : op->planes * T * op->np * 2},
        {(void **)&op->x, copies ? op->planes * T * op->kp * 2 : 0}, {(void **)&op->w, copies ? op->planes * c.out_features * op->kp * 2 : 0},
    };
    uint64_t total = 0;
    for (const auto &x : want) total += round_up(x.bytes, 256);
    char *block = nullptr;
    const int rc = linear_alloc(op, &block, total);
    if (rc != SCAR_OK) return rc;
    for (const auto &x : want)
        if (x.bytes) {
            *x.p = block;
            block += round_up(x.bytes, 256);
        }
    TRAIN_TRY(cudaMemsetAsync(op->rec, 0, sizeof(LinearRecord), op->stream));
    TRAIN_TRY(cudaMemsetAsync(op->left, 0, 4 * strips, op->stream));
    TRAIN_TRY(cudaStreamSynchronize(op->stream));
    return SCAR_OK;
}

}  // namespace

extern "C" {

int scar_linear_init(scar_linear **out, const scar_linear_config *cfg, void *cuda_stream) {
    if (!out) return SCAR_ERR_INVALID_ARG;
    *out = nullptr;
    const uint64_t top = 1ull << 31;
    if (!cfg || !is_operand_type(cfg->dtype) || cfg->activation < SCAR_ACT_IDENTITY || cfg->activation > SCAR_ACT_SILU || !cfg->in_features ||
        !cfg->out_features || cfg->in_features >= top || cfg->out_features >= top || cfg->max_rows >= top)
        return SCAR_ERR_INVALID_ARG;
    scar_linear *op = new (std::nothrow) scar_linear();
    if (!op) return SCAR_ERR_ALLOC;
    op->cfg = *cfg;
    op->dtype = cfg->dtype;
    op->stream = static_cast<cudaStream_t>(cuda_stream);
    int rc;
    try {
        rc = setup(op);
    } catch (...) {
        rc = SCAR_ERR_ALLOC;
    }
    if (rc != SCAR_OK) {
        scar_linear_destroy(op);
        return rc;
    }
    *out = op;
    return SCAR_OK;
}

int scar_linear_forward(scar_linear *op, const void *d_x, uint64_t x_pitch, const void *d_w, uint64_t w_pitch, const void *d_bias,
                        const void *d_residual, uint64_t residual_pitch, const scar_dropout *dropout, uint64_t n_rows, void *d_y, uint64_t y_pitch,
                        void *d_slope) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    const uint64_t K = op->cfg.in_features, N = op->cfg.out_features;
    if (n_rows > op->cfg.max_rows) return SCAR_ERR_CAPACITY;
    const bool any = n_rows != 0;
    int rc = check_matrices(op, {{d_x, x_pitch, n_rows, K, any}, {d_w, w_pitch, N, K, any}, {d_bias, 0, 1, N, false}, {d_residual, residual_pitch, n_rows, N, false},
                                 {d_y, y_pitch, n_rows, N, any}});
    DropRule drop;
    if (rc != SCAR_OK || (rc = make_rule(dropout, &drop)) != SCAR_OK) return rc;
    if ((uintptr_t)d_slope % 16 || (d_slope && !has_slope(op))) return SCAR_ERR_INVALID_ARG;
    if ((rc = check_current_device(op->device)) != SCAR_OK || !any) return rc;
    return guarded(op, [&](auto e) {
        using T = decltype(e);
        return run_forward<T>(op, static_cast<const T *>(d_x), x_pitch, static_cast<const T *>(d_w), w_pitch, static_cast<const T *>(d_bias),
                              static_cast<const T *>(d_residual), residual_pitch, drop, (unsigned)n_rows, static_cast<T *>(d_y), y_pitch, d_slope);
    });
}

int scar_linear_backward(scar_linear *op, const void *d_dy, uint64_t dy_pitch, const void *d_x, uint64_t x_pitch, const void *d_w, uint64_t w_pitch,
                         const void *d_slope, const scar_dropout *dropout, uint64_t n_rows, void *d_dx, uint64_t dx_pitch, void *d_dw, uint64_t dw_pitch,
                         void *d_dbias) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    if (op->cfg.forward_only) return SCAR_ERR_STATE;
    const uint64_t K = op->cfg.in_features, N = op->cfg.out_features;
    if (n_rows > op->cfg.max_rows) return SCAR_ERR_CAPACITY;
    const bool any = n_rows != 0;
    int rc = check_matrices(op, {{d_dy, dy_pitch, n_rows, N, any}, {d_x, x_pitch, n_rows, K, any && d_dw}, {d_w, w_pitch, N, K, any && d_dx},
                                 {d_dx, dx_pitch, n_rows, K, false}, {d_dw, dw_pitch, N, K, false}, {d_dbias, 0, 1, N, false}});
    DropRule drop;
    if (rc != SCAR_OK || (rc = make_rule(dropout, &drop)) != SCAR_OK) return rc;
    if ((uintptr_t)d_slope % 16 || (d_slope != nullptr) != (has_slope(op) && (any || d_slope))) return SCAR_ERR_INVALID_ARG;
    if ((rc = check_current_device(op->device)) != SCAR_OK) return rc;
    return guarded(op, [&](auto e) {
        using T = decltype(e);
        return run_backward<T>(op, static_cast<const T *>(d_dy), dy_pitch, static_cast<const T *>(d_x), x_pitch, static_cast<const T *>(d_w), w_pitch, d_slope,
                               drop, (unsigned)n_rows, static_cast<T *>(d_dx), dx_pitch, static_cast<T *>(d_dw), dw_pitch, static_cast<T *>(d_dbias));
    });
}

uint64_t scar_linear_slope_bytes(const scar_linear *op, uint64_t n_rows) { return op && has_slope(op) ? n_rows * op->np * slope_size(op) : 0; }

int scar_linear_status(scar_linear *op) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    const int rc = check_current_device(op->device);
    if (rc != SCAR_OK) return rc;
    unsigned error = 0;
    TRAIN_TRY(cudaMemcpyAsync(&error, &op->rec->error, sizeof(error), cudaMemcpyDeviceToHost, op->stream));
    TRAIN_TRY(cudaMemsetAsync(&op->rec->error, 0, sizeof(error), op->stream));
    TRAIN_TRY(cudaStreamSynchronize(op->stream));
    return error ? SCAR_ERR_TIMEOUT : SCAR_OK;
}

int scar_linear_selftest_arm_timeout(scar_linear *op) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    op->arm_error = true;
    return SCAR_OK;
}

uint64_t scar_linear_workspace_bytes(const scar_linear *op) { return op ? op->bytes : 0; }
uint64_t scar_linear_launch_count(const scar_linear *op) { return op ? op->launches : 0; }

int scar_linear_destroy(scar_linear *op) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    const bool ok = cudaStreamSynchronize(op->stream) == cudaSuccess;
    for (void *p : op->owned) cudaFree(p);
    delete op;
    if (!ok) cudaGetLastError();
    return ok ? SCAR_OK : SCAR_ERR_CUDA;
}

}  // extern "C"
