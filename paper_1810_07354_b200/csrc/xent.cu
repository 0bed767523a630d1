// Linear softmax cross entropy with its gradient (scar_xent_* of scar.h).
//
// Rows that do not count are dropped first; the others go through the products in pieces, each of which holds the
// logits of its rows until their gradient has taken their place.
#include <algorithm>
#include <new>
#include <vector>

#include "train_common.cuh"

using namespace scar;

namespace {

constexpr int kRowThreads = 1024;
constexpr int kTile = 64;   // edge of a CTA's output tile
constexpr int kTileK = 16;

struct XentRecord {
    double sum;  // of the row losses
    float loss;
    unsigned rows, ignored, bad;
    unsigned error;
};

// Compacts the rows that count: idx[0 .. rows) are their numbers, ascending.  One CTA: the labels of a step are few.
__global__ void __launch_bounds__(kRowThreads)
k_xent_rows(const long long *__restrict__ labels, unsigned n, long long ignore, unsigned n_classes,
            unsigned *__restrict__ idx, float *__restrict__ row_loss, XentRecord *rec) {
    __shared__ unsigned sh[kRowThreads / 32], base, n_ign, n_bad;
    if (threadIdx.x == 0) base = n_ign = n_bad = 0;
    __syncthreads();
    const unsigned lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (unsigned at = 0; at < n; at += kRowThreads) {
        const unsigned t = at + threadIdx.x;
        bool keep = false, bad = false, ign = false;
        if (t < n) {
            const long long y = labels[t];
            ign = y == ignore;
            keep = !ign && y >= 0 && y < (long long)n_classes;
            bad = !ign && !keep;
            if (!keep) row_loss[t] = 0.f;
        }
        const unsigned m = __ballot_sync(0xffffffffu, keep);
        const unsigned mi = __ballot_sync(0xffffffffu, ign), mb = __ballot_sync(0xffffffffu, bad);
        if (lane == 0) {
            sh[warp] = __popc(m);
            if (mi) atomicAdd(&n_ign, __popc(mi));
            if (mb) atomicAdd(&n_bad, __popc(mb));
        }
        __syncthreads();
        unsigned before = base, all = 0;
        for (unsigned w = 0; w < kRowThreads / 32; ++w) {
            if (w < warp) before += sh[w];
            all += sh[w];
        }
        if (keep) idx[before + __popc(m & ((1u << lane) - 1u))] = t;
        __syncthreads();
        if (threadIdx.x == 0) base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        rec->sum = 0.0;
        rec->rows = base;
        rec->ignored = n_ign;
        rec->bad = n_bad;
        rec->error = 0;
        rec->loss = 0.f;
    }
}

// out(m, n) = sum_k A(m, k) B(n, k), 64 x 64 outputs per CTA, float32 throughout.  A, B: load(row, k) or 0 outside.
template <typename FA, typename FB, typename FO>
__device__ __forceinline__ void gemm_tile(unsigned m0, unsigned n0, unsigned K, FA a, FB b, FO out) {
    __shared__ float sa[kTileK][kTile + 4], sb[kTileK][kTile + 4];
    const unsigned tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (unsigned k0 = 0; k0 < K; k0 += kTileK) {
        for (unsigned i = threadIdx.x; i < kTile * kTileK; i += 256) {
            const unsigned r = i / kTileK, k = i % kTileK;
            sa[k][r] = k0 + k < K ? a(m0 + r, k0 + k) : 0.f;
            sb[k][r] = k0 + k < K ? b(n0 + r, k0 + k) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kTileK; ++k) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty * 4 + i], sb[k][tx * 4 + j], acc[i][j]);
        }
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) out(m0 + ty * 4 + i, n0 + tx * 4 + j, acc[i][j]);
}

struct Piece {
    unsigned first, most;  // rows [first, min(first + most, rows)) of the compacted list
    __device__ unsigned rows(const XentRecord *rec) const {
        return rec->rows > first ? min(most, rec->rows - first) : 0u;
    }
};

template <typename T>
__global__ void __launch_bounds__(256)
k_xent_logits(const T *h, uint64_t hp, const T *w, uint64_t wp, unsigned V, unsigned D, const unsigned *idx,
              const XentRecord *rec, Piece p, float *z) {
    const unsigned R = p.rows(rec), m0 = blockIdx.y * kTile;
    if (m0 >= R) return;
    gemm_tile(m0, blockIdx.x * kTile, D,
              [&](unsigned r, unsigned k) { return r < R ? to_f32<T>(h[idx[p.first + r] * hp + k]) : 0.f; },
              [&](unsigned v, unsigned k) { return v < V ? to_f32<T>(w[v * wp + k]) : 0.f; },
              [&](unsigned r, unsigned v, float x) { if (r < R && v < V) z[(uint64_t)r * V + v] = x; });
}

__device__ __forceinline__ float cta_max(float v, float *sh) {
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    v = sh[0];
    for (unsigned w = 1; w < blockDim.x / 32; ++w) v = fmaxf(v, sh[w]);
    __syncthreads();
    return v;
}
__device__ __forceinline__ float cta_add(float v, float *sh) {
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
    for (unsigned w = 0; w < blockDim.x / 32; ++w) v += sh[w];
    __syncthreads();
    return v;
}

// One CTA per row: loss, and with GRAD the row's logits become exp(z - lse) - [v = label].
template <bool GRAD>
__global__ void __launch_bounds__(256)
k_xent_softmax(float *z, unsigned V, const long long *labels, const unsigned *idx, const XentRecord *rec, Piece p,
               float *row_loss) {
    __shared__ float sh[8];
    const unsigned r = blockIdx.x;
    if (r >= p.rows(rec)) return;
    const unsigned t = idx[p.first + r];
    const unsigned y = (unsigned)labels[t];
    float *row = z + (uint64_t)r * V;
    float top = -INFINITY;
    for (unsigned v = threadIdx.x; v < V; v += 256) top = fmaxf(top, row[v]);
    top = cta_max(top, sh);
    float s = 0.f;
    for (unsigned v = threadIdx.x; v < V; v += 256) s += expf(row[v] - top);
    s = cta_add(s, sh);
    const float lse = top + logf(s);
    const float zl = row[y];
    __syncthreads();
    if (threadIdx.x == 0) row_loss[t] = lse - zl;
    if (!GRAD) return;
    for (unsigned v = threadIdx.x; v < V; v += 256) row[v] = v == y ? expm1f(row[v] - lse) : expf(row[v] - lse);
}

__device__ __forceinline__ float grad_factor(const XentRecord *rec, float scale, bool mean) {
    return mean ? scale / (float)max(rec->rows, 1u) : scale;
}

template <typename T>
__global__ void __launch_bounds__(256)
k_xent_dh(const float *dz, const T *w, uint64_t wp, unsigned V, unsigned D, const unsigned *idx, const XentRecord *rec,
          Piece p, float scale, bool mean, T *dh, uint64_t dhp) {
    const unsigned R = p.rows(rec), m0 = blockIdx.y * kTile;
    if (m0 >= R) return;
    const float g = grad_factor(rec, scale, mean);
    gemm_tile(m0, blockIdx.x * kTile, V,
              [&](unsigned r, unsigned v) { return r < R ? dz[(uint64_t)r * V + v] : 0.f; },
              [&](unsigned d, unsigned v) { return d < D ? to_f32<T>(w[v * wp + d]) : 0.f; },
              [&](unsigned r, unsigned d, float x) { if (r < R && d < D) dh[idx[p.first + r] * dhp + d] = from_f32<T>(x * g); });
}

template <typename T>
__global__ void __launch_bounds__(256)
k_xent_dw(const float *dz, const T *h, uint64_t hp, unsigned V, unsigned D, const unsigned *idx, const XentRecord *rec,
          Piece p, float scale, bool mean, bool first, bool last, float *acc, T *dw, uint64_t dwp) {
    const unsigned R = p.rows(rec);
    const float g = grad_factor(rec, scale, mean);
    gemm_tile(blockIdx.y * kTile, blockIdx.x * kTile, R,
              [&](unsigned v, unsigned r) { return v < V ? dz[(uint64_t)r * V + v] : 0.f; },
              [&](unsigned d, unsigned r) { return d < D ? to_f32<T>(h[idx[p.first + r] * hp + d]) : 0.f; },
              [&](unsigned v, unsigned d, float x) {
                  if (v >= V || d >= D) return;
                  if (!first) x += acc[(uint64_t)v * D + d];
                  if (last) dw[v * dwp + d] = from_f32<T>(x * g);
                  else acc[(uint64_t)v * D + d] = x;
              });
}

// Rows of dh that do not count are zero.
template <typename T>
__global__ void __launch_bounds__(256)
k_xent_zero_rows(const long long *labels, long long ignore, unsigned V, unsigned D, T *dh, uint64_t dhp) {
    const long long y = labels[blockIdx.x];
    if (y != ignore && y >= 0 && y < (long long)V) return;
    for (unsigned d = threadIdx.x; d < D; d += 256) dh[blockIdx.x * dhp + d] = from_f32<T>(0.f);
}

__global__ void __launch_bounds__(kRowThreads)
k_xent_loss(const float *row_loss, unsigned n, bool mean, XentRecord *rec, float *d_loss) {
    __shared__ double sh[32];
    double s = 0.0;
    for (unsigned t = threadIdx.x; t < n; t += kRowThreads) s += row_loss[t];
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x) return;
    s = 0.0;
    for (int w = 0; w < 32; ++w) s += sh[w];
    rec->sum = s;
    rec->loss = (float)(mean ? s / (double)max(rec->rows, 1u) : s);
    if (d_loss) *d_loss = rec->loss;
}

}  // namespace

struct scar_xent {
    int device = 0;
    cudaStream_t stream = nullptr;
    scar_xent_config cfg{};
    unsigned piece = 0;  // rows per piece
    unsigned *idx = nullptr;
    float *row_loss = nullptr;
    float *z = nullptr;
    float *acc = nullptr;
    XentRecord *rec = nullptr;
    XentRecord *h_rec = nullptr;  // pinned
    std::vector<void *> owned;
    uint64_t bytes = 0;
    uint64_t launches = 0;
    bool ran = false;
};

namespace {

template <typename P> int xent_alloc(scar_xent *op, P **p, uint64_t bytes) {
    void *q = nullptr;
    bytes = bytes ? bytes : 16;
    if (cudaMalloc(&q, bytes) != cudaSuccess) {
        cudaGetLastError();
        return SCAR_ERR_ALLOC;
    }
    op->owned.push_back(q);
    op->bytes += bytes;
    *p = static_cast<P *>(q);
    return SCAR_OK;
}

int check_call(const scar_xent *op, const void *h, uint64_t hp, const void *w, uint64_t wp, const int64_t *labels,
               uint64_t n) {
    if (!op || !w) return SCAR_ERR_INVALID_ARG;
    const unsigned b = elem_size(op->cfg.dtype);
    if (n > op->cfg.max_tokens) return SCAR_ERR_CAPACITY;
    if (n && (!h || !labels)) return SCAR_ERR_INVALID_ARG;
    if (hp < op->cfg.dim || wp < op->cfg.dim || hp >= (1ull << 40) || wp >= (1ull << 40)) return SCAR_ERR_INVALID_ARG;
    if ((uintptr_t)h % b || (uintptr_t)w % b || (uintptr_t)labels % 8) return SCAR_ERR_INVALID_ARG;
    return check_current_device(op->device);
}

template <typename T>
void run_xent(scar_xent *op, const T *h, uint64_t hp, const T *w, uint64_t wp, const int64_t *labels, unsigned n,
              bool grad, float scale, float *row_loss, float *d_loss, T *dh, uint64_t dhp, T *dw, uint64_t dwp) {
    const unsigned V = (unsigned)op->cfg.n_classes, D = (unsigned)op->cfg.dim;
    const bool mean = op->cfg.reduction == SCAR_MEAN;
    const long long *y = reinterpret_cast<const long long *>(labels);
    cudaStream_t s = op->stream;
    if (!row_loss) row_loss = op->row_loss;
    auto tiles = [](unsigned v) { return (v + kTile - 1) / kTile; };
    k_xent_rows<<<1, kRowThreads, 0, s>>>(y, n, op->cfg.ignore_label, V, op->idx, row_loss, op->rec);
    op->launches++;
    if (grad && n) {
        k_xent_zero_rows<T><<<n, 256, 0, s>>>(y, op->cfg.ignore_label, V, D, dh, dhp);
        op->launches++;
    }
    for (unsigned at = 0; at < std::max(n, 1u); at += op->piece) {
        const Piece p{at, op->piece};
        const unsigned rows = std::min(op->piece, n - at);
        if (rows) {
            k_xent_logits<T><<<dim3(tiles(V), tiles(rows)), 256, 0, s>>>(h, hp, w, wp, V, D, op->idx, op->rec, p, op->z);
            if (grad) k_xent_softmax<true><<<rows, 256, 0, s>>>(op->z, V, y, op->idx, op->rec, p, row_loss);
            else k_xent_softmax<false><<<rows, 256, 0, s>>>(op->z, V, y, op->idx, op->rec, p, row_loss);
            op->launches += 2;
        }
        if (!grad) continue;
        if (rows) {
            k_xent_dh<T><<<dim3(tiles(D), tiles(rows)), 256, 0, s>>>(op->z, w, wp, V, D, op->idx, op->rec, p, scale, mean, dh, dhp);
            op->launches++;
        }
        k_xent_dw<T><<<dim3(tiles(D), tiles(V)), 256, 0, s>>>(op->z, h, hp, V, D, op->idx, op->rec, p, scale, mean, at == 0,
                                                              at + op->piece >= n, op->acc, dw, dwp);
        op->launches++;
    }
    k_xent_loss<<<1, kRowThreads, 0, s>>>(row_loss, n, mean, op->rec, d_loss);
    op->launches++;
}

int call(scar_xent *op, const void *h, uint64_t hp, const void *w, uint64_t wp, const int64_t *labels, uint64_t n,
         bool grad, float scale, float *row_loss, float *d_loss, void *dh, uint64_t dhp, void *dw, uint64_t dwp) {
    dispatch_operand(op->cfg.dtype, [&](auto e) {
        using T = decltype(e);
        run_xent<T>(op, static_cast<const T *>(h), hp, static_cast<const T *>(w), wp, labels, (unsigned)n, grad, scale,
                    row_loss, d_loss, static_cast<T *>(dh), dhp, static_cast<T *>(dw), dwp);
    });
    TRAIN_TRY(cudaGetLastError());
    op->ran = true;
    return SCAR_OK;
}

}  // namespace

extern "C" {

int scar_xent_init(scar_xent **out, const scar_xent_config *cfg, void *cuda_stream) {
    if (!out) return SCAR_ERR_INVALID_ARG;
    *out = nullptr;
    if (!cfg || !is_operand_type(cfg->dtype) || (cfg->reduction != SCAR_MEAN && cfg->reduction != SCAR_SUM))
        return SCAR_ERR_INVALID_ARG;
    const uint64_t top = 1ull << 31;
    if (!cfg->n_classes || !cfg->dim || cfg->n_classes >= top || cfg->dim >= top || cfg->max_tokens >= top)
        return SCAR_ERR_INVALID_ARG;
    scar_xent *op = new (std::nothrow) scar_xent();
    if (!op) return SCAR_ERR_ALLOC;
    op->cfg = *cfg;
    op->stream = static_cast<cudaStream_t>(cuda_stream);
    auto setup = [&]() -> int {
        TRAIN_TRY(cudaGetDevice(&op->device));
        const uint64_t row = 4 * cfg->n_classes, limit = cfg->workspace_bytes ? cfg->workspace_bytes : 1ull << 30;
        uint64_t piece = std::max<uint64_t>(limit / row / 256 * 256, 256);
        const bool sums = cfg->dtype != SCAR_F32;  // dw itself holds the sums of a float32 operator
        if (piece < cfg->max_tokens && !cfg->loss_only &&
            cfg->max_tokens * row <= piece * row + cfg->n_classes * cfg->dim * 4)
            piece = cfg->max_tokens;
        op->piece = (unsigned)std::min<uint64_t>(piece, std::max<uint64_t>(cfg->max_tokens, 1));
        int rc;
        if ((rc = xent_alloc(op, &op->idx, 4 * cfg->max_tokens)) != SCAR_OK) return rc;
        if ((rc = xent_alloc(op, &op->row_loss, 4 * cfg->max_tokens)) != SCAR_OK) return rc;
        if ((rc = xent_alloc(op, &op->rec, sizeof(XentRecord))) != SCAR_OK) return rc;
        if ((rc = xent_alloc(op, &op->z, (uint64_t)op->piece * row)) != SCAR_OK) return rc;
        (void)sums;
        if (!cfg->loss_only && op->piece < cfg->max_tokens &&
            (rc = xent_alloc(op, &op->acc, cfg->n_classes * cfg->dim * 4)) != SCAR_OK)
            return rc;
        if (cudaMallocHost(&op->h_rec, sizeof(XentRecord)) != cudaSuccess) {
            cudaGetLastError();
            return SCAR_ERR_ALLOC;
        }
        TRAIN_TRY(cudaStreamSynchronize(op->stream));
        return SCAR_OK;
    };
    int rc;
    try {
        rc = setup();
    } catch (...) {
        rc = SCAR_ERR_ALLOC;
    }
    if (rc != SCAR_OK) {
        scar_xent_destroy(op);
        return rc;
    }
    *out = op;
    return SCAR_OK;
}

int scar_xent_loss(scar_xent *op, const void *d_h, uint64_t h_pitch, const void *d_w, uint64_t w_pitch,
                   const int64_t *d_labels, uint64_t n_tokens, float *d_row_loss, float *d_loss) {
    const int rc = check_call(op, d_h, h_pitch, d_w, w_pitch, d_labels, n_tokens);
    if (rc != SCAR_OK) return rc;
    return call(op, d_h, h_pitch, d_w, w_pitch, d_labels, n_tokens, false, 0.f, d_row_loss, d_loss, nullptr, 0, nullptr, 0);
}

int scar_xent_loss_grad(scar_xent *op, const void *d_h, uint64_t h_pitch, const void *d_w, uint64_t w_pitch,
                        const int64_t *d_labels, uint64_t n_tokens, float grad_scale, float *d_row_loss,
                        float *d_loss, void *d_dh, uint64_t dh_pitch, void *d_dw, uint64_t dw_pitch) {
    const int rc = check_call(op, d_h, h_pitch, d_w, w_pitch, d_labels, n_tokens);
    if (rc != SCAR_OK) return rc;
    const unsigned b = elem_size(op->cfg.dtype);
    if (op->cfg.loss_only) return SCAR_ERR_STATE;
    if (!d_dw || (n_tokens && !d_dh) || (uintptr_t)d_dh % b || (uintptr_t)d_dw % b) return SCAR_ERR_INVALID_ARG;
    if (dh_pitch < op->cfg.dim || dw_pitch < op->cfg.dim || dh_pitch >= (1ull << 40) || dw_pitch >= (1ull << 40))
        return SCAR_ERR_INVALID_ARG;
    return call(op, d_h, h_pitch, d_w, w_pitch, d_labels, n_tokens, true, grad_scale, d_row_loss, d_loss, d_dh, dh_pitch,
                d_dw, dw_pitch);
}

int scar_xent_status(scar_xent *op, scar_xent_info *out) {
    if (!op || !out) return SCAR_ERR_INVALID_ARG;
    const int rc = check_current_device(op->device);
    if (rc != SCAR_OK) return rc;
    if (!op->ran) return SCAR_ERR_STATE;
    TRAIN_TRY(cudaMemcpyAsync(op->h_rec, op->rec, sizeof(XentRecord), cudaMemcpyDeviceToHost, op->stream));
    TRAIN_TRY(cudaStreamSynchronize(op->stream));
    out->loss = op->h_rec->loss;
    out->rows = op->h_rec->rows;
    out->ignored = op->h_rec->ignored;
    out->bad = op->h_rec->bad;
    return op->h_rec->error ? SCAR_ERR_TIMEOUT : SCAR_OK;
}

uint64_t scar_xent_workspace_bytes(const scar_xent *op) { return op ? op->bytes : 0; }
uint64_t scar_xent_launch_count(const scar_xent *op) { return op ? op->launches : 0; }

int scar_xent_destroy(scar_xent *op) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    const bool ok = cudaStreamSynchronize(op->stream) == cudaSuccess;
    for (void *p : op->owned) cudaFree(p);
    if (op->h_rec) cudaFreeHost(op->h_rec);
    delete op;
    if (!ok) cudaGetLastError();
    return ok ? SCAR_OK : SCAR_ERR_CUDA;
}

}  // extern "C"
