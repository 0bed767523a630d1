// Linear softmax cross entropy with its gradient (scar_xent_* of scar.h).
//
// A call:  rows that count are listed and copied together (k_xent_rows, k_xent_place; float32 is split into three
// bfloat16 planes on the way, w too).  The rows then go through the products in pieces:
//   z = h w^T        the product's epilogue keeps, per row and 128 classes, the maximum and the sum of exponentials, and
//                    for gradients the exponentials relative to that maximum, in float16 (k_tc_gemm, kProb / kStat)
//   dz               k_xent_dz joins a row's groups to lse and turns the exponentials into dz, in place
//   dh = dz w, dw = dz^T h
// so the logits are computed once (6 n V D operations, not 8) and, for 16-bit operands, exist as such in tensor memory alone.
// float32 operands keep float32 logits of the piece beside the same statistics; products with too few tiles to fill the
// GPU (their sum over D is cut into parts) leave float32 parts for k_xent_softmax.  The last CTA of the last softmax adds
// the row losses.
//
// What bounds it, measured: many rows, the tensor cores (4096 x 32000 x 2048 bfloat16: the logits' product 300 us with
// its pipe active 86 % of the time, dh and dw together 594 us, 94 %, at the 1.5 - 1.6 GHz that the power limit leaves;
// 81 us for the dz pass at 5.2 TB/s); few rows, reading w (one row, 128000 x 4096: 5.6 TB/s); small sizes, the chain of
// five to seven launches (16 x 2000 x 512: 34 us).
#include <algorithm>
#include <new>
#include <vector>

#include "tc_gemm.cuh"

using namespace scar;

namespace {

constexpr int kRowThreads = 1024;
constexpr unsigned kNone = 0xffffffffu;

// A row of the softmax kernels has a warp or a CTA of its own.  Loss and gradients, replayed from a graph, dim 64, warp / CTA in us:
//   bfloat16  1184 rows: 2048 classes 34.2 / 36.1, 4000 49.5 / 48.7;  4736 rows: 8192 classes 119 / 127, 16000 222 / 213
//   float32   1184 rows: 1000 classes 58.3 / 57.4, 2048 67.5 / 61.4;  4736 rows: 4000 classes 189 / 194, 8192 314 / 310
// so the limit is one of bytes: rows of 4 KiB (16-bit values or float32 logits) where there is a CTA of them for every SM,
// of 16 KiB where there are four.  512 rows of 256 to 2048 classes: 24.7 / 26.7 to 33.0 / 33.4, float32 63.5 / 56.9: left to CTAs.
constexpr unsigned kWarpRowBytes = 4096;

struct XentRecord {
    float loss;
    unsigned rows, ignored, bad;
    unsigned error; // a wait inside a product gave up
    unsigned done;  // CTAs of the last softmax kernel that are through
    unsigned splits; // parts of the split product that ran last
};

// Every kernel of a call is launched while the one before it may still run; nothing is touched before that one is done.
__device__ __forceinline__ void griddep_start() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Lists the rows that count, in order: row_of[0 .. rows) are their numbers, pos is the inverse (kNone for the rest).  By one
// CTA of kThreads, eight labels per thread at a time (kThreads apart): the labels of a step are few.
constexpr int kLabels = 8;
struct RowList {
    const long long *labels;
    unsigned n;
    long long ignore;
    unsigned n_classes;
    unsigned *row_of, *pos;
    int *label;
    float *row_loss;
    XentRecord *rec;
    float *d_loss;
    unsigned error;  // what the record's begins with: 1 in a self-test
};
template <int kThreads, bool kWrite> __device__ __forceinline__ unsigned list_rows(const RowList &q, unsigned *pos) {
    constexpr int kWarps = kThreads / 32, kCounts = kLabels * kWarps;  // rows that count, by round of labels and warp
    __shared__ unsigned sh[kCounts], total, n_ign, n_bad;
    if (threadIdx.x == 0) n_ign = n_bad = 0;
    const unsigned lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned base = 0, ign = 0, bad = 0;
    for (unsigned long long at = 0; at < q.n; at += kThreads * kLabels) {
        const unsigned long long t0 = at + threadIdx.x;
        long long y[kLabels];
        unsigned before[kLabels], keep = 0;
#pragma unroll
        for (int i = 0; i < kLabels; ++i) y[i] = t0 + i * kThreads < q.n ? q.labels[t0 + i * kThreads] : q.ignore;
#pragma unroll
        for (int i = 0; i < kLabels; ++i) {
            const bool k = y[i] != q.ignore && y[i] >= 0 && y[i] < (long long)q.n_classes;
            const unsigned m = __ballot_sync(0xffffffffu, k);
            before[i] = __popc(m & ((1u << lane) - 1u));
            if (lane == 0) sh[i * kWarps + warp] = __popc(m);
            keep |= (unsigned)k << i;
            if (k || t0 + i * kThreads >= q.n) continue;
            if (y[i] == q.ignore) ++ign;
            else ++bad;
            if (kWrite) q.row_loss[t0 + i * kThreads] = 0.f;
            pos[t0 + i * kThreads] = kNone;
        }
        __syncthreads();
        if (warp == 0) {  // counts become sums of what is before them
            constexpr int kEach = kCounts / 32;
            unsigned c[kEach], sum = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                c[i] = sh[lane * kEach + i];
                sum += c[i];
            }
            unsigned scan = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned v = __shfl_up_sync(0xffffffffu, scan, o);
                if (lane >= o) scan += v;
            }
            if (lane == 31) total = scan;
            scan -= sum;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                sh[lane * kEach + i] = scan;
                scan += c[i];
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLabels; ++i) {
            if (!(keep >> i & 1u)) continue;
            const unsigned r = base + sh[i * kWarps + warp] + before[i];
            if (kWrite) {
                q.row_of[r] = (unsigned)(t0 + i * kThreads);
                q.label[r] = (int)y[i];
            }
            pos[t0 + i * kThreads] = r;
        }
        base += total;
        __syncthreads();
    }
    __syncthreads();
    if (kWrite) {
        if (ign) atomicAdd(&n_ign, ign);
        if (bad) atomicAdd(&n_bad, bad);
        __syncthreads();
        if (threadIdx.x == 0) {
            q.rec->rows = base;
            q.rec->ignored = n_ign;
            q.rec->bad = n_bad;
            q.rec->error = q.error;
            q.rec->done = 0;
            q.rec->loss = 0.f;
            if (q.d_loss && q.n == 0) *q.d_loss = 0.f;
        }
    }
    return base;
}
__global__ void __launch_bounds__(kRowThreads) k_xent_rows(RowList q) {
    griddep_start();
    list_rows<kRowThreads, true>(q, q.pos);
}

union Eight {
    uint4 u;
    __nv_bfloat16 b[8];
    __half h[8];
    unsigned short s[8];
};

// x = p0 + p1 + p2, each the bfloat16 next to what is left.  A finite value above the largest bfloat16 is cut, not
// rounded to infinity; an infinity or a NaN stays in p0.
__device__ __forceinline__ void split3(float x, __nv_bfloat16 &p0, __nv_bfloat16 &p1, __nv_bfloat16 &p2) {
    p0 = __float2bfloat16_rn(x);
    if (!isfinite(__bfloat162float(p0))) {
        p0 = __float2bfloat16_rz(x);
        if (!isfinite(x)) {
            p0 = __float2bfloat16_rn(x);
            p1 = p2 = __float2bfloat16_rn(0.f);
            return;
        }
    }
    const float r1 = x - __bfloat162float(p0);
    p1 = __float2bfloat16_rn(r1);
    p2 = __float2bfloat16_rn(r1 - __bfloat162float(p1));
}

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

// Rows and where they are copied to in the layout the products read: rows of dp elements (zeros behind the last),
// 16-byte aligned, one plane for the 16-bit types and three for float32.
template <typename T> struct Copy {
    const T *src;
    unsigned long long pitch;
    unsigned n;
    bool vec;  // rows of src on 16-byte boundaries
    unsigned short *dst;
    unsigned long long plane;
};
// Eight elements from column c of row r to row `to`.
template <typename T> __device__ __forceinline__ void copy_eight(const Copy<T> &q, unsigned r, unsigned to, unsigned c, unsigned d, unsigned dp) {
    const T *s = q.src + r * q.pitch + c;
    unsigned short *o = q.dst + (unsigned long long)to * dp + c;
    if constexpr (sizeof(T) == 2) {
        Eight x;
        const unsigned by = (unsigned)(uintptr_t)s & 15u;
        if (q.vec && c + 8 <= d) x.u = *reinterpret_cast<const uint4 *>(s);
        else if (c && c + 16 <= d) {  // the two aligned words that hold it lie within the row
            const uint4 *a = reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(s) - by);
            x.u = by ? shifted(a[0], a[1], by) : a[0];
        } else
            for (int j = 0; j < 8; ++j) x.s[j] = c + j < d ? reinterpret_cast<const unsigned short *>(s)[j] : (unsigned short)0;
        *reinterpret_cast<uint4 *>(o) = x.u;
    } else {
        float x[8];
        if (q.vec && c + 8 <= d) {
            const float4 a = *reinterpret_cast<const float4 *>(s), b = *reinterpret_cast<const float4 *>(s + 4);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
            x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
            for (int j = 0; j < 8; ++j) x[j] = c + j < d ? s[j] : 0.f;
        }
        Eight p[3];
#pragma unroll
        for (int j = 0; j < 8; ++j) split3(x[j], p[0].b[j], p[1].b[j], p[2].b[j]);
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4 *>(o + k * q.plane) = p[k].u;
    }
}

// Row t of h goes to pos[t]; rows that do not count are left out and their row of `zero` (dh) is cleared, and the rows
// behind the last one are zero up to a multiple of 64.  Then w, where it has to be copied.  SCAN: every CTA lists the rows
// itself (the first one for all to come), which for up to kScanRows of them takes less time than a launch, unless the copies
// are what takes the time (kScanGroups groups of eight elements: 16 MB of 16-bit values).  A call of 1000 classes, bfloat16,
// listed by every CTA / by a launch: 16 rows of 64 26.7 / 29.5 us, 2048 rows of 64 34.9 / 38.9, of 1024 44.0 / 45.0, of 8192 117 / 114.
constexpr unsigned kScanRows = 2048, kScanGroups = 1u << 20;
template <typename T, bool SCAN>
__global__ void __launch_bounds__(256)
k_xent_place(RowList q, Copy<T> h, Copy<T> w, unsigned d, unsigned dp, T *__restrict__ zero, unsigned long long zero_pitch) {
    __shared__ unsigned spos[SCAN ? kScanRows : 1];
    griddep_start();
    unsigned rows;
    if constexpr (SCAN) {
        static_assert(kScanRows == 256 * kLabels, "one round of labels");
        rows = blockIdx.x == 0 ? list_rows<256, true>(q, spos) : list_rows<256, false>(q, spos);
        __syncthreads();
    } else {
        rows = q.rec->rows;
    }
    const unsigned groups = dp / 8, pad = (rows + 63) / 64 * 64;
    const unsigned long long total = (unsigned long long)(h.n + 64u) * groups, step = (unsigned long long)gridDim.x * 256;
    unsigned long long i = (unsigned long long)blockIdx.x * 256 + threadIdx.x;
    for (; i < total; i += step) {
        const unsigned r = total >> 32 ? (unsigned)(i / groups) : (unsigned)i / groups;
        const unsigned c = (unsigned)(i - (unsigned long long)r * groups) * 8;
        if (r >= h.n) {
            const unsigned to = rows + (r - h.n);
            if (to < pad)
                for (int p = 0; p < (sizeof(T) == 4 ? 3 : 1); ++p) *reinterpret_cast<uint4 *>(h.dst + p * h.plane + (unsigned long long)to * dp + c) = make_uint4(0, 0, 0, 0);
            continue;
        }
        const unsigned to = SCAN ? spos[r] : q.pos[r];
        if (to != kNone) copy_eight(h, r, to, c, d, dp);
        else if (zero)
            for (unsigned j = 0; j < 8 && c + j < d; ++j) zero[r * zero_pitch + c + j] = from_f32<T>(0.f);
    }
    const unsigned long long more = (unsigned long long)w.n * groups;
    for (i -= total; i < more; i += step) {
        const unsigned r = more >> 32 ? (unsigned)(i / groups) : (unsigned)i / groups;
        copy_eight(w, r, r, (unsigned)(i - (unsigned long long)r * groups) * 8, d, dp);
    }
}

struct Piece {
    unsigned first, most;  // rows [first, min(first + most, rows)) of the compacted list
    __device__ unsigned rows(const XentRecord *rec) const {
        return rec->rows > first ? min(most, rec->rows - first) : 0u;
    }
};

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

// dz is rounded once to the operands' type, since the matrix instruction takes both operands in one type; the other way, two
// planes of it, would double the products' time.  Error of dh in the mean square against that of rounding the exact dh alone,
// 256 rows, 32000 classes: bfloat16 0.00187 / 0.00166, float16 2.47e-4 / 2.08e-4 (rounding the exact dz instead gives the same
// three digits: what the exponentials' 11 bits add does not show).
// What the products read as dz: bfloat16 as it is; float16 times 2^15 (|dz| <= 1, and a probability of 1e-6 would be
// next to float16's smallest step), taken out again by the products' scale.
constexpr float kDzF16 = 32768.f;

struct DzOut {
    unsigned short *dz;        // [planes][rows][pitch]
    unsigned long long pitch;  // classes rounded up to a multiple of 8
    unsigned long long plane;
    int dt;
};

// Ends every CTA of a softmax kernel; with `n` (the last piece of a call) the last CTA to get here adds up the call's row
// losses, in an order that depends on n alone.  The loss is NaN once a wait inside a product of the call has given up.
struct LossOut {
    const float *row_loss;
    unsigned n;
    bool mean;
    XentRecord *rec;
    float *d_loss;
};
__device__ __forceinline__ void finish_loss(const LossOut &o) {
    __shared__ double sh[8];
    __shared__ bool last;
    if (!o.n) return;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(&o.rec->done, 1u) == gridDim.x * gridDim.y - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double s = 0.0;
#pragma unroll 4
    for (unsigned t = threadIdx.x; t < o.n; t += 256) s += __ldcg(o.row_loss + t);
    for (int k = 16; k; k >>= 1) s += __shfl_xor_sync(0xffffffffu, s, k);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x) return;
    s = 0.0;
    for (int w = 0; w < 8; ++w) s += sh[w];
    o.rec->loss = __ldcg(&o.rec->error) ? __int_as_float(0x7fffffff) : (float)(o.mean ? s / (double)max(o.rec->rows, 1u) : s);
    if (o.d_loss) *o.d_loss = o.rec->loss;
}

// Maximum and sum over the NT threads of a row: a warp, or the CTA of 256.
template <int NT> __device__ __forceinline__ float row_max(float v, float *sh) {
    if constexpr (NT == 256) v = cta_max(v, sh);
    for (int o = NT == 256 ? 0 : 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
template <int NT> __device__ __forceinline__ float row_add(float v, float *sh) {
    if constexpr (NT == 256) v = cta_add(v, sh);
    for (int o = NT == 256 ? 0 : 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int NT> __device__ __forceinline__ void zero_row(const DzOut &o, unsigned short *row, unsigned tid) {
    for (int q = 0; q < (o.dt == SCAR_F32 ? 3 : 1); ++q)
        for (unsigned v = tid * 8; v < o.pitch; v += NT * 8) *reinterpret_cast<uint4 *>(row + q * o.plane + v) = make_uint4(0, 0, 0, 0);
}

// NT threads (the CTA of 256, or a warp of it) per row of the piece: join the row's groups of 128 classes to lse and the
// loss; with GRAD they turn the row's values into dz: scaled exponentials in place (z = nullptr), or float32 logits.  Rows
// behind the last one up to a multiple of 64 become zero (the dw product runs over whole groups of 64 rows).  Few long
// rows are cut into gridDim.y ranges of `span` classes, each of which joins the groups again.  Bound by HBM: 2 bytes (or
// 4) read and 2 (or 6) written per value.
template <bool GRAD, int NT>
__global__ void __launch_bounds__(256)
k_xent_dz(DzOut o, unsigned V, unsigned span, const float *__restrict__ z, const float2 *__restrict__ stat, unsigned groups, const int *__restrict__ label,
          const float *__restrict__ label_z, const unsigned *__restrict__ row_of, Piece p, float *row_loss, LossOut loss) {
    __shared__ float sh[8];
    griddep_start();
    const unsigned r = blockIdx.x * (256 / NT) + threadIdx.x / NT, tid = threadIdx.x % NT, R = p.rows(loss.rec);
    const float2 *st = stat + (unsigned long long)r * groups;
    float lse = 0.f, zl = 0.f;
    if (r < R) {
        float top = -INFINITY, s = 0.f;
#pragma unroll 4
        for (unsigned i = tid; i < groups; i += NT) {
            const float2 e = st[i];
            top = fmaxf(top, e.y > 0.f ? e.x : -INFINITY);
        }
        top = row_max<NT>(top, sh);
#pragma unroll 4
        for (unsigned i = tid; i < groups; i += NT) {
            const float2 e = st[i];
            if (e.y != 0.f) s = fmaf(e.y, expf(e.x - top), s);  // a NaN sum goes through
        }
        s = row_add<NT>(s, sh);
        lse = top + logf(s * (1.f / kProbScale));
        zl = label_z[p.first + r];
        if (tid == 0 && blockIdx.y == 0) row_loss[row_of[p.first + r]] = lse - zl;
    }
    finish_loss(loss);
    if (!GRAD) return;
    unsigned short *row = o.dz + (unsigned long long)r * o.pitch;
    const unsigned from = blockIdx.y * span;
    if (r >= R) {
        if (r < (R + 63) / 64 * 64 && from == 0) zero_row<NT>(o, row, tid);
        return;
    }
    const unsigned y = (unsigned)label[p.first + r], to = V - from > span ? from + span : V;
    const float held = o.dt == SCAR_F16 ? kDzF16 : 1.f;
    if (o.dt == SCAR_F32) {
        const float *zr = z + (unsigned long long)r * o.pitch;
#pragma unroll 2
        for (unsigned v = from + tid * 8; v < to; v += NT * 8) {
            const float4 a = __ldcs(reinterpret_cast<const float4 *>(zr + v)), b = __ldcs(reinterpret_cast<const float4 *>(zr + v + 4));
            const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            Eight w[3];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = v + j < V ? (v + j == y ? expm1f(zl - lse) : expf(x[j] - lse)) : 0.f;
                split3(d, w[0].b[j], w[1].b[j], w[2].b[j]);
            }
#pragma unroll
            for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4 *>(row + q * o.plane + v) = w[q].u;
        }
        return;
    }
    constexpr int kBatch = 4;  // 16-byte loads of a thread in flight
    for (unsigned v0 = from + tid * 8; v0 < to; v0 += kBatch * NT * 8) {
        Eight x[kBatch];
        float2 e[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const unsigned v = v0 + i * NT * 8;
            if (v >= to) break;
            x[i].u = __ldcs(reinterpret_cast<const uint4 *>(row + v));
            e[i] = st[v >> 7];
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const unsigned v = v0 + i * NT * 8;
            if (v >= to) break;
            const float f = e[i].y != 0.f ? expf(e[i].x - lse) * (held / kProbScale) : 0.f;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float2 w = __half22float2(*reinterpret_cast<const __half2 *>(x[i].h + j));
                if (o.dt == SCAR_F16) *reinterpret_cast<__half2 *>(x[i].h + j) = __floats2half2_rn(w.x * f, w.y * f);
                else *reinterpret_cast<__nv_bfloat162 *>(x[i].b + j) = __floats2bfloat162_rn(w.x * f, w.y * f);
            }
            *reinterpret_cast<uint4 *>(row + v) = x[i].u;
        }
    }
    // the label's value, from its exact logit, by the thread that has just written what was there
    if (y >= from && y < to && (y - from) / 8 % NT == tid) {
        const float d = expm1f(zl - lse) * held;
        if (o.dt == SCAR_F16) reinterpret_cast<__half *>(row)[y] = __float2half_rn(d);
        else reinterpret_cast<__nv_bfloat16 *>(row)[y] = __float2bfloat16_rn(d);
    }
}

// The same from logits whose sum over k was split (their sum replaces the first part): one pass for the running maximum
// and sum of every thread, one for dz.
template <bool GRAD, int NT>
__global__ void __launch_bounds__(256)
k_xent_softmax(const __grid_constant__ TcArgs g, DzOut o, const int *__restrict__ label, const unsigned *__restrict__ row_of, float *row_loss, LossOut loss) {
    __shared__ float sh[8];
    griddep_start();
    const unsigned r = blockIdx.x * (256 / NT) + threadIdx.x / NT, tid = threadIdx.x % NT, R = rows_of(g), V = g.n, pitch = (V + 7) & ~7u;
    const unsigned splits = parts_of(g);
    const unsigned long long stride = (unsigned long long)g.m * pitch;
    float *z = g.part + (unsigned long long)r * pitch;
    float lse = 0.f, zl = 0.f;
    unsigned y = 0;
    if (r < R) {
        float top = -INFINITY, s = 0.f;
#pragma unroll 2
        for (unsigned v = tid * 4; v < V; v += NT * 4) {
            float4 a = *reinterpret_cast<const float4 *>(z + v);
            if (splits > 1) {
#pragma unroll 4
                for (unsigned q = 1; q < splits; ++q) {
                    const float4 b = *reinterpret_cast<const float4 *>(z + q * stride + v);
                    a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
                }
                *reinterpret_cast<float4 *>(z + v) = a;
            }
            const float x[4] = {a.x, v + 1 < V ? a.y : -INFINITY, v + 2 < V ? a.z : -INFINITY, v + 3 < V ? a.w : -INFINITY};
            const float t = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
            if (t > top) {
                s *= expf(top - t);
                top = t;
            }
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int i = 0; i < 4; ++i) s += expf(x[i] - ref);
        }
        const float all = row_max<NT>(top, sh);
        const float ref = all == -INFINITY ? 0.f : all;
        s = row_add<NT>(s != 0.f ? s * expf((top == -INFINITY ? 0.f : top) - ref) : 0.f, sh);
        lse = ref + logf(s);
        y = (unsigned)label[g.first + r];
        __syncwarp();
        zl = z[y];
        if (tid == 0) row_loss[row_of[g.first + r]] = lse - zl;
    }
    finish_loss(loss);
    if (!GRAD) return;
    unsigned short *row = o.dz + (unsigned long long)r * o.pitch;
    if (r >= R) {
        if (r < (R + 63) / 64 * 64) zero_row<NT>(o, row, tid);
        return;
    }
    const float held = o.dt == SCAR_F16 ? kDzF16 : 1.f;
#pragma unroll 2
    for (unsigned v = tid * 8; v < V; v += NT * 8) {
        const float4 a = *reinterpret_cast<const float4 *>(z + v), b = *reinterpret_cast<const float4 *>(z + v + 4);
        const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        Eight w[3];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float d = 0.f;
            if (v + j < V) d = (v + j == y ? expm1f(zl - lse) : expf(x[j] - lse)) * held;
            if (o.dt == SCAR_F32) split3(d, w[0].b[j], w[1].b[j], w[2].b[j]);
            else if (o.dt == SCAR_F16) w[0].h[j] = __float2half_rn(d);
            else w[0].b[j] = __float2bfloat16_rn(d);
        }
        for (int q = 0; q < (o.dt == SCAR_F32 ? 3 : 1); ++q) *reinterpret_cast<uint4 *>(row + q * o.plane + v) = w[q].u;
    }
}

// Adds the parts of a split product and does what the product's own epilogue does without a split.
__global__ void __launch_bounds__(128)
k_xent_combine(const __grid_constant__ TcArgs g) {
    griddep_start();
    const unsigned m = g.dyn == 0 ? rows_of(g) : g.m;
    const unsigned groups = (g.n + 3) / 4, pitch = (g.n + 7) & ~7u, splits = parts_of(g);
    const float f = g.mean ? g.scale / (float)max(*g.rows, 1u) : g.scale;
    const unsigned long long stride = (unsigned long long)g.m * pitch, total = (unsigned long long)m * groups;
    for (unsigned long long i = (unsigned long long)blockIdx.x * 128 + threadIdx.x; i < total; i += (unsigned long long)gridDim.x * 128) {
        const unsigned row = total >> 32 ? (unsigned)(i / groups) : (unsigned)i / groups;
        const unsigned col = (unsigned)(i - (unsigned long long)row * groups) * 4;
        const float *p = g.part + (unsigned long long)row * pitch + col;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (unsigned s = 0; s < splits; ++s) {
            const float4 a = *reinterpret_cast<const float4 *>(p + s * stride);
            x.x += a.x; x.y += a.y; x.z += a.z; x.w += a.w;
        }
        store_out4(g, x, row, g.row_map ? g.row_map[g.first + row] : row, col, f);
    }
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// A 16-bit matrix as the products read it: `planes` of rows x inner, rows `pitch` elements apart.
struct Operand {
    const void *p;
    uint64_t inner, rows, pitch, planes, plane;
};

}  // namespace

struct scar_xent {
    int device = 0;
    cudaStream_t stream = nullptr;
    scar_xent_config cfg{};
    EncodeTiled encode = nullptr;
    unsigned pairs = 74;       // CTA pairs the GPU holds at a time
    unsigned planes = 1;
    unsigned piece = 0;        // rows per piece, a multiple of 64
    uint64_t vp = 0, dp = 0;   // classes and dim, rounded up to a multiple of 8
    uint64_t h_rows = 0;
    unsigned groups = 0;       // groups of 128 classes, two per tile
    unsigned *row_of = nullptr, *pos = nullptr;
    int *label = nullptr;
    float *label_z = nullptr, *row_loss = nullptr;
    unsigned short *h = nullptr;   // compacted h
    unsigned short *w = nullptr;   // w in planes, or copied to 16-byte rows (allocated by the first call that needs it)
    unsigned short *dz = nullptr;  // the piece's exponentials, then dz
    float2 *stat = nullptr;
    float *part = nullptr;         // float32 logits of the piece, or parts of split products
    uint64_t part_bytes = 0;
    float *acc = nullptr;
    XentRecord *rec = nullptr;
    // tensor maps of the workspaces: h as rows (128 a box) and as columns, dz likewise and as a result, w's copy
    CUtensorMap h_rows_map, h_cols_map, dz_rows_map, dz_cols_map, dz_out_map, w_rows_map, w_cols_map;
    std::vector<void *> owned;
    uint64_t bytes = 0;
    uint64_t launches = 0;
    bool ran = false, failed = false, have_w_maps = false;
    bool arm_error = false;  // the next call reports a wait that gave up
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

constexpr uint64_t kPitchEnd = 1ull << 38;  // a tensor map's row is shorter than 2^40 bytes
int check_call(const scar_xent *op, const void *h, uint64_t hp, const void *w, uint64_t wp, const int64_t *labels,
               uint64_t n, const float *row_loss, const float *loss) {
    if (!op || !w) return SCAR_ERR_INVALID_ARG;
    const unsigned b = elem_size(op->cfg.dtype);
    if (n > op->cfg.max_tokens) return SCAR_ERR_CAPACITY;
    if (n && (!h || !labels)) return SCAR_ERR_INVALID_ARG;
    if (hp < op->cfg.dim || wp < op->cfg.dim || hp >= kPitchEnd || wp >= kPitchEnd) return SCAR_ERR_INVALID_ARG;
    if ((uintptr_t)h % b || (uintptr_t)w % b || (uintptr_t)labels % 8 || (uintptr_t)row_loss % 4 || (uintptr_t)loss % 4)
        return SCAR_ERR_INVALID_ARG;
    return check_current_device(op->device);
}

bool rows_aligned(const void *p, uint64_t pitch, unsigned elem) { return (uintptr_t)p % 16 == 0 && pitch * elem % 16 == 0; }

// The tensor map of an operand: boxes of 64 values of k by box_rows rows (K-major), or of 64 of its own dimension by 64
// values of k (MN-major; box_rows = 64); or of a result: boxes of 128 bytes (float32) or 64 (16-bit types) by 32 rows.
int make_map(const scar_xent *op, CUtensorMap *map, const Operand &x, unsigned box_rows, unsigned elem = 2, unsigned box_bytes = 128) {
    const cuuint64_t dims[3] = {x.inner, x.rows, x.planes}, strides[2] = {x.pitch * elem, (x.planes > 1 ? x.plane : x.pitch) * elem};
    const cuuint32_t box[3] = {box_bytes / elem, box_rows, 1}, step[3] = {1, 1, 1};
    const CUtensorMapDataType type = elem == 4                      ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                     : op->cfg.dtype == SCAR_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                                 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const CUresult rc = op->encode(map, type, 3, const_cast<void *>(x.p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, box_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? SCAR_OK : SCAR_ERR_CUDA;
}

// A 16-bit or float32 matrix from rows on 16-byte boundaries to rows anywhere, a warp per row: whole 16-byte words of the
// destination, its ends element by element.
template <typename T>
__global__ void __launch_bounds__(256)
k_xent_unplace(const T *__restrict__ src, unsigned long long src_pitch, unsigned n, unsigned d, T *__restrict__ dst, unsigned long long pitch) {
    griddep_start();
    constexpr unsigned kVec = 16 / sizeof(T);
    const unsigned lane = threadIdx.x & 31;
    for (unsigned long long r = blockIdx.x * 8ull + (threadIdx.x >> 5); r < n; r += gridDim.x * 8ull) {
        const T *s = src + r * src_pitch;
        T *o = dst + r * pitch;
        const unsigned head = min(d, (unsigned)((0u - (unsigned)(uintptr_t)o) & 15u) / (unsigned)sizeof(T)), words = (d - head) / kVec, tail = head + words * kVec;
        if (lane < head) o[lane] = s[lane];
        if (tail + lane < d) o[tail + lane] = s[tail + lane];
        const uint4 *a = reinterpret_cast<const uint4 *>(s);  // head is shorter than a word: word w lies in a[w] and a[w + 1]
#pragma unroll 4
        for (unsigned w = lane; w < words; w += 32)
            *reinterpret_cast<uint4 *>(o + head + w * kVec) = head ? shifted(a[w], a[w + 1], head * (unsigned)sizeof(T)) : a[w];
    }
}

// Maps of the operator's own buffers, made once.
int map_workspaces(scar_xent *op) {
    const uint64_t V = op->cfg.n_classes, D = op->cfg.dim;
    const Operand oh{op->h, D, op->h_rows, op->dp, op->planes, op->h_rows * op->dp};
    const Operand oz{op->dz, V, op->piece, op->vp, op->planes, (uint64_t)op->piece * op->vp};
    int rc;
    if ((rc = make_map(op, &op->h_rows_map, oh, 128)) != SCAR_OK || (rc = make_map(op, &op->h_cols_map, oh, 64)) != SCAR_OK) return rc;
    if (!op->dz) return SCAR_OK;
    if ((rc = make_map(op, &op->dz_rows_map, oz, 128)) != SCAR_OK || (rc = make_map(op, &op->dz_cols_map, oz, 64)) != SCAR_OK) return rc;
    return make_map(op, &op->dz_out_map, oz, 32, 2, 64);
}
int map_w_copy(scar_xent *op) {
    const uint64_t V = op->cfg.n_classes, D = op->cfg.dim;
    const Operand ow{op->w, D, V, op->dp, op->planes, V * op->dp};
    int rc;
    if ((rc = make_map(op, &op->w_rows_map, ow, kBN / 2)) != SCAR_OK || (rc = make_map(op, &op->w_cols_map, ow, 64)) != SCAR_OK) return rc;
    op->have_w_maps = true;
    return SCAR_OK;
}

// Launches a kernel of the call's chain: it may start while the one before it still runs (griddep_start waits for it).
template <typename... P, typename... A> void launch(scar_xent *op, void (*kernel)(P...), dim3 grid, unsigned threads, unsigned smem, A... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = threads;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = op->stream;
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, P(args)...) == cudaSuccess) op->launches++;
    else op->failed = true;
}

// Sets the product's `splits`: 1, or more than 1 where cutting the sum over k pays for all the rows the call has.  Returns
// what it costs, in units of 64 values of k.
float choose_splits(const scar_xent *op, TcArgs &g, float join_s) {
    const uint64_t part = (uint64_t)g.m * round_up(g.n, 8) * 4;
    g.pairs = op->pairs;
    g.planes = op->planes;
    g.join_s = join_s;
    g.most_splits = (unsigned)std::min<uint64_t>(kMostSplits, std::max<uint64_t>(1, part ? op->part_bytes / part : 1));
    g.splits = 1;
    const unsigned kb = (g.k + kBK - 1) / kBK;
    const uint64_t tiles = (uint64_t)((g.m + kBM - 1) / kBM) * ((g.n + kBN - 1) / kBN);
    float best = split_cost(1, tiles, kb, op->pairs, 0.f, join_s, op->planes);
    for (unsigned s = 2; s <= g.most_splits && s <= kb; ++s) {
        const float cost = split_cost(s, tiles, kb, op->pairs, (float)g.m * (float)g.n * 4.f, join_s, op->planes);
        if (cost < best) {
            best = cost;
            g.splits = s;
        }
    }
    return best;
}

uint64_t tiles_of(const TcArgs &g) { return (uint64_t)((g.m + kBM - 1) / kBM) * ((g.n + kBN - 1) / kBN) * (g.splits > 1 ? g.most_splits : 1); }

template <int PL, bool A_MN, bool B_MN, Epi EPI> void launch_tc(scar_xent *op, TcArgs g) {
    if (EPI == Epi::kPart) {
        const uint64_t pitch = round_up(g.n, 8);
        if (make_map(op, &g.c, {g.part, pitch, g.m, pitch, g.splits > 1 ? g.most_splits : 1u, g.m * pitch}, 32, 4) != SCAR_OK) op->failed = true;
    }
    const unsigned pairs = (unsigned)std::min<uint64_t>(tiles_of(g), op->pairs);
    if (pairs) launch(op, k_tc_gemm<PL, A_MN, B_MN, EPI, 1>, 2 * pairs, kGemmThreads, kTcSmem, TcSet<1>{g});
}

template <typename K> bool allow_smem(K kernel) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kTcSmem) == cudaSuccess;
}
template <int PL> bool allow_smem_all() {
    return allow_smem(k_tc_gemm<PL, false, false, Epi::kPart, 1>) && allow_smem(k_tc_gemm<PL, false, true, Epi::kPart, 1>) &&
           allow_smem(k_tc_gemm<PL, true, true, Epi::kPart, 1>) && allow_smem(k_tc_gemm<PL, false, true, Epi::kOut, 1>) &&
           allow_smem(k_tc_gemm<PL, true, true, Epi::kOut, 1>) && allow_smem(k_tc_gemm<PL, false, true, Epi::kOut, 2>);
}

// A product that ends in an output, its sum over k split or not.
template <int PL, bool A_MN> void launch_out(scar_xent *op, const TcArgs &g) {
    if (g.splits == 1) {
        launch_tc<PL, A_MN, true, Epi::kOut>(op, g);
        return;
    }
    launch_tc<PL, A_MN, true, Epi::kPart>(op, g);
    const uint64_t todo = (uint64_t)g.m * ((g.n + 3) / 4);
    launch(op, k_xent_combine, (unsigned)std::min<uint64_t>((todo + 127) / 128, 32 * op->pairs), 128, 0, g);
}

// dh and dw of a piece: one launch without splits, so that the second one's tiles fill the last round of the first one's
// (4096 x 32000 x 2048: 120 tiles of 500 stages leave 28 of 74 pairs idle for half of that time), unless split products
// with launches of their own are worth it (a dh of few tiles whose sum runs over very many classes).  Not where dw goes through the room of w's copy, which dh still reads.
template <int PL> void launch_grads(scar_xent *op, TcArgs dhg, TcArgs dwg, bool through_w) {
    const float apart = choose_splits(op, dhg, kLaunchS) + choose_splits(op, dwg, kLaunchS) + kLaunchS / unit_s(PL);
    const unsigned pairs = op->pairs;
    const float tile0 = (float)((dhg.k + kBK - 1) / kBK + 4), tile1 = (float)((dwg.k + kBK - 1) / kBK + 4);
    const uint64_t tiles0 = (uint64_t)((dhg.m + kBM - 1) / kBM) * ((dhg.n + kBN - 1) / kBN), tiles1 = (uint64_t)((dwg.m + kBM - 1) / kBM) * ((dwg.n + kBN - 1) / kBN);
    // the second one's tiles fill gaps where they are the shorter ones, and come on top where they are not
    const float together = tile1 <= tile0 ? std::max(tile0, ((float)tiles0 * tile0 + (float)tiles1 * tile1) / (float)pairs)
                                          : (float)((tiles0 + pairs - 1) / pairs) * tile0 + (float)((tiles1 + pairs - 1) / pairs) * tile1;
    if (!through_w && together <= apart) {
        dhg.splits = dwg.splits = 1;
        launch(op, k_tc_gemm<PL, false, true, Epi::kOut, 2>, 2 * (unsigned)std::min<uint64_t>(tiles0 + tiles1, pairs), kGemmThreads, kTcSmem, TcSet<2>{{dhg, dwg}});
        return;
    }
    launch_out<PL, false>(op, dhg);
    launch_out<PL, true>(op, dwg);
}

template <typename T>
int run_xent(scar_xent *op, const T *h, uint64_t hp, const T *w, uint64_t wp, const int64_t *labels, unsigned n, bool grad, float scale,
             float *row_loss, float *d_loss, T *dh, uint64_t dhp, T *dw, uint64_t dwp) {
    constexpr int PL = sizeof(T) == 4 ? 3 : 1;
    const unsigned V = (unsigned)op->cfg.n_classes, D = (unsigned)op->cfg.dim;
    const bool mean = op->cfg.reduction == SCAR_MEAN;
    const long long *y = reinterpret_cast<const long long *>(labels);
    int rc;
    if (!row_loss) row_loss = op->row_loss;

    // w in place where its rows lie on 16-byte boundaries, else (and in float32 always) through a copy of its own
    const bool w_copied = PL == 3 || !rows_aligned(w, wp, sizeof(T));
    if (w_copied && !op->w && (rc = xent_alloc(op, &op->w, (uint64_t)PL * V * op->dp * 2)) != SCAR_OK) return rc;
    TcArgs logits{}, dhg{}, dwg{};
    logits.a = op->h_rows_map;
    dwg.b = op->h_cols_map;
    dhg.a = op->dz_rows_map;
    dwg.a = op->dz_cols_map;
    logits.c = op->dz_out_map;
    if (w_copied) {
        if (!op->have_w_maps && (rc = map_w_copy(op)) != SCAR_OK) return rc;
        logits.b = op->w_rows_map;
        dhg.b = op->w_cols_map;
    } else {
        const Operand ow{w, D, V, wp, 1, 0};
        if ((rc = make_map(op, &logits.b, ow, kBN / 2)) != SCAR_OK || (grad && (rc = make_map(op, &dhg.b, ow, 64)) != SCAR_OK)) return rc;
    }

    const RowList list{y, n, op->cfg.ignore_label, V, op->row_of, op->pos, op->label, row_loss, op->rec, d_loss, op->arm_error ? 1u : 0u};
    op->arm_error = false;
    const Copy<T> ch{h, hp, n, rows_aligned(h, hp, sizeof(T)), op->h, op->h_rows * op->dp};
    const Copy<T> cw{w, wp, w_copied ? V : 0u, rows_aligned(w, wp, sizeof(T)), op->w, (uint64_t)V * op->dp};
    const uint64_t groups = ((uint64_t)n + 64 + cw.n) * (op->dp / 8);
    const unsigned place_ctas = (unsigned)std::min<uint64_t>((groups + 255) / 256, 16 * op->pairs);
    if (n <= kScanRows && groups <= kScanGroups) {
        launch(op, k_xent_place<T, true>, place_ctas, 256, 0, list, ch, cw, D, (unsigned)op->dp, grad ? dh : nullptr, dhp);
    } else {
        launch(op, k_xent_rows, 1, kRowThreads, 0, list);
        launch(op, k_xent_place<T, false>, place_ctas, 256, 0, list, ch, cw, D, (unsigned)op->dp, grad ? dh : nullptr, dhp);
    }

    TcArgs base{};
    base.rows = &op->rec->rows;
    base.error = &op->rec->error;
    base.chosen = &op->rec->splits;
    base.loss[0] = &op->rec->loss;
    base.loss[1] = d_loss;
    base.bf16 = op->cfg.dtype != SCAR_F16;
    base.part = op->part;
    base.out_type = op->cfg.dtype;
    base.mean = mean;
    base.scale = op->cfg.dtype == SCAR_F16 ? scale / kDzF16 : scale;
    auto fill = [&](TcArgs &g, unsigned m, unsigned nn, unsigned k, int dyn) {
        const CUtensorMap a = g.a, b = g.b, c = g.c;
        g = base;
        g.a = a;
        g.b = b;
        g.c = c;
        g.m = m;
        g.n = nn;
        g.k = k;
        g.dyn = dyn;
        g.n_fast = nn < m;
        g.splits = 1;
    };
    for (unsigned at = 0; at == 0 || at < n; at += op->piece) {
        const unsigned rows = std::min(op->piece, n - at), rows64 = (rows + 63) / 64 * 64;
        const Piece p{at, op->piece};
        base.first = at;
        base.most = op->piece;
        const DzOut dz{op->dz, op->vp, (uint64_t)op->piece * op->vp, op->cfg.dtype};
        const LossOut loss{row_loss, (uint64_t)at + op->piece >= n ? n : 0u, mean, op->rec, d_loss};
        if (rows) {
            fill(logits, rows, V, D, 0);
            logits.a_row0 = at;
            logits.stat_pitch = op->groups;
            logits.label = op->label;
            logits.label_z = op->label_z;
            choose_splits(op, logits, kLaunchS);  // the softmax of parts takes about that much longer
            logits.stat = logits.splits == 1 ? op->stat : nullptr;
            const bool many = rows >= 16 * op->pairs;
            const uint64_t row_bytes = (uint64_t)V * (PL == 3 ? 4 : 2);
            const bool short_rows = (many && row_bytes <= kWarpRowBytes) || (rows >= 64 * op->pairs && row_bytes <= 4 * kWarpRowBytes);
            if (logits.splits > 1) {
                launch_tc<PL, false, false, Epi::kPart>(op, logits);
                auto kernel = short_rows ? (grad ? k_xent_softmax<true, 32> : k_xent_softmax<false, 32>) : (grad ? k_xent_softmax<true, 256> : k_xent_softmax<false, 256>);
                launch(op, kernel, dim3(short_rows ? (rows64 + 7) / 8 : rows64), 256, 0, logits, dz, op->label, op->row_of, row_loss, loss);
            } else {
                if constexpr (PL == 3) launch_tc<3, false, false, Epi::kPart>(op, logits);
                else if (grad) launch_tc<1, false, false, Epi::kProb>(op, logits);
                else launch_tc<1, false, false, Epi::kStat>(op, logits);
                // The loss alone reads a row's groups of 128 classes only.  Warp / CTA, bfloat16: 1184 rows of 8192 classes
                // 22.6 / 22.6 us, of 32000 43.1 / 39.0; 3000 rows of 16000 51.3 / 55.4, of 64000 142 / 140; 8192 rows of 32000 177 / 193.
                const bool warps = short_rows || (many && !grad && V <= 8ull * rows);
                // Few long rows: ranges of at least 4096 classes, for about four CTAs per SM.  Cut / whole, 128000 classes: 8 rows
                // 101 / 113 us, float32 261 / 325; 64000 classes: 200 rows (two ranges) 74.3 / 79.8, float32 191 / 223; 600 rows 132 / 135,
                // 335 / 338; of 8192 classes 48.3 / 45.9.
                const unsigned ranges = grad && !warps ? std::max(1u, std::min(V / 4096u, 8 * op->pairs / std::max(rows, 1u))) : 1u;
                const unsigned span = (unsigned)round_up((V + ranges - 1) / ranges, 2048);
                auto kernel = warps ? (grad ? k_xent_dz<true, 32> : k_xent_dz<false, 32>) : (grad ? k_xent_dz<true, 256> : k_xent_dz<false, 256>);
                launch(op, kernel, dim3(warps ? (rows64 + 7) / 8 : rows64, (V + span - 1) / span), 256, 0, dz, V, span, op->part, op->stat, op->groups, op->label,
                       op->label_z, op->row_of, p, row_loss, loss);
            }
        }
        if (!grad) continue;
        if (rows) {
            fill(dhg, rows, D, V, 0);
            dhg.out = dh;
            dhg.out_pitch = dhp;
            dhg.out_vec = rows_aligned(dh, dhp, sizeof(T));
            dhg.row_map = op->row_of;
        }
        fill(dwg, V, D, rows, 1);
        dwg.b_row0 = at;
        dwg.out = dw;
        dwg.out_pitch = dwp;
        dwg.out_vec = rows_aligned(dw, dwp, sizeof(T));
        if (n > op->piece) {  // several pieces: their sums in float32, in dw itself when it is float32
            dwg.acc = PL == 3 ? reinterpret_cast<float *>(dw) : op->acc;
            dwg.acc_pitch = PL == 3 ? dwp : op->dp;
            dwg.acc_vec = PL == 3 ? dwg.out_vec : 1;
            dwg.acc_first = at == 0;
            dwg.acc_last = at + (uint64_t)op->piece >= n;
        }
        // Rows of dw that do not lie on 16-byte boundaries would be stored in pieces of lines, at a tenth of the rate: they go
        // through the room of w's copy, which is done with by now, and from there to their places.  A tensor map's store
        // clips rows to whole 16-byte words only, so rows of a length between two go the epilogue's own way.
        const bool through_w = !dwg.acc && !dwg.out_vec && w_copied;
        if (through_w) {
            dwg.out = op->w;
            dwg.out_pitch = op->dp;
            dwg.out_vec = 1;
        }
        dwg.c_map = !dwg.acc && (through_w || (dwg.out_vec && D * sizeof(T) % 16 == 0));
        if (dwg.c_map && (rc = make_map(op, &dwg.c, {dwg.out, D, V, dwg.out_pitch, 1, 0}, 32, sizeof(T), PL == 1 ? 64 : 128)) != SCAR_OK) return rc;
        if (rows) {
            launch_grads<PL>(op, dhg, dwg, through_w);
        } else {
            choose_splits(op, dwg, kLaunchS);
            launch_out<PL, true>(op, dwg);
        }
        if (through_w)
            launch(op, k_xent_unplace<T>, (unsigned)std::min<uint64_t>((V + 7) / 8, 16 * op->pairs), 256, 0, reinterpret_cast<const T *>(op->w), op->dp, V, D, dw, dwp);
        if ((uint64_t)at + op->piece >= n) break;
    }
    if (op->failed) {
        op->failed = false;
        cudaGetLastError();
        return SCAR_ERR_CUDA;
    }
    return SCAR_OK;
}

int call(scar_xent *op, const void *h, uint64_t hp, const void *w, uint64_t wp, const int64_t *labels, uint64_t n,
         bool grad, float scale, float *row_loss, float *d_loss, void *dh, uint64_t dhp, void *dw, uint64_t dwp) {
    int rc = SCAR_OK;
    try {
        dispatch_operand(op->cfg.dtype, [&](auto e) {
            using T = decltype(e);
            rc = run_xent<T>(op, static_cast<const T *>(h), hp, static_cast<const T *>(w), wp, labels, (unsigned)n, grad, scale,
                             row_loss, d_loss, static_cast<T *>(dh), dhp, static_cast<T *>(dw), dwp);
        });
    } catch (...) {
        rc = SCAR_ERR_ALLOC;
    }
    if (rc != SCAR_OK) return rc;
    TRAIN_TRY(cudaGetLastError());
    op->ran = true;
    return SCAR_OK;
}

// Rows per piece and the workspaces that go by it.
int size_workspaces(scar_xent *op) {
    const scar_xent_config &c = op->cfg;
    const uint64_t V = c.n_classes, D = c.dim, T = std::max<uint64_t>(c.max_tokens, 1);
    const bool f32 = c.dtype == SCAR_F32, grad = !c.loss_only;
    op->planes = f32 ? 3 : 1;
    op->vp = round_up(V, 8);
    op->dp = round_up(D, 8);
    op->groups = (unsigned)(2 * ((V + 255) / 256));
    const uint64_t limit = c.workspace_bytes ? c.workspace_bytes : 1ull << 30;
    const uint64_t row = 8ull * op->groups + (f32 ? 4 * op->vp : 0) + (grad ? 2 * op->planes * op->vp : 0);
    uint64_t piece = std::max<uint64_t>(limit / row / 256 * 256, 256);
    if (grad && !f32 && piece < T && (unsigned __int128)T * row <= (unsigned __int128)piece * row + V * D * 4) piece = T;
    op->piece = (unsigned)round_up(std::min(piece, T), 64);
    op->h_rows = round_up(T, 64);
    // parts of split products: as many as choose_splits may ask for, up to 64 MiB
    const uint64_t P = std::min<uint64_t>(op->piece, T);
    uint64_t most = P * op->vp;
    if (grad) most = std::max(most, std::max(P * op->dp, V * op->dp));
    op->part_bytes = std::min<uint64_t>(64ull << 20, most * 4 * 32);
    if (f32) op->part_bytes = std::max(op->part_bytes, P * op->vp * 4);
    // all of it in one allocation: each one costs the caller a few hundred microseconds
    struct {
        void **p;
        uint64_t bytes;
    } const want[] = {
        {(void **)&op->row_of, 4 * T}, {(void **)&op->pos, 4 * T}, {(void **)&op->label, 4 * T}, {(void **)&op->label_z, 4 * T},
        {(void **)&op->row_loss, 4 * T}, {(void **)&op->rec, sizeof(XentRecord)}, {(void **)&op->h, op->planes * op->h_rows * op->dp * 2},
        {(void **)&op->stat, 8ull * op->groups * op->piece}, {(void **)&op->part, op->part_bytes},
        {(void **)&op->dz, grad ? op->planes * (uint64_t)op->piece * op->vp * 2 : 0},
        {(void **)&op->acc, grad && !f32 && op->piece < T ? V * op->dp * 4 : 0},
        {(void **)&op->w, f32 || D % 8 ? op->planes * V * op->dp * 2 : 0},
    };
    uint64_t total = 0;
    for (const auto &x : want) total += round_up(x.bytes, 256);
    char *block = nullptr;
    const int rc = xent_alloc(op, &block, total);
    if (rc != SCAR_OK) return rc;
    for (const auto &x : want)
        if (x.bytes) {
            *x.p = block;
            block += round_up(x.bytes, 256);
        }
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
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        TRAIN_TRY(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found));
        if (found != cudaDriverEntryPointSuccess || !fn) return SCAR_ERR_CUDA;
        op->encode = reinterpret_cast<EncodeTiled>(fn);
        if (cfg->dtype == SCAR_F32 ? !(allow_smem_all<3>())
                                   : !(allow_smem_all<1>() && allow_smem(k_tc_gemm<1, false, false, Epi::kProb, 1>) && allow_smem(k_tc_gemm<1, false, false, Epi::kStat, 1>)))
            return SCAR_ERR_CUDA;
        int sms = 0;
        TRAIN_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, op->device));
        op->pairs = std::max(1, sms / 2);
        int rc = size_workspaces(op);
        if (rc != SCAR_OK || (rc = map_workspaces(op)) != SCAR_OK) return rc;
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
    const int rc = check_call(op, d_h, h_pitch, d_w, w_pitch, d_labels, n_tokens, d_row_loss, d_loss);
    if (rc != SCAR_OK) return rc;
    return call(op, d_h, h_pitch, d_w, w_pitch, d_labels, n_tokens, false, 0.f, d_row_loss, d_loss, nullptr, 0, nullptr, 0);
}

int scar_xent_loss_grad(scar_xent *op, const void *d_h, uint64_t h_pitch, const void *d_w, uint64_t w_pitch,
                        const int64_t *d_labels, uint64_t n_tokens, float grad_scale, float *d_row_loss,
                        float *d_loss, void *d_dh, uint64_t dh_pitch, void *d_dw, uint64_t dw_pitch) {
    const int rc = check_call(op, d_h, h_pitch, d_w, w_pitch, d_labels, n_tokens, d_row_loss, d_loss);
    if (rc != SCAR_OK) return rc;
    const unsigned b = elem_size(op->cfg.dtype);
    if (op->cfg.loss_only) return SCAR_ERR_STATE;
    if (!d_dw || (n_tokens && !d_dh) || (uintptr_t)d_dh % b || (uintptr_t)d_dw % b) return SCAR_ERR_INVALID_ARG;
    if (dh_pitch < op->cfg.dim || dw_pitch < op->cfg.dim || dh_pitch >= kPitchEnd || dw_pitch >= kPitchEnd)
        return SCAR_ERR_INVALID_ARG;
    return call(op, d_h, h_pitch, d_w, w_pitch, d_labels, n_tokens, true, grad_scale, d_row_loss, d_loss, d_dh, dh_pitch,
                d_dw, dw_pitch);
}

int scar_xent_status(scar_xent *op, scar_xent_info *out) {
    if (!op || !out) return SCAR_ERR_INVALID_ARG;
    const int rc = check_current_device(op->device);
    if (rc != SCAR_OK) return rc;
    if (!op->ran) return SCAR_ERR_STATE;
    XentRecord rec;
    TRAIN_TRY(cudaMemcpyAsync(&rec, op->rec, sizeof(XentRecord), cudaMemcpyDeviceToHost, op->stream));
    TRAIN_TRY(cudaStreamSynchronize(op->stream));
    out->loss = rec.loss;
    out->rows = rec.rows;
    out->ignored = rec.ignored;
    out->bad = rec.bad;
    return rec.error ? SCAR_ERR_TIMEOUT : SCAR_OK;
}

int scar_xent_selftest_arm_timeout(scar_xent *op) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    op->arm_error = true;
    return SCAR_OK;
}

uint64_t scar_xent_workspace_bytes(const scar_xent *op) { return op ? op->bytes : 0; }
uint64_t scar_xent_launch_count(const scar_xent *op) { return op ? op->launches : 0; }

int scar_xent_destroy(scar_xent *op) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    const bool ok = cudaStreamSynchronize(op->stream) == cudaSuccess;
    for (void *p : op->owned) cudaFree(p);
    delete op;
    if (!ok) cudaGetLastError();
    return ok ? SCAR_OK : SCAR_ERR_CUDA;
}

}  // extern "C"
