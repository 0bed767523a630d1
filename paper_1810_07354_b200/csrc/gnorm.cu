// Global gradient norm over a list of tensors, and clipping (scar_gnorm_* of scar.h).
//
// The tensors are cut into pieces of kPieceBytes on the host, once, so that every piece but a tensor's first begins on a
// 16-byte boundary.  A CTA walks over pieces with a fixed stride: on one GPU, which CTA adds what depends on the lengths, the
// types and the addresses modulo 16 alone.  The last CTA to finish adds the CTAs' sums in their order: the result is the
// same bits every time.
// Bound by HBM: one read for the norm, one read and one write for the scaled values.  The second kernel is launched
// while the first runs (programmatic launch) and takes the pieces backwards, so that what the first read last is still
// in L2; it has one CTA per piece, started in order, because CTAs that walk over pieces drift apart and then read and
// write all over memory at once (a billion bfloat16 values: norm and scaling 901 us this way, 1077 with walking CTAs).
// The norm alone reads 400 MB in 62 us (6.45 TB/s); pieces of 16 KiB rather than 32 are for lists of short tensors
// (1200 tensors, 80 MB: 43.0 against 43.8 us).
#include <algorithm>
#include <new>
#include <vector>

#include "train_common.cuh"

using namespace scar;

namespace {

constexpr int kNormThreads = 256;
constexpr unsigned kPieceBytes = 16384;  // four 16-byte loads per thread, all in flight together
constexpr int kVecs = kPieceBytes / 16 / kNormThreads;
constexpr unsigned kCtasPerSm = 8;

struct Piece {
    const void *src;
    void *dst;
    unsigned n;   // elements
    int dtype;
};

struct NormRecord {
    double norm;
    double coef;
    unsigned long long nonfinite;
    unsigned long long alone;  // calls that one CTA had to finish (k_gnorm_clip)
};

// One term of the norm, and how two partial results join.
template <int KIND> __device__ __forceinline__ void add_term(float &a, float v) {
    if (KIND == SCAR_GNORM_L2) a = fmaf(v, v, a);
    else if (KIND == SCAR_GNORM_L1) a += fabsf(v);
    else a = (fabsf(v) > a || v != v) ? fabsf(v) : a;  // a NaN stays: nothing compares above it
}
template <int KIND, typename W> __device__ __forceinline__ W join(W a, W b) {
    if (KIND != SCAR_GNORM_MAX) return a + b;
    return (a != a) ? a : ((b > a || b != b) ? b : a);
}

template <int KIND> __device__ __forceinline__ double cta_join(double v, double *sh) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = join<KIND>(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    v = threadIdx.x < kNormThreads / 32 ? sh[threadIdx.x & 31] : 0.0;
    if (threadIdx.x < 32) {
#pragma unroll
        for (int o = 16; o; o >>= 1) v = join<KIND>(v, __shfl_xor_sync(0xffffffffu, v, o));
    }
    return v;  // thread 0
}

template <typename T> union Vec {
    static constexpr int n = 16 / sizeof(T);
    uint4 u;
    T v[n];
};

// A piece as its vector part and what lies before and behind it (fewer elements than a vector each).
template <typename T> struct Split {
    const T *src;
    unsigned head, vecs, n;
    __device__ __forceinline__ explicit Split(const Piece &p) : src(static_cast<const T *>(p.src)), n(p.n) {
        head = min(n, (unsigned)((0u - (unsigned)(uintptr_t)src) & 15u) / (unsigned)sizeof(T));
        vecs = (n - head) / Vec<T>::n;
    }
    // The one element outside the vectors that thread t looks after, or n.
    __device__ __forceinline__ unsigned edge(unsigned t) const {
        const unsigned tail = head + vecs * Vec<T>::n;
        return t < head ? t : min(n, tail + (t - head));
    }
    __device__ __forceinline__ void load(Vec<T> (&x)[kVecs]) const {
        const uint4 *b = reinterpret_cast<const uint4 *>(src + head);
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const unsigned at = threadIdx.x + i * kNormThreads;
            x[i].u = at < vecs ? b[at] : make_uint4(0, 0, 0, 0);
        }
    }
};

// A thread's values of a piece again, in double: a finite value's square is one there, whatever its size.
template <int KIND, typename T> __device__ __noinline__ double wide_terms(Split<T> s) {
    double a = 0.0;
    auto add = [&](double v) { a += KIND == SCAR_GNORM_L2 ? v * v : fabs(v); };
    const unsigned e = s.edge(threadIdx.x);
    if (e < s.n && threadIdx.x < 2 * Vec<T>::n) add(to_f32<T>(s.src[e]));
    for (unsigned at = threadIdx.x; at < s.vecs; at += kNormThreads) {
        const T *v = s.src + s.head + at * Vec<T>::n;
        for (int j = 0; j < Vec<T>::n; ++j) add(to_f32<T>(v[j]));
    }
    return a;
}

// The terms of a thread's values (at most 33 of a 16-bit type): x its vectors, xe its edge element or 0.  They are summed in
// float32, unless the sum leaves its range: squares of values above 1.8e19 are no float32, those of values below 1e-19 lose
// bits or vanish.  A sum of at least 2^-120 has lost less than 2^-24 of itself (33 squares, each off by at most 2^-150); below
// that, or not finite, the values are read again and summed in double (so are NaN and infinities, with the same result): 400 MB
// of which every thread's sum takes that way 84 us, of ordinary values or zeros 67, each call waited for.
template <int KIND, typename T> __device__ __forceinline__ double thread_terms(const Split<T> &s, const Vec<T> (&x)[kVecs], float xe) {
    float a[2] = {0.f, 0.f};
    add_term<KIND>(a[0], xe);
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int j = 0; j < Vec<T>::n; ++j) add_term<KIND>(a[j & 1], to_f32<T>(x[i].v[j]));
    if (KIND != SCAR_GNORM_MAX) {
        const float sum = a[0] + a[1];
        if (!(sum >= (KIND == SCAR_GNORM_L2 ? 0x1p-120f : 0.f) && sum <= 3.402823466e38f)) {
            constexpr unsigned kMagnitude = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
            unsigned any = __float_as_uint(xe) & 0x7fffffffu;
#pragma unroll
            for (int i = 0; i < kVecs; ++i) any |= (x[i].u.x | x[i].u.y | x[i].u.z | x[i].u.w) & kMagnitude;
            if (any) return wide_terms<KIND, T>(s);  // not for zeros alone
        }
    }
    return join<KIND>((double)a[0], (double)a[1]);
}

template <int KIND, typename T> __device__ __forceinline__ double piece_norm(const Piece &p) {
    const Split<T> s(p);
    Vec<T> x[kVecs];
    s.load(x);
    const unsigned e = s.edge(threadIdx.x);
    return thread_terms<KIND, T>(s, x, e < s.n && threadIdx.x < 2 * Vec<T>::n ? to_f32<T>(s.src[e]) : 0.f);
}

// From the joined sums: the record and the caller's copy of the norm.  Returns the factor.
template <int KIND> __device__ __forceinline__ double norm_factor(double &v, float max_norm, bool clip) {
    if (KIND == SCAR_GNORM_L2) v = sqrt(v);
    return clip && !(v <= (double)max_norm) ? (double)max_norm / v : 1.0;
}
template <int KIND> __device__ __forceinline__ void write_record(double v, float max_norm, bool clip, NormRecord *rec, float *d_norm) {
    const double coef = norm_factor<KIND>(v, max_norm, clip);
    rec->norm = v;
    rec->coef = coef;
    rec->nonfinite = !isfinite(v);
    if (d_norm) *d_norm = (float)v;
}

// Every CTA leaves its part; the last one to do so joins them all.
template <int KIND>
__global__ void __launch_bounds__(kNormThreads, kCtasPerSm)
k_gnorm_norm(const Piece *__restrict__ pieces, unsigned n_pieces, double *part, unsigned *ticket, float max_norm, bool clip,
             NormRecord *rec, float *d_norm) {
    __shared__ double sh[32];
    __shared__ bool last;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    double v = 0.0;
    Piece next{};
    if (blockIdx.x < n_pieces) next = pieces[blockIdx.x];
    for (unsigned i = blockIdx.x; i < n_pieces; i += gridDim.x) {
        const Piece p = next;
        if (i + gridDim.x < n_pieces) next = pieces[i + gridDim.x];
        const double w = p.dtype == SCAR_F32    ? piece_norm<KIND, float>(p)
                         : p.dtype == SCAR_BF16 ? piece_norm<KIND, __nv_bfloat16>(p)
                                                : piece_norm<KIND, __half>(p);
        v = join<KIND>(v, w);
    }
    v = cta_join<KIND>(v, sh);
    if (threadIdx.x == 0) {
        part[blockIdx.x] = v;
        __threadfence();
        last = atomicAdd(ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    v = 0.0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += kNormThreads) v = join<KIND>(v, __ldcg(part + i));
    __syncthreads();
    v = cta_join<KIND>(v, sh);
    if (threadIdx.x) return;
    write_record<KIND>(v, max_norm, clip, rec, d_norm);
    *ticket = 0;  // for the next call
}

// The vectors of a piece, scaled, to their places; element by element where those lie differently within 16 bytes.
template <typename T> __device__ __forceinline__ void store_scaled(const Split<T> &s, Vec<T> (&x)[kVecs], T *d, const Piece &p, float coef) {
    const bool vec = (((uintptr_t)p.dst ^ (uintptr_t)p.src) & 15) == 0;
    d += s.head;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const unsigned at = threadIdx.x + i * kNormThreads;
#pragma unroll
        for (int j = 0; j < Vec<T>::n; ++j) x[i].v[j] = from_f32<T>(to_f32<T>(x[i].v[j]) * coef);
        if (at >= s.vecs) continue;
        if (vec) {
            __stcs(reinterpret_cast<uint4 *>(d) + at, x[i].u);
        } else {
#pragma unroll
            for (int j = 0; j < Vec<T>::n; ++j) d[at * Vec<T>::n + j] = x[i].v[j];
        }
    }
}
// A factor below this has lost bits as a float32 or is about to: the values are scaled in double then (a norm far above the
// limit, as only values near float32's largest give it), one by one, since such a call is rare (400 MB: 291 us against 187).
constexpr double kLeastCoef = 0x1p-100;
template <typename T> __device__ __noinline__ void scale_wide(const void *src, void *dst, unsigned n, double coef) {
    const T *s = static_cast<const T *>(src);
    T *d = static_cast<T *>(dst);
    for (unsigned i = threadIdx.x; i < n; i += kNormThreads) d[i] = from_f32<T>((float)((double)to_f32<T>(s[i]) * coef));
}
__device__ __forceinline__ bool is_wide(double coef) { return coef > 0.0 && coef < kLeastCoef; }
template <typename T> __device__ __forceinline__ void scale_piece(const Piece &p, float coef) {
    const Split<T> s(p);
    Vec<T> x[kVecs];
    s.load(x);
    T *d = static_cast<T *>(p.dst);
    const unsigned e = s.edge(threadIdx.x);
    if (e < s.n && threadIdx.x < 2 * Vec<T>::n) d[e] = from_f32<T>(to_f32<T>(s.src[e]) * coef);
    store_scaled(s, x, d, p, coef);
}

__device__ __forceinline__ void scale_any(const Piece &p, double by) {
    if (is_wide(by)) {
        if (p.dtype == SCAR_F32) scale_wide<float>(p.src, p.dst, p.n, by);
        else if (p.dtype == SCAR_BF16) scale_wide<__nv_bfloat16>(p.src, p.dst, p.n, by);
        else scale_wide<__half>(p.src, p.dst, p.n, by);
        return;
    }
    const float coef = (float)by;
    if (p.dtype == SCAR_F32) scale_piece<float>(p, coef);
    else if (p.dtype == SCAR_BF16) scale_piece<__nv_bfloat16>(p, coef);
    else scale_piece<__half>(p, coef);
}

__global__ void __launch_bounds__(kNormThreads, kCtasPerSm)
k_gnorm_scale(const Piece *__restrict__ pieces, const NormRecord *rec) {
    const Piece p = pieces[gridDim.x - 1 - blockIdx.x];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    scale_any(p, rec->coef);
}

// Both steps in one cooperative launch, for lists of so few pieces that every one has a resident CTA (four per SM: up to
// 9.7 MB): a CTA keeps its piece in registers, leaves its part, waits until all parts are there and joins them itself, in the
// order of k_gnorm_norm.  What it saves is the host's second launch.  Calls back to back, one launch / two: 2^20 float32 values
// 7.3 / 10.0 us, 2.3 million 9.3 / 10.1; 590 tensors of 100 8.2 / 10.0, of 4096 9.6 / 10.3.  Replayed from a graph, where the host has no
// part, the two are even for short lists and one launch behind for long ones (10.3 / 9.9 us; 2.3 million 12.3 / 10.3).
//
// ticket[0] counts parts, ticket[1] the CTAs that are done with them; the last of those clears both.  A kernel of another stream
// may keep some of the CTAs from starting for as long as it likes, so the wait has an end (kPatienceNs): a CTA that reaches it
// sets kGaveUp in ticket[0], unless all parts are there by then.  The CTAs agree, since the count cannot reach the grid's
// without the bit once the bit is set: either all of them go on as above, or none does, and each leaves without having written
// anything.  The last one to leave then finds all parts, whenever that is, and finishes the call by itself: same order, same bits
// (2^20 values 0.18 ms, 592 pieces 0.40 ms).  A millisecond: parts are usually there within microseconds of one another, and CTAs
// that wait keep their multiprocessors from whatever the missing ones wait for.
constexpr unsigned kGaveUp = 0x80000000u;
constexpr unsigned long long kPatienceNs = 1000000ull;

// Thread 0 of a CTA whose part is in place: true when all are there, false when the CTAs gave up.
__device__ __forceinline__ bool all_parts(unsigned *ticket, unsigned long long patience_ns) {
    __threadfence();
    atomicAdd(ticket, 1u);
    unsigned long long t0 = 0, now;
    for (unsigned i = 1;; ++i) {
        unsigned got;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(got) : "l"(ticket) : "memory");
        if (got & kGaveUp) return false;
        if (patience_ns) {
            if (got == gridDim.x) return true;
            if (i & 255u) continue;
            asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
            if (!t0) t0 = now;
            if (now - t0 <= patience_ns) continue;
        }
        if (atomicCAS(ticket, got, got | kGaveUp) == got) return false;
    }
}

enum After { kScaleMine, kLeave, kScaleAll };

template <int KIND> __device__ __forceinline__ double join_parts(const double *part, double *sh) {
    double v = 0.0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += kNormThreads) v = join<KIND>(v, __ldcg(part + i));
    __syncthreads();
    return cta_join<KIND>(v, sh);
}

// True for the CTA that is to scale all pieces by *factor.
template <int KIND, typename T>
__device__ __forceinline__ bool clip_piece(const Piece &p, double *part, unsigned *ticket, float max_norm, unsigned long long patience_ns, NormRecord *rec, float *d_norm,
                                           double *sh, double *factor, After *after) {
    const Split<T> s(p);
    Vec<T> x[kVecs];
    s.load(x);
    const unsigned e = s.edge(threadIdx.x);
    const bool edge = e < s.n && threadIdx.x < 2 * Vec<T>::n;
    const float xe = edge ? to_f32<T>(s.src[e]) : 0.f;
    double v = cta_join<KIND>(join<KIND>(0.0, thread_terms<KIND, T>(s, x, xe)), sh);
    if (threadIdx.x == 0) {
        part[blockIdx.x] = v;
        *after = kScaleMine;
        if (!all_parts(ticket, patience_ns)) {
            *after = atomicAdd(ticket + 1, 1u) == gridDim.x - 1 ? kScaleAll : kLeave;
            __threadfence();
        }
    }
    __syncthreads();
    const After then = *after;
    if (then == kLeave) return false;
    v = join_parts<KIND>(part, sh);
    if (threadIdx.x == 0) {
        if (blockIdx.x == 0 || then == kScaleAll) write_record<KIND>(v, max_norm, true, rec, d_norm);
        *factor = norm_factor<KIND>(v, max_norm, true);
        if (then == kScaleAll) rec->alone += 1;
        if (then == kScaleAll || atomicAdd(ticket + 1, 1u) == gridDim.x - 1) ticket[0] = ticket[1] = 0;
    }
    __syncthreads();
    if (then == kScaleAll) return true;
    if (is_wide(*factor)) {
        scale_wide<T>(p.src, p.dst, p.n, *factor);
        return false;
    }
    const float coef = (float)*factor;
    T *d = static_cast<T *>(p.dst);
    if (edge) d[e] = from_f32<T>(xe * coef);
    store_scaled(s, x, d, p, coef);
    return false;
}
template <int KIND>
__global__ void __launch_bounds__(kNormThreads, kCtasPerSm / 2)
k_gnorm_clip(const Piece *__restrict__ pieces, double *part, unsigned *ticket, float max_norm, unsigned long long patience_ns, NormRecord *rec, float *d_norm) {
    __shared__ double sh[32];
    __shared__ double factor;
    __shared__ After after;
    const Piece p = pieces[blockIdx.x];
    bool all;
    if (p.dtype == SCAR_F32) all = clip_piece<KIND, float>(p, part, ticket, max_norm, patience_ns, rec, d_norm, sh, &factor, &after);
    else if (p.dtype == SCAR_BF16) all = clip_piece<KIND, __nv_bfloat16>(p, part, ticket, max_norm, patience_ns, rec, d_norm, sh, &factor, &after);
    else all = clip_piece<KIND, __half>(p, part, ticket, max_norm, patience_ns, rec, d_norm, sh, &factor, &after);
    if (!all) return;
#pragma unroll 1
    for (unsigned i = 0; i < gridDim.x; ++i) scale_any(pieces[i], factor);
}

}  // namespace

struct scar_gnorm {
    int device = 0;
    cudaStream_t stream = nullptr;
    scar_gnorm_kind kind = SCAR_GNORM_L2;
    std::vector<uint64_t> lengths;
    std::vector<int> types;
    std::vector<Piece> h_pieces;
    char *block = nullptr;  // the one allocation, which the pointers below lie in
    Piece *pieces = nullptr;
    double *part = nullptr;
    unsigned *ticket = nullptr;
    NormRecord *rec = nullptr;
    unsigned grid = 1;
    unsigned resident = 0;  // CTAs of k_gnorm_clip that the GPU holds at a time
    bool ran = false;
    bool no_patience = false;  // of the next k_gnorm_clip
    uint64_t launches = 0;
};

namespace {

// Also gives the pieces that tensors of these lengths are cut into, wherever they lie.
int check_tensors(const scar_tensor *t, uint64_t n, uint64_t &pieces) {
    pieces = 0;
    if (n && !t) return SCAR_ERR_INVALID_ARG;
    for (uint64_t i = 0; i < n; ++i) {
        if (!is_operand_type(t[i].dtype)) return SCAR_ERR_INVALID_ARG;
        const unsigned b = elem_size(t[i].dtype);
        if (t[i].n_elems >= (1ull << 48)) return SCAR_ERR_LAYOUT;
        if (t[i].n_elems && !t[i].d_data) return SCAR_ERR_INVALID_ARG;
        if ((uintptr_t)t[i].d_data % b || (uintptr_t)t[i].d_out % b) return SCAR_ERR_INVALID_ARG;
        pieces += (t[i].n_elems * b + kPieceBytes - 1) / kPieceBytes;
    }
    return pieces < (1ull << 31) ? SCAR_OK : SCAR_ERR_CAPACITY;
}

// A tensor of b bytes has ceil(b / kPieceBytes) pieces wherever it lies, so that new addresses change neither the launches nor
// their grids (a captured call stays right).  The first piece takes the elements before a 16-byte boundary and a piece's worth
// behind them; what is left for the last one may then be nothing.
std::vector<Piece> cut(const scar_tensor *t, uint64_t n) {
    std::vector<Piece> got;
    for (uint64_t i = 0; i < n; ++i) {
        const unsigned b = elem_size(t[i].dtype), most = kPieceBytes / b;
        const char *src = static_cast<const char *>(t[i].d_data);
        char *dst = t[i].d_out ? static_cast<char *>(t[i].d_out) : const_cast<char *>(src);
        const unsigned head = (unsigned)((0u - (uintptr_t)src) % 16) / b;
        const uint64_t pieces = (t[i].n_elems + most - 1) / most;
        uint64_t at = 0;
        for (uint64_t p = 0; p < pieces; ++p) {
            const uint64_t left = t[i].n_elems - at, size = std::min<uint64_t>(left, most + (p ? 0 : head));
            got.push_back({src + at * b, dst + at * b, (unsigned)size, t[i].dtype});
            at += size;
        }
    }
    return got;
}

int upload(scar_gnorm *op) {
    if (!op->h_pieces.empty())
        TRAIN_TRY(cudaMemcpyAsync(op->pieces, op->h_pieces.data(), op->h_pieces.size() * sizeof(Piece),
                                  cudaMemcpyHostToDevice, op->stream));
    TRAIN_TRY(cudaStreamSynchronize(op->stream));
    return SCAR_OK;
}

const void *clip_kernel(scar_gnorm_kind kind) {
    return kind == SCAR_GNORM_L2   ? reinterpret_cast<const void *>(k_gnorm_clip<SCAR_GNORM_L2>)
           : kind == SCAR_GNORM_L1 ? reinterpret_cast<const void *>(k_gnorm_clip<SCAR_GNORM_L1>)
                                   : reinterpret_cast<const void *>(k_gnorm_clip<SCAR_GNORM_MAX>);
}

template <int KIND> void launch_norm(scar_gnorm *op, float max_norm, bool clip, float *d_norm) {
    const unsigned n = (unsigned)op->h_pieces.size();
    k_gnorm_norm<KIND><<<op->grid, kNormThreads, 0, op->stream>>>(op->pieces, n, op->part, op->ticket, max_norm, clip, op->rec, d_norm);
    op->launches += 1;
}

int run_norm(scar_gnorm *op, float max_norm, bool clip, float *d_norm) {
    if (op->kind == SCAR_GNORM_L2) launch_norm<SCAR_GNORM_L2>(op, max_norm, clip, d_norm);
    else if (op->kind == SCAR_GNORM_L1) launch_norm<SCAR_GNORM_L1>(op, max_norm, clip, d_norm);
    else launch_norm<SCAR_GNORM_MAX>(op, max_norm, clip, d_norm);
    TRAIN_TRY(cudaGetLastError());
    op->ran = true;
    return SCAR_OK;
}

}  // namespace

extern "C" {

int scar_gnorm_init(scar_gnorm **out, const scar_tensor *h_tensors, uint64_t n_tensors, scar_gnorm_kind kind,
                    void *cuda_stream) {
    if (!out) return SCAR_ERR_INVALID_ARG;
    *out = nullptr;
    if (kind != SCAR_GNORM_L2 && kind != SCAR_GNORM_L1 && kind != SCAR_GNORM_MAX) return SCAR_ERR_INVALID_ARG;
    uint64_t n_pieces = 0;
    int rc = check_tensors(h_tensors, n_tensors, n_pieces);
    if (rc != SCAR_OK) return rc;
    scar_gnorm *op = nullptr;
    try {
        op = new scar_gnorm();
        for (uint64_t i = 0; i < n_tensors; ++i) {
            op->lengths.push_back(h_tensors[i].n_elems);
            op->types.push_back(h_tensors[i].dtype);
        }
        op->h_pieces = cut(h_tensors, n_tensors);
    } catch (...) {
        delete op;
        return SCAR_ERR_ALLOC;
    }
    op->stream = static_cast<cudaStream_t>(cuda_stream);
    op->kind = kind;
    auto setup = [&]() -> int {
        int sms = 0;
        TRAIN_TRY(cudaGetDevice(&op->device));
        TRAIN_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, op->device));
        int coop = 0, per_sm = 0;
        TRAIN_TRY(cudaDeviceGetAttribute(&coop, cudaDevAttrCooperativeLaunch, op->device));
        TRAIN_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, clip_kernel(op->kind), kNormThreads, 0));
        const unsigned most = kCtasPerSm * (unsigned)sms, n = (unsigned)op->h_pieces.size();
        op->grid = n < 1 ? 1 : (n < most ? n : most);
        op->resident = coop ? (unsigned)(per_sm * sms < (int)most ? per_sm * sms : (int)most) : 0u;
        const uint64_t table = round_up(n_pieces * sizeof(Piece), 256), parts = round_up(op->grid * sizeof(double), 256);
        if (cudaMalloc(&op->block, table + parts + 512) != cudaSuccess) {
            cudaGetLastError();
            return SCAR_ERR_ALLOC;
        }
        op->pieces = reinterpret_cast<Piece *>(op->block);
        op->part = reinterpret_cast<double *>(op->block + table);
        op->rec = reinterpret_cast<NormRecord *>(op->block + table + parts);
        op->ticket = reinterpret_cast<unsigned *>(op->block + table + parts + 256);
        TRAIN_TRY(cudaMemsetAsync(op->rec, 0, 512, op->stream));  // the record and the tickets
        return upload(op);
    };
    rc = setup();
    if (rc != SCAR_OK) {
        scar_gnorm_destroy(op);
        return rc;
    }
    *out = op;
    return SCAR_OK;
}

int scar_gnorm_bind(scar_gnorm *op, const scar_tensor *h_tensors, uint64_t n_tensors) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    uint64_t n_pieces = 0;
    int rc = check_tensors(h_tensors, n_tensors, n_pieces);
    if (rc != SCAR_OK) return rc;
    if (n_tensors != op->lengths.size()) return SCAR_ERR_LAYOUT;
    for (uint64_t i = 0; i < n_tensors; ++i)
        if (h_tensors[i].n_elems != op->lengths[i] || h_tensors[i].dtype != op->types[i]) return SCAR_ERR_LAYOUT;
    if ((rc = check_current_device(op->device)) != SCAR_OK) return rc;
    TRAIN_TRY(cudaStreamSynchronize(op->stream));
    try {
        op->h_pieces = cut(h_tensors, n_tensors);
    } catch (...) {
        return SCAR_ERR_ALLOC;
    }
    return upload(op);
}

int scar_gnorm_norm(scar_gnorm *op, float *d_norm) {
    if (!op || (uintptr_t)d_norm % 4) return SCAR_ERR_INVALID_ARG;
    const int rc = check_current_device(op->device);
    if (rc != SCAR_OK) return rc;
    return run_norm(op, 0.f, false, d_norm);
}

int scar_gnorm_clip(scar_gnorm *op, float max_norm, float *d_norm) {
    if (!op || !(max_norm >= 0.f) || (uintptr_t)d_norm % 4) return SCAR_ERR_INVALID_ARG;
    int rc = check_current_device(op->device);
    if (rc != SCAR_OK) return rc;
    if (!op->h_pieces.empty() && op->h_pieces.size() <= op->resident) {
        unsigned long long patience = op->no_patience ? 0 : kPatienceNs;
        void *args[] = {&op->pieces, &op->part, &op->ticket, &max_norm, &patience, &op->rec, &d_norm};
        TRAIN_TRY(cudaLaunchCooperativeKernel(clip_kernel(op->kind), dim3((unsigned)op->h_pieces.size()), dim3(kNormThreads), args, 0, op->stream));
        op->launches += 1;
        op->ran = true;
        op->no_patience = false;
        return SCAR_OK;
    }
    if ((rc = run_norm(op, max_norm, true, d_norm)) != SCAR_OK) return rc;
    if (op->h_pieces.empty()) return SCAR_OK;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = (unsigned)op->h_pieces.size();
    cfg.blockDim = kNormThreads;
    cfg.stream = op->stream;
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    TRAIN_TRY(cudaLaunchKernelEx(&cfg, k_gnorm_scale, (const Piece *)op->pieces, (const NormRecord *)op->rec));
    op->launches += 1;
    return SCAR_OK;
}

namespace {
int read_record(scar_gnorm *op, NormRecord *rec) {
    const int rc = check_current_device(op->device);
    if (rc != SCAR_OK) return rc;
    TRAIN_TRY(cudaMemcpyAsync(rec, op->rec, sizeof(NormRecord), cudaMemcpyDeviceToHost, op->stream));
    TRAIN_TRY(cudaStreamSynchronize(op->stream));
    return SCAR_OK;
}
}  // namespace

int scar_gnorm_status(scar_gnorm *op, scar_gnorm_info *out) {
    if (!op || !out) return SCAR_ERR_INVALID_ARG;
    if (!op->ran) return SCAR_ERR_STATE;
    NormRecord rec;
    const int rc = read_record(op, &rec);
    if (rc != SCAR_OK) return rc;
    out->norm = rec.norm;
    out->coef = rec.coef;
    out->nonfinite = rec.nonfinite;
    return SCAR_OK;
}

int scar_gnorm_selftest_arm_timeout(scar_gnorm *op) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    op->no_patience = true;
    return SCAR_OK;
}

int scar_gnorm_finished_alone(scar_gnorm *op, uint64_t *calls) {
    if (!op || !calls) return SCAR_ERR_INVALID_ARG;
    NormRecord rec;
    const int rc = read_record(op, &rec);
    if (rc == SCAR_OK) *calls = rec.alone;
    return rc;
}

uint64_t scar_gnorm_launch_count(const scar_gnorm *op) { return op ? op->launches : 0; }

int scar_gnorm_destroy(scar_gnorm *op) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    const bool ok = cudaStreamSynchronize(op->stream) == cudaSuccess;
    cudaFree(op->block);
    delete op;
    if (!ok) cudaGetLastError();
    return ok ? SCAR_OK : SCAR_ERR_CUDA;
}

}  // extern "C"
