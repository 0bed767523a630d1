// The norms before and after a residual block with the block's gate and residual scale (scar_resnorm_* of scar.h):
//
//   u = f or N(f; w_post, b_post)      y = x + scale gate u      n = N(y; w_pre, b_pre)
//   N(v) = (v - mean) r w + b, r = 1 / sqrt(mean of (v - mean)^2 + eps)      (RMS: without mean and b)
//
// and the gradients.  A CTA has a whole row at hand, so x, f and the gate are read once and y and n written once; backward
// reads dy, dn, y, f and the gate once and forms the statistics again from them: storing them would save one of two reductions
// and cost the caller a tensor.  With g = dn w_pre, h = du w_post and hats for normalised rows:
//
//   dY = dy + r_y (g - mean g - y^ mean(g y^))          dx = dY           dw_pre = sum dn y^    db_pre = sum dn
//   du = scale gate dY    dgate = scale sum dY u        df = r_f (h - mean h - f^ mean(h f^))   dw_post = sum du f^   db_post = sum du
//
// A row's mean is summed first and its squared deviations from it second: no sum of squares is taken far from the mean, so rows
// whose mean is large beside their deviation keep theirs.
//
// Memory is what bounds it (16384 x 4096 bfloat16, both norms, a gate for each value: 106 us forward, 6.3 TB/s, and 191 backward,
// 5.6), so the next rows are always on their way: a ring of rows in shared memory, filled by bulk copies (cp.async.bulk) that one warp
// issues.  A stage is filled again behind the first barrier that every thread reaches when it is done with the row.  Rows longer than
// 4096 values are cut over the CTAs of a cluster, which exchange their sums through distributed shared memory: a thread has the
// same number of a row's values whatever its length, and its columns' sums over the rows fit its registers.
//
// Sums over rows: a CTA walks a run of rows and keeps its threads' columns in registers; k_resnorm_join adds the CTAs' sums in
// order.  Gates shared by several rows end inside a CTA's run, or reach over its ends: those leave partial sums too.
#include <algorithm>
#include <initializer_list>
#include <new>
#include <type_traits>

#include "barriers.cuh"
#include "pairs.cuh"

using namespace scar;

namespace {

constexpr unsigned kSpan = 4096;  // columns of a CTA at most
constexpr unsigned kMostStages = 6;
// Values of a row that a thread has, rows that a CTA takes at a time, CTAs of an SM that the registers are for.  16 values, so that
// what a thread does once per row (waits, sums over the CTA, addresses) is shared by many: 16384 x 4096 bfloat16 forward 110 us, with
// eight 187; backward 214 and 317.  Backward with means and biases has four sums over rows for every column, for which 128 registers hold
// eight columns: there two 16-bit rows at a time share what is done once (282 us; 16 columns and one CTA an SM 317, eight and a single
// row 324).  Two float32 rows at a time find no room in shared memory.
constexpr int kForwardValues = 16;
__host__ __device__ constexpr int back_values(bool layer) { return layer ? 8 : 16; }
template <typename T> __host__ __device__ constexpr int back_rows(bool layer) { return layer && sizeof(T) == 2 ? 2 : 1; }
template <typename T> __host__ __device__ constexpr int back_ctas(bool layer) { return layer || sizeof(T) == 4 ? 1 : 2; }
__host__ __device__ constexpr int threads_of(int values) { return (int)kSpan / values; }
constexpr unsigned kNoStage = 0xffffffffu;

// Rows that are read: row r of the operator is row r / per of the matrix.
template <typename T> struct In {
    const T *p;
    unsigned long long pitch;
    unsigned per;
    const T *end;  // of its last row
};
enum { kX, kF, kGate, kForwardIn };              // forward
enum { kDy, kDn, kY, kBackF, kBackGate, kBackwardIn };  // backward

template <typename T> struct NormArgs {
    unsigned rows, dim;
    float scale, eps;
    int post, pre, has_f, has_gate;
    In<T> in[kBackwardIn];
    unsigned n_in;  // of them there are
    const T *w_post, *b_post, *w_pre, *b_pre;
    T *y, *n, *df, *dgate;                      // backward: n is dx
    unsigned long long y_pitch, n_pitch, df_pitch, dgate_pitch;
    unsigned cluster, span;                     // CTAs of a row, and columns of each but the last
    unsigned stages, array_bytes, stage_bytes;  // of the ring
    unsigned slot_off, smem;                    // where sums of rows begin, and bytes in all
    unsigned *error;
    int give_up;                                // self-test: a warp of the first CTA takes its first wait as one that ran out
    // backward
    unsigned per_gate, per_run;  // rows
    float *part;                 // [4][runs][dim]: dw_pre, dw_post, db_pre, db_post
    float *part_gate;            // [runs][2][dim]: of a gate that began before the run, of one that ends behind it
    T *dw_post, *db_post, *dw_pre, *db_pre;
};

// A thread's N values of one row.  A warp has 32 N neighbouring columns.  Rows on 16-byte boundaries: 16 bytes of neighbours per
// thread and round.  Rows anywhere: single values, neighbouring threads next to one another, so that a warp's access is one run of
// memory.  Either way the rounds are a constant distance apart.
template <typename T, int N> union Row {
    uint4 u[N * sizeof(T) / 16];
    T v[N];
    __device__ Row() {}
};
template <bool VEC, typename T, int N> __device__ __forceinline__ unsigned col_of(int i) {
    constexpr int kWord = VEC ? 16 / sizeof(T) : 1;
    return (threadIdx.x & ~31u) * N + (threadIdx.x & 31) * kWord + i / kWord * (32 * kWord) + i % kWord;
}
// All of the warp's columns lie in the row.
template <int N> __device__ __forceinline__ bool whole_warp(unsigned cols) { return ((threadIdx.x & ~31u) + 32) * N <= cols; }
template <bool VEC, typename T, int N> __device__ __forceinline__ void load_row(Row<T, N> &r, const T *p, unsigned cols) {
    if (VEC) {  // rows are whole words
#pragma unroll
        for (unsigned k = 0; k < N * sizeof(T) / 16; ++k) {
            const unsigned col = col_of<true, T, N>(k * (16 / sizeof(T)));
            r.u[k] = col < cols ? *reinterpret_cast<const uint4 *>(p + col) : make_uint4(0, 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const unsigned col = col_of<false, T, N>(i);
            r.v[i] = col < cols ? p[col] : from_f32<T>(0.f);
        }
    }
}
template <bool VEC, typename T, int N> __device__ __forceinline__ void store_row(T *p, const Row<T, N> &r, unsigned cols) {
    if (VEC) {
#pragma unroll
        for (unsigned k = 0; k < N * sizeof(T) / 16; ++k) {
            const unsigned col = col_of<true, T, N>(k * (16 / sizeof(T)));
            if (col < cols) *reinterpret_cast<uint4 *>(p + col) = r.u[k];
        }
    } else if (whole_warp<N>(cols)) {
#pragma unroll
        for (int i = 0; i < N; ++i) p[col_of<false, T, N>(i)] = r.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (col_of<false, T, N>(i) < cols) p[col_of<false, T, N>(i)] = r.v[i];
    }
}
// A row from a stage of the ring as float32 pairs; zeros lie behind it there.
template <bool VEC, typename T, int N> __device__ __forceinline__ void fetch_row(float2 (&v)[N / 2], const T *p) {
    Row<T, N> r;
    load_row<VEC>(r, p, ~0u);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = Two<T>::get(r.v + 2 * i);
}
template <bool VEC, typename T, int N> __device__ __forceinline__ void write_row(T *p, const float2 (&v)[N / 2], unsigned cols) {
    Row<T, N> r;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) Two<T>::put(r.v + 2 * i, v[i]);
    store_row<VEC>(p, r, cols);
}
// A thread's own copy of a vector in shared memory, zeros behind its columns.
template <bool VEC, typename T, int N> __device__ __forceinline__ void put_row(T *p, const Row<T, N> &r) { store_row<VEC>(p, r, ~0u); }
template <bool VEC, typename T, int N> __device__ __forceinline__ void take_row(Row<T, N> &r, const T *p) { load_row<VEC>(r, p, ~0u); }
template <bool VEC, typename T, int N> __device__ __forceinline__ void load_vector(Row<T, N> &r, const T *p, unsigned cols, unsigned col0, float otherwise) {
    if (p) {
        load_row<VEC>(r, p + col0, cols);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] = from_f32<T>(col_of<VEC, T, N>(i) < cols ? otherwise : 0.f);
}
// v + shift, but zeros stay behind the row.
template <bool VEC, typename T, int N> __device__ __forceinline__ void shift_row(float2 (&v)[N / 2], float shift, unsigned cols) {
    constexpr int kWord = VEC ? 16 / sizeof(T) : 1;  // all or none of a word's values lie in the row
    if (!VEC && whole_warp<N>(cols)) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) v[i] = add2(v[i], both(shift));
        return;
    }
#pragma unroll
    for (int i = 0; i < N; i += kWord) {
        const float s = col_of<VEC, T, N>(i) < cols ? shift : 0.f;
        if (kWord == 1) {
            float &x = i & 1 ? v[i / 2].y : v[i / 2].x;
            x += s;
        } else {
#pragma unroll
            for (int j = i / 2; j < (i + kWord) / 2; ++j) v[j] = add2(v[j], both(s));
        }
    }
}
template <int M> __device__ __forceinline__ float total(const float2 (&v)[M]) {
    float2 s = v[0];
#pragma unroll
    for (int i = 1; i < M; ++i) s = add2(s, v[i]);
    return s.x + s.y;
}
template <int M> __device__ __forceinline__ float dot(const float2 (&a)[M], const float2 (&b)[M]) {
    float2 s = mul2(a[0], b[0]);
#pragma unroll
    for (int i = 1; i < M; ++i) s = fma2(a[i], b[i], s);
    return s.x + s.y;
}

// The CTA's ring of rows.  Its methods that copy are called by all lanes of one warp and by no other warp: a lane per matrix copies the
// 16-byte words that its row lies in, with what else is in the first and the last one of them.  Where such a word is not the matrix's
// alone (first and last rows), lanes read the row's values in it one by one and put them in place a row later; done for every row, that
// takes 192 us forward and 362 backward for 16384 x 4095 bfloat16 instead of 142 and 309.  At the barrier of a stage every matrix arrives
// once, and the values at the rows' ends together once.
template <typename T, bool VEC, int IN, int R> struct Ring {
    static constexpr int kEnd = 16 / sizeof(T) - 1;                         // values at one end of a row, at most
    static constexpr int kPasses = VEC ? 1 : (2 * kEnd * IN + 31) / 32;     // rounds of a warp over all ends of a row
    const NormArgs<T> &g;
    uint8_t *smem;
    uint32_t full;   // barriers, one per stage
    unsigned *sent;  // where the warp leaves how many rows it had issued when a wait gave up; they take the stages in turn
    unsigned col0, cols;
    T edge[R][kPasses];  // on their way to the stages of the rows that were issued last
    unsigned open[R];    // their matrices, a bit each

    __device__ __forceinline__ const T *source(int a, unsigned row) const {
        const In<T> &m = g.in[a];
        return m.p + (unsigned long long)(m.per > 1 ? row / m.per : row) * m.pitch + col0;
    }
    // Where a row lies in its stage: as far from a 16-byte boundary as in memory.
    __device__ __forceinline__ const T *at(int a, unsigned row, unsigned stage) const {
        const unsigned off = VEC ? 0u : (unsigned)(uintptr_t)source(a, row) & 15u;
        return reinterpret_cast<const T *>(smem + stage * g.stage_bytes + a * g.array_bytes + off);
    }
    // The 16-byte words that a row's values are in, or those that hold nothing else.
    __device__ __forceinline__ bool words(const In<T> &m, const T *p, uintptr_t &from, uintptr_t &to) const {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = a + cols * sizeof(T);
        from = a;
        to = b;
        if (VEC) return true;
        from = a & ~uintptr_t(15);
        to = (b + 15) & ~uintptr_t(15);
        if (from >= reinterpret_cast<uintptr_t>(m.p) && to <= reinterpret_cast<uintptr_t>(m.end)) return true;
        from = (a + 15) & ~uintptr_t(15);
        to = b & ~uintptr_t(15);
        if (to < from) to = from;
        return false;
    }
    // f(matrix, its row, which of the values behind the row's end, which value of the row or none) for each of this lane's ends.
    template <typename F> __device__ __forceinline__ void ends(unsigned row, unsigned open, F f) const {
#pragma unroll
        for (int q = 0; q < kPasses; ++q) {
            const unsigned id = q * 32 + (threadIdx.x & 31), a = id / (2 * kEnd), j = id % (2 * kEnd);
            if (a >= IN || !(open >> a & 1u)) continue;
            const T *p = source(a, row);
            uintptr_t from, to;
            words(g.in[a], p, from, to);
            const unsigned head = min(cols, (unsigned)((from - reinterpret_cast<uintptr_t>(p)) / sizeof(T)));
            const unsigned tail = max(head, (unsigned)((to - reinterpret_cast<uintptr_t>(p)) / sizeof(T)));
            const unsigned i = j < kEnd ? j : tail + j - kEnd;
            if (j < kEnd ? i < head : i < cols) f(q, a, p, i);
        }
    }
    __device__ __forceinline__ void arrive(unsigned stage) const {
        if ((threadIdx.x & 31) == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(full + 8 * stage) : "memory");
    }
    __device__ __forceinline__ void put_edges(unsigned row, unsigned stage, int k = 0) {
        if (VEC || !open[k]) return;
        ends(row, open[k], [&](int q, unsigned a, const T *, unsigned i) { const_cast<T *>(at(a, row, stage))[i] = edge[k][q]; });
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // a later row's copy may write over what was stored here
        __syncwarp();
        arrive(stage);
    }
    __device__ __forceinline__ void issue(unsigned row, unsigned stage, int k = 0) {
        const unsigned a = threadIdx.x & 31;
        bool all = true;
        if (a < IN && g.in[a].p) {
            const uint32_t bar = full + 8 * stage;
            const T *p = source(a, row);
            uintptr_t from, to;
            all = words(g.in[a], p, from, to);
            mbar_expect(bar, (unsigned)(to - from));
            if (to != from)
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                                 smem_addr(at(a, row, stage)) + (uint32_t)((intptr_t)from - (intptr_t)p)),
                             "l"(from), "r"((unsigned)(to - from)), "r"(bar)
                             : "memory");
        }
        if (!VEC) {
            open[k] = __ballot_sync(0xffffffffu, !all);
            if (open[k]) ends(row, open[k], [&](int q, unsigned, const T *p, unsigned i) { edge[k][q] = p[i]; });
            else arrive(stage);
        }
        __syncwarp();
    }
    // After a wait that gave up: no more rows than these n.
    __device__ __forceinline__ void stop(unsigned n) const {
        if ((threadIdx.x & 31) == 0 && !*sent) *sent = n;
    }
    // And at the end of all `rows`: the copies that may still be under way, with a limit.
    __device__ __forceinline__ void drain(unsigned rows) const {
        const unsigned long long until = now_ns() + kWaitNs;
        const unsigned n = *sent ? *sent : rows;
        for (unsigned i = n > g.stages ? n - g.stages : 0u; i < n; ++i)
            while (!mbar_try(full + 8 * (i % g.stages), i / g.stages & 1u) && now_ns() < until) {}
    }
    // Zeros behind a row of the stage that has arrived, each warp in its own columns: there lie the rest of the row's last word and what a
    // row that began further on has left.  Before that row there were zeros again.
    template <int N> __device__ __forceinline__ void close(unsigned row, unsigned stage) const {
        if (VEC || whole_warp<N>(cols)) return;
#pragma unroll
        for (int q = 0; q < (IN * 8 + 31) / 32; ++q) {
            const unsigned id = q * 32 + (threadIdx.x & 31), a = id / 8, j = id % 8, col = cols + j;
            if (a < IN && g.in[a].p && j < kEnd && col / (32 * N) == threadIdx.x / 32) const_cast<T *>(at(a, row, stage))[col] = from_f32<T>(0.f);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
    }
};

// As mbar_wait, for what other CTAs of the cluster have written before they arrived.
__device__ __forceinline__ bool try_cluster(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok;
}
__device__ __forceinline__ bool wait_cluster(uint32_t bar, uint32_t parity, unsigned *error) {
    if (try_cluster(bar, parity)) return true;
    unsigned long long until = 0;
    for (unsigned i = 1;; ++i) {
        if (try_cluster(bar, parity)) return true;
        if ((i & 255u) == 0) {
            const unsigned long long now = now_ns();
            if (!until) until = now + kWaitNs;
            if (now > until) {
                atomicExch(error, 1u);
                return false;
            }
        }
    }
}

// Sums over a row, K at a time.  Within a warp the lanes halve what they carry at every exchange, until each has one of the K sums
// of some lanes (three values: 5 exchanges, not 15).  Warps leave theirs in one half of `slot` (of every CTA of the cluster), and every
// warp adds them up in the same order.  The halves alternate: one is written again only when all warps have arrived at the reduction
// between, and a warp arrives there after it has read.  A wait that gave up (`ok`, a lane's own) is not repeated: the loops go on
// without waiting and end.  Over a cluster such a lane sends nothing more and announces nothing more at its CTA's barrier: the sum
// that it leaves out completes nowhere, so all warps of the cluster give up at it, none later, and no barrier sees an arrival too many.
struct Shared {
    unsigned long long full[kMostStages], red[2];
    unsigned sent;
};
template <int kWarps> struct Sums {  // kWarps: of a CTA at most
    Shared *sh;
    float *slot;  // [2][8][warps of the cluster]
    unsigned half, phase, cluster;
    unsigned *error;
    bool ok;

    template <int K> __device__ __forceinline__ void add(float (&v)[K]) {
        constexpr int P = K == 1 ? 1 : K == 2 ? 2 : K <= 4 ? 4 : 8, kLanes = 32 / P;  // lanes that end up with the same sum
        const unsigned lane = threadIdx.x & 31, warp = threadIdx.x / 32, warps = blockDim.x / 32;
        float w[P];
#pragma unroll
        for (int k = 0; k < P; ++k) w[k] = k < K ? v[k < K ? k : 0] : 0.f;
#pragma unroll
        for (int o = 16, n = P / 2; o >= kLanes; o >>= 1, n >>= 1) {
#pragma unroll
            for (int k = 0; k < P / 2; ++k) {
                if (k >= n) continue;
                const float keep = lane & o ? w[k + n] : w[k], give = lane & o ? w[k] : w[k + n];
                w[k] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
        }
        float x = w[0];
#pragma unroll
        for (int o = kLanes / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if (blockDim.x * cluster == 32) {
            __syncwarp();
        } else {
            float *at = slot + (half * 8 + lane / kLanes) * (warps * cluster);
            const unsigned sub = lane % kLanes;
            if (cluster == 1) {
                if (sub == 0) at[warp] = x;
                __syncthreads();
                x = 0.f;
                constexpr int kOver = kWarps < kLanes ? kWarps : kLanes;  // lanes that share a sum's warps; the others do the same again
#pragma unroll
                for (int e = 0; e < kWarps; e += kOver) {
                    const unsigned i = e + sub % kOver;
                    x += i < warps ? at[i] : 0.f;
                }
#pragma unroll
                for (int o = kOver / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
            } else {
                // Stores that report themselves at the reader's barrier: an arrival that releases would wait for this warp's results
                // on their way to memory (4096 x 16384 bfloat16, forward: 390 us).
                const uint32_t mbar = smem_addr(sh->red + half);
                if (threadIdx.x == 0 && ok) mbar_expect(mbar, P * 4 * warps * cluster);
                if (sub == 0 && ok) {
                    const uint32_t here = smem_addr(at + cluster_rank() * warps + warp);
                    for (unsigned c = 0; c < cluster; ++c)
                        asm volatile("{\n .reg .b32 a, b;\n mapa.shared::cluster.u32 a, %0, %2;\n mapa.shared::cluster.u32 b, %1, %2;\n"
                                     " st.async.shared::cluster.mbarrier::complete_tx::bytes.f32 [a], %3, [b];\n}\n" ::"r"(here), "r"(mbar), "r"(c), "f"(x)
                                     : "memory");
                }
                if (ok) ok = wait_cluster(mbar, phase >> half & 1u, error);
                __syncwarp();
                phase ^= 1u << half;
                x = 0.f;
                for (unsigned i = sub; i < warps * cluster; i += kLanes) x += at[i];
#pragma unroll
                for (int o = kLanes / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
            }
            half ^= 1;
        }
        if (K == 1) {
            v[0] = x;
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] = __shfl_sync(0xffffffffu, x, k * kLanes);
        }
    }
};

// Barriers, and zeros in the ring, before any copy.
template <bool VEC, typename T> __device__ __forceinline__ void start(const NormArgs<T> &g, Shared &sh, uint8_t *smem) {
    for (unsigned i = threadIdx.x; i < g.stages * g.stage_bytes / 16; i += blockDim.x) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if (threadIdx.x == 0) {
        sh.sent = 0;
        for (unsigned i = 0; i < g.stages; ++i) mbar_init(smem_addr(sh.full + i), g.n_in + (VEC ? 0 : 1));
        for (int i = 0; i < 2; ++i) mbar_init(smem_addr(sh.red + i), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (g.cluster > 1) cluster_sync_all();
    else __syncthreads();
}

// No wait has run out, except for the self-test.
template <typename T> __device__ __forceinline__ bool begins_well(const NormArgs<T> &g) {
    const bool ok = !(g.give_up && blockIdx.x == 0 && (int)(threadIdx.x / 32) == g.give_up - 1);
    if (!ok) atomicExch(g.error, 1u);
    return ok;
}

// The end of a CTA.  Where a wait gave up, copies of its own that are under way come first, and the CTAs of a cluster leave together:
// one whose waits gave up is through long before those that still store into its shared memory.  What these have stored by then
// is given a millisecond to arrive; elsewhere the last sum has waited for all of it.
template <typename T, typename R, typename S> __device__ __forceinline__ void leave(const NormArgs<T> &g, const R &ring, const S &sums, unsigned rows) {
    if (!sums.ok && threadIdx.x < 32) ring.drain(rows);
    __syncwarp();
    // relaxed: nothing is handed over, and a release would wait for this warp's results on their way to memory
    if (g.cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
    if (!sums.ok)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
}

// 1 / sqrt(q / dim + eps)
__device__ __forceinline__ float deviation(float q, float inv_dim, float eps) { return rsqrtf(fmaf(q, inv_dim, eps)); }

template <typename T, bool LAYER, bool VEC>
__global__ void __launch_bounds__(threads_of(kForwardValues), 2) k_resnorm_forward(const __grid_constant__ NormArgs<T> g) {
    constexpr int N = kForwardValues;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) Shared sh;
    const unsigned rank = g.cluster > 1 ? cluster_rank() : 0u, first = blockIdx.x / g.cluster, step = gridDim.x / g.cluster;
    const unsigned col0 = rank * g.span, cols = min(g.span, g.dim - col0), warp = threadIdx.x / 32;
    start<VEC>(g, sh, smem);
    Ring<T, VEC, kForwardIn, 1> ring{g, smem, smem_addr(sh.full), &sh.sent, col0, cols};
    Sums<threads_of(N) / 32> sums{&sh, reinterpret_cast<float *>(smem + g.slot_off), 0u, 0u, g.cluster, g.error, true};
    if (warp == 0)
        for (unsigned i = 0; i < g.stages && first + i * step < g.rows; ++i) {
            ring.issue(first + i * step, i);
            ring.put_edges(first + i * step, i);
        }
    Row<T, N> w_post, b_post, w_pre, b_pre;
    load_vector<VEC>(w_post, g.w_post, cols, col0, 1.f);
    load_vector<VEC>(w_pre, g.w_pre, cols, col0, 1.f);
    if (LAYER) {
        load_vector<VEC>(b_post, g.b_post, cols, col0, 0.f);
        load_vector<VEC>(b_pre, g.b_pre, cols, col0, 0.f);
    }
    const float inv_dim = 1.f / (float)g.dim;
    unsigned stage = 0, parity = 0, edges = kNoStage, edge_row = 0;
    sums.ok = begins_well(g);
    for (unsigned row = first; row < g.rows; row += step) {
        if (sums.ok) sums.ok = mbar_wait(smem_addr(sh.full + stage), parity, g.error);
        __syncwarp();
        ring.template close<N>(row, stage);
        // v becomes its deviation from the mean, the result is 1 / its deviation as a whole
        const auto normalise = [&](float2 (&v)[N / 2], auto between) {
            float s[1];
            if (LAYER) {
                s[0] = total(v);
                sums.add(s);
                between();
                shift_row<VEC, T, N>(v, -s[0] * inv_dim, cols);
            }
            s[0] = dot(v, v);
            sums.add(s);
            if (!LAYER) between();
            return deviation(s[0], inv_dim, g.eps);
        };
        float2 y[N / 2];
        fetch_row<VEC, T, N>(y, ring.at(kX, row, stage));
        if (g.has_f) {
            float2 u[N / 2], a[N / 2];
            fetch_row<VEC, T, N>(u, ring.at(kF, row, stage));
            if (g.post) {
                const float2 r = both(normalise(u, []() {}));
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    u[i] = mul2(mul2(u[i], r), Two<T>::get(w_post.v + 2 * i));
                    if (LAYER) u[i] = add2(u[i], Two<T>::get(b_post.v + 2 * i));
                }
            }
            const float2 scale = both(g.scale);
            if (g.has_gate) {
                fetch_row<VEC, T, N>(a, ring.at(kGate, row, stage));
#pragma unroll
                for (int i = 0; i < N / 2; ++i) y[i] = fma2(mul2(a[i], scale), u[i], y[i]);
            } else {
#pragma unroll
                for (int i = 0; i < N / 2; ++i) y[i] = fma2(scale, u[i], y[i]);
            }
        }
        // Called once the CTA is done with the stage: it takes a row further on.
        const auto refill = [&]() {
            if (warp != 0) return;
            if (!VEC && edges != kNoStage) ring.put_edges(edge_row, edges);
            edges = kNoStage;
            const unsigned long long next = row + (unsigned long long)g.stages * step;
            if (next >= g.rows) return;
            if (!__all_sync(0xffffffffu, sums.ok)) {
                ring.stop((row - first) / step + g.stages);
                return;
            }
            ring.issue((unsigned)next, stage);
            edges = stage;
            edge_row = (unsigned)next;
        };
        Row<T, N> out;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            Two<T>::put(out.v + 2 * i, y[i]);
            y[i] = Two<T>::get(out.v + 2 * i);  // the norm is that of the values handed on: backward has them and nothing else
        }
        if (g.y) store_row<VEC>(g.y + row * g.y_pitch + col0, out, cols);
        if (g.pre) {
            const float2 r = both(normalise(y, refill));  // y is zero behind the row, where x, f and the weights are
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                y[i] = mul2(mul2(y[i], r), Two<T>::get(w_pre.v + 2 * i));
                if (LAYER) y[i] = add2(y[i], Two<T>::get(b_pre.v + 2 * i));
            }
            write_row<VEC, T, N>(g.n + row * g.n_pitch + col0, y, cols);
        } else {
            __syncthreads();
            refill();
        }
        if (++stage == g.stages) {
            stage = 0;
            parity ^= 1;
        }
    }
    leave(g, ring, sums, first < g.rows ? (g.rows - first - 1) / step + 1 : 0u);
}

template <bool VEC, typename T, int N> __device__ __forceinline__ void put_part(float *p, const float2 (&v)[N / 2], unsigned cols) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (col_of<VEC, T, N>(i) < cols) p[col_of<VEC, T, N>(i)] = i & 1 ? v[i / 2].y : v[i / 2].x;
}

template <typename T, bool LAYER, bool VEC, bool SHARED>
__global__ void __launch_bounds__(threads_of(back_values(LAYER)), back_ctas<T>(LAYER)) k_resnorm_backward(const __grid_constant__ NormArgs<T> g) {
    constexpr int N = back_values(LAYER), M = N / 2, R = back_rows<T>(LAYER);
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) Shared sh;
    const unsigned rank = g.cluster > 1 ? cluster_rank() : 0u, run = blockIdx.x / g.cluster, runs = gridDim.x / g.cluster;
    const unsigned col0 = rank * g.span, cols = min(g.span, g.dim - col0), warp = threadIdx.x / 32;
    const unsigned r0 = run * g.per_run, r1 = min(g.rows, r0 + g.per_run);
    start<VEC>(g, sh, smem);
    Ring<T, VEC, kBackwardIn, R> ring{g, smem, smem_addr(sh.full), &sh.sent, col0, cols};
    Sums<threads_of(N) / 32> sums{&sh, reinterpret_cast<float *>(smem + g.slot_off), 0u, 0u, g.cluster, g.error, true};
    if (warp == 0)
        for (unsigned i = 0; i < g.stages && r0 + i < r1; ++i) {
            ring.issue(r0 + i, i);
            ring.put_edges(r0 + i, i);
        }
    const float inv_dim = 1.f / (float)g.dim;
    const bool norm_f = g.has_f && g.post;
    const float2 zero = both(0.f);
    float2 a_wpre[M], a_wpost[M], a_bpre[LAYER ? M : 1], a_bpost[LAYER ? M : 1], a_gate[SHARED ? M : 1];
#pragma unroll
    for (int i = 0; i < M; ++i) {
        a_wpre[i] = a_wpost[i] = zero;
        if (SHARED) a_gate[SHARED ? i : 0] = zero;
        if (LAYER) a_bpre[LAYER ? i : 0] = a_bpost[LAYER ? i : 0] = zero;
    }
    // a thread's weights stay in shared memory, where it alone reads them: its registers hold the columns' sums
    T *const w_pre = reinterpret_cast<T *>(smem + g.stages * g.stage_bytes), *const w_post = w_pre + g.array_bytes / sizeof(T);
    T *const b_post = w_post + g.array_bytes / sizeof(T);
    {
        Row<T, N> w;
        load_vector<VEC>(w, g.w_pre, cols, col0, 1.f);
        put_row<VEC>(w_pre, w);
        load_vector<VEC>(w, g.w_post, cols, col0, 1.f);
        put_row<VEC>(w_post, w);
        if (LAYER) {
            load_vector<VEC>(w, g.b_post, cols, col0, 0.f);
            put_row<VEC>(b_post, w);
        }
    }
    T *dx = g.n ? g.n + r0 * g.n_pitch + col0 : nullptr, *df = g.df ? g.df + r0 * g.df_pitch + col0 : nullptr;
    unsigned stage = 0, parity = 0, edges = 0;  // rows whose edges are on their way
    // Called behind a barrier that the CTA reaches when it is done with the rows before: their stages take rows further on.
    const auto refill = [&](unsigned row0) {
        if (warp != 0 || row0 == r0) return;
        const unsigned before = (stage ? stage : g.stages) - R;
        if (!__all_sync(0xffffffffu, sums.ok)) {
            ring.stop(min(row0 - R - r0 + g.stages, r1 - r0));
            return;
        }
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (row0 - R + k + (unsigned long long)g.stages < r1) {
                ring.issue(row0 - R + k + g.stages, before + k, k);
                edges = k + 1;
            }
    };
    sums.ok = begins_well(g);
    for (unsigned row0 = r0; row0 < r1; row0 += R) {
        const unsigned mine = min((unsigned)R, r1 - row0);
        if (!VEC && warp == 0 && edges) {  // of the rows that the last refill issued
            const unsigned before = (stage ? stage : g.stages) - R, earlier = (before ? before : g.stages) - R;
#pragma unroll
            for (int k = 0; k < R; ++k)
                if (k < edges) ring.put_edges(row0 - 2 * R + g.stages + k, earlier + k, k);
            edges = 0;
        }
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (k < mine && sums.ok) sums.ok = mbar_wait(smem_addr(sh.full + stage + k), parity, g.error);
        __syncwarp();
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (k < mine) ring.template close<N>(row0 + k, stage + k);
        // Minus the means of y and f; then, of their deviations y' and f' and with e = dn w_pre: sums of y'^2, e y', f'^2, e.
        constexpr int K = LAYER ? 4 : 3;
        float m[2 * R] = {}, q[K * R] = {};
        if (LAYER && (g.pre || norm_f)) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (k >= mine) continue;
                float2 v[M];
                if (g.pre) {
                    fetch_row<VEC, T, N>(v, ring.at(kY, row0 + k, stage + k));
                    m[2 * k] = total(v);
                }
                if (norm_f) {
                    fetch_row<VEC, T, N>(v, ring.at(kBackF, row0 + k, stage + k));
                    m[2 * k + 1] = total(v);
                }
            }
            sums.add(m);
#pragma unroll
            for (int k = 0; k < 2 * R; ++k) m[k] *= -inv_dim;
        }
        if (g.pre || norm_f) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (k >= mine) continue;
                if (g.pre) {
                    float2 y[M], e[M];
                    Row<T, N> w;
                    take_row<VEC>(w, w_pre);
                    fetch_row<VEC, T, N>(y, ring.at(kY, row0 + k, stage + k));
                    fetch_row<VEC, T, N>(e, ring.at(kDn, row0 + k, stage + k));
                    if (LAYER) shift_row<VEC, T, N>(y, m[2 * k], cols);
#pragma unroll
                    for (int i = 0; i < M; ++i) e[i] = mul2(e[i], Two<T>::get(w.v + 2 * i));
                    if (LAYER) q[K * k + K - 1] = total(e);
                    q[K * k] = dot(y, y);
                    q[K * k + 1] = dot(e, y);
                }
                if (norm_f) {
                    float2 f[M];
                    fetch_row<VEC, T, N>(f, ring.at(kBackF, row0 + k, stage + k));
                    if (LAYER) shift_row<VEC, T, N>(f, m[2 * k + 1], cols);
                    q[K * k + 2] = dot(f, f);
                }
            }
            sums.add(q);
        } else {
            __syncthreads();
        }
        refill(row0);
        // With r = 1 / deviation of y, rf of f and t = r dn:  dY = dy + w_pre t - r mean e - y' r^3 mean(e y'),  dw_pre += t y'
        //   t2 = scale rf dY:  dgate = t2 w_post f' + scale dY b_post,  h = t2 gate (the gradient of f^ times rf, without w_post)
        //   dw_post += h f',  df = h w - mean(h w) - f' rf^2 mean(h w f')
        float2 d[R][M];  // dY, then h w
        float h[(LAYER ? 2 : 1) * R] = {};
        constexpr int H = LAYER ? 2 : 1;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (k >= mine) continue;
            const unsigned row = row0 + k, st = stage + k;
            if (g.in[kDy].p) {
                fetch_row<VEC, T, N>(d[k], ring.at(kDy, row, st));
            } else {
#pragma unroll
                for (int i = 0; i < M; ++i) d[k][i] = zero;
            }
            if (g.pre) {
                float2 y[M], e[M];
                Row<T, N> w;
                take_row<VEC>(w, w_pre);
                fetch_row<VEC, T, N>(y, ring.at(kY, row, st));
                fetch_row<VEC, T, N>(e, ring.at(kDn, row, st));
                if (LAYER) shift_row<VEC, T, N>(y, m[2 * k], cols);
                const float r = deviation(q[K * k], inv_dim, g.eps);
                const float2 rr = both(r), c = both(-(r * r) * (r * q[K * k + 1] * inv_dim));
                if (LAYER) shift_row<VEC, T, N>(d[k], -r * q[K * k + K - 1] * inv_dim, cols);
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    if (LAYER) a_bpre[LAYER ? i : 0] = add2(a_bpre[LAYER ? i : 0], e[i]);
                    const float2 t = mul2(e[i], rr);
                    d[k][i] = fma2(y[i], c, fma2(t, Two<T>::get(w.v + 2 * i), d[k][i]));
                    a_wpre[i] = fma2(t, y[i], a_wpre[i]);
                }
            }
            if (dx) {
                write_row<VEC, T, N>(dx, d[k], cols);
                dx += g.n_pitch;
            }
            if (!g.has_f) continue;
            const float rf = norm_f ? deviation(q[K * k + 2], inv_dim, g.eps) : 1.f;
            float2 f[M], a[M];
            Row<T, N> w, out;
            take_row<VEC>(w, w_post);
            fetch_row<VEC, T, N>(f, ring.at(kBackF, row, st));
            if (LAYER) shift_row<VEC, T, N>(f, m[2 * k + 1], cols);
            if (g.has_gate) {
                fetch_row<VEC, T, N>(a, ring.at(kBackGate, row, st));
            } else {
#pragma unroll
                for (int i = 0; i < M; ++i) a[i] = both(1.f);
            }
            const float2 scale = both(LAYER ? g.scale : g.scale * rf), rr = both(rf);
            Row<T, N> b;
            if (LAYER) take_row<VEC>(b, b_post);
#pragma unroll
            for (int i = 0; i < M; ++i) {
                float2 t = mul2(d[k][i], scale);
                const float2 ww = Two<T>::get(w.v + 2 * i);
                float2 e = zero;
                if (LAYER) {
                    e = mul2(t, Two<T>::get(b.v + 2 * i));
                    a_bpost[LAYER ? i : 0] = fma2(t, a[i], a_bpost[LAYER ? i : 0]);
                    t = mul2(t, rr);
                }
                if (SHARED || g.dgate) {
                    const float2 fw = mul2(f[i], ww);
                    e = LAYER ? fma2(t, fw, e) : mul2(t, fw);
                    if (SHARED) a_gate[SHARED ? i : 0] = add2(a_gate[SHARED ? i : 0], e);
                    else Two<T>::put(out.v + 2 * i, e);
                }
                t = mul2(t, a[i]);
                a_wpost[i] = fma2(t, f[i], a_wpost[i]);
                d[k][i] = mul2(t, ww);
            }
            if constexpr (SHARED) {
                const unsigned gate = row / g.per_gate, begin = gate * g.per_gate, end = g.rows - begin > g.per_gate ? begin + g.per_gate : g.rows;
                if (row + 1 == r1 || row + 1 == end) {
                    if (begin >= r0 && end <= r1) write_row<VEC, T, N>(g.dgate + gate * g.dgate_pitch + col0, a_gate, cols);
                    else put_part<VEC, T, N>(g.part_gate + (run * 2ull + (begin < r0 ? 0 : 1)) * g.dim + col0, a_gate, cols);
#pragma unroll
                    for (int i = 0; i < M; ++i) a_gate[i] = zero;
                }
            } else if (g.dgate) {
                store_row<VEC>(g.dgate + row * g.dgate_pitch + col0, out, cols);
            }
            if (norm_f) {
                h[H * k] = dot(d[k], f);
                if (LAYER) h[H * k + H - 1] = total(d[k]);
            }
        }
        if (norm_f) sums.add(h);
        if (df) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (k >= mine) continue;
                if (norm_f) {
                    float2 f[M];
                    fetch_row<VEC, T, N>(f, ring.at(kBackF, row0 + k, stage + k));
                    if (LAYER) {
                        shift_row<VEC, T, N>(f, m[2 * k + 1], cols);
                        shift_row<VEC, T, N>(d[k], -h[H * k + H - 1] * inv_dim, cols);
                    }
                    const float rf = deviation(q[K * k + 2], inv_dim, g.eps);
                    const float2 c = both(-(rf * rf) * (h[H * k] * inv_dim));
#pragma unroll
                    for (int i = 0; i < M; ++i) d[k][i] = fma2(f[i], c, d[k][i]);
                }
                write_row<VEC, T, N>(df, d[k], cols);
                df += g.df_pitch;
            }
        }
        stage += R;
        if (stage == g.stages) {
            stage = 0;
            parity ^= 1;
        }
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the join: its CTAs get ready while the last sums are written
    const unsigned long long each = (unsigned long long)runs * g.dim, mine = (unsigned long long)run * g.dim + col0;
    if (g.dw_pre) put_part<VEC, T, N>(g.part + mine, a_wpre, cols);
    if (g.dw_post) put_part<VEC, T, N>(g.part + each + mine, a_wpost, cols);
    if constexpr (LAYER) {
        if (g.db_pre) put_part<VEC, T, N>(g.part + 2 * each + mine, a_bpre, cols);
        if (g.db_post) put_part<VEC, T, N>(g.part + 3 * each + mine, a_bpost, cols);
    }
    leave(g, ring, sums, r1 > r0 ? r1 - r0 : 0u);
}

// Adds the runs' sums, 32 columns a CTA, 16 walkers over the rows of the list, in an order that depends on the sizes alone.
// blockIdx.y 0 .. 3: the vectors; the others take turns at the gates whose rows are cut by a run's end.
constexpr unsigned kJoinGates = 32;
template <typename T> __global__ void __launch_bounds__(512) k_resnorm_join(const __grid_constant__ NormArgs<T> g, unsigned runs) {
    __shared__ float sh[16][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const unsigned lane = threadIdx.x & 31, col = blockIdx.x * 32 + lane, walker = threadIdx.x >> 5;
    // rows of `from`, `step` apart; the first lies `skip` further on
    const auto join = [&](const float *from, unsigned long long step, unsigned n, unsigned skip, T *out) {
        float v = 0.f;
        if (col < g.dim) {
#pragma unroll 8
            for (unsigned k = walker; k < n; k += 16) v += from[k * step + (k == 0 ? skip : 0u) + col];
        }
        sh[walker][lane] = v;
        __syncthreads();
        if (walker == 0 && col < g.dim) {
            v = 0.f;
#pragma unroll
            for (int k = 0; k < 16; ++k) v += sh[k][lane];
            out[col] = from_f32<T>(v);
        }
        __syncthreads();
    };
    if (blockIdx.y < 4) {
        T *const out = blockIdx.y == 0 ? g.dw_pre : blockIdx.y == 1 ? g.dw_post : blockIdx.y == 2 ? g.db_pre : g.db_post;
        if (out) join(g.part + blockIdx.y * (unsigned long long)runs * g.dim, g.dim, runs, 0u, out);
        return;
    }
    // gates one by one where they are fewer than runs
    const unsigned gates = (g.rows - 1) / g.per_gate + 1, turns = min(gates, runs);
    for (unsigned i = blockIdx.y - 4; i < turns; i += gridDim.y - 4) {
        const unsigned gate = gates <= runs ? i : (min(g.rows, (i + 1) * g.per_run) - 1) / g.per_gate;
        const unsigned first = gate * g.per_gate, end = g.rows - first > g.per_gate ? first + g.per_gate : g.rows;
        const unsigned c = first / g.per_run, last = (end - 1) / g.per_run;
        if (c == last || (gates > runs && c != i)) continue;
        // the first of its parts is the run's second, the others' their first
        join(g.part_gate + c * 2ull * g.dim, 2ull * g.dim, last - c + 1, g.dim, g.dgate + gate * g.dgate_pitch);
    }
}

}  // namespace

struct scar_resnorm {
    int device = 0;
    cudaStream_t stream = nullptr;
    scar_resnorm_config cfg{};
    unsigned sms = 148, cluster = 1, span = 8, forward_threads = 32, back_threads = 32;
    unsigned forward_fit = 1, back_fit = 1;  // CTAs of an SM
    unsigned most_runs = 1;    // of backward
    float *part = nullptr;     // [6][most_runs][dim]
    unsigned *error = nullptr; // a wait gave up; cleared when its report has been read
    uint64_t launches = 0;
    unsigned armed = 0;        // self-test: which warp of the next call gives up, from 1 on
};

namespace {

template <typename T> bool aligned16(const T *p, uint64_t pitch = 0) { return (uintptr_t)p % 16 == 0 && pitch * sizeof(T) % 16 == 0; }

constexpr unsigned kSmemOfSm = 220 * 1024;  // left to the rings of an SM's CTAs

// The ring of a kernel whose rows consist of `arrays` matrices: as many stages, between two and six, as leave room for
// `resident` CTAs on an SM, if that is possible.
// About 100 KiB of rows on their way to an SM are enough: forward of 16384 x 4096 bfloat16 takes 106 us with that and 124 us with half
// as much again (reads and writes of more rows take turns at the same memory), without a gate 87 and, with a third less, 91.
template <typename T> void set_ring(const scar_resnorm *op, NormArgs<T> &g, unsigned arrays, unsigned vectors, unsigned at_once, unsigned threads, unsigned values, unsigned resident) {
    g.array_bytes = (unsigned)(threads * values * sizeof(T) + 16);  // what the threads read, and up to 15 bytes before it
    g.stage_bytes = arrays * g.array_bytes;
    const unsigned warps = threads / 32 * g.cluster, slots = warps > 1 ? (unsigned)round_up(2 * 8 * 4 * warps, 16) : 0u;
    const unsigned other = vectors * g.array_bytes + slots;
    const unsigned room = kSmemOfSm / resident - (resident > 1 ? (unsigned)sizeof(Shared) + 1024u : 0u);  // 1 KiB a CTA is the system's
    for (const In<T> &m : g.in) g.n_in += m.p != nullptr;
    const unsigned wanted = (100u * 1024u + resident * g.n_in * g.array_bytes / 2) / (resident * g.n_in * g.array_bytes);
    g.stages = std::max(2 * at_once, std::min(std::min(kMostStages, wanted), room > other ? (room - other) / g.stage_bytes : 0u) / at_once * at_once);
    g.slot_off = g.stages * g.stage_bytes + vectors * g.array_bytes;
    g.smem = g.slot_off + slots;
    g.error = op->error;
}

template <typename T> int launch_rows(scar_resnorm *op, void (*kernel)(NormArgs<T>), NormArgs<T> g, unsigned groups, unsigned threads) {
    g.give_up = (int)std::min(op->armed, threads / 32);
    op->armed = 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = groups * g.cluster;
    cfg.blockDim = threads;
    cfg.dynamicSmemBytes = g.smem;
    cfg.stream = op->stream;
    cudaLaunchAttribute size{};
    size.id = cudaLaunchAttributeClusterDimension;
    size.val.clusterDim.x = g.cluster;
    size.val.clusterDim.y = size.val.clusterDim.z = 1;
    cfg.attrs = &size;
    cfg.numAttrs = g.cluster > 1 ? 1 : 0;
    TRAIN_TRY(cudaLaunchKernelEx(&cfg, kernel, g));
    op->launches++;
    return SCAR_OK;
}

template <typename T> auto forward_kernel(bool layer, bool vec) {
    return layer ? (vec ? k_resnorm_forward<T, true, true> : k_resnorm_forward<T, true, false>)
                 : (vec ? k_resnorm_forward<T, false, true> : k_resnorm_forward<T, false, false>);
}
template <typename T> auto backward_kernel(bool layer, bool vec, bool shared) {
    if (shared)
        return layer ? (vec ? k_resnorm_backward<T, true, true, true> : k_resnorm_backward<T, true, false, true>)
                     : (vec ? k_resnorm_backward<T, false, true, true> : k_resnorm_backward<T, false, false, true>);
    return layer ? (vec ? k_resnorm_backward<T, true, true, false> : k_resnorm_backward<T, true, false, false>)
                 : (vec ? k_resnorm_backward<T, false, true, false> : k_resnorm_backward<T, false, false, false>);
}

template <typename T> void set_ends(NormArgs<T> &g) {
    for (In<T> &m : g.in)
        if (m.p && g.rows) m.end = m.p + (g.rows - 1) / m.per * m.pitch + g.dim;
}

template <typename T> int run_forward(scar_resnorm *op, NormArgs<T> g) {
    set_ends(g);
    bool vec = g.dim * sizeof(T) % 16 == 0 && aligned16(g.y, g.y_pitch) && aligned16(g.n, g.n_pitch) && aligned16(g.w_post) && aligned16(g.b_post) &&
               aligned16(g.w_pre) && aligned16(g.b_pre);
    for (const In<T> &m : g.in) vec = vec && aligned16(m.p, m.pitch);
    const bool layer = op->cfg.kind == SCAR_RESNORM_LAYER;
    const unsigned fit = op->forward_fit;
    set_ring(op, g, kForwardIn, 0, 1, op->forward_threads, kForwardValues, fit);
    const unsigned groups = std::min(g.rows, std::max(1u, op->sms * fit / g.cluster));
    return launch_rows(op, forward_kernel<T>(layer, vec), g, groups, op->forward_threads);
}

template <typename T> int run_backward(scar_resnorm *op, NormArgs<T> g) {
    set_ends(g);
    bool vec = g.dim * sizeof(T) % 16 == 0 && aligned16(g.n, g.n_pitch) && aligned16(g.df, g.df_pitch) && aligned16(g.dgate, g.dgate_pitch) &&
               aligned16(g.w_post) && aligned16(g.b_post) && aligned16(g.w_pre);
    for (const In<T> &m : g.in) vec = vec && aligned16(m.p, m.pitch);
    const bool layer = op->cfg.kind == SCAR_RESNORM_LAYER;
    unsigned runs = 0;
    if (g.rows) {
        runs = std::min(g.rows, op->most_runs);
        g.per_run = (g.rows + runs - 1) / runs;
        runs = (g.rows + g.per_run - 1) / g.per_run;
        g.part = op->part;
        g.part_gate = op->part + 4ull * op->most_runs * g.dim;
        set_ring(op, g, kBackwardIn, layer ? 3 : 2, back_rows<T>(layer), op->back_threads, back_values(layer), op->back_fit);
        const bool shared = g.dgate && g.per_gate > 1;
        const int rc = launch_rows(op, backward_kernel<T>(layer, vec, shared), g, runs, op->back_threads);
        if (rc != SCAR_OK) return rc;
    }
    const bool gates = g.dgate && g.per_gate > 1 && runs > 1;
    if (!g.dw_pre && !g.dw_post && !g.db_pre && !g.db_post && !gates) return SCAR_OK;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((g.dim + 31) / 32, 4 + (gates ? std::min(std::min(runs, (g.rows - 1) / g.per_gate + 1), kJoinGates) : 0));
    cfg.blockDim = 512;
    cfg.stream = op->stream;
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    TRAIN_TRY(cudaLaunchKernelEx(&cfg, k_resnorm_join<T>, g, runs));
    op->launches++;
    return SCAR_OK;
}

// Shared memory for the operator's kernels, and how many of their CTAs an SM's registers hold: the fewest over the ways that rows
// may lie and gates be shared, so that the order of sums over rows depends on sizes alone.
template <typename T> int fit_kernels(scar_resnorm *op) {
    const bool layer = op->cfg.kind == SCAR_RESNORM_LAYER;
    int rc = SCAR_OK;
    const auto fit = [&](auto kernel, unsigned threads) {
        cudaFuncAttributes a{};
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemOfSm) != cudaSuccess || cudaFuncGetAttributes(&a, kernel) != cudaSuccess) {
            cudaGetLastError();
            rc = SCAR_ERR_CUDA;
            return 1u;
        }
        return std::max(1u, std::min(32u, 65536u / ((unsigned)round_up(std::max(a.numRegs, 1), 8) * threads)));
    };
    op->forward_fit = std::min(fit(forward_kernel<T>(layer, true), op->forward_threads), fit(forward_kernel<T>(layer, false), op->forward_threads));
    op->back_fit = 32;
    for (int i = 0; i < 4; ++i) op->back_fit = std::min(op->back_fit, fit(backward_kernel<T>(layer, i & 1, i >> 1), op->back_threads));
    return rc;
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
    g.cluster = op->cluster;
    g.span = op->span;
    g.per_gate = (unsigned)std::min<uint64_t>(std::max<uint64_t>(k->rows_per_gate, 1), std::max<uint64_t>(rows, 1));
    g.w_post = k->post ? static_cast<const T *>(k->d_w_post) : nullptr;
    g.b_post = k->post ? static_cast<const T *>(k->d_b_post) : nullptr;
    g.w_pre = k->pre ? static_cast<const T *>(k->d_w_pre) : nullptr;
    g.b_pre = k->pre ? static_cast<const T *>(k->d_b_pre) : nullptr;
    return g;
}
uint64_t gates_of(const scar_resnorm_block *k, uint64_t rows) { return k->rows_per_gate ? (rows + k->rows_per_gate - 1) / k->rows_per_gate : 0; }

int done(int rc) {
    if (rc != SCAR_OK) return rc;
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
        op->cluster = (unsigned)((cfg->dim + kSpan - 1) / kSpan);
        op->span = (unsigned)round_up((cfg->dim + op->cluster - 1) / op->cluster, 8);
        op->forward_threads = (unsigned)round_up((op->span + kForwardValues - 1) / kForwardValues, 32);
        const int back = back_values(cfg->kind == SCAR_RESNORM_LAYER);
        op->back_threads = (unsigned)round_up((op->span + back - 1) / back, 32);
        int rc = SCAR_OK;
        dispatch_operand(cfg->dtype, [&](auto e) { rc = fit_kernels<decltype(e)>(op); });
        if (rc != SCAR_OK) return rc;
        // runs of backward: as many as are held at a time
        op->most_runs = (unsigned)std::max<uint64_t>(1, std::min<uint64_t>(op->sms * op->back_fit / op->cluster, cfg->max_rows));
        const uint64_t floats = cfg->forward_only ? 0 : 6ull * op->most_runs * cfg->dim;
        if (cudaMalloc(&op->part, floats * sizeof(float) + 16) != cudaSuccess) {
            cudaGetLastError();
            op->part = nullptr;
            return SCAR_ERR_ALLOC;
        }
        op->error = reinterpret_cast<unsigned *>(op->part + floats);
        TRAIN_TRY(cudaMemsetAsync(op->error, 0, 16, op->stream));
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
        g.has_f = d_f != nullptr;
        g.has_gate = block->d_gate != nullptr;
        g.in[kX] = {static_cast<const T *>(d_x), x_pitch, 1};
        g.in[kF] = {static_cast<const T *>(d_f), f_pitch, 1};
        g.in[kGate] = {static_cast<const T *>(block->d_gate), block->gate_pitch, g.per_gate};
        g.y = static_cast<T *>(d_y); g.y_pitch = y_pitch;
        g.n = block->pre ? static_cast<T *>(d_n) : nullptr; g.n_pitch = n_pitch;
        rc = run_forward(op, g);
    });
    return done(rc);
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
        g.has_f = d_f != nullptr;
        g.has_gate = block->d_gate != nullptr;
        g.in[kDy] = {static_cast<const T *>(d_dy), dy_pitch, 1};
        if (block->pre) {
            g.in[kDn] = {static_cast<const T *>(d_dn), dn_pitch, 1};
            g.in[kY] = {static_cast<const T *>(d_y), y_pitch, 1};
        }
        g.in[kBackF] = {static_cast<const T *>(d_f), f_pitch, 1};
        g.in[kBackGate] = {static_cast<const T *>(block->d_gate), block->gate_pitch, g.per_gate};
        g.n = static_cast<T *>(d_dx); g.n_pitch = dx_pitch;
        g.df = static_cast<T *>(d_df); g.df_pitch = df_pitch;
        g.dgate = static_cast<T *>(d_dgate); g.dgate_pitch = dgate_pitch;
        g.dw_post = static_cast<T *>(d_dw_post);
        g.db_post = static_cast<T *>(d_db_post);
        g.dw_pre = static_cast<T *>(d_dw_pre);
        g.db_pre = static_cast<T *>(d_db_pre);
        rc = run_backward(op, g);
    });
    return done(rc);
}

int scar_resnorm_status(scar_resnorm *op) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    const int rc = check_current_device(op->device);
    if (rc != SCAR_OK) return rc;
    unsigned error = 0;
    TRAIN_TRY(cudaMemcpyAsync(&error, op->error, sizeof(error), cudaMemcpyDeviceToHost, op->stream));
    TRAIN_TRY(cudaMemsetAsync(op->error, 0, sizeof(error), op->stream));
    TRAIN_TRY(cudaStreamSynchronize(op->stream));
    return error ? SCAR_ERR_TIMEOUT : SCAR_OK;
}

int scar_resnorm_selftest_arm_timeout(scar_resnorm *op) {
    if (!op) return SCAR_ERR_INVALID_ARG;
    op->armed++;
    return SCAR_OK;
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
