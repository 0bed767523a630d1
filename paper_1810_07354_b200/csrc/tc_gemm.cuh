// Matrix products of the training step on the fifth-generation tensor cores.
//
//   C(m, n) = sum_k A(m, k) B(n, k),   A, B 16-bit, C float32 in tensor memory
//
// A pair of CTAs (a cluster of two, one per SM) computes a tile of 256 x 256: each CTA stages its own 128 rows of A
// and its own half of B's rows with TMA, and one thread of the pair's first CTA issues the tcgen05.mma of both.
// Per 64 values of k a CTA reads 32 KiB for 512 clocks of matrix work; a CTA working alone on 128 x 256 would read
// 48 KiB for the same, more than L2 delivers to all SMs at once.  The kernel is persistent: pairs walk over the
// tiles, one warp loads, one issues, eight read the finished accumulators, and with two accumulators in tensor memory the
// products of the next tile run under the epilogue of the last.  Shared memory is the next limit: per 512 clocks a CTA
// writes 32 KiB and its matrix unit reads 32 KiB, which is all of its 128 bytes a clock; a 256 x 128 tile would read
// half as much again (and ran at three quarters of the rate).
//
// An operand may be stored with k contiguous ("K-major") or with its own dimension contiguous ("MN-major"): the
// logits, dh and dw all read h, w and dz where they lie, without a transposed copy.
//
// float32 operands come as three bfloat16 planes x = x0 + x1 + x2 (8 + 8 + 8 bits of the significand).  Six of the
// nine plane products are kept, smallest first; the others are below 2^-25 of the product.  Every 64 values of k
// (24 instructions) have an accumulator of their own and are summed in the epilogue's registers in float32, because
// an accumulator in tensor memory drops the low bits of each of the many additions it takes.
#pragma once
#include <cuda.h>

#include "train_common.cuh"

namespace scar {

constexpr int kBM = 256, kBK = 64;  // a pair's rows of A, and k per stage
constexpr int kEpiWarps = 8;
constexpr int kGemmThreads = (kEpiWarps + 2) * 32;
constexpr unsigned long long kWaitNs = 2000000000ull;  // a wait inside the kernel gives up after two seconds

enum class Epi { kPart, kOut, kProb, kStat };

// The logits of 16-bit operands (Epi::kProb, kStat) are summed in registers over rounds of this many stages (1024
// values of k, 64 instructions): in one accumulator over a dim of 4096 the dropped low bits put a row's loss off by
// 1.2e-6 of itself.  dh and dw are rounded to 16 bits and need no rounds: over 128000 classes one accumulator adds 3 % at most
// to the error that the two roundings (of dz and of the result) have by themselves.
constexpr unsigned kRound = 16;

template <int PL> struct TcShape {
    static constexpr int kABytes = 128 * kBK * 2;  // one plane of one CTA's rows of A, and of its half of B's
    static constexpr int kStageBytes = 2 * PL * kABytes;
    static constexpr int kStages = PL == 1 ? 6 : 2;
};
constexpr int kBN = 256;
constexpr int kAccs = 512 / kBN;
constexpr int kCols = kBN / 2;        // columns of one epilogue thread
constexpr int kWarpStage = 32 * 128;  // epilogue: 32 rows of 128 bytes per warp, on their way to memory
constexpr int kTcSmem = 6 * 2 * 128 * kBK * 2 + kEpiWarps * kWarpStage + 1024;
static_assert(TcShape<1>::kStages * TcShape<1>::kStageBytes == TcShape<3>::kStages * TcShape<3>::kStageBytes, "both fill 192 KiB");

struct TcArgs {
    CUtensorMap a, b, c;     // c: the result, where whole boxes of it can be stored (c_map)
    unsigned m, n, k;        // extents; the one `dyn` names is an upper bound
    int dyn;                 // 0: m, 1: k is the number of rows of this piece
    unsigned first, most;    // the piece's rows of the compacted list
    const unsigned *rows;    // rows that count (device)
    unsigned a_row0, b_row0; // where the piece starts in the row dimension of the tensor maps
    unsigned splits;         // 1, or more: the product then chooses for the rows it finds (pick_splits) ...
    unsigned *chosen;        // ... and leaves its choice here for the kernel that joins the parts
    unsigned pairs;          // CTA pairs the GPU holds
    unsigned most_splits;    // that fit the buffer of parts
    int planes;
    float join_s;            // time of the launch that joins parts
    int n_fast;              // tiles of one row of tiles run first (B is the smaller operand and stays in L2)
    int bf16;
    unsigned *error;
    float *loss[2];          // become NaN where a wait gives up (each may be nullptr)
    int c_map;               // kOut: the result is stored through `c` (kPart and kProb always do)
    // kPart
    float *part;             // [splits][m][n rounded up to 8]
    // kOut
    void *out;
    unsigned long long out_pitch;
    int out_type, out_vec;   // out_vec: base and pitch allow 16-byte stores
    const unsigned *row_map; // row of C -> row of out (from `first`), or nullptr
    float *acc;              // float32 sums over pieces, or nullptr when there is one piece
    unsigned long long acc_pitch;
    int acc_vec, acc_first, acc_last;
    float scale;             // of the result: scale / rows when mean
    int mean;
    // kProb, kStat, and kPart of float32 logits (stat set)
    float2 *stat;            // [row][2 * n tiles]: maximum and sum of exponentials of 128 columns
    unsigned stat_pitch;
    const int *label;        // of the compacted rows
    float *label_z;
};

// A probability is held as 2^15 exp(z - maximum of its group) in float16: 11 bits down to 2^-29 of the group's largest.
constexpr float kProbScale = 32768.f;
constexpr float kProbLog2 = 15.f;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok;
}
__device__ __forceinline__ unsigned long long now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// Bounded wait.  After kWaitNs it records the failure and returns false; the caller leaves its loop.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, unsigned *error) {
    if (mbar_try(bar, parity)) return true;
    const unsigned long long until = now_ns() + kWaitNs;
    for (unsigned i = 1;; ++i) {
        if (mbar_try(bar, parity)) return true;
        if ((i & 255u) == 0 && now_ns() > until) {
            atomicExch(error, 1u);
            return false;
        }
    }
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Arrives at the same barrier in the pair's first CTA.  Relaxed: what it reports are reads of tensor memory that are done
// (tcgen05.wait::ld); releasing would also wait for the warp's stores of the tile before, about 2000 clocks.
__device__ __forceinline__ void mbar_arrive_leader(uint32_t bar) {
    asm volatile(
        "{\n .reg .b32 ra;\n mapa.shared::cluster.u32 ra, %0, 0;\n mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [ra];\n}\n" ::"r"(bar)
        : "memory");
}
// One lane of a converged warp.  The loops below run in all lanes with warp-uniform values and only the issuing of
// copies and matrix instructions is left to one: a loop that a single lane runs keeps its descriptors in per-lane
// registers, and moving them where the instructions take them from cost 200 of 700 clocks per stage.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n selp.u32 %0, 1, 0, q;\n}\n" : "=r"(p));
    return p;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A box of the tensor map into this CTA's shared memory; its bytes are counted at the barrier of the pair's first CTA
// (bit 24 of a shared::cluster address tells the two apart).
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int plane) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(map), "r"(bar & 0xFEFFFFFFu), "r"(x), "r"(y), "r"(plane)
        : "memory");
}
// A box of 32 rows of 128 bytes from a warp's stage (whose swizzle is the tensor map's) to memory; what lies outside the
// tensor is left out.  The copy is asynchronous: stage_free waits until the stage has been read.
__device__ __forceinline__ void tma_store(const CUtensorMap *map, uint32_t src, int x, int y, int plane) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (elect_one()) {
        asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(plane) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    __syncwarp();
}
__device__ __forceinline__ void stage_free() {
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b),
        "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
// Arrives at `bar` of both CTAs once the matrix instructions issued so far are done.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
        : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, float *v) {
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
        "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(addr));
}

__device__ __forceinline__ void tmem_load16(uint32_t addr, float *v) {
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
// The loads above are done: nothing that uses their registers moves before this point.
template <int N> __device__ __forceinline__ void tmem_loaded(float (&v)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+f"(v[j]));
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Shared-memory descriptor of an operand in rows of 128 bytes, swizzled over 1024-byte groups of eight rows.
// K-major: the rows are the operand's, 64 values of k each; groups of eight rows are 1024 bytes apart.
// MN-major: the rows are values of k, 64 of the operand's own dimension each; eight values of k are 1024 bytes apart
// (stride), the next 64 of the own dimension 8192 (leading).
template <bool MN> __device__ __forceinline__ uint64_t smem_desc(uint32_t addr) {
    constexpr uint64_t lead = MN ? 8192 >> 4 : 1, stride = 1024 >> 4;
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | lead << 16 | stride << 32 | 1ull << 46 | 2ull << 61;
}
template <bool MN> __device__ constexpr uint32_t k_step_bytes() { return MN ? 2048 : 32; }  // 16 values of k

// This warp has read its part of an accumulator.
__device__ __forceinline__ void acc_release(uint32_t bar, unsigned lane) {
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncwarp();
    if (lane == 0) mbar_arrive_leader(bar);
}

// How many parts to cut the sum over k into.  In units of one pair's 64 values of k (0.28 us; six times that for planes):
// a wave of tiles costs its length and about four for the exposed part of its epilogue; parts cost their way through
// memory (6.5 TB/s) and, where one is needed, the launch that joins them (`join_s`: about 5 us in a chain of launches).
constexpr float kLaunchS = 5e-6f;
__host__ __device__ inline float unit_s(int planes) { return planes == 3 ? 1.7e-6f : 0.28e-6f; }
__host__ __device__ inline float split_cost(unsigned s, unsigned long long tiles, unsigned kb, unsigned pairs, float out_bytes, float join_s, int planes) {
    const float waves = (float)((tiles * s + pairs - 1) / pairs);
    const float cost = waves * ((float)((kb + s - 1) / s) + 4.f);
    return s == 1 ? cost : cost * 1.03f + (join_s + out_bytes * (float)(2 * s) / 6.5e12f) / unit_s(planes);
}
__host__ __device__ inline unsigned tiles_of(unsigned m, unsigned n) { return (unsigned)(((unsigned long long)m + kBM - 1) / kBM * (((unsigned long long)n + kBN - 1) / kBN)); }
constexpr unsigned kMostSplits = 32;

// The same choice for the rows that really take part, known on the device only: every lane of a warp rates one number.  Only
// the product chooses; who reads its parts takes the number from parts_of, so that no rounding of a cost can part the two.
__device__ __forceinline__ unsigned pick_splits(const TcArgs &g, unsigned m, unsigned k) {
    if (g.splits == 1) return 1;
    const unsigned s = (threadIdx.x & 31) + 1, kb = (k + kBK - 1) / kBK;
    float cost = s <= g.most_splits && s <= max(kb, 1u) ? split_cost(s, tiles_of(m, g.n), kb, g.pairs, (float)m * (float)g.n * 4.f, g.join_s, g.planes) : INFINITY;
    unsigned best = s;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float c = __shfl_xor_sync(0xffffffffu, cost, o);
        const unsigned b = __shfl_xor_sync(0xffffffffu, best, o);
        if (c < cost || (c == cost && b < best)) {
            cost = c;
            best = b;
        }
    }
    return best;
}
__device__ __forceinline__ unsigned rows_of(const TcArgs &g) {
    const unsigned rows = *g.rows;
    return rows > g.first ? min(g.most, rows - g.first) : 0u;
}

__device__ __forceinline__ unsigned parts_of(const TcArgs &g) { return g.splits == 1 ? 1u : *g.chosen; }

struct TileWalk {
    unsigned m, mt, nt, total, kb, splits;
    int n_fast;
    TileWalk() = default;
    __device__ explicit TileWalk(const TcArgs &g) {
        const unsigned mine = rows_of(g), k = g.dyn == 1 ? mine : g.k;
        m = g.dyn == 0 ? mine : g.m;
        mt = (m + kBM - 1) / kBM;
        nt = (g.n + kBN - 1) / kBN;
        splits = pick_splits(g, m, k);
        total = mt * nt * splits;
        kb = (k + kBK - 1) / kBK;
        n_fast = g.n_fast;
    }
};

// One tile (and part of its sum) of a pair's list, the same for all warps of its CTAs.
struct Turn {
    unsigned which, mi, ni, s, k0, k1;
};
// The i-th turn of a pair, or false at the end of its list.  One product: tiles in rounds over the pairs.  Two products
// that do not depend on one another, in one launch: the second one's tiles first go, in rounds, to the pairs that have a
// tile of the first one less than the others and finish early by that; what is left goes in rounds to all.
template <int N> __device__ __forceinline__ bool take_turn(const TileWalk *w, unsigned i, unsigned pair, unsigned pairs, Turn &t) {
    unsigned at = pair + i * pairs;
    t.which = 0;
    if (at >= w[0].total) {
        if (N == 1) return false;
        const unsigned full = w[0].total / pairs, late = w[0].total % pairs;  // pairs below `late` have full + 1 tiles
        const bool early = late && pair >= late;
        const unsigned n_early = late ? pairs - late : 0u, j = i - full - (pair < late ? 1u : 0u);
        const unsigned ahead = late ? min((w[0].kb + 4) / (w[N - 1].kb + 4), w[N - 1].total / n_early) : 0u;
        if (early && j < ahead) at = (pair - late) + j * n_early;
        else at = n_early * ahead + (early ? j - ahead : j) * pairs + (early ? pair - late : n_early + pair);
        if (at >= w[N - 1].total) return false;
        t.which = N - 1;
    }
    const TileWalk &k = w[t.which];
    const unsigned tiles = k.mt * k.nt;
    t.s = N == 1 ? at / tiles : 0u;
    at -= t.s * tiles;
    t.ni = k.n_fast ? at % k.nt : at / k.mt;
    t.mi = k.n_fast ? at / k.nt : at % k.mt;
    t.k0 = (unsigned)((unsigned long long)k.kb * t.s / k.splits);
    t.k1 = (unsigned)((unsigned long long)k.kb * (t.s + 1) / k.splits);
    return true;
}

// ---- Epilogue.  A thread of a warp holds 128 columns of one row.  They go to memory through 4 KiB of shared memory per
// warp, 128 bytes of 32 rows at a time, so that a store of the warp writes whole lines: rows written straight from their
// threads are 32 lines per store and took longer than the products of a tile with few values of k.  16-byte chunk c of
// row r lies at chunk c ^ (r & 7): neither the rows' owners nor the readers of lines meet in a bank.
union Chunk {
    uint4 u;
    float f[4];
    __nv_bfloat16 b[8];
    __half h[8];
    unsigned short s[8];
};
__device__ __forceinline__ uint4 *stage_at(uint8_t *stage, unsigned row, unsigned chunk) {
    return reinterpret_cast<uint4 *>(stage + row * 128 + ((chunk ^ (row & 7)) << 4));
}
template <typename F> __device__ __forceinline__ void stage_fill(uint8_t *stage, unsigned lane, F chunk) {
    stage_free();
#pragma unroll
    for (int c = 0; c < 8; ++c) *stage_at(stage, lane, c) = chunk(c);
    __syncwarp();
}
// Where the warp's rows go: `row` is this lane's row of C, `out` its row of the output.
struct EpiRows {
    unsigned m, row0;  // rows of C; first row of the warp
    unsigned out;
    __device__ __forceinline__ bool has(unsigned i) const { return row0 + i < m; }
    __device__ __forceinline__ unsigned long long to(unsigned i) const { return __shfl_sync(0xffffffffu, out, i); }
};

// Where a tile's float32 values go: a part of a split product, float32 sums over pieces, or a float32 output.
struct F32Out {
    float *p;
    unsigned long long pitch;
    unsigned cols;
    bool vec, add;  // rows on 16-byte boundaries; add to what is there
    float scale;    // of the sum
};

__device__ __forceinline__ float out_scale(const TcArgs &g) { return g.mean ? g.scale / (float)max(*g.rows, 1u) : g.scale; }
template <Epi EPI> __device__ __forceinline__ F32Out f32_out(const TcArgs &g) {
    if (EPI == Epi::kPart) return {g.part, (g.n + 7) & ~7u, (g.n + 7) & ~7u, true, false, 1.f};
    return {g.acc ? g.acc : static_cast<float *>(g.out), g.acc ? g.acc_pitch : g.out_pitch, g.n, g.acc ? g.acc_vec != 0 : g.out_vec != 0,
            g.acc && !g.acc_first, g.acc && !g.acc_last ? 1.f : out_scale(g)};
}
template <Epi EPI> __device__ __forceinline__ EpiRows epi_rows(const TcArgs &g, unsigned m, unsigned row0, unsigned s, unsigned lane) {
    EpiRows rows{m, row0, row0 + lane};
    if (EPI == Epi::kOut && g.row_map && rows.out < m) rows.out = g.row_map[g.first + rows.out];
    if (EPI == Epi::kPart) rows.out += s * g.m;
    return rows;
}

// The code below runs once per tile on eight warps that are all at different places: it is kept short (loops over chunks
// of columns stay loops), since fetching instructions was most of its time when everything was unrolled.

// 32 columns of 32 rows from the stage, kBatch stores at a time.
template <int kBatch>
__device__ __forceinline__ void flush_f32(uint8_t *stage, const F32Out &o, const EpiRows &rows, unsigned col0, unsigned lane) {
    if (o.vec) {
        const unsigned c = lane & 7, col = col0 + c * 4;
        float *const base = o.p + col;
        const bool whole = col + 4 <= o.cols;
#pragma unroll 1
        for (int h = 0; h < 32; h += 4 * kBatch) {
            Chunk x[kBatch];
            float *at[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const unsigned r = h + i * 4 + (lane >> 3);
                at[i] = base + rows.to(r) * o.pitch;
                x[i].u = *stage_at(stage, r, c);
                if (!rows.has(r) || col >= o.cols) at[i] = nullptr;
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                if (!at[i]) continue;
                if (whole) {
                    if (o.add) {
                        const float4 y = *reinterpret_cast<const float4 *>(at[i]);
                        x[i].f[0] += y.x; x[i].f[1] += y.y; x[i].f[2] += y.z; x[i].f[3] += y.w;
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) x[i].f[q] *= o.scale;
                    *reinterpret_cast<uint4 *>(at[i]) = x[i].u;
                } else {
#pragma unroll
                    for (int q = 0; q < 3; ++q)
                        if (col + q < o.cols) at[i][q] = ((o.add ? at[i][q] : 0.f) + x[i].f[q]) * o.scale;
                }
            }
        }
        return;
    }
    const unsigned col = col0 + lane;  // a line per row, wherever it begins
#pragma unroll 4
    for (unsigned r = 0; r < 32; ++r) {
        float *p = o.p + rows.to(r) * o.pitch + col;
        float x = reinterpret_cast<const float *>(stage)[r * 32 + (((lane >> 2) ^ (r & 7)) << 2) + (lane & 3)];
        if (!rows.has(r) || col >= o.cols) continue;
        if (o.add) x += *p;
        *p = x * o.scale;
    }
}

// Four neighbouring results of one row: to the float32 sums over pieces, or scaled and rounded once to the output.
__device__ __forceinline__ void store_out4(const TcArgs &g, float4 v, unsigned long long row, unsigned long long out_row, unsigned col, float f) {
    if (col >= g.n) return;
    const unsigned left = g.n - col;
    float x[4] = {v.x, v.y, v.z, v.w};
    if (g.acc) {
        float *a = g.acc + row * g.acc_pitch + col;
        const bool whole = g.acc_vec && left >= 4;
        if (!g.acc_first) {
            if (whole) {
                const float4 p = *reinterpret_cast<const float4 *>(a);
                x[0] += p.x; x[1] += p.y; x[2] += p.z; x[3] += p.w;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < left) x[i] += a[i];
            }
        }
        if (!g.acc_last) {
            if (whole) {
                *reinterpret_cast<float4 *>(a) = make_float4(x[0], x[1], x[2], x[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < left) a[i] = x[i];
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= f;
    const bool whole = g.out_vec && left >= 4;
    if (g.out_type == SCAR_F32) {
        float *o = static_cast<float *>(g.out) + out_row * g.out_pitch + col;
        if (whole) {
            *reinterpret_cast<float4 *>(o) = make_float4(x[0], x[1], x[2], x[3]);
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) o[i] = x[i];
        return;
    }
    Chunk y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (g.out_type == SCAR_BF16) y.b[i] = __float2bfloat16_rn(x[i]);
        else y.h[i] = __float2half_rn(x[i]);
    }
    unsigned short *o = static_cast<unsigned short *>(g.out) + out_row * g.out_pitch + col;
    if (whole) {
        *reinterpret_cast<uint2 *>(o) = make_uint2(y.u.x, y.u.y);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) o[i] = y.s[i];
}

// Packed 16-bit rows of 64 columns from the stage to `base` (row pitch in elements), columns [0, left) of them.
__device__ __forceinline__ void flush16(uint8_t *stage, unsigned short *base, unsigned long long pitch, bool vec, const EpiRows &rows, unsigned left, unsigned lane) {
    if (vec) {
        const unsigned c = lane & 7;
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
            const unsigned r = i + (lane >> 3);
            const unsigned long long to = rows.to(r);
            Chunk x;
            x.u = *stage_at(stage, r, c);
            if (!rows.has(r) || c * 8 >= left) continue;
            unsigned short *o = base + to * pitch + c * 8;
            if (c * 8 + 8 <= left) {
                *reinterpret_cast<uint4 *>(o) = x.u;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c * 8 + k < left) o[k] = x.s[k];
            }
        }
        return;
    }
    // any row may begin between two 4-byte words: lane l then takes columns 2l + 1 and 2l + 2, and lane 0 the first one
    const unsigned short *st = reinterpret_cast<const unsigned short *>(stage);
#pragma unroll 4
    for (unsigned r = 0; r < 32; ++r) {
        unsigned short *o = base + rows.to(r) * pitch;
        const unsigned odd = (unsigned)((uintptr_t)o >> 1) & 1u, a = 2 * lane + odd, b = a + 1;
        const unsigned short x = st[r * 64 + (((a >> 3) ^ (r & 7)) << 3) + (a & 7)];
        const unsigned short y = b < 64 ? st[r * 64 + (((b >> 3) ^ (r & 7)) << 3) + (b & 7)] : (unsigned short)0;
        if (!rows.has(r)) continue;
        if (b < 64 && b < left) *reinterpret_cast<unsigned *>(o + a) = (unsigned)x | (unsigned)y << 16;
        else if (a < left) o[a] = x;
        if (odd && lane == 0 && left) o[0] = st[r * 64 + ((r & 7) << 3)];
    }
}

// 32 columns of the last of several pieces: added to the float32 sums of the others, scaled and rounded to 16 bits.
__device__ __forceinline__ void flush_last16(uint8_t *stage, const TcArgs &g, const EpiRows &rows, unsigned col0, float f, unsigned lane) {
    const unsigned c = lane & 7;
#pragma unroll 2
    for (int i = 0; i < 32; i += 4) {
        const unsigned r = i + (lane >> 3);
        const unsigned long long to = rows.to(r);
        Chunk x;
        x.u = *stage_at(stage, r, c);
        if (rows.has(r)) store_out4(g, make_float4(x.f[0], x.f[1], x.f[2], x.f[3]), rows.row0 + r, to, col0 + c * 4, f);
    }
}

__device__ __forceinline__ uint4 pack_half8(const float *v) {
    union {
        __half2 h[4];
        uint4 u;
    } x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    return x.u;
}
__device__ __forceinline__ uint4 pack_bf8(const float *v) {
    union {
        __nv_bfloat162 h[4];
        uint4 u;
    } x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    return x.u;
}

// One row's 128 logits of this thread: their maximum, the sum of their exponentials relative to it, the label's logit; with
// KEEP the exponentials take the logits' place.  A group whose maximum is -inf is taken relative to 0 (all zeros).
template <bool KEEP> __device__ __forceinline__ void epi_stat(const TcArgs &g, float (&v)[kCols], bool mine, unsigned row, unsigned col, unsigned group) {
    const unsigned left = g.n > col ? g.n - col : 0u;
    if (left < kCols) {
#pragma unroll
        for (int j = 0; j < kCols; ++j)
            if (j >= left) v[j] = -INFINITY;
    }
    const unsigned at = mine ? (unsigned)g.label[g.first + row] - col : 0xffffffffu;
    if (at < kCols) {
        float z = 0.f;
#pragma unroll
        for (int j = 0; j < kCols; ++j) z = j == at ? v[j] : z;
        g.label_z[g.first + row] = z;
    }
    float top = v[0];
#pragma unroll
    for (int j = 1; j < kCols; ++j) top = fmaxf(top, v[j]);
    const float ref = top == -INFINITY ? 0.f : top;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
        // the difference first: it is small where the exponential is not, and so is its rounding
        const float e = ex2(fmaf(v[j] - ref, kLog2e, kProbLog2));
        s[j & 3] += e;
        if (KEEP) v[j] = e;
    }
    if (mine) g.stat[(unsigned long long)row * g.stat_pitch + group] = make_float2(ref, (s[0] + s[1]) + (s[2] + s[3]));
}

// Packed 16-bit values of 32 rows x 64 columns to memory through the result's map, 32 columns at a time: the two halves of
// the warp's stage alternate, so that one is filled while the other is read.  `half` is the one to fill next.  It changes with
// every store and with nothing else (a last column tile may need one half only, a warp without rows none), so the newest store,
// the one that may still be under way when the wait ends, never reads the half that is filled.
template <typename F> __device__ __forceinline__ void store_halves(const CUtensorMap *map, uint8_t *stage, unsigned &half, unsigned lane, bool any, unsigned cols, int col, int row0, F chunk) {
    if (!any) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (h * 32 >= cols) break;
        uint8_t *at = stage + half * 2048;
        half ^= 1;
        asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 4; ++c) *reinterpret_cast<uint4 *>(at + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)) = chunk(h * 4 + c);
        tma_store(map, smem_addr(at), col + h * 32, row0, 0);
    }
}

// N = 2 runs two products with results of their own (kOut): the first one's A is K-major, the second one's MN-major.
template <int N> struct TcSet {
    TcArgs p[N];
};
template <int PL, bool A_MN, bool B_MN, Epi EPI, int N>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1)
k_tc_gemm(const __grid_constant__ TcSet<N> set) {
    using S = TcShape<PL>;
    __shared__ TileWalk walks[N];
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ __align__(8) unsigned long long bars[2 * S::kStages + 2 * kAccs];
    __shared__ uint32_t tmem_base;
    constexpr bool kLogits = EPI == Epi::kProb || EPI == Epi::kStat;
    constexpr unsigned kPer = PL == 3 ? 1u : kLogits ? kRound : 0xffffffffu;  // stages per accumulator
    const uint32_t stage0 = smem_addr(smem);
    const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages;
    const uint32_t acc_full = empty + 8 * S::kStages, acc_empty = acc_full + 8 * kAccs;
    const unsigned warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const unsigned pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < kAccs; ++i) {
            mbar_init(acc_full + 8 * i, 1);
            mbar_init(acc_empty + 8 * i, 2 * kEpiWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kEpiWarps + 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp < N) {
        const TileWalk w(set.p[warp]);
        if (lane == 0) walks[warp] = w;
        if (EPI == Epi::kPart && lane == 0 && blockIdx.x == 0 && set.p[0].splits > 1) *set.p[0].chosen = w.splits;
    }
    __syncthreads();
    unsigned *const error = set.p[0].error;
    bool ok = true;
    Turn t;

    if (warp == kEpiWarps) {  // loads
        unsigned st = 0, ph = 0;
        for (unsigned i = 0; ok && take_turn<N>(walks, i, pair, pairs, t); ++i) {
            const TcArgs &g = set.p[N == 1 ? 0 : t.which];
            const bool a_mn = N == 1 ? A_MN : t.which == 1;
            const int am = (int)(t.mi * kBM + rank * 128), bn = (int)(t.ni * kBN + rank * (kBN / 2));
            for (unsigned kb = t.k0; kb < t.k1; ++kb) {
                ok = __all_sync(0xffffffffu, mbar_wait(empty + 8 * st, ph ^ 1, error));
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t bar = full + 8 * st, dst = stage0 + st * S::kStageBytes;
                    if (rank == 0) mbar_expect(bar, 2 * S::kStageBytes);
                    const int kk = (int)(kb * kBK);
#pragma unroll
                    for (int p = 0; p < PL; ++p) {
                        const uint32_t da = dst + p * S::kABytes, db = dst + PL * S::kABytes + p * S::kABytes;
                        if (a_mn) {
                            tma_load(da, &g.a, bar, am, (int)g.a_row0 + kk, p);
                            tma_load(da + 8192, &g.a, bar, am + 64, (int)g.a_row0 + kk, p);
                        } else {
                            tma_load(da, &g.a, bar, kk, (int)g.a_row0 + am, p);
                        }
                        if (B_MN) {
                            tma_load(db, &g.b, bar, bn, (int)g.b_row0 + kk, p);
                            tma_load(db + 8192, &g.b, bar, bn + 64, (int)g.b_row0 + kk, p);
                        } else {
                            tma_load(db, &g.b, bar, kk, (int)g.b_row0 + bn, p);
                        }
                    }
                }
                __syncwarp();
                if (++st == S::kStages) {
                    st = 0;
                    ph ^= 1;
                }
            }
        }
    } else if (warp == kEpiWarps + 1) {  // matrix instructions, first CTA of the pair
        if (rank == 0) {
            const uint32_t type = set.p[0].bf16 ? 1u : 0u;
            const uint32_t idesc0 = 1u << 4 | type << 7 | type << 10 | (B_MN ? 1u << 16 : 0u) | (uint32_t)(kBN >> 3) << 17 | (uint32_t)(kBM >> 4) << 24;
            const uint64_t desc_b = smem_desc<B_MN>(stage0 + PL * S::kABytes);
            unsigned st = 0, ph = 0, ac = 0, aph = 1;
            for (unsigned i = 0; ok && take_turn<N>(walks, i, pair, pairs, t); ++i) {
                const bool a_mn = N == 1 ? A_MN : t.which == 1;
                const uint32_t idesc = idesc0 | (a_mn ? 1u << 15 : 0u), a_step = (a_mn ? k_step_bytes<true>() : k_step_bytes<false>()) >> 4;
                const uint64_t desc_a = a_mn ? smem_desc<true>(stage0) : smem_desc<false>(stage0);
                unsigned left = 0;  // stages left of the accumulator
                for (unsigned kb = t.k0; kb < t.k1; ++kb) {
                    const bool fresh = left == 0;
                    if (fresh) {
                        ok = __all_sync(0xffffffffu, mbar_wait(acc_empty + 8 * ac, aph, error));
                        if (!ok) break;
                        left = min(kPer, t.k1 - kb);
                    }
                    ok = __all_sync(0xffffffffu, mbar_wait(full + 8 * st, ph, error));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t d = tmem + ac * kBN;
                    --left;
                    if (elect_one()) {
                        constexpr int kPairs = PL == 1 ? 1 : 6;
                        constexpr int pa[6] = {PL == 1 ? 0 : 2, 1, 0, 1, 0, 0}, pb[6] = {0, 1, 2, 0, 1, 0};
#pragma unroll
                        for (int q = 0; q < kPairs; ++q) {
                            const uint64_t da = desc_a + ((st * S::kStageBytes + pa[q] * S::kABytes) >> 4);
                            const uint64_t db = desc_b + ((st * S::kStageBytes + pb[q] * S::kABytes) >> 4);
#pragma unroll
                            for (int k = 0; k < kBK / 16; ++k)
                                mma_pair(d, da + k * a_step, db + (k * k_step_bytes<B_MN>() >> 4), idesc,
                                         q + k > 0 || !fresh);
                        }
                        mma_commit(empty + 8 * st);
                        if (left == 0) mma_commit(acc_full + 8 * ac);
                    }
                    __syncwarp();
                    if (++st == S::kStages) {
                        st = 0;
                        ph ^= 1;
                    }
                    if (left == 0 && ++ac == kAccs) {
                        ac = 0;
                        aph ^= 1;
                    }
                }
            }
        }
    } else if (warp < kEpiWarps) {  // epilogue
        const unsigned quad = warp & 3, half = warp >> 2;
        uint8_t *stage = smem + S::kStages * S::kStageBytes + warp * kWarpStage;
        constexpr bool kRegs = PL == 3 || kLogits;  // sums over rounds, or a whole row at a time: all columns in registers
        unsigned ac = 0, aph = 0;
        unsigned half_next = 0;  // of the stage, for store_halves
        for (unsigned i = 0; take_turn<N>(walks, i, pair, pairs, t); ++i) {
            const TcArgs &g = set.p[N == 1 ? 0 : t.which];
            const unsigned rounds = t.k1 > t.k0 ? (kPer == 1 ? t.k1 - t.k0 : (t.k1 - t.k0 - 1) / kPer + 1) : 0u;
            const uint32_t lanes = tmem + half * kCols + (quad * 32u << 16);
            if constexpr (kRegs) {
                float v[kCols];
                if (rounds == 0) {
#pragma unroll
                    for (int j = 0; j < kCols; ++j) v[j] = 0.f;
                }
                // the first round is the tile's accumulator itself, later ones are added to it
                if (rounds) {
                    ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * ac, aph, error));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                    for (int j = 0; j < kCols; j += 32) tmem_load32(lanes + ac * kBN + j, v + j);
                    tmem_loaded(v);
                    acc_release(acc_empty + 8 * ac, lane);
                    if (++ac == kAccs) {
                        ac = 0;
                        aph ^= 1;
                    }
                }
#pragma unroll 1
                for (unsigned r = 1; r < rounds; ++r) {
                    ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * ac, aph, error));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                    for (int j = 0; j < kCols; j += 16) {  // 16 at a time: 128 sums and 32 more registers do not fit
                        float u[16];
                        tmem_load16(lanes + ac * kBN + j, u);
                        tmem_loaded(u);
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[j + i] += u[i];
                    }
                    acc_release(acc_empty + 8 * ac, lane);
                    if (++ac == kAccs) {
                        ac = 0;
                        aph ^= 1;
                    }
                }
                if (!ok) break;
                const EpiRows rows = epi_rows<EPI>(g, walks[t.which].m, t.mi * kBM + rank * 128 + quad * 32, t.s, lane);
                const unsigned col = t.ni * kBN + half * kCols;
                if constexpr (kLogits) {
                    const unsigned row = rows.row0 + lane;
                    epi_stat<EPI == Epi::kProb>(g, v, row < rows.m, row, col, 2 * t.ni + half);
                    if constexpr (EPI == Epi::kProb) {
                        const unsigned left = g.n > col ? g.n - col : 0u;
#pragma unroll 1
                        for (int j = 0; j < 2; ++j) {
                            if (j * 64 >= left) break;
                            if (j == 0) store_halves(&g.c, stage, half_next, lane, rows.has(0), left, (int)col, (int)rows.row0, [&](int c) { return pack_half8(v + c * 8); });
                            else store_halves(&g.c, stage, half_next, lane, rows.has(0), left - 64, (int)col + 64, (int)rows.row0, [&](int c) { return pack_half8(v + 64 + c * 8); });
                        }
                    }
                } else {
                    if (EPI == Epi::kPart && g.stat) {
                        const unsigned row = rows.row0 + lane;
                        epi_stat<false>(g, v, row < rows.m, row, col, 2 * t.ni + half);
                    }
                    const F32Out o = f32_out<EPI>(g);
#pragma unroll 1
                    for (int j = 0; j < 4; ++j) {
                        if (col + j * 32 >= o.cols) break;
                        // a map stores what is staged: scaled already
                        const float f = EPI == Epi::kOut && g.c_map ? o.scale : 1.f;
                        auto fill = [&](const float *x) {
                            stage_fill(stage, lane, [&](int c) {
                                return make_uint4(__float_as_uint(x[4 * c] * f), __float_as_uint(x[4 * c + 1] * f), __float_as_uint(x[4 * c + 2] * f), __float_as_uint(x[4 * c + 3] * f));
                            });
                        };
                        if (j == 0) fill(v);
                        else if (j == 1) fill(v + 32);
                        else if (j == 2) fill(v + 64);
                        else fill(v + 96);
                        if (EPI == Epi::kPart || g.c_map) {
                            if (rows.has(0)) tma_store(&g.c, smem_addr(stage), (int)(col + j * 32), (int)rows.row0, EPI == Epi::kPart ? (int)t.s : 0);
                        } else {
                            flush_f32<2>(stage, o, rows, col + j * 32, lane);
                        }
                    }
                }
            } else {
                const EpiRows rows = epi_rows<EPI>(g, walks[t.which].m, t.mi * kBM + rank * 128 + quad * 32, t.s, lane);
                const unsigned col = t.ni * kBN + half * kCols;
                const F32Out o = f32_out<EPI>(g);
                const bool to16 = EPI == Epi::kOut && g.out_type != SCAR_F32;
                const bool last16 = to16 && g.acc && g.acc_last, pack16 = to16 && !g.acc;
                const float f = EPI == Epi::kOut ? out_scale(g) : 1.f;
                if (rounds) {
                    ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * ac, aph, error));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                }
#pragma unroll 1
                for (unsigned j = 0; j < kCols && col + j < g.n;) {
                    if (pack16) {
                        float v[64] = {};
                        if (rounds) {
                            tmem_load32(lanes + ac * kBN + j, v);
                            tmem_load32(lanes + ac * kBN + j + 32, v + 32);
                            tmem_loaded(v);
                        }
#pragma unroll
                        for (int i = 0; i < 64; ++i) v[i] *= f;
                        const bool bf = g.out_type == SCAR_BF16;
                        if (g.c_map) {
                            store_halves(&g.c, stage, half_next, lane, rows.has(0), g.n - (col + j), (int)(col + j), (int)rows.row0,
                                         [&](int c) { return bf ? pack_bf8(v + c * 8) : pack_half8(v + c * 8); });
                            j += 64;
                            continue;
                        }
                        stage_fill(stage, lane, [&](int c) { return bf ? pack_bf8(v + c * 8) : pack_half8(v + c * 8); });
                        flush16(stage, static_cast<unsigned short *>(g.out) + col + j, g.out_pitch, g.out_vec, rows, g.n - (col + j), lane);
                        j += 64;
                    } else {
                        float v[32] = {};
                        if (rounds) {
                            tmem_load32(lanes + ac * kBN + j, v);
                            tmem_loaded(v);
                        }
                        stage_fill(stage, lane, [&](int c) {
                            return make_uint4(__float_as_uint(v[4 * c]), __float_as_uint(v[4 * c + 1]), __float_as_uint(v[4 * c + 2]), __float_as_uint(v[4 * c + 3]));
                        });
                        if (EPI == Epi::kPart) {
                            if (rows.has(0)) tma_store(&g.c, smem_addr(stage), (int)(col + j), (int)rows.row0, (int)t.s);
                        } else if (last16) flush_last16(stage, g, rows, col + j, f, lane);
                        else flush_f32<8>(stage, o, rows, col + j, lane);
                        j += 32;
                    }
                }
                if (rounds) {
                    acc_release(acc_empty + 8 * ac, lane);
                    if (++ac == kAccs) {
                        ac = 0;
                        aph ^= 1;
                    }
                }
            }
        }
    }
    if (warp < kEpiWarps) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");  // this warp's stores are in memory
    if (!ok) {  // let copies and instructions in flight end before the memory they use is given back
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        // for a caller who reads no status: a loss that is written after this is NaN by the error flag
        if (lane == 0)
            for (float *loss : set.p[0].loss)
                if (loss) *loss = __int_as_float(0x7fffffff);
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();
    if (warp == kEpiWarps + 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

}  // namespace scar
