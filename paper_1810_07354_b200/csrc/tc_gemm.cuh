// Matrix products of the training step on the fifth-generation tensor cores.
//
//   C(m, n) = sum_k A(m, k) B(n, k),   A, B 16-bit, C float32 in tensor memory
//
// A pair of CTAs (a cluster of two, one per SM) computes a tile of 256 x BN: each CTA stages its own 128 rows of A
// and its own half of B's rows with TMA, and one thread of the pair's first CTA issues the tcgen05.mma of both.
// Per 64 values of k a CTA reads 32 KiB for 512 clocks of matrix work; a CTA working alone on 128 x 256 would read
// 48 KiB for the same, more than L2 delivers to all SMs at once.  The kernel is persistent: pairs walk over the
// tiles, one warp loads, one issues, eight read the finished accumulators, and with two (or four) accumulators in
// tensor memory the products of the next tile run under the epilogue of the last.
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
// 1.2e-6 of itself.  dh and dw are rounded to 16 bits and need no rounds.
constexpr unsigned kRound = 16;

template <int PL> struct TcShape {
    static constexpr int BN = PL == 1 ? 256 : 128;
    static constexpr int kABytes = 128 * kBK * 2;       // one plane of one CTA's rows of A
    static constexpr int kBBytes = BN / 2 * kBK * 2;    // one plane of one CTA's rows of B
    static constexpr int kStageBytes = PL * (kABytes + kBBytes);
    static constexpr int kStages = PL == 1 ? 6 : 3;
    static constexpr int kAccs = 512 / BN;
    static constexpr int kCols = BN / 2;  // columns of one epilogue thread
    static constexpr int kSmem = kStages * kStageBytes + 1024 + 256;
};

struct TcArgs {
    CUtensorMap a, b;
    unsigned m, n, k;        // extents; the one `dyn` names is an upper bound
    int dyn;                 // 0: m, 1: k is the number of rows of this piece
    unsigned first, most;    // the piece's rows of the compacted list
    const unsigned *rows;    // rows that count (device)
    unsigned a_row0, b_row0; // where the piece starts in the row dimension of the tensor maps
    unsigned splits;
    int n_fast;              // tiles of one row of tiles run first (B is the smaller operand and stays in L2)
    int bf16;
    unsigned *error;
    // kPart
    float *part;             // [splits][m][n]
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
    // kProb, kStat
    __half *prob;
    unsigned long long prob_pitch;
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
// Arrives at the same barrier in the pair's first CTA.
__device__ __forceinline__ void mbar_arrive_leader(uint32_t bar) {
    asm volatile(
        "{\n .reg .b32 ra;\n mapa.shared::cluster.u32 ra, %0, 0;\n mbarrier.arrive.release.cluster.shared::cluster.b64 _, [ra];\n}\n" ::"r"(bar)
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

struct TileWalk {
    unsigned m, k, mt, nt, total, kb, splits;
    int n_fast;
    __device__ TileWalk(const TcArgs &g, int bn) {
        const unsigned rows = *g.rows, mine = rows > g.first ? min(g.most, rows - g.first) : 0u;
        m = g.dyn == 0 ? mine : g.m;
        k = g.dyn == 1 ? mine : g.k;
        mt = (m + kBM - 1) / kBM;
        nt = (g.n + bn - 1) / bn;
        splits = g.splits;
        total = mt * nt * splits;
        kb = (k + kBK - 1) / kBK;
        n_fast = g.n_fast;
    }
    __device__ void at(unsigned t, unsigned &mi, unsigned &ni, unsigned &s, unsigned &k0, unsigned &k1) const {
        const unsigned tiles = mt * nt;
        s = t / tiles;
        t -= s * tiles;
        if (n_fast) {
            ni = t % nt;
            mi = t / nt;
        } else {
            mi = t % mt;
            ni = t / mt;
        }
        k0 = (unsigned)((unsigned long long)kb * s / splits);
        k1 = (unsigned)((unsigned long long)kb * (s + 1) / splits);
    }
};

template <int NC> __device__ __forceinline__ void epi_part(const TcArgs &g, const float (&v)[NC], unsigned m, unsigned row, unsigned col, unsigned s) {
    if (row >= m) return;
    float *p = g.part + ((unsigned long long)s * g.m + row) * g.n + col;
    const bool vec = (g.n & 3u) == 0;
#pragma unroll
    for (int j = 0; j < NC; j += 4) {
        if (vec) {
            if (col + j < g.n) *reinterpret_cast<float4 *>(p + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + j + i < g.n) p[j + i] = v[j + i];
        }
    }
}

// Eight neighbouring results of one row: to the float32 sums over pieces, or scaled and rounded once to the output.
__device__ __forceinline__ void store_out8(const TcArgs &g, float (&x)[8], unsigned long long row, unsigned long long out_row, unsigned col, float f) {
    const unsigned left = g.n - col;
    if (g.acc) {
        float *a = g.acc + row * g.acc_pitch + col;
        const bool whole = g.acc_vec && left >= 8;
        if (!g.acc_first) {
            if (whole) {
                const float4 p = *reinterpret_cast<const float4 *>(a), q = *reinterpret_cast<const float4 *>(a + 4);
                x[0] += p.x; x[1] += p.y; x[2] += p.z; x[3] += p.w;
                x[4] += q.x; x[5] += q.y; x[6] += q.z; x[7] += q.w;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < left) x[i] += a[i];
            }
        }
        if (!g.acc_last) {
            if (whole) {
                *reinterpret_cast<float4 *>(a) = make_float4(x[0], x[1], x[2], x[3]);
                *reinterpret_cast<float4 *>(a + 4) = make_float4(x[4], x[5], x[6], x[7]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < left) a[i] = x[i];
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= f;
    const bool whole = g.out_vec && left >= 8;
    if (g.out_type == SCAR_F32) {
        float *o = static_cast<float *>(g.out) + out_row * g.out_pitch + col;
        if (whole) {
            *reinterpret_cast<float4 *>(o) = make_float4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<float4 *>(o + 4) = make_float4(x[4], x[5], x[6], x[7]);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) o[i] = x[i];
        return;
    }
    union {
        __nv_bfloat16 b[8];
        __half h[8];
        uint4 u;
        unsigned short s[8];
    } y;
    if (g.out_type == SCAR_BF16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y.b[i] = __float2bfloat16_rn(x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) y.h[i] = __float2half_rn(x[i]);
    }
    unsigned short *o = static_cast<unsigned short *>(g.out) + out_row * g.out_pitch + col;
    if (whole) {
        *reinterpret_cast<uint4 *>(o) = y.u;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) o[i] = y.s[i];
}

template <int NC> __device__ __forceinline__ void epi_out(const TcArgs &g, const float (&v)[NC], unsigned m, unsigned row, unsigned col, float f) {
    if (row >= m) return;
    const unsigned long long out_row = g.row_map ? g.row_map[g.first + row] : row;
#pragma unroll
    for (int j = 0; j < NC; j += 8) {
        if (col + j >= g.n) break;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = v[j + i];
        store_out8(g, x, row, out_row, col + j, f);
    }
}

// One row's 128 logits of this thread: their maximum, the sum of their exponentials relative to it, the label's logit,
// and with STORE the exponentials themselves.  A group whose maximum is -inf is taken relative to 0 (all zeros).
template <bool STORE, int NC>
__device__ __forceinline__ void epi_prob(const TcArgs &g, float (&v)[NC], unsigned m, unsigned row, unsigned col, unsigned group) {
    if (row >= m) return;
    const unsigned left = g.n > col ? g.n - col : 0u;
    if (left < NC) {
#pragma unroll
        for (int j = 0; j < NC; ++j)
            if (j >= left) v[j] = -INFINITY;
    }
    const unsigned at = (unsigned)g.label[g.first + row] - col;
    if (at < NC) {
        float z = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) z = j == at ? v[j] : z;
        g.label_z[g.first + row] = z;
    }
    float top = v[0];
#pragma unroll
    for (int j = 1; j < NC; ++j) top = fmaxf(top, v[j]);
    const float ref = top == -INFINITY ? 0.f : top;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    __half *p = STORE ? g.prob + (unsigned long long)row * g.prob_pitch + col : nullptr;
#pragma unroll
    for (int j = 0; j < NC; j += 8) {
        union {
            __half2 h[4];
            uint4 u;
        } y;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            // the difference first: it is small where the exponential is not, and so is its rounding
            const float e0 = ex2(fmaf(v[j + i] - ref, kLog2e, kProbLog2));
            const float e1 = ex2(fmaf(v[j + i + 1] - ref, kLog2e, kProbLog2));
            s[(i >> 1) & 3] += e0 + e1;
            if (STORE) y.h[i >> 1] = __floats2half2_rn(e0, e1);
        }
        if (STORE && j < left) *reinterpret_cast<uint4 *>(p + j) = y.u;
    }
    g.stat[(unsigned long long)row * g.stat_pitch + group] = make_float2(ref, (s[0] + s[1]) + (s[2] + s[3]));
}

template <int PL, bool A_MN, bool B_MN, Epi EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1)
k_tc_gemm(const __grid_constant__ TcArgs g) {
    using S = TcShape<PL>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ __align__(8) unsigned long long bars[2 * S::kStages + 2 * S::kAccs];
    __shared__ uint32_t tmem_base;
    constexpr bool kLogits = EPI == Epi::kProb || EPI == Epi::kStat;
    constexpr unsigned kPer = PL == 3 ? 1u : kLogits ? kRound : 0xffffffffu;  // stages per accumulator
    const uint32_t stage0 = smem_addr(smem);
    const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages;
    const uint32_t acc_full = empty + 8 * S::kStages, acc_empty = acc_full + 8 * S::kAccs;
    const unsigned warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const unsigned pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < S::kAccs; ++i) {
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
    const TileWalk walk(g, S::BN);
    bool ok = true;

    if (warp == kEpiWarps) {  // loads
        unsigned st = 0, ph = 0;
        for (unsigned t = pair; t < walk.total && ok; t += pairs) {
            unsigned mi, ni, s, k0, k1;
            walk.at(t, mi, ni, s, k0, k1);
            const int am = (int)(mi * kBM + rank * 128), bn = (int)(ni * S::BN + rank * (S::BN / 2));
            for (unsigned kb = k0; kb < k1; ++kb) {
                ok = __all_sync(0xffffffffu, mbar_wait(empty + 8 * st, ph ^ 1, g.error));
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t bar = full + 8 * st, dst = stage0 + st * S::kStageBytes;
                    if (rank == 0) mbar_expect(bar, 2 * S::kStageBytes);
                    const int kk = (int)(kb * kBK);
#pragma unroll
                    for (int p = 0; p < PL; ++p) {
                        const uint32_t da = dst + p * S::kABytes, db = dst + PL * S::kABytes + p * S::kBBytes;
                        if (A_MN) {
                            tma_load(da, &g.a, bar, am, (int)g.a_row0 + kk, p);
                            tma_load(da + 8192, &g.a, bar, am + 64, (int)g.a_row0 + kk, p);
                        } else {
                            tma_load(da, &g.a, bar, kk, (int)g.a_row0 + am, p);
                        }
                        if (B_MN) {
                            tma_load(db, &g.b, bar, bn, (int)g.b_row0 + kk, p);
                            if (S::BN == 256) tma_load(db + 8192, &g.b, bar, bn + 64, (int)g.b_row0 + kk, p);
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
            const uint32_t type = g.bf16 ? 1u : 0u;
            const uint32_t idesc = 1u << 4 | type << 7 | type << 10 | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) |
                                   (uint32_t)(S::BN >> 3) << 17 | (uint32_t)(kBM >> 4) << 24;
            const uint64_t desc_a = smem_desc<A_MN>(stage0), desc_b = smem_desc<B_MN>(stage0 + PL * S::kABytes);
            unsigned st = 0, ph = 0, ac = 0, aph = 1;
            for (unsigned t = pair; t < walk.total && ok; t += pairs) {
                unsigned mi, ni, s, k0, k1;
                walk.at(t, mi, ni, s, k0, k1);
                unsigned left = 0;  // stages left of the accumulator
                for (unsigned kb = k0; kb < k1; ++kb) {
                    const bool fresh = left == 0;
                    if (fresh) {
                        ok = __all_sync(0xffffffffu, mbar_wait(acc_empty + 8 * ac, aph, g.error));
                        if (!ok) break;
                        left = min(kPer, k1 - kb);
                    }
                    ok = __all_sync(0xffffffffu, mbar_wait(full + 8 * st, ph, g.error));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t d = tmem + ac * S::BN;
                    --left;
                    if (elect_one()) {
                        constexpr int kPairs = PL == 1 ? 1 : 6;
                        constexpr int pa[6] = {PL == 1 ? 0 : 2, 1, 0, 1, 0, 0}, pb[6] = {0, 1, 2, 0, 1, 0};
#pragma unroll
                        for (int q = 0; q < kPairs; ++q) {
                            const uint64_t da = desc_a + ((st * S::kStageBytes + pa[q] * S::kABytes) >> 4);
                            const uint64_t db = desc_b + ((st * S::kStageBytes + pb[q] * S::kBBytes) >> 4);
#pragma unroll
                            for (int k = 0; k < kBK / 16; ++k)
                                mma_pair(d, da + (k * k_step_bytes<A_MN>() >> 4), db + (k * k_step_bytes<B_MN>() >> 4), idesc,
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
                    if (left == 0 && ++ac == S::kAccs) {
                        ac = 0;
                        aph ^= 1;
                    }
                }
            }
        }
    } else {  // epilogue
        const unsigned quad = warp & 3, half = warp >> 2;
        const float f = EPI == Epi::kOut ? (g.mean ? g.scale / (float)max(*g.rows, 1u) : g.scale) : 0.f;
        unsigned ac = 0;
        for (unsigned t = pair; t < walk.total && ok; t += pairs) {
            unsigned mi, ni, s, k0, k1;
            walk.at(t, mi, ni, s, k0, k1);
            float v[S::kCols];
            const unsigned rounds = k1 > k0 ? (k1 - k0 - 1) / kPer + 1 : 0u;
            if (rounds == 0) {
#pragma unroll
                for (int j = 0; j < S::kCols; ++j) v[j] = 0.f;
            }
            // the first round is the tile's accumulator itself, later ones are added to it
            if (rounds) {
                const unsigned a = ac % S::kAccs;
                ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * a, (ac / S::kAccs) & 1, g.error));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t src = tmem + a * S::BN + half * S::kCols + (quad * 32u << 16);
#pragma unroll
                for (int j = 0; j < S::kCols; j += 32) tmem_load32(src + j, v + j);
                tmem_loaded(v);
                acc_release(acc_empty + 8 * a, lane);
                ++ac;
            }
            for (unsigned r = 1; r < rounds; ++r, ++ac) {
                const unsigned a = ac % S::kAccs;
                ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * a, (ac / S::kAccs) & 1, g.error));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t src = tmem + a * S::BN + half * S::kCols + (quad * 32u << 16);
#pragma unroll
                for (int j = 0; j < S::kCols; j += 16) {  // 16 at a time: 128 sums and 32 more registers do not fit
                    float u[16];
                    tmem_load16(src + j, u);
                    tmem_loaded(u);
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[j + i] += u[i];
                }
                acc_release(acc_empty + 8 * a, lane);
            }
            if (!ok) break;
            const unsigned row = mi * kBM + rank * 128 + quad * 32 + lane, col = ni * S::BN + half * S::kCols;
            if (EPI == Epi::kPart) epi_part(g, v, walk.m, row, col, s);
            else if (EPI == Epi::kOut) epi_out(g, v, walk.m, row, col, f);
            else epi_prob<EPI == Epi::kProb>(g, v, walk.m, row, col, 2 * ni + half);
        }
    }
    if (!ok) {  // let copies and instructions in flight end before the memory they use is given back
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
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
