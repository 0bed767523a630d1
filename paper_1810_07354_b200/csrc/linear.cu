// A hidden layer (scar_linear_* of scar.h): y = residual + m . act(x w^T + b) with its gradients.
//
//   forward    the product's epilogue adds the bias, applies the activation, the mask (computed, mask.cuh) and the residual, and
//              leaves the activation's derivative for backward; where the product's sum is split, and in float32, k_linear_join
//              does the same from the float32 sums
//   backward   k_linear_dz: dz = m . dy . slope, rounded to the operands' type (few rows or values: in two; float32: three bfloat16
//              planes), and its sums over the rows; dx = dz w and dw = dz^T x in one launch (k_tc_gemm)
//
// The derivative and not z is kept: it lies in [-0.13, 1.13], so float16 holds it to 2^-11 of itself or 2^-25 beside bfloat16 (float32 beside
// the other types, where that would show), and backward needs no activation.  Computing z again instead would be 8 rather than 6 T K N operations.
#include <algorithm>
#include <new>
#include <vector>

#include "rows.cuh"
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

// Eight products of a row to the layer's output and slope, for a whole warp (as put8).
template <typename T, int ACT>
__device__ __forceinline__ void finish8(const LayerArgs &l, T *out, unsigned long long out_pitch, bool out_vec, unsigned n, unsigned row, unsigned col, unsigned long long offset, float2 (&z)[4],
                                        bool has, bool next, bool before) {
    float2 slope[4];
    Pack8<T> r;
    if (l.res && has) r = row8(static_cast<const T *>(l.res) + row * l.res_pitch, col, n, l.res_vec);
    if (has) layer8<ACT, T>(l, offset, row, col, n, z, slope);
    if (l.slope && has) {
        const unsigned long long at = (unsigned long long)row * ((n + 7) & ~7u) + col;
        if constexpr (!kHalfSlope<T>) {
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
    put8(out + row * out_pitch, col, n, out_vec, y, has, next, before);
}

// The parts of a product whose sum was split (or its float32 result) to the layer's output: what epi_layer does without a split.
template <typename T, int ACT>
__global__ void __launch_bounds__(128) k_linear_join(const __grid_constant__ TcArgs g) {
    griddep_start();
    const LayerArgs &l = g.layer;
    const unsigned m = rows_of(g), pitch = (g.n + 7) & ~7u, groups = pitch / 8, splits = parts_of(g);
    const unsigned long long stride = (unsigned long long)g.m * pitch, total = (unsigned long long)m * groups;
    const unsigned long long offset = l.drop.on ? l.drop.at() : 0ull;
    const unsigned lane = threadIdx.x & 31;
    for (unsigned long long first = (unsigned long long)blockIdx.x * 128 + (threadIdx.x & ~31u); first < total; first += (unsigned long long)gridDim.x * 128) {
        const unsigned long long i = first + lane;
        const bool has = i < total;
        const unsigned row = total >> 32 ? (unsigned)(i / groups) : (unsigned)i / groups;
        const unsigned col = (unsigned)(i - (unsigned long long)row * groups) * 8;
        const float *p = g.part + (unsigned long long)row * pitch + col;
        float2 z[4] = {};
        if (has) {
#pragma unroll 2
            for (unsigned s = 0; s < splits; ++s) {
                const float4 a = *reinterpret_cast<const float4 *>(p + s * stride), b = *reinterpret_cast<const float4 *>(p + s * stride + 4);
                z[0] = add2(z[0], make_float2(a.x, a.y));
                z[1] = add2(z[1], make_float2(a.z, a.w));
                z[2] = add2(z[2], make_float2(b.x, b.y));
                z[3] = add2(z[3], make_float2(b.z, b.w));
            }
        }
        finish8<T, ACT>(l, static_cast<T *>(g.out), g.out_pitch, g.out_vec, g.n, row, col, offset, z, has, lane < 31 && i + 1 < total && col + 8 < pitch, lane > 0 && col > 0);
    }
}

// ---- Few rows: reading w is everything, so no tile of 256 rows is filled up with zeros.  A CTA has 32 rows of w (eight in
// float32), its eight warps take turns at the k they read, every load is 16 bytes a lane, and the warps' sums meet in shared
// memory, where the layer's epilogue takes them.
// Rows up to which w is read this way, where it lies on 16-byte boundaries and where it does not.  bfloat16, 4096 -> 16384: 32 rows 33 us,
// the product kernel 35 with 64.  2395 -> 16196: one row 46 us, 16 rows 55, 32 rows 74, the product kernel with its copies 58.  float32,
// 4096 -> 8192: 32 rows 104 us, 64 rows 203, the product kernel with its planes 131; 2161 -> 11904, 59 rows: 277 and 120.
constexpr unsigned kFewRows = 32, kFewOdd = 16;
template <typename T> struct FewArgs {
    const T *x, *w;
    unsigned long long x_pitch, w_pitch;
    unsigned rows, n, k;
    unsigned parts;  // CTAs of a cluster that share the sum over k (k_linear_few)
    int x_vec, w_vec;  // rows on 16-byte boundaries
    int act;
    T *out;
    unsigned long long out_pitch;
    int out_vec;
    LayerArgs layer;
};
// The sums `at` of eight columns of a row in every warp's block of `size` floats.
__device__ __forceinline__ void add_warps(const float *at, unsigned size, float2 (&z)[4]) {
#pragma unroll
    for (unsigned w = 0; w < 8; ++w) {
        const float4 a = *reinterpret_cast<const float4 *>(at + w * size), b = *reinterpret_cast<const float4 *>(at + w * size + 4);
        z[0] = add2(z[0], make_float2(a.x, a.y));
        z[1] = add2(z[1], make_float2(a.z, a.w));
        z[2] = add2(z[2], make_float2(b.x, b.y));
        z[3] = add2(z[3], make_float2(b.z, b.w));
    }
}
template <typename T> __device__ __forceinline__ void finish_few(const FewArgs<T> &g, unsigned row, unsigned col, float2 (&z)[4], bool has) {
    const unsigned long long offset = g.layer.drop.on ? g.layer.drop.at() : 0ull;
    if (g.act == SCAR_ACT_IDENTITY) finish8<T, SCAR_ACT_IDENTITY>(g.layer, g.out, g.out_pitch, g.out_vec, g.n, row, col, offset, z, has, false, false);
    else if (g.act == SCAR_ACT_RELU) finish8<T, SCAR_ACT_RELU>(g.layer, g.out, g.out_pitch, g.out_vec, g.n, row, col, offset, z, has, false, false);
    else if (g.act == SCAR_ACT_GELU) finish8<T, SCAR_ACT_GELU>(g.layer, g.out, g.out_pitch, g.out_vec, g.n, row, col, offset, z, has, false, false);
    else finish8<T, SCAR_ACT_SILU>(g.layer, g.out, g.out_pitch, g.out_vec, g.n, row, col, offset, z, has, false, false);
}

template <typename T> __device__ __forceinline__ void mma_16x8x16(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The accumulators of a CTA's warps (and of its cluster's CTAs) to the layer's columns from n0 on; sums:
// [8][8 * NT][kFewPad] floats of shared memory.
constexpr int RM = 2;  // 16 rows of w each
constexpr int kFewPad = 16 * RM + 4;
template <typename T, int NT>
__device__ __forceinline__ void finish_tiles(const FewArgs<T> &g, float *sums, const float (&acc)[RM][NT][4], unsigned part, unsigned n0) {
    constexpr int kTokens = 8 * NT;
    const unsigned warp = threadIdx.x / 32, lane = threadIdx.x & 31, group = lane >> 2, quad = lane & 3;
#pragma unroll
    for (int m = 0; m < RM; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[(warp * kTokens + t * 8 + quad * 2 + (i & 1)) * kFewPad + m * 16 + (i >> 1) * 8 + group] = acc[m][t][i];
    __syncthreads();
    const unsigned row = threadIdx.x / (2 * RM), col = threadIdx.x % (2 * RM) * 8;
    const bool has = row < g.rows && row < kTokens && n0 + col < g.n;
    float2 z[4] = {};
    if (has) add_warps(sums + row * kFewPad + col, kTokens * kFewPad, z);
    if (g.parts > 1) {  // the first CTA adds the others' in order
        float4 *const whole = reinterpret_cast<float4 *>(sums + row * kFewPad + col);  // of the first warp: this thread alone has read it
        if (has) {
            whole[0] = make_float4(z[0].x, z[0].y, z[1].x, z[1].y);
            whole[1] = make_float4(z[2].x, z[2].y, z[3].x, z[3].y);
        }
        cluster_sync_all();
        if (part == 0 && has) {
            const uint32_t here = smem_addr(whole);
            for (unsigned c = 1; c < g.parts; ++c) {
                float4 v[2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %4, %5;\n ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n}\n"
                                 : "=f"(v[i].x), "=f"(v[i].y), "=f"(v[i].z), "=f"(v[i].w)
                                 : "r"(here + i * 16), "r"(c)
                                 : "memory");
                z[0] = add2(z[0], make_float2(v[0].x, v[0].y));
                z[1] = add2(z[1], make_float2(v[0].z, v[0].w));
                z[2] = add2(z[2], make_float2(v[1].x, v[1].y));
                z[3] = add2(z[3], make_float2(v[1].z, v[1].w));
            }
        }
        cluster_sync_all();  // nobody leaves before it has been read
    }
    if (part == 0) finish_few(g, row, n0 + col, z, has);
}

// w's rows are the rows of 16 x 8 x 16 matrix instructions, which tcgen05's 128 would leave empty; x's rows, 8 * NT of them, the
// columns.  A lane's eight values of k of a row are the operands of two instructions: which k a slot of the
// instruction stands for does not matter as long as w and x agree.  float32 values are split into three bfloat16 planes in registers (six
// products of planes, smallest first), and every round's products begin with zeros and are added to sums in registers: an instruction
// drops the low bits of what it adds to (y of 16384 -> 8192 was off by 1.4e-5 of its norm, of positive values by 4.7e-5; so 2.2e-7).
// What a lane reads goes through shared memory, asynchronously and some rounds ahead, and back to the same lane: nothing is
// exchanged there, it takes the place of registers that the loads would wait in (4096 -> 16384 bfloat16: one row 25 us, 16 rows 29;
// loads straight to registers 24 and 39).  Rows anywhere (VEC false): a lane copies the aligned 16-byte words
// that its values begin in, reads the next one from its neighbour's copy, and the last of a row's four lanes has one word more; a word
// that begins before the matrix is copied value by value, and of one that ends behind it what lies in it.
template <typename T, int NT, int AHEAD, bool VEC> struct Few {
    static_assert(VEC || 8 * NT <= (int)kFewOdd, "more rows than that come here on 16-byte boundaries only");
    static constexpr int kRows = 2 * RM + NT;           // of a lane
    static constexpr int kWords = sizeof(T) / 2;        // of 16 bytes, eight values
    static constexpr int kMore = VEC ? 0 : 1024;        // bytes of the words behind the four lanes', a row
    static constexpr int kRow = kWords * 4096 + kMore;  // of all threads
    static constexpr int kRound = kRows * kRow;
    static constexpr int kAhead = AHEAD;                // rounds, with the one that is read
    static constexpr int kSums = 8 * 8 * NT * kFewPad * 4;
    static constexpr int kSmem = kAhead * kRound > kSums ? kAhead * kRound : kSums;
};
__device__ __forceinline__ void copy16(uint32_t to, const void *from, unsigned bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
template <typename T, int NT, int AHEAD, bool VEC>
__global__ void __launch_bounds__(256) k_linear_few(const __grid_constant__ FewArgs<T> g) {
    using S = Few<T, NT, AHEAD, VEC>;
    constexpr int PL = sizeof(T) == 4 ? 3 : 1, kPairs = PL == 1 ? 1 : 6;
    constexpr int pw[6] = {PL == 1 ? 0 : 2, 1, 0, 1, 0, 0}, px[6] = {0, 1, 2, 0, 1, 0};
    extern __shared__ __align__(16) uint8_t few_smem[];
    const unsigned warp = threadIdx.x / 32, lane = threadIdx.x & 31, group = lane >> 2, quad = lane & 3;
    const unsigned part = g.parts > 1 ? cluster_rank() : 0u, n0 = blockIdx.x / g.parts * (16 * RM);
    const T *row[S::kRows];
    bool has[S::kRows];
#pragma unroll
    for (int i = 0; i < S::kRows; ++i) {
        const unsigned r = i < 2 * RM ? n0 + i * 8 + group : (i - 2 * RM) * 8 + group;
        has[i] = r < (i < 2 * RM ? g.n : g.rows);
        row[i] = i < 2 * RM ? g.w + (has[i] ? r : 0u) * g.w_pitch : g.x + (has[i] ? r : 0u) * g.x_pitch;
    }
    griddep_start();
    uint8_t *const mine = few_smem + threadIdx.x * 16, *const more = few_smem + S::kWords * 4096 + (warp * 8 + group) * 16;
    const uint32_t slot0 = smem_addr(mine), more0 = smem_addr(more);
    const auto issue = [&](unsigned round, unsigned slot) {
        const unsigned k = ((round * g.parts + part) * 8 + warp) * 32 + quad * 8;
#pragma unroll
        for (int i = 0; i < S::kRows; ++i) {
            const uint32_t at = slot * S::kRound + i * S::kRow;
            if (VEC) {  // k is a multiple of a word's values
                const bool in = k < g.k && has[i];
                const T *p = row[i] + (k < g.k ? k : 0u);
#pragma unroll
                for (int q = 0; q < S::kWords; ++q) {
                    const bool there = in && k + q * (16 / sizeof(T)) < g.k;
                    copy16(slot0 + at + q * 4096, there ? p + q * (16 / sizeof(T)) : p, there ? 16u : 0u);
                }
            } else {
                // this lane's words, and the bytes from there to the end of the row: what lies behind it is not read
                const unsigned off = (unsigned)(uintptr_t)row[i] & 15u;
                const char *const word = reinterpret_cast<const char *>(row[i]) - off + (unsigned long long)k * sizeof(T);
                const long long to_end = has[i] ? (long long)off + ((long long)g.k - (long long)k) * (long long)sizeof(T) : 0ll;
                const int left = (int)min(max(to_end, 0ll), 64ll);
                if (word < reinterpret_cast<const char *>(i < 2 * RM ? g.w : g.x)) {
                    if (has[i])
#pragma unroll 1
                        for (unsigned j = 0; j < g.k && off + j * sizeof(T) < 16 * S::kWords; ++j)
                            *reinterpret_cast<T *>(mine + at + (off + j * sizeof(T)) / 16 * 4096 + (off + j * sizeof(T)) % 16) = row[i][j];
                } else {
#pragma unroll
                    for (int q = 0; q < S::kWords; ++q) {
                        const int n = min(max(left - q * 16, 0), 16);
                        copy16(slot0 + at + q * 4096, n ? word + q * 16 : reinterpret_cast<const char *>(row[i]) - off + 16, (unsigned)n);
                    }
                }
                if (quad == 3) {
                    const int n = min(max(left - 16 * S::kWords, 0), 16);
                    copy16(more0 + at, n ? word + 16 * S::kWords : reinterpret_cast<const char *>(row[i]) - off + 16, (unsigned)n);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // The eight values of row i from k on, zeros behind the row's end.
    const auto fetch = [&](int i, unsigned k, unsigned slot, Pack8<T> &v) {
        const uint8_t *const from = mine + slot * S::kRound + i * S::kRow;
        uint4 u[S::kWords + 1];
#pragma unroll
        for (int q = 0; q < S::kWords; ++q) u[q] = *reinterpret_cast<const uint4 *>(from + q * 4096);
        if (VEC) {
#pragma unroll
            for (int q = 0; q < S::kWords; ++q) v.u[q] = u[q];
            return;
        }
        u[S::kWords] = *reinterpret_cast<const uint4 *>(quad == 3 ? more + slot * S::kRound + i * S::kRow : from + 16);
        const unsigned off = (unsigned)(uintptr_t)row[i] & 15u;
#pragma unroll
        for (int q = 0; q < S::kWords; ++q) v.u[q] = off ? shifted(u[q], u[q + 1], off) : u[q];
        if (k + 8 > g.k || !has[i]) {
#pragma unroll
            for (unsigned j = 0; j < 8; ++j)
                if (k + j >= g.k || !has[i]) v.v[j] = from_f32<T>(0.f);
        }
    };
    const auto planes = [&](const Pack8<T> &v, uint4 (&p)[PL]) {
        if constexpr (PL == 1) {
            p[0] = v.u[0];
        } else {
            // 8 + 8 + 8 bits are exact.  The first is cut, so nothing overflows, the second rounded, so the third has either sign: what the
            // six products leave out stays below 2^-22 of a product and adds up as chance has it.
            unsigned *const to[3] = {&p[0].x, &p[1].x, &p[2].x};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 x = make_float2(v.v[2 * j], v.v[2 * j + 1]);
                const float2 c0 = make_float2(__uint_as_float(__float_as_uint(x.x) & 0xffff0000u), __uint_as_float(__float_as_uint(x.y) & 0xffff0000u));
                const float2 r1 = add2(x, make_float2(-c0.x, -c0.y));
                __nv_bfloat16 b1[2];
                Two<__nv_bfloat16>::put(b1, r1);
                const float2 c1 = Two<__nv_bfloat16>::get(b1), r2 = add2(r1, make_float2(-c1.x, -c1.y));
                to[0][j] = __byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x7632);
                to[1][j] = *reinterpret_cast<const unsigned *>(b1);
                to[2][j] = __byte_perm(__float_as_uint(r2.x), __float_as_uint(r2.y), 0x7632);
            }
        }
    };
    using M = typename std::conditional<PL == 3, __nv_bfloat16, T>::type;
    float acc[RM][NT][4] = {};
    const unsigned rounds = (g.k + 256 * g.parts - 1) / (256 * g.parts);
#pragma unroll 1
    for (int i = 0; i < S::kAhead - 1; ++i) issue(i, i);
    unsigned slot = 0;
#pragma unroll 1
    for (unsigned r = 0; r < rounds; ++r) {
        if (!VEC) __syncwarp();  // the neighbours have read the slot that is filled now
        issue(r + S::kAhead - 1, slot ? slot - 1 : S::kAhead - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(S::kAhead - 1) : "memory");
        if (!VEC) __syncwarp();
        const unsigned k = ((r * g.parts + part) * 8 + warp) * 32 + quad * 8;
        uint4 a[2 * RM][PL];
        Pack8<T> v;
#pragma unroll
        for (int i = 0; i < 2 * RM; ++i) {
            fetch(i, k, slot, v);
            planes(v, a[i]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            uint4 b[PL];
            fetch(2 * RM + t, k, slot, v);
            planes(v, b);
#pragma unroll
            for (int m = 0; m < RM; ++m) {
                float fresh[4] = {};
                float(&d)[4] = PL == 1 ? acc[m][t] : fresh;
#pragma unroll
                for (int q = 0; q < kPairs; ++q) {
                    const uint4 &p = a[2 * m][pw[q]], &o = a[2 * m + 1][pw[q]], &c = b[px[q]];
                    mma_16x8x16<M>(d, p.x, o.x, p.y, o.y, c.x, c.y);
                    mma_16x8x16<M>(d, p.z, o.z, p.w, o.w, c.z, c.w);
                }
                if (PL == 3) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][t][i] += fresh[i];
                }
            }
        }
        if (++slot == S::kAhead) slot = 0;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    finish_tiles<T, NT>(g, reinterpret_cast<float *>(few_smem), acc, part, n0);
}

// float32, up to four rows: eight rows of w, the products on the ordinary cores, two at an instruction.  A lane's four values of k of a row
// are one load (VEC: one or two rows, with w's on 16-byte boundaries; 4000 -> 4096, one row: 7.8 us) or lie 32 apart, so that neighbouring
// lanes have neighbours wherever rows begin (9.2; four rows of x leave the first form too few registers: 4096 -> 16384 71 us, this one 48;
// 578 -> 9491 with rows 581 apart 9, in planes 24).
template <int TT, bool VEC>
__global__ void __launch_bounds__(256) k_linear_few32(const __grid_constant__ FewArgs<float> g) {
    constexpr int R = 8, V = R * TT;
    __shared__ __align__(16) float sh[8][TT][R];
    griddep_start();
    const unsigned warp = threadIdx.x / 32, lane = threadIdx.x & 31, n0 = blockIdx.x * R;
    const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
    float2 acc[R][TT];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[r][t] = both(0.f);
    for (unsigned k = warp * 128 + lane * (VEC ? 4 : 1); k < g.k; k += 1024) {  // VEC: a multiple of 4, as g.k
        const auto apart = [&](const float *p) {
            return make_float4(p[0], k + 32 < g.k ? p[32] : 0.f, k + 64 < g.k ? p[64] : 0.f, k + 96 < g.k ? p[96] : 0.f);
        };
        float4 w[R], x[TT];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float *p = g.w + (n0 + r) * g.w_pitch + k;
            w[r] = n0 + r >= g.n ? none : VEC ? *reinterpret_cast<const float4 *>(p) : apart(p);
        }
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const float *p = g.x + t * g.x_pitch + k;
            x[t] = t >= (int)g.rows ? none : !VEC ? apart(p) : g.x_vec ? *reinterpret_cast<const float4 *>(p) : make_float4(p[0], p[1], p[2], p[3]);
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = 0; t < TT; ++t)
                acc[r][t] = fma2(make_float2(w[r].z, w[r].w), make_float2(x[t].z, x[t].w), fma2(make_float2(w[r].x, w[r].y), make_float2(x[t].x, x[t].y), acc[r][t]));
    }
    // lanes halve what they carry at every exchange, until each has some lanes' sum of one value
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = acc[i % R][i / R].x + acc[i % R][i / R].y;
#pragma unroll
    for (int o = 16, n = V / 2; o; o >>= 1, n >>= 1) {
        if (n == 0) {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
            continue;
        }
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            if (i >= n) continue;
            const float keep = lane & o ? v[i + n] : v[i], give = lane & o ? v[i] : v[i + n];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    constexpr unsigned kLanes = 32 / V;  // with the same value
    if (lane % kLanes == 0) (&sh[warp][0][0])[lane / kLanes] = v[0];
    __syncthreads();
    const unsigned t = threadIdx.x;
    if (t >= 32) return;
    const bool has = t < TT && t < g.rows;
    float2 z[4] = {};
    if (has) add_warps(&sh[0][t][0], V, z);
    finish_few(g, t, n0, z, has);
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
    unsigned long long plane;  // of three in float32, of two in 16 bits, or 0 there: one
    float *part;         // [CTAs of a strip][np]
    T *dbias;            // or nullptr
    unsigned *left;      // per strip: CTAs that are through
};
// Rows of a warp under way together, and CTAs of an SM that leave the compiler 64 registers: 8192 x 16384 bfloat16 with a mask takes 127 us
// (6.3 TB/s); four rows and two CTAs 144, two and three 171, one and six 139.
constexpr int kDzRows = 2, kDzCtas = 4;
template <typename T>
__global__ void __launch_bounds__(256, kDzCtas) k_linear_dz(const __grid_constant__ DzArgs<T> g) {
    __shared__ float sums[8][256];
    __shared__ bool last;
    griddep_start();
    const unsigned lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 256 + lane * 8;
    const unsigned r1 = min(g.rows, (blockIdx.y + 1) * g.per_cta);
    const unsigned long long offset = g.drop.on ? g.drop.at() : 0ull;
    using S = typename std::conditional<kHalfSlope<T>, __half, float>::type;
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
                    Pack8<T> hi;
                    hi.u[0] = pack8<T>(z);
                    *reinterpret_cast<uint4 *>(o) = hi.u[0];
                    if (g.plane) {  // what the rounding left
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 h = Two<T>::get(hi.v + 2 * j);
                            z[j].x = isinf(h.x) ? 0.f : z[j].x - h.x;
                            z[j].y = isinf(h.y) ? 0.f : z[j].y - h.y;
                        }
                        *reinterpret_cast<uint4 *>(o + g.plane) = pack8<T>(z);
                    }
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
        if (c < g.np) g.part[blockIdx.y * (unsigned long long)g.np + c] = v;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicInc(g.left + blockIdx.x, gridDim.y - 1) == gridDim.y - 1;
        __syncthreads();
        if (!last) return;
        __threadfence();
        // four columns a thread, four threads a column
        const unsigned c4 = blockIdx.x * 256 + (threadIdx.x & 63) * 4, from = threadIdx.x >> 6;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c4 < g.np) {
#pragma unroll 8
            for (unsigned k = from; k < gridDim.y; k += 4) {
                const float4 p = __ldcg(reinterpret_cast<const float4 *>(g.part + k * (unsigned long long)g.np + c4));
                a.x += p.x; a.y += p.y; a.z += p.z; a.w += p.w;
            }
        }
        *reinterpret_cast<float4 *>(&sums[from][(threadIdx.x & 63) * 4]) = a;
        __syncthreads();
        v = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
    }
    if (c < g.n) g.dbias[c] = from_f32<T>(v);
}

// Two matrices of d columns from rows of `src_pitch` on 16-byte boundaries to their places, a warp per row.
template <typename T>
__global__ void __launch_bounds__(256) k_linear_unplace(const T *a, T *to_a, unsigned long long pitch_a, unsigned na, const T *b, T *to_b, unsigned long long pitch_b, unsigned nb,
                                                        unsigned long long src_pitch, unsigned d) {
    griddep_start();
    for (unsigned long long r = blockIdx.x * 8ull + (threadIdx.x >> 5); r < (unsigned long long)na + nb; r += gridDim.x * 8ull) {
        if (r < na) unplace_row(a + r * src_pitch, to_a + r * pitch_a, d);
        else unplace_row(b + (r - na) * src_pitch, to_b + (r - na) * pitch_b, d);
    }
}

// 16 bits: calls whose dz goes to the products as two values, the second one what the first one's rounding left: of few rows, and of few
// values of dz.  That rounding comes on top of the results' own: together they are off by 1.41 times the latter alone where dz has
// many values, by up to 1.9 times where it has few (worst of 12 for 17, 128, 512, 1024, 2048 values: 1.9, 1.6, 1.63, 1.53, 1.45).  It takes more
// launches: 16 x 4096 -> 4096 35 us, 17 rows 28; 32 x 512 -> 32 20 us, rounded once 13.
constexpr unsigned kFineRows = 16, kFineValues = 2048;
bool takes_two(uint64_t rows, uint64_t n) { return rows <= kFineRows || rows * n <= kFineValues; }

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
    unsigned short *twice = nullptr;  // [2][such a call's rows][kp]: x's rows, and again
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

uint64_t slope_size(const scar_linear *op) { return op->cfg.dtype == SCAR_BF16 ? 2 : 4; }
bool has_slope(const scar_linear *op) { return op->cfg.activation != SCAR_ACT_IDENTITY; }

// x and w as the products read them: in place, or copied.
struct Operands {
    Operand x, w;
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

// f(kernel, NT, AHEAD, whether rows lie on 16-byte boundaries, shared memory) for every instance: two or three CTAs of an SM where that
// leaves three rounds or more, else one.
template <typename T, int NT, int AHEAD, bool VEC, typename F> void one_few(F &&f) { f(k_linear_few<T, NT, AHEAD, VEC>, NT, AHEAD, VEC, (unsigned)Few<T, NT, AHEAD, VEC>::kSmem); }
template <typename T, typename F> void for_few(F &&f) {
    if constexpr (sizeof(T) == 2) {
        one_few<T, 1, 4, true>(f);
        one_few<T, 2, 3, true>(f);
        one_few<T, 2, 4, true>(f);
        one_few<T, 4, 3, true>(f);
        one_few<T, 1, 4, false>(f);
        one_few<T, 2, 3, false>(f);
    } else {
        one_few<T, 1, 2, true>(f);
        one_few<T, 2, 2, true>(f);
        one_few<T, 4, 3, true>(f);
        one_few<T, 1, 2, false>(f);
        one_few<T, 2, 2, false>(f);
    }
}
template <typename T> bool allow_few() {
    bool ok = true;
    for_few<T>([&](auto kernel, int, int, bool, unsigned smem) { ok = ok && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess; });
    return ok;
}
template <typename T> void run_few(scar_linear *op, FewArgs<T> g) {
    const unsigned tiles = (g.n + 31) / 32, rounds = (g.k + 255) / 256;
    if constexpr (sizeof(T) == 4) {
        if (g.rows <= 4) {
            auto kernel = g.rows > 2 ? k_linear_few32<4, false> : g.rows == 2 ? (g.w_vec ? k_linear_few32<2, true> : k_linear_few32<2, false>)
                                                                : (g.w_vec ? k_linear_few32<1, true> : k_linear_few32<1, false>);
            launch(op, kernel, dim3((g.n + 7) / 8), 256, 0, g);
            return;
        }
    }
    // A CTA for every SM is enough, and with few rows of w the sum over k is shared by the CTAs of a cluster to get there: 16384 ->
    // 2048, one row 14.0 us, 16 rows 18.5 (half as many CTAs 17.5 and 26.1; CTAs of 16 rows of w, which read x twice as often, 17.3
    // and 21.1).  Weights from memory, 60 calls.
    while (g.parts < 8 && tiles * g.parts < 2 * op->pairs && rounds >= 4 * g.parts) g.parts *= 2;
    const int nt = g.rows <= 8 ? 1 : g.rows <= 16 ? 2 : 4;
    const bool vec = g.w_vec && g.x_vec;
    // 16 bits, up to 16 rows: 96 KiB a CTA, which are two on an SM, or with more CTAs than that 72 KiB and three (16 rows, 8192 -> 4096: 15.9 us
    // with the one and 18.7 with the other; 4096 -> 32768 52.5 and 48.3).  Elsewhere there is one: up to 8 rows four rounds (8192 -> 4096
    // 15.0 us, three 17.5, six 18.0; 4096 -> 32768 47.9, 47.7, 53.5), up to 32 rows three (4096 -> 32768 57.5 us, two 61.9, four 66.2;
    // 16384 -> 2048 20.9, 18.9, 23.2).
    const int ahead = sizeof(T) == 2 && vec && nt == 2 ? (tiles * g.parts > 4 * op->pairs ? 3 : 4) : 0;
    for_few<T>([&](auto kernel, int t, int a, bool v, unsigned smem) {
        if (t == nt && v == vec && (!ahead || a == ahead)) launch_clusters(op, kernel, dim3(tiles * g.parts), 256, smem, g.parts, g);
    });
}

template <typename T>
int run_forward(scar_linear *op, const T *x, uint64_t xp, const T *w, uint64_t wp, const T *bias, const T *res, uint64_t rp, const DropRule &drop,
                unsigned rows, T *y, uint64_t yp, void *slope) {
    constexpr int PL = sizeof(T) == 4 ? 3 : 1;
    const unsigned K = (unsigned)op->cfg.in_features, N = (unsigned)op->cfg.out_features;
    LayerArgs layer{};
    layer.slope = slope;
    layer.bias = bias;
    layer.bias_vec = (uintptr_t)bias % 16 == 0;
    layer.res = res;
    layer.res_pitch = rp;
    layer.res_vec = rows_aligned(res, rp, sizeof(T));
    layer.drop = drop;
    if (rows <= kFewRows) {
        const bool words = K * sizeof(T) % 16 == 0;
        FewArgs<T> f{x, w, xp, wp, rows, N, K, 1, words && rows_aligned(x, rows > 1 ? xp : 0, sizeof(T)), words && rows_aligned(w, N > 1 ? wp : 0, sizeof(T)),
                     op->cfg.activation, y, yp, rows_aligned(y, yp, sizeof(T)), layer};
        if (PL == 1 && f.w_vec && !f.x_vec && (uint64_t)rows * K * 2 <= op->part_bytes) {  // with a copy of x alone, in the parts' room
            const Copy<T> a{x, xp, rows, false, reinterpret_cast<unsigned short *>(op->part), 0}, none{x, xp, 0, false, nullptr, 0};
            launch(op, k_linear_place<T>, (unsigned)std::min<uint64_t>(((uint64_t)rows * (K / 8) + 255) / 256, 16 * op->pairs), 256, 0, a, none, K, K);
            f.x = reinterpret_cast<const T *>(op->part);
            f.x_pitch = K;
            f.x_vec = 1;
        }
        if (rows <= kFewOdd || (f.w_vec && f.x_vec)) {
            run_few(op, f);
            return SCAR_OK;
        }
    }
    Operands o;
    int rc = place(op, x, xp, w, wp, rows, true, true, &o);
    if (rc != SCAR_OK) return rc;
    TcArgs g = product(op, rows, N, K, 0);
    if ((rc = make_map(op, &g.a, o.x, 128)) != SCAR_OK || (rc = make_map(op, &g.b, o.w, kBN / 2)) != SCAR_OK) return rc;
    g.out = y;
    g.out_pitch = yp;
    g.out_vec = rows_aligned(y, yp, sizeof(T));
    LayerArgs &l = g.layer;
    l = layer;
    choose_splits(op, g, PL == 3 ? 0.f : kLaunchS);  // float32 has that launch in any case
    dispatch_activation(op->cfg.activation, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        // Rows off 16-byte boundaries go through float32 and the join where that has room: its threads lie along the rows, the product's
        // across them (1537 x 1001 -> 2003 float16 with such rows, from cold caches: 14 + 11 us against 46).  A tensor map's store clips rows to
        // whole 16-byte words only.
        const bool whole = g.out_vec && N % 8 == 0, parts = (!whole || (res && !l.res_vec)) && (uint64_t)rows * op->np * 4 <= op->part_bytes;
        if (PL == 1 && g.splits == 1 && !parts) {
            g.c_map = whole;
            if (g.c_map) rc = make_map(op, &g.c, {y, N, rows, rows > 1 ? yp : op->np, 1, 0}, 32, 2, 64);
            if (rc == SCAR_OK && slope) rc = make_map(op, &l.slope_map, {slope, op->np, rows, op->np, 1, 0}, 32, (unsigned)slope_size(op), 64);
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
        if (dw) TRAIN_TRY(cudaMemset2DAsync(dw, (N > 1 ? dwp : K) * sizeof(T), 0, K * sizeof(T), N, op->stream));
        if (dbias) TRAIN_TRY(cudaMemsetAsync(dbias, 0, N * sizeof(T), op->stream));
        return SCAR_OK;
    }
    // dy itself where nothing changes it
    const bool direct = PL == 1 && !slope && !drop.on && rows_aligned(dy, dyp, 2);
    const bool fine = PL == 1 && !direct && takes_two(rows, N) && 2ull * rows * op->kp * 4 <= op->part_bytes;
    const uint64_t dz_rows = std::max<uint64_t>(op->cfg.max_rows, 1);
    if (!direct || dbias) {
        const unsigned strips = (N + 255) / 256;
        const unsigned per = (unsigned)round_up((rows + op->dz_ctas - 1) / op->dz_ctas, 8);
        const DzArgs<T> a{dy, dyp, rows_aligned(dy, dyp, sizeof(T)), slope, rows, N, (unsigned)op->np, per, drop, direct ? nullptr : op->dz, PL == 3 ? dz_rows * op->np : fine ? rows * op->np : 0,
                          op->sums, dbias, op->left};
        launch(op, k_linear_dz<T>, dim3(strips, (rows + per - 1) / per), 256, 0, a);
    }
    if (!dx && !dw) return SCAR_OK;
    Operands o;
    if ((rc = place(op, x, xp, w, wp, rows, dw && !fine, dx != nullptr, &o)) != SCAR_OK) return rc;
    const unsigned dz_n = fine ? 2 * rows : rows;
    const Operand dz = direct ? Operand{dy, N, rows, rows > 1 ? dyp : op->np, 1, 0} : Operand{op->dz, N, dz_n, op->np, PL, dz_rows * op->np};
    if (fine && dw) {
        const Copy<T> a{x, xp, rows, rows_aligned(x, xp, 2), op->twice, 0}, b{x, xp, rows, a.vec, op->twice + rows * op->kp, 0};
        o.x = {op->twice, K, dz_n, op->kp, 1, 0};
        launch(op, k_linear_place<T>, (unsigned)std::min<uint64_t>((2 * rows * (op->kp / 8) + 255) / 256, 16 * op->pairs), 256, 0, a, b, K, (unsigned)op->kp);
    }
    if (fine && dx) {  // one product of both values' rows (they fill no tile of 256), joined with its parts
        TcArgs g = product(op, dz_n, K, N, 0);
        if ((rc = make_map(op, &g.a, dz, 128)) != SCAR_OK || (rc = make_map(op, &g.b, o.w, 64)) != SCAR_OK) return rc;
        choose_splits(op, g, 0.f);
        launch_tc<PL, false, true, Epi::kPart>(op, g);
        g.out = dx;
        g.out_pitch = dxp;
        g.out_vec = rows_aligned(dx, dxp, sizeof(T));
        g.m = g.most = rows;
        g.twice = 1;
        launch(op, k_join_parts, (unsigned)std::min<uint64_t>(((uint64_t)rows * ((K + 3) / 4) + 127) / 128, 32 * op->pairs), 128, 0, g);
        if (!dw) return SCAR_OK;
        dx = nullptr;
    }
    TcArgs dxg = product(op, rows, K, N, 0), dwg = product(op, N, K, dz_n, 1);
    // Results of long sums whose rows do not lie on 16-byte boundaries would be stored in pieces of lines: where the parts' room holds
    // them they go there, and from there to their places.  dw alone may go through the room of w's copy, which dx is done
    // with by then.
    // A sum that is worth splitting on its own is joined into any place directly, or stored there.
    const auto split = [&](TcArgs &g) {
        choose_splits(op, g, kLaunchS);
        return g.splits > 1;
    };
    const bool dx_split = dx && split(dxg), dw_split = dw && split(dwg);
    const bool dx_odd = dx && !dx_split && !rows_aligned(dx, dxp, sizeof(T)), dw_odd = dw && !dw_split && !rows_aligned(dw, dwp, sizeof(T));
    const uint64_t dx_room = dx_odd ? round_up((uint64_t)rows * op->kp * sizeof(T), 256) : 0, dw_room = dw_odd ? (uint64_t)N * op->kp * sizeof(T) : 0;
    const bool through = (dx_odd || dw_odd) && dx_room + dw_room <= op->part_bytes;
    const bool through_w = dw_odd && !through && op->w;
    const auto result = [&](TcArgs &g, T *out, uint64_t pitch, unsigned n, bool other, void *room) {
        g.out = other ? room : out;
        g.out_pitch = other ? op->kp : pitch;
        g.out_vec = other || rows_aligned(out, pitch, sizeof(T));
        g.c_map = other || (g.out_vec && K * sizeof(T) % 16 == 0);
        return g.c_map ? make_map(op, &g.c, {g.out, K, n, n > 1 ? g.out_pitch : op->kp, 1, 0}, 32, sizeof(T), PL == 1 ? 64 : 128) : SCAR_OK;
    };
    T *const room = reinterpret_cast<T *>(op->part), *const dw_at = through_w ? reinterpret_cast<T *>(op->w) : room + dx_room / sizeof(T);
    if (dx) {
        if ((rc = make_map(op, &dxg.a, dz, 128)) != SCAR_OK || (rc = make_map(op, &dxg.b, o.w, 64)) != SCAR_OK) return rc;
        if ((rc = result(dxg, dx, dxp, rows, through && dx_odd, room)) != SCAR_OK) return rc;
    }
    if (dw) {
        if ((rc = make_map(op, &dwg.a, dz, 64)) != SCAR_OK || (rc = make_map(op, &dwg.b, o.x, 64)) != SCAR_OK) return rc;
        if ((rc = result(dwg, dw, dwp, N, (through && dw_odd) || through_w, dw_at)) != SCAR_OK) return rc;
    }
    if (through) {  // split ones first: the others then take the parts' room
        if (dx_split) launch_out<PL, false>(op, dxg);
        if (dw_split) launch_out<PL, true>(op, dwg);
        const bool left_dx = dx && !dx_split, left_dw = dw && !dw_split;
        if (left_dx && left_dw) launch_both<PL>(op, dxg, dwg);
        else if (left_dx) launch_tc<PL, false, true, Epi::kOut>(op, dxg);
        else if (left_dw) launch_tc<PL, true, true, Epi::kOut>(op, dwg);
    } else if (dx && dw) {
        // One launch for both leaves sums unsplit that were to be, and rows anywhere to the product.  16 bits are as well off with that (bfloat16,
        // 3000 x 300 -> 3000 backward 48 us and split 55, 4096 x 100 -> 4096 61 and 61, 8192 x 100 -> 8192 143 and 157), float32 is not (2000 x 301
        // -> 2000: 92 and 79).
        const bool split_odd = (dx_split && !dxg.out_vec) || (dw_split && !dwg.out_vec);
        launch_grads<PL>(op, dxg, dwg, through_w || (PL == 3 && split_odd));
    } else if (dx) {
        launch_out<PL, false>(op, dxg);
    } else {
        launch_out<PL, true>(op, dwg);
    }
    const unsigned n0 = through && dx_odd ? rows : 0u, n1 = (through && dw_odd) || through_w ? N : 0u;
    if (n0 + n1)
        launch(op, k_linear_unplace<T>, (unsigned)std::min<uint64_t>(((uint64_t)n0 + n1 + 7) / 8, 32 * op->pairs), 256, 0, room, dx, dxp, n0, dw_at, dw, dwp, n1, op->kp, K);
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
    if (c.dtype == SCAR_BF16 ? !allow_few<__nv_bfloat16>() : c.dtype == SCAR_F16 ? !allow_few<__half>() : !allow_few<float>()) return SCAR_ERR_CUDA;
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
    // rows of a call that takes two values of dz
    const uint64_t fine = std::min<uint64_t>(std::min(T, op->part_bytes / (8 * op->kp)), std::max<uint64_t>(kFineRows, kFineValues / c.out_features));
    struct {
        void **p;
        uint64_t bytes;
    } const want[] = {
        {(void **)&op->rec, sizeof(LinearRecord)}, {(void **)&op->part, op->part_bytes}, {(void **)&op->left, 4 * strips},
        {(void **)&op->sums, c.forward_only ? 0 : 4ull * op->dz_ctas * op->np}, {(void **)&op->dz, c.forward_only ? 0 : std::max(op->planes * T, f32 ? 0 : 2 * fine) * op->np * 2}, {(void **)&op->twice, c.forward_only || f32 ? 0 : 2 * fine * op->kp * 2},
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
