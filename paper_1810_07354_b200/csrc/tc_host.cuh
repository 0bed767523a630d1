// What the operators that multiply matrices (xent.cu, linear.cu) share around the product kernel of tc_gemm.cuh: operands and their
// copies, tensor maps, the choice of splits, launches.
#pragma once
#include <algorithm>

#include "rows.cuh"
#include "tc_gemm.cuh"

namespace scar {

// Every kernel of a call is launched while the one before it may still run; nothing is touched before that one is done.
__device__ __forceinline__ void griddep_start() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
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

// Adds the parts of a split product and does what the product's own epilogue does without a split.
static __global__ void __launch_bounds__(128)
k_join_parts(const __grid_constant__ TcArgs g) {
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

// What a handle's products need to know of it.
struct TcHost {
    int device = 0;
    cudaStream_t stream = nullptr;
    scar_dtype dtype = SCAR_F32;
    EncodeTiled encode = nullptr;
    unsigned pairs = 74;     // CTA pairs the GPU holds at a time
    unsigned planes = 1;
    float *part = nullptr;   // parts of split products, and float32 results on their way to an epilogue of their own
    uint64_t part_bytes = 0;
    uint64_t launches = 0;
    bool failed = false;
};

constexpr uint64_t kPitchEnd = 1ull << 38;  // a tensor map's row is shorter than 2^40 bytes
inline bool rows_aligned(const void *p, uint64_t pitch, unsigned elem) { return (uintptr_t)p % 16 == 0 && pitch * elem % 16 == 0; }

// The tensor map of an operand: boxes of 64 values of k by box_rows rows (K-major), or of 64 of its own dimension by 64
// values of k (MN-major; box_rows = 64); or of a result: boxes of 128 bytes (float32) or 64 (16-bit types) by 32 rows.
inline int make_map(const TcHost *op, CUtensorMap *map, const Operand &x, unsigned box_rows, unsigned elem = 2, unsigned box_bytes = 128) {
    const cuuint64_t dims[3] = {x.inner, x.rows, x.planes}, strides[2] = {x.pitch * elem, (x.planes > 1 ? x.plane : x.pitch) * elem};
    const cuuint32_t box[3] = {box_bytes / elem, box_rows, 1}, step[3] = {1, 1, 1};
    const CUtensorMapDataType type = elem == 4                      ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                     : op->dtype == SCAR_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                                 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const CUresult rc = op->encode(map, type, 3, const_cast<void *>(x.p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, box_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? SCAR_OK : SCAR_ERR_CUDA;
}

// A row on a 16-byte boundary to a row anywhere, by a warp: whole 16-byte words of the destination, its ends element by element.
template <typename T> __device__ __forceinline__ void unplace_row(const T *__restrict__ s, T *__restrict__ o, unsigned d) {
    constexpr unsigned kVec = 16 / sizeof(T);
    const unsigned lane = threadIdx.x & 31;
    const unsigned head = min(d, (unsigned)((0u - (unsigned)(uintptr_t)o) & 15u) / (unsigned)sizeof(T)), words = (d - head) / kVec, tail = head + words * kVec;
    if (lane < head) o[lane] = s[lane];
    if (tail + lane < d) o[tail + lane] = s[tail + lane];
    const uint4 *a = reinterpret_cast<const uint4 *>(s);  // head is shorter than a word: word w lies in a[w] and a[w + 1]
#pragma unroll 4
    for (unsigned w = lane; w < words; w += 32)
        *reinterpret_cast<uint4 *>(o + head + w * kVec) = head ? shifted(a[w], a[w + 1], head * (unsigned)sizeof(T)) : a[w];
}
// A matrix from such rows to rows anywhere, a warp per row.
template <typename T>
static __global__ void __launch_bounds__(256)
k_unplace(const T *__restrict__ src, unsigned long long src_pitch, unsigned n, unsigned d, T *__restrict__ dst, unsigned long long pitch) {
    griddep_start();
    for (unsigned long long r = blockIdx.x * 8ull + (threadIdx.x >> 5); r < n; r += gridDim.x * 8ull) unplace_row(src + r * src_pitch, dst + r * pitch, d);
}

// Launches a kernel of the call's chain: it may start while the one before it still runs (griddep_start waits for it).
template <typename... P, typename... A> void launch_clusters(TcHost *op, void (*kernel)(P...), dim3 grid, unsigned threads, unsigned smem, unsigned cluster, A... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = threads;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = op->stream;
    cudaLaunchAttribute attrs[2]{};
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = cluster;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    cfg.attrs = attrs;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, P(args)...) == cudaSuccess) op->launches++;
    else op->failed = true;
}
template <typename... P, typename... A> void launch(TcHost *op, void (*kernel)(P...), dim3 grid, unsigned threads, unsigned smem, A... args) {
    launch_clusters(op, kernel, grid, threads, smem, 1, args...);
}

// Sets the product's `splits`: 1, or more than 1 where cutting the sum over k pays for all the rows the call has.  Returns
// what it costs, in units of 64 values of k.
inline float choose_splits(const TcHost *op, TcArgs &g, float join_s) {
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

inline uint64_t tiles_of(const TcArgs &g) { return (uint64_t)((g.m + kBM - 1) / kBM) * ((g.n + kBN - 1) / kBN) * (g.splits > 1 ? g.most_splits : 1); }

template <int PL, bool A_MN, bool B_MN, Epi EPI> void launch_tc(TcHost *op, TcArgs g) {
    if (EPI == Epi::kPart) {
        const uint64_t pitch = round_up(g.n, 8);
        if (make_map(op, &g.c, {g.part, pitch, g.m, pitch, g.splits > 1 ? g.most_splits : 1u, g.m * pitch}, 32, 4) != SCAR_OK) op->failed = true;
    }
    const unsigned pairs = (unsigned)std::min<uint64_t>(tiles_of(g), op->pairs);
    if (pairs) launch(op, k_tc_gemm<PL, A_MN, B_MN, EPI, 1>, 2 * pairs, EpiShape<EPI>::kThreads, kTcSmem, TcSet<1>{g});
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
template <int PL, bool A_MN> void launch_out(TcHost *op, const TcArgs &g) {
    if (g.splits == 1) {
        launch_tc<PL, A_MN, true, Epi::kOut>(op, g);
        return;
    }
    launch_tc<PL, A_MN, true, Epi::kPart>(op, g);
    const uint64_t todo = (uint64_t)g.m * ((g.n + 3) / 4);
    launch(op, k_join_parts, (unsigned)std::min<uint64_t>((todo + 127) / 128, 32 * op->pairs), 128, 0, g);
}

// Two products without splits in one launch.
template <int PL> void launch_both(TcHost *op, TcArgs a, TcArgs b) {
    a.splits = b.splits = 1;
    launch(op, k_tc_gemm<PL, false, true, Epi::kOut, 2>, 2 * (unsigned)std::min<uint64_t>(tiles_of(a) + tiles_of(b), op->pairs), EpiShape<Epi::kOut>::kThreads, kTcSmem, TcSet<2>{{a, b}});
}

// dh and dw of a piece: one launch without splits, so that the second one's tiles fill the last round of the first one's
// (4096 x 32000 x 2048: 120 tiles of 500 stages leave 28 of 74 pairs idle for half of that time), unless split products
// with launches of their own are worth it (a dh of few tiles whose sum runs over very many classes).  never_one: dw goes
// through the room of w's copy, which dh still reads, or rows anywhere are better written by the kernel that joins a split sum.
template <int PL> void launch_grads(TcHost *op, TcArgs dhg, TcArgs dwg, bool never_one) {
    const float apart = choose_splits(op, dhg, kLaunchS) + choose_splits(op, dwg, kLaunchS) + kLaunchS / unit_s(PL);
    const unsigned pairs = op->pairs;
    const float tile0 = (float)((dhg.k + kBK - 1) / kBK + 4), tile1 = (float)((dwg.k + kBK - 1) / kBK + 4);
    const uint64_t tiles0 = (uint64_t)((dhg.m + kBM - 1) / kBM) * ((dhg.n + kBN - 1) / kBN), tiles1 = (uint64_t)((dwg.m + kBM - 1) / kBM) * ((dwg.n + kBN - 1) / kBN);
    // the second one's tiles fill gaps where they are the shorter ones, and come on top where they are not
    const float together = tile1 <= tile0 ? std::max(tile0, ((float)tiles0 * tile0 + (float)tiles1 * tile1) / (float)pairs)
                                          : (float)((tiles0 + pairs - 1) / pairs) * tile0 + (float)((tiles1 + pairs - 1) / pairs) * tile1;
    if (!never_one && together <= apart) {
        launch_both<PL>(op, dhg, dwg);
        return;
    }
    launch_out<PL, false>(op, dhg);
    launch_out<PL, true>(op, dwg);
}

}  // namespace scar
