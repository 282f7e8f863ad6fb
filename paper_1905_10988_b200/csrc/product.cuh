// Matrix products of 16-bit operands on the tensor cores of sm_100a with an epilogue of the caller's:
//
//   acc[m][n] = sum_k left[m][k] * right[n][k]      (binary32)
//
// Either operand may lie in memory with k or with its own index as the neighbouring one ("lines": a
// line of memory is one k), and may be a symmetric matrix of which only the blocks of 256 x 256 on
// and above the diagonal exist: a block below it is read from its mirror image with the other layout,
// which the matrix instruction takes as it is, so nothing is ever transposed.
//
// What bounds it: at full clock the path from L2 to an SM (a step of 512 cycles brings 32 KB, 64 bytes
// a cycle), with the tensor pipe active 87 to 91 % of the cycles for 4096 and more k; over a longer time
// the power cap.  8192 x 16384 x 4096: 720 to 750 us a product, 1.47 to 1.53 PFLOP/s.
//
// A pair of blocks (cta_group::2) computes tiles of 256 x 256 one after another, block r of it the
// rows from 128 r on; it brings 128 rows of either operand for every step of 64 k.  Tiles that do not fill
// a round of the chip's pairs are cut along n into two or four (product_split).  One thread of each
// block copies boxes of 64 x 64 into a ring of six stages of 32 KB, one thread of the pair's first
// block issues the matrix instructions, and eight warps read the finished tile out of TMEM, which
// holds two, while the next one is computed.  Both blocks' copies are counted by the first block's
// barrier, so the issuing thread waits once a step.
//
// A job may have several phases, each of which reads what the one before has written: the blocks wait
// for each other between them (a cooperative launch), which takes a third of the time that a launch
// does.
//
// What a caller brings is a Job: maps and layout of the operands, the units of work, and store(), which
// gets the accumulators of a row of the tile, 32 columns at a time.
#pragma once

#include <type_traits>

#include "act8_common.cuh"
#include "tensor_core.cuh"

namespace natcomp {

constexpr int kProductTile = 256;        // m and n of a pair's tile
constexpr int kProductHalf = 128;        // of a block
constexpr int kProductStep = 64;         // k
constexpr int kProductStages = 6;
constexpr int kProductWriters = 8;       // warps: four quarters of the rows, two halves of the columns
constexpr int kProductCopyWarp = kProductWriters, kProductMmaWarp = kProductWriters + 1;
constexpr int kProductThreads = 32 * (kProductWriters + 2);
constexpr int kProductPairs = 74;        // pairs of blocks that a whole chip holds at a time
constexpr uint32_t kProductBox = 64 * 128;                   // bytes of 64 x 64 values
constexpr uint32_t kProductOperand = 2 * kProductBox;        // of a block's half
constexpr uint32_t kProductStage = 2 * kProductOperand;
constexpr uint32_t kProductBars = kProductStages * kProductStage;
constexpr uint32_t kProductRows = 32 * 33 * 4;               // a writer warp's values in passing
constexpr uint32_t kProductSmem =
    kProductBars + 256 + kProductWriters * kProductRows + 1024;

// ---- copies, TMEM and shapes -----------------------------------------------------------------

// a box of 64 x 64 of one of several matrices into this block's shared memory, counted by the barrier at
// the place of `bar` in the pair's first block
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y,
                                              int z, uint32_t bar) {
    asm volatile("{\n\t"
                 ".reg .b32 first;\n\t"
                 "mapa.shared::cluster.u32 first, %5, 0;\n\t"
                 "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile"
                 ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [first];\n\t"
                 "}" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}

// 32 columns of the warp's 32 lanes; the values are there after tmem_wait32
__device__ __forceinline__ void tmem_load32(uint32_t tmem, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
                   "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
                   "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
                   "=r"(r[30]), "=r"(r[31])
                 : "r"(tmem)
                 : "memory");
}

__device__ __forceinline__ void tmem_wait32(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]),
                   "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                   "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]),
                   "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                   "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]),
                   "+r"(r[30]), "+r"(r[31])::"memory");
}

// operands of one type; lines: the contraction index runs over the lines of shared memory, else along
// them
__host__ __device__ constexpr uint32_t mma_shape_of(uint32_t m, uint32_t n, bool bf16, bool a_lines,
                                                    bool b_lines) {
    return (1u << 4) | ((uint32_t)bf16 << 7) | ((uint32_t)bf16 << 10) | ((uint32_t)a_lines << 15) |
           ((uint32_t)b_lines << 16) | ((n >> 3) << 17) | ((m >> 4) << 24);
}

__device__ __forceinline__ float exp2_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// 32 bytes at an address that is a multiple of 32
__device__ __forceinline__ Bytes32 ld_wide(const void* p) {
    Bytes32 r;
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r.v[0]), "=r"(r.v[1]), "=r"(r.v[2]), "=r"(r.v[3]), "=r"(r.v[4]),
                   "=r"(r.v[5]), "=r"(r.v[6]), "=r"(r.v[7])
                 : "l"(p)
                 : "memory");
    return r;
}

__device__ __forceinline__ void st_wide(void* p, const Bytes32& r) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r.v[0]),
                 "r"(r.v[1]), "r"(r.v[2]), "r"(r.v[3]), "r"(r.v[4]), "r"(r.v[5]), "r"(r.v[6]),
                 "r"(r.v[7])
                 : "memory");
}

// brings a map to where tensor copies look it up
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// what this thread has written to global memory is visible to the tensor copies of whoever sees what it
// does next; and what it has seen to its own
__device__ __forceinline__ void fence_global_copies() {
    asm volatile("fence.proxy.async.global;" ::: "memory");
}

__device__ __forceinline__ void grid_arrive(uint32_t* counter) {
    asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(counter) : "memory");
}

__device__ __forceinline__ uint32_t grid_arrived(const uint32_t* counter) {
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
    return v;
}

// Waits until `target` blocks have arrived; gives up after about two seconds, or where its block has.
__device__ __forceinline__ bool grid_wait(const uint32_t* counter, uint32_t target,
                                          volatile uint32_t* gave_up) {
    const long long begin = clock64();
    while (grid_arrived(counter) < target) {
        if (*gave_up) return false;
        if (clock64() - begin > 4000000000ll) {
            *gave_up = 1;
            return false;
        }
    }
    return true;
}

// Launches `kernel`, whose blocks come in pairs and wait for each other, so that all of them run at the same
// time: `grid` blocks, or as many as the device, or the part of it that the context has, holds at a time (a
// question that takes the host 0.2 us).
template <typename Kernel, typename... Args>
inline cudaError_t launch_together(Kernel kernel, dim3 grid, dim3 block, size_t smem,
                                   cudaStream_t stream, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int pairs = 0;
    const cudaError_t asked = cudaOccupancyMaxActiveClusters(&pairs, kernel, &cfg);
    if (asked != cudaSuccess) return asked;
    if (pairs < 1) return cudaErrorCooperativeLaunchTooLarge;
    if (grid.x > 2u * pairs) cfg.gridDim.x = 2u * pairs;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// map of `count` row-major matrices of 16-bit values for boxes of 64 x 64 with 128-byte swizzle; what
// lies beyond a matrix reads as 0
inline bool make_box_map(CUtensorMap* map, const void* p, bool bf16, uint64_t count, uint64_t rows,
                         uint64_t cols, uint64_t ld, uint64_t distance) {
    typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                               const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                               const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                               CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    void* f = nullptr;
    static Encode encode = nullptr;
    if (!encode) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault,
                                             &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return false;
        encode = (Encode)f;
    }
    const cuuint64_t dims[3] = {cols, rows, count};
    const cuuint64_t strides[2] = {2 * ld, 2 * (count > 1 ? distance : rows * ld)};
    const cuuint32_t box[3] = {64, 64, 1}, steps[3] = {1, 1, 1};
    return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                  const_cast<void*>(p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// ---- work ------------------------------------------------------------------------------------

// a tile's place in the product and the part of the contraction that is added up.  steps == 0: the sum
// of nothing, which is 0
struct ProductUnit {
    int m, n, z;                         // z: which of several matrices
    int k, steps;                        // from k on, in steps of 64
    int width;                           // n values: 256, 128 or 64
    uint32_t part;                       // of the job's own
};

// Tiles from `whole` on come in `parts` pieces of 256 / parts columns each.  A round of tiles that leaves
// half of the pairs idle takes about half the time in halves, although the left operand is read once more.
// Updates of five steps: 512 x 512 157 us instead of 225, 1024 x 1024 217 instead of 270, 4096 x 4096
// (256 tiles for 74 pairs) 1321 instead of 1406.
struct ProductSplit {
    uint32_t whole, parts;
    __host__ __device__ __forceinline__ uint32_t units(uint32_t tiles) const {
        return whole + (tiles - whole) * parts;
    }
    // the tile of unit u; its first column in the tile and their number
    __device__ __forceinline__ uint32_t tile(uint32_t u, int& column, int& width) const {
        column = 0;
        width = kProductTile;
        if (u < whole) return u;
        const uint32_t t = (u - whole) / parts;
        width = kProductTile / (int)parts;
        column = (int)(u - whole - t * parts) * width;
        return whole + t;
    }
};

__host__ __device__ __forceinline__ ProductSplit product_split(uint32_t tiles) {
    const uint32_t rest = tiles % kProductPairs;
    ProductSplit s = {tiles - rest, 1};
    if (rest == 0) return s;
    if (rest * 4 <= kProductPairs) s.parts = 4;
    else if (rest * 2 <= kProductPairs) s.parts = 2;
    return s;
}

struct ProductSide {
    bool lines;                          // k runs over the lines of memory
    bool symmetric;                      // the blocks of 256 on and above the diagonal are there
    __device__ __forceinline__ bool by_lines(int row, int k) const {
        return symmetric ? (row & ~(kProductTile - 1)) > (k & ~(kProductTile - 1)) : lines;
    }
};

// the next chain of a unit, or the first of the pair's next unit
template <typename Job>
__device__ __forceinline__ void product_next(const Job& job, uint32_t& u, uint32_t& chain,
                                             uint32_t pairs) {
    if (++chain >= job.chains()) {
        chain = 0;
        u += pairs;
    }
}

struct ProductNothing {};

// a job of one phase
struct ProductOnce {
    static constexpr bool kPhased = false;
    CUtensorMap left, right;
    ProductSide left_side, right_side;
    bool bf16;
    uint32_t phases;
    uint32_t* arrived;
    const CUtensorMap *left_given, *right_given;
    template <typename Job> __device__ __forceinline__ void given_as(const Job* job) {
        left_given = &job->left;
        right_given = &job->right;
    }
    __device__ __forceinline__ void prefetch() const {
        prefetch_map(&left);
        prefetch_map(&right);
    }
    __device__ __forceinline__ const CUtensorMap* left_map() const { return left_given; }
    __device__ __forceinline__ const CUtensorMap* right_map() const { return right_given; }
};

// what a thread that reads a tile out has: one row, half of the columns
struct ProductRead {
    uint32_t tmem;                       // of the warp's lanes and of its first column
    int row, column, columns;            // in the unit: of the thread, of its first value; their number
    int lane, quarter, half;             // quarter: of the block's rows, half: of the columns
    bool ok, nothing;                    // !ok: a wait ran out, no result;  nothing: no steps
    float* rows;                         // the warp's own 32 x 33 words of shared memory
    float* exchange;                     // 32 x 33 words that the two warps of a quarter share
    uint32_t* word;                      // one that all threads that read tiles out share
    template <int N> __device__ __forceinline__ void load(int c, uint32_t (&r)[N]) const {
        if (nothing) {
#pragma unroll
            for (int i = 0; i < N; ++i) r[i] = 0u;
        } else {
            __syncwarp();
            if constexpr (N == 32) {
                tmem_load32(tmem + c, r);
                tmem_wait32(r);
            } else {
                static_assert(N == 16, "");
                uint32_t a[2][8];
                tmem_load8(tmem + c, a[0]);
                tmem_load8(tmem + c + 8, a[1]);
                tmem_wait8(a[0]);
                tmem_wait8(a[1]);
#pragma unroll
                for (int i = 0; i < 16; ++i) r[i] = a[i >> 3][i & 7];
            }
        }
        if (!ok) {
#pragma unroll
            for (int i = 0; i < N; ++i) r[i] = 0x7FC00000u;
        }
    }
};

// the two warps that read the same rows out
__device__ __forceinline__ void product_pair_barrier(const ProductRead& r) {
    asm volatile("bar.sync %0, %1;" ::"r"(1 + r.quarter), "r"(64) : "memory");
}

__device__ __forceinline__ void product_writers_barrier() {
    asm volatile("bar.sync %0, %1;" ::"r"(5), "r"(32 * kProductWriters) : "memory");
}

// tile number u of tiles_m x tiles_n, so that tiles computed at the same time share operands
__device__ __forceinline__ void product_tile(uint32_t u, uint32_t tiles_m, uint32_t tiles_n, int& m,
                                             int& n) {
    const uint32_t g = u / (8 * tiles_n), first = 8 * g, high = min(8u, tiles_m - first);
    const uint32_t r = u - 8 * tiles_n * g;
    m = (int)((first + r % high) * kProductTile);
    n = (int)(r / high * kProductTile);
}

// ---- results in memory -----------------------------------------------------------------------

// where a job's values go: rows of one of the three types, added to what is there or not
struct ProductTarget {
    int dtype;
    bool add;
    RowAccess access;
};

// The rows of a warp: where its lane's own one goes, nullptr: nowhere; and, unless they lie anywhere, where
// the first one goes, how far apart they are in elements, and how many there are.
struct ProductRows {
    void *own, *first;
    uint64_t step;
    int count;
    bool anywhere;
};

// Rows of a matrix at p, of which `rows` are there: those of the thread's warp, whose first is `row0`.
__device__ __forceinline__ ProductRows product_rows(void* p, int dtype, uint64_t ld, uint32_t row0,
                                                    uint32_t rows, uint64_t col, int lane) {
    const int bytes = dtype == NC_DTYPE_F32 ? 4 : 2;
    ProductRows r;
    r.count = row0 < rows ? (int)min(rows - row0, 32u) : 0;
    r.first = static_cast<char*>(p) + bytes * (row0 * ld + col);
    r.own = lane < r.count ? static_cast<char*>(r.first) + bytes * (lane * ld) : nullptr;
    r.step = ld;
    r.anywhere = false;
    return r;
}

template <typename T>
__device__ __forceinline__ void product_store_typed(const ProductTarget& t, const ProductRows& to, int c,
                                                    int cols, float (&v)[32], const ProductRead& r) {
    // a row whose 32 values are there and on 16-byte boundaries is written by its thread
    if (t.access != kRowElement && cols >= 32) {
        if (!to.own) return;
        T* row = static_cast<T*>(to.own) + c;
        const bool wide = t.access == kRowWide;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float o[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = v[16 * h + i];
            if (t.add) {
                float old[16];
                Raw16<T> raw;
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
                    const uint4* p = reinterpret_cast<const uint4*>(row + 16 * h) + 2 * i;
                    const uint4 a = p[0], b = p[1];
                    raw.b[i].v[0] = a.x; raw.b[i].v[1] = a.y; raw.b[i].v[2] = a.z; raw.b[i].v[3] = a.w;
                    raw.b[i].v[4] = b.x; raw.b[i].v[5] = b.y; raw.b[i].v[6] = b.z; raw.b[i].v[7] = b.w;
                }
                unpack16<T>(raw, old);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] += old[i];
            }
            st_raw16<T>(row + 16 * h, pack16<T>(o), wide);
        }
        return;
    }
    // else values change places, so that the lanes write neighbours of one row
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 32; ++i) r.rows[33 * r.lane + i] = v[i];
    __syncwarp();
    const bool in = r.lane < cols;
    if (!to.anywhere) {
        T* p = static_cast<T*>(to.first) + c + r.lane;
#pragma unroll 1
        for (int at = 0; at < to.count; at += 8, p += 8 * to.step) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = r.rows[33 * (at + i) + r.lane];
            if (t.add) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (in && at + i < to.count) x[i] += to_f32<T>(p[i * to.step]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (in && at + i < to.count) p[i * to.step] = from_f32<T>(x[i]);
        }
        return;
    }
#pragma unroll 1
    for (int at = 0; at < 32; at += 8) {
        T* p[8];
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = reinterpret_cast<T*>(
                __shfl_sync(0xFFFFFFFFu, (unsigned long long)(uintptr_t)to.own, at + i));
            x[i] = r.rows[33 * (at + i) + r.lane];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!p[i] || !in) continue;
            p[i] += c + r.lane;
            *p[i] = from_f32<T>(t.add ? to_f32<T>(*p[i]) + x[i] : x[i]);
        }
    }
}

// 32 values of the thread's row, from column c of its part on, of which the first `cols` are there.  All
// lanes of a warp come here with the same c and cols.
__device__ __forceinline__ void product_store(const ProductTarget& t, const ProductRows& to, int c,
                                              int cols, float (&v)[32], const ProductRead& r) {
    if (cols <= 0) return;
    if (t.dtype == NC_DTYPE_F32)
        product_store_typed<float>(t, to, c, cols, v, r);
    else if (t.dtype == NC_DTYPE_BF16)
        product_store_typed<__nv_bfloat16>(t, to, c, cols, v, r);
    else
        product_store_typed<__half>(t, to, c, cols, v, r);
}

// ---- chains ------------------------------------------------------------------------------------

// The `chain`-th of `chains` about equal parts of a unit's steps.  (Divisions in 64 bits only where 32 do not
// hold the product: the thread that issues the matrix instructions makes them between two chains.  6144 x 2048
// x 65536 logits with them always: 1430 us instead of 1340.)
__device__ __forceinline__ void product_chain(ProductUnit& w, uint32_t chain, uint32_t chains) {
    const uint32_t steps = (uint32_t)w.steps;
    uint32_t first, end;
    if ((uint64_t)steps * chains >> 32) {
        first = (uint32_t)((uint64_t)steps * chain / chains);
        end = (uint32_t)((uint64_t)steps * (chain + 1) / chains);
    } else {
        first = steps * chain / chains;
        end = steps * (chain + 1) / chains;
    }
    w.k += (int)first * kProductStep;
    w.steps = (int)(end - first);
}

// The accumulators of a chain added to those of the chains before (first: there are none).
__device__ __forceinline__ void product_keep(const ProductRead& r, bool first, float (&sums)[kProductHalf]) {
#pragma unroll
    for (int c = 0; c < kProductHalf; c += 16) {
        if (c >= r.columns) break;
        uint32_t v[16];
        r.load(c, v);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            sums[c + i] = first ? __uint_as_float(v[i]) : sums[c + i] + __uint_as_float(v[i]);
    }
}

// 32 of the sums of the chains before, those of the thread's columns from c on (0, 32, 64 or 96), added to v.
__device__ __forceinline__ void product_join(const float (&sums)[kProductHalf], int c, uint32_t (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) {       // (selects: an index would put the sums into memory)
        const float low = c & 32 ? sums[32 + i] : sums[i], high = c & 32 ? sums[96 + i] : sums[64 + i];
        v[i] = __float_as_uint((c & 64 ? high : low) + __uint_as_float(v[i]));
    }
}

// ---- sums in parts ---------------------------------------------------------------------------
// A part of a unit's sums lies in memory as [column / 4][256 rows] groups of four columns.

// The part of all threads that read the unit out, to memory (`to`: where the thread's first four columns
// go).  Whether all `splits` parts of the block's rows are there now: the block that brings the last one
// adds them up, in their order.  ticket: of the unit and of the block's half of the rows, 0 at first.
__device__ __forceinline__ bool product_part(const ProductRead& r, float4* to, uint32_t* ticket,
                                             uint32_t splits) {
#pragma unroll 1
    for (int c = 0; c < r.columns; c += 32) {
        uint32_t v[32];
        r.load(c, v);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            to[(c / 4 + i) * kProductTile] =
                make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]),
                            __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
    }
    product_writers_barrier();
    if (threadIdx.x == 0) {
        __threadfence();                 // (covers what all of the block's threads wrote before)
        const uint32_t before = atomicAdd(ticket, 1u);
        *r.word = (before + 1) % splits == 0;            // (the same ticket may serve several times)
        __threadfence();
    }
    product_writers_barrier();
    return *reinterpret_cast<volatile uint32_t*>(r.word) != 0;
}

// 32 columns of the parts' sum; `distance`: from one part to the next, in groups
__device__ __forceinline__ void product_sum(const float4* p, uint64_t distance, uint32_t splits,
                                            uint32_t (&v)[32]) {
    float4 all[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) all[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 2
    for (uint32_t j = 0; j < splits; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 x = __ldcg(p + j * distance + i * kProductTile);
            all[i].x += x.x; all[i].y += x.y; all[i].z += x.z; all[i].w += x.w;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[4 * i] = __float_as_uint(all[i].x);
        v[4 * i + 1] = __float_as_uint(all[i].y);
        v[4 * i + 2] = __float_as_uint(all[i].z);
        v[4 * i + 3] = __float_as_uint(all[i].w);
    }
}

// ---- the kernel ------------------------------------------------------------------------------
//
// Job:
//   ProductSide left_side, right_side;  bool bf16;
//   static bool kPhased;  uint32_t phases;  uint32_t* arrived       phased: their number, and a word that
//                                     is 0 at the beginning
//   void prefetch() const             of its maps
//   void given_as(const Job*)         the job as the kernel was given it (maps must be used where they are)
//   const CUtensorMap* left_map(), right_map()
//   uint32_t begin(uint32_t phase, bool reads_out)   the number of units, for every thread at the beginning
//                                     of each phase (may read what earlier kernels wrote); reads_out: of
//                                     the warps that read tiles out
//   uint32_t chains() const           parts that the sum of a unit is read out in, one after the other
//   ProductUnit unit_of(uint32_t u, uint32_t chain) const
//   struct State                      what a thread keeps from one chain to the next
//   void ahead(const ProductUnit&, const ProductRead&, State&)      loads that store() needs, while the
//                                     product is computed
//   void store(const ProductUnit&, const ProductRead&, State&)      all 256 threads that read tiles out
//
// A wait that runs out leaves NaN: the first block's issuing thread tells both blocks before it lets
// the tile count as complete.
template <typename Job>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1)
product_kernel(const __grid_constant__ Job given) {
    extern __shared__ uint8_t raw[];
    uint8_t* base = reinterpret_cast<uint8_t*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const uint32_t stages = smem_u32(base);
    uint64_t* bars = reinterpret_cast<uint64_t*>(base + kProductBars);
    const uint32_t filled = smem_u32(bars);                  // first block's: both blocks' copies
    const uint32_t empty = filled + 8 * kProductStages;      // operands consumed
    const uint32_t full = empty + 8 * kProductStages;        // [2] a tile's product is complete
    const uint32_t drained = full + 16;                      // [2] first block's: TMEM read out
    uint32_t* words = reinterpret_cast<uint32_t*>(bars + 2 * kProductStages + 4);
    volatile uint32_t* gave_up = words + 1;

    // (the shuffle tells the compiler that a warp has one number)
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (warp == kProductMmaWarp) tmem_alloc_pair(smem_u32(words), 2 * kProductTile);
    if (threadIdx.x == 32 * kProductCopyWarp) given.prefetch();
    if (threadIdx.x == 0) {
        words[1] = 0;
        for (int s = 0; s < kProductStages; ++s) {
            mbar_init(filled + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(full + 8 * b, 1);
            mbar_init(drained + 8 * b, 2 * kProductWriters);
        }
        mbar_init_fence();
    }
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    after_previous();
    let_next_begin();
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, words[0], 0);
    Job job = given;
    job.given_as(&given);
    const uint32_t phases = Job::kPhased ? job.phases : 1;

    if (warp < kProductWriters) {
        ProductRead r;
        r.lane = lane;
        r.quarter = warp & 3;
        r.half = warp >> 2;
        r.row = (int)rank * kProductHalf + 32 * r.quarter + lane;
        r.rows = reinterpret_cast<float*>(base + kProductBars + 256) + warp * (kProductRows / 4);
        r.exchange =
            reinterpret_cast<float*>(base + kProductBars + 256) + r.quarter * (kProductRows / 4);
        r.word = words + 2;
        uint32_t turn = 0;
        typename Job::State state;
        for (uint32_t phase = 0; phase < phases; ++phase) {
            if (Job::kPhased && phase) {     // every block is done with the phase before
                if (threadIdx.x == 0) grid_wait(job.arrived, phase * gridDim.x, gave_up);
                product_writers_barrier();
            }
            const uint32_t units = job.begin(phase, true);
            for (uint32_t u = pair, chain = 0; u < units; product_next(job, u, chain, pairs), ++turn) {
                const ProductUnit w = job.unit_of(u, chain);
                const uint32_t b = turn & 1;
                r.columns = w.width / 2;
                r.column = r.columns * r.half;
                job.ahead(w, r, state);
                const bool ok = mbar_wait(full + 8 * b, (turn >> 1) & 1, gave_up);
                r.ok = __all_sync(0xFFFFFFFFu, ok && !*gave_up);
                r.nothing = w.steps == 0;
                tc_fence_after();
                r.tmem = tmem + b * kProductTile + r.column + ((uint32_t)(32 * r.quarter) << 16);
                job.store(w, r, state);
                tc_fence_before();
                __syncwarp();
                // (a tile that was not waited for was not read: the other block may still be reading it)
                if (lane == 0 && r.ok) mbar_arrive_at(drained + 8 * b, 0);
            }
            if (Job::kPhased && phase + 1 < phases) {
                fence_global_copies();
                product_writers_barrier();       // (one thread's release behind it covers what all wrote)
                // (given up: others must not take this block's phases for done, or those of a block that is
                // late for it; they give up too)
                if (threadIdx.x == 0 && !*gave_up) grid_arrive(job.arrived);
            }
        }
    } else if (warp == kProductCopyWarp) {
        if (lane == 0) {
            uint32_t step = 0, stage = 0, parity = 0;
            bool ok = true;
            for (uint32_t phase = 0; phase < phases && ok; ++phase) {
                if (Job::kPhased && phase) {
                    ok = grid_wait(job.arrived, phase * gridDim.x, gave_up);
                    fence_global_copies();
                }
                const uint32_t units = job.begin(phase, false);
                const CUtensorMap *left = job.left_map(), *right = job.right_map();
                for (uint32_t u = pair, chain = 0; u < units && ok; product_next(job, u, chain, pairs)) {
                    const ProductUnit w = job.unit_of(u, chain);
                    const int m = w.m + (int)rank * kProductHalf;
                    const int n = w.n + (int)rank * (w.width / 2);
                    const bool second = w.width == kProductTile;     // box of the right operand
                    for (int s = 0; s < w.steps; ++s, ++step) {
                        if (step >= kProductStages) ok = mbar_wait(empty + 8 * stage, parity ^ 1, gave_up);
                        if (!ok) break;
                        const int k = w.k + s * kProductStep;
                        const uint32_t bar = filled + 8 * stage, to = stages + stage * kProductStage;
                        if (rank == 0)
                            mbar_expect(bar, 2 * (kProductStage - (second ? 0 : kProductBox)));
                        const bool a = job.left_side.by_lines(m, k);
                        const bool b = job.right_side.by_lines(n, k);
                        for (int h = 0; h < 2; ++h) {
                            tma_load_pair(to + h * kProductBox, left, a ? m + 64 * h : k,
                                          a ? k : m + 64 * h, w.z, bar);
                            if (h == 0 || second)
                                tma_load_pair(to + kProductOperand + h * kProductBox, right,
                                              b ? n + 64 * h : k, b ? k : n + 64 * h, w.z, bar);
                        }
                        stage = stage + 1 == kProductStages ? 0 : stage + 1;
                        parity ^= stage == 0;
                    }
                }
            }
            // both blocks' copies in flight land before the pair ends
            if (rank == 0) {
                const long long begin = clock64();
                for (uint32_t i = step < kProductStages ? 0 : step - kProductStages; i < step; ++i)
                    while (!mbar_try(filled + 8 * (i % kProductStages), (i / kProductStages) & 1) &&
                           clock64() - begin < 4000000000ll) {}
            }
        }
    } else if (rank == 0) {
        // ---- matrix instructions: the whole warp, of which one thread issues
        const bool elected = elect_one();
        const uint64_t operand = mma_operand(stages, kProductBox);     // + bytes / 16: further on
        bool ok = true;
        uint32_t stage = 0, parity = 0, turn = 0;
        for (uint32_t phase = 0; phase < phases && ok; ++phase) {
            const uint32_t units = job.begin(phase, false);
            for (uint32_t u = pair, chain = 0; u < units && ok;
                 product_next(job, u, chain, pairs), ++turn) {
                const ProductUnit w = job.unit_of(u, chain);
                const uint32_t b = turn & 1, to = tmem + b * kProductTile;
                const uint32_t plain = mma_shape_of(kProductTile, w.width, job.bf16, false, false);
                ok = mbar_wait(drained + 8 * b, ((turn >> 1) & 1) ^ 1, gave_up);
                for (int s = 0; s < w.steps; ++s) {
                    if (ok) ok = mbar_wait(filled + 8 * stage, parity, gave_up);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    const int k = w.k + s * kProductStep;
                    const bool a = job.left_side.by_lines(w.m, k);
                    const bool c = job.right_side.by_lines(w.n, k);
                    const uint32_t shape = plain | (uint32_t)a << 15 | (uint32_t)c << 16;
                    // 16 k further on: 16 lines, or 32 bytes of each line
                    const uint32_t da = a ? 128 : 2, dc = c ? 128 : 2;
                    const uint64_t left = operand + stage * (kProductStage / 16);
                    const uint64_t right = left + kProductOperand / 16;
#pragma unroll
                    for (int i = 0; i < kProductStep / 16; ++i)
                        mma_pair(to, left + i * da, right + i * dc, shape, s > 0 || i > 0, elected);
                    mma_commit_pair(empty + 8 * stage, elected);
                    stage = stage + 1 == kProductStages ? 0 : stage + 1;
                    parity ^= stage == 0;
                }
                ok = __all_sync(0xFFFFFFFFu, ok);
                // given up: both blocks know before their writers hear that the tile is complete, for what
                // stands in TMEM is the sum of some of the steps
                if (!ok && elected) {
                    shared_store_at(smem_u32(words + 1), 0, 1);
                    shared_store_at(smem_u32(words + 1), 1, 1);
                    fence_cluster();
                }
                __syncwarp();
                mma_commit_pair(full + 8 * b, elected);
            }
        }
    }
    // the pair stays until both blocks are done with each other's barriers and with TMEM
    __syncwarp();
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    if (warp == kProductMmaWarp) tmem_free_pair(tmem, 2 * kProductTile);
}

// most: an upper bound of the units of a phase
template <typename Job>
inline nc_status product_launch(const Job& job, uint64_t most, cudaStream_t stream) {
    static bool allowed[64];
    if (!allow_dynamic_smem((const void*)product_kernel<Job>, kProductSmem, allowed))
        return NC_ERR_CUDA;
    const unsigned pairs = (unsigned)(most < kProductPairs ? (most ? most : 1) : kProductPairs);
    if (!Job::kPhased) {
        launch_overlapping(product_kernel<Job>, dim3(2 * pairs), dim3(kProductThreads), kProductSmem,
                           stream, job);
        return NC_OK;
    }
    return launch_together(product_kernel<Job>, dim3(2 * pairs), dim3(kProductThreads), kProductSmem,
                           stream, job) == cudaSuccess
               ? NC_OK
               : NC_ERR_CUDA;
}

}  // namespace natcomp
