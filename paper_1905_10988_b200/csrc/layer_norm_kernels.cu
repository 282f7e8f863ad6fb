// Layer norm, forward and backward, with an optional 8-bit checkpoint of the normalised rows
// (act8_common.cuh), for sm_100a.
//
//   xh = (x - mean) * rstd,  y = gamma * xh + beta
//   g = gamma * dy,  dx = rstd * (g - mean(g) - xh * mean(g * xh)) [+ dres]
//   dgamma = sum over rows of dy * xh,  dbeta = sum over rows of dy
//
// By its bytes bound by memory: every row is read once and stays in registers between its statistics
// and its outputs.  What is left above that is the latency of a row's two reductions with the 16 warps
// an SM that the registers allow (bfloat16 16384 x 4096: forward with checkpoint 62 us, 5.4 TB/s;
// backward from the checkpoint with a residual gradient 86 us, 5.5 TB/s; a copy reaches 6.55 TB/s).
// (8 warps an SM backward for binary32 rows of 2048 and 4096 columns from the saved input with a residual
// gradient, whose ring leaves room for one block: 16384 x 4096 242 us, 4.4 TB/s.)
// A warp (up to 512 columns) or more of a block own a row, 16 values a thread.  The backward kernel
// is persistent: a thread keeps the sums of its own columns over all its rows in registers and reads
// a row ahead, the blocks' sums go to the workspace once, and a second kernel adds them in a fixed
// order, so no atomics decide the order of any sum.
#include "act8_common.cuh"
#include "tensor_core.cuh"

namespace natcomp {

constexpr int kLnMaxCols = 32768;
constexpr int kLnThreads = 256;         // most threads of a row in one block; a cluster of 2, 4 or 8
                                        // blocks shares a row of more than 16 * 256 columns
constexpr int kLnMaxParts = 592;        // blocks that write partial parameter gradients

struct LnParams {
    const void *gamma, *beta;           // where absent, the address of some other input
    int dtype;
    bool has_gamma, has_beta;
};

__device__ __forceinline__ float ln_param(const void* p, int dtype, uint32_t col) {
    if (dtype == NC_DTYPE_F32) return __ldg(static_cast<const float*>(p) + col);
    if (dtype == NC_DTYPE_BF16)
        return __bfloat162float(__ldg(static_cast<const __nv_bfloat16*>(p) + col));
    return __half2float(__ldg(static_cast<const __half*>(p) + col));
}

// A vector of parameters as the threads of a group read it: columns 16 * tid + 4 * q .. + 3 at
// table[q * G + tid].  Absent ones are `none`.
__device__ __forceinline__ void ln_table(float4* table, const void* p, bool has, int dtype, int G,
                                         uint32_t origin, uint32_t cols, float none) {
    const bool vector = (reinterpret_cast<uintptr_t>(p) & 15) == 0;
#pragma unroll 4
    for (int i = threadIdx.x; i < 4 * G; i += blockDim.x) {      // i: four columns
        const uint32_t col = 4 * i;
        float f[4] = {none, none, none, none};
        if (has) {
            if (vector && col + 4 <= cols) {
                if (dtype == NC_DTYPE_F32) {
                    const float4 v = __ldg(reinterpret_cast<const float4*>(
                        static_cast<const float*>(p) + origin + col));
                    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
                } else {
                    const uint2 v = __ldg(reinterpret_cast<const uint2*>(
                        static_cast<const unsigned short*>(p) + origin + col));
                    if (dtype == NC_DTYPE_BF16) {
                        unpack2<__nv_bfloat16>(v.x, f[0], f[1]);
                        unpack2<__nv_bfloat16>(v.y, f[2], f[3]);
                    } else {
                        unpack2<__half>(v.x, f[0], f[1]);
                        unpack2<__half>(v.y, f[2], f[3]);
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (col + k < cols) f[k] = ln_param(p, dtype, origin + col + k);
            }
        }
        table[(i & 3) * G + (i >> 2)] = make_float4(f[0], f[1], f[2], f[3]);
    }
}

__device__ __forceinline__ void ln_params(const float4* table, int G, int tid, f32x2 (&v)[8]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float4 f = table[q * G + tid];
        v[2 * q] = pair_of(f.x, f.y);
        v[2 * q + 1] = pair_of(f.z, f.w);
    }
}

// (The empty statement keeps the caller's condition a branch: few threads need it.)
__device__ __forceinline__ void clear_beyond(float (&v)[16], int tid, uint32_t cols) {
    asm volatile("");
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (16u * tid + i >= cols) v[i] = 0.0f;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

__device__ __forceinline__ float sum_of(const f32x2 (&v)[8]) {
    const f32x2 s = add2(add2(add2(v[0], v[1]), add2(v[2], v[3])),
                         add2(add2(v[4], v[5]), add2(v[6], v[7])));
    float a, b;
    of_pair(s, a, b);
    return a + b;
}

// values of warp `w` of the row's block `rank`
__device__ __forceinline__ uint32_t ln_warp_values(int rank, int w, int G, uint32_t all_cols) {
    const uint32_t first = rank * 16 * G + 512u * w;
    return all_cols > first ? min(all_cols - first, 512u) : 0u;
}

// Where a thread stands: a block holds blockDim / G groups of G threads, and a group owns a row at
// a time.  CLUSTER > 1: one group a block, and the blocks of a cluster share a row, block r of it
// owning the columns from r * 16 * G on.
template <int CLUSTER>
struct LnPlace {
    int G, groups, group, tid, warps, warp, lane;
    uint32_t rank, origin, cols;         // the block's first column and how many there are from it
    uint64_t first, step;                // rows
    __device__ __forceinline__ LnPlace(int g, uint32_t all_cols) {
        G = g;
        groups = blockDim.x / G;
        group = threadIdx.x / G;
        tid = threadIdx.x - group * G;
        warps = G >> 5;
        warp = tid >> 5;
        lane = threadIdx.x & 31;
        rank = CLUSTER > 1 ? blockIdx.x % CLUSTER : 0;
        origin = rank * 16 * G;
        cols = all_cols > origin ? all_cols - origin : 0;
        step = (uint64_t)(gridDim.x / CLUSTER) * groups;
        first = (uint64_t)(blockIdx.x / CLUSTER) * groups + group;
    }
};

// whether a wait of the block has run out of time
__device__ __forceinline__ bool ln_gave_up(const uint32_t* word) {
    return *static_cast<const volatile uint32_t*>(word) != 0;
}

// Two numbers of every warp of a row for all of them.  A row has up to 8 warps, or up to 64 in a
// cluster; slots without a warp stay 0.  Two rows use two sets in turn, so that a slot is written
// again only after the readers of the row before have passed the row in between.
//
// One block: a barrier of the group's threads.  Cluster: asynchronous stores to all its blocks, of
// which every block's own barrier counts the bytes; a cluster-wide barrier would wait for the loads
// and stores of global memory in flight as well.
//
// A wait that runs out of time sets the block's word, which ends its other waits at once.  A later wait
// on the same barrier could not tell the phase that never came from its own, so after that nothing
// that the block takes from another passes for a result, and it sends nothing more: whoever does not
// wait for the others may not write to their slots.  Their waits run out in turn.
template <int CLUSTER>
struct LnExchange {
    static constexpr int kSlots = CLUSTER > 1 ? 8 * CLUSTER : 8;      // of a row
    float2* set;                         // of even rows; the other one lies `other` further on
    uint32_t other, bars, bytes;
    // `slots`: [2][kSlots * groups], `words`: two barriers, `word`: the block's;
    // all threads of the cluster call
    __device__ __forceinline__ void begin(float2* slots, uint64_t* words, uint32_t* word,
                                          const LnPlace<CLUSTER>& p) {
        if (threadIdx.x == 0) *word = 0;
        const int all = kSlots * p.groups;
        for (int i = threadIdx.x; i < 2 * all; i += blockDim.x) slots[i] = make_float2(0.0f, 0.0f);
        set = slots + kSlots * p.group;
        other = all;
        bars = smem_u32(words);
        bytes = 8 * CLUSTER * p.warps;
        if (CLUSTER > 1 && threadIdx.x == 0) {
            mbar_init(bars, 1);
            mbar_init(bars + 8, 1);
            mbar_expect(bars, bytes);
            mbar_expect(bars + 8, bytes);
            mbar_init_fence();
        }
        __syncthreads();
        if (CLUSTER > 1) cluster_sync();
    }
    // row number `turn` of the group (0, 1, 2, ...)
    // lost: whether a wait of the block has run out of time; then, what it returns is no result
    __device__ __forceinline__ const float2* send(float2 mine, uint32_t turn,
                                                  const LnPlace<CLUSTER>& p, uint32_t* word,
                                                  bool& lost) {
        float2* slots = set + (turn & 1 ? other : 0u);
        if constexpr (CLUSTER > 1) {
            const uint32_t bar = bars + 8 * (turn & 1);
            if (p.lane < CLUSTER && !lost)
                st_async_pair(smem_u32(&slots[p.rank * p.warps + p.warp]), bar, p.lane, mine);
            lost |= !mbar_wait(bar, (turn >> 1) & 1, word);
            // armed for the row after next: nothing of it arrives before this block has sent
            // its part of the next row
            if (threadIdx.x == 0 && !lost) mbar_expect(bar, bytes);
        } else {
            if (p.lane == 0) slots[p.warp] = mine;
            asm volatile("bar.sync %0, %1;" ::"r"(p.group + 1), "r"(p.G) : "memory");
        }
        return slots;
    }
    // f(slot) summed over the row's slots, the same in every lane
    template <typename F>
    __device__ __forceinline__ float sum(const float2* slots, int lane, bool lost, F f) const {
        constexpr int kLanes = kSlots < 32 ? kSlots : 32;
        float s = f(slots, lane & (kLanes - 1));
        if (kSlots > 32) s += f(slots, lane + 32);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        if (CLUSTER > 1 && lost) s = __uint_as_float(0x7FC00000u);
        return s;
    }
};

// ---- forward -------------------------------------------------------------------------------

enum LnKeep { kKeepNone = 0, kKeepNearest = 1, kKeepRandom = 2 };

struct LnForward {
    const void* x;
    uint64_t rows;
    uint32_t cols;
    uint64_t ldx;
    LnParams params;
    float eps;
    void* y;
    uint64_t ldy;
    int access;
    float *mean, *rstd;
    uint8_t *codes, *scales;
    int keep;
    uint64_t seed;
    uint32_t worker;
};

// Every warp sums up its own values and their squared distances from its own mean; one exchange
// later the row's mean and variance follow from these (the squared distances about the common
// mean are the warps' own plus n_w (mean_w - mean)^2).  A row is read ahead.
// Four-byte values that are not kRegular do not fit 64 registers a thread with a row ahead, so they
// get 80 and three blocks an SM (binary32 with checkpoint, 4097 x 4099: 78 -> 47 us, 40000 x 1001:
// 80 -> 74); two-byte values fit (bfloat16 30000 x 1001: 52 us with four blocks, 58 with three).
template <typename T, int MODE>
constexpr int kLnForwardBlocks = sizeof(T) == 4 && MODE != kRegular ? 3 : 4;

template <typename T, int MODE, int KEEP, int CLUSTER>
__global__ void __launch_bounds__(kLnThreads, kLnForwardBlocks<T, MODE>)
ln_forward_kernel(const __grid_constant__ LnForward a, const int threads,
                  const __grid_constant__ PhiloxKeys keys) {
    __shared__ float2 slots[2 * LnExchange<CLUSTER>::kSlots * (CLUSTER > 1 ? 1 : 8)];
    __shared__ float2 counts[LnExchange<CLUSTER>::kSlots];
    __shared__ __align__(16) uint32_t
        scratches[MODE == kSpread ? kLnThreads / 32 : 1][MODE == kSpread ? kSpreadWords<T> : 4];
    uint32_t* scratch = scratches[MODE == kSpread ? threadIdx.x >> 5 : 0];
    __shared__ uint64_t bars[2];
    __shared__ uint32_t gave_up;
    extern __shared__ float4 tables[];   // gamma, beta
    const LnPlace<CLUSTER> p(threads, a.cols);
    const int row_warps = CLUSTER * p.warps;
    const float inverse_cols = 1.0f / (float)a.cols;
    const bool wide = a.access == kRowWide;
    const T* x = static_cast<const T*>(a.x) + p.origin;
    T* y = static_cast<T*>(a.y) + p.origin;
    const uint32_t pitch = (a.cols + 31) & ~31u;
    const uint32_t own = pitch > p.origin ? pitch - p.origin : 0;    // codes of a row from here on

    Raw16<T> next;
    if (p.first < a.rows) row_load<T, MODE>(x + p.first * a.ldx, p.tid, p.cols, wide, next);
    ln_table(tables, a.params.gamma, a.params.has_gamma, a.params.dtype, p.G, p.origin,
                        p.cols, 1.0f);
    ln_table(tables + 4 * p.G, a.params.beta, a.params.has_beta, a.params.dtype, p.G,
                        p.origin, p.cols, 0.0f);
    // values of each warp of the row and their reciprocal
    for (int w = threadIdx.x; w < LnExchange<CLUSTER>::kSlots; w += blockDim.x) {
        const float n = (float)ln_warp_values(w / p.warps, w % p.warps, p.G, a.cols);
        counts[w] = make_float2(n, n > 0.0f ? 1.0f / n : 0.0f);
    }
    LnExchange<CLUSTER> others;
    others.begin(slots, bars, &gave_up, p);
    const bool whole = MODE == kRegular || 16u * p.tid + 15 < p.cols;
    const float inverse_n = counts[p.rank * p.warps + p.warp].y;

    uint32_t turn = 0;
    for (uint64_t row = p.first; row < a.rows; row += p.step, ++turn) {
        f32x2 v[8];
        row_arrange<T, MODE>(next, scratch);
        unpack16<T>(next, v);
        if (row + p.step < a.rows)
            row_load<T, MODE>(x + (row + p.step) * a.ldx, p.tid, p.cols, wide, next);
        const float sum = warp_sum(sum_of(v));
        float mean = sum * inverse_n;
        float f[16];
        {
            const f32x2 m = pair_of(-mean, -mean);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f32x2 d = add2(v[i], m);
                of_pair(d, f[2 * i], f[2 * i + 1]);
            }
        }
        if (!whole) clear_beyond(f, p.tid, p.cols);
        f32x2 q = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f32x2 d = pair_of(f[2 * i], f[2 * i + 1]);
            q = fma2(d, d, q);
        }
        float square, odd;
        of_pair(q, square, odd);
        square = warp_sum(square + odd);
        if (row_warps > 1) {
            bool lost = CLUSTER > 1 && ln_gave_up(&gave_up);
            const float2* got = others.send(make_float2(sum, square), turn, p, &gave_up, lost);
            mean = others.sum(got, p.lane, lost, [](const float2* s, int w) { return s[w].x; }) *
                   inverse_cols;
            square = others.sum(got, p.lane, lost, [&](const float2* s, int w) {
                const float d = fmaf(s[w].x, counts[w].y, -mean);
                return fmaf(counts[w].x * d, d, s[w].y);
            });
        }
        const float rstd = rsqrtf(fmaf(square, inverse_cols, a.eps));
        if (p.tid == 0 && p.rank == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        {
            const f32x2 m = pair_of(-mean, -mean), s = pair_of(rstd, rstd);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = mul2(add2(v[i], m), s);
                of_pair(v[i], f[2 * i], f[2 * i + 1]);
            }
        }
        if constexpr (KEEP != kKeepNone) {
            float kept[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) kept[i] = f[i];
            if (!whole) clear_beyond(kept, p.tid, p.cols);
            const uint64_t plane = row * pitch + p.origin;
            uint32_t top = max_bits16(kept);
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            const uint32_t scale = act8_scale(top);
            if (16u * p.tid < own) {
                const uint64_t at = (plane >> 4) + p.tid;
                __stcs(reinterpret_cast<uint4*>(a.codes) + at,
                       act8_sixteen<KEEP == kKeepRandom>(
                           kept, scale,
                           act8_draws<KEEP == kKeepRandom>((uint32_t)at, a.worker, keys)));
                if (!(p.tid & 1)) a.scales[at >> 1] = (uint8_t)scale;
            }
        }
        f32x2 gamma[8], beta[8];
        ln_params(tables, p.G, p.tid, gamma);
        ln_params(tables + 4 * p.G, p.G, p.tid, beta);
#pragma unroll
        for (int i = 0; i < 8; ++i) of_pair(fma2(v[i], gamma[i], beta[i]), f[2 * i], f[2 * i + 1]);
        row_store<T, MODE>(y + row * a.ldy, p.tid, p.cols, wide, f, scratch);
    }
    // no block leaves while another may still write to its slots
    if (CLUSTER > 1) cluster_sync();
}

// how the rows are dealt out
struct LnDeal {
    int cluster, G, groups;              // blocks of a row, threads of a group, groups of a block
    uint64_t owners;                     // blocks (clusters) that have a row
};

static LnDeal ln_deal(uint64_t rows, uint64_t cols) {
    LnDeal d;
    d.cluster = 1;
    while (cols > 16u * kLnThreads * d.cluster) d.cluster *= 2;
    const uint64_t share = (cols + d.cluster - 1) / d.cluster;
    d.G = (int)((share + 511) / 512 * 32);
    d.groups = d.cluster == 1 ? kLnThreads / d.G : 1;
    d.owners = (rows + d.groups - 1) / d.groups;
    return d;
}

// launches `kernel` on as many blocks as have rows, at most `threads` threads for every SM
template <typename Kernel, typename... Args>
static nc_status ln_launch(Kernel kernel, const LnDeal& d, int threads, uint64_t most, size_t smem,
                           uint64_t* blocks, cudaStream_t stream, const Args&... args) {
    const int per_sm = threads / (d.G * d.groups);
    uint64_t n = (uint64_t)device_sm_count() * (per_sm < 1 ? 1 : per_sm) / d.cluster;
    if (n > most) n = most;
    if (n > d.owners) n = d.owners;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)n * d.cluster);
    cfg.blockDim = dim3(d.G * d.groups);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = d.cluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = d.cluster > 1 ? 1 : 0;
    if (blocks) *blocks = n;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? NC_OK : NC_ERR_CUDA;
}

// Rows of a multiple of 1024 columns up to 8192 on 32-byte boundaries: 32 values a thread, half
// the reductions a value, and no case to tell apart.
template <typename T, int KEEP>
__global__ void __launch_bounds__(kLnThreads, 2)
ln_forward_regular_kernel(const __grid_constant__ LnForward a, const int threads,
                          const __grid_constant__ PhiloxKeys keys) {
    __shared__ float2 slots[2 * 8 * 8];
    __shared__ uint64_t bars[2];
    __shared__ uint32_t gave_up;
    extern __shared__ float4 tables[];   // gamma, beta of the first and of the second half
    const LnPlace<1> p(threads, a.cols);
    const int G = p.G;
    const float inverse_cols = 1.0f / (float)a.cols;
    const T* x = static_cast<const T*>(a.x) + 16 * p.tid;
    T* y = static_cast<T*>(a.y) + 16 * p.tid;

    Raw16<T> next[2];
    if (p.first < a.rows) {
#pragma unroll
        for (int c = 0; c < 2; ++c) next[c] = ld_raw16<T>(x + p.first * a.ldx + c * 16 * G, true);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const uint32_t origin = c * 16 * G;
        ln_table(tables + 8 * G * c, a.params.gamma, a.params.has_gamma,
                              a.params.dtype, G, origin, a.cols - origin, 1.0f);
        ln_table(tables + 8 * G * c + 4 * G, a.params.beta, a.params.has_beta,
                              a.params.dtype, G, origin, a.cols - origin, 0.0f);
    }
    LnExchange<1> others;
    others.begin(slots, bars, &gave_up, p);

    uint32_t turn = 0;
    for (uint64_t row = p.first; row < a.rows; row += p.step, ++turn) {
        f32x2 v[2][8];
#pragma unroll
        for (int c = 0; c < 2; ++c) unpack16<T>(next[c], v[c]);
        if (row + p.step < a.rows) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
                next[c] = ld_raw16<T>(x + (row + p.step) * a.ldx + c * 16 * G, true);
        }
        const float sum = warp_sum(sum_of(v[0]) + sum_of(v[1]));
        float mean = sum * (1.0f / 1024.0f);
        f32x2 q = 0;
        f32x2 m = pair_of(-mean, -mean);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f32x2 d = add2(v[c][i], m);
                q = fma2(d, d, q);
            }
        float square, odd;
        of_pair(q, square, odd);
        square = warp_sum(square + odd);
        if (p.warps > 1) {
            bool lost = false;
            const float2* got = others.send(make_float2(sum, square), turn, p, &gave_up, lost);
            mean = others.sum(got, p.lane, lost, [](const float2* s, int w) { return s[w].x; }) *
                   inverse_cols;
            square = others.sum(got, p.lane, lost, [&](const float2* s, int w) {
                const float d = fmaf(s[w].x, 1.0f / 1024.0f, -mean);
                return w < p.warps ? fmaf(1024.0f * d, d, s[w].y) : 0.0f;
            });
        }
        const float rstd = rsqrtf(fmaf(square, inverse_cols, a.eps));
        if (p.tid == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        m = pair_of(-mean, -mean);
        const f32x2 s = pair_of(rstd, rstd);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float f[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[c][i] = mul2(add2(v[c][i], m), s);
                of_pair(v[c][i], f[2 * i], f[2 * i + 1]);
            }
            if constexpr (KEEP != kKeepNone) {
                uint32_t top = max_bits16(f);
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                const uint32_t scale = act8_scale(top);
                const uint64_t at = ((row * a.cols) >> 4) + c * G + p.tid;
                __stcs(reinterpret_cast<uint4*>(a.codes) + at,
                       act8_sixteen<KEEP == kKeepRandom>(
                           f, scale,
                           act8_draws<KEEP == kKeepRandom>((uint32_t)at, a.worker, keys)));
                if (!(p.tid & 1)) a.scales[at >> 1] = (uint8_t)scale;
            }
            f32x2 gamma[8], beta[8];
            ln_params(tables + 8 * G * c, G, p.tid, gamma);
            ln_params(tables + 8 * G * c + 4 * G, G, p.tid, beta);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                of_pair(fma2(v[c][i], gamma[i], beta[i]), f[2 * i], f[2 * i + 1]);
            st_raw16<T>(y + row * a.ldy + c * 16 * G, pack16<T>(f), true);
        }
    }
}

// rows on 32-byte boundaries whose values fill every thread of every block
static bool ln_regular(const LnDeal& d, uint64_t cols, int access) {
    return access == kRowWide && d.cluster <= 2 && cols == 16ull * d.G * d.cluster;
}

template <typename T, int KEEP>
static nc_status ln_forward_go(const LnForward& a, cudaStream_t stream) {
    // (few rows: with half the threads a row, one row of 4096 took 8.2 us instead of 6.5)
    if (a.access == kRowWide && a.cols % 1024 == 0 && a.cols <= 8192 && a.rows >= 512) {
        LnDeal d;
        d.cluster = 1;
        d.G = (int)(a.cols / 32);
        // blocks of 128 threads where rows allow it: four of them leave the registers that a thread
        // needs (three blocks of 256 with 80 registers: 70 instead of 63 us for 16384 x 4096; four-byte
        // values, twice the registers ahead: 55 with blocks of 256, 59 with blocks of 128)
        const int block = sizeof(T) == 4 ? kLnThreads : 128;
        d.groups = d.G < block ? block / d.G : 1;
        d.owners = (a.rows + d.groups - 1) / d.groups;
        const size_t smem = 4 * 16 * d.G * sizeof(float);
        static bool allowed[64];
        if (!allow_dynamic_smem((const void*)ln_forward_regular_kernel<T, KEEP>,
                                4 * 16 * kLnThreads * sizeof(float), allowed))
            return NC_ERR_CUDA;
        return ln_launch(ln_forward_regular_kernel<T, KEEP>, d, 512,
                         (uint64_t)1 << 30, smem, nullptr, stream, a, d.G,
                         make_philox_keys(a.seed));
    }
    const LnDeal d = ln_deal(a.rows, a.cols);
    auto pick = [&]() {
        if (ln_regular(d, a.cols, a.access))
            return d.cluster == 1 ? ln_forward_kernel<T, kRegular, KEEP, 1>
                                  : ln_forward_kernel<T, kRegular, KEEP, 2>;
        if (a.access != kRowElement)
            return d.cluster == 1   ? ln_forward_kernel<T, kVector, KEEP, 1>
                   : d.cluster == 2 ? ln_forward_kernel<T, kVector, KEEP, 2>
                   : d.cluster == 4 ? ln_forward_kernel<T, kVector, KEEP, 4>
                                    : ln_forward_kernel<T, kVector, KEEP, 8>;
        return d.cluster == 1   ? ln_forward_kernel<T, kSpread, KEEP, 1>
               : d.cluster == 2 ? ln_forward_kernel<T, kSpread, KEEP, 2>
               : d.cluster == 4 ? ln_forward_kernel<T, kSpread, KEEP, 4>
                                : ln_forward_kernel<T, kSpread, KEEP, 8>;
    };
    const auto kernel = pick();
    const size_t smem = 2 * 16 * d.G * sizeof(float);
    // spread rows of four-byte values need more than the 48 KB that come without asking
    static bool allowed[4][64];
    if (a.access == kRowElement && sizeof(T) == 4 &&
        !allow_dynamic_smem((const void*)kernel, 2 * 16 * kLnThreads * sizeof(float),
                            allowed[31 - __builtin_clz((unsigned)d.cluster)]))
        return NC_ERR_CUDA;
    const int most = ln_regular(d, a.cols, a.access) ? kLnForwardBlocks<T, kRegular>
                                                     : kLnForwardBlocks<T, kVector>;
    return ln_launch(kernel, d, kLnThreads * most, (uint64_t)1 << 30, smem, nullptr, stream, a, d.G,
                     make_philox_keys(a.seed));
}

template <typename T>
static nc_status ln_forward_launch(const LnForward& a, cudaStream_t stream) {
    auto go = a.keep == kKeepNone      ? ln_forward_go<T, kKeepNone>
              : a.keep == kKeepNearest ? ln_forward_go<T, kKeepNearest>
                                       : ln_forward_go<T, kKeepRandom>;
    return go(a, stream);
}

// ---- backward ------------------------------------------------------------------------------

struct LnBackward {
    const void* dy;
    uint64_t rows;
    uint32_t cols;
    uint64_t lddy;
    const void* x;                       // saved input, or
    uint64_t ldx;
    const uint8_t *codes, *scales;       // the checkpoint of xh
    const float *mean, *rstd;
    LnParams params;
    const void* dres;
    uint64_t lddres;
    void* dx;
    uint64_t lddx;
    float* parts;                        // [blocks][2][pitch]
    uint32_t parts_pitch;
    bool wide;
};

// kRegular rows pass through a ring in shared memory, filled by bulk copies that one thread of a group
// issues two or three rows ahead (with the rows ahead held in registers instead, 2051 x 8192 took 31 us
// and 16384 x 4096 from the checkpoint 92).  Places of a row's pieces in a stage, for G threads:
template <typename T, bool SAVED8, bool RES>
struct LnStage {
    static constexpr int kStages = sizeof(T) == 4 ? 2 : 3;
    static constexpr uint32_t kValues = 16 * sizeof(T);              // bytes of a thread
    static constexpr uint32_t kSaved = SAVED8 ? 16 : kValues;
    __host__ __device__ static uint32_t saved(int G) { return kValues * G; }
    __host__ __device__ static uint32_t scales(int G) { return saved(G) + kSaved * G; }
    __host__ __device__ static uint32_t dres(int G) { return scales(G) + (SAVED8 ? G / 2 : 0); }
    __host__ __device__ static uint32_t bytes(int G) { return dres(G) + (RES ? kValues * G : 0); }
};

template <typename T>
__device__ __forceinline__ Raw16<T> ld_shared16(const uint8_t* p) {
    Raw16<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) {
        const uint4 q = reinterpret_cast<const uint4*>(p)[i];
        uint32_t* v = r.b[i >> 1].v + 4 * (i & 1);
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    }
    return r;
}

// what a thread holds of a row before it is unpacked; other rows: loaded one row ahead
template <typename T, bool SAVED8, bool RES>
struct LnRow {
    Raw16<T> dy;
    Raw16<T> x;                          // !SAVED8
    uint4 codes;                         // SAVED8
    uint32_t scale;
    float mean, rstd;
};

template <typename T, int MODE, bool SAVED8, bool RES, int CLUSTER>
__global__ void __launch_bounds__(kLnThreads, 2)
ln_backward_kernel(const __grid_constant__ LnBackward a, const int threads) {
    __shared__ float2 slots[2 * LnExchange<CLUSTER>::kSlots * (CLUSTER > 1 ? 1 : 8)];
    __shared__ __align__(16) uint32_t
        scratches[MODE == kSpread ? kLnThreads / 32 : 1][MODE == kSpread ? kSpreadWords<T> : 4];
    uint32_t* scratch = scratches[MODE == kSpread ? threadIdx.x >> 5 : 0];
    __shared__ uint64_t bars[2], ringbars[MODE == kRegular ? 8 : 1][3];
    __shared__ uint32_t gave_up, fetches[MODE == kRegular ? 8 : 1];
    extern __shared__ float4 table[];    // gamma; several groups: their sums; the ring
    const LnPlace<CLUSTER> p(threads, a.cols);
    float* columns = reinterpret_cast<float*>(table + 4 * p.G);
    const int row_warps = CLUSTER * p.warps;
    const float inverse_cols = 1.0f / (float)a.cols;

    const T* dy = static_cast<const T*>(a.dy) + p.origin;
    const T* x = static_cast<const T*>(a.x) + (SAVED8 ? 0 : p.origin);
    const T* dres = static_cast<const T*>(a.dres) + (RES ? p.origin : 0);
    T* dx = static_cast<T*>(a.dx) + p.origin;
    const uint32_t pitch = (a.cols + 31) & ~31u;
    const uint32_t own = pitch > p.origin ? pitch - p.origin : 0;    // codes of a row from here on

    using Stage = LnStage<T, SAVED8, RES>;
    constexpr bool kRing = MODE == kRegular;
    uint8_t* ring = reinterpret_cast<uint8_t*>(columns + (p.groups > 1 ? 2 * pitch : 0)) +
                    p.group * Stage::kStages * Stage::bytes(p.G);
    const uint32_t arrived = smem_u32(ringbars[p.group]);

    auto load = [&](uint64_t row, LnRow<T, SAVED8, RES>& r) {
        r.rstd = __ldg(a.rstd + row);
        if constexpr (!SAVED8) r.mean = __ldg(a.mean + row);
        if constexpr (!kRing) {
            row_load<T, MODE>(dy + row * a.lddy, p.tid, p.cols, a.wide, r.dy);
            if constexpr (SAVED8) {
                const uint64_t plane = row * pitch + p.origin;
                r.codes = make_uint4(0u, 0u, 0u, 0u);
                r.scale = kAct8MinScale;
                if (16u * p.tid < own) {
                    r.codes = ld_stream_u4(a.codes + plane + 16u * p.tid);
                    r.scale = __ldg(a.scales + ((plane + 16u * p.tid) >> 5));
                }
            } else {
                row_load<T, MODE>(x + row * a.ldx, p.tid, p.cols, a.wide, r.x);
            }
        }
    };
    // one thread: the group's part of a row into stage `s`
    auto fetch = [&](uint64_t row, uint32_t s) {
        const uint32_t bar = arrived + 8 * s, at = smem_u32(ring + s * Stage::bytes(p.G));
        const uint32_t values = Stage::kValues * p.G;
        mbar_expect(bar, Stage::bytes(p.G));
        bulk_load(at, dy + row * a.lddy, values, bar);
        if constexpr (SAVED8) {
            const uint64_t plane = row * pitch + p.origin;
            bulk_load(at + Stage::saved(p.G), a.codes + plane, 16 * p.G, bar);
            bulk_load(at + Stage::scales(p.G), a.scales + (plane >> 5), p.G / 2, bar);
        } else {
            bulk_load(at + Stage::saved(p.G), x + row * a.ldx, values, bar);
        }
        if constexpr (RES) bulk_load(at + Stage::dres(p.G), dres + row * a.lddres, values, bar);
    };

    LnRow<T, SAVED8, RES> next;
    if (p.first < a.rows) load(p.first, next);
    if (kRing && p.tid == 0) {
        for (int s = 0; s < Stage::kStages; ++s) mbar_init(arrived + 8 * s, 1);
        mbar_init_fence();
        fetches[p.group] = 0;
        for (int s = 0; s < Stage::kStages; ++s)
            if (p.first + s * p.step < a.rows) fetch(p.first + s * p.step, s);
    }
    f32x2 dgamma[8], dbeta[8];
    ln_table(table, a.params.gamma, a.params.has_gamma, a.params.dtype, p.G, p.origin, p.cols, 1.0f);
    LnExchange<CLUSTER> others;
    others.begin(slots, bars, &gave_up, p);
    const bool whole = MODE == kRegular || 16u * p.tid + 15 < p.cols;
#pragma unroll
    for (int i = 0; i < 8; ++i) dgamma[i] = dbeta[i] = 0;

    uint32_t turn = 0, stage = 0, parity = 0;
    for (uint64_t row = p.first; row < a.rows; row += p.step, ++turn) {
        f32x2 g[8], xh[8];
        const float rstd = next.rstd;
        const float mean = SAVED8 ? 0.0f : next.mean;
        const uint8_t* here = ring + stage * Stage::bytes(p.G);
        if constexpr (kRing) {
            mbar_wait(arrived + 8 * stage, parity, &gave_up);        // what comes of it: `lost` below
            next.dy = ld_shared16<T>(here + Stage::kValues * p.tid);
            if constexpr (SAVED8) {
                next.codes =
                    *reinterpret_cast<const uint4*>(here + Stage::saved(p.G) + 16 * p.tid);
                next.scale = here[Stage::scales(p.G) + (p.tid >> 1)];
            } else {
                next.x = ld_shared16<T>(here + Stage::saved(p.G) + Stage::kValues * p.tid);
            }
        }
        row_arrange<T, MODE>(next.dy, scratch);
        unpack16<T>(next.dy, g);
        {
            float f[16];
            if constexpr (SAVED8) {
                act8_decode16(next.codes, next.scale, f);
            } else {
                row_arrange<T, MODE>(next.x, scratch);
                unpack16<T>(next.x, f);
#pragma unroll
                for (int i = 0; i < 16; ++i) f[i] = (f[i] - mean) * rstd;
            }
            if (!whole) clear_beyond(f, p.tid, p.cols);
#pragma unroll
            for (int i = 0; i < 8; ++i) xh[i] = pair_of(f[2 * i], f[2 * i + 1]);
        }
        Raw16<T> late;
        // issued here, not with the row ahead: the registers it would hold meanwhile cost more than its
        // latency (binary32 40000 x 1001: 207 -> 150 us, bfloat16 30000 x 1001: 119 -> 97)
        if constexpr (RES && !kRing)
            row_load<T, MODE>(dres + row * a.lddres, p.tid, p.cols, a.wide, late);
        if (row + p.step < a.rows) load(row + p.step, next);
        f32x2 s1 = 0, s2 = 0, gamma[8];
        ln_params(table, p.G, p.tid, gamma);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dbeta[i] = add2(dbeta[i], g[i]);
            dgamma[i] = fma2(g[i], xh[i], dgamma[i]);
            g[i] = mul2(g[i], gamma[i]);
            s1 = add2(s1, g[i]);
            s2 = fma2(g[i], xh[i], s2);
        }
        float m1, m2, odd;
        bool lost = kRing && ln_gave_up(&gave_up);
        of_pair(s1, m1, odd);
        if (kRing && lost) odd = __uint_as_float(0x7FC00000u);       // the row must not pass for a result
        m1 = warp_sum(m1 + odd);
        of_pair(s2, m2, odd);
        m2 = warp_sum(m2 + odd);
        if (row_warps > 1) {
            if (!kRing && CLUSTER > 1) lost = ln_gave_up(&gave_up);
            const float2* got = others.send(make_float2(m1, m2), turn, p, &gave_up, lost);
            m1 = others.sum(got, p.lane, lost, [](const float2* s, int w) { return s[w].x; });
            m2 = others.sum(got, p.lane, lost, [](const float2* s, int w) { return s[w].y; });
        } else if (kRing) {
            __syncwarp();
        }
        if constexpr (kRing) {
            // the whole group has come by, so it is done with the stage of the row before
            const uint32_t before = stage ? stage - 1 : Stage::kStages - 1;
            const uint64_t ahead = row + (Stage::kStages - 1) * p.step;
            if (p.tid == 0 && turn > 0 && ahead < a.rows) {
                if (!lost)
                    fetch(ahead, before);
                else if (!fetches[p.group])
                    fetches[p.group] = turn + Stage::kStages - 1;    // so many before
            }
            if constexpr (RES) late = ld_shared16<T>(here + Stage::dres(p.G) + Stage::kValues * p.tid);
            if (++stage == Stage::kStages) {
                stage = 0;
                parity ^= 1;
            }
        }
        m1 *= inverse_cols;
        m2 *= inverse_cols;
        // rstd * (g - m1 - xh * m2) + dres
        float out[16];
        const f32x2 n1 = pair_of(-m1, -m1), n2 = pair_of(-m2, -m2), s = pair_of(rstd, rstd);
        f32x2 d[8];
        if constexpr (RES) {
            row_arrange<T, MODE>(late, scratch);
            unpack16<T>(late, d);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f32x2 inner = fma2(xh[i], n2, add2(g[i], n1));
            of_pair(RES ? fma2(inner, s, d[i]) : mul2(inner, s), out[2 * i], out[2 * i + 1]);
        }
        row_store<T, MODE>(dx + row * a.lddx, p.tid, p.cols, a.wide, out, scratch);
    }

    let_next_begin();
    // the copies in flight land before the block may end
    if (kRing && p.tid == 0 && ln_gave_up(&gave_up)) {
        const long long begin = clock64();
        const uint32_t n = fetches[p.group] ? fetches[p.group] : turn;
        for (uint32_t i = n < Stage::kStages ? 0 : n - Stage::kStages; i < n; ++i)
            while (!mbar_try(arrived + 8 * (i % Stage::kStages), (i / Stage::kStages) & 1) &&
                   clock64() - begin < 4000000000ll) {}
    }
    float dg[16], db[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        of_pair(dgamma[i], dg[2 * i], dg[2 * i + 1]);
        of_pair(dbeta[i], db[2 * i], db[2 * i + 1]);
    }
    if (kRing && ln_gave_up(&gave_up)) {         // sums of values that may not have come
#pragma unroll
        for (int i = 0; i < 16; ++i) dg[i] = db[i] = __uint_as_float(0x7FC00000u);
    }
    float* out = a.parts + (uint64_t)(blockIdx.x / CLUSTER) * 2 * a.parts_pitch + p.origin;
    float* out2 = out + a.parts_pitch;
    if (p.groups > 1) {                  // the groups add up in order
        out = columns;
        out2 = columns + pitch;
        for (int k = 0; k < p.groups; ++k) {
            if (p.group == k && k > 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t col = 16u * p.tid + i;
                    if (col < p.cols) {
                        dg[i] += out[col];
                        db[i] += out2[col];
                    }
                }
            }
            if (p.group == k && k + 1 < p.groups) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t col = 16u * p.tid + i;
                    if (col < p.cols) {
                        out[col] = dg[i];
                        out2[col] = db[i];
                    }
                }
            }
            __syncthreads();
        }
        out = a.parts + (uint64_t)blockIdx.x * 2 * a.parts_pitch;
        out2 = out + a.parts_pitch;
    }
    if (p.group == p.groups - 1) {
        if (whole) {                     // the workspace's rows start on 16 bytes
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                *reinterpret_cast<float4*>(out + 16 * p.tid + i) =
                    make_float4(dg[i], dg[i + 1], dg[i + 2], dg[i + 3]);
                *reinterpret_cast<float4*>(out2 + 16 * p.tid + i) =
                    make_float4(db[i], db[i + 1], db[i + 2], db[i + 3]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t col = 16u * p.tid + i;
                if (col < p.cols) {
                    out[col] = dg[i];
                    out2[col] = db[i];
                }
            }
        }
    }
    // no block leaves while another may still write to its slots
    if (CLUSTER > 1) cluster_sync();
}

// dgamma, dbeta <- [their values +] the sum of the blocks' parts, in the order of the blocks
// within each of 8 interleaved groups, then of the groups
__global__ void __launch_bounds__(256)
ln_parts_kernel(const float* __restrict__ parts, const int blocks, const uint32_t pitch,
                const uint32_t cols, float* __restrict__ dgamma, float* __restrict__ dbeta,
                const bool accumulate) {
    __shared__ float sums[8][33];
    after_previous();
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const uint32_t col = blockIdx.x * 32 + lane;
    const float* p = parts + (blockIdx.y ? pitch : 0) + col;
    float s = 0.0f;
    if (col < cols) {
#pragma unroll 8
        for (int b = group; b < blocks; b += 8) s += __ldcg(p + (uint64_t)b * 2 * pitch);
    }
    sums[group][lane] = s;
    __syncthreads();
    if (group == 0 && col < cols) {
        s = sums[0][lane];
#pragma unroll
        for (int k = 1; k < 8; ++k) s += sums[k][lane];
        float* out = (blockIdx.y ? dbeta : dgamma) + col;
        *out = accumulate ? *out + s : s;
    }
}

template <typename T, bool SAVED8, bool RES>
static nc_status ln_backward_go(const LnBackward& a, int access, uint64_t* blocks,
                                cudaStream_t stream) {
    const LnDeal d = ln_deal(a.rows, a.cols);
    auto pick = [&]() {
        if (ln_regular(d, a.cols, access))
            return d.cluster == 1 ? ln_backward_kernel<T, kRegular, SAVED8, RES, 1>
                                  : ln_backward_kernel<T, kRegular, SAVED8, RES, 2>;
        if (access != kRowElement)
            return d.cluster == 1   ? ln_backward_kernel<T, kVector, SAVED8, RES, 1>
                   : d.cluster == 2 ? ln_backward_kernel<T, kVector, SAVED8, RES, 2>
                   : d.cluster == 4 ? ln_backward_kernel<T, kVector, SAVED8, RES, 4>
                                    : ln_backward_kernel<T, kVector, SAVED8, RES, 8>;
        return d.cluster == 1   ? ln_backward_kernel<T, kSpread, SAVED8, RES, 1>
               : d.cluster == 2 ? ln_backward_kernel<T, kSpread, SAVED8, RES, 2>
               : d.cluster == 4 ? ln_backward_kernel<T, kSpread, SAVED8, RES, 4>
                                : ln_backward_kernel<T, kSpread, SAVED8, RES, 8>;
    };
    size_t smem =
        16 * d.G * sizeof(float) + (d.groups > 1 ? 2 * act8_pitch(a.cols) * sizeof(float) : 0);
    const auto kernel = pick();
    if (ln_regular(d, a.cols, access)) {
        using Stage = LnStage<T, SAVED8, RES>;
        constexpr size_t kGroups = kLnThreads / 32;      // the most that any G takes
        static bool allowed[2][64];
        if (!allow_dynamic_smem((const void*)kernel,
                                16 * kLnThreads * sizeof(float) + 2 * 4096 * sizeof(float) +
                                    Stage::kStages * kGroups * Stage::bytes(32),
                                allowed[d.cluster - 1]))
            return NC_ERR_CUDA;
        smem += d.groups * Stage::kStages * Stage::bytes(d.G);
    }
    return ln_launch(kernel, d, 512, kLnMaxParts, smem, blocks, stream, a, d.G);
}

template <typename T>
static nc_status ln_backward_launch(const LnBackward& a, int access, float* dgamma, float* dbeta,
                                    bool accumulate, cudaStream_t stream) {
    uint64_t blocks = 0;
    if (a.rows) {
        auto go = a.codes ? (a.dres ? ln_backward_go<T, true, true> : ln_backward_go<T, true, false>)
                          : (a.dres ? ln_backward_go<T, false, true>
                                    : ln_backward_go<T, false, false>);
        const nc_status st = go(a, access, &blocks, stream);
        if (st != NC_OK) return st;
    }
    return launch_overlapping(ln_parts_kernel, dim3((a.cols + 31) / 32, 2), dim3(256), 0, stream,
                              (const float*)a.parts, (int)blocks, a.parts_pitch, a.cols, dgamma,
                              dbeta, accumulate) == cudaSuccess
               ? NC_OK
               : NC_ERR_CUDA;
}

static nc_status ln_backward_call(LnBackward a, int dtype, size_t cols, int param_dtype,
                                  float* dgamma, float* dbeta, int accumulate, void* workspace,
                                  size_t workspace_bytes, cudaStream_t stream) {
    const int bytes = act8_type_bytes(dtype), pbytes = act8_type_bytes(param_dtype);
    if (!bytes || !pbytes) return NC_ERR_UNSUPPORTED;
    if (cols == 0) return NC_OK;
    if (!dgamma || !dbeta) return NC_ERR_INVALID;
    if (a.rows) {
        if (!a.dy || !a.dx || !a.rstd || !workspace || a.lddy < cols || a.lddx < cols ||
            (a.dres && a.lddres < cols))
            return NC_ERR_INVALID;
        if (a.codes ? !a.scales : (!a.x || !a.mean || a.ldx < cols)) return NC_ERR_INVALID;
    }
    if (cols > kLnMaxCols || a.rows > 0x7FFFFFFFu || !act8_fits(a.rows, cols))
        return NC_ERR_TOO_LARGE;
    if (!aligned4(dgamma) || !aligned4(dbeta) || !aligned4(a.rstd) || !aligned4(a.mean) ||
        !element_aligned(a.dy, bytes) || !element_aligned(a.dx, bytes) ||
        !element_aligned(a.x, bytes) || !element_aligned(a.dres, bytes) ||
        !element_aligned(a.params.gamma, pbytes) || !aligned16(a.codes) || !aligned16(a.scales) ||
        !aligned16(workspace))
        return NC_ERR_ALIGN;
    a.cols = (uint32_t)cols;
    a.parts = static_cast<float*>(workspace);
    a.parts_pitch = (uint32_t)act8_pitch(cols);
    if (a.rows && workspace_bytes < nc_layer_norm_workspace_bytes(a.rows, cols))
        return NC_ERR_WORKSPACE;
    a.params.dtype = param_dtype;
    a.params.has_gamma = a.params.gamma != nullptr;
    if (!a.params.has_gamma) a.params.gamma = a.dy;
    int access = row_access(a.dy, a.lddy, bytes, a.rows);
    const int others[3] = {row_access(a.dx, a.lddx, bytes, a.rows),
                           a.dres ? row_access(a.dres, a.lddres, bytes, a.rows) : kRowWide,
                           a.codes ? kRowWide : row_access(a.x, a.ldx, bytes, a.rows)};
    for (int o : others) access = o > access ? o : access;
    a.wide = access == kRowWide;
    if (dtype == NC_DTYPE_F32)
        return ln_backward_launch<float>(a, access, dgamma, dbeta, accumulate != 0, stream);
    if (dtype == NC_DTYPE_BF16)
        return ln_backward_launch<__nv_bfloat16>(a, access, dgamma, dbeta, accumulate != 0,
                                                 stream);
    return ln_backward_launch<__half>(a, access, dgamma, dbeta, accumulate != 0, stream);
}

}  // namespace natcomp

using namespace natcomp;

extern "C" {

size_t nc_layer_norm_workspace_bytes(size_t rows, size_t cols) {
    if (cols == 0 || cols > kLnMaxCols) return 0;    // nothing to do; refused by the calls
    const uint64_t owners = ln_deal(rows, cols).owners;
    return (owners < (uint64_t)kLnMaxParts ? owners : (uint64_t)kLnMaxParts) * 2 *
           act8_pitch(cols) * sizeof(float);
}

nc_status nc_layer_norm_forward(const void* x, int dtype, size_t rows, size_t cols, size_t ldx,
                                const void* gamma, const void* beta, int param_dtype, float eps,
                                void* y, size_t ldy, float* mean, float* rstd, uint8_t* codes,
                                uint8_t* scales, int rounding, uint64_t seed, uint32_t worker,
                                cudaStream_t stream) {
    const int bytes = act8_type_bytes(dtype), pbytes = act8_type_bytes(param_dtype);
    if (!bytes || !pbytes) return NC_ERR_UNSUPPORTED;
    if (rounding != NC_ROUND_NEAREST && rounding != NC_ROUND_RANDOM) return NC_ERR_INVALID;
    if (rows == 0 || cols == 0) return NC_OK;
    if (!x || !y || ldx < cols || ldy < cols || (codes == nullptr) != (scales == nullptr))
        return NC_ERR_INVALID;
    if (cols > kLnMaxCols || rows > 0x7FFFFFFFu || !act8_fits(rows, cols)) return NC_ERR_TOO_LARGE;
    if (!element_aligned(x, bytes) || !element_aligned(y, bytes) ||
        !element_aligned(gamma, pbytes) || !element_aligned(beta, pbytes) || !aligned4(mean) ||
        !aligned4(rstd) || !aligned16(codes) || !aligned16(scales))
        return NC_ERR_ALIGN;
    const LnParams params = {gamma ? gamma : x, beta ? beta : x, param_dtype, gamma != nullptr,
                             beta != nullptr};
    LnForward a = {x, rows, (uint32_t)cols, ldx, params, eps, y, ldy, 0, mean, rstd, codes, scales,
                   kKeepNone, seed, worker};
    const int ax = row_access(x, ldx, bytes, rows), ay = row_access(y, ldy, bytes, rows);
    a.access = ax > ay ? ax : ay;
    if (codes) a.keep = rounding == NC_ROUND_RANDOM ? kKeepRandom : kKeepNearest;
    if (dtype == NC_DTYPE_F32)
        return ln_forward_launch<float>(a, stream);
    if (dtype == NC_DTYPE_BF16) return ln_forward_launch<__nv_bfloat16>(a, stream);
    return ln_forward_launch<__half>(a, stream);
}

nc_status nc_layer_norm_backward(const void* dy, int dtype, size_t rows, size_t cols, size_t lddy,
                                 const void* x, size_t ldx, const float* mean, const float* rstd,
                                 const void* gamma, int param_dtype, const void* dres,
                                 size_t lddres, void* dx, size_t lddx, float* dgamma, float* dbeta,
                                 int accumulate, void* workspace, size_t workspace_bytes,
                                 cudaStream_t stream) {
    LnBackward a = {};
    a.dy = dy; a.rows = rows; a.lddy = lddy; a.x = x; a.ldx = ldx; a.mean = mean; a.rstd = rstd;
    a.params.gamma = gamma; a.dres = dres; a.lddres = lddres; a.dx = dx; a.lddx = lddx;
    return ln_backward_call(a, dtype, cols, param_dtype, dgamma, dbeta, accumulate, workspace,
                            workspace_bytes, stream);
}

nc_status nc_act8_layer_norm_backward(const void* dy, int dtype, size_t rows, size_t cols,
                                      size_t lddy, const uint8_t* codes, const uint8_t* scales,
                                      const float* rstd, const void* gamma, int param_dtype,
                                      const void* dres, size_t lddres, void* dx, size_t lddx,
                                      float* dgamma, float* dbeta, int accumulate, void* workspace,
                                      size_t workspace_bytes, cudaStream_t stream) {
    if (rows && cols && !codes) return NC_ERR_INVALID;
    LnBackward a = {};
    a.dy = dy; a.rows = rows; a.lddy = lddy; a.codes = codes; a.scales = scales; a.rstd = rstd;
    a.params.gamma = gamma; a.dres = dres; a.lddres = lddres; a.dx = dx; a.lddx = lddx;
    return ln_backward_call(a, dtype, cols, param_dtype, dgamma, dbeta, accumulate, workspace,
                            workspace_bytes, stream);
}

}  // extern "C"
