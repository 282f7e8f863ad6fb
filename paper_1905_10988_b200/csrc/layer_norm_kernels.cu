// Layer norm, forward and backward, with an optional 8-bit checkpoint of the normalised rows
// (act8_common.cuh), for sm_100a.
//
//   xh = (x - mean) * rstd,  y = gamma * xh + beta
//   g = gamma * dy,  dx = rstd * (g - mean(g) - xh * mean(g * xh)) [+ dres]
//   dgamma = sum over rows of dy * xh,  dbeta = sum over rows of dy
//
// Bound by memory: every row is read once and stays in registers between its statistics and its
// outputs.  A warp (up to 512 columns) or more of a block own a row, 16 values a thread.  The
// backward kernel is persistent: a thread keeps the sums of its own columns over all its rows in
// registers and reads a row ahead, the blocks' sums go to the workspace once, and a second kernel
// adds them in a fixed order, so no atomics decide the order of any sum.
//
// Two assignments of a row's values to threads, one code: rows that start on multiples of 16
// bytes give a thread 16 neighbouring values at a time; other rows give neighbouring values to
// neighbouring lanes, one element per access.
#include <cooperative_groups.h>

#include "act8_common.cuh"

namespace natcomp {

constexpr int kLnMaxCols = 32768;
constexpr int kLnBackThreads = 512;     // most threads of a backward block; a cluster of 2 or 4
                                        // blocks shares a row of more than 16 * 512 columns
constexpr int kLnMaxParts = 592;        // blocks that write partial parameter gradients

struct LnParams {
    const void *gamma, *beta;           // where absent, the address of some other input
    int dtype;
    bool vector;                        // both may be read 16 bytes at a time
    bool has_gamma, has_beta;
};

// ---- a thread's values of a row ------------------------------------------------------------
// value (c, i) of thread `tid` of G: column 16 * (c * G + tid) + i, or, ELEMENT,
// (16 * c + i) * G + tid
template <bool ELEMENT>
__device__ __forceinline__ uint32_t ln_col(int c, int i, int G, int tid) {
    return ELEMENT ? (uint32_t)(16 * c + i) * G + tid : 16u * (c * G + tid) + i;
}

template <typename T, bool ELEMENT>
__device__ __forceinline__ void ln_load(const T* __restrict__ row, int c, int G, int tid,
                                        uint32_t cols, bool wide, Raw16<T>& r) {
    if (ELEMENT) {
#pragma unroll
        for (int b = 0; b < (int)sizeof(T) / 2; ++b)
#pragma unroll
            for (int i = 0; i < 8; ++i) r.b[b].v[i] = 0u;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t col = ln_col<true>(c, i, G, tid);
            if (col < cols) {
                if constexpr (sizeof(T) == 4)
                    r.b[i >> 3].v[i & 7] = __ldg(reinterpret_cast<const uint32_t*>(row) + col);
                else
                    r.b[0].v[i >> 1] |=
                        (uint32_t)__ldg(reinterpret_cast<const unsigned short*>(row) + col)
                        << (16 * (i & 1));
            }
        }
        return;
    }
    const uint32_t col = ln_col<false>(c, 0, G, tid);
    if (col + 16 <= cols)
        r = ld_raw16<T>(row + col, wide);
    else
        r = ld_raw16_part<T>(row + col, col < cols ? (int)(cols - col) : 0);
}

template <typename T, bool ELEMENT>
__device__ __forceinline__ void ln_store(T* __restrict__ row, int c, int G, int tid, uint32_t cols,
                                         bool wide, const float (&v)[16]) {
    if (ELEMENT) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t col = ln_col<true>(c, i, G, tid);
            if (col < cols) row[col] = from_f32<T>(v[i]);
        }
        return;
    }
    const uint32_t col = ln_col<false>(c, 0, G, tid);
    if (col + 16 <= cols)
        st_raw16<T>(row + col, pack16<T>(v), wide);
    else if (col < cols)
        st_part16<T>(row + col, v, (int)(cols - col));
}

__device__ __forceinline__ float ln_param(const void* p, int dtype, uint32_t col) {
    if (dtype == NC_DTYPE_F32) return __ldg(static_cast<const float*>(p) + col);
    if (dtype == NC_DTYPE_BF16)
        return __bfloat162float(__ldg(static_cast<const __nv_bfloat16*>(p) + col));
    return __half2float(__ldg(static_cast<const __half*>(p) + col));
}

// sixteen parameters in float; absent ones are `none`
template <bool ELEMENT>
__device__ __forceinline__ void ln_params(const void* p, bool has, int dtype, bool vector, int c,
                                          int G, int tid, uint32_t cols, float none,
                                          float (&v)[16]) {
    if (!has) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = none;
        return;
    }
    const uint32_t col = ln_col<false>(c, 0, G, tid);
    if (!ELEMENT && vector && col + 16 <= cols) {
        if (dtype == NC_DTYPE_F32)
            unpack16<float>(ld_raw16<float>(static_cast<const float*>(p) + col, false), v);
        else if (dtype == NC_DTYPE_BF16)
            unpack16<__nv_bfloat16>(
                ld_raw16<__nv_bfloat16>(static_cast<const __nv_bfloat16*>(p) + col, false), v);
        else
            unpack16<__half>(ld_raw16<__half>(static_cast<const __half*>(p) + col, false), v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t at = ln_col<ELEMENT>(c, i, G, tid);
        v[i] = at < cols ? ln_param(p, dtype, at) : 0.0f;
    }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// the threads of group `group` of a block, G of them
__device__ __forceinline__ void group_sync(int group, int G) {
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(G) : "memory");
}

// ---- forward -------------------------------------------------------------------------------

enum LnKeep { kKeepNone = 0, kKeepNearest = 1, kKeepRandom = 2 };

// A block holds blockDim / G groups of G threads; a group takes a row at a time and reads a row
// ahead.  Every warp sums up its own values and their squared distances from its own mean; one
// barrier later the group's mean and variance follow from these (the squared distances about the
// common mean are the warps' own plus n_w (mean_w - mean)^2).
template <typename T, int C, int THREADS, bool ELEMENT, int KEEP>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS)
ln_forward_kernel(const T* __restrict__ x, const uint64_t rows, const uint32_t cols,
                  const uint64_t ldx, const LnParams params, const float eps, T* __restrict__ y,
                  const uint64_t ldy, const bool wide, float* __restrict__ mean_out,
                  float* __restrict__ rstd_out, uint8_t* __restrict__ codes,
                  uint8_t* __restrict__ scales, const uint32_t worker, const int G,
                  const __grid_constant__ PhiloxKeys keys) {
    __shared__ float2 part[2][32];       // sum and squared distances of a warp, two rows in turn
    __shared__ float count[32];          // values of a warp
    const int groups = blockDim.x / G, group = threadIdx.x / G, tid = threadIdx.x - group * G;
    const int warps = G >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint64_t step = (uint64_t)gridDim.x * groups;
    const float inverse_cols = 1.0f / (float)cols;

    int mine = 0;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) mine += ln_col<ELEMENT>(c, i, G, tid) < cols;
    const bool whole = mine == 16 * C;
    const float n_warp = warp_sum((float)mine), inverse_n = n_warp > 0.0f ? 1.0f / n_warp : 0.0f;
    if (lane == 0) count[warp] = n_warp;
    __syncthreads();

    uint64_t row = (uint64_t)blockIdx.x * groups + group;
    Raw16<T> next[C];
    if (row < rows) {
#pragma unroll
        for (int c = 0; c < C; ++c) ln_load<T, ELEMENT>(x + row * ldx, c, G, tid, cols, wide, next[c]);
    }
    for (int turn = 0; row < rows; row += step, turn ^= 1) {
        float v[C][16];
#pragma unroll
        for (int c = 0; c < C; ++c) unpack16<T>(next[c], v[c]);
        if (row + step < rows) {
#pragma unroll
            for (int c = 0; c < C; ++c)
                ln_load<T, ELEMENT>(x + (row + step) * ldx, c, G, tid, cols, wide, next[c]);
        }
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += v[c][i];
        sum = warp_sum(sum);
        float mean = sum * inverse_n, square = 0.0f;
        if (whole) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float d = v[c][i] - mean;
                    square = fmaf(d, d, square);
                }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float d = v[c][i] - mean;
                    if (ln_col<ELEMENT>(c, i, G, tid) < cols) square = fmaf(d, d, square);
                }
        }
        square = warp_sum(square);
        if (warps > 1) {
            // a slot is written again only after the barrier of the row in between, which its
            // readers have passed
            if (lane == 0) part[turn][warp] = make_float2(sum, square);
            group_sync(group, G);
            const bool has = lane < warps;
            const float2 p = has ? part[turn][group * warps + lane] : make_float2(0.0f, 0.0f);
            const float n = has ? count[group * warps + lane] : 0.0f;
            mean = warp_sum(p.x) * inverse_cols;
            const float d = n > 0.0f ? p.x / n - mean : 0.0f;
            square = warp_sum(fmaf(n * d, d, p.y));
        }
        const float rstd = 1.0f / sqrtf(fmaf(square, inverse_cols, eps));
        if (tid == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }

        const uint32_t pitch = (cols + 31) & ~31u;
        const uint64_t plane = row * pitch;              // the row's first code
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[c][i] = (v[c][i] - mean) * rstd;
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (ln_col<ELEMENT>(c, i, G, tid) >= cols) v[c][i] = 0.0f;
            }
            if (KEEP != kKeepNone && !ELEMENT) {
                uint32_t top = max_bits16(v[c]);
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                const uint32_t scale = act8_scale(top);
                const uint32_t col = ln_col<false>(c, 0, G, tid);
                if (col < pitch) {
                    const uint64_t q = (plane + col) >> 4;
                    __stcs(reinterpret_cast<uint4*>(codes) + q,
                           act8_sixteen<KEEP == kKeepRandom>(v[c], scale, q, worker, keys));
                    if (!(tid & 1)) scales[q >> 1] = (uint8_t)scale;
                }
            }
            if (KEEP != kKeepNone && ELEMENT) {
                // step i of the warp is the block of 32 columns that starts at ln_col of lane 0
                uint32_t r[4] = {0u, 0u, 0u, 0u};
                if (KEEP == kKeepRandom) {
                    const uint32_t col =
                        ln_col<true>(c, lane >> 1, G, tid - lane) + 16 * (lane & 1);
                    stream_words4((plane + col) >> 4, worker, kDomainAct8, keys, r);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t first = ln_col<true>(c, i, G, tid - lane);
                    const uint32_t top =
                        __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v[c][i]) & 0x7FFFFFFFu);
                    const uint32_t scale = act8_scale(top);
                    uint32_t draw = 0;
                    if (KEEP == kKeepRandom) {
                        uint32_t word = 0;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t t =
                                __shfl_sync(0xFFFFFFFFu, r[k], 2 * i + (lane >> 4));
                            if (((lane >> 2) & 3) == k) word = t;
                        }
                        draw = (word >> (8 * (lane & 3))) & 0xFFu;
                    }
                    if (first < pitch) {
                        codes[plane + first + lane] = (uint8_t)(
                            scale == kAct8Nan
                                ? 0u
                                : act8_one(v[c][i], act8_inverse(scale, KEEP == kKeepRandom),
                                           KEEP == kKeepRandom, draw));
                        if (lane == 0) scales[(plane + first) >> 5] = (uint8_t)scale;
                    }
                }
            }
            float p[16];
            ln_params<ELEMENT>(params.gamma, params.has_gamma, params.dtype, params.vector, c, G,
                               tid, cols, 1.0f, p);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[c][i] *= p[i];
            ln_params<ELEMENT>(params.beta, params.has_beta, params.dtype, params.vector, c, G, tid,
                               cols, 0.0f, p);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[c][i] += p[i];
            ln_store<T, ELEMENT>(y + row * ldy, c, G, tid, cols, wide, v[c]);
        }
    }
}

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

template <typename T, int C, int THREADS, bool ELEMENT, int KEEP>
static void ln_forward_go(const LnForward& a, int G, cudaStream_t stream) {
    const int groups = G < THREADS ? THREADS / G : 1;
    const uint64_t want = (a.rows + groups - 1) / groups;
    const uint64_t fit = (uint64_t)device_sm_count() * (1024 / (G * groups));
    ln_forward_kernel<T, C, THREADS, ELEMENT, KEEP>
        <<<(unsigned)(want < fit ? want : fit), G * groups, 0, stream>>>(
            static_cast<const T*>(a.x), a.rows, a.cols, a.ldx, a.params, a.eps,
            static_cast<T*>(a.y), a.ldy, a.access == kRowWide, a.mean, a.rstd, a.codes, a.scales,
            a.worker, G, make_philox_keys(a.seed));
}

template <typename T, int C, int THREADS>
static void ln_forward_rows(const LnForward& a, int G, cudaStream_t stream) {
    const bool element = a.access == kRowElement;
    auto go = a.keep == kKeepNone
                  ? (element ? ln_forward_go<T, C, THREADS, true, kKeepNone>
                             : ln_forward_go<T, C, THREADS, false, kKeepNone>)
              : a.keep == kKeepNearest
                  ? (element ? ln_forward_go<T, C, THREADS, true, kKeepNearest>
                             : ln_forward_go<T, C, THREADS, false, kKeepNearest>)
                  : (element ? ln_forward_go<T, C, THREADS, true, kKeepRandom>
                             : ln_forward_go<T, C, THREADS, false, kKeepRandom>);
    go(a, G, stream);
}

template <typename T>
static void ln_forward_launch(const LnForward& a, cudaStream_t stream) {
    if (a.cols <= 4096)
        ln_forward_rows<T, 1, 256>(a, (int)((a.cols + 511) / 512 * 32), stream);
    else if (a.cols <= 16384)
        ln_forward_rows<T, 1, 1024>(a, (int)((a.cols + 511) / 512 * 32), stream);
    else
        ln_forward_rows<T, 2, 1024>(a, (int)((a.cols + 1023) / 1024 * 32), stream);
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

// what a thread holds of a row before it is unpacked: loaded one row ahead
template <typename T, bool SAVED8, bool RES>
struct LnRow {
    Raw16<T> dy;
    Raw16<T> x;                          // !SAVED8
    uint4 codes;                         // SAVED8
    uint32_t scale;
    Raw16<T> dres;                       // RES
    float mean, rstd;
};

// A block holds blockDim / G groups of G threads, a group owns a row at a time, 16 values a
// thread.  CLUSTER > 1: one group a block, and the blocks of a cluster share a row, block r of it
// owning the columns from r * 16 * G on.
template <typename T, bool ELEMENT, bool SAVED8, bool RES, int CLUSTER>
__global__ void __launch_bounds__(kLnBackThreads)
ln_backward_kernel(const __grid_constant__ LnBackward a, const int G) {
    __shared__ float2 part[2][CLUSTER * 16];
    extern __shared__ float columns[];   // several groups: their sums
    const int groups = blockDim.x / G, group = threadIdx.x / G, tid = threadIdx.x - group * G;
    const int warps = G >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CLUSTER > 1 ? blockIdx.x % CLUSTER : 0;
    const uint32_t origin = rank * 16 * G;                          // the block's first column
    const uint32_t cols = a.cols > origin ? a.cols - origin : 0;    // from there on
    const uint64_t step = (uint64_t)(gridDim.x / CLUSTER) * groups;
    const uint64_t begin = (uint64_t)(blockIdx.x / CLUSTER) * groups + group;

    const T* dy = static_cast<const T*>(a.dy) + origin;
    const T* x = static_cast<const T*>(a.x) + (SAVED8 ? 0 : origin);
    const T* dres = static_cast<const T*>(a.dres) + (RES ? origin : 0);
    T* dx = static_cast<T*>(a.dx) + origin;
    const uint32_t pitch = (a.cols + 31) & ~31u;
    const uint32_t own = pitch > origin ? pitch - origin : 0;       // codes from there on
    const uint32_t col0 = ln_col<false>(0, 0, G, tid);

    auto load = [&](uint64_t row, LnRow<T, SAVED8, RES>& r) {
        r.rstd = __ldg(a.rstd + row);
        ln_load<T, ELEMENT>(dy + row * a.lddy, 0, G, tid, cols, a.wide, r.dy);
        if constexpr (SAVED8) {
            const uint64_t plane = row * pitch + origin;
            r.codes = make_uint4(0u, 0u, 0u, 0u);
            r.scale = kAct8MinScale;
            if (!ELEMENT && col0 < own) {
                r.codes = ld_stream_u4(a.codes + plane + col0);
                r.scale = __ldg(a.scales + ((plane + col0) >> 5));
            }
        } else {
            r.mean = __ldg(a.mean + row);
            ln_load<T, ELEMENT>(x + row * a.ldx, 0, G, tid, cols, a.wide, r.x);
        }
        if constexpr (RES)
            ln_load<T, ELEMENT>(dres + row * a.lddres, 0, G, tid, cols, a.wide, r.dres);
    };

    float gamma[16], dgamma[16], dbeta[16];
    {
        const int bytes = a.params.dtype == NC_DTYPE_F32 ? 4 : 2;
        const char* p = static_cast<const char*>(a.params.gamma);
        ln_params<ELEMENT>(p + (size_t)origin * bytes, a.params.has_gamma, a.params.dtype,
                           a.params.vector, 0, G, tid, cols, 1.0f, gamma);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) dgamma[i] = dbeta[i] = 0.0f;

    // the other blocks' slots exist once all blocks of the cluster run
    if (CLUSTER > 1) cooperative_groups::this_cluster().sync();
    LnRow<T, SAVED8, RES> next;
    if (begin < a.rows) load(begin, next);
    int turn = 0;
    for (uint64_t row = begin; row < a.rows; row += step, turn ^= 1) {
        const LnRow<T, SAVED8, RES> r = next;
        if (row + step < a.rows) load(row + step, next);
        float g[16], xh[16];
        unpack16<T>(r.dy, g);
        if constexpr (SAVED8) {
            if (ELEMENT) {
                const uint64_t plane = row * pitch + origin;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t col = ln_col<true>(0, i, G, tid);
                    xh[i] = col < cols ? act8_value(__ldg(a.codes + plane + col),
                                                    __ldg(a.scales + ((plane + col) >> 5)))
                                       : 0.0f;
                }
            } else {
                act8_decode16(r.codes, r.scale, xh);
                if (col0 + 16 > cols) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (col0 + i >= cols) xh[i] = 0.0f;      // of a block that is not finite
                }
            }
        } else {
            unpack16<T>(r.x, xh);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                xh[i] = ln_col<ELEMENT>(0, i, G, tid) < cols ? (xh[i] - r.mean) * r.rstd : 0.0f;
        }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            dbeta[i] += g[i];
            dgamma[i] = fmaf(g[i], xh[i], dgamma[i]);
            g[i] *= gamma[i];
            s1 += g[i];
            s2 = fmaf(g[i], xh[i], s2);
        }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        if (CLUSTER > 1 || warps > 1) {
            // two sets of slots in turn: a slot is written again only after the barrier of the
            // row in between, which its readers have passed
            if constexpr (CLUSTER > 1) {
                cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
                if (lane < CLUSTER)
                    *cluster.map_shared_rank(&part[turn][rank * 16 + warp], lane) =
                        make_float2(s1, s2);
                cluster.sync();
            } else {
                if (lane == 0) part[turn][warp] = make_float2(s1, s2);
                group_sync(group, G);
            }
            s1 = s2 = 0.0f;
            for (int k = 0; k < CLUSTER; ++k)
                for (int w = 0; w < warps; ++w) {
                    const float2 p = part[turn][k * 16 + group * warps + w];
                    s1 += p.x;
                    s2 += p.y;
                }
        }
        const float m1 = s1 / (float)a.cols, m2 = s2 / (float)a.cols;
#pragma unroll
        for (int i = 0; i < 16; ++i) g[i] = r.rstd * fmaf(-xh[i], m2, g[i] - m1);
        if constexpr (RES) {
            float d[16];
            unpack16<T>(r.dres, d);
#pragma unroll
            for (int i = 0; i < 16; ++i) g[i] += d[i];
        }
        ln_store<T, ELEMENT>(dx + row * a.lddx, 0, G, tid, cols, a.wide, g);
    }

    float* out = a.parts + (uint64_t)(blockIdx.x / CLUSTER) * 2 * a.parts_pitch + origin;
    if (groups == 1) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t col = ln_col<ELEMENT>(0, i, G, tid);
            if (col < cols) {
                out[col] = dgamma[i];
                out[a.parts_pitch + col] = dbeta[i];
            }
        }
        // no block leaves while another may still write to its slots
        if (CLUSTER > 1) cooperative_groups::this_cluster().sync();
    } else {
        for (int k = 0; k < groups; ++k) {           // the groups in order
            if (group == k) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t col = ln_col<ELEMENT>(0, i, G, tid);
                    if (col < cols) {
                        columns[col] = dgamma[i] + (k ? columns[col] : 0.0f);
                        columns[pitch + col] = dbeta[i] + (k ? columns[pitch + col] : 0.0f);
                    }
                }
            }
            __syncthreads();
        }
        for (uint32_t col = threadIdx.x; col < cols; col += blockDim.x) {
            out[col] = columns[col];
            out[a.parts_pitch + col] = columns[pitch + col];
        }
    }
}

// dgamma, dbeta <- [their values +] the sum of the blocks' parts, in the order of the blocks
// within each of 8 interleaved groups, then of the groups
__global__ void __launch_bounds__(256)
ln_parts_kernel(const float* __restrict__ parts, const int blocks, const uint32_t pitch,
                const uint32_t cols, float* __restrict__ dgamma, float* __restrict__ dbeta,
                const bool accumulate) {
    __shared__ float sums[8][33];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const uint32_t col = blockIdx.x * 32 + lane;
    const float* p = parts + (blockIdx.y ? pitch : 0) + col;
    float s = 0.0f;
    if (col < cols)
        for (int b = group; b < blocks; b += 8) s += p[(uint64_t)b * 2 * pitch];
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

// how the rows are dealt out
struct LnDeal {
    int cluster, G, groups;              // blocks of a row, threads of a group, groups of a block
    uint64_t owners;                     // blocks (clusters) that are wanted at most
};

static LnDeal ln_deal(uint64_t rows, uint64_t cols) {
    LnDeal d;
    d.cluster = 1;
    while (cols > 16u * kLnBackThreads * d.cluster) d.cluster *= 2;
    const uint64_t share = (cols + d.cluster - 1) / d.cluster;
    d.G = (int)((share + 511) / 512 * 32);
    d.groups = d.G <= 128 ? 256 / d.G : 1;
    const uint64_t owners = (rows + d.groups - 1) / d.groups;
    d.owners = owners < (uint64_t)kLnMaxParts ? owners : (uint64_t)kLnMaxParts;
    return d;
}

template <typename T, bool ELEMENT, bool SAVED8, int CLUSTER>
static nc_status ln_backward_go(const LnBackward& a, const LnDeal& d, uint64_t blocks,
                                cudaStream_t stream) {
    auto kernel = a.dres ? ln_backward_kernel<T, ELEMENT, SAVED8, true, CLUSTER>
                         : ln_backward_kernel<T, ELEMENT, SAVED8, false, CLUSTER>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks * CLUSTER);
    cfg.blockDim = dim3(d.G * d.groups);
    cfg.dynamicSmemBytes = d.groups > 1 ? 2 * act8_pitch(a.cols) * sizeof(float) : 0;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    if (CLUSTER > 1) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = CLUSTER;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
    return cudaLaunchKernelEx(&cfg, kernel, a, d.G) == cudaSuccess ? NC_OK : NC_ERR_CUDA;
}

template <typename T, int CLUSTER>
static nc_status ln_backward_rows(const LnBackward& a, bool element, const LnDeal& d,
                                  uint64_t blocks, cudaStream_t stream) {
    auto go = element ? (a.codes ? ln_backward_go<T, true, true, CLUSTER>
                                 : ln_backward_go<T, true, false, CLUSTER>)
                      : (a.codes ? ln_backward_go<T, false, true, CLUSTER>
                                 : ln_backward_go<T, false, false, CLUSTER>);
    return go(a, d, blocks, stream);
}

template <typename T>
static nc_status ln_backward_launch(LnBackward a, bool element, float* dgamma, float* dbeta,
                                    bool accumulate, cudaStream_t stream) {
    uint64_t blocks = 0;
    if (a.rows) {
        // as many blocks as have the 512 threads that an SM's registers hold
        const LnDeal d = ln_deal(a.rows, a.cols);
        const uint64_t fit =
            (uint64_t)device_sm_count() * (kLnBackThreads / (d.G * d.groups)) / d.cluster;
        blocks = d.owners < fit ? d.owners : fit;
        const nc_status st = d.cluster == 1   ? ln_backward_rows<T, 1>(a, element, d, blocks, stream)
                             : d.cluster == 2 ? ln_backward_rows<T, 2>(a, element, d, blocks, stream)
                                              : ln_backward_rows<T, 4>(a, element, d, blocks, stream);
        if (st != NC_OK) return st;
    }
    ln_parts_kernel<<<dim3((a.cols + 31) / 32, 2), 256, 0, stream>>>(
        a.parts, (int)blocks, a.parts_pitch, a.cols, dgamma, dbeta, accumulate);
    return launch_status();
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
    a.params.vector = aligned16(a.params.gamma);
    a.params.has_gamma = a.params.gamma != nullptr;
    if (!a.params.has_gamma) a.params.gamma = a.dy;
    int access = row_access(a.dy, a.lddy, bytes, a.rows);
    const int others[3] = {row_access(a.dx, a.lddx, bytes, a.rows),
                           a.dres ? row_access(a.dres, a.lddres, bytes, a.rows) : kRowWide,
                           a.codes ? kRowWide : row_access(a.x, a.ldx, bytes, a.rows)};
    for (int o : others) access = o > access ? o : access;
    a.wide = access == kRowWide;
    const bool element = access == kRowElement;
    if (dtype == NC_DTYPE_F32)
        return ln_backward_launch<float>(a, element, dgamma, dbeta, accumulate != 0, stream);
    if (dtype == NC_DTYPE_BF16)
        return ln_backward_launch<__nv_bfloat16>(a, element, dgamma, dbeta, accumulate != 0,
                                                 stream);
    return ln_backward_launch<__half>(a, element, dgamma, dbeta, accumulate != 0, stream);
}

}  // namespace natcomp

using namespace natcomp;

extern "C" {

size_t nc_layer_norm_workspace_bytes(size_t rows, size_t cols) {
    if (cols > kLnMaxCols) return 0;                 // refused by the calls
    return ln_deal(rows, cols).owners * 2 * act8_pitch(cols) * sizeof(float);
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
    const LnParams params = {gamma ? gamma : x, beta ? beta : x, param_dtype,
                             aligned16(gamma) && aligned16(beta), gamma != nullptr,
                             beta != nullptr};
    LnForward a = {x, rows, (uint32_t)cols, ldx, params, eps, y, ldy, 0, mean, rstd, codes, scales,
                   kKeepNone, seed, worker};
    const int ax = row_access(x, ldx, bytes, rows), ay = row_access(y, ldy, bytes, rows);
    a.access = ax > ay ? ax : ay;
    if (codes) a.keep = rounding == NC_ROUND_RANDOM ? kKeepRandom : kKeepNearest;
    if (dtype == NC_DTYPE_F32)
        ln_forward_launch<float>(a, stream);
    else if (dtype == NC_DTYPE_BF16)
        ln_forward_launch<__nv_bfloat16>(a, stream);
    else
        ln_forward_launch<__half>(a, stream);
    return launch_status();
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
