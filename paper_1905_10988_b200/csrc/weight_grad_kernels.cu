// Weight gradient of a linear layer whose input is kept as an 8-bit checkpoint, for sm_100a.
//
//   dW[n][k] = sum_t dY[t][n] * (gamma[k] * xh[t][k] + beta[k])
//            = gamma[k] * (sum_t dY[t][n] * xh[t][k]) + beta[k] * db[n],   db[n] = sum_t dY[t][n]
//
// so one matrix product over the decoded checkpoint serves a layer behind a norm as well, and the
// affine part is a step of the epilogue.  The product runs on the tensor cores in bfloat16 with
// binary32 accumulation; a checkpoint's values are exact in bfloat16, so nothing is rounded on the
// way.  They exist as bfloat16 in shared memory only.
//
// A pair of blocks (cta_group::2) computes 256 x 256 values of dW; block r of it brings 128 of the
// n and 128 of the k.  Both operands have the tokens as their strided dimension, as they lie in
// memory.  A step is 64 tokens:
//   - warp 8 copies the dY tile by tensor copies (rows on 16-byte boundaries), or warps 10 to 17
//     gather it with plain loads (rows at any element);
//   - warps 0 to 7 hold the codes of the next four steps in registers, decode them and store them
//     in the swizzled operand layout;
//   - one thread of warp 9 of the pair's first block issues the matrix instructions.
// Few tiles: the tokens are split over several pairs, whose binary32 parts a second kernel adds in
// order.
#include "act8_common.cuh"
#include "tensor_core.cuh"

namespace natcomp {

constexpr int kWgTile = 256;             // n and k of a pair's tile
constexpr int kWgHalf = 128;             // of a block
constexpr int kWgStep = 64;              // tokens
constexpr int kWgStages = 6;
constexpr int kWgAhead = 4;              // steps whose codes are in flight
constexpr int kWgDecoders = 8, kWgLoaders = 8;       // warps
constexpr uint32_t kWgPanel = kWgStep * 128;         // bytes of 64 values x 64 tokens
constexpr uint32_t kWgOperand = 2 * kWgPanel;        // of a block's half
constexpr uint32_t kWgStageBytes = 2 * kWgOperand;
constexpr uint32_t kWgSmem = kWgStages * kWgStageBytes + 1024 + 256 + 2 * kWgTile * 4;
constexpr int kWgPairs = 74;             // pairs of blocks that the chip holds at a time
constexpr int kWgMinSteps = 8;           // of a split

struct WgArgs {
    const __nv_bfloat16* dy;
    uint64_t rows, n, lddy;
    const uint8_t *codes, *scales;
    uint64_t k, pitch;
    const void *gamma, *beta;
    int param_dtype;
    void* dw;
    int dw_f32;
    uint64_t lddw;
    const float* db;                     // complete when the product's epilogue reads it
    int accumulate, splits;
    bool vector;                         // dw rows may be written 16 bytes at a time
    float* parts;                        // [splits][n, rounded up to tiles][k, likewise]
};

__device__ __forceinline__ float wg_param(const void* p, int dtype, uint64_t i) {
    if (dtype == NC_DTYPE_F32) return static_cast<const float*>(p)[i];
    if (dtype == NC_DTYPE_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}

// what a decoder thread reads of one step: 16 codes in each of the two panels and their scales
struct WgCodes {
    uint4 c[2];
    uint32_t scale[2];
};

__device__ __forceinline__ void wg_load_codes(const WgArgs& a, uint64_t t, uint64_t k, WgCodes& r) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const uint64_t col = k + 64 * p;
        r.c[p] = make_uint4(0u, 0u, 0u, 0u);
        r.scale[p] = 127u;
        if (t < a.rows && col < a.pitch) {
            r.c[p] = __ldg(reinterpret_cast<const uint4*>(a.codes + t * a.pitch + col));
            r.scale[p] = __ldg(a.scales + ((t * a.pitch + col) >> 5));
        }
    }
}

// sixteen codes -> two swizzled 16-byte chunks of the thread's line
__device__ __forceinline__ void wg_decode(const uint4& c, uint32_t scale, uint32_t line,
                                          uint32_t chunk, uint32_t flip) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    uint32_t v[8];
    if (scale <= kAct8MaxFast) {
        const uint32_t fields = act8_fields(scale);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = act8_pair_bf16(w[i >> 1], i & 1, fields);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t two = w[i >> 1] >> (16 * (i & 1));
            v[i] = pack2<__nv_bfloat16>(act8_value(two & 0xFFu, scale),
                                        act8_value((two >> 8) & 0xFFu, scale));
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                         line + (((chunk + h) ^ flip) << 4)),
                     "r"(v[4 * h]), "r"(v[4 * h + 1]), "r"(v[4 * h + 2]), "r"(v[4 * h + 3])
                     : "memory");
}

// eight values of a dY row at any element
__device__ __forceinline__ uint4 wg_load_dy8(const WgArgs& a, uint64_t t, uint64_t n) {
    uint32_t v[4] = {0u, 0u, 0u, 0u};
    if (t < a.rows) {
        const unsigned short* p =
            reinterpret_cast<const unsigned short*>(a.dy) + t * a.lddy + n;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (n + i < a.n) v[i >> 1] |= (uint32_t)__ldg(p + i) << (16 * (i & 1));
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

template <bool COPY>
__global__ void __cluster_dims__(2, 1, 1)
__launch_bounds__(32 * (kWgDecoders + 2 + (COPY ? 0 : kWgLoaders)), 1)
wg_product_kernel(const __grid_constant__ WgArgs a, const __grid_constant__ CUtensorMap map) {
    extern __shared__ uint8_t raw[];
    uint8_t* base = reinterpret_cast<uint8_t*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const uint32_t tiles = smem_u32(base);
    uint64_t* bars = reinterpret_cast<uint64_t*>(base + kWgStages * kWgStageBytes);
    const uint32_t empty = smem_u32(bars);                       // [stages] operands consumed
    const uint32_t copied = empty + 8 * kWgStages;               // [stages] dY tile arrived
    const uint32_t ready = copied + 8 * kWgStages;               // [stages] both blocks' operands
    const uint32_t done = ready + 8 * kWgStages;                 // the tile's product
    uint32_t* words = reinterpret_cast<uint32_t*>(bars + 3 * kWgStages + 1);
    volatile uint32_t* gave_up = words + 1;
    float* affine = reinterpret_cast<float*>(base + kWgStages * kWgStageBytes + 256);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const uint64_t n0 = (uint64_t)(blockIdx.x >> 1) * kWgTile + rank * kWgHalf;   // of A and D rows
    const uint64_t k0 = (uint64_t)blockIdx.y * kWgTile;
    const uint64_t all = (a.rows + kWgStep - 1) / kWgStep;
    const int first = (int)(all * blockIdx.z / a.splits);
    const int steps = (int)(all * (blockIdx.z + 1) / a.splits) - first;
    const uint64_t t0 = (uint64_t)first * kWgStep;

    if (warp == kWgDecoders + 1) tmem_alloc_pair(smem_u32(words), kWgTile);
    if (threadIdx.x == 0) {
        words[1] = 0;
        for (int s = 0; s < kWgStages; ++s) {
            mbar_init(empty + 8 * s, 1);
            mbar_init(copied + 8 * s, 1);
            mbar_init(ready + 8 * s, 2 * (kWgDecoders + (COPY ? 0 : kWgLoaders)));
        }
        mbar_init(done, 1);
        mbar_init_fence();
    }
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = words[0];

    if (warp < kWgDecoders) {
        // ---- decode: the thread's token and its sixteen values of each panel.  Four lanes cover
        // half a line and eight lanes two lines, whose swizzles differ: no bank is hit twice.
        const uint32_t token = threadIdx.x >> 2, quarter = threadIdx.x & 3;
        const uint64_t k = k0 + rank * kWgHalf + 16 * quarter;
        WgCodes r[kWgAhead];
#pragma unroll
        for (int u = 0; u < kWgAhead; ++u)
            if (u < steps) wg_load_codes(a, t0 + u * kWgStep + token, k, r[u]);
        uint32_t stage = 0, parity = 1;
        bool ok = true;
        for (int s0 = 0; s0 < steps && ok; s0 += kWgAhead) {
#pragma unroll
            for (int u = 0; u < kWgAhead; ++u) {
                const int s = s0 + u;
                if (s < steps && ok) {
                    ok = mbar_wait(empty + 8 * stage, parity, gave_up);
                    const uint32_t line =
                        tiles + stage * kWgStageBytes + kWgOperand + token * 128;
#pragma unroll
                    for (int p = 0; p < 2; ++p)
                        wg_decode(r[u].c[p], r[u].scale[p], line + p * kWgPanel, 2 * quarter,
                                  token & 7);
                    if (s + kWgAhead < steps)
                        wg_load_codes(a, t0 + (uint64_t)(s + kWgAhead) * kWgStep + token, k, r[u]);
                    fence_async_proxy();
                    __syncwarp();
                    if (lane == 0) {
                        // the pair's first block hears of the dY tile through the decoders
                        if (COPY && ok) ok = mbar_wait(copied + 8 * stage, parity ^ 1, gave_up);
                        mbar_arrive_at(ready + 8 * stage, 0);
                    }
                    ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
                    if (++stage == kWgStages) {
                        stage = 0;
                        parity ^= 1;
                    }
                }
            }
        }
        // ---- epilogue: lane = row of D, a warp takes half of the columns
        for (int i = threadIdx.x; i < kWgTile; i += 32 * kWgDecoders) {
            const bool in = k0 + i < a.k;
            affine[i] = a.gamma && in ? wg_param(a.gamma, a.param_dtype, k0 + i) : 1.0f;
            affine[kWgTile + i] = a.beta && in ? wg_param(a.beta, a.param_dtype, k0 + i) : 0.0f;
        }
        asm volatile("bar.sync 1, %0;" ::"r"(32 * kWgDecoders) : "memory");
        ok = mbar_wait(done, 0, gave_up) && ok && !*gave_up;
        tc_fence_after();
        const uint64_t n = n0 + 32 * (warp & 3) + lane;
        const int half = (warp >> 2) * kWgHalf;
        const uint64_t padded_n = (uint64_t)(gridDim.x >> 1) * kWgTile;
        const uint64_t padded_k = (uint64_t)gridDim.y * kWgTile;
        const float add = a.splits == 1 && a.beta && n < a.n ? a.db[n] : 0.0f;
#pragma unroll 1
        for (int c = 0; c < kWgHalf; c += 32) {
            float v[32];
            tmem_load32(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + half + c, v);
            if (!ok) {               // a wait ran out: the result must not pass for one
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(0x7FC00000u);
            }
            const uint64_t k = k0 + half + c;
            if (a.splits > 1) {
                float4* p = reinterpret_cast<float4*>(
                    a.parts + (blockIdx.z * padded_n + n) * padded_k + k);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    p[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                continue;
            }
            if (n >= a.n || k >= a.k) continue;
#pragma unroll
            for (int i = 0; i < 32; ++i)
                v[i] = fmaf(v[i], affine[half + c + i], add * affine[kWgTile + half + c + i]);
            if (a.dw_f32) {
                float* p = static_cast<float*>(a.dw) + n * a.lddw + k;
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    if (a.vector && k + i + 4 <= a.k) {
                        float4 o = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                        if (a.accumulate) {
                            const float4 old = *reinterpret_cast<const float4*>(p + i);
                            o.x += old.x; o.y += old.y; o.z += old.z; o.w += old.w;
                        }
                        *reinterpret_cast<float4*>(p + i) = o;
                    } else {
#pragma unroll
                        for (int j = i; j < i + 4; ++j)
                            if (k + j < a.k) p[j] = a.accumulate ? p[j] + v[j] : v[j];
                    }
                }
            } else {
                __nv_bfloat16* p = static_cast<__nv_bfloat16*>(a.dw) + n * a.lddw + k;
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    if (a.vector && k + i + 8 <= a.k) {
                        uint4* q = reinterpret_cast<uint4*>(p + i);
                        uint32_t o[4];
                        if (a.accumulate) {
                            const uint4 old = *q;
                            const uint32_t w[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                float e, f;
                                unpack2<__nv_bfloat16>(w[j], e, f);
                                v[i + 2 * j] += e;
                                v[i + 2 * j + 1] += f;
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            o[j] = pack2<__nv_bfloat16>(v[i + 2 * j], v[i + 2 * j + 1]);
                        *q = make_uint4(o[0], o[1], o[2], o[3]);
                    } else {
#pragma unroll
                        for (int j = i; j < i + 8; ++j)
                            if (k + j < a.k)
                                p[j] = __float2bfloat16_rn(
                                    a.accumulate ? __bfloat162float(p[j]) + v[j] : v[j]);
                    }
                }
            }
        }
        tc_fence_before();
    } else if (warp == kWgDecoders) {
        // ---- copies of the dY tile: two panels of 64 n
        if (COPY && lane == 0) {
            uint32_t stage = 0, parity = 1;
            int s = 0;
            for (; s < steps; ++s) {
                if (!mbar_wait(empty + 8 * stage, parity, gave_up)) break;
                const uint32_t dst = tiles + stage * kWgStageBytes;
                mbar_expect(copied + 8 * stage, kWgOperand);
                for (int p = 0; p < 2; ++p)
                    tma_load_2d(dst + p * kWgPanel, &map, (int)(n0 + 64 * p),
                                (int)(t0 + (uint64_t)s * kWgStep), copied + 8 * stage);
                if (++stage == kWgStages) {
                    stage = 0;
                    parity ^= 1;
                }
            }
            // given up: the copies in flight still land before the block may end
            if (s < steps) {
                const long long begin = clock64();
                for (int back = 1; back <= kWgStages && back <= s; ++back) {
                    const int i = s - back;
                    while (!mbar_try(copied + 8 * (i % kWgStages), (i / kWgStages) & 1) &&
                           clock64() - begin < 4000000000ll) {}
                }
            }
        }
    } else if (warp == kWgDecoders + 1) {
        // ---- matrix instructions
        if (rank == 0 && lane == 0) {
            uint32_t stage = 0, parity = 0;
            const uint32_t shape = mma_shape(kWgTile, kWgTile);
            for (int s = 0; s < steps; ++s) {
                if (!mbar_wait(ready + 8 * stage, parity, gave_up)) break;
                tc_fence_after();
                const uint32_t at = tiles + stage * kWgStageBytes;
#pragma unroll
                for (int i = 0; i < kWgStep / 16; ++i)      // 16 tokens are two groups of lines
                    mma_pair(tmem, mma_operand(at + 2048 * i, kWgPanel),
                             mma_operand(at + kWgOperand + 2048 * i, kWgPanel), shape,
                             s > 0 || i > 0);
                mma_commit_pair(empty + 8 * stage);
                if (++stage == kWgStages) {
                    stage = 0;
                    parity ^= 1;
                }
            }
            mma_commit_pair(done);
        }
    } else if (!COPY) {
        // ---- plain loads of the dY tile, a step ahead: 16 lanes cover the 128 n of a token
        const int i0 = threadIdx.x - 32 * (kWgDecoders + 2);
        const uint32_t chunk = i0 & 15, token0 = i0 >> 4;          // tokens token0 + 16 j
        const uint64_t n = n0 + 8 * chunk;
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = wg_load_dy8(a, t0 + token0 + 16 * j, n);
        uint32_t stage = 0, parity = 1;
        for (int s = 0; s < steps; ++s) {
            bool ok = mbar_wait(empty + 8 * stage, parity, gave_up);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            const uint32_t dst = tiles + stage * kWgStageBytes + (chunk >> 3) * kWgPanel;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t token = token0 + 16 * j;
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                                 dst + token * 128 + (((chunk & 7) ^ (token & 7)) << 4)),
                             "r"(v[j].x), "r"(v[j].y), "r"(v[j].z), "r"(v[j].w)
                             : "memory");
            }
            if (s + 1 < steps) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v[j] = wg_load_dy8(a, t0 + (uint64_t)(s + 1) * kWgStep + token0 + 16 * j, n);
            }
            fence_async_proxy();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(ready + 8 * stage, 0);
            if (++stage == kWgStages) {
                stage = 0;
                parity ^= 1;
            }
        }
    }
    // the pair stays until both blocks are done with each other's barriers and with TMEM
    __syncwarp();
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    if (warp == kWgDecoders + 1) tmem_free_pair(tmem, kWgTile);
}

// dw <- [dw +] gamma * (sum of the parts, in order) + beta * db; no parts: the sum over no tokens
__global__ void __launch_bounds__(256)
wg_join_kernel(const __grid_constant__ WgArgs a, const uint64_t padded_n, const uint64_t padded_k) {
    const uint64_t k = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (k >= a.k) return;
    for (uint64_t n = blockIdx.y; n < a.n; n += gridDim.y) {
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int z = 0; z < a.splits; ++z) {
            const float4 p = __ldcs(
                reinterpret_cast<const float4*>(a.parts + (z * padded_n + n) * padded_k + k));
            s.x += p.x; s.y += p.y; s.z += p.z; s.w += p.w;
        }
        float v[4] = {s.x, s.y, s.z, s.w};
        const float add = a.beta ? a.db[n] : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (k + i >= a.k) break;
            if (a.gamma) v[i] *= wg_param(a.gamma, a.param_dtype, k + i);
            if (a.beta) v[i] = fmaf(add, wg_param(a.beta, a.param_dtype, k + i), v[i]);
            if (a.dw_f32) {
                float* p = static_cast<float*>(a.dw) + n * a.lddw + k + i;
                *p = a.accumulate ? *p + v[i] : v[i];
            } else {
                __nv_bfloat16* p = static_cast<__nv_bfloat16*>(a.dw) + n * a.lddw + k + i;
                *p = __float2bfloat16_rn(a.accumulate ? __bfloat162float(*p) + v[i] : v[i]);
            }
        }
    }
}

// ---- column sums of dY: parts of kWgSumRows rows, then their sum ----------------------------------
constexpr int kWgSumBlocks = 256;

__global__ void __launch_bounds__(256)
wg_sums_kernel(const __nv_bfloat16* __restrict__ dy, const uint64_t rows, const uint64_t n,
               const uint64_t lddy, float* __restrict__ parts) {
    __shared__ float sums[8][33];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const uint64_t col = (uint64_t)blockIdx.x * 32 + lane;
    const uint64_t begin = rows * blockIdx.y / gridDim.y, end = rows * (blockIdx.y + 1) / gridDim.y;
    float s = 0.0f;
    if (col < n)
        for (uint64_t t = begin + group; t < end; t += 8) s += __bfloat162float(dy[t * lddy + col]);
    sums[group][lane] = s;
    __syncthreads();
    if (group == 0 && col < n) {
        s = sums[0][lane];
#pragma unroll
        for (int g = 1; g < 8; ++g) s += sums[g][lane];
        parts[blockIdx.y * n + col] = s;
    }
}

// db <- [db +] the parts' sum; `fresh` (may be db) gets the sum alone
__global__ void __launch_bounds__(256)
wg_sums_join_kernel(const float* __restrict__ parts, const int blocks, const uint64_t n,
                    float* fresh, float* db, const bool accumulate) {
    const uint64_t col = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (col >= n) return;
    float s = 0.0f;
    for (int b = 0; b < blocks; ++b) s += parts[b * n + col];
    if (fresh) fresh[col] = s;
    if (db) db[col] = accumulate ? db[col] + s : s;
}

struct WgPlan {
    uint64_t tiles_n, tiles_k;
    int splits, sum_blocks;
    size_t sum_offset, fresh_offset, bytes;
};

static WgPlan wg_plan(uint64_t rows, uint64_t n, uint64_t k) {
    WgPlan p = {};
    p.tiles_n = (n + kWgTile - 1) / kWgTile;
    p.tiles_k = (k + kWgTile - 1) / kWgTile;
    const uint64_t tiles = p.tiles_n * p.tiles_k, steps = (rows + kWgStep - 1) / kWgStep;
    uint64_t splits = tiles ? kWgPairs / tiles : 1;
    if (splits > steps / kWgMinSteps) splits = steps / kWgMinSteps;
    p.splits = (int)(splits < 1 ? 1 : splits);
    const uint64_t sum_tiles = (n + 31) / 32;
    uint64_t blocks = sum_tiles ? 8 * 148 / sum_tiles : 1;
    if (blocks > (rows + 63) / 64) blocks = (rows + 63) / 64;
    if (blocks > kWgSumBlocks) blocks = kWgSumBlocks;
    p.sum_blocks = (int)(blocks < 1 ? 1 : blocks);
    p.sum_offset = p.splits > 1 ? p.splits * tiles * kWgTile * kWgTile * 4 : 0;
    p.fresh_offset = p.sum_offset + round_up16(p.sum_blocks * n * 4);
    p.bytes = p.fresh_offset + round_up16(n * 4);
    return p;
}

}  // namespace natcomp

using namespace natcomp;

extern "C" {

size_t nc_act8_weight_grad_workspace_bytes(size_t rows, size_t n, size_t k) {
    if (n > ((size_t)1 << 31) || k > ((size_t)1 << 31) || rows > ((size_t)1 << 31)) return 0;
    return wg_plan(rows, n, k).bytes;
}

nc_status nc_act8_weight_grad(const void* dy, size_t rows, size_t n, size_t lddy,
                              const uint8_t* codes, const uint8_t* scales, size_t k,
                              const void* gamma, const void* beta, int param_dtype, void* dw,
                              int dw_dtype, size_t lddw, float* db, int accumulate,
                              void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    const int pbytes = act8_type_bytes(param_dtype);
    if (!pbytes || (dw_dtype != NC_DTYPE_F32 && dw_dtype != NC_DTYPE_BF16))
        return NC_ERR_UNSUPPORTED;
    if (n == 0) return NC_OK;
    if (k && (!dw || lddw < k)) return NC_ERR_INVALID;
    if (rows && (!dy || lddy < n || !workspace || (k && (!codes || !scales))))
        return NC_ERR_INVALID;
    if (rows >= ((size_t)1 << 31) || n >= ((size_t)1 << 31) || k >= ((size_t)1 << 23) ||
        !act8_fits(rows, k))
        return NC_ERR_TOO_LARGE;
    const int wbytes = dw_dtype == NC_DTYPE_F32 ? 4 : 2;
    if (!element_aligned(dy, 2) || !element_aligned(gamma, pbytes) ||
        !element_aligned(beta, pbytes) || !element_aligned(dw, wbytes) || !aligned4(db) ||
        !aligned16(codes) || !aligned16(scales) || !aligned16(workspace))
        return NC_ERR_ALIGN;
    const WgPlan p = wg_plan(rows, n, k);
    if (rows && workspace_bytes < p.bytes) return NC_ERR_WORKSPACE;

    char* ws = static_cast<char*>(workspace);
    float* fresh = reinterpret_cast<float*>(ws + p.fresh_offset);
    const bool with_beta = beta && k && rows;
    if (db || with_beta) {
        float* sums = reinterpret_cast<float*>(ws + p.sum_offset);
        if (rows)
            wg_sums_kernel<<<dim3((unsigned)((n + 31) / 32), p.sum_blocks), 256, 0, stream>>>(
                static_cast<const __nv_bfloat16*>(dy), rows, n, lddy, sums);
        wg_sums_join_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(
            sums, rows ? p.sum_blocks : 0, n, with_beta ? fresh : nullptr, db, accumulate != 0);
    }
    if (k == 0) return launch_status();

    WgArgs a = {};
    a.dy = static_cast<const __nv_bfloat16*>(dy);
    a.rows = rows; a.n = n; a.lddy = lddy; a.codes = codes; a.scales = scales; a.k = k;
    a.pitch = act8_pitch(k); a.gamma = gamma; a.beta = with_beta ? beta : nullptr;
    a.param_dtype = param_dtype; a.dw = dw; a.dw_f32 = dw_dtype == NC_DTYPE_F32; a.lddw = lddw;
    a.db = fresh; a.accumulate = accumulate; a.splits = rows ? p.splits : 0;
    a.vector = row_access(dw, lddw, wbytes, n) != kRowElement;
    a.parts = reinterpret_cast<float*>(ws);
    if (rows) {
        const bool copy = row_access(dy, lddy, 2, rows) != kRowElement;
        CUtensorMap map = {};
        if (copy && !make_tensor_map(&map, dy, rows, n, rows > 1 ? lddy : (n + 7) / 8 * 8, 64,
                                     kWgStep))
            return NC_ERR_CUDA;
        auto kernel = copy ? wg_product_kernel<true> : wg_product_kernel<false>;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kWgSmem) !=
            cudaSuccess)
            return NC_ERR_CUDA;
        const dim3 grid((unsigned)(2 * p.tiles_n), (unsigned)p.tiles_k, (unsigned)p.splits);
        kernel<<<grid, 32 * (kWgDecoders + 2 + (copy ? 0 : kWgLoaders)), kWgSmem, stream>>>(a, map);
    }
    if (a.splits != 1) {
        const unsigned across = (unsigned)((k + 1023) / 1024);
        const unsigned down = (unsigned)(n < 4096 ? n : 4096);
        wg_join_kernel<<<dim3(across, down), 256, 0, stream>>>(a, p.tiles_n * kWgTile,
                                                               p.tiles_k * kWgTile);
    }
    return launch_status();
}

}  // extern "C"
