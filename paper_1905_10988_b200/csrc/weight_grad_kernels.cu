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
// A pair of blocks (cta_group::2) computes tiles of dW one after another: 256 x 256 values, or two
// neighbours along n at a time, 512 x 256; block r of the pair brings 128 of each 256 n and 128 of
// the k.  What bounds a step is shared memory: it takes the dY tile, the decoded tile and the
// codes, and the tensor cores read both tiles.  Two tiles at a time share the decoded one.  Both
// operands have the tokens as their strided dimension, as they lie in memory.  A step is 64 tokens,
// and its operands pass through a ring in shared memory:
//   - one thread copies the dY tile by tensor copies (rows on 16-byte boundaries), or four warps
//     gather it with plain loads (rows at any element);
//   - another thread copies the codes and their scale bytes, which a small kernel has laid out by
//     columns of 128 beforehand, so that a step's are 256 neighbouring bytes and not a byte or four
//     of each of 64 lines;
//   - sixteen warps decode, in four groups that take every fourth step;
//   - one thread of the pair's first block issues the matrix instructions; TMEM holds two tiles, so
//     four more warps write one out while the next is computed.
// A sum over many tokens is made of chains: the accumulator goes to memory after each and is added up
// there (kWgChainF32 below).
// The tiles are dealt out evenly to the chip's 74 pairs, double ones while there are rounds of
// them, then single ones.  What is left over, fewer tiles than pairs, is split along the tokens,
// and a second kernel adds its binary32 parts in order.
//
// 16384 x 4096 x 4096: the product 390 us (1.41 PFLOP/s, the tensor pipe active 77 % of the cycles;
// 400 to 445 us back to back, where the power cap lowers the clock), all kernels 440 to 490 us.
#include "act8_common.cuh"
#include "tensor_core.cuh"

namespace natcomp {

constexpr int kWgTile = 256;             // n and k of a pair's tile
constexpr int kWgHalf = 128;             // of a block
constexpr int kWgStep = 64;              // tokens
constexpr int kWgPlaces = 6;             // places of dY tiles
constexpr int kWgSlots = 5;              // places of codes and of decoded tiles
constexpr int kWgGroups = 4, kWgGroupWarps = 4;      // decoders
// Steps that barriers tell apart.  A wait by parity cannot tell a phase from the one before the last,
// so whoever waits for a step must know that the step which used the barrier before is over: a
// decoding group has waited for that one itself, because it takes every fourth step and the barrier
// comes round after a multiple of four.
constexpr int kWgRing = 8;
static_assert(kWgRing % kWgGroups == 0 && kWgRing >= kWgPlaces && kWgRing >= kWgSlots, "");
constexpr int kWgWriters = 4, kWgLoaders = 4;        // warps
constexpr int kWgCopyWarp = kWgWriters, kWgCodeWarp = kWgWriters + 1, kWgMmaWarp = kWgWriters + 2;
constexpr int kWgDecodeWarp = kWgWriters + 4;        // the first of them, a multiple of four
constexpr int kWgLoadWarp = kWgDecodeWarp + kWgGroups * kWgGroupWarps;
constexpr uint32_t kWgPanel = kWgStep * 128;         // bytes of 64 values x 64 tokens
constexpr uint32_t kWgOperand = 2 * kWgPanel;        // of a block's half
constexpr uint32_t kWgCodeBytes = kWgStep * 128, kWgScaleBytes = kWgStep * 4;
// shared memory: dY tiles, decoded tiles, codes, scales, barriers, gamma and beta
constexpr uint32_t kWgDecoded = kWgPlaces * kWgOperand;
constexpr uint32_t kWgCodes = kWgDecoded + kWgSlots * kWgOperand;
constexpr uint32_t kWgScales = kWgCodes + kWgSlots * kWgCodeBytes;
constexpr uint32_t kWgBars = kWgScales + kWgSlots * kWgScaleBytes;
constexpr uint32_t kWgRows = 32 * 9 * 4;             // a writer warp's rows in passing
constexpr uint32_t kWgSmem = kWgBars + 512 + 2 * kWgTile * 4 + kWgWriters * kWgRows + 1024;
constexpr int kWgPairs = 74;             // pairs of blocks that the chip holds at a time
constexpr int kWgMinSteps = 4;           // of a part
// Most steps that an accumulator adds up before its sums go to memory and are added up there, by the
// type of dW.  The tensor cores cut off what does not fit 24 bits, always towards 0, so the relative
// error grows with the length of a chain: in the norm of a binary32 dW 4.6e-7 after 2048 tokens, 1.1e-6
// after 4096, 2.9e-6 after 8192, 7e-6 after 16384, 4.4e-5 after 65536 (a product in binary32: 5e-7 and
// 1.5e-6 at the last two), and a sum of chains keeps that of one.  Emptying both tiles of TMEM takes 15
// to 20 us, in which the pair's tensor cores stand still.  binary32, 16384 x 4096 x 4096: 415 us as one
// chain, 435 in chains of 8192 tokens, 457 of 4096, 495 of 2048.  Where bfloat16 rounds the result by
// 1.7e-3 the cut is below a hundredth of that up to 16384.
constexpr uint32_t kWgChainF32 = 128;
constexpr uint32_t kWgChainBf16 = 256;
constexpr uint32_t kWgTileFours = kWgTile / 4 * kWgTile;     // groups of four values of a tile

struct WgArgs {
    const __nv_bfloat16* dy;
    uint64_t rows, n, lddy;
    uint64_t k;
    const uint32_t* scales;              // [columns of 128][token_pitch]: four scale bytes each
    uint64_t token_pitch;
    const void *gamma, *beta;
    int param_dtype;
    void* dw;
    int dw_f32;
    uint64_t lddw;
    const float* db;                     // complete when dW is written
    int accumulate;
    bool vector;                         // dw rows may be written 16 bytes at a time
    uint32_t tiles_n, tiles_k;           // of 256 x 256
    uint32_t rounds;                     // of double tiles; double tile i: n tiles 2 (i % m) and
                                         // one more, m = tiles_n / 2, k tile i / m
    uint32_t tiles;                      // single ones after that
    uint32_t whole, splits;              // those from `whole` on are computed in `splits` parts
    float* parts;                        // [tile - whole][part][k / 4][256 n][4]
    uint32_t chain;                      // steps of a chain at most
    float* runs;                         // [pair][half][k / 4][256 n][4]: sums of a tile's chains
};

__device__ __forceinline__ float wg_param(const void* p, int dtype, uint64_t i) {
    if (dtype == NC_DTYPE_F32) return static_cast<const float*>(p)[i];
    if (dtype == NC_DTYPE_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}

// the u-th piece of work of a pair: a chain of the steps of a double tile, of a single one, or of a
// part of one
struct WgUnit {
    uint32_t tile, part, first, steps;   // steps == 0: no more work
    uint32_t chain, chains;              // of the tile or the part
    uint32_t halves;                     // tiles of 256 n
    uint64_t n0, k0;
};

// place of the single tile `i`: first the halves of the double tiles that no round has taken, then
// the last column of an odd number
__device__ __forceinline__ void wg_single(const WgArgs& a, uint32_t i, uint64_t& n0, uint64_t& k0) {
    const uint32_t m = a.tiles_n / 2, taken = a.rounds * kWgPairs, left = 2 * (m * a.tiles_k - taken);
    if (i < left) {
        const uint32_t d = taken + i / 2;
        n0 = (uint64_t)(2 * (d % m) + (i & 1)) * kWgTile;
        k0 = (uint64_t)(d / m) * kWgTile;
    } else {
        n0 = (uint64_t)(a.tiles_n - 1) * kWgTile;
        k0 = (uint64_t)(i - left) * kWgTile;
    }
}

template <bool CHAINS>
__device__ __forceinline__ WgUnit wg_unit(const WgArgs& a, uint32_t pair, uint32_t u) {
    const uint32_t all = (uint32_t)((a.rows + kWgStep - 1) / kWgStep);
    const uint32_t pairs = gridDim.x >> 1, rounds = a.whole / pairs;
    WgUnit w = {};
    w.halves = 1;
    w.chains = CHAINS ? (all + a.chain - 1) / a.chain : 1;
    uint32_t steps = all, piece = CHAINS ? u / w.chains : u;
    if (piece < a.rounds + rounds) {
        w.chain = CHAINS ? u % w.chains : 0;
    } else {                             // the last piece: a part of a tile
        if (pair >= (a.tiles - a.whole) * a.splits) return w;
        w.tile = a.whole + pair / a.splits;
        w.part = pair % a.splits;
        w.first = (uint32_t)((uint64_t)all * w.part / a.splits);
        steps = (uint32_t)((uint64_t)all * (w.part + 1) / a.splits) - w.first;
        w.chain = u - (a.rounds + rounds) * w.chains;
        if (CHAINS) w.chains = (steps + a.chain - 1) / a.chain;
        if (w.chain >= w.chains) return w;
    }
    if (piece < a.rounds) {
        const uint32_t m = a.tiles_n / 2, d = piece * pairs + pair;
        w.halves = 2;
        w.n0 = (uint64_t)(d % m) * (2 * kWgTile);
        w.k0 = (uint64_t)(d / m) * kWgTile;
    } else {
        if (piece < a.rounds + rounds) w.tile = (piece - a.rounds) * pairs + pair;
        wg_single(a, w.tile, w.n0, w.k0);
    }
    w.steps = steps;
    if (CHAINS) {
        const uint32_t begin = (uint32_t)((uint64_t)steps * w.chain / w.chains);
        w.first += begin;
        w.steps = (uint32_t)((uint64_t)steps * (w.chain + 1) / w.chains) - begin;
    }
    return w;
}

// which of the two accumulators in TMEM a unit's tiles use, and how often each was used before
struct WgTurns {
    uint32_t uses[2], next;
    __device__ __forceinline__ WgTurns() : uses{0u, 0u}, next(0u) {}
    __device__ __forceinline__ uint32_t of(const WgUnit& w, uint32_t half) const {
        return w.halves == 2 ? half : next;
    }
    __device__ __forceinline__ void done(const WgUnit& w) {
        if (w.halves == 2) {
            ++uses[0];
            ++uses[1];
        } else {
            if (next) ++uses[1]; else ++uses[0];
            next ^= 1;
        }
    }
    __device__ __forceinline__ uint32_t parity(uint32_t b) const {
        return (b ? uses[1] : uses[0]) & 1;
    }
};

// a place in a pair's sequence of steps
template <bool CHAINS> struct WgWalk {
    WgUnit unit;
    uint32_t u, step;
    __device__ __forceinline__ void begin(const WgArgs& a, uint32_t pair) {
        u = 0;
        step = 0;
        unit = wg_unit<CHAINS>(a, pair, 0);
    }
    __device__ __forceinline__ bool more() const { return unit.steps != 0; }
    __device__ __forceinline__ void advance(const WgArgs& a, uint32_t pair, uint32_t by) {
        step += by;
        while (unit.steps != 0 && step >= unit.steps) {
            step -= unit.steps;
            unit = wg_unit<CHAINS>(a, pair, ++u);
        }
    }
    __device__ __forceinline__ uint64_t token() const {
        return (uint64_t)(unit.first + step) * kWgStep;
    }
};

// a place in the ring of stages
struct WgRing {
    uint32_t stage, parity;
    __device__ __forceinline__ void advance(uint32_t by) {
        stage += by;
        if (stage >= kWgRing) {
            stage -= kWgRing;
            parity ^= 1;
        }
    }
};

// sixteen codes -> eight pairs of bfloat16; FAST: the scale byte is at most kAct8MaxFast
template <bool FAST>
__device__ __forceinline__ void wg_decode(const uint32_t (&w)[4], uint32_t scale, uint32_t (&v)[8]) {
    const uint32_t fields = act8_fields(scale);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (FAST) {
            v[i] = act8_pair_bf16(w[i >> 1], i & 1, fields);
        } else {
            const uint32_t two = w[i >> 1] >> (16 * (i & 1));
            v[i] = pack2<__nv_bfloat16>(act8_value(two & 0xFFu, scale),
                                        act8_value((two >> 8) & 0xFFu, scale));
        }
    }
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

// eight neighbouring values of dW
__device__ __forceinline__ void wg_store8(const WgArgs& a, uint64_t n, uint64_t k, float (&v)[8]) {
    const bool vector = a.vector && k + 8 <= a.k;
    if (a.dw_f32) {
        float* p = static_cast<float*>(a.dw) + n * a.lddw + k;
        if (vector) {
            float4* q = reinterpret_cast<float4*>(p);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float4 o = make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
                if (a.accumulate) {
                    const float4 old = q[h];
                    o.x += old.x; o.y += old.y; o.z += old.z; o.w += old.w;
                }
                q[h] = o;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < a.k) p[i] = a.accumulate ? p[i] + v[i] : v[i];
        }
    } else {
        __nv_bfloat16* p = static_cast<__nv_bfloat16*>(a.dw) + n * a.lddw + k;
        if (vector) {
            uint4* q = reinterpret_cast<uint4*>(p);
            if (a.accumulate) {
                const uint4 old = *q;
                const uint32_t w[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float e, f;
                    unpack2<__nv_bfloat16>(w[i], e, f);
                    v[2 * i] += e;
                    v[2 * i + 1] += f;
                }
            }
            *q = make_uint4(pack2<__nv_bfloat16>(v[0], v[1]), pack2<__nv_bfloat16>(v[2], v[3]),
                            pack2<__nv_bfloat16>(v[4], v[5]), pack2<__nv_bfloat16>(v[6], v[7]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < a.k)
                    p[i] = __float2bfloat16_rn(a.accumulate ? __bfloat162float(p[i]) + v[i] : v[i]);
        }
    }
}

// eight neighbouring values of the 32 rows of a warp, a row a lane, where rows cannot be written by 16
// bytes: they change places in shared memory, so that the lanes write neighbouring values
__device__ __forceinline__ void wg_store_rows(const WgArgs& a, uint64_t n0, uint64_t k,
                                              const float (&v)[8], uint32_t* rows) {
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) rows[lane * 9 + i] = __float_as_uint(v[i]);
    __syncwarp();
    const uint64_t col = k + (lane & 7);
    const uint32_t row = lane >> 3;
    const uint64_t at = (n0 + row) * a.lddw + col, step = 4 * a.lddw;
    const int count = col >= a.k || n0 + row >= a.n ? 0 : (int)min((a.n - n0 - row + 3) / 4, (uint64_t)8);
    if (a.dw_f32) {
        float* p = static_cast<float*>(a.dw) + at;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float o = __uint_as_float(rows[(4 * i + row) * 9 + (lane & 7)]);
            if (i < count) p[i * step] = a.accumulate ? p[i * step] + o : o;
        }
    } else {
        __nv_bfloat16* p = static_cast<__nv_bfloat16*>(a.dw) + at;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float o = __uint_as_float(rows[(4 * i + row) * 9 + (lane & 7)]);
            if (i < count)
                p[i * step] = __float2bfloat16_rn(
                    a.accumulate ? __bfloat162float(p[i * step]) + o : o);
        }
    }
}

// a chain's sums of a warp's 32 rows, to memory or on top of what stands there
__device__ __forceinline__ void wg_empty(float4* sums, uint32_t from, bool ok, bool first) {
#pragma unroll 1
    for (int c = 0; c < kWgTile; c += 32) {
        uint32_t r[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j) tmem_load8(from + c + 8 * j, r[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j) tmem_wait8(r[j]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)              // NaN: a wait ran out, no result
                v[i] = ok ? __uint_as_float(r[j / 2][4 * (j & 1) + i]) : __uint_as_float(0x7FC00000u);
            float4* to = sums + (c / 4 + j) * kWgTile;
            if (first)
                *to = make_float4(v[0], v[1], v[2], v[3]);
            else
                global_add4(to, v[0], v[1], v[2], v[3]);
        }
    }
}

// waits until the barrier of step number `step` among `bars` is over
__device__ __forceinline__ bool wg_wait_step(uint32_t bars, uint32_t step,
                                             volatile uint32_t* gave_up) {
    return mbar_wait(bars + 8 * (step % kWgRing), (step / kWgRing) & 1, gave_up);
}

// CHAINS: a tile's steps are more than one chain
template <bool COPY, bool CHAINS>
__global__ void __cluster_dims__(2, 1, 1)
__launch_bounds__(32 * (kWgLoadWarp + (COPY ? 0 : kWgLoaders)), 1)
wg_product_kernel(const __grid_constant__ WgArgs a, const __grid_constant__ CUtensorMap map,
                  const __grid_constant__ CUtensorMap code_map) {
    extern __shared__ uint8_t raw[];
    uint8_t* base = reinterpret_cast<uint8_t*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const uint32_t tiles = smem_u32(base);
    uint64_t* bars = reinterpret_cast<uint64_t*>(base + kWgBars);
    // Barriers by step (step % kWgRing).  The thread that issues the matrix instructions waits for
    // one of them and commits to one a step: every further wait would leave the tensor cores idle.
    const uint32_t empty = smem_u32(bars);             // operands consumed
    const uint32_t ready = empty + 8 * kWgRing;      // first block's: both blocks' operands are there
    const uint32_t copied = ready + 8 * kWgRing;     // second block's: its dY tiles arrived
    const uint32_t coded = copied + 8 * kWgRing;     // the block's codes arrived
    const uint32_t taken = coded + 8 * kWgRing;      // they were read
    const uint32_t full = taken + 8 * kWgRing;       // [2] a tile's product is complete
    const uint32_t drained = full + 16;                // [2] first block's: TMEM read out
    uint32_t* words = reinterpret_cast<uint32_t*>(bars + 5 * kWgRing + 4);
    volatile uint32_t* gave_up = words + 1;
    float* affine = reinterpret_cast<float*>(base + kWgBars + 512);

    // (the shuffle tells the compiler that a warp has one number)
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x & 1, pair = blockIdx.x >> 1;     // of the cluster of two

    if (warp == kWgMmaWarp) tmem_alloc_pair(smem_u32(words), 2 * kWgTile);
    if (threadIdx.x == 0) {
        words[1] = 0;
        for (int s = 0; s < kWgRing; ++s) {
            mbar_init(empty + 8 * s, 1);
            mbar_init(ready + 8 * s, 2 * (kWgGroupWarps + (COPY ? 1 : kWgLoaders)));
            mbar_init(copied + 8 * s, 1);
            mbar_init(coded + 8 * s, 1);
            mbar_init(taken + 8 * s, kWgGroupWarps);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(full + 8 * b, 1);
            mbar_init(drained + 8 * b, 2 * kWgWriters);
        }
        mbar_init_fence();
    }
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    after_previous();
    let_next_begin();
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, words[0], 0);

    if (warp >= kWgDecodeWarp && warp < kWgLoadWarp) {
        // ---- decode.  Eight lanes read the 128 codes of a token.  Four of them write the even
        // chunks of a line of the first panel while the other four write the odd chunks of the same
        // line of the second, so no bank is hit twice.
        const uint32_t group = (warp - kWgDecodeWarp) / kWgGroupWarps;
        const uint32_t i0 = (threadIdx.x - 32 * kWgDecodeWarp) & (32 * kWgGroupWarps - 1);
        const uint32_t token = i0 >> 3, eighth = i0 & 7;
        const bool odd = eighth >= 4;
        const uint32_t place = kWgDecoded + (odd ? kWgPanel : 0u) + token * 128;
        const uint32_t chunk = (2 * (eighth & 3) + odd) ^ (token & 7);
        uint32_t total = 0, u = 0;
        for (WgUnit w = wg_unit<CHAINS>(a, pair, 0); w.steps; w = wg_unit<CHAINS>(a, pair, ++u)) total += w.steps;
        for (uint32_t step = group; step < total; step += kWgGroups) {
            const uint32_t stage = step % kWgRing, slot = step % kWgSlots;
            bool ok = wg_wait_step(coded, step, gave_up);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            const uint8_t* from = base + kWgCodes + slot * kWgCodeBytes + token * 128 + eighth * 16;
            const uint8_t* scales = base + kWgScales + slot * kWgScaleBytes + token * 4 + (eighth >> 1);
            uint32_t w[4][4], scale[4], most = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 c = *reinterpret_cast<const uint4*>(from + i * (16 * 128));
                w[i][0] = odd ? c.z : c.x;
                w[i][1] = odd ? c.w : c.y;
                w[i][2] = odd ? c.x : c.z;
                w[i][3] = odd ? c.y : c.w;
                scale[i] = scales[i * 64];
                most = max(most, scale[i]);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(taken + 8 * stage);
            uint32_t v[4][8];
            if (most <= kAct8MaxFast) {
#pragma unroll
                for (int i = 0; i < 4; ++i) wg_decode<true>(w[i], scale[i], v[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) wg_decode<false>(w[i], scale[i], v[i]);
            }
            ok = step < kWgSlots || wg_wait_step(empty, step - kWgSlots, gave_up);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            const uint32_t line = tiles + slot * kWgOperand + place;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t at = line + i * (16 * 128);
                shared_store16(at + (chunk << 4), v[i][0], v[i][1], v[i][2], v[i][3]);
                shared_store16(at + ((chunk ^ 1) << 4), v[i][4], v[i][5], v[i][6], v[i][7]);
            }
            fence_async_proxy();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(ready + 8 * stage, 0);
        }
    } else if (warp < kWgWriters) {
        // ---- write a tile out: lane = row
        uint32_t* rows = reinterpret_cast<uint32_t*>(affine + 2 * kWgTile) + warp * (kWgRows / 4);
        uint32_t u = 0;
        WgTurns turns;
        for (WgUnit w = wg_unit<CHAINS>(a, pair, 0); w.steps; w = wg_unit<CHAINS>(a, pair, ++u)) {
            const uint64_t k0 = w.k0;
            const bool part = w.halves == 1 && w.tile >= a.whole && a.splits > 1;
            const bool last = !part && (!CHAINS || w.chain + 1 == w.chains);      // dW is written
            if (last) {
                asm volatile("bar.sync 1, %0;" ::"r"(32 * kWgWriters) : "memory");
                for (int i = threadIdx.x; i < kWgTile; i += 32 * kWgWriters) {
                    const bool in = k0 + i < a.k;
                    affine[i] = a.gamma && in ? wg_param(a.gamma, a.param_dtype, k0 + i) : 1.0f;
                    affine[kWgTile + i] =
                        a.beta && in ? wg_param(a.beta, a.param_dtype, k0 + i) : 0.0f;
                }
                asm volatile("bar.sync 1, %0;" ::"r"(32 * kWgWriters) : "memory");
            }
#pragma unroll 1
            for (uint32_t h = 0; h < w.halves; ++h) {
                const uint32_t b = turns.of(w, h);
                const uint64_t n = w.n0 + h * kWgTile + rank * kWgHalf + 32 * warp + lane;
                const float add = last && a.beta && n < a.n ? a.db[n] : 0.0f;
                bool ok = mbar_wait(full + 8 * b, turns.parity(b), gave_up);
                ok = __all_sync(0xFFFFFFFFu, ok && !*gave_up);
                tc_fence_after();
                const uint32_t from = tmem + b * kWgTile + ((uint32_t)(32 * warp) << 16);
                // four columns of all rows follow each other
                float4* sums = (part ? reinterpret_cast<float4*>(a.parts) +
                                           ((uint64_t)(w.tile - a.whole) * a.splits + w.part) * kWgTileFours
                                     : reinterpret_cast<float4*>(a.runs) +
                                           (uint64_t)(2 * pair + h) * kWgTileFours) +
                               rank * kWgHalf + 32 * warp + lane;
                if (CHAINS && !last) {
                    wg_empty(sums, from, ok, w.chain == 0);
                } else {
                    // (a loop of few instructions: in a short call they are all fetched for the first
                    // time)
                    const int end = part || k0 + kWgTile <= a.k ? kWgTile : (int)((a.k - k0 + 7) & ~7ull);
                    uint32_t next[8];
                    tmem_load8(from, next);
#pragma unroll 1
                    for (int c = 0; c < end; c += 8) {
                        float v[8];
                        float4* to = sums + c / 4 * kWgTile;
                        tmem_wait8(next);
#pragma unroll
                        for (int i = 0; i < 8; ++i)      // NaN: a wait ran out, no result
                            v[i] = ok ? __uint_as_float(next[i]) : __uint_as_float(0x7FC00000u);
                        if (CHAINS && w.chain > 0) {     // on top of the chains before
                            const float4 lo = __ldcg(to), hi = __ldcg(to + kWgTile);
                            v[0] += lo.x; v[1] += lo.y; v[2] += lo.z; v[3] += lo.w;
                            v[4] += hi.x; v[5] += hi.y; v[6] += hi.z; v[7] += hi.w;
                        }
                        if (c + 8 < end) tmem_load8(from + c + 8, next);
                        if (!CHAINS && part) {
                            to[0] = make_float4(v[0], v[1], v[2], v[3]);
                            to[kWgTile] = make_float4(v[4], v[5], v[6], v[7]);
                            continue;
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            v[i] = fmaf(v[i], affine[c + i], add * affine[kWgTile + c + i]);
                        if (!a.vector || k0 + c + 8 > a.k)
                            wg_store_rows(a, n - lane, k0 + c, v, rows);
                        else if (n < a.n)
                            wg_store8(a, n, k0 + c, v);
                    }
                }
                tc_fence_before();
                __syncwarp();
                // (a tile that was not waited for was not read: the other block may still be reading it)
                if (lane == 0 && ok) mbar_arrive_at(drained + 8 * b, 0);
            }
            turns.done(w);
        }
    } else if (warp == kWgCopyWarp) {
        // ---- copies of the dY tiles: two panels of 64 n each.  A place of their ring is free when
        // the step that used it last is done.
        if (COPY && lane == 0) {
            WgWalk<CHAINS> walk;
            const uint32_t arrived = rank ? copied : ready;
            uint32_t place = 0, step = 0, last[kWgPlaces];        // last: step + 1, 0: unused
            for (int s = 0; s < kWgPlaces; ++s) last[s] = 0;
            bool ok = true;
            for (walk.begin(a, pair); walk.more() && ok; walk.advance(a, pair, 1), ++step) {
                const uint32_t bar = arrived + 8 * (step % kWgRing);
                for (uint32_t h = 0; h < walk.unit.halves; ++h) {
                    uint32_t before = 0;
#pragma unroll
                    for (int s = 0; s < kWgPlaces; ++s)
                        if (s == (int)place) {
                            before = last[s];
                            last[s] = step + 1;
                        }
                    if (before) ok = wg_wait_step(empty, before - 1, gave_up);
                    if (!ok) break;
                    if (h == 0) mbar_expect(bar, walk.unit.halves * kWgOperand);
                    for (int p = 0; p < 2; ++p)
                        tma_load_2d(tiles + place * kWgOperand + p * kWgPanel, &map,
                                    (int)(walk.unit.n0 + h * kWgTile + rank * kWgHalf + 64 * p),
                                    (int)walk.token(), bar);
                    place = place + 1 == kWgPlaces ? 0 : place + 1;
                }
            }
            // the copies in flight land before the block may end
            const long long begin = clock64();
            for (uint32_t i = step < kWgRing ? 0 : step - kWgRing; i < step; ++i)
                while (!mbar_try(arrived + 8 * (i % kWgRing), (i / kWgRing) & 1) &&
                       clock64() - begin < 4000000000ll) {}
        }
    } else if (warp == kWgCodeWarp) {
        // ---- copies of the codes and of their scales
        if (lane == 0) {
            WgWalk<CHAINS> walk;
            uint32_t step = 0;
            for (walk.begin(a, pair); walk.more(); walk.advance(a, pair, 1), ++step) {
                const uint32_t slot = step % kWgSlots, bar = coded + 8 * (step % kWgRing);
                if (step >= kWgSlots && !wg_wait_step(taken, step - kWgSlots, gave_up)) break;
                const uint64_t column = walk.unit.k0 + rank * kWgHalf;
                mbar_expect(bar, kWgCodeBytes + kWgScaleBytes);
                tma_load_2d(tiles + kWgCodes + slot * kWgCodeBytes, &code_map, (int)column,
                            (int)walk.token(), bar);
                bulk_load(tiles + kWgScales + slot * kWgScaleBytes,
                          a.scales + (column / 128) * a.token_pitch + walk.token(), kWgScaleBytes,
                          bar);
            }
            const long long begin = clock64();
            for (uint32_t i = step < kWgRing ? 0 : step - kWgRing; i < step; ++i)
                while (!mbar_try(coded + 8 * (i % kWgRing), (i / kWgRing) & 1) &&
                       clock64() - begin < 4000000000ll) {}
        }
    } else if (warp == kWgMmaWarp) {
        if (rank == 0) {
            // ---- matrix instructions: the whole warp, of which one thread issues
            const uint32_t shape = mma_shape(kWgTile, kWgTile);
            const bool elected = elect_one();
            const uint64_t operand = mma_operand(tiles, kWgPanel);   // + bytes / 16: further on
            bool ok = true, here = false;            // here: the next step was seen to be ready
            uint32_t u = 0, place = 0, slot = 0, stage = 0, parity = 0;
            WgTurns turns;
            for (WgUnit w = wg_unit<CHAINS>(a, pair, 0); w.steps && ok; w = wg_unit<CHAINS>(a, pair, ++u)) {
                for (uint32_t h = 0; h < w.halves && ok; ++h) {
                    const uint32_t b = turns.of(w, h);
                    ok = mbar_wait(drained + 8 * b, turns.parity(b) ^ 1, gave_up);
                }
                const uint32_t to = tmem + turns.of(w, 0) * kWgTile;
                const bool twice = w.halves == 2;
                for (uint32_t s = 0; s < w.steps && ok; ++s) {
                    if (!here) ok = mbar_wait(ready + 8 * stage, parity, gave_up);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t right = operand + (kWgDecoded + slot * kWgOperand) / 16;
                    slot = slot + 1 == kWgSlots ? 0 : slot + 1;
                    const uint32_t done = empty + 8 * stage;
                    stage = stage + 1 == kWgRing ? 0 : stage + 1;
                    parity ^= stage == 0;
                    uint64_t left = operand + place * (kWgOperand / 16);
                    place = place + 1 == kWgPlaces ? 0 : place + 1;
#pragma unroll
                    for (int i = 0; i < kWgStep / 16; ++i)   // 16 tokens: two groups of lines
                        mma_pair(to, left + 128 * i, right + 128 * i, shape, s > 0 || i > 0,
                                 elected);
                    if (twice) {
                        left = operand + place * (kWgOperand / 16);
                        place = place + 1 == kWgPlaces ? 0 : place + 1;
#pragma unroll
                        for (int i = 0; i < kWgStep / 16; ++i)
                            mma_pair(to + kWgTile, left + 128 * i, right + 128 * i, shape,
                                     s > 0 || i > 0, elected);
                    }
                    mma_commit_pair(done, elected);
                    here = __all_sync(0xFFFFFFFFu, mbar_test(ready + 8 * stage, parity));
                }
                // given up: both blocks know before their writers hear that the tile is complete, for
                // what stands in TMEM is the sum of some of the steps
                if (!ok && elected) {
                    shared_store_at(smem_u32(words + 1), 0, 1);
                    shared_store_at(smem_u32(words + 1), 1, 1);
                    fence_cluster();
                }
                __syncwarp();
                for (uint32_t h = 0; h < w.halves; ++h)
                    mma_commit_pair(full + 8 * turns.of(w, h), elected);
                turns.done(w);
            }
        } else if (COPY && lane == 0) {
            // ---- the other block: pass on that its dY tiles have arrived
            WgRing ring = {0, 0};
            WgWalk<CHAINS> walk;
            for (walk.begin(a, pair); walk.more(); walk.advance(a, pair, 1)) {
                if (!mbar_wait(copied + 8 * ring.stage, ring.parity, gave_up)) break;
                mbar_arrive_at(ready + 8 * ring.stage, 0);
                ring.advance(1);
            }
        }
    } else if (!COPY && warp >= kWgLoadWarp) {
        // ---- plain loads of the dY tile, a step ahead: 16 lanes cover the 128 n of a token
        const int i0 = threadIdx.x - 32 * kWgLoadWarp;
        const uint32_t chunk = i0 & 15, token0 = i0 >> 4;          // tokens token0 + 8 j
        WgWalk<CHAINS> walk;
        walk.begin(a, pair);
        uint32_t step = 0;
        uint4 v[8];
        if (walk.more()) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] = wg_load_dy8(a, walk.token() + token0 + 8 * j,
                                   walk.unit.n0 + rank * kWgHalf + 8 * chunk);
        }
        while (walk.more()) {
            walk.advance(a, pair, 1);
            const bool free = step < kWgPlaces || wg_wait_step(empty, step - kWgPlaces, gave_up);
            if (!__all_sync(0xFFFFFFFFu, free)) break;
            const uint32_t dst = tiles + step % kWgPlaces * kWgOperand + (chunk >> 3) * kWgPanel;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t token = token0 + 8 * j;
                shared_store16(dst + token * 128 + (((chunk & 7) ^ (token & 7)) << 4), v[j].x, v[j].y,
                               v[j].z, v[j].w);
                if (walk.more())
                    v[j] = wg_load_dy8(a, walk.token() + token,
                                       walk.unit.n0 + rank * kWgHalf + 8 * chunk);
            }
            fence_async_proxy();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(ready + 8 * (step % kWgRing), 0);
            ++step;
        }
    }
    // the pair stays until both blocks are done with each other's barriers and with TMEM
    __syncwarp();
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    if (warp == kWgMmaWarp) tmem_free_pair(tmem, 2 * kWgTile);
}

// the tiles that were computed in parts: dw <- [dw +] gamma * (sum of the parts, in order) +
// beta * db; no parts: the sum over no tokens.  A block takes 32 rows x 32 columns of a tile; the
// parts hold rows side by side, dw columns, so they change places in shared memory.
__global__ void __launch_bounds__(256) wg_join_kernel(const __grid_constant__ WgArgs a) {
    __shared__ float4 sums[8][33];
    after_previous();
    const uint32_t tile = a.whole + blockIdx.x / 64, piece = blockIdx.x % 64;
    uint64_t n, k;
    wg_single(a, tile, n, k);
    n += piece / 8 * 32;
    k += piece % 8 * 32;
    if (n >= a.n || k >= a.k) return;
    {
        const uint32_t row = threadIdx.x & 31, four = threadIdx.x >> 5;
        const float4* p = reinterpret_cast<const float4*>(a.parts) +
                          (uint64_t)(tile - a.whole) * a.splits * (kWgTile / 4 * kWgTile) +
                          (piece % 8 * 8 + four) * kWgTile + piece / 8 * 32 + row;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (uint32_t z = 0; z < a.splits; ++z) {
            const float4 q = __ldcs(p + (uint64_t)z * (kWgTile / 4 * kWgTile));
            s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
        }
        sums[four][row] = s;
    }
    __syncthreads();
    if (!a.vector) {                     // a value at a time, neighbours side by side
        const uint32_t column = threadIdx.x & 31;
        if (k + column >= a.k) return;
        const float gamma = a.gamma ? wg_param(a.gamma, a.param_dtype, k + column) : 1.0f;
        const float beta = a.beta ? wg_param(a.beta, a.param_dtype, k + column) : 0.0f;
        for (uint32_t row = threadIdx.x >> 5; row < 32 && n + row < a.n; row += 8) {
            const float s = reinterpret_cast<const float*>(&sums[column >> 2][row])[column & 3];
            const float v = a.beta ? fmaf(a.db[n + row], beta, s * gamma) : s * gamma;
            const uint64_t at = (n + row) * a.lddw + k + column;
            if (a.dw_f32) {
                float* p = static_cast<float*>(a.dw) + at;
                *p = a.accumulate ? *p + v : v;
            } else {
                __nv_bfloat16* p = static_cast<__nv_bfloat16*>(a.dw) + at;
                *p = __float2bfloat16_rn(a.accumulate ? __bfloat162float(*p) + v : v);
            }
        }
        return;
    }
    if (threadIdx.x >= 128) return;
    const uint32_t row = threadIdx.x >> 2, eight = threadIdx.x & 3;
    n += row;
    k += 8 * eight;
    if (n >= a.n || k >= a.k) return;
    const float4 lo = sums[2 * eight][row], hi = sums[2 * eight + 1][row];
    float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    const float add = a.beta ? a.db[n] : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k + i < a.k) {
            if (a.gamma) v[i] *= wg_param(a.gamma, a.param_dtype, k + i);
            if (a.beta) v[i] = fmaf(add, wg_param(a.beta, a.param_dtype, k + i), v[i]);
        }
    wg_store8(a, n, k, v);
}

// ---- scale bytes by columns of 128: word [c][t] holds the four bytes of token t and of the columns
// from 128 c on; those beyond the checkpoint are a unit of 1.  A block moves 64 tokens x 32 words.
struct WgScales {
    const uint8_t* in;
    uint64_t rows, row_bytes;            // of the checkpoint
    uint32_t* out;
    uint64_t token_pitch, columns;       // of 128, even
    uint32_t across;                     // pieces of 32 columns
    uint64_t pieces;                     // of 64 tokens x 32 columns
};

// the blocks of `down` rows of the grid, this one in row `y` of them, take the pieces in turn
__device__ __forceinline__ void wg_lay_scales(const WgScales& g, int y, int down) {
    __shared__ uint32_t words[32][65];
    const bool whole = g.row_bytes % 4 == 0;                         // words of a row: one access
    for (uint64_t piece = (uint64_t)y * gridDim.x + blockIdx.x; piece < g.pieces;
         piece += (uint64_t)down * gridDim.x) {
        const uint64_t t0 = piece / g.across * 64, c0 = piece % g.across * 32;
#pragma unroll 4
        for (int i = threadIdx.x; i < 64 * 32; i += 256) {
            const uint64_t t = t0 + i / 32, c = c0 + i % 32;
            uint32_t w = 0x7F7F7F7Fu;
            if (whole) {
                if (t < g.rows && 4 * c < g.row_bytes)
                    w = __ldg(reinterpret_cast<const uint32_t*>(g.in + t * g.row_bytes + 4 * c));
            } else if (t < g.rows) {
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    if (4 * c + b < g.row_bytes)
                        w = (w & ~(0xFFu << (8 * b))) |
                            (uint32_t)__ldg(g.in + t * g.row_bytes + 4 * c + b) << (8 * b);
            }
            words[i % 32][i / 32] = w;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 64 * 32; i += 256) {
            const uint64_t t = t0 + i % 64, c = c0 + i / 64;
            if (c < g.columns) g.out[c * g.token_pitch + t] = words[i / 64][i % 64];
        }
        __syncthreads();
    }
}

// where the columns' sums go when there is one range of rows only: `fresh` gets the sum, db <- [db +] it
struct WgDb {
    float *fresh, *db;
    bool accumulate;
    __device__ __forceinline__ void store(uint64_t n, float s) const {
        if (fresh) fresh[n] = s;
        if (db) db[n] = accumulate ? db[n] + s : s;
    }
};

// ---- column sums of dY: a block adds up a range of rows, a thread eight columns, or one where the
// rows are not on 16-byte boundaries.  The blocks of the grid's first rows lay out the scales (as its
// last blocks they came after a full wave: 8192 x 4096 x 1024 took 111 instead of 107 us).
constexpr int kWgSumBlocks = 256;        // ranges at most

template <bool VECTOR>
__global__ void __launch_bounds__(256)
wg_sums_kernel(const __nv_bfloat16* __restrict__ dy, const uint64_t rows, const uint64_t n,
               const uint64_t lddy, float* __restrict__ parts, const int ranges, const WgDb last,
               const __grid_constant__ WgScales scales) {
    let_next_begin();
    const int down = gridDim.y - ranges, range = (int)blockIdx.y - down;
    if (range < 0) {
        wg_lay_scales(scales, blockIdx.y, down);
        return;
    }
    constexpr int W = VECTOR ? 8 : 1;
    __shared__ float sums[8][32 * W + 1];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const uint64_t col = ((uint64_t)blockIdx.x * 32 + lane) * W;
    const uint64_t begin = rows * range / ranges, end = rows * (range + 1) / ranges;
    float s[W];
#pragma unroll
    for (int i = 0; i < W; ++i) s[i] = 0.0f;
    if (col < n) {
        const __nv_bfloat16* p = dy + col;
        if constexpr (VECTOR) {
            for (uint64_t t = begin + group; t < end; t += 32) {     // four loads in flight
                uint4 v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    v[u] = make_uint4(0u, 0u, 0u, 0u);
                    if (t + 8 * u < end)
                        v[u] = __ldg(reinterpret_cast<const uint4*>(p + (t + 8 * u) * lddy));
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float e, f;
                        unpack2<__nv_bfloat16>(w[i], e, f);
                        s[2 * i] += e;
                        s[2 * i + 1] += f;
                    }
                }
            }
        } else {
#pragma unroll 8
            for (uint64_t t = begin + group; t < end; t += 8)
                s[0] += __bfloat162float(__ldg(p + t * lddy));
        }
    }
#pragma unroll
    for (int i = 0; i < W; ++i) sums[group][lane * W + i] = s[i];
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * W; c += 256) {
        const uint64_t at = (uint64_t)blockIdx.x * 32 * W + c;
        if (at >= n) continue;
        float v = sums[0][c];
#pragma unroll
        for (int g = 1; g < 8; ++g) v += sums[g][c];
        if (ranges == 1)
            last.store(at, v);
        else
            parts[range * n + at] = v;
    }
}

// the same for rows that are not on 16-byte boundaries, and a copy of dY whose rows are: a warp
// takes 512 columns of every eighth row
__global__ void __launch_bounds__(256)
wg_align_kernel(const __nv_bfloat16* __restrict__ dy, const uint64_t rows, const uint64_t n,
                const uint64_t lddy, __nv_bfloat16* __restrict__ copy, const uint64_t ldc,
                float* __restrict__ parts, const int ranges, const WgDb last,
                const __grid_constant__ WgScales scales) {
    let_next_begin();
    const int range = blockIdx.y;        // the scales last here, in the shadow of the longer copies
    if (range >= ranges) {
        wg_lay_scales(scales, range - ranges, gridDim.y - ranges);
        return;
    }
    __shared__ float sums[512];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t first = (uint64_t)blockIdx.x * 512;
    const uint32_t cols = (uint32_t)min(n - first, (uint64_t)1024);
    const uint64_t begin = rows * range / ranges, end = rows * (range + 1) / ranges;
    float s[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.0f;
    for (uint64_t t = begin + warp; t < end; t += 8) {
        Raw16<__nv_bfloat16> r;
        row_load<__nv_bfloat16, kSpread>(dy + t * lddy + first, lane, cols, false, r);
        uint32_t* out = reinterpret_cast<uint32_t*>(copy + t * ldc + first);
#pragma unroll
        for (int i = 0; i < 8; ++i)      // rows of the copy hold whole pairs
            if (spread_col<__nv_bfloat16>(i, lane) < cols)
                out[32 * i + lane] = r.b[0].v[i];
        float v[16];
        unpack16<__nv_bfloat16>(r, v);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] += v[i];
    }
    for (int w = 0; w < 8; ++w) {        // the warps in order
        if (warp == w) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t c = spread_col<__nv_bfloat16>(i >> 1, lane) + (i & 1);
                sums[c] = w ? sums[c] + s[i] : s[i];
            }
        }
        __syncthreads();
    }
    for (uint32_t c = threadIdx.x; c < min(cols, 512u); c += 256) {
        if (ranges == 1)
            last.store(first + c, sums[c]);
        else
            parts[range * n + first + c] = sums[c];
    }
}

// db <- [db +] the parts' sum, in the order of the parts within each of 8 interleaved groups, then of
// the groups; `fresh`, where wanted, gets the sum alone
__global__ void __launch_bounds__(256)
wg_sums_join_kernel(const float* __restrict__ parts, const int blocks, const uint64_t n,
                    const WgDb last) {
    __shared__ float sums[8][33];
    let_next_begin();
    after_previous();
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const uint64_t col = (uint64_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (col < n) {
#pragma unroll 8
        for (int b = group; b < blocks; b += 8) s += __ldcg(parts + b * n + col);
    }
    sums[group][lane] = s;
    __syncthreads();
    if (group == 0 && col < n) {
        s = sums[0][lane];
#pragma unroll
        for (int k = 1; k < 8; ++k) s += sums[k][lane];
        last.store(col, s);
    }
}

struct WgPlan {
    uint64_t tiles_n, tiles_k, rounds, tiles, whole;
    uint32_t splits;
    int sum_blocks;
    uint64_t ldc;                        // row stride of the aligned copy of dY
    uint64_t token_pitch;                // tokens of a column of laid out scales
    uint64_t steps;
    size_t runs_offset, sum_offset, fresh_offset, scale_offset, copy_offset, bytes;
};

// `doubles`: double tiles may be used
static WgPlan wg_plan(uint64_t rows, uint64_t n, uint64_t k, bool doubles) {
    WgPlan p = {};
    p.tiles_n = (n + kWgTile - 1) / kWgTile;
    p.tiles_k = (k + kWgTile - 1) / kWgTile;
    p.rounds = doubles ? p.tiles_n / 2 * p.tiles_k / kWgPairs : 0;
    p.tiles = p.tiles_n * p.tiles_k - 2 * kWgPairs * p.rounds;
    const uint64_t steps = (rows + kWgStep - 1) / kWgStep, left = p.tiles % kWgPairs;
    p.steps = steps;
    uint64_t splits = left ? kWgPairs / left : 1;
    if (splits > steps / kWgMinSteps) splits = steps / kWgMinSteps;
    p.whole = p.tiles - left;
    p.splits = splits < 1 ? 1 : (uint32_t)splits;
    // eight blocks for every SM in the column sums
    // (unaligned widths are copied as well: four rows a warp at least)
    const uint64_t across = n % 8 ? (n + 511) / 512 : (n + 255) / 256, least = n % 8 && rows <= 1024 ? 32 : 64;
    uint64_t blocks = across ? 8 * 148 / across : 1;
    if (blocks > (rows + least - 1) / least) blocks = (rows + least - 1) / least;
    if (n % 8 == 0 && rows <= 256) blocks = 1;       // no kernel to join ranges
    if (blocks > kWgSumBlocks) blocks = kWgSumBlocks;
    p.sum_blocks = (int)(blocks < 1 ? 1 : blocks);
    p.runs_offset = p.splits > 1 ? left * p.splits * kWgTileFours * 16 : 0;
    // (the type of dW, and with it the chains, are the call's)
    const uint32_t least_chain = kWgChainF32 < kWgChainBf16 ? kWgChainF32 : kWgChainBf16;
    const bool runs = steps > least_chain && (p.tiles_n * p.tiles_k >= kWgPairs || p.splits == 1);
    p.sum_offset = p.runs_offset + (runs ? 2 * kWgPairs * (size_t)kWgTileFours * 16 : 0);
    p.fresh_offset = p.sum_offset + round_up16(p.sum_blocks * n * 4);
    p.scale_offset = p.fresh_offset + round_up16(n * 4);
    p.token_pitch = steps * kWgStep;
    p.copy_offset = p.scale_offset + 2 * p.tiles_k * p.token_pitch * 4;
    p.ldc = (n + 7) / 8 * 8;
    // a copy is made where the width itself keeps rows off the boundaries
    p.bytes = p.copy_offset + (n % 8 ? rows * p.ldc * 2 : 0);
    return p;
}

}  // namespace natcomp

using namespace natcomp;

extern "C" {

size_t nc_act8_weight_grad_workspace_bytes(size_t rows, size_t n, size_t k) {
    if (n > ((size_t)1 << 31) || k > ((size_t)1 << 31) || rows > ((size_t)1 << 31)) return 0;
    return wg_plan(rows, n, k, true).bytes;
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
    if (rows >= ((size_t)1 << 31) || n >= ((size_t)1 << 31) || k >= ((size_t)1 << 31) ||
        !act8_fits(rows, k) || ((n + 255) / 256) * ((k + 255) / 256) >= ((size_t)1 << 24))
        return NC_ERR_TOO_LARGE;
    const int wbytes = dw_dtype == NC_DTYPE_F32 ? 4 : 2;
    if (!element_aligned(dy, 2) || !element_aligned(gamma, pbytes) ||
        !element_aligned(beta, pbytes) || !element_aligned(dw, wbytes) || !aligned4(db) ||
        !aligned16(codes) || !aligned16(scales) || !aligned16(workspace))
        return NC_ERR_ALIGN;
    const bool aligned = row_access(dy, lddy, 2, rows) != kRowElement;
    const bool copied = !aligned && n % 8 != 0;          // through a copy that is
    const bool f32 = dw_dtype == NC_DTYPE_F32;
    const uint32_t chain = f32 ? kWgChainF32 : kWgChainBf16;
    const WgPlan p = wg_plan(rows, n, k, rows && (aligned || copied));
    if (rows && workspace_bytes < p.bytes) return NC_ERR_WORKSPACE;

    char* ws = static_cast<char*>(workspace);
    float* fresh = reinterpret_cast<float*>(ws + p.fresh_offset);
    const bool with_beta = beta && k && rows;
    float* sums = reinterpret_cast<float*>(ws + p.sum_offset);
    WgScales g = {};
    g.in = scales;
    g.rows = rows;
    g.row_bytes = act8_pitch(k) / 32;
    g.out = reinterpret_cast<uint32_t*>(ws + p.scale_offset);
    g.token_pitch = k ? p.token_pitch : 0;
    g.columns = 2 * p.tiles_k;
    g.across = (uint32_t)((g.columns + 31) / 32);
    g.pieces = g.token_pitch / 64 * g.across;
    const int ranges = rows && (db || with_beta || copied) ? p.sum_blocks : 0;
    const WgDb last = {with_beta ? fresh : nullptr, db, accumulate != 0};
    if (rows) {
        const __nv_bfloat16* in = static_cast<const __nv_bfloat16*>(dy);
        const bool vector = aligned && n % 8 == 0;
        const uint64_t across = (n + (copied ? 511 : vector ? 255 : 31)) /
                                (copied ? 512 : vector ? 256 : 32);
        const uint64_t lay = (g.pieces + across - 1) / across;       // rows of blocks for them
        const unsigned down = ranges + (unsigned)(lay < 4096 ? lay : 4096);
        const dim3 grid((unsigned)across, down);
        if (copied) {
            __nv_bfloat16* copy = reinterpret_cast<__nv_bfloat16*>(ws + p.copy_offset);
            wg_align_kernel<<<grid, 256, 0, stream>>>(in, rows, n, lddy, copy, p.ldc, sums, ranges,
                                                      last, g);
            dy = copy;
            lddy = p.ldc;
        } else if (down) {
            auto kernel = vector ? wg_sums_kernel<true> : wg_sums_kernel<false>;
            kernel<<<grid, 256, 0, stream>>>(in, rows, n, lddy, sums, ranges, last, g);
        }
    }
    if ((db || with_beta) && ranges != 1)
        launch_overlapping(wg_sums_join_kernel, dim3((unsigned)((n + 31) / 32)), dim3(256), 0,
                           stream, (const float*)sums, rows ? p.sum_blocks : 0, (uint64_t)n, last);
    if (k == 0) return launch_status();

    WgArgs a = {};
    a.dy = static_cast<const __nv_bfloat16*>(dy);
    a.rows = rows; a.n = n; a.lddy = lddy; a.k = k; a.scales = g.out;
    a.token_pitch = p.token_pitch;
    a.gamma = rows ? gamma : nullptr;        // no tokens: 0, not 0 * gamma
    a.beta = with_beta ? beta : nullptr;
    a.param_dtype = param_dtype; a.dw = dw; a.dw_f32 = f32; a.lddw = lddw;
    a.db = fresh; a.accumulate = accumulate;
    a.vector = row_access(dw, lddw, wbytes, n) != kRowElement;
    a.tiles_n = (uint32_t)p.tiles_n;
    a.tiles_k = (uint32_t)p.tiles_k;
    a.rounds = (uint32_t)p.rounds;
    a.tiles = (uint32_t)p.tiles;
    a.whole = rows ? (uint32_t)p.whole : 0;
    a.splits = rows ? p.splits : 0;
    a.parts = reinterpret_cast<float*>(ws);
    a.chain = chain;
    a.runs = reinterpret_cast<float*>(ws + p.runs_offset);
    if (rows) {
        const bool copy = aligned || copied;             // by tensor copies
        CUtensorMap map = {}, code_map = {};
        if (copy && !make_tensor_map(&map, dy, true, rows, n, rows > 1 ? lddy : p.ldc, 64, kWgStep))
            return NC_ERR_CUDA;
        if (!make_tensor_map(&code_map, codes, false, rows, act8_pitch(k), act8_pitch(k), 128,
                             kWgStep))
            return NC_ERR_CUDA;
        const bool chains = p.steps > chain;
        auto kernel = copy ? (chains ? wg_product_kernel<true, true> : wg_product_kernel<true, false>)
                           : (chains ? wg_product_kernel<false, true> : wg_product_kernel<false, false>);
        static bool allowed[4][64];
        if (!allow_dynamic_smem((const void*)kernel, kWgSmem, allowed[2 * chains + copy]))
            return NC_ERR_CUDA;
        const uint64_t pairs = p.whole || p.rounds ? kWgPairs : (p.tiles - p.whole) * p.splits;
        launch_overlapping(kernel, dim3((unsigned)(2 * pairs)),
                           dim3(32 * (kWgLoadWarp + (copy ? 0 : kWgLoaders))), kWgSmem, stream, a,
                           map, code_map);
    }
    if (a.splits != 1 && a.whole < a.tiles)
        launch_overlapping(wg_join_kernel, dim3((a.tiles - a.whole) * 64), dim3(256), 0, stream, a);
    return launch_status();
}

}  // extern "C"
