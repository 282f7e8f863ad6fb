// Softmax cross entropy of a linear output layer over a large vocabulary, and its gradient, for
// sm_100a.  With z[t][v] = scale * x[t] . table[v]:
//
//   lse[t]  = log sum_v exp z[t][v],   loss[t] = lse[t] - z[t][target[t]]
//   dz[t][v] = p (dloss[t] + dlse[t]) - [v = target[t]] dloss[t],   p = exp(z[t][v] - lse[t])
//   dx = scale * dz table,   dtable = scale * dz^T x
//
// The logits never reach memory.  Forward, the epilogue of the product keeps a running maximum and a
// sum of exponentials for every row and 256 columns, and the logit of the target; a second kernel
// joins them.  Backward, a piece of the vocabulary at a time: the logits again, whose epilogue writes
// dz in 16 bits (a few hundred megabytes at most), then the two products that read it.
//
// Rows without a target (target < 0) are left out of all products: the rows that count are gathered
// first, side by side.  So a NaN in a row that does not count reaches nothing, a batch that is half
// padding costs half, and rows of any alignment become ones that tensor copies take.
//
// dz is divided by about the largest coefficient of any row before it is rounded to 16 bits and the products
// are multiplied by it again.  That puts the entries of the targets, 1 - p times their coefficient,
// just under 1, where 16 bits are finest relative to the value, and keeps binary16 (with another
// 2^14) clear of its subnormal numbers: a p of 2^-28 is still a normal one.
//
// What bounds it: the tensor cores and the power cap.  2 operations forward and 6 backward for every row,
// column and vocabulary entry.  8192 x 4096 x 65536 backward: 10.6 ms back to back, 1.24 PFLOP/s.
#include "product.cuh"

namespace natcomp {

constexpr float kLog2E = 1.4426950408889634f;
constexpr uint32_t kCeNone = 0xFFFFFFFFu;            // a target beyond the vocabulary: the row is NaN
// Of a piece of dz: 256 MB.  8192 x 2048 x 65536 backward: 5.41 ms; pieces of 64 MB 5.71, of 1 GB 5.37.
constexpr uint64_t kCeDzValues = 1ull << 27;
constexpr uint64_t kCeLeastPiece = 2048;             // vocabulary entries of a piece
// Of a piece of the table that the forward pass copies: 64 MB, 8192 entries of width 4096.  (64 x 101 x 71851
// took 92 us in pieces of 8192 entries, whatever the width.)
constexpr uint64_t kCeCopyValues = 1ull << 25;
constexpr int kCeGatherBlocks = 592;

// the rows that count, side by side
struct CeRows {
    uint32_t* count;                     // [0] of them, [1] the largest coefficient's bits
    uint32_t* origin;                    // where each came from
    uint32_t* target;                    // kCeNone: beyond the vocabulary
    float *lse, *dloss, *both;           // both: dloss + dlse
    float* hit;                          // logit of the target (forward)
    uint2* most;                         // of each gathering block, bits of the largest dloss and of the
                                         // largest of the others
    void* x;                             // pitch values a row
    uint64_t pitch;
};

struct CeGather {
    const unsigned short* x;
    uint64_t rows, width, ldx;
    bool aligned;                        // rows of x are on 16-byte boundaries
    const void* targets;
    int target_bytes;
    uint64_t vocabulary;
    const float *lse, *dloss, *dlse;     // of the backward pass
    float *loss_out, *lse_out;           // of the forward pass
    void* dx;                            // of the backward pass, or nullptr
    uint64_t lddx;
    uint32_t per_block;
    int blocks;                          // that gather; those behind them copy a piece of the table:
    const unsigned short* piece;
    uint64_t piece_rows, ldt;
    unsigned short* piece_to;
    CeRows to;
};

__device__ __forceinline__ int64_t ce_target(const CeGather& g, uint64_t i) {
    return g.target_bytes == 8 ? __ldg(static_cast<const long long*>(g.targets) + i)
                               : (int64_t)__ldg(static_cast<const int*>(g.targets) + i);
}

// bits of a coefficient's magnitude, ordered as the magnitudes are; 0 for one that is not finite: it makes
// its own row what it is, whatever the rows are divided by
__device__ __forceinline__ uint32_t ce_magnitude(float v) {
    const uint32_t bits = __float_as_uint(v) & 0x7FFFFFFFu;
    return bits < 0x7F800000u ? bits : 0u;
}

// eight values of a row at any element to a row on 16-byte boundaries; what lies behind the row becomes 0
__device__ __forceinline__ void ce_copy8(const unsigned short* from, uint64_t width, uint64_t c, uint4* to) {
    uint32_t v[4] = {0u, 0u, 0u, 0u};
    if (c + 8 <= width) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i >> 1] |= (uint32_t)__ldg(from + c + i) << (16 * (i & 1));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < width) v[i >> 1] |= (uint32_t)__ldg(from + c + i) << (16 * (i & 1));
    }
    *to = make_uint4(v[0], v[1], v[2], v[3]);
}

// the rows of a matrix by `threads` threads, this one number `thread`
__device__ __forceinline__ void ce_copy_rows(const unsigned short* from, uint64_t rows, uint64_t width,
                                             uint64_t ld, unsigned short* to, uint64_t pitch,
                                             uint64_t thread, uint64_t threads) {
    const uint64_t eights = (width + 7) / 8, all = rows * eights;
#pragma unroll 2
    for (uint64_t i = thread; i < all; i += threads) {
        // (a division in 64 bits would take longer than the copy)
        const uint64_t r = i >> 32 ? i / eights : (uint64_t)((uint32_t)i / (uint32_t)eights);
        const uint64_t c = (i - r * eights) * 8;
        ce_copy8(from + r * ld, width, c, reinterpret_cast<uint4*>(to + r * pitch + c));
    }
}

// Every block counts the rows before its own, and all of them, for itself: a few reads of the targets
// out of L2 instead of a pass that finds the places first.
__global__ void __launch_bounds__(256) ce_gather_kernel(const __grid_constant__ CeGather g) {
    __shared__ uint32_t sums[8][2];
    __shared__ uint32_t place[256];
    __shared__ uint2 most[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    after_previous();
    let_next_begin();
    if ((int)blockIdx.x >= g.blocks) {
        ce_copy_rows(g.piece, g.piece_rows, g.width, g.ldt, g.piece_to, g.to.pitch,
                     (uint64_t)(blockIdx.x - g.blocks) * 256 + threadIdx.x,
                     (uint64_t)(gridDim.x - g.blocks) * 256);
        return;
    }
    const uint64_t first = (uint64_t)blockIdx.x * g.per_block;
    const uint64_t last = min(first + g.per_block, g.rows);
    uint32_t before = 0, all = 0;
    uint2 top = make_uint2(0u, 0u);      // of dloss, of the others
    // (every block begins at another place, or all of them ask the same parts of L2 at a time)
    for (uint64_t i = threadIdx.x; i < g.rows; i += 8 * 256) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint64_t to = i + j * 256, at = to + first < g.rows ? to + first : to + first - g.rows;
            const uint32_t counts = to < g.rows && ce_target(g, at) >= 0;
            all += counts;
            before += at < first ? counts : 0;
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        all += __shfl_xor_sync(0xFFFFFFFFu, all, d);
        before += __shfl_xor_sync(0xFFFFFFFFu, before, d);
    }
    if (lane == 0) {
        sums[warp][0] = before;
        sums[warp][1] = all;
    }
    __syncthreads();
    before = all = 0;
    for (int w = 0; w < 8; ++w) {
        before += sums[w][0];
        all += sums[w][1];
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) g.to.count[0] = all;
    const uint32_t eights = (uint32_t)(g.to.pitch / 8);
    for (uint64_t chunk = first; chunk < last; chunk += 256) {
        // places of up to 256 rows
        const uint64_t i = chunk + threadIdx.x;
        const int64_t t = i < last ? ce_target(g, i) : -1;
        uint32_t at = t >= 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t other = __shfl_sync(0xFFFFFFFFu, at, lane >= d ? lane - d : lane);
            if (lane >= d) at += other;
        }
        __syncthreads();
        if (lane == 31) sums[warp][0] = at;
        __syncthreads();
        uint32_t base = before, here = 0;
        for (int w = 0; w < 8; ++w) {
            if (w < warp) base += sums[w][0];
            here += sums[w][0];
        }
        at += base - 1;
        place[threadIdx.x] = t >= 0 ? at : kCeNone;
        before += here;
        if (t >= 0) {
            g.to.origin[at] = (uint32_t)i;
            g.to.target[at] = (uint64_t)t < g.vocabulary ? (uint32_t)t : kCeNone;
            if (g.dloss) {
                const float dl = g.dloss[i], ds = g.dlse ? g.dlse[i] : 0.0f, both = dl + ds;
                g.to.lse[at] = g.lse[i];
                g.to.dloss[at] = dl;
                g.to.both[at] = both;
                top.x = max(top.x, ce_magnitude(dl));
                top.y = max(top.y, max(ce_magnitude(ds), ce_magnitude(both)));
            } else {
                g.to.hit[at] = __uint_as_float(0x7FC00000u);
            }
        } else if (i < last && g.loss_out) {
            g.loss_out[i] = 0.0f;
            g.lse_out[i] = 0.0f;
        }
        __syncthreads();
        // a warp copies a row, or clears the gradient of one that does not count
        for (uint64_t r = chunk + warp; r < min(chunk + 256, last); r += 8) {
            const uint32_t to = place[r - chunk];
            if (to == kCeNone) {
                if (g.dx) {
                    unsigned short* p = static_cast<unsigned short*>(g.dx) + r * g.lddx;
                    for (uint64_t c = lane; c < g.width; c += 32) p[c] = 0;
                }
                continue;
            }
            const unsigned short* from = g.x + r * g.ldx;
            uint4* out = reinterpret_cast<uint4*>(static_cast<unsigned short*>(g.to.x) +
                                                  (uint64_t)to * g.to.pitch);
            if (g.aligned && g.width % 8 == 0) {
#pragma unroll 4
                for (uint32_t c = lane; c < g.width / 8; c += 32)
                    out[c] = __ldg(reinterpret_cast<const uint4*>(from) + c);
            } else {
                for (uint64_t c = lane; c < (g.width + 7) / 8; c += 32)
                    ce_copy8(from, g.width, 8 * c, out + c);
            }
        }
    }
    // the last step of the products over the rows reads up to 63 rows more: 0, not what stood there
    const uint64_t end = ((uint64_t)all + 63) & ~(uint64_t)63;
    for (uint64_t r = all + blockIdx.x; r < end; r += g.blocks) {
        uint4* out = reinterpret_cast<uint4*>(static_cast<unsigned short*>(g.to.x) + r * g.to.pitch);
        for (uint32_t c = threadIdx.x; c < eights; c += 256) out[c] = make_uint4(0u, 0u, 0u, 0u);
    }
    if (g.dloss) {
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            top.x = max(top.x, __shfl_xor_sync(0xFFFFFFFFu, top.x, d));
            top.y = max(top.y, __shfl_xor_sync(0xFFFFFFFFu, top.y, d));
        }
        if (lane == 0) most[warp] = top;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < 8; ++w) {
                top.x = max(top.x, most[w].x);
                top.y = max(top.y, most[w].y);
            }
            g.to.most[blockIdx.x] = top;
        }
    }
}

// rows of a table whose rows no tensor copy can take, to ones of `pitch` values
__global__ void __launch_bounds__(256)
ce_copy_kernel(const unsigned short* __restrict__ from, const uint64_t rows, const uint64_t width,
               const uint64_t ld, unsigned short* __restrict__ to, const uint64_t pitch) {
    after_previous();
    let_next_begin();
    ce_copy_rows(from, rows, width, ld, to, pitch, (uint64_t)blockIdx.x * 256 + threadIdx.x,
                 (uint64_t)gridDim.x * 256);
}

// rows of zeros, a warp each
template <typename T>
__global__ void __launch_bounds__(256)
ce_clear_kernel(T* __restrict__ p, const uint64_t rows, const uint64_t width, const uint64_t ld) {
    after_previous();
    let_next_begin();
    for (uint64_t r = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += (uint64_t)gridDim.x * 8)
        for (uint64_t c = threadIdx.x & 31; c < width; c += 32) p[r * ld + c] = from_f32<T>(0.0f);
}

// ---- forward ---------------------------------------------------------------------------------

// The tensor cores cut off what an accumulator of 24 bits cannot hold, always towards 0, so all logits of
// a long sum are too small: by 5e-7 of their size after 1024 products, 9e-7 after 2048, twice that after
// 4096, and the loss with them.  CHAINS: longer sums are read out every 1024 products and added up in
// registers (128 of a thread's), rounded to nearest, while the next ones are computed; the error stays
// that of 1024.  6144 x 2048 x 65536: 1161 us, 1123 as one sum.  (Figures of bfloat16.  A product of binary16
// has more bits than the accumulator has below the sum's first, so something of each is cut off too: 7e-6 after
// 1024 products of one sign.)
constexpr uint32_t kCeChain = 16;                    // steps
// The backward pass makes its logits as the forward pass does, chain by chain, so that they are the same bits
// as those in lse.  As one sum of 4096 products they were 1.8e-6 of their size smaller, and the entry of a
// target with 1 - p = 1e-4 and a logit of 25 was off by a half.  8192 x 4096 x 65536: 10.61 ms, 10.44 as one sum.
constexpr uint32_t kCeDzChain = 16;
// dtable, a sum over the rows: chains of 8192 rows, 4e-6 of it, and in binary16 of 2048, 1.3e-5.  (One sum of
// 131072 rows was 6e-5 and, in binary16, 5e-4 too small; 16384 x 1024 x 65536 into binary32 5.87 ms, 5.82 as one
// sum, 16384 x 1024 x 32768 binary16 3.26 and 3.09.)  dx is rounded to 16 bits and stays one sum a piece.
constexpr uint32_t kCeLongChain = 128;
constexpr uint32_t kCeLongChainF16 = 32;

template <bool CHAINS> struct CeLogits : ProductOnce {
    // left, right: gathered rows, piece of the table
    CeRows rows;
    uint32_t columns, tiles_n;           // of the piece
    uint32_t split;                      // pieces that every tile comes in
    uint32_t first;                      // its first vocabulary entry
    uint32_t steps, parts_of;            // parts_of: chains of a sum
    float unit;                          // scale * log2 e
    float scale;
    float2* parts;                       // [piece of the vocabulary][pitch of the rows]: maximum, sum
    uint64_t part_pitch;
    uint32_t count;

    static constexpr int kColumns = CHAINS ? 16 : 32;        // at a time
    struct State {
        float sums[CHAINS ? kProductHalf : 1];
    };
    __device__ __forceinline__ uint32_t begin(uint32_t, bool) {
        count = __ldcg(rows.count);
        return (count + kProductTile - 1) / kProductTile * tiles_n * split;
    }
    __device__ __forceinline__ uint32_t chains() const { return CHAINS ? parts_of : 1; }
    __device__ __forceinline__ void ahead(const ProductUnit&, const ProductRead&, State&) const {}
    __device__ __forceinline__ ProductUnit unit_of(uint32_t u, uint32_t chain) const {
        ProductUnit w = {};
        product_tile(u / split, (count + kProductTile - 1) / kProductTile, tiles_n, w.m, w.n);
        w.width = kProductTile / (int)split;
        w.n += (int)(u % split) * w.width;
        w.steps = (int)steps;
        if (CHAINS) product_chain(w, chain, parts_of);
        w.part = chain;
        return w;
    }
    __device__ __forceinline__ void store(const ProductUnit& w, const ProductRead& r, State& s) const {
        if constexpr (CHAINS) {
            if (w.part + 1 < parts_of) {
                product_keep(r, w.part == 0, s.sums);
                return;
            }
        }
        const uint32_t row = (uint32_t)(w.m + r.row), col = (uint32_t)(w.n + r.column);
        const uint32_t target = row < count ? __ldcg(rows.target + row) : kCeNone;
        const uint32_t at = target - first - col;            // of the target among these columns
        const bool near = target != kCeNone && target >= first + col && at < (uint32_t)r.columns;
        float top = __uint_as_float(0xFF800000u), sum = 0.0f;
#pragma unroll (CHAINS ? kProductHalf / kColumns : 1)
        for (int c = 0; c < kProductHalf; c += kColumns) {
            if (c >= r.columns || col + c >= columns) break;
            uint32_t v[kColumns];
            r.load(c, v);
            if (CHAINS) {
#pragma unroll
                for (int i = 0; i < kColumns; ++i)
                    v[i] = __float_as_uint(s.sums[c + i] + __uint_as_float(v[i]));
            }
            take(v, col + c, row, near && at >= (uint32_t)c && at < (uint32_t)c + kColumns, at - c, top,
                 sum);
        }
        // the two halves of the columns
        const float lowest = __uint_as_float(0xFF800000u);
        float2* other = reinterpret_cast<float2*>(r.exchange) + r.lane;
        if (r.half) *other = make_float2(top, sum);
        product_pair_barrier(r);
        if (!r.half) {
            const float2 o = *other;
            const float next = fmaxf(top, o.x), from = next == lowest ? 0.0f : next;
            sum = sum * exp2_approx((top - from) * unit) + o.y * exp2_approx((o.x - from) * unit);
            if (row < count)
                parts[(uint64_t)((first + (uint32_t)w.n) / (uint32_t)w.width) * part_pitch + row] =
                    make_float2(next, sum);
        }
        product_pair_barrier(r);
    }
    // neighbouring logits of a row, from vocabulary entry first + col on; here: the target is the `at`-th of them
    __device__ __forceinline__ void take(uint32_t (&v)[kColumns], uint32_t col, uint32_t row, bool here,
                                         uint32_t at, float& top, float& sum) const {
        const float lowest = __uint_as_float(0xFF800000u);
        if (col + kColumns > columns) {
#pragma unroll
            for (int i = 0; i < kColumns; ++i)
                if (col + i >= columns) v[i] = 0xFF800000u;
        }
        if (here) {
            uint32_t hit = 0;
#pragma unroll
            for (int i = 0; i < kColumns; ++i)
                if (at == (uint32_t)i) hit = v[i];
            rows.hit[row] = scale * __uint_as_float(hit);
        }
        float m[4] = {top, lowest, lowest, lowest};
#pragma unroll
        for (int i = 0; i < kColumns; ++i) m[i & 3] = fmaxf(m[i & 3], __uint_as_float(v[i]));
        const float next = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
        const float from = next == lowest ? 0.0f : next;     // nothing but -inf so far
        const float shift = -from * unit;
        float s[4] = {sum * exp2_approx((top - from) * unit), 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kColumns; ++i)
            s[i & 3] += exp2_approx(fmaf(__uint_as_float(v[i]), unit, shift));
        sum = (s[0] + s[1]) + (s[2] + s[3]);
        top = next;
    }
};

// a row's parts -> its logsumexp and loss.  Eight warps share the parts of 32 rows.
__global__ void __launch_bounds__(256)
ce_join_kernel(const CeRows rows, const float2* __restrict__ parts, const uint64_t pitch,
               const uint32_t tiles, const float scale, float* __restrict__ loss,
               float* __restrict__ lse) {
    __shared__ float2 got[8][32];
    after_previous();
    let_next_begin();
    const uint32_t count = __ldcg(rows.count);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float unit = scale * kLog2E, lowest = __uint_as_float(0xFF800000u);
    for (uint64_t first = (uint64_t)blockIdx.x * 32; first < count; first += (uint64_t)gridDim.x * 32) {
        const uint64_t row = first + lane;
        float top = lowest, sum = 0.0f;
        if (row < count) {
#pragma unroll 4
            for (uint32_t t = warp; t < tiles; t += 8) {
                const float2 p = __ldcg(parts + t * pitch + row);
                const float next = fmaxf(top, p.x), from = next == lowest ? 0.0f : next;
                sum = sum * exp2_approx((top - from) * unit) + p.y * exp2_approx((p.x - from) * unit);
                top = next;
            }
        }
        __syncthreads();
        got[warp][lane] = make_float2(top, sum);
        __syncthreads();
        if (warp == 0 && row < count) {
            float high = top;
            for (int w = 1; w < 8; ++w) high = fmaxf(high, got[w][lane].x);
            const float from = high == lowest ? 0.0f : high;
            float s = 0.0f;
            for (int w = 0; w < 8; ++w)
                s += got[w][lane].y * exp2_approx((got[w][lane].x - from) * unit);
            const float l = fmaf(from, scale, logf(s));
            const uint32_t to = __ldcg(rows.origin + row);
            lse[to] = l;
            loss[to] = l - __ldcg(rows.hit + row);
        }
    }
}

// ---- backward --------------------------------------------------------------------------------

// What the rows are divided by: the largest dloss, unless the other coefficients reach more than twice as
// far.  (With the same dloss for all rows the entries of targets of small p become -1, which is exact, also
// where a small dlse makes p's coefficient a little larger.)
__device__ __forceinline__ uint32_t ce_chosen(uint32_t hot, uint32_t others) {
    return __uint_as_float(others) > 2.0f * __uint_as_float(hot) ? others : hot;
}

// the largest coefficient of any row, never so small that its inverse is not finite
__device__ __forceinline__ float ce_largest(uint32_t bits) {
    return fmaxf(__uint_as_float(bits), 1e-33f);
}
// dz / largest in binary16 is at most twice this much
template <typename T> __device__ __forceinline__ constexpr float ce_headroom() {
    return sizeof(T) && std::is_same<T, __half>::value ? 16384.0f : 1.0f;
}

template <typename T, bool CHAINS> struct CeDzJob : ProductOnce {
    // left, right: gathered rows, piece of the table
    CeRows rows;
    uint32_t tiles_n, first, steps, parts_of;            // parts_of: chains of a sum
    float unit;
    T* dz;                               // [row][pitch]
    uint64_t pitch;
    int blocks;                          // of the gathering kernel
    uint32_t count;
    ProductSplit split;
    float inverse;

    __device__ __forceinline__ uint32_t begin(uint32_t, bool reads_out) {
        count = __ldcg(rows.count);
        if (reads_out) {
            uint32_t hot = 0, others = 0;
            for (int i = threadIdx.x & 31; i < blocks; i += 32) {
                const uint2 m = __ldcg(rows.most + i);
                hot = max(hot, m.x);
                others = max(others, m.y);
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) {
                hot = max(hot, __shfl_xor_sync(0xFFFFFFFFu, hot, d));
                others = max(others, __shfl_xor_sync(0xFFFFFFFFu, others, d));
            }
            const uint32_t top = ce_chosen(hot, others);
            if (blockIdx.x == 0 && threadIdx.x == 0) rows.count[1] = top;
            inverse = ce_headroom<T>() / ce_largest(top);
        }
        const uint32_t tiles = (count + kProductTile - 1) / kProductTile * tiles_n;
        split = product_split(tiles);
        return split.units(tiles);
    }
    struct State {
        float sums[CHAINS ? kProductHalf : 1];           // of the chains before
    };
    __device__ __forceinline__ uint32_t chains() const { return CHAINS ? parts_of : 1; }
    __device__ __forceinline__ void ahead(const ProductUnit&, const ProductRead&, State&) const {}
    __device__ __forceinline__ ProductUnit unit_of(uint32_t u, uint32_t chain) const {
        ProductUnit w = {};
        int column;
        const uint32_t t = split.tile(u, column, w.width);
        product_tile(t, (count + kProductTile - 1) / kProductTile, tiles_n, w.m, w.n);
        w.n += column;
        w.steps = (int)steps;
        if (CHAINS) product_chain(w, chain, parts_of);
        w.part = chain;
        return w;
    }
    __device__ __forceinline__ void store(const ProductUnit& w, const ProductRead& r, State& s) const {
        if constexpr (CHAINS) {
            if (w.part + 1 < parts_of) {
                product_keep(r, w.part == 0, s.sums);
                return;
            }
        }
        const uint32_t row = (uint32_t)(w.m + r.row), col = (uint32_t)(w.n + r.column);
        const bool counts = row < count;
        const uint32_t target = counts ? __ldcg(rows.target + row) : 0u;
        const float shift = counts ? -__ldcg(rows.lse + row) * kLog2E : 0.0f;
        const float hot = counts ? __ldcg(rows.dloss + row) * inverse : 0.0f;
        float all = counts ? __ldcg(rows.both + row) * inverse : 0.0f;
        if (target == kCeNone) all = __uint_as_float(0x7FC00000u);
        const uint32_t keep = counts ? 0xFFFFFFFFu : 0u;
        const uint32_t at = target - first - col;            // of the target among these columns
        const bool near = counts && target != kCeNone && target >= first + col &&
                          at < (uint32_t)r.columns;
        T* to = dz + (uint64_t)row * pitch + col;
        const auto put = [&](auto& v, int c) {
            constexpr int N = CHAINS ? 16 : 32;
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] = __float_as_uint(all * exp2_approx(fmaf(__uint_as_float(v[i]), unit, shift)));
            if (near && at >= (uint32_t)c && at < (uint32_t)c + N) {
#pragma unroll
                for (int i = 0; i < N; ++i)      // (a sum, not a store: v stays in registers)
                    v[i] = __float_as_uint(__uint_as_float(v[i]) - (at - c == (uint32_t)i ? hot : 0.0f));
            }
            Bytes32 o[N / 16];
#pragma unroll
            for (int i = 0; i < N / 2; ++i)
                o[i >> 3].v[i & 7] =
                    pack2<T>(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])) & keep;
#pragma unroll
            for (int i = 0; i < N / 16; ++i) st_wide(to + c + 16 * i, o[i]);
        };
        if constexpr (CHAINS) {
#pragma unroll
            for (int c = 0; c < kProductHalf; c += 16) {
                if (c >= r.columns) break;
                uint32_t v[16];
                r.load(c, v);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    v[i] = __float_as_uint(s.sums[c + i] + __uint_as_float(v[i]));
                put(v, c);
            }
        } else {
#pragma unroll 1
            for (int c = 0; c < r.columns; c += 32) {
                uint32_t v[32];
                r.load(c, v);
                put(v, c);
            }
        }
    }
};
template <typename T> using CeDz = CeDzJob<T, false>;

// what the products over dz are multiplied by
__device__ __forceinline__ float ce_factor(uint32_t largest, float scale, bool bf16) {
    return ce_largest(largest) * (bf16 ? scale : scale * (1.0f / 16384.0f));
}

struct CeDx : ProductOnce {
    // left, right: dz, piece of the table
    CeRows rows;
    uint32_t width, tiles_n, steps, splits;
    float scale;
    bool begins, ends;                   // the first, the last piece of the vocabulary
    float* sums;                         // [split][rows' pitch][pitch]
    uint64_t pitch, split_distance;
    void* dx;
    uint64_t lddx;
    ProductTarget target;
    uint32_t count;
    ProductSplit split;
    float factor;

    __device__ __forceinline__ uint32_t begin(uint32_t, bool reads_out) {
        count = __ldcg(rows.count);
        factor = reads_out ? ce_factor(__ldcg(rows.count + 1), scale, bf16) : 0.0f;
        const uint32_t tiles = (count + kProductTile - 1) / kProductTile * tiles_n * splits;
        split = product_split(tiles);
        return split.units(tiles);
    }
    typedef ProductNothing State;
    __device__ __forceinline__ uint32_t chains() const { return 1; }
    __device__ __forceinline__ void ahead(const ProductUnit&, const ProductRead&, State&) const {}
    __device__ __forceinline__ ProductUnit unit_of(uint32_t u, uint32_t) const {
        ProductUnit w = {};
        int column;
        const uint32_t t = split.tile(u, column, w.width);
        w.part = t % splits;
        product_tile(t / splits, (count + kProductTile - 1) / kProductTile, tiles_n, w.m, w.n);
        w.n += column;
        const uint32_t from = (uint32_t)((uint64_t)steps * w.part / splits);
        w.k = (int)from * kProductStep;
        w.steps = (int)((uint32_t)((uint64_t)steps * (w.part + 1) / splits) - from);
        return w;
    }
    __device__ __forceinline__ void store(const ProductUnit& w, const ProductRead& r, State&) const {
        const uint32_t row = (uint32_t)(w.m + r.row), col = (uint32_t)(w.n + r.column);
        float* sum = sums + w.part * split_distance + (uint64_t)row * pitch + col;
        ProductRows to = {};
        to.anywhere = true;              // rows go back to where they were gathered from
        if (ends && splits == 1 && row < count)
            to.own = static_cast<char*>(dx) + 2 * ((uint64_t)__ldcg(rows.origin + row) * lddx + col);
#pragma unroll 1
        for (int c = 0; c < r.columns && col + c < width; c += 32) {
            uint32_t v[32];
            r.load(c, v);
            if (!begins) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const Bytes32 old = ld_wide(sum + c + 8 * i);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        v[8 * i + j] = __float_as_uint(__uint_as_float(v[8 * i + j]) +
                                                       __uint_as_float(old.v[j]));
                }
            }
            if (!ends || splits > 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    Bytes32 o;
#pragma unroll
                    for (int j = 0; j < 8; ++j) o.v[j] = v[8 * i + j];
                    st_wide(sum + c + 8 * i, o);
                }
            } else {
                float o[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = factor * __uint_as_float(v[i]);
                product_store(target, to, c, (int)(width - col) - c, o, r);
            }
        }
    }
};

// dx of a few rows whose sums were split: the parts in order
template <typename T>
__global__ void __launch_bounds__(256)
ce_join_dx_kernel(const CeRows rows, const float* __restrict__ sums, const uint64_t pitch,
                  const uint64_t distance, const uint32_t splits, const float scale, const bool bf16,
                  T* __restrict__ dx, const uint64_t lddx, const uint32_t width) {
    after_previous();
    let_next_begin();
    __shared__ uint32_t word[2];         // (one thread asks for the block)
    if (threadIdx.x < 2) word[threadIdx.x] = __ldcg(rows.count + threadIdx.x);
    __syncthreads();
    const uint32_t count = word[0];
    const float factor = ce_factor(word[1], scale, bf16);
    const uint32_t col = blockIdx.x * 256 + threadIdx.x;
    if (col >= width) return;
    for (uint32_t row = blockIdx.y; row < count; row += gridDim.y) {
        const float* p = sums + (uint64_t)row * pitch + col;
        float s = 0.0f;
#pragma unroll 8
        for (uint32_t i = 0; i < splits; ++i) s += __ldcg(p + i * distance);
        dx[(uint64_t)__ldcg(rows.origin + row) * lddx + col] = from_f32<T>(factor * s);
    }
}

template <bool CHAINS> struct CeDtableJob : ProductOnce {
    // left, right: dz, gathered rows
    CeRows rows;
    uint32_t entries, width, tiles_m, tiles_n, chain_steps;
    float scale;
    void* dtable;                        // of the piece
    uint64_t ldt;
    ProductTarget target;
    uint32_t count, parts_of;            // parts_of: chains of a sum
    ProductSplit split;
    float factor;

    __device__ __forceinline__ uint32_t begin(uint32_t, bool reads_out) {
        count = __ldcg(rows.count);
        parts_of = max(1u, ((count + kProductStep - 1) / kProductStep + chain_steps - 1) / chain_steps);
        factor = reads_out ? ce_factor(__ldcg(rows.count + 1), scale, bf16) : 0.0f;
        split = product_split(tiles_m * tiles_n);
        return split.units(tiles_m * tiles_n);
    }
    struct State {
        float sums[CHAINS ? kProductHalf : 1];           // of the chains before
    };
    __device__ __forceinline__ uint32_t chains() const { return CHAINS ? parts_of : 1; }
    __device__ __forceinline__ void ahead(const ProductUnit&, const ProductRead&, State&) const {}
    __device__ __forceinline__ ProductUnit unit_of(uint32_t u, uint32_t chain) const {
        ProductUnit w = {};
        int column;
        product_tile(split.tile(u, column, w.width), tiles_m, tiles_n, w.m, w.n);
        w.n += column;
        w.steps = (int)((count + kProductStep - 1) / kProductStep);
        if (CHAINS) product_chain(w, chain, parts_of);
        w.part = chain;
        return w;
    }
    __device__ __forceinline__ void store(const ProductUnit& w, const ProductRead& r, State& s) const {
        if constexpr (CHAINS) {
            if (w.part + 1 < parts_of) {
                product_keep(r, w.part == 0, s.sums);
                return;
            }
        }
        const uint32_t row = (uint32_t)(w.m + r.row), col = (uint32_t)(w.n + r.column);
        const ProductRows to =
            product_rows(dtable, target.dtype, ldt, row - r.lane, entries, col, r.lane);
#pragma unroll 1
        for (int c = 0; c < r.columns && col + c < width; c += 32) {
            uint32_t v[32];
            r.load(c, v);
            if constexpr (CHAINS) {              // (few rows may count)
                if (parts_of > 1) product_join(s.sums, c, v);
            }
            float o[32];
#pragma unroll
            for (int i = 0; i < 32; ++i)         // (no row counts: 0, whatever the factor)
                o[i] = count ? factor * __uint_as_float(v[i]) : 0.0f;
            product_store(target, to, c, (int)(width - col) - c, o, r);
        }
    }
};
typedef CeDtableJob<false> CeDtable;

// ---- plans -----------------------------------------------------------------------------------

struct CePlan {
    uint64_t rows_pitch, pitch, vocabulary_pitch, piece;
    uint32_t splits;                     // of dx
    uint32_t pieces;                     // that every tile of the forward pass comes in
    int blocks;
    uint32_t per_block;
    size_t count, origin, target, lse, dloss, both, hit, most, x, copy, parts, dz, sums, bytes;
};

static size_t ce_place(size_t& at, size_t bytes) {
    const size_t here = at;
    at = (at + bytes + 255) & ~(size_t)255;
    return here;
}

static bool ce_fits(size_t rows, size_t width, size_t vocabulary) {
    const size_t most = ((size_t)1 << 31) - 256;
    return rows <= most && width <= most && vocabulary <= most &&
           ((rows + 255) / 256) * ((vocabulary + 255) / 256) < ((size_t)1 << 31) &&
           ((rows + 255) / 256) * ((width + 255) / 256) < ((size_t)1 << 24) &&
           ((vocabulary + 255) / 256) * ((width + 255) / 256) < ((size_t)1 << 31);
}

static CePlan ce_plan(uint64_t rows, uint64_t width, uint64_t vocabulary, bool backward) {
    CePlan p = {};
    p.rows_pitch = (rows + 255) / 256 * 256;
    p.pitch = (width + 15) / 16 * 16;
    p.vocabulary_pitch = (vocabulary + 255) / 256 * 256;
    p.piece = kCeCopyValues / (p.pitch ? p.pitch : 1) / 256 * 256;
    if (p.piece < kCeLeastPiece) p.piece = kCeLeastPiece;
    if (backward) {
        p.piece = p.rows_pitch ? kCeDzValues / p.rows_pitch / 256 * 256 : 0;
        if (p.piece < kCeLeastPiece) p.piece = kCeLeastPiece;
    }
    if (p.piece > p.vocabulary_pitch) p.piece = p.vocabulary_pitch;
    // (a row for every warp at least: with fewer the counting outweighs the copies)
    p.per_block = (uint32_t)((rows + kCeGatherBlocks - 1) / kCeGatherBlocks);
    if (p.per_block < 8) p.per_block = 8;
    p.blocks = (int)((rows + p.per_block - 1) / p.per_block);
    // Fewer tiles of dx than pairs: the sum over the vocabulary is split, eight steps a part at least, and a
    // kernel adds up the parts.  515 x 1001 x 8193: 67 us instead of 93, 200 x 512 x 32768: 56 instead of 194.
    const uint64_t tiles = p.rows_pitch / kProductTile * ((width + kProductTile - 1) / kProductTile);
    const uint64_t steps = (p.piece + kProductStep - 1) / kProductStep;
    uint64_t splits = tiles ? kProductPairs / tiles : 1;
    if (splits > steps / 8) splits = steps / 8;
    p.splits = splits < 1 || p.piece < p.vocabulary_pitch ? 1 : (uint32_t)splits;
    size_t at = 0;
    p.count = ce_place(at, 256);
    p.origin = ce_place(at, 4 * p.rows_pitch);
    p.target = ce_place(at, 4 * p.rows_pitch);
    p.x = ce_place(at, 2 * p.rows_pitch * p.pitch);
    p.copy = ce_place(at, 2 * p.piece * p.pitch);
    if (backward) {
        p.lse = ce_place(at, 4 * p.rows_pitch);
        p.dloss = ce_place(at, 4 * p.rows_pitch);
        p.both = ce_place(at, 4 * p.rows_pitch);
        p.most = ce_place(at, 8 * (size_t)(p.blocks + 1));
        p.dz = ce_place(at, 2 * p.rows_pitch * p.piece);
        if (p.splits > 1 || p.piece < p.vocabulary_pitch)
            p.sums = ce_place(at, 4 * p.splits * p.rows_pitch * ((width + 31) / 32 * 32));
    } else {
        p.hit = ce_place(at, 4 * p.rows_pitch);
        // (a few tiles in pieces: the rule is that of product_split, but for all of them)
        const uint64_t all = p.rows_pitch / 256 * (p.vocabulary_pitch / 256);
        p.pieces = all < kProductPairs ? product_split((uint32_t)all).parts : 1;
        p.parts = ce_place(at, 8 * p.rows_pitch * (p.vocabulary_pitch / 256 * p.pieces));
    }
    p.bytes = at;
    return p;
}

static CeRows ce_rows(const CePlan& p, char* ws) {
    CeRows r = {};
    r.count = reinterpret_cast<uint32_t*>(ws + p.count);
    r.origin = reinterpret_cast<uint32_t*>(ws + p.origin);
    r.target = reinterpret_cast<uint32_t*>(ws + p.target);
    r.lse = reinterpret_cast<float*>(ws + p.lse);
    r.dloss = reinterpret_cast<float*>(ws + p.dloss);
    r.both = reinterpret_cast<float*>(ws + p.both);
    r.hit = reinterpret_cast<float*>(ws + p.hit);
    r.most = reinterpret_cast<uint2*>(ws + p.most);
    r.x = ws + p.x;
    r.pitch = p.pitch;
    return r;
}

// The piece of the table from entry `first` on as tensor copies may read it.  It is copied where they may
// not: the first one beside the gathering of the rows (515 x 1001 x 8193 backward: 66 us instead of 73; 62 with eight values a thread).
struct CeTable {
    const unsigned short* p;
    uint64_t vocabulary, width, ld, pitch;
    bool copied;
    unsigned short* copy;
    cudaStream_t stream;
    unsigned blocks(uint64_t rows) const {
        const uint64_t n = (rows * ((width + 7) / 8) + 255) / 256;
        return (unsigned)(n < 1184 ? n : 1184);
    }
    const void* piece(uint64_t first, uint64_t count, uint64_t& stride) const {
        if (!copied) {
            stride = vocabulary > 1 ? ld : pitch;
            return p + first * ld;
        }
        if (first)
            launch_overlapping(ce_copy_kernel, dim3(blocks(count)), dim3(256), 0, stream, p + first * ld,
                               count, width, ld, copy, pitch);
        stride = pitch;
        return copy;
    }
};

template <typename T>
static nc_status ce_backward(const CePlan& p, const CeRows& rows, const CeTable& table, bool bf16,
                             float scale, char* ws, T* dx, uint64_t lddx, void* dtable,
                             int dtable_dtype, uint64_t lddt, bool accumulate, uint64_t most_rows,
                             cudaStream_t stream) {
    const uint64_t width = table.width, vocabulary = table.vocabulary;
    const uint64_t sums_pitch = (width + 31) / 32 * 32, tiles_n = (width + 255) / 256;
    const uint64_t tiles_t = p.rows_pitch / 256;
    T* dz = reinterpret_cast<T*>(ws + p.dz);
    const uint32_t chain = bf16 ? kCeLongChain : kCeLongChainF16;
    for (uint64_t first = 0; first < vocabulary; first += p.piece) {
        const uint64_t count = vocabulary - first < p.piece ? vocabulary - first : p.piece;
        const uint64_t dz_pitch = (count + 255) / 256 * 256;
        uint64_t stride = 0;
        const void* piece = table.piece(first, count, stride);
        CUtensorMap x_map, table_map, dz_map;
        if (!make_box_map(&x_map, rows.x, bf16, 1, p.rows_pitch, width, p.pitch, 0) ||
            !make_box_map(&table_map, piece, bf16, 1, count, width, stride, 0) ||
            !make_box_map(&dz_map, dz, bf16, 1, p.rows_pitch, count, dz_pitch, 0))
            return NC_ERR_CUDA;
        const auto launch_dz = [&](auto a) {
            a.left = x_map; a.right = table_map; a.bf16 = bf16; a.rows = rows;
            a.tiles_n = (uint32_t)(dz_pitch / 256); a.first = (uint32_t)first;
            a.steps = (uint32_t)((width + kProductStep - 1) / kProductStep);
            a.parts_of = (a.steps + kCeDzChain - 1) / kCeDzChain;
            a.unit = scale * kLog2E; a.dz = dz; a.pitch = dz_pitch; a.blocks = p.blocks;
            return product_launch(a, 4 * tiles_t * a.tiles_n, stream);
        };
        nc_status st = width > (uint64_t)kCeDzChain * kProductStep ? launch_dz(CeDzJob<T, true>{})
                                                                   : launch_dz(CeDz<T>{});
        if (st != NC_OK) return st;
        const auto launch_dtable = [&](auto c) {
            c.left = dz_map; c.right = x_map; c.left_side.lines = c.right_side.lines = true;
            c.bf16 = bf16; c.rows = rows; c.entries = (uint32_t)count; c.width = (uint32_t)width;
            c.tiles_m = (uint32_t)(dz_pitch / 256); c.tiles_n = (uint32_t)tiles_n; c.scale = scale;
            c.chain_steps = chain;
            const int bytes = act8_type_bytes(dtable_dtype);
            c.dtable = static_cast<char*>(dtable) + first * lddt * bytes; c.ldt = lddt;
            c.target.dtype = dtable_dtype; c.target.add = accumulate;
            c.target.access = row_access(dtable, lddt, bytes, vocabulary);
            return product_launch(c, 4 * (uint64_t)c.tiles_m * tiles_n, stream);
        };
        if (dx) {
            CeDx b = {};
            b.left = dz_map; b.right = table_map; b.right_side.lines = true; b.bf16 = bf16;
            b.rows = rows; b.width = (uint32_t)width; b.tiles_n = (uint32_t)tiles_n;
            b.steps = (uint32_t)((count + kProductStep - 1) / kProductStep); b.splits = p.splits;
            b.scale = scale; b.begins = first == 0; b.ends = first + count == vocabulary;
            b.sums = reinterpret_cast<float*>(ws + p.sums); b.pitch = sums_pitch;
            b.split_distance = p.rows_pitch * sums_pitch; b.dx = dx; b.lddx = lddx;
            b.target.dtype = bf16 ? NC_DTYPE_BF16 : NC_DTYPE_F16;
            b.target.access = row_access(dx, lddx, 2, most_rows);
            st = product_launch(b, 4 * tiles_t * tiles_n * p.splits, stream);
            if (st != NC_OK) return st;
        }
        if (dtable) {
            st = most_rows > (uint64_t)chain * kProductStep ? launch_dtable(CeDtableJob<true>{})
                                                            : launch_dtable(CeDtable{});
            if (st != NC_OK) return st;
        }
    }
    if (dx && p.splits > 1)
        launch_overlapping(ce_join_dx_kernel<T>,
                           dim3((unsigned)((width + 255) / 256),
                                (unsigned)(most_rows < 1024 ? most_rows : 1024)),
                           dim3(256), 0, stream, rows, reinterpret_cast<const float*>(ws + p.sums),
                           sums_pitch, p.rows_pitch * sums_pitch, p.splits, scale, bf16, dx, lddx,
                           (uint32_t)width);
    return launch_status();
}

// what both calls ask of their arguments
static nc_status ce_check(const void* x, int dtype, size_t rows, size_t width, size_t ldx,
                          const void* table, size_t vocabulary, size_t ldt, const void* targets,
                          int target_bytes, float scale) {
    if (dtype != NC_DTYPE_BF16 && dtype != NC_DTYPE_F16) return NC_ERR_UNSUPPORTED;
    if (target_bytes != 4 && target_bytes != 8) return NC_ERR_UNSUPPORTED;
    if (!(scale > 0.0f) || !(scale * kLog2E <= 3e38f)) return NC_ERR_INVALID;
    if (width == 0 || vocabulary == 0) return NC_ERR_INVALID;
    if (!table || ldt < width) return NC_ERR_INVALID;
    if (rows && (!x || !targets || ldx < width)) return NC_ERR_INVALID;
    if (!ce_fits(rows, width, vocabulary)) return NC_ERR_TOO_LARGE;
    if (!element_aligned(x, 2) || !element_aligned(table, 2) || !element_aligned(targets, target_bytes))
        return NC_ERR_ALIGN;
    return NC_OK;
}

static void ce_gather(CeGather& g, const CePlan& p, const CeTable& t, uint64_t piece) {
    g.per_block = p.per_block;
    g.blocks = p.blocks;
    unsigned more = 0;
    if (t.copied) {
        g.piece = t.p; g.ldt = t.ld; g.piece_to = t.copy;
        g.piece_rows = piece < t.vocabulary ? piece : t.vocabulary;
        more = t.blocks(g.piece_rows);
    }
    launch_overlapping(ce_gather_kernel, dim3((unsigned)p.blocks + more), dim3(256), 0, t.stream, g);
}

}  // namespace natcomp

using namespace natcomp;

extern "C" {

size_t nc_linear_cross_entropy_forward_workspace_bytes(size_t rows, size_t width, size_t vocabulary) {
    return ce_fits(rows, width, vocabulary) ? ce_plan(rows, width, vocabulary, false).bytes : 0;
}

size_t nc_linear_cross_entropy_backward_workspace_bytes(size_t rows, size_t width, size_t vocabulary) {
    return ce_fits(rows, width, vocabulary) ? ce_plan(rows, width, vocabulary, true).bytes : 0;
}

nc_status nc_linear_cross_entropy_forward(const void* x, int dtype, size_t rows, size_t width,
                                          size_t ldx, const void* table, size_t vocabulary, size_t ldt,
                                          const void* targets, int target_bytes, float scale,
                                          float* loss, float* lse, void* workspace,
                                          size_t workspace_bytes, cudaStream_t stream) {
    const nc_status bad = ce_check(x, dtype, rows, width, ldx, table, vocabulary, ldt, targets,
                                   target_bytes, scale);
    if (bad != NC_OK) return bad;
    if (rows == 0) return NC_OK;
    if (!loss || !lse || !workspace) return NC_ERR_INVALID;
    if (!aligned4(loss) || !aligned4(lse) || !aligned32(workspace)) return NC_ERR_ALIGN;
    const CePlan p = ce_plan(rows, width, vocabulary, false);
    if (workspace_bytes < p.bytes) return NC_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    const bool bf16 = dtype == NC_DTYPE_BF16;
    const CeRows to = ce_rows(p, ws);
    CeGather g = {};
    g.x = static_cast<const unsigned short*>(x); g.rows = rows; g.width = width; g.ldx = ldx;
    g.aligned = row_access(x, ldx, 2, rows) != kRowElement;
    g.targets = targets; g.target_bytes = target_bytes; g.vocabulary = vocabulary;
    g.loss_out = loss; g.lse_out = lse; g.to = to;
    const bool copied = row_access(table, ldt, 2, vocabulary) == kRowElement;
    const CeTable t = {static_cast<const unsigned short*>(table), vocabulary, width, ldt, p.pitch,
                       copied, reinterpret_cast<unsigned short*>(ws + p.copy), stream};
    ce_gather(g, p, t, p.piece);
    const uint64_t step = copied ? p.piece : vocabulary;
    for (uint64_t first = 0; first < vocabulary; first += step) {
        const uint64_t count = vocabulary - first < step ? vocabulary - first : step;
        uint64_t stride = 0;
        const void* piece = t.piece(first, count, stride);
        const uint32_t steps = (uint32_t)((width + kProductStep - 1) / kProductStep);
        CUtensorMap x_map, table_map;
        if (!make_box_map(&x_map, to.x, bf16, 1, p.rows_pitch, width, p.pitch, 0) ||
            !make_box_map(&table_map, piece, bf16, 1, count, width, stride, 0))
            return NC_ERR_CUDA;
        const auto launch = [&](auto a) {
            a.left = x_map; a.right = table_map; a.bf16 = bf16; a.rows = to;
            a.columns = (uint32_t)count; a.tiles_n = (uint32_t)((count + 255) / 256);
            a.first = (uint32_t)first; a.steps = steps; a.parts_of = (steps + kCeChain - 1) / kCeChain;
            a.unit = scale * kLog2E; a.scale = scale;
            a.parts = reinterpret_cast<float2*>(ws + p.parts); a.part_pitch = p.rows_pitch;
            a.split = p.pieces;
            return product_launch(a, p.rows_pitch / 256 * a.tiles_n * a.split, stream);
        };
        const nc_status st = steps > kCeChain ? launch(CeLogits<true>{}) : launch(CeLogits<false>{});
        if (st != NC_OK) return st;
    }
    const uint64_t blocks = (rows + 31) / 32;
    launch_overlapping(ce_join_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0,
                       stream, to, reinterpret_cast<const float2*>(ws + p.parts), p.rows_pitch,
                       (uint32_t)((vocabulary + 256 / p.pieces - 1) / (256 / p.pieces)), scale, loss, lse);
    return launch_status();
}

nc_status nc_linear_cross_entropy_backward(const void* x, int dtype, size_t rows, size_t width,
                                           size_t ldx, const void* table, size_t vocabulary,
                                           size_t ldt, const void* targets, int target_bytes,
                                           float scale, const float* lse, const float* dloss,
                                           const float* dlse, void* dx, size_t lddx, void* dtable,
                                           int dtable_dtype, size_t lddt, int accumulate,
                                           void* workspace, size_t workspace_bytes,
                                           cudaStream_t stream) {
    const nc_status bad = ce_check(x, dtype, rows, width, ldx, table, vocabulary, ldt, targets,
                                   target_bytes, scale);
    if (bad != NC_OK) return bad;
    if (dtable && dtable_dtype != NC_DTYPE_F32 && dtable_dtype != dtype) return NC_ERR_UNSUPPORTED;
    if ((dx && lddx < width) || (dtable && lddt < width)) return NC_ERR_INVALID;
    if (!workspace || (rows && (!lse || !dloss))) return NC_ERR_INVALID;
    if (!aligned4(lse) || !aligned4(dloss) || !aligned4(dlse) || !aligned32(workspace) ||
        !element_aligned(dx, 2) ||
        (dtable && !element_aligned(dtable, act8_type_bytes(dtable_dtype))))
        return NC_ERR_ALIGN;
    const CePlan p = ce_plan(rows, width, vocabulary, true);
    if (workspace_bytes < p.bytes) return NC_ERR_WORKSPACE;
    if (!dx && !dtable) return NC_OK;
    char* ws = static_cast<char*>(workspace);
    const bool bf16 = dtype == NC_DTYPE_BF16;
    const CeRows to = ce_rows(p, ws);
    if (rows == 0) {
        if (dtable && !accumulate) {
            const unsigned blocks = (unsigned)(vocabulary < 8 * 1184 ? (vocabulary + 7) / 8 : 1184);
            if (dtable_dtype == NC_DTYPE_F32)
                launch_overlapping(ce_clear_kernel<float>, dim3(blocks), dim3(256), 0, stream,
                                   static_cast<float*>(dtable), vocabulary, width, lddt);
            else                         // (zeros of either 16-bit type are the same)
                launch_overlapping(ce_clear_kernel<__half>, dim3(blocks), dim3(256), 0, stream,
                                   static_cast<__half*>(dtable), vocabulary, width, lddt);
        }
        return launch_status();
    }
    CeGather g = {};
    g.x = static_cast<const unsigned short*>(x); g.rows = rows; g.width = width; g.ldx = ldx;
    g.aligned = row_access(x, ldx, 2, rows) != kRowElement;
    g.targets = targets; g.target_bytes = target_bytes; g.vocabulary = vocabulary;
    g.lse = lse; g.dloss = dloss; g.dlse = dlse; g.dx = dx; g.lddx = lddx; g.to = to;
    const bool copied = row_access(table, ldt, 2, vocabulary) == kRowElement;
    const CeTable t = {static_cast<const unsigned short*>(table), vocabulary, width, ldt, p.pitch,
                       copied, reinterpret_cast<unsigned short*>(ws + p.copy), stream};
    ce_gather(g, p, t, p.piece);
    if (bf16)
        return ce_backward(p, to, t, bf16, scale, ws, static_cast<__nv_bfloat16*>(dx), lddx, dtable,
                           dtable_dtype, lddt, accumulate != 0, rows, stream);
    return ce_backward(p, to, t, bf16, scale, ws, static_cast<__half*>(dx), lddx, dtable,
                       dtable_dtype, lddt, accumulate != 0, rows, stream);
}

}  // extern "C"
