// Embedding of tokens and its gradient, for sm_100a:
//
//   out[t] = scale * table[token[t]],     dtable[v] = scale * sum of dy[t] over the t of token v
//
// Forward, a warp moves up to 1024 columns of a row.  What bounds it: HBM.
//
// Backward, the tokens are sorted with their places, so that equal ones are neighbours in the order
// of their places, and each row of the gradient is one sum in that order: no atomics, the same bits
// from run to run.  Three kernels:
//   - one cluster of up to eight blocks sorts (radix sort from the low digit, two digits up to a
//     vocabulary of a million), while all other blocks clear the rows of the gradient that no token
//     of the batch names: each scans the tokens for those of its own rows.  So the sort, which a few
//     blocks do, costs nothing where the gradient is large, and every row is written once;
//   - segments of the sorted tokens are added up, a thread eight columns; runs of equal tokens that end
//     inside their segment are finished there, the others leave binary32 sums behind;
//   - those are joined in order.
// What bounds it: HBM, by the gradient that is written and the rows that are read.
#include "act8_common.cuh"
#include "tensor_core.cuh"

namespace natcomp {

constexpr int kEmbedSlab = 1024;         // columns of a warp, forward
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortEach = 8;             // items of a thread in a chunk
constexpr int kSortChunk = kSortThreads * kSortEach;
constexpr int kSortMaxBits = 10;         // of a digit
constexpr int kSortMaxBlocks = 8;        // of the cluster
constexpr int kClearBytes = 16384;       // of shared memory for the rows' flags
constexpr int kSumThreads = 128;
constexpr int kSumColumns = 8 * kSumThreads;
constexpr int kMaxSegment = 32;          // sorted tokens of a block

struct EmbedTokens {
    const void* p;
    int bytes;                           // 4 or 8
    uint64_t count, vocabulary;
    __device__ __forceinline__ int64_t at(uint64_t i) const {
        return bytes == 8 ? __ldg(static_cast<const long long*>(p) + i)
                          : (int64_t)__ldg(static_cast<const int*>(p) + i);
    }
    // the vocabulary's size for a token that is not in it
    __device__ __forceinline__ uint32_t key(uint64_t i) const {
        const int64_t t = at(i);
        return t < 0 || (uint64_t)t >= vocabulary ? (uint32_t)vocabulary : (uint32_t)t;
    }
};

// eight values of a row: neighbours from c on, or, spread, every 32nd from c on
template <typename T>
__device__ __forceinline__ void embed_load8(const T* row, uint64_t c, uint64_t cols, bool vector,
                                            float (&v)[8]) {
    if (vector && c + 8 <= cols) {
        uint32_t w[2 * sizeof(T)];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const uint4 q = __ldg(reinterpret_cast<const uint4*>(row + c) + i);
            w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
        }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) unpack2<T>(w[i], v[2 * i], v[2 * i + 1]);
        }
    } else {
        const int step = vector ? 1 : 32;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i * step < cols ? to_f32<T>(row[c + i * step]) : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void embed_store8(T* row, uint64_t c, uint64_t cols, bool vector, bool add,
                                             float (&v)[8]) {
    if (vector && c + 8 <= cols) {
        uint4* p = reinterpret_cast<uint4*>(row + c);
        if (add) {
            float old[8];
            embed_load8<T>(row, c, cols, true, old);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += old[i];
        }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                p[i] = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                                  __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
        } else {
            *p = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]),
                            pack2<T>(v[6], v[7]));
        }
    } else {
        const int step = vector ? 1 : 32;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i * step < cols) {
                T* p = row + c + i * step;
                *p = from_f32<T>(add ? to_f32<T>(*p) + v[i] : v[i]);
            }
    }
}

// ---- forward ---------------------------------------------------------------------------------

template <typename T, typename O>
__global__ void __launch_bounds__(256)
embed_forward_kernel(const __grid_constant__ EmbedTokens tokens, const T* __restrict__ table,
                     const uint64_t cols, const uint64_t ldt, const float scale, O* __restrict__ out,
                     const uint64_t ldo, const uint32_t slabs, const bool vector) {
    after_previous();
    let_next_begin();
    const int lane = threadIdx.x & 31;
    const uint64_t unit = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const uint64_t t = unit / slabs, base = (unit - t * slabs) * kEmbedSlab;
    if (t >= tokens.count) return;
    const int64_t token = tokens.at(t);
    const bool in = token >= 0 && (uint64_t)token < tokens.vocabulary;
    const float fill = token < 0 ? 0.0f : __uint_as_float(0x7FC00000u);
    const T* row = table + (in ? (uint64_t)token * ldt : 0);
    O* to = out + t * ldo;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t c = base + 256 * i + (vector ? 8 * lane : lane);
        if (in) {
            embed_load8<T>(row, c, cols, vector, v[i]);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[i][k] *= scale;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[i][k] = fill;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        embed_store8<O>(to, base + 256 * i + (vector ? 8 * lane : lane), cols, vector, false, v[i]);
}

// ---- backward: sorted tokens, and the rows without any ------------------------------------------

struct EmbedSort {
    EmbedTokens tokens;
    int blocks;                          // of the cluster that sorts
    int passes, bits;                    // digits, and bits of one
    uint32_t *keys[2], *places[2];       // the sorted ones end up in [0]
    uint32_t* counts;                    // [block][digits]
    uint32_t* valid;                     // [block]: tokens of its part that are in the vocabulary
    char* dtable;                        // rows without a token are cleared, nullptr: not
    uint64_t row_bytes, row_distance;
    bool vector;
};

// Clears rows that no token names.  A block takes every gridDim-th range of rows whose flags fit.
__device__ __forceinline__ void embed_clear(const EmbedSort& s, uint32_t* flags, uint32_t block,
                                            uint32_t blocks) {
    const uint64_t v = s.tokens.vocabulary;
    uint64_t range = (v + blocks - 1) / blocks;
    if (range > 8 * kClearBytes) range = 8 * kClearBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (uint64_t first = block * range; first < v; first += blocks * range) {
        const uint64_t rows = min(range, v - first);
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < (rows + 31) / 32; i += kSortThreads) flags[i] = 0;
        __syncthreads();
#pragma unroll 8
        for (uint64_t i = threadIdx.x; i < s.tokens.count; i += kSortThreads) {
            const uint64_t k = (uint64_t)s.tokens.key(i) - first;
            if (k < rows) atomicOr(flags + (k >> 5), 1u << (k & 31));
        }
        __syncthreads();
        for (uint64_t r = warp; r < rows; r += kSortWarps) {
            if (flags[r >> 5] >> (r & 31) & 1) continue;
            char* p = s.dtable + (first + r) * s.row_distance;
            if (s.vector) {
                const uint64_t n = s.row_bytes / 16;
#pragma unroll 4
                for (uint64_t i = lane; i < n; i += 32)
                    reinterpret_cast<uint4*>(p)[i] = make_uint4(0u, 0u, 0u, 0u);
                for (uint64_t i = 8 * n + lane; i < s.row_bytes / 2; i += 32)
                    reinterpret_cast<unsigned short*>(p)[i] = 0;
            } else {
                for (uint64_t i = lane; i < s.row_bytes / 2; i += 32)
                    reinterpret_cast<unsigned short*>(p)[i] = 0;
            }
        }
    }
}

__global__ void __launch_bounds__(kSortThreads, 1) embed_sort_kernel(const __grid_constant__ EmbedSort s) {
    // of every warp, how many of its items have a digit; then where they go
    extern __shared__ uint16_t ranks[];
    __shared__ uint32_t base[1 << kSortMaxBits];
    __shared__ uint32_t sums[kSortWarps];
    after_previous();
    let_next_begin();
    if ((int)blockIdx.x >= s.blocks) {
        embed_clear(s, reinterpret_cast<uint32_t*>(ranks), blockIdx.x - s.blocks,
                    gridDim.x - s.blocks);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t digits = 1u << s.bits, below = (1u << lane) - 1;
    const uint64_t n = s.tokens.count;
    const uint64_t first = n * blockIdx.x / s.blocks, last = n * (blockIdx.x + 1) / s.blocks;
    uint32_t valid = 0;
    for (int pass = 0; pass < s.passes; ++pass) {
        // from buffer (passes - pass) & 1 to the other one
        const uint32_t* keys = s.keys[(s.passes - pass) & 1];
        const uint32_t* places = s.places[(s.passes - pass) & 1];
        uint32_t* keys_to = s.keys[(s.passes - pass - 1) & 1];
        uint32_t* places_to = s.places[(s.passes - pass - 1) & 1];
        const int shift = pass * s.bits;
        for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) base[d] = 0;
        __syncthreads();
        for (uint64_t i = first + threadIdx.x; i < last; i += kSortThreads) {
            const uint32_t key = pass ? __ldcg(keys + i) : s.tokens.key(i);
            if (pass == 0) valid += key < s.tokens.vocabulary;
            atomicAdd(base + (key >> shift & (digits - 1)), 1u);
        }
        __syncthreads();
        for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads)
            s.counts[blockIdx.x * digits + d] = base[d];
        cluster_sync();
        // a thread a digit: the items of lower digits, and of this one in the blocks before
        uint32_t before = 0, all = 0;
        if (threadIdx.x < digits)
            for (int b = 0; b < s.blocks; ++b) {
                const uint32_t c = __ldcg(s.counts + b * digits + threadIdx.x);
                before += b < (int)blockIdx.x ? c : 0;
                all += c;
            }
        uint32_t up = all;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t other = __shfl_sync(0xFFFFFFFFu, up, lane >= d ? lane - d : lane);
            if (lane >= d) up += other;
        }
        if (lane == 31) sums[warp] = up;
        __syncthreads();
        for (int w = 0; w < warp; ++w) before += sums[w];
        __syncthreads();
        if (threadIdx.x < digits) base[threadIdx.x] = before + up - all;
        for (uint64_t chunk = first; chunk < last; chunk += kSortChunk) {
            // a warp's items are 256 neighbours, 32 at a time
            for (uint32_t i = threadIdx.x; i < kSortWarps * digits / 2; i += kSortThreads)
                reinterpret_cast<uint32_t*>(ranks)[i] = 0;
            __syncthreads();
            uint32_t key[kSortEach], place[kSortEach], rank[kSortEach];
#pragma unroll
            for (int k = 0; k < kSortEach; ++k) {
                const uint64_t i = chunk + (warp * kSortEach + k) * 32 + lane;
                key[k] = i >= last ? 0xFFFFFFFFu : pass ? __ldcg(keys + i) : s.tokens.key(i);
                place[k] = i >= last ? 0 : pass ? __ldcg(places + i) : (uint32_t)i;
            }
            uint16_t* mine = ranks + warp * digits;
#pragma unroll
            for (int k = 0; k < kSortEach; ++k) {
                const uint64_t i = chunk + (warp * kSortEach + k) * 32 + lane;
                const uint32_t d = key[k] >> shift & (digits - 1);
                const uint32_t same = __match_any_sync(0xFFFFFFFFu, i >= last ? digits : d);
                const uint32_t old = i >= last ? 0 : mine[d];
                rank[k] = old + __popc(same & below);
                __syncwarp();
                if (i < last && (same & below) == 0) mine[d] = (uint16_t)(old + __popc(same));
                __syncwarp();
            }
            __syncthreads();
            if (threadIdx.x < digits) {
                uint32_t sum = 0;
                for (int w = 0; w < kSortWarps; ++w) {
                    const uint32_t c = ranks[w * digits + threadIdx.x];
                    ranks[w * digits + threadIdx.x] = (uint16_t)sum;
                    sum += c;
                }
                before = sum;
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kSortEach; ++k) {
                const uint64_t i = chunk + (warp * kSortEach + k) * 32 + lane;
                if (i < last) {
                    const uint32_t d = key[k] >> shift & (digits - 1);
                    const uint32_t to = base[d] + mine[d] + rank[k];
                    keys_to[to] = key[k];
                    places_to[to] = place[k];
                }
            }
            __syncthreads();
            if (threadIdx.x < digits) base[threadIdx.x] += before;
            __syncthreads();
        }
        cluster_sync();
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) valid += __shfl_xor_sync(0xFFFFFFFFu, valid, d);
    if (lane == 0) sums[warp] = valid;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kSortWarps; ++w) valid += sums[w];
        s.valid[blockIdx.x] = valid;
    }
}

// ---- backward: sums --------------------------------------------------------------------------

struct EmbedSum {
    const uint32_t *keys, *places, *valid;
    int blocks;                          // words of valid
    uint32_t segment;                    // sorted tokens of one
    const void* dy;
    uint64_t cols, lddy;
    bool vector;                         // rows of dy and dtable are on 16-byte boundaries
    float scale;
    void* dtable;
    uint64_t ldt;
    bool add;
    float* parts;                        // [segment][2][pitch]: of the run that began before the
    uint64_t pitch;                      // segment, of the one that goes on behind it
};

__device__ __forceinline__ uint32_t embed_valid(const EmbedSum& s) {
    uint32_t n = 0;
    for (int b = 0; b < s.blocks; ++b) n += __ldcg(s.valid + b);
    return n;
}

template <typename T, typename O>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(const __grid_constant__ EmbedSum s) {
    __shared__ uint32_t keys[kMaxSegment + 2], places[kMaxSegment];
    after_previous();
    let_next_begin();
    const uint32_t n = embed_valid(s), first = blockIdx.x * s.segment;
    if (first >= n) return;
    const uint32_t count = min(s.segment, n - first);
    // keys[i + 1] is that of the i-th token; before and behind: of the neighbours, or no token's
    for (uint32_t i = threadIdx.x; i < count + 2; i += kSumThreads)
        keys[i] = first + i == 0 || first + i > n ? 0xFFFFFFFFu : __ldcg(s.keys + first + i - 1);
    for (uint32_t i = threadIdx.x; i < count; i += kSumThreads) places[i] = __ldcg(s.places + first + i);
    __syncthreads();
    const uint64_t c = (uint64_t)blockIdx.y * kSumColumns +
                       (s.vector ? 8 * threadIdx.x : 256 * (threadIdx.x >> 5) + (threadIdx.x & 31));
    if (c >= s.cols) return;
    const T* dy = static_cast<const T*>(s.dy);
    float sum[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
    bool began = keys[1] != keys[0];     // the run began in this segment
    for (uint32_t i = 0; i < count; i += 4) {
        float v[4][8];                   // four rows in flight
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j < count)
                embed_load8<T>(dy + (uint64_t)places[i + j] * s.lddy, c, s.cols, s.vector, v[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (i + j >= count) break;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += v[j][k];
            const bool ends = keys[i + j + 1] != keys[i + j + 2];
            if (!ends && i + j + 1 < count) continue;
            if (began && ends) {
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] *= s.scale;
                embed_store8<O>(static_cast<O*>(s.dtable) + (uint64_t)keys[i + j + 1] * s.ldt, c, s.cols,
                                s.vector, s.add, sum);
            } else {
                embed_store8<float>(s.parts + (2ull * blockIdx.x + (began ? 1 : 0)) * s.pitch, c, s.cols,
                                    s.vector, false, sum);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
            began = true;
        }
    }
}

// The runs that go on behind their segment: a block takes 256 columns and every gridDim-th group of 32
// segments; eight warps add up the parts of a run in turns, and their sums are added in order.
template <typename O>
__global__ void __launch_bounds__(256) embed_join_kernel(const __grid_constant__ EmbedSum s) {
    __shared__ float sums[8][256];
    __shared__ uint32_t ends[8];
    after_previous();
    let_next_begin();
    const uint32_t n = embed_valid(s), segments = (n + s.segment - 1) / s.segment;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint64_t c = (uint64_t)blockIdx.y * 256 + 8 * lane;
    for (uint32_t group = blockIdx.x * 32; group < segments; group += gridDim.x * 32) {
        // (every warp finds out for itself which of the 32 a run begins in that goes on)
        const uint32_t g = group + lane, end = (g + 1) * s.segment;
        bool open = false;
        if (end < n) {
            const uint32_t k = __ldcg(s.keys + end - 1);
            open = k == __ldcg(s.keys + end) &&
                   (g == 0 || __ldcg(s.keys + g * s.segment - 1) != k);
        }
        uint32_t mask = __ballot_sync(0xFFFFFFFFu, open);
        while (mask) {
            const uint32_t from = group + __ffs(mask) - 1;
            mask &= mask - 1;
            const uint32_t k = __ldcg(s.keys + (from + 1) * s.segment - 1);
            // the segment that the run ends in
            uint32_t to = segments;
            for (uint32_t at = from + 1; at < segments && to == segments; at += 256) {
                const uint32_t i = at + threadIdx.x;
                const bool over = i < segments &&
                                  ((i + 1) * (uint64_t)s.segment >= n ||
                                   __ldcg(s.keys + (i + 1) * s.segment) != k);
                const uint32_t hit = __ballot_sync(0xFFFFFFFFu, over);
                __syncthreads();
                if (lane == 0) ends[warp] = hit ? at + 32 * warp + __ffs(hit) - 1 : segments;
                __syncthreads();
                for (int w = 7; w >= 0; --w)
                    if (ends[w] < segments) to = ends[w];
            }
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
            if (c < s.cols) {
#pragma unroll 4
                for (uint32_t i = from + warp; i <= to; i += 8) {
                    const float* p = s.parts + (2ull * i + (i == from ? 1 : 0)) * s.pitch + c;
                    const float4 a = __ldcg(reinterpret_cast<const float4*>(p));
                    const float4 b = __ldcg(reinterpret_cast<const float4*>(p) + 1);
                    v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
                    v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[warp][8 * lane + i] = v[i];
            __syncthreads();
            const uint64_t col = (uint64_t)blockIdx.y * 256 + threadIdx.x;
            if (col < s.cols) {
                float all = sums[0][threadIdx.x];
#pragma unroll
                for (int w = 1; w < 8; ++w) all += sums[w][threadIdx.x];
                all *= s.scale;
                O* p = static_cast<O*>(s.dtable) + (uint64_t)k * s.ldt + col;
                *p = from_f32<O>(s.add ? to_f32<O>(*p) + all : all);
            }
        }
    }
}

struct EmbedPlan {
    int sorters, passes, bits;
    uint32_t segment, segments;
    uint64_t pitch;
    size_t keys[2], places[2], counts, valid, parts, bytes;
};

static EmbedPlan embed_plan(uint64_t rows, uint64_t vocabulary, uint64_t cols) {
    EmbedPlan p = {};
    p.sorters = 1;
    while (p.sorters < kSortMaxBlocks && (uint64_t)p.sorters * kSortChunk < rows) p.sorters *= 2;
    int bits = 1;                        // of the keys 0 .. vocabulary
    while (vocabulary >> bits) ++bits;
    p.passes = (bits + kSortMaxBits - 1) / kSortMaxBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    const uint64_t slabs = (cols + kSumColumns - 1) / kSumColumns;
    p.segment = kMaxSegment;             // shorter ones where the chip would stand idle
    while (p.segment > 8 && (rows + p.segment - 1) / p.segment * slabs < 8 * 148) p.segment /= 2;
    p.segments = (uint32_t)((rows + p.segment - 1) / p.segment);
    p.pitch = (cols + 7) / 8 * 8;
    size_t at = 0;
    auto place = [&](size_t bytes) {
        const size_t here = at;
        at = (at + bytes + 255) & ~(size_t)255;
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = place(4 * rows);
        p.places[i] = place(4 * rows);
    }
    p.counts = place((size_t)4 * kSortMaxBlocks << kSortMaxBits);
    p.valid = place(4 * kSortMaxBlocks);
    p.parts = place(8 * (size_t)p.segments * p.pitch);
    p.bytes = at;
    return p;
}

template <typename T, typename O>
static void embed_sums(const EmbedSum& s, uint32_t segments, cudaStream_t stream) {
    const unsigned slabs = (unsigned)((s.cols + kSumColumns - 1) / kSumColumns);
    launch_overlapping(embed_sum_kernel<T, O>, dim3(segments, slabs), dim3(kSumThreads), 0, stream, s);
    const uint32_t groups = (segments + 31) / 32;
    launch_overlapping(embed_join_kernel<O>, dim3(groups, (unsigned)((s.cols + 255) / 256)), dim3(256),
                       0, stream, s);
}

template <typename T, typename O>
static void embed_forward(const EmbedTokens& tokens, const void* table, uint64_t cols, uint64_t ldt,
                          float scale, void* out, uint64_t ldo, cudaStream_t stream) {
    const bool vector =
        row_access(table, ldt, sizeof(T), tokens.vocabulary) != kRowElement &&
        row_access(out, ldo, sizeof(O), tokens.count) != kRowElement;
    const uint32_t slabs = (uint32_t)((cols + kEmbedSlab - 1) / kEmbedSlab);
    launch_overlapping(embed_forward_kernel<T, O>, dim3((unsigned)((tokens.count * slabs + 7) / 8)),
                       dim3(256), 0, stream, tokens, static_cast<const T*>(table), cols, ldt, scale,
                       static_cast<O*>(out), ldo, slabs, vector);
}

// calls f<T, O>() for two of the types
#define NC_EMBED_TYPES(t, o, f, ...)                                                              \
    do {                                                                                          \
        if (t == NC_DTYPE_F32 && o == NC_DTYPE_F32) f<float, float>(__VA_ARGS__);                 \
        else if (t == NC_DTYPE_F32 && o == NC_DTYPE_BF16) f<float, __nv_bfloat16>(__VA_ARGS__);   \
        else if (t == NC_DTYPE_F32) f<float, __half>(__VA_ARGS__);                                \
        else if (t == NC_DTYPE_BF16 && o == NC_DTYPE_F32) f<__nv_bfloat16, float>(__VA_ARGS__);   \
        else if (t == NC_DTYPE_BF16 && o == NC_DTYPE_BF16)                                        \
            f<__nv_bfloat16, __nv_bfloat16>(__VA_ARGS__);                                         \
        else if (t == NC_DTYPE_BF16) f<__nv_bfloat16, __half>(__VA_ARGS__);                       \
        else if (o == NC_DTYPE_F32) f<__half, float>(__VA_ARGS__);                                \
        else if (o == NC_DTYPE_BF16) f<__half, __nv_bfloat16>(__VA_ARGS__);                       \
        else f<__half, __half>(__VA_ARGS__);                                                      \
    } while (0)

}  // namespace natcomp

using namespace natcomp;

extern "C" {

nc_status nc_embedding_forward(const void* tokens, int token_bytes, size_t rows, const void* table,
                               int dtype, size_t vocabulary, size_t cols, size_t ldt, float scale,
                               void* out, int out_dtype, size_t ldo, cudaStream_t stream) {
    const int tb = act8_type_bytes(dtype), ob = act8_type_bytes(out_dtype);
    if (!tb || !ob || (token_bytes != 4 && token_bytes != 8)) return NC_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return NC_OK;
    if (vocabulary == 0 || !tokens || !table || !out || ldt < cols || ldo < cols)
        return NC_ERR_INVALID;
    const size_t most = (size_t)1 << 31;
    if (rows >= most || cols >= most || vocabulary >= most ||
        rows * ((cols + kEmbedSlab - 1) / kEmbedSlab) >= ((size_t)1 << 33))
        return NC_ERR_TOO_LARGE;
    if (!element_aligned(tokens, token_bytes) || !element_aligned(table, tb) ||
        !element_aligned(out, ob))
        return NC_ERR_ALIGN;
    const EmbedTokens t = {tokens, token_bytes, rows, vocabulary};
    NC_EMBED_TYPES(dtype, out_dtype, embed_forward, t, table, cols, ldt, scale, out, ldo, stream);
    return launch_status();
}

size_t nc_embedding_backward_workspace_bytes(size_t rows, size_t vocabulary, size_t cols) {
    const size_t most = (size_t)1 << 31;
    if (rows >= most || cols >= most || vocabulary >= most) return 0;
    return embed_plan(rows, vocabulary, cols).bytes;
}

nc_status nc_embedding_backward(const void* tokens, int token_bytes, size_t rows, const void* dy,
                                int dtype, size_t cols, size_t lddy, float scale, size_t vocabulary,
                                void* dtable, int dtable_dtype, size_t lddt, int accumulate,
                                void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    const int yb = act8_type_bytes(dtype), tb = act8_type_bytes(dtable_dtype);
    if (!yb || !tb || (token_bytes != 4 && token_bytes != 8)) return NC_ERR_UNSUPPORTED;
    if (vocabulary == 0 || cols == 0) return NC_OK;
    if (!dtable || lddt < cols || !workspace) return NC_ERR_INVALID;
    if (rows && (!tokens || !dy || lddy < cols)) return NC_ERR_INVALID;
    const size_t most = (size_t)1 << 31;
    if (rows >= most || cols >= (size_t)256 * 65535 || vocabulary >= most) return NC_ERR_TOO_LARGE;
    if (!element_aligned(tokens, token_bytes) || !element_aligned(dy, yb) ||
        !element_aligned(dtable, tb) || !aligned16(workspace))
        return NC_ERR_ALIGN;
    const EmbedPlan p = embed_plan(rows, vocabulary, cols);
    if (workspace_bytes < p.bytes) return NC_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    EmbedSort s = {};
    s.tokens = {tokens, token_bytes, rows, vocabulary};
    s.blocks = p.sorters; s.passes = rows ? p.passes : 0; s.bits = p.bits;
    for (int i = 0; i < 2; ++i) {
        s.keys[i] = reinterpret_cast<uint32_t*>(ws + p.keys[i]);
        s.places[i] = reinterpret_cast<uint32_t*>(ws + p.places[i]);
    }
    s.counts = reinterpret_cast<uint32_t*>(ws + p.counts);
    s.valid = reinterpret_cast<uint32_t*>(ws + p.valid);
    if (!accumulate) s.dtable = static_cast<char*>(dtable);
    s.row_bytes = cols * tb; s.row_distance = lddt * tb;
    s.vector = row_access(dtable, lddt, tb, vocabulary) != kRowElement;
    // one block on every SM, in whole clusters; no others than the sorting ones where nothing is cleared
    const int sms = device_sm_count(), clusters = s.dtable ? sms / p.sorters : 1;
    const int grid = (clusters < 2 ? (s.dtable ? 2 : 1) : clusters) * p.sorters;
    const int flags = kSortWarps * 2 << p.bits;
    const int smem = flags > kClearBytes ? flags : kClearBytes;
    static bool allowed[64];
    if (!allow_dynamic_smem((const void*)embed_sort_kernel, kSortWarps * 2 << kSortMaxBits, allowed))
        return NC_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = p.sorters;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaLaunchKernelEx(&cfg, embed_sort_kernel, s);
    if (rows == 0) return launch_status();
    EmbedSum e = {};
    e.keys = s.keys[0]; e.places = s.places[0]; e.valid = s.valid; e.blocks = p.sorters;
    e.segment = p.segment; e.dy = dy; e.cols = cols; e.lddy = lddy;
    e.vector = row_access(dy, lddy, yb, rows) != kRowElement && s.vector;
    e.scale = scale; e.dtable = dtable; e.ldt = lddt; e.add = accumulate != 0;
    e.parts = reinterpret_cast<float*>(ws + p.parts); e.pitch = p.pitch;
    NC_EMBED_TYPES(dtype, dtable_dtype, embed_sums, e, p.segments, stream);
    return launch_status();
}

}  // extern "C"
