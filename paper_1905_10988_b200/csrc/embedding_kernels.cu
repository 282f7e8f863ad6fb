// Embedding of tokens and its gradient, for sm_100a:
//
//   out[t] = scale * table[token[t]],     dtable[v] = scale * sum of dy[t] over the t of token v
//
// Forward, a warp moves up to 1024 columns of a row.  What bounds it: HBM.
//
// Backward, the tokens are sorted with their places, so that equal ones are neighbours in the order
// of their places, and each row of the gradient is a sum in that order or, of many rows, of such sums: no
// atomics, the same bits from run to run.  Rows that no token names are cleared by blocks of their own, each of which scans the
// tokens for those of its rows, so that every row is written once.  Three kernels:
//   - one cluster of up to eight blocks sorts (radix sort from the low digit, two digits up to a
//     vocabulary of a million), while all other blocks clear as many rows as that takes time for;
//   - segments of the sorted tokens are added up, a thread eight columns; runs of equal tokens that are
//     not cut between segments are finished there, the others leave binary32 sums behind; other blocks
//     clear rows meanwhile;
//   - those sums are joined in order.
// Up to 512 tokens there is one kernel: a block for each token, of which the first of equal ones finds
// the others by a scan and adds them up.
// What bounds it: HBM, by the gradient that is written and the rows that are read.
#include <type_traits>

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
// Tokens that are not sorted at most.  512 tokens into 8192 x 768 binary32: 9 us, sorted 19; into 32001 x 1001 26
// and 39; into 65536 x 4096 bfloat16 94 and 96.  With a limit of 2048, which takes more registers: 512 10.6, 27
// and 97; 1024 14, 31 and 112, sorted 20, 39 and 99; 2048 22, 40 and 146, sorted 21, 41 and 103.  So 512 is where
// the largest table breaks even; a small one takes twice as long from 513 tokens on, and would not up to 1500.
constexpr int kDirect = 512;
constexpr int kDirectThreads = 512;
// What is cleared beside the sort.  The blocks that do have scanned the tokens 7 to 8 us before the sort ends
// (4096 tokens: after 4 of 11 us, 16384: after 7 of 15) and clear about 9 MB a microsecond.
constexpr uint64_t kClearBeside = 64 << 20;
// Bytes that a block clears beside the sums.  16384 x 4096 into 65536 rows, 4096 x 2048 into 32768, 8191 x 1001
// into 32001: 137, 39, 48 us; 24 KB 136, 38, 46; 400 KB 142, 76, 88.
constexpr uint64_t kClearBlock = 96 << 10;
// Cuts of a run that one warp joins.  30000 x 768 binary32 of one token: 179 us; left to one warp whatever the
// number 252, all runs by eight warps 196.
constexpr int kJoinShort = 12;

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

// eight values of a row, neighbours from c on or, spread, every 32nd from c on, as they lie in memory, and
// to binary32
template <typename T> struct EmbedRaw {
    uint32_t w[2 * sizeof(T)];
};

// (OWN: of a row that this thread writes later, so not through the cache for what no one writes)
template <typename T, bool OWN = false>
__device__ __forceinline__ EmbedRaw<T> embed_load_raw(const T* row, uint64_t c, uint64_t cols, bool vector) {
    EmbedRaw<T> r;
    if (vector && c + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const uint4* p = reinterpret_cast<const uint4*>(row + c) + i;
            const uint4 q = OWN ? __ldcg(p) : __ldg(p);
            r.w[4 * i] = q.x; r.w[4 * i + 1] = q.y; r.w[4 * i + 2] = q.z; r.w[4 * i + 3] = q.w;
        }
    } else {
        typedef typename std::conditional<sizeof(T) == 4, uint32_t, unsigned short>::type Word;
        const int step = vector ? 1 : 32;
        const Word* p = reinterpret_cast<const Word*>(row) + c;
        uint32_t w[8];
        if (c + 7 * step < cols) {       // (all of them: loads without a question each)
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = OWN ? __ldcg(p + i * step) : __ldg(p + i * step);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = 0u;
                if (c + i * step < cols) w[i] = OWN ? __ldcg(p + i * step) : __ldg(p + i * step);
            }
        }
#pragma unroll
        for (int i = 0; i < 2 * (int)sizeof(T); ++i)
            r.w[i] = sizeof(T) == 4 ? w[i & 7] : w[2 * i & 7] | w[(2 * i + 1) & 7] << 16;
    }
    return r;
}

template <typename T>
__device__ __forceinline__ void embed_unpack(const EmbedRaw<T>& r, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack2<T>(r.w[i], v[2 * i], v[2 * i + 1]);
    }
}

template <typename T>
__device__ __forceinline__ void embed_store8(T* row, uint64_t c, uint64_t cols, bool vector, bool add,
                                             float (&v)[8]) {
    if (vector && c + 8 <= cols) {
        uint4* p = reinterpret_cast<uint4*>(row + c);
        if (add) {
            float old[8];
            embed_unpack<T>(embed_load_raw<T, true>(row, c, cols, true), old);
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
        T* p = row + c;
        if (!add && c + 7 * step < cols) {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i * step] = from_f32<T>(v[i]);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i * step < cols)
                p[i * step] = from_f32<T>(add ? to_f32<T>(p[i * step]) + v[i] : v[i]);
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
    EmbedRaw<T> raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (in)
            raw[i] = embed_load_raw<T>(row, base + 256 * i + (vector ? 8 * lane : lane), cols, vector);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[8];
        if (in) {
            embed_unpack<T>(raw[i], v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= scale;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = fill;
        }
        embed_store8<O>(to, base + 256 * i + (vector ? 8 * lane : lane), cols, vector, false, v);
    }
}

// ---- backward: sorted tokens, and the rows without any ------------------------------------------

struct EmbedClear {
    EmbedTokens tokens;
    char* dtable;
    uint64_t row_bytes, row_distance;
    uint64_t begin, end;                 // rows
};

struct EmbedSort {
    EmbedTokens tokens;
    int blocks;                          // of the cluster that sorts
    int passes, bits;                    // digits, and bits of one
    uint2* items[2];                     // key, place; the sorted ones end up in [0]
    uint32_t* counts;                    // [block][digits]
    uint32_t* valid;                     // tokens in the vocabulary
    EmbedClear clear;
};

// zeros from p on, `bytes` of them (both even)
__device__ __forceinline__ void embed_zero(char* p, uint64_t bytes, int lane) {
    const uint64_t head = min((uint64_t)(-(uintptr_t)p & 15), bytes), n = (bytes - head) / 16;
    if (2 * lane < head) reinterpret_cast<unsigned short*>(p)[lane] = 0;
    uint4* q = reinterpret_cast<uint4*>(p + head);
#pragma unroll 4
    for (uint64_t i = lane; i < n; i += 32) q[i] = make_uint4(0u, 0u, 0u, 0u);
    const uint64_t at = head + 16 * n + 2 * lane;
    if (at < bytes) *reinterpret_cast<unsigned short*>(p + at) = 0;
}

// the first of n sorted items whose key is not below `key`: all threads of the block look at as many places at a
// time
__device__ __forceinline__ uint32_t embed_find(const uint2* items, uint32_t n, uint32_t key) {
    uint32_t low = 0, high = n;          // it is in [low, high]
    while (low < high) {
        const uint32_t step = (high - low + blockDim.x - 1) / blockDim.x;
        const uint64_t at = low + (uint64_t)threadIdx.x * step;
        const int below = __syncthreads_count(at < high && __ldcg(&items[at].x) < key);
        if (below == 0) return low;      // (those below are the first threads')
        const uint64_t next = low + (uint64_t)below * step;
        low = low + (below - 1) * step + 1;
        high = (uint32_t)min(next, (uint64_t)high);
    }
    return low;
}

// Clears the rows from `begin` to `end` that no token names: block `block` of `blocks` takes every so
// many-th range of rows, whose flags fit into its memory.  items: the n sorted ones, or nullptr where they
// are not there yet and all tokens are looked at instead.
__device__ __forceinline__ void embed_clear(const EmbedClear& s, uint32_t* flags, uint32_t block,
                                            uint32_t blocks, const uint2* items, uint32_t n) {
    if (s.begin >= s.end) return;
    uint64_t range = (s.end - s.begin + blocks - 1) / blocks;
    if (range > 8 * kClearBytes) range = 8 * kClearBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    for (uint64_t first = s.begin + block * range; first < s.end; first += blocks * range) {
        const uint64_t rows = min(range, s.end - first);
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < (rows + 31) / 32; i += blockDim.x) flags[i] = 0;
        __syncthreads();
        if (items) {
            for (uint32_t i = embed_find(items, n, (uint32_t)first) + threadIdx.x; i < n; i += blockDim.x) {
                const uint64_t k = (uint64_t)__ldcg(&items[i].x) - first;
                if (k >= rows) break;
                atomicOr(flags + (k >> 5), 1u << (k & 31));
            }
        } else {
            // (every block begins at another place, or all of them ask the same parts of L2 at a time)
            const uint32_t n = (uint32_t)s.tokens.count, turn = (uint32_t)((uint64_t)n * block / blocks);
            for (uint32_t i = threadIdx.x; i < n; i += 4 * blockDim.x) {
                uint32_t key[4];         // (all loads before the first use)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t to = i + j * blockDim.x, at = to < n - turn ? to + turn : to - (n - turn);
                    key[j] = to < n ? s.tokens.key(at) : 0xFFFFFFFFu;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t k = key[j] - (uint32_t)first;
                    if (k < (uint32_t)rows) atomicOr(flags + (k >> 5), 1u << (k & 31));
                }
            }
        }
        __syncthreads();
        for (uint64_t r = warp; r < rows; r += warps)
            if (!(flags[r >> 5] >> (r & 31) & 1))
                embed_zero(s.dtable + (first + r) * s.row_distance, s.row_bytes, lane);
    }
}

// two words to the same place in block `rank` of the cluster
__device__ __forceinline__ void shared_store_pair_at(uint32_t at, uint32_t rank, uint2 v) {
    asm volatile("{\n\t"
                 ".reg .b32 remote;\n\t"
                 "mapa.shared::cluster.u32 remote, %0, %1;\n\t"
                 "st.shared::cluster.v2.u32 [remote], {%2, %3};\n\t"
                 "}" ::"r"(at), "r"(rank), "r"(v.x), "r"(v.y)
                 : "memory");
}

// One digit of a chunk of items: a warp's are neighbours, 32 for each round.  Afterwards rank[k] is that
// of the thread's k-th item among its warp's with the same digit, ranks[warp][digit] how many the warps
// before have, and the result, of thread `digit`, how many there are in the chunk.  ON_CHIP: items are
// those of the chunk, in shared memory.
template <bool ON_CHIP>
__device__ __forceinline__ uint32_t embed_rank(const EmbedSort& s, const uint2* items, int pass, int rounds,
                                               uint64_t chunk, uint64_t last, uint16_t* ranks,
                                               uint2 (&item)[kSortEach], uint32_t (&rank)[kSortEach]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, shift = pass * s.bits;
    const uint32_t digits = 1u << s.bits, below = (1u << lane) - 1;
    for (uint32_t i = threadIdx.x; i < kSortWarps * digits / 2; i += kSortThreads)
        reinterpret_cast<uint32_t*>(ranks)[i] = 0;
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
        if (k >= rounds) break;
        const uint32_t at = (warp * rounds + k) * 32 + lane;
        const uint64_t i = chunk + at;
        item[k] = i >= last    ? make_uint2(0xFFFFFFFFu, 0u)
                  : pass == 0  ? make_uint2(s.tokens.key(i), (uint32_t)i)
                  : ON_CHIP    ? items[at]
                               : __ldcg(items + i);
    }
    __syncthreads();
    uint16_t* mine = ranks + warp * digits;
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
        if (k >= rounds) break;
        const bool in = chunk + (warp * rounds + k) * 32 + lane < last;
        const uint32_t d = item[k].x >> shift & (digits - 1);
        // lanes with the same digit: a vote for each bit (the instruction that finds equal values takes
        // about 118 cycles of an SM with this many different ones, the votes a tenth)
        uint32_t same = __ballot_sync(0xFFFFFFFFu, in);
        for (int b = 0; b < s.bits; ++b) {
            const uint32_t ones = __ballot_sync(0xFFFFFFFFu, d >> b & 1);
            same &= d >> b & 1 ? ones : ~ones;
        }
        const uint32_t old = in ? mine[d] : 0;
        rank[k] = old + __popc(same & below);
        __syncwarp();
        if (in && (same & below) == 0) mine[d] = (uint16_t)(old + __popc(same));
        __syncwarp();
    }
    __syncthreads();
    uint32_t sum = 0;
    if (threadIdx.x < digits) {
#pragma unroll 8
        for (int w = 0; w < kSortWarps; ++w) {
            const uint32_t c = ranks[w * digits + threadIdx.x];
            ranks[w * digits + threadIdx.x] = (uint16_t)sum;
            sum += c;
        }
    }
    return sum;
}

// ON_CHIP: a block's items are one chunk.  Between the passes they are held by the cluster's shared
// memory, block b the places from b * each on, and so are the counts: nothing goes through L2, which the
// blocks that clear keep busy.  (16384 tokens of a vocabulary of 65536: 16 us; 19 through L2 and with the
// instruction that finds equal lanes.)
template <bool ON_CHIP>
__global__ void __launch_bounds__(kSortThreads, 1) embed_sort_kernel(const __grid_constant__ EmbedSort s) {
    // [warp][digit]; ON_CHIP, behind it, of every block how many items have each digit, and the items
    extern __shared__ uint16_t ranks[];
    __shared__ uint32_t base[1 << kSortMaxBits];
    __shared__ uint32_t sums[kSortWarps];
    __shared__ uint32_t valids[kSortMaxBlocks];      // of the first block
    const bool clears = (int)blockIdx.x >= s.blocks;
    if (!clears) cluster_sync();         // all of its blocks run
    after_previous();
    let_next_begin();
    if (clears) {
        embed_clear(s.clear, reinterpret_cast<uint32_t*>(ranks), blockIdx.x - s.blocks,
                    gridDim.x - s.blocks, nullptr, 0);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t digits = 1u << s.bits, number = blockIdx.x;
    uint32_t* counts = reinterpret_cast<uint32_t*>(ranks + kSortWarps * digits);
    uint2* here = reinterpret_cast<uint2*>(counts + s.blocks * digits);
    const uint64_t n = s.tokens.count;
    const uint32_t each = (uint32_t)((n + s.blocks - 1) / s.blocks);
    const uint64_t first = min((uint64_t)number * each, n), last = min(first + each, n);
    // of a warp in a chunk: 32 items each
    const int rounds = min((int)((each + kSortThreads - 1) / kSortThreads), kSortEach);
    uint2 item[kSortEach];
    uint32_t rank[kSortEach];
    uint32_t valid = 0;
    for (int pass = 0; pass < s.passes; ++pass) {
        // from buffer (passes - pass) & 1 to the other one, or through the blocks' own
        const uint2* items = ON_CHIP ? here : s.items[(s.passes - pass) & 1];
        uint2* to = s.items[ON_CHIP ? 0 : (s.passes - pass - 1) & 1];
        const int shift = pass * s.bits;
        // how many items of the block have each digit, by thread
        uint32_t mine = 0;
        if (ON_CHIP) {
            mine = embed_rank<true>(s, items, pass, rounds, first, last, ranks, item, rank);
            if (pass == 0)
#pragma unroll
                for (int k = 0; k < kSortEach; ++k)      // (none: a key beyond all)
                    if (k < rounds) valid += item[k].x < s.tokens.vocabulary;
            if (threadIdx.x < digits)
                for (int b = 0; b < s.blocks; ++b)
                    shared_store_at(smem_u32(counts + number * digits + threadIdx.x), b, mine);
        } else {
            for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) base[d] = 0;
            __syncthreads();
            for (uint64_t i = first + threadIdx.x; i < last; i += kSortThreads) {
                const uint32_t k = pass ? __ldcg(&items[i].x) : s.tokens.key(i);
                if (pass == 0) valid += k < s.tokens.vocabulary;
                atomicAdd(base + (k >> shift & (digits - 1)), 1u);
            }
            __syncthreads();
            if (threadIdx.x < digits) s.counts[number * digits + threadIdx.x] = base[threadIdx.x];
        }
        if (pass == 0) {
#pragma unroll
            for (int d = 16; d; d >>= 1) valid += __shfl_xor_sync(0xFFFFFFFFu, valid, d);
            if (lane == 0) sums[warp] = valid;
            __syncthreads();
            if (threadIdx.x == 0) {
                for (int w = 1; w < kSortWarps; ++w) valid += sums[w];
                shared_store_at(smem_u32(valids + number), 0, valid);
            }
        }
        cluster_sync();
        if (pass == 0 && number == 0 && threadIdx.x == 0) {
            valid = 0;
            for (int b = 0; b < s.blocks; ++b) valid += valids[b];
            *s.valid = valid;
        }
        // the items of lower digits, and of this one in the blocks before
        uint32_t before = 0, all = 0;
        if (threadIdx.x < digits) {
#pragma unroll
            for (int b = 0; b < kSortMaxBlocks; ++b) {
                uint32_t c = 0;
                if (b < s.blocks)
                    c = ON_CHIP ? counts[b * digits + threadIdx.x]
                                : __ldcg(s.counts + b * digits + threadIdx.x);
                before += b < (int)number ? c : 0;
                all += c;
            }
        }
        uint32_t up = all;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t other = __shfl_sync(0xFFFFFFFFu, up, lane >= d ? lane - d : lane);
            if (lane >= d) up += other;
        }
        if (lane == 31) sums[warp] = up;
        __syncthreads();
        uint32_t lower = lane < warp ? sums[lane] : 0;
#pragma unroll
        for (int d = 16; d; d >>= 1) lower += __shfl_xor_sync(0xFFFFFFFFu, lower, d);
        if (threadIdx.x < digits) base[threadIdx.x] = before + lower + up - all;
        for (uint64_t chunk = first; ON_CHIP || chunk < last; chunk += rounds * kSortThreads) {
            if (!ON_CHIP) {
                __syncthreads();
                mine = embed_rank<false>(s, items, pass, rounds, chunk, last, ranks, item, rank);
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kSortEach; ++k) {
                if (k >= rounds) break;
                if (chunk + (warp * rounds + k) * 32 + lane < last) {
                    const uint32_t d = item[k].x >> shift & (digits - 1);
                    const uint32_t at = base[d] + ranks[warp * digits + d] + rank[k];
                    if (ON_CHIP && pass + 1 < s.passes) {
                        const uint32_t owner = at / each;
                        shared_store_pair_at(smem_u32(here + (at - owner * each)), owner, item[k]);
                    } else {
                        to[at] = item[k];
                    }
                }
            }
            if (ON_CHIP) break;
            __syncthreads();
            if (threadIdx.x < digits) base[threadIdx.x] += mine;
        }
        // (the last pass of the chip leaves nothing that a block of the cluster reads)
        if (!ON_CHIP || pass + 1 < s.passes) cluster_sync();
    }
}

// ---- backward: sums --------------------------------------------------------------------------

struct EmbedSum {
    const uint2* items;
    const uint32_t* valid;
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
    uint32_t segments;
    uint32_t across;                     // threads that take eight columns each of a block's 1024
    EmbedClear clear;
};

// tokens in the vocabulary.  One thread of a block asks: asked by every warp of a few thousand blocks, the
// one place in L2 that has it held the joins up by 10 us.
__device__ __forceinline__ uint32_t embed_valid(const EmbedSum& s) {
    __shared__ uint32_t n;
    if (threadIdx.x == 0) n = __ldcg(s.valid);
    __syncthreads();
    return n;
}

// Segment g has the sorted tokens from about g * segment on.  A run of equal ones across that place is
// left to the segment before, where it ends within `segment` tokens; longer ones are cut there.
__device__ __forceinline__ bool embed_cut(const EmbedSum& s, uint32_t g, uint32_t n) {
    const uint64_t p = (uint64_t)g * s.segment;
    if (g == 0 || p + s.segment >= n) return false;
    const uint32_t a = __ldcg(&s.items[p - 1].x), b = __ldcg(&s.items[p].x),
                   c = __ldcg(&s.items[p + s.segment].x);
    return (a == b) & (b == c);          // (three loads at a time)
}

template <typename T, typename O, bool ADD>
__global__ void __launch_bounds__(kSumThreads, ADD ? 5 : 8) embed_sum_kernel(const __grid_constant__ EmbedSum s) {
    // of a block's groups of threads, each with a segment of its own: key and place of up to twice as many
    // tokens, and the keys of the ones before and behind
    __shared__ uint32_t keys[4][2 * kMaxSegment + 2], places[4][2 * kMaxSegment];
    __shared__ uint32_t flags[kClearBytes / 4];
    after_previous();
    let_next_begin();
    const uint32_t n = embed_valid(s), groups = kSumThreads / s.across;
    const uint32_t works = (s.segments + groups - 1) / groups, number = blockIdx.x;
    if (number >= works) {               // (last: evenly between the others they took 1 to 3 us longer)
        embed_clear(s.clear, flags, (number - works) * gridDim.y + blockIdx.y,
                    (gridDim.x - works) * gridDim.y, s.items, n);
        return;
    }
    const uint32_t group = threadIdx.x / s.across, x = threadIdx.x - group * s.across;
    const uint32_t g = number * groups + group, first = g * s.segment;
    const bool any = group < groups && g < s.segments && first < n;
    uint32_t* key = keys[group & 3];
    uint32_t* place = places[group & 3];
    if (any)
        for (uint32_t i = x; i < 2 * s.segment + 2; i += s.across) {
            const uint32_t at = first + i - 1;           // key[i] is that of token `at`
            const bool in = first + i > 0 && at < n;
            const uint2 item = in ? __ldcg(s.items + at) : make_uint2(0xFFFFFFFFu, 0u);
            key[i] = item.x;
            if (i > 0 && i <= 2 * s.segment) place[i - 1] = item.y;
        }
    __syncthreads();
    if (!any) return;
    // from `at` tokens on, the first that begins a run, within a segment's length, or else `at`
    const auto border = [&](uint32_t at) {
        if (first + at >= n || first + at == 0) return min(at, n - first);
        for (uint32_t i = 0; i <= s.segment; ++i)
            if (key[at + i] != key[at + i + 1]) return at + i;
        return at;
    };
    const uint32_t begin = border(0), end = border(s.segment);
    if (begin >= end) return;
    const uint64_t c = (uint64_t)blockIdx.y * kSumColumns +
                       (s.vector ? 8 * x : 256 * (x >> 5) + (x & 31));
    if (c >= s.cols) return;
    const T* dy = static_cast<const T*>(s.dy);
    float sum[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
    bool began = key[begin] != key[begin + 1];           // the run began in this segment
    // Rows at a time: as many as 64 registers hold, so that eight blocks share an SM.  (Eight rows of 16-bit
    // values in 96 registers: 8191 x 1001 62 us instead of 52, 16384 x 2048 of 2001 tokens 48 instead of 41.  With
    // the rows that are added to, five blocks: 14336 x 4096 87 us instead of 98.)
    constexpr int kFlight = 8 / sizeof(T);
    for (uint32_t i = begin; i < end; i += kFlight) {
        EmbedRaw<T> raw[kFlight];
        EmbedRaw<O> old[ADD ? kFlight : 1];              // the rows that the sums are added to
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (i + j < end) {
                raw[j] = embed_load_raw<T>(dy + (uint64_t)place[i + j] * s.lddy, c, s.cols, s.vector);
                if (ADD && key[i + j + 1] != key[i + j + 2])
                    old[j] = embed_load_raw<O, true>(
                        static_cast<const O*>(s.dtable) + (uint64_t)key[i + j + 1] * s.ldt, c, s.cols,
                        s.vector);
            }
#pragma unroll
        for (int j = 0; j < kFlight; ++j) {
            if (i + j >= end) break;
            float v[8];
            embed_unpack<T>(raw[j], v);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += v[k];
            const bool ends = key[i + j + 1] != key[i + j + 2];
            if (!ends && i + j + 1 < end) continue;
            if (began && ends) {
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] *= s.scale;
                if (ADD) {
                    embed_unpack<O>(old[j], v);
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum[k] += v[k];
                }
                embed_store8<O>(static_cast<O*>(s.dtable) + (uint64_t)key[i + j + 1] * s.ldt, c, s.cols,
                                s.vector, false, sum);
            } else {
                embed_store8<float>(s.parts + (2ull * g + (began ? 1 : 0)) * s.pitch, c, s.cols, s.vector,
                                    false, sum);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
            began = true;
        }
    }
}

// The runs that were cut.  A block takes 256 columns and eight segments; a warp joins the run whose first
// cut is at the beginning of its segment, in the order of the segments.  Runs with more than 12 cuts are
// left to all eight warps, which take a run's parts in turns and add up their sums in order.
template <typename O>
__global__ void __launch_bounds__(256) embed_join_kernel(const __grid_constant__ EmbedSum s) {
    __shared__ float sums[8][256];
    __shared__ uint32_t ends[8];         // of each of those runs: the segment after its last cut
    after_previous();
    let_next_begin();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t n = embed_valid(s), segments = (n + s.segment - 1) / s.segment;
    const uint64_t c = (uint64_t)blockIdx.y * 256 + 8 * lane;
    const uint32_t group = blockIdx.x * 8;
    if (group >= segments) return;
    // (every warp finds out for itself which of the eight a run is cut at for the first time)
    const uint32_t g = group + (lane & 7);
    const bool cut = embed_cut(s, g, n), before = embed_cut(s, g ? g - 1 : 0, n);
    const uint32_t mask = __ballot_sync(0xFFFFFFFFu, cut && !before) & 0xFFu;
    if (!mask) return;
    if (mask >> warp & 1) {
        const uint32_t from = group + warp;
        uint32_t to = segments;          // the segment behind the last cut is the first that is not cut
        for (uint32_t at = from + 1; at < segments && to == segments; at += 32) {
            const uint32_t hit = __ballot_sync(0xFFFFFFFFu, !embed_cut(s, at + lane, n));
            if (hit) to = min(at + __ffs(hit) - 1, segments);
        }
        if (lane == 0) ends[warp] = to;
        if (to - from <= kJoinShort && c < s.cols) {
            const uint32_t k = __ldcg(&s.items[(uint64_t)from * s.segment].x);
            float v[8];
            const float4* p = reinterpret_cast<const float4*>(s.parts + (2ull * from - 1) * s.pitch + c);
            *reinterpret_cast<float4*>(v) = __ldcg(p);
            *reinterpret_cast<float4*>(v + 4) = __ldcg(p + 1);
#pragma unroll 4
            for (uint32_t i = from; i < to; ++i) {
                const float4* q = reinterpret_cast<const float4*>(s.parts + 2ull * i * s.pitch + c);
                const float4 a = __ldcg(q), b = __ldcg(q + 1);
                v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
                v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
            }
            // (values of neighbouring columns, also where rows are at any element)
            O* row = static_cast<O*>(s.dtable) + (uint64_t)k * s.ldt;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= s.scale;
            if (s.vector) {
                embed_store8<O>(row, c, s.cols, true, s.add, v);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < s.cols)
                        row[c + i] = from_f32<O>(s.add ? to_f32<O>(row[c + i]) + v[i] : v[i]);
            }
        }
    }
    __syncthreads();
    for (uint32_t m = mask; m; m &= m - 1) {
        const uint32_t which = __ffs(m) - 1, from = group + which, to = ends[which];
        if (to - from <= kJoinShort) continue;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        if (c < s.cols) {
            // (the part before the first cut is the second one of the segment before)
#pragma unroll 4
            for (uint32_t i = from + warp; i <= to; i += 8) {
                const float* p = s.parts + (i == from ? 2ull * from - 1 : 2ull * (i - 1)) * s.pitch + c;
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
            const uint32_t k = __ldcg(&s.items[(uint64_t)from * s.segment].x);
            O* p = static_cast<O*>(s.dtable) + (uint64_t)k * s.ldt + col;
            *p = from_f32<O>(s.add ? to_f32<O>(*p) + all : all);
        }
    }
}

// ---- backward: few tokens ----------------------------------------------------------------------

struct EmbedDirect {
    EmbedTokens tokens;
    const void* dy;
    uint64_t cols, lddy;
    bool vector;
    float scale;
    void* dtable;
    uint64_t ldt;
    bool add;
    uint32_t across;                     // threads that take eight columns each of a block's 1024
    EmbedClear clear;
};

// Blocks of the first tokens.count: the token of the block's number, if it is the first of its kind.
// Threads beyond `across` take other rows of the sum in turns.
template <typename T, typename O>
__global__ void __launch_bounds__(kDirectThreads) embed_direct_kernel(const __grid_constant__ EmbedDirect s) {
    __shared__ uint32_t flags[kClearBytes / 4];
    __shared__ uint32_t counts[kDirectThreads / 32];
    after_previous();
    let_next_begin();
    const uint32_t n = (uint32_t)s.tokens.count;
    if (blockIdx.x >= n) {
        embed_clear(s.clear, flags, (blockIdx.x - n) * gridDim.y + blockIdx.y,
                    (gridDim.x - n) * gridDim.y, nullptr, 0);
        return;
    }
    // places of the tokens like this one, in order, and the sums of the rows' groups in passing
    static_assert(kDirect + 8 * kSumThreads <= kClearBytes / 4, "");
    uint32_t* places = flags;
    float* sums = reinterpret_cast<float*>(flags + kDirect);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t mine = s.tokens.key(blockIdx.x);
    if (mine >= s.tokens.vocabulary) return;
    uint32_t found[kDirect / kDirectThreads];
    bool before = false;
#pragma unroll
    for (int k = 0; k < kDirect / kDirectThreads; ++k) {
        const uint32_t i = k * kDirectThreads + threadIdx.x;
        const bool same = i < n && s.tokens.key(i) == mine;
        before |= same && i < blockIdx.x;
        found[k] = __ballot_sync(0xFFFFFFFFu, same);
    }
    if (__syncthreads_or(before)) return;
    uint32_t count = 0;
#pragma unroll
    for (int k = 0; k < kDirect / kDirectThreads; ++k) {
        __syncthreads();
        if (lane == 0) counts[warp] = __popc(found[k]);
        __syncthreads();
        uint32_t at = count;
        for (int w = 0; w < kDirectThreads / 32; ++w) {
            if (w < warp) at += counts[w];
            count += counts[w];
        }
        if (found[k] >> lane & 1)
            places[at + __popc(found[k] & ((1u << lane) - 1))] = k * kDirectThreads + threadIdx.x;
    }
    __syncthreads();
    const uint32_t groups = kDirectThreads / s.across, group = threadIdx.x / s.across;
    const uint32_t x = threadIdx.x - group * s.across;
    const uint64_t base = (uint64_t)blockIdx.y * kSumColumns;
    const uint64_t c = base + (s.vector ? 8 * x : 256 * (x >> 5) + (x & 31));
    const T* dy = static_cast<const T*>(s.dy);
    float sum[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
    if (group < groups && c < s.cols) {
        for (uint32_t i = group; i < count; i += 4 * groups) {
            EmbedRaw<T> raw[4];          // four rows in flight
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i + j * groups < count)
                    raw[j] = embed_load_raw<T>(dy + (uint64_t)places[i + j * groups] * s.lddy, c, s.cols,
                                               s.vector);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (i + j * groups >= count) break;
                float v[8];
                embed_unpack<T>(raw[j], v);
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] += v[k];
            }
        }
    }
    // the groups' sums in order (none but the first has any where there are fewer rows)
    const uint32_t used = min(groups, count);
    for (uint32_t g = 1; g < used; ++g) {
        __syncthreads();
        if (group == g)
#pragma unroll
            for (int k = 0; k < 8; ++k) sums[k * s.across + x] = sum[k];
        __syncthreads();
        if (group == 0)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += sums[k * s.across + x];
    }
    if (group == 0 && c < s.cols) {
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] *= s.scale;
        embed_store8<O>(static_cast<O*>(s.dtable) + (uint64_t)mine * s.ldt, c, s.cols, s.vector, s.add,
                        sum);
    }
}

struct EmbedPlan {
    int sorters, passes, bits;
    uint32_t segment, segments, across;
    uint64_t pitch;
    size_t items[2], counts, valid, parts, bytes;
};

// threads that share a slab of columns: whole warps, because spread columns need them; one at least, also
// where there are no columns
static uint32_t embed_across(uint64_t cols) {
    const uint64_t eights = (cols + 7) / 8;
    return eights >= kSumThreads ? kSumThreads : eights ? (uint32_t)(eights + 31) / 32 * 32 : 32;
}

// (columns: a grid has 65535 blocks of 256 in its second dimension)
static bool embed_fits(size_t rows, size_t vocabulary, size_t cols) {
    const size_t most = (size_t)1 << 31;
    return rows < most && vocabulary < most && cols < (size_t)256 * 65535;
}

static EmbedPlan embed_plan(uint64_t rows, uint64_t vocabulary, uint64_t cols) {
    EmbedPlan p = {};
    p.sorters = 1;
    while (p.sorters < kSortMaxBlocks && (uint64_t)p.sorters * 2 * kSortThreads <= rows) p.sorters *= 2;
    int bits = 1;                        // of the keys 0 .. vocabulary
    while (vocabulary >> bits) ++bits;
    p.passes = (bits + kSortMaxBits - 1) / kSortMaxBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    const uint64_t slabs = (cols + kSumColumns - 1) / kSumColumns;
    p.across = embed_across(cols);
    const uint64_t groups = kSumThreads / p.across;
    // Shorter segments where the chip would stand idle: 1024 x 768 20 us, in segments of 32 27; 4096 x 2048
    // 40 and 47.
    p.segment = kMaxSegment;
    while (p.segment > 8 && (rows / p.segment + 1) * slabs / groups < 8 * 148) p.segment /= 2;
    p.segments = (uint32_t)((rows + p.segment - 1) / p.segment);
    p.pitch = (cols + 7) / 8 * 8;
    size_t at = 0;
    auto place = [&](size_t bytes) {
        const size_t here = at;
        at = (at + bytes + 255) & ~(size_t)255;
        return here;
    };
    for (int i = 0; i < 2; ++i) p.items[i] = place(8 * rows);
    p.counts = place((size_t)4 * kSortMaxBlocks << kSortMaxBits);
    p.valid = place(4);
    p.parts = place(8 * (size_t)p.segments * p.pitch);
    p.bytes = at;
    return p;
}

template <typename T, typename O>
static void embed_sums(const EmbedSum& s, uint32_t segments, cudaStream_t stream) {
    const unsigned slabs = (unsigned)((s.cols + kSumColumns - 1) / kSumColumns);
    const unsigned columns = (unsigned)((s.cols + 255) / 256);
    // blocks that clear take about as long as those that add up
    const uint32_t groups = kSumThreads / s.across;
    const auto clears = [](const EmbedClear& c, unsigned down) {
        if (c.begin >= c.end) return 0u;
        const uint64_t n = (c.end - c.begin) * c.row_bytes / kClearBlock / down + 1;
        return (unsigned)(n < 65536 ? n : 65536);
    };
    const unsigned clear = clears(s.clear, slabs);
    launch_overlapping(s.add ? embed_sum_kernel<T, O, true> : embed_sum_kernel<T, O, false>,
                       dim3((segments + groups - 1) / groups + clear, slabs), dim3(kSumThreads), 0, stream,
                       s);
    launch_overlapping(embed_join_kernel<O>, dim3((segments + 7) / 8, columns), dim3(256), 0,
                       stream, s);
}

template <typename T, typename O>
static void embed_direct(const EmbedDirect& s, cudaStream_t stream) {
    const unsigned slabs = (unsigned)((s.cols + kSumColumns - 1) / kSumColumns);
    const unsigned clear = s.clear.begin < s.clear.end ? (4 * 148 + slabs - 1) / slabs : 0;
    const unsigned blocks = (unsigned)s.tokens.count + clear;
    if (blocks)
        launch_overlapping(embed_direct_kernel<T, O>, dim3(blocks, slabs), dim3(kDirectThreads), 0,
                           stream, s);
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
    return embed_fits(rows, vocabulary, cols) ? embed_plan(rows, vocabulary, cols).bytes : 0;
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
    if (!embed_fits(rows, vocabulary, cols)) return NC_ERR_TOO_LARGE;
    if (!element_aligned(tokens, token_bytes) || !element_aligned(dy, yb) ||
        !element_aligned(dtable, tb) || !aligned16(workspace))
        return NC_ERR_ALIGN;
    const EmbedPlan p = embed_plan(rows, vocabulary, cols);
    if (workspace_bytes < p.bytes) return NC_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    const bool vector = row_access(dtable, lddt, tb, vocabulary) != kRowElement &&
                        row_access(dy, lddy, yb, rows) != kRowElement;
    EmbedClear clear = {};
    clear.tokens = {tokens, token_bytes, rows, vocabulary};
    clear.dtable = static_cast<char*>(dtable);
    clear.row_bytes = cols * tb; clear.row_distance = lddt * tb;
    clear.end = accumulate ? 0 : vocabulary;
    if (rows <= kDirect) {
        EmbedDirect d = {};
        d.tokens = clear.tokens; d.dy = dy; d.cols = cols; d.lddy = lddy; d.vector = vector;
        d.scale = scale; d.dtable = dtable; d.ldt = lddt; d.add = accumulate != 0; d.clear = clear;
        d.across = p.across;
        NC_EMBED_TYPES(dtype, dtable_dtype, embed_direct, d, stream);
        return launch_status();
    }
    EmbedSort s = {};
    s.tokens = clear.tokens;
    s.blocks = p.sorters; s.passes = p.passes; s.bits = p.bits;
    for (int i = 0; i < 2; ++i) s.items[i] = reinterpret_cast<uint2*>(ws + p.items[i]);
    s.counts = reinterpret_cast<uint32_t*>(ws + p.counts);
    s.valid = reinterpret_cast<uint32_t*>(ws + p.valid);
    // as many rows as are cleared while the sort runs
    s.clear = clear;
    const uint64_t beside = kClearBeside / clear.row_bytes;
    if (beside < clear.end) s.clear.end = beside;
    // a block on most SMs, in clusters: not all SMs, because the chip's parts do not hold whole numbers of
    // clusters, and one that waits for another to end is late (18 clusters of 8 blocks: the last ended
    // after 25 us, the others after 13); none but the sorting one where nothing is cleared
    const int sms = device_sm_count();
    const int fit = p.sorters == 1 ? sms : (p.sorters < kSortMaxBlocks ? sms * 7 / 8 : sms * 3 / 4) / p.sorters;
    const int clusters = s.clear.end ? fit : 1;
    const int grid = (s.clear.end && clusters < 2 ? 2 : clusters) * p.sorters;
    const bool on_chip = (rows + p.sorters - 1) / p.sorters <= (uint64_t)kSortChunk;
    int smem = kSortWarps * 2 << p.bits;
    if (on_chip) smem += (p.sorters * 4 << p.bits) + (int)((rows + p.sorters - 1) / p.sorters) * 8;
    if (smem < kClearBytes) smem = kClearBytes;
    auto kernel = on_chip ? embed_sort_kernel<true> : embed_sort_kernel<false>;
    constexpr int kMost = (kSortWarps * 2 << kSortMaxBits) + (kSortMaxBlocks * 4 << kSortMaxBits) +
                          kSortChunk * 8;
    static bool allowed[2][64];
    if (!allow_dynamic_smem((const void*)kernel, kMost, allowed[on_chip])) return NC_ERR_CUDA;
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
    cudaLaunchKernelEx(&cfg, kernel, s);
    EmbedSum e = {};
    e.items = s.items[0]; e.valid = s.valid; e.across = p.across;
    e.segment = p.segment; e.segments = p.segments; e.dy = dy; e.cols = cols; e.lddy = lddy;
    e.vector = vector; e.scale = scale; e.dtable = dtable; e.ldt = lddt; e.add = accumulate != 0;
    e.parts = reinterpret_cast<float*>(ws + p.parts); e.pitch = p.pitch;
    e.clear = clear;
    e.clear.begin = s.clear.end;
    NC_EMBED_TYPES(dtype, dtable_dtype, embed_sums, e, p.segments, stream);
    return launch_status();
}

}  // extern "C"
