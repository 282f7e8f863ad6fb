// 8-bit activation checkpoints (act8_common.cuh): compression and decompression, for sm_100a.
//
// Bound by memory: 2 + 33/32 bytes per bfloat16 value in either direction.  A thread takes 16
// neighbouring values, half a block: two lanes agree on the block's largest magnitude with one
// shuffle, a 16-byte store takes the codes, and one generator block serves the 16 draws of random
// rounding.  Rows that are not 16-byte aligned are spread over the lanes, an element or a pair of
// two-byte elements an access, and a warp puts them in order in shared memory.
//
// bfloat16 16384 x 4096: nearest 33 us (6.2 TB/s), read back 31 us (6.6 TB/s, a copy's rate), random
// rounding 43 us: 221 instructions for a warp's 512 values, integer pipe and issue slots at 64 % each,
// memory at 47 %, because a thread's loads, generator block and stores follow each other.  binary32
// 4097 x 1001 there and back: 14 us, of two launches, issue-bound.
#include "act8_common.cuh"

namespace natcomp {

struct Act8Rows {
    uint64_t rows, cols, ld;      // of the matrix, in elements
    uint32_t per_row;             // 16-value chunks of a row of the code plane
    uint64_t total;               // chunks of the plane
    int access;                   // RowAccess of the matrix
};

template <typename T, bool RANDOM>
__global__ void __launch_bounds__(kBlockThreads)
act8_compress_kernel(const T* __restrict__ x, const Act8Rows g, const uint32_t worker,
                     uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                     const __grid_constant__ PhiloxKeys keys) {
    const uint64_t i = (uint64_t)blockIdx.x * kBlockThreads + threadIdx.x;
    const bool live = i < g.total;
    Raw16<T> r = {};
    if (live) {
        const uint32_t row = g.rows == 1 ? 0u : (uint32_t)i / g.per_row;
        const uint64_t col = 16ull * ((uint32_t)i - row * g.per_row);
        const T* p = x + row * g.ld + col;
        if (col + 16 <= g.cols)
            r = ld_raw16<T>(p, g.access == kRowWide);
        else if (col < g.cols)
            r = ld_raw16_part<T>(p, (int)(g.cols - col));
    }
    const uint4 draws = act8_draws<RANDOM>((uint32_t)i, worker, keys);   // while the values arrive
    float v[16];
    unpack16<T>(r, v);
    uint32_t top = max_bits16(v);
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    const uint32_t scale = act8_scale(top);
    if (!live) return;
    __stcs(reinterpret_cast<uint4*>(codes) + i, act8_sixteen<RANDOM>(v, scale, draws));
    if (!(i & 1)) scales[i >> 1] = (uint8_t)scale;
}

// rows at any element: a warp takes 512 neighbouring values of a row
template <typename T, bool RANDOM>
__global__ void __launch_bounds__(kBlockThreads)
act8_compress_spread_kernel(const T* __restrict__ x, const Act8Rows g, const uint32_t worker,
                            uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                            const __grid_constant__ PhiloxKeys keys) {
    __shared__ __align__(16) uint32_t scratch[kWarpsPerBlock][kSpreadWords<T>];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t segments = (g.per_row + 31) / 32;
    const uint32_t w = blockIdx.x * kWarpsPerBlock + warp;
    const uint32_t row = w / segments;
    if (row >= g.rows) return;
    const uint32_t segment = w - row * segments;
    const uint64_t first = 512ull * segment;
    Raw16<T> r;
    float v[16];
    row_load<T, kSpread>(x + row * g.ld + first, lane,
                         g.cols > first ? (uint32_t)min(g.cols - first, (uint64_t)1024) : 0u, false,
                         r);
    row_arrange<T, kSpread>(r, scratch[warp]);
    unpack16<T>(r, v);
    uint32_t top = max_bits16(v);
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    const uint32_t scale = act8_scale(top), chunk = 32 * segment + lane;
    if (chunk >= g.per_row) return;
    const uint64_t i = (uint64_t)row * g.per_row + chunk;
    __stcs(reinterpret_cast<uint4*>(codes) + i,
           act8_sixteen<RANDOM>(v, scale, act8_draws<RANDOM>((uint32_t)i, worker, keys)));
    if (!(i & 1)) scales[i >> 1] = (uint8_t)scale;
}

template <typename T>
__global__ void __launch_bounds__(kBlockThreads)
act8_decompress_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                       const Act8Rows g, T* __restrict__ out) {
    const uint64_t i = (uint64_t)blockIdx.x * kBlockThreads + threadIdx.x;
    if (i >= g.total) return;
    const uint32_t row = g.rows == 1 ? 0u : (uint32_t)i / g.per_row;
    const uint64_t col = 16ull * ((uint32_t)i - row * g.per_row);
    if (col >= g.cols) return;
    float v[16];
    act8_decode16(ld_stream_u4(codes + 16 * i), __ldg(scales + (i >> 1)), v);
    T* p = out + row * g.ld + col;
    if (col + 16 <= g.cols)
        st_raw16<T>(p, pack16<T>(v), g.access == kRowWide);
    else
        st_part16<T>(p, v, (int)(g.cols - col));
}

template <typename T>
__global__ void __launch_bounds__(kBlockThreads)
act8_decompress_spread_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                              const Act8Rows g, T* __restrict__ out) {
    __shared__ __align__(16) uint32_t scratch[kWarpsPerBlock][kSpreadWords<T>];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t segments = (g.per_row + 31) / 32;
    const uint32_t w = blockIdx.x * kWarpsPerBlock + warp;
    const uint32_t row = w / segments;
    if (row >= g.rows) return;
    const uint32_t segment = w - row * segments, chunk = 32 * segment + lane;
    const uint64_t first = 512ull * segment, i = (uint64_t)row * g.per_row + chunk;
    if (first >= g.cols) return;
    float v[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = 0.0f;
    if (chunk < g.per_row)
        act8_decode16(ld_stream_u4(codes + 16 * i), __ldg(scales + (i >> 1)), v);
    row_store<T, kSpread>(out + row * g.ld + first, lane,
                          (uint32_t)min(g.cols - first, (uint64_t)1024), false, v, scratch[warp]);
}

// the plane of a matrix: one long row where the matrix has no gaps and whole blocks
static Act8Rows act8_rows(size_t rows, size_t cols, size_t ld, const void* p, int bytes) {
    Act8Rows g;
    g.access = row_access(p, ld, bytes, rows);
    g.total = rows * (act8_pitch(cols) / 16);
    if (cols % 32 == 0 && ld == cols) {
        cols *= rows;
        ld = cols;
        rows = 1;
    }
    g.rows = rows;
    g.cols = cols;
    g.ld = ld;
    g.per_row = (uint32_t)(act8_pitch(cols) / 16);
    return g;
}

static unsigned act8_grid(const Act8Rows& g) {
    if (g.access != kRowElement) return (unsigned)((g.total + kBlockThreads - 1) / kBlockThreads);
    const uint64_t warps = g.rows * ((g.per_row + 31) / 32);
    return (unsigned)((warps + kWarpsPerBlock - 1) / kWarpsPerBlock);
}

template <typename T>
static void act8_compress_launch(const void* x, const Act8Rows& g, bool random, uint64_t seed,
                                 uint32_t worker, uint8_t* codes, uint8_t* scales,
                                 cudaStream_t stream) {
    const PhiloxKeys keys = make_philox_keys(seed);
    auto kernel = g.access == kRowElement
                      ? (random ? act8_compress_spread_kernel<T, true>
                                : act8_compress_spread_kernel<T, false>)
                      : (random ? act8_compress_kernel<T, true> : act8_compress_kernel<T, false>);
    kernel<<<act8_grid(g), kBlockThreads, 0, stream>>>(static_cast<const T*>(x), g, worker, codes,
                                                       scales, keys);
}

template <typename T>
static void act8_decompress_launch(const uint8_t* codes, const uint8_t* scales, const Act8Rows& g,
                                   void* out, cudaStream_t stream) {
    auto kernel = g.access == kRowElement ? act8_decompress_spread_kernel<T>
                                          : act8_decompress_kernel<T>;
    kernel<<<act8_grid(g), kBlockThreads, 0, stream>>>(codes, scales, g, static_cast<T*>(out));
}

}  // namespace natcomp

using namespace natcomp;

extern "C" {

size_t nc_act8_code_bytes(size_t rows, size_t cols) { return rows * act8_pitch(cols); }

size_t nc_act8_scale_bytes(size_t rows, size_t cols) {
    return round_up16(rows * (act8_pitch(cols) / 32));
}

nc_status nc_act8_compress(const void* x, int dtype, size_t rows, size_t cols, size_t ldx,
                           int rounding, uint64_t seed, uint32_t worker, uint8_t* codes,
                           uint8_t* scales, cudaStream_t stream) {
    const int bytes = act8_type_bytes(dtype);
    if (!bytes) return NC_ERR_UNSUPPORTED;
    if (rounding != NC_ROUND_NEAREST && rounding != NC_ROUND_RANDOM) return NC_ERR_INVALID;
    if (rows == 0 || cols == 0) return NC_OK;
    if (!x || !codes || !scales || ldx < cols) return NC_ERR_INVALID;
    if (!act8_fits(rows, cols)) return NC_ERR_TOO_LARGE;
    if (!element_aligned(x, bytes) || !aligned16(codes) || !aligned16(scales)) return NC_ERR_ALIGN;
    const Act8Rows g = act8_rows(rows, cols, ldx, x, bytes);
    const bool random = rounding == NC_ROUND_RANDOM;
    if (dtype == NC_DTYPE_F32)
        act8_compress_launch<float>(x, g, random, seed, worker, codes, scales, stream);
    else if (dtype == NC_DTYPE_BF16)
        act8_compress_launch<__nv_bfloat16>(x, g, random, seed, worker, codes, scales, stream);
    else
        act8_compress_launch<__half>(x, g, random, seed, worker, codes, scales, stream);
    return launch_status();
}

nc_status nc_act8_decompress(const uint8_t* codes, const uint8_t* scales, size_t rows, size_t cols,
                             void* out, int dtype, size_t ldo, cudaStream_t stream) {
    const int bytes = act8_type_bytes(dtype);
    if (!bytes) return NC_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return NC_OK;
    if (!out || !codes || !scales || ldo < cols) return NC_ERR_INVALID;
    if (!act8_fits(rows, cols)) return NC_ERR_TOO_LARGE;
    if (!element_aligned(out, bytes) || !aligned16(codes) || !aligned16(scales))
        return NC_ERR_ALIGN;
    const Act8Rows g = act8_rows(rows, cols, ldo, out, bytes);
    if (dtype == NC_DTYPE_F32)
        act8_decompress_launch<float>(codes, scales, g, out, stream);
    else if (dtype == NC_DTYPE_BF16)
        act8_decompress_launch<__nv_bfloat16>(codes, scales, g, out, stream);
    else
        act8_decompress_launch<__half>(codes, scales, g, out, stream);
    return launch_status();
}

}  // extern "C"
