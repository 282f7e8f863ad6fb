// 8-bit activation checkpoints: the code, its encoder and decoder, and the row accesses that the
// checkpoint, layer-norm and weight-gradient kernels share.
//
// A row is cut into blocks of 32 values.  A block has one unit 2^e, the smallest power of two (at
// least 2^-118) with max|x| <= 127 * 2^e, stored as the byte e + 127, and each value a code byte
// (sign << 7) | magnitude that stands for +-magnitude * 2^e.  A power-of-two unit makes the
// scaling exact, so a code depends on the value and its block's largest magnitude alone, not on
// an order of operations; and magnitude * 2^e has at most 7 significant bits, so the decoded
// value is exact in bfloat16 and the matrix instructions read the very number the checkpoint
// holds.  A block with an inf or a NaN gets the byte 255 and decodes to NaN.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "philox.cuh"

namespace natcomp {

constexpr uint32_t kDomainAct8 = 6u;
constexpr uint32_t kAct8Nan = 255u;        // scale byte of a block that is not finite
constexpr uint32_t kAct8MinScale = 9u;     // e = -118: 2^(8 - e), the finest multiplier, is finite
constexpr uint32_t kAct8MaxFast = 247u;    // up to here (128 + m) * 2^e is finite in bfloat16

constexpr uint64_t kAct8MaxCodes = ((uint64_t)1 << 36) - 32;  // of one call: 32-bit chunk index

__host__ __device__ inline uint64_t act8_pitch(uint64_t cols) { return (cols + 31) & ~(uint64_t)31; }

// ---- values in memory ------------------------------------------------------------------------

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) {
    return __bfloat162float(v);
}
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) {
    return __float2bfloat16_rn(v);
}
template <> __device__ __forceinline__ __half from_f32<__half>(float v) {
    return __float2half_rn(v);
}

template <typename T> __device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b);
template <> __device__ __forceinline__ void unpack2<__nv_bfloat16>(uint32_t w, float& a, float& b) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
}
template <> __device__ __forceinline__ void unpack2<__half>(uint32_t w, float& a, float& b) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x;
    b = f.y;
}

template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// 32 bytes of global memory.  `wide`: the address is a multiple of 32, else of 16.
struct Bytes32 {
    uint32_t v[8];
};

__device__ __forceinline__ Bytes32 ld_bytes32(const void* p, bool wide) {
    Bytes32 r;
    if (wide) {
        asm volatile("ld.global.cs.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r.v[0]), "=r"(r.v[1]), "=r"(r.v[2]), "=r"(r.v[3]), "=r"(r.v[4]),
                       "=r"(r.v[5]), "=r"(r.v[6]), "=r"(r.v[7])
                     : "l"(p));
    } else {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
        const uint4 b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
        r.v[0] = a.x; r.v[1] = a.y; r.v[2] = a.z; r.v[3] = a.w;
        r.v[4] = b.x; r.v[5] = b.y; r.v[6] = b.z; r.v[7] = b.w;
    }
    return r;
}

__device__ __forceinline__ void st_bytes32(void* p, const Bytes32& r, bool wide) {
    if (wide) {
        asm volatile("st.global.cs.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r.v[0]),
                     "r"(r.v[1]), "r"(r.v[2]), "r"(r.v[3]), "r"(r.v[4]), "r"(r.v[5]),
                     "r"(r.v[6]), "r"(r.v[7])
                     : "memory");
    } else {
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(r.v[0], r.v[1], r.v[2], r.v[3]));
        __stcs(reinterpret_cast<uint4*>(p) + 1, make_uint4(r.v[4], r.v[5], r.v[6], r.v[7]));
    }
}

// sixteen values as they lie in memory
template <typename T> struct Raw16 {
    Bytes32 b[sizeof(T) / 2];
};

template <typename T>
__device__ __forceinline__ Raw16<T> ld_raw16(const T* p, bool wide) {
    Raw16<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
        r.b[i] = ld_bytes32(reinterpret_cast<const char*>(p) + 32 * i, wide);
    return r;
}

// the first `count` (< 16) of sixteen values one at a time, the rest 0
template <typename T>
__device__ __forceinline__ Raw16<T> ld_raw16_part(const T* p, int count) {
    Raw16<T> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            r.b[i >> 3].v[i & 7] = i < count ? __ldg(reinterpret_cast<const uint32_t*>(p) + i) : 0u;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned short* h = reinterpret_cast<const unsigned short*>(p) + 2 * i;
            const uint32_t a = 2 * i < count ? __ldg(h) : 0u;
            const uint32_t b = 2 * i + 1 < count ? __ldg(h + 1) : 0u;
            r.b[0].v[i] = a | (b << 16);
        }
    }
    return r;
}

template <typename T>
__device__ __forceinline__ void unpack16(const Raw16<T>& r, float (&v)[16]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r.b[i >> 3].v[i & 7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) unpack2<T>(r.b[0].v[i], v[2 * i], v[2 * i + 1]);
    }
}

template <typename T>
__device__ __forceinline__ Raw16<T> pack16(const float (&v)[16]) {
    Raw16<T> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 16; ++i) r.b[i >> 3].v[i & 7] = __float_as_uint(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.b[0].v[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
    }
    return r;
}

template <typename T>
__device__ __forceinline__ void st_raw16(T* p, const Raw16<T>& r, bool wide) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
        st_bytes32(reinterpret_cast<char*>(p) + 32 * i, r.b[i], wide);
}

template <typename T>
__device__ __forceinline__ void st_part16(T* p, const float (&v)[16], int count) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < count) p[i] = from_f32<T>(v[i]);
}

// ---- pairs of binary32 values: one instruction for two additions, products or both --------------
typedef unsigned long long f32x2;

__device__ __forceinline__ f32x2 pair_of(float lo, float hi) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void of_pair(f32x2 v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

template <typename T>
__device__ __forceinline__ void unpack16(const Raw16<T>& r, f32x2 (&v)[8]) {
    float f[16];
    unpack16<T>(r, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = pair_of(f[2 * i], f[2 * i + 1]);
}

// ---- a thread's sixteen values of a row ---------------------------------------------------------
// Threads share a row, 16 neighbouring values each: thread `tid` has the columns from 16 * tid on.
//   kRegular  rows on 32-byte boundaries, and every thread has sixteen values: no branches
//   kVector   rows on 16-byte boundaries: vector accesses
//   kSpread   rows at any element: neighbouring lanes access neighbouring values (pairs of two-byte
//             ones), and a warp's 512 values change places in shared memory afterwards or before
enum RowMode { kRegular = 0, kVector = 1, kSpread = 2 };

// the warp's i-th spread access: which of its 512 columns lane `lane` has (2-byte types: the first
// of a pair)
template <typename T>
__device__ __forceinline__ uint32_t spread_col(int i, int lane) {
    return sizeof(T) == 4 ? 32u * i + lane : 64u * i + 2 * lane;
}

// where that word lies in shared memory: sixteen values of a lane follow each other, and the lanes
// are four words further apart, so that a lane reads its values by 16 bytes
template <typename T> constexpr int kSpreadPitch = sizeof(T) == 4 ? 20 : 12;
template <typename T> constexpr int kSpreadWords = 32 * kSpreadPitch<T>;      // of a warp

template <typename T>
__device__ __forceinline__ uint32_t spread_place(int i, int lane) {
    return sizeof(T) == 4 ? (2 * i + (lane >> 4)) * 20 + (lane & 15)
                          : (4 * i + (lane >> 3)) * 12 + (lane & 7);
}

// values from `cols` on read as 0; kSpread: still spread, row_arrange() follows
template <typename T, int MODE>
__device__ __forceinline__ void row_load(const T* __restrict__ row, int tid, uint32_t cols,
                                         bool wide, Raw16<T>& r) {
    if constexpr (MODE == kRegular) {
        r = ld_raw16<T>(row + 16u * tid, true);
    } else if constexpr (MODE == kVector) {
        const uint32_t col = 16u * tid;
        if (col + 16 <= cols)
            r = ld_raw16<T>(row + col, wide);
        else
            r = ld_raw16_part<T>(row + col, col < cols ? (int)(cols - col) : 0);
    } else if constexpr (sizeof(T) == 4) {
        const uint32_t first = 16u * (tid & ~31);
        const uint32_t* p = reinterpret_cast<const uint32_t*>(row) + first;
        const int lane = tid & 31;
        if (first + 512 <= cols) {
#pragma unroll
            for (int i = 0; i < 16; ++i) r.b[i >> 3].v[i & 7] = __ldg(p + spread_col<T>(i, lane));
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                r.b[i >> 3].v[i & 7] =
                    first + spread_col<T>(i, lane) < cols ? __ldg(p + spread_col<T>(i, lane)) : 0u;
        }
    } else {
        const uint32_t first = 16u * (tid & ~31);
        const unsigned short* p = reinterpret_cast<const unsigned short*>(row) + first;
        const int lane = tid & 31;
        const bool odd = (reinterpret_cast<uintptr_t>(row) & 2) != 0;
        if (!odd && first + 512 <= cols) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                r.b[0].v[i] = __ldg(reinterpret_cast<const uint32_t*>(p + spread_col<T>(i, lane)));
        } else if (odd && first + 512 < cols) {
            // two words hold a pair's halves; the row's first value has no neighbour to share one
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t* q =
                    reinterpret_cast<const uint32_t*>(p + (int)spread_col<T>(i, lane) - 1);
                const uint32_t lo = i > 0 || tid > 0 ? __ldg(q) : (uint32_t)__ldg(p) << 16;
                r.b[0].v[i] = __funnelshift_r(lo, __ldg(q + 1), 16);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t c = spread_col<T>(i, lane);
                uint32_t w = 0;
                if (first + c < cols) w = __ldg(p + c);
                if (first + c + 1 < cols) w |= (uint32_t)__ldg(p + c + 1) << 16;
                r.b[0].v[i] = w;
            }
        }
    }
}

// kSpread: the lanes' words change places; `scratch` is the warp's own, kSpreadWords<T> words on a
// 16-byte boundary
template <typename T, int MODE>
__device__ __forceinline__ void row_arrange(Raw16<T>& r, uint32_t* scratch) {
    if constexpr (MODE == kSpread) {
        const int lane = threadIdx.x & 31;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) * 4; ++i)
            scratch[spread_place<T>(i, lane)] = r.b[i >> 3].v[i & 7];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) {
            const uint4 q = reinterpret_cast<const uint4*>(scratch + lane * kSpreadPitch<T>)[i];
            uint32_t* v = r.b[i >> 1].v + 4 * (i & 1);
            v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
        }
    }
}

template <typename T, int MODE>
__device__ __forceinline__ void row_store(T* __restrict__ row, int tid, uint32_t cols, bool wide,
                                          const float (&v)[16], uint32_t* scratch) {
    if constexpr (MODE == kRegular) {
        st_raw16<T>(row + 16u * tid, pack16<T>(v), true);
    } else if constexpr (MODE == kVector) {
        const uint32_t col = 16u * tid;
        if (col + 16 <= cols)
            st_raw16<T>(row + col, pack16<T>(v), wide);
        else if (col < cols)
            st_part16<T>(row + col, v, (int)(cols - col));
    } else {
        const int lane = tid & 31;
        const uint32_t first = 16u * (tid & ~31);
        const Raw16<T> r = pack16<T>(v);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) {
            const uint32_t* w = r.b[i >> 1].v + 4 * (i & 1);
            reinterpret_cast<uint4*>(scratch + lane * kSpreadPitch<T>)[i] =
                make_uint4(w[0], w[1], w[2], w[3]);
        }
        __syncwarp();
        if constexpr (sizeof(T) == 4) {
            uint32_t* p = reinterpret_cast<uint32_t*>(row) + first;
            const bool whole = first + 512 <= cols;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t c = spread_col<T>(i, lane), w = scratch[spread_place<T>(i, lane)];
                if (whole || first + c < cols) p[c] = w;
            }
        } else {
            unsigned short* p = reinterpret_cast<unsigned short*>(row) + first;
            const bool odd = (reinterpret_cast<uintptr_t>(row) & 2) != 0;
            const bool whole = first + 512 <= cols;
            if (whole && !odd) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<uint32_t*>(p + spread_col<T>(i, lane)) =
                        scratch[spread_place<T>(i, lane)];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t c = spread_col<T>(i, lane);
                    const uint32_t w = scratch[spread_place<T>(i, lane)];
                    if (whole || first + c < cols) p[c] = (unsigned short)w;
                    if (whole || first + c + 1 < cols) p[c + 1] = (unsigned short)(w >> 16);
                }
            }
        }
    }
}

// ---- encoder ---------------------------------------------------------------------------------

// scale byte of a block from the largest |x| bit pattern.  The patterns order as the magnitudes
// do, and the exponent field of max|x| * (2 / (127 / 64)) rounded down is reached by an integer
// addition: a mantissa above 127/64 (field 0x7E0000) carries into the exponent.
__device__ __forceinline__ uint32_t act8_scale(uint32_t max_bits) {
    if (max_bits >= 0x7F800000u) return kAct8Nan;
    const int s = (int)((max_bits + 0x1FFFFu) >> 23) - 6;
    return s < (int)kAct8MinScale ? kAct8MinScale : (uint32_t)s;
}

// 1 / unit and 256 / unit (a block that is not finite is not scaled: its codes are 0)
__device__ __forceinline__ float act8_inverse(uint32_t scale, bool random) {
    return __uint_as_float(((random ? 262u : 254u) - (scale == kAct8Nan ? 128u : scale)) << 23);
}

// Magnitudes: adding 2^23 leaves rint(|x| * inverse) in the low bits.  Random rounding keeps eight
// more bits, adds the draw to them and drops them: up with probability (their value) / 256, so the
// expectation is |x| rounded to 1/256 unit.
// codes of four neighbouring values; `draws`: their four stream bytes
template <bool RANDOM>
__device__ __forceinline__ uint32_t act8_four(const float* x, float inverse, uint32_t draws) {
    uint32_t f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __float_as_uint(fmaf(fabsf(x[i]), inverse, 8388608.0f));
    uint32_t m;
    if (RANDOM) {      // two 16-bit sums per word: at most 127 * 256 + 255, no carry between them
        const uint32_t lo = __byte_perm(f[0], f[1], 0x5410) + __byte_perm(draws, 0u, 0x4140);
        const uint32_t hi = __byte_perm(f[2], f[3], 0x5410) + __byte_perm(draws, 0u, 0x4342);
        m = __byte_perm(lo, hi, 0x7531);
    } else {
        m = __byte_perm(__byte_perm(f[0], f[1], 0x0040), __byte_perm(f[2], f[3], 0x0040), 0x5410);
    }
    const uint32_t s = __byte_perm(
        __byte_perm(__float_as_uint(x[0]), __float_as_uint(x[1]), 0x0073),
        __byte_perm(__float_as_uint(x[2]), __float_as_uint(x[3]), 0x0073), 0x5410);
    return (m & 0x7F7F7F7Fu) | (s & 0x80808080u);
}

// the largest magnitude of three, NaN if one of them is
__device__ __forceinline__ float max3_abs(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
    return r;
}

__device__ __forceinline__ uint32_t max_bits16(const float (&v)[16]) {
    float a = max3_abs(v[0], v[1], v[2]);
#pragma unroll
    for (int i = 3; i < 15; i += 2) a = max3_abs(a, v[i], v[i + 1]);
    return __float_as_uint(max3_abs(a, v[15], v[15]));
}

// the sixteen stream bytes of the sixteen codes with index q of the code plane, q < 2^32
template <bool RANDOM>
__device__ __forceinline__ uint4 act8_draws(uint32_t q, uint32_t worker, const PhiloxKeys& keys) {
    uint32_t r[4] = {0u, 0u, 0u, 0u};
    if (RANDOM) philox4x32_10(q, 0u, worker, kDomainAct8, keys, r);
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// codes of sixteen neighbouring values, one half of the block whose scale byte is `scale`
template <bool RANDOM>
__device__ __forceinline__ uint4 act8_sixteen(const float (&v)[16], uint32_t scale,
                                              const uint4& draws) {
    if (scale == kAct8Nan) return make_uint4(0u, 0u, 0u, 0u);
    const float inverse = act8_inverse(scale, RANDOM);
    return make_uint4(act8_four<RANDOM>(v, inverse, draws.x),
                      act8_four<RANDOM>(v + 4, inverse, draws.y),
                      act8_four<RANDOM>(v + 8, inverse, draws.z),
                      act8_four<RANDOM>(v + 12, inverse, draws.w));
}

// ---- decoder ---------------------------------------------------------------------------------

// any scale byte, one code at a time
__device__ __forceinline__ float act8_value(uint32_t code, uint32_t scale) {
    if (scale == kAct8Nan) return __uint_as_float(0x7FC00000u);
    const float unit = __uint_as_float(scale ? scale << 23 : 0x00400000u);
    const float v = (float)(code & 0x7Fu) * unit;
    return (code & 0x80u) ? -v : v;
}

// two neighbouring codes (bytes 2h and 2h + 1 of w) as a pair of bfloat16.  With the magnitude m
// in the mantissa field and the exponent field of 128 * 2^e, a word reads +-(128 + m) * 2^e; the
// same word without m reads +-128 * 2^e; their difference +-m * 2^e is exact.
// fields = (scale + 7) << 7 in both halves, scale <= kAct8MaxFast.
__device__ __forceinline__ uint32_t act8_pair_bf16(uint32_t w, int h, uint32_t fields) {
    const uint32_t d = __byte_perm(w, 0u, h ? 0x3322 : 0x1100);      // each code in both bytes
    const uint32_t a = (d & 0x807F807Fu) | fields;
    const uint32_t b = (d & 0x80008000u) | fields;
    uint32_t v;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(v) : "r"(a), "r"(b));
    return v;
}

__device__ __forceinline__ uint32_t act8_fields(uint32_t scale) {
    return ((scale + 7u) << 7) * 0x00010001u;
}

__device__ __forceinline__ void act8_decode16(const uint4& c, uint32_t scale, float (&v)[16]) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    if (scale <= kAct8MaxFast) {
        const uint32_t fields = act8_fields(scale);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            unpack2<__nv_bfloat16>(act8_pair_bf16(w[i >> 1], i & 1, fields), v[2 * i],
                                   v[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = act8_value(w[i >> 2] >> (8 * (i & 3)) & 0xFFu, scale);
    }
}

// ---- arguments -------------------------------------------------------------------------------

inline int act8_type_bytes(int dtype) {
    return dtype == NC_DTYPE_F32 ? 4 : dtype == NC_DTYPE_BF16 || dtype == NC_DTYPE_F16 ? 2 : 0;
}

// rows * pitch codes fit the 32-bit chunk index of one call
inline bool act8_fits(size_t rows, size_t cols) {
    if (cols > kAct8MaxCodes || rows > kAct8MaxCodes) return false;
    const uint64_t pitch = act8_pitch(cols);
    return pitch == 0 || rows <= kAct8MaxCodes / pitch;
}

// how the rows of a matrix may be accessed: every row starts on a multiple of 32 bytes, of 16
// bytes, or of one element only
enum RowAccess { kRowWide = 0, kRow16 = 1, kRowElement = 2 };

inline RowAccess row_access(const void* p, size_t ld, int bytes, size_t rows) {
    const uintptr_t a = (uintptr_t)p | (rows > 1 ? (uintptr_t)(ld * bytes) : 0);
    return (a & 31) == 0 ? kRowWide : (a & 15) == 0 ? kRow16 : kRowElement;
}

inline bool element_aligned(const void* p, int bytes) { return ((uintptr_t)p % bytes) == 0; }

}  // namespace natcomp
