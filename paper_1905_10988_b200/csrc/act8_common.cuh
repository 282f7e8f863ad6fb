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
// G threads share a row, 16 values each.  Value i of thread `tid` is column
//   16 * tid + i                                rows on 16-byte boundaries: vector accesses
//   kSpread, 4-byte types: i * G + tid          any rows: neighbouring lanes, neighbouring values
//   kSpread, 2-byte types: 2 * ((i / 2) * G + tid) + i % 2    the same by pairs of values, so that
//                                               a row on a 4-byte boundary moves a pair at a time
// kRegular: rows on 32-byte boundaries, and every thread has sixteen values; no branches.
enum RowMode { kRegular = 0, kVector = 1, kSpread = 2 };

template <typename T, int MODE>
__device__ __forceinline__ uint32_t row_col(int i, int G, int tid) {
    if (MODE != kSpread) return 16u * tid + i;
    if (sizeof(T) == 4) return (uint32_t)i * G + tid;
    return 2u * ((uint32_t)(i >> 1) * G + tid) + (i & 1);
}

// values from `cols` on read as 0
template <typename T, int MODE>
__device__ __forceinline__ void row_load(const T* __restrict__ row, int G, int tid, uint32_t cols,
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
        const uint32_t* p = reinterpret_cast<const uint32_t*>(row);
        if (row_col<T, kSpread>(15, G, tid) < cols) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                r.b[i >> 3].v[i & 7] = __ldg(p + row_col<T, kSpread>(i, G, tid));
            return;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t col = row_col<T, kSpread>(i, G, tid);
            r.b[i >> 3].v[i & 7] = col < cols ? __ldg(p + col) : 0u;
        }
    } else {
        const unsigned short* p = reinterpret_cast<const unsigned short*>(row);
        const bool odd = (reinterpret_cast<uintptr_t>(row) & 2) != 0;     // the same for all lanes
        if (row_col<T, kSpread>(15, G, tid) < cols) {
            if (!odd) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    r.b[0].v[i] = __ldg(
                        reinterpret_cast<const uint32_t*>(p + row_col<T, kSpread>(2 * i, G, tid)));
            } else {
                // two words hold a pair's halves; the row's first and last value have no
                // neighbour to share a word with
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t col = row_col<T, kSpread>(2 * i, G, tid);
                    const uint32_t* q = reinterpret_cast<const uint32_t*>(p + col - 1);
                    const uint32_t lo = i > 0 || tid > 0 ? __ldg(q) : (uint32_t)__ldg(p) << 16;
                    const uint32_t hi =
                        i < 7 || col + 2 < cols ? __ldg(q + 1) : (uint32_t)__ldg(p + col + 1);
                    r.b[0].v[i] = __funnelshift_r(lo, hi, 16);
                }
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t col = row_col<T, kSpread>(2 * i, G, tid);
            uint32_t w = 0;
            if (col < cols) w = __ldg(p + col);
            if (col + 1 < cols) w |= (uint32_t)__ldg(p + col + 1) << 16;
            r.b[0].v[i] = w;
        }
    }
}

template <typename T, int MODE>
__device__ __forceinline__ void row_store(T* __restrict__ row, int G, int tid, uint32_t cols,
                                          bool wide, const float (&v)[16]) {
    if constexpr (MODE == kRegular) {
        st_raw16<T>(row + 16u * tid, pack16<T>(v), true);
    } else if constexpr (MODE == kVector) {
        const uint32_t col = 16u * tid;
        if (col + 16 <= cols)
            st_raw16<T>(row + col, pack16<T>(v), wide);
        else if (col < cols)
            st_part16<T>(row + col, v, (int)(cols - col));
    } else if constexpr (sizeof(T) == 4) {
        if (row_col<T, kSpread>(15, G, tid) < cols) {
#pragma unroll
            for (int i = 0; i < 16; ++i) row[row_col<T, kSpread>(i, G, tid)] = v[i];
            return;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t col = row_col<T, kSpread>(i, G, tid);
            if (col < cols) row[col] = v[i];
        }
    } else {
        unsigned short* p = reinterpret_cast<unsigned short*>(row);
        const bool odd = (reinterpret_cast<uintptr_t>(row) & 2) != 0;
        const bool whole = row_col<T, kSpread>(15, G, tid) < cols;
        if (whole && !odd) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                *reinterpret_cast<uint32_t*>(p + row_col<T, kSpread>(2 * i, G, tid)) =
                    pack2<T>(v[2 * i], v[2 * i + 1]);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t col = row_col<T, kSpread>(2 * i, G, tid);
            const uint32_t w = pack2<T>(v[2 * i], v[2 * i + 1]);
            if (whole || col < cols) p[col] = (unsigned short)w;
            if (whole || col + 1 < cols) p[col + 1] = (unsigned short)(w >> 16);
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

// magnitude of one value: adding 2^23 leaves rint(|x| * inverse) in the low bits.  Random
// rounding keeps eight more bits, adds the draw to them and drops them: up with probability
// (their value) / 256, so the expectation is |x| rounded to 1/256 unit.
__device__ __forceinline__ uint32_t act8_one(float x, float inverse, bool random, uint32_t draw) {
    const uint32_t f = __float_as_uint(fmaf(fabsf(x), inverse, 8388608.0f));
    const uint32_t m = random ? ((f & 0xFFFFu) + draw) >> 8 : f & 0x7Fu;
    return m | ((__float_as_uint(x) >> 24) & 0x80u);
}

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

// codes of sixteen neighbouring values, one half of the block whose scale byte is `scale`;
// `q` is the index of these sixteen codes in the code plane, which is also their generator block
template <bool RANDOM>
__device__ __forceinline__ uint4 act8_sixteen(const float (&v)[16], uint32_t scale, uint64_t q,
                                              uint32_t worker, const PhiloxKeys& keys) {
    if (scale == kAct8Nan) return make_uint4(0u, 0u, 0u, 0u);
    const float inverse = act8_inverse(scale, RANDOM);
    uint32_t r[4] = {0u, 0u, 0u, 0u};
    if (RANDOM) stream_words4(q, worker, kDomainAct8, keys, r);
    return make_uint4(act8_four<RANDOM>(v, inverse, r[0]), act8_four<RANDOM>(v + 4, inverse, r[1]),
                      act8_four<RANDOM>(v + 8, inverse, r[2]),
                      act8_four<RANDOM>(v + 12, inverse, r[3]));
}

// Codes of a thread's spread values (row_col<T, kSpread>).  `plane`: place of the row's first code,
// `first` = tid - lane, `pitch`: codes of the row.  A step of the warp covers one block (4-byte
// types) or two, of 16 lanes each.  The warp's 32 generator blocks of 16 draws are computed one
// a lane.
template <typename T, bool RANDOM>
__device__ __forceinline__ void act8_encode_spread(const float (&v)[16], uint64_t plane,
                                                   uint32_t pitch, int G, int first,
                                                   uint32_t worker, const PhiloxKeys& keys,
                                                   uint8_t* __restrict__ codes,
                                                   uint8_t* __restrict__ scales) {
    constexpr int PER = sizeof(T) == 4 ? 1 : 2;      // values of a lane in a step
    const int lane = threadIdx.x & 31;
    uint32_t r[4] = {0u, 0u, 0u, 0u};
    if (RANDOM) {
        const int step = lane / (2 * PER), part = lane % (2 * PER);
        const uint32_t col = row_col<T, kSpread>(step * PER, G, first) + 16 * part;
        stream_words4((plane + col) >> 4, worker, kDomainAct8, keys, r);
    }
#pragma unroll
    for (int s = 0; s < 16 / PER; ++s) {
        const uint32_t begin = row_col<T, kSpread>(s * PER, G, first);
        uint32_t top;
        if (PER == 1) {
            top = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v[s]) & 0x7FFFFFFFu);
        } else {
            const float m = max3_abs(v[PER * s], v[PER * s + PER - 1], 0.0f);
            top = __float_as_uint(m);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        }
        const uint32_t scale = act8_scale(top);
        uint32_t word = 0;
        if (RANDOM) {          // the lane's draws: bytes of word (column / 4) mod 4 of its chunk
            const int source = s * 2 * PER + lane * PER / 16, which = (lane * PER >> 2) & 3;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t t = __shfl_sync(0xFFFFFFFFu, r[k], source);
                if (which == k) word = t;
            }
            word >>= 8 * (lane * PER & 3);
        }
        const uint32_t col = begin + lane * PER;
        if (col < pitch) {
            const float inverse = act8_inverse(scale, RANDOM);
            uint32_t code = 0;
            if (scale != kAct8Nan) {
                code = act8_one(v[PER * s], inverse, RANDOM, word & 0xFFu);
                if (PER == 2)
                    code |= act8_one(v[PER * s + PER - 1], inverse, RANDOM, (word >> 8) & 0xFFu)
                            << 8;
            }
            if (PER == 1)
                codes[plane + col] = (uint8_t)code;
            else
                *reinterpret_cast<unsigned short*>(codes + plane + col) = (unsigned short)code;
            if ((col & 31) == 0) scales[(plane + col) >> 5] = (uint8_t)scale;
        }
    }
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

// a thread's spread values of a row of codes; those from `cols` on are 0
template <typename T>
__device__ __forceinline__ void act8_decode_spread(const uint8_t* __restrict__ codes,
                                                   const uint8_t* __restrict__ scales,
                                                   uint64_t plane, int G, int tid, uint32_t cols,
                                                   float (&v)[16]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t col = row_col<T, kSpread>(i, G, tid);
            v[i] = col < cols ? act8_value(__ldg(codes + plane + col),
                                           __ldg(scales + ((plane + col) >> 5)))
                              : 0.0f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t col = row_col<T, kSpread>(2 * i, G, tid);
            v[2 * i] = v[2 * i + 1] = 0.0f;
            if (col < cols) {
                const uint32_t c =
                    __ldg(reinterpret_cast<const unsigned short*>(codes + plane + col));
                const uint32_t scale = __ldg(scales + ((plane + col) >> 5));
                if (scale <= kAct8MaxFast) {
                    unpack2<__nv_bfloat16>(act8_pair_bf16(c, 0, act8_fields(scale)), v[2 * i],
                                           v[2 * i + 1]);
                } else {
                    v[2 * i] = act8_value(c & 0xFFu, scale);
                    v[2 * i + 1] = act8_value(c >> 8, scale);
                }
                if (col + 1 >= cols) v[2 * i + 1] = 0.0f;
            }
        }
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
