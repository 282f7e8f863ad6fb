// What product.cuh and the kernels on it call beyond model.hpp: pairs' copies of boxes, reads of TMEM by
// 32 columns, matrix instructions of both types and layouts, votes and atomics.  (Spliced
// into the translated text after act8_common.cuh and tensor_core.cuh: no includes.)

inline int __ffs(uint32_t v) { return __builtin_ffs((int)v); }
inline int __popc(uint32_t v) { return __builtin_popcount(v); }
inline uint32_t __ballot_sync(uint32_t, int p) {
    const uint64_t* s = model::exchange(p != 0);
    uint32_t mask = 0;
    for (int i = 0; i < 32; ++i) mask |= (uint32_t)(s[i] != 0) << i;
    return mask;
}
inline uint32_t __match_any_sync(uint32_t, uint32_t v) {
    const uint64_t* s = model::exchange(v);
    uint32_t mask = 0;
    for (int i = 0; i < 32; ++i) mask |= (uint32_t)(s[i] == v) << i;
    return mask;
}
inline int __syncthreads_or(int p) {
    static int any;                      // (blocks of a cluster come here one by one)
    __syncthreads();
    any = 0;
    __syncthreads();
    any |= p;
    __syncthreads();
    const int r = any;
    __syncthreads();
    return r;
}
inline int __syncthreads_count(int p) {
    static int sum;
    __syncthreads();
    sum = 0;
    __syncthreads();
    sum += p != 0;
    __syncthreads();
    const int r = sum;
    __syncthreads();
    return r;
}
inline uint32_t atomicAdd(uint32_t* p, uint32_t v) {
    const uint32_t old = *p;
    *p += v;
    return old;
}
inline uint32_t atomicOr(uint32_t* p, uint32_t v) {
    const uint32_t old = *p;
    *p |= v;
    return old;
}
inline cudaError_t cudaMemset2DAsync_model(void* p, size_t pitch, int v, size_t width, size_t height) {
    for (size_t r = 0; r < height; ++r) memset((char*)p + r * pitch, v, width);
    return cudaSuccess;
}
#define cudaMemset2DAsync(p, pitch, v, w, h, s) cudaMemset2DAsync_model(p, pitch, v, w, h)

namespace natcomp {

// of a map of boxes: how many matrices, and how far apart in bytes
inline std::map<const void*, std::pair<uint64_t, uint64_t>> model_matrices;

inline bool make_box_map(CUtensorMap* map, const void* p, bool, uint64_t count, uint64_t rows,
                         uint64_t cols, uint64_t ld, uint64_t distance) {
    if ((uintptr_t)p % 16 || ld % 8 || (count > 1 && distance % 8)) return false;
    *map = {(const uint8_t*)p, rows, cols, 2 * ld, 64, 64, 2};
    model_matrices[p] = {count, 2 * distance};
    return true;
}

inline void tma_load_pair(uint32_t dst, const CUtensorMap* m, int x, int y, int z, uint32_t bar) {
    if (x % 8) model::fail("tensor copy at an x that is not aligned");
    if (dst % 1024) model::fail("tensor copy to a place that is not aligned");
    const auto& [count, distance] = model_matrices[m->p];
    std::vector<uint8_t> d(64 * 128, 0);
    for (uint32_t r = 0; r < 64; ++r)
        for (uint32_t c = 0; c < 64; ++c) {
            if ((uint64_t)y + r >= m->rows || (uint64_t)x + c >= m->cols || (uint64_t)z >= count) continue;
            uint32_t at = r * 128 + c * 2;
            at ^= (at >> 7 & 7) << 4;                        // 128-byte swizzle
            memcpy(&d[at], m->p + z * distance + ((uint64_t)y + r) * m->ld + ((uint64_t)x + c) * 2, 2);
        }
    if (model::dropped()) return;
    model::async_copy(dst, d, model::mapped(bar, 0));
}

inline void tmem_load32(uint32_t at, uint32_t (&r)[32]) {
    for (int i = 0; i < 4; ++i) tmem_load8(at + 8 * i, reinterpret_cast<uint32_t(&)[8]>(r[8 * i]));
}
inline void tmem_wait32(uint32_t (&)[32]) {}
inline void shared_store_pair_at(uint32_t at, uint32_t rank, uint2 v) {
    if (at % 8) model::fail("store that is not aligned");
    memcpy(model::memory(model::mapped(at, rank)), &v, 8);
}
inline void __threadfence() {}
inline void prefetch_map(const CUtensorMap*) {}
inline void fence_global_copies() {}
inline void grid_arrive(uint32_t* counter) { ++*counter; }
inline bool grid_wait(const uint32_t* counter, uint32_t target, volatile uint32_t* gave_up) {
    const long long end = model::W.clock + model::kWaitLimit;
    while (*counter < target) {
        if (*gave_up) return false;
        if (model::W.clock > end) {
            *gave_up = 1;
            return false;
        }
        model::cur->until = end + 201;
        model::wait_on(counter, *counter, true);
    }
    return true;
}
template <typename K, typename... A>
inline cudaError_t launch_together(K kernel, dim3 g, dim3 b, size_t smem, cudaStream_t, const A&... a) {
    if ((int)g.x != model::declared_cluster(kernel))
        model::fail("blocks that wait for each other: one cluster at a time runs here");
    return model::launch_kernel(kernel, g, b, smem, model::declared_cluster(kernel), a...);
}
inline float exp2_approx(float x) { return exp2f(x); }
inline Bytes32 ld_wide(const void* p) {
    if ((uintptr_t)p % 32) model::fail("load that is not aligned");
    return *static_cast<const Bytes32*>(p);
}
inline void st_wide(void* p, const Bytes32& r) {
    if ((uintptr_t)p % 32) model::fail("store that is not aligned");
    *static_cast<Bytes32*>(p) = r;
}

inline constexpr uint32_t mma_shape_of(uint32_t m, uint32_t n, bool bf16, bool a_lines, bool b_lines) {
    return (uint32_t)bf16 | (n >> 6) << 1 | (uint32_t)a_lines << 15 | (uint32_t)b_lines << 16 | (m >> 8) << 17;
}

inline float model_value_of(uint16_t h, bool bf16) {
    if (bf16) return model::half_of(h, 0);
    __half v;
    memcpy(&v, &h, 2);
    return __half2float(v);
}

// 256 x n x 16 of a pair: block r holds the rows from 128 r on and the columns from n / 2 r on.  An operand's address is that of
// its first value of the 16 k: by lines, panels of 64 values and a line for each k; else rows of 128 bytes
inline void product_mma(uint32_t to, uint64_t a, uint64_t b, uint32_t shape, bool add, bool elected) {
    if (!elected) return;
    const int n = (int)(shape >> 1 & 7) * 64;
    if (to % 256 || to >= 512 || (n != 256 && n != 128 && n != 64)) model::fail("matrix instruction");
    model::W.tensor.push_back([=] {
        static float left[256][16], right[16][256];
        const bool bf16 = shape & 1;
        auto read = [&](uint64_t op, bool lines, int r, int k, int i) {
            const uint32_t base = (uint32_t)(op & 0xFFFFFFFF) * 16, panel = (uint32_t)(op >> 32);
            const uint32_t line = lines ? base + panel * (i / 64) + k * 128 : base + i * 128;
            const uint32_t plain = line + (lines ? (i % 64) * 2 : k * 2);
            const uint32_t at = plain ^ ((plain >> 7 & 7) << 4);
            uint16_t h;
            memcpy(&h, model::memory(((uint32_t)(r + 1) << 24) | at), 2);
            return model_value_of(h, bf16);
        };
        for (int r = 0; r < 2; ++r)
            for (int k = 0; k < 16; ++k)
                for (int i = 0; i < 128; ++i) {
                    left[128 * r + i][k] = read(a, shape >> 15 & 1, r, k, i);
                    if (i < n / 2) right[k][n / 2 * r + i] = read(b, shape >> 16 & 1, r, k, i);
                }
        for (int m = 0; m < 256; ++m) {
            float* d = &model::W.tmem[(m / 128 * 128 + m % 128) * 512 + to];
            if (!add) memset(d, 0, n * 4);
            for (int k = 0; k < 16; ++k)
                for (int c = 0; c < n; ++c) d[c] += left[m][k] * right[k][c];
        }
    });
}

}  // namespace natcomp
