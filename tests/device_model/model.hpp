// Runs the library's CUDA kernels on the host, thread by thread: the sources are compiled as C++ with
// the built-ins below in place of the device's.  Every device thread is a fiber; the blocks of a
// cluster run at the same time, clusters one after the other.  Copies, matrix instructions and remote
// stores are queued and take effect later, in any order that the hardware may choose, so that a wait
// that is missing shows in the results.  Memory is checked by the address sanitizer: global buffers
// by their allocation, a block's shared memory by the ranges it has.
//
// Waits: time passes only while nothing else can happen, so a wait that runs out of time is one that
// nothing would have ended.
#pragma once
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <deque>
#include <functional>
#include <map>
#include <memory>
#include <random>
#include <string>
#include <tuple>
#include <unordered_map>
#include <vector>

#include <sanitizer/asan_interface.h>
#include <sanitizer/common_interface_defs.h>

#include "natcomp.h"

struct CUtensorMap_st {
    const uint8_t* p;
    uint64_t rows, cols, ld;             // ld in bytes
    uint32_t box_rows, box_cols, bytes;  // of an element
};
typedef CUtensorMap_st CUtensorMap;

#if !defined(__x86_64__)
#error "fibers are switched in x86-64 assembly"
#endif

// saves the caller's registers on its stack and its stack in *from, and goes on where `to` was saved
extern "C" void model_switch(void** from, void* to);
asm(R"(
.text
.globl model_switch
model_switch:
    push %rbp
    push %rbx
    push %r12
    push %r13
    push %r14
    push %r15
    mov %rsp, (%rdi)
    mov %rsi, %rsp
    pop %r15
    pop %r14
    pop %r13
    pop %r12
    pop %rbx
    pop %rbp
    ret
)");

extern "C" const char* __asan_default_options() { return "detect_leaks=0:detect_stack_use_after_return=0"; }

namespace model {

[[noreturn]] inline void fail(const char* what) {
    fprintf(stderr, "model: %s\n", what);
    abort();
}

constexpr size_t kArena = 512 << 10, kDynamic = 1040, kStatic = 300 << 10;
constexpr long long kWaitLimit = 4000000000ll;
constexpr size_t kShared = 232448, kStackBytes = 96 << 10;

struct Block;
struct Warp {
    uint64_t slot[2][32];
    uint32_t count = 0, gen = 0;
};
struct Counter {
    uint32_t count = 0, gen = 0;
};
struct Thread {
    void* saved;                         // its stack where it stands still
    char* stack;
    void* fake = nullptr;
    Block* block;
    uint32_t index;
    bool done = false;
    const uint32_t* on = nullptr;        // runs again when *on is no longer `seen`,
    uint32_t seen = 0;
    bool timed = false;                  // or, timed, when time has passed
    uint32_t lapse = 0;
    uint32_t tried = 0, parity = 0;      // the barrier it waits for, and from when on
    long long since = 0, until = 0;      // until: when its wait runs out of time
};
struct Block {
    uint32_t id, rank;
    uint8_t* arena;
    size_t dynamic, statics = kStatic;
    std::map<int, uint8_t*> named;
    std::vector<Warp> warps;
    std::map<int, Counter> bars;
};
struct Barrier {
    uint32_t expected = 0, pending = 0, phase = 0;
    int64_t tx = 0;
};

// what a test asks for
struct Inject {
    int drop_rank = -1, drop_nth = -1;   // this block's nth untiled copy or remote store never arrives
    int hold_rank = -1;                  // from its `hold_after`-th read of TMEM on, the first four
    int hold_after = 0;                  // warps of this block stand still until `hold_until`
    long long hold_until = 0;
    int late = 0;                        // one copy in so many arrives when nothing else can happen
};

struct World {
    std::vector<std::unique_ptr<Block>> blocks;          // of the running cluster
    std::vector<std::unique_ptr<Thread>> threads;
    std::unordered_map<uint32_t, Barrier> bars;
    std::vector<std::function<void()>> copies, late;
    std::deque<std::function<void()>> tensor;            // in order
    std::vector<float> tmem;                             // [rank][lane][column]
    Counter cluster;
    uint32_t lapses = 0;
    long long clock = 1000;
    int bulk[16] = {0}, tmem_reads[16] = {0};
    bool ran_out = false;                                // a wait ran out of time
};
inline World W;
inline Inject inject;
inline std::mt19937 rng(1);
inline Thread* cur = nullptr;
inline dim3 grid, block_dim;
inline void* home;
inline const void* home_bottom;
inline size_t home_size;
inline std::function<void()> body;
inline bool any_ran_out = false;
inline long long longest = 0;             // clock at the end of a cluster
inline std::map<const void*, int> cluster_of;
inline size_t launches = 0;
inline int sms = 148;

// ---- fibers
inline void to_home() {
    Thread* t = cur;
    __sanitizer_start_switch_fiber(t->done ? nullptr : &t->fake, home_bottom, home_size);
    model_switch(&t->saved, home);
    __sanitizer_finish_switch_fiber(t->fake, nullptr, nullptr);
}
inline void entry() {
    __sanitizer_finish_switch_fiber(nullptr, &home_bottom, &home_size);
    body();
    cur->done = true;
    to_home();
}
inline void resume(Thread* t) {
    cur = t;
    void* fake = nullptr;
    __sanitizer_start_switch_fiber(&fake, t->stack, kStackBytes);
    model_switch(&home, t->saved);
    __sanitizer_finish_switch_fiber(fake, nullptr, nullptr);
    cur = nullptr;
}
inline void wait_on(const uint32_t* p, uint32_t seen, bool timed = false) {
    cur->on = p;
    cur->seen = seen;
    cur->timed = timed;
    cur->lapse = W.lapses;
    to_home();
    cur->on = nullptr;
}
inline bool runnable(const Thread& t) {
    return !t.done && (!t.on || *t.on != t.seen || (t.timed && t.lapse != W.lapses));
}

inline void run_async() {
    // a few of the copies in any order, a few of the matrix instructions in theirs
    for (size_t k = rng() % 4; k > 0 && !W.copies.empty(); --k) {
        const size_t i = rng() % W.copies.size();
        auto f = std::move(W.copies[i]);
        W.copies.erase(W.copies.begin() + i);
        f();
    }
    for (size_t k = rng() % 6; k > 0 && !W.tensor.empty(); --k) {
        auto f = std::move(W.tensor.front());
        W.tensor.pop_front();
        f();
    }
}

inline void run_cluster(uint32_t first, int size, dim3 g, dim3 b, size_t smem) {
    W.bars.clear();
    W.blocks.clear();
    W.threads.clear();
    W.cluster = Counter();
    W.ran_out = false;
    W.clock = 1000;
    memset(W.bulk, 0, sizeof W.bulk);
    memset(W.tmem_reads, 0, sizeof W.tmem_reads);
    const uint32_t n = b.x;
    if (n % 32 || n > 1024) fail("threads of a block");
    static std::vector<char*> stacks;
    static std::vector<uint8_t*> arenas;
    while (stacks.size() < (size_t)size * n) stacks.push_back((char*)malloc(kStackBytes));
    while (arenas.size() < (size_t)size) arenas.push_back((uint8_t*)aligned_alloc(1 << 16, kArena));
    for (int r = 0; r < size; ++r) {
        auto blk = std::make_unique<Block>();
        blk->id = first + r;
        blk->rank = r;
        blk->arena = arenas[r];
        blk->dynamic = smem;
        __asan_unpoison_memory_region(blk->arena, kArena);
        memset(blk->arena, 0xFF, kArena);
        __asan_poison_memory_region(blk->arena, kArena);
        __asan_unpoison_memory_region(blk->arena + kDynamic, smem);
        blk->warps.resize(n / 32);
        W.blocks.push_back(std::move(blk));
    }
    for (int r = 0; r < size; ++r)
        for (uint32_t i = 0; i < n; ++i) {
            auto t = std::make_unique<Thread>();
            t->stack = stacks[(size_t)r * n + i];
            t->block = W.blocks[r].get();
            t->index = i;
            // a first switch pops six registers and returns to entry()
            void** top = (void**)(((uintptr_t)t->stack + kStackBytes) & ~(uintptr_t)15) - 8;
            __asan_unpoison_memory_region(t->stack, kStackBytes);
            for (int k = 0; k < 6; ++k) top[k] = nullptr;
            top[6] = (void*)&entry;
            top[7] = nullptr;
            t->saved = top;
            W.threads.push_back(std::move(t));
        }
    size_t left = W.threads.size();
    std::vector<uint32_t> order(W.threads.size() / 32);
    for (size_t i = 0; i < order.size(); ++i) order[i] = (uint32_t)i;
    int idle = 0;
    bool looked = false;
    while (left) {
        std::shuffle(order.begin(), order.end(), rng);
        bool moved = false;
        for (uint32_t w : order) {
            for (uint32_t l = 0; l < 32; ++l) {
                Thread* t = W.threads[32 * w + l].get();
                if (!runnable(*t)) continue;
                if (!(t->on && *t->on == t->seen)) moved = true;      // not by time alone
                resume(t);
                if (t->done) --left;
            }
            if (rng() % 4 == 0) run_async();
        }
        if (!W.copies.empty() || !W.tensor.empty()) {
            run_async();
            moved = true;
        }
        W.clock += 100;
        if (moved) {
            idle = 0;
            looked = false;
            continue;
        }
        if (!W.late.empty()) {           // one of those that come late
            const size_t i = rng() % W.late.size();
            W.copies.push_back(std::move(W.late[i]));
            W.late.erase(W.late.begin() + i);
            continue;
        }
        // (a thread that has tried once goes on to wait)
        bool again = false;
        for (auto& t : W.threads) again |= runnable(*t);
        if (again) continue;
        // a waiting thread looks at other things than its barrier now and then
        looked = !looked;
        if (looked) {
            ++W.lapses;
            continue;
        }
        // nothing but time can end a wait: it passes until the first of them runs out
        long long next = 0;
        for (auto& t : W.threads)
            if (!t->done && t->timed && t->on && t->until > W.clock && (!next || t->until < next))
                next = t->until;
        if (!next && ++idle > 20) fail("threads wait for each other");
        W.clock = next ? next : W.clock + 1000000000ll;
        if (W.clock > kWaitLimit) W.ran_out = true;
        ++W.lapses;
    }
    if (!W.copies.empty() || !W.late.empty()) fail("a block ended with copies in flight");
    if (!W.tensor.empty()) fail("a block ended with matrix instructions in flight");
    any_ran_out |= W.ran_out;
    longest = std::max(longest, W.clock);
    for (auto& blk : W.blocks) {
        if (blk->dynamic + (blk->statics - kStatic) > kShared) fail("too much shared memory");
        __asan_unpoison_memory_region(blk->arena, kArena);
    }
}

template <typename F>
inline void launch(F f, int cluster, dim3 g, dim3 b, size_t smem) {
    ++launches;
    if (!g.x || !g.y || g.x % cluster || !b.x) fail("launch shape");
    grid = g;
    block_dim = b;
    body = f;
    for (uint32_t y = 0; y < g.y; ++y)
        for (uint32_t x = 0; x < g.x; x += cluster) run_cluster(y * g.x + x, cluster, g, b, smem);
}

template <typename K, typename... A>
inline cudaError_t launch_kernel(K kernel, dim3 g, dim3 b, size_t smem, int cluster, const A&... a) {
    auto args = std::make_tuple(a...);
    launch([&] { std::apply(kernel, args); }, cluster, g, b, smem);
    return cudaSuccess;
}
template <typename K> inline int declared_cluster(K kernel) {
    auto it = cluster_of.find((const void*)kernel);
    return it == cluster_of.end() ? 1 : it->second;
}
template <typename K> struct Chevrons {
    K kernel;
    dim3 g, b;
    size_t smem;
    template <typename... A> void operator()(const A&... a) {
        launch_kernel(kernel, g, b, smem, declared_cluster(kernel), a...);
    }
};
template <typename K>
inline Chevrons<K> chevrons(K kernel, dim3 g, dim3 b, size_t smem, cudaStream_t) {
    return {kernel, g, b, smem};
}
template <typename... P, typename... A>
inline cudaError_t launch_ex(const cudaLaunchConfig_t* c, void (*kernel)(P...), const A&... a) {
    int cluster = 1;
    for (unsigned i = 0; i < c->numAttrs; ++i)
        if (c->attrs[i].id == cudaLaunchAttributeClusterDimension)
            cluster = c->attrs[i].val.clusterDim.x;
    return launch_kernel(kernel, c->gridDim, c->blockDim, c->dynamicSmemBytes, cluster, a...);
}
inline cudaError_t get_device(int* d) { *d = 0; return cudaSuccess; }
inline cudaError_t get_attribute(int* v, cudaDeviceAttr, int) { *v = sms; return cudaSuccess; }
inline cudaError_t set_attribute(const void*, cudaFuncAttribute, int bytes) {
    return bytes <= (int)kShared ? cudaSuccess : cudaErrorInvalidValue;
}
inline cudaError_t no_error() { return cudaSuccess; }

// ---- shared memory
inline uint8_t* dynamic_memory() { return cur->block->arena + kDynamic; }
inline uint8_t* static_memory(int name, size_t bytes) {
    Block& b = *cur->block;
    uint8_t*& p = b.named[name];
    if (!p) {
        p = b.arena + b.statics;
        __asan_unpoison_memory_region(p, bytes);
        b.statics += (bytes + 64 + 15) / 16 * 16;
    }
    return p;
}
inline uint32_t shared_address(const void* p) {
    const ptrdiff_t at = (const uint8_t*)p - cur->block->arena;
    if (at < 0 || at >= (ptrdiff_t)kArena) fail("not an address of shared memory");
    return ((cur->block->rank + 1) << 24) | (uint32_t)at;
}
inline uint32_t mapped(uint32_t a, uint32_t rank) {
    if (rank >= W.blocks.size()) fail("no such block in the cluster");
    return ((rank + 1) << 24) | (a & 0xFFFFFF);
}
inline uint8_t* memory(uint32_t a) { return W.blocks[(a >> 24) - 1]->arena + (a & 0xFFFFFF); }

// ---- collectives
inline const uint64_t* exchange(uint64_t v) {
    Warp& w = cur->block->warps[cur->index >> 5];
    const uint32_t g = w.gen;
    w.slot[g & 1][cur->index & 31] = v;
    if (++w.count == 32) {
        w.count = 0;
        ++w.gen;
    } else {
        wait_on(&w.gen, g);
    }
    return w.slot[g & 1];
}
inline void meet(Counter& c, uint32_t threads) {
    const uint32_t g = c.gen;
    if (++c.count == threads) {
        c.count = 0;
        ++c.gen;
    } else {
        wait_on(&c.gen, g);
    }
}
inline void named_barrier(int id, uint32_t threads) { meet(cur->block->bars[id], threads); }

// ---- mbarriers
inline Barrier& bar_at(uint32_t a) {
    auto it = W.bars.find(a);
    if (it == W.bars.end()) fail("no barrier at this address");
    return it->second;
}
inline void bar_check(Barrier& b) {
    if (b.pending == 0 && b.tx == 0) {
        ++b.phase;
        b.pending = b.expected;
    }
}
inline void bar_arrive(uint32_t a) {
    Barrier& b = bar_at(a);
    if (!b.pending) {
        fprintf(stderr, "barrier %x, phase %u, %lld bytes to come\n", a, b.phase, (long long)b.tx);
        fail("more arrivals than a barrier expects");
    }
    --b.pending;
    bar_check(b);
}
inline void bar_tx(uint32_t a, int64_t bytes) {
    Barrier& b = bar_at(a);
    b.tx += bytes;
    bar_check(b);
}
inline bool bar_done(uint32_t a, uint32_t parity) { return (bar_at(a).phase & 1) != parity; }

inline bool dropped() {
    const int rank = (int)cur->block->rank;
    return W.bulk[rank]++ == inject.drop_nth && rank == inject.drop_rank;
}
inline void async_copy(uint32_t dst, std::vector<uint8_t> data, uint32_t bar) {
    auto& list = inject.late && rng() % inject.late == 0 ? W.late : W.copies;
    list.push_back([=] {
        memcpy(memory(dst), data.data(), data.size());
        bar_tx(bar, -(int64_t)data.size());
    });
}

// ---- pairs of bfloat16 and float
inline float half_of(uint32_t w, int h) {
    const uint32_t b = h ? w & 0xFFFF0000u : w << 16;
    float f;
    memcpy(&f, &b, 4);
    return f;
}
inline uint16_t to_bf16(float f) {
    const __nv_bfloat16 v = __float2bfloat16_rn(f);
    uint16_t r;
    memcpy(&r, &v, 2);
    return r;
}
inline uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
    return to_bf16(half_of(a, 0) - half_of(b, 0)) |
           (uint32_t)to_bf16(half_of(a, 1) - half_of(b, 1)) << 16;
}

}  // namespace model

// ---- the device's names
struct ModelIndex {
    struct X {
        operator uint32_t() const { return model::cur->index; }
    } x;
};
struct ModelBlockIndex {
    struct X {
        operator uint32_t() const { return model::cur->block->id % model::grid.x; }
    } x;
    struct Y {
        operator uint32_t() const { return model::cur->block->id / model::grid.x; }
    } y;
};
inline ModelIndex threadIdx;
inline ModelBlockIndex blockIdx;
inline dim3& blockDim = model::block_dim;
inline dim3& gridDim = model::grid;
#define cudaGetDevice model::get_device
#define cudaDeviceGetAttribute model::get_attribute
#define cudaFuncSetAttribute(k, w, b) model::set_attribute(k, w, b)
#define cudaPeekAtLastError model::no_error
#define cudaLaunchKernelEx(c, k, ...) model::launch_ex(c, k, __VA_ARGS__)

using std::max;
using std::min;
inline uint32_t max(int a, uint32_t b) { return std::max((uint32_t)a, b); }

template <typename T> inline T __ldg(const T* p) { return *p; }
template <typename T> inline T __ldcs(const T* p) { return *p; }
template <typename T> inline T __ldcg(const T* p) { return *p; }
template <typename T> inline void __stcs(T* p, T v) { *p = v; }
inline uint32_t __float_as_uint(float f) { uint32_t u; memcpy(&u, &f, 4); return u; }
inline float __uint_as_float(uint32_t u) { float f; memcpy(&f, &u, 4); return f; }
inline uint32_t __byte_perm(uint32_t x, uint32_t y, uint32_t s) {
    const uint64_t v = (uint64_t)y << 32 | x;
    uint32_t r = 0;
    for (int i = 0; i < 4; ++i) r |= (uint32_t)(v >> (8 * ((s >> (4 * i)) & 7)) & 0xFF) << (8 * i);
    return r;
}
inline uint32_t __funnelshift_r(uint32_t lo, uint32_t hi, uint32_t s) {
    return (uint32_t)(((uint64_t)hi << 32 | lo) >> (s & 31));
}
inline float rsqrtf(float x) { return 1.0f / sqrtf(x); }
inline long long clock64() { return model::W.clock; }

template <typename T> inline uint64_t model_bits(T v) {
    uint64_t b = 0;
    memcpy(&b, &v, sizeof v);
    return b;
}
template <typename T> inline T model_value(uint64_t b) {
    T v;
    memcpy(&v, &b, sizeof v);
    return v;
}
template <typename T> inline T __shfl_sync(uint32_t, T v, int lane) {
    return model_value<T>(model::exchange(model_bits(v))[lane & 31]);
}
template <typename T> inline T __shfl_xor_sync(uint32_t, T v, int m) {
    const uint32_t lane = model::cur->index & 31;
    return model_value<T>(model::exchange(model_bits(v))[lane ^ m]);
}
inline bool __all_sync(uint32_t, int p) {
    const uint64_t* s = model::exchange(p != 0);
    bool all = true;
    for (int i = 0; i < 32; ++i) all &= s[i] != 0;
    return all;
}
inline void __syncwarp() { model::exchange(0); }
inline void __syncthreads() { model::named_barrier(0, blockDim.x); }

// ---- what the sources call for the barriers, copies and matrix instructions of sm_100a
namespace natcomp {

inline uint32_t smem_u32(const void* p) { return model::shared_address(p); }
inline void cluster_sync() {
    model::meet(model::W.cluster, (uint32_t)model::W.threads.size());
}
inline void mbar_init(uint32_t bar, uint32_t count) {
    model::memory(bar)[0] = model::memory(bar)[7] = 0;       // inside its block's memory
    if (bar % 8) model::fail("barrier not aligned");
    model::Barrier b;
    b.expected = b.pending = count;
    model::W.bars[bar] = b;
}
inline void mbar_init_fence() {}
inline void mbar_expect(uint32_t bar, uint32_t bytes) {
    model::bar_at(bar).tx += bytes;
    model::bar_arrive(bar);
}
inline void mbar_arrive(uint32_t bar) { model::bar_arrive(bar); }
inline void mbar_arrive_at(uint32_t bar, uint32_t rank) { model::bar_arrive(model::mapped(bar, rank)); }
inline void st_async_pair(uint32_t dst, uint32_t bar, uint32_t rank, float2 v) {
    std::vector<uint8_t> d(8);
    memcpy(d.data(), &v, 8);
    if (model::dropped()) return;
    model::async_copy(model::mapped(dst, rank), d, model::mapped(bar, rank));
}
inline bool mbar_test(uint32_t bar, uint32_t parity) { return model::bar_done(bar, parity); }
inline bool mbar_try(uint32_t bar, uint32_t parity) {
    model::Thread& t = *model::cur;
    if (!model::bar_done(bar, parity)) {
        if (t.tried != bar || t.parity != parity) {          // once, then the caller looks at the time
            t.tried = bar;
            t.parity = parity;
            t.since = model::W.clock;
            model::wait_on(nullptr, 0);
        } else {
            t.until = t.since + model::kWaitLimit + 201;
            model::wait_on(&model::bar_at(bar).phase, model::bar_at(bar).phase, true);
        }
    }
    const bool done = model::bar_done(bar, parity);
    if (done) t.tried = 0;
    return done;
}
inline void tma_load_2d(uint32_t dst, const CUtensorMap* m, int x, int y, uint32_t bar) {
    if ((uint64_t)x * m->bytes % 16) model::fail("tensor copy at an x that is not aligned");
    if (dst % (m->bytes == 2 ? 1024 : 128)) model::fail("tensor copy to a place that is not aligned");
    const uint32_t line = m->box_cols * m->bytes;
    std::vector<uint8_t> d((size_t)m->box_rows * line, 0);
    for (uint32_t r = 0; r < m->box_rows; ++r)
        for (uint32_t c = 0; c < m->box_cols; ++c) {
            if ((uint64_t)y + r >= m->rows || (uint64_t)x + c >= m->cols) continue;
            uint32_t at = r * line + c * m->bytes;
            if (m->bytes == 2) at ^= (at >> 7 & 7) << 4;                 // 128-byte swizzle
            memcpy(&d[at], m->p + ((uint64_t)y + r) * m->ld + ((uint64_t)x + c) * m->bytes, m->bytes);
        }
    model::async_copy(dst, d, bar);
}
inline void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    if (dst % 16 || (uintptr_t)src % 16 || bytes % 16) model::fail("bulk copy that is not aligned");
    std::vector<uint8_t> d((const uint8_t*)src, (const uint8_t*)src + bytes);
    if (model::dropped()) return;
    model::async_copy(dst, d, bar);
}
inline void global_add4(float4* p, float a, float b, float c, float d) {
    if ((uintptr_t)p % 16) model::fail("addition that is not aligned");
    p->x += a; p->y += b; p->z += c; p->w += d;
}
inline void fence_async_proxy() {}
inline void shared_store16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    if (at % 16) model::fail("store that is not aligned");
    const uint32_t v[4] = {a, b, c, d};
    memcpy(model::memory(at), v, 16);
}
inline void shared_store_at(uint32_t at, uint32_t rank, uint32_t v) {
    memcpy(model::memory(model::mapped(at, rank)), &v, 4);
}
inline void fence_cluster() {}

inline void tmem_alloc_pair(uint32_t where, uint32_t columns) {
    if (model::W.tmem.size() != 2 * 128 * 512) model::W.tmem.resize(2 * 128 * 512);
    if (columns != 512) model::fail("columns of TMEM");
    std::fill(model::W.tmem.begin(), model::W.tmem.end(), NAN);
    memset(model::memory(where), 0, 4);
}
inline void tmem_free_pair(uint32_t, uint32_t) {
    if (!model::W.tensor.empty()) model::fail("TMEM freed under matrix instructions");
}
inline void tc_fence_before() {}
inline void tc_fence_after() {}
inline void tmem_load8(uint32_t at, uint32_t (&r)[8]) {
    const uint32_t rank = model::cur->block->rank, lanes = at >> 16, column = at & 0xFFFF;
    const uint32_t warp = model::cur->index >> 5, lane = model::cur->index & 31;
    if (lanes != 32 * (warp & 3) || column + 8 > 512) model::fail("TMEM that a warp cannot read");
    if ((int)rank == model::inject.hold_rank &&
        ++model::W.tmem_reads[rank] > model::inject.hold_after)
        while (model::W.clock < model::inject.hold_until) {
            static uint32_t never = 0;
            model::cur->until = model::inject.hold_until;
            model::wait_on(&never, 0, true);
        }
    memcpy(r, &model::W.tmem[(rank * 128 + lanes + lane) * 512 + column], 32);
}
inline void tmem_wait8(uint32_t (&)[8]) {}
inline uint64_t mma_operand(uint32_t address, uint32_t panel) {
    return (uint64_t)(address & 0xFFFFFF) / 16 | (uint64_t)panel << 32;
}
inline constexpr uint32_t mma_shape(uint32_t m, uint32_t n) { return m << 16 | n; }
inline bool elect_one() { return (model::cur->index & 31) == 0; }

inline void model_mma(uint32_t to, uint64_t a, uint64_t b, bool add) {
    // 256 rows x 256 columns x 16: block r holds the rows from 128 r on, of A, and of B the columns
    static float left[2][16][128], right[16][256];
    auto read = [&](uint64_t op, int r, int k, int i) {
        const uint32_t line = (uint32_t)(op & 0xFFFFFFFF) * 16 + (uint32_t)(op >> 32) * (i / 64) + k * 128;
        const uint32_t at = (line + (i % 64) * 2) ^ ((line >> 7 & 7) << 4);
        uint16_t h;
        memcpy(&h, model::memory(((uint32_t)(r + 1) << 24) | at), 2);
        return model::half_of(h, 0);
    };
    for (int r = 0; r < 2; ++r)
        for (int k = 0; k < 16; ++k)
            for (int i = 0; i < 128; ++i) {
                left[r][k][i] = read(a, r, k, i);
                right[k][128 * r + i] = read(b, r, k, i);
            }
    for (int r = 0; r < 2; ++r)
        for (int m = 0; m < 128; ++m) {
            float* d = &model::W.tmem[(r * 128 + m) * 512 + to];
            if (!add) memset(d, 0, 256 * 4);
            for (int k = 0; k < 16; ++k) {
                const float l = left[r][k][m];
                for (int n = 0; n < 256; ++n) d[n] += l * right[k][n];
            }
        }
}
inline void mma_pair(uint32_t tmem, uint64_t a, uint64_t b, uint32_t shape, bool add, bool elected) {
    if (!elected) return;
    if (shape != mma_shape(256, 256) || tmem % 256 || tmem >= 512) model::fail("matrix instruction");
    model::W.tensor.push_back([=] { model_mma(tmem, a, b, add); });
}
inline void mma_commit_pair(uint32_t bar, bool elected) {
    if (!elected) return;
    model::W.tensor.push_back([=] {
        for (uint32_t r = 0; r < 2; ++r) model::bar_arrive(model::mapped(bar, r));
    });
}
inline bool make_tensor_map(CUtensorMap* map, const void* p, bool bf16, uint64_t rows, uint64_t cols,
                            uint64_t ld, uint32_t box_cols, uint32_t box_rows) {
    const uint32_t bytes = bf16 ? 2 : 1;
    if ((uintptr_t)p % 16 || ld * bytes % 16 || box_cols * bytes % 16) return false;
    *map = {(const uint8_t*)p, rows, cols, ld * bytes, box_rows, box_cols, bytes};
    return true;
}
inline void after_previous() {}
inline void let_next_begin() {}
template <typename K, typename... A>
inline cudaError_t launch_overlapping(K kernel, dim3 g, dim3 b, size_t smem, cudaStream_t,
                                      const A&... a) {
    return model::launch_kernel(kernel, g, b, smem, model::declared_cluster(kernel), a...);
}

}  // namespace natcomp

// ---- for the programs
struct Held {                            // memory whose ends the sanitizer checks, at an offset
    std::unique_ptr<uint8_t[]> raw;
    uint8_t* p;
    Held(size_t bytes, size_t offset = 0) : raw(new uint8_t[bytes + offset + 64]) {
        uintptr_t a = ((uintptr_t)raw.get() + 63) & ~(uintptr_t)63;
        p = (uint8_t*)a + offset;
        const uintptr_t end = (uintptr_t)raw.get() + bytes + offset + 64;
        memset(raw.get(), 0xFF, bytes + offset + 64);
        if (end > a + offset + bytes) __asan_poison_memory_region(p + bytes, end - (a + offset + bytes));
    }
    ~Held() { __asan_unpoison_memory_region(raw.get(), 1); }
};

// name=value arguments from `first` on; whether one of them makes a wait run out
inline bool injected(int argc, char** argv, int first) {
    bool ran_out = false;
    for (int i = first; i < argc; ++i) {
        const std::string a = argv[i], name = a.substr(0, a.find('='));
        const long long v = atoll(a.c_str() + a.find('=') + 1);
        if (name == "late") {
            model::inject.late = (int)v;
            continue;
        }
        ran_out = true;
        if (name == "drop_rank") model::inject.drop_rank = (int)v;
        else if (name == "drop_nth") model::inject.drop_nth = (int)v;
        else if (name == "hold_rank") model::inject.hold_rank = (int)v;
        else if (name == "hold_after") model::inject.hold_after = (int)v;
        else if (name == "hold_until") model::inject.hold_until = v;
        else model::fail("argument");
    }
    return ran_out;
}
