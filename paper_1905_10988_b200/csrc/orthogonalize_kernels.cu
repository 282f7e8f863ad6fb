// Orthogonalised update of a weight matrix by Newton-Schulz products, for sm_100a:
//
//   X <- G / (|G| + eps),  then `steps` times  X <- a X + (b A + c A A) X,  A = X X^T,  out = scale X
//
// (|G| the Frobenius norm; of a matrix with more rows than columns A = X^T X and the polynomial is
// applied from the right).  Each step applies the odd polynomial a s + b s^3 + c s^5 to the singular
// values and leaves the singular vectors alone.
//
// The three products of a step run on the tensor cores.  A and b A + c A A are symmetric: only the tiles
// on and above the diagonal are computed, and the products that read them take the others from their
// mirror images, so a step of a square matrix costs four thirds of a product less.  Nothing is
// transposed: either layout is an operand as it lies in memory.
//
// Numbers: operands are binary16, not bfloat16.  All of them are bounded (singular values near 1), so
// range is no concern and the three bits more are: with bfloat16 the result is off by 1 to 2 % of its
// norm, with binary16 by 0.1 to 0.2 %, as much as rounding it to bfloat16 costs.  X is kept in 22 bits,
// as two binary16 values; the term a X takes both, the products the first.  With one value alone the
// rounding of each step would grow like the smallest singular values do (a^steps, several hundred
// times), and a gradient of low rank would come out wrong by 4 %.  The diagonal of the polynomial, which
// is most of it once the singular values are near 1, stays in binary32 and outside the product (off by
// 1.7e-3 of the norm instead of 2.4e-3 for random 256 x 512).  X is scaled by the power of two near
// the root of its longer side, which brings its entries to about 1, A and the polynomial by 2^8: away
// from binary16's subnormal numbers.
//
// All steps are one cooperative launch: a phase costs 3.7 us at least (64 x 64) and 90 us for 4096 x 4096,
// where the power cap bounds it (1.1 ms for five steps, 1.3 back to back; 1.2 PFLOP/s counting half of the
// symmetric products).
#include "product.cuh"

namespace natcomp {

constexpr float kOrthoGramScale = 256.0f;
constexpr int kOrthoSteps = 16;                      // of one launch
constexpr int kOrthoLaunches = 64;
// Steps of a sum that is worth splitting.  Updates of five steps, whole and split: 512 x 1024 121 and 124 us,
// 512 x 1536 133 and 130, 512 x 2048 148 and 133, 128 x 2048 125 and 111.
constexpr uint64_t kOrthoLong = 24;
constexpr float kOrthoLow = 2048.0f;                 // of the second of X's two values
constexpr int kOrthoNormBlocks = 592;                // per matrix at most

// ---- the norm, and the first X ---------------------------------------------------------------

struct OrthoInput {
    const void* g;
    int dtype;
    uint64_t rows, cols, ldg, distance;
    bool vector;                         // rows may be read 16 bytes at a time
    double* parts;                       // [matrix][block]
    int blocks;
    double eps, scale;
    __half *high, *low;
    uint64_t pitch;
    uint32_t* arrived;                   // words that the products count in, cleared here
    int words;
};

// eight values of a row, those beyond it 0
template <typename T>
__device__ __forceinline__ void ortho_load8(const OrthoInput& in, const T* row, uint64_t c,
                                            float (&v)[8]) {
    if (in.vector && c + 8 <= in.cols) {
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
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < in.cols ? to_f32<T>(row[c + i]) : 0.0f;
    }
}

// Sums of squares, in binary64: neither overflows nor vanishes for any binary32 input.
template <typename T>
__global__ void __launch_bounds__(256) ortho_norm_kernel(const __grid_constant__ OrthoInput in) {
    __shared__ double sums[8];
    after_previous();
    let_next_begin();
    const T* g = static_cast<const T*>(in.g) + blockIdx.y * in.distance;
    const uint64_t across = (in.cols + 7) / 8, all = in.rows * across;
    double s = 0.0;
#pragma unroll 4
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (uint64_t)in.blocks * 256) {
        const uint64_t r = i / across;
        float v[8];
        ortho_load8<T>(in, g + r * in.ldg, (i - r * across) * 8, v);
        double t = 0.0;
#pragma unroll
        for (int k = 0; k < 8; ++k) t = fma((double)v[k], (double)v[k], t);
        s += t;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) s += sums[w];
        in.parts[(uint64_t)blockIdx.y * in.blocks + blockIdx.x] = s;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) ortho_start_kernel(const __grid_constant__ OrthoInput in) {
    after_previous();
    let_next_begin();
    __shared__ double sums;
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = threadIdx.x; i < in.words; i += 256) in.arrived[i] = 0;
    if (threadIdx.x < 32) {
        double s = 0.0;
#pragma unroll 8
        for (int i = threadIdx.x; i < in.blocks; i += 32)
            s += __ldcg(in.parts + (uint64_t)blockIdx.y * in.blocks + i);
#pragma unroll
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
        if (threadIdx.x == 0) sums = s;
    }
    __syncthreads();
    const double sum = sums;
    // (of an inf: NaN for all values, not 0 for those that are finite)
    const double by = sum == 0.0      ? 0.0
                      : isfinite(sum) ? in.scale / (sqrt(sum) + in.eps)
                                      : (double)__uint_as_float(0x7FC00000u);
    const bool narrow = by > 1e-37 && by < 1e37;
    const float by32 = (float)by;
    const T* g = static_cast<const T*>(in.g) + blockIdx.y * in.distance;
    const uint64_t across = in.pitch / 8, all = in.rows * across;
    const uint64_t base = (uint64_t)blockIdx.y * in.rows * in.pitch;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (uint64_t)gridDim.x * 256) {
        const uint64_t r = i / across, c = (i - r * across) * 8;
        float v[8];
        ortho_load8<T>(in, g + r * in.ldg, c, v);
        uint32_t h[4], l[4];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = narrow ? v[k] * by32 : (float)((double)v[k] * by);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float a, b;
            h[k] = pack2<__half>(v[2 * k], v[2 * k + 1]);
            unpack2<__half>(h[k], a, b);
            l[k] = pack2<__half>((v[2 * k] - a) * kOrthoLow, (v[2 * k + 1] - b) * kOrthoLow);
        }
        const uint64_t at = base + r * in.pitch + c;
        *reinterpret_cast<uint4*>(in.high + at) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(in.low + at) = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

// ---- products --------------------------------------------------------------------------------

// the u-th tile on or above the diagonal of one of several square matrices of `side` tiles
__device__ __forceinline__ ProductUnit ortho_upper(uint32_t u, uint32_t side) {
    ProductUnit w = {};
    const uint32_t each = side * (side + 1) / 2;
    w.z = (int)(u / each);
    u -= (uint32_t)w.z * each;
    uint32_t row = 0;
    while (u >= side - row) {
        u -= side - row;
        ++row;
    }
    w.m = (int)(row * kProductTile);
    w.n = (int)((row + u) * kProductTile);
    return w;
}

// 16 values of a row of binary16 as they lie in a workspace
__device__ __forceinline__ void ortho_unpack16(const Bytes32& raw, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) unpack2<__half>(raw.v[i], v[2 * i], v[2 * i + 1]);
}
__device__ __forceinline__ void ortho_store16(__half* p, const float (&v)[16]) {
    Bytes32 raw;
#pragma unroll
    for (int i = 0; i < 8; ++i) raw.v[i] = pack2<__half>(v[2 * i], v[2 * i + 1]);
    st_wide(p, raw);
}

// Every step has three phases: A from X, b A + c A A from A, the next X.
struct OrthoJob {
    static constexpr bool kPhased = true;
    CUtensorMap x_map[2], gram_map, poly_map;
    bool bf16;                           // no
    bool tall;
    uint32_t phases;                     // three of every step, or, no steps, one
    uint32_t* arrived;
    uint32_t rows, cols, side, batch;
    uint32_t tiles, tiles_m, tiles_n;    // of a side, of X
    uint64_t pitch, side_pitch;          // row strides of X, and of A and the polynomial
    __half *high[2], *low;
    __half *gram, *poly;
    float* diagonal;                     // of the polynomial: [matrix][side_pitch]; poly has 0 there
    float of_step[3 * kOrthoSteps];      // a, b, c of the launch's steps
    float gram_scale;
    uint32_t splits;                     // of the long sums of A
    float4* parts;                       // [unit][split][column / 4][256 rows]
    uint32_t* tickets;                   // [unit][half of the rows]: 0 at the beginning
    uint32_t turn;                       // which of the two X the first step reads
    void* out;                           // of the last step, nullptr: another launch follows
    uint64_t ldo, out_distance;
    float scale;
    ProductTarget target;
    // of the phase
    ProductSide left_side, right_side;
    ProductSplit split;
    uint32_t kind, step, from, count;    // kind: 0, 1, 2, or 3 for no steps; from: which of the two X is read
    float a, b, c;

    struct State {
        Bytes32 first[2], second[2];     // 32 values of A, or of X's two, a chunk ahead
        float of_column;                 // the lane's diagonal value, tall
    };
    const OrthoJob* self;                // as the kernel was given it: arrays indexed there need no copy
    __device__ __forceinline__ void given_as(const OrthoJob* job) { self = job; }
    __device__ __forceinline__ void prefetch() const {
        prefetch_map(&x_map[0]);
        prefetch_map(&x_map[1]);
        prefetch_map(&gram_map);
        prefetch_map(&poly_map);
    }
    __device__ __forceinline__ const CUtensorMap* left_map() const {
        return kind == 1 ? &self->gram_map : kind == 2 && !tall ? &self->poly_map : &self->x_map[from];
    }
    __device__ __forceinline__ const CUtensorMap* right_map() const {
        return kind == 1 ? &self->gram_map : kind == 2 && tall ? &self->poly_map : &self->x_map[from];
    }
    __device__ __forceinline__ uint32_t chains() const { return 1; }
    __device__ __forceinline__ uint32_t begin(uint32_t phase, bool) {
        step = phase / 3;
        kind = phases == 1 ? 3 : phase - 3 * step;
        from = (turn + step) & 1;
        a = kind == 3 ? 1.0f : self->of_step[3 * step];
        b = self->of_step[3 * step + 1];
        c = kind == 0 ? gram_scale : self->of_step[3 * step + 2] * (1.0f / kOrthoGramScale);
        left_side.symmetric = kind == 1 || (kind == 2 && !tall);
        right_side.symmetric = kind == 1 || (kind == 2 && tall);
        left_side.lines = kind == 0 && tall;
        right_side.lines = kind == 0 ? tall : kind == 2 && !tall;
        const uint32_t longer = tall ? rows : cols;
        count = kind == 3 ? 0 : ((kind == 0 ? longer : side) + kProductStep - 1) / kProductStep;
        const uint32_t all = (kind < 2 ? tiles * (tiles + 1) / 2 : tiles_m * tiles_n) * batch;
        split = product_split(all);
        return split.units(all) * (kind == 0 ? splits : 1);
    }
    __device__ __forceinline__ ProductUnit unit_of(uint32_t u, uint32_t) const {
        int column, width;
        const uint32_t number = u, by = kind == 0 ? splits : 1;
        const uint32_t t = split.tile(u / by, column, width);
        ProductUnit w = {};
        if (kind < 2) {
            w = ortho_upper(t, tiles);
        } else {
            const uint32_t each = tiles_m * tiles_n, z = t / each;
            product_tile(t - z * each, tiles_m, tiles_n, w.m, w.n);
            w.z = (int)z;
        }
        w.n += column;
        w.width = width;
        w.part = number;
        const uint32_t i = number % by, first = count * i / by;
        w.k = (int)first * kProductStep;
        w.steps = (int)(count * (i + 1) / by - first);
        return w;
    }
    __device__ __forceinline__ void load(const ProductUnit& w, const ProductRead& r, int k, State& s) const {
        const uint32_t row = (uint32_t)(w.m + r.row), col = (uint32_t)(w.n + r.column) + k;
        if (kind == 0 || k >= r.columns) return;
        if (kind == 1) {
            if (row >= side) return;
            const __half* p = gram + ((uint64_t)w.z * side + row) * side_pitch + col;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (col + 16 * h < side) s.first[h] = ld_wide(p + 16 * h);
            return;
        }
        if (kind == 2 && tall && col + r.lane < cols)
            s.of_column = __ldcg(diagonal + w.z * side_pitch + col + r.lane);
        if (row >= rows) return;
        const uint64_t at = ((uint64_t)w.z * rows + row) * pitch + col;
        const __half* p = self->high[from];
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (col + 16 * h < cols) {
                s.first[h] = ld_wide(p + at + 16 * h);
                s.second[h] = ld_wide(low + at + 16 * h);
            }
    }
    __device__ __forceinline__ void ahead(const ProductUnit& w, const ProductRead& r, State& s) const {
        load(w, r, 0, s);
    }
    __device__ __forceinline__ void store(const ProductUnit& w, const ProductRead& r, State& s) const {
        if (kind == 0 && splits > 1) {
            uint32_t* ticket = tickets + 2 * (w.part / splits) + r.row / kProductHalf;
            if (product_part(r, part(w, r, w.part), ticket, splits)) store_square<true>(w, r, s);
        } else if (kind < 2)
            store_square<false>(w, r, s);
        else
            store_step(w, r, s);
    }
    __device__ __forceinline__ float4* part(const ProductUnit& w, const ProductRead& r, uint32_t number) const {
        return parts + ((uint64_t)number * (w.width / 4) + r.column / 4) * kProductTile + r.row;
    }
    // A, or b A + c A A without its diagonal.  PARTS: the sums lie in parts.
    template <bool PARTS>
    __device__ __forceinline__ void store_square(const ProductUnit& w, const ProductRead& r, State& s) const {
        const uint32_t row = (uint32_t)(w.m + r.row), col = (uint32_t)(w.n + r.column);
        const bool polynomial = kind == 1;
        __half* to = (polynomial ? poly : gram) + ((uint64_t)w.z * side + row) * side_pitch + col;
#pragma unroll 1
        for (int k = 0; k < r.columns && col + k < side; k += 32) {
            const State now = s;
            load(w, r, k + 32, s);
            uint32_t v[32];
            if (PARTS) {
                product_sum(part(w, r, w.part / splits * splits) + k / 4 * kProductTile,
                            (uint64_t)(w.width / 4) * kProductTile, splits, v);
            } else {
                r.load(k, v);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (row >= side || col + k + 16 * h >= side) continue;
                float o[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = c * __uint_as_float(v[16 * h + i]);
                if (polynomial) {
                    float old[16];
                    ortho_unpack16(now.first[h], old);
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] = fmaf(b, old[i], o[i]);
                    if (row - (col + k + 16 * h) < 16) {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (row == col + k + 16 * h + i) {
                                diagonal[w.z * side_pitch + row] = o[i] * (1.0f / kOrthoGramScale);
                                o[i] = 0.0f;
                            }
                    }
                }
                ortho_store16(to + k + 16 * h, o);
            }
        }
    }
    // a X + diagonal * X + the product, or, no steps, X
    __device__ __forceinline__ void store_step(const ProductUnit& w, const ProductRead& r, State& s) const {
        const uint32_t row = (uint32_t)(w.m + r.row), col = (uint32_t)(w.n + r.column);
        const uint64_t at = ((uint64_t)w.z * rows + row) * pitch + col;
        const bool last = out && (kind == 3 || 3 * step + 3 == phases);
        ProductRows to = {};
        if (last)
            to = product_rows(static_cast<char*>(out) + (target.dtype == NC_DTYPE_F32 ? 4 : 2) *
                                                            (w.z * out_distance),
                              target.dtype, ldo, row - r.lane, rows, col, r.lane);
        const bool by_column = kind == 2 && tall;
        const float of_row =
            kind == 2 && !tall && row < rows ? __ldcg(diagonal + w.z * side_pitch + row) : 0.0f;
        __half* next = self->high[from ^ 1];
#pragma unroll 1
        for (int k = 0; k < r.columns && col + k < cols; k += 32) {
            const State now = s;
            load(w, r, k + 32, s);
            if (by_column) {             // the diagonal of the columns, a lane's each, for all lanes
                __syncwarp();
                r.rows[r.lane] = now.of_column;
                __syncwarp();
            }
            uint32_t v[32];
            r.load(k, v);
            float o[32];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (row >= rows || col + k + 16 * h >= cols) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[16 * h + i] = 0.0f;
                    continue;
                }
                float x[16], y[16];
                ortho_unpack16(now.first[h], x);
                ortho_unpack16(now.second[h], y);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float all = fmaf(y[i], 1.0f / kOrthoLow, x[i]);
                    const float product = fmaf(by_column ? r.rows[16 * h + i] : of_row, x[i],
                                               __uint_as_float(v[16 * h + i]) * (1.0f / kOrthoGramScale));
                    x[i] = fmaf(a, all, product);
                    o[16 * h + i] = scale * x[i];
                }
                if (!last) {
                    Bytes32 first, second;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float p, q;
                        first.v[i] = pack2<__half>(x[2 * i], x[2 * i + 1]);
                        unpack2<__half>(first.v[i], p, q);
                        second.v[i] = pack2<__half>((x[2 * i] - p) * kOrthoLow,
                                                    (x[2 * i + 1] - q) * kOrthoLow);
                    }
                    st_wide(next + at + k + 16 * h, first);
                    st_wide(low + at + k + 16 * h, second);
                }
            }
            if (last)
                product_store(target, to, k, (int)(cols - col) - k, o, r);
        }
    }
};

struct OrthoPlan {
    uint64_t side, pitch, side_pitch;
    int blocks;
    size_t parts, high[2], low, gram, poly, diagonal, arrived, sums, bytes;
    uint32_t splits;
};

static size_t ortho_place(size_t& at, size_t bytes) {
    const size_t here = at;
    at = (at + bytes + 255) & ~(size_t)255;
    return here;
}

static bool ortho_fits(size_t batch, size_t rows, size_t cols) {
    const size_t most = (size_t)1 << 20;
    if (rows > most || cols > most || batch > 65535) return false;
    const uint64_t tiles = ((rows + 255) / 256) * ((cols + 255) / 256);
    return tiles * (batch ? batch : 1) < ((uint64_t)1 << 31) && batch * rows < ((uint64_t)1 << 31);
}

// Whether nothing that is held in binary16 overflows, whatever the matrix: A, whose entries are at most s^2 for
// the largest singular value s of X, and the polynomial's, at most |b s^2 + c s^4| for one of them, both times
// 256.  The singular values are at most 1 before the first step, and at most the largest of |a s + b s^3 + c s^5|
// after one.  (240: 6 % below what overflows, for the roundings.  Beyond it inf met 0 and all became NaN.)
static bool ortho_bounded(const float* coefficients, int steps) {
    double top = 1.0;
    for (int i = 0; i < steps; ++i) {
        const double a = coefficients[3 * i], b = coefficients[3 * i + 1], c = coefficients[3 * i + 2];
        const double square = top * top;
        const auto poly = [&](double u) { return fabs(b * u + c * u * u); };
        const auto next = [&](double u) { return fabs(sqrt(u) * (a + b * u + c * u * u)); };
        if (!(square <= 240.0 && poly(square) <= 240.0)) return false;
        const double middle = -b / (2.0 * c);            // where the slope of b u + c u u is 0
        if (middle > 0.0 && middle < square && !(poly(middle) <= 240.0)) return false;
        // the slope of the step is 0 where a + 3 b u + 5 c u u is; with c = 0, or nearly so, at -a / 3 b
        top = next(square);
        const double root = sqrt(9.0 * b * b - 20.0 * a * c), q = -0.5 * (3.0 * b + (b < 0.0 ? -root : root));
        const double at[2] = {q / (5.0 * c), a / q};
        for (double u : at)
            if (u > 0.0 && u < square && next(u) > top) top = next(u);
    }
    return true;
}

static OrthoPlan ortho_plan(uint64_t batch, uint64_t rows, uint64_t cols) {
    OrthoPlan p = {};
    p.side = rows < cols ? rows : cols;
    p.pitch = (cols + 15) / 16 * 16;
    p.side_pitch = (p.side + 15) / 16 * 16;
    const uint64_t blocks = (rows * ((cols + 7) / 8) + 1023) / 1024;     // four groups of eight a thread
    p.blocks = (int)(blocks < 1 ? 1 : blocks > kOrthoNormBlocks ? kOrthoNormBlocks : blocks);
    size_t at = 0;
    p.parts = ortho_place(at, 8 * batch * p.blocks);
    for (int i = 0; i < 2; ++i) p.high[i] = ortho_place(at, 2 * batch * rows * p.pitch);
    p.low = ortho_place(at, 2 * batch * rows * p.pitch);
    p.gram = ortho_place(at, 2 * batch * p.side * p.side_pitch);
    p.poly = ortho_place(at, 2 * batch * p.side * p.side_pitch);
    p.diagonal = ortho_place(at, 4 * batch * p.side_pitch);
    p.arrived = ortho_place(at, 4 * (kOrthoLaunches + 2 * kProductPairs));
    // Long sums of A by few tiles are split over the idle pairs, four steps a part at least.
    const uint64_t tiles = (p.side + 255) / 256, squares = tiles * (tiles + 1) / 2 * batch;
    const uint64_t steps = ((rows < cols ? cols : rows) + kProductStep - 1) / kProductStep;
    p.splits = 1;
    if (squares < kProductPairs && steps >= kOrthoLong) {
        const ProductSplit s = product_split((uint32_t)squares);
        const uint64_t units = s.units((uint32_t)squares), most = kProductPairs / units;
        p.splits = (uint32_t)(most < steps / 4 ? most : steps / 4);
        if (p.splits > 1)
            p.sums = ortho_place(at, 4 * units * p.splits * kProductTile * (kProductTile / s.parts));
    }
    p.bytes = at;
    return p;
}

template <typename T>
static void ortho_start(const OrthoInput& in, unsigned batch, cudaStream_t stream) {
    launch_overlapping(ortho_norm_kernel<T>, dim3(in.blocks, batch), dim3(256), 0, stream, in);
    const uint64_t blocks = (in.rows * (in.pitch / 8) + 255) / 256;
    launch_overlapping(ortho_start_kernel<T>, dim3((unsigned)(blocks < 1184 ? blocks : 1184), batch),
                       dim3(256), 0, stream, in);
}

}  // namespace natcomp

using namespace natcomp;

extern "C" {

size_t nc_orthogonalize_workspace_bytes(size_t batch, size_t rows, size_t cols) {
    return ortho_fits(batch, rows, cols) ? ortho_plan(batch, rows, cols).bytes : 0;
}

nc_status nc_orthogonalize(const void* g, int dtype, size_t batch, size_t rows, size_t cols,
                           size_t ldg, size_t distance, const float* coefficients, int steps, float eps,
                           float scale, void* out, int out_dtype, size_t ldo, size_t out_distance,
                           void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    const int bytes = act8_type_bytes(dtype), out_bytes = act8_type_bytes(out_dtype);
    if (!bytes || !out_bytes) return NC_ERR_UNSUPPORTED;
    if (steps < 0 || (steps && !coefficients) || !(eps >= 0.0f)) return NC_ERR_INVALID;
    if (batch == 0 || rows == 0 || cols == 0) return NC_OK;
    if (!g || !out || !workspace || ldg < cols || ldo < cols) return NC_ERR_INVALID;
    if (!ortho_fits(batch, rows, cols) || steps > kOrthoSteps * kOrthoLaunches) return NC_ERR_TOO_LARGE;
    if (!ortho_bounded(coefficients, steps)) return NC_ERR_INVALID;
    if (batch > 1 && (distance < (rows - 1) * ldg + cols || out_distance < (rows - 1) * ldo + cols))
        return NC_ERR_INVALID;
    if (!element_aligned(g, bytes) || !element_aligned(out, out_bytes) || !aligned32(workspace))
        return NC_ERR_ALIGN;
    const OrthoPlan p = ortho_plan(batch, rows, cols);
    if (workspace_bytes < p.bytes) return NC_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    __half* high[2] = {reinterpret_cast<__half*>(ws + p.high[0]),
                       reinterpret_cast<__half*>(ws + p.high[1])};
    __half* low = reinterpret_cast<__half*>(ws + p.low);
    __half* gram = reinterpret_cast<__half*>(ws + p.gram);
    __half* poly = reinterpret_cast<__half*>(ws + p.poly);
    float* diagonal = reinterpret_cast<float*>(ws + p.diagonal);
    const uint64_t longer = rows > cols ? rows : cols;
    const bool tall = rows > cols;
    int exponent = 0;                    // 2^exponent about the root of the longer side
    while (((uint64_t)1 << (2 * (exponent + 1))) <= longer) ++exponent;
    const float up = (float)(1 << exponent);

    OrthoInput in = {};
    in.g = g; in.dtype = dtype; in.rows = rows; in.cols = cols; in.ldg = ldg;
    in.distance = batch > 1 ? distance : 0;
    in.vector = row_access(g, ldg, bytes, rows) != kRowElement &&
                (batch == 1 || distance * bytes % 16 == 0);
    in.parts = reinterpret_cast<double*>(ws + p.parts); in.blocks = p.blocks;
    in.eps = eps; in.scale = up; in.high = high[0]; in.low = low; in.pitch = p.pitch;
    in.arrived = reinterpret_cast<uint32_t*>(ws + p.arrived);
    in.words = kOrthoLaunches + 2 * kProductPairs;
    if (dtype == NC_DTYPE_F32) ortho_start<float>(in, (unsigned)batch, stream);
    else if (dtype == NC_DTYPE_BF16) ortho_start<__nv_bfloat16>(in, (unsigned)batch, stream);
    else ortho_start<__half>(in, (unsigned)batch, stream);

    OrthoJob t = {};
    const uint64_t side_distance = p.side * p.side_pitch;
    for (int i = 0; i < 2; ++i)
        if (!make_box_map(&t.x_map[i], high[i], false, batch, rows, cols, p.pitch, rows * p.pitch))
            return NC_ERR_CUDA;
    if (!make_box_map(&t.gram_map, gram, false, batch, p.side, p.side, p.side_pitch, side_distance) ||
        !make_box_map(&t.poly_map, poly, false, batch, p.side, p.side, p.side_pitch, side_distance))
        return NC_ERR_CUDA;
    t.tall = tall; t.rows = (uint32_t)rows; t.cols = (uint32_t)cols; t.side = (uint32_t)p.side;
    t.batch = (uint32_t)batch; t.tiles = (uint32_t)((p.side + 255) / 256);
    t.tiles_m = (uint32_t)((rows + 255) / 256); t.tiles_n = (uint32_t)((cols + 255) / 256);
    t.pitch = p.pitch; t.side_pitch = p.side_pitch;
    t.high[0] = high[0]; t.high[1] = high[1]; t.low = low; t.gram = gram; t.poly = poly;
    t.diagonal = diagonal; t.gram_scale = kOrthoGramScale / (up * up);
    t.splits = p.splits; t.parts = reinterpret_cast<float4*>(ws + p.sums);
    t.tickets = in.arrived + kOrthoLaunches;
    t.ldo = ldo; t.out_distance = batch > 1 ? out_distance : 0; t.scale = scale / up;
    t.target.dtype = out_dtype;
    t.target.access = row_access(out, ldo, out_bytes, rows);
    if (batch > 1) {                     // every matrix starts where the first one might
        const size_t apart = out_distance * out_bytes;
        if (apart % 16) t.target.access = kRowElement;
        else if (apart % 32 && t.target.access == kRowWide) t.target.access = kRow16;
    }
    const uint64_t squares = (uint64_t)t.tiles * (t.tiles + 1) / 2 * batch;
    const uint64_t whole = (uint64_t)t.tiles_m * t.tiles_n * batch;
    for (int i = 0; i == 0 || i < steps; i += kOrthoSteps) {
        const int n = steps - i < kOrthoSteps ? steps - i : kOrthoSteps;
        t.phases = n ? 3 * n : 1;
        for (int k = 0; k < 3 * n; ++k) t.of_step[k] = coefficients[3 * i + k];
        t.turn = i & 1;
        t.out = i + n == steps ? out : nullptr;
        t.arrived = in.arrived + i / kOrthoSteps;
        const nc_status st = product_launch(t, 4 * (squares > whole ? squares : whole) * p.splits, stream);
        if (st != NC_OK) return st;
    }
    return launch_status();
}

}  // extern "C"
