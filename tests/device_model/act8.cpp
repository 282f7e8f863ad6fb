// A checkpoint written and read back on the host model, bit for bit against the definition.
// Arguments: rows cols layout(whole|gap|any) random(0|1) seed.  T is the element type.
using namespace natcomp;

static float value(float v) { return v; }
static float value(__nv_bfloat16 v) { return __bfloat162float(v); }
static void set(float& d, float v) { d = v; }
static void set(__nv_bfloat16& d, float v) { d = __float2bfloat16_rn(v); }

int main(int argc, char** argv) {
    if (argc < 6) return 2;
    const size_t rows = atol(argv[1]), cols = atol(argv[2]);
    const std::string lay = argv[3];
    const bool random = atoi(argv[4]);
    model::rng.seed(atoi(argv[5]));
    const int dtype = sizeof(T) == 4 ? NC_DTYPE_F32 : NC_DTYPE_BF16;
    const size_t v16 = 16 / sizeof(T);
    const size_t ld = lay == "gap" ? (cols + v16 - 1) / v16 * v16 + v16 : lay == "any" ? cols + 1 : cols;
    const size_t off = lay == "gap" ? v16 : lay == "any" ? 1 : 0;
    const size_t size = ((rows - 1) * ld + cols) * sizeof(T), pitch = act8_pitch(cols);
    Held xh(size, off * sizeof(T)), yh(size, off * sizeof(T)), codes(rows * pitch), scales(rows * pitch / 32);
    std::mt19937 g(3);
    std::normal_distribution<float> normal;
    T *x = (T*)xh.p, *y = (T*)yh.p;
    for (size_t r = 0; r < rows; ++r)
        for (size_t c = 0; c < cols; ++c) set(x[r * ld + c], normal(g) * ldexpf(1.0f, (int)(g() % 20) - 10));
    if (rows * cols > 5) set(x[(rows - 1) * ld + cols / 2], INFINITY);
    const PhiloxKeys keys = make_philox_keys(9);
    nc_status st = nc_act8_compress(x, dtype, rows, cols, ld, random, 9, 2, codes.p, scales.p, nullptr);
    if (st == NC_OK) st = nc_act8_decompress(codes.p, scales.p, rows, cols, y, dtype, ld, nullptr);
    if (st != NC_OK) {
        printf("status %d\n", (int)st);
        return 1;
    }
    size_t wrong = 0;
    for (size_t r = 0; r < rows; ++r)
        for (size_t b = 0; b < pitch / 32; ++b) {
            double top = 0;
            for (size_t c = 32 * b; c < std::min(cols, 32 * b + 32); ++c)
                top = std::max(top, (double)fabsf(value(x[r * ld + c])));
            int e = -118;
            while (std::isfinite(top) && top > 127 * ldexp(1.0, e)) ++e;
            const int s = std::isfinite(top) ? e + 127 : 255;
            wrong += scales.p[r * pitch / 32 + b] != s;
            for (size_t c = 32 * b; c < 32 * b + 32; ++c) {
                const size_t j = r * pitch + c;
                const float v = c < cols ? value(x[r * ld + c]) : 0.0f;
                uint32_t word[4];
                philox4x32_10((uint32_t)(j / 16), 0, 2, 6, keys, word);
                const int draw = word[j % 16 / 4] >> (8 * (j % 4)) & 255;
                const double q = fabs(v) / ldexp(1.0, e);
                const int m = s == 255 ? 0 : random ? ((int)nearbyint(256 * q) + draw) / 256 : (int)nearbyint(q);
                const int code = s == 255 ? 0 : m | (std::signbit(v) ? 128 : 0);
                wrong += codes.p[j] != code;
                if (c >= cols) continue;
                const float back = value(y[r * ld + c]);
                wrong += s == 255 ? !std::isnan(back) : back != (code & 128 ? -1 : 1) * (float)(m * ldexp(1.0, e));
            }
        }
    printf(wrong ? "%zu wrong\n" : "ok\n", wrong);
    return wrong != 0;
}
