// Orthogonalised updates on the host model, against the same products in 64 bits.
// Arguments: batch rows cols in(f32|bf16|f16) out(f32|bf16|f16) layout(whole|any) steps seed, then
// name=value pairs.
using namespace natcomp;

static float get(const uint8_t* p, int dtype, size_t i) {
    if (dtype == NC_DTYPE_F32) return ((const float*)p)[i];
    return model_value_of(((const uint16_t*)p)[i], dtype == NC_DTYPE_BF16);
}
static void put(uint8_t* p, int dtype, size_t i, float v) {
    if (dtype == NC_DTYPE_F32) { ((float*)p)[i] = v; return; }
    if (dtype == NC_DTYPE_BF16) ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(v);
    else ((__half*)p)[i] = __float2half_rn(v);
}
static int type_of(const std::string& s) {
    return s == "f32" ? NC_DTYPE_F32 : s == "bf16" ? NC_DTYPE_BF16 : NC_DTYPE_F16;
}
typedef std::vector<double> Matrix;
static Matrix times(const Matrix& a, const Matrix& b, size_t n, size_t k, size_t m, bool second_transposed) {
    Matrix c(n * m, 0.0);
    for (size_t i = 0; i < n; ++i)
        for (size_t l = 0; l < k; ++l)
            for (size_t j = 0; j < m; ++j)
                c[i * m + j] += a[i * k + l] * (second_transposed ? b[j * k + l] : b[l * m + j]);
    return c;
}

int main(int argc, char** argv) {
    if (argc < 9) return 2;
    const size_t batch = atol(argv[1]), rows = atol(argv[2]), cols = atol(argv[3]);
    const int in = type_of(argv[4]), out = type_of(argv[5]), steps = atoi(argv[7]);
    const bool any = std::string(argv[6]) == "any";
    model::rng.seed(atoi(argv[8]));
    const bool injected = ::injected(argc, argv, 9);
    model::cluster_of[(const void*)product_kernel<OrthoJob>] = 2;
    const int ib = in == NC_DTYPE_F32 ? 4 : 2, ob = out == NC_DTYPE_F32 ? 4 : 2;
    const size_t ld = any ? cols + 3 : cols, off = any ? 1 : 0, apart = rows * ld + (any ? 5 : 0);
    const size_t all = (batch - 1) * apart + (rows - 1) * ld + cols;
    Held gh(all * ib, off * ib), oh(all * ob, off * ob);
    std::mt19937 g(7);
    std::normal_distribution<float> normal;
    for (size_t b = 0; b < batch; ++b)
        for (size_t i = 0; i < rows; ++i)
            for (size_t j = 0; j < cols; ++j) put(gh.p, in, b * apart + i * ld + j, 1e-2f * normal(g));
    const size_t bytes = nc_orthogonalize_workspace_bytes(batch, rows, cols);
    Held ws(bytes);
    std::vector<float> co;
    for (int i = 0; i < steps; ++i) {
        co.push_back(3.4445f); co.push_back(-4.775f); co.push_back(2.0315f + 0.01f * i);
    }
    const float scale = 1.5f;
    const nc_status st = nc_orthogonalize(gh.p, in, batch, rows, cols, ld, apart, co.data(), steps, 1e-7f,
                                          scale, oh.p, out, ld, apart, ws.p, bytes, nullptr);
    if (st != NC_OK) { printf("status %d\n", (int)st); return 1; }
    if (model::any_ran_out != injected) {
        printf("waits %s\n", model::any_ran_out ? "ran out of time" : "did not run out of time");
        return 1;
    }
    const size_t n = std::min(rows, cols), m = std::max(rows, cols);
    size_t lost = 0;
    for (size_t b = 0; b < batch; ++b) {
        Matrix x(n * m);
        double norm = 0;
        for (size_t i = 0; i < rows; ++i)
            for (size_t j = 0; j < cols; ++j) {
                const double v = get(gh.p, in, b * apart + i * ld + j);
                x[rows <= cols ? i * m + j : j * m + i] = v;
                norm += v * v;
            }
        for (auto& v : x) v /= sqrt(norm) + 1e-7;
        for (int s = 0; s < steps; ++s) {
            const Matrix a = times(x, x, n, m, n, true), aa = times(a, a, n, n, n, false);
            Matrix p(n * n);
            for (size_t i = 0; i < n * n; ++i) p[i] = co[3 * s + 1] * a[i] + co[3 * s + 2] * aa[i];
            const Matrix y = times(p, x, n, n, m, false);
            for (size_t i = 0; i < n * m; ++i) x[i] = co[3 * s] * x[i] + y[i];
        }
        double off2 = 0, size2 = 0;
        for (size_t i = 0; i < rows; ++i)
            for (size_t j = 0; j < cols; ++j) {
                const double want = scale * x[rows <= cols ? i * m + j : j * m + i];
                const double got = get(oh.p, out, b * apart + i * ld + j);
                if (std::isnan(got)) { ++lost; continue; }
                off2 += (got - want) * (got - want);
                size2 += want * want;
            }
        // Roundings of a step, relative to the norm: half a step of binary16, 2^-11, for each of X, A
        // and the polynomial, times their coefficients (b, c, and the polynomial's largest value, at
        // most 3.5, where X itself is at least 0.6): below 2^-11 * 12; spread over the values by chance
        // a third of it.  Errors of earlier steps shrink or grow with the slope of the polynomial at the
        // singular values, at most 3.45 relative to growing X.  And the result's own rounding.
        const double tol = steps ? 8 * ldexp(1.0, -11) + (out == NC_DTYPE_BF16 ? ldexp(1.0, -8) : 0)
                                 : ldexp(1.0, out == NC_DTYPE_BF16 ? -8 : out == NC_DTYPE_F16 ? -10 : -20);
        if (!injected && !(sqrt(off2) <= tol * sqrt(size2))) {
            printf("matrix %zu is off by %.3g of its norm\n", b, sqrt(off2 / size2));
            return 1;
        }
    }
    if ((lost != 0) != injected) { printf("%zu NaN\n", lost); return 1; }
    printf("ok, %zu NaN, %zu launches\n", lost, model::launches);
    return 0;
}
