// Layer norm on the host model, against the formulas in 64 bits.
// Arguments: forward|backward rows cols layout(whole|gap|any) kept(none|nearest|random; backward: the
// saved input or the checkpoint) gamma(0|1) residual(0|1) accumulate(0|1) sms seed, then name=value
// pairs for what a test injects.  T is the element type.  Prints "ok ..." or what is wrong.
using namespace natcomp;

static float value(float v) { return v; }
static float value(__nv_bfloat16 v) { return __bfloat162float(v); }
static void set(float& d, float v) { d = v; }
static void set(__nv_bfloat16& d, float v) { d = __float2bfloat16_rn(v); }

int main(int argc, char** argv) {
    if (argc < 11) return 2;
    const std::string op = argv[1], lay = argv[4], kept = argv[5];
    const size_t rows = atol(argv[2]), cols = atol(argv[3]);
    const bool with_gamma = atoi(argv[6]), res = atoi(argv[7]), acc = atoi(argv[8]);
    model::sms = atoi(argv[9]);
    model::rng.seed(atoi(argv[10]));
    const bool injected = ::injected(argc, argv, 11);
    const int dtype = sizeof(T) == 4 ? NC_DTYPE_F32 : NC_DTYPE_BF16;
    const double u = ldexp(1.0, -24), round = sizeof(T) == 4 ? u : ldexp(1.0, -8);
    std::mt19937 g(5);
    std::normal_distribution<float> normal;
    const size_t v16 = 16 / sizeof(T);
    const size_t ld = lay == "gap" ? (cols + v16 - 1) / v16 * v16 + v16 : lay == "any" ? cols + 1 : cols;
    const size_t off = lay == "gap" ? v16 : lay == "any" ? 1 : 0;
    const size_t size = ((rows - 1) * ld + cols) * sizeof(T);
    auto matrix = [&](Held& h, std::vector<double>& v, float scale, float shift) {
        v.resize(rows * cols);
        for (size_t r = 0; r < rows; ++r)
            for (size_t c = 0; c < cols; ++c) {
                set(((T*)h.p)[r * ld + c], scale * normal(g) + shift);
                v[r * cols + c] = value(((T*)h.p)[r * ld + c]);
            }
    };
    Held xh(size, off * sizeof(T)), yh(size, off * sizeof(T)), dyh(size, off * sizeof(T)),
        dresh(size, off * sizeof(T));
    Held gam(cols * 4, 4), bet(cols * 4), meanh(rows * 4), rstdh(rows * 4);
    const size_t pitch = act8_pitch(cols);
    Held codes(rows * pitch), scales(rows * pitch / 32);
    float *gamma = (float*)gam.p, *beta = (float*)bet.p, *mean = (float*)meanh.p, *rstd = (float*)rstdh.p;
    std::vector<double> x, dy, dres;
    matrix(xh, x, 1.5f, 0.5f);
    for (size_t c = 0; c < cols; ++c) {
        gamma[c] = 1 + 0.25f * normal(g);
        beta[c] = normal(g);
    }
    std::vector<double> m64(rows, 0.0), r64(rows, 0.0), n64(rows * cols);
    for (size_t r = 0; r < rows; ++r) {
        for (size_t c = 0; c < cols; ++c) m64[r] += x[r * cols + c] / cols;
        for (size_t c = 0; c < cols; ++c) r64[r] += pow(x[r * cols + c] - m64[r], 2) / cols;
        r64[r] = 1 / sqrt(r64[r] + 1e-5);
        for (size_t c = 0; c < cols; ++c) n64[r * cols + c] = (x[r * cols + c] - m64[r]) * r64[r];
    }
    size_t wrong = 0, lost = 0, all = 0;
    auto check = [&](double got, double want, double tol) {
        ++all;
        if (std::isnan(got)) ++lost;
        else if (!(fabs(got - want) <= tol)) ++wrong;
    };
    nc_status st;
    if (op == "forward") {
        const bool keep = kept != "none";
        st = nc_layer_norm_forward(xh.p, dtype, rows, cols, ld, with_gamma ? gamma : nullptr,
                                   with_gamma ? beta : nullptr, NC_DTYPE_F32, 1e-5f, yh.p, ld, mean,
                                   rstd, keep ? codes.p : nullptr, keep ? scales.p : nullptr,
                                   kept == "random" ? NC_ROUND_RANDOM : NC_ROUND_NEAREST, 7, 1, nullptr);
        for (size_t r = 0; r < rows; ++r) {
            const double e = 300 * u * (1 + 1.5 * r64[r]);           // of a normalised value
            check(mean[r], m64[r], 200 * u * 2);
            check(rstd[r], r64[r], 200 * u * 2 * r64[r] * (1 + r64[r]));
            for (size_t c = 0; c < cols; ++c) {
                const double n = n64[r * cols + c], k = with_gamma ? gamma[c] : 1;
                const double w = n * k + (with_gamma ? beta[c] : 0);
                const double en = e * (1 + fabs(n)) * (1 + r64[r]);
                check(value(((T*)yh.p)[r * ld + c]), w, round * (fabs(w) + 1e-3) + en * fabs(k) + 8 * u * fabs(w) + 1e-6);
                if (!keep) continue;
                const int s = scales.p[(r * pitch + c) / 32], code = codes.p[r * pitch + c];
                const double unit = ldexp(1.0, s - 127);
                if (s == 255) ++lost, ++all;
                else check((code & 128 ? -1 : 1) * (code & 127) * unit, n, unit * 1.01 + en);
            }
        }
    } else {
        matrix(dyh, dy, 1.0f, 0.25f);
        matrix(dresh, dres, 1.0f, 0.0f);
        const bool saved8 = kept != "none";
        for (size_t r = 0; r < rows; ++r) {
            mean[r] = (float)m64[r];
            rstd[r] = (float)r64[r];
            for (size_t b = 0; b < pitch / 32; ++b) {
                const int s = 121 + (int)(g() % 3);
                scales.p[r * pitch / 32 + b] = (uint8_t)s;
                for (size_t c = 32 * b; c < 32 * b + 32; ++c) {
                    const int code = c < cols ? (int)(g() & 255) : 0;
                    codes.p[r * pitch + c] = (uint8_t)code;
                    if (c >= cols) continue;
                    n64[r * cols + c] = saved8 ? (code & 128 ? -1 : 1) * ldexp(code & 127, s - 127)
                                               : (x[r * cols + c] - mean[r]) * (double)rstd[r];
                }
            }
        }
        Held dgh(cols * 4, 4), dbh(cols * 4, 8);
        float *dg = (float*)dgh.p, *db = (float*)dbh.p;
        std::vector<double> old(cols);
        for (size_t c = 0; c < cols; ++c) old[c] = dg[c] = db[c] = normal(g);
        const size_t bytes = nc_layer_norm_workspace_bytes(rows, cols);
        Held ws(bytes);
        const float* ga = with_gamma ? gamma : nullptr;
        const void* dr = res ? dresh.p : nullptr;
        st = saved8 ? nc_act8_layer_norm_backward(dyh.p, dtype, rows, cols, ld, codes.p, scales.p, rstd,
                                                  ga, NC_DTYPE_F32, dr, ld, yh.p, ld, dg, db, acc, ws.p,
                                                  bytes, nullptr)
                    : nc_layer_norm_backward(dyh.p, dtype, rows, cols, ld, xh.p, ld, mean, rstd, ga,
                                             NC_DTYPE_F32, dr, ld, yh.p, ld, dg, db, acc, ws.p, bytes,
                                             nullptr);
        std::vector<double> wg(cols, 0.0), wb(cols, 0.0), mg(cols, 0.0), mb(cols, 0.0);
        for (size_t r = 0; r < rows; ++r) {
            double m1 = 0, m2 = 0, a1 = 0, a2 = 0;
            for (size_t c = 0; c < cols; ++c) {
                const double d = dy[r * cols + c], q = d * (with_gamma ? gamma[c] : 1), n = n64[r * cols + c];
                m1 += q / cols;
                m2 += q * n / cols;
                a1 += fabs(q) / cols;
                a2 += fabs(q * n) / cols;
                wg[c] += d * n;
                wb[c] += d;
                mg[c] += fabs(d * n);
                mb[c] += fabs(d);
            }
            for (size_t c = 0; c < cols; ++c) {
                const double q = dy[r * cols + c] * (with_gamma ? gamma[c] : 1), n = n64[r * cols + c];
                double w = rstd[r] * (q - m1 - n * m2);
                const double mag = rstd[r] * (fabs(q) + a1 + fabs(n) * a2);
                if (res) w += dres[r * cols + c];
                check(value(((T*)yh.p)[r * ld + c]), w, round * fabs(w) + 200 * u * mag + 2 * u * fabs(w) + 1e-30);
            }
        }
        for (size_t c = 0; c < cols; ++c) {
            const double o = acc ? old[c] : 0;
            check(dg[c], wg[c] + o, (rows + 20) * 4 * u * mg[c] + u * fabs(wg[c] + o) + 1e-30);
            check(db[c], wb[c] + o, (rows + 20) * u * mb[c] + u * fabs(wb[c] + o) + 1e-30);
        }
    }
    if (st != NC_OK) {
        printf("status %d\n", (int)st);
        return 1;
    }
    if (model::any_ran_out != injected) {
        printf("waits %s\n", model::any_ran_out ? "ran out of time" : "did not run out of time");
        return 1;
    }
    if (wrong || (lost != 0) != injected) {
        printf("%zu wrong values, %zu NaN of %zu\n", wrong, lost, all);
        return 1;
    }
    printf("ok, %zu NaN of %zu, at most %lld limits of waiting\n", lost, all,
           model::longest / model::kWaitLimit);
    return 0;
}
