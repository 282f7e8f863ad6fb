// One weight gradient on the host model, against a product in 64 bits.
// Arguments: rows n k dy_layout(whole|gap|any) dw(f32|bf16) affine(0|1) accumulate(0|1) seed, then
// name=value pairs for what a test injects.  Prints "ok ..." or what is wrong.
using namespace natcomp;

int main(int argc, char** argv) {
    if (argc < 9) return 2;
    const size_t t = atol(argv[1]), n = atol(argv[2]), k = atol(argv[3]);
    const std::string lay = argv[4], kind = argv[5];
    const bool affine = atoi(argv[6]), acc = atoi(argv[7]);
    model::rng.seed(atoi(argv[8]));
    const bool injected = ::injected(argc, argv, 9);
    model::cluster_of[(const void*)wg_product_kernel<true, true>] = 2;
    model::cluster_of[(const void*)wg_product_kernel<true, false>] = 2;
    model::cluster_of[(const void*)wg_product_kernel<false, true>] = 2;
    model::cluster_of[(const void*)wg_product_kernel<false, false>] = 2;
    std::mt19937 g(7);
    std::normal_distribution<float> normal;
    const size_t ld = lay == "gap" ? (n + 7) / 8 * 8 + 8 : lay == "any" ? n + 3 : n;
    const size_t off = lay == "gap" ? 8 : lay == "any" ? 1 : 0;
    Held dyh((t ? (t - 1) * ld + n : 0) * 2, off * 2);
    __nv_bfloat16* dy = (__nv_bfloat16*)dyh.p;
    const size_t pitch = act8_pitch(k);
    Held codes(t * pitch), scales(t * pitch / 32);
    std::vector<double> x(t * k), y(t * n);
    for (size_t i = 0; i < t; ++i) {
        for (size_t j = 0; j < n; ++j) {
            dy[i * ld + j] = __float2bfloat16_rn(normal(g));
            y[i * n + j] = __bfloat162float(dy[i * ld + j]);
        }
        for (size_t b = 0; b < pitch / 32; ++b) {
            const int s = 120 + (int)(g() % 8);
            scales.p[i * pitch / 32 + b] = (uint8_t)s;
            for (size_t c = 32 * b; c < 32 * b + 32; ++c) {
                const uint8_t code = c < k ? (uint8_t)g() : 0;
                codes.p[i * pitch + c] = code;
                if (c < k) x[i * k + c] = (code & 128 ? -1 : 1) * ldexp(code & 127, s - 127);
            }
        }
    }
    const int wb = kind == "f32" ? 4 : 2;
    Held dwh(n * k * wb), dbh(n * 4), gam(k * 4), bet(k * 4);
    float *gamma = (float*)gam.p, *beta = (float*)bet.p, *db = (float*)dbh.p;
    for (size_t j = 0; j < k; ++j) {
        gamma[j] = 1 + 0.25f * normal(g);
        beta[j] = normal(g);
    }
    std::vector<double> old(n * k), oldb(n);
    for (size_t i = 0; i < n * k; ++i) {
        const float v = normal(g);
        if (wb == 4) ((float*)dwh.p)[i] = v; else ((__nv_bfloat16*)dwh.p)[i] = __float2bfloat16_rn(v);
        old[i] = wb == 4 ? v : __bfloat162float(((__nv_bfloat16*)dwh.p)[i]);
    }
    for (size_t i = 0; i < n; ++i) oldb[i] = db[i] = normal(g);
    const size_t bytes = nc_act8_weight_grad_workspace_bytes(t, n, k);
    Held ws(bytes);
    const nc_status st = nc_act8_weight_grad(
        dy, t, n, ld, codes.p, scales.p, k, affine ? gamma : nullptr, affine ? beta : nullptr,
        NC_DTYPE_F32, dwh.p, wb == 4 ? NC_DTYPE_F32 : NC_DTYPE_BF16, k, db, acc, ws.p, bytes, nullptr);
    if (st != NC_OK) {
        printf("status %d\n", (int)st);
        return 1;
    }
    if (model::any_ran_out != injected) {
        printf("waits %s\n", model::any_ran_out ? "ran out of time" : "did not run out of time");
        return 1;
    }
    // a sum in 32 bits, in any order, of t rounded products; the parameters and the result add a few
    const double u = ldexp(1.0, -24), round = wb == 4 ? u : ldexp(1.0, -8);
    std::vector<double> sum(n, 0.0), mag(n, 0.0);
    for (size_t i = 0; i < t; ++i)
        for (size_t j = 0; j < n; ++j) {
            sum[j] += y[i * n + j];
            mag[j] += fabs(y[i * n + j]);
        }
    size_t wrong = 0, lost = 0;
    for (size_t i = 0; i < n; ++i) {
        std::vector<double> want(k, 0.0), size(k, 0.0);
        for (size_t r = 0; r < t; ++r) {
            const double v = y[r * n + i];
            for (size_t j = 0; j < k; ++j) {
                const double p = v * x[r * k + j];
                want[j] += p;
                size[j] += fabs(p);
            }
        }
        for (size_t j = 0; j < k; ++j) {
            double w = want[j], s = size[j];
            if (affine) {
                w = w * gamma[j] + sum[i] * beta[j];
                s = s * fabs(gamma[j]) + mag[i] * fabs(beta[j]);
            }
            if (acc) w += old[i * k + j];
            const double tol = (t + 8) * u * s + (round + u) * fabs(w) + (acc ? u * fabs(w) : 0) + 1e-30;
            const double got = wb == 4 ? ((float*)dwh.p)[i * k + j]
                                       : __bfloat162float(((__nv_bfloat16*)dwh.p)[i * k + j]);
            if (std::isnan(got)) ++lost;
            else if (!(fabs(got - w) <= tol * 1.01)) ++wrong;
        }
        const double wb0 = sum[i] + (acc ? oldb[i] : 0);
        if (!(fabs(db[i] - wb0) <= (t + 8) * u * mag[i] + u * fabs(wb0))) ++wrong;
    }
    if (wrong || (lost != 0) != injected) {
        printf("%zu wrong values, %zu NaN of %zu\n", wrong, lost, n * k);
        return 1;
    }
    printf("ok, %zu NaN of %zu, %zu launches\n", lost, n * k, model::launches);
    return 0;
}
