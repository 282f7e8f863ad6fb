// Forward and backward pass of the cross entropy on the host model, against sums in 64 bits.
// Arguments: rows width vocabulary type(bf16|f16) layout(whole|any) without(every n-th row has no target;
// 0: all have one) dtable(same|f32) accumulate(0|1) dlse(0|1) seed, then name=value pairs.
using namespace natcomp;

static bool g_bf16;
static uint16_t bits_of(float v) {
    uint16_t h;
    if (g_bf16) { const __nv_bfloat16 b = __float2bfloat16_rn(v); memcpy(&h, &b, 2); }
    else { const __half b = __float2half_rn(v); memcpy(&h, &b, 2); }
    return h;
}
static double value_of(uint16_t h) { return model_value_of(h, g_bf16); }

int main(int argc, char** argv) {
    if (argc < 11) return 2;
    const size_t t = atol(argv[1]), d = atol(argv[2]), v = atol(argv[3]);
    g_bf16 = std::string(argv[4]) == "bf16";
    const bool any = std::string(argv[5]) == "any", f32 = std::string(argv[7]) == "f32";
    const size_t without = atol(argv[6]);
    const bool acc = atoi(argv[8]), with_dlse = atoi(argv[9]);
    model::rng.seed(atoi(argv[10]));
    const bool injected = ::injected(argc, argv, 11);
    model::cluster_of[(const void*)product_kernel<CeLogits<false>>] = 2;
    model::cluster_of[(const void*)product_kernel<CeLogits<true>>] = 2;
    model::cluster_of[(const void*)product_kernel<CeDz<__nv_bfloat16>>] = 2;
    model::cluster_of[(const void*)product_kernel<CeDz<__half>>] = 2;
    model::cluster_of[(const void*)product_kernel<CeDx>] = 2;
    model::cluster_of[(const void*)product_kernel<CeDtable>] = 2;
    const int dtype = g_bf16 ? NC_DTYPE_BF16 : NC_DTYPE_F16;
    std::mt19937 g(7);
    std::normal_distribution<float> normal;
    const size_t ld = any ? d + 3 : (d + 7) / 8 * 8, off = any ? 1 : 0;
    const float scale = 0.75f, nan = NAN;
    Held xh(((t ? t - 1 : 0) * ld + (t ? d : 0)) * 2, off * 2), wh(((v - 1) * ld + d) * 2, off * 2);
    Held th(t * 8), lossh(t * 4), lseh(t * 4), dlh(t * 4), dsh(t * 4);
    Held dxh(((t ? t - 1 : 0) * ld + (t ? d : 0)) * 2, off * 2);
    const int wb = f32 ? 4 : 2;
    Held dwh(((v - 1) * ld + d) * wb, off * wb);
    uint16_t *x = (uint16_t*)xh.p, *w = (uint16_t*)wh.p, *dx = (uint16_t*)dxh.p;
    long long* target = (long long*)th.p;
    float *dl = (float*)dlh.p, *ds = (float*)dsh.p, *loss = (float*)lossh.p, *lse = (float*)lseh.p;
    std::vector<double> old(v * d);
    for (size_t i = 0; i < v; ++i)
        for (size_t j = 0; j < d; ++j) {
            w[i * ld + j] = bits_of(2 * normal(g) / sqrtf((float)d));
            const float o = normal(g);
            if (f32) ((float*)dwh.p)[i * ld + j] = o; else ((uint16_t*)dwh.p)[i * ld + j] = bits_of(o);
            old[i * d + j] = f32 ? o : value_of(((uint16_t*)dwh.p)[i * ld + j]);
        }
    for (size_t i = 0; i < t; ++i) {
        const bool counts = !without || i % without != 1 % without;
        target[i] = counts ? (long long)(g() % v) : -1 - (long long)(g() % 5);
        for (size_t j = 0; j < d; ++j) x[i * ld + j] = counts ? bits_of(normal(g)) : bits_of(nan);
        dl[i] = counts ? 1e-3f * (1 + (float)(g() % 100)) : nan;
        ds[i] = counts ? 1e-3f * normal(g) : nan;
    }
    const size_t fb = nc_linear_cross_entropy_forward_workspace_bytes(t, d, v);
    const size_t bb = nc_linear_cross_entropy_backward_workspace_bytes(t, d, v);
    {
        Held ws(fb);
        const nc_status st = nc_linear_cross_entropy_forward(x, dtype, t, d, ld, w, v, ld, target, 8,
                                                             scale, loss, lse, ws.p, fb, nullptr);
        if (st != NC_OK) { printf("forward: status %d\n", (int)st); return 1; }
    }
    size_t wrong = 0, lost = 0, values = 0;
    const double u = ldexp(1.0, -24), r16 = ldexp(1.0, g_bf16 ? -8 : -11);
    std::vector<double> z(t * v), want_lse(t), ez(t);
    for (size_t i = 0; i < t; ++i) {
        if (target[i] < 0) {
            wrong += loss[i] != 0 || lse[i] != 0;
            continue;
        }
        double top = -1e300, most = 0;
        for (size_t k = 0; k < v; ++k) {
            double s = 0, m = 0;
            for (size_t j = 0; j < d; ++j) {
                const double p = value_of(x[i * ld + j]) * value_of(w[k * ld + j]);
                s += p;
                m += fabs(p);
            }
            z[i * v + k] = scale * s;
            top = std::max(top, scale * s);
            most = std::max(most, scale * m);
        }
        double s = 0;
        for (size_t k = 0; k < v; ++k) s += exp(z[i * v + k] - top);
        want_lse[i] = top + log(s);
        // a sum of d products in 32 bits, and four roundings of the exponent's argument
        ez[i] = (d + 8) * u * most;
        const double tol = ez[i] + (v + 16) * u + 8 * u * fabs(want_lse[i]);
        const double want = want_lse[i] - z[i * v + target[i]];
        values += 2;
        if (std::isnan(lse[i])) ++lost;
        else if (!(fabs(lse[i] - want_lse[i]) <= tol)) ++wrong;
        if (std::isnan(loss[i])) ++lost;
        else if (!(fabs(loss[i] - want) <= 2 * tol)) ++wrong;
    }
    if (wrong || (lost && !injected)) {
        printf("forward: %zu wrong values, %zu NaN\n", wrong, lost);
        return 1;
    }
    for (size_t i = 0; i < t; ++i) lse[i] = target[i] < 0 ? nan : (float)want_lse[i];
    {
        Held ws(bb);
        const nc_status st = nc_linear_cross_entropy_backward(
            x, dtype, t, d, ld, w, v, ld, target, 8, scale, lse, dl, with_dlse ? ds : nullptr, dx, ld,
            dwh.p, f32 ? NC_DTYPE_F32 : dtype, ld, acc, ws.p, bb, nullptr);
        if (st != NC_OK) { printf("backward: status %d\n", (int)st); return 1; }
    }
    if (model::any_ran_out != injected) {
        printf("waits %s\n", model::any_ran_out ? "ran out of time" : "did not run out of time");
        return 1;
    }
    double largest = 0;
    std::vector<double> dz(t * v), edz(t * v);
    for (size_t i = 0; i < t; ++i) {
        if (target[i] < 0) continue;
        const double a = dl[i], b = with_dlse ? ds[i] : 0.0;
        largest = std::max(largest, std::max(fabs(a), std::max(fabs(b), fabs(a + b))));
        for (size_t k = 0; k < v; ++k) {
            const double p = exp(z[i * v + k] - (double)lse[i]), hot = (long long)k == target[i];
            dz[i * v + k] = p * (a + b) - hot * a;
            // its rounding, and what the logit and the arithmetic before it are off by
            edz[i * v + k] = r16 * fabs(dz[i * v + k]) +
                             (p * fabs(a + b) + hot * fabs(a)) *
                                 (ez[i] + 8 * u * (1 + fabs(lse[i]) + fabs(z[i * v + k])));
        }
    }
    for (auto& e : edz) e += largest * ldexp(1.0, g_bf16 ? -120 : -38);      // subnormal numbers
    for (size_t i = 0; i < t; ++i)
        for (size_t j = 0; j < d; ++j) {
            double s = 0, m = 0, e = 0;
            if (target[i] >= 0)
                for (size_t k = 0; k < v; ++k) {
                    const double y = value_of(w[k * ld + j]);
                    s += dz[i * v + k] * y;
                    m += fabs(dz[i * v + k] * y);
                    e += edz[i * v + k] * fabs(y);
                }
            const double got = value_of(dx[i * ld + j]);
            ++values;
            if (std::isnan(got)) ++lost;
            else if (!(fabs(got - scale * s) <= scale * (e + (v + 8) * u * m) * 1.01 +
                                                    r16 * fabs(scale * s) * 1.01 + 1e-7)) ++wrong;
        }
    if (wrong) printf("dx: ");
    for (size_t k = 0; k < v && !wrong; ++k)
        for (size_t j = 0; j < d; ++j) {
            double s = 0, m = 0, e = 0;
            for (size_t i = 0; i < t; ++i) {
                if (target[i] < 0) continue;
                const double y = value_of(x[i * ld + j]);
                s += dz[i * v + k] * y;
                m += fabs(dz[i * v + k] * y);
                e += edz[i * v + k] * fabs(y);
            }
            const double want = scale * s + (acc ? old[k * d + j] : 0);
            const double got = f32 ? ((float*)dwh.p)[k * ld + j] : value_of(((uint16_t*)dwh.p)[k * ld + j]);
            ++values;
            if (std::isnan(got)) ++lost;
            else if (!(fabs(got - want) <= scale * (e + (t + 8) * u * m) * 1.01 +
                                               (f32 ? 4 * u : r16) * fabs(want) * 1.01 + 1e-7)) ++wrong;
        }
    if (wrong || (lost != 0) != injected) {
        printf("%zu wrong values, %zu NaN of %zu\n", wrong, lost, values);
        return 1;
    }
    printf("ok, %zu NaN of %zu, %zu launches\n", lost, values, model::launches);
    return 0;
}
