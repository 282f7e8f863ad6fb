// Embedding and its gradient on the host model, against sums in 64 bits.
// Arguments: rows vocabulary cols type out layout(whole|any) kind(few|many|one|none) token_bytes
// accumulate seed.
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

int main(int argc, char** argv) {
    if (argc < 11) return 2;
    const size_t t = atol(argv[1]), v = atol(argv[2]), d = atol(argv[3]);
    const int ty = type_of(argv[4]), to = type_of(argv[5]), bytes = atoi(argv[8]);
    const bool any = std::string(argv[6]) == "any", acc = atoi(argv[9]);
    const std::string kind = argv[7];
    model::rng.seed(atoi(argv[10]));
    const int tb = ty == NC_DTYPE_F32 ? 4 : 2, ob = to == NC_DTYPE_F32 ? 4 : 2;
    const size_t ld = any ? d + 3 : (d + 7) / 8 * 8, off = any ? 1 : 0;
    std::mt19937 g(7);
    std::normal_distribution<float> normal;
    auto matrix = [&](size_t rows) { return rows ? (rows - 1) * ld + d : 0; };
    Held tok(t * bytes), table(matrix(v) * tb, off * tb), out(matrix(t) * ob, off * ob);
    Held dy(matrix(t) * tb, off * tb), dt(matrix(v) * ob, off * ob);
    std::vector<long long> token(t);
    for (size_t i = 0; i < t; ++i) {
        long long k = kind == "one" ? (long long)(v / 2) : kind == "few" ? (long long)(g() % 3 * (v / 3))
                                                                         : (long long)(g() % v);
        if (kind == "none" || (kind == "many" && g() % 9 == 0)) k = -1 - (long long)(g() % 3);
        if (kind == "many" && g() % 50 == 0) k = (long long)(v + g() % 2);
        token[i] = k;
        if (bytes == 8) ((long long*)tok.p)[i] = k; else ((int*)tok.p)[i] = (int)k;
        for (size_t j = 0; j < d; ++j)
            put(dy.p, ty, i * ld + j, k < 0 || k >= (long long)v ? NAN : normal(g));
    }
    std::vector<double> old(v * d), sum(v * d, 0.0), mag(v * d, 0.0);
    std::vector<size_t> times(v, 0);
    for (size_t i = 0; i < v; ++i)
        for (size_t j = 0; j < d; ++j) {
            put(table.p, ty, i * ld + j, normal(g));
            put(dt.p, to, i * ld + j, normal(g));
            old[i * d + j] = get(dt.p, to, i * ld + j);
        }
    const float scale = 1.7f;
    nc_status st = nc_embedding_forward(tok.p, bytes, t, table.p, ty, v, d, ld, scale, out.p, to, ld, nullptr);
    if (st != NC_OK) { printf("forward: status %d\n", (int)st); return 1; }
    const double r = to == NC_DTYPE_F32 ? ldexp(1.0, -24) : ldexp(1.0, to == NC_DTYPE_BF16 ? -8 : -11);
    const double u = ldexp(1.0, -24);
    size_t wrong = 0;
    for (size_t i = 0; i < t; ++i)
        for (size_t j = 0; j < d; ++j) {
            const double got = get(out.p, to, i * ld + j);
            if (token[i] < 0) wrong += got != 0;
            else if (token[i] >= (long long)v) wrong += !std::isnan(got);
            else {
                const double want = scale * (double)get(table.p, ty, token[i] * ld + j);
                wrong += !(fabs(got - want) <= 1.01 * (r + u) * fabs(want) + 1e-7);
                sum[token[i] * d + j] += get(dy.p, ty, i * ld + j);
                mag[token[i] * d + j] += fabs(get(dy.p, ty, i * ld + j));
                times[token[i]] += j == 0;
            }
        }
    if (wrong) { printf("forward: %zu wrong values\n", wrong); return 1; }
    const size_t wb = nc_embedding_backward_workspace_bytes(t, v, d);
    Held ws(wb);
    st = nc_embedding_backward(tok.p, bytes, t, dy.p, ty, d, ld, scale, v, dt.p, to, ld, acc, ws.p, wb, nullptr);
    if (st != NC_OK) { printf("backward: status %d\n", (int)st); return 1; }
    for (size_t i = 0; i < v; ++i)
        for (size_t j = 0; j < d; ++j) {
            const double got = get(dt.p, to, i * ld + j), o = acc ? old[i * d + j] : 0;
            const double want = scale * sum[i * d + j] + o;
            if (!times[i]) wrong += got != o;
            else
                wrong += !(fabs(got - want) <= 1.01 * (scale * (times[i] + 2) * u * mag[i * d + j] +
                                                       (r + u) * fabs(want)) + 1e-7);
        }
    if (wrong) { printf("%zu wrong values\n", wrong); return 1; }
    printf("ok, %zu launches\n", model::launches);
    return 0;
}
