// The 8-bit operators and the block norm run on the CPU (test infrastructure): as
// main.cpp, whose workgroups, tensors and bounds these cases use, for the library's
// sources ff_block_api.cpp, quantize.hip, dense_int8.hip, block_norm.hip and, for the
// gradient from checkpoints, dense.hip.  op is quantize, dequantize, int8, backward_int8,
// block_norm or block_norm_backward.
#define main feed_forward_main
#include "main.cpp"
#undef main

namespace emulate {
// until only a thread's last n loads are under way
void wait_loads_but(int n)
{
    auto& loads = under_way[now];
    const size_t done = loads.size() > (size_t)n ? loads.size() - n : 0;
    for (size_t i = 0; i < done; ++i) land(loads[i].first.data(), loads[i].second);
    loads.erase(loads.begin(), loads.begin() + done);
}
}  // namespace emulate

namespace {

const Type I8{-1, 1, 0, 0};
int8_t& at(const Mat& m, int64_t r, int64_t c) { return reinterpret_cast<int8_t*>(m.p)[r * m.ld + c]; }
float* floats(const Mat& m) { return reinterpret_cast<float*>(m.p); }

void rows8(Case& k, Mat& m, const char* name, int64_t r, int64_t c)
{
    const std::string n(name);
    const int64_t ld = k.f.i(("ld_" + n).c_str(), c + k.f.i(("pad_" + n).c_str(), k.f.i("pad")));
    m.make(I8, r, c, ld, k.f.i(("off_" + n).c_str(), k.f.i("off")));
}
void fill8(Case& k, Mat& m, int most = 127)
{
    if (emulate::dry) return;
    std::uniform_int_distribution<int> d(-most, most);
    for (int64_t r = 0; r < m.rows; ++r)
        for (int64_t c = 0; c < m.cols; ++c) at(m, r, c) = (int8_t)d(k.g);
}
// fp32 [r, n], positive
void fill_scales(Case& k, Mat& m, int64_t r, int64_t n, float size)
{
    m.make(F32, 1, r * n, r * n, 0);
    if (emulate::dry) return;
    std::uniform_real_distribution<float> d(0.5f * size, 1.5f * size);
    for (int64_t i = 0; i < r * n; ++i) m.set(0, i, d(k.g));
}
double value(const Mat& q, const Mat& s, int64_t groups, int64_t r, int64_t c)
{
    return at(q, r, c) * s.get(0, r * groups + (groups > 1 ? c / 128 : 0));
}

int quantize(Case& k)
{
    const int64_t R = k.f.i("rows"), d = k.f.i("d"), group = k.f.i("group"), groups = group ? (d + 127) / 128 : 1;
    Mat x, q, s;
    rows(k, x, "x", R, d);
    x.fill(k.g, (float)(k.f.m.count("size") ? k.f.d("size") : 1.));
    const int64_t special = k.f.i("special");
    if (!emulate::dry && special && R && d) {  // values that are not finite, zeros, ties
        if (special == 1) x.set(R / 2, d / 2, INFINITY), x.set(0, d - 1, NAN);
        if (special == 2)
            for (int64_t c = 0; c < d; ++c) x.set(R - 1, c, 0.f);
        if (special == 3)
            for (int64_t r = 0; r < R; ++r)
                for (int64_t c = 0; c < d; ++c) x.set(r, c, c % 128 ? (float)(c * 37 % 253 - 126) * 0.5f : 127.f);
    }
    rows8(k, q, "q", R, d);
    s.make(F32, 1, R * groups, R * groups, 0);
    const int st = cliffconv_quantize(k.t.code, R, d, x.ptr(), x.ld, group, reinterpret_cast<int8_t*>(q.ptr()), q.ld,
                                      floats(s), nullptr);
    if (emulate::dry || st) return st;
    for (int64_t r = 0; r < R; ++r)
        for (int64_t g = 0; g < groups; ++g) {
            const int64_t c0 = g * 128, c1 = groups > 1 ? std::min(d, c0 + 128) : d;
            double most = 0;
            bool finite = true;
            for (int64_t c = c0; c < c1; ++c) finite &= isfinite(x.get(r, c)), most = std::max(most, fabs(x.get(r, c)));
            const float got = floats(s)[r * groups + g], want = std::max((float)(most / 127), 0x1p-126f);
            if (finite ? got != want : got == got)
                fail("scale (%lld, %lld): %.9g, expected %.9g", (long long)r, (long long)g, got, want);
            for (int64_t c = c0; c < c1; ++c) {
                const int i = finite ? (int)nearbyint(x.get(r, c) / (double)want) : 0;
                if (at(q, r, c) != i)
                    fail("q (%lld, %lld): %d, expected %d", (long long)r, (long long)c, at(q, r, c), i);
            }
        }
    return st;
}

int dequantize(Case& k)
{
    const int64_t R = k.f.i("rows"), d = k.f.i("d"), group = k.f.i("group"), groups = group ? (d + 127) / 128 : 1;
    Mat q, s, y;
    rows8(k, q, "q", R, d);
    fill8(k, q);
    fill_scales(k, s, R, groups, 0.01f);
    rows(k, y, "y", R, d);
    const int st = cliffconv_dequantize(k.t.code, R, d, reinterpret_cast<int8_t*>(q.ptr()), q.ld, floats(s), group,
                                        y.ptr(), y.ld, nullptr);
    if (emulate::dry || st) return st;
    for (int64_t r = 0; r < R; ++r)
        for (int64_t c = 0; c < d; ++c) {
            const double v = value(q, s, groups, r, c);
            expect("y", r, c, y.get(r, c), v, rounded(k.t, U * fabs(v), v));
        }
    return st;
}

int dense_int8(Case& k)
{
    const int64_t M = k.f.i("M"), K = k.f.i("K"), N = k.f.i("N");
    const int a = (int)k.f.i("act");
    const bool in_place = k.f.i("in_place");
    Mat x, w, xs, ws, b, res, y;
    rows8(k, x, "x", M, K);
    rows8(k, w, "w", N, K);
    fill8(k, x, k.f.i("most") ? 128 : 127);
    fill8(k, w);
    if (k.f.i("most") && !emulate::dry)
        for (int64_t c = 0; c < K; ++c) at(x, 0, c) = -128, at(w, 0, c) = -128;
    const float size = (float)(1 / (80 * sqrt((double)K)));
    fill_scales(k, xs, M, 1, 1.f);
    fill_scales(k, ws, N, 1, size / 80);
    if (const int far = (int)k.f.i("far"); far && !emulate::dry) {  // of both signs, far from one: 2^far and 2^-far
        for (int64_t i = 0; i < M; ++i) xs.set(0, i, (float)(ldexp(xs.get(0, i), far) * (i % 2 ? -1 : 1)));
        for (int64_t i = 0; i < N; ++i) ws.set(0, i, (float)(ldexp(ws.get(0, i), -far) * (i / 2 % 2 ? -1 : 1)));
    }
    if (k.f.i("bias")) b.make(k.t, 1, N, N, k.f.i("off")), b.fill(k.g, 1);
    if (k.f.i("residual") && !in_place) rows(k, res, "res", M, N), res.fill(k.g, 1);
    rows(k, y, "y", M, N);
    std::vector<double> before;
    if (in_place && !emulate::dry) {
        y.fill(k.g, 1);
        for (int64_t r = 0; r < M; ++r)
            for (int64_t c = 0; c < N; ++c) before.push_back(y.get(r, c));
    }
    const int64_t need = cliffconv_dense_int8_workspace(M, K, N);
    k.workspace(need);
    const Mat& rr = in_place ? y : res;
    const int st = cliffconv_dense_int8(k.t.code, M, K, N, reinterpret_cast<int8_t*>(x.ptr()), x.ld, floats(xs),
                                        reinterpret_cast<int8_t*>(w.ptr()), w.ld, floats(ws), b.ptr(), a, rr.ptr(), rr.ld,
                                        y.ptr(), y.ld, need ? k.ws.ptr() : nullptr, need, nullptr);
    if (emulate::dry || st) return st;
    const int64_t step = M * N > 1 << 18 ? 7 : 1;  // of the rows that are compared
    for (int64_t r = 0; r < M; r += r + step < M || r == M - 1 ? step : M - 1 - r)
        for (int64_t n = 0; n < N; ++n) {
            int64_t sum = 0;
            for (int64_t i = 0; i < K; ++i) sum += at(x, r, i) * at(w, n, i);
            const double p = (double)sum * xs.get(0, r) * ws.get(0, n), bn = b.p ? b.get(0, n) : 0, s = p + bn;
            const double e = 4 * U * (fabs(p) + fabs(bn)), f = act(a, s);
            double v = f, ev = 1.13 * e + COST * U * (fabs(f) + (a ? fabs(s) : 0));
            if (rr.p) {
                const double o = in_place ? before[r * N + n] : res.get(r, n);
                v += o, ev += 2 * U * fabs(o);
            }
            expect("y", r, n, y.get(r, n), v, rounded(k.t, ev, v));
        }
    return st;
}

int backward_int8(Case& k)
{
    const int64_t M = k.f.i("M"), K = k.f.i("K"), N = k.f.i("N"), xg = k.f.i("x_group"), pg = k.f.i("pre_group");
    const int64_t xgs = xg ? (K + 127) / 128 : 1, pgs = pg ? (N + 127) / 128 : 1;
    const int order = (int)k.f.i("oi"), a = (int)k.f.i("act"), want = (int)k.f.i("want", 7);  // 1 dx, 2 dw, 4 dbias
    Mat x, xs, w, dy, pre, ps, dx, dw, db;
    rows8(k, x, "x", M, K);
    fill8(k, x);
    fill_scales(k, xs, M, xgs, 0.01f);
    rows(k, w, "w", order ? N : K, order ? K : N);
    w.fill(k.g, (float)(1 / sqrt((double)K)));
    rows(k, dy, "dy", M, N);
    dy.fill(k.g, 1);
    if (a) rows8(k, pre, "pre", M, N), fill8(k, pre), fill_scales(k, ps, M, pgs, 0.01f);
    if (want & 1) rows(k, dx, "dx", M, K);
    if (want & 2) rows(k, dw, "dw", order ? N : K, order ? K : N);
    if (want & 4) db.make(k.t, 1, N, N, k.f.i("off"));
    const int64_t need = cliffconv_dense_backward_int8_workspace(k.t.code, M, K, N);
    k.workspace(need);
    const int st = cliffconv_dense_backward_int8(
        k.t.code, M, K, N, dy.ptr(), dy.ld, reinterpret_cast<int8_t*>(x.ptr()), x.ld, floats(xs), xg, w.ptr(), w.ld,
        order, reinterpret_cast<int8_t*>(pre.ptr()), pre.ld, floats(ps), pg, a, k.drop(), dx.ptr(), dx.ld, dw.ptr(),
        dw.ld, db.ptr(), k.ws.ptr(), need, nullptr);
    if (emulate::dry || st) return st;
    const double scale = k.p == 1 ? 0 : 1 / (1 - k.p);
    std::vector<double> g(M * N), eg(M * N), er(M * N);
    for (int64_t r = 0; r < M; ++r)
        for (int64_t n = 0; n < N; ++n) {
            const double z = a ? value(pre, ps, pgs, r, n) : 0, m = factor(k.p, k.rng.get(), r, n);
            const double v = dy.get(r, n) * (a ? slope(a, z) : 1) * m;
            const int64_t i = r * N + n;
            g[i] = v;
            eg[i] = (a ? COST * U * fabs(dy.get(r, n)) * (1 + fabs(z)) * m : 0) + 2 * U * fabs(v);
            er[i] = eg[i] + (a > 1 ? k.t.unit * fabs(v) + 2 * k.t.tiny * scale : 0);
        }
    auto compare = [&](const char* what, const Mat& m, int64_t r, int64_t c, double v, double size, double e, int64_t n) {
        e += (LAMBDA * sqrt((double)std::max<int64_t>(n, 1)) + COST) * U * size;
        expect(what, r, c, m.get(r, c), v, rounded(k.t, e, v));
    };
    auto weight = [&](int64_t i, int64_t n) { return order ? w.get(n, i) : w.get(i, n); };
    if (want & 1)
        for (int64_t r = 0; r < M; ++r)
            for (int64_t i = 0; i < K; ++i) {
                double v = 0, z = 0, e = 0;
                for (int64_t n = 0; n < N; ++n) {
                    v += g[r * N + n] * weight(i, n), z += fabs(g[r * N + n] * weight(i, n));
                    e += er[r * N + n] * fabs(weight(i, n));
                }
                compare("dx", dx, r, i, v, z, e, N);
            }
    if (want & 2) {
        std::vector<double> v(N), z(N), e(N);
        for (int64_t i = 0; i < K; ++i) {
            for (int64_t n = 0; n < N; ++n) v[n] = z[n] = e[n] = 0;
            for (int64_t r = 0; r < M; ++r) {
                const double xv = value(x, xs, xgs, r, i), ex = rounded(k.t, U * fabs(xv), xv) - k.t.unit * fabs(xv);
                for (int64_t n = 0; n < N; ++n)
                    v[n] += xv * g[r * N + n], z[n] += fabs(xv * g[r * N + n]),
                        e[n] += fabs(xv) * er[r * N + n] + ex * (fabs(g[r * N + n]) + er[r * N + n]);
            }
            for (int64_t n = 0; n < N; ++n) compare("dw", dw, order ? n : i, order ? i : n, v[n], z[n], e[n], M);
        }
    }
    if (want & 4)
        for (int64_t n = 0; n < N; ++n) {
            double v = 0, z = 0, e = 0;
            for (int64_t r = 0; r < M; ++r) v += g[r * N + n], z += fabs(g[r * N + n]), e += eg[r * N + n];
            compare("db", db, 0, n, v, z, e, M);
        }
    return st;
}

// A norm of a row v with errors e, in 64 bits: normed values and their errors.
struct Normed {
    double mean = 0, em = 0, rstd = 0, ei = 0;
    std::vector<double> h, eh;
    Normed(const std::vector<double>& v, const std::vector<double>& e, bool rms, double eps)
    {
        const int64_t d = (int64_t)v.size();
        const double s = (LAMBDA * sqrt((double)d) + COST) * U;
        if (!rms) {
            double a = 0;
            for (int64_t c = 0; c < d; ++c) mean += v[c] / d, a += fabs(v[c]) / d, em += e[c] / d;
            em += s * a;
        }
        double q = 0, eq = 0;
        for (int64_t c = 0; c < d; ++c) {
            const double u = v[c] - mean, eu = e[c] + em + U * fabs(v[c]);
            q += u * u / d;
            // (the mean's own error moves the sum of squares in second order only)
            eq += (2 * fabs(u) * e[c] + eu * eu + 2 * U * fabs(u) * fabs(v[c])) / d;
        }
        rstd = 1 / sqrt(q + eps);
        ei = rstd * (0.5 * (eq + s * q + 2 * U * eps) * rstd * rstd + 4 * U);
        if (rstd * rstd * eq > 0.5) ei += 2 * rstd;  // (a variance that is lost in the errors)
        for (int64_t c = 0; c < d; ++c) {
            h.push_back((v[c] - mean) * rstd);
            eh.push_back((e[c] + em + U * fabs(v[c])) * (rstd + ei) + fabs(v[c] - mean) * ei + 4 * U * fabs(h[c]));
        }
    }
    void affine(const Mat& w, const Mat& b)
    {
        for (size_t c = 0; c < h.size(); ++c) {
            if (w.p) h[c] *= w.get(0, c), eh[c] = eh[c] * fabs(w.get(0, c)) + 2 * U * fabs(h[c]);
            if (b.p) eh[c] += 2 * U * (fabs(h[c]) + fabs(b.get(0, c))), h[c] += b.get(0, c);
        }
    }
};

struct NormCase {
    int64_t R, d, gates;
    bool after, before, rms;
    cliff_block_norm_desc desc;
    Mat gate, w, b, nw, nb;
    explicit NormCase(Case& k)
        : R(k.f.i("rows")), d(k.f.i("d")), gates(k.f.i("gates")), after(k.f.i("after", 1)), before(k.f.i("before", 1)),
          rms(k.f.i("rms"))
    {
        desc = {after, before, rms, k.f.m.count("scale") ? k.f.d("scale") : 1., 1e-5, gates};
        auto vector = [&](Mat& m, int64_t n, const char* name, bool is) {
            if (is && k.f.i(name)) m.make(k.t, n, d, d, k.f.i("off")), m.fill(k.g, 0.7f, 0.2f);
        };
        vector(gate, gates, "gates", true);
        vector(w, 1, "w", after);
        vector(b, 1, "b", after);
        vector(nw, 1, "w", before);
        vector(nb, 1, "b", before);
    }
    double g(int64_t r, int64_t c) const { return gate.p ? gate.get(r / (R / gates), c) : 1; }
};

int block_norm(Case& k)
{
    NormCase n(k);
    const int64_t R = n.R, d = n.d;
    const int alias = (int)k.f.i("alias");  // out, normed: 1 residual, own; 2 x, own; 3 residual, x; 4 x, residual
    Mat x, res, out, normed, stats;
    rows(k, x, "x", R, d);
    x.fill(k.g, 1.5f, 0.7f);
    rows(k, res, "res", R, d);
    res.fill(k.g, 1);
    if (!alias) rows(k, out, "y", R, d);
    if (n.before && alias < 3) rows(k, normed, "n", R, d);
    if (!k.f.i("no_stats")) stats.make(F32, 4, R, R, 0);
    std::vector<double> in, rin;
    if (!emulate::dry)
        for (int64_t r = 0; r < R; ++r)
            for (int64_t c = 0; c < d; ++c) in.push_back(x.get(r, c)), rin.push_back(res.get(r, c));
    const Mat& to = alias == 1 || alias == 3 ? res : alias ? x : out;
    const Mat& tn = !n.before ? normed : alias == 3 ? x : alias == 4 ? res : normed;
    const int st = cliffconv_block_norm(k.t.code, R, d, &n.desc, x.ptr(), x.ld, res.ptr(), res.ld, n.gate.ptr(), n.w.ptr(),
                                        n.b.ptr(), n.nw.ptr(), n.nb.ptr(), to.ptr(), to.ld, tn.ptr(), tn.ld, floats(stats),
                                        nullptr);
    if (emulate::dry || st) return st;
    auto statistics = [&](int which, int64_t r, const Normed& v) {
        if (!stats.p) return;
        expect("mean", which, r, stats.get(which, r), v.mean, v.em + 1e-37);
        expect("rstd", which + 1, r, stats.get(which + 1, r), v.rstd, v.ei + 1e-37);
    };
    for (int64_t r = 0; r < R; ++r) {
        std::vector<double> v(in.begin() + r * d, in.begin() + (r + 1) * d), e(d, 0.);
        if (n.after) {
            Normed h(v, e, n.rms, 1e-5);
            statistics(0, r, h);
            h.affine(n.w, n.b);
            v = h.h, e = h.eh;
        }
        for (int64_t c = 0; c < d; ++c) {
            const double gate = n.g(r, c), s = n.desc.scale * rin[r * d + c];
            e[c] = e[c] * fabs(gate) + 3 * U * (fabs(v[c] * gate) + fabs(s));
            v[c] = v[c] * gate + s;
            expect("out", r, c, to.get(r, c), v[c], rounded(k.t, e[c], v[c]));
        }
        if (!n.before) continue;
        Normed h(v, e, n.rms, 1e-5);
        statistics(2, r, h);
        h.affine(n.nw, n.nb);
        for (int64_t c = 0; c < d; ++c) expect("normed", r, c, tn.get(r, c), h.h[c], rounded(k.t, h.eh[c], h.h[c]));
    }
    return st;
}

int block_norm_backward(Case& k)
{
    NormCase n(k);
    const int64_t R = n.R, d = n.d;
    const int alias = (int)k.f.i("alias");  // 1: dx is dout, dresidual dnormed; 2: the other way
    const bool has_dout = !n.before || !k.f.i("no_dout"), params = !k.f.i("no_params");
    Mat dout, dn, x, out, stats, dx, dr, dg, dw, db, dnw, dnb;
    if (has_dout) rows(k, dout, "dy", R, d), dout.fill(k.g, 1);
    if (n.before) rows(k, dn, "dn", R, d), dn.fill(k.g, 1), rows(k, out, "y", R, d), out.fill(k.g, 1.5f, 0.3f);
    const bool reads_x = n.after || (params && n.gate.p);
    if (reads_x) rows(k, x, "x", R, d), k.f.m.count("constant") ? x.fill(k.g, 0, (float)k.f.d("constant")) : x.fill(k.g, 1.5f, 0.7f);
    stats.make(F32, 4, R, R, 0);
    auto statistics = [&](int which, const Mat& v) {
        if (emulate::dry || !v.p) return;
        for (int64_t r = 0; r < R; ++r) {
            double m = 0, q = 0;
            if (!n.rms)
                for (int64_t c = 0; c < d; ++c) m += v.get(r, c) / d;
            stats.set(which, r, (float)m);
            for (int64_t c = 0; c < d; ++c) q += pow(v.get(r, c) - stats.get(which, r), 2) / d;
            stats.set(which + 1, r, (float)(1 / sqrt(q + 1e-5)));
        }
    };
    if (n.after) statistics(0, x);
    if (n.before) statistics(2, out);
    const bool a1 = alias && has_dout && n.before;
    if (!a1) rows(k, dx, "dx", R, d), rows(k, dr, "dr", R, d);
    auto sum = [&](Mat& m, const Mat& of) {
        if (params && of.p) m.make(k.t, of.rows, d, d, k.f.i("off"));
    };
    sum(dg, n.gate), sum(dw, n.w), sum(db, n.b), sum(dnw, n.nw), sum(dnb, n.nb);
    std::vector<double> go, gn;
    if (!emulate::dry)
        for (int64_t r = 0; r < R; ++r)
            for (int64_t c = 0; c < d; ++c)
                go.push_back(has_dout ? dout.get(r, c) : 0), gn.push_back(n.before ? dn.get(r, c) : 0);
    const int64_t need = cliffconv_block_norm_backward_workspace(k.t.code, R, d, n.gate.p ? n.gates : 0);
    k.workspace(need);
    const Mat& tx = a1 ? (alias == 1 ? dout : dn) : dx;
    const Mat& tr = a1 ? (alias == 1 ? dn : dout) : dr;
    const int st = cliffconv_block_norm_backward(
        k.t.code, R, d, &n.desc, dout.ptr(), dout.ld, dn.ptr(), dn.ld, x.ptr(), x.ld, out.ptr(), out.ld, floats(stats),
        n.gate.ptr(), n.w.ptr(), n.b.ptr(), n.nw.ptr(), tx.ptr(), tx.ld, tr.ptr(), tr.ld, dg.ptr(), dw.ptr(), db.ptr(),
        dnw.ptr(), dnb.ptr(), k.ws.ptr(), need, nullptr);
    if (emulate::dry || st) return st;
    const double s = (LAMBDA * sqrt((double)d) + COST) * U, sr = (LAMBDA * sqrt((double)std::max<int64_t>(R, 1)) + COST) * U;
    struct Sum {
        double v = 0, z = 0, e = 0;
        void add(double a, double err) { v += a, z += fabs(a), e += err; }
    };
    const int64_t G = n.gate.p ? n.gates : 1;
    std::vector<Sum> A(G * d), B(G * d), Cs(d), D(d);
    for (int64_t r = 0; r < R; ++r) {
        std::vector<double> t(d), et(d), h(d), eh(d);
        auto values = [&](const Mat& v, int which, std::vector<double>& o, std::vector<double>& e) {
            const double m = stats.get(which, r), i = stats.get(which + 1, r);
            for (int64_t c = 0; c < d; ++c) {
                o[c] = (v.get(r, c) - m) * i;
                e[c] = 4 * U * (fabs(o[c]) + (fabs(v.get(r, c)) + fabs(m)) * i);
            }
            return i;
        };
        // i (q - mean q - h mean(q h)) of q with errors
        auto through = [&](const std::vector<double>& q, const std::vector<double>& eq, double i, std::vector<double>& o,
                           std::vector<double>& e) {
            double m = 0, em = 0, mh = 0, emh = 0, a = 0, ah = 0;
            for (int64_t c = 0; c < d; ++c) {
                m += q[c] / d, a += fabs(q[c]) / d, em += eq[c] / d;
                mh += q[c] * h[c] / d, ah += fabs(q[c] * h[c]) / d, emh += (eq[c] * fabs(h[c]) + (fabs(q[c]) + eq[c]) * eh[c]) / d;
            }
            em += s * a, emh += s * ah;
            if (n.rms) m = em = 0;
            for (int64_t c = 0; c < d; ++c) {
                o[c] = i * (q[c] - m - h[c] * mh);
                e[c] = i * (eq[c] + em + fabs(h[c]) * emh + eh[c] * (fabs(mh) + emh) +
                            COST * U * (fabs(q[c]) + fabs(m) + fabs(h[c] * mh)));
            }
        };
        std::vector<double> q(d), eq(d), o(d), e(d);
        for (int64_t c = 0; c < d; ++c) t[c] = go[r * d + c];
        if (n.before) {
            const double i = values(out, 2, h, eh);
            for (int64_t c = 0; c < d; ++c) {
                const double v = gn[r * d + c], w = n.nw.p ? n.nw.get(0, c) : 1;
                q[c] = v * w, eq[c] = U * fabs(v * w);
                Cs[c].add(v * h[c], fabs(v) * eh[c]);
                D[c].add(v, 0);
            }
            through(q, eq, i, o, e);
            for (int64_t c = 0; c < d; ++c) et[c] = e[c] + 2 * U * (fabs(t[c]) + fabs(o[c])), t[c] += o[c];
        }
        double i = 1;
        if (n.after) {
            i = values(x, 0, h, eh);
        } else {
            for (int64_t c = 0; c < d; ++c) h[c] = reads_x ? x.get(r, c) : 0, eh[c] = 0;
        }
        for (int64_t c = 0; c < d; ++c) {
            const double f = n.g(r, c) * (n.w.p ? n.w.get(0, c) : 1);
            const int64_t j = (n.gate.p ? r / (R / n.gates) : 0) * d + c;
            A[j].add(t[c] * h[c], et[c] * (fabs(h[c]) + eh[c]) + fabs(t[c]) * eh[c]);
            B[j].add(t[c], et[c]);
            q[c] = t[c] * f, eq[c] = et[c] * fabs(f) + 3 * U * fabs(q[c]);
            const double v = n.desc.scale * t[c];
            expect("dresidual", r, c, tr.get(r, c), v, rounded(k.t, fabs(n.desc.scale) * et[c] + 2 * U * fabs(v), v));
        }
        if (n.after) through(q, eq, i, o, e);
        else o = q, e = eq;
        for (int64_t c = 0; c < d; ++c) expect("dx", r, c, tx.get(r, c), o[c], rounded(k.t, e[c], o[c]));
    }
    auto check = [&](const char* what, const Mat& m, int64_t r, int64_t c, const Sum& v) {
        if (m.p) expect(what, r, c, m.get(r, c), v.v, rounded(k.t, v.e + sr * v.z, v.v));
    };
    for (int64_t c = 0; c < d; ++c) {
        Sum w, b;
        for (int64_t g = 0; g < G; ++g) {
            const Sum &a = A[g * d + c], &z = B[g * d + c];
            const double gate = n.gate.p ? n.gate.get(g, c) : 1;
            w.v += gate * a.v, w.z += fabs(gate) * a.z, w.e += fabs(gate) * a.e;
            b.v += gate * z.v, b.z += fabs(gate) * z.z, b.e += fabs(gate) * z.e;
            const double f = n.w.p ? n.w.get(0, c) : 1, o = n.b.p ? n.b.get(0, c) : 0;
            check("dgate", dg, g, c, {f * a.v + o * z.v, fabs(f) * a.z + fabs(o) * z.z, fabs(f) * a.e + fabs(o) * z.e});
        }
        check("dweight", dw, 0, c, w);
        check("dbias", db, 0, c, b);
        check("dnext_weight", dnw, 0, c, Cs[c]);
        check("dnext_bias", dnb, 0, c, D[c]);
    }
    return st;
}

}  // namespace

int main()
{
    std::string line;
    for (int n = 0; std::getline(std::cin, line); ++n) {
        fprintf(stderr, "case %d\n", n);
        Fields f;
        std::istringstream in(line);
        std::string word;
        while (in >> word) {
            const size_t eq = word.find('=');
            f.m[word.substr(0, eq)] = eq == std::string::npos ? "1" : word.substr(eq + 1);
        }
        cliff::assumed_cus = (int)f.i("cus", 256);
        emulate::dry = f.i("dry");
        emulate::late = f.i("late");
        emulate::most_threads = 0;
        next_address = (uintptr_t)1 << 44;
        failure.clear();
        int st = -1;
        {
            Case k(f);
            const std::string op = f.s("op");
            st = op == "quantize" ? quantize(k) : op == "dequantize" ? dequantize(k) : op == "int8" ? dense_int8(k)
               : op == "backward_int8" ? backward_int8(k) : op == "block_norm" ? block_norm(k)
               : op == "block_norm_backward" ? block_norm_backward(k) : -1;
        }
        if (!failure.empty()) printf("FAIL %s\n", failure.c_str());
        else printf("ok %d %llu\n", st, (unsigned long long)emulate::most_threads);
        fflush(stdout);
        fflush(stderr);
    }
    return 0;
}
