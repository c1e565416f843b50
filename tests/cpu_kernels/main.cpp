// The feed-forward operators run on the CPU (test infrastructure): the library's
// own sources (ff_api.cpp, dense.hip, norm.hip, dropout.hip), compiled with
// hip_runtime.h and lds_load.hpp of this folder in the place of HIP's, under
// AddressSanitizer and UndefinedBehaviorSanitizer.  Every tensor of a case is an
// allocation of exactly its size with the elements between its rows poisoned, so
// that a read or write outside a row ends the program; results are compared with
// loops in 64 bits.
//
// Input: one case per line on stdin, fields as key=value; op is dense, backward,
// norm, norm_backward or dropout, cus the compute units that the launchers
// assume; late=1: loads straight to LDS land when their thread waits for them, not
// at once.  dry=1: nothing runs, and tensors are addresses only; the line says what the call
// returned and the largest number of threads along an axis of a grid.
// Output: one line per case, "ok status ..." or "FAIL ...".  stderr: "case" lines,
// followed by what the library prints of its launches.
#include <hip/hip_runtime.h>
#include <math.h>
#include <sanitizer/asan_interface.h>
#include <stdio.h>
#include <stdlib.h>
#include <sys/mman.h>

#include <algorithm>
#include <iostream>
#include <map>
#include <memory>
#include <random>
#include <sstream>
#include <string>
#include <vector>

#include "cliffconv_ff.h"
#include "ff_common.hpp"

// ---- the workgroup's fibers

dim3 threadIdx, blockIdx, blockDim, gridDim;

extern "C" void emulate_switch(void** save, void* to);
__asm__(R"(
.text
.globl emulate_switch
emulate_switch:
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

namespace emulate {

hipError_t last_error = hipSuccess;
bool dry = false;
bool late = false;  // loads straight to LDS land when they are waited for
uint64_t most_threads = 0;

namespace {

constexpr size_t STACK = 512 << 10;
enum State { READY, IN_WAVE, IN_GROUP, DONE };
struct Fiber {
    void* sp;
    State state;
    dim3 tid;
};
struct Wave {
    int kind = 0, came = 0;
    char out[WAVE][128];
    alignas(128) char packed_in[WAVE * 128], packed_out[WAVE * 128];
};
Fiber fibers[1024];
std::vector<std::pair<std::vector<char>, char*>> under_way[1024];  // loads of each thread
Wave waves[16];
char* stacks = nullptr;
void* scheduler;
int now, threads, barrier, alive;
const std::function<void()>* body;
struct Dynamic {
    char* at;
    size_t bytes;
};
std::vector<Dynamic>& dynamics()
{
    static std::vector<Dynamic> v;
    return v;
}

[[noreturn]] void die(const char* what)
{
    fprintf(stderr, "emulation: %s, block (%u, %u), thread %d of %d\n", what, blockIdx.x, blockIdx.y, now, threads);
    fflush(stderr);
    abort();
}

void yield() { emulate_switch(&fibers[now].sp, scheduler); }

void entry()
{
    (*body)();
    fibers[now].state = DONE;
    --alive;
    yield();
    die("a finished thread ran on");
}

void run_group()
{
    alive = threads;
    barrier = 0;
    for (int t = 0; t < threads; ++t) {
        Fiber& f = fibers[t];
        f.state = READY;
        f.tid = dim3(t, 0, 0);
        void** top = reinterpret_cast<void**>(stacks + (t + 1) * STACK);
        *--top = nullptr;  // (the entry's return address is at 16 n + 8)
        *--top = reinterpret_cast<void*>(entry);
        for (int i = 0; i < 6; ++i) *--top = nullptr;
        f.sp = top;
    }
    for (Wave& w : waves) w.came = 0;
    for (auto& l : under_way) l.clear();
    while (alive) {
        bool any = false;
        for (int w0 = 0; w0 < threads; w0 += WAVE) {
            // odd workgroups take the waves from the last one on
            const int w = blockIdx.x & 1 ? threads - WAVE - w0 : w0;
            bool more = true;
            while (more) {
                more = false;
                for (int t = w; t < w + WAVE; ++t)
                    if (fibers[t].state == READY) {
                        now = t;
                        threadIdx = fibers[t].tid;
                        emulate_switch(&scheduler, fibers[t].sp);
                        more = any = true;
                    }
            }
        }
        if (alive && barrier == alive) {
            barrier = 0;
            for (int t = 0; t < threads; ++t)
                if (fibers[t].state == IN_GROUP) fibers[t].state = READY;
        } else if (alive && !any) {
            die("threads wait for others that never come");
        }
    }
}

}  // namespace

DynamicLds::DynamicLds(void* at, size_t bytes) { dynamics().push_back({static_cast<char*>(at), bytes}); }

int lane_id() { return now % WAVE; }

static void land(const char* bytes, char* to) { memcpy(to, bytes, 16); }
void load(const char* from, char* to)
{
    char bytes[16] = {};
    if (from) memcpy(bytes, from, 16);
    if (late) under_way[now].push_back({std::vector<char>(bytes, bytes + 16), to});
    else land(bytes, to);
}
void wait_loads()
{
    for (const auto& l : under_way[now]) land(l.first.data(), l.second);
    under_way[now].clear();
}

void meet_workgroup()
{
    ++barrier;
    fibers[now].state = IN_GROUP;
    yield();
}

void meet(int kind, const void* in, size_t in_size, void* out, size_t out_size, Meet f)
{
    Wave& w = waves[now / WAVE];
    const int lane = now % WAVE, w0 = now - lane;
    if (in_size > 128 || out_size > sizeof w.out[0]) die("operands too large");
    if (w.came && w.kind != kind) die("lanes of a wave meet in different instructions");
    w.kind = kind;
    memcpy(w.packed_in + lane * in_size, in, in_size);
    if (++w.came == WAVE) {
        f(w.packed_in, w.packed_out);
        w.came = 0;
        for (int t = w0; t < w0 + WAVE; ++t) {
            memcpy(w.out[t - w0], w.packed_out + (t - w0) * out_size, out_size);
            if (fibers[t].state == IN_WAVE) fibers[t].state = READY;
        }
    } else {
        fibers[now].state = IN_WAVE;
        yield();
    }
    memcpy(out, w.out[lane], out_size);
}

void launch(dim3 grid, dim3 block, size_t lds, const std::function<void()>& kernel)
{
    const uint64_t n[3] = {(uint64_t)grid.x * block.x, (uint64_t)grid.y * block.y, (uint64_t)grid.z * block.z};
    for (uint64_t v : n) most_threads = std::max(most_threads, v);
    if (!n[0] || !n[1] || !n[2] || n[0] >> 32 || n[1] >> 32 || n[2] >> 32 || grid.y > 65535 || grid.z > 65535 ||
        block.x * block.y * block.z > 1024 || lds > 160 << 10) {
        last_error = 1;
        return;
    }
    if (dry) return;
    if (block.x % WAVE || block.y != 1 || block.z != 1) die("workgroup");
    if (!stacks) {
        stacks = static_cast<char*>(mmap(nullptr, 1024 * STACK, PROT_READ | PROT_WRITE,
                                         MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0));
        if (stacks == MAP_FAILED) die("stacks");
    }
    threads = (int)block.x;
    body = &kernel;
    blockDim = block;
    gridDim = grid;
    for (unsigned z = 0; z < grid.z; ++z)
        for (unsigned y = 0; y < grid.y; ++y)
            for (unsigned x = 0; x < grid.x; ++x) {
                blockIdx = dim3(x, y, z);
                for (const Dynamic& d : dynamics()) {
                    __asan_unpoison_memory_region(d.at, d.bytes);
                    memset(d.at, 0xff, d.bytes);  // NaN
                    __asan_poison_memory_region(d.at + lds, d.bytes - lds);
                }
                run_group();
            }
}

}  // namespace emulate

namespace cliff {
static int assumed_cus = 256;
int device_cus() { return assumed_cus; }
bool debug_enabled() { return true; }
}  // namespace cliff

// ---- the cases

namespace {

std::string failure;
template <typename... A>
void fail(const char* fmt, A... a)
{
    if (!failure.empty()) return;
    char b[400];
    snprintf(b, sizeof b, fmt, a...);
    failure = b;
}

const double U = 0x1p-24, LAMBDA = 8, COST = 16;  // as in ff_oracle.py

struct Type {
    int code, size;
    double unit, tiny;
};
Type type_of(const std::string& s)
{
    if (s == "bf16") return {CLIFF_BF16, 2, 0x1p-8, 1e-37};
    if (s == "fp16") return {CLIFF_F16, 2, 0x1p-11, 0x1p-24};
    return {CLIFF_F32, 4, 0x1p-24, 1e-37};
}

uintptr_t next_address;  // of dry cases

// A matrix of a case: rows of cols elements, ld apart, `offset` elements into its
// allocation, which ends with its last row.
struct Mat {
    Type t;
    int64_t rows = 0, cols = 0, ld = 0;
    char* base = nullptr;
    size_t bytes = 0;
    char* p = nullptr;
    bool mapped = false;
    Mat() = default;
    Mat(const Mat&) = delete;
    Mat& operator=(const Mat&) = delete;
    ~Mat()
    {
        if (!base) return;
        if (mapped) {
            munmap(base, bytes);
        } else {
            __asan_unpoison_memory_region(base, bytes);
            free(base);
        }
    }
    void make(Type t_, int64_t rows_, int64_t cols_, int64_t ld_, int64_t offset)
    {
        t = t_, rows = rows_, cols = cols_, ld = ld_;
        if (emulate::dry) {
            p = reinterpret_cast<char*>(next_address);
            next_address += ((uintptr_t)((rows * ld + cols) * t.size) + 4095) & ~(uintptr_t)4095;
            return;
        }
        bytes = (size_t)((rows ? (rows - 1) * ld + cols : 0) + offset) * t.size;
        if (bytes > (size_t)1 << 30) {
            // rows far from each other: pages that nothing touches take no memory
            mapped = true;
            base = static_cast<char*>(mmap(nullptr, bytes, PROT_READ | PROT_WRITE,
                                           MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0));
            if (base == MAP_FAILED) abort();
            p = base + offset * t.size;
            return;
        }
        base = static_cast<char*>(aligned_alloc(64, (bytes + 64) / 64 * 64 + 64));
        // the allocation ends with the matrix
        const size_t all = (bytes + 64) / 64 * 64 + 64;
        memset(base, 0xff, all);
        p = base + offset * t.size;
        if (offset) __asan_poison_memory_region(base, (size_t)offset * t.size & ~(size_t)7);
        for (int64_t r = 0; r + 1 < rows; ++r)
            if (ld > cols) __asan_poison_memory_region(p + (r * ld + cols) * t.size, (size_t)(ld - cols) * t.size);
        __asan_poison_memory_region(base + bytes, all - bytes);
        bytes = all;
    }
    double get(int64_t r, int64_t c) const
    {
        const char* a = p + (r * ld + c) * t.size;
        if (t.code == CLIFF_F32) {
            float v;
            memcpy(&v, a, 4);
            return v;
        }
        if (t.code == CLIFF_BF16) {
            uint16_t v;
            memcpy(&v, a, 2);
            const uint32_t w = (uint32_t)v << 16;
            float f;
            memcpy(&f, &w, 4);
            return f;
        }
        _Float16 v;
        memcpy(&v, a, 2);
        return (double)v;
    }
    void set(int64_t r, int64_t c, float f)
    {
        char* a = p + (r * ld + c) * t.size;
        if (t.code == CLIFF_F32) {
            memcpy(a, &f, 4);
        } else if (t.code == CLIFF_BF16) {
            uint32_t w;
            memcpy(&w, &f, 4);
            const uint16_t v = (uint16_t)((w + 0x7fff + (w >> 16 & 1)) >> 16);
            memcpy(a, &v, 2);
        } else {
            const _Float16 v = (_Float16)f;
            memcpy(a, &v, 2);
        }
    }
    void fill(std::mt19937& g, float scale, float shift = 0.f)
    {
        if (emulate::dry) return;
        std::uniform_real_distribution<float> d(-1.7f, 1.7f);
        for (int64_t r = 0; r < rows; ++r)
            for (int64_t c = 0; c < cols; ++c) set(r, c, scale * d(g) + shift);
    }
    void* ptr() const { return p; }
};

struct Fields {
    std::map<std::string, std::string> m;
    int64_t i(const char* k, int64_t otherwise = 0) const
    {
        const auto f = m.find(k);
        return f == m.end() ? otherwise : strtoll(f->second.c_str(), nullptr, 0);
    }
    double d(const char* k) const
    {
        const auto f = m.find(k);
        return f == m.end() ? 0. : strtod(f->second.c_str(), nullptr);
    }
    std::string s(const char* k) const
    {
        const auto f = m.find(k);
        return f == m.end() ? "" : f->second;
    }
};

double cdf(double v) { return 0.5 * erfc(-v * sqrt(0.5)); }
double act(int a, double v)
{
    return a == 1 ? (v > 0 ? v : 0) : a == 2 ? v * cdf(v) : a == 3 ? v / (1 + exp(-v)) : v;
}
double slope(int a, double v)
{
    const double s = 1 / (1 + exp(-v));
    return a == 1 ? v > 0 : a == 2 ? cdf(v) + v * exp(-v * v / 2) / sqrt(2 * M_PI) : a == 3 ? s + v * s * (1 - s) : 1;
}

// Dropout's factor of an element, from the generator's definition.
double factor(double p, const int64_t* rng, int64_t r, int64_t c)
{
    if (p == 0) return 1;
    if (p == 1) return 0;
    uint32_t x[4] = {(uint32_t)(c / 4), (uint32_t)r, (uint32_t)(r >> 32), (uint32_t)rng[1]},
             k[2] = {(uint32_t)rng[0], (uint32_t)((uint64_t)rng[0] >> 32)};
    for (int i = 0; i < 7; ++i) {
        const uint64_t a = 0xD2511F53ull * x[0], b = 0xCD9E8D57ull * x[2];
        const uint32_t y[4] = {(uint32_t)(b >> 32) ^ x[1] ^ k[0], (uint32_t)b, (uint32_t)(a >> 32) ^ x[3] ^ k[1],
                               (uint32_t)a};
        memcpy(x, y, sizeof x);
        k[0] += 0x9E3779B9u;
        k[1] += 0xBB67AE85u;
    }
    return x[c & 3] >= nearbyint(p * 4294967296.0) ? 1 / (1 - p) : 0;
}

void expect(const char* what, int64_t r, int64_t c, double got, double want, double bound)
{
    if (!(fabs(got - want) <= bound))
        fail("%s (%lld, %lld): %.9g, expected %.9g +- %.3g", what, (long long)r, (long long)c, got, want, bound);
}
double rounded(const Type& t, double e, double v) { return e * (1 + t.unit) + 2 * t.unit * fabs(v) + t.tiny; }

struct Case {
    const Fields& f;
    Type t;
    std::mt19937 g;
    double p;
    std::unique_ptr<int64_t[]> rng;
    cliff_dropout_desc desc;
    Mat ws;
    explicit Case(const Fields& f_) : f(f_), t(type_of(f.s("type"))), g((unsigned)f.i("seed", 1)), p(f.d("p"))
    {
        rng.reset(new int64_t[2]{0x123456789ABCDEF, 77});
        desc = {p, rng.get()};
    }
    const cliff_dropout_desc* drop() const { return p > 0 ? &desc : nullptr; }
    void workspace(int64_t n) { ws.make({0, 1, 0, 0}, 1, n, n, 0); }
};

// rows of a tensor `name`: its stride is what "ld_<name>" says, else its width and
// "pad_<name>"
void rows(Case& k, Mat& m, const char* name, int64_t r, int64_t c)
{
    const std::string n(name);
    const int64_t ld = k.f.i(("ld_" + n).c_str(), c + k.f.i(("pad_" + n).c_str(), k.f.i("pad")));
    m.make(k.t, r, c, ld, k.f.i(("off_" + n).c_str(), k.f.i("off")));
}

struct Dense {
    int64_t M, K, N;
    int order, a;
    Mat x, w;
    explicit Dense(Case& k) : M(k.f.i("M")), K(k.f.i("K")), N(k.f.i("N")), order((int)k.f.i("oi")), a((int)k.f.i("act"))
    {
        rows(k, x, "x", M, K);
        rows(k, w, "w", order ? N : K, order ? K : N);
        x.fill(k.g, 1);
        w.fill(k.g, (float)(1 / sqrt((double)K)));
    }
    double weight(int64_t k, int64_t n) const { return order ? w.get(n, k) : w.get(k, n); }
};

int dense(Case& k)
{
    Dense d(k);
    const int64_t M = d.M, K = d.K, N = d.N;
    const bool in_place = k.f.i("in_place");
    Mat b, res, pre, y;
    if (k.f.i("bias")) b.make(k.t, 1, N, N, k.f.i("off")), b.fill(k.g, 1);
    if (k.f.i("residual") && !in_place) rows(k, res, "res", M, N), res.fill(k.g, 1);
    if (k.f.i("pre")) rows(k, pre, "pre", M, N);
    rows(k, y, "y", M, N);
    std::vector<double> before;
    if (in_place) {
        y.fill(k.g, 1);
        for (int64_t r = 0; r < M; ++r)
            for (int64_t c = 0; c < N; ++c) before.push_back(y.get(r, c));
    }
    const int64_t need = cliffconv_dense_workspace(k.t.code, M, K, N);
    k.workspace(need);
    const Mat& rr = in_place ? y : res;
    const int st = cliffconv_dense(k.t.code, M, K, N, d.x.ptr(), d.x.ld, d.w.ptr(), d.w.ld, d.order, b.ptr(), d.a, k.drop(),
                                   rr.ptr(), rr.ld, pre.ptr(), pre.ld, y.ptr(), y.ld, need ? k.ws.ptr() : nullptr, need,
                                   nullptr);
    if (emulate::dry || st) return st;
    const int64_t step = M * N > 1 << 18 ? 7 : 1;  // of the rows that are compared
    std::vector<double> wt(K * N);
    for (int64_t i = 0; i < K; ++i)
        for (int64_t n = 0; n < N; ++n) wt[i * N + n] = d.weight(i, n);
    std::vector<double> sum(N), size(N);
    for (int64_t r = 0; r < M; r += r + step < M || r == M - 1 ? step : M - 1 - r) {
        for (int64_t n = 0; n < N; ++n) sum[n] = size[n] = 0;
        for (int64_t i = 0; i < K; ++i) {
            const double v = d.x.get(r, i);
            for (int64_t n = 0; n < N; ++n) sum[n] += v * wt[i * N + n], size[n] += fabs(v * wt[i * N + n]);
        }
        for (int64_t n = 0; n < N; ++n) {
            double s = sum[n], z = size[n];
            if (b.p) s += b.get(0, n), z += fabs(b.get(0, n));
            const double e = (LAMBDA * sqrt((double)K) + COST) * U * z, f = act(d.a, s), m = factor(k.p, k.rng.get(), r, n);
            if (pre.p) expect("pre", r, n, pre.get(r, n), s, rounded(k.t, e, s));
            double v = f * m, ev = (1.13 * e + COST * U * (fabs(f) + (d.a ? fabs(s) : 0))) * m;
            if (rr.p) {
                const double q = in_place ? before[r * N + n] : res.get(r, n);
                v += q, ev += 2 * U * fabs(q);
            }
            expect("y", r, n, y.get(r, n), v, rounded(k.t, ev, v));
        }
    }
    return st;
}

int backward(Case& k)
{
    Dense d(k);
    const int64_t M = d.M, K = d.K, N = d.N;
    const int want = (int)k.f.i("want", 7);  // 1 dx, 2 dw, 4 dbias
    Mat dy, pre, dx, dw, db;
    rows(k, dy, "dy", M, N);
    dy.fill(k.g, 1);
    if (d.a) rows(k, pre, "pre", M, N), pre.fill(k.g, 1);
    if (want & 1) rows(k, dx, "dx", M, K);
    if (want & 2) rows(k, dw, "dw", d.order ? N : K, d.order ? K : N);
    if (want & 4) db.make(k.t, 1, N, N, k.f.i("off"));
    const int64_t need = cliffconv_dense_backward_workspace(k.t.code, M, K, N);
    k.workspace(need);
    const int st = cliffconv_dense_backward(k.t.code, M, K, N, dy.ptr(), dy.ld, d.x.ptr(), d.x.ld, d.w.ptr(), d.w.ld,
                                            d.order, pre.ptr(), pre.ld, d.a, k.drop(), dx.ptr(), dx.ld, dw.ptr(), dw.ld,
                                            db.ptr(), k.ws.ptr(), need, nullptr);
    if (emulate::dry || st) return st;
    const double scale = k.p == 1 ? 0 : 1 / (1 - k.p);
    std::vector<double> g(M * N), eg(M * N), er(M * N);
    for (int64_t r = 0; r < M; ++r)
        for (int64_t n = 0; n < N; ++n) {
            const double m = factor(k.p, k.rng.get(), r, n), v = dy.get(r, n) * (d.a ? slope(d.a, pre.get(r, n)) : 1) * m;
            const int64_t i = r * N + n;
            g[i] = v;
            eg[i] = (d.a ? COST * U * fabs(dy.get(r, n)) * (1 + fabs(pre.get(r, n))) * m : 0) + 2 * U * fabs(v);
            er[i] = eg[i] + (d.a > 1 ? k.t.unit * fabs(v) + 2 * k.t.tiny * scale : 0);
        }
    auto compare = [&](const char* what, const Mat& m, int64_t r, int64_t c, double v, double size, double e, int64_t n) {
        e += (LAMBDA * sqrt((double)std::max<int64_t>(n, 1)) + COST) * U * size;
        expect(what, r, c, m.get(r, c), v, rounded(k.t, e, v));
    };
    if (want & 1)
        for (int64_t r = 0; r < M; ++r)
            for (int64_t i = 0; i < K; ++i) {
                double v = 0, z = 0, e = 0;
                for (int64_t n = 0; n < N; ++n) {
                    const double w = d.weight(i, n);
                    v += g[r * N + n] * w, z += fabs(g[r * N + n] * w), e += er[r * N + n] * fabs(w);
                }
                compare("dx", dx, r, i, v, z, e, N);
            }
    if (want & 2) {
        std::vector<double> v(N), z(N), e(N);
        for (int64_t i = 0; i < K; ++i) {
            for (int64_t n = 0; n < N; ++n) v[n] = z[n] = e[n] = 0;
            for (int64_t r = 0; r < M; ++r) {
                const double x = d.x.get(r, i);
                for (int64_t n = 0; n < N; ++n)
                    v[n] += x * g[r * N + n], z[n] += fabs(x * g[r * N + n]), e[n] += fabs(x) * er[r * N + n];
            }
            for (int64_t n = 0; n < N; ++n)
                compare("dw", dw, d.order ? n : i, d.order ? i : n, v[n], z[n], e[n], M);
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

const Type F32{CLIFF_F32, 4, 0x1p-24, 1e-37};

int norm(Case& k)
{
    const int64_t R = k.f.i("rows"), d = k.f.i("d");
    const bool in_place = k.f.i("in_place");
    const double eps = 1e-5;
    Mat x, w, b, y, mean, rstd;
    rows(k, x, "x", R, d);
    x.fill(k.g, 1.5f, 0.7f);
    if (k.f.i("w")) w.make(k.t, 1, d, d, k.f.i("off")), w.fill(k.g, 1);
    if (k.f.i("b")) b.make(k.t, 1, d, d, k.f.i("off")), b.fill(k.g, 1);
    if (!in_place) rows(k, y, "y", R, d);
    if (!k.f.i("no_stats")) mean.make(F32, 1, R, R, 0), rstd.make(F32, 1, R, R, 0);
    std::vector<double> in;
    if (!emulate::dry)
        for (int64_t r = 0; r < R; ++r)
            for (int64_t c = 0; c < d; ++c) in.push_back(x.get(r, c));
    const Mat& to = in_place ? x : y;
    const int st = cliffconv_layer_norm(k.t.code, R, d, x.ptr(), x.ld, w.ptr(), b.ptr(), eps, to.ptr(), to.ld,
                                        reinterpret_cast<float*>(mean.ptr()), reinterpret_cast<float*>(rstd.ptr()), nullptr);
    if (emulate::dry || st) return st;
    const double s = (LAMBDA * sqrt((double)d) + COST) * U;
    for (int64_t r = 0; r < R; ++r) {
        const double* v = &in[r * d];
        double m = 0, a = 0, q = 0;
        for (int64_t c = 0; c < d; ++c) m += v[c], a += fabs(v[c]);
        m /= d;
        const double em = s * a / d;
        for (int64_t c = 0; c < d; ++c) q += (v[c] - m) * (v[c] - m);
        q /= d;
        const double i = 1 / sqrt(q + eps), ei = i * (0.5 * (em * em + s * q + 2 * U * eps) * i * i + 4 * U);
        if (mean.p) {
            expect("mean", r, 0, mean.get(0, r), m, em + 1e-37);
            expect("rstd", r, 0, rstd.get(0, r), i, ei + 1e-37);
        }
        for (int64_t c = 0; c < d; ++c) {
            double h = (v[c] - m) * i, e = (em + U * fabs(v[c])) * i + fabs(v[c] - m) * ei + 4 * U * fabs(h);
            if (w.p) h *= w.get(0, c), e = e * fabs(w.get(0, c)) + 2 * U * fabs(h);
            if (b.p) e += 2 * U * (fabs(h) + fabs(b.get(0, c))), h += b.get(0, c);
            expect("y", r, c, to.get(r, c), h, rounded(k.t, e, h));
        }
    }
    return st;
}

int norm_backward(Case& k)
{
    const int64_t R = k.f.i("rows"), d = k.f.i("d");
    const bool in_place = k.f.i("in_place");
    const int want = (int)k.f.i("want", 6);  // 2 dweight, 4 dbias
    Mat x, dy, res, w, dx, dw, db, mean, rstd;
    rows(k, x, "x", R, d);
    rows(k, dy, "dy", R, d);
    if (k.f.m.count("constant")) x.fill(k.g, 0, (float)k.f.d("constant"));
    else x.fill(k.g, 1.5f, 0.7f);
    dy.fill(k.g, 1);
    if (k.f.i("residual")) rows(k, res, "res", R, d), res.fill(k.g, 1);
    if (k.f.i("w")) w.make(k.t, 1, d, d, k.f.i("off")), w.fill(k.g, 1);
    if (!in_place) rows(k, dx, "dx", R, d);
    if (want & 2) dw.make(k.t, 1, d, d, k.f.i("off"));
    if (want & 4) db.make(k.t, 1, d, d, k.f.i("off"));
    mean.make(F32, 1, R, R, 0);
    rstd.make(F32, 1, R, R, 0);
    std::vector<double> in;
    if (!emulate::dry)
        for (int64_t r = 0; r < R; ++r) {
            double m = 0, q = 0;
            for (int64_t c = 0; c < d; ++c) m += x.get(r, c);
            mean.set(0, r, (float)(m / d));
            for (int64_t c = 0; c < d; ++c) q += pow(x.get(r, c) - mean.get(0, r), 2), in.push_back(dy.get(r, c));
            rstd.set(0, r, (float)(1 / sqrt(q / d + 1e-5)));
        }
    const int64_t need = want ? cliffconv_layer_norm_backward_workspace(k.t.code, R, d) : 0;
    k.workspace(need);
    const Mat& to = in_place ? dy : dx;
    const int st = cliffconv_layer_norm_backward(
        k.t.code, R, d, dy.ptr(), dy.ld, x.ptr(), x.ld, reinterpret_cast<float*>(mean.ptr()),
        reinterpret_cast<float*>(rstd.ptr()), w.ptr(), res.ptr(), res.ld, to.ptr(), to.ld, dw.ptr(), db.ptr(),
        need ? k.ws.ptr() : nullptr, need, nullptr);
    if (emulate::dry || st) return st;
    const double s = (LAMBDA * sqrt((double)d) + COST) * U, sr = (LAMBDA * sqrt((double)std::max<int64_t>(R, 1)) + COST) * U;
    std::vector<double> sw(d), zw(d), ew(d), sb(d), zb(d);
    for (int64_t r = 0; r < R; ++r) {
        const double m = mean.get(0, r), i = rstd.get(0, r);
        double mq = 0, mqh = 0, aq = 0, aqh = 0, aqe = 0;
        auto h = [&](int64_t c) { return (x.get(r, c) - m) * i; };
        auto eh = [&](int64_t c) { return 4 * U * (fabs(h(c)) + (fabs(x.get(r, c)) + fabs(m)) * i); };
        auto q = [&](int64_t c) { return in[r * d + c] * (w.p ? w.get(0, c) : 1); };
        for (int64_t c = 0; c < d; ++c) {
            mq += q(c), aq += fabs(q(c)), mqh += q(c) * h(c), aqh += fabs(q(c) * h(c)), aqe += fabs(q(c)) * eh(c);
            const double g = in[r * d + c];
            sw[c] += g * h(c), zw[c] += fabs(g * h(c)), ew[c] += fabs(g) * eh(c), sb[c] += g, zb[c] += fabs(g);
        }
        mq /= d, mqh /= d;
        const double emq = s * aq / d, emqh = s * aqh / d + aqe / d;
        for (int64_t c = 0; c < d; ++c) {
            double v = i * (q(c) - mq - h(c) * mqh);
            double e = i * (emq + fabs(h(c)) * emqh + eh(c) * fabs(mqh) + COST * U * (fabs(q(c)) + fabs(mq) + fabs(h(c) * mqh)));
            if (res.p) e += 2 * U * (fabs(v) + fabs(res.get(r, c))), v += res.get(r, c);
            expect("dx", r, c, to.get(r, c), v, rounded(k.t, e, v));
        }
    }
    for (int64_t c = 0; c < d; ++c) {
        if (want & 2) expect("dweight", 0, c, dw.get(0, c), sw[c], rounded(k.t, ew[c] + sr * zw[c], sw[c]));
        if (want & 4) expect("dbias", 0, c, db.get(0, c), sb[c], rounded(k.t, sr * zb[c], sb[c]));
    }
    return st;
}

int dropout(Case& k)
{
    const int64_t R = k.f.i("rows"), d = k.f.i("d");
    const bool in_place = k.f.i("in_place");
    Mat x, res, y;
    rows(k, x, "x", R, d);
    x.fill(k.g, 1);
    if (k.f.i("residual")) rows(k, res, "res", R, d), res.fill(k.g, 1);
    if (!in_place) rows(k, y, "y", R, d);
    std::vector<double> in;
    if (!emulate::dry)
        for (int64_t r = 0; r < R; ++r)
            for (int64_t c = 0; c < d; ++c) in.push_back(x.get(r, c));
    const Mat& to = in_place ? x : y;
    const int st = cliffconv_dropout(k.t.code, R, d, x.ptr(), x.ld, &k.desc, res.ptr(), res.ld, to.ptr(), to.ld, nullptr);
    if (emulate::dry || st) return st;
    for (int64_t r = 0; r < R; ++r)
        for (int64_t c = 0; c < d; ++c) {
            double v = in[r * d + c] * factor(k.p, k.rng.get(), r, c), e = 2 * U * fabs(v);
            if (res.p) e += 2 * U * (fabs(v) + fabs(res.get(r, c))), v += res.get(r, c);
            expect("y", r, c, to.get(r, c), v, rounded(k.t, e, v));
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
            st = op == "dense" ? dense(k) : op == "backward" ? backward(k) : op == "norm" ? norm(k)
               : op == "norm_backward" ? norm_backward(k) : op == "dropout" ? dropout(k) : -1;
        }
        if (!failure.empty()) printf("FAIL %s\n", failure.c_str());
        else printf("ok %d %llu\n", st, (unsigned long long)emulate::most_threads);
        fflush(stdout);
        fflush(stderr);
    }
    return 0;
}
