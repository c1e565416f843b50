// The norms after and before a block, its gate and the scaled residual in one pass
// over rows, and their gradient:
//   out = scale residual + gate n(x),   normed = n(out)
// (n: layer norm with its weight and bias, or the same without mean).
//
// Bound by memory: forward reads x and the residual and writes out and normed,
// backward reads dout, dnormed, x and out and writes dx and dresidual.  A row lies
// in the registers of TPR threads as in layer norm (rows.hpp), between its two norms
// in fp32.  524288 x 128 fp32 forward 216 us (5.0 TB/s), 8192 x 4096 fp32 99 (5.4);
// backward 16384 x 4096 bf16 171 us with its sums (4.7 TB/s), 266 with sixteen columns in
// a thread, vectors loaded anew for each row and no loads ahead; 4 x 4096 bf16 5.4 us.
#include <stdio.h>

#include <algorithm>

#include "rows.hpp"

namespace cliff {
namespace {

// What the vectors [d] hold from column col on; `otherwise` where there is none.
template <typename T>
__device__ inline void vector_or(const void* v, float otherwise, int col, int64_t d, float (&to)[per16<T>])
{
    if (v) {
        load_vector(static_cast<const T*>(v), col, d, to);
    } else {
#pragma unroll
        for (int e = 0; e < per16<T>; ++e) to[e] = otherwise;
    }
}

// The pieces of a vector [d] that a thread has, loaded early and unpacked where they
// are used (of elements past the end, anything).
template <typename T, int TPR, int C>
struct Pieces {
    raw16 r[C];
    __device__ void load(const void* v, int t, int64_t d)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * per16<T>;
            r[c] = raw16{0, 0, 0, 0};
            if (v) r[c] = load_piece(static_cast<const T*>(v), col, d);
        }
    }
    __device__ void get(const void* v, float otherwise, int c, int t, int64_t d, float (&to)[per16<T>]) const
    {
        raw16 p = r[c];
        if (d >= per16<T>) settle16<T>(p, (c * TPR + t) * per16<T>, d);
        unpack16<T>(p, to);
        if (!v)
#pragma unroll
            for (int e = 0; e < per16<T>; ++e) to[e] = otherwise;
    }
};

// Workgroups of the kernels here: 64 threads or fewer per row share one of 256.
constexpr int block_threads(int TPR) { return TPR > 64 ? TPR : 256; }

// The row of the gate that belongs to a row.
template <typename T>
__device__ inline const T* gate_of(const void* gate, int64_t d, int64_t rows_per_gate, int64_t rows, int64_t r)
{
    return static_cast<const T*>(gate) + (rows_per_gate == rows ? 0 : r / rows_per_gate * d);
}

// Mean (zero with rms) and 1 / standard deviation of R rows in registers, columns
// past the end zero.
template <int TPR, int R, int C, int E, int LDS>
__device__ inline void moments(const float (&v)[R][C][E], int t, int d, bool rms, float eps, float (&mean)[R],
                               float (&rstd)[R], float (&lds)[2][LDS], int& turn)
{
    const float inv = 1.0f / (float)d;
#pragma unroll
    for (int r = 0; r < R; ++r) mean[r] = rstd[r] = 0.f;
    if (!rms) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) mean[r] += v[r][c][e];
        row_sums<TPR, R>(mean, lds[turn ^= 1]);
#pragma unroll
        for (int r = 0; r < R; ++r) mean[r] *= inv;
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int have = d - (c * TPR + t) * E;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float u = e < have ? v[r][c][e] - mean[r] : 0.f;
                rstd[r] = fmaf(u, u, rstd[r]);
            }
        }
    row_sums<TPR, R>(rstd, lds[turn ^= 1]);
#pragma unroll
    for (int r = 0; r < R; ++r) rstd[r] = 1.0f / sqrtf(rstd[r] * inv + eps);
}

// How the vectors and rows come.  USED: vectors where they are used, one pass over rows
// per workgroup, several workgroups on a compute unit.  EARLY, for calls of few rows:
// one row, its vectors under way with it.  STREAM, for rows that take a compute unit's
// threads: a workgroup goes over many rows, vectors (but the gate) once, the next rows'
// loads under way while the sums of these are joined.
enum Way { USED, EARLY, STREAM };

template <typename T, int TPR, int EL, int R, Way WAY>
__global__ __launch_bounds__(block_threads(TPR)) void block_norm_kernel(BlockNormArgs a, int64_t rows_per_gate)
{
    constexpr int E = per16<T>, C = EL / E, G = block_threads(TPR) / TPR;
    __shared__ float lds[2][TPR / 64 * R + 1];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, d = (int)a.d;
    int turn = 0;
    struct Rows {
        raw16 x[R][C], res[R][C];
    };
    auto load = [&](Rows& w, int64_t r0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            // rows that do not exist give way to the last one
            const int64_t rr = r0 + (int64_t)g * R + r, row = rr < a.rows ? rr : a.rows - 1;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * TPR + t) * E;
                w.x[r][c] = load_piece(static_cast<const T*>(a.x) + row * a.ldx, col, d);
                w.res[r][c] = load_piece(static_cast<const T*>(a.residual) + row * a.ldr, col, d);
            }
        }
    };
    const int64_t first = (int64_t)blockIdx.x * G * R, step = (int64_t)gridDim.x * G * R;
    Rows now, next;
    if constexpr (WAY == STREAM) load(next, first);
    Pieces<T, TPR, C> pw, pb, pg, pnw, pnb;
    if constexpr (WAY == STREAM) {
        pw.load(a.weight, t, d);
        pb.load(a.bias, t, d);
        pnw.load(a.next_weight, t, d);
        pnb.load(a.next_bias, t, d);
    }
    for (int64_t r0 = first; r0 < a.rows; r0 += step) {
        const int64_t rg = r0 + (int64_t)g * R;
        if constexpr (WAY == STREAM) {
            now = next;
            if (r0 + step < a.rows) load(next, r0 + step);
        } else {
            load(now, r0);
        }
        auto &x = now.x, &res = now.res;
        const int64_t row0 = rg < a.rows ? rg : a.rows - 1;
        if constexpr (WAY != USED && R == 1)
            pg.load(a.gate ? gate_of<T>(a.gate, d, rows_per_gate, a.rows, row0) : nullptr, t, d);
        if constexpr (WAY == EARLY) {
            pw.load(a.weight, t, d);
            pb.load(a.bias, t, d);
            pnw.load(a.next_weight, t, d);
            pnb.load(a.next_bias, t, d);
        }
        settle_rows<T, TPR, R, C>(x, t, d);
        settle_rows<T, TPR, R, C>(res, t, d);
        float v[R][C][E], mean[R], rstd[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) unpack16<T>(x[r][c], v[r][c]);
        auto keep = [&](int which) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (a.stats && t == 0 && rg + r < a.rows) {
                    a.stats[which * a.rows + rg + r] = mean[r];
                    a.stats[(which + 1) * a.rows + rg + r] = rstd[r];
                }
        };
        if (a.after) {
            moments<TPR>(v, t, d, a.rms, a.eps, mean, rstd, lds, turn);
            keep(0);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * E, have = d - col;
            float w[E], b[E];
            if constexpr (WAY != USED) {
                pw.get(a.weight, 1.f, c, t, d, w);
                pb.get(a.bias, 0.f, c, t, d, b);
            } else {
                vector_or<T>(a.weight, 1.f, col, d, w);
                vector_or<T>(a.bias, 0.f, col, d, b);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int64_t row = rg + r < a.rows ? rg + r : a.rows - 1;
                float gate[E], u[E];
                if constexpr (WAY != USED) pg.get(a.gate, 1.f, c, t, d, gate);
                else
                    vector_or<T>(a.gate ? gate_of<T>(a.gate, d, rows_per_gate, a.rows, row) : nullptr, 1.f, col, d, gate);
                unpack16<T>(res[r][c], u);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float h = v[r][c][e];
                    if (a.after) h = fmaf((h - mean[r]) * rstd[r], w[e], b[e]);
                    if (a.gate) h *= gate[e];
                    v[r][c][e] = e < have ? fmaf(a.scale, u[e], h) : 0.f;
                }
                if (rg + r < a.rows) store16(static_cast<T*>(a.out) + (rg + r) * a.ldo + col, v[r][c], have);
            }
        }
        if (!a.before) continue;
        moments<TPR>(v, t, d, a.rms, a.eps, mean, rstd, lds, turn);
        keep(2);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * E, have = d - col;
            float w[E], b[E];
            if constexpr (WAY != USED) {
                pnw.get(a.next_weight, 1.f, c, t, d, w);
                pnb.get(a.next_bias, 0.f, c, t, d, b);
            } else {
                vector_or<T>(a.next_weight, 1.f, col, d, w);
                vector_or<T>(a.next_bias, 0.f, col, d, b);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float u[E];
#pragma unroll
                for (int e = 0; e < E; ++e) u[e] = fmaf((v[r][c][e] - mean[r]) * rstd[r], w[e], b[e]);
                if (rg + r < a.rows) store16(static_cast<T*>(a.normed) + (rg + r) * a.ldn + col, u, have);
            }
        }
    }
}

// Rows that do not fit the registers: one workgroup per row, which forms out anew
// from x and the residual for each step and writes in the last one, each piece by
// the thread that reads it (out and normed may be x or the residual).
constexpr int WIDE = 1024;
template <typename T>
__device__ inline void load_wide(const T* row, int64_t col, int64_t d, float (&v)[per16<T>])
{
    raw16 r = load16(row, col, d);
    settle16<T>(r, col, d);
    unpack16<T>(r, v);
}
template <typename T>
__device__ inline void wide_vector(const void* v, float otherwise, int64_t col, int64_t d, float (&to)[per16<T>])
{
    if (v) {
        load_wide(static_cast<const T*>(v), col, d, to);
    } else {
#pragma unroll
        for (int e = 0; e < per16<T>; ++e) to[e] = otherwise;
    }
}
template <typename T>
__global__ __launch_bounds__(WIDE) void block_norm_wide_kernel(BlockNormArgs a, int64_t rows_per_gate)
{
    constexpr int E = per16<T>;
    __shared__ float lds[2][WIDE / 64];
    int turn = 0;
    const float inv = 1.0f / (float)a.d;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* const x = static_cast<const T*>(a.x) + r * a.ldx;
        const T* const res = static_cast<const T*>(a.residual) + r * a.ldr;
        const T* const gate = a.gate ? gate_of<T>(a.gate, a.d, rows_per_gate, a.rows, r) : nullptr;
        // the sum over the row of what f gives for the values that `values` gives
        auto sum = [&](auto values, auto f) {
            float s[1] = {0.f};
            for (int64_t c = threadIdx.x * (int64_t)E; c < a.d; c += WIDE * E) {
                float v[E];
                values(c, v);
#pragma unroll
                for (int e = 0; e < E; ++e) s[0] += c + e < a.d ? f(v[e]) : 0.f;
            }
            row_sums<WIDE, 1>(s, lds[turn ^= 1]);
            return s[0] * inv;
        };
        float mean = 0.f, rstd = 1.f;
        auto measure = [&](int which, auto values) {
            float m = 0.f;
            if (!a.rms) m = sum(values, [](float v) { return v; });
            const float q = sum(values, [&](float v) { return (v - m) * (v - m); });
            mean = m;
            rstd = 1.0f / sqrtf(q + a.eps);
            if (a.stats && threadIdx.x == 0) {
                a.stats[which * a.rows + r] = mean;
                a.stats[(which + 1) * a.rows + r] = rstd;
            }
        };
        if (a.after) measure(0, [&](int64_t c, float (&v)[E]) { load_wide(x, c, a.d, v); });
        const float mean1 = mean, rstd1 = rstd;
        auto row = [&](int64_t c, float (&v)[E]) {
            float w[E], b[E], g[E], u[E];
            load_wide(x, c, a.d, v);
            load_wide(res, c, a.d, u);
            wide_vector<T>(a.weight, 1.f, c, a.d, w);
            wide_vector<T>(a.bias, 0.f, c, a.d, b);
            wide_vector<T>(gate, 1.f, c, a.d, g);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float h = v[e];
                if (a.after) h = fmaf((h - mean1) * rstd1, w[e], b[e]);
                v[e] = fmaf(a.scale, u[e], h * g[e]);
            }
        };
        if (a.before) measure(2, row);
        for (int64_t c = threadIdx.x * (int64_t)E; c < a.d; c += WIDE * E) {
            const int have = a.d - c < E ? (int)(a.d - c) : E;
            float v[E], w[E], b[E];
            row(c, v);
            // (a piece that passes the end comes with columns of another thread, which may
            // write them, and drops them)
            store16(static_cast<T*>(a.out) + r * a.ldo + c, v, have);
            if (!a.before) continue;
            wide_vector<T>(a.next_weight, 1.f, c, a.d, w);
            wide_vector<T>(a.next_bias, 0.f, c, a.d, b);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = fmaf((v[e] - mean) * rstd, w[e], b[e]);
            store16(static_cast<T*>(a.normed) + r * a.ldn + c, v, have);
        }
    }
}

// ---- the gradient

// The rows are cut into parts, `per_gate` of them for each gate, and a part's sums
// over its rows are [4][d] in the workspace:
//   A = sum t h,  B = sum t,  C = sum dnormed k,  D = sum dnormed.
struct Parts {
    int64_t gates, rows_per_gate, per_gate, chunk;  // chunk: rows of a part
    int64_t all() const { return gates * per_gate; }
};

// The next rows' loads are under way while the sums of these are joined, where the
// registers hold both.
// EACH: every row has a gate of its own, which comes and whose gradient
//   weight A + bias B = v (h weight + bias)
// goes with the row, and the sums over all rows are of gate A and gate B at once
// (bf16, both norms with their vectors: 65536 x 1024 in 238 us, and 2459 with the sums of
// each gate in memory; 16384 x 4096 in 226 and 2341; one gate for all rows 186 and 171).
template <typename T, int TPR, int EL, int R, bool EACH>
__global__ __launch_bounds__(block_threads(TPR), TPR < 1024 ? 2 : 4) void block_norm_backward_kernel(BlockNormBackwardArgs a,
                                                                                              Parts parts, float* sums)
{
    constexpr int E = per16<T>, C = EL / E, NT = block_threads(TPR), G = NT / TPR;
    __shared__ float lds[2][TPR / 64 * 2 * R + 1];
    __shared__ float join[G > 1 ? NT * EL : 1];
    if (blockIdx.y && workgroup_id() >= (uint64_t)parts.gates * parts.per_gate) return;
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, d = (int)a.d;
    const int64_t part = workgroup_id(), which = part / parts.per_gate, sub = part - which * parts.per_gate;
    const int64_t begin = which * parts.rows_per_gate + sub * parts.chunk;
    const int64_t last = (which + 1) * parts.rows_per_gate;
    const int64_t end = begin + parts.chunk < last ? begin + parts.chunk : last;
    const T* const gate = a.gate && !EACH ? static_cast<const T*>(a.gate) + which * a.d : nullptr;
    const float inv = 1.0f / (float)a.d;
    float sum[4][C][E];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[k][c][e] = 0.f;
    int turn = 0;
    struct Rows {
        raw16 dout[R][C], dn[R][C], x[R][C], out[R][C], gate[EACH ? R : 1][C];
        float mean1[R], rstd1[R], mean2[R], rstd2[R];
    };
    auto load = [&](Rows& w, int64_t r0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            // rows that do not exist give way to the last one
            const int64_t row = r0 + (int64_t)g * R + r, m = row < end ? row : end - 1;
            w.mean1[r] = a.after ? a.stats[m] : 0.f;
            w.rstd1[r] = a.after ? a.stats[a.rows + m] : 1.f;
            w.mean2[r] = a.dnormed ? a.stats[2 * a.rows + m] : 0.f;
            w.rstd2[r] = a.dnormed ? a.stats[3 * a.rows + m] : 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * TPR + t) * E;
                w.dout[r][c] = w.dn[r][c] = w.x[r][c] = w.out[r][c] = raw16{0, 0, 0, 0};
                if (a.dout) w.dout[r][c] = load_piece(static_cast<const T*>(a.dout) + m * a.lddo, col, d);
                if (a.dnormed) {
                    w.dn[r][c] = load_piece(static_cast<const T*>(a.dnormed) + m * a.lddn, col, d);
                    w.out[r][c] = load_piece(static_cast<const T*>(a.out) + m * a.ldo, col, d);
                }
                if (a.x) w.x[r][c] = load_piece(static_cast<const T*>(a.x) + m * a.ldx, col, d);
                if constexpr (EACH) w.gate[r][c] = load_piece(static_cast<const T*>(a.gate) + m * a.d, col, d);
            }
        }
    };
    constexpr bool AHEAD = TPR < 1024;
    Rows now, next;
    if constexpr (AHEAD) load(next, begin);
    // the vectors, once for all rows: next_weight, and what t is multiplied by on its way to
    // the norm after the block (without it to dx), gate weight (EACH: weight, and bias)
    float nws[C][E], gws[C][E], bs[EACH ? C : 1][E];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * E;
        float gv[E];
        vector_or<T>(a.next_weight, 1.f, col, d, nws[c]);
        vector_or<T>(a.weight, 1.f, col, d, gws[c]);
        vector_or<T>(gate, 1.f, col, d, gv);
#pragma unroll
        for (int e = 0; e < E; ++e) gws[c][e] *= gv[e];
        if constexpr (EACH) vector_or<T>(a.after ? a.bias : nullptr, 0.f, col, d, bs[c]);
    }
    for (int64_t r0 = begin; r0 < end; r0 += G * R) {
        const int64_t rg = r0 + (int64_t)g * R;
        if constexpr (AHEAD) {
            now = next;
            if (r0 + G * R < end) load(next, r0 + G * R);
        } else {
            load(now, r0);
        }
        auto &dout = now.dout, &dn = now.dn, &x = now.x, &out = now.out;
        auto &mean1 = now.mean1, &rstd1 = now.rstd1, &mean2 = now.mean2, &rstd2 = now.rstd2;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (rg + r >= end) {  // a row that does not exist adds nothing to the sums
                mean1[r] = rstd1[r] = mean2[r] = rstd2[r] = 0.f;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    dout[r][c] = dn[r][c] = x[r][c] = out[r][c] = raw16{0, 0, 0, 0};
                    if constexpr (EACH) now.gate[r][c] = raw16{0, 0, 0, 0};
                }
            }
        if constexpr (EACH) settle_rows<T, TPR, R, C>(now.gate, t, d);
        settle_rows<T, TPR, R, C>(dout, t, d);
        settle_rows<T, TPR, R, C>(dn, t, d);
        settle_rows<T, TPR, R, C>(x, t, d);
        settle_rows<T, TPR, R, C>(out, t, d);
        // the norm before the next block: sums of q and of q (out - mean), which rstd
        // multiplies as a whole (mean times rstd need not be a float)
        float s[2 * R];
        if (a.dnormed) {
#pragma unroll
            for (int r = 0; r < 2 * R; ++r) s[r] = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const auto& w = nws[c];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float n[E], o[E];
                    unpack16<T>(dn[r][c], n);
                    unpack16<T>(out[r][c], o);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float u = o[e] - mean2[r], q = n[e] * w[e];
                        s[2 * r] += q;
                        s[2 * r + 1] = fmaf(q, u, s[2 * r + 1]);
                        sum[2][c][e] = fmaf(n[e], u * rstd2[r], sum[2][c][e]);
                        sum[3][c][e] += n[e];
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) s[2 * r + 1] *= rstd2[r];
            row_sums<TPR, 2 * R>(s, lds[turn ^= 1]);
        }
        // t, and the same sums for the norm after the block
        float tv[R][C][E], z[2 * R];
#pragma unroll
        for (int r = 0; r < 2 * R; ++r) z[r] = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * E, have = d - col;
            const auto &nw = nws[c], &gw = gws[c];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float n[E], o[E], xv[E], dr[E], gv[E], dg[E];
                if constexpr (EACH) unpack16<T>(now.gate[r][c], gv);
                unpack16<T>(dout[r][c], tv[r][c]);
                unpack16<T>(dn[r][c], n);
                unpack16<T>(out[r][c], o);
                unpack16<T>(x[r][c], xv);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float v = tv[r][c][e];
                    if (a.dnormed) {
                        const float k = (o[e] - mean2[r]) * rstd2[r];
                        float q = n[e] * nw[e] - k * (s[2 * r + 1] * inv);
                        if (!a.rms) q -= s[2 * r] * inv;
                        v = fmaf(rstd2[r], q, v);
                    }
                    if (e >= have) v = 0.f;
                    tv[r][c][e] = v;
                    dr[e] = a.scale * v;
                    const float u = xv[e] - mean1[r];
                    float f = v;
                    if constexpr (EACH) {
                        dg[e] = v * fmaf(u * rstd1[r], gw[e], bs[c][e]);
                        f *= gv[e];
                    }
                    const float q = f * gw[e];
                    z[2 * r] += q;
                    z[2 * r + 1] = fmaf(q, u, z[2 * r + 1]);
                    sum[0][c][e] = fmaf(f, u * rstd1[r], sum[0][c][e]);
                    sum[1][c][e] += f;
                }
                if constexpr (EACH)
                    if (a.dgate && rg + r < end) store16(static_cast<T*>(a.dgate) + (rg + r) * a.d + col, dg, have);
                if (rg + r < end) store16(static_cast<T*>(a.dresidual) + (rg + r) * a.lddr + col, dr, have);
            }
        }
        if (a.after) {
#pragma unroll
            for (int r = 0; r < R; ++r) z[2 * r + 1] *= rstd1[r];
            row_sums<TPR, 2 * R>(z, lds[turn ^= 1]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * E, have = d - col;
            const auto& gw = gws[c];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float xv[E], dx[E], gv[E];
                unpack16<T>(x[r][c], xv);
                if constexpr (EACH) unpack16<T>(now.gate[r][c], gv);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float q = tv[r][c][e] * gw[e];
                    if constexpr (EACH) q = tv[r][c][e] * gv[e] * gw[e];
                    if (a.after) {
                        const float h = (xv[e] - mean1[r]) * rstd1[r];
                        q -= h * (z[2 * r + 1] * inv);
                        if (!a.rms) q -= z[2 * r] * inv;
                        q *= rstd1[r];
                    }
                    dx[e] = q;
                }
                if (rg + r < end) store16(static_cast<T*>(a.dx) + (rg + r) * a.lddx + col, dx, have);
            }
        }
    }
    if (!sums) return;
    float* const to = sums + 4 * part * a.d;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (G > 1) {
            // the groups' sums of a column, in order
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) join[g * TPR * EL + (c * TPR + t) * E + e] = sum[k][c][e];
            __syncthreads();
            for (int col = threadIdx.x; col < d; col += NT) {
                float v = 0.f;
                for (int i = 0; i < G; ++i) v += join[i * TPR * EL + col];
                to[k * a.d + col] = v;
            }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * TPR + t) * E;
                float* const at = to + k * a.d + col;
                if (col + E <= d) {
                    __builtin_memcpy(at, sum[k][c], sizeof sum[k][c]);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (col + e < d) at[e] = sum[k][c][e];
                }
            }
        }
    }
}

// Rows that do not fit the registers, in three steps: the rows' sums into row_sums
// [rows][4] (those of the norm before, then after); the sums over rows; dx and
// dresidual, each piece by the thread that reads its inputs.
struct WideRow {
    float mean1, rstd1, mean2, rstd2, s1, s2, z1, z2;
};
__device__ inline WideRow wide_row(const BlockNormBackwardArgs& a, const float* row_sums, int64_t r)
{
    WideRow w{0.f, 1.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.after) w.mean1 = a.stats[r], w.rstd1 = a.stats[a.rows + r];
    if (a.dnormed) w.mean2 = a.stats[2 * a.rows + r], w.rstd2 = a.stats[3 * a.rows + r];
    if (row_sums) w.s1 = row_sums[4 * r], w.s2 = row_sums[4 * r + 1], w.z1 = row_sums[4 * r + 2], w.z2 = row_sums[4 * r + 3];
    return w;
}
template <typename T>
__device__ inline void wide_rows(const void* m, int64_t ld, int64_t r, int64_t c, int64_t d, float (&v)[per16<T>])
{
    wide_vector<T>(m ? static_cast<const T*>(m) + r * ld : nullptr, 0.f, c, d, v);
}
// A piece of t (zero past the end); of dnormed into n and of out's normed values into k.
template <typename T>
__device__ inline void wide_t(const BlockNormBackwardArgs& a, const WideRow& w, int64_t r, int64_t c, float (&t)[per16<T>],
                              float (&n)[per16<T>], float (&k)[per16<T>])
{
    wide_rows<T>(a.dout, a.lddo, r, c, a.d, t);
    if (!a.dnormed) return;
    float nw[per16<T>];
    wide_rows<T>(a.dnormed, a.lddn, r, c, a.d, n);
    wide_rows<T>(a.out, a.ldo, r, c, a.d, k);
    wide_vector<T>(a.next_weight, 1.f, c, a.d, nw);
#pragma unroll
    for (int e = 0; e < per16<T>; ++e) {
        k[e] = (k[e] - w.mean2) * w.rstd2;
        float q = n[e] * nw[e] - k[e] * w.s2;
        if (!a.rms) q -= w.s1;
        t[e] = c + e < a.d ? fmaf(w.rstd2, q, t[e]) : 0.f;
    }
}
// gate weight of a piece, without after the gate alone
template <typename T>
__device__ inline void wide_factor(const BlockNormBackwardArgs& a, const T* gate, int64_t c, float (&f)[per16<T>])
{
    float w[per16<T>];
    wide_vector<T>(gate, 1.f, c, a.d, f);
    wide_vector<T>(a.weight, 1.f, c, a.d, w);
#pragma unroll
    for (int e = 0; e < per16<T>; ++e) f[e] *= w[e];
}

template <typename T>
__global__ __launch_bounds__(WIDE) void block_norm_wide_rows_kernel(BlockNormBackwardArgs a, int64_t rows_per_gate,
                                                                    float* to)
{
    constexpr int E = per16<T>;
    __shared__ float lds[2][2 * WIDE / 64];
    int turn = 0;
    const float inv = 1.0f / (float)a.d;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        WideRow w = wide_row(a, nullptr, r);
        const T* const gate = a.gate ? gate_of<T>(a.gate, a.d, rows_per_gate, a.rows, r) : nullptr;
        if (a.dnormed) {
            float s[2] = {0.f, 0.f};
            for (int64_t c = threadIdx.x * (int64_t)E; c < a.d; c += WIDE * E) {
                float n[E], o[E], nw[E];
                wide_rows<T>(a.dnormed, a.lddn, r, c, a.d, n);
                wide_rows<T>(a.out, a.ldo, r, c, a.d, o);
                wide_vector<T>(a.next_weight, 1.f, c, a.d, nw);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float q = n[e] * nw[e];
                    s[0] += q;
                    s[1] = fmaf(q, o[e] - w.mean2, s[1]);
                }
            }
            s[1] *= w.rstd2;
            row_sums<WIDE, 2>(s, lds[turn ^= 1]);
            w.s1 = s[0] * inv, w.s2 = s[1] * inv;
        }
        if (a.after) {
            float s[2] = {0.f, 0.f};
            for (int64_t c = threadIdx.x * (int64_t)E; c < a.d; c += WIDE * E) {
                float v[E], n[E], k[E], f[E], x[E];
                wide_t<T>(a, w, r, c, v, n, k);
                wide_factor<T>(a, gate, c, f);
                wide_rows<T>(a.x, a.ldx, r, c, a.d, x);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float q = v[e] * f[e];
                    s[0] += q;
                    s[1] = fmaf(q, x[e] - w.mean1, s[1]);
                }
            }
            s[1] *= w.rstd1;
            row_sums<WIDE, 2>(s, lds[turn ^= 1]);
            w.z1 = s[0] * inv, w.z2 = s[1] * inv;
        }
        if (threadIdx.x == 0) to[4 * r] = w.s1, to[4 * r + 1] = w.s2, to[4 * r + 2] = w.z1, to[4 * r + 3] = w.z2;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void block_norm_wide_sums_kernel(BlockNormBackwardArgs a, Parts parts,
                                                                   const float* rows, float* sums, uint32_t blocks)
{
    constexpr int E = per16<T>;
    const uint32_t id = workgroup_id();
    const int64_t part = id / blocks, c = ((id - part * blocks) * 256ll + threadIdx.x) * E;
    if (part >= parts.gates * parts.per_gate || c >= a.d) return;
    const int64_t which = part / parts.per_gate, begin = which * parts.rows_per_gate + (part - which * parts.per_gate) * parts.chunk;
    const int64_t last = (which + 1) * parts.rows_per_gate;
    const int64_t end = begin + parts.chunk < last ? begin + parts.chunk : last;
    float s[4][E];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) s[k][e] = 0.f;
#pragma unroll 2
    for (int64_t r = begin; r < end; ++r) {
        const WideRow w = wide_row(a, rows, r);
        float t[E], n[E], k[E], x[E];
        wide_t<T>(a, w, r, c, t, n, k);
        wide_rows<T>(a.x, a.ldx, r, c, a.d, x);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            s[0][e] = fmaf(t[e], (x[e] - w.mean1) * w.rstd1, s[0][e]);
            s[1][e] += t[e];
            if (a.dnormed) {
                s[2][e] = fmaf(n[e], k[e], s[2][e]);
                s[3][e] += n[e];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e < a.d) sums[(4 * part + k) * a.d + c + e] = s[k][e];
}

template <typename T>
__global__ __launch_bounds__(256) void block_norm_wide_dx_kernel(BlockNormBackwardArgs a, int64_t rows_per_gate,
                                                                 const float* rows, uint32_t blocks)
{
    constexpr int E = per16<T>;
    const uint32_t id = workgroup_id();
    const int64_t r = id / blocks, c = ((id - r * blocks) * 256ll + threadIdx.x) * E;
    if (r >= a.rows || c >= a.d) return;
    const int have = a.d - c < E ? (int)(a.d - c) : E;
    const WideRow w = wide_row(a, rows, r);
    const T* const gate = a.gate ? gate_of<T>(a.gate, a.d, rows_per_gate, a.rows, r) : nullptr;
    float t[E], n[E], k[E], x[E], f[E];
    wide_t<T>(a, w, r, c, t, n, k);
    wide_rows<T>(a.x, a.ldx, r, c, a.d, x);
    wide_factor<T>(a, gate, c, f);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        float q = t[e] * f[e];
        if (a.after) {
            q -= (x[e] - w.mean1) * w.rstd1 * w.z2;
            if (!a.rms) q -= w.z1;
            q *= w.rstd1;
        }
        x[e] = q;
        t[e] *= a.scale;
    }
    store16(static_cast<T*>(a.dresidual) + r * a.lddr + c, t, have);
    store16(static_cast<T*>(a.dx) + r * a.lddx + c, x, have);
}

// One value of a vector [d], or what there is without one.
template <typename T>
__device__ inline float wide_value(const void* v, int64_t i, float otherwise)
{
    return v ? (float)static_cast<const T*>(v)[i] : otherwise;
}

// Joins a gate's parts in a fixed order: 16 columns per workgroup, whose threads are
// [subset][sum][column], every SUBSETS-th part per subset.  Writes dgate, and the sums
// that the gates still have to be joined of, gate A, gate B, C and D, to `each`
// [gates][4][d]; with one gate those are the results.
template <typename T, int SUBSETS>
__global__ __launch_bounds__(64 * SUBSETS) void block_norm_gate_kernel(BlockNormBackwardArgs a, Parts parts,
                                                                       const float* sums, float* each, uint32_t blocks)
{
    __shared__ float s[SUBSETS][4][16];
    const uint32_t id = workgroup_id();
    const int lane = threadIdx.x & 15, k = threadIdx.x >> 4 & 3, subset = threadIdx.x >> 6;
    const int64_t which = id / blocks, c = (id - which * blocks) * 16ll + lane;
    float v = 0.f;
    if (which < parts.gates && c < a.d) {
        const float* const from = sums + 4 * which * parts.per_gate * a.d + k * a.d + c;
#pragma unroll 8
        for (int64_t i = subset; i < parts.per_gate; i += SUBSETS) v += from[4 * i * a.d];
    }
    s[subset][k][lane] = v;
    __syncthreads();
    if (which >= parts.gates || threadIdx.x >= 16 || c >= a.d) return;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < SUBSETS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] += s[i][j][lane];
    if (a.dgate) {
        float g = w[0];
        if (a.after) g = fmaf(g, wide_value<T>(a.weight, c, 1.f), wide_value<T>(a.bias, c, 0.f) * w[1]);
        static_cast<T*>(a.dgate)[which * a.d + c] = (T)g;
    }
    const float gate = wide_value<T>(a.gate, which * a.d + c, 1.f);
    w[0] *= gate;
    w[1] *= gate;
    if (each) {
#pragma unroll
        for (int j = 0; j < 4; ++j) each[(4 * which + j) * a.d + c] = w[j];
        return;
    }
    void* const to[4] = {a.dweight, a.dbias, a.dnext_weight, a.dnext_bias};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (to[j]) static_cast<T*>(to[j])[c] = (T)w[j];
}

// Joins the gates' sums in a fixed order: 64 of the 4 d columns per workgroup, every
// 16th gate per wave.
template <typename T>
__global__ __launch_bounds__(1024) void block_norm_join_kernel(BlockNormBackwardArgs a, const float* each, int64_t gates)
{
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = workgroup_id() * 64ll + lane;
    float v = 0.f;
    if (c < 4 * a.d) {
#pragma unroll 8
        for (int64_t i = wave; i < gates; i += 16) v += each[4 * a.d * i + c];
    }
    s[wave][lane] = v;
    __syncthreads();
    if (wave || c >= 4 * a.d) return;
    v = 0.f;
    for (int i = 0; i < 16; ++i) v += s[i][lane];
    const int64_t k = c / a.d;
    void* const to = k == 0 ? a.dweight : k == 1 ? a.dbias : k == 2 ? a.dnext_weight : a.dnext_bias;
    if (to) static_cast<T*>(to)[c - k * a.d] = (T)v;
}

// How a row is spread, as with_spread: eight elements in a thread, which has four sums
// of each in the gradient, and between its two norms what registers hold of R rows.
template <bool BACKWARD, typename F>
bool with_block_spread(int64_t d, F&& f)
{
    constexpr int R = BACKWARD ? 2 : 4;
    if (d <= 16 * 8) f.template operator()<16, 8, R>();
    else if (d <= 32 * 8) f.template operator()<32, 8, R>();
    else if (d <= 64 * 8) f.template operator()<64, 8, R>();
    else if (d <= 128 * 8) f.template operator()<128, 8, R>();
    else if (d <= 256 * 8) f.template operator()<256, 8, R>();
    else if (d <= 512 * 8) f.template operator()<512, 8, BACKWARD ? 2 : 1>();
    else if (d <= 1024 * 8) f.template operator()<1024, 8, 1>();
    else return false;
    return true;
}

template <typename T>
struct Forward {
    const BlockNormArgs& a;
    int64_t rows_per_gate;
    hipStream_t stream;
    template <int TPR, int EL, int R>
    void operator()()
    {
        // few rows: one each, for every compute unit has one
        const int64_t cus = std::max(device_cus(), 1), groups = block_threads(TPR) / TPR;
        // (4096 columns: 8192 rows of fp32 99 us as a stream and 121 otherwise, 16384 of bf16
        // 111 and 174)
        if constexpr (TPR > 256) launch<TPR, EL, 1, STREAM>(1024 / TPR * cus);
        else if (a.rows <= cus * groups * R) launch<TPR, EL, 1, EARLY>(1 << 20);
        else launch<TPR, EL, R, USED>(1 << 20);
    }
    template <int TPR, int EL, int R, Way WAY>
    void launch(int64_t most)
    {
        constexpr int per_pass = block_threads(TPR) / TPR * R;
        const int64_t blocks = std::min(ceil_div(a.rows, per_pass), most);
        if (debug_enabled())
            fprintf(stderr, "cliffconv: block_norm %lld x %lld, %d threads per row, %lld workgroups\n",
                    (long long)a.rows, (long long)a.d, TPR, (long long)blocks);
        hipLaunchKernelGGL((block_norm_kernel<T, TPR, EL, R, WAY>), dim3((unsigned)blocks), dim3(block_threads(TPR)), 0,
                           stream, a, rows_per_gate);
    }
};

// How the gradient's rows are cut: each part writes 4 d sums, so no more of them than
// keep the memory busy.
struct BackwardParts {
    template <int TPR, int EL, int R>
    void operator()()
    {
        rows_per_pass = block_threads(TPR) / TPR * R;
        per_cu = std::max(1, 512 / block_threads(TPR));
    }
    int64_t rows_per_pass = 16, per_cu = 2;
};
// Every row has a gate of its own, of rows that fit the registers.
bool gate_of_each(int64_t rows, int64_t d, int64_t gates)
{
    BackwardParts b;
    return gates > 1 && gates == rows && with_block_spread<true>(d, b);
}
Parts cut(int64_t rows, int64_t d, int64_t gates)
{
    Parts p;
    BackwardParts b;
    const bool fits = with_block_spread<true>(d, b);
    const int64_t cus = std::max(device_cus(), 1);
    p.gates = gate_of_each(rows, d, gates) ? 1 : std::max<int64_t>(gates, 1);
    p.rows_per_gate = rows / p.gates;
    const int64_t want = fits ? b.per_cu * cus : std::max<int64_t>(1, ceil_div(8 * cus, ceil_div(d, 1024)));
    p.per_gate = std::max<int64_t>(1, std::min(ceil_div(p.rows_per_gate, b.rows_per_pass), ceil_div(want, p.gates)));
    p.chunk = ceil_div(ceil_div(p.rows_per_gate, p.per_gate), b.rows_per_pass) * b.rows_per_pass;
    p.per_gate = std::max<int64_t>(1, p.chunk ? ceil_div(p.rows_per_gate, p.chunk) : 1);
    return p;
}

template <typename T>
struct Backward {
    const BlockNormBackwardArgs& a;
    const Parts& parts;
    float* sums;
    hipStream_t stream;
    template <int TPR, int EL, int R>
    void operator()()
    {
        if (debug_enabled())
            fprintf(stderr, "cliffconv: block_norm_backward %lld x %lld, %d threads per row, %lld workgroups\n",
                    (long long)a.rows, (long long)a.d, TPR, (long long)parts.all());
        constexpr int ROWS = sizeof(T) == 4 ? 1 : R;  // what the registers hold
        if (gate_of_each(a.rows, a.d, a.gate ? a.gates : 0))
            hipLaunchKernelGGL((block_norm_backward_kernel<T, TPR, EL, ROWS, true>), grid_of(parts.all()),
                               dim3(block_threads(TPR)), 0, stream, a, parts, sums);
        else
            hipLaunchKernelGGL((block_norm_backward_kernel<T, TPR, EL, ROWS, false>), grid_of(parts.all()),
                               dim3(block_threads(TPR)), 0, stream, a, parts, sums);
    }
};

// Workspace: the parts' sums, the gates' sums, and the sums of rows that do not fit
// the registers.
struct Space {
    int64_t each, rows, all;
};
Space space(const Parts& p, int64_t rows, int64_t d)
{
    Space s;
    BackwardParts b;
    s.each = ceil_div(p.all() * 16 * d, 256) * 256;
    s.rows = s.each + (p.gates > 1 ? ceil_div(p.gates * 16 * d, 256) * 256 : 0);
    s.all = s.rows + (with_block_spread<true>(d, b) ? 0 : 16 * rows);
    return s;
}

}  // namespace

cliff_status launch_block_norm(int dtype, const BlockNormArgs& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const int64_t rows_per_gate = a.gate ? a.rows / a.gates : a.rows;
        if (!with_block_spread<false>(a.d, Forward<T>{a, rows_per_gate, stream}))
            hipLaunchKernelGGL(block_norm_wide_kernel<T>, dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(WIDE),
                               0, stream, a, rows_per_gate);
        return launched();
    });
}

int64_t block_norm_backward_workspace(int, int64_t rows, int64_t d, int64_t gates)
{
    return space(cut(rows, d, gates), rows, d).all;
}

cliff_status launch_block_norm_backward(int dtype, const BlockNormBackwardArgs& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const Parts parts = cut(a.rows, a.d, a.gates);
        const Space s = space(parts, a.rows, a.d);
        char* const ws = static_cast<char*>(a.workspace);
        float* const sums = reinterpret_cast<float*>(ws);
        float* const rows = reinterpret_cast<float*>(ws + s.rows);
        const bool each_row = gate_of_each(a.rows, a.d, a.gate ? a.gates : 0);
        const bool params = (a.dgate && !each_row) || a.dweight || a.dbias || a.dnext_weight || a.dnext_bias;
        const int64_t blocks = ceil_div(a.d, 256 * per16<T>), cols = ceil_div(a.d, 16);
        // (rows of the grid are 16 bits; matrices of 2^36 elements and more)
        if (std::max(cols * parts.all(), a.d > 8192 ? blocks * a.rows : 0) > GRID_ROW * 0xffff) return CLIFF_EUNSUPPORTED;
        if (a.rows && !with_block_spread<true>(a.d, Backward<T>{a, parts, params ? sums : nullptr, stream})) {
            hipLaunchKernelGGL(block_norm_wide_rows_kernel<T>, dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)),
                               dim3(WIDE), 0, stream, a, parts.rows_per_gate, rows);
            if (params)
                hipLaunchKernelGGL(block_norm_wide_sums_kernel<T>, grid_of(blocks * parts.all()), dim3(256), 0, stream,
                                   a, parts, rows, sums, (uint32_t)blocks);
            hipLaunchKernelGGL(block_norm_wide_dx_kernel<T>, grid_of(blocks * a.rows), dim3(256), 0, stream, a,
                               parts.rows_per_gate, rows, (uint32_t)blocks);
        }
        if (params) {
            float* const each = parts.gates > 1 ? reinterpret_cast<float*>(ws + s.each) : nullptr;
            Parts join = parts;
            BlockNormBackwardArgs left = a;
            if (!a.rows) join.per_gate = 0;
            if (each_row) left.gate = left.dgate = nullptr;  // (the sums have the gates in them)
            if (parts.per_gate >= 16)
                hipLaunchKernelGGL((block_norm_gate_kernel<T, 16>), grid_of(cols * parts.gates), dim3(1024), 0, stream, left,
                                   join, sums, each, (uint32_t)cols);
            else
                hipLaunchKernelGGL((block_norm_gate_kernel<T, 1>), grid_of(cols * parts.gates), dim3(64), 0, stream, left,
                                   join, sums, each, (uint32_t)cols);
            if (each && (a.dweight || a.dbias || a.dnext_weight || a.dnext_bias))
                hipLaunchKernelGGL(block_norm_join_kernel<T>, grid_of(ceil_div(4 * a.d, 64)), dim3(1024), 0, stream, a,
                                   each, parts.gates);
        }
        return launched();
    });
}

}  // namespace cliff
