// Layer norm over the columns of rows, forward and backward.
//
// Both are bound by memory: forward reads x and writes y, backward reads dy, x
// (and the residual's gradient) and writes dx.  A row lies in the registers of
// TPR threads, EL elements each (16-byte pieces, threads next to each other),
// so the mean, the sum of squares about it and the output come from one read;
// R rows at a time keep enough loads in flight and share the barriers.
// 1048576 x 128 fp32 forward 197 us (5.5 TB/s); 16384 x 4096 bf16 backward with a
// residual's gradient 120 us (4.5 TB/s); 4 x 4096 bf16 4 us, a launch.
#include <stdio.h>

#include <algorithm>

#include "rows.hpp"

namespace cliff {
namespace {

// Rows per workgroup and pass: wg_threads / TPR groups of R.
template <typename T, int TPR, int EL, int R>
__global__ __launch_bounds__(wg_threads(TPR)) void norm_kernel(NormArgs a)
{
    constexpr int E = per16<T>, C = EL / E, G = wg_threads(TPR) / TPR;
    __shared__ float lds[2][TPR / 64 * R + 1];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const T* w = static_cast<const T*>(a.weight);
    const T* b = static_cast<const T*>(a.bias);
    const float inv = 1.0f / (float)a.d;
    for (int64_t r0 = (int64_t)blockIdx.x * G * R; r0 < a.rows; r0 += (int64_t)gridDim.x * G * R) {
        const int64_t rg = r0 + (int64_t)g * R;
        int64_t rows[R];  // those that do not exist give way to the last one
#pragma unroll
        for (int r = 0; r < R; ++r) rows[r] = rg + r < a.rows ? rg + r : a.rows - 1;
        raw16 x[R][C];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * TPR + t) * E;
                x[r][c] = load_piece(static_cast<const T*>(a.x) + rows[r] * a.ldx, col, a.d);
            }
        settle_rows<T, TPR, R, C>(x, t, a.d);
        float mean[R], sq[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean[r] = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float v[E];
                unpack16<T>(x[r][c], v);
#pragma unroll
                for (int e = 0; e < E; ++e) mean[r] += v[e];
            }
        }
        row_sums<TPR, R>(mean, lds[0]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean[r] *= inv;
            sq[r] = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int have = (int)a.d - (c * TPR + t) * E;
                float v[E];
                unpack16<T>(x[r][c], v);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float u = e < have ? v[e] - mean[r] : 0.f;
                    sq[r] = fmaf(u, u, sq[r]);
                }
            }
        }
        row_sums<TPR, R>(sq, lds[1]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sq[r] = 1.0f / sqrtf(sq[r] * inv + a.eps);
            if (t == 0 && rg + r < a.rows) {
                if (a.mean) a.mean[rg + r] = mean[r];
                if (a.rstd) a.rstd[rg + r] = sq[r];
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * E, have = (int)a.d - col;
            float vw[E], vb[E];
            if (w) load_vector(w, col, a.d, vw);
            if (b) load_vector(b, col, a.d, vb);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float v[E];
                unpack16<T>(x[r][c], v);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    v[e] = (v[e] - mean[r]) * sq[r];
                    if (w) v[e] *= vw[e];
                    if (b) v[e] += vb[e];
                }
                if (rg + r < a.rows) store16(static_cast<T*>(a.y) + (rg + r) * a.ldy + col, v, have);
            }
        }
    }
}

// The gradient: dx, and each workgroup's sums over its rows for the weight and
// bias into the workspace [workgroup][2][d] (if wanted).
template <typename T, int TPR, int EL, int R>
__global__ __launch_bounds__(wg_threads(TPR), 2) void norm_backward_kernel(NormBackwardArgs a, float* sums)
{
    constexpr int E = per16<T>, C = EL / E, NT = wg_threads(TPR), G = NT / TPR;
    __shared__ float lds[2][TPR / 64 * 2 * R + 1];
    __shared__ float join[G > 1 ? NT * EL : 1];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const T* w = static_cast<const T*>(a.weight);
    const float inv = 1.0f / (float)a.d;
    float dw[C][E], db[C][E];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < E; ++e) dw[c][e] = db[c][e] = 0.f;
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * G * R; r0 < a.rows; r0 += (int64_t)gridDim.x * G * R, turn ^= 1) {
        const int64_t rg = r0 + (int64_t)g * R;
        raw16 x[R][C], dy[R][C], res[R][C];
        float mean[R], rstd[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool row = rg + r < a.rows;
            const int64_t m = row ? rg + r : a.rows - 1;
            mean[r] = row ? a.mean[m] : 0.f;
            rstd[r] = row ? a.rstd[m] : 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * TPR + t) * E;
                x[r][c] = load_piece(static_cast<const T*>(a.x) + m * a.ldx, col, a.d);
                dy[r][c] = load_piece(static_cast<const T*>(a.dy) + m * a.lddy, col, a.d);
                if (!row) x[r][c] = dy[r][c] = raw16{0, 0, 0, 0};  // adds nothing to the sums
                if (a.dresidual)
                    res[r][c] = load_piece(static_cast<const T*>(a.dresidual) + m * a.ldr, col, a.d);
            }
        }
        settle_rows<T, TPR, R, C>(x, t, a.d);
        settle_rows<T, TPR, R, C>(dy, t, a.d);
        if (a.dresidual) settle_rows<T, TPR, R, C>(res, t, a.d);
        // sums of q and of q (x - mean), which rstd multiplies as a whole: elements
        // that do not exist have q zero, and mean times rstd need not be a float
        float s[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) s[2 * r] = s[2 * r + 1] = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * E;
            float wf[E];
            if (w) load_vector(w, col, a.d, wf);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float xv[E], dv[E];
                unpack16<T>(x[r][c], xv);
                unpack16<T>(dy[r][c], dv);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float u = xv[e] - mean[r], q = w ? dv[e] * wf[e] : dv[e];
                    s[2 * r] += q;
                    s[2 * r + 1] = fmaf(q, u, s[2 * r + 1]);
                    dw[c][e] = fmaf(dv[e], u * rstd[r], dw[c][e]);
                    db[c][e] += dv[e];
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) s[2 * r + 1] *= rstd[r];
        row_sums<TPR, 2 * R>(s, lds[turn]);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * E, have = (int)a.d - col;
            float wf[E];
            if (w) load_vector(w, col, a.d, wf);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float xv[E], dv[E], v[E];
                unpack16<T>(x[r][c], xv);
                unpack16<T>(dy[r][c], dv);
                if (a.dresidual) unpack16<T>(res[r][c], v);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float h = (xv[e] - mean[r]) * rstd[r], q = w ? dv[e] * wf[e] : dv[e];
                    const float u = rstd[r] * (q - s[2 * r] * inv - h * (s[2 * r + 1] * inv));
                    v[e] = a.dresidual ? v[e] + u : u;
                }
                if (rg + r < a.rows) store16(static_cast<T*>(a.dx) + (rg + r) * a.lddx + col, v, have);
            }
        }
    }
    if (!sums) return;
    float* const out = sums + 2 * blockIdx.x * a.d;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if constexpr (G > 1) {
            // the groups' sums of a column, in order
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    join[g * TPR * EL + (c * TPR + t) * E + e] = k ? db[c][e] : dw[c][e];
            __syncthreads();
            for (int col = threadIdx.x; col < a.d; col += NT) {
                float v = 0.f;
                for (int i = 0; i < G; ++i) v += join[i * TPR * EL + col];
                out[k * a.d + col] = v;
            }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * TPR + t) * E;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (col + e < a.d) out[k * a.d + col + e] = k ? db[c][e] : dw[c][e];
            }
        }
    }
}

// Rows that do not fit the registers: one workgroup per row at a time, which
// reads the row again for each step.
constexpr int WIDE = 1024;
template <typename T>
__global__ __launch_bounds__(WIDE) void norm_wide_kernel(NormArgs a)
{
    __shared__ float lds[2][WIDE / 64];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.ldx;
        T* y = static_cast<T*>(a.y) + r * a.ldy;
        float m[1] = {0.f}, q[1] = {0.f};
        for (int64_t c = threadIdx.x; c < a.d; c += WIDE) m[0] += (float)x[c];
        row_sums<WIDE, 1>(m, lds[0]);
        const float mean = m[0] / (float)a.d;
        for (int64_t c = threadIdx.x; c < a.d; c += WIDE) {
            const float v = (float)x[c] - mean;
            q[0] = fmaf(v, v, q[0]);
        }
        row_sums<WIDE, 1>(q, lds[1]);
        const float rstd = 1.0f / sqrtf(q[0] / (float)a.d + a.eps);
        for (int64_t c = threadIdx.x; c < a.d; c += WIDE) {
            float v = ((float)x[c] - mean) * rstd;
            if (a.weight) v *= (float)static_cast<const T*>(a.weight)[c];
            if (a.bias) v += (float)static_cast<const T*>(a.bias)[c];
            y[c] = (T)v;
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(WIDE) void norm_wide_dx_kernel(NormBackwardArgs a)
{
    __shared__ float lds[2][2 * WIDE / 64];
    const T* w = static_cast<const T*>(a.weight);
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
        const T* x = static_cast<const T*>(a.x) + r * a.ldx;
        const T* dy = static_cast<const T*>(a.dy) + r * a.lddy;
        const T* res = static_cast<const T*>(a.dresidual) + r * a.ldr;
        T* dx = static_cast<T*>(a.dx) + r * a.lddx;
        const float mean = a.mean[r], rstd = a.rstd[r], inv = 1.0f / (float)a.d;
        float s[2] = {0.f, 0.f};
        for (int64_t c = threadIdx.x; c < a.d; c += WIDE) {
            const float q = (float)dy[c] * (w ? (float)w[c] : 1.f);
            s[0] += q;
            s[1] = fmaf(q, ((float)x[c] - mean) * rstd, s[1]);
        }
        row_sums<WIDE, 2>(s, lds[turn]);
        for (int64_t c = threadIdx.x; c < a.d; c += WIDE) {
            const float q = (float)dy[c] * (w ? (float)w[c] : 1.f);
            float v = rstd * (q - s[0] * inv - ((float)x[c] - mean) * rstd * (s[1] * inv));
            if (a.dresidual) v += (float)res[c];
            dx[c] = (T)v;
        }
    }
}

// The weight's and bias's sums of wide rows: workgroup (column block, part).
template <typename T>
__global__ __launch_bounds__(256) void norm_wide_sums_kernel(NormBackwardArgs a, float* sums, int64_t rows_per_part)
{
    const int64_t c = blockIdx.x * 256ll + threadIdx.x;
    if (c >= a.d) return;
    const int64_t r0 = blockIdx.y * rows_per_part, r1 = r0 + rows_per_part < a.rows ? r0 + rows_per_part : a.rows;
    float t0 = 0.f, t1 = 0.f;
    for (int64_t r = r0; r < r1; ++r) {
        const float g = (float)static_cast<const T*>(a.dy)[r * a.lddy + c];
        t0 = fmaf(g, ((float)static_cast<const T*>(a.x)[r * a.ldx + c] - a.mean[r]) * a.rstd[r], t0);
        t1 += g;
    }
    sums[2 * blockIdx.y * a.d + c] = t0;
    sums[(2 * blockIdx.y + 1) * a.d + c] = t1;
}

// Joins the parts [part][2][d] in a fixed order: 64 of the 2 d columns per
// workgroup, every 16th part per wave.
template <typename T>
__global__ __launch_bounds__(1024) void norm_join_kernel(NormBackwardArgs a, const float* sums, int parts)
{
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = workgroup_id() * 64ll + lane;
    float v = 0.f;
    if (c < 2 * a.d) {
#pragma unroll 8
        for (int i = wave; i < parts; i += 16) v += sums[2 * a.d * i + c];
    }
    s[wave][lane] = v;
    __syncthreads();
    if (wave || c >= 2 * a.d) return;
    v = 0.f;
    for (int i = 0; i < 16; ++i) v += s[i][lane];
    if (c < a.d) {
        if (a.dweight) static_cast<T*>(a.dweight)[c] = (T)v;
    } else if (a.dbias) {
        static_cast<T*>(a.dbias)[c - a.d] = (T)v;
    }
}

// Workgroups of the gradient: each writes 2 d sums, so no more than keep the
// memory busy.
struct BackwardGrid {
    template <int TPR, int EL, int R>
    void operator()()
    {
        const int64_t rows_per_pass = wg_threads(TPR) / TPR * R;
        blocks = std::min<int64_t>(ceil_div(rows, rows_per_pass), (int64_t)cus * 2);
    }
    int64_t rows, cus, blocks = 0;
};

int64_t backward_parts(int64_t rows, int64_t d)
{
    if (rows == 0) return 0;
    BackwardGrid g{rows, std::max(device_cus(), 1)};
    if (with_spread<true>(d, g)) return g.blocks;
    return std::max<int64_t>(1, std::min<int64_t>({ceil_div(rows, 16), ceil_div(2048, ceil_div(d, 256)), 512}));
}

template <typename T>
struct Forward {
    const NormArgs& a;
    hipStream_t stream;
    template <int TPR, int EL, int R>
    void operator()()
    {
        // few rows: one each, for every compute unit has one
        const int64_t cus = std::max(device_cus(), 1), groups = wg_threads(TPR) / TPR;
        if (a.rows <= cus * groups * R)
            launch<TPR, EL, 1>();
        else
            launch<TPR, EL, R>();
    }
    template <int TPR, int EL, int R>
    void launch()
    {
        constexpr int per_pass = wg_threads(TPR) / TPR * R;
        const int64_t blocks = std::min<int64_t>(ceil_div(a.rows, per_pass), 1 << 20);
        if (debug_enabled())
            fprintf(stderr, "cliffconv: layer_norm %lld x %lld, %d threads per row, %lld workgroups\n",
                    (long long)a.rows, (long long)a.d, TPR, (long long)blocks);
        hipLaunchKernelGGL((norm_kernel<T, TPR, EL, R>), dim3((unsigned)blocks), dim3(wg_threads(TPR)), 0, stream, a);
    }
};

template <typename T>
struct Backward {
    const NormBackwardArgs& a;
    hipStream_t stream;
    int64_t parts;
    template <int TPR, int EL, int R>
    void operator()()
    {
        if (debug_enabled())
            fprintf(stderr, "cliffconv: layer_norm_backward %lld x %lld, %d threads per row, %lld workgroups\n",
                    (long long)a.rows, (long long)a.d, TPR, (long long)parts);
        float* const sums = a.dweight || a.dbias ? static_cast<float*>(a.workspace) : nullptr;
        hipLaunchKernelGGL((norm_backward_kernel<T, TPR, EL, R>), dim3((unsigned)parts), dim3(wg_threads(TPR)), 0,
                           stream, a, sums);
    }
};

}  // namespace

int64_t layer_norm_backward_workspace(int, int64_t rows, int64_t d)
{
    return ceil_div(8 * d * backward_parts(rows, d), 16) * 16;
}

cliff_status launch_layer_norm(int dtype, const NormArgs& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (!with_spread<false>(a.d, Forward<T>{a, stream}))
            hipLaunchKernelGGL(norm_wide_kernel<T>, dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(WIDE), 0,
                               stream, a);
        return launched();
    });
}

cliff_status launch_layer_norm_backward(int dtype, const NormBackwardArgs& a, hipStream_t stream)
{
    clear_hip_error();
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const bool params = a.dweight || a.dbias;
        const int64_t parts = backward_parts(a.rows, a.d);
        float* const sums = static_cast<float*>(a.workspace);
        if (a.rows && !with_spread<true>(a.d, Backward<T>{a, stream, parts})) {
            // the sums first: dx may be dy
            if (params)
                hipLaunchKernelGGL(norm_wide_sums_kernel<T>, dim3((unsigned)ceil_div(a.d, 256), (unsigned)parts),
                                   dim3(256), 0, stream, a, sums, ceil_div(a.rows, parts));
            hipLaunchKernelGGL(norm_wide_dx_kernel<T>, dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(WIDE),
                               0, stream, a);
        }
        if (params)
            hipLaunchKernelGGL(norm_join_kernel<T>, grid_of(ceil_div(2 * a.d, 64)), dim3(1024), 0, stream, a,
                               sums, (int)parts);
        return launched();
    });
}

}  // namespace cliff
