// HIP's device language on the CPU, as far as the feed-forward kernels use it
// (test infrastructure; see main.cpp).  Stands in place of hip/hip_runtime.h.
//
// A workgroup's threads are fibers of one OS thread.  What the lanes of a wave do
// together (matrix instructions, lane moves, transposing LDS reads) is a meeting of
// its 64 fibers, a barrier one of the workgroup's; a meeting that some fibers never
// come to ends the program.  A wave barrier is a meeting too: lanes of a wave see
// each other's LDS writes there and nowhere earlier.
#pragma once

#include <math.h>
#include <stddef.h>
#include <stdint.h>
#include <string.h>

#include <functional>

#define __global__
#define __device__
#define __host__
#define __shared__ thread_local
#define __align__(n) __attribute__((aligned(n)))
#define __launch_bounds__(...)

typedef void* hipStream_t;
typedef int hipError_t;
constexpr hipError_t hipSuccess = 0;

struct dim3 {
    unsigned x, y, z;
    dim3(unsigned x_ = 1, unsigned y_ = 1, unsigned z_ = 1) : x(x_), y(y_), z(z_) {}
};
extern dim3 threadIdx, blockIdx, blockDim, gridDim;

namespace emulate {

extern hipError_t last_error;

// Runs a launch to its end; refuses one that a GPU would refuse.
void launch(dim3 grid, dim3 block, size_t lds, const std::function<void()>& kernel);

// The dynamic LDS of a translation unit: its array, and its size.
struct DynamicLds {
    DynamicLds(void* at, size_t bytes);
};

constexpr int WAVE = 64;
int lane_id();

// 16 bytes (nullptr: zeros) to LDS, and the wait for a thread's loads.
void load(const char* from, char* to);
void wait_loads();

// A meeting of the wave: `in` of every lane goes to f(ins, outs), once.
typedef void (*Meet)(const void* ins, void* outs);
void meet(int kind, const void* in, size_t in_size, void* out, size_t out_size, Meet f);
void meet_workgroup();

template <int KIND, typename In, typename Out, void F(const In*, Out*)>
Out together(const In& in)
{
    Out out;
    meet(KIND, &in, sizeof in, &out, sizeof out,
         [](const void* ins, void* outs) { F(static_cast<const In*>(ins), static_cast<Out*>(outs)); });
    return out;
}

enum Kind { BARRIER = 1, FIRST, BALLOT, DPP, SWAP, MFMA, TR16 };

struct Nothing {
    char c;
};
inline void nothing(const Nothing*, Nothing*) {}
inline void wave_barrier() { together<BARRIER, Nothing, Nothing, nothing>(Nothing{}); }

inline void first(const int* in, int* out)
{
    for (int l = 0; l < WAVE; ++l) out[l] = in[0];
}
inline int readfirstlane(int v) { return together<FIRST, int, int, first>(v); }

inline void ballot_of(const int* in, uint64_t* out)
{
    uint64_t m = 0;
    for (int l = 0; l < WAVE; ++l) m |= (uint64_t)(in[l] != 0) << l;
    for (int l = 0; l < WAVE; ++l) out[l] = m;
}
inline uint64_t ballot(int v) { return together<BALLOT, int, uint64_t, ballot_of>(v); }

template <int CTRL>
void dpp_of(const int* in, int* out)
{
    static_assert(CTRL < 0x100 || CTRL == 0x140 || CTRL == 0x141, "control");
    for (int l = 0; l < WAVE; ++l)
        out[l] = CTRL < 0x100 ? in[(l & ~3) | (CTRL >> 2 * (l & 3) & 3)]  // of four lanes
               : CTRL == 0x140 ? in[l ^ 15] : in[l ^ 7];                    // mirrored
}
template <int CTRL>
int dpp(int v)
{
    return together<DPP, int, int, dpp_of<CTRL>>(v);
}

// Rows of N lanes: the odd ones of the first operand and the even ones of the
// second change places.
struct Two {
    uint32_t v[2];
    uint32_t operator[](int i) const { return v[i]; }
};
template <int N>
void swap_of(const Two* in, Two* out)
{
    for (int l = 0; l < WAVE; ++l)
        out[l] = l & N ? Two{{in[l ^ N].v[1], in[l].v[1]}} : Two{{in[l].v[0], in[l ^ N].v[0]}};
}
template <int N>
Two swap_rows(uint32_t a, uint32_t b)
{
    return together<SWAP, Two, Two, swap_of<N>>(Two{{a, b}});
}

// Matrix instructions: D (S x S) = A B + C with K contraction values, E of them
// per lane.  Lane l has A's row and B's column l % S, values E (l / S) on, and of D
// column l % S, rows 8 (e / 4) + 4 (l / S) + e % 4.
template <int S, int E, typename V, typename Acc>
struct Product {
    struct In {
        V a, b;
        Acc c;
    };
    static void f(const In* in, Acc* out)
    {
        constexpr int K = E * WAVE / S, R = S * S / WAVE;
        float a[S][K], b[K][S];
        for (int l = 0; l < WAVE; ++l)
            for (int e = 0; e < E; ++e) {
                a[l % S][E * (l / S) + e] = element(in[l].a, e);
                b[E * (l / S) + e][l % S] = element(in[l].b, e);
            }
        for (int i = 0; i < S; ++i) {
            float d[S];
            // the accumulator that holds row i: register and half of the lanes
            const int e = S == 32 ? i / 8 * 4 + i % 4 : i % 4, h = S == 32 ? i / 4 % 2 : i / 4;
            for (int j = 0; j < S; ++j) d[j] = in[S * h + j].c[e];
            for (int k = 0; k < K; ++k)
                for (int j = 0; j < S; ++j) d[j] += a[i][k] * b[k][j];
            for (int j = 0; j < S; ++j) out[S * h + j][e] = d[j];
        }
        static_assert(R == 16 || R == 4, "accumulators");
    }
    static float element(float v, int) { return v; }
    template <typename U>
    static float element(const U& v, int e)
    {
        return (float)v[e];
    }
};
template <int S, int E, typename V, typename Acc>
Acc mfma(const V& a, const V& b, const Acc& c)
{
    typedef Product<S, E, V, Acc> P;
    return together<MFMA, typename P::In, Acc, P::f>(typename P::In{a, b, c});
}

// Of 16 lanes, lane t gets as its i-th value element t % 4 of what lane 4 i + t / 4
// points to.
typedef short short4_t __attribute__((ext_vector_type(4)));
inline void tr16_of(const short4_t* in, short4_t* out)
{
    for (int l = 0; l < WAVE; ++l)
        for (int i = 0; i < 4; ++i) out[l][i] = in[(l & 48) + 4 * i + (l & 15) / 4][l & 3];
}
template <typename P>
short4_t read_tr16(const P* from)
{
    short4_t v;
    memcpy(&v, (const void*)from, sizeof v);
    return together<TR16, short4_t, short4_t, tr16_of>(v);
}

}  // namespace emulate

inline hipError_t hipGetLastError()
{
    const hipError_t e = emulate::last_error;
    emulate::last_error = hipSuccess;
    return e;
}
#define hipLaunchKernelGGL(k, grid, block, lds, stream, ...)                     \
    do {                                                                         \
        (void)(stream);                                                          \
        const auto kernel_ = k;                                                  \
        emulate::launch(grid, block, lds, [=] { kernel_(__VA_ARGS__); });        \
    } while (0)

#define __syncthreads emulate::meet_workgroup
#define __ballot emulate::ballot
#define __expf expf
#define __builtin_amdgcn_exp2f exp2f
#define __builtin_amdgcn_rcpf(v) (1.0f / (v))
#define __builtin_amdgcn_readfirstlane emulate::readfirstlane
#define __builtin_amdgcn_wave_barrier emulate::wave_barrier
#define __builtin_amdgcn_fence(order, scope) ((void)0)
#define __builtin_amdgcn_s_waitcnt(n) ((void)0)
#define __builtin_amdgcn_sched_barrier(n) ((void)0)
#define __builtin_amdgcn_sched_group_barrier(a, b, c) ((void)0)
#define __builtin_amdgcn_update_dpp(old, v, ctrl, rows, banks, bound) emulate::dpp<ctrl>(v)
#define __builtin_amdgcn_permlane16_swap(a, b, x, y) emulate::swap_rows<16>(a, b)
#define __builtin_amdgcn_permlane32_swap(a, b, x, y) emulate::swap_rows<32>(a, b)
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16 emulate::read_tr16
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) emulate::mfma<32, 8>(a, b, c)
#define __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, x, y, z) emulate::mfma<32, 8>(a, b, c)
#define __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, x, y, z) emulate::mfma<32, 1>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) emulate::mfma<16, 8>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) emulate::mfma<16, 8>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, x, y, z) emulate::mfma<16, 1>(a, b, c)
