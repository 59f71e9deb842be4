// Categorical likelihood of rows of logits and its gradient.
//
// Row i: l = lse - z_t, lse = m + log sum exp(z_j - m); dz_j = scale
// (exp(z_j - lse) - [j = t]).  One read of the logits and one write of the
// gradient: a row stays in the registers of the threads that share it, 16 bytes
// at a time, from the maximum and the sum to the gradient.  A thread's own
// maximum and sum come first, the pairs are then joined over the threads in a
// fixed order.  Rows that do not fit are read twice.
//
// Bound by memory: 8192 rows of 128,000 bf16 classes with gradient 773 us (4.1 GB: 5.3
// TB/s; a large copy 4.8).  16 rows of 32,003 fp32 without gradient, as one workgroup
// each on 16 units, 7 us: latency.
//
// An exponential is off by |z - m| 2^-24 of itself, its argument's rounding: with x =
// m - z, x e^-x 2^-24 of the row's largest, less than the sum's own rounding.  Taking
// that back in would cost the case above 1005 us, and 16 rows 9.4.
#include "token.h"
#include "token_device.h"

namespace nuts {
namespace token {
namespace {

struct Pair {
    float m, s;  // maximum, and the sum of exp(z - m); m = -infinity: nothing
};

__device__ __forceinline__ float finite_max(float m) { return m == -__builtin_inff() ? 0.0f : m; }

__device__ __forceinline__ Pair join(Pair a, Pair b)
{
    const float m = fmaxf(a.m, b.m), safe = finite_max(m);
    return {m, a.s * __expf(a.m - safe) + b.s * __expf(b.m - safe)};
}

// A thread's pair with W more values.
template <int W>
__device__ __forceinline__ Pair more(Pair a, const float (&v)[W])
{
    float m = a.m;
#pragma unroll
    for (int i = 0; i < W; ++i) m = fmaxf(m, v[i]);
    const float safe = finite_max(m);
    float s = a.s * __expf(a.m - safe);
#pragma unroll
    for (int i = 0; i < W; ++i) s += __expf(v[i] - safe);
    return {m, s};
}

// TPR threads a row; PER pieces of it in a thread's registers (0: two reads).
// The elements past the last whole piece lie one each in the first threads.
template <typename T, int TPR, int PER>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void categorical_kernel(nuts_categorical_args a)
{
    constexpr int kThreads = TPR < 256 ? 256 : TPR;
    constexpr int E = 16 / sizeof(T);
    constexpr int kWaves = TPR < 64 ? 1 : TPR / 64;
    __shared__ Pair shared[kWaves];
    const int t = threadIdx.x % TPR;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t i = block * (kThreads / TPR) + threadIdx.x / TPR;
    if (i >= a.M) return;  // (with several waves a row, a workgroup has one row)
    const int64_t target = a.targets[i];
    const T* in = (const T*)a.logits + i * a.ld_logits;
    T* out = a.dlogits ? (T*)a.dlogits + i * a.ld_dlogits : nullptr;
    const bool there = target >= 0 && target < a.V;
    const int pieces = (int)(a.V / E), rest = (int)(a.V % E);

    v4u raw[PER ? PER : 1];
    Pair p = {-__builtin_inff(), 0.0f};
    float zt = 0.0f, tail = -__builtin_inff();
    if (there) {
        if constexpr (PER > 0) {
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (k * TPR + t < pieces) raw[k] = load16(in + (int64_t)k * (TPR * E) + t * E);
        }
        if (t < rest) tail = to_f32(in[(int64_t)pieces * E + t]);
        zt = to_f32(in[target]);
        // (piece by piece, as they arrive)
        float v[E];
        if constexpr (PER > 0) {
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                if (k * TPR + t < pieces) {
                    unpack<T>(raw[k], v);
                    p = more<E>(p, v);
                }
            }
        } else {
            for (int at = t; at < pieces; at += TPR) {
                unpack<T>(load16(in + (int64_t)at * E), v);
                p = more<E>(p, v);
            }
        }
        const float last[1] = {tail};
        p = more<1>(p, last);
#pragma unroll
        for (int o = TPR < 64 ? TPR / 2 : 32; o > 0; o /= 2) {
            const Pair q = {__shfl_xor(p.m, o), __shfl_xor(p.s, o)};
            p = (t & o) ? join(q, p) : join(p, q);
        }
        if constexpr (kWaves > 1) {
            if ((t & 63) == 0) shared[t / 64] = p;
            __syncthreads();
            p = shared[0];
            for (int w = 1; w < kWaves; ++w) p = join(p, shared[w]);
        }
    }
    // no class left: the logarithm of an empty sum
    const bool empty = p.m == -__builtin_inff() && p.s == 0.0f;
    const float logs = __logf(p.s);
    if (t == 0) {
        float l = (p.m - zt) + logs;
        if (empty || (zt == -__builtin_inff() && p.m + logs < __builtin_inff())) l = __builtin_inff();
        a.nll[i] = there ? l : 0.0f;
    }
    if (!out) return;
    const bool live = there && !empty;
    const float scale = (float)a.scale, factor = scale / p.s, safe = finite_max(p.m);
    const int64_t hit = live ? target : -1;
    auto write = [&](int at, v4u r) {
        v4u o = {0, 0, 0, 0};
        if (live) {
            float v[E];
            unpack<T>(r, v);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = __expf(v[e] - safe) * factor;
            if (at == (int)(hit / E)) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e == (int)(hit % E)) v[e] -= scale;
            }
            o = pack<T>(v);
        }
        store16(out + (int64_t)at * E, o);
    };
    if constexpr (PER > 0) {
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (k * TPR + t < pieces) write(k * TPR + t, raw[k]);
    } else {
        for (int at = t; at < pieces; at += TPR) {
            v4u r = {0, 0, 0, 0};
            if (live) r = load16(in + (int64_t)at * E);
            write(at, r);
        }
    }
    if (t < rest) {
        const int64_t c = (int64_t)pieces * E + t;
        float g = live ? __expf(tail - safe) * factor : 0.0f;
        if (c == hit) g -= scale;
        out[c] = from_f32<T>(g);
    }
}

// The sum of the rows' likelihoods, in 64 bits and one order: one workgroup, 8192 rows
// 6 us.
__global__ __launch_bounds__(1024) void total_kernel(const float* nll, int64_t M, double* total)
{
    __shared__ double part[16];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < M; i += 1024) s += (double)nll[i];
#pragma unroll
    for (int o = 32; o > 0; o /= 2) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) s += part[w];
        *total = s;
    }
}

// Threads of a row and their pieces: the fewest threads whose registers hold the
// row, so that a thread has several loads in flight and the joining of its pair
// with the others' costs least.  fp32, 300 MB of logits, with gradient (us; in
// parentheses the neighbour): V = 120 16 x 2 316 (64 x 1: 485), 256 32 x 2 194 (64 x
// 1: 238), 1024 64 x 4 133 (256 x 1: 176), 4000 256 x 4 116 (1024 x 1: 225), 8000 256 x
// 16 119 (1024 x 2: 136; 256 x 8 spills: 210), 16,000 1024 x 8 109 (256 x 16: 120),
// 64,000 1024 x 16 129 (two reads: 163).  bf16 is within 10% of these.
template <typename T>
hipError_t launch(const nuts_categorical_args& a, hipStream_t stream)
{
    constexpr int64_t E = 16 / sizeof(T);
    const int64_t pieces = a.V / E;
    // (past one row of the grid the rows go on in the next)
    auto go = [&](auto* kernel, int tpr) {
        const int threads = tpr < 256 ? 256 : tpr;
        const int64_t blocks = (a.M * tpr + threads - 1) / threads;
        const unsigned row = groups_of(blocks, threads);
        kernel<<<dim3(row, (unsigned)((blocks + row - 1) / row)), threads, 0, stream>>>(a);
    };
    if (pieces <= 32) go(categorical_kernel<T, 16, 2>, 16);
    else if (pieces <= 64) go(categorical_kernel<T, 32, 2>, 32);
    else if (pieces <= 256) go(categorical_kernel<T, 64, 4>, 64);
    else if (pieces <= 1024) go(categorical_kernel<T, 256, 4>, 256);
    else if (pieces <= 2048) go(categorical_kernel<T, 256, 16>, 256);
    else if (pieces <= 8192) go(categorical_kernel<T, 1024, 8>, 1024);
    else if (pieces <= 16384) go(categorical_kernel<T, 1024, 16>, 1024);
    else go(categorical_kernel<T, 1024, 0>, 1024);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_categorical(const nuts_categorical_args& a, hipStream_t stream)
{
    if (a.M > 0) {
        const hipError_t e = a.dtype == NUTS_BF16 ? launch<__bf16>(a, stream) : launch<float>(a, stream);
        if (e != hipSuccess) return e;
    }
    if (a.total) {
        total_kernel<<<1, 1024, 0, stream>>>(a.nll, a.M, a.total);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace token
}  // namespace nuts
