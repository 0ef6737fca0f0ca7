// Root-mean-square norm of the rows of h = x + r:  y = h / sqrt(mean h^2 + eps) * gamma, as values of the inputs' type or as
// E4M3 codes with one scale per row (what the 8-bit projection takes).  Bytes bound: every value is read once and written once, the
// row stays in registers between the sum of squares and the scaling.  4096 x 4096 bfloat16 with a residual 20.2 us = 6.6 TB/s, into codes 2048 rows 13.1
// (4.5 TB/s; the largest value of the row is a second exchange between its threads, and a call this short starts and ends unevenly), 64 rows 3.3,
// called from Python 7.5; float 49.8 (5.4 TB/s), into codes 20.4 (5.4), 64 rows from Python 8.6.  Sums are float: 64 values at most in a thread, then
// over threads, so nothing adds up beyond a few units in the last place.
#include "gelo_internal.h"
#include "e4m3.h"

namespace gelo {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

template <class T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        const u32x4_t w = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    } else {
        const f32x4_t a = *reinterpret_cast<const f32x4_t*>(p), b = *reinterpret_cast<const f32x4_t*>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    }
}

// PAST: past the caches, see norm_of_type (not a flag at run time: the compiler makes one plain store of the two)
template <bool PAST, class T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
        bf16x8_t o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[i];
        if constexpr (PAST) __builtin_nontemporal_store(o, reinterpret_cast<bf16x8_t*>(p));
        else *reinterpret_cast<bf16x8_t*>(p) = o;
    } else {
        const f32x4_t lo = {v[0], v[1], v[2], v[3]}, hi = {v[4], v[5], v[6], v[7]};
        if constexpr (PAST) {
            __builtin_nontemporal_store(lo, reinterpret_cast<f32x4_t*>(p));
            __builtin_nontemporal_store(hi, reinterpret_cast<f32x4_t*>(p + 4));
        } else {
            *reinterpret_cast<f32x4_t*>(p) = lo;
            *reinterpret_cast<f32x4_t*>(p + 4) = hi;
        }
    }
}

// the larger of two, NaN if either is
__device__ __forceinline__ float max_or_nan(float a, float b) { return b > a || b != b ? b : a; }

template <bool MAX>
__device__ __forceinline__ float combine(float a, float b) { return MAX ? max_or_nan(a, b) : a + b; }

// Over the TPR threads of a row, in a fixed order: lanes by halving, then the waves in turn.  part: a slot per wave of the workgroup.
template <int TPR, bool MAX>
__device__ __forceinline__ float over_row(float v, float* part) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = combine<MAX>(v, __shfl_xor(v, off, 64));
    if constexpr (TPR > 64) {
        const int wave = threadIdx.x >> 6, first = wave & ~(TPR / 64 - 1);
        if ((threadIdx.x & 63) == 0) part[wave] = v;
        __syncthreads();
        v = part[first];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) v = combine<MAX>(v, part[first + w]);
    }
    return v;
}

template <class T>
struct NormArgs {
    const T* X; int64_t ldx;
    const T* R; int64_t ldr;
    const T* gamma;
    T* R_out; int64_t ldro;
    T* H; int64_t ldh;
    uint8_t* codes; int64_t ldq; float* scales;
    float eps;
    int n, d;
};

// TPR threads to a row, up to VPT vectors of 8 values in each; WG threads in all.
template <class T, int TPR, int VPT, int WG, bool PAST>
__global__ __launch_bounds__(WG)
void rms_norm_kernel(NormArgs<T> a) {
    __shared__ float part[2][WG / 64];
    const int t = threadIdx.x & (TPR - 1);
    const int64_t want = (int64_t)blockIdx.x * (WG / TPR) + threadIdx.x / TPR;
    const bool live = want < a.n;                             // rows of a last workgroup that are not there: computed again, not stored
    const int64_t row = live ? want : a.n - 1;
    const int vecs = a.d >> 3;
    float h[VPT][8];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = t + i * TPR;
        if (v < vecs) load8(a.X + row * a.ldx + 8 * v, h[i]);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) h[i][e] = 0.f;
        }
    }
    if (a.R) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = t + i * TPR;
            if (v >= vecs) continue;
            float r[8];
            load8(a.R + row * a.ldr + 8 * v, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[i][e] += r[e];
        }
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(h[i][e], h[i][e], ss);
    // every thread of the row has read what it stores below before any of them passes a barrier only where TPR > 64; a thread stores
    // nothing but the vectors it has read itself, so outputs in the inputs' memory are safe either way
    ss = over_row<TPR, false>(ss, part[0]);
    const float inv = rsqrtf(ss / (float)a.d + a.eps);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = t + i * TPR;
        if (v >= vecs) continue;
        if (a.R_out && live) store8<true>(a.R_out + row * a.ldro + 8 * v, h[i]);
        float g[8];
        load8(a.gamma + 8 * v, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[i][e] = h[i][e] * inv * g[e];
            top = max_or_nan(top, fabsf(h[i][e]));
        }
        if (a.H && live) store8<PAST>(a.H + row * a.ldh + 8 * v, h[i]);
    }
    if (!a.codes) return;
    top = over_row<TPR, true>(top, part[1]);
    const E4m3Scale scale = e4m3_scale(top);
    if (!live) return;
    if (t == 0) a.scales[row] = scale.back;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = t + i * TPR;
        if (v >= vecs) continue;
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float q = h[i][e] * scale.times;
            w[e >> 2] |= (q != q ? 0x7Fu : e4m3_code(q)) << (8 * (e & 3));
        }
        *reinterpret_cast<u32x2_t*>(a.codes + row * a.ldq + 8 * v) = u32x2_t{w[0], w[1]};
    }
}

template <class T, int TPR, int VPT, int WG = (TPR > 256 ? TPR : 256)>
hipError_t launch(const NormArgs<T>& a, bool past, hipStream_t stream) {
    const int rows = WG / TPR;
    const dim3 grid((a.n + rows - 1) / rows);
    if (past) hipLaunchKernelGGL((rms_norm_kernel<T, TPR, VPT, WG, true>), grid, dim3(WG), 0, stream, a);
    else hipLaunchKernelGGL((rms_norm_kernel<T, TPR, VPT, WG, false>), grid, dim3(WG), 0, stream, a);
    return hipGetLastError();
}

template <class T>
hipError_t norm_of_type(const RmsNorm& o, hipStream_t stream) {
    NormArgs<T> a;
    a.X = (const T*)o.X; a.ldx = o.ldx; a.R = (const T*)o.R; a.ldr = o.ldr; a.gamma = (const T*)o.gamma;
    a.R_out = (T*)o.R_out; a.ldro = o.ldro; a.H = (T*)o.H; a.ldh = o.ldh;
    a.codes = o.codes; a.ldq = o.ldq; a.scales = o.scales; a.eps = o.eps; a.n = o.n; a.d = o.d;
    // The residual is read again a layer later, so it always passes the caches by: with codes 2048 x 4096 bf16 take 13.6 us instead of 15.0, 4096
    // rows 22.3 (5.3 TB/s) instead of 29.2, the 8-bit product behind them 62.7 and 85.0 together instead of 63.4 and 89.8.  H, which the next kernel
    // reads, goes the same way where both are more than the L2s hold and push the inputs out of them: 4096 x 4096 20.2 us (6.6 TB/s)
    // instead of 26.7, with a kernel behind that reads H 39 instead of 42; at 2048 rows that reader takes 18.8 and 17.1.
    const bool past = ((o.H ? 1.0 : 0.0) + (o.R_out ? 1.0 : 0.0)) * o.n * o.d * sizeof(T) > 40e6;
    const int vecs = o.d / 8;
    if (vecs <= 64) return launch<T, 64, 1>(a, past, stream);
    if (vecs <= 256) return launch<T, 256, 1>(a, past, stream);
    // (4096 x 4096: 512 threads to a row 20.1 and 26.7 us, 256 21.4 and 28.7; with codes, 2048 rows, 15.0 and 14.6)
    if (vecs <= 512 && !o.codes) return launch<T, 512, 1>(a, past, stream);
    if (vecs <= 512) return launch<T, 256, 2>(a, past, stream);
    if (vecs <= 1024) return launch<T, 256, 4>(a, past, stream);
    if (vecs <= 2048) return launch<T, 1024, 2>(a, past, stream);
    return launch<T, 1024, 8>(a, past, stream);
}

}  // namespace

// Rows of one launch: a row of more than 8192 values has a workgroup of 1024 threads, the others at most 512 threads.
int rms_norm_most_rows(int d) { return (int)(kMostThreads / (d > 8192 ? 1024 : 512)); }

hipError_t rms_norm(const RmsNorm& o, int is_bf16, hipStream_t stream) {
    return is_bf16 ? norm_of_type<uint16_t>(o, stream) : norm_of_type<float>(o, stream);
}

}  // namespace gelo
