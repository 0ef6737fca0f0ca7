// What the attention over a cache of values and the one over a cache of 4 bits have in common: a call as its kernels see it, and the join of the parts
// that a cut cache leaves.
#pragma once

#include "gelo_internal.h"
#include "paged.h"

namespace gelo {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x3_t __attribute__((ext_vector_type(3), aligned(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
constexpr float kLog2E = 1.4426950408889634f;

struct AttnArgs {
    const void* Q; int64_t ldq;
    void* O; int64_t ldo;
    float* part_o;               // [chunk][sequence, its row][head][D], where the cache is cut: max_rows places to a sequence
    float* part_ml;              // [chunk][sequence, its row][head][2]: maximum (of log2) and sum
    int n_q_heads, group;        // query heads to a key head
    float scale2;                // |scale| log2 e
    float scale2s;               // scale log2 e
    uint32_t flip;               // sign bits of Q's words where scale is negative
    int causal;
    int chunk, n_chunks, col_tiles, paired, by_head;
    KvCache kv;
    SeqBatch b;
};

__device__ __forceinline__ float across_groups_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float across_groups_sum(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// PAST: cache rows are read past the caches (nobody reads them again soon)
template <class V, bool PAST>
__device__ __forceinline__ V read_row(const void* p) {
    if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
    else return *reinterpret_cast<const V*>(p);
}

// words side by side: 2, 3, 4 or 8
template <int W, bool PAST>
__device__ __forceinline__ void read_words(const uint8_t* p, uint32_t (&w)[W]) {
    if constexpr (W == 2) {
        const u32x2_t x = read_row<u32x2_t, PAST>(p);
        w[0] = x[0]; w[1] = x[1];
    } else if constexpr (W == 3) {
        const u32x3_t x = read_row<u32x3_t, PAST>(p);
        w[0] = x[0]; w[1] = x[1]; w[2] = x[2];
    } else {
#pragma unroll
        for (int i = 0; i < W; i += 4) {
            const u32x4_t x = read_row<u32x4_t, PAST>(p + 4 * i);
#pragma unroll
            for (int u = 0; u < 4; ++u) w[i + u] = x[u];
        }
    }
}

// the place of the part that chunk `chunk` makes of head `head` of a sequence's row i
__device__ __forceinline__ int64_t part_of(const AttnArgs& a, int chunk, int seq, int i, int head) {
    return (((int64_t)chunk * a.b.n_seqs + seq) * a.b.max_rows + i) * a.n_q_heads + head;
}

// What a row's sums are divided by, as a factor.  No weight at all: a row that sees nothing is to give zeros; one that sees only scores of
// -infinity has no softmax.
__device__ __forceinline__ float inverse_of(float total, bool sees) { return total == 0.f ? sees ? __builtin_nanf("") : 0.f : 1.f / total; }

template <class T> __device__ __forceinline__ void store4(T* p, f32x4_t v);
template <> __device__ __forceinline__ void store4<float>(float* p, f32x4_t v) { *reinterpret_cast<f32x4_t*>(p) = v; }
template <> __device__ __forceinline__ void store4<uint16_t>(uint16_t* p, f32x4_t v) {
    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4_t*>(p) = bf16x4_t{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
}

// Joins the chunks' parts of a row's head: O = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.  D / 4 threads (padded to a power of two) take
// a part each P-th chunk's, four components a thread; the P sums are joined in LDS in their order.  With one thread after another through all
// chunks (P = 1) 37 chunks of 96 heads took 31 us: a chain of trips to memory; as it is 4.3.  (Joined by the last workgroup of a tile to end, one launch
// less, 1 x 16384 keys took 23.9 us instead of 18.0, 8 x 2048 15.8 instead of 16.7, with fences between device and memory 52 and 53.)
template <class T, int D, int P>
__global__ __launch_bounds__(256)
void attention_join_kernel(AttnArgs a) {
    constexpr int TH = D == 96 ? 32 : D / 4, ITEMS = 256 / (TH * P);
    __shared__ float ml[P > 1 ? 256 / TH : 1][2];
    __shared__ f32x4_t parts[P > 1 ? 256 : 1];
    const int x = 4 * (threadIdx.x % TH), sub = threadIdx.x / TH, turn = sub % P;
    const int64_t items = (int64_t)a.b.n_rows * a.n_q_heads, item = (int64_t)blockIdx.x * ITEMS + sub / P;
    bool there = item < items && x < D;
    const int row = there ? (int)(item / a.n_q_heads) : 0;
    int used = 0;
    int64_t part0 = 0;                                       // the first chunk's part
    if (there) {
        int seq = row, i = 0, count = 1;
        if (a.b.row_start) {
            int lo = 0, hi = a.b.n_seqs;                     // the number of sequences that end at or before the row
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (a.b.row_start[mid + 1] <= row) lo = mid + 1; else hi = mid;
            }
            seq = lo;
            there = seq < a.b.n_seqs;
            if (there) {
                const NewRows rows = rows_of_sequence(a.b, seq);
                i = row - rows.first;
                count = rows.count;
                there = i >= 0 && i < count;
            }
        }
        if (there) {
            const int kv_len = length_of_sequence(a.b, seq), kv_end = min(kv_len, a.b.max_kv_len);
            const int limit = min(a.causal ? kv_len - count + i : kv_len - 1, kv_end - 1);
            used = limit < 0 ? 0 : limit / a.chunk + 1;
            part0 = part_of(a, 0, seq, i, (int)(item - (int64_t)row * a.n_q_heads));
        }
    }
    float top = -__builtin_inff(), total = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    constexpr int DEEP = 4;                                  // chunks whose parts are sent for together
    const int64_t apart = (int64_t)a.b.n_seqs * a.b.max_rows * a.n_q_heads;      // parts of a chunk
    for (int s0 = turn; s0 < used; s0 += DEEP * P) {
        float2 part[DEEP];
        f32x4_t y[DEEP];
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            const int64_t at = min(s0 + k * P, used - 1) * apart + part0;
            part[k] = *reinterpret_cast<const float2*>(a.part_ml + 2 * at);
            y[k] = *reinterpret_cast<const f32x4_t*>(a.part_o + at * D + x);
        }
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            if (s0 + k * P >= used || part[k].y == 0.f) continue;            // nothing seen: 0 times what it holds need not be 0
            const float m = fmaxf(top, part[k].x), safe = m == -__builtin_inff() ? 0.f : m;
            const float was = __builtin_amdgcn_exp2f(top - safe), is = __builtin_amdgcn_exp2f(part[k].x - safe);
            total = total * was + is * part[k].y;
#pragma unroll
            for (int u = 0; u < 4; ++u) o[u] = o[u] * was + is * y[k][u];
            top = m;
        }
    }
    if constexpr (P > 1) {
        parts[threadIdx.x] = o;
        if (x == 0) { ml[sub][0] = top; ml[sub][1] = total; }
        __syncthreads();
        if (turn != 0) return;
        float m = top;
#pragma unroll
        for (int s = 1; s < P; ++s) m = fmaxf(m, ml[sub + s][0]);
        const float safe = m == -__builtin_inff() ? 0.f : m;
        total = 0.f;
        o = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < P; ++s) {
            if (ml[sub + s][1] == 0.f) continue;
            const float k = __builtin_amdgcn_exp2f(ml[sub + s][0] - safe);
            total += k * ml[sub + s][1];
            const f32x4_t y = parts[threadIdx.x + s * TH];
#pragma unroll
            for (int u = 0; u < 4; ++u) o[u] += k * y[u];
        }
    }
    if (!there) return;
    const float inv = inverse_of(total, used > 0);
#pragma unroll
    for (int u = 0; u < 4; ++u) o[u] *= inv;                 // (nothing was added to o where there was no weight)
    store4((T*)a.O + row * a.ldo + (item - (int64_t)row * a.n_q_heads) * D + x, o);
}

template <class T, int D, int P>
hipError_t join(const AttnArgs& a, hipStream_t stream) {
    constexpr int ITEMS = 256 / ((D == 96 ? 32 : D / 4) * P);
    const int64_t items = (int64_t)a.b.n_rows * a.n_q_heads;
    hipLaunchKernelGGL((attention_join_kernel<T, D, P>), dim3((unsigned)((items + ITEMS - 1) / ITEMS)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

// behind a kernel that left a.n_chunks parts
template <class T, int D>
hipError_t join_parts(const AttnArgs& a, hipStream_t stream) {
    if (a.n_chunks <= 4) return join<T, D, 1>(a, stream);
    return a.n_chunks <= 16 ? join<T, D, 4>(a, stream) : join<T, D, D == 256 ? 4 : 8>(a, stream);
}

// Which kernel, and how the cache is cut: chunks of `chunk` keys, n_chunks of them to the longest sequence.
struct Plan { bool prompt, shared, paired, past, by_head; int chunk, n_chunks; int64_t col_tiles, workgroups; };
constexpr int64_t kMostWorkgroups = kMostThreads / 256;      // all kernels here have workgroups of 256
constexpr int kCus = 256;
constexpr int kFewTarget = 512, kFewLeast = 256;         // workgroups that fill the chip (two to a CU), keys to a chunk at least
constexpr int kPromptTarget = 512, kPromptLeast = 128;

// The cache cut `cuts` times, rounded to whole steps of both kernels.
void cut(Plan* p, int max_kv_len, int64_t cuts) {
    p->chunk = (int)round_up((max_kv_len + cuts - 1) / cuts, 128);
    p->n_chunks = (int)(((int64_t)max_kv_len + p->chunk - 1) / p->chunk);
}
// The join: a launch behind another one, and the parts written and read.
double join_us(const Attention& o, const Plan& p) {
    const double rows = (double)o.batch.n_seqs * o.batch.max_rows;
    return p.n_chunks == 1 ? 0.0 : 5.0 + 8.0 * p.n_chunks * (rows < o.batch.n_rows ? rows : o.batch.n_rows) * o.n_q_heads * o.cache.head_dim / 4e6;
}

}  // namespace
}  // namespace gelo
