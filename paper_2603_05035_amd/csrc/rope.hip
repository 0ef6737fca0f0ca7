// Rotary positions on the way into the paged cache: rows of a fused Q|K|V turn their query and key heads by the row's position; the
// queries go to a matrix, keys and values to the row's place in the cache.  Bytes bound: every value is read once and written once.
// A pair (a, b) of components i becomes (a cos - b sin, b cos + a sin), in float, rounded once; angles are worked out in double when the table is
// filled, since a float of position times frequency would be off by 0.004 at position 65536.  8 prompts of 301 to 512 rows, 32/8 heads of 128,
// bfloat16: 14.1 to 15.9 us = 4.9 to 5.5 TB/s, float 32.9 (4.7; an elementwise kernel over 1 GiB reads and writes at 6.2); one row of each of 64 sequences
// 4.8, called from Python 6.3, float 7.8.
// Stores past the caches: 8 x 512 rows of 32/32 heads 37.8 us instead of 42.8, but with the attention behind them 88.5 instead of 83.8.
#include "gelo_internal.h"
#include "paged.h"

namespace gelo {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

__global__ __launch_bounds__(256)
void rope_table_kernel(RopeTable o) {
    const int half = o.rot / 2;
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= (int64_t)o.count * half) return;
    const int p = (int)(e / half), i = (int)(e - (int64_t)p * half);
    double w = pow(o.base, -2.0 * i / o.rot);
    double keep = 0.0;                                       // the part of the frequency that is not stretched
    if (o.trained > 0.0) {
        keep = (o.trained * w * 0.15915494309189535 - o.low) / (o.high - o.low);       // turns over the trained length: trained w / (2 pi)
        keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
    }
    w *= keep + (1.0 - keep) / o.factor;
    double s, c;
    sincos((o.first + (double)p) * w, &s, &c);
    o.out[2 * e] = (float)c;
    o.out[2 * e + 1] = (float)s;
}

// 8 values of a head
template <class T> struct Eight;
template <> struct Eight<uint16_t> {
    u32x4_t w;
    __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const u32x4_t*>(p); }
    __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<u32x4_t*>(p) = w; }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
        bf16x8_t o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[i];
        w = __builtin_bit_cast(u32x4_t, o);
    }
};
template <> struct Eight<float> {
    f32x4_t a, b;
    __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const f32x4_t*>(p); b = *reinterpret_cast<const f32x4_t*>(p + 4); }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<f32x4_t*>(p) = a; *reinterpret_cast<f32x4_t*>(p + 4) = b; }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    }
    __device__ __forceinline__ void set(const float (&v)[8]) { a = f32x4_t{v[0], v[1], v[2], v[3]}; b = f32x4_t{v[4], v[5], v[6], v[7]}; }
};

// A workgroup takes a row of QKV.  Its work is cut into items of 8 values, or of 8 + 8 where components rot / 2 apart turn together: a
// head that turns has `per_turned` items, rot / 16 such pairs and then the components behind rot; a value head has d / 8.
template <class T>
__global__ __launch_bounds__(256)
void rope_append_kernel(RopeAppend o) {
    const SeqBatch& b = o.batch;
    const KvCache& kv = o.cache;
    const int row = blockIdx.x;
    int seq = row, count = 1, j = 0;
    if (b.row_start) {
        if (row < b.row_start[0]) return;
        seq = sequence_of_row(b.row_start, b.n_seqs, row);
        if (seq >= b.n_seqs) return;                         // a row of no sequence is left alone
        j = row - b.row_start[seq];
        count = b.row_start[seq + 1] - b.row_start[seq];
    }
    const int pos = length_of_sequence(b, seq) - count + j;
    const bool beyond = pos >= b.max_kv_len, placed = pos >= 0 && !beyond;
    const int page = placed ? b.page_table[seq * b.table_ld + (pos >> kv.page_shift)] : -1;
    const bool kept = page >= 0 && page < kv.n_pages;
    const int64_t at = kept ? page * kv.page_stride + (pos & ((1 << kv.page_shift) - 1)) * kv.row_stride : 0;
    const float* angles = o.table + (int64_t)(placed ? pos : 0) * o.rot;

    const int d = kv.head_dim, hq = o.n_q_heads, hkv = kv.n_kv_heads;
    const int turning = o.pairs ? o.rot / 8 : o.rot / 16;    // items of a head that turn
    const int per_turned = turning + (d - o.rot) / 8, turned = (hq + hkv) * per_turned;
    const int items = turned + hkv * (d / 8);
    const T* in = (const T*)o.QKV + (int64_t)row * o.ld;
    for (int e = threadIdx.x; e < items; e += 256) {
        const bool is_value = e >= turned;
        const int per = is_value ? d / 8 : per_turned, e1 = is_value ? e - turned : e;
        const int head = e1 / per, i = e1 - head * per;
        const bool turns = !is_value && i < turning;
        const int col = turns || is_value || o.pairs ? 8 * i : o.rot + 8 * (i - turning);        // first component
        const int from = is_value ? hq + hkv + head : head;                                       // head in the row
        Eight<T> x, y;
        x.load(in + (int64_t)from * d + col);
        const bool two = turns && !o.pairs;
        if (two) y.load(in + (int64_t)from * d + col + o.rot / 2);
        if (turns) {
            float v[8], cs[16];
            x.get(v);
            const int at_angle = two ? 2 * col : col;          // float of the table's row
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (!two && t >= 2) break;
                const f32x4_t c = *reinterpret_cast<const f32x4_t*>(angles + at_angle + 4 * t);
#pragma unroll
                for (int u = 0; u < 4; ++u) cs[4 * t + u] = c[u];
            }
            if (two) {
                float w[8], p[8], q[8];
                y.get(w);
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    p[t] = v[t] * cs[2 * t] - w[t] * cs[2 * t + 1];
                    q[t] = w[t] * cs[2 * t] + v[t] * cs[2 * t + 1];
                }
                x.set(p);
                y.set(q);
            } else {
                float p[8];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    p[2 * t] = v[2 * t] * cs[2 * t] - v[2 * t + 1] * cs[2 * t + 1];
                    p[2 * t + 1] = v[2 * t + 1] * cs[2 * t] + v[2 * t] * cs[2 * t + 1];
                }
                x.set(p);
            }
        }
        T* out;
        if (!is_value && head < hq) {
            out = (T*)o.Q + (int64_t)row * o.ldq + (int64_t)head * d + col;
            if (!placed) {
                float v[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) v[t] = beyond ? __builtin_nanf("") : 0.f;
                x.set(v);
                y = x;
            }
        } else {
            if (!kept) continue;
            const int h = is_value ? head : head - hq;
            out = (T*)(is_value ? kv.v : kv.k) + at + h * kv.head_stride + col;
        }
        x.store(out);
        if (two) y.store(out + o.rot / 2);
    }
}

}  // namespace

hipError_t rope_table(const RopeTable& o, hipStream_t stream) {
    const int64_t n = (int64_t)o.count * (o.rot / 2);
    hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, o);
    return hipGetLastError();
}

hipError_t rope_append(const RopeAppend& o, int is_bf16, hipStream_t stream) {
    if (is_bf16) hipLaunchKernelGGL(rope_append_kernel<uint16_t>, dim3(o.batch.n_rows), dim3(256), 0, stream, o);
    else hipLaunchKernelGGL(rope_append_kernel<float>, dim3(o.batch.n_rows), dim3(256), 0, stream, o);
    return hipGetLastError();
}

}  // namespace gelo
