// Rotary positions on the way into the paged cache: rows of a fused Q|K|V turn their query and key heads by the row's position; the
// queries go to a matrix, keys and values to the row's place in the cache.  Bytes bound: every value is read once and written once.
// A pair (a, b) of components i becomes (a cos - b sin, b cos + a sin), in float, rounded once; angles are worked out in double when the table is
// filled, since a float of position times frequency would be off by 0.004 at position 65536.  8 prompts of 301 to 512 rows, 32/8 heads of 128,
// bfloat16: 14.1 to 15.9 us = 4.9 to 5.5 TB/s, float 32.9 (4.7; an elementwise kernel over 1 GiB reads and writes at 6.2); one row of each of 64 sequences
// 4.8, called from Python 6.3, float 7.8.
// Stores past the caches: 8 x 512 rows of 32/32 heads 37.8 us instead of 42.8, but with the attention behind them 88.5 instead of 83.8.
#include "fp4.h"
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

// Where a row of the batch lies in a cache of 4 bits, and whether it does.
struct Fp4Row {
    int pos, page, in_page;
    bool beyond, placed, kept;
};
__device__ __forceinline__ bool find_row(const SeqBatch& b, const KvCache& kv, int row, Fp4Row* at) {
    int seq = row, count = 1, j = 0;
    if (b.row_start) {
        if (row < b.row_start[0]) return false;
        seq = sequence_of_row(b.row_start, b.n_seqs, row);
        if (seq >= b.n_seqs) return false;                   // a row of no sequence is left alone
        j = row - b.row_start[seq];
        count = b.row_start[seq + 1] - b.row_start[seq];
    }
    at->pos = length_of_sequence(b, seq) - count + j;
    at->beyond = at->pos >= b.max_kv_len;
    at->placed = at->pos >= 0 && !at->beyond;
    at->page = at->placed ? b.page_table[seq * b.table_ld + (at->pos >> kv.page_shift)] : -1;
    at->kept = at->page >= 0 && at->page < kv.n_pages;
    at->in_page = at->pos & ((1 << kv.page_shift) - 1);
    return true;
}
// The row of a wave where a workgroup of 256 has 2^log rows
__device__ __forceinline__ int row_of_thread(int log) { return (blockIdx.x << log) + __builtin_amdgcn_readfirstlane(threadIdx.x >> (8 - log)); }
// Bytes from the start of a head's piece: of four bytes of codes, 8 values, from byte `byte` of the row on where they lie side by side, and of a block's scale.
__device__ __forceinline__ int key_codes_at(int d, int in_page, int byte) { return in_page * (d / 2) + byte; }
__device__ __forceinline__ int value_codes_at(int d, int in_page, int byte) {
    const int unit = d / 32, piece = byte / unit;
    return (in_page >> 2) * 2 * d + (4 * piece + (in_page & 3)) * unit + byte - piece * unit;
}
__device__ __forceinline__ int scale_at(int d, int page_shift, int in_page, int block, bool is_value) {
    const int first = fp4_scales_at(d, page_shift), per = d / 32;
    return is_value ? first + (in_page >> 2) * 4 * per + 4 * block + (in_page & 3) : first + in_page * per + block;
}

// A workgroup takes a row of QKV, or a share of its items (grid y), or a few rows.  Bound by the trips before a row's first store, one behind the other - sequence, length, page, angles:
// 3126 rows of 32/8 heads of 128 17.8 us, 67 MB at 3.8 TB/s; 64 rows of 32/32 4.1.  Where nothing turns the 3126 take 15.0 us, in pairs 16.6, in halves 16.8 to 17.7 (a call after the other).  Keys and values go by items of 8 components, four lanes to a block: each of them loads the components that its own turn
// with, too, so that any rot / 2 will do.  A turned key is worked out in double, where the two products are exact and their sum as good as, and its code is
// that value's: in float one in some millions would fall on the other side of the middle between two codes.  Queries turn as in rope_append_kernel, to the bit.
template <class T>
__global__ __launch_bounds__(256)
void rope_append_fp4_kernel(RopeAppend o, int rows_log) {
    const SeqBatch& b = o.batch;
    const KvCache& kv = o.cache;
    const int threads = 256 >> rows_log, thread = threadIdx.x & (threads - 1), row = row_of_thread(rows_log);
    if (row >= b.n_rows) return;
    Fp4Row at;
    if (!find_row(b, kv, row, &at)) return;
    const float* angles = o.table + (int64_t)(at.placed ? at.pos : 0) * o.rot;
    const int d = kv.head_dim, hq = o.n_q_heads, hkv = kv.n_kv_heads, per_head = d / 8;
    const T* in = (const T*)o.QKV + (int64_t)row * o.ld;
    const int held = 2 * hkv * per_head;                     // items of keys and values: a multiple of 4
    const int turning = o.pairs ? o.rot / 8 : o.rot / 16, per_turned = turning + (d - o.rot) / 8;
    for (int e = blockIdx.y * threads + thread; e < held + hq * per_turned; e += threads * gridDim.y) {
        if (e >= held) {
            const int head = (e - held) / per_turned, i = e - held - head * per_turned;
            const bool turns = i < turning, two = turns && !o.pairs;
            const int col = turns || o.pairs ? 8 * i : o.rot + 8 * (i - turning);
            Eight<T> x, y;
            x.load(in + (int64_t)head * d + col);
            if (two) y.load(in + (int64_t)head * d + col + o.rot / 2);
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
            if (!at.placed) {
                float v[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) v[t] = at.beyond ? __builtin_nanf("") : 0.f;
                x.set(v);
                y = x;
            }
            T* out = (T*)o.Q + (int64_t)row * o.ldq + (int64_t)head * d + col;
            x.store(out);
            if (two) y.store(out + o.rot / 2);
            continue;
        }
        if (!at.kept) continue;
        const int head2 = e / per_head, i = e - head2 * per_head, col = 8 * i;
        const bool is_value = head2 >= hkv;
        const int head = is_value ? head2 - hkv : head2;
        const T* from = in + (int64_t)(hq + head2) * d;
        Eight<T> x;
        x.load(from + col);
        float v[8];
        x.get(v);
        bool finite = true;
#pragma unroll
        for (int t = 0; t < 8; ++t) finite &= fabsf(v[t]) < __builtin_inff();
        if (!is_value && col < o.rot) {
            const int half = o.rot / 2;
            const bool upper = !o.pairs && col >= half;
            float w[8], cs[16];
            if (!o.pairs) {
                Eight<T> y;
                y.load(from + (upper ? col - half : col + half));
                y.get(w);
            }
            const float* c = angles + (o.pairs ? col : 2 * (upper ? col - half : col));
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (o.pairs && t >= 2) break;
                const f32x4_t z = *reinterpret_cast<const f32x4_t*>(c + 4 * t);
#pragma unroll
                for (int u = 0; u < 4; ++u) cs[4 * t + u] = z[u];
            }
            double p[8];
            if (o.pairs) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const double c0 = cs[2 * t], s0 = cs[2 * t + 1], a0 = v[2 * t], b0 = v[2 * t + 1];
                    p[2 * t] = a0 * c0 - b0 * s0;
                    p[2 * t + 1] = b0 * c0 + a0 * s0;
                }
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const double c0 = cs[2 * t], s0 = upper ? cs[2 * t + 1] : -cs[2 * t + 1];
                    p[t] = v[t] * c0 + w[t] * s0;
                }
            }
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                finite &= fabs(p[t]) < (double)__builtin_inff();
                v[t] = odd_float(p[t]);
            }
        }
        float top = 0.f;
#pragma unroll
        for (int t = 0; t < 8; ++t) top = fmaxf(top, fabsf(v[t]));
        top = finite ? top : __builtin_nanf("");
        // the block's: of four lanes; a NaN stays (fmaxf would drop it)
#pragma unroll
        for (int by = 1; by < 4; by *= 2) {
            const float other = __shfl_xor(top, by, 64);
            top = top != top || other != other ? __builtin_nanf("") : fmaxf(top, other);
        }
        const uint32_t byte = top != top ? 255u : fp4_scale_byte(top);
        const uint32_t codes = top != top ? 0u : fp4_codes(v, fp4_scale(byte));
        uint8_t* piece = (uint8_t*)(is_value ? kv.v : kv.k) + at.page * kv.page_stride + head * kv.head_stride;
        if (!is_value || d % 128 == 0) {
            *reinterpret_cast<uint32_t*>(piece + (is_value ? value_codes_at(d, at.in_page, 4 * i) : key_codes_at(d, at.in_page, 4 * i))) = codes;
        } else if (d % 64 == 0) {
#pragma unroll
            for (int t = 0; t < 4; t += 2) *reinterpret_cast<uint16_t*>(piece + value_codes_at(d, at.in_page, 4 * i + t)) = (uint16_t)(codes >> (8 * t));
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t) piece[value_codes_at(d, at.in_page, 4 * i + t)] = (uint8_t)(codes >> (8 * t));
        }
        if ((i & 3) == 0) piece[scale_at(d, kv.page_shift, at.in_page, i / 4, is_value)] = (uint8_t)byte;
    }
}

// Rows of a cache of 4 bits as values: 8 to an item.  4096 rows of 32 heads of 128, 85 MB: 27 us, 3.2 TB/s, two trips before the codes.
template <class T>
__global__ __launch_bounds__(256)
void cache_rows_fp4_kernel(CacheRows o, int rows_log) {
    const KvCache& kv = o.cache;
    const int threads = 256 >> rows_log, thread = threadIdx.x & (threads - 1), row = row_of_thread(rows_log);
    if (row >= o.batch.n_rows) return;
    Fp4Row at;
    if (!find_row(o.batch, kv, row, &at)) return;
    const int d = kv.head_dim, hkv = kv.n_kv_heads, per_head = d / 8;
    for (int e = blockIdx.y * threads + thread; e < 2 * hkv * per_head; e += threads * gridDim.y) {
        const int head2 = e / per_head, i = e - head2 * per_head;
        const bool is_value = head2 >= hkv;
        const int head = is_value ? head2 - hkv : head2;
        T* out = (T*)(is_value ? o.V : o.K);
        if (!out) continue;
        float v[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = at.pos < 0 ? 0.f : __builtin_nanf("");
        if (at.kept) {
            const uint8_t* piece = (const uint8_t*)(is_value ? kv.v : kv.k) + at.page * kv.page_stride + head * kv.head_stride;
            uint32_t codes = 0;
            if (!is_value || d % 128 == 0) {
                codes = *reinterpret_cast<const uint32_t*>(piece + (is_value ? value_codes_at(d, at.in_page, 4 * i) : key_codes_at(d, at.in_page, 4 * i)));
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t) codes |= (uint32_t)piece[value_codes_at(d, at.in_page, 4 * i + t)] << (8 * t);
            }
            const float scale = fp4_scale(piece[scale_at(d, kv.page_shift, at.in_page, i / 4, is_value)]);
            static_for<4>([&](auto ic) {
                constexpr int t = decltype(ic)::value;
                const uint32_t pair = fp4_pair<t>(codes, scale);
                v[2 * t] = __uint_as_float(pair << 16);
                v[2 * t + 1] = __uint_as_float(pair & 0xFFFF0000u);
            });
        }
        Eight<T> x;
        x.set(v);
        x.store(out + (int64_t)row * (is_value ? o.ldv : o.ldk) + head * d + 8 * i);
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

// Rows of a workgroup (the logarithm): two or four where a row has items for no more of its threads (7632 rows of 5/5 heads of 64 20.6 and 15.9 us, read back 12.7 and 10.3;
// 5450 rows of one key head of 128 read back 6.7 and 4.4).
static int rows_log(int items) { return items <= 64 ? 2 : items <= 128 ? 1 : 0; }
// workgroups to a row: as many as its items fill, where the rows leave CUs idle
static int shares(int n_rows, int items) {
    const int most = (items + 255) / 256, idle = 1024 / n_rows;
    return idle < 1 ? 1 : idle < most ? idle : most;
}

hipError_t rope_append_fp4(const RopeAppend& o, int is_bf16, hipStream_t stream) {
    const int d = o.cache.head_dim, items = 2 * o.cache.n_kv_heads * d / 8 + o.n_q_heads * ((o.pairs ? o.rot / 8 : o.rot / 16) + (d - o.rot) / 8);
    const int log = rows_log(items);
    const dim3 grid((o.batch.n_rows + (1 << log) - 1) >> log, shares(o.batch.n_rows, items));
    if (is_bf16) hipLaunchKernelGGL(rope_append_fp4_kernel<uint16_t>, grid, dim3(256), 0, stream, o, log);
    else hipLaunchKernelGGL(rope_append_fp4_kernel<float>, grid, dim3(256), 0, stream, o, log);
    return hipGetLastError();
}

hipError_t cache_rows_fp4(const CacheRows& o, int is_bf16, hipStream_t stream) {
    const int items = 2 * o.cache.n_kv_heads * o.cache.head_dim / 8, log = rows_log(items);
    const dim3 grid((o.batch.n_rows + (1 << log) - 1) >> log, shares(o.batch.n_rows, items));
    if (is_bf16) hipLaunchKernelGGL(cache_rows_fp4_kernel<uint16_t>, grid, dim3(256), 0, stream, o, log);
    else hipLaunchKernelGGL(cache_rows_fp4_kernel<float>, grid, dim3(256), 0, stream, o, log);
    return hipGetLastError();
}

}  // namespace gelo
