// Attention over the paged cache.  For a row's head q and the keys k_p, values v_p it sees: O = sum_p w_p v_p / sum_p w_p, w_p = exp(scale q.k_p - m),
// in one pass over the cache with a running maximum m, sum and weighted sum that are rescaled when m grows.
//
// Keys of one head and all queries that meet it - the rows a sequence brings times the query heads that share the key head - are one
// product: a COLUMN is such a query, 16 columns are a tile.  S^T = K Q^T (rows: keys, columns: queries) leaves in every lane scores of
// one column, so maximum, sum and the rescaling stay in the lane, and the weights are at once the operand of O^T = V^T P^T: the matrix
// instruction sums over keys in any order, as long as both operands agree on it.
//
// attention_few_kernel: decode.  Bound by the cache's bytes.  K and V go from memory to registers with nothing between, as the matrix
// instructions want them; four waves of a workgroup walk different keys and join at the end.
#include "gelo_internal.h"
#include "paged.h"

namespace gelo {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
constexpr float kLog2E = 1.4426950408889634f;

struct AttnArgs {
    const void* Q; int64_t ldq;
    void* O; int64_t ldo;
    float* part_o;               // [chunk][row][head][D], where the cache is cut
    float* part_ml;              // [chunk][row][head][2]: maximum (of log2) and sum
    int n_q_heads, group;        // query heads to a key head
    float scale2;                // scale * log2 e
    int causal;
    int chunk, n_chunks, col_tiles;
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

template <class T, int D> struct Few;

// bfloat16, 32 keys a step.  Lane (g, c) = (lane / 16, lane % 16).
//   S^T, tile t of 16 keys: A = K, row c = key 16 t + c, contraction values 32 s + 8 g ...: 16 bytes of that key; B = Q^T alike.
//   The lane then holds S of column c and keys 16 t + 4 g + r.  O^T: the B operand wants 8 keys of column c: those very ones, slot i =
//   4 t + r.  So A = V^T must have in slot i of group g the key 16 (i / 4) + 4 g + i % 4, for row c: a lane loads VD = D / 16 consecutive values
//   of these 8 keys (16 lanes: one whole row) and transposes its 8 x VD block in registers; instruction j computes components VD m + j.
template <int D>
struct Few<uint16_t, D> {
    static constexpr int KEYS = 32, TILES = 2, KS = D / 32, VD = D / 16, VW = VD / 2;      // VW: 32-bit words of VD values
    typedef bf16x8_t KFrag;
    bf16x8_t q[KS];
    bf16x8_t k[TILES][KS];
    uint32_t v[8][VW];
    __device__ __forceinline__ void load_q(const uint16_t* p, int g) {
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const bf16x8_t*>(p + 32 * s + 8 * g);
    }
    __device__ __forceinline__ void load_k(int t, const uint16_t* row, int g) {
#pragma unroll
        for (int s = 0; s < KS; ++s) k[t][s] = *reinterpret_cast<const bf16x8_t*>(row + 32 * s + 8 * g);
    }
    // r: slot of the tile's group of four
    __device__ __forceinline__ void load_v(int t, int r, const uint16_t* row, int c) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(row) + VW * c;
        if constexpr (VW % 4 == 0) {
#pragma unroll
            for (int w = 0; w < VW; w += 4) {
                const u32x4_t x = *reinterpret_cast<const u32x4_t*>(p + w);
#pragma unroll
                for (int u = 0; u < 4; ++u) v[4 * t + r][w + u] = x[u];
            }
        } else if constexpr (VW == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(p);
            v[4 * t + r][0] = x.x; v[4 * t + r][1] = x.y;
        } else {
            const uint3 x = *reinterpret_cast<const uint3*>(p);                     // 12 bytes, 4-byte aligned
            v[4 * t + r][0] = x.x; v[4 * t + r][1] = x.y; v[4 * t + r][2] = x.z;
        }
    }
    __device__ __forceinline__ f32x4_t scores(int t) const {
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KS; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[t][i], q[i], s, 0, 0, 0);
        return s;
    }
    // operand of O^T for component j of the lane's VD: half j % 2 of word j / 2 of the 8 slots
    __device__ __forceinline__ u32x4_t v_frag(int j) const {
        u32x4_t f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f[i] = __builtin_amdgcn_perm(v[2 * i + 1][j >> 1], v[2 * i][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
        return f;
    }
    static __device__ __forceinline__ bf16x8_t weights(const float (&p)[8]) {
        bf16x8_t o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (__bf16)p[i];
        return o;
    }
    __device__ __forceinline__ void accumulate(f32x4_t (&acc)[VD], const float (&p)[8]) const {
        const bf16x8_t w = weights(p);
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v_frag(j)), w, acc[j], 0, 0, 0);
    }
    __device__ __forceinline__ bool odd_values() const {       // a NaN or an infinity among the values
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int w = 0; w < VW; ++w) odd |= (v[i][w] & 0x7F80u) == 0x7F80u || (v[i][w] & 0x7F800000u) == 0x7F800000u;
        return odd;
    }
    // as accumulate, where some keys are hidden from some columns (seen: bit per slot) and some values are not finite: 0 times those would be
    // NaN in columns that do not see them.  The finite part is summed as ever; how many +inf (-inf, NaN: both) a column sees is counted by two more products.
    __device__ __forceinline__ void accumulate_odd(f32x4_t (&acc)[VD], const float (&p)[8], uint32_t seen) const {
        const bf16x8_t w = weights(p);
        float one[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) one[i] = (seen >> i) & 1 ? 1.f : 0.f;
        const bf16x8_t sees = weights(one);
        for (int j = 0; j < VD; ++j) {
            u32x4_t f = {0, 0, 0, 0}, fin = f, up = {0, 0, 0, 0}, down = {0, 0, 0, 0};
#pragma unroll
            for (int jj = 0; jj < VD; ++jj) if (jj == j) f = v_frag(jj);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t x = (f[i] >> (16 * h)) & 0xFFFFu;
                    const bool odd = (x & 0x7F80u) == 0x7F80u, nan = odd && (x & 0x7Fu);
                    fin[i] |= (odd ? 0u : x) << (16 * h);
                    up[i] |= (odd && (nan || !(x & 0x8000u)) ? 0x3F80u : 0u) << (16 * h);
                    down[i] |= (odd && (nan || (x & 0x8000u)) ? 0x3F80u : 0u) << (16 * h);
                }
            const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
            f32x4_t sum = zero;
#pragma unroll
            for (int jj = 0; jj < VD; ++jj) if (jj == j) sum = acc[jj];
            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, fin), w, sum, 0, 0, 0);
            const f32x4_t ups = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, up), sees, zero, 0, 0, 0);
            const f32x4_t downs = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, down), sees, zero, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[r] += (ups[r] > 0.f ? __builtin_inff() : 0.f) - (downs[r] > 0.f ? __builtin_inff() : 0.f);
#pragma unroll
            for (int jj = 0; jj < VD; ++jj) if (jj == j) acc[jj] = sum;
        }
    }
};

// float, 16 keys a step: v_mfma_f32_16x16x4_f32, one contraction value per lane.  Instruction (s, e) of S^T takes component 16 s + 4 g + e,
// instruction (r, j) of O^T the key 4 g + r, whose weight is register r of the scores.
template <int D>
struct Few<float, D> {
    static constexpr int KEYS = 16, TILES = 1, KS = D / 16, VD = D / 16;
    f32x4_t q[KS], k[1][KS];
    float v[4][VD];
    __device__ __forceinline__ void load_q(const float* p, int g) {
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const f32x4_t*>(p + 16 * s + 4 * g);
    }
    __device__ __forceinline__ void load_k(int, const float* row, int g) {
#pragma unroll
        for (int s = 0; s < KS; ++s) k[0][s] = *reinterpret_cast<const f32x4_t*>(row + 16 * s + 4 * g);
    }
    __device__ __forceinline__ void load_v(int, int r, const float* row, int c) {
        const float* p = row + VD * c;
        if constexpr (VD % 4 == 0) {
#pragma unroll
            for (int w = 0; w < VD; w += 4) {
                const f32x4_t x = *reinterpret_cast<const f32x4_t*>(p + w);
#pragma unroll
                for (int u = 0; u < 4; ++u) v[r][w + u] = x[u];
            }
        } else {
#pragma unroll
            for (int w = 0; w < VD; w += 2) {
                const float2 x = *reinterpret_cast<const float2*>(p + w);
                v[r][w] = x.x; v[r][w + 1] = x.y;
            }
        }
    }
    __device__ __forceinline__ f32x4_t scores(int) const {
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[0][i][e], q[i][e], s, 0, 0, 0);
        return s;
    }
    __device__ __forceinline__ void accumulate(f32x4_t (&acc)[VD], const float (&p)[4]) const {
#pragma unroll
        for (int j = 0; j < VD; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][j], p[r], acc[j], 0, 0, 0);
    }
    __device__ __forceinline__ bool odd_values() const {
        bool odd = false;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < VD; ++j) odd |= (__float_as_uint(v[r][j]) & 0x7F800000u) == 0x7F800000u;
        return odd;
    }
    __device__ __forceinline__ void accumulate_odd(f32x4_t (&acc)[VD], const float (&p)[4], uint32_t seen) const {
#pragma unroll
        for (int j = 0; j < VD; ++j) {
            f32x4_t ups = {0.f, 0.f, 0.f, 0.f}, downs = ups;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = v[r][j], sees = (seen >> r) & 1 ? 1.f : 0.f;
                const bool odd = (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u;
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(odd ? 0.f : x, p[r], acc[j], 0, 0, 0);
                ups = __builtin_amdgcn_mfma_f32_16x16x4f32(odd && !(x < 0.f) ? 1.f : 0.f, sees, ups, 0, 0, 0);
                downs = __builtin_amdgcn_mfma_f32_16x16x4f32(odd && !(x > 0.f) ? 1.f : 0.f, sees, downs, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[j][r] += (ups[r] > 0.f ? __builtin_inff() : 0.f) - (downs[r] > 0.f ? __builtin_inff() : 0.f);
        }
    }
};

template <class T> __device__ __forceinline__ void store4(T* p, f32x4_t v);
template <> __device__ __forceinline__ void store4<float>(float* p, f32x4_t v) { *reinterpret_cast<f32x4_t*>(p) = v; }
template <> __device__ __forceinline__ void store4<uint16_t>(uint16_t* p, f32x4_t v) {
    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4_t*>(p) = bf16x4_t{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
}

constexpr int kFewWaves = 4;

// A workgroup: one tile of 16 columns of one sequence and key head, one chunk of the cache.
template <class T, int D>
__global__ __launch_bounds__(64 * kFewWaves)
void attention_few_kernel(AttnArgs a) {
    typedef Few<T, D> F;
    constexpr int VD = F::VD, SLOTS = 4 * F::TILES;
    __shared__ float joined_o[kFewWaves][16][D + 4];
    __shared__ float joined_ml[kFewWaves][16][2];
    const int chunk = blockIdx.x % a.n_chunks;
    int rest = blockIdx.x / a.n_chunks;
    const int tile = rest % a.col_tiles; rest /= a.col_tiles;
    const int kvh = rest % a.kv.n_kv_heads, seq = rest / a.kv.n_kv_heads;
    const NewRows rows = rows_of_sequence(a.b, seq);
    const int columns = rows.count * a.group;
    if (tile * 16 >= columns) return;
    const int kv_len = a.b.kv_len[seq], kv_end = min(kv_len, a.b.max_kv_len);

    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = tile * 16 + c;
    const bool live = col < columns;
    const int my = live ? col : columns - 1;                 // dead columns repeat the last one
    const int i = my / a.group, head = kvh * a.group + my - i * a.group;
    const int row = rows.first + i;
    const int limit = min(a.causal ? kv_len - rows.count + i : kv_len - 1, kv_end - 1);      // last key this column sees
    // the last column sees most, the first one least
    const int most = __builtin_amdgcn_readlane(limit, 15), least = __builtin_amdgcn_readfirstlane(limit);
    const int begin = chunk * a.chunk, end = min(begin + a.chunk, most + 1);
    if (begin >= end && a.n_chunks > 1) return;              // the join does not look at it

    F f;
    f.load_q((const T*)a.Q + row * a.ldq + (int64_t)head * D, g);
    f32x4_t acc[VD];
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -__builtin_inff(), l = 0.f;
    bool bad_page = false;

    const int last = end - 1, shift = a.kv.page_shift, in_page = (1 << shift) - 1;
    const int32_t* table = a.b.page_table + seq * a.b.table_ld;
    const T* k_head = (const T*)a.kv.k + kvh * a.kv.head_stride;
    const T* v_head = (const T*)a.kv.v + kvh * a.kv.head_stride;
    // keys beyond the end are read as the last key, whose address is good, and get no weight
    auto tile_start = [&](int key) { return min(key, last & ~15); };
    auto page_of = [&](int key) { return table[tile_start(key) >> shift]; };
    auto page_base = [&](int key, int page) {
        const bool good = page >= 0 && page < a.kv.n_pages;
        bad_page |= !good;
        return (good ? page : 0) * a.kv.page_stride + (tile_start(key) & in_page) * a.kv.row_stride;
    };
    auto load_k = [&](int key, const int (&page)[F::TILES]) {
#pragma unroll
        for (int t = 0; t < F::TILES; ++t) {
            const int at = key + 16 * t, r = min(at + c, last) - tile_start(at);
            f.load_k(t, k_head + page_base(at, page[t]) + r * a.kv.row_stride, g);
        }
    };
    auto load_v = [&](int key, const int (&page)[F::TILES]) {
#pragma unroll
        for (int t = 0; t < F::TILES; ++t) {
            const int at = key + 16 * t;
            const T* base = v_head + page_base(at, page[t]);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int r = min(at + 4 * g + u, last) - tile_start(at);
                f.load_v(t, u, base + r * a.kv.row_stride, c);
            }
        }
    };

    constexpr int STRIDE = F::KEYS * kFewWaves;
    int key = begin + wave * F::KEYS;
    if (key < end) {
        int page[F::TILES];
#pragma unroll
        for (int t = 0; t < F::TILES; ++t) page[t] = page_of(key + 16 * t);
        load_k(key, page);
        load_v(key, page);
        for (; key < end; key += STRIDE) {
            const int next = key + STRIDE;
            if (next < end) {
#pragma unroll
                for (int t = 0; t < F::TILES; ++t) page[t] = page_of(next + 16 * t);
            }
            float s[SLOTS];
#pragma unroll
            for (int t = 0; t < F::TILES; ++t) {
                const f32x4_t x = f.scores(t);
#pragma unroll
                for (int r = 0; r < 4; ++r) s[4 * t + r] = x[r] * a.scale2;
            }
            if (next < end) load_k(next, page);
            // hidden: keys beyond what the column sees (uniform test first: most steps have none)
            const bool partly = key + F::KEYS - 1 > min(least, last);
            uint32_t seen = ~0u;
            if (partly) {
                const int upto = min(limit, last);
                seen = 0;
#pragma unroll
                for (int t = 0; t < F::TILES; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const bool sees = key + 16 * t + 4 * g + r <= upto;
                        s[4 * t + r] = sees ? s[4 * t + r] : -__builtin_inff();
                        seen |= (uint32_t)sees << (4 * t + r);
                    }
            }
            float top = s[0];
#pragma unroll
            for (int r = 1; r < SLOTS; ++r) top = fmaxf(top, s[r]);
            const float m_new = fmaxf(m, across_groups_max(top));
            const float m_safe = m_new == -__builtin_inff() ? 0.f : m_new;        // nothing seen yet: all weights are 0
            const float alpha = __builtin_amdgcn_exp2f(m - m_safe);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int r = 0; r < SLOTS; ++r) {
                s[r] = __builtin_amdgcn_exp2f(s[r] - m_safe);
                l += s[r];
            }
            if (__ballot(alpha != 1.f)) {
#pragma unroll
                for (int j = 0; j < VD; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[j][r] *= alpha;
            }
            if (partly && __ballot(f.odd_values())) f.accumulate_odd(acc, s, seen);
            else f.accumulate(acc, s);
            if (next < end) load_v(next, page);
        }
    }
    l = across_groups_sum(l);
    if (bad_page) l = __builtin_nanf("");

    // acc[j][r]: component VD (4 g + r) + j of column c
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < VD; ++j) joined_o[wave][c][VD * (4 * g + r) + j] = acc[j][r];
    if (g == 0) { joined_ml[wave][c][0] = m; joined_ml[wave][c][1] = l; }
    __syncthreads();
    const int first_head = kvh * a.group;
    for (int e = threadIdx.x; e < 16 * (D / 4); e += 64 * kFewWaves) {
        const int cc = e / (D / 4), x = 4 * (e - cc * (D / 4));
        const int cl = tile * 16 + cc;
        if (cl >= columns) continue;
        float top = joined_ml[0][cc][0];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) top = fmaxf(top, joined_ml[w][cc][0]);
        const float safe = top == -__builtin_inff() ? 0.f : top;
        float total = 0.f;
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) {
            if (joined_ml[w][cc][1] == 0.f) continue;        // nothing seen: 0 times what it holds need not be 0
            const float k = __builtin_amdgcn_exp2f(joined_ml[w][cc][0] - safe);
            total += k * joined_ml[w][cc][1];
            const f32x4_t y = *reinterpret_cast<const f32x4_t*>(&joined_o[w][cc][x]);
#pragma unroll
            for (int u = 0; u < 4; ++u) o[u] += k * y[u];
        }
        const int ri = cl / a.group, h = first_head + cl - ri * a.group;
        const int64_t rr = rows.first + ri;
        if (a.n_chunks == 1) {
            const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
            for (int u = 0; u < 4; ++u) o[u] = total == 0.f ? 0.f : o[u] * inv;
            store4((T*)a.O + rr * a.ldo + (int64_t)h * D + x, o);
        } else {
            const int64_t item = ((int64_t)chunk * a.b.n_rows + rr) * a.n_q_heads + h;
            *reinterpret_cast<f32x4_t*>(a.part_o + item * D + x) = o;
            if (x == 0) { a.part_ml[2 * item] = top; a.part_ml[2 * item + 1] = total; }
        }
    }
}

// Joins the chunks' parts of a row's head: O = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.
template <class T, int D>
__global__ __launch_bounds__(256)
void attention_join_kernel(AttnArgs a) {
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t items = (int64_t)a.b.n_rows * a.n_q_heads;
    int64_t item = e / (D / 4);
    const int x = 4 * (int)(e - item * (D / 4));
    const bool there = item < items;
    if (!there) item = items - 1;
    const int row = (int)(item / a.n_q_heads);
    int seq = row, i = 0, count = 1;
    if (a.b.row_start) {
        // the rows of a wave differ by a few at most, yet each thread looks for its own
        int lo = 0, hi = a.b.n_seqs;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (a.b.row_start[mid + 1] <= row) lo = mid + 1; else hi = mid;
        }
        seq = lo;
        if (seq >= a.b.n_seqs) return;
        const NewRows rows = rows_of_sequence(a.b, seq);
        i = row - rows.first;
        count = rows.count;
        if (i < 0 || i >= count) return;
    }
    if (!there) return;
    const int kv_len = a.b.kv_len[seq], kv_end = min(kv_len, a.b.max_kv_len);
    const int limit = min(a.causal ? kv_len - count + i : kv_len - 1, kv_end - 1);
    const int used = limit < 0 ? 0 : limit / a.chunk + 1;
    float top = -__builtin_inff(), total = 0.f;
    for (int s = 0; s < used; ++s) top = fmaxf(top, a.part_ml[2 * (s * items + item)]);
    const float safe = top == -__builtin_inff() ? 0.f : top;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < used; ++s) {
        const int64_t at = s * items + item;
        const float ls = a.part_ml[2 * at + 1];
        if (ls == 0.f) continue;
        const float k = __builtin_amdgcn_exp2f(a.part_ml[2 * at] - safe);
        total += k * ls;
        const f32x4_t y = *reinterpret_cast<const f32x4_t*>(a.part_o + at * D + x);
#pragma unroll
        for (int u = 0; u < 4; ++u) o[u] += k * y[u];
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int u = 0; u < 4; ++u) o[u] = total == 0.f ? 0.f : o[u] * inv;
    store4((T*)a.O + row * a.ldo + (item - (int64_t)row * a.n_q_heads) * D + x, o);
}

// How the cache is cut: chunks of `chunk` keys, n_chunks of them to the longest sequence.
struct Plan { int col_tiles, chunk, n_chunks; int64_t workgroups; };
constexpr int kFewTarget = 1024;         // workgroups that fill the chip
constexpr int64_t kMostWorkgroups = 1 << 23;     // of a launch: 2^31 threads and no more fit HIP's 32-bit counts
constexpr int kFewLeast = 256;           // keys to a chunk, at least

Plan plan_few(const Attention& o) {
    Plan p;
    const int group = o.n_q_heads / o.cache.n_kv_heads;
    p.col_tiles = (int)(((int64_t)o.batch.max_rows * group + 15) / 16);
    const int64_t tiles = (int64_t)o.batch.n_seqs * o.cache.n_kv_heads * p.col_tiles;
    int64_t cuts = kFewTarget / tiles;
    const int64_t most = (o.batch.max_kv_len + kFewLeast - 1) / kFewLeast;
    cuts = cuts < 1 ? 1 : cuts < most ? cuts : most;
    if (cuts < 1) cuts = 1;
    p.chunk = (int)round_up((o.batch.max_kv_len + cuts - 1) / cuts, 128);
    p.n_chunks = p.chunk > 0 ? (o.batch.max_kv_len + p.chunk - 1) / p.chunk : 1;
    if (p.n_chunks < 1) p.n_chunks = 1;
    p.workgroups = tiles * p.n_chunks;
    return p;
}

size_t part_bytes(const Attention& o, const Plan& p) {
    return p.n_chunks == 1 ? 0 : (size_t)p.n_chunks * o.batch.n_rows * o.n_q_heads * (o.cache.head_dim + 2) * sizeof(float);
}

template <class T, int D>
hipError_t launch(const Attention& o, hipStream_t stream) {
    const Plan p = plan_few(o);
    AttnArgs a;
    a.Q = o.Q; a.ldq = o.ldq; a.O = o.O; a.ldo = o.ldo;
    a.n_q_heads = o.n_q_heads; a.group = o.n_q_heads / o.cache.n_kv_heads;
    a.scale2 = o.scale * kLog2E; a.causal = o.causal;
    a.chunk = p.chunk; a.n_chunks = p.n_chunks; a.col_tiles = p.col_tiles;
    a.kv = o.cache; a.b = o.batch;
    const int64_t items = (int64_t)o.batch.n_rows * o.n_q_heads;
    a.part_o = o.workspace;
    a.part_ml = p.n_chunks == 1 ? nullptr : o.workspace + (int64_t)p.n_chunks * items * D;
    hipLaunchKernelGGL((attention_few_kernel<T, D>), dim3((unsigned)p.workgroups), dim3(64 * kFewWaves), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.n_chunks == 1) return e;
    hipLaunchKernelGGL((attention_join_kernel<T, D>), dim3((unsigned)((items * (D / 4) + 255) / 256)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <class T>
hipError_t of_width(const Attention& o, hipStream_t stream) {
    switch (o.cache.head_dim) {
        case 64: return launch<T, 64>(o, stream);
        case 96: return launch<T, 96>(o, stream);
        case 128: return launch<T, 128>(o, stream);
        case 256: return launch<T, 256>(o, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

bool attention_fits(const Attention& o, int) {
    return plan_few(o).workgroups <= kMostWorkgroups && ((int64_t)o.batch.n_rows * o.n_q_heads * (o.cache.head_dim / 4) + 255) / 256 <= kMostWorkgroups;
}
size_t attention_workspace_bytes(const Attention& o, int) { return part_bytes(o, plan_few(o)); }
// a plan with more than one chunk has at most kFewTarget workgroups of 16 columns
size_t attention_workspace_bound(int head_dim) { return (size_t)kFewTarget * 16 * (head_dim + 2) * sizeof(float); }

hipError_t attention(const Attention& o, int is_bf16, hipStream_t stream) {
    return is_bf16 ? of_width<uint16_t>(o, stream) : of_width<float>(o, stream);
}

hipError_t attention_init() { return hipSuccess; }

}  // namespace gelo
