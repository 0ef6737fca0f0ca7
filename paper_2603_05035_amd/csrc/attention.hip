// Attention over the paged cache.  For a row's head q and the keys k_p, values v_p it sees: O = sum_p w_p v_p / sum_p w_p, w_p = exp(scale q.k_p - m),
// in one pass over the cache with a running maximum m, sum and weighted sum that are rescaled when m grows.
//
// Keys of one head and all queries that meet it - the rows a sequence brings times the query heads that share the key head - are one
// product: a COLUMN is such a query, 16 columns are a tile.  S^T = K Q^T (rows: keys, columns: queries) leaves in every lane scores of
// one column, so maximum, sum and the rescaling stay in the lane, and the weights are at once the operand of O^T = V^T P^T: the matrix
// instruction sums over keys in any order, as long as both operands agree on it.
//
// Scores, weights, maximum, sum and weighted sum are float.  Where the values are bfloat16 the second product takes bfloat16 weights.  With few columns
// the matrix pipes have time to spare and a weight is two of them, 16 bits: results are as near as their own rounding.  In the kernel for prompts, which the
// matrix pipes bound, weights (at most 2^8.5) are rounded to one, and their sum is that of the rounded ones: a row that sees one key is then that
// key's value, and rounding moves the others by no more than the values' distance from their mean.
//
// attention_few_kernel: single tokens and a few rows, and float where its prompts do not fill the chip.  Bound by the cache's bytes: every one is read once by one wave, and a
// CU has about 130 KB of them on their way.  K and V go from memory to registers with nothing between, as the matrix instructions want them (15
// of 16 columns are idle where a key head has one query: the matrix pipes have that to spare); four waves of a workgroup walk different keys and join at
// the end.  A single token of each of 64 sequences, 32 heads of 128, bfloat16: 3500 to 4095 rows 626 us (6.3 TB/s of those there are), 400 to 639 rows 93
// (5.9; 92 with weights of 8 bits), 3 sequences of 20000 to 32767 rows of 8 heads 64 and 4.3 for the join (5.8 without it).  In float 1297 (6.1), 200 (5.5) and
// 145 (5.2); of heads of 256, whose 416 registers leave one wave to a SIMD and half the bytes on their way, 64 x 2048 keys of 8 heads 465 (4.6).  Three
// sequences of up to 200 rows 7.7: trips to memory one after another - lengths, page numbers, keys.
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

// the place of the part that chunk `chunk` makes of head `head` of a sequence's row i
__device__ __forceinline__ int64_t part_of(const AttnArgs& a, int chunk, int seq, int i, int head) {
    return (((int64_t)chunk * a.b.n_seqs + seq) * a.b.max_rows + i) * a.n_q_heads + head;
}

// sum + the two bfloat16 of a word: their products with 1
__device__ __forceinline__ float add_pair(uint32_t pair, float sum) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pair), bf16x2_t{(__bf16)1.f, (__bf16)1.f}, sum, false);
}

// PAST: cache rows are read past the caches (nobody reads them again soon)
template <class V, bool PAST>
__device__ __forceinline__ V read_row(const void* p) {
    if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
    else return *reinterpret_cast<const V*>(p);
}

template <class T, int D, bool PAST> struct Few;

// bfloat16, 32 keys a step, of heads of 256 half of that (what follows is for 32): with 32 the registers leave one wave to a SIMD, and few keys
// take long: 14 sequences of 21 rows and 60 keys, 32 heads, 36.4 us with 32 and 22.7 with 16, one row of 256 sequences of 64 keys, 8 heads, 47.6
// and 31.3, of 16 sequences of 2048 keys 54.2 and 51.5.  Lane (g, c) = (lane / 16, lane % 16).
//   S^T, tile t of 16 keys: A = K, row c = key 16 t + c, contraction values 32 s + 8 g ...: 16 bytes of that key; B = Q^T alike.
//   The lane then holds S of column c and keys 16 t + 4 g + r.  O^T: the B operand wants 8 keys of column c: those very ones, slot i =
//   4 t + r.  So A = V^T must have in slot i of group g the key 16 (i / 4) + 4 g + i % 4, for row c: a lane loads VD = D / 16 consecutive values
//   of these 8 keys (16 lanes: one whole row) and transposes its 8 x VD block in registers; instruction j computes components VD m + j.
template <int D, bool PAST>
struct Few<uint16_t, D, PAST> {
    static constexpr int TILES = D < 256 ? 2 : 1, KEYS = 16 * TILES, SLOTS = 4 * TILES;
    static constexpr int KS = D / 32, VD = D / 16, VW = VD / 2;        // VW: 32-bit words of VD values
    typedef uint32_t frag_t __attribute__((ext_vector_type(2 * TILES)));       // SLOTS weights or values
    // Of heads of 256 the last pieces of Q lie in LDS: with all of them in registers some would be kept in memory, and a wait for those is one for
    // the keys and values on their way.
    static constexpr int APART = D < 256 ? 0 : 2;
    bf16x8_t q[KS - APART];
    bf16x8_t* q_apart;                                       // this lane's: 64 lanes to a piece
    bf16x8_t k[TILES][KS];
    uint32_t v[SLOTS][VW];
    // lds: the wave's own, 1 KB to a piece
    __device__ __forceinline__ void load_q(const uint16_t* p, int g, float* lds) {
        q_apart = reinterpret_cast<bf16x8_t*>(lds) + (threadIdx.x & 63);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const bf16x8_t x = *reinterpret_cast<const bf16x8_t*>(p + 32 * s + 8 * g);
            if (s < KS - APART) q[s] = x;
            else q_apart[64 * (s - (KS - APART))] = x;
        }
    }
    __device__ __forceinline__ void load_k(int t, const uint16_t* row, int g) {
#pragma unroll
        for (int s = 0; s < KS; ++s) k[t][s] = read_row<bf16x8_t, PAST>(row + 32 * s + 8 * g);
    }
    // r: slot of the tile's group of four
    __device__ __forceinline__ void load_v(int t, int r, const uint16_t* row, int c) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(row) + VW * c;
        if constexpr (VW % 4 == 0) {
#pragma unroll
            for (int w = 0; w < VW; w += 4) {
                const u32x4_t x = read_row<u32x4_t, PAST>(p + w);
#pragma unroll
                for (int u = 0; u < 4; ++u) v[4 * t + r][w + u] = x[u];
            }
        } else if constexpr (VW == 2) {
            const u32x2_t x = read_row<u32x2_t, PAST>(p);
            v[4 * t + r][0] = x[0]; v[4 * t + r][1] = x[1];
        } else {
            const u32x3_t x = read_row<u32x3_t, PAST>(p);
            v[4 * t + r][0] = x[0]; v[4 * t + r][1] = x[1]; v[4 * t + r][2] = x[2];
        }
    }
    __device__ __forceinline__ f32x4_t scores(int t) const {
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KS - APART; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[t][i], q[i], s, 0, 0, 0);
        if constexpr (APART > 0) {
            asm volatile("" ::: "memory");                   // read here, not kept
#pragma unroll
            for (int i = KS - APART; i < KS; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[t][i], q_apart[64 * (i - (KS - APART))], s, 0, 0, 0);
        }
        return s;
    }
    // operand of O^T for component j of the lane's VD: half j % 2 of word j / 2 of the slots
    __device__ __forceinline__ frag_t v_frag(int j) const {
        frag_t f;
#pragma unroll
        for (int i = 0; i < 2 * TILES; ++i)
            f[i] = __builtin_amdgcn_perm(v[2 * i + 1][j >> 1], v[2 * i][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
        return f;
    }
    // A weight is the sum of two bfloat16: its upper half as it stands and what is left of it.  Neither is nought or negative where the weight is
    // not nought: an infinite value times both is that infinity.
    struct weights_t { frag_t high, low; };
    static __device__ __forceinline__ weights_t weights(const float (&p)[SLOTS]) {
        typedef __bf16 pack_t __attribute__((ext_vector_type(SLOTS)));
        frag_t high;
        pack_t low;
#pragma unroll
        for (int i = 0; i < 2 * TILES; ++i) high[i] = __builtin_amdgcn_perm(__float_as_uint(p[2 * i + 1]), __float_as_uint(p[2 * i]), 0x07060302u);
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            const float up = __uint_as_float(__float_as_uint(p[i]) & 0xFFFF0000u);
            low[i] = (__bf16)fmaxf(p[i] - up, fminf(up, 0x1p-120f));
        }
        return {high, __builtin_bit_cast(frag_t, low)};
    }
    static __device__ __forceinline__ f32x4_t product(frag_t values, frag_t weights, f32x4_t sum) {
        typedef short s16x4_t __attribute__((ext_vector_type(4)));
        if constexpr (TILES == 2) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, values), __builtin_bit_cast(bf16x8_t, weights), sum, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4_t, values), __builtin_bit_cast(s16x4_t, weights), sum, 0, 0, 0);
    }
    __device__ __forceinline__ void accumulate(f32x4_t (&acc)[VD], weights_t w) const {
#pragma unroll
        for (int j = 0; j < VD; ++j) {
            const frag_t f = v_frag(j);
            acc[j] = product(f, w.low, product(f, w.high, acc[j]));
        }
    }
    __device__ __forceinline__ bool odd_values() const {       // a NaN or an infinity among the values
        bool odd = false;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
#pragma unroll
            for (int w = 0; w < VW; ++w) odd |= (v[i][w] & 0x7F80u) == 0x7F80u || (v[i][w] & 0x7F800000u) == 0x7F800000u;
        return odd;
    }
    // as accumulate, where some keys are hidden from some columns (seen: bit per slot) and some values are not finite: 0 times those would be
    // NaN in columns that do not see them.  The finite part is summed as ever; how many +inf (-inf, NaN: both) a column sees is counted by two more products.
    __device__ __forceinline__ void accumulate_odd(f32x4_t (&acc)[VD], weights_t w, uint32_t seen) const {
        float one[SLOTS];
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) one[i] = (seen >> i) & 1 ? 1.f : 0.f;
        const frag_t sees = weights(one).high;
        for (int j = 0; j < VD; ++j) {
            frag_t f = frag_t(0u), fin = f, up = f, down = f;
#pragma unroll
            for (int jj = 0; jj < VD; ++jj) if (jj == j) f = v_frag(jj);
#pragma unroll
            for (int i = 0; i < 2 * TILES; ++i)
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
            sum = product(fin, w.low, product(fin, w.high, sum));
            const f32x4_t ups = product(up, sees, zero), downs = product(down, sees, zero);
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[r] += (ups[r] > 0.f ? __builtin_inff() : 0.f) - (downs[r] > 0.f ? __builtin_inff() : 0.f);
#pragma unroll
            for (int jj = 0; jj < VD; ++jj) if (jj == j) acc[jj] = sum;
            __builtin_amdgcn_sched_barrier(0);               // one component after another: together their masks take registers that the loop needs
        }
    }
};

// float, 16 keys a step: v_mfma_f32_16x16x4_f32, one contraction value per lane.  Instruction (s, e) of S^T takes component 16 s + 4 g + e,
// instruction (r, j) of O^T the key 4 g + r, whose weight is register r of the scores.
template <int D, bool PAST>
struct Few<float, D, PAST> {
    static constexpr int KEYS = 16, TILES = 1, KS = D / 16, VD = D / 16;
    f32x4_t q[KS], k[1][KS];
    float v[4][VD];
    __device__ __forceinline__ void load_q(const float* p, int g, float*) {
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const f32x4_t*>(p + 16 * s + 4 * g);
    }
    __device__ __forceinline__ void load_k(int, const float* row, int g) {
#pragma unroll
        for (int s = 0; s < KS; ++s) k[0][s] = read_row<f32x4_t, PAST>(row + 16 * s + 4 * g);
    }
    __device__ __forceinline__ void load_v(int, int r, const float* row, int c) {
        const float* p = row + VD * c;
        if constexpr (VD % 4 == 0) {
#pragma unroll
            for (int w = 0; w < VD; w += 4) {
                const f32x4_t x = read_row<f32x4_t, PAST>(p + w);
#pragma unroll
                for (int u = 0; u < 4; ++u) v[r][w + u] = x[u];
            }
        } else {
#pragma unroll
            for (int w = 0; w < VD; w += 2) {
                const f32x2_t x = read_row<f32x2_t, PAST>(p + w);
                v[r][w] = x[0]; v[r][w + 1] = x[1];
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
    typedef f32x4_t frag_t;
    typedef frag_t weights_t;
    static __device__ __forceinline__ weights_t weights(const float (&p)[4]) { return f32x4_t{p[0], p[1], p[2], p[3]}; }
    __device__ __forceinline__ void accumulate(f32x4_t (&acc)[VD], frag_t p) const {
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
    __device__ __forceinline__ void accumulate_odd(f32x4_t (&acc)[VD], frag_t p, uint32_t seen) const {
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

// What a row's sums are divided by, as a factor.  No weight at all: a row that sees nothing is to give zeros; one that sees only scores of
// -infinity has no softmax.
__device__ __forceinline__ float inverse_of(float total, bool sees) { return total == 0.f ? sees ? __builtin_nanf("") : 0.f : 1.f / total; }

template <class T> __device__ __forceinline__ void store4(T* p, f32x4_t v);
template <> __device__ __forceinline__ void store4<float>(float* p, f32x4_t v) { *reinterpret_cast<f32x4_t*>(p) = v; }
template <> __device__ __forceinline__ void store4<uint16_t>(uint16_t* p, f32x4_t v) {
    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4_t*>(p) = bf16x4_t{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
}

constexpr int kFewWaves = 4;

// One wave walks the keys `key`, key + stride, ... up to `last` of a tile of 16 columns, KEYS at a time: the running maximum (of log2), the sum of
// weights over the lane's own keys and the weighted sum of the values.  limit: last key this lane's column sees, least: the least of the tile.
template <class T, int D, bool PAST>
__device__ __forceinline__ void walk_keys(const AttnArgs& a, int seq, int kvh, int key, int stride, int last, int least, int limit, int g, int c,
                                          Few<T, D, PAST>& f, f32x4_t (&acc)[Few<T, D, PAST>::VD], float& m, float& l, bool& bad_page) {
    typedef Few<T, D, PAST> F;
    constexpr int VD = F::VD, SLOTS = 4 * F::TILES;
    const int shift = a.kv.page_shift, in_page = (1 << shift) - 1;
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
    if (key > last) return;
    int page[F::TILES];
#pragma unroll
    for (int t = 0; t < F::TILES; ++t) page[t] = page_of(key + 16 * t);
    load_k(key, page);
    load_v(key, page);
    for (; key <= last; key += stride) {
        const int next = key + stride;
        if (next <= last) {
#pragma unroll
            for (int t = 0; t < F::TILES; ++t) page[t] = page_of(next + 16 * t);
        }
        float s[SLOTS];
#pragma unroll
        for (int t = 0; t < F::TILES; ++t) {
            const f32x4_t x = f.scores(t);
#pragma unroll
            for (int r = 0; r < 4; ++r) s[4 * t + r] = x[r] * a.scale2s;
        }
        if (next <= last) load_k(next, page);
        // hidden: keys beyond what the column sees (uniform test first: most steps have none)
        const bool partly = key + F::KEYS - 1 > min(least, last);
        uint32_t seen = ~0u;
        if (partly) {
            int upto = min(limit, last);
            asm volatile("" : "+v"(upto));                   // a branch: as selects it would cost every step
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
#pragma unroll
        for (int r = 0; r < SLOTS; ++r) s[r] = __builtin_amdgcn_exp2f(s[r] - m_safe);
        const typename F::weights_t w = F::weights(s);
        l *= alpha;
#pragma unroll
        for (int r = 0; r < SLOTS; ++r) l += s[r];
        if (__ballot(alpha != 1.f)) {
#pragma unroll
            for (int j = 0; j < VD; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[j][r] *= alpha;
        }
        if (partly && __ballot(f.odd_values())) f.accumulate_odd(acc, w, seen);
        else f.accumulate(acc, w);
        if (next <= last) load_v(next, page);
    }
}

// A workgroup: one tile of 16 columns of one sequence and key head, one chunk of the cache, whose keys its waves share out; or (by_head) one
// sequence and four neighbouring key heads, one to a wave.
template <class T, int D, bool PAST>
__global__ __launch_bounds__(64 * kFewWaves, sizeof(T) == 2 || D < 256 ? 2 : 1)
void attention_few_kernel(AttnArgs a) {
    typedef Few<T, D, PAST> F;
    constexpr int VD = F::VD;
    __shared__ __attribute__((aligned(16))) float joined_o[kFewWaves][16][D + 4];
    __shared__ float joined_ml[kFewWaves][16][2];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = a.n_chunks == 1 ? blockIdx.x : blockIdx.x / a.n_chunks, chunk = blockIdx.x - tile * a.n_chunks;
    const int heads = a.by_head ? kFewWaves : 1;             // key heads of a workgroup
    const int first_kvh = blockIdx.y * heads, kvh = first_kvh + (a.by_head ? wave : 0), seq = blockIdx.z;
    const NewRows rows = rows_of_sequence(a.b, seq);
    const int columns = rows.count * a.group;
    if (tile * 16 >= columns) return;
    const int kv_len = length_of_sequence(a.b, seq), kv_end = min(kv_len, a.b.max_kv_len);

    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int col = tile * 16 + c;
    const bool live = col < columns;
    const int my = live ? col : columns - 1;                 // dead columns repeat the last one
    const int i = my / a.group, head = kvh * a.group + my - i * a.group;
    const int row = rows.first + i;
    auto limit_of = [&](int i) { return min(a.causal ? kv_len - rows.count + i : kv_len - 1, kv_end - 1); };
    const int limit = limit_of(i);                           // last key this column sees
    // the last column sees most, the first one least
    const int most = __builtin_amdgcn_readlane(limit, 15), least = __builtin_amdgcn_readfirstlane(limit);
    const int begin = chunk * a.chunk, end = min(begin + a.chunk, most + 1);
    if (begin >= end && a.n_chunks > 1) return;              // the join does not look at it

    F f;
    f.load_q((const T*)a.Q + row * a.ldq + (int64_t)head * D, g, &joined_o[wave][0][0]);
    f32x4_t acc[VD];
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -__builtin_inff(), l = 0.f;
    bool bad_page = false;

    walk_keys<T, D, PAST>(a, seq, kvh, a.by_head ? begin : begin + wave * F::KEYS, a.by_head ? F::KEYS : F::KEYS * kFewWaves, end - 1, least, limit, g, c, f, acc, m,
                          l, bad_page);
    l = across_groups_sum(l);
    if (bad_page) l = __builtin_nanf("");

    // acc[j][r]: component VD (4 g + r) + j of column c
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < VD; ++j) joined_o[wave][c][VD * (4 * g + r) + j] = acc[j][r];
    if (g == 0) { joined_ml[wave][c][0] = m; joined_ml[wave][c][1] = l; }
    __syncthreads();
    for (int e = threadIdx.x; e < heads * 16 * (D / 4); e += 64 * kFewWaves) {
        const int k16 = e / (D / 4), cc = k16 & 15, hd = k16 >> 4, x = 4 * (e - k16 * (D / 4));
        const int first_head = (first_kvh + hd) * a.group;
        const int from = a.by_head ? hd : 0, to = a.by_head ? hd + 1 : kFewWaves;             // the waves that have parts of this column
        const int cl = tile * 16 + cc;
        if (cl >= columns) continue;
        float top = joined_ml[from][cc][0];
        for (int w = from + 1; w < to; ++w) top = fmaxf(top, joined_ml[w][cc][0]);
        const float safe = top == -__builtin_inff() ? 0.f : top;
        float total = 0.f;
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
        for (int w = from; w < to; ++w) {
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
            const float inv = inverse_of(total, limit_of(ri) >= 0);
#pragma unroll
            for (int u = 0; u < 4; ++u) o[u] *= inv;         // (nothing was added to o where there was no weight)
            store4((T*)a.O + rr * a.ldo + (int64_t)h * D + x, o);
        } else {
            const int64_t item = part_of(a, chunk, seq, ri, h);
            *reinterpret_cast<f32x4_t*>(a.part_o + item * D + x) = o;
            if (x == 0) { a.part_ml[2 * item] = top; a.part_ml[2 * item + 1] = total; }
        }
    }
}

// attention_float_kernel: many columns to a key head, float.  Bound by the matrix instructions and the softmax between them.  A wave has a tile of 16 columns,
// four of them share the keys and values that a workgroup brings into LDS, kFloatKeys at a time, a step ahead: through registers, since the rows' pitch
// is 16 bytes more than they are long (16 lanes read the same piece of 16 rows).  8 x 512 rows, 32 heads of 128: 291 us, 478 with a workgroup to every 16
// columns; 1 x 3000 behind 1000, 32/8 heads: 1133 us = 109 TFLOP/s, of the 154 that a library's product reaches, and 1434.  16 keys at a time 295 and 1163.
constexpr int kFloatWaves = 4, kFloatKeys = 32;
template <int D> constexpr int float_lds() { return 2 * 2 * kFloatKeys * (D + 4) * 4; }        // two steps of K and V

template <int D>
__global__ __launch_bounds__(64 * kFloatWaves, 2)
void attention_float_kernel(AttnArgs a) {
    typedef Few<float, D, false> F;
    constexpr int VD = F::VD, KT = kFloatKeys, TILES = KT / 16, PITCH = D + 4, THREADS = 64 * kFloatWaves, VECS = KT * (D / 4) / THREADS;
    static_assert(KT * (D / 4) % THREADS == 0, "");
    extern __shared__ __attribute__((aligned(16))) float tiles[];
    int set, item;
    if (!deal_to_dies(blockIdx.x, a.col_tiles * a.n_chunks, a.b.n_seqs * a.kv.n_kv_heads, &set, &item)) return;
    const int kvh = set % a.kv.n_kv_heads, seq = set / a.kv.n_kv_heads, chunk = item % a.n_chunks;
    const int tile = a.col_tiles - 1 - item / a.n_chunks;    // the columns that see most first
    const NewRows rows = rows_of_sequence(a.b, seq);
    const int columns = rows.count * a.group, first_col = tile * 16 * kFloatWaves;
    if (first_col >= columns) return;
    const int kv_len = length_of_sequence(a.b, seq), kv_end = min(kv_len, a.b.max_kv_len);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    auto limit_of = [&](int col) { return min(a.causal ? kv_len - rows.count + col / a.group : kv_len - 1, kv_end - 1); };
    const int begin = chunk * a.chunk, end = min(begin + a.chunk, limit_of(min(first_col + 16 * kFloatWaves, columns) - 1) + 1);
    if (begin >= end && a.n_chunks > 1) return;              // the join does not look at it
    const int last = end - 1, steps = end > begin ? (end - begin + KT - 1) / KT : 0;

    const int wave_col = first_col + 16 * wave;
    const bool awake = wave_col < columns;
    const int col = min(wave_col + c, columns - 1), i = col / a.group, head = kvh * a.group + col - i * a.group;     // dead columns repeat the last one
    const int64_t row = rows.first + i;
    const int limit = limit_of(col);
    const int most = awake ? min(__builtin_amdgcn_readlane(limit, 15), last) : -1, least = __builtin_amdgcn_readfirstlane(limit);
    F f;
    f.load_q((const float*)a.Q + row * a.ldq + (int64_t)head * D, g, nullptr);
    f32x4_t acc[VD];
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -__builtin_inff(), l = 0.f;
    bool bad_page = false;

    // this thread's pieces of a step: rows beyond the last key are read as that one
    const int shift = a.kv.page_shift, in_page = (1 << shift) - 1;
    const int32_t* table = a.b.page_table + seq * a.b.table_ld;
    f32x4_t stage[2][VECS];
    auto send = [&](int step) {
#pragma unroll
        for (int u = 0; u < VECS; ++u) {
            const int e = threadIdx.x + u * THREADS, r = e / (D / 4), x = 4 * (e - r * (D / 4));
            const int key = min(begin + step * KT + r, last);
            const int page = table[key >> shift];
            const bool good = page >= 0 && page < a.kv.n_pages;
            bad_page |= !good;
            const int64_t at = (good ? page : 0) * a.kv.page_stride + kvh * a.kv.head_stride + (key & in_page) * a.kv.row_stride + x;
            stage[0][u] = *reinterpret_cast<const f32x4_t*>((const float*)a.kv.k + at);
            stage[1][u] = *reinterpret_cast<const f32x4_t*>((const float*)a.kv.v + at);
        }
    };
    auto put = [&](int step) {
        float* to = tiles + (step & 1) * 2 * KT * PITCH;
#pragma unroll
        for (int u = 0; u < VECS; ++u) {
            const int e = threadIdx.x + u * THREADS, r = e / (D / 4), x = 4 * (e - r * (D / 4));
            *reinterpret_cast<f32x4_t*>(to + r * PITCH + x) = stage[0][u];
            *reinterpret_cast<f32x4_t*>(to + KT * PITCH + r * PITCH + x) = stage[1][u];
        }
    };
    if (steps > 0) { send(0); put(0); }
    __syncthreads();
    for (int step = 0; step < steps; ++step) {
        if (step + 1 < steps) send(step + 1);
        const float* from = tiles + (step & 1) * 2 * KT * PITCH;
        const int key = begin + step * KT;
        if (key <= most) {
            float s[4 * TILES];
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                f.load_k(0, from + (16 * t + c) * PITCH, g);
                const f32x4_t x = f.scores(0);
#pragma unroll
                for (int r = 0; r < 4; ++r) s[4 * t + r] = x[r] * a.scale2s;
            }
            const bool partly = key + KT - 1 > min(least, last);
            uint32_t seen = ~0u;
            if (partly) {
                int upto = min(limit, last);
                asm volatile("" : "+v"(upto));               // a branch: as selects it would cost every step
                seen = 0;
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const bool sees = key + 16 * t + 4 * g + r <= upto;
                        s[4 * t + r] = sees ? s[4 * t + r] : -__builtin_inff();
                        seen |= (uint32_t)sees << (4 * t + r);
                    }
            }
            float top = s[0];
#pragma unroll
            for (int r = 1; r < 4 * TILES; ++r) top = fmaxf(top, s[r]);
            const float m_new = fmaxf(m, across_groups_max(top)), m_safe = m_new == -__builtin_inff() ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m - m_safe);
            m = m_new;
            l *= alpha;
            if (__ballot(alpha != 1.f)) {
#pragma unroll
                for (int j = 0; j < VD; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[j][r] *= alpha;
            }
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
#pragma unroll
                for (int u = 0; u < 4; ++u) f.load_v(0, u, from + (KT + 16 * t + 4 * g + u) * PITCH, c);
                f32x4_t w;
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = __builtin_amdgcn_exp2f(s[4 * t + r] - m_safe);
#pragma unroll
                for (int r = 0; r < 4; ++r) l += w[r];
                if (partly && __ballot(f.odd_values())) f.accumulate_odd(acc, w, seen >> (4 * t));
                else f.accumulate(acc, w);
            }
        }
        if (step + 1 < steps) put(step + 1);                 // into the half that nobody has read since the last barrier
        __syncthreads();
    }
    const bool any_bad = __syncthreads_or(bad_page);
    float total = across_groups_sum(l);
    if (any_bad) total = __builtin_nanf("");
    if (wave_col + c >= columns) return;
    const bool whole = a.n_chunks == 1;
    const float by = whole ? inverse_of(total, limit >= 0) : 1.f;
    const int64_t part = part_of(a, chunk, seq, i, head);
    float* out = whole ? (float*)a.O + row * a.ldo + (int64_t)head * D : a.part_o + part * D;
    // acc[j][r]: component VD (4 g + r) + j
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < VD; j += 2) *reinterpret_cast<f32x2_t*>(out + VD * (4 * g + r) + j) = f32x2_t{acc[j][r] * by, acc[j + 1][r] * by};
    if (!whole && g == 0) { a.part_ml[2 * part] = m; a.part_ml[2 * part + 1] = total; }
}

// attention_prompt_kernel: many columns to a key head, bfloat16.  Bound by the matrix instructions and, beside them, by the exponentials.  A
// workgroup takes kPromptWaves x 32 columns and walks the keys kPromptKeys at a time; K and V come into LDS once for all its waves, by
// direct-to-LDS fetches a step ahead.  v_mfma_f32_32x32x16_bf16: lane (h, c) = (lane / 32, lane % 32); S^T of 32 keys leaves in register r of
// the lane column c and key 8 (r / 4) + 4 h + r % 4, so registers 8 t ... 8 t + 7 are keys 16 t + {4 h + 0..3, 8 + 4 h + 0..3}: the B operand of step t
// of O^T, if A = V^T takes its keys in that order - two transposing reads of four rows each.
// A wave works on three groups of 32 keys at once, whose instructions depend on nothing of each other: the scores of the next group and the
// weighted sum of the last one (matrix pipe) beside the weights of the present one (vector pipe).
// 6000 rows behind 2000, 32/8 heads of 128: 472 us on one chip, 477 to 490 on others = 1.00 to 1.04 PFLOP/s, at 1.83 GHz under the power limit; a library's product
// of 8192^3 reaches 1.24.  Of 507 us (an earlier step) the fetches were 73, maximum and masks 114, the reads of LDS 159, each taken out alone.
// 8 prompts of 301 to 512 rows, 32 heads of 128: 38 to 43 us = 0.26 PFLOP/s of what causal rows see: 12 us for one row of keys, and tiles that end early.
constexpr int kPromptWaves = 4;
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

// lds_addr must be wave-uniform (it travels in M0); lane l's 16 bytes land at lds_addr + 16 l
__device__ __forceinline__ void fetch16(uint32_t offset, const void* base, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(offset), "s"(base), "s"(lds_addr) : "memory", "m0");
}

constexpr int kPromptKeys = 64;
template <int D> constexpr int prompt_lds() { return 2 * 2 * kPromptKeys * D * 2; }        // two steps of K, then two of V

// Where the 16-byte chunk c of row r lies in its row.  K: 16 lanes read the same chunk of 16 rows in a row; V: half a wave reads four chunks of
// four rows.  Either has to meet all 64 banks: 16 chunks of 16 bytes are a round of them.
template <int D> __device__ __forceinline__ int k_pos(int r, int c) {
    if constexpr (D == 64) return c ^ ((r >> 1) & 7);
    else if constexpr (D == 96) return (c + ((r >> 2) & 3)) % 12;
    else return c ^ (r & 15);
}
template <int D> __device__ __forceinline__ int k_chunk(int r, int p) {
    if constexpr (D == 96) return (p + 12 - ((r >> 2) & 3)) % 12;
    else return k_pos<D>(r, p);
}
template <int D> __device__ __forceinline__ int v_pos(int r, int c) {          // its own inverse
    if constexpr (D == 64) return c ^ ((r & 2) << 1);
    else if constexpr (D == 96) return c;
    else return c ^ ((r & 3) << 2);
}

// 0 times a value that is not finite is NaN also in columns that do not see its key.  Such values are rare, and they show in the result: a
// workgroup that finds any there walks its keys once more (ODD) with zeros in their place and adds them to the columns that see them.
// So it does where a base ended far out.  An exponent is s scale2 - base in one rounding, and the base is the rounding of one such product: from 2^32 on
// they can stand 2^8 apart, and the largest weight of a column leaves float's range.  ODD rounds the product of such columns first.  (A base that was far
// below zero and came back has left infinities or nothing: either is found or does not matter.)
template <int D> struct PromptNotes {
    int odd, bad;                                            // results that are not finite or a base far out, page numbers outside the cache
    int first[2][D];                                         // per component the first key whose value is +infinity (-infinity), NaN: both
};

constexpr float kFarBase = 0x1p28f;                         // products of this size are rounded by 16 at most
__device__ __forceinline__ float rounded_exponent(float score, float scale2, float base) {
#pragma clang fp contract(off)
    return score * scale2 - base;
}

// One tile of columns of a sequence and key head, one chunk of the cache.  True: to be done again with ODD.
template <int D, bool ODD>
__device__ __forceinline__ bool prompt_tile(const AttnArgs& a, int seq, int kvh, int chunk, int tile, PromptNotes<D>& notes) {
    constexpr int KT = kPromptKeys, KS = D / 16, DT = D / 32, PITCH = 2 * D, SLOT = KT * PITCH, WIDE = 32 * kPromptWaves;
    constexpr int ROWS = KT / kPromptWaves;                  // rows a wave fetches
    constexpr int NF = ROWS * PITCH / 1024;                  // fetches of 1 KB for them
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    int thread = threadIdx.x;
    asm volatile("" : "+v"(thread));                         // another tile's or pass's addresses are worked out again: kept, they take registers
    const NewRows rows = rows_of_sequence(a.b, seq);
    const int columns = rows.count * a.group, first_col = tile * WIDE;
    if (first_col >= columns) return false;
    const int kv_len = length_of_sequence(a.b, seq), kv_end = min(kv_len, a.b.max_kv_len);
    const int lane = thread & 63, h = lane >> 5, c = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(thread >> 6);

    auto limit_of = [&](int col) { return min(a.causal ? kv_len - rows.count + col / a.group : kv_len - 1, kv_end - 1); };
    const int wg_most = limit_of(min(first_col + WIDE, columns) - 1);
    const int begin = chunk * a.chunk, end = min(begin + a.chunk, wg_most + 1);
    if (begin >= end && a.n_chunks > 1) return false;
    const int last = end - 1, steps = end > begin ? (end - begin + KT - 1) / KT : 0;

    // fetches: this wave's 16 rows of a step, 1 KB at a time; the keys of 16 rows share a page
    const uint32_t lds_base = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)lds);
    const uint32_t my_rows = lds_base + wave * ROWS * PITCH;
    uint32_t k_off[NF], v_off[NF];
    const int shift = a.kv.page_shift, in_page = (1 << shift) - 1;
    const int32_t* table = a.b.page_table + seq * a.b.table_ld;
    const uint16_t* k_head = (const uint16_t*)a.kv.k + kvh * a.kv.head_stride;
    const uint16_t* v_head = (const uint16_t*)a.kv.v + kvh * a.kv.head_stride;
    bool bad_page = false;
    auto group_of = [&](int step) { return min(begin + step * KT + wave * ROWS, last & ~(ROWS - 1)); };
    // (a vector load: beside a scalar one every wait for LDS would be a wait for it as well)
    auto load_page = [&](int step) { return table[(group_of(min(step, steps - 1)) + (lane >> 6)) >> shift]; };
    auto rows_at = [&](int step, int page) {                 // values from the start of a head to these rows
        const bool good = page >= 0 && page < a.kv.n_pages;
        bad_page |= !good;
        return (good ? page : 0) * a.kv.page_stride + (group_of(step) & in_page) * a.kv.row_stride;
    };
    // rows beyond the last key are fetched as that key's (they are masked, but 0 times what lies there might be NaN): in the last step
    auto trim = [&](uint32_t (&off)[NF], int step) {
        const int there = last - group_of(step);             // last row of the 16 that is there
        if (step < steps - 1 || there >= ROWS - 1) return;
#pragma unroll
        for (int i = 0; i < NF; ++i) off[i] -= (uint32_t)(max((i * 1024 + lane * 16) / PITCH - there, 0) * (int)a.kv.row_stride) * 2;
    };

    // this wave's columns, one to a lane (and to the lane 32 further on)
    const int wave_col = first_col + wave * 32;
    const bool awake = wave_col < columns;
    const int most = awake ? min(limit_of(min(wave_col + 32, columns) - 1), last) : -1, least = awake ? limit_of(wave_col) : -1;
    const int my_steps = most >= begin ? (most - begin) / KT + 1 : 0;
    const int col = min(wave_col + c, columns - 1);          // dead columns repeat the last one
    const int limit = limit_of(col);
    auto row_of = [&](int x) { return rows.first + x / a.group; };
    auto head_of = [&](int x) { return kvh * a.group + x % a.group; };
    bf16x8_t q[KS];
    {
        const uint16_t* p = (const uint16_t*)a.Q + row_of(col) * a.ldq + (int64_t)head_of(col) * D + 8 * h;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            u32x4_t w = *reinterpret_cast<const u32x4_t*>(p + 16 * s);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] ^= a.flip;
            q[s] = __builtin_bit_cast(bf16x8_t, w);
        }
    }
    f32x16_t acc[DT], s[2], zero;
    bf16x8_t p[2][2];                                        // weights of two groups of 32 keys
    float m, base, l;                                        // the maximum that weights are relative to, times scale2 as a whole number, their sum
    const float slack = 8.f / a.scale2;
#pragma unroll
    for (int r = 0; r < 16; ++r) zero[r] = 0.f;

    // reads of a step: 32 rows of K from row c on, four rows of V and eight below them; a row's chunks lie alike every 16 rows
    typedef uint8_t __attribute__((address_space(3))) * lds_ptr_t;
    typedef const bf16x8_t __attribute__((address_space(3))) * k_ptr_t;
    typedef s16x4_t __attribute__((address_space(3))) * v_ptr_t;
    const int s16 = lane & 15, nh = (lane >> 4) & 1;
    lds_ptr_t k_at[KS], v_at[DT];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) k_at[ks] = (lds_ptr_t)lds + (c * PITCH + 16 * k_pos<D>(c, 2 * ks + h));
#pragma unroll
    for (int t = 0; t < DT; ++t) {
        const int r = 4 * h + (s16 >> 2);
        v_at[t] = (lds_ptr_t)lds + (3 * SLOT + r * PITCH + 16 * v_pos<D>(r, 4 * t + 2 * nh + ((s16 >> 1) & 1)) + 8 * (s16 & 1));
    }
    // The matrix instructions of a group, in this order: KS for the scores of 32 keys, whose rows begin `kfrom` bytes into the slots of K, then
    // KS for the weighted values of 32 others, `vfrom` bytes into those of V.  Each has one fragment to read, AHEAD instructions before.
    constexpr int N = 2 * KS, AHEAD = 3;
    auto read_k = [&](int ks, int kfrom) { return *(k_ptr_t)(k_at[ks] + (kfrom)); };
    auto read_v = [&](int j, int vfrom) {                    // V^T of component block j % DT and 16 keys
        s16x8_t f;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v_ptr_t)(v_at[j % DT] + (vfrom + (16 * (j / DT) + 8 * half) * PITCH)));
#pragma unroll
            for (int e = 0; e < 4; ++e) f[4 * half + e] = x[e];
        }
        return __builtin_bit_cast(bf16x8_t, f);
    };
    // Both go from slot to slot in the middle of a step: K then reads the next step's, V this one's.
    auto turn_addresses = [&](int by) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) k_at[ks] += by;
#pragma unroll
        for (int t = 0; t < DT; ++t) v_at[t] -= by;
    };
    // The largest of 16 scores, in four pieces.
    float top2[2], top = 0.f;
    auto top_piece = [&](auto ic, const f32x16_t& x) {
        constexpr int i = decltype(ic)::value;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if constexpr (i == 0) top2[u] = fmaxf(fmaxf(x[8 * u], x[8 * u + 1]), x[8 * u + 2]);
            else if constexpr (i < 3) top2[u] = fmaxf(fmaxf(top2[u], x[8 * u + 2 * i + 1]), x[8 * u + 2 * i + 2]);
        }
        if constexpr (i == 3) top = fmaxf(fmaxf(top2[0], x[7]), fmaxf(top2[1], x[15]));
    };
    // Weights of the 32 keys from `key` on, whose scores are s[G] and whose largest score is top; beside them the scores of the next group, their
    // largest one, and the weighted values of the one before.  The order is kept as it stands here (sched_barrier): a matrix instruction, and
    // while it runs a read, a share of the weights and extra(slot).
    auto group = [&](auto g, auto kfrom, auto vfrom, int key, auto&& extra) {
        constexpr int G = decltype(g)::value, KFROM = decltype(kfrom)::value, VFROM = decltype(vfrom)::value;
        bf16x8_t frag[AHEAD + 1];
        static_for<AHEAD>([&](auto ic) { frag[decltype(ic)::value] = read_k(decltype(ic)::value, KFROM); });
        if (key + 31 > min(least, last)) {
            int upto = min(limit, last) - key;
            asm volatile("" : "+v"(upto));                   // a branch: as selects it would cost every step
#pragma unroll
            for (int r = 0; r < 16; ++r) s[G][r] = 8 * (r >> 2) + 4 * h + (r & 3) <= upto ? s[G][r] : -__builtin_inff();
            static_for<4>([&](auto ic) { top_piece(ic, s[G]); });
        }
        // any base that leaves the weights in range gives the same quotient: it moves only where a column's maximum has grown by 2^8, and by
        // whole powers of two, which scale everything there is without a rounding
        if (__ballot(top > m + slack)) {
            const float m_new = fmaxf(m, fmaxf(top, __shfl_xor(top, 32, 64)));
            const float base_new = m_new == -__builtin_inff() ? 0.f : rintf(m_new * a.scale2);       // nothing seen yet: all weights are 0
            const float alpha = m == -__builtin_inff() ? 0.f : ldexpf(1.f, (int)fmaxf(base - base_new, -200.f));
            m = m_new;
            base = base_new;
            l *= alpha;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[t][r] *= alpha;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int e = 0; e < 8; ++e) p[G ^ 1][ks][e] = (__bf16)((float)p[G ^ 1][ks][e] * alpha);
        }
        float from = base;
        if constexpr (ODD) {
            const bool far = fabsf(base) >= kFarBase;
            if (__ballot(far)) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[G][r] = far ? rounded_exponent(s[G][r], a.scale2, base) / a.scale2 : s[G][r];
                from = far ? 0.f : base;
            }
        }
        float part[2] = {0.f, 0.f};
        __builtin_amdgcn_sched_barrier(0);
        static_for<N>([&](auto ic) {
            constexpr int i = decltype(ic)::value, ahead = i + AHEAD;
            if constexpr (ahead < KS) frag[ahead % (AHEAD + 1)] = read_k(ahead, KFROM);
            else if constexpr (ahead < N) frag[ahead % (AHEAD + 1)] = read_v(ahead - KS, VFROM);
            if constexpr (i < KS) s[G ^ 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % (AHEAD + 1)], q[i], i == 0 ? zero : s[G ^ 1], 0, 0, 0);
            else acc[(i - KS) % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % (AHEAD + 1)], p[G ^ 1][(i - KS) / DT], acc[(i - KS) % DT], 0, 0, 0);
            static_for<(i + 1) * 16 / N - i * 16 / N>([&](auto rc) {
                constexpr int r = i * 16 / N + decltype(rc)::value;
                const float w = __builtin_amdgcn_exp2f(s[G][r] * a.scale2 - from);
                s[G][r] = w;
                if constexpr (r % 2 == 0) {
                    asm volatile("" : "+v"(s[G][r]));        // here: extra() may hold branches, behind which it would sink to its use
                } else {
                    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
                    const bf16x2_t pair = {(__bf16)s[G][r - 1], (__bf16)w};
                    p[G][r >> 3][(r & 7) - 1] = pair[0];
                    p[G][r >> 3][r & 7] = pair[1];
                    part[(r >> 1) & 1] = add_pair(__builtin_bit_cast(uint32_t, pair), part[(r >> 1) & 1]);
                    asm volatile("" : "+v"(part[(r >> 1) & 1]));
                }
            });
            // (the scores are there two instructions after the last of them)
            constexpr int j = i - KS - 2, SPAN = KS - 2;
            if constexpr (j >= 0) static_for<(j + 1) * 4 / SPAN - j * 4 / SPAN>([&](auto x) { top_piece(std::integral_constant<int, j * 4 / SPAN + decltype(x)::value>{}, s[G ^ 1]); });
            extra(ic);
            __builtin_amdgcn_sched_barrier(0);
        });
        l += part[0] + part[1];
        asm volatile("" :: "v"(p[G][0]), "v"(p[G][1]), "v"(s[G ^ 1]), "v"(l), "v"(top));      // here, and not where they are used next
    };
    constexpr std::integral_constant<int, 0> c0{};
    constexpr std::integral_constant<int, 1> c1{};
    constexpr std::integral_constant<int, 0> first{};                // where the two groups of a step begin in a slot
    constexpr std::integral_constant<int, 32 * PITCH> second{};

    if constexpr (ODD) {
        for (int x = thread; x < 2 * D; x += 64 * kPromptWaves) (&notes.first[0][0])[x] = 0x7FFFFFFF;
    } else if (thread == 0) {
        notes.odd = notes.bad = 0;
    }
    m = -__builtin_inff();
    base = l = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = zero;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[1][0][e] = p[1][1][e] = (__bf16)0.f;
    // nothing comes before the first group: no weights, and zeros in the place of its values
    for (int x = thread * 16; x < 32 * PITCH; x += 64 * kPromptWaves * 16) *reinterpret_cast<u32x4_t*>(lds + 3 * SLOT + 32 * PITCH + x) = u32x4_t{0, 0, 0, 0};
    int page = 0;                                        // in a lane's register: of the step three further on
    int64_t k_rows = 0, v_rows = 0;                      // where the rows of the next fetches begin
#pragma unroll
    for (int i = 0; i < NF; ++i) {
        const int at = i * 1024 + lane * 16, r = at / PITCH, x = (at - r * PITCH) / 16, rr = wave * ROWS + r;
        k_off[i] = (uint32_t)(r * (int)a.kv.row_stride + 8 * k_chunk<D>(rr, x)) * 2;
        v_off[i] = (uint32_t)(r * (int)a.kv.row_stride + 8 * v_pos<D>(rr, x)) * 2;
    }
    if (steps > 0) {
        const int page0 = load_page(0), page1 = load_page(1);
        page = load_page(2);
        v_rows = rows_at(0, __builtin_amdgcn_readfirstlane(page0));
        trim(k_off, 0);
#pragma unroll
        for (int i = 0; i < NF; ++i) fetch16(k_off[i], k_head + v_rows, my_rows + i * 1024);
        if (steps > 1) {
            k_rows = rows_at(1, __builtin_amdgcn_readfirstlane(page1));
            trim(k_off, 1);
#pragma unroll
            for (int i = 0; i < NF; ++i) fetch16(k_off[i], k_head + k_rows, my_rows + SLOT + i * 1024);
        }
        trim(v_off, 0);
#pragma unroll
        for (int i = 0; i < NF; ++i) fetch16(v_off[i], v_head + v_rows, my_rows + 2 * SLOT + i * 1024);
        if (steps > 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(2 * NF) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(NF) : "memory");
        __builtin_amdgcn_s_barrier();
    }
    int step = 0;
    // between the two groups of a step: its V and the next step's K are there
    auto turn = [&] {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        if constexpr (ODD) {
            // the values that are not finite go, and per component the first key that had one is kept
            for (int x = thread * 16; x < SLOT; x += 64 * kPromptWaves * 16) {
                const int r = x / PITCH, d = 8 * v_pos<D>(r, (x - r * PITCH) / 16);
                s16x8_t* where = reinterpret_cast<s16x8_t*>(lds + (2 + (step & 1)) * SLOT + x);
                s16x8_t v = *where;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if ((v[e] & 0x7F80) != 0x7F80) continue;
                    const bool nan = v[e] & 0x7F;
                    if (nan || v[e] > 0) atomicMin(&notes.first[0][d + e], begin + step * KT + r);
                    if (nan || v[e] < 0) atomicMin(&notes.first[1][d + e], begin + step * KT + r);
                    v[e] = 0;
                }
                *where = v;
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
        }
    };
    // what follows it: V of the next step and K of the one after are sent for, in 1 + 2 NF pieces
    auto send = [&](auto ic) {
        constexpr int i = decltype(ic)::value;
        const int at = step & 1;
        if constexpr (i == 0) {
            if (step + 1 < steps) {
                v_rows = k_rows;
                trim(v_off, step + 1);
                if (step + 2 < steps) {
                    k_rows = rows_at(step + 2, __builtin_amdgcn_readfirstlane(page));
                    trim(k_off, step + 2);
                }
                page = load_page(step + 3);
            }
        } else if constexpr (i <= NF) {
            if (step + 1 < steps) fetch16(v_off[i - 1], v_head + v_rows, my_rows + (3 - at) * SLOT + (i - 1) * 1024);
        } else if constexpr (i <= 2 * NF) {
            if (step + 2 < steps) fetch16(k_off[i - 1 - NF], k_head + k_rows, my_rows + at * SLOT + (i - 1 - NF) * 1024);
        }
    };
    // Behind the last step there is nothing to score: what its second group multiplies beside its weights is not used.
    if (my_steps > 0) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_k(ks, 0), q[ks], ks == 0 ? zero : s[0], 0, 0, 0);
        static_for<4>([&](auto ic) { top_piece(ic, s[0]); });
        do {
            group(c0, second, second, begin + step * KT, [](auto) {});
            turn();
            turn_addresses(step & 1 ? -SLOT : SLOT);
            group(c1, first, first, begin + step * KT + 32, send);
        } while (++step < my_steps);
#pragma unroll
        for (int j = 0; j < KS; ++j) acc[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_v(j, 32 * PITCH), p[1][j / DT], acc[j % DT], 0, 0, 0);
    }
    for (; step < steps; ++step) {                       // for the other waves
        turn();
        static_for<1 + 2 * NF>([&](auto ic) { send(ic); });
    }
    if constexpr (!ODD) {
        bool odd = fabsf(base) >= kFarBase;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) odd |= (__float_as_uint(acc[t][r]) & 0x7F800000u) == 0x7F800000u;
        __syncthreads();
        if (odd) notes.odd = 1;
        if (bad_page) notes.bad = 1;                         // any wave may have met it
        __syncthreads();
        if (notes.odd) return true;
    }
    if (wave_col + c >= columns) return false;
    int my_col = wave_col + c;
    asm volatile("" : "+v"(my_col));                         // (row and head are worked out again: kept, they take registers the loop needs)
    const int row = row_of(my_col), head = head_of(my_col);
    const bool whole = a.n_chunks == 1;
    float total = l + __shfl_xor(l, 32, 64);
    if (notes.bad) total = __builtin_nanf("");
    const float by = whole ? inverse_of(total, limit >= 0) : 1.f;       // (without weights acc is 0: what was not finite is out of it by now)
    const int64_t part = part_of(a, chunk, seq, my_col / a.group, head);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int x = 32 * t + 8 * e + 4 * h;
            f32x4_t o;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                o[u] = acc[t][4 * e + u] * by;
                if (ODD) o[u] += (notes.first[0][x + u] <= limit ? __builtin_inff() : 0.f) - (notes.first[1][x + u] <= limit ? __builtin_inff() : 0.f);
            }
            if (whole) store4((uint16_t*)a.O + row * a.ldo + (int64_t)head * D + x, o);
            else *reinterpret_cast<f32x4_t*>(a.part_o + part * D + x) = o;
        }
    if (!whole && h == 0) { a.part_ml[2 * part] = total == 0.f ? -__builtin_inff() : base; a.part_ml[2 * part + 1] = total; }
    return false;
}

template <int D>
__global__ __launch_bounds__(64 * kPromptWaves, D < 256 ? 2 : 1)
void attention_prompt_kernel(AttnArgs a) {
    __shared__ PromptNotes<D> notes;
    int set, item;
    const int dealt = a.paired ? (a.col_tiles + 1) / 2 : a.col_tiles;
    if (!deal_to_dies(blockIdx.x, dealt * a.n_chunks, a.b.n_seqs * a.kv.n_kv_heads, &set, &item)) return;
    const int kvh = set % a.kv.n_kv_heads, seq = set / a.kv.n_kv_heads;
    const int chunk = item % a.n_chunks;
    int tile = a.col_tiles - 1 - item / a.n_chunks;          // the columns that see most first
    for (;; tile = a.col_tiles - 1 - tile) {
        if (prompt_tile<D, false>(a, seq, kvh, chunk, tile, notes)) prompt_tile<D, true>(a, seq, kvh, chunk, tile, notes);
        if (!a.paired || 2 * tile < a.col_tiles) break;      // the middle one of an odd number has no partner
        __syncthreads();
    }
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

// Which kernel, and how the cache is cut: chunks of `chunk` keys, n_chunks of them to the longest sequence.
struct Plan { bool prompt, shared, paired, past, by_head; int chunk, n_chunks; int64_t col_tiles, workgroups; };
constexpr int64_t kMostWorkgroups = kMostThreads / 256;      // all kernels here have workgroups of 256
static_assert(64 * kFewWaves <= 256 && 64 * kFloatWaves <= 256 && 64 * kPromptWaves <= 256, "");
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

Plan plan_few(const Attention& o, int64_t columns, int bytes, double* us) {
    Plan p;
    p.prompt = p.shared = p.paired = p.past = p.by_head = false;
    p.col_tiles = (columns + 15) / 16;
    const int64_t tiles = (int64_t)o.batch.n_seqs * o.cache.n_kv_heads * p.col_tiles;
    const int64_t most = (o.batch.max_kv_len + kFewLeast - 1) / kFewLeast;
    int64_t cuts = kFewTarget / tiles;
    cut(&p, o.batch.max_kv_len, cuts < 1 ? 1 : cuts < most ? cuts : most);
    p.workgroups = tiles * p.n_chunks;
    // A large cache that is read once passes the caches by: it would not stay there anyway.  64 x 4096 keys of 32 heads of 128, bf16 (4.3 GB), 711
    // and 621 us (6.9 TB/s), 64 x 512 (0.54 GB) 92 and 84, 16 x 8192 of 2 heads (134 MB) 29.8 and 27.9; 67 MB, which the last-level cache
    // holds, 16.8 and 17.7.
    p.past = p.col_tiles == 1 && 2.0 * bytes * tiles * o.batch.max_kv_len * o.cache.head_dim > 100e6;
    // Where the rows of all heads lie side by side, four heads' are one piece of memory: 64 x 4096 keys of 32 heads of 128, bf16, 714 us with
    // the keys of a head shared out over the waves and 653 with a head to each, 64 x 512 94 and 89; with a head's rows side by side 621 and 622.
    p.by_head = p.n_chunks == 1 && p.col_tiles == 1 && o.cache.n_kv_heads % kFewWaves == 0 && o.cache.head_stride == o.cache.head_dim && tiles / kFewWaves >= kFewTarget;
    if (p.by_head) p.workgroups = tiles / kFewWaves;
    // every tile of 16 columns reads the cache's rows again, from L2 as a rule; a wave's step is a trip to memory
    const double rounds = (double)((p.workgroups + kFewTarget - 1) / kFewTarget);
    const double reads = 4.0 * tiles * o.batch.max_kv_len * o.cache.head_dim / 9e6, trips = rounds * (p.chunk / 128) * 1.5;
    *us = 4.0 * rounds + (reads > trips ? reads : trips) + join_us(o, p);
    return p;
}

// Cuts fill the chip but cost the join, and two workgroups on a CU share its matrix pipes: of the counts that fit, the one that this reckoning
// likes best.  A workgroup takes 5 us until its first weights, then per step of 64 keys 1.3 us alone on its CU (a fetch's way) and 1.1 us
// times the width over 128 of the CU's pipes.  With two workgroups on every CU wherever the columns allowed it (at 256 keys to a chunk) 8 x 128
// rows against 512 keys of 32 heads of 128 took 37 us where one cut less takes 22, against 1024 52 and 40, 2 x 300 rows of 8 heads of 256
// against 3000 77 and 54; 512 rows behind 7680, 32/8 heads, take 86 us cut in four and 95 in two.
Plan plan_prompt(const Attention& o, int64_t columns, double* us) {
    Plan best;
    best.prompt = true;
    best.shared = best.past = best.by_head = false;
    best.col_tiles = (columns + 32 * kPromptWaves - 1) / (32 * kPromptWaves);
    const int64_t sets = (int64_t)o.batch.n_seqs * o.cache.n_kv_heads, tiles = sets * best.col_tiles;
    const int d = o.cache.head_dim, per_cu = d == 256 ? 1 : 2;
    const double bytes = 4.0 * sets * o.batch.max_kv_len * d;
    *us = 1e30;
    int64_t most = kPromptTarget / tiles;
    const int64_t whole = (o.batch.max_kv_len + kPromptLeast - 1) / kPromptLeast;
    most = most < 1 ? 1 : most < whole ? most : whole;
    for (int64_t cuts = 1; cuts <= most; ++cuts) {
        Plan p = best;
        cut(&p, o.batch.max_kv_len, cuts);
        p.workgroups = tiles * p.n_chunks;
        const int64_t slots = kCus * per_cu, rounds = (p.workgroups + slots - 1) / slots;
        const int64_t together = rounds > 1 || p.workgroups > kCus ? per_cu : 1;
        const double pipes = 1.1 * d / 128 * together, step = pipes > 1.3 ? pipes : 1.3;
        double main = (double)rounds * (5.0 + p.chunk / 64 * step);
        if (main < 5.0 + bytes / 5.5e6) main = 5.0 + bytes / 5.5e6;
        const double all = main + join_us(o, p);
        if (all < *us) { *us = all; best.chunk = p.chunk; best.n_chunks = p.n_chunks; best.workgroups = p.workgroups; }
    }
    // Causal rows: the last tile of columns walks the most keys, the first one the fewest.  Where the tiles are more than the chip holds at
    // once but no more than twice that, a workgroup takes a long and a short one: all end together.
    const int64_t pairs = sets * ((best.col_tiles + 1) / 2);
    best.paired = o.causal && best.n_chunks == 1 && best.col_tiles > 1 && best.workgroups > kCus * per_cu && pairs <= kCus * per_cu;
    if (best.workgroups <= kMostWorkgroups) best.workgroups = 8 * (int64_t)dies_slots((int)((best.paired ? (best.col_tiles + 1) / 2 : best.col_tiles) * best.n_chunks), (int)sets);
    return best;
}

// Float: tiles of 64 columns pay where they fill the chip, or where they are long ones (every row sees half of the keys at least) and it takes a cut or two.
// 16 columns to a workgroup and 64, us: heads of 128, 8 x 512 rows 478 and 291 (2048 tiles), 64 x 48 on 200 61 and 50 (512), 16 x 24 on 500, 32/8 heads, 72
// and 55 (256), 4 x 200 on 1000, all seen, 109 and 93 (256), 2 x 512 on 2000 99 and 93 (128); 1 x 2000 148 and 162 (256), 32 x 64 on 300 56 and 61
// (256), 1 x 32 on 4096 20 and 33; of 96, 16 x 33 on 1000, 28/4 heads, 92 and 76 (256), 4 x 378 24 and 43 (192).  Heads of 64, where four of the small ones fit a
// CU, and of 256, where one of either does, stay with 16 columns: of 64 one size was timed, 8 x 200 37 and 41, of 256 8 x 300 on 600 386 and 440 but 4 x 378
// on 600 446 and 365, and no count that tells such calls apart.
bool float_shares(const Attention& o, int64_t columns) {
    const int64_t tiles = (int64_t)o.batch.n_seqs * o.cache.n_kv_heads * ((columns + 16 * kFloatWaves - 1) / (16 * kFloatWaves));
    const bool lengthy = !o.causal || o.batch.max_kv_len >= 2 * (int64_t)o.batch.max_rows;
    return (o.cache.head_dim == 96 || o.cache.head_dim == 128) && ((columns >= 48 && tiles >= 512) || (columns >= 96 && tiles >= 128 && lengthy));
}
Plan plan_float(const Attention& o, int64_t columns) {
    Plan p;
    p.shared = true;
    p.prompt = p.paired = p.past = p.by_head = false;
    p.col_tiles = (columns + 16 * kFloatWaves - 1) / (16 * kFloatWaves);
    const int64_t sets = (int64_t)o.batch.n_seqs * o.cache.n_kv_heads, tiles = sets * p.col_tiles;
    const int64_t most = (o.batch.max_kv_len + kFewLeast - 1) / kFewLeast, cuts = kFewTarget / tiles;
    cut(&p, o.batch.max_kv_len, cuts < 1 ? 1 : cuts < most ? cuts : most);
    p.workgroups = tiles * p.n_chunks;
    if (p.workgroups <= kMostWorkgroups) p.workgroups = 8 * (int64_t)dies_slots((int)(p.col_tiles * p.n_chunks), (int)sets);
    return p;
}

Plan plan_of(const Attention& o, int is_bf16) {
    const int64_t columns = (int64_t)o.batch.max_rows * (o.n_q_heads / o.cache.n_kv_heads);
    double few_us, prompt_us;
    const Plan few = plan_few(o, columns, is_bf16 ? 2 : 4, &few_us);
    if (!is_bf16) return float_shares(o, columns) ? plan_float(o, columns) : few;
    if (columns <= 16) return few;
    const Plan prompt = plan_prompt(o, columns, &prompt_us);
    return few_us < prompt_us ? few : prompt;
}

int64_t parts(const Attention& o, const Plan& p) {
    return p.n_chunks == 1 ? 0 : (int64_t)p.n_chunks * o.batch.n_seqs * o.batch.max_rows * o.n_q_heads;
}

template <class T, int D>
hipError_t launch(const Attention& o, hipStream_t stream) {
    const Plan p = plan_of(o, sizeof(T) == 2);
    AttnArgs a;
    a.Q = o.Q; a.ldq = o.ldq; a.O = o.O; a.ldo = o.ldo;
    a.n_q_heads = o.n_q_heads; a.group = o.n_q_heads / o.cache.n_kv_heads;
    a.scale2s = o.scale * kLog2E;
    a.scale2 = o.scale == 0.f ? 1e-30f : fabsf(a.scale2s);      // (-inf, a hidden score, times 0 would be NaN)
    a.flip = o.scale < 0.f ? 0x80008000u : 0u;
    a.causal = o.causal;
    a.chunk = p.chunk; a.n_chunks = p.n_chunks; a.col_tiles = (int)p.col_tiles; a.paired = p.paired; a.by_head = p.by_head;
    a.kv = o.cache; a.b = o.batch;
    a.part_o = o.workspace;
    a.part_ml = p.n_chunks == 1 ? nullptr : o.workspace + parts(o, p) * D;
    if constexpr (sizeof(T) == 2) {
        if (p.prompt)
            hipLaunchKernelGGL((attention_prompt_kernel<D>), dim3((unsigned)p.workgroups), dim3(64 * kPromptWaves), (size_t)prompt_lds<D>(), stream, a);
    }
    if constexpr (sizeof(T) == 4 && (D == 96 || D == 128)) {
        if (p.shared) hipLaunchKernelGGL((attention_float_kernel<D>), dim3((unsigned)p.workgroups), dim3(64 * kFloatWaves), (size_t)float_lds<D>(), stream, a);
    }
    const bool direct = !p.prompt && !p.shared;
    const dim3 few((unsigned)(p.col_tiles * p.n_chunks), (unsigned)(o.cache.n_kv_heads / (p.by_head ? kFewWaves : 1)), (unsigned)o.batch.n_seqs);
    if (direct && p.past) hipLaunchKernelGGL((attention_few_kernel<T, D, true>), few, dim3(64 * kFewWaves), 0, stream, a);
    else if (direct) hipLaunchKernelGGL((attention_few_kernel<T, D, false>), few, dim3(64 * kFewWaves), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.n_chunks == 1) return e;
    if (p.n_chunks <= 4) return join<T, D, 1>(a, stream);
    return p.n_chunks <= 16 ? join<T, D, 4>(a, stream) : join<T, D, D == 256 ? 4 : 8>(a, stream);
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

bool attention_fits(const Attention& o, int is_bf16) {
    if (o.batch.n_seqs > 65535 || o.cache.n_kv_heads > 65535) return false;          // dimensions of a launch
    // (before the plan: a column is a row's head, so what this lets through has few enough of them for the plan's counts)
    if ((int64_t)o.batch.n_rows * o.n_q_heads > kMostWorkgroups) return false;
    return plan_of(o, is_bf16).workgroups <= kMostWorkgroups;
}

namespace {
Attention described(int causal, int n_q_heads, int n_kv_heads, int head_dim, int n_seqs, int n_rows, int max_rows, int max_kv_len) {
    Attention o = {};
    o.causal = causal != 0; o.n_q_heads = n_q_heads;
    o.cache.n_kv_heads = n_kv_heads; o.cache.head_dim = head_dim;
    o.batch.n_seqs = n_seqs; o.batch.n_rows = n_rows; o.batch.max_rows = rows_bound(max_rows, n_rows); o.batch.max_kv_len = max_kv_len;
    return o;
}
}  // namespace

// Which way a call of these sizes goes: 0 few columns, 1 many, 2 many with causal tiles in pairs; plus 4 where the cache is cut; -1: too large.
int attention_way(int is_bf16, int causal, int n_q_heads, int n_kv_heads, int head_dim, int n_seqs, int n_rows, int max_rows, int max_kv_len) {
    const Attention o = described(causal, n_q_heads, n_kv_heads, head_dim, n_seqs, n_rows, max_rows, max_kv_len);
    if (!attention_fits(o, is_bf16)) return -1;
    const Plan p = plan_of(o, is_bf16);
    return (p.prompt ? p.paired ? 2 : 1 : 0) + (p.n_chunks > 1 ? 4 : 0);
}

// Whether a float call goes by tiles of 64 columns: 1, with a cut cache 5; -1: too large.
int attention_float_way(int causal, int n_q_heads, int n_kv_heads, int head_dim, int n_seqs, int n_rows, int max_rows, int max_kv_len) {
    const Attention o = described(causal, n_q_heads, n_kv_heads, head_dim, n_seqs, n_rows, max_rows, max_kv_len);
    if (!attention_fits(o, 0)) return -1;
    const Plan p = plan_of(o, 0);
    return (p.shared ? 1 : 0) + (p.n_chunks > 1 ? 4 : 0);
}

size_t attention_workspace_bytes(const Attention& o, int is_bf16) { return parts(o, plan_of(o, is_bf16)) * (o.cache.head_dim + 2) * sizeof(float); }
// A plan of more than one chunk has at most its target of workgroups, and every part is a column of one of them: parts have places by sequence and row
// of it, so rows that belong to no sequence have none.
size_t attention_workspace_bound(int head_dim) {
    const size_t columns = kPromptTarget * 32 * kPromptWaves;
    static_assert(kFewTarget * 16 <= kPromptTarget * 32 * kPromptWaves, "");
    return columns * (head_dim + 2) * sizeof(float);
}

// attention_workspace_bytes of these sizes
size_t attention_parts(int is_bf16, int causal, int n_q_heads, int n_kv_heads, int head_dim, int n_seqs, int n_rows, int max_rows, int max_kv_len) {
    const Attention o = described(causal, n_q_heads, n_kv_heads, head_dim, n_seqs, n_rows, max_rows, max_kv_len);
    return attention_fits(o, is_bf16) ? attention_workspace_bytes(o, is_bf16) : 0;
}

hipError_t attention(const Attention& o, int is_bf16, hipStream_t stream) {
    return is_bf16 ? of_width<uint16_t>(o, stream) : of_width<float>(o, stream);
}

hipError_t attention_init() {
    const void* kernels[] = {(const void*)&attention_prompt_kernel<64>, (const void*)&attention_prompt_kernel<96>,
                             (const void*)&attention_prompt_kernel<128>, (const void*)&attention_prompt_kernel<256>,
                             (const void*)&attention_float_kernel<96>, (const void*)&attention_float_kernel<128>};
    const int bytes[] = {prompt_lds<64>(), prompt_lds<96>(), prompt_lds<128>(), prompt_lds<256>(), float_lds<96>(), float_lds<128>()};
    for (int i = 0; i < 6; ++i) {
        const hipError_t e = hipFuncSetAttribute(kernels[i], hipFuncAttributeMaxDynamicSharedMemorySize, bytes[i]);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace gelo
