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
#include "attention_prompt.h"

namespace gelo {
namespace {

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
static_assert(64 * kFewWaves <= 256 && 64 * kFloatWaves <= 256 && 64 * kPromptWaves <= 256, "workgroups as kMostWorkgroups has them");
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
            hipLaunchKernelGGL((attention_prompt_kernel<D, false>), dim3((unsigned)p.workgroups), dim3(64 * kPromptWaves), (size_t)prompt_lds<D>(), stream, a);
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
    return join_parts<T, D>(a, stream);
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
    const void* kernels[] = {(const void*)&attention_prompt_kernel<64, false>, (const void*)&attention_prompt_kernel<96, false>,
                             (const void*)&attention_prompt_kernel<128, false>, (const void*)&attention_prompt_kernel<256, false>,
                             (const void*)&attention_float_kernel<96>, (const void*)&attention_float_kernel<128>};
    const int bytes[] = {prompt_lds<64>(), prompt_lds<96>(), prompt_lds<128>(), prompt_lds<256>(), float_lds<96>(), float_lds<128>()};
    for (int i = 0; i < 6; ++i) {
        const hipError_t e = hipFuncSetAttribute(kernels[i], hipFuncAttributeMaxDynamicSharedMemorySize, bytes[i]);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace gelo
