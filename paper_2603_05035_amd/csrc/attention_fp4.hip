// Attention over a paged cache of 4 bits (fp4.h): O = sum_p w_p v_p / sum_p w_p, w_p = exp(scale q.k_p - m), in one pass with a running maximum.
//
// A held key or value is a power of two times a number of two bits after its first one: exact in bfloat16, which the matrix instructions take.  So they
// multiply what is held with nothing rounded on the way.  Queries of bfloat16 are one operand; a float query is the sum of three bfloat16, and a
// weight the sum of two (bfloat16 calls: 16 bits) or three (float calls: all of it), so that float results are as near as float products would leave them, at
// three bfloat16 instructions in the place of eight of float.  Conversions of gfx950 make two bfloat16 of a byte with the block's scale in it, at the rate
// of an addition.
//
// attention_few_fp4_kernel: a COLUMN is a row's query head, 16 columns that meet one key head are a tile.  S^T = K Q^T leaves in every lane scores of one
// column; the weights are at once the operand of O^T = V^T P^T.  Lane (g, c) = (lane / 16, lane % 16).  S^T, 16 keys: the lane's operand is a quarter of key c,
// components (D / 4) g ..., step s of the product takes 8 of them, and of column c's query alike.  It then holds the scores of keys 4 g + r.  O^T: the
// operand's slot 4 t + r of the lane is key 16 t + 4 g + r; the lane has components (D / 16) c + j of it, instruction j takes one of each.
#include "attention_prompt.h"

namespace gelo {
namespace {

typedef uint16_t u16_t;
constexpr int kFewWaves = 4;

// 32 keys a half of a step
template <class T, int D, bool PAST>
struct Few {
    static constexpr bool FLOAT = sizeof(T) == 4;
    static constexpr int HALVES = D < 256 ? 2 : 1, TILES = 2 * HALVES, KEYS = 16 * TILES;
    static constexpr int W = D / 32, KS = D / 32, VD = D / 16, VW = VD / 2;      // words of a lane's load; steps of S^T; components of a lane, pairs of them
    static constexpr int QP = FLOAT ? 3 : 1, WP = FLOAT ? 3 : 2;                 // parts of a query and of a weight
    static constexpr bool APART = FLOAT && D >= 128;                             // a float query's parts lie in LDS, shared by the waves
    typedef bf16x8_t frag_t;
    frag_t q[APART ? 1 : QP][APART ? 1 : KS];
    const frag_t* q_apart;
    // EARLY: the next step's values are sent for with its keys, before this step's arithmetic (64 x 3500-4095 keys of 32 heads of 128 188 us and 179, of heads of 256, whose
    // registers are scarce, 32 x 2000 keys 31.6 and 37.4)
    static constexpr bool EARLY = !FLOAT && D == 128;
    static constexpr int VB = D == 96 ? 2 : 1;                   // blocks a lane's components lie in
    uint32_t k[TILES][W], v[TILES][W], v_next[EARLY ? TILES : 1][W];
    uint32_t k_scale[TILES], v_scale[TILES][VB], v_scale_next[EARLY ? TILES : 1][VB];          // 1 or 2 bytes; 4 rows' bytes of a block

    // to: LDS for the parts of a float query where they lie there (the waves of a workgroup write the same)
    __device__ __forceinline__ void load_q(const T* p, int g, frag_t* to) {
        q_apart = to + (threadIdx.x & 63);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const T* at = p + D / 4 * g + 8 * s;
            if constexpr (!FLOAT) {
                q[0][s] = *reinterpret_cast<const frag_t*>(at);
            } else {
                const f32x4_t x[2] = {*reinterpret_cast<const f32x4_t*>(at), *reinterpret_cast<const f32x4_t*>(at + 4)};
                u16_t part[3][8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float rest = x[e >> 2][e & 3];
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
                        const uint32_t up = __float_as_uint(rest) & 0xFFFF0000u;
                        part[i][e] = (u16_t)(up >> 16);
                        rest -= __uint_as_float(up);
                    }
                }
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    frag_t f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = __builtin_bit_cast(__bf16, part[i][e]);
                    if constexpr (APART) to[64 * (i * KS + s) + (threadIdx.x & 63)] = f;
                    else q[i][s] = f;
                }
            }
        }
    }
    // piece: a head's piece of a page; row: the tile's first in it; scales: where its scale bytes begin
    __device__ __forceinline__ void load_k(int t, const uint8_t* piece, int row, int scales, int g, int c) {
        read_words<W, PAST>(piece + (uint32_t)(row * (D / 2) + (4 * c + g) * (D / 8)), k[t]);
        const uint8_t* s = piece + (uint32_t)(scales + row * (D / 32) + c * (D / 32) + (D == 64 ? g >> 1 : D == 128 ? g : D == 256 ? 2 * g : 24 * g / 32));
        if constexpr (D == 64 || D == 128) k_scale[t] = *s;
        else if constexpr (D == 96) k_scale[t] = s[0] | (uint32_t)s[(24 * g + 23) / 32 - 24 * g / 32] << 8;
        else k_scale[t] = *reinterpret_cast<const u16_t*>(s);
    }
    __device__ __forceinline__ void load_v(int t, const uint8_t* piece, int row, int scales, int g, int c) {
        auto& codes = [&]() -> uint32_t (&)[W] { if constexpr (EARLY) return v_next[t]; else return v[t]; }();
        auto& bytes = [&]() -> uint32_t (&)[VB] { if constexpr (EARLY) return v_scale_next[t]; else return v_scale[t]; }();
        read_words<W, PAST>(piece + (uint32_t)(row * (D / 2) + (16 * g + c) * (D / 8)), codes);
        const uint8_t* s = piece + (uint32_t)(scales + row * (D / 32) + g * (D / 8) + 4 * (VD * c / 32));
        bytes[0] = *reinterpret_cast<const uint32_t*>(s);
        if constexpr (D == 96) bytes[1] = *reinterpret_cast<const uint32_t*>(s + 4 * ((VD * c + 5) / 32 - VD * c / 32));
    }
    __device__ __forceinline__ void turn_values() {              // those sent for early become this step's
        if constexpr (EARLY) {
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
#pragma unroll
                for (int w = 0; w < W; ++w) v[t][w] = v_next[t][w];
                v_scale[t][0] = v_scale_next[t][0];
            }
        }
    }
    __device__ __forceinline__ f32x4_t scores(int t, int g) const {
        f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
        const float s0 = fp4_scale(k_scale[t] & 0xFFu), s1 = D == 96 || D == 256 ? fp4_scale(k_scale[t] >> 8) : s0;
        const int turn = D == 96 ? (32 * (24 * g / 32 + 1) - 24 * g) / 8 : KS / 2;      // the step that begins the second block
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const float scale = D == 96 || D == 256 ? s < turn ? s0 : s1 : s0;
            const u32x4_t x = {fp4_pair<0>(k[t][s], scale), fp4_pair<1>(k[t][s], scale), fp4_pair<2>(k[t][s], scale), fp4_pair<3>(k[t][s], scale)};
            const frag_t f = __builtin_bit_cast(frag_t, x);
#pragma unroll
            for (int i = QP - 1; i >= 0; --i) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, APART ? q_apart[64 * (i * KS + s)] : q[APART ? 0 : i][APART ? 0 : s], sum, 0, 0, 0);
        }
        return sum;
    }
    // acc += the values of 32 keys times their weights p, whose slots are 4 t + r
    __device__ __forceinline__ void accumulate(int half, const float* p, f32x4_t (&acc)[VD], int c) const {
        frag_t w[WP];
        {
            float rest[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) rest[i] = p[i];
#pragma unroll
            for (int j = 0; j + 1 < WP; ++j) {
                u32x4_t up;
#pragma unroll
                for (int i = 0; i < 4; ++i) up[i] = __builtin_amdgcn_perm(__float_as_uint(rest[2 * i + 1]), __float_as_uint(rest[2 * i]), 0x07060302u);
#pragma unroll
                for (int i = 0; i < 8; ++i) rest[i] -= __uint_as_float(__float_as_uint(rest[i]) & 0xFFFF0000u);
                w[j] = __builtin_bit_cast(frag_t, up);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) w[WP - 1][i] = (__bf16)rest[i];
        }
        float scale[VB][8];
#pragma unroll
        for (int b = 0; b < VB; ++b)
#pragma unroll
            for (int i = 0; i < 8; ++i) scale[b][i] = fp4_scale((v_scale[2 * half + (i >> 2)][b] >> (8 * (i & 3))) & 0xFFu);
        const int turn = (32 * (VD * c / 32 + 1) - VD * c) / 2;           // heads of 96: the pair that begins the second block
        static_for<VW>([&](auto wc) {
            constexpr int x = decltype(wc)::value;
            uint32_t pair[8];
            static_for<8>([&](auto ic) {
                constexpr int i = decltype(ic)::value, byte = (i & 3) * VW + x;
                const float by = D == 96 ? x < turn ? scale[0][i] : scale[D == 96 ? 1 : 0][i] : scale[0][i];
                pair[i] = fp4_pair<byte & 3>(v[2 * half + (i >> 2)][byte >> 2], by);
            });
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
                u32x4_t f;
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_perm(pair[2 * i + 1], pair[2 * i], odd ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int j = WP - 1; j >= 0; --j)
                    acc[2 * x + odd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(frag_t, f), w[j], acc[2 * x + odd], 0, 0, 0);
            }
        });
    }
    // slots of a half whose block (of heads of 96: first or second one) is NaN, or has a scale beyond the format's: what lies behind a sequence's end may be anything, and
    // its 6 2^126 are infinities
    __device__ __forceinline__ uint32_t odd_slots(int half, int b) const {
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) odd |= (uint32_t)(((v_scale[2 * half + (i >> 2)][b] >> (8 * (i & 3))) & 0xFFu) > kFp4MostScale) << i;
        return odd;
    }
    // as accumulate, where some keys are hidden from some columns (seen: bit per slot): 0 times NaN would be NaN in those.  How many NaN a column sees of a
    // component is counted by a product more, and the blocks' scales go.
    __device__ __forceinline__ void accumulate_odd(int half, const float* p, f32x4_t (&acc)[VD], int c, uint32_t seen) {
        const uint32_t odd[2] = {odd_slots(half, 0), odd_slots(half, D == 96 ? 1 : 0)};
        frag_t sees;
#pragma unroll
        for (int i = 0; i < 8; ++i) sees[i] = (__bf16)((seen >> i) & 1 ? 1.f : 0.f);
        const int turn = (32 * (VD * c / 32 + 1) - VD * c) / 2;
#pragma unroll
        for (int b = 0; b < VB; ++b)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if ((odd[b] >> i) & 1) v_scale[2 * half + (i >> 2)][b] &= ~(0xFFu << (8 * (i & 3)));
        accumulate(half, p, acc, c);
#pragma unroll
        for (int j = 0; j < VD; ++j) {
            const uint32_t mine = odd[D == 96 && j / 2 >= turn ? 1 : 0];
            frag_t f;
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (__bf16)((mine >> i) & 1 ? 1.f : 0.f);
            const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
            const f32x4_t count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, sees, zero, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[j][r] += count[r] > 0.f ? __builtin_nanf("") : 0.f;
        }
    }
};

// A weight is at most 2^kSlack: the maximum that weights are relative to moves only where a column's has grown by more, which spares most steps the look
// across lanes and the rescaling.
constexpr float kSlack = 8.f;

// One wave walks the keys `key`, key + stride, ... up to `last` of a tile of 16 columns, KEYS at a time: what weights are relative to (of log2), the sum of
// weights over the lane's own keys and the weighted sum of the values.  limit: last key this lane's column sees, least: the least of the tile.
template <class T, int D, bool PAST>
__device__ __forceinline__ void walk_keys(const AttnArgs& a, int seq, int kvh, int key, int stride, int last, int least, int limit, int g, int c,
                                          Few<T, D, PAST>& f, f32x4_t (&acc)[Few<T, D, PAST>::VD], float& m, float& l, bool& bad_page) {
    typedef Few<T, D, PAST> F;
    constexpr int VD = F::VD, SLOTS = 4 * F::TILES;
    const int shift = a.kv.page_shift, in_page = (1 << shift) - 1, scales = fp4_scales_at(D, shift);
    const int32_t* table = a.b.page_table + seq * a.b.table_ld;
    const uint8_t* k_head = (const uint8_t*)a.kv.k + kvh * a.kv.head_stride;
    const uint8_t* v_head = (const uint8_t*)a.kv.v + kvh * a.kv.head_stride;
    // Tiles beyond the end are read as the last one, whose rows are there, and get no weight.  Where a tile lies is worked out once for keys and values: 64-bit
    // products of its own for each were as long as the arithmetic beside them (64 x 3500-4095 keys of 32 heads 202 us).
    const uint32_t page_stride = (uint32_t)a.kv.page_stride;             // (below 2^31)
    uint64_t place[F::TILES];
    int in_piece[F::TILES];
    auto tile_start = [&](int key) { return min(key, last & ~15); };
    auto page_of = [&](int key) { return table[tile_start(key) >> shift]; };
    auto find = [&](int key, const int (&page)[F::TILES]) {
#pragma unroll
        for (int t = 0; t < F::TILES; ++t) {
            const bool good = (uint32_t)page[t] < (uint32_t)a.kv.n_pages;
            bad_page |= !good;
            place[t] = (uint64_t)(good ? (uint32_t)page[t] : 0u) * page_stride;
            in_piece[t] = tile_start(key + 16 * t) & in_page;
        }
    };
    auto load_k = [&] {
#pragma unroll
        for (int t = 0; t < F::TILES; ++t) f.load_k(t, k_head + place[t], in_piece[t], scales, g, c);
    };
    auto load_v = [&] {
#pragma unroll
        for (int t = 0; t < F::TILES; ++t) f.load_v(t, v_head + place[t], in_piece[t], scales, g, c);
    };
    if (key > last) return;
    float base = 0.f;                                        // m, or 0 where nothing has been seen yet: all weights are 0
    int page[F::TILES];
#pragma unroll
    for (int t = 0; t < F::TILES; ++t) page[t] = page_of(key + 16 * t);
    find(key, page);
    load_k();
    load_v();
    f.turn_values();
    for (; key <= last; key += stride) {
        const int next = key + stride;
        if (next <= last) {
#pragma unroll
            for (int t = 0; t < F::TILES; ++t) page[t] = page_of(next + 16 * t);
        }
        if (next <= last) {
            find(next, page);
            if constexpr (F::EARLY) load_v();
        }
        float s[SLOTS];
#pragma unroll
        for (int t = 0; t < F::TILES; ++t) {
            const f32x4_t x = f.scores(t, g);
#pragma unroll
            for (int r = 0; r < 4; ++r) s[4 * t + r] = x[r] * a.scale2s;
        }
        if (next <= last) load_k();
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
        if (__ballot(top > m + kSlack)) {
            const float m_new = fmaxf(m, across_groups_max(top));
            base = m_new == -__builtin_inff() ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m - base);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int j = 0; j < VD; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[j][r] *= alpha;
        }
#pragma unroll
        for (int r = 0; r < SLOTS; ++r) {
            s[r] = __builtin_amdgcn_exp2f(s[r] - base);
            l += s[r];
        }
#pragma unroll
        for (int h = 0; h < F::HALVES; ++h) {
            if (partly && __ballot((f.odd_slots(h, 0) | f.odd_slots(h, D == 96 ? 1 : 0)) != 0)) f.accumulate_odd(h, s + 8 * h, acc, c, seen >> (8 * h));
            else f.accumulate(h, s + 8 * h, acc, c);
        }
        if constexpr (F::EARLY) f.turn_values();
        else if (next <= last) load_v();
    }
}

template <class T, int D> constexpr int few_lds() {
    const int joined = kFewWaves * 16 * (D + 4) * 4, parts = Few<T, D, false>::APART ? 3 * (D / 32) * 1024 : 0;
    return joined > parts ? joined : parts;
}

// A workgroup: one tile of 16 columns of one sequence and key head, one chunk of the cache, whose keys its waves share out; or (by_head) one
// sequence and four key heads, one to a wave.
template <class T, int D, bool PAST>
__global__ __launch_bounds__(64 * kFewWaves, sizeof(T) == 4 && D == 128 ? 3 : 2)
void attention_few_fp4_kernel(AttnArgs a) {
    typedef Few<T, D, PAST> F;
    constexpr int VD = F::VD;
    __shared__ __attribute__((aligned(16))) uint8_t lds[few_lds<T, D>()];      // parts of a float query, and then the waves' sums
    __shared__ float joined_ml[kFewWaves][16][2];
    auto joined_o = reinterpret_cast<float (*)[16][D + 4]>(lds);
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
    f.load_q((const T*)a.Q + row * a.ldq + (int64_t)head * D, g, reinterpret_cast<typename F::frag_t*>(lds));
    if constexpr (F::APART) __syncthreads();
    f32x4_t acc[VD];
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -__builtin_inff(), l = 0.f;
    bool bad_page = false;

    walk_keys<T, D, PAST>(a, seq, kvh, a.by_head ? begin : begin + wave * F::KEYS, a.by_head ? F::KEYS : F::KEYS * kFewWaves, end - 1, least, limit, g, c, f, acc, m, l, bad_page);
    l = across_groups_sum(l);
    if (bad_page) l = __builtin_nanf("");
    if constexpr (F::APART) __syncthreads();                 // nobody reads the query's parts any more

    // acc[j][r]: component VD (4 g + r) + j of column c
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < VD; ++j) joined_o[wave][c][VD * (4 * g + r) + j] = acc[j][r];
    if (g == 0) { joined_ml[wave][c][0] = m; joined_ml[wave][c][1] = l; }
    __syncthreads();
    for (int e = threadIdx.x; e < heads * 16 * (D / 4); e += 64 * kFewWaves) {
        const int k16 = e / (D / 4), cc = k16 & 15, hd = k16 >> 4, x = 4 * (e - k16 * (D / 4)), cl = tile * 16 + cc;
        const int from = a.by_head ? hd : 0, to = a.by_head ? hd + 1 : kFewWaves;             // the waves that have parts of this column
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
        const int ri = cl / a.group, h = (first_kvh + hd) * a.group + cl - ri * a.group;
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

constexpr int kFewLong = 4096, kFewMost = 4096;             // keys; workgroups, whose columns are as many as the workspace's bound has
static_assert(kFewMost * 16 <= kPromptTarget * 32 * kPromptWaves, "");
static_assert(64 * kFewWaves <= 256 && 64 * kPromptWaves <= 256, "workgroups as kMostWorkgroups has them");

Plan plan_few(const Attention& o, int64_t columns, int is_bf16, double* us) {
    Plan p;
    p.prompt = p.shared = p.paired = p.past = p.by_head = false;
    p.col_tiles = (columns + 15) / 16;
    const int64_t tiles = (int64_t)o.batch.n_seqs * o.cache.n_kv_heads * p.col_tiles;
    const int64_t most = (o.batch.max_kv_len + kFewLeast - 1) / kFewLeast;
    // Long caches are cut further, into 4096 keys, once that makes four: sequences of a batch end at lengths of their own, and the longest would work alone at the end (us as few as
    // fill the chip, and so: 6 sequences of 18658-37317 keys of 32 heads 188 and 160, 39 of 21295-42590 of 5 213 and 167, 106 of 26353-52707 of one head of 64, float, 134 and 108; cut in
    // two or three 17 of 6000-12000 of 32 135 and 161; 2048 keys, 16 of 32000 of 4 54 and 60).
    const int64_t fill = kFewTarget / tiles, fine = o.batch.max_kv_len / kFewLong < kFewMost / tiles ? o.batch.max_kv_len / kFewLong : kFewMost / tiles;
    const int64_t cuts = fine >= 4 && fine > fill ? fine : fill;
    cut(&p, o.batch.max_kv_len, cuts < 1 ? 1 : cuts < most ? cuts : most);
    p.workgroups = tiles * p.n_chunks;
    // A head to a wave needs no join, but a wave walks its cache alone: where one round of such workgroups fills the chip.  us with a cache shared out and by head, bfloat16, caches of 85 to 100% of 64,
    // 512, 2000 and 4000 keys:
    //   32 heads of 128   48 sequences 12.3, 25.0, 74, 139 and 7.8, 26.4, 83, 160;  56 15.1, 28.2, 87, 156 and 7.7, 26.8, 90, 163;  63 16.2, 31.2, 96, 178 and 7.9, 28.0, 95, 179
    //                     64 16.2, 31.9, 96, 178 and 8.2, 28.5, 93, 180;  72 19.1, 36.5, 110, 201 and 11.4, 40.9, 133, 251;  96 23.9, 46.9, 145, 261 and 11.7, 42.8, 146, 270
    //   16 heads of 64    128 sequences 10.2, 21.2, 64, 116 and 6.5, 20.6, 73, 138
    // So it is right for short caches on both sides of the border, and takes up to a quarter more where caches are long and the last round nearly empty, or heads narrow: the rule looks at neither.
    p.by_head = (is_bf16 || o.cache.head_dim < 128) && p.n_chunks == 1 && p.col_tiles == 1 && o.cache.n_kv_heads % kFewWaves == 0 && tiles / kFewWaves >= kFewTarget;
    if (p.by_head) p.workgroups = tiles / kFewWaves;
    p.past = p.col_tiles == 1 && 17.0 / 16 * tiles * o.batch.max_kv_len * o.cache.head_dim > 100e6;
    // a wave's step of 64 keys takes its SIMD 1.3 us at a width of 128, and a trip to memory 1.5
    const double rounds = (double)((p.workgroups + kFewTarget - 1) / kFewTarget), steps = (p.chunk + 255) / 256;
    const double work = p.workgroups * steps * 4 / 1024 * 1.3 * o.cache.head_dim / 128, trips = rounds * steps * 1.5;
    *us = 4.0 * rounds + (work > trips ? work : trips) + join_us(o, p);
    return p;
}

Plan plan_of(const Attention& o, int is_bf16) {
    const int64_t columns = (int64_t)o.batch.max_rows * (o.n_q_heads / o.cache.n_kv_heads);
    double few_us, prompt_us;
    const Plan few = plan_few(o, columns, is_bf16, &few_us);
    if (!is_bf16 || columns <= 16) return few;
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
            hipLaunchKernelGGL((attention_prompt_kernel<D, true>), dim3((unsigned)p.workgroups), dim3(64 * kPromptWaves), (size_t)prompt_lds<D>(), stream, a);
    }
    const dim3 few((unsigned)(p.col_tiles * p.n_chunks), (unsigned)(o.cache.n_kv_heads / (p.by_head ? kFewWaves : 1)), (unsigned)o.batch.n_seqs);
    if (p.prompt) {}
    else if (p.past) hipLaunchKernelGGL((attention_few_fp4_kernel<T, D, true>), few, dim3(64 * kFewWaves), 0, stream, a);
    else hipLaunchKernelGGL((attention_few_fp4_kernel<T, D, false>), few, dim3(64 * kFewWaves), 0, stream, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || p.n_chunks == 1 ? e : join_parts<T, D>(a, stream);
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

bool attention_fp4_fits(const Attention& o, int is_bf16) {
    if (o.batch.n_seqs > 65535 || o.cache.n_kv_heads > 65535) return false;          // dimensions of a launch
    if ((int64_t)o.batch.n_rows * o.n_q_heads > kMostWorkgroups) return false;
    return plan_of(o, is_bf16).workgroups <= kMostWorkgroups;
}

size_t attention_fp4_workspace_bytes(const Attention& o, int is_bf16) { return parts(o, plan_of(o, is_bf16)) * (o.cache.head_dim + 2) * sizeof(float); }

namespace {
Attention described(int causal, int n_q_heads, int n_kv_heads, int head_dim, int n_seqs, int n_rows, int max_rows, int max_kv_len) {
    Attention o = {};
    o.causal = causal != 0; o.n_q_heads = n_q_heads;
    o.cache.n_kv_heads = n_kv_heads; o.cache.head_dim = head_dim;
    o.batch.n_seqs = n_seqs; o.batch.n_rows = n_rows; o.batch.max_rows = rows_bound(max_rows, n_rows); o.batch.max_kv_len = max_kv_len;
    return o;
}
}  // namespace

// Which way a call of these sizes goes, as attention_way says it, plus 8 where a wave has a head to itself.
int attention_fp4_way(int is_bf16, int causal, int n_q_heads, int n_kv_heads, int head_dim, int n_seqs, int n_rows, int max_rows, int max_kv_len) {
    const Attention o = described(causal, n_q_heads, n_kv_heads, head_dim, n_seqs, n_rows, max_rows, max_kv_len);
    if (!attention_fp4_fits(o, is_bf16)) return -1;
    const Plan p = plan_of(o, is_bf16);
    return (p.prompt ? p.paired ? 2 : 1 : 0) + (p.n_chunks > 1 ? 4 : 0) + (p.by_head ? 8 : 0);
}
// attention_fp4_workspace_bytes of these sizes
size_t attention_fp4_parts(int is_bf16, int causal, int n_q_heads, int n_kv_heads, int head_dim, int n_seqs, int n_rows, int max_rows, int max_kv_len) {
    const Attention o = described(causal, n_q_heads, n_kv_heads, head_dim, n_seqs, n_rows, max_rows, max_kv_len);
    return attention_fp4_fits(o, is_bf16) ? attention_fp4_workspace_bytes(o, is_bf16) : 0;
}

hipError_t attention_fp4(const Attention& o, int is_bf16, hipStream_t stream) { return is_bf16 ? of_width<uint16_t>(o, stream) : of_width<float>(o, stream); }

hipError_t attention_fp4_init() {
    const void* kernels[] = {(const void*)&attention_prompt_kernel<64, true>, (const void*)&attention_prompt_kernel<96, true>,
                             (const void*)&attention_prompt_kernel<128, true>, (const void*)&attention_prompt_kernel<256, true>};
    const int bytes[] = {prompt_lds<64>(), prompt_lds<96>(), prompt_lds<128>(), prompt_lds<256>()};
    for (int i = 0; i < 4; ++i) {
        const hipError_t e = hipFuncSetAttribute(kernels[i], hipFuncAttributeMaxDynamicSharedMemorySize, bytes[i]);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace gelo
