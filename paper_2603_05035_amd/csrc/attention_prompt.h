// Attention of many columns to a key head, bfloat16: the kernel for prompts, over a cache of values or one of 4 bits, and how its calls are cut.
#pragma once

#include "attention.h"
#include "fp4.h"

namespace gelo {
namespace {

// sum + the two bfloat16 of a word: their products with 1
__device__ __forceinline__ float add_pair(uint32_t pair, float sum) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pair), bf16x2_t{(__bf16)1.f, (__bf16)1.f}, sum, false);
}

// attention_prompt_kernel: many columns to a key head, bfloat16.  Bound by the matrix instructions and, beside them, by the exponentials.  A
// workgroup takes kPromptWaves x 32 columns and walks the keys kPromptKeys at a time; K and V come into LDS once for all its waves, by
// direct-to-LDS fetches a step ahead.  v_mfma_f32_32x32x16_bf16: lane (h, c) = (lane / 32, lane % 32); S^T of 32 keys leaves in register r of
// the lane column c and key 8 (r / 4) + 4 h + r % 4, so registers 8 t ... 8 t + 7 are keys 16 t + {4 h + 0..3, 8 + 4 h + 0..3}: the B operand of step t
// of O^T, if A = V^T takes its keys in that order - two transposing reads of four rows each.
// A wave works on three groups of 32 keys at once, whose instructions depend on nothing of each other: the scores of the next group and the
// weighted sum of the last one (matrix pipe) beside the weights of the present one (vector pipe).
// Weights are rounded to bfloat16 for the product with V, and their sum is that of the rounded ones: what a rounding leaves would be half as many matrix instructions more, and they are what prompts
// wait for.  Distance from 64 bits, relative in the Frobenius norm: 8 x 301-512 rows 0.0021, 6000 behind 2000 0.0023; of these the rounding of the result is 0.0016 to 0.0017.
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
template <int D, bool FP4, bool ODD>
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
    typedef std::conditional_t<FP4, uint8_t, uint16_t> held_t;
    const held_t* k_head = (const held_t*)a.kv.k + kvh * a.kv.head_stride;
    const held_t* v_head = (const held_t*)a.kv.v + kvh * a.kv.head_stride;
    bool bad_page = false;
    auto group_of = [&](int step) { return min(begin + step * KT + wave * ROWS, last & ~(ROWS - 1)); };
    // (a vector load: beside a scalar one every wait for LDS would be a wait for it as well)
    auto load_page = [&](int step) { return table[(group_of(min(step, steps - 1)) + (lane >> 6)) >> shift]; };
    auto rows_at = [&](int step, int page) {                 // values (of 4 bits: bytes) from the start of a head to these rows
        const bool good = page >= 0 && page < a.kv.n_pages;
        bad_page |= !good;
        return (good ? page : 0) * a.kv.page_stride + (group_of(step) & in_page) * (FP4 ? D / 2 : a.kv.row_stride);
    };
    // rows beyond the last key are fetched as that key's (they are masked, but 0 times what lies there might be NaN): in the last step
    auto trim = [&](uint32_t (&off)[NF], int step) {
        const int there = last - group_of(step);             // last row of the 16 that is there
        if (step < steps - 1 || there >= ROWS - 1) return;
#pragma unroll
        for (int i = 0; i < NF; ++i) off[i] -= (uint32_t)(max((i * 1024 + lane * 16) / PITCH - there, 0) * (int)a.kv.row_stride) * 2;
    };

    // Of 4 bits: the wave's 16 rows of a step come into registers, a lane's D / 8 bytes side by side, and are put into LDS as bfloat16 a step later.  Keys: a
    // quarter of row lane / 4; values: D / 16 components of each of the rows 4 (lane / 16) ...
    constexpr int W = D / 32, VW = D / 32;
    [[maybe_unused]] uint32_t k_codes[W], v_codes[W], k_scale, v_scale[D == 96 ? 2 : 1];
    const int scales = fp4_scales_at(D, shift);
    auto scale_rows = [&](int64_t rows, int step) {          // where the scale bytes of these rows are
        return rows + scales - (group_of(step) & in_page) * (D / 2 - D / 32);
    };
    auto read_k4 = [&](int64_t rows, int step, uint32_t (&codes)[W], uint32_t& scale) {
        read_words<W, false>((const uint8_t*)k_head + rows + lane * (D / 8), codes);
        const uint8_t* s = (const uint8_t*)k_head + scale_rows(rows, step) + (lane >> 2) * (D / 32);
        const int quarter = lane & 3;
        if constexpr (D == 64) scale = s[quarter >> 1];
        else if constexpr (D == 96) scale = s[24 * quarter / 32] | (uint32_t)s[(24 * quarter + 23) / 32] << 8;
        else if constexpr (D == 128) scale = s[quarter];
        else scale = *reinterpret_cast<const uint16_t*>(s + 2 * quarter);
    };
    auto read_v4 = [&](int64_t rows, int step) {
        read_words<W, false>((const uint8_t*)v_head + rows + lane * (D / 8), v_codes);
        const uint8_t* s = (const uint8_t*)v_head + scale_rows(rows, step) + (lane >> 4) * (D / 8);
        v_scale[0] = *reinterpret_cast<const uint32_t*>(s + 4 * (D / 16 * (lane & 15) / 32));
        if constexpr (D == 96) v_scale[1] = *reinterpret_cast<const uint32_t*>(s + 4 * ((D / 16 * (lane & 15) + 5) / 32));
    };
    // chunk j of the lane's keys into slot `slot`
    auto put_k4 = [&](auto jc, int slot, const uint32_t (&codes)[W], uint32_t scale) {
        constexpr int j = decltype(jc)::value;
        int my = lane;
        asm volatile("" : "+v"(my));                         // (addresses are worked out again: kept, they take registers the loop needs)
        const int r = my >> 2, quarter = my & 3, turn = D == 96 ? (32 * (24 * quarter / 32 + 1) - 24 * quarter) / 8 : W / 2;
        const float by = fp4_scale(((D == 96 || D == 256) && j >= turn ? scale >> 8 : scale) & 0xFFu);
        const u32x4_t x = {fp4_pair<0>(codes[j], by), fp4_pair<1>(codes[j], by), fp4_pair<2>(codes[j], by), fp4_pair<3>(codes[j], by)};
        *reinterpret_cast<u32x4_t*>(lds + slot * SLOT + (wave * ROWS + r) * PITCH + 16 * k_pos<D>(r, quarter * W + j)) = x;
    };
    // the lane's values of its row r.  Rows beyond the last key get a scale that is a number: they are masked, but 0 times NaN is NaN
    auto trim_v4 = [&](int step) {
        const int there = last - group_of(step);             // last row of the 16 that is there
        if (step < steps - 1 || there >= ROWS - 1) return;
        const int n = min(max(there + 1 - 4 * (lane >> 4), 0), 4);
#pragma unroll
        for (int b = 0; b < (D == 96 ? 2 : 1); ++b) v_scale[b] &= n == 4 ? ~0u : (1u << (8 * n)) - 1;
    };
    auto put_v4 = [&](auto rc, int slot) {
        constexpr int r = decltype(rc)::value;
        int my = lane;
        asm volatile("" : "+v"(my));
        const int row = 4 * (my >> 4) + r, col = my & 15, turn = (32 * (D / 16 * col / 32 + 1) - D / 16 * col) / 2;
        float by[D == 96 ? 2 : 1];
#pragma unroll
        for (int b = 0; b < (D == 96 ? 2 : 1); ++b) by[b] = fp4_scale((v_scale[b] >> (8 * r)) & 0xFFu);
        uint32_t x[VW];
        static_for<VW>([&](auto wc) {
            constexpr int w = decltype(wc)::value, byte = r * VW + w;
            x[w] = fp4_pair<byte & 3>(v_codes[byte >> 2], D == 96 && w >= turn ? by[D == 96 ? 1 : 0] : by[0]);
        });
        uint8_t* to = lds + slot * SLOT + (wave * ROWS + row) * PITCH;
        if constexpr (D == 64) *reinterpret_cast<u32x2_t*>(to + 16 * v_pos<D>(row, col >> 1) + 8 * (col & 1)) = u32x2_t{x[0], x[1]};
        else if constexpr (D == 96) *reinterpret_cast<u32x3_t*>(to + 12 * col) = u32x3_t{x[0], x[1], x[2]};
        else {
#pragma unroll
            for (int i = 0; i < VW / 4; ++i)
                *reinterpret_cast<u32x4_t*>(to + 16 * v_pos<D>(row, VW / 4 * col + i)) = u32x4_t{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
        }
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
    if constexpr (!FP4) {
#pragma unroll
    for (int i = 0; i < NF; ++i) {
        const int at = i * 1024 + lane * 16, r = at / PITCH, x = (at - r * PITCH) / 16, rr = wave * ROWS + r;
        k_off[i] = (uint32_t)(r * (int)a.kv.row_stride + 8 * k_chunk<D>(rr, x)) * 2;
        v_off[i] = (uint32_t)(r * (int)a.kv.row_stride + 8 * v_pos<D>(rr, x)) * 2;
    }
    }
    auto barrier4 = [&] {                                    // what the waves have put into LDS is there
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if (FP4 && steps > 0) {
        const int page0 = load_page(0), page1 = load_page(1), page2 = load_page(2);
        page = load_page(3);
        uint32_t codes0[W], codes1[W], scale0, scale1;
        const int64_t rows0 = rows_at(0, __builtin_amdgcn_readfirstlane(page0));
        read_k4(rows0, 0, codes0, scale0);
        read_v4(rows0, 0);
        if (steps > 1) {
            v_rows = rows_at(1, __builtin_amdgcn_readfirstlane(page1));
            read_k4(v_rows, 1, codes1, scale1);
        }
        if (steps > 2) k_rows = rows_at(2, __builtin_amdgcn_readfirstlane(page2));
        trim_v4(0);
        static_for<W>([&](auto jc) { put_k4(jc, 0, codes0, scale0); });
        static_for<4>([&](auto rc) { put_v4(rc, 2); });
        if (steps > 1) {
            read_v4(v_rows, 1);
            if (steps > 2) read_k4(k_rows, 2, k_codes, k_scale);
            static_for<W>([&](auto jc) { put_k4(jc, 1, codes1, scale1); });
        }
        barrier4();
    }
    if (!FP4 && steps > 0) {
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
        if constexpr (FP4) {
            barrier4();
        } else {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
        }
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
    // (of 4 bits: put into LDS, and those of one step further on are sent for, in 6 + W)
    auto send = [&](auto ic) {
        constexpr int i = decltype(ic)::value;
        const int at = step & 1;
        if constexpr (FP4) {
            if constexpr (i == 0) {
                if (step + 1 < steps) trim_v4(step + 1);
            } else if constexpr (i <= 4) {
                if (step + 1 < steps) put_v4(std::integral_constant<int, i - 1>{}, 3 - at);
            } else if constexpr (i <= 4 + W) {
                if (step + 2 < steps) put_k4(std::integral_constant<int, i - 5>{}, at, k_codes, k_scale);
            } else if constexpr (i == 5 + W) {
                if (step + 2 < steps) {
                    read_v4(k_rows, step + 2);
                    if (step + 3 < steps) {
                        k_rows = rows_at(step + 3, __builtin_amdgcn_readfirstlane(page));
                        read_k4(k_rows, step + 3, k_codes, k_scale);
                    }
                    page = load_page(step + 4);
                }
            }
        } else if constexpr (i == 0) {
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
        static_for<FP4 ? 6 + W : 1 + 2 * NF>([&](auto ic) { send(ic); });
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

template <int D, bool FP4>
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
        if (prompt_tile<D, FP4, false>(a, seq, kvh, chunk, tile, notes)) prompt_tile<D, FP4, true>(a, seq, kvh, chunk, tile, notes);
        if (!a.paired || 2 * tile < a.col_tiles) break;      // the middle one of an odd number has no partner
        __syncthreads();
    }
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

}  // namespace
}  // namespace gelo
