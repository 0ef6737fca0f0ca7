// Low-rank adapters of many requests beside one projection: Z[i] = base[i] + scale_w (H[i] A_w^T) B_w^T, w = which[i] the adapter of row i.  Parts of the
// columns (the queries, keys and values of a fused projection) have an A each: rows k rank ... (k + 1) rank - 1 of A_w belong to part k.
//
// T = H A_w^T for all parts, in float, d cut over workgroups whose sums lie side by side; then base + scale (T B_w^T).  Bound by the bytes of H, base, Z and the
// adapters.
//   few rows   two launches.  The first takes tiles of 16 rows as they come; a tile's adapters go side by side, rows of others count as zeros and their results are
//              dropped.  The second takes row by row; of small rows it does both.
//   many rows  three: the first puts the rows of an adapter together, 64 to a group (rows that are so already stay in runs); then a tile is a group.
// A row's sums do not go by what the rows around it hold or which adapters they have: each is a column of a matrix instruction.  The order of its sums, and whether T is two bfloat16, go by
// the sizes of the call (plan_of), how many rows and adapters it has among them.
//
// bfloat16 takes v_mfma_f32_16x16x32_bf16, and (many rows) the float T of the second product as two bfloat16, 16 bits of it: with one, its rounding would show where what the
// adapter adds is as large as base.  float takes v_mfma_f32_16x16x4_f32.
#include "gelo_internal.h"

namespace gelo {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;

// 16 bytes of each of 16 rows' contraction values to a lane: PER values, 4 PER to a step
template <class T> struct Lane;
template <> struct Lane<uint16_t> {
    static constexpr int PER = 8;
    typedef bf16x8_t piece_t;
    static __device__ __forceinline__ f32x4_t multiply(piece_t a, piece_t b, f32x4_t sum) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, sum, 0, 0, 0); }
};
template <> struct Lane<float> {
    static constexpr int PER = 4;
    typedef f32x4_t piece_t;
    static __device__ __forceinline__ f32x4_t multiply(piece_t a, piece_t b, f32x4_t sum) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], sum, 0, 0, 0);
        return sum;
    }
};
template <class T> __device__ __forceinline__ typename Lane<T>::piece_t none() {
    return __builtin_bit_cast(typename Lane<T>::piece_t, u32x4_t{0, 0, 0, 0});
}

// lane l's 16 bytes land at lds_addr + 16 l (wave-uniform: it travels in M0)
__device__ __forceinline__ void fetch16(const void* from, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" :: "v"(from), "s"(lds_addr) : "memory", "m0");
}

struct AdaptArgs {
    Adapt o;
    int all;                             // rank n_parts: values of a row of T
    int splits, steps;                   // parts of d, `steps` steps of 4 PER values each
    int wide;                            // columns of a workgroup of the second product: a multiple of 64
    int first_block[kMostParts + 1];     // blocks of so many columns before a part
    float* t;                            // [split][row][all]
    // many rows put in order; null: as they come
    int2* groups;                        // of each group its adapter (-1: none) and how many rows it has; n_groups of them, some have none
    int* order;                          // 64 places to each group
    int n_groups;                        // (a multiple of 8)
    bool by_die;                         // the second product of a group on the die that had its first
};

__device__ __forceinline__ int part_of_block(const AdaptArgs& a, int block) {
    int part = 0;
    while (block >= a.first_block[part + 1]) ++part;
    return part;
}

// The adapters of a tile of 16 rows, one after the other: `left` has a bit for every row still to come.
struct Tile {
    int id;                              // of row lane % 16
    uint32_t left;
    bool live;                           // row lane % 16 has the adapter that next() gave
    __device__ __forceinline__ Tile(const Adapt& o, int tile) {
        const int row = tile * 16 + (threadIdx.x & 15);
        id = row < o.n ? o.which[row] : -1;
        if (id >= o.n_adapters) id = -1;
        left = (uint32_t)__ballot(id >= 0) & 0xFFFFu;
    }
    __device__ __forceinline__ int next() {
        const int w = __builtin_amdgcn_readlane(id, __builtin_ctz(left));
        live = id == w;
        left &= ~(uint32_t)__ballot(live);
        return w;
    }
};

// Few rows, the first product.  A workgroup: one of the adapters of a tile, 64 rows of A, one part of d, whose steps its waves share out.  64 rows with 48 adapters of
// 48 x 4096, a row without now and then: 14 MB in 6.5 us; a smaller part of d makes more of T, which every workgroup of the second product adds up again.
template <class T>
__global__ __launch_bounds__(64 * kWaves)
void adapt_few_down_kernel(AdaptArgs a) {
    typedef Lane<T> L;
    typedef typename L::piece_t piece_t;
    constexpr int STEP = 4 * L::PER, RT = 4, AHEAD = 4;
    const Adapt& o = a.o;
    __shared__ f32x4_t sums[kWaves][RT][64];
    const int tile = blockIdx.x >> 4, slot = blockIdx.x & 15, split = blockIdx.y, first_rank = blockIdx.z * 16 * RT;
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = min((a.all - first_rank + 15) / 16, RT);
    Tile rows(o, tile);
    const int begin = split * a.steps, end = min(begin + a.steps, (o.d + STEP - 1) / STEP);
    const int row = min(tile * 16 + c, o.n - 1);
    const T* h = (const T*)o.H + row * o.ldh;
    for (int k = 0; rows.left; ++k) {
        const int w = rows.next();
        if (k != slot) continue;
        const bool live = rows.live;
        const T* A = (const T*)o.A + w * o.a_stride;
        f32x4_t sum[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) sum[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int s0 = begin + wave * AHEAD; s0 < end; s0 += kWaves * AHEAD) {
            piece_t x[AHEAD], y[AHEAD][RT];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int col = (s0 + u) * STEP + g * L::PER;
                const bool there = s0 + u < end && col < o.d;
                x[u] = none<T>();
                if (there && live) x[u] = *reinterpret_cast<const piece_t*>(h + col);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const int r = first_rank + 16 * t + c;
                    y[u][t] = none<T>();
                    if (there && r < a.all) y[u][t] = *reinterpret_cast<const piece_t*>(A + r * o.lda + col);
                }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int t = 0; t < RT; ++t) sum[t] = L::multiply(y[u][t], x[u], sum[t]);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) sums[wave][t][lane] = sum[t];
        __syncthreads();
        // wave t adds up tile t: rank 16 t + 4 g + r of row c
        if (wave < tiles && live) {
            f32x4_t all = sums[0][wave][lane];
#pragma unroll
            for (int i = 1; i < kWaves; ++i) all += sums[i][wave][lane];
            const int r = first_rank + 16 * wave + 4 * g;
            if (r < a.all) *reinterpret_cast<f32x4_t*>(a.t + ((int64_t)split * o.n + row) * a.all + r) = all;
        }
        return;
    }
}

// A row's PER values of T from `t` on, summed over the parts of d
template <class T>
__device__ __forceinline__ void read_t(const AdaptArgs& a, const float* t, float (&v)[Lane<T>::PER]) {
    constexpr int PER = Lane<T>::PER;
#pragma unroll
    for (int e = 0; e < PER; ++e) v[e] = 0.f;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
#pragma unroll
        for (int e = 0; e < PER; e += 4) {
            const f32x4_t x = *reinterpret_cast<const f32x4_t*>(t + (int64_t)s * a.o.n * a.all + e);
#pragma unroll
            for (int u = 0; u < 4; ++u) v[e + u] += x[u];
        }
    }
}
// as an operand: of bfloat16 the upper part, or (rest) what it leaves, of the same sign and not zero: an infinity in B would be NaN by a zero
__device__ __forceinline__ bf16x8_t piece_of(const float (&v)[8], bool rest) {
    bf16x8_t f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float up = __uint_as_float(__float_as_uint(v[e]) & 0xFFFF0000u);
        const float low = v[e] - up;
        f[e] = (__bf16)(rest && fabsf(v[e]) < __builtin_inff() ? low != 0.f ? low : 0x1p-40f * v[e] : rest || v[e] != v[e] ? v[e] : up);
    }
    return f;
}
__device__ __forceinline__ f32x4_t piece_of(const float (&v)[4], bool) { return f32x4_t{v[0], v[1], v[2], v[3]}; }

// 16 bytes of Z: base's and `by` times what lies at `more`, rounded once
__device__ __forceinline__ void add_to(u32x4_t& x, float by, const float* more, uint16_t) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    const f32x4_t a = *reinterpret_cast<const f32x4_t*>(more), b = *reinterpret_cast<const f32x4_t*>(more + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float m0 = i < 2 ? a[2 * i] : b[2 * i - 4], m1 = i < 2 ? a[2 * i + 1] : b[2 * i - 3];
        const bf16x2_t pair = {(__bf16)(__uint_as_float(x[i] << 16) + by * m0), (__bf16)(__uint_as_float(x[i] & 0xFFFF0000u) + by * m1)};
        x[i] = __builtin_bit_cast(uint32_t, pair);
    }
}
__device__ __forceinline__ void add_to(u32x4_t& x, float by, const float* more, float) {
    const f32x4_t a = *reinterpret_cast<const f32x4_t*>(more);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) + by * a[i]);
}

// Rank values go by pieces of PER; of bfloat16 every one comes twice, its upper parts and the rests.  Ranks of up to 16 put both into one instruction.
template <class T> __device__ __forceinline__ int steps_of_rank(int rank) {
    const int pieces = rank / Lane<T>::PER;
    if (sizeof(T) == 4) return (pieces + 3) / 4;
    return pieces <= 2 ? 1 : 2 * ((pieces + 3) / 4);
}
// Which piece lane g has in step s, and whether it is of the rests; `there`: it has one.
struct Rank { int piece; bool rest, there; };
template <class T> __device__ __forceinline__ Rank rank_of(int rank, int s, int g) {
    const int pieces = rank / Lane<T>::PER, half = (pieces + 3) / 4;
    if (sizeof(T) == 4) return Rank{4 * s + g, false, 4 * s + g < pieces};
    if (pieces <= 2) return Rank{g >= pieces ? g - pieces : g, g >= pieces, g < 2 * pieces};
    const int q = 4 * (s >= half ? s - half : s) + g;
    return Rank{q, s >= half, q < pieces};
}

// Few rows, the second product, as sums of products: a row has its adapter to itself as a rule, and a matrix instruction would multiply 15 rows of zeros.  A
// workgroup: one row, kFewCols columns of one part.  Bound by its trips to memory - whose row, T and B, base: 64 rows with 48 adapters, 12288 columns, rank 16, 17 MB in
// 5.5 us (tiles of matrix instructions 10).  A column's rank values lie side by side: from 64 bytes on LANES = 4 lanes take 16 each, of 8 columns (by a lane alone, two columns: both products of
// 40 rows of 11760 columns, rank 64, 19.8 us, 13.7; of 32 of 12288 21.6, 16.9); fewer belong to one lane (64 rows, rank 16, 11.2 us, 14.9 by four).
constexpr int kFewCols = 512;
// WHOLE: the first product too, in the same launch, by every workgroup for itself: a wave has a quarter of the ranks, its lanes the row's values.
constexpr int kWholeRank = 32;
template <class T, int LANES, bool WHOLE>
__global__ __launch_bounds__(256, WHOLE ? 4 : 1)
void adapt_few_up_kernel(AdaptArgs a) {
    const Adapt& o = a.o;
    __shared__ __attribute__((aligned(16))) float t[kMostRank], sums[kFewCols];          // the row's T, and what it adds
    const int blocks = a.first_block[o.n_parts], row = blockIdx.x / blocks, block = blockIdx.x - row * blocks;
    const int id = o.which[row], part = part_of_block(a, block);
    const int first = (part > 0 ? o.part_end[part - 1] : 0) + kFewCols * (block - a.first_block[part]), end = o.part_end[part], col = first + 2 * threadIdx.x;
    const bool in = col < end, has = id >= 0 && id < o.n_adapters;
    if (!has && o.base == o.Z) return;
    typedef T pair_t __attribute__((ext_vector_type(2)));
    pair_t x = {};
    if (in) x = *reinterpret_cast<const pair_t*>((const T*)o.base + row * o.ldb + col);
    if (has) {
        constexpr int PER = 16 / sizeof(T), SLOTS = 256 / LANES, COLS = kFewCols / SLOTS;
        const int q = threadIdx.x % LANES, slot = threadIdx.x / LANES, pieces = o.rank / PER;
        constexpr int DEEP = LANES == 1 ? 2 : 1, APART = LANES == 1 ? 1 : SLOTS;               // pieces sent for together; from one column of a lane to its next
        // (columns behind the last one: that one again; what comes of them is not used)
        const int my_first = first + (LANES == 1 ? COLS * slot : slot);
        const T* B = (const T*)o.B + id * o.b_stride;
        u32x4_t y[DEEP][COLS];
        auto read = [&](int piece) {
#pragma unroll
            for (int u = 0; u < DEEP; ++u) {
                if (piece + u >= pieces) break;
#pragma unroll
                for (int k = 0; k < COLS; ++k) y[u][k] = *reinterpret_cast<const u32x4_t*>(B + min(my_first + k * APART, end - 1) * o.ldbw + (piece + u) * PER);
            }
        };
        read(q);
        if constexpr (WHOLE) {
            constexpr int MINE = kWholeRank / 4;
            const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = o.rank / 4;
            const T* h = (const T*)o.H + row * o.ldh;
            const T* A = (const T*)o.A + id * o.a_stride + (part * o.rank + wave * mine) * o.lda;
            float sum[MINE];
#pragma unroll
            for (int r = 0; r < MINE; ++r) sum[r] = 0.f;
            auto value = [](const u32x4_t& v, int e) {
                return sizeof(T) == 4 ? __uint_as_float(v[e & 3]) : __uint_as_float(e & 1 ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16);
            };
#pragma unroll 2
            for (int c = PER * lane; c < o.d; c += 64 * PER) {
                const u32x4_t x = *reinterpret_cast<const u32x4_t*>(h + c);
                u32x4_t w[MINE];
#pragma unroll
                for (int r = 0; r < MINE; ++r)
                    if (r < mine) w[r] = *reinterpret_cast<const u32x4_t*>(A + r * o.lda + c);
#pragma unroll
                for (int r = 0; r < MINE; ++r) {
                    if (r >= mine) break;
#pragma unroll
                    for (int e = 0; e < PER; ++e) sum[r] += value(x, e) * value(w[r], e);
                }
            }
#pragma unroll
            for (int r = 0; r < MINE; ++r) {
                if (r >= mine) break;
#pragma unroll
                for (int by = 1; by < 64; by *= 2) sum[r] += __shfl_xor(sum[r], by, 64);
                if (lane == 0) t[wave * mine + r] = sum[r];
            }
        } else if ((int)threadIdx.x < o.rank) {
            float sum = 0.f;
            const float* from = a.t + (int64_t)row * a.all + part * o.rank + threadIdx.x;
#pragma unroll 8
            for (int s = 0; s < a.splits; ++s) sum += from[(int64_t)s * o.n * a.all];
            t[threadIdx.x] = sum;
        }
        const float scale = o.scale ? o.scale[id] : 1.f;
        __syncthreads();
        float sum[COLS];
#pragma unroll
        for (int k = 0; k < COLS; ++k) sum[k] = 0.f;
        for (int piece = q; piece - q < pieces; piece += LANES * DEEP) {
#pragma unroll
            for (int u = 0; u < DEEP; ++u) {
                if (piece + u >= pieces) break;
                float with[PER];
#pragma unroll
                for (int e = 0; e < PER; e += 4) *reinterpret_cast<f32x4_t*>(with + e) = *reinterpret_cast<const f32x4_t*>(t + (piece + u) * PER + e);
#pragma unroll
                for (int k = 0; k < COLS; ++k)
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        sum[k] += with[e] * (sizeof(T) == 4 ? __uint_as_float(y[u][k][e & 3]) : __uint_as_float(e & 1 ? y[u][k][e >> 1] & 0xFFFF0000u : y[u][k][e >> 1] << 16));
            }
            read(piece + LANES * DEEP);
        }
        if constexpr (LANES > 1) {
#pragma unroll
            for (int k = 0; k < COLS; ++k) {
#pragma unroll
                for (int by = 1; by < LANES; by *= 2) sum[k] += __shfl_xor(sum[k], by, 64);
                if (q == 0) sums[slot + k * SLOTS] = sum[k];
            }
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float more = scale * (LANES > 1 ? sums[2 * threadIdx.x + k] : sum[k]);
            if constexpr (sizeof(T) == 4) x[k] += more;
            else x[k] = __builtin_bit_cast(uint16_t, (__bf16)(__uint_as_float((uint32_t)x[k] << 16) + more));
        }
    }
    if (in) *reinterpret_cast<pair_t*>((T*)o.Z + row * o.ldz + col) = x;
}

// Many rows: which go together.  One workgroup counts the rows of every adapter (and of none), deals out groups, and puts the rows into their places; where
// among its adapter's a row comes goes by the order of atomic additions, and nothing goes by that.  Groups of one adapter have numbers 8 apart: workgroups of such numbers
// meet on one die, whose L2 then has what they share.
constexpr int kOrderThreads = 1024, kMostBins = 12288, kGroup = 64;
__global__ __launch_bounds__(kOrderThreads)
void adapt_order_kernel(AdaptArgs a) {
    const Adapt& o = a.o;
    __shared__ int bins[kMostBins];
    __shared__ int sums[kOrderThreads / 64];
    const int n_bins = o.n_adapters + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto bin_of = [&](int w) { return w >= 0 && w < o.n_adapters ? w : o.n_adapters; };
    for (int i = threadIdx.x; i < n_bins; i += kOrderThreads) bins[i] = 0;
    __syncthreads();
    // Adds the rows of a wave to their bins and returns where each comes.  Rows of one adapter side by side are one addition: as many from one address are one after
    // the other.
    auto add = [&](int bin, bool there) -> int {
        const uint64_t all = __ballot(there);
        if (!all) return 0;
        const int leader = __builtin_ctzll(all), same = __builtin_amdgcn_readlane(bin, leader);
        if ((__ballot(bin == same) & all) != all) return there ? atomicAdd(&bins[bin], 1) : 0;
        int first = 0;
        if (lane == leader) first = atomicAdd(&bins[same], __popcll(all));
        return __builtin_amdgcn_readlane(first, leader) + __popcll(all & ((1ull << lane) - 1));
    };
    const int rounds = (o.n + kOrderThreads - 1) / kOrderThreads;
    auto row_of = [&](int i) { return i * kOrderThreads + (int)threadIdx.x; };
    auto read = [&](int i) { return row_of(i) < o.n ? bin_of(o.which[row_of(i)]) : 0; };
    constexpr int KEPT = 8;                                  // rounds whose numbers and places stay in registers: the last places of their bins
    int kept[KEPT], place[KEPT];
#pragma unroll
    for (int i = 0; i < KEPT; ++i) kept[i] = read(i);
    for (int i = KEPT; i < rounds; ++i) add(read(i), row_of(i) < o.n);
    if (rounds > KEPT) __syncthreads();
#pragma unroll
    for (int i = 0; i < KEPT; ++i) place[i] = i < rounds ? add(kept[i], row_of(i) < o.n) : 0;
    __syncthreads();
    // groups before each thread's bins
    const int each = (n_bins + kOrderThreads - 1) / kOrderThreads, first = threadIdx.x * each, last = min(first + each, n_bins);
    int mine = 0;
    for (int i = first; i < last; ++i) mine += (bins[i] + kGroup - 1) / kGroup;
    int upto = mine;
    for (int by = 1; by < 64; by *= 2) {
        const int x = __shfl_up(upto, by, 64);
        if (lane >= by) upto += x;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int before = upto - mine, groups = 0;
    for (int i = 0; i < kOrderThreads / 64; ++i) {
        if (i < wave) before += sums[i];
        groups += sums[i];
    }
    const int to_die = (groups + 7) / 8;
    auto number = [&](int k) { return k % to_die * 8 + k / to_die; };            // of the k-th group
    for (int i = threadIdx.x; i < a.n_groups; i += kOrderThreads)
        if (i >> 3 >= to_die || (i & 7) * to_die + (i >> 3) >= groups) a.groups[i] = int2{-1, 0};
    for (int j = 0; j < each; ++j) {
        const int i = first + j, count = i < last ? bins[i] : 0, w = i < o.n_adapters ? i : -1, in_bin = (count + kGroup - 1) / kGroup;
        if (i < last) bins[i] = before * kGroup;
        auto put = [&](int k, int w, int before, int count) { a.groups[number(before + k)] = int2{w, min(count - kGroup * k, kGroup)}; };
        constexpr int FEW = 4;
        for (int k = 0; k < min(in_bin, FEW); ++k) put(k, w, before, count);
        // the other groups of a large bin: its wave
        for (uint64_t large = __ballot(in_bin > FEW); large; large &= large - 1) {
            const int from = __builtin_ctzll(large), all = __shfl(in_bin, from, 64), c = __shfl(count, from, 64), its = __shfl(w, from, 64), at = __shfl(before, from, 64);
            for (int k = FEW + lane; k < all; k += 64) put(k, its, at, c);
        }
        before += in_bin;
    }
    __syncthreads();
    auto put = [&](int i, int at) {
        if (row_of(i) < o.n) a.order[number(at / kGroup) * kGroup + at % kGroup] = row_of(i);
    };
#pragma unroll
    for (int i = 0; i < KEPT; ++i) if (i < rounds) put(i, bins[kept[i]] + place[i]);
    if (rounds <= KEPT) return;
    __syncthreads();
    for (int i = KEPT; i < rounds; ++i) put(i, add(read(i), row_of(i) < o.n));
}

// Rows `first` ... of a group, or, where none were made, of 64 rows as they come, up to SIZE of them: lane l of a wave has row l (the last one's again behind the last),
// its adapter, and whether there is one.
template <int SIZE>
struct Some {
    int count, id, row;
    uint64_t left;                       // rows of adapters still to come
    __device__ __forceinline__ bool find(const AdaptArgs& a, int at, int first) {
        const int lane = threadIdx.x & 63;
        if (a.groups) {
            const int2 group = a.groups[at];
            row = a.order[at * kGroup + first + min(lane, SIZE - 1)];
            count = min(group.y - first, SIZE);
            if (count <= 0) return false;
            const int end = __builtin_amdgcn_readlane(row, count - 1);
            row = lane < count ? row : end;
            id = lane < count ? group.x : -1;
        } else {
            count = min(a.o.n - at * kGroup - first, SIZE);
            if (count <= 0) return false;
            row = at * kGroup + first + min(lane, count - 1);
            id = lane < count ? a.o.which[row] : -1;
        }
        return true;
    }
    // (apart, so that loads of rows do not wait for their numbers)
    __device__ __forceinline__ void look(const AdaptArgs& a) {
        if (id >= a.o.n_adapters) id = -1;
        left = __ballot(id >= 0);
    }
    __device__ __forceinline__ int next(uint64_t* those) {
        const int w = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        *those = __ballot(id == w);
        left &= ~*those;
        return w;
    }
};

// Many rows, the first product.  A workgroup: one group, 64 rows of A, one part of d, whose steps its waves share out.  Columns of rows of other adapters come
// out as they may and are not kept, so the rows are sent for before their adapters are known.  Neighbouring groups go to one die: its L2 then has their A.  A wave's piece of H
// lies in its registers, that of A in its own part of LDS, put there by loads that need no registers: all of it is one trip to memory (tile after tile of A
// through registers, a trip each, 2048 rows of 4096 values, rank 64: 12.8 us, 9.7).  (16 rows and all of d to a workgroup: every 16 rows read A for themselves, 4096 rows 26 us instead of 13.
// Half as many waves: twice the parts of d, which the second product reads once for each of its workgroups, 60 instead of 57.5 for both.)
constexpr int kDownWaves = 8, kDownWaveLds = 16 * 1024;
template <class T>
__global__ __launch_bounds__(64 * kDownWaves, 2)
void adapt_many_down_kernel(AdaptArgs a) {
    typedef Lane<T> L;
    typedef typename L::piece_t piece_t;
    constexpr int STEP = 4 * L::PER, RT = 4, HT = kGroup / 16, AHEAD = 4;
    static_assert(RT * AHEAD * 1024 == kDownWaveLds && HT * RT * 1024 == kDownWaveLds, "");
    const Adapt& o = a.o;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Some<kGroup> rows;
    // (rows as they come: neighbours to one die, as the order has it)
    if (!rows.find(a, a.groups ? blockIdx.x : (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3), 0)) return;
    const int split = blockIdx.y, first_rank = blockIdx.z * 16 * RT;
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rank_tiles = min((a.all - first_rank + 15) / 16, RT);
    const int begin = split * a.steps, end = min(begin + a.steps, (o.d + STEP - 1) / STEP);
    const int each = min((a.steps + kDownWaves - 1) / kDownWaves, AHEAD);        // steps of a wave at a time
    uint8_t* mine = lds + wave * kDownWaveLds;
    const uint32_t mine_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)mine;
    const T* h[HT];
#pragma unroll
    for (int i = 0; i < HT; ++i) h[i] = (const T*)o.H + __shfl(rows.row, 16 * i + c, 64) * o.ldh;
    piece_t x[AHEAD][HT];
    auto read_h = [&](int s0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int col = (s0 + u) * STEP + g * L::PER;
#pragma unroll
            for (int i = 0; i < HT; ++i) {
                x[u][i] = none<T>();
                if (s0 + u < min(s0 + each, end) && col < o.d) x[u][i] = *reinterpret_cast<const piece_t*>(h[i] + col);
            }
        }
    };
    const int first = begin + wave * each;
    read_h(first);
    rows.look(a);
    bool there = true;
    while (rows.left) {
        uint64_t those;
        const int w = rows.next(&those);
        const T* A = (const T*)o.A + w * o.a_stride;
        f32x4_t sum[HT][RT];
#pragma unroll
        for (int i = 0; i < HT; ++i)
#pragma unroll
            for (int t = 0; t < RT; ++t) sum[i][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int s0 = first; s0 < end; s0 += kDownWaves * each) {
            const int upto = min(s0 + each, end);
            // what the wave multiplies lies in its own part of LDS, as its lanes take it (behind A's rows and columns: the last ones again)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if (t >= rank_tiles) break;
                const T* from = A + min(first_rank + 16 * t + c, a.all - 1) * o.lda;
#pragma unroll
                for (int u = 0; u < AHEAD; ++u)
                    if (s0 + u < upto) fetch16(from + min((s0 + u) * STEP + g * L::PER, o.d - L::PER), mine_at + (t * AHEAD + u) * 1024);
            }
            if (!there) read_h(s0);
            there = end - first <= kDownWaves * each;       // nothing came behind them: another adapter finds them there
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if (t >= rank_tiles) break;
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    piece_t y = *reinterpret_cast<const piece_t*>(mine + (t * AHEAD + u) * 1024 + 16 * lane);
                    if (s0 + u >= upto || (s0 + u) * STEP + g * L::PER >= o.d) y = none<T>();
#pragma unroll
                    for (int i = 0; i < HT; ++i) sum[i][t] = L::multiply(y, x[u][i], sum[i][t]);
                }
            }
        }
        // through LDS: wave 2 i + t % 2 and the next add up tile i of rows and t of ranks: rank 16 t + 4 g + r of row c
#pragma unroll
        for (int i = 0; i < HT; ++i)
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if (t >= rank_tiles) break;
                *reinterpret_cast<f32x4_t*>(mine + (i * RT + t) * 1024 + 16 * lane) = sum[i][t];
            }
        __syncthreads();
#pragma unroll
        for (int e = wave; e < HT * RT; e += kDownWaves) {
            const int i = e / RT, t = e % RT, r = first_rank + 16 * t + 4 * g, row = __shfl(rows.row, 16 * i + c, 64);
            if (t >= rank_tiles || r >= a.all || !((those >> (16 * i + c)) & 1)) continue;
            f32x4_t all = *reinterpret_cast<const f32x4_t*>(lds + e * 1024 + 16 * lane);
#pragma unroll
            for (int k = 1; k < kDownWaves; ++k) all += *reinterpret_cast<const f32x4_t*>(lds + k * kDownWaveLds + e * 1024 + 16 * lane);
            *reinterpret_cast<f32x4_t*>(a.t + ((int64_t)split * o.n + row) * a.all + r) = all;
        }
        if (rows.left) __syncthreads();                      // nobody reads what the next adapter's rows overwrite
    }
}

// Many rows, the second product.  A workgroup: half a group, 256 columns of one part, 64 to a wave.  What the matrix instructions leave goes through LDS, so that base is read
// and Z written a row's 256 columns at a time (4096 x 12288 values in and out: 36 us; as the instructions leave them, 16 rows at a time, 41 to 45).  The workgroups of a
// row's columns come one after the other, for memory's sake too (42 where those of a column do).  Where T is a large part of what is read (by_die) they do so on the die whose L2
// has the row's T, each die at rows of its own: 2048 rows of 4096 columns, rank 64, eight parts of d 29.1 us for both products and 26.0; 4096 rows of 12288, rank 16, four 57.3
// and 59.6.  HALF: steps of a rank's upper parts at most.
constexpr int kUpRows = 32, kUpCols = 256;
template <class T, int HALF>
__global__ __launch_bounds__(64 * kWaves, HALF == 1 && sizeof(T) == 2 ? 4 : HALF <= 2 ? 3 : 2)
void adapt_many_up_kernel(AdaptArgs a) {
    typedef Lane<T> L;
    typedef typename L::piece_t piece_t;
    constexpr int PER = L::PER, HT = kUpRows / 16, TWICE = sizeof(T) == 2 ? 2 : 1, THREADS = 64 * kWaves;
    constexpr int VEC = 16 / sizeof(T), TO_ROW = kUpCols / VEC, VECS = kUpRows * TO_ROW / THREADS;         // 16 bytes of a row to a thread
    static_assert(4 * PER * (HALF / 2) < kMostRank, "no rank has so many steps");
    const Adapt& o = a.o;
    __shared__ piece_t z[TWICE * HALF][HT][64];
    __shared__ __attribute__((aligned(16))) float sums[kUpRows][kUpCols + 4];
    const int blocks = a.first_block[o.n_parts], halves = kGroup / kUpRows;
    int block = blockIdx.x % blocks, of_rows = blockIdx.x / blocks;
    if (a.by_die) {
        const int die = blockIdx.x & 7, k = blockIdx.x >> 3, j = k / blocks / halves;
        block = k % blocks;
        of_rows = (a.groups ? 8 * j + die : die * (a.n_groups >> 3) + j) * halves + k / blocks % halves;
    }
    Some<kUpRows> rows;
    if (!rows.find(a, of_rows / halves, kUpRows * (of_rows % halves))) return;
    const bool in_place = o.base == o.Z;
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = part_of_block(a, block);
    const int first = (part > 0 ? o.part_end[part - 1] : 0) + a.wide * (block - a.first_block[part]), end = min(first + a.wide, o.part_end[part]);
    const int pieces = o.rank / PER, steps = steps_of_rank<T>(o.rank), half = (pieces + 3) / 4;
    // base: 16 bytes of row i of the group, 256 columns at a time
    u32x4_t x[VECS];
    auto read = [&](int at) {
#pragma unroll
        for (int k = 0; k < VECS; ++k) {
            const int e = threadIdx.x + k * THREADS, i = e / TO_ROW, col = at + VEC * (e - i * TO_ROW);
            const int64_t row = __shfl(rows.row, i, 64);
            if (col < end && i < rows.count) x[k] = *reinterpret_cast<const u32x4_t*>((const T*)o.base + row * o.ldb + col);
        }
    };
    read(first);
    rows.look(a);
    const uint64_t with = rows.left;                         // rows that have an adapter
    // a row's factor, for its sums as a whole: T times one could leave float's range where the sums do not (T times it, eight values to a thread, was 1 to 3% less time)
    const float factor = rows.id >= 0 && o.scale ? o.scale[rows.id] : 1.f;
    // one row's PER rank values to a thread, those of a row side by side (what a row without an adapter has there is not used)
    const int slots = 4 * half;                              // pieces, and nothing to fill a step up with
    for (int e = threadIdx.x; e < kUpRows * slots; e += THREADS) {
        const int i = e / slots, q = e - i * slots, to = i & 15;
        const int row = __shfl(rows.row, i, 64);
        float v[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) v[k] = 0.f;
        if (q < pieces) read_t<T>(a, a.t + (int64_t)row * a.all + part * o.rank + q * PER, v);
        if constexpr (sizeof(T) == 4) {
            z[q >> 2][i >> 4][16 * (q & 3) + to] = piece_of(v, false);
        } else if (pieces <= 2) {
            // upper parts, rests, nothing
            if (q < pieces) {
                z[0][i >> 4][16 * q + to] = piece_of(v, false);
                z[0][i >> 4][16 * (pieces + q) + to] = piece_of(v, true);
            } else if (q >= 2 * pieces) {
                z[0][i >> 4][16 * q + to] = none<T>();
            }
        } else {
            z[q >> 2][i >> 4][16 * (q & 3) + to] = piece_of(v, false);
            z[half + (q >> 2)][i >> 4][16 * (q & 3) + to] = piece_of(v, true);
        }
    }
    piece_t y[HALF][4];
    auto read_b = [&](int w, int at) {
        const T* B = (const T*)o.B + w * o.b_stride;
#pragma unroll
        for (int s = 0; s < HALF; ++s) {
            if (s >= half) break;
            const Rank r = rank_of<T>(o.rank, s, g);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int j = at + 64 * wave + 16 * t + c;
                y[s][t] = none<T>();
                if (r.there && j < end) y[s][t] = *reinterpret_cast<const piece_t*>(B + j * o.ldbw + r.piece * PER);
            }
        }
    };
    Some<kUpRows> of = rows;
    uint64_t those = 0;
    const int w0 = with ? of.next(&those) : 0;
    const bool alone = those == with;                        // one adapter at most
    if (with && alone) read_b(w0, first);
    for (int at = first; at < end; at += kUpCols) {
        __syncthreads();
        if (with) {
#pragma unroll
            for (int i = 0; i < HT; ++i) {
                f32x4_t sum[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) sum[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                of = rows;
                of.left &= 0xFFFFull << (16 * i);            // this tile's rows
                while (of.left) {
                    const int w = of.next(&those);
                    of.left &= 0xFFFFull << (16 * i);
                    if (!alone) read_b(w, at);
                    const bool live = alone || ((those >> (16 * i + c)) & 1);
#pragma unroll
                    for (int s = 0; s < HALF; ++s) {
                        if (s >= half) break;
                        for (int k = s; k < steps; k += half) {
                            const piece_t zi = z[k][i][lane];
#pragma unroll
                            for (int t = 0; t < 4; ++t) {
                                const f32x4_t more = L::multiply(y[s][t], zi, sum[t]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) sum[t][e] = live ? more[e] : sum[t][e];
                            }
                        }
                    }
                }
                // columns 16 t + 4 g ... of row c
#pragma unroll
                for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4_t*>(&sums[16 * i + c][64 * wave + 16 * t + 4 * g]) = sum[t];
            }
        }
        if (with && alone && at + kUpCols < end) read_b(w0, at + kUpCols);
        __syncthreads();
        u32x4_t was[VECS];
#pragma unroll
        for (int k = 0; k < VECS; ++k) was[k] = x[k];
        if (at + kUpCols < end) read(at + kUpCols);
#pragma unroll
        for (int k = 0; k < VECS; ++k) {
            const int e = threadIdx.x + k * THREADS, i = e / TO_ROW, col = at + VEC * (e - i * TO_ROW);
            const int64_t row = __shfl(rows.row, i, 64);
            const bool has = (with >> i) & 1;
            const float by = __shfl(factor, i, 64);
            if (col >= end || i >= rows.count || (!has && in_place)) continue;
            if (has) add_to(was[k], by, &sums[i][col - at], T());
            *reinterpret_cast<u32x4_t*>((T*)o.Z + row * o.ldz + col) = was[k];
        }
    }
}

int steps_of(int is_bf16, int d) { return (d + (is_bf16 ? 31 : 15)) / (is_bf16 ? 32 : 16); }

// Rows by themselves read their adapters at 7.5 TB/s, from L2 for the most part; groups take three launches and their trips, 10 us more, and read an adapter once for 64
// rows.  4096 -> 12288 columns, rank 16, one adapter, us by rows and by groups: 64 rows 10.9 and 16.2, 96 (75 MB) 16.5 and 16.4, 128 18.2 and 16.4, 256 28.2 and 17.4; 4096 ->
// 4096, rank 128, 64 rows (134 MB) 22.4 and 20.9; 1024 -> 1024, rank 8, 1024 rows (34 MB) 10.9 and 19.3.
// All this goes by how many adapters are described: which of them a batch uses, and in what order, is on the GPU.  The more there are, the more groups there could be, whose workgroups start
// to find nothing, and the counts fit no more than kMostBins: 4096 rows in runs of eight adapters, 4096 -> 12288 columns, rank 16, one set of inputs again and again, 51 us where 8 are described, 60 with
// 9 or 64, 153 with 12287, 326 with 12288, where every row reads its own.
constexpr double kRowsRead = 80e6, kOrderedRead = 110e6;
// Putting rows in order is a launch of 4 to 6 us, and what follows finds its rows a trip later.  Without it a group's adapters follow each other, each a trip to its B and so many more
// instructions.  4096 -> 12288 columns, rank 16, us in order and as they come: 1024 rows of eight adapters in any order 29 and 44, of four 31 as they come; 4096 rows of eight in any
// order 67 and 92, in runs 67 and 57.  So many rows are prompts, whose rows lie side by side, more often than not - but at high ranks a wrong guess costs more: 4096 rows of 2048 values, 2048
// columns, eight adapters of rank 64 in any order 33 and 63, in runs 33 and 25, of rank 128 43 and 101, 43 and 35.
int few_adapters(int n, int rank) { return n >= 2048 && rank <= 32 ? 8 : 4; }
struct Plan { bool many, ordered, by_die, whole; int splits, steps, wide; int64_t most_groups, t_bytes, bytes; };
Plan plan_of(int is_bf16, int n, int d, int p, int rank, int n_parts, int n_adapters) {
    Plan r;
    const double read = (double)n * rank * ((double)n_parts * d + p) * (is_bf16 ? 2 : 4);
    r.many = n_adapters < kMostBins && read > (n_adapters > few_adapters(n, rank) ? kOrderedRead : kRowsRead);
    r.ordered = r.many && n_adapters > few_adapters(n, rank);
    const int all = steps_of(is_bf16, d), rank_groups = (rank * n_parts + 63) / 64;
    const int64_t rows = n, groups = (rows + kGroup - 1) / kGroup;      // (what is added to n may leave 32 bits; adapt_fits refuses such calls, from what is reckoned here)
    const int64_t alone = n_adapters < n ? n_adapters + 1 : n;          // groups that are not full
    r.most_groups = round_up(r.ordered ? rows / kGroup + alone : r.many ? groups : 0, 8);
    // workgroups that fill the chip with the first product, of 8 waves or (few rows, which have an adapter each as a rule) 4; two steps to a wave at least, or four
    const int64_t items = (r.many ? groups : rows) * rank_groups, target = r.many ? 256 : 512;
    int64_t cuts = items >= target ? 1 : target / items;
    const int to_each = r.many ? 2 * kDownWaves : 4 * kWaves, most = (all + to_each - 1) / to_each;
    cuts = cuts < most ? cuts : most;
    cuts = cuts < (r.many ? 8 : 16) ? cuts : (r.many ? 8 : 16);
    r.steps = (int)((all + cuts - 1) / cuts);
    r.splits = (all + r.steps - 1) / r.steps;
    // two blocks of columns to a workgroup of the second product where that leaves 512 of them: it reads T once (4096 rows, us: 62 with one, 57.5, 61 with four; 1024 rows of
    // 12288 columns, 768 workgroups, 34.4 and 32.0)
    r.wide = kFewCols;
    if (r.many) for (r.wide = 2 * kUpCols; r.wide > kUpCols && (rows + kUpRows - 1) / kUpRows * ((p + r.wide - 1) / r.wide) < 512;) r.wide /= 2;
    // One launch for small rows: every workgroup of the second product reads A once more, a few trips one behind the other.  16 rows, us in two launches and in one: of 256 values, rank 16 6.3
    // and 4.3; 1024, rank 32 8.1 and 7.1; 2048, rank 16 7.1 and 6.5, rank 32 8.7 and 9.4; 4096, rank 8 6.5 and 7.3; 256 rows of 2048, 67 MB, 9.9 and 8.7.
    const double row_bytes = (double)d * (is_bf16 ? 2 : 4), reads = rank * row_bytes;
    r.whole = !r.many && rank <= kWholeRank && row_bytes <= 4096 && reads <= 65536 && reads * n * ((p + kFewCols - 1) / kFewCols + n_parts - 1) <= 70e6;
    // (T goes to 8 dies otherwise: where that is a fifth of base and Z)
    r.by_die = 5 * 8 * r.splits * rank * n_parts * (int64_t)sizeof(float) > 2 * (int64_t)p * (is_bf16 ? 2 : 4);
    r.t_bytes = round_up((int64_t)r.splits * n * rank * n_parts * sizeof(float), 256);
    r.bytes = r.t_bytes + (r.ordered ? (8 + 4 * kGroup) * r.most_groups : 0);
    return r;
}

template <class T>
hipError_t launch(const Adapt& o, hipStream_t stream) {
    AdaptArgs a;
    a.o = o;
    a.all = o.rank * o.n_parts;
    const Plan p = plan_of(sizeof(T) == 2, o.n, o.d, o.p, o.rank, o.n_parts, o.n_adapters);
    a.splits = p.splits; a.steps = p.steps; a.wide = p.wide; a.by_die = p.by_die;
    a.first_block[0] = 0;
    for (int k = 0; k < kMostParts; ++k)
        a.first_block[k + 1] = a.first_block[k] + (k < o.n_parts ? (o.part_end[k] - (k ? o.part_end[k - 1] : 0) + a.wide - 1) / a.wide : 0);
    const int blocks = a.first_block[o.n_parts], rank_groups = (a.all + 63) / 64;
    uint8_t* ws = (uint8_t*)o.workspace;
    a.t = (float*)ws;
    a.n_groups = (int)p.most_groups;
    a.groups = p.ordered ? (int2*)(ws + p.t_bytes) : nullptr;
    a.order = (int*)(ws + p.t_bytes + 8 * p.most_groups);
    if (p.many) {
        if (p.ordered) hipLaunchKernelGGL(adapt_order_kernel, dim3(1), dim3(kOrderThreads), 0, stream, a);
        hipLaunchKernelGGL(adapt_many_down_kernel<T>, dim3((unsigned)p.most_groups, a.splits, rank_groups), dim3(64 * kDownWaves), kDownWaves * kDownWaveLds, stream, a);
        const dim3 up((unsigned)(kGroup / kUpRows * p.most_groups * blocks));
        const int half = (o.rank + 4 * Lane<T>::PER - 1) / (4 * Lane<T>::PER);
        if (half <= 1) hipLaunchKernelGGL((adapt_many_up_kernel<T, 1>), up, dim3(64 * kWaves), 0, stream, a);
        else if (half <= 2) hipLaunchKernelGGL((adapt_many_up_kernel<T, 2>), up, dim3(64 * kWaves), 0, stream, a);
        else if (half <= 4) hipLaunchKernelGGL((adapt_many_up_kernel<T, 4>), up, dim3(64 * kWaves), 0, stream, a);
        else if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((adapt_many_up_kernel<T, 8>), up, dim3(64 * kWaves), 0, stream, a);
        return hipGetLastError();
    }
    const int tiles = (o.n + 15) / 16;
    if (!p.whole) hipLaunchKernelGGL(adapt_few_down_kernel<T>, dim3(tiles * 16, a.splits, rank_groups), dim3(64 * kWaves), 0, stream, a);
    const dim3 up((unsigned)(blocks * o.n));
    const int pieces = o.rank / (16 / (int)sizeof(T));
    if (p.whole && pieces < 4) hipLaunchKernelGGL((adapt_few_up_kernel<T, 1, true>), up, dim3(256), 0, stream, a);
    else if (p.whole) hipLaunchKernelGGL((adapt_few_up_kernel<T, 4, true>), up, dim3(256), 0, stream, a);
    else if (pieces < 4) hipLaunchKernelGGL((adapt_few_up_kernel<T, 1, false>), up, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((adapt_few_up_kernel<T, 4, false>), up, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

bool adapt_fits(const Adapt& o, int is_bf16) {
    const Plan p = plan_of(is_bf16, o.n, o.d, o.p, o.rank, o.n_parts, o.n_adapters);
    const int64_t blocks = o.p / p.wide + o.n_parts, most = kMostThreads / (64 * kWaves), rank_groups = (o.rank * o.n_parts + 63) / 64;
    if (p.many) return kGroup / kUpRows * p.most_groups * blocks <= most && 2 * p.most_groups * p.splits * rank_groups <= most;
    const int64_t tiles = ((int64_t)o.n + 15) / 16;
    return o.n * blocks <= most && 16 * tiles * p.splits * rank_groups <= most;
}

size_t adapt_workspace_bytes(const Adapt& o, int is_bf16) { return (size_t)plan_of(is_bf16, o.n, o.d, o.p, o.rank, o.n_parts, o.n_adapters).bytes; }
// What any call of up to so many rows, ranks and adapters needs: the parts of d are at most 512 over the workgroups of one part, of 1 row, or 256, of 64.
size_t adapt_workspace_bound(int n, int rank, int n_parts, int n_adapters) {
    const int64_t grouped = 8 * (int64_t)n < 256 * kGroup ? 8 * (int64_t)n : 256 * kGroup, alone = n_adapters < n ? n_adapters + 1 : n;
    int64_t rows = grouped > 512 ? grouped : 512;
    if (rows < n) rows = n;
    return (size_t)(round_up(rows * rank * n_parts * (int64_t)sizeof(float), 256) + (8 + 4 * kGroup) * round_up(n / kGroup + alone, 8));
}
// Which way a call of these sizes goes: 0 rows by themselves, 1 groups of rows as they come, 2 groups of rows put in order.  adapt_launches: in so many.
int adapt_launches(int is_bf16, int n, int d, int p, int rank, int n_parts, int n_adapters) {
    const Plan r = plan_of(is_bf16, n, d, p, rank, n_parts, n_adapters);
    return r.whole ? 1 : 2 + r.ordered;
}
int adapt_way(int is_bf16, int n, int d, int p, int rank, int n_parts, int n_adapters) {
    const Plan r = plan_of(is_bf16, n, d, p, rank, n_parts, n_adapters);
    return r.many + r.ordered;
}

// adapt_workspace_bytes of these sizes
size_t adapt_needs(int is_bf16, int n, int d, int p, int rank, int n_parts, int n_adapters) {
    return (size_t)plan_of(is_bf16, n, d, p, rank, n_parts, n_adapters).bytes;
}

hipError_t adapt_init() {
    const hipError_t e = hipFuncSetAttribute((const void*)&adapt_many_down_kernel<uint16_t>, hipFuncAttributeMaxDynamicSharedMemorySize, kDownWaves * kDownWaveLds);
    return e != hipSuccess ? e : hipFuncSetAttribute((const void*)&adapt_many_down_kernel<float>, hipFuncAttributeMaxDynamicSharedMemorySize, kDownWaves * kDownWaveLds);
}

hipError_t adapt(const Adapt& o, int is_bf16, hipStream_t stream) { return is_bf16 ? launch<uint16_t>(o, stream) : launch<float>(o, stream); }

}  // namespace gelo
