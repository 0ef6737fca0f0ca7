// Low-rank adapters of many requests beside one projection: Z[i] = base[i] + scale_w (H[i] A_w^T) B_w^T, w = which[i] the adapter of row i.  Parts of the
// columns (the queries, keys and values of a fused projection) have an A each: rows k rank ... (k + 1) rank - 1 of A_w belong to part k.
//
// Two launches: T = H A_w^T for all parts, in float, cut over d where rows are few; then base + scale T B_w^T.  Bound by the bytes of H, base, Z and the
// adapters.  Rows go 16 to a tile, one of a tile's adapters after another: rows of other adapters count as zeros there, and their results are dropped.
//
// bfloat16 takes v_mfma_f32_16x16x32_bf16, and the float T of the second product as two bfloat16, 16 bits of it: with one, its rounding would show where what the
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

struct AdaptArgs {
    Adapt o;
    int all;                             // rank n_parts: values of a row of T
    int slots, splits, steps;            // workgroups that share a tile's adapters; parts of d, `steps` steps of 4 PER values each
    int first_group[kMostParts + 1];     // groups of 64 columns before a part
};

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

// T[split][row][rank of all parts].  A workgroup: the adapters of one tile from `slot` on, 64 rows of A, one part of d, whose steps its waves share out.
template <class T>
__global__ __launch_bounds__(64 * kWaves)
void adapt_down_kernel(AdaptArgs a) {
    typedef Lane<T> L;
    typedef typename L::piece_t piece_t;
    constexpr int STEP = 4 * L::PER, RT = 4, AHEAD = 4;
    const Adapt& o = a.o;
    __shared__ f32x4_t sums[kWaves][RT][64];
    const int tile = blockIdx.x / a.slots, slot = blockIdx.x - tile * a.slots, split = blockIdx.y, first_rank = blockIdx.z * 16 * RT;
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = min((a.all - first_rank + 15) / 16, RT);
    Tile rows(o, tile);
    const int begin = split * a.steps, end = min(begin + a.steps, (o.d + STEP - 1) / STEP);
    const int row = min(tile * 16 + c, o.n - 1);
    const T* h = (const T*)o.H + row * o.ldh;
    for (int k = 0; rows.left; ++k) {
        const int w = rows.next();
        if (k % a.slots != slot) continue;
        const bool live = rows.live;
        const T* A = (const T*)o.A + w * o.a_stride;
        f32x4_t sum[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) sum[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int s0 = begin + wave; s0 < end; s0 += kWaves * AHEAD) {
            piece_t x[AHEAD], y[AHEAD][RT];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int col = (s0 + u * kWaves) * STEP + g * L::PER;
                const bool there = s0 + u * kWaves < end && col < o.d;
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
            if (r < a.all) *reinterpret_cast<f32x4_t*>(o.workspace + ((int64_t)split * o.n + row) * a.all + r) = all;
        }
        __syncthreads();
    }
}

// 4 PER / 4 = PER rank values of a lane, summed over the parts of d and scaled, as the operand's pieces
template <class T>
__device__ __forceinline__ void read_t(const AdaptArgs& a, const float* t, float scale, float (&v)[Lane<T>::PER]) {
    constexpr int PER = Lane<T>::PER;
#pragma unroll
    for (int e = 0; e < PER; ++e) v[e] = 0.f;
    for (int s = 0; s < a.splits; ++s) {
#pragma unroll
        for (int e = 0; e < PER; e += 4) {
            const f32x4_t x = *reinterpret_cast<const f32x4_t*>(t + (int64_t)s * a.o.n * a.all + e);
#pragma unroll
            for (int u = 0; u < 4; ++u) v[e + u] += x[u];
        }
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) v[e] *= scale;
}
// of bfloat16 the upper part, or what it leaves
__device__ __forceinline__ bf16x8_t piece_of(const float (&v)[8], bool rest) {
    bf16x8_t f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float up = __uint_as_float(__float_as_uint(v[e]) & 0xFFFF0000u);
        const float low = fabsf(v[e]) < __builtin_inff() ? v[e] - up : 0.f;
        f[e] = (__bf16)(rest ? low : fabsf(v[e]) <= __builtin_inff() ? up : v[e]);
    }
    return f;
}
__device__ __forceinline__ f32x4_t piece_of(const float (&v)[4], bool) { return f32x4_t{v[0], v[1], v[2], v[3]}; }

template <class T> struct Sixteen;                           // 16 columns of a row
template <> struct Sixteen<uint16_t> {
    u32x4_t w[2];
    __device__ __forceinline__ void load(const uint16_t* p, bool second) {
        w[0] = *reinterpret_cast<const u32x4_t*>(p);
        w[1] = second ? *reinterpret_cast<const u32x4_t*>(p + 8) : u32x4_t{0, 0, 0, 0};
    }
    __device__ __forceinline__ void store(uint16_t* p, bool second) const {
        *reinterpret_cast<u32x4_t*>(p) = w[0];
        if (second) *reinterpret_cast<u32x4_t*>(p + 8) = w[1];
    }
    __device__ __forceinline__ void add(const f32x4_t (&x)[4]) {
        typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t was = w[i >> 2][i & 3];
            const bf16x2_t pair = {(__bf16)(__uint_as_float(was << 16) + x[i >> 1][2 * (i & 1)]), (__bf16)(__uint_as_float(was & 0xFFFF0000u) + x[i >> 1][2 * (i & 1) + 1])};
            w[i >> 2][i & 3] = __builtin_bit_cast(uint32_t, pair);
        }
    }
};
template <> struct Sixteen<float> {
    f32x4_t w[4];
    __device__ __forceinline__ void load(const float* p, bool second) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = i < 2 || second ? *reinterpret_cast<const f32x4_t*>(p + 4 * i) : f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void store(float* p, bool second) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) if (i < 2 || second) *reinterpret_cast<f32x4_t*>(p + 4 * i) = w[i];
    }
    __device__ __forceinline__ void add(const f32x4_t (&x)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] += x[i];
    }
};

// A workgroup: a tile of 16 rows, 64 columns of one part; its waves share the tile's adapters out.  The second product is B T^T: instruction t takes the columns
// 16 (m / 4) + 4 t + m % 4 for its rows m, so that a lane ends with 16 columns of one row side by side.
template <class T>
__global__ __launch_bounds__(64 * kWaves)
void adapt_up_kernel(AdaptArgs a) {
    typedef Lane<T> L;
    typedef typename L::piece_t piece_t;
    constexpr int PER = L::PER, TWICE = sizeof(T) == 2 ? 2 : 1;          // pieces of a rank value: its two halves
    const Adapt& o = a.o;
    const int tile = blockIdx.y, lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int part = 0;
    while ((int)blockIdx.x >= a.first_group[part + 1]) ++part;
    const int first = (part > 0 ? o.part_end[part - 1] : 0) + 64 * (blockIdx.x - a.first_group[part]), end = o.part_end[part];
    Tile rows(o, tile);
    const int row = min(tile * 16 + c, o.n - 1), col = first + 16 * g;
    const bool in = col < end, second = col + 8 < end, in_place = o.base == o.Z;
    const T* base = (const T*)o.base + row * o.ldb + col;
    T* out = (T*)o.Z + row * o.ldz + col;
    if (wave == 0 && rows.id < 0 && tile * 16 + c < o.n && in && !in_place) {          // rows without an adapter
        Sixteen<T> x;
        x.load(base, second);
        x.store(out, second);
    }
    const int pieces = o.rank / PER, steps = (TWICE * pieces + 3) / 4;
    for (int k = 0; rows.left; ++k) {
        const int w = rows.next();
        if (k % kWaves != wave) continue;
        const bool live = rows.live;
        const T* B = (const T*)o.B + w * o.b_stride;
        const float scale = o.scale ? o.scale[w] : 1.f;
        Sixteen<T> x;
        if (live && in) x.load(base, second);
        f32x4_t sum[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) sum[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < steps; ++s) {
            const int q = 4 * s + g, at = (q >= pieces ? q - pieces : q) * PER;
            const bool there = q < TWICE * pieces;
            piece_t y[4], z = none<T>();
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int j = first + 16 * (c >> 2) + 4 * t + (c & 3);
                y[t] = none<T>();
                if (there && j < end) y[t] = *reinterpret_cast<const piece_t*>(B + j * o.ldbw + at);
            }
            if (there && live) {
                float v[PER];
                read_t<T>(a, o.workspace + (int64_t)row * a.all + part * o.rank + at, scale, v);
                z = piece_of(v, q >= pieces);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] = L::multiply(y[t], z, sum[t]);
        }
        if (live && in) {
            x.add(sum);
            x.store(out, second);
        }
    }
}

int steps_of(int is_bf16, int d) { return (d + (is_bf16 ? 31 : 15)) / (is_bf16 ? 32 : 16); }

// Workgroups for the first product: 512 fill the chip.  A tile of few rows has an adapter to each of them as a rule: they go side by side.
void plan(int is_bf16, int n, int d, int rank, int n_parts, int* slots, int* splits, int* steps) {
    const int tiles = (n + 15) / 16, all = steps_of(is_bf16, d), groups = (rank * n_parts + 63) / 64;
    *slots = tiles <= 16 ? 16 : 1;
    const int64_t items = (int64_t)(*slots == 1 ? tiles : n) * groups;
    int64_t cuts = items >= 512 ? 1 : 512 / items;
    const int most = (all + 15) / 16;                        // four steps to a wave
    if (cuts > most) cuts = most;
    if (cuts > 16) cuts = 16;
    *steps = (int)((all + cuts - 1) / cuts);
    *splits = (all + *steps - 1) / *steps;
}

template <class T>
hipError_t launch(const Adapt& o, hipStream_t stream) {
    AdaptArgs a;
    a.o = o;
    a.all = o.rank * o.n_parts;
    plan(sizeof(T) == 2, o.n, o.d, o.rank, o.n_parts, &a.slots, &a.splits, &a.steps);
    a.first_group[0] = 0;
    for (int k = 0; k < kMostParts; ++k)
        a.first_group[k + 1] = a.first_group[k] + (k < o.n_parts ? (o.part_end[k] - (k ? o.part_end[k - 1] : 0) + 63) / 64 : 0);
    const int tiles = (o.n + 15) / 16;
    hipLaunchKernelGGL(adapt_down_kernel<T>, dim3(tiles * a.slots, a.splits, (a.all + 63) / 64), dim3(64 * kWaves), 0, stream, a);
    hipLaunchKernelGGL(adapt_up_kernel<T>, dim3(a.first_group[o.n_parts], tiles), dim3(64 * kWaves), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

bool adapt_fits(const Adapt& o) {
    const int64_t tiles = (o.n + 15) / 16, groups = o.p / 64 + o.n_parts;
    return tiles <= 65535 && tiles * groups <= kMostThreads / 256;
}

size_t adapt_workspace_bytes(int is_bf16, int n, int d, int rank, int n_parts) {
    int slots, splits, steps;
    plan(is_bf16, n, d, rank, n_parts, &slots, &splits, &steps);
    return (size_t)splits * n * rank * n_parts * sizeof(float);
}

hipError_t adapt(const Adapt& o, int is_bf16, hipStream_t stream) { return is_bf16 ? launch<uint16_t>(o, stream) : launch<float>(o, stream); }

}  // namespace gelo
