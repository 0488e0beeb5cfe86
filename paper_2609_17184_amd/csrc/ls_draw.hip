// One token per row of logits from a given uniform number: temperature, top-k,
// top-p and min-p, each row with its own settings.
//
//   w_v = 2^((z_v - max z) log2(e) / T);  ids ranked by (z descending, id ascending), -infinity left out:
//   top-k keeps the first k ranks; top-p, of those, the ranks whose preceding mass is below top_p of the top-k
//   mass; min-p, of those, w_v >= min_p.  The token is the smallest id whose kept mass through it exceeds
//   u * kept mass.  T = 0: the largest logit, lowest id.
//
// One CU reads a row of 49152 fp32 logits in about 19 us, most of it waiting,
// so a row is spread over shards of 4096 ids.  Three launches:
//
//   k_draw_shard  a workgroup per (row, shard): the shard's largest logit, its mass, and, for a row with a
//                 filter, counts and masses over 128 bins of half an octave of weight
//   k_draw_list   (rows with filters) the bins of all shards put together tell the few bins in which the last
//                 kept rank and the min-p threshold lie; each shard adds its logits in them to the row's list
//                 and sums its mass above them
//   k_draw_pick   a workgroup per row: the last kept rank on the list, the shard that holds the token, the token
//
// A token is decided by comparing sums with u times a sum, so weights are taken
// in 64 bits (2^f by a polynomial on [-1/2, 1/2], off by 2^-38.8: each two degrees
// more are a tenth of a large batch's time) and sums have to be the same whatever
// the order of adding: what atomics add are integers, in units of 2^-38 of a power
// of two at a bin's upper end, or 2^-44 of the row's largest weight, and sums of
// doubles run in an order that depends on the vocabulary alone.  Weights are taken
// from differences to the shard's or the row's largest logit, which itself weighs
// exactly 1, so equal logits weigh the same and a u or top-p on the border between
// them falls on the right side of it.  Bins lie on a grid of z log2(e) / T that all
// shards share.
//
// The last kept rank: up to 1024 listed logits are sorted, one a thread (48 rows
// of mixed settings with no longer list: 32 us, through the histogram below 35).  More
// go through a histogram of 2048 bins of 1/32 octave; if the bin that it leaves
// holds no more than 1024, a thread each finds its logit's rank against all
// others, else ranges of the logits' order-preserving integer keys are searched
// the same way down to a single key, whose ties are counted off by id.  A row
// whose list overflows is searched in place.  48 rows of 65536 normal logits of
// deviation 2.5 at T = 1.25 and top-p 0.95, some 4100 listed, take 70 us, of 131072 239,
// at T = 2 and top-p 0.9, which overflows, 316.
//
// Measured (us): 256 rows of 131072 logits 42 in fp32 and 41 in bf16, bound by the
// weights' 64-bit arithmetic (about 8 cycles an operation and wave); at T = 0 27,
// 4.9 TB/s, memory's rate; rows off the loads' alignment (130003) 48 and 49.  256
// rows of 65536 with top-k 50 and top-p 0.9 66, with top-p 0.95 92: the bins' LDS
// atomics, the second read of the shards that hold listed logits, and long lists.
// One row of 49152 with top-p 24.7: 6, 8 and 12 in the three launches, each a chain
// of loads that wait for each other and barriers.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/loopspec.h"

namespace ls {

typedef unsigned long long u64;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kShard = 4096, kShardThreads = 256, kShardEach = kShard / kShardThreads;
constexpr int kCoarse = 128;                          // bins of half an octave, the last one for all below
constexpr int kListMax = 8192;                        // listed logits of a row
constexpr int kDThreads = 1024, kDWaves = kDThreads / 64;
constexpr int kDBins = 2048;                          // two per thread
constexpr int kMembers = kDThreads;
constexpr int kDMaxVocab = 1 << 18, kShardsMax = kDMaxVocab / kShard;
static_assert(kShardsMax == 64, "a shard per lane");

struct Head {                                         // of a shard
    double grid;                                      // the largest logit's place on the grid
    double mass;                                      // in 2^-44 of the largest logit's weight
    float top;
    int arg, bad;                                     // lowest id of the largest logit; NaN or +infinity met
    unsigned finite;
};
struct Entry {
    float v;
    int id;
};
struct RowPlan {                                      // what the listing found, for the pick
    int rank;                                         // the last kept rank lies in the list
    unsigned above_c;                                 // ranks above the listed bins
    double above_m, all;                              // mass above them and in the whole row, in 2^-44 of the largest weight
};

struct DrawArgs {
    const void* z;
    int64_t stride;
    const double* u;
    const float *temperature, *top_p, *min_p;         // per row, or null: the values below
    const int32_t* top_k;
    float temperature1, top_p1, min_p1;
    int32_t top_k1;
    int32_t* token;
    float* prob;
    int32_t* kept;
    int V, S;
    // workspace
    Head* head;                                       // [rows][S]
    u64* bins;                                        // [rows][S][kCoarse]
    double* above;                                    // [rows][S]: the shard's mass above the listed bins, in the head's unit
    RowPlan* plan;                                    // [rows]
    Entry* list;                                      // [rows][kListMax]
    unsigned* listed;                                 // [rows]
};

// a row's settings
struct Setting {
    float T, top_p, min_p;
    int top_k;
    double scale;                                     // log2(e) / T
    bool ok, by_k, by_p, by_m;
    __device__ __forceinline__ Setting(const DrawArgs& a, int row) {
        T = a.temperature ? a.temperature[row] : a.temperature1;
        top_p = a.top_p ? a.top_p[row] : a.top_p1;
        min_p = a.min_p ? a.min_p[row] : a.min_p1;
        top_k = a.top_k ? a.top_k[row] : a.top_k1;
        const double u = a.u[row];
        ok = T >= 0.f && T < INFINITY && top_p > 0.f && top_p <= 1.f && min_p >= 0.f && min_p <= 1.f && u >= 0.0 && u < 1.0;
        const bool draws = ok && T > 0.f;
        scale = draws ? 1.4426950408889634074 / (double)T : 0.0;
        by_k = draws && top_k > 0 && top_k < a.V;
        by_p = draws && top_p < 1.f;
        by_m = draws && min_p > 0.f;
    }
    __device__ __forceinline__ bool filters() const { return by_k || by_p || by_m; }
    // the logit in octaves, rounded: not contracted with what is added to it, so that a threshold lies on the grid
    // where the largest logit does
    __device__ __forceinline__ double octaves(float v) const {
        double t = (double)v * scale;
        asm("" : "+v"(t));
        return t;
    }
    // its place on the grid of half octaves
    __device__ __forceinline__ double grid(float v) const { return floor(2.0 * octaves(v)); }
    // Octaves between a logit and a larger one.  The difference is taken first: it is exact wherever weights matter,
    // while octaves of logits far from zero are rounded, and equal logits weigh exactly 1.
    __device__ __forceinline__ double below(float top, float v) const { return ((double)v - (double)top) * scale; }
};
// the bin of a place: 0 also for one above the largest logit's, where a threshold's slack may reach
__device__ __forceinline__ int coarse(double grid_top, double grid) {
    const double d = grid_top - grid;
    return d < (double)(kCoarse - 1) ? max((int)d, 0) : kCoarse - 1;
}

__device__ __forceinline__ float half_bits(int dt, uint32_t b) {
    return dt == LOOPSPEC_BF16 ? __uint_as_float(b << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)b);
}
template <int DT>
__device__ __forceinline__ float logit(const void* p, int64_t i) {
    if (DT == LOOPSPEC_F32) return ((const float*)p)[i];
    return half_bits(DT, ((const uint16_t*)p)[i]);
}
// four logits from i, one load of its alignment
template <int DT>
__device__ __forceinline__ void load4(const void* p, int64_t i, float* v) {
    if (DT == LOOPSPEC_F32) {
        const u32x4 u = *(const u32x4*)((const float*)p + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(u[k]);
    } else {
        const u32x2 u = *(const u32x2*)((const uint16_t*)p + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = half_bits(DT, k & 1 ? u[k >> 1] >> 16 : u[k >> 1] & 0xFFFFu);
    }
}
// logits id0 + 1024 k + 4 t + (0 .. 3) of thread t and k = 0 .. 3, -infinity from V on.  Four of them are one
// aligned load; rows that lie off that alignment (odd vocabularies) pass through LDS, since a shard of
// unaligned loads took 1.6 times as long.
template <int DT>
__device__ __forceinline__ void load_shard(const DrawArgs& a, int64_t base, int id0, float (&v)[kShardEach], float (&l)[kShard + 4]) {
    const int tid = threadIdx.x, id = id0 + 4 * tid;
    const int off = (int)(((uintptr_t)a.z / (DT == LOOPSPEC_F32 ? 4 : 2) + (uint64_t)base + id0) % 4);
    if (id0 + kShard > a.V) {
#pragma unroll
        for (int k = 0; k < kShardEach; ++k) {
            const int i = id + 1024 * (k / 4) + k % 4;
            v[k] = i < a.V ? logit<DT>(a.z, base + i) : -INFINITY;
        }
    } else if (off == 0) {
#pragma unroll
        for (int k = 0; k < kShardEach / 4; ++k) load4<DT>(a.z, base + id + 1024 * k, v + 4 * k);
    } else {
        // place i of l holds id0 - off + i; the vectors that reach over the shard's ends are taken singly
        float e = 0.f;
        const int i = tid < 4 - off ? tid : kShard - 2 * 4 + tid;   // 4 - off ids at the front, off at the back
        if (tid < 4) e = logit<DT>(a.z, base + id0 + i + (tid < 4 - off ? 0 : 4));
#pragma unroll
        for (int k = 0; k < kShardEach / 4; ++k)
            if (k || tid) load4<DT>(a.z, base + id - off + 1024 * k, v + 4 * k);
        if (tid < 4) l[off + i + (tid < 4 - off ? 0 : 4)] = e;
#pragma unroll
        for (int k = 0; k < kShardEach / 4; ++k)
            if (k || tid)
#pragma unroll
                for (int m = 0; m < 4; ++m) l[4 * tid + 1024 * k + m] = v[4 * k + m];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kShardEach; ++k) v[k] = l[off + 4 * tid + 1024 * (k / 4) + k % 4];
    }
}
// order-preserving integer of a float that is no NaN; both zeros alike
__device__ __forceinline__ uint32_t order_key(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
// 2^(y + up), y small or negative (2^(up - 200) below y = -200): y = n + f, the polynomial
// interpolates 2^f at the Chebyshev points of [-1/2, 1/2] and is 1 at 0.  n comes
// from adding 1.5 * 2^52, whose low word it then is, and goes to the exponent as
// it is: conversions and ldexp take several times an addition's cycles.
__device__ __forceinline__ double weight(double y, int up = 0) {
    constexpr double M = 6755399441055744.0;
    y = fmax(y, -200.0);
    const double t = y + M, f = y - (t - M);
    double p = 1.325080551750225e-06;
    p = fma(p, f, 1.5303700711365693e-05);
    p = fma(p, f, 0.00015403475186530786);
    p = fma(p, f, 0.0013333478473685416);
    p = fma(p, f, 0.00961812913523614);
    p = fma(p, f, 0.055504109063258665);
    p = fma(p, f, 0.24022650695888503);
    p = fma(p, f, 0.6931471805568324);
    p = fma(p, f, 1.0);
    return __hiloint2double(__double2hiint(p) + ((__double2loint(t) + up) << 20), __double2loint(p));
}
// the weight in units of 2^-44, to nearest: adding 2^52 leaves it in the low bits
__device__ __forceinline__ u64 mass44(double y) {
    return (u64)__double_as_longlong(weight(y, 44) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
}

// A bin: how many logits (from bit 51) and their mass in units of 2^-38 of the
// power of two 2^-bin_octaves(b), which no weight of bin b exceeds beside the
// largest one anywhere in bin 0: each is off by 2^-37 of itself at most, however
// far down, and 4096 of them stay below bit 51.
constexpr u64 kOne = 1ull << 51;
__device__ __forceinline__ int bin_octaves(int b) { return (max(b, 1) - 1) >> 1; }
__device__ __forceinline__ u64 binned(double y, int b) {
    return kOne + ((u64)__double_as_longlong(weight(y, 38 + bin_octaves(b)) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull);
}
// its mass in 2^-44
__device__ __forceinline__ double bin_mass(u64 x, int b) { return (double)(x & (kOne - 1)) * __hiloint2double((1029 - bin_octaves(b)) << 20, 0); }

// Exchanges within a full wave by VALU moves (DPP, and swaps of rows and halves):
// a permutation through LDS takes some 50 ns, and a sort of 1024 has 90 of them
// (with those, a row with filters took 3.7 us longer).
template <typename T, typename F>
__device__ __forceinline__ T by_words(T v, F move) {
    static_assert(sizeof(T) == 4 || sizeof(T) == 8, "one or two words");
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, (uint32_t)move(__builtin_bit_cast(uint32_t, v)));
    } else {
        const u64 b = __builtin_bit_cast(u64, v);
        return __builtin_bit_cast(T, (u64)move((uint32_t)(b >> 32)) << 32 | move((uint32_t)b));
    }
}
// what CTRL brings, zero where it brings nothing or the row is not in ROWS
template <int CTRL, int ROWS = 15>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 15, false);
}
// the value of lane ^ J
template <int J, typename T>
__device__ __forceinline__ T from_xor(T v) {
    return by_words(v, [](uint32_t x) -> uint32_t {
        if constexpr (J == 1) return dpp<0xB1>(x);                  // quad_perm [1,0,3,2]
        if constexpr (J == 2) return dpp<0x4E>(x);                  // quad_perm [2,3,0,1]
        if constexpr (J == 4) return dpp<0x1B>(dpp<0x141>(x));      // row_half_mirror, quad_perm [3,2,1,0]
        if constexpr (J == 8) return dpp<0x128>(x);                 // row_ror:8
        if constexpr (J == 16) {
            const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
            return threadIdx.x & 16 ? p[0] : p[1];
        }
        if constexpr (J == 32) {
            const auto p = __builtin_amdgcn_permlane32_swap(x, x, false, false);
            return threadIdx.x & 32 ? p[0] : p[1];
        }
    });
}
template <typename T, typename F>
__device__ __forceinline__ T wave_all(T v, F f) {
    v = f(v, from_xor<1>(v)), v = f(v, from_xor<2>(v)), v = f(v, from_xor<4>(v));
    v = f(v, from_xor<8>(v)), v = f(v, from_xor<16>(v));
    return f(v, from_xor<32>(v));
}
template <typename T>
__device__ __forceinline__ T wave_sum(T v) { return wave_all(v, [](T a, T b) { return a + b; }); }
__device__ __forceinline__ float wave_max(float v) { return wave_all(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ double wave_max(double v) { return wave_all(v, [](double a, double b) { return fmax(a, b); }); }
// sum of the lanes up to the lane's own
template <typename T>
__device__ __forceinline__ T wave_upto(T v) {
    v += by_words(v, dpp<0x111>), v += by_words(v, dpp<0x112>);     // row_shr:1, 2, 4, 8
    v += by_words(v, dpp<0x114>), v += by_words(v, dpp<0x118>);
    v += by_words(v, dpp<0x142, 0xA>);                              // row_bcast:15, then row_bcast:31
    return v + by_words(v, dpp<0x143, 0xC>);
}
// the value of one lane, the same for the wave
template <typename T>
__device__ __forceinline__ T from_lane(T v, int l) {
    l = __builtin_amdgcn_readfirstlane(l);
    return by_words(v, [l](uint32_t x) -> uint32_t { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); });
}

template <int DT>
__global__ void __launch_bounds__(kShardThreads) k_draw_shard(DrawArgs a) {
    __shared__ float shifted[kShard + 4];
    __shared__ u64 bins[kCoarse];
    __shared__ float wf[4];
    __shared__ double wm[4];
    __shared__ unsigned wc[4];
    __shared__ int bad, arg;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, s = blockIdx.x, row = blockIdx.y, id0 = s * kShard;
    float v[kShardEach];
    load_shard<DT>(a, row * a.stride, id0, v, shifted);
    const Setting set(a, row);
    if (tid < kCoarse) bins[tid] = 0;
    if (tid == 0) bad = 0, arg = 0x7FFFFFFF;
    float top = -INFINITY;
    bool wrong = false;
    unsigned n = 0;
#pragma unroll
    for (int k = 0; k < kShardEach; ++k) {
        wrong |= !(v[k] < INFINITY);
        top = fmaxf(top, v[k]);
        n += v[k] > -INFINITY;
    }
    top = wave_max(top);
    n = wave_sum(n);
    if (lane == 0) wf[wv] = top, wc[wv] = n;
    __syncthreads();
    if (wrong) bad = 1;
    top = fmaxf(fmaxf(wf[0], wf[1]), fmaxf(wf[2], wf[3]));
    const double grid = set.grid(top);
    if (set.T > 0.f && top > -INFINITY) {
        double sum = 0.0;
        if (set.filters()) {
#pragma unroll
            for (int k0 = 0; k0 < kShardEach; k0 += 4) {
                u64 m[4];
                int b[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    b[k] = coarse(grid, set.grid(v[k0 + k]));
                    m[k] = binned(set.below(top, v[k0 + k]), b[k]);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (v[k0 + k] > -INFINITY) atomicAdd(&bins[b[k]], m[k]);
            }
            __syncthreads();
            if (tid < kCoarse) sum = bin_mass(bins[tid], tid);
        } else {
            // (-infinity weighs 2^-200)
            double part[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
            for (int k = 0; k < kShardEach; ++k) part[k & 3] += weight(set.below(top, v[k]), 44);
            sum = (part[0] + part[1]) + (part[2] + part[3]);
        }
        sum = wave_sum(sum);
        if (lane == 0) wm[wv] = sum;
    } else {
        if (lane == 0) wm[wv] = 0.0;
        if (set.T == 0.f) {
            int best = 0x7FFFFFFF;
#pragma unroll
            for (int k = kShardEach - 1; k >= 0; --k)
                if (v[k] == top) best = id0 + 4 * tid + 1024 * (k / 4) + k % 4;
            if (best < 0x7FFFFFFF) atomicMin(&arg, best);
        }
    }
    __syncthreads();
    const size_t at = (size_t)row * a.S + s;
    if (set.filters() && tid < kCoarse) a.bins[at * kCoarse + tid] = bins[tid];
    if (tid == 0) {
        a.head[at] = Head{grid, (wm[0] + wm[1]) + (wm[2] + wm[3]), top, arg, bad, wc[0] + wc[1] + wc[2] + wc[3]};
        if (s == 0) a.listed[row] = 0;
    }
}

// what a row's shards have in common; every wave works it out from the heads
struct Whole {
    float top;
    double grid;                                      // of the row's largest logit
    bool bad;
    Head mine;                                        // lane s: shard s's (nothing in it behind the last one)
    __device__ __forceinline__ Whole(const DrawArgs& a, int row) {
        const int lane = threadIdx.x & 63;
        mine = Head{-INFINITY, 0.0, -INFINITY, 0x7FFFFFFF, 0, 0};
        if (lane < a.S) mine = a.head[(size_t)row * a.S + lane];
        if (!(mine.top > -INFINITY)) mine.grid = -INFINITY;
        top = wave_max(mine.top);
        grid = wave_max(mine.grid);
        bad = __any(mine.bad);
    }
};

template <int DT>
__global__ void __launch_bounds__(kShardThreads) k_draw_list(DrawArgs a) {
    __shared__ double he[kShardsMax], part_m[2][kCoarse];   // a shard's largest weight over the row's; halves of the row's bins
    __shared__ float shifted[kShard + 4];
    __shared__ int ho[kShardsMax];
    __shared__ unsigned part_c[2][kCoarse];
    __shared__ int range[2];
    __shared__ double wm[4];
    __shared__ unsigned n, base;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, s = blockIdx.x, row = blockIdx.y;
    const Setting set(a, row);
    if (!set.filters()) return;
    const Whole r(a, row);
    if (r.bad || !(r.top > -INFINITY)) return;
    const size_t row0 = (size_t)row * a.S;
    if (tid < a.S) {
        // (a shard without a finite logit has empty bins, wherever they go)
        he[tid] = weight(set.below(r.top, r.mine.top));
        ho[tid] = r.mine.grid > -INFINITY ? coarse(r.grid, r.mine.grid) : 0;
    }
    if (tid == 0) n = 0;
    __syncthreads();
    // the row's bins: a thread per bin and half of the shards, 8 of them under way; what the last bin holds
    // follows from the whole
    {
        const int b = tid & (kCoarse - 1), h = tid / kCoarse, half = (a.S + 1) / 2, end = min(a.S, (h + 1) * half);
        double m = 0.0;
        unsigned c = 0;
        for (int k0 = h * half; k0 < end; k0 += 8) {
            u64 x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int k = min(k0 + i, end - 1);
                x[i] = a.bins[(row0 + k) * kCoarse + max(b - ho[k], 0)];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k0 + i < end && b >= ho[k0 + i]) m += bin_mass(x[i], b - ho[k0 + i]) * he[k0 + i], c += (unsigned)(x[i] / kOne);
        }
        part_m[h][b] = b < kCoarse - 1 ? m : 0.0, part_c[h][b] = b < kCoarse - 1 ? c : 0u;
    }
    __syncthreads();
    if (wv == 0) {
        const double m0 = part_m[0][2 * lane] + part_m[1][2 * lane];
        double m1 = part_m[0][2 * lane + 1] + part_m[1][2 * lane + 1];
        const unsigned c0 = part_c[0][2 * lane] + part_c[1][2 * lane];
        unsigned c1 = part_c[0][2 * lane + 1] + part_c[1][2 * lane + 1];
        const double all = wave_sum(lane < a.S ? r.mine.mass * he[lane] : 0.0), most = wave_sum(m0 + m1);
        const unsigned finite = wave_sum(r.mine.finite), counted = wave_sum(c0 + c1);
        if (lane == 63) m1 = fmax(all - most, 0.0), c1 = finite - counted;
        const double sm = wave_upto(m0 + m1);
        const unsigned sc = wave_upto(c0 + c1);
        const unsigned long long used = __ballot(c0 + c1 > 0);
        const int last_lane = 63 - __clzll(used), last = 2 * last_lane + (from_lane(c1, last_lane) > 0);
        // first bin that meets a condition on (mass through, count through), the last occupied one when none does
        auto first = [&](auto meets) {
            const bool low = meets(sm - m1, sc - c1), high = meets(sm, sc);
            const unsigned long long hit = __ballot(high);
            if (!hit) return last;
            const int l = __ffsll(hit) - 1;
            return min(2 * l + (from_lane((int)low, l) ? 0 : 1), last);
        };
        int lo = kCoarse, hi = -1;
        double share = all;                           // bounds of the mass that top-k keeps, as far as known
        if (set.by_k) {
            hi = lo = first([&](double, unsigned c) { return c >= (unsigned)set.top_k; });
            const double above = from_lane(sm - m0 - m1, hi / 2) + (hi & 1 ? from_lane(m0, hi / 2) : 0.0);
            share = above;
        }
        if (set.by_p) {
            // (a hair of slack: these sums of doubles and the exact ones need not round alike)
            const double p = (double)set.top_p;
            const int b = first([&](double m, unsigned) { return m >= p * share * (1.0 - 1e-9); });
            const int b2 = first([&](double m, unsigned) { return m >= p * share * (1.0 + 1e-9); });
            lo = min(lo, b);
            hi = max(hi, b2);
        }
        bool rank = set.by_k || set.by_p;
        if (set.by_m) {
            // both bins that the threshold may lie in
            const double t = set.octaves(r.top) + log2((double)set.min_p);
            const int b = min(coarse(r.grid, floor(2.0 * t + 1e-6)), last), b2 = min(coarse(r.grid, floor(2.0 * t - 1e-6)), last);
            if (!rank || b2 < lo) {
                rank = false;
                lo = b, hi = b2;
            } else if (b < lo) {
                lo = b;
            }
        }
        const double am = from_lane(sm - m0 - m1, lo / 2) + (lo & 1 ? from_lane(m0, lo / 2) : 0.0);
        const unsigned ac = from_lane(sc - c0 - c1, lo / 2) + (lo & 1 ? from_lane(c0, lo / 2) : 0u);
        if (lane == 0) {
            range[0] = lo, range[1] = hi;
            if (s == 0) a.plan[row] = RowPlan{rank, ac, am, all};
        }
    }
    __syncthreads();
    const int lo = range[0], hi = range[1];
    // this shard: its mass above the listed bins, its members in them
    double above = 0.0;
    bool some = false;
    if (tid < kCoarse) {
        const int b = min(ho[s] + tid, kCoarse - 1);
        const u64 x = a.bins[(row0 + s) * kCoarse + tid];
        if (b < lo) above = bin_mass(x, tid);
        some = b >= lo && b <= hi && x >= kOne;
    }
    above = wave_sum(above);
    if (lane == 0) wm[wv] = above;
    const bool any = __syncthreads_or(some);
    if (tid == 0) a.above[row0 + s] = wm[0] + wm[1];
    if (!any) return;
    float v[kShardEach];
    load_shard<DT>(a, row * a.stride, s * kShard, v, shifted);
    unsigned at[kShardEach];
#pragma unroll
    for (int k = 0; k < kShardEach; ++k) {
        at[k] = ~0u;
        if (!(v[k] > -INFINITY)) continue;
        const int b = coarse(r.grid, set.grid(v[k]));
        if (b >= lo && b <= hi) at[k] = atomicAdd(&n, 1u);
    }
    __syncthreads();
    if (tid == 0) base = atomicAdd(&a.listed[row], n);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kShardEach; ++k)
        if (at[k] != ~0u && base + at[k] < (unsigned)kListMax)
            a.list[(size_t)row * kListMax + base + at[k]] = Entry{v[k], s * kShard + 4 * tid + 1024 * (k / 4) + k % 4};
}

// the last kept rank: logits above f are kept, and those equal to it up to id
struct Cut {
    float f = -INFINITY;
    int id = -1;
    __device__ __forceinline__ bool keeps(float v, int i) const { return v > f || (v == f && i <= id); }
};

struct Member {
    float v;
    int id;
    u64 mass;
};

struct DrawLds {
    u64 mass[kDBins];
    unsigned count[kDBins];
    Member list[kMembers];
    u64 shard[kShardsMax];                            // kept mass of the searched logits, per shard
    double ws[kShardsMax];                            // kept mass per shard
    u64 wm[kDWaves];
    double wd[kDWaves];
    unsigned wc[kDWaves];
    unsigned first, last, listed, lo, hi, cnt, above_cnt, kept;
    u64 above_mass;
    float cut_f;
    int cut_id;
};

// Logits among which a rank is searched: the row's list, or the whole row.
template <int DT>
struct Search {
    const DrawArgs& a;
    int64_t base;
    const Entry* list;                                // null: the whole row
    int n;
    float top;
    double scale;
    DrawLds& l;
    // f(id, logit)
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        if (list) {
            for (int i = threadIdx.x; i < n; i += kDThreads) {
                const Entry e = list[i];
                f(e.id, e.v);
            }
        } else {
            for (int i = threadIdx.x; i < a.V; i += kDThreads) f(i, logit<DT>(a.z, base + i));
        }
    }
    __device__ __forceinline__ double y(float v) const { return ((double)v - (double)top) * scale; }
    __device__ __forceinline__ int bin(float v) const {
        const float d = (top - v) * (float)(32.0 * scale);
        return d < (float)(kDBins - 1) ? (int)d : kDBins - 1;       // infinity and NaN (0 * inf): the last bin
    }
};

template <bool MASS, bool COUNT>
__device__ __forceinline__ void clear_bins(DrawLds& l) {
    __syncthreads();
    for (int i = threadIdx.x; i < kDBins; i += kDThreads) {
        if (MASS) l.mass[i] = 0;
        if (COUNT) l.count[i] = 0;
    }
    if (threadIdx.x == 0) l.first = kDBins, l.last = 0, l.listed = 0;
    __syncthreads();
}

// l.first and l.last become the smallest `low` and the largest `high` of the
// workgroup that are not -1; both rise with the thread, so a wave has one say
__device__ __forceinline__ void note_first_last(DrawLds& l, int low, int high) {
    const int lane = threadIdx.x & 63;
    const u64 a = __ballot(low >= 0), b = __ballot(high >= 0);
    if (a && lane == __ffsll(a) - 1) atomicMin(&l.first, (unsigned)low);
    if (b && lane == 63 - __clzll(b)) atomicMax(&l.last, (unsigned)high);
}

// The bin that holds the last kept rank: the first one through which the count
// reaches `need` (COUNT), or the mass reaches `goal`; the last occupied one when
// none does.  share > 0: the goal is that share of the bins' whole mass and what
// is above them.  What lies above the bin (above_m and above_c included) is left
// in l, and the bin's count.
template <bool MASS, bool COUNT>
__device__ unsigned pick_bin(DrawLds& l, unsigned need, double share, double* goal, u64 above_m, unsigned above_c) {
    __syncthreads();
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, b0 = 2 * tid;
    u64 m[2] = {0, 0};
    unsigned c[2] = {0, 0};
    if (MASS) m[0] = l.mass[b0], m[1] = l.mass[b0 + 1];
    if (COUNT) c[0] = l.count[b0], c[1] = l.count[b0 + 1];
    u64 sm = MASS ? wave_upto(m[0] + m[1]) : 0;
    unsigned sc = COUNT ? wave_upto(c[0] + c[1]) : 0u;
    if (lane == 63) l.wm[wv] = sm, l.wc[wv] = sc;
    __syncthreads();
    sm += above_m - m[0] - m[1];
    sc += above_c - c[0] - c[1];
    u64 all = 0;
    for (int i = 0; i < kDWaves; ++i) {
        if (i < wv) sm += l.wm[i], sc += l.wc[i];
        all += l.wm[i];
    }
    if (share > 0.0) *goal = share * (double)(above_m + all);
    const u64 am[2] = {sm, sm + m[0]};                // above each of the thread's bins
    const unsigned ac[2] = {sc, sc + c[0]};
    int low = -1, high = -1;                          // the thread's first bin that reaches it, its last occupied one
#pragma unroll
    for (int i = 1; i >= 0; --i) {
        if (COUNT ? !c[i] : !m[i]) continue;
        if (goal ? (double)(am[i] + m[i]) >= *goal : ac[i] + c[i] >= need) low = b0 + i;
        high = max(high, b0 + i);
    }
    note_first_last(l, low, high);
    __syncthreads();
    const unsigned at = l.first < (unsigned)kDBins ? l.first : l.last;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (at == (unsigned)(b0 + i)) l.cnt = c[i], l.above_mass = am[i], l.above_cnt = ac[i];
    __syncthreads();
    return at;
}

// Id of the tie with `ties` ids up to its own among the logits equal to f: by
// halving the ids.
template <int DT>
__device__ int tie_id(const Search<DT>& r, Cut from, float f, unsigned ties) {
    DrawLds& l = r.l;
    int lo = 0, hi = r.a.V - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        unsigned c = 0;
        r.each([&](int id, float v) { c += v == f && id <= mid && from.keeps(v, id); });
        c = wave_sum(c);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) l.wc[threadIdx.x >> 6] = c;
        __syncthreads();
        c = 0;
        for (int i = 0; i < kDWaves; ++i) c += l.wc[i];
        if (c >= ties)
            hi = mid;
        else
            lo = mid + 1;
    }
    __syncthreads();
    return lo;
}

// The last kept rank of what `from` keeps: the first `need` ranks (BY_COUNT), or
// the ranks whose preceding mass is below the goal: `share` of the whole mass
// (above and searched) or, share 0, the given one.  above_c ranks of mass above_m
// lie above all that is searched.
template <bool BY_COUNT, int DT>
__device__ Cut last_kept(const Search<DT>& r, Cut from, unsigned need, double share, double goal, u64 above_m, unsigned above_c) {
    DrawLds& l = r.l;
    const int tid = threadIdx.x;
    double* const goalp = BY_COUNT ? nullptr : &goal;
    clear_bins<!BY_COUNT, BY_COUNT>(l);
    r.each([&](int id, float v) {
        if (!from.keeps(v, id)) return;
        if (BY_COUNT)
            atomicAdd(&l.count[r.bin(v)], 1u);
        else
            atomicAdd(&l.mass[r.bin(v)], mass44(r.y(v)));
    });
    const int picked = (int)pick_bin<!BY_COUNT, BY_COUNT>(l, need, share, goalp, above_m, above_c);
    above_m = l.above_mass, above_c = l.above_cnt;
    __syncthreads();
    if (tid == 0) l.listed = 0, l.cnt = 0;
    __syncthreads();
    r.each([&](int id, float v) {
        if (r.bin(v) != picked || !from.keeps(v, id)) return;
        const unsigned at = atomicAdd(&l.listed, 1u);
        if (at < (unsigned)kMembers) l.list[at] = Member{v, id, BY_COUNT ? 0 : mass44(r.y(v))};
    });
    __syncthreads();
    const unsigned members = l.listed;
    if (members <= (unsigned)kMembers) {
        const Member me = l.list[tid < (int)members ? tid : 0];
        unsigned rank = 0;
        u64 before = 0;
        if ((tid & ~63) < (int)members)
            for (unsigned j = 0; j < members; ++j) {
                const Member o = l.list[j];
                const bool ahead = o.v > me.v || (o.v == me.v && o.id < me.id);
                rank += ahead;
                if (!BY_COUNT) before += ahead ? o.mass : 0;
            }
        const bool kept = tid < (int)members && (BY_COUNT ? above_c + rank < need : (double)(above_m + before) < goal);
        const u64 vote = __ballot(kept);
        if ((tid & 63) == 0 && vote) atomicAdd(&l.cnt, (unsigned)__popcll(vote));
        __syncthreads();
        // (none kept: sums of doubles put the goal just above the members; their first one it is)
        if (tid < (int)members && rank == (l.cnt ? l.cnt - 1 : 0u)) l.cut_f = me.v, l.cut_id = me.id;
        __syncthreads();
        Cut c;
        c.f = l.cut_f, c.id = l.cut_id;
        __syncthreads();
        return c;
    }
    uint32_t lo = 0, hi = 0xFFFFFFFFu;                // keys of the range that holds the last rank
    for (;;) {
        // the ends of what is left, then its histogram
        if (tid == 0) l.lo = 0xFFFFFFFFu, l.hi = 0;
        clear_bins<true, true>(l);
        uint32_t a = 0xFFFFFFFFu, b = 0;
        r.each([&](int id, float v) {
            const uint32_t k = order_key(v);
            if (r.bin(v) == picked && k >= lo && k <= hi && from.keeps(v, id)) a = min(a, k), b = max(b, k);
        });
        if (a <= b) {
            atomicMin(&l.lo, a);
            atomicMax(&l.hi, b);
        }
        __syncthreads();
        lo = l.lo, hi = l.hi;
        int shift = 0;
        while (((hi - lo) >> shift) >= (uint32_t)kDBins) ++shift;
        r.each([&](int id, float v) {
            const uint32_t k = order_key(v);
            if (r.bin(v) != picked || k < lo || k > hi || !from.keeps(v, id)) return;
            const int bin = (int)((hi - k) >> shift);
            atomicAdd(&l.count[bin], 1u);
            if (!BY_COUNT) atomicAdd(&l.mass[bin], mass44(r.y(v)));
        });
        const uint32_t h = hi - (pick_bin<true, true>(l, need, 0.0, goalp, above_m, above_c) << shift);
        above_m = l.above_mass, above_c = l.above_cnt;
        const unsigned n = l.cnt;
        __syncthreads();
        if (shift == 0) {
            // n equal logits, of which the first e are kept
            Cut c;
            c.f = __uint_as_float(h & 0x80000000u ? h & 0x7FFFFFFFu : ~h);
            unsigned e = n;
            if (BY_COUNT) {
                e = min(n, need - above_c);
            } else if (const u64 one = mass44(r.y(c.f))) {
                const double want = (goal - (double)above_m) / (double)one;
                e = want < (double)n ? (unsigned)max(want, 1.0) : n;
                while (e > 1 && (double)(above_m + (u64)(e - 1) * one) >= goal) --e;
                while (e < n && (double)(above_m + (u64)e * one) < goal) ++e;
            }
            c.id = e < n ? tie_id(r, from, c.f, e) : 0x7FFFFFFF;
            if (e == n && c.f == from.f) c.id = from.id;
            return c;
        }
        lo = max(lo, h - ((1u << shift) - 1));
        hi = h;
    }
}

// Up to 1024 listed logits, one a thread, put in the order of their ranks (a
// bitonic sort of key and id; strides below a wave's width by shuffles) and
// their masses summed in it: both filters then are places in that order.
// Returns the last kept rank; e and m are the thread's logit and its mass.
template <int DT>
__device__ Cut sorted_cut(const Search<DT>& r, const Setting& set, double all, u64 above_m, unsigned above_c, Entry* e, u64* m) {
    DrawLds& l = r.l;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    u64 key = ~0ull;
    if (tid < r.n) {
        const Entry x = r.list[tid];
        key = (u64)~order_key(x.v) << 32 | (unsigned)x.id;
    }
    for (int k = 2; k / 2 < r.n; k *= 2) {
        auto step = [&](int j, u64 o) {
            if ((o < key) == (((tid & j) == 0) == ((tid & k) == 0))) key = o;
        };
        for (int j = k / 2; j >= 64; j /= 2) {
            __syncthreads();
            l.mass[tid] = key;
            __syncthreads();
            step(j, l.mass[tid ^ j]);
        }
        if (k >= 64) step(32, from_xor<32>(key));
        if (k >= 32) step(16, from_xor<16>(key));
        if (k >= 16) step(8, from_xor<8>(key));
        if (k >= 8) step(4, from_xor<4>(key));
        if (k >= 4) step(2, from_xor<2>(key));
        step(1, from_xor<1>(key));
    }
    const uint32_t h = ~(uint32_t)(key >> 32);
    const bool in = tid < r.n;
    e->v = in ? __uint_as_float(h & 0x80000000u ? h & 0x7FFFFFFFu : ~h) : -INFINITY;
    e->id = (int)(unsigned)key;
    *m = in ? mass44(r.y(e->v)) : 0;
    u64 upto = wave_upto(*m);
    __syncthreads();
    if (lane == 63) l.wm[wv] = upto;
    if (tid == 0) l.above_mass = 0;
    __syncthreads();
    upto += above_m;
    for (int i = 0; i < wv; ++i) upto += l.wm[i];
    const unsigned rank = above_c + tid;
    auto in_k = [&](unsigned x) { return !set.by_k || x < (unsigned)set.top_k; };
    if (in && in_k(rank) && (tid == r.n - 1 || !in_k(rank + 1))) l.above_mass = upto;
    __syncthreads();
    const double goal = (double)set.top_p * (set.by_k ? (double)l.above_mass : all);
    // (the first listed rank is kept whatever the roundings of sums above it)
    auto in_p = [&](u64 before) { return !set.by_p || (double)before < goal; };
    const bool kept = in && (tid == 0 || (in_k(rank) && in_p(upto - *m)));
    if (kept && (tid == r.n - 1 || !in_k(rank + 1) || !in_p(upto))) l.cut_f = e->v, l.cut_id = e->id;
    __syncthreads();
    Cut c;
    c.f = l.cut_f, c.id = l.cut_id;
    return c;
}

template <int DT>
__global__ void __launch_bounds__(kDThreads) k_draw_pick(DrawArgs a) {
    __shared__ DrawLds l;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const Setting set(a, row);
    const size_t row0 = (size_t)row * a.S;
    // (asked for together; what a row without filters, or a bad one, finds there is not used)
    RowPlan plan = a.plan[row];
    const unsigned listed = set.filters() ? a.listed[row] : 0u;
    const double shard_above = tid < a.S ? a.above[row0 + tid] : 0.0;
    const Whole w(a, row);
    if (!set.ok || w.bad || !(w.top > -INFINITY) || set.T == 0.f) {
        const bool greedy = set.ok && !w.bad && w.top > -INFINITY;
        int best = w.mine.top == w.top ? w.mine.arg : 0x7FFFFFFF;
        best = wave_all(best, [](int a, int b) { return min(a, b); });
        if (tid == 0) {
            a.token[row] = greedy ? best : -1;
            if (a.prob) a.prob[row] = greedy ? 1.f : 0.f;
            if (a.kept) a.kept[row] = greedy ? 1 : 0;
        }
        return;
    }
    const bool filters = set.filters();
    const bool fits = listed <= (unsigned)kListMax;
    Search<DT> r{a, row * a.stride, fits ? a.list + (size_t)row * kListMax : nullptr, fits ? (int)listed : a.V, w.top, set.scale, l};
    if (tid < kShardsMax) l.shard[tid] = 0;
    if (tid == 0) l.kept = 0;
    __syncthreads();
    Cut cut;
    unsigned above_c = 0;
    if (filters) {
        u64 above_m = (u64)rint(plan.above_m);        // masses in units of 2^-44 of the row's largest weight
        above_c = plan.above_c;
        if (!fits) above_m = 0, above_c = 0, plan.rank = set.by_k || set.by_p;
        auto count = [&](int id, float v, u64 m) -> unsigned {
            if (!cut.keeps(v, id) || weight(r.y(v)) < (double)set.min_p) return 0u;
            atomicAdd(&l.shard[id / kShard], m);
            return 1u;
        };
        unsigned n = 0;
        if (fits && listed <= (unsigned)kMembers) {
            Entry e{-INFINITY, 0};
            u64 m = 0;
            if (plan.rank) {
                cut = sorted_cut(r, set, plan.all, above_m, above_c, &e, &m);
            } else if (tid < r.n) {
                e = r.list[tid];
                m = mass44(r.y(e.v));
            }
            if (e.v > -INFINITY) n = count(e.id, e.v, m);
        } else {
            if (plan.rank && set.by_k) cut = last_kept<true>(r, cut, (unsigned)set.top_k, 0.0, 0.0, above_m, above_c);
            if (plan.rank && set.by_p) {
                // (without top-k the row's mass is known; the list alone holds what top-k kept)
                const bool whole = fits && !set.by_k;
                cut = last_kept<false>(r, cut, 0u, whole ? 0.0 : (double)set.top_p, whole ? (double)set.top_p * plan.all : 0.0, above_m, above_c);
            }
            r.each([&](int id, float v) { n += count(id, v, mass44(r.y(v))); });
        }
        n = wave_sum(n);
        if (lane == 0 && n) atomicAdd(&l.kept, n);
        __syncthreads();
    }
    // kept mass per shard, in 2^-44 of the row's largest weight
    if (tid < a.S) {
        double m = 0.0;
        if (w.mine.top > -INFINITY && (!filters || fits))
            m = (filters ? shard_above : w.mine.mass) * weight(r.y(w.mine.top));
        l.ws[tid] = m + (double)l.shard[tid];
    }
    const unsigned finite = wave_sum(w.mine.finite);
    if (tid == 0) l.first = kDThreads, l.last = 0;
    __syncthreads();
    const unsigned kept = filters ? above_c + l.kept : finite;
    // the shard that holds the token, found by every wave (sums may round up to the goal: then the last one
    // with any mass)
    const double here = lane < a.S ? l.ws[lane] : 0.0;
    const double through = wave_upto(here), all = from_lane(through, 63), goal = a.u[row] * all;
    const u64 past = __ballot(here > 0.0 && through > goal), some = __ballot(here > 0.0);
    const int run = past ? __ffsll(past) - 1 : 63 - __clzll(some);
    const double rest = goal - from_lane(through - here, run);
    // its ids in order, four a thread
    double own[4], sum = 0.0;
    const int id0 = run * kShard + 4 * tid;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float v = id0 + k < a.V ? logit<DT>(a.z, r.base + id0 + k) : -INFINITY;
        const double x = weight(r.y(v));
        own[k] = cut.keeps(v, id0 + k) && x >= (double)set.min_p ? x * 17592186044416.0 : 0.0;
        sum += own[k];
    }
    double upto = wave_upto(sum);
    if (lane == 63) l.wd[wv] = upto;
    __syncthreads();
    for (int i = 0; i < wv; ++i) upto += l.wd[i];
    note_first_last(l, sum > 0.0 && upto > rest ? tid : -1, sum > 0.0 ? tid : -1);
    __syncthreads();
    if (tid == (int)(l.first < (unsigned)kDThreads ? l.first : l.last)) {
        // the first id of the thread's whose mass passes the rest, or its last with any mass
        double m = upto - sum, x = 0.0;
        int token = -1;
        bool done = false;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (own[k] > 0.0 && !done) {
                m += own[k];
                token = id0 + k, x = own[k];
                done = m > rest;
            }
        a.token[row] = token;
        if (a.prob) a.prob[row] = (float)(x / all);
        if (a.kept) a.kept[row] = (int)kept;
    }
}

namespace {

// the workspace's parts, each 16-byte aligned; null: its size
uint64_t draw_workspace(int V, int64_t rows, char* p, DrawArgs* a) {
    const int64_t S = (V + kShard - 1) / kShard;
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        char* const q = p ? p + at : nullptr;
        at += (bytes + 15) / 16 * 16;
        return q;
    };
    a->S = (int)S;
    a->head = (Head*)take(rows * S * sizeof(Head));
    a->bins = (u64*)take(rows * S * kCoarse * 8);
    a->above = (double*)take(rows * S * 8);
    a->plan = (RowPlan*)take(rows * sizeof(RowPlan));
    a->list = (Entry*)take(rows * kListMax * sizeof(Entry));
    a->listed = (unsigned*)take(rows * 4);
    return at;
}

template <int DT>
int draw_launch(DrawArgs& a, int rows, bool filters, hipStream_t st) {
    void* args[] = {&a};
    const dim3 grid(a.S, rows);
    if (hipLaunchKernel((const void*)k_draw_shard<DT>, grid, dim3(kShardThreads), args, 0, st) != hipSuccess) return LOOPSPEC_EHIP;
    if (filters && hipLaunchKernel((const void*)k_draw_list<DT>, grid, dim3(kShardThreads), args, 0, st) != hipSuccess) return LOOPSPEC_EHIP;
    return hipLaunchKernel((const void*)k_draw_pick<DT>, dim3(rows), dim3(kDThreads), args, 0, st) == hipSuccess ? LOOPSPEC_OK : LOOPSPEC_EHIP;
}

}  // namespace
}  // namespace ls

extern "C" {

uint64_t loopspec_sample_workspace_bytes(int32_t vocab, int32_t rows) {
    if (vocab < 1 || vocab > ls::kDMaxVocab || rows < 1 || rows > 65535) return 0;
    ls::DrawArgs a{};
    return ls::draw_workspace(vocab, rows, nullptr, &a);
}

int loopspec_sample(const loopspec_sample_cfg* cfg, int32_t rows, const void* logits_dev, int64_t stride, const double* u_dev,
                    int32_t* token_dev, float* prob_dev, int32_t* kept_dev, void* workspace_dev, uint64_t workspace_bytes,
                    void* stream) {
    using namespace ls;
    if (!cfg || rows < 0 || rows > 65535 || stride < 0) return LOOPSPEC_EINVAL;
    if (cfg->vocab < 1 || cfg->vocab > kDMaxVocab) return LOOPSPEC_EINVAL;
    if (cfg->dtype != LOOPSPEC_F32 && cfg->dtype != LOOPSPEC_BF16 && cfg->dtype != LOOPSPEC_F16) return LOOPSPEC_EINVAL;
    if (!cfg->temperature_dev && !(cfg->temperature >= 0.f && cfg->temperature < 3e38f)) return LOOPSPEC_EINVAL;
    if (!cfg->top_p_dev && !(cfg->top_p > 0.f && cfg->top_p <= 1.f)) return LOOPSPEC_EINVAL;
    if (!cfg->min_p_dev && !(cfg->min_p >= 0.f && cfg->min_p <= 1.f)) return LOOPSPEC_EINVAL;
    if (!rows) return LOOPSPEC_OK;            // (empty tensors have no address)
    if (!logits_dev || !u_dev || !token_dev || (uintptr_t)logits_dev % (cfg->dtype == LOOPSPEC_F32 ? 4 : 2)) return LOOPSPEC_EINVAL;
    DrawArgs a{logits_dev, stride, u_dev, cfg->temperature_dev, cfg->top_p_dev, cfg->min_p_dev, cfg->top_k_dev,
               cfg->temperature, cfg->top_p, cfg->min_p, cfg->top_k, token_dev, prob_dev, kept_dev, cfg->vocab};
    if (!workspace_dev || ((uintptr_t)workspace_dev & 15) || workspace_bytes < draw_workspace(cfg->vocab, rows, (char*)workspace_dev, &a))
        return LOOPSPEC_EINVAL;
    const bool filters = cfg->top_k_dev || cfg->top_p_dev || cfg->min_p_dev || (cfg->top_k > 0 && cfg->top_k < cfg->vocab) ||
                         cfg->top_p < 1.f || cfg->min_p > 0.f;
    hipStream_t st = (hipStream_t)stream;
    if (cfg->dtype == LOOPSPEC_F32) return draw_launch<LOOPSPEC_F32>(a, rows, filters, st);
    if (cfg->dtype == LOOPSPEC_BF16) return draw_launch<LOOPSPEC_BF16>(a, rows, filters, st);
    return draw_launch<LOOPSPEC_F16>(a, rows, filters, st);
}

}  // extern "C"
