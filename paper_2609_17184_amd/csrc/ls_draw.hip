// One token per row of logits from a given uniform number: temperature, top-k,
// top-p and min-p, each row with its own settings.
//
//   w_v = 2^((z_v - max z) log2(e) / T);  ids ranked by (z descending, id ascending), -infinity left out:
//   top-k keeps the first k ranks; top-p, of those, the ranks whose preceding mass is below top_p of the top-k
//   mass; min-p, of those, w_v >= min_p.  The token is the smallest id whose kept mass through it exceeds
//   u * kept mass.  T = 0: the largest logit, lowest id.
//
// A row is one workgroup's.  Each of its 16 waves owns a run of ids, four
// consecutive ones a lane; up to 65536 ids the logits stay in registers from
// their only read.  Weights are taken in 64 bits (2^f by a polynomial on
// [-1/2, 1/2], off by 2^-50), since a token is decided by comparing sums with u
// times a sum.  Sums are 64-bit in an order that depends on the vocabulary
// alone; where the order of adding is not fixed (the histograms' atomics),
// masses are integers in units of 2^-44 of the largest weight.
//
// What top-k and top-p keep is the ranks above a boundary.  A histogram over
// 2048 bins of 1/32 octave of weight tells the bin that holds it (counts for
// top-k; masses for top-p, of what top-k kept); the bin's members are listed in
// LDS and searched the same way over ranges of the logits' order-preserving
// integer keys until a bin is a single key, where ties are cut by id.  A bin
// with too many members is searched in place.
//
// The token: the kept mass per wave tells the run of ids, then all threads take
// that run in id order.  A row without filters and of more than 65536 ids is
// read once: every lane sums against its own running maximum.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/loopspec.h"

namespace ls {

typedef unsigned long long u64;
typedef uint32_t u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_a4 __attribute__((ext_vector_type(2), aligned(4)));

constexpr int kDThreads = 1024, kDWaves = kDThreads / 64;
constexpr int kDBins = 2048;                          // two per thread
constexpr int kDList = 4096;
constexpr int kDHeld = 64;                            // logits a thread holds
constexpr int kDMaxVocab = 1 << 18;

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
    int V;
};

__device__ __forceinline__ float half_bits(int dt, uint32_t b) {
    return dt == LOOPSPEC_BF16 ? __uint_as_float(b << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)b);
}
template <int DT>
__device__ __forceinline__ float logit(const void* p, int64_t i) {
    if (DT == LOOPSPEC_F32) return ((const float*)p)[i];
    return half_bits(DT, ((const uint16_t*)p)[i]);
}
// order-preserving integer of a float that is no NaN; both zeros alike
__device__ __forceinline__ uint32_t order_key(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
// 2^(n + up) 2^f of y = n + f <= 0, from 2^-200 on: the polynomial interpolates
// 2^f at the Chebyshev points of [-1/2, 1/2] and is 1 at 0
__device__ __forceinline__ double weight(double y, int up = 0) {
    y = fmax(y, -200.0);
    const double n = rint(y), f = y - n;
    double p = 7.070977866508138e-09;
    p = fma(p, f, 1.0205905413765595e-07);
    p = fma(p, f, 1.3215451633221434e-06);
    p = fma(p, f, 1.5252672924850737e-05);
    p = fma(p, f, 0.00015403530424776529);
    p = fma(p, f, 0.0013333558200794592);
    p = fma(p, f, 0.009618129107618665);
    p = fma(p, f, 0.05550410866465167);
    p = fma(p, f, 0.24022650695910075);
    p = fma(p, f, 0.6931471805599462);
    return ldexp(fma(p, f, 1.0), (int)n + up);
}
// the weight in units of 2^-44, to nearest: adding 2^52 leaves it in the low bits
__device__ __forceinline__ u64 mass44(double y) {
    return (u64)__double_as_longlong(weight(y, 44) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
}

struct DrawLds {
    u64 mass[kDBins];
    unsigned count[kDBins];
    uint2 list[kDList];                               // key, id
    u64 wm[kDWaves];
    double wd[kDWaves];
    unsigned wc[kDWaves];
    float wf[kDWaves];
    unsigned first, last, listed, lo, hi, cnt, above_cnt;
    u64 bin_mass, above_mass;
    int bad, token;
};

template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
    return v;
}

// the row as its workgroup sees it
template <int DT, bool HELD>
struct DrawRow {
    static constexpr int B = 16;                      // logits of a lane's batch: 4 of each of 4 neighbouring rows of 256 ids
    const void* z;
    int64_t base;
    int V, seg;                                       // wave w owns ids [w * seg, (w + 1) * seg)
    bool vec;                                         // 4-byte aligned: four logits a load
    DrawLds& l;
    float top = 0.f;                                  // the largest logit
    double scale = 0.0;                               // log2(e) / T
    float x[HELD ? kDHeld : 1];

    __device__ __forceinline__ float at(int id) const { return logit<DT>(z, base + id); }
    // four logits from id, -infinity outside [., end)
    __device__ __forceinline__ void load4(int id, int end, float* v) const {
        if (id + 4 <= end && vec) {
            if (DT == LOOPSPEC_F32) {
                const u32x4_a4 u = *(const u32x4_a4*)((const float*)z + base + id);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(u[i]);
            } else {
                const u32x2_a4 u = *(const u32x2_a4*)((const uint16_t*)z + base + id);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = half_bits(DT, i & 1 ? u[i >> 1] >> 16 : u[i >> 1] & 0xFFFFu);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = id + i < end ? at(id + i) : -INFINITY;
        }
    }
    __device__ __forceinline__ int first() const { return (threadIdx.x >> 6) * seg + (threadIdx.x & 63) * 4; }
    __device__ __forceinline__ int end() const { return min(((int)(threadIdx.x >> 6) + 1) * seg, V); }
    __device__ __forceinline__ void load_batch(int j, float* v) const {
#pragma unroll
        for (int k = 0; k < B / 4; ++k) load4(first() + (j * (B / 4) + k) * 256, end(), v + 4 * k);
    }
    __device__ __forceinline__ void hold() {
        if constexpr (HELD) {
#pragma unroll
            for (int j = 0; j < kDHeld / B; ++j) load_batch(j, x + j * B);
        }
    }
    // f(id, logit) for every id of the thread, and -infinity for places without one
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        if constexpr (HELD) {
#pragma unroll
            for (int j = 0; j < kDHeld / 4; ++j) {
                if (j * 256 >= seg) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) f(first() + j * 256 + i, x[j * 4 + i]);
            }
        } else {
            for (int j = 0; j * 64 * B < seg; ++j) {
                float v[B];
                load_batch(j, v);
#pragma unroll
                for (int i = 0; i < B; ++i) f(first() + (j * (B / 4) + i / 4) * 256 + i % 4, v[i]);
            }
        }
    }
    __device__ __forceinline__ double y(float v) const { return ((double)v - (double)top) * scale; }
    __device__ __forceinline__ int bin(float v) const {
        const float d = (top - v) * (float)(32.0 * scale);
        return d < (float)(kDBins - 1) ? (int)d : kDBins - 1;       // infinity and NaN (0 * inf): the last bin
    }
};

__device__ __forceinline__ void clear_bins(DrawLds& l) {
    __syncthreads();
    for (int i = threadIdx.x; i < kDBins; i += kDThreads) l.mass[i] = 0, l.count[i] = 0;
    if (threadIdx.x == 0) l.first = kDBins, l.last = 0;
    __syncthreads();
}

// The bin that holds the boundary: the first one through which the count
// reaches `need` (by count) or the mass reaches `goal`, the last occupied one
// when none does.  l.first is its number; l.cnt and l.bin_mass what it holds,
// l.above_* what lies above it, above_m and above_c included.
__device__ void pick_bin(DrawLds& l, bool by_count, unsigned need, double goal, u64 above_m, unsigned above_c) {
    __syncthreads();
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, b0 = 2 * tid;
    const u64 m[2] = {l.mass[b0], l.mass[b0 + 1]};
    const unsigned c[2] = {l.count[b0], l.count[b0 + 1]};
    u64 sm = m[0] + m[1];
    unsigned sc = c[0] + c[1];
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const u64 v = __shfl_up(sm, o);
        const unsigned k = __shfl_up(sc, o);
        if (lane >= o) sm += v, sc += k;
    }
    if (lane == 63) l.wm[wv] = sm, l.wc[wv] = sc;
    __syncthreads();
    sm += above_m - m[0] - m[1];
    sc += above_c - c[0] - c[1];
    for (int i = 0; i < wv; ++i) sm += l.wm[i], sc += l.wc[i];
    u64 am[2] = {sm, sm + m[0]};                      // above each of the thread's bins
    unsigned ac[2] = {sc, sc + c[0]};
#pragma unroll
    for (int i = 1; i >= 0; --i) {
        if (!c[i]) continue;
        atomicMax(&l.last, (unsigned)(b0 + i));
        if (by_count ? ac[i] + c[i] >= need : (double)(am[i] + m[i]) >= goal) atomicMin(&l.first, (unsigned)(b0 + i));
    }
    __syncthreads();
    const unsigned at = l.first < (unsigned)kDBins ? l.first : l.last;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (at == (unsigned)(b0 + i)) l.cnt = c[i], l.bin_mass = m[i], l.above_mass = am[i], l.above_cnt = ac[i];
    __syncthreads();
    if (tid == 0) l.first = at;
    __syncthreads();
}

// Boundary of a filter: keys above `key` are kept, and of those equal to it
// the first `ties` by id of `all`; `mass` is what is kept (by mass only).
struct Bound {
    uint32_t key;
    unsigned ties, all;
};

// Finds it.  The first `need` ranks (by count), or the ranks whose preceding
// mass is below `goal`, among the keys from `floor` on (top-k's boundary, which
// takes `floor_ties` of the keys equal to it: they have ranks, but no effect
// below, since top-p's boundary never lies behind top-k's).
template <int DT, bool HELD>
__device__ Bound boundary(const DrawRow<DT, HELD>& r, bool by_count, unsigned need, double goal, uint32_t floor) {
    DrawLds& l = r.l;
    const int tid = threadIdx.x;
    clear_bins(l);
    r.each([&](int, float v) {
        if (v == -INFINITY || order_key(v) < floor) return;
        const int b = r.bin(v);
        atomicAdd(&l.count[b], 1u);
        if (!by_count) atomicAdd(&l.mass[b], mass44(r.y(v)));
    });
    pick_bin(l, by_count, need, goal, 0, 0);
    const int picked = (int)l.first;
    u64 above_m = l.above_mass;
    unsigned above_c = l.above_cnt, members = l.cnt;
    const bool list = members <= (unsigned)kDList;
    if (tid == 0) l.listed = 0;
    __syncthreads();
    if (list)
        r.each([&](int id, float v) {
            if (v == -INFINITY || r.bin(v) != picked || order_key(v) < floor) return;
            l.list[atomicAdd(&l.listed, 1u)] = make_uint2(__float_as_uint(v), (unsigned)id);
        });
    __syncthreads();
    uint32_t lo = 0, hi = 0xFFFFFFFFu;                // keys of the range that holds the boundary
    auto members_of = [&](auto f) {
        if (list) {
            for (unsigned i = tid; i < members; i += kDThreads) f(__uint_as_float(l.list[i].x));
        } else {
            r.each([&](int, float v) {
                if (v != -INFINITY && r.bin(v) == picked && order_key(v) >= floor) f(v);
            });
        }
    };
    for (;;) {
        // the ends of what is left, then its histogram
        if (tid == 0) l.lo = 0xFFFFFFFFu, l.hi = 0;
        clear_bins(l);
        uint32_t a = 0xFFFFFFFFu, b = 0;
        members_of([&](float v) {
            const uint32_t k = order_key(v);
            if (k >= lo && k <= hi) a = min(a, k), b = max(b, k);
        });
        if (a <= b) {
            atomicMin(&l.lo, a);
            atomicMax(&l.hi, b);
        }
        __syncthreads();
        lo = l.lo, hi = l.hi;
        int shift = 0;
        while (((hi - lo) >> shift) >= (uint32_t)kDBins) ++shift;
        members_of([&](float v) {
            const uint32_t k = order_key(v);
            if (k < lo || k > hi) return;
            const int bin = (int)((hi - k) >> shift);
            atomicAdd(&l.count[bin], 1u);
            if (!by_count) atomicAdd(&l.mass[bin], mass44(r.y(v)));
        });
        pick_bin(l, by_count, need, goal, above_m, above_c);
        above_m = l.above_mass, above_c = l.above_cnt;
        const uint32_t h = hi - (l.first << shift);
        const unsigned n = l.cnt;
        const u64 bin_mass = l.bin_mass;
        __syncthreads();
        if (shift == 0) {
            if (by_count) return Bound{h, min(n, need - above_c), n};
            const u64 one = bin_mass / n;             // equal keys have equal masses
            unsigned e = n;
            if (one) {
                const double want = (goal - (double)above_m) / (double)one;
                e = want < (double)n ? (unsigned)max(want, 0.0) : n;
                while (e > 0 && (double)(above_m + (u64)(e - 1) * one) >= goal) --e;
                while (e < n && (double)(above_m + (u64)e * one) < goal) ++e;
            }
            return Bound{h, e, n};
        }
        lo = max(lo, h - ((1u << shift) - 1));
        hi = h;
    }
}

// The id of tie number `ties` (from 0) among the keys equal to `key`, in id
// order: the first that is left out.  Every thread gets it.
template <int DT, bool HELD>
__device__ int tie_cut(const DrawRow<DT, HELD>& r, uint32_t key, unsigned ties) {
    DrawLds& l = r.l;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    unsigned n = 0;
    r.each([&](int, float v) { n += v != -INFINITY && order_key(v) == key; });
    n = wave_sum(n);
    __syncthreads();
    if (lane == 0) l.wc[wv] = n;
    __syncthreads();
    unsigned before = 0;
    for (int i = 0; i < wv; ++i) before += l.wc[i];
    if (before <= ties && ties < before + n) {
        for (int i = wv * r.seg;; i += 64) {
            const float v = i + lane < r.V ? r.at(i + lane) : -INFINITY;
            const bool tie = v != -INFINITY && order_key(v) == key;
            const u64 m = __ballot(tie);
            if (tie && before + __popcll(m & ((1ull << lane) - 1)) == ties) l.token = i + lane;
            before += __popcll(m);
            if (before > ties) break;
        }
    }
    __syncthreads();
    const int cut = l.token;
    __syncthreads();
    return cut;
}

template <int DT, bool HELD>
__global__ void __launch_bounds__(kDThreads) k_draw(DrawArgs a) {
    __shared__ DrawLds l;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const float T = a.temperature ? a.temperature[row] : a.temperature1;
    const float top_p = a.top_p ? a.top_p[row] : a.top_p1, min_p = a.min_p ? a.min_p[row] : a.min_p1;
    const int top_k = a.top_k ? a.top_k[row] : a.top_k1;
    const double u = a.u[row];
    bool ok = T >= 0.f && T < INFINITY && top_p > 0.f && top_p <= 1.f && min_p >= 0.f && min_p <= 1.f && u >= 0.0 && u < 1.0;
    DrawRow<DT, HELD> r{a.z, row * a.stride, a.V, ((a.V + kDWaves - 1) / kDWaves + 255) / 256 * 256, false, l};
    r.vec = ((uintptr_t)a.z + (uint64_t)r.base * (DT == LOOPSPEC_F32 ? 4 : 2)) % 4 == 0;
    if (T > 0.f) r.scale = 1.4426950408889634074 / (double)T;
    const bool by_k = top_k > 0 && top_k < a.V, by_p = top_p < 1.f, by_m = min_p > 0.f;
    // rows read once: the lane's sum against its own maximum
    const bool once = !HELD && T > 0.f && !by_k && !by_p && !by_m;

    float top = -INFINITY;
    bool bad = false;
    double sum = 0.0;
    unsigned cnt = 0;
    if (once) {
        constexpr int B = DrawRow<DT, HELD>::B;
        float v[B], nx[B];
        r.load_batch(0, v);
        for (int j = 0; j * 64 * B < r.seg; ++j) {
            if ((j + 1) * 64 * B < r.seg) r.load_batch(j + 1, nx);
            float m = v[0];
#pragma unroll
            for (int i = 0; i < B; ++i) {
                bad |= !(v[i] < INFINITY);
                m = fmaxf(m, v[i]);
            }
            if (__any(m > top)) {
                const float now = fmaxf(top, m);
                if (top > -INFINITY) sum *= weight(((double)top - (double)now) * r.scale);
                top = now;
            }
#pragma unroll
            for (int i = 0; i < B; ++i) {
                const double w = weight(((double)v[i] - (double)top) * r.scale);
                if (v[i] != -INFINITY) sum += w, ++cnt;
            }
#pragma unroll
            for (int i = 0; i < B; ++i) v[i] = nx[i];
        }
    } else {
        r.hold();
        r.each([&](int, float v) {
            bad |= !(v < INFINITY);
            top = fmaxf(top, v);
        });
    }
    const float mine = top;
    for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
    if (tid == 0) l.bad = 0, l.token = 0x7FFFFFFF, l.first = kDThreads, l.last = 0;
    if (lane == 0) l.wf[wv] = top;
    __syncthreads();
    if (bad) l.bad = 1;
    for (int i = 0; i < kDWaves; ++i) top = fmaxf(top, l.wf[i]);
    __syncthreads();
    ok = ok && !l.bad && top > -INFINITY;
    if (!ok) {
        if (tid == 0) {
            a.token[row] = -1;
            if (a.prob) a.prob[row] = 0.f;
            if (a.kept) a.kept[row] = 0;
        }
        return;
    }
    if (T == 0.f) {
        int best = 0x7FFFFFFF;
        r.each([&](int i, float v) {
            if (v == top) best = min(best, i);
        });
        if (best < 0x7FFFFFFF) atomicMin(&l.token, best);
        __syncthreads();
        if (tid == 0) {
            a.token[row] = l.token;
            if (a.prob) a.prob[row] = 1.f;
            if (a.kept) a.kept[row] = 1;
        }
        return;
    }
    r.top = top;

    // what is kept: keys above bd.key, those equal to it below the id `cut`, weights from min_p on
    Bound bd{0, 0, 0};
    if (by_k) bd = boundary(r, true, (unsigned)top_k, 0.0, 0);
    if (by_p) {
        // the mass that top-k kept, in integers: whatever falls behind its boundary among the equal keys is
        // taken off again
        u64 all = 0;
        r.each([&](int, float v) {
            if (v != -INFINITY && order_key(v) >= bd.key) all += mass44(r.y(v));
        });
        all = wave_sum(all);
        __syncthreads();
        if (lane == 0) l.wm[wv] = all;
        __syncthreads();
        all = 0;
        for (int i = 0; i < kDWaves; ++i) all += l.wm[i];
        if (bd.ties < bd.all) {
            const uint32_t b = bd.key & 0x80000000u ? bd.key & 0x7FFFFFFFu : ~bd.key;
            all -= (u64)(bd.all - bd.ties) * mass44(r.y(__uint_as_float(b)));
        }
        bd = boundary(r, false, 0u, (double)top_p * (double)all, bd.key);
    }
    const int cut = bd.ties < bd.all ? tie_cut(r, bd.key, bd.ties) : 0x7FFFFFFF;
    auto keeps = [&](int id, float v) {
        const uint32_t k = order_key(v);
        return v != -INFINITY && (k > bd.key || (k == bd.key && id < cut));
    };

    // kept mass and count per wave
    if (once) {
        sum *= mine > -INFINITY ? weight(r.y(mine)) : 0.0;
    } else {
        r.each([&](int id, float v) {
            if (!keeps(id, v)) return;
            const double w = weight(r.y(v));
            if (w >= (double)min_p) sum += w, ++cnt;
        });
    }
    sum = wave_sum(sum);
    cnt = wave_sum(cnt);
    __syncthreads();
    if (tid == 0) l.first = kDThreads, l.last = 0;
    if (lane == 0) l.wd[wv] = sum, l.wc[wv] = cnt;
    __syncthreads();
    double all = 0.0;
    unsigned kept = 0;
    for (int i = 0; i < kDWaves; ++i) all += l.wd[i], kept += l.wc[i];
    // the wave whose run of ids holds the token (sums may round up to the goal: then the last run with any mass)
    const double goal = u * all;
    double before = 0.0, rest = 0.0;
    int run = -1;
    for (int i = 0; i < kDWaves; ++i) {
        const double m = l.wd[i];
        if (m > 0.0 && (run < 0 || before <= goal)) run = i, rest = goal - before;
        if (m > 0.0 && before + m > goal) break;
        before += m;
    }
    // all threads take that run, consecutive ids each
    const int per = r.seg / kDThreads + (r.seg % kDThreads != 0), s0 = run * r.seg, s1 = min(s0 + r.seg, a.V);
    const int i0 = min(s0 + tid * per, s1), i1 = min(i0 + per, s1);
    auto weigh = [&](int id) {
        const float v = r.at(id);
        const double w = weight(r.y(v));
        return keeps(id, v) && w >= (double)min_p ? w : 0.0;
    };
    double own = 0.0;
    for (int id = i0; id < i1; ++id) own += weigh(id);
    double upto = own;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const double v = __shfl_up(upto, o);
        if (lane >= o) upto += v;
    }
    __syncthreads();
    if (lane == 63) l.wd[wv] = upto;
    __syncthreads();
    double at = 0.0;
    for (int i = 0; i < wv; ++i) at += l.wd[i];
    upto += at;
    if (own > 0.0) {
        atomicMax(&l.last, (unsigned)tid);
        if (upto > rest) atomicMin(&l.first, (unsigned)tid);
    }
    __syncthreads();
    if (tid == (int)(l.first < (unsigned)kDThreads ? l.first : l.last)) {
        // the first id of the thread's whose mass passes the rest, or its last with any mass
        double m = upto - own, w = 0.0;
        int token = -1;
        for (int id = i0; id < i1; ++id) {
            const double x = weigh(id);
            if (!(x > 0.0)) continue;
            m += x;
            token = id, w = x;
            if (m > rest) break;
        }
        a.token[row] = token;
        if (a.prob) a.prob[row] = (float)(w / all);
        if (a.kept) a.kept[row] = (int)kept;
    }
}

}  // namespace ls

extern "C" {

int loopspec_sample(const loopspec_sample_cfg* cfg, int32_t rows, const void* logits_dev, int64_t stride, const double* u_dev,
                    int32_t* token_dev, float* prob_dev, int32_t* kept_dev, void* stream) {
    using namespace ls;
    if (!cfg || rows < 0 || !logits_dev || !u_dev || !token_dev || stride < 0) return LOOPSPEC_EINVAL;
    if (cfg->vocab < 1 || cfg->vocab > kDMaxVocab) return LOOPSPEC_EINVAL;
    if (cfg->dtype != LOOPSPEC_F32 && cfg->dtype != LOOPSPEC_BF16 && cfg->dtype != LOOPSPEC_F16) return LOOPSPEC_EINVAL;
    if ((uintptr_t)logits_dev % (cfg->dtype == LOOPSPEC_F32 ? 4 : 2)) return LOOPSPEC_EINVAL;
    if (!cfg->temperature_dev && !(cfg->temperature >= 0.f && cfg->temperature < 3e38f)) return LOOPSPEC_EINVAL;
    if (!cfg->top_p_dev && !(cfg->top_p > 0.f && cfg->top_p <= 1.f)) return LOOPSPEC_EINVAL;
    if (!cfg->min_p_dev && !(cfg->min_p >= 0.f && cfg->min_p <= 1.f)) return LOOPSPEC_EINVAL;
    if (!rows) return LOOPSPEC_OK;
    DrawArgs a{logits_dev, stride, u_dev, cfg->temperature_dev, cfg->top_p_dev, cfg->min_p_dev, cfg->top_k_dev,
               cfg->temperature, cfg->top_p, cfg->min_p, cfg->top_k, token_dev, prob_dev, kept_dev, cfg->vocab};
    const bool held = cfg->vocab <= kDHeld * kDThreads;
    const void* f = cfg->dtype == LOOPSPEC_F32    ? held ? (const void*)k_draw<LOOPSPEC_F32, true> : (const void*)k_draw<LOOPSPEC_F32, false>
                    : cfg->dtype == LOOPSPEC_BF16 ? held ? (const void*)k_draw<LOOPSPEC_BF16, true> : (const void*)k_draw<LOOPSPEC_BF16, false>
                    : held                        ? (const void*)k_draw<LOOPSPEC_F16, true>
                                                  : (const void*)k_draw<LOOPSPEC_F16, false>;
    void* args[] = {&a};
    return hipLaunchKernel(f, dim3(rows), dim3(kDThreads), args, 0, (hipStream_t)stream) == hipSuccess ? LOOPSPEC_OK : LOOPSPEC_EHIP;
}

}  // extern "C"
