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
// What top-k and top-p keep is the ranks down to some last one.  A histogram
// over 2048 bins of 1/32 octave of weight tells the bin that holds it (counts
// for top-k; masses for top-p, of what top-k kept).  The bin's members, when
// there are at most 1024, go to LDS and a thread each finds its member's rank
// against all others; otherwise ranges of the logits' order-preserving integer
// keys are searched the same way until a bin is a single key, and ties are
// counted off by id.
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
constexpr int kDList = kDThreads;
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
// 2^(y + up), y <= 0 (2^(up - 200) below y = -200): y = n + f, the polynomial
// interpolates 2^f at the Chebyshev points of [-1/2, 1/2] and is 1 at 0.  n comes
// from adding 1.5 * 2^52, whose low word it then is, and goes to the exponent as
// it is: conversions and ldexp take several times an addition's cycles.
__device__ __forceinline__ double weight(double y, int up = 0) {
    constexpr double M = 6755399441055744.0;
    y = fmax(y, -200.0);
    const double t = y + M, f = y - (t - M);
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
    p = fma(p, f, 1.0);
    return __hiloint2double(__double2hiint(p) + ((__double2loint(t) + up) << 20), __double2loint(p));
}
// the weight in units of 2^-44, to nearest: adding 2^52 leaves it in the low bits
__device__ __forceinline__ u64 mass44(double y) {
    return (u64)__double_as_longlong(weight(y, 44) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
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
    union {
        u64 mass[kDBins];
        float run[kDBins * 2];                        // the logits of the wave that holds the token
    };
    unsigned count[kDBins];
    Member list[kDList];
    u64 wm[kDWaves];
    double wd[kDWaves];
    unsigned wc[kDWaves];
    float wf[kDWaves];
    unsigned first, last, listed, lo, hi, cnt, above_cnt;
    u64 bin_mass, above_mass;
    int bad, token;
    float cut_f;
    int cut_id;
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
    static constexpr int B = 16;                      // logits of a lane's batch
    const void* z;
    int64_t base;
    int V, seg;                                       // wave w owns ids [w * seg, (w + 1) * seg)
    bool vec;                                         // 4-byte aligned: four logits a load
    DrawLds& l;
    float top = 0.f;                                  // the largest logit
    double scale = 0.0;                               // log2(e) / T
    float x[HELD ? kDHeld : 1];

    __device__ __forceinline__ float at(int id) const { return logit<DT>(z, base + id); }
    // four logits from id, a load for 4-byte aligned rows
    __device__ __forceinline__ void load4(int id, float* v) const {
        if (DT == LOOPSPEC_F32) {
            const u32x4_a4 u = *(const u32x4_a4*)((const float*)z + base + id);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(u[i]);
        } else {
            const u32x2_a4 u = *(const u32x2_a4*)((const uint16_t*)z + base + id);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = half_bits(DT, i & 1 ? u[i >> 1] >> 16 : u[i >> 1] & 0xFFFFu);
        }
    }
    __device__ __forceinline__ int first() const { return (int)(threadIdx.x >> 6) * seg + (int)(threadIdx.x & 63) * 4; }
    __device__ __forceinline__ int end() const { return min(((int)(threadIdx.x >> 6) + 1) * seg, V); }
    // batch j: 4 logits in each of 4 consecutive blocks of 256 ids of the wave; -infinity where there is none
    __device__ __forceinline__ void load_batch(int j, float* v) const {
        const int b = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) * seg + j * (64 * B));
        if (b + 64 * B <= __builtin_amdgcn_readfirstlane(end()) && vec) {
#pragma unroll
            for (int k = 0; k < B / 4; ++k) load4(first() + j * (64 * B) + k * 256, v + 4 * k);
        } else {
#pragma unroll
            for (int k = 0; k < B; ++k) {
                const int id = first() + j * (64 * B) + (k / 4) * 256 + k % 4;
                v[k] = id < end() ? at(id) : -INFINITY;
            }
        }
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

// The bin that holds the last kept rank: the first one through which the count
// reaches `need` (COUNT), or the mass reaches `goal`; the last occupied one when
// none does.  share > 0: the goal is that share of the bins' whole mass.  What
// the bin and (above_m and above_c included) all above it hold is left in l.
template <bool MASS, bool COUNT>
__device__ unsigned pick_bin(DrawLds& l, unsigned need, double share, double* goal, u64 above_m, unsigned above_c) {
    __syncthreads();
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, b0 = 2 * tid;
    u64 m[2] = {0, 0};
    unsigned c[2] = {0, 0};
    if (MASS) m[0] = l.mass[b0], m[1] = l.mass[b0 + 1];
    if (COUNT) c[0] = l.count[b0], c[1] = l.count[b0 + 1];
    u64 sm = m[0] + m[1];
    unsigned sc = c[0] + c[1];
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        if (MASS) {
            const u64 v = __shfl_up(sm, o);
            if (lane >= o) sm += v;
        }
        if (COUNT) {
            const unsigned k = __shfl_up(sc, o);
            if (lane >= o) sc += k;
        }
    }
    if (lane == 63) l.wm[wv] = sm, l.wc[wv] = sc;
    __syncthreads();
    sm += above_m - m[0] - m[1];
    sc += above_c - c[0] - c[1];
    u64 all = 0;
    for (int i = 0; i < kDWaves; ++i) {
        if (i < wv) sm += l.wm[i], sc += l.wc[i];
        all += l.wm[i];
    }
    if (share > 0.0) *goal = share * (double)all;
    const u64 am[2] = {sm, sm + m[0]};                // above each of the thread's bins
    const unsigned ac[2] = {sc, sc + c[0]};
#pragma unroll
    for (int i = 1; i >= 0; --i) {
        if (COUNT ? !c[i] : !m[i]) continue;
        const bool reach = goal ? (double)(am[i] + m[i]) >= *goal : ac[i] + c[i] >= need;
        if (reach) atomicMin(&l.first, (unsigned)(b0 + i));
        atomicMax(&l.last, (unsigned)(b0 + i));
    }
    __syncthreads();
    const unsigned at = l.first < (unsigned)kDBins ? l.first : l.last;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (at == (unsigned)(b0 + i)) l.cnt = c[i], l.bin_mass = m[i], l.above_mass = am[i], l.above_cnt = ac[i];
    __syncthreads();
    return at;
}

// Id of tie number `tie` (from 0, in id order) among the logits equal to f.
template <int DT, bool HELD>
__device__ int tie_id(const DrawRow<DT, HELD>& r, float f, unsigned tie) {
    DrawLds& l = r.l;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    unsigned n = 0;
    r.each([&](int, float v) { n += v == f; });
    n = wave_sum(n);
    __syncthreads();
    if (lane == 0) l.wc[wv] = n;
    __syncthreads();
    unsigned before = 0;
    for (int i = 0; i < wv; ++i) before += l.wc[i];
    if (before <= tie && tie < before + n) {
        for (int i = wv * r.seg;; i += 64) {
            const bool eq = i + lane < r.V && r.at(i + lane) == f;
            const u64 m = __ballot(eq);
            if (eq && before + __popcll(m & ((1ull << lane) - 1)) == tie) l.token = i + lane;
            before += __popcll(m);
            if (before > tie) break;
        }
    }
    __syncthreads();
    const int id = l.token;
    __syncthreads();
    return id;
}

// The last kept rank of what `from` keeps: the first `need` ranks (BY_COUNT), or
// the ranks whose preceding mass is below `share` of all of it.
template <bool BY_COUNT, int DT, bool HELD>
__device__ Cut last_kept(const DrawRow<DT, HELD>& r, Cut from, unsigned need, double share) {
    DrawLds& l = r.l;
    const int tid = threadIdx.x;
    double goal = 0.0, *const goalp = BY_COUNT ? nullptr : &goal;
    clear_bins<!BY_COUNT, BY_COUNT>(l);
    r.each([&](int id, float v) {
        if (!from.keeps(v, id)) return;
        if (BY_COUNT)
            atomicAdd(&l.count[r.bin(v)], 1u);
        else
            atomicAdd(&l.mass[r.bin(v)], mass44(r.y(v)));
    });
    const int picked = (int)pick_bin<!BY_COUNT, BY_COUNT>(l, need, share, goalp, 0, 0);
    u64 above_m = l.above_mass;
    unsigned above_c = l.above_cnt;
    r.each([&](int id, float v) {
        if (r.bin(v) != picked || !from.keeps(v, id)) return;
        const unsigned at = atomicAdd(&l.listed, 1u);
        if (at < (unsigned)kDList) l.list[at] = Member{v, id, BY_COUNT ? 0 : mass44(r.y(v))};
    });
    if (tid == 0) l.cnt = 0;
    __syncthreads();
    const unsigned members = l.listed;
    if (members <= (unsigned)kDList) {
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
        if (kept && rank + 1 == l.cnt) l.cut_f = me.v, l.cut_id = me.id;
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
        const u64 bin_mass = l.bin_mass;
        __syncthreads();
        if (shift == 0) {
            // n equal logits (of equal masses), of which the first e are kept
            unsigned e = n;
            if (BY_COUNT) {
                e = min(n, need - above_c);
            } else if (const u64 one = bin_mass / n) {
                const double want = (goal - (double)above_m) / (double)one;
                e = want < (double)n ? (unsigned)max(want, 0.0) : n;
                while (e > 0 && (double)(above_m + (u64)(e - 1) * one) >= goal) --e;
                while (e < n && (double)(above_m + (u64)e * one) < goal) ++e;
            }
            Cut c;
            c.f = __uint_as_float(h & 0x80000000u ? h & 0x7FFFFFFFu : ~h);
            c.id = tie_id(r, c.f, e - 1);
            return c;
        }
        lo = max(lo, h - ((1u << shift) - 1));
        hi = h;
    }
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

    // what is kept, but for min-p
    Cut cut;
    if (by_k) cut = last_kept<true>(r, cut, (unsigned)top_k, 0.0);
    if (by_p) cut = last_kept<false>(r, cut, 0u, (double)top_p);

    // kept mass and count per wave
    if (once) {
        sum *= mine > -INFINITY ? weight(r.y(mine)) : 0.0;
    } else {
        r.each([&](int id, float v) {
            if (!cut.keeps(v, id)) return;
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
    const int per = HELD ? kDHeld / 16 : (r.seg + kDThreads - 1) / kDThreads, s0 = run * r.seg, s1 = min(s0 + r.seg, a.V);
    const int i0 = min(s0 + tid * per, s1), i1 = min(i0 + per, s1);
    if (HELD) {
        if (wv == run) r.each([&](int id, float v) { l.run[id - s0] = v; });
        __syncthreads();
    }
    auto weigh = [&](int id) {
        const float v = HELD ? l.run[id - s0] : r.at(id);
        const double w = weight(r.y(v));
        return cut.keeps(v, id) && w >= (double)min_p ? w : 0.0;
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
