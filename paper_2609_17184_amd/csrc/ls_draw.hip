// One token per row of logits from a given uniform number: temperature, top-k,
// top-p and min-p, each row with its own settings.
//
//   w_v = 2^((z_v - max z) log2(e) / T);  ids ranked by (z descending, id ascending), -infinity left out:
//   top-k keeps the first k ranks; top-p, of those, the ranks whose preceding mass is below top_p of the top-k
//   mass; min-p, of those, w_v >= min_p.  The token is the smallest id whose kept mass through it exceeds
//   u * kept mass.  T = 0: the largest logit, lowest id.
//
// A token is decided by comparing sums with u times a sum, so sums have to be
// the same whatever the order of adding: weights are taken in 64 bits (a
// polynomial of 2^f on [-1/2, 1/2], off by 2^-50) and masses are integers in
// units of 2^-44 of the largest weight, exact and orderless (a row's sum stays
// below 2^62).
//
// The kept set of top-k and top-p is the ranks above some boundary.  The
// boundary is found on histograms of counts and masses over descending bins:
// first bins of 1/32 octave of weight, then, inside the bin that holds the
// boundary, ranges of the logits' order-preserving integer keys until a bin is
// a single key; ties there are cut by id.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/loopspec.h"

namespace ls {

typedef unsigned long long u64;

constexpr int kDThreads = 1024, kDWaves = kDThreads / 64;
constexpr int kDBins = 2048;
constexpr int kDMaxVocab = 1 << 18;
constexpr double kUnit = 17592186044416.0;            // 2^44

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

template <int DT>
__device__ __forceinline__ float logit(const void* p, int64_t i) {
    if (DT == LOOPSPEC_F32) return ((const float*)p)[i];
    const uint16_t b = ((const uint16_t*)p)[i];
    if (DT == LOOPSPEC_BF16) return __uint_as_float((uint32_t)b << 16);
    return (float)__builtin_bit_cast(_Float16, b);
}
// order-preserving integer of a float that is no NaN; both zeros alike
__device__ __forceinline__ uint32_t order_key(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
// 2^y, y <= 0: 2^n 2^f with the polynomial of 2^f that interpolates at the
// Chebyshev points of [-1/2, 1/2] and is 1 at 0
__device__ __forceinline__ double weight(double y) {
    if (y < -1000.0) return 0.0;
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
    return ldexp(fma(p, f, 1.0), (int)n);
}

struct DrawLds {
    u64 mass[kDBins];
    unsigned count[kDBins];
    u64 wsum[kDWaves];
    unsigned wcnt[kDWaves];
    float wmax[kDWaves];
    unsigned pick, cnt, lo, hi;
    u64 above_mass, bin_mass;
    unsigned above_cnt;
    int bad, token;
};

// the row as its workgroup sees it
template <int DT>
struct Row1 {
    const void* z;
    int64_t base;
    int V, seg;               // wave w holds ids [w * seg, (w + 1) * seg)
    float top;                // the largest logit
    double scale;             // log2(e) / T
    DrawLds& l;

    __device__ __forceinline__ float at(int id) const { return logit<DT>(z, base + id); }
    __device__ __forceinline__ double w(float x) const { return weight(((double)x - (double)top) * scale); }
    __device__ __forceinline__ u64 mass(float x) const { return (u64)rint(w(x) * kUnit); }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        const int w0 = threadIdx.x >> 6, lane = threadIdx.x & 63;
        for (int i = w0 * seg + lane; i < min((w0 + 1) * seg, V); i += 64) f(i, at(i));
    }
    __device__ __forceinline__ int bin(float x) const {
        const float d = (top - x) * (float)(32.0 * scale);
        return d < (float)(kDBins - 1) ? (int)d : kDBins - 1;         // infinity and NaN (0 * inf): the last bin
    }
};

__device__ __forceinline__ u64 wave_sum(u64 v) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ unsigned wave_sum(unsigned v) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
    return v;
}

// The bin that holds the boundary, from the histogram: the first one through
// which the count reaches `need` (by count) or the mass reaches `goal`; the
// last occupied one when none does.  Leaves it in l.pick with what lies above.
__device__ void pick_bin(DrawLds& l, bool by_count, unsigned need, double goal, u64 above_m, unsigned above_c) {
    const int tid = threadIdx.x;
    if (tid < 64) {
        constexpr int PER = kDBins / 64;
        u64 m = 0;
        unsigned c = 0;
        for (int i = 0; i < PER; ++i) m += l.mass[tid * PER + i], c += l.count[tid * PER + i];
        u64 sm = m;
        unsigned sc = c;
        for (int o = 1; o < 64; o *= 2) {
            const u64 v = __shfl_up(sm, o);
            const unsigned x = __shfl_up(sc, o);
            if (tid >= o) sm += v, sc += x;
        }
        sm += above_m - m;                     // above this lane's bins
        sc += above_c - c;
        int at = -1, last = -1;
        u64 am = 0, lm = 0;
        unsigned ac = 0, lc = 0;
        for (int i = 0; i < PER; ++i) {
            const int b = tid * PER + i;
            const unsigned n = l.count[b];
            if (!n) continue;
            last = b, lm = sm, lc = sc;
            const bool reach = by_count ? sc + n >= need : (double)(sm + l.mass[b]) >= goal;
            if (at < 0 && reach) at = b, am = sm, ac = sc;
            sm += l.mass[b];
            sc += n;
        }
        unsigned long long hit = __ballot(at >= 0);
        if (!hit) {
            hit = __ballot(last >= 0);
            at = last, am = lm, ac = lc;
            hit = 1ull << (63 - __clzll(hit));
        }
        if (tid == __ffsll(hit) - 1) {
            l.pick = at;
            l.above_mass = am;
            l.above_cnt = ac;
            l.cnt = l.count[at];
            l.bin_mass = l.mass[at];
        }
    }
    __syncthreads();
}

// Boundary of one filter: keys above `key` are kept, and of those equal to it
// the first `ties` by id; `mass` is what is kept, `all` the number of equal keys.
struct Bound {
    uint32_t key;
    unsigned ties, all;
    u64 mass;
};

template <int DT>
__device__ Bound boundary(const Row1<DT>& r, bool by_count, unsigned need, double goal) {
    DrawLds& l = r.l;
    const int tid = threadIdx.x;
    bool first = true;
    int picked = 0;
    uint32_t lo = 0, hi = 0xFFFFFFFFu;         // keys of the range that holds the boundary
    u64 above_m = 0;
    unsigned above_c = 0;
    for (;;) {
        // the range's own ends: a bin of the first round, or what is left of a range of keys
        if (!first) {
            __syncthreads();
            if (tid == 0) l.lo = 0xFFFFFFFFu, l.hi = 0;
            __syncthreads();
            uint32_t a = 0xFFFFFFFFu, b = 0;
            r.each([&](int, float x) {
                const uint32_t k = order_key(x);
                if (x != -INFINITY && k >= lo && k <= hi && r.bin(x) == picked) a = min(a, k), b = max(b, k);
            });
            atomicMin(&l.lo, a);
            atomicMax(&l.hi, b);
            __syncthreads();
            lo = l.lo, hi = l.hi;
        }
        __syncthreads();
        for (int i = tid; i < kDBins; i += kDThreads) l.mass[i] = 0, l.count[i] = 0;
        __syncthreads();
        int shift = 0;
        while (!first && ((hi - lo) >> shift) >= (uint32_t)kDBins) ++shift;
        r.each([&](int, float x) {
            if (x == -INFINITY) return;
            int b = r.bin(x);
            if (!first) {
                const uint32_t k = order_key(x);
                if (b != picked || k < lo || k > hi) return;
                b = (int)((hi - k) >> shift);
            }
            atomicAdd(&l.count[b], 1u);
            atomicAdd(&l.mass[b], r.mass(x));
        });
        __syncthreads();
        pick_bin(l, by_count, need, goal, above_m, above_c);
        above_m = l.above_mass, above_c = l.above_cnt;
        if (first) {
            picked = l.pick;
            first = false;
            continue;
        }
        const uint32_t h = hi - (l.pick << shift);
        if (shift == 0) {
            const unsigned n = l.cnt;
            const u64 one = l.bin_mass / n;     // equal keys have equal masses
            unsigned e;
            if (by_count) {
                e = min(n, need - above_c);
            } else {
                e = n;
                if (one) {
                    const double want = (goal - (double)above_m) / (double)one;
                    e = want < (double)n ? (unsigned)max(want, 0.0) : n;
                    while (e > 0 && (double)(above_m + (u64)(e - 1) * one) >= goal) --e;
                    while (e < n && (double)(above_m + (u64)e * one) < goal) ++e;
                }
            }
            return Bound{h, e, n, above_m + (u64)e * one};
        }
        lo = max(lo, h - ((1u << shift) - 1));
        hi = h;
    }
}

template <int DT>
__global__ void __launch_bounds__(kDThreads) k_draw(DrawArgs a) {
    __shared__ DrawLds l;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const float T = a.temperature ? a.temperature[row] : a.temperature1;
    const float top_p = a.top_p ? a.top_p[row] : a.top_p1, min_p = a.min_p ? a.min_p[row] : a.min_p1;
    const int top_k = a.top_k ? a.top_k[row] : a.top_k1;
    const double u = a.u[row];
    bool ok = T >= 0.f && T < INFINITY && top_p > 0.f && top_p <= 1.f && min_p >= 0.f && min_p <= 1.f && u >= 0.0 && u < 1.0;
    Row1<DT> r{a.z, row * a.stride, a.V, ((a.V + kDWaves - 1) / kDWaves + 63) / 64 * 64, 0.f, 0.0, l};

    // the largest logit
    float top = -INFINITY;
    bool bad = false;
    r.each([&](int, float x) {
        bad |= !(x < INFINITY);
        top = fmaxf(top, x);
    });
    for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
    if (tid == 0) l.bad = 0, l.token = 0x7FFFFFFF;
    if (lane == 0) l.wmax[wv] = top;
    __syncthreads();
    if (bad) l.bad = 1;
    for (int i = 0; i < kDWaves; ++i) top = fmaxf(top, l.wmax[i]);
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
        r.each([&](int i, float x) {
            if (x == top) best = min(best, i);
        });
        atomicMin(&l.token, best);
        __syncthreads();
        if (tid == 0) {
            a.token[row] = l.token;
            if (a.prob) a.prob[row] = 1.f;
            if (a.kept) a.kept[row] = 1;
        }
        return;
    }
    r.top = top;
    r.scale = 1.4426950408889634074 / (double)T;

    // what is kept: keys above bd.key, ties below the id `cut`, weights from min_p on
    Bound bd{0, 0, 0, 0};
    int cut = 0x7FFFFFFF;
    if (top_k > 0 && top_k < a.V) bd = boundary(r, true, (unsigned)top_k, 0.0);
    if (top_p < 1.f) {
        u64 all = bd.mass;
        if (!all) {
            r.each([&](int, float x) { all += r.mass(x); });
            all = wave_sum(all);
            __syncthreads();
            if (lane == 0) l.wsum[wv] = all;
            __syncthreads();
            all = 0;
            for (int i = 0; i < kDWaves; ++i) all += l.wsum[i];
        }
        bd = boundary(r, false, 0u, (double)top_p * (double)all);
    }
    if (bd.ties < bd.all) {
        // the id of the first tie that is left out
        unsigned n = 0;
        r.each([&](int, float x) { n += order_key(x) == bd.key; });
        n = wave_sum(n);
        __syncthreads();
        if (lane == 0) l.wcnt[wv] = n;
        __syncthreads();
        unsigned before = 0;
        for (int i = 0; i < wv; ++i) before += l.wcnt[i];
        if (before <= bd.ties && bd.ties < before + n) {
            for (int i = wv * r.seg;; i += 64) {
                const bool tie = i + lane < a.V && order_key(r.at(i + lane)) == bd.key;
                const u64 m = __ballot(tie);
                const unsigned c = __popcll(m), mine = before + __popcll(m & ((1ull << lane) - 1));
                if (tie && mine == bd.ties) l.token = i + lane;
                before += c;
                if (before > bd.ties) break;
            }
        }
        __syncthreads();
        cut = l.token;
        __syncthreads();
    }
    // kept mass and count per wave
    u64 sum = 0;
    unsigned cnt = 0;
    auto mass = [&](int i, float x, unsigned* c) -> u64 {
        const uint32_t k = order_key(x);
        if (x == -INFINITY || k < bd.key || (k == bd.key && i >= cut)) return 0;
        const double w = r.w(x);
        if (w < (double)min_p) return 0;
        ++*c;
        return (u64)rint(w * kUnit);
    };
    r.each([&](int i, float x) { sum += mass(i, x, &cnt); });
    sum = wave_sum(sum);
    cnt = wave_sum(cnt);
    if (lane == 0) l.wsum[wv] = sum, l.wcnt[wv] = cnt;
    __syncthreads();
    u64 all = 0, before = 0;
    unsigned kept = 0;
    for (int i = 0; i < kDWaves; ++i) {
        if (i < wv) before += l.wsum[i];
        all += l.wsum[i];
        kept += l.wcnt[i];
    }
    // mass through an id > u * all, in integers: > floor(u * all), which rounding must not raise to all
    const u64 goal = min((u64)(u * (double)all), all - 1);
    if (before <= goal && goal < before + sum) {
        // the token is this wave's
        for (int i = wv * r.seg;; i += 64) {
            unsigned c = 0;
            const u64 m = i + lane < a.V ? mass(i + lane, r.at(i + lane), &c) : 0;
            u64 s = m;
            for (int o = 1; o < 64; o *= 2) {
                const u64 v = __shfl_up(s, o);
                if (lane >= o) s += v;
            }
            const unsigned long long hit = __ballot(before + s > goal);
            if (hit) {
                if (lane == __ffsll(hit) - 1) {
                    a.token[row] = i + lane;
                    if (a.prob) a.prob[row] = (float)((double)m / (double)all);
                    if (a.kept) a.kept[row] = (int)kept;
                }
                break;
            }
            before += __shfl(s, 63);
        }
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
    const void* f = cfg->dtype == LOOPSPEC_F32 ? (const void*)k_draw<LOOPSPEC_F32>
                    : cfg->dtype == LOOPSPEC_BF16 ? (const void*)k_draw<LOOPSPEC_BF16> : (const void*)k_draw<LOOPSPEC_F16>;
    void* args[] = {&a};
    return hipLaunchKernel(f, dim3(rows), dim3(kDThreads), args, 0, (hipStream_t)stream) == hipSuccess ? LOOPSPEC_OK : LOOPSPEC_EHIP;
}

}  // extern "C"
