// The append to a cache held in 8 bits: per-head norm, rotation and codes with
// one scale for 16 positions of a head, in one launch.
//
//   e = max(-64, min{e : max |x| <= 448 * 2^e}) over the block's new elements, and at least the scale of positions
//   that the block keeps;  code = e4m3(x * 2^-e), to nearest even, straight from fp32
//
// 448 is e4m3's largest value: with max |x| = m * 2^t, 1 <= m < 2, e is t - 8 or,
// for m > 1.75, t - 7.  A power of two costs e4m3 no bits, and codes of a block
// whose scale grows later are rounded again only where they become subnormal.
//
// A block's scale follows all of its new tokens, so one workgroup takes a run of
// tokens of one sequence inside one block of 16 positions: the workgroup whose
// tokens hold the run's first.  A wave takes a head of the run: L lanes hold a
// token's head (8 elements and their partners of the rotation each), so that the
// maximum crosses the wave by shuffles and codes leave as 8-byte stores.  Runs of
// a single token put several heads side by side instead.
//
// Bound by memory and by the angles and codes beside it: 16001 tokens of 28 query
// and 4 key and value heads of 128 (bf16, norms, half of a head rotated, 278 MB)
// take 62 us, 4.5 TB/s, of which a large copy's rate is 59; 5 prompts of up to 900
// tokens of 55 heads of 96 (fp16, 176 MB) 51 us, 3.4 TB/s, a head's loads behind the
// angles, the next head's behind its codes, and the angles anew in each slice.  One
// token takes 5 us, a launch and the loads that wait for each other.
#include "ls_paged.h"

#include <algorithm>

namespace ls {

namespace {

constexpr int kT = 512, kW = kT / 64;
constexpr int kLeast = -64;

struct Rope8 {
    const uint16_t *q, *k, *v;
    uint16_t* out;
    int64_t qt, qh, kt, kh, vt, vh, ot, oh;   // strides in elements: token, head
    const double* freq;
    const float *qn, *kn;
    int H, rot;
    float eps;
};

// the smallest e from kLeast on with a <= 448 * 2^e (a finite, >= 0)
__device__ __forceinline__ int exponent8(float a) {
    int t;
    const float m = frexpf(a, &t);            // a = m * 2^t, 0.5 <= m < 1 (0: 0)
    return a > 0.f ? max(t - 9 + (m > 0.875f ? 1 : 0), kLeast) : kLeast;
}

// four codes (the conversion makes infinities NaN; nothing finite is above 448 here)
__device__ __forceinline__ uint32_t encode4(const float* x, float inv) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, lo, true);
}
__device__ __forceinline__ uint32_t rescale4(uint32_t c, float f) {
    const float x[4] = {__builtin_amdgcn_cvt_f32_fp8(c, 0), __builtin_amdgcn_cvt_f32_fp8(c, 1), __builtin_amdgcn_cvt_f32_fp8(c, 2),
                        __builtin_amdgcn_cvt_f32_fp8(c, 3)};
    return encode4(x, f);
}

// Sine and cosine of a fraction of a turn, |x| <= 1/2: Taylor's series on an eighth of a turn to either side, in 64 bits
// (their next terms are below 2^-36 of the result), each rounded once.  fp32's functions are off by up to two roundings,
// and a key's code shows on which side of a border a value lies (against 64 bits its error was twice that of exactly rounded
// angles).  18 products; 5 prompts of 55 heads take 52 us, with fp32's functions 53.
__device__ __forceinline__ void sine_cosine(double x, float* sine, float* cosine) {
    const int quarter = (int)rint(4.0 * x);
    const double a = (x - 0.25 * quarter) * 6.283185307179586477, z = a * a;
    const double s = a * fma(z, fma(z, fma(z, fma(z, fma(z, -1.0 / 39916800, 1.0 / 362880), -1.0 / 5040), 1.0 / 120), -1.0 / 6), 1.0);
    const double c = fma(z, fma(z, fma(z, fma(z, fma(z, fma(z, 1.0 / 479001600, -1.0 / 3628800), 1.0 / 40320), -1.0 / 720), 1.0 / 24), -0.5), 1.0);
    const float fs = (float)s, fc = (float)c;
    const bool odd = quarter & 1;             // a quarter turn on: the sine is the cosine, the cosine the sine's negative
    const float p = odd ? fc : fs, q = odd ? -fs : fc;
    *sine = quarter & 2 ? -p : p;
    *cosine = quarter & 2 ? -q : q;
}

// A run: token t0 + i begins it at `place` of sequence `seq`, n tokens long.
struct Run {
    int n, keep;                              // tokens; positions that its block keeps below it
    int64_t place, k, v, ks, vs;              // own position; the block's first position and its scale (-1: no page)
};

// One wave, one item of it: token slots of L lanes.  ONE: runs of one token, 64 / L heads side by side.
template <bool BF, int L, bool ONE>
__device__ __forceinline__ void heads(const PagedCache& c, const PageScales& sc, const Rope8& a, const Run& r, int t0,
                                      const float (&cs)[16][128], int first, int step) {
    constexpr int SLOTS = 64 / L, TS = ONE ? 1 : SLOTS < 16 ? SLOTS : 16, HW = SLOTS / TS, NP = ONE ? 1 : 16 / TS;
    const int wl = threadIdx.x & 63, lane = wl % L, ts = wl / L % TS, hs = wl / L / TS;
    const int D = c.D, half = a.rot >> 1, ch = a.rot >> 4;
    const int lo = lane < ch ? 8 * lane : 16 * lane, hi = lane < ch ? half + 8 * lane : 16 * lane + 8;
    const int items = a.H + 2 * c.G;
    for (int it0 = first * HW; it0 < items; it0 += step * HW) {
        const int it = it0 + hs;
        const bool query = it < a.H, key = !query && it < a.H + c.G, on = 16 * lane < D && it < items;
        const int g = query ? it : key ? it - a.H : it - a.H - c.G;
        const uint16_t* const from = query ? a.q + g * a.qh : key ? a.k + g * a.kh : a.v + g * a.vh;
        const int64_t next = query ? a.qt : key ? a.kt : a.vt;
        const float* const gain = query ? a.qn : key ? a.kn : nullptr;
        float x[NP][8], y[NP][8];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            u32x4 u0 = {0, 0, 0, 0}, u1 = {0, 0, 0, 0};
            const uint16_t* const src = from + (int64_t)(t0 + ts + p * TS) * next;
            if (on && ts + p * TS < r.n) u0 = *(const u32x4*)(src + lo), u1 = *(const u32x4*)(src + hi);
            unpack8<BF>(u0, x[p]);
            unpack8<BF>(u1, y[p]);
        }
        float amax = 0.f;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            if (query || key) {
                if (gain) {
                    float s = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) s = fmaf(x[p][j], x[p][j], fmaf(y[p][j], y[p][j], s));
                    s = 1.0f / sqrtf(group_sum<L>(s) / (float)D + a.eps);
                    if (on)
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            x[p][j] *= s * gain[lo + j];
                            y[p][j] *= s * gain[hi + j];
                        }
                }
                if (lane < ch && ts + p * TS < r.n)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float cn = cs[ts + p * TS][lo + j], sn = cs[ts + p * TS][64 + lo + j];
                        const float t = x[p][j] * cn - y[p][j] * sn;
                        y[p][j] = y[p][j] * cn + x[p][j] * sn;
                        x[p][j] = t;
                    }
            }
            if (query) {
                if (on && ts + p * TS < r.n) {
                    uint16_t* const d = a.out + g * a.oh + (int64_t)(t0 + ts + p * TS) * a.ot;
                    *(u32x4*)(d + lo) = pack8<BF>(x[p]);
                    *(u32x4*)(d + hi) = pack8<BF>(y[p]);
                }
            } else if (ts + p * TS < r.n) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float u = fabsf(x[p][j]), w = fabsf(y[p][j]);
                    amax = fmaxf(amax, fmaxf(u < INFINITY ? u : 0.f, w < INFINITY ? w : 0.f));
                }
            }
        }
        if (r.k < 0) continue;                // the block's page is none of the cache's
        // (all lanes take part: queries bring 0)
#pragma unroll
        for (int o = 1; o < L * TS; o *= 2) amax = fmaxf(amax, __shfl_xor(amax, o));
        if (query || !on) continue;
        uint8_t* const codes = (uint8_t*)(key ? (void*)c.k : (void*)c.v) + (key ? r.k + g * c.kh : r.v + g * c.vh);
        uint8_t* const scale = key ? sc.k + r.ks + g * sc.kh : sc.v + r.vs + g * sc.vh;
        const int64_t row = key ? c.ks : c.vs;
        int e = exponent8(amax);
        if (r.keep) {
            const int old = (int)*scale - 127;
            if (e > old) {
                const float f = ldexpf(1.f, old - e);
                for (int i = ts; i < r.keep; i += TS) {
                    uint8_t* const d = codes + i * row;
                    u32x2 u = *(const u32x2*)(d + lo), w = *(const u32x2*)(d + hi);
                    u = u32x2{rescale4(u[0], f), rescale4(u[1], f)};
                    w = u32x2{rescale4(w[0], f), rescale4(w[1], f)};
                    *(u32x2*)(d + lo) = u;
                    *(u32x2*)(d + hi) = w;
                }
            }
            e = max(e, old);
        }
        const float inv = ldexpf(1.f, -e);
#pragma unroll
        for (int p = 0; p < NP; ++p)
            if (ts + p * TS < r.n) {
                uint8_t* const d = codes + (r.keep + ts + p * TS) * row;
                *(u32x2*)(d + lo) = u32x2{encode4(x[p], inv), encode4(x[p] + 4, inv)};
                *(u32x2*)(d + hi) = u32x2{encode4(y[p], inv), encode4(y[p] + 4, inv)};
            }
        // after the lanes of this wave that read the old scale: they are in lockstep, and the load has been waited for
        if (ts == 0 && lane == 0) *scale = (uint8_t)(e + 127);
    }
}

// Workgroup x * slices + y: the runs that begin in the `per` tokens from x * per on; slice y of the heads (the slices of a
// run together, since heads share lines).
template <bool BF, int L>
__global__ void __launch_bounds__(kT) k_append8(PagedCache c, PageScales sc, PagedBatch b, Rope8 a, int per, int slices) {
    __shared__ float cs[16][128];             // cosines, then sines at 64
    __shared__ Run runs[16];
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), half = a.rot >> 1;
    const int bx = blockIdx.x / slices, by = blockIdx.x % slices, t0 = bx * per, n = min(per, b.T - t0);
    for (int i = w; i < n; i += kW) {
        const int t = t0 + i;
        int64_t place = -1;
        const int seq = paged_place(b, t, &place);
        Run r{0, 0, place, -1, -1, -1, -1};
        if (seq >= 0 && place >= 0) {
            const int start = b.q_start ? max(b.q_start[seq], 0) : t, end = min(b.q_start ? b.q_start[seq + 1] : t + 1, b.T);
            r.keep = (int)(place & 15);
            if (t == start || r.keep == 0) {
                r.n = min(16 - r.keep, end - t);
                if (place >> 4 < (int64_t)b.width * c.unit) {
                    const int blk = (int)(place >> 4), at = (int)unit_div((unsigned)blk, c.magic);
                    const int page = b.table[seq * b.table_stride + at], u = blk - at * c.unit;
                    if ((unsigned)page < (unsigned)c.n_pages) {
                        r.k = page * c.kp + u * kPageUnit * c.ks;
                        r.v = page * c.vp + u * kPageUnit * c.vs;
                        r.ks = page * sc.kp + u;
                        r.vs = page * sc.vp + u;
                    }
                }
            }
        }
        if ((tid & 63) == 0) runs[i] = r;
    }
    __syncthreads();
    for (int i = 0; i < n; ++i) {
        const Run r = runs[i];
        if (!r.n) continue;                   // the same for the whole workgroup
        for (int j = tid; j < r.n * half; j += kT) {
            const int t = j / half, f = j - t * half;
            const double turns = (double)(b.prefix + r.place + t) * a.freq[f] * 0.15915494309189533577;
            const double part = turns - rint(turns);
            sine_cosine(part, &cs[t][64 + f], &cs[t][f]);
        }
        __syncthreads();
        const int first = by * kW + w, step = slices * kW;
        if (r.n == 1)
            heads<BF, L, true>(c, sc, a, r, t0 + i, cs, first, step);
        else
            heads<BF, L, false>(c, sc, a, r, t0 + i, cs, first, step);
        __syncthreads();
    }
}

template <bool BF>
const void* append8_kernel(int L) {
    switch (L) {
        case 1: return (const void*)k_append8<BF, 1>;
        case 2: return (const void*)k_append8<BF, 2>;
        case 4: return (const void*)k_append8<BF, 4>;
        default: return (const void*)k_append8<BF, 8>;
    }
}

}  // namespace
}  // namespace ls

extern "C" int loopspec_rope_append_quantized(const loopspec_paged_cache* cache, const loopspec_page_scales* scales,
                                              const loopspec_paged_batch* batch, const loopspec_rope_args* args, void* stream) {
    using namespace ls;
    PagedCache c;
    PagedBatch b;
    PageScales s;
    if (!args) return LOOPSPEC_EINVAL;
    int rc = paged_args(cache, batch, &c, &b);
    if (rc || (rc = scale_args(cache, scales, &s))) return rc;
    if ((rc = rope_args(c, b, args))) return rc;
    if (!b.B || !b.T) return LOOPSPEC_OK;
    Rope8 a{(const uint16_t*)args->q_dev, (const uint16_t*)args->k_dev, (const uint16_t*)args->v_dev,
            (uint16_t*)args->q_out_dev, args->q_token, args->q_head, args->k_token, args->k_head, args->v_token,
            args->v_head, args->out_token, args->out_head, args->freq_dev, args->q_norm_dev, args->k_norm_dev,
            args->n_heads, args->rot_dim, args->eps};
    int L = 1;
    while (L * 16 < c.D) L *= 2;
    const int items = a.H + 2 * c.G;
    int per = b.T > 1 << 22 || (b.q_start && b.T >= 8ll * b.B) ? 16 : 1;    // (a grid holds 2^32 threads)
    const int x = (b.T + per - 1) / per;
    // Slices of the heads, each of which takes the run's angles again: 1001 runs of 36 heads 60.6 us in one, 67.0 in two;
    // 214 runs of 165 heads 57.3 in nine, 52.4 in seven, 54.2 in six, 53.2 in five, 65.2 in two: from five to seven is
    // noise, and no other shapes were measured.  Workgroups of 256 threads,
    // whose share of the angles is twice as long, took 61.8 and 54.0 where these took 60.6 and 53, of 1024 67.0 and 58.4.
    const int most = per > 1 ? (items + kW - 1) / kW : (items * L + 64 * kW - 1) / (64 * kW);
    int slices = std::max(1, std::min(most, 1500 / x));
    void* kargs[] = {&c, &s, &b, &a, &per, &slices};
    const void* f = cache->dtype == LOOPSPEC_BF16 ? append8_kernel<true>(L) : append8_kernel<false>(L);
    return hipLaunchKernel(f, dim3(x * slices), dim3(kT), kargs, 0, (hipStream_t)stream) == hipSuccess ? LOOPSPEC_OK : LOOPSPEC_EHIP;
}
