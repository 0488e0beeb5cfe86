// Queries, keys and values of a step's tokens: per-head norm, rotation and the
// append to the paged cache, in one launch.
//
//   x <- g * x / sqrt(mean(x^2) + eps)                     (queries and keys, when gains are given)
//   (x_j, x_{j + rot/2}) <- (x_j cos a - x_{j + rot/2} sin a, x_{j + rot/2} cos a + x_j sin a),  a = position * freq_j
//
// A token's angles are computed once for all of its heads and pass through
// LDS.  The angle is reduced to a fraction of a turn in 64 bits (at position
// 2^20 an fp32 angle is off by 0.06), the sine and cosine of the fraction are
// fp32.  Everything between the load and the store is fp32; the result is
// rounded once.
//
// A head is worked on by D / 16 lanes of a group of L (a power of two): a lane
// holds elements [8c, 8c + 8) and their partners [rot/2 + 8c, ...) of the
// rotated part, or 16 consecutive elements behind it, and both come and go as
// 16-byte accesses.  The norm's sum crosses the group by DPP moves.
//
// Bound by memory: 3340 tokens of 55 query and 55 key and value heads of 96 (fp16,
// no norm, 212 MB) take 47 us, 4.5 TB/s; 16001 tokens of 28 query and 4 key and
// value heads of 128 (bf16, norms, half of a head rotated, 295 MB) take 60 us,
// 4.9 TB/s, which is what a large copy reaches.  One token takes 3 us, a launch
// and the loads that wait for each other (lengths, then pages).
#include "ls_paged.h"

#include <algorithm>

namespace ls {

struct RopeArgs {
    const uint16_t *q, *k, *v;
    uint16_t* out;
    int64_t qt, qh, kt, kh, vt, vh, ot, oh;   // strides in elements: token, head
    const double* freq;
    const float *qn, *kn;
    int H, rot;
    float eps;
};

constexpr int kRopeThreads = 256, kRopeTokens = 4;

// Workgroup (x, y): `per` tokens from x * per on; L threads to an item, which
// stays theirs for all of the tokens (so gains stay in registers): H query
// heads, G key heads, G value heads, cut into gridDim.y slices.  A wave finds
// the place of every fourth token and takes its sines; an item's data is on its
// way under that, the next token's under the work on one.
template <bool BF, int L>
__global__ void __launch_bounds__(kRopeThreads) k_rope_append(PagedCache c, PagedBatch b, RopeArgs a, int per) {
    __shared__ float cs[kRopeTokens][128];    // cosines, then sines at 64
    __shared__ int64_t to_k[kRopeTokens], to_v[kRopeTokens];        // where a token's keys and values go: kNowhere, kPadding
    constexpr int64_t kNowhere = -1, kPadding = -2;
    const int tid = threadIdx.x, D = c.D, half = a.rot >> 1;
    const int lane = tid % L, ch = a.rot >> 4;                      // rotated chunks per half
    const int lo = lane < ch ? 8 * lane : 16 * lane, hi = lane < ch ? half + 8 * lane : 16 * lane + 8;
    const int it = (blockIdx.y * kRopeThreads + tid) / L;
    const bool query = it < a.H, key = !query && it < a.H + c.G, on = 16 * lane < D && it < a.H + 2 * c.G;
    const int g = query ? it : key ? it - a.H : it - a.H - c.G;
    const uint16_t* const from = query ? a.q + g * a.qh : key ? a.k + g * a.kh : a.v + g * a.vh;
    const int64_t next = query ? a.qt : key ? a.kt : a.vt;
    uint16_t* const dst = query ? a.out + g * a.oh : key ? c.k + g * c.kh : c.v + g * c.vh;
    const float* const gain = query ? a.qn : key ? a.kn : nullptr;
    float gl[8], gh[8];
    if (gain && on)
#pragma unroll
        for (int i = 0; i < 8; ++i) gl[i] = gain[lo + i], gh[i] = gain[hi + i];
    const int t0 = blockIdx.x * per, n = min(per, b.T - t0);
    const uint16_t* src = from + t0 * next;
    u32x4 n0 = {0, 0, 0, 0}, n1 = {0, 0, 0, 0};
    if (on) n0 = *(const u32x4*)(src + lo), n1 = *(const u32x4*)(src + hi);
    for (int i = tid >> 6; i < n; i += kRopeThreads / 64) {
        const int j = tid & 63;
        int64_t place = -1, k = kPadding, v = 0;
        const int seq = paged_place(b, t0 + i, &place);
        if (seq >= 0 && place >= 0) {
            k = kNowhere;
            if (place >> 4 < (int64_t)b.width * c.unit) {
                const int at = (int)unit_div((unsigned)(place >> 4), c.magic);
                const int page = b.table[seq * b.table_stride + at];
                const int64_t row = place - at * c.unit * kPageUnit;
                if ((unsigned)page < (unsigned)c.n_pages) k = page * c.kp + row * c.ks, v = page * c.vp + row * c.vs;
            }
            if (j < half) {
                const double turns = (double)(b.prefix + place) * a.freq[j] * 0.15915494309189533577;
                float sn, cn;
                sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cn);
                cs[i][j] = cn;
                cs[i][64 + j] = sn;
            }
        }
        if (j == 0) to_k[i] = k, to_v[i] = v;
    }
    __syncthreads();
    for (int i = 0; i < n; ++i) {
        u32x4 u0 = n0, u1 = n1;
        src += next;
        if (on && i + 1 < n) n0 = *(const u32x4*)(src + lo), n1 = *(const u32x4*)(src + hi);
        const int64_t place = to_k[i];
        if (place == kPadding) continue;                            // the same for the whole workgroup
        if (query || key) {
            float x[8], y[8];
            unpack8<BF>(u0, x);
            unpack8<BF>(u1, y);
            if (gain) {
                float s = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) s = fmaf(x[j], x[j], fmaf(y[j], y[j], s));
                s = 1.0f / sqrtf(group_sum<L>(s) / (float)D + a.eps);
                if (on)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x[j] *= s * gl[j];
                        y[j] *= s * gh[j];
                    }
            }
            if (lane < ch)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float cn = cs[i][lo + j], sn = cs[i][64 + lo + j];
                    const float r = x[j] * cn - y[j] * sn;
                    y[j] = y[j] * cn + x[j] * sn;
                    x[j] = r;
                }
            u0 = pack8<BF>(x);
            u1 = pack8<BF>(y);
        }
        if (on && (query || place != kNowhere)) {
            uint16_t* const d = dst + (query ? (t0 + i) * a.ot : key ? place : to_v[i]);
            *(u32x4*)(d + lo) = u0;
            *(u32x4*)(d + hi) = u1;
        }
    }
}

int paged_args(const loopspec_paged_cache* cache, const loopspec_paged_batch* batch, PagedCache* c, PagedBatch* b) {
    if (!cache || !batch) return LOOPSPEC_EINVAL;
    const int D = cache->head_dim, G = cache->n_kv_heads, ps = cache->page_size;
    if (cache->dtype != LOOPSPEC_F16 && cache->dtype != LOOPSPEC_BF16) return LOOPSPEC_EINVAL;
    if (D != 16 && D != 32 && D != 64 && D != 96 && D != 128) return LOOPSPEC_EINVAL;
    if (G < 1 || G > (1 << 16) || cache->n_pages < 1) return LOOPSPEC_EINVAL;
    if (ps < kPageUnit || ps > kPageMax || ps % kPageUnit) return LOOPSPEC_EINVAL;
    const void* p[2] = {cache->k_dev, cache->v_dev};
    const int64_t st[2][3] = {{cache->k_page, cache->k_head, cache->k_pos}, {cache->v_page, cache->v_head, cache->v_pos}};
    for (int i = 0; i < 2; ++i) {
        if (!p[i] || ((uintptr_t)p[i] & 15)) return LOOPSPEC_EINVAL;
        for (int64_t s : st[i])
            if (s < 0 || s % 8) return LOOPSPEC_EINVAL;
        if (st[i][2] < D || st[i][2] > kStrideMax) return LOOPSPEC_EINVAL;
        if ((G > 1 && st[i][1] < D) || (cache->n_pages > 1 && st[i][0] < D)) return LOOPSPEC_EINVAL;
    }
    if (batch->n_seqs < 0 || batch->n_tokens < 0 || batch->prefix_len < 0 || batch->table_width < 0) return LOOPSPEC_EINVAL;
    if (batch->n_tokens > kTokensMax || batch->prefix_len > kPlacesMax || (int64_t)batch->table_width * ps > kPlacesMax) return LOOPSPEC_EINVAL;
    if (batch->n_seqs > 0 && !batch->seq_len_dev) return LOOPSPEC_EINVAL;
    if (batch->n_seqs > 0 && batch->table_width > 0 && !batch->table_dev) return LOOPSPEC_EINVAL;
    if (batch->n_seqs > 1 && batch->table_stride < batch->table_width) return LOOPSPEC_EINVAL;
    const int unit = ps / kPageUnit;
    *c = PagedCache{(uint16_t*)cache->k_dev, (uint16_t*)cache->v_dev, cache->k_page, cache->k_head, cache->k_pos,
                    cache->v_page, cache->v_head, cache->v_pos, cache->n_pages, G, D, unit,
                    unit > 1 ? (unsigned)(((1ull << 32) + unit - 1) / unit) : 0u};
    *b = PagedBatch{batch->q_start_dev, batch->seq_len_dev, batch->table_dev, batch->table_stride, batch->prefix_table_dev,
                    batch->n_seqs, batch->n_tokens, batch->table_width, batch->prefix_len};
    return LOOPSPEC_OK;
}

// an 8-bit cache's own conditions, beside paged_args'
int scale_args(const loopspec_paged_cache* cache, const loopspec_page_scales* scales, PageScales* s) {
    if (!cache || !scales) return LOOPSPEC_EINVAL;
    for (int64_t st : {cache->k_page, cache->k_head, cache->k_pos, cache->v_page, cache->v_head, cache->v_pos})
        if (st % 16) return LOOPSPEC_EINVAL;
    const int units = cache->page_size / kPageUnit;
    if (!scales->k_dev || !scales->v_dev) return LOOPSPEC_EINVAL;
    for (int64_t st : {scales->k_head, scales->v_head})
        if (st < 0 || (cache->n_kv_heads > 1 && st < units)) return LOOPSPEC_EINVAL;
    for (int64_t st : {scales->k_page, scales->v_page})
        if (st < 0 || (cache->n_pages > 1 && st < units)) return LOOPSPEC_EINVAL;
    *s = PageScales{(uint8_t*)scales->k_dev, (uint8_t*)scales->v_dev, scales->k_page, scales->k_head, scales->v_page, scales->v_head};
    return LOOPSPEC_OK;
}

// rows of 16-byte chunks: element strides and the address keep that alignment
bool rows_ok(const void* p, int64_t token, int64_t head) {
    return p && !((uintptr_t)p & 15) && token >= 0 && head >= 0 && token % 8 == 0 && head % 8 == 0;
}

int rope_args(const PagedCache& c, const PagedBatch& b, const loopspec_rope_args* args) {
    if (args->n_heads < 1 || args->n_heads > (1 << 16) || args->n_heads % c.G) return LOOPSPEC_EINVAL;
    if (args->rot_dim < 0 || args->rot_dim > c.D || args->rot_dim % 16 || (args->rot_dim && !args->freq_dev))
        return LOOPSPEC_EINVAL;
    if (!(args->eps >= 0.f)) return LOOPSPEC_EINVAL;
    if (!b.B || !b.T) return LOOPSPEC_OK;     // (empty tensors have no address)
    if (!rows_ok(args->q_dev, args->q_token, args->q_head) || !rows_ok(args->k_dev, args->k_token, args->k_head) ||
        !rows_ok(args->v_dev, args->v_token, args->v_head) || !rows_ok(args->q_out_dev, args->out_token, args->out_head))
        return LOOPSPEC_EINVAL;
    if ((args->n_heads > 1 && args->out_head < c.D) || (b.T > 1 && args->out_token < c.D)) return LOOPSPEC_EINVAL;
    return LOOPSPEC_OK;
}

namespace {

template <bool BF>
const void* rope_kernel(int L) {
    switch (L) {
        case 1: return (const void*)k_rope_append<BF, 1>;
        case 2: return (const void*)k_rope_append<BF, 2>;
        case 4: return (const void*)k_rope_append<BF, 4>;
        default: return (const void*)k_rope_append<BF, 8>;
    }
}

}  // namespace
}  // namespace ls

extern "C" int loopspec_rope_append(const loopspec_paged_cache* cache, const loopspec_paged_batch* batch,
                                    const loopspec_rope_args* args, void* stream) {
    using namespace ls;
    PagedCache c;
    PagedBatch b;
    if (!args) return LOOPSPEC_EINVAL;
    int rc = paged_args(cache, batch, &c, &b);
    if (rc || (rc = rope_args(c, b, args))) return rc;
    if (!b.B || !b.T) return LOOPSPEC_OK;     // (empty tensors have no address)
    RopeArgs a{(const uint16_t*)args->q_dev, (const uint16_t*)args->k_dev, (const uint16_t*)args->v_dev,
               (uint16_t*)args->q_out_dev, args->q_token, args->q_head, args->k_token, args->k_head, args->v_token,
               args->v_head, args->out_token, args->out_head, args->freq_dev, args->q_norm_dev, args->k_norm_dev,
               args->n_heads, args->rot_dim, args->eps};
    int L = 1;
    while (L * 16 < c.D) L *= 2;
    const int64_t lanes = (int64_t)(a.H + 2 * c.G) * L;
    const int y = (int)((lanes + kRopeThreads - 1) / kRopeThreads);
    // a token a workgroup while there are few; several, with gains kept and loads running ahead, once 4096
    // workgroups stand (one each: 50 and 76 us instead of 47 and 60 at the sizes above; 8 or 16: 1 to 3 % more)
    int per = (int)std::min<int64_t>(kRopeTokens, std::max<int64_t>(1, (int64_t)b.T * y / 4096));
    const int x = (b.T + per - 1) / per;
    void* kargs[] = {&c, &b, &a, &per};
    const void* f = cache->dtype == LOOPSPEC_BF16 ? rope_kernel<true>(L) : rope_kernel<false>(L);
    return hipLaunchKernel(f, dim3(x, y), dim3(kRopeThreads), kargs, 0, (hipStream_t)stream) == hipSuccess ? LOOPSPEC_OK
                                                                                                          : LOOPSPEC_EHIP;
}
