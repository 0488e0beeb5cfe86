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
#include "ls_paged.h"

namespace ls {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct RopeArgs {
    const uint16_t *q, *k, *v;
    uint16_t* out;
    int64_t qt, qh, kt, kh, vt, vh, ot, oh;   // strides in elements: token, head
    const double* freq;
    const float *qn, *kn;
    int H, rot;
    float eps;
};

template <bool BF>
__device__ __forceinline__ void unpack8(const u32x4& u, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = u[i];
        f[2 * i] = BF ? __uint_as_float(w << 16) : h2f((uint16_t)w);
        f[2 * i + 1] = BF ? __uint_as_float(w & 0xFFFF0000u) : h2f((uint16_t)(w >> 16));
    }
}
template <bool BF>
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF)
            u[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)f[2 * i], (__bf16)f[2 * i + 1]});
        else
            u[i] = pack_h2(f[2 * i], f[2 * i + 1]);
    }
    return u;
}

constexpr int kRopeThreads = 256;

// Workgroup (x, y): tokens x, x + gridDim.x, ...; of each token the heads that
// fall to slice y of gridDim.y.  Items of a token: H query heads, G key heads,
// G value heads.
template <bool BF, int L>
__global__ void __launch_bounds__(kRopeThreads) k_rope_append(PagedCache c, PagedBatch b, RopeArgs a) {
    __shared__ float cs[2][128];              // cosines, then sines at 64; one buffer per token parity
    const int tid = threadIdx.x, D = c.D, half = a.rot >> 1;
    const int lane = tid % L, ch = a.rot >> 4;                      // rotated chunks per half
    const int lo = lane < ch ? 8 * lane : 16 * lane, hi = lane < ch ? half + 8 * lane : 16 * lane + 8;
    const bool on = 16 * lane < D;
    const int items = a.H + 2 * c.G, first = (blockIdx.y * kRopeThreads + tid) / L, step = gridDim.y * (kRopeThreads / L);
    int flip = 0;
    for (int t = blockIdx.x; t < b.T; t += gridDim.x) {
        int64_t place = -1;
        const int seq = paged_place(b, t, &place);
        if (seq < 0 || place < 0) continue;                         // padding; the same for the whole workgroup
        if (tid < half) {
            const double turns = (double)(b.prefix + place) * a.freq[tid] * 0.15915494309189533577;
            float sn, cn;
            sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cn);
            cs[flip][tid] = cn;
            cs[flip][64 + tid] = sn;
        }
        // where the token's key and value go: nowhere when its page is not one of the cache's
        const int64_t blk = place >> 4;
        const int64_t pg = blk / c.unit;
        int64_t row = -1, page = -1;
        if (pg < b.width) {
            page = b.table[seq * b.table_stride + pg];
            if ((uint64_t)page < (uint64_t)c.n_pages) row = place - pg * c.unit * kPageUnit;
        }
        __syncthreads();
        for (int it = first; it < items; it += step) {
            if (it >= a.H && row < 0) break;
            const uint16_t* src;
            uint16_t* dst;
            const float* gain = nullptr;
            if (it < a.H) {
                src = a.q + t * a.qt + it * a.qh;
                dst = a.out + t * a.ot + it * a.oh;
                gain = a.qn;
            } else if (it < a.H + c.G) {
                const int g = it - a.H;
                src = a.k + t * a.kt + g * a.kh;
                dst = c.k + page * c.kp + g * c.kh + row * c.ks;
                gain = a.kn;
            } else {
                const int g = it - a.H - c.G;
                src = a.v + t * a.vt + g * a.vh;
                dst = c.v + page * c.vp + g * c.vh + row * c.vs;
            }
            u32x4 u0 = {0, 0, 0, 0}, u1 = {0, 0, 0, 0};
            if (on) {
                u0 = *(const u32x4*)(src + lo);
                u1 = *(const u32x4*)(src + hi);
            }
            if (it < a.H + c.G) {
                float x[8], y[8];
                unpack8<BF>(u0, x);
                unpack8<BF>(u1, y);
                if (gain) {
                    float s = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], fmaf(y[i], y[i], s));
                    s = 1.0f / sqrtf(group_sum<L>(s) / (float)D + a.eps);
                    if (on)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            x[i] *= s * gain[lo + i];
                            y[i] *= s * gain[hi + i];
                        }
                }
                if (lane < ch)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float cn = cs[flip][lo + i], sn = cs[flip][64 + lo + i];
                        const float r = x[i] * cn - y[i] * sn;
                        y[i] = y[i] * cn + x[i] * sn;
                        x[i] = r;
                    }
                u0 = pack8<BF>(x);
                u1 = pack8<BF>(y);
            }
            if (on) {
                *(u32x4*)(dst + lo) = u0;
                *(u32x4*)(dst + hi) = u1;
            }
        }
        flip ^= 1;
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
    if (batch->prefix_len > kPlacesMax || (int64_t)batch->table_width * ps > kPlacesMax) return LOOPSPEC_EINVAL;
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

namespace {

// rows of 16-byte chunks: element strides and the address keep that alignment
bool rows_ok(const void* p, int64_t token, int64_t head) {
    return p && !((uintptr_t)p & 15) && token >= 0 && head >= 0 && token % 8 == 0 && head % 8 == 0;
}

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
    const int rc = paged_args(cache, batch, &c, &b);
    if (rc) return rc;
    if (args->n_heads < 1 || args->n_heads > (1 << 16) || args->n_heads % c.G) return LOOPSPEC_EINVAL;
    if (args->rot_dim < 0 || args->rot_dim > c.D || args->rot_dim % 16 || (args->rot_dim && !args->freq_dev))
        return LOOPSPEC_EINVAL;
    if (!(args->eps >= 0.f)) return LOOPSPEC_EINVAL;
    if (!rows_ok(args->q_dev, args->q_token, args->q_head) || !rows_ok(args->k_dev, args->k_token, args->k_head) ||
        !rows_ok(args->v_dev, args->v_token, args->v_head) || !rows_ok(args->q_out_dev, args->out_token, args->out_head))
        return LOOPSPEC_EINVAL;
    if ((args->n_heads > 1 && args->out_head < c.D) || (b.T > 1 && args->out_token < c.D)) return LOOPSPEC_EINVAL;
    if (!b.B || !b.T) return LOOPSPEC_OK;
    RopeArgs a{(const uint16_t*)args->q_dev, (const uint16_t*)args->k_dev, (const uint16_t*)args->v_dev,
               (uint16_t*)args->q_out_dev, args->q_token, args->q_head, args->k_token, args->k_head, args->v_token,
               args->v_head, args->out_token, args->out_head, args->freq_dev, args->q_norm_dev, args->k_norm_dev,
               args->n_heads, args->rot_dim, args->eps};
    int L = 1;
    while (L * 16 < c.D) L *= 2;
    // one pass over the heads per token while that leaves the chip unfilled
    const int64_t lanes = (int64_t)(a.H + 2 * c.G) * L;
    const int slices = (int)((lanes + kRopeThreads - 1) / kRopeThreads);
    const int y = (int64_t)b.T * slices <= 2048 ? slices : 1;
    const int x = b.T < (1 << 20) ? b.T : 1 << 20;
    void* kargs[] = {&c, &b, &a};
    const void* f = cache->dtype == LOOPSPEC_BF16 ? rope_kernel<true>(L) : rope_kernel<false>(L);
    return hipLaunchKernel(f, dim3(x, y), dim3(kRopeThreads), kargs, 0, (hipStream_t)stream) == hipSuccess ? LOOPSPEC_OK
                                                                                                          : LOOPSPEC_EHIP;
}
