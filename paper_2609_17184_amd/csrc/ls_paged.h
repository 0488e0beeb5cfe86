// A paged key/value cache and the batch of sequences that a call works on, as
// the device sees them (loopspec_paged_cache and loopspec_paged_batch).
#pragma once
#include "../../include/loopspec.h"
#include "ls_common.h"

namespace ls {

constexpr int kPageUnit = 16;                 // a page holds a multiple of 16 positions
constexpr int kPageMax = 1024;
constexpr int64_t kPlacesMax = 1ll << 28;     // positions a page table may span
constexpr int kTokensMax = 1 << 25;           // 2^23 workgroups of 4 tokens: a grid holds 2^32 threads
constexpr int64_t kStrideMax = 1ll << 24;     // elements between neighbouring positions or heads

struct PagedCache {
    uint16_t *k, *v;
    int64_t kp, kh, ks, vp, vh, vs;           // strides in elements: page, head, position
    int n_pages, G, D;
    int unit;                                 // page_size / 16
    unsigned magic;                           // x / unit = x * magic >> 32 for x < 2^26; unit 1 has no magic (0)
};

struct PagedBatch {
    const int32_t* q_start;                   // null: token b belongs to sequence b
    const int32_t* seq_len;
    const int32_t* table;
    int64_t table_stride;
    const int32_t* prefix_table;
    int B, T, width, prefix;
};

// x / unit of a block of 16 positions, x < 2^24: magic = ceil(2^32 / unit)
// overshoots 2^32 / unit by less than 1, so the product is off by less than
// x / 2^32 < 1 / unit while unit <= 64
__host__ __device__ __forceinline__ unsigned unit_div(unsigned x, unsigned magic) {
    return magic ? (unsigned)(((unsigned long long)x * magic) >> 32) : x;
}

// Sequence of token t (-1: none) and the token's own position, which is below
// zero when the sequence is shorter than its tokens.  Every lane of the wave
// calls it with the same t.  q_start is ascending, so the entries at or below t
// are counted rather than searched: the loads do not wait for each other.
__device__ __forceinline__ int paged_place(const PagedBatch& p, int t, int64_t* place) {
    int b = t, end = t + 1;
    if (p.q_start) {
        int n = 0;
        for (int i = threadIdx.x & 63; i <= p.B; i += 64) n += __popcll(__ballot(p.q_start[i] <= t));
        n = __builtin_amdgcn_readfirstlane(n);      // lane 0 took part in every turn
        if (n < 1 || n > p.B) return -1;
        b = n - 1;
        end = p.q_start[n];
    } else if (b >= p.B) {
        return -1;
    }
    *place = (int64_t)p.seq_len[b] - ((int64_t)end - t);
    return b;
}

// scales of 8-bit pages: one byte for 16 positions of a head
struct PageScales {
    uint8_t *k, *v;
    int64_t kp, kh, vp, vh;                   // strides: page, head
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

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
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    if (BF) return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));      // one instruction
}
template <bool BF>
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
    return u32x4{pack2<BF>(f[0], f[1]), pack2<BF>(f[2], f[3]), pack2<BF>(f[4], f[5]), pack2<BF>(f[6], f[7])};
}

template <bool BF>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <bool BF>
__device__ __forceinline__ bool finite16(uint32_t w) {
    constexpr uint32_t e = BF ? 0x7F80u : 0x7C00u;
    return (w & e) != e;
}
// the halves of a word that are finite; *all becomes false when one is not
template <bool BF>
__device__ __forceinline__ uint32_t sane(uint32_t w, bool* all) {
    const uint32_t k = (finite16<BF>(w) ? 0xFFFFu : 0u) | (finite16<BF>(w >> 16) ? 0xFFFF0000u : 0u);
    *all = *all && k == ~0u;
    return w & k;
}

// host: LOOPSPEC_EINVAL unless the structs describe what the kernels take
int scale_args(const loopspec_paged_cache* cache, const loopspec_page_scales* scales, PageScales* s);
bool rows_ok(const void* p, int64_t token, int64_t head);
int rope_args(const PagedCache& c, const PagedBatch& b, const loopspec_rope_args* args);
int paged_args(const loopspec_paged_cache* cache, const loopspec_paged_batch* batch, PagedCache* c, PagedBatch* b);

}  // namespace ls
