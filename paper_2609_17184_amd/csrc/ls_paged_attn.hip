// Attention of a batch over a paged cache: one long prefix that every sequence
// shares, then each sequence's own positions (causal).
//
//   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),   s_j = scale * q . k_j,  m a running reference
//
// Every row of the batch sees the whole prefix, so its rows form one matrix
// per key/value head (tokens x query heads of the group) and the prefix is read
// for up to 16 * NR rows at a time.  A workgroup takes a chunk of positions for
// such a block of rows; own positions are chunked per sequence in the same
// launch.  A second launch joins a row's chunks.
//
// Up to 32 rows: a wave holds a tile of 32 positions of K and V in registers and
// runs all row tiles over it; the four waves take every fourth tile and meet at
// the end of the chunk.  Scores are formed transposed, S^T = K Q^T (K rows straight from
// memory as the MFMA's A operand, Q in registers as the other): a lane ends with
// 8 positions of one query, which after exp are its B operand of
// O^T += V^T P^T when the k index runs over the positions in that order.  V^T's
// operand needs 8 positions of one column per lane: a lane loads D/16
// consecutive columns of those 8 positions and interleaves them (one v_perm per
// word).  Neither K nor V passes through LDS, and no wave waits for another
// inside a chunk.  More rows: see walk_wide.
//
// Softmax: a weight is 2^(c s - m) with a reference m that gives the largest
// score of its time 2^7 and is raised only when a weight could reach 2^15,
// which after the first tiles is rare.  So the largest weight stays inside fp16's
// range and the small ones of a long prefix keep 2^31 of room below it.  In bf16
// these are 2^-36 and 2^-28: the output is divided by the sum of the weights last,
// and so no finite values of 2^28 positions leave fp32 on the way.  Sums are fp32.
// Weights are rounded to the cache's type for the second product, whose operands
// have 16 bits (with a high and a low part of each they would keep twice the bits
// for twice the products).
//
// Measured, both launches (us): three sequences of 40 positions and a prefix of
// 500, 4 heads of 64: 10, two launches and their chains of loads.  32 sequences,
// prefix 8192, 256 own positions, 16 heads of 128 (fp16, 104 MB): 37, 2.8 TB/s,
// bound by the loads of the ragged own positions and 6 us of the join.  48 x 5
// rows, prefix 4007, 300 own, 55 heads of 96 (bf16, 272 MB): 81, 3.4 TB/s, the own
// positions alone 51 + 8.  192 x 4 rows, prefix 32768, 8 heads of 128 (bf16, 103
// GFLOP): 151, 684 TFLOP/s; the matrix cores are busy a third of the time, without
// a stage's loads (and their way to LDS) it would take 34 less, without the
// exponentials 8, and the join takes 11.
#include <algorithm>

#include "ls_paged.h"

namespace ls {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kAThreads = 256;
constexpr int kATile = 32;                    // positions per wave and step
constexpr int kAStep = 4 * kATile;            // positions per workgroup and step
constexpr int kRowsMax = 1 << 25;              // tokens x heads: the join's grid holds 2^32 threads
constexpr int kGroupsMax = 1 << 23;            // workgroups of the prefix, for the same reason
constexpr float kNone = -3e38f;               // the reference before the first score
constexpr float kRoom = 8.0f;                  // octaves that a weight may rise above the one that set the reference
// log2 of the highest weight: a lane's sum of 8 weights up to which none leaves fp16; in bf16, whose exponents are
// fp32's, what keeps the sums over 2^28 positions of any finite values inside fp32
template <bool BF>
constexpr float kTop = BF ? -28.0f : 15.0f;

struct AttnArgs {
    const uint16_t* q;
    int64_t qt, qh;
    uint16_t* out;
    int64_t ot, oh;
    float* lse;
    float* part;                              // [rows][splits][D], rows = tokens x heads
    float* ml;                                // [rows][splits][2]: reference (base 2), sum
    float c;                                  // scale * log2(e)
    int H, per;                               // query heads; per key/value head
    int NP, pchunk;                           // prefix: chunks, positions per chunk
    int NO, oshift;                           // own positions: chunks at most, log2 of the positions per chunk
    int rb, rows;                             // prefix: row blocks, rows of a block
    int ptasks;                               // workgroups of the prefix
};

// Chunks of a sequence's own positions: the last one takes up to half a chunk
// more rather than leave a short one.
__host__ __device__ __forceinline__ int own_chunks(int len, int shift) {
    const int c = (len + (1 << shift) / 2 - 1) >> shift;
    return len <= 0 ? 0 : c > 1 ? c : 1;
}

template <bool BF>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <bool BF>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    if (BF) return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
    return pack_h2(a, b);
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

// D/16 consecutive 16-bit columns of one position: `off` bytes behind a
// wave-uniform address
template <int E>
struct VRow {
    uint32_t w[(E + 1) / 2];
    __device__ __forceinline__ void load(const char* p, uint32_t off) {
        if constexpr (E == 8) {
            const u32x4 u = *(const u32x4*)(p + off);
            w[0] = u[0], w[1] = u[1], w[2] = u[2], w[3] = u[3];
        } else if constexpr (E == 6) {
            const uint32_t* q = (const uint32_t*)(p + off);         // 12 bytes, 4-byte aligned
            w[0] = q[0], w[1] = q[1], w[2] = q[2];
        } else if constexpr (E == 4) {
            const u32x2 u = *(const u32x2*)(p + off);
            w[0] = u[0], w[1] = u[1];
        } else if constexpr (E == 2) {
            w[0] = *(const uint32_t*)(p + off);
        } else {
            w[0] = *(const uint16_t*)(p + off);
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < (E + 1) / 2; ++i) w[i] = 0;
    }
};

// the positions [p0, p1) of one key/value head and a block of rows over them
struct AttnTask {
    const int32_t* table;
    int width;                                // pages of the table
    int g, p0, p1;
    int tok0, r0, rows;                       // row r of the block: row r0 + r of the tokens from tok0 (r < rows)
    int lim0;                                 // visible positions of token tok0; token tok0 + i sees i more (own positions)
    bool causal;
    int split;                                // where the partials go

    __device__ __forceinline__ int token(int r, int per) const { return tok0 + (r0 + r) / per; }
    // visible positions of row r, within the task's
    __device__ __forceinline__ int limit(int r, int per) const { return causal ? min(p1, lim0 + (r0 + r) / per) : p1; }
};

// Keys and values of 32 positions in a wave's registers.
template <bool BF, int D>
struct Tile {
    static constexpr int E = D / 16, NS = (D + 31) / 32;
    u32x4 k[2][NS];
    VRow<E> v[8];

    // page of the 16 positions from p; -1 when the table names none of the cache's
    static __device__ __forceinline__ int look(const PagedCache& c, const AttnTask& t, int p) {
        if (p >= t.p1) return 0;                                    // masked: any page will do
        const int i = (int)unit_div((unsigned)p >> 4, c.magic);
        if (i >= t.width) return -1;
        const int id = ld_uniform(t.table + i);
        return (unsigned)id < (unsigned)c.n_pages ? id : -1;
    }
    // address of the 16 positions from p in page id (any page for a masked or missing one)
    static __device__ __forceinline__ const char* spot(const PagedCache& c, const uint16_t* b, int64_t page, int64_t head, int64_t pos,
                                                       int g, int p, int id) {
        const unsigned blk = (unsigned)p >> 4, off = (blk - unit_div(blk, c.magic) * c.unit) * kPageUnit;
        return (const char*)(b + (id < 0 ? 0 : id) * page + g * head + off * pos);
    }
    __device__ __forceinline__ void load_k(const PagedCache& c, const AttnTask& t, int p, const int (&id)[2]) {
        const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
        const uint32_t lo = (n * (uint32_t)c.ks + 8 * gq) * 2;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const char* b = spot(c, c.k, c.kp, c.kh, c.ks, t.g, p + 16 * a, id[a]);
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                if (D % 32 == 0 || gq < 2)
                    k[a][s] = *(const u32x4*)(b + 64 * s + lo);
                else
                    k[a][s] = u32x4{0, 0, 0, 0};
            }
        }
    }
    __device__ __forceinline__ void load_v(const PagedCache& c, const AttnTask& t, int p, const int (&id)[2]) {
        const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
        const uint32_t lo = (4 * gq * (uint32_t)c.vs + E * n) * 2;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const char* b = spot(c, c.v, c.vp, c.vh, c.vs, t.g, p + 16 * a, id[a]);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[a * 4 + i].load(b + i * (2 * c.vs), lo);
        }
    }
    // the lane's position of row i of v, from the tile's first
    static __device__ __forceinline__ int place(int i) { return 16 * (i >> 2) + 4 * ((threadIdx.x & 63) >> 4) + (i & 3); }
    // operand of 32 positions for the columns E * (lane % 16) + e
    __device__ __forceinline__ u32x4 column(int e) const {
        u32x4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            r[j] = __builtin_amdgcn_perm(v[2 * j + 1].w[e / 2], v[2 * j].w[e / 2], (e & 1) ? 0x07060302u : 0x05040100u);
        return r;
    }
    // Values that no row sees do not reach the second product, whatever they hold: zero from `end` on.
    __device__ __forceinline__ void cut(int p, int end) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (p + place(i) >= end) v[i].zero();
    }
    // Zero where not finite; true when the wave has met any.
    __device__ __forceinline__ bool sane() {
        bool f = true;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < (E + 1) / 2; ++j) v[i].w[j] = ls::sane<BF>(v[i].w[j], &f);
        return __any(!f);
    }
};

__device__ __forceinline__ size_t part_slot(const AttnArgs& a, const AttnTask& t, int r) {
    return ((size_t)t.token(r, a.per) * a.H + t.g * a.per + (t.r0 + r) % a.per) * (a.NP + a.NO) + t.split;
}

// NR tiles of 16 rows in a wave: output (transposed, lane = row), reference of
// the exponent and the lane's share of the sum.
template <bool BF, int D, int NR>
struct Rows {
    static constexpr int E = D / 16, NS = (D + 31) / 32;
    static constexpr float high = BF ? 0x1p-28f : 0x1p15f;          // 2^kTop
    f32x4 o[NR][E];
    float ref[NR], sum[NR];                   // weights are 2^(c * score - ref)

    __device__ __forceinline__ void start() {
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            ref[rt] = kNone, sum[rt] = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) o[rt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // positions from `lim` on do not count for the lane's row
    static __device__ __forceinline__ void hide(int lim, int p, f32x4 (&s)[2]) {
        const int gq = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (p + 4 * gq + i >= lim) s[0][i] = -INFINITY;
            if (p + 16 + 4 * gq + i >= lim) s[1][i] = -INFINITY;
        }
    }
    // A new reference for the lane's row if some weight of its is high: the largest score so far gets the weight
    // 2^(kTop - kRoom).  The tile's other rows keep theirs, since a row's roundings follow its own scores alone.
    __device__ __forceinline__ void raise(int rt, const f32x4 (&s)[2], float part, const AttnArgs& a) {
        part = fmaxf(part, __shfl_xor(part, 16));
        part = fmaxf(part, __shfl_xor(part, 32));
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float now = part > high ? fmaxf(ref[rt], fmaf(mx, a.c, kRoom - kTop<BF>)) : ref[rt], al = __builtin_amdgcn_exp2f(ref[rt] - now);
        ref[rt] = now;
        sum[rt] *= al;
#pragma unroll
        for (int e = 0; e < E; ++e) o[rt][e] *= al;
    }
    // The weights of 32 positions as an operand, and their sum.  No maximum is taken: a lane's sum of 8
    // tells when some weight may leave its range, and then, which is rare after the first tiles, the
    // reference is raised and the weights are taken again.
    struct Weights {
        float x[2][4], part;
        __device__ __forceinline__ void take(const f32x4 (&s)[2], float ref, const AttnArgs& a) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[h][i] = __builtin_amdgcn_exp2f(fmaf(s[h][i], a.c, -ref));
            part = ((x[0][0] + x[0][1]) + (x[0][2] + x[0][3])) + ((x[1][0] + x[1][1]) + (x[1][2] + x[1][3]));
        }
        __device__ __forceinline__ u32x4 packed() const {
            return u32x4{pack2<BF>(x[0][0], x[0][1]), pack2<BF>(x[0][2], x[0][3]), pack2<BF>(x[1][0], x[1][1]), pack2<BF>(x[1][2], x[1][3])};
        }
    };
    __device__ __forceinline__ u32x4 weights(int rt, const f32x4 (&s)[2], const AttnArgs& a) {
        Weights w;
        w.take(s, ref[rt], a);
        if (__any(w.part > high)) {
            raise(rt, s, w.part, a);
            w.take(s, ref[rt], a);
        }
        sum[rt] += w.part;
        return w.packed();
    }
    // the same for all row tiles with one branch, which leaves the products' code whole
    __device__ __forceinline__ void weights(const f32x4 (&s)[NR][2], u32x4 (&p)[NR], const AttnArgs& a) {
        Weights w[NR];
        bool any = false;
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            w[rt].take(s[rt], ref[rt], a);
            any |= w[rt].part > high;
        }
        if (__builtin_expect(__any(any), 0))
#pragma unroll
            for (int rt = 0; rt < NR; ++rt)
                if (__any(w[rt].part > high)) {
                    raise(rt, s[rt], w[rt].part, a);
                    w[rt].take(s[rt], ref[rt], a);
                }
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) sum[rt] += w[rt].part, p[rt] = w[rt].packed();
    }
    // O += V^T P
    __device__ __forceinline__ void add(const Tile<BF, D>& x, const u32x4 (&p)[NR]) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const u32x4 vt = x.column(e);
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) o[rt][e] = mfma16<BF>(vt, p[rt], o[rt][e]);
        }
    }
    // What values that are not finite contribute: the products' operand has zeros in their places, since a
    // zero weight would not keep them out of the rows that do not see them.
    __device__ __forceinline__ void add_odd(const PagedCache& c, const AttnTask& t, int p, const int (&lim)[NR]) {
        const int gq = (threadIdx.x & 63) >> 4;
        for (int i = 0; i < kATile && p + i < t.p1; ++i) {
            const int id = Tile<BF, D>::look(c, t, p + i);
            const uint16_t* row = (const uint16_t*)Tile<BF, D>::spot(c, c.v, c.vp, c.vh, c.vs, t.g, p + i, id) +
                                  ((p + i) & 15) * c.vs + 4 * E * gq;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint16_t b = row[E * k + e];
                    if (finite16<BF>(b)) continue;
                    const float v = BF ? __uint_as_float((uint32_t)b << 16) : h2f(b);
#pragma unroll
                    for (int rt = 0; rt < NR; ++rt)
                        if (p + i < lim[rt]) o[rt][e][k] += v;
                }
        }
    }
    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            sum[rt] += __shfl_xor(sum[rt], 16);
            sum[rt] += __shfl_xor(sum[rt], 32);
        }
    }
    // row rt * 16 + lane % 16 of the block, without a workgroup's other waves
    __device__ __forceinline__ void store(const AttnArgs& a, const AttnTask& t, int row0) {
        const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
        finish();
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            const int r = row0 + rt * 16 + n;
            if (r >= t.rows) continue;
            const size_t slot = part_slot(a, t, r);
            float* p = a.part + slot * D + 4 * E * gq;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) p[E * i + e] = o[rt][e][i];
            if (gq == 0) a.ml[slot * 2] = ref[rt], a.ml[slot * 2 + 1] = sum[rt];
        }
    }
};

// Few rows (16 or 32): Q in registers; the next tile's keys and values come
// into the registers of this one's as soon as a product has read them.  The
// wave takes the tiles p, p + step, ...
template <bool BF, int D, int NR>
__device__ __forceinline__ void walk(const PagedCache& c, const AttnArgs& a, const AttnTask& t, int p, int step, Rows<BF, D, NR>& r) {
    constexpr int NS = (D + 31) / 32;
    using T = Tile<BF, D>;
    const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
    T x;
    int id[2] = {T::look(c, t, p), T::look(c, t, p + 16)}, nx[2];
    r.start();
    if (p >= t.p1) return;
    x.load_k(c, t, p, id);
    x.load_v(c, t, p, id);
    nx[0] = T::look(c, t, p + step), nx[1] = T::look(c, t, p + step + 16);
    u32x4 q[NR][NS];
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
        const int i = rt * 16 + n, tok = t.token(i, a.per), h = t.g * a.per + (t.r0 + i) % a.per;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            q[rt][s] = u32x4{0, 0, 0, 0};
            if (i < t.rows && 32 * s + 8 * gq < D) q[rt][s] = *(const u32x4*)(a.q + tok * a.qt + h * a.qh + 32 * s + 8 * gq);
        }
    }
    const int lo = t.limit(0, a.per), hi = t.limit(t.rows - 1, a.per);
    f32x4 s[NR][2];
    u32x4 w[NR];
    auto scores = [&]() {
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            s[rt][0] = s[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NS; ++k) {
                s[rt][0] = mfma16<BF>(x.k[0][k], q[rt][k], s[rt][0]);
                s[rt][1] = mfma16<BF>(x.k[1][k], q[rt][k], s[rt][1]);
            }
        }
    };
    int bad = 0;
    // a tile that all rows see, with another one behind it
    for (; p + kATile <= lo && p + step < t.p1; p += step) {
        const int nn[2] = {T::look(c, t, p + 2 * step), T::look(c, t, p + 2 * step + 16)};
        bad |= id[0] | id[1];
        scores();
        x.load_k(c, t, p + step, nx);
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) w[rt] = r.weights(rt, s[rt], a);
        r.add(x, w);
        x.load_v(c, t, p + step, nx);
        id[0] = nx[0], id[1] = nx[1], nx[0] = nn[0], nx[1] = nn[1];
    }
    if (bad < 0)
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) r.sum[rt] = NAN;
    int lim[NR];                              // visible positions of the lane's row
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) lim[rt] = rt * 16 + n < t.rows ? t.limit(rt * 16 + n, a.per) : 0;
    while (p < t.p1) {
        scores();
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) r.hide(lim[rt], p, s[rt]);
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) w[rt] = r.weights(rt, s[rt], a);
#pragma unroll
        for (int rt = 0; rt < NR; ++rt)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (id[h] < 0 && p + 16 * h < lim[rt]) r.sum[rt] = NAN;
        x.cut(p, t.p1);
        const bool odd = lo != hi && x.sane();
        r.add(x, w);
        if (odd) r.add_odd(c, t, p, lim);
        p += step;
        if (p >= t.p1) break;
        id[0] = T::look(c, t, p), id[1] = T::look(c, t, p + 16);
        x.load_k(c, t, p, id);
        x.load_v(c, t, p, id);
    }
}

// Many rows: the four waves share the positions and each has its own 16 * NR
// rows, Q in registers.  A stage of 64 positions comes to LDS in operand order
// (a wave brings 16 of them, in registers while the stage before is worked on)
// and every wave reads all of it.
constexpr int kStage = 64;

template <int D>
struct StageLds {
    static constexpr int E = D / 16, NS = (D + 31) / 32;
    u32x4 k[4][NS][64];                       // 16 positions each
    u32x4 v[E][2][64];                        // a column of each lane's, 32 positions each
};

// The order of a run of N reads of operands from LDS, each for NR products: 4
// reads lead.  Left to itself the compiler waits for every read before its
// products, and that and accumulators which did not stay in place cost 8 %.
template <int N, int NR>
__device__ __forceinline__ void ahead() {
    constexpr int LEAD = N < 4 ? N : 4;
    __builtin_amdgcn_sched_group_barrier(0x100, LEAD, 0);
#pragma unroll
    for (int i = 0; i < N - LEAD; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, NR, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x8, NR * LEAD, 0);
}

template <bool BF, int D, int NR>
__device__ __forceinline__ void walk_wide(const PagedCache& c, const AttnArgs& a, const AttnTask& t, StageLds<D> (&l)[2], Rows<BF, D, NR>& r) {
    constexpr int E = D / 16, NS = (D + 31) / 32;
    using T = Tile<BF, D>;
    const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = w * NR * 16;             // the wave's rows of the block
    // this wave's 16 positions of a stage
    u32x4 pk[NS];
    VRow<E> pv[4];
    auto bring = [&](int p, int id) {
        p += 16 * w;
        const char* b = T::spot(c, c.k, c.kp, c.kh, c.ks, t.g, p, id);
        const uint32_t lo = (n * (uint32_t)c.ks + 8 * gq) * 2;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            pk[s] = u32x4{0, 0, 0, 0};
            if (D % 32 == 0 || gq < 2) pk[s] = *(const u32x4*)(b + 64 * s + lo);
        }
        b = T::spot(c, c.v, c.vp, c.vh, c.vs, t.g, p, id);
        const uint32_t vo = (4 * gq * (uint32_t)c.vs + E * n) * 2;
#pragma unroll
        for (int i = 0; i < 4; ++i) pv[i].load(b + i * (2 * c.vs), vo);
    };
    auto put = [&](int p, int id, StageLds<D>& s) {
        p += 16 * w;
        if (id < 0)                           // scores of a page outside the cache are NaN
#pragma unroll
            for (int k = 0; k < NS; ++k) pk[k] = u32x4{~0u, ~0u, ~0u, ~0u};
        if (p + 16 > t.p1)                    // values that no row sees
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (p + 4 * gq + i >= t.p1) pv[i].zero();
#pragma unroll
        for (int k = 0; k < NS; ++k) s.k[w][k][lane] = pk[k];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const unsigned sel = (e & 1) ? 0x07060302u : 0x05040100u;
            ((u32x2*)&s.v[e][w >> 1][lane])[w & 1] = u32x2{__builtin_amdgcn_perm(pv[1].w[e / 2], pv[0].w[e / 2], sel),
                                                          __builtin_amdgcn_perm(pv[3].w[e / 2], pv[2].w[e / 2], sel)};
        }
    };
    int p = t.p0, id = T::look(c, t, p + 16 * w);
    bring(p, id);
    int nx = T::look(c, t, p + kStage + 16 * w);
    u32x4 q[NR][NS];
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
        const int i = row0 + rt * 16 + n, tok = t.token(i, a.per), h = t.g * a.per + (t.r0 + i) % a.per;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            q[rt][s] = u32x4{0, 0, 0, 0};
            if (i < t.rows && 32 * s + 8 * gq < D) q[rt][s] = *(const u32x4*)(a.q + tok * a.qt + h * a.qh + 32 * s + 8 * gq);
        }
    }
    r.start();
    const bool idle = row0 >= t.rows;
    const int lo = idle ? 0 : t.limit(row0, a.per), hi = idle ? 0 : t.limit(min(row0 + NR * 16, t.rows) - 1, a.per);
    // some position that the workgroup brings is hidden from some of the wave's rows; from all of them where they
    // are one token's (lo == hi) and another wave's token is later
    const bool hidden = lo != hi || hi < t.p1;
    put(p, id, l[0]);
    id = nx;
    if (p + kStage < t.p1) bring(p + kStage, id);
    nx = T::look(c, t, p + 2 * kStage + 16 * w);
    __syncthreads();

    f32x4 s[NR][2];
    u32x4 wt[NR];
    auto scores = [&](int h, const StageLds<D>& st) {
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) s[rt][0] = s[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NS; ++k)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const u32x4 f = st.k[2 * h + b][k][lane];
#pragma unroll
                for (int rt = 0; rt < NR; ++rt) s[rt][b] = mfma16<BF>(f, q[rt][k], s[rt][b]);
            }
    };
    // the stage after p's to LDS, the one after that on its way
    int turn = 0;
    auto next = [&]() {
        put(p + kStage, id, l[(turn + 1) & 1]);
        id = nx;
        if (p + 2 * kStage < t.p1) bring(p + 2 * kStage, id);
        nx = T::look(c, t, p + 3 * kStage + 16 * w);
        __syncthreads();
        ++turn, p += kStage;
    };
    // stages that all rows of the wave see (waves of a workgroup may leave at different ones: both loops
    // have one barrier a stage)
    while (p + kStage <= lo) {
        const StageLds<D>& st = l[turn & 1];
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            scores(h, st);
            ahead<2 * NS, NR>();
            r.weights(s, wt, a);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const u32x4 v = st.v[e][h][lane];
#pragma unroll
                for (int rt = 0; rt < NR; ++rt) r.o[rt][e] = mfma16<BF>(v, wt[rt], r.o[rt][e]);
            }
            ahead<E, NR>();
        }
        if (p + kStage >= t.p1) return;
        next();
    }
    int lim[NR];
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) lim[rt] = row0 + rt * 16 + n < t.rows ? t.limit(row0 + rt * 16 + n, a.per) : 0;
    for (;;) {
        const StageLds<D>& st = l[turn & 1];
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            const int ph = p + kATile * h;
            if (ph >= hi) break;
            scores(h, st);
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) r.hide(lim[rt], ph, s[rt]);
            r.weights(s, wt, a);
            bool f = true;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                u32x4 v = st.v[e][h][lane];
                if (hidden) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = sane<BF>(v[j], &f);
                }
#pragma unroll
                for (int rt = 0; rt < NR; ++rt) r.o[rt][e] = mfma16<BF>(v, wt[rt], r.o[rt][e]);
            }
            if (__any(!f)) r.add_odd(c, t, ph, lim);
        }
        if (p + kStage >= t.p1) return;
        next();
    }
}

template <int D, int NR>
struct MeetLds {
    float o[4][16][D + 4];
    float ml[4][NR * 16][2];
};

// the four waves' results of a workgroup's task, summed and stored
template <bool BF, int D, int NR>
__device__ __forceinline__ void meet(const AttnArgs& a, const AttnTask& t, Rows<BF, D, NR>& r, MeetLds<D, NR>& l) {
    constexpr int E = D / 16;
    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, n = lane & 15, gq = lane >> 4;
    r.finish();
    __syncthreads();                          // an earlier task's LDS is read out
#pragma unroll
    for (int rt = 0; rt < NR; ++rt)
        if (gq == 0) l.ml[w][rt * 16 + n][0] = r.ref[rt], l.ml[w][rt * 16 + n][1] = r.sum[rt];
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
        if (rt * 16 >= t.rows) break;
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, l.ml[i][rt * 16 + n][0]);
        const float f = __builtin_amdgcn_exp2f(r.ref[rt] - top);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) l.o[w][n][4 * E * gq + E * i + e] = r.o[rt][e][i] * f;
        __syncthreads();
        for (int i = tid; i < 16 * (D / 4); i += kAThreads) {
            const int rr = i / (D / 4), d = i % (D / 4) * 4, row = rt * 16 + rr;
            if (row >= t.rows) continue;
            f32x4 v = *(const f32x4*)&l.o[0][rr][d];
#pragma unroll
            for (int k = 1; k < 4; ++k) v += *(const f32x4*)&l.o[k][rr][d];
            const size_t slot = part_slot(a, t, row);
            *(f32x4*)(a.part + slot * D + d) = v;
            if (d == 0) {
                float tp = -INFINITY, sm = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) tp = fmaxf(tp, l.ml[k][row][0]);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    sm += l.ml[k][row][1] * __builtin_amdgcn_exp2f(l.ml[k][row][0] - tp);
                a.ml[slot * 2] = tp;
                a.ml[slot * 2 + 1] = sm;
            }
        }
        __syncthreads();
    }
}

// The own positions' tasks, numbered sequence by sequence: (chunk, row block,
// key/value head).  How many there are only the device knows; whoever asks for
// rising numbers walks the sequences once.
struct OwnTasks {
    int base = 0;                             // the sequences before it hold `done` tasks
    int64_t done = 0;

    __device__ bool find(const PagedCache& c, const PagedBatch& b, const AttnArgs& a, int64_t task, int RT, AttnTask& t) {
        constexpr int PER = 4;                // sequences a lane takes at a time
        const int64_t cap = (int64_t)b.width * c.unit * kPageUnit;
        const int lane = threadIdx.x & 63;
        for (; base < b.B; base += 64 * PER) {
            int len[PER], start[PER], n[PER], raw[PER], end[PER];
            int64_t mine[PER], all = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int s = base + lane * PER + i;
                raw[i] = -1, start[i] = 0, end[i] = 0;
                if (s < b.B) {
                    raw[i] = b.seq_len[s];
                    end[i] = b.q_start ? b.q_start[s + 1] : s + 1;
                    start[i] = b.q_start ? b.q_start[s] : s;
                }
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                // a token sees its own position and those before it
                const int64_t first = (int64_t)raw[i] - ((int64_t)end[i] - start[i]) + 1;
                len[i] = (int)min((int64_t)max(raw[i], 0), cap);
                raw[i] = (int)max(min(first, (int64_t)INT32_MAX / 2), (int64_t)-INT32_MAX / 2);
                start[i] = min(max(start[i], 0), b.T);
                n[i] = min(max(end[i], start[i]), b.T) - start[i];
                mine[i] = (int64_t)((n[i] * a.per + RT - 1) / RT) * own_chunks(len[i], a.oshift) * c.G;
                all += mine[i];
            }
            int64_t upto = all;
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                const int64_t v = __shfl_up(upto, o);
                if (lane >= o) upto += v;
            }
            const unsigned long long over = __ballot(done + upto > task);
            if (!over) {
                done += (int64_t)(((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(upto >> 32), 63) << 32) |
                                  (unsigned)__builtin_amdgcn_readlane((int)upto, 63));
                continue;
            }
            // the sequence among the lane's, then (wave-uniform from here, by readlane) the task among its own
            int64_t at = done + upto - all;
            int k = 0;
#pragma unroll
            for (int i = 0; i < PER - 1; ++i)
                if (k == i && at + mine[i] <= task) {
                    at += mine[i], k = i + 1;
                    len[0] = len[i + 1], start[0] = start[i + 1], n[0] = n[i + 1], raw[0] = raw[i + 1];
                }
            const int hit = __ffsll(over) - 1, seq = base + hit * PER + __builtin_amdgcn_readlane(k, hit);
            const unsigned rest = (unsigned)__builtin_amdgcn_readlane((int)(task - at), hit), rest_b = rest / c.G;
            const int own_n = __builtin_amdgcn_readlane(n[0], hit), own_len = __builtin_amdgcn_readlane(len[0], hit);
            const int blocks = (own_n * a.per + RT - 1) / RT, rb = rest_b % blocks, ch = rest_b / blocks;
            t.table = b.table + seq * b.table_stride;
            t.width = b.width;
            t.g = rest % c.G;
            t.split = a.NP + ch;
            t.tok0 = __builtin_amdgcn_readlane(start[0], hit);
            t.r0 = rb * RT;
            t.rows = min(RT, own_n * a.per - t.r0);
            t.lim0 = __builtin_amdgcn_readlane(raw[0], hit);
            t.causal = true;
            t.p0 = ch << a.oshift;
            t.p1 = ch + 1 < own_chunks(own_len, a.oshift) ? t.p0 + (1 << a.oshift) : own_len;
            t.p1 = min(t.p1, t.lim0 + (t.r0 + t.rows - 1) / a.per);
            return true;
        }
        return false;
    }
};

// One launch.  Workgroups below ptasks take the prefix (key/value head, chunk,
// row block): up to 32 rows with the four waves on different positions (WIDE =
// false), or up to 64 * NR rows with the four waves on different rows.  The
// others walk the own positions' tasks: a wave each with 16 rows, or (WIDE_OWN)
// a workgroup each like the prefix.
// Three workgroups a CU where registers and LDS suffice (heads up to 96): 88 -> 83 us
// for 240 rows over 4007 positions of 55 heads of 96; at 128 the registers are two's.
template <bool BF, int D, int NR, bool WIDE, bool WIDE_OWN>
__global__ void __launch_bounds__(kAThreads) __attribute__((amdgpu_waves_per_eu(WIDE && D <= 96 ? 3 : 2)))
k_paged_attn(PagedCache c, PagedBatch b, AttnArgs a) {
    constexpr int ROWS = WIDE ? 64 * NR : 16 * NR;
    union Lds {
        StageLds<(WIDE ? D : 16)> st[2];
        MeetLds<(WIDE ? 16 : D), (WIDE ? 1 : NR)> m;
    };
    __shared__ Lds l;
    const bool prefix = (int)blockIdx.x < a.ptasks;
    if (prefix || WIDE_OWN) {
        OwnTasks own;
        for (int64_t task = (int)blockIdx.x - a.ptasks;; task += gridDim.x - a.ptasks) {
            AttnTask t;
            if (prefix) {
                // the row blocks of one chunk follow each other on one XCD (workgroups go round the 8 XCDs)
                const int j = blockIdx.x / 8, pair = j / a.rb * 8 + blockIdx.x % 8, rb = j % a.rb;
                if (pair >= c.G * a.NP) return;
                t.table = b.prefix_table;
                t.width = (b.prefix + c.unit * kPageUnit - 1) / (c.unit * kPageUnit);
                t.g = pair % c.G;
                t.split = pair / c.G;
                t.p0 = t.split * a.pchunk;
                t.p1 = min(t.p0 + a.pchunk, b.prefix);
                t.tok0 = 0;
                t.r0 = rb * a.rows;
                t.rows = min(a.rows, b.T * a.per - t.r0);
                t.lim0 = 0;
                t.causal = false;
            } else {
                if (!own.find(c, b, a, task, ROWS, t)) return;
                if (t.p1 <= t.p0) continue;   // no row of the block sees the chunk
            }
            Rows<BF, D, NR> r;
            if constexpr (WIDE) {
                __syncthreads();              // an earlier task's LDS is read out
                walk_wide<BF, D, NR>(c, a, t, l.st, r);
                r.store(a, t, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * NR * 16);
            } else {
                walk<BF, D, NR>(c, a, t, t.p0 + kATile * __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kAStep, r);
                meet<BF, D, NR>(a, t, r, l.m);
            }
            if (prefix) return;
        }
    }
    if constexpr (!WIDE_OWN) {
        OwnTasks own;
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        for (int64_t task = ((int)blockIdx.x - a.ptasks) * 4 + w;; task += ((int)gridDim.x - a.ptasks) * 4) {
            AttnTask t;
            if (!own.find(c, b, a, task, 16, t)) return;
            if (t.p1 <= t.p0) continue;
            Rows<BF, D, 1> r;
            walk<BF, D, 1>(c, a, t, t.p0, kATile, r);
            r.store(a, t, 0);
        }
    }
}

// WPR waves per row (token, head) join its chunks: 256 at a time are in the
// lanes of every wave by their references and sums, a wave takes every WPR-th
// group of chunks, a group of lanes (four columns a lane) one chunk each.
template <bool BF, int WPR>
__global__ void __launch_bounds__(WPR > 4 ? 64 * WPR : kAThreads) k_paged_join(PagedCache c, PagedBatch b, AttnArgs a) {
    constexpr int ROWS = WPR > 4 ? 1 : 4 / WPR;
    __shared__ float l[WPR > 1 ? WPR : 1][ROWS][128];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, sub = wv % WPR, rl = wv / WPR, D = c.D;
    const int row = blockIdx.x * ROWS + rl;
    const bool in = row < b.T * a.H;
    const int t = in ? row / a.H : 0, h = row % a.H;
    int64_t place = -1;
    const int seq = in ? paged_place(b, t, &place) : -1;
    const bool live = seq >= 0 && b.seq_len[seq] >= 0;              // padding: its output stays as it is
    const int64_t cap = (int64_t)b.width * c.unit * kPageUnit, see = max(place + 1, (int64_t)0);
    // the sequence's chunks that begin before the row's limit
    const int own = live ? min(own_chunks((int)min((int64_t)b.seq_len[seq], cap), a.oshift), ((int)min(see, cap) + (1 << a.oshift) - 1) >> a.oshift) : 0;
    const int S = a.NP + a.NO, n = live ? a.NP + own : 0;
    const float* ml = a.ml + (size_t)row * S * 2;
    const float* part = a.part + (size_t)row * S * D;
    const int gl = D > 64 ? 32 : D / 4, groups = 64 / gl, g = lane / gl, d = lane % gl * 4;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float top = kNone, sum = 0.f;
    for (int i0 = 0; i0 < n; i0 += 64) {
        float2 v = {kNone, 0.f};
        if (i0 + lane < n) v = *(const float2*)(ml + 2 * (i0 + lane));
        float tp = fmaxf(top, v.x);
#pragma unroll
        for (int o = 1; o < 64; o *= 2) tp = fmaxf(tp, __shfl_xor(tp, o));
        const float old = __builtin_amdgcn_exp2f(top - tp), f = __builtin_amdgcn_exp2f(v.x - tp);
        float s = v.y * f;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) s += __shfl_xor(s, o);
        sum = fmaf(sum, old, s);
        acc *= old;
        top = tp;
        const int m = min(64, n - i0);
        for (int k0 = sub * groups; k0 < m; k0 += 4 * WPR * groups) {
            f32x4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = k0 + j * WPR * groups + g;
                x[j] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (k < m && d < D) x[j] = *(const f32x4*)(part + (size_t)(i0 + k) * D + d);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float fk = __shfl(f, min(k0 + j * WPR * groups + g, 63));
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(x[j][e], fk, acc[e]);
            }
        }
    }
    for (int o = gl; o < 64; o *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o);
    if (WPR > 1) {
        if (g == 0 && d < D) *(f32x4*)&l[sub][rl][d] = acc;
        __syncthreads();
        if (sub == 0 && g == 0 && d < D) {
#pragma unroll
            for (int i = 1; i < WPR; ++i) acc += *(const f32x4*)&l[i][rl][d];
        }
    }
    if (!live || sub) return;
    if (see > cap) sum = NAN;                                       // positions that the table does not hold
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    if (g == 0 && d < D) {
        const u32x2 r = {pack2<BF>(acc[0] * inv, acc[1] * inv), pack2<BF>(acc[2] * inv, acc[3] * inv)};
        *(u32x2*)(a.out + t * a.ot + h * a.oh + d) = r;
    }
    if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -INFINITY : top * 0.69314718055994531f + logf(sum);
}

namespace {

struct AttnPlan {
    int nr;                                   // tiles of 16 rows a wave has
    bool wide, wide_own;
    int rb, rows, NP, pchunk, NO, oshift, ptasks, otasks;
};

// Rows per block, chunks and workgroups from the sizes that the host knows.
int attn_plan(const PagedCache& c, const PagedBatch& b, int H, AttnPlan* pl) {
    const int per = H / c.G;
    const int64_t rows = (int64_t)b.T * per, each = (rows + b.B - 1) / b.B;
    if (rows * c.G > kRowsMax) return LOOPSPEC_EINVAL;
    // Both sides at heads of 128 (us): 4 sequences of 40 rows a head over 2000 own positions, a wave's
    // 16 rows at a time 34, a workgroup's 128 34; of 128 rows 52 and 45.
    pl->wide_own = each > 32;
    // 48 rows over 8192 positions of 16 heads, 32 at a time 32.2, all at a time 32.0 (64 rows: 33.1, 34.3)
    pl->wide = pl->wide_own || (b.prefix > 0 && rows > 32);
    // 32 rows a wave halve what passes through LDS, 16 spread better: 96 rows 43.7 and 38.9, 240 rows
    // 58.6 and 58.0, 768 rows of 8 heads over 32768 positions 151 and 181
    pl->nr = pl->wide ? (pl->wide_own || rows > 256 ? 2 : 1) : b.prefix > 0 && rows > 16 ? 2 : 1;
    // slots: two workgroups a CU, also for heads up to 96, of which three fit (chunks for 768: 91 us instead of 83
    // for 240 rows over 4007 positions of 55 heads of 96)
    const int block = pl->nr * (pl->wide ? 64 : 16), slots = 512;
    pl->rb = (int)((rows + block - 1) / block);
    pl->rows = (int)((rows + pl->rb * 16 - 1) / (pl->rb * 16) * 16);
    // prefix: the number of chunks whose rounds of resident workgroups take the least time, a
    // workgroup's start and end counted as two steps
    pl->NP = pl->pchunk = 0;
    if (b.prefix > 0) {
        const int64_t steps = (b.prefix + kAStep - 1) / kAStep, heads = (int64_t)c.G * pl->rb;
        int64_t best = -1;
        for (int64_t np = 1; np <= std::min<int64_t>(steps, 128); ++np) {
            const int64_t len = (steps + np - 1) / np, n = (steps + len - 1) / len;
            const int64_t cost = (heads * n + slots - 1) / slots * (len + 2);
            if (best < 0 || cost < best) best = cost, pl->NP = (int)n, pl->pchunk = (int)(len * kAStep);
        }
    }
    const int64_t pairs = ((int64_t)c.G * pl->NP + 7) / 8 * 8;
    if (pairs * pl->rb > kGroupsMax) return LOOPSPEC_EINVAL;
    pl->ptasks = (int)(pairs * pl->rb);
    // own positions: about two chunks per resident wave (or workgroup) when every table is full, of at
    // least four tiles a wave (16 instead, or 16 stages for 8: 4 x 40 rows over 2000 positions 34 -> 45 us)
    const int64_t cap = (int64_t)b.width * c.unit * kPageUnit, all = cap * b.B * c.G;
    pl->oshift = pl->wide_own ? 9 : 7;
    while (pl->oshift < 12 && (all >> pl->oshift) > (pl->wide_own ? 2 * slots : 8 * slots)) ++pl->oshift;
    pl->NO = own_chunks((int)cap, pl->oshift);
    const int RT = pl->wide_own ? block : 16;
    const int64_t own = ((rows + RT - 1) / RT + b.B) * pl->NO * c.G;
    pl->otasks = (int)std::min<int64_t>(pl->wide_own ? own : (own + 3) / 4, slots);
    return LOOPSPEC_OK;
}

uint64_t attn_bytes(const PagedCache& c, const PagedBatch& b, int H, const AttnPlan& pl) {
    return (uint64_t)b.T * H * (pl.NP + pl.NO) * (c.D + 2) * 4;
}

template <bool BF, int D>
const void* attn_kernel(const AttnPlan& p) {
    if (p.wide_own) return (const void*)k_paged_attn<BF, D, 2, true, true>;
    if (p.wide) return p.nr == 1 ? (const void*)k_paged_attn<BF, D, 1, true, false> : (const void*)k_paged_attn<BF, D, 2, true, false>;
    return p.nr == 1 ? (const void*)k_paged_attn<BF, D, 1, false, false> : (const void*)k_paged_attn<BF, D, 2, false, false>;
}
template <bool BF>
const void* attn_kernel(int D, const AttnPlan& p) {
    switch (D) {
        case 16: return attn_kernel<BF, 16>(p);
        case 32: return attn_kernel<BF, 32>(p);
        case 64: return attn_kernel<BF, 64>(p);
        case 96: return attn_kernel<BF, 96>(p);
        default: return attn_kernel<BF, 128>(p);
    }
}

template <bool BF>
const void* join_kernel(int wpr) {
    return wpr == 1 ? (const void*)k_paged_join<BF, 1> : wpr == 4 ? (const void*)k_paged_join<BF, 4> : (const void*)k_paged_join<BF, 16>;
}

int attn_check(const loopspec_paged_cache* cache, const loopspec_paged_batch* batch, int n_heads, PagedCache* c,
               PagedBatch* b, AttnPlan* pl) {
    const int rc = paged_args(cache, batch, c, b);
    if (rc) return rc;
    if (n_heads < 1 || n_heads > (1 << 16) || n_heads % c->G) return LOOPSPEC_EINVAL;
    if (b->prefix > 0 && !b->prefix_table) return LOOPSPEC_EINVAL;
    if (!b->B || !b->T) return LOOPSPEC_OK;
    return attn_plan(*c, *b, n_heads, pl);
}

}  // namespace
}  // namespace ls

extern "C" {

uint64_t loopspec_prefix_attention_workspace_bytes(const loopspec_paged_cache* cache, const loopspec_paged_batch* batch,
                                                   int32_t n_heads) {
    ls::PagedCache c;
    ls::PagedBatch b;
    ls::AttnPlan pl{};
    if (ls::attn_check(cache, batch, n_heads, &c, &b, &pl)) return 0;
    if (!b.B || !b.T) return 0;
    return ls::attn_bytes(c, b, n_heads, pl);
}

int loopspec_prefix_attention(const loopspec_paged_cache* cache, const loopspec_paged_batch* batch,
                              const loopspec_attention_args* args, void* workspace_dev, uint64_t workspace_bytes,
                              void* stream) {
    using namespace ls;
    PagedCache c;
    PagedBatch b;
    AttnPlan pl{};
    if (!args) return LOOPSPEC_EINVAL;
    const int rc = attn_check(cache, batch, args->n_heads, &c, &b, &pl);
    if (rc) return rc;
    const float cs = args->scale * 1.44269504088896341f;
    if (!(args->scale > 0.f) || !(cs < 3e38f)) return LOOPSPEC_EINVAL;
    auto ok = [](const void* p, int64_t token, int64_t head) {
        return p && !((uintptr_t)p & 15) && token >= 0 && head >= 0 && token % 8 == 0 && head % 8 == 0;
    };
    if (!b.B || !b.T) return LOOPSPEC_OK;     // (empty tensors have no address)
    if (!ok(args->q_dev, args->q_token, args->q_head) || !ok(args->out_dev, args->out_token, args->out_head)) return LOOPSPEC_EINVAL;
    if ((args->n_heads > 1 && args->out_head < c.D) || (b.T > 1 && args->out_token < c.D)) return LOOPSPEC_EINVAL;
    const uint64_t need = attn_bytes(c, b, args->n_heads, pl);
    if (need && (!workspace_dev || ((uintptr_t)workspace_dev & 15) || workspace_bytes < need)) return LOOPSPEC_EINVAL;
    const uint64_t rows = (uint64_t)b.T * args->n_heads;
    AttnArgs a{(const uint16_t*)args->q_dev, args->q_token, args->q_head, (uint16_t*)args->out_dev, args->out_token, args->out_head,
               args->lse_dev, (float*)workspace_dev, (float*)workspace_dev + rows * (pl.NP + pl.NO) * c.D, cs,
               args->n_heads, args->n_heads / c.G, pl.NP, pl.pchunk, pl.NO, pl.oshift, pl.rb, pl.rows, pl.ptasks};
    hipStream_t st = (hipStream_t)stream;
    void* kargs[] = {&c, &b, &a};
    const bool bf = cache->dtype == LOOPSPEC_BF16;
    if (pl.ptasks + pl.otasks > 0) {
        const void* f = bf ? attn_kernel<true>(c.D, pl) : attn_kernel<false>(c.D, pl);
        if (hipLaunchKernel(f, dim3(pl.ptasks + pl.otasks), dim3(kAThreads), kargs, 0, st) != hipSuccess) return LOOPSPEC_EHIP;
    }
    // Waves per row: one has 4 (D = 128) to 64 chunks in flight at once; with enough rows several each only
    // make more workgroups.  In all (us) with 1, 4 and 16: 8 rows of 128 chunks 37.5, 33.4, 32.6; 512 rows 39.2, 37.6, 40.0;
    // 1024 rows 35.1, 34.2, 41.6; 1536 rows 42.0, 43.8, 53.9; 13200 rows 77, 91, 148.
    const int S = pl.NP + pl.NO, wpr = S <= 8 || rows > 1024 ? 1 : S <= 64 || rows > 256 ? 4 : 16;
    const void* j = bf ? join_kernel<true>(wpr) : join_kernel<false>(wpr);
    const unsigned per_wg = wpr > 4 ? 1 : 4 / wpr;
    if (hipLaunchKernel(j, dim3((unsigned)((rows + per_wg - 1) / per_wg)), dim3(wpr > 4 ? 64 * wpr : kAThreads), kargs, 0, st) != hipSuccess)
        return LOOPSPEC_EHIP;
    return LOOPSPEC_OK;
}

}  // extern "C"
