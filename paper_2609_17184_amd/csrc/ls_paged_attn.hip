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
// A wave holds a tile of 32 positions of K and V in registers and runs all row
// tiles over it; its four waves take every fourth tile and meet at the end of
// the chunk.  Scores are formed transposed, S^T = K Q^T (K rows straight from
// memory as the MFMA's A operand, Q in LDS in operand order): a lane ends with
// 8 positions of one query, which after exp are its B operand of
// O^T += V^T P^T when the k index runs over the positions in that order.  V^T's
// operand needs 8 positions of one column per lane: a lane loads D/16
// consecutive columns of those 8 positions and interleaves them (one v_perm per
// word).  Neither K nor V passes through LDS, and no wave waits for another
// inside a chunk.
//
// Softmax: the reference m is raised only when some score of the tile exceeds
// it by 8 (in the base-2 exponent), which after the first tiles is rare.
// Weights are 2^(s - m + 7), so the largest lies in [2^7, 2^15]: inside fp16's
// range, and the small ones of a long prefix stay 2^31 below it before they
// vanish.  Sums are fp32; weights are rounded to the cache's type for the
// second product.
#include <algorithm>

#include "ls_paged.h"

namespace ls {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x3 __attribute__((ext_vector_type(3)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kAThreads = 256;
constexpr int kATile = 32;                    // positions per wave and step
constexpr int kAStep = 4 * kATile;            // positions per workgroup and step
constexpr float kRaise = 8.0f, kLift = 7.0f;  // log2 of what a weight may exceed the reference's by; of the reference's weight

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
    int NO, ochunk;                           // own positions: chunks at most, positions per chunk
    int rb;                                   // row blocks of the prefix
    int ptasks;                               // workgroups of the prefix
};

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
// both halves of a word finite
template <bool BF>
__device__ __forceinline__ bool finite2(uint32_t w) {
    constexpr uint32_t e = BF ? 0x7F80u : 0x7C00u;
    return (w & e) != e && ((w >> 16) & e) != e;
}

// D/16 consecutive 16-bit columns of one position
template <int E>
struct VRow {
    uint32_t w[(E + 1) / 2];
    __device__ __forceinline__ void load(const uint16_t* p) {
        if constexpr (E == 8) {
            const u32x4 u = *(const u32x4*)p;
            w[0] = u[0], w[1] = u[1], w[2] = u[2], w[3] = u[3];
        } else if constexpr (E == 6) {
            const uint32_t* q = (const uint32_t*)p;         // 12 bytes, 4-byte aligned
            w[0] = q[0], w[1] = q[1], w[2] = q[2];
        } else if constexpr (E == 4) {
            const u32x2 u = *(const u32x2*)p;
            w[0] = u[0], w[1] = u[1];
        } else if constexpr (E == 2) {
            w[0] = *(const uint32_t*)p;
        } else {
            w[0] = *p;
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
};

template <bool BF, int D, int NR>
struct Attend {
    static constexpr int E = D / 16, NS = (D + 31) / 32, LDO = D + 4;
    struct Lds {
        u32x4 q[NR][NS][64];
        float o[4][16][LDO];
        float ml[4][NR * 16][2];
    };
    struct Tile {
        u32x4 k[2][NS];
        VRow<E> v[8];
    };

    // page of the 16 positions from p; -1 when the table names none of the cache's
    static __device__ __forceinline__ int look(const PagedCache& c, const AttnTask& t, int p) {
        if (p >= t.p1) return 0;                                    // masked: any page will do
        const int i = (int)unit_div((unsigned)p >> 4, c.magic);
        if (i >= t.width) return -1;
        const int id = ld_uniform(t.table + i);
        return (unsigned)id < (unsigned)c.n_pages ? id : -1;
    }

    static __device__ __forceinline__ void load(const PagedCache& c, const AttnTask& t, int p, const int (&id)[2], Tile& x) {
        const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const unsigned blk = ((unsigned)p >> 4) + a;
            const int64_t off = (int64_t)(blk - unit_div(blk, c.magic) * c.unit) * kPageUnit;
            const int64_t pg = id[a] < 0 ? 0 : id[a];
            const uint16_t* kb = c.k + pg * c.kp + t.g * c.kh + off * c.ks;
            const uint16_t* vb = c.v + pg * c.vp + t.g * c.vh + off * c.vs;
            const int ko = n * (int)c.ks + 8 * gq, vo = 4 * gq * (int)c.vs + E * n;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                if (D % 32 == 0 || gq < 2)
                    x.k[a][s] = *(const u32x4*)(kb + ko + 32 * s);
                else
                    x.k[a][s] = u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) x.v[a * 4 + i].load(vb + vo + i * (int)c.vs);
        }
    }

    static __device__ void run(const PagedCache& c, const AttnArgs& a, const AttnTask& t, Lds& l) {
        const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 15, gq = lane >> 4;
        __syncthreads();                                            // an earlier task's LDS is read out
        for (int i = tid; i < NR * NS * 64; i += kAThreads) {
            const int la = i & 63, s = (i >> 6) % NS, rt = (i >> 6) / NS, r = rt * 16 + (la & 15), d = 32 * s + 8 * (la >> 4);
            u32x4 u = {0, 0, 0, 0};
            if (r < t.rows && d < D) {
                const int rr = t.r0 + r, tok = t.tok0 + rr / a.per, h = t.g * a.per + rr % a.per;
                u = *(const u32x4*)(a.q + tok * a.qt + h * a.qh + d);
            }
            l.q[rt][s][la] = u;
        }
        // visible positions of the lane's row in each row tile, and of the block's first and last row
        int lim[NR], minlim = t.p1, maxlim = t.p1;
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            const int r = rt * 16 + n;
            lim[rt] = r < t.rows ? t.p1 : 0;
            if (t.causal && r < t.rows) lim[rt] = min(t.p1, t.lim0 + (t.r0 + r) / a.per);
        }
        if (t.causal) {
            minlim = min(t.p1, t.lim0 + t.r0 / a.per);
            maxlim = min(t.p1, t.lim0 + (t.r0 + t.rows - 1) / a.per);
        }
        f32x4 o[NR][E];
        float m[NR], mc[NR], sum[NR];
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            m[rt] = -INFINITY, mc[rt] = 0.f, sum[rt] = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) o[rt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        __syncthreads();

        const float raise = kRaise / a.c;
        Tile cur, nxt;
        int id[2], id_n[2];
        int p = t.p0 + kATile * w;
        if (p < t.p1) {
            id[0] = look(c, t, p), id[1] = look(c, t, p + 16);
            load(c, t, p, id, cur);
            id_n[0] = look(c, t, p + kAStep), id_n[1] = look(c, t, p + kAStep + 16);
        }
        for (; p < t.p1; p += kAStep) {
            int id_2[2] = {0, 0};
            if (p + kAStep < t.p1) {
                load(c, t, p + kAStep, id_n, nxt);
                id_2[0] = look(c, t, p + 2 * kAStep), id_2[1] = look(c, t, p + 2 * kAStep + 16);
            }
            // positions no row sees do not reach the second product, whatever they hold
            if (p + kATile > t.p1) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (p + 16 * (i >> 2) + 4 * gq + (i & 3) >= t.p1) cur.v[i].zero();
            }
            u32x4 vt[E];
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    vt[e][j] = __builtin_amdgcn_perm(cur.v[2 * j + 1].w[e / 2], cur.v[2 * j].w[e / 2],
                                                     (e & 1) ? 0x07060302u : 0x05040100u);
            const bool masked = p + kATile > minlim, bad = (id[0] | id[1]) < 0;
            // some positions hidden from some rows only: a value there that is not finite would reach
            // them as 0 * value
            bool apart = false;
            if (masked && minlim != maxlim) {
                bool f = true;
#pragma unroll
                for (int e = 0; e < E; ++e)
#pragma unroll
                    for (int j = 0; j < 4; ++j) f = f && finite2<BF>(vt[e][j]);
                apart = __any(!f);
            }
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) {
                if (rt && rt * 16 >= t.rows) break;
                f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const u32x4 qf = l.q[rt][s][lane];
                    s0 = mfma16<BF>(cur.k[0][s], qf, s0);
                    s1 = mfma16<BF>(cur.k[1][s], qf, s1);
                }
                if (masked || bad) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (id[0] < 0) s0[i] = NAN;
                        if (id[1] < 0) s1[i] = NAN;
                        if (p + 4 * gq + i >= lim[rt]) s0[i] = -INFINITY;
                        if (p + 16 + 4 * gq + i >= lim[rt]) s1[i] = -INFINITY;
                    }
                }
                float mx = fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])), fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
                if (__any(mx > m[rt] + raise)) {
                    mx = fmaxf(mx, __shfl_xor(mx, 16));
                    mx = fmaxf(mx, __shfl_xor(mx, 32));
                    const float mn = fmaxf(m[rt], mx);
                    const float al = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[rt] - mn) * a.c);
                    m[rt] = mn;
                    mc[rt] = mn == -INFINITY ? 0.f : mn * a.c - kLift;
                    sum[rt] *= al;
#pragma unroll
                    for (int e = 0; e < E; ++e) o[rt][e] *= al;
                }
                float e0[4], e1[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e0[i] = __builtin_amdgcn_exp2f(fmaf(s0[i], a.c, -mc[rt]));
                    e1[i] = __builtin_amdgcn_exp2f(fmaf(s1[i], a.c, -mc[rt]));
                }
                sum[rt] += ((e0[0] + e0[1]) + (e0[2] + e0[3])) + ((e1[0] + e1[1]) + (e1[2] + e1[3]));
                const u32x4 pf = {pack2<BF>(e0[0], e0[1]), pack2<BF>(e0[2], e0[3]), pack2<BF>(e1[0], e1[1]), pack2<BF>(e1[2], e1[3])};
                if (!apart) {
#pragma unroll
                    for (int e = 0; e < E; ++e) o[rt][e] = mfma16<BF>(vt[e], pf, o[rt][e]);
                } else {
                    // one product per limit, over the positions below it, for the rows that have it
                    const int mine = min(lim[rt], p + kATile);
                    for (int lm = max(minlim, p); lm <= min(maxlim, p + kATile); ++lm) {
                        uint32_t keep[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int pos = p + 16 * (j >> 1) + 4 * gq + 2 * (j & 1);
                            keep[j] = (pos < lm ? 0xFFFFu : 0u) | (pos + 1 < lm ? 0xFFFF0000u : 0u);
                        }
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            u32x4 vm;
#pragma unroll
                            for (int j = 0; j < 4; ++j) vm[j] = vt[e][j] & keep[j];
                            const f32x4 part = mfma16<BF>(vm, pf, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[rt][e][i] = mine == lm ? o[rt][e][i] + part[i] : o[rt][e][i];
                        }
                    }
                }
            }
            cur = nxt;
            id[0] = id_n[0], id[1] = id_n[1];
            id_n[0] = id_2[0], id_n[1] = id_2[1];
        }

        // the four waves meet
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            sum[rt] += __shfl_xor(sum[rt], 16);
            sum[rt] += __shfl_xor(sum[rt], 32);
            if (gq == 0) {
                l.ml[w][rt * 16 + n][0] = m[rt] == -INFINITY ? -INFINITY : mc[rt];
                l.ml[w][rt * 16 + n][1] = sum[rt];
            }
        }
        __syncthreads();
        const int S = a.NP + a.NO;
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            if (rt * 16 >= t.rows) break;
            const int r = rt * 16 + n;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, l.ml[i][r][0]);
            const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(l.ml[w][r][0] - top);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) l.o[w][n][4 * E * gq + E * i + e] = o[rt][e][i] * f;
            __syncthreads();
            for (int i = tid; i < 16 * (D / 4); i += kAThreads) {
                const int rr = i / (D / 4), d = i % (D / 4) * 4, row = rt * 16 + rr;
                if (row >= t.rows) continue;
                f32x4 v = *(const f32x4*)&l.o[0][rr][d];
#pragma unroll
                for (int k = 1; k < 4; ++k) v += *(const f32x4*)&l.o[k][rr][d];
                const int gr = t.r0 + row;
                const size_t slot = ((size_t)(t.tok0 + gr / a.per) * a.H + t.g * a.per + gr % a.per) * S + t.split;
                *(f32x4*)(a.part + slot * D + d) = v;
                if (d == 0) {
                    float tp = -INFINITY, sm = 0.f;
#pragma unroll
                    for (int k = 0; k < 4; ++k) tp = fmaxf(tp, l.ml[k][row][0]);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        sm += l.ml[k][row][1] * (tp == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(l.ml[k][row][0] - tp));
                    a.ml[slot * 2] = tp;
                    a.ml[slot * 2 + 1] = sm;
                }
            }
            __syncthreads();
        }
    }
};

// One launch: workgroups below ptasks take the prefix (key/value head, chunk,
// row block), the others walk the own positions' tasks (sequence, chunk, row
// block, key/value head), whose number only the device knows.
template <bool BF, int D, int NR>
__global__ void __launch_bounds__(kAThreads, NR > 2 ? 1 : 2) k_paged_attn(PagedCache c, PagedBatch b, AttnArgs a) {
    using A = Attend<BF, D, NR>;
    __shared__ typename A::Lds l;
    constexpr int RT = 16 * NR;
    if ((int)blockIdx.x < a.ptasks) {
        // the row blocks of one chunk follow each other on one XCD (workgroups go round the 8 XCDs)
        const int j = blockIdx.x / 8, pair = j / a.rb * 8 + blockIdx.x % 8, rb = j % a.rb;
        if (pair >= c.G * a.NP) return;
        AttnTask t;
        t.table = b.prefix_table;
        t.width = (b.prefix + c.unit * kPageUnit - 1) / (c.unit * kPageUnit);
        t.g = pair % c.G;
        t.split = pair / c.G;
        t.p0 = t.split * a.pchunk;
        t.p1 = min(t.p0 + a.pchunk, b.prefix);
        t.tok0 = 0;
        t.r0 = rb * RT;
        t.rows = min(RT, b.T * a.per - t.r0);
        t.lim0 = 0;
        t.causal = false;
        A::run(c, a, t, l);
        return;
    }
    const int64_t cap = (int64_t)b.width * c.unit * kPageUnit;
    const int lane = threadIdx.x & 63;
    int base = 0;                             // sequences [base, base + 64) are in the lanes; those before hold `done` tasks
    int64_t done = 0;
    for (int64_t task = blockIdx.x - a.ptasks;; task += gridDim.x - a.ptasks) {
        int len = 0, start = 0, n = 0, end = 0, blocks = 0, chunks = 0;
        int64_t upto = 0;
        int hit = -1;
        for (; base < b.B; base += 64) {
            const int s = base + lane;
            len = 0, start = 0, n = 0, end = 0;
            if (s < b.B) {
                len = (int)min((int64_t)max(b.seq_len[s], 0), cap);
                end = b.q_start ? b.q_start[s + 1] : s + 1;
                start = min(max(b.q_start ? b.q_start[s] : s, 0), b.T);
                n = min(max(end, start), b.T) - start;
            }
            blocks = (n * a.per + RT - 1) / RT;
            chunks = (len + a.ochunk - 1) / a.ochunk;
            upto = (int64_t)blocks * chunks * c.G;
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                const int64_t v = __shfl_up(upto, o);
                if (lane >= o) upto += v;
            }
            const unsigned long long over = __ballot(done + upto > task);
            if (over) {
                hit = __ffsll(over) - 1;
                break;
            }
            done += __shfl(upto, 63);
        }
        if (hit < 0) return;
        blocks = __shfl(blocks, hit);
        chunks = __shfl(chunks, hit);
        n = __shfl(n, hit), start = __shfl(start, hit), end = __shfl(end, hit), len = __shfl(len, hit);
        const int64_t all = (int64_t)blocks * chunks * c.G;
        const int64_t rest = task - (done + __shfl(upto, hit) - all);
        const int seq = __builtin_amdgcn_readfirstlane(base + hit);
        const int rest_b = (int)(rest / c.G);
        AttnTask t;
        t.table = b.table + seq * b.table_stride;
        t.width = b.width;
        t.g = __builtin_amdgcn_readfirstlane((int)(rest % c.G));
        const int rb = __builtin_amdgcn_readfirstlane(rest_b % blocks), ch = __builtin_amdgcn_readfirstlane(rest_b / blocks);
        t.split = a.NP + ch;
        t.tok0 = __builtin_amdgcn_readfirstlane(start);
        t.r0 = rb * RT;
        t.rows = __builtin_amdgcn_readfirstlane(min(RT, n * a.per - t.r0));
        // a token sees its own position and those before it
        const int64_t first = (int64_t)b.seq_len[seq] - ((int64_t)end - start) + 1;
        t.lim0 = __builtin_amdgcn_readfirstlane((int)max(min(first, (int64_t)INT32_MAX / 2), (int64_t)-INT32_MAX / 2));
        t.causal = true;
        t.p0 = ch * a.ochunk;
        t.p1 = __builtin_amdgcn_readfirstlane(min(min(t.p0 + a.ochunk, len), t.lim0 + (t.r0 + t.rows - 1) / a.per));
        if (t.p1 > t.p0) A::run(c, a, t, l);  // else no row of the block sees the chunk
    }
}

// One wave per row (token, head): its chunks joined in order.
template <bool BF>
__global__ void __launch_bounds__(kAThreads) k_paged_join(PagedCache c, PagedBatch b, AttnArgs a) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6), D = c.D;
    if (row >= b.T * a.H) return;
    const int t = row / a.H, h = row % a.H;
    int64_t place = -1;
    const int seq = paged_place(b, t, &place);
    if (seq < 0 || b.seq_len[seq] < 0) return;                      // padding: its output stays as it is
    const int64_t cap = (int64_t)b.width * c.unit * kPageUnit, see = max(place + 1, (int64_t)0);
    const int own = (int)((min(see, cap) + a.ochunk - 1) / a.ochunk), S = a.NP + a.NO, n = a.NP + own;
    const float* ml = a.ml + (size_t)row * S * 2;
    const float* part = a.part + (size_t)row * S * D;
    float top = -INFINITY;
    for (int i = lane; i < n; i += 64) top = fmaxf(top, ml[2 * i]);
#pragma unroll
    for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
    float x0 = 0.f, x1 = 0.f, sum = 0.f;
    const int d = lane * 2;
    for (int i = 0; i < n; ++i) {
        const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[2 * i] - top);
        sum = fmaf(ml[2 * i + 1], f, sum);
        if (d < D) {
            const float2 v = *(const float2*)(part + (size_t)i * D + d);
            x0 = fmaf(v.x, f, x0);
            x1 = fmaf(v.y, f, x1);
        }
    }
    if (see > cap) sum = NAN;                                       // positions that the table does not hold
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    if (d < D) {
        uint32_t* o = (uint32_t*)(a.out + t * a.ot + h * a.oh + d);
        *o = pack2<BF>(x0 * inv, x1 * inv);
    }
    if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -INFINITY : top * 0.69314718055994531f + logf(sum);
}

namespace {

struct AttnPlan {
    int nr, rb, NP, pchunk, NO, ochunk, ptasks, otasks;
};

// Rows per block, chunks and workgroups from the sizes that the host knows.
int attn_plan(const PagedCache& c, const PagedBatch& b, int H, AttnPlan* pl) {
    const int per = H / c.G;
    const int64_t rows = (int64_t)b.T * per;
    if (rows * c.G > (1 << 30)) return LOOPSPEC_EINVAL;
    const int64_t most = b.prefix > 0 ? rows : (rows + b.B - 1) / b.B;
    pl->nr = most <= 16 ? 1 : most <= 32 ? 2 : 4;
    const int RT = 16 * pl->nr, slots = pl->nr > 2 ? 256 : 512;
    pl->rb = (int)((rows + RT - 1) / RT);
    // prefix: the number of chunks whose rounds of resident workgroups take the least time, a
    // workgroup's start and end counted as one step
    pl->NP = pl->pchunk = 0;
    if (b.prefix > 0) {
        const int64_t steps = (b.prefix + kAStep - 1) / kAStep, heads = (int64_t)c.G * pl->rb;
        int64_t best = -1;
        for (int64_t np = 1; np <= std::min<int64_t>(steps, 128); ++np) {
            const int64_t len = (steps + np - 1) / np, n = (steps + len - 1) / len;
            const int64_t cost = (heads * n + slots - 1) / slots * (len + 1);
            if (best < 0 || cost < best) best = cost, pl->NP = (int)n, pl->pchunk = (int)(len * kAStep);
        }
    }
    const int64_t pairs = ((int64_t)c.G * pl->NP + 7) / 8 * 8;
    if (pairs * pl->rb > (1 << 30)) return LOOPSPEC_EINVAL;
    pl->ptasks = (int)(pairs * pl->rb);
    // own positions: chunks that give about a thousand tasks when every table is full
    const int64_t cap = (int64_t)b.width * c.unit * kPageUnit;
    int64_t chunk = (cap * b.B * c.G / 1024 + kAStep - 1) / kAStep * kAStep;
    chunk = std::min<int64_t>(std::max<int64_t>(chunk, 2 * kAStep), 32 * kAStep);
    pl->ochunk = (int)chunk;
    pl->NO = (int)((cap + chunk - 1) / chunk);
    const int64_t own = ((rows + RT - 1) / RT + b.B) * pl->NO * c.G;
    pl->otasks = (int)std::min<int64_t>(own, slots);
    return LOOPSPEC_OK;
}

uint64_t attn_bytes(const PagedCache& c, const PagedBatch& b, int H, const AttnPlan& pl) {
    return (uint64_t)b.T * H * (pl.NP + pl.NO) * (c.D + 2) * 4;
}

template <bool BF, int D>
const void* attn_kernel(int nr) {
    switch (nr) {
        case 1: return (const void*)k_paged_attn<BF, D, 1>;
        case 2: return (const void*)k_paged_attn<BF, D, 2>;
        default: return (const void*)k_paged_attn<BF, D, 4>;
    }
}
template <bool BF>
const void* attn_kernel(int D, int nr) {
    switch (D) {
        case 16: return attn_kernel<BF, 16>(nr);
        case 32: return attn_kernel<BF, 32>(nr);
        case 64: return attn_kernel<BF, 64>(nr);
        case 96: return attn_kernel<BF, 96>(nr);
        default: return attn_kernel<BF, 128>(nr);
    }
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
    if (!(args->scale > 0.f) || !(cs < 3e38f) || !(kRaise / cs < 3e38f)) return LOOPSPEC_EINVAL;
    auto ok = [](const void* p, int64_t token, int64_t head) {
        return p && !((uintptr_t)p & 15) && token >= 0 && head >= 0 && token % 8 == 0 && head % 8 == 0;
    };
    if (!ok(args->q_dev, args->q_token, args->q_head) || !ok(args->out_dev, args->out_token, args->out_head)) return LOOPSPEC_EINVAL;
    if ((args->n_heads > 1 && args->out_head < c.D) || (b.T > 1 && args->out_token < c.D)) return LOOPSPEC_EINVAL;
    if (!b.B || !b.T) return LOOPSPEC_OK;
    const uint64_t need = attn_bytes(c, b, args->n_heads, pl);
    if (need && (!workspace_dev || ((uintptr_t)workspace_dev & 15) || workspace_bytes < need)) return LOOPSPEC_EINVAL;
    const uint64_t rows = (uint64_t)b.T * args->n_heads;
    AttnArgs a{(const uint16_t*)args->q_dev, args->q_token, args->q_head, (uint16_t*)args->out_dev, args->out_token, args->out_head,
               args->lse_dev, (float*)workspace_dev, (float*)workspace_dev + rows * (pl.NP + pl.NO) * c.D, cs,
               args->n_heads, args->n_heads / c.G, pl.NP, pl.pchunk, pl.NO, pl.ochunk, pl.rb, pl.ptasks};
    hipStream_t st = (hipStream_t)stream;
    void* kargs[] = {&c, &b, &a};
    const bool bf = cache->dtype == LOOPSPEC_BF16;
    if (pl.ptasks + pl.otasks > 0) {
        const void* f = bf ? attn_kernel<true>(c.D, pl.nr) : attn_kernel<false>(c.D, pl.nr);
        if (hipLaunchKernel(f, dim3(pl.ptasks + pl.otasks), dim3(kAThreads), kargs, 0, st) != hipSuccess) return LOOPSPEC_EHIP;
    }
    const void* j = bf ? (const void*)k_paged_join<true> : (const void*)k_paged_join<false>;
    if (hipLaunchKernel(j, dim3((unsigned)((rows + 3) / 4)), dim3(kAThreads), kargs, 0, st) != hipSuccess) return LOOPSPEC_EHIP;
    return LOOPSPEC_OK;
}

}  // extern "C"
