// Attention over a paged cache of 16-bit or 8-bit pages under a window of the
// latest positions and a few first ones.
//
//   o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),   s_j = scale * q . k_j,   j <= p and (p - j < window or j < sinks)
//
// A task is a block of rows (tokens x query heads of a key/value head) of one
// sequence.  What its rows see are two runs of blocks of 16 positions, the first
// ones and the latest; the task's list of blocks is the two put together, cut
// into chunks where there are too few tasks to fill the card.
//
// The products are those of the prefix's attention: S^T = K Q^T with K straight
// from memory as the matrix instruction's first operand, so that a lane holds 4
// positions of each of two blocks for one row; exp of them is the operand of
// O^T += V^T P^T.
//
// 8-bit pages: codes have 4 significant bits and are exact in fp16 and bf16, so
// they are widened (one instruction for two) and multiplied as they are.  A key
// block's scale joins the factor of its scores.  A value block's scale 2^e goes
// into the widening in bf16, whose range holds the result; in fp16 it goes into
// the weights, 2^(c s + e - m), and out of their sum again, so that m bounds the
// product and neither factor leaves fp16.
//
// Softmax: a weight is 2^(c s - m) with a reference m that gives the largest
// score of its time 2^7 and is raised only when a weight could reach 2^15; in
// bf16 these are 2^-36 and 2^-28, and the division by the sum comes last, so that
// no finite values leave fp32.  Sums are fp32, weights are rounded to the
// queries' type for the second product.
//
// Three kernels, since one that held all three ways had the registers of the
// largest (and 135 us where two launches take 73): blocks of 128 rows, whose four
// waves share positions through LDS (k_window_wide); blocks of 16, whose waves
// take every fourth tile and meet at the end (k_window); a wave alone for short
// tasks (k_window_waves).
//
// Measured (us a call), and what bounds it.  64 rows x 4 heads of 8 key/value
// heads of 128 over 4100 of 12000 positions (bf16, 954 MB): 165, 5.8 TB/s; a plain
// stream of reads reaches 7.2.  32 rows of 16 heads of 128 over up to 8192 positions
// (fp16 over 8-bit pages, 584 MB): 117, of which 113 at 5.2 TB/s and 5 the join.
// 8001 rows of 28 heads on 4 of 128 under a window of 2048 (bf16, 206 GFLOP): 234,
// 880 TFLOP/s; the matrix cores are busy 36 % of the cycles and vector instructions
// 41 %, which two waves a SIMD overlap in part only.  250 tokens of 32 heads on 8 of 128 behind
// 8007 positions (bf16 over 8-bit pages, 33 GFLOP): 72, of which the own positions'
// launch and the taking in of partial results 22.  5 prompts of up to 900 tokens,
// 55 heads of 96 (fp16 over 8-bit pages, 66 GFLOP): 143; a task's begin and end
// (lengths, pages, first loads, the two stages that the diagonal cuts) take 13 of
// the 25 that a block of 128 rows over 640 positions does, while the CU's other
// workgroup goes on.  Three tokens of 4 heads: 9.2, of which 3 are an empty launch and
// the rest loads that wait for each other (lengths, pages, scales, keys).
#include <algorithm>

#include "ls_paged.h"

namespace ls {

namespace {

constexpr int kT = 256;
constexpr int kWideRows = 128, kFewRows = 16;  // rows of a block where the waves share positions, and where each has its own
constexpr int kUncut = 24;                    // tiles of 32 positions that blocks of few rows take in one piece
constexpr int kRowsMax = 1 << 25;              // tokens x heads: the join's grid holds 2^32 threads
constexpr int kGroupsMax = 1 << 23;            // workgroups of the prefix, for the same reason
constexpr int kAll = 1 << 30;                 // a window that holds every position
constexpr int kNowhere = INT32_MIN;
constexpr float kNone = -3e38f;               // the reference before the first score
constexpr float kRoom = 8.0f;                  // octaves that a weight may rise above the one that set the reference
template <bool BF>
constexpr float kTop = BF ? -28.0f : 15.0f;    // log2 of the highest weight

struct WinArgs {
    const uint16_t* q;
    int64_t qt, qh;
    uint16_t* out;
    int64_t ot, oh;
    float* lse;
    float* part;                              // [rows][slots][D], rows = tokens x heads
    float* ml;                                // [rows][slots][2]: reference (base 2), sum
    float c;                                  // scale * log2(e)
    int D;
    int H, per;                               // query heads; per key/value head
    unsigned magic;                           // for quotients by per
    int W, S;                                 // window (kAll: none), sinks
    int RT;                                   // rows of a block
    int most;                                 // blocks of 16 positions that a block of rows sees at most
    int NO, CT;                               // chunks at most, tiles of 32 positions per chunk
    int NP, CP;                               // the prefix for the rows of all sequences at once: chunks (0: it is not), tiles per chunk
    int rb, rows, ptasks;                     // blocks of these rows, rows of a block, workgroups
    int slots, fold;                          // partial results of a row; the own tasks take the prefix's in and finish the row
};

// ---- 8-bit operands
template <bool BF, int HALF>
__device__ __forceinline__ uint32_t widen2(uint32_t w, float scale) {
    if constexpr (BF)
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HALF != 0));
    else
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, HALF != 0));
}
template <bool BF>
__device__ __forceinline__ u32x4 widen8(uint32_t a, uint32_t b) {
    return u32x4{widen2<BF, 0>(a, 1.f), widen2<BF, 1>(a, 1.f), widen2<BF, 0>(b, 1.f), widen2<BF, 1>(b, 1.f)};
}
// the exponent of a value block's scale, as far as it matters (below 2^-64 e4m3 values vanish in every output)
__device__ __forceinline__ int value_exp(uint32_t b) { return max((int)b - 127, -64); }

// Columns of the output that lane m of 16 and index e stand for: what a lane loads of a position's values.
template <bool Q8, int E>
__device__ __forceinline__ constexpr int column_of(int m, int e) {
    return Q8 && E == 6 ? (e < 4 ? 4 * m + e : 64 + 2 * m + e - 4) : E * m + e;
}

// Offsets of a lane in 16 positions, in bytes.  `same` says nothing about them to the compiler, which would otherwise make
// 64-bit addresses of them outside the loops and add these to every block's base, 2 registers and an instruction a load.
struct Offsets {
    uint32_t a, b;
    template <bool BOTH>
    __device__ __forceinline__ void same() {
        asm("" : "+v"(a));
        if (BOTH) asm("" : "+v"(b));
    }
};

// A lane's part of the keys of 16 positions.
template <bool BF, bool Q8, int D>
struct Keys;
template <bool BF, int D>
struct Keys<BF, false, D> {
    static constexpr int NS = (D + 31) / 32;
    u32x4 w[NS];
    static __device__ __forceinline__ Offsets offsets(uint32_t row, int gq) { return Offsets{2 * row + 16 * gq, 0}; }
    __device__ __forceinline__ void load(const char* b, const Offsets& o, int gq) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            w[s] = u32x4{0, 0, 0, 0};
            if (D % 32 == 0 || gq < 2) w[s] = *(const u32x4*)(b + o.a + 64 * s);
        }
    }
    __device__ __forceinline__ u32x4 get(int s) const { return w[s]; }
    // element of the head that lane gq has first in step s
    static __device__ __forceinline__ constexpr int first(int s, int gq) { return 32 * s + 8 * gq; }
};
// 16 bytes hold two steps' elements: the contraction's order is free, and the queries follow it
template <bool BF, int D>
struct Keys<BF, true, D> {
    static constexpr int NS = (D + 31) / 32;
    uint32_t w[2 * NS];
    static __device__ __forceinline__ Offsets offsets(uint32_t row, int gq) { return Offsets{row + 16 * gq, row + 8 * gq}; }
    __device__ __forceinline__ void load(const char* b, const Offsets& o, int gq) {
#pragma unroll
        for (int m = 0; m < D / 64; ++m) {
            const u32x4 u = *(const u32x4*)(b + o.a + 64 * m);
            w[4 * m] = u[0], w[4 * m + 1] = u[1], w[4 * m + 2] = u[2], w[4 * m + 3] = u[3];
        }
        if constexpr (D % 64 != 0) {
            u32x2 u = {0, 0};
            if (D % 32 == 0 || gq < 2) u = *(const u32x2*)(b + o.b + D / 64 * 64);
            w[2 * NS - 2] = u[0], w[2 * NS - 1] = u[1];
        }
    }
    __device__ __forceinline__ u32x4 get(int s) const { return widen8<BF>(w[2 * s], w[2 * s + 1]); }
    static __device__ __forceinline__ constexpr int first(int s, int gq) {
        return s < D / 64 * 2 ? s / 2 * 64 + 16 * gq + 8 * (s & 1) : 32 * s + 8 * gq;
    }
};

// A lane's D / 16 columns of one position's values, as loaded and as 16-bit words.
template <bool BF, bool Q8, int E>
struct Vals;
template <bool BF, int E>
struct Vals<BF, false, E> {
    uint32_t w[(E + 1) / 2];
    static __device__ __forceinline__ Offsets offsets(uint32_t row, int n) { return Offsets{2 * row + 2 * E * n, 0}; }
    __device__ __forceinline__ void load(const char* p, const Offsets& f) {
        p += f.a;
        if constexpr (E == 8) {
            const u32x4 u = *(const u32x4*)p;
            w[0] = u[0], w[1] = u[1], w[2] = u[2], w[3] = u[3];
        } else if constexpr (E == 6) {
            const uint32_t* q = (const uint32_t*)p;                 // 12 bytes, 4-byte aligned
            w[0] = q[0], w[1] = q[1], w[2] = q[2];
        } else if constexpr (E == 4) {
            const u32x2 u = *(const u32x2*)p;
            w[0] = u[0], w[1] = u[1];
        } else if constexpr (E == 2) {
            w[0] = *(const uint32_t*)p;
        } else {
            w[0] = *(const uint16_t*)p;
        }
    }
    __device__ __forceinline__ void wide(uint32_t (&o)[(E + 1) / 2], float) const {
#pragma unroll
        for (int i = 0; i < (E + 1) / 2; ++i) o[i] = w[i];
    }
};
template <bool BF, int E>
struct Vals<BF, true, E> {
    uint32_t w[(E + 3) / 4];
    static __device__ __forceinline__ Offsets offsets(uint32_t row, int n) { return Offsets{row + (E == 6 ? 4 : E) * n, row + 2 * n}; }
    __device__ __forceinline__ void load(const char* p, const Offsets& f) {
        if constexpr (E == 8) {
            const u32x2 u = *(const u32x2*)(p + f.a);
            w[0] = u[0], w[1] = u[1];
        } else if constexpr (E == 6) {
            w[0] = *(const uint32_t*)(p + f.a);
            w[1] = *(const uint16_t*)(p + f.b + 64);
        } else if constexpr (E == 4) {
            w[0] = *(const uint32_t*)(p + f.a);
        } else if constexpr (E == 2) {
            w[0] = *(const uint16_t*)(p + f.a);
        } else {
            w[0] = *(const uint8_t*)(p + f.a);
        }
    }
    __device__ __forceinline__ void wide(uint32_t (&o)[(E + 1) / 2], float scale) const {
#pragma unroll
        for (int i = 0; i < (E + 1) / 2; ++i) o[i] = i & 1 ? widen2<BF, 1>(w[i / 2], scale) : widen2<BF, 0>(w[i / 2], scale);
    }
};

// ---- what there is to do

// A sequence as the device finds it: its tokens in this step and the own position of the first of them.
struct Seq {
    int start, n, first;
};
__device__ __forceinline__ Seq seq_at(const PagedBatch& b, int s) {
    const int len = b.seq_len[s];
    int start = b.q_start ? b.q_start[s] : s;
    const int64_t end = b.q_start ? b.q_start[s + 1] : s + 1;
    start = min(max(start, 0), b.T);
    const int n = (int)min((int64_t)max(end, (int64_t)start), (int64_t)b.T) - start;
    const int64_t first = (int64_t)len - (end - start);
    return Seq{start, len < 0 ? 0 : n, (int)min(max(first, (int64_t)-kAll), (int64_t)kAll)};
}

// The blocks of 16 positions that the rows at positions lo .. hi see, numbered through the prefix's blocks and the
// sequence's own: the first `head` of them, then those from `from` on, n in all.
struct Seen {
    int head, from, n;
};
__device__ __forceinline__ int block_of(int j, int P, int PB) { return j < P ? j >> 4 : PB + ((j - P) >> 4); }
__device__ __forceinline__ Seen seen(const PagedBatch& b, const WinArgs& a, int cap, int lo, int hi) {
    const int P = b.prefix, PB = (P + 15) >> 4;
    hi = min(hi, P + cap - 1);                // (a table spans 2^28 positions at most, a prefix as many)
    lo = max(lo, P);
    if (hi < P) return Seen{0, 0, 0};         // (behind the table's end lo may pass hi)
    const int to = block_of(hi, P, PB) + 1;
    if (a.NP) return Seen{0, PB, to - PB};
    const int from = block_of(min(max(lo - a.W + 1, 0), hi), P, PB);
    const int head = a.S > 0 ? min(block_of(min(a.S - 1, hi), P, PB) + 1, from) : 0;
    return Seen{head, from, head + to - from};
}
__device__ __forceinline__ int chunks_of(int n, int CT) { return max(1, ((n + 1) / 2 + CT - 1) / CT); }

struct Task {
    const int32_t* table;
    int b0, b1;                               // its part of the list of blocks (b1 is the list's end or even)
    int g, tok0, lead, rows;                  // row r of the block: row lead + r of the tokens from tok0 on (r < rows, lead < per)
    int pos0;                                 // position of token tok0; kNowhere: all rows stand at hi
    int lo, hi;                               // of the first and last row (lo -1: some rows see nothing)
    int low;                                  // positions above it (or below the sinks) are seen by some row
    Seen s;
    int split, splits;                        // where the partial results go; 1: the results are whole

    __device__ __forceinline__ int offset(int r, const WinArgs& a) const { return (int)unit_div((unsigned)(lead + r), a.magic); }
    __device__ __forceinline__ int token(int r, const WinArgs& a) const { return tok0 + offset(r, a); }
    __device__ __forceinline__ int head(int r, const WinArgs& a) const { return g * a.per + lead + r - a.per * offset(r, a); }
    __device__ __forceinline__ int position(int r, const WinArgs& a) const { return pos0 == kNowhere ? hi : pos0 + offset(r, a); }
    // row r0 of the tokens from t0 on is the block's first
    __device__ __forceinline__ void begin(int t0, int r0, const WinArgs& a) {
        const int q = (int)((unsigned)r0 / (unsigned)a.per);
        tok0 = t0 + q;
        lead = r0 - q * a.per;
    }
};

// 16 positions of a task's list: the first one and how many there are (0: behind the list's end)
struct Blk {
    int j0, nv;
};
__device__ __forceinline__ Blk look(const PagedBatch& b, const Task& t, int i) {
    if (i >= t.b1) return Blk{kAll, 0};
    const int P = b.prefix, PB = (P + 15) >> 4, vb = i < t.s.head ? i : i - t.s.head + t.s.from;
    return vb < PB ? Blk{16 * vb, min(16, P - 16 * vb)} : Blk{P + 16 * (vb - PB), 16};
}
// The list's blocks that all rows from position lo to hi see whole: from w0 to w1, but for one (the prefix's last, if it
// is not full).
struct Inner {
    int w0, w1, pb;
    __device__ __forceinline__ bool holds(int i, int n) const { return i >= w0 && i + n <= w1 && (pb < i || pb >= i + n); }
};
__device__ __forceinline__ Inner inner(const PagedBatch& b, const WinArgs& a, const Task& t, int lo, int hi) {
    const int P = b.prefix, PB = (P + 15) >> 4, shift = t.s.head - t.s.from, x = max(hi - a.W + 1, 0);
    const int vb = block_of(x, P, PB), j0 = vb < PB ? 16 * vb : P + 16 * (vb - PB);
    return Inner{max(t.s.head, vb + (j0 < x) + shift), min(t.b1, block_of(lo + 1, P, PB) + shift), P & 15 ? PB - 1 + shift : -1};
}
// Where 64 blocks of the list are, one in each lane: offsets of the head's keys and values in bytes, and in one word the
// scale bytes (keys', values' << 8), kBad (the page is none of the cache's, or a scale is NaN) and kPart (not in `whole`).
constexpr int kBad = 1 << 16, kPart = 1 << 17;
struct Where {
    int64_t k, v;
    int info;
};
template <bool Q8>
__device__ __forceinline__ Where where(const PagedCache& c, const PageScales& sc, const PagedBatch& b, const Task& t, const Inner& whole, int i) {
    const int PB = (b.prefix + 15) >> 4, vb = i < t.s.head ? i : i - t.s.head + t.s.from;
    const bool pre = vb < PB, in = i < t.b1;
    const unsigned o = pre ? vb : vb - PB, at = unit_div(o, c.magic);
    const int unit = in ? (int)(o - at * c.unit) : 0;
    const bool held = in && (pre || at < (unsigned)b.width);
    const int raw = *(held ? (pre ? b.prefix_table : t.table) + at : b.seq_len);
    const bool ok = held && (unsigned)raw < (unsigned)c.n_pages;
    const int id = ok ? raw : 0;              // (behind the list's end any page will do)
    int info = (in && !ok ? kBad : 0) | (whole.holds(i, 1) ? 0 : kPart);
    if (Q8) {
        const int kb = sc.k[id * sc.kp + t.g * sc.kh + unit], vb8 = sc.v[id * sc.vp + t.g * sc.vh + unit];
        info |= kb | vb8 << 8 | (in && (kb == 255 || vb8 == 255) ? kBad : 0);
    }
    constexpr int size = Q8 ? 1 : 2;
    return Where{(id * c.kp + t.g * c.kh + (int64_t)(unit * kPageUnit) * c.ks) * size,
                 (id * c.vp + t.g * c.vh + (int64_t)(unit * kPageUnit) * c.vs) * size, info};
}
__device__ __forceinline__ int64_t lane_of(int64_t x, int j) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, j));
}
__device__ __forceinline__ Where lane_of(const Where& x, int j) {
    return Where{lane_of(x.k, j), lane_of(x.v, j), __builtin_amdgcn_readlane(x.info, j)};
}
// none of the rows from position lo to hi sees any of it
__device__ __forceinline__ bool hidden(const Blk& x, int lo, int hi, const WinArgs& a) {
    return x.nv == 0 || x.j0 > hi || (x.j0 + 15 <= lo - a.W && x.j0 >= a.S);
}

// The tasks, numbered sequence by sequence: (row block from the last on, chunk, key/value head).  How many there are
// only the device knows; whoever asks for rising numbers walks the sequences once.
// the lane's value added to those of all lanes below (no sum passes 2^32 - 1)
__device__ __forceinline__ unsigned sum_upto(unsigned v) {
    const auto add = [](unsigned x, unsigned y) { return x + y < x ? ~0u : x + y; };
    v = add(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true));         // the lane 1, 2, 4, 8 below, in rows of 16
    v = add(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true));
    v = add(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true));
    v = add(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true));
    v = add(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));        // a row's last lane to the next row
    v = add(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));        // lane 31 to the upper half
    return v;
}

struct Tasks {
    int base = 0;                             // the sequences before it hold `done` tasks
    unsigned done = 0, last = ~0u;            // the last 64 sequences' tasks end there

    template <int RT>
    __device__ bool find(const PagedCache& c, const PagedBatch& b, const WinArgs& a, unsigned task, Task& t) {
        // the same in all lanes, which the compiler does not see
        task = __builtin_amdgcn_readfirstlane(task), last = __builtin_amdgcn_readfirstlane(last);
        done = __builtin_amdgcn_readfirstlane(done), base = __builtin_amdgcn_readfirstlane(base);
        if (task >= last) return false;       // (without asking for the lengths again)
        const int cap = b.width * c.unit * kPageUnit;
        const int lane = threadIdx.x & 63, PB = (b.prefix + 15) >> 4;
        for (; base < b.B; base += 64) {
            Seq q{0, 0, 0};
            if (base + lane < b.B) q = seq_at(b, base + lane);
            const int nb = (q.n * a.per + RT - 1) / RT;             // (rows are below 2^26)
            // chunks of its blocks of rows at most
            int most = (a.NP ? 0 : PB) + ((min(max(q.first + q.n, 0), cap) + 15) >> 4);
            most = min(most, a.most);
            const int nc = a.NO == 1 ? 1 : chunks_of(most, a.CT);
            const unsigned mine = (unsigned)nb * nc * c.G;          // (below 2^31: chunks go down as blocks go up)
            const unsigned upto = sum_upto(mine);
            const unsigned long long over = __ballot(upto > task - done);
            const unsigned all = (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
            if (b.B - base <= 64) last = done + all < done ? ~0u : done + all;
            if (!over) {
                done = done + all < done ? ~0u : done + all;
                continue;
            }
            const int hit = __ffsll(over) - 1, sq = base + hit;
            const unsigned rest = (unsigned)__builtin_amdgcn_readlane((int)(task - done - (upto - mine)), hit);
            const int n = __builtin_amdgcn_readlane(q.n, hit), first = __builtin_amdgcn_readlane(q.first, hit);
            const int ncs = __builtin_amdgcn_readlane(nc, hit), blocks = __builtin_amdgcn_readlane(nb, hit);
            const unsigned rc = rest / (unsigned)c.G, above = ncs == 1 ? rc : rc / (unsigned)ncs;
            if (above >= (unsigned)blocks) return false;            // (only where first tokens do not ascend)
            t.g = (int)(rest - rc * c.G);
            const int ch = (int)(rc - above * ncs), rb = blocks - 1 - (int)above;
            t.table = b.table + sq * b.table_stride;
            t.begin(__builtin_amdgcn_readlane(q.start, hit), rb * RT, a);
            t.pos0 = b.prefix + first + (t.tok0 - __builtin_amdgcn_readlane(q.start, hit));
            t.rows = min(RT, n * a.per - rb * RT);
            t.lo = t.pos0;
            t.hi = t.position(t.rows - 1, a);
            t.s = seen(b, a, cap, t.lo, t.hi);
            t.b0 = 0, t.b1 = t.s.n;
            t.splits = 1;
            if (a.NO > 1) {
                const int n_chunks = chunks_of(t.s.n, a.CT), tiles = (t.s.n + 1) / 2, each = (tiles + n_chunks - 1) / n_chunks;
                t.splits = n_chunks;
                t.b0 = 2 * ch * each;
                t.b1 = min(t.s.n, t.b0 + 2 * each);
            }
            t.split = ch;
            if (!a.fold) t.splits += a.NP, t.split += a.NP;
            t.low = max(t.lo, b.prefix) - a.W;
            if (t.lo < b.prefix) t.lo = -1;
            return true;
        }
        return false;
    }
};

// the prefix's tasks: the blocks of rows of one chunk follow each other on one XCD (workgroups go round the 8 XCDs)
__device__ __forceinline__ bool prefix_task(const PagedCache& c, const PagedBatch& b, const WinArgs& a, Task& t) {
    const int j = blockIdx.x / 8, pair = j / a.rb * 8 + blockIdx.x % 8, rb = j % a.rb, PB = (b.prefix + 15) >> 4;
    if (pair >= c.G * a.NP) return false;
    t.table = nullptr;
    t.g = pair % c.G;
    t.split = pair / c.G;
    t.splits = a.NP + 1;
    t.s = Seen{0, 0, PB};
    t.b0 = 2 * t.split * a.CP;
    t.b1 = min(PB, t.b0 + 2 * a.CP);
    t.begin(0, rb * a.rows, a);
    t.rows = min(a.rows, b.T * a.per - rb * a.rows);
    t.pos0 = kNowhere;
    t.lo = t.hi = b.prefix - 1;
    t.low = t.lo - a.W;
    return true;
}

// ---- a wave's rows

// NR tiles of 16 rows: output (transposed, lane = row), reference of the exponent and the lane's share of the sum.
template <bool BF, bool Q8, int D, int NR>
struct Rows {
    static constexpr int E = D / 16;
    static constexpr float high = BF ? 0x1p-28f : 0x1p15f;          // 2^kTop
    static constexpr bool JOINT = Q8 && !BF;  // the weights hold the values' scale
    f32x4 o[NR][E];
    float ref[NR], sum[NR];                   // weights are 2^(c * score (+ e) - ref)
    int hi[NR];                               // the lane's rows' positions; -1: they see nothing

    __device__ __forceinline__ void start(const Task& t, int P, const WinArgs& a, int row0) {
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            const int i = row0 + rt * 16 + (threadIdx.x & 15), p = t.position(i, a);
            hi[rt] = i < t.rows && (p >= P || t.pos0 == kNowhere) ? p : -1;
            ref[rt] = kNone, sum[rt] = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) o[rt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    static __device__ __forceinline__ bool sees(int j, int hi, const WinArgs& a) { return j <= hi && (j > hi - a.W || j < a.S); }
    // the scores of what the lane's row does not see in a block, where rows from position `lo` to `top` are the wave's
    __device__ __forceinline__ void hide(int rt, const Blk& x, f32x4& s, int lo, int top, const WinArgs& a) const {
        const int first = x.j0 + 4 * ((threadIdx.x & 63) >> 4);     // the lane's positions are first + i
        if (x.j0 + 15 > lo || x.nv < 16) {                          // some row is before the block's end
            const int n = min(hi[rt], x.j0 + x.nv - 1) - first;
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = i <= n ? s[i] : -INFINITY;
        }
        if (x.j0 <= top - a.W && x.j0 + 15 >= a.S) {                // some row's window begins behind the block's first
            const int n = hi[rt] - a.W - first, m = a.S - first;
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = i > n || i < m ? s[i] : -INFINITY;
        }
    }
    struct Weights {
        float x[2][4], part, sum;
        template <bool CAP = false>
        __device__ __forceinline__ void take(const f32x4 (&s)[2], float ref, const float (&ck)[2], const float (&ev)[2]) {
            float p[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float z = JOINT ? ev[h] - ref : -ref;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[h][i] = __builtin_amdgcn_exp2f(fmaf(s[h][i], ck[h], z));
                    if (CAP) x[h][i] = x[h][i] > high ? high : x[h][i];
                }
                p[h] = (x[h][0] + x[h][1]) + (x[h][2] + x[h][3]);
            }
            part = p[0] + p[1];
            sum = JOINT ? fmaf(p[0], __builtin_amdgcn_exp2f(-ev[0]), p[1] * __builtin_amdgcn_exp2f(-ev[1])) : part;
        }
        __device__ __forceinline__ u32x4 packed() const {
            return u32x4{pack2<BF>(x[0][0], x[0][1]), pack2<BF>(x[0][2], x[0][3]), pack2<BF>(x[1][0], x[1][1]), pack2<BF>(x[1][2], x[1][3])};
        }
    };
    // A new reference for the lane's row if some weight of its is high: the largest score so far gets the weight
    // 2^(kTop - kRoom).  The tile's other rows keep theirs, since a row's roundings follow its own scores alone.  Where fp32
    // no longer holds a difference of a reference and a score, the reference is rounded down, so that the largest score's
    // weight is not lost, and weights behind 2^kTop are cut off there: scores that near each other count alike.
    __device__ __forceinline__ void raise(int rt, const f32x4 (&s)[2], float part, const float (&ck)[2], const float (&ev)[2]) {
        part = fmaxf(part, __shfl_xor(part, 16));
        part = fmaxf(part, __shfl_xor(part, 32));
        float mx = -INFINITY;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            mx = fmaxf(mx, fmaf(fmaxf(fmaxf(s[h][0], s[h][1]), fmaxf(s[h][2], s[h][3])), ck[h], JOINT ? ev[h] : 0.f));
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        mx += kRoom - kTop<BF>;
        if (fabsf(mx) > 0x1p18f) mx *= mx > 0.f ? 1.f - 0x1p-21f : 1.f + 0x1p-21f;
        const float now = part > high ? fmaxf(ref[rt], mx) : ref[rt], al = __builtin_amdgcn_exp2f(ref[rt] - now);
        ref[rt] = now;
        sum[rt] *= al;
#pragma unroll
        for (int e = 0; e < E; ++e) o[rt][e] *= al;
    }
    // The weights of 32 positions as operands, and their sums, in two steps.  No maximum is taken: a lane's sum of 8
    // tells when some weight may leave its range, and then, which is rare after the first tiles, the reference is raised.
    __device__ __forceinline__ void take(const f32x4 (&s)[NR][2], Weights (&w)[NR], const float (&ck)[2], const float (&ev)[2]) const {
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) w[rt].take(s[rt], ref[rt], ck, ev);
    }
    __device__ __forceinline__ void settle(const f32x4 (&s)[NR][2], Weights (&w)[NR], u32x4 (&p)[NR], const float (&ck)[2], const float (&ev)[2]) {
        bool any = false;
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) any |= w[rt].part > high;
        if (__builtin_expect(__any(any), 0))
#pragma unroll
            for (int rt = 0; rt < NR; ++rt)
                if (__any(w[rt].part > high)) {
                    raise(rt, s[rt], w[rt].part, ck, ev);
                    w[rt].template take<true>(s[rt], ref[rt], ck, ev);
                }
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) sum[rt] += w[rt].sum, p[rt] = w[rt].packed();
    }
    __device__ __forceinline__ void weights(const f32x4 (&s)[NR][2], u32x4 (&p)[NR], const float (&ck)[2], const float (&ev)[2]) {
        Weights w[NR];
        take(s, w, ck, ev);
        settle(s, w, p, ck, ev);
    }
    // What values that are not finite contribute to the rows that see them, of N blocks: the products' operand has zeros in
    // their places, since a zero weight would not keep them out of the other rows.
    template <int N>
    __device__ __forceinline__ void add_odd(const PagedCache& c, const PageScales& sc, const PagedBatch& b, const WinArgs& a, const Task& t, int at) {
        const int gq = (threadIdx.x & 63) >> 4;
        for (int i = 0; i < 16 * N; ++i) {
            const Blk y = look(b, t, at + (i >> 4));
            const Where w = where<Q8>(c, sc, b, t, Inner{}, at + (i >> 4));
            if ((i & 15) >= y.nv || (w.info & kBad)) continue;
            const int j = y.j0 + (i & 15);
            const char* const from = (const char*)c.v + w.v + (int64_t)(i & 15) * c.vs * (Q8 ? 1 : 2);
            const float scale = Q8 && BF ? ldexpf(1.f, value_exp(w.info >> 8 & 255)) : 1.f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int col = column_of<Q8, E>(4 * gq + k, e);
                    float v;
                    bool odd;
                    if (Q8) {
                        v = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)from)[col], 0) * scale;
                        odd = !(fabsf(v) < INFINITY) || (BF && !finite16<true>(pack2<true>(v, v)));
                    } else {
                        const uint16_t u = ((const uint16_t*)from)[col];
                        odd = !finite16<BF>(u);
                        v = BF ? __uint_as_float((uint32_t)u << 16) : h2f(u);
                    }
                    if (!odd) continue;
#pragma unroll
                    for (int rt = 0; rt < NR; ++rt)
                        if (sees(j, hi[rt], a)) o[rt][e][k] += v;
                }
        }
    }
    __device__ __forceinline__ void finish(int end) {
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
            sum[rt] += __shfl_xor(sum[rt], 16);
            sum[rt] += __shfl_xor(sum[rt], 32);
            if (hi[rt] >= end) sum[rt] = NAN;                       // it sees positions that the table does not hold
        }
    }
};

// The keys and the values of 16 positions in a wave's registers.
template <bool BF, bool Q8, int D>
struct Loader {
    Offsets k, v;
    __device__ __forceinline__ explicit Loader(const PagedCache& c) {
        const int lane = threadIdx.x & 63;
        k = Keys<BF, Q8, D>::offsets((lane & 15) * (uint32_t)c.ks, lane >> 4);
        v = Vals<BF, Q8, D / 16>::offsets(4 * (lane >> 4) * (uint32_t)c.vs, lane & 15);
    }
    __device__ __forceinline__ void keys(Keys<BF, Q8, D>& to, const PagedCache& c, const Where& x) {
        k.template same<Q8 && D % 64 != 0>();
        to.load((const char*)c.k + x.k, k, (threadIdx.x & 63) >> 4);
    }
    __device__ __forceinline__ void values(Vals<BF, Q8, D / 16> (&to)[4], const PagedCache& c, const Where& x) {
        v.template same<Q8 && D == 96>();
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i].load((const char*)c.v + x.v + (int64_t)i * (Q8 ? c.vs : 2 * c.vs), v);
    }
};
// What a block's scale bytes say: the scores' factor (neither 0 nor infinite, which times the -infinity of a hidden position
// or a score of 0 were NaN) and the values' exponent.
template <bool Q8>
__device__ __forceinline__ void scales_of(const WinArgs& a, int info, float* ck, float* ev) {
    *ck = Q8 ? __builtin_amdgcn_fmed3f(ldexpf(a.c, (info & 255) - 127), 0x1p-126f, 0x1p127f) : a.c;
    *ev = Q8 ? (float)value_exp(info >> 8 & 255) : 0.f;
}

template <bool BF, bool Q8, int D, int NR>
__device__ __forceinline__ void load_q(const WinArgs& a, const Task& t, int row0, u32x4 (&q)[NR][(D + 31) / 32]) {
    const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
        const int i = row0 + rt * 16 + n, tok = t.token(i, a), h = t.head(i, a);
#pragma unroll
        for (int s = 0; s < (D + 31) / 32; ++s) {
            const int d = Keys<BF, Q8, D>::first(s, gq);
            q[rt][s] = u32x4{0, 0, 0, 0};
            if (i < t.rows && d < D) q[rt][s] = *(const u32x4*)(a.q + (int64_t)tok * a.qt + h * a.qh + d);
        }
    }
}

// Few rows (16): the wave takes the tiles at, at + step, ... of the task; the next tile's keys and values come into
// the registers of this one's as soon as a product has read them.
template <bool BF, bool Q8, int D>
__device__ __forceinline__ void walk(const PagedCache& c, const PageScales& sc, const PagedBatch& b, const WinArgs& a,
                                     const Task& t, int at, int step, Rows<BF, Q8, D, 1>& r) {
    constexpr int E = D / 16, NS = (D + 31) / 32, EW = (E + 1) / 2;
    const int gq = (threadIdx.x & 63) >> 4;
    r.start(t, b.prefix, a, 0);
    if (at >= t.b1) return;
    u32x4 q[1][NS];                           // (on their way while the pages are looked up)
    load_q<BF, Q8, D, 1>(a, t, 0, q);
    Keys<BF, Q8, D> xk[2];
    Vals<BF, Q8, E> xv[2][4];
    // lane 2 j + h: block h of the wave's tile j of 32
    const int lane = threadIdx.x & 63;
    const int at0 = at + (lane & 1);
    const Inner in = inner(b, a, t, t.lo, t.hi);
    auto find = [&](int j) { return where<Q8>(c, sc, b, t, in, at0 + step * (j + (lane >> 1))); };
    Loader<BF, Q8, D> load(c);
    Where run = find(0);
    int turn = 0, info[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const Where x = lane_of(run, h);
        load.keys(xk[h], c, x);
        load.values(xv[h], c, x);
        info[h] = x.info;
    }
    const bool several = t.position(0, a) != t.hi;
    for (int known = 31;; known += 32) {      // the last tile whose place the lanes hold
    for (; at < t.b1 && turn < known; at += step, ++turn) {
        float ck[2], ev[2];
        bool bad[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            scales_of<Q8>(a, info[h], &ck[h], &ev[h]);
            bad[h] = info[h] & kBad;
        }
        const bool more = at + step < t.b1;
        Where nx[2];
        f32x4 s[1][2] = {{{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}};
#pragma unroll
        for (int k = 0; k < NS; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) s[0][h] = mfma16<BF>(xk[h].get(k), q[0][k], s[0][h]);
        if (more)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                nx[h] = lane_of(run, (2 * turn + 2 + h) & 63);
                load.keys(xk[h], c, nx[h]);
            }
        const bool part = (info[0] | info[1]) & (kBad | kPart);
        Blk x[2];
        if (part)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                x[h] = look(b, t, at + h);
                if (bad[h]) s[0][h] = f32x4{NAN, NAN, NAN, NAN};
                r.hide(0, x[h], s[0][h], t.lo, t.hi, a);
            }
        u32x4 w[1];
        r.weights(s, w, ck, ev);
        uint32_t v[8][EW];
#pragma unroll
        for (int i = 0; i < 8; ++i) xv[i >> 2][i & 3].wide(v[i], Q8 && BF ? ldexpf(1.f, (int)ev[i >> 2]) : 1.f);
        if (more)
#pragma unroll
            for (int h = 0; h < 2; ++h) load.values(xv[h], c, nx[h]), info[h] = nx[h].info;
        bool fine = true;
        if (part) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int k = 4 * gq + (i & 3), j = x[i >> 2].j0 + k;
                // values that no row sees do not reach the product, whatever they hold
                const bool some = k < x[i >> 2].nv && j <= t.hi && (j > t.low || j < a.S) && !bad[i >> 2];
#pragma unroll
                for (int m = 0; m < EW; ++m) {
                    if (!some) v[i][m] = 0;
                    if (several) v[i][m] = sane<BF>(v[i][m], &fine);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const unsigned sel = (e & 1) ? 0x07060302u : 0x05040100u;
            u32x4 f;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = __builtin_amdgcn_perm(v[2 * j + 1][e / 2], v[2 * j][e / 2], sel);
            r.o[0][e] = mfma16<BF>(f, w[0], r.o[0][e]);
        }
        if (part && __any(!fine)) r.template add_odd<2>(c, sc, b, a, t, at);
    }
    if (at >= t.b1) return;
    run = find(turn + 1);                     // 32 more, outside the loop: a branch in it costs copies of the accumulators
    }
}

// Many rows: the four waves share the positions and each has its own 16 * NR rows, Q in registers.  A stage of 64
// positions comes to LDS in operand order and in 16 bits (a wave brings 16 of them, in registers while the stage before is
// worked on) and every wave reads all of it.
constexpr int kBlocks = 4;                    // of 16 positions in a stage, one for each wave

template <int D>
struct StageLds {
    static constexpr int E = D / 16, NS = (D + 31) / 32;
    u32x4 k[kBlocks][NS][64];
    u32x4 v[E][kBlocks / 2][64];              // a column of each lane's, 32 positions each
    float ck[kBlocks], ev[kBlocks];           // 8-bit pages: the scores' factors and the values' exponents
};
// Blocks of a task whose values that are not finite have been left out, as the wave that brought them wrote them down: the
// first kOdd of them, and where more lie.  Only what some row of the task does not see whole is looked at, about 6 blocks a
// wave and all of a prefix where a sequence is shorter than its tokens.
constexpr int kOdd = 8;
struct OddLds {
    alignas(16) int n[kBlocks];
    int at[kBlocks][kOdd], from[kBlocks], to[kBlocks];
};

template <bool BF, bool Q8, int D, int NR>
__device__ __forceinline__ void walk_wide(const PagedCache& c, const PageScales& sc, const PagedBatch& b, const WinArgs& a,
                                          const Task& t, StageLds<D> (&l)[2], OddLds& odd, Rows<BF, Q8, D, NR>& r) {
    constexpr int E = D / 16, NS = (D + 31) / 32, EW = (E + 1) / 2;
    const int lane = threadIdx.x & 63, gq = lane >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = w * NR * 16;             // the wave's rows of the block
    r.start(t, b.prefix, a, row0);
    if (t.b0 >= t.b1) return;
    const int last = min(row0 + 16 * NR, t.rows) - 1;
    const bool idle = last < row0;
    // positions of the wave's first and last row
    const int hi = idle ? -1 : t.position(last, a), first = idle ? -1 : t.position(row0, a);
    const int lo = first < b.prefix && t.pos0 != kNowhere ? -1 : first;
    const Inner in = inner(b, a, t, lo, hi);
    Keys<BF, Q8, D> xk;
    Vals<BF, Q8, E> xv[4];
    // lane j: the block that the wave brings of stage j of 64
    Where run;
    int turn = 0, info = 0;                   // turn: of the stage that is worked on
    auto find = [&](int j) { run = where<Q8>(c, sc, b, t, inner(b, a, t, t.lo, t.hi), t.b0 + kBlocks * (j + lane) + w); };
    Loader<BF, Q8, D> load(c);
    auto bring = [&](int j) {
        const Where x = lane_of(run, j & 63);
        load.keys(xk, c, x);
        load.values(xv, c, x);
        info = x.info;
    };
    auto write_v = [&](StageLds<D>& s, const uint32_t (&v)[4][EW]) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const unsigned sel = (e & 1) ? 0x07060302u : 0x05040100u;
            ((u32x2*)&s.v[e][w >> 1][lane])[w & 1] = u32x2{__builtin_amdgcn_perm(v[1][e / 2], v[0][e / 2], sel),
                                                          __builtin_amdgcn_perm(v[3][e / 2], v[2][e / 2], sel)};
        }
    };
    auto put = [&](int at, StageLds<D>& s) {
        float ck, ev;
        scales_of<Q8>(a, info, &ck, &ev);
        const bool bad = info & kBad;
        const float scale = Q8 && BF ? ldexpf(1.f, (int)ev) : 1.f;
        uint32_t v[4][EW];
#pragma unroll
        for (int i = 0; i < 4; ++i) xv[i].wide(v[i], scale);
#pragma unroll
        for (int k = 0; k < NS; ++k) s.k[w][k][lane] = xk.get(k);
        if (info & (kBad | kPart)) {          // some row does not see some of it: a zero weight keeps no NaN out
            const Blk y = look(b, t, at);
            bool fine = true;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = 4 * gq + i, j = y.j0 + k;
                const bool some = k < y.nv && j <= t.hi && (j > t.low || j < a.S) && !bad;
#pragma unroll
                for (int m = 0; m < EW; ++m) v[i][m] = some ? sane<BF>(v[i][m], &fine) : 0;
            }
            if (__any(!fine) && lane == 0) {
                const int n = odd.n[w]++;
                if (n < kOdd) odd.at[w][n] = at;
                if (n == kOdd) odd.from[w] = at;
                odd.to[w] = at;
            }
            if (bad)                          // its scores are NaN
#pragma unroll
                for (int k = 0; k < NS; ++k) s.k[w][k][lane] = u32x4{~0u, ~0u, ~0u, ~0u};
        }
        write_v(s, v);
        if (Q8 && lane == 0) s.ck[w] = bad ? 1.f : ck, s.ev[w] = bad ? 0.f : ev;
    };
    int at = t.b0;
    if (lane == 0) odd.n[w] = 0;              // (the wave's own until the first stage's barrier)
    // (the queries first: loads come back in order, and one that is still out when the loop begins would be waited for in
    // every stage)
    u32x4 q[NR][NS];
    load_q<BF, Q8, D, NR>(a, t, row0, q);
    find(0);
    bring(0);
    put(at + w, l[0]);
    if (at + kBlocks < t.b1) bring(1);
    // the next stage to LDS, the one after that on its way
    auto next = [&]() {
        if (at + kBlocks < t.b1) {
            put(at + kBlocks + w, l[(turn + 1) & 1]);
            if (at + 2 * kBlocks < t.b1) bring(turn + 2);
        }
    };
    // Operands come from LDS well before their products, past other work: left to itself the compiler reads each into the
    // same registers right before its products and waits for it there.
    u32x4 kf[NS][2], vf[E];
    auto read_k = [&](const StageLds<D>& st, int h) {
#pragma unroll
        for (int k = 0; k < NS; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) kf[k][i] = st.k[2 * h + i][k][lane];
        __builtin_amdgcn_sched_barrier(0);
    };
    auto read_v = [&](const StageLds<D>& st, int h) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < E; ++e) vf[e] = st.v[e][h][lane];
        __builtin_amdgcn_sched_barrier(0);
    };
    f32x4 s[NR][2];
    u32x4 wt[NR];
    auto scores = [&]() {
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) s[rt][0] = s[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NS; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int rt = 0; rt < NR; ++rt) s[rt][i] = mfma16<BF>(kf[k][i], q[rt][k], s[rt][i]);
    };
    float ck[2] = {a.c, a.c}, ev[2] = {0.f, 0.f};
    auto factors = [&](const StageLds<D>& st, int h) {
        if (Q8) ck[0] = st.ck[2 * h], ck[1] = st.ck[2 * h + 1], ev[0] = st.ev[2 * h], ev[1] = st.ev[2 * h + 1];
    };
    auto add = [&]() {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) r.o[rt][e] = mfma16<BF>(vf[e], wt[rt], r.o[rt][e]);
    };
    for (int known = 62;;) {
        // the places of 64 more stages, outside the loops around products: a branch in these costs copies of the
        // accumulators
        if (turn == known) find(turn + 2), known += 64;
        // stages that all rows of the wave see (waves of a workgroup may leave at different ones: both loops have one
        // barrier a stage)
        const int to = !in.holds(at, kBlocks) ? INT32_MIN : in.pb < at ? in.w1 - kBlocks : min(in.w1, in.pb) - kBlocks;
        while (at <= to && turn < known) {
            const StageLds<D>& st = l[turn & 1];
            __syncthreads();                  // the stage is there, and nobody reads the one before
            read_k(st, 0);
            __builtin_amdgcn_s_setprio(1);    // (everybody waits for it: 80 -> 78 us for 1000 rows over 8007 positions)
            next();
            __builtin_amdgcn_s_setprio(0);
            factors(st, 0);
            scores();
            read_v(st, 0);
            r.weights(s, wt, ck, ev);
            factors(st, 1);
            read_k(st, 1);
            add();
            scores();
            read_v(st, 1);
            r.weights(s, wt, ck, ev);
            add();
            ++turn, at += kBlocks;
        }
        if (at >= t.b1) break;
        if (turn == known) continue;
        const StageLds<D>& st = l[turn & 1];
        __syncthreads();
        next();
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            const Blk x[2] = {look(b, t, at + 2 * h), look(b, t, at + 2 * h + 1)};
            if (hidden(x[0], lo, hi, a) && hidden(x[1], lo, hi, a)) continue;
            read_k(st, h);
            scores();
#pragma unroll
            for (int rt = 0; rt < NR; ++rt)
#pragma unroll
                for (int i = 0; i < 2; ++i) r.hide(rt, x[i], s[rt][i], lo, hi, a);
            read_v(st, h);
            factors(st, h);
            r.weights(s, wt, ck, ev);
            add();
        }
        ++turn, at += kBlocks;
        if (at >= t.b1) break;
    }
    // What was left out of a stage is missing to every row that sees it, also in waves that see all of the stage: here, behind
    // the last stage's barrier, for both loops.
    const u32x4 any = *(const u32x4*)odd.n;
    if (!__builtin_amdgcn_readfirstlane(any[0] | any[1] | any[2] | any[3])) return;
#pragma unroll 1
    for (int i = 0; i < kBlocks; ++i) {
        const int n = __builtin_amdgcn_readfirstlane(odd.n[i]);
#pragma unroll 1
        for (int k = 0; k < min(n, kOdd); ++k) r.template add_odd<1>(c, sc, b, a, t, __builtin_amdgcn_readfirstlane(odd.at[i][k]));
        if (n > kOdd)
#pragma unroll 1
            for (int k = odd.from[i]; k <= odd.to[i]; k += kBlocks) r.template add_odd<1>(c, sc, b, a, t, k);
    }
}

// the output of one row, columns D / 16 at a time in the lanes' order
template <bool BF, bool Q8, int E>
__device__ __forceinline__ void put_out(uint16_t* o, int m, const float (&v)[E]) {
    if constexpr (E == 1) {
        o[m] = (uint16_t)pack2<BF>(v[0], 0.f);
    } else {
#pragma unroll
        for (int e = 0; e < E; e += 2) *(uint32_t*)(o + column_of<Q8, E>(m, e)) = pack2<BF>(v[e], v[e + 1]);
    }
}

// The prefix's partial results of a row are taken in: N of its columns v (whose first is `p` in a partial result), its
// reference and sum.  Several at a time, since each comes from memory.
template <int N, class Column>
__device__ __forceinline__ void take_in(const WinArgs& a, size_t row, float* ref, float* sum, float (&v)[N], Column column) {
    constexpr int AHEAD = N > 8 ? 1 : 4;
    const float* const ml = a.ml + row * a.slots * 2;
    const float* const part = a.part + row * a.slots * (size_t)a.D;
    float top = *ref;
    for (int s0 = 0; s0 < a.NP; s0 += 8) {
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = ml[2 * min(s0 + k, a.NP - 1)];
#pragma unroll
        for (int k = 0; k < 8; ++k) top = fmaxf(top, x[k]);
    }
    const float f = __builtin_amdgcn_exp2f(*ref - top);
    *sum *= f;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= f;
    for (int s0 = 0; s0 < a.NP; s0 += AHEAD) {
        float2 m[AHEAD];
        float x[AHEAD][N];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int s = min(s0 + k, a.NP - 1);
            m[k] = *(const float2*)(ml + 2 * s);
#pragma unroll
            for (int i = 0; i < N; ++i) x[k][i] = part[(size_t)s * a.D + column(i)];
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (s0 + k < a.NP) {
                const float g = __builtin_amdgcn_exp2f(m[k].x - top);
                *sum = fmaf(m[k].y, g, *sum);
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = fmaf(x[k][i], g, v[i]);
            }
    }
    *ref = top;
}

// a wave's rows without the workgroup's other waves: partial results, or whole ones
template <bool BF, bool Q8, int D, int NR, bool FOLD>
__device__ __forceinline__ void store(const WinArgs& a, const Task& t, int end, Rows<BF, Q8, D, NR>& r, int row0) {
    constexpr int E = D / 16;
    // Where all registers are in use, the lane is made here: the compiler would hold addresses that hang on it through all of
    // the task, and for them put others into memory.  No kernel here does that; where it is done at the begin of a block
    // that some lanes skip, the lanes' common numbers are lost for these (seen with three waves a SIMD, which need it).
    int lane = threadIdx.x & 63;
    if (!Q8 && D == 128) asm volatile("" : "+v"(lane));
    const int n = lane & 15, gq = lane >> 4;
    r.finish(end);
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
        const int i = row0 + rt * 16 + n;
        if (i >= t.rows) continue;
        const int tok = t.token(i, a), h = t.head(i, a);
        const size_t at = (size_t)tok * a.H + h;
        if (t.splits > 1) {
            const size_t slot = at * a.slots + t.split;
            float* const p = a.part + slot * D;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) p[column_of<Q8, E>(4 * gq + k, e)] = r.o[rt][e][k];
            if (gq == 0) a.ml[slot * 2] = r.ref[rt], a.ml[slot * 2 + 1] = r.sum[rt];
        } else {
            if (FOLD && a.fold && r.hi[rt] >= 0) {
                float v[4 * E];
#pragma unroll
                for (int i = 0; i < 4 * E; ++i) v[i] = r.o[rt][i % E][i / E];
                take_in<4 * E>(a, at, &r.ref[rt], &r.sum[rt], v, [gq](int i) { return column_of<Q8, E>(4 * gq + i / E, i % E); });
#pragma unroll
                for (int i = 0; i < 4 * E; ++i) r.o[rt][i % E][i / E] = v[i];
            }
            const float inv = r.sum[rt] == 0.f ? 0.f : 1.0f / r.sum[rt];
            uint16_t* const o = a.out + (int64_t)tok * a.ot + h * a.oh;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float v[E];
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = r.o[rt][e][k] * inv;
                put_out<BF, Q8, E>(o, 4 * gq + k, v);
            }
            if (a.lse && gq == 0) a.lse[at] = r.sum[rt] == 0.f ? -INFINITY : r.ref[rt] * 0.69314718055994531f + logf(r.sum[rt]);
        }
    }
}

template <int D>
struct MeetLds {
    float o[4][16][D + 4];
    float ml[4][16][2];
};

// the four waves' results of a workgroup's task, summed and stored
template <bool BF, bool Q8, int D>
__device__ __forceinline__ void meet(const WinArgs& a, const Task& t, int prefix, int end, Rows<BF, Q8, D, 1>& r, MeetLds<D>& l) {
    constexpr int E = D / 16;
    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, n = lane & 15, gq = lane >> 4;
    r.finish(end);
    __syncthreads();                          // an earlier task's LDS is read out
    if (gq == 0) l.ml[w][n][0] = r.ref[0], l.ml[w][n][1] = r.sum[0];
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, l.ml[i][n][0]);
    const float f = __builtin_amdgcn_exp2f(r.ref[0] - top);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) l.o[w][n][column_of<Q8, E>(4 * gq + i, e)] = r.o[0][e][i] * f;
    __syncthreads();
    for (int i = tid; i < t.rows * (D / 4); i += kT) {
        const int row = i / (D / 4), d = i % (D / 4) * 4;
        f32x4 v = *(const f32x4*)&l.o[0][row][d];
#pragma unroll
        for (int k = 1; k < 4; ++k) v += *(const f32x4*)&l.o[k][row][d];
        float tp = -INFINITY, sm = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) tp = fmaxf(tp, l.ml[k][row][0]);
#pragma unroll
        for (int k = 0; k < 4; ++k) sm += l.ml[k][row][1] * __builtin_amdgcn_exp2f(l.ml[k][row][0] - tp);
        const int tok = t.token(row, a), h = t.head(row, a);
        const size_t at = (size_t)tok * a.H + h;
        if (t.splits > 1) {
            const size_t slot = at * a.slots + t.split;
            *(f32x4*)(a.part + slot * D + d) = v;
            if (d == 0) a.ml[slot * 2] = tp, a.ml[slot * 2 + 1] = sm;
            continue;
        }
        if (a.fold && t.position(row, a) >= prefix) {               // (others see nothing)
            float x[4] = {v[0], v[1], v[2], v[3]};
            take_in<4>(a, at, &tp, &sm, x, [d](int i) { return d + i; });
            v = f32x4{x[0], x[1], x[2], x[3]};
        }
        const float inv = sm == 0.f ? 0.f : 1.0f / sm;
        const u32x2 o = {pack2<BF>(v[0] * inv, v[1] * inv), pack2<BF>(v[2] * inv, v[3] * inv)};
        *(u32x2*)(a.out + (int64_t)tok * a.ot + h * a.oh + d) = o;
        if (a.lse && d == 0) a.lse[at] = sm == 0.f ? -INFINITY : tp * 0.69314718055994531f + logf(sm);
    }
}

// The next task of a workgroup or wave: the prefix's for workgroups below ptasks, which have one, else the sequences'.
struct Asked {
    Tasks all;
    unsigned task, step;
    bool prefix, done = false;

    __device__ __forceinline__ Asked(const WinArgs& a, int waves) : prefix((int)blockIdx.x < a.ptasks) {
        const int w = waves > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
        task = (blockIdx.x - a.ptasks) * waves + w;
        step = (gridDim.x - a.ptasks) * waves;
    }
    template <int RT>
    __device__ __forceinline__ bool next(const PagedCache& c, const PagedBatch& b, const WinArgs& a, Task& t) {
        if (prefix) {
            if (done) return false;
            done = true;
            return prefix_task(c, b, a, t);
        }
        for (;;) {
            if (!all.template find<RT>(c, b, a, task, t)) return false;
            task = task + step < task ? ~0u : task + step;
            if (t.split < t.splits) return true;                    // (fewer chunks than the sequence's longest block of rows)
        }
    }
    __device__ __forceinline__ int end(const PagedCache& c, const PagedBatch& b) const {
        return prefix ? kAll : b.prefix + b.width * c.unit * kPageUnit;
    }
};

// A workgroup per task of up to 128 rows, the four waves on different rows.
template <bool BF, bool Q8, int D>
__global__ void __launch_bounds__(kT) __attribute__((amdgpu_waves_per_eu(2))) k_window_wide(PagedCache c, PageScales sc, PagedBatch b, WinArgs a) {
    constexpr int NR = kWideRows / 64;
    __shared__ StageLds<D> l[2];
    __shared__ OddLds odd;
    Asked asked(a, 1);
    Task t;
    while (asked.template next<kWideRows>(c, b, a, t)) {
        Rows<BF, Q8, D, NR> r;
        __syncthreads();                      // an earlier task's LDS is read out
        walk_wide<BF, Q8, D, NR>(c, sc, b, a, t, l, odd, r);
        store<BF, Q8, D, NR, false>(a, t, asked.end(c, b), r, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * NR * 16);
    }
}

// A workgroup per task of up to 16 rows, the four waves on every fourth tile.
template <bool BF, bool Q8, int D>
__global__ void __launch_bounds__(kT) __attribute__((amdgpu_waves_per_eu(2))) k_window(PagedCache c, PageScales sc, PagedBatch b, WinArgs a) {
    __shared__ MeetLds<D> l;
    Asked asked(a, 1);
    Task t;
    while (asked.template next<kFewRows>(c, b, a, t)) {
        Rows<BF, Q8, D, 1> r;
        walk<BF, Q8, D>(c, sc, b, a, t, t.b0 + 2 * __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), 8, r);
        meet<BF, Q8, D>(a, t, b.prefix, asked.end(c, b), r, l);
    }
}

// A wave per task of up to 16 rows.
template <bool BF, bool Q8, int D>
__global__ void __launch_bounds__(kT) __attribute__((amdgpu_waves_per_eu(2))) k_window_waves(PagedCache c, PageScales sc, PagedBatch b, WinArgs a) {
    Asked asked(a, 4);
    Task t;
    while (asked.template next<kFewRows>(c, b, a, t)) {
        Rows<BF, Q8, D, 1> r;
        walk<BF, Q8, D>(c, sc, b, a, t, t.b0, 2, r);
        store<BF, Q8, D, 1, true>(a, t, asked.end(c, b), r, 0);
    }
}

// A wave per row (token, head) joins its chunks: their references and sums in the lanes, a group of lanes (four
// columns a lane) one chunk each.
template <bool BF>
__global__ void __launch_bounds__(kT) k_window_join(PagedCache c, PagedBatch b, WinArgs a) {
    const int lane = threadIdx.x & 63, D = c.D, row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= b.T * a.H) return;
    const int t = row / a.H, h = row % a.H;
    int64_t place = -1;
    const int sq = paged_place(b, t, &place);
    if (sq < 0) return;
    const Seq q = seq_at(b, sq);
    if (t - q.start >= q.n) return;           // padding: its output stays as it is
    const int cap = b.width * c.unit * kPageUnit;
    const unsigned r0 = ((t - q.start) * a.per + h % a.per) & ~(a.RT - 1u);       // (RT is a power of two)
    const int lo = (int)(r0 / a.per), hi = min((int)((r0 + a.RT - 1) / a.per), q.n - 1);
    int n = a.NP + chunks_of(seen(b, a, cap, b.prefix + q.first + lo, b.prefix + q.first + hi).n, a.CT);
    if (n == 1) return;                       // finished where it was computed
    if (place < 0) n = 0;                     // (the prefix was worked on for all rows)
    const float* ml = a.ml + (size_t)row * a.slots * 2;
    const float* part = a.part + (size_t)row * a.slots * D;
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
        for (int k0 = 0; k0 < m; k0 += 8 * groups) {
            f32x4 x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int k = k0 + j * groups + g;
                x[j] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (k < m && d < D) x[j] = *(const f32x4*)(part + (size_t)(i0 + k) * D + d);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float fk = __shfl(f, min(k0 + j * groups + g, 63));
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(x[j][e], fk, acc[e]);
            }
        }
    }
    for (int o = gl; o < 64; o *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o);
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    if (g == 0 && d < D) {
        const u32x2 r = {pack2<BF>(acc[0] * inv, acc[1] * inv), pack2<BF>(acc[2] * inv, acc[3] * inv)};
        *(u32x2*)(a.out + (int64_t)t * a.ot + h * a.oh + d) = r;
    }
    if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -INFINITY : top * 0.69314718055994531f + logf(sum);
}

enum { WIDE, SMALL, WAVES };                  // kernels

struct Plan {
    bool wide_own;
    int RT, most, NO, CT, NP, CP, rb, rows, ptasks, groups;
    int own, before, slots;                   // kernels of the sequences' tasks and of the prefix's; partial results of a row
    bool fold;
};

// Rows per block, chunks and workgroups from the sizes that the host knows.
int plan_of(const PagedCache& c, const PagedBatch& b, int H, int W, int S, Plan* p) {
    const int per = H / c.G;
    const int64_t rows = (int64_t)b.T * per, each = (rows + b.B - 1) / b.B;
    if (rows * c.G > kRowsMax) return LOOPSPEC_EINVAL;
    // Blocks of 128 rows or of 16: 16 sequences' 16 tokens (64 rows a head each, 4000 positions) 48 us and 71, 52 and 47 over
    // 8-bit pages; with 12 tokens 45 and 55, 51 and 39; one sequence's 16 tokens 21 and 16.
    p->wide_own = each > 48;
    // Rows of several sequences over the prefix at once, where none has enough of its own: 32 sequences behind 8000 positions
    // 38 us, one by one 72.  Blocks of 128 of them or of 16: 256 rows over 4000 positions 20 us and 31, 128 rows 18 and 25,
    // but the own positions' launch then costs 10 more.  Short prefixes and own positions stay one task a sequence (8 sequences
    // behind 400 positions 13 us, the prefix apart 10 + 5; 64 of them 19 and 12 + 13).
    const int64_t seqs = std::min(b.B, b.T), held = (int64_t)b.width * c.unit;    // blocks of 16 that a table holds
    const int slots = 512;                    // two workgroups a CU
    const bool brief = ((b.prefix + 15) / 16 + held + 1) / 2 <= kUncut && (seqs + std::max<int64_t>(rows - seqs * per, 0) / kFewRows) * c.G <= slots;
    const bool together = b.prefix > 0 && W == kAll && b.B > 1 && !p->wide_own && !brief;
    const bool wide = p->wide_own || (together && rows > 128);
    p->RT = p->wide_own ? kWideRows : kFewRows;
    p->NP = p->CP = p->rb = p->rows = p->ptasks = 0;
    if (together) {
        const int block = wide ? kWideRows : kFewRows;
        p->rb = (int)((rows + block - 1) / block);
        p->rows = (int)((rows + p->rb * 16 - 1) / (p->rb * 16) * 16);
        // The number of chunks that takes the least time, in steps of 128 positions: rounds of resident workgroups, whose start
        // and end count as two, and the partial results (512 rows over 4000 positions: 8 chunks 27 + 26 us, 16 chunks 30 + 37).
        const int64_t steps = (b.prefix + 127) / 128, heads = (int64_t)c.G * p->rb;
        int64_t best = -1;
        for (int64_t np = 1; np <= std::min<int64_t>(steps, 128); ++np) {
            const int64_t len = (steps + np - 1) / np, n = (steps + len - 1) / len;
            const int64_t cost = (heads * n + slots - 1) / slots * (len + 2) * slots + 6 * heads * n;
            if (best < 0 || cost < best) best = cost, p->NP = (int)n, p->CP = (int)(len * 4);
        }
        const int64_t pairs = ((int64_t)c.G * p->NP + 7) / 8 * 8;
        if (pairs * p->rb > kGroupsMax) return LOOPSPEC_EINVAL;
        p->ptasks = (int)(pairs * p->rb);
    }
    // blocks of 16 positions that a block of rows may see
    int64_t most = (together ? 0 : (b.prefix + 15) / 16) + held;
    if (W < kAll) most = std::min(most, ((int64_t)W + p->RT / per + 2 + 15) / 16 + 3 + ((int64_t)S + 15) / 16);
    p->most = (int)most;
    const int64_t tiles = std::max<int64_t>(1, (most + 1) / 2);
    const int64_t blocks = (seqs + std::max<int64_t>(rows - seqs * per, 0) / p->RT) * c.G;
    // About 1024 tasks where the tables are full (over 18 batches of ragged lengths 384 to 1536 are within 3 %), of at least
    // two tiles a wave.  What is short (700 positions 15 us, in chunks of 8 tiles 11 + 5) is not cut, nor are prompts and
    // windows, whose tasks are alike, that fill the card (64 rows over 4096 of 12000 positions 168 us, cut in two 172 + 6).
    // The join's time is not weighed: one row over 100000 positions takes 103 us in 126 chunks a head, in 32 83.
    if ((!p->wide_own && tiles <= kUncut) || ((p->wide_own || W < kAll) && blocks >= slots))
        p->CT = (int)tiles;
    else
        p->CT = (int)std::min<int64_t>(tiles, std::max<int64_t>(p->wide_own ? 16 : 8, (tiles * blocks / 1024 + 1) / 2 * 2));
    p->NO = (int)((tiles + p->CT - 1) / p->CT);
    const int64_t tasks = blocks * p->NO;
    // A wave per task where there are enough short ones (8 heads, up to 250 positions): 128 sequences 22 us, by workgroups 26;
    // 64 of them 19 and 17; 512 of up to 60 positions 29 and 71.
    const bool by_wave = !p->wide_own && p->NO == 1 && p->CT <= 16 && tasks >= 2 * slots;
    p->own = p->wide_own ? WIDE : by_wave ? WAVES : SMALL;
    p->before = wide ? WIDE : SMALL;
    // Workgroups that go on from task to task fill the card once (the same rows cut in two 172 us, with a workgroup each 174);
    // tasks of many rows are too unequal for that.
    p->groups = (int)std::min<int64_t>(by_wave ? (tasks + 3) / 4 : tasks, p->wide_own ? 16384 : slots);
    // Where the prefix has a launch of its own and a row's own positions are one task, that one finishes the row: waves behind
    // 5 chunks 28 us, with a join 21 + 14, behind 16 chunks 37 and 16 + 11; workgroups behind 32 chunks 20 and 13 + 10.
    p->fold = together && p->own != p->before && p->NO == 1 && p->NP <= (by_wave ? 8 : 32);
    p->slots = p->fold ? p->NP : p->NP + p->NO > 1 ? p->NP + p->NO : 0;
    return LOOPSPEC_OK;
}

// for unit_div of numbers below per + 128 by per
unsigned unit_magic(int per) { return per > 1 ? (unsigned)(((1ull << 32) + per - 1) / per) : 0u; }

uint64_t bytes_of(const PagedCache& c, const PagedBatch& b, int H, const Plan& p) {
    return (uint64_t)b.T * H * p.slots * (c.D + 2) * 4;
}

int check(const loopspec_paged_cache* cache, const loopspec_page_scales* scales, const loopspec_paged_batch* batch, int n_heads,
          int window, int sinks, PagedCache* c, PageScales* s, PagedBatch* b, Plan* p) {
    int rc = paged_args(cache, batch, c, b);
    if (rc) return rc;
    *s = PageScales{};
    if (scales && (rc = scale_args(cache, scales, s))) return rc;
    if (n_heads < 1 || n_heads > (1 << 16) || n_heads % c->G) return LOOPSPEC_EINVAL;
    if (window < 0 || sinks < 0) return LOOPSPEC_EINVAL;
    if (b->prefix > 0 && !b->prefix_table) return LOOPSPEC_EINVAL;
    if (!b->B || !b->T) return LOOPSPEC_OK;
    return plan_of(*c, *b, n_heads, window ? std::min(window, kAll) : kAll, std::min(sinks, kAll), p);
}

template <bool BF, bool Q8, int D>
const void* kernel_of(int k) {
    switch (k) {
        case WIDE: return (const void*)k_window_wide<BF, Q8, D>;
        case SMALL: return (const void*)k_window<BF, Q8, D>;
        default: return (const void*)k_window_waves<BF, Q8, D>;
    }
}
template <bool BF, bool Q8>
const void* kernel_of(int D, int k) {
    switch (D) {
        case 16: return kernel_of<BF, Q8, 16>(k);
        case 32: return kernel_of<BF, Q8, 32>(k);
        case 64: return kernel_of<BF, Q8, 64>(k);
        case 96: return kernel_of<BF, Q8, 96>(k);
        default: return kernel_of<BF, Q8, 128>(k);
    }
}

}  // namespace
}  // namespace ls

extern "C" {

uint64_t loopspec_window_attention_workspace_bytes(const loopspec_paged_cache* cache, const loopspec_page_scales* scales,
                                                   const loopspec_paged_batch* batch, int32_t n_heads, int32_t window,
                                                   int32_t sinks) {
    ls::PagedCache c;
    ls::PageScales s;
    ls::PagedBatch b;
    ls::Plan p{};
    if (ls::check(cache, scales, batch, n_heads, window, sinks, &c, &s, &b, &p)) return 0;
    if (!b.B || !b.T) return 0;
    return ls::bytes_of(c, b, n_heads, p);
}

int loopspec_window_attention(const loopspec_paged_cache* cache, const loopspec_page_scales* scales,
                              const loopspec_paged_batch* batch, const loopspec_attention_args* args, int32_t window,
                              int32_t sinks, void* workspace_dev, uint64_t workspace_bytes, void* stream) {
    using namespace ls;
    PagedCache c;
    PageScales s;
    PagedBatch b;
    Plan p{};
    if (!args) return LOOPSPEC_EINVAL;
    const int rc = check(cache, scales, batch, args->n_heads, window, sinks, &c, &s, &b, &p);
    if (rc) return rc;
    const float cs = args->scale * 1.44269504088896341f;
    if (!(args->scale > 0.f) || !(cs < 3e38f)) return LOOPSPEC_EINVAL;
    if (!b.B || !b.T) return LOOPSPEC_OK;     // (empty tensors have no address)
    if (!rows_ok(args->q_dev, args->q_token, args->q_head) || !rows_ok(args->out_dev, args->out_token, args->out_head)) return LOOPSPEC_EINVAL;
    if ((args->n_heads > 1 && args->out_head < c.D) || (b.T > 1 && args->out_token < c.D)) return LOOPSPEC_EINVAL;
    const uint64_t need = bytes_of(c, b, args->n_heads, p);
    if (need && (!workspace_dev || ((uintptr_t)workspace_dev & 15) || workspace_bytes < need)) return LOOPSPEC_EINVAL;
    const uint64_t rows = (uint64_t)b.T * args->n_heads;
    WinArgs a{(const uint16_t*)args->q_dev, args->q_token, args->q_head, (uint16_t*)args->out_dev, args->out_token, args->out_head,
              args->lse_dev, (float*)workspace_dev, (float*)workspace_dev + rows * p.slots * c.D, cs, c.D, args->n_heads,
              args->n_heads / c.G, unit_magic(args->n_heads / c.G), window ? std::min(window, kAll) : kAll, std::min(sinks, kAll), p.RT, p.most, p.NO, p.CT,
              p.NP, p.CP, p.rb, p.rows, 0, p.slots, p.fold};
    hipStream_t st = (hipStream_t)stream;
    const bool bf = cache->dtype == LOOPSPEC_BF16, q8 = scales != nullptr;
    auto run = [&](int kernel, int groups) {
        void* kargs[] = {&c, &s, &b, &a};
        const void* f = bf ? q8 ? kernel_of<true, true>(c.D, kernel) : kernel_of<true, false>(c.D, kernel)
                           : q8 ? kernel_of<false, true>(c.D, kernel) : kernel_of<false, false>(c.D, kernel);
        return hipLaunchKernel(f, dim3((unsigned)groups), dim3(kT), kargs, 0, st) == hipSuccess;
    };
    if (p.ptasks && p.own != p.before) {
        a.ptasks = p.ptasks;
        if (!run(p.before, p.ptasks)) return LOOPSPEC_EHIP;
        a.ptasks = 0;
        if (!run(p.own, p.groups)) return LOOPSPEC_EHIP;
    } else {
        a.ptasks = p.ptasks;
        if (!run(p.own, p.ptasks + p.groups)) return LOOPSPEC_EHIP;
    }
    if (p.NP + p.NO > 1 && !p.fold) {
        void* jargs[] = {&c, &b, &a};
        const void* j = bf ? (const void*)k_window_join<true> : (const void*)k_window_join<false>;
        if (hipLaunchKernel(j, dim3((unsigned)((rows + 3) / 4)), dim3(kT), jargs, 0, st) != hipSuccess) return LOOPSPEC_EHIP;
    }
    return LOOPSPEC_OK;
}

}  // extern "C"
