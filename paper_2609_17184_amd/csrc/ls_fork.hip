// Forks of a batch over a paged cache: whole pages are shared and counted, the
// partly filled last page is copied, pages without a reader are given out again.
//
// Four launches: counts start as the caller's; a wave per child writes its table
// row and one per parent lets pages go (integer atomics, whose order does not
// matter); one workgroup numbers the free pages in rising order and the wants of
// the children in theirs; a workgroup per child and half a cache fills in the
// pages and copies.  For few rows and pages one workgroup does all but the copies.
//
// Which child takes its parent's pages over is found by looking through the
// children before it, so nothing has to be exchanged for it.  It does not take
// over what it would append to and others hold too (a row that was shortened into
// a page it shares): the counts from before the step tell.  Such a page is let go
// only when the free ones have been numbered, since others may copy from it.
//
// Measured, in a queue of calls (us): 192 children of 192 rows of up to 16 pages of
// 64, 6 caches of 8 heads of 128 in 8 bits (48 MB): 28, the four launches 2 + 3 + 4 +
// 14 (3.4 TB/s in the copies, a large copy 4.8) and the host's 28.  8 children of 4
// rows: 22, all of it the host's; 6 + 4 in the two kernels, chains of loads.
#include "ls_paged.h"

#include <algorithm>

namespace ls {

namespace {

constexpr int kT = 256, kMost = 1024;
constexpr int kMany = 16;                     // caches per launch: their descriptions travel with it
constexpr int kWanted = -2;                   // an entry of the new table that is to get a page

struct Fork {
    const int32_t *seq_len, *table, *parent, *refs;
    int64_t stride, out_stride;
    int n, m, width, ps, pages, P, W, S, room;
    int32_t *len_out, *table_out, *refs_out, *lack;
    int32_t* need;                            // [m + 1] pages that a child wants, then the number of the first of them; pages given out
    int32_t* source;                          // [m] page that a child has a copy of, or -1; -2 - page if it is to be let go
    int32_t* free;                            // [pages] the counts as they were, then the pages given out, in rising order
};

struct Copied {
    char *k, *v;
    uint8_t *ks, *vs;
    int64_t kp, kh, kr, vp, vh, vr;           // strides in bytes: page, head, position
    int64_t ksp, ksh, vsp, vsh;
    unsigned G, chunks;                       // heads, 16-byte pieces of a row
};
struct CopySet {
    Copied c[kMany];
    int n;
};

__device__ __forceinline__ bool page_ok(const Fork& f, int x) { return (unsigned)x < (unsigned)f.pages; }
// pages that hold a row's positions (in part)
__device__ __forceinline__ int pages_of(const Fork& f, int64_t positions) {
    return (int)min((positions + f.ps - 1) / f.ps, (int64_t)f.width);
}
// page i holds nothing that the position behind `len` own ones sees
__device__ __forceinline__ bool gone(const Fork& f, int len, int i) {
    if (!f.W) return false;
    const int64_t first = f.P + (int64_t)i * f.ps, next = (int64_t)f.P + len;
    return first + f.ps - 1 <= next - f.W && first >= f.S;
}
// some child below j (of m) continues row p; asked by a whole wave
__device__ __forceinline__ bool has_child(const Fork& f, int p, int j) {
    bool any = false;
    for (int i = threadIdx.x & 63; i < j; i += 64) any |= f.parent[i] == p;
    return __any(any);
}

// the counts: in memory, or in LDS where one workgroup does everything
struct InMemory {
    int32_t* r;
    __device__ __forceinline__ void add(int x, int v) const { atomicAdd(&r[x], v); }
    __device__ __forceinline__ int get(int x) const { return r[x]; }
    __device__ __forceinline__ void set(int x, int v) const { r[x] = v; }
};

// Which lanes' pages x (those that `ask`) others hold beside the row `from`: they count more than the row names them
// (`before`, the counts as they were).
__device__ __forceinline__ bool held_by_others(const Fork& f, const int32_t* before, const int32_t* from, int x, bool ask) {
    const int lane = threadIdx.x & 63, count = ask ? before[x] : 0;
    bool others = false;
    for (unsigned long long left = __ballot(count > 1); left; left &= left - 1) {
        const int l = __ffsll(left) - 1, y = __shfl(x, l);
        int named = 0;
        for (int i0 = 0; i0 < f.width; i0 += 64) named += __popcll(__ballot(i0 + lane < f.width && from[min(i0 + lane, f.width - 1)] == y));
        if (lane == l) others = count > named;
    }
    return others;
}

// A wave's row j of the new table: what it takes over of its parent's, -1 elsewhere, kWanted where it is to get a page.
// Gives the number of these.
template <class R>
__device__ int child_row(const Fork& f, const R& refs, const int32_t* before, int32_t* lack, int j) {
    const int lane = threadIdx.x & 63, p = f.parent[j];
    const int len = (unsigned)p < (unsigned)f.n ? f.seq_len[p] : -1;
    int32_t* const to = f.table_out + j * f.out_stride;
    int wants = 0, source = -1;
    bool heir = false;
    if (len < 0) {
        for (int i = lane; i < f.width; i += 64) to[i] = -1;
    } else {
        heir = !has_child(f, p, j);
        const int32_t* const from = f.table + p * f.stride;
        const int full = (int)min((int64_t)(len / f.ps), (int64_t)f.width), held = pages_of(f, len);
        const int64_t more = (min((int64_t)len, (int64_t)f.width * f.ps) + f.room + f.ps - 1) / f.ps;
        const int want = f.room ? (int)min(more, (int64_t)f.width) : held;
        for (int i0 = 0; i0 < f.width; i0 += 64) {
            const int i = i0 + lane, x = i < f.width ? from[i] : -1;
            const bool ok = page_ok(f, x), off = gone(f, len, i);
            const bool others = heir && held_by_others(f, before, from, x, ok && !off && i >= full);
            int y = -1;
            if (i < f.width) {
                if (heir) {
                    if (others && i < held) {
                        y = kWanted, source = x;                    // (let go later)
                    } else if (ok && (off || others)) {
                        refs.add(x, -1);
                    } else if (ok) {
                        y = x;
                    }
                    if (i >= held && i < want && y < 0) y = kWanted;
                } else if (i < full) {
                    if (ok && !off) y = x, refs.add(x, 1);
                } else if (i < held) {
                    if (ok) y = kWanted, source = x;                // its page of the copy
                } else if (i < want) {
                    y = kWanted;
                }
                to[i] = y;
            }
            wants += __popcll(__ballot(y == kWanted));
        }
        if (f.room && more > f.width && lane == 0) atomicAdd(lack, (int)(more - f.width));
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) source = max(source, __shfl_xor(source, o));
    if (lane == 0) f.source[j] = heir && source >= 0 ? -2 - source : source, f.len_out[j] = len < 0 ? -1 : len;
    return wants;
}

// An heir that has a copy of its last page lets that page go.
template <class R>
__device__ __forceinline__ void let_go(const Fork& f, const R& refs, int j) {
    if (f.source[j] < -1) refs.add(-2 - f.source[j], -1);
}

// A row without a child lets its pages go; a wave's work.
template <class R>
__device__ void end_row(const Fork& f, const R& refs, int p) {
    if (has_child(f, p, f.m) || f.seq_len[p] < 0) return;
    for (int i = threadIdx.x & 63; i < f.width; i += 64) {
        const int x = f.table[p * f.stride + i];
        if (page_ok(f, x)) refs.add(x, -1);
    }
}

// the wanted entries of row j get the free pages from number `at` on; a wave's work
__device__ void fill_row(const Fork& f, const int32_t* free, int j, int at, int given) {
    const int lane = threadIdx.x & 63;
    int32_t* const row = f.table_out + j * f.out_stride;
    for (int i0 = 0; i0 < f.width; i0 += 64) {
        const int i = i0 + lane;
        const bool want = i < f.width && row[i] == kWanted;
        const unsigned long long all = __ballot(want);
        const int k = at + __popcll(all & ((1ull << lane) - 1));
        if (want) row[i] = k < given ? free[k] : -1;
        at += __popcll(all);
    }
}

// sum of v over the threads below, and over all of them
template <int NT>
__device__ __forceinline__ int scan(int v, int* total) {
    __shared__ int part[NT / 64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int upto = v;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int u = __shfl_up(upto, o);
        if (lane >= o) upto += u;
    }
    __syncthreads();                          // an earlier scan's parts are read
    if (lane == 63) part[w] = upto;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
        if (i < w) before += part[i];
        all += part[i];
    }
    *total = all;
    return before + upto - v;
}

// need[j] becomes the number of child j's first page among the free ones, need[m] how many are given out; free lists
// these.  A workgroup's work; returns how many were wanted and not to be had.
template <int NT, class R>
__device__ int hand_out(const Fork& f, const R& refs, int32_t* need, int32_t* free) {
    int wanted = 0, total;
    for (int j0 = 0; j0 < f.m; j0 += NT) {
        const int j = j0 + threadIdx.x, v = j < f.m ? need[j] : 0, at = scan<NT>(v, &total);
        if (j < f.m) need[j] = wanted + at;
        wanted += total;
    }
    constexpr int PER = 8;
    int found = 0;
    for (int x0 = 0; x0 < f.pages && found < wanted; x0 += PER * NT) {
        unsigned mask = 0;
        const int first = x0 + PER * (int)threadIdx.x;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (first + i < f.pages && refs.get(first + i) == 0) mask |= 1u << i;
        int at = found + scan<NT>(__popc(mask), &total);
        for (; mask; mask &= mask - 1, ++at)
            if (at < wanted) {
                const int x = first + __ffs(mask) - 1;
                free[at] = x;
                refs.set(x, 1);
            }
        found += total;
    }
    if (threadIdx.x == 0) need[f.m] = min(found, wanted);
    return max(wanted - found, 0);
}

__global__ void __launch_bounds__(kT) k_fork_start(Fork f) {
    const int i = blockIdx.x * kT + threadIdx.x;
    if (i < f.pages) {
        const int32_t count = f.refs[i];
        f.free[i] = count;
        if (f.refs_out != f.refs) f.refs_out[i] = count;
    }
    if (i == 0) *f.lack = 0;
}
// a wave per child, then one per parent
__global__ void __launch_bounds__(kT) k_fork_rows(Fork f) {
    const int i = blockIdx.x * (kT / 64) + (threadIdx.x >> 6);
    const InMemory refs{f.refs_out};
    if (i < f.m) {
        const int wants = child_row(f, refs, f.free, f.lack, i);
        if ((threadIdx.x & 63) == 0) f.need[i] = wants;
    } else if (i < f.m + f.n) {
        end_row(f, refs, i - f.m);
    }
}
__global__ void __launch_bounds__(kMost) k_fork_free(Fork f) {
    const int lack = hand_out<kMost>(f, InMemory{f.refs_out}, f.need, f.free);
    if (threadIdx.x == 0) *f.lack += lack;
}

// All of it but the copies for few rows and pages, with counts and lists in LDS: 4 rows, 8 children and 190 pages 24 us in
// all instead of 31 (two launches less).  Of more rows a workgroup's 16 waves would take several each, one after another,
// and look for heirs through all children each time.
constexpr int kFewRows = 128, kFewPages = 4096;
struct InLds {
    int* r;
    __device__ __forceinline__ void add(int x, int v) const { atomicAdd(&r[x], v); }
    __device__ __forceinline__ int get(int x) const { return r[x]; }
    __device__ __forceinline__ void set(int x, int v) const { r[x] = v; }
};
__global__ void __launch_bounds__(kMost) k_fork_small(Fork f) {
    __shared__ int refs[kFewPages], free[kFewPages], need[kFewRows + 1], lack;
    const int tid = threadIdx.x, w = tid >> 6;
    for (int i = tid; i < f.pages; i += kMost) refs[i] = free[i] = f.refs[i];
    if (tid == 0) lack = 0;
    __syncthreads();
    for (int i = w; i < f.m + f.n; i += kMost / 64) {
        if (i < f.m) {
            const int wants = child_row(f, InLds{refs}, free, &lack, i);
            if ((tid & 63) == 0) need[i] = wants;
        } else {
            end_row(f, InLds{refs}, i - f.m);
        }
    }
    __syncthreads();
    const int short_of = hand_out<kMost>(f, InLds{refs}, need, free);
    __syncthreads();
    const int given = need[f.m];
    // (a row's wave is the one that wrote it)
    for (int j = w; j < f.m; j += kMost / 64) {
        if ((tid & 63) == 0) let_go(f, InLds{refs}, j);
        fill_row(f, free, j, need[j], given);
    }
    for (int i = tid; i < given; i += kMost) f.free[i] = free[i];
    for (int i = tid; i <= f.m; i += kMost) f.need[i] = need[i];
    if (tid == 0) *f.lack = lack + short_of;
    __syncthreads();
    for (int i = tid; i < f.pages; i += kMost) f.refs_out[i] = refs[i];
}

// Workgroup (child, y, z): positions of the child's last page, half a cache (keys or values) and a share of the pieces
// each; the first one fills in the child's wanted entries and lets go what is left to, as well.
__global__ void __launch_bounds__(kT) k_fork_copy(Fork f, CopySet set, int fill) {
    const int j = blockIdx.x, first = f.need[j], given = f.need[f.m], source = f.source[j], src = source < -1 ? -2 - source : source;
    if (fill && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x < 64) {
        fill_row(f, f.free, j, first, given);
        if (threadIdx.x == 0) let_go(f, InMemory{f.refs_out}, j);
    }
    if (src < 0 || first >= given || (int)blockIdx.y >= 2 * set.n) return;
    const int dst = f.free[first], n = f.len_out[j] % f.ps;         // (the copy's page is the first that the child wants)
    const Copied& c = set.c[blockIdx.y >> 1];
    const bool val = blockIdx.y & 1;
    char* const base = val ? c.v : c.k;
    const int64_t sp = val ? c.vp : c.kp, sh = val ? c.vh : c.kh, sr = val ? c.vr : c.kr;
    const char* const from = base + src * sp;
    char* const to = base + dst * sp;
    const unsigned per = n * c.chunks, all = c.G * per, step = gridDim.z * kT;      // (below 2^30)
    constexpr int AHEAD = 4;                  // pieces on their way
    for (unsigned i0 = blockIdx.z * kT + threadIdx.x; i0 < all; i0 += AHEAD * step) {
        u32x4 x[AHEAD];
        int64_t at[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const unsigned i = min(i0 + k * step, all - 1), g = i / per, r = i - g * per, q = r / c.chunks;
            at[k] = g * sh + q * sr + 16 * (r - q * c.chunks);
            x[k] = *(const u32x4*)(from + at[k]);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i0 + k * step < all) *(u32x4*)(to + at[k]) = x[k];
    }
    if (c.ks && blockIdx.z == 0) {
        uint8_t* const scale = val ? c.vs : c.ks;
        const int64_t tp = val ? c.vsp : c.ksp, th = val ? c.vsh : c.ksh;
        const unsigned blocks = (n + kPageUnit - 1) / kPageUnit;
        for (unsigned i = threadIdx.x; i < c.G * blocks; i += kT) {
            const unsigned g = i / blocks, u = i - g * blocks;
            scale[dst * tp + g * th + u] = scale[src * tp + g * th + u];
        }
    }
}

uint64_t bytes_of(int64_t m, int64_t pages) { return (uint64_t)(2 * m + 1 + pages) * 4; }

}  // namespace
}  // namespace ls

extern "C" {

uint64_t loopspec_fork_pages_workspace_bytes(int32_t n_children, int32_t n_pages) {
    return n_children < 0 || n_children > 65535 || n_pages < 1 ? 0 : ls::bytes_of(n_children, n_pages);
}

int loopspec_fork_pages(const loopspec_fork_args* args, const loopspec_paged_cache* caches,
                        const loopspec_page_scales* scales, int32_t n_caches, void* workspace_dev,
                        uint64_t workspace_bytes, void* stream) {
    using namespace ls;
    if (!args || n_caches < 0 || (n_caches && !caches)) return LOOPSPEC_EINVAL;
    const int n = args->n_seqs, m = args->n_children, width = args->table_width, ps = args->page_size;
    if (n < 0 || n > 65535 || m < 0 || m > 65535 || width < 0 || args->n_pages < 1) return LOOPSPEC_EINVAL;
    if (ps < kPageUnit || ps > kPageMax || ps % kPageUnit || (int64_t)width * ps > kPlacesMax) return LOOPSPEC_EINVAL;
    if ((int64_t)m * width >= 1ll << 31) return LOOPSPEC_EINVAL;
    if (args->prefix_len < 0 || args->prefix_len > kPlacesMax || args->window < 0 || args->sinks < 0) return LOOPSPEC_EINVAL;
    if (args->room < 0 || args->room > (int64_t)width * ps) return LOOPSPEC_EINVAL;
    if ((n && (!args->seq_len_dev || (width && !args->table_dev))) || (n > 1 && args->table_stride < width)) return LOOPSPEC_EINVAL;
    if ((m && (!args->parent_dev || !args->seq_len_out_dev || (width && !args->table_out_dev))) || (m > 1 && args->out_stride < width))
        return LOOPSPEC_EINVAL;
    if (!args->refs_dev || !args->refs_out_dev || !args->short_dev) return LOOPSPEC_EINVAL;
    if (!workspace_dev || ((uintptr_t)workspace_dev & 15) || workspace_bytes < bytes_of(m, args->n_pages)) return LOOPSPEC_EINVAL;
    auto describe = [&](int i, Copied* d) {
        PagedCache c;
        PagedBatch b;
        PageScales s{};
        loopspec_paged_batch none{};
        int rc = paged_args(&caches[i], &none, &c, &b);
        const bool eight = scales && scales[i].k_dev;
        if (!rc && eight) rc = scale_args(&caches[i], &scales[i], &s);
        if (rc || caches[i].page_size != ps || caches[i].n_pages != args->n_pages) return LOOPSPEC_EINVAL;
        const int e = eight ? 1 : 2;
        *d = Copied{(char*)c.k, (char*)c.v, s.k, s.v, c.kp * e, c.kh * e, c.ks * e, c.vp * e, c.vh * e, c.vs * e,
                    s.kp, s.kh, s.vp, s.vh, (unsigned)c.G, (unsigned)(c.D * e / 16)};
        return LOOPSPEC_OK;
    };
    CopySet set{};
    for (int i = 0; i < n_caches; ++i)        // all of them before anything runs
        if (describe(i, &set.c[0])) return LOOPSPEC_EINVAL;
    int32_t* const ws = (int32_t*)workspace_dev;
    Fork f{args->seq_len_dev, args->table_dev, args->parent_dev, args->refs_dev, args->table_stride, args->out_stride,
           n, m, width, ps, args->n_pages, args->prefix_len, args->window, args->sinks, args->room,
           args->seq_len_out_dev, args->table_out_dev, args->refs_out_dev, args->short_dev, ws, ws + m + 1, ws + 2 * m + 1};
    hipStream_t st = (hipStream_t)stream;
    void* kargs[] = {&f};
    auto run = [&](const void* k, dim3 grid, dim3 block, void** a) { return hipLaunchKernel(k, grid, block, a, 0, st) == hipSuccess; };
    int fill = 1;
    if (n + m <= kFewRows && f.pages <= kFewPages) {
        if (!run((const void*)k_fork_small, dim3(1), dim3(kMost), kargs)) return LOOPSPEC_EHIP;
        fill = 0;
    } else {
        if (!run((const void*)k_fork_start, dim3((f.pages + kT - 1) / kT), dim3(kT), kargs)) return LOOPSPEC_EHIP;
        if (!run((const void*)k_fork_rows, dim3((n + m + kT / 64 - 1) / (kT / 64)), dim3(kT), kargs)) return LOOPSPEC_EHIP;
        if (m && !run((const void*)k_fork_free, dim3(1), dim3(kMost), kargs)) return LOOPSPEC_EHIP;
    }
    if (!m) return LOOPSPEC_OK;
    for (int i = 0; i < n_caches || fill; i += kMany, fill = 0) {
        set.n = std::min(kMany, n_caches - i);
        for (int k = 0; k < set.n; ++k) describe(i + k, &set.c[k]);
        void* cargs[] = {&f, &set, &fill};
        const int y = std::max(1, 2 * set.n), z = std::max(1, std::min(16, 1024 / (y * m)));
        if (!run((const void*)k_fork_copy, dim3(m, y, z), dim3(kT), cargs)) return LOOPSPEC_EHIP;
    }
    return LOOPSPEC_OK;
}

}  // extern "C"
