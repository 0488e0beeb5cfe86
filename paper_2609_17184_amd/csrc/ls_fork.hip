// Forks of a batch over a paged cache: whole pages are shared and counted, the
// partly filled last page is copied, pages without a reader are given out again.
//
// Four launches: counts start as the caller's; a workgroup per child writes its
// table row and one per parent lets pages go (integer atomics, whose order does
// not matter); one workgroup numbers the free pages in rising order and the wants
// of the children in theirs; a workgroup per child and slice of the caches fills
// in the pages and copies.
//
// Which child takes its parent's pages over is found by looking through the
// children before it, so nothing has to be exchanged for it.
#include "ls_paged.h"

#include <algorithm>

namespace ls {

namespace {

constexpr int kT = 256;
constexpr int kMany = 16;                     // caches per launch: their descriptions travel with it
constexpr int kWanted = -2;                   // an entry of the new table that is to get a page

struct Fork {
    const int32_t *seq_len, *table, *parent, *refs;
    int64_t stride, out_stride;
    int n, m, width, ps, pages, P, W, S, room;
    int32_t *len_out, *table_out, *refs_out, *lack;
    int32_t* need;                            // [m + 1] pages that a child wants, then the number of the first of them; pages given out
    int32_t* source;                          // [m] page that a child has a copy of, or -1
    int32_t* free;                            // [pages] those given out, in rising order
};

struct Copied {
    char *k, *v;
    uint8_t *ks, *vs;
    int64_t kp, kh, kr, vp, vh, vr;           // strides in bytes: page, head, position
    int64_t ksp, ksh, vsp, vsh;
    int G, chunks;                            // heads, 16-byte pieces of a row
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
// some child below j (of m) continues row p; every thread of the workgroup gets the answer
__device__ __forceinline__ bool has_child(const Fork& f, int p, int j) {
    bool any = false;
    for (int i = threadIdx.x; i < j; i += kT) any |= f.parent[i] == p;
    return __syncthreads_or(any);
}

// Row j of the new table: what it takes over of its parent's, -1 elsewhere, kWanted where it is to get a page.
__device__ void child_row(const Fork& f, int j) {
    __shared__ int wants;
    const int p = f.parent[j];
    const int len = (unsigned)p < (unsigned)f.n ? f.seq_len[p] : -1;
    int32_t* const to = f.table_out + j * f.out_stride;
    if (threadIdx.x == 0) wants = 0;
    const bool heir = len >= 0 && !has_child(f, p, j);
    __syncthreads();
    int mine = 0;
    if (len < 0) {
        for (int i = threadIdx.x; i < f.width; i += kT) to[i] = -1;
        if (threadIdx.x == 0) f.source[j] = -1;
    } else {
        const int32_t* const from = f.table + p * f.stride;
        const int full = (int)min((int64_t)(len / f.ps), (int64_t)f.width), held = pages_of(f, len);
        const int64_t more = (min((int64_t)len, (int64_t)f.width * f.ps) + f.room + f.ps - 1) / f.ps;
        const int want = f.room ? (int)min(more, (int64_t)f.width) : held;
        for (int i = threadIdx.x; i < f.width; i += kT) {
            const int x = from[i];
            const bool ok = page_ok(f, x), off = gone(f, len, i);
            int y = -1;
            if (heir) {
                if (ok && off) atomicSub(&f.refs_out[x], 1);
                if (ok && !off) y = x;
                if (!ok && i >= held && i < want) y = kWanted;
            } else {
                if (i < full) {
                    if (ok && !off) y = x, atomicAdd(&f.refs_out[x], 1);
                } else if (i < held) {
                    if (ok) y = kWanted;
                } else if (i < want) {
                    y = kWanted;
                }
            }
            to[i] = y;
            mine += y == kWanted;
        }
        if (f.room && more > f.width && threadIdx.x == 0) atomicAdd(f.lack, (int)(more - f.width));
        if (threadIdx.x == 0) f.source[j] = !heir && full < held && page_ok(f, from[full]) ? from[full] : -1;
    }
    if (mine) atomicAdd(&wants, mine);
    __syncthreads();
    if (threadIdx.x == 0) f.need[j] = wants, f.len_out[j] = len < 0 ? -1 : len;
    __syncthreads();
}

// A row without a child lets its pages go.
__device__ void end_row(const Fork& f, int p) {
    const bool kept = has_child(f, p, f.m);
    if (kept || f.seq_len[p] < 0) return;
    for (int i = threadIdx.x; i < f.width; i += kT) {
        const int x = f.table[p * f.stride + i];
        if (page_ok(f, x)) atomicSub(&f.refs_out[x], 1);
    }
}

// sum of v over the threads below, and over all of them
__device__ __forceinline__ int scan(int v, int* total) {
    __shared__ int part[kT / 64];
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
    for (int i = 0; i < kT / 64; ++i) {
        if (i < w) before += part[i];
        all += part[i];
    }
    *total = all;
    return before + upto - v;
}

// need[j] becomes the number of child j's first page among the free ones; free lists as many of these as are wanted.
__device__ void hand_out(const Fork& f) {
    int wanted = 0, total;
    for (int j0 = 0; j0 < f.m; j0 += kT) {
        const int j = j0 + threadIdx.x, v = j < f.m ? f.need[j] : 0, at = scan(v, &total);
        if (j < f.m) f.need[j] = wanted + at;
        wanted += total;
    }
    constexpr int PER = 8;
    int found = 0;
    for (int x0 = 0; x0 < f.pages && found < wanted; x0 += PER * kT) {
        unsigned mask = 0;
        const int first = x0 + PER * (int)threadIdx.x;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (first + i < f.pages && f.refs_out[first + i] == 0) mask |= 1u << i;
        int at = found + scan(__popc(mask), &total);
        for (; mask; mask &= mask - 1, ++at)
            if (at < wanted) {
                const int x = first + __ffs(mask) - 1;
                f.free[at] = x;
                f.refs_out[x] = 1;
            }
        found += total;
    }
    if (threadIdx.x == 0) {
        f.need[f.m] = min(found, wanted);     // pages given out
        f.lack[0] += max(wanted - found, 0);
    }
}

__global__ void __launch_bounds__(kT) k_fork_start(Fork f) {
    const int i = blockIdx.x * kT + threadIdx.x;
    if (i < f.pages && f.refs_out != f.refs) f.refs_out[i] = f.refs[i];
    if (i == 0) *f.lack = 0;
}
__global__ void __launch_bounds__(kT) k_fork_rows(Fork f) {
    if ((int)blockIdx.x < f.m)
        child_row(f, blockIdx.x);
    else
        end_row(f, blockIdx.x - f.m);
}
__global__ void __launch_bounds__(kT) k_fork_free(Fork f) { hand_out(f); }

// Workgroup (child, y, z): positions of the child's last page, half a cache (keys or values) and a share of the pieces
// each; the first one fills in the child's wanted entries as well.
__global__ void __launch_bounds__(kT) k_fork_copy(Fork f, CopySet set, int fill) {
    const int j = blockIdx.x, first = f.need[j], given = f.need[f.m], src = f.source[j];
    if (fill && blockIdx.y == 0 && blockIdx.z == 0) {
        int32_t* const row = f.table_out + j * f.out_stride;
        int at = first, total;
        for (int i0 = 0; i0 < f.width; i0 += kT) {
            const int i = i0 + threadIdx.x;
            const bool want = i < f.width && row[i] == kWanted;
            const int k = at + scan(want, &total);
            if (want) row[i] = k < given ? f.free[k] : -1;
            at += total;
        }
    }
    if (src < 0 || first >= given || (int)blockIdx.y >= 2 * set.n) return;
    const int dst = f.free[first], n = f.len_out[j] % f.ps;         // (the copy's page is the first that the child wants)
    const Copied& c = set.c[blockIdx.y >> 1];
    const bool val = blockIdx.y & 1;
    char* const base = val ? c.v : c.k;
    const int64_t sp = val ? c.vp : c.kp, sh = val ? c.vh : c.kh, sr = val ? c.vr : c.kr;
    const char* const from = base + src * sp;
    char* const to = base + dst * sp;
    const int per = n * c.chunks;
    for (int64_t i = blockIdx.z * kT + threadIdx.x; i < (int64_t)c.G * per; i += gridDim.z * kT) {
        const int g = (int)(i / per), r = (int)(i - (int64_t)g * per), q = r / c.chunks, x = r - q * c.chunks;
        const int64_t at = g * sh + q * sr + 16 * x;
        *(u32x4*)(to + at) = *(const u32x4*)(from + at);
    }
    if (c.ks && blockIdx.z == 0) {
        uint8_t* const scale = val ? c.vs : c.ks;
        const int64_t tp = val ? c.vsp : c.ksp, th = val ? c.vsh : c.ksh;
        const int blocks = (n + kPageUnit - 1) / kPageUnit;
        for (int i = threadIdx.x; i < c.G * blocks; i += kT) {
            const int g = i / blocks, u = i - g * blocks;
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
                    s.kp, s.kh, s.vp, s.vh, c.G, c.D * e / 16};
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
    auto run = [&](const void* k, dim3 grid, void** a) { return hipLaunchKernel(k, grid, dim3(kT), a, 0, st) == hipSuccess; };
    if (!run((const void*)k_fork_start, dim3((f.pages + kT - 1) / kT), kargs)) return LOOPSPEC_EHIP;
    if (n + m && !run((const void*)k_fork_rows, dim3(n + m), kargs)) return LOOPSPEC_EHIP;
    if (!m) return LOOPSPEC_OK;
    if (!run((const void*)k_fork_free, dim3(1), kargs)) return LOOPSPEC_EHIP;
    int fill = 1;
    for (int i = 0; i < n_caches || fill; i += kMany, fill = 0) {
        set.n = std::min(kMany, n_caches - i);
        for (int k = 0; k < set.n; ++k) describe(i + k, &set.c[k]);
        void* cargs[] = {&f, &set, &fill};
        const int y = std::max(1, 2 * set.n), z = std::max(1, std::min(16, 1024 / (y * m)));
        if (!run((const void*)k_fork_copy, dim3(m, y, z), cargs)) return LOOPSPEC_EHIP;
    }
    return LOOPSPEC_OK;
}

}  // extern "C"
