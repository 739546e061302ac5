// k_pool.hip -- the life of a paged cache's pages (gfx950): forks, pages for new rows, compaction.
//
// The state is the sequences' tables and a count of the entries that name each page; a free page is one
// that none names.  So nothing is kept beside them, and which page is given follows from it alone: free pages
// are ranked by their number (counts of 4096 pages each, then ranks within), requests by sequence and entry, and the
// r-th request gets the r-th page.  Counts are changed by atomic additions, whose order does not show.  What moves are whole pages of
// every plane and layer, by a fixed number of workgroups that share the copies the earlier launch has listed, however
// many they are.  Bound: HBM (each moved page is read and written once); small calls by their launches.
#include <algorithm>

#include "vkv_internal.h"

namespace vkv {

constexpr int PO_THREADS = 256, PO_WAVES = PO_THREADS / 64, PO_EACH = POOL_BLOCK / PO_THREADS;
constexpr int PO_MOVERS = 2048;          // workgroups that copy
constexpr int PO_PIECE = 16 * 1024;      // bytes that one copies at a time
enum { PO_FREE = 0, PO_PAIRS = 1, PO_HEAD = 64 };   // words of head: free pages; copies

__device__ __forceinline__ bool names(const PoolArgs& a, int e) { return (uint32_t)e < (uint32_t)a.n_pages; }
__device__ __forceinline__ int rows_of(const PoolArgs& a, int n) { return min(max(n, 0), a.width * a.page); }

template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
    return v;
}
// v summed over the workgroup, in every thread
template <typename T>
__device__ __forceinline__ T group_sum(T v, T* lds) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    T s = 0;
#pragma unroll
    for (int i = 0; i < PO_WAVES; ++i) s += lds[i];
    return s;
}
// the sum of v over the threads before this one
__device__ __forceinline__ int group_before(int v, int* lds) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int upto = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int t = __shfl_up(upto, d);
        if (lane >= d) upto += t;
    }
    __syncthreads();
    if (lane == 63) lds[w] = upto;
    __syncthreads();
    int s = upto - v;
    for (int i = 0; i < w; ++i) s += lds[i];
    return s;
}
template <typename T>
__device__ __forceinline__ T sum_of(const int32_t* p, int n, int step, T* lds) {
    T s = 0;
    for (int i = threadIdx.x; i < n; i += PO_THREADS) s += p[(int64_t)step * i];
    return group_sum(s, lds);
}

// ----------------------------------------------------------------------- fork

// the rows of the sequences that become forks, as they are before the call; their pages gain a name
__global__ __launch_bounds__(PO_THREADS) void fork_take_kernel(PoolArgs a, const int32_t* from) {
    const int b = blockIdx.x, s = from[b];
    if (s == b) return;
    int32_t* rows = a.rows + (int64_t)b * (a.width + 1);
    const bool some = s >= 0 && s < a.B;
    const int n = some ? rows_of(a, a.kv_len[s]) : 0;
    const int32_t* t = a.table + (int64_t)(some ? s : 0) * a.tstride;
    for (int j = threadIdx.x; j < (n + a.page - 1) / a.page; j += PO_THREADS) {
        const int e = t[j];
        rows[j] = names(a, e) ? e : -1;
        if (names(a, e)) atomicAdd(a.refs + e, 1);
    }
    if (threadIdx.x == 0) rows[a.width] = n;
}
// the rows in their place; the pages that were there lose a name
__global__ __launch_bounds__(PO_THREADS) void fork_put_kernel(PoolArgs a, const int32_t* from) {
    const int b = blockIdx.x;
    if (from[b] == b) return;
    const int32_t* rows = a.rows + (int64_t)b * (a.width + 1);
    const int n = rows[a.width], np = (n + a.page - 1) / a.page;
    int32_t* t = a.table + (int64_t)b * a.tstride;
    for (int j = threadIdx.x; j < a.width; j += PO_THREADS) {
        const int e = t[j];
        if (names(a, e)) atomicAdd(a.refs + e, -1);
        t[j] = j < np ? rows[j] : -1;
    }
    if (threadIdx.x == 0) a.kv_len[b] = n;
}

// Both in one workgroup, for few entries (launches are what such a call costs): the sequences' sources and lengths in LDS, then
// the entries of all of them, thread by thread.
constexpr int PS_THREADS = 1024, PS_WAVES = PS_THREADS / 64, PS_EACH = POOL_SMALL / PS_THREADS, PS_SEQS = PS_THREADS;

__global__ __launch_bounds__(PS_THREADS) void fork_small_kernel(PoolArgs a, const int32_t* from) {
    __shared__ int src[PS_SEQS], len[PS_SEQS];      // (src[b] = b: stays)
    const int tid = threadIdx.x, entries = a.B * a.width;
    if (tid < a.B) {
        const int s = from[tid];
        const bool some = s >= 0 && s < a.B;
        src[tid] = some ? s : -1;
        len[tid] = some ? rows_of(a, a.kv_len[s]) : 0;
    }
    __syncthreads();
#pragma unroll 4
    for (int i = tid; i < entries; i += PS_THREADS) {
        const int b = i / a.width, j = i - b * a.width, s = src[b];
        if (s == b) continue;
        int e = j < (len[b] + a.page - 1) / a.page ? a.table[(int64_t)s * a.tstride + j] : -1;
        if (names(a, e)) atomicAdd(a.refs + e, 1);
        else e = -1;
        a.rows[i] = e;
    }
    __syncthreads();
#pragma unroll 4
    for (int i = tid; i < entries; i += PS_THREADS) {      // (each thread the entries that it wrote)
        const int b = i / a.width, j = i - b * a.width;
        if (src[b] == b) continue;
        int32_t* t = a.table + (int64_t)b * a.tstride + j;
        const int e = *t;
        if (names(a, e)) atomicAdd(a.refs + e, -1);
        *t = a.rows[i];
    }
    if (tid < a.B && src[tid] != tid) a.kv_len[tid] = len[tid];
}

// -------------------------------------------------------------------- reserve

struct Ask {
    int kv, want, j0, j1;   // rows now and wanted; the entries [j0, j1) that have to name a page
    int shared;             // the page of entry j0 - 1, where it is to be copied, or -1
    int absent;             // entry j0 - 1 holds rows and names no page
};
__device__ __forceinline__ Ask ask(const PoolArgs& a, const int32_t* want, int b) {
    Ask q;
    q.kv = rows_of(a, a.kv_len[b]);
    q.want = rows_of(a, want[b]);
    q.shared = -1;
    q.absent = 0;
    q.j0 = (q.kv + a.page - 1) / a.page;
    q.j1 = (q.want + a.page - 1) / a.page;
    if (q.want > q.kv && q.kv % a.page) {
        const int e = a.table[(int64_t)b * a.tstride + q.j0 - 1];
        if (!names(a, e)) q.absent = 1;
        else if (a.refs[e] > 1) q.shared = e;
    }
    return q;
}

// what a wave's sequence needs: pages, and whether one of them is for a copy
__device__ __forceinline__ int needs(const PoolArgs& a, const int32_t* want, int b, bool* shares) {
    const Ask q = ask(a, want, b);
    int n = 0;
    for (int j = q.j0 + (int)(threadIdx.x & 63); j < q.j1; j += 64) n += !names(a, a.table[(int64_t)b * a.tstride + j]);
    *shares = q.shared >= 0;
    return wave_sum(n) + *shares;
}

// pages of each block that are free (or in use, if used), and what each sequence needs
__global__ __launch_bounds__(PO_THREADS) void pool_count_kernel(PoolArgs a, const int32_t* want, int used) {
    __shared__ int lds[PO_WAVES];
    if ((int)blockIdx.x < a.nb) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < PO_EACH; ++i) {
            const int64_t p = (int64_t)blockIdx.x * POOL_BLOCK + PO_THREADS * i + threadIdx.x;
            if (p < a.n_pages) n += (a.refs[p] > 0) == (used != 0);
        }
        n = group_sum(n, lds);
        if (threadIdx.x == 0) a.block[blockIdx.x] = n;
        if (blockIdx.x == 0 && threadIdx.x == 0) a.head[PO_PAIRS] = 0;
        return;
    }
    const int b = ((int)blockIdx.x - a.nb) * PO_WAVES + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (b >= a.B) return;
    bool shares;
    const int n = needs(a, want, b, &shares);
    if (lane == 0) {
        a.need[2 * b] = n;
        a.need[2 * b + 1] = shares;
    }
}

// the free pages in order, as many as are needed
__global__ __launch_bounds__(PO_THREADS) void reserve_list_kernel(PoolArgs a) {
    __shared__ int lds[PO_WAVES];
    const int64_t p0 = (int64_t)blockIdx.x * POOL_BLOCK + (int64_t)PO_EACH * threadIdx.x;
    __shared__ int64_t wide[PO_WAVES];
    const int64_t most = sum_of(a.need, a.B, 2, wide);   // (more than 32 bits hold, where nobody can have that many)
    const int before = sum_of(a.block, blockIdx.x, 1, lds);
    uint32_t free = 0;
#pragma unroll
    for (int i = 0; i < PO_EACH; ++i)
        if (p0 + i < a.n_pages && a.refs[p0 + i] <= 0) free |= 1u << i;
    int r = before + group_before(__popc(free), lds);
#pragma unroll
    for (int i = 0; i < PO_EACH; ++i)
        if ((free >> i) & 1u) {
            if (r < most) a.list[r] = (int32_t)(p0 + i);
            ++r;
        }
    if ((int)blockIdx.x == a.nb - 1 && threadIdx.x == 0) a.head[PO_FREE] = before + a.block[blockIdx.x];
}

// One wave's sequence b takes its requests, those from `at` on of all, and its copy, the copy-th; list: the free pages in order.
__device__ __forceinline__ void give(const PoolArgs& a, const int32_t* want, int b, int64_t at, int copy, bool shares, int have,
                                     const int32_t* list, int32_t* missing, bool count) {
    const int lane = threadIdx.x & 63;
    const Ask q = ask(a, want, b);      // (its shared is not looked at: the counts change while the call runs)
    int lacks = q.absent;
    int32_t* t = a.table + (int64_t)b * a.tstride;
    if (shares) {
        if (at < have) {
            if (lane == 0) {
                int32_t* entry = t + q.kv / a.page;
                const int e = *entry, to = list[at];
                a.from[copy] = e;
                a.to[copy] = to;
                if (count) atomicMax(a.head + PO_PAIRS, copy + 1);
                atomicAdd(a.refs + e, -1);
                a.refs[to] = 1;
                *entry = to;
            }
        } else {
            ++lacks;
        }
        ++at;
    }
    for (int j = q.j0; j < q.j1; j += 64) {
        const bool open = j + lane < q.j1 && !names(a, t[j + lane]);
        const uint64_t all = __ballot(open);
        const int64_t r = at + __popcll(all & ((1ull << lane) - 1));
        const bool got = open && r < have;
        if (got) {
            const int to = list[r];
            a.refs[to] = 1;
            t[j + lane] = to;
        }
        at += __popcll(all);
        lacks += __popcll(__ballot(open && !got));
    }
    if (lane == 0) missing[b] = lacks;
}
// a wave a sequence: its requests are those from the sum of the sequences' before it on
__global__ __launch_bounds__(PO_THREADS) void reserve_give_kernel(PoolArgs a, const int32_t* want, int32_t* missing) {
    const int b = (int)blockIdx.x * PO_WAVES + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (b >= a.B) return;
    int64_t at = 0;
    int copy = 0;
    for (int i = lane; i < b; i += 64) {
        at += a.need[2 * i];
        copy += a.need[2 * i + 1];
    }
    give(a, want, b, wave_sum(at), wave_sum(copy), a.need[2 * b + 1] != 0, a.head[PO_FREE], a.list, missing, true);
}

// the copies of pairs of pages, shared by workgroups of THREADS

template <int THREADS, typename T>
__device__ __forceinline__ void move_plane(const PoolPlane& s, const int32_t* from, const int32_t* to, int pairs, int wg, int wgs) {
    const int64_t n = s.bytes / (int64_t)sizeof(T);
    const int64_t per = n < THREADS ? THREADS / n : 1;        // small pages: several by one workgroup
    const int64_t pages = (int64_t)pairs * s.layers;
    const int64_t items = per > 1 ? (pages + per - 1) / per : pages * s.pieces;
    for (int64_t k = wg; k < items; k += wgs) {
        int64_t page, i, end;
        if (per > 1) {
            page = k * per + threadIdx.x / n;
            i = threadIdx.x % n;
            end = threadIdx.x < per * n && page < pages ? n : 0;
        } else {
            page = k / s.pieces;
            const int64_t first = (k % s.pieces) * (PO_PIECE / (int64_t)sizeof(T));
            i = first + threadIdx.x;
            end = min(n, first + PO_PIECE / (int64_t)sizeof(T));
        }
        const int pair = (int)(page % max(pairs, 1)), layer = (int)(page / max(pairs, 1));
        if (i >= end) continue;
        const T* src = reinterpret_cast<const T*>(s.base + layer * s.ls + from[pair] * s.ps);
        T* dst = reinterpret_cast<T*>(s.base + layer * s.ls + to[pair] * s.ps);
        if (per > 1) {
            dst[i] = src[i];
            continue;
        }
        if constexpr (sizeof(T) == 16) {
            constexpr int EACH = PO_PIECE / 16 / THREADS;
            T v[EACH];
#pragma unroll
            for (int q = 0; q < EACH; ++q)
                if (i + THREADS * q < end) v[q] = src[i + THREADS * q];
#pragma unroll
            for (int q = 0; q < EACH; ++q)
                if (i + THREADS * q < end) dst[i + THREADS * q] = v[q];
        } else {
            for (; i < end; i += THREADS) dst[i] = src[i];
        }
    }
}
template <int THREADS>
__device__ __forceinline__ void move_pages(const PoolArgs& a, int pairs, int wg, int wgs) {
    for (int k = 0; k < a.n_planes; ++k) {
        const PoolPlane& s = a.plane[k];
        if (s.unit == 16) move_plane<THREADS, u32x4_t>(s, a.from, a.to, pairs, wg, wgs);
        else if (s.unit == 4) move_plane<THREADS, uint32_t>(s, a.from, a.to, pairs, wg, wgs);
        else move_plane<THREADS, uint8_t>(s, a.from, a.to, pairs, wg, wgs);
    }
}

// The three launches above in one workgroup, for pools of few pages: ranks in registers, needs and free pages in LDS (launches are
// what such a call costs: fork and reserve of 4 beams over 2048 rows 26.6 us in six launches, 12.7 in two; of 64 beams over 8192
// rows 26.1 in six and 20.4 in four).  Few bytes are copied there too.
constexpr int PS_SHORT = 8;      // entries up to which a thread looks through its sequence's by itself

// the sum of v over the threads before this one, and over all
__device__ __forceinline__ int small_before(int v, int* lds, int* total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int upto = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int t = __shfl_up(upto, d);
        if (lane >= d) upto += t;
    }
    __syncthreads();
    if (lane == 63) lds[w] = upto;
    __syncthreads();
    int s = upto - v, all = 0;
#pragma unroll
    for (int i = 0; i < PS_WAVES; ++i) {
        if (i < w) s += lds[i];
        all += lds[i];
    }
    *total = all;
    return s;
}

__global__ __launch_bounds__(PS_THREADS) void reserve_small_kernel(PoolArgs a, const int32_t* want, int32_t* missing, int copies) {
    __shared__ int32_t list[POOL_SMALL];
    __shared__ int lds[PS_WAVES], need[PS_SEQS], share[PS_SEQS];
    const int tid = threadIdx.x, w = tid >> 6, p0 = PS_EACH * tid;
    int32_t refs[PS_EACH];
#pragma unroll
    for (int i = 0; i < PS_EACH; ++i) refs[i] = p0 + i < a.n_pages ? a.refs[p0 + i] : 1;
    // a thread a sequence; those with many entries a wave each, after them
    Ask q{};
    q.shared = -1;
    uint32_t open = 0;               // its entries that name no page
    if (tid < a.B) {
        q = ask(a, want, tid);
        if (q.j1 - q.j0 <= PS_SHORT)
            for (int j = 0; j < q.j1 - q.j0; ++j) open |= names(a, a.table[(int64_t)tid * a.tstride + q.j0 + j]) ? 0u : 1u << j;
        need[tid] = __popc(open) + (q.shared >= 0);
        share[tid] = q.j1 - q.j0 > PS_SHORT;
    }
    __syncthreads();
    for (int b = w; b < a.B; b += PS_WAVES)
        if (share[b]) {
            bool shares;
            const int n = needs(a, want, b, &shares);
            if ((tid & 63) == 0) need[b] = min(n, POOL_SMALL + 1);   // (more than there are, and sums within 32 bits)
        }
    int free = 0, have, all, most;
#pragma unroll
    for (int i = 0; i < PS_EACH; ++i) free += refs[i] <= 0;
    int r = small_before(free, lds, &have);
#pragma unroll
    for (int i = 0; i < PS_EACH; ++i)
        if (refs[i] <= 0) list[r++] = p0 + i;
    // (the scan has waited for every wave)
    const int at = small_before(tid < a.B ? need[tid] : 0, lds, &most), copy = small_before(q.shared >= 0, lds, &all);
    const bool wide = tid < a.B && share[tid];
    __syncthreads();
    if (tid < a.B) need[tid] = at, share[tid] = !wide ? INT32_MIN : q.shared >= 0 ? copy : -1 - copy;
    int pairs;
    (void)small_before(q.shared >= 0 && at < have, lds, &pairs);
    if (tid == 0) a.head[PO_PAIRS] = pairs;
    if (tid < a.B && !wide) {
        int n = at, lacks = q.absent;
        int32_t* t = a.table + (int64_t)tid * a.tstride;
        if (q.shared >= 0) {
            if (n < have) {
                const int to = list[n];
                a.from[copy] = q.shared;
                a.to[copy] = to;
                atomicAdd(a.refs + q.shared, -1);
                a.refs[to] = 1;
                t[q.j0 - 1] = to;
            } else {
                ++lacks;
            }
            ++n;
        }
        for (int j = 0; j < q.j1 - q.j0; ++j)
            if ((open >> j) & 1u) {
                if (n < have) {
                    a.refs[list[n]] = 1;
                    t[q.j0 + j] = list[n];
                } else {
                    ++lacks;
                }
                ++n;
            }
        missing[tid] = lacks;
    }
    for (int b = w; b < a.B; b += PS_WAVES) {
        const int s = share[b];
        if (s != INT32_MIN) give(a, want, b, need[b], s < 0 ? -1 - s : s, s >= 0, have, list, missing, false);
    }
    if (!copies) return;
    __syncthreads();   // the pairs are there
    move_pages<PS_THREADS>(a, pairs, 0, 1);
}

// -------------------------------------------------------------------- compact

__global__ __launch_bounds__(PO_THREADS) void compact_list_kernel(PoolArgs a, int32_t* used) {
    __shared__ int lds[PO_WAVES];
    const int64_t p0 = (int64_t)blockIdx.x * POOL_BLOCK + (int64_t)PO_EACH * threadIdx.x;
    const int n = sum_of(a.block, a.nb, 1, lds);
    uint32_t in = 0;
#pragma unroll
    for (int i = 0; i < PO_EACH; ++i)
        if (p0 + i < a.n_pages && a.refs[p0 + i] > 0) in |= 1u << i;
    int r = sum_of(a.block, blockIdx.x, 1, lds);
    r += group_before(__popc(in), lds);          // pages in use before p
#pragma unroll
    for (int i = 0; i < PO_EACH; ++i) {
        const int64_t p = p0 + i;
        if (p >= a.n_pages) break;
        const bool u = (in >> i) & 1u;
        if (p == n) a.head[PO_PAIRS] = n - r;    // as many holes before n as pages behind it
        if (p >= n) {
            a.list[p] = u ? n - 1 - r : -1;
            if (u) a.from[n - 1 - r] = (int32_t)p;
        } else if (!u) {
            a.to[p - r] = (int32_t)p;
        }
        r += u;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *used = n;   // where every page is in use, the counting launch has left no pairs
}

// the count of the pages in use, and the list, in one workgroup, for few pages
__global__ __launch_bounds__(PS_THREADS) void compact_small_kernel(PoolArgs a, int32_t* used) {
    __shared__ int lds[PS_WAVES];
    const int p0 = PS_EACH * threadIdx.x;
    uint32_t in = 0;
#pragma unroll
    for (int i = 0; i < PS_EACH; ++i)
        if (p0 + i < a.n_pages && a.refs[p0 + i] > 0) in |= 1u << i;
    int n, r = small_before(__popc(in), lds, &n);   // pages in use, and before p
#pragma unroll
    for (int i = 0; i < PS_EACH; ++i) {
        const int p = p0 + i;
        if (p >= a.n_pages) break;
        const bool u = (in >> i) & 1u;
        if (p == n) a.head[PO_PAIRS] = n - r;
        if (p >= n) {
            a.list[p] = u ? n - 1 - r : -1;
            if (u) a.from[n - 1 - r] = p;
        } else if (!u) {
            a.to[p - r] = p;
        }
        r += u;
    }
    if (threadIdx.x == 0) {
        if (n >= a.n_pages) a.head[PO_PAIRS] = 0;
        *used = n;
    }
}

// ----------------------------------------------------------------------- copy

__global__ __launch_bounds__(PO_THREADS) void pool_copy_kernel(PoolArgs a) {
    move_pages<PO_THREADS>(a, a.head[PO_PAIRS], blockIdx.x, gridDim.x);
}

// the copies, and beside them the tables and counts of the pages that move
__global__ __launch_bounds__(PO_THREADS) void compact_move_kernel(PoolArgs a, int movers) {
    if ((int)blockIdx.x < movers) {
        move_pages<PO_THREADS>(a, a.head[PO_PAIRS], blockIdx.x, movers);
        return;
    }
    const int pairs = a.head[PO_PAIRS];
    if (pairs == 0) return;
    const int64_t at = (int64_t)(blockIdx.x - movers) * PO_THREADS + threadIdx.x, step = (int64_t)(gridDim.x - movers) * PO_THREADS;
    const int lowest = a.from[pairs - 1];        // of the pages that move
    for (int64_t i = at; i < pairs; i += step) {
        a.refs[a.to[i]] = a.refs[a.from[i]];
        a.refs[a.from[i]] = 0;
    }
    for (int64_t i = at; i < (int64_t)a.B * a.width; i += step) {
        int32_t* t = a.table + (i / a.width) * a.tstride + i % a.width;
        const int e = *t;
        if (!names(a, e) || e < lowest) continue;
        const int r = a.list[e];
        if (r >= 0) *t = a.to[r];
    }
}

// ------------------------------------------------------------------- launches

PoolLayout pool_layout(int64_t B, int64_t n_pages, int64_t width) {
    PoolLayout l{};
    size_t at = 0;
    auto take = [&](int64_t words) {
        const size_t here = at;
        at += ((size_t)words * 4 + 255) & ~(size_t)255;
        return here;
    };
    const int64_t nb = (n_pages + POOL_BLOCK - 1) / POOL_BLOCK;
    l.head = take(PO_HEAD);
    l.block = take(nb);
    l.need = take(2 * B);
    l.list = take(n_pages);
    l.from = take(std::max(n_pages, B));
    l.to = take(std::max(n_pages, B));
    l.rows = take(B * (width + 1));
    l.total = at;
    return l;
}

hipError_t launch_fork(const PoolArgs& a, const int32_t* from, hipStream_t s) {
    if (a.B <= PS_SEQS && (int64_t)a.B * a.width <= POOL_SMALL_TABLE) {
        hipLaunchKernelGGL(fork_small_kernel, dim3(1), dim3(1024), 0, s, a, from);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(fork_take_kernel, dim3((unsigned)a.B), dim3(PO_THREADS), 0, s, a, from);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(fork_put_kernel, dim3((unsigned)a.B), dim3(PO_THREADS), 0, s, a, from);
    return hipGetLastError();
}

// workgroups that copy up to `pairs` pages
static int movers(const PoolArgs& a, int64_t pairs) {
    int64_t n = 0;
    pairs = std::min<int64_t>(pairs, PO_MOVERS);
    for (int k = 0; k < a.n_planes; ++k) n += pairs * a.plane[k].layers * a.plane[k].pieces;
    return (int)std::min<int64_t>(n, PO_MOVERS);
}

hipError_t launch_reserve(const PoolArgs& a, const int32_t* want, int32_t* missing, hipStream_t s) {
    hipError_t e;
    if (a.n_pages <= POOL_SMALL && a.B <= PS_SEQS) {
        int64_t bytes = 0;   // that are copied at the most
        for (int k = 0; k < a.n_planes; ++k) bytes += a.B * a.plane[k].layers * a.plane[k].bytes;
        const int copies = bytes <= POOL_SMALL_COPY;
        hipLaunchKernelGGL(reserve_small_kernel, dim3(1), dim3(PS_THREADS), 0, s, a, want, missing, copies);
        e = hipGetLastError();
        if (e != hipSuccess || copies) return e;
    } else {
        const int seqs = (a.B + PO_WAVES - 1) / PO_WAVES;
        hipLaunchKernelGGL(pool_count_kernel, dim3((unsigned)(a.nb + seqs)), dim3(PO_THREADS), 0, s, a, want, 0);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL(reserve_list_kernel, dim3((unsigned)a.nb), dim3(PO_THREADS), 0, s, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL(reserve_give_kernel, dim3((unsigned)seqs), dim3(PO_THREADS), 0, s, a, want, missing);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const int n = movers(a, a.B);
    if (n == 0) return hipSuccess;
    hipLaunchKernelGGL(pool_copy_kernel, dim3((unsigned)n), dim3(PO_THREADS), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_compact(const PoolArgs& a, int32_t* used, hipStream_t s) {
    hipError_t e;
    if (a.n_pages <= POOL_SMALL) {
        hipLaunchKernelGGL(compact_small_kernel, dim3(1), dim3(PS_THREADS), 0, s, a, used);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    } else {
        hipLaunchKernelGGL(pool_count_kernel, dim3((unsigned)a.nb), dim3(PO_THREADS), 0, s, a, (const int32_t*)nullptr, 1);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL(compact_list_kernel, dim3((unsigned)a.nb), dim3(PO_THREADS), 0, s, a, used);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const int n = movers(a, a.n_pages / 2);
    const int64_t words = std::max<int64_t>((int64_t)a.B * a.width, a.n_pages);
    const int tables = (int)std::min<int64_t>((words + 4 * PO_THREADS - 1) / (4 * PO_THREADS), 1024);
    hipLaunchKernelGGL(compact_move_kernel, dim3((unsigned)(n + tables)), dim3(PO_THREADS), 0, s, a, n);
    return hipGetLastError();
}

}  // namespace vkv
