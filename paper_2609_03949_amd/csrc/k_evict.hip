// k_evict.hip -- the tier of the rows of largest accumulated attention weight, and
// the move of a tier's rows to the front of a paged cache (gfx950).
#include "vkv_internal.h"

namespace vkv {

// ------------------------------------------------------------- the selection
//
// Rows [0, nsink) and [n - recent, n) are kept in any case; of the others the m of
// largest weight, ties to the lower row.  Order by an integer key that grows with the
// weight (NaN below everything, -0 equal to 0).

constexpr int WS_THREADS = 1024, WS_PER = 4;

__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    return key_to_ord(w + 0.0f);
}

// inclusive prefix sum over the block's threads; `total` of all of them
__device__ __forceinline__ int block_prefix(int v, int* s_wave, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = 1; d < 64; d *= 2) {
        const int t = __shfl_up(v, d);
        if (lane >= d) v += t;
    }
    __syncthreads();
    if (lane == 63) s_wave[wave] = v;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int i = 0; i < WS_THREADS / 64; ++i) {
        const int t = s_wave[i];
        if (i < wave) before += t;
        total += t;
    }
    return v + before;
}

__global__ __launch_bounds__(WS_THREADS) void weight_select_kernel(WeightSelArgs a) {
    __shared__ int hist[2048];
    __shared__ int s_wave[WS_THREADS / 64];
    __shared__ int s_bin, s_left;
    const int b = blockIdx.x, tid = threadIdx.x;
    const int n = min(max(a.kv_len[b], 0), a.max_kv), K = a.keep;
    int32_t* kept = a.kept + (int64_t)b * K;
    if (tid == 0) a.count[b] = min(n, K);
    if (n <= K) {
        for (int j = tid; j < K; j += WS_THREADS) kept[j] = j < n ? j : -1;
        return;
    }
    const float* w = a.weight + (int64_t)b * a.stride;
    const int lo = a.nsink, hi = n - a.recent;   // the rows that compete
    int left = K - a.nsink - a.recent;           // how many of them are kept
    // the left-th largest key, 11 + 11 + 10 bits at a time
    uint32_t prefix = 0, mask = 0;
    const int shifts[3] = {21, 10, 0};
    if (left > 0)
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = shifts[pass], bins = pass == 2 ? 1024 : 2048;
            for (int i = tid; i < bins; i += WS_THREADS) hist[i] = 0;
            __syncthreads();
            for (int u = lo + tid; u < hi; u += WS_THREADS) {
                const uint32_t key = weight_key(w[u]);
                if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & (bins - 1)], 1);
            }
            __syncthreads();
            // bins from the top: thread t takes bins - 1 - 2 t and the next one down
            const int i1 = bins - 1 - 2 * tid, c1 = i1 >= 0 ? hist[i1] : 0, c0 = i1 >= 1 ? hist[i1 - 1] : 0;
            int total;
            const int upto = block_prefix(c1 + c0, s_wave, total), above = upto - c1 - c0;
            if (above < left && left <= upto) {
                const bool first = left <= above + c1;
                s_bin = first ? i1 : i1 - 1;
                s_left = left - (first ? above : above + c1);
            }
            __syncthreads();
            prefix |= (uint32_t)s_bin << shift;
            mask |= (uint32_t)(bins - 1) << shift;
            left = s_left;
            __syncthreads();
        }
    // rows above the key, and the first `left` rows that have it, in order
    const bool none = K - a.nsink - a.recent == 0;
    int out = 0, ties = 0;
    for (int u0 = 0; u0 < n; u0 += WS_THREADS * WS_PER) {
        uint32_t key[WS_PER];
        int eq = 0;
#pragma unroll
        for (int i = 0; i < WS_PER; ++i) {
            const int u = u0 + WS_PER * tid + i;
            key[i] = u >= lo && u < hi ? weight_key(w[u]) : 0u;
            eq += u >= lo && u < hi && key[i] == prefix && !none;
        }
        int total_eq, total;
        int at_eq = ties + block_prefix(eq, s_wave, total_eq) - eq;
        bool take[WS_PER];
        int cnt = 0;
#pragma unroll
        for (int i = 0; i < WS_PER; ++i) {
            const int u = u0 + WS_PER * tid + i;
            const bool in = u >= lo && u < hi;
            take[i] = u < n && (!in || (!none && (key[i] > prefix || (key[i] == prefix && at_eq < left))));
            if (in && !none && key[i] == prefix) ++at_eq;
            cnt += take[i];
        }
        int at = out + block_prefix(cnt, s_wave, total) - cnt;
#pragma unroll
        for (int i = 0; i < WS_PER; ++i)
            if (take[i]) kept[at++] = u0 + WS_PER * tid + i;
        ties += total_eq;
        out += total;
    }
}

hipError_t launch_weight_select(const WeightSelArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(weight_select_kernel, dim3((unsigned)a.B), dim3(WS_THREADS), 0, s, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------- the move
//
// The count kept rows (ascending) are to fill slots [0, count).  Kept rows below
// count stay where they are; the r-th slot that holds none (a hole) takes the r-th
// kept row from count on.  Holes and sources are disjoint, so rows move in place
// and in any order, and no row moves that need not.  Slot j lies behind i = the number
// of kept rows below j; it is a hole iff kept[i] is not j, its rank then j - i.
//
// One wave per EV_SLOTS slots: kept rows are found by searches that probe 64 places a
// step; then rows go through registers, all of a wave's loads in flight.

constexpr int EV_SLOTS = 8;
constexpr int EV_LOADS = EV_SLOTS * (D_ROW / 8) / 64;   // 9 loads of 64 pieces

// the number of kept rows below x among the first n (ascending), by a whole wave
__device__ __forceinline__ int kept_below(const int32_t* kept, int n, int x) {
    const int lane = threadIdx.x & 63;
    int lo = 0, len = n;   // the answer is in [lo, lo + len]
    while (len > 0) {
        const int step = (len + 63) / 64;
        const int p = lo + lane * step + step - 1;     // the last place of this lane's piece
        const bool below = p < lo + len && kept[p] < x;
        const int c = __popcll(__ballot(below));       // whole pieces below x
        lo += c * step;
        len = min(step - 1, max(len - c * step, 0));
    }
    return lo;
}

__global__ __launch_bounds__(64) void evict_kernel(EvictArgs a) {
    const int nw = (a.keep + EV_SLOTS - 1) / EV_SLOTS;
    const int b = blockIdx.x / nw, j0 = (blockIdx.x % nw) * EV_SLOTS;
    const int lane = threadIdx.x;
    const int kv = min(max(a.kv_len[b], 0), a.max_kv);
    const int32_t* kept = a.kept + (int64_t)b * a.keep;
    const int n = min(min(max(a.count[b], 0), a.keep), kv);
    const int32_t* table = a.table + (int64_t)b * a.tstride;
    int32_t src = -1;      // lane j < EV_SLOTS: the row that is to lie in slot j0 + j
    if (j0 < n) {
        const int below = kept_below(kept, n, n), i0 = kept_below(kept, below, j0);
        // the kept rows from j0 on: which of the slots hold one
        const int32_t v = i0 + lane < below && lane < EV_SLOTS ? kept[i0 + lane] : -1;
        uint32_t held = 0;
#pragma unroll
        for (int l = 0; l < EV_SLOTS; ++l) {
            const int32_t x = __shfl(v, l) - j0;
            if (x >= 0 && x < EV_SLOTS) held |= 1u << x;
        }
        const int j = j0 + lane;
        if (lane < EV_SLOTS && j < n) {
            const int hole = j - i0 - __popc(held & ((1u << lane) - 1));   // its rank, if slot j is one
            const int p = below + hole;
            src = (held >> lane) & 1u ? j : p >= 0 && p < n ? kept[p] : -1;
            if (src != j && (src < n || src >= kv)) src = -1;   // not a table of ascending rows: nothing is moved
        }
    }
    if (lane < EV_SLOTS && j0 + lane < a.keep) {
        const int64_t at = (int64_t)b * a.keep + j0 + lane;
        if (a.origin) a.origin[at] = src;
        if (a.weight_out) a.weight_out[at] = src >= 0 ? a.weight[(int64_t)b * a.wstride + src] : 0.f;
    }
    // where the rows lie (a row on a page that does not exist stays)
    int64_t from = -1, to = -1;
    if (src >= 0 && src != j0 + lane) {
        const int32_t ps = table[src >> a.shift], pd = table[(j0 + lane) >> a.shift];
        if ((uint32_t)ps < (uint32_t)a.n_pages && (uint32_t)pd < (uint32_t)a.n_pages) {
            from = (int64_t)ps * a.ps + (int64_t)(src & a.page_mask) * a.rs;
            to = (int64_t)pd * a.ps + (int64_t)((j0 + lane) & a.page_mask) * a.rs;
        }
    }
    if (__ballot(from >= 0) == 0) return;
    u32x4_t piece[EV_LOADS];
    int64_t dst[EV_LOADS];
#pragma unroll
    for (int i = 0; i < EV_LOADS; ++i) {
        const int q = 64 * i + lane, r = q / (D_ROW / 8), p = q % (D_ROW / 8);
        const int64_t f = __shfl(from, r), t = __shfl(to, r);
        dst[i] = f >= 0 ? t + 8 * p : -1;
        piece[i] = f >= 0 ? *reinterpret_cast<const u32x4_t*>(a.cache + f + 8 * p) : u32x4_t{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < EV_LOADS; ++i)
        if (dst[i] >= 0) *reinterpret_cast<u32x4_t*>(a.cache + dst[i]) = piece[i];
}

int64_t evict_waves(int64_t keep) { return (keep + EV_SLOTS - 1) / EV_SLOTS; }

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(evict_kernel, dim3((unsigned)(a.B * evict_waves(a.keep))), dim3(64), 0, s, a);
    return hipGetLastError();
}

}  // namespace vkv
