// k_evict.hip -- the tier of the rows of largest accumulated attention weight, and
// the move of a tier's rows to the front of a paged cache (gfx950).
#include <algorithm>

#include "vkv_internal.h"

namespace vkv {

// ------------------------------------------------------------- the selection
//
// Rows [0, nsink) and [n - recent, n) are kept in any case; of the others (those that
// compete) the m of largest weight, ties to the lower row.  Order by an integer key that
// grows with the weight (NaN below everything, -0 equal to 0).
//
// One launch, up to WS_MAX_PARTS workgroups a sequence; each finds the m-th largest key for
// itself and writes its part of the rows.  Up to WS_CAP competing rows lie in LDS; of more,
// a sample of WS_SAMPLE rows brackets the m-th key within 4.5 standard deviations of its
// rank, one pass over all weights counts what lies above the bracket and lists what lies
// in it, and the key is selected among those.  Where the bracket misses (which the
// counts tell) or holds too many, the selection passes over all weights.
//
// Measured at 32 sequences of 131072 rows, m = 4096: 34 us, of which the sample and its
// bracket 7, the pass over the weights 16, the selection among the listed rows 4 and the
// writing 5.  The pass is bound by what one compute unit does for its sequence's rows: two
// comparisons a row and, with a bracket that holds 5% of them, a list write in most waves
// (written without the branch it took as long).  More workgroups a sequence only divide the
// writing: each has to know the key, and joining their counts would take a second launch.

constexpr int WS_THREADS = 1024, WS_WAVES = WS_THREADS / 64;
constexpr int WS_PER = 16, WS_CAP = WS_THREADS * WS_PER;    // listed rows of a thread, and of all
constexpr int WS_SAMPLE = 8192, WS_BINS = 2048;
constexpr int WS_MAX_PARTS = 8;
constexpr int WS_LOADS = 16;                                // loads of a thread in flight

__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    return key_to_ord(w + 0.0f);
}

struct SelShared {
    uint2 list[WS_PER + 1][WS_THREADS];   // listed rows and their weights, each thread its own (the last place: too many)
    int hist[2][WS_BINS];     // one is cleared while the other is read
    int wave[WS_WAVES];
    uint32_t lo[WS_WAVES], hi[WS_WAVES];
    int in[WS_WAVES], most[WS_WAVES];     // rows listed by each wave; whether one of its threads found too many
    uint32_t edge[2];
    int bin, left, size;
};

// v combined with that of other lanes by op, in steps within the rows of 16 lanes and then over
// them, without LDS: lane l ends with all of lanes 0 .. l.  zero: op's neutral value.
template <typename Op>
__device__ __forceinline__ int wave_scan(int v, int zero, Op op) {
    v = op(v, __builtin_amdgcn_update_dpp(zero, v, 0x111, 0xF, 0xF, false));   // row_shr:1
    v = op(v, __builtin_amdgcn_update_dpp(zero, v, 0x112, 0xF, 0xF, false));   // row_shr:2
    v = op(v, __builtin_amdgcn_update_dpp(zero, v, 0x114, 0xF, 0xF, false));   // row_shr:4
    v = op(v, __builtin_amdgcn_update_dpp(zero, v, 0x118, 0xF, 0xF, false));   // row_shr:8
    v = op(v, __builtin_amdgcn_update_dpp(zero, v, 0x142, 0xA, 0xF, false));   // row_bcast:15 to rows 1 and 3
    v = op(v, __builtin_amdgcn_update_dpp(zero, v, 0x143, 0xC, 0xF, false));   // row_bcast:31 to rows 2 and 3
    return v;
}
__device__ __forceinline__ int wave_prefix(int v) {
    return wave_scan(v, 0, [](int x, int y) { return x + y; });
}

// sum over the block's threads (two barriers)
__device__ __forceinline__ int block_sum(int v, SelShared& sh) {
    v = wave_prefix(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sh.wave[threadIdx.x >> 6] = v;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int i = 0; i < WS_WAVES; ++i) total += sh.wave[i];
    return total;
}

// smallest and largest of the threads' values (two barriers)
__device__ __forceinline__ void block_range(uint32_t& lo, uint32_t& hi, SelShared& sh) {
    lo = (uint32_t)wave_scan((int)lo, -1, [](int x, int y) { return (int)min((uint32_t)x, (uint32_t)y); });
    hi = (uint32_t)wave_scan((int)hi, 0, [](int x, int y) { return (int)max((uint32_t)x, (uint32_t)y); });
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sh.lo[threadIdx.x >> 6] = lo, sh.hi[threadIdx.x >> 6] = hi;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WS_WAVES; ++i) lo = min(lo, sh.lo[i]), hi = max(hi, sh.hi[i]);
}

// After the threads' atomics on hist[which] (the other one is cleared here): each thread's two
// bins, counted from the top (bins - 1 - 2 t and the next one down), and what lies above them.
struct TopBins {
    int i1, c1, c0, above;
};
__device__ __forceinline__ TopBins top_bins(int bins, int which, SelShared& sh) {
    const int tid = threadIdx.x, wave = tid >> 6;
    __syncthreads();
    TopBins t;
    t.i1 = bins - 1 - 2 * tid;
    t.c1 = t.i1 >= 0 ? sh.hist[which][t.i1] : 0;
    t.c0 = t.i1 >= 1 ? sh.hist[which][t.i1 - 1] : 0;
    const int upto = wave_prefix(t.c1 + t.c0);
    if ((tid & 63) == 63) sh.wave[wave] = upto;
#pragma unroll
    for (int i = tid; i < WS_BINS; i += WS_THREADS) sh.hist[which ^ 1][i] = 0;
    __syncthreads();
    t.above = upto - t.c1 - t.c0;
#pragma unroll
    for (int i = 0; i < WS_WAVES; ++i) t.above += i < wave ? sh.wave[i] : 0;
    return t;
}

// The rank-th largest (from 1) of the keys that each(f) hands to f, every thread its own ones,
// all in [lo, hi]: returns T such that the rank largest are the keys above T and `left` of those
// equal to T (0 where a digit's bin ends the selection: T is then below the bin).  hist[which] is clear.
template <typename Each>
__device__ __forceinline__ uint32_t radix_select(Each each, uint32_t lo, uint32_t hi, int rank, int& which, SelShared& sh,
                                                 int& left) {
    uint32_t prefix = 0, mask = 0;
    int shift = hi == lo ? 0 : 32 - __clz((int)(hi - lo));   // the digits are those of key - lo
    left = rank;
    while (shift > 0) {
        const int bits = min(shift, 11), bins = 1 << bits;
        shift -= bits;
        each([&](uint32_t k) {
            const uint32_t x = k - lo;
            if ((x & mask) == prefix) atomicAdd(&sh.hist[which][(x >> shift) & (bins - 1)], 1);
        });
        const TopBins t = top_bins(bins, which, sh);
        if (t.above < left && left <= t.above + t.c1 + t.c0) {
            const bool first = left <= t.above + t.c1;
            sh.bin = first ? t.i1 : t.i1 - 1;
            sh.left = left - (first ? t.above : t.above + t.c1);
            sh.size = first ? t.c1 : t.c0;
        }
        __syncthreads();
        prefix |= (uint32_t)sh.bin << shift;
        mask |= (uint32_t)(bins - 1) << shift;
        left = sh.left;
        which ^= 1;
        if (sh.size == left && lo + prefix != 0u) {   // all keys of the bin
            left = 0;
            return lo + prefix - 1u;
        }
    }
    return lo + prefix;
}

__global__ __launch_bounds__(WS_THREADS) void weight_select_kernel(WeightSelArgs a) {
    __shared__ SelShared sh;
    // a sequence's workgroups on one XCD (they go there in turn), whose L2 then holds its weights
    const int b = (int)(blockIdx.x / (8u * a.parts)) * 8 + (int)(blockIdx.x % 8u), part = (int)(blockIdx.x / 8u) % a.parts;
    if (b >= a.B) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = min(max(a.kv_len[b], 0), a.max_kv), K = a.keep;
    int32_t* kept = a.kept + (int64_t)b * K;
    if (part == 0 && tid == 0) a.count[b] = min(n, K);
    if (n <= K) {
        for (int64_t j = (int64_t)part * WS_THREADS + tid; j < K; j += (int64_t)a.parts * WS_THREADS) kept[j] = j < n ? (int)j : -1;
        return;
    }
    const float* w = a.weight + (int64_t)b * a.stride;
    const int lo = a.nsink, hi = n - a.recent, N = hi - lo;   // the rows that compete
    const int m = K - a.nsink - a.recent;                     // how many of them are kept (fewer than N)
    // this workgroup's rows (max_kv is at most 2^30: no overflow below)
    const int size = (n + a.parts - 1) / a.parts;
    const int r0 = min(part * size, n), r1 = min(r0 + size, n);
    const int s0 = min(max(r0, lo), hi);                      // competing rows before r0 are [lo, s0)

    // kept: key > T, or key = T and row <= cut;  before: the competing rows kept before s0
    uint32_t T = 0xFFFFFFFFu;
    int cut = 0x7FFFFFFF, before = 0;
    if (m > 0) {
        uint32_t key[WS_PER];                 // this thread's listed keys, cnt of them
        int cnt = 0, rank = m, which = 0, ties;
        // the count-th lowest of the rows whose complements each(f) hands out
        auto last_row = [&](auto each, int count) {
            int left;
            const uint32_t t = radix_select(each, ~(uint32_t)hi, ~(uint32_t)lo, count, which, sh, left);
            return (int)~t - (left == 0 ? 1 : 0);   // (below the bin: the rows before ~t)
        };
        bool listed = true;
        uint32_t ka = 0xFFFFFFFFu, kb = 0;    // the listed keys' range
        for (int i = tid; i < WS_BINS; i += WS_THREADS) sh.hist[0][i] = 0;
        const bool whole = N <= WS_CAP;
        auto row_of = [&](int i) { return whole ? lo + tid + WS_THREADS * i : (int)sh.list[i][tid].x; };
        if (whole) {
            cnt = max((N - tid + WS_THREADS - 1) / WS_THREADS, 0);
            float v[WS_PER];
#pragma unroll
            for (int i = 0; i < WS_PER; ++i) v[i] = WS_THREADS * i < N ? w[lo + min(tid + WS_THREADS * i, N - 1)] : 0.f;
#pragma unroll
            for (int i = 0; i < WS_PER; ++i) {
                key[i] = weight_key(v[i]);
                if (i < cnt) {
                    ka = min(ka, key[i]);
                    kb = max(kb, key[i]);
                }
            }
            block_range(ka, kb, sh);
        } else {
            // the sample: one row of each of WS_SAMPLE equal pieces, at a place in it that a hash picks
            uint32_t sample[WS_SAMPLE / WS_THREADS];
#pragma unroll
            for (int i = 0; i < WS_SAMPLE / WS_THREADS; ++i) {
                const uint32_t j = tid + WS_THREADS * i;
                const uint32_t h = (j * 2654435761u) ^ (j * 40503u >> 3);
                const int p0 = (int)((int64_t)N * j / WS_SAMPLE), p1 = (int)((int64_t)N * (j + 1) / WS_SAMPLE);
                sample[i] = weight_key(w[lo + p0 + (int)(h % (uint32_t)(p1 - p0))]);
                ka = min(ka, sample[i]);
                kb = max(kb, sample[i]);
            }
            block_range(ka, kb, sh);
            // by a histogram over the sample's range: the bins of the ranks that bracket the m-th key
            const int shift = max(kb == ka ? 0 : 32 - __clz((int)(kb - ka)) - 11, 0);
#pragma unroll
            for (int i = 0; i < WS_SAMPLE / WS_THREADS; ++i) atomicAdd(&sh.hist[0][(sample[i] - ka) >> shift], 1);
            const float p = (float)m / (float)N, e = WS_SAMPLE * p, d = 4.5f * sqrtf(e * (1.0f - p)) + 2.0f;
            const int top = (int)(e - d), low = (int)(e + d) + 1;
            if (tid == 0) sh.edge[0] = 0u, sh.edge[1] = 0xFF800000u;   // no lower one; +inf
            const TopBins t = top_bins(WS_BINS, 0, sh);
            which = 1;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int above = t.above + (i ? t.c1 : 0), c = i ? t.c0 : t.c1;
                const uint32_t bin = ka + ((uint32_t)(t.i1 - i) << shift);
                if (above < low && low <= above + c) sh.edge[0] = bin;
                if (above < top && top <= above + c) sh.edge[1] = min(bin + (1u << shift) - 1u, kb);
            }
            __syncthreads();
            ka = sh.edge[0];
            // the key between the negative numbers and 0 is no weight's (-0 has that of 0), and as a number it is -0, which
            // 0 is not above: rows of weight 0 would be listed with keys outside the bracket
            kb = sh.edge[1] == 0x7FFFFFFFu ? 0x7FFFFFFEu : sh.edge[1];
            listed = ka != 0u;    // (0: NaN, which compares with nothing, or everything)
            int above = 0;
            if (listed) {
                const float fb = ord_to_key(kb), fa = ord_to_key(ka);
                int gt = 0;   // this thread's count
                auto look = [&](float v, int u) __attribute__((always_inline)) {
                    const bool over = v > fb;
                    gt += over;
                    if (v >= fa && !over) {
                        sh.list[min(cnt, WS_PER)][tid] = make_uint2((uint32_t)u, __float_as_uint(v));
                        ++cnt;
                    }
                };
                int above_before = 0;
                for (int half = 0; half < 2; ++half) {        // the rows before s0, then the others
                    const int e1 = half ? hi : s0;
                    int i0 = half ? s0 : lo;
                    above_before = gt;
                    // the next batch's loads are in flight while one is looked at
                    float v[WS_LOADS], next[WS_LOADS];
                    auto load = [&](float (&x)[WS_LOADS]) __attribute__((always_inline)) {
#pragma unroll
                        for (int i = 0; i < WS_LOADS; ++i) x[i] = w[i0 + tid + WS_THREADS * i];
                    };
                    constexpr int STEP = WS_THREADS * WS_LOADS;
                    if (e1 - i0 >= STEP) load(next);
                    while (e1 - i0 >= STEP) {
#pragma unroll
                        for (int i = 0; i < WS_LOADS; ++i) v[i] = next[i];
                        const int u = i0 + tid;
                        i0 += STEP;
                        if (e1 - i0 >= STEP) load(next);
#pragma unroll
                        for (int i = 0; i < WS_LOADS; ++i) look(v[i], u + WS_THREADS * i);
                    }
                    for (int u = i0 + tid; u < e1; u += WS_THREADS) look(w[u], u);
                }
                // over the block: rows above, rows above before s0, rows listed
                gt = wave_prefix(gt);
                above_before = wave_prefix(above_before);
                const int listing = wave_prefix(cnt);
                const bool full = __ballot(cnt > WS_PER) != 0;
                if (lane == 63) {
                    sh.lo[wave] = (uint32_t)gt;
                    sh.hi[wave] = (uint32_t)above_before;
                    sh.in[wave] = listing;
                    sh.most[wave] = full;
                }
                __syncthreads();
                int in = 0;
#pragma unroll
                for (int i = 0; i < WS_WAVES; ++i) {
                    above += (int)sh.lo[i];
                    before += (int)sh.hi[i];
                    in += sh.in[i];
                    listed = listed && !sh.most[i];
                }
                listed = listed && above < m && m <= above + in;
                rank = m - above;
                cnt = listed ? cnt : 0;
#pragma unroll
                for (int i = 0; i < WS_PER; ++i)
                    if (i < cnt) key[i] = key_to_ord(__uint_as_float(sh.list[i][tid].y) + 0.0f);
            }
        }
        if (listed) {
            auto each = [&](auto f) {
#pragma unroll
                for (int i = 0; i < WS_PER; ++i)
                    if (i < cnt) f(key[i]);
            };
            T = radix_select(each, ka, kb, rank, which, sh, ties);
            // rows whose key is T: the ties-th lowest of them
            int c = 0;
            if (ties == 0) {
                cut = -1;
            } else {
                auto rows = [&](auto f) {
#pragma unroll
                    for (int i = 0; i < WS_PER; ++i)
                        if (i < cnt && key[i] == T) f(~(uint32_t)row_of(i));
                };
                cut = last_row(rows, ties);
            }
            if (r0 > lo) {
                c = 0;
#pragma unroll
                for (int i = 0; i < WS_PER; ++i)
                    if (i < cnt) {
                        const int u = row_of(i);
                        c += u < s0 && (key[i] > T || (key[i] == T && u <= cut));
                    }
                before += block_sum(c, sh);
            }
        } else {
            // over all weights
            auto all = [&](int e0, int e1, auto f) {
                for (int i0 = e0 + tid; i0 < e1; i0 += WS_THREADS * WS_LOADS) {
                    float v[WS_LOADS];
#pragma unroll
                    for (int i = 0; i < WS_LOADS; ++i) v[i] = w[min(i0 + WS_THREADS * i, e1 - 1)];
#pragma unroll
                    for (int i = 0; i < WS_LOADS; ++i)
                        if (i0 + WS_THREADS * i < e1) f(weight_key(v[i]), i0 + WS_THREADS * i);
                }
            };
            T = radix_select([&](auto f) { all(lo, hi, [&](uint32_t k, int) { f(k); }); }, 0u, 0xFFFFFFFFu, m, which, sh, ties);
            cut = ties == 0 ? -1 : last_row([&](auto f) { all(lo, hi, [&](uint32_t k, int u) { if (k == T) f(~(uint32_t)u); }); }, ties);
            int c = 0;
            all(lo, s0, [&](uint32_t k, int u) { c += k > T || (k == T && u <= cut); });
            before = block_sum(c, sh);
        }
    }
    // the kept rows of [r0, r1), in order: each wave 1024 consecutive rows at a time
    int out = min(r0, lo) + before + max(r0 - hi, 0);
    constexpr int G = 16;
    for (int u0 = r0; u0 < r1; u0 += WS_THREADS * G) {
        float v[G];
        uint64_t take[G];
        int c = 0;
        const int w0 = u0 + 64 * G * wave;
#pragma unroll
        for (int i = 0; i < G; ++i) v[i] = w[min(w0 + 64 * i + lane, r1 - 1)];
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int u = w0 + 64 * i + lane;
            const uint32_t k = weight_key(v[i]);
            take[i] = __ballot(u < r1 && (u < lo || u >= hi || (m > 0 && (k > T || (k == T && u <= cut)))));
            c += __popcll(take[i]);
        }
        __syncthreads();
        if (lane == 0) sh.wave[wave] = c;
        __syncthreads();
        int at = out;
#pragma unroll
        for (int i = 0; i < WS_WAVES; ++i) {
            const int t = sh.wave[i];
            if (i < wave) at += t;
            out += t;
        }
#pragma unroll
        for (int i = 0; i < G; ++i) {
            if (take[i] >> lane & 1ull) kept[at + __popcll(take[i] & ((1ull << lane) - 1ull))] = w0 + 64 * i + lane;
            at += __popcll(take[i]);
        }
    }
}

// workgroups of a sequence: each passes over all its weights, so more only divide the writing
int weight_select_parts(int64_t B, int64_t max_kv) {
    return (int)std::max<int64_t>(1, std::min<int64_t>({WS_MAX_PARTS, 256 / B, (max_kv + WS_CAP - 1) / WS_CAP}));
}

hipError_t launch_weight_select(const WeightSelArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(weight_select_kernel, dim3((unsigned)((a.B + 7) / 8 * 8 * a.parts)), dim3(WS_THREADS), 0, s, a);
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
// step; then rows go through registers, all of a wave's loads in flight.  Measured: 16
// sequences cut to 1024 rows 9.9 us (37 MB, 3.7 TB/s), one 7.6 us (the launch and the
// chain of searches).

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
    const uint32_t nw = (uint32_t)(a.keep + EV_SLOTS - 1) / EV_SLOTS, wg = workgroup_id();
    if (wg >= (uint32_t)a.B * nw) return;
    const int b = (int)(wg / nw), j0 = (int)(wg % nw) * EV_SLOTS;
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
            // not a row, or not above the entry before it: nothing is moved
            if (src != j && (src < n || src >= kv || (p > 0 && kept[p - 1] >= src))) src = -1;
        }
    }
    const float weight = a.weight_out && src >= 0 ? a.weight[(int64_t)b * a.wstride + src] : 0.f;
    // where the rows lie; one whose page, or whose slot's page, does not exist is in no slot
    int64_t from = -1, to = -1;
    if (src >= 0) {
        const int32_t ps = table[src >> a.shift], pd = table[(j0 + lane) >> a.shift];
        if ((uint32_t)ps >= (uint32_t)a.n_pages || (uint32_t)pd >= (uint32_t)a.n_pages) {
            src = -1;
        } else if (src != j0 + lane) {
            from = (int64_t)ps * a.ps + (int64_t)(src & a.page_mask) * a.rs;
            to = (int64_t)pd * a.ps + (int64_t)((j0 + lane) & a.page_mask) * a.rs;
        }
    }
    u32x4_t piece[EV_LOADS];
    int64_t dst[EV_LOADS];
#pragma unroll
    for (int i = 0; i < EV_LOADS; ++i) {
        const int q = 64 * i + lane, r = q / (D_ROW / 8), p = q % (D_ROW / 8);
        const int64_t f = __shfl(from, r), t = __shfl(to, r);
        dst[i] = f >= 0 ? t + 8 * p : -1;
        piece[i] = f >= 0 ? *reinterpret_cast<const u32x4_t*>(a.cache + f + 8 * p) : u32x4_t{0, 0, 0, 0};
    }
    if (lane < EV_SLOTS && j0 + lane < a.keep) {
        const int64_t at = (int64_t)b * a.keep + j0 + lane;
        if (a.origin) a.origin[at] = src;
        if (a.weight_out) a.weight_out[at] = src >= 0 ? weight : 0.f;
    }
#pragma unroll
    for (int i = 0; i < EV_LOADS; ++i)
        if (dst[i] >= 0) *reinterpret_cast<u32x4_t*>(a.cache + dst[i]) = piece[i];
}

int64_t evict_waves(int64_t keep) { return (keep + EV_SLOTS - 1) / EV_SLOTS; }

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(evict_kernel, grid_of(a.B * evict_waves(a.keep)), dim3(64), 0, s, a);
    return hipGetLastError();
}

}  // namespace vkv
