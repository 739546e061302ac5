// k_weight.hip -- accumulated attention weights of the rows of a paged latent
// cache (gfx950).
//
//   weight[u] = decay * prev[u] + sum_{i, h: u seen} exp(scale * (q_lat . c_u + q_rope . r_u) - lse_ih)
//
// The attention's log-sum-exp is given, so one product S = Q K^T and one
// exponential per score are left: a lane has one cache row (its column of the product) and
// 16 queries a tile, so the sum over the queries is in-lane but for one swap of the lane
// halves, and over tiles or waves.  With many queries the cache rows stay in registers and
// the queries pass by, with few the other way round.  Sums: fp32, 16 terms of a tile first.
// Nothing is added atomically: the same inputs give the same bits.
#include <algorithm>

#include "vkv_pages.h"

namespace vkv {

constexpr int WT_WAVES = 4, WT_THREADS = 64 * WT_WAVES;
constexpr int WT_TILE = 32;                              // queries of a tile
constexpr int WT_STAGE = WT_TILE * 2 * D_ROW;
constexpr int WT_KS = D_ROW / 16;
static_assert(D_LAT == 512 && D_ROW == 576 && WT_TILE == 32 && WT_WAVES == 4, "a latent row per load; one rope load a wave");

// rows new in this chunk start at 0; a sequence without new tokens keeps its weights
__device__ __forceinline__ void finish(const WeightArgs& w, int b, int u, int kv, int old, float sum) {
    const int64_t at = (int64_t)b * w.stride + u;
    if (old == kv)
        w.weight[at] = w.prev ? w.prev[at] : 0.f;
    else
        w.weight[at] = w.prev && w.decay != 0.f && u < old ? __builtin_fmaf(w.decay, w.prev[at], sum) : sum;
}

// --------------------------------------------------------------- many queries
//
// Each of 4 waves holds 64 cache rows (576 dims: 288 of its 512 registers), so that a query
// tile read from LDS feeds two products: with 32 rows a wave, LDS takes as long as the
// matrix cores.  One workgroup per CU then, and the wave overlaps by itself: the scores of a
// tile become weights, and the loads and operand reads of later ones are issued, between the
// products of the present one.  (The products are written as instructions: the scores stay
// in vector registers, most of the cache rows in the accumulation registers.)  One barrier
// per tile; the operand reads run on over it.
//
// The work is cut into WW_RUNS equal runs of (block of 256 rows, query tile) pairs, as the
// device's lengths give it, one workgroup each: no last round of blocks on part of the chip,
// and the workgroups load their rows at different times.  A block that several runs share
// gets its parts through the workspace, added in order by a second kernel.
//
// Measured at 32 tokens of 64 heads over 4 x 65536 rows (lengths from 50021): 451 to 478 us by
// card, 1.06 to 1.13 PFLOP/s, at 2.0 GHz with the matrix cores busy for 53% of the cycles (32 rows a
// wave, two workgroups per CU: 589 us; rows loaded as operands, 15.5 us a block, instead of whole: 485 us).

constexpr int WW_ROWS = 64 * WT_WAVES;                   // cache rows of a block
constexpr int WW_STAGES = 4;
constexpr int WW_LAT = WT_TILE * 2 * D_LAT;              // latent panel: rows of 1 KB; then rows of 128 bytes
constexpr int WW_SD = 5;                                 // operands read ahead of the matrix cores
constexpr int WW_LSE = 4;                                // lse slots of a wave, of 256 bytes
constexpr int WW_ACC = 8;                                // K operands in vector registers, the others in accumulation registers
constexpr int WW_RUNS = 256;
constexpr int WW_LOAD = 3;                               // loading a block's rows counts as so many tiles
static_assert(WT_KS % (WW_SD + 1) == 0, "operands keep their registers from tile to tile");
static_assert((WW_ROWS * WT_TILE) % (WT_TILE * WT_TILE) == 0, "whole tiles per block of new rows and head");

// A sequence's blocks and their query tiles: all ntile for the first `full` blocks; those of the new rows are not
// seen by the first tokens, and begin at tile first, first + step, ... (`some` of them; the rows of tokens past the
// first max_q are seen by none)
struct WeightSpan {
    int kv, nq, old, nblk, ntile, full, first, step, some;
    int64_t cost;             // tiles in all, with WW_LOAD a block before its own (one of a sequence without new tokens)
    int64_t tok0;
    __device__ __forceinline__ int64_t later(int64_t j) const {   // tiles of the first j blocks after the full ones
        const int64_t i = min(j, (int64_t)some);
        return j * WW_LOAD + i * (ntile - first) - (int64_t)step * (i * (i - 1) / 2);
    }
};
__device__ __forceinline__ WeightSpan weight_span(const ChunkArgs& a, int b) {
    WeightSpan s;
    s.kv = min(max(a.kv_len[b], 0), a.max_kv);
    s.tok0 = min(max((int64_t)a.cu[b], (int64_t)0), a.n_tok);
    const int64_t tok1 = min(max((int64_t)a.cu[b + 1], s.tok0), a.n_tok);
    s.nq = (int)min(tok1 - s.tok0, (int64_t)a.max_q);
    s.nblk = (s.kv + WW_ROWS - 1) / WW_ROWS;
    s.ntile = max((s.nq * a.H + WT_TILE - 1) / WT_TILE, 1);
    s.old = rows_before(s.kv, tok1 - s.tok0, a.max_q);
    s.full = s.old < 0 ? 0 : min(s.nblk, s.old / WW_ROWS + 1);
    s.first = s.full < s.nblk ? (int)((int64_t)(s.full * WW_ROWS - s.old) * a.H / WT_TILE) : 0;
    s.step = WW_ROWS / WT_TILE * a.H;
    s.some = min(s.nblk - s.full, (max(s.ntile - s.first, 0) + s.step - 1) / s.step);
    s.cost = (int64_t)s.full * (s.ntile + WW_LOAD) + s.later(s.nblk - s.full);
    return s;
}

// The block of a sequence's tile `off` (< cost): its first tile, and off's place and the number of tiles in it
struct WeightPlace {
    int blk, t0;
    int64_t k, n;
};
__device__ __forceinline__ WeightPlace weight_place(const WeightSpan& s, int64_t off) {
    WeightPlace p;
    const int each = s.ntile + WW_LOAD;
    if (off < (int64_t)s.full * each) {
        p.blk = (int)(off / each);
        p.t0 = 0;
        p.k = off - (int64_t)p.blk * each;
    } else {
        off -= (int64_t)s.full * each;
        int lo = 0, hi = s.nblk - s.full;      // later(lo) <= off < later(hi)
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (s.later(mid) <= off) lo = mid;
            else hi = mid;
        }
        p.blk = s.full + lo;
        p.t0 = s.first + s.step * min(lo, s.some);     // (behind the last tile: none)
        p.k = off - s.later(lo);
    }
    p.n = max(s.ntile - p.t0, 0) + WW_LOAD;
    return p;
}

__device__ __forceinline__ int64_t uniform64(int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)((uint64_t)v >> 32)) << 32 |
                     (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}

// The sum of cost(b) over all sequences; the sequence that holds place x = at(sum) (x < sum), and x's place in it.
template <int THREADS>
struct WeightFind {
    int64_t sum[THREADS + 1];
    int64_t off;
    int b;
};
template <int THREADS, typename Cost, typename At>
__device__ __forceinline__ int64_t weight_find(int B, WeightFind<THREADS>& f, Cost cost, At at, int& b, int64_t& off) {
    const int tid = threadIdx.x, per = (B + THREADS - 1) / THREADS;
    const int b0 = min(tid * per, B), b1 = min(b0 + per, B);
    int64_t mine = 0;
    for (int i = b0; i < b1; ++i) mine += cost(i);
    f.sum[tid + 1] = mine;
    if (tid == 0) f.sum[0] = 0;
    for (int d = 1; d < THREADS; d *= 2) {
        __syncthreads();
        const int64_t v = tid + 1 > d ? f.sum[tid + 1 - d] : 0;
        __syncthreads();
        f.sum[tid + 1] += v;
    }
    if (tid == 0) f.b = 0, f.off = 0;
    __syncthreads();
    const int64_t total = f.sum[THREADS], x = at(total);
    if (f.sum[tid] <= x && x < f.sum[tid + 1]) {
        int64_t o = x - f.sum[tid];
        int i = b0;
        for (; i + 1 < b1; ++i) {
            const int64_t c = cost(i);
            if (o < c) break;
            o -= c;
        }
        f.b = i;
        f.off = o;
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(f.b);
    off = uniform64(f.off);
    return uniform64(total);
}
__device__ __forceinline__ int64_t run_start(int64_t total, int r) {
    return total / WW_RUNS * r + total % WW_RUNS * r / WW_RUNS;
}

__global__ __launch_bounds__(WT_THREADS, 1) void weight_many_kernel(WeightArgs w) {
    __shared__ __align__(256) uint8_t smem[WW_STAGES * WT_STAGE + WT_WAVES * WW_LSE * 256];   // tiles, then their lse values
    __shared__ WeightFind<WT_THREADS> find;
    const ChunkArgs& a = w.c;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), run = blockIdx.x;
    int b;
    int64_t off;
    const int64_t total = weight_find<WT_THREADS>(
        a.B, find, [&](int i) { return weight_span(a, i).cost; }, [&](int64_t n) { return run_start(n, run); }, b, off);
    int64_t left = run_start(total, run + 1) - run_start(total, run);
    while (left > 0) {
        const WeightSpan sp = weight_span(a, b);
        if (off >= sp.cost) {
            ++b;
            off = 0;
            continue;
        }
        const WeightPlace pl = weight_place(sp, off);
        const int n = (int)min(pl.n - pl.k, left);       // tiles of this block
        off += n;
        left -= n;
        const int kv = __builtin_amdgcn_readfirstlane(sp.kv), nq = __builtin_amdgcn_readfirstlane(sp.nq), nrow = nq * a.H;
        const int old = __builtin_amdgcn_readfirstlane(sp.old);
        const int blk = __builtin_amdgcn_readfirstlane(pl.blk);
        const int k0 = __builtin_amdgcn_readfirstlane((int)pl.k) - WW_LOAD, first = __builtin_amdgcn_readfirstlane(pl.t0);
        const int t0 = first + max(k0, 0), t1 = nq > 0 ? first + max(k0 + n, 0) : t0;
        const int64_t tok0 = sp.tok0;
        const int uw = WW_ROWS * blk + 64 * wave;        // the wave's first cache row; this lane's: uw + c and uw + 32 + c
        const uint16_t* ql = a.q_lat + tok0 * a.H * a.qls;
        const uint16_t* qr = a.q_rope + tok0 * a.H * a.qrs;
        const float* lse = w.lse + tok0 * a.H;
        // This wave's loads of tile t, i = 0 .. 9 in order: latent rows wave + 4 i, then a quarter of the rope rows, then
        // the lse (each wave's own copy).  Slot j of a latent row holds piece j ^ (row mod 16), of a rope row piece
        // j ^ (row / 2 mod 8): LDS serves a 128-bit read 16 lanes at a time, lanes {0-3, 12-15, 20-27} or the others of a
        // half wave, and their slots then differ modulo 16.  Rows past the end repeat an earlier one, not counted.
        const uint8_t* lat_row = nullptr;         // (scalar) the next latent row
        const int64_t next_row = 8 * a.qls;       // bytes
        auto seek = [&](int t, auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            const int R = WT_TILE * t + wave + 4 * i;
            if constexpr (i == 0) lat_row = reinterpret_cast<const uint8_t*>(ql + (int64_t)min(R, nrow - 1) * a.qls);
            else if constexpr (i < 8) lat_row += R < nrow ? next_row : 0;
            if constexpr (i < 8) asm volatile("" : "+s"(lat_row));
        };
        auto issue = [&](int t, int s, int slot, auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            uint8_t* st = smem + s * WT_STAGE;
            if constexpr (i < 8) {
                const int r = wave + 4 * i;
                uint32_t at;                      // (computed here each time: not kept for every i across the loop)
                asm volatile("v_xor_b32 %0, %1, %2" : "=v"(at) : "s"(16 * (r & 15)), "v"(16 * lane));
                __builtin_amdgcn_global_load_lds((gbl_void_t*)(lat_row + at), (lds_void_t*)(st + 1024 * r), 16, 0, 0);
            } else if constexpr (i == 8) {
                const int r = 8 * wave + (lane >> 3), R = min(WT_TILE * t + r, nrow - 1);
                __builtin_amdgcn_global_load_lds((gbl_void_t*)(qr + (int64_t)R * a.qrs + 8 * ((lane & 7) ^ ((r >> 1) & 7))),
                                                 (lds_void_t*)(st + WW_LAT + 1024 * wave), 16, 0, 0);
            } else {
                const int R = min(WT_TILE * t + c, nrow - 1);
                __builtin_amdgcn_global_load_lds((gbl_void_t*)(lse + R),
                                                 (lds_void_t*)(smem + WW_STAGES * WT_STAGE + 256 * (WW_LSE * wave + (slot & (WW_LSE - 1)))), 4, 0, 0);
            }
        };

        // K operand: cache row uw + 32 g + c, dims 16 ks + 8 hh .. +8 (rows past the end repeat the last one; a page
        // that does not exist: any row of the cache, not counted)
        bool there[2];
        const uint16_t* row[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int uc = min(uw + 32 * g + c, kv - 1);
            const int32_t page = a.table[(int64_t)b * a.tstride + (uc >> a.shift)];
            there[g] = (uint32_t)page < (uint32_t)a.n_pages;
            row[g] = a.cache + (there[g] ? 8 * ((int64_t)page * a.ps16 + (int64_t)(uc & a.page_mask) * a.rs16) : 0);
        }
        float sum[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) sum[g] = 0.f;
        if (t0 < t1) {
            uint32_t lat[8], rope[4];   // operand of tile row c, piece 2 ks + hh, in a stage: latent ks mod 8, rope
#pragma unroll
            for (int i = 0; i < 8; ++i) lat[i] = c * 1024 + 16 * ((2 * i + hh) ^ (c & 15));
#pragma unroll
            for (int i = 0; i < 4; ++i) rope[i] = WW_LAT + c * 128 + 16 * ((2 * i + hh) ^ ((c >> 1) & 7));
            wg_barrier();      // every wave is done with the stages (of the block before)
            // The cache rows come through the wave's own stage, laid out like a tile, 32 at a time: whole rows, which
            // direct loads fetch three times as fast as operands (32 bytes of a row a load) do.
            bf16x8_t kf[2][WT_KS];
            uint8_t* own = smem + wave * WT_STAGE;
            static_assert(WT_WAVES == WW_STAGES, "a stage for each wave");
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const uint64_t mine = (uint64_t)row[g];
                int ln = lane;
                asm volatile("" : "+v"(ln));     // nothing of this is kept from block to block
#pragma unroll 2
                for (int r = 0; r < 32; ++r) {
                    const uint8_t* base = (const uint8_t*)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), r) << 32 |
                                                           (uint32_t)__builtin_amdgcn_readlane((int)mine, r));
                    __builtin_amdgcn_global_load_lds((gbl_void_t*)(base + ((16u * ln) ^ (16u * (r & 15)))), (lds_void_t*)(own + 1024 * r), 16, 0, 0);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = 8 * j + (ln >> 3);
                    const uint64_t base = (uint64_t)(uint32_t)__shfl((int)(mine >> 32), r) << 32 | (uint32_t)__shfl((int)mine, r);
                    __builtin_amdgcn_global_load_lds((gbl_void_t*)(base + 2 * D_LAT + 16u * ((ln & 7) ^ ((r >> 1) & 7))),
                                                     (lds_void_t*)(own + WW_LAT + 1024 * j), 16, 0, 0);
                }
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
                for (int ks = 0; ks < WT_KS; ++ks)
                    kf[g][ks] = *reinterpret_cast<const bf16x8_t*>(own + (ks < 32 ? lat[ks & 7] + 256 * (ks >> 3) : rope[ks & 3]));
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
                for (int ks = 0; ks < WT_KS; ++ks) {    // read before the next rows come
                    if (g * WT_KS + ks < WW_ACC) asm volatile("" : "+v"(kf[g][ks])::"memory");
                    else asm volatile("" : "+a"(kf[g][ks])::"memory");
                }
            }
            wg_barrier();
            static_for<0, 10>([&](auto ic) { seek(t0, ic); issue(t0, 0, 0, ic); });
            static_for<0, 10>([&](auto ic) { seek(min(t0 + 1, t1 - 1), ic); issue(min(t0 + 1, t1 - 1), 1, 1, ic); });
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            wg_barrier();
            const uint32_t lds0 = lds_addr(smem);
            bf16x8_t qf[WW_SD + 1];
            auto qload = [&](uint32_t st, auto kc) __attribute__((always_inline)) {
                constexpr int ks = decltype(kc)::value;
                if constexpr (ks < 32) qf[ks % (WW_SD + 1)] = lds_read128<256 * (ks >> 3)>(st + lat[ks & 7]);
                else qf[ks % (WW_SD + 1)] = lds_read128<0>(st + rope[ks - 32]);
            };
            // The scores of a tile become weights while the matrix cores work on the next one: y, with
            // the lse z4 of their queries (nothing pending: 0 and inf, whose weights are 0).
            f32x16_t xa[2], xb[2];
            f32x4_t z4[4];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
#pragma unroll
                for (int g = 0; g < 2; ++g) xb[g][i] = 0.f;
                z4[i >> 2][i & 3] = INFINITY;
            }
            auto weight = [&](float x, float l) __attribute__((always_inline)) {
                return __builtin_amdgcn_exp2f(__builtin_fmaf(x, a.scale_log2, -1.4426950408889634f * l));
            };
            // tiles [safe0, safe1) hold whole queries that see all of the wave's rows
            const int64_t full = a.H * ((int64_t)(uw + 63) - old);
            const int safe0 = ((int)max(min(full, (int64_t)nrow), (int64_t)0) + WT_TILE - 1) / WT_TILE, safe1 = nrow / WT_TILE;
            int s = 0;
            static_for<0, WW_SD>([&](auto kc) { qload(lds0, kc); });
            auto tile = [&](int t, f32x16_t (&x)[2], f32x16_t (&y)[2]) __attribute__((always_inline)) {
                const int sn = (s + 1) % WW_STAGES, sl = (s + 2) % WW_STAGES;
                const int tl = min(t + 2, t1 - 1);   // loaded (from the last tile but one on: once more, not used)
                const uint32_t st = lds0 + s * WT_STAGE, stn = lds0 + sn * WT_STAGE;
                s = sn;
                float add[2];
                static_for<0, WT_KS>([&](auto kc) {
                    constexpr int ks = decltype(kc)::value, KB = WT_KS - WW_SD;
                    if constexpr (ks == KB) {
                        // This wave's loads of the next tile have landed (those of the one after are in flight), every
                        // wave's have, and every wave is done with the tile before, whose stage the next tile's loads fill.
                        asm volatile("s_waitcnt vmcnt(10)" ::: "memory");
                        wg_barrier();
                    }
                    auto product = [&](auto gc) __attribute__((always_inline)) {
                        constexpr int g = decltype(gc)::value;
                        constexpr bool acc = g * WT_KS + ks >= WW_ACC;
                        const bf16x8_t& q = qf[ks % (WW_SD + 1)];
                        // (the first product waits for its operand)
                        constexpr int n = g == 1 ? 15 : WW_SD - 1 + (ks >= 34 ? 4 : 0);
                        if constexpr (ks == 0 && acc) asm volatile("s_waitcnt lgkmcnt(%3)\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(x[g]) : "v"(q), "a"(kf[g][ks]), "n"(n));
                        else if constexpr (ks == 0) asm volatile("s_waitcnt lgkmcnt(%3)\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(x[g]) : "v"(q), "v"(kf[g][ks]), "n"(n));
                        else if constexpr (g == 0 && acc) asm volatile("s_waitcnt lgkmcnt(%3)\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(x[g]) : "v"(q), "a"(kf[g][ks]), "n"(n));
                        else if constexpr (g == 0) asm volatile("s_waitcnt lgkmcnt(%3)\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(x[g]) : "v"(q), "v"(kf[g][ks]), "n"(n));
                        else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(x[g]) : "v"(q), "a"(kf[g][ks]));
                        __builtin_amdgcn_sched_barrier(0);
                    };
                    // The compiler does not see that results are in flight and would not wait before it reads or copies
                    // them: the statement of the last products ends when they are through (12 wait states after 8 passes).
                    // Between products nothing names their results (a test of the generated code holds it to that).
                    auto last_products = [&]() __attribute__((always_inline)) {
                        static_assert(WT_KS > WW_ACC, "their operands are in accumulation registers");
                        asm volatile("s_waitcnt lgkmcnt(%5)\n\tv_mfma_f32_32x32x16_bf16 %0, %2, %3, %0\n\tv_mfma_f32_32x32x16_bf16 %1, %2, %4, %1\n\ts_nop 13"
                                     : "+v"(x[0]), "+v"(x[1]) : "v"(qf[(WT_KS - 1) % (WW_SD + 1)]), "a"(kf[0][WT_KS - 1]), "a"(kf[1][WT_KS - 1]), "n"(WW_SD - 1 + 4));
                        __builtin_amdgcn_sched_barrier(0);
                    };
                    // A wave issues in order, and the second product when the first one's passes are over: what
                    // stands between them, and after them, is to fit into 32 cycles each.
                    if constexpr (ks < WT_KS - 1) product(std::integral_constant<int, 0>{});
                    if constexpr (ks == 0) {
#pragma unroll
                        for (int g = 0; g < 2; ++g) asm volatile("" : "+v"(y[g]));
                    }
                    if constexpr (ks >= 1 && ks <= 32) {
                        constexpr int g = (ks - 1) % 2, i = (ks - 1) / 2;
                        const float p = weight(y[g][i], z4[i >> 2][i & 3]);
                        add[g] = i ? add[g] + p : p;
                        asm volatile("" : "+v"(add[g]));   // here, not after the products
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (ks < WT_KS - 1) product(std::integral_constant<int, 1>{});
                    else last_products();
                    if constexpr (ks < KB) qload(st, std::integral_constant<int, ks + WW_SD>{});
                    else qload(stn, std::integral_constant<int, ks - KB>{});
                    if constexpr (ks == 33) {
                        // the lse of tile rows 8 i4 + 4 hh .. +3
                        const uint32_t la = lds0 + WW_STAGES * WT_STAGE + 256 * (WW_LSE * wave + ((t - t0) & (WW_LSE - 1))) + 16 * hh;
                        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:32\n\tds_read_b128 %2, %4 offset:64\n\t"
                                     "ds_read_b128 %3, %4 offset:96"
                                     : "=&v"(z4[0]), "=&v"(z4[1]), "=&v"(z4[2]), "=&v"(z4[3])
                                     : "v"(la));
                    }
                    if constexpr (ks % 3 == 1 && ks < 30) seek(tl, std::integral_constant<int, ks / 3>{});
                    if constexpr (ks % 3 == 2 && ks < 30) issue(tl, sl, t - t0 + 2, std::integral_constant<int, ks / 3>{});
                    __builtin_amdgcn_sched_barrier(0);
                });
                asm volatile("s_waitcnt lgkmcnt(2)" : "+v"(z4[0]), "+v"(z4[1]), "+v"(z4[2]), "+v"(z4[3]));
#pragma unroll
                for (int g = 0; g < 2; ++g) sum[g] += add[g];
                float low = z4[0][0];   // -inf: a query without weights
#pragma unroll
                for (int i = 1; i < 16; ++i) low = fminf(low, z4[i >> 2][i & 3]);
                // x[i] = score of query row 32 t + 8 (i / 4) + 4 hh + i % 4 and cache row u.  Rows the tile's first token
                // does not see, rows past the last query, or a query without weights: at once, score by score
                if (t < safe0 || t >= safe1 || __ballot(low == -INFINITY) != 0) {
                    int ln = lane;
                    asm volatile("" : "+v"(ln));     // nothing of this is kept across the loop
                    const int r0 = WT_TILE * t + 4 * (ln >> 5);
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        // the first query row that sees cache row u (none sees those from kv on)
                        const int first = a.H * min(max(uw + 32 * g + (ln & 31) - old, 0), nq);
                        float part = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int R = r0 + 8 * (i >> 2) + (i & 3);
                            const float l = z4[i >> 2][i & 3], p = weight(x[g][i], l);
                            if (R < nrow && R >= first && l != -INFINITY) part += p;
                            x[g][i] = 0.f;
                        }
                        sum[g] += part;
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) z4[i >> 2][i & 3] = INFINITY;
                }
            };
            auto rest = [&](f32x16_t (&y)[2]) __attribute__((always_inline)) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
                for (int i = 0; i <= WW_SD; ++i) lds_wait<0>(qf[i]);   // the reads after the last tile
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    float add = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) add += weight(y[g][i], z4[i >> 2][i & 3]);
                    sum[g] += add;
                }
            };
            for (int t = t0;; t += 2) {
                tile(t, xa, xb);
                if (t + 1 >= t1) {
                    rest(xa);
                    break;
                }
                tile(t + 1, xb, xa);
                if (t + 2 >= t1) {
                    rest(xb);
                    break;
                }
            }
        }
        // a block within one run is done; the others' sums: the run's first block that began in an earlier one, and its last
        const bool whole = pl.k == 0 && n == pl.n;
        float* slot = w.part + (int64_t)(2 * run + (pl.k == 0)) * WW_ROWS + 64 * wave + c;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int u = uw + 32 * g + c;
            float sums = half_sum(sum[g]);
            if (!there[g]) sums = 0.f;
            if (hh == 1) continue;
            if (!whole) slot[32 * g] = sums;
            else if (u < kv) finish(w, b, u, kv, old, sums);
        }
    }
}

// The sums of the blocks that begin in run blockIdx.x and end in a later one.
__global__ __launch_bounds__(WW_ROWS) void weight_join_kernel(WeightArgs w) {
    __shared__ WeightFind<WW_ROWS> find;
    const int run = blockIdx.x;
    int b;
    int64_t off;
    const int64_t total = weight_find<WW_ROWS>(
        w.c.B, find, [&](int i) { return weight_span(w.c, i).cost; },
        [&](int64_t n) { return max(run_start(n, run + 1) - 1, (int64_t)0); }, b, off);
    const int64_t x0 = run_start(total, run), x1 = run_start(total, run + 1);
    if (x0 == x1) return;
    const WeightSpan sp = weight_span(w.c, b);
    const WeightPlace pl = weight_place(sp, off);        // of the run's last tile
    const int64_t end = x1 - 1 - pl.k + pl.n;
    if (x1 - 1 - pl.k < x0 || end <= x1) return;
    const int row = threadIdx.x, u = WW_ROWS * pl.blk + row;
    float sum = w.part[(int64_t)(2 * run + 1) * WW_ROWS + row];
    for (int r = run + 1; r < WW_RUNS && run_start(total, r) < end; ++r)
        if (run_start(total, r) < run_start(total, r + 1)) sum += w.part[(int64_t)(2 * r) * WW_ROWS + row];
    if (u < sp.kv) finish(w, b, u, sp.kv, sp.old, sum);
}

// ---------------------------------------------------------------- few queries
//
// Up to 256 (token, head) rows, 32 of them in the registers of each wave (the A operand),
// and the cache passes by once: tiles of 32 rows through LDS stages by direct loads, three
// tiles ahead where all 8 waves hold queries; with up to 128 rows two streams of 4 waves
// take the tiles in turn, one tile ahead each.  Reading the cache is the bound: every CU
// takes an equal run of all sequences' tiles.  A wave's sums over its queries meet those of
// the others through LDS, one tile later.
//
// Measured at one token of 128 heads over 16 x 32768 rows: 117 us, 5.2 TB/s.  (Rows held in
// registers as with many queries, two workgroups of 128 rows per CU: 157 us, 3.8 TB/s.)

constexpr int WF_WAVES = 8, WF_THREADS = 64 * WF_WAVES, WF_STAGES = 4;
constexpr int WF_OFF_SUM = WF_STAGES * CK_STAGE;                      // [2][wave][32]: sums of the waves' queries
constexpr int WF_OFF_GONE = WF_OFF_SUM + 2 * WF_WAVES * 32 * 4;       // per stage and wave: which of its tile rows do not exist
constexpr int WF_OFF_PREV = WF_OFF_GONE + WF_STAGES * WF_WAVES * 4;   // the old weights of the rows of 8 tiles: a tile's are read after
constexpr int WF_SMEM = WF_OFF_PREV + 2 * WF_STAGES * 256;            // its stage is loaded again

template <int QW>   // waves of a stream
__global__ __launch_bounds__(WF_THREADS, 2) void weight_few_kernel(WeightArgs w) {
    __shared__ __align__(256) uint8_t smem[WF_SMEM];
    __shared__ WeightFind<WF_THREADS> find;
    constexpr int KSTR = WF_WAVES / QW, PD = WF_STAGES / KSTR - 1;   // streams; tiles loaded ahead
    const ChunkArgs& a = w.c;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), run = blockIdx.x;
    const int qw = wave % QW, ks0 = wave / QW;
    const uint32_t lds0 = lds_addr(smem);
    auto rows_of = [&](int b) { return min(max(a.kv_len[b], 0), a.max_kv); };
    auto tiles_of = [&](int b) { return (int64_t)((rows_of(b) + CK_TILE - 1) / CK_TILE); };
    int b;
    int64_t off;
    const int64_t total = weight_find<WF_THREADS>(a.B, find, tiles_of, [&](int64_t n) { return run_start(n, run); }, b, off);
    int64_t left = run_start(total, run + 1) - run_start(total, run);
    while (left > 0) {
        const int kv = rows_of(b), tiles = (kv + CK_TILE - 1) / CK_TILE;
        if (off >= tiles) {
            ++b;
            off = 0;
            continue;
        }
        const int t0 = (int)off, t1 = (int)min((int64_t)tiles, off + left);
        left -= t1 - t0;
        off = t1;
        const int64_t tok0 = min(max((int64_t)a.cu[b], (int64_t)0), a.n_tok);
        const int64_t tok1 = min(max((int64_t)a.cu[b + 1], tok0), a.n_tok);
        const int nq = (int)min(tok1 - tok0, (int64_t)a.max_q), nrow = nq * a.H, before = rows_before(kv, tok1 - tok0, a.max_q);
        if (nq == 0) {
            for (int u = CK_TILE * t0 + tid; u < min(CK_TILE * t1, kv); u += WF_THREADS) finish(w, b, u, kv, before, 0.f);
            continue;
        }
        const int nw = (nrow + 31) / 32;             // waves of a stream that have queries
        const int row0 = 32 * qw;
        const bool idle = row0 >= nrow;
        const int nit = (t1 - t0 + KSTR - 1) / KSTR;   // tiles of each stream, the last ones perhaps past t1
        auto tile_of = [&](int k) { return t0 + ks0 + KSTR * k; };
        auto stage_of = [&](int k) { return ks0 * (PD + 1) + k % (PD + 1); };
        auto gone_of = [&](int k) { return lds0 + WF_OFF_GONE + stage_of(k) * (WF_WAVES * 4); };
        TileLoader<QW> loader{a, (const_i32_t*)(a.table + (int64_t)b * a.tstride), kv, qw, lane, {}};
        auto prev_of = [&](int k) { return smem + WF_OFF_PREV + 256 * (ks0 * 2 * (PD + 1) + k % (2 * (PD + 1))); };
        const bool old = w.prev && w.decay != 0.f;
        auto issue = [&](int k) {   // tile k of the stream, and the table entries of the next one
            if (old && qw == 0) {
                const int u = min(CK_TILE * tile_of(k) + c, kv - 1);
                __builtin_amdgcn_global_load_lds((gbl_void_t*)(w.prev + (int64_t)b * w.stride + u), (lds_void_t*)prev_of(k), 4, 0, 0);
            }
            loader.issue(tile_of(k), smem + stage_of(k) * CK_STAGE, gone_of(k));
            loader.fetch(tile_of(k + 1));
        };
        // Q operand: query row row0 + c, dims 16 ks + 8 hh .. +8; rows past the end repeat the last one, not counted
        bf16x8_t qf[WT_KS];
        {
            const int64_t row = tok0 * a.H + min(row0 + c, nrow - 1);
            const uint16_t* ql = a.q_lat + row * a.qls + 8 * hh;
            const uint16_t* qr = a.q_rope + row * a.qrs + 8 * hh;
#pragma unroll
            for (int ks = 0; ks < WT_KS; ++ks)
                qf[ks] = *reinterpret_cast<const bf16x8_t*>(ks < D_LAT / 16 ? ql + 16 * ks : qr + 16 * ks - D_LAT);
        }
        // -lse log2 e of this lane's query rows row0 + 8 (i / 4) + 4 hh + i % 4 (-inf: none, or one without weights)
        float z[16];
        bool odd = row0 + 32 > nrow;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int R = row0 + 8 * (i >> 2) + 4 * hh + (i & 3);
            const float l = w.lse[tok0 * a.H + min(R, nrow - 1)];
            odd |= l == -INFINITY;
            z[i] = R < nrow && l != -INFINITY ? -1.4426950408889634f * l : -INFINITY;
        }
        const bool some = __ballot(odd) != 0;
        loader.fetch(tile_of(0));
        issue(0);
        if (PD > 1 && nit > 1) issue(1);
        if (PD > 2 && nit > 2) issue(2);
#pragma unroll
        for (int ks = 0; ks < WT_KS; ++ks) asm volatile("" : "+v"(qf[ks]));   // no wait for them inside the tile loop
#pragma unroll
        for (int i = 0; i < 16; ++i) asm volatile("" : "+v"(z[i]));

        // a tile's sums, over the waves in order (explicit LDS reads: the compiler would make its own wait for the
        // direct loads in flight)
        auto sum_of = [&](int k, int wv) { return lds0 + WF_OFF_SUM + 4 * (((k & 1) * WF_WAVES + wv) * 32 + c); };
        auto close = [&](int k) {
            const int u = CK_TILE * tile_of(k) + c;
            if (qw != k % QW || tile_of(k) >= t1) return;
            const uint32_t at = sum_of(k, ks0 * QW);
            float s[QW];
            static_for<0, QW>([&](auto ic) { s[decltype(ic)::value] = lds_read32<128 * decltype(ic)::value>(at); });
            float pv = lds_read32<0>(lds_addr(prev_of(k)) + 4 * c);
#pragma unroll
            for (int i = 0; i < QW; ++i) lds_wait<0>(s[i]);
            lds_wait<0>(pv);
            float sum = s[0];
#pragma unroll
            for (int i = 1; i < QW; ++i) sum += i < nw ? s[i] : 0.f;
            if (old && u < before) sum = __builtin_fmaf(w.decay, pv, sum);
            if (lane < 32 && u < kv) w.weight[(int64_t)b * w.stride + u] = sum;
        };
        for (int k = 0; k < nit; ++k) {
            // this wave's share of tile k has landed (at most the loads of the PD - 1 tiles behind it are still
            // in flight), and every wave's; the stage loaded next is free
            if (PD > 1 && k + PD - 1 < nit)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PD > 1 ? (PD - 1) * loader.LOADS : 0) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            wg_barrier();
            if (k + PD < nit) issue(k + PD);
            if (k > 0) close(k - 1);
            const int t = tile_of(k), u0 = CK_TILE * t;
            if (t < t1 && !idle) {
                const uint32_t st = lds0 + stage_of(k) * CK_STAGE;
                uint32_t note;   // arrives ahead of the operands
                asm volatile("ds_read_b32 %0, %1" : "=v"(note) : "v"(loader.note(gone_of(k), lane)) : "memory");
                f32x16_t x;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = 0.f;
                {
                    constexpr int SD = 3;   // operands read ahead of the matrix cores
                    bf16x8_t kf[SD + 1];
                    int ln = lane;
                    asm volatile("" : "+v"(ln));   // nothing of the addresses is kept across the tiles
                    // K operand of (tile row c, piece 2 ks + hh), the piece's low bits permuted
                    const uint32_t ka = st + (ln & 31) * CK_LAT_BYTES + 16 * ((ln >> 5) ^ lat_xor(ln & 31));
                    const uint32_t ra = st + CK_OFF_ROPE + (ln & 31) * CK_ROPE_BYTES + 16 * ((ln >> 5) ^ rope_xor(ln & 31));
                    auto kload = [&](auto kc) {
                        constexpr int ks = decltype(kc)::value;
                        if constexpr (ks < D_LAT / 16) kf[ks % (SD + 1)] = lds_read128<256 * (ks >> 3)>(ka ^ (32 * (ks & 7)));
                        else kf[ks % (SD + 1)] = lds_read128<0>(ra ^ (32 * (ks - D_LAT / 16)));
                    };
                    static_for<0, SD>(kload);
                    static_for<0, WT_KS>([&](auto kc) {
                        constexpr int ks = decltype(kc)::value;
                        if constexpr (ks + SD < WT_KS) kload(std::integral_constant<int, ks + SD>{});
                        lds_wait<(ks + SD < WT_KS) ? SD : (WT_KS - 1 - ks)>(kf[ks % (SD + 1)]);
                        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[ks], kf[ks % (SD + 1)], x, 0, 0, 0);
                    });
                    lds_wait<0>(note);
                }
                const uint32_t absent = loader.absent(note);   // tile rows on no page
                float sum = 0.f;
                if (some || u0 + CK_TILE - 1 > before + row0 / a.H) {   // rows that a query does not see, or odd ones
                    // the first query row that sees cache row u0 + c (none sees those from kv on)
                    const int first = a.H * min(max(u0 + c - before, 0), nq);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, z[i]));
                        if (row0 + 8 * (i >> 2) + 4 * hh + (i & 3) >= first && z[i] != -INFINITY) sum += p;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, z[i]));
                }
                sum = half_sum(sum);
                if ((absent >> c) & 1u) sum = 0.f;
                if (hh == 0) asm volatile("ds_write_b32 %0, %1" ::"v"(sum_of(k, wave)), "v"(sum) : "memory");
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wg_barrier();
        close(nit - 1);
        wg_barrier();      // the sums and the stages are free
    }
}

// More than 256 query rows of the longest chunk, which the few-queries form cannot hold.  At 256 (two tokens of 128 heads,
// one in every third sequence) it takes 162 us where runs take 215 (16 sequences of 32768 rows), 16 where they take 26 (one
// of 8192), 47 and 63 (64 of 2048).
static bool many_queries(int64_t H, int64_t max_q) { return max_q * H > 32 * WF_WAVES; }

size_t weight_workspace_bytes(int64_t H, int64_t max_q) {
    return many_queries(H, max_q) ? (size_t)2 * WW_RUNS * WW_ROWS * sizeof(float) : 0;
}

hipError_t launch_weight(const WeightArgs& w, hipStream_t s) {
    if (!many_queries(w.c.H, w.c.max_q)) {
        if ((int64_t)w.c.max_q * w.c.H > 128)
            hipLaunchKernelGGL((weight_few_kernel<8>), dim3(WW_RUNS), dim3(WF_THREADS), 0, s, w);
        else
            hipLaunchKernelGGL((weight_few_kernel<4>), dim3(WW_RUNS), dim3(WF_THREADS), 0, s, w);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(weight_many_kernel, dim3(WW_RUNS), dim3(WT_THREADS), 0, s, w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(weight_join_kernel, dim3(WW_RUNS), dim3(WW_ROWS), 0, s, w);
    return hipGetLastError();
}

}  // namespace vkv
