// k_weight.hip -- accumulated attention weights of the rows of a paged latent
// cache (gfx950).
//
//   weight[u] = decay * prev[u] + sum_{i, h: u seen} exp(scale * (q_lat . c_u + q_rope . r_u) - lse_ih)
//
// The attention's log-sum-exp is given, so one product S = Q K^T and one
// exponential per score are left.  Work split: workgroup = 128 cache rows, two of
// them per CU (one loads its rows while the other computes); each of 4 waves
// holds 32 rows (576 dims) in its registers as the B operand and the queries pass by: tiles
// of 32 (token, head) rows through two LDS stages by direct loads, one barrier per
// tile.  A lane then has one cache row (its column) and 16 queries: the sum over
// the queries is in-lane but for one swap of the lane halves at the end.  Every
// row's sum belongs to one workgroup; where there are few cache rows the queries
// are cut into parts as well, and a second kernel adds those in order.  Nothing
// is added atomically: the same inputs give the same bits.
// Sums: fp32, 16 terms of a tile first, then over the tiles.
#include <algorithm>

#include "vkv_tile.h"

namespace vkv {

constexpr int WT_WAVES = 4, WT_THREADS = 64 * WT_WAVES;
constexpr int WT_ROWS = 32 * WT_WAVES;                   // cache rows of a workgroup
constexpr int WT_TILE = 32;                              // queries of a tile
constexpr int WT_PIECES = D_ROW / 8;
constexpr int WT_ROW_BYTES = 2 * D_ROW;
constexpr int WT_STAGE = WT_TILE * WT_ROW_BYTES;
constexpr int WT_LOADS = WT_STAGE / 1024 / WT_WAVES;     // 9 loads of 1 KB per wave
constexpr int WT_KS = D_ROW / 16;

__global__ __launch_bounds__(WT_THREADS, 2) void weight_kernel(WeightArgs w) {
    __shared__ __align__(256) uint8_t smem[2 * WT_STAGE + 2 * 256];   // tiles, then their lse values
    const ChunkArgs& a = w.c;
    const int nblk = w.nblk;
    const int z = blockIdx.x / (nblk * a.B), rest = blockIdx.x % (nblk * a.B);
    const int b = rest / nblk, u0 = (rest % nblk) * WT_ROWS;
    const int kv = min(max(a.kv_len[b], 0), a.max_kv);
    if (u0 >= kv) return;
    const int64_t tok0 = min(max((int64_t)a.cu[b], (int64_t)0), a.n_tok);
    const int64_t tok1 = min(max((int64_t)a.cu[b + 1], tok0), a.n_tok);
    const int nq = (int)min(tok1 - tok0, (int64_t)a.max_q), nrow = nq * a.H;

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int uw = u0 + 32 * wave;            // the wave's first cache row
    const int u = uw + c;                     // this lane's
    // the queries of this part that see some row of the block: those of the tokens from i0 on
    const int i0 = max(u0 - (kv - nq), 0);
    const int ntile = (nrow + WT_TILE - 1) / WT_TILE;
    const int per = (ntile + w.parts - 1) / w.parts;
    const int t0 = max(z * per, (int)((int64_t)i0 * a.H / WT_TILE)), t1 = min(z * per + per, ntile);

    const uint16_t* ql = a.q_lat + tok0 * a.H * a.qls;
    const uint16_t* qr = a.q_rope + tok0 * a.H * a.qrs;
    const float* lse = w.lse + tok0 * a.H;
    // this wave's loads of tile t: slot q = 72 r + p' holds piece p' ^ (r / 2 mod 8) of tile row r (LDS serves a
    // 128-bit read 16 lanes at a time, lanes {0-3, 12-15, 20-27} or the others of a half wave: their slots differ
    // modulo 16, odd rows lying 8 slots on)
    auto issue = [&](int t, int s) {
        uint8_t* st = smem + s * WT_STAGE;
        int ln = lane;
        asm volatile("" : "+v"(ln));   // keeps the slot arithmetic out of registers across the loop
#pragma unroll
        for (int i = 0; i < WT_LOADS; ++i) {
            const int j = wave + WT_WAVES * i, q = 64 * j + ln, r = q / WT_PIECES, p = (q - WT_PIECES * r) ^ ((r >> 1) & 7);
            const int64_t R = min(WT_TILE * t + r, nrow - 1);   // rows past the end repeat the last one, not counted
            const uint16_t* src = p < D_LAT / 8 ? ql + R * a.qls + 8 * p : qr + R * a.qrs + 8 * (p - D_LAT / 8);
            __builtin_amdgcn_global_load_lds((gbl_void_t*)src, (lds_void_t*)(st + 1024 * j), 16, 0, 0);
        }
        if (wave == 0) {
            const int R = min(WT_TILE * t + c, nrow - 1);
            __builtin_amdgcn_global_load_lds((gbl_void_t*)(lse + R), (lds_void_t*)(smem + 2 * WT_STAGE + 256 * s), 4, 0, 0);
        }
    };

    // K operand: cache row u, dims 16 ks + 8 hh .. +8 (rows past the end repeat the last one; a page that
    // does not exist: any row of the cache, not counted)
    const int uc = min(u, kv - 1);
    const int32_t page = a.table[(int64_t)b * a.tstride + (uc >> a.shift)];
    const bool there = (uint32_t)page < (uint32_t)a.n_pages;
    const uint16_t* row = a.cache + (there ? 8 * ((int64_t)page * a.ps16 + (int64_t)(uc & a.page_mask) * a.rs16) : 0) + 8 * hh;
    float sum = 0.f;
    if (t0 < t1) {
        issue(t0, 0);
        bf16x8_t kf[WT_KS];
#pragma unroll
        for (int ks = 0; ks < WT_KS; ++ks) kf[ks] = *reinterpret_cast<const bf16x8_t*>(row + 16 * ks);
#pragma unroll
        for (int ks = 0; ks < WT_KS; ++ks) asm volatile("" : "+v"(kf[ks]));   // no wait for them inside the tile loop

        const uint32_t lds0 = lds_addr(smem);
        uint32_t qaddr[4];   // Q operand of (tile row c, piece 2 ks + hh), the piece's low three bits permuted
#pragma unroll
        for (int i = 0; i < 4; ++i) qaddr[i] = c * WT_ROW_BYTES + 16 * ((2 * i + hh) ^ ((c >> 1) & 7));
        for (int t = t0; t < t1; ++t) {
            const int s = (t - t0) & 1;
            // this wave's loads of tile t have landed (nothing else is in flight), every wave's
            // have, and every wave is done with the stage loaded next
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            wg_barrier();
            if (t + 1 < t1) issue(t + 1, s ^ 1);
            const uint32_t st = lds0 + s * WT_STAGE;
            f32x16_t x;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = 0.f;
            // the lse of tile rows 8 i4 + 4 hh .. +3
            f32x4_t z4[4];
            const uint32_t la = lds0 + 2 * WT_STAGE + 256 * s + 16 * hh;
            asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:32\n\tds_read_b128 %2, %4 offset:64\n\t"
                         "ds_read_b128 %3, %4 offset:96\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(z4[0]), "=&v"(z4[1]), "=&v"(z4[2]), "=&v"(z4[3])
                         : "v"(la));
            {
                constexpr int SD = 4;   // operands read ahead of the matrix cores
                bf16x8_t qf[SD + 1];
                uint32_t qa[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) qa[i] = st + qaddr[i];
                auto qload = [&](auto kc) {
                    constexpr int ks = decltype(kc)::value;
                    qf[ks % (SD + 1)] = lds_read128<128 * (ks >> 2)>(qa[ks & 3]);
                };
                static_for<0, SD>(qload);
                static_for<0, WT_KS>([&](auto kc) {
                    constexpr int ks = decltype(kc)::value;
                    if constexpr (ks + SD < WT_KS) qload(std::integral_constant<int, ks + SD>{});
                    lds_wait<(ks + SD < WT_KS) ? SD : (WT_KS - 1 - ks)>(qf[ks % (SD + 1)]);
                    x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[ks % (SD + 1)], kf[ks], x, 0, 0, 0);
                });
            }
            // x[i] = score of query row 32 t + 8 (i / 4) + 4 hh + i % 4 and cache row u
            bool dead = false;   // a query without weights (its lse is -inf)
#pragma unroll
            for (int i = 0; i < 16; ++i) dead |= z4[i >> 2][i & 3] == -INFINITY;
            // rows the tile's first token does not see, rows past the last query, or such a query
            const bool masked = uw + 31 > kv - nq + WT_TILE * t / a.H || WT_TILE * t + WT_TILE > nrow || __ballot(dead) != 0;
            float add = 0.f;
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int R = WT_TILE * t + 8 * (i >> 2) + 4 * hh + (i & 3);
                    const float l = z4[i >> 2][i & 3];
                    const bool seen = R < nrow && u <= kv - nq + R / a.H && l != -INFINITY;
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, -l * 1.4426950408889634f));
                    if (seen) add += p;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    add += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, -z4[i >> 2][i & 3] * 1.4426950408889634f));
            }
            sum += add;
        }
    }
    sum = half_sum(sum);
    if (hh == 1 || u >= kv) return;
    if (!there) sum = 0.f;
    if (w.parts > 1) {
        w.part[((int64_t)z * a.B + b) * a.max_kv + u] = sum;
        return;
    }
    // rows new in this chunk start at 0; a sequence without new tokens keeps its weights
    const int64_t at = (int64_t)b * w.stride + u;
    const bool old = w.prev && u < kv - nq;
    if (nq == 0)
        w.weight[at] = w.prev ? w.prev[at] : 0.f;
    else
        w.weight[at] = old && w.decay != 0.f ? __builtin_fmaf(w.decay, w.prev[at], sum) : sum;
}

__global__ __launch_bounds__(256) void weight_join_kernel(WeightArgs w) {
    const ChunkArgs& a = w.c;
    const int nb = (a.max_kv + 255) / 256, b = blockIdx.x / nb, u = (blockIdx.x % nb) * 256 + threadIdx.x;
    const int kv = min(max(a.kv_len[b], 0), a.max_kv);
    if (u >= kv) return;
    const int64_t tok0 = min(max((int64_t)a.cu[b], (int64_t)0), a.n_tok);
    const int64_t tok1 = min(max((int64_t)a.cu[b + 1], tok0), a.n_tok);
    const int nq = (int)min(tok1 - tok0, (int64_t)a.max_q);
    float sum = 0.f;
    for (int z = 0; z < w.parts; ++z) sum += w.part[((int64_t)z * a.B + b) * a.max_kv + u];
    const int64_t at = (int64_t)b * w.stride + u;
    const bool old = w.prev && u < kv - nq;
    if (nq == 0)
        w.weight[at] = w.prev ? w.prev[at] : 0.f;
    else
        w.weight[at] = old && w.decay != 0.f ? __builtin_fmaf(w.decay, w.prev[at], sum) : sum;
}

// parts of the queries: enough workgroups for two per CU, but at least 8 tiles in a part
int64_t weight_parts(int64_t B, int64_t H, int64_t max_q, int64_t max_kv) {
    const int64_t blocks = B * ((max_kv + WT_ROWS - 1) / WT_ROWS), tiles = (max_q * H + WT_TILE - 1) / WT_TILE;
    return std::max<int64_t>(1, std::min(512 / std::max<int64_t>(blocks, 1), tiles / 8));
}

int64_t weight_blocks(int64_t max_kv) { return (max_kv + WT_ROWS - 1) / WT_ROWS; }

hipError_t launch_weight(const WeightArgs& w, hipStream_t s) {
    const int64_t n = (int64_t)w.nblk * w.c.B * w.parts;
    hipLaunchKernelGGL(weight_kernel, dim3((unsigned)n), dim3(WT_THREADS), 0, s, w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || w.parts == 1) return e;
    hipLaunchKernelGGL(weight_join_kernel, dim3((unsigned)((int64_t)w.c.B * ((w.c.max_kv + 255) / 256))), dim3(256), 0, s, w);
    return hipGetLastError();
}

}  // namespace vkv
