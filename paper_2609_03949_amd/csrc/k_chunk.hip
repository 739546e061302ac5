// k_chunk.hip -- attention of a chunk of new tokens over a paged latent cache
// (gfx950).
//
//   s_u = scale * (q_lat . c_u + q_rope . r_u),  u <= kv_len - nq + i,
//   o_i = sum_u softmax_u(s) c_u   (512 dims)
//
// All heads read the same cache rows, so the rows of the products are (token,
// head) pairs: row R of a sequence is head R % H of its new token R / H.  A unit
// is 16 QG of them; a workgroup of 8 waves takes a run of 32-row cache tiles of a
// unit.  A wave holds 16 rows: their queries (576 dims) and outputs (512 dims,
// fp32) stay in its registers (two waves per SIMD), as do the softmax weights: the
// accumulator layout of S^T = K Q^T is the B-operand layout of O^T = V^T P^T when
// the cache rows are fed to the K dimension in a permuted order, which the
// transposing V reads follow.  With QG = 8 the waves share every tile; with QG = 4
// and 2 (few rows: decode) they split into 8 / QG streams that take the tiles in
// turn, each in its own LDS stages, and join at the end through LDS.
//
// Cache rows go to LDS by direct loads, a row's 512 latent dims by one instruction whose
// address is scalar but for the lane; so are the table entries, a tile ahead.  (Row
// addresses per lane took 1100 vector cycles of a wave and tile, half its time.)
// Stage layout: [32 rows][512 dims], then [32 rows][64 dims], 16-byte pieces permuted
// within a row by an XOR with a function of the row that spreads the operand reads over
// the LDS banks.
//
// Work split: up to CK_MAX_UNITS units, the tiles of all units are laid end to end
// and cut into equal runs, at most one per CU, however the lengths differ; a run that
// covers part of a unit leaves (unnormalised O, reference maximum, sum) in fp32 and
// a second kernel joins the parts.  More units than that fill the chip by
// themselves: one workgroup each, the later rows (more tiles) first.
//
// Measured: 512 new tokens of 128 heads behind up to 16384 rows, 3 sequences: 4.43 ms, 1.12
// PFLOP/s (bound: LDS returns, 557 KB a tile at 128 bytes a cycle, 95% of the cycles); one token
// of 128 heads over 32 x 32768 rows 293 us, 0.8 PFLOP/s (the run 275, the join 18); one token of 16
// heads over 8192 rows 20.2 us: launches, and in the run 3 us before the loads are under
// way, 3 us for them and the tile, 4 us for the streams' join, 1 us of stores.
#include <algorithm>

#include "vkv_pages.h"

namespace vkv {

constexpr int CK_WAVES = 8;
constexpr int CK_THREADS = 64 * CK_WAVES;
constexpr int CK_STAGES = 4;
constexpr int CK_KS = D_ROW / 32, CK_DT = D_LAT / 16;
constexpr float CK_SLACK = 8.0f;   // lag allowed to the softmax reference maximum (log2 units)
constexpr float CK_ROOM = 0x1p-40f;   // careful passes and joins: a factor of the weights, so that no sum of finite values overflows
constexpr int CK_OFF_ML = CK_STAGES * CK_STAGE;          // (m, l) of the waves' rows
constexpr int CK_OFF_GONE = CK_OFF_ML + CK_WAVES * 16 * 8;   // per stage and wave: which of its tile rows do not exist
constexpr int CK_SMEM = CK_OFF_GONE + CK_STAGES * CK_WAVES * 4;

// ------------------------------------------------------------ units and runs

struct CkUnit {
    int b, row0, nrow;      // sequence, first row of the block, rows of the sequence
    int64_t tok0;           // first token of the sequence among the packed ones
    int nq, kv;             // new tokens (max_q at most) and cache rows of the sequence
    int old;                // its rows before the new tokens' (below 0: more tokens than rows)
};

__device__ __forceinline__ CkUnit chunk_unit(const ChunkArgs& a, int u, int rows) {
    CkUnit x;
    x.b = u / a.mb;
    x.row0 = (u - x.b * a.mb) * rows;
    const int64_t s = min(max((int64_t)a.cu[x.b], (int64_t)0), a.n_tok);
    const int64_t e = min(max((int64_t)a.cu[x.b + 1], s), a.n_tok);
    x.tok0 = s;
    x.nq = (int)min(e - s, (int64_t)a.max_q);
    x.nrow = x.nq * a.H;
    x.kv = min(max(a.kv_len[x.b], 0), a.max_kv);
    x.old = rows_before(x.kv, e - s, a.max_q);
    return x;
}

// tiles that some row of the block sees; a block of rows that see nothing counts
// one, so that its outputs are written; 0: no rows
__device__ __forceinline__ int unit_tiles(const ChunkArgs& a, const CkUnit& x, int rows) {
    if (x.row0 >= x.nrow) return 0;
    const int last = min(x.row0 + rows, x.nrow) - 1;
    const int seen = max(x.old + last / a.H + 1, 0);
    return max((seen + CK_TILE - 1) / CK_TILE, 1);
}

// Runs the tiles of all units are cut into: at most one per CU, and as a run costs its tiles
// (1.2 us each, or each round of one per stream) and its parts (written and read again: 256 KB,
// or that divided by the streams, 0.075 us of the join), about 4 sqrt(tiles) runs.  Their
// length is a power of two of rounds, so that fewer runs cover parts of two units.  One sequence
// of 32768 rows, 128 heads: 42 us with 128 runs of 8 tiles, 48 with 256; of 8192 rows 32 us
// with 64 of 4, 42 with 256; 16 heads of 32768 rows 29 us with 128, 34 with 256.
__device__ __forceinline__ int run_count(const ChunkArgs& a, int total) {
    int len = a.streams;
    while (2.0f * (float)len <= 0.3525f * sqrtf((float)total)) len *= 2;
    return min(max((total + len - 1) / len, 1), a.runs);
}
__device__ __forceinline__ int run_start(int g, int n, int total) { return (int)((int64_t)g * total / n); }

// ------------------------------------------------------------------ a segment

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));

// natural-log lse from the reference (log2 units) and the sum; nothing seen: -inf
__device__ __forceinline__ float lse_of(float m, float l) {
    return m == -INFINITY && l == 0.f ? -INFINITY : ((m == -INFINITY ? 0.f : m) + log2f(l)) * 0.69314718055994530942f;
}

// this lane's dims 16 dt + 4 g .. +3 of output row `row` (dt = at(0) .. at(N - 1)) from f times what
// o holds, and its lse if `first`; rows that see nothing: 0, -inf
template <int N, typename At>
__device__ __forceinline__ void store_row(const ChunkArgs& a, int64_t row, int g, float m, float l, float f,
                                          const f32x4_t (&o)[N], At at, bool first) {
    const bool none = m == -INFINITY && l == 0.f;
    const float inv = none ? 0.f : (1.0f / l) * f;
    uint16_t* out = a.out + row * D_LAT + 4 * g;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bf16x4_t v = {(__bf16)(o[i][0] * inv), (__bf16)(o[i][1] * inv), (__bf16)(o[i][2] * inv),
                            (__bf16)(o[i][3] * inv)};
        *reinterpret_cast<bf16x4_t*>(out + 16 * at(i)) = v;
    }
    if (g == 0 && first) a.lse[row] = lse_of(m, l);
}

// Tiles [t0, t1) of unit x by one workgroup.  part: where an incomplete unit's
// (O, m, l) go, or null (outputs).  Returns true, and stores nothing, when SAFE is
// false and a result is not finite: a masked row has weight 0 and 0 times a value
// that is not finite is not 0, so with SAFE the tiles that hold masked rows take
// those values apart; and weights above 1 may have made a sum overflow, so with
// SAFE they are small (by a power of two: the same bits but for weights and sums below
// 2^-86, whose roundings are of absolute size).  Parts whose O carries that factor have a
// negative l.
template <int QG, bool SAFE>
__device__ __forceinline__ bool chunk_segment(const ChunkArgs& a, const CkUnit& x, int t0, int t1, float* part_o,
                                              float* part_ml, uint8_t* smem) {
    constexpr int KSTR = CK_WAVES / QG;          // streams of tiles
    constexpr int PD = CK_STAGES / KSTR - 1;     // tiles loaded ahead: 3, 1, 0
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int qg = wave % QG, ks0 = wave / QG;
    const int R = x.row0 + 16 * qg + c;                         // this lane's row
    const int Rc = min(R, x.nrow - 1);                          // rows past the end repeat the last one, never stored
    const int lim = min(x.old + Rc / a.H, x.kv - 1);            // the last cache row it sees
    const int lim_lo = __builtin_amdgcn_readfirstlane(lim);     // of the wave's rows
    const int lim_hi = __builtin_amdgcn_readlane(lim, 15);
    const bool idle = x.row0 + 16 * qg >= x.nrow;
    const int nt = x.kv > 0 ? t1 - t0 : 0;
    const int nit = (nt + KSTR - 1) / KSTR;                     // tiles of each stream, the last ones perhaps past t1

    const uint32_t lds0 = lds_addr(smem);
    TileLoader<QG> loader{a, (const_i32_t*)(a.table + (int64_t)x.b * a.tstride), x.kv, qg, lane, {}};
    auto tile_of = [&](int k) { return t0 + ks0 + KSTR * k; };
    auto stage_of = [&](int k) { return ks0 * (PD + 1) + k % (PD + 1); };
    auto gone_of = [&](int k) { return lds0 + CK_OFF_GONE + stage_of(k) * (CK_WAVES * 4); };
    auto issue = [&](int k) {   // tile k of the stream, and the table entries of the next one
        loader.issue(tile_of(k), smem + stage_of(k) * CK_STAGE, gone_of(k));
        loader.fetch(tile_of(k + 1));
    };
    // Q^T operand: row R, dims 32 ks + 8 g .. +8
    bf16x8_t qf[CK_KS];
    {
        const int64_t row = x.tok0 * a.H + Rc;
        const uint16_t* ql = a.q_lat + row * a.qls + 8 * g;
        const uint16_t* qr = a.q_rope + row * a.qrs + 8 * g;
#pragma unroll
        for (int ks = 0; ks < CK_KS; ++ks)
            qf[ks] = *reinterpret_cast<const bf16x8_t*>(ks < D_LAT / 32 ? ql + 32 * ks : qr + 32 * ks - D_LAT);
    }
    if (nt > 0) {
        loader.fetch(tile_of(0));
        issue(0);
        if (PD > 1 && nit > 1) issue(1);
        if (PD > 2 && nit > 2) issue(2);
    }
#pragma unroll
    for (int ks = 0; ks < CK_KS; ++ks) asm volatile("" : "+v"(qf[ks]));   // no wait for them inside the tile loop

    // Operand addresses are recomputed from an opaque copy of the lane index, so that no
    // registers hold them across the loop.
    auto opaque_lane = [&]() {
        int ln = lane;
        asm volatile("" : "+v"(ln));
        return ln;
    };

    f32x4_t o[CK_DT];
#pragma unroll
    for (int dt = 0; dt < CK_DT; ++dt) o[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    for (int k = 0; k < nit; ++k) {
        // this wave's share of tile k has landed (at most the loads of the PD - 1 tiles behind it are
        // still in flight), and every wave's; the stage loaded next is free
        if (PD > 1 && k + PD - 1 < nit)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PD > 1 ? (PD - 1) * loader.LOADS : 0) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        wg_barrier();
        if (PD > 0 && k + PD < nit) issue(k + PD);
        const int t = tile_of(k), u0 = CK_TILE * t;
        if (t < t1 && !idle && u0 <= lim_hi) {
            const uint32_t st = lds0 + stage_of(k) * CK_STAGE;
            uint32_t note;   // arrives ahead of the K operands
            asm volatile("ds_read_b32 %0, %1" : "=v"(note) : "v"(loader.note(gone_of(k), lane)) : "memory");
            f32x4_t s[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
            {
                constexpr int SD = 2;   // operands read ahead of the matrix cores
                bf16x8_t kf[SD + 1][2];
                // K operand of (row 16 mt + c, piece 4 ks + g), the piece's low bits permuted
                const int ln = opaque_lane(), r = ln & 15;
                const uint32_t kaddr = r * CK_LAT_BYTES + 16 * ((ln >> 4) ^ lat_xor(r));
                const uint32_t raddr = CK_OFF_ROPE + r * CK_ROPE_BYTES + 16 * ((ln >> 4) ^ rope_xor(r));
                uint32_t ka[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) ka[i] = st + (kaddr ^ (64 * i));
                const uint32_t ra[2] = {st + raddr, st + (raddr ^ 64)};
                auto kload = [&](auto kc) {
                    constexpr int ks = decltype(kc)::value;
                    if constexpr (ks < D_LAT / 32) {
                        kf[ks % (SD + 1)][0] = lds_read128<256 * (ks >> 2)>(ka[ks & 3]);
                        kf[ks % (SD + 1)][1] = lds_read128<256 * (ks >> 2) + 16 * CK_LAT_BYTES>(ka[ks & 3]);
                    } else {
                        kf[ks % (SD + 1)][0] = lds_read128<0>(ra[ks & 1]);
                        kf[ks % (SD + 1)][1] = lds_read128<16 * CK_ROPE_BYTES>(ra[ks & 1]);
                    }
                };
                static_for<0, SD>(kload);
                static_for<0, CK_KS>([&](auto kc) {
                    constexpr int ks = decltype(kc)::value;
                    if constexpr (ks + SD < CK_KS) kload(std::integral_constant<int, ks + SD>{});
                    lds_wait<2 * ((ks + SD < CK_KS) ? SD : (CK_KS - 1 - ks))>(kf[ks % (SD + 1)][0], kf[ks % (SD + 1)][1]);
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt)
                        s[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[ks % (SD + 1)][mt], qf[ks], s[mt], 0, 0, 0);
                });
                lds_wait<0>(note);
            }
            const uint32_t absent = loader.absent(note);   // tile rows on no page
            const bool masked = u0 + CK_TILE - 1 > lim_lo || absent != 0;
            // s[mt][i] = score of tile row 16 mt + 4 g + i for row R
            if (masked) {
                const int last = lim - u0 - 4 * g;
                const uint32_t gone = absent >> (4 * g);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (16 * mt + i > last || ((gone >> (16 * mt + i)) & 1u)) s[mt][i] = -INFINITY;
            }
            float cmax = s[0][0];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) cmax = fmaxf(cmax, s[mt][i]);
            cmax = allreduce_groups(cmax, [](float p, float q) { return fmaxf(p, q); }) * a.scale_log2;
            const bool move = cmax > m_run + CK_SLACK;
            const float alpha = move ? __builtin_amdgcn_exp2f(m_run - cmax) : 1.0f;
            if (move) m_run = cmax;
            const float ref = m_run == -INFINITY ? 0.f : m_run;   // nothing but masked scores so far
            bf16x8_t pf;
            float psum = 0.f;
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][i], a.scale_log2, -ref));
                    psum += p;
                    pf[4 * mt + i] = (__bf16)(SAFE ? p * CK_ROOM : p);
                }
            l_run = l_run * alpha + psum;   // this lane's share of the sum
            if (__ballot(move)) {
#pragma unroll
                for (int dt = 0; dt < CK_DT; ++dt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[dt][i] *= alpha;
            }
            // the softmax's cross-lane reads complete before the V reads are issued
            asm volatile("" : "+v"(l_run), "+v"(pf));
            // V operand (transposing reads): lane 4 e + q of 16-lane group g reads rows 4 g + e and 16 + 4 g + e,
            // dims 16 dt + 4 q .. +3, i.e. piece 2 dt + q / 2, half q mod 2
            const int vl = opaque_lane(), vrow = vl >> 2;
            const uint32_t vaddr = vrow * CK_LAT_BYTES + 16 * (((vl >> 1) & 1) ^ lat_xor(vrow)) + 8 * (vl & 1);
            if (SAFE && masked) {
                bf16x8_t seen;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int r = 16 * (j >> 2) + 4 * g + (j & 3);
                    seen[j] = (u0 + r <= lim && !((absent >> r) & 1u)) ? (__bf16)1.0f : (__bf16)0.0f;
                }
#pragma unroll
                for (int dt = 0; dt < CK_DT; ++dt) {
                    const uint32_t va = st + (vaddr ^ (32 * (dt & 7))) + 256 * (dt >> 3);
                    i16x4_t lo = lds_read_tr16<0>(va), hi = lds_read_tr16<16 * CK_LAT_BYTES>(va);
                    lds_wait<0>(lo, hi);
                    bf16x8_t v = join(lo, hi);
                    const bf16x8_t code = split_nonfinite(v);
                    f32x4_t codes = {0.f, 0.f, 0.f, 0.f};
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf, o[dt], 0, 0, 0);
                    codes = __builtin_amdgcn_mfma_f32_16x16x32_bf16(code, seen, codes, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[dt][i] = add_nonfinite(o[dt][i], codes[i]);
                }
            } else {
                // dim blocks in the order dt = e + 8 f, f inner: one address per e
                constexpr int VD = 4;
                i16x4_t vv[VD + 1][2];
                uint32_t va;
                auto vload = [&](auto ic) {
                    constexpr int i = decltype(ic)::value;
                    if constexpr ((i & 3) == 0) va = st + (vaddr ^ (32 * (i >> 2)));
                    vv[i % (VD + 1)][0] = lds_read_tr16<256 * (i & 3)>(va);
                    vv[i % (VD + 1)][1] = lds_read_tr16<256 * (i & 3) + 16 * CK_LAT_BYTES>(va);
                };
                static_for<0, VD>(vload);
                static_for<0, CK_DT>([&](auto ic) {
                    constexpr int i = decltype(ic)::value, dt = (i >> 2) + 8 * (i & 3);
                    if constexpr (i + VD < CK_DT) vload(std::integral_constant<int, i + VD>{});
                    lds_wait<2 * ((i + VD < CK_DT) ? VD : (CK_DT - 1 - i))>(vv[i % (VD + 1)][0], vv[i % (VD + 1)][1]);
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join(vv[i % (VD + 1)][0], vv[i % (VD + 1)][1]), pf, o[dt],
                                                                    0, 0, 0);
                });
            }
        }
        if (PD == 0 && k + 1 < nit) {   // the stream's waves are done with its only stage
            wg_barrier();
            issue(k + 1);
        }
    }
    l_run = allreduce_groups(l_run, [](float p, float q) { return p + q; });

    // ---- the streams of a row join, each wave a part of the dims: its dim blocks of the first half, then of the second
    __syncthreads();
    constexpr int NO = CK_DT / KSTR;             // dim blocks of a wave in the end
    auto block_of = [&](int i) { return KSTR == 1 ? i : 16 * (i / (NO / 2)) + NO / 2 * ks0 + i % (NO / 2); };
    auto finish = [&](const f32x4_t (&o)[NO]) __attribute__((always_inline)) {
        if constexpr (!SAFE) {
            float top = 0.f;
#pragma unroll
            for (int j = 0; j < NO; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = __builtin_fmaf(fabsf(o[j][i]), 0x1p-40f, top);   // not finite where an output is not
            uint32_t* words = reinterpret_cast<uint32_t*>(smem);   // in the stages, which nobody reads any more
            const bool bad = __ballot(!idle && !(top < INFINITY)) != 0;
            if (lane == 0) words[wave] = bad;
            __syncthreads();
            uint32_t any = 0;
#pragma unroll
            for (int i = 0; i < CK_WAVES; ++i) any |= words[i];
            if (__builtin_amdgcn_readfirstlane(any) != 0) {
                __syncthreads();   // every wave has read the words
                return true;
            }
        }
        if (idle) return false;
        if (part_o) {
            float* po = part_o + qg * (16 * D_LAT);
#pragma unroll
            for (int j = 0; j < NO; ++j) *reinterpret_cast<f32x4_t*>(po + (block_of(j) * 64 + lane) * 4) = o[j];
            if (g == 0 && ks0 == 0) {
                part_ml[2 * (16 * qg + c)] = m_run;
                part_ml[2 * (16 * qg + c) + 1] = SAFE ? -l_run : l_run;
            }
        } else if (R < x.nrow) {
            store_row(a, x.tok0 * a.H + R, g, m_run, l_run, SAFE ? 1.0f / CK_ROOM : 1.0f, o, block_of, ks0 == 0);
        }
        return false;
    };
    if constexpr (KSTR == 1) {
        return finish(o);
    } else {
        float* fl = reinterpret_cast<float*>(smem);
        float* sml = fl + CK_OFF_ML / 4;
        if (g == 0) {
            sml[2 * (16 * wave + c)] = m_run;
            sml[2 * (16 * wave + c) + 1] = l_run;
        }
        __syncthreads();
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int j = 0; j < KSTR; ++j) M = fmaxf(M, sml[2 * (16 * (qg + QG * j) + c)]);
        auto weight = [&](float m) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M); };
#pragma unroll
        for (int j = 0; j < KSTR; ++j) {
            const float m = sml[2 * (16 * (qg + QG * j) + c)], l = sml[2 * (16 * (qg + QG * j) + c) + 1];
            L += m == -INFINITY ? l : weight(m) * l;   // nothing seen: l is 0, or NaN from a score that is NaN
        }
        const float w = m_run == -INFINITY ? 1.0f : weight(m_run);   // (without a maximum, o is 0, or NaN)
        m_run = M;
        l_run = L;
        // blocks of 1 KB: [row group][stream][16 dim blocks]
        f32x4_t sum[NO];
        float* rows = fl + qg * (KSTR * 16 * 256) + lane * 4;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (!idle) {
#pragma unroll
                for (int d = 0; d < 16; ++d) {
                    f32x4_t v = o[16 * half + d];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] *= w;
                    *reinterpret_cast<f32x4_t*>(rows + (ks0 * 16 + d) * 256) = v;
                }
            }
            __syncthreads();
            if (!idle) {
#pragma unroll
                for (int k = 0; k < NO / 2; ++k) {
                    f32x4_t v[KSTR];
#pragma unroll
                    for (int j = 0; j < KSTR; ++j)
                        v[j] = *reinterpret_cast<const f32x4_t*>(rows + (j * 16 + NO / 2 * ks0 + k) * 256);
#pragma unroll
                    for (int j = 1; j < KSTR; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[0][i] += v[j][i];
                    sum[NO / 2 * half + k] = v[0];
                }
            }
            __syncthreads();
        }
        return finish(sum);
    }
}

// ------------------------------------------------------------------- kernels

// first tile of every unit in the run of all tiles, and their number, into LDS
__device__ __forceinline__ int scan_units(const ChunkArgs& a, int rows, int* pre) {
    const int tid = threadIdx.x, lane = tid & 63, U = a.B * a.mb;
    auto wave_prefix = [&](int v) {
        for (int d = 1; d < 64; d *= 2) {
            const int t = __shfl_up(v, d);
            if (lane >= d) v += t;
        }
        return v;
    };
    if (U <= 64) {   // every wave for itself, the same values: no barrier
        const int n = lane < U ? unit_tiles(a, chunk_unit(a, lane, rows), rows) : 0;
        const int upto = wave_prefix(n);
        pre[lane] = upto - n;
        return __builtin_amdgcn_readlane(upto, 63);
    }
    constexpr int PER = CK_MAX_UNITS / CK_THREADS;
    __shared__ int waves[CK_WAVES];
    int n[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int u = PER * tid + i;
        n[i] = u < U ? unit_tiles(a, chunk_unit(a, u, rows), rows) : 0;
        sum += n[i];
    }
    const int upto = wave_prefix(sum);
    if (lane == 63) waves[tid >> 6] = upto;
    __syncthreads();
    int at = upto - sum, total = 0;
#pragma unroll
    for (int i = 0; i < CK_WAVES; ++i) {
        if (i < (tid >> 6)) at += waves[i];
        total += waves[i];
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        pre[PER * tid + i] = at;
        at += n[i];
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(total);
}

// The segments of run g of n, one after another; returns whether one is to go again.
template <int QG, bool SAFE>
__device__ __forceinline__ bool chunk_run(const ChunkArgs& a, int g, int n, int total, const int* pre, uint8_t* smem) {
    constexpr int ROWS = 16 * QG;
    const int U = a.B * a.mb;
    const int beg = run_start(g, n, total), end = run_start(g + 1, n, total);
    int u = 0;   // the last unit that starts at or before beg
    for (int step = CK_MAX_UNITS / 2; step > 0; step /= 2)
        if (u + step < U && pre[u + step] <= beg) u += step;
    int at = beg;
    bool again = false;
    while (at < end) {
        u = __builtin_amdgcn_readfirstlane(u);
        at = __builtin_amdgcn_readfirstlane(at);
        const int base = __builtin_amdgcn_readfirstlane(pre[u]);
        const int next = __builtin_amdgcn_readfirstlane(u + 1 < U ? pre[u + 1] : total);
        if (next <= at) {   // a unit without rows
            ++u;
            continue;
        }
        const CkUnit x = chunk_unit(a, u, ROWS);
        const int t0 = at - base, t1 = min(end, next) - base;
        const bool whole = t0 == 0 && t1 == next - base;
        if (threadIdx.x == 0) {   // for the join: the unit's first and last run, and which of its slots the first one fills
            if (t0 == 0) a.span[3 * u] = g, a.span[3 * u + 2] = at > beg;
            if (t1 == next - base) a.span[3 * u + 1] = g;
        }
        const int slot = 2 * g + (at > beg ? 1 : 0);
        float* po = whole ? nullptr : a.part_o + (int64_t)slot * (ROWS * D_LAT);
        float* pml = a.part_ml + (int64_t)slot * (ROWS * 2);
        again |= chunk_segment<QG, SAFE>(a, x, t0, t1, po, pml, smem);
        __syncthreads();   // the stages are free
        at = base + t1;
        ++u;
    }
    return again;
}

// Calls, so that the rare segments' registers are not the ordinary ones'; by value, so that
// nothing of those has an address.
template <int QG>
__device__ __attribute__((noinline)) void chunk_run_again(ChunkArgs a, int g, int n, int total, const int* pre, uint8_t* smem) {
    (void)chunk_run<QG, true>(a, g, n, total, pre, smem);
}
template <int QG>
__device__ __attribute__((noinline)) void chunk_unit_again(ChunkArgs a, int u, int tiles, uint8_t* smem) {
    (void)chunk_segment<QG, true>(a, chunk_unit(a, u, 16 * QG), 0, tiles, nullptr, nullptr, smem);
}

template <int QG>
__global__ __launch_bounds__(CK_THREADS, 2) void chunk_run_kernel(ChunkArgs a) {
    __shared__ __align__(256) uint8_t smem[CK_SMEM];
    __shared__ int pre[CK_MAX_UNITS];
    const int total = scan_units(a, 16 * QG, pre), U = a.B * a.mb;
    const int n = run_count(a, total), g = blockIdx.x;
    if (g == 0)   // units without rows: nothing to join
        for (int u = threadIdx.x; u < U; u += CK_THREADS)
            if ((u + 1 < U ? pre[u + 1] : total) == pre[u]) a.span[3 * u] = a.span[3 * u + 1] = 0;
    if (g >= n) return;
    if (chunk_run<QG, false>(a, g, n, total, pre, smem)) chunk_run_again<QG>(a, g, n, total, pre, smem);
}

template <int QG>
__global__ __launch_bounds__(CK_THREADS, 2) void chunk_unit_kernel(ChunkArgs a) {
    __shared__ __align__(256) uint8_t smem[CK_SMEM];
    const uint32_t wg = workgroup_id();
    if (wg >= (uint32_t)a.B * (uint32_t)a.mb) return;
    const int b = (int)(wg / (uint32_t)a.mb), j = a.mb - 1 - (int)(wg % (uint32_t)a.mb);
    const int u = b * a.mb + j;
    const CkUnit x = chunk_unit(a, u, 16 * QG);
    const int n = unit_tiles(a, x, 16 * QG);
    if (n == 0) return;
    if (chunk_segment<QG, false>(a, x, 0, n, nullptr, nullptr, smem)) chunk_unit_again<QG>(a, u, n, smem);
}

// Joins the parts of a unit that several runs cover: block = (unit, 128 float4 of a
// part, in the order the segments leave them), thread = one of them in every CKJ_GROUPS-th
// part; then the groups join through LDS, in order.
constexpr int CKJ_F = 128, CKJ_GROUPS = 4, CKJ_THREADS = CKJ_F * CKJ_GROUPS, CKJ_BATCH = 4;

struct JoinSum {
    float M, L;
    f32x4_t acc;
};
// x += w y, and the references: weights exp2(m - M), m = -inf where nothing was seen (then 0, or NaN)
__device__ __forceinline__ void join_add(JoinSum& x, float m, float l, const f32x4_t& v, float f) {
    if (m > x.M) {
        const float w = x.M == -INFINITY ? 1.0f : exp2f(x.M - m);
        x.L *= w;
#pragma unroll
        for (int i = 0; i < 4; ++i) x.acc[i] *= w;
        x.M = m;
    }
    const float w = m == -INFINITY ? 1.0f : exp2f(m - x.M);
    x.L += w * l;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.acc[i] += w * f * v[i];
}

__global__ __launch_bounds__(CKJ_THREADS) void chunk_join_kernel(ChunkArgs a, int QG) {
    __shared__ JoinSum sums[CKJ_GROUPS - 1][CKJ_F];
    const int rows = 16 * QG, per = rows * (D_LAT / 4) / CKJ_F;
    const int u = blockIdx.x / per, grp = threadIdx.x / CKJ_F;
    const int f = (blockIdx.x % per) * CKJ_F + threadIdx.x % CKJ_F, lane = f & 63;
    const int r = 16 * (f >> 11) + (lane & 15), d = 16 * ((f >> 6) & 31) + 4 * (lane >> 4);   // row of the unit, first dim
    const int g0 = a.span[3 * u], g1 = a.span[3 * u + 1], late = a.span[3 * u + 2];
    if (g0 == g1) return;
    const CkUnit x = chunk_unit(a, u, rows);
    const int R = x.row0 + r;
    const bool live = R < x.nrow;
    JoinSum t{-INFINITY, 0.f, f32x4_t{0.f, 0.f, 0.f, 0.f}};
    if (live)
        for (int s0 = g0 + grp; s0 <= g1; s0 += CKJ_GROUPS * CKJ_BATCH) {
            float m[CKJ_BATCH], l[CKJ_BATCH];
            f32x4_t v[CKJ_BATCH];
#pragma unroll
            for (int j = 0; j < CKJ_BATCH; ++j) {   // all loads in flight
                const int run = min(s0 + CKJ_GROUPS * j, g1);
                const int64_t slot = 2 * run + (run == g0 ? late : 0);
                const float* ml = a.part_ml + slot * (rows * 2) + 2 * r;
                m[j] = ml[0];
                l[j] = ml[1];
                v[j] = *reinterpret_cast<const f32x4_t*>(a.part_o + slot * (rows * D_LAT) + 4 * f);
            }
#pragma unroll
            for (int j = 0; j < CKJ_BATCH; ++j)   // acc carries the factor; parts with l < 0 do already
                if (s0 + CKJ_GROUPS * j <= g1) join_add(t, m[j], fabsf(l[j]), v[j], l[j] < 0.f ? 1.0f : CK_ROOM);
        }
    if (grp > 0) sums[grp - 1][threadIdx.x % CKJ_F] = t;
    __syncthreads();
    if (grp > 0 || !live) return;
#pragma unroll
    for (int i = 0; i < CKJ_GROUPS - 1; ++i) {
        const JoinSum y = sums[i][threadIdx.x];
        join_add(t, y.M, y.L, y.acc, 1.0f);
    }
    const int64_t row = x.tok0 * a.H + R;
    const bool none = t.M == -INFINITY && t.L == 0.f;
    const float inv = none ? 0.f : (1.0f / t.L) * (1.0f / CK_ROOM);
    const bf16x4_t v4 = {(__bf16)(t.acc[0] * inv), (__bf16)(t.acc[1] * inv), (__bf16)(t.acc[2] * inv), (__bf16)(t.acc[3] * inv)};
    *reinterpret_cast<bf16x4_t*>(a.out + row * D_LAT + d) = v4;
    if (d == 0) a.lse[row] = lse_of(t.M, t.L);
}

ChunkSplit chunk_split(int64_t B, int64_t H, int64_t max_q, int64_t max_kv) {
    ChunkSplit s{};
    const int64_t rows = max_q * H;
    s.qg = rows <= 32 ? 2 : rows <= 64 ? 4 : 8;
    s.mb = (rows + 16 * s.qg - 1) / (16 * s.qg);
    s.units = B * s.mb;
    const int64_t tiles = s.units * std::max<int64_t>(1, (max_kv + CK_TILE - 1) / CK_TILE);
    s.runs = s.units <= CK_MAX_UNITS && tiles < (1ll << 31) ? CK_RUNS : 0;
    s.streams = CK_WAVES / s.qg;
    if (s.runs) {
        s.runs = std::max<int64_t>(1, std::min<int64_t>(s.runs, (tiles + s.streams - 1) / s.streams));
        s.part_o = (size_t)(2 * s.runs) * 16 * s.qg * D_LAT * 4;
        s.part_ml = (size_t)(2 * s.runs) * 16 * s.qg * 2 * 4;
        s.span = (size_t)s.units * 3 * 4;
    }
    return s;
}

hipError_t launch_chunk(const ChunkArgs& a, const ChunkSplit& sp, hipStream_t s) {
    const dim3 block(CK_THREADS);
    if (sp.runs) {
        const dim3 grid((unsigned)sp.runs);
        if (sp.qg == 8) hipLaunchKernelGGL((chunk_run_kernel<8>), grid, block, 0, s, a);
        else if (sp.qg == 2) hipLaunchKernelGGL((chunk_run_kernel<2>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((chunk_run_kernel<4>), grid, block, 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || sp.runs == 1) return e;
        hipLaunchKernelGGL(chunk_join_kernel, dim3((unsigned)(sp.units * 16 * sp.qg * (D_LAT / 4) / CKJ_F)), dim3(CKJ_THREADS), 0, s, a, (int)sp.qg);
        return hipGetLastError();
    }
    const dim3 grid = grid_of(sp.units);
    if (sp.qg == 8) hipLaunchKernelGGL((chunk_unit_kernel<8>), grid, block, 0, s, a);
    else if (sp.qg == 2) hipLaunchKernelGGL((chunk_unit_kernel<2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((chunk_unit_kernel<4>), grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace vkv
