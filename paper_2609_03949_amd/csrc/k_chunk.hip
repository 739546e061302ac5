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
// Cache rows go to LDS by direct loads; their pages' table entries, too, several
// tiles ahead (per wave, so that they need no barrier).  Stage layout: row-major,
// piece p (16 B) of tile row r at slot 72 r + (p ^ (r & 7)).
//
// Work split: up to CK_MAX_UNITS units, the tiles of all units are laid end to end
// and cut into equal runs, one per CU, however the lengths differ; a run that
// covers part of a unit leaves (unnormalised O, reference maximum, sum) in fp32 and
// a second kernel joins the parts.  More units than that fill the chip by
// themselves: one workgroup each, the later rows (more tiles) first.
#include <algorithm>

#include "vkv_tile.h"

namespace vkv {

constexpr int CK_WAVES = 8;
constexpr int CK_THREADS = 64 * CK_WAVES;
constexpr int CK_TILE = 32;                              // cache rows of a tile
constexpr int CK_PIECES = D_ROW / 8;                     // 72 pieces of 16 B per row
constexpr int CK_ROW_BYTES = 2 * D_ROW;
constexpr int CK_STAGE = CK_TILE * CK_ROW_BYTES;         // 36 KB
constexpr int CK_LOADS = CK_STAGE / 1024;                // loads of 1 KB
constexpr int CK_STAGES = 4;
constexpr int CK_ENT = 8;                                // table entries of this many tiles per wave
constexpr int CK_KS = D_ROW / 32, CK_DT = D_LAT / 16;
constexpr float CK_SLACK = 8.0f;   // lag allowed to the softmax reference maximum (log2 units)
constexpr float CK_ROOM = 0x1p-40f;   // careful passes and joins: a factor of the weights, so that no sum of finite values overflows
constexpr int CK_ENT_BYTES = CK_TILE * 4;
constexpr int CK_SMEM = CK_STAGES * CK_STAGE + CK_WAVES * CK_ENT * CK_ENT_BYTES;

// ------------------------------------------------------------ units and runs

struct CkUnit {
    int b, row0, nrow;      // sequence, first row of the block, rows of the sequence
    int64_t tok0;           // first token of the sequence among the packed ones
    int nq, kv;             // new tokens and cache rows of the sequence
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
    return x;
}

// tiles that some row of the block sees; a block of rows that see nothing counts
// one, so that its outputs are written; 0: no rows
__device__ __forceinline__ int unit_tiles(const ChunkArgs& a, const CkUnit& x, int rows) {
    if (x.row0 >= x.nrow) return 0;
    const int last = min(x.row0 + rows, x.nrow) - 1;
    const int seen = max(x.kv - x.nq + last / a.H + 1, 0);
    return max((seen + CK_TILE - 1) / CK_TILE, 1);
}

// runs the tiles of all units are cut into: one per CU, at least CK_MIN_RUN tiles each
__device__ __forceinline__ int run_count(const ChunkArgs& a, int total) {
    return min(max(total / a.min_run, 1), a.runs);
}
__device__ __forceinline__ int run_start(int g, int n, int total) { return (int)((int64_t)g * total / n); }

// ------------------------------------------------------------------ a segment

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));

// this lane's dims 16 dt + 4 g .. +3 of output row `row` from f times what o holds, and
// its lse; rows that see nothing: 0, -inf
__device__ __forceinline__ void store_row(const ChunkArgs& a, int64_t row, int g, float m, float l, float f,
                                          const f32x4_t* o) {
    const bool none = m == -INFINITY && l == 0.f;
    const float inv = none ? 0.f : (1.0f / l) * f;
    uint16_t* out = a.out + row * D_LAT + 4 * g;
#pragma unroll
    for (int dt = 0; dt < CK_DT; ++dt) {
        const bf16x4_t v = {(__bf16)(o[dt][0] * inv), (__bf16)(o[dt][1] * inv), (__bf16)(o[dt][2] * inv),
                            (__bf16)(o[dt][3] * inv)};
        *reinterpret_cast<bf16x4_t*>(out + 16 * dt) = v;
    }
    if (g == 0) a.lse[row] = none ? -INFINITY : ((m == -INFINITY ? 0.f : m) + log2f(l)) * 0.69314718055994530942f;
}

// Tiles [t0, t1) of unit x by one workgroup.  part: where an incomplete unit's
// (O, m, l) go, or null (outputs).  Returns true, and stores nothing, when SAFE is
// false and a result is not finite: a masked row has weight 0 and 0 times a value
// that is not finite is not 0, so with SAFE the tiles that hold masked rows take
// those values apart; and weights above 1 may have made a sum overflow, so with
// SAFE they are small (by a power of two: all else has the same bits).  Parts whose O
// carries that factor have a negative l.
template <int QG, bool SAFE>
__device__ __forceinline__ bool chunk_segment(const ChunkArgs& a, const CkUnit& x, int t0, int t1, float* part_o,
                                              float* part_ml, uint8_t* smem) {
    constexpr int KSTR = CK_WAVES / QG;          // streams of tiles
    constexpr int PD = CK_STAGES / KSTR - 1;     // tiles loaded ahead: 3, 1, 0
    constexpr int NL = (CK_LOADS + QG - 1) / QG; // loads of a tile per wave, at most
    constexpr int NL_MIN = CK_LOADS / QG;        // and at least
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int qg = wave % QG, ks0 = wave / QG;
    const int R = x.row0 + 16 * qg + c;                         // this lane's row
    const int Rc = min(R, x.nrow - 1);                          // rows past the end repeat the last one, never stored
    const int lim = min(x.kv - x.nq + Rc / a.H, x.kv - 1);      // the last cache row it sees
    const int lim_lo = __builtin_amdgcn_readfirstlane(lim);     // of the wave's rows
    const int lim_hi = __builtin_amdgcn_readlane(lim, 15);
    const bool idle = x.row0 + 16 * qg >= x.nrow;
    const int nt = x.kv > 0 ? t1 - t0 : 0;
    const int nit = (nt + KSTR - 1) / KSTR;                     // tiles of each stream, the last ones perhaps past t1

    const int32_t* table = a.table + (int64_t)x.b * a.tstride;
    uint8_t* ents = smem + CK_STAGES * CK_STAGE + wave * (CK_ENT * CK_ENT_BYTES);
    const uint32_t ents_lds = lds_addr(ents);
    auto tile_of = [&](int k) { return t0 + ks0 + KSTR * k; };
    auto stage_of = [&](int k) { return (ks0 * (PD + 1) + k % (PD + 1)) * CK_STAGE; };
    // table entries of the stream's tile k, one per tile row (rows past the end: of the last row)
    auto issue_ent = [&](int k) {
        const int u = min(CK_TILE * tile_of(k) + lane, x.kv - 1);
        if (lane < CK_TILE)
            __builtin_amdgcn_global_load_lds((gbl_void_t*)(table + (u >> a.shift)),
                                             (lds_void_t*)(ents + (k % CK_ENT) * CK_ENT_BYTES), 4, 0, 0);
    };
    // this wave's loads of the stream's tile k: slots 64 j .. 64 j + 63, j = qg + QG i
    auto issue = [&](int k) {
        const int t = tile_of(k);
        uint8_t* st = smem + stage_of(k);
        const uint32_t ent0 = ents_lds + (k % CK_ENT) * CK_ENT_BYTES;
        int ln = lane;
        asm volatile("" : "+v"(ln));   // keeps the slot arithmetic out of registers across the loop
        constexpr int BATCH = NL < 9 ? NL : 9;
#pragma unroll
        for (int i0 = 0; i0 < NL; i0 += BATCH) {
            int32_t e[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int r = min((64 * (qg + QG * (i0 + i)) + ln) / CK_PIECES, CK_TILE - 1);
                asm volatile("ds_read_b32 %0, %1" : "=v"(e[i]) : "v"(ent0 + 4 * r));
            }
            if constexpr (BATCH == 9)
                asm volatile("s_waitcnt lgkmcnt(0)"
                             : "+v"(e[0]), "+v"(e[1]), "+v"(e[2]), "+v"(e[3]), "+v"(e[4]), "+v"(e[5]), "+v"(e[6]), "+v"(e[7]), "+v"(e[8]));
            else
                asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(e[0]), "+v"(e[1]), "+v"(e[2]), "+v"(e[3]), "+v"(e[4]));
            static_assert(BATCH == 9 || BATCH == 5, "entries tied above");
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int j = qg + QG * (i0 + i);
                const int q = 64 * j + ln, r = q / CK_PIECES;
                const int u = min(CK_TILE * t + r, x.kv - 1);
                // a page that does not exist: any row of the cache in its place, masked below
                const bool there = (uint32_t)e[i] < (uint32_t)a.n_pages;
                const int64_t at = there ? (int64_t)e[i] * a.ps + (int64_t)(u & a.page_mask) * a.rs : 0;
                const uint16_t* src = a.cache + at + 8 * ((q - CK_PIECES * r) ^ (r & 7));
                if (j < CK_LOADS)
                    __builtin_amdgcn_global_load_lds((gbl_void_t*)src, (lds_void_t*)(st + 1024 * j), 16, 0, 0);
            }
        }
    };

    if (nt > 0) {
        for (int k = 0; k < max(2 * PD, 1); ++k) issue_ent(k);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (PD == 0) issue_ent(1);
        for (int k = 0; k < max(PD, 1); ++k)
            if (k < nit) issue(k);
    }

    // Q^T operand: row R, dims 32 ks + 8 g .. +8
    bf16x8_t qf[CK_KS];
    {
        const int64_t row = x.tok0 * a.H + Rc;
        const uint16_t* ql = a.q_lat + row * a.qls + 8 * g;
        const uint16_t* qr = a.q_rope + row * a.qrs + 8 * g;
#pragma unroll
        for (int ks = 0; ks < CK_KS; ++ks)
            qf[ks] = *reinterpret_cast<const bf16x8_t*>(ks < D_LAT / 32 ? ql + 32 * ks : qr + 32 * ks - D_LAT);
#pragma unroll
        for (int ks = 0; ks < CK_KS; ++ks) asm volatile("" : "+v"(qf[ks]));   // no wait for them inside the tile loop
    }

    // K operand of (row 16 mt + c, piece 4 ks + g), the piece's low three bits permuted; V operand
    // (transposing reads): lane 4 e + q of 16-lane group g reads rows 4 g + e and 16 + 4 g + e,
    // dims 16 dt + 4 q .. +3, i.e. piece 2 dt + q / 2, half q mod 2
    const uint32_t lds0 = lds_addr(smem);
    uint32_t kaddr[2], vaddr[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) kaddr[i] = c * CK_ROW_BYTES + 16 * ((4 * i + g) ^ (c & 7));
    {
        const int e = c >> 2, q = c & 3, row = 4 * g + e;
#pragma unroll
        for (int i = 0; i < 4; ++i) vaddr[i] = row * CK_ROW_BYTES + 16 * ((2 * i + (q >> 1)) ^ (row & 7)) + 8 * (q & 1);
    }

    f32x4_t o[CK_DT];
#pragma unroll
    for (int dt = 0; dt < CK_DT; ++dt) o[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    for (int k = 0; k < nit; ++k) {
        // tile k has landed: at most the loads of the PD - 1 tiles behind it (and the table
        // entries issued with them) are still in flight
        if (PD > 1 && k + PD - 1 < nit)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(PD > 1 ? (PD - 1) * (NL_MIN + 1) : 0) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        wg_barrier();   // every wave's share has, and the stage loaded next is free
        if (PD > 0 && k + PD < nit) {
            issue_ent(k + 2 * PD);
            issue(k + PD);
        }
        const int t = tile_of(k), u0 = CK_TILE * t;
        if (t < t1 && !idle && u0 <= lim_hi) {
            const uint32_t st = lds0 + stage_of(k);
            int32_t ent;
            asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(ent)
                         : "v"(ents_lds + (k % CK_ENT) * CK_ENT_BYTES + 4 * (lane & 31)));
            const uint32_t absent = (uint32_t)__ballot((uint32_t)ent >= (uint32_t)a.n_pages);   // tile rows on no page
            const bool masked = u0 + CK_TILE - 1 > lim_lo || absent != 0;
            f32x4_t s[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
            {
                constexpr int SD = 3;   // operands read ahead of the matrix cores
                bf16x8_t kf[SD + 1][2];
                const uint32_t ka[2] = {st + kaddr[0], st + kaddr[1]};
                auto kload = [&](auto kc) {
                    constexpr int ks = decltype(kc)::value;
                    kf[ks % (SD + 1)][0] = lds_read128<128 * (ks >> 1)>(ka[ks & 1]);
                    kf[ks % (SD + 1)][1] = lds_read128<128 * (ks >> 1) + 16 * CK_ROW_BYTES>(ka[ks & 1]);
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
            }
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
            uint32_t va[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) va[i] = st + vaddr[i];
            if (SAFE && masked) {
                bf16x8_t seen;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int r = 16 * (j >> 2) + 4 * g + (j & 3);
                    seen[j] = (u0 + r <= lim && !((absent >> r) & 1u)) ? (__bf16)1.0f : (__bf16)0.0f;
                }
#pragma unroll
                for (int dt = 0; dt < CK_DT; ++dt) {
                    i16x4_t lo = lds_read_tr16<0>(va[dt & 3] + 128 * (dt >> 2));
                    i16x4_t hi = lds_read_tr16<16 * CK_ROW_BYTES>(va[dt & 3] + 128 * (dt >> 2));
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
                constexpr int VD = 4;
                i16x4_t vv[VD + 1][2];
                auto vload = [&](auto ic) {
                    constexpr int dt = decltype(ic)::value;
                    vv[dt % (VD + 1)][0] = lds_read_tr16<128 * (dt >> 2)>(va[dt & 3]);
                    vv[dt % (VD + 1)][1] = lds_read_tr16<128 * (dt >> 2) + 16 * CK_ROW_BYTES>(va[dt & 3]);
                };
                static_for<0, VD>(vload);
                static_for<0, CK_DT>([&](auto ic) {
                    constexpr int dt = decltype(ic)::value;
                    if constexpr (dt + VD < CK_DT) vload(std::integral_constant<int, dt + VD>{});
                    lds_wait<2 * ((dt + VD < CK_DT) ? VD : (CK_DT - 1 - dt))>(vv[dt % (VD + 1)][0], vv[dt % (VD + 1)][1]);
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join(vv[dt % (VD + 1)][0], vv[dt % (VD + 1)][1]), pf, o[dt],
                                                                    0, 0, 0);
                });
            }
        }
        if (PD == 0 && k + 1 < nit) {   // the stream's waves are done with its only stage
            wg_barrier();
            issue_ent(k + 2);
            issue(k + 1);
        }
    }
    l_run = allreduce_groups(l_run, [](float p, float q) { return p + q; });

    // ---- the streams of a row join in the first one's wave, through the stages
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // table entries issued past the end have landed
    __syncthreads();
    float* fl = reinterpret_cast<float*>(smem);
    if constexpr (KSTR > 1) {
        float* sml = fl + CK_STAGES * CK_STAGE / 4;   // the table entries' place: (m, l) of every wave's rows
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
        if (m_run != -INFINITY) {   // (without one, o is 0, or NaN)
            const float w = weight(m_run);
#pragma unroll
            for (int dt = 0; dt < CK_DT; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[dt][i] *= w;
        }
        m_run = M;
        l_run = L;
        constexpr int WO = 16 * D_LAT;   // floats of a wave's O
        auto put = [&](float* dst) {
#pragma unroll
            for (int dt = 0; dt < CK_DT; ++dt) *reinterpret_cast<f32x4_t*>(dst + (dt * 64 + lane) * 4) = o[dt];
        };
        auto add = [&](const float* src) {
#pragma unroll
            for (int dt = 0; dt < CK_DT; ++dt) {
                const f32x4_t v = *reinterpret_cast<const f32x4_t*>(src + (dt * 64 + lane) * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[dt][i] += v[i];
            }
        };
#pragma unroll
        for (int half = CK_WAVES / 2; half >= QG; half /= 2) {
            if (wave >= half && wave < 2 * half) put(fl + (wave - half) * WO);
            __syncthreads();
            if (wave < half) add(fl + wave * WO);
            __syncthreads();
        }
    }
    const bool mine = ks0 == 0 && !idle;
    if constexpr (!SAFE) {
        float top = 0.f;
        if (mine)
#pragma unroll
            for (int dt = 0; dt < CK_DT; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) top += fabsf(o[dt][i]) * 0x1p-40f;   // not finite where an output is not
        uint32_t* flag = reinterpret_cast<uint32_t*>(smem);   // in the stages, which nobody reads any more
        if (tid == 0) *flag = 0;
        __syncthreads();
        if (!(top < INFINITY)) *flag = 1;
        __syncthreads();
        const bool again = *flag != 0;
        __syncthreads();
        if (again) return true;
    }
    if (!mine) return false;
    if (part_o) {
        float* po = part_o + qg * (16 * D_LAT);
#pragma unroll
        for (int dt = 0; dt < CK_DT; ++dt) *reinterpret_cast<f32x4_t*>(po + (dt * 64 + lane) * 4) = o[dt];
        if (g == 0) {
            part_ml[2 * (16 * qg + c)] = m_run;
            part_ml[2 * (16 * qg + c) + 1] = SAFE ? -l_run : l_run;
        }
        return false;
    }
    if (R >= x.nrow) return false;
    store_row(a, x.tok0 * a.H + R, g, m_run, l_run, SAFE ? 1.0f / CK_ROOM : 1.0f, o);
    return false;
}

// a call, so that the rare segment's registers are not the ordinary one's; by value, so
// that nothing of the ordinary one has an address
template <int QG>
__device__ __attribute__((noinline)) void chunk_segment_again(ChunkArgs a, int u, int t0, int t1, float* part_o,
                                                              float* part_ml, uint8_t* smem) {
    (void)chunk_segment<QG, true>(a, chunk_unit(a, u, 16 * QG), t0, t1, part_o, part_ml, smem);
}

// ------------------------------------------------------------------- kernels

// first tile of every unit in the run of all tiles, and their number, into LDS
__device__ __forceinline__ int scan_units(const ChunkArgs& a, int rows, int* pre) {
    constexpr int PER = CK_MAX_UNITS / CK_THREADS;
    const int tid = threadIdx.x, U = a.B * a.mb;
    int n[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int u = PER * tid + i;
        n[i] = u < U ? unit_tiles(a, chunk_unit(a, u, rows), rows) : 0;
        sum += n[i];
    }
    pre[tid] = sum;
    __syncthreads();
    for (int d = 1; d < CK_THREADS; d *= 2) {
        const int v = tid >= d ? pre[tid - d] : 0;
        __syncthreads();
        pre[tid] += v;
        __syncthreads();
    }
    const int total = __builtin_amdgcn_readfirstlane(pre[CK_THREADS - 1]);
    int at = pre[tid] - sum;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        pre[PER * tid + i] = at;
        at += n[i];
    }
    __syncthreads();
    return total;
}

template <int QG>
__global__ __launch_bounds__(CK_THREADS, 2) void chunk_run_kernel(ChunkArgs a) {
    __shared__ __align__(256) uint8_t smem[CK_SMEM];
    constexpr int ROWS = 16 * QG;
    __shared__ int pre[CK_MAX_UNITS];
    const int total = scan_units(a, ROWS, pre), U = a.B * a.mb;
    const int n = run_count(a, total), g = blockIdx.x;
    if (g == 0)
        for (int u = threadIdx.x; u <= U; u += CK_THREADS) a.first[u] = u < U ? pre[u] : total;
    if (g >= n) return;
    const int beg = run_start(g, n, total), end = run_start(g + 1, n, total);
    int u = 0;   // the last unit that starts at or before beg
    for (int step = CK_MAX_UNITS / 2; step > 0; step /= 2)
        if (u + step < U && pre[u + step] <= beg) u += step;
    int at = beg;
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
        const int slot = 2 * g + (at > beg ? 1 : 0);
        float* po = whole ? nullptr : a.part_o + (int64_t)slot * (ROWS * D_LAT);
        float* pml = a.part_ml + (int64_t)slot * (ROWS * 2);
        if (chunk_segment<QG, false>(a, x, t0, t1, po, pml, smem)) chunk_segment_again<QG>(a, u, t0, t1, po, pml, smem);
        __syncthreads();   // the stages are free
        at = base + t1;
        ++u;
    }
}

template <int QG>
__global__ __launch_bounds__(CK_THREADS, 2) void chunk_unit_kernel(ChunkArgs a) {
    __shared__ __align__(256) uint8_t smem[CK_SMEM];
    constexpr int ROWS = 16 * QG;
    const int b = blockIdx.x / a.mb, j = a.mb - 1 - (int)(blockIdx.x % a.mb);
    const int u = b * a.mb + j;
    const CkUnit x = chunk_unit(a, u, ROWS);
    const int n = unit_tiles(a, x, ROWS);
    if (n == 0) return;
    if (chunk_segment<QG, false>(a, x, 0, n, nullptr, nullptr, smem)) chunk_segment_again<QG>(a, u, 0, n, nullptr, nullptr, smem);
}

// Joins the parts of a unit that several runs cover: block = (unit, 16 rows, 8 of the
// 32 blocks of 16 dims), thread = 4 dims of a row.
constexpr int CKJ_DT = 8, CKJ_BATCH = 8;

__global__ __launch_bounds__(64 * CKJ_DT) void chunk_join_kernel(ChunkArgs a, int QG) {
    const int rows = 16 * QG;
    constexpr int DP = CK_DT / CKJ_DT;
    const int dp = blockIdx.x % DP, qg = blockIdx.x / DP % QG, u = blockIdx.x / (DP * QG);
    const int U = a.B * a.mb, total = a.first[U], base = a.first[u], next = a.first[u + 1];
    if (next == base) return;
    const int n = run_count(a, total);
    // the runs that hold the unit's first and last tile
    auto run_of = [&](int tile) {
        int g = (int)min((int64_t)tile * n / total, (int64_t)n - 1);
        while (run_start(g + 1, n, total) <= tile) ++g;
        while (run_start(g, n, total) > tile) --g;
        return g;
    };
    const int g0 = run_of(base), g1 = run_of(next - 1);
    if (g0 == g1) return;
    const CkUnit x = chunk_unit(a, u, rows);
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int R = x.row0 + 16 * qg + c;
    const int dt = dp * CKJ_DT + (threadIdx.x >> 6);
    const bool late = run_start(g0, n, total) < base;   // the unit is its first run's last segment, not its first
    float M = -INFINITY, L = 0.f;
    f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int s0 = g0; s0 <= g1; s0 += CKJ_BATCH) {
        float m[CKJ_BATCH], l[CKJ_BATCH];
        f32x4_t v[CKJ_BATCH];
#pragma unroll
        for (int j = 0; j < CKJ_BATCH; ++j) {
            const int run = min(s0 + j, g1);
            const int64_t slot = 2 * run + (run == g0 && late ? 1 : 0);
            const float* ml = a.part_ml + slot * (rows * 2) + 2 * (16 * qg + c);
            m[j] = ml[0];
            l[j] = ml[1];
            v[j] = *reinterpret_cast<const f32x4_t*>(a.part_o + slot * (rows * D_LAT) + qg * (16 * D_LAT) + (dt * 64 + lane) * 4);
        }
        float top = M;
#pragma unroll
        for (int j = 0; j < CKJ_BATCH; ++j)
            if (s0 + j <= g1) top = fmaxf(top, m[j]);
        if (top != M && M != -INFINITY) {
            const float w = exp2f(M - top);
            L *= w;
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] *= w;
        }
        M = top;
#pragma unroll
        for (int j = 0; j < CKJ_BATCH; ++j) {
            if (s0 + j > g1) break;
            const float w = m[j] == -INFINITY ? 1.0f : exp2f(m[j] - M);   // nothing seen: 0, or NaN
            L += w * fabsf(l[j]);
            const float wo = w * (l[j] < 0.f ? 1.0f : CK_ROOM);   // acc carries the factor
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += wo * v[j][i];
        }
    }
    if (R >= x.nrow) return;
    const int64_t row = x.tok0 * a.H + R;
    const bool none = M == -INFINITY && L == 0.f;
    const float inv = none ? 0.f : (1.0f / L) * (1.0f / CK_ROOM);
    const bf16x4_t r = {(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv), (__bf16)(acc[3] * inv)};
    *reinterpret_cast<bf16x4_t*>(a.out + row * D_LAT + 16 * dt + 4 * g) = r;
    if (g == 0 && dt == 0) a.lse[row] = none ? -INFINITY : ((M == -INFINITY ? 0.f : M) + log2f(L)) * 0.69314718055994530942f;
}

ChunkSplit chunk_split(int64_t B, int64_t H, int64_t max_q, int64_t max_kv) {
    ChunkSplit s{};
    const int64_t rows = max_q * H;
    s.qg = rows <= 32 ? 2 : rows <= 64 ? 4 : 8;
    s.mb = (rows + 16 * s.qg - 1) / (16 * s.qg);
    s.units = B * s.mb;
    const int64_t tiles = s.units * std::max<int64_t>(1, (max_kv + CK_TILE - 1) / CK_TILE);
    s.runs = s.units <= CK_MAX_UNITS && tiles < (1ll << 31) ? CK_RUNS : 0;
    s.min_run = 2 * CK_WAVES / s.qg;
    if (s.runs) {
        s.runs = std::max<int64_t>(1, std::min<int64_t>(s.runs, tiles / s.min_run));
        s.part_o = (size_t)(2 * s.runs) * 16 * s.qg * D_LAT * 4;
        s.part_ml = (size_t)(2 * s.runs) * 16 * s.qg * 2 * 4;
        s.first = (size_t)(s.units + 1) * 4;
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
        hipLaunchKernelGGL(chunk_join_kernel, dim3((unsigned)(sp.units * sp.qg * (CK_DT / CKJ_DT))), dim3(64 * CKJ_DT), 0, s, a, (int)sp.qg);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)sp.units);
    if (sp.qg == 8) hipLaunchKernelGGL((chunk_unit_kernel<8>), grid, block, 0, s, a);
    else if (sp.qg == 2) hipLaunchKernelGGL((chunk_unit_kernel<2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((chunk_unit_kernel<4>), grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace vkv
