// k_prompt.hip -- causal attention over whole prompts, packed sequences,
// grouped heads (gfx950).
//
//   s_ij = scale * (q_i . k_j [+ qr_i . kr_j]),  j <= i,   o_i = sum_j softmax_j(s_ij) v_j
//
// Work split: workgroup = (128 query rows, head, sequence), 4 waves of 32 rows;
// two workgroups per CU, so that one's softmax runs beside the other's matrix
// instructions.  Key and value tiles of 64 rows go through two LDS stages by
// direct global->LDS loads: one barrier per tile, the next tile loads while
// the current one is used.  S^T = K Q^T leaves every lane with one query (its
// column) and 16 keys per 32-key block, so the softmax is in-lane but for one
// swap of the lane halves, and P stays in registers: the accumulator layout is
// the B-operand layout of O^T = V^T P^T when the keys are fed to the K dimension
// in a permuted order, which the transposing V reads follow.
// Softmax in the log2 domain against a reference maximum that moves only when
// a score exceeds it by more than 2^8 (P <= 256; most tiles rescale nothing).
// P is rounded to bf16 for the matrix cores (off by at most 2^-8 of a weight, the
// type of V); the sum of the weights is taken before that rounding, in fp32.
//
// Bound: LDS, the matrix cores and the vector units each are busy half of a tile's time,
// and long prompts run at the power limit (1.9 GHz).  Measured: 16384 tokens, 16 heads of
// 192/128 dims 1217 us, 1.13 PFLOP/s; 16 prompts of 17 to 2048 tokens, 32 heads of 128 dims
// 260 to 266 us, 0.72 PFLOP/s (more than a quarter of a workgroup's time lies before its
// second tile and after its last one).  No faster: the weights between the products of the values
// (1256 and 268 us); the next tile's scores ahead of them, which needs registers for
// two tiles' scores (more than 100 spilled).
#include "vkv_tile.h"

namespace vkv {

constexpr int PR_WAVES = 4;
constexpr int PR_ROWS = 32 * PR_WAVES;   // query rows of a workgroup
constexpr int PR_KEYS = 64;              // keys of a tile
constexpr float PR_SLACK = 8.0f;
constexpr float PR_ROOM = 0x1p-40f;   // the careful pass: a factor of the weights, so that no sum of finite values overflows

// Bytes of one stage: panels [64 keys][DN], [64][DR], [64][DV], row-major, 16-byte
// pieces permuted within a row by an XOR with a function of the row that spreads the
// operand reads over the LDS banks.
template <int DN, int DR, int DV>
constexpr int prompt_stage_bytes() {
    return PR_KEYS * 2 * (DN + DR + DV);
}

// K panels: LDS serves a 128-bit read sixteen lanes (rows of one piece) at a time, rows
// {0-3, 12-15, 20-27} and the others; each such group has all of r mod 16, and the even
// rows of it all of r / 2 mod 8 (a 64-wide panel's odd rows lie in the other half of
// the banks), so these spread it over all 16 pieces of a 256-byte sweep
template <int D>
__device__ __forceinline__ int kpiece_xor(int r) {
    return D == 128 ? r & 15 : (r >> 1) & 7;
}
// V panels: the transposing reads take four rows (4 a .. 4 a + 3) of 2 or 4 adjacent
// pieces; the row within the four picks a group of four pieces, so that they cover
// every bank (a 64-wide panel has 8 pieces a row, and odd rows lie in the other half)
template <int DV>
__device__ __forceinline__ int vpiece_xor(int r) {
    return DV == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

// One panel of a tile: D columns of PR_KEYS rows, this wave's share (1 KB per load).  A lane
// keeps the offset of its row and piece of the first load; the rest of the address is scalar
// but in a sequence's last tile, whose rows past the end repeat the last one (address
// arithmetic in the lanes took as long as the exponentials).
template <int D>
struct PanelLoader {
    static constexpr int PC = D / 8;              // pieces per row
    static constexpr int RPL = 64 / PC;           // rows per load
    static constexpr int NL = PR_KEYS * PC / 64 / PR_WAVES;
    const uint8_t* base;
    int64_t row_bytes, off;
    int r0, wave;                                 // row of the first load; the i-th one RPL * PR_WAVES * i on
    template <typename XOR>
    __device__ __forceinline__ PanelLoader(const uint16_t* b, int64_t ts, int wave_, int lane, XOR xr)
        : base(reinterpret_cast<const uint8_t*>(b)), row_bytes(2 * ts), r0(RPL * wave_ + lane / PC), wave(wave_) {
        off = r0 * row_bytes + 16 * ((lane % PC) ^ xr(r0));   // the piece is the same for every i: xr has a period of RPL * PR_WAVES rows
    }
    __device__ __forceinline__ void load(int t0, int len, uint8_t* st) const {
        const uint8_t* tile = base + t0 * row_bytes;
        if (t0 + PR_KEYS <= len) {
#pragma unroll
            for (int i = 0; i < NL; ++i)
                __builtin_amdgcn_global_load_lds((gbl_void_t*)(tile + RPL * PR_WAVES * i * row_bytes + off),
                                                 (lds_void_t*)(st + 1024 * (wave + PR_WAVES * i)), 16, 0, 0);
        } else {
            int first = r0;
            asm volatile("" : "+v"(first));       // nothing of this is kept across the tiles
#pragma unroll 1
            for (int i = 0; i < NL; ++i) {
                const int row = first + RPL * PR_WAVES * i;
                __builtin_amdgcn_global_load_lds((gbl_void_t*)(tile + off + (int64_t)(min(row, len - 1 - t0) - first) * row_bytes),
                                                 (lds_void_t*)(st + 1024 * (wave + PR_WAVES * i)), 16, 0, 0);
            }
        }
    }
};

// One block: SAFE false is the ordinary pass.  A masked key has weight 0, and 0 times
// a value that is not finite is not 0, so such a value would reach rows that do not see
// it.  That shows in the result: the block then returns true and goes again with SAFE,
// over what it stored, which takes the values that are not finite apart in the tiles
// that hold masked keys, and keeps the weights small (by a power of two: the same bits
// but for weights and sums below 2^-86, whose roundings are of absolute size), as those
// above 1 may have made a sum overflow.
template <int DN, int DR, int DV, bool SAFE>
__device__ __forceinline__ bool prompt_block(const PromptArgs& a, uint8_t* smem) {
    constexpr int STAGE = prompt_stage_bytes<DN, DR, DV>();
    constexpr int OFF_R = PR_KEYS * 2 * DN, OFF_V = PR_KEYS * 2 * (DN + DR);
    constexpr int KSN = DN / 16, KSR = DR / 16, KS = KSN + KSR, DT = DV / 32;

    // the longest blocks first; with 8 | H every XCD takes H / 8 neighbouring heads of
    // each sequence (workgroups go to the XCDs in turn), which share K and V in its L2
    const uint32_t npair = (uint32_t)a.n_seq * (uint32_t)a.H;     // (the grid is below 2^31)
    const uint32_t wg = workgroup_id();
    const int qb = a.nqb - 1 - (int)(wg / npair);                 // (below 0: none)
    const int p = (int)(wg % npair);
    int b = p / a.H, h = p % a.H;
    if (a.H % 8 == 0) {
        const int hx = a.H / 8, i = p / 8;
        b = i / hx;
        h = (p % 8) * hx + i % hx;
    }
    const int g = h / (a.H / a.Hk);
    const int64_t start = min(max((int64_t)a.cu[b], (int64_t)0), a.n_tok);
    const int64_t end = min(max((int64_t)a.cu[b + 1], start), a.n_tok);
    const int len = (int)min(end - start, (int64_t)a.max_len);
    const int q0 = qb * PR_ROWS;
    if (q0 >= len || qb < 0) return false;

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int w0 = q0 + 32 * wave;            // the wave's first row
    const int qi = w0 + c;                    // this lane's query
    const int ntile = (min(len, q0 + PR_ROWS) + PR_KEYS - 1) / PR_KEYS;

    const uint16_t* kb = a.k + start * a.kts + (int64_t)g * a.khs;
    const uint16_t* vb = a.v + start * a.vts + (int64_t)g * a.vhs;
    const PanelLoader<DN> kpanel(kb, a.kts, wave, lane, kpiece_xor<DN>);
    const PanelLoader<DR ? DR : 64> rpanel(DR ? a.kr + start * a.rts : kb, a.rts, wave, lane, kpiece_xor<DR ? DR : 64>);
    const PanelLoader<DV> vpanel(vb, a.vts, wave, lane, vpiece_xor<DV>);
    auto issue = [&](int t) {
        uint8_t* st = smem + (t & 1) * STAGE;
        kpanel.load(PR_KEYS * t, len, st);
        if constexpr (DR > 0) rpanel.load(PR_KEYS * t, len, st + OFF_R);
        vpanel.load(PR_KEYS * t, len, st + OFF_V);
    };

    // Q^T operand: query qi, dims 16 ks + 8 hh .. +8 (rows past the end repeat the last one, never stored)
    bf16x8_t qf[KS];
    {
        const uint16_t* src = a.q + (start + min(qi, len - 1)) * a.qts + (int64_t)h * a.qhs + 8 * hh;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8_t*>(src + 16 * ks);
    }
    if constexpr (SAFE) wg_barrier();   // every wave has read the others' words (below)
    issue(0);
    // consume the query loads here, so no wait for them lands inside the tile loop
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));

    const uint32_t lds0 = lds_addr(smem);
    // K operand of (row 32 mt + c, piece 2 ks + hh): a k-step flips bits of the permuted piece
    const uint32_t kaddr = c * (2 * DN) + 16 * (hh ^ kpiece_xor<DN>(c));
    const uint32_t raddr = DR ? OFF_R + c * (2 * DR) + 16 * (hh ^ kpiece_xor<DR ? DR : 64>(c)) : 0;
    // V operand (transposing reads): lane 4 e + q of a 16-lane group reads row
    // 16 s + 8 u + 4 hh + e, dims 32 dt + 16 gi + 4 q .. +3
    uint32_t vaddr[DT][2];
    {
        const int e = (lane >> 2) & 3, q = lane & 3, gi = (lane >> 4) & 1;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int row = 8 * u + 4 * hh + e, piece = 4 * dt + 2 * gi + (q >> 1);
                vaddr[dt][u] = OFF_V + row * (2 * DV) + 16 * (piece ^ vpiece_xor<DV>(row)) + 8 * (q & 1);
            }
    }

    f32x16_t o[DT];
    float m_run, l_run;
    {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
        m_run = -INFINITY;
        l_run = 0.f;
        for (int t = 0; t < ntile; ++t) {
            // this wave's loads of tile t have landed (nothing else is in flight), every wave's
            // have, and every wave is done with tile t - 1, whose stage is loaded next
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            wg_barrier();
            if (t + 1 < ntile) issue(t + 1);
            const int k0 = PR_KEYS * t;
            if (k0 > w0 + 31) continue;   // no key of the tile is seen by a row of this wave
            const bool masked = k0 + PR_KEYS - 1 > w0;
            const uint32_t st = lds0 + (t & 1) * STAGE;
            f32x16_t s[2];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[mt][i] = 0.f;
            {
                constexpr int SD = 3;   // operands read ahead of the matrix cores
                bf16x8_t kf[SD + 1][2];
                auto kload = [&](auto kc) {
                    constexpr int ks = decltype(kc)::value;
                    const uint32_t at = st + (ks < KSN ? kaddr ^ (32 * ks) : raddr ^ (32 * (ks - KSN)));
                    kf[ks % (SD + 1)][0] = lds_read128<0>(at);
                    kf[ks % (SD + 1)][1] = lds_read128<32 * 2 * (ks < KSN ? DN : DR)>(at);
                };
                static_for<0, SD>(kload);
                static_for<0, KS>([&](auto kc) {
                    constexpr int ks = decltype(kc)::value;
                    if constexpr (ks + SD < KS) kload(std::integral_constant<int, ks + SD>{});
                    constexpr int after = 2 * ((ks + SD < KS) ? SD : (KS - 1 - ks));
                    lds_wait<after>(kf[ks % (SD + 1)][0], kf[ks % (SD + 1)][1]);
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt)
                        s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks % (SD + 1)][mt], qf[ks], s[mt], 0, 0, 0);
                });
            }
            // s[mt][i] = score of key k0 + 32 mt + 8 (i / 4) + 4 hh + i % 4 for query qi
            if (masked) {
                const int lim = qi - k0 - 4 * hh;
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (32 * mt + 8 * (i >> 2) + (i & 3) > lim) s[mt][i] = -INFINITY;
            }
            float cmax = s[0][0];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int i = 0; i < 16; ++i) cmax = fmaxf(cmax, s[mt][i]);
            cmax = half_max(cmax) * a.scale_log2;
            const bool move = cmax > m_run + PR_SLACK;
            const float alpha = move ? __builtin_amdgcn_exp2f(m_run - cmax) : 1.0f;
            if (move) m_run = cmax;
            const float ref = m_run == -INFINITY ? 0.f : m_run;   // nothing but masked scores so far
            bf16x8_t pf[4];
            float psum = 0.f;
#pragma unroll
            for (int s4 = 0; s4 < 4; ++s4)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int mt = s4 >> 1, i = 8 * (s4 & 1) + j;
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][i], a.scale_log2, -ref));
                    psum += x;
                    pf[s4][j] = (__bf16)(SAFE ? x * PR_ROOM : x);
                }
            l_run = l_run * alpha + psum;
            if (__ballot(move)) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[dt][i] *= alpha;
            }
            if (SAFE && masked) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    f32x16_t codes;
#pragma unroll
                    for (int i = 0; i < 16; ++i) codes[i] = 0.f;
#pragma unroll
                    for (int s4 = 0; s4 < 4; ++s4) {
                        i16x4_t lo = lds_read_tr16<0>(st + vaddr[dt][0] + 16 * 2 * DV * s4);
                        i16x4_t hi = lds_read_tr16<0>(st + vaddr[dt][1] + 16 * 2 * DV * s4);
                        lds_wait<0>(lo, hi);
                        bf16x8_t v = join(lo, hi), seen;
                        const bf16x8_t code = split_nonfinite(v);
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            seen[j] = k0 + 16 * s4 + 8 * (j >> 2) + 4 * hh + (j & 3) <= qi ? (__bf16)1.0f : (__bf16)0.0f;
                        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[s4], o[dt], 0, 0, 0);
                        codes = __builtin_amdgcn_mfma_f32_32x32x16_bf16(code, seen, codes, 0, 0, 0);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[dt][i] = add_nonfinite(o[dt][i], codes[i]);
                }
                continue;
            }
            // the softmax's cross-lane reads complete before the V reads are issued
            asm volatile("" : "+v"(l_run), "+v"(pf[0]), "+v"(pf[1]), "+v"(pf[2]), "+v"(pf[3]));
            {
                constexpr int VD = 4, N = 4 * DT;
                i16x4_t vv[VD + 1][2];
                auto vload = [&](auto ic) {
                    constexpr int i = decltype(ic)::value, s4 = i / DT, dt = i % DT;
                    vv[i % (VD + 1)][0] = lds_read_tr16<16 * 2 * DV * s4>(st + vaddr[dt][0]);
                    vv[i % (VD + 1)][1] = lds_read_tr16<16 * 2 * DV * s4>(st + vaddr[dt][1]);
                };
                static_for<0, VD>(vload);
                static_for<0, N>([&](auto ic) {
                    constexpr int i = decltype(ic)::value, s4 = i / DT, dt = i % DT;
                    if constexpr (i + VD < N) vload(std::integral_constant<int, i + VD>{});
                    constexpr int after = 2 * ((i + VD < N) ? VD : (N - 1 - i));
                    lds_wait<after>(vv[i % (VD + 1)][0], vv[i % (VD + 1)][1]);
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(join(vv[i % (VD + 1)][0], vv[i % (VD + 1)][1]), pf[s4],
                                                                    o[dt], 0, 0, 0);
                });
            }
        }
        l_run = half_sum(l_run);
    }
    // the workgroup's waves share the tiles, so they go again together; each one's word lies in
    // the stage of the last tile but one, which every wave was done with before the last
    const uint32_t word = lds0 + (ntile & 1) * STAGE;
    if constexpr (!SAFE) {
        float top = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = __builtin_fmaf(fabsf(o[dt][i]), 0x1p-40f, top);   // not finite where an output is not
        const uint32_t again = __ballot(!(top < INFINITY)) != 0;
        asm volatile("ds_write_b32 %0, %1" ::"v"(word + 4 * wave), "v"(again) : "memory");
    }
    if (qi < len) {
        const float inv = (1.0f / l_run) * (SAFE ? 1.0f / PR_ROOM : 1.0f);
        uint16_t* out = a.out + ((start + qi) * a.H + h) * DV + 4 * hh;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
                const bf16x4_t v = {(__bf16)(o[dt][4 * i4] * inv), (__bf16)(o[dt][4 * i4 + 1] * inv),
                                    (__bf16)(o[dt][4 * i4 + 2] * inv), (__bf16)(o[dt][4 * i4 + 3] * inv)};
                *reinterpret_cast<bf16x4_t*>(out + 32 * dt + 8 * i4) = v;
            }
        if (hh == 0) a.lse[(start + qi) * a.H + h] = (m_run + log2f(l_run)) * 0.69314718055994530942f;
    }
    if constexpr (SAFE) return false;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // (no wait for the stores)
    wg_barrier();
    f32x4_t words;
    asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(words) : "v"(word) : "memory");
    const uint32_t any = __float_as_uint(words[0]) | __float_as_uint(words[1]) | __float_as_uint(words[2]) | __float_as_uint(words[3]);
    return __builtin_amdgcn_readfirstlane(any) != 0;
}
static_assert(PR_WAVES == 4, "four words");

// a call, so that the rare block's registers are not the ordinary one's; by value, so
// that nothing of the ordinary one has an address
template <int DN, int DR, int DV>
__device__ __attribute__((noinline)) void prompt_block_again(PromptArgs a, uint8_t* smem) {
    (void)prompt_block<DN, DR, DV, true>(a, smem);
}

template <int DN, int DR, int DV>
__global__ __launch_bounds__(64 * PR_WAVES, 2) void prompt_kernel(PromptArgs a) {
    __shared__ __align__(256) uint8_t smem[2 * prompt_stage_bytes<DN, DR, DV>()];
    if (prompt_block<DN, DR, DV, false>(a, smem)) prompt_block_again<DN, DR, DV>(a, smem);
}

int64_t prompt_blocks(int64_t len) { return (len + PR_ROWS - 1) / PR_ROWS; }

hipError_t launch_prompt(const PromptArgs& a, int dn, int dr, hipStream_t s) {
    const dim3 grid = grid_of((int64_t)a.n_seq * a.H * a.nqb), block(64 * PR_WAVES);
    if (dn == 128 && dr == 64)
        hipLaunchKernelGGL((prompt_kernel<128, 64, 128>), grid, block, 0, s, a);
    else if (dn == 128)
        hipLaunchKernelGGL((prompt_kernel<128, 0, 128>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((prompt_kernel<64, 0, 64>), grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace vkv
