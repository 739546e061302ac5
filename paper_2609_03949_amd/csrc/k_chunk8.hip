// k_chunk8.hip -- attention of a chunk of new tokens over a paged latent cache held in 8 bits
// (gfx950).
//
//   s_u = scale * (q_lat . c_u + q_rope . r_u),  c_u = 2^e code_u,  u <= kv_len - nq + i,
//   o_i = sum_u softmax_u(s) c_u   (512 dims)
//
// Units of (token, head) rows and the runs of cache tiles they are cut into are those of the bf16
// cache's kernel.  A tile is 64 or 32 rows of 640 bytes, three or seven of them in LDS (direct loads).  Every 8-bit value is a
// bf16 and an fp16 value, so the products take operands that are exact: the conversion of the keys multiplies by their power of
// two, and the weights carry it for the product with the values, which is fp16's.  (The 8-bit products of these matrix cores take half the
// time, but over 512 dims of normal data are off by 8e-7 of the sum of the magnitudes on average, 6e-6 at worst, where bf16 products are
// by 6e-10 and 3e-8; the weights would be rounded to 8 bits too.)  The queries stay in registers, so do the
// outputs, 128 dims a wave; weights go through LDS.  What the vector units convert is as long as the products it is for, and
// bounds units of many rows as much as these do; units of few rows are bound by HBM.  So there are three ways to work on a unit,
// by its rows:
//   16       four waves; scores by rows of the tile, so that each code is converted once for either product
//   32, 64   four waves of scores, by rows of the unit, beside four of outputs
//   128      four waves, both in one stream of instructions, the scores of a tile between the outputs of the one before
// 16 sequences of up to 65536 rows, 16 heads: 130 us, 4.6 TB/s.  16 of 32768 rows, 32 and 64 heads: 88 and 119 us.  32 of 32768
// rows, 128 heads: 293 us; 3 x 512 new tokens over 16384 rows, 128 heads: 4.36 ms, 1.14 PFLOP/s.
#include <algorithm>
#include <cmath>

#include "vkv_runs.h"

namespace vkv {

constexpr int C8_TILE = 64, C8_WAVES = 4, C8_THREADS = 64 * C8_WAVES, C8_STAGES = 3;
constexpr int C8_OFF_ROPE = C8_TILE * D_LAT;                    // of a stage: [64][512] codes, [64][64] bf16
constexpr int C8_STAGE = C8_TILE * VKV_ROW8;                    // 40 KB
// what is read at constant offsets lies first (they have 16 bits), the stages after it
constexpr int C8_OFF_WORD = 0;                                  // per stage and row: the word that holds its scale byte
constexpr int C8_OFF_NOTE = C8_OFF_WORD + C8_STAGES * C8_TILE * 4;   // how far to shift it, or C8_ABSENT
constexpr int C8_OFF_TOP = C8_OFF_NOTE + C8_STAGES * C8_TILE * 4;    // [16] per row of the unit: the waves' largest scores
constexpr int C8_OFF_BAD = C8_OFF_TOP + 16 * 16;                // per wave: whether a score that a mask hides is NaN
constexpr int C8_OFF_P = 2048;                                  // weights: [16][64] fp16
constexpr int C8_OFF_STAGE = C8_OFF_P + 16 * 2 * C8_TILE;       // 1 KB aligned, as pieces are chosen by XORs of the address
constexpr int C8_SMEM = C8_OFF_STAGE + C8_STAGES * C8_STAGE;
static_assert(C8_OFF_BAD + 16 <= C8_OFF_P && C8_OFF_STAGE % 1024 == 0 && C8_OFF_P % 1024 == 0, "");
constexpr uint32_t C8_ABSENT = 255;
// The weight of a code is the row's softmax weight times its power of two, against a reference that follows the largest of
// these (in log2 units): a new one makes the largest 2^first, and it is kept until one is above 2^15.  fp16 holds 11 bits of a
// weight down to 2^-14, fewer below, and nothing under 2^-25, so n rows of one segment that are light one by one lose at most
// n 2^-(25 + first) of what the largest adds to an output.  `first` goes by the rows that a segment may have, so that this is 2^-11 (an
// eighth of half a step of the output's bf16) up to 2^28 of them, 2^-9 up to 2^30.  The larger it is the sooner a reference
// moves, and a move multiplies the outputs: with first = 0, 4, 8 and 12 whatever the size, 32 x 32768 rows of 128 heads took 301,
// 311, 329 and 358 us, 16 x 65536 rows of 16 heads 130, 131, 134 and 142.  The products and sums are fp32, and so is the sum of the
// softmax weights themselves, which are 2^-64 to 2^64 times as large, from unrounded ones: between 2^-64 and 2^109.
constexpr float C8_SLACK = 15.0f;
constexpr float C8_MOST = 32768.0f;   // 2^SLACK: weights are taken as if they were no more, and again where one is
// Does the reference m of this lane's row, whose largest is top, move?  Where one of the wave's rows has to, all do that have come
// nearer by a bit or more: the outputs are multiplied for all of them at once, and seldom.
__device__ __forceinline__ bool moves(float top, float m, float first) {
    bool move = top > m + C8_SLACK;
    if (__ballot(move)) move = top > m + (first + 1.0f);
    return move;
}

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// XOR of the 16-byte piece index within the 512 bytes of tile row r, so that what a group of lanes
// reads at a time lies in 16 pieces that differ modulo 16: the keys' 128-bit reads (16 rows, in two sets
// of 8 whose pieces differ by 9: closed under it, as bits 0 and 3 of this are bits 2 and 3 of r) and the
// values' transposing reads (16 rows of one piece, or rows {0-3, 8-11} or {4-7, 12-15} of two neighbours).
__host__ __device__ constexpr int code_xor(int r) { return ((r & 3) << 1) | (r & 8) | ((r >> 2) & 1); }

template <int OFF>
__device__ __forceinline__ u32x2_t lds_read_tr8(uint32_t addr) {
    u32x2_t v;
    asm volatile("ds_read_b64_tr_b8 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
template <int OFF>
__device__ __forceinline__ u32x4_t lds_read_u4(uint32_t addr) {
    u32x4_t v;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
__device__ __forceinline__ uint32_t lds_read_u1(uint32_t addr) {
    uint32_t v;
    asm volatile("ds_read_b32 %0, %1" : "=v"(v) : "v"(addr));
    return v;
}
__device__ __forceinline__ void lds_write_u1(uint32_t addr, uint32_t v) {
    asm volatile("ds_write_b32 %0, %1" ::"v"(addr), "v"(v) : "memory");
}
__device__ __forceinline__ void lds_write_u2(uint32_t addr, const u32x2_t& v) {
    asm volatile("ds_write_b64 %0, %1" ::"v"(addr), "v"(v) : "memory");
}
__device__ __forceinline__ void lds_write_u4(uint32_t addr, const u32x4_t& v) {
    asm volatile("ds_write_b128 %0, %1" ::"v"(addr), "v"(v) : "memory");
}
// every LDS operation of this wave is through, then every wave's
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// eight codes times sc (a power of two), exact
__device__ __forceinline__ bf16x8_t decode8(uint32_t lo, uint32_t hi, float sc) {
    bf16x2_t v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sc, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sc, true),
                     __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sc, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sc, true)};
    bf16x8_t r;
    __builtin_memcpy(&r, v, 16);
    return r;
}
// eight codes, exact
__device__ __forceinline__ f16x8_t value8(uint32_t lo, uint32_t hi) {
    f16x2_t v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true),
                    __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true)};
    f16x8_t r;
    __builtin_memcpy(&r, v, 16);
    return r;
}
__device__ __forceinline__ float log_scale(float f) { return (float)((int)(__float_as_uint(f) >> 23) - 127); }   // of a power of two
// The largest log2 of a code's weight (but for the reference) among four rows of scores s and scales f (powers of two).
__device__ __forceinline__ float top4(float s0, float s1, float s2, float s3, const float* f, float scale_log2) {
    return fmaxf(fmaxf(__builtin_fmaf(s0, scale_log2, log_scale(f[0])), __builtin_fmaf(s1, scale_log2, log_scale(f[1]))),
                 fmaxf(__builtin_fmaf(s2, scale_log2, log_scale(f[2])), __builtin_fmaf(s3, scale_log2, log_scale(f[3]))));
}
// v times 2^d (d <= 0) where 2^d alone may be below what fp32 holds
__device__ __forceinline__ float times_power(float v, float half) { return v * half * half; }
__device__ __forceinline__ uint32_t drop_nan(uint32_t w) {   // NaN codes become 0
    const uint32_t n = (((w & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u;
    return w & ~((n << 8) - n);
}
// Wave w's 16 rows of a tile (at st in LDS) without NaN codes, where a mask hides a row that holds one: 0 times it would
// not be 0.  (A token that sees such a row has a score that is NaN, whatever its values are.)  Rare.
__device__ __attribute__((noinline)) void clean_tile(uint32_t st, int w, int lane) {
    for (int i = 0; i < 8; ++i) {
        const uint32_t at = st + (16 * w + 2 * i) * D_LAT + 16 * lane;
        u32x4_t v = lds_read_u4<0>(at);
        lds_wait<0>(v);
        for (int q = 0; q < 4; ++q) v[q] = drop_nan(v[q]);
        lds_write_u4(at, v);
    }
    lds_barrier();
}
__device__ __forceinline__ float scale_of(uint32_t word, uint32_t note) {
    const uint32_t s = min(max((word >> (note & 31u)) & 255u, (uint32_t)VKV_SCALE_MIN), (uint32_t)VKV_SCALE_MAX);
    return note == C8_ABSENT ? 0.f : __uint_as_float(s << 23);
}

// One wave's share of a tile of 4 NR rows: NR of them, their codes, branch and scale words.  WORD, NOTE: where the words of all
// stages are, and what is noted of each.  HOLD: a lane's offsets in registers of their own across the loop, not found anew for
// every tile (some 60 cycles a load).
template <int NR, int WORD, int NOTE, bool HOLD>
struct Loader8 {
    static constexpr int TILE = 4 * NR, STAGE = TILE * VKV_ROW8, OFF_ROPE = TILE * D_LAT;
    const Chunk8Args& a;
    const_i32_t* table;
    int kv, wt, lane;
    int32_t e[NR];          // the fetched tile's table entries (scalar)
    uint32_t off[HOLD ? NR / 2 + NR / 8 : 1];

    // among 16 rows of the tile, which the XORs go by, NR = 8 are the first or the last
    __device__ __forceinline__ uint32_t late() const { return NR == 8 ? wt & 1 : 0; }

    __device__ __forceinline__ int row(int t, int i) const { return min(TILE * t + NR * wt + i, kv - 1); }
    __device__ __forceinline__ void fetch(int t) {
        e[0] = table[row(t, 0) >> a.shift];
        if (a.page_mask < NR - 1)
#pragma unroll
            for (int i = 1; i < NR; ++i) e[i] = table[row(t, i) >> a.shift];
    }
    // Are tile t's rows of this wave all there and on one page?  Then scalar row addresses and 32 bits of offset a lane do, and
    // the loads can be issued one by one.
    __device__ __forceinline__ bool plain(int t) const {
        return a.page_mask >= NR - 1 && row(t, 0) + NR <= kv && (uint32_t)e[0] < (uint32_t)a.n_pages && a.rs16 < (1u << 24);
    }
    static constexpr int LOADS = NR / 2 + NR / 8 + 1;
    // this lane's place in load J from its first row on: of two rows' codes, half a wave each, or of eight rows' branch, eight
    // lanes each
    template <int J>
    __device__ __forceinline__ uint32_t place(int ln) const {
        const uint32_t rs = 16 * a.rs16;
        if constexpr (J < NR / 2) {
            const uint32_t p16 = (16 * (ln & 31)) ^ (32 * (ln >> 5)) ^ (128 * late());
            return (p16 ^ (16 * code_xor(2 * J))) + (ln >> 5) * rs;
        } else {
            const uint32_t q16 = 16 * ((ln & 7) ^ ((ln >> 4) & 3)) ^ (64 * late());
            return (q16 ^ (64 * (J - NR / 2))) + (ln >> 3) * rs + D_LAT;
        }
    }
    __device__ __forceinline__ void prepare() {
        if constexpr (HOLD) static_for<0, LOADS - 1>([&](auto ic) { off[decltype(ic)::value] = place<decltype(ic)::value>(lane); });
    }
    template <int J>
    __device__ __forceinline__ void part(int t, uint8_t* smem, uint32_t lds0, int sg, int stages, int ln) const {
        uint8_t* st = smem + stages + sg * STAGE;
        const uint32_t r = row(t, 0) & a.page_mask;
        const char* b = reinterpret_cast<const char*>(a.cache8) + 16 * ((uint64_t)(uint32_t)e[0] * a.ps16 + (uint64_t)r * a.rs16);
        if constexpr (J < LOADS - 1) {
            constexpr int i = J < NR / 2 ? 2 * J : 8 * (J - NR / 2);
            const int at = J < NR / 2 ? D_LAT * (NR * wt + i) : OFF_ROPE + 2 * D_ROPE * (NR * wt + i);
            uint32_t o;
            if constexpr (HOLD) o = off[J];
            else o = place<J>(ln);
            __builtin_amdgcn_global_load_lds((gbl_void_t*)(b + (uint64_t)(16 * a.rs16) * i + o), (lds_void_t*)(st + at), 16, 0, 0);
        } else if (ln < NR) {                   // the aligned words around the scale bytes
            const uint64_t s0 = (uint64_t)(uintptr_t)(a.scale + (uint64_t)(uint32_t)e[0] * (uint64_t)a.sstride);
            const uint32_t at = (uint32_t)(s0 & 3) + ((r + ln) >> a.bshift);
            __builtin_amdgcn_global_load_lds((gbl_void_t*)(uintptr_t)((s0 & ~3ull) + (at & ~3u)),
                                             (lds_void_t*)(smem + WORD + (sg * TILE + NR * wt) * 4), 4, 0, 0);
            lds_write_u1(lds0 + NOTE + (sg * TILE + NR * wt + ln) * 4, 8u * (at & 3u));
        }
    }
    // the loads of the fetched tile t into stage sg
    __device__ __forceinline__ void issue(int t, uint8_t* smem, uint32_t lds0, int sg, int stages) const {
        int ln = lane;
        if constexpr (!HOLD) asm volatile("" : "+v"(ln));   // keeps the lane arithmetic out of registers across the loop
        if (plain(t)) static_for<0, LOADS>([&](auto ic) { part<decltype(ic)::value>(t, smem, lds0, sg, stages, ln); });
        else issue_any(t, smem, lds0, sg, stages);
    }
    __device__ __forceinline__ void issue_any(int t, uint8_t* smem, uint32_t lds0, int sg, int stages) const {
        uint8_t* st = smem + stages + sg * STAGE;
        const int u = row(t, 0);
        const char* base[NR];
        const uint8_t* word;     // this lane's (of NR) scale byte
        uint32_t absent;
        int ln = lane;
        asm volatile("" : "+v"(ln));   // keeps the lane arithmetic out of registers across the loop
        const int mine = ln & (NR - 1);
        if (a.page_mask >= NR - 1) {   // the rows lie on one page; rows past the end: the last row's
            const int last = min(kv - 1 - u, NR - 1);
            const bool there = (uint32_t)e[0] < (uint32_t)a.n_pages;
            const uint32_t p = there ? e[0] : 0, r = there ? u & a.page_mask : 0;
            base[0] = reinterpret_cast<const char*>(a.cache8) + 16 * ((uint64_t)p * a.ps16 + (uint64_t)r * a.rs16);
#pragma unroll
            for (int i = 1; i < NR; ++i) base[i] = base[i - 1] + (there && i <= last ? 16 * (uint64_t)a.rs16 : 0);
            word = a.scale + (uint64_t)p * (uint64_t)a.sstride + (there ? (r + (uint32_t)min(mine, last)) >> a.bshift : 0);
            absent = there ? 0 : C8_ABSENT;
        } else {
            uint64_t pl = 0;
            uint32_t rl = 0;
            absent = 0;
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const bool there = (uint32_t)e[i] < (uint32_t)a.n_pages;
                const uint32_t p = there ? e[i] : 0, r = there ? row(t, i) & a.page_mask : 0;
                base[i] = reinterpret_cast<const char*>(a.cache8) + 16 * ((uint64_t)p * a.ps16 + (uint64_t)r * a.rs16);
                if (mine == i) {
                    pl = (uint64_t)p * (uint64_t)a.sstride;
                    rl = r;
                    absent = there ? 0 : C8_ABSENT;
                }
            }
            word = a.scale + pl + (rl >> a.bshift);
        }
        const int hb = ln >> 5;
#pragma unroll
        for (int i = 0; i < NR; i += 2) {
            const char* b = hb ? base[i + 1] : base[i];
            const uint32_t off = 16 * ((uint32_t)(ln & 31) ^ (uint32_t)code_xor(i) ^ (uint32_t)(2 * hb) ^ (8 * late()));
            __builtin_amdgcn_global_load_lds((gbl_void_t*)(b + off), (lds_void_t*)(st + D_LAT * (NR * wt + i)), 16, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < NR; j += 8) {      // eight rows, eight lanes each
            const char* b = base[j];
#pragma unroll
            for (int i = 1; i < 8; ++i) b = (ln >> 3) == i ? base[j + i] : b;
            const int r = j + 8 * (int)late() + (ln >> 3);
            __builtin_amdgcn_global_load_lds((gbl_void_t*)(b + D_LAT + 16 * ((ln & 7) ^ rope_xor(r))),
                                             (lds_void_t*)(st + OFF_ROPE + 2 * D_ROPE * (NR * wt + j)), 16, 0, 0);
        }
        if (ln < NR) {   // the aligned word around the byte
            const uint64_t at = (uint64_t)(uintptr_t)word;
            __builtin_amdgcn_global_load_lds((gbl_void_t*)(uintptr_t)(at & ~3ull),
                                             (lds_void_t*)(smem + WORD + (sg * TILE + NR * wt) * 4), 4, 0, 0);
            lds_write_u1(lds0 + NOTE + (sg * TILE + NR * wt + ln) * 4, absent ? C8_ABSENT : 8u * (uint32_t)(at & 3u));
        }
    }
};

typedef Loader8<16, C8_OFF_WORD, C8_OFF_NOTE, true> Loader64;   // tiles of 64 rows
typedef Loader8<16, C8_OFF_WORD, C8_OFF_NOTE, false> Loader64Lean;

// ------------------------------------------------------------------ a segment

// v *= f for four accumulator registers: said so that the compiler keeps the outputs where the products add to them (with
// plain products it copies all of them to the other registers and back around every tile).  The products that wrote v and
// those that read it next are a barrier away, as far as their wait states go.
__device__ __forceinline__ void scale_acc(float& v0, float& v1, float& v2, float& v3, float f) {
    float t0, t1, t2, t3;
    asm volatile("v_accvgpr_read_b32 %4, %0\n\tv_accvgpr_read_b32 %5, %1\n\tv_accvgpr_read_b32 %6, %2\n\tv_accvgpr_read_b32 %7, %3\n\t"
                 "v_mul_f32 %4, %4, %8\n\tv_mul_f32 %5, %5, %8\n\tv_mul_f32 %6, %6, %8\n\tv_mul_f32 %7, %7, %8\n\t"
                 "v_accvgpr_write_b32 %0, %4\n\tv_accvgpr_write_b32 %1, %5\n\tv_accvgpr_write_b32 %2, %6\n\tv_accvgpr_write_b32 %3, %7"
                 : "+a"(v0), "+a"(v1), "+a"(v2), "+a"(v3), "=&v"(t0), "=&v"(t1), "=&v"(t2), "=&v"(t3) : "v"(f));
}
template <int N, typename V>
__device__ __forceinline__ void scale_all(V& o, float f) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        float v0 = o[i], v1 = o[i + 1], v2 = o[i + 2], v3 = o[i + 3];
        scale_acc(v0, v1, v2, v3, f);
        o[i] = v0, o[i + 1] = v1, o[i + 2] = v2, o[i + 3] = v3;
    }
}

// Tiles [t0, t1) of unit x (16 rows) by one workgroup.  part: where an incomplete unit's (O, m, l) go, or null (outputs).
// Wave w takes the scores of rows 16 w .. + 15 of a tile and the output dims from 128 w on.  Weights are taken against the
// reference that every wave has, while the waves' maxima are exchanged, and again where these move it.
__device__ __forceinline__ void chunk8_segment(const Chunk8Args& a, const CkUnit& x, int t0, int t1, float* part_o,
                                               float* part_ml, uint8_t* smem) {
    constexpr int NO = 8, KS = 2;                 // the outputs' blocks of dims, and steps along the tile
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t lds0 = lds_addr(smem);
    const int Rc = min(x.row0 + c, x.nrow - 1);                 // rows past the end repeat the last one, never stored
    const int lim = min(x.old + Rc / a.H, x.kv - 1);            // the last cache row that this lane's row sees
    const int lim_lo = __builtin_amdgcn_readfirstlane(min(x.old + x.row0 / a.H, x.kv - 1));
    const int nt = x.kv > 0 ? t1 - t0 : 0;

    Loader64 loader{a, (const_i32_t*)(a.table + (int64_t)x.b * a.tstride), x.kv, w, lane, {}, {}};
    loader.prepare();
    // pieces of a key's codes that this lane reads: step s takes piece s ^ 9 (g & 1) ^ 16 (g >> 1), half after half
    const int pg = 9 * (g & 1) ^ 16 * (g >> 1);
    bf16x8_t qf[18];
    {
        const int64_t row = x.tok0 * a.H + Rc;
        const uint16_t* ql = a.q_lat + row * a.qls;
        const uint16_t* qr = a.q_rope + row * a.qrs + 8 * g;
#pragma unroll
        for (int s = 0; s < 16; ++s) qf[s] = *reinterpret_cast<const bf16x8_t*>(ql + 16 * ((s >> 1) ^ pg) + 8 * (s & 1));
#pragma unroll
        for (int s = 0; s < 2; ++s) qf[16 + s] = *reinterpret_cast<const bf16x8_t*>(qr + 32 * s);
    }
    if (nt > 0) {
        loader.fetch(t0);
        loader.issue(t0, smem, lds0, 0, C8_OFF_STAGE);
        loader.fetch(t0 + 1);
        if (nt > 1) {
            loader.issue(t0 + 1, smem, lds0, 1, C8_OFF_STAGE);
            loader.fetch(t0 + 2);
        }
    }
#pragma unroll
    for (int s = 0; s < 18; ++s) asm volatile("" : "+v"(qf[s]));   // no wait for them inside the tile loop

    f32x4_t o[NO];
#pragma unroll
    for (int d = 0; d < NO; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, w_top = 0.f, l_run = 0.f;   // reference, this lane's largest weight since it moved, sum

    int sg = 0;   // the stage of tile k
    for (int k = 0; k < nt; ++k) {
        // this wave's share of tile k has landed, and every wave's; what was read of tile k - 1 and its weights has been used
        if (k + 1 < nt)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Loader64::LOADS) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
        if (k + 2 < nt) loader.issue(t0 + k + 2, smem, lds0, sg == 0 ? 2 : sg - 1, C8_OFF_STAGE);
        const int u0 = C8_TILE * (t0 + k);
        const uint32_t st = lds0 + C8_OFF_STAGE + sg * C8_STAGE;
        const uint32_t wn = lds0 + C8_OFF_WORD + (sg * C8_TILE + lane) * 4;
        sg = sg == 2 ? 0 : sg + 1;

        // ---- scores of rows 16 w .. + 15 of the tile
        uint32_t word = lds_read_u1(wn), note = lds_read_u1(wn + (C8_OFF_NOTE - C8_OFF_WORD));
        const uint32_t ka = st + (16 * w + c) * D_LAT + ((16 * pg) ^ (16 * code_xor(c)));
        const uint32_t ra = st + C8_OFF_ROPE + (16 * w + c) * (2 * D_ROPE) + 16 * (g ^ rope_xor(c));
        constexpr int SD = 3;          // operands read ahead of the matrix cores: 8 of codes, 2 of the branch
        u32x4_t kc[SD + 1];
        auto kload = [&](auto sc_) {
            constexpr int s = decltype(sc_)::value;
            kc[s % (SD + 1)] = lds_read_u4<0>(s < 8 ? ka ^ (16 * s) : ra ^ (64 * (s - 8)));
        };
        static_for<0, SD>(kload);
        lds_wait<SD>(word, note);
        const float sc = scale_of(word, note);                  // of tile row `lane`
        const uint64_t absent = __ballot(sc == 0.f);
        const float sk = __shfl(sc, 16 * w + c);                // of the key this lane decodes
        float sp[4];                                            // of those whose scores it gets: 16 w + 4 g + i
#pragma unroll
        for (int i = 0; i < 4; ++i) sp[i] = __shfl(sc, 16 * w + 4 * g + i);
        f32x4_t s4 = {0.f, 0.f, 0.f, 0.f};
        static_for<0, 10>([&](auto sc_) {
            constexpr int s = decltype(sc_)::value;
            if constexpr (s + SD < 10) kload(std::integral_constant<int, s + SD>{});
            u32x4_t& v = kc[s % (SD + 1)];
            lds_wait<(s + SD < 10) ? SD : 9 - s>(v);
            if constexpr (s < 8) {
                const bf16x8_t k0 = decode8(v[0], v[1], sk), k1 = decode8(v[2], v[3], sk);
                s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[2 * s], s4, 0, 0, 0);
                s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[2 * s + 1], s4, 0, 0, 0);
            } else {
                s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v), qf[8 + s], s4, 0, 0, 0);
            }
        });

        // ---- masks
        bool bad = false;
        if (u0 + C8_TILE - 1 > lim_lo || absent != 0) {
            const uint32_t gone = (uint32_t)(absent >> (16 * w + 4 * g));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (u0 + 16 * w + 4 * g + i > lim || ((gone >> i) & 1u)) {
                    bad |= s4[i] != s4[i];
                    s4[i] = -INFINITY;
                }
        }
        // ---- weights against the reference that every wave has, and again where one of them is too large for it
        float ps, most;
        auto weights = [&]() __attribute__((always_inline)) {
            const float ref = m_run == -INFINITY ? 0.f : m_run;
            f16x4_t p4;
            ps = most = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s4[i], a.scale_log2, -ref)), v = p * sp[i];
                ps += p;
                most = fmaxf(most, v);
                p4[i] = (_Float16)v;
            }
            lds_write_u2(lds0 + C8_OFF_P + c * (2 * C8_TILE) + 16 * ((2 * w + (g >> 1)) ^ rope_xor(c)) + 8 * (g & 1),
                         __builtin_bit_cast(u32x2_t, p4));
        };
        weights();
        const uint32_t flags = (__ballot(most > C8_MOST || m_run == -INFINITY) ? 1u : 0u) | (__ballot(bad) ? 2u : 0u);
        if (lane == 0) lds_write_u1(lds0 + C8_OFF_BAD + 4 * w, flags);
        lds_barrier();
        u32x4_t fl = lds_read_u4<C8_OFF_BAD>(lds0);
        lds_wait<0>(fl);
        const uint32_t any = __builtin_amdgcn_readfirstlane((fl[0] | fl[1]) | (fl[2] | fl[3]));
        if (any & 1u) {
            float top = m_run == -INFINITY ? -INFINITY : m_run + __builtin_amdgcn_logf(w_top);
            top = fmaxf(top, top4(s4[0], s4[1], s4[2], s4[3], sp, a.scale_log2));
            top = allreduce_groups(top, [](float p, float q) { return fmaxf(p, q); });
            if (g == 0) lds_write_u1(lds0 + C8_OFF_TOP + c * 16 + 4 * w, __float_as_uint(top));
            lds_barrier();
            u32x4_t tops = lds_read_u4<C8_OFF_TOP>(lds0 + c * 16);
            lds_wait<0>(tops);
            const float m_top = fmaxf(fmaxf(__uint_as_float(tops[0]), __uint_as_float(tops[1])),
                                      fmaxf(__uint_as_float(tops[2]), __uint_as_float(tops[3])));
            const bool move = moves(m_top, m_run, a.first);
            const float next = move ? m_top - a.first : m_run, half = move ? __builtin_amdgcn_exp2f(0.5f * (m_run - next)) : 1.0f;
            const float al = half * half;
            if (__ballot(move && m_run != -INFINITY)) {   // (else there is nothing yet; the same in every wave)
#pragma unroll
                for (int d = 0; d < NO; ++d) scale_all<4>(o[d], al);
            }
            l_run = times_power(l_run, half);
            m_run = next;
            if (move) w_top = __builtin_amdgcn_exp2f(a.first);
            weights();
            lds_barrier();
        }
        w_top = fmaxf(w_top, most);
        l_run += ps;   // this lane's share of the sum

        // after the waits for every LDS operation, which would be waits for these scalar loads too
        if (k + 2 < nt) loader.fetch(t0 + k + 3);

        // ---- outputs, dims 128 w .. + 127
        u32x4_t pf[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) pf[s] = lds_read_u4<C8_OFF_P>(lds0 + c * (2 * C8_TILE) + 16 * ((4 * s + g) ^ rope_xor(c)));
        const int vr = 8 * g + (c >> 1);       // the row within a lane group's eight, its place among the tile's
        const uint32_t va = st + vr * D_LAT + 16 * ((8 * w) ^ code_xor(vr)) + 8 * (lane & 1);
        if (any & 2u) {
            lds_wait<0>(pf[0], pf[1]);         // nothing is on its way over the call
            clean_tile(st, w, lane);
        }
        constexpr int N = KS * NO, VD = 6;
        u32x2_t vv[VD + 1];
        auto vload = [&](auto ic) {
            constexpr int i = decltype(ic)::value, s = i / NO, d = i % NO;
            vv[i % (VD + 1)] = lds_read_tr8<32 * D_LAT * s>(va ^ (16 * d));
        };
        static_for<0, VD>(vload);
        static_for<0, N>([&](auto ic) {
            constexpr int i = decltype(ic)::value, s = i / NO, d = i % NO;
            if constexpr (i + VD < N) vload(std::integral_constant<int, i + VD>{});
            if constexpr (i == 0) lds_wait<VD + 1>(pf[0], pf[1]);
            lds_wait<(i + VD < N) ? VD : N - 1 - i>(vv[i % (VD + 1)]);
            const f16x8_t v = value8(vv[i % (VD + 1)][0], vv[i % (VD + 1)][1]);
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, __builtin_bit_cast(f16x8_t, pf[s]), o[d], 0, 0, 0);
        });
    }

    // ---- the sums of the waves' rows
    __syncthreads();
    float* sums = reinterpret_cast<float*>(smem + C8_OFF_TOP);   // [row][wave]
    l_run = allreduce_groups(l_run, [](float p, float q) { return p + q; });
    if (g == 0) sums[4 * c + w] = l_run;
    __syncthreads();
    const float l = (sums[4 * c] + sums[4 * c + 1]) + (sums[4 * c + 2] + sums[4 * c + 3]);
    const int R = x.row0 + c;
    if (part_o) {
        // accumulator order: [wave][dim block][64 lanes][4]
#pragma unroll
        for (int d = 0; d < NO; ++d) *reinterpret_cast<f32x4_t*>(part_o + ((w * NO + d) * 64 + lane) * 4) = o[d];
        if (w == 0 && g == 0) {
            part_ml[2 * c] = m_run;
            part_ml[2 * c + 1] = l;
        }
    } else if (R < x.nrow) {
        const int64_t at = x.tok0 * a.H + R;
        const bool none = m_run == -INFINITY && l == 0.f;
        const float inv = none ? 0.f : 1.0f / l;
        uint16_t* out = a.out + at * D_LAT + 128 * w + 4 * g;
#pragma unroll
        for (int d = 0; d < NO; ++d) {
            const bf16x4_t v = {(__bf16)(o[d][0] * inv), (__bf16)(o[d][1] * inv), (__bf16)(o[d][2] * inv), (__bf16)(o[d][3] * inv)};
            *reinterpret_cast<bf16x4_t*>(out + 16 * d) = v;
        }
        if (w == 0 && g == 0) a.lse[at] = lse_of(m_run, l);
    }
}

// What becomes of a row block's outputs (the dims 128 w .. + 127 of row R of a unit of 32 RB rows, 32x32 layout): a part, or the outputs
// at row `at` of the call's if it is one.
template <int RB, typename Out>
__device__ __forceinline__ void finish_rows(const Chunk8Args& a, int64_t at, bool live, int row, int rb, int w, int lane, float m, float l,
                                            Out&& o, float* part_o, float* part_ml) {
    if (part_o) {
        // accumulator order: [wave][dim block][row block][4][64 lanes][4]
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4_t v = {o(d)[4 * q], o(d)[4 * q + 1], o(d)[4 * q + 2], o(d)[4 * q + 3]};
                *reinterpret_cast<f32x4_t*>(part_o + ((((w * 4 + d) * RB + rb) * 4 + q) * 64 + lane) * 4) = v;
            }
        if (w == 0 && lane < 32) {
            part_ml[2 * row] = m;
            part_ml[2 * row + 1] = l;
        }
    } else if (live) {
        const bool none = m == -INFINITY && l == 0.f;
        const float inv = none ? 0.f : 1.0f / l;
        uint16_t* out = a.out + at * D_LAT + 128 * w + 4 * (lane >> 5);
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const bf16x4_t v = {(__bf16)(o(d)[4 * q] * inv), (__bf16)(o(d)[4 * q + 1] * inv), (__bf16)(o(d)[4 * q + 2] * inv),
                                    (__bf16)(o(d)[4 * q + 3] * inv)};
                *reinterpret_cast<bf16x4_t*>(out + 32 * d + 8 * q) = v;
            }
        if (w == 0 && lane < 32) a.lse[at] = lse_of(m, l);
    }
}

// ------------------------------------------------- a segment of a unit of 128 rows

// As above, but the queries of 128 rows do not fit in every wave: wave w takes the scores of rows 32 w .. + 31 of the unit
// against all of the tile's rows, and 128 dims of all rows' outputs.  It has its rows' scores to itself, so
// their reference moves before the weights are written; the other waves learn by how much.
//
// A wave has its SIMD to itself, so what keeps the matrix cores busy while codes are converted (vector instructions,
// about as long as the products that they feed) has to be in the same instruction stream: the scores of tile k + 1 are
// taken between the outputs of tile k, four products of either at a time.
constexpr int B8_P = 128 * 2 * C8_TILE;                         // weights of a tile, [128][64] fp16; two of them
constexpr int B8_OFF_SCALE = C8_OFF_TOP;                        // [64] the tile's scales (every wave writes the same ones)
constexpr int B8_OFF_ALPHA = B8_OFF_SCALE + 4 * C8_TILE;        // two of [128]: by what a row's outputs are to be multiplied
constexpr int B8_OFF_BAD = B8_OFF_ALPHA + 2 * 512;              // two of [4]: the waves' flags, outputs to multiply, a hidden NaN
constexpr int B8_OFF_P = 3 * 1024;
constexpr int B8_OFF_STAGE = B8_OFF_P + 2 * B8_P;
constexpr int B8_SMEM = B8_OFF_STAGE + C8_STAGES * C8_STAGE;
static_assert(B8_OFF_BAD + 32 <= B8_OFF_P && B8_OFF_STAGE % 1024 == 0, "");

// The products of the scores are written as instructions: their results have to lie in the registers that the vector
// units read (the compiler takes accumulators for every product of a kernel that needs some, where these do not fit
// beside the outputs).  It does not see them, so the wait states are here: two from an operand's conversion to the
// product, and after the last products, in their own statement, what a reader of the result has to wait (12 from the
// last one's issue, 8 passes).
__device__ __forceinline__ void score_first(f32x16_t& s, const bf16x8_t& k, const bf16x8_t& q) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "v"(q));
}
template <bool NEAR>   // the conversion is right before (else an output's product and a conversion lie between)
__device__ __forceinline__ void score_next(f32x16_t& s, const bf16x8_t& k, const bf16x8_t& q) {
    if constexpr (NEAR) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "v"(q));
    else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "v"(q));
}
__device__ __forceinline__ void score_last(f32x16_t& s0, f32x16_t& s1, const bf16x8_t& k0, const bf16x8_t& k1, const bf16x8_t& q) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %2, %4, %0\n\tv_mfma_f32_32x32x16_bf16 %1, %3, %4, %1\n\ts_nop 15\n\ts_nop 7"
                 : "+v"(s0), "+v"(s1) : "v"(k0), "v"(k1), "v"(q));
}

// What the fused loop has in flight of LDS reads: in step j (from -AHEAD: before the loop) the keys of step j + AHEAD (two
// reads), the values of step j + AHEAD (one), and at the end of every fourth step the weights of the next four (four).
constexpr int B8_AHEAD = 2, B8_STEPS = 20, B8_OUT = 16;
template <bool SCORES, bool OUT>
constexpr int reads_keys(int j) { return SCORES && j + B8_AHEAD < B8_STEPS ? 2 : 0; }
template <bool SCORES, bool OUT>
constexpr int reads_values(int j) { return OUT && j + B8_AHEAD < B8_OUT ? 1 : 0; }
template <bool SCORES, bool OUT>
constexpr int reads_weights(int j) { return OUT && j >= 0 && j % 4 == 3 && j + 1 < B8_OUT ? 4 : 0; }
// reads behind those of a step's keys or values, at the place where they are waited for
template <bool SCORES, bool OUT>
constexpr int reads_step(int j) { return reads_keys<SCORES, OUT>(j) + reads_values<SCORES, OUT>(j); }
template <bool SCORES, bool OUT>
constexpr int reads_between(int i) {   // of the steps i - AHEAD + 1 .. i - 1, and the weights of step i - AHEAD
    int n = reads_weights<SCORES, OUT>(i - B8_AHEAD);
    for (int j = i - B8_AHEAD + 1; j < i; ++j) n += reads_step<SCORES, OUT>(j) + reads_weights<SCORES, OUT>(j);
    return n;
}
template <bool SCORES, bool OUT>
constexpr int behind_keys(int i) {     // step i's keys, in step i after its reads
    return reads_values<SCORES, OUT>(i - B8_AHEAD) + reads_between<SCORES, OUT>(i) + reads_step<SCORES, OUT>(i);
}
template <bool SCORES, bool OUT>
constexpr int behind_next(int i) {     // step i + 1's keys, in step i before its last product for the outputs (and the read behind it)
    const int w = reads_weights<SCORES, OUT>(i);
    return reads_values<SCORES, OUT>(i + 1 - B8_AHEAD) + reads_between<SCORES, OUT>(i + 1) - w + (w ? 3 : 0);
}
template <bool SCORES, bool OUT>
constexpr int behind_values(int i) {   // step i + 1's values, in step i after its reads
    return reads_between<SCORES, OUT>(i + 1) - reads_weights<SCORES, OUT>(i);
}
static_assert(B8_AHEAD == 2, "");   // (the values' registers are two)

struct Big8 {
    bf16x8_t qf[36];     // Q^T operand: step 2 s + i (i < 2) has dims 32 s + 16 h + 8 i .. + 7, as a 16-byte piece of codes holds them
    f32x16_t o[4][4];    // outputs, [dim block][row block]
    f32x16_t s[2];       // scores: s[b][i] is tile row 32 b + 8 (i / 4) + 4 h + i % 4
};

// Outputs of the tile in stage sv with the weights at pw, and scores of the tile in stage sk.  Returns this lane's scale (of
// tile row `lane` of the latter).
template <bool SCORES, bool OUT>
__device__ __forceinline__ float fused8(Big8& z, uint32_t lds0, uint32_t sv, uint32_t pw, uint32_t sk, uint32_t wn, int w, int lane) {
    int ln = lane;
    asm volatile("" : "+v"(ln));   // operand addresses are found anew from it, so that no registers hold them across the loop
    const int r = ln & 31, hh = ln >> 5;
    // values: a lane group's eight rows of 16, its place among the dims; weights: row r, piece 2 step + h
    const int e = (ln >> 1) & 7, vr = 4 * hh + (e & 3) + 8 * (e >> 2);
    const uint32_t va = sv + vr * D_LAT + 16 * ((8 * w + ((ln >> 4) & 1)) ^ code_xor(vr)) + 8 * (ln & 1);
    const uint32_t pr = pw + r * (2 * C8_TILE) + 16 * (hh ^ rope_xor(r));
    // keys: pieces 2 s + h of rows r and 32 + r
    const uint32_t ka = sk + r * D_LAT + 16 * (hh ^ code_xor(r & 15));
    const uint32_t ra = sk + C8_OFF_ROPE + r * (2 * D_ROPE) + 16 * (hh ^ rope_xor(r));
    constexpr int NB = B8_AHEAD + 1;
    u32x4_t kc[NB][2], pf[4];
    u32x2_t vv[2];
    float sc = 0.f, sk2[2] = {0.f, 0.f};
    auto kload = [&](auto ic) {
        constexpr int i = decltype(ic)::value;
        if constexpr (SCORES && i < B8_STEPS) {
            if constexpr (i < 16) {
                kc[i % NB][0] = lds_read_u4<0>(ka ^ (32 * i));
                kc[i % NB][1] = lds_read_u4<32 * D_LAT>(ka ^ (32 * i));
            } else {
                kc[i % NB][0] = lds_read_u4<0>(ra ^ (32 * (i - 16)));
                kc[i % NB][1] = lds_read_u4<32 * 2 * D_ROPE>(ra ^ (32 * (i - 16)));
            }
        }
    };
    auto vload = [&](auto ic) {
        constexpr int i = decltype(ic)::value;
        if constexpr (OUT && i < B8_OUT) vv[i % 2] = lds_read_tr8<16 * D_LAT * (i >> 2)>(va ^ (32 * (i & 3)));
    };
    auto pload = [&](auto sc_, auto rc) {
        constexpr int s = decltype(sc_)::value, rb = decltype(rc)::value;
        pf[rb] = lds_read_u4<rb * 32 * 2 * C8_TILE>(pr ^ (32 * s));
    };
    uint32_t word = 0, note = C8_ABSENT;
    if constexpr (SCORES) {
        word = lds_read_u1(wn);
        note = lds_read_u1(wn + (C8_OFF_NOTE - C8_OFF_WORD));
    }
    if constexpr (OUT) static_for<0, 4>([&](auto rc) { pload(std::integral_constant<int, 0>{}, rc); });
    static_for<0, B8_AHEAD>([&](auto ic) {
        kload(ic);
        vload(ic);
    });
    if constexpr (SCORES) {
        lds_wait<(OUT ? 4 + 3 * B8_AHEAD : 2 * B8_AHEAD)>(word, note);
        sc = scale_of(word, note);
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(sc), __float_as_uint(sc), false, false);
        sk2[0] = __uint_as_float(sw[0]);     // of rows r and 32 + r
        sk2[1] = __uint_as_float(sw[1]);
    }
    // the operands of the next products: a key's is decoded while the product before it runs, a step's values during the last one
    bf16x8_t kd;
    f16x8_t vd[2];
    auto vwait = [&](auto ic, auto n) {
        lds_wait<decltype(n)::value>(vv[decltype(ic)::value % 2]);
    };
    auto kdecode = [&](auto ic, auto qc) {
        constexpr int i = decltype(ic)::value, q = decltype(qc)::value;
        const u32x4_t& k4 = kc[i % NB][q & 1];
        kd = decode8(k4[2 * (q >> 1)], k4[2 * (q >> 1) + 1], sk2[q & 1]);
    };
    if constexpr (SCORES) {
        lds_wait<(OUT ? 1 : 0) + (B8_AHEAD - 1) * (OUT ? 3 : 2)>(kc[0][0], kc[0][1]);
        kdecode(std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{});
    }
    if constexpr (OUT) {
        vwait(std::integral_constant<int, 0>{}, std::integral_constant<int, (B8_AHEAD - 1) * (SCORES ? 3 : 1)>{});
        vd[0] = value8(vv[0][0], vv[0][1]);
    }
    static_for<0, (SCORES ? B8_STEPS : B8_OUT)>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        constexpr bool out = OUT && i < B8_OUT, more = OUT && i + 1 < B8_OUT;
        kload(std::integral_constant<int, i + B8_AHEAD>{});
        vload(std::integral_constant<int, i + B8_AHEAD>{});
        if constexpr (SCORES && i >= 16) lds_wait<behind_keys<SCORES, OUT>(i)>(kc[i % NB][0], kc[i % NB][1]);
        if constexpr (more) lds_wait<behind_values<SCORES, OUT>(i)>(vv[(i + 1) % 2]);
        static_for<0, 4>([&](auto rc) {      // a product of either kind, and conversions behind each
            constexpr int q = decltype(rc)::value, half = q >> 1, b = q & 1;
            if constexpr (SCORES && i < 16) {
                if constexpr (i == 0 && half == 0) score_first(z.s[b], kd, z.qf[0]);
                else score_next<!more>(z.s[b], kd, z.qf[2 * i + half]);
                if constexpr (q < 3) {
                    kdecode(ic, std::integral_constant<int, q + 1>{});
                } else if constexpr (i + 1 < 16) {
                    lds_wait<behind_next<SCORES, OUT>(i)>(kc[(i + 1) % NB][0], kc[(i + 1) % NB][1]);
                    kdecode(std::integral_constant<int, i + 1>{}, std::integral_constant<int, 0>{});
                }
            } else if constexpr (SCORES && i < B8_STEPS - 1) {
                if constexpr (half == 0) score_next<true>(z.s[b], __builtin_bit_cast(bf16x8_t, kc[i % NB][b]), z.qf[16 + i]);
            } else if constexpr (SCORES && q == 0) {
                score_last(z.s[0], z.s[1], __builtin_bit_cast(bf16x8_t, kc[i % NB][0]), __builtin_bit_cast(bf16x8_t, kc[i % NB][1]), z.qf[16 + i]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (out) {
                constexpr int s = i >> 2, d = i & 3;
                // the weights came at the end of the last step: behind each are the later ones, and this step's keys and values
                if constexpr (d == 0) lds_wait<3 - q + reads_keys<SCORES, OUT>(i) + reads_values<SCORES, OUT>(i)>(pf[q]);
                z.o[d][q] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vd[i & 1], __builtin_bit_cast(f16x8_t, pf[q]), z.o[d][q], 0, 0, 0);
                if constexpr (d == 3 && more) pload(std::integral_constant<int, s + 1>{}, rc);
                if constexpr (more) {        // a quarter of the next step's values
                    const uint32_t word = vv[(i + 1) % 2][q >> 1];
                    const f16x2_t two = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, 1.0f, q & 1);
                    vd[(i + 1) & 1][2 * q] = two[0];
                    vd[(i + 1) & 1][2 * q + 1] = two[1];
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    });
    return sc;
}

__device__ __forceinline__ void chunk8_big_segment(const Chunk8Args& a, const CkUnit& x, int t0, int t1, float* part_o,
                                                   float* part_ml, uint8_t* smem) {
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, h = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t lds0 = lds_addr(smem);
    const int first = min(x.row0 + 32 * w, x.nrow - 1);
    const int Rc = min(x.row0 + 32 * w + c, x.nrow - 1);        // rows past the end repeat the last one, never stored
    const int lim = min(x.old + Rc / a.H, x.kv - 1);            // the last cache row that this lane's row sees
    const int lim_lo = __builtin_amdgcn_readfirstlane(min(x.old + first / a.H, x.kv - 1));
    const int nt = x.kv > 0 ? t1 - t0 : 0;

    Loader64Lean loader{a, (const_i32_t*)(a.table + (int64_t)x.b * a.tstride), x.kv, w, lane, {}, {}};
    Big8 z;
    {
        const int64_t row = x.tok0 * a.H + Rc;
        const uint16_t* ql = a.q_lat + row * a.qls + 16 * h;
        const uint16_t* qr = a.q_rope + row * a.qrs + 8 * h;
#pragma unroll
        for (int s = 0; s < 32; ++s) z.qf[s] = *reinterpret_cast<const bf16x8_t*>(ql + 32 * (s >> 1) + 8 * (s & 1));
#pragma unroll
        for (int s = 0; s < 4; ++s) z.qf[32 + s] = *reinterpret_cast<const bf16x8_t*>(qr + 16 * s);
    }
    if (nt > 0) {
        loader.fetch(t0);
        loader.issue(t0, smem, lds0, 0, B8_OFF_STAGE);
        loader.fetch(t0 + 1);
        if (nt > 1) {
            loader.issue(t0 + 1, smem, lds0, 1, B8_OFF_STAGE);
            loader.fetch(t0 + 2);
        }
    }
#pragma unroll
    for (int s = 0; s < 36; ++s) asm volatile("" : "+v"(z.qf[s]));   // no wait for them inside the tile loop
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) z.o[d][r][i] = 0.f;
    float m_run = -INFINITY, m_top = -INFINITY, l_run = 0.f;   // reference, largest, sum

    // the weights of the tile whose scores are there (rows from u0 on), into buffer k & 1
    auto weights = [&](int k, int u0, float sc) __attribute__((always_inline)) {
        int ln = lane;
        asm volatile("" : "+v"(ln));          // (as above)
        const int c = ln & 31, h = ln >> 5;
        const uint32_t own = lds0 + B8_OFF_SCALE;
        lds_write_u1(own + 4 * ln, __float_as_uint(sc));
        const uint64_t absent = __ballot(sc == 0.f);
        u32x4_t f[8];                         // of the rows whose scores this lane has, in their order
        static_for<0, 8>([&](auto ic) { f[decltype(ic)::value] = lds_read_u4<32 * decltype(ic)::value>(own + 16 * h); });
        bool bad = false;
        if (u0 + C8_TILE - 1 > lim_lo || absent != 0) {
            const int last = lim - u0 - 4 * h;
            const uint64_t gone = absent >> (4 * h);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int row = 32 * b + 8 * (i >> 2) + (i & 3);
                    if (row > last || ((gone >> row) & 1u)) {
                        bad |= z.s[b][i] != z.s[b][i];
                        z.s[b][i] = -INFINITY;
                    }
                }
        }
        static_for<0, 4>([&](auto ic) { lds_wait<0>(f[2 * decltype(ic)::value], f[2 * decltype(ic)::value + 1]); });
        float top = m_top;
        auto tops = [&](bool one) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float scales[4] = {__uint_as_float(f[q][0]), __uint_as_float(f[q][1]), __uint_as_float(f[q][2]), __uint_as_float(f[q][3])};
                const f32x16_t& s = z.s[q >> 2];
                const int i = 4 * (q & 3);
                if (one) top = fmaxf(top, __builtin_fmaf(fmaxf(fmaxf(s[i], s[i + 1]), fmaxf(s[i + 2], s[i + 3])), a.scale_log2, log_scale(scales[0])));
                else top = fmaxf(top, top4(s[i], s[i + 1], s[i + 2], s[i + 3], scales, a.scale_log2));
            }
        };
        if (a.bshift >= 2) tops(true);        // four rows have one scale
        else tops(false);
        m_top = half_max(top);
        const bool move = moves(m_top, m_run, a.first), scaled = move && m_run != -INFINITY;   // (else there is nothing yet)
        const float next = m_top - a.first, half = move ? __builtin_amdgcn_exp2f(0.5f * (m_run - next)) : 1.0f, alpha = half * half;
        if (move) m_run = next;
        l_run = times_power(l_run, half);
        const float ref = m_run == -INFINITY ? 0.f : m_run;
        const uint32_t flags = (__ballot(scaled) ? 1u : 0u) | (__ballot(bad) ? 2u : 0u);
        const uint32_t pa = lds0 + B8_OFF_P + (k & 1) * B8_P + (32 * w + c) * (2 * C8_TILE);
        const uint32_t px = rope_xor(c);
        float psum = 0.f;
        static_for<0, 4>([&](auto ic) {        // 16 rows of the tile, eight of them this lane's
            constexpr int q = decltype(ic)::value, b = q >> 1;
            f16x8_t p8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(z.s[b][8 * (q & 1) + i], a.scale_log2, -ref));
                psum += p;
                p8[i] = (_Float16)(p * __uint_as_float(f[2 * q + (i >> 2)][i & 3]));
            }
            const u32x4_t v = __builtin_bit_cast(u32x4_t, p8);
            lds_write_u4(pa + 16 * ((2 * q + h) ^ px), v);
        });
        l_run += psum;   // this lane's share of the sum
        if (h == 0) lds_write_u1(lds0 + B8_OFF_ALPHA + 512 * (k & 1) + (32 * w + c) * 4, __float_as_uint(alpha));
        if (ln == 0) lds_write_u1(lds0 + B8_OFF_BAD + 16 * (k & 1) + 4 * w, flags);
    };
    auto stage = [&](int sg) { return lds0 + B8_OFF_STAGE + sg * C8_STAGE; };
    auto words = [&](int sg) { return lds0 + C8_OFF_WORD + (sg * C8_TILE + lane) * 4; };

    if (nt > 0) {
        if (nt > 1)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Loader64Lean::LOADS) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
        const float sc = fused8<true, false>(z, lds0, 0, 0, stage(0), words(0), w, lane);
        weights(0, C8_TILE * t0, sc);
    }
    int sg = 0;   // the stage of tile k
    // tile k + 1 has landed, every wave's share; the weights of tile k are there, and nobody reads tile k - 1 any more
    auto turn = [&](int k, auto more) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
        u32x4_t fl = lds_read_u4<B8_OFF_BAD>(lds0 + 16 * (k & 1));
        if (decltype(more)::value && k + 2 < nt) loader.issue(t0 + k + 2, smem, lds0, sg == 0 ? 2 : sg - 1, B8_OFF_STAGE);
        lds_wait<0>(fl);
        const uint32_t all = __builtin_amdgcn_readfirstlane((fl[0] | fl[1]) | (fl[2] | fl[3]));
        if (all & 1u) {
            int ln = lane;
            asm volatile("" : "+v"(ln));          // (as above: an address from memory would wait for the loads just issued)
#pragma unroll
            for (int rb = 0; rb < 4; ++rb) {      // a wave's rows are a row block
                if (!(__builtin_amdgcn_readfirstlane(fl[rb]) & 1u)) continue;
                uint32_t f = lds_read_u1(lds0 + B8_OFF_ALPHA + 512 * (k & 1) + (32 * rb + (ln & 31)) * 4);
                lds_wait<0>(f);
#pragma unroll
                for (int d = 0; d < 4; ++d) scale_all<16>(z.o[d][rb], __uint_as_float(f));
            }
        }
        if (all & 2u) clean_tile(stage(sg), w, lane);
        // after the waits for every LDS operation, which would be waits for these scalar loads too
        if (decltype(more)::value && k + 2 < nt) loader.fetch(t0 + k + 3);
    };
    for (int k = 0; k + 1 < nt; ++k) {
        turn(k, std::true_type{});
        const int next = sg == 2 ? 0 : sg + 1;
        const float sc = fused8<true, true>(z, lds0, stage(sg), lds0 + B8_OFF_P + (k & 1) * B8_P, stage(next), words(next), w, lane);
        weights(k + 1, C8_TILE * (t0 + k + 1), sc);
        sg = next;
    }
    if (nt > 0) {
        turn(nt - 1, std::false_type{});
        (void)fused8<false, true>(z, lds0, stage(sg), lds0 + B8_OFF_P + ((nt - 1) & 1) * B8_P, 0, 0, w, lane);
    }

    // ---- the rows' references and sums, for every wave
    __syncthreads();
    float* ml = reinterpret_cast<float*>(smem + B8_OFF_P);   // [row][2]
    const float l = half_sum(l_run);
    if (h == 0) {
        ml[2 * (32 * w + c)] = m_run;
        ml[2 * (32 * w + c) + 1] = l;
    }
    __syncthreads();
#pragma unroll
    for (int rb = 0; rb < 4; ++rb) {
        const int row = 32 * rb + c, R = x.row0 + row;
        finish_rows<4>(a, x.tok0 * a.H + R, R < x.nrow, row, rb, w, lane, ml[2 * row], ml[2 * row + 1], [&](int d) -> const f32x16_t& { return z.o[d][rb]; }, part_o, part_ml);
    }
}

// --------------------------------------------- a segment of a unit of 32 or 64 rows

// Eight waves, two a SIMD: four take scores and weights, 16 rows of the unit each (and no others, so that a reference is one wave's
// own), four the outputs, 128 dims each, of the tile before; so a SIMD's vector units convert and weigh for one while its
// matrix cores work for the other.  Tiles of 32 rows, seven in LDS: five on their way while two are used.
constexpr int M8_TILE = 32, M8_THREADS = 512, M8_STAGES = 7;
constexpr int M8_OFF_WORD = 0, M8_OFF_NOTE = M8_OFF_WORD + M8_STAGES * M8_TILE * 4;
constexpr int M8_OFF_SCALE = M8_OFF_NOTE + M8_STAGES * M8_TILE * 4;   // [32] the tile's scales (every wave writes the same ones)
constexpr int M8_OFF_ALPHA = M8_OFF_SCALE + 4 * M8_TILE;              // two of [64]: by what a row's outputs are to be multiplied
constexpr int M8_OFF_BAD = M8_OFF_ALPHA + 2 * 256;                    // two of [4]: the waves' flags, outputs to multiply, a hidden NaN
constexpr int M8_OFF_P = 3 * 1024, M8_P = 64 * 2 * M8_TILE;               // weights of a tile, [64][32] fp16; two of them
constexpr int M8_OFF_STAGE = M8_OFF_P + 2 * M8_P;
typedef Loader8<8, M8_OFF_WORD, M8_OFF_NOTE, true> Loader32;
constexpr int M8_SMEM = M8_OFF_STAGE + M8_STAGES * Loader32::STAGE;
static_assert(M8_OFF_BAD + 32 <= M8_OFF_P && M8_OFF_STAGE % 1024 == 0 && Loader32::TILE == M8_TILE, "");

// XOR of the 16-byte piece index within the 64 bytes of a row's weights: 16 rows' reads of a piece differ modulo 256 bytes
__device__ __forceinline__ int weight_xor(int r) { return (r >> 2) & 3; }

// The dims 128 w .. + 127 of a tile (at st), which this wave alone reads any more, without NaN codes (as clean_tile).
__device__ __attribute__((noinline)) void clean_dims(uint32_t st, int w, int lane) {
    for (int i = 0; i < M8_TILE; i += 8) {
        const int r = i + (lane >> 3);
        const uint32_t at = st + r * D_LAT + 16 * ((8 * w + (lane & 7)) ^ code_xor(r & 15));
        u32x4_t v = lds_read_u4<0>(at);
        lds_wait<0>(v);
        for (int q = 0; q < 4; ++q) v[q] = drop_nan(v[q]);
        lds_write_u4(at, v);
    }
}

// Scores and weights of a segment's tiles by the rows 16 w .. + 15 of unit x.
template <int RG>
__device__ __forceinline__ void mid_scores(const Chunk8Args& a, const CkUnit& x, int t0, int nt, uint32_t lds0, int w, int lane, float& m_run,
                                           float& l_run) {
    const int c = lane & 15, g = lane >> 4;
    if (w >= RG || x.row0 + 16 * w >= x.nrow) {                 // no rows: nothing to say
        if (lane < 2) lds_write_u1(lds0 + M8_OFF_BAD + 16 * lane + 4 * w, 0);
        for (int k = -1; k < nt; ++k) lds_barrier();
        return;
    }
    const int Rc = min(x.row0 + 16 * w + c, x.nrow - 1);        // rows past the end repeat the last one, never stored
    const int lim = min(x.old + Rc / a.H, x.kv - 1);            // the last cache row that this lane's row sees
    const int lim_lo = __builtin_amdgcn_readfirstlane(min(x.old + (x.row0 + 16 * w) / a.H, x.kv - 1));
    const int pg = 9 * (g & 1) ^ 16 * (g >> 1);                 // pieces of a key, as for fewer rows
    bf16x8_t qf[18];
    {
        const int64_t row = x.tok0 * a.H + Rc;
        const uint16_t* ql = a.q_lat + row * a.qls;
        const uint16_t* qr = a.q_rope + row * a.qrs + 8 * g;
#pragma unroll
        for (int s = 0; s < 16; ++s) qf[s] = *reinterpret_cast<const bf16x8_t*>(ql + 16 * ((s >> 1) ^ pg) + 8 * (s & 1));
#pragma unroll
        for (int s = 0; s < 2; ++s) qf[16 + s] = *reinterpret_cast<const bf16x8_t*>(qr + 32 * s);
    }
#pragma unroll
    for (int s = 0; s < 18; ++s) asm volatile("" : "+a"(qf[s]));   // no wait for them inside the tile loop

    float w_top = 0.f;   // this lane's largest weight since the reference moved
    int sg = 0;   // the stage of tile k
    for (int k = 0; k < nt; ++k) {
        lds_barrier();
        const int u0 = M8_TILE * (t0 + k);
        const uint32_t st = lds0 + M8_OFF_STAGE + sg * Loader32::STAGE;
        const uint32_t wn = lds0 + M8_OFF_WORD + (sg * M8_TILE + (lane & 31)) * 4;
        sg = sg == M8_STAGES - 1 ? 0 : sg + 1;

        // ---- scores of the 32 rows of the tile: s4[b][i] is row 16 b + 4 g + i
        uint32_t word = lds_read_u1(wn), note = lds_read_u1(wn + (M8_OFF_NOTE - M8_OFF_WORD));
        const uint32_t ka = st + c * D_LAT + ((16 * pg) ^ (16 * code_xor(c)));
        const uint32_t ra = st + Loader32::OFF_ROPE + c * (2 * D_ROPE) + 16 * (g ^ rope_xor(c));
        constexpr int SD = 3;          // operands read ahead of the matrix cores, of the tile's two row blocks: 8 of codes, 2 of the branch
        u32x4_t kc[SD + 1][2];
        auto kload = [&](auto sc_) {
            constexpr int s = decltype(sc_)::value;
            static_for<0, 2>([&](auto bc) {
                constexpr int b = decltype(bc)::value;
                if constexpr (s < 8) kc[s % (SD + 1)][b] = lds_read_u4<16 * D_LAT * b>(ka ^ (16 * s));
                else kc[s % (SD + 1)][b] = lds_read_u4<16 * 2 * D_ROPE * b>(ra ^ (64 * (s - 8)));
            });
        };
        static_for<0, SD>(kload);
        lds_wait<2 * SD>(word, note);
        const float sc = scale_of(word, note);                  // of tile row `lane` & 31
        const uint32_t absent = (uint32_t)__ballot(sc == 0.f);
        if (lane < M8_TILE) lds_write_u1(lds0 + M8_OFF_SCALE + 4 * lane, __float_as_uint(sc));
        float sk[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) sk[b] = __shfl(sc, 16 * b + c);
        f32x4_t s4[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) s4[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        static_for<0, 10>([&](auto sc_) {
            constexpr int s = decltype(sc_)::value;
            if constexpr (s + SD < 10) kload(std::integral_constant<int, s + SD>{});
            constexpr int N = 2 * ((s + SD < 10) ? SD : 9 - s);
            lds_wait<N>(kc[s % (SD + 1)][0], kc[s % (SD + 1)][1]);
#pragma unroll
            for (int i = 0; i < (s < 8 ? 2 : 1); ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const u32x4_t& v = kc[s % (SD + 1)][b];
                    if constexpr (s < 8)
                        s4[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8(v[2 * i], v[2 * i + 1], sk[b]), qf[2 * s + i], s4[b], 0, 0, 0);
                    else
                        s4[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v), qf[8 + s], s4[b], 0, 0, 0);
                }
        });

        // ---- weights, into buffer k & 1
        u32x4_t f[2];                 // the scales of this lane's scores
        static_for<0, 2>([&](auto bc) { f[decltype(bc)::value] = lds_read_u4<M8_OFF_SCALE + 64 * decltype(bc)::value>(lds0 + 16 * g); });
        bool bad = false;
        if (u0 + M8_TILE - 1 > lim_lo || absent != 0) {
            const int last = lim - u0 - 4 * g;
            const uint32_t gone = absent >> (4 * g);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (16 * b + i > last || ((gone >> (16 * b + i)) & 1u)) {
                        bad |= s4[b][i] != s4[b][i];
                        s4[b][i] = -INFINITY;
                    }
        }
        lds_wait<0>(f[0], f[1]);
        const int row = 16 * w + c;
        float psum, most;
        auto store = [&]() __attribute__((always_inline)) {
            const float ref = m_run == -INFINITY ? 0.f : m_run;
            psum = most = 0.f;
            static_for<0, 2>([&](auto bc) {
                constexpr int b = decltype(bc)::value;
                f16x4_t p4;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s4[b][i], a.scale_log2, -ref)), v = p * __uint_as_float(f[b][i]);
                    psum += p;
                    most = fmaxf(most, v);
                    p4[i] = (_Float16)v;
                }
                // slots of a row: in each 16 of them rows 4 h + (0..3, 8..11) for half h
                lds_write_u2(lds0 + M8_OFF_P + M8_P * (k & 1) + row * (2 * M8_TILE) + 16 * ((2 * b + (g & 1)) ^ weight_xor(row)) + 8 * (g >> 1),
                             __builtin_bit_cast(u32x2_t, p4));
            });
        };
        store();
        float alpha = 1.0f;
        bool scaled = false;
        if (__ballot(most > C8_MOST || m_run == -INFINITY)) {
            float top = m_run == -INFINITY ? -INFINITY : m_run + __builtin_amdgcn_logf(w_top);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const float scales[4] = {__uint_as_float(f[b][0]), __uint_as_float(f[b][1]), __uint_as_float(f[b][2]), __uint_as_float(f[b][3])};
                top = fmaxf(top, top4(s4[b][0], s4[b][1], s4[b][2], s4[b][3], scales, a.scale_log2));
            }
            top = allreduce_groups(top, [](float p, float q) { return fmaxf(p, q); });
            const bool move = moves(top, m_run, a.first);
            const float next = top - a.first, half = move ? __builtin_amdgcn_exp2f(0.5f * (m_run - next)) : 1.0f;
            alpha = half * half;
            scaled = move && m_run != -INFINITY;           // (else there is nothing yet)
            l_run = times_power(l_run, half);
            if (move) m_run = next, w_top = __builtin_amdgcn_exp2f(a.first);
            store();
        }
        w_top = fmaxf(w_top, most);
        l_run += psum;                // this lane's share of the sum
        const uint32_t flags = (__ballot(scaled) ? 1u : 0u) | (__ballot(bad) ? 2u : 0u);
        if (g == 0) lds_write_u1(lds0 + M8_OFF_ALPHA + 256 * (k & 1) + row * 4, __float_as_uint(alpha));
        if (lane == 0) lds_write_u1(lds0 + M8_OFF_BAD + 16 * (k & 1) + 4 * w, flags);
    }
    lds_barrier();
}

// Loads of a segment's tiles, and the outputs' dims 128 w .. + 127 of all the unit's rows.
template <int RB>
__device__ __forceinline__ void mid_outputs(const Chunk8Args& a, const CkUnit& x, int t0, int nt, uint8_t* smem, uint32_t lds0, int w, int lane,
                                            f32x16_t (&o)[4][RB]) {
    Loader32 loader{a, (const_i32_t*)(a.table + (int64_t)x.b * a.tstride), x.kv, w, lane, {}, {}};
    loader.prepare();
    constexpr int FIRST = M8_STAGES - 2;
    {
        Loader32 first[FIRST] = {loader, loader, loader, loader, loader};
        static_assert(FIRST == 5, "");
#pragma unroll
        for (int i = 0; i < FIRST; ++i)
            if (i < nt) first[i].fetch(t0 + i);
        loader.fetch(t0 + FIRST);
#pragma unroll
        for (int i = 0; i < FIRST; ++i)
            if (i < nt) first[i].issue(t0 + i, smem, lds0, i, M8_OFF_STAGE);
    }
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][r][i] = 0.f;

    // tile k + 1 has landed; the weights of tile k are there, and nobody reads tile k - 1 any more: tile k + 6 goes into its place
    auto turn = [&](int k, int sg) __attribute__((always_inline)) {
        if (k + 5 < nt)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * Loader32::LOADS) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
        if (k + 6 < nt) loader.issue(t0 + k + 6, smem, lds0, sg, M8_OFF_STAGE);
    };
    turn(-1, FIRST);
    if (FIRST + 1 < nt) loader.fetch(t0 + FIRST + 1);
    int sg = 0;   // the stage of tile k
    for (int k = 0; k < nt; ++k) {
        turn(k, sg == 0 ? M8_STAGES - 1 : sg - 1);
        const uint32_t st = lds0 + M8_OFF_STAGE + sg * Loader32::STAGE;
        sg = sg == M8_STAGES - 1 ? 0 : sg + 1;
        const int r = lane & 31, hh = lane >> 5;
        const uint32_t pr = lds0 + M8_OFF_P + M8_P * (k & 1) + r * (2 * M8_TILE) + 16 * (hh ^ weight_xor(r));
        u32x4_t fl = lds_read_u4<M8_OFF_BAD>(lds0 + 16 * (k & 1));
        u32x4_t pf[2][RB];
        static_for<0, 2>([&](auto sc_) {
            static_for<0, RB>([&](auto rc) {
                constexpr int s = decltype(sc_)::value, rb = decltype(rc)::value;
                pf[s][rb] = lds_read_u4<rb * 32 * 2 * M8_TILE>(pr ^ (32 * s));
            });
        });
        lds_wait<2 * RB>(fl);
        const uint32_t all = __builtin_amdgcn_readfirstlane((fl[0] | fl[1]) | (fl[2] | fl[3]));
        if (all & 1u) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                uint32_t al = lds_read_u1(lds0 + M8_OFF_ALPHA + 256 * (k & 1) + (32 * rb + r) * 4);
                lds_wait<0>(al);
#pragma unroll
                for (int d = 0; d < 4; ++d) scale_all<16>(o[d][rb], __uint_as_float(al));
            }
        }
        if (all & 2u) {
            static_for<0, 2 * RB>([&](auto q) { lds_wait<0>(pf[decltype(q)::value / RB][decltype(q)::value % RB]); });   // (as above)
            clean_dims(st, w, lane);
        }
        const int e = (lane >> 1) & 7, vr = 4 * hh + (e & 3) + 8 * (e >> 2);   // a lane group's eight rows of 16, its place among the dims
        const uint32_t va = st + vr * D_LAT + 16 * ((8 * w + ((lane >> 4) & 1)) ^ code_xor(vr)) + 8 * (lane & 1);
        constexpr int N = 8, VD = 5;
        u32x2_t vv[VD + 1];
        auto vload = [&](auto ic) {
            constexpr int i = decltype(ic)::value;
            vv[i % (VD + 1)] = lds_read_tr8<16 * D_LAT * (i >> 2)>(va ^ (32 * (i & 3)));
        };
        static_for<0, VD>(vload);
        static_for<0, N>([&](auto ic) {
            constexpr int i = decltype(ic)::value, s = i >> 2, d = i & 3;
            if constexpr (i + VD < N) vload(std::integral_constant<int, i + VD>{});
            if constexpr (i == 0) static_for<0, 2 * RB>([&](auto q) { lds_wait<VD + 1>(pf[decltype(q)::value / RB][decltype(q)::value % RB]); });
            lds_wait<(i + VD < N) ? VD : N - 1 - i>(vv[i % (VD + 1)]);
            const f16x8_t v = value8(vv[i % (VD + 1)][0], vv[i % (VD + 1)][1]);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
                o[d][rb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, __builtin_bit_cast(f16x8_t, pf[s][rb]), o[d][rb], 0, 0, 0);
        });
        // after the waits for every LDS operation, which would be waits for these scalar loads too
        if (k + 7 < nt) loader.fetch(t0 + k + 7);
    }
}

template <int RG>
__device__ __forceinline__ void chunk8_mid_segment(const Chunk8Args& a, const CkUnit& x, int t0, int t1, float* part_o,
                                                   float* part_ml, uint8_t* smem) {
    constexpr int RB = RG / 2;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));   // keeps the lane arithmetic of the loops out of registers across the units
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave & 3;
    const uint32_t lds0 = lds_addr(smem);
    const int nt = x.kv > 0 ? t1 - t0 : 0;
    float* ml = reinterpret_cast<float*>(smem + M8_OFF_P);   // [row][2]
    if (wave < 4) {
        float m_run = -INFINITY, l_run = 0.f;
        if (nt > 0) mid_scores<RG>(a, x, t0, nt, lds0, w, lane, m_run, l_run);
        // ---- the rows' references and sums, for every wave
        __syncthreads();
        const float l = allreduce_groups(l_run, [](float p, float q) { return p + q; });
        if (w < RG && lane < 16) {
            ml[2 * (16 * w + lane)] = m_run;
            ml[2 * (16 * w + lane) + 1] = l;
        }
        __syncthreads();
        return;
    }
    f32x16_t o[4][RB];   // [dim block][row block]
    if (nt > 0) {
        mid_outputs<RB>(a, x, t0, nt, smem, lds0, w, lane, o);
    } else {
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][r][i] = 0.f;
    }
    __syncthreads();
    __syncthreads();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = 32 * rb + (lane & 31), R = x.row0 + row;
        finish_rows<RB>(a, x.tok0 * a.H + R, R < x.nrow, row, rb, w, lane, ml[2 * row], ml[2 * row + 1], [&](int d) -> const f32x16_t& { return o[d][rb]; }, part_o, part_ml);
    }
}

// how a unit of 16 RG rows is worked on
template <int RG>
struct Shape8 {
    static constexpr int TILE = RG == 2 || RG == 4 ? M8_TILE : C8_TILE, THREADS = RG == 2 || RG == 4 ? M8_THREADS : C8_THREADS;
    static constexpr int SMEM = RG == 8 ? B8_SMEM : RG == 1 ? C8_SMEM : M8_SMEM;
};

template <int RG>
__device__ __forceinline__ void segment8(const Chunk8Args& a, const CkUnit& x, int t0, int t1, float* part_o, float* part_ml,
                                         uint8_t* smem) {
    if constexpr (RG == 8) chunk8_big_segment(a, x, t0, t1, part_o, part_ml, smem);
    else if constexpr (RG > 1) chunk8_mid_segment<RG>(a, x, t0, t1, part_o, part_ml, smem);
    else chunk8_segment(a, x, t0, t1, part_o, part_ml, smem);
}

// ------------------------------------------------------------------- kernels

// Runs the tiles of all units are cut into: at most one per CU, and as a run costs its tiles and the writing and reading of its
// part, some sqrt(tiles) of them, more where parts are small beside a tile's time.  16 heads over 4 x 8192 rows 20.6 us, 25.0 with
// half as many runs; 32 heads over 4 x 8192 rows 25.4 us, 27.3 with fewer; 128 heads over 32768 rows in units of 128 rows 49.1 us,
// 55.0 with twice as many.
template <int RG>
__device__ __forceinline__ int run_count8(const Chunk8Args& a, int total) {
    int len = 1;
    while (2.0f * (float)len <= (RG == 1 ? 0.12f : 0.25f) * sqrtf((float)total)) len *= 2;
    return min(max((total + len - 1) / len, 1), a.runs);
}

// What scan_units finds, for up to 64 units: each wave for itself, a lane a unit.  What is read of the units goes to LDS as well, behind
// the 64 first tiles, so that nobody waits for it again.
constexpr int UNIT_WORDS = 4;
template <int TILE>
__device__ __forceinline__ int scan_few(const Chunk8Args& a, int rows, int* pre) {
    const int lane = threadIdx.x & 63, U = a.B * a.mb;
    int n = 0;
    if (lane < U) {
        const CkUnit x = chunk_unit(a, lane, rows);
        n = unit_tiles<TILE>(a, x, rows);
        int* at = pre + 64 + UNIT_WORDS * lane;
        at[0] = x.nrow;
        at[1] = (int)x.tok0;      // (n_tok is below 2^31)
        at[2] = x.kv;
        at[3] = x.old;
    }
    int upto = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int t = __shfl_up(upto, d);
        if (lane >= d) upto += t;
    }
    pre[lane] = upto - n;
    return __builtin_amdgcn_readlane(upto, 63);
}
__device__ __forceinline__ CkUnit few_unit(const Chunk8Args& a, int u, int rows, const int* pre) {
    const int* at = pre + 64 + UNIT_WORDS * u;
    CkUnit x{};   // (nq, which gives nrow, is not asked for again)
    x.b = u / a.mb;
    x.row0 = (u - x.b * a.mb) * rows;
    x.nrow = __builtin_amdgcn_readfirstlane(at[0]);
    x.tok0 = __builtin_amdgcn_readfirstlane(at[1]);
    x.kv = __builtin_amdgcn_readfirstlane(at[2]);
    x.old = __builtin_amdgcn_readfirstlane(at[3]);
    return x;
}

template <int RG>
__global__ __launch_bounds__(Shape8<RG>::THREADS, 1) void chunk8_run_kernel(Chunk8Args a) {
    constexpr int ROWS = 16 * RG, TILE = Shape8<RG>::TILE, THREADS = Shape8<RG>::THREADS;
    __shared__ __align__(1024) uint8_t smem[Shape8<RG>::SMEM];
    __shared__ int pre[CK_MAX_UNITS];
    static_assert(64 * (1 + UNIT_WORDS) <= CK_MAX_UNITS, "");
    const int U = a.B * a.mb;
    const bool few = U <= 64;
    const int total = few ? scan_few<TILE>(a, ROWS, pre) : scan_units<TILE, THREADS>(a, ROWS, pre);
    const int n = run_count8<RG>(a, total), g = blockIdx.x;
    if (g == 0)   // units without rows: nothing to join
        for (int u = threadIdx.x; u < U; u += THREADS)
            if ((u + 1 < U ? pre[u + 1] : total) == pre[u]) a.span[3 * u] = a.span[3 * u + 1] = 0;
    if (g >= n) return;
    const int beg = run_start(g, n, total), end = run_start(g + 1, n, total);
    int u = 0;   // the last unit that starts at or before beg
    if (few) {
        const int lane = threadIdx.x & 63;
        u = __popcll(__ballot(lane < U && pre[lane] <= beg)) - 1;
    } else {
        for (int step = CK_MAX_UNITS / 2; step > 0; step /= 2)
            if (u + step < U && pre[u + step] <= beg) u += step;
    }
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
        const CkUnit x = few ? few_unit(a, u, ROWS, pre) : chunk_unit(a, u, ROWS);
        const int t0 = at - base, t1 = min(end, next) - base;
        const bool whole = t0 == 0 && t1 == next - base;
        if (threadIdx.x == 0) {   // for the join: the unit's first and last run, and which of its slots the first one fills
            if (t0 == 0) a.span[3 * u] = g, a.span[3 * u + 2] = at > beg;
            if (t1 == next - base) a.span[3 * u + 1] = g;
        }
        const int64_t slot = 2 * g + (at > beg ? 1 : 0);
        segment8<RG>(a, x, t0, t1, whole ? nullptr : a.part_o + slot * (ROWS * D_LAT), a.part_ml + slot * (ROWS * 2), smem);
        __syncthreads();   // the stages are free
        at = base + t1;
        ++u;
    }
}

template <int RG>
__global__ __launch_bounds__(Shape8<RG>::THREADS, 1) void chunk8_unit_kernel(Chunk8Args a) {
    __shared__ __align__(1024) uint8_t smem[Shape8<RG>::SMEM];
    const uint32_t wg = workgroup_id();
    if (wg >= (uint32_t)a.B * (uint32_t)a.mb) return;
    const int b = (int)(wg / (uint32_t)a.mb), j = a.mb - 1 - (int)(wg % (uint32_t)a.mb);   // the later rows (more tiles) first
    const CkUnit x = chunk_unit(a, b * a.mb + j, 16 * RG);
    const int n = unit_tiles<Shape8<RG>::TILE>(a, x, 16 * RG);
    if (n == 0) return;
    segment8<RG>(a, x, 0, n, nullptr, nullptr, smem);
}

// x += y of reference m: references 2^128 apart still add up right, as a sum may be 2^64 times what its reference stands for
__device__ __forceinline__ void join8_add(JoinSum& x, float m, float l, const f32x4_t& v) {
    if (m > x.M) {
        const float half = x.M == -INFINITY ? 1.0f : exp2f(0.5f * (x.M - m));
        x.L = times_power(x.L, half);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.acc[i] *= half * half;
        x.M = m;
    }
    const float half = m == -INFINITY ? 1.0f : exp2f(0.5f * (m - x.M));
    x.L += times_power(l, half);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.acc[i] += half * half * v[i];
}

// Joins the parts of a unit that several runs cover: block = (unit, F float4 of a part, in the order the segments leave them),
// thread = one of them in every GROUPS-th part; then the groups join through LDS, in order.  Few rows: more groups, as a
// part is small and the loads' latency what counts.
constexpr int C8J_THREADS = 512;

template <int RG, int F>
__global__ __launch_bounds__(C8J_THREADS) void chunk8_join_kernel(Chunk8Args a) {
    constexpr int GROUPS = C8J_THREADS / F, BATCH = F == 32 ? 8 : 4, rows = 16 * RG, per = rows * (D_LAT / 4) / F;
    __shared__ JoinSum sums[GROUPS - 1][F];
    const int u = blockIdx.x / per, grp = threadIdx.x / F;
    const int f = (blockIdx.x % per) * F + threadIdx.x % F, lane = f & 63;
    int r, d;   // row of the unit, first dim
    if constexpr (RG == 1) {
        r = lane & 15;
        d = 16 * (f >> 6) + 4 * (lane >> 4);
    } else {
        constexpr int rb = RG / 2;
        const int q = (f >> 6) & 3, blk = f >> 8;
        r = 32 * (blk % rb) + (lane & 31);
        d = 32 * (blk / rb) + 8 * q + 4 * (lane >> 5);
    }
    const int g0 = a.span[3 * u], g1 = a.span[3 * u + 1], late = a.span[3 * u + 2];
    const CkUnit x = chunk_unit(a, u, rows);
    if (g0 == g1) return;
    const int R = x.row0 + r;
    const bool live = R < x.nrow;
    JoinSum t{-INFINITY, 0.f, f32x4_t{0.f, 0.f, 0.f, 0.f}};
    if (live)
        for (int s0 = g0 + grp; s0 <= g1; s0 += GROUPS * BATCH) {
            float m[BATCH], l[BATCH];
            f32x4_t v[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {   // all loads in flight
                const int run = min(s0 + GROUPS * j, g1);
                const int64_t slot = 2 * run + (run == g0 ? late : 0);
                const float* ml = a.part_ml + slot * (rows * 2) + 2 * r;
                m[j] = ml[0];
                l[j] = ml[1];
                v[j] = *reinterpret_cast<const f32x4_t*>(a.part_o + slot * (rows * D_LAT) + 4 * f);
            }
#pragma unroll
            for (int j = 0; j < BATCH; ++j)
                if (s0 + GROUPS * j <= g1) join8_add(t, m[j], l[j], v[j]);
        }
    if (grp > 0) sums[grp - 1][threadIdx.x % F] = t;
    __syncthreads();
    if (grp > 0 || !live) return;
#pragma unroll
    for (int i = 0; i < GROUPS - 1; ++i) {
        const JoinSum y = sums[i][threadIdx.x];
        join8_add(t, y.M, y.L, y.acc);
    }
    const int64_t row = x.tok0 * a.H + R;
    const bool none = t.M == -INFINITY && t.L == 0.f;
    const float inv = none ? 0.f : 1.0f / t.L;
    const bf16x4_t v4 = {(__bf16)(t.acc[0] * inv), (__bf16)(t.acc[1] * inv), (__bf16)(t.acc[2] * inv), (__bf16)(t.acc[3] * inv)};
    *reinterpret_cast<bf16x4_t*>(a.out + row * D_LAT + d) = v4;
    if (d == 0) a.lse[row] = lse_of(t.M, t.L);
}

ChunkSplit chunk8_split(int64_t B, int64_t H, int64_t max_q, int64_t max_kv) {
    ChunkSplit s{};
    const int64_t rows = max_q * H;
    // Rows of a unit.  Many rows: each code is converted once for all of them.  Fewer rows: more units where the cache alone does not
    // give every CU some tiles to work through, a start and a part that take less time, and the cache is read again from
    // nearby.  128 heads, a token each, units of 32, 64 and 128 rows: one sequence of 8192 rows 26, 30, 44 us, of 131072 rows 85,
    // 66, 81 us; 16 of 32768 rows 262, 204, 187 us.  64 heads, units of 32 and 64 rows: 30 and 33 us, 52 and 49 us, 145 and 113 us.
    const int64_t cache = B * std::max<int64_t>(1, (max_kv + C8_TILE - 1) / C8_TILE);   // tiles
    const int64_t of32 = (rows + 31) / 32 * cache, of64 = (rows + 63) / 64 * cache;
    s.qg = rows <= 16 ? 1 : rows <= 32 || of32 <= 2048 ? 2 : rows <= 64 || of64 <= 8192 ? 4 : 8;
    s.mb = (rows + 16 * s.qg - 1) / (16 * s.qg);
    s.units = B * s.mb;
    const int64_t tiles = s.mb * cache;
    s.runs = s.units <= CK_MAX_UNITS && tiles < (1ll << 30) ? CK_RUNS : 0;   // (tiles of 32 rows are twice as many)
    s.streams = 1;
    if (s.runs) {
        s.runs = std::max<int64_t>(1, std::min<int64_t>(s.runs, tiles));
        s.part_o = (size_t)(2 * s.runs) * 16 * s.qg * D_LAT * 4;
        s.part_ml = (size_t)(2 * s.runs) * 16 * s.qg * 2 * 4;
        s.span = (size_t)s.units * 3 * 4;
    }
    return s;
}

template <int RG>
static hipError_t launch_chunk8_rows(const Chunk8Args& a, const ChunkSplit& sp, hipStream_t s) {
    if (!sp.runs) {
        hipLaunchKernelGGL((chunk8_unit_kernel<RG>), grid_of(sp.units), dim3(Shape8<RG>::THREADS), 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((chunk8_run_kernel<RG>), dim3((unsigned)sp.runs), dim3(Shape8<RG>::THREADS), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || sp.runs == 1) return e;
    // a part in many pieces where few units share the chip (many parts of each), fewer pieces where there are units enough
    const int F = sp.units * RG <= 16 ? 32 : 128;
    const dim3 grid((unsigned)(sp.units * 16 * RG * (D_LAT / 4) / F));
    if (F == 32) hipLaunchKernelGGL((chunk8_join_kernel<RG, 32>), grid, dim3(C8J_THREADS), 0, s, a);
    else hipLaunchKernelGGL((chunk8_join_kernel<RG, 128>), grid, dim3(C8J_THREADS), 0, s, a);
    return hipGetLastError();
}

// log2 of the largest weight where a reference moves, by the rows that a segment may have (run_count8's lengths, a tile's rest)
static int first_weight(const ChunkSplit& sp, int64_t max_kv) {
    const int64_t tile = sp.qg == 2 || sp.qg == 4 ? M8_TILE : C8_TILE, cache = (max_kv + tile - 1) / tile, total = sp.units * cache;
    int64_t rows = max_kv;
    if (sp.runs) rows = std::min(rows, tile * (1 + std::max(1 + total / sp.runs, (int64_t)(0.25 * std::sqrt((double)total)))));
    int log = 0;
    while (log < 30 && (1ll << log) < rows) ++log;
    return std::min(std::max(log - 14, 0), 14);
}

hipError_t launch_chunk8(Chunk8Args a, const ChunkSplit& sp, hipStream_t s) {
    a.first = (float)first_weight(sp, a.max_kv);
    return sp.qg == 1 ? launch_chunk8_rows<1>(a, sp, s) : sp.qg == 2 ? launch_chunk8_rows<2>(a, sp, s)
         : sp.qg == 4 ? launch_chunk8_rows<4>(a, sp, s) : launch_chunk8_rows<8>(a, sp, s);
}

}  // namespace vkv
