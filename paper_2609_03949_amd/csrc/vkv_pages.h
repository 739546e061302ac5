// vkv_pages.h -- tiles of a paged latent cache in LDS (gfx950): their layout, and the
// direct loads that fill them, with scalar table entries and row addresses.
#pragma once

#include "vkv_tile.h"

namespace vkv {

constexpr int CK_TILE = 32;                              // cache rows of a tile
constexpr int CK_LAT_BYTES = 2 * D_LAT, CK_ROPE_BYTES = 2 * D_ROPE;
constexpr int CK_OFF_ROPE = CK_TILE * CK_LAT_BYTES;
constexpr int CK_STAGE = CK_TILE * 2 * D_ROW;            // 36 KB

// XOR of the piece index of tile row r.  LDS serves a 128-bit read sixteen lanes at a
// time, lanes {0-3, 12-15, 20-23, 24-27} and {4-11, 16-19, 28-31} of each half wave, and a
// 64-bit one a half wave at a time; each such group has to touch 16 pieces that differ
// modulo 16 (64 banks).  Latent panel (rows 1 KB apart, so the XOR alone decides): the
// transposing V reads of a half wave take rows 4 a .. 4 a + 3 of four adjacent pieces
// (32x32 products), or of two pieces and the next four rows (16x16): the row within
// the four chooses a block of four pieces, the four's number y(b) the place in it, with
// y = 0, 2, 3, 1, which also keeps the K reads apart (a group has all of r mod 16 in
// 32x32 products; b = 0, 3 of one piece and b = 1, 2 of its neighbour, or the reverse, in
// 16x16 ones).  Branch panel (128 bytes a row: odd rows in the other half of the
// banks): r / 2 mod 8.
__device__ __forceinline__ int lat_xor(int r) {
    const int b = r >> 2;
    return ((r & 3) << 2) | (((b ^ (b >> 1)) & 1) << 1) | ((b >> 1) & 1);
}
__device__ __forceinline__ int rope_xor(int r) { return (r >> 1) & 7; }

// The cache rows before those of a sequence's new tokens: token i sees the rows up to rows_before + i.  (Below -max_q no
// token that is computed sees a row, and no row is older than the tokens: cut there, within 32 bits.)
__device__ __forceinline__ int rows_before(int kv, int64_t tokens, int max_q) {
    return (int)(kv - min(tokens, (int64_t)kv + max_q));
}

typedef __attribute__((address_space(4))) const int32_t const_i32_t;

// One wave's share of the tiles of a stream of WPT waves: NR rows of each.
template <int WPT>
struct TileLoader {
    static constexpr int NR = CK_TILE / WPT;
    static constexpr int LOADS = NR + (NR + 7) / 8;
    const ChunkArgs& a;
    const_i32_t* table;
    int kv, wt, lane;       // rows of the sequence, wave of the stream, lane
    int32_t e[NR];          // the fetched tile's table entries (scalar)

    __device__ __forceinline__ int row(int t, int i) const { return min(CK_TILE * t + NR * wt + i, kv - 1); }
    // rows past the end: the last row's
    __device__ __forceinline__ void fetch(int t) {
        e[0] = table[row(t, 0) >> a.shift];
        if (a.page_mask < NR - 1)
#pragma unroll
            for (int i = 1; i < NR; ++i) e[i] = table[row(t, i) >> a.shift];
    }
    // the loads of the fetched tile t into stage st; gone: where its rows that do not exist are noted
    __device__ __forceinline__ void issue(int t, uint8_t* st, uint32_t gone) const {
        const char* base[NR];
        uint32_t none = 0;
        // on a page that does not exist: the first rows of the cache in place of its own, masked later
        const bool whole = a.page_mask >= NR - 1;   // the rows lie on one page
        if (whole) {
            const int u = row(t, 0), last = min(kv - 1 - u, NR - 1);
            const bool there = (uint32_t)e[0] < (uint32_t)a.n_pages;
            const uint64_t at = (uint64_t)(uint32_t)(there ? e[0] : 0) * a.ps16 + (uint64_t)(uint32_t)(there ? u & a.page_mask : 0) * a.rs16;
            base[0] = reinterpret_cast<const char*>(a.cache) + 16 * at;
#pragma unroll
            for (int i = 1; i < NR; ++i) base[i] = base[i - 1] + (i <= last ? 16 * (uint64_t)a.rs16 : 0);
            none = there ? 0u : (1u << NR) - 1u;
        } else {
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const bool there = (uint32_t)e[i] < (uint32_t)a.n_pages;
                const uint64_t at = (uint64_t)(uint32_t)(there ? e[i] : 0) * a.ps16 +
                                    (uint64_t)(uint32_t)(there ? row(t, i) & a.page_mask : 0) * a.rs16;
                base[i] = reinterpret_cast<const char*>(a.cache) + 16 * at;
                none |= there ? 0u : 1u << i;
            }
        }
        int ln = lane;
        asm volatile("" : "+v"(ln));   // keeps the lane arithmetic out of registers across the loop
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int r = NR * wt + i;
            const uint32_t off = (uint32_t)(16 * ln) ^ (uint32_t)(16 * lat_xor(r));
            __builtin_amdgcn_global_load_lds((gbl_void_t*)(base[i] + off), (lds_void_t*)(st + CK_LAT_BYTES * r), 16, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < NR; j += 8) {      // eight rows, eight lanes each
            const char* b = base[j];
#pragma unroll
            for (int i = 1; i < (NR < 8 ? NR : 8); ++i) b = (ln >> 3) == i ? base[j + i] : b;
            const int r = NR * wt + j + (ln >> 3);
            if (NR >= 8 || ln < 8 * NR)
                __builtin_amdgcn_global_load_lds((gbl_void_t*)(b + CK_LAT_BYTES + 16 * ((ln & 7) ^ rope_xor(r))),
                                                 (lds_void_t*)(st + CK_OFF_ROPE + CK_ROPE_BYTES * (NR * wt + j)), 16, 0, 0);
        }
        asm volatile("ds_write_b32 %0, %1" ::"v"(gone + 4 * wt), "v"(none) : "memory");
    }
    // where this lane reads the notes of a tile, and the mask they make (bit r: tile row r does not exist)
    __device__ __forceinline__ static uint32_t note(uint32_t gone, int ln) { return gone + 4 * (ln % WPT); }
    __device__ __forceinline__ static uint32_t absent(uint32_t w) {
        uint32_t all = 0;
        if (__ballot(w != 0))
#pragma unroll
            for (int i = 0; i < WPT; ++i) all |= (uint32_t)__builtin_amdgcn_readlane(w, i) << (NR * i);
        return all;
    }
};

}  // namespace vkv
