// k_write8.hip -- new rows into a paged latent cache held in 8 bits (gfx950).
//
//   s = max(the block's scale byte if it holds rows before the new ones, least s with amax <= 448 * 2^(s - 127)),
//   code = RNE_e4m3(x 2^(127 - s)),  older codes of a block whose s grows: RNE_e4m3(code 2^(old - s))
//
// A block of R rows of one page is one workgroup's (R >= 4: each of its four waves takes every fourth row) or one
// wave's.  A wave reads a row's 512 bf16 in one 16-byte load a lane and keeps what it read in registers
// until the block's largest magnitude is known, so every input is read once; a bf16's magnitude is compared as
// the integer of its bits, and the scale comes from that integer's exponent.  Bound: HBM (1152 + 640 bytes a row): 28600
// rows in blocks of 16, 12.1 us, 4.2 TB/s; one row of each of 32 sequences 4.2 us, the launch and three loads one after another.
#include <algorithm>

#include "vkv_pages.h"

namespace vkv {

constexpr int W8_WAVES = 4, W8_THREADS = 64 * W8_WAVES;
constexpr uint32_t W8_TOP = 0x63E0;   // bits of 448 * 2^64: larger ones, infinities and NaN are stored as NaN

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int scale_byte(uint32_t top) {   // of the bits of a bf16 magnitude
    const int s = (int)(top >> 7) - 8 + ((top & 0x7Fu) > 0x60u ? 1 : 0);
    return min(max(s, VKV_SCALE_MIN), VKV_SCALE_MAX);
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }   // 2^e, -126 <= e <= 127
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) {
    uint32_t v = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, (int)v, true);
}

template <int R>
__global__ __launch_bounds__(W8_THREADS) void write8_kernel(Write8Args a) {
    constexpr int GW = R >= 4 ? W8_WAVES : 1;    // waves of a block
    constexpr int NR = R / GW;                   // rows of a wave
    __shared__ uint32_t tops[W8_WAVES];
    const Chunk8Args& c = a.c;
    const uint32_t wg = workgroup_id();
    if (wg >= (uint32_t)c.B * (uint32_t)a.mb) return;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = (int)(wg / (uint32_t)a.mb), j = (int)(wg % (uint32_t)a.mb);
    const int64_t s0 = min(max((int64_t)c.cu[b], (int64_t)0), c.n_tok);
    const int64_t e0 = min(max((int64_t)c.cu[b + 1], s0), c.n_tok);
    // A sequence longer than its table keeps its rows' places (cut to max_kv, as where it is read, the length would put new rows
    // over older ones).  No sequence has 2^30 rows and more: such a length stands for max_kv.
    const int n = c.kv_len[b], kv = n >= (1 << 30) ? c.max_kv : max(n, 0);
    const int64_t before = kv - (e0 - s0);                             // the row of token s0
    const int first = (int)max(before, (int64_t)0), end = (int)min(before + min(e0 - s0, (int64_t)c.max_q), (int64_t)c.max_kv);   // rows that are written
    // the block's first row (another sequence may have 2^30 rows to write, so that this passes 31 bits, not 32)
    const uint32_t at0 = (uint32_t)(first / R + (GW == 1 ? W8_WAVES * j + w : j)) * R;
    if (first >= end || at0 >= (uint32_t)end) return;                  // the whole workgroup, or waves that share nothing
    const int u0 = (int)at0;
    const int32_t p = c.table[(int64_t)b * c.tstride + (u0 >> c.shift)];
    if ((uint32_t)p >= (uint32_t)c.n_pages) return;
    const int r0 = u0 & c.page_mask;
    uint8_t* page = a.cache + 16 * ((uint64_t)(uint32_t)p * c.ps16 + (uint64_t)(uint32_t)r0 * c.rs16);
    uint8_t* sb = a.scale + (uint64_t)(uint32_t)p * (uint64_t)c.sstride + (r0 >> c.bshift);
    const int was = u0 < first ? min(max((int)*sb, VKV_SCALE_MIN), VKV_SCALE_MAX) : VKV_SCALE_MIN;

    u32x4_t x[NR];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int u = u0 + w % GW + GW * i;
        x[i] = u32x4_t{0, 0, 0, 0};
        if (u >= first && u < end) x[i] = *reinterpret_cast<const u32x4_t*>(a.lat + (s0 + u - before) * a.ls + 8 * lane);
    }
#pragma unroll
    for (int i = 0; i < NR; i += 8) {            // the branch: eight rows, eight lanes each
        const int k = i + (lane >> 3), u = u0 + w % GW + GW * k;
        if (k < NR && u >= first && u < end)
            *reinterpret_cast<u32x4_t*>(page + (uint64_t)(u - u0) * 16 * c.rs16 + D_LAT + 16 * (lane & 7)) =
                *reinterpret_cast<const u32x4_t*>(a.rope + (s0 + u - before) * a.rs + 8 * (lane & 7));
    }
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t m = (x[i][q] >> (16 * h)) & 0x7FFFu;
                top = max(top, m <= W8_TOP ? m : 0u);
            }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if constexpr (GW > 1) {
        if (lane == 0) tops[w] = top;
        __syncthreads();   // every wave has read the block's scale, too
#pragma unroll
        for (int i = 0; i < W8_WAVES; ++i) top = max(top, tops[i]);
    }
    const int s = max(scale_byte(top), was);
    const float f = power(127 - s);
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int u = u0 + w % GW + GW * i;
        if (u < first || u >= end) continue;
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const uint32_t bits = (x[i][q >> 1] >> (16 * (q & 1))) & 0xFFFFu;
            v[q] = (bits & 0x7FFFu) <= W8_TOP ? __uint_as_float(bits << 16) * f : __uint_as_float(0x7FC00000u);
        }
        *reinterpret_cast<u32x2_t*>(page + (uint64_t)(u - u0) * 16 * c.rs16 + 8 * lane) =
            u32x2_t{code4(v[0], v[1], v[2], v[3]), code4(v[4], v[5], v[6], v[7])};
    }
    if (u0 < first && s > was) {                 // rows that were there before
        const float g = power(max(was - s, -126));   // (from 2^-20 on every code becomes 0)
        for (int i = 0; i < NR; ++i) {
            const int u = u0 + w % GW + GW * i;
            if (u >= first) break;
            u32x2_t* at = reinterpret_cast<u32x2_t*>(page + (uint64_t)(u - u0) * 16 * c.rs16 + 8 * lane);
            u32x2_t v = *at;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(v[q], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(v[q], true);
                v[q] = code4(lo[0] * g, lo[1] * g, hi[0] * g, hi[1] * g);
            }
            *at = v;
        }
    }
    if (lane == 0 && w % GW == 0) *sb = (uint8_t)s;
}

// blocks that up to q rows lie in, wherever they begin, by the workgroup
int64_t write8_blocks(int64_t q, int64_t block) {
    const int64_t n = (q + 2 * block - 2) / block;
    return block >= 4 ? n : (n + W8_WAVES - 1) / W8_WAVES;
}

hipError_t launch_write8(Write8Args a, int64_t q, hipStream_t s) {
    const int64_t R = 1ll << a.c.bshift;
    a.mb = (int)write8_blocks(q, R);
    const dim3 grid = grid_of((int64_t)a.c.B * a.mb), block(W8_THREADS);
    switch (R) {
        case 1: hipLaunchKernelGGL((write8_kernel<1>), grid, block, 0, s, a); break;
        case 2: hipLaunchKernelGGL((write8_kernel<2>), grid, block, 0, s, a); break;
        case 4: hipLaunchKernelGGL((write8_kernel<4>), grid, block, 0, s, a); break;
        case 8: hipLaunchKernelGGL((write8_kernel<8>), grid, block, 0, s, a); break;
        case 16: hipLaunchKernelGGL((write8_kernel<16>), grid, block, 0, s, a); break;
        case 32: hipLaunchKernelGGL((write8_kernel<32>), grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL((write8_kernel<64>), grid, block, 0, s, a); break;
    }
    return hipGetLastError();
}

}  // namespace vkv
