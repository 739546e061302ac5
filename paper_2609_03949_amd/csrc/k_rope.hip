// k_rope.hip -- rotary positions (gfx950): pairs of dims turned by the angle p f_i.
//
// The angles of a token are shared by its heads: a workgroup takes a few tokens (or a part of one's heads, where there are few
// tokens), finds cosine and sine of their dims / 2 angles once, into LDS, while the first rows are on their way.  The angle
// is reduced to one turn in fp64 (far positions times the first frequencies have many turns), its sine and
// cosine are fp32.  Bound: HBM (each element read and written once): 16387 tokens of 16 heads, 64 of 192 dims turned, 50 us, 4.0
// TB/s, where a large copy reaches 4.9; with the input in the last-level cache 40 us, the vector units busy 92% of the cycles.
// 32 tokens of 128 heads 4.6 us.
#include <algorithm>

#include "vkv_internal.h"

namespace vkv {

constexpr int RP_THREADS = 256, RP_ANGLES = 512;   // angles of a workgroup's tokens
constexpr int RP_EACH = 4;                         // pieces a thread has in flight

template <bool FAST>
__global__ __launch_bounds__(RP_THREADS) void rope_kernel(RopeArgs a) {
    __shared__ float turn[2][RP_ANGLES];           // cosines, sines, with the magnitude
    const uint32_t wg = workgroup_id();
    const int64_t tok = (int64_t)(wg / (uint32_t)a.parts) * a.toks;
    if (tok >= a.n_tok) return;
    const int tid = threadIdx.x, half = a.dims / 2;
    const int part = (int)(wg % (uint32_t)a.parts), toks = (int)min((int64_t)a.toks, a.n_tok - tok);
    const int h0 = (int)((int64_t)part * a.H / a.parts), heads = (int)((int64_t)(part + 1) * a.H / a.parts) - h0;
    const bool place = a.x == a.out;
    const uint16_t* x = a.x + tok * a.xts + h0 * a.xhs;
    uint16_t* out = a.out + tok * a.ots + h0 * a.ohs;
    auto angles = [&]() __attribute__((always_inline)) {
        for (int i = tid; i < toks * half; i += RP_THREADS) {
            const int q = i / half;
            const double turns = (double)a.pos[tok + q] * a.freq[i - q * half] * 0.15915494309189533577;
            float s, c;
            sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
            turn[0][i] = a.magnitude * c;
            turn[1][i] = a.transposed ? -(a.magnitude * s) : a.magnitude * s;
        }
        __syncthreads();
    };
    if constexpr (FAST) {
        // eight elements a lane, 16 bytes: whole pairs where they are neighbours, else the pairs' other halves beside them
        const int rot = a.interleaved ? a.dims / 8 : half / 8;      // pieces of a row that turn
        const int rest = place ? 0 : (a.width - a.dims) / 8;        // pieces that are copied
        const uint32_t per = rot + rest, first8 = a.first / 8, row_items = heads * per, items = toks * row_items;
        for (uint32_t i0 = 0; i0 < items; i0 += RP_EACH * RP_THREADS) {
            const u16x8_t* src[RP_EACH];
            u16x8_t* dst[RP_EACH];
            int at[RP_EACH];                                        // the pair's first angle, or -1: copied, -2: none
            u16x8_t v[RP_EACH], y[RP_EACH];
#pragma unroll
            for (int u = 0; u < RP_EACH; ++u) {
                const uint32_t i = i0 + RP_THREADS * u + tid;
                at[u] = -2;
                if (i >= items) continue;
                const uint32_t q = i / row_items, r = i - q * row_items, h = r / per, k = r - h * per;
                const u16x8_t* xr = reinterpret_cast<const u16x8_t*>(x + q * a.xts + h * a.xhs);
                u16x8_t* orow = reinterpret_cast<u16x8_t*>(out + q * a.ots + h * a.ohs);
                uint32_t piece = first8 + k;
                at[u] = (int)(q * half + (a.interleaved ? 4 : 8) * k);
                if (k >= (uint32_t)rot) {
                    piece = k - rot;
                    if (piece >= first8) piece += a.dims / 8;
                    at[u] = -1;
                }
                src[u] = xr + piece;
                dst[u] = orow + piece;
                v[u] = *src[u];
                if (!a.interleaved && at[u] >= 0) y[u] = src[u][rot];
            }
            if (i0 == 0) angles();
#pragma unroll
            for (int u = 0; u < RP_EACH; ++u) {
                if (at[u] == -2) continue;
                if (at[u] >= 0 && a.interleaved) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float p = bf16_to_f32(v[u][2 * j]), q = bf16_to_f32(v[u][2 * j + 1]), c = turn[0][at[u] + j], s = turn[1][at[u] + j];
                        v[u][2 * j] = f32_to_bf16_rne(p * c - q * s);
                        v[u][2 * j + 1] = f32_to_bf16_rne(q * c + p * s);
                    }
                } else if (at[u] >= 0) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float p = bf16_to_f32(v[u][j]), q = bf16_to_f32(y[u][j]), c = turn[0][at[u] + j], s = turn[1][at[u] + j];
                        v[u][j] = f32_to_bf16_rne(p * c - q * s);
                        y[u][j] = f32_to_bf16_rne(q * c + p * s);
                    }
                    dst[u][rot] = y[u];
                }
                *dst[u] = v[u];
            }
        }
    } else {
        angles();
        const int rest = place ? 0 : a.width - a.dims;
        const uint32_t per = half + rest, row_items = heads * per, items = toks * row_items;
        for (uint32_t i = tid; i < items; i += RP_THREADS) {
            const uint32_t q = i / row_items, r = i - q * row_items, h = r / per, k = r - h * per;
            const uint16_t* xr = x + q * a.xts + h * a.xhs;
            uint16_t* orow = out + q * a.ots + h * a.ohs;
            if (k >= (uint32_t)half) {
                const int n = (int)k - half, at = n < a.first ? n : n + a.dims;
                orow[at] = xr[at];
            } else {
                const int i0 = a.first + (int)(a.interleaved ? 2 * k : k), i1 = i0 + (a.interleaved ? 1 : half);
                const float p = bf16_to_f32(xr[i0]), s0 = bf16_to_f32(xr[i1]), c = turn[0][q * half + k], s = turn[1][q * half + k];
                orow[i0] = f32_to_bf16_rne(p * c - s0 * s);
                orow[i1] = f32_to_bf16_rne(s0 * c + p * s);
            }
        }
    }
}

hipError_t launch_rope(RopeArgs a, hipStream_t s) {
    // about four workgroups a CU where the tokens alone are fewer, a head each at the least; where they are many, tokens
    // enough for every thread to have its pieces in flight
    a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(a.H, 1024 / a.n_tok));
    auto al16 = [](const void* p) { return ((uintptr_t)p & 15u) == 0; };
    const bool fast = al16(a.x) && al16(a.out) && a.first % 8 == 0 && (a.dims / 2) % 8 == 0 && a.width % 8 == 0 &&
                      a.xts % 8 == 0 && a.xhs % 8 == 0 && a.ots % 8 == 0 && a.ohs % 8 == 0;
    const int64_t pieces = (int64_t)a.H * std::max(a.width / 8, 1);
    a.toks = a.parts > 1 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({RP_ANGLES / (a.dims / 2), RP_EACH * RP_THREADS / pieces, a.n_tok / 1024}));
    const dim3 grid = grid_of((a.n_tok + a.toks - 1) / a.toks * a.parts), block(RP_THREADS);
    if (fast) hipLaunchKernelGGL((rope_kernel<true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rope_kernel<false>), grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace vkv
