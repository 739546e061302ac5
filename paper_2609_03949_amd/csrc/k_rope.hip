// k_rope.hip -- rotary positions (gfx950): pairs of dims turned by the angle p f_i.
//
// The angles of a token are shared by its heads: a workgroup takes a token's heads (or a part of them,
// where there are few tokens), finds cosine and sine of its dims / 2 angles once, into LDS, and passes over the rows.  The angle
// is reduced to one turn in fp64 (far positions times the first frequencies have many turns), its sine and
// cosine are fp32.  Bound: HBM (each element read and written once).
#include <algorithm>

#include "vkv_internal.h"

namespace vkv {

constexpr int RP_THREADS = 256;

template <bool FAST>
__global__ __launch_bounds__(RP_THREADS) void rope_kernel(RopeArgs a) {
    __shared__ float turn[2][VKV_ROPE_MAX_DIMS / 2];      // cosines, sines, with the magnitude
    const uint32_t wg = workgroup_id();
    if (wg >= (uint32_t)(a.n_tok * a.parts)) return;
    const int tid = threadIdx.x, half = a.dims / 2;
    const int64_t tok = wg / (uint32_t)a.parts;
    const int part = (int)(wg % (uint32_t)a.parts);
    const int h0 = (int)((int64_t)part * a.H / a.parts), h1 = (int)((int64_t)(part + 1) * a.H / a.parts);
    for (int i = tid; i < half; i += RP_THREADS) {
        const double turns = (double)a.pos[tok] * a.freq[i] * 0.15915494309189533577;
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        turn[0][i] = a.magnitude * c;
        turn[1][i] = a.transposed ? -(a.magnitude * s) : a.magnitude * s;
    }
    __syncthreads();
    const uint16_t* x = a.x + tok * a.xts;
    uint16_t* out = a.out + tok * a.ots;
    const bool place = a.x == a.out;
    if constexpr (FAST) {
        // eight elements a lane, 16 bytes: whole pairs where they are neighbours, else the pairs' other halves beside them
        const int rot = a.interleaved ? a.dims / 8 : half / 8;      // pieces of a row that turn
        const int rest = place ? 0 : (a.width - a.dims) / 8;        // pieces that are copied
        const int per = rot + rest, first8 = a.first / 8;
        for (int i = tid; i < (h1 - h0) * per; i += RP_THREADS) {
            const int h = h0 + i / per, k = i % per;
            const u16x8_t* xr = reinterpret_cast<const u16x8_t*>(x + h * a.xhs);
            u16x8_t* orow = reinterpret_cast<u16x8_t*>(out + h * a.ohs);
            if (k >= rot) {
                const int q = k - rot, at = q < first8 ? q : q + a.dims / 8;
                orow[at] = xr[at];
            } else if (a.interleaved) {
                u16x8_t v = xr[first8 + k];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p = bf16_to_f32(v[2 * j]), q = bf16_to_f32(v[2 * j + 1]), c = turn[0][4 * k + j], s = turn[1][4 * k + j];
                    v[2 * j] = f32_to_bf16_rne(p * c - q * s);
                    v[2 * j + 1] = f32_to_bf16_rne(q * c + p * s);
                }
                orow[first8 + k] = v;
            } else {
                u16x8_t v = xr[first8 + k], y = xr[first8 + k + rot];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float p = bf16_to_f32(v[j]), q = bf16_to_f32(y[j]), c = turn[0][8 * k + j], s = turn[1][8 * k + j];
                    v[j] = f32_to_bf16_rne(p * c - q * s);
                    y[j] = f32_to_bf16_rne(q * c + p * s);
                }
                orow[first8 + k] = v;
                orow[first8 + k + rot] = y;
            }
        }
    } else {
        const int rest = place ? 0 : a.width - a.dims, per = half + rest;
        for (int64_t i = tid; i < (int64_t)(h1 - h0) * per; i += RP_THREADS) {
            const int h = h0 + (int)(i / per), k = (int)(i % per);
            const uint16_t* xr = x + h * a.xhs;
            uint16_t* orow = out + h * a.ohs;
            if (k >= half) {
                const int q = k - half, at = q < a.first ? q : q + a.dims;
                orow[at] = xr[at];
            } else {
                const int i0 = a.first + (a.interleaved ? 2 * k : k), i1 = i0 + (a.interleaved ? 1 : half);
                const float p = bf16_to_f32(xr[i0]), q = bf16_to_f32(xr[i1]), c = turn[0][k], s = turn[1][k];
                orow[i0] = f32_to_bf16_rne(p * c - q * s);
                orow[i1] = f32_to_bf16_rne(q * c + p * s);
            }
        }
    }
}

hipError_t launch_rope(RopeArgs a, hipStream_t s) {
    // about four workgroups a CU where the tokens alone are fewer, a head each at the least
    a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(a.H, 1024 / a.n_tok));
    auto al16 = [](const void* p) { return ((uintptr_t)p & 15u) == 0; };
    const bool fast = al16(a.x) && al16(a.out) && a.first % 8 == 0 && (a.dims / 2) % 8 == 0 && a.width % 8 == 0 &&
                      a.xts % 8 == 0 && a.xhs % 8 == 0 && a.ots % 8 == 0 && a.ohs % 8 == 0;
    const dim3 grid = grid_of(a.n_tok * a.parts), block(RP_THREADS);
    if (fast) hipLaunchKernelGGL((rope_kernel<true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rope_kernel<false>), grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace vkv
