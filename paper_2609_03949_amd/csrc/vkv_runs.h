// vkv_runs.h -- how the attention of a chunk over a paged cache is cut (gfx950): units of
// (token, head) rows, the tiles of all units laid end to end, and what joins the parts of a unit.
#pragma once

#include "vkv_pages.h"

namespace vkv {

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
template <int TILE>
__device__ __forceinline__ int unit_tiles(const ChunkArgs& a, const CkUnit& x, int rows) {
    if (x.row0 >= x.nrow) return 0;
    const int last = min(x.row0 + rows, x.nrow) - 1;
    const int seen = max(x.old + last / a.H + 1, 0);
    return max((seen + TILE - 1) / TILE, 1);
}

__device__ __forceinline__ int run_start(int g, int n, int total) { return (int)((int64_t)g * total / n); }

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));

// natural-log lse from the reference (log2 units) and the sum; nothing seen: -inf
__device__ __forceinline__ float lse_of(float m, float l) {
    return m == -INFINITY && l == 0.f ? -INFINITY : ((m == -INFINITY ? 0.f : m) + log2f(l)) * 0.69314718055994530942f;
}

// first tile of every unit in the run of all tiles, and their number, into LDS
template <int TILE, int THREADS>
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
        const int n = lane < U ? unit_tiles<TILE>(a, chunk_unit(a, lane, rows), rows) : 0;
        const int upto = wave_prefix(n);
        pre[lane] = upto - n;
        return __builtin_amdgcn_readlane(upto, 63);
    }
    constexpr int PER = CK_MAX_UNITS / THREADS;
    __shared__ int waves[THREADS / 64];
    int n[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int u = PER * tid + i;
        n[i] = u < U ? unit_tiles<TILE>(a, chunk_unit(a, u, rows), rows) : 0;
        sum += n[i];
    }
    const int upto = wave_prefix(sum);
    if (lane == 63) waves[tid >> 6] = upto;
    __syncthreads();
    int at = upto - sum, total = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
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

}  // namespace vkv
