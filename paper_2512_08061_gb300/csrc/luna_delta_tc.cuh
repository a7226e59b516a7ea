// The gated delta rule on tensor cores: bf16, chunks of 64 rows.
//
// With G_i the sum of a chunk's gates to row i, c(i, j) = exp(G_i - G_j), S the state before the chunk and
//
//     A_ij = b_i c(i, j) k_i . k_j  (j < i),   T = (1 + A)^-1,   P_ij = scale c(i, j) q_i . k_j  (j <= i)
//
// the rows that the chunk writes, its outputs and the state behind it are
//
//     U = T diag(b) (V - diag(c(i, 0)) K S),   O = scale diag(c(i, 0)) Q S + P U,   S' = c(C, 0) S + K^T diag(c(C, j)) U
//
// and with R the gradient of S', that of U's right-hand side and of S
//
//     X = T^T (P^T dO + diag(c(C, j)) K R),   R' = c(C, 0) R + scale Q^T diag(c(i, 0)) dO - K^T diag(b_i c(i, 0)) X.
//
// T and P come from one launch over all chunks; the chains over the chunks then run column by column of the state, a
// warp holding 16 columns (of S^T or R^T: 16 rows by d) in its accumulators.  The accumulators of one product have the
// layout that the next one's left operand wants, so that the whole chain of a chunk stays in a warp's registers and
// warps meet only where tiles arrive in shared memory.  That is why these products are the warps' own matrix
// instructions: through TMEM each of the chain's three products would wait for a round trip and a barrier, in tiles of
// 128 columns, one block a head (32 blocks for a prompt of 32 heads, where this form has 128).
// Precision.  Operands are fp16, scaled by powers of two: 11 bits where bf16 has 8, two terms 22.  The state, U and X
// enter products in two terms, T and (in reverse) P too, so that states and U are off by a few 1e-7; the outputs take
// one term of S, U and P (1.4e-4, under their own rounding).  K, Q, T and P are scaled by chunk, to a largest value of
// 2^12 to 2^13, what a warp holds by its own largest value, so that whatever is 2^-15 of its neighbours still has
// its 22 bits, and a state that all but vanishes within a chunk is off by 2^-35 of what was in its place; K, Q and dO are
// exact down to 2^-26 of their tile's largest value.  What a chunk adds to the
// state is summed by itself and added in fp32, because the tensor cores cut sums off.
#pragma once

#include <cuda_fp16.h>
#include <math.h>

#include "luna_delta.cuh"
#include "luna_prof.cuh"
#include "luna_sm100.cuh"

namespace luna {
int tc_sm_count();

namespace delta {

using namespace sm100;

constexpr int C = kDeltaRows;
constexpr int kTileB = C * C * 2;  // bytes of a 64 x 64 bf16 tile: rows of 128 bytes, 16-byte pieces swizzled
constexpr int kRowsF = kDeltaFactors;

// ---- tiles in shared memory: panels of 64 columns, row r's 16-byte piece p at place p ^ (r % 8)

__device__ __forceinline__ uint32_t tile_at(uint32_t base, int rows, int r, int piece) {
    return base + (piece >> 3) * rows * 128 + r * 128 + (((piece & 7) ^ (r & 7)) << 4);
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool in) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Eight values of a row into shared memory, zeros behind `n` of them: by an asynchronous copy, or one by one where rows do
// not start on 16-byte boundaries (or end inside one)
__device__ __forceinline__ void load_piece(uint32_t dst, const __nv_bfloat16 *src, const void *any, int n, bool vec) {
    if (vec) {
        copy16(dst, n > 0 ? src : any, n > 0);
        return;
    }
    uint32_t w[4] = {0, 0, 0, 0};
    const unsigned short *u = reinterpret_cast<const unsigned short *>(src);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) w[i / 2] |= (uint32_t)u[i] << (i % 2 * 16);
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}
// a tile of `rows` rows (64 of them, DP columns) of a tensor of d columns; zeros behind both
template <int DP>
__device__ __forceinline__ void load_rows(uint32_t dst, const __nv_bfloat16 *src, int64_t st, int rows, int d, bool vec, int tid, int threads) {
    for (int i = tid; i < C * DP / 8; i += threads) {
        const int r = i / (DP / 8), p = i % (DP / 8);
        load_piece(tile_at(dst, C, r, p), src + r * st + p * 8, src, r < rows ? d - p * 8 : 0, vec);
    }
}
// two neighbouring values of a row of which n are left
__device__ __forceinline__ float2 load_pair(const __nv_bfloat16 *p, int n, bool vec) {
    if (vec && n > 0) {
        const uint32_t u = *reinterpret_cast<const uint32_t *>(p);
        return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
    }
    return make_float2(n > 0 ? io_load(p) : 0.0f, n > 1 ? io_load(p + 1) : 0.0f);
}

// What this file's kernels leave for each other lies in global memory as its tile does in shared memory: one copy a tile.
__device__ __forceinline__ void load_tile(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src),
                 "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// ---- matrix instructions

using Frag = uint32_t[4];

__device__ __forceinline__ void ldm(Frag &f, uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(f[0]), "=r"(f[1]), "=r"(f[2]), "=r"(f[3]) : "r"(at));
}
__device__ __forceinline__ void ldm_t(Frag &f, uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(f[0]), "=r"(f[1]), "=r"(f[2]), "=r"(f[3]) : "r"(at));
}
__device__ __forceinline__ void stm_t(uint32_t at, const Frag &f) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(f[0]), "r"(f[1]), "r"(f[2]), "r"(f[3]) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const Frag &a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const Frag &a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Right operands of 16 summed indices and 16 columns (two n-tiles) from a tile that holds a row for each column (n) or
// for each summed index (k).
__device__ __forceinline__ void right_n(Frag &f, uint32_t base, int rows, int n0, int k0, int lane) {
    ldm(f, tile_at(base, rows, n0 + (lane >> 4) * 8 + (lane & 7), (k0 >> 3) + ((lane >> 3) & 1)));
}
__device__ __forceinline__ void right_k(Frag &f, uint32_t base, int rows, int k0, int n0, int lane) {
    ldm_t(f, tile_at(base, rows, k0 + ((lane >> 3) & 1) * 8 + (lane & 7), (n0 >> 3) + (lane >> 4)));
}
// Left operands of 16 rows and 16 summed indices from a tile that holds a row for each row (m) or summed index (k).
__device__ __forceinline__ void left_m(Frag &f, uint32_t base, int rows, int m0, int k0, int lane) {
    ldm(f, tile_at(base, rows, m0 + ((lane >> 3) & 1) * 8 + (lane & 7), (k0 >> 3) + (lane >> 4)));
}
__device__ __forceinline__ void left_k(Frag &f, uint32_t base, int rows, int k0, int m0, int lane) {
    ldm_t(f, tile_at(base, rows, k0 + (lane >> 4) * 8 + (lane & 7), (m0 >> 3) + ((lane >> 3) & 1)));
}

// pairs of bf16 (outputs, V, dO) and of fp16 (operands)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float low(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float high(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 half_pair(uint32_t u) {
    __half2 h;
    memcpy(&h, &u, 4);
    return __half22float2(h);
}
// x = hi + lo to 22 bits
__device__ __forceinline__ void split(float x0, float x1, uint32_t &hi, uint32_t &lo) {
    hi = pack(x0, x1);
    const float2 f = half_pair(hi);
    lo = pack(x0 - f.x, x1 - f.y);
}
// The power of two that takes a largest value of 2^E (to 2^(E+1)) to 2^12, and its inverse.  (Below 2^-113 all is 0; an
// infinity would leave everything else 0, so that all becomes NaN with it.)
struct Scale {
    float by, back;
};
__device__ __forceinline__ Scale scale_of(float most) {
    const uint32_t e = max((__float_as_uint(most) >> 23) & 255u, 14u);
    return Scale{__uint_as_float(e == 255u ? 0x7fffffffu : (254u + 12u - e) << 23), __uint_as_float((e - 12u) << 23)};
}
// of values that are not negative, whose bits are in their order
__device__ __forceinline__ float warp_max(float x) {
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(x)));
}
// the largest of all that a warp holds
template <int N>
__device__ __forceinline__ float most_of(const float (&c)[N][4]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, fmaxf(fmaxf(fabsf(c[i][0]), fabsf(c[i][1])), fmaxf(fabsf(c[i][2]), fabsf(c[i][3]))));
    return warp_max(m);
}
template <int N>
__device__ __forceinline__ Scale scale_of(const float (&c)[N][4]) {
    return scale_of(most_of(c));
}
// the left operand whose 16 summed indices are two neighbouring n-tiles of accumulators
__device__ __forceinline__ void split_left(const float (&c0)[4], const float (&c1)[4], float by, Frag &hi, Frag &lo) {
    split(by * c0[0], by * c0[1], hi[0], lo[0]);
    split(by * c0[2], by * c0[3], hi[1], lo[1]);
    split(by * c1[0], by * c1[1], hi[2], lo[2]);
    split(by * c1[2], by * c1[3], hi[3], lo[3]);
}

// 16 x 16 values of a left operand (or of two neighbouring n-tiles) into a tile
__device__ __forceinline__ void tile_put(uint32_t base, int rows, int r0, int k0, const Frag &f, int lane) {
    const uint32_t at = tile_at(base, rows, r0 + (lane >> 3 & 1) * 8 + (lane & 7), (k0 >> 3) + (lane >> 4));
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(f[0]), "r"(f[1]), "r"(f[2]), "r"(f[3]) : "memory");
}
// shared memory to global memory, by one thread (committed, not waited for)
__device__ __forceinline__ void store_tile(void *dst, uint32_t src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}

template <int N>
__device__ __forceinline__ void zero(float (&c)[N][4]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = 0.0f;
}

__device__ __forceinline__ float inverse2(float back) {  // of a power of two
    return __uint_as_float((254u << 23) - __float_as_uint(back));
}
inline unsigned blocks_of(int64_t a, int64_t b) { return (unsigned)((a + b - 1) / b); }

}  // namespace delta
}  // namespace luna
