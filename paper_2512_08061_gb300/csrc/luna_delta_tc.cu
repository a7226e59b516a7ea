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
// its 22 bits; K, Q and dO are exact down to 2^-26 of their tile's largest value.  What a chunk adds to the
// state is summed by itself and added in fp32, because the tensor cores cut sums off.
#include <cuda_fp16.h>
#include <math.h>

#include "luna_delta.cuh"
#include "luna_prof.cuh"
#include "luna_sm100.cuh"

namespace luna {
int tc_sm_count();

namespace {

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
// The power of two that takes a largest value of 2^E (to 2^(E+1)) to 2^12, and its inverse.  (Below 2^-113 all is 0.)
struct Scale {
    float by, back;
};
__device__ __forceinline__ Scale scale_of(float most) {
    const uint32_t e = max((__float_as_uint(most) >> 23) & 255u, 14u);
    return Scale{__uint_as_float((254u + 12u - e) << 23), __uint_as_float((e - 12u) << 23)};
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int w = 16; w > 0; w /= 2) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, w));
    return x;
}
// one scale for all that a warp holds
template <int N>
__device__ __forceinline__ Scale scale_of(const float (&c)[N][4]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, fmaxf(fmaxf(fabsf(c[i][0]), fabsf(c[i][1])), fmaxf(fabsf(c[i][2]), fabsf(c[i][3]))));
    return scale_of(warp_max(m));
}
// the left operand whose 16 summed indices are two neighbouring n-tiles of accumulators
__device__ __forceinline__ void split_left(const float (&c0)[4], const float (&c1)[4], float by, Frag &hi, Frag &lo) {
    split(by * c0[0], by * c0[1], hi[0], lo[0]);
    split(by * c0[2], by * c0[3], hi[1], lo[1]);
    split(by * c1[0], by * c1[1], hi[2], lo[2]);
    split(by * c1[2], by * c1[3], hi[3], lo[3]);
}

template <int N>
__device__ __forceinline__ void zero(float (&c)[N][4]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = 0.0f;
}

// ---------------------------------------------------------------------------
// T, P and the factors of every chunk.  A block of four warps a chunk, a warp 16 rows of K K^T and Q K^T.  The inverse
// of the diagonal blocks of 16 rows is taken by substitution in fp32, a lane a column; a warp then goes down one block
// column of T, transposed so that each product's accumulators are the next one's left operand:
//
//     T_IJ^T = -(sum_{J <= K < I} T_KJ^T A_IK^T) T_II^T
//
// with both operands in two terms.  It leaves T^T, P and in a chunk's factors: c(i, 0) 2^ek, c(C, i) 2^ek, b,
// scale c(i, 0) 2^eq of its rows, then c(C, 0) in two terms and what T, P, K and Q were scaled down by (the last two
// are 2^ek and 2^eq).  (With the inverse in fp32 by all threads, 13 barriers and 68 KB of shared memory: 248 us for 8192
// chunks.)

constexpr int kPrepThreads = 128;

template <int DP>
struct PrepShared {
    alignas(128) char k[DP / 64][kTileB], q[DP / 64][kTileB], A[2][kTileB];  // A: two planes; T_II in its diagonal blocks
    float diag[4][16][17];
    float hi[C], lo[C], past[C], left[C], b[C], most[5][kPrepThreads / 32], back_T[4];
};

// the half row of a bf16 tile that a thread scales: its largest value; in fp16 to `out`
template <int DP>
__device__ __forceinline__ uint4 prep_piece(uint32_t tile, int tid, int p) {
    uint4 w;
    const uint32_t at = tile_at(tile, C, tid / 2, tid % 2 * (DP / 16) + p);
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(at));
    return w;
}
template <int DP>
__device__ __forceinline__ float prep_most(uint32_t tile, int tid) {
    uint32_t most = 0;
#pragma unroll
    for (int p = 0; p < DP / 16; ++p) {
        const uint4 w = prep_piece<DP>(tile, tid, p);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max(most, max((u[i] << 16) & 0x7fff0000u, u[i] & 0x7fff0000u));
    }
    return __uint_as_float(most);
}
template <int DP>
__device__ __forceinline__ void prep_write(uint32_t tile, float by, __half *out, int tid) {
#pragma unroll
    for (int p = 0; p < DP / 16; ++p) {
        const uint4 w = prep_piece<DP>(tile, tid, p);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
        uint32_t f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = pack(by * low(u[i]), by * high(u[i]));
        *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(out) + tile_at(0, C, tid / 2, tid % 2 * (DP / 16) + p)) = make_uint4(f[0], f[1], f[2], f[3]);
    }
}
// acc += F M^T in two terms each, for F of 16 rows and 16 summed indices, M the 16 x 16 block (n0, k0) of two planes
__device__ __forceinline__ void prep_product(float (&acc)[2][4], const Frag &hi, const Frag &lo, uint32_t planes, int n0, int k0, int lane) {
    Frag f, g;
    right_n(f, planes, C, n0, k0, lane);
    right_n(g, planes + kTileB, C, n0, k0, lane);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        mma(acc[i], hi, f[2 * i], f[2 * i + 1]);
        mma(acc[i], lo, f[2 * i], f[2 * i + 1]);
        mma(acc[i], hi, g[2 * i], g[2 * i + 1]);
    }
}

template <int DP, bool TERMS>  // TERMS: P in two terms
__global__ void __launch_bounds__(kPrepThreads, 4) k_delta_prepare(DeltaArgs a) {
    extern __shared__ __align__(128) char raw[];
    PrepShared<DP> &sm = *reinterpret_cast<PrepShared<DP> *>(raw);
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, q2 = lane % 4 * 2;
    const int64_t at = blockIdx.x, bh = at / a.m;
    const int chunk = (int)(at % a.m), b = (int)(bh / a.H), h = (int)(bh % a.H), t0 = chunk * C;
    const int rows = min(C, head_length(a.lengths, b, a.n) - t0);
    if (at == 0 && tid == 0) *a.status = 0;  // (the waits that set it run for a second)
    if (rows <= 0) return;
    const int hk = h / (a.H / a.k.heads);
    const uint32_t sk = smem_u32(sm.k), sq = smem_u32(sm.q), sA = smem_u32(sm.A);
    load_rows<DP>(sk, static_cast<const __nv_bfloat16 *>(a.k.p) + b * a.k.sb + hk * a.k.sh + t0 * a.k.st, a.k.st, rows, a.d, a.vec, tid, kPrepThreads);
    load_rows<DP>(sq, static_cast<const __nv_bfloat16 *>(a.q.p) + b * a.q.sb + hk * a.q.sh + t0 * a.q.st, a.q.st, rows, a.d, a.vec, tid, kPrepThreads);
    copies_end();
    if (warp == 0)
        delta_gate_sums(lane, [&](int t) { return t < rows ? gate_at<__nv_bfloat16>(a.g, b, h, t0 + t) : 0.0f; }, sm.hi, sm.lo,
                        sm.past, sm.left);
    else if (warp < 3)
        sm.b[tid - 32] = tid - 32 < rows ? gate_at<__nv_bfloat16>(a.b, b, h, t0 + tid - 32) : 0.0f;
    copies_wait<0>();
    __syncthreads();
    auto most_of = [&](int which, float x) {  // to be read after a barrier
        x = warp_max(x);
        if (lane == 0) sm.most[which][warp] = x;
    };
    auto block_scale = [&](int which) {
        const float *m = sm.most[which];
        return scale_of(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
    };
    most_of(2, prep_most<DP>(sk, tid));
    most_of(3, prep_most<DP>(sq, tid));

    const int r0 = warp * 16;
    float kk[8][4], qk[8][4];
    zero(kk);
    zero(qk);
#pragma unroll
    for (int k0 = 0; k0 < DP; k0 += 16) {
        Frag fk, fq;
        left_m(fk, sk, C, r0, k0, lane);
        left_m(fq, sq, C, r0, k0, lane);
#pragma unroll
        for (int n0 = 0; n0 < C; n0 += 16) {
            if (n0 > r0) continue;
            Frag f;
            right_n(f, sk, C, n0, k0, lane);
            mma_bf16(kk[n0 / 8], fk, f[0], f[1]);
            mma_bf16(kk[n0 / 8 + 1], fk, f[2], f[3]);
            mma_bf16(qk[n0 / 8], fq, f[0], f[1]);
            mma_bf16(qk[n0 / 8 + 1], fq, f[2], f[3]);
        }
    }
    float most_p = 0.0f, most_a = 0.0f;
#pragma unroll
    for (int nt = 0; nt < 8; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = r0 + lane / 4 + (e >> 1) * 8, j = nt * 8 + q2 + (e & 1);
            const float c = j <= i ? expf((sm.hi[i] - sm.hi[j]) + (sm.lo[i] - sm.lo[j])) : 0.0f;
            qk[nt][e] = j <= i ? a.scale * c * qk[nt][e] : 0.0f;
            kk[nt][e] = j < i ? sm.b[i] * c * kk[nt][e] : 0.0f;
            most_p = fmaxf(most_p, fabsf(qk[nt][e]));
            most_a = fmaxf(most_a, fabsf(kk[nt][e]));
            if (nt / 2 == warp) sm.diag[warp][i - r0][j - r0] = kk[nt][e];
        }
    most_of(0, most_p);
    most_of(1, most_a);
    __syncthreads();
    const Scale ps = block_scale(0), as = block_scale(1), ks = block_scale(2), qs = block_scale(3);
    if (h % (a.H / a.k.heads) == 0) {  // one head of those that share queries and keys
        const int64_t to = ((int64_t)b * a.k.heads + hk) * a.m + chunk;
        prep_write<DP>(sk, ks.by, a.Kp + to * C * DP, tid);
        prep_write<DP>(sq, qs.by, a.Qp + to * C * DP, tid);
    }
    float *rowf = a.rows + at * kRowsF;
    if (tid < C) {
        rowf[tid] = sm.past[tid] * ks.back;
        rowf[C + tid] = sm.left[tid] * ks.back;
        rowf[2 * C + tid] = sm.b[tid];
        rowf[3 * C + tid] = a.scale * sm.past[tid] * qs.back;
    }
    if (tid == 0) {
        gate_terms(sm.hi[C - 1], rowf[4 * C], rowf[4 * C + 1]);
        rowf[4 * C + 3] = ps.back;
        rowf[4 * C + 4] = ks.back;
        rowf[4 * C + 5] = qs.back;
    }
    char *P = reinterpret_cast<char *>(a.Pp + at * (TERMS ? 2 : 1) * C * C);
#pragma unroll
    for (int nt = 0; nt < 8; ++nt)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            const uint32_t to = tile_at(0, C, r0 + lane / 4 + e * 4, nt) + q2 * 2;
            uint32_t hi, lo;
            split(ps.by * qk[nt][e], ps.by * qk[nt][e + 1], hi, lo);
            *reinterpret_cast<uint32_t *>(P + to) = hi;
            if (TERMS) *reinterpret_cast<uint32_t *>(P + kTileB + to) = lo;
            if (nt / 2 >= warp) continue;  // (its diagonal block waits for T_II)
            split(as.by * kk[nt][e], as.by * kk[nt][e + 1], hi, lo);
            *reinterpret_cast<uint32_t *>(sm.A[0] + to) = hi;
            *reinterpret_cast<uint32_t *>(sm.A[1] + to) = lo;
        }
    // T_II, a lane a column
    {
        float x[16], m = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = i == lane ? 1.0f : 0.0f;
#pragma unroll
            for (int l = 0; l < i; ++l) x[i] = fmaf(-sm.diag[warp][i][l], x[l], x[i]);
            m = fmaxf(m, fabsf(x[i]));
        }
        const Scale s = scale_of(warp_max(m));  // (the lanes without a column hold zeros)
        if (lane == 0) sm.back_T[warp] = s.back;
        if (lane < 16)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float y = s.by * x[i];
                const __half hi = __float2half_rn(y), lo = __float2half_rn(y - __half2float(hi));
                const uint32_t to = tile_at(0, C, r0 + i, (r0 + lane) >> 3) + (lane & 7) * 2;
                *reinterpret_cast<__half *>(sm.A[0] + to) = hi;
                *reinterpret_cast<__half *>(sm.A[1] + to) = lo;
                sm.diag[warp][i][lane] = x[i];
            }
    }
    __syncthreads();
    // block column J = warp of T, transposed: rows j, columns i
    float T[4][2][4];
    Frag hi[3], lo[3];
    float back[3];
#pragma unroll
    for (int I = 0; I < 4; ++I) zero(T[I]);
    left_k(hi[0], sA, C, r0, r0, lane);
    left_k(lo[0], sA + kTileB, C, r0, r0, lane);
    back[0] = sm.back_T[warp];
#pragma unroll
    for (int s = 1; s < 4; ++s) {
        const int I = warp + s;
        if (I > 3) break;
        float acc[2][4], y[2][4];
        zero(acc);
#pragma unroll
        for (int t = 0; t < s; ++t) {
            zero(y);
            prep_product(y, hi[t], lo[t], sA, I * 16, r0 + t * 16, lane);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][e] = fmaf(back[t] * as.back, y[i][e], acc[i][e]);
        }
        const Scale sc = scale_of(acc);
        Frag fh, fl;
        split_left(acc[0], acc[1], sc.by, fh, fl);
        zero(y);
        prep_product(y, fh, fl, sA, I * 16, I * 16, lane);
        const float by = -sc.back * sm.back_T[I];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) T[s][i][e] = by * y[i][e];
        if (s < 3) {
            const Scale st = scale_of(T[s]);
            split_left(T[s][0], T[s][1], st.by, hi[s], lo[s]);
            back[s] = st.back;
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) T[0][i][e] = sm.diag[warp][i * 8 + q2 + (e & 1)][lane / 4 + (e >> 1) * 8];
    float m = 0.0f;
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) m = fmaxf(m, fabsf(T[s][i][e]));
    most_of(4, m);
    __syncthreads();
    const Scale ts = block_scale(4);
    if (tid == 0) rowf[4 * C + 2] = ts.back;
    char *planes = reinterpret_cast<char *>(a.Tp + at * 2 * C * C);
#pragma unroll
    for (int s = 0; s < 4; ++s)  // (block row J + s, or the empty ones before J)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                uint32_t th, tl;
                split(ts.by * T[s][i][e], ts.by * T[s][i][e + 1], th, tl);
                const uint32_t to = tile_at(0, C, r0 + lane / 4 + e * 4, (warp + s) % 4 * 2 + i) + q2 * 2;
                *reinterpret_cast<uint32_t *>(planes + to) = th;
                *reinterpret_cast<uint32_t *>(planes + kTileB + to) = tl;
            }
}

// ---------------------------------------------------------------------------
// The chains.  A block has NG groups of 16 columns of one head's state, a group SP warps: with few heads two, which hold
// half of each column and exchange their shares of K S (and Q S) once a chunk; each then has 230 products a chunk where
// one warp has 420.  The tiles of a chunk come by asynchronous copies while the chunk before is worked on; one barrier a
// chunk.

enum ChainMode {
    kOutputs,   // O (and the last state)
    kKeep,      // U and the states, for the gradients
    kReverse    // dV, X, dO and the gradients of the states
};

template <int DP, int NG, int SP, ChainMode MODE>
struct ChainShared {
    static constexpr int kWarps = NG * SP;
    static constexpr int kPitch = NG * 32 + 16;  // bytes of a row of V or dO: eight rows start in eight banks
    static constexpr bool kQ = MODE != kKeep;    // Q and P are needed
    static constexpr int kPlanes = MODE == kReverse ? 2 : 1;  // of P
    struct Stage {
        alignas(128) char k[DP / 64][kTileB], q[kQ ? DP / 64 : 1][kQ ? kTileB : 16], T[2][kTileB];
        alignas(128) char P[kPlanes][kQ ? kTileB : 16], x[C * kPitch];
        alignas(16) float rows[kRowsF];
    } stage[2];
    uint64_t bar[2];
    alignas(16) char out[kQ ? kWarps : 1][C * 48];  // 16 columns of the outputs, rows of 32 bytes 48 apart
    alignas(128) char planes[MODE != kOutputs && SP == 1 ? kWarps : 1][DP * 32];  // 16 rows of a tile that is kept
    float4 shares[SP == 1 ? 1 : kWarps][SP == 1 ? 1 : 12][32];
};

template <int DP, int NG, int SP, ChainMode MODE>
__device__ __forceinline__ void chain_load(typename ChainShared<DP, NG, SP, MODE>::Stage &st, uint64_t *bar, const DeltaArgs &a,
                                           int64_t bh, int b, int h, int chunk, int len, int col0, int tid) {
    using Sh = ChainShared<DP, NG, SP, MODE>;
    const int t0 = chunk * C, rows = min(C, len - t0);
    if (tid == 0) {
        const int64_t at = bh * a.m + chunk, kat = ((int64_t)b * a.k.heads + h / (a.H / a.k.heads)) * a.m + chunk;
        mbar_arrive_expect_tx(bar, sizeof(st.k) + sizeof(st.T) + sizeof(st.rows) + (Sh::kQ ? sizeof(st.q) + sizeof(st.P) : 0));
        load_tile(st.k, a.Kp + kat * C * DP, sizeof(st.k), bar);
        if (Sh::kQ) load_tile(st.q, a.Qp + kat * C * DP, sizeof(st.q), bar);
        load_tile(st.rows, a.rows + at * kRowsF, sizeof(st.rows), bar);
        load_tile(st.T, a.Tp + at * 2 * C * C, sizeof(st.T), bar);
        if (Sh::kQ) load_tile(st.P, a.Pp + at * a.planes * C * C, sizeof(st.P), bar);
    }
    const RowView &xv = MODE == kReverse ? a.go : a.v;
    const __nv_bfloat16 *x = static_cast<const __nv_bfloat16 *>(xv.p) + b * xv.sb + h * xv.sh + t0 * xv.st + col0;
    const uint32_t sx = smem_u32(st.x);
#pragma unroll
    for (int i = tid; i < C * NG * 2; i += Sh::kWarps * 32) {
        const int r = i / (NG * 2), p = i % (NG * 2);
        load_piece(sx + r * Sh::kPitch + p * 16, x + r * xv.st + p * 8, xv.p, r < rows ? a.dv - col0 - p * 8 : 0, a.vec);
    }
    copies_end();
}

// Rows first, first + 1, .. (n of them) of a warp's 16 columns, given column by column, to the output: transposed through
// shared memory
__device__ __forceinline__ void chain_store(const float (&acc)[8][4], int first, int n, char *mem, __nv_bfloat16 *out, int64_t st, int rows,
                                            int col, int dv, bool vec, int lane) {
    const uint32_t base = smem_u32(mem);
#pragma unroll
    for (int nt = 0; nt < 8; nt += 2) {
        if (nt * 8 < first || nt * 8 >= first + n) continue;
        const Frag f = {pack_bf16(acc[nt][0], acc[nt][1]), pack_bf16(acc[nt][2], acc[nt][3]),
                        pack_bf16(acc[nt + 1][0], acc[nt + 1][1]), pack_bf16(acc[nt + 1][2], acc[nt + 1][3])};
        stm_t(base + (nt * 8 + (lane >> 4) * 8 + (lane & 7)) * 48 + ((lane >> 3) & 1) * 16, f);
    }
    __syncwarp();
    for (int i = 0; i < n / 16; ++i) {
        const int r = first + i * 16 + lane / 2, half = lane % 2;
        if (r < rows && col + half * 8 < dv) {
            const __nv_bfloat16 *from = reinterpret_cast<const __nv_bfloat16 *>(mem + r * 48 + half * 16);
            __nv_bfloat16 *to = out + r * st + col + half * 8;
            if (vec)
                *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from);
            else
                for (int e = 0; e < min(8, dv - col - half * 8); ++e) to[e] = from[e];
        }
    }
    __syncwarp();
}

// 16 rows of a tile that is kept for the gradients, from left operands: through shared memory, from where one copy a panel
// takes them (stored from the registers, four bytes a lane in eight rows, they took a fifth of the chain's time)
__device__ __forceinline__ void plane_room(int lane) {  // the copies before have read what they take
    if (lane == 0) bulk_wait_read();
    __syncwarp();
}
__device__ __forceinline__ void plane_put(char *mem, int k0, const Frag &f, int lane) {
    const int r = (lane >> 3 & 1) * 8 + (lane & 7);
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(smem_u32(mem) + tile_at(0, 16, r, (k0 >> 3) + (lane >> 4))),
                 "r"(f[0]), "r"(f[1]), "r"(f[2]), "r"(f[3])
                 : "memory");
}
__device__ __forceinline__ void plane_send(const char *mem, __half *tile, int rows, int r0, int panels, int lane) {
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
        for (int p = 0; p < panels; ++p)
            asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], 2048;" ::"l"(reinterpret_cast<char *>(tile) + (p * rows + r0) * 128),
                         "r"(smem_u32(mem) + p * 2048)
                         : "memory");
        bulk_commit();
    }
}
// (where a group's warps share rows of 128 bytes) from the registers
__device__ __forceinline__ void plane_store(__half *tile, int rows, int r0, int k0, const Frag &f, int lane) {
    char *p = reinterpret_cast<char *>(tile) + lane % 4 * 4;
    const int r = r0 + lane / 4;
    *reinterpret_cast<uint32_t *>(p + tile_at(0, rows, r, k0 >> 3)) = f[0];
    *reinterpret_cast<uint32_t *>(p + tile_at(0, rows, r + 8, k0 >> 3)) = f[1];
    *reinterpret_cast<uint32_t *>(p + tile_at(0, rows, r, (k0 >> 3) + 1)) = f[2];
    *reinterpret_cast<uint32_t *>(p + tile_at(0, rows, r + 8, (k0 >> 3) + 1)) = f[3];
}

template <int DP, int NG, int SP, ChainMode MODE>
__global__ void __launch_bounds__(NG * SP * 32) k_delta_chain(DeltaArgs a) {
    using Sh = ChainShared<DP, NG, SP, MODE>;
    extern __shared__ __align__(128) char raw[];
    Sh &sm = *reinterpret_cast<Sh *>(raw);
    constexpr bool REV = MODE == kReverse;
    constexpr int ND = DP / 8 / SP;  // n-tiles of a state's row that a warp holds
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, group = warp / SP, part = warp % SP, d0 = part * (DP / SP);
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / a.H), h = (int)(bh % a.H), col0 = blockIdx.y * NG * 16, col = col0 + group * 16;
    const int len = head_length(a.lengths, b, a.n), chunks = (len + C - 1) / C, q2 = lane % 4 * 2;
    const bool mine = col < a.dv;  // the warp has columns
    __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(a.o) + b * a.ob + h * a.oh;  // (not with kKeep)
    // what is kept: by copies where a warp has whole rows of 128 bytes
    char *const mem = sm.planes[SP == 1 ? warp : 0];
    auto put = [&](__half *tile, int k0, const Frag &f) {
        if (SP == 1)
            plane_put(mem, k0, f, lane);
        else
            plane_store(tile, a.dvp, col, k0, f, lane);
    };
    auto room = [&]() {
        if (SP == 1) plane_room(lane);
    };
    auto send = [&](__half *tile, int panels) {
        if (SP == 1) plane_send(mem, tile, a.dvp, col, panels, lane);
    };
    // n-tiles of rows that the warp finishes where a group's warps share that work, for 16 of them (np)
    auto own = [&](int np) { return SP == 1 || np / 2 == part; };
    const int first = SP == 1 ? 0 : part * (C / 2), some = C / SP;

    // S^T or R^T: row lane / 4 (and 8 more) of the warp's columns, values d0 + 8 nt + q2 and the next
    float S[ND][4];
    const float *init = REV ? a.dS1 : a.S0;
    auto place = [&](int nt, int e, int64_t &at) {
        const int c = col + lane / 4 + (e >> 1) * 8, r = d0 + nt * 8 + q2 + (e & 1);
        at = (bh * a.d + r) * a.dv + c;
        return r < a.d && c < a.dv;
    };
#pragma unroll
    for (int nt = 0; nt < ND; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            int64_t at;
            S[nt][e] = init && place(nt, e, at) ? init[at] : 0.0f;
        }
    // the scales of the warp's columns: 0, 1: of the halves of S before a chunk, 2, 3: of R, 4: U, 5: X, 6: dO
    auto scales_of = [&](int chunk) { return a.scales + ((bh * (a.m + 1) + chunk) * (a.dvp / 16) + col / 16) * kDeltaScales; };
    auto keep_scale = [&](int chunk, float back) {
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < 2 / SP; ++i) scales_of(chunk)[(REV ? 2 : 0) + part + i] = back;
    };

    if (tid < 2) mbar_init(&sm.bar[tid], 1);
    fence_mbar_init();
    __syncthreads();
    if (chunks > 0) chain_load<DP, NG, SP, MODE>(sm.stage[0], &sm.bar[0], a, bh, b, h, REV ? chunks - 1 : 0, len, col0, tid);
    for (int step = 0; step < chunks; ++step) {
        const int chunk = REV ? chunks - 1 - step : step, t0 = chunk * C;
        typename Sh::Stage &st = sm.stage[step & 1];
        copies_wait<0>();
        const bool here = mbar_wait_long(&sm.bar[step & 1], (step >> 1) & 1);
        if (__syncthreads_or(!here)) {  // a copy that did not arrive within a second: give up
            if (tid == 0) {
                atomicOr(a.status, 1);
                mbar_wait(&sm.bar[step & 1], (step >> 1) & 1, kDrainNs);
            }
            break;
        }
        if (step + 1 < chunks)
            chain_load<DP, NG, SP, MODE>(sm.stage[(step + 1) & 1], &sm.bar[(step + 1) & 1], a, bh, b, h, REV ? chunk - 1 : chunk + 1, len, col0, tid);
        if (!mine) continue;
        const uint32_t sk = smem_u32(st.k), sq = smem_u32(st.q), sT = smem_u32(st.T), sP = smem_u32(st.P);
        const uint32_t sx = smem_u32(st.x) + ((lane >> 4) * 8 + (lane & 7)) * Sh::kPitch + group * 32 + ((lane >> 3) & 1) * 16;
        const float whole = st.rows[4 * C], rest = st.rows[4 * C + 1], back_T = st.rows[4 * C + 2], back_P = st.rows[4 * C + 3];
        auto factor = [&](int which, int t) { return *reinterpret_cast<const float2 *>(st.rows + which * C + t); };
        const int64_t at = bh * a.m + chunk;
        // S <- c(C, 0) S (first) + F M for a left operand F of 64 summed rows and the tile M (a row for each)
        auto update = [&](const Frag (&fh)[4], const Frag (&fl)[4], float back, uint32_t tile, bool decay) {
#pragma unroll
            for (int np = 0; np < ND / 2; np += 2) {
                float acc[4][4];
                zero(acc);
#pragma unroll
                for (int kt = 0; kt < 4; ++kt) {
                    Frag f, g;
                    right_k(f, tile, C, kt * 16, d0 + np * 16, lane);
                    right_k(g, tile, C, kt * 16, d0 + np * 16 + 16, lane);
                    mma(acc[0], fh[kt], f[0], f[1]);
                    mma(acc[1], fh[kt], f[2], f[3]);
                    mma(acc[2], fh[kt], g[0], g[1]);
                    mma(acc[3], fh[kt], g[2], g[3]);
                    mma(acc[0], fl[kt], f[0], f[1]);
                    mma(acc[1], fl[kt], f[2], f[3]);
                    mma(acc[2], fl[kt], g[0], g[1]);
                    mma(acc[3], fl[kt], g[2], g[3]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float &s = S[2 * np + i][e];
                        s = decay ? fmaf(whole, s, fmaf(rest, s, back * acc[i][e])) : fmaf(back, acc[i][e], s);
                    }
            }
        };
        // the other warp's share of x, and of y's own rows, added to this one's
        auto exchange = [&](float (&x)[8][4], float (&y)[8][4], bool both) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sm.shares[warp][i][lane] = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
            if (both)
#pragma unroll
                for (int i = 0; i < 4; ++i) {  // (the rows that the other one finishes)
                    const float *lo = y[i], *hi = y[4 + i];
                    sm.shares[warp][8 + i][lane] = part ? make_float4(lo[0], lo[1], lo[2], lo[3]) : make_float4(hi[0], hi[1], hi[2], hi[3]);
                }
            asm volatile("bar.sync %0, 64;" ::"r"(1 + group) : "memory");
            const float4 (*other)[32] = sm.shares[warp ^ 1];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 v = other[i][lane];
                x[i][0] += v.x; x[i][1] += v.y; x[i][2] += v.z; x[i][3] += v.w;
            }
            if (both)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 v = other[8 + i][lane];
                    const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y[i][e] += part ? 0.0f : w[e];
                        y[4 + i][e] += part ? w[e] : 0.0f;
                    }
                }
        };
        float x[8][4], y[8][4];
        zero(x);
        zero(y);
        // x = K S (or K R), with it Q S
        const Scale ss = scale_of(S);
        {
            __half *ends = REV ? a.Rp + (bh * (a.m + 1) + chunk + 1) * a.dvp * DP : a.Sp + at * a.dvp * DP;
            if (MODE != kOutputs) {
                keep_scale(REV ? chunk + 1 : chunk, ss.back);
                room();
            }
#pragma unroll
            for (int kt = 0; kt < ND / 2; ++kt) {
                Frag hi, lo;
                split_left(S[2 * kt], S[2 * kt + 1], ss.by, hi, lo);
                if (MODE != kOutputs) put(ends, d0 + kt * 16, hi);
#pragma unroll
                for (int np = 0; np < 4; ++np) {
                    Frag f;
                    right_n(f, sk, C, np * 16, d0 + kt * 16, lane);
                    mma(x[2 * np], hi, f[0], f[1]);
                    mma(x[2 * np + 1], hi, f[2], f[3]);
                    mma(x[2 * np], lo, f[0], f[1]);
                    mma(x[2 * np + 1], lo, f[2], f[3]);
                    if (MODE == kOutputs) {
                        right_n(f, sq, C, np * 16, d0 + kt * 16, lane);
                        mma(y[2 * np], hi, f[0], f[1]);
                        mma(y[2 * np + 1], hi, f[2], f[3]);
                    }
                }
            }
            if (MODE != kOutputs) send(ends, DP / 64);
        }
        Frag fh[4], fl[4];
        if (!REV) {
            float back_s = ss.back;
            if (SP == 2) {
#pragma unroll
                for (int nt = 0; nt < 8; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[nt][e] *= ss.back;
                        y[nt][e] *= ss.back;
                    }
                exchange(x, y, MODE == kOutputs);
                back_s = 1.0f;
            }
            // x = b (V - c(i, 0) K S)
#pragma unroll
            for (int np = 0; np < 4; ++np) {
                Frag v;
                ldm_t(v, sx + np * 16 * Sh::kPitch);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int nt = 2 * np + i, t = nt * 8 + q2;
                    const float2 past = factor(0, t), beta = factor(2, t);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = back_s * (e & 1 ? past.y : past.x), vv = e & 1 ? high(v[2 * i + (e >> 1)]) : low(v[2 * i + (e >> 1)]);
                        x[nt][e] = (e & 1 ? beta.y : beta.x) * fmaf(-p, x[nt][e], vv);
                    }
                }
            }
            // U = T x
            float u[8][4];
            zero(u);
            const Scale xs = scale_of(x);
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                Frag hi, lo;
                split_left(x[2 * kt], x[2 * kt + 1], xs.by, hi, lo);
#pragma unroll
                for (int np = kt; np < 4; ++np) {
                    Frag f;
                    right_k(f, sT, C, kt * 16, np * 16, lane);
                    mma(u[2 * np], hi, f[0], f[1]);
                    mma(u[2 * np + 1], hi, f[2], f[3]);
                    mma(u[2 * np], lo, f[0], f[1]);
                    mma(u[2 * np + 1], lo, f[2], f[3]);
                    right_k(f, sT + kTileB, C, kt * 16, np * 16, lane);
                    mma(u[2 * np], hi, f[0], f[1]);
                    mma(u[2 * np + 1], hi, f[2], f[3]);
                }
            }
            const float back_u = xs.back * back_T;
#pragma unroll
            for (int nt = 0; nt < 8; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) u[nt][e] *= back_u;
            {  // P U, or U's plane
                __half *tile = a.Up + at * a.dvp * C;
                if (MODE == kKeep) room();
#pragma unroll
                for (int nt = 0; nt < 8; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[nt][e] = 0.0f;
                const Scale us = scale_of(u);
#pragma unroll
                for (int kt = 0; kt < 4; ++kt) {
                    const Frag hi = {pack(us.by * u[2 * kt][0], us.by * u[2 * kt][1]), pack(us.by * u[2 * kt][2], us.by * u[2 * kt][3]),
                                     pack(us.by * u[2 * kt + 1][0], us.by * u[2 * kt + 1][1]), pack(us.by * u[2 * kt + 1][2], us.by * u[2 * kt + 1][3])};
                    if (MODE == kKeep && own(kt)) put(tile, kt * 16, hi);
                    if (MODE == kOutputs)
#pragma unroll
                        for (int np = kt; np < 4; ++np) {
                            if (!own(np)) continue;
                            Frag f;
                            right_n(f, sP, C, np * 16, kt * 16, lane);
                            mma(x[2 * np], hi, f[0], f[1]);
                            mma(x[2 * np + 1], hi, f[2], f[3]);
                        }
                }
                if (MODE == kKeep) {
                    send(tile, 1);
                    if (lane == 0) scales_of(chunk)[4] = us.back;
                } else {  // scale c(i, 0) Q S + P U
                    const float back = us.back * back_P;
#pragma unroll
                    for (int nt = 0; nt < 8; ++nt) {
                        const float2 past = factor(3, nt * 8 + q2);
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[nt][e] = fmaf(back_s * (e & 1 ? past.y : past.x), y[nt][e], back * x[nt][e]);
                    }
                    chain_store(y, first, some, sm.out[warp], o + t0 * a.ot, a.ot, min(C, len - t0), col, a.dv, a.vec, lane);
                }
            }
#pragma unroll
            for (int nt = 0; nt < 8; ++nt) {
                const float2 left = factor(1, nt * 8 + q2);
#pragma unroll
                for (int e = 0; e < 4; ++e) u[nt][e] *= e & 1 ? left.y : left.x;
            }
            const Scale ls = scale_of(u);
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) split_left(u[2 * kt], u[2 * kt + 1], ls.by, fh[kt], fl[kt]);
            update(fh, fl, ls.back, sk, true);
        } else {
            // y = P^T dO (this warp's share of the rows);  R <- c(C, 0) R + scale Q^T c(i, 0) dO
            Frag g[4];
            float m = 0.0f, mp = 0.0f;
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                ldm_t(g[kt], sx + kt * 16 * Sh::kPitch);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 past = factor(3, kt * 16 + (i >> 1) * 8 + q2);
                    const float g0 = fabsf(low(g[kt][i])), g1 = fabsf(high(g[kt][i]));
                    m = fmaxf(m, fmaxf(g0, g1));
                    mp = fmaxf(mp, fmaxf(g0 * fabsf(past.x), g1 * fabsf(past.y)));
                }
            }
            const Scale gs = scale_of(warp_max(m)), ps = scale_of(warp_max(mp));
            __half *const go = a.Gp + at * a.dvp * C;  // dO's plane
            if (lane == 0) scales_of(chunk)[6] = gs.back;
            room();
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                Frag gf;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 past = factor(3, kt * 16 + (i >> 1) * 8 + q2);
                    const float g0 = low(g[kt][i]), g1 = high(g[kt][i]);
                    gf[i] = pack(gs.by * g0, gs.by * g1);
                    split(ps.by * (past.x * g0), ps.by * (past.y * g1), fh[kt][i], fl[kt][i]);
                }
                if (own(kt)) put(go, kt * 16, gf);
                if (SP == 2 && (kt == 0 || kt == 3) != (part == 0)) continue;  // five of the ten blocks each
#pragma unroll
                for (int np = 0; np <= kt; ++np) {
                    Frag f;
                    right_k(f, sP, C, kt * 16, np * 16, lane);
                    mma(y[2 * np], gf, f[0], f[1]);
                    mma(y[2 * np + 1], gf, f[2], f[3]);
                    right_k(f, sP + kTileB, C, kt * 16, np * 16, lane);
                    mma(y[2 * np], gf, f[0], f[1]);
                    mma(y[2 * np + 1], gf, f[2], f[3]);
                }
            }
            send(go, 1);
            // x = c(C, j) K R + P^T dO
            const float back = gs.back * back_P;
#pragma unroll
            for (int nt = 0; nt < 8; ++nt) {
                const float2 left = factor(1, nt * 8 + q2);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[nt][e] = fmaf(ss.back * (e & 1 ? left.y : left.x), x[nt][e], back * y[nt][e]);
            }
            if (SP == 2) exchange(x, y, false);
            update(fh, fl, ps.back, sq, true);
            zero(y);
            // X = T^T x
            const Scale xs = scale_of(x);
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                Frag hi, lo;
                split_left(x[2 * kt], x[2 * kt + 1], xs.by, hi, lo);
#pragma unroll
                for (int np = 0; np <= kt; ++np) {
                    Frag f;
                    right_n(f, sT, C, np * 16, kt * 16, lane);
                    mma(y[2 * np], hi, f[0], f[1]);
                    mma(y[2 * np + 1], hi, f[2], f[3]);
                    mma(y[2 * np], lo, f[0], f[1]);
                    mma(y[2 * np + 1], lo, f[2], f[3]);
                    right_n(f, sT + kTileB, C, np * 16, kt * 16, lane);
                    mma(y[2 * np], hi, f[0], f[1]);
                    mma(y[2 * np + 1], hi, f[2], f[3]);
                }
            }
            // X's plane;  dV = b X;  R <- R - K^T b c(i, 0) X
            const float back_x = xs.back * back_T;
#pragma unroll
            for (int nt = 0; nt < 8; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[nt][e] *= back_x;
            const Scale us = scale_of(y);
            if (lane == 0) scales_of(chunk)[5] = us.back;
            room();
            __half *const kept = a.Xp + at * a.dvp * C;
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                if (!own(kt)) continue;
                const Frag hi = {pack(us.by * y[2 * kt][0], us.by * y[2 * kt][1]), pack(us.by * y[2 * kt][2], us.by * y[2 * kt][3]),
                                 pack(us.by * y[2 * kt + 1][0], us.by * y[2 * kt + 1][1]), pack(us.by * y[2 * kt + 1][2], us.by * y[2 * kt + 1][3])};
                put(kept, kt * 16, hi);
            }
            send(kept, 1);
#pragma unroll
            for (int nt = 0; nt < 8; ++nt) {
                const float2 past = factor(0, nt * 8 + q2), beta = factor(2, nt * 8 + q2);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[nt][e] *= e & 1 ? beta.y : beta.x;
                    x[nt][e] = -(e & 1 ? past.y : past.x) * y[nt][e];
                }
            }
            const Scale ws = scale_of(x);
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) split_left(x[2 * kt], x[2 * kt + 1], ws.by, fh[kt], fl[kt]);
            update(fh, fl, ws.back, sk, false);
            chain_store(y, first, some, sm.out[warp], o + t0 * a.ot, a.ot, min(C, len - t0), col, a.dv, a.vec, lane);
        }
    }
    if (REV && mine && chunks > 0) {  // R before the first chunk
        const Scale ss = scale_of(S);
        keep_scale(0, ss.back);
        room();
        __half *tile = a.Rp + bh * (a.m + 1) * a.dvp * DP;
#pragma unroll
        for (int kt = 0; kt < ND / 2; ++kt) {
            Frag hi, lo;
            split_left(S[2 * kt], S[2 * kt + 1], ss.by, hi, lo);
            put(tile, d0 + kt * 16, hi);
        }
        send(tile, DP / 64);
    }
    if (lane == 0) bulk_wait();  // (shared memory is read to the end)
    float *last = REV ? a.dS0 : a.S1;
    if (last)
#pragma unroll
        for (int nt = 0; nt < ND; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                int64_t at;
                if (place(nt, e, at)) last[at] = S[nt][e];
            }
    if (MODE != kKeep)  // rows behind the end, eight columns at a time
        for (int64_t i = tid; i < (int64_t)(a.n - len) * NG * 2; i += Sh::kWarps * 32) {
            const int c = col0 + (int)(i % (NG * 2)) * 8;
            __nv_bfloat16 *to = o + (len + i / (NG * 2)) * a.ot + c;
            if (a.vec && c < a.dv)
                *reinterpret_cast<uint4 *>(to) = make_uint4(0, 0, 0, 0);
            else
                for (int e = 0; e < min(8, a.dv - c); ++e) io_store(to + e, 0.0f);
        }
}

// ---------------------------------------------------------------------------
// Gradients of q, k and the gates (luna_delta.cuh) from the chunk's U, X, dO and states.  A block of eight warps a chunk:
// two groups of 32 rows by four quarters of the columns.  102 KB of shared memory, so that two blocks are on an SM and
// the one's products cover the other's loads: R, then S, then Q lie in the same place, P and W in that of U.

constexpr int kGradThreads = 256, kParts = 4;

template <int DP, int DVT>
struct GradShared {
    alignas(128) char k[DP / 64][kTileB], go[DVT * 128], x[DVT * 128], u[DVT * 128 > 2 * kTileB ? DVT * 128 : 2 * kTileB];
    alignas(128) char s[DVT * DP * 2 > DP / 64 * kTileB ? DVT * DP * 2 : DP / 64 * kTileB];
    uint64_t bar[4];
    float hi[C], lo[C], past[C], left[C], b[C], scales[DVT / 16][kDeltaScales], behind[DVT / 16][2];  // (behind: of R)
    __half2 steps[8][DVT / 16];  // of the products over columns: 16 columns' scale over the largest, that
    float all[8], total[kGradThreads / 32];
    float sums[6][kParts][C];  // of a row's quarters: q . dQ, k . Z without the rows' part, k . (dK), W . K K^T, x . v, b k . Z
    float most[2][kGradThreads / 32], read[C], wrote[C];
};

__device__ __forceinline__ float inverse2(float back) {  // of a power of two
    return __uint_as_float((254u << 23) - __float_as_uint(back));
}

template <int DP, int DVT, typename OUT>
__global__ void __launch_bounds__(kGradThreads, 2) k_delta_grad_tc(DeltaArgs a) {
    using Sh = GradShared<DP, DVT>;
    using Acc = float[2][DP / 32][4];
    extern __shared__ __align__(128) char raw[];
    Sh &sm = *reinterpret_cast<Sh *>(raw);
    constexpr int NT = DP / 32;  // n-tiles of a warp's quarter of the columns of dQ, dK
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, r0 = warp % 2 * 32, quarter = warp / 2, q2 = lane % 4 * 2;
    const int of_half = 2 + quarter / 2 * 3;  // the products with S and R of the warp's half of the columns
    const int64_t at = blockIdx.x, bh = at / a.m;
    const int chunk = (int)(at % a.m), b = (int)(bh / a.H), h = (int)(bh % a.H), t0 = chunk * C;
    const int rows = max(0, min(C, head_length(a.lengths, b, a.n) - t0)), out_rows = min(C, a.n - t0);
    const int hk = h / (a.H / a.k.heads);
    OUT *dq = static_cast<OUT *>(a.dq) + b * a.dqb + h * a.dqh + t0 * a.dqt;
    OUT *dk = static_cast<OUT *>(a.dk) + b * a.dkb + h * a.dkh + t0 * a.dkt;
    __nv_bfloat16 *dg = static_cast<__nv_bfloat16 *>(a.dg.p) + b * a.dg.sb + h * a.dg.sh + t0 * a.dg.st;
    __nv_bfloat16 *db = static_cast<__nv_bfloat16 *>(a.db.p) + b * a.db.sb + h * a.db.sh + t0 * a.db.st;
    for (int i = tid; i < (out_rows - rows) * a.d; i += kGradThreads) {
        const int t = rows + i / a.d, c = i % a.d;
        io_store(dq + t * a.dqt + c, 0.0f);
        io_store(dk + t * a.dkt + c, 0.0f);
    }
    if (tid >= rows && tid < out_rows) {
        io_store(dg + tid * a.dg.st, 0.0f);
        io_store(db + tid * a.db.st, 0.0f);
    }
    if (rows == 0) return;

    const uint32_t sk = smem_u32(sm.k), sgo = smem_u32(sm.go), su = smem_u32(sm.u), sx = smem_u32(sm.x), ss = smem_u32(sm.s);
    const uint32_t sP = su, sW = su + kTileB;
    const int dvp = a.dvp, groups = dvp / 16;
    const int64_t kat = ((int64_t)b * a.k.heads + hk) * a.m + chunk;
    const int64_t slot = bh * (a.m + 1) + chunk;
    const uint32_t of_rows = dvp * C * 2, of_state = dvp * DP * 2;
    if (tid < 4) mbar_init(&sm.bar[tid], 1);
    fence_mbar_init();
    __syncthreads();
    auto load_state = [&](const void *src, uint32_t bytes, int which) {  // (one thread)
        mbar_arrive_expect_tx(&sm.bar[which], bytes);
        load_tile(sm.s, src, bytes, &sm.bar[which]);
    };
    if (tid == 0) {
        mbar_arrive_expect_tx(&sm.bar[0], sizeof(sm.k) + 3 * of_rows);
        load_tile(sm.u, a.Up + at * dvp * C, of_rows, &sm.bar[0]);
        load_tile(sm.x, a.Xp + at * dvp * C, of_rows, &sm.bar[0]);
        load_tile(sm.go, a.Gp + at * dvp * C, of_rows, &sm.bar[0]);
        load_tile(sm.k, a.Kp + kat * C * DP, sizeof(sm.k), &sm.bar[0]);
        load_state(a.Rp + (slot + 1) * dvp * DP, of_state, 1);
        // what comes later, as far as L2
        auto ask = [](const void *p, uint32_t bytes) {
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
        };
        ask(a.Sp + at * dvp * DP, of_state);
        ask(a.Rp + slot * dvp * DP, of_state);
        ask(a.Qp + kat * C * DP, sizeof(sm.k));
    }
    const float *rowf = a.rows + at * kRowsF;
    const float back_k = rowf[4 * C + 4], back_q = rowf[4 * C + 5];
    if (warp == 0)
        delta_gate_sums(lane, [&](int t) { return t < rows ? gate_at<__nv_bfloat16>(a.g, b, h, t0 + t) : 0.0f; }, sm.hi, sm.lo,
                        sm.past, sm.left);
    else if (warp < 3)
        sm.b[tid - 32] = rowf[2 * C + tid - 32];
    for (int i = tid; i < groups * kDeltaScales; i += kGradThreads) (&sm.scales[0][0])[i] = a.scales[slot * groups * kDeltaScales + i];
    if (tid < groups * 2) sm.behind[tid / 2][tid % 2] = a.scales[((slot + 1) * groups + tid / 2) * kDeltaScales + 2 + tid % 2];
    __syncthreads();
    // What is summed over the columns has a scale of its own every 16 of them: the left operand takes the ratio to the
    // largest of them (at most 1, and what it loses is small beside that).  Products: dO U, X U; of either half of the
    // other columns dO S, X S, U R.
    if (tid < 8) {
        const int side = tid < 2 ? 0 : (tid - 2) / 3, which = tid < 2 ? tid : (tid - 2) % 3;
        auto scale = [&](int kt) {
            const float *f = sm.scales[kt];
            return tid < 2 ? f[6 - which] * f[4] : which < 2 ? f[6 - which] * f[side] : f[4] * sm.behind[kt][side];
        };
        float most = 0.0f;
        for (int kt = 0; kt < groups; ++kt) most = fmaxf(most, scale(kt));
        sm.all[tid] = most;
        for (int kt = 0; kt < groups; ++kt) sm.steps[tid][kt] = __float2half2_rn(most > 0.0f ? scale(kt) / most : 0.0f);
    }
    // x . v: a thread a row and a quarter of the columns, while the tiles come
    float xv = 0.0f;
    bool here = mbar_wait_long(&sm.bar[0], 0);
    __syncthreads();
    {
        const int i = tid % C;
        const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(a.v.p) + b * a.v.sb + h * a.v.sh + (t0 + i) * a.v.st;
        if (i < rows)
            for (int c8 = tid / C; c8 * 8 < a.dv; c8 += kParts) {
                uint32_t w[4];
                if (a.vec) {
                    const uint4 w4 = *reinterpret_cast<const uint4 *>(v + c8 * 8);
                    w[0] = w4.x; w[1] = w4.y; w[2] = w4.z; w[3] = w4.w;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 f = load_pair(v + c8 * 8 + 2 * e, a.dv - c8 * 8 - 2 * e, false);
                        w[e] = pack_bf16(f.x, f.y);
                    }
                }
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    unsigned short u;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(u) : "r"(tile_at(sx, dvp, c8 * 8 + e, i >> 3) + (i & 7) * 2));
                    sum = fmaf(e & 1 ? high(w[e / 2]) : low(w[e / 2]), __half2float(__ushort_as_half(u)), sum);
                }
                xv = fmaf(sm.scales[c8 / 2][5], sum, xv);
            }
        sm.sums[4][tid / C][i] = xv;
    }

    // 16 rows (m0) of a left operand from a plane, for the product's 16 columns kt
    auto left_plane = [&](Frag &f, uint32_t tile, int m0, int kt, int product) {
        left_k(f, tile, dvp, kt * 16, m0, lane);
        const __half2 by = sm.steps[product][kt];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __half2 x;
            memcpy(&x, &f[i], 4);
            x = __hmul2(x, by);
            memcpy(&f[i], &x, 4);
        }
    };
    // sums over the four lanes of a row, for this quarter of the columns: rows r0 + 16 mt + lane / 4 and 8 more
    auto row_sums = [&](float x, float y, int mt, int which) {
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        y += __shfl_xor_sync(0xffffffffu, y, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        y += __shfl_xor_sync(0xffffffffu, y, 2);
        if (lane % 4 == 0) {
            sm.sums[which][quarter][r0 + mt * 16 + lane / 4] = x;
            sm.sums[which][quarter][r0 + mt * 16 + lane / 4 + 8] = y;
        }
    };
    const int c0 = quarter * (DP / 4), n0 = quarter * 16;  // first column of the warp's, of P and W
    // acc += F M over the columns of the state: F a plane, M the tile of the state
    auto over_columns = [&](Acc &acc, uint32_t plane, int product) {
#pragma unroll 2
        for (int kt = 0; kt < groups; ++kt) {
            Frag fl[2];
            left_plane(fl[0], plane, r0, kt, product);
            left_plane(fl[1], plane, r0 + 16, kt, product);
#pragma unroll
            for (int np = 0; np < NT / 2; ++np) {
                Frag f;
                right_k(f, ss, dvp, kt * 16, c0 + np * 16, lane);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    mma(acc[mt][2 * np], fl[mt], f[0], f[1]);
                    mma(acc[mt][2 * np + 1], fl[mt], f[2], f[3]);
                }
            }
        }
    };
    // acc += F M over the 64 rows of the chunk: F from P or W (trans: its transpose), M a tile of K or Q
    auto over_rows = [&](Acc &acc, uint32_t from, bool trans, uint32_t tile, uint32_t sign) {
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            if (trans ? kt * 16 < r0 : kt * 16 > r0 + 16) continue;
            Frag fl[2];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                if (trans)
                    left_k(fl[mt], from, C, kt * 16, r0 + mt * 16, lane);
                else
                    left_m(fl[mt], from, C, r0 + mt * 16, kt * 16, lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) fl[mt][i] ^= sign;
            }
#pragma unroll
            for (int np = 0; np < NT / 2; ++np) {
                Frag f;
                right_k(f, tile, C, kt * 16, c0 + np * 16, lane);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    mma(acc[mt][2 * np], fl[mt], f[0], f[1]);
                    mma(acc[mt][2 * np + 1], fl[mt], f[2], f[3]);
                }
            }
        }
    };
    // acc *= by row_factor (of every row)
    auto times_rows = [&](Acc &acc, const float *row_factor, const float *more, float by) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            const int ra = r0 + mt * 16 + lane / 4;
            float fa = by * row_factor[ra], fb = by * row_factor[ra + 8];
            if (more) {
                fa *= more[ra];
                fb *= more[ra + 8];
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[mt][nt][e] *= e & 2 ? fb : fa;
        }
    };
    auto times = [&](Acc &acc, float by) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[mt][nt][e] *= by;
    };
    // sums of the rows times those of K (whose left operands lie as the accumulators do)
    auto dot_k = [&](const Acc &acc, int which) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            float x = 0.0f, y = 0.0f;
#pragma unroll
            for (int np = 0; np < NT / 2; ++np) {
                Frag f;
                left_m(f, sk, C, r0 + mt * 16, c0 + np * 16, lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 k2 = half_pair(f[i]);
                    const float *c = acc[mt][2 * np + i / 2] + (i & 1) * 2;
                    float &to = i & 1 ? y : x;
                    to = fmaf(k2.x, c[0], fmaf(k2.y, c[1], to));
                }
            }
            row_sums(back_k * x, back_k * y, mt, which);
        }
    };
    auto store_rows = [&](const Acc &acc, OUT *out, int64_t st) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = r0 + mt * 16 + lane / 4 + i * 8;
                if (r >= rows) continue;
                OUT *to = out + r * st + c0 + q2;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int left = a.d - (c0 + nt * 8 + q2);  // (an odd width ends inside a pair)
                    if (left <= 0) continue;
                    if (!a.vec) {
                        io_store(to + nt * 8, acc[mt][nt][2 * i]);
                        if (left > 1) io_store(to + nt * 8 + 1, acc[mt][nt][2 * i + 1]);
                    } else if (sizeof(OUT) == 2) {
                        *reinterpret_cast<uint32_t *>(to + nt * 8) = pack_bf16(acc[mt][nt][2 * i], acc[mt][nt][2 * i + 1]);
                    } else {
                        *reinterpret_cast<float2 *>(to + nt * 8) = make_float2(acc[mt][nt][2 * i], acc[mt][nt][2 * i + 1]);
                    }
                }
            }
    };
    auto clear = [&](Acc &acc) {
        zero(acc[0]);
        zero(acc[1]);
    };

    // P_ij = scale c(i, j) dO_i . u_j,  W_ij = b_i c(i, j) x_i . u_j, 16 columns a warp; W . K K^T for db
    float p[2][2][4], w[2][2][4];
    float mp = 0.0f, mw = 0.0f;
    {
        float kk[2][2][4];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            zero(p[mt]);
            zero(w[mt]);
            zero(kk[mt]);
        }
        if (n0 <= r0 + 16) {
#pragma unroll 2
            for (int kt = 0; kt < groups; ++kt) {
                Frag f;
                right_k(f, su, dvp, kt * 16, n0, lane);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    Frag fg, fx;
                    left_plane(fg, sgo, r0 + mt * 16, kt, 0);
                    left_plane(fx, sx, r0 + mt * 16, kt, 1);
                    mma(p[mt][0], fg, f[0], f[1]);
                    mma(p[mt][1], fg, f[2], f[3]);
                    mma(w[mt][0], fx, f[0], f[1]);
                    mma(w[mt][1], fx, f[2], f[3]);
                }
            }
#pragma unroll
            for (int k0 = 0; k0 < DP; k0 += 16) {
                Frag f;
                right_n(f, sk, C, n0, k0, lane);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    Frag fk;
                    left_m(fk, sk, C, r0 + mt * 16, k0, lane);
                    mma(kk[mt][0], fk, f[0], f[1]);
                    mma(kk[mt][1], fk, f[2], f[3]);
                }
            }
        }
        const float by_p = a.scale * sm.all[0], by_w = sm.all[1];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            float dot[2] = {0.0f, 0.0f};
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = r0 + mt * 16 + lane / 4 + (e >> 1) * 8, j = n0 + nt * 8 + q2 + (e & 1);
                    const float c = j <= i ? expf((sm.hi[i] - sm.hi[j]) + (sm.lo[i] - sm.lo[j])) : 0.0f;
                    float &pp = p[mt][nt][e], &ww = w[mt][nt][e];
                    pp = j <= i ? by_p * c * pp : 0.0f;
                    ww = j < i ? by_w * c * ww : 0.0f;
                    if (j < i) dot[e >> 1] = fmaf(ww, kk[mt][nt][e], dot[e >> 1]);
                    ww *= sm.b[i];
                    mp = fmaxf(mp, fabsf(pp));
                    mw = fmaxf(mw, fabsf(ww));
                }
            row_sums(dot[0], dot[1], mt, 3);
        }
        mp = warp_max(mp);
        mw = warp_max(mw);
        if (lane == 0) {
            sm.most[0][warp] = mp;
            sm.most[1][warp] = mw;
        }
    }
    // what dK takes from R
    Acc acc, z;
    clear(acc);
    here = mbar_wait_long(&sm.bar[1], 0) && here;
    if (here) over_columns(acc, su, of_half + 2);
    if (__syncthreads_or(!here)) {  // a copy that did not arrive within a second: give up
        if (tid == 0) {
            atomicOr(a.status, 1);
            for (int i = 0; i < 2; ++i) mbar_wait(&sm.bar[i], 0, kDrainNs);
        }
        return;
    }
    if (tid == 0) load_state(a.Sp + at * dvp * DP, of_state, 2);
    mp = mw = 0.0f;
#pragma unroll
    for (int i = 0; i < kGradThreads / 32; ++i) {
        mp = fmaxf(mp, sm.most[0][i]);
        mw = fmaxf(mw, sm.most[1][i]);
    }
    // P Q and W K are scaled down alike, so that they add up in dK
    const float by = fmaxf(fmaxf(scale_of(mp).back * back_q, scale_of(mw).back * back_k), 0x1p-100f), inv = inverse2(by);
    const float to_p = back_q * inv, to_w = back_k * inv, by_pk = by * back_k * inverse2(back_q);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const uint32_t to = tile_at(0, C, r0 + mt * 16 + lane / 4 + e * 4, quarter * 2 + nt) + q2 * 2;
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(sP + to), "r"(pack(to_p * p[mt][nt][e], to_p * p[mt][nt][e + 1])) : "memory");
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(sW + to), "r"(pack(to_w * w[mt][nt][e], to_w * w[mt][nt][e + 1])) : "memory");
            }
    times_rows(acc, sm.left, nullptr, sm.all[of_half + 2] * inv);
    __syncthreads();
    over_rows(acc, sW, true, sk, 0x80008000u);

    // dQ and Z from S
    here = mbar_wait_long(&sm.bar[2], 0);
    clear(z);
    if (here) over_columns(z, sgo, of_half);
    times_rows(z, sm.past, nullptr, a.scale * sm.all[of_half] * inverse2(by_pk));
    over_rows(z, sP, false, sk, 0);
    times(z, by_pk);
    store_rows(z, dq, a.dqt);
    {  // q . dQ, with Q as it came
        const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(a.q.p) + b * a.q.sb + hk * a.q.sh + t0 * a.q.st + c0 + q2;
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            float dot[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = r0 + mt * 16 + lane / 4 + i * 8;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float2 f = load_pair(q + r * a.q.st + nt * 8, r < rows ? a.d - (c0 + nt * 8 + q2) : 0, a.vec);
                    dot[i] = fmaf(f.x, z[mt][nt][2 * i], fmaf(f.y, z[mt][nt][2 * i + 1], dot[i]));
                }
            }
            row_sums(dot[0], dot[1], mt, 0);
        }
    }
    {  // <S, R> before the chunk: of every 16 columns the diagonal of S^T R, R as it lies in memory (in both the summed
       // values lie in the same, permuted order: a lane's 16 bytes of a row are those of two products)
        float sum = 0.0f;
        if (here && warp < groups) {
            const char *r = reinterpret_cast<const char *>(a.Rp + slot * dvp * DP);
            const int ra = warp * 16 + lane / 4;
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                float c[2][4];
                zero(c);
#pragma unroll
                for (int i = 0; i < DP / 64; ++i) {
                    const int piece = (side * (DP / 64) + i) * 4 + lane % 4;
                    const uint32_t at0 = tile_at(0, dvp, ra, piece), at1 = tile_at(0, dvp, ra + 8, piece);
                    const uint4 s0 = *reinterpret_cast<const uint4 *>(sm.s + at0), s1 = *reinterpret_cast<const uint4 *>(sm.s + at1);
                    const uint4 r0_ = *reinterpret_cast<const uint4 *>(r + at0), r1 = *reinterpret_cast<const uint4 *>(r + at1);
                    const Frag f = {s0.x, s1.x, s0.y, s1.y}, g = {s0.z, s1.z, s0.w, s1.w};
                    mma(c[0], f, r0_.x, r0_.y);
                    mma(c[0], g, r0_.z, r0_.w);
                    mma(c[1], f, r1.x, r1.y);
                    mma(c[1], g, r1.z, r1.w);
                }
                const float *scale = sm.scales[warp];
                float diag = 0.0f;
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (lane / 4 == q2 + e) diag += c[0][e] + c[1][2 + e];
                sum = fmaf(scale[side] * scale[2 + side], diag, sum);
            }
        }
        sum = sum + __shfl_xor_sync(0xffffffffu, sum, 16);
#pragma unroll
        for (int w = 8; w > 0; w /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        if (lane == 0) sm.total[warp] = sum;
    }
    clear(z);
    if (here) over_columns(z, sx, of_half + 1);
    if (__syncthreads_or(!here)) {
        if (tid == 0) {
            atomicOr(a.status, 1);
            mbar_wait(&sm.bar[2], 0, kDrainNs);
        }
        return;
    }
    if (tid == 0) load_state(a.Qp + kat * C * DP, sizeof(sm.k), 3);
    times_rows(z, sm.past, nullptr, sm.all[of_half + 1]);
    dot_k(z, 1);
    times_rows(z, sm.b, nullptr, inv);
    over_rows(z, sW, false, sk, 0);
    times(z, by);
    dot_k(z, 5);

    // dK
    here = mbar_wait_long(&sm.bar[3], 0);
    if (here) over_rows(acc, sP, true, ss, 0);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[mt][nt][e] = fmaf(by, acc[mt][nt][e], -z[mt][nt][e]);
    dot_k(acc, 2);
    store_rows(acc, dk, a.dkt);
    if (__syncthreads_or(!here)) {
        if (tid == 0) {
            atomicOr(a.status, 1);
            mbar_wait(&sm.bar[3], 0, kDrainNs);
        }
        return;
    }
    if (tid < rows) {
        auto sum = [&](int which) {
            return (sm.sums[which][0][tid] + sm.sums[which][1][tid]) + (sm.sums[which][2][tid] + sm.sums[which][3][tid]);
        };
        const float bz = sum(5);
        io_store(db + tid * a.db.st, sum(4) - sum(1) - back_k * back_k * sum(3));
        sm.read[tid] = sum(0) - bz;
        sm.wrote[tid] = sum(2) + bz;
    }
    __syncthreads();
    if (warp == 0) {
        float base = 0.0f;
        for (int w = 0; w < kGradThreads / 32; ++w) base += sm.total[w];
        delta_gate_grads(base, sm.read, sm.wrote, rows, lane, [&](int t, float x) {
            io_store(dg + t * a.dg.st, expf(gate_at<__nv_bfloat16>(a.g, b, h, t0 + t)) == 0.0f ? 0.0f : x);
        });
    }
}

unsigned cdiv(int64_t a, int64_t b) { return (unsigned)((a + b - 1) / b); }

template <int DP, bool TERMS>
cudaError_t prepare(const DeltaArgs &a, cudaStream_t s) {
    cudaError_t e = cudaFuncSetAttribute(k_delta_prepare<DP, TERMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PrepShared<DP>));
    if (e != cudaSuccess) return e;
    LUNA_LAUNCH("delta_prepare", (k_delta_prepare<DP, TERMS>), (unsigned)((int64_t)a.B * a.H * a.m), kPrepThreads, sizeof(PrepShared<DP>), s, a);
    return cudaGetLastError();
}

template <int DP, int NG, int SP, ChainMode MODE>
cudaError_t chain_launch(const DeltaArgs &a, cudaStream_t s) {
    using Sh = ChainShared<DP, NG, SP, MODE>;
    cudaError_t e = cudaFuncSetAttribute(k_delta_chain<DP, NG, SP, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Sh));
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)(a.B * a.H), cdiv(a.dv, NG * 16));
    LUNA_LAUNCH("delta_chain", (k_delta_chain<DP, NG, SP, MODE>), grid, NG * SP * 32, sizeof(Sh), s, a);
    return cudaGetLastError();
}

// With few heads, few columns a block and two warps for 16 of them, so that the chains spread over the SMs.
template <int DP, ChainMode MODE>
cudaError_t chain(const DeltaArgs &a, cudaStream_t s) {
    const int64_t bh = (int64_t)a.B * a.H, sms = tc_sm_count();
    if (a.dv > 64 && bh * cdiv(a.dv, 64) > sms) return chain_launch<DP, 8, 1, MODE>(a, s);
    if (a.dv > 32 && bh * cdiv(a.dv, 32) > sms) return chain_launch<DP, 4, 1, MODE>(a, s);
    return chain_launch<DP, 2, 2, MODE>(a, s);
}

}  // namespace

template <int DP, int DVT, typename OUT>
static cudaError_t grad_launch(const DeltaArgs &a, cudaStream_t s) {
    using Sh = GradShared<DP, DVT>;
    cudaError_t e = cudaFuncSetAttribute(k_delta_grad_tc<DP, DVT, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Sh));
    if (e != cudaSuccess) return e;
    LUNA_LAUNCH("delta_grad_tc", (k_delta_grad_tc<DP, DVT, OUT>), (unsigned)((int64_t)a.B * a.H * a.m), kGradThreads, sizeof(Sh), s, a);
    return cudaGetLastError();
}

template <typename OUT>
static cudaError_t grad(const DeltaArgs &a, cudaStream_t s) {
    if (a.d <= 64) return a.dv <= 64 ? grad_launch<64, 64, OUT>(a, s) : grad_launch<64, 128, OUT>(a, s);
    return a.dv <= 64 ? grad_launch<128, 64, OUT>(a, s) : grad_launch<128, 128, OUT>(a, s);
}

cudaError_t launch_delta_grad_tc(const DeltaArgs &a, luna_dtype out, cudaStream_t s) {
    return out == LUNA_F32 ? grad<float>(a, s) : grad<__nv_bfloat16>(a, s);
}

cudaError_t launch_delta_prepare(const DeltaArgs &a, cudaStream_t s) {
    if (a.d <= 64) return a.planes == 2 ? prepare<64, true>(a, s) : prepare<64, false>(a, s);
    return a.planes == 2 ? prepare<128, true>(a, s) : prepare<128, false>(a, s);
}

cudaError_t launch_delta_chain(const DeltaArgs &a, bool reverse, cudaStream_t s) {
    if (a.d <= 64) return reverse ? chain<64, kReverse>(a, s) : a.Up ? chain<64, kKeep>(a, s) : chain<64, kOutputs>(a, s);
    return reverse ? chain<128, kReverse>(a, s) : a.Up ? chain<128, kKeep>(a, s) : chain<128, kOutputs>(a, s);
}

}  // namespace luna
