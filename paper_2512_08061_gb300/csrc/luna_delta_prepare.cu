// The gated delta rule on tensor cores: what each chunk's rows are to each other.
#include "luna_delta_tc.cuh"

namespace luna {
namespace {

using namespace delta;

// ---------------------------------------------------------------------------
// T, P and the factors of every chunk.  A block of four warps a chunk, a warp 16 rows of K K^T and Q K^T.  The inverse
// of the diagonal blocks of 16 rows is taken by substitution in fp32, a lane a column; a warp then goes down one block
// column of T, transposed so that each product's accumulators are the next one's left operand:
//
//     T_IJ^T = -(sum_{J <= K < I} T_KJ^T A_IK^T) T_II^T
//
// with both operands in two terms.  It leaves T^T, P and in a chunk's factors: c(i, 0) 2^ek, c(C, i) 2^ek, b,
// scale c(i, 0) 2^eq of its rows, then c(C, 0) in two terms and what T, P, K and Q were scaled down by (the last two
// are 2^ek and 2^eq), the largest of c(C, i) 2^ek, of c(i, 0) 2^ek b, of scale c(i, 0) 2^eq, and the sums of the gates
// in two terms.  157 us for 8192 chunks of 128 columns, 89 KB in and out each (4.6 TB/s); bound by
// its stages between barriers, four blocks an SM.  (With the inverse in fp32 by all threads, 13 barriers, 68 KB of shared
// memory and tiles stored from the registers: 248 us.)

constexpr int kPrepThreads = 128;

template <int DP>
struct PrepShared {
    alignas(128) char k[DP / 64][kTileB], q[DP / 64][kTileB], A[2][kTileB];  // A: two planes; T_II in its diagonal blocks
    alignas(16) float diag[4][16][20];
    float hi[C], lo[C], past[C], left[C], b[C], tail[C], most[5][kPrepThreads / 32], back_T[4];  // tail: c(last of its 16, j)
};

// A thread's 16-byte pieces of a bf16 tile, as they lie in memory: their largest value (prep_most), and they themselves in
// fp16 to `out` (prep_write)
template <int DP>
__device__ __forceinline__ float prep_most(const char *tile, int tid) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < C * DP / 8 / kPrepThreads; ++i) {
        const uint4 w = *reinterpret_cast<const uint4 *>(tile + (tid + i * kPrepThreads) * 16);
        most = __vmaxu2(most, __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu)));
    }
    return __uint_as_float(max(most << 16, most & 0x7fff0000u));
}
template <int DP>
__device__ __forceinline__ void prep_write(const char *tile, float by, __half *out, int tid) {
#pragma unroll
    for (int i = 0; i < C * DP / 8 / kPrepThreads; ++i) {
        const uint4 w = *reinterpret_cast<const uint4 *>(tile + (tid + i * kPrepThreads) * 16);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
        uint32_t f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = pack(by * low(u[e]), by * high(u[e]));
        reinterpret_cast<uint4 *>(out)[tid + i * kPrepThreads] = make_uint4(f[0], f[1], f[2], f[3]);
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
    most_of(2, prep_most<DP>(sm.k[0], tid));
    most_of(3, prep_most<DP>(sm.q[0], tid));
    if (tid < C) sm.tail[tid] = expf((sm.hi[tid | 15] - sm.hi[tid]) + (sm.lo[tid | 15] - sm.lo[tid]));
    __syncthreads();

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
    // c(i, j): in the diagonal block of the gates' sums themselves, before it by way of the last row of j's 16
    float most_p = 0.0f, most_a = 0.0f, row_factor[3][2];
#pragma unroll
    for (int J = 0; J < 3; ++J)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int i = r0 + lane / 4 + e * 8, end = J * 16 + 15;
            row_factor[J][e] = J < warp ? expf((sm.hi[i] - sm.hi[end]) + (sm.lo[i] - sm.lo[end])) : 0.0f;
        }
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) {
        if (nt / 2 > warp) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = r0 + lane / 4 + (e >> 1) * 8, j = nt * 8 + q2 + (e & 1);
            float c = 0.0f;
            if (nt / 2 < warp)
                c = row_factor[nt / 2 < 3 ? nt / 2 : 0][e >> 1] * sm.tail[j];
            else if (j <= i)
                c = expf((sm.hi[i] - sm.hi[j]) + (sm.lo[i] - sm.lo[j]));
            qk[nt][e] = j <= i ? a.scale * c * qk[nt][e] : 0.0f;
            kk[nt][e] = j < i ? sm.b[i] * c * kk[nt][e] : 0.0f;
            most_p = fmaxf(most_p, fabsf(qk[nt][e]));
            most_a = fmaxf(most_a, fabsf(kk[nt][e]));
            if (nt / 2 == warp) sm.diag[warp][i - r0][j - r0] = kk[nt][e];
        }
    }
    most_of(0, most_p);
    most_of(1, most_a);
    __syncthreads();
    const Scale ps = block_scale(0), as = block_scale(1), ks = block_scale(2), qs = block_scale(3);
    if (h % (a.H / a.k.heads) == 0) {  // one head of those that share queries and keys
        const int64_t to = ((int64_t)b * a.k.heads + hk) * a.m + chunk;
        prep_write<DP>(sm.k[0], ks.by, a.Kp + to * C * DP, tid);
        prep_write<DP>(sm.q[0], qs.by, a.Qp + to * C * DP, tid);
    }
    float *rowf = a.rows + at * kRowsF;
    if (tid < C) {
        rowf[tid] = sm.past[tid] * ks.back;
        rowf[C + tid] = sm.left[tid] * ks.back;
        rowf[2 * C + tid] = sm.b[tid];
        rowf[3 * C + tid] = a.scale * sm.past[tid] * qs.back;
        rowf[4 * C + 12 + tid] = sm.hi[tid];
        rowf[5 * C + 12 + tid] = sm.lo[tid];
    }
    if (tid == 0) {
        gate_terms(sm.hi[C - 1], rowf[4 * C], rowf[4 * C + 1]);
        rowf[4 * C + 3] = ps.back;
        rowf[4 * C + 4] = ks.back;
        rowf[4 * C + 5] = qs.back;
    }
    Frag ph[4], pl[4];  // P of the warp's rows
#pragma unroll
    for (int np = 0; np < 4; ++np) {
#pragma unroll
        for (int i = 0; i < 4; ++i) ph[np][i] = pl[np][i] = 0;
        if (np > warp) continue;
        split_left(qk[2 * np], qk[2 * np + 1], ps.by, ph[np], pl[np]);
        if (np == warp) continue;  // (its diagonal block waits for T_II)
        Frag hi, lo;
        split_left(kk[2 * np], kk[2 * np + 1], as.by, hi, lo);
        tile_put(sA, C, r0, np * 16, hi, lane);
        tile_put(sA + kTileB, C, r0, np * 16, lo, lane);
    }
    // T_II, a lane a column
    {
        float x[16], m = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = i == lane ? 1.0f : 0.0f;
#pragma unroll
            for (int l4 = 0; l4 < i; l4 += 4) {
                const float4 w4 = *reinterpret_cast<const float4 *>(&sm.diag[warp][i][l4]);
                const float w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                for (int l = 0; l < 4; ++l)
                    if (l4 + l < i) x[i] = fmaf(-w[l], x[l4 + l], x[i]);
            }
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
    // (all have read K and Q, in whose place P goes)
    const uint32_t sP = sk;
#pragma unroll
    for (int np = 0; np < 4; ++np) {
        tile_put(sP, C, r0, np * 16, ph[np], lane);
        if (TERMS) tile_put(sP + kTileB, C, r0, np * 16, pl[np], lane);
    }
    if (warp == 3) {  // (whose block column is the diagonal block alone) the largest of what the chains multiply by
        float m[3];
        for (int i = 0; i < 2; ++i) {
            const int t = lane + i * 32;
            const float x[3] = {sm.left[t], fabsf(sm.past[t] * sm.b[t]), sm.past[t]};
#pragma unroll
            for (int w = 0; w < 3; ++w) m[w] = i ? fmaxf(m[w], x[w]) : x[w];
        }
#pragma unroll
        for (int w = 0; w < 3; ++w) m[w] = warp_max(m[w]);
        if (lane == 0) {
            rowf[4 * C + 6] = m[0] * ks.back;
            rowf[4 * C + 7] = m[1] * ks.back;
            rowf[4 * C + 8] = fabsf(a.scale) * m[2] * qs.back;
        }
    }
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
#pragma unroll
    for (int s = 0; s < 4; ++s) {  // (block row J + s, or the empty ones before J), in the place of A
        Frag th = {0, 0, 0, 0}, tl = {0, 0, 0, 0};
        if (warp + s < 4) split_left(T[s][0], T[s][1], ts.by, th, tl);
        tile_put(sA, C, r0, (warp + s) % 4 * 16, th, lane);
        tile_put(sA + kTileB, C, r0, (warp + s) % 4 * 16, tl, lane);
    }
    fence_proxy_async_smem();
    __syncthreads();
    if (tid == 0) {
        store_tile(a.Tp + at * 2 * C * C, sA, 2 * kTileB);
        store_tile(a.Pp + at * (TERMS ? 2 : 1) * C * C, sP, (TERMS ? 2 : 1) * kTileB);
        bulk_commit();
        bulk_wait();  // (shared memory is read to the end)
    }
}

template <int DP, bool TERMS>
cudaError_t prepare(const DeltaArgs &a, cudaStream_t s) {
    cudaError_t e = cudaFuncSetAttribute(k_delta_prepare<DP, TERMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PrepShared<DP>));
    if (e != cudaSuccess) return e;
    LUNA_LAUNCH("delta_prepare", (k_delta_prepare<DP, TERMS>), (unsigned)((int64_t)a.B * a.H * a.m), kPrepThreads, sizeof(PrepShared<DP>), s, a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_delta_prepare(const DeltaArgs &a, cudaStream_t s) {
    if (a.d <= 64) return a.planes == 2 ? prepare<64, true>(a, s) : prepare<64, false>(a, s);
    return a.planes == 2 ? prepare<128, true>(a, s) : prepare<128, false>(a, s);
}

}  // namespace luna
