// The gated delta rule: argument blocks and launchers.
//
//     S_t = a_t (S_{t-1} - b_t k_t (k_t^T S_{t-1})) + b_t k_t v_t^T,   o_t = scale S_t^T q_t,   a_t = exp(g_t)
//
// With u_t = b_t (v_t - a_t S_{t-1}^T k_t), what a token writes, S_t = a_t S_{t-1} + k_t u_t^T.  The gradients
// carry R, that of the state after a token (R_n = dS1), back through the rows:
//
//     R_t += scale q_t dO_t^T;   x_t = R_t^T k_t;   dV_t = b_t x_t;   R_{t-1} = a_t (R_t - b_t k_t x_t^T)
//     dQ_t = scale S_t dO_t;   Z_t = a_t S_{t-1} x_t;   dK_t = R_t u_t - b_t Z_t
//     db_t = x_t . v_t - k_t . Z_t;   dg_t = <a_t S_{t-1}, R_t - b_t k_t x_t^T>
//
// The columns of S and R (dv of them) never meet, so that S, u and R, x walk the rows in blocks of a few columns;
// what needs whole rows of S and R is then a product over a chunk of 64 rows from the states at its two ends.
// With G_i the sum of a chunk's g to row i, c(i, j) = exp(G_i - G_j), S the state before and R the gradient after
// the chunk, and P_ij = scale c(i, j) dO_i . u_j (j <= i), W_ij = b_i c(i, j) x_i . u_j (j < i):
//
//     dQ_i = scale c(i, 0) S dO_i + sum_j P_ij k_j
//     dK_j = c(C, j) R u_j + sum_i P_ij q_i - sum_i W_ij k_i  -  b_j c(j, 0) S x_j - sum_{l < j} W_jl k_l
//
// and dg is a sum over all pairs of a row at or behind t (or R) that reads and a row before t (or S) that was written:
//
//     dg_t = c(C, 0) <S, R> + sum_{i >= t} (scale c(i, 0) q_i . S dO_i - b_i c(i, 0) k_i . S x_i) + sum_{j < t} c(C, j) k_j . R u_j
//            + sum_{j < t <= i} (P_ij q_i . k_j - W_ij k_i . k_j)
#pragma once

#include <cuda_fp16.h>

#include "luna_decay.cuh"

namespace luna {

constexpr int kDeltaRows = 64;      // rows of a chunk
// tensor-core form: fp32 values of a chunk's factors, and of the scales of 16 columns of it
constexpr int kDeltaFactors = 6 * kDeltaRows + 12, kDeltaScales = 8;

struct GateView {  // a (B, H, n) tensor
    const void *p;
    int64_t sb, sh, st;
};
struct GateOut {
    void *p;
    int64_t sb, sh, st;
};

struct DeltaArgs {
    RowView q, k, v, go;    // go: dO (backward)
    GateView g, b;
    void *o;                // O; (backward) dV
    int64_t ob, oh, ot;
    void *dq, *dk;          // gradients, of type io with strides, or (shared heads) fp32 [B][H][n][d]
    int64_t dqb, dqh, dqt, dkb, dkh, dkt;
    GateOut dg, db;
    const int32_t *lengths;
    const float *S0, *dS1;  // NULL: zero
    float *S1, *dS0;        // NULL: not wanted
    int B, H, n, d, dv, m;  // m: chunks of a head
    float scale;
    // intermediate results
    float *U, *X;           // rows written and their gradients, [B H][n][dv] (CUDA-core form)
    float *before, *after;  // states before chunk i, gradients of the states before chunk i, [B H][m + 1][d][dv]
    // tensor-core form (fp16, scaled; dvp: dv to a multiple of 16, dp: d to 64 or 128), for every chunk: its rows of K
    // and Q ([B Hk][m][64][dp]), the inverse T, transposed, in two planes and the scores P in `planes` of them ([64][64] each),
    // factors of its rows; and for every 16 columns of a chunk U, X and dO ([16][64], transposed), and before it
    // (R: behind the last one too, m + 1 to a head) the states ([16][dp], transposed) and what all these were scaled down by
    __half *Kp, *Qp, *Tp, *Pp, *Up, *Xp, *Gp, *Sp, *Rp;
    float *rows, *scales;
    int planes, dvp;
    bool vec;               // every row of every tensor starts on a 16-byte boundary and has whole vectors
    int *status;            // the call's status word
};

struct DeltaStep {
    const void *q, *k, *v;
    void *o;
    int64_t qb, qh, kb, kh, vb, vh, ob, oh;
    GateView g, b;
    const int32_t *slots;
    float *S;
    int nslots, B, H, Hk, d, dv;
    float scale;
};

template <typename T>
__device__ __forceinline__ float gate_at(const GateView &v, int b, int h, int t) {
    return io_load(static_cast<const T *>(v.p) + b * v.sb + h * v.sh + t * v.st);
}

// exp(g) in two terms: one rounded to fp32 is off the same way at every token of a head whose gate stands still.
__device__ __forceinline__ void gate_terms(float g, float &a, float &rest) {
    if (fabsf(g) < 0.5f) {  // (beyond that a state forgets, or overflows, in some ten tokens)
        const float m1 = expm1f(g);
        a = 1.0f + m1;
        rest = m1 - (a - 1.0f);
    } else {
        a = expf(g);
        rest = 0.0f;
    }
}

// Gates below this forget everything (exp is 0 in fp32); sums of a chunk's gates stay finite.
constexpr float kGateLeast = -120.0f;

// A chunk's gates, by one warp: their sums to each row in 64 bits, kept as two fp32 terms so that differences of near
// rows stay exact, and the factors from the chunk's start (past) and to its end (left).  gate(t) is 0 behind the end.
template <typename F>
__device__ __forceinline__ void delta_gate_sums(int lane, F gate, float *hi, float *lo, float *past, float *left) {
    auto least = [](float g) { return (double)(g < kGateLeast ? kGateLeast : g); };  // (a NaN stays one)
    const double g0 = least(gate(2 * lane)), g1 = least(gate(2 * lane + 1));
    double sum = g0 + g1;
#pragma unroll
    for (int w = 1; w < 32; w *= 2) {
        const double up = __shfl_up_sync(0xffffffffu, sum, w);
        if (lane >= w) sum += up;
    }
    const double total = __shfl_sync(0xffffffffu, sum, 31);
    auto factor = [](double x, float &h, float &l) {
        h = (float)x;
        l = (float)(x - (double)h);
        const float e = expf(h);
        return fmaf(e, l, e);
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const double G = i ? sum : sum - g1;
        float h, l, rh, rl;
        past[2 * lane + i] = factor(G, h, l);
        left[2 * lane + i] = factor(total - G, rh, rl);
        hi[2 * lane + i] = h;
        lo[2 * lane + i] = l;
    }
}

// dg of a chunk's rows, by one warp.  A gate takes part in all that is read at or behind it of what was written before it:
// by R of S (`ends` = c(C, 0) <S, R>), by rows at or behind it of S (read), by R of rows before it (wrote), by the former of the
// latter (crossed).  Each of these has the gate in its factor, so that a strong gate's gradient is a sum of small terms; as
// the difference of what is read up to a row and up to the next it was off by 1e-7 of the large ones (9 % at a gate of -12).
template <typename F>
__device__ __forceinline__ void delta_gate_grads(float ends, const float *read, const float *wrote, const float *crossed,
                                                 int rows, int lane, F store) {
    float r[2], w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int t = 2 * lane + i;
        r[i] = t < rows ? read[t] : 0.0f;
        w[i] = t < rows ? wrote[t] : 0.0f;
    }
    float behind = r[0] + r[1], before = w[0] + w[1];
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
        const float x = __shfl_down_sync(0xffffffffu, behind, m), y = __shfl_up_sync(0xffffffffu, before, m);
        if (lane + m < 32) behind += x;
        if (lane >= m) before += y;
    }
    behind = __shfl_down_sync(0xffffffffu, behind, 1);  // of the other lanes' rows
    before = __shfl_up_sync(0xffffffffu, before, 1);
    if (lane == 31) behind = 0.0f;
    if (lane == 0) before = 0.0f;
    behind += r[1];
    if (2 * lane < rows) store(2 * lane, (ends + crossed[2 * lane]) + ((behind + r[0]) + before));
    if (2 * lane + 1 < rows) store(2 * lane + 1, (ends + crossed[2 * lane + 1]) + (behind + (before + w[0])));
}

cudaError_t launch_delta_rows(const DeltaArgs &a, bool reverse, cudaStream_t s);  // fp32
cudaError_t launch_delta_grad(const DeltaArgs &a, cudaStream_t s);
// bf16, on tensor cores
cudaError_t launch_delta_prepare(const DeltaArgs &a, cudaStream_t s);
cudaError_t launch_delta_chain64(const DeltaArgs &a, bool reverse, cudaStream_t s);   // d <= 64
cudaError_t launch_delta_chain128(const DeltaArgs &a, bool reverse, cudaStream_t s);
cudaError_t launch_delta_grad_tc(const DeltaArgs &a, luna_dtype out, cudaStream_t s);
cudaError_t launch_delta_step(const DeltaStep &a, luna_dtype io, cudaStream_t s);

}  // namespace luna
