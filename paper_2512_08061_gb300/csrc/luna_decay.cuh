// Linear attention with a decay for each head: argument blocks and launchers.
//
// Every pass of the operator, forward or backward, is one "mix" of three row
// sequences a, b (width da) and c (width dc) of a head:
//
//     out_i = p sum_{j <= i} lambda^{i-j} (a_i . b_j) c_j  +  x lambda^{i+e} a_i^T X
//     X'    = lambda^{n} X + u sum_j lambda^{n-j-e} b_j c_j^T
//
// with i, j positions in processing order.  Forward order uses e = 1 (the state
// decays before a token enters it); the reverse order of the gradients of k and
// v uses e = 0 and carries Y = lambda R, R the gradient of the state, so that
// what is left at the first token is the gradient of the initial state:
//
//     O  : a = q,  b = k,  c = v,  X = S      p = x = scale, u = 1
//     dQ : a = dO, b = v,  c = k,  X = S^T    p = x = scale, u = 1
//     dV : a = k,  b = q,  c = dO, X = Y      p = u = scale, x = 1   (reverse order)
//     dK : a = v,  b = dO, c = q,  X = Y^T    p = u = scale, x = 1   (reverse order)
#pragma once

#include "luna_common.cuh"

namespace luna {

struct RowView {          // rows of a (B, heads, n, width) tensor; strides in elements
    const void *p;
    int64_t sb, sh, st;
    int heads;            // heads of the tensor: query head h reads head h / (H / heads)
    bool vec = false;     // (CUDA-core form) rows start on boundaries of four values
};

struct DecayMix {
    RowView a, b, c;
    void *out;            // NULL: only the carry is computed
    int64_t ob, oh, ot;   // strides of out (one head for each of the H)
    bool ovec;            // as RowView::vec
    const float *log_decay;
    const int32_t *lengths;
    int B, H, n, da, dc;
    int reverse;          // processing order; e = reverse ? 0 : 1
    float p, x, u;
    int seg_len, nseg;    // the rows of a head are cut into nseg pieces of seg_len rows
    const float *X;       // carry into piece s of head bh at X + (bh * x_pieces + s) * da * dc, or NULL (zero)
    int x_pieces;         // nseg, or 1 (one piece)
    int x_trans;          // X is stored [dc][da]
    float *Xout;          // carry out of every piece, [bh][s][da][dc], or NULL
    int *status;          // device status word of the call
    int clear;            // first launch of the call: clears it
};

// Carries into the pieces from the pieces' own sums U (carry out of each from zero):
// X[0] = init, X[s + 1] = lambda^{rows of s} X[s] + U[s]; the last one goes to `last`.
struct DecayScan {
    const float *U, *init;  // U [bh][nseg][E]; init [bh][E] or NULL
    float *X, *last;        // X [bh][nseg][E]; last [bh][E] or NULL
    const float *log_decay;
    const int32_t *lengths;
    int B, H, n, seg_len, nseg, reverse;
    int64_t E;              // elements of a state
};

struct DecayStep {
    const void *q, *k, *v;
    void *o;
    int64_t qb, qh, kb, kh, vb, vh, ob, oh;
    const float *log_decay;
    const int32_t *slots;
    float *S;
    int nslots, B, H, Hkv, d, dv;
    float scale;
};

// The first block of a call's first kernel clears the status word; the waits that set it run for a second.
__device__ __forceinline__ void clear_status(const DecayMix &a) {
    if (a.clear && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.status = 0;
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t f2(uint32_t lo, uint32_t hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ uint64_t f2(float lo, float hi) { return f2(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ void unpack2(uint64_t v, float &lo, float &hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// log lambda of a head, with -inf (lambda = 0) as a finite value so that 0 * log lambda is 0.
__device__ __forceinline__ float decay_log(const float *log_decay, int h) {
    const float g = log_decay[h];
    return g < -1e30f ? -1e30f : g;
}

constexpr int kDecaySimtRows = 64;  // rows of a chunk of the CUDA-core form (128 on tensor cores)

cudaError_t launch_decay_mix(const DecayMix &a, luna_dtype io, luna_dtype out, cudaStream_t s);
bool decay_tc_ok(const DecayMix &a, luna_dtype io, luna_dtype out);  // shapes and alignments of the tensor-core form
cudaError_t launch_decay_mix_tc(const DecayMix &a, luna_dtype out, cudaStream_t s);
cudaError_t launch_decay_scan(const DecayScan &a, cudaStream_t s);
cudaError_t launch_decay_step(const DecayStep &a, luna_dtype io, cudaStream_t s);
// Sums groups of G consecutive heads of an fp32 (B, H, n, width) array into a tensor of H / G heads.
cudaError_t launch_decay_group_sum(const float *src, int B, int H, int G, int n, int width, void *dst, int64_t sb,
                                   int64_t sh, int64_t st, luna_dtype io, cudaStream_t s);

}  // namespace luna
