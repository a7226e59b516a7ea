// Matrix products with a fused epilogue: argument blocks and launchers.
//
//     out = act(A B^T + bias) + R,   A: M x K, B: N x K,   z = A B^T + bias kept where asked
//
// The three products of a linear layer are this one with other operands:
//     forward  Y  (m x n): A = X (m x k),    B = W (n x k)
//     backward dX (m x k): A = dZ (m x n),   B = W^T (k x n)
//     backward dW (n x k): A = dZ^T (n x m), B = X^T (k x m)
#pragma once

#include "luna_common.cuh"

namespace luna {

struct MatView {           // element (row, k) at p[row * ld + k], or with kt at p[k * ld + row]
    const void *p;
    int64_t ld;
    bool kt;
    int64_t lo = 0;        // a value's second bf16 term so many elements on, or 0 (tensor cores alone)
};

struct Product {
    MatView A, B;
    int64_t M, N, K;
    const void *bias;      // N values, or NULL
    int act;               // luna_linear_act
    const void *R;         // residual M x N, or NULL
    void *Z, *out;         // Z: pre-activation M x N, or NULL
    int64_t ldr, ldz, ldo;
    float *part;           // fp32 partial products [split][M][N]
    size_t part_bytes;
    void *pad;             // room for copies of operands that TMA cannot read (bf16 with widths that are not
    size_t pad_bytes;      // multiples of 8), or NULL
    int *status;           // device status word
    int clear;             // first launch of the call: clears it
    const int *flags;      // n_flags words of which one is set where an fp32 operand holds an infinity or a
    int n_flags;           // NaN (or NULL): the tensor-core kernel then leaves the product to the other one
};

constexpr int kFlagBlocks = 304;  // blocks that look at an operand, a word for each

// One of p's flags is set; for the whole block.
__device__ __forceinline__ bool flagged(const Product &p) {
    int f = 0;
    if (p.flags)
        for (int i = threadIdx.x; i < p.n_flags; i += blockDim.x) f |= p.flags[i];
    return __syncthreads_or(f) != 0;
}

// The first block of a call's first kernel clears the status word; the waits that set it run for a second.
__device__ __forceinline__ void clear_status(int clear, int *status) {
    if (clear && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0) *status = 0;
}

// The standard normal distribution function and its density.  With fp32 outputs by erfcf, which keeps the
// lower tail (1 + erff(z / sqrt 2) cancels there: 2e-2 of it at z = -4.8, all of it at -6); with bf16
// outputs the upper tail from Abramowitz and Stegun 7.1.26 (erfc(x) = t (a1 + ... + a5 t^4) e^{-x^2},
// t = 1 / (1 + p x)), which shares its exponential with the density and keeps Phi(z) below zero to
// 2^-9 relative down to z = -5: 12 operations against about 40 an element, which the epilogue of a
// product of depth 1024 has no time for.
template <typename IO>
__device__ __forceinline__ float normal_cdf(float z, float &density) {
    if (sizeof(IO) == 4) {
        density = 0.39894228040143268f * expf(-0.5f * z * z);
        return 0.5f * erfcf(z * -0.70710678118654752f);
    }
    const float e = __expf(-0.5f * z * z);
    density = 0.39894228040143268f * e;
    const float t = __fdividef(1.0f, fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.0f));
    float q = fmaf(t, 1.061405429f, -1.453152027f);
    q = fmaf(t, q, 1.421413741f);
    q = fmaf(t, q, -0.284496736f);
    q = fmaf(t, q, 0.254829592f);
    const float tail = 0.5f * t * q * e;
    return z < 0.0f ? tail : 1.0f - tail;
}

// s = 1 / (1 + e^-z) and 1 - s for fp32 outputs, both whole in their tails; the exponential never overflows, and
// the divisor in [1, 2] costs __fdividef 2 units at most.
// (The bf16 forms below use __expf and __fdividef, whose errors grow with |z| to some 2^-17, far under a bf16 unit.)
__device__ __forceinline__ float sigmoid_pair(float z, float &rest) {
    const float e = expf(-fabsf(z)), big = __fdividef(1.0f, 1.0f + e), small = e * big;
    rest = z < 0.0f ? big : small;
    return z < 0.0f ? small : big;
}

template <typename IO>
__device__ __forceinline__ float linear_act(float z, int act) {
    float d;
    switch (act) {
        case LUNA_LINEAR_RELU: return z > 0.0f ? z : (z == z ? 0.0f : z);
        case LUNA_LINEAR_GELU: return z * normal_cdf<IO>(z, d);
        case LUNA_LINEAR_SILU: return sizeof(IO) == 4 ? z * sigmoid_pair(z, d) : __fdividef(z, 1.0f + __expf(-z));
    }
    return z;
}

// d act / d z
template <typename IO>
__device__ __forceinline__ float linear_slope(float z, int act) {
    switch (act) {
        case LUNA_LINEAR_RELU: return z > 0.0f ? 1.0f : 0.0f;
        case LUNA_LINEAR_GELU: {
            float d;
            const float c = normal_cdf<IO>(z, d);
            return fmaf(z, d, c);
        }
        case LUNA_LINEAR_SILU: {
            float s, rest;
            if (sizeof(IO) == 4) {
                s = sigmoid_pair(z, rest);
            } else {
                s = __fdividef(1.0f, 1.0f + __expf(-z));
                rest = 1.0f - s;
            }
            return s * (1.0f + z * rest);
        }
    }
    return 1.0f;
}

// One output value from its sum: z = sum + bias (kept), act, residual.
template <typename IO>
__device__ __forceinline__ void linear_finish(const Product &p, int64_t row, int64_t col, float sum) {
    if (p.bias) sum += io_load(static_cast<const IO *>(p.bias) + col);
    if (p.Z) io_store(static_cast<IO *>(p.Z) + row * p.ldz + col, sum);
    float y = linear_act<IO>(sum, p.act);
    if (p.R) y += io_load(static_cast<const IO *>(p.R) + row * p.ldr + col);
    io_store(static_cast<IO *>(p.out) + row * p.ldo + col, y);
}

// Pieces of K that a product of M x N x K is cut into on a launch of `tiles` blocks: enough to give
// every SM a block, none under `least` of K, and no more than the partial buffer holds.
int linear_splits(const Product &p, int64_t tiles, int64_t least);

cudaError_t launch_product(const Product &p, luna_dtype io, cudaStream_t s);          // picks a kernel
cudaError_t launch_product_simt(const Product &p, luna_dtype io, cudaStream_t s);     // any operands
bool product_rows_ok(const Product &p, luna_dtype io);                                // a few rows of X
cudaError_t launch_product_rows(const Product &p, luna_dtype io, cudaStream_t s);
// On tensor cores: bf16 operands, or with LUNA_F32 operands in three bf16 planes along K (see k_split).
cudaError_t launch_product_tc(const Product &p, luna_dtype io, cudaStream_t s);
// Estimated cycles of the 64-deep steps that a block of that form runs one after another in a bf16 product.
double product_tc_cycles(int64_t M, int64_t N, int64_t K);
cudaError_t launch_product_finish(const Product &p, int splits, luna_dtype io, cudaStream_t s);

}  // namespace luna
