// The norms around a block: argument block, loads and element-wise work shared by the kernels.
#pragma once

#include <string.h>

#include "luna_common.cuh"

namespace luna {

struct NormArgs {
    const void *x, *y, *gate, *dX, *dH;
    void *X, *H, *dx, *dy, *dgate;
    const float *w_post, *b_post, *w_pre, *b_pre;
    float *part;       // [slot][array][cols]: weight-gradient partials (dw_post, db_post, dw_pre, db_pre)
    int64_t rows;
    int cols, groups, layer, act;
    float alpha, eps;
    int64_t ldx, ldy, ldgate, ldX, ldH, lddX, lddH, lddx, lddy, lddgate;
    int gvec;          // vectors of a group
    int gmode;         // how a group is summed: 0 whole row, 1 lanes of a warp, 2 through shared memory
};

// VEC values as they are loaded (16 bytes, or one value), and as fp32.
template <typename IO, int VEC> struct Vec;
template <> struct Vec<float, 4> {
    using Raw = float4;
    static __device__ __forceinline__ void unpack(const Raw &w, float (&v)[4]) { v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w; }
    static __device__ __forceinline__ void store(float *p, const float (&v)[4]) {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
};
template <> struct Vec<__nv_bfloat16, 8> {
    using Raw = uint4;
    static __device__ __forceinline__ void unpack(const Raw &w, float (&v)[8]) {
        const uint32_t b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(b[i] << 16);
            v[2 * i + 1] = __uint_as_float(b[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, const float (&v)[8]) {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 w = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            memcpy(&b[i], &w, 4);
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(b[0], b[1], b[2], b[3]);
    }
};
template <> struct Vec<float, 2> {
    using Raw = float2;
    static __device__ __forceinline__ void unpack(const Raw &w, float (&v)[2]) { v[0] = w.x; v[1] = w.y; }
    static __device__ __forceinline__ void store(float *p, const float (&v)[2]) {
        *reinterpret_cast<float2 *>(p) = make_float2(v[0], v[1]);
    }
};
template <> struct Vec<__nv_bfloat16, 2> {
    using Raw = uint32_t;
    static __device__ __forceinline__ void unpack(const Raw &w, float (&v)[2]) {
        v[0] = __uint_as_float(w << 16);
        v[1] = __uint_as_float(w & 0xffff0000u);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, const float (&v)[2]) {
        *reinterpret_cast<__nv_bfloat162 *>(p) = __floats2bfloat162_rn(v[0], v[1]);
    }
};
template <typename IO> struct Vec<IO, 1> {
    using Raw = IO;
    static __device__ __forceinline__ void unpack(const Raw &w, float (&v)[1]) { v[0] = io_load(&w); }
    static __device__ __forceinline__ void store(IO *p, const float (&v)[1]) { io_store(p, v[0]); }
};

// Element-wise work on VEC values, two an instruction.
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
template <int VEC> struct V {
    // d = a b + c
    static __device__ __forceinline__ void fma(float (&d)[VEC], const float (&a)[VEC], const float (&b)[VEC], const float (&c)[VEC]) {
        if (VEC == 1) { d[0] = fmaf(a[0], b[0], c[0]); return; }
#pragma unroll
        for (int e = 0; e + 1 < VEC; e += 2) {
            uint64_t r;
            asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair(a[e], a[e + 1])), "l"(pair(b[e], b[e + 1])), "l"(pair(c[e], c[e + 1])));
            asm("mov.b64 {%0, %1}, %2;" : "=f"(d[e]), "=f"(d[e + 1]) : "l"(r));
        }
    }
    // d = a s + c
    static __device__ __forceinline__ void fma(float (&d)[VEC], const float (&a)[VEC], float k, const float (&c)[VEC]) {
        if (VEC == 1) { d[0] = fmaf(a[0], k, c[0]); return; }
#pragma unroll
        for (int e = 0; e + 1 < VEC; e += 2) {
            uint64_t r;
            asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair(a[e], a[e + 1])), "l"(pair(k, k)), "l"(pair(c[e], c[e + 1])));
            asm("mov.b64 {%0, %1}, %2;" : "=f"(d[e]), "=f"(d[e + 1]) : "l"(r));
        }
    }
    static __device__ __forceinline__ void mul(float (&d)[VEC], const float (&a)[VEC], const float (&b)[VEC]) {
        if (VEC == 1) { d[0] = a[0] * b[0]; return; }
#pragma unroll
        for (int e = 0; e + 1 < VEC; e += 2) {
            uint64_t r;
            asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair(a[e], a[e + 1])), "l"(pair(b[e], b[e + 1])));
            asm("mov.b64 {%0, %1}, %2;" : "=f"(d[e]), "=f"(d[e + 1]) : "l"(r));
        }
    }
    static __device__ __forceinline__ void mul(float (&d)[VEC], const float (&a)[VEC], float k) {
        if (VEC == 1) { d[0] = a[0] * k; return; }
#pragma unroll
        for (int e = 0; e + 1 < VEC; e += 2) {
            uint64_t r;
            asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair(a[e], a[e + 1])), "l"(pair(k, k)));
            asm("mov.b64 {%0, %1}, %2;" : "=f"(d[e]), "=f"(d[e + 1]) : "l"(r));
        }
    }
    static __device__ __forceinline__ void add(float (&d)[VEC], const float (&a)[VEC], const float (&b)[VEC]) {
        if (VEC == 1) { d[0] = a[0] + b[0]; return; }
#pragma unroll
        for (int e = 0; e + 1 < VEC; e += 2) {
            uint64_t r;
            asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair(a[e], a[e + 1])), "l"(pair(b[e], b[e + 1])));
            asm("mov.b64 {%0, %1}, %2;" : "=f"(d[e]), "=f"(d[e + 1]) : "l"(r));
        }
    }
    static __device__ __forceinline__ float dot(const float (&a)[VEC], const float (&b)[VEC]) {
        if (VEC == 1) return a[0] * b[0];
        uint64_t r = pair(0.0f, 0.0f);
#pragma unroll
        for (int e = 0; e + 1 < VEC; e += 2)
            asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(r) : "l"(pair(a[e], a[e + 1])), "l"(pair(b[e], b[e + 1])));
        float x, y;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(r));
        return x + y;
    }
    static __device__ __forceinline__ float sum(const float (&a)[VEC]) {
        float s = a[0];
#pragma unroll
        for (int e = 1; e < VEC; ++e) s += a[e];
        return s;
    }
};

template <int VEC>
__device__ __forceinline__ void load_w(const float *p, int c, float (&v)[VEC]) {
    if (VEC == 1) {
        v[0] = p[c];
    } else if (VEC == 2) {
        const float2 w = *reinterpret_cast<const float2 *>(p + c);
        v[0] = w.x; v[1 % VEC] = w.y;
    } else {
#pragma unroll
        for (int i = 0; i + 3 < VEC; i += 4) {
            const float4 w = *reinterpret_cast<const float4 *>(p + c + i);
            v[i] = w.x; v[i + 1] = w.y; v[i + 2] = w.z; v[i + 3] = w.w;
        }
    }
}

// 1 / (1 + e^-g) by the hardware's exponential and reciprocal (2 ulp each), without their handling of
// denormal results, which would be as many operations again: those values count as 0.
__device__ __forceinline__ float sigmoidf(float g) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-1.4426950408889634f * g));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return r;
}

// Gates of VEC values: v *= act(g), the choice once for all of them.
template <int VEC> __device__ __forceinline__ void apply_gate(int act, const float (&g)[VEC], float (&v)[VEC]) {
    if (act == LUNA_GATE_SILU) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] *= g[e] * sigmoidf(g[e]);
    } else if (act == LUNA_GATE_SIGMOID) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] *= sigmoidf(g[e]);
    }
}
// act(g) into `value` and its slope into g.
template <int VEC> __device__ __forceinline__ void gate_and_slope(int act, float (&g)[VEC], float (&value)[VEC]) {
    if (act == LUNA_GATE_SILU) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float sg = sigmoidf(g[e]);
            value[e] = g[e] * sg;
            g[e] = fmaf(value[e], 1.0f - sg, sg);
        }
    } else if (act == LUNA_GATE_SIGMOID) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            value[e] = sigmoidf(g[e]);
            g[e] = value[e] * (1.0f - value[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) value[e] = 1.0f;
    }
}

// Floats of shared memory that the kernels for wide rows keep of a row and its groups.
__host__ __device__ constexpr int wide_floats(int cols, int groups) { return ((cols + 3) / 4 * 4 + 2 * (groups + 32) + 4 * groups + 3) / 4 * 4; }

// shared: the sums of the weight gradients in shared memory.
cudaError_t launch_norm_fwd_wide(NormArgs a, luna_dtype io, bool pairs, int grid, int threads, size_t smem, cudaStream_t s);
cudaError_t launch_norm_bwd_wide(NormArgs a, luna_dtype io, int vec, bool bias, bool shared, int grid, int threads, size_t smem,
                                 cudaStream_t s);

}  // namespace luna
