// The norms around a block for rows too wide for a thread's registers (the formulas are in luna_norm.cu).
//
// A block walks a row in passes and reads the inputs again in each (from the caches: the row is its
// only one); x' and the post-norm's output gradient stay in shared memory in fp32, the weight gradients'
// sums too where they fit.  Every warp owns a run of the row's vectors, in pieces that end with the groups.
// Bound by the latency of the passes (at 2913 x 7094 fp32 forward 136 us, backward 243 us, 2 TB/s), with
// the next row asked for in L2 meanwhile.  (Held in registers like narrow rows, 14 values a thread spilled
// beyond the first-level cache: 248 and 1337 us.)
#include "luna_norm.cuh"
#include "luna_prof.cuh"

namespace luna {
namespace {

template <typename IO, int VEC> __device__ __forceinline__ void load_at(const void *p, int64_t off, float (&v)[VEC]) {
    if (p) {
        Vec<IO, VEC>::unpack(*reinterpret_cast<const typename Vec<IO, VEC>::Raw *>(static_cast<const IO *>(p) + off), v);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = 0.0f;
    }
}
template <int VEC> __device__ __forceinline__ void put_w(float *p, int c, const float (&v)[VEC]) {
    if (VEC == 1) {
        p[c] = v[0];
    } else if (VEC == 2) {
        *reinterpret_cast<float2 *>(p + c) = make_float2(v[0], v[1 % VEC]);
    } else {
#pragma unroll
        for (int i = 0; i + 3 < VEC; i += 4) *reinterpret_cast<float4 *>(p + c + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    }
}

struct WideRow {
    int t, warp, lane, threads, v0, v1, groups, gvec;
    float2 *part;        // [groups + warps] sums of the pieces
    float2 *total;       // [groups]
    float *mean, *root;  // [groups] of the post-norm: mean, reciprocal root
    float *row;          // the row in fp32
    __device__ __forceinline__ WideRow(const NormArgs &a, int nvec, float *sm) {
        t = threadIdx.x; warp = t >> 5; lane = t & 31; threads = blockDim.x;
        const int span = (nvec + threads / 32 - 1) / (threads / 32);
        v0 = min(nvec, warp * span);
        v1 = min(nvec, v0 + span);
        groups = a.groups;
        gvec = nvec / groups;
        row = sm;
        part = reinterpret_cast<float2 *>(sm + (a.cols + 3) / 4 * 4);
        total = part + groups + 32;
        mean = reinterpret_cast<float *>(total + groups);
        root = mean + groups;
    }
    // f(group, from, to) of this warp's pieces, with groups of `width` vectors
    template <typename F> __device__ __forceinline__ void pieces(int width, F f) const {
        for (int v = v0; v < v1;) {
            const int g = v / width, e = min(v1, (g + 1) * width);
            f(g, v, e);
            v = e;
        }
    }
    // total[g] = sum of f(group, vector) over each group of `width` vectors
    template <typename F> __device__ __forceinline__ void sums(int width, int count, F f) const {
        pieces(width, [&](int g, int v, int e) {
            float2 s = make_float2(0.f, 0.f);
#pragma unroll 4
            for (int i = v + lane; i < e; i += 32) f(g, i, s);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                s.x += __shfl_xor_sync(0xffffffffu, s.x, o);
                s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
            }
            if (lane == 0) part[g + warp] = s;  // (pieces in order: no other has this sum)
        });
        __syncthreads();
        const int span = max(1, span_());
        for (int g = t; g < count; g += threads) {
            float2 s = make_float2(0.f, 0.f);
            for (int w = g * width / span; w <= (g * width + width - 1) / span; ++w) { s.x += part[g + w].x; s.y += part[g + w].y; }
            total[g] = s;
        }
        __syncthreads();
    }
    __device__ __forceinline__ int span_() const { return (gvec * groups + threads / 32 - 1) / (threads / 32); }
};

// The post-norm's mean and reciprocal root of every group.
template <typename IO, int VEC>
__device__ __forceinline__ void wide_post(const WideRow &w, const NormArgs &a, int64_t off) {
    const float inv = 1.0f / (float)(w.gvec * VEC);
    if (a.layer) {
        w.sums(w.gvec, w.groups, [&](int, int i, float2 &s) {
            float z[VEC];
            load_at<IO, VEC>(a.y, off + (int64_t)i * VEC, z);
            s.x += V<VEC>::sum(z);
        });
        for (int g = w.t; g < w.groups; g += w.threads) w.mean[g] = w.total[g].x * inv;
    } else {
        for (int g = w.t; g < w.groups; g += w.threads) w.mean[g] = 0.0f;
    }
    __syncthreads();
    w.sums(w.gvec, w.groups, [&](int g, int i, float2 &s) {
        float z[VEC];
        load_at<IO, VEC>(a.y, off + (int64_t)i * VEC, z);
#pragma unroll
        for (int e = 0; e < VEC; ++e) z[e] -= w.mean[g];
        s.x += V<VEC>::dot(z, z);
    });
    for (int g = w.t; g < w.groups; g += w.threads) w.root[g] = rsqrtf(fmaf(w.total[g].x, inv, a.eps));
    __syncthreads();
}

// u = norm(y) w_post + b_post of a vector (or y), and norm(y) in z.
template <typename IO, int VEC>
__device__ __forceinline__ void wide_u(const WideRow &w, const NormArgs &a, int64_t off, int g, int i, float (&z)[VEC], float (&u)[VEC]) {
    load_at<IO, VEC>(a.y, off + (int64_t)i * VEC, z);
    if (a.w_post) {
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) z[e] = (z[e] - w.mean[g]) * w.root[g];
        load_w<VEC>(a.w_post, i * VEC, v);
        V<VEC>::mul(u, z, v);
        if (a.b_post) {
            load_w<VEC>(a.b_post, i * VEC, v);
            V<VEC>::add(u, u, v);
        }
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) u[e] = z[e];
    }
}

__device__ __forceinline__ void prefetch_row(const void *p, int64_t off, int cols, int size, int t, int threads) {
    if (!p) return;
    const char *q = static_cast<const char *>(p) + off * size;
    for (int b = t * 128; b < cols * size; b += threads * 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + b));
}

template <typename IO, int VEC>
__global__ void __launch_bounds__(1024) k_norm_fwd_wide(NormArgs a) {
    extern __shared__ __align__(16) float sm[];
    const int nvec = a.cols / VEC;
    const WideRow w(a, nvec, sm);
    const float inv = 1.0f / (float)a.cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t next = row + gridDim.x;
        if (next < a.rows) {
            prefetch_row(a.x, next * a.ldx, a.cols, sizeof(IO), w.t, w.threads);
            prefetch_row(a.y, next * a.ldy, a.cols, sizeof(IO), w.t, w.threads);
            prefetch_row(a.gate, next * a.ldgate, a.cols, sizeof(IO), w.t, w.threads);
        }
        if (a.y && a.w_post) wide_post<IO, VEC>(w, a, row * a.ldy);
        w.pieces(a.w_post ? w.gvec : nvec, [&](int g, int v, int e) {
#pragma unroll 2
            for (int i = v + w.lane; i < e; i += 32) {
                float x[VEC], z[VEC], u[VEC], gt[VEC];
                load_at<IO, VEC>(a.x, row * a.ldx + (int64_t)i * VEC, x);
                if (a.y) {
                    load_at<IO, VEC>(a.gate, row * a.ldgate + (int64_t)i * VEC, gt);
                    wide_u<IO, VEC>(w, a, row * a.ldy, g, i, z, u);
                    apply_gate<VEC>(a.act, gt, u);
                    V<VEC>::fma(x, u, a.alpha, x);
                }
                if (a.X) Vec<IO, VEC>::store(static_cast<IO *>(a.X) + row * a.ldX + (int64_t)i * VEC, x);
                put_w<VEC>(w.row, i * VEC, x);
            }
        });
        if (!a.w_pre) {
            __syncthreads();  // (the groups' values are read before the next row's)
            continue;
        }
        __syncwarp();  // (a warp reads what it wrote itself)
        float m = 0.0f;
        if (a.layer) {
            w.sums(nvec, 1, [&](int, int i, float2 &s) {
                float x[VEC];
                load_w<VEC>(w.row, i * VEC, x);
                s.x += V<VEC>::sum(x);
            });
            m = w.total[0].x * inv;
            __syncthreads();
        }
        w.sums(nvec, 1, [&](int, int i, float2 &s) {
            float x[VEC];
            load_w<VEC>(w.row, i * VEC, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] -= m;
            s.x += V<VEC>::dot(x, x);
        });
        const float r = rsqrtf(fmaf(w.total[0].x, inv, a.eps));
#pragma unroll 2
        for (int i = w.v0 + w.lane; i < w.v1; i += 32) {
            float x[VEC], p[VEC];
            load_w<VEC>(w.row, i * VEC, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = (x[e] - m) * r;
            load_w<VEC>(a.w_pre, i * VEC, p);
            V<VEC>::mul(x, x, p);
            if (a.b_pre) {
                load_w<VEC>(a.b_pre, i * VEC, p);
                V<VEC>::add(x, x, p);
            }
            Vec<IO, VEC>::store(static_cast<IO *>(a.H) + row * a.ldH + (int64_t)i * VEC, x);
        }
        __syncthreads();  // (total is read before the next row's sums)
    }
}

// SHARED: the weight gradients' sums in shared memory, or else where they end up.
template <typename IO, int VEC, bool BIAS, bool SHARED>
__global__ void __launch_bounds__(1024) k_norm_bwd_wide(NormArgs a) {
    extern __shared__ __align__(16) float sm[];
    const int nvec = a.cols / VEC, cols = a.cols;
    const WideRow w(a, nvec, sm);
    constexpr int ARRAYS = BIAS ? 4 : 2;
    float *out = a.part ? a.part + (int64_t)blockIdx.x * ARRAYS * cols : nullptr;
    const int lda = SHARED ? (cols + 3) / 4 * 4 : cols;
    float *acc = SHARED ? sm + wide_floats(cols, a.groups) : out;  // w_post, w_pre, b_post, b_pre
    // (every lane adds to its own columns alone)
    auto add_to = [&](int array, int i, const float (&v)[VEC]) {
        if (!acc) return;
        float *p = acc + (int64_t)array * lda + i * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) p[e] += v[e];
    };
    if (acc)
        for (int k = 0; k < ARRAYS; ++k)
            for (int i = w.v0 + w.lane; i < w.v1; i += 32)
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[(int64_t)k * lda + i * VEC + e] = 0.0f;
    const float inv = 1.0f / (float)cols, ginv = 1.0f / (float)(w.gvec * VEC);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t next = row + gridDim.x;
        if (next < a.rows) {
            prefetch_row(a.x, next * a.ldx, cols, sizeof(IO), w.t, w.threads);
            prefetch_row(a.y, next * a.ldy, cols, sizeof(IO), w.t, w.threads);
            prefetch_row(a.gate, next * a.ldgate, cols, sizeof(IO), w.t, w.threads);
            prefetch_row(a.dX, next * a.lddX, cols, sizeof(IO), w.t, w.threads);
            prefetch_row(a.dH, next * a.lddH, cols, sizeof(IO), w.t, w.threads);
        }
        if (a.y && a.w_post) wide_post<IO, VEC>(w, a, row * a.ldy);
        float m = 0.0f, r = 0.0f, mz = 0.0f, md = 0.0f;
        if (a.w_pre) {
            // x', and what its norm and that norm's gradient sum
            w.pieces(a.w_post ? w.gvec : nvec, [&](int g, int v, int e) {
#pragma unroll 2
                for (int i = v + w.lane; i < e; i += 32) {
                    float x[VEC], z[VEC], u[VEC], gt[VEC];
                    load_at<IO, VEC>(a.x, row * a.ldx + (int64_t)i * VEC, x);
                    if (a.y) {
                        load_at<IO, VEC>(a.gate, row * a.ldgate + (int64_t)i * VEC, gt);
                        wide_u<IO, VEC>(w, a, row * a.ldy, g, i, z, u);
                        apply_gate<VEC>(a.act, gt, u);
                        V<VEC>::fma(x, u, a.alpha, x);
                    }
                    put_w<VEC>(w.row, i * VEC, x);
                }
            });
            __syncwarp();  // (a warp reads what it wrote itself)
            if (a.layer) {
                w.sums(nvec, 1, [&](int, int i, float2 &s) {
                    float x[VEC], d[VEC], p[VEC];
                    load_w<VEC>(w.row, i * VEC, x);
                    load_at<IO, VEC>(a.dH, row * a.lddH + (int64_t)i * VEC, d);
                    load_w<VEC>(a.w_pre, i * VEC, p);
                    s.x += V<VEC>::sum(x);
                    s.y += V<VEC>::dot(d, p);
                });
                m = w.total[0].x * inv;
                md = w.total[0].y * inv;
                __syncthreads();
            }
            w.sums(nvec, 1, [&](int, int i, float2 &s) {  // sum d xhat = r sum d (x' - mean)
                float x[VEC], d[VEC], p[VEC];
                load_w<VEC>(w.row, i * VEC, x);
                load_at<IO, VEC>(a.dH, row * a.lddH + (int64_t)i * VEC, d);
                load_w<VEC>(a.w_pre, i * VEC, p);
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[e] -= m;
                V<VEC>::mul(d, d, p);
                s.x += V<VEC>::dot(x, x);
                s.y += V<VEC>::dot(x, d);
            });
            r = rsqrtf(fmaf(w.total[0].x, inv, a.eps));
            mz = w.total[0].y * r * inv;
            __syncthreads();
        }
        auto grads = [&](int g, int i, float2 &s) {
            const int64_t c = (int64_t)i * VEC;
            float d[VEC], z[VEC], u[VEC], gt[VEC], act[VEC], p[VEC];
            load_at<IO, VEC>(a.dX, row * a.lddX + c, d);
            if (a.w_pre) {
                float x[VEC], dh[VEC];
                load_w<VEC>(w.row, i * VEC, x);
                load_at<IO, VEC>(a.dH, row * a.lddH + c, dh);
                load_w<VEC>(a.w_pre, i * VEC, p);
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[e] = (x[e] - m) * r;
                if (BIAS) add_to(3, i, dh);
#pragma unroll
                for (int e = 0; e < VEC; ++e) u[e] = dh[e] * x[e];
                add_to(1, i, u);
#pragma unroll
                for (int e = 0; e < VEC; ++e) d[e] += r * (dh[e] * p[e] - x[e] * mz - md);
            }
            if (a.dx) Vec<IO, VEC>::store(static_cast<IO *>(a.dx) + row * a.lddx + c, d);
            if (!a.y) return;
            load_at<IO, VEC>(a.gate, row * a.ldgate + c, gt);
            wide_u<IO, VEC>(w, a, row * a.ldy, g, i, z, u);
            gate_and_slope<VEC>(a.act, gt, act);
            V<VEC>::mul(d, d, a.alpha);
            if (a.gate) {
                V<VEC>::mul(u, d, u);
                V<VEC>::mul(u, u, gt);
                V<VEC>::mul(d, d, act);
                Vec<IO, VEC>::store(static_cast<IO *>(a.dgate) + row * a.lddgate + c, u);
            }
            if (a.w_post) {
                if (BIAS) add_to(2, i, d);
                V<VEC>::mul(u, d, z);
                add_to(0, i, u);
                load_w<VEC>(a.w_post, i * VEC, p);
                V<VEC>::mul(d, d, p);
                s.x += V<VEC>::dot(d, z);
                s.y += V<VEC>::sum(d);
                put_w<VEC>(w.row, i * VEC, d);
            } else {
                Vec<IO, VEC>::store(static_cast<IO *>(a.dy) + row * a.lddy + c, d);
            }
        };
        if (!a.y || !a.w_post) {
            float2 none = make_float2(0.f, 0.f);
            for (int i = w.v0 + w.lane; i < w.v1; i += 32) grads(0, i, none);
        } else {
            w.sums(w.gvec, w.groups, grads);
            w.pieces(w.gvec, [&](int g, int v, int e) {
                const float gz = w.total[g].x * ginv, gd = a.layer ? w.total[g].y * ginv : 0.0f, gm = w.mean[g], gr = w.root[g];
#pragma unroll 4
                for (int i = v + w.lane; i < e; i += 32) {
                    float d[VEC], z[VEC];
                    load_w<VEC>(w.row, i * VEC, d);
                    load_at<IO, VEC>(a.y, row * a.ldy + (int64_t)i * VEC, z);
#pragma unroll
                    for (int k = 0; k < VEC; ++k) d[k] = gr * (d[k] - (z[k] - gm) * gr * gz - gd);
                    Vec<IO, VEC>::store(static_cast<IO *>(a.dy) + row * a.lddy + (int64_t)i * VEC, d);
                }
            });
        }
        __syncthreads();  // (the groups' values are read before the next row's)
    }
    if (SHARED && out)
        for (int k = 0; k < ARRAYS; ++k)
            for (int i = w.v0 + w.lane; i < w.v1; i += 32)
#pragma unroll
                for (int e = 0; e < VEC; ++e) out[(int64_t)k * cols + i * VEC + e] = acc[(int64_t)k * lda + i * VEC + e];
}

template <typename K>
cudaError_t launch(K kernel, const char *name, NormArgs a, int grid, int threads, size_t smem, cudaStream_t s) {
    if (!a.w_post) a.groups = 1;
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    LUNA_LAUNCH(name, kernel, grid, threads, smem, s, a);
    return cudaGetLastError();
}

template <typename IO, int VEC>
cudaError_t bwd(const NormArgs &a, bool bias, bool shared, int grid, int threads, size_t smem, cudaStream_t s) {
    if (bias)
        return shared ? launch(k_norm_bwd_wide<IO, VEC, true, true>, "norm_bwd", a, grid, threads, smem, s)
                      : launch(k_norm_bwd_wide<IO, VEC, true, false>, "norm_bwd", a, grid, threads, smem, s);
    return shared ? launch(k_norm_bwd_wide<IO, VEC, false, true>, "norm_bwd", a, grid, threads, smem, s)
                  : launch(k_norm_bwd_wide<IO, VEC, false, false>, "norm_bwd", a, grid, threads, smem, s);
}

}  // namespace

cudaError_t launch_norm_fwd_wide(NormArgs a, luna_dtype io, bool pairs, int grid, int threads, size_t smem, cudaStream_t s) {
    if (io == LUNA_F32)
        return pairs ? launch(k_norm_fwd_wide<float, 2>, "norm_fwd", a, grid, threads, smem, s)
                     : launch(k_norm_fwd_wide<float, 1>, "norm_fwd", a, grid, threads, smem, s);
    return pairs ? launch(k_norm_fwd_wide<__nv_bfloat16, 2>, "norm_fwd", a, grid, threads, smem, s)
                 : launch(k_norm_fwd_wide<__nv_bfloat16, 1>, "norm_fwd", a, grid, threads, smem, s);
}

cudaError_t launch_norm_bwd_wide(NormArgs a, luna_dtype io, int vec, bool bias, bool shared, int grid, int threads, size_t smem,
                                 cudaStream_t s) {
    if (io == LUNA_F32)
        return vec == 4   ? bwd<float, 4>(a, bias, shared, grid, threads, smem, s)
               : vec == 2 ? bwd<float, 2>(a, bias, shared, grid, threads, smem, s)
                          : bwd<float, 1>(a, bias, shared, grid, threads, smem, s);
    return vec == 8   ? bwd<__nv_bfloat16, 8>(a, bias, shared, grid, threads, smem, s)
           : vec == 2 ? bwd<__nv_bfloat16, 2>(a, bias, shared, grid, threads, smem, s)
                      : bwd<__nv_bfloat16, 1>(a, bias, shared, grid, threads, smem, s);
}

}  // namespace luna
