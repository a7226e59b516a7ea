// The norms after and before a block, fused with the block's gate and residual scale:
//
//     u = norm_g(y) w_post + b_post        (norm over each of the row's groups; or u = y)
//     x' = x + alpha u act(gate)           (act: none, sigmoid or silu)
//     h = norm(x') w_pre + b_pre           (norm over the row)
//
// norm(z) = z / sqrt(mean(z^2) + eps), with the mean of z taken out first for the layer kind.
// Gradients of one row, from dX = dL/dx' and dH = dL/dh, with zhat = norm(z), r = 1 / root:
//
//     norm's input gradient from d (its output's):  r (d - zhat mean(d zhat) - [layer] mean(d))
//     g = dX + that of dH w_pre;   dx = g;   dgate = alpha g u act'(gate);   du = alpha g act(gate)
//     dy = that of du w_post;      dw_post = sum_rows du yhat;   dw_pre = sum_rows dH xhat
//
// Bound by bytes and, in the backward pass, by the latency of a row's reductions (16384 x 2048 bf16, 16
// groups, silu gate: forward 67 us, 5.0 TB/s; backward 146 us, 3.7 TB/s, at 16 warps an SM): every row is
// read once and written once, held in registers
// between the reductions (the statistics are recomputed by the backward pass, which has to read
// the same rows anyway), and the weight gradients are summed in registers over the rows of a
// block and joined by a second small kernel in a fixed order.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "luna_norm.cuh"
#include "luna_prof.cuh"

namespace luna {

int tc_sm_count();

namespace {

constexpr int kMaxCols = 16384;

// Launch shapes.  A thread takes NV vectors (16 bytes, or one value where rows are not aligned) of a row.
// `threads`: the threads of a row at most; `resident`: the threads an SM holds, which sets a thread's
// registers (65536 / resident) and the grid.
struct Limits {
    int threads, resident;
};
constexpr Limits limits(int vec, int nv, bool backward) {
    if (vec == 1) return nv == 4 ? Limits{256, backward ? 512 : 1024} : Limits{512, 512};  // (32: narrow groups alone)
    if (nv == 1) return backward ? Limits{512, 512} : Limits{256, 1024};
    if (nv == 2) return backward ? Limits{512, 512} : Limits{256, 512};
    return Limits{kMaxCols / vec / nv, kMaxCols / vec / nv};
}

// The threads of one row: a warp (eight rows a block) or the whole block.  Vector i of thread t is
// number t + i * threads of the row.
template <int NV>
struct RowTeam {
    int t, threads;     // this thread's number in the row, threads of the row
    int wpad;           // warps of the row, rounded up to a power of two
    bool warp_row;
    float *red;         // block rows: [2][32][2] sums of the warps
    float *gsm;         // group sums through shared memory: [vectors][2] then [groups][2]
    int nvec, buf;

    __device__ __forceinline__ void sync() const {
        if (warp_row) __syncwarp();
        else __syncthreads();
    }

    // Sum of (a, b) over the row, to every thread.
    // `two`: b as well (the same for all threads).
    __device__ __forceinline__ float2 row_sum(float2 v, bool two) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        if (two)
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
        if (warp_row) return v;
        float2 *r = reinterpret_cast<float2 *>(red) + 32 * buf;
        buf ^= 1;  // the buffer after next is free: every thread has passed the barrier in between
        if ((t & 31) == 0) r[t >> 5] = v;
        __syncthreads();
        // every group of `wpad` lanes holds the warps' sums
        const int w = t & (wpad - 1);
        v = w < threads / 32 ? r[w] : make_float2(0.f, 0.f);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            if (o < wpad) {
                v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
                if (two) v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
            }
        return v;
    }

    // Sums over each group of the thread's vectors (v in, sums of the vector's group out).
    __device__ __forceinline__ void group_sum(float2 (&v)[NV], const NormArgs &a, const int (&grp)[NV], bool two) {
        if (a.gmode == 0) {
            float2 s = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i) { s.x += v[i].x; s.y += v[i].y; }
            s = row_sum(s, two);
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = s;
        } else if (a.gmode == 1) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int o = 16; o > 0; o >>= 1)
                    if (o < a.gvec) {
                        v[i].x += __shfl_xor_sync(0xffffffffu, v[i].x, o);
                        if (two) v[i].y += __shfl_xor_sync(0xffffffffu, v[i].y, o);
                    }
        } else {
            float2 *p = reinterpret_cast<float2 *>(gsm), *g = p + nvec;
            sync();  // the last call's sums have been read
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (t + i * threads < nvec) p[t + i * threads] = v[i];
            sync();
            for (int q = t >> 5; q < a.groups; q += threads / 32) {  // a warp for each group
                float2 s = make_float2(0.f, 0.f);
                for (int j = t & 31; j < a.gvec; j += 32) { s.x += p[q * a.gvec + j].x; s.y += p[q * a.gvec + j].y; }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    s.x += __shfl_xor_sync(0xffffffffu, s.x, o);
                    s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
                }
                if ((t & 31) == 0) g[q] = s;
            }
            sync();
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (t + i * threads < nvec) v[i] = g[grp[i]];
        }
    }
};

template <int NV>
__device__ __forceinline__ RowTeam<NV> make_team(const NormArgs &a, int nvec, float *sm) {
    RowTeam<NV> t;
    t.warp_row = blockDim.y > 1;
    t.t = threadIdx.x;
    t.threads = blockDim.x;
    t.wpad = next_pow2(blockDim.x / 32);
    t.red = sm;
    t.nvec = nvec;
    t.gsm = sm + 128 + threadIdx.y * 2 * (nvec + a.groups);
    t.buf = 0;
    return t;
}

// z -> norm(z) over each group (or the row), in place; r[i] the reciprocal root of vector i's group.
template <int VEC, int NV>
__device__ __forceinline__ void normalise(float (&z)[NV][VEC], float (&r)[NV], RowTeam<NV> &tm, const NormArgs &a,
                                          bool grouped, const int (&grp)[NV], int active) {
    const float inv = 1.0f / (float)(grouped ? a.cols / a.groups : a.cols);
    float2 s[NV];
    auto sum = [&]() {
        if (grouped) {
            tm.group_sum(s, a, grp, false);
        } else {
            float2 q = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i) { q.x += s[i].x; q.y += s[i].y; }
            q = tm.row_sum(q, false);
#pragma unroll
            for (int i = 0; i < NV; ++i) s[i] = q;
        }
    };
    if (a.layer) {
#pragma unroll
        for (int i = 0; i < NV; ++i) s[i] = make_float2(V<VEC>::sum(z[i]), 0.f);
        sum();
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < active)
#pragma unroll
                for (int e = 0; e < VEC; ++e) z[i][e] -= s[i].x * inv;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) s[i] = make_float2(V<VEC>::dot(z[i], z[i]), 0.f);
    sum();
    // (a vector past the row's end may be a group of its own, whose root of 0 + eps with eps = 0 has no reciprocal)
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        r[i] = i < active ? rsqrtf(fmaf(s[i].x, inv, a.eps)) : 0.0f;
        V<VEC>::mul(z[i], z[i], r[i]);
    }
}

// A thread's part of one row of a matrix, as loaded; zeros for an absent matrix and past the row's end.
template <typename IO, int VEC, int NV> struct RowPart {
    typename Vec<IO, VEC>::Raw raw[NV];
    __device__ __forceinline__ RowPart() {
#pragma unroll
        for (int i = 0; i < NV; ++i) memset(&raw[i], 0, sizeof(raw[i]));
    }
    __device__ __forceinline__ void fetch(const void *p, int64_t off, int t, int threads, int active) {
        if (!p) return;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < active)
                raw[i] = *reinterpret_cast<const typename Vec<IO, VEC>::Raw *>(static_cast<const IO *>(p) + off +
                                                                              (int64_t)(t + i * threads) * VEC);
    }
    __device__ __forceinline__ void get(float (&v)[NV][VEC]) const {
#pragma unroll
        for (int i = 0; i < NV; ++i) Vec<IO, VEC>::unpack(raw[i], v[i]);
    }
};

template <typename IO, int VEC, int NV>
__device__ __forceinline__ void store_row(void *p, int64_t off, const float (&v)[NV][VEC], int t, int threads, int active) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i < active) Vec<IO, VEC>::store(static_cast<IO *>(p) + off + (int64_t)(t + i * threads) * VEC, v[i]);
}

// Vectors of this thread (0 .. NV) and their groups.
template <int VEC, int NV>
__device__ __forceinline__ int my_vectors(const NormArgs &a, int nvec, int (&grp)[NV]) {
    int active = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int q = threadIdx.x + i * blockDim.x;
        if (q < nvec) active = i + 1;
        grp[i] = a.gmode == 2 ? min(q / a.gvec, a.groups - 1) : 0;
    }
    return active;
}

template <typename IO, int VEC, int NV>
__global__ void __launch_bounds__(limits(VEC, NV, false).threads, limits(VEC, NV, false).resident / limits(VEC, NV, false).threads)
    k_norm_fwd(NormArgs a) {
    extern __shared__ float sm[];
    const int nvec = a.cols / VEC;
    RowTeam<NV> tm = make_team<NV>(a, nvec, sm);
    int grp[NV];
    const int active = my_vectors<VEC, NV>(a, nvec, grp);
    const int t = tm.t, T = tm.threads;
    // the next row is on its way while this one is worked on
    constexpr bool AHEAD = VEC > 1 && NV <= 2;
    RowPart<IO, VEC, NV> px, py, pg;
    auto fetch = [&](int64_t row) {
        px.fetch(a.x, row * a.ldx, t, T, active);
        py.fetch(a.y, row * a.ldy, t, T, active);
        pg.fetch(a.gate, row * a.ldgate, t, T, active);
    };
    const int64_t slots = (int64_t)gridDim.x * blockDim.y;
    int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (AHEAD && row < a.rows) fetch(row);
    for (; row < a.rows; row += slots) {
        if (!AHEAD) fetch(row);
        float z[NV][VEC], x[NV][VEC], g[NV][VEC], r[NV];
        px.get(x);
        py.get(z);
        pg.get(g);
        if (AHEAD && row + slots < a.rows) fetch(row + slots);
        if (a.y) {
            if (a.w_post) {
                normalise<VEC, NV>(z, r, tm, a, true, grp, active);
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (i < active) {
                        const int c = (tm.t + i * tm.threads) * VEC;
                        float w[VEC];
                        load_w<VEC>(a.w_post, c, w);
                        V<VEC>::mul(z[i], z[i], w);
                        if (a.b_post) {
                            load_w<VEC>(a.b_post, c, w);
                            V<VEC>::add(z[i], z[i], w);
                        }
                    }
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                apply_gate<VEC>(a.act, g[i], z[i]);
                V<VEC>::fma(z[i], z[i], a.alpha, x[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) z[i][e] = x[i][e];
        }
        if (a.X) store_row<IO, VEC, NV>(a.X, row * a.ldX, z, tm.t, tm.threads, active);
        if (a.w_pre) {
            normalise<VEC, NV>(z, r, tm, a, false, grp, active);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < active) {
                    const int c = (tm.t + i * tm.threads) * VEC;
                    float w[VEC];
                    load_w<VEC>(a.w_pre, c, w);
                    V<VEC>::mul(z[i], z[i], w);
                    if (a.b_pre) {
                        load_w<VEC>(a.b_pre, c, w);
                        V<VEC>::add(z[i], z[i], w);
                    }
                }
            store_row<IO, VEC, NV>(a.H, row * a.ldH, z, tm.t, tm.threads, active);
        }
    }
}

// d -> the gradient of norm's input: r (d - zhat mean(d zhat) - [layer] mean(d)).
template <int VEC, int NV>
__device__ __forceinline__ void normalise_grad(float (&d)[NV][VEC], const float (&zhat)[NV][VEC], const float (&r)[NV],
                                               RowTeam<NV> &tm, const NormArgs &a, bool grouped, const int (&grp)[NV],
                                               int active) {
    const int count = grouped ? a.cols / a.groups : a.cols;
    if (count == 1) {  // the difference below cancels to r d (1 - zhat^2) = r d eps r^2, or to 0 without the mean
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) d[i][e] = a.layer ? 0.0f : d[i][e] * r[i] * (a.eps * r[i] * r[i]);
        return;
    }
    const float inv = 1.0f / (float)count;
    float2 s[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        s[i] = make_float2(V<VEC>::dot(d[i], zhat[i]), a.layer ? V<VEC>::sum(d[i]) : 0.0f);
    }
    if (grouped) {
        tm.group_sum(s, a, grp, a.layer);
    } else {
        float2 q = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i) { q.x += s[i].x; q.y += s[i].y; }
        q = tm.row_sum(q, a.layer);
#pragma unroll
        for (int i = 0; i < NV; ++i) s[i] = q;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const float mz = s[i].x * inv, md = a.layer ? s[i].y * inv : 0.0f;
        if (i < active) {
            if (a.layer)
#pragma unroll
                for (int e = 0; e < VEC; ++e) d[i][e] -= md;
            V<VEC>::fma(d[i], zhat[i], -mz, d[i]);
            V<VEC>::mul(d[i], d[i], r[i]);
        }
    }
}

// BIAS: the biases' gradients are summed too.
template <typename IO, int VEC, int NV, bool BIAS>
__global__ void __launch_bounds__(limits(VEC, NV, true).threads, limits(VEC, NV, true).resident / limits(VEC, NV, true).threads)
    k_norm_bwd(NormArgs a) {
    extern __shared__ float sm[];
    const int nvec = a.cols / VEC;
    RowTeam<NV> tm = make_team<NV>(a, nvec, sm);
    int grp[NV];
    const int active = my_vectors<VEC, NV>(a, nvec, grp);
    const int t = tm.t, T = tm.threads;
    float sw_post[NV][VEC], sw_pre[NV][VEC], sb_post[BIAS ? NV : 1][VEC], sb_pre[BIAS ? NV : 1][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            sw_post[i][e] = sw_pre[i][e] = 0.0f;
            if (BIAS) sb_post[i][e] = sb_pre[i][e] = 0.0f;
        }
    const int64_t slots = (int64_t)gridDim.x * blockDim.y, slot = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    constexpr bool AHEAD = VEC > 1 && NV == 1;  // as in the forward pass, where the registers suffice
    RowPart<IO, VEC, NV> px, py, pg, pdX, pdH;
    auto fetch = [&](int64_t row) {
        py.fetch(a.y, row * a.ldy, t, T, active);
        pg.fetch(a.gate, row * a.ldgate, t, T, active);
        px.fetch(a.x, row * a.ldx, t, T, active);
        pdX.fetch(a.dX, row * a.lddX, t, T, active);
        pdH.fetch(a.dH, row * a.lddH, t, T, active);
    };
    if (AHEAD && slot < a.rows) fetch(slot);
    for (int64_t row = slot; row < a.rows; row += slots) {
        if (!AHEAD) fetch(row);
        float z[NV][VEC], g[NV][VEC], x[NV][VEC], d[NV][VEC], dh[NV][VEC], ry[NV], rx[NV];
        py.get(z);
        pg.get(g);
        px.get(x);
        pdX.get(d);
        pdH.get(dh);
        if (AHEAD && row + slots < a.rows) fetch(row + slots);
        if (a.y && a.w_post) normalise<VEC, NV>(z, ry, tm, a, true, grp, active);
        // u (kept in place of y where there is no norm), and the gate's value and slope in place of the gate
        float u[NV][VEC], act[NV][VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) u[i][e] = z[i][e];
            if (a.w_post && i < active) {
                const int c = (t + i * T) * VEC;
                float w[VEC];
                load_w<VEC>(a.w_post, c, w);
                V<VEC>::mul(u[i], u[i], w);
                if (a.b_post) {
                    load_w<VEC>(a.b_post, c, w);
                    V<VEC>::add(u[i], u[i], w);
                }
            }
            gate_and_slope<VEC>(a.act, g[i], act[i]);
        }
        if (a.w_pre) {
            if (a.y) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (i < active) {
                        float v[VEC];
                        V<VEC>::mul(v, u[i], act[i]);
                        V<VEC>::fma(x[i], v, a.alpha, x[i]);
                    }
            }
            // without a mean, norm's statistic and the sum that its gradient needs are one reduction over x':
            // sum d xhat = r sum d x'
            const bool fused = !a.layer && a.cols > 1;
            float mz = 0.0f;
            if (!fused) {
                normalise<VEC, NV>(x, rx, tm, a, false, grp, active);
            } else {
                float2 q = make_float2(0.f, 0.f);
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (i < active) {
                        float w[VEC];
                        load_w<VEC>(a.w_pre, (t + i * T) * VEC, w);
                        V<VEC>::mul(w, w, dh[i]);
                        q.x += V<VEC>::dot(x[i], x[i]);
                        q.y += V<VEC>::dot(x[i], w);
                    }
                q = tm.row_sum(q, true);
                const float inv = 1.0f / (float)a.cols, r = rsqrtf(fmaf(q.x, inv, a.eps));
                mz = q.y * r * inv;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    rx[i] = r;
                    V<VEC>::mul(x[i], x[i], r);
                }
            }
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < active) {
                    float w[VEC];
                    load_w<VEC>(a.w_pre, (t + i * T) * VEC, w);
                    V<VEC>::fma(sw_pre[i], dh[i], x[i], sw_pre[i]);
                    if (BIAS) V<VEC>::add(sb_pre[i], sb_pre[i], dh[i]);
                    V<VEC>::mul(dh[i], dh[i], w);
                }
            if (!fused) {
                normalise_grad<VEC, NV>(dh, x, rx, tm, a, false, grp, active);
#pragma unroll
                for (int i = 0; i < NV; ++i) V<VEC>::add(d[i], d[i], dh[i]);
            } else {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    V<VEC>::fma(dh[i], x[i], -mz, dh[i]);
                    V<VEC>::fma(d[i], dh[i], rx[i], d[i]);
                }
            }
        }
        if (a.dx) store_row<IO, VEC, NV>(a.dx, row * a.lddx, d, t, T, active);
        if (!a.y) continue;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < active) {
                float dg[VEC];
                V<VEC>::mul(d[i], d[i], a.alpha);
                if (a.gate) {
                    V<VEC>::mul(dg, d[i], u[i]);
                    V<VEC>::mul(dg, dg, g[i]);
                    V<VEC>::mul(d[i], d[i], act[i]);
                    Vec<IO, VEC>::store(static_cast<IO *>(a.dgate) + row * a.lddgate + (int64_t)(t + i * T) * VEC, dg);
                }
                if (a.w_post) {
                    float w[VEC];
                    load_w<VEC>(a.w_post, (t + i * T) * VEC, w);
                    V<VEC>::fma(sw_post[i], d[i], z[i], sw_post[i]);
                    if (BIAS) V<VEC>::add(sb_post[i], sb_post[i], d[i]);
                    V<VEC>::mul(d[i], d[i], w);
                }
            }
        if (a.w_post) normalise_grad<VEC, NV>(d, z, ry, tm, a, true, grp, active);
        store_row<IO, VEC, NV>(a.dy, row * a.lddy, d, t, T, active);
    }
    // this slot's sums: [dw_post | dw_pre | db_post | db_pre] of a row's columns
    if (a.part) {
        float *p = a.part + slot * (BIAS ? 4 : 2) * a.cols;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < active)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int c = (t + i * T) * VEC + e;
                    p[c] = sw_post[i][e];
                    p[a.cols + c] = sw_pre[i][e];
                    if (BIAS) {
                        p[2 * a.cols + c] = sb_post[i][e];
                        p[3 * a.cols + c] = sb_pre[i][e];
                    }
                }
    }
}

struct NormSum {
    const float *part;
    float *out[4];
    int slots, arrays, cols;
};

// Sums the slots of 32 columns of one array: eight warps take slots w, w + 8, ..., joined in order.
__global__ void __launch_bounds__(256) k_norm_sum(NormSum a) {
    __shared__ float s[8][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, arr = blockIdx.y;
    float *out = a.out[arr];
    if (!out) return;
    float acc = 0.0f;
    if (c < a.cols) {
        const float *p = a.part + (int64_t)arr * a.cols + c;
#pragma unroll 4
        for (int i = w; i < a.slots; i += 8) acc += p[(int64_t)i * a.arrays * a.cols];
    }
    s[w][lane] = acc;
    __syncthreads();
    if (w == 0 && c < a.cols) {
#pragma unroll
        for (int i = 1; i < 8; ++i) acc += s[i][lane];
        out[c] = acc;
    }
}

// ---------------------------------------------------------------------------

// Vectors of a group from which a row may go to the kernels for wide rows (8192 bf16 columns, backward: groups of
// 64 vectors 242 us against 296, of 16 vectors 390 against 252; not aligned, registers cost four times as much).
constexpr int wide_group(bool vectors) { return vectors ? 32 : 8; }

struct Shape {
    int vec, nv, threads, rows_per_block, blocks;
    size_t smem;
    bool wide, shared;   // the kernels for wide rows; sums of the weight gradients in shared memory
};

// The fewest vectors a thread with which a row fits its threads.  A row of at most 32 vectors is a warp's.
// Rows that would take more values a thread than its registers hold go to the kernels for wide rows, unless
// their groups are narrow (a warp takes a group at a time).  Aligned rows keep to registers in the forward pass,
// which needs fewer (4104 bf16 columns 48 us against 104).
Shape shape_of(int cols, int groups, bool vectors, int vec_io, bool backward, bool bias) {
    Shape s;
    s.wide = s.shared = false;
    s.vec = vectors ? vec_io : 1;
    const int nvec = cols / s.vec;
    s.nv = vectors ? 1 : 4;
    while (s.nv < (vectors ? 4 : 32) && nvec > s.nv * limits(s.vec, s.nv, backward).threads) s.nv *= vectors ? 2 : 8;
    if (s.nv * s.vec > (vectors ? 8 : 4) && (backward || !vectors) && nvec / groups >= wide_group(vectors)) {
        const size_t row = sizeof(float) * wide_floats(cols, groups);
        const size_t sums = sizeof(float) * (cols + 3) / 4 * 4 * (bias ? 4 : 2);
        s.wide = true;
        s.shared = backward && row + sums <= 200 * 1024;
        s.smem = row + (s.shared ? sums : 0);
        s.rows_per_block = 1;
        s.threads = s.smem <= 100 * 1024 ? 512 : 1024;
        s.blocks = tc_sm_count() * (s.threads == 512 ? 2 : 1);
        return s;
    }
    s.threads = ((nvec + s.nv - 1) / s.nv + 31) / 32 * 32;
    s.rows_per_block = s.threads == 32 ? 8 : 1;
    s.blocks = tc_sm_count() * std::max(1, limits(s.vec, s.nv, backward).resident / (s.threads * s.rows_per_block));
    s.smem = sizeof(float) * 128;
    return s;
}

// Blocks that stay for all rows: no more than the device holds at once.
int grid_of(int64_t rows, const Shape &sh) {
    return (int)std::min<int64_t>(sh.blocks, (rows + sh.rows_per_block - 1) / sh.rows_per_block);
}

void group_mode(NormArgs &a, Shape &s) {
    a.gmode = 0;
    a.gvec = a.cols / s.vec / a.groups;
    if (a.w_post && a.groups > 1) {
        a.gmode = a.gvec <= 32 && (a.gvec & (a.gvec - 1)) == 0 ? 1 : 2;
        if (a.gmode == 2) s.smem += sizeof(float) * 2 * s.rows_per_block * (a.cols / s.vec + a.groups);
    }
}

bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

bool vectors_ok(const NormArgs &a, int vec) {
    if (a.cols % vec || (a.w_post && (a.cols / a.groups) % vec)) return false;
    for (const void *p : {a.w_post, a.b_post, a.w_pre, a.b_pre})
        if (!al16(p)) return false;
    // (the leading dimension of a matrix that the call does not have means nothing)
    const struct { const void *p; int64_t ld; } rows[] = {{a.x, a.ldx}, {a.y, a.ldy}, {a.gate, a.ldgate}, {a.X, a.ldX},
                                                          {a.H, a.ldH}, {a.dX, a.lddX}, {a.dH, a.lddH}, {a.dx, a.lddx},
                                                          {a.dy, a.lddy}, {a.dgate, a.lddgate}};
    for (const auto &r : rows)
        if (r.p && (!al16(r.p) || r.ld % vec)) return false;
    return true;
}

template <typename K>
cudaError_t big_smem(K kernel, size_t smem) {
    if (smem <= 48 * 1024) return cudaSuccess;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
}

template <typename IO, int VEC, int NV>
cudaError_t fwd_launch(const NormArgs &a, const Shape &sh, cudaStream_t s) {
    cudaError_t e = big_smem(k_norm_fwd<IO, VEC, NV>, sh.smem);
    if (e != cudaSuccess) return e;
    const int grid = grid_of(a.rows, sh);
    LUNA_LAUNCH("norm_fwd", (k_norm_fwd<IO, VEC, NV>), grid, dim3(sh.threads, sh.rows_per_block), sh.smem, s, a);
    return cudaGetLastError();
}

template <typename IO, int VECIO>
cudaError_t fwd(NormArgs a, cudaStream_t s) {
    const bool v = vectors_ok(a, VECIO);
    Shape sh = shape_of(a.cols, a.w_post ? a.groups : 1, v, VECIO, false, false);
    if (sh.wide)
        return launch_norm_fwd_wide(a, IOType<IO>::code, vectors_ok(a, 2), grid_of(a.rows, sh), sh.threads, sh.smem, s);
    group_mode(a, sh);
    if (v) {
        if (sh.nv == 1) return fwd_launch<IO, VECIO, 1>(a, sh, s);
        if (sh.nv == 2) return fwd_launch<IO, VECIO, 2>(a, sh, s);
        return fwd_launch<IO, VECIO, 4>(a, sh, s);
    }
    if (sh.nv == 4) return fwd_launch<IO, 1, 4>(a, sh, s);
    return fwd_launch<IO, 1, 32>(a, sh, s);
}

template <typename IO, int VEC, int NV, bool BIAS>
cudaError_t bwd_launch(const NormArgs &a, const Shape &sh, int grid, cudaStream_t s) {
    cudaError_t e = big_smem(k_norm_bwd<IO, VEC, NV, BIAS>, sh.smem);
    if (e != cudaSuccess) return e;
    LUNA_LAUNCH("norm_bwd", (k_norm_bwd<IO, VEC, NV, BIAS>), grid, dim3(sh.threads, sh.rows_per_block), sh.smem, s, a);
    return cudaGetLastError();
}

template <typename IO, int VECIO, bool BIAS>
cudaError_t bwd(NormArgs a, float *const (&out)[4], cudaStream_t s) {
    const bool v = vectors_ok(a, VECIO);
    Shape sh = shape_of(a.cols, a.w_post ? a.groups : 1, v, VECIO, true, BIAS);
    if (!sh.wide) group_mode(a, sh);
    const int grid = grid_of(a.rows, sh);
    cudaError_t e;
    if (sh.wide) {
        e = launch_norm_bwd_wide(a, IOType<IO>::code, v ? VECIO : vectors_ok(a, 2) ? 2 : 1, BIAS, sh.shared, grid, sh.threads,
                                 sh.smem, s);
    } else if (v) {
        if (sh.nv == 1) e = bwd_launch<IO, VECIO, 1, BIAS>(a, sh, grid, s);
        else if (sh.nv == 2) e = bwd_launch<IO, VECIO, 2, BIAS>(a, sh, grid, s);
        else e = bwd_launch<IO, VECIO, 4, BIAS>(a, sh, grid, s);
    } else {
        if (sh.nv == 4) e = bwd_launch<IO, 1, 4, BIAS>(a, sh, grid, s);
        else e = bwd_launch<IO, 1, 32, BIAS>(a, sh, grid, s);
    }
    if (e != cudaSuccess || !a.part) return e;
    NormSum n{a.part, {out[0], out[1], out[2], out[3]}, grid * sh.rows_per_block, BIAS ? 4 : 2, a.cols};
    LUNA_LAUNCH("norm_sum", k_norm_sum, dim3((a.cols + 31) / 32, BIAS ? 4 : 2), 256, 0, s, n);
    return cudaGetLastError();
}

luna_status check(const luna_norm_desc *nd) {
    if (!nd) return LUNA_ERR_INVALID_ARG;
    if (nd->rows < 0 || nd->cols < 1 || nd->groups < 1 || nd->cols % nd->groups) return LUNA_ERR_INVALID_ARG;
    if (nd->kind != LUNA_NORM_RMS && nd->kind != LUNA_NORM_LAYER) return LUNA_ERR_INVALID_ARG;
    if (nd->gate < LUNA_GATE_NONE || nd->gate > LUNA_GATE_SILU) return LUNA_ERR_INVALID_ARG;
    if (nd->io != LUNA_F32 && nd->io != LUNA_BF16) return LUNA_ERR_INVALID_ARG;
    if (!(nd->eps >= 0.0f) || isinf(nd->eps) || !isfinite(nd->alpha)) return LUNA_ERR_INVALID_ARG;
    for (int64_t ld : {nd->ldx, nd->ldy, nd->ldgate, nd->ldX, nd->ldH, nd->lddX, nd->lddH, nd->lddx, nd->lddy, nd->lddgate})
        if (ld != 0 && ld < nd->cols) return LUNA_ERR_INVALID_ARG;
    if (nd->cols > kMaxCols || nd->rows > (int64_t(1) << 31) - 1) return LUNA_ERR_UNSUPPORTED;
    return LUNA_OK;
}

NormArgs args(const luna_norm_desc *nd, const void *x, const void *y, const void *gate, const float *w_post,
              const float *b_post, const float *w_pre, const float *b_pre) {
    NormArgs a;
    memset(&a, 0, sizeof(a));
    a.x = x; a.y = y;
    a.gate = nd->gate == LUNA_GATE_NONE ? nullptr : gate;
    a.w_post = w_post; a.b_post = b_post; a.w_pre = w_pre; a.b_pre = b_pre;
    a.rows = nd->rows; a.cols = nd->cols; a.groups = nd->groups;
    a.layer = nd->kind == LUNA_NORM_LAYER; a.act = nd->gate;
    a.alpha = nd->alpha; a.eps = nd->eps;
    auto ld = [&](int64_t v) { return v ? v : (int64_t)nd->cols; };
    a.ldx = ld(nd->ldx); a.ldy = ld(nd->ldy); a.ldgate = ld(nd->ldgate); a.ldX = ld(nd->ldX); a.ldH = ld(nd->ldH);
    a.lddX = ld(nd->lddX); a.lddH = ld(nd->lddH); a.lddx = ld(nd->lddx); a.lddy = ld(nd->lddy);
    a.lddgate = ld(nd->lddgate);
    return a;
}

// The combinations a call may ask for: something to norm or add, a gate and a post-norm only with y.
bool combination_ok(const luna_norm_desc *nd, const void *x, const void *y, const void *gate, const float *w_post,
                    const float *b_post, const float *w_pre, const float *b_pre) {
    if (!x && !y) return false;
    if (!y && (w_post || nd->gate != LUNA_GATE_NONE)) return false;
    if (nd->gate != LUNA_GATE_NONE && !gate) return false;
    if ((b_post && !w_post) || (b_pre && !w_pre)) return false;
    return true;
}

// The partial sums of the launch shape with vectors or without, whichever has more.
size_t partial_bytes(const luna_norm_desc *nd) {
    size_t slots = 0;
    for (int form = 0; form < 8; ++form) {
        const Shape sh = shape_of(nd->cols, form & 1 ? nd->groups : 1, form & 2, nd->io == LUNA_F32 ? 4 : 8, true, form & 4);
        slots = std::max(slots, (size_t)grid_of(nd->rows, sh) * sh.rows_per_block);
    }
    return slots * 4 * nd->cols * sizeof(float);
}

luna_status cuda_status(cudaError_t e) { return e == cudaSuccess ? LUNA_OK : LUNA_ERR_CUDA; }

}  // namespace
}  // namespace luna

using namespace luna;

extern "C" {

luna_status luna_norm_workspace_size(const luna_norm_desc *nd, size_t *bytes) {
    if (!bytes) return LUNA_ERR_INVALID_ARG;
    const luna_status st = check(nd);
    if (st != LUNA_OK) return st;
    *bytes = nd->rows ? (size_t)align256((int64_t)partial_bytes(nd)) : 256;
    return LUNA_OK;
}

luna_status luna_norm_fwd(const luna_norm_desc *nd, const void *x, const void *y, const void *gate,
                          const float *w_post, const float *b_post, const float *w_pre, const float *b_pre, void *X,
                          void *H, void *stream) {
    const luna_status st = check(nd);
    if (st != LUNA_OK) return st;
    if (nd->rows == 0) return LUNA_OK;
    if (!combination_ok(nd, x, y, gate, w_post, b_post, w_pre, b_pre)) return LUNA_ERR_INVALID_ARG;
    if ((w_pre && !H) || (!w_pre && !X)) return LUNA_ERR_INVALID_ARG;
    NormArgs a = args(nd, x, y, gate, w_post, b_post, w_pre, b_pre);
    a.X = X;
    a.H = w_pre ? H : nullptr;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return cuda_status(nd->io == LUNA_F32 ? fwd<float, 4>(a, s) : fwd<__nv_bfloat16, 8>(a, s));
}

luna_status luna_norm_bwd(const luna_norm_desc *nd, const void *x, const void *y, const void *gate,
                          const float *w_post, const float *b_post, const float *w_pre, const void *dX, const void *dH,
                          void *dx, void *dy, void *dgate, float *dw_post, float *db_post, float *dw_pre,
                          float *db_pre, void *workspace, size_t ws_bytes, void *stream) {
    const luna_status st = check(nd);
    if (st != LUNA_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    float *const out[4] = {dw_post, dw_pre, db_post, db_pre};
    if (nd->rows == 0) {  // sums over no rows
        for (float *p : out)
            if (p && cudaMemsetAsync(p, 0, sizeof(float) * nd->cols, s) != cudaSuccess) return LUNA_ERR_CUDA;
        return LUNA_OK;
    }
    if (!combination_ok(nd, x, y, gate, w_post, b_post, w_pre, nullptr)) return LUNA_ERR_INVALID_ARG;
    if ((w_pre && !dH) || (!w_pre && !dX)) return LUNA_ERR_INVALID_ARG;
    if ((x && !dx) || (y && !dy) || (nd->gate != LUNA_GATE_NONE && !dgate)) return LUNA_ERR_INVALID_ARG;
    if (((dw_post || db_post) && !w_post) || ((dw_pre || db_pre) && !w_pre)) return LUNA_ERR_INVALID_ARG;
    const bool sums = dw_post || db_post || dw_pre || db_pre;
    if (sums && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255))) return LUNA_ERR_INVALID_ARG;
    if (sums && ws_bytes < partial_bytes(nd)) return LUNA_ERR_WORKSPACE;
    NormArgs a = args(nd, x, y, gate, w_post, b_post, w_pre, nullptr);
    a.dX = dX;
    a.dH = w_pre ? dH : nullptr;
    a.dx = x ? dx : nullptr; a.dy = y ? dy : nullptr; a.dgate = a.gate ? dgate : nullptr;
    a.part = sums ? static_cast<float *>(workspace) : nullptr;
    const bool bias = db_post || db_pre;
    cudaError_t e;
    if (nd->io == LUNA_F32)
        e = bias ? bwd<float, 4, true>(a, out, s) : bwd<float, 4, false>(a, out, s);
    else
        e = bias ? bwd<__nv_bfloat16, 8, true>(a, out, s) : bwd<__nv_bfloat16, 8, false>(a, out, s);
    return cuda_status(e);
}

}  // extern "C"
