// The gated delta rule in fp32, on CUDA cores: the recurrence four rows at a time, its gradients by chunk; and single
// tokens of either type.
#include <math.h>

#include "luna_delta.cuh"
#include "luna_prof.cuh"

namespace luna {
int tc_sm_count();

namespace {

// ---------------------------------------------------------------------------
// The recurrence, forward (S, from which u and o) and in reverse (R, from which x and dV).
//
// A column of the state takes part in no other: eight lanes hold one column, 16 values each at d = 128.  Four rows go at a time: their dot products with the state before them are summed over the
// eight lanes together, and what they do to each other is known from the dot products of the rows themselves:
//
//     u_i = b_i (v_i - A_i k_i . S - sum_{j < i} M_ij u_j),   o_i = scale (A_i q_i . S + sum_{j <= i} N_ij u_j)
//     S <- A S + sum_j L_j k_j u_j
//
// with A_i = exp(g_0 + .. + g_i), M_ij and N_ij = exp(g_{j+1} + .. + g_i) times k_i . k_j and q_i . k_j.  In reverse the
// rows of the four count from the last, G_i is scale dO_i, N_ij from k_i . q_j, a row's decay comes behind it, and
//
//     x_i = A_i k_i . R + sum_{j <= i} N_ij G_j - sum_{j < i} M_ij b_j x_j,   R <- A R + sum_j L_j (q_j G_j - b_j k_j x_j)
//
// Rows come in tiles of 16 through shared memory.  A warp carries four columns; four more warps of a block fetch the tile after the next,
// work out the rows' own products of the next and write the outputs of the one before, so that the columns' warps, whose
// chain bounds the pass, do nothing else: 199 ns a row at d = 128 (with all of that in the same warps 430 ns, whether four
// rows go at a time or one).

constexpr int kLoaders = 128, kTile = 16, kFour = 4;

struct Four {  // of four rows
    float b[kFour], A[kFour], L[kFour], M[kFour][kFour], N[kFour][kFour], all, rest;
};

// sums over the eight lanes of a column
__device__ __forceinline__ float lanes8(float x) {
    x += __shfl_xor_sync(0xffffffffu, x, 1);
    x += __shfl_xor_sync(0xffffffffu, x, 2);
    return x + __shfl_xor_sync(0xffffffffu, x, 4);
}

// a s + x for a in two terms, rounded once: where the state moves by a little at every row the same way, a rounding
// of a s alone would be off the same way at every row too (2e-4 of the state after 20000 rows of a = 1 - 1e-6).
__device__ __forceinline__ float decayed(float a, float rest, float s, float x) { return fmaf(a, s, fmaf(rest, s, x)); }

template <int JD, int COLS>
struct RowTile {
    float4 k[kTile][8 * JD + 1], q[kTile][8 * JD + 1];  // (the padding: rows start in different banks)
    float x[kTile][COLS], y[kTile][COLS], z[kTile][COLS], g[kTile];
    Four four[kTile / kFour];
};

template <int JD, bool REV, int COLS, int CPL>  // CPL: columns of a lane
__global__ void __launch_bounds__(COLS / CPL * 8 + kLoaders, JD == 4 ? 2 : 3) k_delta_rows(DeltaArgs a) {
    constexpr int DP = 32 * JD, PER = kTile * DP / kLoaders;  // padded width; values of k (and q) a loader fetches
    constexpr int XPER = kTile * COLS / kLoaders;             // of v or dO
    __shared__ RowTile<JD, COLS> tile_[2];
    constexpr int CARRY = COLS / CPL * 8;                     // threads that carry the columns
    const bool loads = threadIdx.x >= CARRY;
    const int tid = loads ? threadIdx.x - CARRY : threadIdx.x, p = tid % 8, cl = tid / 8;
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / a.H), h = (int)(bh % a.H), col0 = blockIdx.y * COLS;
    const int len = head_length(a.lengths, b, a.n), tiles = (len + kTile - 1) / kTile;
    const int64_t E = (int64_t)a.d * a.dv;
    const RowView &xv = REV ? a.go : a.v;
    float *o = a.o ? static_cast<float *>(a.o) + b * a.ob + h * a.oh : nullptr;
    if (!REV && bh == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.status = 0;  // (the call's first kernel; none of this form sets it)
    auto tile_of = [&](int step) { return REV ? tiles - 1 - step : step; };
    auto at = [](int f, int i) { return f * kFour + (REV ? kFour - 1 - i : i); };  // rows of a four in the order they are taken

    if (loads) {
        const int hk = h / (a.H / a.k.heads);
        const float *k = static_cast<const float *>(a.k.p) + b * a.k.sb + hk * a.k.sh;
        const float *q = static_cast<const float *>(a.q.p) + b * a.q.sb + hk * a.q.sh;
        const float *x = static_cast<const float *>(xv.p) + b * xv.sb + h * xv.sh;
        float *U = REV ? a.X : a.U;
        if (U) U += bh * a.n * a.dv;
        float nk[PER], nq[PER], nx[XPER], ng = 0.0f, nb = 0.0f;
        auto fetch = [&](int tile) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int w = tid + i * kLoaders, t = tile * kTile + w / DP, c = w % DP;
                const bool in = t < len && c < a.d;
                nk[i] = in ? k[t * a.k.st + c] : 0.0f;
                nq[i] = in ? q[t * a.q.st + c] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < XPER; ++i) {
                const int w = tid + i * kLoaders, t = tile * kTile + w / COLS, c = col0 + w % COLS;
                nx[i] = t < len && c < a.dv ? x[t * xv.st + c] : 0.0f;
            }
            if (tid < kTile) {
                const int t = tile * kTile + tid;
                ng = t < len ? gate_at<float>(a.g, b, h, t) : 0.0f;  // (behind the end: k = q = b = g = 0, which changes nothing)
                nb = t < len ? gate_at<float>(a.b, b, h, t) : 0.0f;
            }
        };
        // the fetched rows into a tile, and what its fours need
        auto prepare = [&](RowTile<JD, COLS> &sm) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int w = tid + i * kLoaders;
                reinterpret_cast<float *>(sm.k[w / DP])[w % DP] = nk[i];
                reinterpret_cast<float *>(sm.q[w / DP])[w % DP] = nq[i];
            }
#pragma unroll
            for (int i = 0; i < XPER; ++i) (&sm.x[0][0])[tid + i * kLoaders] = nx[i];
            if (tid < kTile) {
                sm.g[tid] = ng;
                sm.four[tid / kFour].b[REV ? kFour - 1 - tid % kFour : tid % kFour] = nb;
            }
            asm volatile("bar.sync 1, %0;" ::"n"(kLoaders) : "memory");
            // two threads a dot product: of the 16 of a four those with j <= i, k_i . k_j (j < i) and N's
            const int f = tid / 32, lane = tid % 32, i = lane / 8, j = lane / 2 % 4, part = lane % 2;
            Four &four = sm.four[f];
            float kk = 0.0f, nn = 0.0f;
            if (j <= i) {
                const float4 *ki = sm.k[at(f, i)], *kj = sm.k[at(f, j)], *qi = sm.q[at(f, REV ? j : i)];
#pragma unroll 4
                for (int c = part; c < DP / 4; c += 2) {
                    const float4 x4 = ki[c], y4 = kj[c], z4 = qi[c], w4 = REV ? x4 : y4;
                    kk = fmaf(x4.x, y4.x, fmaf(x4.y, y4.y, fmaf(x4.z, y4.z, fmaf(x4.w, y4.w, kk))));
                    nn = fmaf(w4.x, z4.x, fmaf(w4.y, z4.y, fmaf(w4.z, z4.z, fmaf(w4.w, z4.w, nn))));
                }
            }
            kk += __shfl_xor_sync(0xffffffffu, kk, 1);
            nn += __shfl_xor_sync(0xffffffffu, nn, 1);
            // gates between: forward those of j + 1 .. i, in reverse of j .. i - 1
            auto between = [&](int from, int to) {
                float sum = 0.0f;
#pragma unroll
                for (int r = 0; r < kFour; ++r)
                    if (r >= from && r < to) sum += sm.g[at(f, r)];
                return sum;
            };
            if (part == 0 && j <= i) {
                const float c = expf(REV ? between(j, i) : between(j + 1, i + 1));
                four.M[i][j] = c * kk;
                four.N[i][j] = REV ? a.scale * c * nn : c * nn;
            }
            if (lane < kFour) {
                four.A[lane] = expf(REV ? between(0, lane) : between(0, lane + 1));
                four.L[lane] = expf(REV ? between(lane, kFour) : between(lane + 1, kFour));
            }
            if (lane == kFour) gate_terms(between(0, kFour), four.all, four.rest);
        };
        auto write = [&](const RowTile<JD, COLS> &sm, int tile) {
#pragma unroll
            for (int i = 0; i < XPER; ++i) {
                const int w = tid + i * kLoaders, t = w / COLS, c = w % COLS;
                const int64_t r = tile * kTile + t;
                if (r < len && col0 + c < a.dv) {
                    if (o) o[r * a.ot + col0 + c] = sm.y[t][c];
                    if (U) U[r * a.dv + col0 + c] = sm.z[t][c];
                }
            }
        };
        if (tiles > 0) {
            fetch(tile_of(0));
            prepare(tile_[0]);
        }
        if (tiles > 1) fetch(tile_of(1));
        __syncthreads();
        for (int step = 0; step < tiles; ++step) {
            if (step > 0) write(tile_[(step - 1) & 1], tile_of(step - 1));
            if (step + 1 < tiles) prepare(tile_[(step + 1) & 1]);  // (which leaves y and z alone)
            if (step + 2 < tiles) fetch(tile_of(step + 2));
            __syncthreads();
        }
        if (tiles > 0) write(tile_[(tiles - 1) & 1], tile_of(tiles - 1));
        if (o)
            for (int64_t i = tid; i < (int64_t)(a.n - len) * COLS; i += kLoaders) {
                const int c = col0 + (int)(i % COLS);
                if (c < a.dv) o[(len + i / COLS) * a.ot + c] = 0.0f;
            }
        return;
    }

    float *ends = REV ? a.after : a.before;
    if (ends) ends += bh * (a.m + 1) * E;
    const float *init = REV ? a.dS1 : a.S0;
    float *last = REV ? a.dS0 : a.S1;
    float s[CPL][JD][4];  // of columns cl, cl + COLS / CPL, ..
    auto row = [&](int j, int e) { return j * 32 + p * 4 + e; };
    auto column = [&](int c) { return cl + c * (COLS / CPL); };
    auto keep = [&](float *to) {
#pragma unroll
        for (int c = 0; c < CPL; ++c)
            if (col0 + column(c) < a.dv)
#pragma unroll
                for (int j = 0; j < JD; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (row(j, e) < a.d) to[(int64_t)row(j, e) * a.dv + col0 + column(c)] = s[c][j][e];
    };
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
        for (int j = 0; j < JD; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = row(j, e), to = col0 + column(c);
                s[c][j][e] = init && to < a.dv && r < a.d ? init[bh * E + (int64_t)r * a.dv + to] : 0.0f;
            }
    constexpr int kTiles = kDeltaRows / kTile;  // of a chunk
    if (REV && ends) keep(ends + (int64_t)((len + kDeltaRows - 1) / kDeltaRows) * E);
    __syncthreads();
    for (int step = 0; step < tiles; ++step) {
        RowTile<JD, COLS> &sm = tile_[step & 1];
        const int tile = tile_of(step);
        if (!REV && ends && tile % kTiles == 0) keep(ends + (int64_t)(tile / kTiles) * E);
#pragma unroll 1
        for (int r = 0; r < kTile / kFour; ++r) {
            const int f = REV ? kTile / kFour - 1 - r : r;
            const Four &four = sm.four[f];
            float dk[CPL][kFour], dq[CPL][kFour], u[CPL][kFour];
#pragma unroll
            for (int i = 0; i < kFour; ++i) {
                float x0[CPL], x1[CPL], y0[CPL], y1[CPL];
#pragma unroll
                for (int c = 0; c < CPL; ++c) x0[c] = x1[c] = y0[c] = y1[c] = 0.0f;
#pragma unroll
                for (int j = 0; j < JD; ++j) {
                    const float4 kk = sm.k[at(f, i)][j * 8 + p];
#pragma unroll
                    for (int c = 0; c < CPL; ++c) {
                        x0[c] = fmaf(kk.x, s[c][j][0], fmaf(kk.y, s[c][j][1], x0[c]));
                        x1[c] = fmaf(kk.z, s[c][j][2], fmaf(kk.w, s[c][j][3], x1[c]));
                    }
                    if (!REV) {
                        const float4 qq = sm.q[at(f, i)][j * 8 + p];
#pragma unroll
                        for (int c = 0; c < CPL; ++c) {
                            y0[c] = fmaf(qq.x, s[c][j][0], fmaf(qq.y, s[c][j][1], y0[c]));
                            y1[c] = fmaf(qq.z, s[c][j][2], fmaf(qq.w, s[c][j][3], y1[c]));
                        }
                    }
                }
#pragma unroll
                for (int c = 0; c < CPL; ++c) {
                    dk[c][i] = x0[c] + x1[c];
                    dq[c][i] = y0[c] + y1[c];
                }
            }
#pragma unroll
            for (int c = 0; c < CPL; ++c)
#pragma unroll
                for (int i = 0; i < kFour; ++i) {
                    dk[c][i] = lanes8(dk[c][i]);
                    if (!REV) dq[c][i] = lanes8(dq[c][i]);
                }
#pragma unroll
            for (int c = 0; c < CPL; ++c)
#pragma unroll
                for (int i = 0; i < kFour; ++i) {
                    const float xc = sm.x[at(f, i)][column(c)];
                    float &y = sm.y[at(f, i)][column(c)], &z = sm.z[at(f, i)][column(c)];
                    if (!REV) {
                        float w = fmaf(-four.A[i], dk[c][i], xc);
#pragma unroll
                        for (int j = 0; j < i; ++j) w = fmaf(-four.M[i][j], u[c][j], w);
                        u[c][i] = four.b[i] * w;
                        float out = four.A[i] * dq[c][i];
#pragma unroll
                        for (int j = 0; j <= i; ++j) out = fmaf(four.N[i][j], u[c][j], out);
                        if (p == 0) { y = a.scale * out; z = u[c][i]; }
                    } else {
                        dq[c][i] = xc;  // (dO_i)
                        float w = four.A[i] * dk[c][i];
#pragma unroll
                        for (int j = 0; j <= i; ++j) w = fmaf(four.N[i][j], dq[c][j], w);
#pragma unroll
                        for (int j = 0; j < i; ++j) w = fmaf(-four.M[i][j], u[c][j], w);
                        u[c][i] = four.b[i] * w;
                        if (p == 0) { y = u[c][i]; z = w; }
                    }
                }
#pragma unroll
            for (int c = 0; c < CPL; ++c)
#pragma unroll
                for (int i = 0; i < kFour; ++i) {
                    dq[c][i] *= a.scale * four.L[i];
                    u[c][i] *= REV ? -four.L[i] : four.L[i];
                }
#pragma unroll
            for (int j = 0; j < JD; ++j) {
                float t[CPL][4];
#pragma unroll
                for (int c = 0; c < CPL; ++c) t[c][0] = t[c][1] = t[c][2] = t[c][3] = 0.0f;
#pragma unroll
                for (int i = 0; i < kFour; ++i) {
                    const float4 kk = sm.k[at(f, i)][j * 8 + p];
#pragma unroll
                    for (int c = 0; c < CPL; ++c) {
                        t[c][0] = fmaf(kk.x, u[c][i], t[c][0]); t[c][1] = fmaf(kk.y, u[c][i], t[c][1]);
                        t[c][2] = fmaf(kk.z, u[c][i], t[c][2]); t[c][3] = fmaf(kk.w, u[c][i], t[c][3]);
                    }
                    if (REV) {
                        const float4 qq = sm.q[at(f, i)][j * 8 + p];
#pragma unroll
                        for (int c = 0; c < CPL; ++c) {
                            t[c][0] = fmaf(qq.x, dq[c][i], t[c][0]); t[c][1] = fmaf(qq.y, dq[c][i], t[c][1]);
                            t[c][2] = fmaf(qq.z, dq[c][i], t[c][2]); t[c][3] = fmaf(qq.w, dq[c][i], t[c][3]);
                        }
                    }
                }
#pragma unroll
                for (int c = 0; c < CPL; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[c][j][e] = decayed(four.all, four.rest, s[c][j][e], t[c][e]);
            }
        }
        if (REV && ends && tile % kTiles == 0) keep(ends + (int64_t)(tile / kTiles) * E);
        __syncthreads();
    }
    if (!REV && ends) keep(ends + (int64_t)((len + kDeltaRows - 1) / kDeltaRows) * E);
    if (last) keep(last + bh * E);
}

// ---------------------------------------------------------------------------
// Gradients of q, k and the gates from the states at the two ends of a chunk: four products of 64 x 64 and seven of 64 rows by
// d columns, each thread with 4 rows and one or two times 4 columns of them, two multiply-adds an instruction.  The
// operands come from L2 in steps of 16 of the summed index; bound by that and its barriers: 102 us for 300 chunks of
// 40 x 72.  (91 us with a gate's gradient as a difference of sums over the rows, without the products q_i . k_j and
// k_i . k_j; of that form every 16th column a thread's and one multiply-add an instruction took 1.3 times as long.)

constexpr int kGradThreads = 256, kGradK = 16;

struct GradShared {
    alignas(16) float A[kGradK][kDeltaRows + 4], B[kGradK][kMaxD + 4];
    float P[kDeltaRows][kDeltaRows + 1], W[kDeltaRows][kDeltaRows + 1];
    float reads[kDeltaRows][kDeltaRows + 1];  // what row i reads of row j < i; then from row i to the chunk's end
    float hi[kDeltaRows], lo[kDeltaRows], b[kDeltaRows], past[kDeltaRows], left[kDeltaRows];
    float read[kDeltaRows], wrote[kDeltaRows], crossed[kDeltaRows], total[kGradThreads / 32];
};

// A thread's c-th column
__device__ __forceinline__ int grad_column(int tx, int c) { return tx * 4 + c % 4 + c / 4 * 64; }

// acc[r][c] += sum_k A(ty * 4 + r, k) B(k, grad_column(tx, c)); BT: B is stored with k contiguous
template <bool BT, int NC, typename FA, typename FB>
__device__ __forceinline__ void grad_product(GradShared &sm, float (&acc)[4][NC], int K, FA fa, FB fb) {
    const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    uint64_t two[4][NC / 2];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NC / 2; ++c) two[r][c] = f2(acc[r][2 * c], acc[r][2 * c + 1]);
    for (int k0 = 0; k0 < K; k0 += kGradK) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = k0 + tid % kGradK, r = tid / kGradK + 16 * i;
            sm.A[k - k0][r] = k < K ? fa(r, k) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int at = tid + i * kGradThreads;
            const int k = BT ? k0 + at % kGradK : k0 + at / (16 * NC), c = BT ? at / kGradK : at % (16 * NC);
            sm.B[k - k0][c] = k < K ? fb(k, c) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kGradK; ++k) {
            const float4 x = *reinterpret_cast<const float4 *>(&sm.A[k][ty * 4]);
            const uint64_t xx[4] = {f2(x.x, x.x), f2(x.y, x.y), f2(x.z, x.z), f2(x.w, x.w)};
#pragma unroll
            for (int c = 0; c < NC / 4; ++c) {
                const float4 y = *reinterpret_cast<const float4 *>(&sm.B[k][tx * 4 + c * 64]);
                const uint64_t lo = f2(y.x, y.y), hi = f2(y.z, y.w);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    two[r][2 * c] = fma2(xx[r], lo, two[r][2 * c]);
                    two[r][2 * c + 1] = fma2(xx[r], hi, two[r][2 * c + 1]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NC / 2; ++c) unpack2(two[r][c], acc[r][2 * c], acc[r][2 * c + 1]);
}

__global__ void __launch_bounds__(kGradThreads) k_delta_grad(DeltaArgs a) {
    extern __shared__ char raw[];
    GradShared &sm = *reinterpret_cast<GradShared *>(raw);
    constexpr int NC = kMaxD / 16, C = kDeltaRows;
    const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    const int64_t bh = blockIdx.x / a.m;
    const int chunk = (int)(blockIdx.x % a.m), b = (int)(bh / a.H), h = (int)(bh % a.H), t0 = chunk * C;
    const int len = head_length(a.lengths, b, a.n), rows = max(0, min(C, len - t0));
    const int hk = h / (a.H / a.k.heads);
    const float *q = static_cast<const float *>(a.q.p) + b * a.q.sb + hk * a.q.sh + t0 * a.q.st;
    const float *k = static_cast<const float *>(a.k.p) + b * a.k.sb + hk * a.k.sh + t0 * a.k.st;
    const float *v = static_cast<const float *>(a.v.p) + b * a.v.sb + h * a.v.sh + t0 * a.v.st;
    const float *go = static_cast<const float *>(a.go.p) + b * a.go.sb + h * a.go.sh + t0 * a.go.st;
    float *dq = static_cast<float *>(a.dq) + b * a.dqb + h * a.dqh + t0 * a.dqt;
    float *dk = static_cast<float *>(a.dk) + b * a.dkb + h * a.dkh + t0 * a.dkt;
    float *dg = static_cast<float *>(a.dg.p) + b * a.dg.sb + h * a.dg.sh + t0 * a.dg.st;
    float *db = static_cast<float *>(a.db.p) + b * a.db.sb + h * a.db.sh + t0 * a.db.st;
    const int out_rows = min(C, a.n - t0);
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
    const int64_t E = (int64_t)a.d * a.dv;
    const float *S = a.before + (bh * (a.m + 1) + chunk) * E, *R = a.after + (bh * (a.m + 1) + chunk + 1) * E;
    const float *U = a.U + (bh * a.n + t0) * a.dv, *X = a.X + (bh * a.n + t0) * a.dv;
    const int d = a.d, dv = a.dv;

    if (tid < 32)
        delta_gate_sums(tid, [&](int t) { return t < rows ? gate_at<float>(a.g, b, h, t0 + t) : 0.0f; }, sm.hi, sm.lo,
                        sm.past, sm.left);
    else if (tid < 32 + C)
        sm.b[tid - 32] = tid - 32 < rows ? gate_at<float>(a.b, b, h, t0 + tid - 32) : 0.0f;
    __syncthreads();
    auto gap = [&](int i, int j) { return expf((sm.hi[i] - sm.hi[j]) + (sm.lo[i] - sm.lo[j])); };
    auto at = [&](const float *x, int64_t st, int t, int c, int w) { return t < rows && c < w ? io_load(x + t * st + c) : 0.0f; };
    auto in = [&](const float *x, int t, int c) { return t < rows && c < dv ? x[(int64_t)t * dv + c] : 0.0f; };
    auto fK = [&](int kk, int c) { return at(k, a.k.st, kk, c, d); };
    auto fQ = [&](int kk, int c) { return at(q, a.q.st, kk, c, d); };
    auto zero = [](auto &acc) {
#pragma unroll
        for (auto &r : acc)
#pragma unroll
            for (auto &x : r) x = 0.0f;
    };
    // sums over the 16 threads of a row
    auto rowsum = [&](float x) {
#pragma unroll
        for (int w = 1; w < 16; w *= 2) x += __shfl_xor_sync(0xffffffffu, x, w);
        return x;
    };

    {  // P and W
        float acc[4][4];
        zero(acc);
        grad_product<true>(sm, acc, dv, [&](int r, int kk) { return at(go, a.go.st, r, kk, dv); }, [&](int kk, int c) { return in(U, c, kk); });
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int i = ty * 4 + r, j = grad_column(tx, c);
                sm.P[i][j] = j <= i ? a.scale * gap(i, j) * acc[r][c] : 0.0f;
            }
        zero(acc);
        grad_product<true>(sm, acc, dv, [&](int r, int kk) { return in(X, r, kk); }, [&](int kk, int c) { return in(U, c, kk); });
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int i = ty * 4 + r, j = grad_column(tx, c);
                sm.W[i][j] = j < i ? gap(i, j) * acc[r][c] : 0.0f;
            }
        // P_ij q_i . k_j - b_i W_ij k_i . k_j  (a thread's values of P, W and these are its own)
        zero(acc);
        grad_product<true>(sm, acc, d, [&](int r, int kk) { return at(q, a.q.st, r, kk, d); }, [&](int kk, int c) { return at(k, a.k.st, c, kk, d); });
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int i = ty * 4 + r, j = grad_column(tx, c);
                sm.reads[i][j] = j < i ? sm.P[i][j] * acc[r][c] : 0.0f;
            }
        zero(acc);
        grad_product<true>(sm, acc, d, [&](int r, int kk) { return at(k, a.k.st, r, kk, d); }, [&](int kk, int c) { return at(k, a.k.st, c, kk, d); });
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int i = ty * 4 + r, j = grad_column(tx, c);
                if (j < i) sm.reads[i][j] = fmaf(-sm.b[i] * sm.W[i][j], acc[r][c], sm.reads[i][j]);
            }
    }
    float acc[4][NC], z[4][NC];
    auto fS = [&](int kk, int c) { return c < d && kk < dv ? S[(int64_t)c * dv + kk] : 0.0f; };
    auto fR = [&](int kk, int c) { return c < d && kk < dv ? R[(int64_t)c * dv + kk] : 0.0f; };
    // dQ
    zero(acc);
    grad_product<true>(sm, acc, dv, [&](int r, int kk) { return at(go, a.go.st, r, kk, dv); }, fS);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[r][c] *= a.scale * sm.past[ty * 4 + r];
    auto dot = [&](const float *x, int64_t st, const float (&with)[4][NC], int r) {  // of row i = ty * 4 + r
        const int i = ty * 4 + r;
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (i < rows && grad_column(tx, c) < d) sum = fmaf(io_load(x + i * st + grad_column(tx, c)), with[r][c], sum);
        return rowsum(sum);
    };
    auto store = [&](float *to, int64_t st, const float (&from)[4][NC]) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (ty * 4 + r < rows && grad_column(tx, c) < d) io_store(to + (ty * 4 + r) * st + grad_column(tx, c), from[r][c]);
    };
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float of_s = dot(q, a.q.st, acc, r);
        if (tx == 0) sm.read[ty * 4 + r] = of_s;
    }
    grad_product<false>(sm, acc, C, [&](int r, int kk) { return sm.P[r][kk]; }, fK);
    store(dq, a.dqt, acc);
    // Z, and with it db
    zero(z);
    grad_product<true>(sm, z, dv, [&](int r, int kk) { return in(X, r, kk); }, fS);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) z[r][c] *= sm.past[ty * 4 + r];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float of_s = dot(k, a.k.st, z, r);
        if (tx == 0) sm.read[ty * 4 + r] -= sm.b[ty * 4 + r] * of_s;
    }
    grad_product<false>(sm, z, C, [&](int r, int kk) { return sm.W[r][kk]; }, fK);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = ty * 4 + r;
        float xv = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int cc = grad_column(tx, c);
            if (i < rows && cc < dv) xv = fmaf(io_load(v + i * a.v.st + cc), X[(int64_t)i * dv + cc], xv);
        }
        xv = rowsum(xv);
        const float kz = dot(k, a.k.st, z, r);
        if (tx == 0 && i < rows) io_store(db + i * a.db.st, xv - kz);
    }
    // dK
    zero(acc);
    grad_product<true>(sm, acc, dv, [&](int r, int kk) { return in(U, r, kk); }, fR);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[r][c] *= sm.left[ty * 4 + r];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float by_r = dot(k, a.k.st, acc, r);
        if (tx == 0) sm.wrote[ty * 4 + r] = by_r;
    }
    grad_product<false>(sm, acc, C, [&](int r, int kk) { return sm.P[kk][r]; }, fQ);
    grad_product<false>(sm, acc, C, [&](int r, int kk) { return -sm.b[kk] * sm.W[kk][r]; }, fK);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[r][c] = fmaf(-sm.b[ty * 4 + r], z[r][c], acc[r][c]);
    store(dk, a.dkt, acc);
    // dg
    if (tid < C) {
        float sum = 0.0f;
        for (int i = C - 1; i > tid; --i) sm.reads[i][tid] = sum += sm.reads[i][tid];
    }
    float pass = 0.0f;
    for (int64_t i = tid; i < E; i += kGradThreads) pass = fmaf(S[i], R[i], pass);
#pragma unroll
    for (int w = 1; w < 32; w *= 2) pass += __shfl_xor_sync(0xffffffffu, pass, w);
    if (tid % 32 == 0) sm.total[tid / 32] = pass;
    __syncthreads();
    if (tid < C) {
        float sum = 0.0f;
        for (int j = 0; j < tid; ++j) sum += sm.reads[tid][j];
        sm.crossed[tid] = sum;
    }
    __syncthreads();
    if (tid < 32) {
        float all = 0.0f;
        for (int w = 0; w < kGradThreads / 32; ++w) all += sm.total[w];
        delta_gate_grads(sm.past[C - 1] * all, sm.read, sm.wrote, sm.crossed, rows, tid, [&](int t, float x) {
            io_store(dg + t * a.dg.st, expf(gate_at<float>(a.g, b, h, t0 + t)) == 0.0f ? 0.0f : x);
        });
    }
}

// ---------------------------------------------------------------------------
// One token.  A block owns 32 columns of one head's state, a float4 of columns and every 32nd row a thread, all of
// them in registers before the first is used; the sums with k over the rows are joined through shared memory, then
// what the token writes goes in and the sums with q are joined the same way.  The state is read and written once,
// which bounds the step: 51 us for 270 MB of states and tokens (5.2 TB/s).

constexpr int kStepThreads = 256, kStepCols = 32;

template <typename IO, bool VEC>
__global__ void __launch_bounds__(kStepThreads, 6) k_delta_step(DeltaStep a) {
    __shared__ float sq[kMaxD], sk[kMaxD], sgate[3];
    __shared__ float so[2][kStepThreads / 32][kStepCols];
    const int tid = threadIdx.x;
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / a.H), h = (int)(bh % a.H), hk = h / (a.H / a.Hk);
    const int col0 = blockIdx.y * kStepCols;
    const int slot = a.slots ? a.slots[b] : b;
    IO *o = static_cast<IO *>(a.o) + b * a.ob + h * a.oh;
    if (slot < 0 || slot >= a.nslots) {
        if (tid < kStepCols && col0 + tid < a.dv) io_store(o + col0 + tid, 0.0f);
        return;
    }
    const IO *q = static_cast<const IO *>(a.q) + b * a.qb + hk * a.qh;
    const IO *k = static_cast<const IO *>(a.k) + b * a.kb + hk * a.kh;
    const IO *v = static_cast<const IO *>(a.v) + b * a.vb + h * a.vh;
    float *S = a.S + ((int64_t)slot * a.H + h) * a.d * a.dv;
    const int cg = tid % 8, rg = tid / 8, c = col0 + 4 * cg;  // column group of four, row
    constexpr int R = kMaxD / (kStepThreads / 8);
    float s[R][4];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int f = rg + i * (kStepThreads / 8);
        const float *p = S + (int64_t)f * a.dv + c;
        if (VEC) {
            const float4 w = f < a.d && c < a.dv ? *reinterpret_cast<const float4 *>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
            s[i][0] = w.x; s[i][1] = w.y; s[i][2] = w.z; s[i][3] = w.w;
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t) s[i][t] = f < a.d && c + t < a.dv ? p[t] : 0.0f;
        }
    }
    for (int i = tid; i < kMaxD; i += kStepThreads) {
        sq[i] = i < a.d ? io_load(q + i) : 0.0f;
        sk[i] = i < a.d ? io_load(k + i) : 0.0f;
    }
    float vc[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) vc[t] = c + t < a.dv ? io_load(v + c + t) : 0.0f;
    if (tid == kStepThreads - 1) {
        gate_terms(gate_at<IO>(a.g, b, h, 0), sgate[0], sgate[1]);
        sgate[2] = gate_at<IO>(a.b, b, h, 0);
    }
    __syncthreads();
    const float lam = sgate[0], rest = sgate[1], beta = sgate[2];
    // the four rows of a warp, then the warps in order
    auto join = [&](float (&acc)[4], float (*to)[kStepCols]) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            acc[t] += __shfl_xor_sync(0xffffffffu, acc[t], 8);
            acc[t] += __shfl_xor_sync(0xffffffffu, acc[t], 16);
        }
        if ((tid & 31) < 8) {
#pragma unroll
            for (int t = 0; t < 4; ++t) to[tid / 32][4 * cg + t] = acc[t];
        }
        __syncthreads();
    };
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const float kf = sk[rg + i * (kStepThreads / 8)];
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] = fmaf(kf, s[i][t], acc[t]);
    }
    join(acc, so[0]);
    float u[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < kStepThreads / 32; ++w) y += so[0][w][4 * cg + t];
        u[t] = beta * (vc[t] - fmaf(lam, y, rest * y));
        acc[t] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int f = rg + i * (kStepThreads / 8);
        const float kf = sk[f], qf = sq[f];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[i][t] = decayed(lam, rest, s[i][t], kf * u[t]);
            acc[t] = fmaf(qf, s[i][t], acc[t]);
        }
        float *p = S + (int64_t)f * a.dv + c;
        if (f < a.d) {
            if (VEC) {
                if (c < a.dv) *reinterpret_cast<float4 *>(p) = make_float4(s[i][0], s[i][1], s[i][2], s[i][3]);
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (c + t < a.dv) p[t] = s[i][t];
            }
        }
    }
    join(acc, so[1]);
    if (tid < kStepCols && col0 + tid < a.dv) {
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < kStepThreads / 32; ++w) y += so[1][w][tid];
        io_store(o + col0 + tid, a.scale * y);
    }
}

unsigned cdiv(int64_t a, int64_t b) { return (unsigned)((a + b - 1) / b); }

template <int JD, bool REV, int COLS, int CPL>
void rows_launch(const DeltaArgs &a, cudaStream_t s) {
    const dim3 grid((unsigned)(a.B * a.H), cdiv(a.dv, COLS));
    LUNA_LAUNCH("delta_rows", (k_delta_rows<JD, REV, COLS, CPL>), grid, COLS / CPL * 8 + kLoaders, 0, s, a);
}

// Two columns a lane where blocks of 16 columns would be more than the SMs hold at a time: the rows are read from shared
// memory, which then bounds the pass, half as often.  (64 heads of 2048 x 128 x 128: 852 us forward, with one column
// a lane 1190.)
template <bool REV>
cudaError_t rows(const DeltaArgs &a, cudaStream_t s) {
    const bool wide = (int64_t)a.B * a.H * cdiv(a.dv, 16) > (int64_t)(a.d > 64 ? 2 : 3) * tc_sm_count();
    if (a.d <= 32)
        wide ? rows_launch<1, REV, 32, 2>(a, s) : rows_launch<1, REV, 16, 1>(a, s);
    else if (a.d <= 64)
        wide ? rows_launch<2, REV, 32, 2>(a, s) : rows_launch<2, REV, 16, 1>(a, s);
    else
        wide ? rows_launch<4, REV, 32, 2>(a, s) : rows_launch<4, REV, 16, 1>(a, s);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_delta_rows(const DeltaArgs &a, bool reverse, cudaStream_t s) {
    return reverse ? rows<true>(a, s) : rows<false>(a, s);
}

cudaError_t launch_delta_grad(const DeltaArgs &a, cudaStream_t s) {
    cudaError_t e = cudaFuncSetAttribute(k_delta_grad, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(GradShared));
    if (e != cudaSuccess) return e;
    LUNA_LAUNCH("delta_grad", k_delta_grad, (unsigned)((int64_t)a.B * a.H * a.m), kGradThreads, sizeof(GradShared), s, a);
    return cudaGetLastError();
}

cudaError_t launch_delta_step(const DeltaStep &a, luna_dtype io, cudaStream_t s) {
    // 16-byte accesses need rows of whole float4s and an aligned state
    const bool vec = a.dv % 4 == 0 && (reinterpret_cast<uintptr_t>(a.S) & 15) == 0;
    const dim3 grid((unsigned)(a.B * a.H), cdiv(a.dv, kStepCols));
    if (io == LUNA_F32) {
        if (vec)
            LUNA_LAUNCH("delta_step", (k_delta_step<float, true>), grid, kStepThreads, 0, s, a);
        else
            LUNA_LAUNCH("delta_step", (k_delta_step<float, false>), grid, kStepThreads, 0, s, a);
    } else {
        if (vec)
            LUNA_LAUNCH("delta_step", (k_delta_step<__nv_bfloat16, true>), grid, kStepThreads, 0, s, a);
        else
            LUNA_LAUNCH("delta_step", (k_delta_step<__nv_bfloat16, false>), grid, kStepThreads, 0, s, a);
    }
    return cudaGetLastError();
}

}  // namespace luna
