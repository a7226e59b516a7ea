// The gated delta rule on tensor cores: the chains over the chunks (a translation unit for each width of keys).
#pragma once

#include "luna_delta_tc.cuh"

namespace luna {
namespace {

using namespace delta;

// ---------------------------------------------------------------------------
// The chains.  A block has NG groups of 16 columns of one head's state, a group SP warps: with few heads two, which hold
// half of each column and exchange their shares of K S (and Q S) once a chunk; each then has 230 products a chunk where
// one warp has 420.  The tiles of a chunk come by asynchronous copies while the chunk before is worked on; one barrier a
// chunk.  With two warps a group a further warp issues those copies (the chain waits less: 1.31 to 1.18 ms below); with one,
// all warps do: eight of them and a ninth would not have 255 registers each (0.32 to 0.36 ms).  Bound by the chain: a chunk
// of 128 x 128 takes two warps 2.3 us where heads are few (32 heads of 32768 rows 1.18 ms, with one warp a group 2.1 ms),
// eight warps 4.9 us (128 heads of 4096 rows 0.32 ms, 0.47 in reverse), of which the products alone would take 3.5.

enum ChainMode {
    kOutputs,   // O (and the last state)
    kKeep,      // U and the states, for the gradients
    kReverse    // dV, X, dO and the gradients of the states
};

template <int DP, int NG, int SP, ChainMode MODE>
struct ChainShared {
    static constexpr int kWarps = NG * SP;
    static constexpr int kLoaders = SP == 2 ? 32 : kWarps * 32;         // threads that fetch tiles: with two warps a group, one more
    static constexpr int kThreads = kWarps * 32 + (SP == 2 ? 32 : 0);
    static constexpr int kPitch = NG * 32 + 16;  // bytes of a row of V or dO: eight rows start in eight banks
    static constexpr bool kQ = MODE != kKeep;    // Q and P are needed
    static constexpr int kPlanes = MODE == kReverse ? 2 : 1;  // of P
    struct Stage {
        alignas(128) char k[DP / 64][kTileB], q[kQ ? DP / 64 : 1][kQ ? kTileB : 16], T[2][kTileB];
        alignas(128) char P[kPlanes][kQ ? kTileB : 16], x[C * kPitch];
        alignas(16) float rows[4 * C + 12];  // (the gates' sums behind them are not needed)
    } stage[2];
    uint64_t bar[2];
    // 16 columns of the outputs (one warp a group: they take the place of its columns of V or dO)
    alignas(16) char out[kQ && SP == 2 ? kWarps : 1][kQ && SP == 2 ? C * 48 : 16];
    alignas(128) char planes[MODE != kOutputs && SP == 1 ? kWarps : 1][MODE != kOutputs && SP == 1 ? DP * 32 : 16];  // 16 rows of a tile that is kept
    float4 shares[SP == 1 ? 1 : kWarps][SP == 1 ? 1 : 12][32];
};

template <int DP, int NG, int SP, ChainMode MODE, bool VEC>
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
    for (int i = tid; i < C * NG * 2; i += Sh::kLoaders) {
        const int r = i / (NG * 2), p = i % (NG * 2);
        load_piece(sx + r * Sh::kPitch + p * 16, x + r * xv.st + p * 8, xv.p, r < rows ? a.dv - col0 - p * 8 : 0, VEC);
    }
    copies_end();
}

// Rows first, first + 1, .. (n of them) of a warp's 16 columns, given column by column, to the output: transposed through
// shared memory, in rows of 32 bytes `pitch` apart (a multiple of 16 whose eight first multiples fall into eight banks)
__device__ __forceinline__ void chain_store(const float (&acc)[8][4], int first, int n, char *mem, int pitch, __nv_bfloat16 *out, int64_t st, int rows,
                                            int col, int dv, bool vec, int lane) {
    const uint32_t base = smem_u32(mem);
#pragma unroll
    for (int nt = 0; nt < 8; nt += 2) {
        if (nt * 8 < first || nt * 8 >= first + n) continue;
        const Frag f = {pack_bf16(acc[nt][0], acc[nt][1]), pack_bf16(acc[nt][2], acc[nt][3]),
                        pack_bf16(acc[nt + 1][0], acc[nt + 1][1]), pack_bf16(acc[nt + 1][2], acc[nt + 1][3])};
        stm_t(base + (nt * 8 + (lane >> 4) * 8 + (lane & 7)) * pitch + ((lane >> 3) & 1) * 16, f);
    }
    __syncwarp();
    for (int i = 0; i < n / 16; ++i) {
        const int r = first + i * 16 + lane / 2, half = lane % 2;
        if (r < rows && col + half * 8 < dv) {
            const __nv_bfloat16 *from = reinterpret_cast<const __nv_bfloat16 *>(mem + r * pitch + half * 16);
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
__device__ __forceinline__ void plane_send(const char *mem, __half *tile, int rows, int r0, int panels, int lane) {
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
        for (int p = 0; p < panels; ++p) store_tile(reinterpret_cast<char *>(tile) + (p * rows + r0) * 128, smem_u32(mem) + p * 2048, 2048);
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

template <int DP, int NG, int SP, ChainMode MODE, bool VEC>
__global__ void __launch_bounds__(ChainShared<DP, NG, SP, MODE>::kThreads) k_delta_chain(DeltaArgs a) {
    using Sh = ChainShared<DP, NG, SP, MODE>;
    extern __shared__ __align__(128) char raw[];
    Sh &sm = *reinterpret_cast<Sh *>(raw);
    constexpr bool REV = MODE == kReverse;
    constexpr int ND = DP / 8 / SP;  // n-tiles of a state's row that a warp holds
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, group = warp / SP, part = warp % SP, d0 = part * (DP / SP);
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / a.H), h = (int)(bh % a.H), col0 = blockIdx.y * NG * 16, col = col0 + group * 16;
    const int len = head_length(a.lengths, b, a.n), chunks = (len + C - 1) / C, q2 = lane % 4 * 2;
    const bool mine = warp < Sh::kWarps && col < a.dv;  // the warp has columns
    const int loader = SP == 2 ? tid - Sh::kWarps * 32 : tid;  // (not negative: fetches tiles)
    __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(a.o) + b * a.ob + h * a.oh;  // (not with kKeep)
    // what is kept: by copies where a warp has whole rows of 128 bytes
    char *const mem = sm.planes[SP == 1 ? warp : 0];
    auto put = [&](__half *tile, int k0, const Frag &f) {
        if (SP == 1)
            tile_put(smem_u32(mem), 16, 0, k0, f, lane);
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
        return mine && r < a.d && c < a.dv;
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
    if (chunks > 0 && loader >= 0)
        chain_load<DP, NG, SP, MODE, VEC>(sm.stage[0], &sm.bar[0], a, bh, b, h, REV ? chunks - 1 : 0, len, col0, loader);
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
        if (step + 1 < chunks && loader >= 0)
            chain_load<DP, NG, SP, MODE, VEC>(sm.stage[(step + 1) & 1], &sm.bar[(step + 1) & 1], a, bh, b, h, REV ? chunk - 1 : chunk + 1, len, col0, loader);
        if (!mine) continue;
        const uint32_t sk = smem_u32(st.k), sq = smem_u32(st.q), sT = smem_u32(st.T), sP = smem_u32(st.P);
        const uint32_t sx = smem_u32(st.x) + ((lane >> 4) * 8 + (lane & 7)) * Sh::kPitch + group * 32 + ((lane >> 3) & 1) * 16;
        const float whole = st.rows[4 * C], rest = st.rows[4 * C + 1], back_T = st.rows[4 * C + 2], back_P = st.rows[4 * C + 3];
        auto factor = [&](int which, int t) { return *reinterpret_cast<const float2 *>(st.rows + which * C + t); };
        const int64_t at = bh * a.m + chunk;
        char *const out = SP == 2 ? sm.out[warp] : st.x + group * 32;
        constexpr int out_pitch = SP == 2 ? 48 : Sh::kPitch;
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
            const float back_u = xs.back * back_T, most_u = most_of(u);  // (u is U over back_u)
            {  // P U, or U's plane
                __half *tile = a.Up + at * a.dvp * C;
                if (MODE == kKeep) room();
#pragma unroll
                for (int nt = 0; nt < 8; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[nt][e] = 0.0f;
                const Scale us = scale_of(most_u);
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
                    if (lane == 0) scales_of(chunk)[4] = us.back * back_u;
                } else {  // scale c(i, 0) Q S + P U
                    const float back = us.back * back_u * back_P;
#pragma unroll
                    for (int nt = 0; nt < 8; ++nt) {
                        const float2 past = factor(3, nt * 8 + q2);
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[nt][e] = fmaf(back_s * (e & 1 ? past.y : past.x), y[nt][e], back * x[nt][e]);
                    }
                    chain_store(y, first, some, out, out_pitch, o + t0 * a.ot, a.ot, min(C, len - t0), col, a.dv, VEC, lane);
                }
            }
#pragma unroll
            for (int nt = 0; nt < 8; ++nt) {
                const float2 left = factor(1, nt * 8 + q2);
#pragma unroll
                for (int e = 0; e < 4; ++e) u[nt][e] *= e & 1 ? left.y : left.x;
            }
            const Scale ls = scale_of(most_u * st.rows[4 * C + 6]);
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) split_left(u[2 * kt], u[2 * kt + 1], ls.by, fh[kt], fl[kt]);
            update(fh, fl, ls.back * back_u, sk, true);
        } else {
            // y = P^T dO (this warp's share of the rows);  R <- c(C, 0) R + scale Q^T c(i, 0) dO
            Frag g[4];
            uint32_t pairs = 0;
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                ldm_t(g[kt], sx + kt * 16 * Sh::kPitch);
#pragma unroll
                for (int i = 0; i < 4; ++i) pairs = __vmaxu2(pairs, g[kt][i] & 0x7fff7fffu);
            }
            const float most_g = warp_max(__uint_as_float(max(pairs << 16, pairs & 0x7fff0000u)));
            const Scale gs = scale_of(most_g), ps = scale_of(most_g * st.rows[4 * C + 8]);
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
            const float back_x = xs.back * back_T, most_y = most_of(y);  // (y is X over back_x)
            const Scale us = scale_of(most_y);
            if (lane == 0) scales_of(chunk)[5] = us.back * back_x;
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
                    y[nt][e] *= back_x * (e & 1 ? beta.y : beta.x);
                    x[nt][e] = -(e & 1 ? past.y : past.x) * y[nt][e];
                }
            }
            const Scale ws = scale_of(most_y * back_x * st.rows[4 * C + 7]);
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) split_left(x[2 * kt], x[2 * kt + 1], ws.by, fh[kt], fl[kt]);
            update(fh, fl, ws.back, sk, false);
            chain_store(y, first, some, out, out_pitch, o + t0 * a.ot, a.ot, min(C, len - t0), col, a.dv, VEC, lane);
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
        for (int64_t i = tid; i < (int64_t)(a.n - len) * NG * 2; i += Sh::kThreads) {
            const int c = col0 + (int)(i % (NG * 2)) * 8;
            __nv_bfloat16 *to = o + (len + i / (NG * 2)) * a.ot + c;
            if (VEC && c < a.dv)
                *reinterpret_cast<uint4 *>(to) = make_uint4(0, 0, 0, 0);
            else
                for (int e = 0; e < min(8, a.dv - c); ++e) io_store(to + e, 0.0f);
        }
}

template <int DP, int NG, int SP, ChainMode MODE, bool VEC>
cudaError_t chain_launch(const DeltaArgs &a, cudaStream_t s) {
    using Sh = ChainShared<DP, NG, SP, MODE>;
    cudaError_t e = cudaFuncSetAttribute(k_delta_chain<DP, NG, SP, MODE, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Sh));
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)(a.B * a.H), blocks_of(a.dv, NG * 16));
    LUNA_LAUNCH("delta_chain", (k_delta_chain<DP, NG, SP, MODE, VEC>), grid, Sh::kThreads, sizeof(Sh), s, a);
    return cudaGetLastError();
}

// With few heads, few columns a block and two warps for 16 of them, so that the chains spread over the SMs; states of at most
// 32 columns always that way, however many heads (not measured against others).  (Rows that do not start on 16-byte
// boundaries: no blocks of all 128 columns.)  On 152 SMs at 128 columns the forms change at 39 and 77 heads in all; times
// were taken at 32 and 128 (above), none in between, where half of the SMs' quarters have no warp.
template <int DP, ChainMode MODE>
cudaError_t chain(const DeltaArgs &a, cudaStream_t s) {
    const int64_t bh = (int64_t)a.B * a.H, sms = tc_sm_count();
    if (a.vec && a.dv > 64 && bh * blocks_of(a.dv, 64) > sms) return chain_launch<DP, 8, 1, MODE, true>(a, s);
    if (a.dv > 32 && bh * blocks_of(a.dv, 32) > sms)
        return a.vec ? chain_launch<DP, 4, 1, MODE, true>(a, s) : chain_launch<DP, 4, 1, MODE, false>(a, s);
    return a.vec ? chain_launch<DP, 2, 2, MODE, true>(a, s) : chain_launch<DP, 2, 2, MODE, false>(a, s);
}
template <int DP>
cudaError_t chain_of(const DeltaArgs &a, bool reverse, cudaStream_t s) {
    return reverse ? chain<DP, kReverse>(a, s) : a.Up ? chain<DP, kKeep>(a, s) : chain<DP, kOutputs>(a, s);
}

}  // namespace
}  // namespace luna
