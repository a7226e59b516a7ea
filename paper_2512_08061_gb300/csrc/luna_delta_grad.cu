// The gated delta rule on tensor cores: gradients by chunk.
#include "luna_delta_tc.cuh"

namespace luna {
namespace {

using namespace delta;

// ---------------------------------------------------------------------------
// Gradients of q, k and the gates (luna_delta.cuh) from the chunk's U, X, dO and states.  A block of eight warps a chunk:
// two groups of 32 rows by four quarters of the columns.  107 KB of shared memory, so that two blocks are on an SM and
// the one's products cover the other's loads: R, then S, then Q lie in the same place, P and W in that of U.  546 us for
// 8192 chunks of 128 x 128; bound by the waits between those.  (466 us with P and W in one unit, which loses dQ where a chunk's
// queries or keys are 0, and with a gate's gradient as a difference, which loses it where the gate is strong; of that form, with
// everything in place at once, 16 warps and one block an SM 804 us.)

constexpr int kGradThreads = 256, kParts = 4;

template <int DP, int DVT>
struct GradShared {
    alignas(128) char k[DP / 64][kTileB], go[DVT * 128], x[DVT * 128], u[DVT * 128 > 2 * kTileB ? DVT * 128 : 2 * kTileB];
    alignas(128) char s[DVT * DP * 2 > DP / 64 * kTileB ? DVT * DP * 2 : DP / 64 * kTileB];
    uint64_t bar[4];
    alignas(16) float rows[kRowsF];
    alignas(16) float scales[2 * DVT / 16][kDeltaScales];  // of this chunk and, behind it, of the next place
    float past[C], left[C];
    __half2 steps[8][DVT / 16];  // of the products over columns: 16 columns' scale over the largest, that
    float all[8], total[kGradThreads / 32];
    // of a row's quarters: q . dQ, k . Z and k . dK, all of the states' parts alone, W . K K^T, x . v; and what its reads of the rows of an
    // earlier 16 (the quarter) add up to, of its own 16 what crosses its gate; of a row as written, what each later 16 reads
    float sums[6][kParts][C], written[kParts][C];
    float most[2][kGradThreads / 32], read[C], wrote[C], crossed[C];
};

template <int DP, int DVT, typename OUT, bool VEC>
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
        const uint32_t of_scales = 2 * groups * kDeltaScales * 4;
        mbar_arrive_expect_tx(&sm.bar[0], sizeof(sm.k) + 3 * of_rows + sizeof(sm.rows) + of_scales);
        load_tile(sm.rows, a.rows + at * kRowsF, sizeof(sm.rows), &sm.bar[0]);
        load_tile(sm.scales, a.scales + slot * groups * kDeltaScales, of_scales, &sm.bar[0]);
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
        ask(a.Qp + kat * C * DP, sizeof(sm.k));
    }
    // x . v: a thread a row and a quarter of the columns, while the tiles come
    uint32_t v[DVT / 8 / kParts][4];
    {
        const int i = tid % C;
        const __nv_bfloat16 *from = static_cast<const __nv_bfloat16 *>(a.v.p) + b * a.v.sb + h * a.v.sh + (t0 + i) * a.v.st;
#pragma unroll
        for (int j = 0; j < DVT / 8 / kParts; ++j) {
            const int c = (tid / C + j * kParts) * 8;
            if (VEC) {
                const uint4 w4 = i < rows && c < a.dv ? *reinterpret_cast<const uint4 *>(from + c) : make_uint4(0, 0, 0, 0);
                v[j][0] = w4.x; v[j][1] = w4.y; v[j][2] = w4.z; v[j][3] = w4.w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 f = load_pair(from + c + 2 * e, i < rows ? a.dv - c - 2 * e : 0, false);
                    v[j][e] = pack_bf16(f.x, f.y);
                }
            }
        }
    }
    bool here = mbar_wait_long(&sm.bar[0], 0);
    const float back_k = sm.rows[4 * C + 4], back_q = sm.rows[4 * C + 5];
    const float *gate_b = sm.rows + 2 * C, *hi = sm.rows + 4 * C + 12, *lo = hi + C;
    // What is summed over the columns has a scale of its own every 16 of them: the left operand takes the ratio to the
    // largest of them (at most 1, and what it loses is small beside that).  Products: dO U, X U; of either half of the
    // other columns dO S, X S, U R.
    if (tid < 64) {
        const int product = tid / 8, kt = tid % 8, side = product < 2 ? 0 : (product - 2) / 3, which = product < 2 ? product : (product - 2) % 3;
        float scale = 0.0f;
        if (kt < groups) {
            const float *f = sm.scales[kt], *g = sm.scales[groups + kt];  // (behind the chunk: R)
            scale = product < 2 ? f[6 - which] * f[4] : which < 2 ? f[6 - which] * f[side] : f[4] * g[2 + side];
        }
        float most = scale;
#pragma unroll
        for (int w = 4; w > 0; w /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, w));
        if (kt == 0) sm.all[product] = most;
        if (kt < groups) sm.steps[product][kt] = __float2half2_rn(most > 0.0f ? scale * inverse2(most) : 0.0f);
    } else if (tid < 64 + C) {
        // from the sums of the gates: the chains' factors have K's scale in them, and none of their bits where K is 0
        const int t = tid - 64;
        auto factor = [](float h, float l) {
            const float e = expf(h);
            return fmaf(e, l, e);
        };
        sm.past[t] = factor(hi[t], lo[t]);
        sm.left[t] = expf((hi[C - 1] - hi[t]) + (lo[C - 1] - lo[t]));
    }
    {
        const int i = tid % C;
        float xv = 0.0f;
#pragma unroll
        for (int j = 0; j < DVT / 8 / kParts; ++j) {
            const int c8 = tid / C + j * kParts;
            if (c8 * 8 >= dvp) continue;
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                unsigned short u;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(u) : "r"(tile_at(sx, dvp, c8 * 8 + e, i >> 3) + (i & 7) * 2));
                sum = fmaf(e & 1 ? high(v[j][e / 2]) : low(v[j][e / 2]), __half2float(__ushort_as_half(u)), sum);
            }
            xv = fmaf(sm.scales[c8 / 2][5], sum, xv);
        }
        sm.sums[4][tid / C][i] = xv;
    }
    __syncthreads();

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
    // acc += by F M over the 64 rows of the chunk: F from P or W (trans: its transpose), M a tile of K or Q.  Summed by itself
    // and scaled as it is added, in fp32: `by` may be any power of two (of a tile of nothing or of very little), and
    // its inverse is never taken.
    auto over_rows = [&](Acc &acc, uint32_t from, bool trans, uint32_t tile, float by) {
#pragma unroll
        for (int np = 0; np < NT / 2; ++np) {
            float sum[2][2][4];
            zero(sum[0]);
            zero(sum[1]);
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                if (trans ? kt * 16 < r0 : kt * 16 > r0 + 16) continue;
                Frag f;
                right_k(f, tile, C, kt * 16, c0 + np * 16, lane);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    Frag fl;
                    if (trans)
                        left_k(fl, from, C, kt * 16, r0 + mt * 16, lane);
                    else
                        left_m(fl, from, C, r0 + mt * 16, kt * 16, lane);
                    mma(sum[mt][0], fl, f[0], f[1]);
                    mma(sum[mt][1], fl, f[2], f[3]);
                }
            }
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[mt][2 * np + i][e] = fmaf(by, sum[mt][i][e], acc[mt][2 * np + i][e]);
        }
    };
    // acc *= by row_factor (of every row)
    auto times_rows = [&](Acc &acc, const float *row_factor, float by) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            const int ra = r0 + mt * 16 + lane / 4;
            const float fa = by * row_factor[ra], fb = by * row_factor[ra + 8];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[mt][nt][e] *= e & 2 ? fb : fa;
        }
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
                    if (!VEC) {
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
        float kk[2][2][4], qk[2][2][4];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            zero(p[mt]);
            zero(w[mt]);
            zero(kk[mt]);
            zero(qk[mt]);
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
            // Q as it lies in memory (in both the summed values lie in the same, permuted order: a lane's 16 bytes of a row
            // are those of two products)
            const char *q = reinterpret_cast<const char *>(a.Qp + kat * C * DP);
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) {
                const int piece = i * 4 + lane % 4, rk = n0 + lane / 4;
                const uint4 k_0 = *reinterpret_cast<const uint4 *>(sm.k[0] + tile_at(0, C, rk, piece));
                const uint4 k_1 = *reinterpret_cast<const uint4 *>(sm.k[0] + tile_at(0, C, rk + 8, piece));
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    const int rq = r0 + mt * 16 + lane / 4;
                    const uint4 q0 = __ldg(reinterpret_cast<const uint4 *>(q + tile_at(0, C, rq, piece)));
                    const uint4 q1 = __ldg(reinterpret_cast<const uint4 *>(q + tile_at(0, C, rq + 8, piece)));
                    const Frag f = {q0.x, q1.x, q0.y, q1.y}, g = {q0.z, q1.z, q0.w, q1.w};
                    mma(qk[mt][0], f, k_0.x, k_0.y);
                    mma(qk[mt][0], g, k_0.z, k_0.w);
                    mma(qk[mt][1], f, k_1.x, k_1.y);
                    mma(qk[mt][1], g, k_1.z, k_1.w);
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
                    const float c = j <= i ? expf((hi[i] - hi[j]) + (lo[i] - lo[j])) : 0.0f;
                    float &pp = p[mt][nt][e], &ww = w[mt][nt][e];
                    pp = j <= i ? by_p * c * pp : 0.0f;
                    ww = j < i ? by_w * c * ww : 0.0f;
                    if (j < i) dot[e >> 1] = fmaf(ww, kk[mt][nt][e], dot[e >> 1]);
                    ww *= gate_b[i];
                    mp = fmaxf(mp, fabsf(pp));
                    mw = fmaxf(mw, fabsf(ww));
                    // what row i reads of row j, which crosses the gates between them
                    float &read = qk[mt][nt][e];
                    read = j < i ? pp * (read * back_q * back_k) - ww * (kk[mt][nt][e] * back_k * back_k) : 0.0f;
                }
            row_sums(dot[0], dot[1], mt, 3);
            const int I = r0 / 16 + mt;  // (of the 16 rows; those of the columns are `quarter`)
            if (I > quarter) {
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x = qk[mt][nt][e] + qk[mt][nt][2 + e];
#pragma unroll
                        for (int m = 4; m < 32; m *= 2) x += __shfl_xor_sync(0xffffffffu, x, m);
                        if (lane < 4) sm.written[I][n0 + nt * 8 + q2 + e] = x;
                    }
            } else if (I == quarter) {  // columns' sums from their end to each row; of them those before the row cross its gate
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float &x = qk[mt][nt][e], &y = qk[mt][nt][2 + e];  // rows lane / 4 and 8 more
#pragma unroll
                        for (int m = 4; m < 32; m *= 2) {
                            const float x_ = __shfl_down_sync(0xffffffffu, x, m), y_ = __shfl_down_sync(0xffffffffu, y, m);
                            if (lane + m < 32) {
                                x += x_;
                                y += y_;
                            }
                        }
                        x += __shfl_sync(0xffffffffu, y, lane % 4);
                        const int j = nt * 8 + q2 + e, i = lane / 4;
                        x = j < i ? x : 0.0f;
                        y = j < i + 8 ? y : 0.0f;
                    }
            }
            row_sums((qk[mt][0][0] + qk[mt][0][1]) + (qk[mt][1][0] + qk[mt][1][1]),
                     (qk[mt][0][2] + qk[mt][0][3]) + (qk[mt][1][2] + qk[mt][1][3]), mt, 5);
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
    // P and W each by its own largest value, whatever Q, K and each other are
    const Scale ps = scale_of(mp), ws = scale_of(mw);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const uint32_t to = tile_at(0, C, r0 + mt * 16 + lane / 4 + e * 4, quarter * 2 + nt) + q2 * 2;
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(sP + to), "r"(pack(ps.by * p[mt][nt][e], ps.by * p[mt][nt][e + 1])) : "memory");
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(sW + to), "r"(pack(ws.by * w[mt][nt][e], ws.by * w[mt][nt][e + 1])) : "memory");
            }
    times_rows(acc, sm.left, sm.all[of_half + 2]);
    dot_k(acc, 2);
    __syncthreads();
    over_rows(acc, sW, true, sk, -ws.back * back_k);

    // dQ and Z from S
    here = mbar_wait_long(&sm.bar[2], 0);
    clear(z);
    if (here) over_columns(z, sgo, of_half);
    times_rows(z, sm.past, a.scale * sm.all[of_half]);
    {  // q . dQ of the state's part, with Q as it came
        const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(a.q.p) + b * a.q.sb + hk * a.q.sh + t0 * a.q.st + c0 + q2;
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            float dot[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = r0 + mt * 16 + lane / 4 + i * 8;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float2 f = load_pair(q + r * a.q.st + nt * 8, r < rows ? a.d - (c0 + nt * 8 + q2) : 0, VEC);
                    dot[i] = fmaf(f.x, z[mt][nt][2 * i], fmaf(f.y, z[mt][nt][2 * i + 1], dot[i]));
                }
            }
            row_sums(dot[0], dot[1], mt, 0);
        }
    }
    over_rows(z, sP, false, sk, ps.back * back_k);
    store_rows(z, dq, a.dqt);
    {  // <S, R> of the states at the chunk's two ends: of every 16 columns the diagonal of S^T R, R as Q above
        float sum = 0.0f;
        if (here && warp < groups) {
            const char *r = reinterpret_cast<const char *>(a.Rp + (slot + 1) * dvp * DP);
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
                    const uint4 r0_ = __ldg(reinterpret_cast<const uint4 *>(r + at0)), r1 = __ldg(reinterpret_cast<const uint4 *>(r + at1));
                    const Frag f = {s0.x, s1.x, s0.y, s1.y}, g = {s0.z, s1.z, s0.w, s1.w};
                    mma(c[0], f, r0_.x, r0_.y);
                    mma(c[0], g, r0_.z, r0_.w);
                    mma(c[1], f, r1.x, r1.y);
                    mma(c[1], g, r1.z, r1.w);
                }
                const float *scale = sm.scales[warp], *scale_r = sm.scales[groups + warp];
                float diag = 0.0f;
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (lane / 4 == q2 + e) diag += c[0][e] + c[1][2 + e];
                sum = fmaf(scale[side] * scale_r[2 + side], diag, sum);
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
    times_rows(z, sm.past, sm.all[of_half + 1]);
    dot_k(z, 1);
    times_rows(z, gate_b, 1.0f);
    over_rows(z, sW, false, sk, ws.back * back_k);

    // dK
    here = mbar_wait_long(&sm.bar[3], 0);
    if (here) over_rows(acc, sP, true, ss, ps.back * back_q);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[mt][nt][e] -= z[mt][nt][e];
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
        io_store(db + tid * a.db.st, sum(4) - sum(1) - back_k * back_k * sum(3));
        sm.read[tid] = sum(0) - gate_b[tid] * sum(1);
        sm.wrote[tid] = sum(2);
    }
    if (tid >= C && tid < 2 * C) {  // what crosses gate t of its 16: reads of rows at or behind it of rows before it
        const int t = tid - C, T = t / 16, c = t % 16;
        const float(*of)[C] = sm.sums[5];
        float read = 0.0f, wrote = 0.0f;  // in its own 16, of and by the others
        for (int J = 0; J < T; ++J) read += of[J][t];
        for (int I = T + 1; I < 4; ++I) wrote += sm.written[I][t];
        float around = T == 1 ? of[0][32 + c] + of[0][48 + c] : T == 2 ? of[0][48 + c] + of[1][48 + c] : 0.0f;
#pragma unroll
        for (int m = 1; m < 16; m *= 2) {
            const float r = __shfl_down_sync(0xffffffffu, read, m, 16), w = __shfl_up_sync(0xffffffffu, wrote, m, 16);
            if (c + m < 16) read += r;
            if (c >= m) wrote += w;
            around += __shfl_xor_sync(0xffffffffu, around, m, 16);
        }
        wrote = __shfl_up_sync(0xffffffffu, wrote, 1, 16);
        sm.crossed[t] = (of[T][t] + read) + (around + (c > 0 ? wrote : 0.0f));
    }
    __syncthreads();
    if (warp == 0) {
        float base = 0.0f;
        for (int w = 0; w < kGradThreads / 32; ++w) base += sm.total[w];
        delta_gate_grads(sm.rows[4 * C] * base, sm.read, sm.wrote, sm.crossed, rows, lane, [&](int t, float x) {
            const float g = t > 0 ? (hi[t] - hi[t - 1]) + (lo[t] - lo[t - 1]) : hi[0];
            io_store(dg + t * a.dg.st, expf(g) == 0.0f ? 0.0f : x);
        });
    }
}

template <int DP, int DVT, typename OUT, bool VEC>
cudaError_t grad_launch(const DeltaArgs &a, cudaStream_t s) {
    using Sh = GradShared<DP, DVT>;
    cudaError_t e = cudaFuncSetAttribute(k_delta_grad_tc<DP, DVT, OUT, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Sh));
    if (e != cudaSuccess) return e;
    LUNA_LAUNCH("delta_grad_tc", (k_delta_grad_tc<DP, DVT, OUT, VEC>), (unsigned)((int64_t)a.B * a.H * a.m), kGradThreads, sizeof(Sh), s, a);
    return cudaGetLastError();
}

template <typename OUT, bool VEC>
cudaError_t grad(const DeltaArgs &a, cudaStream_t s) {
    if (a.d <= 64) return a.dv <= 64 ? grad_launch<64, 64, OUT, VEC>(a, s) : grad_launch<64, 128, OUT, VEC>(a, s);
    return a.dv <= 64 ? grad_launch<128, 64, OUT, VEC>(a, s) : grad_launch<128, 128, OUT, VEC>(a, s);
}

}  // namespace

cudaError_t launch_delta_grad_tc(const DeltaArgs &a, luna_dtype out, cudaStream_t s) {
    if (out == LUNA_F32) return a.vec ? grad<float, true>(a, s) : grad<float, false>(a, s);
    return a.vec ? grad<__nv_bfloat16, true>(a, s) : grad<__nv_bfloat16, false>(a, s);
}

}  // namespace luna
