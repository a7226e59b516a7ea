// Linear attention with a decay for each head on tensor cores (bf16, tcgen05 / TMEM / TMA).
//
// A block walks one piece of a head's rows in chunks of 128 (a, b, c as in luna_decay.cuh) and keeps the
// state X (da x dc) in fp32 registers.  Per chunk of nv rows, m a row's number in processing order:
//     MMA    P = a b^T,  E = a X                       (X as a bf16 operand)
//     warps  P masked and decayed, as bf16 back into TMEM;  E scaled by x lambda^{m+e} in place
//            b scaled by lambda^{nv-m-e} into bf16 terms b1 + b2 (+ b3)
//     MMA    U = (b1 + b2 (+ b3))^T c,  E += P c
//     warps  out = E;  X = lambda^{nv} X + u U, and its bf16 operand
// The decay sits on b alone, so c enters U as it is; one bf16 rounding of the scaled b would cost the
// state 1.7e-3, two terms leave 3e-6 and three 2^-24.  Passes whose state leaves the kernel use three,
// the others two (their state only enters outputs as one more bf16 rounding).
//
// Bound: by its bytes the pass is (da + dc) * 4 bytes a row at HBM rate; the shared-memory traffic of
// the products' operands and of the scaled terms comes next (about 4/5 of that at d = 128).  Two groups
// of warps (P and out; X and the scaled b) work on their halves of a chunk side by side, and the
// next tiles load while they do: a ring of four slots takes a, b, c in turn.
#include <math.h>
#include <string.h>

#include "luna_decay.cuh"
#include "luna_prof.cuh"
#include "luna_sm100.cuh"

namespace luna {

bool tc_make_map_nd(CUtensorMap *m, const void *base, int rank, const uint64_t *dims, const uint64_t *strides,
                    const uint32_t *box);

namespace {
using namespace sm100;

constexpr int kRows = 128;   // rows of a chunk
constexpr int kSlots = 4;

template <int D, int NT, bool STATE> struct Cfg {
    static constexpr int NW = D / 16;               // warps of a group (8 or 4)
    static constexpr int GT = NW * 32;              // threads of a group
    static constexpr int GROUPS = STATE ? 1 : 2;
    static constexpr int THREADS = GROUPS * GT + 64;
    static constexpr int KB = D / 64;               // 64-column blocks of a row
    static constexpr uint32_t BLK = kRows * 128;    // one block of a tile
    static constexpr uint32_t TILE = KB * BLK;
    static constexpr uint32_t XBLK = D * 128, XOP = KB * XBLK;  // X operand: [64-column block][feature][64]
    static constexpr uint32_t SMEM = kSlots * TILE + (NT - 1) * TILE + (STATE ? 0 : XOP) + 1024 + 1024;
    static_assert(SMEM <= 227 * 1024, "shared memory");
    // TMEM columns: P (then its bf16 form in the first half) | E | U
    static constexpr uint32_t cP = 0, cE = 128, cU = STATE ? 0 : 128 + D;
    static constexpr uint32_t COLS = STATE ? D : D == 64 ? 256 : 512;
    static constexpr int CPT = D == 64 ? 64 : D * D / GT;  // state columns of a thread (D = 64: 16 lanes of a warp)
};

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&v);
}
__device__ __forceinline__ uint8_t *align_1024(uint8_t *p) {
    return p + ((1024u - (smem_u32(p) & 1023u)) & 1023u);
}
__device__ __forceinline__ uint64_t dadd(uint64_t desc, uint32_t bytes) { return desc + (bytes >> 4); }

// D[tmem] (+)= A[tmem, bf16 pairs] * B[smem desc]
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                            uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// 32 scores of row i, columns 32 jb ..: masked, decayed, times p.  Off the diagonal block the decay is a
// factor of the row times one of the column (both at most 1 for lambda <= 1), on it a table lookup.
__device__ __forceinline__ void decay_scores(float (&v)[32], int i, int jb, bool reverse, int nv, float p,
                                             const float *pw) {
    const int ib = i >> 5, li = i & 31, j0 = 32 * jb;
    if (jb == ib) {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const int dist = reverse ? j - li : li - j;
            const bool on = dist >= 0 && i < nv && j0 + j < nv;
            v[j] = on ? v[j] * (p * pw[on ? dist : 0]) : 0.0f;
        }
        return;
    }
    if (reverse ? jb < ib : jb > ib) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = 0.0f;
        return;
    }
    const float row = p * (reverse ? pw[j0 - i] : pw[i - j0 - 31]);
    const float4 *t = reinterpret_cast<const float4 *>(pw);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        // forward: column j of the block decays by 31 - j, reverse: by j
        const float4 w = reverse ? t[q] : t[7 - q];
        const float c[4] = {reverse ? w.x : w.w, reverse ? w.y : w.z, reverse ? w.z : w.y, reverse ? w.w : w.x};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool on = i < nv && j0 + 4 * q + k < nv;
            v[4 * q + k] = on ? v[4 * q + k] * (row * c[k]) : 0.0f;
        }
    }
}

template <int D, int NT, bool STATE, typename OUT>
__global__ void __launch_bounds__(Cfg<D, NT, STATE>::THREADS, D == 64 ? 2 : 1)
    k_decay_tc(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
               const __grid_constant__ CUtensorMap mapC, const __grid_constant__ DecayMix a) {
    using C = Cfg<D, NT, STATE>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sm = align_1024(smem_raw);
    uint8_t *terms = sm + kSlots * C::TILE;           // b2, b3 (b1 overwrites b in its slot)
    uint8_t *Xop = terms + (NT - 1) * C::TILE;
    float *pw = reinterpret_cast<float *>(Xop + (STATE ? 0 : C::XOP));  // lambda^0 .. lambda^128
    uint64_t *bars = reinterpret_cast<uint64_t *>(pw + 132);
    uint64_t *full = bars, *freeb = bars + kSlots, *pready = bars + 2 * kSlots;
    uint64_t *eready = pready + 1, *scaled = pready + 2, *uready = pready + 3, *xready = pready + 4;
    uint64_t *masked = pready + 5, *oready = pready + 6, *efree = pready + 7;
    uint32_t *tslot = reinterpret_cast<uint32_t *>(pready + 8);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int kTma = C::GROUPS * C::NW, kMma = kTma + 1;

    const int seg = blockIdx.x % a.nseg;
    const int64_t bh = blockIdx.x / a.nseg;
    const int b = (int)(bh / a.H), h = (int)(bh % a.H);
    const int len = head_length(a.lengths, b, a.n);
    const int r0 = seg * a.seg_len, rend = min(a.n, r0 + a.seg_len), r1 = max(r0, min(len, rend));
    const int nch = (r1 - r0 + kRows - 1) / kRows;
    const int e = a.reverse ? 0 : 1;
    const float g = decay_log(a.log_decay, h);
    auto chunk_row = [&](int c) { return r0 + (a.reverse ? nch - 1 - c : c) * kRows; };

    if (tid == 0) {
        for (int i = 0; i < kSlots; ++i) { mbar_init(full + i, 1); mbar_init(freeb + i, 1); }
        mbar_init(pready, 1); mbar_init(eready, 1); mbar_init(uready, 1); mbar_init(oready, 1);
        mbar_init(scaled, C::GT); mbar_init(xready, C::GT); mbar_init(masked, C::GT); mbar_init(efree, C::GT);
        fence_mbar_init();
    }
    if (warp == kMma) { tmem_alloc(tslot, C::COLS); tmem_relinquish(); }
    for (int i = tid; i <= kRows; i += C::THREADS) pw[i] = expf(g * (float)i);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tb = *tslot;
    bool failed = false;
    auto wait = [&](uint64_t *bar, uint32_t parity) {  // bounded; a no-op once it has run out
        if (!failed && !mbar_wait(bar, parity)) {
            failed = true;
            atomicOr(a.status, 1);
        }
    };
    // the slot and use of load number L: a (not for states), b, c of each chunk in turn
    constexpr int LOADS = STATE ? 2 : 3;

    if (warp == kTma) {
        if (lane == 0) {
            const int ha = h / (a.H / a.a.heads), hb = h / (a.H / a.b.heads), hc = h / (a.H / a.c.heads);
            int L = 0;
            for (int c = 0; c < nch && !failed; ++c) {
                const int row = chunk_row(c);
#pragma unroll
                for (int w = 3 - LOADS; w < 3; ++w, ++L) {
                    const int s = L % kSlots;
                    if (L >= kSlots) wait(freeb + s, ((L / kSlots) - 1) & 1);
                    if (failed) break;
                    const CUtensorMap *m = w == 0 ? &mapA : w == 1 ? &mapB : &mapC;
                    const int hh = w == 0 ? ha : w == 1 ? hb : hc;
                    mbar_arrive_expect_tx(full + s, C::TILE);
                    for (int k = 0; k < C::KB; ++k)
                        tma_load_4d(sm + s * C::TILE + k * C::BLK, m, 64 * k, row, hh, b, full + s);
                }
            }
        }
    } else if (warp == kMma) {
        if (lane == 0) {
            const uint32_t base = smem_u32(sm);
            const uint64_t dX = sdesc(smem_u32(Xop), C::XBLK, 1024, kSwizzle128);
            const uint64_t dT = sdesc(smem_u32(terms), C::BLK, 1024, kSwizzle128);
            constexpr uint32_t idP = idesc_bf16(128, 128, false, false);
            constexpr uint32_t idE = idesc_bf16(128, D, false, true);
            constexpr uint32_t idU = idesc_bf16(D, D, true, true);
            for (int c = 0; c < nch && !failed; ++c) {
                const int La = c * LOADS, Lb = La + LOADS - 2, Lc = Lb + 1;
                const uint32_t ph = c & 1;
                const uint32_t ta = base + (La % kSlots) * C::TILE, tbb = base + (Lb % kSlots) * C::TILE;
                const uint32_t tc = base + (Lc % kSlots) * C::TILE;
                wait(full + Lb % kSlots, (Lb / kSlots) & 1);
                if (!STATE) {
                    wait(full + La % kSlots, (La / kSlots) & 1);
                    if (c > 0) wait(efree, (c - 1) & 1);
                    if (failed) break;
                    tc_fence_after();
                    const uint64_t dA = sdesc(ta, 16, 1024, kSwizzle128), dB = sdesc(tbb, 16, 1024, kSwizzle128);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t o = (k / 4) * C::BLK + 32 * (k % 4);
                        mma_bf16_ss(tb + C::cP, dadd(dA, o), dadd(dB, o), idP, k > 0);
                    }
                    mma_commit(pready);
                    wait(xready, ph);
                    if (failed) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t o = (k / 4) * C::BLK + 32 * (k % 4);
                        mma_bf16_ss(tb + C::cE, dadd(dA, o), dadd(dX, 2048 * k), idE, k > 0);
                    }
                    mma_commit(eready);
                    mma_commit(freeb + La % kSlots);
                }
                wait(scaled, ph);
                wait(full + Lc % kSlots, (Lc / kSlots) & 1);
                if (failed) break;
                tc_fence_after();
                const uint64_t dB1 = sdesc(tbb, C::BLK, 1024, kSwizzle128), dC = sdesc(tc, C::BLK, 1024, kSwizzle128);
#pragma unroll
                for (int q = 0; q < NT; ++q)
#pragma unroll
                    for (int k = 0; k < kRows / 16; ++k)
                        mma_bf16_ss(tb + C::cU, q == 0 ? dadd(dB1, 2048 * k) : dadd(dT, (q - 1) * C::TILE + 2048 * k),
                                    dadd(dC, 2048 * k), idU, (q | k) != 0);
                mma_commit(uready);
                mma_commit(freeb + Lb % kSlots);
                if (STATE) {
                    mma_commit(freeb + Lc % kSlots);
                } else {
                    wait(masked, ph);
                    if (failed) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < kRows / 16; ++k)
                        mma_bf16_ts(tb + C::cE, tb + C::cP + 8 * k, dadd(dC, 2048 * k), idE, 1);
                    mma_commit(oready);
                    mma_commit(freeb + Lc % kSlots);
                }
            }
        }
    } else if (!STATE && warp < C::NW) {
        // scores and outputs: thread (row, column part); warps w and w + 4 share the rows of quarter w % 4
        constexpr int PARTS = C::NW / 4, PC = kRows / PARTS, EC = D / PARTS;
        const int quarter = warp & 3, part = warp >> 2, i = quarter * 32 + lane;
        const uint32_t lb = (uint32_t)(quarter * 32) << 16;
        OUT *O = static_cast<OUT *>(a.out) + b * a.ob + (int64_t)h * a.oh;
        for (int c = 0; c < nch; ++c) {
            const int row0 = chunk_row(c), nv = min(kRows, r1 - row0);
            const uint32_t ph = c & 1;
            wait(pready, ph);
            tc_fence_after();
            {
                uint32_t w[PC / 2];
#pragma unroll
                for (int q = 0; q < PC / 32; ++q) {
                    uint32_t x[32];
                    tmem_ld32(tb + lb + C::cP + part * PC + 32 * q, x);
                    tmem_wait_ld();
                    float v[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(x[k]);
                    decay_scores(v, i, part * (PC / 32) + q, a.reverse != 0, nv, a.p, pw);
#pragma unroll
                    for (int k = 0; k < 16; ++k) w[16 * q + k] = pack2(v[2 * k], v[2 * k + 1]);
                }
                // the bf16 scores overwrite the first half of P: after both warps of the rows have read theirs
                if (PARTS > 1) {
                    tc_fence_before();
                    asm volatile("bar.sync %0, %1;" ::"r"(1 + quarter), "n"(PARTS * 32) : "memory");
                    tc_fence_after();
                }
#pragma unroll
                for (int q = 0; q < PC / 32; ++q) {
                    uint32_t y[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) y[k] = w[16 * q + k];
                    tmem_st16(tb + lb + C::cP + part * (PC / 2) + 16 * q, y);
                }
            }
            wait(eready, ph);
            tc_fence_after();
            const int m = a.reverse ? nv - 1 - i : i;
            const float xs = a.x * pw[max(0, m) + e];
#pragma unroll
            for (int q = 0; q < EC / 16; ++q) {
                uint32_t x[16];
                tmem_ld16(tb + lb + C::cE + part * EC + 16 * q, x);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(xs * __uint_as_float(x[k]));
                tmem_st16(tb + lb + C::cE + part * EC + 16 * q, x);
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(masked);
            wait(oready, ph);
            tc_fence_after();
            OUT *o = O + (int64_t)(row0 + i) * a.ot + part * EC;
#pragma unroll
            for (int q = 0; q < EC / 32; ++q) {
                uint32_t x[32];
                tmem_ld32(tb + lb + C::cE + part * EC + 32 * q, x);
                tmem_wait_ld();
                if (q == EC / 32 - 1) {
                    tc_fence_before();
                    mbar_arrive(efree);
                }
                if (i < nv) {
#pragma unroll
                    for (int k = 0; k < 32; k += 8)
                        if (part * EC + 32 * q + k < a.dc) {  // dc is a multiple of 8
                            if (sizeof(OUT) == 4) {
                                uint4 *dst = reinterpret_cast<uint4 *>(o + 32 * q + k);
                                dst[0] = make_uint4(x[k], x[k + 1], x[k + 2], x[k + 3]);
                                dst[1] = make_uint4(x[k + 4], x[k + 5], x[k + 6], x[k + 7]);
                            } else {
                                auto f = [&](int z) { return __uint_as_float(x[k + z]); };
                                *reinterpret_cast<uint4 *>(o + 32 * q + k) =
                                    make_uint4(pack2(f(0), f(1)), pack2(f(2), f(3)), pack2(f(4), f(5)), pack2(f(6), f(7)));
                            }
                        }
                }
                __syncwarp();
            }
        }
        // rows at and past the length
        OUT *z = O + (int64_t)r1 * a.ot;
        for (int64_t k = tid; k < (int64_t)(rend - r1) * a.dc; k += C::GT) io_store(z + (k / a.dc) * a.ot + k % a.dc, 0.0f);
    } else {
        // state: thread (feature f, columns c0 ..); the accumulator's row f is lane f, or with 64 rows lane
        // 32 (f / 16) + f % 16
        const int gt = tid - (STATE ? 0 : C::GT), gw = gt >> 5, quarter = warp & 3;
        const bool own = D == 128 || lane < 16;
        const int f = D == 128 ? quarter * 32 + lane : quarter * 16 + (lane & 15);
        const int c0 = D == 128 ? (gw >> 2) * C::CPT : 0;
        const uint32_t lb = (uint32_t)(quarter * 32) << 16;
        const int fr = gt & (kRows - 1), fp = gt / kRows;  // scaling: row of b, part of its 16-byte pieces
        constexpr int FP = C::GT / kRows, PIECES = D / 8 / FP;
        float X[C::CPT];
        {
            const float *x = a.X ? a.X + (bh * a.x_pieces + (a.x_pieces > 1 ? seg : 0)) * a.da * a.dc : nullptr;
#pragma unroll
            for (int k = 0; k < C::CPT; ++k)
                X[k] = x && own && f < a.da && c0 + k < a.dc
                           ? (a.x_trans ? x[(int64_t)(c0 + k) * a.da + f] : x[(int64_t)f * a.dc + c0 + k]) : 0.0f;
        }
        auto put_operand = [&]() {  // X as the bf16 operand
            if (own) {
#pragma unroll
                for (int k = 0; k < C::CPT; k += 8) {
                    const int cc = c0 + k;
                    *reinterpret_cast<uint4 *>(Xop + (cc / 64) * C::XBLK + sw128_chunk(f, (cc % 64) / 8)) =
                        make_uint4(pack2(X[k], X[k + 1]), pack2(X[k + 2], X[k + 3]), pack2(X[k + 4], X[k + 5]),
                                   pack2(X[k + 6], X[k + 7]));
                }
            }
            fence_proxy_async_smem();
            mbar_arrive(xready);
        };
        if (!STATE) put_operand();
        for (int c = 0; c < nch; ++c) {
            const int row0 = chunk_row(c), nv = min(kRows, r1 - row0);
            const uint32_t ph = c & 1;
            const int Lb = c * LOADS + LOADS - 2, Lc = Lb + 1;
            uint8_t *tbb = sm + (Lb % kSlots) * C::TILE, *tcc = sm + (Lc % kSlots) * C::TILE;
            wait(full + Lb % kSlots, (Lb / kSlots) & 1);
            if (!STATE) wait(pready, ph);  // P has read b
            const float w = fr < nv ? pw[nv - (a.reverse ? nv - 1 - fr : fr) - e] : 0.0f;
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                const int piece = fp * PIECES + q;
                const uint32_t off = (piece / 8) * C::BLK + sw128_chunk(fr, piece % 8);
                uint4 v = *reinterpret_cast<const uint4 *>(tbb + off);
                const uint32_t in[4] = {v.x, v.y, v.z, v.w};
                uint32_t o1[4], o2[4], o3[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float lo = __uint_as_float(in[k] << 16) * w, hi = __uint_as_float(in[k] & 0xffff0000u) * w;
                    if (fr >= nv) lo = hi = 0.0f;
                    o1[k] = pack2(lo, hi);
                    lo -= __uint_as_float(o1[k] << 16);
                    hi -= __uint_as_float(o1[k] & 0xffff0000u);
                    o2[k] = pack2(lo, hi);
                    if (NT == 3)
                        o3[k] = pack2(lo - __uint_as_float(o2[k] << 16), hi - __uint_as_float(o2[k] & 0xffff0000u));
                }
                *reinterpret_cast<uint4 *>(tbb + off) = make_uint4(o1[0], o1[1], o1[2], o1[3]);
                *reinterpret_cast<uint4 *>(terms + off) = make_uint4(o2[0], o2[1], o2[2], o2[3]);
                if (NT == 3) *reinterpret_cast<uint4 *>(terms + C::TILE + off) = make_uint4(o3[0], o3[1], o3[2], o3[3]);
            }
            if (nv < kRows) {  // rows past the length may hold anything: c without them
                wait(full + Lc % kSlots, (Lc / kSlots) & 1);
                if (fr >= nv) {
#pragma unroll
                    for (int q = 0; q < PIECES; ++q) {
                        const int piece = fp * PIECES + q;
                        *reinterpret_cast<uint4 *>(tcc + (piece / 8) * C::BLK + sw128_chunk(fr, piece % 8)) =
                            make_uint4(0, 0, 0, 0);
                    }
                }
            }
            fence_proxy_async_smem();
            mbar_arrive(scaled);
            wait(uready, ph);
            tc_fence_after();
            const float dec = pw[nv];
#pragma unroll
            for (int q = 0; q < C::CPT / 16; ++q) {
                uint32_t x[16];
                tmem_ld16(tb + lb + C::cU + c0 + 16 * q, x);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 16; ++k) X[16 * q + k] = fmaf(dec, X[16 * q + k], a.u * __uint_as_float(x[k]));
            }
            tc_fence_before();
            if (!STATE && c + 1 < nch) {
                wait(eready, ph);  // E has read the operand
                put_operand();
            }
        }
        if (a.Xout && own && f < a.da) {
            float *x = a.Xout + (bh * a.nseg + seg) * a.da * a.dc + (int64_t)f * a.dc;
#pragma unroll
            for (int k = 0; k < C::CPT; k += 4)
                if (c0 + k < a.dc) *reinterpret_cast<float4 *>(x + c0 + k) = make_float4(X[k], X[k + 1], X[k + 2], X[k + 3]);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kMma) tmem_dealloc(tb, C::COLS);
}

bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

bool row_map(CUtensorMap *m, const RowView &v, int B, int n, int width) {
    const uint64_t dims[4] = {(uint64_t)width, (uint64_t)n, (uint64_t)v.heads, (uint64_t)B};
    // the stride of a dimension with one entry is never used, but has to be a valid one
    auto st = [&](int64_t s, int ext) { return ext > 1 ? (uint64_t)s * 2 : (uint64_t)256; };
    const uint64_t strides[3] = {st(v.st, n), st(v.sh, v.heads), st(v.sb, B)};
    const uint32_t box[4] = {64, kRows, 1, 1};
    return tc_make_map_nd(m, v.p, 4, dims, strides, box);
}

bool view_ok(const RowView &v, int B, int n) {
    auto ok = [](int64_t s, int ext) { return ext <= 1 || (s > 0 && s % 8 == 0); };
    return al16(v.p) && ok(v.st, n) && ok(v.sh, v.heads) && ok(v.sb, B);
}

template <int D, int NT, bool STATE, typename OUT>
cudaError_t launch(const DecayMix &a, cudaStream_t s) {
    using C = Cfg<D, NT, STATE>;
    CUtensorMap mA, mB, mC;
    if (!row_map(&mB, a.b, a.B, a.n, a.da) || !row_map(&mC, a.c, a.B, a.n, a.dc)) return cudaErrorInvalidValue;
    mA = mB;
    if (!STATE && !row_map(&mA, a.a, a.B, a.n, a.da)) return cudaErrorInvalidValue;
    cudaError_t e = cudaFuncSetAttribute(k_decay_tc<D, NT, STATE, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)((int64_t)a.B * a.H * a.nseg);
    LUNA_LAUNCH(STATE ? "decay_state_tc" : "decay_mix_tc", (k_decay_tc<D, NT, STATE, OUT>), grid, C::THREADS, C::SMEM, s, mA,
                mB, mC, a);
    return cudaGetLastError();
}

template <int D>
cudaError_t pick(const DecayMix &a, luna_dtype out, cudaStream_t s) {
    if (!a.out) return launch<D, 3, true, float>(a, s);
    if (out == LUNA_F32) return a.Xout ? launch<D, 3, false, float>(a, s) : launch<D, 2, false, float>(a, s);
    return a.Xout ? launch<D, 3, false, __nv_bfloat16>(a, s) : launch<D, 2, false, __nv_bfloat16>(a, s);
}

}  // namespace

bool decay_tc_ok(const DecayMix &a, luna_dtype io, luna_dtype out) {
    if (io != LUNA_BF16 || a.da % 8 || a.dc % 8 || !view_ok(a.b, a.B, a.n) || !view_ok(a.c, a.B, a.n)) return false;
    if (a.Xout && !al16(a.Xout)) return false;
    if (!a.out) return true;
    return view_ok(a.a, a.B, a.n) && al16(a.out) && a.ob % 8 == 0 && a.oh % 8 == 0 && a.ot % 8 == 0;
}

cudaError_t launch_decay_mix_tc(const DecayMix &a, luna_dtype out, cudaStream_t s) {
    return a.da <= 64 && a.dc <= 64 ? pick<64>(a, out, s) : pick<128>(a, out, s);
}

}  // namespace luna
