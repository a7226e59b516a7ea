// Linear attention with a decay for each head on tensor cores (bf16, tcgen05 / TMEM / TMA).
//
// A block walks pieces of heads' rows, one after another, in chunks of 128 (a, b, c as in luna_decay.cuh) and keeps the
// state X (da x dc, fp32) in TMEM.  Per chunk of nv rows, m a row's number in processing order:
//     MMA    P = a b^T,  E = a X                       (X as a bf16 operand)
//     warps  P masked and decayed, as bf16 back into TMEM;  E scaled by x lambda^{m+e} in place
//            b scaled by lambda^{nv-m-e} into bf16 terms b1 + b2 (+ b3)
//     MMA    U = (b1 + b2 (+ b3))^T c,  E += P c
//     warps  out = E;  X = lambda^{nv} X + u U, and its bf16 operand
// The decay sits on b alone, so c enters U as it is; one bf16 rounding of the scaled b would cost the
// state 1.7e-3, two terms leave 3e-6 and three 2^-24.  Passes whose state leaves the kernel use three,
// the others two (their state only enters outputs as one more bf16 rounding).  X is not accumulated by
// the products themselves: their additions onto a large X round toward zero, chunk after chunk.
//
// P and the operand X are one bf16 rounding each, which outputs carry beside their own (2.3e-3 to 2.5e-3 off where
// that alone leaves 1.7e-3) and no state does.  A second term of both would add a D-deep and a 128-deep product to the
// chain below, and at D = 128 another 32 KB of operand to shared memory, which is full.
//
// Measured: 115 us for 128 heads of 4096 rows at d = dv = 128 (537 MB, 4.7 TB/s), issue 34 %, tensor 31 %.
// Bound: the chain of the steps above, some 5000 cycles a chunk at d = 128.  By its bytes the pass is (da + dc) * 4
// bytes a row at HBM rate; the shared-memory traffic of the products' operands and of the scaled terms comes next
// (about 2/3 of that at d = 128).  Three
// groups of warps (the scaled b; X; P and out) work on their parts of neighbouring chunks side by side,
// and the next tiles load while they do: a ring of four slots takes a, b, c in turn.
#include <math.h>
#include <string.h>

#include "luna_decay.cuh"
#include "luna_prof.cuh"
#include "luna_sm100.cuh"

namespace luna {

int tc_sm_count();
bool tc_make_map_nd(CUtensorMap *m, const void *base, int rank, const uint64_t *dims, const uint64_t *strides,
                    const uint32_t *box, int swizzle = 128);

namespace {
using namespace sm100;

constexpr int kRows = 128;   // rows of a chunk
constexpr int kAhead = 2;    // chunks whose tiles L2 is asked for in advance

template <int D, int NT, bool STATE> struct Cfg {
    static constexpr int SCALE = 8, STATEW = 8, SCORE = 8;  // warps of each of the three groups
    static constexpr int WARPS = SCALE + STATEW + (STATE ? 0 : SCORE);
    // At D = 64 there is room for two chunks and more, and a block stays for many (short) pieces, whose
    // starts and ends then pass under each other's work; at D = 128 that costs registers that the score
    // warps do not have (5 % at 152 long pieces).
    static constexpr int SLOTS = D == 64 ? 8 : 4;
    static constexpr bool STAYS = D == 64;
    static constexpr int THREADS = WARPS * 32 + 64;
    static constexpr int KB = D / 64;               // 64-column blocks of a row
    static constexpr uint32_t BLK = kRows * 128;    // one block of a tile
    static constexpr uint32_t TILE = KB * BLK;
    static constexpr uint32_t XBLK = D * 128, XOP = KB * XBLK;  // X operand: [64-column block][feature][64]
    // the terms of b, half a chunk at a time: b1 takes b's own place where there is no room beside it, and
    // then waits for P to have read b
    static constexpr bool INPLACE = D == 128 && NT == 3;
    static constexpr int TERMS = INPLACE ? NT - 1 : NT;
    static constexpr uint32_t SMEM = SLOTS * TILE + TERMS * TILE + (STATE ? 0 : XOP) + 2048 + 1024;
    static_assert(SMEM <= 227 * 1024, "shared memory");
    // TMEM columns: U | E | P (the bf16 form of each 64 columns in their first 32) | X
    static constexpr uint32_t cU = 0, cE = D, cP = 2 * D, cX = STATE ? D : 2 * D + 128;
    static constexpr uint32_t COLS = STATE ? 2 * D : 512;
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

__device__ __forceinline__ uint32_t pack2(uint64_t v) {
    float lo, hi;
    unpack2(v, lo, hi);
    return pack2(lo, hi);
}
__device__ __forceinline__ uint64_t widen2(uint32_t bf) { return f2(bf << 16, bf & 0xffff0000u); }

// Decays of the diagonal block by x = column - row + 31: four copies, the m-th shifted by m, so that any
// row's 32 are whole 16-byte loads, and 72 floats apart, so that a warp's fall into different banks.
constexpr int kDiagCopy = 72;

// 32 scores of row i, columns 32 jb .. (TMEM address `taddr`): masked, decayed, times p, as bf16 pairs.
// Off the diagonal block the decay is a factor of the row times one of the column (both at most 1 for
// lambda <= 1), on it it comes from the table of decays by distance, 0 where the distance is negative.
__device__ __forceinline__ void decay_scores(uint32_t taddr, int i, int jb, bool reverse, int nv, float p,
                                             const float *pw, const float *diag, const float *cols, uint32_t (&w)[16]) {
    const int ib = i >> 5, li = i & 31, j0 = 32 * jb;
    if (reverse ? jb < ib : jb > ib) {  // the same for the whole warp
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] = 0u;
        return;
    }
    uint32_t x[32];
    tmem_ld32(taddr, x);
    if (jb == ib) {
        const int m = (31 - li) & 3;
        const float4 *t = reinterpret_cast<const float4 *>(diag + m * kDiagCopy + 31 - li - m);
        tmem_wait_ld();
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float4 c = t[q];
            w[2 * q] = pack2(mul2(f2(x[4 * q], x[4 * q + 1]), f2(c.x, c.y)));
            w[2 * q + 1] = pack2(mul2(f2(x[4 * q + 2], x[4 * q + 3]), f2(c.z, c.w)));
        }
    } else {
        const float row = p * (reverse ? pw[j0 - i] : pw[i - j0 - 31]);
        const uint64_t row2 = f2(row, row);
        const float4 *t = reinterpret_cast<const float4 *>(cols);
        tmem_wait_ld();
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float4 c = t[q];
            w[2 * q] = pack2(mul2(f2(x[4 * q], x[4 * q + 1]), mul2(row2, f2(c.x, c.y))));
            w[2 * q + 1] = pack2(mul2(f2(x[4 * q + 2], x[4 * q + 3]), mul2(row2, f2(c.z, c.w))));
        }
    }
    if (nv < kRows) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t keep = i >= nv ? 0u : (j0 + 2 * j < nv ? 0xffffu : 0u) | (j0 + 2 * j + 1 < nv ? 0xffff0000u : 0u);
            w[j] &= keep;
        }
    }
}

// One piece of a head's rows.
struct Piece {
    int seg, b, h, r0, rend, r1, nch, reverse;  // rows r0 .. rend, those below r1 valid, nch chunks of them
    int64_t bh;
    float g;
    __device__ __forceinline__ Piece(const DecayMix &a, int item) {
        seg = item % a.nseg;
        bh = item / a.nseg;
        b = (int)(bh / a.H);
        h = (int)(bh % a.H);
        r0 = seg * a.seg_len;
        rend = min(a.n, r0 + a.seg_len);
        r1 = max(r0, min(head_length(a.lengths, b, a.n), rend));
        nch = (r1 - r0 + kRows - 1) / kRows;
        reverse = a.reverse;
        g = decay_log(a.log_decay, h);
    }
    __device__ __forceinline__ int row(int c) const { return r0 + (reverse ? nch - 1 - c : c) * kRows; }
    __device__ __forceinline__ int valid(int c) const { return min(kRows, r1 - row(c)); }
    __device__ __forceinline__ float power(int k) const { return expf(g * (float)k); }
};

template <int D, int NT, bool STATE, typename OUT>
__global__ void __launch_bounds__(Cfg<D, NT, STATE>::THREADS, 1)
    k_decay_tc(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
               const __grid_constant__ CUtensorMap mapC, const __grid_constant__ CUtensorMap mapO,
               const __grid_constant__ DecayMix a) {
    using C = Cfg<D, NT, STATE>;
    constexpr bool STAGED = !STATE && sizeof(OUT) == 2;  // bf16 outputs leave by TMA from the chunk's c slot
    constexpr int kSlots = C::SLOTS, kScaleWarps = C::SCALE, kStateWarps = C::STATEW, kScoreWarps = C::SCORE;
    extern __shared__ uint8_t smem_raw[];
    clear_status(a);
    uint8_t *sm = align_1024(smem_raw);
    uint8_t *terms = sm + kSlots * C::TILE;
    uint8_t *Xop = terms + C::TERMS * C::TILE;
    float *pw = reinterpret_cast<float *>(Xop + (STATE ? 0 : C::XOP));  // lambda^0 .. lambda^128 of the scores' warps' piece
    float *diag = pw + 132;
    float *cols = diag + 4 * kDiagCopy;  // of column j of a block: lambda^{31 - j}, in reverse order lambda^j
    uint64_t *bars = reinterpret_cast<uint64_t *>(cols + 32);
    uint64_t *full = bars, *freeb = bars + kSlots, *pready = bars + 2 * kSlots;
    uint64_t *eready = pready + 1, *scaled = pready + 2 /* of each half */, *uread = pready + 4 /* of each half */;
    uint64_t *xready = pready + 6, *masked = pready + 7, *oready = pready + 8, *efree = pready + 9, *ufree = pready + 10;
    uint64_t *stored = pready + 11;
    uint32_t *tslot = reinterpret_cast<uint32_t *>(pready + 12);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int kTma = C::WARPS, kMma = kTma + 1;
    constexpr int kScoreWarp0 = kScaleWarps + kStateWarps;

    const int items = a.B * a.H * a.nseg, e = a.reverse ? 0 : 1;

    if (tid == 0) {
        for (int i = 0; i < kSlots; ++i) { mbar_init(full + i, 1); mbar_init(freeb + i, 1); }
        mbar_init(pready, 1); mbar_init(eready, 1); mbar_init(oready, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(scaled + i, kScaleWarps); mbar_init(uread + i, 1); }
        mbar_init(xready, kStateWarps); mbar_init(ufree, kStateWarps);
        mbar_init(masked, kScoreWarps); mbar_init(efree, kScoreWarps); mbar_init(stored, kScoreWarps * D / 128);
        fence_mbar_init();
    }
    if (warp == kMma) { tmem_alloc(tslot, C::COLS); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tb = *tslot;
    bool failed = false;
    auto wait = [&](uint64_t *bar, uint32_t parity) {  // bounded; a no-op once it has run out
        // (the states' kernel, whose code is small, has the waits in line: 9 % there)
        if (!failed && !(STATE ? mbar_wait(bar, parity) : mbar_wait_long(bar, parity))) {
            failed = true;
            atomicOr(a.status, 1);
        }
    };
    auto arrive = [&](uint64_t *bar) {  // once for the warp, after all its lanes
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
    };
    // the slot and use of load number L: a (not for states), b, c of each chunk in turn; every role counts the
    // chunks of all its block's pieces (gc), and barrier phases and loads go by that count
    constexpr int LOADS = STATE ? 2 : 3;
    int base_c = 0;

    if (warp == kTma) {
        if (lane == 0) {
            uint32_t uses = 0;  // bit s: parity of the phases of freeb[s] waited for
            int issued = 0;
            for (int item = blockIdx.x; item < items && !failed; item += gridDim.x) {
                const Piece t(a, item);
                const int head[3] = {t.h / (a.H / a.a.heads), t.h / (a.H / a.b.heads), t.h / (a.H / a.c.heads)};
                for (int c = 0; c < t.nch && !failed; ++c) {
                    // the slots hold little more than a chunk, less than a load's way from DRAM: ask L2 for the tiles
                    // two chunks ahead
                    for (int cp = c == 0 ? 1 : c + kAhead; cp <= c + kAhead && cp < t.nch; ++cp)
#pragma unroll
                        for (int w = 3 - LOADS; w < 3; ++w)
                            for (int k = 0; k < C::KB; ++k)
                                tma_prefetch_4d(w == 0 ? &mapA : w == 1 ? &mapB : &mapC, 64 * k, t.row(cp), head[w], t.b);
                    const int row = t.row(c);
#pragma unroll
                    for (int w = 3 - LOADS; w < 3; ++w) {
                        const int L = (base_c + c) * LOADS + w - (3 - LOADS), s = L % kSlots;
                        if (STAGED && L >= kSlots && (L - kSlots) % LOADS == LOADS - 1) {
                            wait(stored, ((L - kSlots) / LOADS) & 1);  // the slot held c and then the outputs
                        } else if (L >= kSlots) {
                            wait(freeb + s, (uses >> s) & 1);
                            uses ^= 1u << s;
                        }
                        if (failed) break;
                        const CUtensorMap *m = w == 0 ? &mapA : w == 1 ? &mapB : &mapC;
                        mbar_arrive_expect_tx(full + s, C::TILE);
                        for (int k = 0; k < C::KB; ++k)
                            tma_load_4d(sm + s * C::TILE + k * C::BLK, m, 64 * k, row, head[w], t.b, full + s);
                        issued = L + 1;
                    }
                }
                if (!C::STAYS) break;
                base_c += t.nch;
            }
            // no load may be on its way when the block ends, which one that has given up elsewhere would not wait for
            for (int L = max(0, issued - kSlots); L < issued; ++L) mbar_wait(full + L % kSlots, (L / kSlots) & 1, kDrainNs);
        }
    } else if (warp == kMma) {
        if (lane == 0) {
            const uint32_t base = smem_u32(sm);
            const uint64_t dX = sdesc(smem_u32(Xop), C::XBLK, 1024, kSwizzle128);
            const uint64_t dT = sdesc(smem_u32(terms), C::BLK, 1024, kSwizzle128);
            constexpr uint32_t idP = idesc_bf16(128, 128, false, false);
            constexpr uint32_t idE = idesc_bf16(128, D, false, true);
            constexpr uint32_t idU = idesc_bf16(D, D, true, true);
            auto slot_addr = [&](int L) { return base + (L % kSlots) * C::TILE; };
            auto scores = [&](int gc) {  // P = a b^T of chunk gc
                const int La = gc * LOADS, Lb = La + 1;
                wait(full + La % kSlots, (La / kSlots) & 1);
                wait(full + Lb % kSlots, (Lb / kSlots) & 1);
                if (gc > 0) wait(oready, (gc - 1) & 1);  // the last chunk's scores have been read
                if (failed) return;
                tc_fence_after();
                const uint64_t dA = sdesc(slot_addr(La), 16, 1024, kSwizzle128), dB = sdesc(slot_addr(Lb), 16, 1024, kSwizzle128);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t o = (k / 4) * C::BLK + 32 * (k % 4);
                    mma_bf16_ss(tb + C::cP, dadd(dA, o), dadd(dB, o), idP, k > 0);
                }
                mma_commit(pready);
            };
            for (int item = blockIdx.x; item < items && !failed; item += gridDim.x) {
                const int nch = Piece(a, item).nch;
                for (int c = 0; c < nch && !failed; ++c) {
                    const int gc = base_c + c, La = gc * LOADS, Lb = La + LOADS - 2, Lc = Lb + 1;
                    const uint32_t ph = gc & 1;
                    if (!STATE && c == 0) scores(gc);
                    if (!STATE) {
                        wait(xready, ph);
                        if (gc > 0) wait(efree, (gc - 1) & 1);
                        if (failed) break;
                        tc_fence_after();
                        const uint64_t dA = sdesc(slot_addr(La), 16, 1024, kSwizzle128);
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint32_t o = (k / 4) * C::BLK + 32 * (k % 4);
                            mma_bf16_ss(tb + C::cE, dadd(dA, o), dadd(dX, 2048 * k), idE, k > 0);
                        }
                        mma_commit(eready);
                        mma_commit(freeb + La % kSlots);
                    }
                    wait(full + Lc % kSlots, (Lc / kSlots) & 1);
                    if (STATE && gc > 0) wait(ufree, (gc - 1) & 1);  // (otherwise before X was ready)
                    const uint64_t dB1 = sdesc(C::INPLACE ? slot_addr(Lb) : smem_u32(terms), C::BLK, 1024, kSwizzle128);
                    const uint64_t dB2 = sdesc(smem_u32(terms) + (C::INPLACE ? 0 : C::TILE), C::BLK, 1024, kSwizzle128);
                    const uint64_t dC = sdesc(slot_addr(Lc), C::BLK, 1024, kSwizzle128);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        wait(scaled + half, ph);
                        if (failed) break;
                        tc_fence_after();
#pragma unroll
                        for (int q = 0; q < NT; ++q)
#pragma unroll
                            for (int k = 4 * half; k < 4 * half + 4; ++k)
                                mma_bf16_ss(tb + C::cU, q == 0 ? dadd(dB1, 2048 * k) : dadd(dB2, (q - 1) * C::TILE + 2048 * k),
                                            dadd(dC, 2048 * k), idU, (half | q | (k & 3)) != 0);
                        mma_commit(uread + half);
                    }
                    if (failed) break;
                    mma_commit(freeb + Lb % kSlots);
                    if (STATE) {
                        mma_commit(freeb + Lc % kSlots);
                    } else {
                        wait(masked, ph);
                        if (failed) break;
                        tc_fence_after();
#pragma unroll
                        for (int k = 0; k < kRows / 16; ++k)
                            mma_bf16_ts(tb + C::cE, tb + C::cP + 64 * (k / 4) + 8 * (k % 4), dadd(dC, 2048 * k), idE, 1);
                        mma_commit(oready);
                        if (!STAGED) mma_commit(freeb + Lc % kSlots);
                        if (c + 1 < nch) scores(gc + 1);
                    }
                }
                if (!C::STAYS) break;
                base_c += nch;
            }
        }
    } else if (warp < kScaleWarps) {
        // the scaled terms of b, rows of the first half and then of the second: thread (row, part of its pieces)
        constexpr int PIECES = D / 8 / (kScaleWarps * 32 / 64);
        const int hr = tid & 63, piece0 = (tid >> 6) * PIECES;
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            const Piece t(a, item);
            for (int c = 0; c < t.nch; ++c) {
                const int nv = t.valid(c), gc = base_c + c;
                const uint32_t ph = gc & 1;
                const int Lb = gc * LOADS + LOADS - 2, Lc = Lb + 1;
                uint8_t *tbb = sm + (Lb % kSlots) * C::TILE, *tcc = sm + (Lc % kSlots) * C::TILE;
                uint8_t *t1 = C::INPLACE ? tbb : terms, *t2 = terms + (C::INPLACE ? 0 : C::TILE);
                wait(full + Lb % kSlots, (Lb / kSlots) & 1);
                if (!STATE && C::INPLACE) wait(pready, ph);  // P has read b
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    const int r = half * 64 + hr;
                    const bool on = r < nv;
                    const float w = on ? a.u * t.power(nv - (a.reverse ? nv - 1 - r : r) - e) : 0.0f;
                    const uint64_t w2 = f2(w, w), minus = f2(-1.0f, -1.0f);
                    uint4 in4[PIECES];
#pragma unroll
                    for (int q = 0; q < PIECES; ++q)
                        in4[q] = *reinterpret_cast<const uint4 *>(tbb + ((piece0 + q) / 8) * C::BLK +
                                                                  sw128_chunk(r, (piece0 + q) % 8));
                    if (gc > 0) wait(uread + half, (gc - 1) & 1);  // the last chunk's terms have been read
#pragma unroll
                    for (int q = 0; q < PIECES; ++q) {
                        const uint32_t off = ((piece0 + q) / 8) * C::BLK + sw128_chunk(r, (piece0 + q) % 8);
                        uint4 v = in4[q];
                        if (!on) v = make_uint4(0, 0, 0, 0);  // rows past the length may hold anything
                        const uint32_t in[4] = {v.x, v.y, v.z, v.w};
                        uint32_t o1[4], o2[4], o3[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint64_t x = mul2(widen2(in[k]), w2);
                            o1[k] = pack2(x);
                            x = fma2(widen2(o1[k]), minus, x);
                            o2[k] = pack2(x);
                            if (NT == 3) o3[k] = pack2(fma2(widen2(o2[k]), minus, x));
                        }
                        *reinterpret_cast<uint4 *>(t1 + off) = make_uint4(o1[0], o1[1], o1[2], o1[3]);
                        *reinterpret_cast<uint4 *>(t2 + off) = make_uint4(o2[0], o2[1], o2[2], o2[3]);
                        if (NT == 3) *reinterpret_cast<uint4 *>(t2 + C::TILE + off) = make_uint4(o3[0], o3[1], o3[2], o3[3]);
                    }
                    if (nv < kRows) {  // c without the rows past the length
                        wait(full + Lc % kSlots, (Lc / kSlots) & 1);
                        if (!on) {
#pragma unroll
                            for (int q = 0; q < PIECES; ++q)
                                *reinterpret_cast<uint4 *>(tcc + ((piece0 + q) / 8) * C::BLK + sw128_chunk(r, (piece0 + q) % 8)) =
                                    make_uint4(0, 0, 0, 0);
                        }
                    }
                    fence_proxy_async_smem();
                    // These warps read b alone, and b's slot held an a before: its load is known to be complete only by P
                    // of that chunk, and without that the wait for b would take the phase before a's load for b's.  Before
                    // the arrival that lets this chunk's last products go ahead, so that P is never two phases on.
                    if (!STATE && !C::INPLACE && half == 1) wait(pready, ph);
                    arrive(scaled + half);
                }
            }
            if (!C::STAYS) break;
            base_c += t.nch;
        }
    } else if (warp < kScoreWarp0) {
        constexpr int SC = D / (kStateWarps / 4);
        // state: thread (feature f, SC of the columns); an accumulator's row f is lane f, or with 64 rows lane
        // 32 (f / 16) + f % 16
        const int quarter = warp & 3, cc0 = ((warp - kScaleWarps) >> 2) * SC;
        const bool own = D == 128 || lane < 16;
        const int f = D == 128 ? quarter * 32 + lane : quarter * 16 + (lane & 15);
        const uint32_t lb = (uint32_t)(quarter * 32) << 16;
        auto put_operand = [&](int cc, const float (&x)[16]) {  // columns cc .. of X as bf16
            if (own) {
#pragma unroll
                for (int k = 0; k < 16; k += 8)
                    *reinterpret_cast<uint4 *>(Xop + ((cc + k) / 64) * C::XBLK + sw128_chunk(f, ((cc + k) % 64) / 8)) =
                        make_uint4(pack2(x[k], x[k + 1]), pack2(x[k + 2], x[k + 3]), pack2(x[k + 4], x[k + 5]),
                                   pack2(x[k + 6], x[k + 7]));
            }
        };
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            const Piece t(a, item);
            const float *X0 = a.X ? a.X + (t.bh * a.x_pieces + (a.x_pieces > 1 ? t.seg : 0)) * a.da * a.dc : nullptr;
#pragma unroll 1
            for (int cc = cc0; cc < cc0 + SC; cc += 16) {
                float x[16];
                uint32_t y[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    x[k] = X0 && own && f < a.da && cc + k < a.dc
                               ? (a.x_trans ? X0[(int64_t)(cc + k) * a.da + f] : X0[(int64_t)f * a.dc + cc + k]) : 0.0f;
                    y[k] = __float_as_uint(x[k]);
                }
                tmem_st16(tb + lb + C::cX + cc, y);
                if (!STATE && t.nch > 0) put_operand(cc, x);
            }
            tmem_wait_st();
            if (!STATE && t.nch > 0) {
                fence_proxy_async_smem();
                arrive(xready);
            }
            for (int c = 0; c < t.nch; ++c) {
                const uint32_t ph = (base_c + c) & 1;
                const float dec = t.power(t.valid(c));
                wait(uread + 1, ph);
                if (!STATE) wait(eready, ph);  // E has read the operand
                tc_fence_after();
                const uint64_t dec2 = f2(dec, dec);
                // (one copy of the code where two more groups of warps compete for the instruction cache)
                constexpr int kUnroll = STATE ? SC / 16 : 1;
#pragma unroll kUnroll
                for (int c1 = 0; c1 < SC; c1 += 16) {
                    const int cc = cc0 + c1;
                    uint32_t xu[16], xx[16];
                    tmem_ld16(tb + lb + C::cU + cc, xu);
                    tmem_ld16(tb + lb + C::cX + cc, xx);
                    tmem_wait_ld();
                    float x[16];
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        unpack2(fma2(dec2, f2(xx[k], xx[k + 1]), f2(xu[k], xu[k + 1])), x[k], x[k + 1]);
                        xx[k] = __float_as_uint(x[k]);
                        xx[k + 1] = __float_as_uint(x[k + 1]);
                    }
                    tmem_st16(tb + lb + C::cX + cc, xx);
                    if (!STATE && c + 1 < t.nch) put_operand(cc, x);
                }
                tmem_wait_st();
                tc_fence_before();
                if (STATE) {
                    arrive(ufree);
                } else if (c + 1 < t.nch) {
                    fence_proxy_async_smem();
                    arrive(xready);
                }
            }
            if (a.Xout) {
                float *X = a.Xout + (t.bh * a.nseg + t.seg) * a.da * a.dc + (int64_t)f * a.dc;
#pragma unroll 1
                for (int cc = cc0; cc < cc0 + SC; cc += 16) {
                    uint32_t x[16];
                    tmem_ld16(tb + lb + C::cX + cc, x);
                    tmem_wait_ld();
                    if (own && f < a.da) {
#pragma unroll
                        for (int k = 0; k < 16; k += 4)
                            if (cc + k < a.dc) *reinterpret_cast<uint4 *>(X + cc + k) = make_uint4(x[k], x[k + 1], x[k + 2], x[k + 3]);
                    }
                    __syncwarp();
                }
            }
            if (!C::STAYS) break;
            base_c += t.nch;
        }
    } else if (!STATE) {
        // scores and outputs: thread (row, 1 / PARTS of the columns); PARTS warps share a quarter's rows
        constexpr int PARTS = kScoreWarps / 4, PC = kRows / PARTS, EC = D / PARTS;
        const int gw = warp - kScoreWarp0, quarter = warp & 3, part = gw >> 2, i = quarter * 32 + lane;
        const uint32_t lb = (uint32_t)(quarter * 32) << 16;
        constexpr int GT = kScoreWarps * 32;
        const int gt = tid - kScoreWarp0 * 32;
        const bool stores = lane == 0 && (D == 128 || part == 0);
        auto give_slot = [&]() {  // the last chunk's outputs have left their slot
            if (stores) {
                bulk_wait_read();
                mbar_arrive(stored);
            }
            __syncwarp();
        };
        auto group_sync = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(GT) : "memory"); };
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            const Piece t(a, item);
            OUT *O = static_cast<OUT *>(a.out) + t.b * a.ob + (int64_t)t.h * a.oh;
            group_sync();  // the last piece's decays have been used
            for (int k = gt; k <= kRows; k += GT) pw[k] = t.power(k);
            for (int k = gt; k < 4 * kDiagCopy; k += GT) {
                const int dist = (k % kDiagCopy + k / kDiagCopy - 31) * (a.reverse ? 1 : -1);
                diag[k] = dist >= 0 && dist < 32 ? a.p * t.power(dist) : 0.0f;
            }
            if (gt < 32) cols[gt] = t.power(a.reverse ? gt : 31 - gt);
            group_sync();
            for (int c = 0; c < t.nch; ++c) {
                const int row0 = t.row(c), nv = t.valid(c), gc = base_c + c;
                const uint32_t ph = gc & 1;
                wait(pready, ph);
                tc_fence_after();
#pragma unroll 1
                for (int q = 0; q < PC / 32; ++q) {  // the bf16 scores take the place of columns that this warp has read
                    const int blk = part * (PC / 32) + q;
                    uint32_t w[16];
                    decay_scores(tb + lb + C::cP + 32 * blk, i, blk, a.reverse != 0, nv, a.p, pw, diag, cols, w);
                    tmem_st16(tb + lb + C::cP + 64 * (blk / 2) + 16 * (blk % 2), w);
                }
                if (STAGED && gc > 0) give_slot();
                wait(eready, ph);
                tc_fence_after();
                const int m = a.reverse ? nv - 1 - i : i;
                const float xs = a.x * pw[max(0, m) + e];
                const uint64_t xs2 = f2(xs, xs);
#pragma unroll 1
                for (int q = 0; q < EC / 32; ++q) {
                    uint32_t x[32];
                    tmem_ld32(tb + lb + C::cE + part * EC + 32 * q, x);
                    tmem_wait_ld();
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        uint32_t y[16];
#pragma unroll
                        for (int k = 0; k < 16; k += 2) {
                            float lo, hi;
                            unpack2(mul2(xs2, f2(x[16 * s + k], x[16 * s + k + 1])), lo, hi);
                            y[k] = __float_as_uint(lo);
                            y[k + 1] = __float_as_uint(hi);
                        }
                        tmem_st16(tb + lb + C::cE + part * EC + 32 * q + 16 * s, y);
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                arrive(masked);
                wait(oready, ph);
                tc_fence_after();
                const int Lc = gc * LOADS + LOADS - 1;
                uint8_t *tcc = sm + (Lc % kSlots) * C::TILE;  // U and the scores' product have read c
                OUT *o = O + (int64_t)(row0 + i) * a.ot + part * EC;
#pragma unroll 1
                for (int q = 0; q < EC / 32; ++q) {
                    uint32_t x[32];
                    tmem_ld32(tb + lb + C::cE + part * EC + 32 * q, x);
                    tmem_wait_ld();
                    if (q == EC / 32 - 1) {
                        tc_fence_before();
                        arrive(efree);
                    }
                    const int cc = part * EC + 32 * q;
                    if (STAGED) {
#pragma unroll
                        for (int k = 0; k < 32; k += 8) {
                            uint4 v = make_uint4(0, 0, 0, 0);
                            if (i < nv)
                                v = make_uint4(pack2(f2(x[k], x[k + 1])), pack2(f2(x[k + 2], x[k + 3])),
                                               pack2(f2(x[k + 4], x[k + 5])), pack2(f2(x[k + 6], x[k + 7])));
                            *reinterpret_cast<uint4 *>(tcc + (cc / 64) * C::BLK + sw128_chunk(i, (cc % 64 + k) / 8)) = v;
                        }
                    } else if (i < nv) {
#pragma unroll
                        for (int k = 0; k < 32; k += 8)
                            if (cc + k < a.dc) {  // dc is a multiple of 8
                                uint4 *dst = reinterpret_cast<uint4 *>(o + 32 * q + k);
                                dst[0] = make_uint4(x[k], x[k + 1], x[k + 2], x[k + 3]);
                                dst[1] = make_uint4(x[k + 4], x[k + 5], x[k + 6], x[k + 7]);
                            }
                    }
                    __syncwarp();
                }
                if (STAGED) {  // 32 rows of a 64-column block at a time: a warp's own, or with D = 64 its pair's
                    fence_proxy_async_smem();
                    if (D == 64) asm volatile("bar.sync %0, 64;" ::"r"(2 + quarter) : "memory");
                    else __syncwarp();
                    if (stores) {
                        const int blk = D == 128 ? part : 0, row = row0 + quarter * 32;
                        if (row < a.n && 64 * blk < a.dc)
                            tma_store_4d(&mapO, tcc + blk * C::BLK + quarter * 4096, 64 * blk, row, t.h, t.b);
                        bulk_commit();
                    }
                    __syncwarp();
                }
            }
            // rows at and past the length
            constexpr int ZB = 16 / (int)sizeof(OUT);
            const int pieces = a.dc / ZB, step = GT / pieces;
            const int zr = STAGED ? min(t.rend, t.r0 + t.nch * kRows) : t.r1;  // staged chunks have written theirs
            OUT *z = O + (int64_t)zr * a.ot + (gt % pieces) * ZB;
            if (gt < step * pieces)
                for (int k = gt / pieces; k < t.rend - zr; k += step)
                    *reinterpret_cast<uint4 *>(z + (int64_t)k * a.ot) = make_uint4(0, 0, 0, 0);
            if (!C::STAYS) break;
            base_c += t.nch;
        }
        if (STAGED && stores) bulk_wait();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kMma) tmem_dealloc(tb, C::COLS);
}

bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

bool row_map(CUtensorMap *m, const RowView &v, int B, int n, int width, int rows = kRows) {
    const uint64_t dims[4] = {(uint64_t)width, (uint64_t)n, (uint64_t)v.heads, (uint64_t)B};
    // the stride of a dimension with one entry is never used, but has to be a valid one
    auto st = [&](int64_t s, int ext) { return ext > 1 ? (uint64_t)s * 2 : (uint64_t)256; };
    const uint64_t strides[3] = {st(v.st, n), st(v.sh, v.heads), st(v.sb, B)};
    const uint32_t box[4] = {64, (uint32_t)rows, 1, 1};
    return tc_make_map_nd(m, v.p, 4, dims, strides, box);
}

bool view_ok(const RowView &v, int B, int n) {
    auto ok = [](int64_t s, int ext) { return ext <= 1 || (s > 0 && s % 8 == 0); };
    return al16(v.p) && ok(v.st, n) && ok(v.sh, v.heads) && ok(v.sb, B);
}

template <int D, int NT, bool STATE, typename OUT>
cudaError_t launch(const DecayMix &a, cudaStream_t s) {
    using C = Cfg<D, NT, STATE>;
    CUtensorMap mA, mB, mC, mO;
    if (!row_map(&mB, a.b, a.B, a.n, a.da) || !row_map(&mC, a.c, a.B, a.n, a.dc)) return cudaErrorInvalidValue;
    mA = mO = mB;
    if (!STATE && !row_map(&mA, a.a, a.B, a.n, a.da)) return cudaErrorInvalidValue;
    if (!STATE && sizeof(OUT) == 2 && !row_map(&mO, RowView{a.out, a.ob, a.oh, a.ot, a.H}, a.B, a.n, a.dc, 32))
        return cudaErrorInvalidValue;
    cudaError_t e = cudaFuncSetAttribute(k_decay_tc<D, NT, STATE, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    if (e != cudaSuccess) return e;
    const int64_t items = (int64_t)a.B * a.H * a.nseg;
    const unsigned grid = (unsigned)(C::STAYS && items > tc_sm_count() ? tc_sm_count() : items);
    LUNA_LAUNCH(STATE ? "decay_state_tc" : "decay_mix_tc", (k_decay_tc<D, NT, STATE, OUT>), grid, C::THREADS, C::SMEM, s, mA,
                mB, mC, mO, a);
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
