// Matrix products with a fused epilogue on tensor cores (bf16, tcgen05 / TMEM / TMA).
//
// Persistent blocks walk the output tiles.  One thread loads 64-deep slices of A and B by TMA into a
// ring of shared-memory stages, one thread issues the products of each full stage into one of two
// TMEM accumulators, and eight warps carry the other accumulator through the epilogue (bias, kept
// pre-activation, activation, residual, one rounding), so that the products of the next tile never
// wait for it.  Either operand may be stored along the other dimension (k x rows, as the gradients'
// operands are): its slices then are read as MN-major operands, without a transposed copy.
//
// CG = 2: two CTAs of a cluster share a 256 x BN tile.  Each holds its 128 rows of A and half of B
// (a CTA alone has to read A and all of B from its shared memory for every product, which the
// shared-memory bandwidth does not sustain at 128 x 256), and the leader's thread issues the products
// of both.  TMA zero-fills past every edge and drops what a store holds past it.  The epilogue's warps
// hand 32 x 32 pieces to TMA stores (a lane's own row, written directly, would touch 32 lines an
// instruction: 20 to 40 % of the whole product at a depth of 1024).  At 16333 x 4096 x 1024: 95 us (1440
// TFLOP/s), with gelu 132 us, where the epilogue bounds it.
//
// fp32 operands come as three bf16 planes, x = x0 + x1 + x2 exactly (eight bits each), and a b is the sum
// of the six products a2 b0 + a1 b1 + a0 b2 + a1 b0 + a0 b1 + a0 b0; what is left out is under 2^-21 of
// |a| |b|.  A stage holds one plane of both operands, and the products of three stages run together, the
// small ones first: loading each product's planes anew took the L2 twice the bytes and half as long
// again (917 us at 4096 x 4096 x 4096, now 719 to 726 us, of which the splitting takes 60).  The tensor
// cores add to their fp32 accumulator by cutting off, which at a depth of 1024 has lost 1.7e-6 of a sum of
// positive products and at 64 1e-7 (measured), so after every 64 of K the epilogue's warps add the
// accumulator to an fp32 sum that they keep in TMEM beside it.  bf16 sums over more than 65536 of K are joined like this every 16384 (LONG): cut off all the
// way, 2^20 rows of positive products lost 6.9e-3 of a weight's gradient, twice its bf16 rounding, 65536 rows
// 1e-4.  The fp32 sum takes the place of the second accumulator there (5.14 ms at 2^20 x 1600
// x 1600 against 5.05 without it).
#include "luna_linear.cuh"

#include <algorithm>

#include "luna_prof.cuh"
#include "luna_sm100.cuh"

namespace luna {

int tc_sm_count();
bool tc_make_map_nd(CUtensorMap *m, const void *base, int rank, const uint64_t *dims, const uint64_t *strides,
                    const uint32_t *box, int swizzle = 128);

namespace {
using namespace sm100;

constexpr int kEpiWarps = 8, kWarpTma = 8, kWarpMma = 9, kTcThreads = 320;
constexpr int kDepth = 64;  // K of a stage

template <typename IO, int CG, int BN, bool LONG = false> struct Tile {
    static constexpr bool PLANES = sizeof(IO) == 4;   // fp32 operands in three bf16 planes
    static constexpr bool JOIN = PLANES || LONG;      // accumulators joined in an fp32 sum
    static constexpr int BM = 128;                    // rows of a CTA
    static constexpr int NB = BN / CG;                // B rows a CTA holds
    static constexpr int NBL = NB < 64 ? 64 : NB;     // ... and loads (an MN-major slice is 64 wide)
    static constexpr uint32_t A_BYTES = BM * 128, B_BYTES = NBL * 128, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = (int)((192 * 1024) / STAGE) > 8 ? 8 : (int)((192 * 1024) / STAGE);
    static constexpr int ACCS = LONG ? 1 : 2;         // accumulators, and after them the fp32 sum
    static constexpr uint32_t COLS = PLANES ? 4 * BN : 2 * BN;
    static constexpr uint32_t OUT = kEpiWarps * 4096;   // two 32 x 32 pieces of every epilogue warp
    static constexpr uint32_t SMEM = STAGES * STAGE + OUT + 1024 + 256;
    static_assert(SMEM <= 227 * 1024, "shared memory");
};

struct ProductTc {
    Product p;
    int tiles_m, tiles_n, splits, k_steps, steps_per_split;  // tiles of BM * CG rows, BN columns
    int per;        // 64-deep slices of an operand (of each plane of it)
    int join;       // steps of an accumulator, where they are joined
    int terms;      // of a bf16 operand's values: steps of the first and of the second alternate
    bool swap;      // the product is computed transposed: A = the layer's B (few rows of X)
    bool vec;       // outputs and residual on 16-byte boundaries: the epilogue stores by TMA
};

__device__ __forceinline__ uint8_t *align_1024(uint8_t *p) {
    return p + ((1024u - (smem_u32(p) & 1023u)) & 1023u);
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&v);
}

// Work unit -> tile: runs of eight tile rows are walked column by column, so that the blocks at work
// share slices of A and of B in L2.
__device__ __forceinline__ void unit_tile(const ProductTc &a, int u, int &tm, int &tn, int &split) {
    split = u % a.splits;
    u /= a.splits;
    constexpr int G = 8;
    const int per = G * a.tiles_n, g = u / per, rows = min(G, a.tiles_m - g * G), r = u - g * per;
    tm = g * G + r % rows;
    tn = r / rows;
}

constexpr int kPlanes = 3, kTerms = 6;
constexpr int kLong = 65536, kJoin = 16384;  // K of a bf16 sum from which it is joined, and every how many

// 32 columns of a lane's row (`cols` of them inside the output) into the warp's pieces (64-byte rows,
// swizzled) and on to the output's rows row0 .. row0 + 31; there are two pieces.
template <typename IO>
__device__ __forceinline__ void store_piece(uint8_t *pieces, int &stored, const CUtensorMap *map, int64_t col, int64_t row0,
                                            int cols, const float (&v)[32], int lane) {
    constexpr int N = 64 / sizeof(IO);  // columns of a piece
#pragma unroll
    for (int h = 0; h < 32 / N; ++h) {
        if (h * N >= cols) break;
        uint8_t *piece = pieces + (stored++ & 1) * 2048;
        if (lane == 0) bulk_wait_read_but_one();
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint4 w;
            if (sizeof(IO) == 2)
                w = make_uint4(pack2(v[8 * q], v[8 * q + 1]), pack2(v[8 * q + 2], v[8 * q + 3]),
                               pack2(v[8 * q + 4], v[8 * q + 5]), pack2(v[8 * q + 6], v[8 * q + 7]));
            else
                w = make_uint4(__float_as_uint(v[(h * N + 4 * q) % 32]), __float_as_uint(v[(h * N + 4 * q + 1) % 32]),
                               __float_as_uint(v[(h * N + 4 * q + 2) % 32]), __float_as_uint(v[(h * N + 4 * q + 3) % 32]));
            *reinterpret_cast<uint4 *>(piece + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) = w;
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            tma_store_2d(map, piece, (int)((col + h * N) * (sizeof(IO) / 2)), (int)row0);  // (the map counts 2 bytes)
            bulk_commit();
        }
    }
}

// v += 32 values on a 16-byte boundary
template <typename IO>
__device__ __forceinline__ void add32(float (&v)[32], const IO *p) {
#pragma unroll
    for (int h = 0; h < 32; h += 64 / sizeof(IO)) {  // 64 bytes at a time
        uint4 w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = reinterpret_cast<const uint4 *>(p + h)[q];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t x[4] = {w[q].x, w[q].y, w[q].z, w[q].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (sizeof(IO) == 2) {
                    v[(8 * q + 2 * i) % 32] += __uint_as_float(x[i] << 16);
                    v[(8 * q + 2 * i + 1) % 32] += __uint_as_float(x[i] & 0xffff0000u);
                } else {
                    v[(h + 4 * q + i) % 32] += __uint_as_float(x[i]);
                }
            }
        }
    }
}

// Element (r, c) of a warp's 4096 bytes as a piece of 32 x 32.
template <typename IO>
__device__ __forceinline__ IO *piece_at(uint8_t *piece, int r, int c) {
    if (sizeof(IO) == 4) return reinterpret_cast<IO *>(piece) + r * 32 + (c ^ r);
    return reinterpret_cast<IO *>(piece + r * 64 + (((c >> 3) ^ ((r >> 1) & 3)) << 4)) + (c & 7);
}

// The same for outputs that TMA cannot write: the piece's rows one after another, a lane for each column.
template <typename IO>
__device__ __forceinline__ void write_piece(uint8_t *piece, IO *out, int64_t ld, int rows, int cols, const float (&v)[32],
                                            int lane) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 32; ++i) io_store(piece_at<IO>(piece, lane, i), v[i]);
    __syncwarp();
    if (lane < cols)
        for (int r = 0; r < rows; ++r) out[r * ld + lane] = *piece_at<IO>(piece, r, lane);
    __syncwarp();
}
template <typename IO>
__device__ __forceinline__ void add_piece(uint8_t *piece, const IO *in, int64_t ld, int rows, int cols, float (&v)[32],
                                          int lane) {
    __syncwarp();
    for (int r = 0; r < rows; ++r)
        if (lane < cols) *piece_at<IO>(piece, r, lane) = in[r * ld + lane];
    __syncwarp();
    if (lane < rows)
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (i < cols) v[i] += io_load(piece_at<IO>(piece, lane, i));
    __syncwarp();
}

template <typename IO, int ACT> __device__ __forceinline__ void act32(float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = linear_act<IO>(v[i], ACT);
}

template <typename IO, int CG, int BN, bool LONG>
__global__ void __launch_bounds__(kTcThreads, 1)
    k_product_tc(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
                 const __grid_constant__ CUtensorMap mapO, const __grid_constant__ CUtensorMap mapZ,
                 const __grid_constant__ ProductTc a) {
    using T = Tile<IO, CG, BN, LONG>;
    constexpr int S = T::STAGES;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sm = align_1024(smem_raw);
    uint8_t *pieces = sm + S * T::STAGE;
    uint64_t *bars = reinterpret_cast<uint64_t *>(pieces + T::OUT);
    uint64_t *full = bars, *empty = bars + S, *tfull = bars + 2 * S, *tempty = tfull + 2;
    uint32_t *tslot = reinterpret_cast<uint32_t *>(tempty + 2);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    clear_status(a.p.clear, a.p.status);
    if (T::PLANES && flagged(a.p)) return;
    if (tid == 0) {
        for (int i = 0; i < S; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(tfull + i, 1); mbar_init(tempty + i, CG * kEpiWarps); }
        fence_mbar_init();
    }
    if (warp == 0) {
        if (CG == 2) { tmem_alloc_pair(tslot, T::COLS); tmem_relinquish_pair(); }
        else { tmem_alloc(tslot, T::COLS); tmem_relinquish(); }
    }
    tc_fence_before();
    if (CG == 2) cluster_sync();
    else __syncthreads();
    tc_fence_after();
    const uint32_t tbase = *tslot;
    const Product &p = a.p;
    const int units = a.tiles_m * a.tiles_n * a.splits;
    const int first = blockIdx.x / CG, stride = gridDim.x / CG;
    bool failed = false;
    auto wait = [&](uint64_t *bar, uint32_t parity) {
        if (!failed && !mbar_wait(bar, parity)) {
            failed = true;
            atomicOr(p.status, 1);
        }
    };

    if (warp == kWarpTma) {
        if (lane == 0) {
            int it = 0;
            for (int u = first; u < units && !failed; u += stride) {
                int tm, tn, sp;
                unit_tile(a, u, tm, tn, sp);
                const int s0 = sp * a.steps_per_split, s1 = min(a.k_steps, s0 + a.steps_per_split);
                const int ra = (tm * CG + (int)rank) * T::BM, rb = tn * BN + (int)rank * T::NB;
                for (int s = s0; s < s1 && !failed; ++s, ++it) {
                    const int st = it % S;
                    wait(empty + st, ((it / S) & 1) ^ 1);
                    if (failed) break;
                    uint8_t *sa = sm + st * T::STAGE, *sb = sa + T::A_BYTES;
                    if (rank == 0) mbar_arrive_expect_tx(full + st, CG * T::STAGE);
                    const uint32_t bar = CG == 2 ? leader_addr(full + st) : 0;
                    auto load = [&](uint8_t *dst, const CUtensorMap *m, int x, int y) {
                        if (CG == 2) tma_load_2d_pair(dst, m, x, y, bar);
                        else tma_load_2d(dst, m, x, y, full + st);
                    };
                    const int second = !T::PLANES && a.terms == 2 ? s & 1 : 0;
                    const int k = (T::PLANES ? s % kPlanes * a.per + s / kPlanes : a.terms == 2 ? s >> 1 : s) * kDepth;
                    const int xa = second * (int)p.A.lo, xb = second * (int)p.B.lo;  // (multiples of 64)
                    if (p.A.kt) {
                        for (int b = 0; b < T::BM / 64; ++b) load(sa + b * 8192, &mapA, xa + ra + 64 * b, k);
                    } else {
                        load(sa, &mapA, xa + k, ra);
                    }
                    if (p.B.kt) {
                        for (int b = 0; b < T::NBL / 64; ++b) load(sb + b * 8192, &mapB, xb + rb + 64 * b, k);
                    } else {
                        load(sb, &mapB, xb + k, rb);
                    }
                }
            }
            // no load may be on its way when the block ends, which one that has given up elsewhere would not wait for
            // (the leader's barriers count the pair's, and the other block waits for it)
            if (rank == 0)
                for (int i = max(0, it - S); i < it; ++i) mbar_wait(full + i % S, (i / S) & 1, kDrainNs);
        }
    } else if (warp == kWarpMma) {
        if (lane == 0 && rank == 0) {
            const uint32_t id = idesc_bf16(CG * T::BM, BN, p.A.kt, p.B.kt);
            const uint32_t lboA = p.A.kt ? 8192 : 16, lboB = p.B.kt ? 8192 : 16;
            const uint32_t stepA = p.A.kt ? 2048 : 32, stepB = p.B.kt ? 2048 : 32;  // bytes of 16 of K
            int it = 0, n = 0;
            for (int u = first; u < units && !failed; u += stride) {
                int tm, tn, sp;
                unit_tile(a, u, tm, tn, sp);
                const int from = sp * a.steps_per_split, to = min(a.k_steps, from + a.steps_per_split);
                auto product = [&](uint32_t d, int sa, int sb, bool fresh) {  // of A in one stage, B in another
                    const uint64_t da = sdesc(smem_u32(sm + sa * T::STAGE), lboA, 1024, kSwizzle128);
                    const uint64_t db = sdesc(smem_u32(sm + sb * T::STAGE) + T::A_BYTES, lboB, 1024, kSwizzle128);
#pragma unroll
                    for (int k = 0; k < kDepth / 16; ++k) {
                        const uint64_t ka = da + ((k * stepA) >> 4), kb = db + ((k * stepB) >> 4);
                        if (CG == 2) mma_bf16_ss_pair(d, ka, kb, id, !fresh || k > 0);
                        else mma_bf16_ss(d, ka, kb, id, !fresh || k > 0);
                    }
                };
                auto release = [&](int st) {
                    if (CG == 2) mma_commit_pair(empty + st);
                    else mma_commit(empty + st);
                };
                // (one accumulator for all of them, for every three planes, or for every `join` steps)
                for (int s = from; s < to && !failed; ++n) {
                    const int acc = n % T::ACCS;
                    wait(tempty + acc, ((n / T::ACCS) & 1) ^ 1);
                    tc_fence_after();
                    const uint32_t d = tbase + acc * BN;
                    if (T::PLANES) {
                        int st[kPlanes];
                        for (int q = 0; q < kPlanes; ++q, ++s, ++it) {
                            st[q] = it % S;
                            wait(full + st[q], (it / S) & 1);
                        }
                        if (failed) break;
                        tc_fence_after();
                        product(d, st[2], st[0], true);
                        product(d, st[1], st[1], false);
                        product(d, st[0], st[2], false);
                        product(d, st[1], st[0], false);
                        product(d, st[0], st[1], false);
                        product(d, st[0], st[0], false);
                        for (int q = 0; q < kPlanes; ++q) release(st[q]);
                    } else {
                        const int end = T::JOIN ? min(to, s + a.join) : to;
                        for (bool fresh = true; s < end; ++s, ++it, fresh = false) {
                            const int st = it % S;
                            wait(full + st, (it / S) & 1);
                            if (failed) break;
                            tc_fence_after();
                            product(d, st, st, fresh);
                            release(st);
                        }
                        if (failed) break;
                    }
                    if (CG == 2) mma_commit_pair(tfull + acc);
                    else mma_commit(tfull + acc);
                }
            }
        }
    } else {
        const int quarter = warp & 3, half = warp >> 2;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tempty_leader[2] = {CG == 2 ? leader_addr(tempty) : 0, CG == 2 ? leader_addr(tempty + 1) : 0};
        int n = 0, stored = 0;
        constexpr int CH = BN / 32;  // chunks of 32 columns, in halves
        const int c0 = half * ((CH + 1) / 2), c1 = half ? CH : (CH + 1) / 2;
        const uint32_t sum = tbase + lane_base + T::ACCS * BN;
        for (int u = first; u < units && !failed; u += stride, ++n) {
            int tm, tn, sp;
            unit_tile(a, u, tm, tn, sp);
            int more = 0;  // accumulators before the last one
            if (T::JOIN) {
                const int steps = min(a.k_steps - sp * a.steps_per_split, a.steps_per_split);
                more = (steps - 1) / a.join;
                for (int i = 0; i < more && !failed; ++i, ++n) {
                    const int acc = n % T::ACCS;
                    wait(tfull + acc, (n / T::ACCS) & 1);
                    if (__any_sync(0xffffffffu, failed)) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = c0; c < c1; ++c) {
                        uint32_t x[32];
                        tmem_ld32(tbase + lane_base + acc * BN + 32 * c, x);
                        if (i) {
                            uint32_t y[32];
                            tmem_ld32(sum + 32 * c, y);
                            tmem_wait_ld();
#pragma unroll
                            for (int j = 0; j < 32; ++j) x[j] = __float_as_uint(__uint_as_float(x[j]) + __uint_as_float(y[j]));
                        } else {
                            tmem_wait_ld();
                        }
                        tmem_st32(sum + 32 * c, x);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if (CG == 2) mbar_arrive_cluster(tempty_leader[acc]);
                        else mbar_arrive(tempty + acc);
                    }
                }
                if (__any_sync(0xffffffffu, failed)) break;
            }
            const int acc = n % T::ACCS;
            wait(tfull + acc, (n / T::ACCS) & 1);
            if (__any_sync(0xffffffffu, failed)) break;
            tc_fence_after();
            const int64_t row = (int64_t)(tm * CG + (int)rank) * T::BM + quarter * 32 + lane;
            const bool last_split_empty = a.steps_per_split * sp >= a.k_steps;
#pragma unroll 1
            for (int c = c0; c < c1; ++c) {
                const int64_t col = (int64_t)tn * BN + 32 * c;
                uint32_t x[32];
                tmem_ld32(tbase + lane_base + acc * BN + 32 * c, x);
                tmem_wait_ld();
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = last_split_empty ? 0.0f : __uint_as_float(x[i]);
                if (T::JOIN && more) {
                    tmem_ld32(sum + 32 * c, x);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] += __uint_as_float(x[i]);
                }
                const int64_t M = a.swap ? p.N : p.M, N = a.swap ? p.M : p.N;  // of the computed product
                const int w = row < M ? (int)max((int64_t)0, min((int64_t)32, N - col)) : 0;
                if (!a.swap && a.splits == 1) {  // the whole warp, for its 32 rows
                    using B = IO;
                    const int64_t row0 = row - lane;
                    if (row0 < M && col < N) {
                        const int rows = (int)min((int64_t)32, M - row0), cols = (int)min((int64_t)32, N - col);
                        uint8_t *piece = pieces + warp * 4096;
                        if (p.bias) {
                            if (a.vec && cols == 32) {
                                add32<B>(v, static_cast<const B *>(p.bias) + col);
                            } else {
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (i < cols) v[i] += io_load(static_cast<const B *>(p.bias) + col + i);
                            }
                        }
                        if (p.Z) {
                            if (a.vec) store_piece<B>(piece, stored, &mapZ, col, row0, cols, v, lane);
                            else write_piece(piece, static_cast<B *>(p.Z) + row0 * p.ldz + col, p.ldz, rows, cols, v, lane);
                        }
                        switch (p.act) {
                            case LUNA_LINEAR_RELU: act32<B, LUNA_LINEAR_RELU>(v); break;
                            case LUNA_LINEAR_GELU: act32<B, LUNA_LINEAR_GELU>(v); break;
                            case LUNA_LINEAR_SILU: act32<B, LUNA_LINEAR_SILU>(v); break;
                            default: break;
                        }
                        if (p.R) {
                            if (!a.vec)
                                add_piece(piece, static_cast<const B *>(p.R) + row0 * p.ldr + col, p.ldr, rows, cols, v, lane);
                            else if (row < M && cols == 32)
                                add32<B>(v, static_cast<const B *>(p.R) + row * p.ldr + col);
                            else if (row < M)
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (i < cols) v[i] += io_load(static_cast<const B *>(p.R) + row * p.ldr + col + i);
                        }
                        if (a.vec) store_piece<B>(piece, stored, &mapO, col, row0, cols, v, lane);
                        else write_piece(piece, static_cast<B *>(p.out) + row0 * p.ldo + col, p.ldo, rows, cols, v, lane);
                    }
                } else if (w == 0) {
                    // nothing of the row in this chunk
                } else if (a.swap) {
                    if (a.splits > 1) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i < w) p.part[((int64_t)sp * p.M + col + i) * p.N + row] = v[i];
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i < w) linear_finish<IO>(p, col + i, row, v[i]);
                    }
                } else {
                    float *o = p.part + ((int64_t)sp * p.M + row) * p.N + col;
                    if (w == 32 && p.N % 4 == 0) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            *reinterpret_cast<float4 *>(o + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i < w) o[i] = v[i];
                    }
                }
                __syncwarp();  // the TMEM load of the next chunk is the whole warp's
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 2) mbar_arrive_cluster(tempty_leader[acc]);
                else mbar_arrive(tempty + acc);
            }
        }
        if (lane == 0) bulk_wait();
    }
    __syncwarp();
    tc_fence_before();
    if (CG == 2) cluster_sync();  // the leader's products read this CTA's slices, its loads signal the leader
    else __syncthreads();
    if (warp == 0) {
        if (CG == 2) tmem_dealloc_pair(tbase, T::COLS);
        else tmem_dealloc(tbase, T::COLS);
    }
}

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Map of an operand whose slices are `rows` rows x 64 deep.  (Where values have a second term, what lies between
// the terms is read too: of rows past the operand's, whose outputs are dropped, or of depths past its, zeros.)
bool operand_map(CUtensorMap *m, const MatView &v, int64_t rows, int64_t K, int slice_rows) {
    const uint64_t dims[2] = {(uint64_t)(v.lo + (v.kt ? rows : K)), (uint64_t)(v.kt ? K : rows)};
    const uint64_t strides[1] = {(uint64_t)v.ld * 2};
    const uint32_t box[2] = {64, (uint32_t)(v.kt ? kDepth : slice_rows)};
    return tc_make_map_nd(m, v.p, 2, dims, strides, box);
}

// (an fp32 output as twice as many columns of 2 bytes)
bool output_map(CUtensorMap *m, const void *p, int64_t ld, int64_t M, int64_t N, int halves) {
    const uint64_t dims[2] = {(uint64_t)(N * halves), (uint64_t)M}, strides[1] = {(uint64_t)ld * 2 * halves};
    const uint32_t box[2] = {32, 32};
    return tc_make_map_nd(m, p, 2, dims, strides, box, 64);
}

// Cycles of a tile's 64-deep step (its products at 8/10 to 9/10 of the tensor rate, measured on large
// products) and of what a block does around its steps, for choosing between tiles.
template <int CG, int BN> constexpr int step_cycles() {
    return CG == 2 ? (BN == 256 ? 560 : 300) : BN == 256 ? 640 : BN == 128 ? 360 : 250;
}
constexpr int kTileCycles = 2500;

struct Choice {
    int splits;
    double steps, cycles;  // cycles of the steps, and with what is around them
};
template <typename IO, int CG, int BN>
Choice cost(const Product &p) {
    const int64_t tiles = ((p.M + 128 * CG - 1) / (128 * CG)) * ((p.N + BN - 1) / BN), steps = (p.K + kDepth - 1) / kDepth * (sizeof(IO) == 4 ? kTerms : 1);
    const int splits = linear_splits(p, tiles * CG, 256);
    const int64_t rounds = (tiles * splits * CG + tc_sm_count() - 1) / tc_sm_count();
    const double run = (double)rounds * ((double)((steps + splits - 1) / splits) * step_cycles<CG, BN>());
    return Choice{splits, run, run + kTileCycles + (splits > 1 ? kTileCycles : 0)};
}

template <typename IO, int CG, int BN, bool LONG = false>
cudaError_t launch(ProductTc a, cudaStream_t s) {
    using T = Tile<IO, CG, BN, LONG>;
    Product &p = a.p;
    const int64_t M = a.swap ? p.N : p.M, N = a.swap ? p.M : p.N;
    if (a.swap) std::swap(p.A, p.B);
    a.tiles_m = (int)cdiv(M, T::BM * CG);
    a.tiles_n = (int)cdiv(N, BN);
    a.per = (int)cdiv(p.K, kDepth);
    a.terms = p.A.lo || p.B.lo ? 2 : 1;
    a.k_steps = a.per * (T::PLANES ? kPlanes : a.terms);
    a.join = T::PLANES ? kPlanes : kJoin / kDepth;
    const int64_t K = T::PLANES ? 3 * (int64_t)a.per * kDepth : p.K;  // of the operands as they are stored
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
    a.splits = linear_splits(p, tiles * CG, 256);
    a.steps_per_split = (int)cdiv(a.k_steps, a.splits);
    if (T::PLANES) a.steps_per_split = (int)cdiv(a.steps_per_split, kPlanes) * kPlanes;
    a.splits = (int)cdiv(a.k_steps, a.steps_per_split);
    CUtensorMap mA, mB, mO, mZ;
    a.vec = a.vec && !a.swap && a.splits == 1;
    if (!operand_map(&mA, p.A, M, K, T::BM) || !operand_map(&mB, p.B, N, K, T::NBL)) return cudaErrorInvalidValue;
    mO = mZ = mA;
    if (a.vec && (!output_map(&mO, p.out, p.ldo, M, N, sizeof(IO) / 2) || (p.Z && !output_map(&mZ, p.Z, p.ldz, M, N, sizeof(IO) / 2))))
        return cudaErrorInvalidValue;
    cudaError_t e = cudaFuncSetAttribute(k_product_tc<IO, CG, BN, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, T::SMEM);
    if (e != cudaSuccess) return e;
    const int sms = tc_sm_count() / CG * CG;
    const int grid = (int)std::min<int64_t>(tiles * a.splits * CG, sms);
    const int splits = a.splits;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = CG;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kTcThreads);
    cfg.dynamicSmemBytes = T::SMEM;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = CG == 2 ? 1 : 0;
    prof_before("product_tc", s);
    e = cudaLaunchKernelEx(&cfg, k_product_tc<IO, CG, BN, LONG>, mA, mB, mO, mZ, a);
    prof_after("product_tc", s);
    if (e != cudaSuccess || (e = cudaGetLastError()) != cudaSuccess || splits == 1) return e;
    return launch_product_finish(p, splits, T::PLANES ? LUNA_F32 : LUNA_BF16, s);
}

}  // namespace

double product_tc_cycles(int64_t M, int64_t N, int64_t K) {
    using B = __nv_bfloat16;
    Product p{};
    p.M = M; p.N = N; p.K = K;
    p.part_bytes = size_t(64) << 20;  // (what the partial products take at most)
    if (M <= 64) {  // transposed, as below
        std::swap(p.M, p.N);
        return cost<B, 1, 64>(p).steps;
    }
    const Choice pair = cost<B, 2, 256>(p), wide = cost<B, 1, 256>(p), half = cost<B, 1, 128>(p);
    return pair.cycles <= wide.cycles && pair.cycles <= half.cycles ? pair.steps : wide.cycles <= half.cycles ? wide.steps : half.steps;
}

cudaError_t launch_product_tc(const Product &p, luna_dtype io, cudaStream_t s) {
    using B = __nv_bfloat16;
    const int unit = io == LUNA_F32 ? 4 : 8;
    ProductTc a;
    a.p = p;
    a.swap = false;
    a.vec = al16(p.out) && al16(p.R) && al16(p.Z) && al16(p.bias) && p.ldo % unit == 0 && (!p.R || p.ldr % unit == 0) &&
            (!p.Z || p.ldz % unit == 0);
    const auto is_long = [&](int splits) { return cdiv(p.K, splits) > kLong; };
    if (p.M <= 64) {  // few rows of X: the weight's rows fill the tile's 128 rows, X's are its columns
        a.swap = true;
        // (an MN-major slice is 64 wide)
        const bool narrow = p.M <= 32 && !p.A.kt;
        if (io == LUNA_F32) return narrow ? launch<float, 1, 32>(a, s) : launch<float, 1, 64>(a, s);
        if (is_long(linear_splits(p, cdiv(p.N, 128), 256))) return launch<B, 1, 64, true>(a, s);
        return narrow ? launch<B, 1, 32>(a, s) : launch<B, 1, 64>(a, s);
    }
    if (io == LUNA_F32)  // (the fp32 sum leaves no room for 256 columns in TMEM)
        return cost<float, 2, 128>(p).cycles <= cost<float, 1, 128>(p).cycles ? launch<float, 2, 128>(a, s)
                                                                             : launch<float, 1, 128>(a, s);
    const Choice pair = cost<B, 2, 256>(p), wide = cost<B, 1, 256>(p), half = cost<B, 1, 128>(p);
    const bool paired = pair.cycles <= wide.cycles && pair.cycles <= half.cycles, widest = wide.cycles <= half.cycles;
    if (is_long(paired ? pair.splits : widest ? wide.splits : half.splits))
        return pair.cycles <= wide.cycles ? launch<B, 2, 256, true>(a, s) : launch<B, 1, 256, true>(a, s);
    if (paired) return launch<B, 2, 256>(a, s);
    return widest ? launch<B, 1, 256>(a, s) : launch<B, 1, 128>(a, s);
}

}  // namespace luna
