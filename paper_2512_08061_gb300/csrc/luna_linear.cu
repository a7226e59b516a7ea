// Linear layers: the C ABI, the CUDA-core product for every type and stride, the joining of
// partial products, and the gradient of the activation with the bias gradient's column sums.
#include "luna_linear.cuh"

#include <math.h>
#include <string.h>

#include <algorithm>

#include "luna_prof.cuh"

namespace luna {

int tc_sm_count();

namespace {

constexpr int kT = 128, kK = 16, kThreads = 256;  // tile, depth of a step

// element (row, k) of an operand; rows past `rows` and depths past `k1` read as 0
template <typename IO>
__device__ __forceinline__ float at(const MatView &v, int64_t row, int64_t rows, int64_t k, int64_t k1) {
    if (row >= rows || k >= k1) return 0.0f;
    return io_load(static_cast<const IO *>(v.p) + (v.kt ? k * v.ld + row : row * v.ld + k));
}

// VEC values (16 bytes, or one) as fp32.
template <typename IO, int VEC>
__device__ __forceinline__ void load_vec(const IO *p, float (&v)[VEC]) {
    if (VEC == 1) {
        v[0] = io_load(p);
    } else {
        const uint4 w = *reinterpret_cast<const uint4 *>(p);
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (sizeof(IO) == 4) {
                v[i] = __uint_as_float(x[i]);
            } else {
                v[2 * i % VEC] = __uint_as_float(x[i] << 16);
                v[(2 * i + 1) % VEC] = __uint_as_float(x[i] & 0xffff0000u);
            }
        }
    }
}
template <typename IO, int VEC>
__device__ __forceinline__ void store_vec(IO *p, const float (&v)[VEC]) {
    if (VEC == 1) {
        io_store(p, v[0]);
    } else {
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (sizeof(IO) == 4) {
                x[i] = __float_as_uint(v[i]);
            } else {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i % VEC], v[(2 * i + 1) % VEC]);
                memcpy(&x[i], &b, 4);
            }
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(x[0], x[1], x[2], x[3]);
    }
}

// Four consecutive values as fp32.
template <typename IO>
__device__ __forceinline__ void load_quad(const IO *p, float (&v)[4]) {
    if (sizeof(IO) == 4) {
        const float4 w = *reinterpret_cast<const float4 *>(p);
        v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
    } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(p);
        v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u);
        v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
    }
}

// 128 x 128 tile of A B^T over one piece of K: operands staged in shared memory 16 deep, eight by eight
// sums a thread in fp32, two multiply-adds an instruction, the next step's values loaded while this one's
// are multiplied.  Bound by the fp32 FMA rate (116 us at 5727 x 656 x 576: 37 TFLOP/s).
// QUAD: loads of four values along the contiguous dimension (rows on their boundaries).
template <typename IO, bool QUAD>
__global__ void __launch_bounds__(kThreads, 2) k_product(Product p, int64_t depth, int splits) {
    __shared__ __align__(16) float sA[kK][kT + 4], sB[kK][kT + 4];
    const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    clear_status(p.clear, p.status);
    if (p.flags && !flagged(p)) return;
    const int64_t row0 = (int64_t)blockIdx.x * kT, col0 = (int64_t)blockIdx.y * kT;
    const int64_t k0 = (int64_t)blockIdx.z * depth, k1 = min(p.K, k0 + depth);
    uint64_t acc[8][4];  // pairs of columns
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0;
    float ra[8], rb[8];
    constexpr int W = QUAD ? 4 : 1;  // values of a load
    // load i of a thread, along the contiguous dimension of each operand: its first row and depth in the tile
    auto place = [&](bool kt, int i, int &r, int &k) {
        const int e = tid + i * kThreads;
        if (kt) { r = e % (kT / W) * W; k = e / (kT / W); } else { k = e % (kK / W) * W; r = e / (kK / W); }
    };
    auto fetch_one = [&](const MatView &v, int64_t base, int64_t rows, int64_t kb, float (&out)[8]) {
#pragma unroll
        for (int i = 0; i < 8 / W; ++i) {
            int r, k;
            place(v.kt, i, r, k);
            if (QUAD) {  // (four rows or four depths are in or out together)
                const bool in = base + r < rows && kb + k < k1;
                const IO *q = static_cast<const IO *>(v.p) + (v.kt ? (kb + k) * v.ld + base + r : (base + r) * v.ld + kb + k);
                float x[4] = {0.f, 0.f, 0.f, 0.f};
                if (in) load_quad<IO>(q, x);
#pragma unroll
                for (int j = 0; j < 4; ++j) out[(4 * i + j) % 8] = x[j];
            } else {
                out[i % 8] = at<IO>(v, base + r, rows, kb + k, k1);
            }
        }
    };
    auto put_one = [&](const MatView &v, float (&tile)[kK][kT + 4], const float (&in)[8]) {
#pragma unroll
        for (int i = 0; i < 8 / W; ++i) {
            int r, k;
            place(v.kt, i, r, k);
#pragma unroll
            for (int j = 0; j < W; ++j) tile[k + (v.kt ? 0 : j)][r + (v.kt ? j : 0)] = in[(W * i + j) % 8];
        }
    };
    auto fetch = [&](int64_t kb) {
        fetch_one(p.A, row0, p.M, kb, ra);
        fetch_one(p.B, col0, p.N, kb, rb);
    };
    fetch(k0);
    for (int64_t kb = k0; kb < k1; kb += kK) {
        __syncthreads();
        put_one(p.A, sA, ra);
        put_one(p.B, sB, rb);
        __syncthreads();
        if (kb + kK < k1) fetch(kb + kK);
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            float a[8];
            uint64_t b[4];
            *reinterpret_cast<float4 *>(a) = *reinterpret_cast<const float4 *>(&sA[k][ty * 4]);
            *reinterpret_cast<float4 *>(a + 4) = *reinterpret_cast<const float4 *>(&sA[k][64 + ty * 4]);
            *reinterpret_cast<ulonglong2 *>(b) = *reinterpret_cast<const ulonglong2 *>(&sB[k][tx * 4]);
            *reinterpret_cast<ulonglong2 *>(b + 2) = *reinterpret_cast<const ulonglong2 *>(&sB[k][64 + tx * 4]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint64_t aa;
                asm("mov.b64 %0, {%1, %1};" : "=l"(aa) : "f"(a[i]));
#pragma unroll
                for (int j = 0; j < 4; ++j) asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc[i][j]) : "l"(aa), "l"(b[j]));
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t row = row0 + (i < 4 ? ty * 4 + i : 60 + ty * 4 + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t col = col0 + (j < 4 ? tx * 4 + j : 60 + tx * 4 + j);
            if (row >= p.M || col >= p.N) continue;
            float v[2];
            asm("mov.b64 {%0, %1}, %2;" : "=f"(v[0]), "=f"(v[1]) : "l"(acc[i][j / 2]));
            if (splits > 1) p.part[((int64_t)blockIdx.z * p.M + row) * p.N + col] = v[j % 2];
            else linear_finish<IO>(p, row, col, v[j % 2]);
        }
    }
}

// Joins the pieces of K in order.
template <typename IO>
__global__ void __launch_bounds__(256) k_product_finish(Product p, int splits) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, MN = p.M * p.N;
    if (p.flags && flagged(p)) return;
    if (i >= MN) return;
    float acc = 0.0f;
#pragma unroll 8
    for (int s = 0; s < splits; ++s) acc += p.part[s * MN + i];
    linear_finish<IO>(p, i / p.N, i % p.N, acc);
}

// A few rows of X (eight of them, or the blockIdx.y-th eight) against rows of W, both along k: a warp owns
// RW rows of W and `split` warps share them, each with its part of k; every lane has its sums for all rows
// of X, so W is read once, 16 bytes a lane and RW loads in flight, and X comes from the first-level cache.
// Bound by the bytes of W (17 us for 67 MB of them: 4 TB/s).
template <typename IO, int VEC, int MR>
__global__ void __launch_bounds__(256) k_product_rows(Product p, int split) {
    constexpr int RW = 4;
    __shared__ float part[8][MR * RW];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    clear_status(p.clear, p.status);
    const int64_t row0 = ((int64_t)blockIdx.x * (8 / split) + warp / split) * RW;
    const int64_t units = p.K / VEC;  // (VEC = 1 otherwise)
    const int64_t u0 = units * (warp % split) / split, u1 = units * (warp % split + 1) / split;
    const IO *W = static_cast<const IO *>(p.B.p), *X = static_cast<const IO *>(p.A.p);
    const int64_t m0 = (int64_t)blockIdx.y * MR;
    float acc[MR][RW];
#pragma unroll
    for (int i = 0; i < MR; ++i)
#pragma unroll
        for (int r = 0; r < RW; ++r) acc[i][r] = 0.0f;
    const IO *w[RW];
#pragma unroll
    for (int r = 0; r < RW; ++r) w[r] = W + min(row0 + r, p.N - 1) * p.B.ld;
#pragma unroll 2
    for (int64_t u = u0 + lane; u < u1; u += 32) {
        float wv[RW][VEC];
#pragma unroll
        for (int r = 0; r < RW; ++r) load_vec<IO, VEC>(w[r] + u * VEC, wv[r]);
#pragma unroll
        for (int i = 0; i < MR; ++i) {
            float xv[VEC];
            load_vec<IO, VEC>(X + min(m0 + i, p.M - 1) * p.A.ld + u * VEC, xv);
#pragma unroll
            for (int r = 0; r < RW; ++r)
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[i][r] = fmaf(xv[e], wv[r][e], acc[i][r]);
        }
    }
#pragma unroll
    for (int i = 0; i < MR; ++i)
#pragma unroll
        for (int r = 0; r < RW; ++r) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) acc[i][r] += __shfl_xor_sync(0xffffffffu, acc[i][r], o);
            if (lane == 0) part[warp][i * RW + r] = acc[i][r];
        }
    __syncthreads();
    // one thread an output: group of `split` warps, row of X, row of W
    for (int t = threadIdx.x; t < (8 / split) * MR * RW; t += 256) {
        const int g = t / (MR * RW), j = t % (MR * RW);
        const int64_t row = m0 + j / RW, col = ((int64_t)blockIdx.x * (8 / split) + g) * RW + j % RW;
        float sum = 0.0f;
        for (int k = 0; k < split; ++k) sum += part[g * split + k][j];
        if (row < p.M && col < p.N) linear_finish<IO>(p, row, col, sum);
    }
}

// dZ = dY act'(Z) (not written where there is no activation; rows lddz apart) and the column sums of dZ over a
// block's rows, one partial row a block.  32 column pieces x 8 rows of threads; bound by the bytes.
// TWO: a value's rounding error goes into a second term lo elements on, and the columns between
// are set to 0 (an infinity or a NaN is its first term alone).
template <typename IO, int VEC, bool TWO>
__global__ void __launch_bounds__(256) k_linear_dz(const IO *dY, int64_t lddy, const IO *Z, int64_t ldz, IO *dZ,
                                                   int64_t lddz, int64_t lo, int64_t m, int n, int act, int64_t rows,
                                                   float *part, int *status) {
    __shared__ float s[8][32 * VEC + 1];
    clear_status(1, status);
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = (blockIdx.x * 32 + lane) * VEC;
    const int64_t r0 = (int64_t)blockIdx.y * rows, r1 = min(m, r0 + rows);
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
    if (c < n) {
#pragma unroll 4
        for (int64_t r = r0 + w; r < r1; r += 8) {
            float d[VEC];
            load_vec<IO, VEC>(dY + r * lddy + c, d);
            if (act != LUNA_LINEAR_NONE) {
                float z[VEC];
                load_vec<IO, VEC>(Z + r * ldz + c, z);
#pragma unroll
                for (int e = 0; e < VEC; ++e) d[e] *= linear_slope<IO>(z[e], act);
                store_vec<IO, VEC>(dZ + r * lddz + c, d);
                if (TWO) {
                    float rest[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float first = __bfloat162float(__float2bfloat16_rn(d[e]));
                        rest[e] = fabsf(first) < INFINITY ? d[e] - first : 0.0f;
                    }
                    store_vec<IO, VEC>(dZ + r * lddz + lo + c, rest);
                }
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] += d[e];
        }
    } else if (TWO && c < lo) {
        const float none[VEC] = {};
        for (int64_t r = r0 + w; r < r1; r += 8) store_vec<IO, VEC>(dZ + r * lddz + c, none);
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) s[w][lane * VEC + e] = acc[e];
    __syncthreads();
    if (part)
        for (int t = threadIdx.x; t < 32 * VEC; t += 256) {
            const int col = blockIdx.x * 32 * VEC + t;
            float a = s[0][t];
#pragma unroll
            for (int i = 1; i < 8; ++i) a += s[i][t];
            if (col < n) part[(int64_t)blockIdx.y * n + col] = a;
        }
}

// Rows of `width` bf16 values, `ld` apart, into rows `ldp` (a multiple of 8) apart: 16 bytes a thread.
__global__ void __launch_bounds__(256) k_pad_rows(const __nv_bfloat16 *src, int64_t ld, __nv_bfloat16 *dst, int64_t ldp,
                                                  int64_t rows, int64_t width) {
    const int64_t per = ldp / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * per) return;
    const int64_t r = i / per, c = (i % per) * 8;
    const uint16_t *p = reinterpret_cast<const uint16_t *>(src) + r * ld + c;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t lo = c + 2 * k < width ? p[2 * k] : 0, hi = c + 2 * k + 1 < width ? p[2 * k + 1] : 0;
        w[k] = lo | (hi << 16);
    }
    *reinterpret_cast<uint4 *>(dst + r * ldp + c) = make_uint4(w[0], w[1], w[2], w[3]);
}

// An fp32 operand as three bf16 planes, x = x0 + x1 + x2: each takes the upper eight bits of what the last
// one left, cut off, not rounded (a value near the largest stays finite), and the third takes the rest.
// Rows (of K where the operand is stored k x rows) and columns that only fill up to whole slices are zeros.
// An infinity or a NaN sets the block's flag: its planes' products would be NaN where the product is not.
// Bound by the bytes (18 us for 10.5 million values, 16 bytes each with the planes: 5.8 TB/s over both).
struct Split {
    const float *src;
    int64_t ld, rows, cols;           // as stored
    __nv_bfloat16 *dst;
    int64_t ldp, prow, pcol, plane;   // rows and columns (a multiple of 8) to write, from plane to plane
    bool vec;                         // 16-byte loads
};
__global__ void __launch_bounds__(256) k_split(Split a, Split b, int *flags, int clear, int *status) {
    const Split &v = blockIdx.y ? b : a;
    clear_status(clear, status);
    const uint32_t per = (uint32_t)(v.pcol / 8);
    const int64_t total = v.prow * per;
    int bad = 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = total >> 32 ? i / per : (int64_t)((uint32_t)i / per), c = (i - r * per) * 8;
        float x[8];
        const float *p = v.src + r * v.ld + c;
        if (v.vec && r < v.rows && c + 8 <= v.cols) {
            const float4 lo = reinterpret_cast<const float4 *>(p)[0], hi = reinterpret_cast<const float4 *>(p)[1];
            x[0] = lo.x; x[1] = lo.y; x[2] = lo.z; x[3] = lo.w;
            x[4] = hi.x; x[5] = hi.y; x[6] = hi.z; x[7] = hi.w;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = r < v.rows && c + k < v.cols ? p[k] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) bad |= (__float_as_uint(x[k]) & 0x7f800000u) == 0x7f800000u;
        __nv_bfloat16 *o = v.dst + r * v.ldp + c;
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t lo = __float_as_uint(x[2 * k]) & 0xffff0000u, hi = __float_as_uint(x[2 * k + 1]) & 0xffff0000u;
                w[k] = lo >> 16 | hi;
                x[2 * k] -= __uint_as_float(lo);
                x[2 * k + 1] -= __uint_as_float(hi);
            }
            *reinterpret_cast<uint4 *>(o + q * v.plane) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) flags[blockIdx.y * kFlagBlocks + blockIdx.x] = bad;
}

template <typename IO>
__global__ void __launch_bounds__(256) k_linear_db(const float *part, int parts, int n, IO *db) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= n) return;
    float acc = 0.0f;
#pragma unroll 8
    for (int i = 0; i < parts; ++i) acc += part[(int64_t)i * n + c];
    io_store(db + c, acc);
}

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
luna_status cuda_status(cudaError_t e) { return e == cudaSuccess ? LUNA_OK : LUNA_ERR_CUDA; }

template <typename IO>
cudaError_t simt(const Product &p, cudaStream_t s) {
    const int64_t gx = cdiv(p.M, kT), gy = cdiv(p.N, kT);
    const int splits = p.flags ? 1 : linear_splits(p, gx * gy, 64);  // (a step of 16 takes about a microsecond when alone)
    const int64_t depth = std::max<int64_t>(1, cdiv(cdiv(p.K, splits), kK)) * kK;
    const int used = (int)std::max<int64_t>(1, cdiv(p.K, depth));
    auto quad = [](const MatView &v, int64_t rows, int64_t K) {
        return reinterpret_cast<uintptr_t>(v.p) % (4 * sizeof(IO)) == 0 && v.ld % 4 == 0 && (v.kt ? rows : K) % 4 == 0;
    };
    const dim3 grid((unsigned)gx, (unsigned)gy, used);
    if (quad(p.A, p.M, p.K) && quad(p.B, p.N, p.K))
        LUNA_LAUNCH("product", (k_product<IO, true>), grid, kThreads, 0, s, p, depth, used);
    else
        LUNA_LAUNCH("product", (k_product<IO, false>), grid, kThreads, 0, s, p, depth, used);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || used == 1) return e;
    return launch_product_finish(p, used, IOType<IO>::code, s);
}

constexpr int64_t kDzRows = 256;  // rows of a block of the column sums

bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename IO, int VEC>
void dz_launch(const void *dY, int64_t lddy, const void *Z, int64_t ldz, void *dZ, int64_t lddz, int64_t lo, int64_t m, int n,
               int act, float *part, int parts, int *status, cudaStream_t s) {
    const dim3 grid((unsigned)cdiv(std::max<int64_t>(n, lo), 32 * VEC), parts);
    if constexpr (sizeof(IO) == 2)
        if (lo) {
            LUNA_LAUNCH("linear_dz", (k_linear_dz<IO, VEC, true>), grid, 256, 0, s, static_cast<const IO *>(dY), lddy,
                        static_cast<const IO *>(Z), ldz, static_cast<IO *>(dZ), lddz, lo, m, n, act, kDzRows, part, status);
            return;
        }
    LUNA_LAUNCH("linear_dz", (k_linear_dz<IO, VEC, false>), grid, 256, 0, s, static_cast<const IO *>(dY), lddy,
                static_cast<const IO *>(Z), ldz, static_cast<IO *>(dZ), lddz, lo, m, n, act, kDzRows, part, status);
}

template <typename IO>
cudaError_t dz(const void *dY, int64_t lddy, const void *Z, int64_t ldz, void *dZ, int64_t lddz, int64_t lo, int64_t m, int n,
               int act, float *part, void *db, int *status, cudaStream_t s) {
    constexpr int VEC = 16 / (int)sizeof(IO);
    const int parts = (int)cdiv(m, kDzRows);
    const bool a = act != LUNA_LINEAR_NONE;
    if (n % VEC == 0 && al16(dY) && lddy % VEC == 0 && (!a || (al16(Z) && ldz % VEC == 0)))
        dz_launch<IO, VEC>(dY, lddy, Z, ldz, dZ, lddz, lo, m, n, act, db ? part : nullptr, parts, status, s);
    else
        dz_launch<IO, 1>(dY, lddy, Z, ldz, dZ, lddz, lo, m, n, act, db ? part : nullptr, parts, status, s);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !db) return e;
    LUNA_LAUNCH("linear_db", k_linear_db<IO>, (unsigned)cdiv(n, 256), 256, 0, s, part, parts, n, static_cast<IO *>(db));
    return cudaGetLastError();
}

template <typename IO, int VEC>
cudaError_t rows_launch(const Product &p, cudaStream_t s) {
    // warps that share four rows of W: as many as keep some 2000 warps at work, with 16 loads each at least
    int split = 1;
    while (split < 8 && cdiv(p.N, 4) * split < 2000 && p.K / VEC / (split * 2) >= 128) split *= 2;
    const dim3 grid((unsigned)cdiv(cdiv(p.N, 4) * split, 8), (unsigned)cdiv(p.M, 8));
    if (p.M == 1) LUNA_LAUNCH("product_rows", (k_product_rows<IO, VEC, 1>), grid, 256, 0, s, p, split);
    else if (p.M == 2) LUNA_LAUNCH("product_rows", (k_product_rows<IO, VEC, 2>), grid, 256, 0, s, p, split);
    else if (p.M <= 4) LUNA_LAUNCH("product_rows", (k_product_rows<IO, VEC, 4>), grid, 256, 0, s, p, split);
    else LUNA_LAUNCH("product_rows", (k_product_rows<IO, VEC, 8>), grid, 256, 0, s, p, split);
    return cudaGetLastError();
}

luna_status check(const luna_linear_desc *ld) {
    if (!ld) return LUNA_ERR_INVALID_ARG;
    if (ld->m < 0 || ld->n < 0 || ld->k < 0) return LUNA_ERR_INVALID_ARG;
    if (ld->act < LUNA_LINEAR_NONE || ld->act > LUNA_LINEAR_SILU) return LUNA_ERR_INVALID_ARG;
    if (ld->io != LUNA_F32 && ld->io != LUNA_BF16) return LUNA_ERR_INVALID_ARG;
    const struct { int64_t ld; int width; } w[] = {{ld->ldx, ld->k}, {ld->ldw, ld->k}, {ld->ldy, ld->n}, {ld->ldr, ld->n},
                                                   {ld->ldz, ld->n}, {ld->lddy, ld->n}, {ld->lddx, ld->k}};
    for (const auto &x : w)
        if (x.ld != 0 && x.ld < x.width) return LUNA_ERR_INVALID_ARG;
    if (ld->m > (1 << 23) || ld->n > (1 << 20) || ld->k > (1 << 20)) return LUNA_ERR_UNSUPPORTED;
    return LUNA_OK;
}

struct Plan {
    size_t o_part = 256, o_dz, o_pad_fwd, o_pad_bwd, pad_fwd = 0, pad_bwd = 0, part_fwd, part_bwd, fwd, bwd;
};

int64_t up8(int64_t x) { return (x + 7) / 8 * 8; }
constexpr double kTwoTermCycles = 2000;
constexpr int64_t kTwoTermRows = 64;

int64_t up64(int64_t x) { return (x + 63) / 64 * 64; }

// bf16 layers: whether dZ goes to its products in two bf16 terms (2^-17 of it) instead of one.  One rounding of
// dZ adds to each gradient as much as the gradient's own (sqrt 2 of it in all, and more where few values have to
// average it out); two terms take that away for twice the products' steps, and are taken where the launches nearly
// hide them: to 64 rows and 2000 cycles of steps that costs 0.8 to 2.3 us of 15 to 25 (20 x 16 x 4096 22.8 -> 23.6 us,
// 2 x 3680 x 128 16.2 -> 17.9, 64 x 512 x 512 18.9 -> 21.2), beyond them 3.5 to 12 (128^3 19.7 -> 23.2, 2048 x 64 x 64
// 28.9 -> 34.3, 4 x 4096 x 4096 32.0 -> 36.9, 2048 x 1024 x 1024 49.0 -> 60.5).
bool two_terms(const luna_linear_desc *ld) {
    return ld->io == LUNA_BF16 && ld->act != LUNA_LINEAR_NONE && ld->m > 0 && ld->m <= kTwoTermRows && ld->n > 0 && ld->k > 0 &&
           product_tc_cycles(ld->m, ld->k, ld->n) + product_tc_cycles(ld->n, ld->k, ld->m) <= kTwoTermCycles;
}
// Bytes of a row of dZ.
int64_t dz_row(const luna_linear_desc *ld) { return two_terms(ld) ? 4 * up64(ld->n) : up8(ld->n) * (ld->io == LUNA_F32 ? 4 : 2); }

// Pieces of K of a product of M x N x K on a launch of `tiles` blocks: enough to give every SM a block, none
// under `least` of K, at most 32, and at most 64 MiB of partial products.
int pieces(int64_t M, int64_t N, int64_t K, int64_t tiles, int64_t least) {
    if (tiles >= tc_sm_count()) return 1;
    int64_t s = std::min<int64_t>(tc_sm_count() / tiles, K / least);
    s = std::min<int64_t>(s, (int64_t(64) << 20) / (4 * M * N));
    return (int)std::max<int64_t>(1, std::min<int64_t>(s, 32));
}

// Room for the partial products of the kernels that may take a product (`rows`: the one for a few rows takes it
// whole): every tile shape on tensor cores, and the CUDA cores' for operands off their boundaries.
size_t part_bytes(int64_t M, int64_t N, int64_t K, bool rows) {
    if (M == 0 || N == 0 || rows) return 0;
    int most = pieces(M, N, K, cdiv(M, kT) * cdiv(N, kT), 64);
    if (M <= 64) {
        most = std::max(most, pieces(M, N, K, cdiv(N, 128), 256));
    } else {
        for (const int64_t tiles : {2 * cdiv(M, 256) * cdiv(N, 256), cdiv(M, 128) * cdiv(N, 256), 2 * cdiv(M, 256) * cdiv(N, 128)})
            most = std::max(most, pieces(M, N, K, tiles, 256));
    }
    return most > 1 ? (size_t)(M * N * 4 * most) : 0;
}

// Whether an fp32 product is taken to tensor cores in bf16 planes: estimated microseconds of both ways.  The
// CUDA cores carry 35 TFLOP/s in whole tiles; the planes take three launches, 16 bytes a value of the operands
// and six products at 1 PFLOP/s.
bool planes_pay(int64_t M, int64_t N, int64_t K) {
    const double macs = (double)M * N * K;
    const double simt = 2.0 * (double)(cdiv(M, kT) * kT) * (double)(cdiv(N, kT) * kT) * K / 35e6;
    return M > 8 && K > 0 && simt > 12.0 + 12.0 * macs / 1e9 + 16.0 * (double)(M + N) * K / 4e6;
}
// Rows of X that go to the kernel for a few rows, eight at a time in fp32.
constexpr int kRows = 8, kRowsF32 = 32;
// Bytes of the planes of an operand of `rows` rows.
int64_t plane_bytes(int64_t rows, int64_t K, bool kt) { return align256(3 * up64(K) * (kt ? up8(rows) : rows) * 2); }
constexpr int64_t kFlagBytes = 2 * kFlagBlocks * sizeof(int) / 256 * 256 + 256;
int64_t planes_room(int64_t M, int64_t N, int64_t K, bool akt, bool bkt) {
    return planes_pay(M, N, K) ? kFlagBytes + plane_bytes(M, K, akt) + plane_bytes(N, K, bkt) : 0;
}

Plan make_plan(const luna_linear_desc *ld) {
    Plan p;
    const bool few = ld->k > 0 && ld->m <= (ld->io == LUNA_F32 ? kRowsF32 : kRows);
    p.part_fwd = (size_t)align256((int64_t)part_bytes(ld->m, ld->n, ld->k, few));
    p.part_bwd = std::max(part_bytes(ld->m, ld->k, ld->n, false), part_bytes(ld->n, ld->k, ld->m, false));
    p.part_bwd = std::max(p.part_bwd, (size_t)(cdiv(ld->m, kDzRows) * ld->n * 4));  // the bias gradient's
    p.part_bwd = (size_t)align256((int64_t)p.part_bwd);
    p.fwd = p.o_part + p.part_fwd;
    p.o_dz = p.o_part + p.part_bwd;
    p.bwd = p.o_dz + (ld->act == LUNA_LINEAR_NONE ? 0 : (size_t)align256(ld->m * dz_row(ld)));
    p.o_pad_fwd = p.fwd;
    p.o_pad_bwd = p.bwd;
    // bf16 widths that are not multiples of 8: copies of the operands whose rows are 16-byte aligned
    if (ld->io == LUNA_BF16 && (ld->n % 8 || ld->k % 8)) {
        const int64_t X = align256(ld->m * up8(ld->k) * 2), W = align256(ld->n * up8(ld->k) * 2);
        p.pad_fwd = ld->k % 8 ? (size_t)(X + W) : 0;
        p.pad_bwd = (size_t)(align256(ld->m * up8(ld->n) * 2) + std::max(X, W));  // dz and one of the others at a time
        p.fwd += p.pad_fwd;
        p.bwd += p.pad_bwd;
    } else if (two_terms(ld)) {  // (the CUDA cores' product, for operands off their boundaries, takes no second term)
        p.pad_bwd = (size_t)align256(std::max(ld->m, (int64_t)ld->n) * up8(ld->k) * 2);
        p.bwd += p.pad_bwd;
    }
    if (ld->io == LUNA_F32) {  // fp32 operands in three bf16 planes
        p.pad_fwd = ld->m <= kRowsF32 ? 0 : (size_t)planes_room(ld->m, ld->n, ld->k, false, false);
        p.pad_bwd = (size_t)std::max(planes_room(ld->m, ld->k, ld->n, false, true), planes_room(ld->n, ld->k, ld->m, true, true));
        p.fwd += p.pad_fwd;
        p.bwd += p.pad_bwd;
    }
    return p;
}

bool ws_ok(const void *ws) { return ws && (reinterpret_cast<uintptr_t>(ws) & 255) == 0; }

}  // namespace

int linear_splits(const Product &p, int64_t tiles, int64_t least) {
    const int64_t room = (int64_t)(p.part_bytes / (sizeof(float) * p.M * p.N));
    return (int)std::max<int64_t>(1, std::min<int64_t>(pieces(p.M, p.N, p.K, tiles, least), room));
}

cudaError_t launch_product_simt(const Product &p, luna_dtype io, cudaStream_t s) {
    return io == LUNA_F32 ? simt<float>(p, s) : simt<__nv_bfloat16>(p, s);
}

cudaError_t launch_product_finish(const Product &p, int splits, luna_dtype io, cudaStream_t s) {
    const unsigned grid = (unsigned)cdiv(p.M * p.N, 256);
    if (io == LUNA_F32)
        LUNA_LAUNCH("product_finish", k_product_finish<float>, grid, 256, 0, s, p, splits);
    else
        LUNA_LAUNCH("product_finish", k_product_finish<__nv_bfloat16>, grid, 256, 0, s, p, splits);
    return cudaGetLastError();
}

// Copies what TMA cannot read of p's operands into p.pad and points p at the copies; false if there is no
// room (an operand whose width would do, but whose address or leading dimension does not).
static bool pad_operands(Product &p, cudaStream_t s, cudaError_t *err) {
    size_t used = 0;
    *err = cudaSuccess;
    for (int i = 0; i < 2; ++i) {
        MatView &v = i ? p.B : p.A;
        if (al16(v.p) && v.ld % 8 == 0) continue;
        const int64_t width = v.kt ? (i ? p.N : p.M) : p.K, rows = v.kt ? p.K : (i ? p.N : p.M), ldp = up8(width);
        const size_t bytes = (size_t)align256(rows * ldp * 2);
        if (!p.pad || used + bytes > p.pad_bytes) return false;
        __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(static_cast<char *>(p.pad) + used);
        used += bytes;
        LUNA_LAUNCH("pad_rows", k_pad_rows, (unsigned)cdiv(rows * (ldp / 8), 256), 256, 0, s,
                    static_cast<const __nv_bfloat16 *>(v.p), v.ld, dst, ldp, rows, width);
        if ((*err = cudaGetLastError()) != cudaSuccess) return false;
        v.p = dst;
        v.ld = ldp;
    }
    return true;
}

// The operands of p into three planes each in p.pad; p then points at them.
static cudaError_t split_operands(Product &p, cudaStream_t s) {
    int *flags = static_cast<int *>(p.pad);
    char *to = static_cast<char *>(p.pad) + kFlagBytes;
    Split sp[2];
    for (int i = 0; i < 2; ++i) {
        MatView &v = i ? p.B : p.A;
        Split &q = sp[i];
        const int64_t rows = i ? p.N : p.M, Kp = up64(p.K);
        q.src = static_cast<const float *>(v.p);
        q.ld = v.ld;
        q.rows = v.kt ? p.K : rows;
        q.cols = v.kt ? rows : p.K;
        q.dst = reinterpret_cast<__nv_bfloat16 *>(to);
        q.prow = v.kt ? Kp : rows;
        q.pcol = v.kt ? up8(rows) : Kp;
        q.ldp = v.kt ? q.pcol : 3 * Kp;
        q.plane = v.kt ? Kp * q.ldp : Kp;
        q.vec = al16(v.p) && v.ld % 4 == 0;
        to += plane_bytes(rows, p.K, v.kt);
        v.p = q.dst;
        v.ld = q.ldp;
    }
    LUNA_LAUNCH("split", k_split, dim3(kFlagBlocks, 2), 256, 0, s, sp[0], sp[1], flags, p.clear, p.status);
    p.clear = 0;
    p.flags = flags;
    p.n_flags = 2 * kFlagBlocks;
    return cudaGetLastError();
}

bool product_rows_ok(const Product &p, luna_dtype io) {
    return p.M <= (io == LUNA_F32 ? kRowsF32 : kRows) && p.K > 0 && !p.A.kt && !p.B.kt;
}

cudaError_t launch_product_rows(const Product &p, luna_dtype io, cudaStream_t s) {
    const int vec = io == LUNA_F32 ? 4 : 8;
    const bool v = p.K % vec == 0 && al16(p.A.p) && al16(p.B.p) && p.A.ld % vec == 0 && p.B.ld % vec == 0;
    if (io == LUNA_F32) return v ? rows_launch<float, 4>(p, s) : rows_launch<float, 1>(p, s);
    return v ? rows_launch<__nv_bfloat16, 8>(p, s) : rows_launch<__nv_bfloat16, 1>(p, s);
}

// Up to eight rows of X the product is a read of W (at m = 8, n = 8192, k = 4096 the fp32 sums take about
// as long as the bytes); beyond that tensor cores take bf16, if need be from aligned copies of the operands
// (which cost their bytes twice over; the CUDA-core product would take ten to thirty times the tensor cores').
cudaError_t launch_product(const Product &p, luna_dtype io, cudaStream_t s) {
    if (product_rows_ok(p, io)) return launch_product_rows(p, io, s);
    if (io == LUNA_BF16 && p.K >= 1) {
        Product q = p;
        cudaError_t e;
        if (pad_operands(q, s, &e)) return launch_product_tc(q, io, s);
        if (e != cudaSuccess) return e;
        if (p.A.lo) return cudaErrorInvalidValue;  // (has its copies always)
    }
    if (io == LUNA_F32 && planes_pay(p.M, p.N, p.K) &&
        p.pad_bytes >= (size_t)planes_room(p.M, p.N, p.K, p.A.kt, p.B.kt)) {
        Product q = p;
        cudaError_t e = split_operands(q, s);
        if (e == cudaSuccess) e = launch_product_tc(q, io, s);
        if (e != cudaSuccess) return e;
        Product r = p;  // takes the product if an operand holds an infinity or a NaN
        r.clear = 0;
        r.flags = q.flags;
        r.n_flags = q.n_flags;
        return launch_product_simt(r, io, s);
    }
    return launch_product_simt(p, io, s);
}

}  // namespace luna

using namespace luna;

extern "C" {

luna_status luna_linear_workspace_size(const luna_linear_desc *ld, int backward, size_t *bytes) {
    if (!bytes) return LUNA_ERR_INVALID_ARG;
    const luna_status st = check(ld);
    if (st != LUNA_OK) return st;
    const Plan p = make_plan(ld);
    *bytes = backward ? p.bwd : p.fwd;
    return LUNA_OK;
}

luna_status luna_linear_fwd(const luna_linear_desc *ld, const void *X, const void *W, const void *bias, const void *R,
                            void *Y, void *Z, void *workspace, size_t ws_bytes, void *stream) {
    const luna_status st = check(ld);
    if (st != LUNA_OK) return st;
    if (ld->m == 0 || ld->n == 0) return LUNA_OK;
    if ((ld->k > 0 && (!X || !W)) || !Y || !ws_ok(workspace)) return LUNA_ERR_INVALID_ARG;
    const Plan pl = make_plan(ld);
    if (ws_bytes < pl.fwd) return LUNA_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char *ws = static_cast<char *>(workspace);
    Product p;
    memset(&p, 0, sizeof(p));
    p.A = MatView{X, ld->ldx ? ld->ldx : ld->k, false};
    p.B = MatView{W, ld->ldw ? ld->ldw : ld->k, false};
    p.M = ld->m; p.N = ld->n; p.K = ld->k;
    p.bias = bias; p.act = ld->act; p.R = R; p.Z = Z; p.out = Y;
    p.ldr = ld->ldr ? ld->ldr : ld->n; p.ldz = ld->ldz ? ld->ldz : ld->n; p.ldo = ld->ldy ? ld->ldy : ld->n;
    p.part = reinterpret_cast<float *>(ws + pl.o_part); p.part_bytes = pl.part_fwd;
    p.pad = pl.pad_fwd ? ws + pl.o_pad_fwd : nullptr; p.pad_bytes = pl.pad_fwd;
    p.status = reinterpret_cast<int *>(ws);
    p.clear = 1;
    return cuda_status(launch_product(p, ld->io, s));
}

luna_status luna_linear_bwd(const luna_linear_desc *ld, const void *X, const void *W, const void *Z, const void *dY,
                            void *dX, void *dW, void *db, void *workspace, size_t ws_bytes, void *stream) {
    const luna_status st = check(ld);
    if (st != LUNA_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int64_t m = ld->m, n = ld->n, k = ld->k, eb = ld->io == LUNA_F32 ? 4 : 2;
    if (n == 0 && (m == 0 || k == 0)) return LUNA_OK;
    if (m == 0 || n == 0 || k == 0) {  // sums over nothing
        if (m == 0 && dW && k > 0 && cudaMemsetAsync(dW, 0, n * k * eb, s) != cudaSuccess) return LUNA_ERR_CUDA;
        if (n == 0 && dX && cudaMemset2DAsync(dX, (ld->lddx ? ld->lddx : k) * eb, 0, k * eb, m, s) != cudaSuccess)
            return LUNA_ERR_CUDA;
        if (m == 0 && db && cudaMemsetAsync(db, 0, n * eb, s) != cudaSuccess) return LUNA_ERR_CUDA;
        if (!(k == 0 && m > 0 && n > 0 && db)) return LUNA_OK;
    }
    const bool act = ld->act != LUNA_LINEAR_NONE;
    if (!dY || (act && !Z) || (dX && k > 0 && !W) || (dW && k > 0 && !X) || !ws_ok(workspace)) return LUNA_ERR_INVALID_ARG;
    const Plan pl = make_plan(ld);
    if (ws_bytes < pl.bwd) return LUNA_ERR_WORKSPACE;
    char *ws = static_cast<char *>(workspace);
    float *part = reinterpret_cast<float *>(ws + pl.o_part);
    int *status = reinterpret_cast<int *>(ws);
    const int64_t lddy = ld->lddy ? ld->lddy : n, ldz = ld->ldz ? ld->ldz : n;
    cudaError_t e = cudaSuccess;
    const int64_t lo = act && two_terms(ld) ? up64(n) : 0, ldg = act ? dz_row(ld) / eb : lddy;
    if (act || db) {
        void *dZ = ws + pl.o_dz;
        e = ld->io == LUNA_F32 ? dz<float>(dY, lddy, Z, ldz, dZ, ldg, lo, m, (int)n, ld->act, part, db, status, s)
                               : dz<__nv_bfloat16>(dY, lddy, Z, ldz, dZ, ldg, lo, m, (int)n, ld->act, part, db, status, s);
        if (e != cudaSuccess) return LUNA_ERR_CUDA;
    }
    if (k == 0) return LUNA_OK;
    const void *G = act ? ws + pl.o_dz : dY;
    const int64_t ldx = ld->ldx ? ld->ldx : k, ldw = ld->ldw ? ld->ldw : k;
    Product p;
    memset(&p, 0, sizeof(p));
    p.act = LUNA_LINEAR_NONE;
    p.part = part; p.part_bytes = pl.part_bwd;
    p.pad = pl.pad_bwd ? ws + pl.o_pad_bwd : nullptr; p.pad_bytes = pl.pad_bwd;
    p.status = status;
    p.clear = !(act || db);
    if (dX) {
        p.A = MatView{G, ldg, false, lo};
        p.B = MatView{W, ldw, true};
        p.M = m; p.N = k; p.K = n;
        p.out = dX; p.ldo = ld->lddx ? ld->lddx : k;
        if ((e = launch_product(p, ld->io, s)) != cudaSuccess) return LUNA_ERR_CUDA;
        p.clear = 0;
    }
    if (dW) {
        p.A = MatView{G, ldg, true, lo};
        p.B = MatView{X, ldx, true};
        p.M = n; p.N = k; p.K = m;
        p.out = dW; p.ldo = k;
        if ((e = launch_product(p, ld->io, s)) != cudaSuccess) return LUNA_ERR_CUDA;
    }
    return LUNA_OK;
}

}  // extern "C"
