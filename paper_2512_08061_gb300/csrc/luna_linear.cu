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

// 128 x 128 tile of A B^T over one piece of K: operands staged in shared memory 16 deep, eight by
// eight sums a thread in fp32, the next step's values loaded while this one's are multiplied.
// Bound by the fp32 FMA rate.
template <typename IO>
__global__ void __launch_bounds__(kThreads) k_product(Product p, int64_t depth, int splits) {
    __shared__ float sA[kK][kT + 4], sB[kK][kT + 4];
    const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    const int64_t row0 = (int64_t)blockIdx.x * kT, col0 = (int64_t)blockIdx.y * kT;
    const int64_t k0 = (int64_t)blockIdx.z * depth, k1 = min(p.K, k0 + depth);
    float acc[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = 0.0f;
    float ra[8], rb[8];
    // element i of a thread: along the contiguous dimension of each operand
    auto place = [&](bool kt, int i, int &r, int &k) {
        const int e = tid + i * kThreads;
        if (kt) { r = e % kT; k = e / kT; } else { k = e % kK; r = e / kK; }
    };
    auto fetch = [&](int64_t kb) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int r, k;
            place(p.A.kt, i, r, k);
            ra[i] = at<IO>(p.A, row0 + r, p.M, kb + k, k1);
            place(p.B.kt, i, r, k);
            rb[i] = at<IO>(p.B, col0 + r, p.N, kb + k, k1);
        }
    };
    fetch(k0);
    for (int64_t kb = k0; kb < k1; kb += kK) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int r, k;
            place(p.A.kt, i, r, k);
            sA[k][r] = ra[i];
            place(p.B.kt, i, r, k);
            sB[k][r] = rb[i];
        }
        __syncthreads();
        if (kb + kK < k1) fetch(kb + kK);
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            float a[8], b[8];
            *reinterpret_cast<float4 *>(a) = *reinterpret_cast<const float4 *>(&sA[k][ty * 4]);
            *reinterpret_cast<float4 *>(a + 4) = *reinterpret_cast<const float4 *>(&sA[k][64 + ty * 4]);
            *reinterpret_cast<float4 *>(b) = *reinterpret_cast<const float4 *>(&sB[k][tx * 4]);
            *reinterpret_cast<float4 *>(b + 4) = *reinterpret_cast<const float4 *>(&sB[k][64 + tx * 4]);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[i][j] = fmaf(a[i], b[j], acc[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t row = row0 + (i < 4 ? ty * 4 + i : 60 + ty * 4 + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t col = col0 + (j < 4 ? tx * 4 + j : 60 + tx * 4 + j);
            if (row >= p.M || col >= p.N) continue;
            if (splits > 1) p.part[((int64_t)blockIdx.z * p.M + row) * p.N + col] = acc[i][j];
            else linear_finish<IO>(p, row, col, acc[i][j]);
        }
    }
}

// Joins the pieces of K in order.
template <typename IO>
__global__ void __launch_bounds__(256) k_product_finish(Product p, int splits) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, MN = p.M * p.N;
    if (i >= MN) return;
    float acc = 0.0f;
#pragma unroll 8
    for (int s = 0; s < splits; ++s) acc += p.part[s * MN + i];
    linear_finish<IO>(p, i / p.N, i % p.N, acc);
}

// dZ = dY act'(Z) (not written where there is no activation) and the column sums of dZ over a
// block's rows, one partial row a block.  32 columns x 8 rows of threads.
template <typename IO>
__global__ void __launch_bounds__(256) k_linear_dz(const IO *dY, int64_t lddy, const IO *Z, int64_t ldz, IO *dZ, int64_t m,
                                                   int n, int act, int64_t rows, float *part) {
    __shared__ float s[8][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
    const int64_t r0 = (int64_t)blockIdx.y * rows, r1 = min(m, r0 + rows);
    float acc = 0.0f;
    if (c < n)
        for (int64_t r = r0 + w; r < r1; r += 8) {
            float d = io_load(dY + r * lddy + c);
            if (act != LUNA_LINEAR_NONE) {
                d *= linear_slope(io_load(Z + r * ldz + c), act);
                io_store(dZ + r * n + c, d);
            }
            acc += d;
        }
    s[w][threadIdx.x & 31] = acc;
    __syncthreads();
    if (part && w == 0 && c < n) {
#pragma unroll
        for (int i = 1; i < 8; ++i) acc += s[i][threadIdx.x & 31];
        part[(int64_t)blockIdx.y * n + c] = acc;
    }
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
    const int splits = linear_splits(p, gx * gy, 512);
    const int64_t depth = std::max<int64_t>(1, cdiv(cdiv(p.K, splits), kK)) * kK;
    const int used = (int)std::max<int64_t>(1, cdiv(p.K, depth));
    LUNA_LAUNCH("product", k_product<IO>, dim3((unsigned)gx, (unsigned)gy, used), kThreads, 0, s, p, depth, used);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || used == 1) return e;
    return launch_product_finish(p, used, IOType<IO>::code, s);
}

constexpr int64_t kDzRows = 256;  // rows of a block of the column sums

template <typename IO>
cudaError_t dz(const void *dY, int64_t lddy, const void *Z, int64_t ldz, void *dZ, int64_t m, int n, int act, float *part,
               void *db, cudaStream_t s) {
    const int parts = (int)cdiv(m, kDzRows);
    LUNA_LAUNCH("linear_dz", k_linear_dz<IO>, dim3((unsigned)cdiv(n, 32), parts), 256, 0, s, static_cast<const IO *>(dY), lddy,
                static_cast<const IO *>(Z), ldz, static_cast<IO *>(dZ), m, n, act, kDzRows, db ? part : nullptr);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !db) return e;
    LUNA_LAUNCH("linear_db", k_linear_db<IO>, (unsigned)cdiv(n, 256), 256, 0, s, part, parts, n, static_cast<IO *>(db));
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
    size_t o_part = 256, o_dz, part_fwd, part_bwd, fwd, bwd;
};

// Partial products: up to 32 pieces of K of a product with few tiles, at most 64 MiB.
size_t part_bytes(int64_t M, int64_t N) { return (size_t)std::min<int64_t>(M * N * 4 * 32, int64_t(64) << 20); }

Plan make_plan(const luna_linear_desc *ld) {
    Plan p;
    const int64_t eb = ld->io == LUNA_F32 ? 4 : 2;
    p.part_fwd = (size_t)align256((int64_t)part_bytes(ld->m, ld->n));
    p.part_bwd = std::max(part_bytes(ld->m, ld->k), part_bytes(ld->n, ld->k));
    p.part_bwd = std::max(p.part_bwd, (size_t)(cdiv(ld->m, kDzRows) * ld->n * 4));  // the bias gradient's
    p.part_bwd = (size_t)align256((int64_t)p.part_bwd);
    p.fwd = p.o_part + p.part_fwd;
    p.o_dz = p.o_part + p.part_bwd;
    p.bwd = p.o_dz + (ld->act == LUNA_LINEAR_NONE ? 0 : (size_t)align256(ld->m * ld->n * eb));
    return p;
}

bool ws_ok(const void *ws) { return ws && (reinterpret_cast<uintptr_t>(ws) & 255) == 0; }

}  // namespace

int linear_splits(const Product &p, int64_t tiles, int64_t least) {
    if (!p.part || tiles >= tc_sm_count()) return 1;
    int64_t s = std::min<int64_t>(tc_sm_count() / tiles, p.K / least);
    s = std::min<int64_t>(s, (int64_t)(p.part_bytes / (sizeof(float) * p.M * p.N)));
    return (int)std::max<int64_t>(1, std::min<int64_t>(s, 32));
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

cudaError_t launch_product(const Product &p, luna_dtype io, cudaStream_t s) {
    return io == LUNA_BF16 && product_tc_ok(p) ? launch_product_tc(p, s) : launch_product_simt(p, io, s);
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
    p.status = reinterpret_cast<int *>(ws);
    if (cudaMemsetAsync(ws, 0, sizeof(int), s) != cudaSuccess) return LUNA_ERR_CUDA;
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
    if (cudaMemsetAsync(ws, 0, sizeof(int), s) != cudaSuccess) return LUNA_ERR_CUDA;
    const int64_t lddy = ld->lddy ? ld->lddy : n, ldz = ld->ldz ? ld->ldz : n;
    cudaError_t e = cudaSuccess;
    if (act || db) {
        void *dZ = ws + pl.o_dz;
        e = ld->io == LUNA_F32 ? dz<float>(dY, lddy, Z, ldz, dZ, m, (int)n, ld->act, part, db, s)
                               : dz<__nv_bfloat16>(dY, lddy, Z, ldz, dZ, m, (int)n, ld->act, part, db, s);
        if (e != cudaSuccess) return LUNA_ERR_CUDA;
    }
    if (k == 0) return LUNA_OK;
    const void *G = act ? ws + pl.o_dz : dY;
    const int64_t ldg = act ? n : lddy, ldx = ld->ldx ? ld->ldx : k, ldw = ld->ldw ? ld->ldw : k;
    Product p;
    memset(&p, 0, sizeof(p));
    p.act = LUNA_LINEAR_NONE;
    p.part = part; p.part_bytes = pl.part_bwd;
    p.status = reinterpret_cast<int *>(ws);
    if (dX) {
        p.A = MatView{G, ldg, false};
        p.B = MatView{W, ldw, true};
        p.M = m; p.N = k; p.K = n;
        p.out = dX; p.ldo = ld->lddx ? ld->lddx : k;
        if ((e = launch_product(p, ld->io, s)) != cudaSuccess) return LUNA_ERR_CUDA;
    }
    if (dW) {
        p.A = MatView{G, ldg, true};
        p.B = MatView{X, ldx, true};
        p.M = n; p.N = k; p.K = m;
        p.out = dW; p.ldo = k;
        if ((e = launch_product(p, ld->io, s)) != cudaSuccess) return LUNA_ERR_CUDA;
    }
    return LUNA_OK;
}

}  // extern "C"
