// Linear attention with a decay for each head on CUDA cores in fp32: the form for
// every type, width and stride (the tensor-core form covers bf16 at aligned
// widths), the scan of the pieces' states, the sum over grouped heads, and the
// single-token step.
#include "luna_decay.cuh"
#include "luna_prof.cuh"

namespace luna {
namespace {

constexpr int kCh = 32;        // rows of a chunk
constexpr int kCols = 32;      // columns of c of a block
constexpr int kMixThreads = 256;

template <typename T>
__device__ __forceinline__ const T *row_base(const RowView &v, int b, int h, int H) {
    return static_cast<const T *>(v.p) + b * v.sb + (int64_t)(h / (H / v.heads)) * v.sh;
}

// One block: piece s of head (b, h), columns [32 * blockIdx.y, +32) of c.  The columns of the
// state are independent, so blocks that share a head read a and b again but exchange nothing.
// The state slice (da x 32) stays in shared memory; per chunk of 32 rows
//     P = (a b^T) masked and decayed,  out = p P c + x lambda^{m+e} a X,  X = lambda^{nv} X + u (b w)^T c
// Bound by the shared-memory reads of the three small products (fp32 on CUDA cores).
template <typename IO, typename OUT>
__global__ void __launch_bounds__(kMixThreads) k_decay_mix(DecayMix a) {
    extern __shared__ float sm[];
    clear_status(a);
    const int da = a.da, lda = da + 1;
    float *sa = sm, *sb = sa + kCh * lda, *sc = sb + kCh * lda, *sP = sc + kCh * (kCols + 1);
    float *sX = sP + kCh * (kCh + 1), *pw = sX + da * kCols;
    const int tid = threadIdx.x;
    const int64_t item = blockIdx.x;
    const int seg = (int)(item % a.nseg);
    const int64_t bh = item / a.nseg;
    const int b = (int)(bh / a.H), h = (int)(bh % a.H);
    const int col0 = blockIdx.y * kCols;
    const int e = a.reverse ? 0 : 1;
    const float g = decay_log(a.log_decay, h);
    for (int i = tid; i <= kCh; i += kMixThreads) pw[i] = expf(g * (float)i);
    const int len = head_length(a.lengths, b, a.n);
    const int r0 = seg * a.seg_len, rend = min(a.n, r0 + a.seg_len);
    const int r1 = max(r0, min(len, rend));
    const IO *A = row_base<IO>(a.a, b, h, a.H), *Bm = row_base<IO>(a.b, b, h, a.H), *Cm = row_base<IO>(a.c, b, h, a.H);
    OUT *O = a.out ? static_cast<OUT *>(a.out) + b * a.ob + (int64_t)h * a.oh : nullptr;
    {
        const float *X = a.X ? a.X + (bh * a.x_pieces + (a.x_pieces > 1 ? seg : 0)) * da * a.dc : nullptr;
        for (int i = tid; i < da * kCols; i += kMixThreads) {
            const int f = i / kCols, c = col0 + i % kCols;
            sX[i] = X && c < a.dc ? (a.x_trans ? X[(int64_t)c * da + f] : X[(int64_t)f * a.dc + c]) : 0.0f;
        }
    }
    const int nch = (r1 - r0 + kCh - 1) / kCh;
    for (int ci = 0; ci < nch; ++ci) {
        const int row0 = r0 + (a.reverse ? nch - 1 - ci : ci) * kCh;
        const int nv = min(kCh, r1 - row0);
        __syncthreads();
        for (int i = tid; i < kCh * da; i += kMixThreads) {
            const int r = i / da, f = i % da;
            const bool on = r < nv;
            if (O) sa[r * lda + f] = on ? io_load(A + (int64_t)(row0 + r) * a.a.st + f) : 0.0f;
            sb[r * lda + f] = on ? io_load(Bm + (int64_t)(row0 + r) * a.b.st + f) : 0.0f;
        }
        for (int i = tid; i < kCh * kCols; i += kMixThreads) {
            const int r = i / kCols, c = i % kCols;
            sc[r * (kCols + 1) + c] =
                r < nv && col0 + c < a.dc ? io_load(Cm + (int64_t)(row0 + r) * a.c.st + col0 + c) : 0.0f;
        }
        __syncthreads();
        if (O) {
            const int r = tid / 8, j0 = tid % 8;
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
            for (int f = 0; f < da; ++f) {
                const float av = sa[r * lda + f];
#pragma unroll
                for (int t = 0; t < 4; ++t) acc[t] = fmaf(av, sb[(j0 + 8 * t) * lda + f], acc[t]);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int j = j0 + 8 * t, dist = a.reverse ? j - r : r - j;
                sP[r * (kCh + 1) + j] = dist >= 0 ? a.p * acc[t] * pw[dist] : 0.0f;
            }
            __syncthreads();
            float in[4] = {0.f, 0.f, 0.f, 0.f}, ex[4] = {0.f, 0.f, 0.f, 0.f};
            const int c0 = (tid % 8) * 4;
            for (int j = 0; j < nv; ++j) {
                const float pv = sP[r * (kCh + 1) + j];
#pragma unroll
                for (int t = 0; t < 4; ++t) in[t] = fmaf(pv, sc[j * (kCols + 1) + c0 + t], in[t]);
            }
            for (int f = 0; f < da; ++f) {
                const float av = sa[r * lda + f];
#pragma unroll
                for (int t = 0; t < 4; ++t) ex[t] = fmaf(av, sX[f * kCols + c0 + t], ex[t]);
            }
            if (r < nv) {
                const float w = a.x * pw[(a.reverse ? nv - 1 - r : r) + e];
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (col0 + c0 + t < a.dc) io_store(O + (int64_t)(row0 + r) * a.ot + col0 + c0 + t, fmaf(w, ex[t], in[t]));
            }
            __syncthreads();
        }
        const float dec = pw[nv];
        const int c = tid % kCols;
        for (int f = tid / kCols; f < da; f += kMixThreads / kCols) {
            float acc = 0.0f;
            for (int r = 0; r < nv; ++r) {
                const int m = a.reverse ? nv - 1 - r : r;
                acc = fmaf(pw[nv - m - e] * sb[r * lda + f], sc[r * (kCols + 1) + c], acc);
            }
            sX[f * kCols + c] = fmaf(dec, sX[f * kCols + c], a.u * acc);
        }
    }
    __syncthreads();
    if (O) {  // rows at and past the length
        const int w = min(kCols, a.dc - col0);
        for (int64_t i = tid; i < (int64_t)(rend - r1) * w; i += kMixThreads)
            io_store(O + (r1 + i / w) * a.ot + col0 + i % w, 0.0f);
    }
    if (a.Xout) {
        float *X = a.Xout + (bh * a.nseg + seg) * da * a.dc;
        for (int i = tid; i < da * kCols; i += kMixThreads) {
            const int f = i / kCols, cc = col0 + i % kCols;
            if (cc < a.dc) X[(int64_t)f * a.dc + cc] = sX[i];
        }
    }
}

__global__ void __launch_bounds__(256) k_decay_scan(DecayScan a) {
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / a.H), h = (int)(bh % a.H);
    const int64_t i = (int64_t)blockIdx.y * blockDim.x + threadIdx.x;
    if (i >= a.E) return;
    const float g = decay_log(a.log_decay, h);
    const int len = head_length(a.lengths, b, a.n);
    float x = a.init ? a.init[bh * a.E + i] : 0.0f;
    for (int t = 0; t < a.nseg; ++t) {
        const int s = a.reverse ? a.nseg - 1 - t : t;
        const int r0 = s * a.seg_len, rows = min(len, r0 + a.seg_len) - r0;
        if (a.X) a.X[(bh * a.nseg + s) * a.E + i] = x;
        if (rows > 0) x = fmaf(expf(g * (float)rows), x, a.U[(bh * a.nseg + s) * a.E + i]);
    }
    if (a.last) a.last[bh * a.E + i] = x;
}

template <typename IO>
__global__ void __launch_bounds__(256) k_decay_group_sum(const float *src, int H, int G, int n, int width, IO *dst,
                                                         int64_t sb, int64_t sh, int64_t st, int64_t total) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= total) return;
    const int w = (int)(i % width);
    const int64_t row = i / width;
    const int t = (int)(row % n);
    const int64_t bk = row / n;
    const int Hk = H / G, b = (int)(bk / Hk), hk = (int)(bk % Hk);
    const float *p = src + (((int64_t)b * H + (int64_t)hk * G) * n + t) * width + w;
    float acc = 0.0f;
    for (int j = 0; j < G; ++j) acc += p[(int64_t)j * n * width];
    io_store(dst + b * sb + (int64_t)hk * sh + (int64_t)t * st + w, acc);
}

// ---------------------------------------------------------------------------
// One token: S <- lambda S + k v^T, o = scale q^T S.  A block owns 32 columns of one
// head's state: 8 lanes x 16 bytes cover a row's 128 bytes, four rows a warp, 32 rows a
// block at a time, every load of a thread in flight before the first is used.  The state is
// read and written once, which bounds the step; the column split keeps one sequence's 32
// heads on 128 blocks.

constexpr int kStepThreads = 256;

template <typename IO, bool VEC>
__global__ void __launch_bounds__(kStepThreads) k_decay_step(DecayStep a) {
    __shared__ float sq[kMaxD], sk[kMaxD];
    __shared__ float so[kStepThreads / 32][kCols];
    const int tid = threadIdx.x;
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / a.H), h = (int)(bh % a.H), hk = h / (a.H / a.Hkv);
    const int col0 = blockIdx.y * kCols;
    const int slot = a.slots ? a.slots[b] : b;
    IO *o = static_cast<IO *>(a.o) + b * a.ob + h * a.oh;
    const bool live = slot >= 0 && slot < a.nslots;
    if (!live) {
        if (tid < kCols && col0 + tid < a.dv) io_store(o + col0 + tid, 0.0f);
        return;
    }
    const IO *q = static_cast<const IO *>(a.q) + b * a.qb + h * a.qh;
    const IO *k = static_cast<const IO *>(a.k) + b * a.kb + hk * a.kh;
    const IO *v = static_cast<const IO *>(a.v) + b * a.vb + hk * a.vh;
    float *S = a.S + ((int64_t)slot * a.H + h) * a.d * a.dv;
    const int cg = tid % 8, rg = tid / 8;  // column group of four, row
    const int c = col0 + 4 * cg;
    constexpr int R = kMaxD / (kStepThreads / 8);
    float4 s[R];
    float vc[4];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int f = rg + i * (kStepThreads / 8);
        s[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (f < a.d) {
            const float *p = S + (int64_t)f * a.dv + c;
            if (VEC) {
                if (c < a.dv) s[i] = *reinterpret_cast<const float4 *>(p);
            } else {
                if (c < a.dv) s[i].x = p[0];
                if (c + 1 < a.dv) s[i].y = p[1];
                if (c + 2 < a.dv) s[i].z = p[2];
                if (c + 3 < a.dv) s[i].w = p[3];
            }
        }
    }
    for (int i = tid; i < a.d; i += kStepThreads) { sq[i] = io_load(q + i); sk[i] = io_load(k + i); }
#pragma unroll
    for (int t = 0; t < 4; ++t) vc[t] = c + t < a.dv ? io_load(v + c + t) : 0.0f;
    const float lam = expf(decay_log(a.log_decay, h));
    __syncthreads();
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int f = rg + i * (kStepThreads / 8);
        if (f < a.d) {
            const float kf = sk[f], qf = sq[f];
            float4 w = s[i];
            w.x = fmaf(lam, w.x, kf * vc[0]); w.y = fmaf(lam, w.y, kf * vc[1]);
            w.z = fmaf(lam, w.z, kf * vc[2]); w.w = fmaf(lam, w.w, kf * vc[3]);
            float *p = S + (int64_t)f * a.dv + c;
            if (VEC) {
                if (c < a.dv) *reinterpret_cast<float4 *>(p) = w;
            } else {
                if (c < a.dv) p[0] = w.x;
                if (c + 1 < a.dv) p[1] = w.y;
                if (c + 2 < a.dv) p[2] = w.z;
                if (c + 3 < a.dv) p[3] = w.w;
            }
            acc[0] = fmaf(qf, w.x, acc[0]); acc[1] = fmaf(qf, w.y, acc[1]);
            acc[2] = fmaf(qf, w.z, acc[2]); acc[3] = fmaf(qf, w.w, acc[3]);
        }
    }
    // the four rows of a warp, then the warps in order
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        acc[t] += __shfl_xor_sync(0xffffffffu, acc[t], 8);
        acc[t] += __shfl_xor_sync(0xffffffffu, acc[t], 16);
    }
    if ((tid & 31) < 8) {
#pragma unroll
        for (int t = 0; t < 4; ++t) so[tid / 32][4 * cg + t] = acc[t];
    }
    __syncthreads();
    if (tid < kCols && col0 + tid < a.dv) {
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < kStepThreads / 32; ++w) y += so[w][tid];
        io_store(o + col0 + tid, a.scale * y);
    }
}

int cdiv(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

template <typename IO, typename OUT>
cudaError_t mix(const DecayMix &a, cudaStream_t s) {
    const size_t smem = sizeof(float) * (2 * kCh * (a.da + 1) + kCh * (kCols + 1) + kCh * (kCh + 1) + a.da * kCols + kCh + 1);
    cudaError_t e = cudaFuncSetAttribute(k_decay_mix<IO, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)((int64_t)a.B * a.H * a.nseg), cdiv(a.dc, kCols));
    LUNA_LAUNCH("decay_mix", (k_decay_mix<IO, OUT>), grid, kMixThreads, smem, s, a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_decay_mix(const DecayMix &a, luna_dtype io, luna_dtype out, cudaStream_t s) {
    if (decay_tc_ok(a, io, out)) return launch_decay_mix_tc(a, out, s);
    if (io == LUNA_F32) return mix<float, float>(a, s);
    return out == LUNA_F32 ? mix<__nv_bfloat16, float>(a, s) : mix<__nv_bfloat16, __nv_bfloat16>(a, s);
}

cudaError_t launch_decay_scan(const DecayScan &a, cudaStream_t s) {
    LUNA_LAUNCH("decay_scan", k_decay_scan, dim3((unsigned)(a.B * a.H), cdiv(a.E, 256)), 256, 0, s, a);
    return cudaGetLastError();
}

cudaError_t launch_decay_group_sum(const float *src, int B, int H, int G, int n, int width, void *dst, int64_t sb,
                                   int64_t sh, int64_t st, luna_dtype io, cudaStream_t s) {
    const int64_t total = (int64_t)B * (H / G) * n * width;
    const unsigned grid = (unsigned)cdiv(total, 256);
    if (io == LUNA_F32)
        LUNA_LAUNCH("decay_group_sum", k_decay_group_sum<float>, grid, 256, 0, s, src, H, G, n, width,
                    static_cast<float *>(dst), sb, sh, st, total);
    else
        LUNA_LAUNCH("decay_group_sum", k_decay_group_sum<__nv_bfloat16>, grid, 256, 0, s, src, H, G, n, width,
                    static_cast<__nv_bfloat16 *>(dst), sb, sh, st, total);
    return cudaGetLastError();
}

cudaError_t launch_decay_step(const DecayStep &a, luna_dtype io, cudaStream_t s) {
    // 16-byte accesses need rows of whole float4s and an aligned state
    const bool vec = a.dv % 4 == 0 && (reinterpret_cast<uintptr_t>(a.S) & 15) == 0;
    const dim3 grid((unsigned)(a.B * a.H), cdiv(a.dv, kCols));
    if (io == LUNA_F32) {
        if (vec)
            LUNA_LAUNCH("decay_step", (k_decay_step<float, true>), grid, kStepThreads, 0, s, a);
        else
            LUNA_LAUNCH("decay_step", (k_decay_step<float, false>), grid, kStepThreads, 0, s, a);
    } else {
        if (vec)
            LUNA_LAUNCH("decay_step", (k_decay_step<__nv_bfloat16, true>), grid, kStepThreads, 0, s, a);
        else
            LUNA_LAUNCH("decay_step", (k_decay_step<__nv_bfloat16, false>), grid, kStepThreads, 0, s, a);
    }
    return cudaGetLastError();
}

}  // namespace luna
