// Linear attention with a decay for each head on CUDA cores in fp32: the form for
// every type, width and stride (the tensor-core form covers bf16 at aligned
// widths), the scan of the pieces' states, the sum over grouped heads, and the
// single-token step.
#include "luna_decay.cuh"
#include "luna_prof.cuh"

#include <string.h>

namespace luna {
namespace {

constexpr int kMixThreads = 256;
constexpr int kCols = 32;      // state columns of a block of the single-token step

template <typename T>
__device__ __forceinline__ const T *row_base(const RowView &v, int b, int h, int H) {
    return static_cast<const T *>(v.p) + b * v.sb + (int64_t)(h / (H / v.heads)) * v.sh;
}

// Four consecutive values of a row, zeros past `width`.
template <typename IO>
__device__ __forceinline__ float4 load4(const IO *p, int c, int width, bool vec) {
    if (vec && c + 4 <= width) {
        if (sizeof(IO) == 4) return *reinterpret_cast<const float4 *>(p + c);
        const uint2 w = *reinterpret_cast<const uint2 *>(p + c);
        return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                           __uint_as_float(w.y & 0xffff0000u));
    }
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = c + i < width ? io_load(p + c + i) : 0.0f;
    return make_float4(v[0], v[1], v[2], v[3]);
}
template <typename OUT>
__device__ __forceinline__ void store4(OUT *p, int c, int width, bool vec, const float *v) {
    if (vec && c + 4 <= width && sizeof(OUT) == 4) {
        *reinterpret_cast<float4 *>(p + c) = make_float4(v[0], v[1], v[2], v[3]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (c + i < width) io_store(p + c + i, v[i]);
}

// One block: piece s of head (b, h), chunks of 64 rows.  DA, DC: widths rounded up (64 or 128).
//     P = (a b^T) masked and decayed,  out = p P c + x lambda^{m+e} a X,  X = lambda^{nv} X + u (b w)^T c
// Every product runs from shared memory with a register tile a thread (4 x 4 scores, 4 rows x DC / 16
// outputs, DA / 16 x DC / 16 of the state, which stays in registers and is copied to shared memory for
// the outputs), 16-byte reads without bank conflicts, two multiply-adds an instruction.  Bound by the
// fp32 FMA rate at width 128 (2.6 ms in two passes for 160 heads of 5276 rows at 128 x 64 in fp32, some
// 24 TFLOP/s), by the loads' latency at small widths, where two blocks share an SM.
// CH: rows of a chunk, 64, or 16 where no sequence is longer than that.
template <typename IO, typename OUT, int DA, int DC, int CH>
__global__ void __launch_bounds__(kMixThreads, DA + DC <= 128 ? 2 : 1) k_decay_mix(DecayMix a) {
    extern __shared__ float4 sm4[];
    clear_status(a);
    constexpr int LA = DA + 4, LC = DC + 4, LP = CH + 4, RT = CH / 16, FT = DA / 64, CT = DC / 64;
    float *sa = reinterpret_cast<float *>(sm4), *sb = sa + CH * LA, *sc = sb + CH * LA, *sP = sc + CH * LC;
    float *sX = sP + CH * LP, *pw = sX + DA * LC;
    const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    const int seg = (int)(blockIdx.x % a.nseg);
    const int64_t bh = blockIdx.x / a.nseg;
    const int b = (int)(bh / a.H), h = (int)(bh % a.H);
    const int e = a.reverse ? 0 : 1;
    const float g = decay_log(a.log_decay, h);
    for (int i = tid; i <= CH; i += kMixThreads) pw[i] = expf(g * (float)i);
    const int len = head_length(a.lengths, b, a.n);
    const int r0 = seg * a.seg_len, rend = min(a.n, r0 + a.seg_len);
    const int r1 = max(r0, min(len, rend));
    const IO *A = row_base<IO>(a.a, b, h, a.H), *Bm = row_base<IO>(a.b, b, h, a.H), *Cm = row_base<IO>(a.c, b, h, a.H);
    OUT *O = a.out ? static_cast<OUT *>(a.out) + b * a.ob + (int64_t)h * a.oh : nullptr;
    // this thread's part of the state: rows 4 ty + 64 i + k, columns 4 tx + 64 j + l
    uint64_t X[4 * FT][2 * CT];  // columns in pairs
    {
        const float *x = a.X ? a.X + (bh * a.x_pieces + (a.x_pieces > 1 ? seg : 0)) * a.da * a.dc : nullptr;
#pragma unroll
        for (int i = 0; i < 4 * FT; ++i)
#pragma unroll
            for (int j = 0; j < 2 * CT; ++j) {
                const int f = 4 * ty + 64 * (i / 4) + i % 4, c = 4 * tx + 64 * (j / 2) + 2 * (j % 2);
                float v[2];
#pragma unroll
                for (int l = 0; l < 2; ++l)
                    v[l] = x && f < a.da && c + l < a.dc
                               ? (a.x_trans ? x[(int64_t)(c + l) * a.da + f] : x[(int64_t)f * a.dc + c + l]) : 0.0f;
                X[i][j] = f2(v[0], v[1]);
            }
    }
    const int na = (a.da + 3) / 4, nc = (a.dc + 3) / 4;  // float4 pieces of a row
    const int nch = (r1 - r0 + CH - 1) / CH;
    for (int ci = 0; ci < nch; ++ci) {
        const int row0 = r0 + (a.reverse ? nch - 1 - ci : ci) * CH;
        const int nv = min(CH, r1 - row0);
        __syncthreads();
        // the pieces of b, c and (where outputs are wanted) a, eight loads of a thread in flight
        const int nb = CH * na, total = nb + CH * nc + (O ? nb : 0);
#pragma unroll 1
        for (int i0 = tid; i0 < total; i0 += 8 * kMixThreads) {
            float4 v[8];
            float *to[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                int i = i0 + q * kMixThreads;
                const bool is_b = i < nb, is_c = !is_b && i < nb + CH * nc;
                const int per = is_c ? nc : na;
                to[q] = i < total ? (is_b ? sb : is_c ? sc : sa) : nullptr;
                i -= is_b ? 0 : is_c ? nb : nb + CH * nc;
                const int r = i / per, c = 4 * (i % per);
                const RowView &w = is_b ? a.b : is_c ? a.c : a.a;
                const IO *p = is_b ? Bm : is_c ? Cm : A;
                v[q] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (to[q]) {
                    to[q] += r * (is_c ? LC : LA) + c;
                    if (r < nv) v[q] = load4<IO>(p + (int64_t)(row0 + r) * w.st, c, is_c ? a.dc : a.da, w.vec);
                }
            }
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (to[q]) *reinterpret_cast<float4 *>(to[q]) = v[q];
        }
        if (O) {
#pragma unroll
            for (int i = 0; i < 4 * FT; ++i)
#pragma unroll
                for (int j = 0; j < CT; ++j)
                    *reinterpret_cast<ulonglong2 *>(sX + (4 * ty + 64 * (i / 4) + i % 4) * LC + 4 * tx + 64 * j) =
                        make_ulonglong2(X[i][2 * j], X[i][2 * j + 1]);
        }
        __syncthreads();
        if (O) {
            {  // scores of rows ty + 16 i, columns tx + 16 j
                uint64_t acc[RT][RT];  // two partial sums each
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int j = 0; j < RT; ++j) acc[i][j] = 0;
#pragma unroll 2
                for (int k = 0; k < na; ++k) {
                    float4 u[RT], v[RT];
#pragma unroll
                    for (int i = 0; i < RT; ++i) {
                        u[i] = *reinterpret_cast<const float4 *>(sa + (ty + 16 * i) * LA + 4 * k);
                        v[i] = *reinterpret_cast<const float4 *>(sb + (tx + 16 * i) * LA + 4 * k);
                    }
#pragma unroll
                    for (int i = 0; i < RT; ++i)
#pragma unroll
                        for (int j = 0; j < RT; ++j) {
                            acc[i][j] = fma2(f2(u[i].x, u[i].y), f2(v[j].x, v[j].y), acc[i][j]);
                            acc[i][j] = fma2(f2(u[i].z, u[i].w), f2(v[j].z, v[j].w), acc[i][j]);
                        }
                }
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int j = 0; j < RT; ++j) {
                        const int r = ty + 16 * i, c = tx + 16 * j, dist = a.reverse ? c - r : r - c;
                        float lo, hi;
                        unpack2(acc[i][j], lo, hi);
                        sP[r * LP + c] = dist >= 0 ? a.p * (lo + hi) * pw[dist] : 0.0f;
                    }
            }
            __syncthreads();
            uint64_t out[RT][2 * CT];  // rows ty + 16 i, columns 4 tx + 64 j + l in pairs
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < 2 * CT; ++j) out[i][j] = 0;
            // out (+)= left (rows of lda) times right (rows of LC), over n pieces of four
            auto product = [&](const float *left, int lda, const float *right, int n) {
#pragma unroll 1
                for (int k = 0; k < n; ++k) {
                    float4 u[RT];
#pragma unroll
                    for (int i = 0; i < RT; ++i) u[i] = *reinterpret_cast<const float4 *>(left + (ty + 16 * i) * lda + 4 * k);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int j = 0; j < CT; ++j) {
                            const float4 v = *reinterpret_cast<const float4 *>(right + (4 * k + q) * LC + 4 * tx + 64 * j);
#pragma unroll
                            for (int i = 0; i < RT; ++i) {
                                const float w = q == 0 ? u[i].x : q == 1 ? u[i].y : q == 2 ? u[i].z : u[i].w;
                                out[i][2 * j] = fma2(f2(w, w), f2(v.x, v.y), out[i][2 * j]);
                                out[i][2 * j + 1] = fma2(f2(w, w), f2(v.z, v.w), out[i][2 * j + 1]);
                            }
                        }
                }
            };
            product(sa, LA, sX, na);  // (a's columns past da are zeros to a whole piece, and so are X's rows)
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int r = ty + 16 * i;
                const float w = a.x * pw[max(0, a.reverse ? nv - 1 - r : min(r, CH - 1)) + e];
#pragma unroll
                for (int j = 0; j < 2 * CT; ++j) out[i][j] = mul2(out[i][j], f2(w, w));
            }
            product(sP, LP, sc, CH / 4);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int r = ty + 16 * i;
                if (r < nv)
#pragma unroll
                    for (int j = 0; j < CT; ++j) {
                        float v[4];
                        unpack2(out[i][2 * j], v[0], v[1]);
                        unpack2(out[i][2 * j + 1], v[2], v[3]);
                        store4<OUT>(O + (int64_t)(row0 + r) * a.ot, 4 * tx + 64 * j, a.dc, a.ovec, v);
                    }
            }
        }
        if (ci == nch - 1 && !a.Xout) break;  // (the state is wanted no further)
        const float dec = pw[nv];
#pragma unroll
        for (int i = 0; i < 4 * FT; ++i)
#pragma unroll
            for (int j = 0; j < 2 * CT; ++j) X[i][j] = mul2(X[i][j], f2(dec, dec));
#pragma unroll 2
        for (int r = 0; r < nv; ++r) {
            const float w = a.u * pw[nv - (a.reverse ? nv - 1 - r : r) - e];
            float4 v[CT];
#pragma unroll
            for (int j = 0; j < CT; ++j) v[j] = *reinterpret_cast<const float4 *>(sc + r * LC + 4 * tx + 64 * j);
#pragma unroll
            for (int i = 0; i < FT; ++i) {
                const float4 u = *reinterpret_cast<const float4 *>(sb + r * LA + 4 * ty + 64 * i);
                const float uw[4] = {w * u.x, w * u.y, w * u.z, w * u.w};
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int j = 0; j < CT; ++j) {
                        X[4 * i + k][2 * j] = fma2(f2(uw[k], uw[k]), f2(v[j].x, v[j].y), X[4 * i + k][2 * j]);
                        X[4 * i + k][2 * j + 1] = fma2(f2(uw[k], uw[k]), f2(v[j].z, v[j].w), X[4 * i + k][2 * j + 1]);
                    }
            }
        }
    }
    if (O)  // rows at and past the length
        for (int i = tid; i < (rend - r1) * nc; i += kMixThreads) {  // (under 2^29: a row has at most 32 pieces)
            const float z[4] = {0.f, 0.f, 0.f, 0.f};
            store4<OUT>(O + (int64_t)(r1 + i / nc) * a.ot, 4 * (i % nc), a.dc, a.ovec, z);
        }
    if (a.Xout) {
        float *x = a.Xout + (bh * a.nseg + seg) * a.da * a.dc;
#pragma unroll
        for (int i = 0; i < 4 * FT; ++i)
#pragma unroll
            for (int j = 0; j < 2 * CT; ++j) {
                const int f = 4 * ty + 64 * (i / 4) + i % 4, c = 4 * tx + 64 * (j / 2) + 2 * (j % 2);
                float v[2];
                unpack2(X[i][j], v[0], v[1]);
                if (f < a.da && c < a.dc) x[(int64_t)f * a.dc + c] = v[0];
                if (f < a.da && c + 1 < a.dc) x[(int64_t)f * a.dc + c + 1] = v[1];
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

// Four columns a thread; bound by the bytes of src (21 us for 480 heads of 313 rows of 128, 4 TB/s).
template <typename IO>
__global__ void __launch_bounds__(256) k_decay_group_sum(const float *src, int H, int G, int n, int width, IO *dst,
                                                         int64_t sb, int64_t sh, int64_t st) {
    const int per = (width + 3) / 4, Hk = H / G, b = blockIdx.x / Hk, hk = blockIdx.x % Hk;
    const float *head = src + ((int64_t)b * H + (int64_t)hk * G) * n * width;
    IO *out = dst + b * sb + (int64_t)hk * sh;
    const bool vec = width % 4 == 0 && st % 4 == 0 && sb % 4 == 0 && sh % 4 == 0 && reinterpret_cast<uintptr_t>(dst) % 16 == 0;
    const int total = n * per;  // under 2^29
    for (int i = blockIdx.y * 256 + threadIdx.x; i < total; i += gridDim.y * 256) {
        const int t = i / per, c = (i - t * per) * 4;
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < G; ++j) {
            const float4 v = load4<float>(head + ((int64_t)j * n + t) * width, c, width, width % 4 == 0);
            acc[0] += v.x; acc[1] += v.y; acc[2] += v.z; acc[3] += v.w;
        }
        IO *o = out + (int64_t)t * st;
        if (vec && sizeof(IO) == 2) {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(acc[0], acc[1]), hi = __floats2bfloat162_rn(acc[2], acc[3]);
            uint2 w;
            memcpy(&w.x, &lo, 4);
            memcpy(&w.y, &hi, 4);
            *reinterpret_cast<uint2 *>(o + c) = w;
        } else {
            store4<IO>(o, c, width, vec, acc);
        }
    }
}

// ---------------------------------------------------------------------------
// One token: S <- lambda S + k v^T, o = scale q^T S.  A block owns 32 columns of one
// head's state: 8 lanes x 16 bytes cover a row's 128 bytes, four rows a warp, 32 rows a
// block at a time, every load of a thread in flight before the first is used.  The state is
// read and written once, which bounds the step (45 to 47 us for 270 MB of states and tokens, 5.7 to 6 TB/s);
// the column split keeps one sequence's 32 heads on 128 blocks.
// lambda has a second term: rounded to fp32 alone it is off by up to 3e-8 the same way at every token, which
// after 30000 tokens of slow decay has been 1.1e-3 of the state.

constexpr int kStepThreads = 256;

template <typename IO, bool VEC>
__global__ void __launch_bounds__(kStepThreads) k_decay_step(DecayStep a) {
    __shared__ float sq[kMaxD], sk[kMaxD], slam[2];
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
    if (tid == kStepThreads - 1) {  // (once a block: by every thread 16.4 us at 64 x 32 heads of 64 x 64, so 14.5)
        const float g = decay_log(a.log_decay, h), m1 = expm1f(g);
        const bool slow = fabsf(g) < 0.5f;  // (beyond that a state forgets, or overflows, in some ten tokens)
        slam[0] = slow ? 1.0f + m1 : expf(g);
        slam[1] = slow ? m1 - (slam[0] - 1.0f) : 0.0f;
    }
    __syncthreads();
    const float lam = slam[0], rest = slam[1];
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int f = rg + i * (kStepThreads / 8);
        if (f < a.d) {
            const float kf = sk[f], qf = sq[f];
            float4 w = s[i];
            w.x = fmaf(lam, w.x, fmaf(rest, w.x, kf * vc[0])); w.y = fmaf(lam, w.y, fmaf(rest, w.y, kf * vc[1]));
            w.z = fmaf(lam, w.z, fmaf(rest, w.z, kf * vc[2])); w.w = fmaf(lam, w.w, fmaf(rest, w.w, kf * vc[3]));
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

template <typename IO, typename OUT, int DA, int DC, int CH>
cudaError_t mix_launch(const DecayMix &a, cudaStream_t s) {
    const size_t smem = sizeof(float) * (2 * CH * (DA + 4) + CH * (DC + 4) + CH * (CH + 4) + DA * (DC + 4) + CH + 4);
    cudaError_t e = cudaFuncSetAttribute(k_decay_mix<IO, OUT, DA, DC, CH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)((int64_t)a.B * a.H * a.nseg);
    LUNA_LAUNCH("decay_mix", (k_decay_mix<IO, OUT, DA, DC, CH>), grid, kMixThreads, smem, s, a);
    return cudaGetLastError();
}

template <typename IO, typename OUT, int CH>
cudaError_t mix_width(const DecayMix &a, cudaStream_t s) {
    if (a.da <= 64) return a.dc <= 64 ? mix_launch<IO, OUT, 64, 64, CH>(a, s) : mix_launch<IO, OUT, 64, 128, CH>(a, s);
    return a.dc <= 64 ? mix_launch<IO, OUT, 128, 64, CH>(a, s) : mix_launch<IO, OUT, 128, 128, CH>(a, s);
}

template <typename IO, typename OUT>
cudaError_t mix(DecayMix a, cudaStream_t s) {
    // loads of four values: rows that start on their boundary
    auto quad = [](const void *p, int64_t sb, int64_t sh, int64_t st, size_t size) {
        return (reinterpret_cast<uintptr_t>(p) % (4 * size)) == 0 && sb % 4 == 0 && sh % 4 == 0 && st % 4 == 0;
    };
    for (RowView *v : {&a.a, &a.b, &a.c}) v->vec = quad(v->p, v->sb, v->sh, v->st, sizeof(IO));
    a.ovec = quad(a.out, a.ob, a.oh, a.ot, sizeof(OUT));
    return a.n <= 16 ? mix_width<IO, OUT, 16>(a, s) : mix_width<IO, OUT, kDecaySimtRows>(a, s);
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
    const int64_t blocks = ((int64_t)n * ((width + 3) / 4) + 255) / 256;
    const dim3 grid((unsigned)(B * (H / G)), (unsigned)(blocks < 4096 ? blocks : 4096));
    if (io == LUNA_F32)
        LUNA_LAUNCH("decay_group_sum", k_decay_group_sum<float>, grid, 256, 0, s, src, H, G, n, width,
                    static_cast<float *>(dst), sb, sh, st);
    else
        LUNA_LAUNCH("decay_group_sum", k_decay_group_sum<__nv_bfloat16>, grid, 256, 0, s, src, H, G, n, width,
                    static_cast<__nv_bfloat16 *>(dst), sb, sh, st);
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
