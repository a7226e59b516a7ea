// C ABI of linear attention with decay: argument checks, piece planning, dispatch.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "luna_decay.cuh"

namespace luna {
int tc_sm_count();
}
using namespace luna;

namespace {

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
luna_status cuda_status(cudaError_t e) { return e == cudaSuccess ? LUNA_OK : LUNA_ERR_CUDA; }

// A tensor's strides with the contiguous default filled in.
luna_strides filled(luna_strides s, int heads, int n, int width) {
    if (s.b == 0 && s.h == 0 && s.t == 0) s = luna_strides{(int64_t)heads * n * width, (int64_t)n * width, width};
    return s;
}

// Whether no two elements of an output share an address: every dimension's stride is at
// least the extent of the dimensions with smaller strides.
bool disjoint(const luna_strides &s, int B, int heads, int n, int width) {
    struct D { int64_t stride, ext; } d[3] = {{s.b, B}, {s.h, heads}, {s.t, n}};
    std::sort(d, d + 3, [](const D &x, const D &y) { return x.stride < y.stride; });
    int64_t span = width;
    for (const D &x : d) {
        if (x.ext <= 1) continue;
        if (x.stride < span) return false;
        span += (x.ext - 1) * x.stride;
    }
    return true;
}

bool negative(const luna_strides &s) { return s.b < 0 || s.h < 0 || s.t < 0; }

luna_status check(const luna_decay_desc *dd) {
    if (!dd) return LUNA_ERR_INVALID_ARG;
    if (dd->B < 0 || dd->H < 0 || dd->Hkv < 0 || dd->n < 0 || dd->d < 1 || dd->dv < 1) return LUNA_ERR_INVALID_ARG;
    if (dd->io != LUNA_F32 && dd->io != LUNA_BF16) return LUNA_ERR_INVALID_ARG;
    if (!isfinite(dd->scale)) return LUNA_ERR_INVALID_ARG;
    if (dd->H > 0 && (dd->Hkv < 1 || dd->H % dd->Hkv != 0)) return LUNA_ERR_INVALID_ARG;
    for (const luna_strides *s : {&dd->q, &dd->k, &dd->v, &dd->o, &dd->gq, &dd->gk, &dd->gv, &dd->go})
        if (negative(*s)) return LUNA_ERR_INVALID_ARG;
    if (dd->d > kMaxD || dd->dv > kMaxD || dd->n > (1 << 24) || (int64_t)dd->B * dd->H > (1 << 24))
        return LUNA_ERR_UNSUPPORTED;
    return LUNA_OK;
}

struct Plan {
    int seg_len, nseg;
    size_t state;  // bytes of one set of piece states (none with one piece: the pass itself carries the state)
    size_t o_U = 256, o_X = 0, o_R = 0, o_part = 0, fwd = 0, bwd = 0;
};

// Pieces of the rows.  More pieces fill more SMs, but with more than one the states before each have to
// be summed first, a pass over two of the four tensors; the piece count with the least of (pieces of a
// block) x (chunks of a piece, and about half of one to start it) x (passes) is taken.
Plan make_plan(const luna_decay_desc *dd) {
    Plan p;
    const bool tc = dd->io == LUNA_BF16 && dd->d % 8 == 0 && dd->dv % 8 == 0;
    const int rows = tc ? 128 : kDecaySimtRows;
    const int64_t BH = (int64_t)dd->B * dd->H, chunks = cdiv(std::max(1, dd->n), rows);
    const double room = (double)tc_sm_count() * (!tc && std::max(dd->d, dd->dv) <= 64 ? 2 : 1);  // blocks the SMs hold
    int64_t best = 1;
    double least = 1e300;
    for (int64_t ns = 1; ns <= std::min<int64_t>(64, chunks); ++ns) {
        const double rounds = ceil((double)(BH * ns) / room);
        const double cost = (rounds * ((double)cdiv(chunks, ns) + 0.5) + 1) * (ns > 1 ? 1.45 : 1.0);
        if (cost < least) { least = cost; best = ns; }
    }
    p.seg_len = (int)(cdiv(chunks, best) * rows);
    p.nseg = (int)cdiv(std::max(1, dd->n), p.seg_len);
    p.state = p.nseg == 1 ? 0 : (size_t)align256((int64_t)BH * p.nseg * dd->d * dd->dv * 4);
    p.o_X = p.o_U + p.state;
    p.fwd = p.o_X + p.state;
    p.o_R = p.fwd;
    p.o_part = p.o_R + p.state;
    p.bwd = p.o_part;
    if (dd->H != dd->Hkv)  // gradients of shared keys or values, one for each query head
        p.bwd += (size_t)align256(BH * dd->n * std::max(dd->d, dd->dv) * 4);
    return p;
}

bool empty(const luna_decay_desc *dd) { return (int64_t)dd->B * dd->H == 0; }

RowView view(const void *p, const luna_strides &s, int heads) { return RowView{p, s.b, s.h, s.t, heads}; }

// What all passes of a call share.
DecayMix base(const luna_decay_desc *dd, const Plan &p, const float *log_decay, const int32_t *lengths, char *ws) {
    DecayMix a{};
    a.status = reinterpret_cast<int *>(ws);
    a.log_decay = log_decay;
    a.lengths = lengths;
    a.B = dd->B; a.H = dd->H; a.n = dd->n;
    a.seg_len = p.seg_len; a.nseg = p.nseg;
    a.p = a.x = a.u = 1.0f;
    return a;
}

// The carries into every piece of a sequence of states, from the pieces' own sums (two launches);
// with one piece, nothing (the pass itself starts from `init` and leaves `last`).
cudaError_t carries(DecayMix a, const Plan &p, luna_dtype io, char *ws, const float *init, float *X, float *last,
                    cudaStream_t s) {
    if (p.nseg == 1) return cudaSuccess;
    float *U = reinterpret_cast<float *>(ws + p.o_U);
    a.out = nullptr;
    a.X = nullptr;
    a.Xout = U;
    cudaError_t e = launch_decay_mix(a, io, io, s);
    if (e != cudaSuccess) return e;
    DecayScan sc{U, init, X, last, a.log_decay, a.lengths, a.B, a.H, a.n, p.seg_len, p.nseg, a.reverse,
                 (int64_t)a.da * a.dc};
    return launch_decay_scan(sc, s);
}

}  // namespace

extern "C" {

luna_status luna_decay_workspace_size(const luna_decay_desc *dd, int backward, size_t *bytes) {
    if (!bytes) return LUNA_ERR_INVALID_ARG;
    const luna_status st = check(dd);
    if (st != LUNA_OK) return st;
    const Plan p = make_plan(dd);
    *bytes = empty(dd) ? 256 : backward ? p.bwd : p.fwd;
    return LUNA_OK;
}

luna_status luna_decay_fwd(const luna_decay_desc *dd, const float *log_decay, const void *Q, const void *K,
                           const void *V, const int32_t *lengths, const float *S0, void *O, float *S1,
                           void *workspace, size_t ws_bytes, void *stream) {
    luna_status st = check(dd);
    if (st != LUNA_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (empty(dd)) return LUNA_OK;
    const size_t SB = (size_t)dd->B * dd->H * dd->d * dd->dv * 4;
    if (dd->n == 0) {
        if (!S1 || S1 == S0) return LUNA_OK;
        return cuda_status(S0 ? cudaMemcpyAsync(S1, S0, SB, cudaMemcpyDeviceToDevice, s) : cudaMemsetAsync(S1, 0, SB, s));
    }
    if (!log_decay || !Q || !K || !V || !O || !workspace || !aligned(workspace, 256)) return LUNA_ERR_INVALID_ARG;
    const luna_strides sq = filled(dd->q, dd->H, dd->n, dd->d), sk = filled(dd->k, dd->Hkv, dd->n, dd->d);
    const luna_strides sv = filled(dd->v, dd->Hkv, dd->n, dd->dv), so = filled(dd->o, dd->H, dd->n, dd->dv);
    if (!disjoint(so, dd->B, dd->H, dd->n, dd->dv)) return LUNA_ERR_INVALID_ARG;
    const Plan p = make_plan(dd);
    if (ws_bytes < p.fwd) return LUNA_ERR_WORKSPACE;
    char *ws = static_cast<char *>(workspace);

    DecayMix a = base(dd, p, log_decay, lengths, ws);
    a.a = view(Q, sq, dd->H); a.b = view(K, sk, dd->Hkv); a.c = view(V, sv, dd->Hkv);
    a.da = dd->d; a.dc = dd->dv;
    a.p = a.x = dd->scale;
    float *X = reinterpret_cast<float *>(ws + p.o_X);
    a.clear = 1;
    cudaError_t e = carries(a, p, dd->io, ws, S0, X, S1, s);
    if (e != cudaSuccess) return LUNA_ERR_CUDA;
    a.out = O;
    a.ob = so.b; a.oh = so.h; a.ot = so.t;
    a.clear = p.nseg == 1;
    a.X = p.nseg == 1 ? S0 : X;
    a.x_pieces = p.nseg;
    a.Xout = p.nseg == 1 ? S1 : nullptr;
    return cuda_status(launch_decay_mix(a, dd->io, dd->io, s));
}

luna_status luna_decay_bwd(const luna_decay_desc *dd, const float *log_decay, const void *Q, const void *K,
                           const void *V, const void *dO, const int32_t *lengths, const float *S0, const float *dS1,
                           void *dQ, void *dK, void *dV, float *dS0, void *workspace, size_t ws_bytes,
                           void *stream) {
    luna_status st = check(dd);
    if (st != LUNA_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (empty(dd)) return LUNA_OK;
    const size_t SB = (size_t)dd->B * dd->H * dd->d * dd->dv * 4;
    if (dd->n == 0) {
        if (!dS0 || dS0 == dS1) return LUNA_OK;
        return cuda_status(dS1 ? cudaMemcpyAsync(dS0, dS1, SB, cudaMemcpyDeviceToDevice, s)
                               : cudaMemsetAsync(dS0, 0, SB, s));
    }
    if (!log_decay || !Q || !K || !V || !dO || !dQ || !dK || !dV || !workspace || !aligned(workspace, 256))
        return LUNA_ERR_INVALID_ARG;
    const int H = dd->H, Hkv = dd->Hkv, n = dd->n, d = dd->d, dv = dd->dv, G = H / Hkv;
    const luna_strides sq = filled(dd->q, H, n, d), sk = filled(dd->k, Hkv, n, d), sv = filled(dd->v, Hkv, n, dv);
    const luna_strides go = filled(dd->go, H, n, dv), gq = filled(dd->gq, H, n, d);
    const luna_strides gk = filled(dd->gk, Hkv, n, d), gv = filled(dd->gv, Hkv, n, dv);
    if (!disjoint(gq, dd->B, H, n, d) || !disjoint(gk, dd->B, Hkv, n, d) || !disjoint(gv, dd->B, Hkv, n, dv))
        return LUNA_ERR_INVALID_ARG;
    const Plan p = make_plan(dd);
    if (ws_bytes < p.bwd) return LUNA_ERR_WORKSPACE;
    char *ws = static_cast<char *>(workspace);
    const RowView q = view(Q, sq, H), k = view(K, sk, Hkv), v = view(V, sv, Hkv), g = view(dO, go, H);
    float *X = reinterpret_cast<float *>(ws + p.o_X), *R = reinterpret_cast<float *>(ws + p.o_R);
    float *part = reinterpret_cast<float *>(ws + p.o_part);
    cudaError_t e;

    // states before every piece, gradients of the states after every piece
    DecayMix a = base(dd, p, log_decay, lengths, ws);
    a.a = k; a.b = k; a.c = v; a.da = d; a.dc = dv;
    a.clear = 1;
    if ((e = carries(a, p, dd->io, ws, S0, X, nullptr, s)) != cudaSuccess) return LUNA_ERR_CUDA;
    a.clear = 0;
    a.reverse = 1;
    a.a = q; a.b = q; a.c = g;
    a.u = dd->scale;
    if ((e = carries(a, p, dd->io, ws, dS1, R, dS0, s)) != cudaSuccess) return LUNA_ERR_CUDA;

    a = base(dd, p, log_decay, lengths, ws);
    a.x_pieces = p.nseg;
    a.x_trans = 1;
    a.p = a.x = dd->scale;
    a.a = g; a.b = v; a.c = k; a.da = dv; a.dc = d;
    a.X = p.nseg == 1 ? S0 : X;
    a.out = dQ; a.ob = gq.b; a.oh = gq.h; a.ot = gq.t;
    a.clear = p.nseg == 1;
    if ((e = launch_decay_mix(a, dd->io, dd->io, s)) != cudaSuccess) return LUNA_ERR_CUDA;
    a.clear = 0;

    a.reverse = 1;
    a.x = 1.0f;
    a.p = a.u = dd->scale;
    a.X = p.nseg == 1 ? dS1 : R;
    const int64_t rows = (int64_t)n;
    // dK, then dV, whose carry with one piece is dS0 (which may be dS1 itself, read by both)
    for (int side = 1; side >= 0; --side) {
        const int w = side == 0 ? dv : d;
        const luna_strides &so = side == 0 ? gv : gk;
        void *dst = side == 0 ? dV : dK;
        a.a = side == 0 ? k : v;
        a.b = side == 0 ? q : g;
        a.c = side == 0 ? g : q;
        a.da = side == 0 ? d : dv;
        a.dc = w;
        a.x_trans = side;
        a.Xout = side == 0 && p.nseg == 1 ? dS0 : nullptr;
        if (G == 1) {
            a.out = dst; a.ob = so.b; a.oh = so.h; a.ot = so.t;
            if ((e = launch_decay_mix(a, dd->io, dd->io, s)) != cudaSuccess) return LUNA_ERR_CUDA;
        } else {
            a.out = part; a.ob = (int64_t)H * rows * w; a.oh = rows * w; a.ot = w;
            if ((e = launch_decay_mix(a, dd->io, LUNA_F32, s)) != cudaSuccess) return LUNA_ERR_CUDA;
            e = launch_decay_group_sum(part, dd->B, H, G, n, w, dst, so.b, so.h, so.t, dd->io, s);
            if (e != cudaSuccess) return LUNA_ERR_CUDA;
        }
    }
    return LUNA_OK;
}

luna_status luna_decay_step(const luna_decay_desc *dd, const float *log_decay, const void *q, const void *k,
                            const void *v, const int32_t *slots, int nslots, float *S, void *o, void *stream) {
    const luna_status st = check(dd);
    if (st != LUNA_OK) return st;
    if (nslots < 0 || (!slots && nslots < dd->B)) return LUNA_ERR_INVALID_ARG;
    if (empty(dd)) return LUNA_OK;
    if (!log_decay || !q || !k || !v || !o || (nslots > 0 && !S)) return LUNA_ERR_INVALID_ARG;
    const luna_strides sq = filled(dd->q, dd->H, 1, dd->d), sk = filled(dd->k, dd->Hkv, 1, dd->d);
    const luna_strides sv = filled(dd->v, dd->Hkv, 1, dd->dv), so = filled(dd->o, dd->H, 1, dd->dv);
    if (!disjoint(so, dd->B, dd->H, 1, dd->dv)) return LUNA_ERR_INVALID_ARG;
    DecayStep a{q, k, v, o, sq.b, sq.h, sk.b, sk.h, sv.b, sv.h, so.b, so.h, log_decay, slots, S, nslots,
                dd->B, dd->H, dd->Hkv, dd->d, dd->dv, dd->scale};
    return cuda_status(launch_decay_step(a, dd->io, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
