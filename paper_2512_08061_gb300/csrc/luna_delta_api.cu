// C ABI of the gated delta rule: argument checks, workspace, dispatch.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "luna_delta.cuh"

using namespace luna;

namespace {

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
luna_status cuda_status(cudaError_t e) { return e == cudaSuccess ? LUNA_OK : LUNA_ERR_CUDA; }

// A tensor's strides with the contiguous default filled in (width 0: one value a row).
luna_strides filled(luna_strides s, int heads, int n, int width) {
    const int64_t w = std::max(width, 1);
    if (s.b == 0 && s.h == 0 && s.t == 0) s = luna_strides{(int64_t)heads * n * w, (int64_t)n * w, w};
    return s;
}

// Whether no two elements of an output share an address: every dimension's stride is at
// least the extent of the dimensions with smaller strides.
bool disjoint(const luna_strides &s, int B, int heads, int n, int width) {
    struct D { int64_t stride, ext; } d[3] = {{s.b, B}, {s.h, heads}, {s.t, n}};
    std::sort(d, d + 3, [](const D &x, const D &y) { return x.stride < y.stride; });
    int64_t span = std::max(width, 1);
    for (const D &x : d) {
        if (x.ext <= 1) continue;
        if (x.stride < span) return false;
        span += (x.ext - 1) * x.stride;
    }
    return true;
}

luna_status check(const luna_delta_desc *dd) {
    if (!dd) return LUNA_ERR_INVALID_ARG;
    if (dd->B < 0 || dd->H < 0 || dd->Hk < 0 || dd->n < 0 || dd->d < 1 || dd->dv < 1) return LUNA_ERR_INVALID_ARG;
    if (dd->io != LUNA_F32 && dd->io != LUNA_BF16) return LUNA_ERR_INVALID_ARG;
    if (!isfinite(dd->scale)) return LUNA_ERR_INVALID_ARG;
    if (dd->H > 0 && (dd->Hk < 1 || dd->H % dd->Hk != 0)) return LUNA_ERR_INVALID_ARG;
    for (const luna_strides *s : {&dd->q, &dd->k, &dd->v, &dd->o, &dd->g, &dd->beta, &dd->gq, &dd->gk, &dd->gv, &dd->go,
                                  &dd->gg, &dd->gbeta})
        if (s->b < 0 || s->h < 0 || s->t < 0) return LUNA_ERR_INVALID_ARG;
    if (dd->d > kMaxD || dd->dv > kMaxD || dd->n > (1 << 24) || (int64_t)dd->B * dd->H > (1 << 24) ||
        (int64_t)dd->B * dd->H * cdiv(dd->n, kDeltaRows) >= (int64_t(1) << 31))
        return LUNA_ERR_UNSUPPORTED;
    return LUNA_OK;
}

bool empty(const luna_delta_desc *dd) { return (int64_t)dd->B * dd->H == 0; }

// Offsets of the parts of a workspace.
struct Plan {
    int m, dvp, dp;
    size_t dq = 0, dk = 0;                          // gradients of shared queries and keys, one for each head
    size_t U = 0, X = 0, before = 0, after = 0;      // CUDA-core form
    size_t K = 0, Q = 0, T = 0, P = 0, rows = 0;     // tensor-core form, in a forward pass too
    size_t Up = 0, Xp = 0, Gp = 0, Sp = 0, Rp = 0, scales = 0;  // (gradients)
    size_t fwd = 256, bwd = 256;
};

// fp32 runs on CUDA cores, bf16 on tensor cores.
bool on_tc(const luna_delta_desc *dd) { return dd->io == LUNA_BF16; }
bool whole_vectors(const luna_delta_desc *dd) { return dd->d % 8 == 0 && dd->dv % 8 == 0; }

Plan make_plan(const luna_delta_desc *dd) {
    Plan p;
    const int64_t BH = (int64_t)dd->B * dd->H;
    p.m = (int)cdiv(dd->n, kDeltaRows);
    p.dvp = (int)cdiv(dd->dv, 16) * 16;
    p.dp = dd->d <= 64 ? 64 : 128;
    size_t at = 256;
    auto take = [&](int64_t bytes) { const size_t o = at; at += (size_t)align256(bytes); return o; };
    const int64_t tile = (int64_t)kDeltaRows * kDeltaRows * 2, chunks = BH * p.m;
    if (on_tc(dd)) {
        p.rows = take(chunks * kDeltaFactors * 4);
        p.K = take((int64_t)dd->B * dd->Hk * p.m * kDeltaRows * p.dp * 2);
        p.Q = take((int64_t)dd->B * dd->Hk * p.m * kDeltaRows * p.dp * 2);
        p.T = take(chunks * 2 * tile);
        p.P = take(chunks * tile);
        p.fwd = at;
        at = p.P;
        take(chunks * 2 * tile);  // (in two planes)
        p.Up = take(chunks * p.dvp * kDeltaRows * 2);
        p.Xp = take(chunks * p.dvp * kDeltaRows * 2);
        p.Gp = take(chunks * p.dvp * kDeltaRows * 2);
        p.Sp = take(chunks * p.dvp * p.dp * 2);
        p.Rp = take((chunks + BH) * p.dvp * p.dp * 2);
        p.scales = take((chunks + BH) * (p.dvp / 16) * kDeltaScales * 4);
    } else {
        p.U = take(BH * dd->n * dd->dv * 4);
        p.X = take(BH * dd->n * dd->dv * 4);
        p.before = take(BH * (p.m + 1) * dd->d * dd->dv * 4);
        p.after = take(BH * (p.m + 1) * dd->d * dd->dv * 4);
    }
    if (dd->H != dd->Hk) {
        p.dq = take(BH * dd->n * dd->d * 4);
        p.dk = take(BH * dd->n * dd->d * 4);
    }
    p.bwd = at;
    return p;
}

// Whether rows start on 16-byte boundaries.
bool rows16(const void *p, const luna_strides &s) {
    return aligned(p, 16) && s.b % 8 == 0 && s.h % 8 == 0 && s.t % 8 == 0;
}
bool rows16(const RowView &v) { return rows16(v.p, luna_strides{v.sb, v.sh, v.st}); }

RowView view(const void *p, const luna_strides &s, int heads) { return RowView{p, s.b, s.h, s.t, heads}; }
GateView gate(const void *p, const luna_strides &s) { return GateView{p, s.b, s.h, s.t}; }

// What all passes of a call share.
DeltaArgs base(const luna_delta_desc *dd, const Plan &p, const void *g, const void *beta, const void *Q, const void *K,
               const void *V, const int32_t *lengths, void *ws) {
    DeltaArgs a{};
    a.status = static_cast<int *>(ws);
    a.q = view(Q, filled(dd->q, dd->Hk, dd->n, dd->d), dd->Hk);
    a.k = view(K, filled(dd->k, dd->Hk, dd->n, dd->d), dd->Hk);
    a.v = view(V, filled(dd->v, dd->H, dd->n, dd->dv), dd->H);
    a.g = gate(g, filled(dd->g, dd->H, dd->n, 0));
    a.b = gate(beta, filled(dd->beta, dd->H, dd->n, 0));
    a.lengths = lengths;
    a.B = dd->B; a.H = dd->H; a.n = dd->n; a.d = dd->d; a.dv = dd->dv; a.m = p.m;
    a.scale = dd->scale;
    a.dvp = p.dvp;
    return a;
}

// The tensor-core form's parts of the workspace.
void tc_parts(DeltaArgs &a, const Plan &p, char *ws, bool backward) {
    auto at = [&](size_t o) { return reinterpret_cast<__half *>(ws + o); };
    a.rows = reinterpret_cast<float *>(ws + p.rows);
    a.Kp = at(p.K); a.Qp = at(p.Q); a.Tp = at(p.T); a.Pp = at(p.P);
    a.planes = backward ? 2 : 1;
    if (!backward) return;
    a.Up = at(p.Up); a.Xp = at(p.Xp); a.Gp = at(p.Gp); a.Sp = at(p.Sp); a.Rp = at(p.Rp);
    a.scales = reinterpret_cast<float *>(ws + p.scales);
}

cudaError_t run_chain(const DeltaArgs &a, bool reverse, cudaStream_t s) {
    return a.d <= 64 ? launch_delta_chain64(a, reverse, s) : launch_delta_chain128(a, reverse, s);
}

}  // namespace

extern "C" {

luna_status luna_delta_workspace_size(const luna_delta_desc *dd, int backward, size_t *bytes) {
    if (!bytes) return LUNA_ERR_INVALID_ARG;
    const luna_status st = check(dd);
    if (st != LUNA_OK) return st;
    const Plan p = make_plan(dd);
    *bytes = empty(dd) || dd->n == 0 ? 256 : backward ? p.bwd : p.fwd;
    return LUNA_OK;
}

luna_status luna_delta_fwd(const luna_delta_desc *dd, const void *log_decay, const void *beta, const void *Q, const void *K,
                           const void *V, const int32_t *lengths, const float *S0, void *O, float *S1,
                           void *workspace, size_t ws_bytes, void *stream) {
    const luna_status st = check(dd);
    if (st != LUNA_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (empty(dd)) return LUNA_OK;
    const size_t SB = (size_t)dd->B * dd->H * dd->d * dd->dv * 4;
    if (dd->n == 0) {
        if (!S1 || S1 == S0) return LUNA_OK;
        return cuda_status(S0 ? cudaMemcpyAsync(S1, S0, SB, cudaMemcpyDeviceToDevice, s) : cudaMemsetAsync(S1, 0, SB, s));
    }
    if (!log_decay || !beta || !Q || !K || !V || !O || !workspace || !aligned(workspace, 256)) return LUNA_ERR_INVALID_ARG;
    const luna_strides so = filled(dd->o, dd->H, dd->n, dd->dv);
    if (!disjoint(so, dd->B, dd->H, dd->n, dd->dv)) return LUNA_ERR_INVALID_ARG;
    const Plan p = make_plan(dd);
    if (ws_bytes < p.fwd) return LUNA_ERR_WORKSPACE;
    DeltaArgs a = base(dd, p, log_decay, beta, Q, K, V, lengths, workspace);
    a.o = O; a.ob = so.b; a.oh = so.h; a.ot = so.t;
    a.S0 = S0;
    a.S1 = S1;
    if (!on_tc(dd)) return cuda_status(launch_delta_rows(a, false, s));
    a.vec = whole_vectors(dd) && rows16(a.q) && rows16(a.k) && rows16(a.v) && rows16(O, so);
    tc_parts(a, p, static_cast<char *>(workspace), false);
    if (launch_delta_prepare(a, s) != cudaSuccess) return LUNA_ERR_CUDA;
    return cuda_status(run_chain(a, false, s));
}

luna_status luna_delta_bwd(const luna_delta_desc *dd, const void *log_decay, const void *beta, const void *Q, const void *K,
                           const void *V, const void *dO, const int32_t *lengths, const float *S0, const float *dS1,
                           void *dQ, void *dK, void *dV, void *dlog_decay, void *dbeta, float *dS0, void *workspace,
                           size_t ws_bytes, void *stream) {
    const luna_status st = check(dd);
    if (st != LUNA_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (empty(dd)) return LUNA_OK;
    const size_t SB = (size_t)dd->B * dd->H * dd->d * dd->dv * 4;
    if (dd->n == 0) {
        if (!dS0 || dS0 == dS1) return LUNA_OK;
        return cuda_status(dS1 ? cudaMemcpyAsync(dS0, dS1, SB, cudaMemcpyDeviceToDevice, s)
                               : cudaMemsetAsync(dS0, 0, SB, s));
    }
    if (!log_decay || !beta || !Q || !K || !V || !dO || !dQ || !dK || !dV || !dlog_decay || !dbeta || !workspace ||
        !aligned(workspace, 256))
        return LUNA_ERR_INVALID_ARG;
    const int B = dd->B, H = dd->H, Hk = dd->Hk, n = dd->n, d = dd->d, dv = dd->dv;
    const luna_strides gq = filled(dd->gq, Hk, n, d), gk = filled(dd->gk, Hk, n, d), gv = filled(dd->gv, H, n, dv);
    const luna_strides gg = filled(dd->gg, H, n, 0), gb = filled(dd->gbeta, H, n, 0);
    if (!disjoint(gq, B, Hk, n, d) || !disjoint(gk, B, Hk, n, d) || !disjoint(gv, B, H, n, dv) ||
        !disjoint(gg, B, H, n, 0) || !disjoint(gb, B, H, n, 0))
        return LUNA_ERR_INVALID_ARG;
    const Plan p = make_plan(dd);
    if (ws_bytes < p.bwd) return LUNA_ERR_WORKSPACE;
    char *ws = static_cast<char *>(workspace);
    const bool shared = H != Hk;

    DeltaArgs a = base(dd, p, log_decay, beta, Q, K, V, lengths, workspace);
    a.go = view(dO, filled(dd->go, H, n, dv), H);
    a.S0 = S0;
    a.dS1 = dS1;
    a.U = reinterpret_cast<float *>(ws + p.U);
    a.X = reinterpret_cast<float *>(ws + p.X);
    a.before = reinterpret_cast<float *>(ws + p.before);
    a.after = reinterpret_cast<float *>(ws + p.after);
    float *part_q = reinterpret_cast<float *>(ws + p.dq), *part_k = reinterpret_cast<float *>(ws + p.dk);
    a.dq = shared ? (void *)part_q : dQ;
    a.dk = shared ? (void *)part_k : dK;
    const luna_strides part{(int64_t)H * n * d, (int64_t)n * d, d};
    const luna_strides &sq = shared ? part : gq, &sk = shared ? part : gk;
    a.dqb = sq.b; a.dqh = sq.h; a.dqt = sq.t;
    a.dkb = sk.b; a.dkh = sk.h; a.dkt = sk.t;
    a.dg = GateOut{dlog_decay, gg.b, gg.h, gg.t};
    a.db = GateOut{dbeta, gb.b, gb.h, gb.t};

    const bool tc = on_tc(dd);
    a.vec = whole_vectors(dd) && rows16(a.q) && rows16(a.k) && rows16(a.v) && rows16(a.go) && rows16(dV, gv) &&
            (shared || (rows16(dQ, gq) && rows16(dK, gk)));
    cudaError_t e = cudaSuccess;
    if (tc) {
        tc_parts(a, p, ws, true);
        e = launch_delta_prepare(a, s);
        if (e == cudaSuccess) e = run_chain(a, false, s);
    } else {
        e = launch_delta_rows(a, false, s);
    }
    if (e != cudaSuccess) return LUNA_ERR_CUDA;
    DeltaArgs r = a;
    r.o = dV; r.ob = gv.b; r.oh = gv.h; r.ot = gv.t;
    r.dS0 = dS0;
    e = tc ? run_chain(r, true, s) : launch_delta_rows(r, true, s);
    if (e != cudaSuccess) return LUNA_ERR_CUDA;
    const luna_dtype out = shared ? LUNA_F32 : dd->io;
    e = tc ? launch_delta_grad_tc(a, out, s) : launch_delta_grad(a, s);
    if (e != cudaSuccess) return LUNA_ERR_CUDA;
    if (!shared) return LUNA_OK;
    e = launch_decay_group_sum(part_q, B, H, H / Hk, n, d, dQ, gq.b, gq.h, gq.t, dd->io, s);
    if (e != cudaSuccess) return LUNA_ERR_CUDA;
    return cuda_status(launch_decay_group_sum(part_k, B, H, H / Hk, n, d, dK, gk.b, gk.h, gk.t, dd->io, s));
}

luna_status luna_delta_step(const luna_delta_desc *dd, const void *log_decay, const void *beta, const void *q, const void *k,
                            const void *v, const int32_t *slots, int nslots, float *S, void *o, void *stream) {
    const luna_status st = check(dd);
    if (st != LUNA_OK) return st;
    if (nslots < 0 || (!slots && nslots < dd->B)) return LUNA_ERR_INVALID_ARG;
    if (empty(dd)) return LUNA_OK;
    if (!log_decay || !beta || !q || !k || !v || !o || (nslots > 0 && !S)) return LUNA_ERR_INVALID_ARG;
    const luna_strides sq = filled(dd->q, dd->Hk, 1, dd->d), sk = filled(dd->k, dd->Hk, 1, dd->d);
    const luna_strides sv = filled(dd->v, dd->H, 1, dd->dv), so = filled(dd->o, dd->H, 1, dd->dv);
    if (!disjoint(so, dd->B, dd->H, 1, dd->dv)) return LUNA_ERR_INVALID_ARG;
    DeltaStep a{q, k, v, o, sq.b, sq.h, sk.b, sk.h, sv.b, sv.h, so.b, so.h,
                gate(log_decay, filled(dd->g, dd->H, 1, 0)), gate(beta, filled(dd->beta, dd->H, 1, 0)),
                slots, S, nslots, dd->B, dd->H, dd->Hk, dd->d, dd->dv, dd->scale};
    return cuda_status(launch_delta_step(a, dd->io, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
