// Beam search over recurrent states: the best continuations of every sequence, and the states that follow them.
#include <math.h>

#include <algorithm>

#include "luna_common.cuh"
#include "luna_prof.cuh"

namespace luna {
int tc_sm_count();

namespace {

constexpr int kMaxBeams = 32;                  // a warp's lanes
constexpr int kThreads = 256;
// values of a piece that a thread holds: of many rows 64 bytes, of few 8 values
template <typename T> constexpr int kPer = 64 / (int)sizeof(T);
constexpr int kFew = 8;

// Values as integers in the same order; larger is better.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) {
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ uint64_t ordered(double x) {
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    return u >> 63 ? ~u : u | (uint64_t(1) << 63);
}
__device__ __forceinline__ double unordered(uint64_t u) {
    return __longlong_as_double((long long)(u >> 63 ? u & ~(uint64_t(1) << 63) : ~u));
}

// A candidate of one row: its logit, and at equal logits the lower token first.  0: none.
struct RowKey {
    uint64_t v = 0;
    __device__ bool over(const RowKey &o) const { return v > o.v; }
    __device__ RowKey lane(int l) const { return RowKey{__shfl_sync(0xffffffffu, v, l)}; }
};
// A candidate of a sequence: its score, and at equal scores the lower beam, then the lower token first.  v = 0: none.
struct SeqKey {
    uint64_t v = 0;
    uint32_t i = 0;  // ~(beam * V + token)
    __device__ bool over(const SeqKey &o) const { return (v > o.v) | ((v == o.v) & (i > o.i)); }
    __device__ SeqKey lane(int l) const { return SeqKey{__shfl_sync(0xffffffffu, v, l), __shfl_sync(0xffffffffu, i, l)}; }
};

// Exchanges of a warp's 32 candidates over lanes w apart, w = from, from / 2, .. 1: the better one goes to the lower lane
// where `down`.
template <typename Key>
__device__ __forceinline__ void exchange(Key &key, int from, bool down) {
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int w = 16; w > 0; w /= 2) {
        if (w > from) continue;
        const Key other = key.lane(lane ^ w);
        const bool take = other.over(key) == (((lane & w) == 0) == down);
        key.v = take ? other.v : key.v;
        if constexpr (sizeof(Key) > 8) key.i = take ? other.i : key.i;
    }
}
// a warp's candidates in order, the best in lane 0
template <typename Key>
__device__ __forceinline__ void sort_warp(Key &key) {
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int size = 2; size <= 32; size *= 2) exchange(key, size / 2, (lane & size) == 0 || size == 32);
}
// The best 32 of two ordered lists, in order: lane by lane the better of the one and of the other from its end, which
// are all that stay, and rise and fall once.
template <typename Key>
__device__ __forceinline__ void merge_warp(Key &key, const Key &from_end) {
    const bool take = from_end.over(key);
    key.v = take ? from_end.v : key.v;
    if constexpr (sizeof(Key) > 8) key.i = take ? from_end.i : key.i;
    exchange(key, 16, true);
}
// The best 32 of the block's candidates, given as the warps' ordered lists: in list[0..31] and in warp 0's lanes.  All
// threads call it; `list` may be written again after a barrier.
template <typename Key>
__device__ __forceinline__ void join_warps(Key &key, Key *list) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    list[threadIdx.x] = key;
    __syncthreads();
#pragma unroll
    for (int w = kThreads / 64; w > 0; w /= 2) {
        if (warp < w) {
            merge_warp(key, list[(warp + w) * 32 + 31 - lane]);
            list[threadIdx.x] = key;  // (in the next round read by another warp than it is written by)
        }
        __syncthreads();
    }
}
// The best 32 of candidate(0..count - 1), as join_warps
template <typename Key, typename F>
__device__ __forceinline__ void best_of(int count, F candidate, Key &key, Key *list) {
    const int lane = threadIdx.x % 32;
    key = Key{};
    for (int at = threadIdx.x - lane; at < count; at += kThreads) {
        Key next = at + lane < count ? candidate(at + lane) : Key{};
        sort_warp(next);
        merge_warp(key, next.lane(31 - lane));
    }
    join_warps(key, list);
}

// 2^x to 2^-22 of itself
__device__ __forceinline__ float power2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;

struct BeamArgs {
    const void *logits;
    int64_t ld;
    const float *scores;
    const uint8_t *done;
    float *scores_out;
    int32_t *tokens, *parents;
    uint8_t *done_out;
    int B, K, V, end, S;  // S: pieces of a row
    uint64_t *keys;       // [B K][S][K]
    float2 *stats;        // [B K][S]: maximum, sum of exp over it
};

// One part of one row: its maximum, its sum of exponentials and its K best values, in one reading.  A thread holds PER
// values of a piece of 256 PER.  Of the first piece only what reaches the K-th best of the threads' largest is kept
// (there are K as good, and at most K threads have some), of the others too; a few dozen values are sorted at the end,
// or before, where the kept ones run out of room (values that rise along a row).
// Few rows come in pieces of 2048 values, so that more SMs share them.  The next piece is on its way to shared memory
// meanwhile, each thread's own part of it.  Which thread takes which tokens does not hang on where the row starts, so that rows of
// equal values have equal sums and their beams are ordered by their place: where a row does not start on a 16-byte
// boundary, a thread's values lie in two vectors, the second of which its neighbour has.  34 us for 256 rows of 128256 bf16 values (1.8 TB/s), 38 % of the
// issue slots used: a piece's instructions are some 13 us of it, the rest waits at the sorts of a block's first piece and
// of its end, at barriers, and for blocks (512 where the SMs hold 608); 8 us for 4 rows of 50257, the chain of one piece.
template <typename T, int PER>
__global__ void __launch_bounds__(kThreads, PER == kFew ? 1 : 4) k_beam_rows(BeamArgs a) {
    constexpr int VEC = 16 / sizeof(T), NV = PER / VEC, PIECE = kThreads * PER;
    constexpr int POOL = kMaxBeams * (PER + 1) + 512;  // (of a piece at most kMaxBeams threads' after the block's best are known)
    __shared__ RowKey list[kThreads], pool[POOL];
    __shared__ int count;
    __shared__ float smax[kThreads / 32], ssum[kThreads / 32];
    const int tid = threadIdx.x, row = blockIdx.y, part = blockIdx.x;
    if (a.done && a.done[row]) return;
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    const int off = (int)((reinterpret_cast<uintptr_t>(x) % 16) / sizeof(T));  // of the row from the 16-byte boundary before it
    const int pieces = (a.V + PIECE - 1) / PIECE;
    const int first = (int)((int64_t)pieces * part / a.S), last = (int)((int64_t)pieces * (part + 1) / a.S);
    float top = -INFINITY, sum = 0.0f, rest = 0.0f;  // rest: what roundings of the sum left
    RowKey bar;  // K candidates are at least as good (none: v = 0)
    auto floor_of = [](const RowKey &k) { return k.v ? unordered((uint32_t)(k.v >> 32)) : -INFINITY; };
    extern __shared__ uint4 ahead[];  // [2][NV][kThreads], behind them [2][NV][kThreads / 32]
    uint4 *const beside = ahead + 2 * NV * kThreads;  // what comes behind a warp's vectors
    auto first_of = [&](int piece, int j) { return (piece * (PIECE / VEC) + j * kThreads + tid) * VEC; };  // every 256 VEC tokens
    auto fetch_one = [&](uint4 *to, int t) {  // from a 16-byte boundary, where all of it is the row's
        if (t >= 0 && t + VEC <= a.V)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(x + t) : "memory");
    };
    auto fetch = [&](int piece) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int t = first_of(piece, j) - off, at = ((piece - first) & 1) * NV + j;
            fetch_one(&ahead[at * kThreads + tid], t);
            if (off && tid % 32 == 31) fetch_one(&beside[at * (kThreads / 32) + tid / 32], t + VEC);
        }
    };
    if (first < last) fetch(first);
    asm volatile("cp.async.commit_group;" ::: "memory");
    for (int piece = first; piece < last; ++piece) {
        if (piece + 1 < last) fetch(piece + 1);
        asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 1;" ::: "memory");
        float val[PER];
        auto token = [&](int i) { return first_of(piece, i / VEC) + i % VEC; };
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int t = token(j * VEC), at = ((piece - first) & 1) * NV + j;
            uint4 w = ahead[at * kThreads + tid];
            if (off) {  // (the same for the whole block) the values from `off` on, of two vectors
                uint32_t u[8] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) u[4 + i] = __shfl_down_sync(0xffffffffu, u[i], 1);
                if (tid % 32 == 31) {
                    const uint4 next = beside[at * (kThreads / 32) + tid / 32];
                    u[4] = next.x; u[5] = next.y; u[6] = next.z; u[7] = next.w;
                }
                const int bytes = off * (int)sizeof(T);
#pragma unroll
                for (int i = 0; i < 6; ++i) u[i] = bytes & 8 ? u[i + 2] : u[i];
#pragma unroll
                for (int i = 0; i < 5; ++i) u[i] = bytes & 4 ? u[i + 1] : u[i];
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = __funnelshift_r(u[i], u[i + 1], bytes % 4 * 8);
                w = make_uint4(u[0], u[1], u[2], u[3]);
            }
            if (off ? t >= off && t - off + 2 * VEC <= a.V : t + VEC <= a.V) {
                T e[VEC];
                memcpy(e, &w, 16);
#pragma unroll
                for (int i = 0; i < VEC; ++i) val[j * VEC + i] = io_load(&e[i]);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    val[j * VEC + i] = t + i < a.V ? io_load(x + t + i) : -INFINITY;
            }
        }
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < PER; ++i) m = fmaxf(m, val[i]);
        const float now = fmaxf(top, m), shift = now == -INFINITY ? 0.0f : now;
        float part_sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < PER; ++i) part_sum[i % 4] += power2((val[i] - shift) * kLog2e);
        // one addition to the sum a piece, and its rounding kept: beside a large value thousands of small ones would be cut off
        const float scale = power2((top - shift) * kLog2e), more = (part_sum[0] + part_sum[1]) + (part_sum[2] + part_sum[3]);
        const float was = sum * scale, total = was + more, added = total - was;
        rest = fmaf(rest, scale, (was - (total - added)) + (more - added));
        sum = total;
        top = now;
        // the key of a value, or none: behind the row's ends, or a NaN (k_beam_join sees by the sum that such a row has no scores)
        auto key = [&](int i, float v) {
            const int t = token(i);
            RowKey k;
            if (t < a.V && v == v) k.v = (uint64_t)ordered(v + 0.0f) << 32 | (uint32_t)~t;  // (-0 is 0)
            return k;
        };
        auto best_of_thread = [&]() {  // the first of its largest (tokens rise with i) that is a token's
            RowKey k;
            int at = -1;
#pragma unroll
            for (int i = PER - 1; i >= 0; --i)
                if (val[i] == m && token(i) < a.V) at = i;
            if (at >= 0) k = key(at, m);
            return k;
        };
        // the K-th best of the threads' largest: K candidates are as good, and no more than K threads have some
        auto threshold = [&]() {
            RowKey k = best_of_thread();
            sort_warp(k);
            join_warps(k, list);
            return list[a.K - 1];
        };
        if (piece == first) {
            if (tid == 0) count = 0;
            bar = threshold();  // (none where fewer than K threads have a value)
        } else {
            const int had = count;  // (before the barrier: behind it faster warps add to it)
            const int hits = __syncthreads_count(m >= floor_of(bar));
            if (hits == 0) continue;
            if (had + hits * PER > POOL) {
                RowKey k;
                best_of(had, [&](int i) { return pool[i]; }, k, list);
                const RowKey kth = list[a.K - 1];
                if (tid < a.K) pool[tid] = k;
                __syncthreads();
                if (tid == 0) count = a.K;  // (what is none among them stays so)
                const RowKey least = threshold();
                bar = least.over(kth) ? least : kth;
            }
        }
        const float lowest = floor_of(bar);
        uint32_t mask = 0;
        if (m >= lowest) {
#pragma unroll
            for (int i = 0; i < PER; ++i) mask |= val[i] >= lowest ? 1u << i : 0u;
        }
        while (mask) {  // (few: their values are read again)
            const int i = __ffs(mask) - 1, t = token(i);
            mask &= mask - 1;
            if (t >= a.V) continue;
            const RowKey c = key(i, io_load(x + t));
            if (c.v && !bar.over(c)) pool[atomicAdd(&count, 1)] = c;
        }
        __syncthreads();
    }
    RowKey best;
    best_of(last > first ? count : 0, [&](int i) { return pool[i]; }, best, list);  // (fewer pieces than parts)
    const int64_t at = (int64_t)row * a.S + part;
    if (tid < a.K) a.keys[at * a.K + tid] = best.v;
    float m = top;
#pragma unroll
    for (int w = 16; w > 0; w /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
    float s = (sum + rest) * power2((top - (m == -INFINITY ? 0.0f : m)) * kLog2e);
#pragma unroll
    for (int w = 16; w > 0; w /= 2) s += __shfl_xor_sync(0xffffffffu, s, w);
    if (tid % 32 == 0) { smax[tid / 32] = m; ssum[tid / 32] = s; }
    __syncthreads();
    if (tid == 0) {
        float all = 0.0f;
        m = smax[0];
        for (int w = 1; w < kThreads / 32; ++w) m = fmaxf(m, smax[w]);
        const float b = m == -INFINITY ? 0.0f : m;
        for (int w = 0; w < kThreads / 32; ++w) all += ssum[w] * power2((smax[w] - b) * kLog2e);
        a.stats[at] = make_float2(m, all);
    }
}

// The K best of a sequence from its rows' candidates.  Scores are in 64 bits, so that two of one beam come in the order of
// their logits; the logarithm is that of a sum in fp32, so that two of different beams may come in either order where they
// are nearer than some 1e-6.  64-bit arithmetic is scarce here, so one warp takes the logarithms of all rows at once and a
// candidate costs two sums (exponentials and logarithms by a warp a row took 16 to 37 us, so 9 to 17).  One block a
// sequence: K S K candidates, which its warps sort 32 at a time.
__global__ void __launch_bounds__(kThreads) k_beam_join(BeamArgs a) {
    __shared__ SeqKey list[kThreads];
    __shared__ double base[kMaxBeams];  // score - log sum exp(logit - most)
    __shared__ float score[kMaxBeams], most[kMaxBeams], sums[kMaxBeams];
    __shared__ uint8_t done[kMaxBeams], dead[kMaxBeams];  // dead: no candidate of its has a score
    const int tid = threadIdx.x, b = blockIdx.x, K = a.K, S = a.S;
    for (int k = tid / 32; k < K; k += kThreads / 32) {  // a warp a row
        const int row = b * K + k, lane = tid % 32;
        const bool over = a.done && a.done[row];
        float m = -INFINITY, sum = 0.0f;
        if (!over) {
            for (int s = lane; s < S; s += 32) m = fmaxf(m, a.stats[(int64_t)row * S + s].x);
#pragma unroll
            for (int w = 16; w > 0; w /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
            for (int s = lane; s < S; s += 32) {
                const float2 p = a.stats[(int64_t)row * S + s];
                sum += p.x == -INFINITY ? p.y : p.y * power2((p.x - m) * kLog2e);
            }
#pragma unroll
            for (int w = 16; w > 0; w /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        }
        if (lane == 0) {
            done[k] = over;
            score[k] = a.scores[row];
            most[k] = m;
            sums[k] = sum;
        }
    }
    __syncthreads();
    if (tid < K) {
        const double x = (double)score[tid] - log((double)sums[tid]);
        base[tid] = x;
        dead[tid] = !done[tid] && !(isfinite(x) && isfinite(most[tid]));
    }
    __syncthreads();
    const int N = K * S * K;
    auto candidate = [&](int n) {
        const int k = n / (S * K), j = n - k * (S * K);
        SeqKey c;
        int token;
        if (done[k] || dead[k]) {
            // an ended beam goes on as itself; what no score can be given to comes behind everything, by its place
            if (j >= K) return c;
            token = done[k] ? (j == 0 ? a.end : j - (j <= a.end)) : j;
            if (token >= a.V) return c;
            c.v = ordered(done[k] && j == 0 && score[k] == score[k] ? (double)(score[k] + 0.0f) : -(double)INFINITY);
        } else {
            const uint64_t key = a.keys[(int64_t)b * N + n];
            if (!key) return c;
            token = (int)~(uint32_t)key;
            // (the largest logit comes off first: a row may be masked by its type's lowest value throughout)
            const double v = base[k] + ((double)unordered((uint32_t)(key >> 32)) - (double)most[k]);
            c.v = __double_as_longlong(v) << 1 == 0 ? uint64_t(1) << 63 : ordered(v);  // (-0 is 0)
        }
        c.i = ~(uint32_t)(k * a.V + token);
        return c;
    };
    SeqKey best;
    best_of(N, candidate, best, list);
    if (tid < K) {
        const uint32_t at = ~best.i;
        const int parent = (int)(at / a.V), token = (int)(at - (uint32_t)parent * a.V);
        a.scores_out[b * K + tid] = (float)unordered(best.v);
        a.tokens[b * K + tid] = token;
        a.parents[b * K + tid] = parent;
        if (a.done_out) a.done_out[b * K + tid] = done[parent] || token == a.end;
    }
}

// ---------------------------------------------------------------------------
// The states follow their beams: the first child of a beam keeps its slot, further children get copies in the slots
// of beams without a child, so that sources and destinations of the copies never meet and each copied state moves
// once.  A block works out the K beams of its sequence in one warp and copies its part of every state that moves;
// bound by the bytes of those (50 us for 284 MB read and written, 5.7 TB/s).

constexpr int kCopyThreads = 256, kCopyVecs = 4;

template <typename V>
__global__ void __launch_bounds__(kCopyThreads) k_beam_reorder(const int32_t *parents, const int32_t *slots, int K,
                                                               int nslots, char *pool, int64_t slot_bytes, int32_t *out) {
    __shared__ int from[kMaxBeams], to[kMaxBeams], moves;
    const int tid = threadIdx.x, b = blockIdx.y;
    if (tid < 32) {
        const bool in = tid < K;
        int p = in ? parents[b * K + tid] : -1;
        if (p < 0 || p >= K) p = -1;
        const unsigned same = __match_any_sync(0xffffffffu, p), below = (1u << tid) - 1;
        const bool keeps = p >= 0 && (same & below) == 0;
        const unsigned kept = __reduce_or_sync(0xffffffffu, p >= 0 ? 1u << p : 0u);
        const unsigned others = __ballot_sync(0xffffffffu, in && !keeps);
        const unsigned beams = K == 32 ? 0xffffffffu : (1u << K) - 1;
        int place = p;
        if (in && !keeps) place = __fns(beams & ~kept, 0, __popc(others & below) + 1);
        const int slot = in ? slots[b * K + place] : -1;
        if (in && blockIdx.x == 0) out[b * K + tid] = slot;
        const int src = in && p >= 0 ? slots[b * K + p] : -1;
        const bool copies = in && !keeps && p >= 0 && src >= 0 && src < nslots && slot >= 0 && slot < nslots;
        const unsigned all = __ballot_sync(0xffffffffu, copies);
        if (copies) {
            from[__popc(all & below)] = src;
            to[__popc(all & below)] = slot;
        }
        if (tid == 0) moves = __popc(all);
    }
    __syncthreads();
    const int64_t vecs = slot_bytes / (int64_t)sizeof(V), step = (int64_t)gridDim.x * kCopyThreads * kCopyVecs;
    for (int64_t v0 = (int64_t)blockIdx.x * kCopyThreads * kCopyVecs + tid; v0 < vecs; v0 += step)
        for (int c = 0; c < moves; ++c) {
            const V *src = reinterpret_cast<const V *>(pool + (int64_t)from[c] * slot_bytes);
            V *dst = reinterpret_cast<V *>(pool + (int64_t)to[c] * slot_bytes);
            V w[kCopyVecs];
#pragma unroll
            for (int i = 0; i < kCopyVecs; ++i)
                if (v0 + i * kCopyThreads < vecs) w[i] = src[v0 + i * kCopyThreads];
#pragma unroll
            for (int i = 0; i < kCopyVecs; ++i)
                if (v0 + i * kCopyThreads < vecs) dst[v0 + i * kCopyThreads] = w[i];
        }
}

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

luna_status check(const luna_beam_desc *bd) {
    if (!bd || bd->B < 0 || bd->K < 1 || bd->V < 0) return LUNA_ERR_INVALID_ARG;
    if (bd->io != LUNA_F32 && bd->io != LUNA_BF16) return LUNA_ERR_INVALID_ARG;
    if (bd->end < -1 || (bd->V > 0 && bd->end >= bd->V) || bd->ld < 0 || (bd->ld > 0 && bd->ld < bd->V))
        return LUNA_ERR_INVALID_ARG;
    if (bd->K > kMaxBeams || bd->V > (1 << 24) || (int64_t)bd->B * bd->K > 65535) return LUNA_ERR_UNSUPPORTED;
    return LUNA_OK;
}

// How rows are cut: the values that a thread holds of a piece, and the parts of a row.  Many rows: large pieces and as
// many blocks as the SMs hold at four each; few, whose large pieces leave most SMs without one: small pieces.
struct Cut {
    int per, parts;
};
Cut cut(const luna_beam_desc *bd) {
    const int64_t rows = std::max<int64_t>(1, (int64_t)bd->B * bd->K), sms = tc_sm_count(), V = bd->V;
    const int large = bd->io == LUNA_F32 ? kPer<float> : kPer<__nv_bfloat16>;
    const int per = rows * cdiv(V, kThreads * large) < sms ? kFew : large;
    const int64_t most = std::max<int64_t>(1, 4 * sms / rows);
    return Cut{per, (int)std::min(cdiv(V, kThreads * per), most)};
}

template <typename T, int PER>
cudaError_t launch_rows(const BeamArgs &a, cudaStream_t s) {
    const size_t ahead = 2 * sizeof(T) * PER * (kThreads + kThreads / 32);
    cudaError_t e = cudaFuncSetAttribute(k_beam_rows<T, PER>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ahead);
    if (e != cudaSuccess) return e;
    LUNA_LAUNCH("beam_rows", (k_beam_rows<T, PER>), dim3((unsigned)a.S, (unsigned)(a.B * a.K)), kThreads, ahead, s, a);
    return cudaGetLastError();
}

size_t workspace(const luna_beam_desc *bd) {
    const int64_t rows = (int64_t)bd->B * bd->K, S = cut(bd).parts;
    return (size_t)(256 + align256(rows * S * bd->K * 8) + align256(rows * S * 8));
}

}  // namespace
}  // namespace luna

using namespace luna;

extern "C" {

luna_status luna_beam_workspace_size(const luna_beam_desc *bd, size_t *bytes) {
    if (!bytes) return LUNA_ERR_INVALID_ARG;
    const luna_status st = check(bd);
    if (st != LUNA_OK) return st;
    *bytes = bd->V > 0 ? workspace(bd) : 256;
    return LUNA_OK;
}

luna_status luna_beam_select(const luna_beam_desc *bd, const void *logits, const float *scores, const uint8_t *done,
                             float *scores_out, int32_t *tokens, int32_t *parents, uint8_t *done_out, void *ws,
                             size_t ws_bytes, void *stream) {
    const luna_status st = check(bd);
    if (st != LUNA_OK) return st;
    if (bd->V < 1 || (bd->end < 0 && (done || done_out))) return LUNA_ERR_INVALID_ARG;
    if (bd->B == 0) return LUNA_OK;
    if (!logits || !scores || !scores_out || !tokens || !parents || !ws || reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        return LUNA_ERR_INVALID_ARG;
    if (ws_bytes < workspace(bd)) return LUNA_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Cut how = cut(bd);
    BeamArgs a{logits, bd->ld ? bd->ld : bd->V, scores, done, scores_out, tokens, parents, done_out,
               bd->B, bd->K, bd->V, bd->end, how.parts};
    a.keys = reinterpret_cast<uint64_t *>(static_cast<char *>(ws) + 256);
    a.stats = reinterpret_cast<float2 *>(static_cast<char *>(ws) + 256 + align256((int64_t)bd->B * bd->K * a.S * bd->K * 8));
    const bool few = how.per == kFew;
    cudaError_t e;
    if (bd->io == LUNA_F32)
        e = few ? launch_rows<float, kFew>(a, s) : launch_rows<float, kPer<float>>(a, s);
    else
        e = few ? launch_rows<__nv_bfloat16, kFew>(a, s) : launch_rows<__nv_bfloat16, kPer<__nv_bfloat16>>(a, s);
    if (e != cudaSuccess) return LUNA_ERR_CUDA;
    LUNA_LAUNCH("beam_join", k_beam_join, (unsigned)bd->B, kThreads, 0, s, a);
    return cudaGetLastError() == cudaSuccess ? LUNA_OK : LUNA_ERR_CUDA;
}

luna_status luna_beam_reorder(const luna_beam_desc *bd, const int32_t *parents, const int32_t *slots, int nslots,
                              void *pool, size_t slot_bytes, int32_t *new_slots, void *stream) {
    const luna_status st = check(bd);
    if (st != LUNA_OK) return st;
    if (nslots < 0 || slot_bytes > (size_t(1) << 40)) return LUNA_ERR_INVALID_ARG;
    if (bd->B == 0) return LUNA_OK;
    if (!parents || !slots || !new_slots || new_slots == slots || new_slots == parents || (slot_bytes > 0 && nslots > 0 && !pool)) return LUNA_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const uintptr_t at = reinterpret_cast<uintptr_t>(pool) | slot_bytes;
    const int vec = at % 16 == 0 ? 16 : at % 4 == 0 ? 4 : 1;
    const int64_t blocks = cdiv((int64_t)slot_bytes, (int64_t)vec * kCopyThreads * kCopyVecs);
    const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>(blocks, 4096)), (unsigned)bd->B);
    const int n = slot_bytes > 0 ? nslots : 0;
    char *p = static_cast<char *>(pool);
    if (vec == 16)
        LUNA_LAUNCH("beam_reorder", k_beam_reorder<uint4>, grid, kCopyThreads, 0, s, parents, slots, bd->K, n, p, (int64_t)slot_bytes, new_slots);
    else if (vec == 4)
        LUNA_LAUNCH("beam_reorder", k_beam_reorder<uint32_t>, grid, kCopyThreads, 0, s, parents, slots, bd->K, n, p, (int64_t)slot_bytes, new_slots);
    else
        LUNA_LAUNCH("beam_reorder", k_beam_reorder<uint8_t>, grid, kCopyThreads, 0, s, parents, slots, bd->K, n, p, (int64_t)slot_bytes, new_slots);
    return cudaGetLastError() == cudaSuccess ? LUNA_OK : LUNA_ERR_CUDA;
}

}  // extern "C"
