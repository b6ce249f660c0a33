// What is answered with a row of logits x[0..V): log probabilities of given tokens, the entropy, the best alternatives; and
// the gradient of the first two.  With m = max x, S = sum exp(x - m):
//     log p(v) = (x_v - m) - log S,   H = log S - sum exp(x - m) (x - m) / S,
//     dx_v = sum of g_t over ids t equal to v - p_v * (sum of g_t + g_H * (log p_v + H)).
// m and log S are kept apart: their sum, the usual normaliser, would round away 1e-6 of every probability.
//
// Forward: one pass over the logits.  A lane keeps a reference r (an element of its own, at most 8 below its maximum), the
// sums of exp(x - r) and exp(x - r)(x - r), and its largest element; 16 bytes are loaded per lane and step, rows may start at
// any element (what lies before the first and behind the last whole 16 bytes is done one element per lane).  A logit of -inf
// adds nothing (its difference is cut at -200, whose exponential is 0 in fp32); NaN and +inf make the sum NaN, which is
// looked at once at the end.
// Alternatives cost the pass only the lanes' maxima.  At its end the lanes are folded to 64 groups, whose n-th largest
// maximum tau is at most the n-th largest logit: only the few lanes that hold something of at least tau read their own
// elements again, and sorted lists of 64 per wavefront, one entry per lane, take in what passes.  The order is by logit and
// then by id, so the result does not depend on which wavefront saw what.
// Few rows are cut into parts, one workgroup each, which a second launch joins.
#include <float.h>
#include <limits.h>

#include "../../include/specee.h"
#include "device_utils.h"
#include "kernels.h"

namespace specee {

namespace {

constexpr int kT = 512;  // threads of a workgroup
constexpr int kWaves = kT / kWave;
constexpr int kUnroll = 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.f;   // how far a lane's reference may lie below its maximum
constexpr float kFloor = -200.f;
constexpr int kMaxParts = 16;  // of a row

template <typename E>
struct Granule {  // 16 bytes of logits
    static constexpr int n = 16 / sizeof(E);
    E v[n] __attribute__((aligned(16)));
};

template <typename E>
__device__ __forceinline__ Granule<E> load_granule(const E *p) {
    Granule<E> g;
    *reinterpret_cast<uintx4 *>(&g) = *reinterpret_cast<const uintx4 *>(p);
    return g;
}

// A row: `head` elements, then `whole` granules at 16-byte boundaries, then the rest
template <typename E>
struct RowView {
    const E *p;
    int head, whole, tail;
    __device__ RowView(const E *row, int V) : p(row) {
        head = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(E);
        head = head < V ? head : V;
        whole = (V - head) / Granule<E>::n;
        tail = V - head - whole * Granule<E>::n;
    }
    __device__ int index(int g) const { return head + g * Granule<E>::n; }
};

struct LaneSum {
    float r, s, sx;  // reference, sum of exp(x - r), sum of exp(x - r)(x - r)
    float best;
    int at;  // granule of best
};

__device__ __forceinline__ void raise(LaneSum &a, float c) {
    if (c > a.r + kSlack) {
        if (a.s > 0.f) {
            const float d = a.r - c, f = exp2f(d * kLog2e);
            a.sx = f > 0.f ? (a.sx + a.s * d) * f : 0.f;
            a.s *= f;
        }
        a.r = c;
    }
}

__device__ __forceinline__ void add(LaneSum &a, float x) {
    const float t = x - a.r, e = __builtin_amdgcn_exp2f(t * kLog2e);
    a.s += e;
    a.sx = fmaf(e, fmaxf(t, kFloor), a.sx);
}

template <typename E>
__device__ __forceinline__ void take(LaneSum &a, const Granule<E> &g, int at) {
    float c = (float)g.v[0];
#pragma unroll
    for (int j = 1; j < Granule<E>::n; ++j) c = fmaxf(c, (float)g.v[j]);
    raise(a, c);
#pragma unroll
    for (int j = 0; j < Granule<E>::n; ++j) add(a, (float)g.v[j]);
    if (c > a.best) {
        a.best = c;
        a.at = at;
    }
}

// Joins sums (r, s, sx) of which each may be empty (s == 0) into one about M >= every r
__device__ __forceinline__ void shift(float r, float &s, float &sx, float M) {
    if (s == 0.f) {
        sx = 0.f;
        return;
    }
    const float d = fmaxf(r - M, kFloor), f = exp2f(d * kLog2e);
    sx = (sx + s * d) * f;
    s *= f;
}

__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_f32<kDppXor1>(v));
    v = fmaxf(v, dpp_f32<kDppXor2>(v));
    v = fmaxf(v, dpp_f32<kDppHalfMirror>(v));
    v = fmaxf(v, dpp_f32<kDppMirror>(v));
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    return fmaxf(v, __shfl_xor(v, 32, kWave));
}

// What a row's sums mean.  NaN or +inf among the logits: everything NaN; nothing above -inf: nothing has a probability.
struct RowStats {
    float m, log_sum, entropy;
    bool bad, empty;
    __device__ RowStats(float M, float s, float sx) {
        bad = !(s == s);
        empty = s == 0.f;
        const float nan = quiet_nan();
        log_sum = bad ? nan : empty ? -INFINITY : logf(s);
        entropy = bad ? nan : empty ? 0.f : fmaxf(log_sum - sx / s, 0.f);
        m = bad ? nan : M;
    }
    __device__ float log_prob(float x) const { return bad ? quiet_nan() : empty ? -INFINITY : (x - m) - log_sum; }
};

__device__ __forceinline__ void write_row(const LogprobsParams &p, int n, const RowStats &st) {
    if (p.max_logit) p.max_logit[n] = st.m;
    if (p.log_sum) p.log_sum[n] = st.log_sum;
    if (p.entropy) p.entropy[n] = st.entropy;
}

template <typename E>
__device__ __forceinline__ void write_tokens(const LogprobsParams &p, int n, const E *row, const RowStats &st, int t) {
    if (t >= p.T) return;
    const int id = p.ids[(size_t)n * p.T + t];
    p.logprobs[(size_t)n * p.T + t] = (unsigned)id < (unsigned)p.V ? st.log_prob((float)row[id]) : quiet_nan();
}

__device__ __forceinline__ void write_alternative(const LogprobsParams &p, int n, int k, const RowStats &st, float x,
                                                  int id) {
    const bool none = st.bad || x == -INFINITY;
    p.top_ids[(size_t)n * p.K + k] = none ? -1 : id;
    p.top_logprobs[(size_t)n * p.K + k] = st.bad ? quiet_nan() : none ? -INFINITY : st.log_prob(x);
}

// A wavefront's list, entry i on lane i, by logit and then by id
struct TopList {
    float v;
    int id;
    float last;  // the K-th
    __device__ TopList() : v(-INFINITY), id(INT_MAX), last(-INFINITY) {}
    // x, i: the same on all lanes; ids come in ascending order
    __device__ __forceinline__ void insert(float x, int i, int K) {
        const int lane = threadIdx.x & (kWave - 1);
        const int pos = __popcll(__ballot(v >= x));
        const float uv = __shfl_up(v, 1, kWave);
        const int ui = __shfl_up(id, 1, kWave);
        v = lane < pos ? v : lane == pos ? x : uv;
        id = lane < pos ? id : lane == pos ? i : ui;
        last = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), K - 1));
    }
    // lanes hold n values each (first id `at`), in ascending order of ids over the lanes; has: the lane holds any
    template <int n, typename E>
    __device__ __forceinline__ void scan(const E *x, int at, bool has, float tau, int K) {
        float c = -INFINITY;
#pragma unroll
        for (int j = 0; j < n; ++j) c = fmaxf(c, (float)x[j]);
        unsigned long long who = __ballot(has && c >= tau && c > last);
        while (who) {
            const int l = __ffsll(who) - 1;
            who &= who - 1;
            const int first = __builtin_amdgcn_readlane(at, l);
#pragma unroll
            for (int j = 0; j < n; ++j) {
                const float v1 = __builtin_bit_cast(
                    float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, (float)x[j]), l));
                if (v1 >= tau && v1 > last) insert(v1, first + j, K);
            }
        }
    }
};

template <typename E>
__global__ __launch_bounds__(kT) void logprobs_kernel(LogprobsParams p) {
    constexpr int G = Granule<E>::n;
    const int n = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const RowView<E> row(static_cast<const E *>(p.logits) + (long long)n * p.stride, p.V);
    const int g0 = (int)((long long)row.whole * part / p.parts), g1 = (int)((long long)row.whole * (part + 1) / p.parts);
    const int heads = part == 0 ? row.head : 0, tails = part == p.parts - 1 ? row.tail : 0;
    const E *body = row.p + row.head, *end = row.p + p.V - row.tail;

    LaneSum a{-FLT_MAX, 0.f, 0.f, -INFINITY, 0};
    int g = g0 + tid;
    for (; g + (kUnroll - 1) * kT < g1; g += kUnroll * kT) {
        Granule<E> x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) x[u] = load_granule(body + (size_t)(g + u * kT) * G);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) take(a, x[u], g + u * kT);
    }
    for (; g < g1; g += kT) take(a, load_granule(body + (size_t)g * G), g);
    if (tid < heads + tails) {
        const float x = (float)(tid < heads ? row.p[tid] : end[tid - heads]);
        raise(a, x);
        add(a, x);
    }

    // the workgroup's maximum and sums about it
    __shared__ float red[3][kWaves];
    __shared__ float lane_best[kT];
    {
        float m = a.best;
        if (tid < heads + tails) m = fmaxf(m, (float)(tid < heads ? row.p[tid] : end[tid - heads]));
        m = wave_max(m);
        if (lane == 0) red[0][wave] = m;
    }
    lane_best[tid] = a.best;
    __syncthreads();
    float M = red[0][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, red[0][w]);
    shift(a.r, a.s, a.sx, M);
    const float ws = wave_sum(a.s), wx = wave_sum(a.sx);
    if (lane == 0) {
        red[1][wave] = ws;
        red[2][wave] = wx;
    }
    __syncthreads();
    float s = 0.f, sx = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        s += red[1][w];
        sx += red[2][w];
    }
    const RowStats st(M, s, sx);
    float *sums = p.part_sums + ((size_t)n * p.parts + part) * 4;
    if (p.parts > 1) {
        if (tid == 0) {
            sums[0] = M;
            sums[1] = s;
            sums[2] = sx;
        }
    } else {
        if (tid == 0) write_row(p, n, st);
        write_tokens(p, n, row.p, st, tid);
    }
    if (p.K == 0) return;

    // tau: the K-th largest of 64 groups of lanes
    float tau;
    {
        float c = lane_best[lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) c = fmaxf(c, lane_best[w * kWave + lane]);
        int rank = 0;
#pragma unroll 8
        for (int l = 0; l < kWave; ++l) {
            const float o = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, c), l));
            rank += o > c || (o == c && l < lane);
        }
        const int l = __ffsll(__ballot(rank == p.K - 1)) - 1;
        tau = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, c), l));
    }
    // the lanes that read again, in ascending order
    __shared__ int sel[kT], count[kWaves + 1];
    const bool again = a.best >= tau && a.best > -INFINITY;
    const unsigned long long mask = __ballot(again);
    if (lane == 0) count[wave] = __popcll(mask);
    __shared__ int entries;
    if (tid == 0) entries = 0;
    __syncthreads();
    int before = 0, nsel = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        before += w < wave ? count[w] : 0;
        nsel += count[w];
    }
    if (again) sel[before + __popcll(mask & ((1ull << lane) - 1))] = tid;
    __syncthreads();

    TopList top;
    if (wave == 0 && heads) top.scan<1>(row.p + (lane < heads ? lane : 0), lane, lane < heads, tau, p.K);
    const int steps = (g1 - g0 + kT - 1) / kT, todo = steps * nsel;
    for (int e0 = wave * kWave; e0 < todo; e0 += kUnroll * kT) {
        Granule<E> x[kUnroll];
        int at[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int e = e0 + u * kT + lane, i = e / nsel;
            const int gi = g0 + i * kT + sel[e < todo ? e - i * nsel : 0];
            at[u] = e < todo && gi < g1 ? gi : -1;
            x[u] = load_granule(body + (size_t)(at[u] >= 0 ? at[u] : g0) * G);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) top.scan<G>(x[u].v, row.index(at[u]), at[u] >= 0, tau, p.K);
    }
    if (wave == 0 && tails) top.scan<1>(end + (lane < tails ? lane : 0), p.V - row.tail + lane, lane < tails, tau, p.K);

    // the lists' entries, in any order, each to the place that its rank gives it
    __shared__ float ev[kWaves * SPECEE_TOP_MAX];
    __shared__ int ei[kWaves * SPECEE_TOP_MAX];
    {
        const bool mine = lane < p.K && top.v > -INFINITY;
        const int c = __popcll(__ballot(mine));
        int first = 0;
        if (lane == 0 && c) first = atomicAdd(&entries, c);
        first = __builtin_amdgcn_readfirstlane(first);
        if (mine) {
            ev[first + lane] = top.v;
            ei[first + lane] = top.id;
        }
    }
    __syncthreads();
    const int C = entries;
    float v = -INFINITY;
    int id = INT_MAX, rank = tid;
    if (tid < C) {
        v = ev[tid];
        id = ei[tid];
        rank = 0;
        for (int k = 0; k < C; ++k) rank += ev[k] > v || (ev[k] == v && ei[k] < id);
    }
    if (rank < p.K) {
        if (p.parts > 1) {
            p.part_vals[((size_t)n * p.parts + part) * p.K + rank] = v;
            p.part_ids[((size_t)n * p.parts + part) * p.K + rank] = id;
        } else {
            write_alternative(p, n, rank, st, v, id);
        }
    }
}

// Joins the parts of a row: one workgroup of two wavefronts, one for the alternatives and one for the tokens.
template <typename E>
__global__ __launch_bounds__(2 * kWave) void logprobs_join_kernel(LogprobsParams p) {
    const int n = blockIdx.x, lane = threadIdx.x & (kWave - 1);
    const E *row = static_cast<const E *>(p.logits) + (long long)n * p.stride;
    __shared__ float lv[kMaxParts][SPECEE_TOP_MAX];
    __shared__ int li[kMaxParts][SPECEE_TOP_MAX];
    for (int e = threadIdx.x; e < p.parts * p.K; e += blockDim.x) {
        lv[e / p.K][e % p.K] = p.part_vals[(size_t)n * p.parts * p.K + e];
        li[e / p.K][e % p.K] = p.part_ids[(size_t)n * p.parts * p.K + e];
    }
    float r = -INFINITY, s = 0.f, sx = 0.f;
    if (lane < p.parts) {
        const float *sums = p.part_sums + ((size_t)n * p.parts + lane) * 4;
        r = sums[0];
        s = sums[1];
        sx = sums[2];
    }
    const float M = wave_max(r);
    shift(r, s, sx, M);
    const RowStats st(M, wave_sum(s), wave_sum(sx));
    __syncthreads();
    if (threadIdx.x >= kWave) {
        if (lane == 0) write_row(p, n, st);
        write_tokens(p, n, row, st, lane);
        return;
    }
    // the parts' lists are sorted: the best of their first entries, K times
    float mv = -INFINITY;
    int mi = INT_MAX, at = 0;
    for (int k = 0; k < p.K; ++k) {
        const bool has = lane < p.parts && at < p.K;
        float v = has ? lv[lane][at] : -INFINITY;
        int id = has ? li[lane][at] : INT_MAX;
        const int mine = id;
        row16_argmax(v, id);
        if (mine == id && mine != INT_MAX) ++at;
        // (lanes of row 0 hold the parts; the winner is read from its first lane)
        v = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
        id = __builtin_amdgcn_readfirstlane(id);
        if (lane == k) {
            mv = v;
            mi = id;
        }
    }
    if (lane < p.K) write_alternative(p, n, lane, st, mv, mi);
}

// Gradient: elementwise, one workgroup per kGradSteps * 512 granules of a row; the ids that fall into its share are looked
// for once and kept in LDS, in their order, so that ids that repeat add up the same way every time.
constexpr int kGradSteps = 4;

struct GradRow {
    float m, log_sum, entropy, factor, g_entropy;
    __device__ __forceinline__ float operator()(float x) const {
        const float lp = fmaxf((x - m) - log_sum, kFloor);
        return -__builtin_amdgcn_exp2f(lp * kLog2e) * fmaf(g_entropy, lp + entropy, factor);
    }
};

template <typename E>
__global__ __launch_bounds__(kT) void logprobs_grad_kernel(LogprobsGradParams p) {
    constexpr int G = Granule<E>::n;
    const int n = blockIdx.y, tid = threadIdx.x, lane = tid & (kWave - 1);
    const RowView<E> row(static_cast<const E *>(p.logits) + (long long)n * p.stride, p.V);
    E *out = static_cast<E *>(p.grad) + (long long)n * p.grad_stride;
    const int g0 = blockIdx.x * (kGradSteps * kT), g1 = min(row.whole, g0 + kGradSteps * kT);
    const bool first = blockIdx.x == 0, last = blockIdx.x == gridDim.x - 1;
    const E *body = row.p + row.head;
    // elements of this workgroup
    const int v0 = first ? 0 : row.index(g0), v1 = last ? p.V : row.index(g1);

    __shared__ int hit_id[SPECEE_IDS_MAX], hits;
    __shared__ float hit_g[SPECEE_IDS_MAX], factor;
    if (tid < kWave) {
        int id = -1;
        float gt = 0.f;
        if (lane < p.T) {
            id = p.ids[(size_t)n * p.T + lane];
            if ((unsigned)id < (unsigned)p.V) gt = p.g_logprobs[(size_t)n * p.T + lane];
        }
        const float sum = wave_sum(gt);
        const bool here = id >= v0 && id < v1;
        const unsigned long long who = __ballot(here);
        if (here) {
            const int at = __popcll(who & ((1ull << lane) - 1));
            hit_id[at] = id;
            hit_g[at] = gt;
        }
        if (lane == 0) {
            hits = __popcll(who);
            factor = sum;
        }
    }
    Granule<E> x[kGradSteps];
#pragma unroll
    for (int u = 0; u < kGradSteps; ++u) {
        const int g = g0 + u * kT + tid;
        if (g < g1) x[u] = load_granule(body + (size_t)g * G);
    }
    const int extras = (first ? row.head : 0) + (last ? row.tail : 0);
    int extra = -1;
    float xe = 0.f;
    if (tid < extras) {
        extra = first && tid < row.head ? tid : p.V - extras + tid;
        xe = (float)row.p[extra];
    }
    GradRow f{p.max_logit[n], p.log_sum[n], 0.f, 0.f, 0.f};
    if (p.g_entropy) {
        f.entropy = p.entropy[n];
        f.g_entropy = p.g_entropy[n];
    }
    __syncthreads();
    f.factor = factor;
    const int H = hits;
    const bool empty = f.m == -INFINITY;  // no token has a probability: nothing to move
    const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15) == 0;
#pragma unroll
    for (int u = 0; u < kGradSteps; ++u) {
        const int g = g0 + u * kT + tid;
        if (g < g1) {
            const int at = row.index(g);
            float d[G];
#pragma unroll
            for (int j = 0; j < G; ++j) d[j] = f((float)x[u].v[j]);
            for (int h = 0; h < H; ++h) {
                const int j0 = hit_id[h] - at;
                if ((unsigned)j0 < (unsigned)G)
#pragma unroll
                    for (int j = 0; j < G; ++j) d[j] += j == j0 ? hit_g[h] : 0.f;
            }
            Granule<E> o;
#pragma unroll
            for (int j = 0; j < G; ++j) o.v[j] = (E)(empty ? 0.f : d[j]);
            if (same)
                *reinterpret_cast<uintx4 *>(out + at) = *reinterpret_cast<const uintx4 *>(&o);
            else
#pragma unroll
                for (int j = 0; j < G; ++j) out[at + j] = o.v[j];
        }
    }
    if (extra >= 0) {
        float d = f(xe);
        for (int h = 0; h < H; ++h) d += hit_id[h] == extra ? hit_g[h] : 0.f;
        out[extra] = (E)(empty ? 0.f : d);
    }
}

}  // namespace

// Parts of a row: as many workgroups as make two per CU, as long as each has a granule for every thread
int logprobs_parts(int N, int V, bool half) {
    const int whole = V / (half ? 8 : 4);
    int parts = 512 / (N > 0 ? N : 1);
    if (parts > whole / kT) parts = whole / kT;
    return parts < 1 ? 1 : parts > kMaxParts ? kMaxParts : parts;
}

hipError_t launch_logprobs(const LogprobsParams &p, bool half, hipStream_t s) {
    const dim3 grid((unsigned)p.N * p.parts);
    if (half)
        hipLaunchKernelGGL(logprobs_kernel<half_t>, grid, dim3(kT), 0, s, p);
    else
        hipLaunchKernelGGL(logprobs_kernel<float>, grid, dim3(kT), 0, s, p);
    if (p.parts > 1) {
        if (half)
            hipLaunchKernelGGL(logprobs_join_kernel<half_t>, dim3(p.N), dim3(2 * kWave), 0, s, p);
        else
            hipLaunchKernelGGL(logprobs_join_kernel<float>, dim3(p.N), dim3(2 * kWave), 0, s, p);
    }
    return hipGetLastError();
}

hipError_t launch_logprobs_grad(const LogprobsGradParams &p, bool half, hipStream_t s) {
    const int whole = p.V / (half ? 8 : 4), share = kGradSteps * kT;
    const dim3 grid(whole < 1 ? 1 : (whole + share - 1) / share, p.N);
    if (half)
        hipLaunchKernelGGL(logprobs_grad_kernel<half_t>, grid, dim3(kT), 0, s, p);
    else
        hipLaunchKernelGGL(logprobs_grad_kernel<float>, grid, dim3(kT), 0, s, p);
    return hipGetLastError();
}

}  // namespace specee
