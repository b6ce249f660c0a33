// What is answered with a row of logits x[0..V): log probabilities of given tokens, the entropy, the best alternatives; and
// the gradient of the first two.  With m = max x, S = sum exp(x - m):
//     log p(v) = (x_v - m) - log S,   H = log S - sum exp(x - m) (x - m) / S,
//     dx_v = sum of g_t over ids t equal to v - p_v * (sum of g_t + g_H * (log p_v + H)).
// m and log S are kept apart: their sum, the usual normaliser, would round away 1e-6 of every probability.  So are the 1 that m
// itself is in S, and the rest u: where one token is all but certain, log S = log(1 + u) is about u, and S as one number would
// hold u to 6e-8 of 1 instead of 6e-8 of itself.
//
// Forward: one pass over the logits, bound by their bytes from a few hundred rows on (4096 x 128256 fp32, 2.1 GB: 319 us, 6.6
// TB/s) and by launch and latency below (1 x 32000: 6.7 us).  A lane keeps its largest element out of its sums, and of the others
// the sums of exp(x - r) and exp(x - r)(x - r) about a reference r (an element of its own, at most 8 below its maximum): a new
// maximum seldom costs it a rescaling.  The largest of 16 bytes and the rest come from minima and maxima in pairs, one
// instruction per element (with S as one number: 1 x 32000 6.4 us, 64 x 128256 14.1 against 14.5, 2043 x 32003 fp16 27.6
// against 28.8).  16 bytes are loaded per lane and step; rows may start at any element (what lies before the first and behind the
// last whole 16 bytes is done one element per lane).  A logit of -inf adds nothing (its t is cut at -300, and 2^-300 is 0 in
// fp32); NaN makes the sum NaN, +inf is the maximum: both are looked at once at the end.
// Rows of 64 KB (2043 x 32003 fp16: 28.8 us, 4.5 TB/s) are bound by what each does one after the other, loads, meetings and
// second reads, with four rows on a CU: neither twice the loads in flight nor a fifth fewer vector instructions made a difference.
// Alternatives cost the pass three instructions per 16 bytes: a lane keeps its largest granule's place and the maximum of the
// others.  Behind the pass groups of lanes meet, and the n-th largest of their maxima, tau, is at most the n-th largest logit:
// only what reaches tau is read again, and taken into a sorted list per wavefront, one entry per lane (a few alternatives), or
// gathered and ranked as it is (many).  The order is by logit and then by id, so the result does not depend on which wavefront
// saw what.
// A few long rows are cut into parts that registers hold, one workgroup each, which a second launch joins.
#include <float.h>
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "../../include/specee.h"
#include "device_utils.h"
#include "kernels.h"

namespace specee {

namespace {

constexpr int kT = 512;  // threads of a workgroup
constexpr int kUnroll = 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;   // how far a lane's reference may lie below its maximum
constexpr float kFloor = -300.f;
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
template <typename E>
__device__ __forceinline__ Granule<E> load_granule_once(const E *p) {
    return __builtin_bit_cast(Granule<E>, __builtin_nontemporal_load(reinterpret_cast<const uintx4 *>(p)));
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

// Sums about a reference r, in base 2: t = (x - r) log2 e.  fp16 logits form t in one mixed instruction from x and the rounded
// product r log2 e (about_exactly puts back what was rounded off); fp32 logits, which may be near the ends of their type, from x - r.
template <typename E>
struct LaneSum {
    static constexpr bool kMixed = sizeof(E) == 2;
    static constexpr float kLowest = kMixed ? -1e6f : -FLT_MAX;
    float r;      // an element, or kLowest while there is none
    float r2;     // kMixed: r log2 e
    float s, st;  // sum of 2^t, of 2^t t

    __device__ __forceinline__ void about(float ref) {
#pragma clang fp contract(off)  // the rounded product, also where it is subtracted
        r = ref;
        r2 = kMixed ? ref * kLog2e : 0.f;
    }
    __device__ __forceinline__ explicit LaneSum(float ref) : s(0.f), st(0.f) { about(ref); }
    __device__ __forceinline__ float distance(float x) const { return kMixed ? fmaf(x, kLog2e, -r2) : (x - r) * kLog2e; }
    // skip: x counts as nothing
    __device__ __forceinline__ void add(float x, bool skip = false) {
        const float t = distance(x), e = skip ? 0.f : __builtin_amdgcn_exp2f(t);
        s += e;
        st = fmaf(e, fmaxf(t, kFloor), st);
    }
    // The same sums about M >= r
    __device__ __forceinline__ void move(float M) {
        const LaneSum to(M);
        if (s == 0.f) {  // empty: r may be anything
            st = 0.f;
        } else {
            const float d = kMixed ? r2 - to.r2 : (r - M) * kLog2e, f = __builtin_amdgcn_exp2f(d);
            st = f > 0.f ? (st + s * d) * f : 0.f;
            s *= f;
        }
        r = to.r;
        r2 = to.r2;
    }
    // ... about the largest of the elements to come
    __device__ __forceinline__ void raise(float c) {
        if (c > r + kSlack) {
            if (s > 0.f)
                move(c);
            else
                about(c);  // (nothing yet; or NaN, which stays)
        }
    }
};

// The largest element, and the others in any order.  NaN stays among the others.
__device__ __forceinline__ float split(const Granule<float> &g, float *low) {
    float hi[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        hi[j] = __builtin_elementwise_maximum(g.v[j], g.v[j + 2]);
        low[j] = __builtin_elementwise_minimum(g.v[j], g.v[j + 2]);
    }
    low[2] = __builtin_elementwise_minimum(hi[0], hi[1]);
    return fmaxf(hi[0], hi[1]);
}
__device__ __forceinline__ float split(const Granule<half_t> &g, float *low) {
    half2_t x[4], l[3];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = half2_t{g.v[2 * j], g.v[2 * j + 1]};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        l[j] = __builtin_elementwise_minimum(x[j], x[j + 2]);
        x[j] = __builtin_elementwise_maximum(x[j], x[j + 2]);
    }
    l[2] = __builtin_elementwise_minimum(x[0], x[1]);
    x[0] = __builtin_elementwise_maximum(x[0], x[1]);
#pragma unroll
    for (int j = 0; j < 6; ++j) low[j] = (float)l[j / 2][j % 2];
    low[6] = (float)__builtin_elementwise_minimum(x[0][0], x[0][1]);
    return fmaxf((float)x[0][0], (float)x[0][1]);
}

template <typename E>
__device__ __forceinline__ float largest(const Granule<E> &g) {
    float c = -INFINITY;
#pragma unroll
    for (int j = 0; j < Granule<E>::n; ++j) c = fmaxf(c, (float)g.v[j]);
    return c;
}

__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_f32<kDppXor1>(v));
    v = fmaxf(v, dpp_f32<kDppXor2>(v));
    v = fmaxf(v, dpp_f32<kDppHalfMirror>(v));
    v = fmaxf(v, dpp_f32<kDppMirror>(v));
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    return fmaxf(v, __shfl_xor(v, 32, kWave));
}

// Sums about the rounded M log2 e, in base 2, as sums about M log2 e
__device__ __forceinline__ void about_exactly(float M, float *s, float *st) {
    if (fabsf(M) == INFINITY) return;
    const float off = fmaf(-M, kLog2e, M * kLog2e), f = __builtin_amdgcn_exp2f(off);
    *st = fmaf(off, *s, *st) * f;
    *s *= f;
}

// log(1 + u), u >= 0, to its relative precision: u' = (1 + u) - 1 is what the logarithm saw of u (Kahan's correction)
__device__ __forceinline__ float log_above_one(float u) {
    const float one = 1.f + u, seen = one - 1.f;
    return seen > 0.f ? logf(one) * (u / seen) : u;
}

// What a row's sums mean.  NaN or +inf among the logits: everything NaN; nothing above -inf: nothing has a probability.
struct RowStats {
    float m, log_sum, entropy;
    bool bad, empty;
    // M: the row's largest logit, `tops` times; s, st: the sums of the others about it, in base 2.  S = tops + s, and what S has
    // above 1 is held by itself: of a confident row it is all that log S, and minus the best token's log probability, consist of.
    __device__ RowStats(float M, float tops, float s, float st) {
        bad = !(s == s) || M == INFINITY;
        empty = M == -INFINITY;
        const float nan = quiet_nan(), above = s + (tops - 1.f), ln = log_above_one(above);
        log_sum = bad ? nan : empty ? -INFINITY : ln;
        entropy = bad ? nan : empty ? 0.f : ln - kLn2 * (st / (1.f + above));
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

__device__ __forceinline__ int from_lane_below(int v) {
    constexpr int kDppWaveShr1 = 0x138;
    return __builtin_amdgcn_update_dpp(v, v, kDppWaveShr1, 0xF, 0xF, false);
}

// The K-th largest of the groups' maxima, or a little less: floats as integers of the same order, whose last six bits are the
// group, so that no two are equal.  Each wavefront counts for GROUPS / WAVES of them; tau is there behind the next meeting.
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, v);
    return bits ^ (bits >> 31 ? 0xffffffffu : 0x80000000u);
}
template <int GROUPS, int WAVES>
__device__ __forceinline__ void kth_largest(float c, int K, float *tau) {
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t key = (lane < GROUPS ? ordered(c) & ~63u : 0u) | (63 - lane);
#pragma unroll
    for (int k = 0; k < GROUPS / WAVES; ++k) {
        const uint32_t mine = (uint32_t)__builtin_amdgcn_readlane((int)key, wave * (GROUPS / WAVES) + k);
        if (__popcll(__ballot(key > mine)) == K - 1 && lane == 0) {
            const uint32_t b = mine & ~63u;
            const float t = __builtin_bit_cast(float, b >> 31 ? b ^ 0x80000000u : ~b);
            *tau = t == t ? t : -INFINITY;  // (below -inf, in this order, there are NaNs)
        }
    }
}

// A wavefront's list, entry i on lane i, by logit and then by id
struct TopList {
    float v;
    int id;
    float last;  // the K-th
    int last_id;
    __device__ TopList() : v(-INFINITY), id(INT_MAX), last(-INFINITY), last_id(INT_MAX) {}
    // x, i: the same on all lanes
    __device__ __forceinline__ void insert(float x, int i, int K) {
        const int lane = threadIdx.x & (kWave - 1);
        const int pos = __popcll(__ballot(v > x || (v == x && id < i)));
        const float uv = __builtin_bit_cast(float, from_lane_below(__builtin_bit_cast(int, v)));
        const int ui = from_lane_below(id);
        v = lane < pos ? v : lane == pos ? x : uv;
        id = lane < pos ? id : lane == pos ? i : ui;
        last = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), K - 1));
        last_id = __builtin_amdgcn_readlane(id, K - 1);
    }
    // n values on each lane that has any, the first with id `at`; c: the largest of them
    template <int n, typename E>
    __device__ __forceinline__ void scan(const E *x, float c, int at, bool has, float tau, int K) {
        unsigned long long who = __ballot(has && c >= tau && c >= last && c > -INFINITY);
        while (who) {
            const int l = __ffsll(who) - 1;
            who &= who - 1;
            const int first = __builtin_amdgcn_readlane(at, l);
#pragma unroll
            for (int j = 0; j < n; ++j) {
                const float v1 = __builtin_bit_cast(
                    float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, (float)x[j]), l));
                if (v1 >= tau && (v1 > last || (v1 == last && first + j < last_id))) insert(v1, first + j, K);
            }
        }
    }
};

// Calls put(rank, x, id) on one lane for each of the C entries (in LDS) whose rank is below K, by x and then by id.  Up to 64: an
// entry per lane, and the wavefronts count for their share of them; more: a thread counts for its own.
template <int WAVES, typename F>
__device__ __forceinline__ void rank_entries(const float *v, const int *id, int C, int K, const F &put) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    if (C > kWave) {
        for (int e = tid; e < C; e += WAVES * kWave) {
            const float x = v[e];
            const int i = id[e];
            int rank = 0;
#pragma unroll 8
            for (int o = 0; o < C; ++o) rank += v[o] > x || (v[o] == x && id[o] < i);
            if (rank < K) put(rank, x, i);
        }
        return;
    }
    const float mv = lane < C ? v[lane] : -INFINITY;
    const int mi = lane < C ? id[lane] : INT_MAX;
    for (int e = wave; e < C; e += WAVES) {
        const float x = v[e];
        const int i = id[e];
        const int rank = __popcll(__ballot(mv > x || (mv == x && mi < i)));
        if (rank < K && lane == 0) put(rank, x, i);
    }
}

// What a workgroup's wavefronts leave for its end: their sums, and candidates for the alternatives in any order
template <int WAVES>
struct RowEnd {
    // (room for every wavefront's best, and for rows that have fewer granules than there are alternatives)
    static constexpr int kMost = WAVES < 8 ? 8 * SPECEE_TOP_MAX : WAVES * SPECEE_TOP_MAX;
    float s[WAVES], st[WAVES];
    int tops[WAVES];
    int entries;  // 0 at a meeting of the workgroup before the first candidate; more than kMost: some had no place
    float v[kMost];
    int id[kMost];

    // of a wavefront: lanes' sums without what equals the maximum, and how often that was
    __device__ __forceinline__ void sums(float sum, float sumt, int top) {
        sum = wave_sum(sum);
        sumt = wave_sum(sumt);
        if ((threadIdx.x & (kWave - 1)) == 0) {
            s[threadIdx.x / kWave] = sum;
            st[threadIdx.x / kWave] = sumt;
            tops[threadIdx.x / kWave] = top;
        }
    }
    // Places for c entries of a wavefront
    __device__ __forceinline__ int places(int c) {
        int first = 0;
        if ((threadIdx.x & (kWave - 1)) == 0) first = atomicAdd(&entries, c);
        return __builtin_amdgcn_readfirstlane(first);
    }
    // Whatever reaches tau; arguments as for TopList
    template <int n, typename E>
    __device__ __forceinline__ void scan(const E *x, float c, int at, bool has, float tau, int) {
        const int lane = threadIdx.x & (kWave - 1);
        const bool any = has && c >= tau && c > -INFINITY;
        if (!__ballot(any)) return;
        unsigned long long who[n];
        int c_all = 0;
#pragma unroll
        for (int j = 0; j < n; ++j) {
            who[j] = __ballot(any && (float)x[j] >= tau && (float)x[j] > -INFINITY);
            c_all += __popcll(who[j]);
        }
        int first = places(c_all);
#pragma unroll
        for (int j = 0; j < n; ++j) {
            const int k = first + __popcll(who[j] & ((1ull << lane) - 1));
            if ((who[j] >> lane & 1) && k < kMost) {
                v[k] = (float)x[j];
                id[k] = at + j;
            }
            first += __popcll(who[j]);
        }
    }
    __device__ __forceinline__ void leave(const TopList &top, int K) {
        const int lane = threadIdx.x & (kWave - 1);
        const bool mine = lane < K && top.v > -INFINITY;
        const int c = __popcll(__ballot(mine));
        const int first = c ? places(c) : 0;
        if (mine) {
            v[first + lane] = top.v;
            id[first + lane] = top.id;
        }
    }
    // The workgroup's candidates; each(to, tau) shows a wavefront's to to.scan().  MANY: all that reach tau, where they have a
    // place (they nearly always do: without equal logits K alternatives have about K to 1.5 K of them); else each wavefront's
    // best.  Follows and ends with a meeting.
    template <bool MANY, typename F>
    __device__ __forceinline__ void gather(float tau, int K, float sum, float sumt, int top, const F &each) {
        if (MANY) {
            sums(sum, sumt, top);
            each(*this, tau);
            __syncthreads();
            if (entries <= kMost) return;
            __syncthreads();
            if (threadIdx.x == 0) entries = 0;
            __syncthreads();
        }
        TopList list;
        each(list, tau);
        if (!MANY) sums(sum, sumt, top);
        leave(list, K);
        __syncthreads();
    }
    // Behind a meeting: the row's outputs, or what a PART of one leaves.  An entry's place is its rank.
    template <bool PART, typename E>
    __device__ __forceinline__ void write(const LogprobsParams &p, int n, int part, const E *row, float M) const {
        const int tid = threadIdx.x;
        float S = 0.f, ST = 0.f;
        int top = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            S += s[w];
            ST += st[w];
            top += tops[w];
        }
        if (LaneSum<E>::kMixed) about_exactly(M, &S, &ST);
        const RowStats stats(M, (float)top, S, ST);
        const size_t at = (size_t)n * p.parts + part;
        if (PART) {
            if (tid == 0) {
                p.part_sums[at * 4] = M;
                p.part_sums[at * 4 + 1] = S;
                p.part_sums[at * 4 + 2] = ST;
                p.part_sums[at * 4 + 3] = (float)top;
            }
        } else {
            if (tid == 0) write_row(p, n, stats);
            write_tokens(p, n, row, stats, tid);
        }
        if (p.K == 0) return;
        const int C = entries;
        auto put = [&](int k, float x, int i) {
            if (PART) {
                p.part_vals[at * p.K + k] = x;
                p.part_ids[at * p.K + k] = i;
            } else {
                write_alternative(p, n, k, stats, x, i);
            }
        };
        rank_entries<WAVES>(v, id, C, p.K, put);
        if (tid >= C && tid < p.K) put(tid, -INFINITY, INT_MAX);
    }
};

// Groups of 16 lanes, or 64 groups for many alternatives, whose tau comes the closer to the last of them
template <int T, bool MANY>
struct Groups {
    static constexpr int n = MANY ? kWave : T / 16, lanes = T / n;
    static_assert(lanes == 4 || lanes == 8 || lanes == 16, "");
    __device__ static __forceinline__ float max(float v) {
        v = fmaxf(v, dpp_f32<kDppXor1>(v));
        v = fmaxf(v, dpp_f32<kDppXor2>(v));
        if (lanes > 4) v = fmaxf(v, dpp_f32<kDppHalfMirror>(v));
        if (lanes > 8) v = fmaxf(v, dpp_f32<kDppMirror>(v));
        return v;
    }
};

// A part of a row that a workgroup holds in registers, U granules per lane: the maximum first, then the sums about it and the
// alternatives, all from the registers.
template <typename E, int U, bool MANY>
__global__ __launch_bounds__(kT, 8) void logprobs_held_kernel(LogprobsParams p) {
    constexpr int T = kT, G = Granule<E>::n, WAVES = T / kWave;
    const int n = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const RowView<E> row(static_cast<const E *>(p.logits) + (long long)n * p.stride, p.V);
    const int g0 = (int)((long long)row.whole * part / p.parts), g1 = (int)((long long)row.whole * (part + 1) / p.parts);
    const int heads = part == 0 ? row.head : 0, tails = part == p.parts - 1 ? row.tail : 0;
    const E *body = row.p + row.head, *end = row.p + p.V - row.tail;
    using Group = Groups<T, MANY>;
    __shared__ float groups[Group::n], tau;
    __shared__ RowEnd<WAVES> last;

    uintx4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = uintx4{0, 0, 0, 0};
    if (g0 < g1) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int g = min(g0 + u * T + tid, g1 - 1);
            raw[u] = __builtin_nontemporal_load(reinterpret_cast<const uintx4 *>(body + (size_t)g * G));
        }
    }
    float xe = -INFINITY;  // one of the elements before and behind the granules
    if (tid < heads + tails) xe = (float)(tid < heads ? row.p[tid] : end[tid - heads]);
    if (tid == 0) last.entries = 0;
    float c = xe == xe ? xe : -INFINITY;
    const uint32_t nothing = sizeof(E) == 4 ? 0xff800000u : 0xfc00fc00u;  // -inf
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (g0 + u * T + tid >= g1) raw[u] = uintx4{nothing, nothing, nothing, nothing};
        c = fmaxf(c, largest(__builtin_bit_cast(Granule<E>, raw[u])));
        // (fp16 logits are widened again below: kept as floats they would cost half of the workgroups that a CU holds)
        if (sizeof(E) == 2) asm volatile("" : "+v"(raw[u]));
    }
    const float mine = c;
    c = Group::max(c);
    if (tid % Group::lanes == 0) groups[tid / Group::lanes] = c;
    __syncthreads();
    c = lane < Group::n ? groups[lane] : -INFINITY;
    if (p.K) kth_largest<Group::n, WAVES>(c, p.K, &tau);
    const float M = wave_max(c);
    LaneSum<E> a(fmaxf(M, LaneSum<E>::kLowest));
    int tops = 0;
    auto add = [&](float x, auto with_top) {
        const bool top = with_top && x == M;
        if (with_top) tops += __popcll(__ballot(top));
        a.add(x, top);
    };
    auto add_all = [&](auto with_top) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Granule<E> x = __builtin_bit_cast(Granule<E>, raw[u]);
#pragma unroll
            for (int j = 0; j < G; ++j) add((float)x.v[j], with_top);
            if (sizeof(E) == 2) asm volatile("" : "+v"(raw[u]));
        }
        add(xe, with_top);
    };
    if (__ballot(mine == M)) {
        asm volatile("" : "+v"(a.r), "+v"(a.r2));  // (differences formed once for both ways would not fit the registers)
        add_all(std::true_type());
    } else {
        add_all(std::false_type());
    }
    if (p.K) {
        __syncthreads();
        last.template gather<MANY>(tau, p.K, a.s, a.st, tops, [&](auto &to, float least) {
            if (wave == 0 && heads) to.template scan<1>(&xe, xe, lane, lane < heads, least, p.K);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int g = g0 + u * T + tid;
                const Granule<E> x = __builtin_bit_cast(Granule<E>, raw[u]);
                to.template scan<G>(x.v, largest(x), row.index(g), g < g1, least, p.K);
            }
            if (wave == 0 && tails)
                to.template scan<1>(&xe, xe, p.V - row.tail + lane - heads, lane >= heads && lane < heads + tails, least, p.K);
        });
    } else {
        last.sums(a.s, a.st, tops);
        __syncthreads();
    }
    last.template write<true>(p, n, part, row.p, M);
}

// A row of any length, in steps.  A lane keeps its largest element, out of its sums, its place, and the maximum of the other
// granules.  Behind the pass the row's maximum is known, and what equals it stays out of the sums for good; the lanes whose
// largest reaches tau read its granule again, and the few of which another does, all of theirs.
template <typename E, int T, bool MANY>
__global__ __launch_bounds__(T, 8) void logprobs_kernel(LogprobsParams p) {
    constexpr int G = Granule<E>::n, WAVES = T / kWave;
    const int n = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const RowView<E> row(static_cast<const E *>(p.logits) + (long long)n * p.stride, p.V);
    const E *body = row.p + row.head, *end = row.p + p.V - row.tail;
    using Group = Groups<T, MANY>;
    __shared__ float groups[Group::n], tau;
    __shared__ RowEnd<WAVES> last;

    LaneSum<E> a(LaneSum<E>::kLowest);
    float best = -INFINITY, others = -INFINITY;
    int place = 0;
    auto take = [&](const Granule<E> &x, int g) {
        float low[G];
        const float c = split(x, low), less = fminf(c, best);
        a.raise(c);
        a.add(less);
#pragma unroll
        for (int j = 0; j < G - 1; ++j) a.add(low[j]);
        others = fmaxf(others, less);
        place = c > best ? g : place;
        best = fmaxf(best, c);
    };
    // Rows with less than a granule per lane: dealt out to the groups in turn, so that as many as can have one
    const int lane0 = row.whole < T ? tid % Group::lanes * Group::n + tid / Group::lanes : tid;
    int g0 = 0;
    for (; g0 + kUnroll * T <= row.whole; g0 += kUnroll * T) {
        Granule<E> x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) x[u] = load_granule_once(body + (size_t)(g0 + u * T + lane0) * G);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) take(x[u], g0 + u * T + lane0);
    }
    // The rest: at once in short rows, where its loads one after the other would take as long as all before (2043 x 32003 fp16
    // 34.5 -> 31 us); one by one in long ones, where other rows fill that time (4096 x 128256 fp32 327 us, at once 337)
    if (row.whole > 32 * T) {
        for (int g = g0 + lane0; g < row.whole; g += T) take(load_granule(body + (size_t)g * G), g);
    } else if (g0 < row.whole) {
        Granule<E> x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            x[u] = load_granule_once(body + (size_t)min(g0 + u * T + lane0, row.whole - 1) * G);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (g0 + u * T + lane0 < row.whole) take(x[u], g0 + u * T + lane0);
    }
    const bool extra = tid < row.head + row.tail;
    float xe = -INFINITY;
    if (extra) xe = (float)(tid < row.head ? row.p[tid] : end[tid - row.head]);
    if (tid == 0) last.entries = 0;
    float c = Group::max(fmaxf(best, xe == xe ? xe : -INFINITY));
    if (tid % Group::lanes == 0) groups[tid / Group::lanes] = c;
    __syncthreads();
    c = lane < Group::n ? groups[lane] : -INFINITY;
    const float M = wave_max(c);
    if (p.K) kth_largest<Group::n, WAVES>(c, p.K, &tau);
    a.move(M);
    int tops = 0;
    auto rest = [&](float x) {
        const bool top = x == M;
        tops += __popcll(__ballot(top));
        a.add(x, top);
    };
    rest(best);
    rest(xe);
    if (p.K) {
        __syncthreads();
        last.template gather<MANY>(tau, p.K, a.s, a.st, tops, [&](auto &to, float least) {
            to.template scan<1>(&xe, xe, tid < row.head ? tid : p.V - row.tail + tid - row.head, extra, least, p.K);
            const bool several = others >= least && others > -INFINITY;
            if (__ballot(best >= least && best > -INFINITY && !several)) {
                Granule<E> x = {};
                if (best >= least && !several && row.whole > 0) x = load_granule(body + (size_t)place * G);
                to.template scan<G>(x.v, best, row.index(place), !several, least, p.K);
            }
            unsigned long long who = __ballot(several);
            const int steps = (row.whole + T - 1) / T;
            while (who) {
                const int l = __ffsll(who) - 1;
                who &= who - 1;
                for (int i0 = 0; i0 < steps; i0 += kWave) {
                    const int gi = (i0 + lane) * T + (tid - lane) + l;
                    const bool has = gi < row.whole;
                    const Granule<E> x = load_granule(body + (size_t)(has ? gi : 0) * G);
                    to.template scan<G>(x.v, largest(x), row.index(gi), has, least, p.K);
                }
            }
        });
    } else {
        last.sums(a.s, a.st, tops);
        __syncthreads();
    }
    last.template write<false>(p, n, 0, row.p, M);
}

// Joins the parts of a row.  A thread holds one of their candidates, as an integer of the same order (by logit, where the two
// zeros are one, and then by id), and counts those above it among a share of all; the wavefronts that would hold none take
// further shares.
constexpr int kJoinMost = kMaxParts * SPECEE_TOP_MAX;
template <typename E>
__global__ __launch_bounds__(2 * kJoinMost) void logprobs_join_kernel(LogprobsParams p) {
    const int n = blockIdx.x, tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const E *row = static_cast<const E *>(p.logits) + (long long)n * p.stride;
    __shared__ unsigned long long keys[kJoinMost];
    __shared__ int above[kJoinMost], real;
    const int C = p.parts * p.K;
    float x = -INFINITY;  // (places without a candidate hold -inf)
    int id = INT_MAX;
    if (tid < C) {
        x = p.part_vals[(size_t)n * C + tid];
        id = p.part_ids[(size_t)n * C + tid];
        keys[tid] = (unsigned long long)ordered(x + 0.f) << 32 | (uint32_t)~id;
        above[tid] = 0;
    }
    if (tid == 0) real = 0;
    float r = -INFINITY, tops = 0.f;
    LaneSum<float> a(0.f);
    if (lane < p.parts) {
        const float *sums = p.part_sums + ((size_t)n * p.parts + lane) * 4;
        r = sums[0];
        a.about(r);
        a.s = sums[1];
        a.st = sums[2];
        tops = sums[3];
    }
    const float M = wave_max(r);
    if (r != M) {  // a part's maxima that are not the row's; of a part of -inf alone they are nothing
        if (r > -INFINITY) a.s += tops;
        tops = 0.f;
    }
    a.move(M);
    const RowStats st(M, wave_sum(tops), wave_sum(a.s), wave_sum(a.st));
    if (tid == 0) write_row(p, n, st);
    write_tokens(p, n, row, st, tid);
    if (p.K == 0) return;
    __syncthreads();
    const int groups = (C + kWave - 1) / kWave, shares = blockDim.x / kWave / groups, share = wave / groups;
    const int mine = wave % groups * kWave + lane;
    if (share < shares) {
        const unsigned long long key = keys[min(mine, C - 1)];
        int count = 0;
#pragma unroll 8
        for (int e = share; e < C; e += shares) count += keys[e] > key;
        if (mine < C && count) atomicAdd(&above[mine], count);
    }
    const int has = __popcll(__ballot(x > -INFINITY));
    if (lane == 0 && has) atomicAdd(&real, has);
    __syncthreads();
    if (x > -INFINITY && above[tid] < p.K) write_alternative(p, n, above[tid], st, x, id);
    if (tid >= real && tid < p.K) write_alternative(p, n, tid, st, -INFINITY, INT_MAX);
}

// Gradient: elementwise, one workgroup per kGradSteps * T granules of a row; the ids that fall into its share are looked for
// once and kept in LDS, in their order, so that ids that repeat add up the same way every time.  At an id the definition is a
// difference, of g and p g of the same token, which is all that a confident target has: of a token that has more than half it is
// formed as g (1 - p) by itself.
constexpr int kGradSteps = 4;

struct GradRow {
    float m, log_sum, entropy, factor, g_entropy;
    // (exp(-200) is 0; a NaN, which m and log_sum of a row without meaning are, stays one)
    __device__ __forceinline__ float log_prob(float x) const {
        return __builtin_elementwise_maximum((x - m) - log_sum, -200.f);
    }
    // factor: the sum of the gradients of all tokens' log probabilities, or of those of the others
    __device__ __forceinline__ float by_others(float p, float lp, float others) const {
        return -p * fmaf(g_entropy, lp + entropy, others);
    }
    __device__ __forceinline__ float operator()(float x) const {
        const float lp = log_prob(x);
        return by_others(__builtin_amdgcn_exp2f(lp * kLog2e), lp, factor);
    }
    // A token of p > 1/2: 1 - p to its relative precision, by log p over what the logarithm of the rounded p is (Kahan's correction)
    __device__ __forceinline__ float likely(float lp, float g, float others) const {
        const float p = __builtin_amdgcn_exp2f(lp * kLog2e), seen = 1.f - p;
        const float rest = seen > 0.f ? seen * (lp * kLog2e) * __builtin_amdgcn_rcpf(__builtin_amdgcn_logf(p)) : -lp;
        return fmaf(g, rest, by_others(p, lp, others));
    }
};

// ONCE: gradients that no cache keeps until they are read
template <typename E, int T, bool ONCE>
__global__ __launch_bounds__(T) void logprobs_grad_kernel(LogprobsGradParams p) {
    constexpr int G = Granule<E>::n;
    const int n = blockIdx.y, tid = threadIdx.x, lane = tid & (kWave - 1);
    const RowView<E> row(static_cast<const E *>(p.logits) + (long long)n * p.stride, p.V);
    E *out = static_cast<E *>(p.grad) + (long long)n * p.grad_stride;
    const int g0 = blockIdx.x * (kGradSteps * T), g1 = min(row.whole, g0 + kGradSteps * T);
    const bool first = blockIdx.x == 0, last = blockIdx.x == gridDim.x - 1;
    const E *body = row.p + row.head;
    // elements of this workgroup
    const int v0 = first ? 0 : row.index(g0), v1 = last ? p.V : row.index(g1);

    __shared__ int hit_id[SPECEE_IDS_MAX], hits;
    __shared__ int all_id[kWave];
    __shared__ float hit_g[SPECEE_IDS_MAX], all_g[kWave], factor;
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
        all_id[lane] = id;
        all_g[lane] = gt;
        if (lane == 0) {
            hits = __popcll(who);
            factor = sum;
        }
    }
    Granule<E> x[kGradSteps];
#pragma unroll
    for (int u = 0; u < kGradSteps; ++u) {
        const int g = g0 + u * T + tid;
        if (g < g1) x[u] = load_granule_once(body + (size_t)g * G);
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
    // d with the gradient g of its token x; of one that has more than half of all, from the sums of its own and the others'
    auto with_id = [&](int id, float g, float x, float d) {
        const float lp = f.log_prob(x);
        if (!(lp > -kLn2)) return d + g;
        float own = 0.f, others = 0.f;
        for (int t = 0; t < p.T; ++t) {
            own += all_id[t] == id ? all_g[t] : 0.f;
            others += all_id[t] == id ? 0.f : all_g[t];
        }
        return f.likely(lp, own, others);
    };
    const bool same = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15) == 0;
#pragma unroll
    for (int u = 0; u < kGradSteps; ++u) {
        const int g = g0 + u * T + tid;
        if (g < g1) {
            const int at = row.index(g);
            float d[G];
#pragma unroll
            for (int j = 0; j < G; ++j) d[j] = f((float)x[u].v[j]);
            for (int h = 0; h < H; ++h) {
                const int j0 = hit_id[h] - at;
                if ((unsigned)j0 < (unsigned)G) {
                    float xh = 0.f, dh = 0.f;
#pragma unroll
                    for (int j = 0; j < G; ++j) {
                        xh = j == j0 ? (float)x[u].v[j] : xh;
                        dh = j == j0 ? d[j] : dh;
                    }
                    dh = with_id(hit_id[h], hit_g[h], xh, dh);
#pragma unroll
                    for (int j = 0; j < G; ++j) d[j] = j == j0 ? dh : d[j];
                }
            }
            Granule<E> o;
#pragma unroll
            for (int j = 0; j < G; ++j) o.v[j] = (E)(empty ? 0.f : d[j]);
            if (same)
                if constexpr (ONCE)
                    __builtin_nontemporal_store(__builtin_bit_cast(uintx4, o), reinterpret_cast<uintx4 *>(out + at));
                else
                    *reinterpret_cast<uintx4 *>(out + at) = __builtin_bit_cast(uintx4, o);
            else
#pragma unroll
                for (int j = 0; j < G; ++j) out[at + j] = o.v[j];
        }
    }
    if (extra >= 0) {
        float d = f(xe);
        for (int h = 0; h < H; ++h)
            if (hit_id[h] == extra) d = with_id(extra, hit_g[h], xe, d);
        out[extra] = (E)(empty ? 0.f : d);
    }
}

}  // namespace

// How rows are dealt out: one workgroup per row, of 1024 threads where no CU has two rows and a row is long enough to give each
// thread two steps (256 x 32000 fp32 with five alternatives 9.6 us, of 512 threads 10.5; 1 x 32000 7.0 and 7.2), else of 512 (511
// x 32000 14.7 us, of 1024 threads 15.7; 1 x 8000 5.1 of either), and of 256 where there are many short ones (one alternative,
// 3317 x 777 fp32 11 us, of 512 threads 18.5; 4096 x 8000 27 and 30, fp16 21 and 29; but 600 x 8000 7.9 and 8.3, 2043 x 32003 46.9
// and 45.3).  A few rows of more than 224 KB in parts of at most 64 KB (fp16: 32 KB), which workgroups of 512 threads hold and a
// second launch joins (1 x 128256 fp32 8.6 us, in one workgroup 14.0; 64 x 128256 14.4 and 17.2, 80 would be 15.9 and 17.3, 100 17.8
// and 17.5; 1 x 50280 8.2 and 8.1).
namespace {
struct Deal {
    int parts, threads, granules;  // granules per thread that are held; 0: in steps
};
Deal deal(int N, int V, bool half) {
    const int whole = V / (half ? 8 : 4), most = (half ? 4 : 8) * kT;  // (8 of fp16 leave the registers)
    if (N > 0 && N <= kLogprobsRowsInParts && whole > 14336 && whole <= kMaxParts * (most - 1)) {
        int parts = std::min(512 / N, kMaxParts);
        while ((whole + parts - 1) / parts + 1 > most) ++parts;
        return Deal{parts, kT, (whole + parts - 1) / parts + 1 <= 4 * kT ? 4 : 8};
    }
    return Deal{1, N <= 256 && whole > 2048 ? 1024 : N > 1024 && whole <= 2048 ? 256 : kT, 0};
}
// More than a few alternatives, which is more than the fewest groups of lanes (16) could bear, in kernels of their own (2043 x 8000
// fp16: 20 of them 19.4 us; five 14.7, in the kernels for many 15.9)
constexpr int kFew = 8;
template <typename E, bool MANY>
hipError_t launch_rows(const LogprobsParams &p, const Deal &d, hipStream_t s) {
    const dim3 grid((unsigned)p.N * p.parts), threads(d.threads);
    if (d.granules == 0) {
        if (d.threads == 1024)
            hipLaunchKernelGGL((logprobs_kernel<E, 1024, MANY>), grid, threads, 0, s, p);
        else if (d.threads == 256)
            hipLaunchKernelGGL((logprobs_kernel<E, 256, MANY>), grid, threads, 0, s, p);
        else
            hipLaunchKernelGGL((logprobs_kernel<E, kT, MANY>), grid, threads, 0, s, p);
        return hipGetLastError();
    }
    if constexpr (sizeof(E) == 4) {
        if (d.granules == 8) hipLaunchKernelGGL((logprobs_held_kernel<E, 8, MANY>), grid, threads, 0, s, p);
    }
    if (d.granules == 4) hipLaunchKernelGGL((logprobs_held_kernel<E, 4, MANY>), grid, threads, 0, s, p);
    // (1 x 128256 fp32, 20 alternatives: 14.9 us with 512 threads, 12.1 with 1024; five: 8.4 and 8.5)
    hipLaunchKernelGGL(logprobs_join_kernel<E>, dim3(p.N), dim3(p.parts * p.K > 128 ? 2 * kJoinMost : kJoinMost), 0, s, p);
    return hipGetLastError();
}
}  // namespace

int logprobs_parts(int N, int V, bool half) {
    return deal(N, V, half).parts;
}

hipError_t launch_logprobs(const LogprobsParams &p, bool half, hipStream_t s) {
    const Deal d = deal(p.N, p.V, half);
    if (p.K > kFew) return half ? launch_rows<half_t, true>(p, d, s) : launch_rows<float, true>(p, d, s);
    return half ? launch_rows<half_t, false>(p, d, s) : launch_rows<float, false>(p, d, s);
}

namespace {
template <typename E, int T, bool ONCE>
hipError_t launch_grad(const LogprobsGradParams &p, int whole, hipStream_t s) {
    const int share = kGradSteps * T;
    hipLaunchKernelGGL((logprobs_grad_kernel<E, T, ONCE>), dim3(whole < 1 ? 1 : (whole + share - 1) / share, p.N), dim3(T), 0, s, p);
    return hipGetLastError();
}

template <typename E>
hipError_t launch_grad(const LogprobsGradParams &p, hipStream_t s) {
    // no cache keeps more than this until it is read (4096 x 32000 fp16, 262 MB: 101 us without the hint, 91 with it; 128 MB of
    // fp32 51.6 and 48.0, 96 MB of fp16 38.5 and 38.2; but 77 MB of fp32 29.0 and 30.6)
    const bool once = (size_t)p.N * p.V * sizeof(E) > (96u << 20);
    // many short rows by two wavefronts each (4096 x 1030 fp32 14.2 -> 9.4 us, 4096 x 2000 fp16 15.7 -> 10.4; but 60 x 777 2.9 and
    // 3.2)
    const int whole = p.V / Granule<E>::n;
    if (p.N > 512 && whole <= kGradSteps * 128)
        return once ? launch_grad<E, 128, true>(p, whole, s) : launch_grad<E, 128, false>(p, whole, s);
    return once ? launch_grad<E, kT, true>(p, whole, s) : launch_grad<E, kT, false>(p, whole, s);
}
}  // namespace

hipError_t launch_logprobs_grad(const LogprobsGradParams &p, bool half, hipStream_t s) {
    return half ? launch_grad<half_t>(p, s) : launch_grad<float>(p, s);
}

}  // namespace specee
