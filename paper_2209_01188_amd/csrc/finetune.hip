// Scoring and the client's ends of a fine-tuning step: log probabilities, distillation loss with its gradient, gradient of
// the embedding lookup.  (The LM head's backward product is in head_backward.hip.)
#include <math.h>

#include "../../include/petals_finetune.h"
#include "../../include/petals_span.h"
#include "client_internal.h"
#include "common.h"
#include "host_util.h"
#include "ln_backward.h"

namespace {

// ------------------------------------------------------------------------------------ a row's softmax statistics
//
// One pass over the row: every thread keeps the maximum m of what it has seen, S = sum of e^t and D = sum of t e^t with
// t = (l - m) / T, and rescales the two when m grows.  The exponentials are fp32 (base 2: x = t log2(e), D in that unit as
// well); the sums are fp64, so that S - 1, what is left beside the largest token, keeps its digits where that token has
// nearly everything: log S and -D / S are the two parts of the entropy, both >= 0, and nothing cancels between them.
//
// Bound by the bytes of the logits where there are many rows: 1024 x 250880 with the 20 best of each in 189 us, 5.4 TB/s (a copy
// within the memory reaches 4.8); with few rows by the latency of two launches, 1 x 250880 in 13 us with 5 of them, in 18 with 50.
constexpr double LN2 = 0.69314718055994530942, LOG2E = 1.4426950408889634074;

struct RowStat {
    float m;
    double S, D;
};
// s in terms of a maximum m that is at least its own.  (A part without any logit above -infinity: S = D = 0, or NaN, and its
// distance to m is no number to multiply with.)
__device__ __forceinline__ void rescale(RowStat &s, float m, double invT) {
    if (s.m != -INFINITY) {
        const double t = ((double)s.m - m) * invT, e = exp_f64(t);
        s.D = e * fma(t * LOG2E, s.S, s.D);
        s.S *= e;
    }
    s.m = m;
}
__device__ __forceinline__ void merge(RowStat &s, RowStat o, double invT) {
    const float m = fmaxf(s.m, o.m);
    rescale(s, m, invT);
    rescale(o, m, invT);
    s.S += o.S;
    s.D += o.D;
}
__device__ __forceinline__ RowStat wave_merge(RowStat s, double invT) {
    rescale(s, wave_max(s.m), invT);
    return RowStat{s.m, wave_sum(s.S), wave_sum(s.D)};
}
// over the workgroup, in a fixed order; every thread gets it.  sm: NW of them
template <int NW>
__device__ __forceinline__ RowStat block_merge(RowStat s, double invT, RowStat *sm) {
    s = wave_merge(s, invT);
    const int lane = threadIdx.x & 63;
    if (lane == 0) sm[threadIdx.x >> 6] = s;
    __syncthreads();
    s = lane < NW ? sm[lane] : RowStat{-INFINITY, 0.0, 0.0};
    return wave_merge(s, invT);
}
// N further logits of a thread; returns the largest of them
template <int N, bool WITH_D>
__device__ __forceinline__ float accumulate(RowStat &s, const float (&l)[N], float c, double invT) {
    float cm = l[0];
#pragma unroll
    for (int i = 1; i < N; i++) cm = fmaxf(cm, l[i]);
    if (cm > s.m) rescale(s, cm, invT);
    const float m = s.m == -INFINITY ? 0.0f : s.m;
    float d = 0.0f;                                                          // (a step's terms have one sign: their sum in fp32 is off by 2^-20 of itself)
#pragma unroll
    for (int i = 0; i < N; i++) {
        const float x = (l[i] - m) * c, e = __builtin_amdgcn_exp2f(x);
        s.S += (double)e;
        if (WITH_D) d = fmaf(e, fmaxf(x, -1e30f), d);                         // (a token ruled out: 0 times a number)
    }
    if (WITH_D) s.D += (double)d;
    return cm;
}

constexpr int ROW_NT = 256, ROW_NW = ROW_NT / 64;   // threads of a workgroup that has a row or a part of one
constexpr int ROW_PER = 16;                         // logits of a thread per step
constexpr int WAVE_STEP = 64 * ROW_PER, ROW_STEP = ROW_NW * WAVE_STEP;
// Workgroups that a call is cut into at least, if it has the steps: 4 and 8 per compute unit.  (Log probabilities of 1024 x 250880
// with 1024, 1536: 188, 205 us, each split starts a list of its own; distillation of 128 x 250880 with 1024, 2048: 74, 73.)
constexpr int LOGPROBS_GROUPS = 1024, DISTILL_GROUPS = 2048;
constexpr int MAX_GRID = 1 << 14;                   // rows of a launch
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));     // rows of an odd vocabulary begin anywhere

// A call of few rows shares each row out over workgroups, a whole number of steps to each.
struct RowSplit {
    int splits, range;
};
RowSplit row_split(int M, int V, int groups, int most) {
    const int steps = (V + ROW_STEP - 1) / ROW_STEP, want = max(1, min(min(steps, most), (groups + M - 1) / M)), per = (steps + want - 1) / want;
    return RowSplit{(steps + per - 1) / per, per * ROW_STEP};
}

// logit 4 q + e of a thread's step is column v0 + 256 q + 4 lane + e, v0 = the wave's first; what lies behind the row is -infinity
template <bool LAST>
__device__ __forceinline__ void load_logits(const float *row, int v0, int end, float (&l)[ROW_PER]) {
    const int first = v0 + 4 * (threadIdx.x & 63);
    if (v0 + WAVE_STEP <= end) {
#pragma unroll
        for (int q = 0; q < ROW_PER / 4; q++) {
            const v4f f = LAST ? __builtin_nontemporal_load((const v4f_any *)(row + first + 256 * q)) : *(const v4f_any *)(row + first + 256 * q);
#pragma unroll
            for (int e = 0; e < 4; e++) l[4 * q + e] = f[e];
        }
    } else {
#pragma unroll
        for (int i = 0; i < ROW_PER; i++) {
            const int v = first + 256 * (i >> 2) + (i & 3);
            l[i] = v < end ? row[v] : -INFINITY;
        }
    }
}
// the steps of this wave in [begin, end): step(first column, logits).  (The other waves of the compute unit cover the wait for
// a step's logits: with the next step's asked for ahead, in 16 more registers, 1024 x 250880 took 223 instead of 218 us.)
template <int NT, bool LAST = false, typename F>
__device__ __forceinline__ void walk_row(const float *row, int begin, int end, F step) {
    for (int v = begin + (threadIdx.x >> 6) * WAVE_STEP; v < end; v += NT / 64 * WAVE_STEP) {
        float l[ROW_PER];
        load_logits<LAST>(row, v, end, l);
        step(v, l);
    }
}

// ------------------------------------------------------------------------------------ the largest logits of a row
//
// A key is (value, lower index first) as one 64-bit number; no two are equal.  A wave keeps the best keys it has seen in falling order
// in LDS.  A step's logits are compared with the last key that still counts; what passes, after the first few hundred logits of random
// order little, waits in LDS as well, and goes in many at a time: each key's place in the list is the number of larger ones.  The waves
// of a workgroup share what they know of the top_k-th best.  (Keys inserted one by one, 120 cycles each, every wave for itself: the 50
// best of 1 x 250880 54 us instead of 18, of 300 x 50257 87 instead of 38, of 2048 x 250880 456 instead of 376; the 5 best of 1 x 250880
// 11.5 instead of 13.)
__device__ __forceinline__ uint32_t order_key(float f) {                   // orders like the floats (-0 as +0)
    const uint32_t u = __float_as_uint(f + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint64_t key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float((u & 0x80000000u) ? u & 0x7fffffffu : ~u);
}
// (in range also where a row of NaN has left a place of the list empty)
__device__ __forceinline__ int key_index(uint64_t key) { return key ? (int)~(uint32_t)key : 0; }
constexpr int LIST = 64, LIST_FLUSH = 16;                                  // at least the most a caller can ask for
static_assert(PETALS_LOGPROBS_TOP_MAX <= LIST, "a lane for each");
// how many keys of a list in falling order are larger
__device__ __forceinline__ int larger_in(const uint64_t *list, uint64_t key) {
    int n = 0;
#pragma unroll
    for (int step = LIST / 2; step; step /= 2) n += list[n + step - 1] > key ? step : 0;
    return n + (list[n] > key);
}
// the rank-th largest of a wave's values (at least that many are as large)
__device__ __forceinline__ float wave_ranked(float v, int rank) {
    int above = 0;
#pragma unroll
    for (int i = 0; i < 64; i++) above += __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), i)) > v;
    return -wave_max(above < rank ? -v : -INFINITY);
}
struct TopList {
    uint64_t *list;                                // of this wave, in LDS: its list, and what waits
    // What every wave has a share of the top_k keys of, in LDS: all together have top_k that reach the lowest of these.  (They rise while
    // others read them; an old one is a bound as well, so the results do not depend on when it is read.)
    volatile uint64_t *reached = nullptr;
    uint64_t floor = 0;                            // what is no larger does not come in
    int waiting = 0;
    __device__ __forceinline__ TopList(uint64_t (*lists)[2 * LIST]) : list(lists[threadIdx.x >> 6]) { list[threadIdx.x & 63] = 0; }
    // from here on only values from this one on
    __device__ __forceinline__ void start(float value) { floor = ((uint64_t)order_key(value) << 32) - 1; }
    __device__ __forceinline__ void offer(uint64_t key, int top_k) {      // one key per lane, 0: none
        unsigned long long who = __ballot(key > floor);
        if (!who) return;
        if (waiting + __popcll(who) > LIST) {
            flush(top_k);
            who = __ballot(key > floor);
        }
        if (key > floor) list[LIST + waiting + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = key;
        waiting += __popcll(who);
    }
    __device__ __forceinline__ void flush(int top_k) {
        const int lane = threadIdx.x & 63;
        const uint64_t a = list[lane], b = lane < waiting ? list[LIST + lane] : 0;
        int at_a = lane, at_b = larger_in(list, b);
#pragma unroll 4
        for (int i = 0; i < waiting; i++) {
            const uint64_t k = list[LIST + i];
            at_a += k > a;
            at_b += k > b;
        }
        place(a, at_a, b, at_b);
        waiting = 0;
        floor = max(floor, list[top_k - 1]);
        if (reached) {
            if (lane == 0) reached[threadIdx.x >> 6] = list[share(top_k) - 1];
            uint64_t lowest = reached[0];
#pragma unroll
            for (int w = 1; w < ROW_NW; w++) lowest = min(lowest, (uint64_t)reached[w]);
            floor = max(floor, lowest);
        }
    }
    static __device__ __forceinline__ int share(int top_k) { return (top_k + ROW_NW - 1) / ROW_NW; }
    // the list becomes these keys at their places (of those that are none, 0, there may be several at one place)
    __device__ __forceinline__ void place(uint64_t a, int at_a, uint64_t b, int at_b) {
        list[threadIdx.x & 63] = 0;
        if (a && at_a < LIST) list[at_a] = a;
        if (b && at_b < LIST) list[at_b] = b;
    }
    // the first wave's becomes that of all (nw waves have one), for the first wave to read
    __device__ __forceinline__ void join(uint64_t (*lists)[2 * LIST], int top_k, int nw) {
        if (waiting) flush(top_k);
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        for (int w = 1; w < nw; w *= 2) {
            __syncthreads();
            if (wave % (2 * w) == 0 && wave + w < nw) {
                const uint64_t *other = lists[wave + w], a = list[lane], b = other[lane];
                const int at_a = lane + larger_in(other, a), at_b = lane + larger_in(list, b);
                place(a, at_a, b, at_b);
            }
        }
    }
};

struct LogprobsOut {
    const float *logits;
    const int32_t *tokens;
    float *logprob, *entropy;
    int32_t *top;
    float *top_logprob;
};
// the results of a row from its statistics (in every thread) and, in the first wave, the row's list
__device__ __forceinline__ void logprobs_store(const LogprobsOut &o, int t, int V, double invT, int top_k, const RowStat &s, const uint64_t *top) {
    const double lse = log(s.S);                            // above (m / T)
    const bool none = s.S == 0.0;
    if (threadIdx.x == 0) {
        if (o.logprob) {
            const int v = o.tokens[t];
            o.logprob[t] = v < 0 || v >= V ? 0.0f : none ? -INFINITY : (float)(((double)o.logits[(size_t)t * V + v] - s.m) * invT - lse);
        }
        if (o.entropy) o.entropy[t] = none ? 0.0f : (float)(lse - LN2 * s.D / s.S);
    }
    if ((int)threadIdx.x < top_k) {                         // at most 64
        o.top[(size_t)t * top_k + threadIdx.x] = key_index(top[threadIdx.x]);
        o.top_logprob[(size_t)t * top_k + threadIdx.x] = none ? -INFINITY : (float)(((double)key_value(top[threadIdx.x]) - s.m) * invT - lse);
    }
}

// workgroup (split, row): the split's part of the row, and with one split the results
__global__ void __launch_bounds__(ROW_NT) k_logprobs(LogprobsOut o, int V, int range, double invT, int top_k, RowStat *__restrict__ stats,
                                                     uint64_t *__restrict__ tops) {
    __shared__ RowStat sm[ROW_NW];
    __shared__ uint64_t lists[ROW_NW][2 * LIST];
    __shared__ uint64_t reached[ROW_NW];
    __shared__ float sf[ROW_NW];
    const int t = blockIdx.y, lane = threadIdx.x & 63, begin = blockIdx.x * range, end = min(V, begin + range);
    const bool all_waves = begin + (ROW_NW - 1) * WAVE_STEP < end;
    const float c = (float)(invT * LOG2E);
    RowStat s{-INFINITY, 0.0, 0.0};
    TopList list(lists);
    walk_row<ROW_NT>(o.logits + (size_t)t * V, begin, end, [&](int v0, const float (&l)[ROW_PER]) {
        const float most = accumulate<ROW_PER, true>(s, l, c, invT);
        // The bound to begin with: of each lane's largest of the first step, at least top_k in the workgroup are as large, if all waves have
        // some; else in the wave.
        if (top_k && v0 < begin + ROW_STEP) {
            float bound = wave_ranked(most, all_waves ? TopList::share(top_k) : top_k);
            if (all_waves) {
                if (lane == 0) {
                    sf[threadIdx.x >> 6] = bound;
                    reached[threadIdx.x >> 6] = 0;
                }
                __syncthreads();
                list.reached = reached;
#pragma unroll
                for (int w = 0; w < ROW_NW; w++) bound = fminf(bound, sf[w]);
            }
            list.start(bound);
        }
        if (top_k && __ballot(!(most < key_value(list.floor + 1)))) {
#pragma unroll
            for (int i = 0; i < ROW_PER; i++) {
                const int v = v0 + 4 * lane + 256 * (i >> 2) + (i & 3);
                list.offer(v < end ? (uint64_t)order_key(l[i]) << 32 | (uint32_t)~v : 0, top_k);
            }
            if (list.waiting >= LIST_FLUSH) list.flush(top_k);
        }
    });
    s = block_merge<ROW_NW>(s, invT, sm);
    if (top_k) list.join(lists, top_k, ROW_NW);
    if (gridDim.x == 1) {
        logprobs_store(o, t, V, invT, top_k, s, lists[0]);
        return;
    }
    const size_t at = (size_t)t * gridDim.x + blockIdx.x;
    if (threadIdx.x == 0) stats[at] = s;
    if ((int)threadIdx.x < top_k) tops[at * top_k + threadIdx.x] = lists[0][threadIdx.x];
}

// What the splits of a row have found.  Of their lists, in falling order, the top_k-th largest of the first keys of each, together some
// 2 top_k, is a bound that all but a few do not reach.
template <int JOIN_NT>
__global__ void __launch_bounds__(JOIN_NT) k_logprobs_join(LogprobsOut o, int V, int splits, double invT, int top_k,
                                                           const RowStat *__restrict__ stats, const uint64_t *__restrict__ tops) {
    constexpr int JOIN_NW = JOIN_NT / 64;
    __shared__ uint64_t lists[JOIN_NW][2 * LIST], firsts[LOGPROBS_GROUPS + 2 * LIST], bound;
    const int t = blockIdx.x, n = splits * top_k, lane = threadIdx.x & 63;
    const uint64_t *keys = tops + (size_t)t * n;
    uint64_t key = (int)threadIdx.x < n ? keys[threadIdx.x] : 0;                   // (asked for early)
    RowStat s{-INFINITY, 0.0, 0.0};
    for (int i = lane; i < splits; i += 64) merge(s, stats[(size_t)t * splits + i], invT);          // by every wave
    if (top_k) {
        const int each = min(top_k, (2 * top_k + splits - 1) / splits), some = splits * each;          // top_k .. splits + 2 top_k
        for (int i = threadIdx.x; i < some; i += JOIN_NT) firsts[i] = keys[i / each * top_k + i % each];
        if (threadIdx.x == 0) bound = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < some; i += JOIN_NT) {
            const uint64_t f = firsts[i];
            int larger = 0;
#pragma unroll 8
            for (int j = 0; j < some; j++) larger += firsts[j] > f;
            if (f && larger == top_k - 1) bound = f - 1;
        }
        __syncthreads();
        TopList list(lists);
        list.floor = bound;
        for (int i = threadIdx.x; i < (n + 63) / 64 * 64; i += JOIN_NT) {
            list.offer(key, top_k);
            key = i + JOIN_NT < n ? keys[i + JOIN_NT] : 0;
        }
        list.join(lists, top_k, min(JOIN_NW, (n + 63) / 64));
    }
    s = wave_merge(s, invT);
    logprobs_store(o, t, V, invT, top_k, s, lists[0]);
}

// ------------------------------------------------------------------------------------ distillation
//
// Two passes over the logits: the softmax statistics, then w q.  From DISTILL_WHOLE rows on a workgroup has a row and both passes: the
// second finds the logits in the cache in front of the memory, and workgroups that read run beside others that write.  Fewer rows are cut
// into parts, with a launch for each pass.
//
// Bound by the memory: 2048 x 250880 in 870 us (a copy of the logits takes 862), 701 x 50257 in 74 (59).  Rows as a whole against parts with
// a launch for each pass: 64 x 250880 54 and 36 us, 128 67 and 68, 191 94 and 100; 128 x 50257 24 and 21, 150 25 and 28, 300 39 and 44,
// 2048 196 and 303.  512 against 1024 threads to a row: 300 x 20000 20 and 25 us, 701 x 50257 71 and 72, 701 x 100003 140 and 133, 2048 x
// 250880 1086 and 955.  Few rows wait for two launches: 1 x 20000 12.3 us (13.2 where the workgroup of a row's first part had the list).
struct DistillIn {
    const float *logits;
    const int32_t *ids;
    const float *vals;
    const float *loss_grad;
    float *loss, *grad;
    int V, K, range;
    double T, invT;
};
struct DistillPart {                   // of a row and split
    float m;
    double S;
};
struct DistillRow {                    // of a row, from its list
    double max, norm;                  // of the teacher's logits, and 1 / sum of e^((logit - max) / T)
    double term, mass;                 // sum p (log p - (z - ref) / T) and sum p: with log q = z / T - lse the loss is T^2 (term + mass (lse - ref / T))
    double ref;                        // the list's largest z, so that large logits cancel exactly
    int listed;
};
constexpr int DISTILL_WHOLE = 140, DISTILL_WIDE = 65536;     // rows from which on one is a workgroup's; vocabulary beyond which it has 1024 threads, not 512
template <int NT>
constexpr int LIST_PER = (PETALS_DISTILL_TOP_MAX + NT - 1) / NT;

// entry k of a row's list; an entry that counts for nothing has value -infinity
__device__ __forceinline__ float teacher_entry(const DistillIn &d, int t, int k, int &id) {
    id = -1;
    if (k >= d.K) return -INFINITY;
    id = d.ids[(size_t)t * d.K + k];
    if (id < 0 || id >= d.V) id = -1;
    return id < 0 ? -INFINITY : d.vals[(size_t)t * d.K + k];
}

// PARTS: the logits of a part of the row (part), or the list (part null); otherwise both, of the whole row
template <int NT, bool PARTS>
__device__ __forceinline__ void distill_stats(const DistillIn &d, int t, int split, DistillPart *part, DistillRow *out, RowStat *sm, double *sd,
                                              float *sf) {
    const float *row = d.logits + (size_t)t * d.V;
    const float c = (float)(d.invT * LOG2E);
    const int begin = split * d.range, end = min(d.V, begin + d.range);
    float val[LIST_PER<NT>], mx = -INFINITY;
    int id[LIST_PER<NT>];
    bool some = false;
#pragma unroll
    for (int i = 0; i < LIST_PER<NT>; i++) {
        val[i] = -INFINITY;
        id[i] = -1;
        if (i * NT < d.K) val[i] = teacher_entry(d, t, i * NT + threadIdx.x, id[i]);
        mx = fmaxf(mx, val[i]);
        some |= !(val[i] == -INFINITY);
    }
    const bool listed = __syncthreads_or(some);
    if (!PARTS || !part) {
        DistillRow r{0.0, 0.0, 0.0, 0.0, 0.0, listed};
        if (listed) {
            float z[LIST_PER<NT>], most = -INFINITY;
#pragma unroll
            for (int i = 0; i < LIST_PER<NT>; i++) {
                z[i] = val[i] == -INFINITY ? -INFINITY : row[id[i]];
                most = fmaxf(most, z[i]);
            }
            mx = block_max<NT / 64>(mx, sf);
            most = block_max<NT / 64>(most, sf);
            const double ref = most == -INFINITY ? 0.0 : (double)most;
            double sum = 0.0, term = 0.0, mass = 0.0;
#pragma unroll
            for (int i = 0; i < LIST_PER<NT>; i++)
                if (i * NT < d.K) sum += val[i] == -INFINITY ? 0.0 : exp_f64(((double)val[i] - mx) * d.invT);
            sum = block_sum<NT / 64>(sum, sd);
            const double ls = log(sum);
#pragma unroll
            for (int i = 0; i < LIST_PER<NT>; i++) {
                if (val[i] == -INFINITY) continue;
                const double tt = ((double)val[i] - mx) * d.invT, p = exp_f64(tt) / sum;
                if (!(p == 0.0)) {
                    term += p * (tt - ls - ((double)z[i] - ref) * d.invT);
                    mass += p;
                }
            }
            term = block_sum<NT / 64>(term, sd);
            mass = block_sum<NT / 64>(mass, sd);
            r = DistillRow{(double)mx, 1.0 / sum, term, mass, ref, 1};
        }
        if (threadIdx.x == 0) *out = r;
        if (PARTS) return;
    }
    if (!listed) return;                                   // nobody reads the part
    RowStat s{-INFINITY, 0.0, 0.0};
    walk_row<NT>(row, begin, end, [&](int, const float (&l)[ROW_PER]) { accumulate<ROW_PER, false>(s, l, c, d.invT); });
    s = block_merge<NT / 64>(s, d.invT, sm);
    if (threadIdx.x == 0) *part = DistillPart{s.m, s.S};
}

// The gradient of a workgroup's range (logits and gradient may be the same memory: what a thread overwrites it has read, and
// the list's logits are read before the barrier), and by the first workgroup of the row its loss.  The list's columns get
// theirs, w (q - p) in fp64, after the others.
template <int NT>
__device__ __forceinline__ void distill_grad(const DistillIn &d, int t, int split, int splits, const DistillPart *parts, const DistillRow *stats, int *s_id,
                                             double *s_p) {
    const int lane = threadIdx.x & 63;
    const float *row = d.logits + (size_t)t * d.V;
    const float c = (float)(d.invT * LOG2E);
    const int begin = split * d.range, end = min(d.V, begin + d.range);
    if (!d.grad && split) return;
    const DistillRow r = *stats;
    RowStat s{-INFINITY, 0.0, 0.0};
    if (r.listed) {
        for (int i = lane; i < splits; i += 64) {          // by every wave
            const DistillPart p = parts[i];
            merge(s, RowStat{p.m, p.S, 0.0}, d.invT);
        }
        s = wave_merge(s, d.invT);
    }
    const bool none = s.S == 0.0, zero = !r.listed || none;
    if (split == 0 && threadIdx.x == 0 && d.loss)
        d.loss[t] = !r.listed ? 0.0f : none ? INFINITY : (float)(d.T * d.T * (r.term + r.mass * (((double)s.m - r.ref) * d.invT + log(s.S))));
    if (!d.grad) return;
    float *out = d.grad + (size_t)t * d.V;
    const double w = d.T * (d.loss_grad ? (double)d.loss_grad[t] : 1.0);
    int id[LIST_PER<NT>];
    float at[LIST_PER<NT>];
    if (!zero) {
        bool mine = false;
#pragma unroll
        for (int i = 0; i < LIST_PER<NT>; i++) {
            id[i] = -1;
            const int k = i * NT + threadIdx.x;
            if (i * NT < d.K) {
                const float val = teacher_entry(d, t, k, id[i]);
                if (k < d.K) {
                    s_id[k] = id[i];
                    s_p[k] = val == -INFINITY ? 0.0 : exp_f64(((double)val - r.max) * d.invT) * r.norm;
                }
                if (id[i] < begin || id[i] >= end) id[i] = -1;
                mine |= id[i] >= 0;
            }
        }
        __syncthreads();
        if (mine) {
#pragma unroll
            for (int i = 0; i < LIST_PER<NT>; i++) {
                if (id[i] < 0) continue;
                double p = 0.0;
                for (int j = 0; j < d.K; j++) p += s_id[j] == id[i] ? s_p[j] : 0.0;
                at[i] = (float)(w * (exp_f64(((double)row[id[i]] - s.m) * d.invT) / s.S - p));
            }
        }
        __syncthreads();
    }
    const float f = zero ? 0.0f : (float)(w / s.S), m = s.m;
    const auto store = [&](int v0, const float (&g)[ROW_PER]) {
        if (v0 + WAVE_STEP <= end) {
#pragma unroll
            for (int q = 0; q < ROW_PER / 4; q++)
                __builtin_nontemporal_store(v4f{g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]}, (v4f_any *)(out + v0 + 4 * lane + 256 * q));
        } else {
#pragma unroll
            for (int i = 0; i < ROW_PER; i++) {
                const int v = v0 + 4 * lane + 256 * (i >> 2) + (i & 3);
                if (v < end) out[v] = g[i];
            }
        }
    };
    if (zero) {
        const float g[ROW_PER] = {};
        for (int v0 = begin + (threadIdx.x >> 6) * WAVE_STEP; v0 < end; v0 += NT / 64 * WAVE_STEP) store(v0, g);
        return;
    }
    walk_row<NT, true>(row, begin, end, [&](int v0, const float (&l)[ROW_PER]) {
        float g[ROW_PER];
#pragma unroll
        for (int i = 0; i < ROW_PER; i++) g[i] = f * __builtin_amdgcn_exp2f((l[i] - m) * c);
        store(v0, g);
    });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < LIST_PER<NT>; i++)
        if (id[i] >= 0) out[id[i]] = at[i];                // (entries with the same token write the same)
}

template <int NT>
struct DistillShared {
    RowStat sm[NT / 64];
    double sd[NT / 64];
    float sf[NT / 64];
    int id[PETALS_DISTILL_TOP_MAX];
    double p[PETALS_DISTILL_TOP_MAX];
};
// One of the two passes, a workgroup for each row and split.  In the first, M in front of them have the lists, which take longest.
template <bool SECOND>
__global__ void __launch_bounds__(ROW_NT) k_distill_part(DistillIn d, int M, int splits, DistillPart *__restrict__ parts, DistillRow *__restrict__ rows) {
    __shared__ DistillShared<ROW_NT> sh;
    const int b = (int)blockIdx.x - (SECOND ? 0 : M), t = __builtin_amdgcn_readfirstlane(b < 0 ? (int)blockIdx.x : b / splits), split = b < 0 ? 0 : b - t * splits;
    if (SECOND) distill_grad<ROW_NT>(d, t, split, splits, parts + (size_t)t * splits, rows + t, sh.id, sh.p);
    else distill_stats<ROW_NT, true>(d, t, split, b < 0 ? nullptr : parts + b, rows + t, sh.sm, sh.sd, sh.sf);
}
// both passes of row first + blockIdx.x
template <int NT>
__global__ void __launch_bounds__(NT) k_distill_row(DistillIn d, int first) {
    __shared__ DistillShared<NT> sh;
    __shared__ DistillPart part;
    __shared__ DistillRow row;
    const int t = first + blockIdx.x;
    distill_stats<NT, false>(d, t, 0, &part, &row, sh.sm, sh.sd, sh.sf);
    __syncthreads();
    distill_grad<NT>(d, t, 0, 1, &part, &row, sh.id, sh.p);
}

// ------------------------------------------------------------------------------------ gradient of the lookup
//
// The LayerNorm's derivative is linear in the gradient, and its statistics belong to the token, not to the position: the
// gradients of a token's positions are summed first and go through it once.
//
// Places in token order by counting: place of position i = number of j with (token_j, j) < (token_i, i).  No order of
// atomics enters, and a call of a few thousand positions is a few million comparisons.
//
// 4096 x 4096 with 1300 different tokens: places 7.5 us, sums and short lists 19.5, the long lists' tokens 5.5; its 65 MB (gradients
// once, matrix rows, results) are 14 us at the rate of a copy.  Few rows (128 x 4096, 16 tokens: 12 us) wait for three launches, each
// of which reads an address before it reads a row.
struct __align__(16) Place {
    int position, token, before, count;      // a position and its token; how many earlier ones have the same, and how many in all
};
// A token's list of fewer than RUN_PIECE positions is one workgroup's, the whole row of each.  A longer one goes in pieces of 32 to 63
// positions, and a workgroup has 1024 columns of one: few tokens that stand everywhere are spread over the chip as well as many.
constexpr int RUN_PIECE = 32, PIECE_COLUMNS = 1024;
constexpr int PLACE_ROWS = 16;        // positions of a workgroup, compared with all of the call's by 64 groups of 16 threads

// first: a byte per place, 1 where a token begins
__global__ void __launch_bounds__(1024) k_token_places(const int32_t *__restrict__ ids, int M, int V, Place *__restrict__ places,
                                                       uint8_t *__restrict__ first) {
    constexpr int TILE = 4096;                         // ids in LDS at a time
    __shared__ __align__(16) int tile[TILE];
    __shared__ int sums[3][64][PLACE_ROWS];
    const int g = threadIdx.x / PLACE_ROWS, r = threadIdx.x % PLACE_ROWS, i0 = blockIdx.x * PLACE_ROWS, i = i0 + r;
    const int own = min(max(ids[min(i, M - 1)], 0), V - 1);
    int place = 0, n_before = 0, n_all = 0;
    for (int j0 = 0; j0 < M; j0 += TILE) {
        const int here = min(TILE, (M - j0 + 3) / 4 * 4);
        __syncthreads();
        for (int u = threadIdx.x; u < here; u += 1024) tile[u] = j0 + u < M ? min(max(ids[j0 + u], 0), V - 1) : 0x7fffffff;      // (no token)
        __syncthreads();
        // four ids at a time; of those before this workgroup's positions equal ones count as less, of its own those before i
        for (int q = g * 4; q < here; q += 256) {
            const v4i o = *(const v4i *)(tile + q);
            const int j = j0 + q;
            if (j + 4 <= i0 || j >= i0 + PLACE_ROWS) {
                const int border = own + (j < i0);
                int n = 0;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    place += o[e] < border;
                    n += o[e] == own;
                }
                n_all += n;
                n_before += j < i0 ? n : 0;
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const bool same = o[e] == own, before = same && j + e < i;
                    place += o[e] < own || before;
                    n_all += same;
                    n_before += before;
                }
            }
        }
    }
    sums[0][g][r] = place;
    sums[1][g][r] = n_before;
    sums[2][g][r] = n_all;
    __syncthreads();
    if (threadIdx.x < 64) {                                                         // 4 lanes share a position's 64 sums
        const int p = threadIdx.x >> 2, part = threadIdx.x & 3, token = __shfl(own, p);
        uint32_t n[3];
#pragma unroll
        for (int c = 0; c < 3; c++) {
            n[c] = 0;
#pragma unroll
            for (int u = 0; u < 16; u++) n[c] += sums[c][part * 16 + u][p];
            n[c] = group_reduce<4>(n[c], [](uint32_t a, uint32_t b) { return a + b; });
        }
        if (part == 0 && i0 + p < M) {
            places[n[0]] = Place{i0 + p, token, (int)n[1], (int)n[2]};
            first[n[0]] = n[1] == 0;
        }
    }
}

// How many pieces a list of n positions has, each of RUN_PIECE but the last, which takes what is left over as well (0: not in pieces).
// Pieces begin at least RUN_PIECE places apart: their sums are row (place / RUN_PIECE) of `parts`.
__device__ __forceinline__ int run_pieces(int n) { return n / RUN_PIECE; }
// the one of places s RUN_PIECE .. + RUN_PIECE for which holds(place), -1: none; by every wave
template <typename F>
__device__ __forceinline__ int find_place(const Place *__restrict__ places, int s, int M, F holds) {
    const int lane = threadIdx.x & 63, q = s * RUN_PIECE + lane;
    const unsigned long long who = __ballot(lane < RUN_PIECE && q < M && holds(places[min(q, M - 1)]));
    return who ? s * RUN_PIECE + __builtin_ctzll(who) : -1;
}

// Number of different tokens before place p, over the workgroup: each thread's first flags (8 places; the memory behind `first` reaches
// to a multiple of that) asked for early, then the waves' sums, and behind a barrier all of them.
__device__ __forceinline__ uint64_t token_flags(const uint8_t *__restrict__ first, int p, int q) {
    if (q >= p) return 0;
    const uint64_t w = *(const uint64_t *)(first + q);
    return p - q >= 8 ? w : w & ((1ull << (8 * (p - q))) - 1);
}
template <int NT>
__device__ __forceinline__ void count_tokens(const uint8_t *__restrict__ first, int p, uint64_t flags, int *sm) {
    int n = __popcll(flags);
    for (int q = (threadIdx.x + NT) * 8; q < p; q += NT * 8) n += __popcll(token_flags(first, p, q));
    const float of_wave = wave_sum((float)n);                        // at most 2^24 of them
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = (int)of_wave;
}
template <int NT>
__device__ __forceinline__ int counted_tokens(const int *sm) {
    const int lane = threadIdx.x & 63;
    return (int)wave_sum(lane < NT / 64 ? (float)sm[lane] : 0.0f);
}

// One workgroup for each RUN_PIECE places and PIECE_COLUMNS columns, in which a piece may begin; behind those (`pieces` of them) one per
// place, at which a token with a short list may begin.
template <int NT, int PER>
__global__ void __launch_bounds__(NT, PER == 1 ? 8 : 4) k_embed_backward(const __half *__restrict__ grad, int M, int H, const __half *__restrict__ E, const __half *__restrict__ g, float eps,
                                                       const Place *__restrict__ places, const uint8_t *__restrict__ first, int pieces,
                                                       float *__restrict__ parts, int32_t *__restrict__ tokens_out,
                                                       float *__restrict__ grads_out, int32_t *__restrict__ count_out) {
    constexpr int COLS = PIECE_COLUMNS / 8, GROUPS = NT / COLS;
    __shared__ union __align__(16) {
        struct {
            double sd[NT / 64][4];
            int si[NT / 64];
        };
        float sums[GROUPS][PIECE_COLUMNS];
    } sm;
    if ((int)blockIdx.x < pieces) {
        const int per = (H + PIECE_COLUMNS - 1) / PIECE_COLUMNS, s = blockIdx.x / per, c0 = (blockIdx.x - s * per) * PIECE_COLUMNS;
        const int p = find_place(places, s, M, [](const Place &pl) { return pl.before % RUN_PIECE == 0 && pl.before / RUN_PIECE < run_pieces(pl.count); });
        if (p < 0) return;
        const Place pl = places[p];
        const int n = pl.before / RUN_PIECE == run_pieces(pl.count) - 1 ? pl.count - pl.before : RUN_PIECE;
        const int group = threadIdx.x / COLS, k0 = c0 + threadIdx.x % COLS * 8;
        float acc[1][8] = {};
        add_rows<NT, 1, _Float16, 4>(acc, (n - group + GROUPS - 1) / GROUPS, k0, H,
                                     [&](int r) { return (const _Float16 *)grad + (size_t)places[p + group + GROUPS * r].position * H; });
#pragma unroll
        for (int h = 0; h < 2; h++)
            *(v4f *)&sm.sums[group][threadIdx.x % COLS * 8 + 4 * h] = v4f{acc[0][4 * h], acc[0][4 * h + 1], acc[0][4 * h + 2], acc[0][4 * h + 3]};
        __syncthreads();
        for (int k = threadIdx.x; k < min(PIECE_COLUMNS, H - c0); k += NT) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < GROUPS; i++) sum += sm.sums[i][k];
            parts[(size_t)s * H + c0 + k] = sum;
        }
        return;
    }
    const int p = blockIdx.x - pieces;
    const Place pl = places[p];
    if (p == M - 1) {
        count_tokens<NT>(first, M, token_flags(first, M, threadIdx.x * 8), sm.si);
        __syncthreads();
        const int n = counted_tokens<NT>(sm.si);
        if (threadIdx.x == 0) *count_out = n;
        __syncthreads();
    }
    if (pl.before || run_pieces(pl.count)) return;
    const uint64_t flags = token_flags(first, p, threadIdx.x * 8);
    LnRow<PER> row;
    ln_load<NT, PER>(row, E + (size_t)pl.token * H, g, H);
    float acc[PER][8] = {};
    add_some_rows<NT, PER, _Float16, 1>(acc, 0, threadIdx.x * 8, H, [&](int) { return (const _Float16 *)grad + (size_t)pl.position * H; });
    add_rows<NT, PER, _Float16, 8>(acc, pl.count - 1, threadIdx.x * 8, H,
                                   [&](int r) { return (const _Float16 *)grad + (size_t)places[p + 1 + r].position * H; });
    count_tokens<NT>(first, p, flags, sm.si);
    ln_backward<NT, PER>(acc, row, H, eps, sm.sd);
    const int u = counted_tokens<NT>(sm.si);
    ln_store<NT, PER>(acc, grads_out + (size_t)u * H, H);
    if (threadIdx.x == 0) tokens_out[u] = pl.token;
}

// The lists that went in pieces: workgroup s looks for one that begins at places s RUN_PIECE ..  (Joined in the launch before, by the
// workgroup that is done last with a list: 34 us there instead of 20 + 5 here, the eight L2 caches have to be brought in line.)
template <int NT, int PER>
__global__ void __launch_bounds__(NT) k_embed_backward_join(int M, int H, const __half *__restrict__ E, const __half *__restrict__ g, float eps,
                                                            const Place *__restrict__ places, const uint8_t *__restrict__ first,
                                                            const float *__restrict__ parts, int32_t *__restrict__ tokens_out,
                                                            float *__restrict__ grads_out) {
    __shared__ double sd[NT / 64][4];
    __shared__ int si[NT / 64];
    const int p = find_place(places, blockIdx.x, M, [](const Place &pl) { return pl.before == 0 && run_pieces(pl.count) > 0; });
    if (p < 0) return;
    const Place pl = places[p];
    LnRow<PER> row;
    const uint64_t flags = token_flags(first, p, threadIdx.x * 8);
    ln_load<NT, PER>(row, E + (size_t)pl.token * H, g, H);
    float acc[PER][8] = {};
    add_rows<NT, PER, float, 4>(acc, run_pieces(pl.count), threadIdx.x * 8, H, [&](int r) { return parts + (size_t)(p / RUN_PIECE + r) * H; });
    count_tokens<NT>(first, p, flags, si);
    ln_backward<NT, PER>(acc, row, H, eps, sd);
    const int u = counted_tokens<NT>(si);
    ln_store<NT, PER>(acc, grads_out + (size_t)u * H, H);
    if (threadIdx.x == 0) tokens_out[u] = pl.token;
}

// A call of few positions in one launch: workgroup i has the token of position i if that is its first.  Against the launches above, 16 tokens
// in turn: 128 x 1024 6.9 us instead of 8.9, 128 x 4096 7.1 instead of 9.8; 31 different ones of 14336 7.9 instead of 10.2.  One compute unit
// reads some 65 GB/s, so the limit is where a single token costs some 5 us more than in pieces (128 x 4096 16 and 11); 256 x 1024 9 and 9, with
// a single token 21 and 11.
constexpr int FEW = 128;              // positions at most
constexpr size_t FEW_VALUES = 512 << 10;
template <int NT, int PER>
__global__ void __launch_bounds__(NT) k_embed_backward_few(const int32_t *__restrict__ ids, const __half *__restrict__ grad, int M, int V, int H,
                                                           const __half *__restrict__ E, const __half *__restrict__ g, float eps,
                                                           int32_t *__restrict__ tokens_out, float *__restrict__ grads_out,
                                                           int32_t *__restrict__ count_out) {
    constexpr int GROUPS = NT / FEW;
    __shared__ __align__(16) int token[FEW];
    __shared__ int list[FEW], first[GROUPS][FEW], n_same[NT / 64], n_less[NT / 64], n_all[NT / 64];
    __shared__ double sd[NT / 64][4];
    const int i = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = threadIdx.x % FEW, group = threadIdx.x / FEW;
    const int own = min(max(ids[i], 0), V - 1), mine = j < M ? min(max(ids[j], 0), V - 1) : 0x7fffffff;      // (no token)
    LnRow<PER> row;
    ln_load<NT, PER>(row, E + (size_t)own * H, g, H);
    float acc[PER][8] = {};
    add_some_rows<NT, PER, _Float16, 1>(acc, 0, threadIdx.x * 8, H, [&](int) { return (const _Float16 *)grad + (size_t)i * H; });
    if (group == 0) token[j] = mine;
    const unsigned long long same = __ballot(group == 0 && mine == own);
    if (lane == 0) n_same[wave] = __popcll(same);
    if (__syncthreads_or(mine == own && j < i)) return;
    // the token's positions in order
    int n = 0, before = 0;
#pragma unroll
    for (int w = 0; w < FEW / 64; w++) {
        before += w < wave ? n_same[w] : 0;
        n += n_same[w];
    }
    if (same >> lane & 1) list[before + __popcll(same & ((1ull << lane) - 1))] = j;
    // the first position of token j, by a share of the positions
    int f = FEW;
    for (int q = (M - 1) / (4 * GROUPS) * GROUPS + group; q >= 0; q -= GROUPS) {
        const v4i o = q * 4 < FEW ? *(const v4i *)(token + q * 4) : v4i{-1, -1, -1, -1};
#pragma unroll
        for (int e = 3; e >= 0; e--) f = o[e] == mine ? q * 4 + e : f;
    }
    first[group][j] = f;
    __syncthreads();
    for (int u = 0; u < GROUPS; u++) f = min(f, first[u][j]);
    const bool is_first = group == 0 && j < M && f == j;
    const unsigned long long all = __ballot(is_first), less = __ballot(is_first && mine < own);
    if (lane == 0) {
        n_all[wave] = __popcll(all);
        n_less[wave] = __popcll(less);
    }
    add_rows<NT, PER, _Float16, 8>(acc, n - 1, threadIdx.x * 8, H, [&](int r) { return (const _Float16 *)grad + (size_t)list[r + 1] * H; });
    ln_backward<NT, PER>(acc, row, H, eps, sd);                      // (with a barrier)
    int u = 0, count = 0;
#pragma unroll
    for (int w = 0; w < FEW / 64; w++) {
        u += n_less[w];
        count += n_all[w];
    }
    ln_store<NT, PER>(acc, grads_out + (size_t)u * H, H);
    if (threadIdx.x == 0) {
        tokens_out[u] = own;
        if (i == 0) *count_out = count;                              // (position 0 is its token's first)
    }
}

struct EmbedBackward {
    const int32_t *ids;
    const __half *grad, *E, *g;
    int M, V, H;
    float eps;
    Place *places;
    uint8_t *first;
    float *parts;
    int32_t *tokens_out;
    float *grads_out;
    int32_t *count_out;
};
template <int NT, int PER>
int embed_backward(const EmbedBackward &c, hipStream_t st) {
    if (c.M <= FEW && (size_t)c.M * c.H <= FEW_VALUES) {
        k_embed_backward_few<NT, PER><<<c.M, NT, 0, st>>>(c.ids, c.grad, c.M, c.V, c.H, c.E, c.g, c.eps, c.tokens_out, c.grads_out, c.count_out);
        HIP_TRY(hipGetLastError());
        return PETALS_OK;
    }
    const int runs = c.M < RUN_PIECE ? 0 : (c.M + RUN_PIECE - 1) / RUN_PIECE, pieces = runs * ((c.H + PIECE_COLUMNS - 1) / PIECE_COLUMNS);
    k_token_places<<<(c.M + PLACE_ROWS - 1) / PLACE_ROWS, 1024, 0, st>>>(c.ids, c.M, c.V, c.places, c.first);
    HIP_TRY(hipGetLastError());
    k_embed_backward<NT, PER><<<pieces + c.M, NT, 0, st>>>(c.grad, c.M, c.H, c.E, c.g, c.eps, c.places, c.first, pieces, c.parts, c.tokens_out,
                                                           c.grads_out, c.count_out);
    HIP_TRY(hipGetLastError());
    if (runs) {
        k_embed_backward_join<NT, PER><<<runs, NT, 0, st>>>(c.M, c.H, c.E, c.g, c.eps, c.places, c.first, c.parts, c.tokens_out, c.grads_out);
        HIP_TRY(hipGetLastError());
    }
    return PETALS_OK;
}

int check_call(const petals_client_config &cfg, int32_t M) {
    if (M < 1) return ps_fail(PETALS_ERR_INVALID_ARG, "M must be positive");
    if (M > cfg.max_rows_per_call) return ps_fail(PETALS_ERR_CAPACITY, "%d rows exceed max_rows_per_call %d", M, cfg.max_rows_per_call);
    if (cfg.vocab > 1 << 30) return ps_fail(PETALS_ERR_UNSUPPORTED, "vocabulary %d exceeds 2^30", cfg.vocab);
    return PETALS_OK;
}
bool usable_temperature(float t) { return t >= 1e-38f && t < INFINITY; }     // (log2(e) / t is a number in fp32)

}  // namespace

extern "C" {

int petals_client_logprobs(petals_client *client, const float *logits, const int32_t *tokens, int32_t M, float temperature,
                           int32_t top_k, float *logprob_out, float *entropy_out, int32_t *top_out, float *top_logprob_out,
                           void *stream) {
    if (!client || !logits) return ps_fail(PETALS_ERR_INVALID_ARG, "null pointer");
    const ps_client_view c = ps_view(client);
    if (int rc = check_call(*c.cfg, M)) return rc;
    if (!tokens != !logprob_out) return ps_fail(PETALS_ERR_INVALID_ARG, "tokens and logprob_out go together");
    if (top_k < 0) return ps_fail(PETALS_ERR_INVALID_ARG, "top_k must not be negative");
    if (top_k > PETALS_LOGPROBS_TOP_MAX) return ps_fail(PETALS_ERR_UNSUPPORTED, "top_k %d exceeds %d", top_k, PETALS_LOGPROBS_TOP_MAX);
    if (top_k > c.cfg->vocab) return ps_fail(PETALS_ERR_INVALID_ARG, "top_k %d exceeds the vocabulary %d", top_k, c.cfg->vocab);
    if ((top_k > 0) != (top_out != nullptr) || (top_k > 0) != (top_logprob_out != nullptr))
        return ps_fail(PETALS_ERR_INVALID_ARG, "top_out and top_logprob_out go with top_k > 0");
    if (!logprob_out && !entropy_out && !top_out) return ps_fail(PETALS_ERR_INVALID_ARG, "no output requested");
    if (!usable_temperature(temperature)) return ps_fail(PETALS_ERR_INVALID_ARG, "temperature must be positive and finite");
    hipStream_t st = (hipStream_t)stream;
    const int V = c.cfg->vocab;
    const double invT = 1.0 / (double)temperature;
    // per row and split in the workspace: its statistics and its list
    const size_t per = sizeof(RowStat) + sizeof(uint64_t) * top_k;
    const RowSplit sp = row_split(M, V, LOGPROBS_GROUPS, (int)min((size_t)1 << 20, c.scratch_bytes / ((size_t)M * per)));
    RowStat *stats = (RowStat *)c.scratch;
    uint64_t *tops = (uint64_t *)(stats + (size_t)M * sp.splits);
    for (int t0 = 0; t0 < M; t0 += MAX_GRID) {
        const int rows = min(MAX_GRID, M - t0);
        const LogprobsOut r{logits + (size_t)t0 * V, tokens ? tokens + t0 : nullptr, logprob_out ? logprob_out + t0 : nullptr,
                            entropy_out ? entropy_out + t0 : nullptr, top_out ? top_out + (size_t)t0 * top_k : nullptr,
                            top_logprob_out ? top_logprob_out + (size_t)t0 * top_k : nullptr};
        k_logprobs<<<dim3(sp.splits, rows), ROW_NT, 0, st>>>(r, V, sp.range, invT, top_k, stats, tops);
        HIP_TRY(hipGetLastError());
        if (sp.splits > 1) {
            if (sp.splits * top_k <= 1024) k_logprobs_join<256><<<rows, 256, 0, st>>>(r, V, sp.splits, invT, top_k, stats, tops);
            else k_logprobs_join<1024><<<rows, 1024, 0, st>>>(r, V, sp.splits, invT, top_k, stats, tops);
            HIP_TRY(hipGetLastError());
        }
    }
    return PETALS_OK;
}

int petals_client_distill(petals_client *client, const float *logits, int32_t M, const int32_t *teacher_tokens,
                          const float *teacher_logits, int32_t K, float temperature, const float *loss_grad, float *loss_out,
                          float *grad_logits_out, void *stream) {
    if (!client || !logits || !teacher_tokens || !teacher_logits) return ps_fail(PETALS_ERR_INVALID_ARG, "null pointer");
    const ps_client_view c = ps_view(client);
    if (int rc = check_call(*c.cfg, M)) return rc;
    if (K < 1) return ps_fail(PETALS_ERR_INVALID_ARG, "K must be positive");
    if (K > PETALS_DISTILL_TOP_MAX) return ps_fail(PETALS_ERR_UNSUPPORTED, "K %d exceeds %d", K, PETALS_DISTILL_TOP_MAX);
    if (!loss_out && !grad_logits_out) return ps_fail(PETALS_ERR_INVALID_ARG, "neither loss nor gradient requested");
    const void *const outs[] = {loss_out, grad_logits_out}, *const ins[] = {teacher_tokens, teacher_logits, loss_grad};
    for (const void *o : outs)
        for (const void *i : ins)
            if (o && o == i) return ps_fail(PETALS_ERR_INVALID_ARG, "an output and an input alias");
    if (loss_out == logits || loss_out == grad_logits_out) return ps_fail(PETALS_ERR_INVALID_ARG, "loss and logits or gradient alias");
    if (!usable_temperature(temperature)) return ps_fail(PETALS_ERR_INVALID_ARG, "temperature must be positive and finite");
    hipStream_t st = (hipStream_t)stream;
    const int V = c.cfg->vocab;
    DistillIn d{logits, teacher_tokens, teacher_logits, loss_grad, loss_out, grad_logits_out, V, K, V, (double)temperature, 1.0 / (double)temperature};
    if (M >= DISTILL_WHOLE) {
        for (int t0 = 0; t0 < M; t0 += MAX_GRID) {
            const int n = min(MAX_GRID, M - t0);
            if (V <= DISTILL_WIDE) k_distill_row<512><<<n, 512, 0, st>>>(d, t0);
            else k_distill_row<1024><<<n, 1024, 0, st>>>(d, t0);
            HIP_TRY(hipGetLastError());
        }
        return PETALS_OK;
    }
    DistillRow *rows = (DistillRow *)c.scratch;
    DistillPart *parts = (DistillPart *)(rows + M);
    const size_t room = (c.scratch_bytes - sizeof(DistillRow) * M) / ((size_t)M * sizeof(DistillPart));
    const RowSplit sp = row_split(M, V, DISTILL_GROUPS, (int)min((size_t)1 << 20, room));
    d.range = sp.range;
    k_distill_part<false><<<M + M * sp.splits, ROW_NT, 0, st>>>(d, M, sp.splits, parts, rows);
    HIP_TRY(hipGetLastError());
    k_distill_part<true><<<M * sp.splits, ROW_NT, 0, st>>>(d, M, sp.splits, parts, rows);
    HIP_TRY(hipGetLastError());
    return PETALS_OK;
}

int petals_client_embed_backward(petals_client *client, const int32_t *token_ids, const void *grad_hidden, int32_t M,
                                 int32_t *tokens_out, float *grads_out, int32_t *count_out, void *stream) {
    if (!client || !token_ids || !grad_hidden || !tokens_out || !grads_out || !count_out) return ps_fail(PETALS_ERR_INVALID_ARG, "null pointer");
    const ps_client_view c = ps_view(client);
    if (int rc = check_call(*c.cfg, M)) return rc;
    if (M > PETALS_BACKWARD_ROWS_MAX) return ps_fail(PETALS_ERR_UNSUPPORTED, "%d rows exceed %d", M, PETALS_BACKWARD_ROWS_MAX);
    if (token_ids == tokens_out || grad_hidden == (const void *)grads_out) return ps_fail(PETALS_ERR_INVALID_ARG, "an output and an input alias");
    const int H = c.cfg->hidden;
    // M places of 16 bytes and their flags, then a row of partial sums for every RUN_PIECE places: some 17 M + (M / 32 + 1) 4 H bytes
    Place *places = (Place *)c.scratch;
    uint8_t *first = (uint8_t *)(places + M);
    float *parts = (float *)(c.scratch + ((size_t)(first - c.scratch) + M + 255) / 256 * 256);
    const EmbedBackward call{token_ids, (const __half *)grad_hidden, (const __half *)c.p->embeddings, (const __half *)c.p->emb_ln_g, M, c.cfg->vocab, H,
                             c.cfg->ln_eps, places, first, parts, tokens_out, grads_out, count_out};
    hipStream_t st = (hipStream_t)stream;
    return H <= 2048 ? embed_backward<256, 1>(call, st) : H <= 4096 ? embed_backward<512, 1>(call, st)
                     : H <= 8192 ? embed_backward<1024, 1>(call, st) : embed_backward<1024, 2>(call, st);
}

}  // extern "C"
