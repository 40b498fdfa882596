// Routing of tokens to experts: scores, choice, weights, the plan that products grouped by expert go by, and the weights'
// gradient with respect to the logits.
//
// Choice.  A warp takes a token; lane l holds experts l, l + 32, ...  Without a bias scores grow with the logits, so the choice
// goes by the logits themselves, exactly.  With a bias (or where sums of scores decide between groups) the keys are fp32 numbers
// with a known error bound: whenever two keys whose order matters are nearer than that, the warp takes the token again with keys
// in 64 bits.  The choice is therefore that of 64-bit scores, at the cost of fp32 ones.
//
// Plan.  A counting sort in three launches: a block takes a run of tokens and counts its slots by expert; the counts are added up
// over the runs (few experts: by the last launch); a block ranks the slots of its run.  Slots of an expert keep their order, and
// nothing depends on the order in which blocks run.  Few tokens: one cluster does it all.
//
// Bound: for few tokens the launches and a token's chain of dependent steps (1 x 64 top 6 4.2 us in a replayed graph, 1 x 256 in groups
// 5.8, 512 x 8 5.4); for many, each warp's own chain: 16384 x 256 top 8 of four in eight groups take 40 us, 28 of them the choice, whose 1100
// instructions a token fill 55 % of the issue slots, 16 warps an SM waiting on their own results most of the rest.
#include "real_rows.cuh"
#include "tc_ptx.cuh"

namespace {

constexpr int ROUTE_MAX_EXPERTS = 1024, ROUTE_MAX_TOP = 32, ROUTE_MAX_GROUPS = 32;
constexpr int PLAN_THREADS = 1024;
// Threads of a block whose lanes hold V experts each: V numbers of four kinds have to fit the registers (256 experts in groups, one token:
// half a microsecond less with 512 threads of 128 registers than with 1024 of 64; 16384 tokens: the same).
__host__ __device__ constexpr int choose_threads(int v) { return v <= 4 ? 1024 : 512; }
// Warps that rank a run's slots, each with counts of its own.
__host__ __device__ constexpr int rank_warps(int experts) { return experts <= 256 ? 32 : experts <= 512 ? 16 : 8; }
constexpr int MAX_RUNS = 148;                                 // of tokens, a block each
constexpr int ALONE_RUNS = 8;                                 // blocks of the cluster that few tokens are left to
constexpr int64_t ROUTE_MAX_SLOTS = (1ll << 30) - 1;         // (tokens past the last are counted in 31 bits)

struct RouteParams {
    const void *logits;
    int type;
    int64_t ld;
    int tokens, experts, top;
    bool sigmoid, renormalise, by_sums;                       // by_sums: groups are judged by the sum of their two largest keys
    const float *bias;
    int groups, top_groups, each, log_lanes, pitch;           // experts, lanes (a power of two) and key pitch of a group
    uint32_t group_of;                                        // ceil(2^20 / each): e / each = e * group_of >> 20 for e < 1024
    bool whole;                                               // groups of 32: register v holds group v
    float factor;
    const uint8_t *mask;
    int32_t *chosen;
    float *weights;
    int32_t *order, *place, *offsets;                         // NULL: no plan
    int32_t *counts;                                          // [experts][pitch_runs], behind them [experts] rows of each
    int runs, run, pitch_runs;                                // tokens of a run; runs in whole fours
    bool scanned;                                             // counts are added up over the runs by a launch of its own
};

// Numbers as unsigned ones of the same order (not for NaN).  An expert that is not to be chosen has key -infinity.
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
constexpr uint32_t NO_KEY = 0x007FFFFFu;                      // ordered(-infinity); below the key of any finite number whatever its lowest bits
constexpr uint32_t INFINITE_KEY = 0xFF800000u;                // ordered(infinity); NaN (as max.NaN gives it) is above
__device__ __forceinline__ float reciprocal(float v) {       // off by one step at most; 0 where the result would be subnormal
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ unsigned long long ordered(double v) {
    const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.0);
    return !(v > __longlong_as_double(0xFFF0000000000000ll)) ? 0ull : (b >> 63) ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ float warp_add(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v = __fadd_rn(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
__device__ __forceinline__ double warp_add(double v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ float warp_most(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
__device__ __forceinline__ unsigned long long warp_max_key(unsigned long long k) {
    const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
    return (unsigned long long)hi << 32 | lo;
}

__device__ __forceinline__ float load_as_f32(const void *p, int type, int64_t i) {
    if (type == QNN_F32) return static_cast<const float *>(p)[i];
    if (type == QNN_BF16) return to_f32(static_cast<const __nv_bfloat16 *>(p)[i]);
    return to_f32(static_cast<const __half *>(p)[i]);
}
// Element i of a row by its type; the branch lies outside the loop that the caller unrolls.
template <int V> __device__ __forceinline__ void load_row(const void *p, int type, int64_t at, int n, float (&l)[V]) {
    const int lane = threadIdx.x & 31;
    const float none = __int_as_float(0xFF800000);
    if (type == QNN_F32) {
        const float *q = static_cast<const float *>(p) + at;
#pragma unroll
        for (int v = 0; v < V; ++v) l[v] = lane + 32 * v < n ? q[lane + 32 * v] : none;
    } else if (type == QNN_BF16) {
        const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p) + at;
#pragma unroll
        for (int v = 0; v < V; ++v) l[v] = lane + 32 * v < n ? to_f32(q[lane + 32 * v]) : none;
    } else {
        const __half *q = static_cast<const __half *>(p) + at;
#pragma unroll
        for (int v = 0; v < V; ++v) l[v] = lane + 32 * v < n ? to_f32(q[lane + 32 * v]) : none;
    }
}

// Two fp32 keys nearer than this may be in the wrong order.
struct Margin {
    float relative, bias;
    __device__ __forceinline__ bool close(float a, float b) const {
        return __fadd_rn(a, -b) <= __fmaf_rn(relative, __fadd_rn(fmaxf(fabsf(a), fabsf(b)), bias), 1e-37f);
    }
};
__device__ __forceinline__ int group_of(const RouteParams &p, int e) { return (int)((uint32_t)e * p.group_of >> 20); }

// worth: of lane's group (-infinity in lanes without one), which lies at lane `at` of 32, every `stride`-th lane holding one.
// Returns the lanes whose groups stay; `narrow` whether the worst of them is too close to the best of the others.
template <class K> __device__ __forceinline__ unsigned best_groups(const RouteParams &p, K worth, bool holds, int stride, Margin margin, bool &narrow) {
    const int lane = threadIdx.x & 31;
    int better = 0;
#pragma unroll 4
    for (int g = 0; g < p.groups; ++g) {
        const K other = __shfl_sync(0xffffffffu, worth, g * stride);
        better += other > worth || (other == worth && g * stride < lane);
    }
    const unsigned stay = __ballot_sync(0xffffffffu, holds && better < p.top_groups);
    narrow = false;
    if constexpr (sizeof(K) == 4) {
        const uint32_t key = holds ? ordered(__fadd_rn(worth, 0.0f)) : 0u;
        const bool mine = stay >> lane & 1u;
        const float worst = from_ordered(__reduce_min_sync(0xffffffffu, mine ? key : 0xffffffffu));
        const uint32_t next = __reduce_max_sync(0xffffffffu, mine ? 0u : key);
        margin.bias *= 2.0f;                                  // sums of two keys
        margin.relative *= 2.0f;
        narrow = next > NO_KEY && margin.close(worst, from_ordered(next));      // (else only groups without experts go)
    }
    return stay;
}

// The sum of a group's two largest keys; -infinity where there are not two.  A sum of fp32 keys may be beyond fp32: it becomes the largest
// finite number there, near enough to others' for 64 bits to decide.
__device__ __forceinline__ double sum_of_two(double first, double second) {
    return second > __longlong_as_double(0xFFF0000000000000ll) ? first + second : second;
}
__device__ __forceinline__ float sum_of_two(float first, float second) {
    const float most = 3.402823466e38f, inf = __int_as_float(0x7F800000), sum = fmaxf(__fadd_rn(first, second), -most);
    return second > -inf ? (first < inf ? fminf(sum, most) : sum) : second;
}

// The worth of lane >> log_lanes' group: its largest number, or the sum of its two largest.  worth: -infinity where an expert is not to
// be chosen.  By way of shared memory, for groups of any size.
template <class K, int V>
__device__ __forceinline__ K group_worth(const RouteParams &p, const K (&worth)[V], K *scratch) {
    const int lane = threadIdx.x & 31;
    const K none = -(K)__int_as_float(0x7F800000);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = lane + 32 * v;
        if (e < p.experts) scratch[e + group_of(p, e) * (p.pitch - p.each)] = worth[v];
    }
    __syncwarp();
    const int lanes = 1 << p.log_lanes, group = lane >> p.log_lanes, sub = lane & (lanes - 1);
    K first = none, second = none;
    if (group < p.groups)
#pragma unroll 4
        for (int i = sub; i < p.each; i += lanes) {
            const K k = scratch[group * p.pitch + i];
            second = k > first ? first : (k > second ? k : second);
            first = k > first ? k : first;
        }
    __syncwarp();
    for (int d = 1; d < lanes; d <<= 1) {
        const K a = __shfl_xor_sync(0xffffffffu, first, d), b = __shfl_xor_sync(0xffffffffu, second, d);
        const K low = a > first ? first : a, high = a > first ? a : first;
        second = b > second ? b : second;
        second = low > second ? low : second;
        first = high;
    }
    return p.by_sums ? sum_of_two(first, second) : first;
}
// The same for groups of 32 experts: register v of the lanes holds group v, as ordered numbers.  The two largest of every group by
// one exchange that halves the registers at each of its first steps: lane l ends up with group l / (32 / V), where group_worth has it.
template <int V> __device__ __forceinline__ float whole_group_worth(const RouteParams &p, const uint32_t (&worth)[V]) {
    const int lane = threadIdx.x & 31;
    uint32_t first[V], second[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { first[v] = worth[v]; second[v] = NO_KEY; }
#pragma unroll
    for (int half = V / 2, d = 16; d >= 1; half /= 2, d /= 2) {
        if (half >= 1) {
            const bool upper = lane & d;
#pragma unroll
            for (int v = 0; v < half; ++v) {
                const uint32_t a = upper ? first[v] : first[v + half], mine = upper ? first[v + half] : first[v], b = __shfl_xor_sync(0xffffffffu, a, d);
                uint32_t low = min(mine, b);
                if (d < 16) {                                 // (at the first step there is one number of each group)
                    const uint32_t s = upper ? second[v] : second[v + half], own = upper ? second[v + half] : second[v];
                    low = max(low, max(own, __shfl_xor_sync(0xffffffffu, s, d)));
                }
                first[v] = max(mine, b);
                second[v] = low;
            }
        } else {
            const uint32_t b = __shfl_xor_sync(0xffffffffu, first[0], d), t = __shfl_xor_sync(0xffffffffu, second[0], d);
            second[0] = max(min(first[0], b), max(second[0], t));
            first[0] = max(first[0], b);
        }
    }
    return p.by_sums ? sum_of_two(from_ordered(first[0]), from_ordered(second[0])) : from_ordered(first[0]);
}
// Lanes whose group is at bit group << log_lanes of a warp's mask.
__device__ __forceinline__ bool holds_group(const RouteParams &p) {
    const int lane = threadIdx.x & 31;
    return lane >> p.log_lanes < p.groups && (lane & ((1 << p.log_lanes) - 1)) == 0;
}
template <class U, int V> __device__ __forceinline__ void keep_groups(const RouteParams &p, unsigned stay, U (&keys)[V], U no_key) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = lane + 32 * v;
        if (e < p.experts && !(stay >> ((p.whole ? v : group_of(p, e)) << p.log_lanes) & 1u)) keys[v] = no_key;
    }
}

// The `top` largest keys in order, ties to the lowest expert: lane i gets choice i (-1 where nothing is left).
template <class U, int V>
__device__ __forceinline__ int take_top(int top, U (&keys)[V]) {
    const int lane = threadIdx.x & 31;
    int mine = -1;
#pragma unroll 1
    for (int i = 0; i < top; ++i) {
        U best = keys[0];
#pragma unroll
        for (int v = 1; v < V; ++v) best = keys[v] > best ? keys[v] : best;
        best = warp_max_key(best);
        if (best == 0) break;
        int e = 0x7FFFFFFF;
#pragma unroll
        for (int v = V - 1; v >= 0; --v) e = keys[v] == best ? lane + 32 * v : e;
        e = (int)__reduce_min_sync(0xffffffffu, (unsigned)e);
#pragma unroll
        for (int v = 0; v < V; ++v) keys[v] = lane + 32 * v == e ? (U)0 : keys[v];
        if (lane == i) mine = e;
    }
    return mine;
}

// Largest first.
template <int V> __device__ __forceinline__ void sort_keys(uint32_t (&k)[V]) {
    // odd-even merge sort of a power of two of numbers
#pragma unroll
    for (int p = 1; p < V; p *= 2)
#pragma unroll
        for (int q = p; q >= 1; q /= 2)
#pragma unroll
            for (int j = q % p; j + q < V; j += 2 * q)
#pragma unroll
                for (int i = 0; i < q; ++i)
                    if (i + j + q < V && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
                        const uint32_t a = k[i + j], b = k[i + j + q];
                        k[i + j] = max(a, b);
                        k[i + j + q] = min(a, b);
                    }
}

// Choices lo .. hi - 1 with V - 1 - v in the lowest bits of a key in place of its own: the lanes' keys are sorted, and each round a lane
// gives its head away, which carries the expert with it.  Lane i gets choice i (-1 where nothing is left); best: the next head.
template <int V> __device__ __forceinline__ void take_sorted(uint32_t (&keys)[V], int lo, int hi, int &mine, uint32_t &best) {
    const int lane = threadIdx.x & 31;
    constexpr uint32_t LOW = V - 1;
    int from = 0;
    uint32_t key = NO_KEY;
#pragma unroll 1
    for (int i = lo; i < hi && best > NO_KEY; ++i) {
        const int owner = __ffs(__ballot_sync(0xffffffffu, keys[0] == best)) - 1;
        from = lane == i ? owner : from;
        key = lane == i ? best : key;
        const bool gives = lane == owner;
#pragma unroll
        for (int v = 0; v + 1 < V; ++v) keys[v] = gives ? keys[v + 1] : keys[v];
        keys[V - 1] = gives ? NO_KEY : keys[V - 1];
        best = __reduce_max_sync(0xffffffffu, keys[0]);
    }
    if (key > NO_KEY) mine = from + 32 * (int)(LOW - (key & LOW));
}

// 1 / (1 + exp(-x)): for the exponential t of -|x| one over 1 + t, which is between 1 and 2, by Newton's iteration from fp32's.
__device__ __forceinline__ double sigmoid_64(double x) {
    const double t = exp(-fabs(x)), y = 1.0 + t;
    double r = (double)reciprocal((float)y);
    r = fma(r, fma(-y, r, 1.0), r);
    r = fma(r, fma(-y, r, 1.0), r);
    return x >= 0.0 ? r : t * r;
}
// Scores of a token's experts in 64 bits.
template <int V> __device__ __forceinline__ void scores_64(const RouteParams &p, const float (&l)[V], double (&s)[V]) {
    if (p.sigmoid) {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = sigmoid_64((double)l[v]);
    } else {
        float most = l[0];
#pragma unroll
        for (int v = 1; v < V; ++v) most = fmaxf(most, l[v]);
        most = warp_most(most);
        double sum = 0.0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            s[v] = exp((double)l[v] - (double)most);
            sum += s[v];
        }
        sum = warp_add(sum);
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] /= sum;
    }
}
// The groups that stay, by 64-bit keys: a mask for keep_groups.
template <int V>
__device__ __noinline__ unsigned groups_in_64_bits(const RouteParams &p, int64_t token, double *scratch) {
    const int lane = threadIdx.x & 31;
    float l[V];
    load_row<V>(p.logits, p.type, token * p.ld, p.experts, l);
    double s[V];
    scores_64<V>(p, l, s);
    const double none = -(double)__int_as_float(0x7F800000);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float b = p.bias && lane + 32 * v < p.experts ? p.bias[lane + 32 * v] : 0.0f;
        s[v] = l[v] > __int_as_float(0xFF800000) && b == b ? s[v] + (double)b : none;
    }
    bool close;
    return best_groups<double>(p, group_worth<double, V>(p, s, scratch), holds_group(p), 1 << p.log_lanes, Margin{}, close);
}
// All decisions with 64-bit keys; stay: the groups.
template <int V>
__device__ __noinline__ int choose_in_64_bits(const RouteParams &p, int64_t token, unsigned stay) {
    const int lane = threadIdx.x & 31;
    float l[V];
    load_row<V>(p.logits, p.type, token * p.ld, p.experts, l);
    double s[V];
    unsigned long long keys[V];
    if (p.bias) scores_64<V>(p, l, s);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = lane + 32 * v;
        keys[v] = 0;
        if (e < p.experts && l[v] > __int_as_float(0xFF800000)) {
            if (p.bias) s[v] += (double)p.bias[e];
            keys[v] = p.bias ? ordered(s[v]) : ordered((double)l[v]);
        }
    }
    if (p.groups > 1) keep_groups<unsigned long long, V>(p, stay, keys, 0ull);
    return take_top(p.top, keys);
}

// The same by candidates alone: those in lanes 0 .. count - 1 are put in order by 64-bit keys; the keys of all others are
// at most `rest` (NO_KEY: there are none), and where that is too near all decisions are taken so.
template <int V>
__device__ __noinline__ int order_in_64_bits(const RouteParams &p, int64_t token, int candidate, int count, uint32_t rest, Margin margin, unsigned stay) {
    const int lane = threadIdx.x & 31;
    const bool valid = lane < count && candidate >= 0;
    const double none = -(double)__int_as_float(0x7F800000);
    const double x = valid ? (double)load_as_f32(p.logits, p.type, token * p.ld + candidate) : none;
    double key = x;
    if (p.bias) {
        if (p.sigmoid) {
            key = sigmoid_64(x);
        } else {
            float l[V];
            load_row<V>(p.logits, p.type, token * p.ld, p.experts, l);
            float most = l[0];
#pragma unroll
            for (int v = 1; v < V; ++v) most = fmaxf(most, l[v]);
            most = warp_most(most);
            double sum = 0.0;
#pragma unroll 1
            for (int v = 0; v < V; ++v) sum += exp((double)l[v] - (double)most);
            key = exp(x - (double)most) / warp_add(sum);
        }
        key = valid ? key + (double)p.bias[candidate] : none;
    }
    int rank = 0, mine = -1;
#pragma unroll 4
    for (int j = 0; j < count; ++j) {
        const double k = __shfl_sync(0xffffffffu, key, j);
        const int e = __shfl_sync(0xffffffffu, candidate, j);
        rank += e >= 0 && (k > key || (k == key && e < candidate));
    }
#pragma unroll 4
    for (int j = 0; j < count; ++j) {
        const int r = __shfl_sync(0xffffffffu, rank, j), e = __shfl_sync(0xffffffffu, candidate, j);
        if (e >= 0 && r == lane && lane < p.top) mine = e;
    }
    if (rest > NO_KEY) {
        const unsigned last = __ballot_sync(0xffffffffu, valid && rank == p.top - 1);
        const double least = __shfl_sync(0xffffffffu, key, __ffs(last) - 1), most = (double)from_ordered(rest);
        if (p.bias ? margin.close((float)least, (float)most) : !(least > most)) return choose_in_64_bits<V>(p, token, stay);
    }
    return mine;
}

// Choice and weights of one token, by a warp.  Lane i < top writes choice i and returns it (-1: none).
template <int V>
__device__ __forceinline__ int route_token(const RouteParams &p, int64_t token, const float (&bias)[V], float bias_most, double *scratch) {
    const int lane = threadIdx.x & 31;
    float l[V];
    load_row<V>(p.logits, p.type, token * p.ld, p.experts, l);
    const bool there = !p.mask || p.mask[token];
    const float none = __int_as_float(0xFF800000);
    float most = l[0];
#pragma unroll
    for (int v = 1; v < V; ++v) most = max_or_nan(most, l[v]);
    const uint32_t highest = __reduce_max_sync(0xffffffffu, ordered(max_or_nan(most, none)));
    const bool bad = highest > INFINITE_KEY || (!p.sigmoid && highest == INFINITE_KEY);
    most = from_ordered(highest);
    int mine = -1;
    float x = none, scale = 1.0f;                             // the chosen logit, one over softmax's sum
    if (there && !bad && highest > NO_KEY) {
        const bool scored = p.bias || (p.groups > 1 && p.by_sums);
        float s[V];
        if (scored || (!p.sigmoid && !p.renormalise)) {
            if (p.sigmoid) {
#pragma unroll
                for (int v = 0; v < V; ++v) s[v] = reciprocal(__fadd_rn(1.0f, expf(-l[v])));
            } else {
                float sum = 0.0f;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    s[v] = expf(__fadd_rn(l[v], -most));
                    sum = __fadd_rn(sum, s[v]);
                }
                scale = reciprocal(warp_add(sum));
#pragma unroll
                for (int v = 0; v < V; ++v) s[v] = __fmul_rn(s[v], scale);
            }
        }
        uint32_t keys[V];
        // A score is off by at most (sigmoid) expf's two steps, half a step of the sum and one of the quotient, 1.75 * 2^-22; (softmax)
        // besides by the roundings of a difference of logits that matters up to some 88 and of a sum, 40 * 2^-22 in all.  The sum with
        // the bias is off by 2^-24.  Two keys: twice that.
        const Margin margin{(p.sigmoid ? 5.0f : 80.0f) * 2.384185791015625e-07f, bias_most};
        unsigned stay = 0;
        if (p.bias) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                s[v] = l[v] > none ? __fadd_rn(s[v], bias[v]) : none;
                keys[v] = ordered(s[v]);
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) keys[v] = ordered(__fadd_rn(l[v], 0.0f));       // (-0 is 0)
        }
        if (p.groups > 1) {
            float worth;
            if (p.whole && scored && !p.bias) {
                uint32_t by_scores[V];
#pragma unroll
                for (int v = 0; v < V; ++v) by_scores[v] = l[v] > none ? ordered(s[v]) : NO_KEY;
                worth = whole_group_worth<V>(p, by_scores);
            } else if (p.whole) {
                worth = whole_group_worth<V>(p, keys);
            } else {
                float numbers[V];
#pragma unroll
                for (int v = 0; v < V; ++v) numbers[v] = scored && l[v] > none ? s[v] : l[v];
                worth = group_worth<float, V>(p, numbers, reinterpret_cast<float *>(scratch));
            }
            bool close;
            stay = best_groups<float>(p, worth, holds_group(p), 1 << p.log_lanes, margin, close);
            if (close && scored) stay = groups_in_64_bits<V>(p, token, scratch);       // (logits are compared exactly)
            keep_groups<uint32_t, V>(p, stay, keys, NO_KEY);
        }
        constexpr uint32_t LOW = V - 1;
#pragma unroll
        for (int v = 0; v < V; ++v) keys[v] = (keys[v] & ~LOW) | (LOW - v);
        sort_keys<V>(keys);
        uint32_t best = __reduce_max_sync(0xffffffffu, keys[0]);
        take_sorted<V>(keys, 0, p.top, mine, best);
        // Is that order certain?  The keys again, whole, each against the one behind it; the last against the most that any other can be.
        if (mine >= 0) x = load_as_f32(p.logits, p.type, token * p.ld + mine);
        float key = x;
        if (p.bias && mine >= 0)
            key = __fadd_rn(p.sigmoid ? reciprocal(__fadd_rn(1.0f, expf(-x))) : __fmul_rn(expf(__fadd_rn(x, -most)), scale), p.bias[mine]);
        float behind = __shfl_down_sync(0xffffffffu, key, 1);
        int expert = __shfl_down_sync(0xffffffffu, mine, 1);
        bool near;
        if (p.bias) {
            if (lane == p.top - 1) {
                behind = from_ordered(best | LOW);
                expert = best > NO_KEY ? 0 : -1;
            }
            near = lane < p.top && mine >= 0 && expert >= 0 && margin.close(key, behind);
        } else {                                              // (narrow types lose nothing with the lowest bits)
            near = lane < p.top - 1 ? expert >= 0 && (key < behind || (key == behind && mine > expert))
                                    : lane == p.top - 1 && mine >= 0 && p.type == QNN_F32 && ordered(__fadd_rn(key, 0.0f)) <= (best | LOW) && best > NO_KEY;
        }
        bool open = __any_sync(0xffffffffu, near);
        if (open && !p.bias) {                                // equal logits whose lowest bits were not needed (all 0, say) are in order
            load_row<V>(p.logits, p.type, token * p.ld, p.experts, l);
            uint32_t cut = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) cut |= __float_as_uint(l[v]) & LOW;
            open = __any_sync(0xffffffffu, cut != 0);
        }
        if (open) {
            const int count = min(32, p.top + 8);
            take_sorted<V>(keys, p.top, count, mine, best);
            mine = order_in_64_bits<V>(p, token, mine, count, best > NO_KEY ? best | LOW : NO_KEY, margin, stay);
            x = mine >= 0 ? load_as_f32(p.logits, p.type, token * p.ld + mine) : none;
        }
    }
    const float t = expf(-fabsf(x));                          // sigmoid: 1 / (1 + t), or t / (1 + t) below 0
    float w = 0.0f;
    if (p.renormalise) {
        // shares of the chosen scores, with the largest one's power taken out, so that none underflows alone
        const float high = __shfl_sync(0xffffffffu, p.bias ? warp_most(x) : x, 0);      // (without a bias the first is the largest)
        float u = 0.0f;
        if (mine >= 0) {
            if (!p.sigmoid) u = expf(__fadd_rn(x, -high));
            else u = __fmul_rn(x >= 0.0f ? 1.0f : high >= 0.0f ? t : expf(__fadd_rn(x, -high)), reciprocal(__fadd_rn(1.0f, t)));
        }
        const float total = warp_add(u);
        if (mine >= 0) w = __fmul_rn(u, reciprocal(total));
    } else if (mine >= 0) {
        w = p.sigmoid ? __fmul_rn(x >= 0.0f ? 1.0f : t, reciprocal(__fadd_rn(1.0f, t))) : __fmul_rn(expf(__fadd_rn(x, -most)), scale);
    }
    if (lane < p.top) {
        p.chosen[token * p.top + lane] = mine;
        p.weights[token * p.top + lane] = there && bad ? __int_as_float(0x7FC00000) : __fmul_rn(w, p.factor);
    }
    return mine;
}

// A block's shared memory, in words: rows of each expert ahead of its run, in all runs, and in its own; each ranking warp's counts, sums;
// then each warp's keys.
struct RouteSmem {
    static __host__ __device__ int all(int experts) { return experts; }
    static __host__ __device__ int own(int experts) { return 2 * experts; }
    static __host__ __device__ int ranks(int experts) { return 3 * experts; }
    static __host__ __device__ int sums(int experts) { return (3 + rank_warps(experts)) * experts; }
    static __host__ __device__ int keys(int experts) { return (sums(experts) + 40 + 3) / 4 * 4; }
};

// The places of a run's slots, whose warps take segments of whole 32s in order.  count(): each warp's slots of every expert, which needs
// nothing of the other runs; place(): their rows, once the counts are the rows ahead of each warp's.
struct RunRanks {
    const RouteParams &p;
    int32_t *counts;                                          // [warps][experts]
    int first, lo, hi, warps, e0;                             // the run's first slot, the warp's segment; lane's first slot's expert
    unsigned same0;
    __device__ __forceinline__ RunRanks(const RouteParams &params, int run, int32_t *words) : p(params), counts(words + RouteSmem::ranks(params.experts)) {
        const int warp = threadIdx.x >> 5, log_warps = 31 - __clz(min(rank_warps(p.experts), (int)blockDim.x >> 5));
        const int slots = max(0, min(p.tokens - run * p.run, p.run)) * p.top, segment = ((slots - 1) >> (log_warps + 5)) + 1 << 5;      // (fewer than 2^31)
        warps = 1 << log_warps;
        first = run * p.run * p.top;
        lo = min(slots, warp * segment);
        hi = warp < warps ? min(slots - lo, segment) + lo : lo;
        e0 = -1;
        same0 = 0;
    }
    __device__ __forceinline__ void load() { e0 = lo + (int)(threadIdx.x & 31) < hi ? p.chosen[first + lo + (threadIdx.x & 31)] : -1; }
    __device__ __forceinline__ int expert(int i) const {
        const int at = i + (threadIdx.x & 31);
        return i == lo ? e0 : at < hi ? p.chosen[first + at] : -1;      // (up to 32 slots a warp stay in registers)
    }
    __device__ __forceinline__ void count() {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        int32_t *mine = counts + warp * p.experts;
        if (warp < warps)
            for (int e = lane; e < p.experts; e += 32) mine[e] = 0;
        __syncwarp();
        same0 = __match_any_sync(0xffffffffu, e0);
        for (int i = lo; i < hi; i += 32) {
            const int e = expert(i);
            const unsigned same = i == lo ? same0 : __match_any_sync(0xffffffffu, e);
            if (e >= 0 && __ffs(same) - 1 == lane) mine[e] += __popc(same);
            __syncwarp();
        }
    }
    __device__ __forceinline__ void place() {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        int32_t *mine = counts + warp * p.experts;
        for (int i = lo; i < hi; i += 32) {
            const int e = expert(i);
            const unsigned same = i == lo ? same0 : __match_any_sync(0xffffffffu, e);
            const int at = e >= 0 ? mine[e] + __popc(same & ((1u << lane) - 1u)) : -1;
            __syncwarp();
            if (e >= 0 && __ffs(same) - 1 == lane) mine[e] += __popc(same);
            __syncwarp();
            if (i + lane < hi) p.place[first + i + lane] = at;
            if (e >= 0) p.order[at] = first + i + lane;
        }
    }
};

// From the rows of every expert ahead of the run and in all: offsets where it is given, order's rest by `blocks` blocks, and the run's
// places.
__device__ __forceinline__ void plan_run(const RouteParams &p, RunRanks &ranks, int32_t *words, int32_t *offsets, int block, int blocks) {
    const int32_t *ahead = words, *all = words + RouteSmem::all(p.experts);
    int32_t *warp_sums = words + RouteSmem::sums(p.experts);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, each = (p.experts + blockDim.x - 1) / blockDim.x, first = threadIdx.x * each;
    int v = 0;
    for (int e = first; e < min(first + each, p.experts); ++e) v += all[e];
    int incl = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    // every warp adds up the sums ahead of it itself
    const int sum = lane < (int)(blockDim.x >> 5) ? warp_sums[lane] : 0;
    const int before = __reduce_add_sync(0xffffffffu, lane < warp ? sum : 0), total = __reduce_add_sync(0xffffffffu, sum);
    int at = before + incl - v;
    for (int e = first; e < min(first + each, p.experts); ++e) {
        if (offsets) offsets[e] = at;
        int row = at + ahead[e];
#pragma unroll 8
        for (int w = 0; w < ranks.warps; ++w) {
            const int c = ranks.counts[w * p.experts + e];
            ranks.counts[w * p.experts + e] = row;
            row += c;
        }
        at += all[e];
    }
    if (offsets && threadIdx.x == 0) offsets[p.experts] = total;
    for (int64_t i = total + (int64_t)block * blockDim.x + threadIdx.x; i < (int64_t)p.tokens * p.top; i += (int64_t)blocks * blockDim.x) p.order[i] = -1;
    __syncthreads();
    ranks.place();
}

// Choices of a run of tokens; ALONE: the plan as well, the runs being the blocks of one cluster, which read one another's counts.
template <int V, bool ALONE>
__global__ void __launch_bounds__(choose_threads(V)) route_choose_kernel(const __grid_constant__ RouteParams p) {
    extern __shared__ __align__(16) int32_t words[];
    start_next();
    wait_for_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int32_t *counts = words + RouteSmem::own(p.experts);
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) counts[e] = 0;
    float bias[V], bias_most = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        bias[v] = p.bias && lane + 32 * v < p.experts ? p.bias[lane + 32 * v] : 0.0f;
        if (bias[v] != bias[v]) bias[v] = __int_as_float(0xFF800000);
        if (fabsf(bias[v]) <= 3.402823466e38f) bias_most = fmaxf(bias_most, fabsf(bias[v]));
    }
    bias_most = warp_most(bias_most);
    double *scratch = reinterpret_cast<double *>(words + RouteSmem::keys(p.experts)) + warp * (p.groups > 1 ? p.groups * p.pitch : 0);
    const int first = blockIdx.x * p.run, last = first + min(p.tokens - first, p.run);
    int32_t *next = words + RouteSmem::sums(p.experts) + 36;     // warps fetch their tokens: one that took a decision again falls behind
    if (threadIdx.x == 0) *next = first + (int)(blockDim.x >> 5);
    __syncthreads();
    for (int t = first + warp; t < last;) {
        const int e = route_token<V>(p, t, bias, bias_most, scratch);
        if (lane < p.top && e >= 0) atomicAdd(&counts[e], 1);
        if (lane == 0) t = atomicAdd(next, 1);
        t = __shfl_sync(0xffffffffu, t, 0);
    }
    if (!p.order) return;                                     // (for every block)
    if constexpr (!ALONE) {
        __syncthreads();
        for (int e = threadIdx.x; e < p.experts; e += blockDim.x) p.counts[(int64_t)e * p.pitch_runs + blockIdx.x] = counts[e];
    } else {
        __syncthreads();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        RunRanks ranks(p, blockIdx.x, words);
        ranks.load();
        ranks.count();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        for (int e = threadIdx.x; e < p.experts; e += blockDim.x) {
            int a = 0, b = 0;
            const uint32_t mine = smem_u32(counts + e);
#pragma unroll
            for (int r = 0; r < ALONE_RUNS; ++r)
                if (r < (int)gridDim.x) {
                    uint32_t there;
                    int c;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(r));
                    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(c) : "r"(there) : "memory");
                    b += c;
                    a += r < (int)blockIdx.x ? c : 0;
                }
            words[e] = a;
            words[RouteSmem::all(p.experts) + e] = b;
        }
        __syncthreads();
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // nobody leaves while its counts are read
        plan_run(p, ranks, words, blockIdx.x == 0 ? p.offsets : nullptr, blockIdx.x, gridDim.x);
        __syncwarp();
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
}

// counts of an expert's runs -> its rows in the runs ahead, and in all; a warp takes an expert, a lane up to five runs in a row.
__global__ void __launch_bounds__(256) route_scan_kernel(const __grid_constant__ RouteParams p) {
    start_next();
    wait_for_previous();
    const int e = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (e >= p.experts) return;
    int32_t *counts = p.counts + (int64_t)e * p.pitch_runs;
    int c[MAX_RUNS / 32 + 1], sum = 0;
    constexpr int EACH = MAX_RUNS / 32 + 1;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        c[i] = lane * EACH + i < p.runs ? counts[lane * EACH + i] : 0;
        sum += c[i];
    }
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    int at = incl - sum;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (lane * EACH + i < p.runs) counts[lane * EACH + i] = at;
        at += c[i];
    }
    if (lane == 31) p.counts[(int64_t)p.experts * p.pitch_runs + e] = incl;
}

// The plan of a run.
__global__ void __launch_bounds__(PLAN_THREADS) route_plan_kernel(const __grid_constant__ RouteParams p) {
    extern __shared__ __align__(16) int32_t words[];
    start_next();
    wait_for_previous();
    RunRanks ranks(p, blockIdx.x, words);
    ranks.load();
    int32_t *ahead = words, *all = words + RouteSmem::all(p.experts);
    if (p.scanned) {
        for (int e = threadIdx.x; e < p.experts; e += blockDim.x) {
            ahead[e] = p.counts[(int64_t)e * p.pitch_runs + blockIdx.x];
            all[e] = p.counts[(int64_t)p.experts * p.pitch_runs + e];
        }
        ranks.count();
    } else {                                                  // eight lanes add up an expert's runs, four at a time
        const int sub = threadIdx.x & 7, me = blockIdx.x;
        const int whole = (p.experts + 3) / 4 * 4;            // (all lanes of a warp go round together)
        for (int e = threadIdx.x >> 3; e < whole; e += blockDim.x >> 3) {
            const int4 *counts = reinterpret_cast<const int4 *>(p.counts + (int64_t)min(e, p.experts - 1) * p.pitch_runs);
            int a = 0, b = 0;
            constexpr int MOST = (MAX_RUNS + 31) / 32;
            int4 c[MOST];
#pragma unroll
            for (int i = 0; i < MOST; ++i) c[i] = (sub + 8 * i) * 4 < p.runs ? counts[sub + 8 * i] : make_int4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < MOST; ++i) {
                const int r = (sub + 8 * i) * 4;
                const int n[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int v = r + k < p.runs ? n[k] : 0;  // (the last pack of a row ends past the runs)
                    b += v;
                    a += r + k < me ? v : 0;
                }
            }
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) {
                a += __shfl_xor_sync(0xffffffffu, a, d);
                b += __shfl_xor_sync(0xffffffffu, b, d);
            }
            if (sub == 0 && e < p.experts) { ahead[e] = a; all[e] = b; }
        }
        ranks.count();
    }
    __syncthreads();
    plan_run(p, ranks, words, blockIdx.x == 0 ? p.offsets : nullptr, blockIdx.x, gridDim.x);
}

// ------------------------------------------------------------------------------------------------ backward

// dlogits of the weights' gradient; a warp takes a token, lane i its choice i.
//   d score_i:  factor * dw_i, renormalised: factor / S * (dw_i - sum_j dw_j s_j / S)
//   sigmoid:    dl_e = d score_i * s_i (1 - s_i) at the chosen experts, 0 elsewhere
//   softmax:    dl_e = s_e * (d score_e - sum_j d score_j s_j); renormalised, that sum is 0 and s_i / S needs the chosen logits alone
struct RouteBackParams {
    const float *dweights;
    const void *logits;
    int type;
    int64_t ld;
    const int32_t *chosen;
    int tokens, experts, top;
    bool sigmoid, renormalise;
    float factor;
    void *dlogits;
    int64_t ldd;
};

template <class T, int V>
__global__ void __launch_bounds__(256) route_back_kernel(const RouteBackParams p) {
    start_next();
    wait_for_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int64_t token = (int64_t)blockIdx.x * 8 + warp; token < p.tokens; token += (int64_t)gridDim.x * 8) {
        int e = lane < p.top ? p.chosen[token * p.top + lane] : -1;
        if (e >= p.experts) e = -1;
        const float x = e >= 0 ? load_as_f32(p.logits, p.type, token * p.ld + e) : __int_as_float(0xFF800000);
        const float dw = e >= 0 ? __fmul_rn(p.dweights[token * p.top + lane], p.factor) : 0.0f;
        float g = 0.0f, rest = 0.0f;                          // dl at the chosen expert; of every expert, times its score
        float l[V], scale = 0.0f;
        // a token without an expert has a gradient of zeros, whatever its logits hold
        const bool dense = !p.renormalise && !p.sigmoid && __any_sync(0xffffffffu, e >= 0);
        if (p.renormalise) {
            const float high = warp_most(x);
            float u = 0.0f;
            if (e >= 0) {
                if (!p.sigmoid) u = expf(__fadd_rn(x, -high));
                else if (x >= 0.0f) u = __fdiv_rn(1.0f, __fadd_rn(1.0f, expf(-x)));
                else u = __fdiv_rn(expf(__fadd_rn(x, -fminf(high, 0.0f))), __fadd_rn(1.0f, expf(x)));
            }
            const float total = warp_add(u), share = e >= 0 ? __fdiv_rn(u, total) : 0.0f;
            const float mean = warp_add(__fmul_rn(dw, share));
            g = __fmul_rn(share, __fadd_rn(dw, -mean));
            if (p.sigmoid && e >= 0) g = __fdiv_rn(g, __fadd_rn(1.0f, expf(x)));                 // 1 - s
        } else if (p.sigmoid) {
            if (e >= 0) g = __fmul_rn(dw, __fmul_rn(__fdiv_rn(1.0f, __fadd_rn(1.0f, expf(-x))), __fdiv_rn(1.0f, __fadd_rn(1.0f, expf(x)))));
        } else if (dense) {
            load_row<V>(p.logits, p.type, token * p.ld, p.experts, l);
            float most = __int_as_float(0xFF800000), sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) most = fmaxf(most, l[v]);
            most = warp_most(most);
            most = most > __int_as_float(0xFF800000) ? most : 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                l[v] = expf(__fadd_rn(l[v], -most));
                sum = __fadd_rn(sum, l[v]);
            }
            sum = warp_add(sum);
            scale = sum > 0.0f ? __fdiv_rn(1.0f, sum) : 0.0f;
            const float s = e >= 0 ? __fmul_rn(expf(__fadd_rn(x, -most)), scale) : 0.0f;
            g = __fmul_rn(dw, s);
            rest = warp_add(g);
        }
        T *out = static_cast<T *>(p.dlogits) + token * p.ldd;
        float d[V];
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = dense ? -__fmul_rn(__fmul_rn(l[v], scale), rest) : 0.0f;
        for (int i = 0; i < p.top; ++i) {
            const int at = __shfl_sync(0xffffffffu, e, i);
            const float add = __shfl_sync(0xffffffffu, g, i);
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (at == lane + 32 * v) d[v] = __fadd_rn(d[v], add);
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (lane + 32 * v < p.experts) out[lane + 32 * v] = from_f32<T>(d[v]);
    }
}

// ------------------------------------------------------------------------------------------------ host side

// Few tokens are left to one launch: a cluster of one to eight blocks, of eight tokens and more, the fewer the more work a token is.
// (In a replayed graph and from Python: 100 x 64 top 6 5.2 and 5.4 us so, 6.4 and 7.2 in two launches; 512 x 8 7.9 and 8.1 so, 5.4
// and 8.3 in two.)  Others make as many runs as there are SMs, of at least eight tokens.  Sized for 148 SMs, so that workspace
// queries and calls agree.
bool route_alone(int64_t tokens, int experts) { return tokens <= (experts <= 64 ? 256 : experts <= 128 ? 128 : 64); }
int route_runs(int64_t tokens, int experts) {
    if (route_alone(tokens, experts)) {
        int runs = 1;
        while (runs < ALONE_RUNS && runs * 8 < tokens) runs *= 2;
        return runs;
    }
    const int64_t each = (tokens + MAX_RUNS - 1) / MAX_RUNS, run = each < 8 ? 8 : each;
    return (int)((tokens + run - 1) / run);
}

template <auto KERNEL> int launch_route(int blocks, int cluster, int threads, int smem, cudaStream_t st, const RouteParams &p) {
    if (smem > 48 * 1024 && !allow_shared_memory<KERNEL>(200 * 1024)) return QNN_E_CUDA;
    LaunchAttrs attrs(cluster);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attrs.a;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, KERNEL, p) == cudaSuccess) return QNN_OK;
    cudaGetLastError();
    return QNN_E_CUDA;
}
// Threads of the blocks that rank runs, and whether a launch of its own adds up the counts ahead of them: where eight lanes an expert would
// go round more than once (2000 x 256: 15.4 us with it, 17.4 without; 4096 x 64: 10.1 and 9.1).
int plan_threads(const RouteParams &p) { return p.run * p.top <= 256 && p.experts * (p.runs + 31) / 32 <= 64 ? 256 : PLAN_THREADS; }
bool plan_scanned(const RouteParams &p) { return p.experts > PLAN_THREADS / 8; }
template <int V> int route_launch(const RouteParams &p, cudaStream_t st) {
    constexpr int threads = choose_threads(V);
    const int fixed = RouteSmem::keys(p.experts) * 4, smem = fixed + (p.groups > 1 ? threads / 32 * p.groups * p.pitch * 8 : 0);
    if (route_alone(p.tokens, p.experts)) {
        // a warp for each token, and at least half a thread for each expert: barriers of idle warps take longer than their work
        const int some = max(p.run, (p.experts + 63) / 64) * 32;
        return launch_route<route_choose_kernel<V, true>>(p.runs, p.runs, some < threads ? some : threads, smem, st, p);
    }
    const int some = p.run * 32;
    const int rc = launch_route<route_choose_kernel<V, false>>(p.runs, 1, some < threads ? some : threads, smem, st, p);
    if (rc != QNN_OK || !p.order) return rc;
    const int scanned = p.scanned ? launch_early(route_scan_kernel, dim3((p.experts + 7) / 8), dim3(256), st, p) : QNN_OK;
    return scanned != QNN_OK ? scanned : launch_route<route_plan_kernel>(p.runs, 1, plan_threads(p), fixed, st, p);
}
template <class T, int V> int back_launch(const RouteBackParams &p, cudaStream_t st) {
    const int64_t blocks = ((int64_t)p.tokens + 7) / 8;
    return launch_early(route_back_kernel<T, V>, dim3((unsigned)(blocks < 148 * 8 ? blocks : 148 * 8)), dim3(256), st, p);
}
template <class T> int back_typed(const RouteBackParams &p, cudaStream_t st) {
    if (p.experts <= 64) return back_launch<T, 2>(p, st);
    if (p.experts <= 256) return back_launch<T, 8>(p, st);
    return back_launch<T, 32>(p, st);
}

bool route_sizes_ok(int64_t tokens, int experts, int top) {
    return tokens >= 0 && experts >= 1 && experts <= ROUTE_MAX_EXPERTS && top >= 1 && top <= experts && top <= ROUTE_MAX_TOP;
}
bool route_slots_ok(int64_t tokens, int top) { return tokens <= ROUTE_MAX_SLOTS / top; }      // (tokens * top could wrap around)

}  // namespace

extern "C" size_t qnn_route_workspace(int64_t tokens, int experts, int top) {
    if (!route_sizes_ok(tokens, experts, top) || !route_slots_ok(tokens, top) || route_alone(tokens, experts)) return 0;
    return ((size_t)((route_runs(tokens, experts) + 3) / 4 * 4 + 1) * (size_t)experts * sizeof(int32_t) + 255) / 256 * 256;
}

extern "C" int qnn_route(const void *logits, int type, int64_t tokens, int experts, int64_t ld, int top, unsigned flags, const float *bias,
                         int groups, int top_groups, float factor, const uint8_t *mask, int32_t *chosen, float *weights, int32_t *order,
                         int32_t *place, int32_t *offsets, void *workspace, size_t workspace_bytes, void *stream) {
    if (!g4_type_ok(type) || !route_sizes_ok(tokens, experts, top) || ld < experts || flags > 7u || groups < 1 || groups > ROUTE_MAX_GROUPS ||
        experts % groups != 0 || top_groups < 1 || top_groups > groups || top > top_groups * (experts / groups) ||
        (groups > 1 && (flags & QNN_ROUTE_GROUPS_BY_TWO) && experts / groups < 2))
        return QNN_E_ARG;
    if (!(fabsf(factor) <= 3.0e38f)) return QNN_E_SCALE;
    if (!route_slots_ok(tokens, top)) return QNN_E_RANGE;
    if (!qnn_aligned(bias, 4) || !qnn_aligned(order, 4) || !qnn_aligned(place, 4) || !qnn_aligned(offsets, 4)) return QNN_E_ALIGN;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (tokens == 0)
        return !offsets || cudaMemsetAsync(offsets, 0, (size_t)(experts + 1) * 4, st) == cudaSuccess ? QNN_OK : QNN_E_CUDA;
    if (!logits || !chosen || !weights || !(order ? place && offsets : !place && !offsets)) return QNN_E_ARG;
    if (!qnn_aligned(logits, g4_type_bytes(type)) || !qnn_aligned(chosen, 4) || !qnn_aligned(weights, 4)) return QNN_E_ALIGN;
    const size_t need = order ? qnn_route_workspace(tokens, experts, top) : 0;
    if (need && (!workspace || workspace_bytes < need)) return QNN_E_ARG;
    if (need && !qnn_aligned(workspace, 256)) return QNN_E_ALIGN;
    RouteParams p{};
    p.logits = logits; p.type = type; p.ld = ld;
    p.tokens = (int)tokens; p.experts = experts; p.top = top;
    p.sigmoid = flags & QNN_ROUTE_SIGMOID;
    p.renormalise = flags & QNN_ROUTE_RENORMALISE;
    p.by_sums = flags & QNN_ROUTE_GROUPS_BY_TWO;
    p.bias = bias; p.groups = groups; p.top_groups = top_groups; p.each = experts / groups;
    while ((2 << p.log_lanes) * groups <= 32) ++p.log_lanes;
    p.pitch = p.each | 1;                                      // (odd: lanes that walk along groups of their own meet no bank conflicts)
    p.group_of = (uint32_t)(((1u << 20) + p.each - 1) / p.each);
    p.whole = p.each == 32;
    p.factor = factor; p.mask = mask; p.chosen = chosen; p.weights = weights;
    p.order = order; p.place = place; p.offsets = offsets;
    p.counts = static_cast<int32_t *>(workspace);
    p.runs = route_runs(tokens, experts);
    p.run = (int)((tokens + p.runs - 1) / p.runs);
    p.pitch_runs = (p.runs + 3) / 4 * 4;
    p.scanned = plan_scanned(p);
    if (experts <= 32) return route_launch<1>(p, st);
    if (experts <= 64) return route_launch<2>(p, st);
    if (experts <= 128) return route_launch<4>(p, st);
    if (experts <= 256) return route_launch<8>(p, st);
    if (experts <= 512) return route_launch<16>(p, st);
    return route_launch<32>(p, st);
}

extern "C" int qnn_route_backward(const float *dweights, const void *logits, int type, int64_t tokens, int experts, int64_t ld, int top,
                                  unsigned flags, const int32_t *chosen, float factor, void *dlogits, int64_t ldd, void *stream) {
    if (!g4_type_ok(type) || !route_sizes_ok(tokens, experts, top) || ld < experts || ldd < experts || flags > 7u) return QNN_E_ARG;
    if (!(fabsf(factor) <= 3.0e38f)) return QNN_E_SCALE;
    if (!route_slots_ok(tokens, top)) return QNN_E_RANGE;
    if (tokens == 0) return QNN_OK;
    if (!dweights || !logits || !chosen || !dlogits) return QNN_E_ARG;
    if (!qnn_aligned(logits, g4_type_bytes(type)) || !qnn_aligned(dlogits, g4_type_bytes(type)) || !qnn_aligned(dweights, 4) || !qnn_aligned(chosen, 4))
        return QNN_E_ALIGN;
    const RouteBackParams p{dweights, logits, type, ld, chosen, (int)tokens, experts, top, (flags & QNN_ROUTE_SIGMOID) != 0,
                            (flags & QNN_ROUTE_RENORMALISE) != 0, factor, dlogits, ldd};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (type == QNN_F32) return back_typed<float>(p, st);
    if (type == QNN_BF16) return back_typed<__nv_bfloat16>(p, st);
    return back_typed<__half>(p, st);
}
