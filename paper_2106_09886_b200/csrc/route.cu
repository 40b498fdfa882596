// Routing of tokens to experts: scores, choice, weights, the plan that products grouped by expert go by, and the weights'
// gradient with respect to the logits.
//
// Choice.  A warp takes a token; lane l holds experts l, l + 32, ...  Without a bias scores grow with the logits, so the choice
// goes by the logits themselves, exactly.  With a bias (or where sums of scores decide between groups) the keys are fp32 numbers
// with a known error bound: whenever two keys whose order matters are nearer than that, the warp takes the token again with keys
// in 64 bits.  The choice is therefore that of 64-bit scores, at the cost of fp32 ones.
//
// Plan.  A counting sort: a block takes a run of tokens, counts its slots by expert, and writes the counts; behind all of them,
// the block that ranks the same slots adds up the counts of the runs ahead.  Slots of an expert keep their order, and nothing
// depends on the order in which blocks run.  Few tokens: one block does both.
//
// Bound: reading the logits and issue (some 50 instructions for each of a token's choices).
#include "real_rows.cuh"
#include "tc_ptx.cuh"

namespace {

constexpr int ROUTE_MAX_EXPERTS = 1024, ROUTE_MAX_TOP = 32, ROUTE_MAX_GROUPS = 32;
constexpr int PLAN_THREADS = 1024;
// Threads of a block whose lanes hold V experts each: V numbers of four kinds have to fit the registers.
__host__ __device__ constexpr int choose_threads(int v) { return v <= 8 ? 1024 : 512; }
constexpr int RANK_WARPS = 8;                                 // that rank a run's slots, each with its own counts
constexpr int64_t ROUTE_MAX_SLOTS = (1ll << 31) - 1;

struct RouteParams {
    const void *logits;
    int type;
    int64_t ld;
    int tokens, experts, top;
    bool sigmoid, renormalise, by_sums;                       // by_sums: groups are judged by the sum of their two largest keys
    const float *bias;
    int groups, top_groups, each, lanes, pitch;               // experts, lanes and key pitch of a group
    float factor;
    const uint8_t *mask;
    int32_t *chosen;
    float *weights;
    int32_t *order, *place, *offsets;                         // NULL: no plan
    int32_t *counts;                                          // [runs][experts]
    int runs, run;                                            // tokens of a run
};

// Keys as unsigned numbers of the same order; 0 is kept for "not to be chosen" (NaN and -infinity).
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(__fadd_rn(v, 0.0f));           // (-0 is 0)
    return !(v > __int_as_float(0xFF800000)) ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
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
__device__ __forceinline__ uint32_t warp_max_key(uint32_t k) { return __reduce_max_sync(0xffffffffu, k); }
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

// What decides between experts and groups, as numbers of type K (float, or double where fp32 is not enough).
template <class K> struct Margin {                            // two keys nearer than this may be in the wrong order
    float relative, bias;
    __device__ __forceinline__ bool close(K a, K b) const {
        if constexpr (sizeof(K) == 8) return false;
        else return __fadd_rn(a, -b) <= __fmaf_rn(relative, __fadd_rn(fmaxf(fabsf(a), fabsf(b)), bias), 1e-37f);
    }
};

// Experts of groups that are not among the best top_groups get key 0 in `keys`.  worth: keys[] as numbers, or the scores where
// sums of them decide and the keys are logits.  Returns whether the decision was too close.
template <class K, class U, int V>
__device__ __forceinline__ bool keep_groups(const RouteParams &p, const K (&worth)[V], U (&keys)[V], K *scratch, Margin<K> margin) {
    const int lane = threadIdx.x & 31;
    const K none = -(K)__int_as_float(0x7F800000);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = lane + 32 * v;
        if (e < p.experts) {
            const int g = e / p.each;
            scratch[g * p.pitch + e - g * p.each] = keys[v] ? worth[v] : none;
        }
    }
    __syncwarp();
    const int group = lane / p.lanes, sub = lane - group * p.lanes;
    K first = none, second = none;
    if (group < p.groups)
        for (int i = sub; i < p.each; i += p.lanes) {
            const K k = scratch[group * p.pitch + i];
            second = k > first ? first : (k > second ? k : second);
            first = k > first ? k : first;
        }
    __syncwarp();
    for (int d = 1; d < p.lanes; d <<= 1) {
        const K a = __shfl_xor_sync(0xffffffffu, first, d), b = __shfl_xor_sync(0xffffffffu, second, d);
        const K low = a > first ? first : a, high = a > first ? a : first;
        second = b > second ? b : second;
        second = low > second ? low : second;
        first = high;
    }
    const K mine = p.by_sums ? first + second : first;
    int better = 0;
    bool close = false;
    for (int g = 0; g < p.groups; ++g) {
        const K other = __shfl_sync(0xffffffffu, mine, g * p.lanes);
        better += other > mine || (other == mine && g < group);
    }
    const bool kept = group < p.groups && better < p.top_groups;
    if constexpr (sizeof(K) == 4) {
        // the worst group that stays against the best that goes
        float worst = kept ? mine : __int_as_float(0x7F800000), best = group < p.groups && !kept ? mine : none;
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            worst = fminf(worst, __shfl_xor_sync(0xffffffffu, worst, d));
            best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, d));
        }
        margin.bias *= 2.0f;                                  // sums of two keys
        margin.relative *= 2.0f;
        close = p.top_groups < p.groups && margin.close(worst, best);
    }
    const unsigned stay = __ballot_sync(0xffffffffu, kept);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = lane + 32 * v;
        if (e < p.experts && !((stay >> (e / p.each * p.lanes)) & 1u)) keys[v] = 0;
    }
    return close;
}

// The `top` largest keys in order, ties to the lowest expert: lane i gets choice i (-1 where nothing is left).  CHECK: whether two
// keys in a row, the first that was not chosen among them, are too close.
template <bool CHECK, class U, int V>
__device__ __forceinline__ bool take_top(int top, U (&keys)[V], int &mine, Margin<float> margin) {
    const int lane = threadIdx.x & 31;
    bool close = false;
    U previous = 0;
    mine = -1;
#pragma unroll 1
    for (int i = 0; i < top + (CHECK ? 1 : 0); ++i) {
        U best = keys[0];
#pragma unroll
        for (int v = 1; v < V; ++v) best = keys[v] > best ? keys[v] : best;
        best = warp_max_key(best);
        if (best == 0) break;
        if constexpr (CHECK) {
            if (i > 0) close |= margin.close(from_ordered((uint32_t)previous), from_ordered((uint32_t)best));
            previous = best;
            if (i == top) break;
        }
        int e = 0x7FFFFFFF;
#pragma unroll
        for (int v = V - 1; v >= 0; --v) e = keys[v] == best ? lane + 32 * v : e;
        e = (int)__reduce_min_sync(0xffffffffu, (unsigned)e);
#pragma unroll
        for (int v = 0; v < V; ++v) keys[v] = lane + 32 * v == e ? (U)0 : keys[v];
        if (lane == i) mine = e;
    }
    return close;
}

// The same decisions with 64-bit keys.
template <int V>
__device__ __noinline__ int choose_in_64_bits(const RouteParams &p, int64_t token, double *scratch) {
    const int lane = threadIdx.x & 31;
    float l[V];
    load_row<V>(p.logits, p.type, token * p.ld, p.experts, l);
    double s[V];
    unsigned long long keys[V];
    if (p.sigmoid) {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = 1.0 / (1.0 + exp(-(double)l[v]));
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
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = lane + 32 * v;
        keys[v] = 0;
        if (e < p.experts && l[v] > __int_as_float(0xFF800000)) {
            if (p.bias) s[v] += (double)p.bias[e];
            keys[v] = p.bias ? ordered(s[v]) : ordered((double)l[v]);
        }
    }
    if (p.groups > 1) keep_groups<double, unsigned long long, V>(p, s, keys, scratch, Margin<double>{});
    int mine;
    take_top<false>(p.top, keys, mine, Margin<float>{});
    return mine;
}

// Choice and weights of one token, by a warp.  Lane i < top writes choice i and returns it (-1: none).
template <int V>
__device__ __forceinline__ int route_token(const RouteParams &p, int64_t token, const float (&bias)[V], float bias_most, double *scratch) {
    const int lane = threadIdx.x & 31;
    float l[V];
    load_row<V>(p.logits, p.type, token * p.ld, p.experts, l);
    const bool there = !p.mask || p.mask[token];
    bool bad = false;
    float most = __int_as_float(0xFF800000);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        bad |= l[v] != l[v];
        most = fmaxf(most, l[v]);
    }
    most = warp_most(most);
    bad = __any_sync(0xffffffffu, bad) || (!p.sigmoid && most == __int_as_float(0x7F800000));
    int mine = -1;
    float sum = 1.0f;
    if (there && !bad && most > __int_as_float(0xFF800000)) {
        const bool scored = p.bias || (p.groups > 1 && p.by_sums);
        float s[V];
        if (scored || (!p.sigmoid && !p.renormalise)) {
            if (p.sigmoid) {
#pragma unroll
                for (int v = 0; v < V; ++v) s[v] = __fdiv_rn(1.0f, __fadd_rn(1.0f, expf(-l[v])));
            } else {
                sum = 0.0f;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    s[v] = expf(__fadd_rn(l[v], -most));
                    sum = __fadd_rn(sum, s[v]);
                }
                sum = warp_add(sum);
#pragma unroll
                for (int v = 0; v < V; ++v) s[v] = __fdiv_rn(s[v], sum);
            }
        }
        uint32_t keys[V];
        // fp32 scores: expf within 2 steps, a sum and a quotient rounded once each; softmax's exponent is rounded besides, by up to
        // 2^-24 of a difference that matters up to some 88
        const Margin<float> margin{p.sigmoid ? 9.5367431640625e-07f : 2.288818359375e-05f, bias_most};          // 2^-20, 1.5 * 2^-16
        bool close = false;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (p.bias) s[v] = __fadd_rn(s[v], bias[v]);
            keys[v] = l[v] > __int_as_float(0xFF800000) ? ordered(p.bias ? s[v] : l[v]) : 0u;
        }
        if (p.groups > 1) {
            if (scored) close = keep_groups<float, uint32_t, V>(p, s, keys, reinterpret_cast<float *>(scratch), margin);
            else keep_groups<float, uint32_t, V>(p, l, keys, reinterpret_cast<float *>(scratch), margin);
        }
        if (p.bias) close |= take_top<true>(p.top, keys, mine, margin);
        else take_top<false>(p.top, keys, mine, margin);
        if (close) mine = choose_in_64_bits<V>(p, token, scratch);
    }
    if (lane < p.top) {
        const float x = mine >= 0 ? load_as_f32(p.logits, p.type, token * p.ld + mine) : 0.0f;
        float w = 0.0f;
        const unsigned lanes = p.top == 32 ? 0xffffffffu : (1u << p.top) - 1u;
        if (p.renormalise) {
            // shares of the chosen scores, with the largest one's power taken out, so that none underflows alone
            float high = mine >= 0 ? x : __int_as_float(0xFF800000), u = 0.0f, total = 0.0f;
            for (int i = 0; i < p.top; ++i) high = fmaxf(high, __shfl_sync(lanes, high, i));
            if (mine >= 0) {
                if (!p.sigmoid) u = expf(__fadd_rn(x, -high));
                else if (x >= 0.0f) u = __fdiv_rn(1.0f, __fadd_rn(1.0f, expf(-x)));
                else u = __fdiv_rn(expf(__fadd_rn(x, -fminf(high, 0.0f))), __fadd_rn(1.0f, expf(x)));
            }
            for (int i = 0; i < p.top; ++i) total = __fadd_rn(total, __shfl_sync(lanes, u, i));
            if (mine >= 0) w = __fdiv_rn(u, total);
        } else if (mine >= 0) {
            w = p.sigmoid ? __fdiv_rn(1.0f, __fadd_rn(1.0f, expf(-x))) : __fdiv_rn(expf(__fadd_rn(x, -most)), sum);
        }
        w = there && bad ? __int_as_float(0x7FC00000) : __fmul_rn(w, p.factor);
        p.chosen[token * p.top + lane] = mine;
        p.weights[token * p.top + lane] = w;
    }
    return mine;
}

// Places of the slots of one run.  base[e]: in, the first row of expert e for this run.  counts: [RANK_WARPS][experts].
__device__ void rank_run(const RouteParams &p, int run, int32_t *base, int32_t *counts) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t first = (int64_t)run * p.run * p.top, end_token = min((int64_t)p.tokens, (int64_t)(run + 1) * p.run);
    const int64_t slots = end_token * p.top - first, segment = (slots + RANK_WARPS * 32 - 1) / (RANK_WARPS * 32) * 32;
    for (int i = threadIdx.x; i < RANK_WARPS * p.experts; i += blockDim.x) counts[i] = 0;
    __syncthreads();
    const int64_t lo = warp * segment, hi = min(slots, lo + segment);
    if (warp < RANK_WARPS)
        for (int64_t i = lo; i < hi; i += 32) {
            const int e = i + lane < hi ? p.chosen[first + i + lane] : -1;
            const unsigned same = __match_any_sync(0xffffffffu, e);
            if (e >= 0 && __ffs(same) - 1 == lane) counts[warp * p.experts + e] += __popc(same);
            __syncwarp();
        }
    __syncthreads();
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) {
        int at = base[e];
#pragma unroll
        for (int w = 0; w < RANK_WARPS; ++w) {
            const int c = counts[w * p.experts + e];
            counts[w * p.experts + e] = at;
            at += c;
        }
    }
    __syncthreads();
    if (warp < RANK_WARPS)
        for (int64_t i = lo; i < hi; i += 32) {
            const bool in = i + lane < hi;
            const int e = in ? p.chosen[first + i + lane] : -1;
            const unsigned same = __match_any_sync(0xffffffffu, e);
            const int at = e >= 0 ? counts[warp * p.experts + e] + __popc(same & ((1u << lane) - 1u)) : -1;
            __syncwarp();
            if (e >= 0 && __ffs(same) - 1 == lane) counts[warp * p.experts + e] += __popc(same);
            __syncwarp();
            if (in) p.place[first + i + lane] = at;
            if (e >= 0) p.order[at] = (int32_t)(first + i + lane);
        }
}

// counts[e] of every expert -> the experts' first rows, into offsets too where that is given; returns the rows in all.  warp_sums: 33
// numbers of shared memory.
__device__ __forceinline__ int scan_experts(int32_t *counts, int experts, int32_t *warp_sums, int32_t *offsets) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, each = (experts + blockDim.x - 1) / blockDim.x;      // (1 or 2)
    const int first = threadIdx.x * each;
    int v = 0;
    for (int e = first; e < min(first + each, experts); ++e) v += counts[e];
    int incl = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        const int own = lane < (int)(blockDim.x >> 5) ? warp_sums[lane] : 0;
        int w = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, w, d);
            if (lane >= d) w += o;
        }
        warp_sums[lane] = w - own;
        if (lane == 31) warp_sums[32] = w;
    }
    __syncthreads();
    const int total = warp_sums[32];
    int at = warp_sums[warp] + incl - v;
    for (int e = first; e < min(first + each, experts); ++e) {
        const int c = counts[e];
        counts[e] = at;
        if (offsets) offsets[e] = at;
        at += c;
    }
    if (offsets && threadIdx.x == 0) offsets[experts] = total;
    return total;
}

// A block's shared memory: counts of its run, the ranks' counts, sums; then each warp's keys.
struct RouteSmem {
    static __host__ __device__ int ranks(int experts) { return experts; }
    static __host__ __device__ int sums(int experts) { return (1 + RANK_WARPS) * experts; }
    static __host__ __device__ int keys(int experts) { return ((1 + RANK_WARPS) * experts + 40 + 3) / 4 * 4; }      // in words
};

// Choices of a run of tokens; ALONE: the plan as well (one run).
template <int V, bool ALONE>
__global__ void __launch_bounds__(choose_threads(V)) route_choose_kernel(const __grid_constant__ RouteParams p) {
    extern __shared__ __align__(16) int32_t words[];
    start_next();
    wait_for_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) words[e] = 0;
    float bias[V], bias_most = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        bias[v] = p.bias && lane + 32 * v < p.experts ? p.bias[lane + 32 * v] : 0.0f;
        if (fabsf(bias[v]) <= 3.402823466e38f) bias_most = fmaxf(bias_most, fabsf(bias[v]));
    }
    bias_most = warp_most(bias_most);
    double *scratch = reinterpret_cast<double *>(words + RouteSmem::keys(p.experts)) + warp * (p.groups > 1 ? p.groups * p.pitch : 0);
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * p.run, last = min((int64_t)p.tokens, first + p.run);
    for (int64_t t = first + warp; t < last; t += choose_threads(V) / 32) {
        const int e = route_token<V>(p, t, bias, bias_most, scratch);
        if (lane < p.top && e >= 0) atomicAdd(&words[e], 1);
    }
    if (!p.order) return;
    __syncthreads();
    if constexpr (!ALONE) {
        for (int e = threadIdx.x; e < p.experts; e += blockDim.x) p.counts[(int64_t)blockIdx.x * p.experts + e] = words[e];
    } else {
        const int total = scan_experts(words, p.experts, words + RouteSmem::sums(p.experts), p.offsets);
        for (int i = total + threadIdx.x; i < p.tokens * p.top; i += blockDim.x) p.order[i] = -1;
        __syncthreads();
        rank_run(p, 0, words, words + RouteSmem::ranks(p.experts));
    }
}

// The plan of a run, behind the counts of all.
__global__ void __launch_bounds__(PLAN_THREADS) route_plan_kernel(const __grid_constant__ RouteParams p) {
    extern __shared__ __align__(16) int32_t words[];
    start_next();
    wait_for_previous();
    // counts of an expert in all runs and in those ahead, by as many threads as fit
    int32_t *ahead = words, *all = words + RouteSmem::ranks(p.experts);
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) ahead[e] = all[e] = 0;
    __syncthreads();
    const int width = (p.experts + 31) / 32 * 32, parts = PLAN_THREADS / width, part = threadIdx.x / width, expert = threadIdx.x - part * width;
    if (part < parts && expert < p.experts) {
        int a = 0, b = 0;
#pragma unroll 16
        for (int r = part; r < p.runs; r += parts) {
            const int c = p.counts[(int64_t)r * p.experts + expert];
            b += c;
            a += r < (int)blockIdx.x ? c : 0;
        }
        atomicAdd(&ahead[expert], a);
        atomicAdd(&all[expert], b);
    }
    __syncthreads();
    const int total = scan_experts(all, p.experts, words + RouteSmem::sums(p.experts), blockIdx.x == 0 ? p.offsets : nullptr);
    __syncthreads();
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) ahead[e] += all[e];
    for (int64_t i = total + (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < (int64_t)p.tokens * p.top; i += (int64_t)gridDim.x * blockDim.x) p.order[i] = -1;
    __syncthreads();
    rank_run(p, blockIdx.x, words, words + RouteSmem::ranks(p.experts));
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
        } else {
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
        const bool dense = !p.renormalise && !p.sigmoid;
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

// Runs of tokens: one for so few that a block's warps take two each (a second launch costs more than that), else as many as there are
// SMs, of at least 32 tokens.  Sized for 148 SMs, so that workspace queries and calls agree.
int route_run(int64_t tokens) {
    if (tokens <= 64) return 64;
    const int64_t each = (tokens + 147) / 148;
    return (int)(each < 32 ? 32 : each);
}
int route_runs(int64_t tokens) { return (int)((tokens + route_run(tokens) - 1) / route_run(tokens)); }

template <class K> int launch_route(K kernel, int blocks, int threads, int smem, cudaStream_t st, const RouteParams &p) {
    if (smem > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return QNN_E_CUDA;
    LaunchAttrs attrs(1);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attrs.a;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess) return QNN_OK;
    cudaGetLastError();
    return QNN_E_CUDA;
}
template <int V> int route_launch(const RouteParams &p, cudaStream_t st) {
    constexpr int threads = choose_threads(V);
    const int fixed = RouteSmem::keys(p.experts) * 4, smem = fixed + (p.groups > 1 ? threads / 32 * p.groups * p.pitch * 8 : 0);
    if (p.runs == 1) return launch_route(route_choose_kernel<V, true>, 1, threads, smem, st, p);
    const int rc = launch_route(route_choose_kernel<V, false>, p.runs, threads, smem, st, p);
    return rc != QNN_OK || !p.order ? rc : launch_route(route_plan_kernel, p.runs, PLAN_THREADS, fixed, st, p);
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

}  // namespace

extern "C" size_t qnn_route_workspace(int64_t tokens, int experts, int top) {
    if (!route_sizes_ok(tokens, experts, top) || tokens == 0 || tokens * top > ROUTE_MAX_SLOTS || route_runs(tokens) == 1) return 0;
    return ((size_t)route_runs(tokens) * (size_t)experts * sizeof(int32_t) + 255) / 256 * 256;
}

extern "C" int qnn_route(const void *logits, int type, int64_t tokens, int experts, int64_t ld, int top, unsigned flags, const float *bias,
                         int groups, int top_groups, float factor, const uint8_t *mask, int32_t *chosen, float *weights, int32_t *order,
                         int32_t *place, int32_t *offsets, void *workspace, size_t workspace_bytes, void *stream) {
    if (!g4_type_ok(type) || !route_sizes_ok(tokens, experts, top) || ld < experts || flags > 7u || groups < 1 || groups > ROUTE_MAX_GROUPS ||
        experts % groups != 0 || top_groups < 1 || top_groups > groups || top > top_groups * (experts / groups) ||
        (groups > 1 && (flags & QNN_ROUTE_GROUPS_BY_TWO) && experts / groups < 2))
        return QNN_E_ARG;
    if (!(fabsf(factor) <= 3.0e38f)) return QNN_E_SCALE;
    if (tokens * top > ROUTE_MAX_SLOTS) return QNN_E_RANGE;
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
    p.lanes = 1;
    while (p.lanes * 2 * groups <= 32) p.lanes *= 2;
    p.pitch = p.each | 1;                                      // (odd: lanes that walk along groups of their own meet no bank conflicts)
    p.factor = factor; p.mask = mask; p.chosen = chosen; p.weights = weights;
    p.order = order; p.place = place; p.offsets = offsets;
    p.counts = static_cast<int32_t *>(workspace);
    p.run = route_run(tokens);
    p.runs = route_runs(tokens);
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
    if (tokens * top > ROUTE_MAX_SLOTS) return QNN_E_RANGE;
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
