// qmm_router.cu -- a router's choice of experts from its logits, and the gradient of the logits.
//
//   s = softmax(l) over all experts, or sigmoid(l);  c = s + bias
//   groups of E / G consecutive experts are valued by the sum of their one or two largest c, the best top_groups stay
//   the topk largest c among them are chosen, larger first, equal ones by lower index;  w = scale * s (/ the chosen ones' sum)
//
// One warp per token.  A token's logits are read once into registers; lane i holds P consecutive experts.  Who is chosen is decided in fp32 where
// fp32 can tell and in fp64 where two neighbours of the order are nearer to one another than the fp32 scores are exact (kTieSigmoid, kTieSoftmax), so that the choice is that
// of the formula.  Without a bias the order of the scores is the order of the logits, which is exact as it stands.
#include "qmm_launch.cuh"
#include "qmm_mx.cuh"
#include "qmm_route.cuh"

#include <float.h>

namespace qmm {

using namespace mx;

constexpr int kRouteWarps = 4;

struct RouteP {
    int T, E, topk, sigmoid, groups, top_groups, group_top, renorm, vec;      // vec: P logits of a lane are one or more 16-byte loads
    int64_t ld;
    const float* bias;
    float scale;
    int* idx;
    float* w;
};

// A logit as the rules read it: NaN counts as -inf, +inf as the largest finite value.
__device__ __forceinline__ float route_logit(float v) { return v == v ? fminf(v, FLT_MAX) : -INFINITY; }

template <typename T, int P> __device__ __forceinline__ void load_logits(const T* __restrict__ row, int E, int lane, int vec, float (&l)[P])
{
    constexpr int V = 16 / (int)sizeof(T) < P ? 16 / (int)sizeof(T) : P;     // elements per load
    if (vec && V > 1) {
#pragma unroll
        for (int i = 0; i < P; i += V) {
            const int e = lane * P + i;
            if (e < E) {
                uint32_t u[V * sizeof(T) / 4 ? V * sizeof(T) / 4 : 1];
                if constexpr (V * sizeof(T) == 16) {
                    const uint4 q = __ldg(reinterpret_cast<const uint4*>(row + e));
                    u[0] = q.x, u[1] = q.y, u[2] = q.z, u[3] = q.w;
                } else if constexpr (V * sizeof(T) == 8) {
                    const uint2 q = __ldg(reinterpret_cast<const uint2*>(row + e));
                    u[0] = q.x, u[1] = q.y;
                } else if constexpr (V * sizeof(T) == 4) {
                    u[0] = __ldg(reinterpret_cast<const uint32_t*>(row + e));
                }
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    if constexpr (sizeof(T) == 4) {
                        l[i + k] = route_logit(__uint_as_float(u[k]));
                    } else {
                        const float2 f = Dt<T>::up2(u[k >> 1]);
                        l[i + k] = route_logit(k & 1 ? f.y : f.x);
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k) l[i + k] = -INFINITY;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int e = lane * P + i;
            l[i] = e < E ? route_logit(Dt<T>::up(row[e])) : -INFINITY;
        }
    }
}

__device__ __forceinline__ float warp_max(float v) { return route_unkey(__reduce_max_sync(0xFFFFFFFFu, route_key(v))); }
template <typename F> __device__ __forceinline__ F warp_sum(F v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Largest magnitude beyond which exp(-l) of a sigmoid leaves fp32's range: there sigmoid(l) = exp(l) to the last bit.
constexpr float kSigmoidEnd = -80.0f;
__device__ __forceinline__ float sigmoid_f(float l) { return l < kSigmoidEnd ? expf(l) : 1.0f / (1.0f + expf(-l)); }

// Order of fp64 values as unsigned numbers, as route_key; 0 is left for "none".
__device__ __forceinline__ unsigned long long key_of(double v)
{
    const unsigned long long u = (unsigned long long)__double_as_longlong(v + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ unsigned key_of(float v) { return route_key(v); }
// The largest key of the warp, and among the lanes that hold it the lowest expert.  In two words: the upper ones first.
__device__ __forceinline__ unsigned top_key(unsigned k) { return __reduce_max_sync(0xFFFFFFFFu, k); }
__device__ __forceinline__ unsigned long long top_key(unsigned long long k)
{
    const unsigned hi = __reduce_max_sync(0xFFFFFFFFu, (unsigned)(k >> 32));
    const unsigned lo = __reduce_max_sync(0xFFFFFFFFu, (unsigned)(k >> 32) == hi ? (unsigned)k : 0u);
    return (unsigned long long)hi << 32 | lo;
}

// The groups that stay open, a bit for each: values are the sums of a group's group_top largest c (shared memory, -inf: not to be chosen).  32 / groups lanes, as a power of two,
// look through each group.  near: whether the last group that stays and the first that does not are within `tie` of one another (fp32).
template <typename F> __device__ __forceinline__ unsigned open_groups(const F* sc, const RouteP& p, int lane, F tie, bool& near)
{
    const F none = (F)-INFINITY;
    const int per = p.E / p.groups;
    const int share = 31 - __clz(32 / p.groups), L = 1 << share, g = lane >> share;
    F a = none, b = none;
    if (g < p.groups)
        for (int i = lane & (L - 1); i < per; i += L) {
            const F v = sc[g * per + i];
            b = v < a ? (v > b ? v : b) : a;
            a = v > a ? v : a;
        }
    for (int o = 1; o < L; o <<= 1) {
        const F a2 = __shfl_xor_sync(0xFFFFFFFFu, a, o), b2 = __shfl_xor_sync(0xFFFFFFFFu, b, o);
        const F low = a < a2 ? a : a2, high = b > b2 ? b : b2;
        b = low > high ? low : high;
        a = a > a2 ? a : a2;
    }
    const F value = p.group_top == 2 && b > none ? a + b : a;
    int rank = 0;
    for (int k = 0; k < p.groups; ++k) {
        const F v = __shfl_sync(0xFFFFFFFFu, value, k << share);
        rank += v > value || (v == value && k < g);
    }
    const bool stays = g < p.groups && rank < p.top_groups;
    if constexpr (sizeof(F) == 4) {
        const float last = route_unkey(__reduce_min_sync(0xFFFFFFFFu, stays ? route_key(value) : 0xFFFFFFFFu));
        const unsigned next = __reduce_max_sync(0xFFFFFFFFu, !stays && g < p.groups && value > none ? route_key(value) : 0u);
        near = next != 0u && !(last - route_unkey(next) > tie);
    }
    return __ballot_sync(0xFFFFFFFFu, (lane & (L - 1)) == 0 && stays);        // bit g << share
}

// One pass of a choice: the largest key left and its expert; that key is taken out.  false: nothing left.
template <int P, typename K> __device__ __forceinline__ bool take_top(K (&key)[P], int lane, K& top, int& e)
{
    K best = 0;
    int best_i = 0;
#pragma unroll
    for (int i = 0; i < P; ++i)
        if (key[i] > best) {
            best = key[i];
            best_i = i;
        }
    top = top_key(best);
    if (top == 0) return false;
    e = (int)__reduce_min_sync(0xFFFFFFFFu, best == top ? (unsigned)(lane * P + best_i) : 0x7FFFFFFFu);
#pragma unroll
    for (int i = 0; i < P; ++i)
        if (lane * P + i == e) key[i] = 0;                 // (constant indices: the array stays in registers)
    return true;
}

// The choice in 64 bits, for a token whose fp32 scores leave it open.  l: the token's logits; sd: E fp64 numbers of shared memory where there are groups (over the logits, which
// the caller restores).  Lane j < topk returns its expert, -1 if none.
template <int P> __device__ __noinline__ int route_exactly(const float (&l)[P], double* sd, const RouteP& p, int lane)
{
    double c[P], m = 0.0, z = 1.0;
    if (!p.sigmoid) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < P; ++i) top = fmaxf(top, l[i]);
        m = (double)warp_max(top);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) c[i] = l[i] > -INFINITY ? exp(p.sigmoid ? -(double)l[i] : (double)l[i] - m) : 0.0;
    if (!p.sigmoid) {
        z = 0.0;
#pragma unroll
        for (int i = 0; i < P; ++i) z += c[i];
        z = warp_sum(z);
    }
    unsigned long long key[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int e = lane * P + i;
        const double s = p.sigmoid ? 1.0 / (1.0 + c[i]) : c[i] / z;
        c[i] = p.bias && e < p.E ? s + (double)__ldg(p.bias + e) : s;
        if (!(l[i] > -INFINITY) || !(c[i] == c[i])) c[i] = -INFINITY;
        key[i] = c[i] > -INFINITY ? key_of(p.bias ? c[i] : (double)l[i]) : 0;      // without a bias: the scores' order is that of the logits
    }
    if (p.groups > 1) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (lane * P + i < p.E) sd[lane * P + i] = c[i];
        __syncwarp();
        bool near;
        const unsigned open = open_groups<double>(sd, p, lane, 0.0, near);
        const int per = p.E / p.groups, share = 31 - __clz(32 / p.groups);
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (!(open >> (((lane * P + i) / per << share) & 31) & 1u)) key[i] = 0;
    }
    int mine = -1;
    for (int j = 0; j < p.topk; ++j) {
        unsigned long long top;
        int e;
        if (!take_top(key, lane, top, e)) break;
        if (lane == j) mine = e;
    }
    return mine;
}

// Two fp32 scores that differ by less than this (plus the roundings of the bias's addition) are compared in 64 bits.  sigmoid: expf off by 2 ulp moves 1 / (1 + e) by
// 6e-8 at most, the sum and the division add 1.2e-7: two of them 4e-7.  softmax, relative to the token's largest score: 2 ulp of expf, |l - m| e^-|l - m| 2^-24 of its argument,
// a rounding, for both, and the denominator's 37 additions, which scale both alike: 3e-6.
constexpr float kTieSigmoid = 6e-7f, kTieSoftmax = 4e-6f;

template <typename T, int P>
__global__ void __launch_bounds__(32 * kRouteWarps) expert_route_kernel(const T* __restrict__ logits, const RouteP p)
{
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ __align__(16) float s_row[];         // per warp: E logits, and E scores where there are groups
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int t = blockIdx.x * kRouteWarps + warp;
    if (t >= p.T) return;
    float* sl = s_row + warp * p.E * (p.groups > 1 ? 2 : 1);
    float l[P], c[P];
    load_logits<T, P>(logits + t * p.ld, p.E, lane, p.vec, l);
    auto keep_logits = [&] {
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (lane * P + i < p.E) sl[lane * P + i] = l[i];
        __syncwarp();
    };
    keep_logits();
    const bool scored = p.bias || (p.groups > 1 && p.group_top == 2);        // whether scores are compared, not logits alone
    float m = -INFINITY, z = 1.0f;
    if (!p.sigmoid && (scored || !p.renorm)) {
#pragma unroll
        for (int i = 0; i < P; ++i) m = fmaxf(m, l[i]);
        m = warp_max(m);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            c[i] = l[i] > -INFINITY ? expf(l[i] - m) : 0.0f;
            sum += c[i];
        }
        z = warp_sum(sum);
    }
    const float per_z = z > 0.0f ? 1.0f / z : 0.0f;        // (0: nothing left to choose from)
    bool open = false;                                     // whether fp32 leaves the choice open
    float tie = 0.0f;
    if (scored) {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int e = lane * P + i;
            const float s = p.sigmoid ? sigmoid_f(l[i]) : c[i] * per_z;
            c[i] = p.bias && e < p.E ? s + __ldg(p.bias + e) : s;
            c[i] = l[i] > -INFINITY && c[i] == c[i] ? c[i] : -INFINITY;
            if (c[i] > -INFINITY) most = fmaxf(most, fabsf(c[i]));
        }
        tie = fmaf(warp_max(most), 2.4e-7f, p.sigmoid ? kTieSigmoid : kTieSoftmax * per_z);          // (the largest softmax is 1 / z)
    } else {
#pragma unroll
        for (int i = 0; i < P; ++i) c[i] = l[i];
    }
    unsigned key[P];                                       // 0: no such expert, not to be chosen, or chosen already
#pragma unroll
    for (int i = 0; i < P; ++i) key[i] = c[i] > -INFINITY ? route_key(scored && !p.bias ? l[i] : c[i]) : 0u;
    if (p.groups > 1) {
        float* sc = sl + p.E;
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (lane * P + i < p.E) sc[lane * P + i] = c[i];
        __syncwarp();
        bool near = false;
        const unsigned stay = open_groups<float>(sc, p, lane, 2.0f * tie, near);
        if (scored) open = near;
        const int per = p.E / p.groups, share = 31 - __clz(32 / p.groups);
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (!(stay >> (((lane * P + i) / per << share) & 31) & 1u)) key[i] = 0u;
    }
    // the topk largest keys, and one more where neighbours are compared
    const int passes = p.bias ? p.topk + 1 : p.topk;
    int sel = -1, after = -1;
    unsigned sel_key = 0u, after_key = 0u;                 // lane j: the j-th choice; after: what follows the last one
    for (int j = 0; j < passes; ++j) {
        unsigned top;
        int e;
        if (!take_top(key, lane, top, e)) break;
        if (j == p.topk) {
            after = e;
            after_key = top;
        } else if (lane == j) {
            sel = e;
            sel_key = top;
        }
    }
    if (p.bias) {
        // lane j against what follows it; equal logits and biases give equal scores in 64 bits too
        const int next_lane = lane + 1 < 32 ? lane + 1 : 31;
        int next = __shfl_sync(0xFFFFFFFFu, sel, next_lane);
        unsigned next_key = __shfl_sync(0xFFFFFFFFu, sel_key, next_lane);
        if (lane == p.topk - 1) next = after, next_key = after_key;
        bool near = false;
        if (lane < p.topk && sel >= 0 && next >= 0)
            near = !(route_unkey(sel_key) - route_unkey(next_key) > tie) && !(sl[sel] == sl[next] && __ldg(p.bias + sel) == __ldg(p.bias + next));
        open = open || __any_sync(0xFFFFFFFFu, near);
    }
    if (open) {
        sel = route_exactly<P>(l, reinterpret_cast<double*>(sl), p, lane);
        if (p.groups > 1) {
            __syncwarp();
            keep_logits();
        }
    }
    const float v = sel >= 0 ? sl[sel] : -INFINITY;
    float w = 0.0f;
    if (!p.renorm) {
        if (sel >= 0) w = p.sigmoid ? sigmoid_f(v) : expf(v - m) * per_z;
    } else {
        // weights relative to the largest chosen score: no underflow, whatever the logits
        const float top = warp_max(v);
        if (sel >= 0) w = p.sigmoid ? (top < kSigmoidEnd ? expf(v - top) : sigmoid_f(v)) : expf(v - top);
        const float sum = warp_sum(w);
        if (sel >= 0) w /= sum;
    }
    if (lane < p.topk) {
        p.idx[(int64_t)t * p.topk + lane] = sel;
        p.w[(int64_t)t * p.topk + lane] = sel >= 0 ? p.scale * w : 0.0f;
    }
}

// ------------------------------------------------------------------ gradient

struct RouteGradP {
    int T, E, topk, sigmoid, renorm, vec;                  // vec: elements of a 16-byte access, 1 if the rows' alignment does not allow it
    int64_t ld, ldo;
    float scale;
    const int* idx;
    const float* dw;
};

// One warp per token: lane j works out what flows into the logit of choice j; every other logit gets zero, or -s (g . s) where the weights are a softmax over all
// experts.  Differences of g are summed instead of the difference of sums: sum_j p_j (g_i - g_j) loses nothing where one weight is nearly 1.
template <typename T, int P>
__global__ void __launch_bounds__(32 * kRouteWarps)
expert_route_grad_kernel(const T* __restrict__ logits, const RouteGradP p, T* __restrict__ dlogits)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int t = blockIdx.x * kRouteWarps + (threadIdx.x >> 5);
    if (t >= p.T) return;
    const T* row = logits + t * p.ld;
    T* out = dlogits + t * p.ldo;
    int e = -1;
    float g = 0.0f, v = -INFINITY;
    if (lane < p.topk) e = __ldg(p.idx + (int64_t)t * p.topk + lane);
    if (e < 0 || e >= p.E) e = -1;
    if (e >= 0) {
        g = p.scale * __ldg(p.dw + (int64_t)t * p.topk + lane);
        v = route_logit(Dt<T>::up(row[e]));
        if (!(v > -INFINITY)) e = -1, g = 0.0f;
    }
    float d = 0.0f, m = 0.0f, z = 1.0f, dot = 0.0f, s = 0.0f, l[P];
    if (!p.sigmoid && !p.renorm) {
        load_logits<T, P>(row, p.E, lane, p.vec > 1, l);
        m = -INFINITY;
#pragma unroll
        for (int i = 0; i < P; ++i) m = fmaxf(m, l[i]);
        m = warp_max(m);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            l[i] = l[i] > -INFINITY ? expf(l[i] - m) : 0.0f;
            sum += l[i];
        }
        z = warp_sum(sum);
        s = e >= 0 ? expf(v - m) / z : 0.0f;
        dot = warp_sum(g * s);
        d = s * (g - dot);
    } else if (!p.renorm) {
        if (e >= 0) d = g * sigmoid_f(v) * sigmoid_f(-v);
    } else {
        const float top = warp_max(v);
        float w = 0.0f;
        if (e >= 0) w = p.sigmoid ? (top < kSigmoidEnd ? expf(v - top) : sigmoid_f(v)) : expf(v - top);
        w /= fmaxf(warp_sum(w), FLT_MIN);
        float sum = 0.0f;
        for (int j = 0; j < p.topk; ++j) sum = fmaf(__shfl_sync(0xFFFFFFFFu, w, j), g - __shfl_sync(0xFFFFFFFFu, g, j), sum);
        d = e >= 0 ? w * sum : 0.0f;
        if (p.sigmoid && e >= 0) d *= sigmoid_f(-v);
    }
    const bool full = !p.sigmoid && !p.renorm;
    // an expert that stands in several slots gets their sum, from the last of them
    const unsigned same = __match_any_sync(0xFFFFFFFFu, e);
    if (__any_sync(0xFFFFFFFFu, e >= 0 && (same & ((1u << lane) - 1u)))) {
        float sum = 0.0f;
        int last = lane;
        for (int j = 0; j < p.topk; ++j) {
            const float dj = __shfl_sync(0xFFFFFFFFu, full ? g : d, j);
            if (__shfl_sync(0xFFFFFFFFu, e, j) == e) {
                sum += dj;
                last = j;
            }
        }
        d = full ? s * (sum - dot) : sum;
        if (last != lane) e = -1;
    }
    // the whole row, then the chosen ones over it (the same warp: its stores to an address stay in order)
    const float all = z > 0.0f ? -dot / z : 0.0f;          // (0: every expert masked)
    constexpr int V = 16 / (int)sizeof(T) < P ? 16 / (int)sizeof(T) : P;
    if (p.vec > 1 && V > 1) {
#pragma unroll
        for (int i = 0; i < P; i += V) {
            const int at = lane * P + i;
            if (at >= p.E) continue;
            uint32_t u[V * sizeof(T) / 4 ? V * sizeof(T) / 4 : 1];
#pragma unroll
            for (int k = 0; k < (int)(V * sizeof(T) / 4); ++k) {
                if constexpr (sizeof(T) == 4) u[k] = __float_as_uint(full ? l[i + k] * all : 0.0f);
                else u[k] = full ? Dt<T>::down2(l[i + 2 * k] * all, l[i + 2 * k + 1 < P ? i + 2 * k + 1 : 0] * all) : 0u;
            }
            if constexpr (V * sizeof(T) == 16) *reinterpret_cast<uint4*>(out + at) = make_uint4(u[0], u[1], u[2], u[3]);
            else if constexpr (V * sizeof(T) == 8) *reinterpret_cast<uint2*>(out + at) = make_uint2(u[0], u[1]);
            else if constexpr (V * sizeof(T) == 4) *reinterpret_cast<uint32_t*>(out + at) = u[0];
        }
    } else {
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (lane * P + i < p.E) out[lane * P + i] = Dt<T>::down(full ? l[i] * all : 0.0f);
    }
    __syncwarp();
    if (e >= 0) out[e] = Dt<T>::down(d);
}

// ------------------------------------------------------------------ launches

// Whether the P logits of a lane can be read (written) in 16-byte pieces, or in one piece of 4 or 8 bytes where P is smaller than that.
static bool route_vec(const void* p, int64_t ld, int E, int P, int size)
{
    const int V = 16 / size < P ? 16 / size : P;
    const uintptr_t bytes = (uintptr_t)V * size;
    return V > 1 && E % V == 0 && (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) % bytes == 0;
}

template <typename F> static qmm_status route_by_type(int dtype, int E, F f)
{
    const int need = (E + 31) / 32;
    auto by_p = [&](auto type) {
        if (need <= 1) return f(type, std::integral_constant<int, 1>());
        if (need <= 2) return f(type, std::integral_constant<int, 2>());
        if (need <= 4) return f(type, std::integral_constant<int, 4>());
        if (need <= 8) return f(type, std::integral_constant<int, 8>());
        if (need <= 16) return f(type, std::integral_constant<int, 16>());
        return f(type, std::integral_constant<int, 32>());
    };
    if (dtype == QMM_F16) return by_p(__half());
    if (dtype == QMM_BF16) return by_p(__nv_bfloat16());
    return by_p(float());
}

qmm_status launch_expert_route(int dtype, const void* logits, int64_t ld, int T, int E, int topk, int sigmoid, const float* bias, int groups, int top_groups,
                               int group_top, int renorm, float scale, int* idx, float* w, cudaStream_t st)
{
    RouteP p = {T, E, topk, sigmoid, groups, top_groups, group_top, renorm, 0, ld, bias, scale, idx, w};
    return route_by_type(dtype, E, [&](auto type, auto per) {
        using D = decltype(type);
        constexpr int P = decltype(per)::value;
        p.vec = route_vec(logits, ld, E, P, (int)sizeof(D));
        const size_t smem = (size_t)kRouteWarps * E * (groups > 1 ? 2 : 1) * 4;               // 32 KB at most
        return launch_pdl(expert_route_kernel<D, P>, dim3((unsigned)((T + kRouteWarps - 1) / kRouteWarps)), 32 * kRouteWarps, smem, 1, st, "expert route launch",
                          (const D*)logits, p);
    });
}

qmm_status launch_expert_route_grad(int dtype, const float* dw, const void* logits, int64_t ld, const int* idx, int T, int E, int topk, int sigmoid, int renorm,
                                    float scale, void* dlogits, int64_t ldo, cudaStream_t st)
{
    RouteGradP p = {T, E, topk, sigmoid, renorm, 1, ld, ldo, scale, idx, dw};
    return route_by_type(dtype, E, [&](auto type, auto per) {
        using D = decltype(type);
        constexpr int P = decltype(per)::value;
        p.vec = route_vec(logits, ld, E, P, (int)sizeof(D)) && route_vec(dlogits, ldo, E, P, (int)sizeof(D)) ? 2 : 1;
        return launch_pdl(expert_route_grad_kernel<D, P>, dim3((unsigned)((T + kRouteWarps - 1) / kRouteWarps)), 32 * kRouteWarps, 0, 1, st,
                          "expert route gradient launch", (const D*)logits, p, (D*)dlogits);
    });
}

}  // namespace qmm
