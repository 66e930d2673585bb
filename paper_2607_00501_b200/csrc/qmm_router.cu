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
    int per, share, per_inverse;                           // experts of a group; 2^share lanes look through one; ceil(2^20 / per)
    int64_t ld;
    const float* bias;
    int bias_vec;
    float scale;
    int* idx;
    float* w;
};

// A logit as the rules read it: NaN counts as -inf, +inf as the largest finite value.
__device__ __forceinline__ float route_logit(float v) { return v == v ? fminf(v, FLT_MAX) : -INFINITY; }

// NC: nobody writes the row meanwhile (the gradient may take the logits' place).
template <bool NC, typename V> __device__ __forceinline__ V load_as(const void* p) { return NC ? __ldg(reinterpret_cast<const V*>(p)) : *reinterpret_cast<const V*>(p); }
template <typename T, int P, bool NC = true> __device__ __forceinline__ void load_logits(const T* row, int E, int lane, int vec, float (&l)[P])
{
    constexpr int V = 16 / (int)sizeof(T) < P ? 16 / (int)sizeof(T) : P;     // elements per load
    if (vec && V > 1) {
#pragma unroll
        for (int i = 0; i < P; i += V) {
            const int e = lane * P + i;
            if (e < E) {
                uint32_t u[V * sizeof(T) / 4 ? V * sizeof(T) / 4 : 1];
                if constexpr (V * sizeof(T) == 16) {
                    const uint4 q = load_as<NC, uint4>(row + e);
                    u[0] = q.x, u[1] = q.y, u[2] = q.z, u[3] = q.w;
                } else if constexpr (V * sizeof(T) == 8) {
                    const uint2 q = load_as<NC, uint2>(row + e);
                    u[0] = q.x, u[1] = q.y;
                } else if constexpr (V * sizeof(T) == 4) {
                    u[0] = load_as<NC, uint32_t>(row + e);
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

// P consecutive numbers of fp32 per lane, zeros from E on; vec: 16-byte loads.
template <int P> __device__ __forceinline__ void load_floats(const float* __restrict__ from, int E, int lane, int vec, float (&v)[P])
{
    if constexpr (P >= 4) {
        if (vec) {
#pragma unroll
            for (int i = 0; i < P; i += 4) {
                const float4 q = lane * P + i < E ? __ldg(reinterpret_cast<const float4*>(from + lane * P + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
                v[i] = q.x, v[i + 1] = q.y, v[i + 2] = q.z, v[i + 3] = q.w;
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = lane * P + i < E ? __ldg(from + lane * P + i) : 0.0f;
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
__device__ __forceinline__ float sigmoid_f(float l) { return l < kSigmoidEnd ? expf(l) : __fdividef(1.0f, 1.0f + expf(-l)); }          // (a reciprocal off by 1 ulp)
// The same for comparisons: below -87 it is 0, which is nearer than they look.
__device__ __forceinline__ float sigmoid_score(float l) { return __fdividef(1.0f, 1.0f + expf(-l)); }

// Shares of the chosen scores in their sum.  v: the lane's chosen logit, -inf for none; top: the largest.  Scores relative to the largest one where exp(top) leaves fp32's range; a score
// below that range beside a larger one is its ratio to that one, so that a share underflows only where it is below fp32 itself.
__device__ __forceinline__ float chosen_share(float v, float top, bool there, int sigmoid, float least)
{
    float w = 0.0f;
    if (there) w = sigmoid ? (top < kSigmoidEnd ? expf(v - top) : sigmoid_f(v)) : expf(v - top);
    const float sum = fmaxf(warp_sum(w), least);
    if (there) w = sigmoid && v < kSigmoidEnd && top >= kSigmoidEnd && top < 0.0f ? expf(v - top) * (expf(top) / sum) : w / sum;
    return w;
}

// Order of fp64 values as unsigned numbers, as route_key; 0 is left for "none".
__device__ __forceinline__ unsigned long long key_of(double v)
{
    const unsigned long long u = (unsigned long long)__double_as_longlong(v + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}
// The largest key of the warp, in two words: the upper ones first.
__device__ __forceinline__ unsigned long long top_key(unsigned long long k)
{
    const unsigned hi = __reduce_max_sync(0xFFFFFFFFu, (unsigned)(k >> 32));
    const unsigned lo = __reduce_max_sync(0xFFFFFFFFu, (unsigned)(k >> 32) == hi ? (unsigned)k : 0u);
    return (unsigned long long)hi << 32 | lo;
}

// The groups that stay open, a bit for each: values are the sums of a group's group_top largest c (-inf: not to be chosen).  32 / groups lanes, as a power of two,
// look through each group.  near: whether the last group that stays and the first that does not are within `tie` of one another (fp32).
// Where the lanes' P consecutive experts make up whole groups (inside) they are looked through in registers, c, else in shared memory, sc (stored: they are there).
template <typename F, int P> __device__ __forceinline__ unsigned open_groups(const F (&c)[P], F* sc, const RouteP& p, int lane, F tie, bool& near, bool stored = false)
{
    const F none = (F)-INFINITY;
    const int per = p.per, share = p.share, L = 1 << share, g = lane >> share;
    F a = none, b = none;
    auto take = [&](F v) {
        b = v < a ? (v > b ? v : b) : a;
        a = v > a ? v : a;
    };
    if (!stored && per == P << share) {
#pragma unroll
        for (int i = 0; i < P; ++i) take(c[i]);
    } else {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (!stored && lane * P + i < p.E) sc[lane * P + i] = c[i];
        __syncwarp();
        if (g < p.groups)
            for (int i = lane & (L - 1); i < per; i += L) take(sc[g * per + i]);
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

// Takes out the keys of closed groups (open: bit group << share).
template <int P, typename K> __device__ __forceinline__ void close_groups(K (&key)[P], unsigned open, const RouteP& p, int lane)
{
    if (p.per == P << p.share) {                           // a lane's experts belong to one group
        const bool stays = open >> (lane >> p.share << p.share) & 1u;
#pragma unroll
        for (int i = 0; i < P; ++i) key[i] = stays ? key[i] : 0;
    } else {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int g = (lane * P + i) * p.per_inverse >> 20;                // e / per: e < 1024, so the product's error stays below 1 / per
            if (!(open >> ((g << p.share) & 31) & 1u)) key[i] = 0;
        }
    }
}

// A lane's own numbers, largest first (odd-even merge sort; P a power of two).
template <int P> __device__ __forceinline__ void sort_down(unsigned (&v)[P])
{
#pragma unroll
    for (int p = 1; p < P; p *= 2)
#pragma unroll
        for (int k = p; k >= 1; k /= 2)
#pragma unroll
            for (int j = k % p; j + k < P; j += 2 * k)
#pragma unroll
                for (int i = 0; i < k; ++i)
                    if (i + j + k < P && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                        const unsigned hi = max(v[i + j], v[i + j + k]), lo = min(v[i + j], v[i + j + k]);
                        v[i + j] = hi;
                        v[i + j + k] = lo;
                    }
}

// What turns a logit into its score in 64 bits: the largest logit and the sum of a softmax.
struct Score64 {
    double m, z;
};
template <typename T> __device__ __forceinline__ Score64 score64_of(const T* __restrict__ row, const RouteP& p, int lane)
{
    Score64 q = {0.0, 1.0};
    if (!p.sigmoid) {
        float top = -INFINITY;
        for (int e = lane; e < p.E; e += 32) top = fmaxf(top, route_logit(Dt<T>::up(row[e])));
        q.m = (double)warp_max(top);
        q.z = 0.0;
#pragma unroll 1
        for (int e = lane; e < p.E; e += 32) {
            const float l = route_logit(Dt<T>::up(row[e]));
            q.z += l > -INFINITY ? exp((double)l - q.m) : 0.0;
        }
        q.z = warp_sum(q.z);
    }
    return q;
}
// Score and bias of expert e, -inf if it is not to be chosen.
template <typename T> __device__ __forceinline__ double value64(const T* __restrict__ row, int e, const Score64& q, const RouteP& p)
{
    const double l = (double)route_logit(Dt<T>::up(row[e]));
    const double v = exp(p.sigmoid ? -l : l - q.m);
    double c = p.sigmoid ? 1.0 / (1.0 + v) : v / q.z;
    if (p.bias) c += (double)__ldg(p.bias + e);
    return l > -INFINITY && c == c ? c : -INFINITY;
}

// The four places below take over where fp32 leaves something open, about one token in a thousand.  Their code is cold: what it takes is mostly its way into the instruction
// cache, so loops stay rolled.

// Open groups in 64 bits: sc holds the scores of 32 bits (shared memory).  false: a group's second and third are too near to one another as well.
template <typename T> __device__ __noinline__ bool open_groups_exactly(const T* __restrict__ row, const float* sc, const RouteP& p, int lane, float tie, unsigned& open)
{
    const Score64 q = score64_of(row, p, lane);
    double value = -INFINITY;
    bool near = false;
    if (lane < p.groups) {
        float a = -INFINITY, b = -INFINITY, c = -INFINITY; // the group's three largest, and where the first two are
        int ea = -1, eb = -1;
#pragma unroll 1
        for (int e = lane * p.per; e < (lane + 1) * p.per; ++e) {
            const float v = sc[e];
            if (v > a) c = b, b = a, eb = ea, a = v, ea = e;
            else if (v > b) c = b, b = v, eb = e;
            else if (v > c) c = v;
        }
        const float last = p.group_top == 2 ? b : a, next = p.group_top == 2 ? c : b;
        near = next > -INFINITY && !(last - next > tie);
        double sum = 0.0;
#pragma unroll 1
        for (int k = 0; k < p.group_top; ++k) {
            const int e = k ? eb : ea;
            if (e >= 0) sum += value64(row, e, q, p);
        }
        if (ea >= 0) value = sum;
    }
    if (__any_sync(0xFFFFFFFFu, near)) return false;
    int rank = 0;
#pragma unroll 1
    for (int k = 0; k < p.groups; ++k) {
        const double v = __shfl_sync(0xFFFFFFFFu, value, k);
        rank += v > value || (v == value && k < lane);
    }
    const unsigned stay = __ballot_sync(0xFFFFFFFFu, lane < p.groups && rank < p.top_groups);
    open = 0u;                                             // bit g << share
#pragma unroll 1
    for (int k = 0; k < p.groups; ++k) open |= (stay >> k & 1u) << (k << p.share);
    return true;
}

// Whether an expert behind the last one chosen (`last`: its key's upper bits, and in the bits `low` what the expert leaves of them) may be better than it.  Of one key's upper
// bits any expert may be the best, so all that follow are looked at; those of the same logit and bias are in order.  m, per_z: of a softmax.
template <typename T> __device__ __noinline__ bool overtaken(const T* __restrict__ row, unsigned last, unsigned low, float m, float per_z, const RouteP& p, int lane, float tie)
{
    auto score = [&](float l) { return p.sigmoid ? sigmoid_score(l) : expf(l - m) * per_z; };
    const int at = (int)(low - (last & low));
    const float v = route_logit(Dt<T>::up(row[at])), b = __ldg(p.bias + at), c = score(v) + b;
    bool any = false;
#pragma unroll 1
    for (int e = lane; e < p.E; e += 32) {
        const float l = route_logit(Dt<T>::up(row[e])), o = __ldg(p.bias + e), x = score(l) + o;
        const unsigned k = l > -INFINITY && x > -INFINITY ? (route_key(x) & ~low) | (low - (unsigned)e) : 0u;
        any |= k != 0u && k < last && !(c - x > tie) && !(l == v && o == b);
    }
    return __any_sync(0xFFFFFFFFu, any);
}

// The topk best of the candidates that the lanes hold (mine: the key's upper bits, and in the bits `low` what the expert leaves of them; 0: none), compared in 64 bits.  rest: the largest key that no lane holds.
// Lane j < topk returns its expert; false: an expert that no lane holds may belong among them.
template <typename T> __device__ __noinline__ bool refine(const T* __restrict__ row, unsigned mine, unsigned rest, unsigned low, const RouteP& p, int lane, float tie, int& sel)
{
    const Score64 q = score64_of(row, p, lane);
    const int e = mine ? (int)(low - (mine & low)) : 0x7FFFFFFF;
    double v = -INFINITY;
    if (mine) v = value64(row, e, q, p);
    int rank = 0;
    const int held = __popc(__ballot_sync(0xFFFFFFFFu, mine != 0u));           // (the first lanes)
#pragma unroll 1
    for (int k = 0; k < held; ++k) {
        const double o = __shfl_sync(0xFFFFFFFFu, v, k);
        const int oe = __shfl_sync(0xFFFFFFFFu, e, k);
        rank += o > v || (o == v && oe < e);
    }
    sel = -1;
    double last = INFINITY;                                // the last one chosen
#pragma unroll 1
    for (int j = 0; j < p.topk; ++j) {
        const unsigned who = __ballot_sync(0xFFFFFFFFu, mine && rank == j);
        if (!who) break;
        const int from = __ffs(who) - 1, ej = __shfl_sync(0xFFFFFFFFu, e, from);
        last = __shfl_sync(0xFFFFFFFFu, v, from);
        if (lane == j) sel = ej;
    }
    return rest == 0u || last > (double)route_unkey(rest | low) + (double)tie;
}

// The whole choice in 64 bits.  sd: E fp64 numbers of shared memory.  Lane j < topk returns its expert, -1 if none.
template <typename T> __device__ __noinline__ int route_exactly(const T* __restrict__ row, double* sd, const RouteP& p, int lane)
{
    const double none = -INFINITY;
    const Score64 q = score64_of(row, p, lane);
    // without a bias the scores' order is that of the logits, which do not run into one another where scores do; sums of two scores are needed for groups alone
    const bool by_logit = !p.bias && !(p.groups > 1 && p.group_top == 2);
#pragma unroll 1
    for (int e = lane; e < p.E; e += 32) sd[e] = by_logit ? (double)route_logit(Dt<T>::up(row[e])) : value64(row, e, q, p);
    __syncwarp();
    if (p.groups > 1) {
        const double unused[1] = {none};
        bool near;
        const unsigned open = open_groups<double, 1>(unused, sd, p, lane, 0.0, near, true);
#pragma unroll 1
        for (int e = lane; e < p.E; e += 32)
            if (!(open >> (((e * p.per_inverse >> 20) << p.share) & 31) & 1u)) sd[e] = none;
    }
    if (!p.bias && !by_logit)
#pragma unroll 1
        for (int e = lane; e < p.E; e += 32)
            if (sd[e] > none) sd[e] = (double)route_logit(Dt<T>::up(row[e]));
    int mine = -1;
#pragma unroll 1
    for (int j = 0; j < p.topk; ++j) {                     // a lane's experts lie 32 apart: lower ones first
        double best = none;
        int at = 0x7FFFFFFF;
#pragma unroll 4
        for (int e = lane; e < p.E; e += 32) {
            const double v = sd[e];
            if (v > best) {
                best = v;
                at = e;
            }
        }
        const unsigned long long key = best > none ? key_of(best) : 0ull, top = top_key(key);
        if (top == 0) break;
        at = (int)__reduce_min_sync(0xFFFFFFFFu, key == top ? (unsigned)at : 0x7FFFFFFFu);
        if ((at & 31) == lane) sd[at] = none;
        if (lane == j) mine = at;
    }
    __syncwarp();
    return mine;
}

// Two fp32 scores that differ by less than this (plus the roundings of the bias's addition) are compared in 64 bits.  sigmoid: expf off by 2 ulp moves 1 / (1 + e) by
// 6e-8 at most, the sum and the reciprocal (1 ulp) add 1.8e-7: two of them 4.8e-7.  softmax, relative to the token's largest score: 2 ulp of expf, |l - m| e^-|l - m| 2^-24 of its argument,
// a rounding, for both, and the denominator's 37 additions, which scale both alike: 3e-6.
constexpr float kTieSigmoid = 6e-7f, kTieSoftmax = 4e-6f;

template <typename T, int P>
__device__ __forceinline__ void route_one(const T* __restrict__ row, int64_t t, const float (&l)[P], const float (&bias)[P], double* sd, const RouteP& p, int lane)
{
    float c[P];
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
            const float s = p.sigmoid ? sigmoid_score(l[i]) : c[i] * per_z;
            c[i] = p.bias ? s + bias[i] : s;
            c[i] = l[i] > -INFINITY ? c[i] : -INFINITY;
            const bool live = c[i] > -INFINITY;            // (a NaN is not)
            c[i] = live ? c[i] : -INFINITY;
            most = fmaxf(most, live ? fabsf(c[i]) : 0.0f);
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
        bool near = false;
        float* sc = reinterpret_cast<float*>(sd);
        unsigned stay = open_groups<float, P>(c, sc, p, lane, 2.0f * tie, near);
        if (scored && near) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < P; ++i)
                if (lane * P + i < p.E) sc[lane * P + i] = c[i];
            __syncwarp();
            open = !open_groups_exactly<T>(row, sc, p, lane, tie, stay);
        }
        close_groups(key, stay, p, lane);
    }
    // The topk largest, and one more to see what follows: by the keys' upper 22 to 27 bits with the expert in the lower ones.  That is one number to compare, so a lane keeps its own
    // in order and a pass is one reduction and one step down in the lane that won.
    int sel = -1;
    float v = -INFINITY;
    if (!open) {
        constexpr unsigned low = 32 * P - 1;               // bits of an expert's number
        unsigned packed[P], mine = 0u;                     // lane j: the j-th largest
#pragma unroll
        for (int i = 0; i < P; ++i) packed[i] = key[i] ? (key[i] & ~low) | (low - (unsigned)(lane * P + i)) : 0u;
        sort_down(packed);
        auto pass = [&](int j) {                           // (0: nothing left, and nothing changes)
            const unsigned top = __reduce_max_sync(0xFFFFFFFFu, packed[0]);
            const bool won = packed[0] == top;
            mine = lane == j ? top : mine;
#pragma unroll
            for (int i = 0; i + 1 < P; ++i) packed[i] = won ? packed[i + 1] : packed[i];
            packed[P - 1] = won ? 0u : packed[P - 1];
        };
        const int passes = p.topk < 32 ? p.topk + 1 : 32;
#pragma unroll 2
        for (int j = 0; j < passes; ++j) pass(j);
        unsigned follow = __shfl_down_sync(0xFFFFFFFFu, mine, 1);
        if (p.topk == 32) {
            const unsigned rest = __reduce_max_sync(0xFFFFFFFFu, packed[0]);
            if (lane == 31) follow = rest;
        }
        sel = lane < p.topk && mine ? (int)(low - (mine & low)) : -1;
        const int next = lane < p.topk && follow ? (int)(low - (follow & low)) : -1;
        if (sel >= 0) v = route_logit(Dt<T>::up(row[sel]));
        // Neighbours that agree in these bits (for 16-bit logits without a bias: are equal, and in order), or whose scores of 32 bits are nearer than these are exact, are
        // compared as logits, or in 64 bits, with eight that follow.  Equal logits and biases give equal scores there too.
        bool near = false, border = false;                 // border: the last one chosen is within reach of what follow's upper bits allow, whatever follow itself is
        if (next >= 0) {
            near = !(sizeof(T) == 2 && !p.bias) && (mine & ~low) == (follow & ~low);
            if (p.bias) {
                const float l2 = route_logit(Dt<T>::up(row[next])), b1 = __ldg(p.bias + sel), b2 = __ldg(p.bias + next);
                const float s1 = p.sigmoid ? sigmoid_score(v) : expf(v - m) * per_z, s2 = p.sigmoid ? sigmoid_score(l2) : expf(l2 - m) * per_z;
                near = (near || !((s1 + b1) - (s2 + b2) > tie)) && !(v == l2 && b1 == b2);
                border = lane == p.topk - 1 && !((s1 + b1) - route_unkey(follow | low) > tie);
            }
        }
        bool look = __any_sync(0xFFFFFFFFu, near || border);
        if (look && p.bias && !__any_sync(0xFFFFFFFFu, near))
            look = overtaken<T>(row, __shfl_sync(0xFFFFFFFFu, mine, p.topk - 1), low, m, per_z, p, lane, tie);
        if (look) {
            unsigned rest;
            if (!p.bias) {                                 // the logits themselves decide: neighbours change places until they are in order
                int e = mine ? (int)(low - (mine & low)) : 0x7FFFFFFF;
                float own = mine ? route_logit(Dt<T>::up(row[e])) : -INFINITY;
#pragma unroll 1
                for (int r = 0; r < passes; ++r) {
                    const int with = r & 1 ? ((lane + 1) ^ 1) - 1 : lane ^ 1;
                    const float o = __shfl_sync(0xFFFFFFFFu, own, with & 31);
                    const int oe = __shfl_sync(0xFFFFFFFFu, e, with & 31);
                    const bool behind = with > lane ? o > own || (o == own && oe < e) : own > o || (own == o && e < oe);
                    if (behind && with >= 0 && with < passes && lane < passes) own = o, e = oe;
                }
                rest = __reduce_max_sync(0xFFFFFFFFu, packed[0]);              // the largest that no lane holds
                const unsigned lowest = __shfl_sync(0xFFFFFFFFu, mine, passes - 1);
                open = rest != 0u && (rest & ~low) == (lowest & ~low);
                sel = lane < p.topk && e < p.E ? e : -1;
            } else {
#pragma unroll 1
                for (int j = passes; j < 32 && j < passes + 8; ++j) pass(j);
                rest = __reduce_max_sync(0xFFFFFFFFu, packed[0]);
                open = !refine<T>(row, mine, rest, low, p, lane, tie, sel);
            }
            v = sel >= 0 ? route_logit(Dt<T>::up(row[sel])) : -INFINITY;
        }
    }
    if (open) {
        sel = route_exactly<T>(row, sd, p, lane);
        v = sel >= 0 ? route_logit(Dt<T>::up(row[sel])) : -INFINITY;
    }
    float w = 0.0f;
    if (!p.renorm) {
        if (sel >= 0) w = p.sigmoid ? sigmoid_f(v) : expf(v - m) * per_z;
    } else {
        w = chosen_share(v, warp_max(v), sel >= 0, p.sigmoid, 0.0f);
    }
    if (lane < p.topk) {
        p.idx[(int64_t)t * p.topk + lane] = sel;
        p.w[(int64_t)t * p.topk + lane] = sel >= 0 ? p.scale * w : 0.0f;
    }
}

// Bound by the latency of a token's chain of reductions: with many tokens (16384 x 128 fp32: 12 us for 9.4 MB; the bytes take 1.4) issue slots are 45 % busy at 43 % of the
// warps an SM can have, with few (4 x 128: 2.2 us; 2048 x 256 bf16 with a bias and groups 7.8) the launch and one chain are all there is.
template <typename T, int P> __global__ void __launch_bounds__(32 * kRouteWarps, P <= 4 ? 8 : P == 8 ? 6 : 4) expert_route_kernel(const T* __restrict__ logits, const RouteP p)
{
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ __align__(16) double s_row[];        // per warp: E scores
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int t = blockIdx.x * kRouteWarps + warp;
    if (t >= p.T) return;
    float l[P], bias[P];
    load_logits<T, P>(logits + t * p.ld, p.E, lane, p.vec, l);
    if (p.bias) load_floats<P>(p.bias, p.E, lane, p.bias_vec, bias);
    route_one<T, P>(logits + t * p.ld, t, l, bias, s_row + warp * p.E, p, lane);
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
// Bound by latency: a warp's row is 512 bytes, read, exchanged and written (16384 x 128 fp32, all of the four forms: 18 MB in 5.7 to 7.4 us; the bytes take 2.8).
template <typename T, int P>
__global__ void __launch_bounds__(32 * kRouteWarps)
expert_route_grad_kernel(const T* logits, const RouteGradP p, T* dlogits)
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
        load_logits<T, P, false>(row, p.E, lane, p.vec > 1, l);
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
        const float w = chosen_share(v, warp_max(v), e >= 0, p.sigmoid, FLT_MIN);
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
    __syncwarp();                                          // dlogits may be logits: the warp has read its row
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
    const int per_group = E / groups;
    int share = 0;                                         // the largest power of two of lanes that all groups can have
    while ((2 << share) * groups <= 32) ++share;
    RouteP p = {T, E, topk, sigmoid, groups, top_groups, group_top, renorm, 0, per_group, share, ((1 << 20) + per_group - 1) / per_group, ld, bias,
                E % 4 == 0 && aligned(bias, 16), scale, idx, w};
    return route_by_type(dtype, E, [&](auto type, auto per) {
        using D = decltype(type);
        constexpr int P = decltype(per)::value;
        p.vec = route_vec(logits, ld, E, P, (int)sizeof(D));
        const size_t smem = (size_t)kRouteWarps * E * 8;                                       // 32 KB at most
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
