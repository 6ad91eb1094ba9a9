// Routing to experts: scores of a token's logits, its best experts and their weights; and the gradient of the logits.
//
// A token is LPT lanes of a wave, EPL neighbouring experts to each.  The order of experts is that of score + bias (of the logits, where scores grow with them and
// nothing is added), equal ones by index; a round takes the best that is left.
//
// Bound by the latency of a token's rounds, each a maximum over its lanes and one removed, and of many tokens by their instructions; the logits are read once (12608 x 128 of fp32, 6.5 MB, 1.3 us at
// 5 TB/s; 7.0 us, both directions back to back 10.1).
#include "abft_device.h"
#include "gemm_epilogue.h"
#include "route_args.h"

namespace abft {

template <int DT> __device__ __forceinline__ float logit_at(const uint8_t *row, int e)
{
    if constexpr (DT == DT_F32) return reinterpret_cast<const float *>(row)[e];
    else if constexpr (DT == DT_BF16) return bf16_bits_to_f32(reinterpret_cast<const uint16_t *>(row)[e]);
    else return f16_bits_to_f32(reinterpret_cast<const uint16_t *>(row)[e]);
}

// A lane's EPL logits: experts e0 ..; those past the last are -Inf.  Rows are whole 16 bytes, so the chunk of the last expert is there.
template <int DT, int EPL> __device__ __forceinline__ void load_logits(const uint8_t *row, int e0, int E, float (&x)[EPL])
{
    constexpr int ES = DT == DT_F32 ? 4 : 2, C = EPL * ES < 16 ? EPL : 16 / ES;
#pragma unroll
    for (int c = 0; c < EPL / C; ++c) {
        const int at = min(e0 + c * C, (E - 1) / C * C);
        uint32_t w[4] = {0, 0, 0, 0};
        if constexpr (C * ES == 16) {
            const i32x4 v = *reinterpret_cast<const i32x4 *>(row + at * ES);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (uint32_t)v[i];
        } else if constexpr (C * ES == 8) {
            const uint2 v = *reinterpret_cast<const uint2 *>(row + at * ES);
            w[0] = v.x; w[1] = v.y;
        } else if constexpr (C * ES == 4) {
            w[0] = *reinterpret_cast<const uint32_t *>(row + at * ES);
        } else {
            w[0] = *reinterpret_cast<const uint16_t *>(row + at * ES);
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float v;
            if constexpr (DT == DT_F32) v = __uint_as_float(w[i]);
            else {
                const uint32_t h = w[i >> 1] >> (16 * (i & 1)) & 0xFFFFu;
                v = DT == DT_BF16 ? bf16_bits_to_f32(h) : f16_bits_to_f32(h);
            }
            x[c * C + i] = e0 + c * C + i < E ? v : -__builtin_inff();
        }
    }
}

// And back, rounded once; nothing past the last.
template <int DT, int EPL> __device__ __forceinline__ void store_logits(uint8_t *row, int e0, int E, const float (&v)[EPL])
{
    constexpr int ES = DT == DT_F32 ? 4 : 2, C = EPL * ES < 16 ? EPL : 16 / ES, W = C * ES / 4;
#pragma unroll
    for (int c = 0; c < EPL / C; ++c) {
        const int e = e0 + c * C;
        uint32_t w[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (DT == DT_F32) w[i] = __float_as_uint(v[c * C + i]);
            else w[i] = pack2<DT>(v[c * C + 2 * i], v[c * C + 2 * i + 1]);
        }
        uint8_t *const at = row + (long)e * ES;
        if (e + C <= E) {
            if constexpr (W == 4) *reinterpret_cast<i32x4 *>(at) = i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
            else if constexpr (W == 2) *reinterpret_cast<uint2 *>(at) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t *>(at) = w[0];
        } else {
            for (int i = 0; i < C && e + i < E; ++i) {
                if constexpr (DT == DT_F32) reinterpret_cast<uint32_t *>(at)[i] = w[i];
                else reinterpret_cast<uint16_t *>(at)[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
            }
        }
    }
}

// ---------------------------------------------------------------- over the LPT lanes of a token
template <int CTRL> __device__ __forceinline__ double dpp_get64(double v)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)dpp_mov<CTRL>((int)(uint32_t)u), hi = (uint32_t)dpp_mov<CTRL>((int)(uint32_t)(u >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int CTRL> __device__ __forceinline__ float other(float v) { return dpp_get<CTRL>(v); }
template <int CTRL> __device__ __forceinline__ int other(int v) { return dpp_mov<CTRL>(v); }
template <int CTRL> __device__ __forceinline__ double other(double v) { return dpp_get64<CTRL>(v); }
// Across the rows of 16 lanes and the halves of a wave: the row-swap instructions, whose two results are the lane's own value and the other's, in either order.
template <int D> __device__ __forceinline__ void far_pair(uint32_t v, uint32_t (&p)[2])
{
    if constexpr (D == 16) {
        auto q = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        p[0] = q[0]; p[1] = q[1];
    } else {
        auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        p[0] = q[0]; p[1] = q[1];
    }
}
template <int D, typename V, typename OP> __device__ __forceinline__ V with_far(V v, const OP &op)
{
    uint32_t p[2], q[2];
    if constexpr (sizeof(V) == 4) {
        far_pair<D>(__builtin_bit_cast(uint32_t, v), p);
        return op(__builtin_bit_cast(V, p[0]), __builtin_bit_cast(V, p[1]));
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        far_pair<D>((uint32_t)u, p);
        far_pair<D>((uint32_t)(u >> 32), q);
        return op(__builtin_bit_cast(V, (uint64_t)q[0] << 32 | p[0]), __builtin_bit_cast(V, (uint64_t)q[1] << 32 | p[1]));
    }
}
template <int CTRL> __device__ __forceinline__ long long other(long long v)
{
    return __builtin_bit_cast(long long, dpp_get64<CTRL>(__builtin_bit_cast(double, v)));
}
template <int LPT, typename V, typename OP> __device__ __forceinline__ V over_token(V v, const OP &op)
{
    v = op(v, other<0xB1>(v));     // lane ^ 1
    v = op(v, other<0x4E>(v));     // lane ^ 2
    v = op(v, other<0x141>(v));    // i <-> 7 - i inside 8 lanes
    v = op(v, other<0x140>(v));    // i <-> 15 - i inside 16 lanes
    if constexpr (LPT == 64) {
        v = with_far<16>(v, op);
        v = with_far<32>(v, op);
    }
    return v;
}
struct Larger { template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a > b ? a : b; } };
struct Smaller { template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a < b ? a : b; } };
struct Plus { template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; } };

__device__ __forceinline__ void wave_lds_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------- keys in the order they are chosen by
// As integers: of fp32 (zeros of either sign alike), and of fp64.  NONE: behind all, -Inf too.
template <typename KEY> struct Order;
template <> struct Order<float> {
    typedef int type;
    static constexpr int NONE = -0x7FFFFFFF - 1;
    __device__ static __forceinline__ int of(float k)
    {
        const int i = __float_as_int(k + 0.f);
        return i ^ ((i >> 31) & 0x7FFFFFFF);
    }
    __device__ static __forceinline__ float value(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7FFFFFFF)); }
};
template <> struct Order<double> {
    typedef long long type;
    static constexpr long long NONE = -0x7FFFFFFFFFFFFFFFll - 1;
    __device__ static __forceinline__ long long of(double k)
    {
        const long long i = __double_as_longlong(k + 0.0);
        return i ^ ((i >> 63) & 0x7FFFFFFFFFFFFFFFll);
    }
};

// Scores, and the largest there can be.  In fp32, with d = x - max x, a softmax's exponential is off by (2 |d| + 2) 2^-24 of itself (d, its multiple and the instruction are each
// rounded), their sum by as much of its terms and by up to 22 2^-24 for its additions, the quotient by 3 2^-24: with |d| of up to 20 where it counts (a term of a larger one is below 2^-28 of
// the sum) below 2^-17 s.  A sigmoid is off by 2^-23 (1 + (1 - s)(|x| + 2) / 2) s or less, below 2^-22.
template <typename KEY, int LPT, int EPL> __device__ __forceinline__ void scores(bool sigmoid, const float (&x)[EPL], float top, KEY (&s)[EPL], float *largest)
{
    *largest = 1.f;
    if (sigmoid) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            if constexpr (sizeof(KEY) == 8) s[i] = 1.0 / (1.0 + exp(-(double)x[i]));
            else s[i] = __builtin_amdgcn_rcpf(1.f + __expf(-x[i]));
        }
        return;
    }
    const float m = top > -__builtin_inff() ? top : 0.f;
    KEY sum = 0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        if constexpr (sizeof(KEY) == 8) s[i] = exp((double)x[i] - (double)m);
        else s[i] = __expf(x[i] - m);
        sum += s[i];
    }
    sum = over_token<LPT>(sum, Plus{});
    if constexpr (sizeof(KEY) == 8) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) s[i] /= sum;
    } else {
        const float inv = __builtin_amdgcn_rcpf(sum);
        *largest = inv;
#pragma unroll
        for (int i = 0; i < EPL; ++i) s[i] *= inv;
    }
}

// What a token's lanes share in LDS: keys of its experts and values of its groups, and the choices.
template <int LPT, int EPL, bool GROUPED> struct RouteLds {
    double keys[GROUPED ? LPT * EPL : 1], values[GROUPED ? ROUTE_MAX_GROUPS : 1];
    int chosen[LPT + 1];
};

// The experts of a token: lane j gets the j-th, -1 where none is left.  False in fp32: keys are so near each other that fp32 may have their order, or what is chosen, wrong; 64 bits then
// tell.  Told apart are neighbours among the chosen and the first that is not, and the last group that stays and the first that
// does not.  Keys of fp32 logits are exact.
template <typename KEY, int LPT, int EPL, bool GROUPED>
__device__ __forceinline__ bool choose(const RouteArgs &a, const float (&x)[EPL], float top, RouteLds<LPT, EPL, GROUPED> &lds, int l, int *mine)
{
    typedef Order<KEY> O;
    typedef typename O::type order_t;
    constexpr bool ROUNDED = sizeof(KEY) == 4;
    const int E = a.experts, e0 = l * EPL;
    const float inf = __builtin_inff();
    order_t key[EPL];
    KEY s[EPL];
    bool sure = true;
    const bool scored = !a.by_logit;
    float largest = 1.f;
    if (scored) {
        scores<KEY, LPT, EPL>(a.sigmoid, x, top, s, &largest);
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const KEY k = a.bias ? s[i] + (KEY)a.bias[min(e0 + i, E - 1)] : s[i];
            s[i] = x[i] > -inf && k > -(KEY)inf ? k : -(KEY)inf;             // (a NaN too)
        }
    } else {
#pragma unroll
        for (int i = 0; i < EPL; ++i) s[i] = (KEY)x[i];
    }
    // without a bias logits are in the order of the scores
#pragma unroll
    for (int i = 0; i < EPL; ++i) key[i] = s[i] > -(KEY)inf ? O::of(a.bias ? s[i] : (KEY)x[i]) : O::NONE;
    if constexpr (GROUPED) {
        const int G = a.groups, per = E / G;
        KEY *const keys = reinterpret_cast<KEY *>(lds.keys), *const values = reinterpret_cast<KEY *>(lds.values);
        [[maybe_unused]] float margins[ROUTE_MAX_GROUPS / LPT];                  // of the lane's groups
#pragma unroll
        for (int i = 0; i < EPL; ++i) keys[e0 + i] = s[i];
        wave_lds_fence();
#pragma unroll
        for (int n = 0; n < ROUTE_MAX_GROUPS / LPT; ++n) {
            const int g = n * LPT + l;
            if (g >= G) break;
            KEY b0 = -(KEY)inf, b1 = -(KEY)inf;
#pragma unroll 8
            for (int i = 0; i < per; ++i) {
                const KEY k = keys[g * per + i];
                b1 = k > b0 ? b0 : k > b1 ? k : b1;
                b0 = k > b0 ? k : b0;
            }
            KEY v = b0;
            if (a.group_best == 2 && b1 > -(KEY)inf) {
                v = b0 + b1;
                // (two near the lowest fp32 number: still ahead of a group without an expert)
                if constexpr (ROUNDED) v = fmaxf(v, -__FLT_MAX__);
            }
            values[g] = v;
            // What a value is off by at most: two scores; and, in parts of the larger key, since keys of either sign cancel in a sum, 2^-24 for each of them, 2 2^-24 for the sum
            // and 2 2^-24 for the comparison below.
            if constexpr (ROUNDED) {
                const float size = fmaxf(b0 > -inf ? fabsf(b0) : 0.f, b1 > -inf ? fabsf(b1) : 0.f);
                margins[n] = (a.sigmoid ? 0x1p-20f : 0x1p-15f * largest) + 0x1p-21f * size;
            }
        }
        wave_lds_fence();
        uint64_t stay = 0;
        KEY in_min = (KEY)inf, out_max = -(KEY)inf;
#pragma unroll
        for (int n = 0; n < ROUTE_MAX_GROUPS / LPT; ++n) {
            const int g0 = n * LPT, g = g0 + l;
            if (g0 >= G) break;
            int rank = 0;
            const KEY v = values[min(g, G - 1)];
#pragma unroll 8
            for (int h = 0; h < G; ++h) {
                const KEY w = values[h];
                rank += w > v || (w == v && h < g) ? 1 : 0;
            }
            const bool in = g < G && rank < a.top_groups;
            KEY margin = 0;
            if constexpr (ROUNDED) margin = margins[n];
            if (in && v - margin < in_min) in_min = v - margin;
            if (g < G && !in && v + margin > out_max) out_max = v + margin;
            const uint64_t b = __ballot(in) >> ((threadIdx.x & 63) & ~(LPT - 1));
            stay |= (LPT == 64 ? b : b & ((1ull << (LPT & 63)) - 1)) << g0;
        }
        if (ROUNDED && scored) {
            in_min = over_token<LPT>(in_min, Smaller{});
            out_max = over_token<LPT>(out_max, Larger{});
            // (groups without an expert are the last in any arithmetic)
            sure = out_max == -(KEY)inf || in_min > out_max;
        }
#pragma unroll
        for (int i = 0; i < EPL; ++i) key[i] = stay >> (min(e0 + i, E - 1) / per) & 1 ? key[i] : O::NONE;
    }
    // rounds: the best that is left, of equal ones that of the first lane, there the first.  Its lane writes it down.
    const bool check = ROUNDED && a.bias != nullptr;                         // then one round more, for the first that is not chosen
    const int lane = threadIdx.x & 63;
    [[maybe_unused]] const uint64_t below = ((1ull << lane) - 1) & ~((1ull << (lane & ~(LPT - 1))) - 1);         // the token's lanes ahead of this one
    float my_key = 0.f, last_key = 0.f;
    for (int j = 0; j < a.topk + (check ? 1 : 0); ++j) {
        order_t best = O::NONE;
#pragma unroll
        for (int i = 0; i < EPL; ++i) best = key[i] > best ? key[i] : best;
        const order_t own = best;
        best = over_token<LPT>(best, Larger{});
        const uint64_t who = __ballot(own == best);
        const bool owner = LPT == 64 ? l == (int)__builtin_ctzll(who) : own == best && !(who & below);
        int slot = 0;
        bool left = owner;                                       // (masks: scalar instructions beside the vector ones)
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const bool here = left && key[i] == best;
            left = left && !here;
            key[i] = here ? O::NONE : key[i];
            slot = here ? i : slot;
        }
        if (owner) lds.chosen[j] = best != O::NONE ? e0 + slot : -1;
        if constexpr (ROUNDED) {
            last_key = O::value(best);
            my_key = l == j ? last_key : my_key;
        }
    }
    wave_lds_fence();
    *mine = l < a.topk ? lds.chosen[l] : -1;
    if constexpr (ROUNDED) {
        if (check) {
            const int next = l < a.topk ? lds.chosen[l + 1] : -1;
            const float down = __shfl_down(my_key, 1), next_key = l == a.topk - 1 ? last_key : down;             // (no lane keeps the key of round 64)
            // twice what two keys are off, twice over; of a softmax by the larger of the two scores.  All that are not chosen are held against the last that is, and behind the first of
            // them there may be one of a larger score, off by more: there by the largest there can be.  (12608 x 128 with a bias 12.6 us; by the largest of those that are not chosen 14.2.)
            if (next >= 0) {
                const float score = l == a.topk - 1 ? largest : fabsf(fmaxf(my_key - a.bias[lds.chosen[l]], next_key - a.bias[next]));
                const float far = (a.sigmoid ? 0x1p-20f : 0x1p-15f * score) + 0x1p-21f * fmaxf(fabsf(my_key), fabsf(next_key));
                if (!(my_key - next_key > far)) sure = false;
            }
        }
        return over_token<LPT>((int)sure, Smaller{}) != 0;
    }
    return true;
}

// What the weights of chosen logits are in proportion to, m the largest of them: exp(x - m), or the sigmoid times a power of e that keeps the largest away from
// zero.
__device__ __forceinline__ float chosen_share(bool sigmoid, float x, float m)
{
    if (!sigmoid) return expf(x - m);
    return m < 0.f ? expf(x - m) / (1.f + expf(x)) : 1.f / (1.f + expf(-x));
}

template <int DT, int LPT, int EPL, bool GROUPED> __global__ __launch_bounds__(256) void route_kernel(RouteArgs a)
{
    constexpr int TOKENS = 256 / LPT;
    __shared__ RouteLds<LPT, EPL, GROUPED> lds[TOKENS];
    fetch_args<RouteArgs>();
    const int l = threadIdx.x % LPT, slot = threadIdx.x / LPT;
    const long t = (long)blockIdx.x * TOKENS + slot;
    const uint8_t *row = a.logits + (t < a.tokens ? t : a.tokens - 1) * a.ld;
    const float none = -__builtin_inff();
    float x[EPL];
    load_logits<DT, EPL>(row, l * EPL, a.experts, x);
    bool bad = false;
    float top = none;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        bad |= !(x[i] < __builtin_inff());
        top = fmaxf(top, x[i]);
    }
    bad = over_token<LPT>((int)bad, Larger{}) != 0;
    top = over_token<LPT>(top, Larger{});
    int e;
    // (a token without scores is not worth the second look)
    const bool sure = choose<float, LPT, EPL, GROUPED>(a, x, top, lds[slot], l, &e) || bad;
    if (__builtin_expect(__any(!sure), 0)) choose<double, LPT, EPL, GROUPED>(a, x, top, lds[slot], l, &e);
    const bool there = l < a.topk && e >= 0;
    const float xe = there ? logit_at<DT>(row, e) : none;
    float w;
    if (a.normalise) {
        const float m = over_token<LPT>(xe, Larger{});
        const float s = there ? chosen_share(a.sigmoid, xe, m) : 0.f;
        w = s / over_token<LPT>(s, Plus{});
    } else if (a.sigmoid) {
        w = 1.f / (1.f + expf(-xe));
    } else {
        const float m = top > none ? top : 0.f;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) sum += expf(x[i] - m);
        w = expf(xe - m) / over_token<LPT>(sum, Plus{});
    }
    if (l < a.topk && t < a.tokens) {
        a.expert[t * a.topk + l] = bad ? l : e;
        a.weight[t * a.topk + l] = bad ? __builtin_nanf("") : there ? a.scale * w : 0.f;
    }
}

// The gradient.  With p the normalised shares and D = sum p dw: chosen logits get scale p (dw - D), times 1 - sigmoid where scores are sigmoids; without
// normalising, s (g - sum g s) over all experts, or scale dw s (1 - s) for the chosen.
template <int DT, int LPT, int EPL> __global__ __launch_bounds__(256) void route_grad_kernel(RouteArgs a)
{
    constexpr int TOKENS = 256 / LPT;
    constexpr uint32_t EMPTY = 0x7FC0A5A5u;                      // (a NaN that hardly ever is a gradient; one that is goes the longer way below)
    __shared__ float lds[TOKENS * LPT * EPL];
    fetch_args<RouteArgs>();
    const int l = threadIdx.x % LPT, slot = threadIdx.x / LPT, e0 = l * EPL;
    const long t = (long)blockIdx.x * TOKENS + slot, tt = t < a.tokens ? t : a.tokens - 1;
    const uint8_t *row = a.logits + tt * a.ld;
    const float none = -__builtin_inff();
    float *const g = lds + slot * LPT * EPL;
    float x[EPL];
    load_logits<DT, EPL>(row, e0, a.experts, x);
    bool bad = false;
    float top = none;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        bad |= !(x[i] < __builtin_inff());
        top = fmaxf(top, x[i]);
        g[e0 + i] = __uint_as_float(EMPTY);
    }
    bad = over_token<LPT>((int)bad, Larger{}) != 0;
    const int e = l < a.topk ? a.expert[tt * a.topk + l] : -1;
    const bool in = e >= 0 && e < a.experts;
    const float xe = in ? logit_at<DT>(row, e) : none;
    const bool there = in && xe > none;
    const float dw = there ? a.scale * a.dweight[tt * a.topk + l] : 0.f;
    wave_lds_fence();
    const bool spread = !a.normalise && !a.sigmoid;              // the gradient reaches experts that were not chosen
    float m = 0.f, sum = 1.f;
    if (spread) {
        top = over_token<LPT>(top, Larger{});
        m = top > none ? top : 0.f;
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) sum += expf(x[i] - m);
        sum = over_token<LPT>(sum, Plus{});
        if (!(top > none)) sum = 1.f;                            // (no expert: all scores are zero)
    }
    float d;                                                     // of the chosen logit; spread: of its score
    if (a.normalise) {
        const float mc = over_token<LPT>(there ? xe : none, Larger{});
        const float s = there ? chosen_share(a.sigmoid, xe, mc) : 0.f;
        const float total = over_token<LPT>(s, Plus{}), p = total > 0.f ? s / total : 0.f;
        d = p * (dw - over_token<LPT>(p * dw, Plus{}));
        if (a.sigmoid) d *= 1.f / (1.f + expf(xe));
    } else if (a.sigmoid) {
        const float s = 1.f / (1.f + expf(-xe));
        d = dw * s / (1.f + expf(xe));
    } else {
        d = dw;
    }
    if (there) g[e] = d;
    wave_lds_fence();
    const float D = spread ? over_token<LPT>(there ? dw * expf(xe - m) / sum : 0.f, Plus{}) : 0.f;
    float v[EPL];
    int filled = 0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        v[i] = g[e0 + i];
        const bool full = __float_as_uint(v[i]) != EMPTY;
        filled += __popcll(__ballot(full));
        v[i] = full ? v[i] : 0.f;
    }
    // fewer places than choices: some token of the wave names an expert twice.  (Additions to begin with: 11.6 us for 10.9, both directions of 12608 x 128.)
    if (__builtin_expect(filled != __popcll(__ballot(there)), 0)) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) g[e0 + i] = 0.f;
        wave_lds_fence();
        if (there) unsafeAtomicAdd(g + e, d);
        wave_lds_fence();
#pragma unroll
        for (int i = 0; i < EPL; ++i) v[i] = g[e0 + i];
    }
    if (t >= a.tokens) return;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        if (spread) v[i] = expf(x[i] - m) / sum * (v[i] - D);
        if (bad) v[i] = __builtin_nanf("");
    }
    store_logits<DT, EPL>(a.dlogits + t * a.ldd, e0, a.experts, v);
}

// ------------------------------------------------------------------------------------------
template <int DT, int LPT, int EPL> static hipError_t launch_one(const RouteArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)(((long)a.tokens + 256 / LPT - 1) / (256 / LPT)));
    if (a.groups > 1) hipLaunchKernelGGL((route_kernel<DT, LPT, EPL, true>), grid, dim3(256), 0, st, a);
    else              hipLaunchKernelGGL((route_kernel<DT, LPT, EPL, false>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}
template <int DT, int LPT, int EPL> static hipError_t launch_grad(const RouteArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL((route_grad_kernel<DT, LPT, EPL>), dim3((unsigned)(((long)a.tokens + 256 / LPT - 1) / (256 / LPT))), dim3(256), 0, st, a);
    return hipGetLastError();
}
template <int DT> static hipError_t launch_type(const RouteArgs &a, hipStream_t st)
{
    // Many tokens of few experts: sixteen lanes to a token, four of which share a wave's instructions.  Else a wave, with shorter lists in its lanes.  (us in a graph, fp32, 8 choices, sixteen lanes /
    // a wave: softmax, 12608 tokens 64 experts in 8 groups 9.8 / 14.6, 128 experts 5.8 / 9.2, 256 in 8 groups 22.3 / 21.6, 6000 x 64 3.8 / 5.1, 4096 x 64 3.6 / 4.1; sigmoid with bias, 12608 x 256
    // 20.9 / 14.6, 6000 x 128 11.0 / 7.7, 4096 x 64 4.5 / 4.6, 4096 x 128 9.9 / 7.0, 2048 x 256 15.9 / 7.7; a second look in 64 bits by a few tokens is in those of the bias, four to a wave.)
    if (a.experts <= 128 && a.topk < 16 && a.tokens > 4096) {
        if (a.experts <= 32)  return launch_one<DT, 16, 2>(a, st);
        if (a.experts <= 64)  return launch_one<DT, 16, 4>(a, st);
        return launch_one<DT, 16, 8>(a, st);
    }
    if (a.experts <= 64)  return launch_one<DT, 64, 1>(a, st);
    if (a.experts <= 128) return launch_one<DT, 64, 2>(a, st);
    if (a.experts <= 256) return launch_one<DT, 64, 4>(a, st);
    if (a.experts <= 512) return launch_one<DT, 64, 8>(a, st);
    return launch_one<DT, 64, 16>(a, st);
}
template <int DT> static hipError_t launch_grad_type(const RouteArgs &a, hipStream_t st)
{
    if (a.experts <= 256 && a.topk <= 16) {
        if (a.experts <= 32)  return launch_grad<DT, 16, 2>(a, st);
        if (a.experts <= 64)  return launch_grad<DT, 16, 4>(a, st);
        if (a.experts <= 128) return launch_grad<DT, 16, 8>(a, st);
        return launch_grad<DT, 16, 16>(a, st);
    }
    if (a.experts <= 256) return launch_grad<DT, 64, 4>(a, st);
    if (a.experts <= 512) return launch_grad<DT, 64, 8>(a, st);
    return launch_grad<DT, 64, 16>(a, st);
}
template <int DT> static hipError_t launch_either(bool grad, const RouteArgs &a, hipStream_t st) { return grad ? launch_grad_type<DT>(a, st) : launch_type<DT>(a, st); }
hipError_t launch_route(int dt, bool grad, const RouteArgs &a, hipStream_t st)
{
    return dt == DT_F32 ? launch_either<DT_F32>(grad, a, st) : dt == DT_BF16 ? launch_either<DT_BF16>(grad, a, st) : launch_either<DT_F16>(grad, a, st);
}

}  // namespace abft
