// Training the router: routing with per-expert counts and a balance loss, and the gradient of the logits.
//   balance   pi = softmax(logits), K = top-k;  counts[e] = #{t : e in K_t}, P[e] = mean_t pi_t[e],  loss = E sum_e f_e P_e with
//             f_e = counts[e] / (k n), over the n tokens of a group that count
//   logits    g_t[e] = [e in K_t] dw + d_loss (E / n) f_e,   d_logits = pi (g - <pi, g>)
// A token lies in G lanes, eight consecutive experts to a lane: one 16-byte piece of a bf16 row, so that a wave's loads are
// contiguous where the experts fill the lanes.
#include "rows.hpp"

namespace swimba {

// Order of 16-bit pairs of bf16 bits as unsigned numbers: -0 as +0, NaN outside the numbers by sign.
__device__ __forceinline__ uint32_t order_of_pair(uint32_t u)
{
    typedef int16_t __attribute__((ext_vector_type(2))) s16x2;
    const uint32_t neg = __builtin_bit_cast(uint32_t, __builtin_bit_cast(s16x2, u) >> (int16_t)15);
    const uint32_t add = (neg & 0x80018001u) ^ 0x80008000u;            // positive u: u + 2^15; negative: ~u + 1
    return __builtin_bit_cast(uint32_t, (s16x2)(__builtin_bit_cast(s16x2, u ^ neg) + __builtin_bit_cast(s16x2, add)));
}
__device__ __forceinline__ uint32_t order_of(float f)
{
    const uint32_t u = __float_as_uint(f + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t umin(uint32_t a, uint32_t b) { return a < b ? a : b; }

// One token in G lanes, 8 NP experts to a lane: piece i of lane l are the experts from 8 (l + G i) on.
// A key is larger the earlier its expert is picked, and 0 past the last expert.  Its lowest bits are the expert's, counted
// down, so that all keys differ and name their experts; above them lie all 16 bits of a bf16 logit's order, or the upper 24 of
// an fp32 one's, which do not decide between logits that agree that far: those are picked by the whole of them (`close`).
// FULL: the experts fill the lanes.
template <typename T, int NP, int G, bool FULL> struct Token {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int SIZE = 8 * NP * G, ROUNDS = SIZE < SWIMBA_MAX_TOPK ? SIZE : SWIMBA_MAX_TOPK, SLOTS = (ROUNDS + G - 1) / G;
    static constexpr uint32_t LOW = BF ? 0xffffu : 0xffu;
    const Piece<T, 8> (&p)[NP];
    const int l, E;
    uint32_t key[NP][8], best;
    float top;                                                 // largest logit

    __device__ __forceinline__ int expert(int i, int j) const { return 8 * (l + G * i) + j; }
    __device__ __forceinline__ bool real(int i, int j) const { return FULL || expert(i, j) < E; }
    __device__ __forceinline__ Token(const Piece<T, 8> (&pieces)[NP], int lane, int experts) : p(pieces), l(lane), E(experts)
    {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t low = LOW - expert(i, j);
                uint32_t k;
                if constexpr (BF) {
                    const uint32_t s = order_of_pair(p[i].v[j / 2]);
                    k = j % 2 ? (s & 0xffff0000u) | low : s << 16 | low;
                } else {
                    const uint32_t s = order_of(p[i].get(j));
                    most = umax(most, real(i, j) ? s : 0);
                    k = (s & ~LOW) | low;
                }
                key[i][j] = real(i, j) ? k : 0;
            }
        best = over([&](int i, int j) { return key[i][j]; }, umax);
        if constexpr (BF) {
            const uint32_t s = best >> 16;
            top = __uint_as_float((s & 0x8000u ? s ^ 0x8000u : 0u - s) << 16);
        } else {
            most = over_group<G>(most, umax);
            top = __uint_as_float(most & 0x80000000u ? most ^ 0x80000000u : ~most);
        }
    }
    template <typename F> __device__ __forceinline__ uint32_t over(F f, uint32_t (*op)(uint32_t, uint32_t)) const
    {
        uint32_t v = f(0, 0);
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v = op(v, f(i, j));
        return over_group<G>(v, op);
    }
    // largest key below `best`: at the smallest distance under it, those at and above it being far away
    __device__ __forceinline__ uint32_t next(uint32_t best) const
    {
        return best - 1 - over([&](int i, int j) { return best - 1 - key[i][j]; }, umin);
    }
    static __device__ __forceinline__ int expert_of(uint32_t k) { return (int)(LOW - (k & LOW)); }

    // The K picks: lane l keeps the experts of rounds l, l + G, ...
    __device__ __forceinline__ void picks(int K, int (&e)[SLOTS]) const
    {
        uint32_t b = best;
        bool close = false;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            uint32_t mine = 0;
            const int rounds = min(K - i * G, G);
#pragma unroll 1
            for (int r = 0; r < rounds; ++r) {
                mine = l == r ? b : mine;
                const uint32_t n = next(b);
                if (!BF) close = close || ((b ^ n) & ~LOW) == 0;
                b = n;
            }
            e[i] = expert_of(mine);
        }
        if constexpr (!BF) {
            if (__any(close)) {                                // whole keys, equal ones by the expert
                uint32_t last = ~0u;
                int x = -1;
                auto order = [&](int i, int j) { return order_of(p[i].get(j)); };
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r)
                    if (r < K) {
                        auto behind = [&](int i, int j) {
                            const uint32_t o = order(i, j);
                            return real(i, j) && (r == 0 || o < last || (o == last && expert(i, j) > x));
                        };
                        const uint32_t o = over([&](int i, int j) { return behind(i, j) ? order(i, j) : 0u; }, umax);
                        x = (int)over([&](int i, int j) { return behind(i, j) && order(i, j) == o ? (uint32_t)expert(i, j) : 1u << 20; }, umin);
                        last = o;
                        if (l == r % G) e[r / G] = x;
                    }
            }
        }
    }
};

// loss of a group from the sums of its probabilities and its counts, which the threads below E hold
__device__ __forceinline__ void balance_finish(float p, int c, int64_t grp, int E, int K, int32_t *counts, float *prob_mean,
                                               float *loss, double (*lds)[4])
{
    // E <= 256: four waves hold the experts
    const int e = threadIdx.x;
    auto total = [&](double v, int row) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
        if (e < 256 && (e & 63) == 0) lds[row][e >> 6] = v;
        __syncthreads();
        return lds[row][0] + lds[row][1] + lds[row][2] + lds[row][3];
    };
    const double all = total(e < E ? (double)c : 0., 0);       // k n
    const float mean = all > 0. ? (float)((double)p * K / all) : 0.f;
    const double l = total(e < E && all > 0. ? (double)c / all * mean : 0., 1);
    if (e < E) {
        counts[grp * E + e] = c;
        if (prob_mean) prob_mean[grp * E + e] = mean;
    }
    if (e == 0) loss[grp] = (float)(E * l);
}

// Threads of the largest block: more experts to a lane take more registers.
constexpr int balance_most(int NP) { return NP > 2 ? 512 : 1024; }

// A block walks its slice of a group's tokens; part (groups, slices, E): {sum of probabilities, count}.  With one slice to a
// group the block has all of it and finishes the loss itself.
template <typename T, int NP, int G, bool FULL>
__global__ void __launch_bounds__(balance_most(NP))
balance_kernel(const T *__restrict__ logits, const uint8_t *__restrict__ mask, int32_t *__restrict__ topk_idx,
               float *__restrict__ topk_w, float2 *__restrict__ part, int64_t tokens, int slices, int E, int K,
               int32_t *__restrict__ counts, float *__restrict__ prob_mean, float *__restrict__ loss)
{
    typedef Token<T, NP, G, FULL> Tok;
    __shared__ float psum[balance_most(NP) / 64][Tok::SIZE];
    __shared__ int csum[Tok::SIZE];
    __shared__ double fin[2][4];
    const int64_t grp = blockIdx.x / slices;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane % G, at = lane / G;
    const int64_t stride = (int64_t)slices * (blockDim.x / G);
    const T *const z = logits + grp * tokens * E;
    if (threadIdx.x < Tok::SIZE) csum[threadIdx.x] = 0;
    __syncthreads();
    float acc[NP][8] = {};
    struct Step {
        Piece<T, 8> p[NP];
        uint8_t on;
    };
    auto fetch = [&](Step &s, int64_t t) __attribute__((always_inline)) {        // t: first token of the wave
        const bool in = t + at < tokens;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int e = 8 * (l + G * i);
            s.p[i].template load<!FULL>(z + t * E + (uint32_t)(at * E + e), in ? E - e : 0);
        }
        s.on = in && (!mask || mask[grp * tokens + t + at]);
    };
    int64_t t = (int64_t)(blockIdx.x % slices) * (blockDim.x / G) + wave * (64 / G);
    Step next;
    if (t < tokens) fetch(next, t);
    for (; t < tokens; t += stride) {
        const Step s = next;
        if (t + stride < tokens) fetch(next, t + stride);
        const Tok tok(s.p, l, E);
        int e[Tok::SLOTS];
        tok.picks(K, e);
        const float m = tok.top;
        bool on = s.on;
        if (__any(m == -INFINITY)) {                           // a token whose logits are all -inf does not count
            uint32_t other = 0;
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) other |= tok.real(i, j) && s.p[i].get(j) != -INFINITY;
            on = on && over_group<G>(other, umax);
        }
        float p[NP][8], Z = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                p[i][j] = tok.real(i, j) ? route_exp(s.p[i].get(j) - m) : 0.f;
                Z += p[i][j];
            }
        const float invZ = 1.0f / group_sum<G>(Z);
        if (t + at < tokens) {
            const int64_t row = grp * tokens + t + at;
#pragma unroll
            for (int i = 0; i < Tok::SLOTS; ++i) {
                const int r = i * G + l;
                if (r < K) {
                    if (topk_idx) topk_idx[row * K + r] = e[i];
                    if (topk_w) topk_w[row * K + r] = route_exp(to_float(logits[row * E + e[i]]) - m) * invZ;
                    if (on) atomicAdd(&csum[e[i]], 1);         // whole numbers: the order does not matter
                }
            }
        }
        if (on) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[i][j] += p[i][j] * invZ;
        }
    }
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = __uint_as_float(over_lanes<G, 64>(__float_as_uint(acc[i][j]), add_f32));
            if (lane < G) psum[wave][8 * (l + G * i) + j] = v;
        }
    __syncthreads();
    const int x = threadIdx.x;
    float v = 0.f;
    int c = 0;
    if (x < E) {
        c = csum[x];
        for (int w = 0; w < (int)blockDim.x / 64; ++w) v += psum[w][x];
    }
    if (slices == 1) balance_finish(v, c, grp, E, K, counts, prob_mean, loss, fin);
    else if (x < E) part[(int64_t)blockIdx.x * E + x] = make_float2(v, __int_as_float(c));
}

// The slices joined, each thread every (1024 / width)-th of an expert, 16 of them under way.
__global__ void __launch_bounds__(1024)
balance_loss_kernel(const float2 *__restrict__ part, int slices, int width, int E, int K, int32_t *__restrict__ counts,
                    float *__restrict__ prob_mean, float *__restrict__ loss)
{
    __shared__ float2 lds[1024];
    __shared__ double fin[2][4];
    const int64_t grp = blockIdx.x;
    const int e = threadIdx.x % width, n = 1024 / width;
    int c = 0;
    float p = 0.f;
    if (e < E) {
#pragma unroll 16
        for (int s = threadIdx.x / width; s < slices; s += n) {
            const float2 v = part[(grp * slices + s) * E + e];
            p += v.x;
            c += __float_as_int(v.y);
        }
    }
    lds[threadIdx.x] = make_float2(p, __int_as_float(c));
    __syncthreads();
    p = 0.f;
    c = 0;
    if (threadIdx.x < width)
        for (int i = 0; i < n; ++i) {
            p += lds[i * width + e].x;
            c += __float_as_int(lds[i * width + e].y);
        }
    balance_finish(p, c, grp, E, K, counts, prob_mean, loss, fin);
}

namespace {

int power_of_two(int n)
{
    int p = 1;
    while (p < n) p *= 2;
    return p;
}
int lanes_of(int E) { return power_of_two((E + 7) / 8); }      // of a token, eight experts to a lane
// Eight lanes at most for the routing: steps over lanes cost as much as three experts of a lane, and with few tokens to a wave
// so does what is done once for all of them.
int pieces_of(int E) { return E <= 64 ? 1 : E <= 128 ? 2 : 4; }
int routing_lanes_of(int E) { return E <= 64 ? lanes_of(E) : 8; }

// Threads of a block and slices of a group.  A group that a block walks in four steps or less stays with one block, without a
// second launch; beyond, a slice is a step or more, and the slices of all groups are some 256 (a few more where groups are
// many), which fill the chip with waves and are soon added up.
struct Slices { int threads; int64_t count; };
Slices balance_slices(int64_t groups, int64_t tokens, int E)
{
    const int most = balance_most(pieces_of(E));
    const int64_t threads = tokens * routing_lanes_of(E), steps = (threads + most - 1) / most;
    if (steps <= 4 || groups >= 256) {
        int n = 256;
        while (n < most && n < threads) n *= 2;
        return {n, 1};
    }
    const int64_t slices = 1024 / most * 256 / groups + 1;
    return {most, steps < slices ? steps : slices};
}

// f(lanes, whether the last piece is short, whether the experts fill the lanes) as constants
template <typename F>
void with_lanes(int E, F &&f)
{
    using std::integral_constant;
    auto tail = [&](auto g) {
        if (E % 8) f(g, std::true_type(), std::false_type());
        else if (E < 8 * g) f(g, std::false_type(), std::false_type());
        else f(g, std::false_type(), std::true_type());
    };
    switch (lanes_of(E)) {
    case 1: return tail(integral_constant<int, 1>());
    case 2: return tail(integral_constant<int, 2>());
    case 4: return tail(integral_constant<int, 4>());
    case 8: return tail(integral_constant<int, 8>());
    case 16: return tail(integral_constant<int, 16>());
    default: return tail(integral_constant<int, 32>());
    }
}

}  // namespace

size_t balance_bytes(int64_t groups, int64_t tokens, int E)
{
    const int64_t n = balance_slices(groups, tokens, E).count;
    return n > 1 ? (size_t)groups * n * E * sizeof(float2) : 0;
}

swimba_status launch_router_balance(int64_t groups, int64_t tokens, int E, int K, int io_dtype, const void *logits,
                                    const uint8_t *mask, int32_t *topk_idx, float *topk_w, int32_t *counts, float *prob_mean,
                                    float *loss, void *part, hipStream_t st)
{
    if (groups == 0) return SWIMBA_OK;
    const Slices s = balance_slices(groups, tokens, E);
    with_lanes(E, [&](auto lanes, auto, auto full) {
        constexpr int G = lanes() < 8 ? lanes() : 8, NP = lanes() / G;
        auto go = [&](auto kernel, auto *z) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(groups * s.count)), dim3(s.threads), 0, st, z, mask, topk_idx, topk_w, (float2 *)part,
                               tokens, (int)s.count, E, K, counts, prob_mean, loss);
        };
        if (io_dtype == SWIMBA_BF16) go(balance_kernel<bf16, NP, G, full()>, (const bf16 *)logits);
        else go(balance_kernel<float, NP, G, full()>, (const float *)logits);
    });
    SWIMBA_CHECK_LAUNCH();
    if (s.count > 1) {
        hipLaunchKernelGGL(balance_loss_kernel, dim3((unsigned)groups), dim3(1024), 0, st, (const float2 *)part, (int)s.count, power_of_two(E), E, K,
                           counts, prob_mean, loss);
        SWIMBA_CHECK_LAUNCH();
    }
    return SWIMBA_OK;
}

// The gradients of a token's routing weights are laid at their experts through LDS: a wave's 64 / G tokens are 512 floats,
// element j of lane i at 8 i + j.
template <typename T, int G, bool TAIL>
__global__ void __launch_bounds__(256)
router_bwd_kernel(const T *__restrict__ logits, const uint8_t *__restrict__ mask, const int32_t *__restrict__ topk_idx,
                  const float *__restrict__ d_topk_w, const int32_t *__restrict__ counts, const float *__restrict__ d_loss,
                  T *__restrict__ d_logits, int64_t tokens, int64_t per_group, int E, int K)
{
    constexpr int SLOTS = Token<T, 1, G, true>::SLOTS;
    __shared__ float lds[4][512];
    const int64_t grp = blockIdx.x / per_group;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane % G, at = lane / G;
    float *const mine = lds[wave] + 8 * lane, *const token = lds[wave] + 8 * (lane - l);
    float share[8] = {};                                        // d_loss (E / n) f_e
    if (counts) {
        double all = 0.;
        int c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            c[j] = 8 * l + j < E ? counts[grp * E + 8 * l + j] : 0;
            all += c[j];
        }
#pragma unroll
        for (int o = 1; o < G; o *= 2) all += __shfl_xor(all, o);
        const double scale = all > 0. ? (double)d_loss[grp] * E * K / all : 0.;
#pragma unroll
        for (int j = 0; j < 8; ++j) share[j] = all > 0. ? (float)(scale * (c[j] / all)) : 0.f;
    }
    const T *const z = logits + grp * tokens * E;
    T *const out = d_logits + grp * tokens * E;
    const int64_t stride = per_group * (256 / G);
    struct Step {
        Piece<T, 8> p;
        float dw[SLOTS];
        int e[SLOTS];
        uint8_t on;
    };
    auto fetch = [&](Step &s, int64_t t) __attribute__((always_inline)) {
        const bool in = t + at < tokens;
        const int64_t row = grp * tokens + t + at;
        s.p.template load<TAIL>(z + t * E + (uint32_t)(at * E + 8 * l), in ? E - 8 * l : 0);
        s.on = in && counts && (!mask || mask[row]);
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            const int r = i * G + l;
            s.e[i] = -1;
            s.dw[i] = 0.f;
            if (d_topk_w && in && r < K) {
                s.e[i] = topk_idx[row * K + r];
                s.dw[i] = d_topk_w[row * K + r];
            }
        }
    };
    int64_t t = (blockIdx.x % per_group) * (256 / G) + wave * (64 / G);
    Step next;
    if (t < tokens) fetch(next, t);
    for (; t < tokens; t += stride) {
        const Step s = next;
        if (t + stride < tokens) fetch(next, t + stride);
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = s.on ? share[j] : 0.f;
        uint32_t some = s.on;                                   // whether the token has a gradient at all
        if (d_topk_w) {
#pragma unroll
            for (int j = 0; j < 8; ++j) mine[j] = g[j];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                some |= s.dw[i] != 0.f;
                if ((uint32_t)s.e[i] < (uint32_t)E) atomicAdd(token + s.e[i], s.dw[i]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = mine[j];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        float f[8], m = -INFINITY;
        uint32_t any = 0;                                       // whether it has a logit above -inf
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = 8 * l + j < E ? s.p.get(j) : -INFINITY;
            m = fmaxf(m, f[j]);
            any |= f[j] != -INFINITY;
        }
        m = __uint_as_float(over_group<G>(__float_as_uint(m), max_f32));
        const uint32_t both = over_group<G>(any | some << 1, or_u32);
        float p[8], Z = 0.f, dot = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            p[j] = 8 * l + j < E ? route_exp(f[j] - m) : 0.f;
            Z += p[j];
            dot += 8 * l + j < E ? p[j] * g[j] : 0.f;
        }
        const float invZ = 1.0f / group_sum<G>(Z);
        dot = group_sum<G>(dot) * invZ;
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = both == 3 ? p[j] * invZ * (g[j] - dot) : 0.f;
        if (t + at < tokens) store_piece<TAIL>(out + t * E + (uint32_t)(at * E + 8 * l), p, E - 8 * l);
    }
}

swimba_status launch_router_bwd(int64_t groups, int64_t tokens, int E, int K, int io_dtype, const void *logits, const uint8_t *mask,
                                const int32_t *topk_idx, const float *d_topk_w, const int32_t *counts, const float *d_loss,
                                void *d_logits, hipStream_t st)
{
    if (groups == 0 || tokens == 0) return SWIMBA_OK;
    const int64_t need = (tokens * lanes_of(E) + 255) / 256, fit = groups < 2048 ? 2048 / groups : 1, per_group = need < fit ? need : fit;
    with_lanes(E, [&](auto g, auto tail, auto) {
        auto go = [&](auto kernel, auto *z, auto *out) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(groups * per_group)), dim3(256), 0, st, z, mask, topk_idx, d_topk_w, counts, d_loss, out,
                               tokens, per_group, E, K);
        };
        if (io_dtype == SWIMBA_BF16) go(router_bwd_kernel<bf16, g(), tail()>, (const bf16 *)logits, (bf16 *)d_logits);
        else go(router_bwd_kernel<float, g(), tail()>, (const float *)logits, (float *)d_logits);
    });
    SWIMBA_CHECK_LAUNCH();
    return SWIMBA_OK;
}

}  // namespace swimba
