// Training the router: routing with per-expert counts and a balance loss, and the gradient of the logits.
//   balance   pi = softmax(logits), K = top-k;  counts[e] = #{t : e in K_t}, P[e] = mean_t pi_t[e],  loss = E sum_e f_e P_e with
//             f_e = counts[e] / (k n), over the n tokens of a group that count
//   logits    g_t[e] = [e in K_t] dw + d_loss (E / n) f_e,   d_logits = pi (g - <pi, g>)
// A token lies in G lanes, in pieces of eight consecutive experts: 16 bytes of a bf16 row, so that a wave's loads are contiguous
// where the experts fill the lanes.
// Few experts are bound by memory and by their launches (2 x 16384 x 16 with padding 11.2 us, its gradient 4.8); many by what
// the vector units have to issue: of the 30 us of 131072 x 256 top-8 in bf16 (75 MB, 13 us for a kernel that only moves them) they
// are busy nine tenths, half of it with the picks.  In fp32 more than 64 experts take 231 to 240 registers: two waves to a SIMD
// (65536 x 256 27 us, the units busy six tenths).  65 to 255 experts in bf16 and 33 to 63 in fp32 spill 2 to 6 registers.
// The gradient is bound by memory in fp32 (65536 x 256 29.5 us, 4.7 TB/s); in bf16, with twice the tokens for the bytes, the vector units
// are busy three quarters of the time (131072 x 256 37 us, 26 for the bytes alone).
#include "rows.hpp"

namespace swimba {

// Place of a logit among all: smaller the larger it is, -0 as +0, NaN outside the numbers by sign.  Of two bf16 at once,
// as 16-bit numbers, and of a float.
__device__ __forceinline__ uint32_t place_of_pair(uint32_t u)
{
    typedef uint16_t __attribute__((ext_vector_type(2))) u16x2;
    typedef int16_t __attribute__((ext_vector_type(2))) s16x2;
    const uint32_t neg = __builtin_bit_cast(uint32_t, __builtin_bit_cast(s16x2, u) >> (int16_t)15);
    const uint32_t from = (neg & 0x80018001u) ^ 0x7fff7fffu;           // positive u: 2^15 - 1 - u; negative: -2 - ~u
    return __builtin_bit_cast(uint32_t, (u16x2)(__builtin_bit_cast(u16x2, from) - __builtin_bit_cast(u16x2, u ^ neg)));
}
__device__ __forceinline__ float at_place(uint32_t place)              // of a bf16, in the lower half
{
    const uint32_t s = ~place;
    return __uint_as_float((s & 0x8000u ? s ^ 0x8000u : 0u - s) << 16);
}
__device__ __forceinline__ uint32_t place_of(float f)
{
    const uint32_t u = __float_as_uint(f + 0.0f);
    return u ^ (~(uint32_t)((int32_t)u >> 31) & 0x7fffffffu);
}
__device__ __forceinline__ float at_whole_place(uint32_t place) { return __uint_as_float(place & 0x80000000u ? place : place ^ 0x7fffffffu); }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t umin(uint32_t a, uint32_t b) { return a < b ? a : b; }

// One token in G lanes, 8 NP experts to a lane: piece i of lane l are the experts from 8 (l + G i) on.
// A key is smaller the earlier its expert is picked.  Its lowest bits are the expert's number, so that all keys differ and
// name their experts; above them lies the place of a bf16 logit, or the upper 24 bits of an fp32 one's, which do not decide
// between logits that agree that far: those are put in order by the whole of them (`close`).  The lane's part of the number, 8 l,
// is not in the stored keys: it is added to what a lane has found.  FULL: the experts fill the lanes.
template <typename T, int NP, int G, bool FULL> struct Token {
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int SIZE = 8 * NP * G, ROUNDS = SIZE < SWIMBA_MAX_TOPK ? SIZE : SWIMBA_MAX_TOPK, SLOTS = (ROUNDS + G - 1) / G;
    static constexpr uint32_t LOW = BF ? 0xffffu : 0xffu, NONE = ~0u;
    const Piece<T, 8> (&p)[NP];
    const int l, E;
    uint32_t key[NP][8], best;
    float top;                                                 // largest logit

    __device__ __forceinline__ int expert(int i, int j) const { return 8 * (l + G * i) + j; }
    __device__ __forceinline__ bool real(int i, int j) const { return FULL || expert(i, j) < E; }
    __device__ __forceinline__ Token(const Piece<T, 8> (&pieces)[NP], int lane, int experts) : p(pieces), l(lane), E(experts)
    {
        uint32_t whole = NONE;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t low = 8 * G * i + j;
                uint32_t k;
                if constexpr (BF) {
                    const uint32_t s = place_of_pair(p[i].v[j / 2]);
                    k = j % 2 ? (s & 0xffff0000u) | low : s << 16 | low;
                } else {
                    const uint32_t s = place_of(p[i].get(j));
                    whole = umin(whole, real(i, j) ? s : NONE);
                    k = (s & ~LOW) | low;
                }
                key[i][j] = real(i, j) ? k : NONE - 8 * l;
                asm("" : "+v"(key[i][j]));                     // the whole key: taken apart, it would cost every pick an addition
            }
        best = over([&](int i, int j) { return key[i][j]; }, umin, 8 * l);
        top = BF ? at_place(best >> 16) : at_whole_place(over_group<G>(whole, umin));
    }
    // op over the lanes of f over the lane's experts, with `more` added in each lane
    template <typename F> __device__ __forceinline__ uint32_t over(F f, uint32_t (*op)(uint32_t, uint32_t), uint32_t more = 0) const
    {
        uint32_t v = f(0, 0);
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v = op(v, f(i, j));
        return over_group<G>(v + more, op);
    }
    // smallest key above `last`: at the smallest distance over it, those at and below it being far away
    __device__ __forceinline__ uint32_t next(uint32_t last) const
    {
        const uint32_t from = last + 1 - 8 * l;
        return last + 1 + over([&](int i, int j) { return key[i][j] - from; }, umin);
    }

    __device__ __forceinline__ bool names(uint32_t k) const { return k != NONE && (int)(k & LOW) < E; }
    static __device__ __forceinline__ bool near(uint32_t a, uint32_t b) { return ((a ^ b) & ~LOW) == 0; }

    // The K picks: lane l keeps the experts of rounds l, l + G, ... and, of bf16, their logits.  Of fp32 logits, whether some agree
    // in their keys' upper bits, down to the pick behind the last, which is `behind` (-1: there is none).
    __device__ __forceinline__ bool picks(int K, int (&e)[SLOTS], float (&v)[SLOTS], int &behind) const
    {
        uint32_t b = best;
        bool close = false, end = false;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            uint32_t mine = 0;
            const int rounds = min(K - i * G, G);
#pragma unroll 1
            for (int r = 0; r < rounds; ++r) {
                mine = l == r ? b : mine;
                if (BF && i * G + r == K - 1) break;
                const uint32_t n = next(b);
                if (!BF) {
                    end = n > b && near(b, n);
                    close = close || end;
                    if (i * G + r == K - 1) behind = n > b && names(n) ? (int)(n & LOW) : -1;
                }
                b = n;
            }
            e[i] = mine & LOW;
            v[i] = BF ? at_place(mine >> 16) : 0.f;
        }
        if constexpr (!BF) {
            // agreement that goes on behind that pick leaves the choice to settle()
            if (__any(end) && end && behind >= 0) {
                const uint32_t n = next(b);
                if (n > b && near(b, n)) behind = -2;
            }
        }
        return close;
    }
    // Which of the logits that agree with the last pick in their keys' upper bits are picked, where more do than there are picks left
    // (`open`): by the lower bits of their places, equal ones by the expert.  The picks with other upper bits stay.
    __device__ __forceinline__ void settle(int K, int (&e)[SLOTS], const float (&v)[SLOTS], bool open) const
    {
        uint32_t upper = 0, before = 0;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) upper = i * G + l < K ? umax(upper, place_of(v[i]) & ~LOW) : upper;
        upper = over_group<G>(upper, umax);
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) before += i * G + l < K && place_of(v[i]) < upper;
        int r = open ? (int)over_group<G>(before, add_u32) : K;
        uint32_t from = 0;
        while (__any(r < K)) {
            const uint32_t n = over([&](int i, int j) {
                const uint32_t o = place_of(p[i].get(j)) - upper, k = o << 8 | expert(i, j);
                return o <= LOW && real(i, j) && k >= from ? k : NONE;
            }, umin);
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) e[i] = r < K && i * G + l == r ? (int)(n & LOW) : e[i];
            from = n + 1;
            ++r;
        }
    }
    // Where the picks that lie in the lanes, and the one behind them, stand among themselves by whole places: rank[i] of the lane's
    // own, the result that of the one behind.
    __device__ __forceinline__ int rank_of(int K, const int (&e)[SLOTS], const float (&v)[SLOTS], int behind, float vb, int (&rank)[SLOTS]) const
    {
        const int from = (threadIdx.x & 63) - l;
        uint32_t mine[SLOTS];
        int over_b = 0;
        const uint32_t pb = behind >= 0 ? place_of(vb) : NONE;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            mine[i] = place_of(v[i]);
            rank[i] = pb < mine[i] || (pb == mine[i] && behind < e[i]);
            rank[i] = behind >= 0 ? rank[i] : 0;
        }
#pragma unroll
        for (int q = 0; q < SLOTS; ++q) {
            const int rounds = min(K - q * G, G);
#pragma unroll 1
            for (int r = 0; r < rounds; ++r) {
                const uint32_t o = (uint32_t)__shfl((int)mine[q], from + r);
                const int x = __shfl(e[q], from + r);
#pragma unroll
                for (int i = 0; i < SLOTS; ++i) rank[i] += o < mine[i] || (o == mine[i] && x < e[i]);
                over_b += o < pb || (o == pb && x < behind);
            }
        }
        return behind >= 0 ? over_b : K;
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

// Threads of the largest block: 32 fp32 logits to a lane take the registers of two.
constexpr int balance_most(int NP, int element) { return NP > 2 && element == 4 ? 512 : 1024; }

// A block walks its slice of a group's tokens; part (groups, slices, E): {sum of probabilities, count}.  With one slice to a
// group the block has all of it and finishes the loss itself.
template <typename T, int NP, int G, bool FULL>
__global__ void __launch_bounds__(balance_most(NP, sizeof(T)))
balance_kernel(const T *__restrict__ logits, const uint8_t *__restrict__ mask, int32_t *__restrict__ topk_idx,
               float *__restrict__ topk_w, float2 *__restrict__ part, int64_t tokens, int slices, int E, int K,
               int32_t *__restrict__ counts, float *__restrict__ prob_mean, float *__restrict__ loss)
{
    typedef Token<T, NP, G, FULL> Tok;
    __shared__ float psum[balance_most(NP, sizeof(T)) / 64][Tok::SIZE];
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
    constexpr bool AHEAD = NP < 4;                             // with more experts to a lane, its registers serve another wave better
    Step next;
    if (AHEAD && t < tokens) fetch(next, t);
    for (; t < tokens; t += stride) {
        Step s;
        if constexpr (AHEAD) {
            s = next;
            if (t + stride < tokens) fetch(next, t + stride);
        } else
            fetch(s, t);
        const Tok tok(s.p, l, E);
        const int64_t row = grp * tokens + (t + at < tokens ? t + at : tokens - 1);
        int e[Tok::SLOTS], rank[Tok::SLOTS], behind = -1, rank_b = K;
        float v[Tok::SLOTS];
        bool close = tok.picks(K, e, v, behind);
        if constexpr (!Tok::BF) {                              // the keys do not hold the whole of the logits
            auto take = [&] {
#pragma unroll
                for (int i = 0; i < Tok::SLOTS; ++i)
                    if (i * G + l < K) v[i] = to_float(logits[row * E + e[i]]);
            };
            take();
            close = close && t + at < tokens;                  // (behind the last token all logits are zero)
            if (__any(close && behind == -2)) {
                tok.settle(K, e, v, close && behind == -2);
                take();
            }
            if (behind == -2) behind = -1;
        }
#pragma unroll
        for (int i = 0; i < Tok::SLOTS; ++i) rank[i] = i * G + l;
        if constexpr (!Tok::BF) {
            if (__any(close)) rank_b = tok.rank_of(K, e, v, behind, to_float(logits[row * E + (behind >= 0 ? behind : 0)]), rank);
        }
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
        // exp(f - m) as exp2(f c - m c) in one rounding, with m c as it is rounded: the weights and their sum have the same factor
        // then, which is 1.01 at most up to |m| = 10^5.  Beyond, the difference is taken first: by each token for itself, so that
        // nothing depends on the tokens beside it.
        float p[NP][8], Z = 0.f;
        const float mc = m * LOG2E;
        const bool far = !(fabsf(m) <= 1e5f);
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                p[i][j] = tok.real(i, j) ? fast_exp2(fmaf(s.p[i].get(j), LOG2E, -mc)) : 0.f;
        if (__any(far)) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) p[i][j] = !tok.real(i, j) ? 0.f : far ? route_exp(s.p[i].get(j) - m) : p[i][j];
        }
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) Z += p[i][j];
        const float invZ = 1.0f / group_sum<G>(Z);
        if (t + at < tokens) {
            auto put = [&](int r, int x, float f) __attribute__((always_inline)) {
                if (topk_idx) topk_idx[row * K + r] = x;
                if (topk_w) topk_w[row * K + r] = (far ? route_exp(f - m) : fast_exp2(fmaf(f, LOG2E, -mc))) * invZ;
                if (on) atomicAdd(&csum[x], 1);                // whole numbers: the order does not matter
            };
#pragma unroll
            for (int i = 0; i < Tok::SLOTS; ++i)
                if (i * G + l < K && rank[i] < K) put(rank[i], e[i], v[i]);
            if (!Tok::BF && l == 0 && rank_b < K) put(rank_b, behind, to_float(logits[row * E + behind]));
        }
        if (on) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[i][j] += p[i][j] * invZ;
        }
    }
    float sum[8 * NP];
    int first = 0;
#pragma unroll
    for (int i = 0; i < 8 * NP; ++i) sum[i] = acc[i / 8][i % 8];
    sum_over<32, G>(sum, first, lane);
    constexpr int LEFT = NP * G > 8 ? NP * G / 8 : 1;
#pragma unroll
    for (int i = 0; i < LEFT; ++i) psum[wave][8 * (l + G * ((first + i) / 8)) + (first + i) % 8] = sum[i];  // one from several lanes: the same
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

// The slices of a group joined by a block of 1024 threads: WIDTH threads side by side have PER experts each, the others every
// (1024 / WIDTH)-th slice, 16 of them under way.
template <int WIDTH, int PER>
__global__ void __launch_bounds__(1024)
balance_loss_kernel(const float2 *__restrict__ part, int slices, int E, int K, int32_t *__restrict__ counts,
                    float *__restrict__ prob_mean, float *__restrict__ loss)
{
    constexpr int ROWS = 1024 / WIDTH;
    __shared__ float2 lds[ROWS][WIDTH * PER];
    __shared__ double fin[2][4];
    const int64_t grp = blockIdx.x;
    const int row = threadIdx.x / WIDTH, e = threadIdx.x % WIDTH * PER, n = E - e;
    float p[PER] = {};
    int c[PER] = {};
    const float2 *const from = part + grp * slices * E + e;
    if (n > 0) {
#pragma unroll 16
        for (int s = row; s < slices; s += ROWS) {
            Piece<float, 2 * PER> v;                           // the last expert of an odd number stands alone
            v.template load<PER == 2>((const float *)(from + (int64_t)s * E), 2 * n);
#pragma unroll
            for (int i = 0; i < PER; ++i) { p[i] += v.get(2 * i); c[i] += (int)v.v[2 * i + 1]; }
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) lds[row][e + i] = make_float2(p[i], __int_as_float(c[i]));
    __syncthreads();
    float sum = 0.f;
    int count = 0;
    if (threadIdx.x < WIDTH * PER) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            sum += lds[i][threadIdx.x].x;
            count += __float_as_int(lds[i][threadIdx.x].y);
        }
    }
    balance_finish(sum, count, grp, E, K, counts, prob_mean, loss, fin);
}

namespace {

int lanes_of(int E)                                            // of a token, eight experts to a lane
{
    int n = 1;
    while (8 * n < E) n *= 2;
    return n;
}
// Eight lanes at most for the routing: steps over lanes cost as much as three experts of a lane, and with few tokens to a wave
// so does what is done once for all of them.
constexpr int pieces_for(int lanes) { return lanes <= 4 ? 1 : lanes <= 8 ? 2 : 4; }
int pieces_of(int E) { return pieces_for(lanes_of(E)); }
int routing_lanes_of(int E) { return lanes_of(E) / pieces_of(E); }

// Threads of a block and slices of a group.  A group that a block walks in one step, or in two with eight experts to a lane, stays
// with it, without a second launch (8.7 us with 64 tokens of 256 experts top-8 in a step; with 512 in four steps 26.3, in two
// launches 13).  So does each of more than 128 groups, of which two slices would be more than the compute units: 129 groups of 2048 x 16
// 11.3 us, 128 in two launches 13.5; of 2048 x 256, though, 100 and 57, until 255 groups fill the chip (103).
// In all other cases a slice is a step or more, and the slices of all groups are no more than the compute units: a block of
// 1024 threads fills one, and a 257th would run by itself (131072 x 256: 53.0 us with 257, 35.6 with 256).  Smaller blocks where
// they are enough for that.
struct Slices { int threads; int64_t count; };
int64_t routing_threads(int64_t tokens, int E) { return tokens * routing_lanes_of(E); }
bool one_block(int64_t groups, int64_t tokens, int E, int element)
{
    return groups > 128 || groups == 0 || routing_threads(tokens, E) <= balance_most(pieces_of(E), element) * (pieces_of(E) == 1 ? 2 : 1);
}
Slices balance_slices(int64_t groups, int64_t tokens, int E, int element)
{
    const int most = balance_most(pieces_of(E), element);
    const int64_t threads = routing_threads(tokens, E), slices = one_block(groups, tokens, E, element) ? 1 : 256 / groups;
    int n = 256;
    while (n < most && (threads + n - 1) / n > slices) n *= 2;
    const int64_t steps = (threads + n - 1) / n;
    return {n, slices == 1 || steps < 2 ? 1 : steps < slices ? steps : slices};
}

// f(lanes, how the last piece is read, whether the experts fill the lanes) as constants
template <typename F>
void with_lanes(int E, F &&f)
{
    using std::integral_constant;
    auto tail = [&](auto g) {
        if constexpr (g == 1) {
            if (E < 8) return f(g, integral_constant<Tail, BY_ELEMENT>(), std::false_type());
        }
        if (tail_of(E, 8) == MOVED) f(g, integral_constant<Tail, MOVED>(), std::false_type());
        else if (E < 8 * g) f(g, integral_constant<Tail, NO_TAIL>(), std::false_type());
        else f(g, integral_constant<Tail, NO_TAIL>(), std::true_type());
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
    // for either type, and for fewer tokens as well
    if (one_block(groups, tokens, E, 2) && one_block(groups, tokens, E, 4)) return 0;
    const int64_t n = groups * ((routing_threads(tokens, E) + 255) / 256);
    return (size_t)(n < 256 ? n : 256) * E * sizeof(float2);
}

swimba_status launch_router_balance(int64_t groups, int64_t tokens, int E, int K, int io_dtype, const void *logits,
                                    const uint8_t *mask, int32_t *topk_idx, float *topk_w, int32_t *counts, float *prob_mean,
                                    float *loss, void *work, hipStream_t st)
{
    if (groups == 0) return SWIMBA_OK;
    const Slices s = balance_slices(groups, tokens, E, io_dtype == SWIMBA_BF16 ? 2 : 4);
    float2 *const part = (float2 *)work;
    with_lanes(E, [&](auto lanes, auto, auto full) {
        constexpr int NP = pieces_for(lanes()), G = lanes() / NP;
        auto go = [&](auto kernel, auto *z) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(groups * s.count)), dim3(s.threads), 0, st, z, mask, topk_idx, topk_w, part, tokens,
                               (int)s.count, E, K, counts, prob_mean, loss);
        };
        if (io_dtype == SWIMBA_BF16) go(balance_kernel<bf16, NP, G, full()>, (const bf16 *)logits);
        else go(balance_kernel<float, NP, G, full()>, (const float *)logits);
    });
    SWIMBA_CHECK_LAUNCH();
    if (s.count > 1) {
        const auto kernel = E <= 64 ? balance_loss_kernel<64, 1> : balance_loss_kernel<128, 2>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(1024), 0, st, part, (int)s.count, E, K, counts, prob_mean, loss);
        SWIMBA_CHECK_LAUNCH();
    }
    return SWIMBA_OK;
}

// The gradients of a token's routing weights are laid at their experts through LDS: a wave's 64 / G tokens are 512 floats,
// element j of lane i at 8 i + j.
template <typename T, int G, Tail TAIL>
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
        int c[8];
        uint32_t low = 0, high = 0;                             // the sum of all counts, which may pass 2^32, in two halves
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            c[j] = 8 * l + j < E ? counts[grp * E + 8 * l + j] : 0;
            low += (uint32_t)c[j] & 0xffff;
            high += (uint32_t)c[j] >> 16;
        }
        const double all = 65536. * over_group<G>(high, add_u32) + over_group<G>(low, add_u32);
        const double scale = all > 0. ? (double)d_loss[grp] * E * K / (all * all) : 0.;
#pragma unroll
        for (int j = 0; j < 8; ++j) share[j] = (float)(scale * c[j]);
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
    // (the last piece moved: 131072 x 100 bf16 23.0 -> 20.6 us; the routing itself gains nothing by it)
    const Part<TAIL, 8> part(8 * l, E, false);
    auto fetch = [&](Step &s, int64_t t) __attribute__((always_inline)) {
        const bool in = t + at < tokens;
        const int64_t row = grp * tokens + t + at;
        if constexpr (TAIL == MOVED) s.p.template load<false>(z + t * E + (uint32_t)(at * E + part.at), in ? 8 : 0);
        else s.p.template load<TAIL == BY_ELEMENT>(z + t * E + (uint32_t)(at * E + 8 * l), in ? E - 8 * l : 0);
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
        Step s = next;
        if (t + stride < tokens) fetch(next, t + stride);
        part.settle(s.p);
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
        if (t + at < tokens) store_piece<TAIL != NO_TAIL>(out + t * E + (uint32_t)(at * E + 8 * l), p, E - 8 * l);
    }
}

// Most blocks: what the chip holds at once; every further block would read the counts for itself (131072 x 128 bf16: 21.4 us, with
// 4096 blocks 26.3, with 8192 37).
constexpr int64_t BWD_BLOCKS = 1536;

swimba_status launch_router_bwd(int64_t groups, int64_t tokens, int E, int K, int io_dtype, const void *logits, const uint8_t *mask,
                                const int32_t *topk_idx, const float *d_topk_w, const int32_t *counts, const float *d_loss,
                                void *d_logits, hipStream_t st)
{
    if (groups == 0 || tokens == 0) return SWIMBA_OK;
    const int64_t need = (tokens * lanes_of(E) + 255) / 256, fit = groups < BWD_BLOCKS ? BWD_BLOCKS / groups : 1, per_group = need < fit ? need : fit;
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
