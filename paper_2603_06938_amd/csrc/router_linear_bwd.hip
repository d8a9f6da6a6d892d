// Backward pass of the router's linear map:  du = dl W + du_add,  dW = dl^T u   (dl: gradient of the logits).
// Bound by memory up to 64 experts in bf16, some 32 in fp32: u is read once (for every 64 experts; again from the cache, where its
// blocks follow each other on one XCD), du written once.  Neither product
// goes through LDS: a wave owns 128 columns, eight consecutive ones to a lane, and column n of tile i is feature 8 n + i, so
// that operands come as whole pieces of rows and a lane's results are consecutive features as well.  A bf16 matrix
// instruction wants eight rows of one column in a lane: 8 x 8 elements are transposed in registers.
//   dW  k runs over the tokens: the wave keeps its sums (16 experts a tile) while it walks its tokens; the sums of a block's
//       waves are joined in LDS, those of the blocks by a second launch
//   du  k runs over the experts: W is kept in registers, 16 tokens at a time
// 16384 x 768 x 8 bf16 with both products (51 MB) 14.5 us, 4.1 of them the second launch; 32768 x 2048 x 64 with du_add (407 MB)
// 95.8 us, 4.25 TB/s; 16384 x 2048 x 256 82.7 us, 415 TFLOP/s: neither memory nor matrix units (busy 18 %) bound it there, two waves
// to a SIMD wait for loads, without registers for du's next step; 16384 x 2048 x 128 fp32 175 us, 98 of 154 TFLOP/s.
#include "rows.hpp"

namespace swimba {

typedef __attribute__((ext_vector_type(4))) float f32x4_t;
__device__ __forceinline__ f32x4_t mfma16(const uint32_t (&a)[4], const uint32_t (&b)[4], f32x4_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
// element i (of each row's piece) of rows 2q and 2q + 1
__device__ __forceinline__ uint32_t pair_of(uint32_t even, uint32_t odd, int i)
{
    return __builtin_amdgcn_perm(odd, even, i % 2 ? 0x07060302u : 0x05040100u);
}

__device__ __forceinline__ f32x4_t mfma4(uint32_t a, uint32_t b, f32x4_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a), __uint_as_float(b), c, 0, 0, 0);
}

template <typename T> constexpr int dw_step() { return sizeof(T) == 2 ? 32 : 16; }
constexpr int LB_COLS = 128;           // features of a wave
constexpr int LB_WAVES = 4;
typedef f32x4_t Join[4][2][64];       // a tile of a wave: rows 4 kg + v, halves of a lane's eight columns

// Where the last pieces of a row would pass its end (columns of u and du, experts of dl), they are moved to end with it: the
// lane then has some elements that its neighbour has as well, and stores, or takes into a sum, only those from `own` on.
struct Cols {
    int at, own;                       // first element of the lane's piece, and of those that are its own
    __device__ __forceinline__ Cols(int first, int size, int W) : at(size >= W ? min(first, size - W) : first), own(first) {}
};

// dW: ME tiles of 16 experts, row m of tile j is expert e0 + ME m + j, so that a lane's experts are consecutive.
// A step is 32 tokens, 8 kg .. 8 kg + 7 in a lane, in bf16 (one instruction), and 16, kg + 4 j, in fp32 (four).
template <typename T, int ME>
__device__ __forceinline__ void dw_block(const T *__restrict__ u, const T *__restrict__ dl, float *__restrict__ part,
                                         Join *lds, int64_t tokens, int D, int E, int col, int eb, int64_t split,
                                         int64_t share)
{
    constexpr bool BF = sizeof(T) == 2;
    constexpr int STEP = dw_step<T>(), R = STEP / 4, EVERY = BF ? 1 : 4;        // rows of a lane, and the distance between them
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, kg = lane >> 4;
    const int own = BF ? 8 * kg : kg;                                           // the lane's first row of a step
    const int64_t t0 = split * share, t1 = min(t0 + share, tokens);
    const Cols c(col * LB_COLS + 8 * n, D, 8), x(eb * 16 * ME + ME * n, E, ME);
    f32x4_t acc[ME][8] = {};
    struct Step {
        Piece<T, 8> u[R];
        uint32_t g[R][BF ? (ME + 1) / 2 : ME];
    };
    const uint32_t uo = own * D + c.at, go = own * E + x.at;
    auto experts = [&](uint32_t *g, const T *p) __attribute__((always_inline)) {
        constexpr int BYTES = ME * sizeof(T);
        if constexpr (BYTES == 2) g[0] = *reinterpret_cast<const uint16_t *>(p);
        else if constexpr (BYTES == 4) g[0] = *reinterpret_cast<const any_u32_t *>(p);
        else if constexpr (BYTES == 8) {
            const any_u32x2_t v = *reinterpret_cast<const any_u32x2_t *>(p);
            g[0] = v.x; g[1] = v.y;
        } else {
            const any_u32x4_t v = *reinterpret_cast<const any_u32x4_t *>(p);
            g[0] = v.x; g[1] = v.y; g[2] = v.z; g[3] = v.w;
        }
    };
    auto fetch = [&](Step &s, int64_t t) __attribute__((always_inline)) {
        const T *ur = u + t * D, *gr = dl + t * E;
        if (t + STEP <= t1 && D >= 8) {
#pragma unroll
            for (int j = 0; j < R; ++j, ur += EVERY * D, gr += EVERY * E) {
                s.u[j].template load<false>(ur + uo, 8);
                experts(s.g[j], gr + go);
            }
            return;
        }
        // tokens that are not the block's add nothing, whatever memory holds there
#pragma unroll
        for (int j = 0; j < R; ++j, ur += EVERY * D, gr += EVERY * E) {
            const bool in = t + own + EVERY * j < t1;
            s.u[j].template load<true>(ur + uo, in ? (D >= 8 ? 8 : D - c.at) : 0);
#pragma unroll
            for (uint32_t &g : s.g[j]) g = 0;
            if (in) experts(s.g[j], gr + go);
        }
    };
    Step next;
    int64_t t = t0 + STEP * wave;
    if (t < t1) fetch(next, t);
    for (; t < t1; t += STEP * LB_WAVES) {
        const Step s = next;
        if (t + STEP * LB_WAVES < t1) fetch(next, t + STEP * LB_WAVES);
        if constexpr (BF) {
            uint32_t a[ME][4];
#pragma unroll
            for (int j = 0; j < ME; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) a[j][q] = pair_of(s.g[2 * q][j / 2], s.g[2 * q + 1][j / 2], j);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t b[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) b[q] = pair_of(s.u[2 * q].v[i / 2], s.u[2 * q + 1].v[i / 2], i);
#pragma unroll
                for (int j = 0; j < ME; ++j) acc[j][i] = mfma16(a[j], b, acc[j][i]);
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int j = 0; j < ME; ++j) acc[j][i] = mfma4(s.g[r][j], s.u[r].v[i], acc[j][i]);
        }
    }
    // A tile's rows 4 kg + v of the four waves are joined by wave v, in the order of the waves.
    const int m = 4 * kg + wave;
    const Cols ce(eb * 16 * ME + ME * m, E, ME);
#pragma unroll
    for (int j = 0; j < ME; ++j) {
        if (j) __syncthreads();
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                lds[wave][v][h][lane] = f32x4_t{acc[j][4 * h][v], acc[j][4 * h + 1][v], acc[j][4 * h + 2][v], acc[j][4 * h + 3][v]};
        __syncthreads();
        f32x4_t sum[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            sum[h] = lds[0][wave][h][lane];
#pragma unroll
            for (int w = 1; w < LB_WAVES; ++w) sum[h] += lds[w][wave][h][lane];
        }
        const int e = ce.at + j;
        if (e < ce.own || e >= E) continue;
        float *const to = part + (split * E + e) * D + c.at;
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = sum[i / 4][i % 4];
        if (c.at == c.own) store_piece<true>(to, f, D - c.at);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= c.own - c.at) to[i] = f[i];
        }
    }
}

// du: KS steps of 32 (bf16) or 16 (fp32) experts, NT tiles of 16 columns (16 NT columns to a wave, NT consecutive ones to a
// lane).  In a step a lane has the experts 8 kg .. 8 kg + 7, one instruction, or 4 kg .. 4 kg + 3, one instruction for each.
template <typename T, int KS, int NT>
__device__ __forceinline__ void du_block(const T *__restrict__ Wg, const T *__restrict__ dl, const T *du_add, T *du,
                                         int64_t tokens, int D, int E, int col, int64_t split, int64_t share)
{
    constexpr bool BF = sizeof(T) == 2, AHEAD = KS * (BF ? 2 : 1) <= 4;         // the operand of many experts leaves no registers
    constexpr int R = BF ? 8 : 4;                                               // experts of a lane in a step
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, kg = lane >> 4;
    const int64_t t0 = split * share, t1 = min(t0 + share, tokens);
    const Cols c(col * 16 * NT + NT * n, D, NT);
    const int width = D >= NT ? (c.own < D ? NT : 0) : D - c.at;       // elements of the lane's piece that exist and count
    struct Step {
        Piece<T, R> a[KS];
        Piece<T, NT> add[4];
    };
    auto fetch = [&](Step &s, int64_t t) __attribute__((always_inline)) {
        const T *g = dl + t * E, *add = du_add + t * D;
        const int left = (int)min((int64_t)16, t1 - t);
        const uint32_t row = min(n, left - 1) * E;
        int first = R * kg;
        asm volatile("" : "+v"(first));                        // the places of all steps, kept, would take the registers
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const Cols x(4 * R * k + first, E, R);
            if (E < R) s.a[k].template load<true>(g + row + x.at, E - x.at);
            else s.a[k].template load<false>(g + row + x.at, R);
        }
        if (du_add) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
                s.add[v].template load<true>(add + (uint32_t)((4 * kg + v) * D + c.at), 4 * kg + v < left ? width : 0);
        }
    };
    Step next;
    int64_t t = t0 + 16 * wave;
    if (AHEAD && t < t1) fetch(next, t);
    uint32_t w[KS][NT][4];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        Piece<T, NT> p[R];
        const Cols x(R * (4 * k + kg), E, R);
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const T *const row = Wg + (uint32_t)((x.at + j) * D + c.at);
            if (E >= R && D >= NT) p[j].template load<false>(row, NT);
            else p[j].template load<true>(row, x.at + j < E ? width : 0);
        }
        if (4 * R * (k + 1) > E) {
#pragma unroll
            for (int j = 0; j < R; ++j)
#pragma unroll
                for (uint32_t &q : p[j].v) q = x.at + j < x.own ? 0 : q;
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if constexpr (BF) w[k][i][q] = pair_of(p[2 * q].v[i / 2], p[2 * q + 1].v[i / 2], i);
                else w[k][i][q] = p[q].v[i];
            }
    }
    for (; t < t1; t += 16 * LB_WAVES) {
        Step s;
        if constexpr (AHEAD) {
            s = next;
            if (t + 16 * LB_WAVES < t1) fetch(next, t + 16 * LB_WAVES);
        } else
            fetch(s, t);
        f32x4_t acc[NT] = {};
        int first = R * kg;
        asm volatile("" : "+v"(first));
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const Cols x(4 * R * k + first, E, R);
            if (4 * R * (k + 1) > E) s.a[k].drop(x.own - x.at);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                if constexpr (BF) acc[i] = mfma16(s.a[k].v, w[k][i], acc[i]);
                else {
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[i] = mfma4(s.a[k].v[q], w[k][i][q], acc[i]);
                }
            }
        }
        T *const out = du + t * D;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            float o[NT];
#pragma unroll
            for (int i = 0; i < NT; ++i) o[i] = acc[i][v] + (du_add ? s.add[v].get(i) : 0.f);
            if (t + 4 * kg + v >= t1) continue;
            T *const p = out + (uint32_t)((4 * kg + v) * D + c.at);
            if (c.at == c.own) store_piece<true>(p, o, width);
            else {
#pragma unroll
                for (int i = 0; i < NT; ++i)
                    if (i >= c.own - c.at) p[i] = from_float<T>(o[i]);
            }
        }
    }
}

// Tokens of a block's share, and how many shares there are.
struct Shares { int64_t share, count; };

// One launch does both: the first wblocks blocks sum dW, the others write du, so that the two streams of memory overlap.
template <typename T, int ME, int KS, int NT>
__global__ void __launch_bounds__(64 * LB_WAVES) __attribute__((amdgpu_waves_per_eu(ME == 4 || sizeof(T) == 4 ? 2 : 3)))
linear_bwd_kernel(const T *__restrict__ u, const T *__restrict__ Wg, const T *__restrict__ dl, const T *du_add, T *du,
                  float *__restrict__ part, int64_t tokens, int D, int E, unsigned wblocks, Shares ws, Shares us)
{
    __shared__ Join lds[LB_WAVES];
    if (blockIdx.x < wblocks) {
        // the blocks of one share and its columns, which read the same u, follow each other on one XCD
        const int cols = (D + LB_COLS - 1) / LB_COLS, eblocks = (E + 16 * ME - 1) / (16 * ME);
        const int64_t id = xcd_logical_id(blockIdx.x, wblocks), col = id / eblocks % cols, split = id / eblocks / cols;
        if (split < ws.count) dw_block<T, ME>(u, dl, part, lds, tokens, D, E, (int)col, (int)(id % eblocks), split, ws.share);
    } else {
        const int cols = (D + 16 * NT - 1) / (16 * NT);
        const int64_t id = blockIdx.x - wblocks;
        du_block<T, KS, NT>(Wg, dl, du_add, du, tokens, D, E, (int)(id % cols), id / cols, us.share);
    }
}

__global__ void __launch_bounds__(512)
linear_reduce_kernel(const float *__restrict__ part, int rows, int64_t n, float *__restrict__ dW)
{
    sum_rows(part, rows, n, [&](int64_t c, float s) { dW[c] = s; });
}

namespace {

// Shares of whole steps (`step` tokens), as many as bring the blocks, `per_share` of them to a share, to `want`: that many at
// most, a number that does not fall as the tokens grow, and what is left of them where a share is the same number of steps for all.
int64_t most_shares(int64_t tokens, int64_t per_share, int64_t step, int64_t want)
{
    const int64_t most = per_share < want ? want / per_share : 1, steps = (tokens + step - 1) / step;
    return steps < most ? steps : most;
}
Shares shares_of(int64_t tokens, int64_t per_share, int64_t step, int64_t want)
{
    if (tokens == 0) return {step, 0};
    const int64_t steps = (tokens + step - 1) / step, count = most_shares(tokens, per_share, step, want);
    const int64_t share = (steps + count - 1) / count * step;
    return {share, (tokens + share - 1) / share};
}
int experts_of(int E) { return E <= 16 ? 16 : E <= 32 ? 32 : 64; }                 // of a block of dW
// Blocks that sum dW, half of those that the chip holds at once at the kernels' registers: of two to a compute unit in fp32 and
// for the sums of 64 experts, of three below (16384 x 1024 x 16 bf16: 17.3 us with 384 blocks, 18.6 with 512; 16384 x 768 x 8
// fp32: 22.2 with 256, 24.3 with 384).  With 17 to 32 experts a few more are faster (16384 x 2048 x 32: 29.5 us with 512, 33.8
// with 384), because shares come in whole steps.  du has three times as many, which start as others end, so that both streams of
// memory run to the end (16384 x 2048 x 16: 30.1 us, 34.6 with as many as dW has; x 64 35.1 and 41.5).
int64_t blocks_of(int E, int element) { return element == 4 || E > 32 ? 256 : E > 16 ? 512 : 384; }
int64_t dw_per_share(int D, int E) { return (int64_t)((D + LB_COLS - 1) / LB_COLS) * ((E + experts_of(E) - 1) / experts_of(E)); }
constexpr int DW_STEP = dw_step<bf16>() * LB_WAVES;                                 // of a block in bf16; in fp32 half of it
Shares dw_shares(int64_t tokens, int D, int E, int element)
{
    return shares_of(tokens, dw_per_share(D, E), DW_STEP, blocks_of(E, element));
}

template <typename T>
swimba_status linear_bwd(int64_t tokens, int D, int E, const void *u, const void *Wg, const void *dl, const void *du_add, void *du,
                         bool dW, float *part, hipStream_t st)
{
    const Shares sh = dw_shares(tokens, D, E, sizeof(T));
    auto go = [&](auto me, auto ks, auto nt) {
        const int64_t cols = (D + 16 * nt - 1) / (16 * nt);
        const Shares us = shares_of(tokens, cols, 16 * LB_WAVES, 3 * blocks_of(E, sizeof(T)));
        const unsigned wb = dW ? (unsigned)xcd_padded(dw_per_share(D, E) * sh.count) : 0;
        const unsigned ub = du ? (unsigned)(cols * us.count) : 0;
        if (wb + ub == 0) return;
        hipLaunchKernelGGL((linear_bwd_kernel<T, me(), ks(), nt()>), dim3(wb + ub), dim3(64 * LB_WAVES), 0, st, (const T *)u,
                           (const T *)Wg, (const T *)dl, (const T *)du_add, (T *)du, part, tokens, D, E, wb, sh, us);
    };
    constexpr std::integral_constant<int, 1> one;
    constexpr std::integral_constant<int, 2> two;
    constexpr std::integral_constant<int, 4> four;
    constexpr std::integral_constant<int, 8> eight;
    constexpr std::integral_constant<int, 16> sixteen;
    // W's operand is at most 128 registers: with more than 128 (bf16) or 32 (fp32) experts, of fewer columns
    if constexpr (sizeof(T) == 2) {
        if (E <= 16) go(one, one, eight);
        else if (E <= 32) go(two, one, eight);
        else if (E <= 64) go(four, two, eight);
        else if (E <= 128) go(four, four, eight);
        else go(four, eight, four);
    } else {
        if (E <= 16) go(one, one, eight);
        else if (E <= 32) go(two, two, eight);
        else if (E <= 64) go(four, four, four);
        else if (E <= 128) go(four, eight, four);
        else go(four, sixteen, two);
    }
    SWIMBA_CHECK_LAUNCH();
    return SWIMBA_OK;
}

}  // namespace

// For bf16, which has as many shares as fp32 or more, and for fewer tokens as well, which may have more of smaller shares.
size_t router_linear_bwd_bytes(int64_t tokens, int D, int E)
{
    const int64_t n = most_shares(tokens, dw_per_share(D, E), DW_STEP, blocks_of(E, 2));
    return n > 1 ? (size_t)n * E * D * sizeof(float) : 0;
}

swimba_status launch_router_linear_bwd(int64_t tokens, int D, int E, int io_dtype, const void *u, const void *Wg, const void *dl,
                                       const void *du_add, void *du, float *dW, void *work, hipStream_t st)
{
    const int64_t shares = dw_shares(tokens, D, E, io_dtype == SWIMBA_BF16 ? 2 : 4).count;
    // the sums of one share are dW itself
    float *const part = shares == 1 ? dW : (float *)work;
    if (tokens > 0) {
        const auto go = io_dtype == SWIMBA_BF16 ? linear_bwd<bf16> : linear_bwd<float>;
        const swimba_status s = go(tokens, D, E, u, Wg, dl, du_add, du, dW != nullptr, part, st);
        if (s != SWIMBA_OK) return s;
    }
    if (dW && shares != 1) {
        const int64_t n = (int64_t)E * D;
        hipLaunchKernelGGL(linear_reduce_kernel, dim3((unsigned)((n + 31) / 32)), dim3(512), 0, st, part, (int)shares, n, dW);
        SWIMBA_CHECK_LAUNCH();
    }
    return SWIMBA_OK;
}

}  // namespace swimba
