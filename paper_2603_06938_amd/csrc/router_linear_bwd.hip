// Backward pass of the router's linear map:  du = dl W + du_add,  dW = dl^T u   (dl: gradient of the logits).
// Bound by memory up to some hundred experts: u is read once, du written once.  Neither product goes through LDS: a wave owns
// 128 columns, eight consecutive ones to a lane (16-byte pieces of the rows), and takes the operand of a 16 x 16 matrix
// instruction out of eight rows by transposing 8 x 8 elements in registers; column n of tile i is then feature 8 n + i, so
// that a lane's results are consecutive features as well.
//   dW  k runs over the tokens: the wave keeps its sums (16 experts a tile) while it walks its tokens, 32 at a time; the sums
//       of a block's waves are joined in LDS, those of the blocks by a second launch
//   du  k runs over the experts: W is kept in registers, 16 tokens at a time
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

constexpr int LB_COLS = 128;           // features of a wave
constexpr int LB_WAVES = 4;

// Where the last pieces of a row would pass its end (columns of u and du, experts of dl), they are moved to end with it: the
// lane then works on some columns that its neighbour has as well, and stores only what is past `own`.
struct Cols {
    int at, own;                       // first element of the lane's piece, and of those that are its own
    __device__ __forceinline__ Cols(int first, int size, int W) : at(size >= W ? min(first, size - W) : first), own(first) {}
};

// dW: ME tiles of 16 experts, row m of tile j is expert e0 + ME m + j, so that a lane's experts are consecutive.
template <int ME>
__device__ __forceinline__ void dw_block(const bf16 *__restrict__ u, const bf16 *__restrict__ dl, float *__restrict__ part,
                                         float (*lds)[LB_COLS + 4], int64_t tokens, int D, int E, int col, int eb, int64_t split,
                                         int64_t share)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, kg = lane >> 4;
    const int64_t t0 = split * share, t1 = min(t0 + share, tokens);
    const Cols c(col * LB_COLS + 8 * n, D, 8), x(eb * 16 * ME + ME * n, E, ME);
    f32x4_t acc[ME][8] = {};
    struct Step {
        Piece<bf16, 8> u[8];
        uint32_t g[8][(ME + 1) / 2];
    };
    const uint32_t uo = 8 * kg * D + c.at, go = 8 * kg * E + x.at;
    auto experts = [&](uint32_t *g, const bf16 *p) __attribute__((always_inline)) {
        if constexpr (ME == 1) g[0] = p->bits;
        else if constexpr (ME == 2) g[0] = *reinterpret_cast<const any_u32_t *>(p);
        else {
            const any_u32x2_t v = *reinterpret_cast<const any_u32x2_t *>(p);
            g[0] = v.x; g[1] = v.y;
        }
    };
    auto fetch = [&](Step &s, int64_t t) __attribute__((always_inline)) {
        const bf16 *ur = u + t * D, *gr = dl + t * E;
        if (t + 32 <= t1 && D >= 8) {
#pragma unroll
            for (int j = 0; j < 8; ++j, ur += D, gr += E) {
                s.u[j].template load<false>(ur + uo, 8);
                experts(s.g[j], gr + go);
            }
            return;
        }
        // tokens that are not the block's add nothing, whatever memory holds there
#pragma unroll
        for (int j = 0; j < 8; ++j, ur += D, gr += E) {
            const bool in = t + 8 * kg + j < t1;
            s.u[j].template load<true>(ur + uo, in ? (D >= 8 ? 8 : D - c.at) : 0);
#pragma unroll
            for (int i = 0; i < (ME + 1) / 2; ++i) s.g[j][i] = 0;
            if (in) experts(s.g[j], gr + go);
        }
    };
    Step next;
    int64_t t = t0 + 32 * wave;
    if (t < t1) fetch(next, t);
    for (; t < t1; t += 32 * LB_WAVES) {
        const Step s = next;
        if (t + 32 * LB_WAVES < t1) fetch(next, t + 32 * LB_WAVES);
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
    }
    // lds[e][column], counted from the block's first
    for (int w = 0; w < LB_WAVES; ++w) {
        if (wave == w) {
#pragma unroll
            for (int j = 0; j < ME; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    float *row = &lds[ME * (4 * kg + v) + j][8 * n];
#pragma unroll
                    for (int i = 0; i < 8; ++i) row[i] = w ? row[i] + acc[j][i][v] : acc[j][i][v];
                }
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < 16 * ME * LB_COLS; i += 64 * LB_WAVES) {
        const int r = i / LB_COLS, q = i % LB_COLS;
        // row r and column q of the tiles are expert and feature
        const Cols ce(eb * 16 * ME + r / ME * ME, E, ME), cd(col * LB_COLS + q / 8 * 8, D, 8);
        const int e = ce.at + r % ME, d = cd.at + q % 8;
        if (e >= ce.own && e < E && d >= cd.own && d < D) part[(split * E + e) * D + d] = lds[r][q];
    }
}

// du: KS steps of 32 experts, NT tiles of 16 columns (16 NT columns to a wave, NT consecutive ones to a lane)
template <int KS, int NT>
__device__ __forceinline__ void du_block(const bf16 *__restrict__ Wg, const bf16 *__restrict__ dl, const bf16 *du_add, bf16 *du,
                                         int64_t tokens, int D, int E, int col, int64_t split, int64_t share)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, kg = lane >> 4;
    const int64_t t0 = split * share, t1 = min(t0 + share, tokens);
    const Cols c(col * 16 * NT + NT * n, D, NT);
    const int width = D >= NT ? (c.own < D ? NT : 0) : D - c.at;       // elements of the lane's piece that exist
    struct Step {
        Piece<bf16, 8> a[KS];
        Piece<bf16, NT> add[4];
    };
    auto fetch = [&](Step &s, int64_t t) __attribute__((always_inline)) {
        const bf16 *g = dl + t * E, *add = du_add + t * D;
        const int left = (int)min((int64_t)16, t1 - t);
        const uint32_t row = min(n, left - 1) * E;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int e = 32 * k + 8 * kg;
            s.a[k].template load<true>(g + row + e, E - e);
        }
        if (du_add) {
#pragma unroll
            for (int v = 0; v < 4; ++v)
                s.add[v].template load<true>(add + (uint32_t)((4 * kg + v) * D + c.at), 4 * kg + v < left ? width : 0);
        }
    };
    Step next;
    int64_t t = t0 + 16 * wave;
    if (t < t1) fetch(next, t);
    uint32_t w[KS][NT][4];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        Piece<bf16, NT> p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = 32 * k + 8 * kg + j;
            p[j].template load<true>(Wg + (uint32_t)(e * D + c.at), e < E ? width : 0);
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) w[k][i][q] = pair_of(p[2 * q].v[i / 2], p[2 * q + 1].v[i / 2], i);
    }
    for (; t < t1; t += 16 * LB_WAVES) {
        const Step s = next;
        if (t + 16 * LB_WAVES < t1) fetch(next, t + 16 * LB_WAVES);
        f32x4_t acc[NT] = {};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < NT; ++i) acc[i] = mfma16(s.a[k].v, w[k][i], acc[i]);
        bf16 *const out = du + t * D;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            float o[NT];
#pragma unroll
            for (int i = 0; i < NT; ++i) o[i] = acc[i][v] + (du_add ? s.add[v].get(i) : 0.f);
            if (t + 4 * kg + v >= t1) continue;
            bf16 *const p = out + (uint32_t)((4 * kg + v) * D + c.at);
            if (c.at == c.own) store_piece<true>(p, o, width);
            else {
#pragma unroll
                for (int i = 0; i < NT; ++i)
                    if (i >= c.own - c.at) p[i] = from_float<bf16>(o[i]);
            }
        }
    }
}

// Tokens of a block's share, and how many shares there are.
struct Shares { int64_t share, count; };

// One launch does both: the first wblocks blocks sum dW, the others write du, so that the two streams of memory overlap.
template <int ME, int KS, int NT>
__global__ void __launch_bounds__(64 * LB_WAVES) __attribute__((amdgpu_waves_per_eu(KS == 8 ? 1 : ME == 4 ? 2 : 3)))
linear_bwd_bf16_kernel(const bf16 *__restrict__ u, const bf16 *__restrict__ Wg, const bf16 *__restrict__ dl, const bf16 *du_add,
                       bf16 *du, float *__restrict__ part, int64_t tokens, int D, int E, unsigned wblocks, Shares ws, Shares us)
{
    __shared__ float lds[16 * ME][LB_COLS + 4];
    if (blockIdx.x < wblocks) {
        // the blocks of one share and its columns, which read the same u, follow each other on one XCD
        const int cols = (D + LB_COLS - 1) / LB_COLS, eblocks = (E + 16 * ME - 1) / (16 * ME);
        const int64_t id = xcd_logical_id(blockIdx.x, wblocks), col = id / eblocks % cols, split = id / eblocks / cols;
        if (split < ws.count) dw_block<ME>(u, dl, part, lds, tokens, D, E, (int)col, (int)(id % eblocks), split, ws.share);
    } else {
        const int cols = (D + 16 * NT - 1) / (16 * NT);
        const int64_t id = blockIdx.x - wblocks;
        du_block<KS, NT>(Wg, dl, du_add, du, tokens, D, E, (int)(id % cols), id / cols, us.share);
    }
}

__global__ void __launch_bounds__(512)
linear_reduce_kernel(const float *__restrict__ part, int rows, int64_t n, float *__restrict__ dW)
{
    sum_rows(part, rows, n, [&](int64_t c, float s) { dW[c] = s; });
}

// fp32: one element by one, for now
__global__ void __launch_bounds__(256)
linear_du_f32_kernel(const float *__restrict__ Wg, const float *__restrict__ dl, const float *du_add, float *du, int64_t tokens, int D, int E)
{
    const int64_t n = tokens * D;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / D, d = i % D;
        float s = 0.f;
        for (int e = 0; e < E; ++e) s += dl[t * E + e] * Wg[e * (int64_t)D + d];
        if (du_add) s += du_add[i];
        du[i] = s;
    }
}
__global__ void __launch_bounds__(256)
linear_dw_f32_kernel(const float *__restrict__ u, const float *__restrict__ dl, float *__restrict__ part, int64_t tokens, int D, int E,
                     int64_t share)
{
    const int d = blockIdx.x * 256 + threadIdx.x, e = blockIdx.y;
    if (d >= D) return;
    const int64_t t0 = blockIdx.z * share, t1 = min(t0 + share, tokens);
    float s = 0.f;
    for (int64_t t = t0; t < t1; ++t) s += dl[t * E + e] * u[t * D + d];
    part[((int64_t)blockIdx.z * E + e) * D + d] = s;
}

namespace {

// Shares of whole steps (`step` tokens), as many as bring the blocks, `per_share` of them to a share, to `want`.
Shares shares_of(int64_t tokens, int64_t per_share, int64_t step, int64_t want)
{
    const int64_t most = per_share < want ? want / per_share : 1, steps = (tokens + step - 1) / step;
    const int64_t count = steps < most ? (steps > 0 ? steps : 1) : most, share = (steps + count - 1) / count * step;
    return {share, tokens > 0 ? (tokens + share - 1) / share : 0};
}
int experts_of(int E) { return E <= 16 ? 16 : E <= 32 ? 32 : 64; }                 // of a block of dW
// Blocks that the chip holds at once at the kernels' registers, half of them for each product.
int64_t blocks_of(int E) { return E <= 32 ? 512 : 256; }
int64_t dw_per_share(int D, int E) { return (int64_t)((D + LB_COLS - 1) / LB_COLS) * ((E + experts_of(E) - 1) / experts_of(E)); }
Shares dw_shares(int64_t tokens, int D, int E) { return shares_of(tokens, dw_per_share(D, E), 32 * LB_WAVES, blocks_of(E)); }

}  // namespace

size_t router_linear_bwd_bytes(int64_t tokens, int D, int E) { return (size_t)dw_shares(tokens, D, E).count * E * D * sizeof(float); }

swimba_status launch_router_linear_bwd(int64_t tokens, int D, int E, int io_dtype, const void *u, const void *Wg, const void *dl,
                                       const void *du_add, void *du, float *dW, void *work, hipStream_t st)
{
    const Shares sh = dw_shares(tokens, D, E);
    float *part = (float *)work;
    if (tokens > 0 && io_dtype == SWIMBA_BF16) {
        auto go = [&](auto kernel, int wide) {
            const int64_t cols = (D + wide - 1) / wide;
            const Shares us = shares_of(tokens, cols, 16 * LB_WAVES, blocks_of(E));
            const unsigned wb = dW ? (unsigned)xcd_padded(dw_per_share(D, E) * sh.count) : 0;
            const unsigned ub = du ? (unsigned)(cols * us.count) : 0;
            if (wb + ub == 0) return;
            hipLaunchKernelGGL(kernel, dim3(wb + ub), dim3(64 * LB_WAVES), 0, st, (const bf16 *)u, (const bf16 *)Wg, (const bf16 *)dl,
                               (const bf16 *)du_add, (bf16 *)du, part, tokens, D, E, wb, sh, us);
        };
        if (E <= 16) go(linear_bwd_bf16_kernel<1, 1, 8>, 128);
        else if (E <= 32) go(linear_bwd_bf16_kernel<2, 1, 8>, 128);
        else if (E <= 64) go(linear_bwd_bf16_kernel<4, 2, 8>, 128);
        else if (E <= 128) go(linear_bwd_bf16_kernel<4, 4, 8>, 128);
        else go(linear_bwd_bf16_kernel<4, 8, 4>, 64);
        SWIMBA_CHECK_LAUNCH();
    } else if (tokens > 0) {
        if (du)
            hipLaunchKernelGGL(linear_du_f32_kernel, dim3((unsigned)((tokens * D + 255) / 256 < 65536 ? (tokens * D + 255) / 256 : 65536)),
                               dim3(256), 0, st, (const float *)Wg, (const float *)dl, (const float *)du_add, (float *)du, tokens, D, E);
        SWIMBA_CHECK_LAUNCH();
        if (dW)
            hipLaunchKernelGGL(linear_dw_f32_kernel, dim3((unsigned)((D + 255) / 256), (unsigned)E, (unsigned)sh.count), dim3(256), 0, st,
                               (const float *)u, (const float *)dl, part, tokens, D, E, sh.share);
        SWIMBA_CHECK_LAUNCH();
    }
    if (dW) {
        const int64_t n = (int64_t)E * D;
        hipLaunchKernelGGL(linear_reduce_kernel, dim3((unsigned)((n + 31) / 32)), dim3(512), 0, st, part, (int)sh.count, n, dW);
        SWIMBA_CHECK_LAUNCH();
    }
    return SWIMBA_OK;
}

}  // namespace swimba
