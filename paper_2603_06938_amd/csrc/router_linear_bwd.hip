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

// ME tiles of 16 experts: row m of tile j is expert e0 + ME m + j, so that a lane's experts are consecutive.
template <int ME>
__global__ void __launch_bounds__(64 * LB_WAVES)
linear_dw_bf16_kernel(const bf16 *__restrict__ u, const bf16 *__restrict__ dl, float *__restrict__ part, int64_t tokens, int D, int E,
                      int cols, int eblocks, int64_t share)
{
    __shared__ float lds[16 * ME][LB_COLS + 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, kg = lane >> 4;
    const int col = blockIdx.x % cols, eb = blockIdx.x / cols % eblocks;
    const int64_t split = blockIdx.x / cols / eblocks, t0 = split * share, t1 = min(t0 + share, tokens);
    const int d = col * LB_COLS + 8 * n, e = eb * 16 * ME + ME * n;
    f32x4_t acc[ME][8] = {};
    struct Step {
        Piece<bf16, 8> u[8];
        uint32_t g[8][(ME + 1) / 2];
    };
    auto fetch = [&](Step &s, int64_t t) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t tt = t + 8 * kg + j;
            const bool in = tt < t1;
            s.u[j].template load<true>(u + tt * D + d, in ? D - d : 0);
            const bf16 *g = dl + tt * E + e;
            if (in && e + ME <= E) {
                if constexpr (ME == 1) s.g[j][0] = g[0].bits;
                else if constexpr (ME == 2) s.g[j][0] = *reinterpret_cast<const any_u32_t *>(g);
                else {
                    const any_u32x2_t a = *reinterpret_cast<const any_u32x2_t *>(g);
                    s.g[j][0] = a.x; s.g[j][1] = a.y;
                }
            } else {
#pragma unroll
                for (int i = 0; i < (ME + 1) / 2; ++i) s.g[j][i] = 0;
#pragma unroll
                for (int i = 0; i < ME - 1; ++i)
                    if (in && e + i < E) s.g[j][i / 2] |= (uint32_t)g[i].bits << (i % 2 * 16);
            }
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
    const int most = min(16 * ME, E - eb * 16 * ME), wide = min(LB_COLS, D - col * LB_COLS);
    float *out = part + (split * E + eb * 16 * ME) * D + col * LB_COLS;
    for (int i = threadIdx.x; i < most * LB_COLS; i += 64 * LB_WAVES) {
        const int r = i / LB_COLS, c = i % LB_COLS;
        if (c < wide) out[(int64_t)r * D + c] = lds[r][c];
    }
}

__global__ void __launch_bounds__(512)
linear_reduce_kernel(const float *__restrict__ part, int rows, int64_t n, float *__restrict__ dW)
{
    sum_rows(part, rows, n, [&](int64_t c, float s) { dW[c] = s; });
}

// KS steps of 32 experts, NT tiles of 16 columns: 16 NT columns to a wave, NT consecutive ones to a lane
template <int KS, int NT>
__global__ void __launch_bounds__(64 * LB_WAVES)
linear_du_bf16_kernel(const bf16 *__restrict__ Wg, const bf16 *__restrict__ dl, const bf16 *du_add, bf16 *du, int64_t tokens, int D,
                      int E, int cols, int64_t share)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, kg = lane >> 4;
    const int col = blockIdx.x % cols;
    const int64_t t0 = blockIdx.x / cols * share, t1 = min(t0 + share, tokens);
    const int d = col * 16 * NT + NT * n;
    uint32_t w[KS][NT][4];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        Piece<bf16, NT> p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = 32 * k + 8 * kg + j;
            p[j].template load<true>(Wg + (int64_t)e * D + d, e < E ? D - d : 0);
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) w[k][i][q] = pair_of(p[2 * q].v[i / 2], p[2 * q + 1].v[i / 2], i);
    }
    for (int64_t t = t0 + 16 * wave; t < t1; t += 16 * LB_WAVES) {
        const int64_t ta = min(t + n, tokens - 1);
        f32x4_t acc[NT] = {};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            Piece<bf16, 8> a;
            const int e = 32 * k + 8 * kg;
            a.template load<true>(dl + ta * E + e, E - e);
#pragma unroll
            for (int i = 0; i < NT; ++i) acc[i] = mfma16(a.v, w[k][i], acc[i]);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int64_t tt = t + 4 * kg + v;
            const int left = tt < t1 ? D - d : 0;
            float o[NT];
            Piece<bf16, NT> p;
            if (du_add) p.template load<true>(du_add + tt * D + d, left);
#pragma unroll
            for (int i = 0; i < NT; ++i) o[i] = acc[i][v] + (du_add ? p.get(i) : 0.f);
            store_piece<true>(du + tt * D + d, o, left);
        }
    }
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

// Tokens of a block's share of dW: whole steps of its waves, and so few shares that the blocks are some 512.
struct Shares { int64_t share, count; };
Shares dw_shares(int64_t tokens, int D, int E)
{
    const int64_t blocks = (int64_t)((D + LB_COLS - 1) / LB_COLS) * ((E + 63) / 64), step = 32 * LB_WAVES;
    const int64_t want = blocks < 512 ? 512 / blocks : 1, steps = (tokens + step - 1) / step;
    const int64_t count = steps < want ? (steps > 0 ? steps : 1) : want, share = (steps + count - 1) / count * step;
    return {share, tokens > 0 ? (tokens + share - 1) / share : 0};
}

}  // namespace

size_t router_linear_bwd_bytes(int64_t tokens, int D, int E) { return (size_t)dw_shares(tokens, D, E).count * E * D * sizeof(float); }

swimba_status launch_router_linear_bwd(int64_t tokens, int D, int E, int io_dtype, const void *u, const void *Wg, const void *dl,
                                       const void *du_add, void *du, float *dW, void *work, hipStream_t st)
{
    const Shares sh = dw_shares(tokens, D, E);
    float *part = (float *)work;
    const bool bf = io_dtype == SWIMBA_BF16;
    if (du && tokens > 0) {
        if (bf) {
            auto go = [&](auto kernel, int wide) {
                const int cols = (D + wide - 1) / wide;
                int64_t shares = 2048 / cols > 0 ? 2048 / cols : 1, steps = (tokens + 63) / 64;
                const int64_t share = (steps + shares - 1) / shares * 64;
                shares = (tokens + share - 1) / share;
                hipLaunchKernelGGL(kernel, dim3((unsigned)(cols * shares)), dim3(64 * LB_WAVES), 0, st, (const bf16 *)Wg, (const bf16 *)dl,
                                   (const bf16 *)du_add, (bf16 *)du, tokens, D, E, cols, share);
            };
            if (E <= 32) go(linear_du_bf16_kernel<1, 8>, 128);
            else if (E <= 64) go(linear_du_bf16_kernel<2, 8>, 128);
            else if (E <= 128) go(linear_du_bf16_kernel<4, 8>, 128);
            else go(linear_du_bf16_kernel<8, 4>, 64);
        } else {
            hipLaunchKernelGGL(linear_du_f32_kernel, dim3((unsigned)((tokens * D + 255) / 256 < 65536 ? (tokens * D + 255) / 256 : 65536)), dim3(256), 0, st,
                               (const float *)Wg, (const float *)dl, (const float *)du_add, (float *)du, tokens, D, E);
        }
        SWIMBA_CHECK_LAUNCH();
    }
    if (dW) {
        if (sh.count > 0) {
            if (bf) {
                auto go = [&](auto kernel, int experts) {
                    const int cols = (D + LB_COLS - 1) / LB_COLS, eblocks = (E + experts - 1) / experts;
                    hipLaunchKernelGGL(kernel, dim3((unsigned)(cols * eblocks * sh.count)), dim3(64 * LB_WAVES), 0, st, (const bf16 *)u,
                                       (const bf16 *)dl, part, tokens, D, E, cols, eblocks, sh.share);
                };
                if (E <= 16) go(linear_dw_bf16_kernel<1>, 16);
                else if (E <= 32) go(linear_dw_bf16_kernel<2>, 32);
                else go(linear_dw_bf16_kernel<4>, 64);
            } else {
                hipLaunchKernelGGL(linear_dw_f32_kernel, dim3((unsigned)((D + 255) / 256), (unsigned)E, (unsigned)sh.count), dim3(256), 0,
                                   st, (const float *)u, (const float *)dl, part, tokens, D, E, sh.share);
            }
            SWIMBA_CHECK_LAUNCH();
        }
        const int64_t n = (int64_t)E * D;
        hipLaunchKernelGGL(linear_reduce_kernel, dim3((unsigned)((n + 31) / 32)), dim3(512), 0, st, part, (int)sh.count, n, dW);
        SWIMBA_CHECK_LAUNCH();
    }
    return SWIMBA_OK;
}

}  // namespace swimba
