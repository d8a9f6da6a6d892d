// Layer norm of token features and its backward pass.
//   forward   r = x (+ residual, rounded to the type it is stored in), u = (r - m) s gamma + beta
//   backward  dx = s (g - mean g - xh mean(g xh)) + d_sum with g = du gamma, xh = (r - m) s;  dgamma = sum_t du xh, dbeta = sum_t du
// Both are bound by memory: every row is read once into registers, where the mean (of fp32 rows in 64 bits), then the centred
// squares (or both sums of the backward pass) are taken in fp32, and written once.  16384 x 768 of bf16 into an fp32 stream
// 25.3 us (151 MB, 6.0 TB/s), back 39.5 (201 MB, 5.1 TB/s); 32768 x 4096 of bf16 114 us (4.7 TB/s), back 153 (5.3 TB/s); one token
// 2.4 us of kernel.
// Where a row does not end with a piece, the last one is moved to end with it: 20490 x 2047 of bf16 back 84 us, 131 with loads by
// element, of which each waits for the one before.  2048 wide takes 51: the moved lane's stores by element cost 22 us at 2044 to 2046
// wide (74), rows that start inside a dword 10 more.
#include "rows.hpp"

namespace swimba {

// A row lies in the registers of LPR lanes (16 to 64 of a wave, or all of 4, 8 or 16 waves), W NV elements to a lane: piece i of
// lane l are the elements from W (l + LPR i) on.
constexpr int norm_threads(int LPR) { return LPR < 256 ? 256 : LPR; }
constexpr int rows_per_block(int LPR) { return norm_threads(LPR) / LPR; }

// Pieces that end before the narrowest row of those that LPR lanes with NV pieces are chosen for.
constexpr int whole_pieces(int LPR, int NV) { return LPR <= 64 || NV < 4 ? NV - 1 : NV - 2; }

// Piece i of a lane.  Where it may be moved, its place is worked out anew wherever it is asked for: kept for all pieces, the places
// would take the registers of a wave.
template <Tail TAIL, int W, int LPR, int NV> __device__ __forceinline__ Part<TAIL, W> row_part(int lane, int i, int D)
{
    const bool whole = i < whole_pieces(LPR, NV);
    uint32_t from = W * (lane + LPR * i);
    if (TAIL == MOVED && !whole) asm volatile("" : "+v"(from));
    return Part<TAIL, W>(from, D, whole);
}

// Threads of a block of the backward pass, of which two fit on a compute unit at the registers that its pieces take.
constexpr int bwd_threads(int LPR, int NV) { return LPR > 64 ? LPR : NV == 1 ? 1024 : NV == 2 ? 512 : 256; }

// sums of N values over the row's lanes, in every one of them; `round` alternates, so that one barrier a round is enough
template <int LPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*lds)[N][16], int round)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = group_sum<LPR < 64 ? LPR : 64>(v[i]);
    if constexpr (LPR > 64) {
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < N; ++i) lds[round & 1][i][wave] = v[i];
        lds_barrier();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < LPR / 64; ++w) v[i] += lds[round & 1][i][w];
        }
    }
}

// the same of one value, in 64 bits
template <int LPR> __device__ __forceinline__ double row_sum(double v, double (*lds)[16], int round)
{
    v = group_sum<LPR < 64 ? LPR : 64>(v);
    if constexpr (LPR > 64) {
        lds[round & 1][threadIdx.x >> 6] = v;
        lds_barrier();
        v = 0.;
#pragma unroll
        for (int w = 0; w < LPR / 64; ++w) v += lds[round & 1][w];
    }
    return v;
}

// first row of the thread's lanes in the block
template <int LPR> __device__ __forceinline__ int row_slot()
{
    return LPR < 64 ? threadIdx.x / LPR : __builtin_amdgcn_readfirstlane(threadIdx.x / 64) / (LPR / 64);
}

template <typename T, typename R, int W, int NV, int LPR, Tail TAIL>
__global__ void __launch_bounds__(norm_threads(LPR))
norm_fwd_kernel(const T *x, const R *residual, const float *__restrict__ gamma, const float *__restrict__ beta, float eps,
                T *__restrict__ u, R *sum, float *__restrict__ mean, float *__restrict__ rstd, int64_t tokens, int D, double per_width)
{
    // What a mean is off by shifts every deviation, and its square goes into the variance.  Rows of bf16 are summed in 32 bits:
    // equal elements exactly (8 bits each, at most 2^14 of them), others to some 2^-18 of the largest, where each is stored to 2^-9.
    // Rows of fp32 are summed in 64, and what the mean loses in 32 bits is taken off the deviations as well; in 32 bits a row of
    // 1000 times 12345.678 would come out at 0.5 instead of 0.  64 bits and 32: 16384 x 1024 22.8 us both, 16384 x 4096 96.5 and
    // 99.8, 4096 x 16384 119.4 and 118.5, 262144 x 64 23.4 and 23.2.
    constexpr bool WIDE = sizeof(R) == 4;
    __shared__ float lds[2][1][16];
    __shared__ double lds64[2][16];
    constexpr int RPB = rows_per_block(LPR);                   // rows a block has at a time
    const int lane = threadIdx.x % LPR;
    const float width = (float)D;
    auto part = [&](int i) __attribute__((always_inline)) { return row_part<TAIL, W, LPR, NV>(lane, i, D); };
    int round = 0;
    // Gain and bias are under way with the row where it lies in one wave (16384 x 768 13.0 -> 11.0 us); more lanes to a row have
    // other waves to wait with and lose by the registers (16384 x 8192 118 -> 136 us).
    constexpr bool EARLY = LPR <= 64;
    Piece<float, W> g[EARLY ? NV : 1], b[EARLY ? NV : 1];
    auto weights = [&](int i, int k) __attribute__((always_inline)) {
        const auto at = part(i);
        if (gamma) at.load(g[k], gamma);
        if (beta) at.load(b[k], beta);
    };
    if constexpr (EARLY) {
#pragma unroll
        for (int i = 0; i < NV; ++i) weights(i, i);
    }
    for (int64_t t = (int64_t)blockIdx.x * RPB + row_slot<LPR>(); t < tokens; t += (int64_t)gridDim.x * RPB) {
        const T *const xr = x + t * D;
        const R *const rr = residual + t * D;
        R *const sr = sum + t * D;
        T *const ur = u + t * D;
        Piece<T, W> px[NV];
        Piece<R, W> pr[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const auto at = part(i);
            at.load(px[i], xr);
            if (residual) at.load(pr[i], rr);
        }
        float r[NV][W], s[1];
        std::conditional_t<WIDE, double, float> total = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const auto at = part(i);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                r[i][j] = px[i].get(j);
                if (residual) r[i][j] = to_float(from_float<R>(r[i][j] + pr[i].get(j)));
                total += TAIL != MOVED || at.own(j) ? r[i][j] : 0.f;
            }
            if (sum) at.store(sr, r[i]);
        }
        float m, rest = 0.f;                                   // the mean, and what it has beyond 32 bits
        if constexpr (WIDE) {
            const double all = row_sum<LPR>(total, lds64, round++);
            double q = all * per_width;
            const double off = fma(-q, (double)D, all);        // divided, so that a constant row is centred to zero
            q = off == off ? fma(off, per_width, q) : q;       // (an infinite row's mean stays infinite)
            m = (float)q;
            rest = (float)(q - m);
        } else {
            s[0] = total;
            row_sums<LPR>(s, lds, round++);
            m = s[0] / width;
        }
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const auto at = part(i);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                r[i][j] -= m;
                if constexpr (WIDE) r[i][j] -= rest;
                s[0] += at.own(j) ? r[i][j] * r[i][j] : 0.f;
            }
        }
        row_sums<LPR>(s, lds, round++);
        const float is = 1.0f / sqrtf(s[0] / width + eps);
        if (lane == 0) {
            if (mean) mean[t] = m;
            if (rstd) rstd[t] = is;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = EARLY ? i : 0;
            if constexpr (!EARLY) weights(i, 0);
#pragma unroll
            for (int j = 0; j < W; ++j) r[i][j] = r[i][j] * is * (gamma ? g[k].get(j) : 1.f) + (beta ? b[k].get(j) : 0.f);
            part(i).store(ur, r[i]);
        }
    }
}

// The blocks keep sums of their own for dgamma and dbeta: part (blocks, 2, D), or the two themselves where there is one block.
template <typename T, typename R, int W, int NV, int LPR, Tail TAIL>
__global__ void __launch_bounds__(bwd_threads(LPR, NV))
norm_bwd_kernel(const T *__restrict__ du, const R *__restrict__ r, const float *__restrict__ gamma,
                const float *__restrict__ mean, const float *__restrict__ rstd, const R *d_sum, R *dx, T *__restrict__ dx_io,
                float *__restrict__ pgamma, float *__restrict__ pbeta, int64_t tokens, int D)
{
    constexpr int THREADS = bwd_threads(LPR, NV), RPB = THREADS / LPR, SPAN = LPR * W;
    constexpr bool AHEAD = NV * W <= (sizeof(T) + sizeof(R) == 4 ? 24 : 16);   // more leave no registers for it, nor for the gain
    __shared__ float lds[2][2][16];
    __shared__ float comb[RPB > 1 ? RPB * 2 * NV * SPAN : 1];
    const int lane = threadIdx.x % LPR, slot = row_slot<LPR>();
    const float width = (float)D;
    auto part = [&](int i) __attribute__((always_inline)) { return row_part<TAIL, W, LPR, NV>(lane, i, D); };
    const int64_t stride = (int64_t)gridDim.x * RPB;
    float dg[NV][W] = {}, db[NV][W] = {}, w[NV][W];
    auto gain = [&] {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Piece<float, W> p;
            const auto at = part(i);
            if (gamma) at.load(p, gamma);
#pragma unroll
            for (int j = 0; j < W; ++j) w[i][j] = TAIL == MOVED && !at.own(j) ? 0.f : gamma ? p.get(j) : 1.f;
        }
    };
    if constexpr (AHEAD) gain();
    struct Row {
        Piece<T, W> g[NV];
        Piece<R, W> x[NV], a[NV];
        float m, s;
    };
    auto fetch = [&](Row &q, int64_t t) __attribute__((always_inline)) {
        q.m = mean[t];
        q.s = rstd[t];
        const R *const row = r + t * D, *const add = d_sum + t * D;
        const T *const grad = du + t * D;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const auto at = part(i);
            at.load(q.x[i], row);
            at.load(q.g[i], grad);
            if (AHEAD && d_sum) at.load(q.a[i], add);
        }
    };
    Row next;
    int64_t t = (int64_t)blockIdx.x * RPB + slot;
    if (AHEAD && t < tokens) fetch(next, t);
    for (int round = 0; t < tokens; t += stride, ++round) {
        Row q;
        if constexpr (AHEAD) {
            q = next;
            if (t + stride < tokens) fetch(next, t + stride);
        } else {
            fetch(q, t);
            gain();
        }
        float xh[NV][W], g[NV][W], s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const auto at = part(i);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                xh[i][j] = at.own(j) ? (q.x[i].get(j) - q.m) * q.s : 0.f;
                g[i][j] = TAIL != MOVED || at.own(j) ? q.g[i].get(j) : 0.f;
                dg[i][j] += g[i][j] * xh[i][j];
                db[i][j] += g[i][j];
                g[i][j] *= w[i][j];
                s[0] += g[i][j];
                s[1] += g[i][j] * xh[i][j];
            }
        }
        row_sums<LPR>(s, lds, round);
        const float mg = s[0] / width, mx = s[1] / width;
        R *const out = dx + t * D;
        T *const out_io = dx_io + t * D;
        const R *const add = d_sum + t * D;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const auto at = part(i);
            if (!AHEAD && d_sum) at.load(q.a[i], add);
#pragma unroll
            for (int j = 0; j < W; ++j) g[i][j] = q.s * (g[i][j] - mg - xh[i][j] * mx) + (d_sum ? q.a[i].get(j) : 0.f);
            at.store(out, g[i]);
            if (dx_io) at.store(out_io, g[i]);
        }
    }
    float *const pg = pgamma + (int64_t)blockIdx.x * 2 * D, *const pb = pbeta + (int64_t)blockIdx.x * 2 * D;
    if (!pgamma && !pbeta) return;
    if constexpr (RPB > 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const auto at = part(i);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                if (!at.own(j)) continue;
                const int d = at.at + j;
                comb[(slot * 2) * NV * SPAN + d] = dg[i][j];
                comb[(slot * 2 + 1) * NV * SPAN + d] = db[i][j];
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * D; c += THREADS) {
            const int at = c < D ? c : c - D + NV * SPAN;
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < RPB; ++k) s += comb[k * 2 * NV * SPAN + at];
            if (c < D && pgamma) pg[c] = s;
            if (c >= D && pbeta) pb[c - D] = s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (pgamma) part(i).store(pg, dg[i]);
            if (pbeta) part(i).store(pb, db[i]);
        }
    }
}

// the blocks' sums joined; columns behind D are dbeta's
__global__ void __launch_bounds__(512)
norm_reduce_kernel(const float *__restrict__ part, int rows, int D, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    sum_rows(part, rows, 2 * D, [&](int64_t c, float s) {
        float *out = c < D ? dgamma : dbeta;
        if (out) out[c < D ? c : c - D] = s;
    });
}

namespace {

// Lanes of a row: one piece to a lane up to 256 features; beyond, 16 elements at most, or 24 where that keeps more lanes at work
// (42 million elements of bf16, 24 and 16 to a lane: rows of 4104 39.3 us and 51.0, 5204 36.7 and 46.7, 6144 33.5 and 39.0, 8200 47.9 and
// 68.1, 10240 41.5 and 57.7, 12288 38.4 and 53.9; back 4104 51.6 and 62.9, 5204 55.3 and 71.0, 6144 the same).  Four-byte rows of 4096 to
// 6144 gain nothing by it.  The backward pass has up to 32 in 512 lanes, without the next row under way: 1024 have 128 registers
// each and spill (2560 x 16384 fp32 104 us, 96 with 512; 4660 x 9000 113 and 94).
int lanes_per_row(int D, bool bf, bool back)
{
    if (D <= 1024) return D <= 64 ? 16 : D <= 128 ? 32 : 64;
    return D <= (bf ? 6144 : 4096) ? 256 : D <= 12288 || back ? 512 : 1024;
}

// f(elements of a piece, pieces, lanes of a row, how the last piece is read) as constants.  Pieces of 16 bytes for
// wide rows of bf16 alone (32768 x 2048 forward 62 us with 8 bytes, 58.6 with 16; backward 85 and 79); of 4 elements elsewhere,
// which fill the lanes of a narrow row better.
template <typename T, typename R, bool BACK, typename F>
void with_row(int D, F &&f)
{
    using std::integral_constant;
    constexpr bool BF = sizeof(T) + sizeof(R) == 4;
    constexpr integral_constant<int, 1> one;
    constexpr integral_constant<int, 2> two;
    constexpr integral_constant<int, 3> three;
    constexpr integral_constant<int, 4> four;
    constexpr integral_constant<int, BF ? 8 : 4> wide;
    constexpr integral_constant<int, 16 / wide> most;
    constexpr integral_constant<int, 24 / wide> more;
    auto tail = [&](auto w, auto pieces, auto lanes) {
        if constexpr (lanes == 16) {
            if (tail_of(D, w) == BY_ELEMENT) return f(w, pieces, lanes, integral_constant<Tail, BY_ELEMENT>());
        }
        if (tail_of(D, w) == MOVED) f(w, pieces, lanes, integral_constant<Tail, MOVED>());
        else f(w, pieces, lanes, integral_constant<Tail, NO_TAIL>());
    };
    switch (lanes_per_row(D, BF, BACK)) {
    case 16: return tail(four, one, integral_constant<int, 16>());
    case 32: return tail(four, one, integral_constant<int, 32>());
    case 64: {
        constexpr integral_constant<int, 64> lanes;
        return D <= 256 ? tail(four, one, lanes) : D <= 512 ? tail(four, two, lanes) : D <= 768 ? tail(four, three, lanes) : tail(four, four, lanes);
    }
    case 256: {
        constexpr integral_constant<int, 256> lanes;
        if constexpr (BF) {
            if (D > 4096) return tail(wide, more, lanes);
        }
        return D <= 2048 ? tail(wide, integral_constant<int, most / 2>(), lanes) : tail(wide, most, lanes);
    }
    case 512: {
        constexpr integral_constant<int, 512> lanes;
        if constexpr (BACK) {
            if (D > 12288) return tail(wide, integral_constant<int, 32 / wide>(), lanes);
        }
        return D > 8192 ? tail(wide, more, lanes) : tail(wide, most, lanes);
    }
    default:
        if constexpr (!BACK) tail(wide, most, integral_constant<int, 1024>());
    }
}

int64_t blocks_for(int64_t tokens, int rpb, int64_t most)
{
    const int64_t need = (tokens + rpb - 1) / rpb;
    return need < most ? need : most;
}

template <typename T, typename R>
swimba_status norm_fwd(int64_t tokens, int D, const void *x, const void *residual, const float *gamma, const float *beta,
                       float eps, void *u, void *sum, float *mean, float *rstd, hipStream_t st)
{
    auto go = [&](auto w, auto nv, auto lpr, auto tail) {
        hipLaunchKernelGGL((norm_fwd_kernel<T, R, w(), nv(), lpr(), tail()>), dim3((unsigned)blocks_for(tokens, rows_per_block(lpr), 1 << 20)),
                           dim3(norm_threads(lpr)), 0, st, (const T *)x, (const R *)residual, gamma, beta, eps, (T *)u, (R *)sum, mean,
                           rstd, tokens, D, 1. / D);
    };
    with_row<T, R, false>(D, go);
    SWIMBA_CHECK_LAUNCH();
    return SWIMBA_OK;
}

// Blocks of the backward pass, which keep sums of their own: one, whose sums need no second launch, for up to four rounds of
// its rows; no more than two to a compute unit, or one for the widest rows.  The same for all types: only rows of more than a wave
// lie in other numbers of lanes, one of them to a block.
int64_t bwd_blocks(int64_t tokens, int D)
{
    const int lpr = lanes_per_row(D, true, true), rpb = bwd_threads(lpr, (D + 4 * lpr - 1) / (4 * lpr)) / lpr;
    return tokens <= 4 * rpb ? (tokens > 0) : blocks_for(tokens, rpb, D > 8192 ? 256 : 512);
}

template <typename T, typename R>
swimba_status norm_bwd(int64_t tokens, int D, const void *du, const void *r, const float *gamma, const float *mean,
                       const float *rstd, const void *d_sum, void *dx, void *dx_io, float *pgamma, float *pbeta, hipStream_t st)
{
    auto go = [&](auto w, auto nv, auto lpr, auto tail) {
        hipLaunchKernelGGL((norm_bwd_kernel<T, R, w(), nv(), lpr(), tail()>), dim3((unsigned)bwd_blocks(tokens, D)),
                           dim3(bwd_threads(lpr, nv)), 0, st, (const T *)du, (const R *)r, gamma, mean, rstd, (const R *)d_sum, (R *)dx,
                           (T *)dx_io, pgamma, pbeta, tokens, D);
    };
    with_row<T, R, true>(D, go);
    SWIMBA_CHECK_LAUNCH();
    return SWIMBA_OK;
}

}  // namespace

size_t layer_norm_bwd_bytes(int64_t tokens, int D)
{
    const int64_t n = bwd_blocks(tokens, D);
    return n > 1 ? (size_t)n * 2 * D * sizeof(float) : 0;
}

swimba_status launch_layer_norm(int64_t tokens, int D, int io_dtype, int res_dtype, const void *x, const void *residual,
                                const float *gamma, const float *beta, float eps, void *u, void *sum, float *mean, float *rstd,
                                hipStream_t st)
{
    if (tokens == 0) return SWIMBA_OK;
    const auto go = io_dtype == SWIMBA_F32 ? norm_fwd<float, float> : res_dtype == SWIMBA_F32 ? norm_fwd<bf16, float> : norm_fwd<bf16, bf16>;
    return go(tokens, D, x, residual, gamma, beta, eps, u, sum, mean, rstd, st);
}

swimba_status launch_layer_norm_bwd(int64_t tokens, int D, int io_dtype, int res_dtype, const void *du, const void *r,
                                    const float *gamma, const float *mean, const float *rstd, const void *d_sum, void *dx,
                                    void *dx_io, float *dgamma, float *dbeta, float *part, hipStream_t st)
{
    const int64_t blocks = bwd_blocks(tokens, D);
    const bool join = blocks != 1 && (dgamma || dbeta);
    if (tokens > 0) {
        const auto go = io_dtype == SWIMBA_F32 ? norm_bwd<float, float> : res_dtype == SWIMBA_F32 ? norm_bwd<bf16, float> : norm_bwd<bf16, bf16>;
        const swimba_status s = go(tokens, D, du, r, gamma, mean, rstd, d_sum, dx, dx_io, join ? part : dgamma, join ? part + D : dbeta, st);
        if (s != SWIMBA_OK) return s;
    }
    if (join) {
        hipLaunchKernelGGL(norm_reduce_kernel, dim3((unsigned)((2 * D + 31) / 32)), dim3(512), 0, st, part, (int)blocks, D, dgamma, dbeta);
        SWIMBA_CHECK_LAUNCH();
    }
    return SWIMBA_OK;
}

}  // namespace swimba
