// Device helpers of the kernels that go over rows of features or logits: vectors of elements whose rows start where they
// start, sums over lanes.
#pragma once

#include "common.hpp"
#include "mfma_util.hpp"

#include <type_traits>

namespace swimba {

// 16 and 8 bytes at an address that is a multiple of the element size only (rows of an odd width): global memory is read and
// written in one piece all the same.
typedef uint32_t __attribute__((ext_vector_type(4), aligned(2))) any_u32x4_t;
typedef uint32_t __attribute__((ext_vector_type(2), aligned(2))) any_u32x2_t;
typedef uint32_t __attribute__((aligned(2))) any_u32_t;

// W (2, 4 or 8) consecutive elements of a row as they lie in memory: loaded long before they are used, they take few registers.
template <typename T, int W> struct Piece {
    static constexpr int WORDS = W * (int)sizeof(T) / 4;
    uint32_t v[WORDS];
    // the first n of the elements (n <= 0: none); the others become zero.  TAIL: n may lie between 0 and W
    template <bool TAIL> __device__ __forceinline__ void load(const T *p, int n)
    {
        if (n >= W) {
            if constexpr (WORDS == 1) {
                v[0] = *reinterpret_cast<const any_u32_t *>(p);
            } else if constexpr (WORDS == 2) {
                const any_u32x2_t a = *reinterpret_cast<const any_u32x2_t *>(p);
                v[0] = a.x; v[1] = a.y;
            } else {
#pragma unroll
                for (int i = 0; i < WORDS; i += 4) {
                    const any_u32x4_t a = *reinterpret_cast<const any_u32x4_t *>(p + i * 4 / sizeof(T));
                    v[i] = a.x; v[i + 1] = a.y; v[i + 2] = a.z; v[i + 3] = a.w;
                }
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < WORDS; ++i) v[i] = 0;
        if constexpr (TAIL) {
#pragma unroll
            for (int i = 0; i < W - 1; ++i)
                if (i < n) {
                    if constexpr (sizeof(T) == 2) v[i / 2] |= (uint32_t)p[i].bits << (i % 2 * 16);
                    else v[i] = __float_as_uint(p[i]);
                }
        }
    }
    __device__ __forceinline__ void drop(int n)                // the first n become zero
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if constexpr (sizeof(T) == 4) v[i] = i < n ? 0 : v[i];
            else v[i] = 2 * i + 1 < n ? 0 : 2 * i < n ? v[i] & 0xffff0000u : v[i];
        }
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(v[i]);
        else return i % 2 ? bf_hi(v[i / 2]) : bf_lo(v[i / 2]);
    }
};

// the first n of W floats to a row, rounded to its type
template <bool TAIL, typename T, int W> __device__ __forceinline__ void store_piece(T *p, const float (&f)[W], int n)
{
    if (n >= W) {
        uint32_t v[Piece<T, W>::WORDS];
#pragma unroll
        for (int i = 0; i < Piece<T, W>::WORDS; ++i) {
            if constexpr (sizeof(T) == 4) v[i] = __float_as_uint(f[i]);
            else v[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
        }
        if constexpr (Piece<T, W>::WORDS == 1) *reinterpret_cast<any_u32_t *>(p) = v[0];
        else if constexpr (Piece<T, W>::WORDS == 2) *reinterpret_cast<any_u32x2_t *>(p) = any_u32x2_t{v[0], v[1]};
        else {
#pragma unroll
            for (int i = 0; i < Piece<T, W>::WORDS; i += 4)
                *reinterpret_cast<any_u32x4_t *>(p + i * 4 / sizeof(T)) = any_u32x4_t{v[i], v[i + 1], v[i + 2], v[i + 3]};
        }
        return;
    }
    if constexpr (TAIL) {
#pragma unroll
        for (int i = 0; i < W - 1; ++i)
            if (i < n) p[i] = from_float<T>(f[i]);
    }
}

// How a row's last piece is read, where it is shorter than the others: it is not, by element, or (in rows of a piece or more) moved
// to end with the row, so that it has some elements of its neighbour in front of its own.  By element, a load waits for the one
// before it, at every row.
enum Tail { NO_TAIL, BY_ELEMENT, MOVED };
constexpr Tail tail_of(int D, int W) { return D % W == 0 ? NO_TAIL : D < W ? BY_ELEMENT : MOVED; }

// A lane's piece of a row of D: W elements that start at d, or with `whole` are there for certain.
template <Tail TAIL, int W> struct Part {
    const uint32_t d, at;              // where it starts, and where it is read
    const int D;
    const bool whole;
    __device__ __forceinline__ Part(uint32_t from, int width, bool certain)
        : d(from), at(TAIL == MOVED && !certain ? min(from, (uint32_t)(width - W)) : from), D(width), whole(certain) {}
    __device__ __forceinline__ bool own(int j) const { return whole || (TAIL == MOVED ? j >= (int)(d - at) : (int)d + j < D); }
    // elements that are not its own: a neighbour's where it is moved, zero otherwise
    template <typename T> __device__ __forceinline__ void load(Piece<T, W> &p, const T *row) const
    {
        if (whole || TAIL == MOVED) p.template load<false>(row + at, W);
        else p.template load<TAIL == BY_ELEMENT>(row + d, D - (int)d);
    }
    // its own elements to the places that they would have, zero behind them
    template <typename T> __device__ __forceinline__ void settle(Piece<T, W> &p) const
    {
        if constexpr (TAIL == MOVED) {
            constexpr int WORDS = Piece<T, W>::WORDS;
            const int by = d - at;
            if (by == 0) return;
            const int words = by * (int)sizeof(T) / 4;
#pragma unroll
            for (int b = WORDS / 2; b > 0; b /= 2)
#pragma unroll
                for (int i = 0; i < WORDS; ++i) p.v[i] = words & b ? (i + b < WORDS ? p.v[i + b] : 0) : p.v[i];
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                if (sizeof(T) == 2) p.v[i] = by % 2 ? p.v[i] >> 16 | (i + 1 < WORDS ? p.v[i + 1] << 16 : 0) : p.v[i];
                p.v[i] = by < W ? p.v[i] : 0;
            }
        }
    }
    template <typename T> __device__ __forceinline__ void store(T *row, const float (&f)[W]) const
    {
        if (whole || (TAIL == MOVED && d == at)) store_piece<false>(row + at, f, W);
        else if (TAIL == MOVED) {
#pragma unroll
            for (int j = 1; j < W; ++j)
                if (own(j)) row[at + j] = from_float<T>(f[j]);
        } else
            store_piece<TAIL == BY_ELEMENT>(row + d, f, D - (int)d);
    }
};

// out[c] = sum over `rows` rows of part (rows, n), c < n, in an order that the sizes alone decide.  32 columns to a block of 512
// threads, whose 16 half waves take every 16th row each: a piece of a row is a line of memory, and up to 16 x 8 are under way.
template <typename Store>
__device__ __forceinline__ void sum_rows(const float *__restrict__ part, int rows, int64_t n, Store store)
{
    __shared__ float lds[16][33];
    const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x % 32;
    const int slice = threadIdx.x / 32;
    float s = 0.f;
    if (c < n) {
#pragma unroll 8
        for (int i = slice; i < rows; i += 16) s += part[i * n + c];
    }
    lds[slice][threadIdx.x % 32] = s;
    __syncthreads();
    if (slice || c >= n) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += lds[i][threadIdx.x];
    store(c, s);
}

// The value of the lane at distance D, once the lanes at smaller distances agree (for D = 4 and 8 another lane of those
// stands in).  Register moves, no LDS pass.
template <int D>
__device__ __forceinline__ uint32_t partner(uint32_t v)
{
    static_assert(D == 1 || D == 2 || D == 4 || D == 8, "inside a row of 16 lanes");
    constexpr int ctrl = D == 1 ? 0xB1 : D == 2 ? 0x4E : D == 4 ? 0x141 : 0x128;   // quad_perm, half mirror, row_ror:8
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, true);
}
// op over lanes whose numbers differ in the bits from FROM to below TO, in every one of them
template <int FROM, int TO, typename Op>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, Op op)
{
    if constexpr (FROM < TO) {
        if constexpr (FROM >= 16) {
            const auto r = FROM == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
            v = op(r[0], r[1]);
        } else if constexpr (FROM == 4) {
            v = op(v, (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x101f));          // xor 4
        } else
            v = op(v, partner<FROM>(v));
        return over_lanes<FROM * 2, TO>(v, op);
    }
    return v;
}
// the same over the lanes of an aligned group of G
template <int G, typename Op>
__device__ __forceinline__ uint32_t over_group(uint32_t v, Op op)
{
    if constexpr (G > 1) v = op(v, partner<1>(v));
    if constexpr (G > 2) v = op(v, partner<2>(v));
    if constexpr (G > 4) v = op(v, partner<4>(v));
    return over_lanes<8, G>(v, op);
}
__device__ __forceinline__ uint32_t add_f32(uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }
__device__ __forceinline__ uint32_t max_f32(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
__device__ __forceinline__ uint32_t add_u32(uint32_t a, uint32_t b) { return a + b; }
__device__ __forceinline__ uint32_t or_u32(uint32_t a, uint32_t b) { return a | b; }
template <int G> __device__ __forceinline__ float group_sum(float v) { return __uint_as_float(over_group<G>(__float_as_uint(v), add_f32)); }
// the same in 64 bits, whose halves move one after the other; D: distance of the step
template <int G, int D = 1> __device__ __forceinline__ double group_sum(double v)
{
    if constexpr (D < G) {
        const uint32_t lo = (uint32_t)__double2loint(v), hi = (uint32_t)__double2hiint(v);
        if constexpr (D >= 16) {
            const auto a = D == 16 ? __builtin_amdgcn_permlane16_swap(lo, lo, false, false) : __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
            const auto b = D == 16 ? __builtin_amdgcn_permlane16_swap(hi, hi, false, false) : __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
            v = __hiloint2double((int)b[0], (int)a[0]) + __hiloint2double((int)b[1], (int)a[1]);
        } else
            v += __hiloint2double((int)partner<D>(hi), (int)partner<D>(lo));
        return group_sum<G, 2 * D>(v);
    }
    return v;
}

// Sums of N values over the lanes whose numbers differ in the bits from G to below 2 D.  While a lane has several, a step halves
// them: the lanes with bit D clear keep the lower half, the others the upper.  v[i] is then the sum of value `first` + i.
template <int D, int G, int N, int LEFT = N>
__device__ __forceinline__ void sum_over(float (&v)[N], int &first, int lane)
{
    if constexpr (D >= G) {
        if constexpr (LEFT > 1) {
#pragma unroll
            for (int i = 0; i < LEFT / 2; ++i) {
                uint32_t a = __float_as_uint(v[i]), b = __float_as_uint(v[i + LEFT / 2]);
                if constexpr (D >= 16) {
                    const auto r = D == 16 ? __builtin_amdgcn_permlane16_swap(a, b, false, false) : __builtin_amdgcn_permlane32_swap(a, b, false, false);
                    v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
                } else {
                    const bool hi = lane & D;
                    const uint32_t keep = hi ? b : a, send = hi ? a : b;
                    uint32_t got;
                    if constexpr (D == 4) got = (uint32_t)__builtin_amdgcn_ds_swizzle((int)send, 0x101f);
                    else got = partner<D>(send);
                    v[i] = __uint_as_float(keep) + __uint_as_float(got);
                }
            }
            first += lane & D ? LEFT / 2 : 0;
            sum_over<D / 2, G, N, LEFT / 2>(v, first, lane);
        } else {
            v[0] = __uint_as_float(over_lanes<D, 2 * D>(__float_as_uint(v[0]), add_f32));
            sum_over<D / 2, G, N, 1>(v, first, lane);
        }
    }
}

}  // namespace swimba
