// Element types of the recognition operators and their wide loads and stores.
//
// A thread takes 16 bytes of a row at once: 4 floats, 8 bfloat16 or 2 doubles.  Rows may
// begin at any multiple of the element's size (odd widths, strided rows): the vector types
// below carry the element's alignment only, and the hardware takes such global accesses.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gpps {

struct bf16_t {
    uint16_t bits;
};

// Acc: the type of sums, states and parameters beside arrays of T.
template <typename T> struct Elem;
template <> struct Elem<float> {
    using Acc = float;
    using Store = float;
    static constexpr int V = 4;
    __device__ static float up(float s) { return s; }
    __device__ static float down(float a) { return a; }
};
template <> struct Elem<double> {
    using Acc = double;
    using Store = double;
    static constexpr int V = 2;
    __device__ static double up(double s) { return s; }
    __device__ static double down(double a) { return a; }
};
template <> struct Elem<bf16_t> {
    using Acc = float;
    using Store = uint16_t;
    static constexpr int V = 8;
    __device__ static float up(uint16_t s) { return __uint_as_float(uint32_t(s) << 16); }
    // to nearest, ties to even: the one rounding of a result computed in 32 bits
    __device__ static uint16_t down(float a) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(a)); }
};

// N values of type S, aligned as one of them.
template <typename S, int N>
struct Wide {
    typedef S type __attribute__((ext_vector_type(N), aligned(sizeof(S))));
};

// n of the V values at p (the others are zero).
template <typename S, int V>
__device__ inline typename Wide<S, V>::type load_some(const S *p, int n) {
    using W = typename Wide<S, V>::type;
    if (n >= V) return *reinterpret_cast<const W *>(p);
    W r = 0;
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (v < n) r[v] = p[v];
    return r;
}

template <typename S, int V>
__device__ inline void store_some(S *p, int n, typename Wide<S, V>::type x) {
    using W = typename Wide<S, V>::type;
    if (n >= V) {
        *reinterpret_cast<W *>(p) = x;
        return;
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (v < n) p[v] = x[v];
}

// x of the lane that the DPP control names.
template <int CTRL>
__device__ inline float lane_of(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false));
}
template <int CTRL>
__device__ inline double lane_of(double x) {
    const long long u = __double_as_longlong(x);
    const int lo = __builtin_amdgcn_update_dpp(0, int(u), CTRL, 0xf, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, int(u >> 32), CTRL, 0xf, 0xf, false);
    return __longlong_as_double((long long)hi << 32 | (unsigned)lo);
}

// Sum over groups of WIDTH neighbouring lanes (8, 16, 32 or 64), the same bits in each of them.
// Within 16 lanes by DPP moves (the neighbour, the other pair, the other four, the other eight).
template <int WIDTH, typename A>
__device__ inline A lanes_sum(A x) {
    x += lane_of<0xb1>(x);                   // quad_perm 1, 0, 3, 2
    x += lane_of<0x4e>(x);                   // quad_perm 2, 3, 0, 1
    x += lane_of<0x141>(x);                  // row_half_mirror
    if constexpr (WIDTH >= 16) x += lane_of<0x140>(x);       // row_mirror
    if constexpr (WIDTH >= 32) x += __shfl_xor(x, 16);
    if constexpr (WIDTH >= 64) x += __shfl_xor(x, 32);
    return x;
}

}  // namespace gpps
