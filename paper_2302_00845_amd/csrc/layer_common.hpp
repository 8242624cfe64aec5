// Per-example gradients of layers: element types, rows of examples, sums over lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cdgrab {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// N consecutive elements at any element address.  (Global memory takes 16-byte accesses at any address; rows of
// odd length need no path of their own.)
template <typename T, int N>
struct AnyVec {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <typename T, int N, bool ONCE = false>  // ONCE: not to be kept in the caches
__device__ __forceinline__ void load_any(const T *p, T (&v)[N]) {
    if constexpr (N == 1) {
        v[0] = *p;
    } else {
        typename AnyVec<T, N>::type x;
        if constexpr (ONCE && N * sizeof(T) == 16) {
            typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
            x = __builtin_bit_cast(typename AnyVec<T, N>::type, __builtin_nontemporal_load(reinterpret_cast<const words *>(p)));
        } else {
            x = *reinterpret_cast<const typename AnyVec<T, N>::type *>(p);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = x[j];
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_any(T *p, const T (&v)[N]) {
    if constexpr (N == 1) {
        *p = v[0];
    } else {
        typename AnyVec<T, N>::type x;
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = v[j];
        *reinterpret_cast<typename AnyVec<T, N>::type *>(p) = x;
    }
}

// The rows of the examples: example e has `count[e]` rows (NULL: `tokens`) from row `first[e]` (NULL: e * tokens) on.
// What of that lies outside the array's `rows` rows, or beyond `tokens`, is cut off, whatever the arrays hold.
struct TokenRows {
    int64_t examples, rows, tokens;
    const int64_t *first;
    const int32_t *count;
    int64_t base;  // a launch's first example
};
struct RowSpan { int64_t first, count; };
__device__ __forceinline__ RowSpan rows_of(const TokenRows &t, int64_t e) {
    RowSpan s{t.first ? t.first[e] : e * t.tokens, t.count ? (int64_t)t.count[e] : t.tokens};
    if (s.first < 0 || s.first > t.rows) return RowSpan{0, 0};
    if (s.count > t.tokens) s.count = t.tokens;
    if (s.count > t.rows - s.first) s.count = t.rows - s.first;
    if (s.count < 0) s.count = 0;
    return s;
}

// Sum over the LANES consecutive lanes that hold a row, left in every one of them: DPP within sixteen, row swaps beyond.
template <int CTRL>
__device__ __forceinline__ float dpp_add_f32(float x) {
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
    static_assert(LANES == 8 || LANES == 16 || LANES == 32 || LANES == 64, "");
    x = dpp_add_f32<0xB1>(x);   // quad_perm 1 0 3 2
    x = dpp_add_f32<0x4E>(x);   // quad_perm 2 3 0 1
    x = dpp_add_f32<0x141>(x);  // row_half_mirror
    if constexpr (LANES >= 16) x = dpp_add_f32<0x140>(x);  // row_mirror
    if constexpr (LANES >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_int(x), __float_as_int(x), false, false);
        x = __int_as_float((int)p[0]) + __int_as_float((int)p[1]);
    }
    if constexpr (LANES >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
        x = __int_as_float((int)p[0]) + __int_as_float((int)p[1]);
    }
    return x;
}

// Workgroup b of `total` as the position in an order in which neighbours run on the same XCD (workgroups go round
// the eight XCDs): what neighbouring tiles read in common then comes from one L2.
__device__ __forceinline__ uint32_t xcd_neighbours(uint32_t b, uint32_t total) {
    const uint32_t per = total >> 3, rest = total & 7, x = b & 7, at = b >> 3;
    return x * per + (x < rest ? x : rest) + at;
}

}  // namespace cdgrab
