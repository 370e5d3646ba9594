// Elements, rows and activations on the device, shared by the operators on feature rows.
#pragma once

#include <type_traits>

#include "rows_internal.h"

namespace aug {

// Calls f with whether no lane's stretch ends outside the row.
template <class F> hipError_t with_full(bool full, F f) { return full ? f(std::true_type()) : f(std::false_type()); }
// Calls f with a value of the element type.
template <class F> hipError_t with_type(int dtype, F f) {
    return dtype == AUG_BF16 ? f((__bf16)0) : dtype == AUG_F16 ? f((_Float16)0) : f(0.f);
}

template <class T> __device__ inline const T* row_in(const aug_rows& m, int64_t r) { return static_cast<const T*>(m.data) + r * m.ld; }
template <class T> __device__ inline T* row_out(const aug_rows& m, int64_t r) { return static_cast<T*>(m.data) + r * m.ld; }

// N elements next to each other, aligned as one element is: wide accesses, which the hardware allows at any such address.
template <class T, int N> struct Pack {
    T v[N];
};
// Elements 0 .. valid - 1 of the N at p (zeros behind them; valid may be negative); nothing else is touched.
template <class T, int N> __device__ inline Pack<T, N> load_pack(const T* p, int valid) {
    Pack<T, N> r;
    if (valid >= N) {
        __builtin_memcpy(r.v, p, sizeof r);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) r.v[i] = i < valid ? p[i] : (T)0;
    }
    return r;
}
template <class T, int N> __device__ inline void store_pack(T* p, const Pack<T, N>& r, int valid) {
    if (valid >= N) {
        __builtin_memcpy(p, r.v, sizeof r);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < valid) p[i] = r.v[i];
}

// A stretch of channels of row r.  FULL: all of it is there, one access without a branch; else `valid` elements of it.  (With a branch per
// load the loads of several rows wait for one another where the branches meet: the short convolution of 64 utterances 157 us, so 95.)
template <class T, int VE, bool FULL> __device__ inline Pack<T, VE> load_part(const aug_rows& m, int64_t r, int col, int valid) {
    if constexpr (FULL) {
        Pack<T, VE> v;
        __builtin_memcpy(v.v, row_in<T>(m, r) + col, sizeof v);
        return v;
    } else {
        return load_pack<T, VE>(row_in<T>(m, r) + col, valid);
    }
}
template <class T, int VE, bool FULL> __device__ inline void store_part(const aug_rows& m, int64_t r, int col, const Pack<T, VE>& v, int valid) {
    if constexpr (FULL) __builtin_memcpy(row_out<T>(m, r) + col, v.v, sizeof v);
    else store_pack<T, VE>(row_out<T>(m, r) + col, v, valid);
}

// The sum over LN (a power of two) neighbouring lanes, in all of them: quads by permutation, then mirrored halves and swapped rows, whose
// lanes hold equal sums already.
template <int CTRL> __device__ inline float dpp_add(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int LN> __device__ inline float lanes_sum(float v) {
    if constexpr (LN >= 2) v = dpp_add<0xB1>(v);
    if constexpr (LN >= 4) v = dpp_add<0x4E>(v);
    if constexpr (LN >= 8) v = dpp_add<0x141>(v);
    if constexpr (LN >= 16) v = dpp_add<0x140>(v);
    if constexpr (LN >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (LN >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}
// Four sums over the lanes of a quad, lane q of it gets the q-th: halved twice by the bits of q, nine instructions where four sums and
// their selection take twelve.
__device__ inline float quad_sums(const float (&v)[4]) {
    const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
    auto pass = [](float x, auto ctrl) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl.value, 0xf, 0xf, true)); };
    const std::integral_constant<int, 0xB1> next;
    const std::integral_constant<int, 0x4E> second;
    const float low = (odd ? v[1] : v[0]) + pass(odd ? v[0] : v[1], next), up = (odd ? v[3] : v[2]) + pass(odd ? v[2] : v[3], next);
    return (high ? up : low) + pass(high ? low : up, second);
}
// The largest of so many neighbouring lanes' values likewise; `lanes` is the same for the whole wavefront.
template <int CTRL> __device__ inline unsigned dpp_max(unsigned v) {
    const unsigned o = __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
    return v > o ? v : o;
}
__device__ inline unsigned lanes_max(unsigned v, int lanes) {
    if (lanes >= 2) v = dpp_max<0xB1>(v);
    if (lanes >= 4) v = dpp_max<0x4E>(v);
    if (lanes >= 8) v = dpp_max<0x141>(v);
    if (lanes >= 16) v = dpp_max<0x140>(v);
    if (lanes >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = r[0] > r[1] ? r[0] : r[1];
    }
    if (lanes >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = r[0] > r[1] ? r[0] : r[1];
    }
    return v;
}

constexpr float kLog2e = 1.44269504088896341f;

// exp(x) by the hardware's power of two, whose argument's rounding is 2^-24 |x log2 e| of the result.
__device__ inline float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
__device__ inline float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + exp_fast(-x)); }      // 0 and 1 at the infinities
// ln(1 + exp(x)) = max(x, 0) + ln(1 + e), e = exp(-|x|).  With w = 1 + e rounded and r = e - (w - 1), which is exact, ln(1 + e) =
// ln(w) + ln(1 + r / w); r is at most 2^-24, so that r alone is off by r e / w, 2^-24 of the value.  (For e below half a step of 1, w is 1
// and the value e.)
__device__ inline float softplus(float x) {
    const float e = exp_fast(-fabsf(x)), w = 1.f + e;
    return fmaxf(x, 0.f) + fmaf(__builtin_amdgcn_logf(w), 0.693147180559945309f, e - (w - 1.f));      // (a NaN is in e, whatever fmaxf drops)
}

}  // namespace aug
