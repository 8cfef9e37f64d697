// Device helpers of the sequence operators (gfx950, wave64).
#pragma once

#include "seq_internal.h"

namespace {

using bf16 = __bf16;
using f16 = _Float16;

// N consecutive elements as one access.  Global memory takes accesses of any
// alignment of an element, so a vector only has to lie inside its row.
template <class T, int N>
struct Vec {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <class T>
struct Vec<T, 1> {
    typedef T type;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float sigmoid(float x) {
    return rcp_fast(1.0f + exp2_fast(-kLog2e * x));
}

// softplus(x) = max(x, 0) + log(1 + e) with e = exp(-|x|), and
// log(1 + e) = 2 artanh(s), s = e / (2 + e) <= 1/3, by the artanh series:
// relative error below 1e-7 down to the smallest results, where log(1 + e)
// itself would lose the low bits of e.  sig: its derivative, sigmoid(x).
__device__ __forceinline__ float softplus(float x, float& sig) {
    const float e = exp2_fast(-kLog2e * fabsf(x));
    const float r = rcp_fast(1.0f + e);
    sig = x >= 0.0f ? r : e * r;
    const float s = e * rcp_fast(2.0f + e);
    const float q = s * s;
    float p = fmaf(q, 1.0f / 15.0f, 1.0f / 13.0f);
    p = fmaf(p, q, 1.0f / 11.0f);
    p = fmaf(p, q, 1.0f / 9.0f);
    p = fmaf(p, q, 1.0f / 7.0f);
    p = fmaf(p, q, 1.0f / 5.0f);
    p = fmaf(p, q, 1.0f / 3.0f);
    p = fmaf(p, q, 1.0f);
    return fmaf(s + s, p, fmaxf(x, 0.0f));
}

// N values of a row as they lie in memory, and as fp32.  n: how many of them
// are inside (the others read as zero).  PK: the row may be packed; N values
// that straddle two blocks have two scales.
template <class T, int N, bool PK>
struct Raw {
    static constexpr int BYTES = N * sizeof(T), WORDS = (BYTES + 3) / 4;
    union {
        typename Vec<T, N>::type v;
        T e[N];
        unsigned w[WORDS];     // packed: byte i in word i / 4
    };
    float scale[PK ? 2 : 1];
};

template <class T, int N, bool PK>
__device__ __forceinline__ void raw_load(Raw<T, N, PK>& r, const SeqT& s, long long b, long long t, int T_, int c,
                                         int n) {
    if constexpr (PK) {
        if (s.packed) {
            const long long at = (b * T_ + t) * s.row + c;
            const unsigned char* p = reinterpret_cast<const unsigned char*>(s.p) + at;
            unsigned w[(N + 3) / 4] = {};
            if (n >= N) {
                __builtin_memcpy(w, p, N);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) w[i / 4] |= (i < n ? (unsigned)p[i] : 0u) << (8 * (i % 4));
            }
#pragma unroll
            for (int i = 0; i < (N + 3) / 4; ++i) r.w[i] = w[i];
            const float* sc = s.scale + (b * T_ + t) * s.blocks;
            const int k = c / SNN_SEQ_BLOCK, split = (k + 1) * SNN_SEQ_BLOCK - c;
            r.scale[0] = n > 0 ? sc[k] : 0.0f;
            r.scale[1] = split < min(n, N) ? sc[k + 1] : r.scale[0];
            return;
        }
    }
    const T* p = reinterpret_cast<const T*>(s.p) + b * s.sample + t * s.row + c;
    if (n >= N) {
        r.v = *reinterpret_cast<const typename Vec<T, N>::type*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) r.e[i] = i < n ? p[i] : T(0.0f);
    }
}

template <class T, int N, bool PK>
__device__ __forceinline__ void raw_get(const Raw<T, N, PK>& r, const SeqT& s, int c, float (&o)[N]) {
    if constexpr (PK) {
        if (s.packed) {
            const int split = (c / SNN_SEQ_BLOCK + 1) * SNN_SEQ_BLOCK - c;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int w = (int)r.w[i / 4];
                const float x = i % 4 == 0   ? __builtin_amdgcn_cvt_f32_fp8(w, 0)
                                : i % 4 == 1 ? __builtin_amdgcn_cvt_f32_fp8(w, 1)
                                : i % 4 == 2 ? __builtin_amdgcn_cvt_f32_fp8(w, 2)
                                             : __builtin_amdgcn_cvt_f32_fp8(w, 3);
                o[i] = x * (i < split ? r.scale[0] : r.scale[1]);
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = (float)r.e[i];
}

template <class T, int N>
__device__ __forceinline__ void store_vec(const SeqT& s, long long b, long long t, int c, int n, const float (&o)[N]) {
    T* p = reinterpret_cast<T*>(s.p) + b * s.sample + t * s.row + c;
    if (n >= N) {
        if constexpr (N == 1) *p = (T)o[0];
        else {
            typename Vec<T, N>::type v;
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = (T)o[i];
            *reinterpret_cast<typename Vec<T, N>::type*>(p) = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) p[i] = (T)o[i];
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp_f32(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true));
}
// DPP controls: within quads, and within rows of 16 lanes
constexpr int kQuadXor1 = 0xB1, kQuadXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140, kRor = 0x120;

// Sum over S neighbouring lanes, in every one of them.
template <int S>
__device__ __forceinline__ float lanes_sum(float x) {
    if constexpr (S >= 2) x += dpp_f32<kQuadXor1>(x);
    if constexpr (S >= 4) x += dpp_f32<kQuadXor2>(x);
    if constexpr (S >= 8) x += dpp_f32<kHalfMirror>(x);
    if constexpr (S >= 16) x += dpp_f32<kMirror>(x);
    return x;
}

__device__ __forceinline__ int clamp_len(const int* lengths, int b, int T) {
    if (!lengths) return T;
    const int l = lengths[b];
    return l < 0 ? 0 : l > T ? T : l;
}

// A call of a template for the element type.
#define SEQ_BY_TYPE(dtype, T, ...)                      \
    do {                                                \
        if ((dtype) == SNN_F32) {                       \
            using T = float;                            \
            __VA_ARGS__;                                \
        } else if ((dtype) == SNN_BF16) {               \
            using T = bf16;                             \
            __VA_ARGS__;                                \
        } else {                                        \
            using T = f16;                              \
            __VA_ARGS__;                                \
        }                                               \
    } while (0)

}  // namespace
