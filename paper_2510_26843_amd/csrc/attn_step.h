// What kv4.hip, paged.hip and logprobs.hip share: launches, sums and maxima over
// a wave, and the attention's tile step (a wave's running softmax state, and one
// key tile's part of it).
#pragma once
#include "kernel_common.h"

#include <cfloat>

namespace cas {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// A launch that reports its own error, not an earlier call's (and without the
// call-configuration calls of the <<<>>> form: 2.35 us of the host for 2.55).
template <typename... P>
static hipError_t launch_checked(void (*kernel)(P...), dim3 grid, unsigned threads, hipStream_t s, P... args) {
    void* at[] = {(void*)&args...};
    return hipLaunchKernel((const void*)kernel, grid, dim3(threads), at, 0, s);
}

// Inclusive sum over the lanes up to one's own, by cross-lane operands: six adds
// (through LDS, as shuffles go, each step waits 100 cycles).
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_or_0(int x) {
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_or_0(float x) {
    return __uint_as_float((uint32_t)dpp_or_0<CTRL, ROWS>((int)__float_as_uint(x)));
}
template <typename V> __device__ __forceinline__ V wave_scan(V x) {
    x += dpp_or_0<0x111, 0xf>(x);  // the row's lane - 1, - 2, - 4, - 8
    x += dpp_or_0<0x112, 0xf>(x);
    x += dpp_or_0<0x114, 0xf>(x);
    x += dpp_or_0<0x118, 0xf>(x);
    x += dpp_or_0<0x142, 0xa>(x);  // the last lane of the row before, to rows 1 and 3
    x += dpp_or_0<0x143, 0xc>(x);  // lane 31, to rows 2 and 3
    return x;
}
template <typename V> __device__ __forceinline__ V wave_total(V x) {
    return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_scan(x)), 63));
}
// The largest of the lanes' values, the same for every lane (no NaN).
__device__ __forceinline__ float wave_top(float x) {
    auto up = [&](auto ctrl, auto rows) {
        const int y = __builtin_amdgcn_update_dpp((int)0xff800000, (int)__float_as_uint(x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        x = fmaxf(x, __uint_as_float((uint32_t)y));
    };
    up(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});
    up(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    up(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    up(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    up(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
    up(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), 63));
}
__device__ __forceinline__ int wave_most(int x) {  // of values >= 0
    x = max(x, dpp_or_0<0x111, 0xf>(x));
    x = max(x, dpp_or_0<0x112, 0xf>(x));
    x = max(x, dpp_or_0<0x114, 0xf>(x));
    x = max(x, dpp_or_0<0x118, 0xf>(x));
    x = max(x, dpp_or_0<0x142, 0xa>(x));
    x = max(x, dpp_or_0<0x143, 0xc>(x));
    return __builtin_amdgcn_readlane(x, 63);
}

__device__ __forceinline__ uint32_t pack_bf(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// Running softmax state of a wave for a query tile: per lane its row's
// reference score m (before scaling), the score that moves it, the factor c of its
// exponents and m c, the sum l (the same in all four elements) and O.
//
// A probability's exponent is S c less m c, fused, and as good as m c in fp32: half a
// step of it, 2^4 at a reference of ATTN_FAR, scales all of a row's probabilities
// alike.  Further out that could pass what an exponential holds, but there scores
// that differ differ by 128 or more: whatever is below the largest has a probability
// below 2^-16, and the power of two next to c, by which m goes without a rounding,
// serves.  The factor is chosen with the reference (2048 rows behind 6001 slots 209.9
// us, with one factor for all 209.1, chosen for each tile 219).
static constexpr float ATTN_FAR = 0x1p31f, ATTN_FAR_C = 0.125f;
template <int HD> struct AttnState {
    float m, top, c, mc;
    f32x4 l, O[HD / 16];
    __device__ __forceinline__ void clear() {
        m = -FLT_MAX;  // (any score that is a number passes the top)
        top = -INFINITY;
        c = ATTN_FAR_C;
        mc = m * c;
        l = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < HD / 16; ++dt) O[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
};

// Values of a pair of d tiles that are not finite, as 1.0 where they are and 0
// elsewhere; the values themselves become 0.
__device__ __forceinline__ i32x4 take_nonfinite(i32x4& v) {
    i32x4 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = (uint32_t)v[i];
        const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
        f[i] = (int)(0x3f803f80u & (lo | hi));
        v[i] = (int)(w & ~(lo | hi));
    }
    return f;
}

// Takes a row's reference score to its largest one (mt: a lane's largest of a
// tile), where that passes it by ATTN_SLACK (in log2 units): probabilities are
// then at most 2^ATTN_SLACK, which neither bf16 nor the fp32 sums mind, and the
// rescaling of O leaves most tiles' path.  The reference scales the
// probabilities before their rounding, so it takes the row's own scores only:
// what a row gives does not hang on its neighbours.
static constexpr float ATTN_SLACK = 8.f;
template <int HD> __device__ __forceinline__ void attn_follow(AttnState<HD>& st, float mt, float c) {
    const float mr = pair_max32(pair_max16(mt));
    const float mn = mr > st.top ? mr : st.m;
    const float f = __builtin_amdgcn_exp2f((st.m - mn) * c);
    st.l *= f;
#pragma unroll
    for (int dt = 0; dt < HD / 16; ++dt) st.O[dt] *= f;
    st.m = mn;
    st.top = mn + ATTN_SLACK / c;
    asm volatile("" : "+v"(st.m));  // (the rest last: moved up, it took the 2048 rows 213 us)
    st.c = fabsf(st.m) > ATTN_FAR ? ATTN_FAR_C : c;
    st.mc = st.m * st.c;
}

// The probabilities of a tile's scores (mc: the scaled reference), as the B operand of
// P V: in one bf16 term, off by 2^-8 of each, or in two, the second what the first
// leaves, off by 2^-16.
template <int TERMS>
__device__ __forceinline__ void attn_probs(i32x4 (&P)[TERMS], const f32x4 (&S)[2], float mc, float c) {
    static_assert(TERMS == 1 || TERMS == 2, "terms");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(S[i >> 1][2 * (i & 1)], c, -mc));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(S[i >> 1][2 * (i & 1) + 1], c, -mc));
        const uint32_t w = pack_bf(p0, p1);
        P[0][i] = (int)w;
        if constexpr (TERMS == 2) P[1][i] = (int)pack_bf(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xffff0000u));
    }
}

// One key tile: S are the scores of its 32 slots, V(m, f) gives the value
// fragments of d tiles 2m and 2m + 1.  next() computes the next tile's scores:
// its MFMA run while this one's probabilities and values are converted.
// MASKED: vm has the visibility of the lane's 8 slots to its row of each query
// tile; CARE: values of unseen slots may not be finite.
// The sum of the (rounded) probabilities is one more row of the PV product.
template <int HD, int JT, bool MASKED, bool CARE, int TERMS = 1, typename VF, typename NF>
__device__ __forceinline__ void attn_step(AttnState<HD> (&st)[JT], f32x4 (&S)[JT][2], float c, VF V,
                                         const uint32_t (&vm)[JT], NF next) {
    constexpr int NDT = HD / 16;
    if constexpr (MASKED) {
#pragma unroll
        for (int j = 0; j < JT; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) S[j][e >> 2][e & 3] = (vm[j] >> e) & 1u ? S[j][e >> 2][e & 3] : -INFINITY;
    }
    float mt[JT];
    bool grow = false;
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        mt[j] = S[j][0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mt[j] = fmaxf(mt[j], S[j][e >> 2][e & 3]);
        grow = grow || mt[j] > st[j].top;
    }
    if (__any(grow)) {
        mfma_result_pad();
#pragma unroll
        for (int j = 0; j < JT; ++j) attn_follow(st[j], mt[j], c);
    }
    next();
    i32x4 P[JT][TERMS];
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        attn_probs(P[j], S[j], st[j].mc, st[j].c);
        const int one = 0x3f803f80;
#pragma unroll
        for (int k = 0; k < TERMS; ++k) st[j].l = mfma_step<ET_BF16>(i32x4{one, one, one, one}, P[j][k], st[j].l);
    }
#pragma unroll
    for (int m = 0; m < NDT / 2; ++m) {
        i32x4 Vf[2];
        V(m, Vf);
        if constexpr (CARE) {
            i32x4 bad[2] = {take_nonfinite(Vf[0]), take_nonfinite(Vf[1])};
            int any = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) any |= bad[0][i] | bad[1][i];
            if (__any(any)) {  // rows that see a bad value's slot: NaN
#pragma unroll
                for (int j = 0; j < JT; ++j) {
                    i32x4 seen;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        seen[i] = (int)(((vm[j] >> (2 * i)) & 1u ? 0x3f80u : 0u) |
                                        ((vm[j] >> (2 * i + 1)) & 1u ? 0x3f800000u : 0u));
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const f32x4 n = mfma_step<ET_BF16>(bad[h], seen, f32x4{0.f, 0.f, 0.f, 0.f});
                        mfma_result_pad();
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (n[i] > 0.f) st[j].O[2 * m + h][i] = NAN;
                    }
                }
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < JT; ++j)
#pragma unroll
                for (int k = 0; k < TERMS; ++k) st[j].O[2 * m + h] = mfma_step<ET_BF16>(Vf[h], P[j][k], st[j].O[2 * m + h]);
    }
}

}  // namespace cas
