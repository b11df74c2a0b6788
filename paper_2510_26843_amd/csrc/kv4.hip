// gfx950 kernels of the 4-bit KV cache: appending rows, packing the decoder's
// bf16 cache, reading back, and tree attention.
//
// The cache quantisation of activation-quantised drafts (App. C, "(partial) KV
// cache").  Form (OCP Microscaling, E2M1 elements, blocks of 32, E8M0 scales):
// 32 consecutive elements x of a token's head row share the scale 2^e,
//   e = max(floor(log2 max|x|) - 2, -125), stored as the byte e + 127,
// and an element is the nearest of +-{0, .5, 1, 1.5, 2, 3, 4, 6} to x / 2^e,
// ties to the even code, saturating at 6.  A block with a NaN or an infinity
// has the byte 255 and reads as NaN.  Every value held is exact in bf16, so
// the cache reads as a bf16 cache of those values would: 17/64 of its bytes.
//
// A record holds 32 slots of one kv head (34 * hd bytes: key codes, value
// codes, key scales, value scales), each part in the order in which the
// attention's lanes read it (kv4_* below; MFMA operands as in kernels.hip):
//   lane (g, r) of a wave reads, in one 16-byte (hd 128; 8 at hd 64) load per
//   half s, the key codes of slot 8 (r/4) + 4 s + r%4, d = g hd/4 + [0, hd/4),
//   which lie in one block: one key scale per lane and half;
//   and in 16-byte loads the value codes of slots 8g + [0, 8) at the d of
//   block r/w (w = 512 / hd) with d % w = r % w: one scale per slot and lane,
//   and the two d of a byte are w apart, so one conversion serves two of the
//   PV product's d tiles.
// The conversion (two codes and a scale to two bf16) is one instruction.
#include "kernel_common.h"

namespace cas {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- the form

// The scale 2^(b - 127) of a scale byte; 255 gives an infinity, with which the
// conversions return NaN.
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
// Two codes (byte B of w) as a pair of bf16 values.
template <int B> __device__ __forceinline__ uint32_t kv4_pair(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}
__device__ __forceinline__ i32x4 kv4_values8(uint32_t w, float scale) {
    return i32x4{(int)kv4_pair<0>(w, scale), (int)kv4_pair<1>(w, scale), (int)kv4_pair<2>(w, scale),
                 (int)kv4_pair<3>(w, scale)};
}
// Low / high halves of two dwords side by side.
__device__ __forceinline__ uint32_t halves_lo(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t halves_hi(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Value from the quad's lane ^ 1 / ^ 2 (the four lanes of a block).
__device__ __forceinline__ uint32_t quad_xor1(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t quad_xor2(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true);
}

// Quantises a block of 32 held by a quad of lanes, 8 elements each: the lane's
// 8 codes (element 0 in the low bits) and the block's scale byte.  Scaling by
// a power of two is exact; the conversion rounds to nearest even and saturates.
__device__ __forceinline__ uint32_t kv4_quantise(const float (&x)[8], uint32_t* byte) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);  // orders magnitudes, NaN on top
    m = max(m, quad_xor1(m));
    m = max(m, quad_xor2(m));
    const bool bad = m >= 0x7f800000u;
    const int e = max((int)(m >> 23) - 129, -125);
    *byte = bad ? 255u : (uint32_t)(e + 127);
    const float s = kv4_scale((uint32_t)(e + 127));
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
    return bad ? 0u : w;
}

// Places within a record of the 8 elements d0 .. d0 + 7 (d0 a multiple of 8)
// of slot sl.
template <int HD> __device__ __forceinline__ int kv4_key_row(int sl) { return (sl >> 3) * 4 + (sl & 3); }
template <int HD> __device__ __forceinline__ int kv4_key_at(int sl, int d0) {  // 4 bytes
    const int g = d0 / (HD / 4), u = d0 % (HD / 4) / 8, s = (sl >> 2) & 1;
    return (((s * 4 + g) * 16 + kv4_key_row<HD>(sl)) * (HD / 32) + u) * 4;
}
template <int HD> __device__ __forceinline__ int kv4_key_scale_at(int sl, int b) {
    return 32 * HD + (b * 16 + kv4_key_row<HD>(sl)) * 2 + ((sl >> 2) & 1);
}
// the byte of row rr (0 .. w - 1) of the pair of d tiles m: d = 32b + w (2m + half) + rr
template <int HD> __device__ __forceinline__ int kv4_val_at(int sl, int b, int m, int rr) {
    constexpr int W = 512 / HD;
    return 16 * HD + (((m >> 1) * 4 + (sl >> 3)) * 16 + b * W + rr) * 16 + (m & 1) * 8 + (sl & 7);
}
template <int HD> __device__ __forceinline__ int kv4_val_scale_at(int sl, int b) { return 33 * HD + b * 32 + sl; }

// Writes the codes w of elements d0 .. d0 + 7 of slot sl, held by lane q of the
// block's quad, and the block's scale byte.
template <int HD, bool KEY>
__device__ __forceinline__ void kv4_put(uint8_t* rec, int sl, int d0, uint32_t w, uint32_t byte) {
    const int b = d0 >> 5, q = (d0 >> 3) & 3;
    if (KEY) {
        *(uint32_t*)(rec + kv4_key_at<HD>(sl, d0)) = w;
        if (q == 0) rec[kv4_key_scale_at<HD>(sl, b)] = (uint8_t)byte;
    } else {
        uint32_t lo, hi;  // nibbles of 4 rows each: the low and the high ones of 4 bytes
        int m, r0;
        if (HD == 128) {  // the lane's 8 elements are two d tiles of 4 rows
            lo = w;
            hi = w >> 16;
            m = q;
            r0 = 0;
        } else {  // d tile q of 8 rows; its pair is the neighbour's: rows 0-3 are the even lane's to write
            const uint32_t o = quad_xor1(w);
            lo = (q & 1) ? o >> 16 : w;
            hi = (q & 1) ? w >> 16 : o;
            m = q >> 1;
            r0 = (q & 1) * 4;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            rec[kv4_val_at<HD>(sl, b, m, r0 + i)] = (uint8_t)(((lo >> (4 * i)) & 15u) | (((hi >> (4 * i)) & 15u) << 4));
        if (q == 0) rec[kv4_val_scale_at<HD>(sl, b)] = (uint8_t)byte;
    }
}

// 8 bf16 of a row, as 16 bytes where the row allows it.
__device__ __forceinline__ i32x4 ld8_bf(const uint16_t* p, bool vec) {
    if (vec) return *(const i32x4*)p;
    i32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (int)((uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16));
    return v;
}

// ---------------------------------------------------------------- append

// One workgroup = one record (32 slots of a kv head); a quad of lanes holds a
// block, so a wave's loads run along the rows.  A record that the call fills
// whole is put together in LDS and stored 16 bytes per lane; the slots of any
// other are stored in place (4 bytes of key codes, single bytes of value
// codes), its other slots' bytes untouched: no byte belongs to two slots.
// Keys are rotated in 64 bits and rounded once to fp32, so that the code next
// to a border does not depend on how a product was fused.
static constexpr int KV4_THREADS = 256;
template <int HD> __global__ void __launch_bounds__(KV4_THREADS) k_kv4_append(const Kv4AppendArgs a) {
    constexpr int CH = HD / 8;  // 8-element pieces of a row
    __shared__ __attribute__((aligned(16))) uint8_t img[34 * HD];
    const int tile = (a.slot0 >> 5) + blockIdx.x, h = blockIdx.y;
    uint8_t* rec = a.kv4 + ((size_t)h * (a.ctx_cap >> 5) + tile) * (34 * HD);
    const int first = max(a.slot0 - tile * 32, 0), last = min(a.slot0 + a.T - tile * 32, 32);
    const bool full = first == 0 && last == 32;
    const int n_items = (last - first) * CH;  // the covered slots' pieces, of keys and of values each
    for (int it = threadIdx.x; it < 2 * n_items; it += KV4_THREADS) {
        const bool key = it < n_items;
        const int item = key ? it : it - n_items;
        const int sl = first + item / CH, d0 = item % CH * 8;
        const int t = tile * 32 + sl - a.slot0;
        float x[8];
        const uint16_t* row = key ? a.k + (size_t)t * a.ldk : a.v + (size_t)t * a.ldv;
        const i32x4 v = ld8_bf(row + h * HD + d0, a.vec);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = piece_val<uint16_t>(v, i);
        if (key && a.cos) {
            const int half = HD / 2, c0 = d0 % half;
            const i32x4 o = ld8_bf(row + h * HD + (d0 < half ? d0 + half : d0 - half), a.vec);
            const int pos = a.pos ? a.pos[t] : a.slot0 + t;
            const bool ok = pos >= 0 && pos < a.n_pos;
            const size_t at = (size_t)(ok ? pos : 0) * half + c0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double c = (double)a.cos[at + i], s = (double)a.sin[at + i];
                const double p = (double)x[i], q = (double)piece_val<uint16_t>(o, i) * s;
                const float y = (float)fma(p, c, d0 < half ? -q : q);
                x[i] = ok ? y : NAN;  // a position outside the table: the row reads as NaN
            }
        }
        uint32_t byte;
        const uint32_t w = kv4_quantise(x, &byte);
        if (full) {
            if (key) kv4_put<HD, true>(img, sl, d0, w, byte);
            else kv4_put<HD, false>(img, sl, d0, w, byte);
        } else {
            if (key) kv4_put<HD, true>(rec, sl, d0, w, byte);
            else kv4_put<HD, false>(rec, sl, d0, w, byte);
        }
    }
    if (!full) return;
    __syncthreads();
    for (int i = threadIdx.x; i < 34 * HD / 16; i += KV4_THREADS) ((i32x4*)rec)[i] = ((const i32x4*)img)[i];
}

hipError_t launch_kv4_append(const Kv4AppendArgs& a, hipStream_t s) {
    if (a.T < 1 || a.slot0 < 0 || a.slot0 > a.ctx_cap - a.T || a.Hkv < 1) return hipErrorInvalidValue;
    const dim3 grid(((a.slot0 + a.T - 1) >> 5) - (a.slot0 >> 5) + 1, a.Hkv);
    if (a.hd == 128) hipLaunchKernelGGL(k_kv4_append<128>, grid, dim3(KV4_THREADS), 0, s, a);
    else if (a.hd == 64) hipLaunchKernelGGL(k_kv4_append<64>, grid, dim3(KV4_THREADS), 0, s, a);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

// ---------------------------------------------------------------- read back

// One workgroup = one record: its bytes to LDS, its slots out as bf16 rows
// [Hkv][n][hd], 16 bytes per lane along a row.
template <int HD> __global__ void __launch_bounds__(KV4_THREADS) k_kv4_read(const Kv4ReadArgs a) {
    constexpr int CH = HD / 8;
    __shared__ __attribute__((aligned(16))) uint8_t img[34 * HD];
    const int tile = (a.slot0 >> 5) + blockIdx.x, h = blockIdx.y;
    const uint8_t* rec = a.kv4 + ((size_t)h * (a.ctx_cap >> 5) + tile) * (34 * HD);
    for (int i = threadIdx.x; i < 34 * HD / 16; i += KV4_THREADS) ((i32x4*)img)[i] = ((const i32x4*)rec)[i];
    __syncthreads();
    const int first = max(a.slot0 - tile * 32, 0), last = min(a.slot0 + a.n - tile * 32, 32);
    const int n_items = (last - first) * CH;
    for (int it = threadIdx.x; it < n_items; it += KV4_THREADS) {
        const int sl = first + it / CH, d0 = it % CH * 8, b = d0 >> 5, q = (d0 >> 3) & 3;
        const size_t o = ((size_t)h * a.n + (tile * 32 + sl - a.slot0)) * HD + d0;
        *(i32x4*)(a.k + o) = kv4_values8(*(const uint32_t*)(img + kv4_key_at<HD>(sl, d0)),
                                         kv4_scale(img[kv4_key_scale_at<HD>(sl, b)]));
        const float s = kv4_scale(img[kv4_val_scale_at<HD>(sl, b)]);
        uint32_t p[8];
#pragma unroll
        for (int i = 0; i < 512 / HD; ++i)
            p[i] = kv4_pair<0>(img[kv4_val_at<HD>(sl, b, HD == 128 ? q : q >> 1, i)], s);
        i32x4 v;
        if (HD == 128) {
            v = i32x4{(int)halves_lo(p[0], p[1]), (int)halves_lo(p[2], p[3]), (int)halves_hi(p[0], p[1]),
                      (int)halves_hi(p[2], p[3])};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = (int)((q & 1) ? halves_hi(p[2 * i], p[2 * i + 1]) : halves_lo(p[2 * i], p[2 * i + 1]));
        }
        *(i32x4*)(a.v + o) = v;
    }
}

hipError_t launch_kv4_read(const Kv4ReadArgs& a, hipStream_t s) {
    if (a.n < 1 || a.slot0 < 0 || a.slot0 > a.ctx_cap - a.n || a.Hkv < 1) return hipErrorInvalidValue;
    const dim3 grid(((a.slot0 + a.n - 1) >> 5) - (a.slot0 >> 5) + 1, a.Hkv);
    if (a.hd == 128) hipLaunchKernelGGL(k_kv4_read<128>, grid, dim3(KV4_THREADS), 0, s, a);
    else if (a.hd == 64) hipLaunchKernelGGL(k_kv4_read<64>, grid, dim3(KV4_THREADS), 0, s, a);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

// ---------------------------------------------------------------- attention

// Workgroup = (run of key tiles, kv head, JT query tiles of 16 rows); its four
// waves take the run's tiles (32 slots) in turn, each with the running maximum
// and sum of a softmax of its own, and join them through LDS at the end.
// MFMA operands as in k_attn_bf16: scores come out with slots along the row
// index, which is the k-order of P in the PV product, so probabilities stay in
// registers.  Tiles of the 4-bit cache are converted to bf16 in registers;
// the next tile's codes are loaded before the current one is used.  The
// probabilities enter the PV product as bf16, each off by at most 2^-8 of
// itself; their sum and the output stay in fp32.
//
// A tile whose slots some row does not see whole takes the masked form: the
// scores of unseen slots are replaced before use, and values that are not
// finite (an unused slot may hold anything) are taken out of the product, in
// which a probability of 0 does not hide them, and given back to the rows
// that see their slot.

template <int HD> struct Kv4Tile {  // a lane's share of a record
    uint32_t k[2][HD / 32];
    uint32_t ks;
    i32x4 v[HD / 64];
    i32x2 vs;
};
template <int HD> __device__ __forceinline__ Kv4Tile<HD> kv4_load(const uint8_t* rec, int lane) {
    const int r = lane & 15, g = lane >> 4;
    Kv4Tile<HD> t;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        if constexpr (HD == 128) {
            const i32x4 w = *(const i32x4*)(rec + (s * 64 + lane) * 16);
#pragma unroll
            for (int u = 0; u < 4; ++u) t.k[s][u] = (uint32_t)w[u];
        } else {
            const i32x2 w = *(const i32x2*)(rec + (s * 64 + lane) * 8);
            t.k[s][0] = (uint32_t)w[0];
            t.k[s][1] = (uint32_t)w[1];
        }
    }
    t.ks = *(const uint16_t*)(rec + 32 * HD + ((HD == 128 ? g : g >> 1) * 16 + r) * 2);
#pragma unroll
    for (int m = 0; m < HD / 64; ++m) t.v[m] = *(const i32x4*)(rec + 16 * HD + (m * 64 + lane) * 16);
    t.vs = *(const i32x2*)(rec + 33 * HD + (r / (512 / HD)) * 32 + 8 * g);
    return t;
}

// First d of the 4 consecutive ones that lane group g holds of d tile dt.
template <int HD> __device__ __forceinline__ int kv4_out_d(int g, int dt) {
    return HD == 128 ? 32 * g + 4 * dt : 32 * (g >> 1) + 8 * dt + 4 * (g & 1);
}

// Running softmax state of a wave for JT query tiles: per lane its row's
// maximum score m (before scaling), its own slots' share of the sum l, and O.
template <int HD, int JT> struct Kv4State {
    float m[JT], l[JT];
    f32x4 O[JT][HD / 16];
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

// One key tile: K(h2) gives the key fragments of half h2, V(m, a, b) the value
// fragments of d tiles 2m and 2m + 1.  vm: the rows' visibility of the lane's
// 8 slots, all ones where not MASKED.
template <int HD, int JT, bool MASKED, typename KF, typename VF>
__device__ __forceinline__ void kv4_step(Kv4State<HD, JT>& st, const i32x4 (&Q)[JT][HD / 32], const uint32_t (&vm)[JT],
                                         float c, KF K, VF V) {
    constexpr int UD = HD / 32, NDT = HD / 16;
    f32x4 S[JT][2];
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2) {
        i32x4 Kf[UD];
        K(h2, Kf);
#pragma unroll
        for (int j = 0; j < JT; ++j) {
            S[j][h2] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < UD; ++u) S[j][h2] = mfma_step<ET_BF16>(Kf[u], Q[j][u], S[j][h2]);
        }
    }
    float x[JT][8];
    float mn[JT];
    bool grow = false;
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        float mt = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[j][e] = S[j][e >> 2][e & 3];
            if (MASKED) x[j][e] = (vm[j] >> e) & 1u ? x[j][e] : -INFINITY;
            mt = fmaxf(mt, x[j][e]);
        }
        mn[j] = fmaxf(st.m[j], pair_max32(pair_max16(mt)));
        grow = grow || mn[j] > st.m[j];
    }
    if (__any(grow)) {
        mfma_result_pad();
#pragma unroll
        for (int j = 0; j < JT; ++j) {
            const float f = __builtin_amdgcn_exp2f((st.m[j] - mn[j]) * c);
            st.l[j] *= f;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) st.O[j][dt] *= f;
            st.m[j] = mn[j];
        }
    }
    i32x4 P[JT];
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        const float mc = st.m[j] * c;
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = __builtin_amdgcn_exp2f(fmaf(x[j][e], c, -mc));
            st.l[j] += p[e];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) P[j][i] = (int)((uint32_t)f2bf(p[2 * i]) | ((uint32_t)f2bf(p[2 * i + 1]) << 16));
    }
#pragma unroll
    for (int m = 0; m < NDT / 2; ++m) {
        i32x4 Vf[2];
        V(m, Vf[0], Vf[1]);
        if constexpr (MASKED) {
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
                        f32x4 n = mfma_step<ET_BF16>(bad[h], seen, f32x4{0.f, 0.f, 0.f, 0.f});
                        mfma_result_pad();
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (n[i] > 0.f) st.O[j][2 * m + h][i] = NAN;
                    }
                }
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < JT; ++j) st.O[j][2 * m + h] = mfma_step<ET_BF16>(Vf[h], P[j], st.O[j][2 * m + h]);
    }
}

// TAIL: where slots from n4 on are: 0 none, 1 bf16 rows [Hkv][kv_cap][hd], 2
// the decoder's bf16 cache (tiled).
template <int HD, int JT, int TAIL>
__global__ void __launch_bounds__(256) k_attn_kv4(const Kv4AttnArgs k4, float c) {
    constexpr int UD = HD / 32, DG = HD / 4, NDT = HD / 16, RS = HD + 4, W = ATT_WAVES;
    const AttnArgs& a = k4.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int S = gridDim.x, split = blockIdx.x, kvh = blockIdx.y, rc = blockIdx.z;
    const int Lc = a.sp ? a.sp->Lc : a.Lc_host, n_tree = a.sp ? a.sp->n_tree : a.n_tree_host, n_slots = Lc + n_tree;
    if (a.sp && !dcheck(a.chk, Lc >= 0 && n_slots <= a.sp->cap && a.sp->cap <= a.ctx_cap, CHK_ATTN_SLOTS)) return;
    const int n4 = a.sp ? Lc & ~31 : k4.n4, t4 = (n4 + 31) >> 5;
    const AttnWindow win(Lc, n_tree, a.win_sink, a.win_len);
    const int T = a.T, G = a.H / a.Hkv, Rp = attn_head_rows(T);
    const int nct = attn_query_tiles(T, G);
    const uint16_t* q = (const uint16_t*)a.q;

    bool rv[JT];
    uint64_t an0[JT], an1[JT];
    i32x4 Q[JT][UD];
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        const int ct = JT * rc + j, p = ct * 16 + r, hg = p / Rp, tr = p % Rp;
        rv[j] = ct < nct && hg < G && tr < T;
        const int t = min(tr, T - 1), head = kvh * G + min(hg, G - 1);
#pragma unroll
        for (int u = 0; u < UD; ++u) Q[j][u] = *(const i32x4*)(q + ((size_t)t * a.H + head) * HD + g * DG + u * 8);
        an0[j] = a.anc[2 * t];
        an1[j] = a.anc[2 * t + 1];
    }
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        if (!rv[j]) {
#pragma unroll
            for (int u = 0; u < UD; ++u) Q[j][u] = i32x4{0, 0, 0, 0};
            an0[j] = an1[j] = 0ull;
        }
    }
    Kv4State<HD, JT> st;
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        st.m[j] = -1e30f;
        st.l[j] = 0.f;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) st.O[j][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // logical tiles [lt0, lt1) of this workgroup; the 4-bit ones come first
    const int lt0 = (int)((long)win.n_log * split / S), lt1 = (int)((long)win.n_log * (split + 1) / S);
    auto whole = [&](int pt) {  // every row sees every slot of the tile
        const int b = pt * 32;
        return b + 32 <= win.csink || (b >= win.wstart && b + 32 <= Lc);
    };
    auto masks = [&](int pt, uint32_t (&vm)[JT]) {
#pragma unroll
        for (int j = 0; j < JT; ++j) vm[j] = attn_vis8(pt * 32 + 8 * g, Lc, n_slots, win, an0[j], an1[j]);
    };
    const uint8_t* rec0 = k4.kv4 + (size_t)kvh * (a.ctx_cap >> 5) * (34 * HD);
    int lt = lt0 + wave;
    auto in4 = [&](int l) { return l < lt1 && win.phys(l) < t4; };
    auto step4 = [&](const Kv4Tile<HD>& t, int pt) {
        auto K = [&](int h2, i32x4 (&Kf)[UD]) {
            const float s = kv4_scale((t.ks >> (8 * h2)) & 0xffu);
#pragma unroll
            for (int u = 0; u < UD; ++u) Kf[u] = kv4_values8(t.k[h2][u], s);
        };
        float vs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) vs[e] = kv4_scale(((uint32_t)t.vs[e >> 2] >> (8 * (e & 3))) & 0xffu);
        auto V = [&](int m, i32x4& va, i32x4& vb) {
            const uint32_t w0 = (uint32_t)t.v[m >> 1][2 * (m & 1)], w1 = (uint32_t)t.v[m >> 1][2 * (m & 1) + 1];
            const uint32_t p[8] = {kv4_pair<0>(w0, vs[0]), kv4_pair<1>(w0, vs[1]), kv4_pair<2>(w0, vs[2]),
                                   kv4_pair<3>(w0, vs[3]), kv4_pair<0>(w1, vs[4]), kv4_pair<1>(w1, vs[5]),
                                   kv4_pair<2>(w1, vs[6]), kv4_pair<3>(w1, vs[7])};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                va[i] = (int)halves_lo(p[2 * i], p[2 * i + 1]);
                vb[i] = (int)halves_hi(p[2 * i], p[2 * i + 1]);
            }
        };
        uint32_t vm[JT];
        if (whole(pt)) {
            kv4_step<HD, JT, false>(st, Q, vm, c, K, V);
        } else {
            masks(pt, vm);
            kv4_step<HD, JT, true>(st, Q, vm, c, K, V);
        }
    };
    if (in4(lt)) {
        Kv4Tile<HD> cur = kv4_load<HD>(rec0 + (size_t)win.phys(lt) * (34 * HD), lane);
        while (true) {
            const int nx = lt + W;
            const bool more = in4(nx);
            const Kv4Tile<HD> next = kv4_load<HD>(rec0 + (size_t)win.phys(more ? nx : lt) * (34 * HD), lane);
            step4(cur, win.phys(lt));
            lt = nx;
            if (!more) break;
            cur = next;
        }
        mfma_result_pad();
    }
    if constexpr (TAIL != 0) {
        for (; lt < lt1; lt += W) {
            const int pt = win.phys(lt);
            uint32_t vm[JT];
            masks(pt, vm);
            const uint16_t *kt, *vt;
            if constexpr (TAIL == 1) {
                kt = k4.kr + (size_t)kvh * k4.kv_cap * HD;
                vt = k4.vr + (size_t)kvh * k4.kv_cap * HD;
            } else {
                kt = (const uint16_t*)a.kc + ((size_t)kvh * a.ctx_cap + pt * 32) * HD;
                vt = (const uint16_t*)a.vt + ((size_t)kvh * a.ctx_cap + pt * 32) * HD;
            }
            auto row = [&](int sl) { return (size_t)(min(pt * 32 + sl, n_slots - 1) - n4) * HD; };
            auto K = [&](int h2, i32x4 (&Kf)[UD]) {
#pragma unroll
                for (int u = 0; u < UD; ++u) {
                    if constexpr (TAIL == 1) Kf[u] = *(const i32x4*)(kt + row(8 * (r >> 2) + 4 * h2 + (r & 3)) + g * DG + u * 8);
                    else Kf[u] = *(const i32x4*)(kt + (h2 * UD + u) * 512 + lane * 8);
                }
            };
            auto V = [&](int m, i32x4& va, i32x4& vb) {
                constexpr int WR = 512 / HD;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int d = 32 * (r / WR) + WR * (2 * m + h) + r % WR;
                    i32x4 f;
                    if constexpr (TAIL == 1) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            f[i] = (int)((uint32_t)vt[row(8 * g + 2 * i) + d] | ((uint32_t)vt[row(8 * g + 2 * i + 1) + d] << 16));
                    } else {
                        f = *(const i32x4*)(vt + ((d >> 4) * 64 + g * 16 + (d & 15)) * 8);
                    }
                    if (h == 0) va = f;
                    else vb = f;
                }
            };
            kv4_step<HD, JT, true>(st, Q, vm, c, K, V);
        }
        mfma_result_pad();
    }

    // ---- join the four waves, one query tile after another
    __shared__ float sm_m[W][16], sm_l[W][16];
    __shared__ __attribute__((aligned(16))) float sm_o[W][16][RS];
    constexpr int D4 = HD / 4;
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        const float l = pair_sum32(pair_sum16(st.l[j]));
        if (j) __syncthreads();
        if (g == 0) {
            sm_m[wave][r] = st.m[j] * c;
            sm_l[wave][r] = l;
        }
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) *(f32x4*)(&sm_o[wave][r][kv4_out_d<HD>(g, dt)]) = st.O[j][dt];
        __syncthreads();
        for (int idx = threadIdx.x; idx < 16 * D4; idx += 64 * W) {
            const int rr = idx / D4, d4 = (idx % D4) * 4;
            const int ct = JT * rc + j, p = ct * 16 + rr, hg = p / Rp, t = p % Rp;
            if (ct >= nct || hg >= G || t >= T) continue;
            float mw[W], M = -INFINITY;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                mw[w] = sm_m[w][rr];
                M = fmaxf(M, mw[w]);
            }
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            float L = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float f = attn_merge_weight(mw[w], M);
                attn_merge_o(acc, *(const f32x4*)(&sm_o[w][rr][d4]), f);
                attn_merge_l(L, sm_l[w][rr], f);
            }
            if (k4.direct) {
                const float inv = L != 0.f ? 1.f / L : 0.f;  // no slot seen: 0 (a NaN sum stays one)
                st4((uint16_t*)a.out, (size_t)t * a.H * HD + (kvh * G + hg) * HD + d4, acc[0] * inv, acc[1] * inv,
                    acc[2] * inv, acc[3] * inv);
            } else {
                const size_t o = ((size_t)split * a.H + kvh * G + hg) * T + t;
                *(f32x4*)(a.part_o + o * HD + d4) = acc;
                if (d4 == 0) *(float2*)(a.part_ml + o * 2) = make_float2(M, L);
            }
        }
    }
}

static int kv4_jt(int T, int G) {
    const int nct = attn_query_tiles(T, G);
    return nct >= 2 ? 2 : 1;
}

int kv4_attention_splits(int Lc, int n_tree, int T, int H, int Hkv, int win_sink, int win_len) {
    const int n_log = AttnWindow(Lc, n_tree, win_sink, win_len).n_log;
    const int G = H / Hkv, jt = kv4_jt(T, G), z = (attn_query_tiles(T, G) + jt - 1) / jt;
    const int most = (n_log + 2 * ATT_WAVES - 1) / (2 * ATT_WAVES);  // two tiles per wave
    const int want = (1024 + Hkv * z - 1) / (Hkv * z);
    return max(1, min(min(most, want), ATT_MAX_SPLITS));
}

template <int HD, int JT> static hipError_t attn_kv4_go(const Kv4AttnArgs& k, dim3 grid, int tail, float c, hipStream_t s) {
    if (tail == 0) hipLaunchKernelGGL((k_attn_kv4<HD, JT, 0>), grid, dim3(64 * ATT_WAVES), 0, s, k, c);
    else if (tail == 1) hipLaunchKernelGGL((k_attn_kv4<HD, JT, 1>), grid, dim3(64 * ATT_WAVES), 0, s, k, c);
    else hipLaunchKernelGGL((k_attn_kv4<HD, JT, 2>), grid, dim3(64 * ATT_WAVES), 0, s, k, c);
    return hipGetLastError();
}

hipError_t launch_attention_kv4(const Kv4AttnArgs& k, hipStream_t s) {
    const AttnArgs& a = k.a;
    if (a.T < 1 || a.T > 128 || a.Hkv < 1 || a.H % a.Hkv || a.ctx_cap % 32) return hipErrorInvalidValue;
    const int G = a.H / a.Hkv, jt = kv4_jt(a.T, G), nct = attn_query_tiles(a.T, G);
    const int S = kv4_attention_splits(a.Lc_host, a.n_tree_host, a.T, a.H, a.Hkv, a.win_sink, a.win_len);
    const dim3 grid(S, a.Hkv, (nct + jt - 1) / jt);
    // (the decoder's whole-tile copy always leaves slots to its bf16 cache)
    const int tail = a.sp ? 2 : k.n4 < a.Lc_host + a.n_tree_host ? 1 : 0;
    const float c = (1.0f / sqrtf((float)a.hd)) * 1.4426950408889634f;
    Kv4AttnArgs k2 = k;
    k2.direct = S == 1 && !a.out_tiled && !a.qout && !a.no_merge;
    hipError_t e = hipErrorInvalidValue;
    if (a.hd == 128)
        e = jt == 2 ? attn_kv4_go<128, 2>(k2, grid, tail, c, s) : attn_kv4_go<128, 1>(k2, grid, tail, c, s);
    else if (a.hd == 64)
        e = jt == 2 ? attn_kv4_go<64, 2>(k2, grid, tail, c, s) : attn_kv4_go<64, 1>(k2, grid, tail, c, s);
    if (e != hipSuccess || k2.direct || a.no_merge) return e;
    return launch_attn_merge(a, S, s);
}

}  // namespace cas
