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
//   half s, the key codes of slot 8 (r/4) + 4 s + r%4, d = g hd/4 + [0, hd/4):
//   with the block's scale (one per lane and half) an operand of the scaled
//   MFMA as it stands, the keys are never converted;
//   and in 16-byte loads the value codes of slots 8g + [0, 8) at the d of
//   block r/w (w = 512 / hd) with d % w = r % w: one scale per slot and lane,
//   and the two d of a byte are w apart, so one conversion (two codes and a
//   scale to two bf16, one instruction) serves two of the PV product's d tiles.
#include "attn_step.h"

namespace cas {

typedef unsigned short uint16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- the form

// The scale 2^(b - 127) of a scale byte; 255 gives an infinity, with which the
// conversions return NaN.
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
// The scale of byte e of a dword for a conversion, which takes the exponent
// field alone: sign and mantissa are the neighbours' bits.
__device__ __forceinline__ float kv4_scale_of(uint32_t w, int e) {
    return __uint_as_float(e < 3 ? w << (23 - 8 * e) : w >> 1);
}
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

// Writes the key codes w of elements d0 .. d0 + 7 of slot sl and, from a
// block's first piece, its scale byte.
template <int HD> __device__ __forceinline__ void kv4_put_key(uint8_t* rec, int sl, int d0, uint32_t w, uint32_t byte) {
    *(uint32_t*)(rec + kv4_key_at<HD>(sl, d0)) = w;
    if ((d0 & 31) == 0) rec[kv4_key_scale_at<HD>(sl, d0 >> 5)] = (uint8_t)byte;
}
// The slot that byte o of a record belongs to.
template <int HD> __device__ __forceinline__ int kv4_slot_of(int o) {
    if (o < 16 * HD) {
        const int lane = o / (HD / 8);  // s, g, row
        return ((lane >> 2) & 3) * 8 + (lane >> 6) * 4 + (lane & 3);
    }
    if (o < 32 * HD) return ((o >> 8) & 3) * 8 + (o & 7);  // (16 HD is a multiple of 1024)
    if (o < 33 * HD) return ((o >> 3) & 3) * 8 + (o & 1) * 4 + ((o >> 1) & 3);
    return o & 31;
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

// One workgroup = one record (32 slots of a kv head).  Keys are rotated in 64
// bits and rounded once to fp32, so that the code next to a border does not
// depend on how a product was fused.
//
// Waves 0 and 1 take the record's keys, a lane two pieces of 8 elements hd/2
// apart (a rotation's two halves); waves 2 and 3 its values, a lane one piece
// of four consecutive slots, whose codes it turns into the record's order (4
// slots to a dword) with byte permutations.  All loads are issued first and
// run along the rows; the record is put together in LDS and stored 16 bytes
// per lane, or, where the call covers some of its slots only, by dwords and
// bytes of those (no byte belongs to two slots; the rows of the others are
// stand-ins).  Records of which it covers at most KV4_FEW slots take a shorter
// way, one piece per lane stored in place: one token's append 2.5 us against
// 4.4, 28 slots of a record 5.0 against 4.5.
static constexpr int KV4_THREADS = 256;

template <int HD>
__device__ __forceinline__ void kv4_rotate(const float* cos, const float* sin, size_t at, bool ok, float (&x)[8],
                                           float (&o)[8]) {  // pieces d0 .. and d0 + hd/2 .. of a row
    const f32x4 cs[2] = {*(const f32x4*)(cos + at), *(const f32x4*)(cos + at + 4)};
    const f32x4 sn[2] = {*(const f32x4*)(sin + at), *(const f32x4*)(sin + at + 4)};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double c = (double)cs[i >> 2][i & 3], s = (double)sn[i >> 2][i & 3], a = (double)x[i], b = (double)o[i];
        x[i] = ok ? (float)fma(a, c, -(b * s)) : NAN;  // a position outside the table: the row reads as NaN
        o[i] = ok ? (float)fma(b, c, a * s) : NAN;
    }
}

// A record of a tile's rows in LDS.  SRC: rows k(sl, d0) of 8 key elements, v4(s4,
// d0, x) of four slots' 8 value elements, and rot(sl, d0, x, y), which turns the
// keys' pieces at d0 and d0 + hd/2.
template <int HD, typename K, typename V, typename R>
__device__ __forceinline__ void kv4_record(uint8_t* img, K k, V v4, R rot) {
    constexpr int CH = HD / 8;
    const int tid = threadIdx.x;
    if (tid < 128) {
        constexpr int PR = CH / 2, NK = 32 * PR / 128;  // pairs of pieces per row, and per thread
        i32x4 lo[NK], hi[NK];
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int item = i * 128 + tid;
            lo[i] = k(item / PR, item % PR * 8);
            hi[i] = k(item / PR, item % PR * 8 + HD / 2);
        }
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int item = i * 128 + tid, sl = item / PR, d0 = item % PR * 8;
            float x[8], y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = piece_val<uint16_t>(lo[i], e);
                y[e] = piece_val<uint16_t>(hi[i], e);
            }
            rot(sl, d0, x, y);
            uint32_t byte;
            uint32_t w = kv4_quantise(x, &byte);
            kv4_put_key<HD>(img, sl, d0, w, byte);
            w = kv4_quantise(y, &byte);
            kv4_put_key<HD>(img, sl, d0 + HD / 2, w, byte);
        }
    } else if (tid < 128 + 8 * CH) {
        const int item = tid - 128, d0 = item % CH * 8, s4 = item / CH * 4;  // slots s4 .. s4 + 3
        float x[4][8];
        v4(s4, d0, x);
        const int b = d0 >> 5, q = (d0 >> 3) & 3;
        uint32_t e[4], o[4], scales = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t byte;
            uint32_t w = kv4_quantise(x[j], &byte);
            scales |= byte << (8 * j);
            if (HD == 64) {  // a d tile's 8 rows pair with the neighbour's: rows 0-3 to the even lane
                const uint32_t n = quad_xor1(w);
                w = (q & 1) ? (n >> 16) | (w & 0xffff0000u) : (w & 0xffffu) | (n << 16);
            }
            // codes n0 .. n7 to the bytes n0 | n4 << 4, n2 | n6 << 4 (e) and n1 | n5 << 4, n3 | n7 << 4 (o)
            e[j] = w & 0x0f0f0f0fu;
            o[j] = (w >> 4) & 0x0f0f0f0fu;
            e[j] |= e[j] >> 12;
            o[j] |= o[j] >> 12;
        }
        const int m = HD == 128 ? q : q >> 1, r0 = HD == 128 ? 0 : (q & 1) * 4;
        uint32_t four[4];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            const uint32_t* p = z ? o : e;
            const uint32_t a01 = __builtin_amdgcn_perm(p[1], p[0], 0x05010400u);  // bytes 0 of both, bytes 1 of both
            const uint32_t a23 = __builtin_amdgcn_perm(p[3], p[2], 0x05010400u);
            four[z] = halves_lo(a01, a23);
            four[2 + z] = halves_hi(a01, a23);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) *(uint32_t*)(img + kv4_val_at<HD>(s4, b, m, r0 + i)) = four[i];
        if (q == 0) *(uint32_t*)(img + kv4_val_scale_at<HD>(s4, b)) = scales;
    }
}

static constexpr int KV4_FEW = 8;  // pieces of 8 slots' keys and values: one per thread
template <int HD>
__device__ __forceinline__ void kv4_pieces(const Kv4AppendArgs& a, int tile, int h, int first, int last, uint8_t* rec) {
    constexpr int CH = HD / 8;
    const int n_items = (last - first) * CH, it = threadIdx.x;
    if (it >= 2 * n_items) return;
    const bool key = it < n_items;
    const int item = key ? it : it - n_items;
    const int sl = first + item / CH, d0 = item % CH * 8, t = tile * 32 + sl - a.slot0;
    const uint16_t* row = (key ? a.k + (size_t)t * a.ldk : a.v + (size_t)t * a.ldv) + h * HD;
    const i32x4 v = ld8_bf(row + d0, a.vec);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = piece_val<uint16_t>(v, i);
    if (key && a.cos) {
        const bool low = d0 < HD / 2;
        const i32x4 o = ld8_bf(row + (low ? d0 + HD / 2 : d0 - HD / 2), a.vec);
        const int pos = a.pos ? a.pos[t] : a.slot0 + t;
        const bool ok = pos >= 0 && pos < a.n_pos;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = piece_val<uint16_t>(o, i);
        const size_t at = (size_t)(ok ? pos : 0) * (HD / 2) + d0 % (HD / 2);
        if (low) kv4_rotate<HD>(a.cos, a.sin, at, ok, x, y);
        else kv4_rotate<HD>(a.cos, a.sin, at, ok, y, x);
    }
    uint32_t byte;
    const uint32_t w = kv4_quantise(x, &byte);
    const uint32_t n = quad_xor1(w);  // (the quads' lanes are here together)
    if (key) {
        kv4_put_key<HD>(rec, sl, d0, w, byte);
        return;
    }
    const int b = d0 >> 5, q = (d0 >> 3) & 3;
    // 4 bytes' low and high codes, as in kv4_record
    const uint32_t lo = HD == 128 ? w : (q & 1) ? n >> 16 : w, hi = HD == 128 ? w >> 16 : (q & 1) ? w >> 16 : n;
    const int m = HD == 128 ? q : q >> 1, r0 = HD == 128 ? 0 : (q & 1) * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        rec[kv4_val_at<HD>(sl, b, m, r0 + i)] = (uint8_t)(((lo >> (4 * i)) & 15u) | (((hi >> (4 * i)) & 15u) << 4));
    if (q == 0) rec[kv4_val_scale_at<HD>(sl, b)] = (uint8_t)byte;
}

template <int HD> __global__ void __launch_bounds__(KV4_THREADS) k_kv4_append(const Kv4AppendArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t img[34 * HD];
    const int tile = (a.slot0 >> 5) + blockIdx.x, h = blockIdx.y;
    uint8_t* rec = a.kv4 + ((size_t)h * (a.ctx_cap >> 5) + tile) * (34 * HD);
    const int first = max(a.slot0 - tile * 32, 0), last = min(a.slot0 + a.T - tile * 32, 32);
    if (last - first <= KV4_FEW) {
        kv4_pieces<HD>(a, tile, h, first, last, rec);
        return;
    }
    auto row = [&](int sl) { return (size_t)min(max(tile * 32 + sl - a.slot0, 0), a.T - 1); };
    kv4_record<HD>(
        img, [&](int sl, int d0) { return ld8_bf(a.k + row(sl) * a.ldk + h * HD + d0, a.vec); },
        [&](int s4, int d0, float (&x)[4][8]) {
            i32x4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = ld8_bf(a.v + row(s4 + j) * a.ldv + h * HD + d0, a.vec);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j][e] = piece_val<uint16_t>(v[j], e);
        },
        [&](int sl, int d0, float (&x)[8], float (&y)[8]) {
            if (!a.cos) return;
            const int pos = a.pos ? a.pos[row(sl)] : tile * 32 + sl;
            const bool ok = pos >= 0 && pos < a.n_pos;
            kv4_rotate<HD>(a.cos, a.sin, (size_t)(ok ? pos : 0) * (HD / 2) + d0, ok, x, y);
        });
    __syncthreads();
    if (first == 0 && last == 32) {
        for (int i = threadIdx.x; i < 34 * HD / 16; i += KV4_THREADS) ((i32x4*)rec)[i] = ((const i32x4*)img)[i];
        return;
    }
    for (int o = 4 * threadIdx.x; o < 34 * HD; o += 4 * KV4_THREADS) {
        bool in[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int sl = kv4_slot_of<HD>(o + i);
            in[i] = sl >= first && sl < last;
        }
        if (in[0] && in[1] && in[2] && in[3]) {
            *(uint32_t*)(rec + o) = *(const uint32_t*)(img + o);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (in[i]) rec[o + i] = img[o + i];
        }
    }
}

hipError_t launch_kv4_append(const Kv4AppendArgs& a, hipStream_t s) {
    if (a.T < 1 || a.slot0 < 0 || a.slot0 > a.ctx_cap - a.T || a.Hkv < 1) return hipErrorInvalidValue;
    const dim3 grid(((a.slot0 + a.T - 1) >> 5) - (a.slot0 >> 5) + 1, a.Hkv);
    if (a.hd == 128) return launch_checked(k_kv4_append<128>, grid, KV4_THREADS, s, a);
    if (a.hd == 64) return launch_checked(k_kv4_append<64>, grid, KV4_THREADS, s, a);
    return hipErrorInvalidValue;
}

// Records tile0 .. tile0 + gridDim.x - 1 of every (layer, kv head) from the
// decoder's bf16 cache (whole 32-slot tiles; its keys are rotated).
template <int HD>
__global__ void __launch_bounds__(KV4_THREADS) k_kv4_pack(const uint16_t* kc, const uint16_t* vt, int ctx_cap, int tile0,
                                                          uint8_t* kv4) {
    __shared__ __attribute__((aligned(16))) uint8_t img[34 * HD];
    const int tile = tile0 + blockIdx.x;
    const size_t src = ((size_t)blockIdx.y * ctx_cap + (size_t)tile * 32) * HD;
    kv4_record<HD>(
        img, [&](int sl, int d0) { return *(const i32x4*)(kc + src + kv_k_tiled(sl, d0, HD)); },
        [&](int s4, int d0, float (&x)[4][8]) {
            i32x2 v[8];  // four slots at a d are 8 bytes
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = *(const i32x2*)(vt + src + kv_v_tiled(s4, d0 + e, HD));
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t w = (uint32_t)v[e][j >> 1];
                    x[j][e] = __uint_as_float((j & 1) ? (w & 0xffff0000u) : (w << 16));
                }
        },
        [](int, int, float (&)[8], float (&)[8]) {});
    __syncthreads();
    i32x4* rec = (i32x4*)(kv4 + ((size_t)blockIdx.y * (ctx_cap >> 5) + tile) * (34 * HD));
    for (int i = threadIdx.x; i < 34 * HD / 16; i += KV4_THREADS) rec[i] = ((const i32x4*)img)[i];
}

hipError_t launch_kv4_pack(const void* kc, const void* vt, int heads, int hd, int ctx_cap, int tile0, int tiles,
                           uint8_t* kv4, hipStream_t s) {
    if (tiles < 1 || tile0 < 0 || tile0 + tiles > ctx_cap >> 5 || heads < 1 || heads > 65535) return hipErrorInvalidValue;
    const dim3 grid(tiles, heads);
    const uint16_t *k = (const uint16_t*)kc, *v = (const uint16_t*)vt;
    if (hd == 128) return launch_checked(k_kv4_pack<128>, grid, KV4_THREADS, s, k, v, ctx_cap, tile0, kv4);
    if (hd == 64) return launch_checked(k_kv4_pack<64>, grid, KV4_THREADS, s, k, v, ctx_cap, tile0, kv4);
    return hipErrorInvalidValue;
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
    if (a.hd == 128) return launch_checked(k_kv4_read<128>, grid, KV4_THREADS, s, a);
    if (a.hd == 64) return launch_checked(k_kv4_read<64>, grid, KV4_THREADS, s, a);
    return hipErrorInvalidValue;
}

// ---------------------------------------------------------------- attention

// Workgroup = (run of key tiles, kv head, JT query tiles of 16 rows); its eight
// waves share the run's tiles (32 slots), each with the running maximum and sum
// of a softmax of its own, and join them through LDS at the end.  The scores
// come out of the scaled MFMA with slots along the row index, which is the
// k-order of P in the PV product (on bf16 MFMA, its values converted in
// registers), so probabilities stay in registers.  They enter that product as
// bf16, each off by at most 2^-8 of itself; their sum, which is of the rounded
// ones, and the output stay in fp32.  The output's error is 0.0023 of its norm
// (0.0017 is its own rounding), the cache's quantisation 0.1.  With the rest of
// each as a second bf16 term, as in k_attn_bf16, it is 0.0017, and 128 rows of
// 8B heads over 16001 slots take 48.3 us for 38.5, 64 rows of 13B heads over
// 2048 10.8 for 9.6, one row over 131071 31.8 for 31.1.  One fp16 term (2^-11)
// ends at 2^-31 of a row's largest, and the sums over the others would miss it.
//
// Whole tiles, which every row sees, are a wave's main loop: a ring of three
// tiles' codes in registers, loaded two steps ahead, the next tile's scores
// issued under this one's exponentials and conversions.  The others, the edge
// tiles (Kv4Tiles), take the masked form and are spread over the waves first:
// the scores of unseen slots are replaced before use, and values that are not
// finite (an unused slot may hold anything) are taken out of the product, in
// which a probability of 0 does not hide them, and given back to the rows that
// see their slot.
//
// What bounds it: for few rows the bytes (one row of 8B heads over 131072
// slots: 142.6 MB in 27 us, and 4 to join); for many the vector unit and the
// matrix cores, which take turns (128 rows of 8B heads over 16001 slots: 33.7
// GFLOP in 39.7 us, 850 TFLOP/s, 69% and 34% busy): per tile and query tile 8
// exponentials a lane at twice an instruction's cost, 4 conversions of P, and
// at hd 128 32 of the values' codes and 32 to bring the two d tiles apart,
// shared by JT; for short calls the launch, the query's conversion and the two
// joins.

template <int HD> struct Kv4Tile {  // a lane's share of a record
    uint32_t k[2][HD / 32];
    uint32_t ks;
    i32x4 v[HD / 64];
    i32x2 vs;
};
// A kv head's records, loaded through a buffer descriptor: a tile's place is a
// scalar, a lane's places in a record are constants of the wave, so that a load
// costs the vector unit nothing (with 64-bit addresses 10 instructions a tile:
// 64 rows of 13B heads over 2048 slots 9.9 us, 9.55 so).
template <int HD> struct Kv4Records {
    __amdgpu_buffer_rsrc_t rec;
    int key, val, ks, vs;
    __device__ __forceinline__ Kv4Records(const uint8_t* head, int tiles, int lane) {
        const int r = lane & 15, g = lane >> 4;
        // (the last word: 32-bit data, which untyped loads ignore but for its being valid)
        rec = __builtin_amdgcn_make_buffer_rsrc((void*)head, 0, tiles * (34 * HD), 0x27000);
        key = lane * (HD / 8);
        val = 16 * HD + lane * 16;
        ks = 32 * HD + ((HD == 128 ? g : g >> 1) * 16 + r) * 2;
        vs = 33 * HD + (r / (512 / HD)) * 32 + 8 * g;
    }
    __device__ __forceinline__ Kv4Tile<HD> load(int tile) const {
        const int at = tile * (34 * HD);
        Kv4Tile<HD> t;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if constexpr (HD == 128) {
                const auto w = __builtin_amdgcn_raw_buffer_load_b128(rec, key + s * 64 * 16, at, 0);
#pragma unroll
                for (int u = 0; u < 4; ++u) t.k[s][u] = w[u];
            } else {
                const auto w = __builtin_amdgcn_raw_buffer_load_b64(rec, key + s * 64 * 8, at, 0);
                t.k[s][0] = w[0];
                t.k[s][1] = w[1];
            }
        }
        t.ks = __builtin_amdgcn_raw_buffer_load_b16(rec, ks, at, 0);
#pragma unroll
        for (int m = 0; m < HD / 64; ++m)
            t.v[m] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rec, val + m * 64 * 16, at, 0));
        t.vs = __builtin_bit_cast(i32x2, __builtin_amdgcn_raw_buffer_load_b64(rec, vs, at, 0));
        return t;
    }
};

// First d of the 4 consecutive ones that lane group g holds of d tile dt.
template <int HD> __device__ __forceinline__ int kv4_out_d(int g, int dt) {
    return HD == 128 ? 32 * g + 4 * dt : 32 * (g >> 1) + 8 * dt + 4 * (g & 1);
}

// The query rows of a tile as the B operand of the scaled MFMA, whose A operand
// a record's key codes and scales are as they stand (16 x 16 x 128; block kg
// of its k, 32 wide, is d = 32 kg + [0, 32) at hd 128, and d = 16 kg + [0, 16)
// and zeros at hd 64).  A row is the sum of two fp8 (e4m3) rows, in each block
// hi at scale 2^s and lo at 2^(s - 5), with the block's largest element in
// [2^7, 2^8) 2^s: hi and lo have four significant bits each, which is bf16's
// eight, so the sum is exact but for elements below 2^-15 of the block's
// largest, which are off by at most 2^-22 of it.  Two of these MFMA per half
// tile take the place of the keys' conversion (32 of a tile's instructions at
// hd 128) and four bf16 ones.
// Lane (g, r) holds row r's k = 16 g + [0, 16) and 64 + 16 g + [0, 16), and the
// scale of block g.  The workgroup's threads convert 8 elements each and hand
// them over in LDS (every wave converting for itself took 1 us more).
template <int HD> struct Kv4Query {
    i32x8 hi, lo;
    int sh, sl;
    // scores of half HALF of a record's slots (codes k, scale byte HALF of ks), in two parts
    template <int HALF> __device__ __forceinline__ f32x4 hi_scores(const i32x8 k, int ks) const {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, hi, f32x4{0.f, 0.f, 0.f, 0.f}, 4, 0, HALF, ks, 0, sh);
    }
    template <int HALF> __device__ __forceinline__ f32x4 lo_scores(const i32x8 k, int ks, f32x4 c) const {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, lo, c, 4, 0, HALF, ks, 0, sl);
    }
};
struct Kv4QueryLds {  // of one tile
    __attribute__((aligned(16))) uint8_t hi[4][16][32], lo[4][16][32];
    uint8_t scale[4][16];
};
// Piece `part` of block kg of row r: 8 elements v (16 bytes of bf16) of a
// block held by HD / 32 neighbouring lanes.
template <int HD> __device__ __forceinline__ void kv4_query_put(Kv4QueryLds& q, int r, int kg, int part, i32x4 v) {
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = max(m, max(((uint32_t)v[w] << 16) & 0x7fff0000u, (uint32_t)v[w] & 0x7fff0000u));
    m = max(m, quad_xor1(m));
    if (HD == 128) m = max(m, quad_xor2(m));
    const bool bad = m >= 0x7f800000u;  // not finite: the row's scores are NaN
    const int s = max((int)(m >> 23) - 134, -120);
    const float down = __uint_as_float((uint32_t)(127 - s) << 23);
    int h[2], l[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = bad ? 0.f : piece_val<uint16_t>(v, 4 * w + e) * down;
        h[w] = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
        h[w] = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], h[w], true);
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(h[w], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(h[w], true);
        l[w] = __builtin_amdgcn_cvt_pk_fp8_f32((x[0] - a[0]) * 32.f, (x[1] - a[1]) * 32.f, 0, false);
        l[w] = __builtin_amdgcn_cvt_pk_fp8_f32((x[2] - b[0]) * 32.f, (x[3] - b[1]) * 32.f, l[w], true);
    }
    const int k = 32 * kg + 8 * part, g = k % 64 / 16, at = k / 64 * 16 + k % 16;
    *(i32x2*)(&q.hi[g][r][at]) = i32x2{h[0], h[1]};
    *(i32x2*)(&q.lo[g][r][at]) = i32x2{l[0], l[1]};
    if (part == 0) q.scale[kg][r] = bad ? 255 : (uint8_t)(s + 127);
}
template <int HD> __device__ __forceinline__ Kv4Query<HD> kv4_query_get(const Kv4QueryLds& q, int g, int r) {
    Kv4Query<HD> x{};
    if (HD == 128 || !(g & 1)) {  // (hd 64: the other lanes' k are the zeros)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const i32x4 a = *(const i32x4*)(&q.hi[g][r][16 * h]), b = *(const i32x4*)(&q.lo[g][r][16 * h]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x.hi[4 * h + i] = a[i];
                x.lo[4 * h + i] = b[i];
            }
        }
    }
    x.sh = q.scale[g][r];
    x.sl = x.sh == 255 ? 255 : x.sh - 5;
    return x;
}

// The scores of a tile of the 4-bit cache, and its step.
template <int HD, int JT>
__device__ __forceinline__ void kv4_scores(f32x4 (&S)[JT][2], const Kv4Tile<HD>& t, const Kv4Query<HD> (&Q)[JT]) {
    i32x8 k0 = {}, k1 = {};
#pragma unroll
    for (int u = 0; u < HD / 32; ++u) {
        k0[u] = (int)t.k[0][u];
        k1[u] = (int)t.k[1][u];
    }
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        S[j][0] = Q[j].template hi_scores<0>(k0, (int)t.ks);
        S[j][1] = Q[j].template hi_scores<1>(k1, (int)t.ks);
    }
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        S[j][0] = Q[j].template lo_scores<0>(k0, (int)t.ks, S[j][0]);
        S[j][1] = Q[j].template lo_scores<1>(k1, (int)t.ks, S[j][1]);
    }
}
template <int HD, int JT, bool MASKED, bool CARE, typename NF>
__device__ __forceinline__ void kv4_step4(AttnState<HD> (&st)[JT], f32x4 (&S)[JT][2], const Kv4Tile<HD>& t, float c,
                                          const uint32_t (&vm)[JT], NF next) {
    float vs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) vs[e] = kv4_scale_of((uint32_t)t.vs[e >> 2], e & 3);
    auto V = [&](int m, i32x4 (&f)[2]) {
        const uint32_t w0 = (uint32_t)t.v[m >> 1][2 * (m & 1)], w1 = (uint32_t)t.v[m >> 1][2 * (m & 1) + 1];
        const uint32_t p[8] = {kv4_pair<0>(w0, vs[0]), kv4_pair<1>(w0, vs[1]), kv4_pair<2>(w0, vs[2]),
                               kv4_pair<3>(w0, vs[3]), kv4_pair<0>(w1, vs[4]), kv4_pair<1>(w1, vs[5]),
                               kv4_pair<2>(w1, vs[6]), kv4_pair<3>(w1, vs[7])};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[0][i] = (int)halves_lo(p[2 * i], p[2 * i + 1]);
            f[1][i] = (int)halves_hi(p[2 * i], p[2 * i + 1]);
        }
    };
    attn_step<HD, JT, MASKED, CARE>(st, S, c, V, vm, next);
}

static constexpr int KV4_WAVES = 8;

// The key tiles of a call: those that are in the 4-bit cache and that every
// row sees whole (the sink's, then the others), and the rest (the sink's and
// the window's ends, the last committed slots, the round, bf16 tiles).
struct Kv4Tiles {
    int a1, b0, n_whole;      // whole: [0, a1) and from b0 on
    int s1, p0, b1, n_edge;   // edges: [a1, s1), [p0, b0), from b1 on
    __device__ Kv4Tiles(const AttnWindow& win, int Lc, int n_slots, int n4) {
        const int n_tiles = (n_slots + 31) >> 5, last = min(Lc >> 5, n4 >> 5);
        a1 = min(win.csink >> 5, last);
        if (win.wstart >= Lc) {  // no window: the committed slots are one run
            s1 = p0 = b0 = b1 = a1;
        } else {
            s1 = win.st;
            p0 = win.pt0;
            b0 = max(p0, (win.wstart + 31) >> 5);
            b1 = last;
            if (b1 <= b0) b0 = b1 = p0;
        }
        n_whole = a1 + b1 - b0;
        n_edge = s1 - a1 + b0 - p0 + n_tiles - b1;
    }
    __device__ int whole(int i) const { return i < a1 ? i : i - a1 + b0; }
    __device__ int edge(int e) const {
        if (e < s1 - a1) return a1 + e;
        e -= s1 - a1;
        return e < b0 - p0 ? p0 + e : e - (b0 - p0) + b1;
    }
};

// TAIL: where slots from n4 on are: 0 none, 1 bf16 rows [Hkv][kv_cap][hd], 2
// the decoder's bf16 cache (tiled).
template <int HD, int JT, int TAIL>
__global__ void __launch_bounds__(64 * KV4_WAVES, 2) k_attn_kv4(const Kv4AttnArgs k4, float c) {
    constexpr int UD = HD / 32, DG = HD / 4, NDT = HD / 16, RS = HD + 4, W = KV4_WAVES, D = 3;
    const AttnArgs& a = k4.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int S = gridDim.x, split = blockIdx.x, kvh = blockIdx.y, rc = blockIdx.z;
    const int Lc = a.sp ? a.sp->Lc : a.Lc_host, n_tree = a.sp ? a.sp->n_tree : a.n_tree_host, n_slots = Lc + n_tree;
    if (a.sp && !dcheck(a.chk, Lc >= 0 && n_slots <= a.sp->cap && a.sp->cap <= a.ctx_cap, CHK_ATTN_SLOTS)) return;
    const int n4 = a.sp ? Lc & ~31 : k4.n4;
    const AttnWindow win(Lc, n_tree, a.win_sink, a.win_len);
    const int T = a.T, G = k4.G, Rp = k4.Rp;
    const uint16_t* q = (const uint16_t*)a.q;
    // packed row p's token and head of the group (rows past the group's: a valid row, not stored)
    auto head_of = [&](int p) { return k4.inv_Rp ? (int)__umulhi((uint32_t)p, k4.inv_Rp) : p; };
    auto row_of = [&](int p, int* t) {
        const int hg = head_of(p);
        *t = min(p - hg * Rp, T - 1);
        return q + ((size_t)*t * a.H + kvh * G + min(hg, G - 1)) * HD;
    };

    // this thread's piece of the query rows
    __shared__ Kv4QueryLds sm_q[JT];
    __shared__ float sm_m[W][16], sm_l[W][16];
    __shared__ __attribute__((aligned(16))) float sm_o[W][16][RS];  // a wave's part: 32 x (hd + 4) bf16 or its state
    constexpr int PP = HD / 32;
    const int qj = threadIdx.x / (64 * PP), qr = threadIdx.x / (4 * PP) % 16, qk = threadIdx.x / PP % 4,
              qp = threadIdx.x % PP;
    i32x4 qv = {0, 0, 0, 0};
    int tok;
    if (qj < JT) qv = *(const i32x4*)(row_of((JT * rc + qj) * 16 + qr, &tok) + qk * DG + qp * 8);
    // (each wave takes edge tiles for one of the query tiles, ej; this lane's row of it)
    const int ej = JT == 1 ? 0 : wave % JT;
    const uint16_t* qrow = row_of((JT * rc + ej) * 16 + r, &tok);
    const uint64_t an0 = a.anc[2 * tok], an1 = a.anc[2 * tok + 1];

    // The split's share of the whole tiles, and the wave's run [w0, w0 + n) of
    // it.  Edge tiles are dealt to the splits, then to the waves from the last
    // on; a wave with one takes EC whole tiles less, the time that it takes:
    // at(w) tiles lie before wave w's (a sum that rises by cost / W per wave,
    // less EC per edge tile; it ends at ns, so cut to [0, ns] it never falls).
    constexpr int EC = (TAIL ? 4 : 2) / JT, WJ = W / JT;
    const Kv4Tiles tl(win, Lc, n_slots, n4);
    auto by_S = [&](int x) { return k4.inv_S ? (int)__umulhi((uint32_t)x, k4.inv_S) : x; };
    const int s0 = by_S(tl.n_whole * split), ns = by_S(tl.n_whole * (split + 1)) - s0;
    const int workers = S * WJ, e_all = by_S(tl.n_edge) / WJ, e_more = tl.n_edge - e_all * workers;
    const int more = by_S(max(e_more - split + S - 1, 0)) * JT;  // the last waves that take one more
    const int cost = ns + EC * (W * e_all + more);
    auto at = [&](int w) { return min(max(cost * w / W - EC * (e_all * w + max(0, w - (W - more))), 0), ns); };
    const int w0 = s0 + at(wave), n = at(wave + 1) - at(wave);
    const Kv4Records<HD> recs(k4.kv4 + (size_t)kvh * (a.ctx_cap >> 5) * (34 * HD), a.ctx_cap >> 5, lane);
    Kv4Tile<HD> ring[D];
    if (n > 0) {
#pragma unroll
        for (int k = 0; k < D; ++k) ring[k] = recs.load(tl.whole(w0 + min(k, n - 1)));
    }
    if (qj < JT) kv4_query_put<HD>(sm_q[qj], qr, qk, qp, qv);
    __syncthreads();

    // the edge tiles, over the splits and the waves of each query tile
    AttnState<HD> es[1];
    es[0].clear();
    for (int e = split + S * (WJ - 1 - wave / JT); e < tl.n_edge; e += workers) {
        const int pt = tl.edge(e);
        const uint32_t vm[1] = {attn_vis8(pt * 32 + 8 * g, Lc, n_slots, win, an0, an1)};
        f32x4 Sc[1][2] = {{{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}};
        if (TAIL == 0 || pt * 32 < n4) {
            const Kv4Tile<HD> t = recs.load(pt);
            const Kv4Query<HD> Q[1] = {kv4_query_get<HD>(sm_q[ej], g, r)};
            kv4_scores<HD, 1>(Sc, t, Q);
            // (scales of 252 and more, whose values bf16 may not hold)
            uint32_t big = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t x = (uint32_t)t.vs[i], y = x & (x << 1);
                big |= y & (y << 2) & (y << 4) & 0x80808080u;
            }
            if (__any(big)) kv4_step4<HD, 1, true, true>(es, Sc, t, c, vm, [] {});
            else kv4_step4<HD, 1, true, false>(es, Sc, t, c, vm, [] {});
        } else if constexpr (TAIL != 0) {
            // keys and values of bf16 as MFMA fragments; rows' values come as 16-byte
            // pieces along the rows and are turned in the wave's part of sm_o
            // (gathered by 2 bytes from memory they took 5 us)
            constexpr int NV = HD / 16, VS = HD + 4, WR = 512 / HD;  // pieces per lane or d tiles; row stride in LDS
            const uint16_t* kt = TAIL == 1 ? k4.kr + (size_t)kvh * k4.kv_cap * HD
                                           : (const uint16_t*)a.kc + ((size_t)kvh * a.ctx_cap + pt * 32) * HD;
            const uint16_t* vt = TAIL == 1 ? k4.vr + (size_t)kvh * k4.kv_cap * HD
                                           : (const uint16_t*)a.vt + ((size_t)kvh * a.ctx_cap + pt * 32) * HD;
            auto row = [&](int sl) { return (size_t)(min(pt * 32 + sl, n_slots - 1) - n4) * HD; };
            i32x4 ek[UD][2], ev[NV];
#pragma unroll
            for (int u = 0; u < UD; ++u)
#pragma unroll
                for (int h2 = 0; h2 < 2; ++h2)
                    ek[u][h2] = *(const i32x4*)(TAIL == 1 ? kt + row(8 * (r >> 2) + 4 * h2 + (r & 3)) + g * DG + u * 8
                                                         : kt + (h2 * UD + u) * 512 + lane * 8);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int p = i * 64 + lane, d = 32 * (r / WR) + WR * i + r % WR;
                ev[i] = *(const i32x4*)(TAIL == 1 ? vt + row(p / (HD / 8)) + p % (HD / 8) * 8
                                                  : vt + ((d >> 4) * 64 + g * 16 + (d & 15)) * 8);
            }
            uint16_t* stage = (uint16_t*)&sm_o[wave][0][0];
            uint16x2 most = {0, 0};
#pragma unroll
            for (int i = 0; i < NV; ++i) {
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    most = __builtin_elementwise_max(most, __builtin_bit_cast(uint16x2, (uint32_t)ev[i][w] & 0x7fff7fffu));
                if constexpr (TAIL == 1) {
                    const int p = i * 64 + lane;
                    i32x2* to = (i32x2*)(stage + p / (HD / 8) * VS + p % (HD / 8) * 8);
                    to[0] = i32x2{ev[i][0], ev[i][1]};
                    to[1] = i32x2{ev[i][2], ev[i][3]};
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int u = 0; u < UD; ++u) {
                const i32x4 Qf = *(const i32x4*)(qrow + g * DG + u * 8);
#pragma unroll
                for (int h2 = 0; h2 < 2; ++h2) Sc[0][h2] = mfma_step<ET_BF16>(ek[u][h2], Qf, Sc[0][h2]);
            }
            auto V = [&](int m, i32x4 (&f)[2]) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if constexpr (TAIL == 1) {
                        const uint16_t* at = stage + 8 * g * VS + 32 * (r / WR) + WR * (2 * m + h) + r % WR;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            f[h][i] = (int)((uint32_t)at[2 * i * VS] | ((uint32_t)at[(2 * i + 1) * VS] << 16));
                    } else {
                        f[h] = ev[2 * m + h];
                    }
                }
            };
            if (__any(most[0] >= 0x7f80 || most[1] >= 0x7f80)) attn_step<HD, 1, true, true>(es, Sc, c, V, vm, [] {});
            else attn_step<HD, 1, true, false>(es, Sc, c, V, vm, [] {});
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
    mfma_result_pad();
    AttnState<HD> st[JT];
    Kv4Query<HD> Q[JT];
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        if (j == ej) st[j] = es[0];
        else st[j].clear();
        Q[j] = kv4_query_get<HD>(sm_q[j], g, r);
    }

    // the whole tiles
    if (n > 0) {
        const uint32_t all[JT] = {};
        f32x4 Sc[D][JT][2];
        kv4_scores<HD, JT>(Sc[0], ring[0], Q);
        mfma_result_pad();  // (the loop's branch follows)
        // Of the two waves of a SIMD the elder goes first wherever both can, and
        // ends at two thirds of the other's time, which is then alone: it
        // yields in every third step (128 rows of 8B heads over 16001 slots
        // 41.5 -> 40.1 us).
        if (wave >= W / 2) __builtin_amdgcn_s_setprio(1);
        for (int i = 0; i < n;) {
#pragma unroll
            for (int k = 0; k < D; ++k) {
                if (wave < W / 2) k == 1 ? __builtin_amdgcn_s_setprio(0) : __builtin_amdgcn_s_setprio(2);
                kv4_step4<HD, JT, false, false>(st, Sc[k], ring[k], c, all,
                                         [&] { kv4_scores<HD, JT>(Sc[(k + 1) % D], ring[(k + 1) % D], Q); });
                // (pins them to this step: the compiler would move them to their use)
#pragma unroll
                for (int j = 0; j < JT; ++j) asm volatile("" : "+v"(Sc[(k + 1) % D][j][0]), "+v"(Sc[(k + 1) % D][j][1]));
                ring[k] = recs.load(tl.whole(w0 + min(i + D, n - 1)));
                if (++i >= n) break;
            }
        }
        __builtin_amdgcn_s_setprio(0);
    }
    mfma_result_pad();

    // ---- join the waves, one query tile after another
    constexpr int D4 = HD / 4;
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        if (j) __syncthreads();
        if (g == 0) {
            sm_m[wave][r] = st[j].m * c;
            sm_l[wave][r] = st[j].l[0];
        }
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) *(f32x4*)(&sm_o[wave][r][kv4_out_d<HD>(g, dt)]) = st[j].O[dt];
        __syncthreads();
        for (int idx = threadIdx.x; idx < 16 * D4; idx += 64 * W) {
            const int rr = idx / D4, d4 = (idx % D4) * 4;
            const int p = (JT * rc + j) * 16 + rr, hg = head_of(p), t = p - hg * Rp;
            if (hg >= G || t >= T) continue;
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
                const float f = __builtin_amdgcn_exp2f(mw[w] - M);
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

// The join of S splits' partial states: SG (at most 256 / (hd / 4)) groups of
// hd/4 threads per row take every SG-th split, four at a time, and join through
// LDS: with 32 splits of one row one round of loads where a thread that takes
// all splits waits for four (32 heads' row: 4.0 us for 4.6).
static constexpr int KV4_MERGE_THREADS = 256;
template <int HD> __global__ void __launch_bounds__(KV4_MERGE_THREADS) k_kv4_merge(const AttnArgs a, int S, int SG) {
    constexpr int D4 = HD / 4, NG = KV4_MERGE_THREADS / D4;
    __shared__ float2 sm_ml[NG];
    __shared__ f32x4 sm_o[NG][D4];
    const int gi = threadIdx.x / D4, d4 = threadIdx.x % D4 * 4;
    const int row = blockIdx.x * (NG / SG) + gi / SG, sub = gi % SG;  // row = head * T + t
    const size_t rows = (size_t)a.H * a.T;
    const bool live = row < (int)rows;
    const size_t rr = live ? row : 0;
    float M = -FLT_MAX, L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = sub; s0 < S; s0 += 4 * SG) {
        float2 ml[4];
        f32x4 po[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const size_t at = (size_t)min(s0 + k * SG, S - 1) * rows + rr;
            ml[k] = *(const float2*)(a.part_ml + at * 2);
            po[k] = *(const f32x4*)(a.part_o + at * HD + d4);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (s0 + k * SG < S) {
                const f32x4 o[1] = {po[k]};
                f32x4 A[1] = {acc};
                attn_merge_split<1>(A, L, M, o, ml[k].y, ml[k].x);
                acc = A[0];
            }
    }
    if (SG > 1) {
        if (d4 == 0) sm_ml[gi] = make_float2(M, L);
        sm_o[gi][d4 / 4] = acc;
        __syncthreads();
        if (sub == 0)
            for (int i = 1; i < SG; ++i) {
                const f32x4 o[1] = {sm_o[gi + i][d4 / 4]};
                f32x4 A[1] = {acc};
                attn_merge_split<1>(A, L, M, o, sm_ml[gi + i].y, sm_ml[gi + i].x);
                acc = A[0];
            }
    }
    if (sub != 0 || !live) return;
    const float inv = L != 0.f ? 1.f / L : 0.f;  // no slot seen: 0 (a NaN sum stays one)
    const int t = row % a.T, k = row / a.T * HD + d4;
    const size_t o = a.out_tiled ? xt_off(t, k, col_tiles(a.T), 8) : (size_t)t * a.H * HD + k;
    st4((uint16_t*)a.out, o, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
}
template <int HD> static hipError_t kv4_merge_go(const AttnArgs& a, int S, hipStream_t s) {
    constexpr int NG = KV4_MERGE_THREADS / (HD / 4);
    int SG = 1;
    while (SG < NG && SG * 2 <= S) SG *= 2;
    const unsigned wgs = ((unsigned)(a.H * a.T) + NG / SG - 1) / (NG / SG);
    return launch_checked(k_kv4_merge<HD>, dim3(wgs), KV4_MERGE_THREADS, s, a, S, SG);
}

// Query tiles per workgroup (jt) and splits of the key tiles (S), by the time
// that a call takes as the sum of its parts in microseconds, fitted to calls of
// 1 to 128 rows over 33 to 131071 slots with every jt and S up to 32 (13% off
// in the mean): the rounds in which 256 CUs take the workgroups one at a time
// (two waves per SIMD), each its start and end and its waves' steps, and the
// merge of the partials.  Two query tiles share a step's conversions but leave
// fewer workgroups, which end later: 128 rows of 8B heads over 16001 slots take
// 38.3 us with 2 tiles and 2 splits, 40.2 with 1 and 1; 64 rows of 13B heads
// over 2048 slots 9.6 with 1 and 1, 14.2 with 2 and 1.  One split needs no
// merge: one row of 13B heads over 500 slots takes 5.5 us with it, 7.1 with two.
Kv4Plan kv4_plan(int Lc, int n_tree, int T, int H, int Hkv, int hd, int win_sink, int win_len, int max_S) {
    const int n_log = AttnWindow(Lc, n_tree, win_sink, win_len).n_log;
    const int nct = attn_query_tiles(T, H / Hkv);
    Kv4Plan best{1, 1};
    float least = INFINITY;
    for (int jt = 1; jt <= (nct > 1 ? 2 : 1); ++jt) {
        const int z = (nct + jt - 1) / jt;
        for (const int S : {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 16, 20, 24, 28, 32, 40, 48, 56, ATT_MAX_SPLITS}) {
            if (S > 1 && (S > max_S || S > n_log)) break;
            const float wgs = (float)Hkv * z * S;
            const int rounds = (int)((wgs + 255) / 256);
            const int steps = ((n_log + S - 1) / S + KV4_WAVES - 1) / KV4_WAVES;
            const float step = (jt == 1 ? 0.68f : 0.95f) * (hd == 128 ? 1.f : 0.59f);
            float us = rounds * ((jt == 1 ? 2.3f : 3.5f) + steps * step);
            if (S > 1) us += 2.9f + 0.33e-6f * S * H * T * hd * 8;
            if (us < least) {
                least = us;
                best = Kv4Plan{jt, S};
            }
        }
    }
    return best;
}

template <int HD, int JT> static hipError_t attn_kv4_go(const Kv4AttnArgs& k, dim3 grid, int tail, float c, hipStream_t s) {
    return launch_checked(tail == 0   ? k_attn_kv4<HD, JT, 0>
                      : tail == 1 ? k_attn_kv4<HD, JT, 1>
                                  : k_attn_kv4<HD, JT, 2>,
                      grid, 64 * KV4_WAVES, s, k, c);
}

hipError_t launch_attention_kv4(const Kv4AttnArgs& k, hipStream_t s) {
    const AttnArgs& a = k.a;
    if (a.T < 1 || a.T > 128 || a.Hkv < 1 || a.H % a.Hkv || a.ctx_cap % 32) return hipErrorInvalidValue;
    if (k.plan.S < 1 || k.plan.S > ATT_MAX_SPLITS || (k.plan.jt != 1 && k.plan.jt != 2)) return hipErrorInvalidValue;
    const int S = k.plan.S, jt = k.plan.jt, nct = attn_query_tiles(a.T, a.H / a.Hkv);
    const dim3 grid(S, a.Hkv, (nct + jt - 1) / jt);
    // (the decoder's whole-tile copy always leaves slots to its bf16 cache)
    const int tail = a.sp ? 2 : k.n4 < a.Lc_host + a.n_tree_host ? 1 : 0;
    const float c = (1.0f / sqrtf((float)a.hd)) * 1.4426950408889634f;
    Kv4AttnArgs k2 = k;
    k2.G = a.H / a.Hkv;
    k2.Rp = attn_head_rows(a.T);
    // (multiplying by these and taking the high word divides by up to 128 exactly below 2^25)
    auto inverse = [](int d) { return d > 1 ? (uint32_t)((((uint64_t)1 << 32) + d - 1) / d) : 0u; };
    k2.inv_Rp = inverse(k2.Rp);
    k2.inv_S = inverse(S);
    k2.direct = S == 1 && !a.out_tiled && !a.qout && !a.no_merge;
    hipError_t e = hipErrorInvalidValue;
    if (a.hd == 128)
        e = jt == 2 ? attn_kv4_go<128, 2>(k2, grid, tail, c, s) : attn_kv4_go<128, 1>(k2, grid, tail, c, s);
    else if (a.hd == 64)
        e = jt == 2 ? attn_kv4_go<64, 2>(k2, grid, tail, c, s) : attn_kv4_go<64, 1>(k2, grid, tail, c, s);
    if (e != hipSuccess || k2.direct || a.no_merge) return e;
    if (a.qout) return launch_attn_merge(a, S, s);  // (the output's codes need whole rows)
    return a.hd == 128 ? kv4_merge_go<128>(a, S, s) : kv4_merge_go<64>(a, S, s);
}

}  // namespace cas
