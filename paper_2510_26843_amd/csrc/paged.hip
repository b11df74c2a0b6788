// gfx950 kernels of the paged KV cache: appending the new rows of several
// sequences with their rotation, and attention of those rows over it.
//
// A page holds page_size slots (a power of two of 32-slot tiles) of every kv
// head, keys then values: [n_pages][2][Hkv][page_size / 32] tiles of 32 * hd
// bf16 in the decoder's order of MFMA fragments (kv_k_tiled, kv_v_tiled), so a
// wave reads a fragment as 1 KB in one piece and no tile crosses a page.
// Sequence b of a batch has the slots [0, first + T): ctx_len[b] committed ones,
// nodes[b] earlier ones of its round, and the T = seq_start[b + 1] -
// seq_start[b] rows of the call at the slots from first on.
//
// Lengths, tables and positions are read on the device, so that a captured
// call serves batches of other lengths: nothing they hold makes a kernel leave
// its buffers.  Pages outside the pool store nothing and read as NaN, sequences
// whose lengths do not fit get rows of NaN.
#include "attn_step.h"

#include <algorithm>

namespace cas {

// ---------------------------------------------------------------- sequences

struct PagedSeq {
    int b, row0, T, Lc, first;
    bool fits;
    __device__ __forceinline__ int n_slots() const { return first + T; }
};

// Sequence b's lengths (T = 0 past the last one, or where its rows are not rows
// of the call).
__device__ __forceinline__ PagedSeq paged_seq(const PagedBatch& p, int b, bool tree) {
    PagedSeq s;
    const int i = min(b, p.B - 1);
    const int s0 = p.seq_start[i], s1 = p.seq_start[i + 1], nodes = p.nodes ? p.nodes[i] : 0;
    s.b = i;
    s.row0 = s0;
    s.T = b < p.B && s0 >= 0 && s0 < s1 && s1 <= p.N ? s1 - s0 : 0;
    s.Lc = p.ctx_len[i];
    s.fits = s.Lc >= 0 && s.Lc <= p.cap && nodes >= 0 && nodes <= p.cap && s.Lc + nodes <= p.cap - s.T &&
             (!tree || nodes + s.T <= 128);
    s.first = s.Lc + nodes;
    return s;
}

// A page number: the same for the whole wave, by the scalar unit.
__device__ __forceinline__ int paged_page(const PagedBatch& p, int b, int tile) {
    typedef const __attribute__((address_space(4))) int* at;
    return ((at)(p.table + (size_t)b * p.table_len))[(uint32_t)tile >> p.tshift];
}

// ---------------------------------------------------------------- append

// One workgroup = one tile (32 slots) that new rows fall into, for one kv head
// and the query heads of its group.  A sequence of T rows touches at most T / 32 +
// 2 tiles, so those of sequence b are numbered from row0 / 32 + 2 b on: no sum
// over the sequences before it.
//
// A whole tile: all loads run along the rows and are issued first, a thread's
// angles serve its key and its queries, and the tile is put together in LDS and
// stored 16 bytes per lane in one piece.  Another tile's few rows are stored in
// place, a piece of 8 elements per thread.
//
// What bounds it: many rows, memory (16384 rows of 32 + 8 + 8 heads of 128, 411 MB:
// 84 us, 4.9 TB/s, a copy's rate; with every tile stored in place and the heads of
// a tile apart 111); one row, its chain of loads (4.4 us).
static constexpr int PAPP_THREADS = 256;

__device__ __forceinline__ i32x4 paged_ld8(const uint16_t* p, bool vec) {
    if (vec) return *(const i32x4*)p;
    i32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (int)((uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16));
    return v;
}

// The pieces x (elements d0 ..) and y (d0 + hd/2 ..) of a head row, rotated in
// fp32 (each product's error 2^-24 of it) and rounded to bf16 once.
__device__ __forceinline__ void paged_rotate(const f32x4 (&cs)[2], const f32x4 (&sn)[2], bool ok, i32x4& x, i32x4& y) {
    float lo[8], hi[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float a = piece_val<uint16_t>(x, e), b = piece_val<uint16_t>(y, e);
        lo[e] = ok ? rope_lo(a, b, cs[e >> 2][e & 3], sn[e >> 2][e & 3]) : NAN;
        hi[e] = ok ? rope_hi(a, b, cs[e >> 2][e & 3], sn[e >> 2][e & 3]) : NAN;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = (int)pack_bf(lo[2 * i], lo[2 * i + 1]);
        y[i] = (int)pack_bf(hi[2 * i], hi[2 * i + 1]);
    }
}

template <int HD> __global__ void __launch_bounds__(PAPP_THREADS) k_paged_append(const PagedAppendArgs a) {
    const PagedBatch& p = a.p;
    // (the heads of a tile follow each other: rows are read as a whole)
    const int lane = threadIdx.x & 63, place = blockIdx.x / p.Hkv;
    // the last sequence whose tiles start at or before this one
    int b = -1;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int i = min(b0 + lane, p.B - 1);
        const uint64_t in = __ballot(b0 + lane < p.B && (int64_t)(p.seq_start[i] >> 5) + 2 * i <= (int64_t)place);
        if (in) b = b0 + 63 - __builtin_clzll(in);
    }
    b = __builtin_amdgcn_readfirstlane(b);
    if (b < 0) return;
    const PagedSeq s = paged_seq(p, b, false);
    if (s.T == 0 || !s.fits) return;
    const int tile = (s.first >> 5) + place - ((s.row0 >> 5) + 2 * b);
    const int lo = max(s.first, tile * 32), hi = min(s.first + s.T, tile * 32 + 32);
    if (lo >= hi) return;
    const int row = s.row0 + tile * 32 - s.first;  // of the tile's slot 0
    const int h = blockIdx.x % p.Hkv, G = a.q ? a.H / p.Hkv : 0, tid = threadIdx.x;
    const int pid = paged_page(p, b, tile);
    const bool paged = (uint32_t)pid < (uint32_t)p.n_pages;  // (else nothing is stored)
    uint16_t* kt = p.pages + ((((size_t)(paged ? pid : 0) * 2 * p.Hkv + h) << p.tshift) + (tile & ((1 << p.tshift) - 1))) * (32 * HD);
    uint16_t* vt = kt + (((size_t)p.Hkv << p.tshift) * (32 * HD));
    constexpr int PR = HD / 16;  // pairs of pieces of a head row
    auto k_at = [&](int sl, int d0) { return a.k + (size_t)(row + sl) * a.ldk + (size_t)h * HD + d0; };
    auto q_at = [&](int sl, int g, int d0) { return a.q + (size_t)(row + sl) * a.ldq + (size_t)(h * G + g) * HD + d0; };
    auto v_at = [&](int sl, int d0) { return a.v + (size_t)(row + sl) * a.ldv + (size_t)h * HD + d0; };
    auto q_to = [&](int sl, int g, int d0, const i32x4 x, const i32x4 y) {
        uint16_t* to = a.q_out + ((size_t)(row + sl) * a.H + h * G + g) * HD + d0;
        *(i32x4*)to = x;
        *(i32x4*)(to + HD / 2) = y;
    };
    // dwords of slots s4, s4 + 1 and s4 + 2, s4 + 3 at element e of four rows' pieces
    auto turned = [](const i32x4 (&x)[4], int e) {
        const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
        return make_uint2(__builtin_amdgcn_perm((uint32_t)x[1][e >> 1], (uint32_t)x[0][e >> 1], sel),
                          __builtin_amdgcn_perm((uint32_t)x[3][e >> 1], (uint32_t)x[2][e >> 1], sel));
    };
    if (hi - lo == 32) {
        // (every 256 bytes 16 further on: a row's pieces lie 256 bytes apart)
        constexpr int PIECES = 32 * HD / 8;
        __shared__ i32x4 ki[PIECES + PIECES / 16], vi[PIECES + PIECES / 16];
        auto spread = [](int element) { return element + element / 128 * 8; };
        constexpr int QB = 4;                                 // query heads at a time
        const bool kq = tid < 32 * PR;                        // a pair of pieces of a slot: its key's and its queries'
        const int vt0 = HD == 128 ? 0 : 128;                  // the threads of the values, four slots of 8 elements each
        const bool vv = tid >= vt0 && tid < vt0 + HD;
        const int sl = tid / PR % 32, d0 = tid % PR * 8, dv = (tid - vt0) % (HD / 8) * 8, s4 = (tid - vt0) / (HD / 8) * 4;
        i32x4 kx, ky, v[4], qx[QB], qy[QB];
        if (kq) {
            kx = paged_ld8(k_at(sl, d0), a.vec);
            ky = paged_ld8(k_at(sl, d0 + HD / 2), a.vec);
        }
        if (vv) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = paged_ld8(v_at(s4 + j, dv), a.vec);
        }
        auto load_q = [&](int g0) {
#pragma unroll
            for (int g = 0; g < QB; ++g)
                if (g0 + g < G) {
                    qx[g] = paged_ld8(q_at(sl, g0 + g, d0), a.vec);
                    qy[g] = paged_ld8(q_at(sl, g0 + g, d0 + HD / 2), a.vec);
                }
        };
        if (kq) load_q(0);
        bool ok = false;
        f32x4 cs[2], sn[2];
        if (kq && a.cos) {
            const int pos = a.pos ? a.pos[row + sl] : tile * 32 + sl;
            ok = pos >= 0 && pos < a.n_pos;
            const size_t at = (size_t)(ok ? pos : 0) * (HD / 2) + d0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                cs[i] = *(const f32x4*)(a.cos + at + 4 * i);
                sn[i] = *(const f32x4*)(a.sin + at + 4 * i);
            }
        }
        if (kq) {
            if (a.cos) paged_rotate(cs, sn, ok, kx, ky);
            *(i32x4*)((uint16_t*)ki + spread((int)kv_k_tiled(sl, d0, HD))) = kx;
            *(i32x4*)((uint16_t*)ki + spread((int)kv_k_tiled(sl, d0 + HD / 2, HD))) = ky;
        }
        if (vv) {
#pragma unroll
            for (int e = 0; e < 8; ++e) *(uint2*)((uint16_t*)vi + spread((int)kv_v_tiled(s4, dv + e, HD))) = turned(v, e);
        }
        if (kq) {
            for (int g0 = 0; g0 < G; g0 += QB) {
                if (g0) load_q(g0);
#pragma unroll
                for (int g = 0; g < QB; ++g)
                    if (g0 + g < G) {
                        if (a.cos) paged_rotate(cs, sn, ok, qx[g], qy[g]);
                        q_to(sl, g0 + g, d0, qx[g], qy[g]);
                    }
            }
        }
        __syncthreads();
        if (!paged) return;
        for (int i = tid; i < PIECES; i += PAPP_THREADS) {
            ((i32x4*)kt)[i] = ki[i + i / 16];
            ((i32x4*)vt)[i] = vi[i + i / 16];
        }
        return;
    }
    const int s_lo = lo - tile * 32, s_hi = hi - tile * 32, n = s_hi - s_lo;
    const int nk = n * PR, nq = nk * G, g_lo = s_lo >> 2, nv = (((s_hi + 3) >> 2) - g_lo) * (HD / 8);
    for (int it = tid; it < nk + nq + nv; it += PAPP_THREADS) {
        if (it < nk + nq) {  // a pair of pieces of a key or query
            const bool key = it < nk;
            const int i = key ? it : it - nk, d0 = i % PR * 8, g = key ? 0 : i / PR % G, sl = s_lo + (key ? i / PR : i / PR / G);
            const uint16_t* from = key ? k_at(sl, d0) : q_at(sl, g, d0);
            i32x4 x = paged_ld8(from, a.vec), y = paged_ld8(from + HD / 2, a.vec);
            if (a.cos) {
                const int pos = a.pos ? a.pos[row + sl] : tile * 32 + sl;
                const bool ok = pos >= 0 && pos < a.n_pos;
                const size_t at = (size_t)(ok ? pos : 0) * (HD / 2) + d0;
                const f32x4 cs[2] = {*(const f32x4*)(a.cos + at), *(const f32x4*)(a.cos + at + 4)};
                const f32x4 sn[2] = {*(const f32x4*)(a.sin + at), *(const f32x4*)(a.sin + at + 4)};
                paged_rotate(cs, sn, ok, x, y);
            }
            if (!key) {
                q_to(sl, g, d0, x, y);
            } else if (paged) {
                *(i32x4*)(kt + kv_k_tiled(sl, d0, HD)) = x;
                *(i32x4*)(kt + kv_k_tiled(sl, d0 + HD / 2, HD)) = y;
            }
        } else if (paged) {  // four slots' values at 8 elements
            const int i = it - nk - nq, d0 = i % (HD / 8) * 8, s4 = (g_lo + i / (HD / 8)) * 4;
            i32x4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = paged_ld8(v_at(min(max(s4 + j, s_lo), s_hi - 1), d0), a.vec);
            const bool whole = s4 >= s_lo && s4 + 4 <= s_hi;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint2 w = turned(x, e);
                uint16_t* to = vt + kv_v_tiled(s4, d0 + e, HD);
                if (whole) {
                    *(uint2*)to = w;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (s4 + j >= s_lo && s4 + j < s_hi) to[j] = (uint16_t)((j & 2 ? w.y : w.x) >> (16 * (j & 1)));
                }
            }
        }
    }
}

hipError_t launch_paged_append(const PagedAppendArgs& a, hipStream_t s) {
    const PagedBatch& p = a.p;
    if (p.N < 1 || p.B < 1 || p.Hkv < 1 || (a.q && a.H % p.Hkv)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)paged_append_grid(p));
    if (p.hd == 128) return launch_checked(k_paged_append<128>, grid, PAPP_THREADS, s, a);
    if (p.hd == 64) return launch_checked(k_paged_append<64>, grid, PAPP_THREADS, s, a);
    return hipErrorInvalidValue;
}

// ---------------------------------------------------------------- attention: the work and its shares

// Slots that a row sees.  Causal: those up to its own; with a window, of the
// ones before it the first `sink` and the last `window`.  Tree: committed slots
// (the first `sink` and the last `window` of them) and the nodes of its mask.
// A call's tiles for the rows [t0, t1) of a sequence: the sink's, then from pt0.
struct PagedRange {
    int st, pt0, n_log;  // tiles [0, st) and [pt0, pt0 + n_log - st)
    int wlo, whi;        // whole for every row: tiles in [wlo, whi) and below ...
    int slo;             // ... slo
    __device__ __forceinline__ int phys(int lt) const { return lt < st ? lt : lt - st + pt0; }
    __device__ __forceinline__ bool whole(int tile) const { return (tile >= wlo && tile < whi) || tile < slo; }
    __device__ PagedRange(const PagedSeq& s, int t0, int t1, bool tree, int sink, int window) {
        // slots every row sees as committed: [0, all), and those any row sees: [0, any)
        const int all = tree ? s.Lc : s.first + t0 + 1, any = tree ? s.n_slots() : s.first + t1;
        const int n_tiles = (any + 31) >> 5;
        st = 0;
        pt0 = 0;
        wlo = 0;
        whi = all >> 5;
        slo = 0;
        if (window > 0) {
            const int w0 = max((tree ? s.Lc : s.first + t0) - window, 0);      // the first row's window starts
            const int w1 = max((tree ? s.Lc : s.first + t1 - 1) - window, 0);  // the last row's
            st = min((min(sink, all) + 31) >> 5, n_tiles);
            pt0 = min(max(w0 >> 5, st), n_tiles);
            slo = min(sink, all) >> 5;
            wlo = (w1 + 31) >> 5;
        }
        n_log = st + n_tiles - pt0;
    }
};

// Visibility of the 8 slots base .. to row t of a sequence.
__device__ __forceinline__ uint32_t paged_vis8(const PagedSeq& s, int t, int base, bool tree, uint64_t an0, uint64_t an1,
                                               int sink, int window) {
    if (tree) return attn_vis8(base, s.Lc, s.n_slots(), AttnWindow(s.Lc, s.n_slots() - s.Lc, sink, window), an0, an1);
    const int own = s.first + t;
    if (window == 0) return bits8(0, own + 1 - base);
    return bits8(0, min(sink, own) - base) | bits8(own - window - base, own + 1 - base);
}

// How the work is shared out.  A unit is (sequence, query tile of R packed
// rows, kv head); the split rule gives a sequence of more than C tiles ns =
// ceil(tiles / C) shares per unit, with C such that the batch has about
// `target` shares of C tiles, so that one long sequence among short ones is
// split and equal ones that fill the chip by themselves are not.  Every wave
// sums the sequences' work and finds its own share, 64 sequences at a time:
// the kernels need no plan made before them, and a replayed call shares out
// the lengths of its own time.
//   shares in all:            sum nq ns <= sum nq + target    (ns - 1 < tiles / C)
//   shares of split units:    <= 2 target                     (ns < 2 tiles / C)
//   split units:              <= target
struct PagedShare {
    PagedSeq s;
    int ns, nq, local, part;  // local: place among the sequence's; part: first partial of the sequence's
    bool found;
};
// The least tiles of a share: one for each of eight waves (1 row over 4095 slots 9.0
// us, at least 16 tiles 9.4, 32 tiles 10.7; 32 rows at 1000 12.4, 13.9, 14.6).
static constexpr int PAGED_LEAST = 8;
template <bool MERGE>
__device__ __forceinline__ PagedShare paged_share(const PagedAttnArgs& a, int R, int item) {
    const PagedBatch& p = a.p;
    const int lane = threadIdx.x & 63, G = a.G;
    const bool tree = a.anc != nullptr;
    struct Seq {
        PagedSeq s;
        int nq, tiles;
    };
    auto seq = [&](int b) {
        Seq q;
        q.s = paged_seq(p, b, tree);
        q.nq = (int)(((int64_t)q.s.T * G + R - 1) >> __builtin_ctz(R));
        q.tiles = !q.s.fits || q.s.T == 0 ? 0 : (q.s.n_slots() + 31) >> 5;
        if (a.window > 0) {  // (the most that one of its query tiles walks)
            const int t = tree ? q.s.n_slots() - q.s.Lc : min(q.s.T, R / G + 2);
            q.tiles = min(q.tiles, ((a.sink + 31) >> 5) + ((min(a.window, p.cap) + t + 31) >> 5) + 1);
        }
        return q;
    };
    const Seq own = seq(lane);
    // tiles / C rounded up, or one less where that is a hair above a whole number
    auto parts_of = [](int tiles, int C, float rC) {
        const int ns = max((int)((float)tiles * rC), 1);
        return ns + ((int64_t)ns * C < tiles ? 1 : 0);
    };
    auto shares_of = [&](int C) {
        const float rC = __builtin_amdgcn_rcpf((float)C);
        int n = own.nq * parts_of(own.tiles, C, rC);
        for (int b0 = 64; b0 < p.B; b0 += 64) {
            const Seq q = seq(b0 + lane);
            n += q.nq * parts_of(q.tiles, C, rC);
        }
        return wave_total<int>(n);
    };
    int C = 1 << 30;
    if (a.target > 0) {
        // (many: nothing hangs on how many; sequences that overlap could pass 32 bits)
        constexpr int MANY = 1 << 24;
        int nq = min(own.nq, MANY), most = own.tiles;
        float w = (float)own.nq * own.tiles;
        for (int b0 = 64; b0 < p.B; b0 += 64) {
            const Seq q = seq(b0 + lane);
            nq = min(nq + min(q.nq, MANY), MANY);
            most = max(most, q.tiles);
            w += (float)q.nq * q.tiles;
        }
        nq = wave_total<int>(nq);
        // (a lane's 1024 sums and the wave's: off by at most 1100 2^-24 of it.  Never
        // below what it stands for, as the bounds need)
        w = wave_total<float>(w) * 1.0001f;
        most = wave_most(most);
        auto share = [&](int n) {
            return max(PAGED_LEAST, (int)fminf(1073741824.f, ceilf(w * __builtin_amdgcn_rcpf((float)n))));
        };
        if (most > a.whole) {
            C = share(a.target);
            // With room left by the units: as many shares as run at once, if the longest
            // is then no longer than two rounds of the finer ones (and the partial states
            // of 128 rows, as many bytes written and read as eight tiles: 5 ragged chunks
            // of up to 400 rows, 40 heads, 53.7 us without, 50.2 with).  On 32 rows only if
            // the finer ones do not run at once (64 rows, 8 sequences at 16000 slots, 8
            // heads: unsplit 160 us, in halves 109); on 16 a share too many costs more
            // than a CU left over (8 sequences at 4095: three shares each 26 us, four 28).
            if (nq < a.target) {
                const int D = share(a.target - nq);
                if (min(D, most) <= 2 * C + (R == 128 ? 8 : 0) && (R != 32 || shares_of(C) > a.target)) C = D;
            }
            // Where a workgroup has its CU to itself a tile takes it 0.57 us, where two
            // share one 0.87; the partial states of twice the shares cost 5 us more.
            if (nq < a.single) {
                const int A = share(a.single - nq);
                auto longest = [&](int c) {
                    return (float)most * __builtin_amdgcn_rcpf(ceilf((float)most * __builtin_amdgcn_rcpf((float)c)));
                };
                if (0.57f * longest(A) <= 0.87f * longest(C) + 5.f) C = A;
            }
        }
    }
    const float rC = __builtin_amdgcn_rcpf((float)C);
    PagedShare r;
    r.found = false;
    int before = 0, parts = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const Seq q = b0 ? seq(b0 + lane) : own;
        const int ns = parts_of(q.tiles, C, rC);
        int n = MERGE ? (ns > 1 ? q.nq : 0) : q.nq * ns, np = ns > 1 ? q.nq * ns : 0;
        const int n_own = n, np_own = np;
        n = wave_scan(n);
        np = wave_scan(np);
        const uint64_t past = __ballot(before + n > item);
        if (past) {
            const int l = __builtin_ctzll(past);
            auto of = [&](int x) { return (int)__builtin_amdgcn_readlane(x, l); };
            r.s.b = b0 + l;
            r.s.row0 = of(q.s.row0);
            r.s.T = of(q.s.T);
            r.s.Lc = of(q.s.Lc);
            r.s.first = of(q.s.first);
            r.s.fits = of(q.s.fits);
            r.ns = of(ns);
            r.nq = of(q.nq);
            r.local = item - before - of(n - n_own);
            r.part = parts + of(np - np_own);
            r.found = true;
            return r;
        }
        before += __builtin_amdgcn_readlane(n, 63);
        parts += __builtin_amdgcn_readlane(np, 63);
    }
    return r;
}

// A lane's largest scores of a tile.
template <int JT> __device__ __forceinline__ void paged_tops(float (&t)[JT], const f32x4 (&x)[JT][2]) {
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        t[j] = x[j][0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) t[j] = fmaxf(t[j], x[j][e >> 2][e & 3]);
    }
}

// attn_step for a tile that some row of the wave does not see whole (vm: the
// visibility of the lane's slots), or of a page outside the pool: the scores of
// unseen slots go to -infinity.  Kept short, since few tiles run it and most of
// those for the first time.  Values that are not finite, which a probability of 0
// would not hide, show in their products with zeros; looking at their exponents
// took a decoded token over 500 slots 0.4 us more, 128 rows of a fresh cache 1.3.
template <int HD, int JT, int TERMS>
__device__ __forceinline__ void paged_end(AttnState<HD> (&st)[JT], f32x4 (&S)[JT][2], i32x4 (&vf)[HD / 16], uint32_t (&vm)[JT],
                                          bool outside, float c) {
    constexpr int NDT = HD / 16;
    f32x4 z[2] = {};
#pragma unroll
    for (int f = 0; f < NDT; ++f) z[f & 1] = mfma_step<ET_BF16>(vf[f], i32x4{0, 0, 0, 0}, z[f & 1]);
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)vm[j], e, 1);
            S[j][e >> 2][e & 3] = __uint_as_float((__float_as_uint(S[j][e >> 2][e & 3]) & m) | (0xff800000u & ~m));
        }
    if (outside) {
#pragma unroll
        for (int j = 0; j < JT; ++j) {
            asm volatile("" : "+v"(vm[j]));  // (no 16 conditions kept from here on)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if ((vm[j] >> e) & 1u) S[j][e >> 2][e & 3] = NAN;
        }
    }
    float t[JT];
    paged_tops<JT>(t, S);
    mfma_result_pad();
    const f32x4 y = z[0] + z[1];
    const bool odd = __any(y[0] + y[1] + y[2] + y[3] != 0.f);
    bool grow = false;
#pragma unroll
    for (int j = 0; j < JT; ++j) grow = grow || t[j] > st[j].top;
    if (__any(grow)) {
        mfma_result_pad();
#pragma unroll
        for (int j = 0; j < JT; ++j) attn_follow(st[j], t[j], c);
    }
    i32x4 P[JT][TERMS];
    const int one = 0x3f803f80;
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        attn_probs(P[j], S[j], st[j].mc, st[j].c);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) st[j].l = mfma_step<ET_BF16>(i32x4{one, one, one, one}, P[j][k], st[j].l);
    }
    // (one arm each: with two that both write O the compiler copies or spills it)
    if (!odd) {
#pragma unroll
        for (int f = 0; f < NDT; ++f)
#pragma unroll
            for (int j = 0; j < JT; ++j)
#pragma unroll
                for (int k = 0; k < TERMS; ++k) st[j].O[f] = mfma_step<ET_BF16>(vf[f], P[j][k], st[j].O[f]);
    }
    mfma_result_pad();
    if (odd) {  // taken out, and given back as NaN to the rows that see them
        i32x4 seen[JT];
#pragma unroll
        for (int j = 0; j < JT; ++j) {
            asm volatile("" : "+v"(vm[j]));
#pragma unroll
            for (int w = 0; w < 4; ++w)
                seen[j][w] = (int)(((vm[j] >> (2 * w)) & 1u ? 0x3f80u : 0u) | ((vm[j] >> (2 * w + 1)) & 1u ? 0x3f800000u : 0u));
        }
#pragma unroll
        for (int f = 0; f < NDT; ++f) {
            const i32x4 bad = take_nonfinite(vf[f]);
#pragma unroll
            for (int j = 0; j < JT; ++j) {
                const f32x4 n = mfma_step<ET_BF16>(bad, seen[j], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int k = 0; k < TERMS; ++k) st[j].O[f] = mfma_step<ET_BF16>(vf[f], P[j][k], st[j].O[f]);
                mfma_result_pad();
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float to = n[e] > 0.f ? NAN : 0.f;
                    asm volatile("" : "+v"(to));  // (here, not as 64 conditions at the end)
                    st[j].O[f][e] += to;
                }
            }
        }
    }
}

// ---------------------------------------------------------------- attention: few rows

// Workgroup = (share of a unit, kv head): JT query tiles of 16 packed rows (row
// p = token p / G, head p % G of the group), the share's key tiles over eight
// waves, each with the running maximum and sum of a softmax of its own (attn_step),
// joined through LDS at the end.  K and V fragments go from memory to the
// registers that the MFMA reads: no other wave wants them.
//
// What bounds it: 16 rows, memory (32 sequences of up to 8190 slots, 8 heads, 276
// MB: 64 us with the join, 4.3 TB/s; one of 131072, 537 MB: 101, 5.3 TB/s.  With keys
// and values of a tile loaded together the 32 took 66 where this took 54, over inputs
// of which the memory-side cache keeps a part); 32 rows, memory (trees of 8 sequences,
// 119 MB: 3.7 TB/s), and the L2s where several units read the same slots; few slots,
// the waits at the start and the joins (one row over 500 slots 6.0 us, over 1000 7.7,
// over 4095, in shares, 9.0).
static constexpr int PAGED_WAVES = 8;
static_assert(64 * PAGED_WAVES <= PAGED_MOST_THREADS);

template <int HD, int JT>
__device__ __forceinline__ void paged_scores(f32x4 (&S)[JT][2], const i32x4 (&k)[HD / 16], const i32x4 (&Q)[JT][HD / 32]) {
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            S[j][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < HD / 32; ++u) S[j][h] = mfma_step<ET_BF16>(k[h * (HD / 32) + u], Q[j][u], S[j][h]);
        }
}

template <int HD, int JT, int TERMS>
__global__ void __launch_bounds__(64 * PAGED_WAVES, 2) k_paged_attn(const PagedAttnArgs a, float c) {
    constexpr int UD = HD / 32, DG = HD / 4, NDT = HD / 16, RS = HD + 4, W = PAGED_WAVES, R = 16 * JT;
    const PagedBatch& p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4, G = a.G;
    const int kvh = blockIdx.x % p.Hkv;
    const PagedShare sh = paged_share<false>(a, R, blockIdx.x / p.Hkv);
    if (!sh.found) return;
    const PagedSeq& s = sh.s;
    const bool tree = a.anc != nullptr;
    const int qt = sh.local % sh.nq, split = sh.local / sh.nq;
    auto token = [&](int x) { return a.by_G(x); };
    const int rows = s.T * G, p0 = qt * R;
    const int t0 = token(p0), t1 = token(min(p0 + R, rows) - 1) + 1;

    __shared__ float sm_m[W][16], sm_l[W][16];
    __shared__ __attribute__((aligned(16))) float sm_o[W][16][RS];
    AttnState<HD> st[JT];
#pragma unroll
    for (int j = 0; j < JT; ++j) st[j].clear();
    if (s.fits) {
        i32x4 Q[JT][UD];
        int tok[JT];
        uint64_t an[JT][2];
#pragma unroll
        for (int j = 0; j < JT; ++j) {
            const int x = min(p0 + 16 * j + r, rows - 1);
            tok[j] = token(x);
            const size_t row = (size_t)(s.row0 + tok[j]);
            const uint16_t* q = a.q + (row * a.H + kvh * G + (x - tok[j] * G)) * HD + g * DG;
#pragma unroll
            for (int u = 0; u < UD; ++u) Q[j][u] = *(const i32x4*)(q + u * 8);
            an[j][0] = tree ? a.anc[2 * row] : 0;
            an[j][1] = tree ? a.anc[2 * row + 1] : 0;
        }
        const PagedRange rg(s, t0, t1, tree, a.sink, a.window);
        const int lo = (int)((int64_t)rg.n_log * split / sh.ns), n = (int)((int64_t)rg.n_log * (split + 1) / sh.ns) - lo;
        const int w0 = lo + n * wave / W, w1 = lo + n * (wave + 1) / W;
        // A tile's fragments, keys and values apart: the next tile's keys are loaded
        // once this one's scores are there, its values after the product with them.
        const uint32_t tmask = (1u << p.tshift) - 1, vtiles = (uint32_t)p.Hkv << p.tshift;
        i32x4 kf[NDT], vf[NDT];
        int tile, pid;
        uint32_t at;
        auto look_up = [&](int lt) {
            tile = rg.phys(lt);
            pid = paged_page(p, s.b, tile);
        };
        auto load_k = [&] {
            const uint32_t pg = (uint32_t)pid < (uint32_t)p.n_pages ? (uint32_t)pid : 0u;
            at = ((pg * (2 * p.Hkv) + kvh) << p.tshift) + ((uint32_t)tile & tmask);
            const uint16_t* k = p.pages + (size_t)at * (32 * HD);
#pragma unroll
            for (int f = 0; f < NDT; ++f) kf[f] = *(const i32x4*)(k + f * 512 + lane * 8);
        };
        auto load_v = [&] {
            const uint16_t* v = p.pages + (size_t)(at + vtiles) * (32 * HD);
#pragma unroll
            for (int f = 0; f < NDT; ++f) vf[f] = *(const i32x4*)(v + f * 512 + lane * 8);
        };
        auto V = [&](int m, i32x4 (&f)[2]) {
            f[0] = vf[2 * m];
            f[1] = vf[2 * m + 1];
        };
        uint32_t vm[JT];
        f32x4 S[JT][2];
        if (w0 < w1) {
            look_up(w0);
            load_k();
            load_v();
        }
        for (int lt = w0; lt < w1;) {
            while (rg.whole(tile) && (uint32_t)pid < (uint32_t)p.n_pages) {
                look_up(min(lt + 1, w1 - 1));
                paged_scores<HD, JT>(S, kf, Q);
                load_k();
                attn_step<HD, JT, false, false, TERMS>(st, S, c, V, vm, [] {});
                load_v();
                if (++lt >= w1) break;
            }
            mfma_result_pad();
            if (lt >= w1) break;
            paged_scores<HD, JT>(S, kf, Q);
            mfma_result_pad();
#pragma unroll
            for (int j = 0; j < JT; ++j)
                vm[j] = paged_vis8(s, tok[j], tile * 32 + 8 * g, tree, an[j][0], an[j][1], a.sink, a.window);
            paged_end<HD, JT, TERMS>(st, S, vf, vm, (uint32_t)pid >= (uint32_t)p.n_pages, c);
            mfma_result_pad();
            if (++lt < w1) {
                look_up(lt);
                load_k();
                load_v();
            }
        }
    }

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
        for (int dt = 0; dt < NDT; ++dt) *(f32x4*)(&sm_o[wave][r][16 * dt + 4 * g]) = st[j].O[dt];
        __syncthreads();
        for (int idx = threadIdx.x; idx < 16 * D4; idx += 64 * W) {
            const int rr = idx / D4, d4 = (idx % D4) * 4, x = p0 + 16 * j + rr;
            if (x >= rows) continue;
            float mw[W], M = -INFINITY;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                mw[w] = sm_m[w][rr];
                M = fmaxf(M, mw[w]);
            }
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            float L = s.fits ? 0.f : NAN;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float f = __builtin_amdgcn_exp2f(mw[w] - M);
                attn_merge_o(acc, *(const f32x4*)(&sm_o[w][rr][d4]), f);
                attn_merge_l(L, sm_l[w][rr], f);
            }
            if (sh.ns == 1) {
                const float inv = L != 0.f ? 1.f / L : 0.f;  // no slot seen: 0 (a NaN sum stays one)
                const int t = token(x);
                st4(a.out, ((size_t)(s.row0 + t) * a.H + kvh * G + (x - t * G)) * HD + d4, acc[0] * inv, acc[1] * inv,
                    acc[2] * inv, acc[3] * inv);
            } else {
                const size_t o = ((size_t)(sh.part + sh.local) * p.Hkv + kvh) * R + 16 * j + rr;
                *(f32x4*)(a.part_o + o * HD + d4) = acc;
                if (d4 == 0) *(float2*)(a.part_ml + o * 2) = make_float2(M, L);
            }
        }
    }
}

// ---------------------------------------------------------------- attention: many rows

// Workgroup = (share of a unit of 128 packed rows, kv head): four waves of two
// 16-row query tiles each.  The share's key tiles pass through LDS in a ring of
// four, keys one tile ahead of the values, with direct-to-LDS loads (the
// fragments lie in memory as the MFMA reads them: no swizzle, no conflict), two
// tiles a stage, one barrier per stage.  A tile's scores are computed under the
// exponentials of the one before it.
//
// What bounds it: the matrix cores, at the rate that a large product reaches: 2048
// rows of 8B heads behind 6001 slots, 236 GFLOP, 204 us, 1154 TFLOP/s (one tile a
// stage, in the compiler's order, 294; 256 rows, four query tiles per wave, 372).
// Two workgroups share a CU: a tile takes one 0.87 us beside another, 0.57 alone.
static constexpr int PROWS_WAVES = 4, PROWS_JT = 2, PROWS_R = 16 * PROWS_JT * PROWS_WAVES, PROWS_D = 4;

template <int HD>
__global__ void __launch_bounds__(64 * PROWS_WAVES, 2) k_paged_rows(const PagedAttnArgs a, float c) {
    constexpr int UD = HD / 32, DG = HD / 4, NDT = HD / 16, JT = PROWS_JT, R = PROWS_R, D = PROWS_D;
    __shared__ i32x4 sk[D * NDT * 64], sv[D * NDT * 64];
    const PagedBatch& p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4, G = a.G;
    const int kvh = blockIdx.x % p.Hkv;
    const PagedShare sh = paged_share<false>(a, R, blockIdx.x / p.Hkv);
    if (!sh.found) return;
    const PagedSeq& s = sh.s;
    const bool tree = a.anc != nullptr;
    // The last rows see the most slots: their shares start first.  Where all of a
    // sequence's run at once, two to a CU, the second half goes the other way, so
    // that a long one shares its CU with a short one (a prompt's first 2048 rows, 8B
    // heads: 54 us, else 57).
    const int split = sh.local / sh.nq, at = sh.local - split * sh.nq, half = (sh.nq + 1) / 2;
    const int qt = a.fold && at >= half ? at - half : sh.nq - 1 - at;
    auto token = [&](int x) { return a.by_G(x); };
    const int rows = s.T * G, p0 = qt * R, w0 = p0 + wave * 16 * JT;
    const bool live = w0 < rows && s.fits;

    AttnState<HD> st[JT];
    i32x4 Q[JT][UD];
    int tok[JT];
    uint64_t an[JT][2];
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        st[j].clear();
        const int x = min(w0 + 16 * j + r, rows - 1);
        tok[j] = token(x);
        const size_t row = (size_t)(s.row0 + tok[j]);
        const uint16_t* q = a.q + (row * a.H + kvh * G + (x - tok[j] * G)) * HD + g * DG;
#pragma unroll
        for (int u = 0; u < UD; ++u) Q[j][u] = *(const i32x4*)(q + u * 8);
        an[j][0] = tree ? a.anc[2 * row] : 0;
        an[j][1] = tree ? a.anc[2 * row + 1] : 0;
    }
    const PagedRange rg(s, token(p0), token(min(p0 + R, rows) - 1) + 1, tree, a.sink, a.window);
    // the wave's own rows
    const PagedRange wr(s, token(min(w0, rows - 1)), token(min(w0 + 16 * JT, rows) - 1) + 1, tree, a.sink, a.window);
    const int w_end = wr.pt0 + wr.n_log - wr.st;
    auto sees = [&](int tile) { return live && tile < w_end && (tile < wr.st || tile >= wr.pt0); };
    const int lo = s.fits ? (int)((int64_t)rg.n_log * split / sh.ns) : 0;
    const int n = s.fits ? (int)((int64_t)rg.n_log * (split + 1) / sh.ns) - lo : 0;
    if (n > 0) {
        // Two tiles a stage: the stage of step i (even) has the keys of i + 1 and i + 2
        // and the values of i and i + 1, a tile for each wave to load, one stage
        // ahead of its use.  A tile's keys are tile (pid 2 Hkv + kvh) 2^tshift + (tile
        // mod 2^tshift) of the pool, its values Hkv 2^tshift tiles on.
        const uint32_t tmask = (1u << p.tshift) - 1, head = (uint32_t)kvh + (wave & 1 ? (uint32_t)p.Hkv : 0u);
        auto tile_at = [&](int i) { return rg.phys(lo + min(i, n - 1)); };
        const int ahead = (wave & 1 ? 0 : 1) + (wave >> 1);  // the wave's tile of a stage: i + ahead
        const uint32_t ring = (wave & 1 ? lds_addr(sv) : lds_addr(sk));
        int mine = tile_at(ahead), pid = paged_page(p, s.b, mine);
        auto load = [&](int i) {  // tile i, by this wave
            const uint32_t pg = (uint32_t)pid < (uint32_t)p.n_pages ? (uint32_t)pid : 0u;
            const uint32_t at = ((pg * (2 * p.Hkv) + head) << p.tshift) + ((uint32_t)mine & tmask);
            lds_load_tile<NDT>((const char*)p.pages + (size_t)at * (NDT * 1024), lane * 16,
                               ring + ((uint32_t)i % D) * (NDT * 1024));
        };
        auto look_up = [&](int i) {  // the page of the wave's next tile, after step i's stage
            mine = tile_at(i + 2 + ahead);
            pid = paged_page(p, s.b, mine);
        };
        // whether a page of the share lies outside the pool: then every tile is looked at
        bool strange = false;
        for (int i = lane; i < n; i += 64)
            strange = strange || (uint32_t)p.table[(size_t)s.b * p.table_len + (rg.phys(lo + i) >> p.tshift)] >= (uint32_t)p.n_pages;
        strange = __any(strange);
        f32x4 S[JT][2], N[JT][2];
        auto scores = [&](f32x4 (&x)[JT][2], int i) {
            const i32x4* k = sk + ((uint32_t)i % D) * (NDT * 64) + lane;
            i32x4 kf[NDT];
#pragma unroll
            for (int f = 0; f < NDT; ++f) kf[f] = k[f * 64];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < UD; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < JT; ++j)
                        x[j][h] = mfma_step<ET_BF16>(kf[h * UD + u], Q[j][u], u ? x[j][h] : f32x4{0.f, 0.f, 0.f, 0.f});
        };
        auto advance = [&](int i) {
            stage_wait<0>();  // what was loaded is there, what was used is free
            if (i + 2 + ahead < n) load(i + 2 + ahead);
        };
        if (wave == 0) {  // the first keys, which no stage has
            const int pid0 = paged_page(p, s.b, tile_at(0));
            const uint32_t pg = (uint32_t)pid0 < (uint32_t)p.n_pages ? (uint32_t)pid0 : 0u;
            const uint32_t at = ((pg * (2 * p.Hkv) + kvh) << p.tshift) + ((uint32_t)tile_at(0) & tmask);
            lds_load_tile<NDT>((const char*)p.pages + (size_t)at * (NDT * 1024), lane * 16, lds_addr(sk));
        }
        load(ahead);
        look_up(0);
        // (the queries are here: no wait for them, which would be one for the loads in flight, in the loops)
#pragma unroll
        for (int j = 0; j < JT; ++j)
#pragma unroll
            for (int u = 0; u < UD; ++u) asm volatile("" : "+v"(Q[j][u]));
        stage_wait<0>();
        scores(S, 0);
        mfma_result_pad();
        // A whole tile: attn_step with the order of its instructions laid down.  x: its
        // scores, y: the next one's, t: a lane's largest of x, and then of y.  The
        // keys are read first, the values under them; the next tile's scores run
        // under this one's exponentials, its largest scores are taken under the
        // product with the values.  The scores and exponentials go before the product of
        // the other workgroup's wave (2048 rows behind 6001 slots 225 -> 211 us: the
        // waves of a SIMD fall out of step, one's exponentials under the other's
        // products).
        auto turn = [&](f32x4 (&x)[JT][2], f32x4 (&y)[JT][2], float (&t)[JT], int i, bool last) {
            const i32x4* k = sk + ((uint32_t)(i + 1) % D) * (NDT * 64) + lane;
            const i32x4* v = sv + ((uint32_t)i % D) * (NDT * 64) + lane;
            i32x4 kf[NDT], vf[NDT];
#pragma unroll
            for (int f = 0; f < NDT; ++f) kf[f] = k[f * 64];
            bool grow = false;
#pragma unroll
            for (int j = 0; j < JT; ++j) grow = grow || t[j] > st[j].top;
            if (__any(grow)) {
                mfma_result_pad();
#pragma unroll
                for (int j = 0; j < JT; ++j) attn_follow(st[j], t[j], c);
            }
#pragma unroll
            for (int f = 0; f < NDT; ++f) vf[f] = v[f * 64];
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int u = 0; u < UD; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < JT; ++j)
                        y[j][h] = mfma_step<ET_BF16>(kf[h * UD + u], Q[j][u], u ? y[j][h] : f32x4{0.f, 0.f, 0.f, 0.f});
            i32x4 P[JT][1];
#pragma unroll
            for (int j = 0; j < JT; ++j) attn_probs(P[j], x[j], st[j].mc, st[j].c);
#pragma unroll
            for (int f = 0; f < NDT * JT; ++f) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
            }
            // (here: a scalar load in flight makes every LDS read's wait one for all of them)
            if (last) look_up(i + 1);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
            const int one = 0x3f803f80;
#pragma unroll
            for (int j = 0; j < JT; ++j) st[j].l = mfma_step<ET_BF16>(i32x4{one, one, one, one}, P[j][0], st[j].l);
#pragma unroll
            for (int f = 0; f < NDT; ++f)
#pragma unroll
                for (int j = 0; j < JT; ++j) st[j].O[f] = mfma_step<ET_BF16>(vf[f], P[j][0], st[j].O[f]);
            paged_tops<JT>(t, y);
#pragma unroll
            for (int f = 0; f < (NDT + 1) * JT; ++f) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        // A tile at the ends of a walk.
        auto turn_end = [&](int i) {
            const i32x4* v = sv + ((uint32_t)i % D) * (NDT * 64) + lane;
            i32x4 vf[NDT];
#pragma unroll
            for (int f = 0; f < NDT; ++f) vf[f] = v[f * 64];
            __builtin_amdgcn_sched_barrier(0);
            const int tile = tile_at(i);
            uint32_t vm[JT];
#pragma unroll
            for (int j = 0; j < JT; ++j)
                vm[j] = paged_vis8(s, tok[j], tile * 32 + 8 * g, tree, an[j][0], an[j][1], a.sink, a.window);
            paged_end<HD, JT, 1>(st, S, vf, vm, strange && (uint32_t)paged_page(p, s.b, tile) >= (uint32_t)p.n_pages, c);
            mfma_result_pad();
        };
        // two tiles that every row of the workgroup sees whole
        auto plain = [&](int i) { return i + 1 < n && rg.whole(tile_at(i)) && rg.whole(tile_at(i + 1)) && !strange; };
        for (int i = 0; i < n;) {
            float top[JT];
            paged_tops<JT>(top, S);
            while (plain(i)) {
                advance(i);
                turn(S, N, top, i, false);
                turn(N, S, top, i + 1, true);
                i += 2;
            }
            mfma_result_pad();
            if (i >= n) break;
            advance(i);
#pragma unroll 1
            for (const int end = i + 2; i < end; ++i) {
                if (i < n && sees(tile_at(i))) turn_end(i);
                scores(S, i + 1);
                mfma_result_pad();
            }
            look_up(i);
        }
        stage_wait<0>();  // (no load outlives the workgroup's LDS)
    }
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        const int x = w0 + 16 * j + r;
        if (x >= rows) continue;
        const float L = s.fits ? st[j].l[0] : NAN;
        if (sh.ns == 1) {
            const float inv = L != 0.f ? 1.f / L : 0.f;  // no slot seen: 0 (a NaN sum stays one)
            uint16_t* o = a.out + ((size_t)(s.row0 + tok[j]) * a.H + kvh * G + (x - tok[j] * G)) * HD + 4 * g;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
                *(uint2*)(o + 16 * dt) = make_uint2(pack_bf(st[j].O[dt][0] * inv, st[j].O[dt][1] * inv),
                                                    pack_bf(st[j].O[dt][2] * inv, st[j].O[dt][3] * inv));
        } else {
            const size_t at = ((size_t)(sh.part + split * sh.nq + qt) * p.Hkv + kvh) * R + x - p0;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) *(f32x4*)(a.part_o + at * HD + 16 * dt + 4 * g) = st[j].O[dt];
            if (g == 0) *(float2*)(a.part_ml + at * 2) = make_float2(st[j].m * c, L);
        }
    }
}

// The join of the shares of split units: hd / 4 threads per row and group; the
// groups take a row each, or with many shares up to eight take every eighth
// share of a row, four at a time, and join through LDS.  Bound by latency: each
// workgroup sums the sequences' lengths (paged_share), then reads its rows once.
// Small workgroups, a unit's over y: with 1024 threads each, units of 16 rows
// took a microsecond more, and 15 shares of 128 rows 3 us more.
static constexpr int PMERGE_THREADS = 256;
template <int HD> __global__ void __launch_bounds__(PMERGE_THREADS) k_paged_merge(const PagedAttnArgs a, int R) {
    constexpr int D4 = HD / 4, NG = PMERGE_THREADS / D4;
    __shared__ float2 sm_ml[NG];
    __shared__ f32x4 sm_o[NG][D4];
    const PagedBatch& p = a.p;
    const int kvh = blockIdx.x % p.Hkv, G = a.G;
    // (one wave looks: up to eight workgroups share a CU)
    __shared__ PagedShare sm_sh;
    if (threadIdx.x < 64) {
        const PagedShare found = paged_share<true>(a, R, blockIdx.x / p.Hkv);
        if (threadIdx.x == 0) sm_sh = found;
    }
    __syncthreads();
    const PagedShare sh = sm_sh;
    if (!sh.found) return;
    const int ns = sh.ns, NS = ns > 16 ? 8 : ns > 8 ? 4 : ns > 4 ? 2 : 1;
    const int gi = threadIdx.x / D4, d4 = threadIdx.x % D4 * 4, sub = gi % NS;
    const int p0 = sh.local * R, rows = min(sh.s.T * G - p0, R);
    for (int i0 = blockIdx.y * (NG / NS); i0 < rows; i0 += gridDim.y * (NG / NS)) {  // (the same for every thread)
        const int i = min(i0 + gi / NS, rows - 1);
        float M = -FLT_MAX, L = 0.f;
        f32x4 acc[1] = {{0.f, 0.f, 0.f, 0.f}};
        for (int k0 = sub; k0 < ns; k0 += 4 * NS) {
            float2 ml[4];
            f32x4 po[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int sp = min(k0 + k * NS, ns - 1);
                const size_t o = ((size_t)(sh.part + sp * sh.nq + sh.local) * p.Hkv + kvh) * R + i;
                ml[k] = *(const float2*)(a.part_ml + o * 2);
                po[k] = *(const f32x4*)(a.part_o + o * HD + d4);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k0 + k * NS < ns) {
                    const f32x4 o[1] = {po[k]};
                    attn_merge_split<1>(acc, L, M, o, ml[k].y, ml[k].x);
                }
        }
        if (NS > 1) {
            if (d4 == 0) sm_ml[gi] = make_float2(M, L);
            sm_o[gi][d4 / 4] = acc[0];
            __syncthreads();
            if (sub == 0)
                for (int k = 1; k < NS; ++k) {
                    const f32x4 o[1] = {sm_o[gi + k][d4 / 4]};
                    attn_merge_split<1>(acc, L, M, o, sm_ml[gi + k].y, sm_ml[gi + k].x);
                }
        }
        if (sub == 0 && i0 + gi / NS < rows) {
            const float inv = L != 0.f ? 1.f / L : 0.f;
            const int x = p0 + i, t = a.by_G(x);
            st4(a.out, ((size_t)(sh.s.row0 + t) * a.H + kvh * G + (x - t * G)) * HD + d4, acc[0][0] * inv,
                acc[0][1] * inv, acc[0][2] * inv, acc[0][3] * inv);
        }
        if (NS > 1) __syncthreads();
    }
}

// Packed rows of a unit, the shares aimed at and the least tiles of one.
// 16, 32 or 128 rows.  The caches of 8 sequences at 4000 slots, 32 heads, read by 48
// rows: 117 us in units of 32, 108 of 128, since the keys and values go to every 32
// rows again.  But where the units of 32 rows leave CUs free, a workgroup of eight
// waves, each with every eighth key tile, is done sooner: 64 rows on one sequence of
// 4000 slots, 8 heads, 14 us of 32 and 19 of 128, at 64000 slots 48 and 57; 256 rows
// at 1000 slots 14 and 17, at 8000 22 and 27, at 64000 97 and 87.
// Not split: calls whose sequences have up to 32 tiles on 16 rows (one of 1000 slots
// 7.5 us, in two shares 9.6), up to 16 on more (128 rows behind 300 slots 11.7 us,
// split 13.3): a split costs the second kernel's 2.6 us even if it finds nothing,
// which a table that allows no longer sequence saves too.
// Probabilities go into the product with the values in two bf16 terms where a sequence
// has up to 32 packed rows, as in the decoder's attention, and in one where it has more.
// Up to 32 rows wait for memory: the second term takes 32 decoding sequences 53.5 ->
// 53.9 us, one row at 131072 slots nothing, at 500 5.9 -> 6.0, 64 sequences of up to
// 300 8.7 -> 9.1, draft trees of 8 conversations 32.0 -> 32.8.  More rows wait for the
// matrix cores: 256 at 8000 slots 23 -> 25.4, a chunk of 509 rows among 8 decoding
// sequences 65.5 -> 84.5, 2048 rows behind 6001 slots 211 -> 287.  Against 64 bits
// an output is off by 0.0016 of the norm in two terms, its own rounding, by 0.0023 in one.
static constexpr int PAGED_CUS = 256;

PagedPlan paged_plan(const PagedBatch& p, int H, int max_rows) {
    PagedPlan q;
    const int64_t most = (int64_t)std::min(max_rows, p.N) * (H / p.Hkv);  // packed rows of a sequence
    const bool few = ((int64_t)p.N * (H / p.Hkv) / 32 + p.B) * p.Hkv <= PAGED_CUS;
    q.R = most <= 16 ? 16 : most <= 32 || (few && (most <= 64 || p.cap <= 8192)) ? 32 : PROWS_R;
    q.terms = most <= 32 ? 2 : 1;
    q.units = (int)(((int64_t)p.N * (H / p.Hkv)) / q.R) + p.B;
    q.target = (PAGED_CUS * (q.R == PROWS_R ? 2 : 1) + p.Hkv - 1) / p.Hkv;
    q.whole = q.R == 16 ? 32 : 16;
    if ((p.cap >> 5) <= q.whole) q.target = 0;  // no sequence is split
    q.work = q.target ? (size_t)2 * q.target * p.Hkv * q.R * (p.hd + 2) * sizeof(float) : 0;
    return q;
}

template <int HD> static hipError_t paged_attn_go(const PagedAttnArgs& a, const PagedPlan& q, float c, hipStream_t s) {
    const PagedBatch& p = a.p;
    const dim3 grid((unsigned)paged_attn_grid(p, q));
    hipError_t e = q.R == 16   ? launch_checked(k_paged_attn<HD, 1, 2>, grid, 64 * PAGED_WAVES, s, a, c)
                   : q.R == 32 ? launch_checked(q.terms == 2 ? k_paged_attn<HD, 2, 2> : k_paged_attn<HD, 2, 1>, grid,
                                                64 * PAGED_WAVES, s, a, c)
                               : launch_checked(k_paged_rows<HD>, grid, 64 * PROWS_WAVES, s, a, c);
    if (e != hipSuccess || q.target == 0) return e;
    const unsigned units = (unsigned)std::min(q.units, q.target);
    // As many workgroups as the chip holds by half, where the units are few (most of
    // the bound may find nothing to do, and each has to look: with 64 for each of
    // 512 units this kernel took 36 us); four for 128 rows, where they are many (one:
    // 80 us instead of 72 for a chunk of 509 rows among 8 decoding sequences).
    const unsigned y = std::max(q.R == PROWS_R ? 4u : 1u, std::min(std::min(32u, (unsigned)q.R), 1024u / (units * p.Hkv)));
    return launch_checked(k_paged_merge<HD>, dim3(units * p.Hkv, y), PMERGE_THREADS, s, a, q.R);
}

hipError_t launch_attention_paged(const PagedAttnArgs& args, const PagedPlan& q, hipStream_t s) {
    PagedAttnArgs a = args;
    const PagedBatch& p = a.p;
    if (p.N < 1 || p.B < 1 || p.Hkv < 1 || a.H % p.Hkv) return hipErrorInvalidValue;
    a.G = a.H / p.Hkv;
    a.by_G = Quotient(a.G);
    a.target = q.target;
    a.single = q.R == PROWS_R ? (PAGED_CUS + p.Hkv - 1) / p.Hkv : 0;
    a.whole = q.whole;
    a.fold = (int64_t)(q.units - p.B) * p.Hkv <= 2 * PAGED_CUS;
    a.part_ml = a.part_o + (size_t)2 * q.target * p.Hkv * q.R * p.hd;
    const float c = (1.0f / sqrtf((float)p.hd)) * 1.4426950408889634f;
    if (p.hd == 128) return paged_attn_go<128>(a, q, c, s);
    if (p.hd == 64) return paged_attn_go<64>(a, q, c, s);
    return hipErrorInvalidValue;
}

}  // namespace cas
