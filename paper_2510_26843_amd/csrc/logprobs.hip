// gfx950 kernels of token scoring: log probabilities of given tokens, entropy
// and top alternatives of rows of logits.
//
// With M a row's largest logit and l_v = scale (x_v - M):
//   S = sum e^{l_v},  logp_t = l_t - log S,  entropy = log S - sum e^{l_v} l_v / S.
// A row is read once, by one workgroup or, where there are few rows, in parts by
// several; a part is walked in chunks that the workgroup holds in registers (the
// next one in flight), each wave with a running maximum, S and U = sum e^l l of
// its own.  Exponents are in log2 units.
//
// The K best: a wave keeps a list (in LDS) of what may be among its K best.  The
// K-th largest of its 64 lanes' running maxima bounds its K-th best from below,
// and closely (the 20th lane is about the 24th logit), so after the first chunk
// few logits pass it; when the list fills up the bound is taken again and the
// list sifted.  Equal logits can defeat it: then the list is cut to its K best by
// rank, and a chunk with too many of them gives its K best one after another.
// The lists are joined by rank, over the waves and then over a row's parts.
// Every list is sorted by (logit, id), so no order of arrival shows.
//
// What bounds it: for many rows the bytes (1501 rows of 128256 fp32 logits, 20
// alternatives); for one row the latency of its two kernels.
#include "attn_step.h"

#include <algorithm>

namespace cas {

static constexpr int LP_THREADS = 256, LP_WAVES = LP_THREADS / 64, LP_MAX_K = 32;
static constexpr int LP_LIST = 256;  // entries of a wave's list
static constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ bool lp_better(float a, int ia, float b, int ib) { return a > b || (a == b && ia < ib); }
__device__ __forceinline__ float lp_lane(float x, int l) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), l));
}

// The K-th largest of the lanes' values (no NaN), the same for every lane.
__device__ __forceinline__ float lp_kth(float x, int K) {
    const int lane = threadIdx.x & 63;
    int above = 0;
#pragma unroll 8
    for (int l = 0; l < 64; ++l) {
        const float o = lp_lane(x, l);
        above += o > x || (o == x && l < lane) ? 1 : 0;
    }
    return lp_lane(x, __builtin_ctzll(__ballot(above == K - 1)));
}

// The K best of a wave's list of n, in order, to its front (fewer: all, in
// order); returns their number.
__device__ __forceinline__ int lp_rank(float* v, int* id, int n, int K) {
    const int lane = threadIdx.x & 63;
    float x[LP_LIST / 64];
    int xi[LP_LIST / 64], rank[LP_LIST / 64];
#pragma unroll
    for (int q = 0; q < LP_LIST / 64; ++q) {
        const int i = q * 64 + lane;
        x[q] = i < n ? v[i] : -INFINITY;
        xi[q] = i < n ? id[i] : 0x7fffffff;
        rank[q] = 0;
    }
    for (int j = 0; j < n; ++j) {  // (broadcast reads)
        const float o = v[j];
        const int oi = id[j];
#pragma unroll
        for (int q = 0; q < LP_LIST / 64; ++q) rank[q] += lp_better(o, oi, x[q], xi[q]) ? 1 : 0;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int q = 0; q < LP_LIST / 64; ++q)
        if (q * 64 + lane < n && rank[q] < K) {
            v[rank[q]] = x[q];
            id[rank[q]] = xi[q];
        }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return min(n, K);
}

// Drops what is below tau from a wave's list of n.
__device__ __forceinline__ int lp_sift(float* v, int* id, int n, float tau) {
    const int lane = threadIdx.x & 63;
    int kept = 0;
    for (int i0 = 0; i0 < n; i0 += 64) {
        const int i = i0 + lane;
        const float x = i < n ? v[i] : -INFINITY;
        const int xi = i < n ? id[i] : 0;
        const bool keep = i < n && x >= tau;
        const uint64_t m = __ballot(keep);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (keep) {
            const int to = kept + __popcll(m & (((uint64_t)1 << lane) - 1));
            v[to] = x;
            id[to] = xi;
        }
        kept += __popcll(m);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return kept;
}

// A row's running sums relative to its largest logit.
struct LpSums {
    float m, s, u;  // log2 units but for m
    __device__ __forceinline__ float ref() const { return m == -INFINITY ? 0.f : m; }
    // relative to a larger m
    __device__ __forceinline__ void lift(float mn, float c) {
        const float d = m == -INFINITY ? 0.f : fmaxf((m - mn) * c, -1e30f), f = __builtin_amdgcn_exp2f(d);
        u = fmaf(d, s, u) * f;
        s *= f;
        m = mn;
    }
};

// What a row gives from its sums: a token's log probability is (x - m) scale -
// log_s.  A row with a NaN, an infinite logit or no finite one has none.
struct LpRow {
    float m, log_s, entropy;
    bool none;
    __device__ __forceinline__ LpRow(const LpSums& t) {
        none = !(t.s > 0.f && t.s < INFINITY) || !(fabsf(t.m) < INFINITY);
        m = t.m;
        log_s = none ? NAN : logf(t.s);
        entropy = log_s - t.u / t.s * LN2;
    }
    __device__ __forceinline__ float logp(float x, float scale) const { return (x - m) * scale - log_s; }
};
__device__ __forceinline__ float lp_logit(const LogprobArgs& a, int row, int t) {
    const size_t o = (size_t)row * a.ld + t;
    return a.bf16 ? bf2f(((const uint16_t*)a.x)[o]) : ((const float*)a.x)[o];
}
template <int THREADS> __device__ __forceinline__ void lp_tokens(const LogprobArgs& a, int row, const LpRow& r) {
    if (threadIdx.x == 0 && a.entropy) a.entropy[row] = r.entropy;
    for (int j = threadIdx.x; j < a.m; j += THREADS) {
        const int t = a.tokens[(size_t)row * a.m + j];
        a.logp[(size_t)row * a.m + j] = t >= 0 && t < a.V ? r.logp(lp_logit(a, row, t), a.scale) : NAN;
    }
}

// A part's record: m, s, u, and its K best: values, then ids.
static int lp_words(int K) { return 4 + 2 * K; }

// Workgroup = (row, part): chunks [part span, (part + 1) span) of EACH logits per
// thread.  One part: it gives the row's results itself.
template <bool BF16, int EACH>
__global__ void __launch_bounds__(LP_THREADS) k_logprob_part(const LogprobArgs a, int parts, int span, int words) {
    constexpr int E = BF16 ? 8 : 4, NV = EACH / E, CHUNK = LP_THREADS * EACH, W = LP_WAVES;
    struct __attribute__((packed, aligned(BF16 ? 2 : 4))) Piece { i32x4 v; };
    __shared__ float sm_v[W][LP_LIST], sm_sum[W][3];
    __shared__ int sm_i[W][LP_LIST], sm_n[W];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = blockIdx.x % parts, row = blockIdx.x / parts, K = a.K;
    const int begin = part * span * CHUNK, end = min(a.V, begin + span * CHUNK);
    const char* x0 = (const char*)a.x + (size_t)row * a.ld * (BF16 ? 2 : 4);
    const float c = a.scale * LOG2E;
    float *v = sm_v[wave], lm = -INFINITY, tau = -INFINITY;
    int *id = sm_i[wave], n = 0;
    LpSums t = {-INFINITY, 0.f, 0.f};  // (s and u: the lane's)
    auto load = [&](i32x4 (&r)[NV], int base) {  // pieces that lie in the part as a whole
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int o = base + (i * LP_THREADS + (int)threadIdx.x) * E;
            if constexpr (BF16) r[i] = i32x4{(int)0xff80ff80, (int)0xff80ff80, (int)0xff80ff80, (int)0xff80ff80};
            else r[i] = i32x4{(int)0xff800000, (int)0xff800000, (int)0xff800000, (int)0xff800000};
            if (o + E <= end) r[i] = ((const Piece*)(x0 + (size_t)o * (BF16 ? 2 : 4)))->v;
        }
    };
    i32x4 raw[NV];
    load(raw, begin);
    for (int base = begin; base < end; base += CHUNK) {
        float x[EACH + 1];
#pragma unroll
        for (int e = 0; e < EACH; ++e) x[e] = piece_val<std::conditional_t<BF16, uint16_t, float>>(raw[e / E], e % E);
        // the logits past the last whole piece: one for each of the first threads
        x[EACH] = -INFINITY;
        const int odd = end - end % E;  // (a part ends at a chunk's end or the row's)
        if (base + CHUNK >= end && odd + (int)threadIdx.x < end)
            x[EACH] = BF16 ? bf2f(((const uint16_t*)x0)[odd + threadIdx.x]) : ((const float*)x0)[odd + threadIdx.x];
        if (base + CHUNK < end) load(raw, base + CHUNK);
        float cm = -INFINITY;  // (fmaxf passes over NaN: s finds it)
#pragma unroll
        for (int e = 0; e <= EACH; ++e) cm = fmaxf(cm, x[e]);
        lm = fmaxf(lm, cm);
        const float wm = wave_max(cm);
        if (wm > t.m) t.lift(wm, c);
        const float ref = t.ref();
#pragma unroll
        for (int e = 0; e <= EACH; ++e) {
            const float l = (x[e] - ref) * c, p = __builtin_amdgcn_exp2f(l);
            t.s += p;
            t.u = fmaf(p, fmaxf(l, -1e30f), t.u);  // (nothing where p is 0)
        }
        if (K > 0) {
            if (base == begin) tau = lp_kth(lm, K);
            if (wm >= tau && wm > -INFINITY) {
                auto id_of = [&](int e) {
                    return e == EACH ? odd + (int)threadIdx.x : base + ((e / E) * LP_THREADS + (int)threadIdx.x) * E + e % E;
                };
                int mine, upto, all;  // the lane's candidates, those up to its own, the wave's
                auto count = [&] {
                    mine = 0;
                    if (cm >= tau) {
#pragma unroll
                        for (int e = 0; e <= EACH; ++e) mine += x[e] >= tau && x[e] > -INFINITY ? 1 : 0;
                    }
                    upto = mine;
#pragma unroll
                    for (int o = 1; o < 64; o <<= 1) {
                        const int y = __shfl_up(upto, o);
                        upto += lane >= o ? y : 0;
                    }
                    all = __builtin_amdgcn_readlane(upto, 63);
                };
                for (int pass = 0;; ++pass) {
                    count();
                    if (n + all <= LP_LIST || pass) break;
                    tau = lp_kth(lm, K);
                    n = lp_sift(v, id, n, tau);
                    if (n > LP_LIST / 2) n = lp_rank(v, id, n, K);
                }
                if (n + all <= LP_LIST) {
                    int to = n + upto - mine;
                    if (mine) {
#pragma unroll
                        for (int e = 0; e <= EACH; ++e)
                            if (x[e] >= tau && x[e] > -INFINITY) {
                                v[to] = x[e];
                                id[to++] = id_of(e);
                            }
                    }
                    n += all;
                } else {  // the chunk's K best, one after another
                    if (n > LP_LIST - LP_MAX_K) n = lp_rank(v, id, n, K);
                    float pv = INFINITY;
                    int pi = -1;
                    for (int k = 0; k < K; ++k) {
                        float bv = -INFINITY;
                        int bi = 0x7fffffff;
#pragma unroll
                        for (int e = 0; e <= EACH; ++e)
                            if (lp_better(pv, pi, x[e], id_of(e)) && lp_better(x[e], id_of(e), bv, bi)) {
                                bv = x[e];
                                bi = id_of(e);
                            }
#pragma unroll
                        for (int o = 32; o >= 1; o >>= 1) {
                            const float ov = __shfl_xor(bv, o);
                            const int oi = __shfl_xor(bi, o);
                            if (lp_better(ov, oi, bv, bi)) {
                                bv = ov;
                                bi = oi;
                            }
                        }
                        if (bi == 0x7fffffff) break;
                        if (lane == 0) {
                            v[n] = bv;
                            id[n] = bi;
                        }
                        ++n;
                        pv = bv;
                        pi = bi;
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
        }
    }
    if (K > 0) {
        n = lp_sift(v, id, n, lp_kth(lm, K));
        n = lp_rank(v, id, n, K);
    }
    // ---- join the waves
    t.s = wave_sum(t.s);
    t.u = wave_sum(t.u);
    if (lane == 0) {
        sm_sum[wave][0] = t.m;
        sm_sum[wave][1] = t.s;
        sm_sum[wave][2] = t.u;
        sm_n[wave] = n;
    }
    __syncthreads();
    LpSums r = {-INFINITY, 0.f, 0.f};
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, sm_sum[w][0]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        LpSums q = {sm_sum[w][0], sm_sum[w][1], sm_sum[w][2]};
        q.lift(m, c);
        r.s += q.s;
        r.u += q.u;
    }
    r.m = m;
    const LpRow out(r);
    float* rec = a.work + (size_t)blockIdx.x * words;
    if (parts == 1) {
        lp_tokens<LP_THREADS>(a, row, out);
    } else if (threadIdx.x == 0) {
        rec[0] = r.m;
        rec[1] = r.s;
        rec[2] = r.u;
    }
    if (K > 0) {
        float* best = parts == 1 ? a.best + (size_t)row * K : rec + 4;
        int* ids = parts == 1 ? a.ids + (size_t)row * K : (int*)rec + 4 + K;
        int total = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) total += sm_n[w];
        // a wave's entries count those of all lists that are better
        if (lane < n) {
            const float y = v[lane];
            const int yi = id[lane];
            int rank = 0;
#pragma unroll
            for (int w = 0; w < W; ++w)
                for (int j = 0; j < sm_n[w]; ++j) rank += lp_better(sm_v[w][j], sm_i[w][j], y, yi) ? 1 : 0;
            if (rank < K) {
                best[rank] = parts > 1 ? y : out.none ? NAN : out.logp(y, a.scale);
                ids[rank] = parts == 1 && out.none ? -1 : yi;
            }
        }
        for (int i = total + (int)threadIdx.x; i < K; i += LP_THREADS) {  // fewer than K finite logits
            best[i] = parts == 1 && out.none ? NAN : -INFINITY;
            ids[i] = -1;
        }
    }
}

// One wave = one row in parts: their sums by a butterfly, the best of their
// bests, and the tokens asked for.
__global__ void __launch_bounds__(64) k_logprob_join(const LogprobArgs a, int parts, int words) {
    extern __shared__ float sm[];  // [parts * K] values, then ids
    const int row = blockIdx.x, lane = threadIdx.x, K = a.K;
    const float* rec = a.work + (size_t)row * parts * words;
    const float c = a.scale * LOG2E;
    LpSums t = {-INFINITY, 0.f, 0.f};
    float tau = -INFINITY;  // every part's K-th best is no better than the row's
    for (int k = lane; k < parts; k += 64) {
        const float* q = rec + (size_t)k * words;
        LpSums p = {q[0], q[1], q[2]};
        if (K > 0) tau = fmaxf(tau, q[3 + K]);
        const float m = fmaxf(t.m, p.m);
        t.lift(m, c);
        p.lift(m, c);
        t.s += p.s;
        t.u += p.u;
    }
    const float m = wave_max(t.m);
    t.lift(m, c);
    t.s = wave_sum(t.s);
    t.u = wave_sum(t.u);
    const LpRow out(t);
    lp_tokens<64>(a, row, out);
    if (K == 0) return;
    tau = wave_max(tau);
    float *best = a.best + (size_t)row * K, *v = sm;
    int *ids = a.ids + (size_t)row * K, *id = (int*)(sm + (size_t)parts * K), n = 0;
    for (int i0 = 0; i0 < parts * K; i0 += 64) {
        const int i = min(i0 + lane, parts * K - 1);
        const float* q = rec + (size_t)(i / K) * words + 4;
        const float x = q[i % K];
        const int xi = ((const int*)q)[K + i % K];
        const bool keep = i0 + lane < parts * K && x >= tau && x > -INFINITY;
        const uint64_t in = __ballot(keep);
        if (keep) {
            const int to = n + __popcll(in & (((uint64_t)1 << lane) - 1));
            v[to] = x;
            id[to] = xi;
        }
        n += __popcll(in);
    }
    __syncthreads();
    for (int i = lane; i < n; i += 64) {
        const float x = v[i];
        const int xi = id[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += lp_better(v[j], id[j], x, xi) ? 1 : 0;
        if (rank < K) {
            best[rank] = out.none ? NAN : out.logp(x, a.scale);
            ids[rank] = out.none ? -1 : xi;
        }
    }
    for (int i = n + lane; i < K; i += 64) {
        best[i] = out.none ? NAN : -INFINITY;
        ids[i] = -1;
    }
}

// Chunks of 8192 logits, or of 2048 where a row's would leave the chip empty, and
// parts such that there are a few workgroups per CU.
struct LpPlan {
    int each, parts, span;
};
static LpPlan lp_plan(int n, int V) {
    LpPlan p;
    p.each = (int64_t)n * ((V + 8191) / 8192) >= 512 ? 32 : 8;
    const int chunk = LP_THREADS * p.each, chunks = (V + chunk - 1) / chunk;
    const int want = (int)std::min<int64_t>(chunks, std::max<int64_t>(1, 2048 / n));
    p.span = (chunks + want - 1) / want;
    p.parts = (chunks + p.span - 1) / p.span;
    return p;
}
size_t logprob_work_bytes(int n, int V, int K) {
    const LpPlan p = lp_plan(n, V);
    return std::max<size_t>(16, (size_t)n * p.parts * lp_words(K) * 4);
}

hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t s) {
    if (a.n < 1 || a.V < 1 || a.K < 0 || a.K > LP_MAX_K || a.m < 0) return hipErrorInvalidValue;
    const LpPlan p = lp_plan(a.n, a.V);
    const int words = lp_words(a.K);
    const dim3 grid((unsigned)a.n * p.parts);
    auto kernel = p.each == 32 ? (a.bf16 ? k_logprob_part<true, 32> : k_logprob_part<false, 32>)
                               : (a.bf16 ? k_logprob_part<true, 8> : k_logprob_part<false, 8>);
    const hipError_t e = launch_checked(kernel, grid, LP_THREADS, s, a, p.parts, p.span, words);
    if (e != hipSuccess || p.parts == 1) return e;
    LogprobArgs b = a;
    int c = p.parts, w = words;
    void* at[] = {(void*)&b, (void*)&c, (void*)&w};
    return hipLaunchKernel((const void*)k_logprob_join, dim3(a.n), dim3(64), at, (size_t)p.parts * a.K * 8, s);
}

}  // namespace cas
