// gfx950 kernels of token scoring: log probabilities of given tokens, entropy
// and top alternatives of rows of logits.
//
// With M the row's largest logit x_v and l_v = scale (x_v - M):
//   S = sum e^{l_v},  logp_t = l_t - log S,  entropy = log S - sum e^{l_v} l_v / S.
// A row is read once, in chunks of 8192 logits: a workgroup holds its chunk in
// registers, takes the chunk's (M, S, U = sum e^l l) and its K best, and a
// second kernel joins the row's chunks.
#include "attn_step.h"

namespace cas {

static constexpr int LP_THREADS = 256, LP_EACH = 32, LP_CHUNK = LP_THREADS * LP_EACH, LP_MAX_K = 32;

static int lp_chunks(int V) { return (V + LP_CHUNK - 1) / LP_CHUNK; }
// Per (row, chunk): M, S, U, and the K best as values, then ids.
static int lp_words(int K) { return 4 + 2 * K; }
size_t logprob_work_bytes(int n, int V, int K) { return (size_t)n * lp_chunks(V) * lp_words(K) * 4; }

__device__ __forceinline__ bool lp_better(float a, int ia, float b, int ib) { return a > b || (a == b && ia < ib); }

// The scaled difference x - M of finite M in log2 units goes through exp2.
static constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// The K best of `n` candidates (in LDS; better(a, b) is a strict order): every
// candidate counts those better than itself.
__device__ __forceinline__ void lp_rank(const float* v, const int* id, int n, int K, float* best, int* ids) {
    for (int i = threadIdx.x; i < n; i += LP_THREADS) {
        const float x = v[i];
        const int xi = id[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += lp_better(v[j], id[j], x, xi) ? 1 : 0;
        if (rank < K) {
            best[rank] = x;
            ids[rank] = xi;
        }
    }
    for (int i = n + threadIdx.x; i < K; i += LP_THREADS) {  // fewer than K finite logits
        best[i] = -INFINITY;
        ids[i] = -1;
    }
}

template <bool BF16> __global__ void __launch_bounds__(LP_THREADS) k_logprob_part(const LogprobArgs a, int chunks, int words) {
    constexpr int W = LP_THREADS / 64, NV = LP_EACH / (BF16 ? 8 : 4), E = BF16 ? 8 : 4, CAP = 64;
    __shared__ float sm_m[W], sm_s[W], sm_u[W], sm_v[W * CAP];
    __shared__ int sm_i[W * CAP], sm_n;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int chunk = blockIdx.x % chunks, row = blockIdx.x / chunks;
    const int base = chunk * LP_CHUNK, n = min(a.V - base, LP_CHUNK);
    float* rec = a.work + (size_t)blockIdx.x * words;
    float x[LP_EACH];
    const size_t at = (size_t)row * a.ld + base;
    // element e of piece i: base + (i * threads + thread) * E + e
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int o = (i * LP_THREADS + (int)threadIdx.x) * E;
#pragma unroll
        for (int e = 0; e < E; ++e) x[i * E + e] = -INFINITY;
        if (o + E <= n) {
            if constexpr (BF16) {
                struct __attribute__((packed, aligned(2))) P { i32x4 v; };
                const i32x4 v = ((const P*)((const uint16_t*)a.x + at + o))->v;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i * E + e] = piece_val<uint16_t>(v, e);
            } else {
                struct __attribute__((packed, aligned(4))) P { f32x4 v; };
                const f32x4 v = ((const P*)((const float*)a.x + at + o))->v;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i * E + e] = v[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (o + e < n) x[i * E + e] = BF16 ? bf2f(((const uint16_t*)a.x)[at + o + e]) : ((const float*)a.x)[at + o + e];
        }
    }
    if (threadIdx.x == 0) sm_n = 0;
    float lm = -INFINITY;  // (fmaxf passes over NaN: S finds it)
#pragma unroll
    for (int e = 0; e < LP_EACH; ++e) lm = fmaxf(lm, x[e]);
    const float wm = wave_max(lm);
    if (lane == 0) sm_m[wave] = wm;
    __syncthreads();
    float M = sm_m[0];
#pragma unroll
    for (int w = 1; w < W; ++w) M = fmaxf(M, sm_m[w]);
    const float ref = M == -INFINITY ? 0.f : M;
    const float c = a.scale * LOG2E;
    float s = 0.f, u = 0.f;
#pragma unroll
    for (int e = 0; e < LP_EACH; ++e) {
        const float l = (x[e] - ref) * c;
        const float p = __builtin_amdgcn_exp2f(l);
        s += p;
        u = fmaf(p, fmaxf(l, -1e30f), u);  // (nothing where p is 0)
    }
    s = wave_sum(s);
    u = wave_sum(u);
    if (lane == 0) {
        sm_s[wave] = s;
        sm_u[wave] = u;
    }
    if (a.K > 0) {
        // The wave's K-th largest lane maximum bounds its K best from below.  (Two
        // NaN-free maxima: lanes without a finite logit hold -inf.)
        int above = 0;
#pragma unroll
        for (int l = 0; l < 64; ++l) {
            const float o = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lm), l));
            above += o > lm || (o == lm && l < lane) ? 1 : 0;
        }
        const uint64_t kth = __ballot(above == a.K - 1);
        const float tau = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lm), __builtin_ctzll(kth)));
        int mine = 0;
        if (lm >= tau) {
#pragma unroll
            for (int e = 0; e < LP_EACH; ++e) mine += x[e] >= tau && x[e] > -INFINITY ? 1 : 0;
        }
        int all = mine;
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) all += __shfl_xor(all, o);
        auto id = [&](int e) { return base + ((e / E) * LP_THREADS + (int)threadIdx.x) * E + e % E; };
        if (all <= CAP) {
            if (mine) {
                int to = atomicAdd(&sm_n, mine);  // (their order does not matter)
#pragma unroll
                for (int e = 0; e < LP_EACH; ++e)
                    if (x[e] >= tau && x[e] > -INFINITY) {
                        sm_v[to] = x[e];
                        sm_i[to++] = id(e);
                    }
            }
        } else {  // many equal ones, or few lanes with a finite logit: the K best one after another
            int to = lane == 0 ? atomicAdd(&sm_n, a.K) : 0;
            to = __builtin_amdgcn_readfirstlane(to);
            float pv = INFINITY;
            int pi = -1;
            for (int k = 0; k < a.K; ++k) {
                float bv = -INFINITY;
                int bi = 0x7fffffff;
#pragma unroll
                for (int e = 0; e < LP_EACH; ++e)
                    if (lp_better(pv, pi, x[e], id(e)) && lp_better(x[e], id(e), bv, bi)) {
                        bv = x[e];
                        bi = id(e);
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
                if (lane == 0) {
                    sm_v[to + k] = bv;
                    sm_i[to + k] = bi;
                }
                pv = bv;
                pi = bi;
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        float S = sm_s[0], U = sm_u[0];
#pragma unroll
        for (int w = 1; w < W; ++w) {
            S += sm_s[w];
            U += sm_u[w];
        }
        rec[0] = M;
        rec[1] = S;
        rec[2] = U;
    }
    if (a.K > 0) lp_rank(sm_v, sm_i, sm_n, a.K, rec + 4, (int*)rec + 4 + a.K);
}

// One workgroup = one row: its chunks' sums in chunk order, the best of their
// bests, and the tokens asked for.
__global__ void __launch_bounds__(LP_THREADS) k_logprob_join(const LogprobArgs a, int chunks, int words) {
    extern __shared__ float sm[];  // [chunks * K] values, then ids
    const int row = blockIdx.x;
    const float* rec = a.work + (size_t)row * chunks * words;
    const float c = a.scale * LOG2E;
    float M = -INFINITY;
    for (int k = 0; k < chunks; ++k) M = fmaxf(M, rec[(size_t)k * words]);
    float S = 0.f, U = 0.f;
    for (int k = 0; k < chunks; ++k) {
        const float* q = rec + (size_t)k * words;
        // (a chunk without a finite logit: sums of exact zeros, but for a NaN)
        const float d = q[0] == -INFINITY ? 0.f : fmaxf((q[0] - M) * c, -1e30f), f = __builtin_amdgcn_exp2f(d);
        S = fmaf(q[1], f, S);
        U = fmaf(fmaf(q[1], d, q[2]), f, U);
    }
    // no finite logit, an infinite one or a NaN: no distribution
    const bool none = !(S > 0.f && S < INFINITY) || !(fabsf(M) < INFINITY);
    const float logS = none ? NAN : logf(S);
    if (threadIdx.x == 0 && a.entropy) a.entropy[row] = logS - U / S * LN2;
    for (int j = threadIdx.x; j < a.m; j += LP_THREADS) {
        const int t = a.tokens[(size_t)row * a.m + j];
        float y = NAN;
        if (t >= 0 && t < a.V) {
            const size_t o = (size_t)row * a.ld + t;
            const float x = a.bf16 ? bf2f(((const uint16_t*)a.x)[o]) : ((const float*)a.x)[o];
            y = (x - M) * a.scale - logS;
        }
        a.logp[(size_t)row * a.m + j] = y;
    }
    if (a.K == 0) return;
    float* best = a.best + (size_t)row * a.K;
    int* ids = a.ids + (size_t)row * a.K;
    if (none) {
        for (int k = threadIdx.x; k < a.K; k += LP_THREADS) {
            best[k] = NAN;
            ids[k] = -1;
        }
        return;
    }
    // candidates: what is no worse than every chunk's K-th
    float tau = -INFINITY;
    for (int k = 0; k < chunks; ++k) tau = fmaxf(tau, rec[(size_t)k * words + 3 + a.K]);
    float* v = sm;
    int* id = (int*)(sm + (size_t)chunks * a.K);
    __shared__ int count;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < chunks * a.K; i += LP_THREADS) {
        const float* q = rec + (size_t)(i / a.K) * words + 4;
        const float x = q[i % a.K];
        if (x >= tau && x > -INFINITY) {
            const int to = atomicAdd(&count, 1);
            v[to] = x;
            id[to] = ((const int*)q)[a.K + i % a.K];
        }
    }
    __syncthreads();
    const int n = count;
    for (int i = threadIdx.x; i < n; i += LP_THREADS) {
        const float x = v[i];
        const int xi = id[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += lp_better(v[j], id[j], x, xi) ? 1 : 0;
        if (rank < a.K) {
            best[rank] = (x - M) * a.scale - logS;
            ids[rank] = xi;
        }
    }
    for (int i = n + threadIdx.x; i < a.K; i += LP_THREADS) {
        best[i] = -INFINITY;
        ids[i] = -1;
    }
}

hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t s) {
    if (a.n < 1 || a.V < 1 || a.K < 0 || a.K > LP_MAX_K || a.m < 0) return hipErrorInvalidValue;
    const int chunks = lp_chunks(a.V), words = lp_words(a.K);
    const dim3 grid((unsigned)a.n * chunks);
    const hipError_t e = a.bf16 ? launch_checked(k_logprob_part<true>, grid, LP_THREADS, s, a, chunks, words)
                                : launch_checked(k_logprob_part<false>, grid, LP_THREADS, s, a, chunks, words);
    if (e != hipSuccess) return e;
    LogprobArgs b = a;
    int c = chunks, w = words;
    void* at[] = {(void*)&b, (void*)&c, (void*)&w};
    return hipLaunchKernel((const void*)k_logprob_join, dim3(a.n), dim3(LP_THREADS), at, (size_t)chunks * a.K * 8, s);
}

}  // namespace cas
