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
// The K best: the walk notes in LDS each thread's largest logit of each chunk, no
// more.  The K-th largest of the threads' largest logits bounds the K-th best from
// below, and closely (of 1024 threads the 20th is about the 20th logit), so that
// few (thread, chunk) pairs reach it, whose logits are read once more; what
// reaches the bound is ordered by rank.  (Collecting candidates during the walk,
// against a bound of the first chunk, cost as much as the sums.)  Equal logits can
// defeat the bound: where more than LP_LIST reach it, the K best come one after
// another, each from a pass over the part.  Everything is ordered by (logit, id),
// so no order of arrival shows.
//
// What bounds it: for many rows the bytes (1501 rows of 128256 logits, K = 20: 151
// us, 5.1 TB/s, what a copy reaches); for few rows a chain of waits (a row's first
// logits 2 us, the join 3.5 us, of which 2 for what other workgroups wrote).
#include "attn_step.h"
#include "logprob_plan.h"

namespace cas {

static constexpr int LP_MAX_K = 32;
static constexpr int LP_RANKED = 128;  // candidates that the join ranks against each other
static constexpr int LP_LIST = 512;  // candidates of a workgroup, of which a list holds
static constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ bool lp_better(float a, int ia, float b, int ib) { return a > b || (a == b && ia < ib); }

// Values in the order of unsigned numbers, and back (below the finite ones: -infinity).
__device__ __forceinline__ uint32_t lp_key(float x) {
    const uint32_t b = __float_as_uint(x);
    return b ^ ((int)b < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float lp_value(uint32_t key) {
    return key < 0x00800000u ? -INFINITY : __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
// Bounds, the same for every lane, that K lanes' x and J lanes' y reach (no NaN): the
// K-th and the J-th largest but for the last 12 bits, found from the top by the
// count of lanes that reach (with every lane's rank, of 64 comparisons, this took
// 16 waves of a CU 3 us).
static constexpr int LP_BITS = 12;
__device__ __forceinline__ void lp_kth(float x, int K, float* kth, float y, int J, float* jth) {
    const uint32_t key = lp_key(x), key_j = lp_key(y);
    uint32_t k = 0, j = 0;
#pragma unroll
    for (int bit = 31; bit >= LP_BITS; --bit) {
        const uint32_t k1 = k | 1u << bit, j1 = j | 1u << bit;
        k = (int)__popcll(__ballot(key >= k1)) >= K ? k1 : k;
        j = (int)__popcll(__ballot(key_j >= j1)) >= J ? j1 : j;
    }
    *kth = lp_value(k);
    *jth = lp_value(j);
}

// How many of a list's n entries (16-byte aligned; up to three -infinity behind
// them) are better than (x, xi), four at a time.
__device__ __forceinline__ int lp_count(const float* v, const int* id, int n, float x, int xi) {
    int k = 0;
#pragma unroll 2
    for (int j = 0; j < n; j += 4) {
        const f32x4 o = *(const f32x4*)(v + j);
        const i32x4 oi = *(const i32x4*)(id + j);
#pragma unroll
        for (int e = 0; e < 4; ++e) k += lp_better(o[e], oi[e], x, xi) ? 1 : 0;
    }
    return k;
}
__device__ __forceinline__ void lp_pad(float* v, int* id, int n) {
    const int lane = threadIdx.x & 63;
    if (lane < 3) {
        v[n + lane] = -INFINITY;
        id[n + lane] = 0x7fffffff;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
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
// The logit of a row's j-th token: NaN for an id outside the row.
__device__ __forceinline__ float lp_token(const LogprobArgs& a, int row, int j) {
    const int t = a.tokens[(size_t)row * a.m + j];
    return t >= 0 && t < a.V ? lp_logit(a, row, t) : NAN;
}
// (x: the logit of the thread's first token)
template <int THREADS> __device__ __forceinline__ void lp_tokens(const LogprobArgs& a, int row, const LpRow& r, float x) {
    if (threadIdx.x == 0 && a.entropy) a.entropy[row] = r.entropy;
    for (int j = threadIdx.x; j < a.m; j += THREADS)
        a.logp[(size_t)row * a.m + j] = r.logp(j < THREADS ? x : lp_token(a, row, j), a.scale);
}

// Workgroup = (row, part): chunks [part span, (part + 1) span) of EACH logits per
// thread.  One part: it gives the row's results itself.  Dynamic LDS: the largest
// logit of each (chunk, thread) of the part.
template <bool BF16, int EACH, int THREADS>
__global__ void __launch_bounds__(THREADS) k_logprob_part(const LogprobArgs a, int parts, int span, int words) {
    constexpr int E = BF16 ? 8 : 4, NV = EACH / E, CHUNK = THREADS * EACH, W = THREADS / 64;
    constexpr int LIST = THREADS > LP_LIST ? THREADS : LP_LIST;
    struct __attribute__((packed, aligned(BF16 ? 2 : 4))) Piece { i32x4 v; };
    extern __shared__ __attribute__((aligned(16))) float sm_top[];
    __shared__ __attribute__((aligned(16))) float sm_v[LIST + 4];
    __shared__ __attribute__((aligned(16))) int sm_i[LIST + 4];
    __shared__ float sm_sum[W][5];  // m, s, u, and the wave's K-th and ceil(K / W)-th largest thread
    __shared__ float sm_tau;
    __shared__ int sm_n[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = blockIdx.x % parts, row = blockIdx.x / parts, K = a.K;
    const int begin = part * span * CHUNK, end = min(a.V, begin + span * CHUNK);
    const char* x0 = (const char*)a.x + (size_t)row * a.ld * (BF16 ? 2 : 4);
    const float c = a.scale * LOG2E;
    const int odd = end - end % E;  // (a part ends at a chunk's end or the row's) the logits past the last whole piece
    auto load = [&](i32x4 (&r)[NV], int base) {  // pieces that lie in the part as a whole
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int o = base + (i * THREADS + tid) * E;
            if constexpr (BF16) r[i] = i32x4{(int)0xff80ff80, (int)0xff80ff80, (int)0xff80ff80, (int)0xff80ff80};
            else r[i] = i32x4{(int)0xff800000, (int)0xff800000, (int)0xff800000, (int)0xff800000};
            if (o + E <= end) r[i] = ((const Piece*)(x0 + (size_t)o * (BF16 ? 2 : 4)))->v;
        }
    };
    // a chunk's logits: its pieces', and one of the odd ones for each of the first threads
    auto unpack = [&](float (&x)[EACH + 1], const i32x4 (&r)[NV], int base) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) x[e] = piece_val<std::conditional_t<BF16, uint16_t, float>>(r[e / E], e % E);
        x[EACH] = -INFINITY;
        if (base + CHUNK >= end && odd + tid < end) x[EACH] = BF16 ? bf2f(((const uint16_t*)x0)[odd + tid]) : ((const float*)x0)[odd + tid];
    };
    auto id_of = [&](int base, int e) { return e == EACH ? odd + tid : base + ((e / E) * THREADS + tid) * E + e % E; };
    LpSums t = {-INFINITY, 0.f, 0.f};  // (s and u: the thread's)
    float lm = -INFINITY;
    i32x4 raw[NV];
    load(raw, begin);
    const float asked = parts == 1 && tid < a.m ? lp_token(a, row, tid) : NAN;
    for (int base = begin, k = 0; base < end; base += CHUNK, ++k) {
        float x[EACH + 1];
        unpack(x, raw, base);
        if (base + CHUNK < end) load(raw, base + CHUNK);
        float cm = -INFINITY;  // (fmaxf passes over NaN: s finds it)
#pragma unroll
        for (int e = 0; e <= EACH; ++e) cm = fmaxf(cm, x[e]);
        if (K > 0) sm_top[k * THREADS + tid] = cm;
        lm = fmaxf(lm, cm);
        const float wm = wave_top(cm);
        if (wm > t.m) t.lift(wm, c);
        const float ref = t.ref();
#pragma unroll
        for (int e = 0; e <= EACH; ++e) {
            const float l = (x[e] - ref) * c, p = __builtin_amdgcn_exp2f(l);
            t.s += p;
            t.u = fmaf(p, fmaxf(l, -1e30f), t.u);  // (nothing where p is 0)
        }
    }
    // Of W waves at least K threads reach each of: the K-th largest thread of any
    // wave, and the smallest of the waves' ceil(K / W)-th.
    float kth = 0.f, jth = 0.f;
    if (K > 0) lp_kth(lm, K, &kth, lm, (K + W - 1) / W, &jth);
    t.s = wave_sum(t.s);
    t.u = wave_sum(t.u);
    if (lane == 0) {
        sm_sum[wave][0] = t.m;
        sm_sum[wave][1] = t.s;
        sm_sum[wave][2] = t.u;
        sm_sum[wave][3] = kth;
        sm_sum[wave][4] = jth;
    }
    if (tid < 2) sm_n[tid] = 0;
    __syncthreads();
    LpSums r = {-INFINITY, 0.f, 0.f};
    float m = -INFINITY, least = -INFINITY, low = INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        m = fmaxf(m, sm_sum[w][0]);
        least = fmaxf(least, sm_sum[w][3]);
        low = fminf(low, sm_sum[w][4]);
    }
    least = fmaxf(least, low);
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
        lp_tokens<THREADS>(a, row, out, asked);
    } else if (tid == 0) {
        rec[0] = r.m;
        rec[1] = r.s;
        rec[2] = r.u;
    }
    if (K == 0) return;
    float* best = parts == 1 ? a.best + (size_t)row * K : rec + 4;
    int* ids = parts == 1 ? a.ids + (size_t)row * K : (int*)rec + 4 + K;
    auto give = [&](int rank, float y, int yi) {
        best[rank] = parts > 1 ? y : out.none ? NAN : out.logp(y, a.scale);
        ids[rank] = parts == 1 && out.none ? -1 : yi;
    };
    // the K-th largest of all threads' largest logits, of those that reach `least`
    auto push = [&](bool in, float y, int yi, int* count) {
        const uint64_t b = __ballot(in);
        int to = 0;
        if (lane == 0 && b) to = atomicAdd(count, (int)__popcll(b));
        to = __builtin_amdgcn_readfirstlane(to) + __popcll(b & (((uint64_t)1 << lane) - 1));
        if (in && to < LIST) {
            sm_v[to] = y;
            sm_i[to] = yi;
        }
    };
    push(lm >= least, lm, tid, &sm_n[0]);
    __syncthreads();
    const int nt = sm_n[0];
    if (tid < 64) lp_pad(sm_v, sm_i, nt);
    __syncthreads();
    if (tid < nt) {
        const float y = sm_v[tid];
        if (lp_count(sm_v, sm_i, nt, y, sm_i[tid]) == K - 1) sm_tau = y;
    }
    __syncthreads();
    const float tau = sm_tau;
    // the logits that reach it: each thread's chunks that have some, one after another
    uint32_t hit = 0;
    for (int base = begin, k = 0; base < end; base += CHUNK, ++k) {
        const float cm = sm_top[k * THREADS + tid];
        if (cm >= tau && cm > -INFINITY) hit |= 1u << k;
    }
    // (from the last on, which is still here)
    while (hit) {
        const int k = 31 - __builtin_clz(hit), base = begin + k * CHUNK;
        hit ^= 1u << k;
        float x[EACH + 1];
        if (base + CHUNK < end) load(raw, base);
        unpack(x, raw, base);
#pragma unroll
        for (int e = 0; e <= EACH; ++e)
            if (x[e] >= tau && x[e] > -INFINITY) {
                const int to = atomicAdd(&sm_n[1], 1);
                if (to < LIST) {
                    sm_v[to] = x[e];
                    sm_i[to] = id_of(base, e);
                }
            }
    }
    __syncthreads();
    const int n = sm_n[1];
    if (n <= LP_LIST) {
        if (tid < 64) lp_pad(sm_v, sm_i, n);
        __syncthreads();
        for (int i = tid; i < n; i += THREADS) {
            const float y = sm_v[i];
            const int yi = sm_i[i], rank = lp_count(sm_v, sm_i, n, y, yi);
            if (rank < K) give(rank, y, yi);
        }
        for (int i = n + tid; i < K; i += THREADS) {  // fewer than K finite logits
            best[i] = parts == 1 && out.none ? NAN : -INFINITY;
            ids[i] = -1;
        }
        return;
    }
    float pv = INFINITY;
    int pi = -1;
    for (int k = 0; k < K; ++k) {
        float bv = -INFINITY;
        int bi = 0x7fffffff;
        for (int base = begin; base < end; base += CHUNK) {
            float x[EACH + 1];
            load(raw, base);
            unpack(x, raw, base);
#pragma unroll
            for (int e = 0; e <= EACH; ++e) {
                const int id = id_of(base, e);
                if (lp_better(pv, pi, x[e], id) && lp_better(x[e], id, bv, bi)) {
                    bv = x[e];
                    bi = id;
                }
            }
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
        __syncthreads();
        if (lane == 0) {
            sm_v[wave] = bv;
            sm_i[wave] = bi;
        }
        __syncthreads();
        bv = sm_v[0];
        bi = sm_i[0];
        for (int w = 1; w < W; ++w)
            if (lp_better(sm_v[w], sm_i[w], bv, bi)) {
                bv = sm_v[w];
                bi = sm_i[w];
            }
        if (tid == 0) give(k, bv, bi);  // (more than LP_LIST finite logits: there is one)
        pv = bv;
        pi = bi;
    }
}

// One wave = one row in parts: their sums by a butterfly, the best of their
// bests, and the tokens asked for.  All it reads is asked for at the start: what
// other workgroups wrote takes 2 us to come.
__global__ void __launch_bounds__(64) k_logprob_join(const LogprobArgs a, int parts, int words, uint32_t inv_K) {
    extern __shared__ __attribute__((aligned(16))) float sm[];  // values, then ids
    constexpr int AT_ONCE = 8;
    const int row = blockIdx.x, lane = threadIdx.x, K = a.K, all = parts * K;
    const float* rec = a.work + (size_t)row * parts * words;
    const float c = a.scale * LOG2E;
    auto part_of = [&](int i) { return inv_K ? (int)__umulhi((uint32_t)i, inv_K) : i; };
    float cv[AT_ONCE];
    int ci[AT_ONCE];
    auto candidates = [&](int i0) {
#pragma unroll
        for (int q = 0; q < AT_ONCE; ++q) {
            const int i = min(i0 + q * 64 + lane, all - 1), k = part_of(i);
            const float* at = rec + (size_t)k * words + 4 + (i - k * K);
            cv[q] = at[0];
            ci[q] = ((const int*)at)[K];
        }
    };
    if (K > 0) candidates(0);
    const float asked = lane < a.m ? lp_token(a, row, lane) : NAN;
    LpSums t = {-INFINITY, 0.f, 0.f};
    // At least K logits reach each of: a part's K-th best, the smallest of the parts'
    // ceil(K / parts)-th best, the K-th of the lanes' best, and the ceil(K / 4)-th of
    // their fourth best.
    const int J = (K + parts - 1) / parts;
    float tau = -INFINITY, low = INFINITY, first = -INFINITY, fourth = -INFINITY;
    if (lane < parts) {
        const float* q = rec + (size_t)lane * words;
        t = {q[0], q[1], q[2]};
        if (K > 0) {
            tau = q[3 + K];
            low = q[3 + J];
            first = q[4];
            if (K > 8) fourth = q[7];
        }
    }
    t.lift(wave_top(t.m), c);
    t.s = wave_sum(t.s);
    t.u = wave_sum(t.u);
    const LpRow out(t);
    lp_tokens<64>(a, row, out, asked);
    if (K == 0) return;
    float kth, jth = -INFINITY, none;
    if (K > 8) lp_kth(first, K, &kth, fourth, (K + 3) / 4, &jth);
    else lp_kth(first, K, &kth, first, 1, &none);
    tau = fmaxf(fmaxf(wave_top(tau), -wave_top(-low)), fmaxf(kth, jth));
    float *best = a.best + (size_t)row * K, *v = sm;
    int *ids = a.ids + (size_t)row * K, *id = (int*)(sm + ((all + 7) & ~3)), n = 0;
    for (int i0 = 0; i0 < all; i0 += AT_ONCE * 64) {
        if (i0) candidates(i0);
#pragma unroll
        for (int q = 0; q < AT_ONCE; ++q) {
            const bool keep = i0 + q * 64 + lane < all && cv[q] >= tau && cv[q] > -INFINITY;
            const uint64_t in = __ballot(keep);
            if (keep) {
                const int to = n + __popcll(in & (((uint64_t)1 << lane) - 1));
                v[to] = cv[q];
                id[to] = ci[q];
            }
            n += __popcll(in);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // Many: to a bound by the count of those that reach it, as in lp_kth (32 parts of
    // 64000 logits, K = 32: 600 reached, and ranking them took 50 us).
    if (n > LP_RANKED) {
        uint32_t bound = 0;
        for (int bit = 31; bit >= LP_BITS; --bit) {
            int reach = 0;
            for (int i0 = 0; i0 < n; i0 += 64)
                reach += (int)__popcll(__ballot(i0 + lane < n && lp_key(v[min(i0 + lane, n - 1)]) >= (bound | 1u << bit)));
            if (reach >= K) bound |= 1u << bit;
        }
        const float least = lp_value(bound);  // (the zeros are equal)
        int kept = 0;
        for (int i0 = 0; i0 < n; i0 += 64) {
            const int i = min(i0 + lane, n - 1);
            const float x = v[i];
            const int xi = id[i];
            const bool keep = i0 + lane < n && x >= least;
            const uint64_t in = __ballot(keep);
            if (keep) {  // (at or below i0 + lane)
                const int to = kept + __popcll(in & (((uint64_t)1 << lane) - 1));
                v[to] = x;
                id[to] = xi;
            }
            kept += __popcll(in);
        }
        n = kept;
    }
    lp_pad(v, id, n);
    for (int i = lane; i < n; i += 64) {
        const float x = v[i];
        const int xi = id[i], rank = lp_count(v, id, n, x, xi);
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

size_t logprob_work_bytes(int n, int V, int K) { return lp_work_bytes(n, V, K); }

hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t s) {
    if (a.n < 1 || a.V < 1 || a.K < 0 || a.K > LP_MAX_K || a.m < 0) return hipErrorInvalidValue;
    const LpPlan p = lp_plan(a.n, a.V);
    const int words = lp_words(a.K);
    if (p.parts > 1 && a.work_bytes < (size_t)a.n * p.parts * words * 4) return hipErrorInvalidValue;
    const dim3 grid((unsigned)a.n * p.parts);
    auto kernel = p.threads == 1024 ? (a.bf16 ? k_logprob_part<true, 32, 1024> : k_logprob_part<false, 32, 1024>)
                  : p.each == 32      ? (a.bf16 ? k_logprob_part<true, 32, 256> : k_logprob_part<false, 32, 256>)
                                      : (a.bf16 ? k_logprob_part<true, 8, 256> : k_logprob_part<false, 8, 256>);
    LogprobArgs b = a;
    int c = p.parts, sp = p.span, w = words;
    void* part_at[] = {(void*)&b, (void*)&c, (void*)&sp, (void*)&w};
    const hipError_t e = hipLaunchKernel((const void*)kernel, grid, dim3(p.threads), part_at,
                                         a.K > 0 ? (size_t)p.span * p.threads * 4 : 0, s);
    if (e != hipSuccess || p.parts == 1) return e;
    // (multiplying by it and taking the high word divides by up to 128 exactly below 2^25)
    uint32_t inv_K = a.K > 1 ? (uint32_t)((((uint64_t)1 << 32) + a.K - 1) / a.K) : 0u;
    void* at[] = {(void*)&b, (void*)&c, (void*)&w, (void*)&inv_K};
    return hipLaunchKernel((const void*)k_logprob_join, dim3(a.n), dim3(64), at, (size_t)(p.parts * a.K + 8) * 8, s);
}

}  // namespace cas
