// What is learned from drawn tokens: the log probabilities of given tokens and their gradient, a clipped policy loss with a KL term and a
// loss over pairs of a preferred and a rejected answer, each with the gradient of the logits.
//
//   logp_t = l[target] - max l - log sum exp(l - max l);   d logp_t / d l_v = [v = target] - exp(l_v - max l) / sum
//
// Bound: bytes.  A row of 128,256 logits is 250 or 500 KB and a loss needs its normaliser before the first element of its gradient.
//   As many rows as SMs or more: a CTA streams a row, once from memory for the statistics and once from L2 for the gradient (token_stream_kernel).  3000 rows of
//     128,256 bf16, policy loss and gradient: 300 us, 5.1 TB/s, 78 % of the copy rate; log probabilities of 1200 such rows 56 us, 84 %.
//   Fewer rows: a cluster of up to eight CTAs holds a row in shared memory, a part each (token_row_kernel): 21 rows of 128,256 fp32 12 us (streamed 24), 120 rows 35
//     (39), log probabilities of 7 rows 5 (10).
// The second way, for many rows too, took 362 us for the 3000: a meeting of CTAs in every row, behind which nothing is in flight; with clusters that stay and fetch
// their next row meanwhile it took 626 us, for the meeting then waits for the stores of the row before.
// Where the slope of the loss follows from the token alone (the policy loss), logits are read from memory once and the gradient is written once.  A loss over pairs needs
// all rows of both answers first: a pass for the log probabilities, one for the gradient that begins with the rows that are still in L2.
#include "common.cuh"
#include "fp32_math.cuh"
#include "sm100_sync.cuh"

#include <cooperative_groups.h>

#include <algorithm>
#include <mutex>

namespace cg = cooperative_groups;

namespace bitlinear {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxRanks = 8;          // CTAs of a cluster
constexpr int kMaxPieces = 12;        // copies of a part; arithmetic on one begins when it has landed
constexpr int kPartBytes = 72 * 1024;  // three parts to an SM
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;  // where running maxima begin: a row may hold -infinity, and -inf - (-inf) is NaN

// What a pass over the rows is for.
constexpr int kLogp = 0;    // log probabilities and statistics
constexpr int kPolicy = 1;  // the policy loss and the gradient

struct RowArgs {
    const void* logits;
    long long stride;  // elements from a row to the next
    const int* targets;
    int V;
    int part;    // 16-byte units of a row's aligned middle per CTA
    int piece;   // of those, per copy
    float* logprobs;
    float2* stats;      // (max, sum of exp(l - max)); nullable
    float* grad;        // nullable: set to 0, for rows that no later kernel gives a slope
    // policy
    const float* old;
    const float* advantages;
    const float* weights;  // nullable
    const float* ref;      // nullable
    float clip_low, clip_high, kl;
    float* token_loss;
    void* dlogits;  // nullable
    long long d_stride;
    int* status;
};

template <typename T>
struct Vec;  // sixteen bytes of logits
template <>
struct Vec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void split(const uint4& v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 join(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    static __device__ __forceinline__ float most(const uint4& v) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    static __device__ __forceinline__ float load(const float* p) { return *p; }
    static __device__ __forceinline__ void store(float* p, float x) { *p = x; }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void split(const uint4& v, float (&x)[8]) {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint4 join(const float (&x)[8]) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            u[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
    static __device__ __forceinline__ float most(const uint4& v) {  // (a NaN counts only where nothing else stands)
        uint32_t a, b;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
        asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
        return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
    }
    static __device__ __forceinline__ float load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
};

// exp(x - m) for x <= m: the difference is rounded once, so what weighs most is off least
__device__ __forceinline__ float exp_below(float x, float m) { return ex2((x - m) * kLog2e); }

// The same exponentials by one multiply-add, for many elements of a row: 2^(x log2(e) - c) with c = fl(m log2(e)).  That is off from exp(x - m) by
// the factor 2^(m log2(e) - c), the same for all elements, which is put right once (`residue`).  For |m| of 2^20 and more that factor leaves the range of
// a float sooner or later: such rows go through exp_below.
constexpr float kPlain = 1048576.0f;
__device__ __forceinline__ float residue(float m, float c) { return ex2(-fmaf(m, kLog2e, -c)); }
template <int N>
__device__ __forceinline__ void exps(const float (&x)[N], float c, float (&e)[N]) {
#pragma unroll
    for (int j = 0; j < N; j += 2) {
        const float2 t = fma2(make_float2(x[j], x[j + 1]), splat(kLog2e), splat(-c));
        e[j] = ex2(t.x), e[j + 1] = ex2(t.y);
    }
}

// A row's elements before its first 16-byte border, and the number of whole 16-byte units behind that.
template <typename T>
struct RowShape {
    int head, units;
    __device__ __forceinline__ RowShape(const T* row, int V) {
        head = min((int)((16u - ((uint32_t)reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) / (int)sizeof(T), V);
        units = (V - head) / Vec<T>::N;
    }
};

// f exp(l - m) of sixteen bytes of logits
template <typename T>
struct RowWeights {
    float m, f, c, g;
    bool plain;
    __device__ __forceinline__ RowWeights(float m, float f) : m(m), f(f), c(m * kLog2e), g(f * residue(m, m * kLog2e)), plain(fabsf(m) < kPlain) {}
};
template <typename T>
__device__ __forceinline__ void weigh(const uint4& raw, float (&v)[Vec<T>::N], const RowWeights<T>& w) {
    constexpr int N = Vec<T>::N;
    float x[N];
    Vec<T>::split(raw, x);
    if (w.plain) {
        exps(x, w.c, v);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] *= w.g;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = exp_below(x[j], w.m) * w.f;
    }
}

// a running maximum and the sum of exp(x - maximum); one that met nothing is (kLowest, 0)
__device__ __forceinline__ void join_stats(float& m, float& s, float m2, float s2) {
    const float n = fmaxf(m, m2);
    s = s * exp_below(m, n) + s2 * exp_below(m2, n);
    m = n;
}

// A thread's statistics while it goes over a row: the running maximum, itself and in base 2, and the sum in two halves.
struct Running {
    float m = kLowest, c = kLowest;
    float2 sum = make_float2(0.0f, 0.0f);
    template <typename T>
    __device__ __forceinline__ void add(const uint4& raw) {
        constexpr int N = Vec<T>::N;
        float v[N], e[N];
        Vec<T>::split(raw, v);
        const float top = Vec<T>::most(raw);
        if (top > m) {
            // Rounded up, c is nowhere below the product, and finite below -2^127: no element's exponential passes 1, whatever c's rounding is worth under a maximum of large
            // magnitude (masked tokens in front of others). To the nearest, such a sum became infinite, and NaN with the next factor of 0.
            const float next = __fmul_ru(top, kLog2e);
            sum.x *= ex2(c - next), sum.y *= ex2(c - next);
            m = top, c = next;
        }
        exps(v, c, e);
        // sixteen bytes' terms among themselves first: fewer roundings at the size of the sum
#pragma unroll
        for (int w = N / 2; w > 1; w /= 2)
#pragma unroll
            for (int j = 0; j < w; ++j) e[j] += e[j + w];
        sum.x += e[0], sum.y += e[1];
    }
    __device__ __forceinline__ bool plain() const { return fabsf(m) < kPlain; }  // else the thread goes over its elements again, with exp_below and m
    __device__ __forceinline__ float total() const { return (sum.x + sum.y) * (m > kLowest ? residue(m, c) : 1.0f); }
};
template <typename T>
__device__ __forceinline__ float sum_below(const uint4& raw, float m) {
    float v[Vec<T>::N], s = 0.0f;
    Vec<T>::split(raw, v);
#pragma unroll
    for (int j = 0; j < Vec<T>::N; ++j) s += exp_below(v[j], m);
    return s;
}

// A log probability in two parts, chosen - m - log(sum): rounded to fp32 alone it is off by a part in 2^24 of log(sum), which is ten or more, and the ratio of two
// models' probabilities by as much.  log(sum) = k ln 2 + log(rest), rest about 1; k times the upper bits of ln 2 is exact.
struct LogProb {
    float hi, lo;
};
// x - y and what its rounding took
__device__ __forceinline__ float difference(float x, float y, float& lost) {
    const float d = __fsub_rn(x, y), z = __fsub_rn(d, x);
    lost = __fsub_rn(__fsub_rn(x, __fsub_rn(d, z)), __fadd_rn(y, z));
    return d;
}
__device__ __forceinline__ LogProb log_prob(float chosen, float m, float sum) {
    const int bits = __float_as_int(sum), k = (bits - 0x3f3504f3) >> 23;  // rest between sqrt(1/2) and sqrt(2)
    const float rest = __int_as_float(bits - (k << 23)), big = (float)k * 0x1.62e4p-1f;  // (fifteen bits)
    const float small = fmaf((float)k, 0x1.7f7d1cp-20f, logf(sum > 0.0f && sum < INFINITY ? rest : sum));
    float a_lo, b_lo, c_lo;
    const float hi = difference(difference(difference(chosen, m, a_lo), big, b_lo), small, c_lo), lo = a_lo + b_lo + c_lo;
    return {hi, fabsf(hi) < 1e30f && fabsf(lo) < 1.0f ? lo : 0.0f};
}

// The policy loss of one token and its slope with the log probability: r = exp(logp - old),
//   -min(r A, clip(r, 1 - low, 1 + high) A) + kl (exp(ref - logp) - (ref - logp) - 1).
__device__ __forceinline__ void policy_token(LogProb logp, float old, float adv, float ref, float low, float high, float kl, float& loss, float& slope) {
    float r = expf((logp.hi - old) + logp.lo);
    if (adv == 0.0f && r == INFINITY) r = 0.0f;  // 0 times a ratio past fp32 is 0
    const float free = r * adv, cut = fminf(fmaxf(r, 1.0f - low), 1.0f + high) * adv;
    const bool inside = free <= cut;
    loss = inside ? -free : -cut;
    slope = inside ? -free : 0.0f;
    if (free != free) loss = slope = free;
    if (kl != 0.0f) {
        const float d = (ref - logp.hi) - logp.lo, e = expm1f(d);
        // e - d cancels for small d: the series there, its first term left out (d^8 / 8! of d^2 / 2) below 2^-26
        const float near = d * d * fmaf(d, fmaf(d, fmaf(d, fmaf(d, fmaf(d, 1.0f / 5040.0f, 1.0f / 720.0f), 1.0f / 120.0f), 1.0f / 24.0f), 1.0f / 6.0f), 0.5f);
        loss = fmaf(kl, fabsf(d) < 0.25f ? near : e - d, loss);
        slope = fmaf(-kl, e, slope);
    }
}

template <typename T, int MODE>
__global__ void __launch_bounds__(kThreads, 3) token_row_kernel(const RowArgs a) {
    constexpr int N = Vec<T>::N;
    extern __shared__ __align__(128) uint8_t part_s[];
    __shared__ float2 warp_stats[kWarps], cta_stats;
    __shared__ uint64_t bars[kMaxPieces];
    __shared__ int abort_flag;
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = blockIdx.x / ranks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const T* x = static_cast<const T*>(a.logits) + (size_t)row * a.stride;
    T* d = MODE == kPolicy && a.dlogits ? static_cast<T*>(a.dlogits) + (size_t)row * a.d_stride : nullptr;
    const RowShape<T> shape(x, a.V);
    // this CTA's units, and (at the ends of the row) its single elements: lane l of warp 0 has one at most
    const int u0 = min(rank * a.part, shape.units), u1 = min(u0 + a.part, shape.units), n = u1 - u0;
    const T* body = x + shape.head;
    int single = -1;
    if (warp == 0) {
        if (rank == 0 && lane < shape.head) single = lane;
        const int tail = shape.head + shape.units * N + lane - 16;
        if (rank == ranks - 1 && lane >= 16 && tail < a.V) single = tail;
    }
    if (tid == 0) {
        abort_flag = 0;
        for (int i = 0; i < kMaxPieces; ++i) mbar_init(smem_u32(bars + i), 1);
        mbar_init_fence();
    }
    __syncthreads();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int target = a.targets[row];
    const float weight = MODE == kPolicy && a.weights ? a.weights[row] : 1.0f;
    const bool counts = target >= 0 && target < a.V;  // else the row is not read: 0 all over
    float slope = 0.0f;
    LogProb logp = {0.0f, 0.0f};
    float2 all = make_float2(0.0f, 1.0f);
    float xs = kLowest;
    if (counts) {
        if (tid == 0) {
            const uint64_t once = l2_evict_first_policy();
            for (int p = 0, at = 0; at < n; ++p, at += a.piece) {
                const uint32_t bytes = 16u * (uint32_t)min(a.piece, n - at), bar = smem_u32(bars + p);
                mbar_expect_tx(bar, bytes);
                const void* src = body + (size_t)(u0 + at) * N;
                if (MODE == kPolicy) bulk_load_once(smem_u32(part_s) + 16u * at, src, bytes, bar, once);
                else bulk_load(smem_u32(part_s) + 16u * at, src, bytes, bar);
            }
        }
        const float chosen = Vec<T>::load(x + target);  // (before the cluster meets: the gradient may go where the logits are)
        if (single >= 0) xs = Vec<T>::load(x + single);
        Running run;
        for (int p = 0, at = 0; at < n; ++p, at += a.piece) {
            if (!mbar_wait(smem_u32(bars + p), 0, &abort_flag)) break;
            const int end = min(at + a.piece, n);
            for (int i = at + tid; i < end; i += kThreads) run.add<T>(*reinterpret_cast<const uint4*>(part_s + 16 * (size_t)i));
        }
        float m = run.m, s = run.total();
        if (!run.plain()) {
            s = 0.0f;
            for (int i = tid; i < n; i += kThreads) s += sum_below<T>(*reinterpret_cast<const uint4*>(part_s + 16 * (size_t)i), m);
        }
        if (single >= 0) join_stats(m, s, xs, xs > kLowest ? 1.0f : exp_below(xs, kLowest));
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const float m2 = __shfl_xor_sync(0xffffffffu, m, off), s2 = __shfl_xor_sync(0xffffffffu, s, off);
            join_stats(m, s, m2, s2);
        }
        if (lane == 0) warp_stats[warp] = make_float2(m, s);
        __syncthreads();
        if (warp == 0) {
            const float2 w = lane < kWarps ? warp_stats[lane] : make_float2(kLowest, 0.0f);
            m = w.x, s = w.y;
#pragma unroll
            for (int off = kWarps / 2; off > 0; off >>= 1) {
                const float m2 = __shfl_xor_sync(0xffffffffu, m, off), s2 = __shfl_xor_sync(0xffffffffu, s, off);
                join_stats(m, s, m2, s2);
            }
            if (lane == 0) cta_stats = make_float2(m, s);
        }
        cluster.sync();
        {  // every thread of every CTA joins the parts in the same order
            float2 o[kMaxRanks];
#pragma unroll
            for (int r = 0; r < kMaxRanks; ++r) o[r] = *cluster.map_shared_rank(&cta_stats, min(r, ranks - 1));
            all = o[0];
#pragma unroll
            for (int r = 1; r < kMaxRanks; ++r)
                if (r < ranks) join_stats(all.x, all.y, o[r].x, o[r].y);
        }
        cluster.barrier_arrive();
        logp = log_prob(chosen, all.x, all.y);
    }
    float loss = 0.0f;
    if constexpr (MODE == kPolicy) {
        if (counts && weight != 0.0f) {  // a token of weight 0 counts for nothing, whatever stands beside it
            policy_token(logp, a.old[row], a.advantages[row], a.ref ? a.ref[row] : 0.0f, a.clip_low, a.clip_high, a.kl, loss, slope);
            loss *= weight, slope *= weight;
        }
    }
    if (rank == 0 && tid == 0) {
        a.logprobs[row] = logp.hi;
        if (a.stats) a.stats[row] = all;
        if (a.grad) a.grad[row] = 0.0f;
        if (MODE == kPolicy) a.token_loss[row] = loss;
    }
    if constexpr (MODE == kPolicy) {
        if (d != nullptr) {
            const bool live = counts && (weight != 0.0f);
            const float f = live ? -slope / all.y : 0.0f, at_target = -slope * expm1f(logp.hi);
            const RowWeights<T> weights(all.x, f);
            T* to = d + shape.head;
            const bool aligned = ((reinterpret_cast<uintptr_t>(to)) & 15) == 0;
            for (int i = tid; i < n; i += kThreads) {
                float v[N];
                if (live) {
                    weigh(*reinterpret_cast<const uint4*>(part_s + 16 * (size_t)i), v, weights);
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j) v[j] = 0.0f;
                }
                const int e = (u0 + i) * N;
                const int hit = target - shape.head - e;
                if (live && hit >= 0 && hit < N) {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (j == hit) v[j] = at_target;
                }
                if (aligned) __stcs(reinterpret_cast<uint4*>(to + e), Vec<T>::join(v));
                else
#pragma unroll
                    for (int j = 0; j < N; ++j) Vec<T>::store(to + e + j, v[j]);
            }
            if (single >= 0) Vec<T>::store(d + single, !live ? 0.0f : single == target ? at_target : exp_below(xs, all.x) * f);
        }
    }
    if (counts) cluster.barrier_wait();  // no CTA leaves while another reads its shared memory
    if (abort_flag && tid == 0 && a.status != nullptr) atomicExch(a.status, BITLINEAR_ERR_TIMEOUT);
    if (abort_flag) abort_drain();
}

// Many rows: a CTA to a row, which it streams from memory for the statistics and, for the gradient, once more - from L2, as far as that holds the rows under way, two to
// an SM: 76 MB of 128,256 bf16 logits, but 152 MB of as many in fp32, of which some come from memory again (1500 rows 367 us; the same bytes as 3000 rows of bf16 325, of
// 64,128 fp32 305; in slices for the clusters of the other kernel 468).  No CTA waits for another, so that loads and stores of several rows are under way at any time.
constexpr int kStreamThreads = 512;
__host__ __device__ constexpr int stream_units(int mode) { return mode == kPolicy ? 8 : 4; }  // loads in flight a thread

template <typename T, int MODE>
__global__ void __launch_bounds__(kStreamThreads, MODE == kPolicy ? 2 : 3) token_stream_kernel(const RowArgs a) {
    constexpr int N = Vec<T>::N, kWarpsHere = kStreamThreads / 32, kStreamUnits = stream_units(MODE);
    __shared__ float2 warp_stats[kWarpsHere];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const T* x = static_cast<const T*>(a.logits) + (size_t)row * a.stride;
    T* d = MODE == kPolicy && a.dlogits ? static_cast<T*>(a.dlogits) + (size_t)row * a.d_stride : nullptr;
    const RowShape<T> shape(x, a.V);
    const T* body = x + shape.head;
    int single = -1;  // the elements at the row's ends: lane l of warp 0 has one at most
    if (warp == 0) {
        const int tail = shape.head + shape.units * N + lane - 16;
        single = lane < 16 ? (lane < shape.head ? lane : -1) : tail < a.V ? tail : -1;
    }
    const int target = a.targets[row];
    const bool counts = target >= 0 && target < a.V;  // else the row is not read: 0 all over
    float weight = 1.0f, old = 0.0f, adv = 0.0f, ref = 0.0f;
    if constexpr (MODE == kPolicy) {
        if (a.weights) weight = a.weights[row];
        old = a.old[row], adv = a.advantages[row], ref = a.ref ? a.ref[row] : 0.0f;
    }
    float slope = 0.0f, loss = 0.0f, xs = kLowest;
    LogProb logp = {0.0f, 0.0f};
    float2 all = make_float2(0.0f, 1.0f);
    if (counts) {
        const float chosen = Vec<T>::load(x + target);  // (before the CTA meets: the gradient may go where the logits are)
        if (single >= 0) xs = Vec<T>::load(x + single);
        Running run;
        for (int i0 = tid; i0 < shape.units; i0 += kStreamUnits * kStreamThreads) {
            uint4 raw[kStreamUnits];
#pragma unroll
            for (int k = 0; k < kStreamUnits; ++k) {
                const int i = i0 + k * kStreamThreads;
                if (i < shape.units) raw[k] = MODE == kPolicy ? *(reinterpret_cast<const uint4*>(body) + i) : __ldcs(reinterpret_cast<const uint4*>(body) + i);
            }
#pragma unroll
            for (int k = 0; k < kStreamUnits; ++k) {
                const int i = i0 + k * kStreamThreads;
                if (i >= shape.units) break;
                run.add<T>(raw[k]);
            }
        }
        float m = run.m, s = run.total();
        if (!run.plain()) {
            s = 0.0f;
            for (int i = tid; i < shape.units; i += kStreamThreads) s += sum_below<T>(*(reinterpret_cast<const uint4*>(body) + i), m);
        }
        if (single >= 0) join_stats(m, s, xs, xs > kLowest ? 1.0f : exp_below(xs, kLowest));
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const float m2 = __shfl_xor_sync(0xffffffffu, m, off), s2 = __shfl_xor_sync(0xffffffffu, s, off);
            join_stats(m, s, m2, s2);
        }
        if (lane == 0) warp_stats[warp] = make_float2(m, s);
        __syncthreads();
        all = warp_stats[lane % kWarpsHere];  // every warp joins all in the same order
#pragma unroll
        for (int off = kWarpsHere / 2; off > 0; off >>= 1) {
            const float m2 = __shfl_xor_sync(0xffffffffu, all.x, off), s2 = __shfl_xor_sync(0xffffffffu, all.y, off);
            join_stats(all.x, all.y, m2, s2);
        }
        all.x = __shfl_sync(0xffffffffu, all.x, 0), all.y = __shfl_sync(0xffffffffu, all.y, 0);
        logp = log_prob(chosen, all.x, all.y);
    }
    if constexpr (MODE == kPolicy) {
        if (counts && weight != 0.0f) {  // a token of weight 0 counts for nothing, whatever stands beside it
            policy_token(logp, old, adv, ref, a.clip_low, a.clip_high, a.kl, loss, slope);
            loss *= weight, slope *= weight;
        }
    }
    if (tid == 0) {
        a.logprobs[row] = logp.hi;
        if (a.stats) a.stats[row] = all;
        if (a.grad) a.grad[row] = 0.0f;
        if (MODE == kPolicy) a.token_loss[row] = loss;
    }
    if constexpr (MODE == kPolicy) {
        if (d == nullptr) return;
        const bool live = counts && weight != 0.0f;
        const float f = live ? -slope / all.y : 0.0f, at_target = -slope * expm1f(logp.hi);
        const RowWeights<T> weights(all.x, f);
        T* to = d + shape.head;
        const bool aligned = (reinterpret_cast<uintptr_t>(to) & 15) == 0;
        for (int i0 = tid; i0 < shape.units; i0 += kStreamUnits * kStreamThreads) {
            uint4 raw[kStreamUnits];
#pragma unroll
            for (int k = 0; k < kStreamUnits; ++k) {
                const int i = i0 + k * kStreamThreads;
                if (live && i < shape.units) raw[k] = __ldcs(reinterpret_cast<const uint4*>(body) + i);
            }
#pragma unroll
            for (int k = 0; k < kStreamUnits; ++k) {
                const int i = i0 + k * kStreamThreads;
                if (i >= shape.units) break;
                float v[N];
                if (live) {
                    weigh(raw[k], v, weights);
                    const int hit = target - shape.head - i * N;
                    if (hit >= 0 && hit < N) {
#pragma unroll
                        for (int j = 0; j < N; ++j)
                            if (j == hit) v[j] = at_target;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j) v[j] = 0.0f;
                }
                if (aligned) __stcs(reinterpret_cast<uint4*>(to) + i, Vec<T>::join(v));
                else
#pragma unroll
                    for (int j = 0; j < N; ++j) Vec<T>::store(to + (size_t)i * N + j, v[j]);
            }
        }
        if (single >= 0) Vec<T>::store(d + single, !live ? 0.0f : single == target ? at_target : exp_below(xs, all.x) * f);
    }
}

// The gradient from statistics that are there: every element on its own.  A CTA takes 256 x 4 units of a row, all loads in flight.
struct GradArgs {
    const void* logits;
    long long stride;
    const int* targets;
    const float2* stats;
    const float* grad;
    void* dlogits;
    long long d_stride;
    int T, V, slabs;
};
constexpr int kGradUnits = 4;

template <typename T>
__global__ void __launch_bounds__(kThreads) token_grad_kernel(const GradArgs a) {
    constexpr int N = Vec<T>::N;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // the last rows first: after a pass over all rows they are the ones that may still be in L2
    const int at = (int)(gridDim.x - 1 - blockIdx.x), row = at / a.slabs, slab = at - row * a.slabs, tid = threadIdx.x;
    const T* x = static_cast<const T*>(a.logits) + (size_t)row * a.stride;
    T* d = static_cast<T*>(a.dlogits) + (size_t)row * a.d_stride;
    const RowShape<T> shape(x, a.V);
    const int target = a.targets[row];
    const float g = a.grad[row];
    const float2 st = a.stats[row];
    const bool live = target >= 0 && target < a.V && g != 0.0f;  // else zeros, whatever the row holds
    const float f = live ? -g / st.y : 0.0f;
    // 1 - p of the target from its own logit, which the thread that holds it has read: the gradient may go where the logits are
    auto at_target = [&](float l) { return -g * expm1f((l - st.x) - logf(st.y)); };
    const RowWeights<T> weights(st.x, f);
    const T* body = x + shape.head;
    T* to = d + shape.head;
    const bool aligned = (reinterpret_cast<uintptr_t>(to) & 15) == 0;
    uint4 raw[kGradUnits];
#pragma unroll
    for (int k = 0; k < kGradUnits; ++k) {
        const int u = (slab * kGradUnits + k) * kThreads + tid;
        raw[k] = live && u < shape.units ? __ldcs(reinterpret_cast<const uint4*>(body) + u) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < kGradUnits; ++k) {
        const int u = (slab * kGradUnits + k) * kThreads + tid;
        if (u >= shape.units) break;
        float v[N];
        if (live) {
            weigh(raw[k], v, weights);
            const int hit = target - shape.head - u * N;
            if (hit >= 0 && hit < N) {
                float x[N];
                Vec<T>::split(raw[k], x);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (j == hit) v[j] = at_target(x[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = 0.0f;
        }
        if (aligned) __stcs(reinterpret_cast<uint4*>(to) + u, Vec<T>::join(v));
        else
#pragma unroll
            for (int j = 0; j < N; ++j) Vec<T>::store(to + (size_t)u * N + j, v[j]);
    }
    if (slab == 0 && tid < 32) {  // the elements at the row's ends
        const int tail = shape.head + shape.units * N + tid - 16;
        const int single = tid < 16 ? (tid < shape.head ? tid : -1) : tail < a.V ? tail : -1;
        if (single >= 0) {
            const float l = live ? Vec<T>::load(x + single) : 0.0f;
            Vec<T>::store(d + single, !live ? 0.0f : single == target ? at_target(l) : exp_below(l, st.x) * f);
        }
    }
}

// sum of n numbers times scale in fp64, always in the same order: thread t adds every 1024th from t on, then a tree
__global__ void __launch_bounds__(1024) loss_sum_kernel(const float* x, int n, double scale, float* out) {
    __shared__ double part[32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += 1024) s += (double)x[i];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x < 32) {
        s = part[threadIdx.x];
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        if (threadIdx.x == 0) *out = (float)(s * scale);
    }
}

// A pair's answers: warps 0 .. 3 sum the preferred one's log probabilities, 4 .. 7 the other's (fp64, always in the same order), then all
// write the tokens' slopes.  Rows of no answer keep the slope 0 that they were given before.  One CTA alone writes the mean, too.
__global__ void __launch_bounds__(256) pair_kernel(const float* logprobs, const int* targets, const int* cu, const float* ref,
                                                   int T, int V, int pairs, float beta, float smooth, float* pair_loss, float* seq_logprobs,
                                                   float* grad, float* loss) {
    __shared__ double part[8];
    double total = 0.0;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int half = threadIdx.x >> 7, t = threadIdx.x & 127;
    for (int i = blockIdx.x; i < pairs; i += gridDim.x) {
        const int begin = min(max(cu[2 * i + half], 0), T), end = min(max(cu[2 * i + half + 1], begin), T);
        double s = 0.0;
        for (int j = begin + t; j < end; j += 128)
            if (targets[j] >= 0 && targets[j] < V) s += (double)logprobs[j];
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        __syncthreads();  // (the pair before this one has been read)
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
        __syncthreads();
        const double chosen = (part[0] + part[1]) + (part[2] + part[3]), rejected = (part[4] + part[5]) + (part[6] + part[7]);
        const float delta = (float)((double)beta * ((chosen - (double)ref[2 * i]) - (rejected - (double)ref[2 * i + 1])));
        // log sigma(x) = min(x, 0) - log1p(exp(-|x|))
        const float soft = log1pf(expf(-fabsf(delta)));
        const float up = fminf(delta, 0.0f) - soft, down = fminf(-delta, 0.0f) - soft;
        const float slope = (float)(-(double)beta / pairs) * (1.0f / (1.0f + expf(delta)) - smooth);
        if (threadIdx.x == 0) {
            // (an answer of probability zero makes one of the two infinite: times a factor of 0 it would be NaN)
            const float value = (smooth < 1.0f ? -(1.0f - smooth) * up : 0.0f) - (smooth > 0.0f ? smooth * down : 0.0f);
            pair_loss[i] = value;
            total += (double)value;
            seq_logprobs[2 * i] = (float)chosen;
            seq_logprobs[2 * i + 1] = (float)rejected;
        }
        if (grad != nullptr)
            for (int j = begin + t; j < end; j += 128) grad[j] = half ? -slope : slope;
    }
    if (loss != nullptr && threadIdx.x == 0) *loss = (float)(total / pairs);
}

// ---------------------------------------------------------------------------------------------- host side

int dtype_bytes(int dtype) { return dtype == BITLINEAR_F32 ? 4 : dtype == BITLINEAR_BF16 ? 2 : 0; }

void launch_dependent(cudaLaunchConfig_t& cfg, cudaLaunchAttribute (&attr)[2], int clusters) {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)clusters;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = clusters > 1 ? 2 : 1;
}

template <typename T, int MODE>
int launch_rows(RowArgs a, int rows, int sm_count, cudaStream_t st) {
    constexpr int kMost = 200 * 1024;
    static std::mutex mu;
    static bool done[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return finish(cudaErrorInvalidDevice);
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!done[dev]) {
            if (cudaFuncSetAttribute(token_row_kernel<T, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost) != cudaSuccess) return finish(cudaErrorUnknown);
            done[dev] = true;
        }
    }
    const long long units = (long long)a.V * (int)sizeof(T) / 16;
    if (rows >= sm_count) {
        cudaLaunchAttribute attr[2];
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)rows);
        cfg.blockDim = dim3(kStreamThreads);
        cfg.stream = st;
        launch_dependent(cfg, attr, 1);
        return finish(cudaLaunchKernelEx(&cfg, token_stream_kernel<T, MODE>, a));
    }
    int ranks = 1;
    auto part = [&] { return (units + ranks - 1) / ranks; };
    while (ranks < kMaxRanks && part() * 16 > kPartBytes) ranks *= 2;
    // few rows: more CTAs to each while SMs are idle and a part keeps 4 KB
    while (ranks < kMaxRanks && (long long)rows * ranks * 2 <= sm_count && part() >= 512) ranks *= 2;
    a.part = (int)std::max(part(), 1ll);
    // (whole rounds of the CTA's threads: a thread that goes over the part again without regard to pieces meets the units whose maximum it has)
    a.piece = std::max(512, ((a.part + kMaxPieces - 1) / kMaxPieces + kThreads - 1) / kThreads * kThreads);
    if (a.part * 16 > kMost || (long long)rows * ranks > 0x7fffffffll) return BITLINEAR_ERR_SHAPE;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * ranks));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)a.part * 16;
    cfg.stream = st;
    launch_dependent(cfg, attr, ranks);
    return finish(cudaLaunchKernelEx(&cfg, token_row_kernel<T, MODE>, a));
}

template <int MODE>
int rows_pass(const RowArgs& a, int dtype, int rows, cudaStream_t st) {
    int sm_count = 0;
    if (const int rc = device_sm_count(&sm_count)) return rc;
    return dtype == BITLINEAR_F32 ? launch_rows<float, MODE>(a, rows, sm_count, st) : launch_rows<__nv_bfloat16, MODE>(a, rows, sm_count, st);
}

int grad_pass(GradArgs a, int dtype, cudaStream_t st) {
    const long long units = (long long)a.V * dtype_bytes(dtype) / 16;
    a.slabs = (int)std::max(1ll, (units + kThreads * kGradUnits - 1) / (kThreads * kGradUnits));
    if ((long long)a.T * a.slabs > 0x7fffffffll) return BITLINEAR_ERR_SHAPE;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.T * a.slabs));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    launch_dependent(cfg, attr, 1);
    return finish(dtype == BITLINEAR_F32 ? cudaLaunchKernelEx(&cfg, token_grad_kernel<float>, a) : cudaLaunchKernelEx(&cfg, token_grad_kernel<__nv_bfloat16>, a));
}

int sum_pass(const float* x, int n, double scale, float* out, cudaStream_t st) {
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1);
    cfg.blockDim = dim3(1024);
    cfg.stream = st;
    launch_dependent(cfg, attr, 1);
    return finish(cudaLaunchKernelEx(&cfg, loss_sum_kernel, x, n, scale, out));
}

// what all entry points ask of logits (and gradients) of T rows
int check_logits(int dtype, int T, int V, long long stride) {
    if (dtype_bytes(dtype) == 0) return BITLINEAR_ERR_DTYPE;
    if (T < 0 || T > (1 << 24) || V <= 0 || V > BITLINEAR_SAMPLE_MAX_VOCAB || stride < V) return BITLINEAR_ERR_SHAPE;
    return BITLINEAR_OK;
}
bool element_aligned(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % (unsigned)dtype_bytes(dtype) == 0; }

}  // namespace

}  // namespace bitlinear

using namespace bitlinear;

extern "C" {

int bitlinear_token_logprobs(const void* logits, int logits_dtype, int T, int V, long long row_stride, const int32_t* targets, float* logprobs, float* stats, void* stream) {
    if (const int rc = check_logits(logits_dtype, T, V, row_stride)) return rc;
    if (T == 0) return BITLINEAR_OK;
    if (!logits || !targets || !logprobs || !stats) return BITLINEAR_ERR_NULL;
    if (!element_aligned(logits, logits_dtype) || reinterpret_cast<uintptr_t>(stats) % 8) return BITLINEAR_ERR_ALIGN;
    RowArgs a = {};
    a.logits = logits, a.stride = row_stride, a.targets = targets, a.V = V, a.logprobs = logprobs;
    a.stats = reinterpret_cast<float2*>(stats), a.status = device_status_word();
    return rows_pass<kLogp>(a, logits_dtype, T, static_cast<cudaStream_t>(stream));
}

int bitlinear_token_logprobs_backward(const void* logits, int logits_dtype, int T, int V, long long row_stride, const int32_t* targets, const float* stats, const float* grad,
                                      void* dlogits, long long d_stride, void* stream) {
    if (const int rc = check_logits(logits_dtype, T, V, row_stride)) return rc;
    if (d_stride < V) return BITLINEAR_ERR_SHAPE;
    if (T == 0) return BITLINEAR_OK;
    if (!logits || !targets || !stats || !grad || !dlogits) return BITLINEAR_ERR_NULL;
    if (logits == dlogits && d_stride != row_stride) return BITLINEAR_ERR_SHAPE;
    if (!element_aligned(logits, logits_dtype) || !element_aligned(dlogits, logits_dtype) || reinterpret_cast<uintptr_t>(stats) % 8) return BITLINEAR_ERR_ALIGN;
    int sm_count = 0;
    if (const int rc = device_sm_count(&sm_count)) return rc;  // (for the device's architecture; the grid does not hang on the number)
    const GradArgs a = {logits, row_stride, targets, reinterpret_cast<const float2*>(stats), grad, dlogits, d_stride, T, V, 0};
    return grad_pass(a, logits_dtype, static_cast<cudaStream_t>(stream));
}

int bitlinear_policy_loss(const void* logits, int logits_dtype, int T, int V, long long row_stride, const int32_t* targets, const float* old_logprobs, const float* advantages,
                          const float* weights, const float* ref_logprobs, float clip_low, float clip_high, float kl_coef, float* loss, float* token_loss, float* logprobs,
                          void* dlogits, long long d_stride, void* stream) {
    if (const int rc = check_logits(logits_dtype, T, V, row_stride)) return rc;
    if ((dlogits && d_stride < V) || !(clip_low >= 0.0f) || !(clip_high >= 0.0f) || !(kl_coef - kl_coef == 0.0f)) return BITLINEAR_ERR_SHAPE;
    if (!loss || (T > 0 && (!logits || !targets || !old_logprobs || !advantages || !token_loss || !logprobs || (kl_coef != 0.0f && !ref_logprobs)))) return BITLINEAR_ERR_NULL;
    if (logits == dlogits && T > 0 && d_stride != row_stride) return BITLINEAR_ERR_SHAPE;
    if (!element_aligned(logits, logits_dtype) || !element_aligned(dlogits, logits_dtype)) return BITLINEAR_ERR_ALIGN;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T > 0) {
        RowArgs a = {};
        a.logits = logits, a.stride = row_stride, a.targets = targets, a.V = V, a.logprobs = logprobs, a.status = device_status_word();
        a.old = old_logprobs, a.advantages = advantages, a.weights = weights, a.ref = ref_logprobs;
        a.clip_low = clip_low, a.clip_high = clip_high, a.kl = kl_coef;
        a.token_loss = token_loss, a.dlogits = dlogits, a.d_stride = d_stride;
        if (const int rc = rows_pass<kPolicy>(a, logits_dtype, T, st)) return rc;
    }
    return sum_pass(token_loss, T, 1.0, loss, st);
}

size_t bitlinear_preference_loss_workspace_bytes(int T) { return T <= 0 || T > (1 << 24) ? 0 : align_up((size_t)T * 12, 16); }

int bitlinear_preference_loss(const void* logits, int logits_dtype, int T, int V, long long row_stride, const int32_t* targets, const int32_t* cu_tokens, int pairs,
                              const float* ref_logprobs, float beta, float label_smoothing, float* loss, float* pair_loss, float* seq_logprobs, float* logprobs, void* dlogits,
                              long long d_stride, void* ws, size_t ws_bytes, void* stream) {
    if (const int rc = check_logits(logits_dtype, T, V, row_stride)) return rc;
    if (pairs <= 0 || pairs > (1 << 24) || (dlogits && d_stride < V) || !(beta - beta == 0.0f) || !(label_smoothing >= 0.0f && label_smoothing <= 1.0f))
        return BITLINEAR_ERR_SHAPE;
    if (!cu_tokens || !ref_logprobs || !loss || !pair_loss || !seq_logprobs || (T > 0 && (!logits || !targets || !logprobs))) return BITLINEAR_ERR_NULL;
    if (logits == dlogits && T > 0 && d_stride != row_stride) return BITLINEAR_ERR_SHAPE;
    if (!element_aligned(logits, logits_dtype) || !element_aligned(dlogits, logits_dtype)) return BITLINEAR_ERR_ALIGN;
    if (T > 0 && (!ws || !aligned16(ws) || ws_bytes < bitlinear_preference_loss_workspace_bytes(T))) return BITLINEAR_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    float2* stats = static_cast<float2*>(ws);
    float* grad = T > 0 && dlogits ? reinterpret_cast<float*>(stats + T) : nullptr;
    if (T > 0) {
        RowArgs a = {};
        a.logits = logits, a.stride = row_stride, a.targets = targets, a.V = V, a.logprobs = logprobs, a.stats = stats, a.grad = grad, a.status = device_status_word();
        if (const int rc = rows_pass<kLogp>(a, logits_dtype, T, st)) return rc;
    }
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = {};
    const bool few = pairs <= 8;  // one CTA after the other takes less than the launch of a sum
    cfg.gridDim = dim3(few ? 1u : (unsigned)std::min(pairs, 1024));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    launch_dependent(cfg, attr, 1);
    if (const int rc = finish(cudaLaunchKernelEx(&cfg, pair_kernel, (const float*)logprobs, targets, cu_tokens, ref_logprobs, T, V, pairs, beta, label_smoothing, pair_loss,
                                                 seq_logprobs, grad, few ? loss : nullptr)))
        return rc;
    if (!few)
        if (const int rc = sum_pass(pair_loss, pairs, 1.0 / pairs, loss, st)) return rc;
    if (!grad) return BITLINEAR_OK;
    const GradArgs g = {logits, row_stride, targets, stats, grad, dlogits, d_stride, T, V, 0};
    return grad_pass(g, logits_dtype, st);
}

}  // extern "C"
