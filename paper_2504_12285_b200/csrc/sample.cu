// The draw of the next token from a row of logits: temperature, top-k, top-p, min-p and one given random number per row.
//
//   w_i = exp((l_i - max l) / T);  keep the top_k largest, of those the shortest run from the largest down whose mass reaches
//   top_p of theirs, of those the ones with w_i >= min_p;  the token is the first in the order of ids whose running sum of
//   kept weights exceeds u times their total.  Equal logits rank by id.
//
// A row is read from memory once: a cluster of CTAs holds it in shared memory, a contiguous part each, and every later
// pass runs there.  No row is sorted.  A threshold (the k-th largest, the end of a mass) is found by histograms, best
// bins first: one over the logits' distance from the largest, linear, so that the elements spread over its bins, and then
// over an order-preserving integer image of the logits within the bin that holds the threshold, until that bin is taken
// whole or holds equal logits only.
//
// One row of 128,256 with every filter takes 16 us: load 2, each pass over the row 2 to 5, each meeting of the cluster 0.7;
// 16 rows of mixed settings 34 us, those with a wide top-p set the time: four shared-memory additions per element.
//
// Which token comes out hangs on sums next to a border, so weights are formed in fp64 and summed as integers in units of
// 2^-44 of the largest: sums of any order are the same, and no two machines' rounding of a sum decides a token.  The kernel without filters
// meets the largest on its way and holds to this within a part of a row only (see there).
#include "common.cuh"

#include <cooperative_groups.h>

#include <algorithm>
#include <mutex>

namespace cg = cooperative_groups;

namespace bitlinear {

namespace {

constexpr int kMaxCluster = 8;
constexpr int kMaxShard = 45056;  // floats of a row that one CTA holds
constexpr double kUnit44 = 17592186044416.0;  // 2^44
constexpr uint32_t kLowKey = 0x007fffffu;     // key of -inf

struct SampleArgs {
    const void* logits;
    long long stride;  // elements from a row to the next
    int M, V, shard, per;  // shard: elements per CTA; per: per thread (odd, so that a thread's own run meets every bank once)
    const float* u;
    const float* temperature;
    const int* top_k;
    const float* top_p;
    const float* min_p;
    int* ids;
    float* logprobs;
};

// at most 1e29; NaN stays NaN, which is not above 0
__device__ __forceinline__ float temperature_of(const SampleArgs& a, int row) {
    const float t = a.temperature ? a.temperature[row] : 1.0f;
    return t > 1e29f ? 1e29f : t;
}

// larger float, larger integer; -0 and 0 are equal
__device__ __forceinline__ uint32_t key_of(float l) {
    const uint32_t b = __float_as_uint(l + 0.0f);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float float_of(uint32_t key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu)); }

struct Crossing {
    int bin;
    uint32_t count_above, count;
    unsigned long long mass_above;
};

// kThreads: of a CTA
template <int kThreads>
struct SampleShared {
    static constexpr int kBinBits = kThreads == 512 ? 10 : 9;
    static constexpr int kBins = 1 << kBinBits;  // two per thread: a row has two CTAs at least, and each merges its share of the bins
    static constexpr int kList = kThreads;      // candidates of a row that one CTA finishes with
    double pow2[16];                            // 2^(j / 16): one entry to a pair of banks
    float top, low;             // largest logit of the part, smallest finite one
    int first;                  // lowest id of the largest logit in the part
    uint32_t ties;
    unsigned long long total;   // kept mass of the part
    Crossing cross;
    uint32_t slice_count;       // what this CTA's share of the merged bins holds
    unsigned long long slice_mass;
    unsigned long long warp_mass[kThreads / 32];
    uint32_t warp_count[kThreads / 32];
    float warp_top[kThreads / 32], warp_low[kThreads / 32];
    int cut_index;
    union {
        struct {
            uint32_t count[kBins];
            uint32_t mass[3][kBins];  // sums of the weights' low, middle and high 16 bits: shared memory adds 32-bit integers natively
        };
        struct {  // rank 0: the row's candidates in the order of ids, once they are few
            unsigned long long list_mass[kList];
            uint32_t list_key[kList];
            int list_id[kList];
        };
    };
};

struct Row {
    float top;        // largest logit
    float least;      // logits below weigh less than 2^-48 of the largest and are taken as this
    double top_d;
    double scale;     // 16 log2(e) / T
    const double* pow2;
    bool alone;       // nothing but the largest weighs anything: it is +infinity, or the next lower float is 34 temperatures away (or -infinity)
};
__device__ __forceinline__ Row relative_to(float top, float temp, const double* pow2) {
    const float least = top - 34.0f * temp;
    const bool alone = top == INFINITY || top < -3e38f || float_of(key_of(top) - 1) < least;
    return {top, least, (double)top, 16.0 * 1.4426950408889634074 / (double)temp, pow2, alone};
}

// exp((l - top) / T) = 2^(n / 16) * 2^(f / 16), n whole, |f| <= 1/2: the first from the table, the second by 1 + f q(f), q of degree 3 interpolating
// (2^(f / 16) - 1) / f at the Chebyshev nodes of -1/2 .. 1/2 (within 2^-37 of 2^(f / 16), exact at 0).  Returned as the two factors.  The table's
// entries lie in different banks, so lookups do not queue up; without it the series takes four more fp64 operations (42 cycles
// per 32 weights and scheduler against 35).
__device__ __forceinline__ void weight_factors(const Row& r, float l, double& series, double& power) {
    constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52: the sum's low bits are n
    const double d = (double)fmaxf(l, r.least) - r.top_d;
    const double t = fma(d, r.scale, kRound);
    const double f = fma(d, r.scale, kRound - t);
    const int n = __double2loint(t);
    double q = fma(f, 1.4676329855091502e-07, 1.3551125679403628e-05);
    q = fma(f, q, 0.0009383847927372583);
    q = fma(f, q, 0.043321698775062194);
    series = fma(f, q, 1.0);
    const double base = r.pow2[n & 15];
    power = __hiloint2double(__double2hiint(base) + ((n << 16) & 0xfff00000), __double2loint(base));
}
__device__ __forceinline__ double weight_of(const Row& r, float l) {
    double series, power;
    weight_factors(r, l, series, power);
    return series * power;
}
// the weight in units of 2^-44, rounded to nearest: the last bits of its sum with 256
constexpr unsigned long long kBits256 = 0x4070000000000000ull;
__device__ __forceinline__ unsigned long long fixed_of(const Row& r, float l) {
    double series, power;
    weight_factors(r, l, series, power);
    return (unsigned long long)__double_as_longlong(fma(series, power, 256.0)) - kBits256;
}

// the running sum that the drawn token is the first to exceed
__device__ __forceinline__ unsigned long long drawn_at(float u, unsigned long long all) {
    const double goal = u > 0.0f ? (double)u * (double)all : 0.0;
    const unsigned long long at = goal < 9.2e18 ? (unsigned long long)goal : all;  // sum > goal, in whole numbers: > its floor
    return at >= all ? all - 1 : at;                                               // u = 1: the last token that is kept
}

template <class T>
__device__ __forceinline__ float load_logit(const T* p);
template <>
__device__ __forceinline__ float load_logit<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float load_logit<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }

// 2^(j / 16)
__device__ const double kPow2Table[16] = {1.0, 1.0442737824274138, 1.0905077326652577, 1.1387886347566916, 1.189207115002721, 1.241857812073484, 1.2968395546510096, 1.3542555469368927, 1.4142135623730951, 1.4768261459394993, 1.5422108254079407, 1.6104903319492543, 1.681792830507429, 1.7562521603732995, 1.8340080864093424, 1.9152065613971474};

// 512 threads and an SM to itself where every CTA can have one; else 256, of which three CTAs share an SM, so that some load while
// others compute (192 rows of 128,256 without filters: two CTAs of 512 took 77 us, three of 256 took 64)
template <class T, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 512 ? 1 : 3) sample_kernel(const SampleArgs a) {
    using Shared = SampleShared<kThreads>;
    constexpr int kBins = Shared::kBins, kList = Shared::kList;
        extern __shared__ __align__(16) uint8_t sample_raw[];
    Shared& sh = *reinterpret_cast<Shared*>(sample_raw);
    float* room = reinterpret_cast<float*>(sample_raw + (sizeof(Shared) + 15) / 16 * 16);
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = blockIdx.x / ranks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid < 16) sh.pow2[tid] = kPow2Table[tid];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long begin = (long long)rank * a.shard;
    const int n = (int)max(0ll, min((long long)a.shard, a.V - begin));
    const T* src = static_cast<const T*>(a.logits) + (size_t)row * a.stride + begin;
    const float temp = temperature_of(a, row);
    const int k = a.top_k ? a.top_k[row] : 0;
    const float p = a.top_p ? a.top_p[row] : 1.0f;
    const float given_mp = a.min_p ? a.min_p[row] : 0.0f;
    const float u = a.u[row];

    // ---- the part into shared memory; the largest and (where a histogram will want it) the smallest finite logit
    const bool use_k = k > 0 && k < a.V, use_p = p < 1.0f, want_low = use_k || use_p;
    float top = -INFINITY, low = INFINITY;
    auto take = [&](float l) {
        l = l == l ? l : -INFINITY;  // NaN: never drawn
        top = fmaxf(top, l);
        if (want_low) low = fminf(low, l > -INFINITY ? l : INFINITY);
        return l;
    };
    constexpr int VEC = 16 / sizeof(T), AHEAD = 4;
    const int head = (int)min((long long)n, (long long)(((16 - (reinterpret_cast<uintptr_t>(src) & 15)) & 15) / sizeof(T)));
    const int n_vec = (n - head) / VEC;
    float* vals = room + ((4 - (head & 3)) & 3);  // what comes 16 bytes at a time goes there 16 bytes at a time
    const uint4* vsrc = reinterpret_cast<const uint4*>(src + head);
    for (int v0 = tid; v0 < n_vec; v0 += AHEAD * kThreads) {
        uint4 x[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (v0 + j * kThreads < n_vec) x[j] = __ldcs(vsrc + v0 + j * kThreads);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (v0 + j * kThreads >= n_vec) break;
            const T* e = reinterpret_cast<const T*>(&x[j]);
            float4* dst = reinterpret_cast<float4*>(vals + head + (v0 + j * kThreads) * VEC);
#pragma unroll
            for (int i = 0; i < VEC / 4; ++i)
                dst[i] = make_float4(take(load_logit(e + 4 * i)), take(load_logit(e + 4 * i + 1)), take(load_logit(e + 4 * i + 2)), take(load_logit(e + 4 * i + 3)));
        }
    }
    for (int i = tid; i < head; i += kThreads) vals[i] = take(load_logit(src + i));
    for (int i = head + n_vec * VEC + tid; i < n; i += kThreads) vals[i] = take(load_logit(src + i));
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, off));
    }
    if (lane == 0) sh.warp_top[warp] = top, sh.warp_low[warp] = low;
    if (tid == 0) sh.first = 0x7fffffff;
    __syncthreads();
    if (warp == 0) {
        top = sh.warp_top[lane & (kThreads / 32 - 1)];
        low = sh.warp_low[lane & (kThreads / 32 - 1)];
#pragma unroll
        for (int off = kThreads / 64; off > 0; off >>= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            low = fminf(low, __shfl_xor_sync(0xffffffffu, low, off));
        }
        if (lane == 0) sh.top = top, sh.low = low;
    }
    cluster.sync();
    {
        float tops[kMaxCluster], lows[kMaxCluster];
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) {
            const Shared* o = cluster.map_shared_rank(&sh, r < ranks ? r : 0);
            tops[r] = o->top;
            lows[r] = o->low;
        }
        top = tops[0], low = lows[0];
#pragma unroll
        for (int r = 1; r < kMaxCluster; ++r) top = fmaxf(top, tops[r]), low = fminf(low, lows[r]);
    }
    const int i0 = min(tid * a.per, n), i1 = min(i0 + a.per, n);
    const bool empty = top == -INFINITY, greedy = !(temp > 0.0f);
    if (empty || greedy) {  // the same in every CTA of the cluster
        if (!empty) {
            for (int i = i0; i < i1; ++i)
                if (vals[i] == top) {
                    atomicMin(&sh.first, (int)(begin + i));
                    break;
                }
            cluster.sync();
        }
        if (rank == 0 && tid == 0) {
            int first = 0x7fffffff;
            for (int r = 0; r < ranks; ++r) first = min(first, cluster.map_shared_rank(&sh, r)->first);
            a.ids[row] = empty ? -1 : first;
            if (a.logprobs) a.logprobs[row] = empty ? -INFINITY : 0.0f;
        }
        cluster.sync();  // no CTA leaves while another reads its shared memory
        return;
    }
    Row rw = relative_to(top, temp, sh.pow2);
    if (rw.alone) {  // as if the largest were 0 and all else -infinity, at any temperature
        for (int i = i0; i < i1; ++i) vals[i] = vals[i] == top ? 0.0f : -INFINITY;
        top = low = 0.0f;
        rw = relative_to(top, 1.0f, sh.pow2);
        __syncthreads();
    }
    const uint32_t top_key = key_of(top);
    const double mp = given_mp > 0.0f ? fmin((double)given_mp, 1.0) : 0.0;  // the largest, of weight 1, always stays

    // kept so far: keys above floor_key, and of those equal to it the ones up to floor_index
    uint32_t floor_key = 0;
    int floor_index = 0x7fffffff;
    auto kept = [&](uint32_t key, int i) { return key > floor_key || (key == floor_key && (int)begin + i <= floor_index); };
    // f(logit, place, whether it is kept) for the elements of this thread's run; four at a time and without branches, so that
    // the chains of dependent operations of several elements run side by side
    auto each = [&](auto&& f) {
        int i = i0;
        for (; i + 4 <= i1; i += 4) {
            const float l[4] = {vals[i], vals[i + 1], vals[i + 2], vals[i + 3]};
            bool in[4] = {true, true, true, true};
            if (floor_key != 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j) in[j] = kept(key_of(l[j]), i + j);
            }
            f(l, in, i);
        }
        if (i < i1) {
            float l[4];
            bool in[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) l[j] = vals[min(i + j, i1 - 1)], in[j] = i + j < i1 && kept(key_of(l[j]), i + j);
            f(l, in, i);
        }
    };
    // Two cluster barriers make up a pass: its sums are ready, and everyone has read them.  The second is waited for only where
    // the fields it guards are written again.
    bool pending = false;
    auto settle = [&]() {
        if (pending) cluster.barrier_wait();
        pending = false;
    };
    auto read_done = [&]() {
        cluster.barrier_arrive();
        pending = true;
    };

    // ---- thresholds
    // linear bins of the first histogram: distances from the largest up to where weights vanish or the logits end
    const float span = fminf(top - low, 40.0f * temp);
    const float to_bin = span > 0.0f ? (float)kBins / span : 0.0f;
    auto linear_bin = [&](float l) {  // monotone: a larger logit never gets a later bin
        const float d = (top - l) * to_bin;
        return d < (float)(kBins - 1) ? (int)d : kBins - 1;  // the last takes the rest, -inf and inf - inf too
    };
    // the smallest key whose linear bin is `bin` or an earlier one; each step of the search tries 32 keys
    auto first_key = [&](int bin) {
        uint32_t lo = kLowKey, hi = top_key + 1;  // the answer lies in lo .. hi; hi: none
        while (lo < hi) {
            const uint32_t step = (hi - lo) / 32 + 1, at = lo + lane * step;  // (keys end at infinity's: no overflow)
            const unsigned m = __ballot_sync(0xffffffffu, at >= hi || linear_bin(float_of(at)) <= bin);
            const uint32_t f = m ? (uint32_t)__ffs((int)m) - 1 : 32u;
            if (f < 32) hi = min(hi, lo + f * step);
            if (f > 0) lo = lo + (f - 1) * step + 1;
        }
        return hi;
    };
    // one histogram over the part's elements to which bin_of gives a bin, merged over the cluster; the bin in which the running
    // count (or mass) reaches the target
    // (sparse: few elements have a bin, so weights are formed for those alone; a target below 0 becomes top_p of the mass of all bins)
    auto find = [&](bool by_mass, bool sparse, uint32_t want, double& target, uint32_t count0, unsigned long long mass0, auto&& bin_of) {
        settle();
        for (int b = tid; b < kBins; b += kThreads) {
            sh.count[b] = 0;
            if (by_mass) sh.mass[0][b] = sh.mass[1][b] = sh.mass[2][b] = 0;
        }
        __syncthreads();
        auto add = [&](int b, unsigned long long w) {
            const uint32_t w2 = (uint32_t)(w >> 32);
            atomicAdd(&sh.count[b], 1u);
            atomicAdd(&sh.mass[0][b], (uint32_t)w & 0xffffu);
            atomicAdd(&sh.mass[1][b], (uint32_t)w >> 16);
            if (w2) atomicAdd(&sh.mass[2][b], w2);
        };
        if (by_mass && !sparse) {
            each([&](const float (&l)[4], const bool (&in)[4], int) {
                unsigned long long w[4];
                int b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = fixed_of(rw, l[j]), b[j] = in[j] ? bin_of(l[j], key_of(l[j])) : -1;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (b[j] >= 0) add(b[j], w[j]);
            });
        } else if (by_mass) {
            each([&](const float (&l)[4], const bool (&in)[4], int) {
                int b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) b[j] = in[j] ? bin_of(l[j], key_of(l[j])) : -1;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (b[j] >= 0) add(b[j], fixed_of(rw, l[j]));
            });
        } else {
            each([&](const float (&l)[4], const bool (&in)[4], int) {
                int b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) b[j] = in[j] ? bin_of(l[j], key_of(l[j])) : -1;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (b[j] >= 0) atomicAdd(&sh.count[b[j]], 1u);
            });
        }
        cluster.sync();
        // each CTA merges its share of the bins, one per thread
        const int share = kBins / ranks, bin = rank * share + tid;
        uint32_t c = 0;
        unsigned long long m = 0;
        if (tid < share) {
            uint32_t x[kMaxCluster];
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r) x[r] = r < ranks ? cluster.map_shared_rank(&sh, r)->count[bin] : 0u;
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r) c += x[r];
            if (by_mass) {
#pragma unroll
                for (int j = 0; j < 3; ++j) {
#pragma unroll
                    for (int r = 0; r < kMaxCluster; ++r) x[r] = r < ranks ? cluster.map_shared_rank(&sh, r)->mass[j][bin] : 0u;
                    unsigned long long t = 0;
#pragma unroll
                    for (int r = 0; r < kMaxCluster; ++r) t += x[r];
                    m += t << (16 * j);
                }
            }
        }
        uint32_t ci = c;
        unsigned long long mi = m;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t cu = __shfl_up_sync(0xffffffffu, ci, d);
            const unsigned long long mu = __shfl_up_sync(0xffffffffu, mi, d);
            if (lane >= d) ci += cu, mi += mu;
        }
        if (lane == 31) sh.warp_count[warp] = ci, sh.warp_mass[warp] = mi;
        __syncthreads();
        uint32_t ca = ci - c, cs = 0;
        unsigned long long ma = mi - m, ms = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w * 32 >= share) break;
            const uint32_t ct = sh.warp_count[w];
            const unsigned long long mt = sh.warp_mass[w];
            if (w < warp) ca += ct, ma += mt;
            cs += ct, ms += mt;
        }
        if (tid == 0) sh.slice_count = cs, sh.slice_mass = ms;
        cluster.sync();
        ca += count0, ma += mass0;
        {
            uint32_t ct[kMaxCluster];
            unsigned long long mt[kMaxCluster], total = 0;
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r) {
                const Shared* o = cluster.map_shared_rank(&sh, min(r, ranks - 1));
                ct[r] = o->slice_count, mt[r] = o->slice_mass;
            }
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r) {
                if (r < rank) ca += ct[r], ma += mt[r];
                if (r < ranks) total += mt[r];
            }
            if (by_mass && target < 0.0) target = fmax((double)p * (double)total, 0.5);
        }
        const bool here = by_mass ? (double)ma < target && (double)(ma + m) >= target : ca < want && ca + c >= want;
        if (here && c > 0)
            for (int r = 0; r < ranks; ++r) cluster.map_shared_rank(&sh, r)->cross = {bin, ca, c, ma};
        cluster.sync();
        return sh.cross;
    };
    // of the elements equal to floor_key the first `keep` by id stay: the id of the last of them
    auto cut_ties = [&](uint32_t keep) {
        settle();
        uint32_t mine = 0;
        each([&](const float (&l)[4], const bool (&in)[4], int) {
#pragma unroll
            for (int j = 0; j < 4; ++j) mine += in[j] && key_of(l[j]) == floor_key;
        });
        uint32_t incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += up;
        }
        __syncthreads();
        if (lane == 31) sh.warp_count[warp] = incl;
        __syncthreads();
        uint32_t before = incl - mine;
        for (int w = 0; w < warp; ++w) before += sh.warp_count[w];
        if (tid == kThreads - 1) sh.ties = before + mine;
        if (tid == 0) sh.cut_index = -1;
        cluster.sync();
        for (int r = 0; r < rank; ++r) before += cluster.map_shared_rank(&sh, r)->ties;
        if (before < keep && before + mine >= keep) {
            uint32_t left = keep - before;
            each([&](const float (&l)[4], const bool (&in)[4], int i) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (in[j] && key_of(l[j]) == floor_key && --left == 0) sh.cut_index = (int)begin + i + j;
            });
        }
        cluster.sync();
        int cut = -1;
        for (int r = 0; r < ranks; ++r) cut = max(cut, cluster.map_shared_rank(&sh, r)->cut_index);
        floor_index = cut;
        read_done();
    };
    // Narrows what is kept to the run from the largest down that reaches the target.  The bin that holds the run's end
    // is split until the run takes all of it or it is a single key, whose elements then go by id.
    auto narrow = [&](Crossing x, bool by_mass, uint32_t want, double target) {
        uint32_t lo = first_key(x.bin), hi = (x.bin == 0 ? top_key + 1 : first_key(x.bin - 1)) - 1;
        while (x.count > 1 && lo < hi && (by_mass || x.count_above + x.count != want)) {
            const int shift = max(0, 32 - __clz((int)(hi - lo)) - Shared::kBinBits);  // hi - lo < 2^(shift + kBinBits)
            const uint32_t from = hi, to = lo;
            x = find(by_mass, true, want, target, x.count_above, x.mass_above, [&](float, uint32_t key) { return key >= to && key <= from ? (int)((from - key) >> shift) : -1; });
            hi = from - ((uint32_t)x.bin << shift);
            lo = hi - to >= (1u << shift) ? hi - ((1u << shift) - 1u) : to;
        }
        uint32_t keep = x.count;
        if (by_mass && x.count > 1) {
            const double each = (double)fixed_of(rw, float_of(lo)), need = ceil((target - (double)x.mass_above) / fmax(each, 1.0));
            keep = need < 1.0 ? 1u : need > (double)x.count ? x.count : (uint32_t)need;
        } else if (!by_mass) {
            keep = want - x.count_above;
        }
        if (lo > floor_key) floor_key = lo, floor_index = 0x7fffffff;  // an earlier cut was among another key's ties
        if (keep < x.count) cut_ties(keep);
    };
    // sum of v over the threads in front of this one, and over all
    auto scan_mass = [&](unsigned long long v, unsigned long long& all) {
        unsigned long long incl = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned long long up = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += up;
        }
        __syncthreads();
        if (lane == 31) sh.warp_mass[warp] = incl;
        __syncthreads();
        unsigned long long before = incl - v;
        all = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            const unsigned long long t = sh.warp_mass[w];
            if (w < warp) before += t;
            all += t;
        }
        return before;
    };
    // Few candidates are left, those in the bins up to last_bin: rank 0 takes them all, one per thread in the order of ids, ranks
    // them by counting, and draws; the other CTAs are done.  want: top_k, or 0; target: top_p's mass, below 0 where it is to be formed from
    // the top_k here.
    auto finish = [&](int last_bin, uint32_t want, double target) {
        settle();
        uint32_t mine = 0;
        each([&](const float (&l)[4], const bool (&in)[4], int) {
#pragma unroll
            for (int j = 0; j < 4; ++j) mine += in[j] && linear_bin(l[j]) <= last_bin;
        });
        uint32_t incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += up;
        }
        __syncthreads();
        if (lane == 31) sh.warp_count[warp] = incl;
        __syncthreads();
        uint32_t at = incl - mine, there = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            const uint32_t t = sh.warp_count[w];
            if (w < warp) at += t;
            there += t;
        }
        if (tid == 0) sh.ties = there;
        cluster.sync();
        {
            uint32_t t[kMaxCluster];
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r) t[r] = r < ranks ? cluster.map_shared_rank(&sh, r)->ties : 0;
            there = 0;
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r) {
                if (r < rank) at += t[r];
                there += t[r];
            }
        }
        Shared* first = cluster.map_shared_rank(&sh, 0);
        if (mine)
            each([&](const float (&l)[4], const bool (&in)[4], int i) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (in[j] && linear_bin(l[j]) <= last_bin) {
                        first->list_key[at] = key_of(l[j]);
                        first->list_id[at++] = (int)begin + i + j;
                    }
            });
        cluster.sync();
        if (rank != 0) return;
        const int m = (int)there;
        const bool in = tid < m;
        const uint32_t key = in ? sh.list_key[tid] : 0;
        int place = 0;  // how many are larger, or equal with a lower id
        if (warp * 32 < m) {
            int j = 0;
            for (; j < m; ++j) {
                const uint32_t o = sh.list_key[j];
                place += o > key || (o == key && j < tid);
            }
        }
        const float l = float_of(key);
        const double w = in ? weight_of(rw, l) : 0.0;
        unsigned long long mass = in && (want == 0 || place < (int)want) ? fixed_of(rw, l) : 0, total;
        bool stays = in && (want == 0 || place < (int)want);
        if (use_p) {
            sh.list_mass[tid] = 0;
            __syncthreads();
            if (stays) sh.list_mass[place] = mass;
            __syncthreads();
            const unsigned long long ahead = scan_mass(sh.list_mass[tid], total);
            if (target < 0.0) target = fmax((double)p * (double)total, 0.5);
            __syncthreads();
            sh.list_mass[tid] = ahead;
            __syncthreads();
            if (stays) stays = (double)sh.list_mass[place] < target;
        }
        if (w < mp) stays = false;
        if (!stays) mass = 0;
        const unsigned long long ahead = scan_mass(mass, total);
        const unsigned long long goal = drawn_at(u, total);
        if (ahead <= goal && goal < ahead + mass) {
            a.ids[row] = sh.list_id[tid];
            if (a.logprobs) a.logprobs[row] = (float)log(w * kUnit44 / (double)total);
        }
    };
    // mass of what is kept and weighs at least `least`, over the cluster; `mine`: this thread's run, `before`: what lies in front of it
    auto kept_mass = [&](double least, unsigned long long& mine, unsigned long long& before) {
        settle();
        mine = 0;
        if (floor_key == 0 && least == 0.0) {  // nothing is left out: the loop carries no tests, and 256's bits are taken off at its end
            int i = i0;
#pragma unroll 1
            for (; i + 4 <= i1; i += 4) {
                const float l[4] = {vals[i], vals[i + 1], vals[i + 2], vals[i + 3]};
#pragma unroll
                for (int j = 0; j < 4; ++j) mine += fixed_of(rw, l[j]) + kBits256;
            }
            for (; i < i1; ++i) mine += fixed_of(rw, vals[i]) + kBits256;
            mine -= (unsigned long long)(i1 - i0) * kBits256;
        } else {
            each([&](const float (&l)[4], const bool (&in)[4], int) {
                double series[4], power[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) weight_factors(rw, l[j], series[j], power[j]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool stays = in[j] && (least == 0.0 || series[j] * power[j] >= least);
                    mine += stays ? (unsigned long long)__double_as_longlong(fma(series[j], power[j], 256.0)) - kBits256 : 0ull;
                }
            });
        }
        unsigned long long incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned long long up = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += up;
        }
        __syncthreads();
        if (lane == 31) sh.warp_mass[warp] = incl;
        __syncthreads();
        before = incl - mine;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w)
            if (w < warp) before += sh.warp_mass[w];
        if (tid == kThreads - 1) sh.total = before + mine;
        cluster.sync();
        unsigned long long t[kMaxCluster], all = 0;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) t[r] = r < ranks ? cluster.map_shared_rank(&sh, r)->total : 0;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) {
            if (r < rank) before += t[r];
            all += t[r];
        }
        read_done();
        return all;
    };

    unsigned long long mine, before;
    auto by_distance = [&](float l, uint32_t) { return linear_bin(l); };
    if (use_k) {
        double none = 0.0;
        const Crossing x = find(false, false, (uint32_t)k, none, 0, 0, by_distance);
        if (x.count_above + x.count <= kList) return finish(x.bin, (uint32_t)k, -1.0);
        narrow(x, false, (uint32_t)k, 0.0);
    }
    if (use_p) {
        double target = -1.0;
        const Crossing x = find(true, false, 0, target, 0, 0, by_distance);
        if (x.count_above + x.count <= kList) return finish(x.bin, 0, target);
        narrow(x, true, 0, target);
    }
    const unsigned long long all = kept_mass(mp, mine, before);
    const unsigned long long at = drawn_at(u, all);
    // the thread whose run holds it; its warp finds the element
    const unsigned holds = __ballot_sync(0xffffffffu, before <= at && at < before + mine);
    if (holds) {
        const int who = __ffs((int)holds) - 1;
        unsigned long long run = __shfl_sync(0xffffffffu, before, who);
        const int j0 = __shfl_sync(0xffffffffu, i0, who), j1 = __shfl_sync(0xffffffffu, i1, who);
        for (int j = j0; j < j1; j += 32) {
            const int i = j + lane;
            double w = 0.0;
            unsigned long long f = 0;
            if (i < j1 && kept(key_of(vals[i]), i)) {
                w = weight_of(rw, vals[i]);
                if (w >= mp) f = fixed_of(rw, vals[i]);
            }
            unsigned long long incl = f;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const unsigned long long up = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += up;
            }
            const unsigned past = __ballot_sync(0xffffffffu, run + incl > at);
            if (past) {
                if (lane == __ffs((int)past) - 1) {
                    a.ids[row] = (int)begin + i;
                    if (a.logprobs) a.logprobs[row] = (float)log(w * kUnit44 / (double)all);
                }
                break;
            }
            run += __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    settle();  // no CTA leaves while another reads its shared memory
}

// The draw without filters: no threshold is wanted, so nothing is kept of a row.  Each warp of a cluster streams a contiguous part, its
// weights relative to the largest logit it has met (a larger one rescales its sum, at most 24 times at the largest vocabulary, each by a
// factor good to 2^-37: a total is good to 2^-31 and depends in its last bits on where the parts begin); the cluster joins the warps' sums, and the
// warp in whose part the goal lies goes over that part once more.  The weights' fp64 operations alone, 35 cycles per 32 weights and
// scheduler, are 24 us for 192 rows of 128,256; the kernel takes 52 us (the one with filters 64): four CTAs of 256 threads per SM
// beat two of 512 (63 us), eight elements per lane with the next eight on their way beat sixteen (62 us), and one join by the
// first warps beat two barriers (80 us).
constexpr int kPlainThreads = 256, kPlainWarps = kPlainThreads / 32;
constexpr int kLane = 8;  // elements that a lane takes at a time
struct PlainShared {
    double pow2[16];
    float warp_top[kPlainWarps];
    unsigned long long warp_mass[kPlainWarps];
    unsigned long long best[kPlainWarps];  // greedy: key of the largest logit, ~id
    unsigned long long first;
};

template <class T>
__global__ void __launch_bounds__(kPlainThreads, 4) sample_plain_kernel(const SampleArgs a) {
    __shared__ PlainShared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = blockIdx.x / ranks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid < 16) sh.pow2[tid] = kPow2Table[tid];
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float temp = temperature_of(a, row);
    const float u = a.u[row];
    const T* src = static_cast<const T*>(a.logits) + (size_t)row * a.stride;
    // the row: elements up to a 16-byte border (worker 0), 16-byte vectors dealt to the workers in equal runs, the rest (the last worker)
    constexpr int VEC = 16 / sizeof(T), SUB = kLane / VEC;  // vectors of a lane's elements
    const int head = min(a.V, (int)(((16 - (reinterpret_cast<uintptr_t>(src) & 15)) & 15) / sizeof(T)));
    const int n_vec = (a.V - head) / VEC, tail = head + n_vec * VEC;
    const int workers = ranks * kPlainWarps, me = rank * kPlainWarps + warp;
    const uint4* vsrc = reinterpret_cast<const uint4*>(src + head);
    // f(logits, id of the first, ids between subs, elements of a sub) over worker w's part in the order of ids until it returns true; what does not
    // exist, and NaN, is -inf
    auto over_part = [&](int w, auto&& f) {
        const int v0 = (int)((long long)n_vec * w / workers), v1 = (int)((long long)n_vec * (w + 1) / workers);
        auto single = [&](int from, int to) {  // fewer than 8 elements, one per lane
            float l[kLane];
#pragma unroll
            for (int i = 0; i < kLane; ++i) l[i] = -INFINITY;
            if (from + lane < to) l[0] = fmaxf(load_logit(src + from + lane), -INFINITY);
            return f(l, from + lane, 0, 1);
        };
        if (w == 0 && head > 0 && single(0, head)) return;
        uint4 x[SUB], y[SUB];
        auto fetch = [&](uint4 (&z)[SUB], int v) {
#pragma unroll
            for (int j = 0; j < SUB; ++j)
                if (v + 32 * j + lane < v1) z[j] = __ldcs(vsrc + v + 32 * j + lane);
        };
        fetch(x, v0);
        for (int v = v0; v < v1; v += 32 * SUB) {
            fetch(y, v + 32 * SUB);  // the next ones come in while these are worked on
            float l[kLane];
#pragma unroll
            for (int j = 0; j < SUB; ++j) {
                const T* e = reinterpret_cast<const T*>(&x[j]);
                const bool in = v + 32 * j + lane < v1;
#pragma unroll
                for (int i = 0; i < VEC; ++i) l[j * VEC + i] = in ? fmaxf(load_logit(e + i), -INFINITY) : -INFINITY;
            }
            if (f(l, head + (v + lane) * VEC, 32 * VEC, VEC)) return;
#pragma unroll
            for (int j = 0; j < SUB; ++j) x[j] = y[j];
        }
        if (w == workers - 1 && tail < a.V) single(tail, a.V);
    };
    if (!(temp > 0.0f)) {  // greedy: the largest, lowest id first
        unsigned long long best = 0;
        over_part(me, [&](const float (&l)[kLane], int id, int step, int n) {
#pragma unroll
            for (int i = 0; i < kLane; ++i)
                if (step > 0 || i == 0)
                    best = max(best, ((unsigned long long)key_of(l[i]) << 32) | (0xffffffffu - (uint32_t)(id + (i / VEC) * step + i % VEC)));
            return false;
        });
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, off));
        if (lane == 0) sh.best[warp] = best;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kPlainWarps; ++w) best = max(best, sh.best[w]);
            sh.first = best;
        }
        cluster.sync();
        if (rank == 0 && tid == 0) {
            for (int r = 0; r < ranks; ++r) best = max(best, cluster.map_shared_rank(&sh, r)->first);
            const bool none = (uint32_t)(best >> 32) <= kLowKey;
            a.ids[row] = none ? -1 : (int)(0xffffffffu - (uint32_t)best);
            if (a.logprobs) a.logprobs[row] = none ? -INFINITY : 0.0f;
        }
        cluster.sync();  // no CTA leaves while another reads its shared memory
        return;
    }
    auto fixed_at = [&](const Row& r, float l) { return r.alone ? (l == r.top ? 1ull << 44 : 0ull) : fixed_of(r, l); };
    Row rw = {-INFINITY, 0.0f, 0.0, 0.0, sh.pow2, false};
    unsigned long long mass = 0;  // this lane's, in units of 2^-44 of the weight of rw.top
    over_part(me, [&](const float (&l)[kLane], int, int, int) {
        float top = l[0];
#pragma unroll
        for (int i = 1; i < kLane; ++i) top = fmaxf(top, l[i]);
        if (__any_sync(0xffffffffu, top > rw.top)) {
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const Row next = relative_to(top, temp, sh.pow2);
            mass = rw.top <= next.least || next.alone ? 0ull : (unsigned long long)__double2ll_rn((double)mass * weight_of(next, rw.top));
            rw = next;
        }
        if (rw.top == -INFINITY) return false;
        if (rw.alone) {
#pragma unroll
            for (int i = 0; i < kLane; ++i) mass += l[i] == rw.top ? 1ull << 44 : 0ull;
            return false;
        }
        unsigned long long sum = 0;
#pragma unroll
        for (int i = 0; i < kLane; ++i) sum += fixed_of(rw, l[i]) + kBits256;
        mass += sum - kLane * kBits256;
        return false;
    });
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, off);
    if (lane == 0) sh.warp_top[warp] = rw.top, sh.warp_mass[warp] = mass;
    cluster.sync();
    if (warp > 0) {  // the first warp of every CTA joins the sums of all; what it has read it needs no more
        cluster.barrier_arrive();
        cluster.barrier_wait();
        return;
    }
    constexpr int EACH = kMaxCluster * kPlainWarps / 32;  // lane l holds the sums of workers EACH l ...
    float tops[EACH];
    unsigned long long sums[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int w = EACH * lane + i;
        const PlainShared* o = cluster.map_shared_rank(&sh, min(w / kPlainWarps, ranks - 1));
        tops[i] = w < workers ? o->warp_top[w % kPlainWarps] : -INFINITY;
        sums[i] = w < workers ? o->warp_mass[w % kPlainWarps] : 0ull;
    }
    cluster.barrier_arrive();
    float top = tops[0];
#pragma unroll
    for (int i = 1; i < EACH; ++i) top = fmaxf(top, tops[i]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    if (top == -INFINITY) {
        if (rank == 0 && tid == 0) {
            a.ids[row] = -1;
            if (a.logprobs) a.logprobs[row] = -INFINITY;
        }
        cluster.barrier_wait();
        return;
    }
    const Row rt = relative_to(top, temp, sh.pow2);
    unsigned long long joined = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const double factor = tops[i] == top ? 1.0 : tops[i] <= rt.least || rt.alone ? 0.0 : weight_of(rt, tops[i]);
        sums[i] = (unsigned long long)__double2ll_rn((double)sums[i] * factor);
        joined += sums[i];
    }
    unsigned long long incl = joined;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long up = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += up;
    }
    const unsigned long long all = __shfl_sync(0xffffffffu, incl, 31);
    const unsigned long long at = drawn_at(u, all);
    // the worker in whose part the goal lies, and what lies in front of it
    const int holder = __ffs((int)__ballot_sync(0xffffffffu, incl > at)) - 1;
    int owner = EACH * lane;
    unsigned long long before = incl - joined;
#pragma unroll
    for (int i = 0; i < EACH - 1; ++i)
        if (owner == EACH * lane + i && before + sums[i] <= at) before += sums[i], ++owner;
    owner = __shfl_sync(0xffffffffu, owner, holder);
    before = __shfl_sync(0xffffffffu, before, holder);
    if (owner / kPlainWarps == rank) {
        // sums of single weights may differ from the joined ones in the last units: where they end short of the goal, the last
        // element of any weight is the one, or the largest where each alone rounds to none
        unsigned long long run = before;
        int last = -1, big = 0;
        float last_l = 0.0f, big_l = -INFINITY;
        over_part(owner, [&](const float (&l)[kLane], int id, int step, int n) {
#pragma unroll
            for (int j = 0; j < SUB; ++j) {
                if (step == 0 && j > 0) break;
                unsigned long long f[VEC], sum = 0;
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    f[i] = i < n ? fixed_at(rt, l[j * VEC + i]) : 0ull;
                    if (f[i]) last = id + j * step + i, last_l = l[j * VEC + i];
                    if (i < n && l[j * VEC + i] > big_l) big = id + j * step + i, big_l = l[j * VEC + i];
                    sum += f[i];
                }
                unsigned long long upto = sum;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const unsigned long long up = __shfl_up_sync(0xffffffffu, upto, d);
                    if (lane >= d) upto += up;
                }
                const unsigned past = __ballot_sync(0xffffffffu, run + upto > at);
                if (past) {
                    if (lane == __ffs((int)past) - 1) {
                        unsigned long long s = run + upto - sum;
                        bool taken = false;
#pragma unroll
                        for (int i = 0; i < VEC; ++i) {
                            s += f[i];
                            if (!taken && s > at) taken = true, last = id + j * step + i, last_l = l[j * VEC + i];
                        }
                    } else {
                        last = -1;
                    }
                    return true;
                }
                run += __shfl_sync(0xffffffffu, upto, 31);
            }
            return false;
        });
        if (!__any_sync(0xffffffffu, last >= 0)) {
            float most_l = big_l;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) most_l = fmaxf(most_l, __shfl_xor_sync(0xffffffffu, most_l, off));
            if (big_l == most_l) last = big, last_l = big_l;
        }
        int most = last;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, off));
        if (last == most && last >= 0) {
            a.ids[row] = last;
            if (a.logprobs) a.logprobs[row] = (float)log((rt.alone ? 1.0 : weight_of(rt, last_l)) * kUnit44 / (double)all);
        }
    }
    cluster.barrier_wait();
}

int launch_rows(const void* kernel, SampleArgs a, int ranks, int threads, size_t smem, cudaStream_t st) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.M * ranks));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    void* args[1] = {&a};
    if (cudaLaunchKernelExC(&cfg, kernel, args) != cudaSuccess) {
        cudaGetLastError();
        return BITLINEAR_ERR_CUDA;
    }
    return BITLINEAR_OK;
}

template <class T, int kThreads>
int sample_launch(SampleArgs a, int ranks, cudaStream_t st) {
    static std::mutex mu;
    static bool done[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return BITLINEAR_ERR_CUDA;
    }
    constexpr size_t fixed = (sizeof(SampleShared<kThreads>) + 15) / 16 * 16;
    const void* kernel = reinterpret_cast<const void*>(sample_kernel<T, kThreads>);
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!done[dev]) {
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(fixed + (kMaxShard + 4) * sizeof(float))) != cudaSuccess) {
                cudaGetLastError();
                return BITLINEAR_ERR_CUDA;
            }
            done[dev] = true;
        }
    }
    a.per = (a.shard + kThreads - 1) / kThreads | 1;
    return launch_rows(kernel, a, ranks, kThreads, fixed + (size_t)(a.shard + 4) * sizeof(float), st);
}

}  // namespace

}  // namespace bitlinear

using namespace bitlinear;

extern "C" int bitlinear_sample(const void* logits, int logits_dtype, int M, int V, long long row_stride, const float* u, const float* temperature,
                                const int32_t* top_k, const float* top_p, const float* min_p, int32_t* ids, float* logprobs, void* stream) {
    if (logits_dtype != BITLINEAR_F32 && logits_dtype != BITLINEAR_BF16) return BITLINEAR_ERR_DTYPE;
    if (M < 0 || M > (1 << 24) || V <= 0 || V > BITLINEAR_SAMPLE_MAX_VOCAB || row_stride < V) return BITLINEAR_ERR_SHAPE;
    if (M == 0) return BITLINEAR_OK;
    if (!logits || !u || !ids) return BITLINEAR_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(logits) % (logits_dtype == BITLINEAR_F32 ? 4 : 2)) return BITLINEAR_ERR_ALIGN;
    int sm_count = 0;
    if (const int rc = device_sm_count(&sm_count)) return rc;
    // CTAs per row: two at least (each merges its share of the bins, one per thread), more for long rows
    int ranks = 2;
    while (ranks < kMaxCluster && V > 2048 * ranks) ranks *= 2;
    SampleArgs a = {logits, row_stride, M, V, 0, 0, u, temperature, top_k, top_p, min_p, ids, logprobs};
    a.shard = ((V + ranks - 1) / ranks + 7) / 8 * 8;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!top_k && !top_p && !min_p) {
        const void* kernel = logits_dtype == BITLINEAR_F32 ? reinterpret_cast<const void*>(sample_plain_kernel<float>)
                                                           : reinterpret_cast<const void*>(sample_plain_kernel<__nv_bfloat16>);
        return launch_rows(kernel, a, ranks, kPlainThreads, 0, st);
    }
    const bool alone = (long long)M * ranks <= sm_count;
    if (logits_dtype == BITLINEAR_F32) return alone ? sample_launch<float, 512>(a, ranks, st) : sample_launch<float, 256>(a, ranks, st);
    return alone ? sample_launch<__nv_bfloat16, 512>(a, ranks, st) : sample_launch<__nv_bfloat16, 256>(a, ranks, st);
}
