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
// Which token comes out hangs on sums next to a border, so weights are formed in fp64 and summed as integers in units of
// 2^-44: sums of any order are the same, and no two machines' rounding of a sum decides a token.
#include "common.cuh"

#include <cooperative_groups.h>

#include <algorithm>
#include <mutex>

namespace cg = cooperative_groups;

namespace bitlinear {

namespace {

constexpr int kThreads = 512;
constexpr int kBins = 1024;  // two per thread
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

struct Shared {
    double pow2[64];            // 2^(j / 64)
    float top, low;             // largest logit of the part, smallest finite one
    int first;                  // lowest id of the largest logit in the part
    uint32_t ties;
    unsigned long long total;   // kept mass of the part
    Crossing cross;
    unsigned long long warp_mass[kThreads / 32];
    uint32_t warp_count[kThreads / 32];
    float warp_top[kThreads / 32], warp_low[kThreads / 32];
    int cut_index;
    __align__(16) uint32_t count[kBins];
    __align__(16) uint32_t mass[3][kBins];  // sums of the weights' low, middle and high 16 bits: shared memory adds 32-bit integers natively
};

struct Row {
    float top;        // largest logit
    double top_d;
    double scale;     // 64 log2(e) / T
    bool top_inf;
    const double* pow2;
};

// exp((l - top) / T), by 2^(n / 64) from the table and the series of exp to its fourth power on what is left (at most ln 2 / 128:
// the next term is below 2^-44); 0 for -inf
__device__ __forceinline__ double weight_of(const Row& r, float l) {
    if (r.top_inf) return l == r.top ? 1.0 : 0.0;
    // fp32 -> fp64 by hand (conversions run at a quarter of the rate of the rest): right but for denormals, which come out
    // below 2^-126 as well
    const uint32_t b = __float_as_uint(l);
    const double d = __hiloint2double((int)((b & 0x80000000u) | (((b & 0x7fffffffu) >> 3) + 0x38000000u)), (int)(b << 29)) - r.top_d;
    double x = d * r.scale;
    if (!(x > -64.0 * 48) || l == -INFINITY) return 0.0;
    constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52
    const double t = x + kRound;
    const int n = __double2loint(t);
    x = (x - (t - kRound)) * 0.010830424696249145;  // ln 2 / 64
    double e = fma(x, 1.0 / 24.0, 1.0 / 6.0);
    e = fma(x, e, 0.5);
    e = fma(x, e, 1.0);
    e = fma(x, e, 1.0) * r.pow2[n & 63];
    return __hiloint2double(__double2hiint(e) + ((n >> 6) << 20), __double2loint(e));
}
// in units of 2^-44, rounded to nearest: the bits behind 256
__device__ __forceinline__ unsigned long long fixed_of(double w) { return (unsigned long long)__double_as_longlong(w + 256.0) & 0xfffffffffffffull; }

template <class T>
__device__ __forceinline__ float load_logit(const T* p);
template <>
__device__ __forceinline__ float load_logit<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float load_logit<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }

template <class T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleArgs a) {
    extern __shared__ __align__(16) uint8_t sample_raw[];
    Shared& sh = *reinterpret_cast<Shared*>(sample_raw);
    float* vals = reinterpret_cast<float*>(sample_raw + (sizeof(Shared) + 15) / 16 * 16);
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = blockIdx.x / ranks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid < 64) sh.pow2[tid] = exp2((double)tid / 64.0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long begin = (long long)rank * a.shard;
    const int n = (int)max(0ll, min((long long)a.shard, a.V - begin));
    const T* src = static_cast<const T*>(a.logits) + (size_t)row * a.stride + begin;
    const float temp = a.temperature ? a.temperature[row] : 1.0f;
    const int k = a.top_k ? a.top_k[row] : 0;
    const float p = a.top_p ? a.top_p[row] : 1.0f;
    const float given_mp = a.min_p ? a.min_p[row] : 0.0f;
    const float u = a.u[row];

    // ---- the part into shared memory; the largest and the smallest finite logit
    float top = -INFINITY, low = INFINITY;
    auto take = [&](float l) {
        l = l == l ? l : -INFINITY;  // NaN: never drawn
        top = fmaxf(top, l);
        low = fminf(low, l > -INFINITY ? l : INFINITY);
        return l;
    };
    constexpr int VEC = 16 / sizeof(T), AHEAD = 4;
    const int head = (int)min((long long)n, (long long)(((16 - (reinterpret_cast<uintptr_t>(src) & 15)) & 15) / sizeof(T)));
    const int n_vec = (n - head) / VEC;
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
            float* dst = vals + head + (v0 + j * kThreads) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i) dst[i] = take(load_logit(e + i));
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
    if (tid == 0) {
        for (int w = 1; w < kThreads / 32; ++w) top = fmaxf(top, sh.warp_top[w]), low = fminf(low, sh.warp_low[w]);
        sh.top = top;
        sh.low = low;
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
    const Row rw = {top, (double)top, 64.0 * 1.4426950408889634074 / (double)temp, top == INFINITY, sh.pow2};
    const uint32_t top_key = key_of(top);
    const double mp = given_mp > 0.0f ? fmin((double)given_mp, 1.0) : 0.0;  // the largest, of weight 1, always stays
    const bool use_k = k > 0 && k < a.V, use_p = p < 1.0f;

    // kept so far: keys above floor_key, and of those equal to it the ones up to floor_index
    uint32_t floor_key = 0;
    int floor_index = 0x7fffffff;
    auto kept = [&](uint32_t key, int i) { return key > floor_key || (key == floor_key && (int)begin + i <= floor_index); };

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
            const uint32_t step = (hi - lo) / 32 + 1;
            const unsigned long long at = (unsigned long long)lo + (unsigned long long)lane * step;
            const bool good = at >= hi || linear_bin(float_of((uint32_t)at)) <= bin;
            const unsigned m = __ballot_sync(0xffffffffu, good);
            if (m == 0) lo = lo + 31 * step + 1;
            else {
                const uint32_t f = (uint32_t)__ffs((int)m) - 1;
                hi = (uint32_t)min((unsigned long long)hi, (unsigned long long)lo + (unsigned long long)f * step);
                if (f > 0) lo = lo + (f - 1) * step + 1;
            }
        }
        return hi;
    };
    // one histogram over the part's elements to which bin_of gives a bin, merged over the cluster; the bin in which the running
    // count (or mass) reaches the target
    auto find = [&](bool by_mass, uint32_t want, double target, uint32_t count0, unsigned long long mass0, auto&& bin_of) {
        settle();
        const uint2 none = make_uint2(0u, 0u);
        reinterpret_cast<uint2*>(sh.count)[tid] = none;
        if (by_mass) {
#pragma unroll
            for (int j = 0; j < 3; ++j) reinterpret_cast<uint2*>(sh.mass[j])[tid] = none;
        }
        __syncthreads();
        for (int i = i0; i < i1; ++i) {
            const float l = vals[i];
            const uint32_t key = key_of(l);
            if (!kept(key, i)) continue;
            const int b = bin_of(l, key);
            if (b < 0) continue;
            atomicAdd(&sh.count[b], 1u);
            if (by_mass) {
                const unsigned long long w = fixed_of(weight_of(rw, l));
                const uint32_t w0 = (uint32_t)w & 0xffffu, w1 = (uint32_t)w >> 16, w2 = (uint32_t)(w >> 32);
                if (w0) atomicAdd(&sh.mass[0][b], w0);
                if (w1) atomicAdd(&sh.mass[1][b], w1);
                if (w2) atomicAdd(&sh.mass[2][b], w2);
            }
        }
        cluster.sync();
        uint32_t c[2] = {0, 0};
        unsigned long long m[2] = {0, 0};
        {
            uint2 x[kMaxCluster];
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r) x[r] = r < ranks ? reinterpret_cast<const uint2*>(cluster.map_shared_rank(&sh, r)->count)[tid] : none;
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r) c[0] += x[r].x, c[1] += x[r].y;
            if (by_mass) {
#pragma unroll
                for (int j = 0; j < 3; ++j) {
#pragma unroll
                    for (int r = 0; r < kMaxCluster; ++r) x[r] = r < ranks ? reinterpret_cast<const uint2*>(cluster.map_shared_rank(&sh, r)->mass[j])[tid] : none;
#pragma unroll
                    for (int r = 0; r < kMaxCluster; ++r) m[0] += (unsigned long long)x[r].x << (16 * j), m[1] += (unsigned long long)x[r].y << (16 * j);
                }
            }
        }
        read_done();
        const uint32_t cs = c[0] + c[1];
        const unsigned long long ms = m[0] + m[1];
        uint32_t ci = cs;
        unsigned long long mi = ms;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t cu = __shfl_up_sync(0xffffffffu, ci, d);
            const unsigned long long mu = __shfl_up_sync(0xffffffffu, mi, d);
            if (lane >= d) ci += cu, mi += mu;
        }
        if (lane == 31) sh.warp_count[warp] = ci, sh.warp_mass[warp] = mi;
        __syncthreads();
        uint32_t ca = count0 + ci - cs;
        unsigned long long ma = mass0 + mi - ms;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w)
            if (w < warp) ca += sh.warp_count[w], ma += sh.warp_mass[w];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bool here = by_mass ? (double)ma < target && (double)(ma + m[j]) >= target : ca < want && ca + c[j] >= want;
            if (here && c[j] > 0) sh.cross = {2 * tid + j, ca, c[j], ma};
            ca += c[j];
            ma += m[j];
        }
        __syncthreads();
        return sh.cross;
    };
    // of the elements equal to floor_key the first `keep` by id stay: the id of the last of them
    auto cut_ties = [&](uint32_t keep) {
        settle();
        uint32_t mine = 0;
        for (int i = i0; i < i1; ++i) {
            const uint32_t key = key_of(vals[i]);
            mine += key == floor_key && kept(key, i);
        }
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
            for (int i = i0; i < i1; ++i) {
                const uint32_t key = key_of(vals[i]);
                if (key == floor_key && kept(key, i) && --left == 0) {
                    sh.cut_index = (int)begin + i;
                    break;
                }
            }
        }
        cluster.sync();
        int cut = -1;
        for (int r = 0; r < ranks; ++r) cut = max(cut, cluster.map_shared_rank(&sh, r)->cut_index);
        floor_index = cut;
        read_done();
    };
    // Narrows what is kept to the run from the largest down that reaches the target.  The bin that holds the run's end
    // is split until the run takes all of it or it is a single key, whose elements then go by id.
    auto narrow = [&](bool by_mass, uint32_t want, double target) {
        Crossing x = find(by_mass, want, target, 0, 0, [&](float l, uint32_t) { return linear_bin(l); });
        uint32_t lo = first_key(x.bin), hi = (x.bin == 0 ? top_key + 1 : first_key(x.bin - 1)) - 1;
        while (x.count > 1 && lo < hi && (by_mass || x.count_above + x.count != want)) {
            const int shift = max(0, 32 - __clz((int)(hi - lo)) - 10);
            const uint32_t from = hi, to = lo;
            x = find(by_mass, want, target, x.count_above, x.mass_above, [&](float, uint32_t key) { return key >= to && key <= from ? (int)((from - key) >> shift) : -1; });
            hi = from - ((uint32_t)x.bin << shift);
            lo = hi - to >= (1u << shift) ? hi - ((1u << shift) - 1u) : to;
        }
        uint32_t keep = x.count;
        if (by_mass && x.count > 1) {
            const double each = (double)fixed_of(weight_of(rw, float_of(lo))), need = ceil((target - (double)x.mass_above) / fmax(each, 1.0));
            keep = need < 1.0 ? 1u : need > (double)x.count ? x.count : (uint32_t)need;
        } else if (!by_mass) {
            keep = want - x.count_above;
        }
        if (lo > floor_key) floor_key = lo, floor_index = 0x7fffffff;  // an earlier cut was among another key's ties
        if (keep < x.count) cut_ties(keep);
    };
    // mass of what is kept and weighs at least `least`, over the cluster; `mine`: this thread's run, `before`: what lies in front of it
    auto kept_mass = [&](double least, unsigned long long& mine, unsigned long long& before) {
        settle();
        mine = 0;
        for (int i = i0; i < i1; ++i) {
            const float l = vals[i];
            if (!kept(key_of(l), i)) continue;
            const double w = weight_of(rw, l);
            if (w >= least) mine += fixed_of(w);
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
    if (use_k) narrow(false, (uint32_t)k, 0.0);
    if (use_p) {
        const unsigned long long all = kept_mass(0.0, mine, before);
        narrow(true, 0, fmax((double)p * (double)all, 0.5));
    }
    const unsigned long long all = kept_mass(mp, mine, before);
    const double goal = u > 0.0f ? (double)u * (double)all : 0.0;
    unsigned long long at = goal < 9.2e18 ? (unsigned long long)goal : all;  // running sum > goal, in integers: > its floor
    if (at >= all) at = all - 1;                                             // u = 1: the last token that is kept
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
                if (w >= mp) f = fixed_of(w);
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

template <class T>
int sample_launch(SampleArgs a, int ranks, cudaStream_t st) {
    static std::mutex mu;
    static bool done[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return BITLINEAR_ERR_CUDA;
    }
    constexpr size_t fixed = (sizeof(Shared) + 15) / 16 * 16;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!done[dev]) {
            if (cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(fixed + kMaxShard * sizeof(float))) != cudaSuccess) {
                cudaGetLastError();
                return BITLINEAR_ERR_CUDA;
            }
            done[dev] = true;
        }
    }
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.M * ranks));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = fixed + (size_t)a.shard * sizeof(float);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, sample_kernel<T>, a) != cudaSuccess) {
        cudaGetLastError();
        return BITLINEAR_ERR_CUDA;
    }
    return BITLINEAR_OK;
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
    int ranks = 1;
    while (ranks < kMaxCluster && V > 2048 * ranks) ranks *= 2;
    SampleArgs a = {logits, row_stride, M, V, 0, 0, u, temperature, top_k, top_p, min_p, ids, logprobs};
    a.shard = ((V + ranks - 1) / ranks + 7) / 8 * 8;
    a.per = (a.shard + kThreads - 1) / kThreads | 1;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return logits_dtype == BITLINEAR_F32 ? sample_launch<float>(a, ranks, st) : sample_launch<__nv_bfloat16>(a, ranks, st);
}
