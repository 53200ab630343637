// The draw of the next token from a row of logits: temperature, top-k, top-p, min-p and one given random number per row.
//
//   w_i = exp((l_i - max l) / T);  keep the top_k largest, of those the shortest run from the largest down whose mass reaches
//   top_p of theirs, of those the ones with w_i >= min_p;  the token is the first in the order of ids whose running sum of
//   kept weights exceeds u times their total.  Equal logits rank by id.
//
// A row is read from memory once: a cluster of CTAs holds it in shared memory, a contiguous part each, and every later
// pass runs there.  No row is sorted.  A threshold (the k-th largest, the end of a mass) is found by histograms, best
// bins first: one over the logits' distance from the largest, linear, so that the elements spread over its bins, and
// three over the bits of an order-preserving integer image within the bin that holds the threshold.
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
constexpr int kBins = 2048;
constexpr int kLinearBins = 1024;
constexpr int kMaxCluster = 8;
constexpr int kMaxShard = 45056;  // floats of a row that one CTA holds
constexpr double kUnit44 = 17592186044416.0;  // 2^44

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

// larger float, larger integer; -inf and below: NaN was turned into -inf
__device__ __forceinline__ uint32_t key_of(float l) {
    const uint32_t b = __float_as_uint(l + 0.0f);  // -0 and 0 are equal
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

struct Crossing {
    int bin;
    uint32_t count_above, count;
    unsigned long long mass_above;
};

struct Shared {
    unsigned long long best;    // (key of the largest, ~index)
    float low;                  // the smallest finite logit of the part
    unsigned long long total;   // kept mass of the part
    uint32_t ties;
    Crossing cross;
    unsigned long long warp_mass[kThreads / 32];
    uint32_t warp_count[kThreads / 32];
    float warp_low[kThreads / 32];
    int cut_index;
    uint32_t count[kBins];
    uint32_t mass[3][kBins];  // sums of the weights' low, middle and high 16 bits: shared memory adds 32-bit integers natively
};

struct Row {
    float top;       // largest logit
    double scale;    // log2(e) / T
    bool top_inf;
};

// exp((l - top) / T); 0 for -inf
__device__ __forceinline__ double weight_of(const Row& r, float l) {
    if (r.top_inf) return l == r.top ? 1.0 : 0.0;
    const double x = ((double)l - (double)r.top) * r.scale;
    return x > -64.0 ? exp2(x) : 0.0;  // NaN (-inf at T = inf) compares false
}
__device__ __forceinline__ unsigned long long fixed_of(double w) { return (unsigned long long)__double2ll_rn(w * kUnit44); }

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
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long begin = (long long)rank * a.shard;
    const int n = (int)max(0ll, min((long long)a.shard, a.V - begin));
    const T* src = static_cast<const T*>(a.logits) + (size_t)row * a.stride + begin;

    // ---- the part into shared memory; the largest and the smallest finite logit
    unsigned long long best = 0;
    float low = INFINITY;
    auto take = [&](int i, float l) {
        l = l == l ? l : -INFINITY;  // NaN: never drawn
        const unsigned long long c = ((unsigned long long)key_of(l) << 32) | (0xffffffffu - (uint32_t)(begin + i));
        best = max(best, c);
        if (l > -INFINITY) low = fminf(low, l);
        return l;
    };
    constexpr int VEC = 16 / sizeof(T);
    const int head = (int)min((long long)n, (long long)(((16 - (reinterpret_cast<uintptr_t>(src) & 15)) & 15) / sizeof(T)));
    const int n_vec = (n - head) / VEC;
    for (int i = tid; i < head; i += kThreads) vals[i] = take(i, load_logit(src + i));
    for (int v = tid; v < n_vec; v += kThreads) {
        const uint4 x = __ldcs(reinterpret_cast<const uint4*>(src + head) + v);
        const T* e = reinterpret_cast<const T*>(&x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int i = head + v * VEC + j;
            vals[i] = take(i, load_logit(e + j));
        }
    }
    for (int i = head + n_vec * VEC + tid; i < n; i += kThreads) vals[i] = take(i, load_logit(src + i));
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        best = max(best, __shfl_xor_sync(0xffffffffu, best, off));
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, off));
    }
    if (lane == 0) sh.warp_mass[warp] = best, sh.warp_low[warp] = low;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kThreads / 32; ++w) best = max(best, sh.warp_mass[w]), low = fminf(low, sh.warp_low[w]);
        sh.best = best;
        sh.low = low;
    }
    cluster.sync();
    for (int r = 0; r < ranks; ++r) {
        const Shared* o = cluster.map_shared_rank(&sh, r);
        best = r == 0 ? o->best : max(best, o->best);
        low = r == 0 ? o->low : fminf(low, o->low);
    }
    const uint32_t top_key = (uint32_t)(best >> 32);
    const int top_index = (int)(0xffffffffu - (uint32_t)best);
    Row rw;
    rw.top = __uint_as_float(top_key ^ ((top_key >> 31) ? 0x80000000u : 0xffffffffu));
    rw.top_inf = rw.top == INFINITY;
    const float temp = a.temperature ? a.temperature[row] : 1.0f;
    const bool empty = rw.top == -INFINITY, greedy = !(temp > 0.0f);
    if (empty || greedy) {  // the same in every CTA of the cluster
        if (rank == 0 && tid == 0) {
            a.ids[row] = empty ? -1 : top_index;
            if (a.logprobs) a.logprobs[row] = empty ? -INFINITY : 0.0f;
        }
        cluster.sync();  // no CTA leaves while another reads its shared memory
        return;
    }
    rw.scale = 1.4426950408889634074 / (double)temp;
    const int k = a.top_k ? a.top_k[row] : 0;
    const float p = a.top_p ? a.top_p[row] : 1.0f;
    const float given_mp = a.min_p ? a.min_p[row] : 0.0f;
    const double mp = given_mp > 0.0f ? fmin((double)given_mp, 1.0) : 0.0;  // the largest, of weight 1, always stays
    const bool use_k = k > 0 && k < a.V, use_p = p < 1.0f;
    const int i0 = min(tid * a.per, n), i1 = min(i0 + a.per, n);

    // kept so far: keys above floor_key, and of those equal to it the ones up to floor_index
    uint32_t floor_key = 0;
    long long floor_index = 0x7fffffffffffffffll;
    auto kept = [&](uint32_t key, int i) { return key > floor_key || (key == floor_key && begin + i <= floor_index); };

    // ---- thresholds
    // linear bins of the first histogram: distances from the largest up to where weights vanish or the logits end
    const float span = fminf(rw.top - low, 40.0f * temp);
    const float to_bin = span > 0.0f ? (float)kLinearBins / span : 0.0f;
    auto linear_bin = [&](float l) {  // monotone: a larger logit never gets a later bin
        const float d = (rw.top - l) * to_bin;
        return d < (float)(kLinearBins - 1) ? (int)d : kLinearBins - 1;  // the last takes the rest, -inf and inf - inf too
    };
    // one histogram over the part's elements that `in` admits, merged over the cluster; the bin in which the running count
    // (or mass) reaches the target
    auto find = [&](int bins, bool by_mass, uint32_t want, double target, uint32_t count0, unsigned long long mass0, auto&& bin_of) {
        for (int b = tid; b < bins; b += kThreads) {
            sh.count[b] = 0;
            if (by_mass) sh.mass[0][b] = sh.mass[1][b] = sh.mass[2][b] = 0;
        }
        __syncthreads();
        for (int i = i0; i < i1; ++i) {
            const float l = vals[i];
            const int b = bin_of(l, key_of(l), i);
            if (b < 0) continue;
            atomicAdd(&sh.count[b], 1u);
            if (by_mass) {
                const unsigned long long w = fixed_of(weight_of(rw, l));
                if (w & 0xffffu) atomicAdd(&sh.mass[0][b], (uint32_t)(w & 0xffffu));
                if ((w >> 16) & 0xffffu) atomicAdd(&sh.mass[1][b], (uint32_t)((w >> 16) & 0xffffu));
                if (w >> 32) atomicAdd(&sh.mass[2][b], (uint32_t)(w >> 32));
            }
        }
        cluster.sync();
        const int per = bins / kThreads;  // 2 or 4 neighbouring bins
        uint32_t c[4] = {0, 0, 0, 0};
        unsigned long long m[4] = {0, 0, 0, 0};
        for (int r = 0; r < ranks; ++r) {
            const Shared* o = cluster.map_shared_rank(&sh, r);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j >= per) break;
                const int b = tid * per + j;
                c[j] += o->count[b];
                if (by_mass) m[j] += o->mass[0][b] + ((unsigned long long)o->mass[1][b] << 16) + ((unsigned long long)o->mass[2][b] << 32);
            }
        }
        uint32_t cs = c[0] + c[1] + c[2] + c[3], ci = cs;
        unsigned long long ms = m[0] + m[1] + m[2] + m[3], mi = ms;
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
        for (int w = 0; w < warp; ++w) ca += sh.warp_count[w], ma += sh.warp_mass[w];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool here = by_mass ? (double)ma < target && (double)(ma + m[j]) >= target : ca < want && ca + c[j] >= want;
            if (here && c[j] > 0) sh.cross = {tid * per + j, ca, c[j], ma};
            ca += c[j];
            ma += m[j];
        }
        cluster.sync();  // the crossing is known, and nobody reads another's bins any more
        return sh.cross;
    };
    // threshold over the kept elements: the key that ends the run, how many of it belong to the run, how many there are
    auto threshold = [&](bool by_mass, uint32_t want, double target, uint32_t& key_out, uint32_t& keep, uint32_t& there) {
        Crossing x = find(kLinearBins, by_mass, want, target, 0, 0, [&](float l, uint32_t key, int i) { return kept(key, i) ? linear_bin(l) : -1; });
        const int bin0 = x.bin;
        uint32_t prefix = 0;
        for (int level = 0; level < 3; ++level) {
            const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
            const uint32_t above_mask = level == 0 ? 0u : level == 1 ? 0xffe00000u : 0xfffffc00u;
            x = find(1 << bits, by_mass, want, target, x.count_above, x.mass_above, [&](float l, uint32_t key, int i) {
                if (!kept(key, i) || (key & above_mask) != prefix || linear_bin(l) != bin0) return -1;
                return (1 << bits) - 1 - (int)((key >> shift) & ((1u << bits) - 1u));
            });
            prefix |= (uint32_t)((1 << bits) - 1 - x.bin) << shift;
        }
        key_out = prefix;
        there = x.count;
        if (by_mass) {
            const float l = __uint_as_float(prefix ^ ((prefix >> 31) ? 0x80000000u : 0xffffffffu));
            const double each = (double)fixed_of(weight_of(rw, l));
            const double need = ceil((target - (double)x.mass_above) / fmax(each, 1.0));
            keep = need < 1.0 ? 1u : need > (double)there ? there : (uint32_t)need;
        } else {
            keep = want - x.count_above;
        }
    };
    // of the elements equal to floor_key the first `keep` by id stay: the id of the last of them
    auto cut_ties = [&](uint32_t keep, uint32_t there) {
        if (keep >= there) return;
        uint32_t mine = 0;
        for (int i = i0; i < i1; ++i) mine += key_of(vals[i]) == floor_key && begin + i <= floor_index;
        uint32_t incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += up;
        }
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
            for (int i = i0; i < i1; ++i)
                if (key_of(vals[i]) == floor_key && begin + i <= floor_index && --left == 0) {
                    sh.cut_index = (int)(begin + i);
                    break;
                }
        }
        cluster.sync();
        int cut = -1;
        for (int r = 0; r < ranks; ++r) cut = max(cut, cluster.map_shared_rank(&sh, r)->cut_index);
        floor_index = cut;
        cluster.sync();  // before the shared fields are written again
    };
    // mass of what is kept, over the cluster; `mine`: this thread's run, `before_cta`: the parts in front of this one
    auto kept_mass = [&](double least, unsigned long long& mine, unsigned long long& before, unsigned long long& before_cta) {
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
        if (lane == 31) sh.warp_mass[warp] = incl;
        __syncthreads();
        before = incl - mine;
        for (int w = 0; w < warp; ++w) before += sh.warp_mass[w];
        if (tid == kThreads - 1) sh.total = before + mine;
        cluster.sync();
        unsigned long long all = 0;
        before_cta = 0;
        for (int r = 0; r < ranks; ++r) {
            const unsigned long long t = cluster.map_shared_rank(&sh, r)->total;
            if (r < rank) before_cta += t;
            all += t;
        }
        return all;
    };

    unsigned long long mine, before, before_cta;
    if (use_k) {
        uint32_t key, keep, there;
        threshold(false, (uint32_t)k, 0.0, key, keep, there);
        floor_key = key;
        cut_ties(keep, there);
    }
    if (use_p) {
        const unsigned long long all = kept_mass(0.0, mine, before, before_cta);
        cluster.sync();  // totals are read before they are written again
        const double target = fmax((double)p * (double)all, 0.5);
        uint32_t key, keep, there;
        threshold(true, 0, target, key, keep, there);
        if (key != floor_key) floor_key = key, floor_index = 0x7fffffffffffffffll;  // top_k's cut was among another key's ties
        cut_ties(keep, there);
    }
    const unsigned long long all = kept_mass(mp, mine, before, before_cta);
    const float u = a.u[row];
    const double goal = u > 0.0f ? (double)u * (double)all : 0.0;
    unsigned long long at = (unsigned long long)goal;  // running sum > goal, in integers: > its floor
    if (at >= all) at = all - 1;                       // u = 1: the last token that is kept
    before += before_cta;
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
                    a.ids[row] = (int)(begin + i);
                    if (a.logprobs) a.logprobs[row] = (float)log(w * kUnit44 / (double)all);
                }
                break;
            }
            run += __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    cluster.sync();
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
