// Block tables and slot maps of a paged cache, built on the GPU from the requests' lengths.
//
// Three running sums over the requests decide everything: blocks needed, tokens to place, blocks given back.  The free
// blocks are a stack; finished requests push theirs in the order of the requests, and the k-th block that this step
// needs is the k-th from the top.  Every CTA forms the three sums over all requests itself (a few kilobytes from L2),
// which costs less than a second launch or a grid barrier; then it fills its share of the token arrays, four tokens per
// thread and 16 bytes per store.  A small step is one CTA and bound by its chain of dependent loads (16 requests: 5.7 us,
// launch included), a large one by the same chain and the bytes it writes (4096 requests, a million slots: 12.6 us, 1.4 TB/s).
//
// Nothing is read that another CTA writes: new table entries lie behind the ones that are looked up, blocks given back are
// stored above the old top of the stack and taken from the tables where this step hands them out again, and lengths
// and the stack's height are written by a second launch where they are updated in place by more than one CTA.
#include "common.cuh"

#include <algorithm>

namespace bitlinear {

namespace {

struct TablesArgs {
    const int* lengths;
    const int* new_tokens;
    int* tables;
    int* free_blocks;
    const int* n_free;
    int R, max_blocks, block_rows, n_blocks, t_cap;
    int* lengths_out;
    int* n_free_out;
    int* served;
    int* cu_tokens;
    int* seq_ids;
    int* positions;
    int* row_lengths;
    int* slots;
};

// what one request asks for; a length outside the table row counts as the nearest one inside
struct Ask {
    int len, used, n, need, back, fresh;  // fresh: new_tokens as given
};
// blocks that n rows take; n + rows - 1 may pass 2^31, not 2^32
__device__ __forceinline__ int blocks_of(int n, int rows) { return (int)(((unsigned)n + (unsigned)rows - 1u) / (unsigned)rows); }
__device__ __forceinline__ Ask ask_of(const TablesArgs& a, int r) {
    const int cap = a.max_blocks * a.block_rows;
    Ask k;
    k.fresh = a.new_tokens[r];
    k.len = min(max(a.lengths[r], 0), cap);
    k.used = blocks_of(k.len, a.block_rows);
    const bool adds = k.fresh > 0 && k.fresh <= cap - k.len;
    k.n = adds ? k.fresh : 0;
    k.need = adds ? blocks_of(k.len + k.n, a.block_rows) - k.used : 0;
    k.back = k.fresh < 0 ? k.used : 0;
    return k;
}

struct Sums {
    long long n;
    int need, back;
};
__device__ __forceinline__ Sums operator+(const Sums& x, const Sums& y) { return {x.n + y.n, x.need + y.need, x.back + y.back}; }
__device__ __forceinline__ Sums shfl_up(const Sums& x, int d) {
    return {__shfl_up_sync(0xffffffffu, x.n, d), __shfl_up_sync(0xffffffffu, x.need, d), __shfl_up_sync(0xffffffffu, x.back, d)};
}

constexpr int kTablesThreads = 1024;

// the largest c in 0 .. n-1 with v[c] <= x (v ascending, v[0] <= x)
template <class T>
__device__ __forceinline__ int chunk_of(const T* v, int n, T x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (v[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// commit: lengths and n_free may be written here (one CTA, or outputs of their own)
__global__ void __launch_bounds__(kTablesThreads) block_tables_kernel(const TablesArgs a, int commit) {
    __shared__ long long cum_n[kTablesThreads];  // sums over the requests before a thread's chunk
    __shared__ int cum_need[kTablesThreads], cum_back[kTablesThreads];
    __shared__ Sums warp_sum[33];
    __shared__ int cut_s;           // the first request that does not fit: none behind it is served
    __shared__ long long cut_n;     // tokens and blocks of the requests before it
    __shared__ int cut_need;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
    const int per = blocks_of(a.R, threads);  // requests per chunk
    const long long first = (long long)tid * per;
    const int r0 = (int)min(first, (long long)a.R), r1 = (int)min(first + per, (long long)a.R);
    const int n_free = min(max(*a.n_free, 0), a.n_blocks);
    if (tid == 0) cut_s = a.R;
    Sums mine = {0, 0, 0};
    for (int r = r0; r < r1; ++r) {
        const Ask k = ask_of(a, r);
        mine = mine + Sums{k.n, k.need, k.back};
    }
    Sums incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const Sums up = shfl_up(incl, d);
        if (lane >= d) incl = incl + up;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        const Sums own = lane < warps ? warp_sum[lane] : Sums{0, 0, 0};
        Sums w = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const Sums up = shfl_up(w, d);
            if (lane >= d) w = w + up;
        }
        if (lane < warps) warp_sum[lane] = {w.n - own.n, w.need - own.need, w.back - own.back};
        if (lane == 31) warp_sum[32] = w;
    }
    __syncthreads();
    const Sums before = {warp_sum[warp].n + incl.n - mine.n, warp_sum[warp].need + incl.need - mine.need, warp_sum[warp].back + incl.back - mine.back};
    const Sums all = warp_sum[32];
    cum_n[tid] = before.n;
    cum_need[tid] = before.need;
    cum_back[tid] = before.back;
    const long long have = (long long)n_free + all.back;
    // the sums only grow, so the requests served are those before the first one that does not fit
    if (all.n > a.t_cap || all.need > have) {
        if (before.n + mine.n > a.t_cap || before.need + mine.need > have) {
            Sums s = before;
            for (int r = r0; r < r1; ++r) {
                const Ask k = ask_of(a, r);
                if (k.n > 0 && (s.n + k.n > a.t_cap || (long long)s.need + k.need > have)) {
                    atomicMin(&cut_s, r);
                    break;
                }
                s = s + Sums{k.n, k.need, k.back};
            }
        }
        __syncthreads();
        if (cut_s >= r0 && cut_s < r1) {
            Sums s = before;
            for (int r = r0; r < cut_s; ++r) {
                const Ask k = ask_of(a, r);
                s = s + Sums{k.n, k.need, k.back};
            }
            cut_n = s.n;
            cut_need = s.need;
        }
    } else if (tid == 0) {
        cut_n = all.n;
        cut_need = all.need;
    }
    __syncthreads();
    const int cut = cut_s;
    const long long live = cut_n;
    const int taken = cut_need;

    // block k (in the order in which they are handed out) comes off the top of the stack
    auto given_back = [&](int j) {  // block j of those given back in this step
        const int c = chunk_of(cum_back, threads, j);
        int left = j - cum_back[c];
        for (int r = c * per;; ++r) {
            const Ask k = ask_of(a, r);
            if (left < k.back) return a.tables[(long long)r * a.max_blocks + left];
            left -= k.back;
        }
    };
    auto block_at = [&](int k) {
        const long long place = have - 1 - k;
        return place < n_free ? a.free_blocks[place] : given_back((int)(place - n_free));
    };

    // tokens, four per thread
    const int stride = gridDim.x * threads;
    for (long long t0 = 4ll * (blockIdx.x * threads + tid); t0 < a.t_cap; t0 += 4ll * stride) {
        int4 seq = make_int4(-1, -1, -1, -1), pos = seq, slot = seq, len = make_int4(0, 0, 0, 0);
        if (t0 < live) {
            const int c = chunk_of(cum_n, threads, t0);
            int r = c * per;
            long long base = cum_n[c];  // tokens before request r
            int need0 = cum_need[c];    // blocks before it
            Ask k = ask_of(a, r);
            int block = -1, block_index = -1, owner = -1;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const long long t = t0 + e;
                if (t < live) {
                    while (t >= base + k.n) {
                        base += k.n;
                        need0 += k.need;
                        k = ask_of(a, ++r);
                    }
                    const int p = k.len + (int)(t - base), b = p / a.block_rows;
                    if (b != block_index || r != owner) {
                        block_index = b, owner = r;
                        int* entry = a.tables + (long long)r * a.max_blocks + b;
                        if (b < k.used) block = *entry;
                        else {
                            block = block_at(need0 + b - k.used);
                            if (p == b * a.block_rows) *entry = block;
                        }
                    }
                    (&seq.x)[e] = r;
                    (&pos.x)[e] = p;
                    (&len.x)[e] = p + 1;
                    (&slot.x)[e] = block >= 0 && block < a.n_blocks ? block * a.block_rows + (p - b * a.block_rows) : -1;
                }
            }
        }
        if (t0 + 4 <= a.t_cap) {
            *reinterpret_cast<int4*>(a.seq_ids + t0) = seq;
            *reinterpret_cast<int4*>(a.positions + t0) = pos;
            *reinterpret_cast<int4*>(a.row_lengths + t0) = len;
            *reinterpret_cast<int4*>(a.slots + t0) = slot;
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e) {
                if (t0 + e >= a.t_cap) break;
                a.seq_ids[t0 + e] = (&seq.x)[e];
                a.positions[t0 + e] = (&pos.x)[e];
                a.row_lengths[t0 + e] = (&len.x)[e];
                a.slots[t0 + e] = (&slot.x)[e];
            }
        }
    }
    // blocks given back go above the old top
    for (long long j = blockIdx.x * threads + tid; j < all.back && n_free + j < a.n_blocks; j += stride) a.free_blocks[n_free + j] = given_back((int)j);
    if (gridDim.x == 1) __syncthreads();  // lengths may be updated in place: every thread has read them
    // requests: chunk c belongs to CTA c % grid
    if (tid % gridDim.x == blockIdx.x) {
        long long s = before.n;
        for (int r = r0; r < r1; ++r) {
            const Ask k = ask_of(a, r);
            const bool ok = k.fresh <= 0 || (k.n > 0 && r < cut);
            if (r < cut) s += k.n;
            a.served[r] = ok;
            a.cu_tokens[r + 1] = (int)min(s, live);
            if (commit) a.lengths_out[r] = k.fresh < 0 ? 0 : k.len + (ok ? k.n : 0);
        }
    }
    if (blockIdx.x == 0 && tid == 0) {
        a.cu_tokens[0] = 0;
        if (commit) *a.n_free_out = (int)min(have - taken, (long long)a.n_blocks);
    }
}

// lengths and the stack's height updated in place after a launch of several CTAs
__global__ void __launch_bounds__(kTablesThreads) block_tables_commit_kernel(const TablesArgs a) {
    __shared__ int delta;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (threadIdx.x == 0) delta = 0;
    __syncthreads();
    int d = 0;
    for (long long i = threadIdx.x; i < a.R; i += blockDim.x) {
        const int r = (int)i;
        const Ask k = ask_of(a, r);
        const bool ok = a.served[r] != 0;
        d += k.back - (ok ? k.need : 0);
        a.lengths_out[r] = k.fresh < 0 ? 0 : k.len + (ok ? k.n : 0);
    }
    atomicAdd(&delta, d);
    __syncthreads();
    if (threadIdx.x == 0) *a.n_free_out = min(min(max(*a.n_free, 0), a.n_blocks) + delta, a.n_blocks);
}

}  // namespace

}  // namespace bitlinear

using namespace bitlinear;

extern "C" int bitlinear_block_tables(const int32_t* lengths, const int32_t* new_tokens, int n_requests, int32_t* tables, int max_blocks,
                                      int32_t* free_blocks, const int32_t* n_free, int n_blocks, int block_rows, int t_cap,
                                      int32_t* lengths_out, int32_t* n_free_out, int32_t* served, int32_t* cu_tokens, int32_t* seq_ids,
                                      int32_t* positions, int32_t* row_lengths, int32_t* slots, void* stream) {
    constexpr long long kMost = 0x7fffffff;
    if (n_requests < 0 || max_blocks <= 0 || n_blocks <= 0 || block_rows <= 0 || t_cap < 0 || (long long)max_blocks * block_rows > kMost ||
        (long long)n_blocks * block_rows > kMost || (long long)n_requests * max_blocks > kMost)
        return BITLINEAR_ERR_SHAPE;
    if (!n_free || !n_free_out || !free_blocks || !cu_tokens || (n_requests > 0 && (!lengths || !new_tokens || !tables || !lengths_out || !served)) ||
        (t_cap > 0 && (!seq_ids || !positions || !row_lengths || !slots)))
        return BITLINEAR_ERR_NULL;
    if (!aligned16(seq_ids) || !aligned16(positions) || !aligned16(row_lengths) || !aligned16(slots)) return BITLINEAR_ERR_ALIGN;
    auto apart = [](const int32_t* x, const int32_t* y, size_t n) { return x == y || x + n <= y || y + n <= x; };
    if (!apart(lengths, lengths_out, n_requests)) return BITLINEAR_ERR_SHAPE;
    int sm_count = 0;
    if (const int rc = device_sm_count(&sm_count)) return rc;
    const TablesArgs a = {lengths, new_tokens, tables, free_blocks, n_free, n_requests, max_blocks, block_rows, n_blocks, t_cap,
                          lengths_out, n_free_out, served, cu_tokens, seq_ids, positions, row_lengths, slots};
    // threads: enough for a request or four tokens each; more than one CTA once the tokens fill one
    const int wanted = std::max(n_requests, (int)((t_cap + 3ll) / 4));
    const int threads = wanted <= 128 ? 128 : wanted <= 512 ? 512 : kTablesThreads;
    const int ctas = std::max(1, (int)std::min<long long>(sm_count, (t_cap + 4ll * threads - 1) / (4 * threads)));
    const bool in_place = lengths_out == lengths || n_free_out == n_free;
    const int commit = ctas == 1 || !in_place;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, block_tables_kernel, a, commit) != cudaSuccess) {
        cudaGetLastError();
        return BITLINEAR_ERR_CUDA;
    }
    if (!commit) {
        cfg.gridDim = dim3(1);
        cfg.blockDim = dim3(kTablesThreads);
        if (cudaLaunchKernelEx(&cfg, block_tables_commit_kernel, a) != cudaSuccess) {
            cudaGetLastError();
            return BITLINEAR_ERR_CUDA;
        }
    }
    return BITLINEAR_OK;
}
