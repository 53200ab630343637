// Attention of many rows over an 8-bit paged cache where groups of rows share their first cache rows: answers to one prompt, or the tokens of a
// prompt's chunk, each of which sees those in front of it.  A group's shared rows are read and multiplied once for all of its rows.
//
//   out[m] = sum_t exp(s_t - max s) v_t / sum_t exp(s_t - max s),  s_t = q[m] . k_t / sqrt(D),  over the rows 0 .. lengths[m] - 1
//
// The query rows of a group and KV head - a row of the call is n_q / n_kv of them - are the 128 rows of a tensor-core tile, 128 cache rows the other side:
// S = Q K^T and O += P V by tcgen05.mma (f16 operands, fp32 accumulators in tensor memory).  Codes arrive by tensor-map copies and become f16 in shared
// memory, which is exact; their scales go onto the scores and the softmax weights in fp32.  Queries are f16 times a power of two per row, exact too.
//
// A CTA runs two streams of such tiles, each with a Q tile, a score tile, an accumulator and four softmax warps of its own.  A stream works in half steps of 64
// cache rows: while the softmax is at one half's scores, the products of the other half - its weights with the values, then the next step's scores in their
// place - run, so neither waits for the other.  Where a group has more than 128 query rows, the streams take two tiles of them over the same
// cache rows (which are then converted once); else they take different cache rows.  What a row does not share is work of the same kind, with the few
// query rows of that row alone.  All of it is cut into equal runs, one per CTA, whatever the lengths; parts of a row meet in a last launch.
//
//   warp 0      the queries of rows' own tiles, ahead of the softmax
//   warps 1, 2  one thread of each issues a stream's products
//   warp 3      copies: block tables -> tensor-map copies of code tiles, and the work list that the other warps follow (not on the scheduler of the softmax warps that
//               have the first rows: where a tile has few query rows they have all the work)
//   warps 4-11  softmax, one thread per query row; four warps per stream
//   warps 12-19 codes -> f16, four warps to a tile
//
// Bound by its instruction caches: five warps of different roles to a scheduler, and two of them at any time wait for instructions.  So loops stay loops wherever a round
// of them hides its own latency, and one loop does for whole and for partial tiles (conversion unrolled by four, once for either: ragged groups 86 -> 84 us, 64 answers over
// 32,768 shared rows 100 -> 95).  A half step of 64 cache rows takes 3000 to 3500 cycles, of which the tensor cores need 1280: 64 answers over 32,768 rows 95 us (floor 13),
// two chunks of 900 .. 1100 tokens behind 3000 .. 6000 223 us (71), 530 Tflop/s.
#include <cuda.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <mutex>

#include "common.cuh"
#include "kv8.cuh"
#include "sm100_sync.cuh"
#include "tensor_map.cuh"

namespace bitlinear {

namespace {

constexpr int kTile = 128;         // query rows and cache rows of a product
constexpr int kPlanThreads = 1024;
constexpr int kFewGroups = 1024;
constexpr int kPlanRows = 4;  // a thread and round
constexpr int kThreads = 640;
constexpr int kHalf = 64;            // columns of a half step
constexpr int kSoftmaxRegs = 144, kOtherRegs = 64;  // a thread, of eight and of twelve warps
constexpr int kSharedCtas = 160;   // parts are reserved for this many
constexpr int kDescs = 4;
constexpr float kWeightScale = 128.0f;  // weights of up to 2^8 (the maximum is followed lazily) stay below f16's largest

// Workspace.  A part: fp32 values of its query rows, then (max, sum) of each.
struct SharedLayout {
    size_t rows, pairs, cum_pairs, cum_rows, starts, pair_rows, item_ctas, totals, parts_w, parts_s, total;
    int max_pairs;
};
struct SharedArgs {
    const __nv_bfloat16* q;
    const float* k_scale;
    const float* v_scale;
    const int* tables;
    const int* lengths;
    const int* seq_ids;
    const int* group_starts;
    const int* shared_rows;
    int M, n_groups, n_q, n_kv, group, n_seq, max_blocks, log2_rows, n_blocks;
    float scale_log2;  // log2(e) / sqrt(D)
    __nv_bfloat16* out;
    int4* rows;       // of each row: cache rows it shares, its length, its group's first pair (-1: none), that group's first query row
    int4* pairs;      // of each pair of query tiles: its first query row, query rows, sequence, cache rows
    int* cum_pairs;   // units of the pairs in front, all heads
    int* cum_rows;    // tiles of the rows' own parts in front, and a place for each part's start, all heads
    int* starts;      // group_starts, in range and not decreasing
    int* pair_rows;   // of each pair: cache rows
    int4* item_ctas;  // of each pair and head: its first unit, the first and last CTA that have some of it
    int* totals;      // pairs, units of pairs, tiles of rows
    float* parts_w;
    float* parts_s;
    int max_pairs;
    int* status;
};

__host__ __device__ inline size_t part_floats(int rows, int D) { return (size_t)rows * D + ((2 * rows + 3) & ~3); }  // (a multiple of sixteen bytes)

// the places 0 .. total - 1 in equal runs: worker w has begin(w) .. begin(w + 1) - 1
struct EqualRuns {
    int each, more;
    __device__ __forceinline__ EqualRuns(int total, int workers) : each((int)((unsigned)total / (unsigned)workers)), more(total - each * workers) {}
    __device__ __forceinline__ int begin(int w) const { return w * each + min(w, more); }
    __device__ __forceinline__ int owner(int at) const {
        const int border = more * (each + 1);
        return at < border ? (int)((unsigned)at / (unsigned)(each + 1)) : more + (int)((unsigned)(at - border) / (unsigned)each);
    }
};
// A CTA's share: units of pairs (two places each: a step of both streams), then tiles of rows (one place), the first half of them the first stream's.
struct Share {
    int w0, w1, s0, s1;
    __device__ __forceinline__ Share(const EqualRuns& runs, int units, int cta) {
        const int p0 = runs.begin(cta), p1 = runs.begin(cta + 1), border = 2 * units;
        w0 = min((p0 + 1) >> 1, units), w1 = min((p1 + 1) >> 1, units);
        s0 = max(p0 - border, 0), s1 = max(p1 - border, 0);
    }
    __device__ __forceinline__ int middle() const { return s0 + ((s1 - s0 + 1) >> 1); }
};

// ---------------------------------------------------------------------------------------------- plan

__device__ __forceinline__ int block_exclusive_scan(int x, int* warp_sums, int& total) {  // of kPlanThreads numbers
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += up;
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    int w = warp_sums[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, w, d);
        if (lane >= d) w += up;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const int before = __shfl_sync(0xffffffffu, w, max(warp - 1, 0));
    return incl - x + (warp > 0 ? before : 0);
}
__device__ __forceinline__ int block_max_scan(int x, int* warp_sums) {  // inclusive, of numbers that are not negative
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x = max(x, up);
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    int w = warp_sums[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, w, d);
        if (lane >= d) w = max(w, up);
    }
    const int before = __shfl_sync(0xffffffffu, w, max(warp - 1, 0));
    return warp > 0 ? max(x, before) : x;
}

// One CTA: which rows share what, the pairs of query tiles, and how many units lie in front of each pair and row.
__global__ void __launch_bounds__(kPlanThreads) shared_plan_kernel(const SharedArgs a, int ctas) {
    __shared__ int warp_sums[32];
    __shared__ int few[2][kFewGroups + 1];
    __shared__ int few_pairs[kFewGroups];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tid = threadIdx.x, cap = a.max_blocks << a.log2_rows;
    // what the phases hand on lies in shared memory where it fits: a phase costs a microsecond less than by way of L2
    int* const starts = a.n_groups <= kFewGroups ? few[0] : a.starts;
    int* const first_pairs = a.n_groups <= kFewGroups ? few[1] : a.cum_pairs;  // (overwritten later)
    int* const pair_rows = a.max_pairs <= kFewGroups ? few_pairs : a.pair_rows;
    // the groups' borders
    int carry = 0;
    for (int g0 = 0; g0 <= a.n_groups; g0 += kPlanThreads) {
        const int g = g0 + tid;
        const int x = g <= a.n_groups ? min(max(a.group_starts[g], 0), a.M) : 0;
        const int y = max(block_max_scan(x, warp_sums), carry);
        if (g <= a.n_groups) starts[g] = y;
        __syncthreads();
        carry = starts[min(g0 + kPlanThreads - 1, a.n_groups)];
    }
    __syncthreads();
    // the groups' pairs; a row on its own shares nothing.  pair_rows: the most that a pair's rows share
    int n_pairs = 0;
    for (int g0 = 0; g0 < a.n_groups; g0 += kPlanThreads) {
        const int g = g0 + tid;
        int n = 0, first = 0, query_rows = 0;
        if (g < a.n_groups) {
            first = starts[g];
            const int rows = starts[g + 1] - first;
            query_rows = rows * a.group;
            if (rows > 1 && a.shared_rows[g] > 0) n = (query_rows + 2 * kTile - 1) / (2 * kTile);
        }
        int total;
        const int at = n_pairs + block_exclusive_scan(n, warp_sums, total);
        for (int i = 0; i < n; ++i) {
            a.pairs[at + i] = make_int4(first * a.group + i * 2 * kTile, min(2 * kTile, query_rows - i * 2 * kTile), 0, 0);
            pair_rows[at + i] = 0;
        }
        if (g < a.n_groups) first_pairs[g] = n > 0 ? at : -1;
        n_pairs += total;
    }
    __syncthreads();
    int tiles_before = 0;
    const int each = a.M > kPlanThreads ? kPlanRows : 1;
    for (int m0 = 0; m0 < a.M; m0 += each * kPlanThreads) {
        const int m1 = m0 + each * tid, m2 = min(m1 + each, a.M);  // this thread's rows, their loads in flight together
        int seqs[kPlanRows], lens[kPlanRows], tiles[kPlanRows], sum = 0;
#pragma unroll
        for (int k = 0; k < kPlanRows; ++k) {
            const int m = m1 + k;
            seqs[k] = m < m2 ? (a.seq_ids ? a.seq_ids[m] : m) : -1;
            lens[k] = m < m2 ? a.lengths[m] : 0;
        }
#pragma unroll
        for (int k = 0; k < kPlanRows; ++k) {
            const int m = m1 + k;
            tiles[k] = 0;
            if (m >= m2) break;
            const int len = seqs[k] < 0 || seqs[k] >= a.n_seq ? 0 : min(max(lens[k], 0), cap);
            // the last group that begins at or before the row, if the row is not behind its end
            int lo = 0, hi = a.n_groups;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (starts[mid] <= m) lo = mid;
                else hi = mid - 1;
            }
            int4 info = make_int4(0, len, -1, 0);
            if (lo < a.n_groups && starts[lo] <= m && first_pairs[lo] >= 0) {
                const int flat0 = starts[lo] * a.group;
                info = make_int4(min(len, a.shared_rows[lo]), len, first_pairs[lo], flat0);
                if (info.x > 0) {
                    const int p0 = info.z + (m * a.group - flat0) / (2 * kTile), p1 = info.z + (m * a.group + a.group - 1 - flat0) / (2 * kTile);
                    for (int p = p0; p <= p1; ++p)
                        if (pair_rows[p] < info.x) atomicMax(&pair_rows[p], info.x);
                }
            }
            a.rows[m] = info;
            // a place for each head's start, too
            if (len > info.x) tiles[k] = ((len - ((info.x >> a.log2_rows) << a.log2_rows) + kTile - 1) / kTile + 1) * a.n_kv;
            sum += tiles[k];
        }
        int total;
        int at = tiles_before + block_exclusive_scan(sum, warp_sums, total);
#pragma unroll
        for (int k = 0; k < kPlanRows; ++k) {
            if (m1 + k >= m2) break;
            a.cum_rows[m1 + k] = at;
            at += tiles[k];
        }
        tiles_before += total;
    }
    __syncthreads();
    int units_before = 0;
    for (int p0 = 0; p0 < n_pairs; p0 += kPlanThreads) {
        const int p = p0 + tid;
        int units = 0;
        if (p < n_pairs) {
            int4 info = a.pairs[p];
            info.w = pair_rows[p];
            const int span = info.y > kTile ? kTile : 2 * kTile;  // a unit: one tile of cache rows for two query tiles, or two for one
            units = (info.w + span - 1) / span * a.n_kv;
            // It is read by the table of a row that has all of its cache rows; others' tables may end before.  The last row of a chunk is one, and any row of answers behind
            // their prompt, so the search begins at the end (with the maximum and its row in one 64-bit atomic the plan of two chunks took 10 us more).
            int row = 0;
            if (info.w > 0) {
                row = (info.x + info.y - 1) / a.group;
                for (bool found = a.rows[row].x == info.w; !found;) {
                    constexpr int AT_ONCE = 8;
                    const int from = row, first = info.x / a.group;
                    int x[AT_ONCE];
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k) x[k] = a.rows[max(from - 1 - k, first)].x;
#pragma unroll
                    for (int k = AT_ONCE - 1; k >= 0; --k)
                        if (x[k] == info.w) row = max(from - 1 - k, first), found = true;
                    if (!found) {
                        row = max(from - AT_ONCE, first);
                        found = row == first;  // (never without one)
                    }
                }
            }
            info.z = a.seq_ids ? a.seq_ids[row] : row;  // (no row has anything in the cache: no units)
            a.pairs[p] = info;
        }
        int total;
        const int at = units_before + block_exclusive_scan(units, warp_sums, total);
        if (p < n_pairs) a.cum_pairs[p] = at;
        units_before += total;
    }
    if (tid == 0) {
        a.cum_pairs[n_pairs] = units_before;
        a.cum_rows[a.M] = tiles_before;
        a.totals[0] = n_pairs, a.totals[1] = units_before, a.totals[2] = tiles_before;
    }
    __syncthreads();
    const EqualRuns runs(2 * units_before + tiles_before, ctas);
    for (int i = tid; i < n_pairs * a.n_kv; i += kPlanThreads) {
        const int p = i / a.n_kv, h = i - p * a.n_kv, c = a.cum_pairs[p], n = (a.cum_pairs[p + 1] - c) / a.n_kv, u0 = c + h * n;
        a.item_ctas[i] = make_int4(u0, runs.owner(2 * u0), runs.owner(2 * (u0 + max(n, 1) - 1)), 0);
    }
}

// ---------------------------------------------------------------------------------------------- tensor-core pieces

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Operand tiles: rows of 128 bytes (64 f16), 128-byte swizzle, groups of eight rows 1024 bytes apart; the second 64 columns follow 128 rows later.
// Read along the rows (queries and keys: the product's sum runs over dims) the leading offset has no meaning; read across them (values: the sum runs over cache
// rows) it leads from 64 dims to the next 64.
constexpr uint32_t kHalfTile = kTile * 128;
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t leading) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(leading >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// D fp32, A and B f16; B read across its rows where `across`
__host__ __device__ constexpr uint32_t instruction(int n, bool across) {
    return (1u << 4) | (across ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
}

#define TM32(r) \
    "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), \
        "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),     \
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
// lane l of the warp: 32 columns of its row
__device__ __forceinline__ void tm_load(uint32_t at, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : TM32(r)
        : "r"(at)
        : "memory");
}
__device__ __forceinline__ void tm_load16(uint32_t at, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
                   "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tm_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_store16(uint32_t at, const uint32_t (&v)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                 "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
                 : "memory");
}
__device__ __forceinline__ void tm_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Queries: a row is scaled by the power of two that brings its largest magnitude to 2^8 .. 2^9; bf16 values then fit f16 without loss down to 2^-22 of it.
// (Magnitudes by their bits: infinity and NaN are above all others, exponent 255.)
__device__ __forceinline__ uint32_t largest_bits(const uint4& v) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
    uint32_t most = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) most = max(most, max((u[e] << 16) & 0x7fffffffu, u[e] & 0x7fff0000u));
    return most;
}
__device__ __forceinline__ int query_exponent(uint32_t most) { return max((int)(most >> 23), 9); }
__device__ __forceinline__ float query_up(uint32_t most) { return __int_as_float((262 - query_exponent(most)) << 23); }
// what scores are multiplied by; a row that is not finite gives NaN
__device__ __forceinline__ float query_down(int exponent) { return exponent == 255 ? NAN : __int_as_float((exponent - 8) << 23); }
// eight queries, the `unit`-th sixteen bytes of row r of a Q tile
__device__ __forceinline__ void store_queries(uint32_t tile, int r, int unit, const uint4& v, float up) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
    uint32_t h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = pack_f16(__uint_as_float(u[e] << 16) * up, __uint_as_float(u[e] & 0xffff0000u) * up);
    sts128(tile + (uint32_t)r * 128u + (uint32_t)(unit >> 3) * kHalfTile + (uint32_t)(((unit & 7) ^ (r & 7)) << 4), h[0], h[1], h[2], h[3]);
}

__device__ __forceinline__ void code_rows(uint32_t dst, const CUtensorMap* map, int row, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(0), "r"(row), "r"(bar)
                 : "memory");
}

// ---------------------------------------------------------------------------------------------- main kernel

// One stream's half of a step.
constexpr int kLive = 1, kFirst = 2, kLast = 4, kOwn = 8;  // there is one; its softmax begins, ends with it; a tile of what a row has for itself (else of a pair)
struct Side {
    int flags;
    int row0, rows;         // query rows
    int head;
    int base;               // first cache row
    int cache_rows;         // of the tile, those that any query row uses
    int lost;               // bit i: cache rows 16 i .. 16 i + 15 belong to no block
    int part;               // where the result goes
    int lower, upper;       // kOwn: the cache rows that the row uses
};
struct __align__(16) Desc {
    float ks[2][8], vs[2][8];  // scales of each sixteen rows
    Side side[2];
    int end, common;           // no more steps; both streams use the first one's cache rows
    int pad[2];
};

template <int D>
struct SharedSmem {
    static constexpr int kOperands = D == 128 ? 4 : 6;  // tiles of f16
    static constexpr int kStages = D == 128 ? 2 : 8;    // tiles of codes
    static_assert(kOperands % 2 == 0 && kStages % 2 == 0, "a place belongs to the same four conversion warps every time, which then wait for each of its phases");
    static constexpr uint32_t kOperandBytes = kTile * D * 2, kCodeBytes = kTile * D;
    // what is small lies in front of the tiles
    static constexpr uint32_t exponents = 0, descs = 2 * 2 * kTile, bars = descs + kDescs * sizeof(Desc);
    // barriers
    static constexpr int code_full = 0, code_empty = code_full + kStages, op_full = code_empty + kStages, op_empty = op_full + kOperands, desc_full = op_empty + kOperands,
                         desc_empty = desc_full + kDescs, q_full = desc_empty + kDescs, q_free = q_full + 2, s_full = q_free + 2, p_full = s_full + 4, o_full = p_full + 4,
                         pv_done = o_full + 2, n_bars = pv_done + 2;
    static constexpr uint32_t small = bars + n_bars * 8 + 8, q = (small + 1023) / 1024 * 1024, operands = q + 2 * kOperandBytes, codes = operands + kOperands * kOperandBytes;
    static constexpr uint32_t total = codes + kStages * kCodeBytes;
};

template <int D, int KIND>
__global__ void __launch_bounds__(kThreads, 1) shared_attention_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const SharedArgs a) {
    using L = SharedSmem<D>;
    extern __shared__ __align__(1024) uint8_t smem[];  // (the tiles' swizzle wants borders of 1024; there is no other shared memory in front)
    const uint32_t base_s = smem_u32(smem);
    if (base_s & 1023u) {  // (never so far: copies to other borders would fault)
        if (threadIdx.x == 0 && a.status != nullptr) atomicExch(a.status, BITLINEAR_ERR_CUDA);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    Desc* descs = reinterpret_cast<Desc*>(smem + L::descs);
    auto bar = [&](int i) { return base_s + L::bars + 8u * (uint32_t)i; };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::bars + L::n_bars * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    if (tid == 0) {
        *abort_flag = 0;
        for (int i = 0; i < L::kStages; ++i) mbar_init(bar(L::code_full + i), 1), mbar_init(bar(L::code_empty + i), 4);
        for (int i = 0; i < L::kOperands; ++i) mbar_init(bar(L::op_full + i), 4), mbar_init(bar(L::op_empty + i), 2);
        for (int i = 0; i < kDescs; ++i) mbar_init(bar(L::desc_full + i), 1 + 32), mbar_init(bar(L::desc_empty + i), 2 + 1 + 8 + 8);
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar(L::q_full + s), 4);
            mbar_init(bar(L::q_free + s), 1);
            mbar_init(bar(L::o_full + s), 1);
            mbar_init(bar(L::pv_done + s), 1);
        }
        for (int i = 0; i < 4; ++i) mbar_init(bar(L::s_full + i), 1), mbar_init(bar(L::p_full + i), 4);
        mbar_init_fence();
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    auto tm_s = [&](int s) { return tmem + (uint32_t)(s * kTile); };            // scores, then weights, of a stream
    auto tm_o = [&](int s) { return tmem + (uint32_t)(2 * kTile + s * D); };  // its accumulator
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // A wait that runs out raises the abort flag and lets its warp go on; every role looks at the flag once a step (a vote after each wait cost the products a
    // hundred cycles apiece).  Until then it works on what is there: nothing leaves its bounds.
    auto wait = [&](int i, uint32_t parity) {
        if (!mbar_try_wait(bar(i), parity)) mbar_wait(bar(i), parity, abort_flag);
        __syncwarp();
    };
    auto aborted = [&] { return __any_sync(0xffffffffu, *abort_flag != 0); };

    // All roles walk the steps in the same order of products: S of step 0 (both streams), then for every step and stream O, and S of the step behind.
    // Operand tiles are made and used in that order.
    if (warp >= 4 && warp < 12) {
        // The softmax holds 64 scores in registers: its eight warps take what the other twelve leave of the launch's (256 * 144 + 384 * 64 of 640 * 96).
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        // ------------------------------------------------------------------ softmax
        const int s = (warp - 4) >> 2, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lane_at = (uint32_t)(quad * 32) << 16;
        const uint32_t ts = tm_s(s) + lane_at, to = tm_o(s) + lane_at;
        float f = 0.0f, m_run = -INFINITY, l_run = 0.0f, v_ref = 0.0f, per_ref = 0.0f;  // per_ref: the weights' scale by v_ref
        int lower = 0, upper = 0;
        uint32_t s_phase = 0, o_phase = 0, item = 0, halves = 0;  // items, half steps so far
        // A finished item's accumulator is read after the next item's queries are on their way.
        bool finished = false, after_pairs = false;
        float* part = nullptr;
        int part_rows = 0;
        bool in_part = false, any_in_part = false;
        auto hand_over = [&] {
            finished = false;
            wait(L::o_full + s, o_phase);
            o_phase ^= 1u;
            tc_fence_after();
            if (any_in_part) {
                const float unscale = v_ref * (1.0f / kWeightScale);
#pragma unroll 1
                for (int i = 0; i < D / 16; ++i) {
                    uint32_t o[16];
                    tm_load16(to + 16 * i, o);
                    tm_load_wait();
                    if (in_part) {
#pragma unroll
                        for (int e = 0; e < 16; e += 4)  // (four dims of all rows lie together, so that a warp writes whole lines)
                            *reinterpret_cast<float4*>(part + (size_t)((4 * i + e / 4) * part_rows + r) * 4) =
                                make_float4(__uint_as_float(o[e]) * unscale, __uint_as_float(o[e + 1]) * unscale, __uint_as_float(o[e + 2]) * unscale,
                                            __uint_as_float(o[e + 3]) * unscale);
                    }
                }
                if (in_part) *reinterpret_cast<float2*>(part + (size_t)part_rows * D + 2 * r) = make_float2(m_run, l_run);
            }
            tc_fence_before();
        };
        for (int p = 0; !aborted(); ++p) {
            const int slot = p % kDescs;
            wait(L::desc_full + slot, (uint32_t)(p / kDescs) & 1u);
            const Desc& d = descs[slot];
            if (d.end) {
                if (finished) hand_over();
                break;
            }
            const Side& x = d.side[s];
            const int flags = x.flags;
            if (!(flags & kLive)) {
                if (finished) hand_over();
                if (lane == 0) mbar_arrive(bar(L::desc_empty + slot));
                continue;
            }
            const int n_rows = x.rows, part_at = x.part, base = x.base, lost = x.lost;
            const bool mine = r < n_rows, any = quad * 32 < n_rows;
            if (flags & kFirst) {
                if (flags & kOwn) {
                    lower = x.lower, upper = x.upper;
                    if (after_pairs && quad == 0 && lane == 0) mbar_arrive(bar(L::q_free + s));
                    after_pairs = false;
                } else {
                    after_pairs = true;
                    // sixteen (eight) lanes bring a row together, eight loads in flight (a row to each lane took the L1 cache 32 lines a load: 8,000 cycles for a tile)
                    constexpr int LANES = D / 8, AT_ONCE = 32 / LANES;
                    const int unit = lane % LANES;
                    uint8_t* exponents = smem + L::exponents + (s * 2 + (item & 1u)) * kTile;
                    if (any) {
#pragma unroll 1
                        for (int i0 = 0; i0 < LANES; i0 += 8) {
                            uint4 v[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const int row = quad * 32 + (i0 + i) * AT_ONCE + lane / LANES, flat = x.row0 + min(row, n_rows - 1), m = flat / a.group, j = flat - m * a.group;
                                v[i] = *(reinterpret_cast<const uint4*>(a.q + ((size_t)m * a.n_q + (size_t)x.head * a.group + j) * D) + unit);
                            }
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const int row = quad * 32 + (i0 + i) * AT_ONCE + lane / LANES;
                                uint32_t most = largest_bits(v[i]);
#pragma unroll
                                for (int off = LANES / 2; off > 0; off >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, off));
                                store_queries(base_s + L::q + (uint32_t)s * L::kOperandBytes, row, unit, v[i], query_up(most));
                                if (unit == 0) exponents[row] = (uint8_t)query_exponent(most);
                            }
                        }
                        __syncwarp();
                        if (mine) {
                            lower = 0, upper = a.rows[(x.row0 + r) / a.group].x;
                            f = query_down(exponents[r]) * a.scale_log2;
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(L::q_full + s));
                }
                if (finished) hand_over();
                m_run = -INFINITY, l_run = 0.0f, v_ref = 0.0f, per_ref = 0.0f;
            }
            // what this row uses of the tile
            const int lo = max(lower - base, 0), hi = min(upper - base, kTile);
            const bool all_used = __all_sync(0xffffffffu, !mine || (lo == 0 && hi == kTile && lost == 0));
#pragma unroll 1
            for (int h = 0; h < 2; ++h, ++halves) {
                // what does not hang on the scores comes before them
                const float4 k4 = *reinterpret_cast<const float4*>(&d.ks[s][4 * h]), w4 = *reinterpret_cast<const float4*>(&d.vs[s][4 * h]);
                float ks[4] = {k4.x, k4.y, k4.z, k4.w}, rs[4] = {w4.x, w4.y, w4.z, w4.w};
                wait(L::s_full + 2 * s + h, s_phase);
                tc_fence_after();
                if ((flags & (kFirst | kOwn)) == (kFirst | kOwn) && h == 0 && mine) f = query_down(smem[L::exponents + (s * 2 + (item & 1u)) * kTile + r]) * a.scale_log2;
                if (any) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) ks[i] *= f;
                    if (!all_used) {  // what the row does not use scores -infinity, whatever lies there; its scales count for nothing
                        const int l = max(lo - kHalf * h, 0), n = min(max(hi - kHalf * h, 0), kHalf);
                        unsigned long long live = n > l ? (~0ull >> (64 - n)) & (~0ull << l) : 0ull;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if ((lost >> (4 * h + i)) & 1) live &= ~(0xffffull << (16 * i));
                            const bool none = ((uint32_t)(live >> (16 * i)) & 0xffffu) == 0u;
                            if (none || ks[i] == 0.0f) ks[i] = 1e-30f;  // -infinity times a scale of zero would be NaN; finite scores stay next to zero
                            if (none) rs[i] = 0.0f;
                        }
#pragma unroll 1
                        for (int i = 0; i < 4; ++i) {
                            uint32_t x[16];
                            tm_load16(ts + kHalf * h + 16 * i, x);
                            const uint32_t used = (uint32_t)(live >> (16 * i));
                            tm_load_wait();
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                if (!((used >> e) & 1u)) x[e] = 0xff800000u;
                            tm_store16(ts + kHalf * h + 16 * i, x);
                        }
                        tm_store_wait();
                    }
                    uint32_t v[2][32];
                    tm_load(ts + kHalf * h, v[0]);
                    tm_load(ts + kHalf * h + 32, v[1]);
                    const float vs = fmaxf(fmaxf(rs[0], rs[1]), fmaxf(rs[2], fmaxf(rs[3], 0.0f)));
                    float ww[4];  // the weights' factors, if the largest scale of values stays
#pragma unroll
                    for (int i = 0; i < 4; ++i) ww[i] = rs[i] * per_ref;
                    tm_load_wait();
                    float top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t* x16 = v[i >> 1] + 16 * (i & 1);
                        float t = __uint_as_float(x16[15]);
#pragma unroll
                        for (int e = 0; e < 14; e += 2) t = fmaxf(fmaxf(t, __uint_as_float(x16[e])), __uint_as_float(x16[e + 1]));
                        top = fmaxf(top, fmaxf(t, __uint_as_float(x16[14])) * ks[i]);
                    }
                    // The maximum is followed only where it grows by more than 2^8: weights stay within f16, and the accumulator is rarely scaled.
                    const bool grows = top > m_run + 8.0f || (m_run == -INFINITY && top > -INFINITY), wider = vs > v_ref;
                    if (__any_sync(0xffffffffu, grows || wider)) {
                        const float n = grows ? top : m_run, nv = fmaxf(v_ref, vs);
                        const float c = m_run == -INFINITY ? 0.0f : ex2(m_run - n);  // (nothing there yet: zeros)
                        const float fo = nv > 0.0f ? c * (v_ref / nv) : c;
                        l_run *= c;
                        if (!(flags & kFirst) || h == 1) {
                            wait(L::pv_done + s, (halves - 1u) & 1u);  // (the half in front of the last is in, or these scores would not be here)
                            tc_fence_after();
#pragma unroll 1
                            for (int i = 0; i < D / 16; ++i) {
                                uint32_t o[16];
                                tm_load16(to + 16 * i, o);
                                tm_load_wait();
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * fo);
                                tm_store16(to + 16 * i, o);
                            }
                        }
                        m_run = n;
                        v_ref = nv;
                        per_ref = v_ref > 0.0f ? __fdividef(kWeightScale, v_ref) : 0.0f;
#pragma unroll
                        for (int i = 0; i < 4; ++i) ww[i] = rs[i] * per_ref;
                    }
                    // Weights, times their rows' scale of values, are rounded to f16 in units of the largest scale met so far: up to 2^-11 of each, an eighth of what the result's
                    // rounding to bf16 may cost, and below 2^-21 of those units, where f16 has no more normal numbers, up to 2^-32 of them.  Their sum takes them unrounded.
                    // They go over the scores.
                    float2 sum = make_float2(0.0f, 0.0f);
                    const float2 bb = splat(m_run == -INFINITY ? 0.0f : -m_run);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t w[16];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float2 kk = splat(ks[2 * c + i]), factor = splat(ww[2 * c + i]);
#pragma unroll
                            for (int e = 0; e < 16; e += 2) {
                                float2 t = fma2(make_float2(__uint_as_float(v[c][16 * i + e]), __uint_as_float(v[c][16 * i + e + 1])), kk, bb);
                                t.x = ex2(t.x), t.y = ex2(t.y);
                                sum = add2(sum, t);
                                t = mul2(t, factor);
                                w[8 * i + e / 2] = pack_f16(t.x, t.y);
                            }
                        }
                        tm_store16(ts + kHalf * h + 16 * c, w);
                    }
                    l_run += sum.x + sum.y;
                    tm_store_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(L::p_full + 2 * s + h));
            }
            s_phase ^= 1u;
            if (lane == 0) mbar_arrive(bar(L::desc_empty + slot));
            if (flags & kLast) {
                ++item;
                finished = true, in_part = mine, any_in_part = any;
                part_rows = flags & kOwn ? a.group : kTile;
                part = (flags & kOwn ? a.parts_s : a.parts_w) + (size_t)part_at * part_floats(part_rows, D);
            }
        }
    } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == 3) {
        // ------------------------------------------------------------------ copies and the work list
        // Half of the lanes keep the books of either stream.
        const int s = lane >> 4, l16 = lane & 15;
        const int units = a.totals[1], tiles = a.totals[2];
        const Share share(EqualRuns(2 * units + tiles, gridDim.x), units, cta);
        // the entry of cum[0 .. n] (not decreasing) that holds `at`, the last one that is not above it; in a half whose `wanted` is false: 0
        auto find = [&](const int* cum, int n, int at, bool wanted) {
            int lo = 0, hi = wanted ? n : 1;  // cum[lo] <= at < cum[hi]
            while (__any_sync(0xffffffffu, hi - lo > 1)) {
                const int step = max(1, (hi - lo) / 16), probe = min(lo + step * (l16 + 1), hi);
                const bool past = probe >= hi || cum[probe] > at;
                const unsigned above = (__ballot_sync(0xffffffffu, past) >> (16 * s)) & 0xffffu;
                if (hi - lo > 1) {
                    const int i = __ffs((int)above) - 1;  // (the last lane may probe below hi)
                    if (i < 0) lo += 16 * step;
                    else {
                        hi = min(lo + step * (i + 1), hi);
                        lo += step * i;
                    }
                }
            }
            return lo;
        };
        // units of pairs, the same for both streams
        int wu = share.w0, w_head = 0, w_unit = 0, w_units = 1;
        int pair = find(a.cum_pairs, a.totals[0], wu, wu < share.w1);
        int4 pair_info = make_int4(0, 0, 0, 0);
        if (wu < share.w1) {
            const int c = a.cum_pairs[pair];
            w_units = (a.cum_pairs[pair + 1] - c) / a.n_kv;
            w_head = (wu - c) / w_units;
            w_unit = wu - c - w_head * w_units;
            pair_info = a.pairs[pair];
        }
        // tiles of rows
        const int s_begin = s ? share.middle() : share.s0, s_end = s ? share.s1 : share.middle();
        int su = s_begin, s_head = 0, s_tile = 0, s_tiles = 1, seq = 0;
        bool fresh = true;  // the next tile is its item's first of this run
        int m = find(a.cum_rows, a.M, su, su < s_end);
        int2 row = make_int2(0, 0);  // cache rows shared, length
        auto enter_row = [&] {
            s_tiles = (a.cum_rows[m + 1] - a.cum_rows[m]) / a.n_kv - 1;
            const int4 info = a.rows[m];
            row = make_int2(info.x, info.y);
            seq = a.seq_ids ? a.seq_ids[m] : m;
        };
        if (su < s_end) {
            enter_row();
            const int at = su - a.cum_rows[m];
            s_head = at / (s_tiles + 1);
            s_tile = at - s_head * (s_tiles + 1) - 1;
            if (s_tile < 0) s_tile = 0, ++su;  // the place that stands for the start
        }
        const int per_tile = kTile >> a.log2_rows;  // blocks
        struct Tile {  // of a step and stream: lane i has block i
            int id, head;
            bool there;
        };
        int made = 0;  // code tiles so far
        // publishes step p; false at the end
        auto publish = [&](int p, Tile& now) {
            const int slot = p % kDescs;
            if (p >= kDescs) wait(L::desc_empty + slot, (uint32_t)(p / kDescs - 1) & 1u);
            Desc& d = descs[slot];
            const bool pairs_left = wu < share.w1, row_left = !pairs_left && su < s_end;
            const bool end = !__any_sync(0xffffffffu, pairs_left || row_left), common = pairs_left && pair_info.y > kTile;
            Side x = {};
            if (pairs_left) {
                const int tile = common ? w_unit : 2 * w_unit + s, rows = pair_info.w;
                const bool first = wu == share.w0 || w_unit == 0, last = wu == share.w1 - 1 || (tile + (common ? 1 : 2)) * kTile >= rows;
                x.flags = tile * kTile < rows ? kLive | (first ? kFirst : 0) | (last ? kLast : 0) : 0;
                x.row0 = pair_info.x + (common ? s * kTile : 0);
                x.rows = common ? (s ? pair_info.y - kTile : kTile) : pair_info.y;
                x.head = w_head;
                x.base = tile * kTile;
                x.cache_rows = min(rows - x.base, kTile);
                x.part = (pair * a.n_kv + w_head + cta) * 2 + s;
            } else if (row_left) {
                x.flags = kLive | kOwn | (fresh ? kFirst : 0) | (s_tile == s_tiles - 1 || su == s_end - 1 ? kLast : 0);
                fresh = false;
                x.row0 = m * a.group;
                x.rows = a.group;
                x.head = s_head;
                x.base = ((row.x >> a.log2_rows) << a.log2_rows) + s_tile * kTile;
                x.cache_rows = min(row.y - x.base, kTile);
                x.part = m * a.n_kv + s_head + 2 * cta + s;
                x.lower = row.x, x.upper = row.y;
            }
            const bool live = x.flags & kLive;
            now.there = live && !(common && s == 1);
            now.head = x.head;
            now.id = -1;
            if (now.there && l16 < per_tile && (l16 << a.log2_rows) < x.cache_rows) {
                const int id = a.tables[(size_t)(pairs_left ? pair_info.z : seq) * a.max_blocks + (x.base >> a.log2_rows) + l16];
                now.id = id < a.n_blocks ? id : -1;
            }
            const int from = common ? 0 : 16 * s;
            const unsigned have = __ballot_sync(0xffffffffu, now.id >= 0) >> from;
            if (live) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (!((have >> ((16 * i) >> a.log2_rows)) & 1u)) x.lost |= 1 << i;
            }
            // scales: the lower eight lanes of a half bring those of cache rows 16 i .. of the keys, the upper ones of the values
            {
                const int i = l16 & 7, id = __shfl_sync(0xffffffffu, now.id, from + ((16 * i) >> a.log2_rows));
                float* to = &(l16 >> 3 ? d.vs : d.ks)[s][i];
                if (id >= 0) {
                    const float* src = (l16 >> 3 ? a.v_scale : a.k_scale) + (size_t)id * a.n_kv + x.head;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(to)), "l"(src) : "memory");
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar(L::desc_full + slot)) : "memory");
                } else {
                    *to = 0.0f;
                    mbar_arrive(bar(L::desc_full + slot));
                }
            }
            if (l16 == 0) d.side[s] = x;
            if (lane == 0) d.end = end, d.common = common;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(L::desc_full + slot));
            // on to the next step
            if (pairs_left) {
                ++wu;
                if (++w_unit == w_units && wu < share.w1) {
                    w_unit = 0;
                    if (++w_head == a.n_kv) {
                        w_head = 0;
                        do ++pair;
                        while (a.cum_pairs[pair + 1] == a.cum_pairs[pair]);
                        w_units = (a.cum_pairs[pair + 1] - a.cum_pairs[pair]) / a.n_kv;
                        pair_info = a.pairs[pair];
                    }
                }
            } else if (row_left) {
                ++su;
                if (++s_tile == s_tiles && ++su < s_end) {
                    s_tile = 0, fresh = true;
                    if (++s_head == a.n_kv) {
                        s_head = 0;
                        do ++m;
                        while (a.cum_rows[m + 1] == a.cum_rows[m]);
                        enter_row();
                    }
                }
            }
            __syncwarp();
            return !end;
        };
        auto load = [&](const Tile& now, int which, const CUtensorMap* map) {
            if (!__shfl_sync(0xffffffffu, (int)now.there, 16 * which)) return;
            const int place = made % L::kStages;
            if (made >= L::kStages) wait(L::code_empty + place, (uint32_t)(made / L::kStages - 1) & 1u);
            ++made;
            const bool mine = s == which && now.id >= 0;
            const unsigned present = __ballot_sync(0xffffffffu, mine);
            const uint32_t full = bar(L::code_full + place), block_bytes = (uint32_t)D << a.log2_rows;
            if (lane == 0) mbar_expect_tx(full, (uint32_t)__popc(present) * block_bytes);
            __syncwarp();
            if (mine) code_rows(base_s + L::codes + (uint32_t)place * L::kCodeBytes + (uint32_t)l16 * block_bytes, map, (now.id * a.n_kv + now.head) << a.log2_rows, full);
        };
        Tile now = {-1, 0, false}, next = now;
        bool ended = false;
        for (int p = -1; !aborted(); ++p) {
#pragma unroll 1
            for (int i = 0; i < 2; ++i) {  // values of step p, keys of the next, for either stream
                load(now, i, &map_v);
                if (i == 0 && !publish(p + 1, next)) next.there = false, ended = true;
                load(next, i, &map_k);
            }
            if (ended) break;
            now = next;
        }
    } else if (warp == 1 || warp == 2) {
        // ------------------------------------------------------------------ products, a warp for each stream: one thread starts a product every 55 cycles at most
        // (What the instructions take is made the same for all lanes first: they want it in uniform registers.)
        const int s = __shfl_sync(0xffffffffu, warp - 1, 0);
        const uint32_t scores_at = __shfl_sync(0xffffffffu, tm_s(s), 0), sums_at = __shfl_sync(0xffffffffu, tm_o(s), 0);
        const uint32_t s_full = __shfl_sync(0xffffffffu, bar(L::s_full + 2 * s), 0), o_full = __shfl_sync(0xffffffffu, bar(L::o_full + s), 0);
        const uint32_t q_free = __shfl_sync(0xffffffffu, bar(L::q_free + s), 0), pv_done = __shfl_sync(0xffffffffu, bar(L::pv_done + s), 0);
        constexpr uint32_t kScores = instruction(kHalf, false), kValues = instruction(D, true);
        const uint64_t q_tile = operand(__shfl_sync(0xffffffffu, base_s + L::q + (uint32_t)s * L::kOperandBytes, 0), 16);
        const uint32_t at1 = __shfl_sync(0xffffffffu, scores_at + kHalf, 0), rows1 = __shfl_sync(0xffffffffu, 512, 0);  // the second half: 64 rows of 128 bytes, in sixteens
        const uint32_t full1 = __shfl_sync(0xffffffffu, s_full + 8, 0);
        uint32_t q_phase = 0, p_phase = 0;
        int made = 0;                // operand tiles so far, of both streams
        int now = 0, other_now = 0;  // flags of step p, this stream's and the other's
        bool common_now = false;
        auto filled = [&](int tile) { wait(L::op_full + tile % L::kOperands, (uint32_t)(tile / L::kOperands) & 1u); };
        // the other stream's tile: one is free when both warps have passed it
        auto pass = [&](int tile) {
            filled(tile);
            if (lane == 0) mbar_arrive(bar(L::op_empty + tile % L::kOperands));
        };
        // Half by half, step p's values, then the scores of the next, of this stream.
        for (int p = -1; !aborted(); ++p) {
            const int slot = (p + 1) % kDescs;
            wait(L::desc_full + slot, (uint32_t)((p + 1) / kDescs) & 1u);
            const Desc& d = descs[slot];
            const bool more = !d.end, common = d.common;
            const int next = __shfl_sync(0xffffffffu, d.side[s].flags, 0), other = __shfl_sync(0xffffffffu, d.side[1 - s].flags, 0);
            // tiles in the order in which they are made: values of the first stream, its next keys, the second's values, its next keys
            const bool v0 = (s ? other_now : now) & kLive, k0 = (s ? other : next) & kLive, v1 = ((s ? now : other_now) & kLive) && !common_now, k1 = ((s ? next : other) & kLive) && !common;
            const int tile_v0 = made, tile_k0 = tile_v0 + v0, tile_v1 = tile_k0 + k0, tile_k1 = tile_v1 + v1;
            made = tile_k1 + k1;
            const int value = s && !common_now ? tile_v1 : tile_v0, key = s && !common ? tile_k1 : tile_k0;
            if (s == 1) {
                if (v0 && !common_now) pass(tile_v0);
                if (k0 && !common) pass(tile_k0);
            }
            const bool has_value = now & kLive, has_key = next & kLive;
            const uint32_t tiles_at = base_s + L::operands;
            const uint64_t v_tile = operand(__shfl_sync(0xffffffffu, tiles_at + (uint32_t)(value % L::kOperands) * L::kOperandBytes, 0), kHalfTile);
            const uint64_t k_tile = operand(__shfl_sync(0xffffffffu, tiles_at + (uint32_t)(key % L::kOperands) * L::kOperandBytes, 0), 16);
            const uint32_t v_done = __shfl_sync(0xffffffffu, bar(L::op_empty + value % L::kOperands), 0), k_done = __shfl_sync(0xffffffffu, bar(L::op_empty + key % L::kOperands), 0);
            const bool one = elect_one();
            if (has_value) filled(value);
            // (A pair's queries come from softmax threads that first finish what is under way: then both halves' values go first.)
            const bool late = has_key && (next & (kFirst | kOwn)) == kFirst;
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
                const int h = late ? i & 1 : i >> 1;
                const bool values = late ? i < 2 : !(i & 1);
                const uint32_t at = h ? at1 : scores_at, rows = h ? rows1 : 0u, full = h ? full1 : s_full;
                if (values && has_value) {
                    wait(L::p_full + 2 * s + h, p_phase);
                    tc_fence_after();
                    if (one) {
#pragma unroll
                        for (int k = 0; k < kHalf / 16; ++k) mma_ts(sums_at, at + 8 * k, v_tile + rows + 128u * k, kValues, !((now & kFirst) && h == 0 && k == 0));
                        tc_commit(pv_done);
                        if (h == 1) {
                            if (now & kLast) tc_commit(o_full);
                            tc_commit(v_done);
                        }
                    }
                }
                if (!values && has_key) {
                    if (h == 0) {
                        filled(key);
                        if (next & kFirst) {
                            wait(L::q_full + s, q_phase);
                            q_phase ^= 1u;
                        }
                    }
                    if (one) {
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint32_t off = ((uint32_t)(k / 4) * kHalfTile + (uint32_t)(k % 4) * 32u) >> 4;
                            mma_ss(at, q_tile + off, k_tile + rows + off, kScores, k > 0);
                        }
                        tc_commit(full);
                        if (h == 1) {
                            tc_commit(k_done);
                            if ((next & (kLast | kOwn)) == (kLast | kOwn)) tc_commit(q_free);
                        }
                    }
                }
                __syncwarp();
            }
            if (has_value) p_phase ^= 1u;
            if (p >= 0 && lane == 0) mbar_arrive(bar(L::desc_empty + p % kDescs));
            __syncwarp();
            if (!more) break;
            if (s == 0) {
                if (v1) pass(tile_v1);
                if (k1) pass(tile_k1);
            }
            now = next, other_now = other, common_now = common;
        }
    } else if (warp == 0) {
        // ------------------------------------------------------------------ queries of rows' own tiles
        // q_free completes once for each of a stream's own items, when its scores are made, and once before the first of them if pairs' items are in front, when the softmax
        // has seen the last one's scores.  This warp waits for every one in turn: it may fall steps behind a stream's pairs, and a barrier that moved on by two phases
        // meanwhile would look as if it had not moved.
        uint32_t items[2] = {0u, 0u}, freed[2] = {0u, 0u};
        for (int p = 0; !aborted(); ++p) {
            const int slot = p % kDescs;
            wait(L::desc_full + slot, (uint32_t)(p / kDescs) & 1u);
            const Desc& d = descs[slot];
            if (d.end) break;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const Side& x = d.side[s];
                if ((x.flags & (kLive | kFirst)) != (kLive | kFirst)) continue;
                const uint32_t item = items[s]++;
                if (!(x.flags & kOwn)) continue;  // (a pair's: its rows' softmax warps bring them)
                if (item > 0) wait(L::q_free + s, freed[s]++ & 1u);  // the scores of the item in front are made
                const int r = lane >> 2, c = lane & 3;  // four lanes to a row, eight rows at most
                uint4 v[D / 32];
                uint32_t most = 0u;
                if (r < x.rows) {
                    const uint4* src = reinterpret_cast<const uint4*>(a.q + ((size_t)x.row0 + (size_t)(x.row0 / a.group) * (a.n_q - a.group) + (size_t)x.head * a.group + r) * D) + c * (D / 32);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) v[i] = src[i], most = max(most, largest_bits(v[i]));
                }
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                if (r < x.rows) {
                    const float up = query_up(most);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) store_queries(base_s + L::q + (uint32_t)s * L::kOperandBytes, r, c * (D / 32) + i, v[i], up);
                    if (c == 0) smem[L::exponents + (s * 2 + (item & 1u)) * kTile + r] = (uint8_t)query_exponent(most);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane < 4) mbar_arrive(bar(L::q_full + s));
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(L::desc_empty + slot));
        }
    } else if (warp >= 12) {
        // ------------------------------------------------------------------ codes -> f16
        const int t = tid & 127, mine = (warp - 12) >> 2;  // of every two tiles, the first four warps take one, the others the next
        // A thread takes sixteen codes of every 16th (32nd) row, always of the same columns.  Eight neighbouring lanes read eight different sixteen-byte columns
        // of the banks and write eight: four pieces of a row, the other four of its neighbour (which the swizzle moves by one sixteen-byte unit).
        const int chunk = t % (D / 16), row = D == 128 ? (t / 8) ^ (chunk >> 2) : t / 4;
        const uint32_t in_at = (uint32_t)(row * D) + (uint32_t)((D == 128 ? chunk ^ (row & 7) : chunk ^ ((row >> 1) & 3)) << 4);
        const uint32_t out_at = (uint32_t)(chunk >> 2) * kHalfTile + (uint32_t)row * 128u + (uint32_t)(((2 * (chunk & 3)) ^ (row & 7)) << 4);
        int made = 0;
        auto convert = [&](int p, int s, bool value) {
            const Desc& d = descs[p % kDescs];
            const Side& x = d.side[s];
            if (!(x.flags & kLive) || (d.common && s == 1)) return;
            if ((made & 1) != mine) {
                ++made;
                return;
            }
            const int from = made % L::kStages, to = made % L::kOperands;
            wait(L::code_full + from, (uint32_t)(made / L::kStages) & 1u);
            if (made >= L::kOperands) wait(L::op_empty + to, (uint32_t)(made / L::kOperands - 1) & 1u);
            ++made;
            const uint32_t src = base_s + L::codes + (uint32_t)from * L::kCodeBytes, dst = base_s + L::operands + (uint32_t)to * L::kOperandBytes;
            const int cache_rows = x.cache_rows, lost = x.lost;
            const bool whole = !value || (cache_rows == kTile && lost == 0);
            const uint32_t in = src + in_at, out0 = dst + out_at, out1 = dst + (out_at ^ 16u);
            constexpr int STEP = 128 * 16 / D;  // rows from a thread's piece to its next
            // Values of no one's rows become 0: they may hold NaN, and zero times NaN is NaN.
            const int there = whole ? kTile : cache_rows, gone = whole ? 0 : lost;
#pragma unroll 1
            for (int i = 0; i < D / 16; ++i) {
                uint32_t w[4], h[8];
                const int r = row + i * STEP;
                lds128(in + i * STEP * D, w);
                if (r >= there || ((gone >> (r >> 4)) & 1)) w[0] = w[1] = w[2] = w[3] = 0u;
#pragma unroll
                for (int j = 0; j < 4; ++j) codes_to_f16<KIND>(w[j], h[2 * j], h[2 * j + 1]);
                sts128(out0 + i * STEP * 128, h[0], h[1], h[2], h[3]);
                sts128(out1 + i * STEP * 128, h[4], h[5], h[6], h[7]);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(bar(L::op_full + to));
                mbar_arrive(bar(L::code_empty + from));
            }
        };
        for (int p = -1; !aborted(); ++p) {
            bool more = false;
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {  // values of step p, keys of the next, for either stream
                if (i == 1) {
                    wait(L::desc_full + (p + 1) % kDescs, (uint32_t)((p + 1) / kDescs) & 1u);
                    more = !descs[(p + 1) % kDescs].end;
                }
                if (i & 1 ? more : p >= 0) convert(i & 1 ? p + 1 : p, i >> 1, !(i & 1));
            }
            __syncwarp();
            if (p >= 0 && lane == 0) mbar_arrive(bar(L::desc_empty + p % kDescs));
            if (!more) break;
        }
    }
    }
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        abort_drain();
        if (tid == 0 && a.status != nullptr) atomicExch(a.status, BITLINEAR_ERR_TIMEOUT);
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ---------------------------------------------------------------------------------------------- the parts of a row

// A query head's parts, by four warps: each takes 32 parts in turn of each of the two kinds.  Lane l first finds the l-th of a round's parts and weighs it;
// then all lanes add up the rounds' values, a few dims each, eight parts' loads in flight.
constexpr int kJoinWarps = 4;
template <int D>
__global__ void __launch_bounds__(32 * kJoinWarps, 6) shared_combine_kernel(const SharedArgs a, int ctas) {
    constexpr int DIMS = D / 32, AT_ONCE = 8;
    __shared__ float2 joined[kJoinWarps];
    __shared__ float values[kJoinWarps][D];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int item = (int)blockIdx.x, m = item / a.n_q, head = item - m * a.n_q, h = head / a.group, j = head - h * a.group;
    const int units = a.totals[1], tiles = a.totals[2];
    const EqualRuns runs(2 * units + tiles, ctas);
    const int4 row = a.rows[m];
    float top = -INFINITY, l = 0.0f, acc[DIMS] = {};
    // n parts of n_rows query rows (a lane finds its own by `find`: nullptr where it is none; which of the rows)
    auto gather = [&](int n, int n_rows, auto find) {
        for (int i0 = 32 * warp; i0 < n; i0 += 32 * kJoinWarps) {
            const float* part = nullptr;
            int r = 0;
            if (i0 + lane < n) part = find(i0 + lane, r);
            float2 ml = make_float2(-INFINITY, 0.0f);
            if (part) ml = *reinterpret_cast<const float2*>(part + (size_t)n_rows * D + 2 * r);
            const float* mine = part ? part + 4 * r : nullptr;
            float most = ml.x;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
            const float now = fmaxf(top, most), f0 = top == -INFINITY ? 0.0f : ex2(top - now);
            // (a part whose scores are all NaN has a sum that is NaN and no maximum)
            const float f = ml.x == -INFINITY ? (ml.y == ml.y ? 0.0f : NAN) : ex2(ml.x - now);
            float sum = ml.y * f;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            l = l * f0 + sum;
            top = now;
#pragma unroll
            for (int e = 0; e < DIMS; ++e) acc[e] *= f0;
            unsigned have = __ballot_sync(0xffffffffu, mine != nullptr && !(f == 0.0f));
            while (have) {
                float v[AT_ONCE][DIMS], g[AT_ONCE];
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) {
                    const int src = have ? __ffs((int)have) - 1 : 0;
                    const float* p = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, (unsigned long long)mine, src));
                    g[k] = have ? __shfl_sync(0xffffffffu, f, src) : 0.0f;
                    if (have) {
                        if constexpr (DIMS == 4) *reinterpret_cast<float4*>(v[k]) = *reinterpret_cast<const float4*>(p + (size_t)(4 * lane) * n_rows);
                        else *reinterpret_cast<float2*>(v[k]) = *reinterpret_cast<const float2*>(p + (size_t)(4 * (lane >> 1)) * n_rows + 2 * (lane & 1));
                    } else {
#pragma unroll
                        for (int e = 0; e < DIMS; ++e) v[k][e] = 0.0f;
                    }
                    have &= have - 1;
                }
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
                    for (int e = 0; e < DIMS; ++e) acc[e] = fmaf(v[k][e], g[k], acc[e]);
            }
        }
    };
    if (row.z >= 0 && row.x > 0) {
        const int in_group = m * a.group + j - row.w, pair = row.z + in_group / (2 * kTile), r0 = in_group % (2 * kTile);
        const int4 info = a.pairs[pair];
        const bool two = info.y > kTile;
        const int4 where = a.item_ctas[pair * a.n_kv + h];  // its first unit, the first and last CTA that have some of it
        const int u0 = where.x, c0 = where.y, c1 = where.z;
        gather((c1 - c0 + 1) * (two ? 1 : 2), kTile, [&](int i, int& r) -> const float* {
            const int c = c0 + (two ? i : i >> 1), s = two ? r0 / kTile : i & 1;
            r = r0 % kTile;
            if (!two || runs.each < 2) {
                const Share share(runs, units, c);
                if (share.w0 >= share.w1) return nullptr;                                                      // (a CTA with one place may have the second half of a unit's)
                if (!two && s == 1 && (2 * max(share.w0 - u0, 0) + 1) * kTile >= info.w) return nullptr;  // the second stream had no tile
            }
            return a.parts_w + ((size_t)(pair * a.n_kv + h + c) * 2 + s) * part_floats(kTile, D);
        });
    }
    if (row.y > row.x) {
        const int n = (a.cum_rows[m + 1] - a.cum_rows[m]) / a.n_kv - 1, t0 = a.cum_rows[m] + h * (n + 1) + 1;
        auto worker = [&](int t) {
            const int c = runs.owner(2 * units + t);
            return 2 * c + (t >= Share(runs, units, c).middle() ? 1 : 0);
        };
        const int first = worker(t0), last = worker(t0 + n - 1);
        gather(last - first + 1, a.group, [&](int i, int& r) -> const float* {
            const int k = first + i;
            r = j;
            const Share share(runs, units, k >> 1);
            if (((k & 1) ? share.s1 - share.middle() : share.middle() - share.s0) <= 0) return nullptr;  // (the second stream of a CTA with one tile)
            return a.parts_s + (size_t)(m * a.n_kv + h + k) * part_floats(a.group, D);
        });
    }
    if (lane == 0) joined[warp] = make_float2(top, l);
#pragma unroll
    for (int e = 0; e < DIMS; ++e) values[warp][DIMS * lane + e] = acc[e];
    __syncthreads();
    if (warp != 0) return;
    float most = top;
#pragma unroll
    for (int k = 1; k < kJoinWarps; ++k) most = fmaxf(most, joined[k].x);
    const float f0 = top == -INFINITY ? (l == l ? 0.0f : NAN) : ex2(top - most);
    l *= f0;
#pragma unroll
    for (int e = 0; e < DIMS; ++e) acc[e] *= f0;
#pragma unroll
    for (int k = 1; k < kJoinWarps; ++k) {
        const float2 o = joined[k];
        const float f = o.x == -INFINITY ? (o.y == o.y ? 0.0f : NAN) : ex2(o.x - most);
        l = fmaf(o.y, f, l);
#pragma unroll
        for (int e = 0; e < DIMS; ++e) acc[e] = fmaf(values[k][DIMS * lane + e], f, acc[e]);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // no row: zeros; a sum that is NaN stays one
    uint32_t out[DIMS / 2];
#pragma unroll
    for (int e = 0; e < DIMS; e += 2) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(acc[e] * inv, acc[e + 1] * inv);
        out[e / 2] = *reinterpret_cast<const uint32_t*>(&b);
    }
    __nv_bfloat16* dst = a.out + (size_t)item * D + DIMS * lane;
    if constexpr (DIMS == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(out[0], out[1]);
    else *reinterpret_cast<uint32_t*>(dst) = out[0];
}

// The same for many rows: a warp takes all query heads of a row and KV head, which have the same parts, so that what leads to them is looked up once (a warp to a
// query head: 27 us for 2173 rows of 20 heads).
template <int D>
__global__ void __launch_bounds__(128) shared_combine_rows_kernel(const SharedArgs a, int ctas) {
    constexpr int DIMS = D / 32, HEADS = 4;  // query heads at a time
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int item = (int)blockIdx.x * 4 + warp, m = item / a.n_kv, h = item - m * a.n_kv;
    if (m >= a.M) return;
    const int4 row = a.rows[m];
    const int units = a.totals[1], tiles = a.totals[2];
    const EqualRuns runs(2 * units + tiles, ctas);
    const int c_row0 = a.cum_rows[m], c_row1 = a.cum_rows[m + 1];
    for (int j0 = 0, nj; j0 < a.group; j0 += nj) {
        // heads j0 .. j0 + nj - 1: of one pair of query tiles, and of one tile
        nj = min(HEADS, a.group - j0);
        int r0 = 0, pair = 0;
        const bool shares = row.z >= 0 && row.x > 0;
        if (shares) {
            const int in_group = m * a.group + j0 - row.w;
            pair = row.z + in_group / (2 * kTile), r0 = in_group % (2 * kTile);
            nj = min(nj, kTile - r0 % kTile);
        }
        float top[HEADS], l[HEADS], acc[HEADS][DIMS];
#pragma unroll
        for (int k = 0; k < HEADS; ++k) {
            top[k] = -INFINITY, l[k] = 0.0f;
#pragma unroll
            for (int e = 0; e < DIMS; ++e) acc[k][e] = 0.0f;
        }
        auto gather = [&](int n, int n_rows, int first_row, auto find) {
            for (int i0 = 0; i0 < n; i0 += 32) {
                const float* part = i0 + lane < n ? find(i0 + lane) : nullptr;
                float2 ml[HEADS];
                float f[HEADS];
#pragma unroll
                for (int k = 0; k < HEADS; ++k) ml[k] = part && k < nj ? *reinterpret_cast<const float2*>(part + (size_t)n_rows * D + 2 * (first_row + k)) : make_float2(-INFINITY, 0.0f);
#pragma unroll
                for (int k = 0; k < HEADS; ++k) {
                    float most = ml[k].x;
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
                    const float now = fmaxf(top[k], most), f0 = top[k] == -INFINITY ? 0.0f : ex2(top[k] - now);
                    f[k] = ml[k].x == -INFINITY ? (ml[k].y == ml[k].y ? 0.0f : NAN) : ex2(ml[k].x - now);
                    float sum = ml[k].y * f[k];
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
                    l[k] = l[k] * f0 + sum;
                    top[k] = now;
#pragma unroll
                    for (int e = 0; e < DIMS; ++e) acc[k][e] *= f0;
                }
                for (unsigned left = __ballot_sync(0xffffffffu, part != nullptr); left; left &= left - 1) {
                    const int src = __ffs((int)left) - 1;
                    const float* p = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, (unsigned long long)part, src));
                    float v[HEADS][DIMS];
#pragma unroll
                    for (int k = 0; k < HEADS; ++k) {
                        const float* at = p + 4 * (size_t)(first_row + min(k, nj - 1));
                        if constexpr (DIMS == 4) *reinterpret_cast<float4*>(v[k]) = *reinterpret_cast<const float4*>(at + (size_t)(4 * lane) * n_rows);
                        else *reinterpret_cast<float2*>(v[k]) = *reinterpret_cast<const float2*>(at + (size_t)(4 * (lane >> 1)) * n_rows + 2 * (lane & 1));
                    }
#pragma unroll
                    for (int k = 0; k < HEADS; ++k) {
                        const float w = __shfl_sync(0xffffffffu, f[k], src);
#pragma unroll
                        for (int e = 0; e < DIMS; ++e) acc[k][e] = w == 0.0f ? acc[k][e] : fmaf(v[k][e], w, acc[k][e]);  // (what weighs nothing may hold anything)
                    }
                }
            }
        };
        if (shares) {
            const int4 info = a.pairs[pair], where = a.item_ctas[pair * a.n_kv + h];  // its first unit, the first and last CTA that have some of it
            const bool two = info.y > kTile;
            gather((where.z - where.y + 1) * (two ? 1 : 2), kTile, r0 % kTile, [&](int i) -> const float* {
                const int c = where.y + (two ? i : i >> 1), s = two ? r0 / kTile : i & 1;
                if (!two || runs.each < 2) {
                    const Share share(runs, units, c);
                    if (share.w0 >= share.w1) return nullptr;
                    if (!two && s == 1 && (2 * max(share.w0 - where.x, 0) + 1) * kTile >= info.w) return nullptr;
                }
                return a.parts_w + ((size_t)(pair * a.n_kv + h + c) * 2 + s) * part_floats(kTile, D);
            });
        }
        if (row.y > row.x) {
            const int n = (c_row1 - c_row0) / a.n_kv - 1, t0 = c_row0 + h * (n + 1) + 1;
            auto worker = [&](int t) {
                const int c = runs.owner(2 * units + t);
                return 2 * c + (t >= Share(runs, units, c).middle() ? 1 : 0);
            };
            const int first = worker(t0), last = worker(t0 + n - 1);
            gather(last - first + 1, a.group, j0, [&](int i) -> const float* {
                const int k = first + i;
                const Share share(runs, units, k >> 1);
                if (((k & 1) ? share.s1 - share.middle() : share.middle() - share.s0) <= 0) return nullptr;
                return a.parts_s + (size_t)(m * a.n_kv + h + k) * part_floats(a.group, D);
            });
        }
#pragma unroll
        for (int k = 0; k < HEADS; ++k) {
            if (k >= nj) break;
            const float inv = l[k] == 0.0f ? 0.0f : 1.0f / l[k];  // no row: zeros; a sum that is NaN stays one
            uint32_t out[DIMS / 2];
#pragma unroll
            for (int e = 0; e < DIMS; e += 2) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(acc[k][e] * inv, acc[k][e + 1] * inv);
                out[e / 2] = *reinterpret_cast<const uint32_t*>(&b);
            }
            __nv_bfloat16* dst = a.out + ((size_t)m * a.n_q + (size_t)h * a.group + j0 + k) * D + DIMS * lane;
            if constexpr (DIMS == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(out[0], out[1]);
            else *reinterpret_cast<uint32_t*>(dst) = out[0];
        }
    }
}

// ---------------------------------------------------------------------------------------------- host side

SharedLayout shared_layout(int M, int n_groups, int n_q, int n_kv, int D) {
    SharedLayout l;
    const int group = n_q / n_kv;
    l.max_pairs = (int)((long long)M * group / (2 * kTile)) + std::min(n_groups, M / 2);  // groups of one row have none
    size_t at = 0;
    auto room = [&](size_t bytes) {
        const size_t here = at;
        at = align_up(at + bytes, 256);
        return here;
    };
    l.rows = room((size_t)M * sizeof(int4));
    l.pairs = room((size_t)l.max_pairs * sizeof(int4));
    l.cum_pairs = room(((size_t)std::max(l.max_pairs, n_groups) + 1) * sizeof(int));
    l.cum_rows = room(((size_t)M + 1) * sizeof(int));
    l.starts = room(((size_t)n_groups + 1) * sizeof(int));
    l.pair_rows = room((size_t)l.max_pairs * sizeof(int));
    l.item_ctas = room((size_t)l.max_pairs * n_kv * sizeof(int4));
    l.totals = room(3 * sizeof(int));
    l.parts_w = room(l.max_pairs == 0 ? 0 : ((size_t)l.max_pairs * n_kv + kSharedCtas) * 2 * part_floats(kTile, D) * sizeof(float));
    l.parts_s = room(((size_t)M * n_kv + 2 * kSharedCtas) * part_floats(group, D) * sizeof(float));
    l.total = at;
    return l;
}

bool shared_sizes_ok(int M, int n_groups, int n_q, int n_kv, int hd) {
    return M >= 0 && M <= 65535 && n_groups >= 0 && n_groups <= 65535 && n_q > 0 && n_kv > 0 && n_q % n_kv == 0 && n_q / n_kv <= 8 && (hd == 64 || hd == 128) && n_kv <= 65535 && (long long)M * n_q < (1ll << 30);
}

// rows = every (block, head, row) of the pool, columns = D bytes; a box is a block's rows, swizzled by the row's width
bool make_block_map(CUtensorMap* map, const void* pool, long long rows, int hd, int block_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)hd, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)hd};
    const cuuint32_t box[2] = {(cuuint32_t)hd, (cuuint32_t)block_rows};
    const cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(pool), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              hd == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int KIND>
int shared_launch(const CUtensorMap& map_k, const CUtensorMap& map_v, const SharedArgs& a, int ctas, cudaStream_t st) {
    constexpr uint32_t kBytes = SharedSmem<D>::total;
    static_assert(kBytes <= 227 * 1024, "shared memory");
    static std::mutex mu;
    static bool done[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return finish(cudaErrorInvalidDevice);
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!done[dev]) {
            if (cudaFuncSetAttribute(shared_attention_kernel<D, KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kBytes) != cudaSuccess) return finish(cudaErrorUnknown);
            // the warps' register split waits for ever unless the launch brings all of it
            cudaFuncAttributes attr;
            if (cudaFuncGetAttributes(&attr, shared_attention_kernel<D, KIND>) != cudaSuccess || attr.numRegs * kThreads < 256 * kSoftmaxRegs + (kThreads - 256) * kOtherRegs)
                return finish(cudaErrorUnknown);
            done[dev] = true;
        }
    }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3(1);
    cfg.blockDim = dim3(kPlanThreads);
    if (const int rc = finish(cudaLaunchKernelEx(&cfg, shared_plan_kernel, a, ctas))) return rc;
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kBytes;
    if (const int rc = finish(cudaLaunchKernelEx(&cfg, shared_attention_kernel<D, KIND>, map_k, map_v, a))) return rc;
    // four warps per query head; one per row and KV head where there are thousands of rows, which have few parts each (2173 rows: 27 us with a warp per query head, 22 so;
    // but 144 rows of six groups 17 and 25)
    const long long heads = (long long)a.M * a.n_q, items = (long long)a.M * a.n_kv;
    cfg.blockDim = dim3(32 * kJoinWarps);
    cfg.dynamicSmemBytes = 0;
    if (heads >= 128ll * ctas) {
        cfg.gridDim = dim3((unsigned)((items + 3) / 4));
        return finish(cudaLaunchKernelEx(&cfg, shared_combine_rows_kernel<D>, a, ctas));
    }
    cfg.gridDim = dim3((unsigned)heads);
    return finish(cudaLaunchKernelEx(&cfg, shared_combine_kernel<D>, a, ctas));
}

}  // namespace

}  // namespace bitlinear

using namespace bitlinear;

extern "C" {

size_t bitlinear_attention_shared_kv8_workspace_bytes(int M, int n_groups, int n_q_heads, int n_kv_heads, int head_dim) {
    return shared_sizes_ok(M, n_groups, n_q_heads, n_kv_heads, head_dim) ? shared_layout(M, n_groups, n_q_heads, n_kv_heads, head_dim).total : 0;
}

int bitlinear_attention_shared_kv8(const void* q_bf16, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale, const int32_t* tables,
                                   const int32_t* lengths, const int32_t* seq_ids, const int32_t* group_starts, const int32_t* shared_rows, int M, int n_groups, int n_q_heads,
                                   int n_kv_heads, int head_dim, int kv_dtype, int n_blocks, int block_rows, int n_seq, int max_blocks, void* out_bf16, void* ws, size_t ws_bytes,
                                   void* stream) {
    if (kv_dtype != BITLINEAR_KV_INT8 && kv_dtype != BITLINEAR_KV_E4M3) return BITLINEAR_ERR_DTYPE;
    if (!shared_sizes_ok(M, n_groups, n_q_heads, n_kv_heads, head_dim) || n_seq <= 0 || max_blocks <= 0 ||
        !kv8_dims_ok(n_q_heads, n_kv_heads, head_dim, kv_dtype, n_blocks, block_rows) || (long long)max_blocks * block_rows > (1ll << 30) || (!seq_ids && n_seq < M) ||
        (double)M * n_kv_heads * ((double)max_blocks * block_rows / kTile + 4) * 2 > 2147483000.0)
        return BITLINEAR_ERR_SHAPE;
    if (M == 0) return BITLINEAR_OK;
    if (!q_bf16 || !k_cache || !v_cache || !k_scale || !v_scale || !tables || !lengths || !group_starts || (n_groups > 0 && !shared_rows) || !out_bf16) return BITLINEAR_ERR_NULL;
    if (!aligned16(q_bf16) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out_bf16)) return BITLINEAR_ERR_ALIGN;
    const SharedLayout l = shared_layout(M, n_groups, n_q_heads, n_kv_heads, head_dim);
    if (!ws || !aligned16(ws) || ws_bytes < l.total) return BITLINEAR_ERR_WORKSPACE;
    int sm_count = 0;
    if (const int rc = device_sm_count(&sm_count)) return rc;
    const long long pool_rows = (long long)n_blocks * n_kv_heads * block_rows;
    CUtensorMap map_k, map_v;
    if (!make_block_map(&map_k, k_cache, pool_rows, head_dim, block_rows) || !make_block_map(&map_v, v_cache, pool_rows, head_dim, block_rows)) return BITLINEAR_ERR_CUDA;
    uint8_t* w = static_cast<uint8_t*>(ws);
    SharedArgs a = {static_cast<const __nv_bfloat16*>(q_bf16), k_scale, v_scale, tables, lengths, seq_ids, group_starts, shared_rows, M, n_groups, n_q_heads, n_kv_heads,
                    n_q_heads / n_kv_heads, n_seq, max_blocks, log2_of(block_rows), n_blocks, 1.4426950408889634f / sqrtf((float)head_dim), static_cast<__nv_bfloat16*>(out_bf16),
                    reinterpret_cast<int4*>(w + l.rows), reinterpret_cast<int4*>(w + l.pairs), reinterpret_cast<int*>(w + l.cum_pairs), reinterpret_cast<int*>(w + l.cum_rows),
                    reinterpret_cast<int*>(w + l.starts), reinterpret_cast<int*>(w + l.pair_rows), reinterpret_cast<int4*>(w + l.item_ctas), reinterpret_cast<int*>(w + l.totals), reinterpret_cast<float*>(w + l.parts_w), reinterpret_cast<float*>(w + l.parts_s),
                    l.max_pairs, device_status_word()};
    const int ctas = std::min(sm_count, kSharedCtas);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (head_dim == 128)
        return kv_dtype == BITLINEAR_KV_INT8 ? shared_launch<128, BITLINEAR_KV_INT8>(map_k, map_v, a, ctas, st) : shared_launch<128, BITLINEAR_KV_E4M3>(map_k, map_v, a, ctas, st);
    return kv_dtype == BITLINEAR_KV_INT8 ? shared_launch<64, BITLINEAR_KV_INT8>(map_k, map_v, a, ctas, st) : shared_launch<64, BITLINEAR_KV_E4M3>(map_k, map_v, a, ctas, st);
}

}  // extern "C"
