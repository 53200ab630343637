// A paged key/value cache held in 8 bits with one scale per block of rows and KV head: the append (rotary embedding and
// quantisation) and grouped-query decode attention over it.
//
// Layout: pools [n_blocks][n_kv][block_rows][D] of codes (int8, or e4m3 floats), scales fp32 [n_blocks][n_kv]; a row's value is
// code * scale.  A (block, head) tile is contiguous, so attention fetches it with one tensor-map copy.
#include "common.cuh"
#include "sm100_sync.cuh"
#include "tensor_map.cuh"

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <mutex>
#include <type_traits>

namespace bitlinear {

namespace {

// ---------------------------------------------------------------------------------------------- append

constexpr int kAppendThreads = 128;
constexpr double kAmaxFloor = 1e-30;  // below this a block counts as all zero

// The scale a block with this largest magnitude needs.  int8: amax / 127, rounded once.  e4m3: the smallest power of two whose
// 448-fold is no less than amax - the codes are floating point, so a finer scale would gain nothing, and bringing
// codes to a larger power of two is exact but for the subnormal ones.
template <int KIND>
__device__ __forceinline__ float scale_for(double amax) {
    amax = fmax(amax, kAmaxFloor);
    if constexpr (KIND == BITLINEAR_KV_INT8) return (float)__ddiv_rn(amax, 127.0);
    const int hi = __double2hiint(amax);
    int k = (hi >> 20) - 1023 - 8;  // amax = f * 2^(k + 8), 448 = 1.75 * 2^8
    const double f = __hiloint2double((hi & 0x000fffff) | 0x3ff00000, __double2loint(amax));
    if (f > 1.75) ++k;
    return __int_as_float(min(k + 127, 254) << 23);
}

// The code nearest to value / scale, ties to even, decided on the quotient in 64 bits: in 32 the rotation's and the quotient's
// own roundings move about one code in a million across the middle between two.
// e4m3: the scale is a power of two, so the quotient is exact; it goes to fp32 with the last bit sticky (round to odd),
// and the conversion to e4m3 then rounds as if it saw all bits.
template <int KIND>
__device__ __forceinline__ uint32_t code_of(double value, double scale) {
    const double x = __ddiv_rn(value, scale);
    if constexpr (KIND == BITLINEAR_KV_INT8) return (uint32_t)(int)fmin(fmax(rint(x), -127.0), 127.0) & 0xffu;
    float f = __double2float_rz(x);
    if ((double)f != x) f = __int_as_float(__float_as_int(f) | 1);
    return (uint32_t)__nv_cvt_float_to_fp8(f, __NV_SATFINITE, __NV_E4M3);
}
// The same from an fp32 value and the reciprocal of the scale; false where they cannot tell: next to the middle between two codes.
// `off` bounds the error of value * inv.  For keys a rotated pair's components are at most sqrt 2 of the block's largest magnitude
// before the turn, two products and a sum round by 2^-24 each, and that magnitude is at most 127 (448) steps: 6e-5 (2.1e-4) with the
// reciprocal's and the product's own rounding.  Values come as they are: 2.3e-5 (5.4e-5, and none where the scale is a power of two, as it
// is unless something else wrote the block's first rows).
template <int KIND>
__device__ __forceinline__ float quick_error(bool keys) {
    return KIND == BITLINEAR_KV_INT8 ? (keys ? 1e-4f : 4e-5f) : (keys ? 3e-4f : 1e-4f);
}
// Eight codes in two words; false if one of them cannot be told.  int8: adding 1.5 * 2^23 rounds to the nearest whole number, ties to even, and
// leaves it in the low bits (no value is more than 127 steps: the scale is what the largest needs, or more).  e4m3: both ends of the
// error are converted, two values to an instruction.
template <int KIND>
__device__ __forceinline__ bool quick_codes(const float (&x)[8], float inv, float off, uint32_t (&word)[2]) {
    if constexpr (KIND == BITLINEAR_KV_INT8) {
        constexpr float kRound = 12582912.0f;
        bool sure = true;
        uint32_t t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float y = fmaf(x[e], inv, kRound);
            sure = sure && fabsf(fmaf(x[e], inv, kRound - y)) < 0.5f - off;
            t[e] = __float_as_uint(y);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) word[h] = __byte_perm(__byte_perm(t[4 * h], t[4 * h + 1], 0x0040), __byte_perm(t[4 * h + 2], t[4 * h + 3], 0x0040), 0x5410);
        return sure;
    } else {
        uint32_t differ = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t low[2], high[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float a = x[4 * h + 2 * j] * inv, b = x[4 * h + 2 * j + 1] * inv;
                low[j] = __nv_cvt_float2_to_fp8x2(make_float2(a - off, b - off), __NV_SATFINITE, __NV_E4M3);
                high[j] = __nv_cvt_float2_to_fp8x2(make_float2(a + off, b + off), __NV_SATFINITE, __NV_E4M3);
            }
            word[h] = __byte_perm(low[0], low[1], 0x5410);
            differ |= word[h] ^ __byte_perm(high[0], high[1], 0x5410);
        }
        return differ == 0;
    }
}
// int8, where some value of a row is next to the middle between two codes: the value in fp64 against the middle nearest to its
// approximate quotient, times the scale (exact), instead of a division
template <int KIND>
__device__ __forceinline__ uint32_t close_code(double value, float inv, double scale) {
    const float low = floorf((float)(value * (double)inv));  // the middle above it is the only one within 0.5
    const double gap = value - ((double)low + 0.5) * scale;
    const int c = (int)low + (gap > 0.0 || (gap == 0.0 && ((int)low & 1)) ? 1 : 0);
    return (uint32_t)min(max(c, -127), 127) & 0xffu;
}
template <int KIND>
__device__ __forceinline__ double decoded(uint32_t code) {
    if constexpr (KIND == BITLINEAR_KV_INT8) return (double)(int)(int8_t)code;
    const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3);
    return (double)__half2float(__half(h));
}

// the larger; NaN if either is
__device__ __forceinline__ float max_nan(float x, float y) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(x), "f"(y));
    return m;
}

struct AppendArgs {
    const float* q;
    const float* k;
    const float* v;
    const int* positions;
    const int* slots;
    const float2* table;
    int T, t_max, n_q, n_kv, log2_rows, n_blocks;
    __nv_bfloat16* q_out;
    uint8_t* k_cache;
    uint8_t* v_cache;
    float* k_scale;
    float* v_scale;
    int tile;       // tokens per CTA of the key/value part
    int kv_ctas;    // CTAs of the key/value part; those behind it rotate q
};

// eight values of a row: four dims from i4 on and their rotation partners, with the angles' (cos, sin)
template <int D>
struct RowValues {
    float l[4], u[4], c[4], s[4];
    __device__ __forceinline__ void load(const float* row, int i4) {
        const float4 lo = *reinterpret_cast<const float4*>(row + i4), hi = *reinterpret_cast<const float4*>(row + i4 + D / 2);
        l[0] = lo.x, l[1] = lo.y, l[2] = lo.z, l[3] = lo.w;
        u[0] = hi.x, u[1] = hi.y, u[2] = hi.z, u[3] = hi.w;
    }
    __device__ __forceinline__ void load_angles(const float2* table, int pos, int i4) {
        const float4* cs = reinterpret_cast<const float4*>(table + (size_t)pos * (D / 2) + i4);
        const float4 c0 = cs[0], c1 = cs[1];
        c[0] = c0.x, c[1] = c0.z, c[2] = c1.x, c[3] = c1.z;
        s[0] = c0.y, s[1] = c0.w, s[2] = c1.y, s[3] = c1.w;
    }
    // the fp32 operations of the other append calls, in their order
    __device__ __forceinline__ void turned(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = __fsub_rn(__fmul_rn(l[e], c[e]), __fmul_rn(u[e], s[e]));
            x[4 + e] = __fadd_rn(__fmul_rn(u[e], c[e]), __fmul_rn(l[e], s[e]));
        }
    }
    // one of them in fp64, where the products are exact
    __device__ __forceinline__ double exact(int e) const {
        const int j = e & 3;
        return e < 4 ? __dsub_rn((double)l[j] * (double)c[j], (double)u[j] * (double)s[j]) : __dadd_rn((double)u[j] * (double)c[j], (double)l[j] * (double)s[j]);
    }
};

// Key/value part: one CTA per (tile of tokens, KV head, keys or values).  The tokens of one block stand next to each other in a
// call; the first of such a run leads it: its CTA finds the run's largest magnitude, settles the block's scale
// (scale = max(old, needed) where the block has rows in front of the run, else what is needed), brings the earlier rows' codes
// to the new scale if it grew, and writes the run's codes.  So a block's scale has one writer and no atomics.
// The result is that of fp64 arithmetic, the work mostly fp32: only values next to the largest, and next to the middle between two
// codes, are formed again in fp64.  16,500 tokens of 20 + 5 heads of 128: 82 us, 4.4 TB/s of the bytes it cannot do without (all in
// fp64 130 us); the queries' half alone takes 34 us (part of what it writes is still in L2 then), this half waits on its chain of
// loads (run, positions, rows, scale).
// Tried and slower: more rows per thread in flight, 256 threads, alternating the two kinds of CTA.  One token of 16 sequences:
// 4.4 us, launch and that chain.
template <int D, int KIND>
__device__ __forceinline__ void append_run(const AppendArgs& a, int m0, int block, int h, int which) {
    constexpr int TPR = D / 8;  // threads per row
    constexpr int ROWS = kAppendThreads / TPR, WARPS = kAppendThreads / 32;
    __shared__ float red[WARPS];
    __shared__ double red_d[WARPS];
    __shared__ int first_s[WARPS];
    __shared__ float scale_s[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int sub = tid / TPR, i4 = 4 * (tid % TPR);
    const float* src = (which == 0 ? a.k : a.v) + (size_t)h * D;
    const size_t row_stride = (size_t)a.n_kv * D;
    int end = m0 + 1;
    while (end < a.T) {  // the run's end, 32 tokens at a time, the same in every warp
        const int s = end + lane < a.T ? a.slots[end + lane] : -1;
        const unsigned other = __ballot_sync(0xffffffffu, s < 0 || s >> a.log2_rows != block);
        if (other) {
            end += __ffs((int)other) - 1;
            break;
        }
        end += 32;
    }
    RowValues<D> r;
    float x[8];
    auto load = [&](int m, int pos) {
        r.load(src + (size_t)m * row_stride, i4);
        if (which == 0) {
            r.load_angles(a.table, pos, i4);
            r.turned(x);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = r.l[e], x[4 + e] = r.u[e];
        }
    };
    // the largest magnitude, in fp32 (NaN if a value is), and the run's first row in the block
    float top = 0.0f;
    int first = 1 << a.log2_rows;
#pragma unroll 2
    for (int m = m0 + sub; m < end; m += ROWS) {
        const int pos = a.positions[m];
        if (pos < 0 || pos >= a.t_max) continue;
        load(m, pos);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max_nan(top, fabsf(x[e]));
        first = min(first, a.slots[m] - (block << a.log2_rows));
    }
    const float own_top = top;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, off));
        first = min(first, __shfl_xor_sync(0xffffffffu, first, off));
    }
    if (lane == 0) red[warp] = top, first_s[warp] = first;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = max_nan(top, red[w]), first = min(first, first_s[w]);
    if (first >> a.log2_rows) {  // no token of the run has a place in the table of angles
        __syncthreads();
        return;
    }
    if (which == 0) {  // keys: the largest in fp64 is among those within the fp32 errors of the largest in fp32
        double amax = 0.0;
        const float near = top * (1.0f - 1.0f / 524288.0f);
        if (own_top >= near) {
            for (int m = m0 + sub; m < end; m += ROWS) {
                const int pos = a.positions[m];
                if (pos < 0 || pos >= a.t_max) continue;
                load(m, pos);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (fabsf(x[e]) >= near) amax = fmax(amax, fabs(r.exact(e)));
            }
        }
        if (__any_sync(0xffffffffu, own_top >= near)) {
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) amax = fmax(amax, __shfl_xor_sync(0xffffffffu, amax, off));
        }
        if (lane == 0) red_d[warp] = amax;
        __syncthreads();
    }
    uint8_t* tile = (which == 0 ? a.k_cache : a.v_cache) + (((size_t)block * a.n_kv + h) << a.log2_rows) * D;
    if (tid == 0) {  // the one reader and writer of the scale
        float* scale = (which == 0 ? a.k_scale : a.v_scale) + (size_t)block * a.n_kv + h;
        double amax = (double)top;
        if (which == 0 && top == top) {
            amax = red_d[0];
#pragma unroll
            for (int w = 1; w < WARPS; ++w) amax = fmax(amax, red_d[w]);
        }
        // a value that is not finite leaves the block without a scale until its first row is written again: what reads it gets NaN
        const float need = amax < (double)INFINITY ? scale_for<KIND>(amax) : NAN, old = first > 0 ? *scale : need;
        const float now = first > 0 ? max_nan(old, need) : need;
        *scale = now;
        scale_s[0] = old, scale_s[1] = now;
    }
    __syncthreads();
    const float old = scale_s[0], now = scale_s[1];
    const double s = (double)now;
    const float inv = __frcp_rn(now), off = quick_error<KIND>(which == 0);
    const bool overflow = !(top < INFINITY);  // a rotated value beyond fp32
    const bool broken = now != now;
#pragma unroll 2
    for (int m = m0 + sub; m < end; m += ROWS) {
        const int pos = a.positions[m];
        if (pos < 0 || pos >= a.t_max) continue;
        load(m, pos);
        uint32_t word[2];
        if (broken || overflow || !quick_codes<KIND>(x, inv, off, word)) {
            word[0] = word[1] = 0u;
#pragma unroll
            for (int e = 0; e < 8 && !broken; ++e) {
                const double value = which == 0 ? r.exact(e) : (double)x[e];
                word[e >> 2] |= (KIND == BITLINEAR_KV_INT8 ? close_code<KIND>(value, inv, s) : code_of<KIND>(value, s)) << (8 * (e & 3));
            }
        }
        uint8_t* dst = tile + (size_t)(a.slots[m] - (block << a.log2_rows)) * D;
        *reinterpret_cast<uint32_t*>(dst + i4) = word[0];
        *reinterpret_cast<uint32_t*>(dst + i4 + D / 2) = word[1];
    }
    if (first > 0 && now > old) {
        uint32_t* words = reinterpret_cast<uint32_t*>(tile);
        for (int i = tid; i < first * (D / 4); i += kAppendThreads) {
            const uint32_t w = words[i];
            uint32_t v = 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) v |= code_of<KIND>(decoded<KIND>((w >> (8 * e)) & 0xffu) * (double)old, s) << (8 * e);
            words[i] = v;
        }
    }
}

template <int D, int KIND>
__global__ void __launch_bounds__(kAppendThreads) rope_kv8_kernel(const AppendArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if ((int)blockIdx.x < a.kv_ctas) {
        const int n_slots = a.n_blocks << a.log2_rows, lane = threadIdx.x & 31;
        const int item = blockIdx.x % (2 * a.n_kv), t0 = (int)(blockIdx.x / (2 * a.n_kv)) * a.tile;
        // the blocks of the tile's tokens (at most 31) and of the one in front, one per lane; a token leads a run if its block is another
        // than that of the token in front
        const int m = t0 - 1 + lane;
        const int s = m >= 0 && m < a.T && lane <= a.tile ? a.slots[m] : -1;
        const int block = s >= 0 && s < n_slots ? s >> a.log2_rows : -1;
        const int front = __shfl_up_sync(0xffffffffu, block, 1);
        unsigned leads = __ballot_sync(0xffffffffu, lane > 0 && block >= 0 && block != front);
        for (; leads; leads &= leads - 1) {
            const int at = __ffs((int)leads) - 1;
            append_run<D, KIND>(a, t0 - 1 + at, __shfl_sync(0xffffffffu, block, at), item >> 1, item & 1);
        }
    } else {
        // rotated queries, a token at a time; a thread's dims are the same in every head that it meets, so the angles are read once
        constexpr int UNITS = D / 8;
        static_assert(kAppendThreads % UNITS == 0, "a thread keeps its dims from head to head");
        const int i4 = 4 * (threadIdx.x % UNITS), units = a.n_q * UNITS;
        const int step = gridDim.x - a.kv_ctas;
        int m = blockIdx.x - a.kv_ctas, pos = m < a.T ? a.positions[m] : -1;
        for (; m < a.T; m += step) {
            const bool placed = pos >= 0 && pos < a.t_max;  // a row without a position: zeros
            RowValues<D> r;
            if (placed) r.load_angles(a.table, pos, i4);
            if (m + step < a.T) pos = a.positions[m + step];
            const float* row = a.q + (size_t)m * a.n_q * D + i4;
            __nv_bfloat16* out = a.q_out + (size_t)m * a.n_q * D + i4;
            for (int u0 = threadIdx.x; u0 < units; u0 += 3 * kAppendThreads) {
                float4 lo[3], hi[3];
#pragma unroll
                for (int j = 0; j < 3; ++j) {
                    const float* src = row + (size_t)(min(u0 + j * kAppendThreads, units - 1) / UNITS) * D;
                    lo[j] = __ldcs(reinterpret_cast<const float4*>(src));
                    hi[j] = __ldcs(reinterpret_cast<const float4*>(src + D / 2));
                }
#pragma unroll
                for (int j = 0; j < 3; ++j) {
                    const int u = u0 + j * kAppendThreads;
                    if (u >= units) break;
                    uint2 lo2 = make_uint2(0u, 0u), hi2 = lo2;
                    if (placed) {
                        float x[8];
                        r.l[0] = lo[j].x, r.l[1] = lo[j].y, r.l[2] = lo[j].z, r.l[3] = lo[j].w;
                        r.u[0] = hi[j].x, r.u[1] = hi[j].y, r.u[2] = hi[j].z, r.u[3] = hi[j].w;
                        r.turned(x);
                        auto pair = [](float p, float q) {
                            const __nv_bfloat162 b = __floats2bfloat162_rn(p, q);
                            return *reinterpret_cast<const uint32_t*>(&b);
                        };
                        lo2 = make_uint2(pair(x[0], x[1]), pair(x[2], x[3]));
                        hi2 = make_uint2(pair(x[4], x[5]), pair(x[6], x[7]));
                    }
                    *reinterpret_cast<uint2*>(out + (size_t)(u / UNITS) * D) = lo2;
                    *reinterpret_cast<uint2*>(out + (size_t)(u / UNITS) * D + D / 2) = hi2;
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- decode attention

// cache rows a warp takes at a time: 8 KB of codes either way (32 rows of 64 dims, half of that, left the copy rate at 3.4 TB/s: a unit's fixed
// cost - issuing, softmax statistics - was as long as its arithmetic)
constexpr int unit_rows(int D) { return D == 64 ? 64 : 32; }
constexpr int kMinUnit = 32;
constexpr int kMaxCtas = 160;    // one CTA per SM; partial results are reserved for this many
constexpr int kMaxStages = 8;

// One (row, KV head) pair is the work of one softmax.  All units of all pairs, in the order (row, head, unit), are cut into equal
// runs, one per warp of the grid, so that a batch of any lengths loads every SM alike.  A run covers pairs in whole
// (finished by the warp) and at most two in part; those meet in shared memory with the neighbouring warps' and,
// where a pair reaches beyond the CTA, in global memory, where a second launch merges them.  A pair counts for one place
// more than it has units: starting and ending it takes a warp about as long as a unit does, and without that place the warps
// that meet many short sequences finished last (by a sixth of the time of a batch of 97 sequences of 1 to 16,384 rows).
// Bound: the bytes of the cache while the rings are full - a batch of 97 such sequences (246 MB) takes 51.5 us, 4.8 TB/s, and its
// steady part runs at the copy rate; the rest is the chain lengths -> table -> first rows in front (3 us cold), the parts' merge (1 us)
// and the second launch (2.5 us).  16 sequences of 4096 rows (e4m3) 22.8 us, one (int8) 11.1 us.  Twelve warps rather than
// eight: 78 -> 68 us at the time; keys on the integer tensor cores rather than converted were part of that step.
struct AttnArgs {
    const __nv_bfloat16* q;
    const float* k_scale;
    const float* v_scale;
    const int* tables;
    const int* lengths;
    const int* seq_ids;
    int M, n_q, n_kv, n_seq, max_blocks, log2_rows, n_blocks;
    int stages;
    float scale_log2;  // log2(e) / sqrt(D)
    __nv_bfloat16* out;
    float* part;       // [CTA][2][group * D values, then (max, sum) of each head]
    int2* desc;        // [CTA][2] (pair, last CTA that holds a part of it); pair -1: none
    int* status;
};

struct __align__(16) UnitMeta {
    int m, h;
    int flags;           // 1: first unit of this run's part of the pair, 2: last
    int unit;            // its number in the pair,
    int units;           // of how many
    int at;              // its place in the order of all
    uint32_t rows[2];    // live rows, one bit each
    float ks[4], vs[4];  // scales of each sixteen rows
};

struct __align__(16) PartHead {
    int begin, end;  // places of the pair's units in the order of all
    int m, h, used, pad[3];
    float m_run[8], l_run[8];
};

__device__ __forceinline__ int row_len(const AttnArgs& a, int m) {
    const int seq = a.seq_ids ? a.seq_ids[m] : m;
    if (seq < 0 || seq >= a.n_seq) return 0;
    return min(max(a.lengths[m], 0), a.max_blocks << a.log2_rows);
}
__device__ __forceinline__ int clamped_len(const AttnArgs& a, int seq, int len) {
    return seq < 0 || seq >= a.n_seq ? 0 : min(max(len, 0), a.max_blocks << a.log2_rows);
}
// units of a (row, head) pair: at least one, so that an empty row has someone to write its zeros
template <int UNIT>
__device__ __forceinline__ int units_of(int len) { return max(1, (len + UNIT - 1) / UNIT); }

// The order in which the rows of an eight-row group take the tensor core's row slots.  Any order is right as long as scores and
// values use the same one; in this one neither read of a swizzled tile meets a bank twice (checked for 64- and 128-byte rows).
__device__ __forceinline__ int row_of_slot(int i) { return (0x25346170 >> (4 * i)) & 7; }

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movmatrix_t16(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// 2^x to two units in the last place; results below 2^-126 are 0
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Four codes of a word -> two pairs of f16, exactly.  int8: the code plus 128 becomes the low bits of 1024 + x, and
// 1152 is taken off.  e4m3: the conversion instruction.
template <int KIND>
__device__ __forceinline__ void to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    if constexpr (KIND == BITLINEAR_KV_INT8) {
        const uint32_t u = w ^ 0x80808080u;
        const uint32_t off = 0x64806480u, l = __byte_perm(u, 0x64646464u, 0x4140), h = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 a = __hsub2(*reinterpret_cast<const __half2*>(&l), *reinterpret_cast<const __half2*>(&off));
        const __half2 b = __hsub2(*reinterpret_cast<const __half2*>(&h), *reinterpret_cast<const __half2*>(&off));
        lo = *reinterpret_cast<const uint32_t*>(&a);
        hi = *reinterpret_cast<const uint32_t*>(&b);
    } else {
        asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
    }
}

__device__ __forceinline__ void lds128(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void lds64(uint32_t addr, uint32_t (&r)[2]) {
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr));
}

__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, int row, uint32_t bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(dst),
        "l"(map), "r"(0), "r"(row), "r"(bar), "l"(policy)
        : "memory");
}

// a warp's partial result in shared memory: head, then group * D values
__host__ __device__ inline size_t part_smem(int group, int D) { return sizeof(PartHead) + (size_t)group * D * sizeof(float); }
__host__ __device__ inline size_t part_floats(int group, int D) { return (size_t)group * D + 2 * group; }

// shared memory: [rings: warp][stage][unit] [unit heads] [first parts] [barriers] [abort flag] [which second parts exist]
struct AttnSmem {
    size_t meta, parts, bars, total;
};
__host__ __device__ inline AttnSmem attn8_smem(int group, int D, int warps, int stages) {
    AttnSmem s;
    s.meta = (size_t)warps * stages * 2 * (D == 64 ? 64 : 32) * D;
    s.parts = s.meta + (size_t)warps * stages * sizeof(UnitMeta);
    s.bars = s.parts + warps * part_smem(group, D);
    s.total = s.bars + (size_t)warps * stages * 8 + 16 + (size_t)warps * 4;
    return s;
}

// the places 0 .. total - 1 in equal runs: worker w has begin(w) .. begin(w + 1) - 1
struct Runs {
    int each, more;  // the first `more` workers have one place more
    __device__ __forceinline__ Runs(int total, int workers) : each((int)((unsigned)total / (unsigned)workers)), more(total - each * workers) {}
    __device__ __forceinline__ int begin(int w) const { return w * each + min(w, more); }
    __device__ __forceinline__ int owner(int at) const {
        const int border = more * (each + 1);
        return at < border ? (int)((unsigned)at / (unsigned)(each + 1)) : more + (int)((unsigned)(at - border) / (unsigned)each);
    }
};

// a word from global memory into shared memory; the barrier is told when it has landed
__device__ __forceinline__ void copy_word(uint32_t dst, const float* src, uint32_t bar) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// NARROW: groups of at most four query heads, which leave half of the tensor core's eight columns free.
template <int D, int KIND, int WARPS, bool NARROW>
__global__ void __launch_bounds__(WARPS * 32, 1) attn_decode_kv8_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                                        const AttnArgs a) {
    constexpr int KS = D / 16;     // 16-dim tiles of the result
    constexpr int VW = D / 32;     // 32-bit words of a value row per lane
    constexpr bool INT8 = KIND == BITLINEAR_KV_INT8;
    constexpr int UNIT = D == 64 ? 64 : 32, PIECES = UNIT / 16;  // the tensor core takes sixteen rows at a time
    constexpr uint32_t kUnitBytes = 2u * UNIT * D;  // keys, then values
    extern __shared__ uint8_t attn8_raw[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, qd = lane & 3;
    const int group = a.n_q / a.n_kv, stages = a.stages;
    uint8_t* smem = attn8_raw + ((1024u - (smem_u32(attn8_raw) & 1023u)) & 1023u);
    const AttnSmem lay = attn8_smem(group, D, WARPS, stages);
    const uint32_t ring = smem_u32(smem) + (uint32_t)warp * stages * kUnitBytes;
    UnitMeta* meta = reinterpret_cast<UnitMeta*>(smem + lay.meta) + warp * stages;
    uint8_t* parts0 = smem + lay.parts;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + lay.bars);
    const uint32_t full = smem_u32(bars + warp * stages);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + WARPS * stages);
    int* second_used = const_cast<int*>(abort_flag) + 4;
    if (tid == 0) *abort_flag = 0;
    if (lane == 0) {
        for (int s = 0; s < stages; ++s) mbar_init(full + 8u * s, 1 + 2 * PIECES);  // the copies' announcement and the scales
        mbar_init_fence();
        reinterpret_cast<PartHead*>(parts0 + warp * part_smem(group, D))->used = 0;
        second_used[warp] = 0;
    }
    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __syncthreads();

    // ---- this warp's run of units.  256 rows' lengths at a time, all loads of a batch in flight at once; up to 256 rows they
    // are read once.
    constexpr int BATCH = 8;
    const int workers = gridDim.x * WARPS, me = blockIdx.x * WARPS + warp;
    int lens[BATCH];
    auto load_lens = [&](int m0) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int m = m0 + 32 * i + lane;
            lens[i] = m < a.M ? row_len(a, m) : -1;
        }
    };
    int total = 0;
    for (int m0 = 0; m0 < a.M; m0 += 32 * BATCH) {
        load_lens(m0);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) total += lens[i] >= 0 ? units_of<UNIT>(lens[i]) + 1 : 0;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
    const Runs runs(total * a.n_kv, workers);
    const int u0 = runs.begin(me), u1 = runs.begin(me + 1);
    // where the run begins: row pm (its length and units), head ph, unit p_unit of the pair, at place `next`
    int pm = a.M, ph = 0, p_len = 0, p_units = 1, p_unit = 0, next = u0;
    if (u0 < u1) {
        int base = 0;
        for (int m0 = 0; m0 < a.M && pm == a.M; m0 += 32 * BATCH) {
            if (a.M > 32 * BATCH) load_lens(m0);
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                if (pm < a.M || m0 + 32 * i >= a.M) break;
                const int n = lens[i] >= 0 ? (units_of<UNIT>(lens[i]) + 1) * a.n_kv : 0;
                int incl = n;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int up = __shfl_up_sync(0xffffffffu, incl, d);
                    if (lane >= d) incl += up;
                }
                const unsigned past = __ballot_sync(0xffffffffu, base + incl > u0);
                if (past) {
                    const int src = __ffs((int)past) - 1;
                    pm = m0 + 32 * i + src;
                    p_len = __shfl_sync(0xffffffffu, lens[i], src);
                    p_units = units_of<UNIT>(p_len);
                    const int in_row = u0 - base - __shfl_sync(0xffffffffu, incl - n, src);
                    ph = (int)((unsigned)in_row / (unsigned)(p_units + 1));
                    p_unit = in_row - ph * (p_units + 1) - 1;
                    if (p_unit < 0) p_unit = 0, ++next;  // the place that stands for the pair's start
                }
                base += __shfl_sync(0xffffffffu, incl, 31);
            }
        }
    }

    // ---- producer side: issue the next unit of the run into its ring place
    const uint64_t once = l2_evict_first_policy();
    const int rows_log2 = a.log2_rows, per_unit = max(1, UNIT >> a.log2_rows);  // blocks a unit spans
    int w_id = -1, w_base = 0, w_end = 0;  // lane l holds entry w_base + l of row pm's table, up to w_end
    int p_seq = 0, n_seq_raw = 0, n_len_raw = 0;  // the row's sequence; the next row's, fetched while this one is at work
    auto fetch_next_row = [&]() {
        if (pm + 1 < a.M) {
            n_seq_raw = a.seq_ids ? a.seq_ids[pm + 1] : pm + 1;
            n_len_raw = a.lengths[pm + 1];
        }
    };
    if (next < u1) {
        p_seq = a.seq_ids ? a.seq_ids[pm] : pm;
        fetch_next_row();
    }
    int issued = 0;
    auto issue = [&]() {
        const int place = issued % stages;
        const int b = (p_unit * UNIT) >> rows_log2;
        if (b < w_base || b + per_unit > w_end) {
            w_base = b;
            w_end = b + 32;
            const int idx = b + lane;
            w_id = ((long long)idx << rows_log2) < p_len ? a.tables[(size_t)p_seq * a.max_blocks + idx] : -1;
            if (w_id >= a.n_blocks) w_id = -1;
        }
        int id[PIECES];  // the block of each sixteen rows
#pragma unroll
        for (int i = 0; i < PIECES; ++i) id[i] = __shfl_sync(0xffffffffu, w_id, ((p_unit * UNIT + 16 * i) >> rows_log2) - w_base);
        const bool pair_end = p_unit == p_units - 1;
        const int after = next + (pair_end ? 2 : 1);
        const uint32_t bar = full + 8u * place;
        UnitMeta& w = meta[place];
        if (lane < 2 * PIECES) {  // scales: keys of every piece, then values
            const int i = lane % PIECES;
            int block = id[0];
#pragma unroll
            for (int j = 1; j < PIECES; ++j) block = i == j ? id[j] : block;
            float* dst = (lane < PIECES ? w.ks : w.vs) + i;
            const float* src = (lane < PIECES ? a.k_scale : a.v_scale) + (size_t)max(block, 0) * a.n_kv + ph;
            if (block >= 0) copy_word(smem_u32(dst), src, bar);
            else {
                *dst = 0.0f;
                mbar_arrive(bar);
            }
        }
        if (lane == 0) {
            const int live = min(max(p_len - p_unit * UNIT, 0), UNIT);
            unsigned long long rows = live == 64 ? ~0ull : (1ull << live) - 1ull;
            uint32_t there = 0;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                if (id[i] < 0) rows &= ~(0xffffull << (16 * i));
                else ++there;
            }
            *reinterpret_cast<int4*>(&w.m) = make_int4(pm, ph, (issued == 0 || p_unit == 0 ? 1 : 0) | (pair_end || after >= u1 ? 2 : 0), p_unit);
            *reinterpret_cast<int4*>(&w.units) = make_int4(p_units, next, (int)(uint32_t)rows, (int)(uint32_t)(rows >> 32));
            const uint32_t dst = ring + (uint32_t)place * kUnitBytes;
            mbar_expect_tx(bar, there * (kUnitBytes / PIECES));
            const int off = (p_unit * UNIT) & ((1 << rows_log2) - 1), step = PIECES / per_unit;  // pieces of a copy
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                if (i % step != 0 || id[i] < 0) continue;
                const int row = ((id[i] * a.n_kv + ph) << rows_log2) + (per_unit == 1 ? off : 0);
                tma_rows(dst + 16 * i * D, &map_k, row, bar, once);
                tma_rows(dst + kUnitBytes / 2 + 16 * i * D, &map_v, row, bar, once);
            }
        }
        ++issued;
        next = after;
        ++p_unit;
        if (pair_end) {  // on to the next pair
            p_unit = 0;
            if (++ph == a.n_kv) {
                ph = 0;
                w_end = 0;
                ++pm;
                p_seq = n_seq_raw;
                p_len = clamped_len(a, n_seq_raw, n_len_raw);
                p_units = units_of<UNIT>(p_len);
                if (next < u1) fetch_next_row();
            }
        }
        __syncwarp();  // the unit's head is written
    };

    // ---- consumer side
    // The queries as the tensor core's second operand.  int8 codes go to the integer tensor cores as they are, the queries as three
    // digits of 8, 7 and 8 bits, 23 bits of each head's largest magnitude, and sums are exact.  Two digits, 15 bits, left the small channels
    // beside a large one too few: one of 200 times the others moved results by more than their rounding to bf16.  The third costs
    // 4 to 7 % of a long batch (97 ragged sequences 49.5 -> 51.5 us, 64 x 6000 rows of 28 / 4 heads 76.6 -> 82.1).  With at most four heads the
    // first two digits share the eight columns.  e4m3 codes are converted to f16, the queries too.
    constexpr int QB = INT8 ? D / 32 : D / 16;  // steps along the dims
    constexpr int MID = NARROW ? 0 : QB, LOW = MID + QB;  // where the second and third digits lie
    constexpr float kQueryUnits = 127.0f * 128.0f * 256.0f;
    uint32_t qb[INT8 ? LOW + QB : QB][2];
    float o[KS][4], m_run[2], l_run[2], f_head[2], v_ref = 1.0f;
    int first_unit = 0;          // the number, in its pair, of the first unit of this run's part
    const int r_lo = row_of_slot(g);
    const int r_v[2] = {row_of_slot(2 * qd), row_of_slot(2 * qd + 1)};

    auto begin_pair = [&](int m, int h) {
        // The order of the dims over the k-slots is that in which the key codes arrive: those of 16-byte chunk qd (and qd + 4) of a row.
        const int head = INT8 && NARROW ? g & 3 : g;
        const uint4* row = reinterpret_cast<const uint4*>(a.q + ((size_t)m * a.n_q + (size_t)h * group + min(head, group - 1)) * D);
        float x[D / 4];
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const uint4 t = row[8 * (i >> 1) + 2 * qd + (i & 1)];
            const uint32_t u[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[8 * i + 2 * j] = __uint_as_float(u[j] << 16);
                x[8 * i + 2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
            }
        }
        uint32_t most = 0u;  // the largest magnitude by its bits: infinity and NaN are above all others
#pragma unroll
        for (int i = 0; i < D / 4; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
        float amax = __uint_as_float(most), f;
        if constexpr (INT8) {
            amax = fmaxf(amax, 1e-30f);
            const float inv = kQueryUnits / amax;
            f = amax * (1.0f / kQueryUnits) * a.scale_log2;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {  // four dims to a word
                uint32_t hi = 0u, mid = 0u, lo = 0u;
#pragma unroll
                for (int j = 0; j < 4; ++j) {  // v = 32768 d + 256 (w - 128 d) + (v - 256 w), each digit the nearest: -127 .. 127, -64 .. 63, -128 .. 127
                    const int v = head < group ? __float2int_rn(x[4 * i + j] * inv) : 0, w = (v + 128) >> 8, d = (w + 64) >> 7;
                    hi |= ((uint32_t)d & 0xffu) << (8 * j);
                    mid |= ((uint32_t)(w - 128 * d) & 0xffu) << (8 * j);
                    lo |= ((uint32_t)(v - 256 * w) & 0xffu) << (8 * j);
                }
                if constexpr (NARROW) qb[i >> 1][i & 1] = g < 4 ? hi : mid;
                else qb[i >> 1][i & 1] = hi, qb[MID + (i >> 1)][i & 1] = mid;
                qb[LOW + (i >> 1)][i & 1] = lo;  // (NARROW: in both halves of the columns)
            }
        } else {
            // each head is scaled by the power of two that brings its largest magnitude to 2^8 .. 2^9: bf16 values then fit f16
            // without loss down to 2^-22 of the largest, and the scores are scaled back in fp32
            const int be = max(__float_as_int(amax) >> 23, 9);
            const float up = __int_as_float((262 - be) << 23), down = __int_as_float((be - 8) << 23);  // 2^(135 - be), its inverse
#pragma unroll
            for (int i = 0; i < D / 8; ++i) qb[i >> 1][i & 1] = head < group ? pack_f16(x[2 * i] * up, x[2 * i + 1] * up) : 0u;
            f = down * a.scale_log2;
        }
        if (most >= 0x7f800000u) f = NAN;  // scores of a head that is not finite
        const int col = INT8 && NARROW ? 8 * (qd & 1) : 8 * qd;  // lane of column 2 qd (qd & 1: both digits' lanes hold the whole score)
        f_head[0] = __shfl_sync(0xffffffffu, f, col);
        f_head[1] = __shfl_sync(0xffffffffu, f, col + 4);
        m_run[0] = m_run[1] = -INFINITY;
        l_run[0] = l_run[1] = 0.0f;
        v_ref = 0.0f;
#pragma unroll
        for (int t = 0; t < KS; ++t) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.0f;
    };

    auto consume = [&](uint32_t base, const UnitMeta& w) {
        const uint32_t rows[2] = {w.rows[0], UNIT == 64 ? w.rows[1] : 0xffffffffu};
        const bool whole = (rows[0] & rows[1]) == 0xffffffffu;
        const uint32_t vbase = base + kUnitBytes / 2;
        if (!whole) {  // dead rows may hold any bits, and zero times NaN is NaN: overwrite their values
            for (int i = lane; i < UNIT * (D / 16); i += 32) {
                const int row = i / (D / 16);
                if (!((rows[row >> 5] >> (row & 31)) & 1u))
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(vbase + 16u * i), "r"(0u) : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the ring place is a copy's target again later
            __syncwarp();
        }
        // scores of every piece: S^T (16 rows x 8 heads) = K (16 x D) Q^T
        float sv[PIECES][4];
#pragma unroll
        for (int hb = 0; hb < PIECES; ++hb) {
            const uint32_t row_lo = base + (uint32_t)(16 * hb + r_lo) * D, row_hi = row_lo + 8 * D;
            uint32_t x[D / 64][4], y[D / 64][4];
#pragma unroll
            for (int hf = 0; hf < D / 64; ++hf) {
                const uint32_t c = D == 128 ? (uint32_t)(((qd + 4 * hf) ^ r_lo) << 4) : (uint32_t)((qd ^ ((r_lo >> 1) & 3)) << 4);
                lds128(row_lo + c, x[hf]);
                lds128(row_hi + c, y[hf]);
            }
            float s[4];
            if constexpr (INT8) {
                int hi[4] = {0, 0, 0, 0}, mid[4] = {0, 0, 0, 0}, lo[4] = {0, 0, 0, 0};
#pragma unroll
                for (int hf = 0; hf < D / 64; ++hf)
#pragma unroll
                    for (int st = 0; st < 2; ++st) {
                        const int i = 2 * hf + st;
                        mma_s8(hi, x[hf][2 * st], y[hf][2 * st], x[hf][2 * st + 1], y[hf][2 * st + 1], qb[i][0], qb[i][1]);
                        if constexpr (!NARROW) mma_s8(mid, x[hf][2 * st], y[hf][2 * st], x[hf][2 * st + 1], y[hf][2 * st + 1], qb[MID + i][0], qb[MID + i][1]);
                        mma_s8(lo, x[hf][2 * st], y[hf][2 * st], x[hf][2 * st + 1], y[hf][2 * st + 1], qb[LOW + i][0], qb[LOW + i][1]);
                    }
#pragma unroll
                for (int e = 0; e < 4; ++e) {  // the upper digits' sum stays below 2^28, the last one's below 2^21
                    int v;
                    if constexpr (NARROW) {
                        v = qd < 2 ? hi[e] << 7 : hi[e];  // lanes 0, 1 of four hold the first digits' columns, 2, 3 the second digits'
                        v += __shfl_xor_sync(0xffffffffu, v, 2);
                    } else {
                        v = (hi[e] << 7) + mid[e];
                    }
                    s[e] = fmaf((float)v, 256.0f, (float)lo[e]);
                }
            } else {
                float s0[4] = {0.0f, 0.0f, 0.0f, 0.0f}, s1[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int hf = 0; hf < D / 64; ++hf)
#pragma unroll
                    for (int st = 0; st < 4; ++st) {
                        uint32_t f[4];
                        to_f16<KIND>(x[hf][st], f[0], f[2]);
                        to_f16<KIND>(y[hf][st], f[1], f[3]);
                        if (st & 1) mma_f16(s1, f, qb[4 * hf + st][0], qb[4 * hf + st][1]);
                        else mma_f16(s0, f, qb[4 * hf + st][0], qb[4 * hf + st][1]);
                    }
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = s0[e] + s1[e];
            }
            const float ks0 = w.ks[hb] * f_head[0], ks1 = w.ks[hb] * f_head[1];
            sv[hb][0] = s[0] * ks0;
            sv[hb][1] = s[1] * ks1;
            sv[hb][2] = s[2] * ks0;
            sv[hb][3] = s[3] * ks1;
        }
        if (!whole) {  // a dead row may hold anything: selected away
#pragma unroll
            for (int hb = 0; hb < PIECES; ++hb) {
                const uint32_t piece = rows[hb >> 1] >> (16 * (hb & 1));
                if (!((piece >> r_lo) & 1u)) sv[hb][0] = sv[hb][1] = -INFINITY;
                if (!((piece >> (8 + r_lo)) & 1u)) sv[hb][2] = sv[hb][3] = -INFINITY;
            }
        }
        float mx0 = fmaxf(sv[0][0], sv[0][2]), mx1 = fmaxf(sv[0][1], sv[0][3]);
#pragma unroll
        for (int hb = 1; hb < PIECES; ++hb) {
            mx0 = fmaxf(mx0, fmaxf(sv[hb][0], sv[hb][2]));
            mx1 = fmaxf(mx1, fmaxf(sv[hb][1], sv[hb][3]));
        }
        // The values' scales ride on the weights: o is held in units of the largest scale met so far.
        float vs = w.vs[0];
#pragma unroll
        for (int hb = 1; hb < PIECES; ++hb) vs = fmaxf(vs, w.vs[hb]);
        if (__any_sync(0xffffffffu, mx0 > m_run[0] || mx1 > m_run[1] || vs > v_ref)) {
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) {
                mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, off));
                mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, off));
            }
            const float n0 = fmaxf(m_run[0], mx0), n1 = fmaxf(m_run[1], mx1), nv = fmaxf(v_ref, vs);
            const float fv = nv > 0.0f ? v_ref / nv : 0.0f;
            const float c0 = n0 == -INFINITY ? 1.0f : ex2(m_run[0] - n0), c1 = n1 == -INFINITY ? 1.0f : ex2(m_run[1] - n1);
            l_run[0] *= c0;
            l_run[1] *= c1;
#pragma unroll
            for (int t = 0; t < KS; ++t) {
                o[t][0] *= c0 * fv;
                o[t][1] *= c1 * fv;
                o[t][2] *= c0 * fv;
                o[t][3] *= c1 * fv;
            }
            m_run[0] = n0;
            m_run[1] = n1;
            v_ref = nv;
        }
        const float b0 = m_run[0] == -INFINITY ? 0.0f : m_run[0], b1 = m_run[1] == -INFINITY ? 0.0f : m_run[1];
        const float per_ref = v_ref > 0.0f ? __fdividef(32768.0f, v_ref) : 0.0f;
#pragma unroll
        for (int hb = 0; hb < PIECES; ++hb) {
            // O^T (D x 8 heads) += V^T (D x 16 rows) P; lane (g, qd) holds dims 2 KS g ... of rows in slots 2qd, 2qd+1 (+8)
            uint32_t x[4][VW];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = r_v[j & 1];
                const uint32_t row = vbase + (uint32_t)(16 * hb + 8 * (j >> 1) + r) * D;
                if constexpr (D == 128) lds128(row + (uint32_t)((g ^ r) << 4), x[j]);
                else lds64(row + (uint32_t)((((g >> 1) ^ ((r >> 1) & 3)) << 4) + ((g & 1) << 3)), x[j]);
            }
            const float p0 = ex2(sv[hb][0] - b0), p1 = ex2(sv[hb][1] - b1), p2 = ex2(sv[hb][2] - b0), p3 = ex2(sv[hb][3] - b1);
            l_run[0] += p0 + p2;  // this lane's rows; summed over the lanes at the pair's end
            l_run[1] += p1 + p3;
            // Weights as f16, scaled by 2^15 so that the smallest ones keep their bits: an error of up to 2^-11 of a weight (rows of equal
            // weights err alike, so it does not average out), an eighth of the result's own rounding to bf16, up to 2^-8.  The sum
            // that divides the result takes them unrounded.
            const float wv = w.vs[hb] * per_ref;
            const uint32_t w0 = movmatrix_t16(pack_f16(p0 * wv, p1 * wv)), w1 = movmatrix_t16(pack_f16(p2 * wv, p3 * wv));
#pragma unroll
            for (int q = 0; q < VW; ++q) {
                const uint32_t t0 = __byte_perm(x[0][q], x[1][q], 0x5140), t1 = __byte_perm(x[2][q], x[3][q], 0x5140);
                const uint32_t t2 = __byte_perm(x[0][q], x[1][q], 0x7362), t3 = __byte_perm(x[2][q], x[3][q], 0x7362);
                uint32_t f[4];
                to_f16<KIND>(t0, f[0], f[1]);
                to_f16<KIND>(t1, f[2], f[3]);
                mma_f16(o[2 * q], f, w0, w1);
                to_f16<KIND>(t2, f[0], f[1]);
                to_f16<KIND>(t3, f[2], f[3]);
                mma_f16(o[2 * q + 1], f, w0, w1);
            }
        }
    };

    // lane (g, qd) holds dims (2 KS) g + 0 .. 2 KS - 1 of heads 2qd, 2qd + 1: o[t][e] is dim 2t, o[t][2 + e] dim 2t + 1
    auto end_pair = [&](const UnitMeta& w) {
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) {
            l_run[0] += __shfl_xor_sync(0xffffffffu, l_run[0], off);
            l_run[1] += __shfl_xor_sync(0xffffffffu, l_run[1], off);
        }
        const float unscale = v_ref * (1.0f / 32768.0f);
        if (first_unit == 0 && w.unit == w.units - 1) {  // the whole pair
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int head = 2 * qd + e;
                if (head < group) {
                    const float f = l_run[e] == 0.0f ? 0.0f : unscale / l_run[e];  // no row: zeros; a sum that is NaN stays one
                    uint32_t r[KS];
#pragma unroll
                    for (int t = 0; t < KS; ++t) {
                        const __nv_bfloat162 b = __floats2bfloat162_rn(o[t][e] * f, o[t][2 + e] * f);
                        r[t] = *reinterpret_cast<const uint32_t*>(&b);
                    }
                    uint4* dst = reinterpret_cast<uint4*>(a.out + ((size_t)w.m * a.n_q + (size_t)w.h * group + head) * D + 2 * KS * g);
#pragma unroll
                    for (int i = 0; i < KS / 4; ++i) dst[i] = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
                }
            }
            return;
        }
        // a part: the pair began before this run (first place), or goes on behind it (second place: this warp's ring, whose
        // copies have all landed - a pair that goes on is the run's last)
        const bool second = first_unit == 0;
        uint8_t* at = second ? smem + (size_t)warp * stages * kUnitBytes : parts0 + warp * part_smem(group, D);
        PartHead* head_p = reinterpret_cast<PartHead*>(at);
        float* val = reinterpret_cast<float*>(at + sizeof(PartHead));
        __syncwarp();
        if (lane == 0) {
            head_p->begin = w.at - w.unit;
            head_p->end = w.at - w.unit + w.units;
            head_p->m = w.m, head_p->h = w.h, head_p->used = 1;
            if (second) second_used[warp] = 1;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int head = 2 * qd + e;
            if (head < group) {
                if (g == 0) head_p->m_run[head] = m_run[e], head_p->l_run[head] = l_run[e];
#pragma unroll
                for (int t = 0; t < KS; ++t)
                    *reinterpret_cast<float2*>(val + head * D + 2 * KS * g + 2 * t) = make_float2(o[t][e] * unscale, o[t][2 + e] * unscale);
            }
        }
    };

    for (int n = 0; n < stages && next < u1; ++n) issue();
    for (int n = 0; n < issued; ++n) {
        const int place = n % stages;
        if (meta[place].flags & 1) {  // (the head is this warp's own and needs no waiting: the queries come in beside the copies)
            begin_pair(meta[place].m, meta[place].h);
            first_unit = meta[place].unit;
        }
        const bool landed = mbar_wait(full + 8u * place, (uint32_t)(n / stages) & 1u, abort_flag);
        if (!__all_sync(0xffffffffu, landed)) break;
        const UnitMeta w = meta[place];
        consume(ring + (uint32_t)place * kUnitBytes, w);
        if (w.flags & 2) end_pair(w);
        __syncwarp();
        if (next < u1) issue();
    }

    __syncthreads();
    if (*abort_flag) {
        if (tid == 0) {
            if (a.status != nullptr) atomicExch(a.status, BITLINEAR_ERR_TIMEOUT);
            a.desc[2 * blockIdx.x] = a.desc[2 * blockIdx.x + 1] = make_int2(-1, 0);
        }
        abort_drain();
        return;
    }
    // ---- merge the warps' parts; parts of one pair stand next to each other in the order (warp, place)
    const int c0 = runs.begin(blockIdx.x * WARPS), c1 = runs.begin(blockIdx.x * WARPS + WARPS);
    auto part_at = [&](int i) {
        const int w = i >> 1;
        return reinterpret_cast<const PartHead*>((i & 1) ? smem + (size_t)w * stages * kUnitBytes : parts0 + w * part_smem(group, D));
    };
    uint32_t used = 0;  // bit i: part i exists
    if (lane < 2 * WARPS) used = (lane & 1) ? second_used[lane >> 1] != 0 : part_at(lane)->used != 0;
    used = __ballot_sync(0xffffffffu, used != 0);
    int2 desc0 = make_int2(-1, 0), desc1 = desc0;
    while (used) {
        const PartHead* lead = part_at(__ffs((int)used) - 1);
        uint32_t mask = 0;
        if (lane < 2 * WARPS && ((used >> lane) & 1u)) mask = part_at(lane)->begin == lead->begin;
        mask = __ballot_sync(0xffffffffu, mask != 0);
        used &= ~mask;
        const bool whole = lead->begin >= c0 && lead->end <= c1;
        const int slot = lead->begin < c0 ? 0 : 1;
        float* dst = a.part + ((size_t)blockIdx.x * 2 + slot) * part_floats(group, D);
        for (int e = 2 * tid; e < group * D; e += WARPS * 64) {
            const int head = e / D;
            // lane i weighs part i (the 64 elements of a warp belong to one head)
            const bool mine = lane < 2 * WARPS && ((mask >> lane) & 1u);
            const float pm_ = mine ? part_at(lane)->m_run[head] : -INFINITY;
            const float pl = mine ? part_at(lane)->l_run[head] : 0.0f;
            float top;
            asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(top) : "f"(pm_));
            const float f = pm_ == -INFINITY ? 0.0f : ex2(pm_ - top);
            float l = pl * f;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
            float2 acc = make_float2(0.0f, 0.0f);
            for (uint32_t mk = mask; mk;) {  // four parts at a time, their loads side by side
                float2 v[4];
                float w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool on = mk != 0;
                    const int i = __ffs((int)(on ? mk : mask)) - 1;
                    mk &= mk - 1;
                    v[k] = *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(part_at(i) + 1) + e);
                    w[k] = __shfl_sync(0xffffffffu, f, i);
                    if (!on) w[k] = 0.0f;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    acc.x = fmaf(v[k].x, w[k], acc.x);
                    acc.y = fmaf(v[k].y, w[k], acc.y);
                }
            }
            if (whole) {
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                *reinterpret_cast<__nv_bfloat162*>(a.out + ((size_t)lead->m * a.n_q + (size_t)lead->h * group) * D + e) = __floats2bfloat162_rn(acc.x * inv, acc.y * inv);
            } else {
                *reinterpret_cast<float2*>(dst + e) = acc;
                if (e % D == 0) dst[group * D + 2 * head] = top, dst[group * D + 2 * head + 1] = l;
            }
        }
        if (!whole) {  // and the CTA that holds the pair's last unit
            const int2 d = make_int2(lead->m * a.n_kv + lead->h, runs.owner(lead->end - 1) / WARPS);
            if (slot == 0) desc0 = d;
            else desc1 = d;
        }
    }
    if (tid == 0) *reinterpret_cast<int4*>(a.desc + 2 * blockIdx.x) = make_int4(desc0.x, desc0.y, desc1.x, desc1.y);
}

// Merges the parts of a pair that several CTAs share: CTA c does nothing unless a pair begins in attention CTA c and goes on
// behind it.  A thread per head and dim (a CTA per head is 0.8 us slower); a lane weighs one part of a round, in every warp alike.  Rounds of four where a pair has
// that few parts (16 sequences: 24 us a call against 28 with one size of 32), of 16 otherwise (one sequence: 11 us against 14
// with 32).
template <int D>
__global__ void __launch_bounds__(8 * D) attn_decode_kv8_combine_kernel(const float* __restrict__ part, const int2* __restrict__ desc, int group, int n_kv,
                                                                    __nv_bfloat16* __restrict__ out) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int c = blockIdx.x, head = threadIdx.y, lane = threadIdx.x & 31;
    const int2 own = desc[2 * c + 1];
    if (own.x < 0) return;
    const size_t stride = part_floats(group, D);
    const float* base = part + head * D + threadIdx.x;
    float top = -INFINITY, l = 0.0f, acc = 0.0f;
    // N parts from p0 on; CTA c's part is its second, the others' their first (a CTA that has no unit at all has none)
    auto round = [&](auto n_tag, int p0) {
        constexpr int N = decltype(n_tag)::value;
        const int p = min(p0 + lane, own.y);
        const bool in = lane < N && p0 + lane <= own.y && (p == c || desc[2 * p].x == own.x);
        const float2 ml = *reinterpret_cast<const float2*>(part + ((size_t)p * 2 + (p == c ? 1 : 0)) * stride + group * D + 2 * head);
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {  // (asm: all loads of a round are in flight before the first result is used)
            const int q = min(p0 + i, own.y);
            asm volatile("ld.global.f32 %0, [%1];" : "=f"(v[i]) : "l"(base + ((size_t)q * 2 + (q == c ? 1 : 0)) * stride));
        }
        const float pm = in ? ml.x : -INFINITY;
        float n = pm;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) n = fmaxf(n, __shfl_xor_sync(0xffffffffu, n, off));
        n = fmaxf(n, top);
        const float f0 = top == -INFINITY ? 0.0f : ex2(top - n), f = pm == -INFINITY ? 0.0f : ex2(pm - n);
        float lt = in ? ml.y * f : 0.0f;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) lt += __shfl_xor_sync(0xffffffffu, lt, off);
        l = fmaf(l, f0, lt);
        acc *= f0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float w = __shfl_sync(0xffffffffu, in ? f : -1.0f, i);
            acc = w < 0.0f ? acc : fmaf(v[i], w, acc);  // (a part that does not exist may hold anything; one that is NaN counts)
        }
        top = n;
    };
    if (own.y - c < 4) round(std::integral_constant<int, 4>{}, c);
    else
        for (int p0 = c; p0 <= own.y; p0 += 16) round(std::integral_constant<int, 16>{}, p0);
    const int m = own.x / n_kv, h = own.x - m * n_kv;
    out[(((size_t)m * n_kv + h) * group + head) * D + threadIdx.x] = __float2bfloat16_rn(l == 0.0f ? 0.0f : acc / l);
}

// ---------------------------------------------------------------------------------------------- host side

bool kv8_dims_ok(int n_q, int n_kv, int hd, int kind, int n_blocks, int block_rows) {
    return n_q > 0 && n_kv > 0 && n_q % n_kv == 0 && n_q / n_kv <= 8 && (hd == 64 || hd == 128) && (kind == BITLINEAR_KV_INT8 || kind == BITLINEAR_KV_E4M3) &&
           n_blocks > 0 && (block_rows == 16 || block_rows == 32 || block_rows == 64 || block_rows == 128) &&
           (long long)n_blocks * n_kv * block_rows <= (1ll << 31) - 256;
}

int log2_of(int block_rows) { return block_rows == 16 ? 4 : block_rows == 32 ? 5 : block_rows == 64 ? 6 : 7; }

// rows = every (block, head, row) of the pool, columns = D bytes; a box is a unit's rows, or a block's where that is fewer, swizzled by the row's width
bool make_kv8_map(CUtensorMap* map, const void* pool, long long rows, int hd, int block_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)hd, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)hd};
    const cuuint32_t box[2] = {(cuuint32_t)hd, (cuuint32_t)std::min(block_rows, unit_rows(hd))};
    const cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(pool), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              hd == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr size_t kAttnMaxSmem = 227 * 1024;

template <int D, int KIND, int WARPS, bool NARROW>
int attn8_launch(const CUtensorMap& map_k, const CUtensorMap& map_v, AttnArgs a, int ctas, cudaStream_t st) {
    // opted in once per device and kernel
    static std::mutex mu;
    static bool done[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return BITLINEAR_ERR_CUDA;
    }
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!done[dev]) {
            if (cudaFuncSetAttribute(attn_decode_kv8_kernel<D, KIND, WARPS, NARROW>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kAttnMaxSmem) !=
                cudaSuccess) {
                cudaGetLastError();
                return BITLINEAR_ERR_CUDA;
            }
            done[dev] = true;
        }
    }
    const int group = a.n_q / a.n_kv;
    a.stages = kMaxStages;
    while (a.stages > 1 && 1024 + attn8_smem(group, D, WARPS, a.stages).total > kAttnMaxSmem) --a.stages;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(WARPS * 32);
    cfg.dynamicSmemBytes = 1024 + attn8_smem(group, D, WARPS, a.stages).total;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, attn_decode_kv8_kernel<D, KIND, WARPS, NARROW>, map_k, map_v, a) != cudaSuccess) {
        cudaGetLastError();
        return BITLINEAR_ERR_CUDA;
    }
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(D, (unsigned)group);
    cfg.dynamicSmemBytes = 0;
    if (cudaLaunchKernelEx(&cfg, attn_decode_kv8_combine_kernel<D>, (const float*)a.part, (const int2*)a.desc, group, a.n_kv, a.out) != cudaSuccess) {
        cudaGetLastError();
        return BITLINEAR_ERR_CUDA;
    }
    return BITLINEAR_OK;
}

// Twelve warps with rings of two units each, where the parts of a group of at most four heads (or heads of 64) leave the room; eleven
// otherwise (64 x 6000 rows, 28 / 4 heads of 128, two digits then: 79 us for int8, 73 for e4m3; with ten or eight warps 84 to 86 and 79).
template <int D, int KIND>
int attn8_dispatch(const CUtensorMap& map_k, const CUtensorMap& map_v, const AttnArgs& a, int ctas, cudaStream_t st) {
    if (a.n_q / a.n_kv <= 4) return attn8_launch<D, KIND, 12, true>(map_k, map_v, a, ctas, st);
    return attn8_launch<D, KIND, D == 64 ? 12 : 11, false>(map_k, map_v, a, ctas, st);
}

}  // namespace

}  // namespace bitlinear

using namespace bitlinear;

extern "C" {

int bitlinear_rope_kv8(const float* q, const float* k, const float* v, const int32_t* positions, const int32_t* slots, const float* rope_table, int T,
                       int t_max, int n_q_heads, int n_kv_heads, int head_dim, void* q_out_bf16, void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                       int kv_dtype, int n_blocks, int block_rows, void* stream) {
    if (kv_dtype != BITLINEAR_KV_INT8 && kv_dtype != BITLINEAR_KV_E4M3) return BITLINEAR_ERR_DTYPE;
    if (T < 0 || t_max <= 0 || !kv8_dims_ok(n_q_heads, n_kv_heads, head_dim, kv_dtype, n_blocks, block_rows) || (long long)T * n_q_heads * head_dim > (1ll << 40) ||
        n_kv_heads > 65535)
        return BITLINEAR_ERR_SHAPE;
    if (T == 0) return BITLINEAR_OK;
    if (!q || !k || !v || !positions || !slots || !rope_table || !q_out_bf16 || !k_cache || !v_cache || !k_scale || !v_scale) return BITLINEAR_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(rope_table) || !aligned16(q_out_bf16) || !aligned16(k_cache) || !aligned16(v_cache))
        return BITLINEAR_ERR_ALIGN;
    int sm_count = 0;
    if (const int rc = device_sm_count(&sm_count)) return rc;
    AppendArgs a = {q, k, v, positions, slots, reinterpret_cast<const float2*>(rope_table), T, t_max, n_q_heads, n_kv_heads, log2_of(block_rows), n_blocks,
                    static_cast<__nv_bfloat16*>(q_out_bf16), static_cast<uint8_t*>(k_cache), static_cast<uint8_t*>(v_cache), k_scale, v_scale, 1, 0};
    // a CTA per token and head while that fits the GPU a few times over, else per tile of tokens (most of them lead no run)
    a.tile = (long long)T * 2 * n_kv_heads <= 64ll * sm_count ? 1 : 16;
    const long long kv_ctas = (long long)((T + a.tile - 1) / a.tile) * 2 * n_kv_heads;
    const long long q_ctas = std::min((long long)T, 16ll * sm_count);
    if (kv_ctas + q_ctas > 0x7fffffffll) return BITLINEAR_ERR_SHAPE;
    a.kv_ctas = (int)kv_ctas;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(kv_ctas + q_ctas));
    cfg.blockDim = dim3(kAppendThreads);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const bool i8 = kv_dtype == BITLINEAR_KV_INT8;
    const cudaError_t rc = head_dim == 128 ? (i8 ? cudaLaunchKernelEx(&cfg, rope_kv8_kernel<128, BITLINEAR_KV_INT8>, a)
                                                 : cudaLaunchKernelEx(&cfg, rope_kv8_kernel<128, BITLINEAR_KV_E4M3>, a))
                                           : (i8 ? cudaLaunchKernelEx(&cfg, rope_kv8_kernel<64, BITLINEAR_KV_INT8>, a)
                                                 : cudaLaunchKernelEx(&cfg, rope_kv8_kernel<64, BITLINEAR_KV_E4M3>, a));
    if (rc != cudaSuccess) {
        cudaGetLastError();
        return BITLINEAR_ERR_CUDA;
    }
    return BITLINEAR_OK;
}

size_t bitlinear_attention_kv8_workspace_bytes(int n_q_heads, int n_kv_heads, int head_dim) {
    if (n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > 8 || (head_dim != 64 && head_dim != 128)) return 0;
    return align_up(kMaxCtas * 2 * sizeof(int2), 256) + kMaxCtas * 2 * part_floats(n_q_heads / n_kv_heads, head_dim) * sizeof(float);
}

int bitlinear_attention_decode_kv8(const void* q_bf16, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                                   const int32_t* tables, const int32_t* lengths, const int32_t* seq_ids, int M, int n_q_heads, int n_kv_heads, int head_dim,
                                   int kv_dtype, int n_blocks, int block_rows, int n_seq, int max_blocks, void* out_bf16, void* ws, size_t ws_bytes,
                                   void* stream) {
    if (kv_dtype != BITLINEAR_KV_INT8 && kv_dtype != BITLINEAR_KV_E4M3) return BITLINEAR_ERR_DTYPE;
    if (M < 0 || M > 65535 || n_seq <= 0 || max_blocks <= 0 || !kv8_dims_ok(n_q_heads, n_kv_heads, head_dim, kv_dtype, n_blocks, block_rows) ||
        (long long)max_blocks * block_rows > (1ll << 30) || (!seq_ids && n_seq < M) ||
        (double)M * n_kv_heads * (((double)max_blocks * block_rows + kMinUnit - 1) / kMinUnit + 1) > 2147483000.0)
        return BITLINEAR_ERR_SHAPE;
    if (M == 0) return BITLINEAR_OK;
    if (!q_bf16 || !k_cache || !v_cache || !k_scale || !v_scale || !tables || !lengths || !out_bf16) return BITLINEAR_ERR_NULL;
    if (!aligned16(q_bf16) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out_bf16)) return BITLINEAR_ERR_ALIGN;
    if (!ws || !aligned16(ws) || ws_bytes < bitlinear_attention_kv8_workspace_bytes(n_q_heads, n_kv_heads, head_dim)) return BITLINEAR_ERR_WORKSPACE;
    int sm_count = 0;
    if (const int rc = device_sm_count(&sm_count)) return rc;
    const long long pool_rows = (long long)n_blocks * n_kv_heads * block_rows;
    CUtensorMap map_k, map_v;
    if (!make_kv8_map(&map_k, k_cache, pool_rows, head_dim, block_rows) || !make_kv8_map(&map_v, v_cache, pool_rows, head_dim, block_rows))
        return BITLINEAR_ERR_CUDA;
    AttnArgs a = {static_cast<const __nv_bfloat16*>(q_bf16), k_scale, v_scale, tables, lengths, seq_ids, M, n_q_heads, n_kv_heads, n_seq, max_blocks, log2_of(block_rows),
                  n_blocks, 1, 1.4426950408889634f / sqrtf((float)head_dim), static_cast<__nv_bfloat16*>(out_bf16),
                  reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + align_up(kMaxCtas * 2 * sizeof(int2), 256)), static_cast<int2*>(ws), device_status_word()};
    const int ctas = std::min(sm_count, kMaxCtas);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (head_dim == 128)
        return kv_dtype == BITLINEAR_KV_INT8 ? attn8_dispatch<128, BITLINEAR_KV_INT8>(map_k, map_v, a, ctas, st)
                                             : attn8_dispatch<128, BITLINEAR_KV_E4M3>(map_k, map_v, a, ctas, st);
    return kv_dtype == BITLINEAR_KV_INT8 ? attn8_dispatch<64, BITLINEAR_KV_INT8>(map_k, map_v, a, ctas, st)
                                         : attn8_dispatch<64, BITLINEAR_KV_E4M3>(map_k, map_v, a, ctas, st);
}

}  // extern "C"
