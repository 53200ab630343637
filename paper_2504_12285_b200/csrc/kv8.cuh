// What the kernels over the 8-bit paged cache share: its dimensions, and codes as f16.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "bitlinear.h"
#include "fp32_math.cuh"

namespace bitlinear {

inline bool kv8_dims_ok(int n_q, int n_kv, int hd, int kind, int n_blocks, int block_rows) {
    return n_q > 0 && n_kv > 0 && n_q % n_kv == 0 && n_q / n_kv <= 8 && (hd == 64 || hd == 128) && (kind == BITLINEAR_KV_INT8 || kind == BITLINEAR_KV_E4M3) &&
           n_blocks > 0 && (block_rows == 16 || block_rows == 32 || block_rows == 64 || block_rows == 128) &&
           (long long)n_blocks * n_kv * block_rows <= (1ll << 31) - 256;
}

inline int log2_of(int block_rows) { return block_rows == 16 ? 4 : block_rows == 32 ? 5 : block_rows == 64 ? 6 : 7; }

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Four codes of a word -> two pairs of f16, exactly.  int8: the code plus 128 becomes the low bits of 1024 + x, and
// 1152 is taken off.  e4m3: the conversion instruction.
template <int KIND>
__device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
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
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

}  // namespace bitlinear
