// The paged cache of 8-bit codes: what its kernels share.  A block is 64 tokens of one sequence and KV head; whole blocks are
// codes with one scale per tensor (K [64][D], V [D][64] bytes), the unfinished one is 16-bit values (K and V [64][D]).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kvc {

constexpr int kPBT = 64;  // tokens of a block and page

enum : int { kF16 = 0, kBF16 = 1 };
enum : int { kI8 = 0, kE4M3 = 1 };

// Flags in the cache's fault word.
constexpr uint32_t kFaultPage = 1u, kFaultTail = 2u, kFaultPosition = 4u, kFaultLength = 8u, kFaultNonfinite = 16u;

// Cache and sequences of one call, by value to the kernels.
struct PagedGeo {
    int H, G, n_pages, n_tails, max_pages, batch;
    uint8_t *k_codes, *v_codes;
    float *scales;
    uint16_t *k_tail, *v_tail;
    uint32_t *fault;
    const int32_t *__restrict__ lens;
    const int32_t *__restrict__ table;
    const int32_t *__restrict__ tails;
};

struct PagedNew {
    int n_tokens;
    const int32_t *__restrict__ starts;
    const uint16_t *__restrict__ k;
    const uint16_t *__restrict__ v;
    const uint16_t *q;
    uint16_t *q_out;
    size_t k_stride, v_stride, q_stride, q_out_stride;
    const float *__restrict__ cos_sin;
    const int32_t *__restrict__ positions;
    int n_positions, rot_dim, interleaved;
    int edge[2];  // first pair of the second and of the third axis
};

hipError_t launch_paged_append(const PagedGeo &g, const PagedNew &n, int head_dim, int data_type, int code_type, hipStream_t s);

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

__device__ __forceinline__ void flag(uint32_t *fault, uint32_t bit) {
    __hip_atomic_fetch_or(fault, bit, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// 16-bit values in the low or high half of a word.
template <int T>
__device__ __forceinline__ float wide_lo(uint32_t w) {
    if constexpr (T == kBF16) return __uint_as_float(w << 16);
    else return (float)__builtin_bit_cast(half2v, w)[0];
}
template <int T>
__device__ __forceinline__ float wide_hi(uint32_t w) {
    if constexpr (T == kBF16) return __uint_as_float(w & 0xffff0000u);
    else return (float)__builtin_bit_cast(half2v, w)[1];
}
// Two values rounded to nearest even and packed.
template <int T>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
    if constexpr (T == kBF16) {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        const bf2 v = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, v);
    } else {
        const half2v v = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, v);
    }
}
template <int T>
constexpr uint32_t kInfBits = T == kBF16 ? 0x7f80u : 0x7c00u;  // magnitudes from here on are Inf or NaN
template <int T>
constexpr uint32_t kNanBits = T == kBF16 ? 0x7fc0u : 0x7e00u;

}  // namespace kvc
