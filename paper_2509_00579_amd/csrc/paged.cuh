// The paged cache of 8-bit codes: what its kernels share.  A block is 64 tokens of one sequence and KV head; whole blocks are
// codes with one scale per tensor (K [64][D], V [D][64] bytes), the unfinished one is 16-bit values (K and V [64][D]).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "paged_plan.h"

namespace kvc {

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
    int stream_q;
};

// One attention call: queries and outputs [rows][Hq][D] with their strides in elements.
struct PagedAttn {
    const uint16_t *__restrict__ q;
    uint16_t *__restrict__ out;
    size_t q_stride, out_stride;
    float scale;  // times log2(e): the softmax runs on powers of two
    int window;   // keys that a row sees, 0 = all before it
    uint32_t *tickets;
    float *partials;
};

constexpr int kDecodeRows = 32;       // query rows per KV head that a decode call may have
constexpr int kDecodeWGs = 256;       // its largest grid
constexpr int kMaxDecodeBatch = 4096;
// Workspace: tickets, then two partial states per workgroup (o[D], m, l of each row, padded to whole 16 bytes).
constexpr int kTicketWords = 1024;
constexpr int partial_pitch(int D) { return D + 4; }

constexpr int kPrefillStateRows = 1 << 17;  // rows of states that a prefill launch that splits the keys may leave

hipError_t launch_paged_prefill(const PagedGeo &g, const PagedAttn &a, const int32_t *starts, int n_tokens, int max_new, int max_len,
                                int head_dim, int data_type, int code_type, hipStream_t s);
hipError_t launch_paged_decode(const PagedGeo &g, const PagedAttn &a, int q_len, int max_len, int head_dim, int data_type, int code_type,
                               hipStream_t s);
hipError_t launch_paged_append(const PagedGeo &g, const PagedNew &n, int head_dim, int data_type, int code_type, hipStream_t s);

// Lets a kernel have `most` bytes of dynamic LDS on the current device; `done` remembers for which devices (a bit each) that has
// been said.
inline hipError_t allow_lds(const void *kernel, size_t most, std::atomic<uint64_t> &done) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    if (e == hipSuccess && dev < 64) done.fetch_or(bit, std::memory_order_release);
    return e;
}

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
// Eight codes as eight fp16 values, exactly.  int8: the bytes with their sign bit turned become the low bits of 1024 + 128 + code.
template <int C>
__device__ __forceinline__ half8v widen8(uint32_t a, uint32_t b) {
    half2v r[4];
    if constexpr (C == kI8) {
        a ^= 0x80808080u;
        b ^= 0x80808080u;
        const half2v off = {(_Float16)1152.f, (_Float16)1152.f};
        r[0] = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u)) - off;
        r[1] = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u)) - off;
        r[2] = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)) - off;
        r[3] = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)) - off;
    } else {
        r[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false);
        r[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true);
        r[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false);
        r[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true);
    }
    return half8v{r[0][0], r[0][1], r[1][0], r[1][1], r[2][0], r[2][1], r[3][0], r[3][1]};
}

// bf16 values reach the fp16 matrix instructions times a power of two that brings the largest of them to 2^14..2^15: a value is
// then exact unless it is below 2^-28 of that one, and off by at most 2^-40 of it otherwise.
__device__ __forceinline__ int bf16_shift(uint32_t largest_bits) { return 141 - (int)(largest_bits >> 7); }
__device__ __forceinline__ uint32_t bf16_to_half2(uint32_t w, int shift) {
    const half2v v = {(_Float16)ldexpf(wide_lo<kBF16>(w), shift), (_Float16)ldexpf(wide_hi<kBF16>(w), shift)};
    return __builtin_bit_cast(uint32_t, v);
}
// Both halves of two words compared as unsigned numbers; 16-bit magnitudes are ordered like the values they stand for.
__device__ __forceinline__ uint32_t max16(uint32_t a, uint32_t b) {
    typedef unsigned short us2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
}
// The largest finite magnitude (a bit pattern) among `count` times eight bf16 values.
template <int count>
__device__ __forceinline__ uint32_t bf16_largest(const uint4 (&w)[count]) {
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < count; k++)
        m = max16(max16(max16(max16(m, w[k].x & 0x7fff7fffu), w[k].y & 0x7fff7fffu), w[k].z & 0x7fff7fffu), w[k].w & 0x7fff7fffu);
    m = max(m & 0xffffu, m >> 16);
    if (m >= 0x7f80u) {  // Inf or NaN: leave them out
        m = 0;
#pragma unroll
        for (int k = 0; k < count; k++)
#pragma unroll
            for (int c = 0; c < 4; c++) {
                const uint32_t x = c == 0 ? w[k].x : c == 1 ? w[k].y : c == 2 ? w[k].z : w[k].w, lo = x & 0x7fffu, hi = (x >> 16) & 0x7fffu;
                m = lo < 0x7f80u && lo > m ? lo : m;
                m = hi < 0x7f80u && hi > m ? hi : m;
            }
    }
    return m;
}

// Across the four groups of 16 lanes of a wave, and across its halves.
__device__ __forceinline__ float max_rows(float v) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float sum_rows(float v) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ uint32_t max_rows_u(uint32_t v) {
    auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = a[0] > a[1] ? a[0] : a[1];
    a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return a[0] > a[1] ? a[0] : a[1];
}

template <int T>
constexpr uint32_t kInfBits = T == kBF16 ? 0x7f80u : 0x7c00u;  // magnitudes from here on are Inf or NaN
template <int T>
constexpr uint32_t kNanBits = T == kBF16 ? 0x7fc0u : 0x7e00u;

}  // namespace kvc
