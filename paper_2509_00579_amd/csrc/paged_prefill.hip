// Attention of prompt chunks over the paged cache of 8-bit codes: ragged chunks, causal, optionally within a sliding window.
//
// Bound by the matrix cores and, nearly as much, by the vector ALUs that the softmax runs on (512 tokens on 32 k: 0.97 to 1.02
// PFLOP/s from box to box; a large library product in fp16 reaches 1.21); with heads of 64 by the vector ALUs.  A workgroup owns one KV
// head and a tile of query rows: consecutive tokens times the group of query heads, so that every K and V block it stages serves whole groups.
// The codes of a block are widened to fp16 once per workgroup, on their way to LDS (two buffers, one barrier a block); a
// wave multiplies its 32 rows, S^T = K Q^T and O^T = V^T P^T on 32x32x16 products.  Row r of K's 32 is token
// 16 (r / 16) + 8 (r / 4 % 2) + 4 (r / 8 % 2) + r % 4, so that a lane receives the scores of eight consecutive tokens: its
// part of P^T for the second product, without an exchange.
//
// K's scale multiplies the scores.  V's scale is 2^e times a mantissa: the mantissa is added to the exponents of P (and taken
// out of their sum again), 2^e goes into the codes as they are widened, relative to the accumulators' unit, so that a block's
// product adds to them as it is.  The unit is the largest e so far, until a block lies so far below that fp16 could not hold its
// codes: then the unit comes down to the block, since the larger ones may be hidden from a row or have no weight in it.  All
// this is exact, down to 2^-91 of the largest scale that the workgroup has met; V below that counts as zero.
//
// P is rounded to fp16 (11 bits, relative to each weight: the reference leaves 2^8 to 2^14 above one, so weights down to 2^-22 of
// a row's largest keep all of them), and the sum of the weights is taken from the rounded ones: the second product runs on one
// operand instead of two, and an output is off by up to 2^-10 of its values' weighted magnitudes (fp16 against 64 bits, the
// root of the mean square: 2.6e-4 of them, 2.1e-4 with weights in 32 bits).
// The exponent is one fused product of the score's factors minus the reference, which was rounded: all weights of a row are off
// by one common factor, which the division takes out as long as it is neither 0 nor infinite; from scores of 2^26 on it
// could be, and the product is rounded by itself.  (With the mantissa's logarithm in it the reference is rounded once more for every
// block, by 2^-25 of itself, as much as the scores of its size are.)
// The reference moves only when a score would pass 2^14 above it, which spares most tiles the rescaling of the accumulators.
//
// Few rows over a long axis: the keys are split among workgroups, and a second launch joins their states.
#include <algorithm>
#include <cmath>

#include "huff_decode.cuh"
#include "paged.cuh"
#include "split_combine.cuh"

namespace kvc {

namespace {

// What the unfinished block counts for when the keys are split: it is turned in LDS and nothing overlaps with it.  1, 2, 3, 4:
// 27.0 25.2 25.3 26.2 us for 4 chunks of 16 tokens on 4001 (8 KV heads, groups of 4), 555 560 558 558 for 512 tokens on 32 k.
constexpr int kTailBlocks = 3;
constexpr float kRefLead = 8.f, kRefMost = 14.f, kFarScore = 67108864.f;
constexpr int kNoExponent = -10000;  // of a scale of zero

// The unit 2^e of the output's accumulators while blocks with V scales of other exponents go by.
template <int C>
struct VUnit {
    // fp16's smallest step is 2^-24 and the smallest code 1 (int8) or 2^-9 (e4m3).
    static constexpr int kExactBelow = C == kI8 ? 24 : 15;
    // How far the unit may lie below the largest: 2^26 keys with weights of 2^15 and codes of 2^9 stay within binary32.
    static constexpr int kDeepest = 76;
    int e = kNoExponent, largest = kNoExponent;
    __device__ __forceinline__ bool fits(int block) const { return (uint32_t)(e - block) <= (uint32_t)kExactBelow; }
    // A block with exponent `block` comes next; returns what that adds to e.
    __device__ __forceinline__ int next(int block) {
        if (__builtin_expect(fits(block), 1)) return 0;
        const int was = e;
        if (block > e) e = block;
        else if (block != kNoExponent) e = max(block, largest - kDeepest);
        largest = max(largest, e);
        return e - was;
    }
    // What the block's codes are widened with.
    __device__ __forceinline__ float factor(int block) const { return fits(block) ? __uint_as_float((uint32_t)(block - e + 127) << 23) : 0.f; }
};

struct PrefillArgs {
    PagedGeo g;
    PagedAttn a;
    int n_tokens, units, splits;
    int per_tile;  // tokens of a row tile
    const int32_t *__restrict__ starts;
    Divide by_heads, by_splits, by_group, by_tile;
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float16v mfma32(half8v a, half8v b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// How many of the waves' registers a CU has room for, with W waves of 32 rows.
constexpr int workgroups_per_cu(int D, int W) { return W == 8 ? 1 : D == 128 ? 2 : 4; }

// The row tile of a unit: which sequence, its first token among the sequence's new ones.
struct RowTile {
    int b, start, fresh, len, tail, place;
    bool bad;
};
// All lanes of a wave together.  b < 0: no such unit.  Everything that is read of 64 sequences is on its way at once.
__device__ __forceinline__ RowTile find_tile(const PrefillArgs &p, int unit, int lane) {
    RowTile r;
    r.b = -1;
    for (int base = 0; base < p.g.batch; base += 64) {
        int tiles = 0, s0 = 0, s1 = 0, len = 0, tail = 0;
        if (base + lane < p.g.batch) {
            s0 = p.starts[base + lane];
            s1 = p.starts[base + lane + 1];
            len = p.g.lens[base + lane];
            tail = p.g.tails[base + lane];
            asm volatile("" ::"v"(len), "v"(tail));
            if (s0 >= 0 && s1 > s0 && s1 <= p.n_tokens) tiles = (int)p.by_tile.of(s1 - s0 + p.per_tile - 1);
            else if (s1 != s0 || s0 < 0 || s1 > p.n_tokens) flag(p.g.fault, kFaultLength);
        }
        const int before = (int)wave_excl_scan((uint32_t)tiles, lane);
        const unsigned long long past = __builtin_amdgcn_ballot_w64(before + tiles > unit);
        if (r.b >= 0) continue;
        if (!past) {
            unit -= __builtin_amdgcn_readlane(before + tiles, 63);
            continue;
        }
        const int at = uniform(__builtin_ctzll(past));
        r.b = base + at;
        r.place = uniform(unit - __builtin_amdgcn_readlane(before, at)) * p.per_tile;
        r.start = __builtin_amdgcn_readlane(s0, at);
        r.fresh = __builtin_amdgcn_readlane(s1, at) - r.start;
        r.len = __builtin_amdgcn_readlane(len, at);
        r.tail = __builtin_amdgcn_readlane(tail, at);
        const bool long_ = (unsigned)r.len > (unsigned)p.g.max_pages * kPBT, no_tail = r.len % kPBT && (unsigned)r.tail >= (unsigned)p.g.n_tails;
        r.bad = long_ || no_tail;
        if (r.bad && lane == 0) flag(p.g.fault, long_ ? kFaultLength : kFaultTail);
        if (blockIdx.x) break;  // the first workgroup looks at all sequences
    }
    return r;
}

// Eight codes as fp16 times 2^k (`by`), exactly unless that is below fp16's smallest step.
template <int C>
__device__ __forceinline__ uint4 widen8_by(uint32_t a, uint32_t b, float by) {
    half2v r[4];
    if constexpr (C == kI8) {
        a ^= 0x80808080u;
        b ^= 0x80808080u;
        const _Float16 f = (_Float16)by, o = (_Float16)(-1152.f * by);
        const half2v ff = {f, f}, oo = {o, o};
        r[0] = __builtin_elementwise_fma(__builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u)), ff, oo);
        r[1] = __builtin_elementwise_fma(__builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u)), ff, oo);
        r[2] = __builtin_elementwise_fma(__builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)), ff, oo);
        r[3] = __builtin_elementwise_fma(__builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)), ff, oo);
    } else {
        r[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, by, false);
        r[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, by, true);
        r[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, by, false);
        r[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, by, true);
    }
    return make_uint4(__builtin_bit_cast(uint32_t, r[0]), __builtin_bit_cast(uint32_t, r[1]), __builtin_bit_cast(uint32_t, r[2]),
                      __builtin_bit_cast(uint32_t, r[3]));
}

// The LDS tiles in units of 16 bytes (eight fp16 values): K [64 tokens][D], V [D][64 tokens]; the units of a row change places so
// that sixteen rows' units of one number hit sixteen different places of 256 bytes.
template <int D>
__device__ __forceinline__ int k_unit(int token, int chunk) {
    if constexpr (D == 128) return token * 16 + (chunk ^ (token & 15));
    else return token * 8 + (chunk ^ ((token >> 1) & 7));
}
__device__ __forceinline__ int v_unit(int channel, int chunk) { return channel * 8 + (chunk ^ ((channel >> 1) & 7)); }

// The order of `count` products and the LDS reads of their left operands: four reads ahead, no more (left to itself the
// compiler reads all of them first and runs out of registers).
template <int count>
__device__ __forceinline__ void ahead() {
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < count - 4; i += 2) {
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
}

// A barrier that waits for LDS only: loads from memory stay on their way.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// What a wave has gathered for its 32 rows; lane (n, half) has row n.
template <int D>
struct RowState {
    float16v o[D / 32];
    float ref, sum;
};

template <int T, int D>
__device__ __forceinline__ void store_rows(uint16_t *out, int half, const RowState<D> &st, float f) {
#pragma unroll
    for (int c = 0; c < D / 32; c++)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<uint2 *>(out + 32 * c + 2 * i + 4 * half) =
                make_uint2(narrow2<T>(st.o[c][i] * f, st.o[c][i + 1] * f), narrow2<T>(st.o[c][i + 2] * f, st.o[c][i + 3] * f));
}

template <int T, int C, int D, int W>
__global__ __launch_bounds__(64 * W, workgroups_per_cu(D, W)) void paged_prefill_kernel(PrefillArgs p) {
    constexpr int kPreRows = 32 * W, kPreThreads = 64 * W;
    constexpr int kUnits = kPBT * D / 8, kPieces = (kPBT * D / 16 + kPreThreads - 1) / kPreThreads;  // 16-byte units of a tile; pieces of 16 codes per thread
    extern __shared__ __align__(16) uint4 s_tiles[];  // [2 buffers][K, V][kUnits]
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), n = lane & 31, half = lane >> 5;
    const int rest = (int)p.by_heads.of(blockIdx.x), h = (int)blockIdx.x - rest * p.g.H, from_last = (int)p.by_splits.of(rest);
    const int split = rest - from_last * p.splits, unit = p.units - 1 - from_last;
    const RowTile rt = find_tile(p, unit, lane);
    if (rt.b < 0) return;
    const int G = p.g.G, r = 32 * wave + n, in_tile = (int)p.by_group.of(r), place = rt.place + in_tile, head = h * G + r - in_tile * G;
    const bool live = r < p.per_tile * G && place < rt.fresh;
    const int past = rt.len - rt.fresh;
    const int pos = live ? past + place : -1;
    const int last_pos = past + min(rt.place + p.per_tile, rt.fresh) - 1;  // of the tile's last row
    const int first_pos = past + rt.place;
    // blocks that any row sees, and this workgroup's share of them
    const int from = p.a.window > 0 && first_pos >= p.a.window ? (first_pos - p.a.window + 1) / kPBT : 0;
    const int blocks = rt.bad || last_pos < 0 ? 0 : last_pos / kPBT + 1 - from;
    const int unfinished = rt.len / kPBT;  // this block is in 16 bits
    const int shares = blocks + (from + blocks > unfinished ? kTailBlocks - 1 : 0);
    auto share = [&](int k) { return uniform(from + min((int)p.by_splits.of(shares * k), blocks)); };
    const int t0 = share(split), t1 = share(split + 1);

    constexpr int KS = D / 16;
    // Page numbers first, then the queries: what hangs on the former is asked for while the latter come.
    const int32_t *pages = p.g.table + (size_t)rt.b * p.g.max_pages;
    const int t_pages = min(t1, max(t0, unfinished));  // the last share can be empty
    auto page_of = [&](int t) { return t + lane < t_pages ? pages[t + lane] : 0; };
    const int first_pages = page_of(t0);
    half8v qf[KS];
    float q_factor = fabsf(p.a.scale);
    uint4 qw[KS];
    {
        const uint16_t *q = p.a.q + (size_t)(rt.start + place) * p.a.q_stride + (size_t)head * D + 8 * half;
#pragma unroll
        for (int k = 0; k < KS; k++) qw[k] = live ? *reinterpret_cast<const uint4 *>(q + 16 * k) : make_uint4(0, 0, 0, 0);
    }
    auto ready_queries = [&]() __attribute__((always_inline)) {
        const uint32_t turn = p.a.scale < 0.f ? 0x80008000u : 0u;
        uint4 w[KS];
#pragma unroll
        for (int k = 0; k < KS; k++) w[k] = make_uint4(qw[k].x ^ turn, qw[k].y ^ turn, qw[k].z ^ turn, qw[k].w ^ turn);
        if constexpr (T == kBF16) {
            const uint32_t big = bf16_largest(w);
            const auto both = __builtin_amdgcn_permlane32_swap(big, big, false, false);
            const int shift = bf16_shift(max(both[0], both[1]));
            q_factor = ldexpf(q_factor, -shift);
#pragma unroll
            for (int k = 0; k < KS; k++)
                w[k] = make_uint4(bf16_to_half2(w[k].x, shift), bf16_to_half2(w[k].y, shift), bf16_to_half2(w[k].z, shift),
                                  bf16_to_half2(w[k].w, shift));
        }
#pragma unroll
        for (int k = 0; k < KS; k++) qf[k] = __builtin_bit_cast(half8v, w[k]);
    };
    RowState<D> st;
#pragma unroll
    for (int c = 0; c < D / 32; c++)
#pragma unroll
        for (int i = 0; i < 16; i++) st.o[c][i] = 0.f;
    st.ref = -INFINITY;
    st.sum = 0.f;
    VUnit<C> unit_v;  // of st.o

    const int token_row = 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);  // of K's 32, see above
    // the last key that this wave's rows see, and the first row's
    const int wave_last = uniform(past + min(rt.place + (int)p.by_group.of(min(32 * wave + 31, p.per_tile * G - 1)), rt.fresh - 1));
    const int wave_first = uniform(past + rt.place + (int)p.by_group.of(32 * wave));
    auto some_hidden = [&](int t) { return t * kPBT + kPBT - 1 > wave_first || (p.a.window > 0 && t * kPBT <= wave_last - p.a.window); };

    float16v s[2];       // scores
    uint32_t pw[2][8];   // weights, fp16
    auto rescale = [&](float by) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < D / 32; c++) st.o[c] *= by;
    };
    // Where this lane reads K and V of a buffer: the numbers of the 16-byte units within a row differ in bits that the addresses
    // have to themselves, so each is one exclusive or away from these (which are kept out of the compiler's sight: it
    // would hold all of them in registers over the loop).
    const char *tiles = reinterpret_cast<const char *>(s_tiles);
    const uint32_t k_first = 16 * k_unit<D>(token_row, half), v_first = 16 * v_unit(n, half);
    auto scores = [&](int buffer) __attribute__((always_inline)) {
        uint32_t at = k_first + buffer * (2 * kUnits * 16);
        asm volatile("" : "+v"(at));
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int i = 0; i < 16; i++) s[j][i] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; k++)
#pragma unroll
            for (int j = 0; j < 2; j++)
                s[j] = mfma32(*reinterpret_cast<const half8v *>(tiles + (at ^ (k << 5)) + j * 32 * D * 2), qf[k], s[j]);
        ahead<2 * KS>();
    };
    // Scores of block t to weights; mant: log2 of its V scale's mantissa, inv: one over that mantissa, by_e brings the accumulators to the unit that V is staged in.
    auto weigh = [&](int t, float k_scale, float mant, float inv, float by_e, bool masked) __attribute__((always_inline)) {
        float f = k_scale * q_factor;
        uint32_t seen[2] = {~0u, ~0u};  // a bit per key of mine
        if (masked) {
            const int low = p.a.window > 0 ? pos - p.a.window : -1;
#pragma unroll
            for (int j = 0; j < 2; j++) {
                seen[j] = 0;
#pragma unroll
                for (int x = 0; x < 2; x++) {  // eight keys in a row
                    const int key = t * kPBT + 32 * j + 16 * x + 8 * half;
                    const uint32_t upto = 1u << min(max(pos + 1 - key, 0), 8), below = 1u << min(max(low + 1 - key, 0), 8);
                    seen[j] |= (upto - below) << (8 * x);
                }
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const uint32_t m = (uint32_t)((int32_t)(seen[j] << (31 - i)) >> 31);
                    s[j][i] = __uint_as_float((m & __float_as_uint(s[j][i])) | (~m & 0xff800000u));
                }
            }
        }
        const bool sees = (seen[0] | seen[1]) != 0, times_zero = !(f > 0.f);
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int i = 0; i < 16; i++) mx = fmaxf(mx, s[j][i]);
        {
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * f;
        }
        const bool move = mx - st.ref > kRefMost;
        if (__builtin_amdgcn_ballot_w64(move) != 0 || by_e != 1.f) {
            const float ref = move ? fmaxf(mx, kLowestRef) - kRefLead : st.ref;
            const float alpha = move ? __builtin_amdgcn_exp2f(st.ref - ref) : 1.f;
            st.ref = ref;
            st.sum *= alpha;
            rescale(alpha * by_e);
        }
        const float ref = fmaxf(st.ref, kLowestRef);  // nothing met yet but hidden keys and scores of -Inf: their weights are zero
        float off = mant - ref;
        if (__builtin_amdgcn_ballot_w64(sees && fabsf(mx) > kFarScore) != 0) {  // see above
#pragma unroll
            for (int j = 0; j < 2; j++)
#pragma unroll
                for (int i = 0; i < 16; i++) s[j][i] = s[j][i] * f - ref;
            f = 1.f;
            off = mant;
        }
        float sum = 0.f;
        const half2v ones = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float a = __builtin_amdgcn_exp2f(fmaf(s[j][i], f, off)), b = __builtin_amdgcn_exp2f(fmaf(s[j][i + 1], f, off));
                pw[j][i >> 1] = narrow2<kF16>(a, b);
            }
        if (masked && __builtin_amdgcn_ballot_w64(times_zero) != 0) {  // -Inf times a scale of zero
#pragma unroll
            for (int j = 0; j < 2; j++)
#pragma unroll
                for (int i = 0; i < 8; i++)
                    pw[j][i] &= ((seen[j] >> (2 * i)) & 1 ? 0xffffu : 0u) | ((seen[j] >> (2 * i + 1)) & 1 ? 0xffff0000u : 0u);
        }
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int i = 0; i < 8; i++) sum = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, pw[j][i]), ones, sum, false);
        st.sum = fmaf(sum, inv, st.sum);
    };
    auto add_values = [&](int buffer) __attribute__((always_inline)) {
        uint32_t at = v_first + buffer * (2 * kUnits * 16) + kUnits * 16;
        asm volatile("" : "+v"(at));
#pragma unroll
        for (int x = 0; x < 4; x++) {
            const uint32_t *w = pw[x >> 1] + 4 * (x & 1);
            const half8v pf = __builtin_bit_cast(half8v, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
            for (int c = 0; c < D / 32; c++)
                st.o[c] = mfma32(*reinterpret_cast<const half8v *>(tiles + (at ^ (x << 5)) + c * 32 * kPBT * 2), pf, st.o[c]);
        }
        ahead<D / 8>();
    };

    // Page numbers and scales of 64 blocks, a block a lane; V's as its exponent, log2 of its mantissa and what takes that out again.
    int known = t0, known_page = 0, known_e = kNoExponent;
    float known_k = 0.f, known_mant = 0.f, known_inv = 1.f;
    auto learn_pages = [&](int t, int page) __attribute__((always_inline)) {
        known = t;
        const bool ok = (unsigned)page < (unsigned)p.g.n_pages;
        if (!ok) flag(p.g.fault, kFaultPage);
        known_page = ok ? page : 0;
        float2 sc = *reinterpret_cast<const float2 *>(p.g.scales + ((size_t)known_page * p.g.H + h) * 2);
        if (!ok) sc.x = __builtin_nanf("");
        return sc;
    };
    auto learn_scales = [&](float2 sc) __attribute__((always_inline)) {
        known_k = sc.x;
        const bool any = sc.y > 0.f;
        known_e = any ? ilogbf(sc.y) : kNoExponent;
        known_mant = any ? __builtin_amdgcn_logf(ldexpf(sc.y, -known_e)) : 0.f;
        known_inv = __builtin_amdgcn_exp2f(-known_mant);
    };
    auto e_of = [&](int t) { return __builtin_amdgcn_readlane(known_e, t - known); };
    auto power_of_2 = [&](int e) { return __uint_as_float((uint32_t)max(e + 127, 0) << 23); };  // 0 below the normal range

    // Two halves of the workgroup's waves, one of each on every SIMD, take turns: while one multiplies (block t's weights with V,
    // then its queries with block t + 1's K), the other weighs its scores and widens its share of the codes of a later block.
    constexpr int kGroups = W == 8 ? 2 : 1;
    const int lead = kGroups == 2 ? wave >> 2 : 0;
    constexpr int kTilePieces = kPBT * D / 16;
    const int k_piece = tid, v_piece = kTilePieces < kPreThreads ? (tid + kPreThreads / 2) % kPreThreads : tid;
    uint4 ck[kPieces], cv[kPieces];
    VUnit<C> staged;
    // Behind the last block the same is done with it again, into buffers that nobody will read: a branch around it would cost the
    // loop copies of whatever it leaves in registers.
    auto fetch_k = [&](int t, uint4 (&c)[kPieces]) __attribute__((always_inline)) {
        t = min(t, t_pages - 1);
        const uint4 *k = reinterpret_cast<const uint4 *>(p.g.k_codes + ((size_t)__builtin_amdgcn_readlane(known_page, t - known) * p.g.H + h) * kPBT * D);
#pragma unroll
        for (int i = 0; i < kPieces; i++)
            if (k_piece + i * kPreThreads < kTilePieces) c[i] = k[k_piece + i * kPreThreads];
    };
    auto fetch_v = [&](int t) __attribute__((always_inline)) {
        t = min(t, t_pages - 1);
        const uint4 *v = reinterpret_cast<const uint4 *>(p.g.v_codes + ((size_t)__builtin_amdgcn_readlane(known_page, t - known) * p.g.H + h) * kPBT * D);
#pragma unroll
        for (int i = 0; i < kPieces; i++)
            if (v_piece + i * kPreThreads < kTilePieces) cv[i] = v[v_piece + i * kPreThreads];
    };
    auto stage_k = [&](uint4 *sk, const uint4 (&c)[kPieces]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kPieces; i++) {
            const int piece = k_piece + i * kPreThreads, token = piece / (D / 16), chunk = piece % (D / 16) * 2;
            if (piece >= kTilePieces) break;
            sk[k_unit<D>(token, chunk)] = widen8_by<C>(c[i].x, c[i].y, 1.f);
            sk[k_unit<D>(token, chunk + 1)] = widen8_by<C>(c[i].z, c[i].w, 1.f);
        }
    };
    auto stage_v = [&](int t, uint4 *sv) __attribute__((always_inline)) {
        const int e = e_of(min(t, t_pages - 1));
        staged.next(e);
        const float by = staged.factor(e);
#pragma unroll
        for (int i = 0; i < kPieces; i++) {
            const int piece = v_piece + i * kPreThreads, channel = piece / 4, part = piece % 4 * 2;
            if (piece >= kTilePieces) break;
            sv[v_unit(channel, part)] = widen8_by<C>(cv[i].x, cv[i].y, by);
            sv[v_unit(channel, part + 1)] = widen8_by<C>(cv[i].z, cv[i].w, by);
        }
    };
    // The unfinished block's rows, asked for before the others where there are registers to hold them.
    constexpr bool kTailAhead = D == 128;
    constexpr int kRowUnits = D / 8, kMine = kUnits / kPreThreads;
    uint4 rk[kMine], rv[kMine];
    auto ask_tail = [&]() __attribute__((always_inline)) {
        const size_t at = ((size_t)rt.tail * p.g.H + h) * kPBT * D;
        const uint4 *tk = reinterpret_cast<const uint4 *>(p.g.k_tail + at), *tv = reinterpret_cast<const uint4 *>(p.g.v_tail + at);
#pragma unroll
        for (int i = 0; i < kMine; i++) {
            const int u = tid + i * kPreThreads;
            const bool in = u / kRowUnits < rt.len - unfinished * kPBT;
            rk[i] = in ? tk[u] : make_uint4(0, 0, 0, 0);
            rv[i] = in ? tv[u] : make_uint4(0, 0, 0, 0);
        }
    };
    if (t0 < t_pages) {
        auto buffer = [&](int t) { return s_tiles + ((t - t0) & 1) * 2 * kUnits; };
        uint4 c0[kPieces];
        const float2 first_scales = learn_pages(t0, first_pages);
        fetch_k(t0, c0);
        fetch_k(t0 + 1, ck);
        fetch_v(t0);
        learn_scales(first_scales);
        ready_queries();
        stage_k(s_tiles, c0);
        if (lead) {
            stage_k(s_tiles + 2 * kUnits, ck);
            stage_v(t0, s_tiles + kUnits);
            fetch_k(t0 + 2, ck);
            fetch_v(t0 + 1);
        }
        if (kTailAhead && t_pages < t1) ask_tail();
        lds_barrier();
        scores(0);
        if (lead) lds_barrier();
        for (int t = t0; t < t_pages; t++) {
            if (t + 4 > known + 64) learn_scales(learn_pages(t, page_of(t)));
            const int mine = (t - t0) & 1;
            const float by_e = power_of_2(-unit_v.next(e_of(t)));
            weigh(t, bcast(known_k, t - known), bcast(known_mant, t - known), bcast(known_inv, t - known), by_e, some_hidden(t));
            stage_k(buffer(t + 1 + lead), ck);
            stage_v(t + lead, buffer(t + lead) + kUnits);
            fetch_k(t + 2 + lead, ck);
            fetch_v(t + 1 + lead);
            lds_barrier();
            __builtin_amdgcn_s_setprio(1);
            add_values(mine);
            scores(1 - mine);
            __builtin_amdgcn_s_setprio(0);
            if (kGroups == 2) lds_barrier();
        }
        if (kGroups == 2 && !lead) lds_barrier();
    } else {
        if (kTailAhead && t_pages < t1) ask_tail();
        ready_queries();
    }
    if (t_pages < t1) {
        // The block that is still in 16 bits, on products of its own type: K as it is, V turned.  fp16: the accumulators change to units of
        // one; bf16: to a unit that no sum of its values overflows, and the weights are taken to it in two parts.
        const int t = unfinished;
        uint4 *sk = s_tiles, *sv = sk + kUnits;
        if (!kTailAhead) ask_tail();
        const int e_ref = T == kBF16 ? max(24, unit_v.largest - VUnit<C>::kDeepest) : 0;
        int up = unit_v.e - e_ref;
        if (up < -100) {  // in two steps: the pages' values are there still, though 2^up may be none
            rescale(power_of_2(-100));
            up += 100;
        }
        const float by_e = power_of_2(up);
        unit_v.e = e_ref;
        const float w_by = power_of_2(-e_ref);
        __syncthreads();  // the tiles are free
#pragma unroll
        for (int i = 0; i < kMine; i++) {
            const int u = tid + i * kPreThreads, row = u / kRowUnits, chunk = u % kRowUnits;
            sk[k_unit<D>(row, chunk)] = rk[i];
            const uint32_t w[4] = {rv[i].x, rv[i].y, rv[i].z, rv[i].w};
#pragma unroll
            for (int c = 0; c < 8; c++) {
                const uint32_t x = c & 1 ? w[c >> 1] >> 16 : w[c >> 1] & 0xffffu;
                reinterpret_cast<uint16_t *>(sv + v_unit(8 * chunk + c, row >> 3))[row & 7] = (uint16_t)x;
            }
        }
        __syncthreads();
        if constexpr (T == kF16) {
            scores(0);
            weigh(t, 1.f, 0.f, 1.f, by_e, true);
            add_values(0);
        } else {
            constexpr float kBack = 6.103515625e-05f;  // 2^-14: the queries' largest between 1 and 2, exactly
            typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
#pragma unroll
            for (int j = 0; j < 2; j++)
#pragma unroll
                for (int i = 0; i < 16; i++) s[j][i] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; k++) {
                uint32_t w[4];
#pragma unroll
                for (int x = 0; x < 4; x++) w[x] = narrow2<kBF16>((float)qf[k][2 * x] * kBack, (float)qf[k][2 * x + 1] * kBack);
                const bf8 q = __builtin_bit_cast(bf8, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
                for (int j = 0; j < 2; j++)
                    s[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        *reinterpret_cast<const bf8 *>(tiles + (k_first ^ (k << 5)) + j * 32 * D * 2), q, s[j], 0, 0, 0);
            }
            weigh(t, 1.f / kBack, 0.f, 1.f, by_e, true);
#pragma unroll
            for (int part = 0; part < 2; part++)
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) {  // a weight's 11 bits are two times 8
                        const uint32_t both = pw[x >> 1][4 * (x & 1) + i];
                        const float a = wide_lo<kF16>(both) * w_by, b = wide_hi<kF16>(both) * w_by;
                        w[i] = narrow2<kBF16>(a, b);
                        if (part) w[i] = narrow2<kBF16>(a - wide_lo<kBF16>(w[i]), b - wide_hi<kBF16>(w[i]));
                    }
                    const bf8 pf = __builtin_bit_cast(bf8, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
                    for (int c = 0; c < D / 32; c++)
                        st.o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            *reinterpret_cast<const bf8 *>(tiles + ((v_first + kUnits * 16) ^ (x << 5)) + c * 32 * kPBT * 2), pf, st.o[c], 0, 0, 0);
                }
        }
    }

    float sum;
    {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(st.sum), __float_as_uint(st.sum), false, false);
        sum = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    }
    const int e_ref = max(unit_v.e, -140);  // nothing was met: any
    if (p.splits == 1) {
        if (!live) return;
        const float f = rt.bad ? __builtin_nanf("") : sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int c = 0; c < D / 32; c++) st.o[c] *= f;  // first: with their unit they could be too large
        store_rows<T, D>(p.a.out + (size_t)(rt.start + place) * p.a.out_stride + (size_t)head * D, half, st, ldexpf(1.f, e_ref));
        return;
    }
    float *part = p.a.partials + (((size_t)(unit * p.g.H + h) * p.splits + split) * kPreRows + r) * partial_pitch(D);
    if (!live) return;
#pragma unroll
    for (int c = 0; c < D / 32; c++)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<float4 *>(part + 32 * c + 2 * i + 4 * half) =
                make_float4(st.o[c][i], st.o[c][i + 1], st.o[c][i + 2], st.o[c][i + 3]);
    if (half == 0) {
        part[D] = st.ref;
        part[D + 1] = rt.bad ? __builtin_nanf("") : sum;
        part[D + 2] = (float)e_ref;
    }
}

// Joins the splits of a row tile: R rows per wave, their loads on the way together, D / 64 channels a lane.  Lane s has the states of
// split s, so all weights of a row are known after one load.
constexpr int kJoinWaves = 4, kMaxKeySplits = 64;
template <int T, int D, int R>
__global__ __launch_bounds__(64 * kJoinWaves) void paged_join_kernel(PrefillArgs p, int tile_rows) {
    constexpr int kMine = D / 64, kJoinRows = R, kBatch = R == 1 ? 8 : 4;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t groups = tile_rows / (kJoinWaves * kJoinRows);  // a power of two
    const int group = blockIdx.x & (groups - 1), rest = blockIdx.x >> __builtin_ctz(groups);
    const int unit = (int)p.by_heads.of(rest), h = rest - unit * p.g.H, r0 = (group * kJoinWaves + wave) * kJoinRows;
    const RowTile rt = find_tile(p, unit, lane);
    if (rt.b < 0) return;
    const int rows = min(p.per_tile, rt.fresh - rt.place) * p.g.G - r0;  // that there are from here on
    if (rows <= 0) return;
    const float *part = p.a.partials + ((size_t)(unit * p.g.H + h) * p.splits * tile_rows + r0) * partial_pitch(D);
    const size_t step = (size_t)tile_rows * partial_pitch(D);
    float4 state[kJoinRows];
#pragma unroll
    for (int i = 0; i < kJoinRows; i++)
        state[i] = lane < p.splits && i < rows ? *reinterpret_cast<const float4 *>(part + lane * step + i * partial_pitch(D) + D)
                                               : make_float4(-INFINITY, 0.f, -140.f, 0.f);
    float w[kJoinRows], by[kJoinRows], unit_v[kJoinRows], o[kJoinRows][kMine] = {};
    auto fetch = [&](int s, float (&v)[kBatch][kJoinRows][kMine]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < kBatch; k++)
#pragma unroll
            for (int i = 0; i < kJoinRows; i++)
#pragma unroll
                for (int c = 0; c < kMine; c++)
                    v[k][i][c] = s + k < p.splits && i < rows ? part[(s + k) * step + i * partial_pitch(D) + lane * kMine + c] : 0.f;
    };
    float v[kBatch][kJoinRows][kMine];
    fetch(0, v);
#pragma unroll
    for (int i = 0; i < kJoinRows; i++) {
        const float m = state[i].x, l = state[i].y, e = state[i].z;
        const bool met = m != -INFINITY;  // a split that met nothing takes no part
        const float top = wave_max(m);
        const float f = met ? __builtin_amdgcn_exp2f(m - top) : 0.f;
        const float sum = wave_sum(met ? l * f : l != l ? l : 0.f);
        // The output's unit is that of the split that counts most, with its weight taken in: one with large values that the row
        // gave next to no weight may not push the others' out of binary32.
        const float e_top = wave_max(met ? e + ceilf(fmaxf(m - top, -1000.f)) : -2000.f);
        w[i] = ldexpf(f, (int)(e - e_top));
        by[i] = sum == 0.f ? 0.f : 1.f / sum;
        unit_v[i] = ldexpf(1.f, (int)e_top);
    }
    for (int s = 0;;) {
#pragma unroll
        for (int k = 0; k < kBatch; k++)
#pragma unroll
            for (int i = 0; i < kJoinRows; i++)
#pragma unroll
                for (int c = 0; c < kMine; c++) o[i][c] = fmaf(v[k][i][c], bcast(w[i], (s + k) & 63), o[i][c]);
        s += kBatch;
        if (s >= p.splits) break;
        fetch(s, v);
    }
#pragma unroll
    for (int i = 0; i < kJoinRows; i++) {
        if (i >= rows) break;
        const int r = r0 + i, in_tile = (int)p.by_group.of(r);
        uint16_t *out = p.a.out + (size_t)(rt.start + rt.place + in_tile) * p.a.out_stride + (size_t)(h * p.g.G + r - in_tile * p.g.G) * D + lane * kMine;
        if constexpr (D == 128) *reinterpret_cast<uint32_t *>(out) = narrow2<T>(o[i][0] * by[i] * unit_v[i], o[i][1] * by[i] * unit_v[i]);
        else *out = (uint16_t)narrow2<T>(o[i][0] * by[i] * unit_v[i], 0.f);
    }
}

template <int T, int C, int D, int W>
hipError_t launch_tiles(PrefillArgs p, int max_len, hipStream_t s) {
    constexpr size_t kLds = (size_t)4 * kPBT * D * 2;
    auto kernel = paged_prefill_kernel<T, C, D, W>;
    static std::atomic<uint64_t> allowed{0};
    hipError_t e = allow_lds(reinterpret_cast<const void *>(kernel), kLds, allowed);
    if (e != hipSuccess) return e;
    p.per_tile = 32 * W / p.g.G;
    // every sequence has at most one row tile that is not full
    const int some = p.g.batch < p.n_tokens ? p.g.batch : p.n_tokens;
    p.units = p.n_tokens / p.per_tile + some;
    const long long base = (long long)p.units * p.g.H;
    const int pages = max_len > 0 && max_len < p.g.max_pages * kPBT ? (max_len + kPBT - 1) / kPBT : p.g.max_pages;
    // Splits of the keys, by what they would take, in blocks on a CU: a workgroup has its share of the longest range (an unfinished
    // block counts for more, see above) and what it does before the first and behind the last block; workgroups that have to wait
    // for others are rounds, those that run beside others on a CU slow them down; the join reads every state.  A split more has to
    // be worth it.  us with 1, 2, 4, 6, 8, 11, 16 splits: a chunk of 16 tokens on 484 (8 KV heads, groups of 4) 18.5 15.5 12.6 12.2
    // 11.6, 4 of 16 on 984 30.7 23.2 18.2 16.4 17.2 19.9 21.2, 4 of 16 on 4001 105 59.8 35.9 28.8 25.3 27.2 25.0.
    const double tiles = std::max<double>(some, (p.n_tokens + p.per_tile - 1) / p.per_tile + 0.5 * (some - 1)) * p.g.H;
    const double longest = p.a.window > 0 ? std::min<double>(pages, (p.a.window + p.per_tile) / kPBT + 2) : pages;
    const double mean = std::max(longest / 2, longest - (double)p.n_tokens / some / kPBT / 2);
    constexpr double kAround = 3, kBeside = D == 128 ? 0.75 : 0.6;
    double best = 0;
    p.splits = 1;
    for (int k = 1; k <= kMaxKeySplits && k <= longest && (k == 1 || base * k * 32 * W <= kPrefillStateRows); k++) {
        const double share = tiles * k / 256;
        const double rounds = share <= 1 ? 1 : workgroups_per_cu(D, W) == 1 ? std::ceil(share) : std::max(1.5, kBeside * share);
        auto work = [&](double blocks) { return kAround + std::ceil((blocks + kTailBlocks - 1) / k); };
        const double cost = std::max(rounds * work(mean), work(longest)) + (k == 1 ? 0 : 3 + 0.1 * k + 0.005 * k * tiles);
        if (k == 1 || cost < 0.95 * best) {
            best = cost;
            p.splits = k;
        }
    }
    p.by_heads = Divide(p.g.H);
    p.by_splits = Divide(p.splits);
    p.by_group = Divide(p.g.G);
    p.by_tile = Divide(p.per_tile);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(base * p.splits)), dim3(64 * W), kLds, s, p);
    if (p.splits > 1) {
        // One row per wave while all waves are on the chip at once, or in two goes; four share the work around them.  us of the whole
        // call with one, four: 4 chunks of 16 tokens on 4001 (6144 rows) 25.4 26.7, one of 8 on 30 k 34.3 39.8; 16 of 16 on 1984
        // (24576 rows) 42.8 40.2, 512 tokens on 32 k (34816) 564 559, 32 of 16 on 3984, heads of 64 (49152) 76.8 71.0.
        const long long rows = base * 32 * W;
        if (rows > 16384) hipLaunchKernelGGL((paged_join_kernel<T, D, 4>), dim3((unsigned)(rows / (kJoinWaves * 4))), dim3(64 * kJoinWaves), 0, s, p, 32 * W);
        else hipLaunchKernelGGL((paged_join_kernel<T, D, 1>), dim3((unsigned)(rows / kJoinWaves)), dim3(64 * kJoinWaves), 0, s, p, 32 * W);
    }
    return hipGetLastError();
}

// Eight waves, 256 rows, two sets that take turns on the matrix cores, where the chunks fill more than half of them; else four.  us with
// four and eight waves: a prompt of 8192 tokens 632 607, 512 tokens on 32 k 585 560, 4 chunks of 16 on 4001 25.3 31.3.  Heads of 64 leave
// registers for four workgroups of four waves on a CU: 100 us for 16 chunks of up to 700 tokens in a window, with two of eight waves 144.
template <int T, int C, int D>
hipError_t launch(const PrefillArgs &p, int max_new, int max_len, hipStream_t s) {
    if constexpr (D == 128) {
        if (max_new == 0 || (long long)max_new * p.g.G > 128) return launch_tiles<T, C, D, 8>(p, max_len, s);
    }
    return launch_tiles<T, C, D, 4>(p, max_len, s);
}

}  // namespace

hipError_t launch_paged_prefill(const PagedGeo &g, const PagedAttn &a, const int32_t *starts, int n_tokens, int max_new, int max_len,
                                int head_dim, int data_type, int code_type, hipStream_t s) {
    PrefillArgs p = {g, a, n_tokens, 0, 0, 0, starts};
    auto by_dim = [&](auto t, auto c) {
        if (head_dim == 64) return launch<decltype(t)::value, decltype(c)::value, 64>(p, max_new, max_len, s);
        return launch<decltype(t)::value, decltype(c)::value, 128>(p, max_new, max_len, s);
    };
    auto by_code = [&](auto t) {
        if (code_type == kI8) return by_dim(t, std::integral_constant<int, kI8>());
        return by_dim(t, std::integral_constant<int, kE4M3>());
    };
    if (data_type == kF16) return by_code(std::integral_constant<int, kF16>());
    return by_code(std::integral_constant<int, kBF16>());
}

}  // namespace kvc
