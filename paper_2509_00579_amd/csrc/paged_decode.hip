// Decode attention over the paged cache of 8-bit codes: up to 32 query rows per KV head (a token or a few drafted ones, times
// the group of query heads).  out = sum_j p_j v_j / sum_j p_j with p_j = 2^(s_j - m), s_j = log2(e) scale q.k_j, one pass with
// the running maximum m.
//
// Bound by HBM: every code is read once (32 heads of 32768 tokens, 268 MB: 56 us, 4.8 TB/s, where the caches hold none of them; a large
// plain read reaches 6.1, and the way to the first codes and the joins take 8 us).  A tile is one block (64 tokens) of a KV head; the tiles of all
// sequences and heads form one list that is dealt evenly to the waves, whatever the sequences' lengths are, so a wave has a
// range of tiles of one head, or the end of one, some whole ones and the beginning of another.  States of heads that are
// spread over several waves meet in LDS, over several workgroups in the workspace, where the last workgroup to arrive joins
// them in order.  A short call is bound by the chain of dependent loads and by the fetching of its code, which is run once: loops
// beat unrolled code outside the tiles (one head of 1000 tokens: 7.6 us a call, replayed).
//
// Both products run on the fp16 matrix cores, S^T = K Q^T and O^T = V^T P^T, with the codes as the left operand straight
// from their 16-byte loads: K rows are tokens, V pages have channels as rows.  Row r of the s-th group of 16 tokens is token
// 16 (r / 4) + 4 s + r % 4, so that lane group g receives the scores of tokens 16 g .. 16 g + 15: the very tokens whose V
// codes its loads bring, and P needs no exchange between lanes.  Codes are exact in fp16.  P goes in as two fp16 parts (the matrix
// cores have nothing else to do), 22 bits of it; the reference m is 15 below the largest score, so that fp16's smallest step,
// 2^-24, is 2^-39 of the largest weight and thousands of faint keys keep theirs.  Scales multiply the products: K's the scores, V's the tile's sum.
#include "huff_decode.cuh"
#include "paged.cuh"
#include "split_combine.cuh"

namespace kvc {

namespace {

struct DecodeArgs {
    PagedGeo g;
    PagedAttn a;
    int q_len, rows;
    uint32_t inv_g;  // 2^16 / G, rounded up: row * inv_g / 2^16 is row / G for the 32 rows that there are at most
};
__device__ __forceinline__ int place_of(const DecodeArgs &p, int row) { return (int)(((uint32_t)row * p.inv_g) >> 16); }

__device__ __forceinline__ float4v mfma16(half8v a, half8v b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ half8v as_half8(uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    return __builtin_bit_cast(half8v, make_uint4(x, y, z, w));
}
// The same with 16-bit values of type T as they are in memory.
template <int T>
__device__ __forceinline__ float4v product(uint4 a, uint4 b, float4v c) {
    typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
    if constexpr (T == kBF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
    else return mfma16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c);
}
// Queries for products with keys that are still in 16 bits.  bf16 ones come back from fp16 exactly, their largest between 1 and 2, so
// that no key overflows a product that binary32 could hold.
constexpr float kBackFromHalf = 6.103515625e-05f;  // 2^-14
template <int T>
__device__ __forceinline__ uint4 raw_queries(half8v v) {
    if constexpr (T == kF16) return __builtin_bit_cast(uint4, v);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; k++) w[k] = narrow2<kBF16>((float)v[2 * k] * kBackFromHalf, (float)v[2 * k + 1] * kBackFromHalf);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Codes are read once a call, yet by plain loads: where the last-level cache (256 MB) still holds some from the call before, they are
// faster, and elsewhere about as fast as ones past the caches.  us, past them -> plain, one cache again and again: 32 heads of 32768
// 56.2 -> 45.4, 8 x 8 heads of up to 16422 43.8 -> 38.5, 64 x 8 of up to 1102 15.3 -> 14.6; six caches in turn: 57.6 -> 56.5, 43.3 ->
// 45.0, 17.1 -> 15.6.
__device__ __forceinline__ uint4 load16(const uint8_t *p) { return *reinterpret_cast<const uint4 *>(p); }
constexpr float kRefBelow = 15.f;
// What an unfinished block costs, in pages: twice the bytes, and its loads start behind the pages'.  us with 2, 3, 4, 6, 8 pages: 8 x 8
// heads of up to 16422 tokens 39.4 38.7 37.8 37.8 36.8, 64 x 8 of up to 1102 14.4 14.9 14.5 14.5 15.2.
constexpr int kTailUnits = 4;
// Units that a workgroup has at least, while there are others without any: a wave alone on its SIMD is through with a page in less
// than half the time of two.  us with 1, 2, 3, 4, 8 units: one head of 1000 7.6 7.6 7.9 8.0 9.5, 8 heads of 2000 in groups of 4 9.3
// 8.7 8.5 8.9 10.7, one head in a group of 8 of 4000 13.7 10.7 10.0 9.7 11.6, 8 heads of 300 7.4 7.5 7.6 7.9 7.1.
constexpr uint32_t kLeastUnits = 2;
// bf16: the accumulators hold 2^-40 of the sums, so that neither the largest values overflow them (2^15 of a weight, 2^26 keys)
// nor the largest weight's of anything that a page holds (2^-100 and more) drops below binary32's normal range; the factor
// is a multiplication of its own, since with it the smallest scales would.
template <int T>
constexpr float kVUnit = T == kBF16 ? 9.094947017729282e-13f : 1.f;
constexpr float kNan = __builtin_nanf("");

// T, C: types; D: channels; R: groups of 16 query rows.
template <int T, int C, int D, int R>
struct Wave {
    static constexpr int CT = D / 16;  // channels CT r + i, i < CT, are row r of the i-th product with V
    static constexpr int KJ = D / 64, KS = D / 32;
    const DecodeArgs &p;
    const int lane, n, g4;
    half8v qf[R][KS];
    uint4 qw[R][KS];
    float q_factor[R];
    int q_place[R];  // token of the row among the call's
    float m[R], l[R];
    float4v o[R][CT];
    uint4 kr[4][KJ], vr[CT];

    __device__ __forceinline__ Wave(const DecodeArgs &p_, int lane_) : p(p_), lane(lane_), n(lane_ & 15), g4(lane_ >> 4) {
#pragma unroll
        for (int r = 0; r < R; r++) q_place[r] = place_of(p, 16 * r + n);
    }

    // A head's queries are asked for, and made ready once something else is on its way too.
    __device__ __forceinline__ void ask_queries(int b, int h) {
#pragma unroll
        for (int r = 0; r < R; r++) {
            const int row = 16 * r + n;
            const bool have = row < p.rows;
            const uint16_t *q = p.a.q + ((size_t)b * p.q_len + q_place[r]) * p.a.q_stride + (size_t)(h * p.g.G + row - q_place[r] * p.g.G) * D;
#pragma unroll
            for (int k = 0; k < KS; k++)
                qw[r][k] = have ? *reinterpret_cast<const uint4 *>(q + (k >> 1) * 64 + g4 * 16 + (k & 1) * 8) : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void begin() {
#pragma unroll
        for (int r = 0; r < R; r++) {
            uint4 w[KS];
#pragma unroll
            for (int k = 0; k < KS; k++) w[k] = qw[r][k];
            q_factor[r] = 1.f;
            if constexpr (T == kBF16) {
                uint32_t big = bf16_largest(w);
                big = max_rows_u(big);
                const int shift = bf16_shift(big);
                q_factor[r] = ldexpf(1.f, -shift);
#pragma unroll
                for (int k = 0; k < KS; k++)
                    w[k] = make_uint4(bf16_to_half2(w[k].x, shift), bf16_to_half2(w[k].y, shift), bf16_to_half2(w[k].z, shift),
                                      bf16_to_half2(w[k].w, shift));
            }
#pragma unroll
            for (int k = 0; k < KS; k++) qf[r][k] = __builtin_bit_cast(half8v, w[k]);
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int i = 0; i < CT; i++) o[r][i] = float4v{0.f, 0.f, 0.f, 0.f};
        }
    }

    __device__ __forceinline__ int token_of(int s) const { return 16 * (n >> 2) + 4 * s + (n & 3); }

    __device__ __forceinline__ void load_k(int page, int h) {
        const uint8_t *t = p.g.k_codes + ((size_t)page * p.g.H + h) * kPBT * D + 16 * g4;
#pragma unroll
        for (int s = 0; s < 4; s++)
#pragma unroll
            for (int j = 0; j < KJ; j++) kr[s][j] = load16(t + token_of(s) * D + 64 * j);
    }
    __device__ __forceinline__ void load_v(int page, int h) {
        const uint8_t *t = p.g.v_codes + ((size_t)page * p.g.H + h) * kPBT * D + 16 * g4;
#pragma unroll
        for (int i = 0; i < CT; i++) vr[i] = load16(t + (CT * n + i) * kPBT);
    }

    // Scores of tokens base + 16 g4 + j, j < 16, in powers of two; hidden ones are -Inf whatever they were.
    __device__ __forceinline__ void scores(const float4v (&s)[R][4], float factor, int base, int len, float (&x)[R][16]) const {
        const int first_row = len - p.q_len;  // position of the call's first token
        const bool masked = base + kPBT - 1 > first_row || (p.a.window > 0 && base + p.a.window < len);
#pragma unroll
        for (int r = 0; r < R; r++) {
            const float f = factor * q_factor[r];
#pragma unroll
            for (int j = 0; j < 16; j++) x[r][j] = s[r][j >> 2][j & 3] * f;
            if (masked) {
                const int pos = first_row + q_place[r];
                const int low = p.a.window > 0 ? pos - p.a.window : -1;
#pragma unroll
                for (int j = 0; j < 16; j++) {
                    const int t = base + 16 * g4 + j;
                    if (t > pos || t <= low) x[r][j] = -INFINITY;
                }
            }
        }
    }

    // The scores of row group r become weights; returns what the state so far is to be multiplied with.
    __device__ __forceinline__ float weigh(int r, float (&x)[16]) {
        float mx = x[0];
#pragma unroll
        for (int j = 1; j < 16; j++) mx = fmaxf(mx, x[j]);
        mx = fmaxf(fmaxf(m[r], max_rows(mx) - kRefBelow), kLowestRef);
        const float alpha = __builtin_amdgcn_exp2f(m[r] - mx);
        m[r] = mx;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 16; j++) {
            x[j] = __builtin_amdgcn_exp2f(x[j] - mx);
            sum += x[j];
        }
        l[r] = l[r] * alpha + sum;
        return alpha;
    }
    // ... and those P as two fp16 parts.
    __device__ __forceinline__ void softmax(float (&x)[R][16], half8v (&hi)[R][2], half8v (&lo)[R][2], float (&alpha)[R]) {
#pragma unroll
        for (int r = 0; r < R; r++) {
            alpha[r] = weigh(r, x[r]);
            uint32_t ph[8], pl[8];
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
                const float a = x[r][j], b = x[r][j + 1];
                const auto h = __builtin_amdgcn_cvt_pkrtz(a, b);
                ph[j >> 1] = __builtin_bit_cast(uint32_t, h);
                pl[j >> 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a - (float)h[0], b - (float)h[1]));
            }
#pragma unroll
            for (int k = 0; k < 2; k++) {
                hi[r][k] = as_half8(ph[4 * k], ph[4 * k + 1], ph[4 * k + 2], ph[4 * k + 3]);
                lo[r][k] = as_half8(pl[4 * k], pl[4 * k + 1], pl[4 * k + 2], pl[4 * k + 3]);
            }
        }
    }

    __device__ __forceinline__ void add_v(int i, half8v v0, half8v v1, const half8v (&hi)[R][2], const half8v (&lo)[R][2],
                                          const float (&alpha)[R], float factor) {
#pragma unroll
        for (int r = 0; r < R; r++) {
            float4v acc = {0.f, 0.f, 0.f, 0.f};
            acc = mfma16(v0, hi[r][0], acc);
            acc = mfma16(v1, hi[r][1], acc);
            acc = mfma16(v0, lo[r][0], acc);
            acc = mfma16(v1, lo[r][1], acc);
#pragma unroll
            for (int k = 0; k < 4; k++) o[r][i][k] = fmaf(T == kBF16 ? acc[k] * kVUnit<T> : acc[k], factor, o[r][i][k] * alpha[r]);
        }
    }

    // Pages [i0, whole) of a head whose first tile is `first`; i0 < whole.
    __device__ __forceinline__ void run(int b, int h, int first, int i0, int whole, int len) {
        const int32_t *pages = p.g.table + (size_t)b * p.g.max_pages + first;
        // page numbers and scales of 64 tiles, a tile a lane
        int known = i0, known_page = 0;
        float known_k = 0.f, known_v = 0.f;
        auto page_of = [&](int i) { return i + lane < whole ? pages[i + lane] : 0; };
        auto learn = [&](int i, int page) {
            known = i;
            const bool ok = (unsigned)page < (unsigned)p.g.n_pages;
            if (!ok) {
                flag(p.g.fault, kFaultPage);
                page = 0;
            }
            known_page = page;
            const float2 sc = *reinterpret_cast<const float2 *>(p.g.scales + ((size_t)page * p.g.H + h) * 2);
            known_k = ok ? sc.x : kNan;
            known_v = sc.y;
        };
        auto page_at = [&](int i) { return __builtin_amdgcn_readlane(known_page, i - known); };
        const int page0 = page_of(i0);
        ask_queries(b, h);  // behind the page numbers, which are waited for first
        learn(i0, page0);
        load_k(page_at(i0), h);
        load_v(page_at(i0), h);
        begin();
        for (int i = i0; i < whole; i++) {
            float4v s[R][4];
#pragma unroll
            for (int t = 0; t < 4; t++) {
#pragma unroll
                for (int r = 0; r < R; r++) s[r][t] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < KJ; j++) {
                    const half8v k0 = widen8<C>(kr[t][j].x, kr[t][j].y), k1 = widen8<C>(kr[t][j].z, kr[t][j].w);
#pragma unroll
                    for (int r = 0; r < R; r++) {
                        s[r][t] = mfma16(k0, qf[r][2 * j], s[r][t]);
                        s[r][t] = mfma16(k1, qf[r][2 * j + 1], s[r][t]);
                    }
                }
            }
            const float ks = bcast(known_k, i - known), vs = bcast(known_v, i - known);
            const bool more = i + 1 < whole;
            if (more) {
                if (i + 1 == known + 64) learn(i + 1, page_of(i + 1));
                load_k(page_at(i + 1), h);
            }
            float x[R][16], alpha[R];
            half8v hi[R][2], lo[R][2];
            scores(s, ks * p.a.scale, (first + i) * kPBT, len, x);
            softmax(x, hi, lo, alpha);
#pragma unroll
            for (int c = 0; c < CT; c++)
                add_v(c, widen8<C>(vr[c].x, vr[c].y), widen8<C>(vr[c].z, vr[c].w), hi, lo, alpha, vs);
            if (more) load_v(page_at(i + 1), h);
        }
    }

    // The block that is still in 16 bits, on products of its own type: K as it is, V turned in registers, rows behind the end left out.
    __device__ __forceinline__ void unfinished(int b, int h, int len, int tail, bool alone) {
        const int count = len % kPBT;
        const size_t at = ((size_t)tail * p.g.H + h) * kPBT * D;
        if (alone) ask_queries(b, h);
        uint4 kt[4][KS];
        uint32_t vt[16][CT / 2];  // token 16 g4 + j, channels CT n ..
#pragma unroll
        for (int s = 0; s < 4; s++) {
            const uint16_t *k = p.g.k_tail + at + min(token_of(s), count - 1) * D + 16 * g4;
#pragma unroll
            for (int x = 0; x < KS; x++) kt[s][x] = *reinterpret_cast<const uint4 *>(k + (x >> 1) * 64 + (x & 1) * 8);
        }
#pragma unroll
        for (int j = 0; j < 16; j++) {
            const uint16_t *v = p.g.v_tail + at + min(16 * g4 + j, count - 1) * D + CT * n;
            if constexpr (CT == 8) {
                const uint4 w = *reinterpret_cast<const uint4 *>(v);
                vt[j][0] = w.x; vt[j][1] = w.y; vt[j][2] = w.z; vt[j][3] = w.w;
            } else {
                const uint2 w = *reinterpret_cast<const uint2 *>(v);
                vt[j][0] = w.x; vt[j][1] = w.y;
            }
        }
        if (alone) begin();
        float4v s[R][4];
#pragma unroll
        for (int r = 0; r < R; r++) {
            uint4 qt[KS];
#pragma unroll
            for (int x = 0; x < KS; x++) qt[x] = raw_queries<T>(qf[r][x]);
#pragma unroll
            for (int t = 0; t < 4; t++) {
                s[r][t] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < KS; x++) s[r][t] = product<T>(kt[t][x], qt[x], s[r][t]);
            }
        }
        float x[R][16], alpha[R];
        constexpr int kParts = T == kBF16 ? 3 : 2;  // of 8 and of 11 bits
        uint32_t parts[R][kParts][8];
        scores(s, T == kBF16 ? p.a.scale / kBackFromHalf : p.a.scale, len - count, len, x);
#pragma unroll
        for (int r = 0; r < R; r++) {
            alpha[r] = weigh(r, x[r]);
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
                float a = x[r][j] * kVUnit<T>, c = x[r][j + 1] * kVUnit<T>;  // bf16 has the exponents for it
#pragma unroll
                for (int k = 0; k < kParts; k++) {
                    const uint32_t w = narrow2<T>(a, c);
                    parts[r][k][j >> 1] = w;
                    a -= wide_lo<T>(w);
                    c -= wide_hi<T>(w);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 16; j++)
#pragma unroll
            for (int w = 0; w < CT / 2; w++) vt[j][w] = 16 * g4 + j < count ? vt[j][w] : 0u;
#pragma unroll
        for (int c = 0; c < CT; c++) {
            uint32_t a[8];  // tokens 2 k and 2 k + 1 of channel CT n + c
#pragma unroll
            for (int k = 0; k < 8; k++)
                a[k] = __builtin_amdgcn_perm(vt[2 * k + 1][c >> 1], vt[2 * k][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int r = 0; r < R; r++) {
                float4v acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < kParts; k++)
#pragma unroll
                    for (int h8 = 0; h8 < 2; h8++)
                        acc = product<T>(make_uint4(a[4 * h8], a[4 * h8 + 1], a[4 * h8 + 2], a[4 * h8 + 3]),
                                         make_uint4(parts[r][k][4 * h8], parts[r][k][4 * h8 + 1], parts[r][k][4 * h8 + 2], parts[r][k][4 * h8 + 3]), acc);
#pragma unroll
                for (int k = 0; k < 4; k++) o[r][c][k] = fmaf(o[r][c][k], alpha[r], acc[k]);
            }
        }
    }

    // Lane (n, g4) holds channels CT (4 g4 + k) + c of row 16 r + n.
    __device__ __forceinline__ void store(int b, int h) {
#pragma unroll
        for (int r = 0; r < R; r++) {
            const float sum = sum_rows(l[r]), f = sum == 0.f ? 0.f : (1.f / kVUnit<T>) / sum;
            const int row = 16 * r + n;
            if (row >= p.rows) continue;
            uint16_t *out = p.a.out + ((size_t)b * p.q_len + q_place[r]) * p.a.out_stride + (size_t)(h * p.g.G + row - q_place[r] * p.g.G) * D;
#pragma unroll
            for (int k = 0; k < 4; k++) {
                uint32_t w[CT / 2];
#pragma unroll
                for (int c = 0; c < CT; c += 2) w[c >> 1] = narrow2<T>(o[r][c][k] * f, o[r][c + 1][k] * f);
                uint32_t *at = reinterpret_cast<uint32_t *>(out + CT * (4 * g4 + k));
                if constexpr (CT == 8) *reinterpret_cast<uint4 *>(at) = make_uint4(w[0], w[1], w[2], w[3]);
                else *reinterpret_cast<uint2 *>(at) = make_uint2(w[0], w[1]);
            }
        }
    }
    __device__ __forceinline__ void park(float *slot) {
#pragma unroll
        for (int r = 0; r < R; r++) {
            const float sum = sum_rows(l[r]);
            const int row = 16 * r + n;
            if (row >= p.rows) continue;
            float *at = slot + row * partial_pitch(D);
#pragma unroll
            for (int k = 0; k < 4; k++)
#pragma unroll
                for (int c = 0; c < CT; c += 4)
                    *reinterpret_cast<float4 *>(at + CT * (4 * g4 + k) + c) =
                        make_float4(o[r][c][k], o[r][c + 1][k], o[r][c + 2][k], o[r][c + 3][k]);
            if (g4 == 0) {
                at[D] = m[r];
                at[D + 1] = sum;
            }
        }
    }
};

__device__ __forceinline__ void store_agent2(float *p, float a, float b) {
    __hip_atomic_store(reinterpret_cast<unsigned long long *>(p), (unsigned long long)__float_as_uint(b) << 32 | __float_as_uint(a),
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_agent2(const float *p) {
    const unsigned long long w = __hip_atomic_load(reinterpret_cast<const unsigned long long *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32)));
}

constexpr size_t kDecodeLdsBytes = 159 * 1024;  // what the kernels may have apart from their own few words

template <int T, int D>
__device__ __forceinline__ void store_row4(const DecodeArgs &p, int b, int h, int row, int c, const float (&o)[4], float sum) {
    const float f = sum == 0.f ? 0.f : (1.f / kVUnit<T>) / sum;
    const int place = place_of(p, row);
    uint16_t *out = p.a.out + ((size_t)b * p.q_len + place) * p.a.out_stride + (size_t)(h * p.g.G + row - place * p.g.G) * D + c;
    *reinterpret_cast<uint2 *>(out) = make_uint2(narrow2<T>(o[0] * f, o[1] * f), narrow2<T>(o[2] * f, o[3] * f));
}

template <int T, int C, int D, int R, int W>
__global__ __launch_bounds__(64 * W) void paged_decode_kernel(DecodeArgs p) {
    constexpr int kWaves = W, kThreads = 64 * kWaves, kSlots = 2 * kWaves, kPitch = partial_pitch(D), kQuads = D / 4;
    extern __shared__ __align__(16) float s_dyn[];
    __shared__ int4 s_of[kSlots];  // whose state is parked: sequence (-1: none), head, the head's first unit and how many have an owner
    __shared__ uint32_t s_last[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int slot_floats = p.rows * kPitch;
    uint32_t *before = reinterpret_cast<uint32_t *>(s_dyn + max(kSlots * slot_floats, kThreads * 6));  // units of one head of the sequences before

    // Units of work of one head of a sequence: a page is one, an unfinished block `kTailUnits` (none: an empty place, or one that
    // does not fit).  Every wave takes the sums for itself and leaves the same words in LDS, so nobody waits.
    auto sane = [&](int len, int tail) {
        return (unsigned)len <= (unsigned)p.g.max_pages * kPBT && (len % kPBT == 0 || (unsigned)tail < (unsigned)p.g.n_tails);
    };
    auto pages_of = [&](int len) { return len / kPBT - tiles_of(len, p.q_len, p.a.window).first; };
    const bool few = p.g.batch <= 64;  // then a sequence is a lane, and nothing goes through LDS
    uint32_t sum = 0, lane_units = 0, lane_before = 0;
    int lane_len = 0, lane_tail = 0;
    for (int base = 0; base < p.g.batch; base += 64) {
        lane_units = 0;
        if (base + lane < p.g.batch) {
            const int len = p.g.lens[base + lane], tail = p.g.tails[base + lane];
            asm volatile("" ::"v"(tail));  // both are on their way at once
            if (sane(len, tail) && len > 0) lane_units = pages_of(len) + (len % kPBT ? kTailUnits : 0);
            lane_len = len;
            lane_tail = tail;
        }
        lane_before = wave_excl_scan(lane_units, lane);
        if (!few && base + lane < p.g.batch) before[base + lane] = sum + lane_before;
        sum += __builtin_amdgcn_readlane(lane_before + lane_units, 63);
    }
    if (!few && lane == 0) before[p.g.batch] = sum;
    if (lane < 2) s_of[2 * wave + lane].x = -1;
    wave_sync();
    auto before_of = [&](int b) { return (uint32_t)(few ? __builtin_amdgcn_readlane((int)lane_before, b) : uniform((int)before[b])); };
    auto units_of = [&](int b) { return (uint32_t)(few ? __builtin_amdgcn_readlane((int)lane_units, b) : uniform((int)(before[b + 1] - before[b]))); };
    // Empty places: zeros; those that do not fit: NaN.
    auto fill_empty = [&]() {
        for (int b = blockIdx.x; b < p.g.batch; b += gridDim.x) {
            if (units_of(b) != 0) continue;
            const int len = p.g.lens[b];
            const bool ok = sane(len, p.g.tails[b]);
            if (!ok && tid == 0) flag(p.g.fault, (unsigned)len <= (unsigned)p.g.max_pages * kPBT ? kFaultTail : kFaultLength);
            const uint32_t w = ok ? 0u : kNanBits<T> * 0x10001u;
            const int per_row = p.g.H * p.g.G * D / 8;
            for (int i = tid; i < p.q_len * per_row; i += kThreads)
                *reinterpret_cast<uint4 *>(p.a.out + ((size_t)b * p.q_len + i / per_row) * p.a.out_stride + (size_t)(i % per_row) * 8) = make_uint4(w, w, w, w);
        }
    };
    const uint32_t H = p.g.H, total = sum * H;
    const uint32_t active = min((uint32_t)gridDim.x, (total + kLeastUnits - 1) / kLeastUnits), wg = blockIdx.x;
    if (wg >= active) {
        fill_empty();
        return;
    }
    const Deal deal(total, active);
    const uint32_t wg_begin = deal.begin(wg), wg_end = deal.begin(wg + 1);
    const Deal inner(wg_end - wg_begin, kWaves);
    uint32_t t = uniform((int)(wg_begin + inner.begin(wave)));
    const uint32_t t_end = uniform((int)(wg_begin + inner.begin(wave + 1)));

    Wave<T, C, D, R> w(p, lane);
    int b = 0, parked = 0;
    if (t < t_end) {  // the sequence of the first unit
        if (few) {
            b = __builtin_ctzll(__builtin_amdgcn_ballot_w64((lane_before + lane_units) * H > t));
        } else {
            int lo = 0, hi = p.g.batch;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (before_of(mid) * H <= t) lo = mid; else hi = mid;
            }
            b = lo;
        }
    }
    while (t < t_end) {
        const uint32_t base = before_of(b), tiles = units_of(b);
        if ((base + tiles) * H <= t) {
            b++;
            continue;
        }
        const uint32_t in_seq = t - base * H, h = in_seq / tiles, i0 = in_seq - h * tiles, i1 = min(tiles, i0 + (t_end - t));
        const int len = few ? __builtin_amdgcn_readlane(lane_len, b) : uniform(p.g.lens[b]);
        t += i1 - i0;
        const uint32_t pages = pages_of(len), tail = len % kPBT ? 1 : 0;
        if (i0 >= pages + tail) continue;  // the rest of an unfinished block's units: it belongs to the first one's owner
        if (i0 < pages) w.run(b, (int)h, tiles_of(len, p.q_len, p.a.window).first, (int)i0, (int)min(i1, pages), len);
        if (tail && i0 <= pages && pages < i1) {
            const int slot = few ? __builtin_amdgcn_readlane(lane_tail, b) : uniform(p.g.tails[b]);
            w.unfinished(b, (int)h, len, slot, i0 == pages);
        }
        if (i0 == 0 && i1 >= pages + tail) {
            w.store(b, (int)h);
        } else {
            w.park(s_dyn + (size_t)(2 * wave + parked) * slot_floats);
            if (lane == 0) s_of[2 * wave + parked] = make_int4(b, (int)h, (int)(base * H + h * tiles), (int)(pages + tail));
            parked++;
        }
    }
    fill_empty();
    __syncthreads();

    // Join the parked states of each head; a head that other workgroups have a part of leaves its state in the workspace.
    int open = 0, open_b[2], open_h[2];
    uint32_t open_from[2], open_parts[2];  // workgroups that the head is spread over
    const int4 of = s_of[min(lane, kSlots - 1)];  // a slot a lane
    uint32_t left = (uint32_t)__builtin_amdgcn_ballot_w64(of.x >= 0 && lane < kSlots);
    while (left) {
        const int s0 = __builtin_ctz(left);
        const int sb = __builtin_amdgcn_readlane(of.x, s0), sh = __builtin_amdgcn_readlane(of.y, s0);
        const uint32_t begin = __builtin_amdgcn_readlane(of.z, s0), units = __builtin_amdgcn_readlane(of.w, s0);
        const uint32_t mine = (uint32_t)__builtin_amdgcn_ballot_w64(of.x == sb && of.y == sh && lane < kSlots);
        left &= ~mine;
        const bool complete = begin >= wg_begin && begin + units <= wg_end;
        for (int item = tid; item < p.rows * kQuads; item += kThreads) {
            const int row = item / kQuads, c = (item - row * kQuads) * 4;
            const float *at = s_dyn + row * kPitch;
            float top = kLowestRef, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
            for (uint32_t rest = mine; rest;) {  // four states on their way at once
                float m[4], l[4];
                float4 v[4];
                float now = top;
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    const bool have = rest != 0;
                    const float *from = at + (have ? __builtin_ctz(rest) : s0) * slot_floats;
                    rest &= rest - 1;
                    m[x] = have ? from[D] : -INFINITY;
                    l[x] = from[D + 1];
                    v[x] = *reinterpret_cast<const float4 *>(from + c);
                }
#pragma unroll
                for (int x = 0; x < 4; x++) now = fmaxf(now, m[x]);
                float f = __builtin_amdgcn_exp2f(top - now);
                top = now;
                sum *= f;
#pragma unroll
                for (int k = 0; k < 4; k++) acc[k] *= f;
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    f = __builtin_amdgcn_exp2f(m[x] - now);
                    sum = fmaf(l[x], f, sum);
                    acc[0] = fmaf(v[x].x, f, acc[0]);
                    acc[1] = fmaf(v[x].y, f, acc[1]);
                    acc[2] = fmaf(v[x].z, f, acc[2]);
                    acc[3] = fmaf(v[x].w, f, acc[3]);
                }
            }
            if (complete) {
                store_row4<T, D>(p, sb, sh, row, c, acc, sum);
            } else {
                float *to = p.a.partials + ((size_t)(2 * wg + (begin < wg_begin ? 0 : 1)) * p.rows + row) * kPitch;
                store_agent2(to + c, acc[0], acc[1]);
                store_agent2(to + c + 2, acc[2], acc[3]);
                if (c == 0) store_agent2(to + D, top, sum);
            }
        }
        if (!complete) {
            const int k = open++ & 1;  // two at most: the one that began before, the one that goes on behind
            open_b[k] = sb;
            open_h[k] = sh;
            open_from[k] = deal.owner(begin);  // here, while the states are on their way
            open_parts[k] = deal.owner(begin + units - 1) - open_from[k] + 1;
        }
    }
    if (!open) return;
    // every wave: its partial stores have completed before the barrier is passed
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    for (int k = 0; k < open; k++) {
        const uint32_t from = open_from[k], parts = open_parts[k];
        if (tid == 0) {
            const uint32_t ticket = __hip_atomic_fetch_add(p.a.tickets + from, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last[k] = ticket == parts - 1;
        }
        __syncthreads();
        if (!s_last[k]) continue;
        // The last to arrive: groups of threads take the parts in turn, everything that a thread needs of four parts on its way at
        // once; the groups meet in LDS.
        const int items = p.rows * kQuads, groups = max(1, min(kThreads / items, (int)(parts + 3) / 4));
        for (int at = 0; at < items; at += kThreads) {  // one round, unless there are more items than threads
            const int local = groups > 1 ? tid % items : tid, group = groups > 1 ? tid / items : 0, item = at + local;
            const bool live = item < items && group < groups;
            const int row = live ? item / kQuads : 0, c = live ? (item - row * kQuads) * 4 : 0;
            float top = kLowestRef, total_l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
            if (live) {
                for (uint32_t i = group; i < parts; i += 4 * groups) {
                    float2 ml[4], lo[4], hi[4];
#pragma unroll
                    for (int x = 0; x < 4; x++) {
                        const uint32_t part = min(i + x * groups, parts - 1);
                        const float *v = p.a.partials + ((size_t)(2 * (from + part) + (part == 0 ? 1 : 0)) * p.rows + row) * kPitch;
                        ml[x] = load_agent2(v + D);
                        lo[x] = load_agent2(v + c);
                        hi[x] = load_agent2(v + c + 2);
                    }
                    float now = top;
#pragma unroll
                    for (int x = 0; x < 4; x++) {
                        if (i + x * groups >= parts) ml[x] = make_float2(-INFINITY, 0.f);
                        now = fmaxf(now, ml[x].x);
                    }
                    const float old = __builtin_amdgcn_exp2f(top - now);
                    top = now;
                    total_l *= old;
#pragma unroll
                    for (int y = 0; y < 4; y++) acc[y] *= old;
#pragma unroll
                    for (int x = 0; x < 4; x++) {
                        const float f = __builtin_amdgcn_exp2f(ml[x].x - now);
                        total_l = fmaf(ml[x].y, f, total_l);
                        acc[0] = fmaf(lo[x].x, f, acc[0]);
                        acc[1] = fmaf(lo[x].y, f, acc[1]);
                        acc[2] = fmaf(hi[x].x, f, acc[2]);
                        acc[3] = fmaf(hi[x].y, f, acc[3]);
                    }
                }
            }
            if (groups > 1) {
                float *mine = s_dyn + 6 * tid;
                mine[0] = top; mine[1] = total_l; mine[2] = acc[0]; mine[3] = acc[1]; mine[4] = acc[2]; mine[5] = acc[3];
                __syncthreads();
                if (live && group == 0) {
                    for (int gr = 1; gr < groups; gr++) {
                        const float *v = s_dyn + 6 * (gr * items + local);
                        const float now = fmaxf(top, v[0]), old = __builtin_amdgcn_exp2f(top - now), f = __builtin_amdgcn_exp2f(v[0] - now);
                        top = now;
                        total_l = fmaf(v[1], f, total_l * old);
#pragma unroll
                        for (int x = 0; x < 4; x++) acc[x] = fmaf(v[2 + x], f, acc[x] * old);
                    }
                }
            }
            if (live && group == 0) store_row4<T, D>(p, open_b[k], open_h[k], row, c, acc, total_l);
        }
        if (tid == 0) __hip_atomic_store(p.a.tickets + from, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
    }
}

template <int T, int C, int D, int R, int W>
hipError_t launch_waves(const DecodeArgs &p, int max_len, hipStream_t s) {
    constexpr int kThreads = 64 * W;
    const size_t states = (size_t)2 * W * p.rows * partial_pitch(D), join = (size_t)kThreads * 6;
    const size_t lds = 4 * ((states > join ? states : join) + p.g.batch + 1);
    auto kernel = paged_decode_kernel<T, C, D, R, W>;
    static std::atomic<uint64_t> allowed{0};
    hipError_t e = allow_lds(reinterpret_cast<const void *>(kernel), kDecodeLdsBytes, allowed);
    if (e != hipSuccess) return e;
    if (lds > kDecodeLdsBytes) return hipErrorInvalidValue;
    // units of work that there could be: no more workgroups than they can busy
    const int pages = max_len > 0 && max_len < p.g.max_pages * kPBT ? (max_len + kPBT - 1) / kPBT : p.g.max_pages;
    const size_t most = (size_t)p.g.batch * p.g.H * (pages + kTailUnits), wgs = (most + kLeastUnits - 1) / kLeastUnits;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(wgs < (size_t)kDecodeWGs ? wgs : (size_t)kDecodeWGs)), dim3(kThreads), lds, s, p);
    return hipGetLastError();
}

// Waves of a workgroup, one of which fills a CU: their states of two heads each have to fit the LDS, and twelve with fewer registers
// each take a third longer over 32 heads x 32768 tokens (61 us against 46).
template <int T, int C, int D, int R>
hipError_t launch(const DecodeArgs &p, int max_len, hipStream_t s) {
    return launch_waves<T, C, D, R, R == 1 ? 8 : 4>(p, max_len, s);
}

}  // namespace

hipError_t launch_paged_decode(const PagedGeo &g, const PagedAttn &a, int q_len, int max_len, int head_dim, int data_type, int code_type,
                               hipStream_t s) {
    DecodeArgs p = {g, a, q_len, q_len * g.G, (65536u + g.G - 1) / g.G};
    auto by_rows = [&](auto t, auto c, auto d) {
        if (p.rows <= 16) return launch<decltype(t)::value, decltype(c)::value, decltype(d)::value, 1>(p, max_len, s);
        return launch<decltype(t)::value, decltype(c)::value, decltype(d)::value, 2>(p, max_len, s);
    };
    auto by_dim = [&](auto t, auto c) {
        if (head_dim == 64) return by_rows(t, c, std::integral_constant<int, 64>());
        return by_rows(t, c, std::integral_constant<int, 128>());
    };
    auto by_code = [&](auto t) {
        if (code_type == kI8) return by_dim(t, std::integral_constant<int, kI8>());
        return by_dim(t, std::integral_constant<int, kE4M3>());
    };
    if (data_type == kF16) return by_code(std::integral_constant<int, kF16>());
    return by_code(std::integral_constant<int, kBF16>());
}

}  // namespace kvc
