// Appending to the paged cache of 8-bit codes: rotate, round to 16 bits, and either quantize a block that ends into its page or
// store the unfinished block's new rows in its tail; the queries of the same tokens are rotated along.
//
// Bound by HBM for prompts (16421 tokens of 8 KV and 32 query heads: 379 MB in 76 us, 5.0 TB/s, what a large copy reaches; 65 to 67
// where the caches hold some of it) and by the launch for single tokens (one sequence: 2.6 us a call, replayed).  One workgroup of
// 16 * D / 16 threads owns a block of 64 tokens of one KV head: thread (rg, item) holds four consecutive tokens x two chunks of
// eight channels of K and of V in registers
// (all of its sixteen 16-byte loads are on their way together), so that the block's largest magnitudes are one reduction
// and every value is read once.  The two chunks are the partners of the split rotation, so both results of a pair come
// from registers.  The four tokens make the bytes of a V channel's word; V leaves through LDS because its page has the
// channels outermost (attention multiplies by V with the tokens as the inner dimension).
//
// A tail is read (tokens from before the call) and written (tokens behind the block that ends) by the same workgroup, the one
// that owns the sequence's first touched block; nobody else may write there while it reads.
#include "huff_decode.cuh"
#include "paged.cuh"

namespace kvc {

namespace {

// Eight cosines and sines of pairs 8 * item .. + 7 at the positions of token t (one per axis); false: a position is out of range.
struct Turn {
    float c[8], s[8];
};
__device__ __forceinline__ bool load_turn(Turn &r, const PagedNew &n, int item, int t, int own_pos) {
    bool fine = true;
#pragma unroll
    for (int half = 0; half < 2; half++) {  // four pairs have one axis
        const int p = 8 * item + 4 * half;
        int pos = own_pos;
        if (n.positions) pos = n.positions[(size_t)((p >= n.edge[0]) + (p >= n.edge[1])) * n.n_tokens + t];
        if ((unsigned)pos >= (unsigned)n.n_positions) {
            fine = false;
            pos = 0;
        }
        const float *row = n.cos_sin + (size_t)pos * n.rot_dim + p;
        const float4 c = *reinterpret_cast<const float4 *>(row), s = *reinterpret_cast<const float4 *>(row + n.rot_dim / 2);
        r.c[4 * half] = c.x; r.c[4 * half + 1] = c.y; r.c[4 * half + 2] = c.z; r.c[4 * half + 3] = c.w;
        r.s[4 * half] = s.x; r.s[4 * half + 1] = s.y; r.s[4 * half + 2] = s.z; r.s[4 * half + 3] = s.w;
    }
    return fine;
}

// The chunks (eight channels each) of an item: partners of the split rotation, neighbours otherwise.
__device__ __forceinline__ void chunks_of(const PagedNew &n, int item, int &c0, int &c1) {
    const int pairs = n.rot_dim / 16;
    if (item < pairs && !n.interleaved) {
        c0 = item;
        c1 = item + pairs;
    } else {
        c0 = 2 * item;
        c1 = c0 + 1;
    }
}

// (a, b) -> (a cos - b sin, b cos + a sin) for the item's eight pairs, binary32, one rounding each.
template <int T>
__device__ __forceinline__ void turn(uint32_t (&x)[2][4], const Turn &r, bool interleaved) {
    if (interleaved) {
#pragma unroll
        for (int c = 0; c < 2; c++)
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float a = wide_lo<T>(x[c][w]), b = wide_hi<T>(x[c][w]), co = r.c[4 * c + w], si = r.s[4 * c + w];
                x[c][w] = narrow2<T>(a * co - b * si, b * co + a * si);
            }
    } else {
#pragma unroll
        for (int w = 0; w < 4; w++) {
            const float a0 = wide_lo<T>(x[0][w]), a1 = wide_hi<T>(x[0][w]), b0 = wide_lo<T>(x[1][w]), b1 = wide_hi<T>(x[1][w]);
            x[0][w] = narrow2<T>(a0 * r.c[2 * w] - b0 * r.s[2 * w], a1 * r.c[2 * w + 1] - b1 * r.s[2 * w + 1]);
            x[1][w] = narrow2<T>(b0 * r.c[2 * w] + a0 * r.s[2 * w], b1 * r.c[2 * w + 1] + a1 * r.s[2 * w + 1]);
        }
    }
}

__device__ __forceinline__ void load16(uint32_t (&w)[4], const uint16_t *p) {
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
}
__device__ __forceinline__ void store16(uint16_t *p, const uint32_t (&w)[4]) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// ... past the caches
__device__ __forceinline__ void stream16(uint16_t *p, const uint32_t (&w)[4]) {
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    const u4 v = {w[0], w[1], w[2], w[3]};
    __builtin_nontemporal_store(v, reinterpret_cast<u4 *>(p));
}
// Values that are Inf or NaN: zero in V, and a NaN in the same token's K marks the token for whoever reads it.
template <int T>
__device__ __forceinline__ bool poison(uint32_t (&k)[2][4], uint32_t (&v)[2][4]) {
    uint32_t mk = 0, mv = 0;
#pragma unroll
    for (int c = 0; c < 2; c++)
#pragma unroll
        for (int w = 0; w < 4; w++) {
            mk = max16(mk, k[c][w] & 0x7fff7fffu);
            mv = max16(mv, v[c][w] & 0x7fff7fffu);
        }
    const uint32_t m = max16(mk, mv);
    if (max(m & 0xffffu, m >> 16) < kInfBits<T>) return false;
    k[0][0] = (k[0][0] & 0xffff0000u) | kNanBits<T>;
#pragma unroll
    for (int c = 0; c < 2; c++)
#pragma unroll
        for (int w = 0; w < 4; w++) {
            if ((v[c][w] & 0x7fffu) >= kInfBits<T>) v[c][w] &= 0xffff0000u;
            if (((v[c][w] >> 16) & 0x7fffu) >= kInfBits<T>) v[c][w] &= 0xffffu;
        }
    return true;
}

// Four bytes of codes of four values times inv.  int8: adding 1.5 * 2^23 rounds the product to the nearest even integer, which
// is the sum's low byte.
template <int C>
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d, float inv) {
    if constexpr (C == kI8) {
        constexpr float kRound = 12582912.f;
        const uint32_t x = __float_as_uint(a * inv + kRound), y = __float_as_uint(b * inv + kRound),
                       z = __float_as_uint(c * inv + kRound), w = __float_as_uint(d * inv + kRound);
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w, z, 0x0c0c0400u), __builtin_amdgcn_perm(y, x, 0x0c0c0400u), 0x05040100u);
    } else {
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, r, true);
    }
}

constexpr float kTinyBlock = 7.888609052210118e-31f;  // 2^-100: below it, 127 / amax could overflow
template <int C>
constexpr float kMostCode = C == kI8 ? 127.f : 448.f;

constexpr int kRowGroups = 16;   // four tokens each
// Rows of queries per thread (16421 tokens, 8 KV and 32 query heads, with 1, 2, 4, 8: 72.3 66.9 67.4 67.6 us).
constexpr int kQRows = 2;
constexpr int kVPitch = 17;      // words of a V channel in LDS: 16, and one so that the writers of eight channels hit eight banks

template <int T, int C, int D>
__global__ __launch_bounds__(kRowGroups * D / 16) void paged_append_kernel(PagedGeo g, PagedNew n, int block_units, Divide by_heads, Divide by_q_heads) {
    constexpr int kItems = D / 16, kThreads = kRowGroups * kItems;
    __shared__ uint32_t s_v[D * kVPitch];
    __shared__ uint32_t s_max[2];
    const int tid = threadIdx.x, item = tid % kItems, rg = tid / kItems, lane = tid & 63;
    const int pairs16 = n.rot_dim / 16;
    const bool turned = item < pairs16;
    int c0, c1;
    chunks_of(n, item, c0, c1);
    c0 *= 8;
    c1 *= 8;

    if ((int)blockIdx.x >= block_units) {
        // queries of chunks: kQRows rows (token, head) per thread, which are heads of one token where they go into a token's
        // heads evenly; then its cosines and sines are read once
        const int Hq = g.H * g.G;
        const uint32_t rows = (uint32_t)n.n_tokens * (uint32_t)Hq;
        const uint32_t r0 = ((blockIdx.x - block_units) * (uint32_t)kRowGroups + rg) * kQRows;
        const int n_first = n.starts[0], n_used = n.starts[g.batch];
        uint32_t x[kQRows][2][4];
        int tok[kQRows], head[kQRows];
#pragma unroll
        for (int k = 0; k < kQRows; k++) {
            const uint32_t r = r0 + k;
            tok[k] = (int)by_q_heads.of(r);
            head[k] = (int)(r - (uint32_t)tok[k] * (uint32_t)Hq);
            if (r >= rows || tok[k] >= n_used || tok[k] < n_first) tok[k] = -1;
            if (tok[k] < 0) continue;
            const uint16_t *p = n.q + (size_t)tok[k] * n.q_stride + head[k] * D;
            load16(x[k][0], p + c0);
            load16(x[k][1], p + c1);
        }
        bool fine = true, ok = true;
        int b = -1;
        Turn t;
#pragma unroll
        for (int k = 0; k < kQRows; k++) {
            if (tok[k] < 0) continue;
            if (turned) {
                if (k == 0 || tok[k] != tok[k - 1]) {
                    int pos = 0;
                    if (!n.positions) {
                        if (b < 0) {  // the last sequence that starts at or before the token
                            int lo = 0, hi = g.batch;
                            while (hi - lo > 1) {
                                const int mid = (lo + hi) >> 1;
                                if (n.starts[mid] <= tok[k]) lo = mid; else hi = mid;
                            }
                            b = lo;
                        } else {
                            while (b + 1 < g.batch && n.starts[b + 1] <= tok[k]) b++;
                        }
                        pos = g.lens[b] - n.starts[b + 1] + tok[k];
                    }
                    ok = load_turn(t, n, item, tok[k], pos);
                }
                turn<T>(x[k], t, n.interleaved);
                if (!ok) {
                    x[k][0][0] = x[k][1][0] = kNanBits<T> * 0x10001u;
                    fine = false;
                }
            }
            uint16_t *p = n.q_out + (size_t)tok[k] * n.q_out_stride + head[k] * D;
            if (n.stream_q) {
                stream16(p + c0, x[k][0]);
                stream16(p + c1, x[k][1]);
            } else {
                store16(p + c0, x[k][0]);
                store16(p + c1, x[k][1]);
            }
        }
        if (!fine) flag(g.fault, kFaultPosition);
        return;
    }

    // which block of which sequence
    int unit = (int)by_heads.of(blockIdx.x);
    const int h = blockIdx.x - unit * g.H;
    int b, start, fresh, len, tail;  // first new row, new tokens
    bool bad = false;
    if (!n.starts) {
        b = unit;
        unit = 0;
        len = g.lens[b];
        tail = g.tails[b];
        fresh = len == 0 ? 0 : 1;
        start = b;
        bad = len < 0 || len > g.max_pages * kPBT;
    } else {
        b = -1;
        for (int base = 0; base < g.batch; base += 64) {
            int blocks = 0, s0 = 0, s1 = 0, l = 0, t = 0;
            if (base + lane < g.batch) {
                s0 = n.starts[base + lane];
                s1 = n.starts[base + lane + 1];
                l = g.lens[base + lane];
                t = g.tails[base + lane];
                asm volatile("" ::"v"(l), "v"(t));  // all on their way at once
                if (s0 < 0 || s1 < s0 || s1 > n.n_tokens || l < s1 - s0 || l > g.max_pages * kPBT) {
                    if (blockIdx.x == 0 && tid < 64) flag(g.fault, kFaultLength);
                } else if (s1 > s0) {
                    blocks = (l - 1) / kPBT - (l - (s1 - s0)) / kPBT + 1;
                }
            }
            const int before = (int)wave_excl_scan((uint32_t)blocks, lane);
            const unsigned long long past = __builtin_amdgcn_ballot_w64(before + blocks > unit);
            if (b >= 0) continue;
            if (past) {
                const int at = __builtin_ctzll(past);
                b = base + at;
                unit -= __builtin_amdgcn_readlane(before, at);
                start = __builtin_amdgcn_readlane(s0, at);
                fresh = __builtin_amdgcn_readlane(s1, at) - start;
                len = __builtin_amdgcn_readlane(l, at);
                tail = __builtin_amdgcn_readlane(t, at);
                if (blockIdx.x) break;  // the first workgroup looks at all sequences
            } else {
                unit -= __builtin_amdgcn_readlane(before + blocks, 63);
            }
        }
        if (b < 0) return;
    }

    if (!n.starts && n.q && fresh) {
        // single tokens: the queries of this KV head, first by the half of the threads that does not have the token's K and V (one
        // sequence, groups of 4, replayed, by the one half and the other: 2.6 and 3.3 us a call)
        for (int i = tid ^ ((len - 1) % kPBT < kPBT / 2 ? kThreads / 2 : 0); i < g.G * kItems; i += kThreads) {
            const int qi = i % kItems, head = h * g.G + i / kItems;
            int d0, d1;
            chunks_of(n, qi, d0, d1);
            uint32_t x[2][4];
            const uint16_t *p = n.q + (size_t)b * n.q_stride + (size_t)head * D;
            load16(x[0], p + 8 * d0);
            load16(x[1], p + 8 * d1);
            if (qi < pairs16) {
                Turn t;
                const bool ok = load_turn(t, n, qi, b, len - 1);
                turn<T>(x, t, n.interleaved);
                if (!ok) {
                    x[0][0] = x[1][0] = kNanBits<T> * 0x10001u;
                    flag(g.fault, kFaultPosition);
                }
            }
            uint16_t *o = n.q_out + (size_t)b * n.q_out_stride + (size_t)head * D;
            store16(o + 8 * d0, x[0]);
            store16(o + 8 * d1, x[1]);
        }
    }
    if (bad) {
        if (tid == 0 && h == 0) flag(g.fault, kFaultLength);
        return;
    }
    if (fresh == 0) return;
    if ((unsigned)tail >= (unsigned)g.n_tails) {
        if (tid == 0) flag(g.fault, kFaultTail);
        return;
    }
    const int past = len - fresh, first = past / kPBT, last = len / kPBT;  // `last`: the unfinished block, if len % 64
    int blk = first + unit;
    if (blk == last && unit) return;  // the workgroup of the first block stores the tail
    const int32_t *pages = g.table + (size_t)b * g.max_pages;
    const int page = blk == last ? 0 : pages[blk];  // long before it is needed
    const int page_of_lane = unit == 0 && first + lane < last ? pages[first + lane] : 0;
    const size_t tail_at = ((size_t)tail * g.H + h) * kPBT * D;

    uint32_t kx[4][2][4], vx[4][2][4];
    bool odd = false, off = false;  // non-finite values, positions out of range
    // rows [lo, hi) of block `blk`, four per thread; rows below `lo` are in the tail if `from_tail`
    auto fetch = [&](int blk_, int lo, int hi, bool from_tail) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int r = 4 * rg + i;
            const uint16_t *kp, *vp;
            if (r >= lo && r < hi) {
                const size_t t = (size_t)(start + blk_ * kPBT + r - past);
                kp = n.k + t * n.k_stride + h * D;
                vp = n.v + t * n.v_stride + h * D;
            } else if (r < lo && from_tail) {
                kp = g.k_tail + tail_at + r * D;
                vp = g.v_tail + tail_at + r * D;
            } else {
                continue;
            }
            load16(kx[i][0], kp + c0);
            load16(kx[i][1], kp + c1);
            load16(vx[i][0], vp + c0);
            load16(vx[i][1], vp + c1);
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int r = 4 * rg + i;
            if (r < lo || r >= hi) continue;
            if (turned) {
                Turn t;
                const int place = blk_ * kPBT + r;
                const bool ok = load_turn(t, n, item, start + place - past, place);
                turn<T>(kx[i], t, n.interleaved);
                if (!ok) {
                    kx[i][0][0] = kNanBits<T> * 0x10001u;
                    off = true;
                }
            }
            odd |= poison<T>(kx[i], vx[i]);
        }
    };
    auto keep = [&](int lo, int hi) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int r = 4 * rg + i;
            if (r < lo || r >= hi) continue;
            store16(g.k_tail + tail_at + r * D + c0, kx[i][0]);
            store16(g.k_tail + tail_at + r * D + c1, kx[i][1]);
            store16(g.v_tail + tail_at + r * D + c0, vx[i][0]);
            store16(g.v_tail + tail_at + r * D + c1, vx[i][1]);
        }
    };
    if (blk == last) {
        fetch(blk, past - blk * kPBT, len - blk * kPBT, false);
        keep(past - blk * kPBT, len - blk * kPBT);
    } else {
        const int begun = unit == 0 ? past - first * kPBT : 0;
        fetch(blk, begun, kPBT, true);
        // the largest magnitudes: 16-bit patterns without their sign are ordered like the values they stand for
        uint32_t mk = 0, mv = 0;
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int c = 0; c < 2; c++)
#pragma unroll
                for (int w = 0; w < 4; w++) {
                    mk = max16(mk, kx[i][c][w] & 0x7fff7fffu);
                    mv = max16(mv, vx[i][c][w] & 0x7fff7fffu);
                }
        uint32_t m = max(mk & 0xffffu, mk >> 16) | max(mv & 0xffffu, mv >> 16) << 16;
        m = max16(m, dpp_u<kDppXor1>(m));
        m = max16(m, dpp_u<kDppXor2>(m));
        m = max16(m, dpp_u<kDppHalfMirror>(m));
        m = max16(m, dpp_u<kDppMirror>(m));
        m = max16(max16(__builtin_amdgcn_readlane(m, 0), __builtin_amdgcn_readlane(m, 16)),
                  max16(__builtin_amdgcn_readlane(m, 32), __builtin_amdgcn_readlane(m, 48)));
        if constexpr (kThreads > 64) {
            if (lane == 0) s_max[tid >> 6] = m;
            __syncthreads();
            m = max16(s_max[0], s_max[1]);
        }
        const bool nan_k = (m & 0xffffu) >= kInfBits<T>;
        const float ak = wide_lo<T>(m), av = wide_hi<T>(m);
        const bool live_k = !nan_k && ak >= kTinyBlock, live_v = av >= kTinyBlock;
        const float ik = live_k ? kMostCode<C> / ak : 0.f, iv = live_v ? kMostCode<C> / av : 0.f;
        const bool page_ok = (unsigned)page < (unsigned)g.n_pages;
        const size_t tile = ((size_t)page * g.H + h) * kPBT * D;
        if (page_ok) {
            if (tid == 0) {
                float2 sc;
                sc.x = nan_k ? __uint_as_float(0x7fc00000u) : live_k ? ak / kMostCode<C> : 0.f;
                sc.y = live_v ? av / kMostCode<C> : 0.f;
                *reinterpret_cast<float2 *>(g.scales + ((size_t)page * g.H + h) * 2) = sc;
            }
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int c = 0; c < 2; c++) {
                    uint2 w;
                    w.x = code4<C>(wide_lo<T>(kx[i][c][0]), wide_hi<T>(kx[i][c][0]), wide_lo<T>(kx[i][c][1]), wide_hi<T>(kx[i][c][1]), ik);
                    w.y = code4<C>(wide_lo<T>(kx[i][c][2]), wide_hi<T>(kx[i][c][2]), wide_lo<T>(kx[i][c][3]), wide_hi<T>(kx[i][c][3]), ik);
                    if (nan_k) w = make_uint2(0, 0);
                    *reinterpret_cast<uint2 *>(g.k_codes + tile + (4 * rg + i) * D + (c ? c1 : c0)) = w;
                }
#pragma unroll
            for (int c = 0; c < 2; c++)
#pragma unroll
                for (int w = 0; w < 4; w++) {
                    uint32_t *at = s_v + ((c ? c1 : c0) + 2 * w) * kVPitch + rg;
                    at[0] = code4<C>(wide_lo<T>(vx[0][c][w]), wide_lo<T>(vx[1][c][w]), wide_lo<T>(vx[2][c][w]), wide_lo<T>(vx[3][c][w]), iv);
                    at[kVPitch] = code4<C>(wide_hi<T>(vx[0][c][w]), wide_hi<T>(vx[1][c][w]), wide_hi<T>(vx[2][c][w]), wide_hi<T>(vx[3][c][w]), iv);
                }
        } else if (tid == 0) {
            flag(g.fault, kFaultPage);
        }
        __syncthreads();  // the V codes are in LDS, and the tail's old rows in registers
        if (page_ok) {
#pragma unroll
            for (int k = 0; k < D * 4 / kThreads; k++) {
                const int piece = tid + k * kThreads, ch = piece >> 2, part = (piece & 3) * 4;
                const uint32_t *from = s_v + ch * kVPitch + part;
                *reinterpret_cast<uint4 *>(g.v_codes + tile + (size_t)piece * 16) = make_uint4(from[0], from[1], from[2], from[3]);
            }
        }
        if (unit == 0 && last * kPBT < len) {
            // the tail keeps its old rows where any block of the sequence has no page: then the call can be repeated
            bool fits = (unsigned)page_of_lane < (unsigned)g.n_pages;
            for (int i = first + 64 + lane; i < last; i += 64) fits &= (unsigned)pages[i] < (unsigned)g.n_pages;
            if (__builtin_amdgcn_ballot_w64(!fits) == 0) {
                fetch(last, 0, len - last * kPBT, false);
                keep(0, len - last * kPBT);
            }
        }
    }
    if (odd) flag(g.fault, kFaultNonfinite);
    if (off) flag(g.fault, kFaultPosition);
}

template <int T, int C, int D>
void launch(const PagedGeo &g, PagedNew n, hipStream_t s) {
    // every sequence touches at most one block more than its new tokens fill, and one more where it starts inside a block
    const size_t units = n.starts ? (size_t)n.n_tokens / kPBT + 2 * (size_t)g.batch : (size_t)g.batch;
    const size_t most = n.starts && (size_t)n.n_tokens < units ? (size_t)n.n_tokens : units;
    const size_t q_rows = n.starts && n.q ? (size_t)n.n_tokens * g.H * g.G : 0;
    // rotated queries that the L2s (8 x 4 MiB) cannot keep for the attention behind go past them: 78.8 -> 66.9 us for 134 MB (79.5 ->
    // 76.1 with other tokens every time), but 19.9 -> 20.5 for 19 MB
    n.stream_q = q_rows * D * 2 > (size_t)32 << 20;
    const size_t q_units = (q_rows + kRowGroups * kQRows - 1) / (kRowGroups * kQRows);
    hipLaunchKernelGGL((paged_append_kernel<T, C, D>), dim3((unsigned)(most * g.H + q_units)), dim3(kRowGroups * D / 16), 0, s, g, n,
                       (int)(most * g.H), Divide(g.H), Divide(g.H * g.G));
}

}  // namespace

hipError_t launch_paged_append(const PagedGeo &g, const PagedNew &n, int head_dim, int data_type, int code_type, hipStream_t s) {
    auto by_code = [&](auto t, auto d) {
        if (code_type == kI8) launch<decltype(t)::value, kI8, decltype(d)::value>(g, n, s);
        else launch<decltype(t)::value, kE4M3, decltype(d)::value>(g, n, s);
    };
    auto by_dim = [&](auto t) {
        if (head_dim == 64) by_code(t, std::integral_constant<int, 64>());
        else by_code(t, std::integral_constant<int, 128>());
    };
    if (data_type == kF16) by_dim(std::integral_constant<int, kF16>());
    else by_dim(std::integral_constant<int, kBF16>());
    return hipGetLastError();
}

}  // namespace kvc
