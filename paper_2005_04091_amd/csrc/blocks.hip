// Block scores and block selection (spconv_block_scores, spconv_select_blocks).
#include "batch.h"
#include "split.h"

namespace {

constexpr float kInf = __builtin_huge_valf();

// Ones of a ballot, as a signed number.
__device__ __forceinline__ int bits(uint64_t x) { return (int)__popcll(x); }

struct ScoreArgs {
    spconv_batch B;
    const void *q;
    int64_t q_token, q_head;
    const float *sums;
    float *scores;
    int64_t items;
    int heads, group, dim, tiles;  // tiles: workgroups along the table
    Div tile_div, head_div, group_div;
    int aligned;
};

// The eight components of a row that lane part `part` holds of every 32 from d0 on: d0 + 4*part .. +4 and 16 behind
// them (the order of the components in a product is free; so the four parts' 16-byte loads of fp32 rows are neighbours).
// dim is a multiple of 8: each half is all there or not.
template <typename T>
__device__ __forceinline__ Floats<8> load_part(const T *p, int d0, int part, int dim, bool aligned) {
    Floats<8> r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int d = d0 + i * 16 + part * 4;
        Floats<4> f;
#pragma unroll
        for (int k = 0; k < 4; ++k) f.v[k] = 0.0f;
        if (d < dim) {
            if (aligned) {
                f = load_floats<T, 4>(p + d);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) f.v[k] = (float)p[d + k];
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) r.v[i * 4 + k] = f.v[k];
    }
    return r;
}

// bf16 parts of queries: bf16 ones are one part, fp16 ones (11 bits) two, fp32 ones three; exact but for fp32's
// least bits below 2^-110.
template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 3 : 2;
template <>
constexpr int kParts<__bf16> = 1;

// Parts of eight components, one 16-byte vector each.
template <typename T>
__device__ __forceinline__ void query_parts(const Floats<8> &x, u32x4_t (&p)[kParts<T>]) {
    Parts s;
#pragma unroll
    for (int i = 0; i < 4; ++i) split2(s, i, x.v[2 * i], x.v[2 * i + 1]);
    p[0] = s.h;
    if constexpr (kParts<T> > 1) p[1] = s.m;
    if constexpr (kParts<T> > 2) p[2] = s.l;
}

__device__ __forceinline__ f32x4 mma_bits(u32x4_t a, u32x4_t b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Unit (16 bytes) u of pair m's row of one part in LDS: 16 lanes read one unit of 16 rows.
template <int UPR>
__device__ __forceinline__ int pair_unit(int m, int u) {
    return UPR >= 16 ? u ^ (m & 15) : u ^ ((m >> 1) & (UPR - 1));
}

// Blocks of a workgroup: with one tile of pairs a wave has 16, and more waves hide the loads; with many, 32.
constexpr int score_blocks(bool one) { return one ? 64 : 256; }

// One workgroup 64 or 256 blocks of a (row, head), a wave 16 at a time: their key sums, as three bf16 parts of each
// fp32 value (split.h), are the rows of 16x16 matrix tiles, and the row's (token, head) pairs pass
// as columns. A product takes the part products of weight 2^-16 or more (three for bf16 queries, five for
// fp16, six for fp32), which is closer than a chain of fp32 products, at a fifth to a tenth of the time of the fp32
// matrix instructions. Lane l holds eight components of every 32 of block l%16, and of pair l%16.
// Pairs: 16 or less (ONE) stay in registers; more lie in LDS, kPairs at a time. Sums that are not
// finite, or whose products are not, are taken again in fp32.
// Neighbouring workgroups take the heads of the same blocks, whose sums lie side by side (of single tokens, 27 -> 23 us).
// 32 single tokens over 20000 to 65536 keys, 8 heads of 128 components, bf16: 23 us, 3.6 TB/s, bound by the latency of
// length, page and sums one after another. 8192 tokens in rows of 64, 4 queries a head, over 16384 keys: 58 us, 12.9 GFLOP
// of products (three times that on the matrix unit), bound by the reads of the pairs from LDS and the waits before them.
template <typename T, int NK, bool ONE>
__global__ __launch_bounds__(ONE ? 256 : 512, NK <= 4 ? 4 : 2) void scores_kernel(ScoreArgs a) {
    constexpr int kCols = ONE ? 1 : 2;                     // column tiles in work at a time
    constexpr int kWaves = ONE ? 4 : 8, kTiles = ONE ? 1 : 2;  // row tiles of a wave
    constexpr int kBlocks = score_blocks(ONE);
    constexpr int DP = NK * 32, UPR = DP / 8, NP = kParts<T>;
    // Pairs in LDS: a power of two, 64 KiB or less.
    constexpr int kFit = 32768 / (NP * DP), kPairs = ONE ? 16 : kFit >= 256 ? 256 : kFit >= 128 ? 128 : kFit >= 64 ? 64 : 32;
    __shared__ __attribute__((aligned(16))) uint16_t qs[ONE ? 1 : kPairs * NP * DP];
    __shared__ float kept[kBlocks];  // maxima of the chunks of pairs so far
    const int64_t idx = grid_index();
    if (idx >= a.items) return;
    const uint32_t rt = (uint32_t)idx / a.head_div;
    const int h = (int)((uint32_t)idx - rt * a.head_div.d);
    const int row = (int)(rt / a.tile_div), tile = (int)(rt - row * a.tile_div.d);
    const spconv_batch &B = a.B;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, part = lane >> 4;
    const Row r = find_row(B, row);
    const int p1 = r.n > 0 ? r.p0 + r.n - 1 : -1;
    const int visible = p1 < 0 ? 0 : min(p1 / B.block + 1, B.max_blocks);
    const int c_base = tile * kBlocks;
    float *out = a.scores + ((int64_t)row * a.heads + h) * B.max_blocks;
    if (c_base >= visible) {
        const int j = c_base + (int)threadIdx.x;
        if (threadIdx.x < kBlocks && j < B.max_blocks) out[j] = -kInf;
        return;
    }
    // Pages of this wave's blocks: tile i of it is blocks c_base + (kWaves*i + wave)*16 and on.
    const int mine = c_base + ((lane >> 4) * kWaves + wave) * 16 + col;
    const int pages = lane < 16 * kTiles && mine < visible ? page_of(B, r.b, mine) : -1;
    const int pairs = r.n * a.group;
    auto query_at = [&](int m) {
        const int i = (uint32_t)m / a.group_div, g = m - i * (int)a.group_div.d;
        return (const T *)a.q + (int64_t)(r.t0 + i) * a.q_token + (int64_t)(h * a.group + g) * a.q_head;
    };
    Floats<8> none;
#pragma unroll
    for (int i = 0; i < 8; ++i) none.v[i] = 0.0f;

    u32x4_t q1[ONE ? NK : 1][NP];
    if constexpr (ONE) {
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            query_parts<T>(col < pairs ? load_part(query_at(col), k * 32, part, a.dim, a.aligned) : none, q1[k]);
        }
    }
    // Key sums of tile i, fp32.
    Floats<8> raw[NK];
    auto fetch = [&](int i) {
        const int page = __shfl(pages, i * 16 + col);
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            raw[k] = page >= 0 ? load_part(a.sums + ((int64_t)page * a.heads + h) * a.dim, k * 32, part, a.dim, true) : none;
        }
    };
    // Rows of a result are blocks c0 + 4*part + e, columns pairs.
    auto bounds = [&](int i, int (&key0)[4], float (&inv)[4]) {
        const int c0 = c_base + (i * kWaves + wave) * 16;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = c0 + part * 4 + e;
            key0[e] = __shfl(pages, i * 16 + part * 4 + e) >= 0 ? j * B.block : 0x7fffffff;
            inv[e] = 1.0f / (float)clamp_int(r.kv - j * B.block, 1, B.block);
        }
    };
    // Maxima over the columns, to lane 16*part + e of each four rows.
    auto finish = [&](int i, float (&best)[4]) {
#pragma unroll
        for (int o = 8; o > 0; o >>= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) best[e] = fmaxf(best[e], __shfl_xor(best[e], o));
        const int at = (i * kWaves + wave) * 16 + part * 4 + (col & 3), j = c_base + at;
        const float v = (col & 3) == 0 ? best[0] : (col & 3) == 1 ? best[1] : (col & 3) == 2 ? best[2] : best[3];
        if (col < 4) kept[at] = v;
        if (col < 4 && j < B.max_blocks) out[j] = v;
    };

    // Tiles of this wave that have visible blocks.
    const int tiles = clamp_int((visible - c_base - wave * 16 + 16 * kWaves - 1) / (16 * kWaves), 0, kTiles);
    uint32_t again = 0;
    for (int m_base = 0; m_base < pairs; m_base += kPairs) {
        const int n_pairs = min(pairs - m_base, kPairs);
        if constexpr (!ONE) {
            __syncthreads();
            for (int u = threadIdx.x; u < n_pairs * UPR; u += 64 * kWaves) {
                const int m = u / UPR, k = (u % UPR) >> 2;
                u32x4_t p[NP];
                query_parts<T>(load_part(query_at(m_base + m), k * 32, u & 3, a.dim, a.aligned), p);
#pragma unroll
                for (int i = 0; i < NP; ++i)
                    *reinterpret_cast<u32x4_t *>(qs + ((m * NP + i) * UPR + pair_unit<UPR>(m, u % UPR)) * 8) = p[i];
            }
            __syncthreads();
        }
#pragma unroll 1
        for (int i = 0; i < tiles; ++i) {
            fetch(i);
            auto split = [&](int k) {
                Parts s;
#pragma unroll
                for (int e = 0; e < 4; ++e) split2(s, e, raw[k].v[2 * e], raw[k].v[2 * e + 1]);
                return s;
            };
            Parts parts[ONE ? 1 : NK];
            if constexpr (!ONE) {
#pragma unroll
                for (int k = 0; k < NK; ++k) parts[k] = split(k);
            }
            int key0[4];
            float inv[4], best[4] = {-kInf, -kInf, -kInf, -kInf};  // best: of the sums, before the division by the keys
            bounds(i, key0, inv);
            const bool whole = __all(max(max(key0[0], key0[1]), max(key0[2], key0[3])) <= r.p0);  // seen by every pair
            uint32_t largest = 0;  // magnitude's bits
            for (int m0 = 0; m0 < n_pairs; m0 += 16 * kCols) {
                f32x4 hi[kCols], lo[kCols];
#pragma unroll
                for (int n = 0; n < kCols; ++n) hi[n] = lo[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    const Parts s = ONE ? split(k) : parts[ONE ? 0 : k];
                    u32x4_t x[kCols][NP];
#pragma unroll
                    for (int n = 0; n < kCols; ++n)
#pragma unroll
                        for (int e = 0; e < NP; ++e) {
                            const int m = m0 + n * 16 + col;
                            if constexpr (ONE)
                                x[n][e] = q1[k][e];
                            else
                                x[n][e] = *reinterpret_cast<const u32x4_t *>(
                                    qs + ((m * NP + e) * UPR + pair_unit<UPR>(m, k * 4 + part)) * 8);
                        }
                    auto add = [&](f32x4 (&c)[kCols], u32x4_t s, int e) {
#pragma unroll
                        for (int n = 0; n < kCols; ++n) c[n] = mma_bits(s, x[n][e], c[n]);
                    };
                    add(lo, s.m, 0);
                    add(hi, s.h, 0);
                    add(lo, s.l, 0);
                    if constexpr (NP > 1) {
                        add(lo, s.h, 1);
                        add(lo, s.m, 1);
                    }
                    if constexpr (NP > 2) add(lo, s.h, 2);
                }
#pragma unroll
                for (int n = 0; n < kCols; ++n) {
                    f32x4 v = hi[n] + lo[n];
                    if (whole && m0 + n * 16 + 16 <= n_pairs) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            best[e] = fmaxf(best[e], v[e]);
                            largest = max(largest, __float_as_uint(v[e]) & 0x7fffffffu);
                        }
                    } else {
                        const int m = m0 + n * 16 + col;
                        const int p = m < n_pairs ? r.p0 + (int)((uint32_t)(m_base + m) / a.group_div) : -1;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool seen = p >= key0[e];
                            best[e] = fmaxf(best[e], seen ? v[e] : -kInf);
                            largest = max(largest, seen ? __float_as_uint(v[e]) & 0x7fffffffu : 0u);
                        }
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                best[e] *= inv[e];
                if (m_base > 0) best[e] = fmaxf(best[e], kept[(i * kWaves + wave) * 16 + part * 4 + e]);
            }
            const bool bad = largest >= 0x7f800000u;
            if (__ballot(bad)) again |= 1u << i;
            finish(i, best);
        }
        // Tiles of this wave behind the visible blocks.
        if (m_base == 0)
            for (int i = tiles; i < kTiles; ++i) {
                const int j = c_base + (i * kWaves + wave) * 16 + lane;
                if (lane < 16 && j < B.max_blocks) out[j] = -kInf;
            }
    }
    // Again in fp32, by the mean keys: a product with the sum may pass the range where that with the mean does not.
    for (int i = 0; again != 0; ++i, again >>= 1) {
        if (!(again & 1)) continue;
        fetch(i);
        int key0[4];
        float inv[4], best[4] = {-kInf, -kInf, -kInf, -kInf};
        bounds(i, key0, inv);
        const float keys = (float)clamp_int(r.kv - (c_base + (i * kWaves + wave) * 16 + col) * B.block, 1, B.block);
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) raw[k].v[e] /= keys;
        for (int m0 = 0; m0 < pairs; m0 += 16) {
            const int m = m0 + col;
            const int p = m < pairs ? r.p0 + (int)((uint32_t)m / a.group_div) : -1;
            f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                const Floats<8> x = p >= 0 ? load_part(query_at(m), k * 32, part, a.dim, a.aligned) : none;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(raw[k].v[e], x.v[e], acc, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (p >= key0[e]) best[e] = fmaxf(best[e], acc[e]);
        }
        finish(i, best);
    }
}

struct SelectArgs {
    spconv_batch B;
    const float *scores;
    int32_t *blocks, *counts;
    int64_t items;  // rows * heads
    int heads, keep, sink, local;
    int each;       // items a wave takes
    Div head_div;
};

// Order of the values as unsigned numbers: 0 stands for "no candidate", NaN counts as -infinity
// (0x007fffff), -0 as +0.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (!(x > -kInf)) return 0x007fffffu;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// What a row may choose from: n blocks seen, of which [0, sink) and [low, n) are always listed.
struct Choice {
    int n, sink, low, want;  // want: how many of the others
};

__device__ __forceinline__ Choice choice_of(const SelectArgs &a, const Row &r) {
    const spconv_batch &B = a.B;
    Choice c;
    const int p1 = r.n > 0 ? r.p0 + r.n - 1 : -1;
    c.n = p1 < 0 ? 0 : min(p1 / B.block + 1, B.max_blocks);
    c.sink = min(a.sink, c.n);
    c.low = c.n;
    if (a.local > 0) c.low = clamp_int(max(r.p0, 0) / B.block - a.local + 1, 0, c.n);
    const int forced = c.low <= c.sink ? c.n : c.sink + c.n - c.low;
    c.want = a.keep - forced;
    return c;
}

// The value whose order is u (not that of NaN).
__device__ __forceinline__ float value_of(uint32_t u) { return __uint_as_float((u & 0x80000000u) ? u & 0x7fffffffu : ~u); }

// Ones of a ballot in the lanes below this one.
__device__ __forceinline__ int before(uint64_t x) {
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(x >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)x, 0));
}

// Maximum over the wave: neighbours 1, 2, 4 and 8 lanes back in each row of 16, then the last lanes of the rows
// before; lane 63 has it all.
__device__ __forceinline__ float wave_max(float x) {
    auto step = [&](float v) { x = fmaxf(x, v); };
#define SPCONV_DPP(ctrl) \
    step(__int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), ctrl, 0xf, 0xf, false)))
    SPCONV_DPP(0x111);
    SPCONV_DPP(0x112);
    SPCONV_DPP(0x114);
    SPCONV_DPP(0x118);
    SPCONV_DPP(0x142);
    SPCONV_DPP(0x143);
#undef SPCONV_DPP
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// One (row, head) of at most 64*NI blocks by one wave, held in registers. Bound by instructions (a count over all
// values is 3*NI of them), so few counts are taken: a lower bound from the lanes' highest values, or halving the range
// of the values, soon leaves 64 or less that can be the want-th highest (many equal or infinite
// ones end at the most steps, and then the range of their order is halved). Those go to one register, where a count
// is one instruction, and the search ends there, by trying one of them after another (log2 of them or so). Of the
// want-th highest's equals the lowest indices are taken. Then the list is written in order.
// 256 lists of 64 of up to 1024 blocks 8 us (latency of one list); 32776 lists of 32 of 125 to 512 blocks 36 us, 1.3 TB/s.
template <int NI>
__device__ __forceinline__ void select_row(const SelectArgs &a, const Choice &c, int64_t item, int lane, float *few) {
    int32_t *blocks = a.blocks + item * a.keep;
    const int count = min(c.n, a.keep);
    if (lane == 0) a.counts[item] = count;
    if (c.n <= a.keep) {
        for (int i = lane; i < a.keep; i += 64) blocks[i] = i < c.n ? i : -1;
        return;
    }
    const float *s = a.scores + item * a.B.max_blocks;
    // Candidates' values; NaN, which no comparison finds, for blocks that are none.
    float v[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) v[i] = s[min(i * 64 + lane, c.n - 1)];
    float mine = __builtin_nanf("");  // this lane's highest
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int j = i * 64 + lane;
        v[i] = v[i] > -kInf ? v[i] : -kInf;  // NaN counts as -infinity
        v[i] = j >= c.sink && j < c.low ? v[i] : __builtin_nanf("");
        mine = fmaxf(mine, v[i]);
    }
    float cut = __builtin_nanf("");  // what is not below it is taken: none without candidates to choose
    int ties = 0x7fffffff;           // and of those equal to it so many
    if (c.want > 0) {
        auto not_below = [&](float t) {
            int n = 0;
#pragma unroll
            for (int i = 0; i < NI; ++i) n += bits(__ballot(v[i] >= t));
            return n;
        };
        // want or more are not below lo, less are not below hi (from above the maximum on).
        const float most = wave_max(mine);
        float hi = most, lo = -kInf;
        int at_lo = c.low - c.sink, at_hi = 0;
        // A value that want or a few more lanes' highest reach is not far below the want-th highest of all.
        if (c.want < bits(__ballot(mine > -kInf))) {
            lo = -wave_max(-mine);
            for (int i = 0; i < 8; ++i) {
                const float t = 0.5f * lo + 0.5f * hi;
                const int n = bits(__ballot(mine >= t));
                if (n >= c.want) lo = t;
                else hi = t;
                if (n >= c.want && n <= c.want + 4) break;
            }
            hi = most;
            at_lo = not_below(lo);
        }
        bool open = true;  // hi is the maximum, and may be the one
        for (int i = 0; i < 10 && at_lo != c.want && at_lo - at_hi > 64; ++i) {
            const float t = 0.5f * lo + 0.5f * hi;
            if (!(t > lo && t < hi)) break;
            const int n = not_below(t);
            if (n >= c.want) {
                lo = t;
                at_lo = n;
            } else {
                hi = t;
                at_hi = n;
                open = false;
            }
        }
        uint32_t a0 = order_of(lo), a1 = order_of(hi) + (open ? 1u : 0u);  // the same in orders: [a0, a1)
        while (at_lo != c.want && at_lo - at_hi > 64 && a1 - a0 > 1) {
            const uint32_t t = a0 + (a1 - a0) / 2;
            const int n = not_below(value_of(t));
            if (n >= c.want) {
                a0 = t;
                at_lo = n;
            } else {
                a1 = t;
                at_hi = n;
                open = false;
            }
        }
        if (at_lo != c.want && a1 - a0 > 1) {
            const float from = value_of(a0), to = open ? __builtin_nanf("") : value_of(a1);
            int at = 0;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const bool in = v[i] >= from && !(v[i] >= to);
                const uint64_t all = __ballot(in);
                few[in ? at + before(all) : 64] = v[i];  // (behind the list: what is not in it)
                at += bits(all);
            }
            __builtin_amdgcn_wave_barrier();
            const float x = lane < at ? few[lane] : __builtin_nanf("");
            // One of those that can still be it at a time: with how many are above it and equal to it, it is the one or
            // leaves those on one side.
            uint64_t left = __ballot(lane < at);
            while (left != 0) {
                const float t = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), __builtin_ctzll(left)));
                const uint64_t gt = __ballot(x > t), ge = __ballot(x >= t);
                if (at_hi + bits(gt) >= c.want) {
                    left &= gt;
                } else if (at_hi + bits(ge) < c.want) {
                    left &= ~ge;
                } else {
                    cut = t;
                    at_lo = at_hi + bits(ge);
                    at_hi += bits(gt);
                    break;
                }
            }
        } else {
            cut = value_of(a0);
        }
        if (at_lo != c.want) ties = c.want - at_hi;  // the cut is the want-th highest, at_hi are above it
    }
    int at = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        if (i * 64 >= c.n) break;
        const int j = i * 64 + lane;
        bool take = v[i] >= cut;
        if (ties != 0x7fffffff) {
            const uint64_t eq = __ballot(v[i] == cut);
            take = take && !(v[i] == cut && before(eq) >= ties);
            ties = max(0, ties - bits(eq));
        }
        if (i * 64 < c.sink || i * 64 + 64 > c.low) take = j < c.n && (take || j < c.sink || j >= c.low);
        const uint64_t all = __ballot(take);
        const int pos = at + before(all);
        if (take && pos < a.keep) blocks[pos] = j;
        at += bits(all);
    }
    for (int i = at + lane; i < a.keep; i += 64) blocks[i] = -1;
}

// One wave `each` neighbouring (row, head): where there are more of them than waves on the GPU, a row is looked up
// once for several of its heads.
template <int NI>
__global__ __launch_bounds__(256) void select_wave_kernel(SelectArgs a) {
    __shared__ float lists[4][65];
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    const int64_t first = (grid_index() * 4 + wave) * a.each, end = min(first + a.each, a.items);
    if (first >= a.items) return;
    Row r;
    Choice c;
    int row = -1;
    for (int64_t item = first; item < end; ++item) {
        if ((int)((uint32_t)item / a.head_div) != row) {
            row = (int)((uint32_t)item / a.head_div);
            r = find_row(a.B, row);
            c = choice_of(a, r);
        }
        if (NI > 4 && c.n <= NI * 32)
            select_row<NI / 2>(a, c, item, lane, lists[wave]);
        else
            select_row<NI>(a, c, item, lane, lists[wave]);
    }
}

// One workgroup of 1024 threads a (row, head) of more blocks: wave w takes the w-th
// sixteenth of them, in `per` steps of 64, the first kHeld of which (8192 blocks in all) stay in registers, the others
// come from the cache each time. The want-th highest is found eight bits of its
// order at a time, from the highest: how many of those that share the bits above have each of the 256 next ones is
// counted in LDS (each number in eight places, so that lanes that count the same one wait less).
// Two workgroups a CU, bound by the latency of its passes: 8192 blocks, 128 lists 12 us with the launch, 4096 lists
// 101 us (134 MB); halving the order, 32 counts with a barrier each, took 54 and 426.
__global__ __launch_bounds__(1024, 8) void select_block_kernel(SelectArgs a, int per) {
    __shared__ int counts[2][16];
    __shared__ int bins[256][8];
    __shared__ __attribute__((aligned(16))) int sums[256];
    __shared__ int found[3];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t item = grid_index();
    if (item >= a.items) return;
    const int row = (int)((uint32_t)item / a.head_div);
    const Row r = find_row(a.B, row);
    const Choice c = choice_of(a, r);
    int32_t *blocks = a.blocks + item * a.keep;
    const int count = min(c.n, a.keep);
    if (threadIdx.x == 0) a.counts[item] = count;
    if (c.n <= a.keep) {
        for (int i = threadIdx.x; i < a.keep; i += 1024) blocks[i] = i < c.n ? i : -1;
        return;
    }
    const float *s = a.scores + item * a.B.max_blocks;
    const int first = wave * per * 64;
    const int steps = clamp_int((c.n - first + 63) / 64, 0, per);  // of this wave; behind them nothing is taken
    int turn = 0;
    // Sum over the workgroup of a wave's number, and of the waves before this one.
    auto total = [&](int n, int &ahead) {
        if (lane == 0) counts[turn][wave] = n;
        __syncthreads();
        int all = 0;
        ahead = 0;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) ahead += counts[turn][w];
            all += counts[turn][w];
        }
        turn ^= 1;  // the next one's slots: nobody is still reading those
        return all;
    };
    constexpr int kHeld = 8;
    float loaded[kHeld];
    uint32_t held[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) loaded[i] = s[min(first + i * 64 + lane, c.n - 1)];
    auto order = [&](int j, float x) { return j >= c.sink && j < c.low ? order_of(x) : 0u; };
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = order(first + i * 64 + lane, loaded[i]);
    // f(block, order of its value) for this wave's blocks.
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (i < steps) f(first + i * 64 + lane, held[i]);
#pragma unroll 4
        for (int i = kHeld; i < steps; ++i) {
            const int j = first + i * 64 + lane;
            f(j, order(j, s[min(j, c.n - 1)]));
        }
    };
    uint32_t cut = 0xffffffffu;  // what is above it is taken (no order is that high)
    int ties = 0;                // and so many of those equal to it
    if (c.want > 0) {
        int want = c.want, equal = 0;  // of those that share the bits found so far
        cut = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = threadIdx.x; i < 256 * 8; i += 1024) bins[0][i] = 0;
            __syncthreads();
            each([&](int, uint32_t v) {
                if (v != 0 && ((uint64_t)v >> (shift + 8)) == (uint64_t)cut >> (shift + 8))
                    atomicAdd(&bins[(v >> shift) & 255][lane & 7], 1);
            });
            __syncthreads();
            if (threadIdx.x < 256) {
                int n = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) n += bins[threadIdx.x][i];
                sums[threadIdx.x] = n;
            }
            __syncthreads();
            if (wave == 0) {  // lane l: bins 4l .. 4l + 3
                int n[4], mine = 0, above;
#pragma unroll
                for (int e = 0; e < 4; ++e) mine += n[e] = sums[lane * 4 + e];
                above = mine;  // with all lanes behind
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const int x = __shfl_down(above, o);
                    above += lane + o < 64 ? x : 0;
                }
                above -= mine;
#pragma unroll
                for (int e = 3; e >= 0; --e) {
                    if (above < want && above + n[e] >= want) {  // one bin of one lane
                        found[0] = lane * 4 + e;
                        found[1] = above;
                        found[2] = n[e];
                    }
                    above += n[e];
                }
            }
            __syncthreads();
            cut |= (uint32_t)found[0] << shift;
            want -= found[1];
            equal = found[2];
            if (equal == want) break;  // all of them, whatever the bits below
        }
        if (equal == want) {
            cut = max(cut, 1u) - 1;  // (no candidate's order is 0)
        } else {
            int eq = 0, ahead;
            each([&](int, uint32_t v) { eq += bits(__ballot(v == cut)); });
            total(eq, ahead);
            ties = max(0, want - ahead);
        }
    }
    // Taken by this wave, then by those before it, then the list.
    int mine = 0, at = 0;
    for (int pass = 0; pass < 2; ++pass) {
        int left = ties, n = 0;
        each([&](int j, uint32_t v) {
            const uint64_t eq = __ballot(v == cut);
            const bool tie = v == cut && before(eq) < left;
            const bool take = j < c.n && (j < c.sink || j >= c.low || v > cut || tie);
            left = max(0, left - bits(eq));
            const uint64_t all = __ballot(take);
            const int pos = at + n + before(all);
            if (pass == 1 && take && pos < a.keep) blocks[pos] = j;
            n += bits(all);
        });
        if (pass == 0) mine = total(n, at);
    }
    for (int i = mine + (int)threadIdx.x; i < a.keep; i += 1024) blocks[i] = -1;
}

template <typename T, bool ONE>
int scores_of(const ScoreArgs &a, hipStream_t stream) {
    const dim3 grid = grid_of(a.items);
    constexpr int threads = ONE ? 256 : 512;
    if (a.dim <= 64)
        scores_kernel<T, 2, ONE><<<grid, threads, 0, stream>>>(a);
    else if (a.dim <= 128)
        scores_kernel<T, 4, ONE><<<grid, threads, 0, stream>>>(a);
    else
        scores_kernel<T, 8, ONE><<<grid, threads, 0, stream>>>(a);
    return launched();
}

template <typename T>
int scores_by_pairs(const ScoreArgs &a, hipStream_t stream) {
    return row_tokens(&a.B) * a.group <= 16 ? scores_of<T, true>(a, stream) : scores_of<T, false>(a, stream);
}

}  // namespace

extern "C" int spconv_block_scores(int dtype, const spconv_batch *batch, const void *q, int64_t q_token, int64_t q_head,
                                   int q_heads, int heads, int dim, const float *sums, float *scores,
                                   hipStream_t stream) {
    if (!batch_ok(batch) || !batch_arrays_ok(batch) || !dtype_ok(dtype) || q == nullptr || sums == nullptr ||
        scores == nullptr || !heads_ok(q_heads, heads, dim) || q_token < 0 || q_head < 0 || !aligned16(sums))
        return SPCONV_EINVAL;
    const int per = score_blocks(row_tokens(batch) * (q_heads / heads) <= 16);
    const int tiles = (batch->max_blocks + per - 1) / per;
    const int64_t rows = rows_of(batch);
    if (rows * heads * tiles >= ((int64_t)1 << 31)) return SPCONV_EINVAL;
    ScoreArgs a{*batch, q, q_token, q_head, sums, scores, rows * heads * tiles, heads, q_heads / heads, dim, tiles,
                make_div((uint32_t)tiles), make_div((uint32_t)heads), make_div((uint32_t)(q_heads / heads)),
                rows_aligned16(q, q_token, q_head, size_of(dtype))};
    if (dtype == SPCONV_F32) return scores_by_pairs<float>(a, stream);
    if (dtype == SPCONV_F16) return scores_by_pairs<_Float16>(a, stream);
    return scores_by_pairs<__bf16>(a, stream);
}

extern "C" int spconv_select_blocks(const spconv_batch *batch, int heads, const float *scores, int keep, int sink,
                                    int local, int32_t *blocks, int32_t *counts, hipStream_t stream) {
    if (!batch_ok(batch) || !batch_arrays_ok(batch) || scores == nullptr || blocks == nullptr || counts == nullptr ||
        heads < 1 || heads > 65535 || keep < 1 || sink < 0 || local < 0)
        return SPCONV_EINVAL;
    const int64_t always = (int64_t)sink + local + (batch->q_block - 1 + batch->block - 1) / batch->block;
    const int64_t items = rows_of(batch) * heads;
    if (keep < always || items >= ((int64_t)1 << 31) || items * keep >= ((int64_t)1 << 40)) return SPCONV_EINVAL;
    SelectArgs a{*batch, scores, blocks, counts, items, heads, keep, sink, local, 1, make_div((uint32_t)heads)};
    const int n = (batch->max_blocks + 63) / 64;
    // A wave's registers hold 2048 values: 4096 lists of 2048 blocks take 20 us, by workgroups 65 (128 lists: 12 and 10).
    if (n <= 32) {
        a.each = (int)std::min<int64_t>(std::max<int64_t>(items / 8192, 1), heads);  // 8192 waves fill the GPU
        const dim3 grid = grid_of(((items + a.each - 1) / a.each + 3) / 4);
        if (n <= 4)
            select_wave_kernel<4><<<grid, 256, 0, stream>>>(a);
        else if (n <= 8)
            select_wave_kernel<8><<<grid, 256, 0, stream>>>(a);
        else if (n <= 16)
            select_wave_kernel<16><<<grid, 256, 0, stream>>>(a);
        else
            select_wave_kernel<32><<<grid, 256, 0, stream>>>(a);
    } else {
        select_block_kernel<<<grid_of(items), 1024, 0, stream>>>(a, (n + 15) / 16);
    }
    return launched();
}
