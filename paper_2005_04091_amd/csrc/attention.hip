// Attention over listed blocks (spconv_block_attention).
//
// For a query q and the keys S that its row lists and its position lets it see:
//   out = sum_S exp(x_j - m) v_j / sum_S exp(x_j - m),  x_j = scale * q.k_j, m = max_S x_j,
// in one pass over the keys: when a tile raises the running maximum from m to m',
// sum and output so far are multiplied by exp(m - m'). Everything is held in powers of two
// (x in units of ln 2), in fp32.
//
// Matrix tiles are formed transposed: S^T = K Q^T has queries as columns, so that a lane
// holds weights of one query only, its maximum and sum are a lane's own numbers, and the
// weights are already where the second product O^T = V^T P^T wants its right
// operand: the order of the keys inside a product is free, so V^T's rows are read in the order
// in which the weights came out (slot 8*(l/16) + 4*t + i of lane l is key 16*t + 4*(l/16) + i).
#include "batch.h"

#include <type_traits>

namespace {

constexpr float kInf = __builtin_huge_valf();
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

template <typename T>
struct Frag8 {
    typedef T type __attribute__((ext_vector_type(8)));
};

template <typename T>
using frag_t = typename Frag8<T>::type;

// acc += A B for 16x16 tiles, 32 deep: eight elements of a row of A and of a column of B per lane.
__device__ __forceinline__ f32x4 mma(frag_t<__bf16> a, frag_t<__bf16> b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(frag_t<_Float16> a, frag_t<_Float16> b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(frag_t<float> a, frag_t<float> b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

template <typename T>
__device__ __forceinline__ frag_t<T> zero_frag() {
    frag_t<T> z;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = (T)0.0f;
    return z;
}

// x, as a value that the compiler knows nothing about: what is derived from it is formed where it
// is used, and not kept in registers through the loops before.
__device__ __forceinline__ int fresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// Max and sum over the four lanes that hold one column (lanes l, l+16, l+32, l+48).
__device__ __forceinline__ float column_max(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const uint32_t w = __float_as_uint(y);
    const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ float column_sum(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const uint32_t w = __float_as_uint(y);
    const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

struct AttnArgs {
    spconv_batch B;
    const void *q;
    int64_t q_token, q_head;
    const void *k_cache, *v_cache;
    const int32_t *blocks, *counts;
    void *out;
    int64_t o_token, o_head;
    float *lse;
    float *part, *stat;  // workspace, items from `whole` on: [item][split][tile_pairs][dim], [item][split][tile_pairs] of (maximum, sum, rounded sum, -)
    int64_t items;       // rows * heads * tiles
    int64_t whole;       // items [0, whole) are one workgroup each, those behind them `splits`
    int heads, group, dim, keep, tiles, splits, q_aligned, o_aligned;
    int tile_pairs;      // pairs of a tile
    float scale2;        // scale / ln 2
    Div tile_div, head_div, group_div, split_div, slab_div, pair_div;
};

// The (token, head) pairs of a tile of a row, token by token: pair m is token m / group, head m % group.
struct Pairs {
    Row r;
    int h, m0, end;   // pairs [m0, end)
    int last;         // position of the tile's last token, -1 if it has none
    int listed;       // what counts says of the row's list
    int64_t rh;
};

__device__ __forceinline__ Pairs find_pairs(const AttnArgs &a, uint32_t item) {
    Pairs p;
    const uint32_t rh = item / a.tile_div;
    p.m0 = (int)(item - rh * a.tile_div.d) * a.tile_pairs;
    const int row = (int)(rh / a.head_div);
    p.h = (int)(rh - row * a.head_div.d);
    p.rh = rh;
    p.listed = a.counts ? a.counts[rh] : a.keep;  // (on its way while the row is looked up)
    p.r = find_row(a.B, row);
    p.end = min(p.r.n * a.group, p.m0 + a.tile_pairs);
    p.last = p.end > p.m0 ? p.r.p0 + (int)((uint32_t)(p.end - 1) / a.group_div) : -1;
    if (p.end <= p.m0) p.r.n = 0;
    return p;
}

// Output and log-sum-exp of a sum of weights relative to 2^ref; 0 and -infinity of an empty one.
__device__ __forceinline__ float weighted(float acc, float sum) { return sum == 0.0f ? 0.0f : acc / sum; }
__device__ __forceinline__ float log_sum(float ref, float sum) {
    return sum == 0.0f ? -kInf : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
}

// The keys that a tile may read, 16 at a time (slabs: a sixteenth of a page's rows or more lie
// side by side): the first key of each and its place in the cache, looked up for kSlabs of them at a time.
constexpr int kSlabs = 256;

// What a workgroup does: share `split` of `splits` of an item. Neighbouring whole items go to one XCD.
struct Work {
    uint32_t item;
    int split, splits;
};

__device__ __forceinline__ bool find_work(const AttnArgs &a, Work &w) {
    int64_t idx = grid_index();
    if (idx < a.whole) {
        if (a.whole <= kGridX) idx = xcd_linear_id((int)idx, (int)a.whole);
        w.item = (uint32_t)idx;
        w.split = 0;
        w.splits = 1;
        return true;
    }
    idx -= a.whole;
    if (idx >= (a.items - a.whole) * a.splits) return false;
    const uint32_t i = (uint32_t)idx / a.split_div;
    w.item = (uint32_t)a.whole + i;
    w.split = (int)((uint32_t)idx - i * a.split_div.d);
    w.splits = a.splits;
    return true;
}

struct Slabs {
    int64_t base[kSlabs + 16];  // elements; 0 behind the last
    int key[kSlabs + 16];       // -1: nothing of it is seen
    uint64_t part[kSlabs / 64]; // a bit for each slab: not all of it is seen by every pair
};

// Slabs [s0, s0 + kSlabs) of a row's list, those below s_hi; THREADS threads. first_pos: the first pair's position.
template <int THREADS>
__device__ __forceinline__ void look_up(Slabs &S, const AttnArgs &a, const Pairs &P, int64_t s0, int64_t s_hi,
                                        int first_pos) {
    const spconv_batch &B = a.B;
    const int spb = B.block >> 4;
    const int e0 = (int)(s0 / spb), r0 = (int)(s0 - (int64_t)e0 * spb);
    for (int i = threadIdx.x; i < kSlabs + 64; i += THREADS) {  // whole waves
        int key = -1;
        int64_t base = 0;
        if (i < kSlabs && s0 + i < s_hi) {
            const int de = (uint32_t)(r0 + i) / a.slab_div, sub = r0 + i - de * spb;
            const int j = a.blocks ? a.blocks[P.rh * a.keep + e0 + de] : e0 + de;
            if (j >= 0 && j < B.max_blocks && j <= P.last / B.block) {
                const int page = page_of(B, P.r.b, j), k0 = j * B.block + sub * 16;
                if (page >= 0 && k0 <= P.last) {
                    key = k0;
                    base = (((int64_t)page * a.heads + P.h) * B.block + sub * 16) * a.dim;
                }
            }
        }
        if (i < kSlabs + 16) {
            S.key[i] = key;
            S.base[i] = base;
        }
        const uint64_t part = __ballot(key < 0 || key + 15 > first_pos);
        if ((threadIdx.x & 63) == 0 && i < kSlabs) S.part[i >> 6] = part;
    }
}

// Slabs of the row's list.
__device__ __forceinline__ int64_t slabs_of(const AttnArgs &a, const Pairs &P) {
    int entries = 0;
    if (P.last >= 0)
        entries = !a.blocks ? min(P.last / a.B.block + 1, a.B.max_blocks)
                            : clamp_int(P.listed, 0, a.keep);
    return (int64_t)entries * (a.B.block >> 4);
}

__device__ __forceinline__ int64_t uniform64(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// Where unit c (16 bytes) of row r of a wave's values lies in its LDS: 32 lanes read two units of eight rows at a
// time (16-bit types) or four units of two rows, and touch all 64 banks.
template <int UPR, int SIZE>
__device__ __forceinline__ int row_unit(int r, int c) {
    if (SIZE == 4) return c ^ (((r >> 2) & 3) << 2);
    return UPR >= 16 ? c ^ ((r & 7) << 1) : c ^ (((r >> 1) & 3) << 1);
}

// One workgroup a (row, head, 16 pairs, share of the row's keys). Its four waves take 32
// keys in turn, each with a running maximum, sum and output of its own, joined
// at the end; shares of a row (splits) are joined by join_kernel. NK*32 components are laid out, NC*32 computed.
// The keys are read once for 16 pairs, so single tokens are bound by HBM: 64 tokens, 8 heads of 4 queries, 128
// components, bf16, lists of 2048 keys, 97 us, 5.5 TB/s. Two workgroups a CU (one of more than 128 components, whose
// tiles fill the registers): 16 tokens, 4 heads of 8 queries, 256 components, 42 us, 3.2 TB/s; fp32 92 us, 2.9 TB/s.
// Lists of prompts that come from the caches: 1000 rows of one token, 4 heads of 4
// queries, 512 keys, 117 us, 9 TB/s.
template <typename T, int NK, int NC>
__global__ __launch_bounds__(256, sizeof(T) == 2 && NC <= 4 ? 2 : 1) void rows_kernel(AttnArgs a) {
    constexpr int DP = NK * 32, W = kPer16<T>, UPR = DP / W;  // 16-byte units of a row
    constexpr int NU = 16 * UPR / 64;                         // units a lane holds of 16 rows
    constexpr int kTile = 32 * DP * (int)sizeof(T);
    constexpr int kJoin = 16 * (DP + 4) * 4;
    constexpr int kPerWave = kTile > kJoin ? kTile : kJoin;
    // Addresses are formed anew for each tile where registers are short (fp32, 256 components: 128 -> 107 us; others lose
    // 2%), and there the queries lie in LDS (-> 92 us).
    constexpr bool kFresh = NC == 8 && sizeof(T) == 4;
    __shared__ __attribute__((aligned(16))) T q_lds[kFresh ? 16 * (DP + 4) : 1];
    __shared__ __attribute__((aligned(16))) char lds[4 * kPerWave];
    __shared__ Slabs S;
    __shared__ float w_max[4][16], w_sum[4][16];
    typedef typename VecOf<T, W>::type V;

    Work work;
    if (!find_work(a, work)) return;
    const Pairs P = find_pairs(a, work.item);
    if (P.r.n == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, part = lane >> 4;
    const int D = a.dim;

    // Query of this lane's column.
    const int m = P.m0 + col, tok = (uint32_t)m / a.group_div;
    const int pos = tok < P.r.n ? P.r.p0 + tok : -1;
    frag_t<T> q[kFresh ? 1 : NC];
    {
        const T *src = (const T *)a.q + (int64_t)(P.r.t0 + tok) * a.q_token +
                       (int64_t)(P.h * a.group + (m - tok * a.group)) * a.q_head;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            const int d = k * 32 + part * 8;
            frag_t<T> x = zero_frag<T>();
            if (tok < P.r.n && d < D) {
                if (a.q_aligned) {
                    x = *reinterpret_cast<const frag_t<T> *>(src + d);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = src[d + i];
                }
            }
            if constexpr (kFresh) {
                if (wave == 0) {  // (read behind the first barrier of the walk)
#pragma unroll
                    for (int i = 0; i < 8; ++i) q_lds[col * (DP + 4) + d + i] = x[i];
                }
            } else {
                q[k] = x;
            }
        }
    }

    // This share of the row's slabs.
    const int64_t slabs = slabs_of(a, P);
    const int64_t per = ((slabs + 1) / 2 + work.splits - 1) / work.splits * 2;
    const int64_t s_lo = min(per * work.split, slabs), s_hi = min(s_lo + per, slabs);
    const int first_pos = P.r.p0 + (int)((uint32_t)P.m0 / a.group_div);  // position of the tile's first token

    constexpr int NT = NC * 2;
    f32x4 o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float top = -kInf, sum = 0.0f;
    T *vt = reinterpret_cast<T *>(lds + wave * kPerWave);

    // Keys go from memory into the operands of the first product, values by rows through LDS, which hands
    // them out by columns. The next tile's loads start as soon as this one's registers are free.
    frag_t<T> kf[2][NC];
    V vf[2][NU];
    auto fetch_keys = [&](int s) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const T *src = (const T *)a.k_cache + S.base[s + t] + col * D;
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                const int d = k * 32 + part * 8;
                kf[t][k] = *reinterpret_cast<const frag_t<T> *>(src + (d < D ? d : 0));
            }
        }
    };
    auto fetch_values = [&](int s) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const T *src = (const T *)a.v_cache + S.base[s + t];
            const int ln = kFresh ? fresh(lane) : lane;
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                const int u = i * 64 + ln, c = u % UPR;
                vf[t][i] = *reinterpret_cast<const V *>(src + u / UPR * D + (c * W < D ? c * W : 0));
            }
        }
    };

    for (int64_t c0 = s_lo; c0 < s_hi; c0 += kSlabs) {
        __syncthreads();
        look_up<256>(S, a, P, c0, s_hi, first_pos);
        __syncthreads();
        const int n_slabs = (int)min(s_hi - c0, (int64_t)kSlabs);
        if (2 * wave < n_slabs) {
            fetch_keys(2 * wave);
            fetch_values(2 * wave);
        }
        for (int s = 2 * wave; s < n_slabs; s += 8) {
            int key0[2];
            bool there[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                key0[t] = __builtin_amdgcn_readfirstlane(S.key[s + t]);
                there[t] = key0[t] >= 0;
            }
            f32x4 x[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                // fp32 products in chains of 64 components or less: the sum's own roundings grow with a chain's length.
                constexpr int kChain = sizeof(T) == 2 ? NC : NC == 2 ? 1 : 2;
#pragma unroll
                for (int k0 = 0; k0 < NC; k0 += kChain) {
                    f32x4 sum4 = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int k = k0; k < k0 + kChain; ++k) {
                        frag_t<T> f = kf[t][k];
                        if (k * 32 + part * 8 >= D) f = zero_frag<T>();
                        if constexpr (kFresh) {
                            union {
                                V h[2];
                                frag_t<T> f;
                            } u;
                            const V *at = reinterpret_cast<const V *>(q_lds + col * (DP + 4) + k * 32 + part * 8);
                            u.h[0] = at[0];
                            u.h[1] = at[1];
                            sum4 = mma(f, u.f, sum4);
                        } else {
                            sum4 = mma(f, q[k], sum4);
                        }
                    }
                    x[t] = k0 == 0 ? sum4 : x[t] + sum4;
                    if (NC > 4 && sizeof(T) == 4) __builtin_amdgcn_sched_barrier(0);  // (short of registers)
                }
            }
            if (s + 8 < n_slabs) fetch_keys(s + 8);
            // Values that no query of the tile sees become zero, whatever lies there: their weights are zero too,
            // and zero times infinity is not. Of a tile that some see a part of, those that are not finite come
            // in a pass of their own.
            bool odd = false;
            if (!there[0] || !there[1] || max(key0[0], key0[1]) + 15 > first_pos) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < NU; ++i) {
                        const int u = i * 64 + lane;
                        const bool seen = there[t] && key0[t] + u / UPR <= P.last;
#pragma unroll
                        for (int e = 0; e < W; ++e) {
                            const bool bad = not_finite((float)vf[t][i][e]);
                            odd = odd || (seen && bad);
                            if (!seen || bad) vf[t][i][e] = (T)0.0f;
                        }
                    }
            }
            const int ln = kFresh ? fresh(lane) : lane;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    const int u = i * 64 + ln, r = t * 16 + u / UPR;
                    *reinterpret_cast<V *>(vt + r * DP + row_unit<UPR, (int)sizeof(T)>(r, u % UPR) * W) = vf[t][i];
                }
            if (s + 8 < n_slabs) fetch_values(s + 8);
            // Weights.
            float hi8 = -kInf;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool seen = there[t] && key0[t] + part * 4 + i <= pos;
                    x[t][i] = seen ? x[t][i] * a.scale2 : -kInf;
                    hi8 = fmaxf(hi8, x[t][i]);
                }
            const float next = fmaxf(top, column_max(hi8));
            const float ref = next == -kInf ? 0.0f : next;
            const float shrink = __builtin_amdgcn_exp2f(top - ref);
            top = next;
            frag_t<T> w;
            float total = 0.0f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // (fp16 and bf16: rounded for the matrix unit, half a step each. The sum is that of the weights before it:
                    // each wave's largest is exactly 1, so that no rounding of a weight that outweighs the others is left to
                    // cancel, as there is in the tiles below.)
                    const float p = __builtin_amdgcn_exp2f(x[t][i] - ref);
                    total += p;
                    w[t * 4 + i] = (T)p;
                }
            sum = sum * shrink + total;
            if (__ballot(shrink != 1.0f)) {
#pragma unroll
                for (int t = 0; t < NT; ++t) o[t] *= shrink;
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (t * 16 >= D) continue;
                frag_t<T> f;
                if constexpr (sizeof(T) == 2) {
                    typedef short s16x4 __attribute__((ext_vector_type(4)));
                    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                    union {
                        s16x4 h[2];
                        frag_t<T> f;
                    } u;
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int col = ln & 15, part = ln >> 4, lr = b * 16 + part * 4 + (col >> 2);
                        const int c = t * 2 + ((col & 3) >> 1);
                        T *src = vt + lr * DP + row_unit<UPR, 2>(lr, c) * W + (col & 1) * 4;
                        u.h[b] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)src);
                    }
                    f = u.f;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int lr = (i >> 2) * 16 + (ln >> 4) * 4 + (i & 3), d = t * 16 + (ln & 15);
                        f[i] = vt[lr * DP + row_unit<UPR, 4>(lr, d >> 2) * 4 + (d & 3)];
                    }
                }
                o[t] = mma(f, w, o[t]);
            }
            if (__ballot(odd)) {
                // Values that are not finite, in a tile of which some queries see a part only: one by one, those of the
                // half that all see too (both halves were cleaned).
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (!there[t]) continue;
                    for (int kr = 0; kr < 16; ++kr) {
                        if (key0[t] + kr > pos) continue;
                        const T *src = (const T *)a.v_cache + S.base[s + t] + kr * D;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const int d = n * 16 + part * 4;
                            const Floats<4> v = load_floats<T, 4>(src + min(d, D - 4));
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[n][i] += not_finite(v.v[i]) ? v.v[i] : 0.0f;  // (behind D: not used)
                            asm volatile("" ::: "memory");  // one load at a time: this is no place for registers
                        }
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
    sum = column_sum(sum);

    // Join the waves.
    __syncthreads();
    float *mine = reinterpret_cast<float *>(lds + wave * kPerWave);
#pragma unroll
    for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4 *>(mine + col * (DP + 4) + t * 16 + part * 4) = o[t];
    if (part == 0) {
        w_max[wave][col] = top;
        w_sum[wave][col] = sum;
    }
    __syncthreads();
    const int pairs = P.end - P.m0;
    for (int i = tid; i < pairs * DP; i += 256) {
        const int c = i / DP, d = i % DP;
        if (d >= D) continue;
        float mx = -kInf;
#pragma unroll
        for (int w = 0; w < 4; ++w) mx = fmaxf(mx, w_max[w][c]);
        const float ref = mx == -kInf ? 0.0f : mx;
        float acc = 0.0f, l = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(w_max[w][c] - ref);
            l += f * w_sum[w][c];
            acc += f * reinterpret_cast<const float *>(lds + w * kPerWave)[c * (DP + 4) + d];
        }
        if (work.splits == 1) {
            const int mm = P.m0 + c, tk = (uint32_t)mm / a.group_div, g = P.h * a.group + (mm - tk * a.group);
            ((T *)a.out)[(int64_t)(P.r.t0 + tk) * a.o_token + (int64_t)g * a.o_head + d] = (T)weighted(acc, l);
            if (a.lse && d == 0) a.lse[(int64_t)(P.r.t0 + tk) * (a.heads * a.group) + g] = log_sum(ref, l);
        } else {
            const int64_t at = ((work.item - a.whole) * a.splits + work.split) * 16 + c;
            a.part[at * D + d] = acc;
            if (d == 0) {
                *reinterpret_cast<f32x4 *>(a.stat + at * 4) = f32x4{mx, l, l, 0.0f};
            }
        }
    }
}

// ---- many pairs: 32x32 tiles, keys and values staged in LDS for all waves ----

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mma32(frag_t<__bf16> a, frag_t<__bf16> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(frag_t<_Float16> a, frag_t<_Float16> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(frag_t<float> a, frag_t<float> b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

// Sum of the weights as they are rounded for the second product: the output is divided by it, so that the rounding of a
// weight that outweighs all others cancels (the lazily raised maximum leaves it anywhere below 2^8). The log-sum-exp takes
// the sum before rounding.
template <typename T, int N>
__device__ __forceinline__ float rounded_sum(const frag_t<T> (&w)[N]) {
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            if constexpr (std::is_same<T, __bf16>::value) {
                typedef __bf16 v2 __attribute__((ext_vector_type(2)));
                s[(i >> 1) & 1] = __builtin_amdgcn_fdot2_f32_bf16(v2{w[n][i], w[n][i + 1]}, v2{(__bf16)1.0f, (__bf16)1.0f},
                                                                  s[(i >> 1) & 1], false);
            } else if constexpr (std::is_same<T, _Float16>::value) {
                typedef _Float16 v2 __attribute__((ext_vector_type(2)));
                s[(i >> 1) & 1] =
                    __builtin_amdgcn_fdot2(v2{w[n][i], w[n][i + 1]}, v2{(_Float16)1.0f, (_Float16)1.0f}, s[(i >> 1) & 1], false);
            } else {
                s[(i >> 1) & 1] += w[n][i] + w[n][i + 1];
            }
        }
    return s[0] + s[1];
}

// x, formed where this stands.
__device__ __forceinline__ float settled(float x) {
    asm volatile("" : "+v"(x));
    return x;
}

// Max and sum over the two lanes that hold one column (lanes l, l+32).
__device__ __forceinline__ float half_max(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float half_sum(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Where unit c (16 bytes) of row r lies in a staged tile of UPR units a row: keys are
// read by 16 lanes at the same unit of 16 rows, values (16-bit ones) by 32 lanes at four units of
// four rows; each such group of reads touches all 64 banks once.
template <int UPR>
__device__ __forceinline__ int key_unit(int r, int c) {
    return UPR >= 16 ? c ^ (r & 15) : c ^ ((r >> 1) & (UPR - 1));
}
template <int UPR, int SIZE>
__device__ __forceinline__ int value_unit(int r, int c) {
    if (SIZE == 4) return c;
    return UPR >= 16 ? c ^ ((r & 3) << 2) : c ^ (((r >> 1) & 1) << 2);
}

// One workgroup a (row, head, 32 pairs for each of its waves, share of the row's keys): the waves
// walk the keys together, KT at a time, staged in LDS, each with the queries, the
// statistics and the output of its own 32 pairs in registers.
// While a tile is computed the next one is on its way to registers; from there it is put into the other
// half of the LDS. Bound by the matrix unit and, at four waves or less, by what those wait for. 8192 tokens in rows of
// 64, 8 heads of 4 queries, 128 components, bf16, lists of 2048 keys: 349 us, 760 TFLOP/s of the products that count
// (no masked ones) with eight waves a workgroup, 367 us with four. Wide ones have no room for eight: 4096
// tokens of 2 sequences, 4 queries a head, 192 components 365 TFLOP/s, 256 components 273. fp32 runs at half of
// its matrix unit's rate (128 components, 78 TFLOP/s), 256 components, in part in scratch memory, at 33.
// The running maximum is raised only when a tile passes it by a factor of 2^8 or more: weights up
// to 2^8 are as exact as those up to 1, and the output is rescaled a few times a row instead of
// nearly every tile.
template <typename T, int NK, int NC, int KT, int THREADS>
__global__ __launch_bounds__(THREADS, NK <= 4 && sizeof(T) == 2 ? 2 : 1) void tiles_kernel(AttnArgs a) {
    constexpr int DP = NK * 32, W = kPer16<T>, UPR = DP / W, SIZE = (int)sizeof(T);
    constexpr int NL = KT * UPR / THREADS;  // units a thread stages of a tile's keys, and of its values
    constexpr int NS = KT / 16, NB = KT / 32, NQ = NC * 2, NT = NC;
    __shared__ __attribute__((aligned(16))) T lds[2][2][KT * DP];
    __shared__ Slabs S;
    __shared__ int any_odd;
    typedef typename VecOf<T, W>::type V;
    typedef typename VecOf<T, 4>::type V4;

    Work work;
    if (!find_work(a, work)) return;
    const Pairs P = find_pairs(a, work.item);
    if (P.r.n == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int D = a.dim;

    // Query of this lane's column. The sign of the scale goes into it.
    const int m = P.m0 + wave * 32 + col, tok = (uint32_t)m / a.group_div;
    const bool live = m < P.end;
    const int pos = live ? P.r.p0 + tok : -1;
    const float scale2 = fabsf(a.scale2);
    const int64_t head = (int64_t)P.h * a.group + (m - tok * a.group);
    frag_t<T> q[NQ];
    {
        const T *src = (const T *)a.q + (int64_t)(P.r.t0 + tok) * a.q_token + head * a.q_head;
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
            const int d = k * 16 + half * 8;
            q[k] = zero_frag<T>();
            if (live && d < D) {
                if (a.q_aligned) {
                    q[k] = *reinterpret_cast<const frag_t<T> *>(src + d);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) q[k][i] = src[d + i];
                }
                if (a.scale2 < 0.0f) q[k] = -q[k];
            }
        }
    }
    const int first_pos = P.r.p0 + (int)((uint32_t)P.m0 / a.group_div);
    const bool busy = P.m0 + wave * 32 < P.end;

    const int64_t slabs = slabs_of(a, P);
    const int64_t per = ((slabs + NS - 1) / NS + work.splits - 1) / work.splits * NS;
    const int64_t s_lo = min(per * work.split, slabs), s_hi = min(s_lo + per, slabs);

    f32x16 o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
    float top = -kInf, sum = 0.0f, norm = 0.0f;  // top: of the products before scaling; norm: sum of the rounded weights

    constexpr bool two = THREADS == 512;  // two waves a SIMD
    const bool late = wave >= 4;
    f32x16 x[NB];      // products of a tile, keys by pairs
    frag_t<T> w[NS];   // weights of a tile
    auto phase_end = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        __builtin_amdgcn_sched_barrier(0);
    };

    // What this thread stages of a tile: unit (lane % UPR) of rows lane / UPR from its wave's first
    // ones on; a wave's units of one turn lie in one slab.
    const int my_row = lane / UPR, my_unit = lane % UPR;
    const bool my = my_unit * W < D;
    const uint32_t my_at = my ? (uint32_t)(my_row * D + my_unit * W) : 0u;

    for (int64_t c0 = s_lo; c0 < s_hi; c0 += kSlabs) {
        __syncthreads();
        look_up<THREADS>(S, a, P, c0, s_hi, first_pos);
        if (tid == 0) any_odd = 0;
        __syncthreads();
        const int n_slabs = (int)min(s_hi - c0, (int64_t)kSlabs);
        bool odd = false;
        // Slabs that some pair does not see all of, a bit each.
        uint64_t part[kSlabs / 64];
#pragma unroll
        for (int i = 0; i < kSlabs / 64; ++i) part[i] = (uint64_t)uniform64((int64_t)S.part[i]);
        auto partial = [&](int t) {
            const int s = t * NS;
            const uint64_t lo = s & 64 ? part[1] : part[0], hi = s & 64 ? part[3] : part[2];
            return (((s & 128 ? hi : lo) >> (s & 63)) & ((1u << NS) - 1)) != 0;
        };
        auto keys_of = [&](int t, int (&k)[NS]) {
#pragma unroll
            for (int n = 0; n < NS; ++n) k[n] = __builtin_amdgcn_readfirstlane(S.key[t * NS + n]);
        };
        V kr[NL], vr[NL];
        // Where this thread's rows of a tile lie. (Of slabs that are not there the first page's rows are read, and
        // masked or zeroed below.)
        struct Places {
            int64_t at[NL];
        };
        auto places = [&](int t) {
            Places p;
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                p.at[i] = S.base[t * NS + (i * THREADS + wave * 64) / UPR / 16];
                if (NK == 8) p.at[i] = uniform64(p.at[i]);  // (the widest ones are short of vector registers)
            }
            return p;
        };
        auto fetch = [&](V (&r)[NL], const void *cache, const Places &p) {
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int row0 = (i * THREADS + wave * 64) / UPR;
                r[i] = *reinterpret_cast<const V *>((const T *)cache + p.at[i] + ((row0 & 15) * D + my_at));
            }
        };
        auto put_keys = [&](int t) {
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int row = (i * THREADS + wave * 64) / UPR + my_row;
                u32x4 v = __builtin_bit_cast(u32x4, kr[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = my ? v[e] : 0u;  // components behind the last one are zero
                *reinterpret_cast<u32x4 *>(&lds[0][t & 1][row * DP + key_unit<UPR>(row, my_unit) * W]) = v;
            }
        };
        auto put_values = [&](int t) {
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int row = (i * THREADS + wave * 64) / UPR + my_row;
                *reinterpret_cast<V *>(&lds[1][t & 1][row * DP + value_unit<UPR, SIZE>(row, my_unit) * W]) = vr[i];
            }
        };
        // Of a tile that some pairs do not see all of: values that no pair sees become zero, whatever lies there
        // (their weights are zero, and zero times infinity is not), and all others that are not finite too;
        // those come back in a pass of their own. Each thread for what it has put there.
        auto clean_values = [&](int t) {
            const int ln = fresh(lane), my_row = ln / UPR, my_unit = ln % UPR;
            if (my_unit * W >= D) return;
#pragma unroll 1
            for (int i = 0; i < NL; ++i) {
                const int row0 = (i * THREADS + wave * 64) / UPR, row = row0 + my_row;
                const int k0 = S.key[t * NS + row0 / 16];
                const bool seen = k0 >= 0 && k0 + (row & 15) <= P.last;
                V *at = reinterpret_cast<V *>(&lds[1][t & 1][row * DP + value_unit<UPR, SIZE>(row, my_unit) * W]);
                V v = *at;
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    const bool bad = not_finite((float)v[e]);
                    odd = odd || (seen && bad);
                    if (!seen || bad) v[e] = (T)0.0f;
                }
                *at = v;
            }
        };
        // Eight keys of values, as rows of the second product: components t*32 + col, slots of step n.
        auto value_frag = [&](const T *v, int t, int n, int lane) {
            const int half = lane >> 5, col = lane & 31;
            frag_t<T> f;
            if constexpr (SIZE == 2) {
                typedef short s16x4 __attribute__((ext_vector_type(4)));
                typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                union {
                    s16x4 h[2];
                    frag_t<T> f;
                } u;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int r = n * 16 + b * 8 + half * 4 + ((lane & 15) >> 2);
                    const int d = t * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
                    const T *src = v + r * DP + value_unit<UPR, SIZE>(r, d / W) * W + (d & (W - 1));
                    u.h[b] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)src);
                }
                f = u.f;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = v[(n * 16 + (i >> 2) * 8 + half * 4 + (i & 3)) * DP + t * 32 + col];
            }
            return f;
        };

        // Eight components of keys, as rows of the first product: keys b*32 + col, components k*16 + half*8 and on.
        auto key_frag = [&](const T *ks, int b, int k) {
            const int r = b * 32 + col;
            if constexpr (SIZE == 2) {
                return *reinterpret_cast<const frag_t<T> *>(ks + r * DP + key_unit<UPR>(r, k * 2 + half) * W);
            } else {
                union {
                    V h[2];
                    frag_t<T> f;
                } u;
                u.h[0] = *reinterpret_cast<const V *>(ks + r * DP + key_unit<UPR>(r, k * 4 + half * 2) * W);
                u.h[1] = *reinterpret_cast<const V *>(ks + r * DP + key_unit<UPR>(r, k * 4 + half * 2 + 1) * W);
                return u.f;
            }
        };
        // O^T += V^T P^T of tile t, if any, then S^T = K Q^T of tile t + 1. LDS reads run kLead matrix instructions
        // ahead of those that they feed.
        auto multiply = [&](auto with_outputs, int t) {
            constexpr int kOut = decltype(with_outputs)::value ? NS * NT : 0, kAll = kOut + NQ * NB, kLead = SIZE == 2 ? 4 : 2;
            const T *vs = lds[1][t & 1], *ks = lds[0][(t + 1) & 1];
            frag_t<T> f[kLead];
            auto read = [&](int i) {
                return i < kOut ? value_frag(vs, i % NT, i / NT, lane) : key_frag(ks, (i - kOut) % NB, (i - kOut) / NB);
            };
#pragma unroll
            for (int i = 0; i < kLead; ++i) f[i] = read(i);
#pragma unroll
            for (int i = 0; i < kAll; ++i) {
                if (i < kOut) {
                    o[i % NT] = mma32(f[i % kLead], w[i / NT], o[i % NT]);
                } else {
                    const int b = (i - kOut) % NB, k = (i - kOut) / NB;
                    f32x16 c = x[b];
                    if (k == 0) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) c[e] = 0.0f;
                    }
                    x[b] = mma32(f[i % kLead], q[k], c);
                }
                if (i + kLead < kAll) f[i % kLead] = read(i + kLead);
                if (SIZE == 4) __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (SIZE == 2) {
                // (Without this the compiler puts each read right before its use.)
                constexpr int kFirst = kOut >= kLead ? 2 * kLead : kLead;
                __builtin_amdgcn_sched_group_barrier(0x100, kFirst, 0);
#pragma unroll
                for (int i = 0; i < kAll; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    if (i < 2 * NL) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);  // the next tile's loads
                    if (i + kLead < kOut)
                        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                    else if (i + kLead < kAll)
                        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
            }
        };
        // Weights of tile t from its products.
        auto weights = [&](int t) {
            if (partial(t)) {
                int key0[NS];
                keys_of(t, key0);
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int k0 = key0[b * 2 + (i >> 3)], key = k0 + ((i >> 2) & 1) * 8 + half * 4 + (i & 3);
                        x[b][i] = k0 >= 0 && key <= pos ? x[b][i] : -kInf;
                    }
            }
            float hi4[4] = {-kInf, -kInf, -kInf, -kInf};
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) hi4[(i >> 1) & 3] = fmaxf(hi4[(i >> 1) & 3], x[b][i]);
            const float hi32 = half_max(fmaxf(fmaxf(hi4[0], hi4[1]), fmaxf(hi4[2], hi4[3])));
            if (__ballot((hi32 - top) * scale2 > 8.0f)) {
                const float up = fmaxf(top, hi32);
                const float shrink = up == -kInf ? 1.0f : __builtin_amdgcn_exp2f((top - up) * scale2);
                top = up;
                sum *= shrink;
                norm *= shrink;
#pragma unroll
                for (int n = 0; n < NT; ++n) o[n] *= shrink;
            }
            const float ref = top == -kInf ? 0.0f : -top * scale2;
            // (In steps of their own: the compiler would otherwise put each exponential behind
            // its argument and before its sum, and wait for each.)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[b][i] = fmaf(x[b][i], scale2, ref);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[b][i] = __builtin_amdgcn_exp2f(x[b][i]);
            __builtin_amdgcn_sched_barrier(0);
            float total[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    total[i & 3] += x[b][i];
                    w[b * 2 + (i >> 3)][i & 7] = (T)x[b][i];
                }
            // (The sums are needed in the next tile only; formed there, they would keep all weights in registers.)
            sum = settled(sum + ((total[0] + total[1]) + (total[2] + total[3])));
            norm = settled(norm + rounded_sum<T, NS>(w));
        };

        // Each tile takes a phase of matrix products (outputs of the tile before, products of this one) and
        // one of exponentials. With eight waves two share a SIMD: the second four run a phase
        // behind the first, so that the matrix unit and the vector unit of a SIMD are both busy; a barrier
        // parts the phases (with four waves or less, other workgroups fill the gaps, and one barrier a
        // tile is enough). Keys of tile t + 1 and values of tile t are put into LDS in the
        // products' phase of tile t: at that time nobody reads those halves of the LDS any more, and
        // their first reader comes a barrier later. The loads for the next such phase start there too.
        const int tiles = (n_slabs + NS - 1) / NS;
        auto stage = [&](int t, const Places &keys, const Places &values) {
            put_keys(t + 1);
            put_values(t);
            fetch(kr, a.k_cache, keys);
            fetch(vr, a.v_cache, values);
        };
        fetch(kr, a.k_cache, places(0));
        fetch(vr, a.v_cache, places(0));
        put_keys(0);
        fetch(kr, a.k_cache, places(1));
        __syncthreads();
        if (two && late) phase_end();
        stage(0, places(2), places(1));
        if (partial(0)) clean_values(0);
        // (The products behind the last tile are of what the LDS holds, and not used: a loop that
        // is left in its middle makes the compiler copy the accumulators.)
        if (busy) {
            multiply(std::false_type{}, -1);
            if (two) phase_end();
            for (int t = 0; t < tiles; ++t) {
                const Places keys = places(t + 3), values = places(t + 2);
                weights(t);
                phase_end();
                stage(t + 1, keys, values);
                multiply(std::true_type{}, t);
                if (partial(t + 1)) clean_values(t + 1);
                if (two) phase_end();
            }
        } else {
            if (two) phase_end();
            for (int t = 0; t < tiles; ++t) {
                phase_end();
                stage(t + 1, places(t + 3), places(t + 2));
                if (partial(t + 1)) clean_values(t + 1);
                if (two) phase_end();
            }
        }
        if (two && !late) phase_end();
        if (odd) any_odd = 1;
        __syncthreads();
        if (any_odd) {
            // Values that are not finite, where some see a part of the tile only: products of
            // who sees a key (1 or 0) with where its value is +infinity or NaN, then
            // -infinity or NaN, say which outputs take part.
            for (int u = 0; u < tiles; ++u) {
                if (!partial(u)) continue;
                int key0[NS];
                keys_of(u, key0);
                for (int sign = 0; sign < 2; ++sign) {
                    const int ln = fresh(lane), my_row = ln / UPR, my_unit = ln % UPR;
#pragma unroll 1
                    for (int i = 0; i < NL; ++i) {
                        const int row0 = (i * THREADS + wave * 64) / UPR, row = row0 + my_row;
                        const int k0 = S.key[u * NS + row0 / 16];
                        const bool seen = k0 >= 0 && k0 + (row & 15) <= P.last && my_unit * W < D;
                        V v;
#pragma unroll
                        for (int e = 0; e < W; ++e) v[e] = (T)0.0f;
                        if (seen)
                            v = *reinterpret_cast<const V *>((const T *)a.v_cache + S.base[u * NS + row0 / 16] +
                                                             (row & 15) * D + my_unit * W);
#pragma unroll
                        for (int e = 0; e < W; ++e) {
                            const float f = (float)v[e];
                            v[e] = (T)(f != f || f == (sign ? -kInf : kInf) ? 1.0f : 0.0f);
                        }
                        *reinterpret_cast<V *>(&lds[1][0][row * DP + value_unit<UPR, SIZE>(row, my_unit) * W]) = v;
                    }
                    __syncthreads();
                    const int p0 = fresh(pos) - (ln >> 5) * 4;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        f32x16 hit;
#pragma unroll
                        for (int i = 0; i < 16; ++i) hit[i] = 0.0f;
#pragma unroll
                        for (int n = 0; n < NS; ++n) {
                            frag_t<T> see;
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                see[i] = (T)(key0[n] >= 0 && key0[n] + (i >> 2) * 8 + (i & 3) <= p0 ? 1.0f : 0.0f);
                            hit = mma32(value_frag(lds[1][0], t, n, ln), see, hit);
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (hit[i] > 0.0f) o[t][i] += sign ? -kInf : kInf;
                    }
                    __syncthreads();
                }
            }
        }
    }
    if (!live) return;
    // (Addresses are formed anew: kept through the loops they would take registers from them.)
    const int ln = fresh(lane), out_half = ln >> 5, out_m = P.m0 + wave * 32 + (ln & 31);
    const int out_tok = (uint32_t)out_m / a.group_div;
    const int64_t o_head_at = (int64_t)P.h * a.group + (out_m - out_tok * a.group);
    sum = half_sum(sum);
    norm = half_sum(norm);
    const float ref = top == -kInf ? 0.0f : top * scale2;
    if (work.splits == 1) {
        T *dst = (T *)a.out + (int64_t)(P.r.t0 + out_tok) * a.o_token + o_head_at * a.o_head;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = t * 32 + (i >> 2) * 8 + out_half * 4;
                if (d >= D) continue;
                V4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (T)weighted(o[t][i + e], norm);
                if (a.o_aligned) {
                    *reinterpret_cast<V4 *>(dst + d) = v;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) dst[d + e] = v[e];
                }
            }
        if (a.lse && out_half == 0) a.lse[(int64_t)(P.r.t0 + out_tok) * (a.heads * a.group) + o_head_at] = log_sum(ref, sum);
    } else {
        const int64_t at = ((work.item - a.whole) * a.splits + work.split) * a.tile_pairs + wave * 32 + (ln & 31);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = t * 32 + (i >> 2) * 8 + out_half * 4;
                if (d < D)
                    *reinterpret_cast<f32x4 *>(a.part + at * D + d) = f32x4{o[t][i], o[t][i + 1], o[t][i + 2], o[t][i + 3]};
            }
        if (out_half == 0) {
            *reinterpret_cast<f32x4 *>(a.stat + at * 4) = f32x4{top == -kInf ? -kInf : top * scale2, sum, norm, 0.0f};
        }
    }
}

constexpr int kMostSplits = 512, kFewSplits = 16;

// Joins many shares of a pair (64 shares of 32 pairs of 128 components 4.5 us, the latency of two dependent loads and
// the launch): one workgroup a (row, head, tile, pair). The factors of the shares are formed by a
// thread each, then the shares are summed by 256 / (dim / 4) groups of threads, four components a thread, eight loads ahead.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(AttnArgs a) {
    __shared__ float factor[kMostSplits];
    __shared__ float red[12];
    __shared__ f32x4 sums[256];
    const int64_t idx = grid_index();
    if (idx >= (a.items - a.whole) * a.tile_pairs) return;
    const uint32_t item = (uint32_t)idx / a.pair_div;  // from `whole` on
    const int c = (int)((uint32_t)idx - item * a.pair_div.d);
    const Pairs P = find_pairs(a, (uint32_t)a.whole + item);
    if (P.r.n == 0 || P.m0 + c >= P.end) return;
    const int step = a.tile_pairs;  // from share to share
    const f32x4 *stat = reinterpret_cast<const f32x4 *>(a.stat) + ((int64_t)item * a.splits * step + c);
    const float *part = a.part + ((int64_t)item * a.splits * step + c) * a.dim;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    static_assert(kMostSplits == 2 * 256, "two shares a thread");
    f32x4 x[2];
    float mx = -kInf;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int s = tid + i * 256;
        x[i] = f32x4{-kInf, 0.0f, 0.0f, 0.0f};
        if (s < a.splits) x[i] = stat[s * step];
        mx = fmaxf(mx, x[i][0]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
    if (lane == 0) red[wave] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float ref = mx == -kInf ? 0.0f : mx;
    float l = 0.0f, norm = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float f = __builtin_amdgcn_exp2f(x[i][0] - ref);
        factor[tid + i * 256] = f;
        l += f * x[i][1];
        norm += f * x[i][2];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        l += __shfl_xor(l, o);
        norm += __shfl_xor(norm, o);
    }
    if (lane == 0) {
        red[4 + wave] = l;
        red[8 + wave] = norm;
    }
    __syncthreads();
    l = (red[4] + red[5]) + (red[6] + red[7]);
    norm = (red[8] + red[9]) + (red[10] + red[11]);

    const int quads = a.dim / 4, groups = 256 / quads, g = tid / quads, u = tid - g * quads;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    if (g < groups) {
        const int64_t stride = (int64_t)step * a.dim;
#pragma unroll 8
        for (int s = g; s < a.splits; s += groups)
            acc += factor[s] * *reinterpret_cast<const f32x4 *>(part + s * stride + u * 4);
    }
    sums[tid] = acc;
    __syncthreads();
    if (tid >= quads) return;
    for (int k = 1; k < groups; ++k) acc += sums[k * quads + u];
    const int m = P.m0 + c, tok = (uint32_t)m / a.group_div, head = P.h * a.group + (m - tok * a.group);
    T *dst = (T *)a.out + (int64_t)(P.r.t0 + tok) * a.o_token + (int64_t)head * a.o_head + u * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = (T)weighted(acc[e], norm);
    if (a.lse && tid == 0) a.lse[(int64_t)(P.r.t0 + tok) * (a.heads * a.group) + head] = log_sum(ref, l);
}

// The same for few shares: `lanes` (a power of two, 16 to 64, dim / 4 or more) threads a pair, four components each, over
// all shares; a workgroup's pairs are of one tile. (A workgroup a pair spends its time on being started: 248 tiles of 128
// pairs, two shares of 64 components, whole call 75 us by that and 30 by this; 42 shares of 16 tiles 23 and 32.)
template <typename T>
__global__ __launch_bounds__(256) void join_few_kernel(AttnArgs a, int lanes_log2) {
    const int pairs = 256 >> lanes_log2;  // of a workgroup
    const int64_t idx = grid_index() * pairs;
    if (idx >= (a.items - a.whole) * a.tile_pairs) return;
    const uint32_t item = (uint32_t)idx / a.pair_div;  // from `whole` on
    const int c = (int)((uint32_t)idx - item * a.pair_div.d) + (int)(threadIdx.x >> lanes_log2);
    const Pairs P = find_pairs(a, (uint32_t)a.whole + item);
    const int u = threadIdx.x & ((1 << lanes_log2) - 1);
    if (P.r.n == 0 || P.m0 + c >= P.end || u * 4 >= a.dim) return;
    const int step = a.tile_pairs;  // from share to share
    const f32x4 *stat = reinterpret_cast<const f32x4 *>(a.stat) + ((int64_t)item * a.splits * step + c);
    const float *part = a.part + ((int64_t)item * a.splits * step + c) * a.dim + u * 4;
    float mx = -kInf;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) mx = fmaxf(mx, stat[s * step][0]);
    const float ref = mx == -kInf ? 0.0f : mx;
    float l = 0.0f, norm = 0.0f;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
        const f32x4 x = stat[s * step];
        const float f = __builtin_amdgcn_exp2f(x[0] - ref);
        l += f * x[1];
        norm += f * x[2];
        acc += f * *reinterpret_cast<const f32x4 *>(part + (int64_t)s * step * a.dim);
    }
    const int m = P.m0 + c, tok = (uint32_t)m / a.group_div, head = P.h * a.group + (m - tok * a.group);
    T *dst = (T *)a.out + (int64_t)(P.r.t0 + tok) * a.o_token + (int64_t)head * a.o_head + u * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = (T)weighted(acc[e], norm);
    if (a.lse && u == 0) a.lse[(int64_t)(P.r.t0 + tok) * (a.heads * a.group) + head] = log_sum(ref, l);
}

struct Plan {
    int64_t items, whole;
    int waves;  // of the tiles kernel; 0: the rows kernel
    int tile_pairs, tiles, splits;
    spconv_batch batch;  // with the rows of this call
    int64_t part_bytes, bytes;
};

// False for sizes out of range.
bool plan_of(int dtype, const spconv_batch *B, int q_heads, int heads, int dim, int keep, Plan *p) {
    const int group = q_heads / heads;
    const int most = dtype == SPCONV_F32 || dim > 128 ? 4 : 8;  // waves of a tile: two a SIMD where registers allow
    p->batch = *B;
    // Without lists rows mean nothing to the result: they are as long as a tile has room for, and sequences tokens.
    // (Two sequences, 1000 tokens, 4 heads of 4 queries and 128 components, rows of one token given: 549 -> 66 us.)
    if (keep == 0 && !B->q_start) p->batch.q_block = 1;  // (then no row is empty)
    if (keep == 0 && B->q_start) {
        const int64_t tokens = (B->tokens + B->sequences - 1) / B->sequences;
        int q = std::min(std::max(most * 32 / group, 1), 128);
        while (q > 1 && (q + 1) / 2 >= tokens) q = (q + 1) / 2;
        p->batch.q_block = q;
    }
    B = &p->batch;
    const int64_t pairs = (int64_t)row_tokens(B) * group;
    p->waves = 0;
    p->tile_pairs = 16;
    // Rows of more pairs than these are tiles of 32 pairs for each of some waves. (128 components, bf16, 2000 tokens: 16
    // pairs 73 us by rows and 123 by tiles, 32 pairs 74 and 64; fp32 of 64 components, 32 pairs: 86 and 107. Wide ones
    // keep a CU busy with four waves only, of which few pairs leave three or two idle: 32 pairs of 2000 tokens, 256
    // components, 239 us by tiles and 210 by rows; fp32 1134 and 531, 64 pairs 712 and 528.)
    const bool f32 = dtype == SPCONV_F32;
    const int few = dim <= 64 ? (f32 ? 32 : 16) : dim <= 128 ? 16 : f32 ? 64 : dim > 192 ? 32 : 16;
    // (fp32 of more than 192: five and a half tiles of 16 pairs cost one of 128; 132 pairs 615 and 737 us.)
    const bool by_rows = pairs <= few || (f32 && dim > 192 && (pairs + 15) / 16 * 2 < (pairs + 127) / 128 * 11);
    if (!by_rows) {
        p->waves = dim > 192 ? 4 : 2;  // (the widest ones' registers hold a quarter of a tile's loads, not a half)
        while (p->waves < most && p->waves * 32 < pairs) p->waves *= 2;
        p->tile_pairs = p->waves * 32;
    }
    p->tiles = (int)((pairs + p->tile_pairs - 1) / p->tile_pairs);
    p->items = rows_of(B) * heads * p->tiles;
    if (p->items >= ((int64_t)1 << 27)) return false;
    // The GPU holds `slots` workgroups at a time: one of eight waves or of wide rows on a CU, two of the others. Items that
    // do not fill a round of them are split along their keys (128 keys a share at least), so that they do.
    const int64_t slots = p->waves == 8 || (p->waves == 0 && dim > (f32 ? 64 : 128)) ? 256 : 512;
    const int64_t keys = (int64_t)(keep ? keep : B->max_blocks) * B->block;
    const int64_t rest = p->items % slots;
    // (Behind sixteen full rounds the last one does not matter.)
    // Without lists rows' keys differ, by sequence or by position: single tokens of several sequences, or tiles that would
    // fill more than half a round, get two rounds of shares to even that out (48 sequences of 100 to 16384 keys, one head
    // of 256 components: 99 -> 66 us; 4096 tokens, 16-bit, 192: 645 -> 368; of equal lengths, 16 sequences: 36 -> 41).
    const bool uneven = keep == 0 && (p->waves == 0 ? B->sequences > 1 : rest > slots / 2);
    // Few keys are walked sooner than a second launch comes (8 lists of 512 keys of 128 components, bf16: 19 us, split 24;
    // fp32 28 and 23).
    const bool short_rows = p->waves == 0 ? keys * dim * size_of(dtype) <= 128 << 10 : keys <= 256;
    const int64_t splits = rest && !short_rows && p->items <= 16 * slots
                               ? std::min({(uneven ? 2 : 1) * slots / rest, (keys + 127) / 128, (int64_t)kMostSplits})
                               : 1;
    p->splits = (int)std::max<int64_t>(1, splits);
    p->whole = p->splits > 1 ? p->items - rest : p->items;
    p->part_bytes = p->bytes = 0;
    if (p->splits > 1) {
        p->part_bytes = rest * p->splits * p->tile_pairs * dim * 4;
        p->bytes = p->part_bytes + rest * p->splits * p->tile_pairs * 4 * 4;
    }
    return true;
}

template <typename T, int NK, int NC, int KT>
void launch_tiles(const AttnArgs &a, int waves, dim3 grid, hipStream_t stream) {
    if (waves == 4) {
        tiles_kernel<T, NK, NC, KT, 256><<<grid, 256, 0, stream>>>(a);
    } else if (waves == 2) {
        if constexpr (NC <= (sizeof(T) == 2 ? 6 : 4)) tiles_kernel<T, NK, NC, KT, 128><<<grid, 128, 0, stream>>>(a);
    } else {
        if constexpr (sizeof(T) == 2 && NK <= 4) tiles_kernel<T, NK, NC, KT, 512><<<grid, 512, 0, stream>>>(a);
    }
}

template <typename T>
int attention_of(const AttnArgs &a, const Plan &p, hipStream_t stream) {
    const dim3 grid = grid_of(a.whole + (a.items - a.whole) * a.splits);
    if (p.waves == 0) {
        if (a.dim <= 64)
            rows_kernel<T, 2, 2><<<grid, 256, 0, stream>>>(a);
        else if (a.dim <= 128)
            rows_kernel<T, 4, 4><<<grid, 256, 0, stream>>>(a);
        else if (a.dim <= 192)
            rows_kernel<T, 8, 6><<<grid, 256, 0, stream>>>(a);
        else
            rows_kernel<T, 8, 8><<<grid, 256, 0, stream>>>(a);
    } else {
        if (a.dim <= 64)
            launch_tiles<T, 2, 2, sizeof(T) == 4 ? 32 : 64>(a, p.waves, grid, stream);
        else if (a.dim <= 128)
            launch_tiles<T, 4, 4, sizeof(T) == 4 ? 32 : 64>(a, p.waves, grid, stream);
        else if (a.dim <= 192)
            launch_tiles<T, 8, 6, 32>(a, p.waves, grid, stream);
        else
            launch_tiles<T, 8, 8, 32>(a, p.waves, grid, stream);
    }
    if (hipGetLastError() != hipSuccess) return SPCONV_EHIP;
    if (a.splits > 1) {
        const int64_t pairs = (a.items - a.whole) * a.tile_pairs;
        if (a.splits <= kFewSplits) {
            const int lanes_log2 = a.dim <= 64 ? 4 : a.dim <= 128 ? 5 : 6;
            const int64_t per = 256 >> lanes_log2;
            join_few_kernel<T><<<grid_of((pairs + per - 1) / per), 256, 0, stream>>>(a, lanes_log2);
        } else {
            join_kernel<T><<<grid_of(pairs), 256, 0, stream>>>(a);
        }
        return launched();
    }
    return SPCONV_OK;
}

}  // namespace

extern "C" int spconv_attention_workspace(int dtype, const spconv_batch *batch, int q_heads, int heads, int dim, int keep,
                                          int64_t *bytes) {
    Plan p;
    if (!batch_ok(batch) || !dtype_ok(dtype) || !heads_ok(q_heads, heads, dim) || keep < 0 || bytes == nullptr ||
        !plan_of(dtype, batch, q_heads, heads, dim, keep, &p))
        return SPCONV_EINVAL;
    *bytes = p.bytes;
    return SPCONV_OK;
}

extern "C" int spconv_block_attention(int dtype, const spconv_batch *batch, const void *q, int64_t q_token,
                                      int64_t q_head, int q_heads, int heads, int dim, const void *k_cache,
                                      const void *v_cache, float scale, const int32_t *blocks, const int32_t *counts,
                                      int keep, void *out, int64_t out_token, int64_t out_head, float *lse,
                                      void *workspace, int64_t workspace_bytes, hipStream_t stream) {
    Plan p;
    if (!batch_ok(batch) || !batch_arrays_ok(batch) || !dtype_ok(dtype) || !heads_ok(q_heads, heads, dim) ||
        q == nullptr || k_cache == nullptr || v_cache == nullptr || out == nullptr || q_token < 0 || q_head < 0 ||
        !out_strides_ok(batch->tokens, q_heads, dim, out_token, out_head) || !aligned16(k_cache) ||
        !aligned16(v_cache) || !std::isfinite(scale * kLog2e) || keep < 0 || (blocks == nullptr) != (keep == 0) ||
        (counts != nullptr && blocks == nullptr) || out == q || !plan_of(dtype, batch, q_heads, heads, dim, keep, &p))
        return SPCONV_EINVAL;
    if (p.bytes > 0 && (workspace == nullptr || !aligned16(workspace) || workspace_bytes < p.bytes)) return SPCONV_EINVAL;
    // Zero times what is masked, -infinity, would be NaN: the least number stands for a scale of zero (products
    // below 2^100 come out as 0 all the same).
    const float scale2 = scale == 0.0f ? 0x1p-149f : scale * kLog2e;
    AttnArgs a{p.batch, q, q_token, q_head, k_cache, v_cache, blocks, counts, out, out_token, out_head, lse,
               (float *)workspace, nullptr, p.items, p.whole, heads, q_heads / heads, dim, keep, p.tiles, p.splits,
               rows_aligned16(q, q_token, q_head, size_of(dtype)),
               rows_aligned16(out, out_token, out_head, size_of(dtype)), p.tile_pairs, scale2,
               make_div((uint32_t)p.tiles), make_div((uint32_t)heads), make_div((uint32_t)(q_heads / heads)),
               make_div((uint32_t)p.splits), make_div((uint32_t)(batch->block / 16)), make_div((uint32_t)p.tile_pairs)};
    if (p.bytes > 0) a.stat = (float *)((char *)workspace + p.part_bytes);
    if (dtype == SPCONV_F32) return attention_of<float>(a, p, stream);
    if (dtype == SPCONV_F16) return attention_of<_Float16>(a, p, stream);
    return attention_of<__bf16>(a, p, stream);
}
