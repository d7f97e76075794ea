// Rotary positions and the paged cache's append (spconv_rope, spconv_cache_append).
//
// Both only move data: a rotated pair takes four products and a sine and cosine
// that all heads of a token share, so both are bound by HBM (each element read and
// written once) or, for single tokens, by the launch.
//
// Angles: position * frequency is rounded to fp64 once. How many half turns that is, less whole turns, is formed
// there with 1/pi in two parts and the product's own rounding, so that positions near 2^31, which turn the fastest pair
// 3e8 times, lose nothing. The rest, at most half a turn, goes through fp32 sine and cosine of a multiple
// of pi, and what its rounding to fp32 left out comes in by their derivatives: each is within 2^-23 + 2^-25 of that of
// the fp64 angle whatever the position. (In fp64 throughout: 84 -> 100 us for rot 26 of 88, append of 14001 tokens 33 -> 35.)
#include "batch.h"

namespace {

struct CosSin {
    float c, s;
};

__device__ __forceinline__ CosSin rope_angle(int position, double freq, float sign, float amplitude) {
    constexpr double kHigh = 0.3183098861837907, kLow = -1.9678676675182486e-17;  // 1 / pi
    const double angle = (double)position * freq, half_turns = angle * kHigh;
    const double tail = fma(angle, kHigh, -half_turns) + angle * kLow;
    const double part = half_turns - 2.0 * rint(0.5 * half_turns) + tail;
    const float near = (float)part, rest = (float)(part - near) * 3.14159265f;  // sin(a + r) = sin a + r cos a
    float s, c;
    sincospif(near, &s, &c);
    return {fmaf(-s, rest, c) * amplitude, fmaf(c, rest, s) * amplitude * sign};
}

// W pairs: x of the first components, y of the second ones (half layout), or, in
// the interleaved layout of W > 1, 2W neighbours (x then y).
template <int W, bool INTER>
__device__ __forceinline__ void rotate(Floats<W> &x, Floats<W> &y, const CosSin (&a)[W]) {
    if constexpr (INTER && W > 1) {
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
            const float u = x.v[2 * i], v = x.v[2 * i + 1], p = y.v[2 * i], q = y.v[2 * i + 1];
            const CosSin m = a[i], n = a[W / 2 + i];
            x.v[2 * i] = u * m.c - v * m.s;
            x.v[2 * i + 1] = v * m.c + u * m.s;
            y.v[2 * i] = p * n.c - q * n.s;
            y.v[2 * i + 1] = q * n.c + p * n.s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float u = x.v[i], v = y.v[i];
            x.v[i] = u * a[i].c - v * a[i].s;
            y.v[i] = v * a[i].c + u * a[i].s;
        }
    }
}

// Where the two vectors of pairs [u*W, u*W + W) start.
template <int W, bool INTER>
__device__ __forceinline__ void pair_at(int u, int rot, int &d0, int &d1) {
    d0 = INTER ? 2 * u * W : u * W;
    d1 = INTER ? d0 + W : d0 + rot / 2;
}

struct RopeArgs {
    const void *x;
    void *out;
    int64_t x_token, x_head, o_token, o_head;
    const int32_t *positions;
    const double *freq;
    int64_t tokens;
    int heads, dim, rot, group;  // group: tokens a workgroup takes at a time
    Div half, units, row;        // rot/2; vectors of a head (pairs and copies); heads * units
    float sign, amplitude;
};

// A workgroup takes `group` tokens: their sines and cosines into LDS, once for all
// heads, then every (token, head, vector pair) by one thread. Vectors are the widest that pairs and copies split into.
// 16384 tokens, 32 heads, bf16: 128 components in whole vectors 44 us, 6.1 TB/s (of inputs that the last-level cache
// does not hold 50 us, 5.4); rot 40 of 96 by four components 4.4 TB/s, rot 36 of 80 by two 4.0, rot 26 of
// 88, one by one, 2.2, bound by the number of its loads and stores.
template <typename T, int W, bool INTER>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    extern __shared__ CosSin table[];
    const int tid = threadIdx.x;
    const T *x = (const T *)a.x;
    T *out = (T *)a.out;
    const int64_t groups = (a.tokens + a.group - 1) / a.group;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t t0 = g * a.group;
        const int n = (int)min((int64_t)a.group, a.tokens - t0);
        __syncthreads();
        for (int i = tid; i < n * (int)a.half.d; i += 256) {
            const int t = (uint32_t)i / a.half;
            table[i] = rope_angle(a.positions[t0 + t], a.freq[i - t * (int)a.half.d], a.sign, a.amplitude);
        }
        __syncthreads();
        const int total = n * (int)a.row.d;
        // Narrow vectors: as many on their way as make 16 bytes, four at most.
        constexpr int kAhead = 16 / (W * (int)sizeof(T)) < 4 ? 16 / (W * (int)sizeof(T)) : 4;
        for (int i0 = tid; i0 < total; i0 += 256 * kAhead) {
            typedef typename VecOf<T, W>::type V;
            V p[kAhead], q[kAhead];
            T *y0[kAhead], *y1[kAhead];
            const CosSin *angles[kAhead];  // null: copied
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int i = min(i0 + 256 * k, total - 1);
                const int t = (uint32_t)i / a.row, r = i - t * (int)a.row.d;
                const int h = (uint32_t)r / a.units, u = r - h * (int)a.units.d;
                const T *xr = x + (t0 + t) * a.x_token + h * a.x_head;
                T *yr = out + (t0 + t) * a.o_token + h * a.o_head;
                int d0 = a.rot / 2 + u * W, d1 = d0;  // copied: rot + (u - rot/2/W) * W
                const bool pair = u * W < a.rot / 2;
                if (pair) pair_at<W, INTER>(u, a.rot, d0, d1);
                angles[k] = pair ? table + t * (int)a.half.d + u * W : nullptr;
                p[k] = *reinterpret_cast<const V *>(xr + d0);
                q[k] = *reinterpret_cast<const V *>(xr + d1);
                y0[k] = yr + d0;
                y1[k] = yr + d1;
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (kAhead > 1 && i0 + 256 * k >= total) break;
                if (angles[k]) {
                    Floats<W> f = floats_of<T, W>(p[k]), g = floats_of<T, W>(q[k]);
                    CosSin m[W];
#pragma unroll
                    for (int e = 0; e < W; ++e) m[e] = angles[k][e];
                    rotate<W, INTER>(f, g, m);
                    store_floats<T, W>(y0[k], f);
                    store_floats<T, W>(y1[k], g);
                } else {
                    *reinterpret_cast<V *>(y0[k]) = p[k];
                }
            }
        }
    }
}

struct AppendArgs {
    spconv_batch B;
    const void *k, *v;
    int64_t k_token, k_head, v_token, v_head;
    void *k_cache, *v_cache;
    float *sums;
    const int32_t *positions;
    const double *freq;
    int64_t items;  // touched pages
    int heads, dim, rot;
    int each;       // heads that a workgroup takes one after another
    int rows;       // rows of a page whose sines fit the table at a time
    int table_len;
    int all_units, all_vecs;             // vectors of a key (pairs and copies) and of a value
    Div parts, head_groups;              // workgroups that share a page's components; heads / each
    Div units, vecs, half;               // of a part: vectors of a key and of a value, pairs
    float amplitude;
};

constexpr int kTable = 4096;  // sines and cosines in LDS at most

// One workgroup a (touched page, group of heads, part of the components: one part where there are enough pages and heads
// for the GPU; 2254 tokens of 4 sequences, one head of 192, pages of 128 keys: 26 us by one part, 15 by three).
// The pages that sequence b touches are items
// q_start[b]/block + 2b and on: a sequence of n tokens touches n/block + 2 pages at
// most. Sines and cosines of the page's new tokens are formed once for the group's heads, in LDS. Threads hold one
// vector pair of a key each and walk the page's rows in strides, so that the
// page's sum is a sum of a thread's rows and then of 256/units threads, always in the same order: no atomics.
// Bound by HBM where the page is new; single tokens read the page's older keys, for the sum, and are bound by
// the latency of length, page and keys one after another.
template <typename T, int W, bool INTER>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
    extern __shared__ CosSin table[];                             // sines of the new rows, then
    float *part = reinterpret_cast<float *>(table + a.table_len);  // [groups][dim] partial sums
    typedef typename VecOf<T, W>::type V;
    const int64_t idx = grid_index();
    if (idx >= a.items * a.head_groups.d * a.parts.d) return;
    const uint32_t whole = (uint32_t)idx / a.parts;
    const int share = (int)((uint32_t)idx - whole * a.parts.d);
    const uint32_t item = whole / a.head_groups;
    const int h0 = (int)(whole - item * a.head_groups.d) * a.each;
    const spconv_batch &B = a.B;
    const Seq s = find_seq(B, (int)item, B.block, 2);
    if (s.b < 0 || s.at < 0 || s.n == 0 || s.kv == 0) return;
    const int from = s.kv - s.n;  // position of the first new token (tokens at negative ones are dropped)
    const int64_t block64 = max(from, 0) / B.block + (int64_t)s.at;
    if (block64 > (s.kv - 1) / B.block) return;
    const int j = (int)block64;
    const int page = uniform(page_of(B, s.b, j));
    if (page < 0) return;
    const int s0 = max(from - j * B.block, 0), s1 = min(s.kv - j * B.block, B.block);
    const int t_off = s.first + j * B.block - from;  // token of slot s: s + t_off
    const int tid = threadIdx.x;

    const int units = a.units.d, groups = 256 / units;
    const int g = (uint32_t)tid / a.units, ul = tid - g * units, u0 = share * units, u = u0 + ul;
    const bool mine = g < groups && u < a.all_units;
    const bool pair = u * W < a.rot / 2;
    // Where vector u of a key starts, and a pair's second one.
    auto place = [&](int u, int &d0, int &d1) {
        d0 = d1 = a.rot / 2 + u * W;
        if (u * W < a.rot / 2) pair_at<W, INTER>(u, a.rot, d0, d1);
    };
    int d0, d1;
    place(u, d0, d1);
    const int v0 = share * (int)a.vecs.d, vecs = min((int)a.vecs.d, a.all_vecs - v0);

    auto angles = [&](int r0, int r1) {  // of slots [r0, r1)
        if (u0 * W >= a.rot / 2) return;
        for (int i = tid; i < (r1 - r0) * (int)a.half.d; i += 256) {
            const int r = (uint32_t)i / a.half, t = r0 + r + t_off, f = u0 * W + i - r * (int)a.half.d;
            if (f < a.rot / 2)
                table[i] = rope_angle(a.positions ? a.positions[t] : j * B.block + r0 + r, a.freq[f], 1.0f, a.amplitude);
        }
    };
    const bool once = s1 - s0 <= a.rows;
    if (once) angles(s0, s1);
    for (int h = h0; h < min(h0 + a.each, a.heads); ++h) {
        const int64_t base = ((int64_t)page * a.heads + h) * B.block * a.dim;
        T *kc = (T *)a.k_cache + base, *vc = (T *)a.v_cache + base;
        // Values: copied.
        const int nv = vecs > 0 ? (s1 - s0) * (int)a.vecs.d : 0;
        for (int i = tid; i < nv; i += 256) {
            // (Behind a part's last vector: that again.)
            const int r = (uint32_t)i / a.vecs, c = (v0 + min(i - r * (int)a.vecs.d, vecs - 1)) * W;
            const V x = *reinterpret_cast<const V *>((const T *)a.v + (int64_t)(s0 + r + t_off) * a.v_token + h * a.v_head + c);
            __builtin_nontemporal_store(x, reinterpret_cast<V *>(vc + (int64_t)(s0 + r) * a.dim + c));
        }
        // Keys: rotated, stored, summed, older ones only summed; as many new rows at a time as the table holds.
        Floats<W> sum0, sum1;
#pragma unroll
        for (int i = 0; i < W; ++i) sum0.v[i] = sum1.v[i] = 0.0f;
        for (int n0 = s0; n0 < s1; n0 += a.rows) {
            const int n1 = min(n0 + a.rows, s1);
            if (!once) {
                __syncthreads();
                angles(n0, n1);
            }
            __syncthreads();
            if (!mine) continue;
            for (int r = (n0 > s0 ? n0 : a.sums ? 0 : s0) + g; r < n1; r += groups) {
                T *dst = kc + (int64_t)r * a.dim;
                const T *src = r < s0 ? dst : (const T *)a.k + (int64_t)(r + t_off) * a.k_token + h * a.k_head;
                Floats<W> p = load_floats<T, W>(src + d0), q = load_floats<T, W>(src + d1);
                if (r >= s0) {
                    if (pair) {
                        CosSin m[W];
#pragma unroll
                        for (int k = 0; k < W; ++k) m[k] = table[(r - n0) * (int)a.half.d + ul * W + k];
                        rotate<W, INTER>(p, q, m);
                        q = store_floats<T, W>(dst + d1, q);
                    }
                    p = store_floats<T, W>(dst + d0, p);
                }
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    sum0.v[i] += p.v[i];
                    sum1.v[i] += q.v[i];  // (of a copied vector: not used)
                }
            }
        }
        if (a.sums == nullptr) continue;
        const int first = units * W, row = 2 * first;  // the first vectors of all units, then the second ones
        if (mine) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                part[g * row + ul * W + i] = sum0.v[i];
                if (pair) part[g * row + first + ul * W + i] = sum1.v[i];
            }
        }
        __syncthreads();
        float *sums = a.sums + ((int64_t)page * a.heads + h) * a.dim;
        for (int x = tid; x < row; x += 256) {
            const bool second = x >= first;
            const int v = u0 + (x - (second ? first : 0)) / W;
            if (v >= a.all_units || (second && v * W >= a.rot / 2)) continue;  // (a copied vector has no second)
            float t = 0.0f;
            for (int k = 0; k < groups; ++k) t += part[k * row + x];
            int e0, e1;
            place(v, e0, e1);
            sums[(second ? e1 : e0) + x % W] = t;
        }
        __syncthreads();
    }
}

// Whether heads of dim components split into vectors of w: whole vectors of pairs, whole ones behind them.
bool splits_into(int dim, int rot, int w) { return (rot / 2) % w == 0 && (dim - rot) % w == 0; }

template <typename T, int W>
int launch_rope(const RopeArgs &a, bool inter, int blocks, size_t lds, hipStream_t stream) {
    if (inter)
        rope_kernel<T, W, true><<<blocks, 256, lds, stream>>>(a);
    else
        rope_kernel<T, W, false><<<blocks, 256, lds, stream>>>(a);
    return launched();
}

template <typename T>
int rope_of(RopeArgs &a, bool inter, hipStream_t stream) {
    // The widest vectors that pairs and copies split into and that rows are aligned for.
    int w = kPer16<T>;
    while (w > 1 && !(splits_into(a.dim, a.rot, w) && rows_aligned(a.x, a.x_token, a.x_head, sizeof(T), w) &&
                      rows_aligned(a.out, a.o_token, a.o_head, sizeof(T), w)))
        w /= 2;
    const int units = (a.dim - a.rot / 2) / w;
    a.units = make_div((uint32_t)units);
    a.row = make_div((uint32_t)units * (uint32_t)a.heads);
    // Tokens a workgroup takes at a time: about 1024 vector pairs, sines within 32 KiB, and
    // workgroups for every CU as long as there are tokens for it.
    int64_t group = std::max<int64_t>(1, 1024 / ((int64_t)units * a.heads));
    group = std::min<int64_t>(group, std::max<int64_t>(1, a.tokens / 1024));
    group = std::min<int64_t>(group, 4096 / std::max(a.rot / 2, 1));
    a.group = (int)group;
    const int64_t groups = (a.tokens + group - 1) / group;
    const int blocks = (int)std::min<int64_t>(groups, 1 << 20);
    const size_t lds = (size_t)group * (a.rot / 2) * sizeof(CosSin);
    if (w == 8) {
        if constexpr (kPer16<T> == 8) return launch_rope<T, 8>(a, inter, blocks, lds, stream);
    }
    if (w == 4) return launch_rope<T, 4>(a, inter, blocks, lds, stream);
    if (w == 2) return launch_rope<T, 2>(a, inter, blocks, lds, stream);
    return launch_rope<T, 1>(a, inter, blocks, lds, stream);
}

template <typename T, int W>
int launch_append(AppendArgs &a, bool inter, hipStream_t stream) {
    a.all_units = (a.dim - a.rot / 2) / W;
    a.all_vecs = a.dim / W;
    // Heads a workgroup takes: as many as leave four workgroups for every CU.
    a.each = (int)std::min<int64_t>(std::max<int64_t>(a.items * a.heads / 1024, 1), a.heads);
    a.head_groups = make_div((uint32_t)((a.heads + a.each - 1) / a.each));
    // Parts of the components: as many as leave two workgroups for every CU, and pieces of 64 bytes of a key.
    const int64_t items = a.items * a.head_groups.d;
    const int least = std::max(64 / (W * (int)sizeof(T)), 1);
    const int64_t parts = std::max<int64_t>(std::min<int64_t>(512 / items, a.all_units / least), 1);
    a.units = make_div((uint32_t)((a.all_units + parts - 1) / parts));
    a.parts = make_div((uint32_t)((a.all_units + a.units.d - 1) / a.units.d));
    a.vecs = make_div((uint32_t)((a.all_vecs + a.parts.d - 1) / a.parts.d));
    const int pairs = std::min((int)a.units.d * W, a.rot / 2);
    a.half = make_div((uint32_t)std::max(pairs, 1));
    a.rows = std::min(kTable / std::max(pairs, 1), a.B.q_start ? a.B.block : 1);
    a.table_len = a.rows * pairs;
    const size_t lds = a.table_len * sizeof(CosSin) + (a.sums ? 256 / a.units.d * a.units.d * 2 * W * sizeof(float) : 0);
    const dim3 grid = grid_of(items * a.parts.d);
    if (inter)
        append_kernel<T, W, true><<<grid, 256, lds, stream>>>(a);
    else
        append_kernel<T, W, false><<<grid, 256, lds, stream>>>(a);
    return launched();
}

template <typename T>
int append_of(AppendArgs &a, bool inter, hipStream_t stream) {
    constexpr int V = kPer16<T>;
    const bool vec = splits_into(a.dim, a.rot, V) && rows_aligned16(a.k, a.k_token, a.k_head, sizeof(T)) &&
                     rows_aligned16(a.v, a.v_token, a.v_head, sizeof(T));
    return vec ? launch_append<T, V>(a, inter, stream) : launch_append<T, 1>(a, inter, stream);
}

}  // namespace

extern "C" int spconv_batch_rows(const spconv_batch *batch, int64_t *rows) {
    if (!batch_ok(batch) || rows == nullptr) return SPCONV_EINVAL;
    *rows = rows_of(batch);
    return SPCONV_OK;
}

extern "C" int spconv_rope_frequencies(int rot, double base, const spconv_rope_scaling *scaling, double *freq) {
    if (freq == nullptr || rot < 2 || rot % 2 != 0 || !std::isfinite(base) || base <= 0.0) return SPCONV_EINVAL;
    const int kind = scaling ? scaling->kind : SPCONV_ROPE_PLAIN;
    if (kind < SPCONV_ROPE_PLAIN || kind > SPCONV_ROPE_BY_PARTS) return SPCONV_EINVAL;
    if (kind != SPCONV_ROPE_PLAIN && !(std::isfinite(scaling->factor) && scaling->factor >= 1.0)) return SPCONV_EINVAL;
    if (kind == SPCONV_ROPE_BASE) {
        if (rot == 2) return SPCONV_EINVAL;
        base *= std::pow(scaling->factor, (double)rot / (rot - 2));
        if (!std::isfinite(base)) return SPCONV_EINVAL;
    }
    if (kind == SPCONV_ROPE_BY_PARTS &&
        !(scaling->low > 0.0 && scaling->high > scaling->low && std::isfinite(scaling->high) &&
          scaling->original > 0.0 && std::isfinite(scaling->original)))
        return SPCONV_EINVAL;
    for (int i = 0; i < rot / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot);
        if (kind == SPCONV_ROPE_LINEAR) f /= scaling->factor;
        if (kind == SPCONV_ROPE_BY_PARTS) {
            const double turns = scaling->original * f / 6.283185307179586477;  // original / wavelength
            double t = (turns - scaling->low) / (scaling->high - scaling->low);
            t = t < 0.0 ? 0.0 : t > 1.0 ? 1.0 : t;
            f = (1.0 - t) * f / scaling->factor + t * f;
        }
        freq[i] = f;
    }
    return SPCONV_OK;
}

extern "C" int spconv_rope(int dtype, const void *x, int64_t x_token, int64_t x_head, int64_t tokens, int heads, int dim,
                           const int32_t *positions, const double *freq, int rot, uint32_t flags, float amplitude,
                           void *out, int64_t out_token, int64_t out_head, hipStream_t stream) {
    if (!dtype_ok(dtype) || x == nullptr || out == nullptr || positions == nullptr || (freq == nullptr && rot != 0))
        return SPCONV_EINVAL;
    if (tokens < 1 || tokens > 0x7fffffff || heads < 1 || heads > 65535 || dim < 1 || dim > 1024 || rot < 0 ||
        rot > dim || rot % 2 != 0 || (flags & ~(SPCONV_ROPE_INTERLEAVED | SPCONV_ROPE_INVERSE)) != 0 ||
        !std::isfinite(amplitude) || x_token < 0 || x_head < 0 || !out_strides_ok(tokens, heads, dim, out_token, out_head))
        return SPCONV_EINVAL;
    if (x == out && (x_token != out_token || x_head != out_head)) return SPCONV_EINVAL;
    RopeArgs a{x, out, x_token, x_head, out_token, out_head, positions, freq, tokens, heads, dim, rot, 1,
               make_div((uint32_t)std::max(rot / 2, 1)), {}, {}, (flags & SPCONV_ROPE_INVERSE) ? -1.0f : 1.0f, amplitude};
    if (rot == 0) a.half.d = 0;  // no angles
    const bool inter = (flags & SPCONV_ROPE_INTERLEAVED) != 0;
    if (dtype == SPCONV_F32) return rope_of<float>(a, inter, stream);
    if (dtype == SPCONV_F16) return rope_of<_Float16>(a, inter, stream);
    return rope_of<__bf16>(a, inter, stream);
}

extern "C" int spconv_cache_append(int dtype, const spconv_batch *batch, const void *k, int64_t k_token, int64_t k_head,
                                   const void *v, int64_t v_token, int64_t v_head, int heads, int dim,
                                   const int32_t *positions, const double *freq, int rot, uint32_t flags,
                                   float amplitude, void *k_cache, void *v_cache, float *sums, hipStream_t stream) {
    if (!batch_ok(batch) || !batch_arrays_ok(batch) || !dtype_ok(dtype) || k == nullptr || v == nullptr ||
        k_cache == nullptr || v_cache == nullptr)
        return SPCONV_EINVAL;
    if (!heads_ok(heads, heads, dim) || rot < 0 || rot > dim || rot % 2 != 0 || (freq == nullptr) != (rot == 0) ||
        (flags & ~SPCONV_ROPE_INTERLEAVED) != 0 || !std::isfinite(amplitude) || k_token < 0 || k_head < 0 ||
        v_token < 0 || v_head < 0 || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(sums))
        return SPCONV_EINVAL;
    // Touched pages of all sequences; one each without q_start.
    const int64_t items =
        batch->q_start ? batch->tokens / batch->block + 2 * (int64_t)batch->sequences : (int64_t)batch->sequences;
    if (items * heads > 0x7fffffff) return SPCONV_EINVAL;
    AppendArgs a{*batch, k, v, k_token, k_head, v_token, v_head, k_cache, v_cache, sums, positions, freq, items, heads,
                 dim, rot, 1, 1, 0, 0, 0, {}, {}, {}, {}, {}, amplitude};
    const bool inter = (flags & SPCONV_ROPE_INTERLEAVED) != 0;
    if (dtype == SPCONV_F32) return append_of<float>(a, inter, stream);
    if (dtype == SPCONV_F16) return append_of<_Float16>(a, inter, stream);
    return append_of<__bf16>(a, inter, stream);
}
