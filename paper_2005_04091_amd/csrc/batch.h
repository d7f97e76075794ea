// Shared by the calls of spconv_attention.h: element types, rows and sequences of
// a batch, host checks (internal header).
#pragma once

#include "common.h"
#include "rows.h"
#include "spconv_attention.h"

#include <cmath>

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T, int W>
struct VecOf {
    typedef T type __attribute__((ext_vector_type(W)));
};
template <typename T>
struct VecOf<T, 1> {
    typedef T type;
};

// Elements of one 16-byte load.
template <typename T>
constexpr int kPer16 = 16 / (int)sizeof(T);

template <int W>
struct Floats {
    float v[W];
};

template <typename T, int W>
__device__ __forceinline__ Floats<W> floats_of(typename VecOf<T, W>::type v) {
    Floats<W> r;
    if constexpr (W == 1) {
        r.v[0] = (float)v;
    } else {
        typedef typename VecOf<float, W>::type F;
        const F f = __builtin_convertvector(v, F);
#pragma unroll
        for (int i = 0; i < W; ++i) r.v[i] = f[i];
    }
    return r;
}

template <typename T, int W>
__device__ __forceinline__ Floats<W> load_floats(const T *p) {
    return floats_of<T, W>(*reinterpret_cast<const typename VecOf<T, W>::type *>(p));
}

// Rounds (to nearest even) and stores W elements; what was stored comes back.
template <typename T, int W>
__device__ __forceinline__ Floats<W> store_floats(T *p, Floats<W> x) {
    if constexpr (W == 1) {
        const T t = (T)x.v[0];
        *p = t;
        x.v[0] = (float)t;
    } else {
        typedef typename VecOf<T, W>::type V;
        typedef typename VecOf<float, W>::type F;
        F f;
#pragma unroll
        for (int i = 0; i < W; ++i) f[i] = x.v[i];
        const V t = __builtin_convertvector(f, V);
        *reinterpret_cast<V *>(p) = t;
        f = __builtin_convertvector(t, F);
#pragma unroll
        for (int i = 0; i < W; ++i) x.v[i] = f[i];
    }
    return x;
}

// x / d with the magic of div_magic (x < 2^31).
struct Div {
    uint32_t d, magic;
    int shift;
};

inline Div make_div(uint32_t d) {
    Div v{d, 0, 0};
    div_magic(d, &v.magic, &v.shift);
    return v;
}

__device__ __forceinline__ uint32_t operator/(uint32_t x, const Div &d) { return fast_div(x, d.magic, d.shift); }

// Grids are laid out in two dimensions: the threads of one have to stay under 2^32.
constexpr int64_t kGridX = 1 << 20;

inline dim3 grid_of(int64_t n) {
    return n <= kGridX ? dim3((uint32_t)n) : dim3((uint32_t)kGridX, (uint32_t)((n + kGridX - 1) / kGridX));
}

__device__ __forceinline__ int64_t grid_index() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// The last sequence b whose start, q_start[b]/div + mul*b, is at most x (the same for the whole wave, as is
// the result), found by the whole wave, 64 starts a step, each step between two of the last one's, and its
// tokens. The starts do not decrease; where they do (the array is the caller's) some sequence or none comes
// out, with its tokens taken into the batch.
struct Seq {
    int b;          // -1: none
    int first, n;   // tokens [first, first + n)
    int at;         // x - start of b (negative: x is no item of b)
    int kv;         // keys
};

__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return min(max(x, lo), hi); }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ Seq find_seq(const spconv_batch &B, int x, int div, int mul) {
    Seq s;
    const int tokens = (int)B.tokens;
    x = uniform(x);
    if (B.q_start == nullptr) {  // (x is a sequence: one item each)
        s.b = x;
        s.first = x;
        s.n = 1;
        s.at = 0;
    } else {
        const int lane = threadIdx.x & (kWave - 1);
        s.b = 0;
        for (int left = B.sequences, step; left > 0; left = step > 1 ? min(step, left) : 0) {  // among [s.b, s.b + left)
            step = (left + kWave - 1) / kWave;
            const int64_t i = (int64_t)lane * step;
            bool in = false;
            if (i < left) {
                const int b = s.b + (int)i;
                in = (int64_t)(clamp_int(B.q_start[b], 0, tokens) / div) + (int64_t)mul * b <= (int64_t)x;
            }
            const int last = (int)__popcll(__ballot(in)) - 1;
            if (last < 0) {  // (before the first start; behind the first step the first of them is one)
                s.b = -1;
                s.first = s.n = s.at = s.kv = 0;
                return s;
            }
            s.b += last * step;
            left -= last * step;
        }
        s.first = clamp_int(uniform(B.q_start[s.b]), 0, tokens);
        s.n = max(clamp_int(uniform(B.q_start[s.b + 1]), 0, tokens) - s.first, 0);
        s.at = (int)((int64_t)x - (s.first / div) - (int64_t)mul * s.b);
    }
    s.kv = clamp_int(uniform(B.kv_len[s.b]), 0, B.max_blocks * B.block);
    return s;
}

// A row: its sequence, its tokens [t0, t0 + n) and the first one's position.
struct Row {
    int b, t0, n, p0, kv;
};

__device__ __forceinline__ Row find_row(const spconv_batch &B, int row) {
    if (B.q_start == nullptr) {
        const int b = sequence_of_row(uniform(row), B.q_block, B.sequences);
        if (b < 0) return {-1, 0, 0, 0, 0};
        const Seq s = find_seq(B, b, 1, 0);
        return {b, b, 1, s.kv - 1, s.kv};
    }
    const Seq s = B.q_block == 1 ? find_seq(B, row, 1, 0) : find_seq(B, row, B.q_block, 1);
    Row r{s.b, 0, 0, 0, s.kv};
    if (s.b < 0 || s.at < 0) return r;
    const int64_t i0 = (int64_t)s.at * B.q_block;
    if (i0 >= s.n) return r;
    r.t0 = s.first + (int)i0;
    r.n = min(s.n - (int)i0, B.q_block);
    r.p0 = s.kv - s.n + (int)i0;
    return r;
}

// Page of block j of sequence b, -1 if there is none.
__device__ __forceinline__ int page_of(const spconv_batch &B, int b, int j) {
    const int page = B.table[(int64_t)b * B.table_stride + j];
    return (uint32_t)page < (uint64_t)B.pages ? page : -1;
}

// ---- host ----

inline bool batch_ok(const spconv_batch *B) {
    if (B == nullptr) return false;
    if (B->sequences < 1 || B->block < 16 || B->block > 256 || B->block % 16 != 0 || B->max_blocks < 1 ||
        (int64_t)B->max_blocks * B->block >= ((int64_t)1 << 31) || B->q_block < 1 || B->q_block > 128 || B->tokens < 1 ||
        B->tokens > 0x7fffffff || B->pages < 1 || B->pages > 0x7fffffff || B->table_stride < B->max_blocks)
        return false;
    return B->q_start != nullptr || B->tokens == B->sequences;
}

inline bool batch_arrays_ok(const spconv_batch *B) { return B->table != nullptr && B->kv_len != nullptr; }

inline int64_t rows_of(const spconv_batch *B) {
    return B->q_block == 1 ? B->tokens : B->tokens / B->q_block + B->sequences;
}

// Tokens that a row has at most.
inline int row_tokens(const spconv_batch *B) { return B->q_start ? B->q_block : 1; }

inline bool dtype_ok(int dtype) { return dtype == SPCONV_F32 || dtype == SPCONV_F16 || dtype == SPCONV_BF16; }

inline int size_of(int dtype) { return dtype == SPCONV_F32 ? 4 : 2; }

inline bool heads_ok(int q_heads, int heads, int dim) {
    return heads >= 1 && q_heads >= heads && q_heads <= 65535 && q_heads % heads == 0 && dim >= 8 && dim <= 256 &&
           dim % 8 == 0;
}

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// Whether rows of these strides (elements of `size` bytes) can be read by vectors of w elements, a power of two.
inline bool rows_aligned(const void *p, int64_t a, int64_t b, int size, int w) {
    return ((uintptr_t)p & (uintptr_t)(size * w - 1)) == 0 && a % w == 0 && b % w == 0;
}
inline bool rows_aligned16(const void *p, int64_t a, int64_t b, int size) { return rows_aligned(p, a, b, size, 16 / size); }

// Strides of a tensor that is written: no two rows of dim elements overlap along one axis.
inline bool out_strides_ok(int64_t tokens, int heads, int dim, int64_t token, int64_t head) {
    return token >= 0 && head >= 0 && (tokens == 1 || token >= dim) && (heads == 1 || head >= dim);
}

inline int launched() { return hipGetLastError() == hipSuccess ? SPCONV_OK : SPCONV_EHIP; }

}  // namespace
