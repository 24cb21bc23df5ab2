// What the kernels of attention with a window and first tokens share: the rule, the element types, argument checks.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "ptx.cuh"

namespace window {

// Lengths and bounds stay below this, so that sums of two stay in 32 bits.
constexpr int MOST = (1 << 30) - 2;

// Bits 0 .. n - 1 of 32 (n of any size or sign).
__device__ __forceinline__ uint32_t bits_below(int n) {
    uint32_t d;
    asm("bmsk.clamp.b32 %0, %1, %2;" : "=r"(d) : "r"(0), "r"(max(n, 0)));
    return d;
}

struct Rule {
    int n_q, n_kv;               // places of a sequence
    int left, right;             // -1: no bound
    int n_sink, n_full;
    const int32_t* q_len;
    const int32_t* kv_len;
    __device__ __forceinline__ int rows(int b) const { return q_len ? min(max(__ldcg(q_len + b), 0), n_q) : n_q; }
    __device__ __forceinline__ int keys(int b) const { return kv_len ? min(max(__ldcg(kv_len + b), 0), n_kv) : n_kv; }
    // The row at position p sees the keys j < hi with j >= lo or j < n_sink.  near: as if no row were full.
    __host__ __device__ __forceinline__ void near(int p, int keys, int& lo, int& hi) const {
        lo = left < 0 ? 0 : max(p - left, 0);
        hi = right < 0 ? keys : min(keys, max(p + right + 1, 0));
    }
    __host__ __device__ __forceinline__ void seen(int p, int keys, int& lo, int& hi) const {
        near(p, keys, lo, hi);
        if ((unsigned)p < (unsigned)n_full) {
            lo = 0;
            hi = keys;
        }
    }
    __host__ __device__ __forceinline__ int count(int p, int keys) const {
        int lo, hi;
        seen(p, keys, lo, hi);
        return max(hi - lo, 0) + max(min(n_sink, min(lo, hi)), 0);
    }
    // The same of the 64 keys from key0 on, as bits.
    __device__ __forceinline__ void seen_bits(int p, int keys, int key0, uint32_t (&bits)[2]) const {
        int lo, hi;
        seen(p, keys, lo, hi);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = key0 + 32 * h;
            bits[h] = bits_below(hi - k) & (~bits_below(lo - k) | bits_below(n_sink - k));
        }
    }
};

// Blocks of 64 that a tile works on: 0 .. first - 1, then from .. to - 1 (from >= first).
struct Blocks {
    int first, from, to;
    __device__ __forceinline__ int count() const { return first + to - from; }
    __device__ __forceinline__ int at(int i) const { return i < first ? i : from + i - first; }
    __device__ __forceinline__ Blocks join(const Blocks& o) const {
        Blocks r;
        r.from = count() == 0 ? o.from : o.count() == 0 ? from : min(from, o.from);
        r.to = max(to, o.to);
        r.first = min(max(first, o.first), r.from);
        return r;
    }
};
__device__ __forceinline__ Blocks blocks_of(int first_end, int lo, int hi) {
    Blocks r;
    r.to = max(0, (hi + 63) >> 6);
    r.from = min(max(0, lo >> 6), r.to);
    r.first = min((first_end + 63) >> 6, r.from);
    return r;
}
// The key blocks of query rows [row0, row1) (row1 <= rows) of a sequence: a row's bounds rise with its position, but for full rows.
__device__ __forceinline__ Blocks key_blocks(const Rule& w, int row0, int row1, int rows, int keys) {
    if (row0 >= row1) return {0, 0, 0};
    const int p0 = row0 + keys - rows, p1 = row1 - 1 + keys - rows;
    if (p0 < w.n_full && p1 >= 0) return blocks_of(0, 0, keys);
    int lo, hi, lo1, hi1;
    w.seen(p0, keys, lo, hi1);
    w.seen(p1, keys, lo1, hi);
    return blocks_of(min(w.n_sink, hi), lo, hi);
}

// ------------------------------------------------------------------ 16-bit types
template <int TYPE>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    if constexpr (TYPE == RAPID3_BF16) return ptx::pack_bf16(lo, hi);
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
template <int TYPE>
__device__ __forceinline__ float2 unpack16(uint32_t v) {
    if constexpr (TYPE == RAPID3_BF16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
// Instruction descriptor of kind::f16 for two operands of the type (format 1 = bf16, 0 = f16).
template <int TYPE>
__host__ __device__ constexpr uint32_t idesc16(int M, int N, int a_mn_major, int b_mn_major) {
    return ptx::idesc_bf16(M, N, a_mn_major, b_mn_major) & (TYPE == RAPID3_BF16 ? ~0u : ~((7u << 7) | (7u << 10)));
}
// Lane c of a quad of lanes holds words 0..3 of the column pairs c, c + 4, c + 8, c + 12 (16x256b fragments); afterwards words 4 c .. 4 c + 3.
__device__ __forceinline__ uint4 quad_transpose(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, int c) {
    const bool b0 = c & 1, b1 = c & 2;
    const uint32_t x = __shfl_xor_sync(0xffffffffu, b0 ? w0 : w1, 1), y = __shfl_xor_sync(0xffffffffu, b0 ? w2 : w3, 1);
    const uint32_t p0 = b0 ? x : w0, p1 = b0 ? w1 : x, q0 = b0 ? y : w2, q1 = b0 ? w3 : y;
    const uint32_t r0 = __shfl_xor_sync(0xffffffffu, b1 ? p0 : q0, 2), r1 = __shfl_xor_sync(0xffffffffu, b1 ? p1 : q1, 2);
    return b1 ? make_uint4(r0, r1, q0, q1) : make_uint4(p0, p1, r0, r1);
}

// A tensor as the kernels address it, strides in elements.
struct Rows {
    char* data;
    long long b, h, n;
    __device__ __forceinline__ char* row(int ib, int ih, int in) const { return data + 2 * (ib * b + ih * h + in * n); }
};
inline Rows rows_arg(const rapid3_rows* t) { return {static_cast<char*>(t->data), t->stride_b, t->stride_h, t->stride_n}; }

// Host side (k8_window.cu): the arguments of a call; a tensor map of boxes of 64 channels x 64 rows, 128-byte swizzle.
int check(const rapid3_window* w);
int check_rows(const rapid3_window* w, const rapid3_rows* t, int heads, int n);
Rule rule_of(const rapid3_window* w);
int tensor_map(const rapid3_window* w, const rapid3_rows* t, int heads, int n, CUtensorMap* map);

}  // namespace window

// K9: few query rows for each key head (H / H_kv * n_q <= 16), from caches of any length.
bool window_rows_fit(const rapid3_window* w);
cudaError_t launch_window_rows(const rapid3_window* w, const rapid3_rows* q, const rapid3_rows* k, const rapid3_rows* v, const rapid3_rows* out,
                               float* lse, cudaStream_t s);
