// K9: attention with a window and first tokens for few query rows, from a cache: the single tokens of serving.  The rows of all query
// heads that share a key head (16 at most) are one tile of mma.m16n8k16, so K and V are read once; tcgen05's tiles of 128 rows would stand
// empty.  Bound by HBM: 4 D bytes a visible key.
//
// A warp takes sixteen keys at a time straight into the registers that the products want them in, without shared memory: the
// channels of a product's contraction may come in any order that Q and K share, and the columns of the second one are channels
// in any order, so both fragments are made of 16-byte loads: K by key (four lanes 64 bytes of one), V by key (eight lanes 128 bytes),
// pairs of keys put together with byte permutes.  The next sixteen keys' loads go out as soon as the registers are free, so that nearly all of
// a warp's 8 KB (D = 128) are always on their way.
//
// The keys of a (sequence, key head) are split over the warps of a cluster of thread blocks.  Their partial results (sums not divided, row
// sums and maxima) meet in shared memory, the thread blocks' in distributed shared memory, each doing a share of the channels: one
// launch, no workspace, and an order that is always the same.
#include <float.h>

#include <algorithm>
#include <atomic>

#include "window.cuh"

using namespace window;

namespace {

constexpr int WARPS = 4, CHUNK = 16, MAX_ROWS = 16, MAX_CLUSTER = 16;

struct RowsParams {
    Rule w;
    Rows q, k, v, out;
    float* lse;
    int H, H_kv, group;          // query heads of a key head
    float scale_log2;
};

template <int TYPE>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (TYPE == RAPID3_BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// (past the L1: what is read may have been written by the kernel right in front)
__device__ __forceinline__ uint4 load16(const char* p) { return __ldcg(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ float peer_float(uint32_t addr, uint32_t rank) {
    float v;
    asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}" : "=f"(v) : "r"(addr), "r"(rank) : "memory");
    return v;
}

template <int TYPE, int D>
__global__ void __launch_bounds__(32 * WARPS) window_rows_kernel(const __grid_constant__ RowsParams p) {
    constexpr int KV = D / 32;                           // 16-byte loads of a lane for eight keys of K, or for two keys of V by halves: D / 64 blocks
    constexpr int DB = D / 64;
    __shared__ float o_sh[WARPS][MAX_ROWS][D + 4];
    __shared__ float m_sh[WARPS][MAX_ROWS], l_sh[WARPS][MAX_ROWS];
    __shared__ float weight[WARPS][MAX_ROWS];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane >> 2, c = lane & 3;
    const int rank = (int)cluster_rank(), size = (int)cluster_size();
    const int pair = blockIdx.x / size, b = pair / p.H_kv, hk = pair - b * p.H_kv;
    const int n_rows = p.group * p.w.n_q;
    grid_dependency_wait();
    const int rows = p.w.rows(b), keys = p.w.keys(b);

    // rows g and g + 8 of the tile: row r is query r % n_q of head r / n_q of the group
    int lo[2], hi[2];
    uint32_t qf[D / 16][4];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int r = g + 8 * x, head = r / p.w.n_q, i = r - head * p.w.n_q;
        const bool there = r < n_rows && i < rows;
        lo[x] = hi[x] = 0;
        if (there) p.w.seen(i + keys - rows, keys, lo[x], hi[x]);
        const char* src = p.q.row(b, hk * p.group + (there ? head : 0), there ? i : 0) + 16 * c;
#pragma unroll
        for (int s = 0; s < KV; ++s) {
            const uint4 v = there ? load16(src + 64 * s) : make_uint4(0, 0, 0, 0);
            qf[2 * s][x] = v.x; qf[2 * s][2 + x] = v.y;
            qf[2 * s + 1][x] = v.z; qf[2 * s + 1][2 + x] = v.w;
        }
    }
    // the keys that any row sees: first ones, then a window
    const bool any0 = hi[0] > 0, any1 = hi[1] > 0;
    int from = min(any0 ? lo[0] : keys, any1 ? lo[1] : keys), to = max(hi[0], hi[1]);
    from = __reduce_min_sync(0xffffffffu, from);
    to = __reduce_max_sync(0xffffffffu, to);
    from = min(from, to);
    const int first_end = min(min(p.w.n_sink, from), to);
    const int first_chunks = (first_end + CHUNK - 1) / CHUNK, chunks = first_chunks + (to - from + CHUNK - 1) / CHUNK;

    const char* kp = p.k.row(b, hk, 0) + 16 * c;
    const char* vp = p.v.row(b, hk, 0) + 16 * g;
    const long long kn = 2 * p.k.n, vn = 2 * p.v.n;
    uint4 kr[2][KV], vr[4][DB];
    auto span = [&](int chunk, int& base, int& end) {
        const bool f = chunk < first_chunks;
        base = f ? chunk * CHUNK : from + (chunk - first_chunks) * CHUNK;
        end = f ? first_end : to;
    };
    auto load_k = [&](int chunk) {
        int base, end;
        span(chunk, base, end);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = base + 8 * t + g;
#pragma unroll
            for (int s = 0; s < KV; ++s) kr[t][s] = key < end ? load16(kp + key * kn + 64 * s) : make_uint4(0, 0, 0, 0);
        }
    };
    auto load_v = [&](int chunk) {
        int base, end;
        span(chunk, base, end);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int key = base + 2 * c + (t & 1) + 8 * (t >> 1);
#pragma unroll
            for (int s = 0; s < DB; ++s) vr[t][s] = key < end ? load16(vp + key * vn + 128 * s) : make_uint4(0, 0, 0, 0);
        }
    };
    float o[DB * 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < DB * 8; ++t) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.f;
    // a thread block's chunks lie side by side, its warps take them by turns
    const int last = (int)((long long)chunks * (rank + 1) / size);
    int chunk = (int)((long long)chunks * rank / size) + warp;
    if (chunk < last) {
        load_k(chunk);
        load_v(chunk);
    }
    for (; chunk < last; chunk += WARPS) {
        float s[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
#pragma unroll
            for (int x = 0; x < KV; ++x) {
                mma16816<TYPE>(s[t], qf[2 * x], kr[t][x].x, kr[t][x].y);
                mma16816<TYPE>(s[t], qf[2 * x + 1], kr[t][x].z, kr[t][x].w);
            }
        }
        const bool more = chunk + WARPS < last;
        if (more) load_k(chunk + WARPS);
        int base, end;
        span(chunk, base, end);
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = base + 8 * t + 2 * c + (e & 1), x = e >> 1;
                const bool seen = j < min(hi[x], end) && (j >= lo[x] || j < p.w.n_sink);
                s[t][e] = seen ? s[t][e] * p.scale_log2 : -INFINITY;
                top[x] = fmaxf(top[x], s[t][e]);
            }
        float shift[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 1));
            top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 2));
            const float next = fmaxf(m[x], top[x]);
            shift[x] = next == -INFINITY ? 0.f : next;
            const float f = ptx::ex2(m[x] - shift[x]);   // 0 where nothing was seen so far
            l[x] *= f;
            m[x] = next;
            if (__any_sync(0xffffffffu, f != 1.f))
#pragma unroll
                for (int t = 0; t < DB * 8; ++t) {
                    o[t][2 * x] *= f;
                    o[t][2 * x + 1] *= f;
                }
        }
        uint32_t pf[4];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t][e] = ptx::ex2(s[t][e] - shift[e >> 1]);
            l[0] += s[t][0] + s[t][1];
            l[1] += s[t][2] + s[t][3];
            pf[2 * t] = pack16<TYPE>(s[t][0], s[t][1]);
            pf[2 * t + 1] = pack16<TYPE>(s[t][2], s[t][3]);
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const uint32_t w[4][4] = {{vr[0][db].x, vr[0][db].y, vr[0][db].z, vr[0][db].w}, {vr[1][db].x, vr[1][db].y, vr[1][db].z, vr[1][db].w},
                                      {vr[2][db].x, vr[2][db].y, vr[2][db].z, vr[2][db].w}, {vr[3][db].x, vr[3][db].y, vr[3][db].z, vr[3][db].w}};
#pragma unroll
            for (int t = 0; t < 8; ++t) {                // column g of product t is channel 64 db + 8 g + t
                const uint32_t pick = t & 1 ? 0x7632u : 0x5410u;
                mma16816<TYPE>(o[8 * db + t], pf, __byte_perm(w[0][t >> 1], w[1][t >> 1], pick), __byte_perm(w[2][t >> 1], w[3][t >> 1], pick));
            }
        }
        if (more) load_v(chunk + WARPS);
    }
    // ---- the warps' results, then the thread blocks'
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
        if (c == 0) {
            m_sh[warp][g + 8 * x] = m[x];
            l_sh[warp][g + 8 * x] = l[x];
        }
#pragma unroll
        for (int t = 0; t < DB * 8; ++t) {
            float* to = &o_sh[warp][g + 8 * x][64 * (t >> 3) + (t & 7)];
            to[8 * (2 * c)] = o[t][2 * x];
            to[8 * (2 * c + 1)] = o[t][2 * x + 1];
        }
    }
    __syncthreads();
    if (threadIdx.x < MAX_ROWS) {
        const int r = threadIdx.x;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int x = 0; x < WARPS; ++x) top = fmaxf(top, m_sh[x][r]);
#pragma unroll
        for (int x = 0; x < WARPS; ++x) {
            const float f = m_sh[x][r] == -INFINITY ? 0.f : ptx::ex2(m_sh[x][r] - top);
            weight[x][r] = f;
            sum = fmaf(f, l_sh[x][r], sum);
        }
        m_sh[0][r] = top;
        l_sh[0][r] = sum;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < MAX_ROWS * D; x += 32 * WARPS) {
        const int r = x / D, d = x % D;
        float sum = 0.f;
#pragma unroll
        for (int y = 0; y < WARPS; ++y) sum = fmaf(weight[y][r], o_sh[y][r][d], sum);
        o_sh[0][r][d] = sum;
    }
    grid_dependency_launch();
    cluster_sync();
    // this thread block's share of the tile, two channels a thread
    const uint32_t o_at = ptx::smem_u32(&o_sh[0][0][0]), m_at = ptx::smem_u32(&m_sh[0][0]), l_at = ptx::smem_u32(&l_sh[0][0]);
    for (int x = rank * 32 * WARPS + threadIdx.x; x < n_rows * (D / 2); x += size * 32 * WARPS) {
        const int r = x / (D / 2), d = 2 * (x % (D / 2)), head = r / p.w.n_q, i = r - head * p.w.n_q;
        float top = -INFINITY, sum = 0.f, a = 0.f, bb = 0.f;
        for (int y = 0; y < size; ++y) top = fmaxf(top, peer_float(m_at + 4 * r, y));
        for (int y = 0; y < size; ++y) {
            const float my = peer_float(m_at + 4 * r, y), f = my == -INFINITY ? 0.f : ptx::ex2(my - top);
            sum = fmaf(f, peer_float(l_at + 4 * r, y), sum);
            a = fmaf(f, peer_float(o_at + 4 * (r * (D + 4) + d), y), a);
            bb = fmaf(f, peer_float(o_at + 4 * (r * (D + 4) + d + 1), y), bb);
        }
        if (i >= rows) continue;                         // a place behind the sequence's rows
        const float inv = sum > 0.f ? 1.f / sum : 0.f;   // a row that sees nothing: zeros
        *reinterpret_cast<uint32_t*>(p.out.row(b, hk * p.group + head, i) + 2 * d) = pack16<TYPE>(a * inv, bb * inv);
        if (p.lse && d == 0)
            p.lse[((long long)b * p.H + hk * p.group + head) * p.w.n_q + i] = sum > 0.f ? (top + log2f(sum)) * 0.69314718055994531f : -INFINITY;
    }
    cluster_sync();                                      // no thread block leaves while others read its shared memory
}

}  // namespace

bool window_rows_fit(const rapid3_window* w) { return (long long)(w->H / w->H_kv) * w->n_q <= MAX_ROWS; }

cudaError_t launch_window_rows(const rapid3_window* w, const rapid3_rows* q, const rapid3_rows* k, const rapid3_rows* v, const rapid3_rows* out,
                               float* lse, cudaStream_t s) {
    RowsParams p;
    p.w = rule_of(w);
    p.q = rows_arg(q);
    p.k = rows_arg(k);
    p.v = rows_arg(v);
    p.out = rows_arg(out);
    p.lse = lse;
    p.H = w->H;
    p.H_kv = w->H_kv;
    p.group = w->H / w->H_kv;
    p.scale_log2 = w->softmax_scale * 1.4426950408889634f;
    const bool bf = w->type == RAPID3_BF16;
    const auto kernel = w->D == 128 ? (bf ? window_rows_kernel<RAPID3_BF16, 128> : window_rows_kernel<RAPID3_F16, 128>)
                                    : (bf ? window_rows_kernel<RAPID3_BF16, 64> : window_rows_kernel<RAPID3_F16, 64>);
    // Keys that a sequence's rows may see; as many thread blocks for them as give every warp 64, while SMs are free.
    long long keys = w->n_kv;
    if (w->left >= 0 && w->n_full == 0) keys = std::min<long long>(keys, (long long)w->left + 1 + std::max(w->right, 0) + w->n_q + w->n_sink);
    const long long pairs = (long long)w->B * w->H_kv;
    int size = 1;
    while (size < MAX_CLUSTER && pairs * size * 2 <= 4 * SM_COUNT && keys >= 64ll * WARPS * size * 2) size *= 2;
    if (size > 8) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    return launch_kernel_cluster(kernel, dim3((unsigned)(pairs * size)), dim3(32 * WARPS), 0, s, size, p);
}
