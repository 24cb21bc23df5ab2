// K7: rotary positions of Q and K heads, alone or behind the RMS normalisation of each head, and the gradients of both.
// Per row x[D] of one (sequence, head, token):
//     y = x / sqrt(mean(x^2) + eps) * gain            (NORM; else y = x)
//     z = amplitude * R(position . freq) y            on the turned channel pairs, z = y on the others
// and, from dz (BACK), with g = amplitude * R^T dz, u = x r, r = 1 / sqrt(mean(x^2) + eps):
//     dx = r (g gain - u mean(g gain u)),  dgain = sum over all rows of g u          (NORM; else dx = g)
// All of it in fp32, one rounding to the tensors' type.  The angles of far positions need more: position * freq / 2 pi is taken in
// fp64, its fraction alone goes on to sincospif.
//
// Bound by HBM: a row is read once (BACK with NORM: two rows) and written once, so that what counts besides is how few instructions a
// row takes.  A group of lanes holds a row, a lane four channel pairs, so the rotation is the lane's own in both layouts and the lanes of a row
// add up its squares by shuffles.  A group stays with one token and goes through its heads: cosines and sines, times the gains where
// both are factors, are computed once and stay in registers, and the arithmetic goes in packed pairs.  The rows come by asynchronous copies
// through a ring of the warp's own in shared memory, DEPTH of them on their way (in registers, with as many warps as these allow, no more than
// 32 to 64 KB an SM were, and the kernel waited for memory half of the time).
//
// Measured at D = 128, bf16: Q and K of three sequences of 4608 tokens and 24 heads, normed and turned, 339.7 MB in 70 us, 4.9 TB/s, 0.74 of a
// copy's rate; gradients of 32 + 8 heads of 8191 tokens, gains' included, 251.6 MB in 56 us, 4.5 TB/s.  At D = 64, fp16: gradients of 24 + 24 heads
// of two sequences of 4429 tokens, 163 MB in 40 us.  Instructions are issued in 39 to 46 of 100 cycles, also in the gradients, which take a row at a time a
// lane group with 16 warps an SM: of the 6.4 cycles between two instructions of a warp 1.5 are the arithmetic's own latency, 1.1 the rows on their way, 0.5 shuffles
// and shared memory; and 512 thread blocks are 1.73 rounds of the 296 that are resident.  Sixteen channels a lane instead of eight take
// half of the shuffles and 115 to 155 registers: 71 us, and 53 for the 41 of the gradients.  Single tokens: 9 to 10 us a call, the launch.
#include <math.h>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "common.cuh"
#include "ptx.cuh"

namespace {

using ptx::fma2;
using ptx::mul2;
using ptx::of_pair;
using ptx::pair_of;

constexpr int WARPS = 8, MAX_D = 256, MAX_AXES = 4;
constexpr int GRAD_BLOCKS_PER_SM = 4;                   // thread blocks of a backward launch: each leaves one partial sum of the gains' gradients
constexpr int MAX_GRAD_BLOCKS = GRAD_BLOCKS_PER_SM * SM_COUNT;

struct RowsArg {
    const char* in;              // x
    const char* grad;            // BACK with NORM: dz (else dz takes the place of x)
    char* out;
    const float* gain;
    long long in_b, in_h, in_n, grad_b, grad_h, grad_n, out_b, out_h, out_n;   // bytes
    int H;
};

struct TurnArg {
    const double* freq;
    const int32_t* pos;
    long long pos_b, pos_n;
    int pos0, pairs, axes;
    int axis_end[MAX_AXES];      // pairs up to axis_end[a] turn by coordinate a (the first that holds)
    float amplitude;
};

struct Args {
    RowsArg t[2];                // Q, K
    TurnArg turn;
    float eps, inv_D;
    int N, D, log_tokens, tiles; // tokens of a thread block (a power of two), thread blocks of a sequence
    int n_tiles;                 // of all sequences
    int heads_per_block;
    float* partial;              // BACK with NORM: [thread block][2][D]
};

// A lane's eight channels of a row, as they lie in memory: two runs of four.
template <int TYPE>
struct Raw {
    uint2 lo, hi;
};
template <>
struct Raw<RAPID3_F32> {
    uint4 lo, hi;
};
template <int TYPE, bool HALVES>
__device__ __forceinline__ Raw<TYPE> read_raw(const char* p, int at0, int at1) {
    Raw<TYPE> r;
    if constexpr (TYPE == RAPID3_F32) {
        r.lo = *reinterpret_cast<const uint4*>(p + 4 * at0);
        r.hi = *reinterpret_cast<const uint4*>(p + 4 * at1);
    } else if constexpr (HALVES) {
        r.lo = *reinterpret_cast<const uint2*>(p + 2 * at0);
        r.hi = *reinterpret_cast<const uint2*>(p + 2 * at1);
    } else {
        const uint4 v = *reinterpret_cast<const uint4*>(p + 2 * at0);   // the two runs lie side by side
        r.lo = make_uint2(v.x, v.y);
        r.hi = make_uint2(v.z, v.w);
    }
    return r;
}
// 16 bytes to shared memory, past the L1; zeros where there is nothing to read.
__device__ __forceinline__ void copy16(uint32_t to, const char* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
template <int TYPE>
__device__ __forceinline__ float2 wide2(uint32_t v) {
    if constexpr (TYPE == RAPID3_BF16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
template <int TYPE>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
    if constexpr (TYPE == RAPID3_BF16) {
        const __nv_bfloat162 u = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&u);
    }
    const __half2 u = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&u);
}
// Four channel pairs, packed by twos: first members a, second members b.
struct Pairs {
    uint64_t a[2], b[2];
};
template <int TYPE, bool HALVES>
__device__ __forceinline__ Pairs widen(const Raw<TYPE>& r) {
    float2 w[4];                                         // the lane's eight channels in order
    if constexpr (TYPE == RAPID3_F32) {
        w[0] = make_float2(__uint_as_float(r.lo.x), __uint_as_float(r.lo.y));
        w[1] = make_float2(__uint_as_float(r.lo.z), __uint_as_float(r.lo.w));
        w[2] = make_float2(__uint_as_float(r.hi.x), __uint_as_float(r.hi.y));
        w[3] = make_float2(__uint_as_float(r.hi.z), __uint_as_float(r.hi.w));
    } else {
        w[0] = wide2<TYPE>(r.lo.x);
        w[1] = wide2<TYPE>(r.lo.y);
        w[2] = wide2<TYPE>(r.hi.x);
        w[3] = wide2<TYPE>(r.hi.y);
    }
    Pairs p;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        p.a[i] = HALVES ? pair_of(w[i].x, w[i].y) : pair_of(w[2 * i].x, w[2 * i + 1].x);
        p.b[i] = HALVES ? pair_of(w[2 + i].x, w[2 + i].y) : pair_of(w[2 * i].y, w[2 * i + 1].y);
    }
    return p;
}
template <int TYPE, bool HALVES>
__device__ __forceinline__ void store_pairs(char* p, int at0, int at1, const Pairs& z) {
    const float2 a0 = of_pair(z.a[0]), a1 = of_pair(z.a[1]), b0 = of_pair(z.b[0]), b1 = of_pair(z.b[1]);
    if constexpr (TYPE == RAPID3_F32) {
        *reinterpret_cast<float4*>(p + 4 * at0) = HALVES ? make_float4(a0.x, a0.y, a1.x, a1.y) : make_float4(a0.x, b0.x, a0.y, b0.y);
        *reinterpret_cast<float4*>(p + 4 * at1) = HALVES ? make_float4(b0.x, b0.y, b1.x, b1.y) : make_float4(a1.x, b1.x, a1.y, b1.y);
    } else if constexpr (HALVES) {
        *reinterpret_cast<uint2*>(p + 2 * at0) = make_uint2(narrow2<TYPE>(a0.x, a0.y), narrow2<TYPE>(a1.x, a1.y));
        *reinterpret_cast<uint2*>(p + 2 * at1) = make_uint2(narrow2<TYPE>(b0.x, b0.y), narrow2<TYPE>(b1.x, b1.y));
    } else {
        *reinterpret_cast<uint4*>(p + 2 * at0) = make_uint4(narrow2<TYPE>(a0.x, b0.x), narrow2<TYPE>(a0.y, b0.y), narrow2<TYPE>(a1.x, b1.x), narrow2<TYPE>(a1.y, b1.y));
    }
}
__device__ __forceinline__ uint64_t twice(float x) { return pair_of(x, x); }
// Sum of squares, or of products, of a lane's eight numbers.
__device__ __forceinline__ float dot8(const Pairs& x, const Pairs& y) {
    const float2 s = of_pair(fma2(x.a[0], y.a[0], fma2(x.a[1], y.a[1], fma2(x.b[0], y.b[0], mul2(x.b[1], y.b[1])))));
    return s.x + s.y;
}

// Rows of a lane group on their way at once.
__host__ __device__ constexpr int depth_of(int type, bool grads) { return type == RAPID3_F32 ? (grads ? 3 : 4) : grads ? 6 : 8; }
__host__ __device__ constexpr size_t ring_bytes(int type, bool grads) { return (size_t)WARPS * depth_of(type, grads) * (grads ? 2 : 1) * 256 * (type == RAPID3_F32 ? 4 : 2); }

// LPR lanes hold a row: lane c the channel pairs 4 c .. 4 c + 3.
template <int TYPE, int LPR, bool HALVES, bool NORM, bool BACK>
__global__ void __launch_bounds__(32 * WARPS) rotary_kernel(const __grid_constant__ Args p) {
    constexpr int RPW = 32 / LPR, SLOTS = WARPS * RPW;   // rows of a warp, of a thread block, at a time
    constexpr bool GRADS = NORM && BACK;
    constexpr int SIZE = TYPE == RAPID3_F32 ? 4 : 2, DEPTH = depth_of(TYPE, GRADS), STREAMS = GRADS ? 2 : 1, U = NORM && !BACK ? DEPTH / 2 : 1;
    constexpr int ROW = 8 * LPR * SIZE, STEP = 256 * SIZE;              // bytes of a row's place, of a warp's rows
    extern __shared__ __align__(16) char ring[];        // [warp][DEPTH][x, dz][row of the warp]
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, c = lane % LPR, slot = warp * RPW + lane / LPR;
    const int D = p.D, half = p.turn.pairs;
    const bool here = 8 * c < D;
    // the lane's channels: two runs of four
    const bool split = HALVES && 4 * c < half;
    const int at0 = split ? 4 * c : 8 * c, at1 = split ? half + 4 * c : 8 * c + 4;
    Pairs acc[GRADS ? 2 : 1];
#pragma unroll
    for (int w = 0; w < (GRADS ? 2 : 1); ++w) acc[w].a[0] = acc[w].a[1] = acc[w].b[0] = acc[w].b[1] = 0ull;
    // the slot's token of a tile, and its share of the heads
    const int mine = slot & ((1 << p.log_tokens) - 1), head0 = slot >> p.log_tokens, head_step = SLOTS >> p.log_tokens;
    char* const ring_at = ring + warp * (DEPTH * STREAMS * STEP) + (lane / LPR) * ROW;
    const uint32_t my_ring = ptx::smem_u32(ring_at);
    grid_dependency_wait();
    // gain_kernel's few thread blocks may be there and wait where an SM has room (gradients of 24 + 24 heads at D = 64: 43.0 -> 40.7 us); other
    // launches that wait beside this one only take its SMs' room (rotation alone 12.7 -> 13.6)
    if (GRADS) grid_dependency_launch();
    for (uint32_t tile = blockIdx.x; tile < (uint32_t)p.n_tiles; tile += gridDim.x) {      // (a tile and a grid may be 2^31 - 1, their sum is no int)
        const int b = (int)tile / p.tiles, n = (((int)tile - b * p.tiles) << p.log_tokens) + mine;
        const bool live = n < p.N && here;
        // this thread block's heads among those of Q and then K; a slot's steps through them
        int first_head[2], heads[2], steps[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int before = w ? p.t[0].H : 0;
            first_head[w] = max(0, (int)blockIdx.y * p.heads_per_block - before);
            heads[w] = max(0, min(p.t[w].H, ((int)blockIdx.y + 1) * p.heads_per_block - before) - first_head[w]);
            steps[w] = (heads[w] + head_step - 1) / head_step;
        }
        // the copies, Q's rows and then K's
        const char *in = nullptr, *grad = nullptr;
        long long in_step = 0, grad_step = 0;
        int issued = 0, coming = 0;                      // heads of the tensor that the slot has still to fetch: this many / head_step, rounded up
        auto source = [&](int w) {
            const RowsArg& t = p.t[w];
            const int h = (w ? first_head[1] : first_head[0]) + head0;
            coming = n < p.N ? (w ? heads[1] : heads[0]) - head0 : 0;
            in = t.in + b * t.in_b + h * t.in_h + n * t.in_n;
            in_step = t.in_h * head_step;
            if constexpr (GRADS) {
                grad = t.grad + b * t.grad_b + h * t.grad_h + n * t.grad_n;
                grad_step = t.grad_h * head_step;
            }
        };
        source(steps[0] > 0 ? 0 : 1);
        auto issue = [&]() {
            if (issued < steps[0] + steps[1]) {
                if (issued == steps[0] && issued > 0) source(1);
                const uint32_t to = my_ring + (issued % DEPTH) * (STREAMS * STEP);
#pragma unroll
                for (int k = 0; k < SIZE / 2; ++k) {     // (lanes side by side fetch pieces side by side)
                    const int piece = c + k * LPR;
                    const bool there = coming > 0 && piece * 16 < D * SIZE;
                    copy16(to + 16 * piece, there ? in + 16 * piece : reinterpret_cast<const char*>(p.t[0].in), there);
                    if constexpr (GRADS) copy16(to + STEP + 16 * piece, there ? grad + 16 * piece : reinterpret_cast<const char*>(p.t[0].in), there);
                }
                coming -= head_step;
                in += in_step;
                if constexpr (GRADS) grad += grad_step;
            }
            ++issued;
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        for (int u = 0; u < DEPTH; ++u) issue();
        int step = 0;
        Pairs cs, sn;                                    // of the first and second members alike
        {
            float cosine[4], sine[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int pair = 4 * c + i;
                cosine[i] = 1.f;
                sine[i] = 0.f;
                if (pair < half && live) {
                    int axis = 0;
                    while (axis + 1 < p.turn.axes && pair >= p.turn.axis_end[axis]) ++axis;
                    const int at = p.turn.pos ? __ldcg(p.turn.pos + b * p.turn.pos_b + n * p.turn.pos_n + axis) : p.turn.pos0 + n;
                    double turns = (double)at * (__ldcg(p.turn.freq + pair) * 0.15915494309189533577);
                    turns -= rint(turns);
                    sincospif(2.f * (float)turns, &sine[i], &cosine[i]);
                    sine[i] *= BACK ? -p.turn.amplitude : p.turn.amplitude;     // the transposed rotation turns back
                    cosine[i] *= p.turn.amplitude;
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                cs.a[i] = cs.b[i] = pair_of(cosine[2 * i], cosine[2 * i + 1]);
                sn.a[i] = pair_of(sine[2 * i], sine[2 * i + 1]);
                sn.b[i] = pair_of(-sine[2 * i], -sine[2 * i + 1]);
            }
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const RowsArg& t = p.t[w];
            if (heads[w] == 0) continue;
            Pairs gain = {};
            if (NORM && here) {
                float ga[4], gb[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ga[i] = __ldcg(t.gain + (HALVES ? at0 + i : at0 + 2 * i));
                    gb[i] = __ldcg(t.gain + (HALVES ? at1 + i : at0 + 2 * i + 1));
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    gain.a[i] = pair_of(ga[2 * i], ga[2 * i + 1]);
                    gain.b[i] = pair_of(gb[2 * i], gb[2 * i + 1]);
                }
            }
            // z.a = x.a fc.a + x.b fs.b, z.b = x.a fs.a + x.b fc.b; forward with the gains as factors
            Pairs fc = cs, fs = sn;
            if (NORM && !BACK) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    fc.a[i] = mul2(cs.a[i], gain.a[i]);
                    fc.b[i] = mul2(cs.b[i], gain.b[i]);
                    fs.a[i] = mul2(sn.a[i], gain.a[i]);
                    fs.b[i] = mul2(sn.b[i], gain.b[i]);
                }
            }
            auto turned = [&](const Pairs& x) {
                Pairs z;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    z.a[i] = fma2(x.a[i], fc.a[i], mul2(x.b[i], fs.b[i]));
                    z.b[i] = fma2(x.a[i], fs.a[i], mul2(x.b[i], fc.b[i]));
                }
                return z;
            };
            int left = live ? heads[w] - head0 : 0;      // as `coming`, of the rows to be written
            char* out = t.out + b * t.out_b + (long long)(first_head[w] + head0) * t.out_h + n * t.out_n;
            const long long out_step = t.out_h * head_step;
            // U rows at a time, whose chains of shuffles run beside one another
            for (int s0 = 0; s0 < steps[w]; s0 += U) {
                const int rows = min(U, steps[w] - s0);
                asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - U) : "memory");
                __syncwarp();
                Raw<TYPE> x[U], d[GRADS ? U : 1];
#pragma unroll
                for (int u = 0; u < U; ++u) {            // (of a row too many: what the place holds; nothing is done with it)
                    const char* const from = ring_at + ((step + u) % DEPTH) * (STREAMS * STEP);
                    x[u] = read_raw<TYPE, HALVES>(from, at0, at1);
                    if constexpr (GRADS) d[u] = read_raw<TYPE, HALVES>(from + STEP, at0, at1);
                }
                __syncwarp();                            // all lanes have read: the places can be filled again
                step += rows;
                for (int u = 0; u < rows; ++u) issue();
                Pairs z[U];
                if constexpr (!GRADS) {
                    float ss[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const Pairs v = widen<TYPE, HALVES>(x[u]);
                        if constexpr (NORM) ss[u] = dot8(v, v);
                        z[u] = turned(v);
                    }
                    if constexpr (NORM) {
#pragma unroll
                        for (int o = 1; o < LPR; o <<= 1)
#pragma unroll
                            for (int u = 0; u < U; ++u) ss[u] += __shfl_xor_sync(0xffffffffu, ss[u], o);
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            const uint64_t r = twice(rsqrtf(ss[u] * p.inv_D + p.eps));
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                z[u].a[i] = mul2(z[u].a[i], r);
                                z[u].b[i] = mul2(z[u].b[i], r);
                            }
                        }
                    }
                } else {
                    static_assert(!GRADS || U == 1, "a row too many would count");
                    const Pairs v = widen<TYPE, HALVES>(x[0]), y = turned(widen<TYPE, HALVES>(d[0]));     // y: gradient of the normed row
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        z[0].a[i] = mul2(y.a[i], gain.a[i]);
                        z[0].b[i] = mul2(y.b[i], gain.b[i]);
                    }
                    float ss = dot8(v, v), dot = dot8(z[0], v);
#pragma unroll
                    for (int o = 1; o < LPR; o <<= 1) {
                        ss += __shfl_xor_sync(0xffffffffu, ss, o);
                        dot += __shfl_xor_sync(0xffffffffu, dot, o);
                    }
                    // (a slot without a row counts for nothing, also where eps is 0 and 1 / sqrt(0) infinite)
                    const float r1 = left > 0 ? rsqrtf(ss * p.inv_D + p.eps) : 0.f;
                    const uint64_t r = twice(r1), m = twice(-dot * r1 * r1 * p.inv_D);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        acc[w].a[i] = fma2(y.a[i], mul2(v.a[i], r), acc[w].a[i]);
                        acc[w].b[i] = fma2(y.b[i], mul2(v.b[i], r), acc[w].b[i]);
                        z[0].a[i] = mul2(r, fma2(m, v.a[i], z[0].a[i]));
                        z[0].b[i] = mul2(r, fma2(m, v.b[i], z[0].b[i]));
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (left > 0) store_pairs<TYPE, HALVES>(out, at0, at1, z[u]);
                    left -= head_step;
                    out += out_step;
                }
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
    }
    if (!GRADS) grid_dependency_launch();
    if constexpr (GRADS) {
        // the lanes' sums of the thread block, in a fixed order: rows of a warp, then warps; through the ring's memory
        static_assert(sizeof(float) * WARPS * 2 * MAX_D <= ring_bytes(TYPE, true), "the sums fit the ring");
        float (*sums)[2 * MAX_D] = reinterpret_cast<float (*)[2 * MAX_D]>(ring);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 v = of_pair(e < 4 ? acc[w].a[e >> 1 & 1] : acc[w].b[e >> 1 & 1]);
                float s = e & 1 ? v.y : v.x;
#pragma unroll
                for (int o = LPR; o < 32; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                const int i = e & 3, channel = HALVES ? (e < 4 ? at0 : at1) + i : at0 + 2 * i + (e >> 2);
                if (lane < LPR && here) sums[warp][w * D + channel] = s;
            }
        __syncthreads();
        float* to = p.partial + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * D;
        for (int x = threadIdx.x; x < 2 * D; x += 32 * WARPS) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) s += sums[w][x];
            to[x] = s;
        }
    }
}

// The gains' gradients: the thread blocks' sums, added up in fp64 in a fixed order.  Eight channels a thread block.
__global__ void __launch_bounds__(512) gain_kernel(const float* partial, int blocks, int D, float* dq_gain, float* dk_gain) {
    __shared__ double sums[16][8];
    grid_dependency_wait();
    grid_dependency_launch();
    const int x = threadIdx.x % 8, y = threadIdx.x / 8, channel = blockIdx.x * 8 + x;    // 2 D is a multiple of 32
    double s = 0.0;
#pragma unroll 8
    for (int b = y; b < blocks; b += 64) s += (double)__ldcg(partial + (size_t)b * 2 * D + channel);
    s += __shfl_xor_sync(0xffffffffu, s, 8);
    s += __shfl_xor_sync(0xffffffffu, s, 16);
    if (threadIdx.x % 32 < 8) sums[threadIdx.x / 32][x] = s;
    __syncthreads();
    if (threadIdx.x >= 8) return;
    s = 0.0;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += sums[w][x];
    float* to = channel < D ? dq_gain + channel : dk_gain ? dk_gain + channel - D : nullptr;
    if (to) *to = (float)s;
}

template <int TYPE, int LPR, bool HALVES>
auto pick_way(bool norm, bool back) {
    return norm ? (back ? rotary_kernel<TYPE, LPR, HALVES, true, true> : rotary_kernel<TYPE, LPR, HALVES, true, false>)
                : (back ? rotary_kernel<TYPE, LPR, HALVES, false, true> : rotary_kernel<TYPE, LPR, HALVES, false, false>);
}
template <int TYPE, int LPR>
auto pick_layout(bool halves, bool norm, bool back) {
    return halves ? pick_way<TYPE, LPR, true>(norm, back) : pick_way<TYPE, LPR, false>(norm, back);
}
template <int TYPE>
auto pick_lanes(int lanes, bool halves, bool norm, bool back) {
    return lanes == 32 ? pick_layout<TYPE, 32>(halves, norm, back) : lanes == 16 ? pick_layout<TYPE, 16>(halves, norm, back)
           : lanes == 8 ? pick_layout<TYPE, 8>(halves, norm, back) : pick_layout<TYPE, 4>(halves, norm, back);
}

int element_size(int type) { return type == RAPID3_F32 ? 4 : 2; }

// Strides of dimensions of one entry are free; the others hold whole rows apart (an output's; `in`: heads or tokens may not lie over
// one another either) and keep every row on 16 bytes.
int check_rows(const rapid3_heads* s, const rapid3_rows* t, int H) {
    if (!t || !t->data || reinterpret_cast<uintptr_t>(t->data) % 16) return RAPID3_ERR_INVALID_ARG;
    const int unit = 16 / element_size(s->type);
    const int64_t stride[3] = {t->stride_b, t->stride_h, t->stride_n};
    const int size[3] = {s->B, H, s->N};
    for (int i = 0; i < 3; ++i)
        if (size[i] > 1 && (stride[i] < s->D || stride[i] % unit)) return RAPID3_ERR_INVALID_ARG;
    return RAPID3_OK;
}

int check_heads(const rapid3_heads* s, const rapid3_turn* turn) {
    if (!s || !turn) return RAPID3_ERR_INVALID_ARG;
    if (s->type != RAPID3_BF16 && s->type != RAPID3_F16 && s->type != RAPID3_F32) return RAPID3_ERR_INVALID_ARG;
    if (s->B < 1 || s->N < 1 || s->H_q < 1 || s->H_k < 0) return RAPID3_ERR_INVALID_ARG;
    if (s->D < 16 || s->D > MAX_D || s->D % 16) return RAPID3_ERR_UNSUPPORTED;
    if (s->H_q > 65535 || s->H_k > 65535 || s->N > (1 << 30) || (long long)s->B * s->N > (1ll << 31) - 1) return RAPID3_ERR_UNSUPPORTED;
    if (turn->layout != RAPID3_TURN_PAIRS && turn->layout != RAPID3_TURN_HALVES) return RAPID3_ERR_INVALID_ARG;
    if (turn->channels < 0 || turn->channels > s->D || turn->channels % 2) return RAPID3_ERR_INVALID_ARG;
    if (turn->layout == RAPID3_TURN_HALVES && turn->channels % 8) return RAPID3_ERR_UNSUPPORTED;
    if (turn->axes < 1 || turn->axes > MAX_AXES) return RAPID3_ERR_INVALID_ARG;
    if (turn->channels && !turn->freq) return RAPID3_ERR_INVALID_ARG;
    if (!isfinite(turn->amplitude)) return RAPID3_ERR_INVALID_ARG;
    if (!turn->pos && (turn->axes != 1 || turn->pos0 < 0 || turn->pos0 > (1 << 30))) return RAPID3_ERR_INVALID_ARG;
    if (turn->pos && (turn->pos_stride_b < 0 || turn->pos_stride_n < 0)) return RAPID3_ERR_INVALID_ARG;
    int pairs = 0;
    for (int a = 0; a < turn->axes; ++a) {
        if (turn->axis_pairs[a] < 0 || turn->axis_pairs[a] > s->D / 2) return RAPID3_ERR_INVALID_ARG;
        pairs += turn->axis_pairs[a];
    }
    return pairs == turn->channels / 2 ? RAPID3_OK : RAPID3_ERR_INVALID_ARG;
}

int run_rotary(const rapid3_heads* s, const rapid3_rows* const (&in)[2], const rapid3_rows* const (&grad)[2], const rapid3_rows* const (&out)[2],
               const float* const (&gain)[2], float eps, const rapid3_turn* turn, bool norm, bool back, float* dq_gain, float* dk_gain,
               void* workspace, int64_t workspace_bytes, void* stream) {
    int r = check_heads(s, turn);
    if (r != RAPID3_OK) return r;
    const bool grads = norm && back;
    if (norm && (!(eps >= 0.f) || !isfinite(eps))) return RAPID3_ERR_INVALID_ARG;
    Args a = {};
    const int size = element_size(s->type), H[2] = {s->H_q, s->H_k};
    for (int w = 0; w < 2; ++w) {
        RowsArg& t = a.t[w];
        t.H = H[w];
        if (H[w] == 0) continue;
        if ((r = check_rows(s, in[w], H[w])) || (r = check_rows(s, out[w], H[w]))) return r;
        if (grads && (r = check_rows(s, grad[w], H[w]))) return r;
        if (norm && !gain[w]) return RAPID3_ERR_INVALID_ARG;
        t.in = static_cast<const char*>(in[w]->data);
        t.out = static_cast<char*>(out[w]->data);
        t.gain = gain[w];
        t.in_b = in[w]->stride_b * size; t.in_h = in[w]->stride_h * size; t.in_n = in[w]->stride_n * size;
        t.out_b = out[w]->stride_b * size; t.out_h = out[w]->stride_h * size; t.out_n = out[w]->stride_n * size;
        if (grads) {
            t.grad = static_cast<const char*>(grad[w]->data);
            t.grad_b = grad[w]->stride_b * size; t.grad_h = grad[w]->stride_h * size; t.grad_n = grad[w]->stride_n * size;
        }
    }
    if (grads) {
        if (!dq_gain || (s->H_k && !dk_gain) || !workspace || reinterpret_cast<uintptr_t>(workspace) % 16) return RAPID3_ERR_INVALID_ARG;
        if (workspace_bytes < rapid3_norm_rotary_workspace_bytes(s)) return RAPID3_ERR_WORKSPACE;
    }
    TurnArg& t = a.turn;
    t.freq = turn->freq;
    t.pos = turn->pos;
    t.pos_b = turn->pos_stride_b;
    t.pos_n = turn->pos_stride_n;
    t.pos0 = turn->pos0;
    t.pairs = turn->channels / 2;
    t.axes = turn->axes;
    t.amplitude = turn->amplitude;
    for (int x = 0, end = 0; x < turn->axes; ++x) t.axis_end[x] = end += turn->axis_pairs[x];
    a.eps = eps;
    a.inv_D = 1.f / (float)s->D;
    a.N = s->N;
    a.D = s->D;
    int lanes = 4;
    while (8 * lanes < s->D) lanes *= 2;
    const int slots = WARPS * (32 / lanes);
    while ((1 << a.log_tokens) < std::min(s->N, slots)) ++a.log_tokens;
    const int tokens = 1 << a.log_tokens;
    a.tiles = (s->N + tokens - 1) / tokens;
    a.n_tiles = s->B * a.tiles;
    a.partial = static_cast<float*>(workspace);
    // Where the tiles leave SMs without work their heads are shared out, down to one pass of a thread block's warps.
    const int heads = s->H_q + s->H_k, pass = slots / tokens;
    int groups = std::min((heads + pass - 1) / pass, std::max(1, 2 * SM_COUNT / a.n_tiles));
    a.heads_per_block = (heads + groups - 1) / groups;
    groups = (heads + a.heads_per_block - 1) / a.heads_per_block;
    const int blocks = grads ? std::min(a.n_tiles, std::max(1, MAX_GRAD_BLOCKS / groups)) : a.n_tiles;
    const bool halves = turn->layout == RAPID3_TURN_HALVES;
    const auto kernel = s->type == RAPID3_BF16 ? pick_lanes<RAPID3_BF16>(lanes, halves, norm, back)
                        : s->type == RAPID3_F16 ? pick_lanes<RAPID3_F16>(lanes, halves, norm, back)
                                                : pick_lanes<RAPID3_F32>(lanes, halves, norm, back);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (launch_kernel(kernel, dim3(blocks, groups), dim3(32 * WARPS), ring_bytes(s->type, grads), st, a) != cudaSuccess)
        return RAPID3_ERR_CUDA;
    if (grads && launch_kernel(gain_kernel, dim3(2 * s->D / 8), dim3(512), 0, st, (const float*)a.partial, blocks * groups, s->D, dq_gain,
                               dk_gain) != cudaSuccess)
        return RAPID3_ERR_CUDA;
    return RAPID3_OK;
}

}  // namespace

extern "C" {

int rapid3_rotary(const rapid3_heads* s, const rapid3_rows* q, const rapid3_rows* k, const rapid3_turn* turn, int backward,
                  const rapid3_rows* q_out, const rapid3_rows* k_out, void* stream) {
    return run_rotary(s, {q, k}, {nullptr, nullptr}, {q_out, k_out}, {nullptr, nullptr}, 0.f, turn, false, backward != 0, nullptr, nullptr, nullptr,
                      0, stream);
}

int rapid3_norm_rotary(const rapid3_heads* s, const rapid3_rows* q, const rapid3_rows* k, const float* q_gain, const float* k_gain, float eps,
                       const rapid3_turn* turn, const rapid3_rows* q_out, const rapid3_rows* k_out, void* stream) {
    return run_rotary(s, {q, k}, {nullptr, nullptr}, {q_out, k_out}, {q_gain, k_gain}, eps, turn, true, false, nullptr, nullptr, nullptr, 0, stream);
}

int64_t rapid3_norm_rotary_workspace_bytes(const rapid3_heads* s) {
    if (!s || s->D < 16 || s->D > MAX_D || s->D % 16) return RAPID3_ERR_UNSUPPORTED;
    return (int64_t)MAX_GRAD_BLOCKS * 2 * s->D * sizeof(float);
}

int rapid3_norm_rotary_backward(const rapid3_heads* s, const rapid3_rows* dq_out, const rapid3_rows* dk_out, const rapid3_rows* q,
                                const rapid3_rows* k, const float* q_gain, const float* k_gain, float eps, const rapid3_turn* turn,
                                const rapid3_rows* dq, const rapid3_rows* dk, float* dq_gain, float* dk_gain, void* workspace,
                                int64_t workspace_bytes, void* stream) {
    return run_rotary(s, {q, k}, {dq_out, dk_out}, {dq, dk}, {q_gain, k_gain}, eps, turn, true, true, dq_gain, dk_gain, workspace,
                      workspace_bytes, stream);
}

int rapid3_rotary_freqs(int channels, double base, int scaling, double factor, int trained, double fast_turns, double slow_turns, double* freq_host,
                        float* amplitude) {
    if (channels < 2 || channels % 2 || !(base > 1.0) || !isfinite(base) || !freq_host || !amplitude) return RAPID3_ERR_INVALID_ARG;
    if (scaling < RAPID3_SCALE_NONE || scaling > RAPID3_SCALE_PARTS) return RAPID3_ERR_INVALID_ARG;
    if (scaling != RAPID3_SCALE_NONE && (!(factor >= 1.0) || !isfinite(factor))) return RAPID3_ERR_INVALID_ARG;
    if (scaling == RAPID3_SCALE_PARTS && (trained < 1 || !(slow_turns > 0.0) || !(fast_turns > slow_turns) || !isfinite(fast_turns)))
        return RAPID3_ERR_INVALID_ARG;
    if (scaling == RAPID3_SCALE_BASE) base *= channels > 2 ? pow(factor, (double)channels / (channels - 2)) : 1.0;
    for (int i = 0; i < channels / 2; ++i) {
        double f = pow(base, -2.0 * i / channels);
        if (scaling == RAPID3_SCALE_LINEAR) f /= factor;
        if (scaling == RAPID3_SCALE_PARTS) {
            // how often the pair turns over the trained length: often, it keeps its frequency; seldom, its positions are interpolated
            const double turns = trained * f / 6.283185307179586477;
            const double keep = fmin(1.0, fmax(0.0, (turns - slow_turns) / (fast_turns - slow_turns)));
            f = f * keep + f / factor * (1.0 - keep);
        }
        freq_host[i] = f;
    }
    *amplitude = scaling == RAPID3_SCALE_PARTS ? (float)(1.0 + 0.1 * log(factor)) : 1.f;
    return RAPID3_OK;
}

}  // extern "C"
