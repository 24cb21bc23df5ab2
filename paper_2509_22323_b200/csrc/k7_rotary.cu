// K7: rotary positions of Q and K heads, alone or behind the RMS normalisation of each head, and the gradients of both.
// Per row x[D] of one (sequence, head, token):
//     y = x / sqrt(mean(x^2) + eps) * gain            (NORM; else y = x)
//     z = amplitude * R(position . freq) y            on the turned channel pairs, z = y on the others
// and, from dz (BACK), with g = amplitude * R^T dz, u = x r, r = 1 / sqrt(mean(x^2) + eps):
//     dx = r (g gain - u mean(g gain u)),  dgain = sum over all rows of g u          (NORM; else dx = g)
// All of it in fp32, one rounding to the tensors' type.  The angles of far positions need more: position * freq / 2 pi is taken in
// fp64, its fraction alone goes on to sincospif.
//
// Bound by HBM: a row is read once (BACK with NORM: two rows) and written once.  A lane holds four channel pairs, so the rotation is
// the lane's own in both layouts; the lanes of a row add up its squares by shuffles.  A thread block does TOKENS tokens of one
// sequence for many heads, which share the tokens' cosines and sines: these are computed once, into shared memory, while the first rows
// are on their way (for 48 heads 4 % of the instructions; from a table in memory they would be a second read of up to a row a token).
#include <math.h>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "common.cuh"

namespace {

constexpr int WARPS = 8, TOKENS = 16, MAX_D = 256, MAX_AXES = 4;
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
    float eps;
    int N, D, log_tokens, tiles; // tokens of a thread block (a power of two), thread blocks of a sequence
    int n_tiles;                 // of all sequences
    int heads_per_block;
    float* partial;              // BACK with NORM: [thread block][2][D]
};

// Four consecutive channels, widened.
template <int TYPE>
__device__ __forceinline__ void load4(const char* p, float (&x)[4]) {
    if constexpr (TYPE == RAPID3_F32) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(p));
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
        const uint2 v = __ldcg(reinterpret_cast<const uint2*>(p));
        if constexpr (TYPE == RAPID3_BF16) {
            x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
            x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
        } else {
            const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&v.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
            x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
        }
    }
}
template <int TYPE>
__device__ __forceinline__ void store4(char* p, float a, float b, float c, float d) {
    if constexpr (TYPE == RAPID3_F32) {
        *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
    } else if constexpr (TYPE == RAPID3_BF16) {
        const __nv_bfloat162 u = __floats2bfloat162_rn(a, b), v = __floats2bfloat162_rn(c, d);
        *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&u), *reinterpret_cast<const uint32_t*>(&v));
    } else {
        const __half2 u = __floats2half2_rn(a, b), v = __floats2half2_rn(c, d);
        *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&u), *reinterpret_cast<const uint32_t*>(&v));
    }
}

// LPR lanes hold a row: lane c the channel pairs 4 c .. 4 c + 3, a their first members and b their second ones.
template <int TYPE, int LPR, bool HALVES, bool NORM, bool BACK>
__global__ void __launch_bounds__(32 * WARPS) rotary_kernel(const __grid_constant__ Args p) {
    constexpr int RPW = 32 / LPR, SIZE = TYPE == RAPID3_F32 ? 4 : 2;
    constexpr bool GRADS = NORM && BACK;
    constexpr int AHEAD = GRADS ? 2 : 4;                // rows of a lane on their way at once
    extern __shared__ float4 table[];                   // [token][cos, sin][LPR]: four pairs; unturned ones (1, 0)
    __shared__ float sums[GRADS ? WARPS : 1][GRADS ? 2 * MAX_D : 1];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, c = lane % LPR, r0 = lane / LPR;
    const int D = p.D, half = p.turn.pairs;
    const bool here = 8 * c < D;
    // the lane's channels: two runs of four
    const bool split = HALVES && 4 * c < half;
    const int at0 = split ? 4 * c : 8 * c, at1 = split ? half + 4 * c : 8 * c + 4;
    float acc[GRADS ? 2 : 1][8];
#pragma unroll
    for (int w = 0; w < (GRADS ? 2 : 1); ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[w][e] = 0.f;
    grid_dependency_wait();
    for (int tile = blockIdx.x; tile < p.n_tiles; tile += gridDim.x) {
        const int b = tile / p.tiles, n0 = (tile - b * p.tiles) << p.log_tokens, tokens = min(1 << p.log_tokens, p.N - n0);
        __syncthreads();                                // the tile before is through with the table
        for (int x = threadIdx.x; x < tokens * 4 * LPR; x += 32 * WARPS) {
            const int t = x / (4 * LPR), pair = x % (4 * LPR);
            float sine = 0.f, cosine = 1.f;
            if (pair < half) {
                int axis = 0;
                while (axis + 1 < p.turn.axes && pair >= p.turn.axis_end[axis]) ++axis;
                const int at = p.turn.pos ? __ldcg(p.turn.pos + b * p.turn.pos_b + (n0 + t) * p.turn.pos_n + axis) : p.turn.pos0 + n0 + t;
                double turns = (double)at * (__ldcg(p.turn.freq + pair) * 0.15915494309189533577);
                turns -= rint(turns);
                sincospif(2.f * (float)turns, &sine, &cosine);
                sine *= p.turn.amplitude;
                cosine *= p.turn.amplitude;
            }
            float* to = reinterpret_cast<float*>(table + (t * 2) * LPR + pair / 4) + pair % 4;
            to[0] = cosine;
            to[4 * LPR] = BACK ? -sine : sine;          // the transposed rotation turns back
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const RowsArg& t = p.t[w];
            // this thread block's heads among those of Q and then K
            const int before = w ? p.t[0].H : 0;
            const int h0 = max(0, (int)blockIdx.y * p.heads_per_block - before), h1 = min(t.H, ((int)blockIdx.y + 1) * p.heads_per_block - before);
            const int rows = h1 > h0 ? (h1 - h0) << p.log_tokens : 0;
            if (rows == 0) continue;
            float ga[4], gb[4];
            if (NORM && here) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ga[i] = __ldcg(t.gain + (HALVES ? at0 + i : at0 + 2 * i));
                    gb[i] = __ldcg(t.gain + (HALVES ? at1 + i : at0 + 2 * i + 1));
                }
            }
            const char* in = t.in + b * t.in_b + (long long)h0 * t.in_h + (long long)n0 * t.in_n;
            const char* grad = GRADS ? t.grad + b * t.grad_b + (long long)h0 * t.grad_h + (long long)n0 * t.grad_n : nullptr;
            char* out = t.out + b * t.out_b + (long long)h0 * t.out_h + (long long)n0 * t.out_n;
            float lo[AHEAD][4], hi[AHEAD][4], dlo[GRADS ? AHEAD : 1][4], dhi[GRADS ? AHEAD : 1][4];
            for (int first = warp * RPW + r0; first - r0 < rows; first += AHEAD * WARPS * RPW) {
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const int row = first + u * WARPS * RPW, h = row >> p.log_tokens, n = row & ((1 << p.log_tokens) - 1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        lo[u][i] = hi[u][i] = 0.f;
                        if (GRADS) dlo[GRADS ? u : 0][i] = dhi[GRADS ? u : 0][i] = 0.f;
                    }
                    if (row < rows && n < tokens && here) {
                        const char* x = in + h * t.in_h + n * t.in_n;
                        load4<TYPE>(x + at0 * SIZE, lo[u]);
                        load4<TYPE>(x + at1 * SIZE, hi[u]);
                        if constexpr (GRADS) {
                            const char* d = grad + h * t.grad_h + n * t.grad_n;
                            load4<TYPE>(d + at0 * SIZE, dlo[u]);
                            load4<TYPE>(d + at1 * SIZE, dhi[u]);
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const int row = first + u * WARPS * RPW, h = row >> p.log_tokens, n = row & ((1 << p.log_tokens) - 1);
                    if (row - r0 >= rows) break;        // the same for the whole warp
                    float xa[4], xb[4], za[4], zb[4];
                    auto pairs_of = [&](const float (&l)[4], const float (&m)[4], float (&a)[4], float (&bb)[4]) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            a[i] = HALVES ? l[i] : i < 2 ? l[2 * i] : m[2 * i - 4];
                            bb[i] = HALVES ? m[i] : i < 2 ? l[2 * i + 1] : m[2 * i - 3];
                        }
                    };
                    pairs_of(lo[u], hi[u], xa, xb);
                    const int tt = min(n, tokens - 1);  // lanes without a row read some token's
                    const float4 co = table[(tt * 2) * LPR + c], si = table[(tt * 2 + 1) * LPR + c];
                    const float cs[4] = {co.x, co.y, co.z, co.w}, sn[4] = {si.x, si.y, si.z, si.w};
                    if constexpr (!GRADS) {
                        float r = 1.f;
                        if constexpr (NORM) {
                            float ss = 0.f;
#pragma unroll
                            for (int i = 0; i < 4; ++i) ss = fmaf(xa[i], xa[i], fmaf(xb[i], xb[i], ss));
#pragma unroll
                            for (int o = 1; o < LPR; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
                            r = rsqrtf(ss / (float)D + p.eps);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float a = NORM ? xa[i] * r * ga[i] : xa[i], bb = NORM ? xb[i] * r * gb[i] : xb[i];
                            za[i] = fmaf(a, cs[i], -(bb * sn[i]));
                            zb[i] = fmaf(a, sn[i], bb * cs[i]);
                        }
                    } else {
                        float da[4], db[4], ss = 0.f, dot = 0.f;
                        pairs_of(dlo[u], dhi[u], da, db);
                        float ya[4], yb[4];             // gradient of the normed row
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            ya[i] = fmaf(da[i], cs[i], -(db[i] * sn[i]));
                            yb[i] = fmaf(da[i], sn[i], db[i] * cs[i]);
                            ss = fmaf(xa[i], xa[i], fmaf(xb[i], xb[i], ss));
                            za[i] = ya[i] * ga[i];
                            zb[i] = yb[i] * gb[i];
                            dot = fmaf(za[i], xa[i], fmaf(zb[i], xb[i], dot));
                        }
                        if (!here) dot = 0.f;           // (gains of lanes without channels are not loaded)
#pragma unroll
                        for (int o = 1; o < LPR; o <<= 1) {
                            ss += __shfl_xor_sync(0xffffffffu, ss, o);
                            dot += __shfl_xor_sync(0xffffffffu, dot, o);
                        }
                        const float r = rsqrtf(ss / (float)D + p.eps), m = dot * r * r / (float)D;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            acc[w][i] = fmaf(ya[i], xa[i] * r, acc[w][i]);
                            acc[w][4 + i] = fmaf(yb[i], xb[i] * r, acc[w][4 + i]);
                            za[i] = r * fmaf(-m, xa[i], za[i]);
                            zb[i] = r * fmaf(-m, xb[i], zb[i]);
                        }
                    }
                    if (row < rows && n < tokens && here) {
                        char* z = out + h * t.out_h + n * t.out_n;
                        if (HALVES) {
                            store4<TYPE>(z + at0 * SIZE, za[0], za[1], za[2], za[3]);
                            store4<TYPE>(z + at1 * SIZE, zb[0], zb[1], zb[2], zb[3]);
                        } else {
                            store4<TYPE>(z + at0 * SIZE, za[0], zb[0], za[1], zb[1]);
                            store4<TYPE>(z + at1 * SIZE, za[2], zb[2], za[3], zb[3]);
                        }
                    }
                }
            }
        }
    }
    grid_dependency_launch();
    if constexpr (GRADS) {
        // the lanes' sums of the thread block, in a fixed order: rows of a warp, then warps
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float s = acc[w][e];
#pragma unroll
                for (int o = LPR; o < 32; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                const int i = e & 3, channel = HALVES ? (e < 4 ? at0 : at1) + i : at0 + 2 * i + (e >> 2);
                if (r0 == 0 && here) sums[warp][w * D + channel] = s;
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

// The gains' gradients: the thread blocks' sums, added up in fp64 in a fixed order.  32 channels a thread block.
__global__ void __launch_bounds__(1024) gain_kernel(const float* partial, int blocks, int D, float* dq_gain, float* dk_gain) {
    __shared__ double sums[32][33];
    grid_dependency_wait();
    grid_dependency_launch();
    const int x = threadIdx.x % 32, y = threadIdx.x / 32, channel = blockIdx.x * 32 + x;
    double s = 0.0;
    if (channel < 2 * D)
        for (int b = y; b < blocks; b += 32) s += (double)__ldcg(partial + (size_t)b * 2 * D + channel);
    sums[y][x] = s;
    __syncthreads();
    s = sums[x][y];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int mine = blockIdx.x * 32 + y;
    if (x == 0 && mine < 2 * D) {
        float* to = mine < D ? dq_gain + mine : dk_gain ? dk_gain + mine - D : nullptr;
        if (to) *to = (float)s;
    }
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
    a.N = s->N;
    a.D = s->D;
    while ((1 << a.log_tokens) < std::min(s->N, TOKENS)) ++a.log_tokens;
    const int tokens = 1 << a.log_tokens;
    a.tiles = (s->N + tokens - 1) / tokens;
    a.n_tiles = s->B * a.tiles;
    a.partial = static_cast<float*>(workspace);
    int lanes = 4;
    while (8 * lanes < s->D) lanes *= 2;
    // Where the tiles leave SMs without work their heads are shared out, down to one pass of a thread block's warps.
    const int heads = s->H_q + s->H_k, pass = std::max(1, WARPS * (32 / lanes) / tokens);
    int groups = std::min((heads + pass - 1) / pass, std::max(1, 2 * SM_COUNT / a.n_tiles));
    a.heads_per_block = (heads + groups - 1) / groups;
    groups = (heads + a.heads_per_block - 1) / a.heads_per_block;
    const int blocks = grads ? std::min(a.n_tiles, std::max(1, MAX_GRAD_BLOCKS / groups)) : a.n_tiles;
    const bool halves = turn->layout == RAPID3_TURN_HALVES;
    const auto kernel = s->type == RAPID3_BF16 ? pick_lanes<RAPID3_BF16>(lanes, halves, norm, back)
                        : s->type == RAPID3_F16 ? pick_lanes<RAPID3_F16>(lanes, halves, norm, back)
                                                : pick_lanes<RAPID3_F32>(lanes, halves, norm, back);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (launch_kernel(kernel, dim3(blocks, groups), dim3(32 * WARPS), (size_t)tokens * 2 * lanes * sizeof(float4), st, a) != cudaSuccess)
        return RAPID3_ERR_CUDA;
    if (grads && launch_kernel(gain_kernel, dim3((2 * s->D + 31) / 32), dim3(1024), 0, st, (const float*)a.partial, blocks * groups, s->D, dq_gain,
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
