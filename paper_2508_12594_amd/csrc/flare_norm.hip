// Residual norm: what stands between two blocks, in one pass over a token's channels.  Per row,
//     u = post(y),  a = u act(gate),  x' = x + alpha a,  h = pre(x')
// with post and pre a layer norm, an RMS norm or nothing.  Both norms are taken from fp32 rows that stay in registers (mean,
// then the squares of what is left), h from x' before x' is rounded to its storage type.
//
// Backward, with xh and uh the normalised rows and r their scales:
//     gx = dx' + r_pre (w dh - mean(w dh) - xh mean(w dh xh))          (RMS: without the first mean),  dx = gx
//     da = alpha gx,  du = da act(gate),  dgate = da u act'(gate)
//     dy = r_post (w du - mean(w du) - uh mean(w du uh))
//     dw_pre = sum dh xh,  db_pre = sum dh,  dw_post = sum du uh,  db_post = sum du      over the rows
// Sums over rows are kept in registers over all rows of a workgroup, and the workgroups' sums are added in a fixed order.
//
// Bound by memory: the forward reads x, y (and a gate of each token) and writes x' and h, the backward reads x, y, dx', dh and
// writes dx and dy; x' is formed again rather than read, which costs the same bytes and saves its rounding.
#include "flare_mfma_common.h"

namespace flare {
namespace {

struct NormArgs {
    const void *x, *y, *gate;
    const float *pre_w, *pre_b, *post_w, *post_b;
    void *x_out, *h;
    float *stats;                    // [rows][4]: mean and scale of pre, then of post; or NULL
    const void *dx_out, *dh;         // backward
    void *dx, *dy, *dgate;
    float *part, *gate_part;         // [workgroups][4][C], [units][C]
    long long rows, rows_per_gate;
    long long units, unit_rows, units_per_group;   // backward: a unit is a piece of the rows that share a gate
    int units_per_block;
    int C, pre, post, act, want;     // want: which of the four sums over rows are asked for
    float alpha, eps;
};
enum { WANT_PRE_W = 1, WANT_PRE_B = 2, WANT_POST_W = 4, WANT_POST_B = 8 };

template <int LPR>
struct Lanes {
    static constexpr int THREADS = LPR > 256 ? LPR : 256, ROWS = THREADS / LPR;
};

// Sum over the LPR lanes of a row, the same bits in each.  `red` has two halves that calls take in turn, so that one
// barrier a call is enough.
template <int LPR, int K>
__device__ __forceinline__ void row_sum(float (&v)[K], float *red, int &turn)
{
    constexpr int IN_WAVE = LPR < 64 ? LPR : 64;
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int s = 1; s < IN_WAVE; s *= 2) v[k] += __shfl_xor(v[k], s);
    }
    if constexpr (LPR > 64) {
        constexpr int WAVES = LPR / 64;       // (a row of more than 64 lanes has 128, 256 or 512: a part of the workgroup)
        const int wave = threadIdx.x >> 6, first = wave / WAVES * WAVES;
        float *slot = red + turn * 2 * 8;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) slot[2 * wave + k] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v[k] += slot[2 * (first + w) + k];
        }
    }
}

// Channel of element e of piece p.  VEC: 8 neighbouring channels a piece (16 bytes of 16-bit rows); otherwise, where rows are
// not whole 16-byte pieces, neighbouring lanes take neighbouring channels.
template <int LPR, bool VEC>
__device__ __forceinline__ int channel(int l, int p, int e) { return VEC ? (p * LPR + l) * 8 + e : (p * 8 + e) * LPR + l; }

template <int DT, int LPR, int NP, bool VEC>
__device__ __forceinline__ void load_row(const void *row, int l, int C, float (&v)[8 * NP])
{
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        if constexpr (VEC) {
            const int c = channel<LPR, true>(l, p, 0);
            if (c < C) {
                if constexpr (DT == FLARE_F32) {
                    const float4 a = *reinterpret_cast<const float4 *>(static_cast<const float *>(row) + c),
                                 b = *reinterpret_cast<const float4 *>(static_cast<const float *>(row) + c + 4);
                    v[8 * p] = a.x; v[8 * p + 1] = a.y; v[8 * p + 2] = a.z; v[8 * p + 3] = a.w;
                    v[8 * p + 4] = b.x; v[8 * p + 5] = b.y; v[8 * p + 6] = b.z; v[8 * p + 7] = b.w;
                } else {
                    const u32x4 w = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(row) + c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[8 * p + 2 * e] = elem_lo<DT == FLARE_F16>(w[e]);
                        v[8 * p + 2 * e + 1] = elem_hi<DT == FLARE_F16>(w[e]);
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[8 * p + e] = 0.f;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = channel<LPR, false>(l, p, e);
                float t = 0.f;
                if (c < C) {
                    if constexpr (DT == FLARE_F32) t = static_cast<const float *>(row)[c];
                    else t = elem_value<DT == FLARE_F16>(static_cast<const uint16_t *>(row)[c]);
                }
                v[8 * p + e] = t;
            }
        }
    }
}
template <int DT, int LPR, int NP, bool VEC>
__device__ __forceinline__ void store_row(void *row, int l, int C, const float (&v)[8 * NP])
{
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        if constexpr (VEC) {
            const int c = channel<LPR, true>(l, p, 0);
            if (c < C) {
                if constexpr (DT == FLARE_F32) {
                    float *d = static_cast<float *>(row) + c;
                    *reinterpret_cast<float4 *>(d) = make_float4(v[8 * p], v[8 * p + 1], v[8 * p + 2], v[8 * p + 3]);
                    *reinterpret_cast<float4 *>(d + 4) = make_float4(v[8 * p + 4], v[8 * p + 5], v[8 * p + 6], v[8 * p + 7]);
                } else {
                    u32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = pack_elems<DT == FLARE_F16>(v[8 * p + 2 * e], v[8 * p + 2 * e + 1]);
                    *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(row) + c) = w;
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = channel<LPR, false>(l, p, e);
                if (c < C) {
                    if constexpr (DT == FLARE_F32) static_cast<float *>(row)[c] = v[8 * p + e];
                    else static_cast<uint16_t *>(row)[c] = (uint16_t)rne_elem<DT == FLARE_F16>(v[8 * p + e]);
                }
            }
        }
    }
}
// a norm's weights (1) or biases (0 where there are none)
template <int LPR, int NP, bool VEC>
__device__ __forceinline__ void load_param(const float *w, float otherwise, int l, int C, float (&v)[8 * NP])
{
    if (w) {
        load_row<FLARE_F32, LPR, NP, VEC>(w, l, C, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8 * NP; ++i) v[i] = otherwise;
    }
}
template <int DT>
__device__ __forceinline__ const void *row_at(const void *p, long long row, int C)
{
    return static_cast<const char *>(p) + row * C * (DT == FLARE_F32 ? 4 : 2);
}
template <int DT>
__device__ __forceinline__ void *row_at(void *p, long long row, int C)
{
    return static_cast<char *>(p) + row * C * (DT == FLARE_F32 ? 4 : 2);
}
__device__ __forceinline__ float sigmoid(float g) { return 1.f / (1.f + __expf(-g)); }
__device__ __forceinline__ float act_of(int act, float g)
{
    return act == FLARE_GATE_PLAIN ? g : act == FLARE_GATE_SIGMOID ? sigmoid(g) : g * sigmoid(g);
}

// mean and scale of a row
template <int LPR, int NP, bool VEC>
__device__ __forceinline__ void row_stats(const float (&v)[8 * NP], int kind, int l, int C, float eps, float *red, int &turn,
                                          float &mean, float &scale)
{
    mean = 0.f;
    float s[1] = {0.f};
    if (kind == FLARE_NORM_LAYER) {
#pragma unroll
        for (int i = 0; i < 8 * NP; ++i) s[0] += v[i];          // (zero beyond C)
        row_sum<LPR>(s, red, turn);
        mean = s[0] / (float)C;
    }
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < 8 * NP; ++i) {
        const float t = channel<LPR, VEC>(l, i / 8, i % 8) < C ? v[i] - mean : 0.f;
        s[0] = fmaf(t, t, s[0]);
    }
    row_sum<LPR>(s, red, turn);
    scale = 1.f / sqrtf(s[0] / (float)C + eps);
}

template <int DT, int XT, int LPR, int NP, bool VEC>
__global__ __launch_bounds__(Lanes<LPR>::THREADS) void residual_norm_kernel(const NormArgs a)
{
    using L = Lanes<LPR>;
    __shared__ float red[2 * 2 * 8];
    const int l = threadIdx.x % LPR, C = a.C;
    int turn = 0;
    for (long long row0 = (long long)blockIdx.x * L::ROWS; row0 < a.rows; row0 += (long long)gridDim.x * L::ROWS) {
        const long long wanted = row0 + threadIdx.x / LPR, row = wanted < a.rows ? wanted : a.rows - 1;
        const bool live = wanted < a.rows;
        float x[8 * NP], w[8 * NP], mean, scale;
        load_row<XT, LPR, NP, VEC>(row_at<XT>(a.x, row, C), l, C, x);
        if (a.y) {
            float y[8 * NP];
            load_row<DT, LPR, NP, VEC>(row_at<DT>(a.y, row, C), l, C, y);
            float g[8 * NP];
            if (a.act != FLARE_GATE_NONE) load_row<DT, LPR, NP, VEC>(row_at<DT>(a.gate, row / a.rows_per_gate, C), l, C, g);
            if (a.post != FLARE_NORM_NONE) {
                row_stats<LPR, NP, VEC>(y, a.post, l, C, a.eps, red, turn, mean, scale);
                if (a.stats && live && l == 0) *reinterpret_cast<float2 *>(a.stats + 4 * row + 2) = make_float2(mean, scale);
                load_param<LPR, NP, VEC>(a.post_w, 1.f, l, C, w);
#pragma unroll
                for (int i = 0; i < 8 * NP; ++i) y[i] = (y[i] - mean) * scale * w[i];
                load_param<LPR, NP, VEC>(a.post_b, 0.f, l, C, w);
#pragma unroll
                for (int i = 0; i < 8 * NP; ++i) y[i] += w[i];
            }
            if (a.act != FLARE_GATE_NONE) {
#pragma unroll
                for (int i = 0; i < 8 * NP; ++i) y[i] *= act_of(a.act, g[i]);
            }
#pragma unroll
            for (int i = 0; i < 8 * NP; ++i)
                x[i] = channel<LPR, VEC>(l, i / 8, i % 8) < C ? fmaf(a.alpha, y[i], x[i]) : 0.f;
            if (live) store_row<XT, LPR, NP, VEC>(row_at<XT>(a.x_out, row, C), l, C, x);
        }
        if (a.pre != FLARE_NORM_NONE) {
            row_stats<LPR, NP, VEC>(x, a.pre, l, C, a.eps, red, turn, mean, scale);
            if (a.stats && live && l == 0) *reinterpret_cast<float2 *>(a.stats + 4 * row) = make_float2(mean, scale);
            load_param<LPR, NP, VEC>(a.pre_w, 1.f, l, C, w);
#pragma unroll
            for (int i = 0; i < 8 * NP; ++i) x[i] = (x[i] - mean) * scale * w[i];
            load_param<LPR, NP, VEC>(a.pre_b, 0.f, l, C, w);
#pragma unroll
            for (int i = 0; i < 8 * NP; ++i) x[i] += w[i];
            if (live) store_row<DT, LPR, NP, VEC>(row_at<DT>(a.h, row, C), l, C, x);
        }
    }
}

// The sums of a workgroup's row slots (threads of the same l), added in their order.
template <int LPR, int NP, bool VEC, typename Put>
__device__ __forceinline__ void slot_sums(float (&v)[8 * NP], float *lds, int C, const Put &put)
{
    using L = Lanes<LPR>;
    const int l = threadIdx.x % LPR, r = threadIdx.x / LPR;
    if constexpr (L::ROWS > 1) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8 * NP; ++i) lds[(r * 8 * NP + i) * LPR + l] = v[i];
        __syncthreads();
        if (r == 0) {
#pragma unroll
            for (int i = 0; i < 8 * NP; ++i) {
                float s = v[i];
                for (int k = 1; k < L::ROWS; ++k) s += lds[(k * 8 * NP + i) * LPR + l];
                v[i] = s;
            }
        }
    }
    if (r == 0) put(v, l);
}

template <int DT, int XT, int LPR, int NP, bool VEC>
__global__ __launch_bounds__(Lanes<LPR>::THREADS) void residual_norm_backward_kernel(const NormArgs a)
{
    using L = Lanes<LPR>;
    constexpr int N8 = 8 * NP;
    __shared__ float red[2 * 2 * 8];
    __shared__ float slots[L::ROWS > 1 ? L::ROWS * N8 * LPR : 1];
    const int l = threadIdx.x % LPR, slot = threadIdx.x / LPR, C = a.C;
    int turn = 0;
    float pre_w_sum[N8], pre_b_sum[N8], post_w_sum[N8], post_b_sum[N8];
#pragma unroll
    for (int i = 0; i < N8; ++i) pre_w_sum[i] = pre_b_sum[i] = post_w_sum[i] = post_b_sum[i] = 0.f;
    const bool shared_gate = a.act != FLARE_GATE_NONE && a.rows_per_gate > 1;
    const long long u0 = (long long)blockIdx.x * a.units_per_block;
    const long long u1 = u0 + a.units_per_block < a.units ? u0 + a.units_per_block : a.units;
    for (long long unit = u0; unit < u1; ++unit) {
        const long long group_rows = shared_gate ? a.rows_per_gate : a.rows;
        const long long group = unit / a.units_per_group, in_group = unit % a.units_per_group * a.unit_rows;
        const long long begin = group * group_rows + in_group;
        const long long end = begin + (a.unit_rows < group_rows - in_group ? a.unit_rows : group_rows - in_group);
        float gate_sum[N8];
#pragma unroll
        for (int i = 0; i < N8; ++i) gate_sum[i] = 0.f;
        for (long long row0 = begin; row0 < end; row0 += L::ROWS) {
            const bool live = row0 + slot < end;
            const long long row = live ? row0 + slot : end - 1;
            float x[N8], y[N8], gx[N8], g[N8], w[N8], dh[N8];
            float4 st = make_float4(0.f, 1.f, 0.f, 1.f);
            if (a.stats) st = *reinterpret_cast<const float4 *>(a.stats + 4 * row);
            if (a.dx_out) {
                load_row<XT, LPR, NP, VEC>(row_at<XT>(a.dx_out, row, C), l, C, gx);
            } else {
#pragma unroll
                for (int i = 0; i < N8; ++i) gx[i] = 0.f;
            }
            if (a.dh) load_row<DT, LPR, NP, VEC>(row_at<DT>(a.dh, row, C), l, C, dh);
            if (a.dh) load_row<XT, LPR, NP, VEC>(row_at<XT>(a.x, row, C), l, C, x);
            if (a.y) {
                load_row<DT, LPR, NP, VEC>(row_at<DT>(a.y, row, C), l, C, y);
                if (a.act != FLARE_GATE_NONE) load_row<DT, LPR, NP, VEC>(row_at<DT>(a.gate, row / a.rows_per_gate, C), l, C, g);
                if (a.post != FLARE_NORM_NONE) {
#pragma unroll
                    for (int i = 0; i < N8; ++i) y[i] = (y[i] - st.z) * st.w;
                }
            }
            // u of element i (y holds the normalised branch)
            float pb[N8];
            if (a.post != FLARE_NORM_NONE) {
                load_param<LPR, NP, VEC>(a.post_w, 1.f, l, C, w);
                load_param<LPR, NP, VEC>(a.post_b, 0.f, l, C, pb);
            } else {
#pragma unroll
                for (int i = 0; i < N8; ++i) { w[i] = 1.f; pb[i] = 0.f; }
            }
            if (a.dh) {
                if (a.y) {
#pragma unroll
                    for (int i = 0; i < N8; ++i) {
                        float u = fmaf(y[i], w[i], pb[i]);
                        if (a.act != FLARE_GATE_NONE) u *= act_of(a.act, g[i]);
                        x[i] = fmaf(a.alpha, u, x[i]);
                    }
                }
                float pw[N8], s[2] = {0.f, 0.f};
                load_param<LPR, NP, VEC>(a.pre_w, 1.f, l, C, pw);
#pragma unroll
                for (int i = 0; i < N8; ++i) {
                    x[i] = (x[i] - st.x) * st.y;
                    if (live) {
                        pre_w_sum[i] = fmaf(dh[i], x[i], pre_w_sum[i]);
                        pre_b_sum[i] += dh[i];
                    }
                    dh[i] *= pw[i];              // (zero beyond C: so is dh)
                    s[0] += dh[i];
                    s[1] = fmaf(dh[i], x[i], s[1]);
                }
                row_sum<LPR>(s, red, turn);
                const float m0 = a.pre == FLARE_NORM_LAYER ? s[0] / (float)C : 0.f, m1 = s[1] / (float)C;
#pragma unroll
                for (int i = 0; i < N8; ++i) gx[i] += st.y * (dh[i] - m0 - x[i] * m1);
            }
            if (live && a.dx) store_row<XT, LPR, NP, VEC>(row_at<XT>(a.dx, row, C), l, C, gx);
            if (a.y) {
                float s[2] = {0.f, 0.f};
#pragma unroll
                for (int i = 0; i < N8; ++i) {
                    const bool in = channel<LPR, VEC>(l, i / 8, i % 8) < C;
                    float d = in ? a.alpha * gx[i] : 0.f;
                    if (a.act != FLARE_GATE_NONE) {
                        const float u = fmaf(y[i], w[i], pb[i]);
                        float act, slope;
                        if (a.act == FLARE_GATE_PLAIN) {
                            act = g[i];
                            slope = 1.f;
                        } else {
                            const float sg = sigmoid(g[i]);
                            act = a.act == FLARE_GATE_SIGMOID ? sg : g[i] * sg;
                            slope = a.act == FLARE_GATE_SIGMOID ? sg * (1.f - sg) : sg * (1.f + g[i] * (1.f - sg));
                        }
                        g[i] = d * u * slope;
                        if (live) gate_sum[i] += g[i];
                        d *= act;
                    }
                    if (a.post != FLARE_NORM_NONE) {
                        if (live) {
                            post_w_sum[i] = fmaf(d, y[i], post_w_sum[i]);
                            post_b_sum[i] += d;
                        }
                        d *= w[i];
                        s[0] += d;
                        s[1] = fmaf(d, in ? y[i] : 0.f, s[1]);
                    }
                    gx[i] = d;
                }
                if (live && a.dgate && a.act != FLARE_GATE_NONE && !shared_gate)
                    store_row<DT, LPR, NP, VEC>(row_at<DT>(a.dgate, row, C), l, C, g);
                if (a.post != FLARE_NORM_NONE) {
                    row_sum<LPR>(s, red, turn);
                    const float m0 = a.post == FLARE_NORM_LAYER ? s[0] / (float)C : 0.f, m1 = s[1] / (float)C;
#pragma unroll
                    for (int i = 0; i < N8; ++i) gx[i] = st.w * (gx[i] - m0 - y[i] * m1);
                }
                if (live && a.dy) store_row<DT, LPR, NP, VEC>(row_at<DT>(a.dy, row, C), l, C, gx);
            }
        }
        if (shared_gate && a.dgate) {
            slot_sums<LPR, NP, VEC>(gate_sum, slots, C, [&](const float (&v)[N8], int lane) {
                if (a.units_per_group == 1) store_row<DT, LPR, NP, VEC>(row_at<DT>(a.dgate, group, C), lane, C, v);
                else store_row<FLARE_F32, LPR, NP, VEC>(a.gate_part + unit * C, lane, C, v);
            });
        }
    }
    const auto put = [&](float (&v)[N8], int which, int bit) {
        if (!(a.want & bit)) return;
        slot_sums<LPR, NP, VEC>(v, slots, C, [&](const float (&t)[N8], int lane) {
            store_row<FLARE_F32, LPR, NP, VEC>(a.part + ((long long)blockIdx.x * 4 + which) * C, lane, C, t);
        });
    };
    put(pre_w_sum, 0, WANT_PRE_W);
    put(pre_b_sum, 1, WANT_PRE_B);
    put(post_w_sum, 2, WANT_POST_W);
    put(post_b_sum, 3, WANT_POST_B);
}

// out[c] = sum of `count` rows `stride` apart, in a fixed order: 16 channels and 64 slices of the rows a workgroup.
struct SumJob { const float *part; void *out; long long count, stride; };
struct SumArgs { SumJob job[4]; long long part_step, out_step; int C, tiles; };   // (steps per blockIdx.y)
template <int DT>
__global__ __launch_bounds__(1024) void norm_sum_kernel(const SumArgs a)
{
    __shared__ float sum[64][17];
    const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
    const int tile = blockIdx.x % a.tiles;
    const long long group = blockIdx.x / a.tiles;
    const SumJob &job = a.job[blockIdx.y];
    if (!job.out) return;
    const int ch = tile * 16 + c;
    float s = 0.f;
    if (ch < a.C) {
        const float *p = job.part + group * a.part_step + ch;
#pragma unroll 4
        for (long long i = r; i < job.count; i += 64) s += p[i * job.stride];
    }
    sum[r][c] = s;
    __syncthreads();
    if (r == 0 && ch < a.C) {
        s = 0.f;
        for (int i = 0; i < 64; ++i) s += sum[i][c];
        const long long at = group * a.out_step + ch;
        if constexpr (DT == FLARE_F32) static_cast<float *>(job.out)[at] = s;
        else static_cast<uint16_t *>(job.out)[at] = (uint16_t)rne_elem<DT == FLARE_F16>(s);
    }
}

// ---- launch ----------------------------------------------------------------------------------------------------
// Lanes and pieces of a row: the fewest lanes whose pieces (8 channels, at most 2 a lane) hold it.
int row_capacity(int C, bool vec)
{
    if (!vec) return C <= 512 ? 512 : C <= 2048 ? 2048 : 8192;
    int cap = 64;
    while (cap < C) cap *= 2;
    return cap;
}
bool whole_pieces(const flare_norm_shape &s) { return s.C % 8 == 0; }
int row_slots(int cap) { return cap >= 2048 ? 1 : 2048 / cap; }   // rows a workgroup works on at a time

struct NormPlan {
    long long units, unit_rows, units_per_group;
    int units_per_block, blocks;
    size_t part_bytes, gate_bytes;
};
NormPlan norm_plan(const flare_norm_shape &s)
{
    NormPlan p{};
    const int slots = row_slots(row_capacity(s.C, whole_pieces(s)));
    const bool shared = s.gate != FLARE_GATE_NONE && s.rows_per_gate > 1;
    const long long group_rows = shared ? s.rows_per_gate : s.rows, groups = s.rows / group_rows;
    // about 1024 workgroups, of at least four rounds of rows
    long long want = s.rows / (4LL * slots);
    want = want < 1 ? 1 : want > 1024 ? 1024 : want;
    p.units_per_group = groups >= want ? 1 : (want + groups - 1) / groups;
    long long rows = (group_rows + p.units_per_group - 1) / p.units_per_group;
    rows = (rows + slots - 1) / slots * slots;
    p.unit_rows = rows;
    p.units_per_group = (group_rows + rows - 1) / rows;
    p.units = groups * p.units_per_group;
    p.units_per_block = (int)((p.units + want - 1) / want);
    p.blocks = (int)((p.units + p.units_per_block - 1) / p.units_per_block);
    p.part_bytes = (size_t)p.blocks * 4 * s.C * 4;
    p.gate_bytes = shared && p.units_per_group > 1 ? (size_t)p.units * s.C * 4 : 0;
    return p;
}
size_t pad256(size_t x) { return (x + 255) & ~(size_t)255; }

template <int DT, int XT, int LPR, int NP, bool VEC>
void launch_norm(const NormArgs &a, bool backward, int blocks, hipStream_t stream)
{
    using L = Lanes<LPR>;
    if (backward) {
        residual_norm_backward_kernel<DT, XT, LPR, NP, VEC><<<blocks, L::THREADS, 0, stream>>>(a);
    } else {
        const long long want = (a.rows + L::ROWS - 1) / L::ROWS;
        residual_norm_kernel<DT, XT, LPR, NP, VEC><<<(unsigned)(want < 8192 ? want : 8192), L::THREADS, 0, stream>>>(a);
    }
}
template <int DT, int XT>
void launch_norm_size(const NormArgs &a, bool vec, bool backward, int blocks, hipStream_t stream)
{
    if (!vec) {
        switch (row_capacity(a.C, false)) {
            case 512: return launch_norm<DT, XT, 64, 1, false>(a, backward, blocks, stream);
            case 2048: return launch_norm<DT, XT, 256, 1, false>(a, backward, blocks, stream);
            default: return launch_norm<DT, XT, 512, 2, false>(a, backward, blocks, stream);
        }
    }
    switch (row_capacity(a.C, true)) {
        case 64: return launch_norm<DT, XT, 8, 1, true>(a, backward, blocks, stream);
        case 128: return launch_norm<DT, XT, 16, 1, true>(a, backward, blocks, stream);
        case 256: return launch_norm<DT, XT, 32, 1, true>(a, backward, blocks, stream);
        case 512: return launch_norm<DT, XT, 64, 1, true>(a, backward, blocks, stream);
        case 1024: return launch_norm<DT, XT, 128, 1, true>(a, backward, blocks, stream);
        case 2048: return launch_norm<DT, XT, 256, 1, true>(a, backward, blocks, stream);
        case 4096: return launch_norm<DT, XT, 256, 2, true>(a, backward, blocks, stream);
        default: return launch_norm<DT, XT, 512, 2, true>(a, backward, blocks, stream);
    }
}
void launch_norm_any(const flare_norm_shape &s, const NormArgs &a, bool backward, int blocks, hipStream_t stream)
{
    const bool vec = whole_pieces(s);
    switch (s.dtype) {
        case FLARE_F32: return launch_norm_size<FLARE_F32, FLARE_F32>(a, vec, backward, blocks, stream);
        case FLARE_BF16:
            return s.x_f32 ? launch_norm_size<FLARE_BF16, FLARE_F32>(a, vec, backward, blocks, stream)
                           : launch_norm_size<FLARE_BF16, FLARE_BF16>(a, vec, backward, blocks, stream);
        default:
            return s.x_f32 ? launch_norm_size<FLARE_F16, FLARE_F32>(a, vec, backward, blocks, stream)
                           : launch_norm_size<FLARE_F16, FLARE_F16>(a, vec, backward, blocks, stream);
    }
}
NormArgs norm_args(const flare_norm_shape &s, const flare_norm_params &p, const void *x, const void *y, const void *gate, float alpha,
                   float eps)
{
    NormArgs a{};
    a.x = x;
    a.y = y;
    a.gate = gate;
    a.pre_w = p.pre_weight;
    a.pre_b = p.pre_bias;
    a.post_w = p.post_weight;
    a.post_b = p.post_bias;
    a.rows = s.rows;
    a.rows_per_gate = s.gate == FLARE_GATE_NONE ? 1 : s.rows_per_gate;
    a.C = s.C;
    a.pre = s.pre;
    a.post = s.post;
    a.act = s.gate;
    a.alpha = alpha;
    a.eps = eps;
    return a;
}

}  // namespace

size_t norm_bwd_bytes(const flare_norm_shape &s)
{
    const NormPlan p = norm_plan(s);
    return pad256(p.part_bytes) + pad256(p.gate_bytes);
}

int norm_forward(const flare_norm_shape &s, const flare_norm_params &p, const void *x, const void *y, const void *gate, void *x_out,
                 void *h, float *stats, float alpha, float eps, hipStream_t stream)
{
    NormArgs a = norm_args(s, p, x, y, gate, alpha, eps);
    a.x_out = x_out;
    a.h = h;
    a.stats = stats;
    LaunchTimer timer(KID_NORM_FORWARD, stream);
    launch_norm_any(s, a, false, 0, stream);
    return check_launch();
}

int norm_backward(const flare_norm_shape &s, const flare_norm_params &p, const void *x, const void *y, const void *gate,
                  const float *stats, const void *dx_out, const void *dh, void *dx, void *dy, void *dgate, float *dpre_weight,
                  float *dpre_bias, float *dpost_weight, float *dpost_bias, float alpha, void *ws, hipStream_t stream)
{
    const NormPlan plan = norm_plan(s);
    NormArgs a = norm_args(s, p, x, y, gate, alpha, 0.f);
    a.stats = const_cast<float *>(stats);
    a.dx_out = dx_out;
    a.dh = dh;
    a.dx = dx;
    a.dy = dy;
    a.dgate = dgate;
    a.part = static_cast<float *>(ws);
    a.gate_part = reinterpret_cast<float *>(static_cast<char *>(ws) + pad256(plan.part_bytes));
    a.units = plan.units;
    a.unit_rows = plan.unit_rows;
    a.units_per_group = plan.units_per_group;
    a.units_per_block = plan.units_per_block;
    a.want = (dpre_weight ? WANT_PRE_W : 0) | (dpre_bias ? WANT_PRE_B : 0) | (dpost_weight ? WANT_POST_W : 0) |
             (dpost_bias ? WANT_POST_B : 0);
    {
        LaunchTimer timer(KID_NORM_BACKWARD, stream);
        launch_norm_any(s, a, true, plan.blocks, stream);
    }
    const int tiles = (s.C + 15) / 16;
    if (a.want) {
        SumArgs b{};
        float *const outs[4] = {dpre_weight, dpre_bias, dpost_weight, dpost_bias};
        for (int i = 0; i < 4; ++i) b.job[i] = SumJob{a.part + (size_t)i * s.C, outs[i], plan.blocks, 4LL * s.C};
        b.C = s.C;
        b.tiles = tiles;
        LaunchTimer timer(KID_NORM_SUM, stream);
        norm_sum_kernel<FLARE_F32><<<dim3(tiles, 4), 1024, 0, stream>>>(b);
    }
    if (dgate && plan.gate_bytes) {
        SumArgs b{};
        b.job[0] = SumJob{a.gate_part, dgate, plan.units_per_group, s.C};
        b.part_step = plan.units_per_group * s.C;
        b.out_step = s.C;
        b.C = s.C;
        b.tiles = tiles;
        const unsigned blocks = (unsigned)(s.rows / s.rows_per_gate * tiles);
        LaunchTimer timer(KID_NORM_SUM, stream);
        if (s.dtype == FLARE_F32) norm_sum_kernel<FLARE_F32><<<blocks, 1024, 0, stream>>>(b);
        else if (s.dtype == FLARE_BF16) norm_sum_kernel<FLARE_BF16><<<blocks, 1024, 0, stream>>>(b);
        else norm_sum_kernel<FLARE_F16><<<blocks, 1024, 0, stream>>>(b);
    }
    return check_launch();
}

}  // namespace flare
