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
// writes dx and dy; x' is formed again rather than read, which costs the same bytes and saves its rounding.  A lane holds eight
// channels of a row, 8 to 1024 lanes a row; a workgroup keeps the weights of its channels in registers and asks for its next rows before it
// works on these.
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
    int C, pre, post, act, want;     // want: a bit for each of the sums over rows (weights, biases) that is asked for
    float alpha, eps;
};

template <int LPR>
struct Lanes {
    static constexpr int THREADS = LPR > 256 ? LPR : 256, ROWS = THREADS / LPR;   // rows a workgroup works on at a time
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
        constexpr int WAVES = LPR / 64;       // (of a row; a workgroup of 256 may hold two such rows)
        const int wave = threadIdx.x >> 6, first = wave / WAVES * WAVES;
        float *slot = red + turn * 2 * 16;
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

// Channel of a lane's element e.  VEC: 8 neighbouring channels a lane (16 bytes of 16-bit rows); otherwise, where C is not a
// multiple of eight, neighbouring lanes take neighbouring channels, an element at a time.
template <int LPR, bool VEC>
__device__ __forceinline__ int channel(int l, int e) { return VEC ? l * 8 + e : e * LPR + l; }

// Eight elements of a row as they are in memory (what is asked for ahead), zeros beyond C
template <int DT, bool VEC>
struct Raw {
    uint32_t w[DT == FLARE_F32 || !VEC ? 8 : 4];
};
template <int DT, int LPR, bool VEC>
__device__ __forceinline__ void fetch(const void *tensor, long long row, int l, int C, Raw<DT, VEC> &raw)
{
    const char *p = static_cast<const char *>(tensor) + row * C * (DT == FLARE_F32 ? 4 : 2);
    if constexpr (VEC) {
        u32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
        if (l * 8 < C) {
            a = *reinterpret_cast<const u32x4 *>(p + l * (DT == FLARE_F32 ? 32 : 16));
            if constexpr (DT == FLARE_F32) b = *reinterpret_cast<const u32x4 *>(p + l * 32 + 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            raw.w[i] = a[i];
            if constexpr (DT == FLARE_F32) raw.w[4 + i] = b[i];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = e * LPR + l;
            raw.w[e] = 0;
            if (c < C) {
                if constexpr (DT == FLARE_F32) raw.w[e] = reinterpret_cast<const uint32_t *>(p)[c];
                else raw.w[e] = reinterpret_cast<const uint16_t *>(p)[c];
            }
        }
    }
}
template <int DT, bool VEC>
__device__ __forceinline__ void values(const Raw<DT, VEC> &raw, float (&v)[8])
{
    if constexpr (DT == FLARE_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(raw.w[e]);
    } else if constexpr (VEC) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = elem_lo<DT == FLARE_F16>(raw.w[e]);
            v[2 * e + 1] = elem_hi<DT == FLARE_F16>(raw.w[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = elem_value<DT == FLARE_F16>(raw.w[e]);
    }
}
template <int DT, int LPR, bool VEC>
__device__ __forceinline__ void store_row(void *tensor, long long row, int l, int C, const float (&v)[8])
{
    char *p = static_cast<char *>(tensor) + row * C * (DT == FLARE_F32 ? 4 : 2);
    if constexpr (VEC) {
        if (l * 8 < C) {
            if constexpr (DT == FLARE_F32) {
                *reinterpret_cast<float4 *>(p + l * 32) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4 *>(p + l * 32 + 16) = make_float4(v[4], v[5], v[6], v[7]);
            } else {
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pack_elems<DT == FLARE_F16>(v[2 * e], v[2 * e + 1]);
                *reinterpret_cast<u32x4 *>(p + l * 16) = w;
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = e * LPR + l;
            if (c < C) {
                if constexpr (DT == FLARE_F32) reinterpret_cast<float *>(p)[c] = v[e];
                else reinterpret_cast<uint16_t *>(p)[c] = (uint16_t)rne_elem<DT == FLARE_F16>(v[e]);
            }
        }
    }
}
// a norm's weights (1) or biases (0 where there are none)
template <int LPR, bool VEC>
__device__ __forceinline__ void load_param(const float *w, float otherwise, int l, int C, float (&v)[8])
{
    if (w) {
        Raw<FLARE_F32, VEC> raw;
        fetch<FLARE_F32, LPR, VEC>(w, 0, l, C, raw);
        values<FLARE_F32, VEC>(raw, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = otherwise;
    }
}
// (v_exp_f32 and v_rcp_f32: a few steps of 2^-24.  An exponential that overflows has the reciprocal 0.)
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + fast_exp2(-kLog2e * g)); }
__device__ __forceinline__ float act_of(int act, float g)
{
    return act == FLARE_GATE_PLAIN ? g : act == FLARE_GATE_SIGMOID ? sigmoid(g) : g * sigmoid(g);
}

// mean and scale of a row
template <int LPR, bool VEC>
__device__ __forceinline__ void row_stats(const float (&v)[8], int kind, int l, int C, float eps, float *red, int &turn,
                                          float &mean, float &scale)
{
    mean = 0.f;
    float s[1] = {0.f};
    if (kind == FLARE_NORM_LAYER) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] += v[i];          // (zero beyond C)
        row_sum<LPR>(s, red, turn);
        mean = s[0] * (1.f / (float)C);
    }
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = channel<LPR, VEC>(l, i) < C ? v[i] - mean : 0.f;
        s[0] = fmaf(t, t, s[0]);
    }
    row_sum<LPR>(s, red, turn);
    scale = 1.f / sqrtf(s[0] * (1.f / (float)C) + eps);
}

// RICH: there is a post norm or a gate.
template <int DT, int XT, int LPR, bool VEC, bool RICH>
__global__ __launch_bounds__(Lanes<LPR>::THREADS) void residual_norm_kernel(const NormArgs a)
{
    using L = Lanes<LPR>;
    __shared__ float red[2 * 2 * 16];
    const int l = threadIdx.x % LPR, C = a.C;
    int turn = 0;
    float pre_w[8], pre_b[8], post_w[8], post_b[8];
    load_param<LPR, VEC>(a.pre_w, 1.f, l, C, pre_w);
    load_param<LPR, VEC>(a.pre_b, 0.f, l, C, pre_b);
    if constexpr (RICH) {
        load_param<LPR, VEC>(a.post_w, 1.f, l, C, post_w);
        load_param<LPR, VEC>(a.post_b, 0.f, l, C, post_b);
    }
    Raw<XT, VEC> rx{};
    Raw<DT, VEC> ry{}, rg{};
    const auto ask = [&](long long row) {
        if (row >= a.rows) row = a.rows - 1;
        fetch<XT, LPR, VEC>(a.x, row, l, C, rx);
        if (a.y) fetch<DT, LPR, VEC>(a.y, row, l, C, ry);
        if (RICH && a.act != FLARE_GATE_NONE)
            fetch<DT, LPR, VEC>(a.gate, a.rows_per_gate == 1 ? row : (unsigned)row / (unsigned)a.rows_per_gate, l, C, rg);
    };
    const long long step = (long long)gridDim.x * L::ROWS;
    long long row = (long long)blockIdx.x * L::ROWS + threadIdx.x / LPR;
    const long long end = ((a.rows + L::ROWS - 1) / L::ROWS) * L::ROWS;      // (the lanes of a row behind the last go along)
    if (row < end) ask(row);
    for (; row < end; row += step) {
        const bool live = row < a.rows;
        float x[8], y[8], g[8], mean, scale;
        values<XT, VEC>(rx, x);
        values<DT, VEC>(ry, y);
        if constexpr (RICH) values<DT, VEC>(rg, g);
        if (row + step < end) ask(row + step);
        if (a.y) {
            if constexpr (RICH) {
                if (a.post != FLARE_NORM_NONE) {
                    row_stats<LPR, VEC>(y, a.post, l, C, a.eps, red, turn, mean, scale);
                    if (a.stats && live && l == 0) *reinterpret_cast<float2 *>(a.stats + 4 * row + 2) = make_float2(mean, scale);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = fmaf((y[i] - mean) * scale, post_w[i], post_b[i]);
                }
                if (a.act != FLARE_GATE_NONE) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] *= act_of(a.act, g[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = channel<LPR, VEC>(l, i) < C ? fmaf(a.alpha, y[i], x[i]) : 0.f;
            if (live) store_row<XT, LPR, VEC>(a.x_out, row, l, C, x);
        }
        if (a.pre != FLARE_NORM_NONE) {
            row_stats<LPR, VEC>(x, a.pre, l, C, a.eps, red, turn, mean, scale);
            if (a.stats && live && l == 0) *reinterpret_cast<float2 *>(a.stats + 4 * row) = make_float2(mean, scale);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = fmaf((x[i] - mean) * scale, pre_w[i], pre_b[i]);
            if (live) store_row<DT, LPR, VEC>(a.h, row, l, C, x);
        }
    }
}

// The sums of a workgroup's row slots (threads of the same l), added in their order.
template <int LPR, typename Put>
__device__ __forceinline__ void slot_sums(float (&v)[8], float *lds, const Put &put)
{
    using L = Lanes<LPR>;
    const int l = threadIdx.x % LPR, r = threadIdx.x / LPR;
    if constexpr (L::ROWS > 1) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) lds[(r * 8 + i) * LPR + l] = v[i];
        __syncthreads();
        if (r == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float s = v[i];
                for (int k = 1; k < L::ROWS; ++k) s += lds[(k * 8 + i) * LPR + l];
                v[i] = s;
            }
        }
    }
    if (r == 0) put(v, l);
}

template <int DT, int XT, int LPR, bool VEC, bool RICH>
__global__ __launch_bounds__(Lanes<LPR>::THREADS) void residual_norm_backward_kernel(const NormArgs a)
{
    using L = Lanes<LPR>;
    __shared__ float red[2 * 2 * 16];
    __shared__ float slots[L::ROWS > 1 ? L::ROWS * 8 * LPR : 1];
    const int l = threadIdx.x % LPR, slot = threadIdx.x / LPR, C = a.C;
    int turn = 0;
    // 1024 lanes have 128 registers each: no room for the weights, nor for a row asked for ahead (two rows ahead are no faster), and
    // with a post norm or a gate the sums over the rows lie in LDS (4096 rows of 8192 channels: 447 us with them spilled).
    constexpr bool KEEP = LPR < 1024, SUMS_IN_LDS = LPR == 1024 && RICH;
    __shared__ float4 lds_sums[SUMS_IN_LDS ? 4 * 2 * LPR : 1];
    const auto add_in_lds = [&](int which, const float (&v)[8]) {
        if (!(a.want >> which & 1)) return;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float4 &t = lds_sums[(2 * which + k) * LPR + l];
            t = make_float4(t.x + v[4 * k], t.y + v[4 * k + 1], t.z + v[4 * k + 2], t.w + v[4 * k + 3]);
        }
    };
    if constexpr (SUMS_IN_LDS) {
#pragma unroll
        for (int k = 0; k < 8; ++k) lds_sums[k * LPR + l] = make_float4(0.f, 0.f, 0.f, 0.f);    // (each lane its own)
    }
    float pre_w_sum[8], pre_b_sum[8], post_w_sum[8], post_b_sum[8], gate_sum[8], pre_w[8], post_w[8], post_b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) pre_w_sum[i] = pre_b_sum[i] = post_w_sum[i] = post_b_sum[i] = 0.f;
    const auto weights = [&]() {
        load_param<LPR, VEC>(a.pre_w, 1.f, l, C, pre_w);
        if constexpr (RICH) {
            load_param<LPR, VEC>(a.post_w, 1.f, l, C, post_w);
            load_param<LPR, VEC>(a.post_b, 0.f, l, C, post_b);
        }
    };
    if constexpr (KEEP) weights();
    const float per_channel = 1.f / (float)C;
    const bool gated = RICH && a.act != FLARE_GATE_NONE, normed = RICH && a.post != FLARE_NORM_NONE;
    const bool shared_gate = gated && a.rows_per_gate > 1;
    const long long u0 = (long long)blockIdx.x * a.units_per_block;
    const long long u1 = u0 + a.units_per_block < a.units ? u0 + a.units_per_block : a.units;
    struct Row {
        Raw<XT, VEC> x{}, d{};
        Raw<DT, VEC> y{}, g{}, h{};
        float4 stats = make_float4(0.f, 1.f, 0.f, 1.f);
    };
    Row ahead;
    Raw<DT, VEC> group_gate{};
    for (long long unit = u0; unit < u1; ++unit) {
        const long long group_rows = shared_gate ? a.rows_per_gate : a.rows;
        const long long group = unit / a.units_per_group, in_group = unit % a.units_per_group * a.unit_rows;
        const long long begin = group * group_rows + in_group;
        const long long end = begin + (a.unit_rows < group_rows - in_group ? a.unit_rows : group_rows - in_group);
        const auto ask = [&](Row &to, long long row) {
            if (row >= end) row = end - 1;
            if (a.dh) fetch<XT, LPR, VEC>(a.x, row, l, C, to.x);
            if (a.dx_out) fetch<XT, LPR, VEC>(a.dx_out, row, l, C, to.d);
            if (a.dh) fetch<DT, LPR, VEC>(a.dh, row, l, C, to.h);
            if (a.y) fetch<DT, LPR, VEC>(a.y, row, l, C, to.y);
            if (gated && !shared_gate) fetch<DT, LPR, VEC>(a.gate, row, l, C, to.g);
            if (a.stats) to.stats = *reinterpret_cast<const float4 *>(a.stats + 4 * row);
        };
        if (shared_gate) fetch<DT, LPR, VEC>(a.gate, group, l, C, group_gate);
#pragma unroll
        for (int i = 0; i < 8; ++i) gate_sum[i] = 0.f;
        const auto work_on = [&](Row &here, long long row0) {
            const long long row = row0 + slot;
            const bool live = row < end;
            float x[8], y[8], gx[8], g[8], dh[8];
            if constexpr (!KEEP) weights();
            values<XT, VEC>(here.x, x);
            values<XT, VEC>(here.d, gx);
            values<DT, VEC>(here.h, dh);
            values<DT, VEC>(here.y, y);
            if constexpr (RICH) values<DT, VEC>(shared_gate ? group_gate : here.g, g);
            const float4 st = here.stats;
            if (KEEP && row0 + L::ROWS < end) ask(here, row + L::ROWS);
            if (normed) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = (y[i] - st.z) * st.w;        // the normalised branch
            }
            const auto branch = [&](int i) { return RICH ? fmaf(y[i], post_w[i], post_b[i]) : y[i]; };   // u (weights 1, 0 without a norm)
            float act[8];                       // the gate's value; g becomes its slope
            if (gated) {
                if (a.act == FLARE_GATE_PLAIN) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) { act[i] = g[i]; g[i] = 1.f; }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        // 1 - sigmoid from the exponential where it is small (the difference has no bits left at g = 17)
                        const float t = fast_exp2(-kLog2e * g[i]), sg = __builtin_amdgcn_rcpf(1.f + t), rest = g[i] > 0.f ? t * sg : 1.f - sg;
                        act[i] = a.act == FLARE_GATE_SIGMOID ? sg : g[i] * sg;
                        g[i] = a.act == FLARE_GATE_SIGMOID ? sg * rest : sg * fmaf(g[i], rest, 1.f);
                    }
                }
            }
            if (a.dh) {
                if (a.y) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = fmaf(a.alpha, gated ? branch(i) * act[i] : branch(i), x[i]);
                }
                float s[2] = {0.f, 0.f};
                if constexpr (SUMS_IN_LDS) add_in_lds(1, dh);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] = (x[i] - st.x) * st.y;
                    if constexpr (SUMS_IN_LDS) pre_w_sum[i] = dh[i] * x[i];
                    else if (live) {
                        pre_w_sum[i] = fmaf(dh[i], x[i], pre_w_sum[i]);
                        pre_b_sum[i] += dh[i];
                    }
                    dh[i] *= pre_w[i];              // (zero beyond C: so is dh)
                    s[0] += dh[i];
                    s[1] = fmaf(dh[i], x[i], s[1]);
                }
                if constexpr (SUMS_IN_LDS) add_in_lds(0, pre_w_sum);
                row_sum<LPR>(s, red, turn);
                const float m0 = a.pre == FLARE_NORM_LAYER ? s[0] * per_channel : 0.f, m1 = s[1] * per_channel;
#pragma unroll
                for (int i = 0; i < 8; ++i) gx[i] += st.y * (dh[i] - m0 - x[i] * m1);
            }
            if (live && a.dx) store_row<XT, LPR, VEC>(a.dx, row, l, C, gx);
            if (a.y) {
                float s[2] = {0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool in = channel<LPR, VEC>(l, i) < C;
                    float d = in ? a.alpha * gx[i] : 0.f;
                    if (gated) {
                        const float dg = d * branch(i) * g[i];
                        if (live) gate_sum[i] = shared_gate ? gate_sum[i] + dg : dg;
                        d *= act[i];
                    }
                    if (normed) {
                        if constexpr (SUMS_IN_LDS) {
                            post_w_sum[i] = d * y[i];
                            post_b_sum[i] = d;
                        } else if (live) {
                            post_w_sum[i] = fmaf(d, y[i], post_w_sum[i]);
                            post_b_sum[i] += d;
                        }
                        d *= post_w[i];
                        s[0] += d;
                        s[1] = fmaf(d, in ? y[i] : 0.f, s[1]);
                    }
                    gx[i] = d;
                }
                if (live && a.dgate && gated && !shared_gate) store_row<DT, LPR, VEC>(a.dgate, row, l, C, gate_sum);
                if (normed) {
                    if constexpr (SUMS_IN_LDS) {
                        add_in_lds(2, post_w_sum);
                        add_in_lds(3, post_b_sum);
                    }
                    row_sum<LPR>(s, red, turn);
                    const float m0 = a.post == FLARE_NORM_LAYER ? s[0] * per_channel : 0.f, m1 = s[1] * per_channel;
#pragma unroll
                    for (int i = 0; i < 8; ++i) gx[i] = st.w * (gx[i] - m0 - y[i] * m1);
                }
                if (live && a.dy) store_row<DT, LPR, VEC>(a.dy, row, l, C, gx);
            }
        };
        if (KEEP) ask(ahead, begin + slot);
        for (long long row0 = begin; row0 < end; row0 += L::ROWS) {
            if (!KEEP) ask(ahead, row0 + slot);
            work_on(ahead, row0);
        }
        if (shared_gate && a.dgate) {
            slot_sums<LPR>(gate_sum, slots, [&](const float (&v)[8], int lane) {
                if (a.units_per_group == 1) store_row<DT, LPR, VEC>(a.dgate, group, lane, C, v);
                else store_row<FLARE_F32, LPR, VEC>(a.gate_part, unit, lane, C, v);
            });
        }
    }
    const auto put = [&](float (&v)[8], int which) {
        if (!(a.want >> which & 1)) return;
        if constexpr (SUMS_IN_LDS) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float4 t = lds_sums[(2 * which + k) * LPR + l];
                v[4 * k] = t.x;
                v[4 * k + 1] = t.y;
                v[4 * k + 2] = t.z;
                v[4 * k + 3] = t.w;
            }
        }
        slot_sums<LPR>(v, slots, [&](const float (&t)[8], int lane) {
            store_row<FLARE_F32, LPR, VEC>(a.part, (long long)blockIdx.x * 4 + which, lane, C, t);
        });
    };
    put(pre_w_sum, 0);
    put(pre_b_sum, 1);
    if constexpr (RICH) {
        put(post_w_sum, 2);
        put(post_b_sum, 3);
    }
}

// out[c] = sum of `count` rows `stride` apart, in a fixed order: 16 channels and 64 slices of the rows a workgroup.  Four jobs are the
// weights' and biases' gradients, the fifth the gate's (a sum for each of its rows).
struct SumJob {
    const float *part;
    void *out;
    long long count, stride;
    int groups, dtype;        // sums side by side: `count` rows of `part`, a row of `out` each
};
struct SumArgs { SumJob job[5]; int C, tiles; };
__global__ __launch_bounds__(1024) void norm_sum_kernel(const SumArgs a)
{
    __shared__ float sum[64][17];
    const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
    const int tile = blockIdx.x % a.tiles, group = blockIdx.x / a.tiles;
    const SumJob &job = a.job[blockIdx.y];
    if (!job.out || group >= job.groups) return;
    const int ch = tile * 16 + c;
    float s = 0.f;
    if (ch < a.C) {
        const float *p = job.part + group * job.count * job.stride + ch;
#pragma unroll 4
        for (long long i = r; i < job.count; i += 64) s += p[i * job.stride];
    }
    sum[r][c] = s;
    __syncthreads();
    if (r == 0 && ch < a.C) {
        s = 0.f;
        for (int i = 0; i < 64; ++i) s += sum[i][c];
        const long long at = (long long)group * a.C + ch;
        if (job.dtype == FLARE_F32) static_cast<float *>(job.out)[at] = s;
        else static_cast<uint16_t *>(job.out)[at] = (uint16_t)(job.dtype == FLARE_F16 ? rne_elem<true>(s) : rne_elem<false>(s));
    }
}

// ---- launch ----------------------------------------------------------------------------------------------------
// Lanes of a row: eight channels each.  Where C is not a multiple of eight there are kernels of three sizes only, so that up to three
// quarters of a lane's elements may lie behind the row (250 channels, fp32, 15003 rows: forward and backward 25 and 42 us, 12 and
// 17 us of bytes), and beyond 2048 channels the backward's 1024 lanes spill 74 ... 162 values with a post norm or a gate.
int row_lanes(int C)
{
    const bool vec = C % 8 == 0;
    if (!vec) return C <= 512 ? 64 : C <= 2048 ? 256 : 1024;
    int lanes = 8;
    while (8 * lanes < C) lanes *= 2;
    return lanes;
}
int row_slots(int lanes) { return lanes >= 256 ? 1 : 256 / lanes; }   // rows a workgroup works on at a time

struct NormPlan {
    long long units, unit_rows, units_per_group;
    int units_per_block, blocks;
    size_t part_bytes, gate_bytes;
};
NormPlan norm_plan(const flare_norm_shape &s)
{
    NormPlan p{};
    const int lanes = row_lanes(s.C), slots = row_slots(lanes);
    const bool shared = s.gate != FLARE_GATE_NONE && s.rows_per_gate > 1;
    const long long group_rows = shared ? s.rows_per_gate : s.rows, groups = s.rows / group_rows;
    // as many workgroups as are on the chip together (two or three waves a SIMD), of at least four rounds of rows; rows that share a
    // gate have their own rounds (128 rows of 128 channels, a gate for every two: 14.5 us, 98 us with full rounds counted)
    const long long most = lanes <= 256 ? 768 : lanes == 512 ? 512 : 256;
    long long want = (shared ? groups * ((group_rows + slots - 1) / slots) : s.rows / slots) / 4;
    want = want < 1 ? 1 : want > most ? most : want;
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

template <int DT, int XT, int LPR, bool VEC, bool RICH>
void launch_norm(const NormArgs &a, bool backward, int blocks, hipStream_t stream)
{
    using L = Lanes<LPR>;
    if (backward) {
        residual_norm_backward_kernel<DT, XT, LPR, VEC, RICH><<<blocks, L::THREADS, 0, stream>>>(a);
    } else {
        const long long want = (a.rows + L::ROWS - 1) / L::ROWS, most = LPR <= 256 ? 8192 : 2048 * 512 / L::THREADS;
        residual_norm_kernel<DT, XT, LPR, VEC, RICH><<<(unsigned)(want < most ? want : most), L::THREADS, 0, stream>>>(a);
    }
}
template <int DT, int XT, bool RICH>
void launch_norm_size(const NormArgs &a, bool backward, int blocks, hipStream_t stream)
{
    const int lanes = row_lanes(a.C);
    if (a.C % 8 != 0) {
        switch (lanes) {
            case 64: return launch_norm<DT, XT, 64, false, RICH>(a, backward, blocks, stream);
            case 256: return launch_norm<DT, XT, 256, false, RICH>(a, backward, blocks, stream);
            default: return launch_norm<DT, XT, 1024, false, RICH>(a, backward, blocks, stream);
        }
    }
    switch (lanes) {
        case 8: return launch_norm<DT, XT, 8, true, RICH>(a, backward, blocks, stream);
        case 16: return launch_norm<DT, XT, 16, true, RICH>(a, backward, blocks, stream);
        case 32: return launch_norm<DT, XT, 32, true, RICH>(a, backward, blocks, stream);
        case 64: return launch_norm<DT, XT, 64, true, RICH>(a, backward, blocks, stream);
        case 128: return launch_norm<DT, XT, 128, true, RICH>(a, backward, blocks, stream);
        case 256: return launch_norm<DT, XT, 256, true, RICH>(a, backward, blocks, stream);
        case 512: return launch_norm<DT, XT, 512, true, RICH>(a, backward, blocks, stream);
        default: return launch_norm<DT, XT, 1024, true, RICH>(a, backward, blocks, stream);
    }
}
template <int DT, int XT>
void launch_norm_rich(const NormArgs &a, bool backward, int blocks, hipStream_t stream)
{
    if (a.post != FLARE_NORM_NONE || a.act != FLARE_GATE_NONE) launch_norm_size<DT, XT, true>(a, backward, blocks, stream);
    else launch_norm_size<DT, XT, false>(a, backward, blocks, stream);
}
void launch_norm_any(const flare_norm_shape &s, const NormArgs &a, bool backward, int blocks, hipStream_t stream)
{
    switch (s.dtype) {
        case FLARE_F32: return launch_norm_rich<FLARE_F32, FLARE_F32>(a, backward, blocks, stream);
        case FLARE_BF16:
            return s.x_f32 ? launch_norm_rich<FLARE_BF16, FLARE_F32>(a, backward, blocks, stream)
                           : launch_norm_rich<FLARE_BF16, FLARE_BF16>(a, backward, blocks, stream);
        default:
            return s.x_f32 ? launch_norm_rich<FLARE_F16, FLARE_F32>(a, backward, blocks, stream)
                           : launch_norm_rich<FLARE_F16, FLARE_F16>(a, backward, blocks, stream);
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
    float *const outs[4] = {dpre_weight, dpre_bias, dpost_weight, dpost_bias};
    for (int i = 0; i < 4; ++i) a.want |= outs[i] ? 1 << i : 0;
    {
        LaunchTimer timer(KID_NORM_BACKWARD, stream);
        launch_norm_any(s, a, true, plan.blocks, stream);
    }
    SumArgs b{};
    b.C = s.C;
    b.tiles = (s.C + 15) / 16;
    for (int i = 0; i < 4; ++i) b.job[i] = SumJob{a.part + (size_t)i * s.C, outs[i], plan.blocks, 4LL * s.C, 1, FLARE_F32};
    int groups = 1, jobs = a.want ? 4 : 0;
    if (dgate && plan.gate_bytes) {
        groups = (int)(s.rows / s.rows_per_gate);
        jobs = 5;
        b.job[4] = SumJob{a.gate_part, dgate, plan.units_per_group, s.C, groups, s.dtype};
    }
    if (jobs) {
        LaunchTimer timer(KID_NORM_SUM, stream);
        norm_sum_kernel<<<dim3(b.tiles * groups, jobs), 1024, 0, stream>>>(b);
    }
    return check_launch();
}

}  // namespace flare
