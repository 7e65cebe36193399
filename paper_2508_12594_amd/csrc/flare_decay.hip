// Decay mixer: causal linear attention with a decay for each head.  Per (b,h), with l = exp(log_decay) and S a d x d matrix,
//     S_t = l S_{t-1} + k_t v_t^T,      o_t = scale * S_t^T q_t.
//
// Everything is one scan.  With three token sequences x, y, z and a state C,
//     out_t = x_t (p sum_{u <= t} l^(t-u) <x_t, y_u> z_u)  +  w l^(t+lead) x_t C,
//     C    <- l^n C + m sum_u l^(n-u-lead) y_u z_u^T                                  (n tokens later)
// the forward is (x,y,z) = (q,k,v); dQ is (dO,v,k) with the transposed state; with time running backwards dK is (v,dO,q)
// and dV (k,q,dO), whose state is the gradient of S.  (Forwards lead = 1: a state counts from the token before.
// Backwards lead = 0: what is carried is the gradient of the state before the token, l already in it.)
//
// Tokens are taken 32 at a time.  A wave owns 32 columns of z and of the state: all d x 32 entries of the state stay in
// its matrix accumulators (fp32) from the first token of its segment to the last.  Per 32 tokens, with the layouts of
// v_mfma_f32_32x32x16 (flare_mfma_common.h):
//   P^T = Y X^T            lane = token of x, registers = tokens of y; weighted by l^(t-u) (0 above the diagonal)
//   O^T = C^T X^T          the state's accumulators, rounded, are the A operand as they lie: a contraction index in
//                          accumulator order, which X's rows are read in too
//   O^T += Z^T P^T         likewise P^T's accumulators are the B operand
//   C   += Y^T (weight Z)  Y and Z read down their columns (transposing LDS reads)
// so that nothing but the three token tiles passes through LDS.
#include "flare_mfma_common.h"

namespace flare {
namespace {

// 8 elements of a matrix operand
template <int DT>
struct Frag { u32x4 w; };
template <>
struct Frag<FLARE_F32> { float v[8]; };

template <int DT>
__device__ __forceinline__ f32x16 mma(const Frag<DT> &a, const Frag<DT> &b, f32x16 c)
{
    if constexpr (DT == FLARE_F32) {
        // v_mfma_f32_32x32x2_f32: lane (row, half) holds one element of contraction slot `half`.  Element e of all lanes
        // is a step of its own, so eight steps contract the same 16 indices as one 16-bit step.
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
        return c;
    } else {
        return mfma_s<DT == FLARE_F16>(as_bf16x8(a.w), as_bf16x8(b.w), c);
    }
}
template <int DT>
__device__ __forceinline__ Frag<DT> pack8(const float (&x)[8])
{
    Frag<DT> f;
    if constexpr (DT == FLARE_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f.v[e] = x[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f.w[e] = pack_elems<DT == FLARE_F16>(x[2 * e], x[2 * e + 1]);
    }
    return f;
}
template <int DT>
__device__ __forceinline__ float elem_of(const Frag<DT> &f, int e)
{
    if constexpr (DT == FLARE_F32) return f.v[e];
    else return (e & 1) ? elem_hi<DT == FLARE_F16>(f.w[e >> 1]) : elem_lo<DT == FLARE_F16>(f.w[e >> 1]);
}

struct ScanJob {
    const void *x, *y, *z;
    void *out;
    const float *first;    // state before the first token, [B][H][d][d], or NULL (zero)
    float *last;           // state behind the last token, or NULL
    float p, w, m;         // see above
    int reverse;           // tokens from the last to the first (then lead = 0)
    int first_turned;      // `first` is the transposed state
};
struct ScanArgs {
    ScanJob job[3];
    const float *log_decay;   // [H]
    const int *lengths;       // [B] or NULL
    float *slots;             // [job][B*H][segments][d][d]: a segment's own sum, then the state before it
    TokStride ts;
    int H, N, BH, segments, seg_len;
};

template <int DT, int D>
struct Tile {
    static constexpr int DP = D < 32 ? 32 : D;              // columns in LDS (d = 16: the upper 16 stay zero)
    static constexpr int WAVES = DP / 32, THREADS = 64 * WAVES;
    static constexpr int ES = DT == FLARE_F32 ? 4 : 2;
    static constexpr int ROW = DP * ES + 16, BYTES = 32 * ROW;
    static constexpr int ROW_PIECES = D * ES / 16, PIECES = 32 * ROW_PIECES / THREADS;   // 16-byte pieces, and each thread's
    static constexpr int BUFFERS = 6 * BYTES <= 64 * 1024 ? 2 : 1;
    // planes of the weighted z: what the state sums is good to 2^-22 (fp16) or 2^-24 (bf16) of a term
    static constexpr int PLANES = DT == FLARE_F32 ? 1 : DT == FLARE_F16 ? 2 : 3;
};

// One head's decay in log2 units per token.  (Far below what fp32 weights resolve it makes no difference, and 0 * inf would.)
__device__ __forceinline__ float decay_log2(float g) { return g <= 0.f ? fmaxf(g * kLog2e, -3000.f) : __builtin_nanf(""); }
__device__ __forceinline__ int item_length(const int *lengths, int b, int N) { return lengths ? min(max(lengths[b], 0), N) : N; }

template <int DT, int D>
__device__ __forceinline__ Frag<DT> row_frag(const char *tile, int row, int s, int hh)
{
    using T = Tile<DT, D>;
    const char *p = tile + row * T::ROW + (16 * s + 4 * hh) * T::ES;
    Frag<DT> f;
    if constexpr (DT == FLARE_F32) {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 32);
        f.v[0] = a.x; f.v[1] = a.y; f.v[2] = a.z; f.v[3] = a.w;
        f.v[4] = b.x; f.v[5] = b.y; f.v[6] = b.z; f.v[7] = b.w;
    } else {
        const u32x2 a = *reinterpret_cast<const u32x2 *>(p), b = *reinterpret_cast<const u32x2 *>(p + 16);
        f.w[0] = a[0]; f.w[1] = a[1]; f.w[2] = b[0]; f.w[3] = b[1];
    }
    return f;
}
// Column 32 * ct + lane % 32 of the tile, 8 tokens of step ks in accumulator order
template <int DT, int D>
__device__ __forceinline__ Frag<DT> col_frag(const char *tile, int ct, int ks, int lane)
{
    using T = Tile<DT, D>;
    Frag<DT> f;
    if constexpr (DT == FLARE_F32) {
        const char *p = tile + (32 * ct + (lane & 31)) * 4 + (16 * ks + 4 * (lane >> 5)) * T::ROW;
#pragma unroll
        for (int e = 0; e < 8; ++e) f.v[e] = *reinterpret_cast<const float *>(p + (8 * (e >> 2) + (e & 3)) * T::ROW);
    } else {
        const int g = lane >> 4, q = lane & 15;
        const char *p = tile + (16 * ks + 4 * (g >> 1) + (q >> 2)) * T::ROW + (32 * ct + 16 * (g & 1) + 4 * (q & 3)) * 2;
        const u32x2 a = lds_read_tr16(reinterpret_cast<const uint16_t *>(p));
        const u32x2 b = lds_read_tr16(reinterpret_cast<const uint16_t *>(p + 8 * T::ROW));
        f.w[0] = a[0]; f.w[1] = a[1]; f.w[2] = b[0]; f.w[3] = b[1];
    }
    return f;
}

// fp16 operands made of fp32 values (the state, P, the weighted z) are scaled by a power of two that the whole wave shares, so
// that the largest of them lies between 2^2 and 2^15: a sum of many tokens may exceed 65504, and products of small
// gradients lie among the subnormals.  `e` is kept from chunk to chunk; returns with the exponent to take off.
__device__ __forceinline__ void fit_exponent(int &e, float largest)
{
    const bool some = __any(largest > 0.f);
    while (e < 96 && __any(ldexpf(largest, -e) > 32768.f)) e += 12;
    while (some && e > -96 && !__any(ldexpf(largest, -e) > 4.f)) e -= 12;
}

// SUM: only the segment's own sum (the state it adds), into its slot.
template <int DT, int D, bool SUM>
__global__ __launch_bounds__((Tile<DT, D>::THREADS), 2) void decay_scan_kernel(const ScanArgs a)
{
    using T = Tile<DT, D>;
    constexpr int STEPS = D / 16, CT = T::DP / 32;
    constexpr bool F16 = DT == FLARE_F16;
    __shared__ __align__(16) char lds[T::BUFFERS * 3 * T::BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, hh = lane >> 5;
    const int seg = blockIdx.x % a.segments, bh = blockIdx.x / a.segments, h = bh % a.H;
    const ScanJob &job = a.job[blockIdx.y];
    const bool reverse = job.reverse != 0;
    const int lead = reverse ? 0 : 1;
    const int len = item_length(a.lengths, bh / a.H, a.N);
    const int t_begin = seg * a.seg_len, t_end = min(t_begin + a.seg_len, len);
    const size_t base = tok_base(a.ts, bh, a.H);
    const float e2 = decay_log2(a.log_decay[h]);

    if constexpr (SUM) {
        if (t_begin + a.seg_len >= len) return;       // nobody reads the sum of the last segment
    } else {
        // rows of the padding
        const int z0 = max(t_begin, len), z1 = min(t_begin + a.seg_len, a.N);
        for (int q = tid; q < (z1 - z0) * T::ROW_PIECES; q += T::THREADS)
            *reinterpret_cast<u32x4 *>(static_cast<char *>(job.out) +
                                       (base + tok_off(a.ts, z0 + q / T::ROW_PIECES)) * T::ES + q % T::ROW_PIECES * 16) = u32x4{0, 0, 0, 0};
        if (seg != 0 && t_begin >= len) return;
    }
    const size_t slot = (((size_t)blockIdx.y * a.BH + bh) * a.segments + seg) * (D * D);

    // the state before the segment: column 32 wave + l32, rows in accumulator order
    f32x16 acc[CT];
    const int col = 32 * wave + l32;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[ct] = splat16(0.f);
    if constexpr (!SUM) {
        const bool from_slot = a.segments > 1;
        const float *s = from_slot ? a.slots + slot : job.first ? job.first + (size_t)bh * (D * D) : nullptr;
        if (s && col < D) {
            const bool turned = !from_slot && job.first_turned;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = 32 * ct + perm_index(r >> 3, hh, r & 7);
                    if (D >= 32 || row < D) acc[ct][r] = turned ? s[(size_t)col * D + row] : s[(size_t)row * D + col];
                }
        }
    }

    // weights, as far as they are the same in every chunk
    float wp[16], wi = 0.f, wu[16];
    if constexpr (!SUM) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int gap = l32 - perm_index(r >> 3, hh, r & 7);
            wp[r] = gap >= 0 ? job.p * fast_exp2(e2 * gap) : 0.f;
        }
        wi = job.w * fast_exp2(e2 * (l32 + lead));
    }
    const auto update_weights = [&](int n) {
#pragma unroll
        for (int r = 0; r < 16; ++r) wu[r] = job.m * fast_exp2(e2 * max(n - lead - perm_index(r >> 3, hh, r & 7), 0));
    };
    update_weights(32);
    float fade = fast_exp2(e2 * 32.f);
    int e_state = 0, e_p = 0, e_z = 0;    // fp16: of the state as an operand, of P, of the weighted z (the accumulators hold C 2^-e_z)

    if constexpr (D < 32) {       // the columns that no load ever writes
        for (int q = tid; q < T::BUFFERS * 3 * T::BYTES / 16; q += T::THREADS) reinterpret_cast<u32x4 *>(lds)[q] = u32x4{0, 0, 0, 0};
        __syncthreads();
    }

    u32x4 px[SUM ? 1 : T::PIECES], py[T::PIECES], pz[T::PIECES];
    const auto load = [&](int t0) {
#pragma unroll
        for (int i = 0; i < T::PIECES; ++i) {
            const int q = tid + i * T::THREADS, t = t0 + q / T::ROW_PIECES;
            const int tc = min(t, t_end - 1);
            const size_t off = (base + tok_off(a.ts, reverse ? len - 1 - tc : tc)) * T::ES + q % T::ROW_PIECES * 16;
            if constexpr (!SUM) px[i] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(job.x) + off);
            py[i] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(job.y) + off);
            pz[i] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(job.z) + off);
            if (t >= t_end) {
                if constexpr (!SUM) px[i] = u32x4{0, 0, 0, 0};
                py[i] = u32x4{0, 0, 0, 0};
                pz[i] = u32x4{0, 0, 0, 0};
            }
        }
    };
    if (t_begin < t_end) load(t_begin);
    int buf = 0;
    for (int t0 = t_begin; t0 < t_end; t0 += 32) {
        char *const tx = lds + buf * 3 * T::BYTES, *const ty = tx + T::BYTES, *const tz = ty + T::BYTES;
        if constexpr (T::BUFFERS == 1) __syncthreads();
#pragma unroll
        for (int i = 0; i < T::PIECES; ++i) {
            const int q = tid + i * T::THREADS, at = q / T::ROW_PIECES * T::ROW + q % T::ROW_PIECES * 16;
            if constexpr (!SUM) *reinterpret_cast<u32x4 *>(tx + at) = px[i];
            *reinterpret_cast<u32x4 *>(ty + at) = py[i];
            *reinterpret_cast<u32x4 *>(tz + at) = pz[i];
        }
        __syncthreads();
        if (t0 + 32 < t_end) load(t0 + 32);
        if (t0 + 32 > t_end) {
            update_weights(t_end - t0);
            fade = fast_exp2(e2 * (t_end - t0));
        }

        const Frag<DT> zc[2] = {col_frag<DT, D>(tz, wave, 0, lane), col_frag<DT, D>(tz, wave, 1, lane)};
        if constexpr (!SUM) {
            float scale_state = 1.f;
            if constexpr (F16) {
                float largest = 0.f;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int r = 0; r < 16; ++r) largest = fmaxf(largest, fabsf(acc[ct][r]));
                fit_exponent(e_state, largest);
                scale_state = ldexpf(1.f, -e_state);
            }
            f32x16 p = splat16(0.f), o = splat16(0.f);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const Frag<DT> xf = row_frag<DT, D>(tx, l32, s, hh), yf = row_frag<DT, D>(ty, l32, s, hh);
                p = mma<DT>(yf, xf, p);
                float c8[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) c8[e] = F16 ? acc[s >> 1][8 * (s & 1) + e] * scale_state : acc[s >> 1][8 * (s & 1) + e];
                o = mma<DT>(pack8<DT>(c8), xf, o);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) p[r] *= wp[r];
            float scale_o = wi, scale_out = 1.f;
            if constexpr (F16) {
                float largest = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) largest = fmaxf(largest, fabsf(p[r]));
                fit_exponent(e_p, largest);
                const float down = ldexpf(1.f, -e_p);
#pragma unroll
                for (int r = 0; r < 16; ++r) p[r] *= down;
                scale_o = ldexpf(wi, e_state + e_z - e_p);
                scale_out = ldexpf(1.f, e_p);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) o[r] *= scale_o;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                float p8[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) p8[e] = p[8 * ks + e];
                o = mma<DT>(zc[ks], pack8<DT>(p8), o);
            }
            const int t = t0 + l32;
            if (t < t_end) {
                char *const row = static_cast<char *>(job.out) +
                                  (base + tok_off(a.ts, reverse ? len - 1 - t : t) + 32 * wave) * T::ES;
#pragma unroll
                for (int g = 0; g < (D < 32 ? 2 : 4); ++g) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = F16 ? o[4 * g + e] * scale_out : o[4 * g + e];
                    if constexpr (DT == FLARE_F32) {
                        *reinterpret_cast<float4 *>(row + (8 * g + 4 * hh) * 4) = make_float4(v[0], v[1], v[2], v[3]);
                    } else {
                        u32x2 w;
                        w[0] = pack_elems<F16>(v[0], v[1]);
                        w[1] = pack_elems<F16>(v[2], v[3]);
                        *reinterpret_cast<u32x2 *>(row + (8 * g + 4 * hh) * 2) = w;
                    }
                }
            }
        }
        float weighted[16], fade_acc = fade;
#pragma unroll
        for (int r = 0; r < 16; ++r) weighted[r] = elem_of<DT>(zc[r >> 3], r & 7) * wu[r];
        if constexpr (F16) {
            float largest = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) largest = fmaxf(largest, fabsf(weighted[r]));
            const int before = e_z;
            fit_exponent(e_z, largest);
            fade_acc = ldexpf(fade, before - e_z);
            const float down = ldexpf(1.f, -e_z);
#pragma unroll
            for (int r = 0; r < 16; ++r) weighted[r] *= down;
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[ct][r] *= fade_acc;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            float left[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) left[e] = weighted[8 * ks + e];
            Frag<DT> plane[T::PLANES];
#pragma unroll
            for (int k = 0; k < T::PLANES; ++k) {
                plane[k] = pack8<DT>(left);
#pragma unroll
                for (int e = 0; e < 8; ++e) left[e] -= elem_of<DT>(plane[k], e);
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const Frag<DT> yc = col_frag<DT, D>(ty, ct, ks, lane);
#pragma unroll
                for (int k = 0; k < T::PLANES; ++k) acc[ct] = mma<DT>(yc, plane[k], acc[ct]);
            }
        }
        if constexpr (T::BUFFERS == 2) buf ^= 1;
    }

    float *dst = nullptr;
    if constexpr (SUM) dst = a.slots + slot;
    else if (job.last && t_begin + a.seg_len >= len) dst = job.last + (size_t)bh * (D * D);
    if (dst && col < D) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = 32 * ct + perm_index(r >> 3, hh, r & 7);
                if (D >= 32 || row < D) dst[(size_t)row * D + col] = F16 ? ldexpf(acc[ct][r], e_z) : acc[ct][r];
            }
    }
}

// Segments' sums -> the state before each segment, in place: thread = four neighbouring entries of a state.
__global__ __launch_bounds__(256) void decay_carry_kernel(const ScanArgs a, int d)
{
    const int dd = d * d, tiles = (dd / 4 + 255) / 256;
    const int i = 4 * (blockIdx.x % tiles * 256 + threadIdx.x), jbh = blockIdx.x / tiles;
    if (i >= dd) return;
    const int bh = jbh % a.BH, jb = jbh / a.BH;
    const ScanJob &job = a.job[jb];
    const int len = item_length(a.lengths, bh / a.H, a.N);
    const int used = (len + a.seg_len - 1) / a.seg_len;
    const float fade = fast_exp2(decay_log2(a.log_decay[bh % a.H]) * (float)a.seg_len);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (job.first) {
        const float *f = job.first + (size_t)bh * dd;
        if (job.first_turned) {
            const int row = i / d, col = i % d;
            s = make_float4(f[(size_t)col * d + row], f[(size_t)(col + 1) * d + row], f[(size_t)(col + 2) * d + row],
                            f[(size_t)(col + 3) * d + row]);
        } else {
            s = *reinterpret_cast<const float4 *>(f + i);
        }
    }
    float *slot = a.slots + (size_t)jbh * a.segments * dd + i;
    for (int g = 0; g < max(used, 1); ++g, slot += dd) {
        float4 u = make_float4(0.f, 0.f, 0.f, 0.f);
        if (g + 1 < used) u = *reinterpret_cast<const float4 *>(slot);
        *reinterpret_cast<float4 *>(slot) = s;
        s = make_float4(fmaf(s.x, fade, u.x), fmaf(s.y, fade, u.y), fmaf(s.z, fade, u.z), fmaf(s.w, fade, u.w));
    }
}

// ---- one token -------------------------------------------------------------------------------------------------
template <int DT>
__device__ __forceinline__ float load_elem(const void *p, size_t i)
{
    if constexpr (DT == FLARE_F32) return static_cast<const float *>(p)[i];
    else return elem_value<DT == FLARE_F16>(static_cast<const uint16_t *>(p)[i]);
}
template <int DT>
__device__ __forceinline__ void store_elem(void *p, size_t i, float x)
{
    if constexpr (DT == FLARE_F32) static_cast<float *>(p)[i] = x;
    else static_cast<uint16_t *>(p)[i] = (uint16_t)rne_elem<DT == FLARE_F16>(x);
}
// Workgroup = (b,h) and a block of COLS columns of its state.  A thread owns four columns and every (256 / (COLS/4))-th
// row; all of its rows are requested before the first is used.
template <int DT, int D, int COLS>
__global__ __launch_bounds__(256) void decay_step_kernel(const void *q, const void *k, const void *v, const float *log_decay,
                                                         const int *active, const float *state_in, float *state_out, void *o,
                                                         float scale, int H)
{
    constexpr int LANES = COLS / 4, GROUPS = 256 / LANES, ROWS = (D + GROUPS - 1) / GROUPS;
    __shared__ float sum[GROUPS][COLS];
    const int bh = blockIdx.x / (D / COLS), c0 = blockIdx.x % (D / COLS) * COLS;
    const int c = threadIdx.x % LANES * 4, g = threadIdx.x / LANES;
    const size_t row = (size_t)bh * D, at = row * D + c0 + c;
    const bool on = !active || active[bh / H] > 0;
    float4 s[ROWS];
    float qr[ROWS], kr[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = min(g + i * GROUPS, D - 1);
        s[i] = *reinterpret_cast<const float4 *>(state_in + at + (size_t)r * D);
        qr[i] = load_elem<DT>(q, row + r);
        kr[i] = load_elem<DT>(k, row + r);
    }
    float vc[4], acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e) vc[e] = load_elem<DT>(v, row + c0 + c + e);
    const float fade = fast_exp2(decay_log2(log_decay[bh % H]));
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = g + i * GROUPS;
        if (r < D) {
            float4 t = s[i];
            if (on) t = make_float4(fmaf(kr[i], vc[0], fade * t.x), fmaf(kr[i], vc[1], fade * t.y), fmaf(kr[i], vc[2], fade * t.z),
                                    fmaf(kr[i], vc[3], fade * t.w));
            *reinterpret_cast<float4 *>(state_out + at + (size_t)r * D) = t;
            acc[0] = fmaf(qr[i], t.x, acc[0]);
            acc[1] = fmaf(qr[i], t.y, acc[1]);
            acc[2] = fmaf(qr[i], t.z, acc[2]);
            acc[3] = fmaf(qr[i], t.w, acc[3]);
        }
    }
    *reinterpret_cast<float4 *>(&sum[g][c]) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    __syncthreads();
    if (threadIdx.x < COLS) {
        float total = 0.f;
#pragma unroll 8
        for (int i = 0; i < GROUPS; ++i) total += sum[i][threadIdx.x];
        store_elem<DT>(o, row + c0 + threadIdx.x, on ? scale * total : 0.f);
    }
}

TokStride decay_stride(const flare_decay_shape &s)
{
    const long long H = s.H, N = s.N, d = s.d;
    if (s.layout == FLARE_BNHD) return TokStride{N * H * d, d, H * d, 0};
    return TokStride{H * N * d, N * d, d, 0};
}
struct DecayPlan { int segments, seg_len; };
DecayPlan decay_plan(const flare_decay_shape &s, int jobs)
{
    const long long waves = (s.d < 32 ? 1 : s.d / 32) * (long long)s.B * s.H * jobs;
    long long want = (2048 + waves - 1) / waves;
    const long long most = (s.N + 255) / 256;
    if (want > most) want = most;
    if (want < 1) want = 1;
    const long long len = ((s.N + want - 1) / want + 31) / 32 * 32;
    return DecayPlan{(int)((s.N + len - 1) / len), (int)len};
}
size_t slot_bytes(const flare_decay_shape &s, int jobs)
{
    const DecayPlan p = decay_plan(s, jobs);
    return p.segments > 1 ? (size_t)jobs * s.B * s.H * p.segments * s.d * s.d * 4 : 0;
}

template <int DT, int D>
int run_scan(const flare_decay_shape &s, ScanArgs &a, int jobs, int kid, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.BH * (long long)a.segments), jobs);
    if (a.segments > 1) {
        {
            LaunchTimer timer(KID_DECAY_SUM, stream);
            decay_scan_kernel<DT, D, true><<<grid, Tile<DT, D>::THREADS, 0, stream>>>(a);
        }
        LaunchTimer timer(KID_DECAY_CARRY, stream);
        decay_carry_kernel<<<(D * D / 4 + 255) / 256 * a.BH * jobs, 256, 0, stream>>>(a, D);
    }
    LaunchTimer timer(kid, stream);
    decay_scan_kernel<DT, D, false><<<grid, Tile<DT, D>::THREADS, 0, stream>>>(a);
    return check_launch();
}
template <int DT>
int run_scan_d(const flare_decay_shape &s, ScanArgs &a, int jobs, int kid, hipStream_t stream)
{
    switch (s.d) {
        case 16: return run_scan<DT, 16>(s, a, jobs, kid, stream);
        case 32: return run_scan<DT, 32>(s, a, jobs, kid, stream);
        case 64: return run_scan<DT, 64>(s, a, jobs, kid, stream);
        case 128: return run_scan<DT, 128>(s, a, jobs, kid, stream);
        default: return FLARE_EUNSUPPORTED;
    }
}
int run_scan_any(const flare_decay_shape &s, ScanArgs &a, int jobs, int kid, const float *log_decay, const int *lengths, void *ws,
                 hipStream_t stream)
{
    const DecayPlan p = decay_plan(s, jobs);
    a.log_decay = log_decay;
    a.lengths = lengths;
    a.slots = static_cast<float *>(ws);
    a.ts = decay_stride(s);
    a.H = s.H;
    a.N = s.N;
    a.BH = s.B * s.H;
    a.segments = p.segments;
    a.seg_len = p.seg_len;
    switch (s.dtype) {
        case FLARE_F32: return run_scan_d<FLARE_F32>(s, a, jobs, kid, stream);
        case FLARE_BF16: return run_scan_d<FLARE_BF16>(s, a, jobs, kid, stream);
        default: return run_scan_d<FLARE_F16>(s, a, jobs, kid, stream);
    }
}

template <int DT, int D>
int run_step(const flare_decay_shape &s, const void *q, const void *k, const void *v, const float *log_decay, const int *active,
             const float *state_in, float *state_out, void *o, float scale, hipStream_t stream)
{
    const int BH = s.B * s.H;
    constexpr int NARROW = D < 32 ? D : 32;
    LaunchTimer timer(KID_DECAY_STEP, stream);
    if (D > 32 && BH >= 512)
        decay_step_kernel<DT, D, D><<<BH, 256, 0, stream>>>(q, k, v, log_decay, active, state_in, state_out, o, scale, s.H);
    else
        decay_step_kernel<DT, D, NARROW><<<BH * (D / NARROW), 256, 0, stream>>>(q, k, v, log_decay, active, state_in, state_out, o,
                                                                               scale, s.H);
    return check_launch();
}
template <int DT>
int run_step_d(const flare_decay_shape &s, const void *q, const void *k, const void *v, const float *log_decay, const int *active,
               const float *state_in, float *state_out, void *o, float scale, hipStream_t stream)
{
    switch (s.d) {
        case 16: return run_step<DT, 16>(s, q, k, v, log_decay, active, state_in, state_out, o, scale, stream);
        case 32: return run_step<DT, 32>(s, q, k, v, log_decay, active, state_in, state_out, o, scale, stream);
        case 64: return run_step<DT, 64>(s, q, k, v, log_decay, active, state_in, state_out, o, scale, stream);
        case 128: return run_step<DT, 128>(s, q, k, v, log_decay, active, state_in, state_out, o, scale, stream);
        default: return FLARE_EUNSUPPORTED;
    }
}

}  // namespace

size_t decay_fwd_bytes(const flare_decay_shape &s) { return slot_bytes(s, 1); }
size_t decay_bwd_bytes(const flare_decay_shape &s) { return slot_bytes(s, 3); }

int decay_forward(const flare_decay_shape &s, const void *q, const void *k, const void *v, const float *log_decay,
                  const int *lengths, const float *state_in, void *o, float *state_out, float scale, void *ws,
                  hipStream_t stream)
{
    ScanArgs a{};
    a.job[0] = ScanJob{q, k, v, o, state_in, state_out, scale, scale, 1.f, 0, 0};
    return run_scan_any(s, a, 1, KID_DECAY_FORWARD, log_decay, lengths, ws, stream);
}

int decay_backward(const flare_decay_shape &s, const void *q, const void *k, const void *v, const float *log_decay,
                   const int *lengths, const float *state_in, const void *d_o, const float *dstate_out, void *dq, void *dk,
                   void *dv, float *dstate_in, float scale, void *ws, hipStream_t stream)
{
    ScanArgs a{};
    a.job[0] = ScanJob{d_o, v, k, dq, state_in, nullptr, scale, scale, 1.f, 0, 1};
    a.job[1] = ScanJob{v, d_o, q, dk, dstate_out, nullptr, scale, 1.f, scale, 1, 1};
    a.job[2] = ScanJob{k, q, d_o, dv, dstate_out, dstate_in, scale, 1.f, scale, 1, 0};
    return run_scan_any(s, a, 3, KID_DECAY_BACKWARD, log_decay, lengths, ws, stream);
}

int decay_step(const flare_decay_shape &s, const void *q, const void *k, const void *v, const float *log_decay, const int *active,
               const float *state_in, float *state_out, void *o, float scale, hipStream_t stream)
{
    switch (s.dtype) {
        case FLARE_F32: return run_step_d<FLARE_F32>(s, q, k, v, log_decay, active, state_in, state_out, o, scale, stream);
        case FLARE_BF16: return run_step_d<FLARE_BF16>(s, q, k, v, log_decay, active, state_in, state_out, o, scale, stream);
        default: return run_step_d<FLARE_F16>(s, q, k, v, log_decay, active, state_in, state_out, o, scale, stream);
    }
}

}  // namespace flare
