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
//   O^T = C^T X^T          the state's accumulators, rounded, are the A operand as they lie
//   O^T += Z^T P^T         likewise P^T's accumulators are the B operand: a contraction index in accumulator order
//   C   += Y^T (weight Z)  Y and Z read down their columns (transposing LDS reads), Y's columns in the order that makes the
//                          state's registers eight neighbouring rows (state_row)
// so that nothing but the token tiles passes through LDS.  These come by direct loads into LDS, two or three chunks ahead.
// dK and dV share their four tiles: a workgroup of theirs has waves in two roles.
//
// Where (b,h) are too few to fill the chip the tokens are cut into segments: a first pass takes each segment's own sum, a
// second turns the sums into the states before the segments, a third is the scan.
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

// What a wave does: which of the loaded tiles it takes for x, y and z, and where its states and results go.
struct Role {
    void *out;
    const float *first;    // state before the first token, [B][H][d][d], or NULL (zero)
    float *last;           // state behind the last token, or NULL
    int turned;            // `first` and the slots hold the transposed state
};
struct ScanArgs {
    const void *in[2][4];     // the tiles of either job (two jobs only where segments are summed)
    Role role[2];
    float p, w, m[2];         // see above; m of either job
    int reverse[2];           // tokens from the last to the first (then lead = 0)
    const float *log_decay;   // [H]
    const int *lengths;       // [B] or NULL
    float *slots;             // [job][B*H][segments][d][d]: a segment's own sum, then the state before it
    TokStride ts;
    int H, N, BH, segments, seg_len;
};

// SUM: a segment's own sum (tiles y, z); FORWARD: one role (x, y, z), also dQ; DKDV: two (q, k, v, dO).
enum ScanKind { SUM = 0, FORWARD = 1, DKDV = 2 };

template <int DT, int D, int KIND>
struct Scan {
    static constexpr int CT = D < 32 ? 1 : D / 32;                 // blocks of 32 columns (and of 32 rows of the state)
    static constexpr int ROLES = KIND == DKDV ? 2 : 1, TILES = KIND == SUM ? 2 : KIND == FORWARD ? 3 : 4;
    static constexpr int WAVES = CT * ROLES, THREADS = 64 * WAVES;
    static constexpr int ES = DT == FLARE_F32 ? 4 : 2;
    static constexpr int ROW = D * ES, BYTES = 32 * ROW, SET = TILES * BYTES;
    static constexpr int PIECES = ROW / 16;                        // of a row
    static constexpr int TILE_LOADS = BYTES / 1024;                // wave-wide loads of a tile; those of all tiles go round the waves
    static constexpr int LOADS = TILES * TILE_LOADS / WAVES;       // and so many of them are each wave's
    // Chunks held in LDS: as many as leave room for eight waves on a CU, two at least, four at most.
    static constexpr int FIT = 160 * 1024 / (SET * (WAVES < 8 ? 8 / WAVES : 1));
    static constexpr int STAGES = FIT < 2 ? 2 : FIT > 4 ? 4 : FIT;
    static constexpr int STORES = KIND == SUM ? 0 : (D < 32 ? 1 : 2) * (ES / 2);   // of a wave, each full chunk
    static constexpr int PER_SIMD = WAVES * (160 * 1024 / (STAGES * SET)) >= 8 ? 2 : 1;   // waves (fp32, d = 128: one)
    static_assert(TILES * TILE_LOADS % WAVES == 0 && STAGES * SET <= 160 * 1024, "");
};

// One head's decay in log2 units per token.  (Far below what fp32 weights resolve it makes no difference, and 0 * inf would.)
__device__ __forceinline__ float decay_log2(float g) { return g <= 0.f ? fmaxf(g * kLog2e, -3000.f) : __builtin_nanf(""); }
__device__ __forceinline__ int item_length(const int *lengths, int b, int N) { return lengths ? min(max(lengths[b], 0), N) : N; }

// l^n for a factor that is applied again and again: the two fp32 numbers around it, of which `next` gives the one that takes
// the product of all factors so far back towards the exact power.  (One of them alone is off by up to 2^-25, always the same
// way: 2^-18 after a hundred chunks.)
struct Fade {
    float up, down, err_up, err_down, drift;
    __device__ __forceinline__ Fade(float g, int n)
    {
        const double exact = g <= 0.f ? exp(fmax((double)g, -2080.0) * n) : (double)__builtin_nanf("");
        up = down = (float)exact;
        if ((double)up < exact) up = __uint_as_float(__float_as_uint(up) + 1);
        else if ((double)down > exact) down = __uint_as_float(__float_as_uint(down) - 1);
        err_up = exact > 0.0 ? (float)((double)up / exact - 1.0) : 0.f;
        err_down = exact > 0.0 ? (float)((double)down / exact - 1.0) : 0.f;
        drift = 0.f;
    }
    __device__ __forceinline__ float next()
    {
        const bool high = drift < 0.f;
        drift += high ? err_up : err_down;
        return high ? up : down;
    }
};

// Rows lie in LDS one behind the other (the direct loads write 1024 bytes in lane order), so that a column would lie in few
// banks: the 16-byte pieces of row r change places, piece c lying at c ^ swizzle(r).  Sixteen rows of a 16-byte read, and four
// rows of a transposing one, then lie in different banks.
template <int ROW>
__device__ __forceinline__ int swizzle(int r)
{
    if constexpr (ROW >= 256) return (r & 7) << 1 | (r >> 3 & 1);
    else if constexpr (ROW == 128) return (r >> 1 & 3) << 1 | (r >> 3 & 1);
    else if constexpr (ROW == 64) return r >> 2 & 3;
    else return r >> 3 & 1;
}
template <int ROW>
__device__ __forceinline__ const char *piece_at(const char *tile, int r, int c) { return tile + r * ROW + ((c ^ swizzle<ROW>(r)) << 4); }

// Row `row`, columns 16 s + 8 hh + 0..7
template <int DT, int D>
__device__ __forceinline__ Frag<DT> row_frag(const char *tile, int row, int s, int hh)
{
    constexpr int ROW = D * (DT == FLARE_F32 ? 4 : 2);
    Frag<DT> f;
    if constexpr (DT == FLARE_F32) {
        const float4 a = *reinterpret_cast<const float4 *>(piece_at<ROW>(tile, row, 4 * s + 2 * hh)),
                     b = *reinterpret_cast<const float4 *>(piece_at<ROW>(tile, row, 4 * s + 2 * hh + 1));
        f.v[0] = a.x; f.v[1] = a.y; f.v[2] = a.z; f.v[3] = a.w;
        f.v[4] = b.x; f.v[5] = b.y; f.v[6] = b.z; f.v[7] = b.w;
    } else {
        f.w = *reinterpret_cast<const u32x4 *>(piece_at<ROW>(tile, row, 2 * s + hh));
    }
    return f;
}
// Row m of the A operand Y^T is this column of Y: accumulator register r of the product then holds row
// 16 (r/8) + 8 hh + r % 8 of the state, eight neighbours for each step of 16 (what row_frag reads).
__device__ __forceinline__ int state_col(int m) { return (m & 16) + 8 * (m >> 2 & 1) + 4 * (m >> 3 & 1) + (m & 3); }
__device__ __forceinline__ int state_row(int ct, int r, int hh) { return 32 * ct + 16 * (r >> 3) + 8 * hh + (r & 7); }
// 32 columns from 32 * ct, 8 tokens of step ks in accumulator order: lane % 32 = column, or (STATE) row of Y^T as above
template <int DT, int D, bool STATE>
__device__ __forceinline__ Frag<DT> col_frag(const char *tile, int ct, int ks, int lane)
{
    constexpr int ROW = D * (DT == FLARE_F32 ? 4 : 2);
    Frag<DT> f;
    if constexpr (DT == FLARE_F32) {
        int c = lane & 31;
        if constexpr (STATE) c = state_col(c);
        if constexpr (D < 32) c &= 15;
        const int t = 16 * ks + 4 * (lane >> 5);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = *reinterpret_cast<const float *>(piece_at<ROW>(tile, t + 8 * (e >> 2) + (e & 3), 8 * ct + (c >> 2)) + 4 * (c & 3));
            f.v[e] = D < 32 && (lane & 16) ? 0.f : x;
        }
    } else {
        const int g = lane >> 4, q = lane & 15, pc = q & 3, t = 16 * ks + 4 * (g >> 1) + (q >> 2);
        const int block = D < 32 ? 0 : 4 * ct + 2 * (g & 1);
        const int c = block + (STATE ? pc & 1 : pc >> 1), at = 8 * (STATE ? pc >> 1 : pc & 1);
        const u32x2 a = lds_read_tr16(reinterpret_cast<const uint16_t *>(piece_at<ROW>(tile, t, c) + at));
        const u32x2 b = lds_read_tr16(reinterpret_cast<const uint16_t *>(piece_at<ROW>(tile, t + 8, c) + at));
        f.w[0] = a[0]; f.w[1] = a[1]; f.w[2] = b[0]; f.w[3] = b[1];
        if (D < 32 && (g & 1)) f.w = u32x4{0, 0, 0, 0};      // d = 16: the upper half of the block is not there
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

// EXACT: the state is an output.  PLANES of the weighted z: what the state sums is then good to 2^-22 (fp16) or 2^-24 (bf16)
// of a term; otherwise, as it only meets x rounded to 16 bits, to 2^-16 with bf16.
template <int DT, int D, int KIND, bool EXACT>
__global__ __launch_bounds__((Scan<DT, D, KIND>::THREADS), (Scan<DT, D, KIND>::PER_SIMD)) void decay_scan_kernel(const ScanArgs a)
{
    using T = Scan<DT, D, KIND>;
    constexpr int STEPS = D / 16, CT = T::CT;
    constexpr bool F16 = DT == FLARE_F16;
    constexpr int PLANES = DT == FLARE_F32 ? 1 : DT == FLARE_BF16 && EXACT ? 3 : 2;
    __shared__ __align__(1024) char lds[T::STAGES * T::SET];
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = wave % CT, which = wave / CT;
    // Neighbouring heads of a segment on one XCD (workgroups go round the eight): with [B][N][H][d] their rows share lines.
    const int total = a.BH * a.segments, each = gridDim.x >> 3, work = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
    if (work >= total) return;
    const int seg = work / a.BH, bh = work % a.BH, h = bh % a.H, job = blockIdx.y;
    const Role &role = a.role[which];
    const bool reverse = a.reverse[job] != 0;
    const int lead = reverse ? 0 : 1;
    const int len = item_length(a.lengths, bh / a.H, a.N);
    const int t_begin = seg * a.seg_len, t_end = min(t_begin + a.seg_len, len);
    const size_t base = tok_base(a.ts, bh, a.H);
    const float g = a.log_decay[h], e2 = decay_log2(g);

    if constexpr (KIND == SUM) {
        if (t_begin + a.seg_len >= len) return;       // nobody reads the sum of the last segment
    } else {
        // rows of the padding
        const int z0 = max(t_begin, len), z1 = min(t_begin + a.seg_len, a.N);
        for (int q = tid % (64 * CT); q < (z1 - z0) * T::PIECES; q += 64 * CT)
            *reinterpret_cast<u32x4 *>(static_cast<char *>(role.out) + (base + tok_off(a.ts, z0 + q / T::PIECES)) * T::ES +
                                       q % T::PIECES * 16) = u32x4{0, 0, 0, 0};
        if (seg != 0 && t_begin >= len) return;
    }

    // ---- loads of a chunk: 16 bytes a lane, 1024 a wave, straight into LDS ----
    const unsigned row_bytes = (unsigned)a.ts.sn * T::ES;
    const auto offset_of = [&](int i, int valid) {      // of load i, from the chunk's first row in memory
        const int q = (i * T::WAVES + wave) % T::TILE_LOADS * 64 + lane, r = q / T::PIECES;
        const int c = (q % T::PIECES) ^ swizzle<T::ROW>(r), rc = min(r, valid - 1);   // behind the end: the last row again
        return (unsigned)(reverse ? 31 - rc : rc) * row_bytes + 16 * c;
    };
    unsigned offset[T::LOADS];
#pragma unroll
    for (int i = 0; i < T::LOADS; ++i) offset[i] = offset_of(i, 32);
    const auto load = [&](int t0, int stage) {
        const int n0 = reverse ? len - 32 - t0 : t0, valid = t_end - t0;
        const long long at = ((long long)base + (long long)n0 * (long long)a.ts.sn) * T::ES;
#pragma unroll
        for (int i = 0; i < T::LOADS; ++i) {
            const int k = i * T::WAVES + wave;
            const char *src = static_cast<const char *>(a.in[job][k / T::TILE_LOADS]) + at;
            const unsigned off = valid >= 32 ? offset[i] : offset_of(i, valid);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(src + off),
                                             (__attribute__((address_space(3))) void *)(lds + stage * T::SET + k * 1024), 16, 0, 0);
        }
    };
    const int chunks = t_begin < t_end ? (t_end - t_begin + 31) / 32 : 0;
#pragma unroll
    for (int i = 0; i < T::STAGES - 1; ++i)
        if (i < chunks) load(t_begin + 32 * i, i);

    // the state before the segment: column 32 part + l32
    f32x16 acc[CT];
    const int col = 32 * part + l32;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[ct] = splat16(0.f);
    const size_t slot = (((size_t)job * a.BH + bh) * a.segments + seg) * (D * D);
    if constexpr (KIND != SUM) {
        const float *s = a.segments > 1 ? a.slots + slot : role.first ? role.first + (size_t)bh * (D * D) : nullptr;
        if (s && col < D) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = state_row(ct, r, hh);
                    if (D >= 32 || row < D) acc[ct][r] = role.turned ? s[(size_t)col * D + row] : s[(size_t)row * D + col];
                }
        }
    }

    // weights, as far as they are the same in every chunk
    float wp[16], wi = 0.f, wu[16];
    if constexpr (KIND != SUM) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int gap = l32 - perm_index(r >> 3, hh, r & 7);
            wp[r] = gap >= 0 ? a.p * fast_exp2(e2 * gap) : 0.f;
        }
        wi = a.w * fast_exp2(e2 * (l32 + lead));
    }
    const auto update_weights = [&](int n) {       // (a token behind the end weighs nothing)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int u = perm_index(r >> 3, hh, r & 7);
            wu[r] = u < n ? a.m[job] * fast_exp2(e2 * (n - lead - u)) : 0.f;
        }
    };
    update_weights(32);
    Fade fade(g, 32);
    int e_state = 0, e_p = 0, e_z = 0;    // fp16: of the state as an operand, of P, of the weighted z (the accumulators hold C 2^-e_z)

    // tiles of this wave's role
    constexpr int X = KIND == FORWARD ? 0 : -1, Y = KIND == SUM ? 0 : KIND == FORWARD ? 1 : -1, Z = KIND == SUM ? 1 : KIND == FORWARD ? 2 : -1;
    const int x_at = (KIND == DKDV ? (which ? 1 : 2) : X) * T::BYTES, y_at = (KIND == DKDV ? (which ? 0 : 3) : Y) * T::BYTES,
              z_at = (KIND == DKDV ? (which ? 3 : 0) : Z) * T::BYTES;

    int stage = 0;
    for (int i = 0; i < chunks; ++i) {
        const int t0 = t_begin + 32 * i;
        // This wave's part of chunk i is there when no more is on its way than what was asked for behind it: the loads of
        // STAGES - 2 chunks, and the stores of the chunks since (full ones; the barrier makes it everyone's part).  Its own reads
        // of chunk i - 1 have returned.
        if (i + T::STAGES - 1 > chunks) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        else if (i < T::STAGES - 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((T::STAGES - 2) * T::LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((T::STAGES - 2) * T::LOADS + (T::STAGES - 1) * T::STORES) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // (everyone is done with chunk i - 1, whose place this takes)
        if (i + T::STAGES - 1 < chunks) load(t0 + 32 * (T::STAGES - 1), stage == 0 ? T::STAGES - 1 : stage - 1);
        const char *const set = lds + stage * T::SET;
        const char *const tx = set + x_at, *const ty = set + y_at, *const tz = set + z_at;
        const int valid = t_end - t0;
        float faded = fade.next();
        if (valid < 32) {
            update_weights(valid);
            faded = fast_exp2(e2 * valid);
        }

        const Frag<DT> zc[2] = {col_frag<DT, D, false>(tz, part, 0, lane), col_frag<DT, D, false>(tz, part, 1, lane)};
        if constexpr (KIND != SUM) {
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
                char *const row = static_cast<char *>(role.out) +
                                  (base + tok_off(a.ts, reverse ? len - 1 - t : t) + 32 * part) * T::ES;
                if constexpr (F16) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[r] *= scale_out;
                }
                if constexpr (DT == FLARE_F32) {
#pragma unroll
                    for (int q = 0; q < (D < 32 ? 2 : 4); ++q)
                        *reinterpret_cast<float4 *>(row + (8 * q + 4 * hh) * 4) =
                            make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
                } else {
                    // register group q holds columns 8 q + 4 hh + 0..3: the halves of the wave trade groups, for 16 bytes a lane
#pragma unroll
                    for (int q = 0; q < (D < 32 ? 1 : 2); ++q) {
                        u32x4 w;
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const auto both = __builtin_amdgcn_permlane32_swap(pack_elems<F16>(o[8 * q + 2 * k], o[8 * q + 2 * k + 1]),
                                                                               pack_elems<F16>(o[8 * q + 4 + 2 * k], o[8 * q + 5 + 2 * k]),
                                                                               false, false);
                            w[k] = both[0];
                            w[2 + k] = both[1];
                        }
                        *reinterpret_cast<u32x4 *>(row + (16 * q + 8 * hh) * 2) = w;
                    }
                }
            }
        }
        float weighted[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) weighted[r] = elem_of<DT>(zc[r >> 3], r & 7) * wu[r];
        if constexpr (F16) {
            float largest = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) largest = fmaxf(largest, fabsf(weighted[r]));
            const int before = e_z;
            fit_exponent(e_z, largest);
            faded = ldexpf(faded, before - e_z);
            const float down = ldexpf(1.f, -e_z);
#pragma unroll
            for (int r = 0; r < 16; ++r) weighted[r] *= down;
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[ct][r] *= faded;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            float left[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) left[e] = weighted[8 * ks + e];
            Frag<DT> plane[PLANES];
#pragma unroll
            for (int k = 0; k < PLANES; ++k) {
                plane[k] = pack8<DT>(left);
#pragma unroll
                for (int e = 0; e < 8; ++e) left[e] -= elem_of<DT>(plane[k], e);
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const Frag<DT> yc = col_frag<DT, D, true>(ty, ct, ks, lane);
#pragma unroll
                for (int k = 0; k < PLANES; ++k) acc[ct] = mma<DT>(yc, plane[k], acc[ct]);
            }
        }
        stage = stage + 1 == T::STAGES ? 0 : stage + 1;
    }

    float *dst = nullptr;
    if constexpr (KIND == SUM) dst = a.slots + slot;
    else if (role.last && t_begin + a.seg_len >= len) dst = role.last + (size_t)bh * (D * D);
    if (dst && col < D) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = state_row(ct, r, hh);
                if (D >= 32 || row < D) dst[(size_t)row * D + col] = F16 ? ldexpf(acc[ct][r], e_z) : acc[ct][r];
            }
    }
}

// Segments' sums -> the state before each segment, in place: thread = four neighbouring entries of a state.
struct CarryArgs {
    const float *first[2];   // state before the first token of either job, or NULL
    int turned[2];
    const float *log_decay;
    const int *lengths;
    float *slots;
    int H, N, BH, segments, seg_len, d;
};
__global__ __launch_bounds__(256) void decay_carry_kernel(const CarryArgs a)
{
    const int d = a.d, dd = d * d, tiles = (dd / 4 + 255) / 256;
    const int i = 4 * (blockIdx.x % tiles * 256 + threadIdx.x), jbh = blockIdx.x / tiles;
    if (i >= dd) return;
    const int bh = jbh % a.BH, jb = jbh / a.BH;
    const int len = item_length(a.lengths, bh / a.H, a.N);
    const int used = (len + a.seg_len - 1) / a.seg_len;
    Fade fade(a.log_decay[bh % a.H], a.seg_len);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.first[jb]) {
        const float *f = a.first[jb] + (size_t)bh * dd;
        if (a.turned[jb]) {
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
        const float f = fade.next();
        s = make_float4(fmaf(s.x, f, u.x), fmaf(s.y, f, u.y), fmaf(s.z, f, u.z), fmaf(s.w, f, u.w));
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
// How the tokens are cut.  The slots of a forward pass are one job's, of a backward pass two (S and its gradient).
struct DecayPlan { int segments, seg_len; };
DecayPlan decay_plan(const flare_decay_shape &s, bool backward)
{
    const long long waves = (s.d < 32 ? 1 : s.d / 32) * (long long)s.B * s.H;
    long long want = (2048 + waves - 1) / waves;
    const long long most = (s.N + 255) / 256;
    if (want > most) want = most;
    if (want < 1) want = 1;
    const long long len = ((s.N + want - 1) / want + 31) / 32 * 32;
    return DecayPlan{(int)((s.N + len - 1) / len), (int)len};
}
size_t slot_bytes(const flare_decay_shape &s, bool backward)
{
    const DecayPlan p = decay_plan(s, backward);
    return p.segments > 1 ? (size_t)(backward ? 2 : 1) * s.B * s.H * p.segments * s.d * s.d * 4 : 0;
}

// What the host knows of a call, whatever its type and d.
struct DecayCall {
    const flare_decay_shape *s;
    const void *q, *k, *v, *d_o;
    const float *log_decay;
    const int *lengths;
    const float *state_in, *dstate_out;
    void *o, *dq, *dk, *dv;
    float *state_out, *dstate_in;
    float scale;
    float *slots;
    hipStream_t stream;
};
ScanArgs scan_args(const DecayCall &c, const DecayPlan &p)
{
    ScanArgs a{};
    a.log_decay = c.log_decay;
    a.lengths = c.lengths;
    a.slots = c.slots;
    a.ts = decay_stride(*c.s);
    a.H = c.s->H;
    a.N = c.s->N;
    a.BH = c.s->B * c.s->H;
    a.segments = p.segments;
    a.seg_len = p.seg_len;
    return a;
}
template <int DT, int D, int KIND>
void launch_scan(const ScanArgs &a, int jobs, bool exact, int kid, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.BH * (long long)a.segments + 7) / 8 * 8), jobs);
    LaunchTimer timer(kid, stream);
    if (exact && DT == FLARE_BF16)       // (the other types make no difference)
        decay_scan_kernel<DT, D, KIND, DT == FLARE_BF16><<<grid, Scan<DT, D, KIND>::THREADS, 0, stream>>>(a);
    else
        decay_scan_kernel<DT, D, KIND, false><<<grid, Scan<DT, D, KIND>::THREADS, 0, stream>>>(a);
}
void launch_carry(const DecayCall &c, const DecayPlan &p, int jobs, const float *first0, int turned0, const float *first1)
{
    CarryArgs a{};
    a.first[0] = first0;
    a.first[1] = first1;
    a.turned[0] = turned0;
    a.log_decay = c.log_decay;
    a.lengths = c.lengths;
    a.slots = c.slots;
    a.H = c.s->H;
    a.N = c.s->N;
    a.BH = c.s->B * c.s->H;
    a.segments = p.segments;
    a.seg_len = p.seg_len;
    a.d = c.s->d;
    LaunchTimer timer(KID_DECAY_CARRY, c.stream);
    decay_carry_kernel<<<(a.d * a.d / 4 + 255) / 256 * a.BH * jobs, 256, 0, c.stream>>>(a);
}

struct ForwardPass {
    template <int DT, int D>
    static int run(const DecayCall &c)
    {
        const DecayPlan p = decay_plan(*c.s, false);
        const bool exact = c.state_out != nullptr;
        if (p.segments > 1) {
            ScanArgs a = scan_args(c, p);
            a.in[0][0] = c.k;
            a.in[0][1] = c.v;
            a.m[0] = 1.f;
            launch_scan<DT, D, SUM>(a, 1, exact, KID_DECAY_SUM, c.stream);
            launch_carry(c, p, 1, c.state_in, 0, nullptr);
        }
        ScanArgs a = scan_args(c, p);
        a.in[0][0] = c.q;
        a.in[0][1] = c.k;
        a.in[0][2] = c.v;
        a.role[0] = Role{c.o, c.state_in, c.state_out, 0};
        a.p = a.w = c.scale;
        a.m[0] = 1.f;
        launch_scan<DT, D, FORWARD>(a, 1, exact, KID_DECAY_FORWARD, c.stream);
        return check_launch();
    }
};
struct BackwardPass {
    template <int DT, int D>
    static int run(const DecayCall &c)
    {
        const DecayPlan p = decay_plan(*c.s, true);
        const bool exact = c.dstate_in != nullptr;
        if (p.segments > 1) {
            // job 0: the transposed S (rows by v), forwards; job 1: its gradient (rows by q), backwards
            ScanArgs a = scan_args(c, p);
            a.in[0][0] = c.v;
            a.in[0][1] = c.k;
            a.in[1][0] = c.q;
            a.in[1][1] = c.d_o;
            a.m[0] = 1.f;
            a.m[1] = c.scale;
            a.reverse[1] = 1;
            launch_scan<DT, D, SUM>(a, 2, exact, KID_DECAY_SUM, c.stream);
            launch_carry(c, p, 2, c.state_in, 1, c.dstate_out);
        }
        const bool slots = p.segments > 1;
        ScanArgs a = scan_args(c, p);
        a.in[0][0] = c.d_o;
        a.in[0][1] = c.v;
        a.in[0][2] = c.k;
        a.role[0] = Role{c.dq, c.state_in, nullptr, slots ? 0 : 1};
        a.p = a.w = c.scale;
        a.m[0] = 1.f;
        launch_scan<DT, D, FORWARD>(a, 1, false, KID_DECAY_DQ, c.stream);
        a = scan_args(c, p);
        a.in[0][0] = c.q;
        a.in[0][1] = c.k;
        a.in[0][2] = c.v;
        a.in[0][3] = c.d_o;
        a.role[0] = Role{c.dk, c.dstate_out, nullptr, 1};            // x = v, y = dO, z = q
        a.role[1] = Role{c.dv, c.dstate_out, c.dstate_in, 0};        // x = k, y = q, z = dO
        a.p = c.scale;
        a.w = 1.f;
        a.m[0] = c.scale;
        a.reverse[0] = 1;
        if (slots) a.slots += (size_t)a.BH * p.segments * D * D;
        launch_scan<DT, D, DKDV>(a, 1, exact, KID_DECAY_DKDV, c.stream);
        return check_launch();
    }
};
template <typename Pass, int DT>
int run_pass_d(const DecayCall &c)
{
    switch (c.s->d) {
        case 16: return Pass::template run<DT, 16>(c);
        case 32: return Pass::template run<DT, 32>(c);
        case 64: return Pass::template run<DT, 64>(c);
        case 128: return Pass::template run<DT, 128>(c);
        default: return FLARE_EUNSUPPORTED;
    }
}
template <typename Pass>
int run_pass(const DecayCall &c)
{
    switch (c.s->dtype) {
        case FLARE_F32: return run_pass_d<Pass, FLARE_F32>(c);
        case FLARE_BF16: return run_pass_d<Pass, FLARE_BF16>(c);
        default: return run_pass_d<Pass, FLARE_F16>(c);
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

size_t decay_fwd_bytes(const flare_decay_shape &s) { return slot_bytes(s, false); }
size_t decay_bwd_bytes(const flare_decay_shape &s) { return slot_bytes(s, true); }

int decay_forward(const flare_decay_shape &s, const void *q, const void *k, const void *v, const float *log_decay,
                  const int *lengths, const float *state_in, void *o, float *state_out, float scale, void *ws,
                  hipStream_t stream)
{
    DecayCall c{};
    c.s = &s;
    c.q = q;
    c.k = k;
    c.v = v;
    c.log_decay = log_decay;
    c.lengths = lengths;
    c.state_in = state_in;
    c.o = o;
    c.state_out = state_out;
    c.scale = scale;
    c.slots = static_cast<float *>(ws);
    c.stream = stream;
    return run_pass<ForwardPass>(c);
}

int decay_backward(const flare_decay_shape &s, const void *q, const void *k, const void *v, const float *log_decay,
                   const int *lengths, const float *state_in, const void *d_o, const float *dstate_out, void *dq, void *dk,
                   void *dv, float *dstate_in, float scale, void *ws, hipStream_t stream)
{
    DecayCall c{};
    c.s = &s;
    c.q = q;
    c.k = k;
    c.v = v;
    c.d_o = d_o;
    c.log_decay = log_decay;
    c.lengths = lengths;
    c.state_in = state_in;
    c.dstate_out = dstate_out;
    c.dq = dq;
    c.dk = dk;
    c.dv = dv;
    c.dstate_in = dstate_in;
    c.scale = scale;
    c.slots = static_cast<float *>(ws);
    c.stream = stream;
    return run_pass<BackwardPass>(c);
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
