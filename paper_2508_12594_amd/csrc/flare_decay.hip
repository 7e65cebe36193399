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
//   O^T = C^T X^T          the state's accumulators, as two numbers of 16 bits, are the A operand as they lie
//   O^T += Z^T P^T         likewise P^T's accumulators are the B operand: a contraction index in accumulator order
//   C   += Y^T (weight Z)  Y and Z read down their columns (transposing LDS reads), Y's columns in the order that makes the
//                          state's registers eight neighbouring rows (state_row)
// so that nothing but the token tiles passes through LDS.  These come by direct loads into LDS, one to three chunks ahead.
// dK and dV share their four tiles: up to d = 64 a workgroup of theirs has waves in two roles.
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
    const void *in[2][4];     // the tiles of either job
    int jobs;                 // 2: neighbouring workgroups of an XCD take one job each (dK and dV, which share tiles)
    Role role[2];
    float p, w, m;            // see above
    int reverse;              // tokens from the last to the first (then lead = 0)
    int whole;                // (sums) of the last segment too: the state behind it is asked for
    const float *log_decay;   // [H]
    const int *lengths;       // [B] or NULL
    float *slots;             // [B*H][segments][d][d]: a segment's own sum, then the state before it
    TokStride ts;
    int H, N, BH, segments, seg_len;
};

constexpr float kSlow = 0x1p-16f;

// SUM: a segment's own sum (tiles y, z); FORWARD: one role (x, y, z), also dQ, and dK and dV as two jobs; DKDV: two roles
// (q, k, v, dO), d < 128.
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
    // Chunks held in LDS: as many as leave room for eight waves on a CU, at most four (the sums, which have least to do with a
    // chunk; dK and dV).  Scans of three tiles need no more than two: 127 us, 142 with three
    // (16 heads, 32768 tokens, d = 128, bf16).  What hides a load is the other waves: the compiler takes an LDS read and a direct load
    // for possibly the same bytes, and lets a wave wait for all its loads before a chunk's first read.  Stages as arrays of
    // their own, with the code once for each, take that wait out of every other chunk, and registers with it (with operands of one
    // number): 256 x 4096 tokens, d = 32, 53 -> 52 us; fp32, d = 64, 16 x 10007, 68 -> 64; d = 128 spills, 118 -> 119.  So there is
    // one array.
    static constexpr int FIT = 160 * 1024 / (SET * (WAVES < 8 ? 8 / WAVES : 1));
    static constexpr int STAGES = FIT <= 2 || KIND == FORWARD ? 2 : FIT > 4 ? 4 : FIT;
    static constexpr int STORES = (D < 32 ? 1 : 2) * (ES / 2);   // of a wave, each full chunk
    static constexpr int GROUP = ROW >= 256 ? 1 : 256 / ROW;       // heads side by side in 256 bytes
    static constexpr int PER_SIMD = WAVES * (160 * 1024 / (STAGES * SET)) >= 8 ? 2 : 1;   // waves (fp32, d = 128: one)
    static_assert(TILES * TILE_LOADS % WAVES == 0 && STAGES * SET <= 160 * 1024, "");
};

// One head's decay in log2 units per token.  (Far below what fp32 weights resolve it makes no difference, and 0 * inf would.)
__device__ __forceinline__ float decay_log2(float g) { return g <= 0.f ? fmaxf(g * kLog2e, -3000.f) : __builtin_nanf(""); }
__device__ __forceinline__ int item_length(const int *lengths, int b, int N) { return lengths ? min(max(lengths[b], 0), N) : N; }

// A value that is the same in all lanes, in a scalar register
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
// l^n
__device__ __forceinline__ double exact_decay(float g, int n)
{
    return g <= 0.f ? exp(fmax((double)g, -2080.0) * n) : (double)__builtin_nanf("");
}
// l^n for a factor that is applied again and again: the two fp32 numbers around it, of which `next` gives the one that takes
// the product of all factors so far back towards the exact power.  (One of them alone is off by up to 2^-25, always the same
// way: 2^-18 after a hundred chunks.)
struct Fade {
    float up, down, err_up, err_down, drift;
    __device__ __forceinline__ Fade(float g, int n)
    {
        const double exact = exact_decay(g, n);
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
__device__ __forceinline__ const char *piece_at(const char *tile, int r, int c)
{
    return tile + r * ROW + ((c ^ swizzle<ROW>(r)) << 4);
}

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
            const char *const at = piece_at<ROW>(tile, t + 8 * (e >> 2) + (e & 3), 8 * ct + (c >> 2)) + 4 * (c & 3);
            const float x = *reinterpret_cast<const float *>(at);
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
// gradients lie among the subnormals.  The exponent is kept from chunk to chunk, and moves in steps of 12 (every step leads
// into the 13 octaves, so that at most one direction is taken).
constexpr int kExponentStep = 12;
// 0 where `largest` (already scaled) is fit for fp16, else the step that its exponent has to take
__device__ __forceinline__ int exponent_step(float largest, int e)
{
    if (e < 96 && __any(largest > 32768.f)) return kExponentStep;
    if (e > -96 && !__any(largest > 4.f) && __any(largest > 0.f)) return -kExponentStep;
    return 0;
}
template <int N>
__device__ __forceinline__ float largest_of(const f32x16 (&v)[N])
{
    float largest = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) largest = fmaxf(largest, fabsf(v[i][r]));
    return largest;
}
// Scales v until it is fit, or until what it is added to (whose largest magnitude, before that, is `held`) would come near the end of
// fp32 (what is lost then is 2^-80 of that); returns the factor it took.
template <int N, typename Held>
__device__ __forceinline__ float fit_exponent(float (&v)[N], int &e, const Held &held)
{
    float took = 1.f;
    for (;;) {
        float largest = 0.f;
#pragma unroll
        for (int r = 0; r < N; ++r) largest = fmaxf(largest, fabsf(v[r]));
        const int step = exponent_step(largest, e);
        if (step == 0 || (step < 0 && __any(held() * took > 0x1p84f))) return took;
        e += step;
        const float by = step > 0 ? 1.f / (1 << kExponentStep) : (float)(1 << kExponentStep);
        took *= by;
#pragma unroll
        for (int r = 0; r < N; ++r) v[r] *= by;
    }
}

// Which (b,h) and segment a workgroup has.  Workgroups go round the eight XCDs: neighbouring heads whose rows share lines
// (with [B][N][H][d]) go to one.  In a padded batch the segments that hold tokens come first, or the workgroups that have
// anything to do would share some CUs and leave others empty (8 items of 0 to 4097 tokens, 16 heads, d = 128, fp16: sums and scan
// 201 us, 161 us like this).
struct Work { int bh, seg; bool none; int job; };
template <int GROUP>
__device__ __forceinline__ Work work_of(const ScanArgs &a)
{
    const int job = a.jobs == 2 ? blockIdx.x >> 3 & 1 : 0, turn = blockIdx.x >> (a.jobs == 2 ? 4 : 3);
    const int work = (turn / GROUP * 8 + (blockIdx.x & 7)) * GROUP + turn % GROUP;
    if (work >= a.BH * a.segments) return Work{0, 0, true, 0};
    // (with one segment each there is nothing to look for; with more (b,h) are few)
    if (!a.lengths || a.segments == 1) return Work{work % a.BH, work / a.BH, false, job};
    const int lane = threadIdx.x & 63, items = a.BH / a.H, h = work % a.H;
    int t = work / a.H;       // of the segments that hold tokens (the first of an empty item, too), then of the others
    for (int other = 0; other < 2; ++other) {
        for (int b0 = 0; b0 < items; b0 += 64) {
            const int b = b0 + lane;
            int used = 0;
            if (b < items) used = max((item_length(a.lengths, b, a.N) + a.seg_len - 1) / a.seg_len, 1);
            const int mine = b < items ? (other ? a.segments - used : used) : 0;
            int upto = mine;                   // of the items up to this one
#pragma unroll
            for (int s = 1; s < 64; s *= 2) {
                const int below = __shfl_up(upto, s);
                if (lane >= s) upto += below;
            }
            const unsigned long long here = __ballot(upto > t);
            if (here) {
                const int l = __ffsll(here) - 1;
                const int seg = t - (__shfl(upto, l) - __shfl(mine, l)) + (other ? __shfl(used, l) : 0);
                return Work{(b0 + __builtin_amdgcn_readfirstlane(l)) * a.H + h, __builtin_amdgcn_readfirstlane(seg), false, job};
            }
            t -= __shfl(upto, 63);
        }
    }
    return Work{0, 0, true, 0};                // (not reached: the two lists hold every segment)
}

// Loads of a chunk of tokens: 16 bytes a lane, 1024 a wave, straight into LDS, the loads of all tiles going round the waves.
template <typename T>
struct Loader {
    const ScanArgs &a;
    int job;
    long long base;          // element offset of the (b,h) slice
    int len, t_end, wave, lane;
    // (of a wave's loads, those of a tile lie like those of the next where the loads of a tile go evenly round the waves)
    static constexpr int OFFSETS = T::TILE_LOADS % T::WAVES == 0 ? T::TILE_LOADS / T::WAVES : T::LOADS;
    unsigned row_bytes, offset[OFFSETS];
    __device__ __forceinline__ Loader(const ScanArgs &args, int j, int bh, int length, int end, int w, int l)
        : a(args), job(j), base((long long)tok_base(args.ts, bh, args.H)), len(length), t_end(end), wave(w), lane(l),
          row_bytes((unsigned)args.ts.sn * T::ES)
    {
#pragma unroll
        for (int i = 0; i < OFFSETS; ++i) {
            const int q = place(i), r = q / T::PIECES, c = (q % T::PIECES) ^ swizzle<T::ROW>(r);
            offset[i] = (unsigned)(a.reverse ? 31 - r : r) * row_bytes + 16 * c;
        }
    }
    __device__ __forceinline__ int place(int i) const { return (i * T::WAVES + wave) % T::TILE_LOADS * 64 + lane; }
    // of load i, from the chunk's first row in memory
    __device__ __forceinline__ unsigned offset_of(int i, int valid) const
    {
        const unsigned off = offset[i % OFFSETS];
        if (valid >= 32) return off;
        const unsigned back = (unsigned)max(place(i) / T::PIECES - valid + 1, 0) * row_bytes;    // behind the end: the last row again
        return a.reverse ? off + back : off - back;
    }
    __device__ __forceinline__ void load(int t0, char *set) const
    {
        const int n0 = a.reverse ? len - 32 - t0 : t0, valid = t_end - t0;
        const long long at = (base + (long long)n0 * (long long)a.ts.sn) * T::ES;
#pragma unroll
        for (int i = 0; i < T::LOADS; ++i) {
            const int k = i * T::WAVES + wave;
            const char *src = static_cast<const char *>(a.in[job][k / T::TILE_LOADS]) + at;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(src + offset_of(i, valid)),
                                             (__attribute__((address_space(3))) void *)(set + k * 1024), 16, 0, 0);
        }
    }
};

// The bf16 (fp16) planes of 8 fp32 values: their sum is the value but for 2^-8 (2^-11) to the power of their number.
template <int DT, int PLANES>
__device__ __forceinline__ void split_planes(const float *x, Frag<DT> (&plane)[PLANES])
{
    float left[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) left[e] = x[e];
#pragma unroll
    for (int k = 0; k < PLANES; ++k) {
        plane[k] = pack8<DT>(left);
        if (k + 1 < PLANES) {
#pragma unroll
            for (int e = 0; e < 8; ++e) left[e] -= elem_of<DT>(plane[k], e);
        }
    }
}
template <int DT, bool EXACT>
constexpr int planes() { return DT == FLARE_F32 ? 1 : DT == FLARE_BF16 && EXACT ? 3 : 2; }
// ... of the weighted scores and of the state where it meets x: one alone would add as much to an output's error as the rounding of
// the output itself (bf16 2.3e-3 of the norm, 1.7e-3 with two).  The second costs 1 ... 5 % of a pass (16 heads of 131072 tokens, d = 128,
// forward 674 -> 682 us; 32 x 8 x 4096, d = 32, with its gradients 251 -> 259 us; 16 x 32768, d = 128, 639 -> 672 us), and 333 tokens of
// 8 heads, one chunk after the other, take 19.6 us for 16.4.
template <int DT>
constexpr int operand_planes() { return DT == FLARE_F32 ? 1 : 2; }

// A segment's own sum, into its slot: sum_u l^(n-u-lead) y_u z_u^T.  From the segment's last chunk to its first, so that its
// first tokens are the last to be read before the scan reads them again (256 MB of memory-side cache), and nothing has to be
// multiplied but the weights.  EXACT: the state behind the sequence is an output.
template <int DT, int D, bool EXACT>
__global__ __launch_bounds__((Scan<DT, D, SUM>::THREADS), 2) void decay_sum_kernel(const ScanArgs a)
{
    using T = Scan<DT, D, SUM>;
    constexpr int CT = T::CT, PLANES = planes<DT, EXACT>();
    constexpr bool F16 = DT == FLARE_F16;
    __shared__ __align__(1024) char lds[T::STAGES * T::SET];
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int part = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Work work = work_of<T::GROUP>(a);
    if (work.none) return;
    const int h = work.bh % a.H, lead = a.reverse ? 0 : 1, len = item_length(a.lengths, work.bh / a.H, a.N);
    const int t_begin = work.seg * a.seg_len, t_end = min(t_begin + a.seg_len, len);
    if (t_begin >= len || (t_end == len && !a.whole)) return;      // nothing there, or nobody asks for it
    const float g = a.log_decay[h], e2 = decay_log2(g);
    int chunks = (t_end - t_begin + 31) / 32;
    // What a token adds has 2^-64 of its weight left 64 halvings later, where fp32 sums no longer see it.
    const int first = e2 < 0.f ? max(0, chunks - 1 - (int)fminf(ceilf(-2.f / e2), 0x1p24f)) : 0;
    const Loader<T> loader(a, 0, work.bh, len, t_end, part, lane);
    chunks -= first;
    const int t_first = t_begin + 32 * first;
#pragma unroll
    for (int i = 0; i < T::STAGES - 1; ++i)
        if (i < chunks) loader.load(t_first + 32 * (chunks - 1 - i), lds + i * T::SET);

    f32x16 acc[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[ct] = splat16(0.f);
    float wu[16];
    const auto weights = [&](int n) {       // (a token behind the end weighs nothing)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int u = perm_index(r >> 3, hh, r & 7);
            wu[r] = u < n ? a.m * fast_exp2(e2 * (n - lead - u)) : 0.f;
        }
    };
    const int last_n = t_end - t_first - 32 * (chunks - 1);
    weights(last_n);
    Fade fade(g, 32);
    float behind = 1.f;                      // the decay of what lies behind the chunk
    int e_z = 0, stage = 0;                  // fp16: the accumulators hold the sum times down_z = 2^-e_z
    float down_z = 1.f;
    for (int i = 0; i < chunks; ++i) {
        if (i + T::STAGES - 1 > chunks) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((T::STAGES - 2) * T::LOADS) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (i + T::STAGES - 1 < chunks)
            loader.load(t_first + 32 * (chunks - T::STAGES - i), lds + (stage == 0 ? T::STAGES - 1 : stage - 1) * T::SET);
        const char *const ty = lds + stage * T::SET, *const tz = ty + T::BYTES;
        stage = stage + 1 == T::STAGES ? 0 : stage + 1;
        const Frag<DT> zc[2] = {col_frag<DT, D, false>(tz, part, 0, lane), col_frag<DT, D, false>(tz, part, 1, lane)};
        float weighted[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) weighted[r] = elem_of<DT>(zc[r >> 3], r & 7) * (wu[r] * (behind * down_z));
        if constexpr (F16) {
            const float took = fit_exponent(weighted, e_z, [&]() { return largest_of(acc); });
            if (took != 1.f) {
                down_z *= took;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[ct][r] *= took;
            }
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            Frag<DT> plane[PLANES];
            split_planes<DT, PLANES>(weighted + 8 * ks, plane);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const Frag<DT> yc = col_frag<DT, D, true>(ty, ct, ks, lane);
#pragma unroll
                for (int k = 0; k < PLANES; ++k) acc[ct] = mma<DT>(yc, plane[k], acc[ct]);
            }
        }
        if (i == 0 && last_n < 32) {
            behind = fast_exp2(e2 * last_n);
            weights(32);
        } else {
            behind *= fade.next();
        }
    }
    float *const dst = a.slots + ((size_t)work.bh * a.segments + work.seg) * (D * D);
    const int col = 32 * part + l32;
    if (col < D) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = state_row(ct, r, hh);
                if (D >= 32 || row < D) dst[(size_t)row * D + col] = F16 ? ldexpf(acc[ct][r], e_z) : acc[ct][r];
            }
    }
}

// The scan of a segment.  EXACT: its last state is an output (of one segment; of several it comes out of the sums).
template <int DT, int D, int KIND, bool EXACT>
__global__ __launch_bounds__((Scan<DT, D, KIND>::THREADS), (Scan<DT, D, KIND>::PER_SIMD)) void decay_scan_kernel(const ScanArgs a)
{
    using T = Scan<DT, D, KIND>;
    constexpr int STEPS = D / 16, CT = T::CT, PLANES = planes<DT, EXACT>(), OPERAND = operand_planes<DT>();
    constexpr bool F16 = DT == FLARE_F16;
    __shared__ __align__(1024) char lds[T::STAGES * T::SET];
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = wave % CT, which = wave / CT;
    const Work work = work_of<T::GROUP>(a);
    if (work.none) return;
    const int seg = work.seg, bh = work.bh, h = bh % a.H;
    const Role &role = a.role[KIND == DKDV ? which : work.job];
    const bool reverse = a.reverse != 0;
    const int lead = reverse ? 0 : 1;
    const int len = item_length(a.lengths, bh / a.H, a.N);
    const int t_begin = seg * a.seg_len, t_end = min(t_begin + a.seg_len, len);
    const size_t base = tok_base(a.ts, bh, a.H);
    const float g = a.log_decay[h], e2 = decay_log2(g);

    // rows of the padding
    const int z0 = max(t_begin, len), z1 = min(t_begin + a.seg_len, a.N);
    for (int q = tid % (64 * CT); q < (z1 - z0) * T::PIECES; q += 64 * CT)
        *reinterpret_cast<u32x4 *>(static_cast<char *>(role.out) + (base + tok_off(a.ts, z0 + q / T::PIECES)) * T::ES +
                                   q % T::PIECES * 16) = u32x4{0, 0, 0, 0};
    if (seg != 0 && t_begin >= len) return;

    const Loader<T> loader(a, work.job, bh, len, t_end, wave, lane);
    const int chunks = t_begin < t_end ? (t_end - t_begin + 31) / 32 : 0;
#pragma unroll
    for (int i = 0; i < T::STAGES - 1; ++i)
        if (i < chunks) loader.load(t_begin + 32 * i, lds + i * T::SET);

    // the state before the segment: column 32 part + l32
    f32x16 acc[CT];
    const int col = 32 * part + l32;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[ct] = splat16(0.f);
    {
        const float *s = a.slots ? a.slots + ((size_t)bh * a.segments + seg) * (D * D)
                                 : role.first ? role.first + (size_t)bh * (D * D) : nullptr;
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
    float wp[16], wu[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int gap = l32 - perm_index(r >> 3, hh, r & 7);
        wp[r] = gap >= 0 ? a.p * fast_exp2(e2 * gap) : 0.f;
    }
    const float wi = a.w * fast_exp2(e2 * (l32 + lead));
    const auto update_weights = [&](int n) {       // (a token behind the end weighs nothing)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int u = perm_index(r >> 3, hh, r & 7);
            wu[r] = u < n ? a.m * fast_exp2(e2 * (n - lead - u)) : 0.f;
        }
    };
    update_weights(32);
    Fade fade(g, 32);
    // of the last chunk, if that is a part of one, as two numbers: calls of a few tokens each apply the same one over and over
    const double part_exact = exact_decay(g, max(t_end - t_begin, 0) % 32);
    const float part_faded = uniform((float)part_exact), part_rest = uniform((float)(part_exact - (double)(float)part_exact));
    // The accumulators hold C / (f 2^e_z).  With slow decays f takes up the decay of the chunks, and is multiplied in where it has
    // become small, so that it is never below 2^-16; otherwise (a chunk leaves less than that) the accumulators themselves are
    // multiplied in each chunk.
    float f = 1.f;
    // fp16: exponents of the weighted z, of P (in wp too) and of the state as an operand
    int e_z = 0, e_p = 0, e_state = 0;
    float down_z = 1.f, down_state = 1.f;

    // tiles of this wave's role
    const int x_at = (KIND == FORWARD ? 0 : which ? 1 : 2) * T::BYTES, y_at = (KIND == FORWARD ? 1 : which ? 0 : 3) * T::BYTES,
              z_at = (KIND == FORWARD ? 2 : which ? 3 : 0) * T::BYTES;

    const auto fit_state = [&]() {
        if constexpr (F16) {
            const float largest = largest_of(acc);
            for (;;) {
                const int step = exponent_step(largest * down_state, e_state);
                if (step == 0) break;
                e_state += step;
                down_state = ldexpf(1.f, -e_state);
            }
        }
    };
    fit_state();
    // One chunk.  PLAIN: of 32 tokens, and slow decays.  The weighted z goes in planes: what the state sums is then good to 2^-22
    // (fp16) or 2^-24 (bf16) of a term; a state that is no output only goes into results of 16 bits, and 2^-16 will do with bf16.
    const auto chunk = [&](auto plain_tag, int t0, const char *set) {
        constexpr bool PLAIN = decltype(plain_tag)::value;
        const char *const tx = set + x_at, *const ty = set + y_at, *const tz = set + z_at;
        __builtin_amdgcn_s_setprio(1);       // (the waves of a SIMD then are less often in the same part)
        float faded = fade.next(), rest = 0.f;
        const bool partial = !PLAIN && t0 + 32 > t_end;
        if (partial) {
            update_weights(t_end - t0);
            faded = part_faded;
            rest = part_rest;
        }

        const Frag<DT> zc[2] = {col_frag<DT, D, false>(tz, part, 0, lane), col_frag<DT, D, false>(tz, part, 1, lane)};
        {
            f32x16 p = splat16(0.f), o = splat16(0.f);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const Frag<DT> xf = row_frag<DT, D>(tx, l32, s, hh), yf = row_frag<DT, D>(ty, l32, s, hh);
                p = mma<DT>(yf, xf, p);
                float c8[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) c8[e] = F16 ? acc[s >> 1][8 * (s & 1) + e] * down_state : acc[s >> 1][8 * (s & 1) + e];
                Frag<DT> plane[OPERAND];
                split_planes<DT, OPERAND>(c8, plane);
#pragma unroll
                for (int k = 0; k < OPERAND; ++k) o = mma<DT>(plane[k], xf, o);
            }
            float p16[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) p16[r] = p[r] * wp[r];
            float scale_o = wi * f, scale_out = 1.f;
            if constexpr (F16) {
                const float took = fit_exponent(p16, e_p, []() { return 0.f; });
                if (took != 1.f) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) wp[r] *= took;
                }
                scale_o = ldexpf(scale_o, e_state + e_z - e_p);
                scale_out = ldexpf(1.f, e_p);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) o[r] *= scale_o;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                Frag<DT> plane[OPERAND];
                split_planes<DT, OPERAND>(p16 + 8 * ks, plane);
#pragma unroll
                for (int k = 0; k < OPERAND; ++k) o = mma<DT>(zc[ks], plane[k], o);
            }
            const int t = t0 + l32;
            char *const row = static_cast<char *>(role.out) +
                              (base + tok_off(a.ts, reverse ? len - 1 - t : t) + 32 * part) * T::ES;
            if constexpr (F16) {
#pragma unroll
                for (int r = 0; r < 16; ++r) o[r] *= scale_out;
            }
            if constexpr (DT == FLARE_F32) {
#pragma unroll
                for (int q = 0; q < (D < 32 ? 2 : 4); ++q)
                    if (PLAIN || t < t_end)
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
                    if (PLAIN || t < t_end) *reinterpret_cast<u32x4 *>(row + (16 * q + 8 * hh) * 2) = w;
                }
            }
        }
        __builtin_amdgcn_s_setprio(0);
        sched_fence();
        if constexpr (PLAIN) f *= faded;
        float weighted[16];
        const float lift = PLAIN ? down_z / f : down_z;
#pragma unroll
        for (int r = 0; r < 16; ++r) weighted[r] = elem_of<DT>(zc[r >> 3], r & 7) * (PLAIN || F16 ? wu[r] * lift : wu[r]);
        if constexpr (F16) {
            const float took = fit_exponent(weighted, e_z, [&]() { return largest_of(acc); });
            if (took != 1.f) {
                down_z *= took;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[ct][r] *= took;
            }
        }
        if constexpr (!PLAIN) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[ct][r] = partial ? fmaf(acc[ct][r], faded, acc[ct][r] * rest) : acc[ct][r] * faded;
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            Frag<DT> plane[PLANES];
            split_planes<DT, PLANES>(weighted + 8 * ks, plane);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const Frag<DT> yc = col_frag<DT, D, true>(ty, ct, ks, lane);
#pragma unroll
                for (int k = 0; k < PLANES; ++k) acc[ct] = mma<DT>(yc, plane[k], acc[ct]);
            }
        }
        fit_state();
    };
    int i = 0, stage = 0;
    const auto next_chunk = [&]() {
        // This wave's part of chunk i is there when no more is on its way than what was asked for behind it: the loads of
        // STAGES - 2 chunks, and the stores of the chunks since (full ones; the barrier makes it everyone's part).  Its own
        // reads of chunk i - 1 have returned.
        if (i + T::STAGES - 1 > chunks) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        else if (i < T::STAGES - 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((T::STAGES - 2) * T::LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((T::STAGES - 2) * T::LOADS + (T::STAGES - 1) * T::STORES) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // (everyone is done with chunk i - 1, whose place this takes)
        if (i + T::STAGES - 1 < chunks)
            loader.load(t_begin + 32 * (i + T::STAGES - 1), lds + (stage == 0 ? T::STAGES - 1 : stage - 1) * T::SET);
        const char *const set = lds + stage * T::SET;
        stage = stage + 1 == T::STAGES ? 0 : stage + 1;
        return set;
    };
    const auto take_up = [&]() {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[ct][r] *= f;
        f = 1.f;
        fit_state();
    };
    if (fade.down >= kSlow) {
        const int full = t_begin < t_end ? (t_end - t_begin) / 32 : 0;
        for (; i < full; ++i) {
            const char *const set = next_chunk();
            if (f * fade.down < kSlow) take_up();
            chunk(PlainTag<true>{}, t_begin + 32 * i, set);
        }
        take_up();
    }
    for (; i < chunks; ++i) {
        const char *const set = next_chunk();
        chunk(PlainTag<false>{}, t_begin + 32 * i, set);
    }

    float *const dst = role.last ? role.last + (size_t)bh * (D * D) : nullptr;
    int here = lane;
    asm volatile("" : "+v"(here));      // (addresses formed anew, not kept over the chunks)
    const int to = 32 * part + (here & 31);
    if (dst && to < D) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = state_row(ct, r, here >> 5);
                if (D >= 32 || row < D) dst[(size_t)row * D + to] = F16 ? ldexpf(acc[ct][r], e_z) : acc[ct][r];
            }
    }
}

// Segments' sums -> the state before each segment, in place: thread = four neighbouring entries of a state.
struct CarryArgs {
    const float *first;      // state before the first token, or NULL
    float *last;             // state behind the last one, or NULL
    const float *log_decay;
    const int *lengths;
    float *slots;
    int H, N, BH, segments, seg_len, d;
};
__global__ __launch_bounds__(256) void decay_carry_kernel(const CarryArgs a)
{
    const int d = a.d, dd = d * d, tiles = (dd / 4 + 255) / 256;
    const int i = 4 * (blockIdx.x % tiles * 256 + threadIdx.x), bh = blockIdx.x / tiles;
    if (i >= dd) return;
    const int len = item_length(a.lengths, bh / a.H, a.N);
    const int used = (len + a.seg_len - 1) / a.seg_len, sums = a.last ? used : used - 1;
    const float g = a.log_decay[bh % a.H];
    // The sums are asked for AHEAD segments before they are added (the slots are written over behind).
    constexpr int AHEAD = 8;
    float *const slot = a.slots + (size_t)bh * a.segments * dd + i;
    float4 u[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
        if (k < sums) u[k] = *reinterpret_cast<const float4 *>(slot + (size_t)k * dd);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.first) s = *reinterpret_cast<const float4 *>(a.first + (size_t)bh * dd + i);
    Fade fade(g, a.seg_len);
    for (int g0 = 0; g0 < max(used, 1); g0 += AHEAD) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int at = g0 + k;
            if (at >= max(used, 1)) break;
            const float4 v = u[k];
            if (at + AHEAD < sums) u[k] = *reinterpret_cast<const float4 *>(slot + (size_t)(at + AHEAD) * dd);
            *reinterpret_cast<float4 *>(slot + (size_t)at * dd) = s;
            if (at < sums) {
                const float f = at + 1 < used ? fade.next() : fast_exp2(decay_log2(g) * (float)(len - at * a.seg_len));
                s = make_float4(fmaf(s.x, f, v.x), fmaf(s.y, f, v.y), fmaf(s.z, f, v.z), fmaf(s.w, f, v.w));
            }
        }
    }
    if (a.last) *reinterpret_cast<float4 *>(a.last + (size_t)bh * dd + i) = s;
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
    // l as two fp32 numbers: one alone is off by up to 2^-25, in every step the same way (16384 steps: 5e-4 of the oldest terms);
    // with both a step rounds its result and nothing else.
    const double exact = exact_decay(log_decay[bh % H], 1);
    const float fade = (float)exact, rest = (float)(exact - (double)fade);
    const auto next = [&](float old, float kr, float vc) { return fmaf(kr, vc, fmaf(old, fade, old * rest)); };
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = g + i * GROUPS;
        if (r < D) {
            float4 t = s[i];
            if (on) t = make_float4(next(t.x, kr[i], vc[0]), next(t.y, kr[i], vc[1]), next(t.z, kr[i], vc[2]), next(t.w, kr[i], vc[3]));
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
DecayPlan decay_plan(const flare_decay_shape &s, bool padded, bool backward)
{
    // As many segments as keep the scan's waves resident together (two on a SIMD; fp32 from d = 64 on: one, and at d = 32
    // the six that a CU's LDS has room for).  The backward's dK and dV are twice as many waves: from d = 64 on, and of fp32
    // from d = 32 on, half as many segments fill the chip.  (fp32, d = 32: 256 x 2048 tokens forward 110 us, 128 with segments
    // for eight waves a CU; 64 x 8192 backward 269 us with segments for four, 317 for eight; bf16, 256 x 4096, the backward's sums, dK
    // and dV: 138, 131.)
    const long long waves = (s.d < 32 ? 1 : s.d / 32) * (long long)s.B * s.H;
    const bool f32 = s.dtype == FLARE_F32;
    const long long room = f32 && s.d >= 32 ? (backward || s.d >= 64 ? 1024 : 1536) : backward && s.d >= 64 ? 1024 : 2048;
    // A padded batch holds about half of its tokens: twice as many segments, of which as many are empty.
    long long want = (padded ? 2 : 1) * room / waves;
    // Sums and carry cost two launches, about 13 us: as much as 9 to 12 chunks one after the other (fp32: 4).  And each segment costs
    // the carry 0.2 us, each chunk of a segment both passes 1.6 us and more: together least at about sqrt(5 N) tokens a segment.
    // (8 heads of 1000 tokens, d = 64, bf16, kernel times: 48 us in one, 34 us in segments of 256, 24 us in the 64 that this gives.)
    const long long least = (long long)(sqrt(5.0 * s.N) / 32.0 + 0.5) * 32;
    const long long most = s.N <= (f32 ? 128 : 384) ? 1 : (s.N + least - 1) / least;
    if (want > most) want = most;
    if (want < 1) want = 1;
    const long long len = ((s.N + want - 1) / want + 31) / 32 * 32;
    return DecayPlan{(int)((s.N + len - 1) / len), (int)len};
}
size_t slot_bytes(const flare_decay_shape &s, bool padded, bool backward)
{
    const DecayPlan p = decay_plan(s, padded, backward);
    return p.segments > 1 ? (size_t)s.B * s.H * p.segments * s.d * s.d * 4 : 0;
}

// What the host knows of a call, whatever its type and d.
struct DecayCall {
    const flare_decay_shape *s;
    const void *q, *k, *v, *d_o;
    const float *log_decay;
    const int *lengths;
    const float *state_in, *dstate_out, *marks_in;
    void *o, *dq, *dk, *dv;
    float *state_out, *dstate_in;
    float scale;
    float *slots;        // of the forward: its marks, if they are asked for
    hipStream_t stream;
};
ScanArgs scan_args(const DecayCall &c, const DecayPlan &p, const void *in0, const void *in1, const void *in2, const void *in3)
{
    ScanArgs a{};
    a.in[0][0] = in0;
    a.in[0][1] = in1;
    a.in[0][2] = in2;
    a.in[0][3] = in3;
    a.jobs = 1;
    a.log_decay = c.log_decay;
    a.lengths = c.lengths;
    a.ts = decay_stride(*c.s);
    a.H = c.s->H;
    a.N = c.s->N;
    a.BH = c.s->B * c.s->H;
    a.segments = p.segments;
    a.seg_len = p.seg_len;
    return a;
}
template <typename T>
unsigned scan_blocks(const ScanArgs &a)
{
    const long long round = 8 * T::GROUP;
    return (unsigned)((a.BH * (long long)a.segments + round - 1) / round * round * a.jobs);
}
template <int DT, int D, int KIND>
void launch_scan(const ScanArgs &a, bool exact, int kid, hipStream_t stream)
{
    using T = Scan<DT, D, KIND>;
    LaunchTimer timer(kid, stream);
    if (exact && DT == FLARE_BF16)       // (to the other types it makes no difference)
        decay_scan_kernel<DT, D, KIND, DT == FLARE_BF16><<<scan_blocks<T>(a), T::THREADS, 0, stream>>>(a);
    else
        decay_scan_kernel<DT, D, KIND, false><<<scan_blocks<T>(a), T::THREADS, 0, stream>>>(a);
}
// The states before the segments of the scan (x), y, z, into slots, and the state behind the last (or NULL).
template <int DT, int D>
void launch_states(const DecayCall &c, const DecayPlan &p, const void *y, const void *z, float m, bool reverse, const float *first,
                   float *last, float *slots)
{
    using T = Scan<DT, D, SUM>;
    ScanArgs a = scan_args(c, p, y, z, nullptr, nullptr);
    a.slots = slots;
    a.m = m;
    a.reverse = reverse;
    a.whole = last != nullptr;
    {
        LaunchTimer timer(KID_DECAY_SUM, c.stream);
        if (last && DT == FLARE_BF16) decay_sum_kernel<DT, D, DT == FLARE_BF16><<<scan_blocks<T>(a), T::THREADS, 0, c.stream>>>(a);
        else decay_sum_kernel<DT, D, false><<<scan_blocks<T>(a), T::THREADS, 0, c.stream>>>(a);
    }
    CarryArgs b{};
    b.first = first;
    b.last = last;
    b.log_decay = c.log_decay;
    b.lengths = c.lengths;
    b.slots = slots;
    b.H = a.H;
    b.N = a.N;
    b.BH = a.BH;
    b.segments = p.segments;
    b.seg_len = p.seg_len;
    b.d = D;
    LaunchTimer timer(KID_DECAY_CARRY, c.stream);
    decay_carry_kernel<<<(D * D / 4 + 255) / 256 * a.BH, 256, 0, c.stream>>>(b);
}

struct ForwardPass {
    template <int DT, int D>
    static int run(const DecayCall &c)
    {
        const DecayPlan p = decay_plan(*c.s, c.lengths != nullptr, false);
        const bool split = p.segments > 1;
        if (split) launch_states<DT, D>(c, p, c.k, c.v, 1.f, false, c.state_in, c.state_out, c.slots);
        ScanArgs a = scan_args(c, p, c.q, c.k, c.v, nullptr);
        a.slots = split ? c.slots : nullptr;
        a.role[0] = Role{c.o, c.state_in, split ? nullptr : c.state_out, 0};
        a.p = a.w = c.scale;
        a.m = 1.f;
        launch_scan<DT, D, FORWARD>(a, a.role[0].last != nullptr, KID_DECAY_FORWARD, c.stream);
        return check_launch();
    }
};
struct BackwardPass {
    template <int DT, int D>
    static int run(const DecayCall &c)
    {
        // dQ: cut as the forward is, from its states S (transposed: rows by v)
        DecayPlan p = decay_plan(*c.s, c.lengths != nullptr, false);
        bool split = p.segments > 1;
        const float *marks = c.marks_in;
        if (split && !marks) {
            launch_states<DT, D>(c, p, c.k, c.v, 1.f, false, c.state_in, nullptr, c.slots);
            marks = c.slots;
        }
        ScanArgs a = scan_args(c, p, c.d_o, c.v, c.k, nullptr);
        a.slots = split ? const_cast<float *>(marks) : nullptr;
        a.role[0] = Role{c.dq, c.state_in, nullptr, 1};
        a.p = a.w = c.scale;
        a.m = 1.f;
        launch_scan<DT, D, FORWARD>(a, false, KID_DECAY_DQ, c.stream);
        // dK and dV: from the gradient of S (rows by q), time running backwards
        p = decay_plan(*c.s, c.lengths != nullptr, true);
        split = p.segments > 1;
        if (split) launch_states<DT, D>(c, p, c.q, c.d_o, c.scale, true, c.dstate_out, c.dstate_in, c.slots);
        // x = v, y = dO, z = q and x = k, y = q, z = dO.  d = 128: as two workgroups side by side, which do not wait for each other
        // (16 heads of 32768 tokens: 226 us, 278 us in one; fp32 8 x 20000: 354, 342).  d < 128: as two roles in one workgroup, which
        // loads q and dO once (d = 64: 99 us, 109 us in two; fp32 d = 64, 16 x 10007: 89, 115; d = 32, 256 x 4096: 97, 107).
        const Role dk{c.dk, c.dstate_out, nullptr, 1}, dv{c.dv, c.dstate_out, split ? nullptr : c.dstate_in, 0};
        if constexpr (D == 128) {
            a = scan_args(c, p, c.v, c.d_o, c.q, nullptr);
            a.in[1][0] = c.k;
            a.in[1][1] = c.q;
            a.in[1][2] = c.d_o;
            a.jobs = 2;
        } else {
            a = scan_args(c, p, c.q, c.k, c.v, c.d_o);
        }
        a.slots = split ? c.slots : nullptr;
        a.role[0] = dk;
        a.role[1] = dv;
        a.p = c.scale;
        a.w = 1.f;
        a.m = c.scale;
        a.reverse = 1;
        launch_scan<DT, D, D == 128 ? FORWARD : DKDV>(a, dv.last != nullptr, KID_DECAY_DKDV, c.stream);
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
    // The blocks of a state all read the whole of q and k: o may lie over those only where one workgroup has them all (it reads them
    // before its barrier, and writes o behind it).
    const bool over = o == q || o == k;
    if (D > 32 && (BH >= 512 || over))
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

size_t decay_marks_bytes(const flare_decay_shape &s, bool padded) { return slot_bytes(s, padded, false); }
size_t decay_fwd_bytes(const flare_decay_shape &s, bool padded, bool marks) { return marks ? 0 : slot_bytes(s, padded, false); }
size_t decay_bwd_bytes(const flare_decay_shape &s, bool padded, bool marks)
{
    const size_t states = marks ? 0 : slot_bytes(s, padded, false), gradients = slot_bytes(s, padded, true);   // one after the other
    return states > gradients ? states : gradients;
}

int decay_forward(const flare_decay_shape &s, const void *q, const void *k, const void *v, const float *log_decay,
                  const int *lengths, const float *state_in, void *o, float *state_out, float *marks, float scale, void *ws,
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
    c.slots = marks ? marks : static_cast<float *>(ws);
    c.stream = stream;
    return run_pass<ForwardPass>(c);
}

int decay_backward(const flare_decay_shape &s, const void *q, const void *k, const void *v, const float *log_decay,
                   const int *lengths, const float *state_in, const float *marks, const void *d_o, const float *dstate_out,
                   void *dq, void *dk, void *dv, float *dstate_in, float scale, void *ws, hipStream_t stream)
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
    c.marks_in = marks;
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
