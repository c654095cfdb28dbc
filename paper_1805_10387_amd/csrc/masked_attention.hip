// Attention under interval masks, forward and backward, any length (paper Section 3.1 arithmetic; the softmax an fp32 part).
//
// One pass over the keys with a running maximum and sum: for a tile of keys S^T = K Q^T on the matrix cores, p = exp(s - max), and
// O^T = O^T exp(max_old - max) + V^T P; scores stay in registers.  Transposed throughout: a lane owns ONE query (column of S^T),
// so the row statistics are one register a lane, and the packed probabilities are the second operand of the next product without
// a move.  Backward recomputes the probabilities from the kept log-sum-exp: one kernel per tile of queries for dq, one per
// tile of keys for dk and dv, so that every gradient has one owner and no atomics (7 products instead of the 5 that one pass
// with atomics would take).
//
// Bound: the matrix cores and the vector work of the scores beside them for long rows; for short ones the chain of a workgroup's start
// (range, first tiles, first product: a kernel whose workgroups have one tile takes 5.5 us).  8 heads of 128 over 2, 12289 causal
// rows: forward (2 products) 358 to 374 us, backward 1220 to 1265, one call after the other; by the profiler, which holds launches apart,
// 389 us (0.80 PFLOP/s of the 1.19 that a library product of 8192^3 reaches here), dq (3 products) 496 (0.94), dk and dv (4) 803 (0.77).
// 16 heads of 64, 8192 rows in 15 documents: 50, 60 and 85 us by the profiler (0.30 PFLOP/s of what is visible, to which the tiles
// add 16 %).
// 32 x 32 tiles of 16 deep are the widest matrix instructions; 128 rows of own, 64 of the other side, and fragments of tiles in LDS
// (filled by loads that pass the registers by, one tile ahead) keep the operands of two tiles and the results in 256 registers; dk and dv
// of heads above 64 take 60 to 170 more, and so have one wave a SIMD.
//
// Masks: query r sees keys [lo, hi).  Whether a tile of pairs is empty, whole or neither follows from four numbers of a 64-row tile
// (least lo, greatest hi, greatest lo, least hi) that the mask keeps behind the rows' own; only tiles that are neither look at
// single pairs.
//
// What is hidden must not be felt, though 0 x NaN is NaN: scores of hidden pairs are replaced, not added to; and in tiles that are
// not whole, non-finite elements of the matrices that a zero probability would multiply are zeroed on their way into LDS.
// Those that are visible still show.  Forward, an element of v by a NaN score in its place (or by the product), one of q or k by what
// it makes of the score: q k^T is finite where both rows are (128 x 65504^2 is far from the end of fp32) and never where one is not, and
// an infinite score becomes NaN before a cap or an exponential could make something finite of it.  Backward because a query that sees one
// has a non-finite lse or delta, and its lse is made so low that its probabilities are infinite.
#include "attn_lds.hpp"
#include "mask_rule.hpp"

#include <limits.h>
#include <math.h>

namespace mp {

constexpr int   JOIN_THREADS = 256;
constexpr int   MA_Q       = 128;   // queries of a workgroup, 32 a wave (dk/dv: keys)
constexpr int   MA_K       = 64;    // keys of a tile (dk/dv: queries)
constexpr float LOG2E      = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float POISON = -3e38f;
constexpr float P_LOG2 = 10.f, P_SCALE = 1024.f;  // dv's probabilities: of 10^5 keys one has 10^-5, which fp16 has to three digits only

struct AttnArgs {
    const uint16_t *q, *k, *v, *ctx, *dctx;
    uint16_t *      out, *dq, *dk, *dv;
    float*          lse;                 // forward: out
    const float *   lse_in, *slopes;
    float *         lse2, *delta;        // backward: [n_heads, rows_pad]; delta twice, the second over P_SCALE
    float*          part;                // dk and dv of a part of a group's heads: [kv_heads * parts, rows_k, 2, d]
    const int2*     range;
    const int4*     tile;
    int             rows_q, rows_k, heads, group, part_heads, d, rows_pad;
    int             ld_q, ld_k, ld_v, ld_ctx, ld_dq, ld_dk, ld_dv, ld_dctx;
    float           alpha, cap;
};

// ------------------------------------------------------------------------------------------------ masks
// One wave per 64 rows.
__global__ __launch_bounds__(64) void mask_kernel(int rows, int rows_k, int n_docs, const int* __restrict__ start, const int* __restrict__ prefix,
                                                  int causal, int window, const int* __restrict__ los, const int* __restrict__ his,
                                                  int2* __restrict__ range, int4* __restrict__ tile) {
    const int r  = blockIdx.x * 64 + threadIdx.x;
    int       lo = 0, hi = 0;
    if (r < rows) {
        if (los) {
            lo = max(los[r], 0);
            hi = min(his[r], rows_k);
        } else if (n_docs > 0 && r >= start[0] && r < start[n_docs]) {
            int a = 0, b = n_docs;  // start[a] <= r < start[b]; seven places a trip to memory
            while (b - a > 1) {
                const int part = (b - a + 7) / 8;
                int       last = a;
#pragma unroll
                for (int i = 1; i < 8; ++i) {
                    const int c = min(a + part * i, b);
                    if (start[c] <= r) last = c;
                }
                b = min(last + part, b);
                a = last;
            }
            seen_in_document(r, max(start[a], 0), min(start[b], rows), causal, prefix != nullptr, prefix ? prefix[a] : 0, window, lo, hi);
        }
        if (lo >= hi) lo = hi = 0;
    }
    range[r]        = make_int2(lo, hi);  // (rows up to the next multiple of 64 too)
    const bool some = lo < hi;
    int        a = some ? lo : INT_MAX, b = some ? hi : 0, c = some ? lo : INT_MAX, d = some ? hi : 0;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        a = min(a, __shfl_xor(a, s, 64));
        b = max(b, __shfl_xor(b, s, 64));
        c = max(c, __shfl_xor(c, s, 64));
        d = min(d, __shfl_xor(d, s, 64));
    }
    if (threadIdx.x == 0) tile[blockIdx.x] = make_int4(a, b, c, d);
}

// ------------------------------------------------------------------------------------------------ scores
// What is done to q k^T: nothing but the scale (to base 2: one factor beside the exponential's), a distance bias, a cap, or both.
enum { PLAIN = 0, BIAS = 1, CAP = 2 };
// Scores in place, to base 2 once they are multiplied by unit(): a factor that costs nothing beside the exponential's.  Lanes own one
// index, registers the other; dist: query less key (or the reverse) at register 0.
// FWD: a score whose cap made it finite becomes NaN.  Backward leaves tanh where there is a cap, and a bias beside it to exponent().
template <int MODE, bool FWD>
__device__ __forceinline__ float unit(const AttnArgs& a) { return MODE == CAP || (MODE & CAP && !FWD) ? a.cap * LOG2E : MODE == PLAIN ? a.alpha * LOG2E : 1.f; }
template <int MODE, bool FWD>
__device__ __forceinline__ void scores(const AttnArgs& a, f32x16& s, float slope2, int dist) {
    if (MODE == PLAIN) return;
    const float k = MODE & CAP ? a.alpha / a.cap * (2.f * LOG2E) : a.alpha * LOG2E, c = a.cap * LOG2E, at = (float)dist;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        // tanh(x) = 1 - 2 / (exp(2x) + 1): an absolute error of 1e-7, which is what counts for a score
        if (MODE & CAP) s[r] = fmaf(-2.f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[r] * k) + 1.f), FWD ? fmaf(s[r], 0.f, 1.f) : 1.f);
        else s[r] *= k;
        if (MODE == (CAP | BIAS) && FWD) s[r] *= c;
        if (MODE == BIAS || (MODE & BIAS && FWD)) s[r] = fmaf(-slope2, fabsf(at + (float)(8 * (r >> 2) + (r & 3))), s[r]);
    }
}
// Backward: log2 of a probability (times P_SCALE) from what scores() left of register r.
template <int MODE>
__device__ __forceinline__ float exponent(float s, float c, float lse2, float slope2, float at, int r) {
    return fmaf(s, c, MODE == (CAP | BIAS) ? fmaf(-slope2, fabsf(at + (float)(8 * (r >> 2) + (r & 3))), -lse2) : -lse2);
}
// d s / d (alpha q k^T) = 1 - tanh^2; 0 for a hidden score's -inf.  (tanh out of a score that holds a bias as well would be off by that
// one's rounding over the cap.)
__device__ __forceinline__ float fade(float tanh) { return fmaxf(fmaf(-tanh, tanh, 1.f), 0.f); }

// ------------------------------------------------------------------------------------------------ tiles
__device__ __forceinline__ f32x16 zero16() { return f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }

// Rows of a result tile D[i = column][j = row], scaled, to memory: this lane's row, 16-byte pieces.
template <int DT>
__device__ __forceinline__ void store_rows(uint16_t* row, const f32x16 (&o)[DT], float scale, int d, int hf) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int    e = 8 * c;
            const u32x4m p = trade8(pack_f16(o[dt][e] * scale, o[dt][e + 1] * scale), pack_f16(o[dt][e + 2] * scale, o[dt][e + 3] * scale),
                                    pack_f16(o[dt][e + 4] * scale, o[dt][e + 5] * scale), pack_f16(o[dt][e + 6] * scale, o[dt][e + 7] * scale));
            const int col = 32 * dt + 16 * c + 8 * hf;
            if (row && col < d) *reinterpret_cast<u32x4m*>(row + col) = p;
        }
}

// What 128 queries see: of the workgroup, of this wave's 32 and of this lane's.
struct QueryRange {
    int lo, hi;
    int wlo, whi, wlo_max, whi_min;
    int glo, ghi, glo_max, ghi_min;
    __device__ __forceinline__ QueryRange(const AttnArgs& a, int m0, int m) {
        const int2 v = m < a.rows_q ? a.range[m] : make_int2(0, 0);
        lo           = max(v.x, 0);
        hi           = min(v.y, a.rows_k);
        if (lo >= hi) lo = hi = 0;
        int p = lo < hi ? lo : INT_MAX, q = hi, r = p, t = hi;
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
            p = min(p, __shfl_xor(p, s, 64));
            q = max(q, __shfl_xor(q, s, 64));
            r = max(r, __shfl_xor(r, s, 64));
            t = min(t, __shfl_xor(t, s, 64));
        }
        wlo = __builtin_amdgcn_readfirstlane(p), whi = __builtin_amdgcn_readfirstlane(q);
        wlo_max = __builtin_amdgcn_readfirstlane(r), whi_min = __builtin_amdgcn_readfirstlane(t);
        int4 x = a.tile[m0 / 64];
        if (m0 + 64 < a.rows_q) {
            const int4 y = a.tile[m0 / 64 + 1];
            x            = make_int4(min(x.x, y.x), max(x.y, y.y), max(x.z, y.z), min(x.w, y.w));
        } else {
            x.z = INT_MAX;  // rows behind the last one: not whole
        }
        // (where nothing is seen, x.x is the largest number there is, and tiles are counted on from glo; a mask may have been made for more
        // keys, and a tile that ends behind the last one is not whole)
        glo = __builtin_amdgcn_readfirstlane(min(max(x.x, 0), a.rows_k)), ghi = __builtin_amdgcn_readfirstlane(min(x.y, a.rows_k));
        glo_max = __builtin_amdgcn_readfirstlane(x.z), ghi_min = __builtin_amdgcn_readfirstlane(min(x.w, a.rows_k));
    }
    __device__ __forceinline__ bool whole(int kb) const { return glo_max <= kb && ghi_min >= kb + MA_K; }
    __device__ __forceinline__ bool none(int kb) const { return wlo >= kb + MA_K || whi <= kb; }
    __device__ __forceinline__ bool all(int kb) const { return wlo_max <= kb && whi_min >= kb + MA_K; }
};

// This lane's row of a matrix as second operands (zeros outside).
template <int KK>
__device__ __forceinline__ void row_frags(f16x8 (&f)[KK], const uint16_t* row, int d, int hf) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        u32x4m p = {0u, 0u, 0u, 0u};
        if (row && 16 * kk + 8 * hf < d) p = *reinterpret_cast<const u32x4m*>(row + 16 * kk + 8 * hf);
        f[kk] = frag8(p);
    }
}
// Fragments have come from memory here: otherwise the first use of them in a loop would wait for every load in flight, in each turn.
template <int KK>
__device__ __forceinline__ void settle(f16x8 (&f)[KK]) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(f[kk]));
}

__device__ __forceinline__ f32x16 mma(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f16x8  words(const unsigned (&w)[8], int e) { return frag8(u32x4m{w[e], w[e + 1], w[e + 2], w[e + 3]}); }
// A barrier behind which the loads of every wave have arrived.
__device__ __forceinline__ void arrive() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ void step() { __builtin_amdgcn_sched_barrier(0); }
template <int DT>
__device__ __forceinline__ bool finite(const f32x16 (&o)[DT]) {
    bool is = true;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) is = is && fabsf(o[dt][r]) < INFINITY;
    return is;
}
// Whether it holds for any lane of the workgroup.  Behind it everybody is through with the tiles in LDS.
__device__ __forceinline__ bool any_of_workgroup(bool it, int* vote) {
    if (threadIdx.x == 0) *vote = 0;
    lds_barrier();
    if (__any(it)) *vote = 1;
    lds_barrier();
    return __builtin_amdgcn_readfirstlane(*vote) != 0;
}

// ------------------------------------------------------------------------------------------------ forward
constexpr float LAZY = 8.f;  // the maximum that exponentials refer to follows when it is 2^8 behind

// 128 queries a workgroup, 32 a wave.  SPLIT: so many teams of four waves share the workgroup's tiles of keys in turn, each with buffers and
// sums of its own, and are joined at the end.
template <int D, int MODE, int SPLIT>
__global__ __launch_bounds__(256 * SPLIT, 2) void masked_fwd_kernel(AttnArgs a) {
    constexpr int KK = D / 16, DT = D / 32, ROWB = D <= 64 ? 128 : 256;
    constexpr unsigned SIZE = MA_K * ROWB;
    typedef TileLoad<ROWB, 4> Load;
    typedef LdsTile<ROWB>     Tile;
    __shared__ __align__(256) char tiles_of[SPLIT][2][2][SIZE];  // keys, values of two tiles
    __shared__ __align__(16) float bads[SPLIT][MA_K];

    const int tiles = (a.rows_q + MA_Q - 1) / MA_Q;
    const int h = blockIdx.x % a.heads, qt = tiles - 1 - blockIdx.x / a.heads, kvh = h / a.group;
    const int lane = threadIdx.x & 63, wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = wave8 & 3, team = wave8 >> 2, hf = lane >> 5;
    const int m0 = qt * MA_Q, m = m0 + 32 * wave + (lane & 31);
    const QueryRange x(a, m0, m);
    const uint16_t*  K = a.k + kvh * a.d;
    const uint16_t*  V = a.v + kvh * a.d;
    float*           bad = bads[team];
    Load             lk, lv;
    lk.init(a.ld_k, a.d, wave, lane);
    lv.init(a.ld_v, a.d, wave, lane);
    if (x.glo + MA_K * team < x.ghi) {
        lk.issue(K, a.ld_k, x.glo + MA_K * team, a.rows_k, a.d, tiles_of[team][0][0], wave);
        lv.issue(V, a.ld_v, x.glo + MA_K * team, a.rows_k, a.d, tiles_of[team][0][1], wave);
    }
    f16x8 qf[KK];
    row_frags<KK>(qf, m < a.rows_q ? a.q + (long long)m * a.ld_q + h * a.d : nullptr, a.d, hf);
    const float slope2 = MODE && a.slopes ? a.slopes[h] * LOG2E : 0.f;
    const float c      = unit<MODE, true>(a);  // scores to base 2
    f32x16      o[DT];
    float       ref = -INFINITY, sum = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = zero16();
    settle<KK>(qf);
    const unsigned at_k = lds_address(tiles_of[team][0][0]) + Tile::plain(lane), at_v = lds_address(tiles_of[team][0][1]) + Tile::across(lane);

    int b = 0;
    for (int k0 = x.glo; k0 < x.ghi; k0 += MA_K * SPLIT, b ^= 1) {
        const int kb = k0 + MA_K * team, next = kb + MA_K * SPLIT;
        arrive();
        if (next < x.ghi) {
            lk.issue(K, a.ld_k, next, a.rows_k, a.d, tiles_of[team][b ^ 1][0], wave);
            lv.issue(V, a.ld_v, next, a.rows_k, a.d, tiles_of[team][b ^ 1][1], wave);
        }
        const bool whole = x.whole(kb);
        if (!(x.whole(k0) && (SPLIT == 1 || x.whole(k0 + MA_K * (SPLIT - 1))))) {
            if (!whole && kb < x.ghi) Load::clean(tiles_of[team][b][1], bad, wave, lane);
            lds_barrier();
        }
        if (x.none(kb)) continue;
        const unsigned xk = at_k + b * 2 * SIZE, xv = at_v + b * 2 * SIZE;
        f32x16         s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = zero16();
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) s[t] = mma(Tile::frag(xk, 32 * t, kk), qf[kk], s[t]);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) scores<MODE, true>(a, s[t], slope2, kb + 32 * t + 4 * hf - m);
        // (without a cap +inf and NaN show by themselves; -inf is the largest word there is of a number)
        if (whole && !(MODE & CAP)) {
            unsigned low = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) low = max(low, __builtin_bit_cast(unsigned, (float)s[t][r]));
            sum = low >= 0xFF800000u ? NAN : sum;
        }
        if (!whole) {  // (also where this wave's queries see all of it: values were zeroed)
            const int      n0  = kb + 4 * hf - x.lo;
            const unsigned len = x.hi - x.lo;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int   n = 32 * t + 8 * (r >> 2) + (r & 3);
                    const float v = s[t][r] + (MODE & CAP ? bad[n + 4 * hf] : fmaf(s[t][r], 0.f, bad[n + 4 * hf]));
                    s[t][r]       = (unsigned)(n0 + n) < len ? v : -INFINITY;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
        top             = join_halves(top, [](float p, float q) { return fmaxf(p, q); }) * c;
        const bool late = top > ref + LAZY;
        if (__any(late)) {  // (each query by itself: its bits do not depend on its neighbours)
            const float fix = late ? __builtin_amdgcn_exp2f(ref - top) : 1.f;
            ref             = late ? top : ref;
            sum *= fix;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[dt][r] *= fix;
        }
        const float base = ref == -INFINITY ? 0.f : ref;  // (nothing seen yet: exp(-inf - 0) = 0)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            unsigned pk[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(s[t][2 * e], c, -base)), p1 = __builtin_amdgcn_exp2f(fmaf(s[t][2 * e + 1], c, -base));
                sum += p0 + p1;
                pk[e] = pack_f16(p0, p1);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] = mma(Tile::frag_t(xv, 32 * t + 16 * u, dt), words(pk, 4 * u), o[dt]);
        }
    }
    sum = join_halves(sum, [](float p, float q) { return p + q; });
    if constexpr (SPLIT > 1) {  // the second team's sums to the first, through the tiles' LDS
        static_assert(sizeof(tiles_of) >= (16 * DT + 2) * 256 * sizeof(float), "the sums fit");
        float* const ex = reinterpret_cast<float*>(tiles_of) + (threadIdx.x & 255);
        lds_barrier();
        if (team == 1) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) ex[256 * (16 * dt + r)] = o[dt][r];
            ex[256 * (16 * DT)]     = ref;
            ex[256 * (16 * DT + 1)] = sum;
        }
        lds_barrier();
        if (team == 1) return;
        const float ref1 = ex[256 * (16 * DT)], top = fmaxf(ref, ref1);
        const float f0 = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - top), f1 = ref1 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref1 - top);
        sum = sum * f0 + ex[256 * (16 * DT + 1)] * f1;
        ref = top;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] = o[dt][r] * f0 + ex[256 * (16 * dt + r)] * f1;
    }
    if (m < a.rows_q && hf == 0) a.lse[(long long)h * a.rows_q + m] = sum == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * LN2;
    store_rows<DT>(m < a.rows_q ? a.out + (long long)m * a.ld_ctx + h * a.d : nullptr, o, sum == 0.f ? 0.f : 1.f / sum, a.d, hf);
}

// ------------------------------------------------------------------------------------------------ backward
// dq of 128 queries, 32 of them a wave; teams as in the forward kernel.  Leaves the rows' statistics for the kernel of dk and dv: lse in base 2
// (+inf where a row sees nothing: its probabilities are then 0; POISON where it or delta is not a number to go by: a visible score's
// probability is then infinite, and that of a hidden one, exp(-inf - POISON), still 0) less log2 of P_SCALE, so that p and with it
// ds = p (dp - delta) come out times P_SCALE, and delta.
// ds is an fp16 operand: of 10^4 even probabilities and the gradients of a loss over 10^7 elements it is near 10^-8, where fp16 ends, so
// it keeps the factor.  A workgroup whose sums overflow that way, with a ds above 64, is done again without it, and then ends where ds
// itself does.  (Not for rows whose sums are not finite anyway; dk and dv of keys that such rows see are done twice.)
// delta = sum p dp is formed as sum dctx ctx from the ctx that was stored in fp16, whose rounding moves it by 2^-12 |dctx| |ctx|: gradients are
// off by 3e-4 of their norm as with an exact one, by 4 to 6e-4 where p (dp - delta) cancels.  Taking sum p dp itself out of ds afterwards
// would need sum p k, a fourth product with results of its own, and heads of 128 have no registers left here.
template <int D, int MODE, int SPLIT>
__global__ __launch_bounds__(256 * SPLIT, 2) void masked_dq_kernel(AttnArgs a) {
    constexpr int      KK = D / 16, DT = D / 32, ROWB = D <= 64 ? 128 : 256;
    constexpr unsigned SIZE = MA_K * ROWB;
    typedef TileLoad<ROWB, 4> Load;
    typedef LdsTile<ROWB>     Tile;
    __shared__ __align__(256) char tiles_of[SPLIT][2][2][SIZE];  // keys, values of two tiles
    __shared__ int vote;

    const int tiles = (a.rows_q + MA_Q - 1) / MA_Q;
    const int h = blockIdx.x % a.heads, qt = tiles - 1 - blockIdx.x / a.heads, kvh = h / a.group;
    const int lane = threadIdx.x & 63, wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = wave8 & 3, team = wave8 >> 2, hf = lane >> 5;
    const int m0 = qt * MA_Q, m = m0 + 32 * wave + (lane & 31);
    const QueryRange x(a, m0, m);
    const uint16_t*  K = a.k + kvh * a.d;
    const uint16_t*  V = a.v + kvh * a.d;
    Load             lk, lv;
    lk.init(a.ld_k, a.d, wave, lane);
    lv.init(a.ld_v, a.d, wave, lane);
    if (x.glo + MA_K * team < x.ghi) {
        lk.issue(K, a.ld_k, x.glo + MA_K * team, a.rows_k, a.d, tiles_of[team][0][0], wave);
        lv.issue(V, a.ld_v, x.glo + MA_K * team, a.rows_k, a.d, tiles_of[team][0][1], wave);
    }
    f16x8 qf[KK], gf[KK];
    row_frags<KK>(qf, m < a.rows_q ? a.q + (long long)m * a.ld_q + h * a.d : nullptr, a.d, hf);
    row_frags<KK>(gf, m < a.rows_q ? a.dctx + (long long)m * a.ld_dctx + h * a.d : nullptr, a.d, hf);
    const float slope2 = MODE && a.slopes ? a.slopes[h] * LOG2E : 0.f;
    const float c      = unit<MODE, false>(a);
    float       lse2 = INFINITY, delta = 0.f;
    if (m < a.rows_q) {
        lse2 = a.lse_in[(long long)h * a.rows_q + m] * LOG2E;
        f16x8 cf[KK];
        row_frags<KK>(cf, a.ctx + (long long)m * a.ld_ctx + h * a.d, a.d, hf);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int i = 0; i < 8; ++i) delta = fmaf((float)cf[kk][i], (float)gf[kk][i], delta);
    }
    delta = join_halves(delta, [](float p, float q) { return p + q; });
    if (x.lo >= x.hi || lse2 == -INFINITY)
        lse2 = INFINITY, delta = 0.f;
    else if (!(fabsf(lse2) < INFINITY && fabsf(delta) < INFINITY))
        lse2 = POISON, delta = 0.f;
    lse2 -= P_LOG2;
    if (team == 0 && hf == 0 && m < a.rows_pad) {
        a.lse2[(long long)h * a.rows_pad + m]              = lse2;
        a.delta[(long long)h * a.rows_pad + m]             = delta;
        a.delta[(long long)(h + a.heads) * a.rows_pad + m] = delta * (1.f / P_SCALE);
    }
    f32x16 o[DT];
    float  kept = 1.f;  // of P_SCALE, that ds has
    settle<KK>(qf);
    settle<KK>(gf);
    asm volatile("" : "+v"(lse2), "+v"(delta));
    const unsigned at_k = lds_address(tiles_of[team][0][0]) + Tile::plain(lane), at_v = lds_address(tiles_of[team][0][1]) + Tile::plain(lane);
    const unsigned at_t = lds_address(tiles_of[team][0][0]) + Tile::across(lane);

again:
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = zero16();
    int b = 0;
    for (int k0 = x.glo; k0 < x.ghi; k0 += MA_K * SPLIT, b ^= 1) {
        const int kb = k0 + MA_K * team, next = kb + MA_K * SPLIT;
        arrive();
        if (next < x.ghi) {
            lk.issue(K, a.ld_k, next, a.rows_k, a.d, tiles_of[team][b ^ 1][0], wave);
            lv.issue(V, a.ld_v, next, a.rows_k, a.d, tiles_of[team][b ^ 1][1], wave);
        }
        if (!(x.whole(k0) && (SPLIT == 1 || x.whole(k0 + MA_K * (SPLIT - 1))))) {
            if (!x.whole(kb) && kb < x.ghi) {
                Load::clean(tiles_of[team][b][0], nullptr, wave, lane);
                Load::clean(tiles_of[team][b][1], nullptr, wave, lane);
            }
            lds_barrier();
        }
        if (x.none(kb)) continue;
        const bool     all    = x.all(kb);
        const int      n0     = kb + 4 * hf - x.lo;
        const unsigned len    = x.hi - x.lo;
        const unsigned xk = at_k + b * 2 * SIZE, xv = at_v + b * 2 * SIZE, xt = at_t + b * 2 * SIZE;
        f32x16         s[2], dp[2];
        unsigned       ds[2][8];
        // Steps as in the kernel of dk and dv: scores and dp of 32 keys (u), of the other 32, dq of the first, of the other.
        constexpr int PP = D / 32, GP = D == 128 ? 2 : 1, PER = 2 * DT / GP, STEPS = 2 * PP + 2 * GP;
        f16x8         F[2][PER > 4 ? PER : 4];
        const auto    read = [&](int i) {
            if (i < 2 * PP) {
                const int u = i / PP, part = i % PP;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    F[i & 1][2 * j]     = Tile::frag(xk, 32 * u, 2 * part + j);
                    F[i & 1][2 * j + 1] = Tile::frag(xv, 32 * u, 2 * part + j);
                }
            } else {
                const int u = (i - 2 * PP) / GP, part = (i - 2 * PP) % GP;
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    const int w = (part * PER + j) / DT, dt = (part * PER + j) % DT;
                    F[i & 1][j] = Tile::frag_t(xt, 32 * u + 16 * w, dt);
                }
            }
        };
        const auto multiply = [&](int i) {
            if (i < 2 * PP) {
                const int u = i / PP, part = i % PP;
                if (part == 0) s[u] = dp[u] = zero16();
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    s[u]  = mma(F[i & 1][2 * j], qf[2 * part + j], s[u]);
                    dp[u] = mma(F[i & 1][2 * j + 1], gf[2 * part + j], dp[u]);
                }
            } else {
                const int u = (i - 2 * PP) / GP, part = (i - 2 * PP) % GP;
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    const int w = (part * PER + j) / DT, dt = (part * PER + j) % DT;
                    o[dt] = mma(F[i & 1][j], words(ds[u], 4 * w), o[dt]);
                }
            }
        };
        const auto weights = [&](int u, int first, int last) {  // ds of pairs of keys
            const float at = (float)(kb + 32 * u + 4 * hf - m);
#pragma unroll
            for (int e = first; e < last; ++e) {
                float d[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int   r = 2 * e + y;
                    const float p = __builtin_amdgcn_exp2f(exponent<MODE>(s[u][r], c, lse2, slope2, at, r));  // (times P_SCALE)
                    d[y] = p * fmaf(dp[u][r], kept, -delta);
                    if (MODE & CAP) d[y] *= fade(s[u][r]);
                }
                ds[u][e] = pack_f16(d[0], d[1]);
            }
        };
        const auto prepare = [&](int u) {
            scores<MODE, false>(a, s[u], slope2, kb + 32 * u + 4 * hf - m);
            if (!all) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = (unsigned)(n0 + 32 * u + 8 * (r >> 2) + (r & 3)) < len ? s[u][r] : -INFINITY;
            }
        };
        read(0);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            if (i == PP) prepare(0);
            if (i == 2 * PP) prepare(1);
            step();
            if (i + 1 < STEPS) read(i + 1);
            multiply(i);
            if (i >= PP && i < 2 * PP) weights(0, 8 * (i - PP) / PP, 8 * (i - PP + 1) / PP);
            if (i >= 2 * PP && i < 2 * PP + GP) weights(1, 8 * (i - 2 * PP) / GP, 8 * (i - 2 * PP + 1) / GP);
        }
    }
    if (kept == 1.f && any_of_workgroup(fabsf(lse2) < 1e38f && !finite(o), &vote)) {
        kept = 1.f / P_SCALE;
        delta *= kept;
        if (x.glo + MA_K * team < x.ghi) {
            lk.issue(K, a.ld_k, x.glo + MA_K * team, a.rows_k, a.d, tiles_of[team][0][0], wave);
            lv.issue(V, a.ld_v, x.glo + MA_K * team, a.rows_k, a.d, tiles_of[team][0][1], wave);
        }
        goto again;
    }
    if constexpr (SPLIT > 1) {  // the second team's sums to the first, through the tiles' LDS
        static_assert(sizeof(tiles_of) >= 16 * DT * 256 * sizeof(float), "the sums fit");
        float* const ex = reinterpret_cast<float*>(tiles_of) + (threadIdx.x & 255);
        lds_barrier();
        if (team == 1) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) ex[256 * (16 * dt + r)] = o[dt][r];
        }
        lds_barrier();
        if (team == 1) return;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] += ex[256 * (16 * dt + r)];
    }
    // (a row that sees nothing may hold anything in q and dctx, and 0 x NaN has reached its sums)
    if (x.lo >= x.hi) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = zero16();
    }
    // (a query whose scores are all -inf has probabilities of 0 all the same)
    store_rows<DT>(m < a.rows_q ? a.dq + (long long)m * a.ld_dq + h * a.d : nullptr, o, lse2 < -1e38f ? NAN : a.alpha / (P_SCALE * kept), a.d, hf);
}

// dk and dv of 128 keys, 32 of them a wave, over the tiles of 64 queries that see any of them, head by head: of all heads that share
// the keys, or of a.part_heads of them, whose sums the join kernel adds up.  Teams as above, each with every SPLITth tile.
template <int D, int MODE, int SPLIT>
__global__ __launch_bounds__(256 * SPLIT, D <= 64 ? 2 : 1) void masked_dkv_kernel(AttnArgs a) {
    constexpr int      KK = D / 16, DT = D / 32, ROWB = D <= 64 ? 128 : 256;
    constexpr unsigned SIZE = MA_K * ROWB;
    typedef TileLoad<ROWB, 4> Load;
    typedef LdsTile<ROWB>     Tile;
    struct Stats {
        float lse2[MA_K], delta[MA_K];
        int2  range[2 * MA_K];  // (a wave's load is twice as long)
    };
    __shared__ __align__(256) char tiles_of[SPLIT][2][2][SIZE];  // queries, gradients of two tiles
    __shared__ __align__(16) Stats stats_of[SPLIT][2];
    __shared__ int vote;

    const int kv_heads = a.heads / a.group, parts = a.group / a.part_heads, per = kv_heads * parts;
    const int id = blockIdx.x % per, kvh = id / parts, h0 = kvh * a.group + id % parts * a.part_heads, kt = blockIdx.x / per;
    const int lane = threadIdx.x & 63, wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = wave8 & 3, team = wave8 >> 2, hf = lane >> 5;
    Stats* const stats = stats_of[team];
    const int k0 = kt * MA_Q, n0 = k0 + 32 * wave, n = n0 + (lane & 31);
    const int qtiles = a.rows_pad / MA_K;

    // the tiles to come, one by one
    const int          end = h0 + a.part_heads;
    int                h = h0, base = -64, q0 = 0;
    int4               bounds = make_int4(0, 0, 0, 0), t4 = bounds;
    unsigned long long todo = 0;
    const auto         advance = [&]() {
        while (todo == 0) {
            if (h == end) return false;  // (asked again behind the end: no more either)
            base += 64;
            if (base >= qtiles) {
                base = 0;
                if (++h == end) return false;
            }
            bounds = base + lane < qtiles ? a.tile[base + lane] : make_int4(INT_MAX, 0, INT_MAX, 0);
            todo   = __ballot(bounds.x < k0 + MA_Q && bounds.y > k0);  // (the same in every wave)
        }
        const int i = __builtin_ctzll(todo);
        todo &= todo - 1;
        q0 = (base + i) * MA_K;
        t4 = make_int4(__builtin_amdgcn_readlane(bounds.x, i), __builtin_amdgcn_readlane(bounds.y, i), __builtin_amdgcn_readlane(bounds.z, i),
                       __builtin_amdgcn_readlane(bounds.w, i));
        return true;
    };
    // a step: one tile for each team
    struct Step {
        int  q0, h;
        int4 t;
        bool mine, whole;  // whether this team has a tile; whether all keys are seen whole in every team's
    };
    const auto take = [&](Step& x) {
        x.mine = false, x.whole = true;
        for (int i = 0; i < SPLIT; ++i) {
            if (!advance()) return i > 0;
            x.whole = x.whole && t4.z <= k0 && t4.w >= k0 + MA_Q;
            if (i == team) x.mine = true, x.q0 = q0, x.h = h, x.t = t4;
        }
        return true;
    };
    Load lq, lg;
    lq.init(a.ld_q, a.d, wave, lane);
    lg.init(a.ld_dctx, a.d, wave, lane);
    float        kept = 1.f;  // of P_SCALE, that ds has
    const float* delta = a.delta;
    const auto issue = [&](int b, const Step& x) {
        if (!x.mine) return;
        lq.issue(a.q + x.h * a.d, a.ld_q, x.q0, a.rows_q, a.d, tiles_of[team][b][0], wave);
        lg.issue(a.dctx + x.h * a.d, a.ld_dctx, x.q0, a.rows_q, a.d, tiles_of[team][b][1], wave);
        const long long at = (long long)x.h * a.rows_pad + x.q0;
        if (wave == 0) load_words(a.lse2 + at, stats[b].lse2, lane);
        if (wave == 1) load_words(delta + at, stats[b].delta, lane);
        if (wave == 2) load_ranges(a.range + x.q0, stats[b].range, lane);
    };
    Step now, next;
    bool more = take(next);
    if (more) issue(0, next);
    f16x8 kf[KK], vf[KK];
    row_frags<KK>(kf, n < a.rows_k ? a.k + (long long)n * a.ld_k + kvh * a.d : nullptr, a.d, hf);
    row_frags<KK>(vf, n < a.rows_k ? a.v + (long long)n * a.ld_v + kvh * a.d : nullptr, a.d, hf);
    f32x16 dk[DT], dv[DT];
    settle<KK>(kf);
    settle<KK>(vf);
    const float c = unit<MODE, false>(a);

    const unsigned at_q = lds_address(tiles_of[team][0][0]) + Tile::plain(lane), at_g = at_q + SIZE;
    const unsigned at_tq = lds_address(tiles_of[team][0][0]) + Tile::across(lane), at_tg = at_tq + SIZE;
    bool           ever = false;  // (the other half of the wave has the other queries)
again:
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dk[dt] = dv[dt] = zero16();
    for (int b = 0; more; b ^= 1) {
        now = next;
        arrive();
        more = take(next);
        if (more) issue(b ^ 1, next);
        const int4 t = now.t;
        if (!now.whole) {
            if (now.mine && !(t.z <= k0 && t.w >= k0 + MA_Q)) {
                Load::clean(tiles_of[team][b][0], nullptr, wave, lane);
                Load::clean(tiles_of[team][b][1], nullptr, wave, lane);
            }
            lds_barrier();
        }
        if (!now.mine || t.x >= n0 + 32 || t.y <= n0) continue;
        const int m0 = now.q0, head = now.h;
        const float slope2 = MODE && a.slopes ? a.slopes[head] * LOG2E : 0.f;
        const unsigned xq = at_q + b * 2 * SIZE, xg = at_g + b * 2 * SIZE, tq = at_tq + b * 2 * SIZE, tg = at_tg + b * 2 * SIZE;
        // which of this lane's 16 queries of each half see its key
        unsigned   seen[2] = {0xFFFFu, 0xFFFFu};
        const bool all     = t.z <= n0 && t.w >= n0 + 32;
        if (!all) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                seen[u] = 0;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int2 g = stats[b].range[32 * u + 8 * (r >> 2) + 4 * hf + (r & 3)];
                    seen[u] |= (unsigned)(n - g.x) < (unsigned)(g.y - g.x) ? 1u << r : 0u;
                    if ((r & 7) == 7) step();
                }
            }
        }
        ever |= (seen[0] | seen[1]) != 0;
        f32x16         s[2], dp[2];
        unsigned       pk[2][8], dsk[2][8];
        // Steps, each the products of fragments that were read during the one before: scores and dp of 32 queries (u), the same of
        // the other 32, dv and dk of the first, of the other; what lies between products of one u rides beside those of the other.
        constexpr int PARTS = D / 32, CK = KK / PARTS, PAIRS = 2 * DT / PARTS, STEPS = 4 * PARTS;
        static_assert(KK % PARTS == 0 && 2 * DT % PARTS == 0, "whole parts");
        f16x8      F[2][2 * (CK > PAIRS ? CK : PAIRS)];
        const auto read = [&](int i) {
            const int u = i / PARTS & 1, part = i % PARTS;
            if (i < 2 * PARTS) {
#pragma unroll
                for (int j = 0; j < CK; ++j) {
                    F[i & 1][2 * j]     = Tile::frag(xq, 32 * u, part * CK + j);
                    F[i & 1][2 * j + 1] = Tile::frag(xg, 32 * u, part * CK + j);
                }
            } else {
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) {
                    const int w = (part * PAIRS + j) / DT, dt = (part * PAIRS + j) % DT;
                    F[i & 1][2 * j]     = Tile::frag_t(tg, 32 * u + 16 * w, dt);
                    F[i & 1][2 * j + 1] = Tile::frag_t(tq, 32 * u + 16 * w, dt);
                }
            }
        };
        const auto multiply = [&](int i) {
            const int u = i / PARTS & 1, part = i % PARTS;
            if (i < 2 * PARTS) {
                if (part == 0) s[u] = dp[u] = zero16();
#pragma unroll
                for (int j = 0; j < CK; ++j) {
                    s[u]  = mma(F[i & 1][2 * j], kf[part * CK + j], s[u]);
                    dp[u] = mma(F[i & 1][2 * j + 1], vf[part * CK + j], dp[u]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) {
                    const int e = (part * PAIRS + j) / DT * 4, dt = (part * PAIRS + j) % DT;
                    dv[dt] = mma(F[i & 1][2 * j], words(pk[u], e), dv[dt]);
                    dk[dt] = mma(F[i & 1][2 * j + 1], words(dsk[u], e), dk[dt]);
                }
            }
        };
        const auto weights = [&](int u, int part) {  // probabilities and ds
            const float at = (float)(m0 + 32 * u + 4 * hf - n);
#pragma unroll
            for (int e = 4 * part / PARTS; e < 4 * (part + 1) / PARTS; ++e) {
                const int   i0 = 32 * u + 8 * e + 4 * hf;
                const f32x4 l4 = *reinterpret_cast<const f32x4*>(stats[b].lse2 + i0), d4 = *reinterpret_cast<const f32x4*>(stats[b].delta + i0);
                float       p[4], d[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int r = 4 * e + x;
                    p[x]        = __builtin_amdgcn_exp2f(exponent<MODE>(s[u][r], c, l4[x], slope2, at, r));  // (P_SCALE is in it)
                    d[x]        = p[x] * fmaf(dp[u][r], kept, -d4[x]);
                    if (MODE & CAP) d[x] *= fade(s[u][r]);
                }
                pk[u][2 * e]      = pack_f16(p[0], p[1]);
                pk[u][2 * e + 1]  = pack_f16(p[2], p[3]);
                dsk[u][2 * e]     = pack_f16(d[0], d[1]);
                dsk[u][2 * e + 1] = pack_f16(d[2], d[3]);
            }
        };
        const auto prepare = [&](int u) {
            scores<MODE, false>(a, s[u], slope2, m0 + 32 * u + 4 * hf - n);
            if (!all) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = seen[u] >> r & 1 ? s[u][r] : -INFINITY;
            }
        };
        read(0);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            if (i == PARTS) prepare(0);
            if (i == 2 * PARTS) prepare(1);
            step();
            if (i + 1 < STEPS) read(i + 1);
            multiply(i);
            if (i >= PARTS && i < 3 * PARTS) weights(i / PARTS - 1, i % PARTS);
        }
    }
    const bool seen_once = __ballot(ever) >> (lane & 31) & 0x100000001ull;
    if (kept == 1.f && any_of_workgroup(seen_once && !finite(dk), &vote)) {
        kept = 1.f / P_SCALE, delta += (long long)a.heads * a.rows_pad;
        h = h0, base = -64, todo = 0;
        more = take(next);
        if (more) issue(0, next);
        goto again;
    }
    if (!seen_once) {  // (a key that nobody sees may hold anything, and 0 x NaN has reached its sums)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) dk[dt] = dv[dt] = zero16();
    }
    if constexpr (SPLIT > 1) {  // the second team's sums to the first, through the tiles' LDS
        static_assert(sizeof(tiles_of) >= 32 * DT * 256 * sizeof(float), "the sums fit");
        float* const ex = reinterpret_cast<float*>(tiles_of) + (threadIdx.x & 255);
        lds_barrier();
        if (team == 1) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    ex[512 * (16 * dt + r)]       = dk[dt][r];
                    ex[512 * (16 * dt + r) + 256] = dv[dt][r];
                }
        }
        lds_barrier();
        if (team == 1) return;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                dk[dt][r] += ex[512 * (16 * dt + r)];
                dv[dt][r] += ex[512 * (16 * dt + r) + 256];
            }
    }
    if (a.part_heads == a.group) {
        const bool in = n < a.rows_k;
        store_rows<DT>(in ? a.dv + (long long)n * a.ld_dv + kvh * a.d : nullptr, dv, 1.f / P_SCALE, a.d, hf);
        store_rows<DT>(in ? a.dk + (long long)n * a.ld_dk + kvh * a.d : nullptr, dk, a.alpha / (P_SCALE * kept), a.d, hf);
    } else if (n < a.rows_k) {
        float*      to = a.part + ((long long)id * a.rows_k + n) * 2 * a.d;
        const float k  = 1.f / (P_SCALE * kept);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int col = 32 * dt + 8 * e + 4 * hf;
                if (col < a.d) {
                    *reinterpret_cast<f32x4*>(to + col)       = f32x4{dk[dt][4 * e] * k, dk[dt][4 * e + 1] * k, dk[dt][4 * e + 2] * k, dk[dt][4 * e + 3] * k};
                    *reinterpret_cast<f32x4*>(to + a.d + col) = f32x4{dv[dt][4 * e], dv[dt][4 * e + 1], dv[dt][4 * e + 2], dv[dt][4 * e + 3]};
                }
            }
    }
}

// Sums of the parts of a key / value head, in order: 4 columns a thread.
__global__ __launch_bounds__(JOIN_THREADS) void masked_join_kernel(AttnArgs a) {
    const int       kv_heads = a.heads / a.group, parts = a.group / a.part_heads, per = a.d / 4;
    const long long i = (long long)blockIdx.x * JOIN_THREADS + threadIdx.x, row = i / per / kv_heads;
    if (row >= a.rows_k) return;
    const int kvh = (int)(i / per % kv_heads), col = (int)(i % per) * 4;
    f32x4     dk = {0.f, 0.f, 0.f, 0.f}, dv = dk;
    for (int p = 0; p < parts; ++p) {
        const float* from = a.part + ((long long)(kvh * parts + p) * a.rows_k + row) * 2 * a.d + col;
        dk += *reinterpret_cast<const f32x4*>(from);
        dv += *reinterpret_cast<const f32x4*>(from + a.d);
    }
    const float k = a.alpha, v = 1.f / P_SCALE;
    *reinterpret_cast<u32x2m*>(a.dk + row * a.ld_dk + kvh * a.d + col) = u32x2m{pack_f16(dk[0] * k, dk[1] * k), pack_f16(dk[2] * k, dk[3] * k)};
    *reinterpret_cast<u32x2m*>(a.dv + row * a.ld_dv + kvh * a.d + col) = u32x2m{pack_f16(dv[0] * v, dv[1] * v), pack_f16(dv[2] * v, dv[3] * v)};
}

// ------------------------------------------------------------------------------------------------ entry points
static int rows64(int rows) { return rows > 0 ? (rows + 63) / 64 : 0; }
static size_t mask_rows_bytes(int rows) { return (size_t)rows64(rows) * 64 * sizeof(int2); }

static int check_desc(const char* who, const mp_attn_desc* d) {
    MP_REQUIRE(d != nullptr, "%s: desc is NULL", who);
    MP_REQUIRE(d->rows_q >= 0 && d->rows_k >= 0 && d->n_heads > 0 && d->n_kv_heads > 0 && d->d_head > 0, "%s: bad shape", who);
    MP_REQUIRE(d->n_heads % d->n_kv_heads == 0, "%s: %d heads do not share %d key / value heads evenly", who, d->n_heads, d->n_kv_heads);
    MP_REQUIRE(d->alpha > 0.f && d->alpha < INFINITY && d->cap >= 0.f && d->cap < INFINITY, "%s: alpha must be positive and cap not negative", who);
    MP_REQUIRE(d->reserved == 0, "%s: reserved is not 0", who);
    // (tanh is good to 2^-22 in absolute terms, which a larger cap would make errors of a score that fp16 shows)
    if (d->cap > 0.f && (d->cap > 1024.f || !(d->alpha / d->cap < 1e30f))) {
        set_error("%s: cap %g above 1024 or too small for alpha %g", who, (double)d->cap, (double)d->alpha);
        return MP_E_UNSUPPORTED;
    }
    if (d->d_head > 128 || (d->d_head & 7)) {
        set_error("%s: head size %d is not a multiple of 8 up to 128", who, d->d_head);
        return MP_E_UNSUPPORTED;
    }
    const long long w = (long long)d->n_heads * d->d_head, wk = (long long)d->n_kv_heads * d->d_head;
    MP_REQUIRE(w < (1 << 24), "%s: too many heads", who);
    MP_REQUIRE(d->rows_q <= 0x7FFFFF00 && d->rows_k <= 0x7FFFFF00, "%s: too many rows", who);
    MP_REQUIRE(grid_fits(((long long)d->rows_q + MA_Q) / MA_Q * d->n_heads, 256) && grid_fits(((long long)d->rows_k + MA_Q) / MA_Q * d->n_heads, 256),
               "%s: too many rows and heads", who);
    MP_REQUIRE(d->ld_q >= w && d->ld_k >= wk && d->ld_v >= wk && d->ld_ctx >= w, "%s: a leading dimension is smaller than its rows", who);
    if (((d->ld_q | d->ld_k | d->ld_v | d->ld_ctx) & 7) || (d->ld_q | d->ld_k | d->ld_v | d->ld_ctx) >= (1 << 22)) {
        set_error("%s: leading dimensions must be multiples of 8 below 2^22", who);
        return MP_E_UNSUPPORTED;
    }
    return MP_OK;
}
static int check_aligned(const char* who, std::initializer_list<const void*> ps) {
    for (const void* p : ps)
        if (!aligned16(p)) {
            set_error("%s: matrices must be 16-byte aligned", who);
            return MP_E_UNSUPPORTED;
        }
    return MP_OK;
}
static AttnArgs attn_args(const mp_attn_desc* d, const void* mask, const float* slopes) {
    AttnArgs a   = {};
    a.part_heads = d->n_heads / d->n_kv_heads;
    a.slopes   = slopes;
    a.range    = static_cast<const int2*>(mask);
    a.tile     = reinterpret_cast<const int4*>(static_cast<const char*>(mask) + mask_rows_bytes(d->rows_q));
    a.rows_q = d->rows_q, a.rows_k = d->rows_k, a.heads = d->n_heads, a.group = d->n_heads / d->n_kv_heads, a.d = d->d_head;
    a.rows_pad = rows64(d->rows_q) * 64;
    a.ld_q = d->ld_q, a.ld_k = d->ld_k, a.ld_v = d->ld_v, a.ld_ctx = d->ld_ctx;
    a.ld_dq = d->ld_dq, a.ld_dk = d->ld_dk, a.ld_dv = d->ld_dv, a.ld_dctx = d->ld_dctx;
    a.alpha = d->alpha, a.cap = d->cap;
    return a;
}
// The kernel of the head size (rounded up to a multiple of 32) and of what is done to the scores.
#define MA_CASE(D, M, kernel, threads, grid, a, hs, ...) \
    case D / 32 * 4 + M: hipLaunchKernelGGL((kernel<D, M, ##__VA_ARGS__>), dim3((unsigned)(grid)), dim3(threads), 0, hs, a); break
#define MA_CASES(D, ...) MA_CASE(D, PLAIN, __VA_ARGS__); MA_CASE(D, BIAS, __VA_ARGS__); MA_CASE(D, CAP, __VA_ARGS__); MA_CASE(D, CAP + BIAS, __VA_ARGS__)
#define MA_LAUNCH(kernel, threads, grid, a, ...)                                                                  \
    switch (((a).d + 31) / 32 * 4 + ((a).cap > 0.f ? CAP : 0) + ((a).slopes ? BIAS : 0)) {                          \
        MA_CASES(32, kernel, threads, grid, a, __VA_ARGS__); MA_CASES(64, kernel, threads, grid, a, __VA_ARGS__);  \
        MA_CASES(96, kernel, threads, grid, a, __VA_ARGS__); MA_CASES(128, kernel, threads, grid, a, __VA_ARGS__); \
    }
// the same where only the kernels of head sizes up to 64 exist
#define MA_LAUNCH_64(kernel, threads, grid, a, ...)                                                                \
    switch (((a).d + 31) / 32 * 4 + ((a).cap > 0.f ? CAP : 0) + ((a).slopes ? BIAS : 0)) {                          \
        MA_CASES(32, kernel, threads, grid, a, __VA_ARGS__); MA_CASES(64, kernel, threads, grid, a, __VA_ARGS__);  \
    }

// Two teams a workgroup where there are fewer workgroups than these.  A compute unit takes two workgroups of one team or one of two, so
// teams fill the chip with half as many; with more workgroups than that, one team each balances better (it has no join, and long
// workgroups run beside short ones).  us with two teams / one.  Forward, every key seen, 8192 rows: heads of 128, 256 workgroups
// 150 / 181, 512 330 / 302, 768 453 / 448, 1024 579 / 552; causal 776 353 / 487; heads of 64, 256 workgroups 100 / 130, 512 166 / 172;
// 1024 of documents of about 500 rows 52 / 46.  (All calls of a size take one rule, so causal ones decide for 768.)  dq likewise: causal 776
// workgroups of heads of 128, whole backward 1242 / 1350.  dk and dv, heads up to 64, whole backward, causal: 256 workgroups of one document
// 118 / 138, of documents of 64 rows 38 / 41, 384 130 / 149, 512 of documents of 512 rows 59 / 54.  Heads above 64 need a wave's
// full registers there, which leaves no room for a second team.
constexpr long long ONE_TEAM = 1024, ONE_TEAM_DKV = 512;

}  // namespace mp

using namespace mp;

extern "C" size_t mp_attention_mask_bytes(int rows_q) {
    return rows_q < 0 ? 0 : mask_rows_bytes(rows_q) + (size_t)rows64(rows_q) * sizeof(int4) + 16;
}

static int build_mask(const char* who, int rows, int rows_k, int n_docs, const int32_t* start, const int32_t* prefix, int causal, int window,
                      const int32_t* lo, const int32_t* hi, void* mask, mp_stream stream) {
    MP_REQUIRE(aligned16(mask), "%s: mask must be 16-byte aligned", who);
    if (rows == 0) return MP_OK;
    int2* range = static_cast<int2*>(mask);
    int4* tile  = reinterpret_cast<int4*>(static_cast<char*>(mask) + mask_rows_bytes(rows));
    hipLaunchKernelGGL(mask_kernel, dim3(rows64(rows)), dim3(64), 0, as_stream(stream), rows, rows_k, n_docs, start, prefix, causal, window, lo, hi,
                       range, tile);
    MP_LAUNCH_CHECK(who);
    return MP_OK;
}

extern "C" int mp_attention_mask_docs(int rows, int n_docs, const int32_t* doc_start, const int32_t* prefix, int causal, int window,
                                      void* mask, mp_stream stream) {
    const char* who = "mp_attention_mask_docs";
    MP_REQUIRE(rows >= 0 && rows <= 0x7FFFFF00 && n_docs >= 0 && n_docs < INT_MAX && window >= 0, "%s: bad shape", who);
    MP_REQUIRE(mask && (n_docs == 0 || doc_start), "%s: NULL argument", who);
    MP_REQUIRE(!prefix || (causal && !window), "%s: a prefix is for causal masks without a window", who);
    return build_mask(who, rows, rows, n_docs, doc_start, prefix, causal, window, nullptr, nullptr, mask, stream);
}

extern "C" int mp_attention_mask_ranges(int rows_q, int rows_k, const int32_t* lo, const int32_t* hi, void* mask, mp_stream stream) {
    const char* who = "mp_attention_mask_ranges";
    MP_REQUIRE(rows_q >= 0 && rows_q <= 0x7FFFFF00 && rows_k >= 0 && rows_k <= 0x7FFFFF00, "%s: bad shape", who);
    MP_REQUIRE(mask && (rows_q == 0 || (lo && hi)), "%s: NULL argument", who);
    return build_mask(who, rows_q, rows_k, 0, nullptr, nullptr, 0, 0, lo, hi, mask, stream);
}

extern "C" int mp_attention_masked_fwd(const mp_attn_desc* desc, const void* mask, const mp_half* q, const mp_half* k, const mp_half* v,
                                       const float* slopes, mp_half* ctx, float* lse, mp_stream stream) {
    const char* who = "mp_attention_masked_fwd";
    int         rc  = check_desc(who, desc);
    if (rc) return rc;
    if (desc->rows_q == 0) return MP_OK;
    MP_REQUIRE(mask && q && ctx && lse && (desc->rows_k == 0 || (k && v)), "%s: NULL argument", who);
    rc = check_aligned(who, {mask, q, k, v, ctx});
    if (rc) return rc;
    AttnArgs a = attn_args(desc, mask, slopes);
    a.q = q, a.k = k, a.v = v, a.out = ctx, a.lse = lse;
    const long long wgs = (long long)((desc->rows_q + MA_Q - 1) / MA_Q) * desc->n_heads;
    if (wgs >= ONE_TEAM)
        MA_LAUNCH(masked_fwd_kernel, 256, wgs, a, as_stream(stream), 1)
    else
        MA_LAUNCH(masked_fwd_kernel, 512, wgs, a, as_stream(stream), 2)
    MP_LAUNCH_CHECK(who);
    return MP_OK;
}

// How many of the heads that share keys a workgroup of dk and dv takes: all of them where that gives every compute unit two workgroups
// (their sums then stay in registers), else one, with sums in fp32 through memory.  8 heads of 128 over 2, one document of 12289 rows
// (194 workgroups or 776): 2.61 ms with all, 1.98 apart (when it was made; 0.81 with the steps that followed).  Parts of the queries instead, of 12
// tiles or more, gained 13 % for one long document without shared keys and cost up to 26 % elsewhere: their sums go through memory.
static int part_heads(const mp_attn_desc* d) {
    const int group = d->n_heads / d->n_kv_heads;
    return (long long)((d->rows_k + MA_Q - 1) / MA_Q) * d->n_kv_heads >= 512 ? group : 1;
}
static size_t stats_bytes(const mp_attn_desc* d) { return (size_t)rows64(d->rows_q) * 64 * d->n_heads * 3 * sizeof(float); }
static size_t parts_bytes(const mp_attn_desc* d) {
    const int group = d->n_heads / d->n_kv_heads;
    return group == part_heads(d) ? 0 : (size_t)d->n_heads * d->rows_k * 2 * d->d_head * sizeof(float);
}

extern "C" size_t mp_attention_masked_bwd_workspace_bytes(const mp_attn_desc* desc) {
    if (check_desc("mp_attention_masked_bwd_workspace_bytes", desc) != MP_OK) return 0;
    return stats_bytes(desc) + parts_bytes(desc) + 256;
}

extern "C" int mp_attention_masked_bwd(const mp_attn_desc* desc, const void* mask, const mp_half* q, const mp_half* k, const mp_half* v,
                                       const float* slopes, const mp_half* ctx, const float* lse, const mp_half* dctx, mp_half* dq,
                                       mp_half* dk, mp_half* dv, void* ws, size_t ws_bytes, mp_stream stream) {
    const char* who = "mp_attention_masked_bwd";
    int         rc  = check_desc(who, desc);
    if (rc) return rc;
    const mp_attn_desc& d = *desc;
    const int           w = d.n_heads * d.d_head, wk = d.n_kv_heads * d.d_head;
    MP_REQUIRE(d.ld_dq >= w && d.ld_dk >= wk && d.ld_dv >= wk && d.ld_dctx >= w, "%s: a leading dimension is smaller than its rows", who);
    if (((d.ld_dq | d.ld_dk | d.ld_dv | d.ld_dctx) & 7) || (d.ld_dq | d.ld_dk | d.ld_dv | d.ld_dctx) >= (1 << 22)) {
        set_error("%s: leading dimensions must be multiples of 8 below 2^22", who);
        return MP_E_UNSUPPORTED;
    }
    if (d.rows_q == 0 && d.rows_k == 0) return MP_OK;
    MP_REQUIRE((d.rows_q == 0 || (mask && q && ctx && lse && dctx && dq)) && (d.rows_k == 0 || (k && v && dk && dv)), "%s: NULL argument", who);
    rc = check_aligned(who, {mask, q, k, v, ctx, dctx, dq, dk, dv});
    if (rc) return rc;
    if (!ws || !aligned16(ws) || ws_bytes < mp_attention_masked_bwd_workspace_bytes(desc)) {
        set_error("%s: workspace missing, misaligned or smaller than mp_attention_masked_bwd_workspace_bytes", who);
        return MP_E_WORKSPACE;
    }
    hipStream_t hs = as_stream(stream);
    AttnArgs    a  = attn_args(desc, mask, slopes);
    a.q = q, a.k = k, a.v = v, a.ctx = ctx, a.lse_in = lse, a.dctx = dctx, a.dq = dq, a.dk = dk, a.dv = dv;
    a.lse2  = static_cast<float*>(ws);
    a.delta = a.lse2 + (size_t)a.rows_pad * a.heads;
    a.part  = a.delta + (size_t)a.rows_pad * a.heads * 2;
    a.part_heads = part_heads(desc);
    if (d.rows_q > 0) {
        const long long wgs = (long long)((d.rows_q + MA_Q - 1) / MA_Q) * d.n_heads;
        if (wgs >= ONE_TEAM)
            MA_LAUNCH(masked_dq_kernel, 256, wgs, a, hs, 1)
        else
            MA_LAUNCH(masked_dq_kernel, 512, wgs, a, hs, 2)
        MP_LAUNCH_CHECK(who);
    }
    if (d.rows_k > 0) {
        const long long wgs = (long long)((d.rows_k + MA_Q - 1) / MA_Q) * (d.n_heads / a.part_heads);
        if (d.d_head > 64 || wgs >= ONE_TEAM_DKV)
            MA_LAUNCH(masked_dkv_kernel, 256, wgs, a, hs, 1)
        else
            MA_LAUNCH_64(masked_dkv_kernel, 512, wgs, a, hs, 2)
        MP_LAUNCH_CHECK(who);
        if (a.part_heads < a.group) {
            const long long quads = (long long)d.rows_k * d.n_kv_heads * (d.d_head / 4);
            hipLaunchKernelGGL(masked_join_kernel, dim3((unsigned)((quads + JOIN_THREADS - 1) / JOIN_THREADS)), dim3(JOIN_THREADS), 0, hs, a);
            MP_LAUNCH_CHECK(who);
        }
    }
    return MP_OK;
}
