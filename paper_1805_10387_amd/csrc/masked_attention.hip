// Attention under interval masks, forward and backward, any length (paper Section 3.1 arithmetic; the softmax an fp32 part).
//
// One pass over the keys with a running maximum and sum: for a tile of keys S^T = K Q^T on the matrix cores, p = exp(s - max), and
// O^T = O^T exp(max_old - max) + V^T P; scores stay in registers.  Transposed throughout: a lane owns ONE query (column of S^T),
// so the row statistics are one register a lane, and the packed probabilities are the second operand of the next product without
// a move.  Backward recomputes the probabilities from the kept log-sum-exp: one kernel per tile of queries for dq, one per
// tile of keys for dk and dv, so that every gradient has one owner and no atomics (7 products instead of the 5 that one pass
// with atomics would take).
//
// Masks: query r sees keys [lo, hi).  Whether a tile of pairs is empty, whole or neither follows from four numbers of a 64-row tile
// (least lo, greatest hi, greatest lo, least hi) that the mask keeps behind the rows' own; only tiles that are neither look at
// single pairs.
//
// What is hidden must not be felt, though 0 x NaN is NaN: scores of hidden pairs are replaced, not added to; and in tiles that are
// not whole, non-finite elements of the matrices that a zero probability would multiply are zeroed on their way into LDS.
// Those that are visible still show: forward by a NaN score in their place, backward because a query that sees one has a non-finite
// lse or delta, and its lse is made a NaN.
#include "attn_lds.hpp"

#include <limits.h>
#include <math.h>

namespace mp {

constexpr int   MA_THREADS = 256;
constexpr int   MA_Q       = 128;   // queries of a workgroup, 32 a wave (dk/dv: keys)
constexpr int   MA_K       = 64;    // keys of a tile (dk/dv: queries)
constexpr float LOG2E      = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float P_SCALE    = 1024.f;  // dv's probabilities: of 10^5 keys one has 10^-5, which fp16 has to three digits only

struct AttnArgs {
    const uint16_t *q, *k, *v, *ctx, *dctx;
    uint16_t *      out, *dq, *dk, *dv;
    float*          lse;                 // forward: out
    const float *   lse_in, *slopes;
    float *         lse2, *delta;        // backward: [n_heads, rows_pad]
    const int2*     range;
    const int4*     tile;
    int             rows_q, rows_k, heads, group, d, rows_pad;
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
            int a = 0, b = n_docs;  // start[a] <= r < start[b]
            while (b - a > 1) {
                const int c = (a + b) >> 1;
                if (start[c] <= r) a = c; else b = c;
            }
            const int s = max(start[a], 0), e = min(start[b], rows);
            lo = s;
            hi = causal ? r + 1 : e;
            if (prefix) hi = max(hi, min(e, s + min(prefix[a], rows)));
            if (window) {
                lo = max(lo, r - window + 1);
                if (window < rows) hi = min(hi, r + window);
            }
        }
        if (lo >= hi) lo = hi = 0;
        range[r] = make_int2(lo, hi);
    }
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
// Base-2 scores of a block of accumulators; lanes own one index, registers the other (`at0` + 8 (r / 4) + r % 4).
// th (backward): tanh of the capped score.
template <bool GENERAL>
__device__ __forceinline__ void scores(const AttnArgs& a, f32x16& s, float slope2, int dist0, f32x16* th = nullptr) {
    if (!GENERAL) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= a.alpha * LOG2E;
        return;
    }
    if (a.cap > 0.f) {
        // tanh(x) = 1 - 2 / (exp(2x) + 1): an absolute error of 1e-7, which is what counts for a score
        const float k = a.alpha / a.cap * (2.f * LOG2E), c = a.cap * LOG2E;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float t = fmaf(-2.f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[r] * k) + 1.f), 1.f);
            if (th) (*th)[r] = t;
            s[r] = c * t;
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= a.alpha * LOG2E;
    }
    if (a.slopes) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = fmaf(-slope2, (float)abs(dist0 + 8 * (r >> 2) + (r & 3)), s[r]);
    }
}

// ------------------------------------------------------------------------------------------------ staging
// ROWS rows of a matrix from `row0` on, columns [0, d), into registers; rows outside [0, rows) and columns from d on are zero.
template <int D, int ROWS>
struct Stage {
    static constexpr int ROWB = D <= 64 ? 128 : 256, C = ROWB / 16, N = ROWS * C / MA_THREADS;
    u32x4m               r[N];
    __device__ __forceinline__ void load(const uint16_t* M, int ld, int row0, int rows, int d) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int v = threadIdx.x + MA_THREADS * j, row = row0 + v / C, col = (v % C) * 8;
            r[j]        = u32x4m{0u, 0u, 0u, 0u};
            if (row < rows && col < d) r[j] = *reinterpret_cast<const u32x4m*>(M + (long long)row * ld + col);
        }
    }
    __device__ __forceinline__ void store(char* X) const {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int v = threadIdx.x + MA_THREADS * j;
            *reinterpret_cast<u32x4m*>(LdsTile<ROWB>::piece(X, v / C, v % C)) = r[j];
        }
    }
    // Zeroes non-finite elements; bad (may be null): per row, NaN if it had one, else 0.
    __device__ __forceinline__ void clean(float* bad) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            bool any = false;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const unsigned x = r[j][w];
                const bool     l = (x & 0x7C00u) == 0x7C00u, h = (x & 0x7C000000u) == 0x7C000000u;
                r[j][w]          = x & ((l ? 0u : 0xFFFFu) | (h ? 0u : 0xFFFF0000u));
                any |= l | h;
            }
            if (bad) {  // the C pieces of a row are with C neighbouring lanes
                const unsigned long long m    = __ballot(any);
                const int                lane = threadIdx.x & 63, first = lane / C * C;
                if (lane == first) bad[(threadIdx.x + MA_THREADS * j) / C] = (m >> first) & ((1ull << C) - 1) ? NAN : 0.f;
            }
        }
    }
};

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

// What the keys of 128 queries are: of the workgroup and of this wave's 32.
struct QueryRange {
    int lo, hi;                        // this lane's query
    int wlo, whi, wlo_max, whi_min;    // the wave's
    int glo, ghi, glo_max, ghi_min;    // the workgroup's
};
__device__ __forceinline__ QueryRange query_range(const AttnArgs& a, int m, int m0) {
    QueryRange x;
    const int2 r = m < a.rows_q ? a.range[m] : make_int2(0, 0);
    x.lo         = max(r.x, 0);
    x.hi         = min(r.y, a.rows_k);
    if (x.lo >= x.hi) x.lo = x.hi = 0;
    const bool some = x.lo < x.hi;
    x.wlo = some ? x.lo : INT_MAX, x.whi = some ? x.hi : 0, x.wlo_max = some ? x.lo : INT_MAX, x.whi_min = some ? x.hi : 0;
#pragma unroll
    for (int s = 1; s < 32; s *= 2) {
        x.wlo     = min(x.wlo, __shfl_xor(x.wlo, s, 64));
        x.whi     = max(x.whi, __shfl_xor(x.whi, s, 64));
        x.wlo_max = max(x.wlo_max, __shfl_xor(x.wlo_max, s, 64));
        x.whi_min = min(x.whi_min, __shfl_xor(x.whi_min, s, 64));
    }
    x.wlo     = __builtin_amdgcn_readfirstlane(x.wlo);
    x.whi     = __builtin_amdgcn_readfirstlane(x.whi);
    x.wlo_max = __builtin_amdgcn_readfirstlane(x.wlo_max);
    x.whi_min = __builtin_amdgcn_readfirstlane(x.whi_min);
    int4 t    = a.tile[m0 / 64];
    if (m0 + 64 < a.rows_q) {
        const int4 u = a.tile[m0 / 64 + 1];
        t            = make_int4(min(t.x, u.x), max(t.y, u.y), max(t.z, u.z), min(t.w, u.w));
    } else {
        t.z = INT_MAX;  // rows behind the last one: not whole
    }
    x.glo = max(t.x, 0), x.ghi = min(t.y, a.rows_k), x.glo_max = t.z, x.ghi_min = t.w;
    return x;
}

// ------------------------------------------------------------------------------------------------ forward
template <int D, bool GENERAL>
__global__ __launch_bounds__(MA_THREADS, 2) void masked_fwd_kernel(AttnArgs a) {
    constexpr int KK = D / 16, DT = D / 32;
    typedef Stage<D, MA_K>        St;
    typedef LdsTile<St::ROWB>     Tile;
    __shared__ __align__(16) char Ks[MA_K * St::ROWB], Vs[MA_K * St::ROWB];
    __shared__ float              bad[MA_K];

    const int tiles = (a.rows_q + MA_Q - 1) / MA_Q;
    const int h = blockIdx.x % a.heads, qt = tiles - 1 - blockIdx.x / a.heads, kvh = h / a.group;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hf = lane >> 5;
    const int m0 = qt * MA_Q, m = m0 + 32 * wave + (lane & 31);
    const QueryRange x = query_range(a, m, m0);
    const uint16_t*  K = a.k + kvh * a.d;
    const uint16_t*  V = a.v + kvh * a.d;

    f16x8 qf[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        u32x4m p = {0u, 0u, 0u, 0u};
        if (m < a.rows_q && 16 * kk + 8 * hf < a.d) p = *reinterpret_cast<const u32x4m*>(a.q + (long long)m * a.ld_q + h * a.d + 16 * kk + 8 * hf);
        qf[kk] = frag8(p);
    }
    const float slope2 = GENERAL && a.slopes ? a.slopes[h] * LOG2E : 0.f;
    f32x16      o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = zero16();
    float mx = -INFINITY, sum = 0.f;

    St rk, rv;
    if (x.glo < x.ghi) {
        rk.load(K, a.ld_k, x.glo, a.rows_k, a.d);
        rv.load(V, a.ld_v, x.glo, a.rows_k, a.d);
    }
    for (int kb = x.glo; kb < x.ghi; kb += MA_K) {
        const bool whole = x.glo_max <= kb && x.ghi_min >= kb + MA_K;
        __syncthreads();  // every wave is done with the tile before
        if (!whole) rv.clean(bad);
        rk.store(Ks);
        rv.store(Vs);
        __syncthreads();
        if (kb + MA_K < x.ghi) {
            rk.load(K, a.ld_k, kb + MA_K, a.rows_k, a.d);
            rv.load(V, a.ld_v, kb + MA_K, a.rows_k, a.d);
        }
        if (x.wlo >= kb + MA_K || x.whi <= kb) continue;  // nothing for this wave
        f32x16 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = zero16();
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
                s[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(Tile::frag(Ks, 32 * t + (lane & 31), kk, hf), qf[kk], s[t], 0, 0, 0);
            scores<GENERAL>(a, s[t], slope2, kb + 32 * t + 4 * hf - m);
        }
        if (!whole) {  // (also where this wave's own queries see all of it: values were zeroed)
            const bool     mine = x.wlo_max <= kb && x.whi_min >= kb + MA_K;
            const int      n0   = kb + 4 * hf - x.lo;
            const unsigned len  = x.hi - x.lo;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int n = 32 * t + 8 * (r >> 2) + (r & 3);
                    s[t][r] += bad[n + 4 * hf];
                    if (!mine) s[t][r] = (unsigned)(n0 + n) < len ? s[t][r] : -INFINITY;
                }
        }
        float top = mx;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
        top              = join_halves(top, [](float p, float q) { return fmaxf(p, q); });
        const float base = top == -INFINITY ? 0.f : top;  // (nothing seen yet: exp(-inf - 0) = 0)
        const float fix  = __builtin_amdgcn_exp2f(mx - base);
        mx               = top;
        sum *= fix;
        unsigned pk[2][8];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float p0 = __builtin_amdgcn_exp2f(s[t][2 * e] - base), p1 = __builtin_amdgcn_exp2f(s[t][2 * e + 1] - base);
                sum += p0 + p1;
                pk[t][e] = pack_f16(p0, p1);
            }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] *= fix;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(Tile::frag_t(Vs, 32 * dt, 32 * t + 16 * u + 4 * hf, lane),
                                                                   frag8(u32x4m{pk[t][4 * u], pk[t][4 * u + 1], pk[t][4 * u + 2], pk[t][4 * u + 3]}),
                                                                   o[dt], 0, 0, 0);
        }
    }
    sum = join_halves(sum, [](float p, float q) { return p + q; });
    if (m < a.rows_q && hf == 0) a.lse[(long long)h * a.rows_q + m] = sum == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * LN2;
    store_rows<DT>(m < a.rows_q ? a.out + (long long)m * a.ld_ctx + h * a.d : nullptr, o, sum == 0.f ? 0.f : 1.f / sum, a.d, hf);
}

// ------------------------------------------------------------------------------------------------ backward
// Row statistics: lse in base 2 (+inf where a row sees nothing: its probabilities are then 0; NaN where it or delta is not a number
// to go by) and delta.  16 lanes a (row, head) pair.
__global__ __launch_bounds__(MA_THREADS) void masked_stats_kernel(AttnArgs a) {
    const long long pair = (long long)blockIdx.x * (MA_THREADS / 16) + (threadIdx.x >> 4);
    const int       row = (int)(pair / a.heads), h = (int)(pair - (long long)row * a.heads), c = (threadIdx.x & 15) * 8;
    if (row >= a.rows_pad) return;
    float s = 0.f;
    if (row < a.rows_q && c < a.d) {
        const f16x8 p = *reinterpret_cast<const f16x8*>(a.ctx + (long long)row * a.ld_ctx + h * a.d + c);
        const f16x8 g = *reinterpret_cast<const f16x8*>(a.dctx + (long long)row * a.ld_dctx + h * a.d + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf((float)p[i], (float)g[i], s);
    }
#pragma unroll
    for (int i = 1; i < 16; i *= 2) s += __shfl_xor(s, i, 64);
    if (threadIdx.x & 15) return;
    float l = INFINITY;
    if (row < a.rows_q) {
        const int2 r = a.range[row];
        l            = a.lse_in[(long long)h * a.rows_q + row] * LOG2E;
        if (max(r.x, 0) >= min(r.y, a.rows_k) || l == -INFINITY)
            l = INFINITY, s = 0.f;
        else if (!(fabsf(l) < INFINITY && fabsf(s) < INFINITY))
            l = NAN, s = 0.f;
    }
    a.lse2[(long long)h * a.rows_pad + row]  = l;
    a.delta[(long long)h * a.rows_pad + row] = s;
}

// dq of 128 queries: the forward kernel's walk over the keys.
template <int D, bool GENERAL>
__global__ __launch_bounds__(MA_THREADS, 2) void masked_dq_kernel(AttnArgs a) {
    constexpr int KK = D / 16, DT = D / 32;
    typedef Stage<D, MA_K>        St;
    typedef LdsTile<St::ROWB>     Tile;
    __shared__ __align__(16) char Ks[MA_K * St::ROWB], Vs[MA_K * St::ROWB];

    const int tiles = (a.rows_q + MA_Q - 1) / MA_Q;
    const int h = blockIdx.x % a.heads, qt = tiles - 1 - blockIdx.x / a.heads, kvh = h / a.group;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hf = lane >> 5;
    const int m0 = qt * MA_Q, m = m0 + 32 * wave + (lane & 31);
    const QueryRange x = query_range(a, m, m0);
    const uint16_t*  K = a.k + kvh * a.d;
    const uint16_t*  V = a.v + kvh * a.d;

    f16x8 qf[KK], gf[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        u32x4m p = {0u, 0u, 0u, 0u}, g = p;
        if (m < a.rows_q && 16 * kk + 8 * hf < a.d) {
            p = *reinterpret_cast<const u32x4m*>(a.q + (long long)m * a.ld_q + h * a.d + 16 * kk + 8 * hf);
            g = *reinterpret_cast<const u32x4m*>(a.dctx + (long long)m * a.ld_dctx + h * a.d + 16 * kk + 8 * hf);
        }
        qf[kk] = frag8(p);
        gf[kk] = frag8(g);
    }
    const float slope2 = GENERAL && a.slopes ? a.slopes[h] * LOG2E : 0.f;
    float       lse2 = INFINITY, delta = 0.f;
    if (m < a.rows_q) {
        lse2  = a.lse2[(long long)h * a.rows_pad + m];
        delta = a.delta[(long long)h * a.rows_pad + m];
    }
    f32x16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = zero16();

    St rk, rv;
    if (x.glo < x.ghi) {
        rk.load(K, a.ld_k, x.glo, a.rows_k, a.d);
        rv.load(V, a.ld_v, x.glo, a.rows_k, a.d);
    }
    for (int kb = x.glo; kb < x.ghi; kb += MA_K) {
        const bool whole = x.glo_max <= kb && x.ghi_min >= kb + MA_K;
        __syncthreads();
        if (!whole) {
            rk.clean(nullptr);
            rv.clean(nullptr);
        }
        rk.store(Ks);
        rv.store(Vs);
        __syncthreads();
        if (kb + MA_K < x.ghi) {
            rk.load(K, a.ld_k, kb + MA_K, a.rows_k, a.d);
            rv.load(V, a.ld_v, kb + MA_K, a.rows_k, a.d);
        }
        if (x.wlo >= kb + MA_K || x.whi <= kb) continue;
        const bool     mine = x.wlo_max <= kb && x.whi_min >= kb + MA_K;
        const int      n0   = kb + 4 * hf - x.lo;
        const unsigned len  = x.hi - x.lo;
        unsigned       ds[2][8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x16 s = zero16(), dp = zero16(), th;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                s  = __builtin_amdgcn_mfma_f32_32x32x16_f16(Tile::frag(Ks, 32 * t + (lane & 31), kk, hf), qf[kk], s, 0, 0, 0);
                dp = __builtin_amdgcn_mfma_f32_32x32x16_f16(Tile::frag(Vs, 32 * t + (lane & 31), kk, hf), gf[kk], dp, 0, 0, 0);
            }
            scores<GENERAL>(a, s, slope2, kb + 32 * t + 4 * hf - m, &th);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float p = __builtin_amdgcn_exp2f(s[r] - lse2);
                if (!mine) p = (unsigned)(n0 + 32 * t + 8 * (r >> 2) + (r & 3)) < len ? p : 0.f;
                float d = p * (dp[r] - delta);
                if (GENERAL && a.cap > 0.f) d *= fmaf(-th[r], th[r], 1.f);
                s[r] = d;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) ds[t][e] = pack_f16(s[2 * e], s[2 * e + 1]);
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(Tile::frag_t(Ks, 32 * dt, 32 * t + 16 * u + 4 * hf, lane),
                                                                   frag8(u32x4m{ds[t][4 * u], ds[t][4 * u + 1], ds[t][4 * u + 2], ds[t][4 * u + 3]}),
                                                                   o[dt], 0, 0, 0);
    }
    // (a row that sees nothing may hold anything in q and dctx, and 0 x NaN has reached its sums)
    if (x.lo >= x.hi) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = zero16();
    }
    store_rows<DT>(m < a.rows_q ? a.dq + (long long)m * a.ld_dq + h * a.d : nullptr, o, a.alpha, a.d, hf);
}

// dk and dv of 128 keys: 32 of them a wave, over the tiles of 64 queries that see any of them, head by head.
template <int D, bool GENERAL>
__global__ __launch_bounds__(MA_THREADS, 1) void masked_dkv_kernel(AttnArgs a) {
    constexpr int KK = D / 16, DT = D / 32;
    typedef Stage<D, MA_K>        St;
    typedef LdsTile<St::ROWB>     Tile;
    __shared__ __align__(16) char Qs[MA_K * St::ROWB], Gs[MA_K * St::ROWB];
    __shared__ __align__(16) float lse2[MA_K], delta[MA_K];
    __shared__ __align__(16) int   los[MA_K], lens[MA_K];

    const int kv_heads = a.heads / a.group, kvh = blockIdx.x % kv_heads, kt = blockIdx.x / kv_heads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hf = lane >> 5;
    const int k0 = kt * MA_Q, n0 = k0 + 32 * wave, n = n0 + (lane & 31);
    const int qtiles = (a.rows_q + MA_K - 1) / MA_K;

    f16x8 kf[KK], vf[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        u32x4m p = {0u, 0u, 0u, 0u}, g = p;
        if (n < a.rows_k && 16 * kk + 8 * hf < a.d) {
            p = *reinterpret_cast<const u32x4m*>(a.k + (long long)n * a.ld_k + kvh * a.d + 16 * kk + 8 * hf);
            g = *reinterpret_cast<const u32x4m*>(a.v + (long long)n * a.ld_v + kvh * a.d + 16 * kk + 8 * hf);
        }
        kf[kk] = frag8(p);
        vf[kk] = frag8(g);
    }
    f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dk[dt] = dv[dt] = zero16();

    St rq, rg;
    for (int h = kvh * a.group; h < (kvh + 1) * a.group; ++h) {
        const uint16_t* Q      = a.q + h * a.d;
        const uint16_t* G      = a.dctx + h * a.d;
        const float     slope2 = GENERAL && a.slopes ? a.slopes[h] * LOG2E : 0.f;
        for (int base = 0; base < qtiles; base += 64) {
            int4 mine = make_int4(INT_MAX, 0, INT_MAX, 0);
            if (base + lane < qtiles) mine = a.tile[base + lane];
            unsigned long long todo = __ballot(mine.x < k0 + MA_Q && mine.y > k0);  // (the same in every wave)
            bool               have = false;
            while (todo) {
                const int i = __builtin_ctzll(todo);
                todo &= todo - 1;
                const int q0 = (base + i) * MA_K;
                if (!have) {
                    rq.load(Q, a.ld_q, q0, a.rows_q, a.d);
                    rg.load(G, a.ld_dctx, q0, a.rows_q, a.d);
                }
                const int4 t4 = make_int4(__builtin_amdgcn_readlane(mine.x, i), __builtin_amdgcn_readlane(mine.y, i),
                                          __builtin_amdgcn_readlane(mine.z, i), __builtin_amdgcn_readlane(mine.w, i));
                const bool whole = t4.z <= k0 && t4.w >= k0 + MA_Q && q0 + MA_K <= a.rows_q;
                __syncthreads();
                if (!whole) {
                    rq.clean(nullptr);
                    rg.clean(nullptr);
                }
                rq.store(Qs);
                rg.store(Gs);
                if (threadIdx.x < MA_K) {
                    const int  m = q0 + threadIdx.x;
                    const int2 r = m < a.rows_q ? a.range[m] : make_int2(0, 0);
                    los[threadIdx.x]   = r.x;
                    lens[threadIdx.x]  = max(r.y - r.x, 0);
                    lse2[threadIdx.x]  = a.lse2[(long long)h * a.rows_pad + m];
                    delta[threadIdx.x] = a.delta[(long long)h * a.rows_pad + m];
                }
                __syncthreads();
                have = todo != 0;
                if (have) {
                    const int next = (base + __builtin_ctzll(todo)) * MA_K;
                    rq.load(Q, a.ld_q, next, a.rows_q, a.d);
                    rg.load(G, a.ld_dctx, next, a.rows_q, a.d);
                }
                if (t4.x >= n0 + 32 || t4.y <= n0) continue;
                const bool all = t4.z <= n0 && t4.w >= n0 + 32 && q0 + MA_K <= a.rows_q;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    f32x16 s = zero16(), dp = zero16(), th;
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk) {
                        s  = __builtin_amdgcn_mfma_f32_32x32x16_f16(Tile::frag(Qs, 32 * t + (lane & 31), kk, hf), kf[kk], s, 0, 0, 0);
                        dp = __builtin_amdgcn_mfma_f32_32x32x16_f16(Tile::frag(Gs, 32 * t + (lane & 31), kk, hf), vf[kk], dp, 0, 0, 0);
                    }
                    scores<GENERAL>(a, s, slope2, q0 + 32 * t + 4 * hf - n, &th);
                    unsigned pk[8], dsk[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int   i0 = 32 * t + 8 * e + 4 * hf;
                        const f32x4 l4 = *reinterpret_cast<const f32x4*>(lse2 + i0), d4 = *reinterpret_cast<const f32x4*>(delta + i0);
                        float       p[4], d[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const int r = 4 * e + c;
                            p[c]        = __builtin_amdgcn_exp2f(s[r] - l4[c]);
                            d[c]        = p[c] * (dp[r] - d4[c]);
                            if (GENERAL && a.cap > 0.f) d[c] *= fmaf(-th[r], th[r], 1.f);
                            if (!all) {  // (this lane's key may be one that holds anything)
                                const bool seen = (unsigned)(n - los[i0 + c]) < (unsigned)lens[i0 + c];
                                p[c]            = seen ? p[c] : 0.f;
                                d[c]            = seen ? d[c] : 0.f;
                            }
                        }
                        pk[2 * e]      = pack_f16(p[0] * P_SCALE, p[1] * P_SCALE);
                        pk[2 * e + 1]  = pack_f16(p[2] * P_SCALE, p[3] * P_SCALE);
                        dsk[2 * e]     = pack_f16(d[0], d[1]);
                        dsk[2 * e + 1] = pack_f16(d[2], d[3]);
                    }
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const int i0 = 32 * t + 16 * u + 4 * hf;
                            dv[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(Tile::frag_t(Gs, 32 * dt, i0, lane),
                                                                            frag8(u32x4m{pk[4 * u], pk[4 * u + 1], pk[4 * u + 2], pk[4 * u + 3]}), dv[dt], 0, 0, 0);
                            dk[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(Tile::frag_t(Qs, 32 * dt, i0, lane),
                                                                            frag8(u32x4m{dsk[4 * u], dsk[4 * u + 1], dsk[4 * u + 2], dsk[4 * u + 3]}), dk[dt], 0, 0, 0);
                        }
                }
            }
        }
    }
    const bool in = n < a.rows_k;
    store_rows<DT>(in ? a.dv + (long long)n * a.ld_dv + kvh * a.d : nullptr, dv, 1.f / P_SCALE, a.d, hf);
    store_rows<DT>(in ? a.dk + (long long)n * a.ld_dk + kvh * a.d : nullptr, dk, a.alpha, a.d, hf);
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
    if (d->d_head > 128 || (d->d_head & 7)) {
        set_error("%s: head size %d is not a multiple of 8 up to 128", who, d->d_head);
        return MP_E_UNSUPPORTED;
    }
    const long long w = (long long)d->n_heads * d->d_head, wk = (long long)d->n_kv_heads * d->d_head;
    MP_REQUIRE(w < (1 << 24), "%s: too many heads", who);
    MP_REQUIRE(d->rows_q <= 0x7FFFFF00 && d->rows_k <= 0x7FFFFF00, "%s: too many rows", who);
    MP_REQUIRE(((long long)d->rows_q + MA_Q) / MA_Q * d->n_heads < (1ll << 31) && ((long long)d->rows_k + MA_Q) / MA_Q * d->n_heads < (1ll << 31),
               "%s: too many rows and heads", who);
    MP_REQUIRE(d->ld_q >= w && d->ld_k >= wk && d->ld_v >= wk && d->ld_ctx >= w, "%s: a leading dimension is smaller than its rows", who);
    if ((d->ld_q | d->ld_k | d->ld_v | d->ld_ctx) & 7) {
        set_error("%s: leading dimensions must be multiples of 8", who);
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
    AttnArgs a = {};
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
// The kernel of the head size (rounded up to a multiple of 32) and of plain or general scores.
#define MA_LAUNCH(kernel, grid, a, hs)                                                                       \
    do {                                                                                                     \
        const bool general = (a).cap > 0.f || (a).slopes;                                                    \
        const dim3 g((unsigned)(grid)), b(MA_THREADS);                                                       \
        switch (((a).d + 31) / 32 * 2 + general) {                                                           \
            case 2: hipLaunchKernelGGL((kernel<32, false>), g, b, 0, hs, a); break;                          \
            case 3: hipLaunchKernelGGL((kernel<32, true>), g, b, 0, hs, a); break;                           \
            case 4: hipLaunchKernelGGL((kernel<64, false>), g, b, 0, hs, a); break;                          \
            case 5: hipLaunchKernelGGL((kernel<64, true>), g, b, 0, hs, a); break;                           \
            case 6: hipLaunchKernelGGL((kernel<96, false>), g, b, 0, hs, a); break;                          \
            case 7: hipLaunchKernelGGL((kernel<96, true>), g, b, 0, hs, a); break;                           \
            case 8: hipLaunchKernelGGL((kernel<128, false>), g, b, 0, hs, a); break;                         \
            default: hipLaunchKernelGGL((kernel<128, true>), g, b, 0, hs, a); break;                         \
        }                                                                                                    \
    } while (0)

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
    MA_LAUNCH(masked_fwd_kernel, (long long)((desc->rows_q + MA_Q - 1) / MA_Q) * desc->n_heads, a, as_stream(stream));
    MP_LAUNCH_CHECK(who);
    return MP_OK;
}

extern "C" size_t mp_attention_masked_bwd_workspace_bytes(const mp_attn_desc* desc) {
    if (check_desc("mp_attention_masked_bwd_workspace_bytes", desc) != MP_OK) return 0;
    return (size_t)rows64(desc->rows_q) * 64 * desc->n_heads * 2 * sizeof(float) + 256;
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
    if ((d.ld_dq | d.ld_dk | d.ld_dv | d.ld_dctx) & 7) {
        set_error("%s: leading dimensions must be multiples of 8", who);
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
    if (d.rows_q > 0) {
        const long long pairs = (long long)a.rows_pad * a.heads, per = MA_THREADS / 16;
        hipLaunchKernelGGL(masked_stats_kernel, dim3((unsigned)((pairs + per - 1) / per)), dim3(MA_THREADS), 0, hs, a);
        MP_LAUNCH_CHECK(who);
        MA_LAUNCH(masked_dq_kernel, (long long)((d.rows_q + MA_Q - 1) / MA_Q) * d.n_heads, a, hs);
        MP_LAUNCH_CHECK(who);
    }
    if (d.rows_k > 0) {
        MA_LAUNCH(masked_dkv_kernel, (long long)((d.rows_k + MA_Q - 1) / MA_Q) * d.n_kv_heads, a, hs);
        MP_LAUNCH_CHECK(who);
    }
    return MP_OK;
}
