// Queries and keys before attention: the RMS norm of each head and the rotation of its pairs by position, in one pass each way.
//
// With x one head's d values, r = (mean x^2 + eps)^-1/2, x^ = x r and n = g x^, a pair (a, b) of n at the angle t becomes
// (a cos t - b sin t, a sin t + b cos t).  Backward with u = the gradient turned back by -t: dg = sum u x^, v = u g,
// dx = r (v - x^ mean(v x^)); r is formed again from x, so forward keeps nothing.
//
// Bound by HBM: forward moves 4 bytes, backward 6 bytes an element.  The angle depends on token and pair only, so a workgroup takes
// some tokens, forms their cosines and sines once into LDS, and all heads of these tokens read them there.
// A lane owns "units" of 2 W columns: W and their partners where halves are paired, 2 W neighbours where neighbours are; a head
// is then d / (2 W) lanes, filled up to a power of two, whose sums go through lane permutations.
#include <cmath>

#include "common.hpp"

namespace mp {

constexpr int RO_THREADS = 256;
constexpr int RO_WAVES   = RO_THREADS / 64;

template <int W>
__device__ __forceinline__ void load_piece(const uint16_t* p, float* f) {
    typedef f16 vec __attribute__((ext_vector_type(W)));
    const vec   q = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int k = 0; k < W; ++k) f[k] = (float)q[k];
}
template <int W>
__device__ __forceinline__ void store_piece(uint16_t* p, const float* f) {
    typedef f16 vec __attribute__((ext_vector_type(W)));
    vec         q;
#pragma unroll
    for (int k = 0; k < W; ++k) q[k] = (f16)f[k];
    *reinterpret_cast<vec*>(p) = q;
}

// Sum over aligned groups of `lanes` lanes (a power of two, the same for the whole launch); all of a group get it.
__device__ __forceinline__ float group_sum(float v, const int lanes) {
    const auto dpp = [&](auto ctrl) {
        const int i = __builtin_bit_cast(int, v);
        v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, decltype(ctrl)::value, 0xF, 0xF, false));
    };
    const auto swap = [&](const auto r) {
        const unsigned a = r[0], b = r[1];
        v                = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
    };
    if (lanes > 1) dpp(std::integral_constant<int, 0xB1>{});    // quad: lanes 1 0 3 2
    if (lanes > 2) dpp(std::integral_constant<int, 0x4E>{});    // quad: lanes 2 3 0 1
    if (lanes > 4) dpp(std::integral_constant<int, 0x141>{});   // mirror of 8 lanes (quads are alike by now)
    if (lanes > 8) dpp(std::integral_constant<int, 0x140>{});   // mirror of 16
    if (lanes > 16) swap(__builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false));
    if (lanes > 32) swap(__builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false));
    return v;
}

struct RopeArgs {
    int             rows, d, rot, units, lanes;  // units a head, lanes a head (units rounded up to a power of two)
    int             tokens;                      // a workgroup's
    float           eps;
    const int32_t*  positions;                   // [axes][rows]
    const double*   freqs;                       // [rot / 2]
    struct Part {
        int             heads, ld_x, ld_y, ld_d; // x, y / dy, dx
        const uint16_t *x, *g, *dy;
        uint16_t *      y, *dx;
    } part[2];                                   // queries, keys
    float*  sums;                                // backward: [workgroups][2][d]
    uint8_t axis[MP_ROPE_PAIRS];
};

// Cosines and sines of `tokens` tokens from `first` on, [token][pair] each.  Angles in revolutions and 64 bits: a position of 2^31 still
// has its angle to 2^-20, where a product in 32 bits has lost it at some thousands.
__device__ __forceinline__ void rope_angles(const RopeArgs& a, const int first, const int tokens, float* cosines, float* sines) {
    const int pairs = a.rot >> 1;
    for (int e = threadIdx.x; e < tokens * pairs; e += RO_THREADS) {
        const int t = e / pairs, i = e - t * pairs;
        double    turn = (double)a.positions[(long long)a.axis[i] * a.rows + first + t] * (a.freqs[i] * 0.15915494309189533577);
        turn -= rint(turn);
        float s, c;
        sincospif(2.0f * (float)turn, &s, &c);
        cosines[e] = c;
        sines[e]   = s;
    }
}

// Where a lane's unit lies: columns of its two pieces, and the first of its W pairs (or -1: columns that are not turned).
template <int W, bool ADJ>
struct Unit {
    int  col0, col1, pair;
    bool there;
    __device__ __forceinline__ Unit(const RopeArgs& a) {
        const int u      = threadIdx.x & (a.lanes - 1);
        const int turned = a.rot / (2 * W);
        there            = u < a.units;
        pair             = u < turned ? u * W : -1;
        if (ADJ || u >= turned) {
            col0 = u * 2 * W;
            col1 = col0 + W;
        } else {
            col0 = u * W;
            col1 = col0 + (a.rot >> 1);
        }
    }
};

// The unit's values turned by the angles at c and s (SIGN -1: back).
template <int W, bool ADJ, int SIGN>
__device__ __forceinline__ void turn_unit(float* f, const float* c, const float* s) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
        float&      x0 = f[ADJ ? 2 * k : k];
        float&      x1 = f[ADJ ? 2 * k + 1 : W + k];
        const float sn = SIGN * s[k], y0 = x0 * c[k] - x1 * sn, y1 = x0 * sn + x1 * c[k];
        x0 = y0;
        x1 = y1;
    }
}

// Items of a workgroup: (token, head) with the heads fastest, one to a group of `lanes` lanes.
struct Items {
    int token, head, step_token, step_head, heads;
    __device__ __forceinline__ Items(int group, int groups, int heads_)
        : token(group / heads_), head(group - token * heads_), step_token(groups / heads_), step_head(groups - step_token * heads_), heads(heads_) {}
    __device__ __forceinline__ void next() {
        token += step_token;
        head += step_head;
        if (head >= heads) {
            head -= heads;
            ++token;
        }
    }
};

template <int W, bool ADJ, bool NORM>
__global__ __launch_bounds__(RO_THREADS) void rope_fwd_kernel(const RopeArgs a) {
    extern __shared__ float lds[];
    const int    first = blockIdx.x * a.tokens, tokens = min(a.tokens, a.rows - first), pairs = a.rot >> 1;
    float *const cosines = lds, *const sines = lds + a.tokens * pairs;
    rope_angles(a, first, tokens, cosines, sines);
    __syncthreads();
    const Unit<W, ADJ> at(a);
    const int          group = threadIdx.x / a.lanes, groups = RO_THREADS / a.lanes;
    const float        inv   = 1.0f / (float)a.d;
    for (int p = 0; p < 2; ++p) {
        const RopeArgs::Part& h = a.part[p];
        float                 g[2 * W];
        if (NORM && at.there) {
            load_piece<W>(h.g + at.col0, g);
            load_piece<W>(h.g + at.col1, g + W);
        }
        for (Items it(group, groups, h.heads); it.token < tokens; it.next()) {
            float f[2 * W];
#pragma unroll
            for (int k = 0; k < 2 * W; ++k) f[k] = 0.f;
            if (at.there) {
                const uint16_t* x = h.x + (long long)(first + it.token) * h.ld_x + it.head * a.d;
                load_piece<W>(x + at.col0, f);
                load_piece<W>(x + at.col1, f + W);
            }
            if (NORM) {
                float q = 0.f;
#pragma unroll
                for (int k = 0; k < 2 * W; ++k) q += f[k] * f[k];
                const float r = rsqrtf(group_sum(q, a.lanes) * inv + a.eps);
#pragma unroll
                for (int k = 0; k < 2 * W; ++k) f[k] = f[k] * r * g[k];
            }
            if (at.pair >= 0) {
                const int e = it.token * pairs + at.pair;
                turn_unit<W, ADJ, 1>(f, cosines + e, sines + e);
            }
            if (at.there) {
                uint16_t* y = h.y + (long long)(first + it.token) * h.ld_y + it.head * a.d;
                store_piece<W>(y + at.col0, f);
                store_piece<W>(y + at.col1, f + W);
            }
        }
    }
}

// Workgroups take blocks of tokens in turn, so that the weights' gradients are few partial rows: [workgroup][queries, keys][d].
template <int W, bool ADJ, bool NORM>
__global__ __launch_bounds__(RO_THREADS) void rope_bwd_kernel(const RopeArgs a) {
    extern __shared__ float lds[];
    const int          pairs = a.rot >> 1;
    float *const       cosines = lds, *const sines = lds + a.tokens * pairs;
    const Unit<W, ADJ> at(a);
    const int          group = threadIdx.x / a.lanes, groups = RO_THREADS / a.lanes;
    const float        inv   = 1.0f / (float)a.d;
    float              acc[2][NORM ? 2 * W : 1], g[2][NORM ? 2 * W : 1];
    if (NORM) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int k = 0; k < 2 * W; ++k) acc[p][k] = g[p][k] = 0.f;
            if (at.there) {
                load_piece<W>(a.part[p].g + at.col0, g[p]);
                load_piece<W>(a.part[p].g + at.col1, g[p] + W);
            }
        }
    }
    for (long long first = (long long)blockIdx.x * a.tokens; first < a.rows; first += (long long)gridDim.x * a.tokens) {
        const int tokens = min((long long)a.tokens, a.rows - first);
        __syncthreads();
        rope_angles(a, (int)first, tokens, cosines, sines);
        __syncthreads();
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const RopeArgs::Part& h = a.part[p];
            for (Items it(group, groups, h.heads); it.token < tokens; it.next()) {
                float f[2 * W], x[NORM ? 2 * W : 1];
                if (at.there) {
                    const uint16_t* dy = h.dy + (first + it.token) * h.ld_y + it.head * a.d;
                    load_piece<W>(dy + at.col0, f);
                    load_piece<W>(dy + at.col1, f + W);
                    if (NORM) {
                        const uint16_t* xs = h.x + (first + it.token) * h.ld_x + it.head * a.d;
                        load_piece<W>(xs + at.col0, x);
                        load_piece<W>(xs + at.col1, x + W);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 2 * W; ++k) f[k] = 0.f;
                    if (NORM) {
#pragma unroll
                        for (int k = 0; k < 2 * W; ++k) x[k] = 0.f;
                    }
                }
                if (at.pair >= 0) {
                    const int e = it.token * pairs + at.pair;
                    turn_unit<W, ADJ, -1>(f, cosines + e, sines + e);
                }
                if (NORM) {
                    float q = 0.f, vx = 0.f;
#pragma unroll
                    for (int k = 0; k < 2 * W; ++k) {
                        q += x[k] * x[k];
                        vx += f[k] * g[p][k] * x[k];
                    }
                    const float r = rsqrtf(group_sum(q, a.lanes) * inv + a.eps);
                    const float m = group_sum(vx, a.lanes) * inv * r * r;  // mean(v x^) r
#pragma unroll
                    for (int k = 0; k < 2 * W; ++k) {
                        acc[p][k] += f[k] * (x[k] * r);
                        f[k] = r * (f[k] * g[p][k] - x[k] * m);
                    }
                }
                if (at.there) {
                    uint16_t* dx = h.dx + (first + it.token) * h.ld_d + it.head * a.d;
                    store_piece<W>(dx + at.col0, f);
                    store_piece<W>(dx + at.col1, f + W);
                }
            }
        }
    }
    if (NORM) {
        // lanes that own the same columns, then the waves, in order
        __syncthreads();
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int k = 0; k < 2 * W; ++k)
                for (int far = 32; far >= a.lanes; far >>= 1) acc[p][k] += __shfl_xor(acc[p][k], far, 64);
            if (at.there && lane < a.lanes) {
#pragma unroll
                for (int k = 0; k < 2 * W; ++k) lds[(wave * 2 + p) * a.d + (k < W ? at.col0 + k : at.col1 + k - W)] = acc[p][k];
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * a.d; c += RO_THREADS) {
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < RO_WAVES; ++w) t += lds[w * 2 * a.d + c];
            a.sums[(long long)blockIdx.x * 2 * a.d + c] = t;
        }
    }
}

// Column sums of the partial rows, 32 columns by 32 lanes of rows a workgroup, in a fixed order.
__global__ __launch_bounds__(1024) void rope_finish_kernel(const float* __restrict__ sums, const int nparts, const int d, uint16_t* dgq, uint16_t* dgk,
                                                           mp_scale_state* st) {
    __shared__ float sm[32][33];
    const int        cl = threadIdx.x & 31, q = threadIdx.x >> 5, c = blockIdx.x * 32 + cl;
    float            acc = 0.f;
    if (c < 2 * d) {
        for (int p = q; p < nparts; p += 32 * 8) {
            float t[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) t[u] = p + 32 * u < nparts ? sums[(long long)(p + 32 * u) * 2 * d + c] : 0.f;
#pragma unroll
            for (int u = 0; u < 8; ++u) acc += t[u];
        }
    }
    sm[q][cl] = acc;
    __syncthreads();
    bool bad = false;
    if (q == 0 && c < 2 * d) {
        float t = 0.f;
#pragma unroll
        for (int j = 0; j < 32; ++j) t += sm[j][cl];
        const uint16_t h = f2h(t);
        if (c < d) dgq[c] = h;
        else dgk[c - d] = h;
        bad = half_nonfinite(h);
    }
    if (st != nullptr && __any(bad)) {
        if ((threadIdx.x & 63) == 0) atomicOr(&st->found_inf, 1);
    }
}

}  // namespace mp

using namespace mp;

namespace {

// Tokens a workgroup takes at once: enough for its waves to have several items each, few enough that the launch fills the chip.
int rope_tokens(int rows) {
    int t = 16;
    while (t > 1 && (rows + t - 1) / t < 1024) t >>= 1;
    return t;
}
int rope_bwd_blocks(int rows) {
    const int t = rope_tokens(rows), n = (rows + t - 1) / t;
    return n < 1024 ? n : 1024;
}
size_t rope_bwd_bytes(const mp_rope_desc* d) { return (size_t)rope_bwd_blocks(d->rows) * 2 * d->d_head * sizeof(float); }

int rope_check(const mp_rope_desc* d, const char* what) {
    MP_REQUIRE(d, "%s: NULL argument", what);
    MP_REQUIRE(d->rows >= 0 && d->n_heads > 0 && d->n_kv_heads > 0 && d->d_head > 0, "%s: bad shape rows=%d heads=%d kv_heads=%d d_head=%d", what, d->rows,
               d->n_heads, d->n_kv_heads, d->d_head);
    MP_REQUIRE(d->rot > 0 && d->rot <= d->d_head && d->rot % 2 == 0, "%s: %d columns of %d to be turned", what, d->rot, d->d_head);
    MP_REQUIRE(d->n_axes > 0 && d->n_axes <= MP_ROPE_AXES, "%s: %d axes of positions", what, d->n_axes);
    MP_REQUIRE(d->adjacent == 0 || d->adjacent == 1, "%s: adjacent=%d", what, d->adjacent);
    MP_REQUIRE(d->reserved == 0, "%s: reserved field is not 0", what);
    MP_REQUIRE(d->eps >= 0.f && std::isfinite(d->eps), "%s: eps is negative or not finite", what);
    if (d->d_head % 8 != 0 || d->d_head > 2 * MP_ROPE_PAIRS || d->rot % 4 != 0) {
        set_error("%s: heads of %d with %d columns turned unsupported (multiples of 8 up to %d, of 4)", what, d->d_head, d->rot, 2 * MP_ROPE_PAIRS);
        return MP_E_UNSUPPORTED;
    }
    for (int i = 0; i < d->rot / 2; ++i) MP_REQUIRE(d->axis[i] < d->n_axes, "%s: pair %d follows axis %d of %d", what, i, d->axis[i], d->n_axes);
    return MP_OK;
}

int rope_matrix(const char* what, const char* name, const void* p, int ld, long long cols) {
    MP_REQUIRE(p, "%s: NULL argument", what);
    MP_REQUIRE(ld >= cols, "%s: leading dimension of %s is %d, of %lld columns", what, name, ld, cols);
    if (ld % 8 != 0 || !aligned16(p)) {
        set_error("%s: %s needs to be 16-byte aligned with a leading dimension that is a multiple of 8", what, name);
        return MP_E_UNSUPPORTED;
    }
    return MP_OK;
}

RopeArgs rope_args(const mp_rope_desc* d, int w, const int32_t* positions, const double* freqs) {
    RopeArgs a{};
    a.rows  = d->rows;
    a.d     = d->d_head;
    a.rot   = d->rot;
    a.units = d->d_head / (2 * w);
    a.lanes = 1;
    while (a.lanes < a.units) a.lanes *= 2;
    a.tokens    = rope_tokens(d->rows);
    a.eps       = d->eps;
    a.positions = positions;
    a.freqs     = freqs;
    for (int i = 0; i < d->rot / 2; ++i) a.axis[i] = d->axis[i];
    return a;
}

// the widest pieces that neither the turned columns nor the others cut
int rope_width(const mp_rope_desc* d) {
    if (d->d_head % 16 == 0 && d->rot % 16 == 0) return 8;
    return d->rot % 8 == 0 ? 4 : 2;
}

template <typename F>
int rope_dispatch(int w, bool adj, bool norm, F&& f) {
    const auto by_norm = [&](auto wc, auto ac) { return norm ? f(wc, ac, std::true_type{}) : f(wc, ac, std::false_type{}); };
    const auto by_adj  = [&](auto wc) { return adj ? by_norm(wc, std::true_type{}) : by_norm(wc, std::false_type{}); };
    if (w == 8) return by_adj(std::integral_constant<int, 8>{});
    if (w == 4) return by_adj(std::integral_constant<int, 4>{});
    return by_adj(std::integral_constant<int, 2>{});
}

}  // namespace

extern "C" int mp_qk_norm_rope_fwd(const mp_rope_desc* d, const mp_half* q, const mp_half* k, const mp_half* gq, const mp_half* gk,
                                   const int32_t* positions, const double* freqs, mp_half* yq, mp_half* yk, mp_stream stream) {
    const char* const what = "mp_qk_norm_rope_fwd";
    int               rc   = rope_check(d, what);
    if (rc != MP_OK) return rc;
    const long long cq = (long long)d->n_heads * d->d_head, ck = (long long)d->n_kv_heads * d->d_head;
    MP_REQUIRE((gq != nullptr) == (gk != nullptr), "%s: a norm's weights for one of queries and keys", what);
    if (d->rows == 0) return MP_OK;
    MP_REQUIRE(positions && freqs && aligned(positions, 4) && aligned(freqs, 8), "%s: positions or freqs are NULL or misaligned", what);
    if ((rc = rope_matrix(what, "q", q, d->ld_q, cq)) != MP_OK || (rc = rope_matrix(what, "k", k, d->ld_k, ck)) != MP_OK ||
        (rc = rope_matrix(what, "yq", yq, d->ld_yq, cq)) != MP_OK || (rc = rope_matrix(what, "yk", yk, d->ld_yk, ck)) != MP_OK)
        return rc;
    if (gq && (!aligned16(gq) || !aligned16(gk))) {
        set_error("%s: weights need to be 16-byte aligned", what);
        return MP_E_UNSUPPORTED;
    }
    const int w = rope_width(d);
    RopeArgs  a = rope_args(d, w, positions, freqs);
    a.part[0]   = {d->n_heads, d->ld_q, d->ld_yq, 0, q, gq, nullptr, yq, nullptr};
    a.part[1]   = {d->n_kv_heads, d->ld_k, d->ld_yk, 0, k, gk, nullptr, yk, nullptr};
    const dim3   grid((unsigned)(((long long)d->rows + a.tokens - 1) / a.tokens));
    const size_t lds = (size_t)a.tokens * d->rot * sizeof(float);
    MP_REQUIRE(grid_fits(grid.x, RO_THREADS), "%s: too many rows", what);
    return rope_dispatch(w, d->adjacent != 0, gq != nullptr, [&](auto wc, auto ac, auto nc) {
        hipLaunchKernelGGL((rope_fwd_kernel<decltype(wc)::value, decltype(ac)::value, decltype(nc)::value>), grid, dim3(RO_THREADS), lds, as_stream(stream), a);
        MP_LAUNCH_CHECK("mp_qk_norm_rope_fwd");
        return (int)MP_OK;
    });
}

extern "C" size_t mp_qk_norm_rope_bwd_workspace_bytes(const mp_rope_desc* d) {
    return rope_check(d, "mp_qk_norm_rope_bwd") == MP_OK ? rope_bwd_bytes(d) + 16 : 0;
}

extern "C" int mp_qk_norm_rope_bwd(const mp_rope_desc* d, const mp_half* q, const mp_half* k, const mp_half* gq, const mp_half* gk,
                                   const int32_t* positions, const double* freqs, const mp_half* dyq, const mp_half* dyk, mp_half* dq, mp_half* dk,
                                   mp_half* dgq, mp_half* dgk, mp_scale_state* st, void* ws, size_t ws_bytes, mp_stream stream) {
    const char* const what = "mp_qk_norm_rope_bwd";
    int               rc   = rope_check(d, what);
    if (rc != MP_OK) return rc;
    const long long cq = (long long)d->n_heads * d->d_head, ck = (long long)d->n_kv_heads * d->d_head;
    const bool      norm = gq != nullptr;
    MP_REQUIRE(norm == (gk != nullptr), "%s: a norm's weights for one of queries and keys", what);
    MP_REQUIRE(norm == (dgq != nullptr) && norm == (dgk != nullptr), "%s: weights and their gradients are given together", what);
    MP_REQUIRE(aligned(dgq, 2) && aligned(dgk, 2) && aligned(st, 4), "%s: misaligned pointer", what);
    const bool some = d->rows > 0;
    if (!some && !norm) return MP_OK;
    if (some) {
        MP_REQUIRE(positions && freqs && aligned(positions, 4) && aligned(freqs, 8), "%s: positions or freqs are NULL or misaligned", what);
        if ((rc = rope_matrix(what, "dyq", dyq, d->ld_dyq, cq)) != MP_OK || (rc = rope_matrix(what, "dyk", dyk, d->ld_dyk, ck)) != MP_OK ||
            (rc = rope_matrix(what, "dq", dq, d->ld_dq, cq)) != MP_OK || (rc = rope_matrix(what, "dk", dk, d->ld_dk, ck)) != MP_OK)
            return rc;
        if (norm && ((rc = rope_matrix(what, "q", q, d->ld_q, cq)) != MP_OK || (rc = rope_matrix(what, "k", k, d->ld_k, ck)) != MP_OK)) return rc;
        if (norm && (!aligned16(gq) || !aligned16(gk))) {
            set_error("%s: weights need to be 16-byte aligned", what);
            return MP_E_UNSUPPORTED;
        }
    }
    const int nb = rope_bwd_blocks(d->rows);
    if (norm && (!ws || !aligned16(ws) || ws_bytes < rope_bwd_bytes(d))) {
        set_error("%s: 16-byte aligned workspace of %zu bytes needed, %zu given", what, rope_bwd_bytes(d), ws_bytes);
        return MP_E_WORKSPACE;
    }
    if (some) {
        const int w = rope_width(d);
        RopeArgs  a = rope_args(d, w, positions, freqs);
        a.part[0]   = {d->n_heads, d->ld_q, d->ld_dyq, d->ld_dq, q, gq, dyq, nullptr, dq};
        a.part[1]   = {d->n_kv_heads, d->ld_k, d->ld_dyk, d->ld_dk, k, gk, dyk, nullptr, dk};
        a.sums      = static_cast<float*>(ws);
        const size_t tables = (size_t)a.tokens * d->rot, partial = norm ? (size_t)RO_WAVES * 2 * d->d_head : 0;
        const size_t lds = (tables > partial ? tables : partial) * sizeof(float);
        rc               = rope_dispatch(w, d->adjacent != 0, norm, [&](auto wc, auto ac, auto nc) {
            hipLaunchKernelGGL((rope_bwd_kernel<decltype(wc)::value, decltype(ac)::value, decltype(nc)::value>), dim3(nb), dim3(RO_THREADS), lds,
                               as_stream(stream), a);
            MP_LAUNCH_CHECK("mp_qk_norm_rope_bwd");
            return (int)MP_OK;
        });
        if (rc != MP_OK) return rc;
    }
    if (norm) {
        hipLaunchKernelGGL(rope_finish_kernel, dim3((2 * d->d_head + 31) / 32), dim3(1024), 0, as_stream(stream), static_cast<const float*>(ws), some ? nb : 0,
                           d->d_head, dgq, dgk, st);
        MP_LAUNCH_CHECK("mp_qk_norm_rope_bwd(finish)");
    }
    return MP_OK;
}
