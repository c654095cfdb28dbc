// Queries and keys before attention: the RMS norm of each head and the rotation of its pairs by position, in one pass each way.
//
// With x one head's d values, r = (mean x^2 + eps)^-1/2, x^ = x r and n = g x^, a pair (a, b) of n at the angle t becomes
// (a cos t - b sin t, a sin t + b cos t).  Backward with u = the gradient turned back by -t: dg = sum u x^, v = u g,
// dx = r (v - x^ mean(v x^)); r is formed again from x, so forward keeps nothing.
//
// Bound by HBM: forward moves 4 bytes, backward 6 bytes an element (16384 tokens of 16 + 4 heads of 128 in a row: 36 us, 4.6 TB/s, and 60 us, 4.2
// TB/s, without norms 36 us each way; one launch by itself, whose last stores are still in a cache at its end, 28 and 51 + 5 us).  Times below are
// of calls in a row, captured and replayed over buffers beyond the caches.  The angle depends on token and pair only, so a workgroup takes
// some tokens, forms their cosines and sines once into LDS, and all heads of these tokens read them there.
// A lane owns "units" of 2 W columns: W and their partners where halves are paired, 2 W neighbours where neighbours are; a head
// is then d / (2 W) lanes, filled up to a power of two, whose sums go through lane permutations.
#include <cmath>

#include "common.hpp"

namespace mp {

constexpr int RO_THREADS = 256;
constexpr int RO_WAVES   = RO_THREADS / 64;

template <int W>
struct Vec {
    typedef f16 type __attribute__((ext_vector_type(W)));
};
template <int W>
__device__ __forceinline__ typename Vec<W>::type load_piece(const uint16_t* p) {
    return *reinterpret_cast<const typename Vec<W>::type*>(p);
}
template <int W>
__device__ __forceinline__ void widen(const typename Vec<W>::type a, const typename Vec<W>::type b, float* f) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
        f[k]     = (float)a[k];
        f[W + k] = (float)b[k];
    }
}
template <int W>
__device__ __forceinline__ void store_piece(uint16_t* p, const float* f) {
    typename Vec<W>::type q;
#pragma unroll
    for (int k = 0; k < W; ++k) q[k] = (f16)f[k];
    *reinterpret_cast<typename Vec<W>::type*>(p) = q;
}

template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
    const int i = __builtin_bit_cast(int, v);
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CTRL, 0xF, 0xF, false));
}
template <int ROWS>  // 16 or 32 lanes apart
__device__ __forceinline__ float add_far(float v) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto     r = ROWS == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false) : __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned a = r[0], b = r[1];
    return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}
constexpr int LANES_1032 = 0xB1, LANES_2301 = 0x4E, MIRROR_8 = 0x141, MIRROR_16 = 0x140, TURN_4 = 0x124, TURN_8 = 0x128;

// Sum over aligned groups of `lanes` lanes (a power of two, the same for the whole launch); all of a group get it.
__device__ __forceinline__ float group_sum(float v, const int lanes) {
    if (lanes > 1) v = add_dpp<LANES_1032>(v);
    if (lanes > 2) v = add_dpp<LANES_2301>(v);
    if (lanes > 4) v = add_dpp<MIRROR_8>(v);   // (quads are alike by now)
    if (lanes > 8) v = add_dpp<MIRROR_16>(v);
    if (lanes > 16) v = add_far<16>(v);
    if (lanes > 32) v = add_far<32>(v);
    return v;
}
// Sums over the groups, lane by lane.
template <int N>
__device__ __forceinline__ void sums_over_groups(float* v, const int lanes) {
    const auto each = [&](auto&& f) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = f(v[k]);
    };
    if (lanes <= 32) each([](float x) { return add_far<32>(x); });
    if (lanes <= 16) each([](float x) { return add_far<16>(x); });
    if (lanes <= 8) each([](float x) { return add_dpp<TURN_8>(x); });
    if (lanes <= 4) each([](float x) { return add_dpp<TURN_4>(x); });  // (halves of a row of 16 are alike by now)
    if (lanes <= 2) each([](float x) { return add_dpp<LANES_2301>(x); });
    if (lanes <= 1) each([](float x) { return add_dpp<LANES_1032>(x); });
}

constexpr int RO_POS = 4;  // positions a thread has on their way

struct RopeArgs {
    int             rows, d, rot, units, lanes;  // units a head, lanes a head (units rounded up to a power of two)
    int             tokens, pair_log;            // a workgroup's at a time; log2 of the pairs, rounded up.  tokens 2^pair_log <= 4 x 256
    float           eps;
    const int32_t*  positions;                   // [axes][rows]
    const double*   freqs;                       // [rot / 2]
    struct Part {
        int             heads, ld_x, ld_y, ld_d; // x, y / dy, dx
        const uint16_t *x, *g, *dy;
        uint16_t *      y, *dx, *dg;
    } part[2];                                   // queries, keys
    float*          sums;                        // backward: [workgroups][2][d]
    mp_scale_state* st;
    unsigned        axis[MP_ROPE_PAIRS / 16];    // two bits a pair
};

// Cosines and sines of a workgroup's tokens, [token][pair] each.  A thread has one pair, whose frequency it loads once, and tokens
// RO_THREADS / 2^pair_log apart.  Angles in revolutions and 64 bits: a position of 2^31 still has its angle to 2^-20, where a product in 32
// bits has lost it at some thousands.
struct Angles {
    const RopeArgs& a;
    double          freq;
    int             pos[RO_POS];
    __device__ __forceinline__ int  pair() const { return threadIdx.x & ((1 << a.pair_log) - 1); }
    __device__ __forceinline__ int  token(int k) const { return ((int)threadIdx.x >> a.pair_log) + k * (RO_THREADS >> a.pair_log); }
    __device__ __forceinline__ void fetch(long long first, int tokens) {
        const int i    = min(pair(), (a.rot >> 1) - 1);
        unsigned  word = 0;
#pragma unroll
        for (int w = 0; w < MP_ROPE_PAIRS / 16; ++w) word = i >> 4 == w ? a.axis[w] : word;
        const int32_t* p = a.positions + (long long)((word >> 2 * (i & 15)) & 3) * a.rows + first;
        freq             = a.freqs[i];
#pragma unroll
        for (int k = 0; k < RO_POS; ++k) pos[k] = p[min(token(k), tokens - 1)];
    }
    __device__ __forceinline__ void form(int tokens, float* cosines, float* sines) const {
        const int pairs = a.rot >> 1;
#pragma unroll
        for (int k = 0; k < RO_POS; ++k) {
            if (k * (RO_THREADS >> a.pair_log) >= tokens) break;
            double turn = (double)pos[k] * (freq * 0.15915494309189533577);
            turn -= rint(turn);
            float s, c;
            sincospif(2.0f * (float)turn, &s, &c);
            if (token(k) < tokens && pair() < pairs) {
                cosines[token(k) * pairs + pair()] = c;
                sines[token(k) * pairs + pair()]   = s;
            }
        }
    }
};

// Where a lane's unit lies: columns of its two pieces, and the first of its W pairs (or -1: columns that are not turned).  Lanes behind
// a head's last unit read the first one's columns, so that no load needs a branch.
template <int W, bool ADJ>
struct Unit {
    int  col0, col1, pair;
    bool there;
    __device__ __forceinline__ Unit(const RopeArgs& a, const int lanes) {
        int       u      = threadIdx.x & (lanes - 1);
        const int turned = a.rot / (2 * W);
        there            = u < a.units;
        u                = there ? u : 0;
        pair             = there && u < turned ? u * W : -1;
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

// An item's values are on their way while the one before it is worked on, the first ones' while the angles are formed.  LANES: of a head, 0:
// whatever a.lanes says.
template <int W, bool ADJ, bool NORM, int LANES>
__global__ __launch_bounds__(RO_THREADS) void rope_fwd_kernel(const RopeArgs a) {
    extern __shared__ float lds[];
    typedef typename Vec<W>::type vec;
    const int          lanes = LANES ? LANES : a.lanes, first = blockIdx.x * a.tokens, tokens = min(a.tokens, a.rows - first), pairs = a.rot >> 1;
    const int          heads_q = a.part[0].heads;
    float *const       cosines = lds, *const sines = lds + a.tokens * pairs;
    uint16_t* const    weights = reinterpret_cast<uint16_t*>(sines + a.tokens * pairs);  // [2][d]
    const Unit<W, ADJ> at(a, lanes);
    Angles             angles{a};
    angles.fetch(first, tokens);
    uint16_t w0 = 0, w1 = 0;
    if (NORM) {
        w0 = a.part[0].g[min((int)threadIdx.x, a.d - 1)];
        w1 = a.part[1].g[min((int)threadIdx.x, a.d - 1)];
    }
    const uint16_t *const xq = a.part[0].x + (long long)first * a.part[0].ld_x, *const xk = a.part[1].x + (long long)first * a.part[1].ld_x;
    uint16_t *const       yq = a.part[0].y + (long long)first * a.part[0].ld_y, *const yk = a.part[1].y + (long long)first * a.part[1].ld_y;
    struct Item {
        vec v0, v1;
        int token, head;
    };
    Items      it(threadIdx.x / lanes, RO_THREADS / lanes, heads_q + a.part[1].heads);
    const auto fetch = [&](Item& m) {
        m.token             = it.token;
        m.head              = it.head;
        const bool      key = it.head >= heads_q;
        const int       off = min(it.token, tokens - 1) * (key ? a.part[1].ld_x : a.part[0].ld_x) + (key ? it.head - heads_q : it.head) * a.d;
        const uint16_t* x   = (key ? xk : xq) + off;
        m.v0 = load_piece<W>(x + at.col0);
        m.v1 = load_piece<W>(x + at.col1);
        it.next();  // (behind the last item the last token's, for nothing)
    };
    const float inv  = 1.0f / (float)a.d;
    const auto  work = [&](const Item& m) {
        if (m.token >= tokens) return;
        float f[2 * W];
        widen<W>(m.v0, m.v1, f);
        const bool key = m.head >= heads_q;
        if (NORM) {
            float q = 0.f, g[2 * W];
#pragma unroll
            for (int k = 0; k < 2 * W; ++k) q = fmaf(f[k], f[k], q);
            if (a.units != lanes) q = at.there ? q : 0.f;
            const float     r    = rsqrtf(group_sum(q, lanes) * inv + a.eps);
            const uint16_t* gain = weights + (key ? a.d : 0);
            widen<W>(load_piece<W>(gain + at.col0), load_piece<W>(gain + at.col1), g);
#pragma unroll
            for (int k = 0; k < 2 * W; ++k) f[k] = f[k] * r * g[k];
        }
        if (at.pair >= 0) turn_unit<W, ADJ, 1>(f, cosines + m.token * pairs + at.pair, sines + m.token * pairs + at.pair);
        if (at.there) {
            uint16_t* y = (key ? yk : yq) + m.token * (key ? a.part[1].ld_y : a.part[0].ld_y) + (key ? m.head - heads_q : m.head) * a.d;
            store_piece<W>(y + at.col0, f);
            store_piece<W>(y + at.col1, f + W);
        }
    };
    Item m, n;
    fetch(m);
    fetch(n);
    if (NORM && (int)threadIdx.x < a.d) {
        weights[threadIdx.x]       = w0;
        weights[a.d + threadIdx.x] = w1;
    }
    angles.form(tokens, cosines, sines);
    lds_barrier();
    while (m.token < tokens) {
        work(m);
        fetch(m);
        work(n);
        fetch(n);
    }
}

// Queries, then keys: the sums for their weights are all that a lane keeps from item to item.  A workgroup has one block of tokens, several
// only where there are more than some thousands of these, so that the weights' gradients are few partial rows: [workgroup][queries, keys][d].
// The only workgroup writes the gradients themselves.  Three waves a SIMD for W 8 with norms: their values, sums and addresses take 162 to
// 165 registers, and held to the 128 that four waves leave they spill (36.8 against 31.0 us for 8192 tokens of 16 + 16 heads of 64, 38.0 against 28.4
// for 12289 of 8 + 2 of 128); narrower ones fit.
template <int W, bool ADJ, bool NORM, int LANES>
__global__ __launch_bounds__(RO_THREADS, W == 8 && NORM ? 3 : 4) void rope_bwd_kernel(const RopeArgs a) {
    extern __shared__ float lds[];
    typedef typename Vec<W>::type vec;
    const int          lanes = LANES ? LANES : a.lanes, pairs = a.rot >> 1, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float *const       cosines = lds, *const sines = lds + a.tokens * pairs, *const partial = sines + a.tokens * pairs;
    const Unit<W, ADJ> at(a, lanes);
    Angles             angles{a};
    const float        inv  = 1.0f / (float)a.d;
    const long long    step = (long long)gridDim.x * a.tokens;
    bool               bad  = false;
    struct Item {
        vec u0, u1, x0, x1;
        int token, head;
    };
#pragma unroll 1
    for (int p = 0; p < 2; ++p) {
        const RopeArgs::Part& h = a.part[p];
        float                 acc[NORM ? 2 * W : 1];
        vec                   g[2];
#pragma unroll 1
        for (long long first = (long long)blockIdx.x * a.tokens; first < a.rows; first += step) {
            const int  tokens = min((long long)a.tokens, a.rows - first);
            const bool turn   = p == 0 || step < a.rows;  // (the keys of a workgroup's only block have the queries' angles)
            if (turn) angles.fetch(first, tokens);
            const uint16_t *const dy = h.dy + first * h.ld_y, *const xs = h.x + first * h.ld_x;
            uint16_t* const       dx = h.dx + first * h.ld_d;
            Items                 it(threadIdx.x / lanes, RO_THREADS / lanes, h.heads);
            const auto            fetch = [&](Item& m) {
                m.token     = it.token;
                m.head      = it.head;
                const int t = min(it.token, tokens - 1), o = it.head * a.d, y = t * h.ld_y + o;
                m.u0 = load_piece<W>(dy + y + at.col0);
                m.u1 = load_piece<W>(dy + y + at.col1);
                if (NORM) {
                    const int x = t * h.ld_x + o;
                    m.x0 = load_piece<W>(xs + x + at.col0);
                    m.x1 = load_piece<W>(xs + x + at.col1);
                }
                it.next();
            };
            const auto work = [&](Item& m) {
                if (m.token >= tokens) return;
                float f[2 * W];
                widen<W>(m.u0, m.u1, f);
                if (at.pair >= 0) turn_unit<W, ADJ, -1>(f, cosines + m.token * pairs + at.pair, sines + m.token * pairs + at.pair);
                if (NORM) {
                    // (halves are widened by the instructions that use them: kept as floats from the first use to the last, x and g cost 16
                    // registers more)
                    const auto x_ = [&](int k) { return (float)(k < W ? m.x0 : m.x1)[k % W]; };
                    const auto g_ = [&](int k) { return (float)g[k / W][k % W]; };
                    float      q = 0.f, vx = 0.f;
#pragma unroll
                    for (int k = 0; k < 2 * W; ++k) {
                        q  = fmaf(x_(k), x_(k), q);
                        vx = fmaf(f[k] * g_(k), x_(k), vx);
                    }
                    asm("" : "+v"(m.x0), "+v"(m.x1), "+v"(g[0]), "+v"(g[1]));
                    if (a.units != lanes) {
                        q  = at.there ? q : 0.f;
                        vx = at.there ? vx : 0.f;
                    }
                    const float r = rsqrtf(group_sum(q, lanes) * inv + a.eps);
                    const float w = group_sum(vx, lanes) * inv * r * r;  // mean(v x^) r, as dx = r v - x^ (mean(v x^) r)
#pragma unroll
                    for (int k = 0; k < 2 * W; ++k) {
                        const float hat = x_(k) * r;
                        acc[k]          = fmaf(f[k], hat, acc[k]);
                        f[k]            = r * (f[k] * g_(k)) - hat * w;
                    }
                }
                if (at.there) {
                    uint16_t* d = dx + m.token * h.ld_d + m.head * a.d;
                    store_piece<W>(d + at.col0, f);
                    store_piece<W>(d + at.col1, f + W);
                }
            };
            Item m, n;
            fetch(m);
            if (NORM && first < step) {  // the workgroup's first block
                g[0] = load_piece<W>(h.g + at.col0);
                g[1] = load_piece<W>(h.g + at.col1);
#pragma unroll
                for (int k = 0; k < 2 * W; ++k) acc[k] = 0.f;
            }
            fetch(n);
            if (turn) {
                lds_barrier();
                angles.form(tokens, cosines, sines);
                lds_barrier();
            }
            while (m.token < tokens) {
                work(m);
                fetch(m);
                work(n);
                fetch(n);
            }
        }
        if (NORM) {
            // lanes that own the same columns, then the waves, in order
            sums_over_groups<2 * W>(acc, lanes);
            lds_barrier();
            if (at.there && lane < lanes) {
#pragma unroll
                for (int k = 0; k < 2 * W; ++k) partial[wave * a.d + (k < W ? at.col0 + k : at.col1 + k - W)] = acc[k];
            }
            lds_barrier();
            for (int c = threadIdx.x; c < a.d; c += RO_THREADS) {
                float t = 0.f;
#pragma unroll
                for (int w = 0; w < RO_WAVES; ++w) t += partial[w * a.d + c];
                if (gridDim.x > 1) {
                    a.sums[((long long)blockIdx.x * 2 + p) * a.d + c] = t;
                } else {
                    h.dg[c] = f2h(t);
                    bad |= half_nonfinite(f2h(t));
                }
            }
        }
    }
    if (NORM && gridDim.x == 1 && a.st != nullptr && __any(bad)) {
        if (lane == 0) atomicOr(&a.st->found_inf, 1);
    }
}

// Column sums of the partial rows, 16 columns by 64 lanes of rows a workgroup, in a fixed order.  Bound by its one or two trips to memory.
__global__ __launch_bounds__(1024) void rope_finish_kernel(const float* __restrict__ sums, const int nparts, const int d, uint16_t* dgq, uint16_t* dgk,
                                                           mp_scale_state* st) {
    __shared__ float sm[64][17];
    const int        cl = threadIdx.x & 15, q = threadIdx.x >> 4, c = blockIdx.x * 16 + cl;
    float            acc = 0.f;
    for (int p = q; p < nparts; p += 64 * 8) {
        float t[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) t[u] = p + 64 * u < nparts ? sums[(long long)(p + 64 * u) * 2 * d + c] : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) acc += t[u];
    }
    sm[q][cl] = acc;
    __syncthreads();
    bool bad = false;
    if (threadIdx.x < 16) {
        float t = 0.f;
#pragma unroll
        for (int j = 0; j < 64; ++j) t += sm[j][cl];
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

int rope_pair_log(const mp_rope_desc* d) {
    int n = 0;
    while (1 << n < d->rot / 2) ++n;
    return n;
}
// the widest pieces that neither the turned columns nor the others cut
int rope_width(const mp_rope_desc* d) {
    if (d->d_head % 16 == 0 && d->rot % 16 == 0) return 8;
    return d->rot % 8 == 0 ? 4 : 2;
}
// Tokens a workgroup takes at once, up to 16, which a thread's RO_POS positions cover.  A thousand workgroups, which the chip holds together (16 + 16
// heads of 64 forward, 1, 2, 4, 8 and 16 tokens: 1000 tokens 4.5, 4.4, 4.5, 5.4, 7.6 us; 4096 11.6, 10.1, 8.9, 9.5, 10.9).
int rope_most_tokens(const mp_rope_desc* d) {
    const int most = RO_POS * RO_THREADS >> rope_pair_log(d);
    return most < 16 ? most : 16;
}
int rope_tokens(const mp_rope_desc* d) {
    const int most = rope_most_tokens(d), t = d->rows / 1024 + (d->rows % 1024 != 0);
    return t < 1 ? 1 : t < most ? t : most;
}
// Backward with norms, in pieces of 8: 256 workgroups, as each adds its weights' sums up over its lanes and leaves a row of them (16 + 16 heads of 64,
// 1, 2, 4, 8 and 16 tokens: 1000 tokens 17.0, 12.4, 11.0, 11.6, 14.0 us; 2048 23.6, 18.0, 13.1, 13.0, 14.7; 8192 73, 51, 35.5, 33.0, 30.5); up to 8 tokens
// one, which leaves none (4 tokens: 8.3 us in four, 6.2 in one).  Narrower pieces have more passes a token (16 + 16 of 80, 40 turned: 4096 tokens 38.4,
// 28.4, 26.0, 28.3, 36.0).
int rope_bwd_tokens(const mp_rope_desc* d, bool norm) {
    if (!norm || rope_width(d) < 8) return rope_tokens(d);
    const int most = rope_most_tokens(d);
    if (d->rows <= 8 && d->rows <= most) return d->rows < 1 ? 1 : d->rows;
    int t = 1;
    while (t < most && t < d->rows / 256.0) t *= 2;
    return t;
}
int rope_bwd_blocks(const mp_rope_desc* d, bool norm) {
    const int t = rope_bwd_tokens(d, norm), n = d->rows / t + (d->rows % t != 0);
    return n < 1024 ? n : 1024;
}
// (for the same heads and as many rows or fewer, of which some have more workgroups)
size_t rope_most_bytes(const mp_rope_desc* d) { return (size_t)(d->rows < 1024 ? d->rows : 1024) * 2 * d->d_head * sizeof(float); }
size_t rope_bwd_bytes(const mp_rope_desc* d) { return (size_t)rope_bwd_blocks(d, true) * 2 * d->d_head * sizeof(float); }

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
    if (ld % 8 != 0 || ld >= 1 << 22 || !aligned16(p)) {
        set_error("%s: %s needs to be 16-byte aligned with a leading dimension that is a multiple of 8 below 2^22", what, name);
        return MP_E_UNSUPPORTED;
    }
    return MP_OK;
}

RopeArgs rope_args(const mp_rope_desc* d, int w, int tokens, const int32_t* positions, const double* freqs) {
    RopeArgs a{};
    a.rows  = d->rows;
    a.d     = d->d_head;
    a.rot   = d->rot;
    a.units = d->d_head / (2 * w);
    a.lanes = 1;
    while (a.lanes < a.units) a.lanes *= 2;
    a.tokens    = tokens;
    a.pair_log  = rope_pair_log(d);
    a.eps       = d->eps;
    a.positions = positions;
    a.freqs     = freqs;
    for (int i = 0; i < d->rot / 2; ++i) a.axis[i / 16] |= (unsigned)d->axis[i] << 2 * (i % 16);
    return a;
}

template <typename F>
int rope_dispatch(const RopeArgs& a, int w, bool adj, bool norm, F&& f) {
    const auto by_norm = [&](auto wc, auto ac, auto lc) { return norm ? f(wc, ac, std::true_type{}, lc) : f(wc, ac, std::false_type{}, lc); };
    const auto by_adj  = [&](auto wc, auto lc) { return adj ? by_norm(wc, std::true_type{}, lc) : by_norm(wc, std::false_type{}, lc); };
    typedef std::integral_constant<int, 0> Any;
    typedef std::integral_constant<int, 8> W8;
    if (w == 8 && a.lanes == 4) return by_adj(W8{}, std::integral_constant<int, 4>{});  // heads of 64
    if (w == 8 && a.lanes == 8) return by_adj(W8{}, W8{});                              // of 80 to 128
    if (w == 8) return by_adj(W8{}, Any{});
    if (w == 4) return by_adj(std::integral_constant<int, 4>{}, Any{});
    return by_adj(std::integral_constant<int, 2>{}, Any{});
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
    RopeArgs  a = rope_args(d, w, rope_tokens(d), positions, freqs);
    a.part[0]   = {d->n_heads, d->ld_q, d->ld_yq, 0, q, gq, nullptr, yq, nullptr, nullptr};
    a.part[1]   = {d->n_kv_heads, d->ld_k, d->ld_yk, 0, k, gk, nullptr, yk, nullptr, nullptr};
    const dim3   grid((unsigned)(((long long)d->rows + a.tokens - 1) / a.tokens));
    const size_t lds = (size_t)a.tokens * d->rot * sizeof(float) + (gq ? 2 * (size_t)d->d_head * sizeof(uint16_t) : 0);
    MP_REQUIRE(grid_fits(grid.x, RO_THREADS), "%s: too many rows", what);
    return rope_dispatch(a, w, d->adjacent != 0, gq != nullptr, [&](auto wc, auto ac, auto nc, auto lc) {
        hipLaunchKernelGGL((rope_fwd_kernel<decltype(wc)::value, decltype(ac)::value, decltype(nc)::value, decltype(lc)::value>), grid, dim3(RO_THREADS), lds, as_stream(stream), a);
        MP_LAUNCH_CHECK("mp_qk_norm_rope_fwd");
        return (int)MP_OK;
    });
}

extern "C" size_t mp_qk_norm_rope_bwd_workspace_bytes(const mp_rope_desc* d) {
    return rope_check(d, "mp_qk_norm_rope_bwd") == MP_OK ? rope_most_bytes(d) + 16 : 0;
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
    const int nb = rope_bwd_blocks(d, norm);
    if (norm && (!ws || !aligned16(ws) || ws_bytes < rope_bwd_bytes(d))) {
        set_error("%s: 16-byte aligned workspace of %zu bytes needed, %zu given", what, rope_bwd_bytes(d), ws_bytes);
        return MP_E_WORKSPACE;
    }
    if (some) {
        const int w = rope_width(d);
        RopeArgs  a = rope_args(d, w, rope_bwd_tokens(d, norm), positions, freqs);
        a.part[0]   = {d->n_heads, d->ld_q, d->ld_dyq, d->ld_dq, q, gq, dyq, nullptr, dq, dgq};
        a.part[1]   = {d->n_kv_heads, d->ld_k, d->ld_dyk, d->ld_dk, k, gk, dyk, nullptr, dk, dgk};
        a.sums      = static_cast<float*>(ws);
        a.st        = st;
        const size_t lds = ((size_t)a.tokens * d->rot + (norm ? (size_t)RO_WAVES * d->d_head : 0)) * sizeof(float);
        rc               = rope_dispatch(a, w, d->adjacent != 0, norm, [&](auto wc, auto ac, auto nc, auto lc) {
            hipLaunchKernelGGL((rope_bwd_kernel<decltype(wc)::value, decltype(ac)::value, decltype(nc)::value, decltype(lc)::value>), dim3(nb), dim3(RO_THREADS), lds,
                               as_stream(stream), a);
            MP_LAUNCH_CHECK("mp_qk_norm_rope_bwd");
            return (int)MP_OK;
        });
        if (rc != MP_OK) return rc;
    }
    if (norm && nb != 1) {
        hipLaunchKernelGGL(rope_finish_kernel, dim3(d->d_head / 8), dim3(1024), 0, as_stream(stream), static_cast<const float*>(ws), some ? nb : 0,
                           d->d_head, dgq, dgk, st);
        MP_LAUNCH_CHECK("mp_qk_norm_rope_bwd(finish)");
    }
    return MP_OK;
}
