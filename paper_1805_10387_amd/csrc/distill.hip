// Distillation from a teacher's top logits: fp32 loss and loss-scaled fp16 seed gradient in one pass over the student's logits.
//
// With z = x / temperature, p = softmax z, A the classes that the teacher's list names, q_u its probability of class u (entries of one
// class added up), Q = sum q, and r what is left for all other classes together (0 where lists are renormalised):
//     L = sum_A q_u (ln q_u - ln p_u) + r (ln r - ln p_rest),       dL/dz_j = (Q + r) p_j - (j in A ? q_j : r p_j / p_rest)
//     dx_j = S / rows (weight / temperature dL/dz_j + hard (softmax(x)_j - 1[j = target]))
//
// Bound by HBM: 2 bytes a class read, 2 written.  A workgroup holds a row in registers from its sums to its gradient; several of them
// on a compute unit are in different parts of that (8192 x 32768 with 64 listed and the rest: 204 us, 5.3 TB/s).  Of rows beyond 65536 classes a unit's
// registers hold one, and nothing is on its way while it is worked on (1021 x 131071 with 100 listed: 146 us, 3.7 TB/s, with the rest 158; in
// chunks, read twice, 194 and 208).  Times here are of calls in a row, captured and replayed over the same buffers.
// Outside A the gradient is one factor a row times the exponential.  The classes of A, at most 128, are one wave's work: their
// gradients wait in LDS, and a map from pieces to entries tells each piece which of its elements to replace.  For r the sum over
// "all others" is formed without A, not as a difference of sums, which would lose it where the student is sure of A.
//
// Rows longer than 135160 classes, or too few for the chip, are cut into chunks: one launch for the sums, one for the gradient.
#include <cmath>

#include "vocab_rows.hpp"

namespace mp {

constexpr int DI_TARGET = MP_TOP_MAX;  // the entry of the target, behind the list's

struct DistillArgs {
    int             rows, vocab, ld, top, chunks, chunk;
    float           c2, weight, inv_temperature, hard;
    const uint16_t* logits;
    const int32_t * ids, *targets;
    const float*    teacher;
    const mp_scale_state* st;
    uint16_t*       dlogits;  // may be logits
    float*          row_loss;
    float*          sums;     // chunks: [row][chunk][4]
    float*          chosen;   // chunks: [row][MP_TOP_MAX + 1], the student's logits of the entries
};

// The entries of a row, in LDS: one wave's work.  The last one is the target's.
struct EntryLds {
    int      id[MP_TOP_MAX + 1];
    float    q[MP_TOP_MAX], x[MP_TOP_MAX + 1];                 // q, the student's logit
    unsigned info[MP_TOP_MAX + 1];                             // as in the map; there for those behind the first one of a word
    int      again[MP_TOP_MAX];                                // an earlier entry names the class too
};
// A word of the map, 0 where there is no entry: the next entry of the word + 1, the element's place among the word's, flags, its gradient.
constexpr unsigned MAP_NEXT = 0xFFu, MAP_TARGET = 1u << 12, MAP_THERE = 1u << 13, MAP_FIRST = 1u << 14;
__device__ __forceinline__ int map_place(unsigned w) { return (int)(w >> 8) & 15; }
// Hard labels: TWO_NONE without these or at temperature 1; TWO_ANY: exponentials of their own; TWO_SQUARES, at temperature 2: squares of the
// others (1021 x 131071 with 100 listed: without hard labels 146 us, with squares 151, with exponentials 170; 8192 x 32768 with 64 208, 212 and 240).
enum { TWO_NONE, TWO_ANY, TWO_SQUARES };
struct RowFactors {
    float a, ref, b, ref2;  // gradient outside A: a 2^(c2 x - ref) + b 2^(log2(e) x - ref2); TWO_SQUARES: e = 2^(c2 x - ref), e (a + b e)
    int   none;             // a zero row, whatever it holds
};

// One wave's view of a row's entries: lane l has entries l and l + 64, lane 0 the target's as well.  SHIFT: 2^SHIFT elements share a word
// of the map.
template <int SHIFT>
struct Entries {
    const DistillArgs& a;
    EntryLds&          l;
    unsigned*          map;
    int                first;              // class that the stretch begins with
    int                target;
    bool               some, listed, twice;  // entries that there are; the target is in A; some class is named more than once

    __device__ __forceinline__ static int lane() { return threadIdx.x & 63; }
    __device__ __forceinline__ bool       there(int c) const { return c >= 0 && c < a.vocab; }
    // f(slot, entry) for the lane's entries
    template <typename F>
    __device__ __forceinline__ void each(F&& f) const {
        if (lane() < a.top) f(0, lane());
        if (a.top > 64 && lane() + 64 < a.top) f(1, lane() + 64);
    }
    // word of the map for class c, or -1: another stretch's, or none
    __device__ __forceinline__ int word(const Stretch& z, int c) const { return c >= first && c < a.vocab && c - first < z.len ? (c - first + z.head) >> SHIFT : -1; }

    // the row's list on its way, and then in place
    struct List {
        int   id[2], target;
        float t[2];
    };
    __device__ __forceinline__ List fetch(long long row) const {
        List h;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const long long e = row * a.top + min(lane() + 64 * s, a.top - 1);
            h.id[s]           = a.ids[e];
            h.t[s]            = a.teacher[e];
        }
        h.target = a.targets ? a.targets[row] : -1;
        return h;
    }
    __device__ __forceinline__ void settle(const List& h) {
        each([&](int s, int e) { l.id[e] = h.id[s]; });
        target = h.target;
        if (lane() == 0) l.id[DI_TARGET] = target;
    }
    // the student's logits of the entries
    struct Logits {
        uint16_t x[2], target;
    };
    __device__ __forceinline__ Logits fetch_logits(long long row, const List& list) const {
        const uint16_t* z = a.logits + row * a.ld;
        Logits          h;
#pragma unroll
        for (int s = 0; s < 2; ++s) h.x[s] = z[there(list.id[s]) ? list.id[s] : 0];
        h.target = z[there(target) ? target : 0];
        return h;
    }
    __device__ __forceinline__ void settle_logits(const Logits& h) {
        each([&](int s, int e) { l.x[e] = h2f(h.x[s]); });
        if (lane() == 0) l.x[DI_TARGET] = h2f(h.target);
    }
    // into the map of the row's pieces, those that lie in the stretch
    __device__ __forceinline__ void insert(const Stretch& z, const List& h) {
        bool any = false, eq = false;
        each([&](int s, int) {
            any |= there(h.id[s]);
            eq |= h.id[s] == target;
        });
        some   = __any(any);
        listed = __any(eq) && there(target);
        bool again = false;
        if (a.chunks > 1) {  // (entries of one class may all lie in another chunk: the map is a hash table of the whole list first)
            each([&](int s, int e) {
                if (there(h.id[s])) l.info[e] = atomicExch(&map[h.id[s] & 255], (unsigned)e + 1);
            });
            __builtin_amdgcn_wave_barrier();
            each([&](int s, int e) {
                if (there(h.id[s]))
                    for (unsigned o = l.info[e]; o; o = l.info[o - 1]) again |= l.id[o - 1] == h.id[s];
            });
            __builtin_amdgcn_wave_barrier();
            each([&](int s, int) { map[h.id[s] & 255] = 0; });
        }
        unsigned   info[2] = {0, 0}, info_t = 0;
        int        at[2]   = {-1, -1}, at_t = -1;
        const auto enter = [&](int c, int e, unsigned flag, int& w, unsigned& i) {
            w = word(z, c);
            if (w < 0) return;
            i         = atomicExch(&map[w], (unsigned)e + 1) | (unsigned)((c - first + z.head) & ((1 << SHIFT) - 1)) << 8 | flag | MAP_THERE;
            l.info[e] = i;
        };
        each([&](int s, int e) { enter(h.id[s], e, 0u, at[s], info[s]); });
        if (lane() == 0 && !listed) enter(target, DI_TARGET, MAP_TARGET, at_t, info_t);
        __builtin_amdgcn_wave_barrier();
        each([&](int s, int) {
            for (unsigned o = info[s] & MAP_NEXT; o; o = l.info[o - 1] & MAP_NEXT) again |= l.id[o - 1] == h.id[s];
        });
        twice = __any(again);
        // the first one of a word moves into it; indices are below 256 and what moves in is above
        const auto head = [&](int e, int w, unsigned i) {
            if (w >= 0 && map[w] == (unsigned)e + 1) map[w] = l.info[e] = i | MAP_FIRST;
        };
        each([&](int s, int e) { head(e, at[s], info[s]); });
        if (lane() == 0 && !listed) head(DI_TARGET, at_t, info_t);
    }
    // the entry's gradient, where its word of the map will find it
    __device__ __forceinline__ void put(const Stretch& z, int e, int c, unsigned info, float value) const {
        const int w = word(z, c);
        if (w < 0) return;
        const unsigned full = info | (unsigned)f2h(value) << 16;
        if (full & MAP_FIRST) map[w] = full;
        else l.info[e] = full;
    }
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int far = 32; far; far >>= 1) v += __shfl_xor(v, far, 64);
    return v;
}

// One wave's work on a row: the teacher's side while the row is on its way, then what the other waves wait for (factors and the entries'
// gradients), then the loss.
template <bool TAIL, int TWO, int SHIFT>
struct RowWork {
    const Entries<SHIFT>& n;
    float                 sum_q, sum_r, r;     // Q, what 1 - Q leaves, and that or 0 where nothing outside A can be
    float                 wc, hs, u;           // S / rows times weight / temperature and hard; Q + r
    Sums<false>           one, all, at1;       // sums outside A (TAIL), over all, at temperature 1
    int                   id[2];               // the lane's entries: class (-1: none), the student's logit, q
    float                 x[2], q[2];
    bool                  first[2];            // of its class

    __device__ __forceinline__ explicit RowWork(const Entries<SHIFT>& n_) : n(n_), one(1.f), all(1.f), at1(1.f) {}

    __device__ __forceinline__ void teacher(const typename Entries<SHIFT>::List& h) {
        EntryLds& l = n.l;
        sum_r       = 0.f;
        if (TAIL) {
            double sum = 0.0;
            n.each([&](int s, int e) {
                const double v = n.there(h.id[s]) ? exp((double)h.t[s]) : 0.0;  // (64 bits: 1 minus their sum is often next to nothing)
                l.q[e]         = (float)v;
                sum += v;
            });
            sum   = wave_sum64(sum);
            sum_q = (float)sum;
            if (n.some && sum < 1.0) sum_r = (float)(1.0 - sum);
        } else {
            float m = -INFINITY, sum = 0.f, v[2] = {0.f, 0.f};
            n.each([&](int s, int) { m = fmaxf(m, n.there(h.id[s]) ? h.t[s] : -INFINITY); });
            m = wave_max(m);
            m = m == -INFINITY ? 0.f : m;
            n.each([&](int s, int) {
                v[s] = n.there(h.id[s]) ? expf(h.t[s] - m) : 0.f;
                sum += v[s];
            });
            sum             = wave_sum(sum);
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            n.each([&](int s, int e) { l.q[e] = v[s] * inv; });
            sum_q = sum * inv;
        }
        __builtin_amdgcn_wave_barrier();
        if (n.twice) {  // a class counts once, with the sum of its entries in their order
            float v[2];
            n.each([&](int s, int e) {
                bool again = false;
                v[s]       = 0.f;
                for (int j = 0; j < n.a.top; ++j)
                    if (l.id[j] == h.id[s]) {
                        v[s] += l.q[j];
                        again |= j < e;
                    }
                l.again[e] = again;
            });
            __builtin_amdgcn_wave_barrier();
            n.each([&](int s, int e) { l.q[e] = v[s]; });
        }
    }
    // s1, s2: sums at the temperature and (TWO) at 1, without A if TAIL
    __device__ __forceinline__ void factors(const Stretch& z, const Sums<false>& s1, const Sums<false>& s2, RowFactors& out) {
        const DistillArgs& a     = n.a;
        EntryLds&          l     = n.l;
        const bool         real  = n.there(n.target);
        const float        scale = (float)((double)a.st->scale / (double)a.rows);
        wc = n.some ? a.weight * a.inv_temperature * scale : 0.f, hs = real ? a.hard * scale : 0.f;
        one = all = s1, at1 = s2;
        unsigned info[2];
        n.each([&](int s, int e) {
            id[s]    = l.id[e];
            x[s]     = l.x[e];
            q[s]     = l.q[e];
            info[s]  = l.info[e];
            first[s] = !n.twice || !l.again[e];
        });
        r = one.s > 0.f ? sum_r : 0.f, u = sum_q + r;
        if (TAIL) {
            float top = -INFINITY;
            n.each([&](int s, int) { top = fmaxf(top, n.there(id[s]) ? x[s] : -INFINITY); });
            top                    = wave_max(top);
            const auto with_listed = [&](Sums<false>& t, float c2) {
                t.move(fmaxf(t.ref, top * c2));
                float sum = 0.f;
                n.each([&](int s, int) {
                    if (n.there(id[s]) && first[s]) sum += __builtin_amdgcn_exp2f(fmaf(x[s], c2, -t.ref));
                });
                t.s += wave_sum(sum);
            };
            with_listed(all, a.c2);
            if (TWO) with_listed(at1, LOG2E);
        }
        const float inv_s = 1.f / all.s, rest = TAIL ? __builtin_amdgcn_exp2f(one.ref - all.ref) : 1.f, inv_1 = TWO ? 1.f / at1.s : inv_s;
        RowFactors  f;
        f.a    = wc * (u * (rest * inv_s) - (TAIL && r > 0.f ? r / one.s : 0.f)) + (TWO ? 0.f : hs * (rest * inv_s));
        f.ref  = one.ref;
        f.b    = TWO ? hs * inv_1 : 0.f;
        f.ref2 = at1.ref;
        f.none = !n.some && !real;
        if (n.lane() == 0) {
            out = f;
            if (TWO == TWO_SQUARES) out.b = f.b * __builtin_amdgcn_exp2f(2.f * f.ref - f.ref2);  // (the other's reference may be a listed logit)
        }
        n.each([&](int s, int e) {
            if (!n.there(id[s])) return;
            const float p  = __builtin_amdgcn_exp2f(fmaf(x[s], a.c2, -all.ref)) * inv_s;
            const float p1 = TWO ? __builtin_amdgcn_exp2f(fmaf(x[s], LOG2E, -at1.ref)) * inv_1 : p;
            n.put(z, e, id[s], info[s], wc * (p * u - q[s]) + (real ? hs * (p1 - (id[s] == n.target ? 1.f : 0.f)) : 0.f));
        });
        if (n.lane() == 0 && real && !n.listed) {
            const float xt = l.x[DI_TARGET], e = __builtin_amdgcn_exp2f(fmaf(xt, a.c2, -f.ref));
            n.put(z, DI_TARGET, n.target, l.info[DI_TARGET], f.a * e + (TWO ? f.b * __builtin_amdgcn_exp2f(fmaf(xt, LOG2E, -f.ref2)) : 0.f) - hs);
        }
    }
    __device__ __forceinline__ void loss(float* out) {
        const DistillArgs& a     = n.a;
        EntryLds&          l     = n.l;
        const float        log_s = log2f(all.s);
        float              kl    = 0.f;
        n.each([&](int s, int) {
            if (n.there(id[s]) && first[s] && q[s] != 0.f) kl += q[s] * (logf(q[s]) - LN2 * (fmaf(x[s], a.c2, -all.ref) - log_s));
        });
        kl = wave_sum(kl);
        if (TAIL && r > 0.f) kl += r * (logf(r) - LN2 * ((one.ref - all.ref) + (log2f(one.s) - log_s)));
        float       sum = n.some ? a.weight * kl : 0.f;
        const float xt  = l.x[DI_TARGET];
        if (n.there(n.target)) sum -= a.hard * (LN2 * (TWO ? fmaf(xt, LOG2E, -at1.ref) - log2f(at1.s) : fmaf(xt, a.c2, -all.ref) - log_s));
        if (n.lane() == 0) *out = sum;
    }
};

// half k of a piece
__device__ __forceinline__ void set_half(u32x4& q, int k, unsigned h) {
#pragma unroll
    for (int w = 0; w < 4; ++w)
        if (w == k >> 1) q[w] = (k & 1) ? (q[w] & 0xFFFFu) | (h << 16) : (q[w] & 0xFFFF0000u) | h;
}

template <int SHIFT>
__host__ __device__ constexpr int map_words(int len) { return (len + 7 + (1 << SHIFT) - 1) >> SHIFT; }

// FUSED: a workgroup has a whole row.  SUMS, GRADIENT: one chunk of one, its sums out or all of them in through a.sums.
enum { DI_SUMS, DI_GRADIENT, DI_FUSED };

template <int THREADS, int VECS, bool TAIL, int TWO, int MODE, int SHIFT>
__global__ __launch_bounds__(THREADS, THREADS == 768 ? 3 : 4) void distill_kernel(const DistillArgs a) {
    extern __shared__ unsigned map[];
    __shared__ EntryLds        l;
    __shared__ RowFactors      factors;
    __shared__ float           red[THREADS / 64][4];
    constexpr int              NW = THREADS / 64, G = VECS % 4 == 0 && !TAIL ? 4 : VECS % 2 == 0 ? 2 : 1;
    const int                  tid = threadIdx.x, wave = tid >> 6;
    const long long            row   = MODE == DI_FUSED ? blockIdx.x : blockIdx.x / a.chunks;
    const int                  chunk = MODE == DI_FUSED ? 0 : blockIdx.x - (int)row * a.chunks, first = chunk * a.chunk, len = min(a.chunk, a.vocab - first);
    const Stretch              z(a.logits + row * a.ld + first, len);
    Entries<SHIFT>             n{a, l, map, first, -1, false, false, false};
    RowWork<TAIL, TWO, SHIFT>  work(n);
    u32x4                      raw[VECS], last;
    typename Entries<SHIFT>::List   list;
    typename Entries<SHIFT>::Logits logits;
    if (wave == 0) list = n.fetch(row);  // (ahead of the row: what comes back first is waited for first)
    load_pieces<THREADS>(z, tid, raw, last);
    for (int v = tid; v < map_words<SHIFT>(a.chunk); v += THREADS) map[v] = 0;
    lds_barrier();
    if (wave == 0) {
        n.settle(list);
        if (MODE != DI_GRADIENT) logits = n.fetch_logits(row, list);
        n.insert(z, list);
    }
    // f(place in the piece, word of the map) for the entries of piece v
    const auto entries_of = [&](int v, auto&& f) {
        if (v < z.pieces())
            for (unsigned w = map[v >> (SHIFT - 3)]; w; w = (w & MAP_NEXT) ? l.info[(w & MAP_NEXT) - 1] : 0u)
                if (SHIFT == 3 || (map_place(w) >> 3) == (v & 1)) f(map_place(w) & 7, w);
    };
    if (TAIL && MODE != DI_GRADIENT) lds_barrier();  // the map is there: sums without A
    if (wave == 0 && MODE != DI_SUMS) work.teacher(list);
    int at = tid;
    asm("" : "+v"(at));  // (places of the pieces are formed again, not kept in registers)
    if (MODE != DI_GRADIENT) {
        Sums<false> one(a.c2), two(LOG2E);
#pragma unroll
        for (int i = 0; i < VECS; i += G) {
#pragma unroll
            for (int j = 0; j < G; ++j) settle<THREADS>(z, i + j, at, raw[i + j], last);
            if (i * THREADS < z.pieces()) {
                u32x4 q[G];
#pragma unroll
                for (int j = 0; j < G; ++j) {
                    q[j] = raw[i + j];
                    if (TAIL)
                        entries_of((i + j) * THREADS + at, [&](int k, unsigned w) {
                            if (!(w & MAP_TARGET)) set_half(q[j], k, 0xFC00u);
                        });
                    asm("" : "+v"(q[j]));
                }
                const float m = max_of<G>(q);
                if (TWO == TWO_SQUARES) {
                    add_pieces_and_squares<G>(one, two, q, a.c2, m);
                } else {
                    one.template add_pieces<G>(q, a.c2, m);
                    if (TWO) two.template add_pieces<G>(q, LOG2E, m);
                }
            }
        }
        one.over_wave();
        if (TWO) two.over_wave();
        if ((tid & 63) == 0) {
            red[wave][0] = one.ref;
            red[wave][1] = one.s;
            red[wave][2] = two.ref;
            red[wave][3] = two.s;
        }
        lds_barrier();
    }
    if (wave == 0) {
        Sums<false> s1(a.c2), s2(LOG2E);
        float*      chosen = a.chosen + row * (MP_TOP_MAX + 1);
        if (MODE == DI_GRADIENT) {
            for (int c = tid; c < a.chunks; c += 64) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(a.sums + (row * a.chunks + c) * 4);
                s1.add_sums(v[0], v[1], 0.f);
                if (TWO) s2.add_sums(v[2], v[3], 0.f);
            }
            n.each([&](int, int e) { l.x[e] = chosen[e]; });
            if (tid == 0) l.x[DI_TARGET] = chosen[DI_TARGET];
        } else {
            n.settle_logits(logits);
            if (tid < NW) {
                s1.add_sums(red[tid][0], red[tid][1], 0.f);
                if (TWO) s2.add_sums(red[tid][2], red[tid][3], 0.f);
            }
        }
        s1.over_wave();
        if (TWO) s2.over_wave();
        if (MODE == DI_SUMS) {
            if (tid == 0) *reinterpret_cast<f32x4*>(a.sums + (row * a.chunks + chunk) * 4) = f32x4{s1.ref, s1.s, s2.ref, s2.s};
            if (chunk == 0) {
                n.each([&](int, int e) { chosen[e] = l.x[e]; });
                if (tid == 0) chosen[DI_TARGET] = l.x[DI_TARGET];
            }
        } else {
            work.factors(z, s1, s2, factors);
        }
    }
    if (MODE == DI_SUMS) return;
    lds_barrier();
    if (wave == 0 && first == 0) work.loss(a.row_loss + row);
    const auto  uniform = [](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); };
    const float fa = uniform(factors.a), ref = uniform(factors.ref), fb = uniform(factors.b), ref2 = uniform(factors.ref2);
    const bool  none = __builtin_amdgcn_readfirstlane(factors.none);
    uint16_t*   dz   = a.dlogits + row * a.ld + first;
    asm("" : "+v"(at));
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        if (i * THREADS < z.pieces()) {
            const int v = i * THREADS + at;
            u32x4     o = {0, 0, 0, 0};
            if (MODE == DI_GRADIENT) settle<THREADS>(z, i, at, raw[i], last);
            asm("" : "+v"(raw[i]));  // (or the compiler keeps the sums' halves, taken apart, in twice the registers until here)
            if (!none) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float d[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float x = (float)as_pair(raw[i][k])[h];
                        const float e = __builtin_amdgcn_exp2f(fmaf(x, a.c2, -ref));
                        d[h]          = TWO == TWO_SQUARES ? e * fmaf(fb, e, fa) : fa * e;
                        if (TWO == TWO_ANY) d[h] = fmaf(fb, __builtin_amdgcn_exp2f(fmaf(x, LOG2E, -ref2)), d[h]);
                    }
                    o[k] = (unsigned)f2h(d[0]) | ((unsigned)f2h(d[1]) << 16);
                }
                entries_of(v, [&](int k, unsigned w) { set_half(o, k, w >> 16); });
            }
            z.store(dz, v, o);
        }
    }
}

}  // namespace mp

using namespace mp;

namespace {

constexpr int DI_CHUNK = 256 * 8;    // 16-byte pieces of a chunk at most
constexpr int DI_FULL  = 512 * 16;   // of a row that leaves room for another one in a compute unit's registers
constexpr int DI_MOST  = 768 * 22;   // of a row in registers

int least_chunks(int vocab) { return (vocab + 8 * DI_CHUNK - 9) / (8 * DI_CHUNK - 8); }
struct DistillPlan {
    int chunks, chunk;  // 0 chunks: rows in registers
};
// Chunks where rows do not fit, and where a long row would keep few compute units long: us, in registers / in chunks, 1, 64 and 128 rows of
// 100000 classes 19.7 / 12.0, 23.7 / 20.1, 25.3 / 26.2, of 131071 22.1 / 12.4, 26.9 / 21.3, 29.6 / 34.2; of 50021 13.5 / 12.2, 18.7 / 20.8, 19.5 / 23.3.
// Chunks are at least 4096 classes, and no more than fill the chip.  even: rows start at 16-byte pieces.  (Others may take a piece more.)
DistillPlan distill_plan(int rows, int vocab, bool even) {
    const int pieces = (vocab + (even ? 7 : 14)) / 8;
    if (pieces <= (rows <= 64 ? DI_FULL : DI_MOST)) return {0, vocab};
    int n = least_chunks(vocab);
    while ((long long)rows * n * 2 <= 256 && vocab / (n * 2) >= 4096) n *= 2;
    const int chunk = ((vocab + n - 1) / n + 7) / 8 * 8;
    return {(vocab + chunk - 1) / chunk, chunk};
}
size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t distill_bytes(int rows, const DistillPlan& p) {
    return round256((size_t)rows * sizeof(float)) + (p.chunks ? (size_t)rows * (p.chunks * 16 + (MP_TOP_MAX + 1) * sizeof(float)) : 0);
}
// for as many rows or fewer, of which some are cut where more are not, or into more chunks, and at any alignment
size_t distill_most_bytes(int rows, int vocab) {
    const int pieces = (vocab + 14) / 8;
    size_t    n      = round256((size_t)rows * sizeof(float));
    if (pieces > DI_FULL) {
        const size_t cut = pieces > DI_MOST || rows < 64 ? rows : 64, chunks = cut * least_chunks(vocab);
        n += (chunks > 256 ? chunks : 256) * 16 + cut * (MP_TOP_MAX + 1) * sizeof(float);
    }
    return n;
}

int distill_check(const mp_distill_desc* d, const char* what) {
    MP_REQUIRE(d, "%s: NULL argument", what);
    MP_REQUIRE(d->rows > 0 && d->vocab > 0 && d->ld >= d->vocab && d->top > 0, "%s: bad shape rows=%d vocab=%d ld=%d top=%d", what, d->rows, d->vocab, d->ld, d->top);
    MP_REQUIRE(d->inv_temperature >= 0x1p-8f && d->inv_temperature <= 0x1p8f, "%s: 1 / temperature outside 2^-8 .. 2^8", what);
    MP_REQUIRE(std::isfinite(d->weight) && std::isfinite(d->hard_weight), "%s: a weight is not finite", what);
    MP_REQUIRE((d->tail == 0 || d->tail == 1) && d->reserved == 0, "%s: tail=%d, reserved=%d", what, d->tail, d->reserved);
    if (d->top > MP_TOP_MAX || d->vocab > MP_VOCAB_MAX) {
        set_error("%s: up to %d classes of a list, of %d", what, MP_TOP_MAX, MP_VOCAB_MAX);
        return MP_E_UNSUPPORTED;
    }
    return MP_OK;
}

// ONLY: 1, 0: for calls with a tail, without one.  2: for both.
template <int THREADS, int VECS, int MODE, int ONLY = 2>
int launch_distill(const DistillArgs& a, const mp_distill_desc* d, long long workgroups, hipStream_t hs) {
    constexpr int SHIFT = THREADS * VECS > 8192 ? 4 : 3;  // (a map within 64 KB)
    MP_REQUIRE(grid_fits(workgroups, THREADS), "mp_distill_scaled: too many rows");
    const int two = d->hard_weight == 0.f || d->inv_temperature == 1.f ? TWO_NONE : d->inv_temperature == 0.5f ? TWO_SQUARES : TWO_ANY;
    const auto launch = [&](auto tail, auto second) {
        hipLaunchKernelGGL((distill_kernel<THREADS, VECS, decltype(tail)::value, decltype(second)::value, MODE, SHIFT>), dim3((unsigned)workgroups), dim3(THREADS),
                           map_words<SHIFT>(a.chunk) * sizeof(unsigned), hs, a);
    };
    const auto by_second = [&](auto tail) {
        if (two == TWO_NONE) launch(tail, std::integral_constant<int, TWO_NONE>{});
        else if (two == TWO_SQUARES) launch(tail, std::integral_constant<int, TWO_SQUARES>{});
        else launch(tail, std::integral_constant<int, TWO_ANY>{});
    };
    if constexpr (ONLY == 2) d->tail ? by_second(std::true_type{}) : by_second(std::false_type{});
    else by_second(std::integral_constant<bool, ONLY == 1>{});
    MP_LAUNCH_CHECK("mp_distill_scaled");
    return MP_OK;
}

}  // namespace

extern "C" size_t mp_distill_workspace_bytes(const mp_distill_desc* d) {
    return distill_check(d, "mp_distill_scaled") == MP_OK ? distill_most_bytes(d->rows, d->vocab) : 0;
}

extern "C" int mp_distill_scaled_parts(const mp_distill_desc* d, const mp_half* logits, const int32_t* teacher_ids, const float* teacher_logp,
                                       const int32_t* targets, const mp_scale_state* st, mp_half* dlogits, void* ws, size_t ws_bytes, mp_mean_parts* parts,
                                       mp_stream stream) {
    const char* const what = "mp_distill_scaled";
    int               rc   = distill_check(d, what);
    if (rc != MP_OK) return rc;
    MP_REQUIRE(logits && teacher_ids && teacher_logp && st && dlogits && parts, "%s: NULL argument", what);
    MP_REQUIRE(targets || d->hard_weight == 0.f, "%s: a weight of hard labels without these", what);
    MP_REQUIRE(aligned(logits, 2) && aligned(dlogits, 2) && aligned(teacher_ids, 4) && aligned(teacher_logp, 4) && aligned(targets, 4) && aligned(st, 4),
               "%s: misaligned pointer", what);
    const bool        even = aligned16(logits) && d->ld % 8 == 0;
    const DistillPlan p    = distill_plan(d->rows, d->vocab, even);
    const size_t      need = distill_bytes(d->rows, p);
    if (!ws || !aligned16(ws) || ws_bytes < need) {
        set_error("%s: 16-byte aligned workspace of %zu bytes needed, %zu given", what, need, ws_bytes);
        return MP_E_WORKSPACE;
    }
    float* const row_loss = static_cast<float*>(ws);
    DistillArgs  a{d->rows, d->vocab, d->ld, d->top, p.chunks ? p.chunks : 1, p.chunk, d->inv_temperature * LOG2E, d->weight, d->inv_temperature, d->hard_weight,
                  logits, teacher_ids, d->hard_weight == 0.f ? nullptr : targets, teacher_logp, st, dlogits, row_loss, nullptr, nullptr};
    hipStream_t  hs = as_stream(stream);
    if (p.chunks) {
        a.sums   = reinterpret_cast<float*>(static_cast<char*>(ws) + round256((size_t)d->rows * sizeof(float)));
        a.chosen = a.sums + (size_t)d->rows * p.chunks * 4;
        const long long n = (long long)d->rows * p.chunks;
        rc = launch_distill<256, 8, DI_SUMS>(a, d, n, hs);
        if (rc == MP_OK) rc = launch_distill<256, 8, DI_GRADIENT>(a, d, n, hs);
    } else {
        const int  pieces = (d->vocab + (even ? 7 : 14)) / 8;
        const long long n = d->rows;
        // Waves of a row, and pieces a lane: what was fastest of two or three forms each, us for 8192 rows with 64 classes listed, r 0 or with the rest as
        // one: 4000 classes 4 a lane 39 / 45, 8 (half as many lanes) 42 / 47; 8192 classes 4 a lane 56 / 63, 2 70 / 76, 8 57 / 63; 16384: 8 109 / 111, 4 108
        // / 109, 2 131 / 148; 32768: 16 217 / 212, 8 207 / 198, 4 202 / 213; 1024 x 65536: 16 59 / 62, 8 63 / 69.
        if (pieces <= 64) rc = launch_distill<64, 1, DI_FUSED>(a, d, n, hs);
        else if (pieces <= 64 * 2) rc = launch_distill<64, 2, DI_FUSED>(a, d, n, hs);
        else if (pieces <= 64 * 4) rc = launch_distill<64, 4, DI_FUSED>(a, d, n, hs);
        else if (pieces <= 128 * 4) rc = launch_distill<128, 4, DI_FUSED>(a, d, n, hs);
        else if (pieces <= 256 * 4) rc = launch_distill<256, 4, DI_FUSED>(a, d, n, hs);
        else if (pieces <= 256 * 8) rc = launch_distill<256, 8, DI_FUSED>(a, d, n, hs);
        else if (pieces <= 512 * 8 && d->tail) rc = launch_distill<512, 8, DI_FUSED, 1>(a, d, n, hs);
        else if (pieces <= 512 * 8) rc = launch_distill<1024, 4, DI_FUSED, 0>(a, d, n, hs);
        else if (pieces <= 512 * 16) rc = launch_distill<512, 16, DI_FUSED>(a, d, n, hs);
        else rc = launch_distill<768, 22, DI_FUSED>(a, d, n, hs);
    }
    if (rc == MP_OK) *parts = mp_mean_parts{row_loss, (double)d->rows, d->rows, 0};
    return rc;
}

extern "C" int mp_distill_scaled(const mp_distill_desc* d, const mp_half* logits, const int32_t* teacher_ids, const float* teacher_logp, const int32_t* targets,
                                 const mp_scale_state* st, float* loss, mp_half* dlogits, void* ws, size_t ws_bytes, mp_stream stream) {
    MP_REQUIRE(loss && aligned(loss, 4), "mp_distill_scaled: loss is NULL or misaligned");
    mp_mean_parts parts;
    const int     rc = mp_distill_scaled_parts(d, logits, teacher_ids, teacher_logp, targets, st, dlogits, ws, ws_bytes, &parts, stream);
    return rc == MP_OK ? finish_mean_launch(parts, loss, as_stream(stream)) : rc;
}
