// Log probabilities of given tokens, entropy, and the most likely alternatives of every row of logits; their gradient.
//
// z = x / temperature, lse = log sum exp z, logp = z[target] - lse, entropy = lse - sum p z.  One pass: a workgroup holds a row (or a
// chunk of one) in registers, sums against a running reference (vocab_rows.hpp), and picks the alternatives out of the
// registers.  Bound by HBM with many rows of many classes (8192 x 32768: 101 to 105 us, 5.1 to 5.3 TB/s; with 64 alternatives 109 to 111 us), by the
// search for the alternatives with short rows (8192 x 2000 with 20: 15.9 us, 8.8 without), by the chain of trips to memory and barriers with few
// (1 x 32768 with 20: 7.7 us).  Times here are of calls in a row, captured and replayed over the same buffers; where forward and backward take
// turns, forward (8192 x 32768) is 135 to 141 us, as it begins on the gradient's last stores, and backward 175.
//
// The top `k` of a chunk: the k-th largest of the lanes' own maxima (or the least of what each wave finds for its share of k) is a bound that at
// least k elements reach, and with values that are spread over the lanes hardly more.  These are gathered in LDS, and each finds its place by
// counting those ahead of it, ties by index.  Where the bound says nothing (fewer lanes with finite values than k, NaN) or too many reach it (ties), the k-th largest value
// is found bit by bit instead, all 16 of them, and of its ties those with the lowest indices are taken.
#include <cmath>

#include "vocab_rows.hpp"

namespace mp {

constexpr int LP_FOUND  = 512;    // elements gathered; k is at most MP_TOP_MAX
constexpr int LP_LOCAL  = 65536;  // elements of a chunk at most

typedef unsigned long long u64;

// fp16 as unsigned numbers in the same order; -0 is 0, and every NaN is above all others
__device__ __forceinline__ unsigned order_key(unsigned h) {
    if ((h & 0x7FFFu) > 0x7C00u) return 0xFFFFu;
    if ((h & 0x7FFFu) == 0) return 0x8000u;
    return (h & 0x8000u) ? (~h & 0xFFFFu) : (h | 0x8000u);
}
__device__ __forceinline__ float key_value(unsigned key) {
    return key == 0xFFFFu ? NAN : h2f((uint16_t)((key & 0x8000u) ? key & 0x7FFFu : ~key & 0xFFFFu));
}
// An element of a chunk in one word, larger is better: its key, then the lower index.  0 is none (no key is).
__device__ __forceinline__ unsigned make_entry(unsigned key, int local) { return (key << 16) | (unsigned)(LP_LOCAL - 1 - local); }
__device__ __forceinline__ unsigned entry_key(unsigned e) { return e >> 16; }
__device__ __forceinline__ int      entry_local(unsigned e) { return LP_LOCAL - 1 - (int)(e & (LP_LOCAL - 1)); }
// ... of a row
__device__ __forceinline__ u64      far_entry(unsigned key, int index) { return ((u64)key << 32) | (0x7FFFFFFFu - (unsigned)index); }
__device__ __forceinline__ unsigned far_key(u64 e) { return (unsigned)(e >> 32); }
__device__ __forceinline__ int      far_index(u64 e) { return (int)(0x7FFFFFFFu - (unsigned)e); }

template <int THREADS>
struct TopLds {
    static constexpr int WAVES = THREADS / 64, HELD = WAVES > 4 ? 64 : WAVES > 1 ? 128 : 160;
    u32x4          found[LP_FOUND / 4];  // entries, zeros behind them up to a multiple of 16
    u32x4          piece[WAVES][HELD];   // pieces with an element that reaches the bound
    unsigned short place[WAVES][HELD];   // and which they are
    unsigned short best[256];            // bound_of_all()
    float          bound;
    int            count, equal[WAVES];
    __device__ __forceinline__ unsigned& entry(int i) { return reinterpret_cast<unsigned*>(found)[i]; }
};

__device__ __forceinline__ unsigned half_of(const u32x4 q, int k) { return (k & 1) ? q[k >> 1] >> 16 : q[k >> 1] & 0xFFFFu; }

// k-th largest of the wave's 64 N keys as a value.  (Not above -inf where fewer than k have one.)
template <int N>
__device__ __forceinline__ float kth_of(const unsigned (&key)[N], int k) {
    unsigned best = 0;
#pragma unroll
    for (int b = 15; b >= 0; --b) {
        const unsigned c = best | (1u << b);
        int            n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__ballot(key[i] >= c));
        if (n >= k) best = c;
    }
    return key_value(best);
}

__device__ __forceinline__ int lanes_ahead(u64 mask) {  // set bits of lower lanes
    return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u));
}

// The k largest of the chunk by value, bit by bit: any values, k elements exactly.  A lane with one piece keeps it, otherwise they are read
// again (the row is in a cache by now; four pieces a lane kept take 140 registers, and 4096 x 2000 with 100 alternatives 26 us, not 19).
template <int THREADS, int VECS>
__device__ __forceinline__ int gather_exact(const u32x4 (&raw)[VECS], const Stretch& z, const int k, TopLds<THREADS>& t) {
    constexpr int  WAVES = THREADS / 64;
    constexpr bool KEPT = WAVES == 1 && VECS == 1;
    const int      tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rounds = (z.pieces() + THREADS - 1) / THREADS;
    // f(key + 1, or 0 outside the stretch; element)
    const auto each = [&](int v, const u32x4 q, auto&& f) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = 8 * v + j - z.head;
            f(e >= 0 && e < z.len ? order_key(half_of(q, j)) + 1 : 0u, e);
        }
    };
    const auto every_piece = [&](auto&& f) {
        if (KEPT) {
            f(tid, raw[0]);
        } else {
#pragma unroll 1
            for (int i = 0; i < rounds; ++i) f(i * THREADS + tid, z.load(i * THREADS + tid));
        }
    };
    const auto count = [&](unsigned from) {  // elements whose key + 1 is at least that
        int n = 0;
        every_piece([&](int v, const u32x4 q) { each(v, q, [&](unsigned key, int) { n += KEPT ? __popcll(__ballot(key >= from)) : (int)(key >= from); }); });
        if (KEPT) return n;
        n = (int)wave_sum((float)n);
        if (WAVES == 1) return n;
        lds_barrier();
        if (lane == 0) t.equal[wave] = n;
        lds_barrier();
        int s = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += t.equal[w];
        return s;
    };
    unsigned best = 0;  // a key + 1
    for (int b = 16; b >= 0; --b) {
        const unsigned c = best | (1u << b);
        if (c <= 0x10000u && count(c) >= k) best = c;
    }
    int left = k - count(best + 1);  // of the elements equal to it, in the order of their indices
    if (tid == 0) t.count = 0;
    every_piece([&](int v, const u32x4 q) {
        unsigned same = 0, hit = 0;
        int      j    = 0;
        each(v, q, [&](unsigned key, int) {
            same |= (unsigned)(key == best) << j;
            hit |= (unsigned)(key > best) << j;
            ++j;
        });
        int upto = __popc(same);  // inclusive sum over the wave's lanes
        for (int far = 1; far < 64; far <<= 1) {
            const int n = __shfl_up(upto, far, 64);
            if (lane >= far) upto += n;
        }
        lds_barrier();
        if (lane == 63) t.equal[wave] = upto;
        lds_barrier();
        int ahead = upto - __popc(same), all = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            ahead += w < wave ? t.equal[w] : 0;
            all += t.equal[w];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((same >> i) & 1) hit |= (unsigned)(ahead++ < left) << i;
        left -= min(left, all);
        int at = atomicAdd(&t.count, __popc(hit));
        j      = 0;
        each(v, q, [&](unsigned key, int e) {
            if ((hit >> j++) & 1) t.entry(at++) = make_entry(key - 1, e);
        });
    });
    lds_barrier();
    return t.count;
}

// Keys of the largest elements of a lane's pieces, each N-th of these together.
template <int N, int VECS>
__device__ __forceinline__ void lane_keys(const u32x4 (&raw)[VECS], unsigned (&key)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int j = i; j < VECS; j += N) top = fmaxf(top, max_of<1>(&raw[j]));
        key[i] = order_key(f2h(top));
    }
}
// A value that at least k of the wave's elements reach, and not many more: the k-th largest of the lanes' maxima.  A wave by itself, whose
// lanes are few beside k, takes those of pieces, or of halves of them where they would be fewer than twice k (8192 x 1000, 20 and 100
// alternatives: pieces 12.3 and 39.6 us, halves 14.4 and 27.7).
template <int THREADS, int VECS>
__device__ __forceinline__ float wave_bound(const u32x4 (&raw)[VECS], float lane_top, int k) {
    if constexpr (THREADS == 64) {
        if (VECS <= 2 && k > 32 * VECS) {
            unsigned halves[2 * VECS];
#pragma unroll
            for (int i = 0; i < 2 * VECS; ++i) halves[i] = order_key(f2h(max_of_half(raw[i >> 1], i & 1)));
            return kth_of<2 * VECS>(halves, k);
        }
        unsigned pieces[VECS];
        lane_keys<VECS>(raw, pieces);
        return kth_of<VECS>(pieces, k);
    } else if constexpr (THREADS == 128) {
        unsigned two[2];
        lane_keys<2>(raw, two);
        return kth_of<2>(two, k);
    } else {
        const unsigned one[1] = {order_key(f2h(lane_top))};
        return kth_of<1>(one, k);
    }
}
// The same of all waves' elements, 256 keys of a lane, of two lanes or of half a lane's pieces: keys_in() before a barrier, bound_of_all()
// behind it.  Ends with a barrier.
template <int THREADS, int VECS>
__device__ __forceinline__ void keys_in(const u32x4 (&raw)[VECS], float lane_top, TopLds<THREADS>& t) {
    const int tid = threadIdx.x;
    if constexpr (THREADS == 128) {
        unsigned two[2];
        lane_keys<2>(raw, two);
        t.best[tid]           = (unsigned short)two[0];
        t.best[THREADS + tid] = (unsigned short)two[1];
    } else {
        constexpr int SHARE = THREADS / 256;
        const float   top   = SHARE == 2 ? fmaxf(lane_top, __shfl_xor(lane_top, 1, 64)) : lane_top;
        if (tid % SHARE == 0) t.best[tid / SHARE] = (unsigned short)order_key(f2h(top));
    }
}
template <int THREADS>
__device__ __forceinline__ float bound_of_all(int k, TopLds<THREADS>& t) {
    if (threadIdx.x < 64) {
        unsigned key[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) key[i] = t.best[i * 64 + threadIdx.x];
        const float b = kth_of<4>(key, k);
        if (threadIdx.x == 0) t.bound = b;
    }
    lds_barrier();
    return t.bound;
}

// The k largest of the chunk, and few others, into t.found in any order; returns their number.  All threads, t.count 0; ends with a barrier.
// bound: a value that at least k elements reach.
template <int THREADS, int VECS>
__device__ __forceinline__ int gather_top(u32x4 (&raw)[VECS], const Stretch& z, int k, float bound, bool plain, TopLds<THREADS>& t) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tid = threadIdx.x;
    if (plain && bound > -INFINITY) {
        // each wave its pieces, then eight of these at a time, a lane an element
        constexpr int HELD  = TopLds<THREADS>::HELD;
        int           held  = 0;
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            asm("" : "+v"(raw[i]));  // (or the compiler keeps 100 registers of halves from the sums until here)
            const bool hit  = max_of<1>(&raw[i]) >= bound;
            const u64  mask = __ballot(hit);
            if (mask) {
                const int at = held + lanes_ahead(mask);
                if (hit && at < HELD) {
                    t.piece[wave][at] = raw[i];
                    t.place[wave][at] = (unsigned short)(i * THREADS + tid);
                }
                held += __popcll(mask);
            }
        }
        __builtin_amdgcn_wave_barrier();
        for (int b = 0; b < min(held, HELD); b += 8) {
            const int p = b + (lane >> 3), j = lane & 7;
            unsigned  h = 0xFC00u;
            if (p < min(held, HELD)) h = reinterpret_cast<const unsigned short*>(&t.piece[wave][p])[j];
            const bool ok   = h2f((uint16_t)h) >= bound;
            const u64  mask = __ballot(ok);
            int        base = 0;
            if (lane == 0) base = atomicAdd(&t.count, __popcll(mask));
            const int at = __builtin_amdgcn_readfirstlane(base) + lanes_ahead(mask);
            if (ok && at < LP_FOUND) t.entry(at) = make_entry(order_key(h), 8 * t.place[wave][p] + j - z.head);
        }
        if (held > HELD && lane == 0) atomicAdd(&t.count, LP_FOUND + 1);
        lds_barrier();
        const int n = t.count;
        if (n <= LP_FOUND) return n;
    }
    return gather_exact<THREADS, VECS>(raw, z, k, t);
}

// f(place, entry) for the k best of n entries, each placed by the number ahead of it.
template <int THREADS, typename F>
__device__ __forceinline__ void place_entries(TopLds<THREADS>& t, int n, int k, F&& f) {
    const int tid = threadIdx.x, padded = (n + 15) & ~15;
    if (tid < padded - n) t.entry(n + tid) = 0;
    lds_barrier();
    for (int i = tid; i < n; i += THREADS) {
        const unsigned mine  = t.entry(i);
        int            place = 0;
        for (int j = 0; j < padded / 4; j += 4) {
            u32x4 e[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) e[u] = t.found[j + u];
#pragma unroll
            for (int u = 0; u < 16; ++u) place += e[u >> 2][u & 3] > mine;
        }
        if (place < k) f(place, mine);
    }
}

struct RowArgs {
    int             vocab, ld, top, chunks, chunk;  // chunk: elements of one, a multiple of 8 where there are several
    const uint16_t* logits;
    const int32_t*  targets;
    float           c2;
    float *         logp, *entropy, *lse, *top_logp;
    int32_t*        top_ids;
    float*          sums;   // several chunks: [row][chunk][4]
    u64*            lists;  // [row][chunk][top]
};

struct RowOut {
    const RowArgs& a;
    long long      row;
    float          ref, s, t;
    __device__ __forceinline__ float of(float x) const { return LN2 * (fmaf(x, a.c2, -ref) - log2f(s)); }
    __device__ __forceinline__ void  row_values() const {
        if (a.targets && a.logp) {
            const int y = a.targets[row];
            a.logp[row] = y >= 0 && y < a.vocab ? of(h2f(a.logits[row * a.ld + y])) : 0.f;
        }
        const float log_s = log2f(s);
        if (a.lse) a.lse[row] = s == 0.f ? -INFINITY : LN2 * (ref + log_s);
        if (a.entropy) a.entropy[row] = LN2 * (log_s - t / s);
    }
    __device__ __forceinline__ void alternative(int place, int index, unsigned key) const {
        a.top_ids[row * a.top + place]  = index;
        a.top_logp[row * a.top + place] = of(key_value(key));
    }
};

template <int THREADS, int VECS, bool TOP>
__global__ __launch_bounds__(THREADS) void token_logprobs_kernel(const RowArgs a) {
    constexpr int    WAVES = THREADS / 64;
    __shared__ float red[WAVES][4];
    __shared__ std::conditional_t<TOP, TopLds<THREADS>, int> top;
    const long long  row   = blockIdx.x / a.chunks;
    const int        chunk = blockIdx.x - (int)row * a.chunks, first = chunk * a.chunk, len = min(a.chunk, a.vocab - first);
    const Stretch    z(a.logits + row * a.ld + first, len);
    const int        tid = threadIdx.x;
    u32x4            raw[VECS], last;
    load_pieces<THREADS>(z, tid, raw, last);
    constexpr int G = VECS < 4 ? VECS : THREADS > 256 ? 2 : 4;
    Sums<true>    sum(a.c2);
    float         lane_top = -INFINITY;
#pragma unroll
    for (int i = 0; i < VECS; i += G) {
#pragma unroll
        for (int j = 0; j < G; ++j) settle<THREADS>(z, i + j, tid, raw[i + j], last);
        if (i * THREADS < z.pieces()) {
            const float m = max_of<G>(raw + i);
            sum.add_pieces<G>(raw + i, a.c2, m);
            lane_top = fmaxf(lane_top, m);
        }
    }
    // The waves find their bounds side by side ahead of the barrier, each for its share of k, and take the least; where the shares are long, which
    // makes that one loose, one wave finds it from all lanes behind it (8192 x 8192, 20, 64 and 128 alternatives: shares 34.9, 44.1 and 61.4 us,
    // one wave 35.5, 41.9 and 56.7; 1 x 32768, 20: 7.9 and 8.5).
    constexpr int SHARE = THREADS == 128 ? 16 : 6;  // of lanes with two keys, one
    const int     k = min(a.top, len);
    const bool    shares = WAVES == 1 || k <= SHARE * WAVES;
    float         bound  = -INFINITY;
    if constexpr (TOP) {
        if (tid == 0) top.count = 0;
        if (shares) bound = wave_bound<THREADS, VECS>(raw, lane_top, (k + WAVES - 1) / WAVES);
        else if constexpr (WAVES > 1) keys_in<THREADS, VECS>(raw, lane_top, top);
    }
    sum.over_wave();
    if (WAVES > 1) {
        if ((tid & 63) == 0) {
            red[tid >> 6][0] = sum.ref;
            red[tid >> 6][1] = sum.s;
            red[tid >> 6][2] = sum.t;
            red[tid >> 6][3] = bound;
        }
        lds_barrier();
        sum = Sums<true>(a.c2);
#pragma unroll 4
        for (int w = 0; w < WAVES; ++w) {
            sum.add_sums(red[w][0], red[w][1], red[w][2]);
            bound = fminf(bound, red[w][3]);
        }
        asm("" : "+v"(sum.ref), "+v"(sum.s), "+v"(sum.t));  // (or what they are made of stays in registers to the end)
    }
    const RowOut out{a, row, sum.ref, sum.s, sum.t};
    if constexpr (TOP) {
        if constexpr (WAVES > 1) {
            if (shares && bound == -INFINITY) {  // (a wave has too few finite elements: are there enough in all lanes?)
                keys_in<THREADS, VECS>(raw, lane_top, top);
                lds_barrier();
                bound = bound_of_all(k, top);
            } else if (!shares) {
                bound = bound_of_all(k, top);
            }
        }
        const int  n    = gather_top<THREADS, VECS>(raw, z, k, bound, sum.s < INFINITY, top);
        u64* const list = a.lists + (row * a.chunks + chunk) * a.top;
        place_entries<THREADS>(top, n, k, [&](int place, unsigned e) {
            const int index = first + entry_local(e);
            if (a.chunks == 1) out.alternative(place, index, entry_key(e));
            else list[place] = far_entry(entry_key(e), index);
        });
        if (a.chunks > 1)
            for (int i = k + tid; i < a.top; i += THREADS) list[i] = 0;
    }
    if (tid == THREADS - 64) {  // (a wave that has few of the places to find, or none)
        if (a.chunks == 1) out.row_values();
        else *reinterpret_cast<f32x4*>(a.sums + (row * a.chunks + chunk) * 4) = f32x4{sum.ref, sum.s, sum.t, 0.f};
    }
}

// Chunks of a row joined: sums, and of the sorted lists the first `top`.  Every list has at least ceil(top / chunks) entries that reach
// the least of the lists' entries at that place; those that do are gathered and placed by counting.
constexpr int JOIN_THREADS = 256;
__global__ __launch_bounds__(JOIN_THREADS) void token_logprobs_join_kernel(const RowArgs a) {
    extern __shared__ u64 found[];
    __shared__ int        count;
    const long long       row = blockIdx.x;
    const int             n = a.chunks * a.top, tid = threadIdx.x, lane = tid & 63;
    const u64*            lists = a.lists + row * n;
    Sums<true>            all(a.c2);
    f32x4                 v = {all.ref, 0.f, 0.f, 0.f};
    u64                   bound = ~0ull;
    if (lane < a.chunks) {
        v = *reinterpret_cast<const f32x4*>(a.sums + (row * a.chunks + lane) * 4);
        if (a.top) bound = lists[lane * a.top + (a.top + a.chunks - 1) / a.chunks - 1];
    }
    all.add_sums(v[0], v[1], v[2]);
    all.over_wave();
    const RowOut out{a, row, all.ref, all.s, all.t};
    if (tid == 0) out.row_values();
    if (a.top == 0) return;
    for (int far = 32; far; far >>= 1) bound = min(bound, (u64)__shfl_xor((unsigned long long)bound, far, 64));
    if (tid == 0) count = 0;
    lds_barrier();
    for (int i = tid; i < n; i += JOIN_THREADS) {
        const u64 e = lists[i];
        if (e != 0 && e >= bound) found[atomicAdd(&count, 1)] = e;
    }
    lds_barrier();
    const int m = count;
    if (tid < ((m + 7) & ~7) - m) found[m + tid] = 0;
    lds_barrier();
    for (int i = tid; i < m; i += JOIN_THREADS) {
        const u64 mine  = found[i];
        int       place = 0;
        for (int j = 0; j < m; j += 8)
#pragma unroll
            for (int u = 0; u < 8; ++u) place += found[j + u] > mine;
        if (place < a.top) out.alternative(place, far_index(mine), far_key(mine));
    }
}

// dx = RNE16(S c (g (1[target] - p) - h p (ln p + entropy))), S c = scale / temperature; bound by HBM (4 bytes an element; 8192 x 32768 194 us,
// 5.5 TB/s).
constexpr int LPB_VECS = 4, LPB_THREADS = 256;
__global__ __launch_bounds__(LPB_THREADS) void token_logprobs_bwd_kernel(const int vocab, const int ld, const int pieces, const uint16_t* logits,
                                                                        const int32_t* __restrict__ targets, const float c,
                                                                        const float* __restrict__ entropy, const float* __restrict__ lse,
                                                                        const float* __restrict__ dlogp, const float* __restrict__ dentropy,
                                                                        const mp_scale_state* __restrict__ st, uint16_t* dlogits) {
    const long long row   = blockIdx.x / pieces;
    const int       piece = blockIdx.x - (int)row * pieces;
    const Stretch   z(logits + row * ld, vocab);
    u32x4           raw[LPB_VECS];
#pragma unroll
    for (int i = 0; i < LPB_VECS; ++i) raw[i] = z.load((piece * LPB_VECS + i) * LPB_THREADS + threadIdx.x);
    const int   y  = targets ? targets[row] : -1;
    const float sc = (st ? st->scale : 1.f) * c, g = dlogp && y >= 0 && y < vocab ? sc * dlogp[row] : 0.f, h = dentropy ? sc * dentropy[row] : 0.f;
    const float a = -(g + (dentropy ? h * entropy[row] : 0.f)), l = -lse[row];
    const bool  none = g == 0.f && h == 0.f;  // (whatever the row holds)
    const int   vt = g != 0.f ? (y + z.head) >> 3 : -1, kt = (y + z.head) & 7;
#pragma unroll
    for (int i = 0; i < LPB_VECS; ++i) {
        const int v = (piece * LPB_VECS + i) * LPB_THREADS + threadIdx.x;
        float     d[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float lp = fmaf((float)as_pair(raw[i][k >> 1])[k & 1], c, l);
            d[k]           = none ? 0.f : __builtin_amdgcn_exp2f(lp * LOG2E) * fmaf(-h, fmaxf(lp, -150.f), a);
        }
        if (v == vt) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k == kt) d[k] += g;
        }
        u32x4 q;
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = (unsigned)f2h(d[2 * k]) | ((unsigned)f2h(d[2 * k + 1]) << 16);
        z.store(dlogits + row * ld, v, q);
    }
}

}  // namespace mp

using namespace mp;

namespace {

constexpr int LP_MOST = LP_LOCAL;  // elements of a chunk that starts at a piece

struct ChunkPlan {
    int chunks, chunk;
};
// As few chunks as hold a row: the second launch, which joins them, and the trips of more workgroups cost what shorter chunks save (20 alternatives,
// us of 1, 2, 4, 8 and 16 chunks: 1 x 32768 8.0, 10.3, 9.4, 9.2, 10.6; 1 x 65536 10.2, 11.8, 10.4, 9.4, 9.9; 16 x 50021 10.8, 13.2, 11.3, 10.8, 11.1;
// 8 alternatives, 2, 4, 8 and 16 chunks: 1 x 131071 9.9, 9.9, 9.9, 9.7; 64 x 131071 14.3, 14.8, 14.0, 15.2; 200 x 131071 27.0, 28.3, 26.7, 28.8).
// even: rows start at 16-byte pieces.  (Others may take a piece more.)
ChunkPlan chunk_plan(int rows, int vocab, bool even) {
    const int most = even ? LP_MOST : LP_MOST - 8;
    const int n    = (vocab + most - 1) / most;
    if (n == 1) return {1, vocab};
    const int chunk = ((vocab + n - 1) / n + 7) / 8 * 8;
    return {(vocab + chunk - 1) / chunk, chunk};
}
size_t lists_offset(int rows, const ChunkPlan& p) { return (size_t)rows * p.chunks * 16; }
size_t logprobs_bytes(int rows, int vocab, int top, bool even) {
    const ChunkPlan p = chunk_plan(rows, vocab, even);
    return p.chunks == 1 ? 0 : lists_offset(rows, p) + (size_t)rows * p.chunks * top * sizeof(u64);
}
int logprobs_check(const char* what, int rows, int vocab, int ld, float inv_temperature) {
    MP_REQUIRE(rows >= 0 && vocab > 0 && ld >= vocab, "%s: bad shape rows=%d vocab=%d ld=%d", what, rows, vocab, ld);
    MP_REQUIRE(inv_temperature >= 0x1p-8f && inv_temperature <= 0x1p8f, "%s: 1 / temperature outside 2^-8 .. 2^8", what);
    if (vocab > MP_VOCAB_MAX) {
        set_error("%s: vocabularies up to %d", what, MP_VOCAB_MAX);
        return MP_E_UNSUPPORTED;
    }
    return MP_OK;
}

}  // namespace

extern "C" size_t mp_token_logprobs_workspace_bytes(int rows, int vocab, int top) {
    if (rows <= 0 || vocab <= 0 || vocab > MP_VOCAB_MAX || top < 0 || top > MP_TOP_MAX || top > vocab) return 0;
    const size_t even = logprobs_bytes(rows, vocab, top, true), any = logprobs_bytes(rows, vocab, top, false);
    return even > any ? even : any;
}

extern "C" int mp_token_logprobs(int rows, int vocab, int top, const mp_half* logits, int ld, const int32_t* targets, float inv_temperature, float* logp,
                                 float* entropy, float* lse, int32_t* top_ids, float* top_logp, void* ws, size_t ws_bytes, mp_stream stream) {
    const char* const what = "mp_token_logprobs";
    int               rc   = logprobs_check(what, rows, vocab, ld, inv_temperature);
    if (rc != MP_OK) return rc;
    MP_REQUIRE(top >= 0 && top <= vocab, "%s: %d alternatives of %d", what, top, vocab);
    if (top > MP_TOP_MAX) {
        set_error("%s: up to %d alternatives", what, MP_TOP_MAX);
        return MP_E_UNSUPPORTED;
    }
    if (rows == 0) return MP_OK;
    MP_REQUIRE(logits, "%s: NULL argument", what);
    MP_REQUIRE((targets != nullptr) == (logp != nullptr), "%s: targets and their log probabilities are given together", what);
    MP_REQUIRE((top > 0) == (top_ids != nullptr) && (top > 0) == (top_logp != nullptr), "%s: ids and log probabilities of alternatives go with top > 0", what);
    MP_REQUIRE(aligned(logits, 2) && aligned(targets, 4) && aligned(logp, 4) && aligned(entropy, 4) && aligned(lse, 4) && aligned(top_ids, 4) && aligned(top_logp, 4),
               "%s: misaligned pointer", what);
    const bool      even = aligned16(logits) && ld % 8 == 0;
    const ChunkPlan p    = chunk_plan(rows, vocab, even);
    const size_t    need = logprobs_bytes(rows, vocab, top, even);
    if (need > 0 && (!ws || !aligned16(ws) || ws_bytes < need)) {
        set_error("%s: 16-byte aligned workspace of %zu bytes needed, %zu given", what, need, ws_bytes);
        return MP_E_WORKSPACE;
    }
    RowArgs a{vocab, ld, top, p.chunks, p.chunk, logits, targets, inv_temperature * LOG2E, logp, entropy, lse, top_logp, top_ids, static_cast<float*>(ws), nullptr};
    if (p.chunks > 1) a.lists = reinterpret_cast<u64*>(static_cast<char*>(ws) + lists_offset(rows, p));
    hipStream_t hs     = as_stream(stream);
    const auto  launch = [&](auto threads, auto vecs) -> int {
        constexpr int T = decltype(threads)::value, V = decltype(vecs)::value;
        MP_REQUIRE(grid_fits((long long)rows * p.chunks, T), "%s: too many rows", what);
        const dim3 grid((unsigned)(rows * p.chunks));
        if (top) hipLaunchKernelGGL((token_logprobs_kernel<T, V, true>), grid, dim3(T), 0, hs, a);
        else hipLaunchKernelGGL((token_logprobs_kernel<T, V, false>), grid, dim3(T), 0, hs, a);
        MP_LAUNCH_CHECK("mp_token_logprobs");
        return MP_OK;
    };
    const int pieces = (p.chunk + (even ? 7 : 14)) / 8;
    typedef std::integral_constant<int, 64>   W1;
    typedef std::integral_constant<int, 128>  W2;
    typedef std::integral_constant<int, 256>  W4;
    typedef std::integral_constant<int, 512>  W8;
    typedef std::integral_constant<int, 1>    V1;
    typedef std::integral_constant<int, 2>    V2;
    typedef std::integral_constant<int, 4>    V4;
    typedef std::integral_constant<int, 8>    V8;
    typedef std::integral_constant<int, 16>   V16;
    // Waves of a row and pieces a lane, us with 8 alternatives, 8192 rows and 1: of 2000 64 x 4 14.9 and 5.7, 128 x 2 18.2 and 5.2; of 4000 128 x 4 22.8
    // and 5.3 (1024 rows 6.8, 512 6.7), 256 x 2 28.5 and 5.0 (7.3, 5.9); of 8192 128 x 8 32.3 and 6.0, 256 x 4 35.4 and 5.4; of 16384 256 x 8 51.7 and 6.1,
    // 512 x 4 74.7 and 6.2; of 32768 256 x 16 101 and 7.9, 512 x 8 118 and 7.3 (128 rows alike, 256 rows 9.2 and 9.4).
    if (pieces <= 64) rc = launch(W1{}, V1{});
    else if (pieces <= 128) rc = launch(W1{}, V2{});
    else if (pieces <= 256) rc = launch(W1{}, V4{});
    else if (pieces <= 512 && rows >= 1024) rc = launch(W2{}, V4{});
    else if (pieces <= 512) rc = launch(W4{}, V2{});
    else if (pieces <= 1024) rc = launch(W4{}, V4{});
    else if (pieces <= 2048) rc = launch(W4{}, V8{});
    else if (pieces <= 4096 && rows <= 64) rc = launch(W8{}, V8{});
    else if (pieces <= 4096) rc = launch(W4{}, V16{});
    else rc = launch(W8{}, V16{});
    if (rc != MP_OK) return rc;
    if (p.chunks > 1) {
        hipLaunchKernelGGL(token_logprobs_join_kernel, dim3(rows), dim3(JOIN_THREADS), ((size_t)p.chunks * top + 8) * sizeof(u64), hs, a);
        MP_LAUNCH_CHECK("mp_token_logprobs(join)");
    }
    return MP_OK;
}

extern "C" int mp_token_logprobs_bwd(int rows, int vocab, const mp_half* logits, int ld, const int32_t* targets, float inv_temperature, const float* entropy,
                                     const float* lse, const float* dlogp, const float* dentropy, const mp_scale_state* st, mp_half* dlogits,
                                     mp_stream stream) {
    const char* const what = "mp_token_logprobs_bwd";
    const int         rc   = logprobs_check(what, rows, vocab, ld, inv_temperature);
    if (rc != MP_OK) return rc;
    if (rows == 0) return MP_OK;
    MP_REQUIRE(logits && lse && dlogits && (dlogp || dentropy), "%s: NULL argument", what);
    MP_REQUIRE((targets != nullptr) == (dlogp != nullptr), "%s: targets and the gradient of their log probabilities are given together", what);
    MP_REQUIRE(!dentropy || entropy, "%s: a gradient of the entropy needs the entropy", what);
    MP_REQUIRE(aligned(logits, 2) && aligned(dlogits, 2) && aligned(st, 4) && aligned(targets, 4) && aligned(entropy, 4) && aligned(lse, 4) && aligned(dlogp, 4) && aligned(dentropy, 4),
               "%s: misaligned pointer", what);
    const int pieces = ((vocab + 7 + 7) / 8 + LPB_VECS * LPB_THREADS - 1) / (LPB_VECS * LPB_THREADS);
    MP_REQUIRE(grid_fits((long long)rows * pieces, LPB_THREADS), "%s: too many rows", what);
    hipLaunchKernelGGL(token_logprobs_bwd_kernel, dim3((unsigned)(rows * pieces)), dim3(LPB_THREADS), 0, as_stream(stream), vocab, ld, pieces, logits, targets,
                       inv_temperature, entropy, lse, dlogp, dentropy, st, dlogits);
    MP_LAUNCH_CHECK("mp_token_logprobs_bwd");
    return MP_OK;
}
