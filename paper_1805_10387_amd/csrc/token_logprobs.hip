// Log probabilities of given tokens, entropy, and the most likely alternatives of every row of logits; their gradient.
//
// z = x / temperature, lse = log sum exp z, logp = z[target] - lse, entropy = lse - sum p z.  One pass: a workgroup holds a row (or a
// chunk of one) in registers, sums against a running reference (vocab_rows.hpp), and picks the alternatives out of the
// registers.  Bound by HBM with many rows, by the chain of trips to memory and barriers with few, where rows are cut into more chunks
// and a second launch joins these.
//
// The top `k` of a chunk: the k-th largest of the lanes' own maxima is a bound that at least k elements reach, and with values that are
// spread over the lanes hardly more.  These are gathered in LDS, and each finds its place by counting those ahead of it, ties by
// index.  Where the bound says nothing (fewer lanes with finite values than k, NaN) or too many reach it (ties), the k-th largest value
// is found bit by bit instead, all 16 of them, and of its ties those with the lowest indices are taken.
#include <cmath>

#include "vocab_rows.hpp"

namespace mp {

constexpr int LP_THREADS = 256, LP_WAVES = LP_THREADS / 64;
constexpr int LP_FOUND   = 512;  // elements gathered; k is at most MP_TOP_MAX
constexpr int LP_CHUNKS  = 48;   // a row is cut into at most so many

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
// larger is better: the value, then the lower index.  0 is none.
__device__ __forceinline__ u64 make_entry(unsigned key, int index) { return ((u64)(key + 1) << 32) | (0x7FFFFFFFu - (unsigned)index); }
__device__ __forceinline__ unsigned entry_key(u64 e) { return (unsigned)(e >> 32) - 1; }
__device__ __forceinline__ int      entry_index(u64 e) { return (int)(0x7FFFFFFFu - (unsigned)e); }

struct TopLds {
    u64 found[LP_FOUND];
    int count, equal[LP_WAVES];
    unsigned short lane_key[LP_THREADS];
    float bound;
};

__device__ __forceinline__ unsigned half_of(const u32x4 q, int k) { return (k & 1) ? q[k >> 1] >> 16 : q[k >> 1] & 0xFFFFu; }

// k-th largest of the lanes' maxima as a value, by one wave; -inf where fewer have one
__device__ __forceinline__ float kth_of_lanes(const unsigned short* lane_key, int k) {
    unsigned key[LP_WAVES];
#pragma unroll
    for (int i = 0; i < LP_WAVES; ++i) key[i] = lane_key[i * 64 + (threadIdx.x & 63)];
    unsigned best = 0;
#pragma unroll
    for (int b = 15; b >= 0; --b) {
        const unsigned c = best | (1u << b);
        int            n = 0;
#pragma unroll
        for (int i = 0; i < LP_WAVES; ++i) n += __popcll(__ballot(key[i] >= c));
        if (n >= k) best = c;
    }
    return key_value(best);
}

// The same by value, bit by bit, from memory (the row is in a cache by now): any values, k elements exactly.
__device__ __forceinline__ int gather_exact(const Stretch z, const int first, const int k, TopLds& t) {
    const int  tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rounds = (z.pieces() + LP_THREADS - 1) / LP_THREADS;
    const auto each = [&](int v, const u32x4 q, auto&& pred) {  // elements of the stretch that are pred, as bits
        unsigned hit = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = 8 * v + j - z.head;
            hit |= (unsigned)(e >= 0 && e < z.len && pred(order_key(half_of(q, j)))) << j;
        }
        return hit;
    };
    const auto total = [&](int n) {  // over the workgroup, for every thread
        for (int far = 32; far; far >>= 1) n += __shfl_xor(n, far, 64);
        lds_barrier();
        if (lane == 0) t.equal[wave] = n;
        lds_barrier();
        int s = 0;
#pragma unroll
        for (int w = 0; w < LP_WAVES; ++w) s += t.equal[w];
        return s;
    };
    const auto count = [&](auto&& pred) {
        int n = 0;
        for (int i = 0; i < rounds; ++i) n += __popc(each(i * LP_THREADS + tid, z.load(i * LP_THREADS + tid), pred));
        return total(n);
    };
    unsigned best = 0;
    for (int b = 15; b >= 0; --b) {
        const unsigned c = best | (1u << b);
        if (count([&](unsigned key) { return key >= c; }) >= k) best = c;
    }
    int left = k - count([&](unsigned key) { return key > best; });  // of the elements equal to it, in the order of their indices
    if (tid == 0) t.count = 0;
    for (int i = 0; i < rounds; ++i) {
        const int      v    = i * LP_THREADS + tid;
        const u32x4    q    = z.load(v);
        const unsigned same = each(v, q, [&](unsigned key) { return key == best; });
        unsigned       hit  = each(v, q, [&](unsigned key) { return key > best; });
        int            upto = __popc(same);  // inclusive sum over the wave's lanes
        for (int far = 1; far < 64; far <<= 1) {
            const int n = __shfl_up(upto, far, 64);
            if (lane >= far) upto += n;
        }
        lds_barrier();
        if (lane == 63) t.equal[wave] = upto;
        lds_barrier();
        int ahead = upto - __popc(same), all = 0;
#pragma unroll
        for (int w = 0; w < LP_WAVES; ++w) {
            ahead += w < wave ? t.equal[w] : 0;
            all += t.equal[w];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if ((same >> j) & 1) hit |= (unsigned)(ahead++ < left) << j;
        left -= min(left, all);
        int at = atomicAdd(&t.count, __popc(hit));
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if ((hit >> j) & 1) t.found[at++] = make_entry(order_key(half_of(q, j)), first + 8 * v + j - z.head);
    }
    lds_barrier();
    return t.count;
}

// The k largest of the chunk into t.found, any order; returns their number or more.  All threads; ends with a barrier.
template <int VECS>
__device__ int gather_top(u32x4 (&raw)[VECS], const Stretch& z, int first, int k, float lane_top, bool plain, TopLds& t) {
    const int tid = threadIdx.x, wave = tid >> 6;
    t.lane_key[tid] = (unsigned short)order_key(f2h(lane_top));
    if (tid == 0) t.count = 0;
    lds_barrier();
    if (wave == 0) {
        const float b = kth_of_lanes(t.lane_key, k);
        if (tid == 0) t.bound = b;
    }
    lds_barrier();
    const float bound = t.bound;
    if (plain && bound > -INFINITY) {
        if (lane_top >= bound) {
#pragma unroll
            for (int i = 0; i < VECS; ++i) {
                asm("" : "+v"(raw[i]));  // (or the compiler keeps 100 registers of halves from the sums until here)
                if (max_of<1>(&raw[i]) >= bound) {
                    unsigned hit = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) hit |= (unsigned)(h2f((uint16_t)half_of(raw[i], j)) >= bound) << j;
                    const int at = atomicAdd(&t.count, __popc(hit));
                    int       n  = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if ((hit >> j) & 1) {
                            if (at + n < LP_FOUND) t.found[at + n] = make_entry(order_key(half_of(raw[i], j)), first + 8 * (i * LP_THREADS + tid) + j - z.head);
                            ++n;
                        }
                }
            }
        }
        lds_barrier();
        const int n = t.count;
        if (n <= LP_FOUND) return n;
    }
    return gather_exact(z, first, k, t);
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
    __device__ __forceinline__ void alternative(int place, u64 e) const {
        a.top_ids[row * a.top + place]  = entry_index(e);
        a.top_logp[row * a.top + place] = of(key_value(entry_key(e)));
    }
};

template <int VECS, bool TOP>
__global__ __launch_bounds__(LP_THREADS) void token_logprobs_kernel(const RowArgs a) {
    __shared__ float  red[LP_WAVES][4];
    const long long   row   = blockIdx.x / a.chunks;
    const int         chunk = blockIdx.x - (int)row * a.chunks, first = chunk * a.chunk, len = min(a.chunk, a.vocab - first);
    const Stretch     z(a.logits + row * a.ld + first, len);
    const int         tid = threadIdx.x;
    u32x4             raw[VECS];
#pragma unroll
    for (int i = 0; i < VECS; ++i) raw[i] = z.load(i * LP_THREADS + tid);
    constexpr int G = VECS < 4 ? VECS : 4;
    Sums<true>    sum(a.c2);
    float         lane_top = -INFINITY;
#pragma unroll
    for (int i = 0; i < VECS; i += G) {
        const float m = max_of<G>(raw + i);
        sum.add_pieces<G>(raw + i, a.c2, m);
        lane_top = fmaxf(lane_top, m);
    }
    sum.over_wave();
    if ((tid & 63) == 0) {
        red[tid >> 6][0] = sum.ref;
        red[tid >> 6][1] = sum.s;
        red[tid >> 6][2] = sum.t;
    }
    lds_barrier();
    Sums<true> all(a.c2);
#pragma unroll
    for (int w = 0; w < LP_WAVES; ++w) all.add_sums(red[w][0], red[w][1], red[w][2]);
    const RowOut out{a, row, all.ref, all.s, all.t};
    if (tid == 0) {
        if (a.chunks == 1) {
            out.row_values();
        } else {
            *reinterpret_cast<f32x4*>(a.sums + (row * a.chunks + chunk) * 4) = f32x4{all.ref, all.s, all.t, 0.f};
        }
    }
    if constexpr (TOP) {
        __shared__ TopLds top;
        const int         k = min(a.top, len), n = gather_top<VECS>(raw, z, first, k, lane_top, all.s < INFINITY, top);
        for (int i = tid; i < n; i += LP_THREADS) {
            const u64 mine  = top.found[i];
            int       place = 0;
            for (int j = 0; j < n; ++j) place += top.found[j] > mine;
            if (place < k) {
                if (a.chunks == 1) out.alternative(place, mine);
                else a.lists[(row * a.chunks + chunk) * a.top + place] = mine;
            }
        }
        if (a.chunks > 1)
            for (int i = k + tid; i < a.top; i += LP_THREADS) a.lists[(row * a.chunks + chunk) * a.top + i] = 0;
    }
}

// Chunks of a row joined: sums, and of the sorted lists the first `top`, each entry placed by how many are ahead of it in every list.
__global__ __launch_bounds__(LP_THREADS) void token_logprobs_join_kernel(const RowArgs a) {
    extern __shared__ u64 lists[];
    const long long       row = blockIdx.x;
    const int             n   = a.chunks * a.top;
    for (int i = threadIdx.x; i < n; i += LP_THREADS) lists[i] = a.lists[row * n + i];
    Sums<true> all(a.c2);
    for (int c = 0; c < a.chunks; ++c) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(a.sums + (row * a.chunks + c) * 4);
        all.add_sums(v[0], v[1], v[2]);
    }
    const RowOut out{a, row, all.ref, all.s, all.t};
    if (threadIdx.x == 0) out.row_values();
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += LP_THREADS) {
        const u64 mine = lists[i];
        if (mine == 0) continue;
        int place = 0;
        for (int c = 0; c < a.chunks && place < a.top; ++c) {
            int lo = 0, hi = a.top;  // entries of list c ahead of mine
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (lists[c * a.top + mid] > mine) lo = mid + 1;
                else hi = mid;
            }
            place += lo;
        }
        if (place < a.top) out.alternative(place, mine);
    }
}

// dx = RNE16(S c (g (1[target] - p) - h p (ln p + entropy))), S c = scale / temperature; bound by HBM (4 bytes an element).
constexpr int LPB_VECS = 4;
__global__ __launch_bounds__(LP_THREADS) void token_logprobs_bwd_kernel(const int vocab, const int ld, const int pieces, const uint16_t* logits,
                                                                        const int32_t* __restrict__ targets, const float c,
                                                                        const float* __restrict__ entropy, const float* __restrict__ lse,
                                                                        const float* __restrict__ dlogp, const float* __restrict__ dentropy,
                                                                        const mp_scale_state* __restrict__ st, uint16_t* dlogits) {
    const long long row   = blockIdx.x / pieces;
    const int       piece = blockIdx.x - (int)row * pieces;
    const Stretch   z(logits + row * ld, vocab);
    u32x4           raw[LPB_VECS];
#pragma unroll
    for (int i = 0; i < LPB_VECS; ++i) raw[i] = z.load((piece * LPB_VECS + i) * LP_THREADS + threadIdx.x);
    const int   y  = targets ? targets[row] : -1;
    const float sc = (st ? st->scale : 1.f) * c, g = dlogp && y >= 0 && y < vocab ? sc * dlogp[row] : 0.f, h = dentropy ? sc * dentropy[row] : 0.f;
    const float a = -(g + (dentropy ? h * entropy[row] : 0.f)), l = -lse[row];
    const bool  none = g == 0.f && h == 0.f;  // (whatever the row holds)
    const int   vt = g != 0.f ? (y + z.head) >> 3 : -1, kt = (y + z.head) & 7;
#pragma unroll
    for (int i = 0; i < LPB_VECS; ++i) {
        const int v = (piece * LPB_VECS + i) * LP_THREADS + threadIdx.x;
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

constexpr int LP_MOST = 16 * 8 * LP_THREADS;  // elements of a chunk that starts at a piece

struct ChunkPlan {
    int chunks, chunk;
};
// One chunk a row where that fills the chip; else as many as do, of 2048 elements or more.
// even: rows start at 16-byte pieces.  (Others may take a piece more.)
ChunkPlan chunk_plan(int rows, int vocab, bool even) {
    const int most = even ? LP_MOST : LP_MOST - 8;
    int       n    = (vocab + most - 1) / most;
    while (n * 2 <= LP_CHUNKS && (long long)rows * n * 2 <= 256 && vocab / (n * 2) >= 2048) n *= 2;
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
    const int         rc   = logprobs_check(what, rows, vocab, ld, inv_temperature);
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
    MP_REQUIRE(grid_fits((long long)rows * p.chunks, LP_THREADS), "%s: too many rows", what);
    RowArgs a{vocab, ld, top, p.chunks, p.chunk, logits, targets, inv_temperature * LOG2E, logp, entropy, lse, top_logp, top_ids, static_cast<float*>(ws), nullptr};
    if (p.chunks > 1) a.lists = reinterpret_cast<u64*>(static_cast<char*>(ws) + lists_offset(rows, p));
    hipStream_t hs     = as_stream(stream);
    const dim3  grid((unsigned)(rows * p.chunks)), block(LP_THREADS);
    const auto  launch = [&](auto vecs) {
        constexpr int V = decltype(vecs)::value;
        if (top) hipLaunchKernelGGL((token_logprobs_kernel<V, true>), grid, block, 0, hs, a);
        else hipLaunchKernelGGL((token_logprobs_kernel<V, false>), grid, block, 0, hs, a);
    };
    const int pieces = (p.chunk + (even ? 7 : 14)) / 8;
    if (pieces <= LP_THREADS) launch(std::integral_constant<int, 1>{});
    else if (pieces <= 2 * LP_THREADS) launch(std::integral_constant<int, 2>{});
    else if (pieces <= 4 * LP_THREADS) launch(std::integral_constant<int, 4>{});
    else if (pieces <= 8 * LP_THREADS) launch(std::integral_constant<int, 8>{});
    else launch(std::integral_constant<int, 16>{});
    MP_LAUNCH_CHECK("mp_token_logprobs");
    if (p.chunks > 1) {
        hipLaunchKernelGGL(token_logprobs_join_kernel, dim3(rows), block, (size_t)p.chunks * top * sizeof(u64), hs, a);
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
    const int pieces = ((vocab + 7 + 7) / 8 + LPB_VECS * LP_THREADS - 1) / (LPB_VECS * LP_THREADS);
    MP_REQUIRE(grid_fits((long long)rows * pieces, LP_THREADS), "%s: too many rows", what);
    hipLaunchKernelGGL(token_logprobs_bwd_kernel, dim3((unsigned)(rows * pieces)), dim3(LP_THREADS), 0, as_stream(stream), vocab, ld, pieces, logits, targets,
                       inv_temperature, entropy, lse, dlogp, dentropy, st, dlogits);
    MP_LAUNCH_CHECK("mp_token_logprobs_bwd");
    return MP_OK;
}
