// Embedding lookup with scaling, and the table's gradient by sorted tokens.
//
// Both are bound by HBM: forward reads a table row per token (or finds it in the caches) and writes a row, backward reads a gradient row
// per token and writes the whole table's gradient.  Gradient rows of one token are summed in fp32 in the order of their positions:
//   1. sort    runs of SORT_RUN tokens (value, then position: one 32-bit key); the other workgroups of the launch clear dw
//   2. merge   up to MERGE_RUNS runs into one, each key's place by binary searches (not for a single run)
//   3. sum     a chunk of sorted positions a group of lanes, however they are spread over tokens: a token's sum that lies inside a
//              chunk is stored, one that crosses a border is left as partial sums
//   4. join    partial sums, in the order of the chunks
// so that a token that comes once costs no more than its row, without an atomic addition.  A frequent one does: its partial sums are joined by
// one group of lanes, 16 chunks a trip to memory.  One word taking none, a quarter, a half of the tokens, the whole gradient in us: 8192
// rows of 1024 36 / 56 / 79, 65521 of 515 78 / 124 / 181, 2^20 of 128 354 / 950 / 1597.
// us forward / sort / merge / sum / join, the word of rank r about as often as 1 / (r + 3): 61 rows of 192 2.8 / 2.7 / - / 7.7 / 3.5 (launches),
// 8192 of 1024 and 32768 words 8.4 (4.0 TB/s) / 11.8 (the clearing, 5.7 TB/s) / 6.4 / 12.7 / 6.6, 65521 of 515 and 50021 words
// 31.9 (3.7 TB/s) / 9.6 / 21.6 / 42.5 / 9.4.
#include "common.hpp"

namespace mp {

typedef unsigned u32x4e __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int EMB_THREADS = 256;
constexpr int SORT_RUN    = 2048;   // 11 bits of position beside 21 bits of token
constexpr int SORT_BITS   = 11;
constexpr int MERGE_RUNS  = 32;
constexpr int EMB_BATCH   = 8;
constexpr int FILL_WGS    = 2048;

// The product rounded to fp32 before it is rounded to fp16: the compiler else makes one instruction of the two in some places,
// which rounds once (an element in 10^4 differs, and a call with `add` from one without).
__device__ __forceinline__ float scaled(float x, float scale) {
    x *= scale;
    asm("" : "+v"(x));
    return x;
}

// 8 elements of a row that may begin at any element.  A load asks for the four words, or five, that hold them: each holds one of the 8 at
// least, so nothing behind a page is touched.
typedef u32x4e   u32x4e_any __attribute__((aligned(2)));
typedef u32x4e   u32x4e_word __attribute__((aligned(4)));
typedef f32x4    f32x4_word __attribute__((aligned(4)));
struct Words {
    unsigned v[5];
    int      odd;
    __device__ __forceinline__ Words() {}
    __device__ __forceinline__ explicit Words(const uint16_t* p) {
        odd               = (int)(reinterpret_cast<uintptr_t>(p) >> 1) & 1;
        const unsigned* q = reinterpret_cast<const unsigned*>(p - odd);
        const u32x4e    w = *reinterpret_cast<const u32x4e_word*>(q);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = w[k];
        v[4] = q[3 + odd];
    }
    __device__ __forceinline__ Words(const uint16_t* p, int n) {  // the first n, the others 0
        odd = 0;
#pragma unroll
        for (int k = 0; k < 5; ++k) v[k] = (2 * k < n ? p[2 * k] : 0u) | (2 * k + 1 < n ? (unsigned)p[2 * k + 1] << 16 : 0u);
    }
};
struct Part {
    float x[8];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = 0.f;
    }
    __device__ __forceinline__ void load(const uint16_t* p) { set(Words(p)); }
    __device__ __forceinline__ void set(const Words& w) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned v = __builtin_amdgcn_alignbit(w.v[k + 1], w.v[k], 16 * w.odd);
            x[2 * k]         = h2f((uint16_t)v);
            x[2 * k + 1]     = h2f((uint16_t)(v >> 16));
        }
    }
    __device__ __forceinline__ void store(uint16_t* p, int first, int end) const {  // elements first .. end-1
        if (end - first == 8) {
            u32x4e q;
#pragma unroll
            for (int k = 0; k < 4; ++k) q[k] = (unsigned)f2h(x[2 * k]) | ((unsigned)f2h(x[2 * k + 1]) << 16);
            *reinterpret_cast<u32x4e_any*>(p) = q;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k >= first && k < end) p[k] = f2h(x[k]);
        }
    }
};

// ------------------------------------------------------------------------------------------------ forward
// A thread has one piece of 8 columns of a row, the rows' pieces one behind the other.  The last piece of a row of 8 or more is its last 8
// columns, which may repeat some of the piece before it; only its own (from `skip`) are stored.  TINY: rows of fewer.
struct Piece {
    long long row;
    int       col, skip, end;
    __device__ Piece(int d, int pieces) {
        const long long base = (long long)blockIdx.x * EMB_THREADS;  // (one long division a workgroup)
        const long long r    = base / pieces;
        const unsigned  i    = (unsigned)(base - r * pieces) + threadIdx.x, down = i / (unsigned)pieces;
        const int       first = (int)(i - down * (unsigned)pieces) * 8;
        row                   = r + down;
        col                   = max(min(first, d - 8), 0);
        skip                  = first - col;
        end                   = min(d - col, 8);
    }
};
template <bool TINY>
__device__ __forceinline__ Words load_piece(const uint16_t* p, const Piece& at) {
    return TINY ? Words(p, at.end) : Words(p);
}

template <bool TINY>
__global__ __launch_bounds__(EMB_THREADS) void embedding_fwd_kernel(int rows, int vocab, int d, int pieces, const int* __restrict__ tokens,
                                                                    const uint16_t* __restrict__ w, float scale, uint16_t* __restrict__ y) {
    const Piece at(d, pieces);
    if (at.row >= rows) return;
    const int v = tokens[at.row];
    Part      p;
    p.zero();
    if ((unsigned)v < (unsigned)vocab) p.set(load_piece<TINY>(w + (long long)v * d + at.col, at));
#pragma unroll
    for (int k = 0; k < 8; ++k) p.x[k] = scaled(p.x[k], scale);
    p.store(y + at.row * d + at.col, at.skip, at.end);
}

// ------------------------------------------------------------------------------------------------ sort
// The value of the lane whose number differs in bit X.
template <int X>
__device__ __forceinline__ unsigned other_lane(unsigned v, int lane) {
    const auto dpp = [](unsigned x, auto ctrl) { return (unsigned)__builtin_amdgcn_update_dpp((int)x, (int)x, decltype(ctrl)::value, 0xF, 0xF, true); };
    if constexpr (X == 1) return dpp(v, std::integral_constant<int, 0xB1>{});                                            // quad: 1 0 3 2
    if constexpr (X == 2) return dpp(v, std::integral_constant<int, 0x4E>{});                                            // quad: 2 3 0 1
    if constexpr (X == 4) return dpp(dpp(v, std::integral_constant<int, 0x141>{}), std::integral_constant<int, 0x1B>{});  // 7 - i, quad: 3 2 1 0
    if constexpr (X == 8) return dpp(v, std::integral_constant<int, 0x128>{});                                           // row of 16 rotated by 8
    if constexpr (X == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return lane & 16 ? r[0] : r[1];
    }
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return lane & 32 ? r[0] : r[1];
}
// Bitonic steps of distances J, J/2 .. 1 in registers: a lane has elements 2 lane and 2 lane + 1.
template <int J>
__device__ __forceinline__ void sort_steps(unsigned& x, unsigned& y, bool up, int lane) {
    if constexpr (J == 1) {
        const unsigned lo = min(x, y), hi = max(x, y);
        x = up ? lo : hi;
        y = up ? hi : lo;
    } else {
        const unsigned p = other_lane<J / 2>(x, lane), q = other_lane<J / 2>(y, lane);
        const bool     least = up == ((lane & (J / 2)) == 0);
        x = least ? min(x, p) : max(x, p);
        y = least ? min(y, q) : max(y, q);
        sort_steps<J / 2>(x, y, up, lane);
    }
}

// The first `runs` workgroups sort; the others clear dw (or copy add into it, or only look at an add that is dw), in words and a last
// half word.
__global__ __launch_bounds__(1024) void embedding_sort_kernel(int rows, int vocab, int runs, const int* __restrict__ tokens, u64* __restrict__ keys,
                                                              uint16_t* __restrict__ dw, const uint16_t* __restrict__ add, size_t n, mp_scale_state* st) {
    __shared__ uint2 s[2][SORT_RUN / 2];
    if ((int)blockIdx.x >= runs) {
        const size_t step = (size_t)(gridDim.x - runs) * 1024, first = (size_t)(blockIdx.x - runs) * 1024 + threadIdx.x;
        const size_t head = min(n, (size_t)((16 - (reinterpret_cast<uintptr_t>(dw) & 15)) & 15) / 2), n8 = (n - head) / 8;
        u32x4e*      q    = reinterpret_cast<u32x4e*>(dw + head);
        bool         bad  = false;
        const auto   one  = [&](size_t i) {
            const uint16_t x = add ? add[i] : 0;
            bad |= half_nonfinite(x);
            if (add != dw) dw[i] = x;
        };
        for (size_t i = first; i < n8; i += step) {
            u32x4e x = {0u, 0u, 0u, 0u};
            if (add) x = *reinterpret_cast<const u32x4e_any*>(add + head + 8 * i);
#pragma unroll
            for (int k = 0; k < 4; ++k) bad |= half_nonfinite((uint16_t)x[k]) || half_nonfinite((uint16_t)(x[k] >> 16));
            if (add != dw) q[i] = x;
        }
        if (first < head) one(first);
        if (first < n - head - n8 * 8) one(head + n8 * 8 + first);
        if (add && st && __any(bad) && (threadIdx.x & 63) == 0) atomicOr(&st->found_inf, 1);
        return;
    }
    // A thread has two neighbours.  Distances up to 64 lie in a wave and take no LDS; the ten larger ones go through it, from one half
    // to the other and so with one barrier (2048 keys: 14 us with every step in LDS, 6 this way).
    const int base = blockIdx.x * SORT_RUN, t = threadIdx.x, lane = t & 63;
    unsigned  key[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int i = 2 * t + j, p = base + i;
        key[j] = 0xFFFFFFFFu;
        if (p < rows) {
            const int v = tokens[p];
            key[j]      = ((unsigned)v < (unsigned)vocab ? (unsigned)v : (unsigned)vocab) << SORT_BITS | (unsigned)i;
        }
    }
    sort_steps<1>(key[0], key[1], (lane & 1) == 0, lane);
    sort_steps<2>(key[0], key[1], (lane & 2) == 0, lane);
    sort_steps<4>(key[0], key[1], (lane & 4) == 0, lane);
    sort_steps<8>(key[0], key[1], (lane & 8) == 0, lane);
    sort_steps<16>(key[0], key[1], (lane & 16) == 0, lane);
    sort_steps<32>(key[0], key[1], (lane & 32) == 0, lane);
    sort_steps<64>(key[0], key[1], (t & 64) == 0, lane);
    int b = 0;
    // (what lies behind the last key is the largest: runs of nothing else need no merging)
    for (int k = 256; k <= SORT_RUN && k / 2 < rows - base; k *= 2) {
        const bool up = k == SORT_RUN || (t & (k / 2)) == 0;
        for (int j = k / 2; j >= 128; j /= 2, b ^= 1) {
            s[b][t] = make_uint2(key[0], key[1]);
            __syncthreads();
            const uint2 o     = s[b][t ^ (j / 2)];
            const bool  least = up == ((t & (j / 2)) == 0);
            key[0] = least ? min(key[0], o.x) : max(key[0], o.x);
            key[1] = least ? min(key[1], o.y) : max(key[1], o.y);
        }
        sort_steps<64>(key[0], key[1], up, lane);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int i = base + 2 * t + j;
        if (i < rows) keys[i] = (u64)(key[j] >> SORT_BITS) << 32 | (unsigned)(base + (int)(key[j] & (SORT_RUN - 1)));
    }
}

// Groups of MERGE_RUNS sorted runs of `run` keys (a power of two) into one each: a key's place is the number of smaller ones, run by run
// (all keys differ).  A workgroup places MERGE_KEYS neighbours of one run.  What lies between the first and the last of them in the other
// runs, about as many keys of each, goes through LDS and is searched there; a search of each key in memory takes ten times as long.
constexpr int MERGE_KEYS = 256, MERGE_THREADS = 1024, MERGE_TILE = 8192;
__global__ __launch_bounds__(MERGE_THREADS) void embedding_merge_kernel(int rows, int run, const u64* __restrict__ in, u64* __restrict__ out) {
    __shared__ unsigned tile[MERGE_TILE];                              // tokens
    __shared__ int      low[MERGE_RUNS], before[MERGE_RUNS + 1], smaller[MERGE_KEYS];
    const int       tid = threadIdx.x, mine = tid % MERGE_KEYS, share = tid / MERGE_KEYS;
    const long long p0 = (long long)blockIdx.x * MERGE_KEYS, group = p0 / ((long long)run * MERGE_RUNS) * run * MERGE_RUNS;
    const long long p1   = min((long long)rows, p0 + MERGE_KEYS);
    const int       own  = (int)((p0 - group) / run);
    const u64       key  = in[min(p0 + mine, p1 - 1)], head = in[p0], tail = in[p1 - 1];
    const unsigned  t    = (unsigned)(key >> 32);
    {  // 32 lanes to a run look at 32 places of it at a time
        const int       r = tid / 32, lane = tid % 32, half = (tid & 32);
        const long long start = group + (long long)r * run;
        const int       len   = r == own ? 0 : (int)max(0ll, min((long long)run, rows - start));
        int             lo = 0, hi = 0;
        for (int width = run;;) {
            const int  part = max(width / 32, 1);
            const int  a = lo + (lane + 1) * part - 1, b = hi + (lane + 1) * part - 1;
            const bool in_width = (lane + 1) * part <= width;
            const u64  less_a = __ballot(in_width && a < len && in[start + min(a, max(len - 1, 0))] < head);
            const u64  less_b = __ballot(in_width && b < len && in[start + min(b, max(len - 1, 0))] < tail);
            lo += part * __popc((unsigned)(less_a >> half));
            hi += part * __popc((unsigned)(less_b >> half));
            if (part == 1) break;
            width = part;
        }
        if (lane == 0) {
            low[r]    = lo;
            before[r] = hi - lo;
        }
    }
    __syncthreads();
    if (tid < 64) {  // before[r]: keys of the windows in front of run r's
        const int n = tid < MERGE_RUNS ? before[tid] : 0;
        int       sum = n;
        for (int j = 1; j < MERGE_RUNS; j *= 2) {
            const int x = __shfl_up(sum, j);
            if (tid >= j) sum += x;
        }
        int lows = tid < MERGE_RUNS ? low[tid] : 0;
        for (int j = 1; j < 64; j *= 2) lows += __shfl_xor(lows, j);
        if (tid < MERGE_RUNS) before[tid] = sum - n;
        if (tid == MERGE_RUNS - 1) before[MERGE_RUNS] = sum;
        for (int i = tid; i < MERGE_KEYS; i += 64) smaller[i] = lows;
    }
    __syncthreads();
    const int all = before[MERGE_RUNS];
    int       count = 0;
    for (int base = 0; base < all; base += MERGE_TILE) {
        const int here = min(all - base, MERGE_TILE);
        for (int i = tid; i < here; i += MERGE_THREADS) {
            int r = 0;
#pragma unroll
            for (int step = MERGE_RUNS / 2; step > 0; step /= 2)
                if (before[r + step] <= base + i) r += step;
            tile[i] = (unsigned)(in[group + (long long)r * run + low[r] + (base + i - before[r])] >> 32);
        }
        __syncthreads();
        for (int r = share; r < MERGE_RUNS; r += MERGE_THREADS / MERGE_KEYS) {
            const int      a = max(before[r] - base, 0), len = min(before[r + 1] - base, here) - a;
            const unsigned than = t + (r < own ? 1 : 0);  // equal tokens of an earlier run come first
            int            n = 0;
            if (len > 0)
                for (int step = 1 << (31 - __clz(len)); step > 0; step /= 2) {
                    const int next = n + step;
                    if (next <= len && tile[a + next - 1] < than) n = next;
                }
            count += n;
        }
        __syncthreads();
    }
    if (count) atomicAdd(&smaller[mine], count);
    __syncthreads();
    if (tid < MERGE_KEYS && p0 + tid < p1) out[group + (p0 - group) % run + tid + smaller[tid]] = key;
}

// ------------------------------------------------------------------------------------------------ sums
__device__ __forceinline__ unsigned token_of(u64 k) { return (unsigned)(k >> 32); }

template <bool TINY>
__device__ __forceinline__ bool finish_row(const Part& sum, float scale, uint16_t* dw, const uint16_t* add, const Piece& at) {
    Part r, a;
    if (add) a.set(load_piece<TINY>(add, at));
    bool bad = false;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        r.x[k] = scaled(sum.x[k], scale);
        if (add) r.x[k] = round16(r.x[k]) + a.x[k];
        bad |= k >= at.skip && half_nonfinite(f2h(r.x[k]));
    }
    r.store(dw, at.skip, at.end);
    return bad;
}
__device__ __forceinline__ void store_part(float* o, const Part& s) {
    *reinterpret_cast<f32x4_word*>(o)     = f32x4{s.x[0], s.x[1], s.x[2], s.x[3]};
    *reinterpret_cast<f32x4_word*>(o + 4) = f32x4{s.x[4], s.x[5], s.x[6], s.x[7]};
}

// A chunk is some batches of 8 positions.  All rows of a batch are on their way at once, with the keys of the next.  Then they pass through
// the first registers one by one: a loop whose code were there for each of them would come from memory too, which a small call waits for.
template <bool TINY>
__global__ __launch_bounds__(EMB_THREADS) void embedding_sum_kernel(int rows, int vocab, int d, int pieces, int pitch, int chunk,
                                                                    const u64* __restrict__ keys, const uint16_t* __restrict__ dy, float scale,
                                                                    const uint16_t* add, uint16_t* dw, float* __restrict__ part, mp_scale_state* st) {
    const Piece     at(d, pieces);
    const long long p0 = at.row * chunk, p1 = min((long long)rows, p0 + chunk);
    bool            bad = false;
    if (p0 < rows) {
        const unsigned before = p0 > 0 ? token_of(keys[p0 - 1]) : ~0u, behind = p1 < rows ? token_of(keys[p1]) : ~0u;
        u64            key[EMB_BATCH];
        const auto     ask = [&](long long p) {
#pragma unroll
            for (int j = 0; j < EMB_BATCH; ++j) key[j] = p + j < p1 ? keys[p + j] : ~0ull;
        };
        ask(p0);
        Part sum;
        bool whole = token_of(key[0]) != before;  // whether the open sum began in this chunk
        sum.zero();
#pragma unroll 1
        for (long long p = p0; p < p1; p += EMB_BATCH) {
            unsigned token[EMB_BATCH + 1];
            Words    x[EMB_BATCH];
#pragma unroll
            for (int j = 0; j < EMB_BATCH; ++j) {
                token[j] = token_of(key[j]);
                // (a token outside the table is the last one; what is loaded for it is not used)
                x[j] = load_piece<TINY>(dy + (token[j] < (unsigned)vocab ? (long long)(unsigned)key[j] * d : 0) + at.col, at);
            }
            ask(p + EMB_BATCH);
            token[EMB_BATCH] = p + EMB_BATCH < p1 ? token_of(key[0]) : behind;
#pragma unroll 1
            for (int j = 0; j < EMB_BATCH; ++j) {
                const unsigned t = token[0];
                if (t >= (unsigned)vocab) break;
                Part one;
                one.set(x[0]);
#pragma unroll
                for (int k = 0; k < 8; ++k) sum.x[k] += one.x[k];
                if (token[1] != t) {
                    if (whole) bad |= finish_row<TINY>(sum, scale, dw + (long long)t * d + at.col, add ? add + (long long)t * d + at.col : nullptr, at);
                    else store_part(part + at.row * 2 * pitch + at.col, sum);
                    sum.zero();
                    whole = true;
                } else if (p + j + 1 == p1) {
                    store_part(part + (at.row * 2 + (whole ? 1 : 0)) * pitch + at.col, sum);
                }
#pragma unroll
                for (int i = 0; i < EMB_BATCH; ++i) token[i] = token[i + 1];
#pragma unroll
                for (int i = 0; i + 1 < EMB_BATCH; ++i) x[i] = x[i + 1];
            }
        }
    }
    if (st && __any(bad) && (threadIdx.x & 63) == 0) atomicOr(&st->found_inf, 1);
}

// Sums that cross a border, by the chunk they begin in.  A frequent token's partial sums are asked for several at a time, whether or not
// they are still its own.
constexpr int JOIN_AHEAD = 16;
template <bool TINY>
__global__ __launch_bounds__(EMB_THREADS) void embedding_join_kernel(int rows, int vocab, int d, int pieces, int pitch, int chunk, const u64* __restrict__ keys,
                                                                     float scale, const uint16_t* add, uint16_t* dw, const float* __restrict__ part,
                                                                     mp_scale_state* st) {
    const Piece     at(d, pieces);
    const long long p0 = at.row * chunk, p1 = p0 + chunk;
    bool            bad = false;
    if (p1 < rows) {
        const unsigned t = token_of(keys[p1 - 1]), first = token_of(keys[p0]), behind = token_of(keys[p1]),
                       before = p0 > 0 ? token_of(keys[p0 - 1]) : ~0u;
        if (t < (unsigned)vocab && behind == t && (first != t || before != t)) {
            Part         sum;
            const float* o = part + (at.row * 2 + 1) * pitch + at.col;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum.x[k] = o[k];
            const long long chunks = ((long long)rows + chunk - 1) / chunk;
            bool            more   = true;
            for (long long c = at.row + 1; more; c += JOIN_AHEAD) {
                f32x4    x[JOIN_AHEAD][2];
                unsigned next[JOIN_AHEAD];  // token behind chunk c + i
#pragma unroll
                for (int i = 0; i < JOIN_AHEAD; ++i) {
                    const long long j = min(c + i, chunks - 1);
                    next[i]           = (c + i + 1) * chunk < rows ? token_of(keys[(c + i + 1) * chunk]) : ~0u;
                    x[i][0]           = *reinterpret_cast<const f32x4_word*>(part + j * 2 * pitch + at.col);
                    x[i][1]           = *reinterpret_cast<const f32x4_word*>(part + j * 2 * pitch + at.col + 4);
                }
#pragma unroll
                for (int i = 0; i < JOIN_AHEAD; ++i) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum.x[k] = more ? sum.x[k] + x[i][k / 4][k % 4] : sum.x[k];
                    more = more && next[i] == t;
                }
            }
            bad = finish_row<TINY>(sum, scale, dw + (long long)t * d + at.col, add ? add + (long long)t * d + at.col : nullptr, at);
        }
    }
    if (st && __any(bad) && (threadIdx.x & 63) == 0) atomicOr(&st->found_inf, 1);
}

static size_t keys_bytes(int rows) { return ((size_t)rows * sizeof(u64) + 255) / 256 * 256; }
static int pieces_of(int d) { return (int)(((long long)d + 7) / 8); }
static int pitch_of(int d) { return d < 8 ? 8 : d; }
// Sorted positions of a chunk: more of them, up to 64, as long as there are 2^17 threads.  Long chunks leave fewer partial sums; with few
// threads they leave memory waiting.  Gradients, words by Zipf's law: 65536 rows of 1024 of 50021 words 138 us in chunks of 8, 101 so
// (of 32); 262144 rows 493 us, 278 so (of 64); 16384 rows of 32768 words 52 us in chunks of 8, 47 so (of 16), 53 with chunks for half the threads.
static int chunk_of(int rows, int d) {
    int chunk = EMB_BATCH;
    while (chunk < 64 && (long long)rows / (2 * chunk) * pieces_of(d) >= (1 << 17)) chunk *= 2;
    return chunk;
}
static long long chunks_of(int rows, int d) { return ((long long)rows + chunk_of(rows, d) - 1) / chunk_of(rows, d); }

static long long sum_wgs(int rows, int d) { return (chunks_of(rows, d) * pieces_of(d) + EMB_THREADS - 1) / EMB_THREADS; }

static int launch_sums(int rows, int vocab, int d, const u64* keys, const mp_half* dy, float scale, const mp_half* add, mp_half* dw, float* part,
                       mp_scale_state* st, hipStream_t hs) {
    const int       pieces = pieces_of(d);
    const long long wgs    = sum_wgs(rows, d);
    const dim3 grid((unsigned)wgs), block(EMB_THREADS);
    const auto sums = d < 8 ? embedding_sum_kernel<true> : embedding_sum_kernel<false>;
    const auto join = d < 8 ? embedding_join_kernel<true> : embedding_join_kernel<false>;
    hipLaunchKernelGGL(sums, grid, block, 0, hs, rows, vocab, d, pieces, pitch_of(d), chunk_of(rows, d), keys, dy, scale, add, dw, part, st);
    MP_LAUNCH_CHECK("mp_embedding_bwd(sum)");
    hipLaunchKernelGGL(join, grid, block, 0, hs, rows, vocab, d, pieces, pitch_of(d), chunk_of(rows, d), keys, scale, add, dw, part, st);
    MP_LAUNCH_CHECK("mp_embedding_bwd(join)");
    return MP_OK;
}

}  // namespace mp

using namespace mp;

static int embedding_check(const char* who, int rows, int vocab, int d) {
    MP_REQUIRE(rows >= 0 && vocab > 0 && d > 0, "%s: bad shape %d x %d, vocabulary %d", who, rows, d, vocab);
    return MP_OK;
}

extern "C" int mp_embedding_fwd(int rows, int vocab, int d, const int32_t* tokens, const mp_half* w, float scale, mp_half* y, mp_stream stream) {
    int rc = embedding_check("mp_embedding_fwd", rows, vocab, d);
    if (rc) return rc;
    if (rows == 0) return MP_OK;
    MP_REQUIRE(tokens && w && y, "mp_embedding_fwd: NULL argument");
    MP_REQUIRE(((reinterpret_cast<uintptr_t>(w) | reinterpret_cast<uintptr_t>(y)) & 1) == 0, "mp_embedding_fwd: w or y is not element-aligned");
    const int       pieces = pieces_of(d);
    const long long wgs    = ((long long)rows * pieces + EMB_THREADS - 1) / EMB_THREADS;
    MP_REQUIRE(grid_fits(wgs, EMB_THREADS), "mp_embedding_fwd: too many rows and columns");
    hipLaunchKernelGGL(d < 8 ? embedding_fwd_kernel<true> : embedding_fwd_kernel<false>, dim3((unsigned)wgs), dim3(EMB_THREADS), 0, as_stream(stream), rows,
                       vocab, d, pieces, tokens, w, scale, y);
    MP_LAUNCH_CHECK("mp_embedding_fwd");
    return MP_OK;
}

extern "C" size_t mp_embedding_bwd_workspace_bytes(int rows, int vocab, int d) {
    if (rows < 0 || vocab <= 0 || d <= 0) return 0;
    return 2 * keys_bytes(rows) + (size_t)chunks_of(rows, d) * 2 * pitch_of(d) * sizeof(float) + 256;
}

extern "C" int mp_embedding_bwd(int rows, int vocab, int d, const int32_t* tokens, const mp_half* dy, float scale, const mp_half* add, mp_half* dw,
                                mp_scale_state* st, void* ws, size_t ws_bytes, mp_stream stream) {
    int rc = embedding_check("mp_embedding_bwd", rows, vocab, d);
    if (rc) return rc;
    MP_REQUIRE(dw && (rows == 0 || (tokens && dy)), "mp_embedding_bwd: NULL argument");
    MP_REQUIRE(((reinterpret_cast<uintptr_t>(dy) | reinterpret_cast<uintptr_t>(add) | reinterpret_cast<uintptr_t>(dw)) & 1) == 0,
               "mp_embedding_bwd: dy, add or dw is not element-aligned");
    if (rows > (1 << 24) || vocab >= (1 << (32 - SORT_BITS))) {
        set_error("mp_embedding_bwd: more than 2^24 rows or a vocabulary of 2^21 or more (%d, %d)", rows, vocab);
        return MP_E_UNSUPPORTED;
    }
    MP_REQUIRE(grid_fits(sum_wgs(rows, d), EMB_THREADS), "mp_embedding_bwd: too many rows and columns");
    if (!ws || !aligned16(ws) || ws_bytes < mp_embedding_bwd_workspace_bytes(rows, vocab, d)) {
        set_error("mp_embedding_bwd: workspace missing, misaligned or smaller than mp_embedding_bwd_workspace_bytes");
        return MP_E_WORKSPACE;
    }
    hipStream_t  hs   = as_stream(stream);
    u64*         keys = static_cast<u64*>(ws);
    u64*         more = reinterpret_cast<u64*>(static_cast<char*>(ws) + keys_bytes(rows));
    float*       part = reinterpret_cast<float*>(static_cast<char*>(ws) + 2 * keys_bytes(rows));
    const int    runs = (rows + SORT_RUN - 1) / SORT_RUN;
    const size_t n    = (size_t)vocab * d;
    const bool   fill = add != dw || st;  // (in place: rows without a token keep what they have, and it is looked at)
    const size_t want = (n + 8191) / 8192;
    const int    wgs  = runs + (fill ? (int)(want < FILL_WGS ? want : FILL_WGS) : 0);
    if (wgs == 0) return MP_OK;
    hipLaunchKernelGGL(embedding_sort_kernel, dim3(wgs), dim3(1024), 0, hs, rows, vocab, runs, tokens, keys, dw, add, n, st);
    MP_LAUNCH_CHECK("mp_embedding_bwd(sort)");
    if (rows == 0) return MP_OK;
    for (long long run = SORT_RUN; run < rows; run *= MERGE_RUNS) {
        hipLaunchKernelGGL(embedding_merge_kernel, dim3((rows + MERGE_KEYS - 1) / MERGE_KEYS), dim3(MERGE_THREADS), 0, hs, rows, (int)run, keys,
                           more);
        MP_LAUNCH_CHECK("mp_embedding_bwd(merge)");
        u64* t = keys;
        keys   = more;
        more   = t;
    }
    return launch_sums(rows, vocab, d, keys, dy, scale, add, dw, part, st, hs);
}
