// Embedding lookup with scaling, and the table's gradient by sorted tokens.
//
// Both are bound by HBM: forward reads a table row per token (or finds it in the caches) and writes a row, backward reads a gradient row
// per token and writes the whole table's gradient.  Gradient rows of one token are summed in fp32 in the order of their positions:
//   1. sort    runs of SORT_RUN tokens in LDS (value, then position: one 32-bit key); the other workgroups of the launch clear dw
//   2. merge   up to MERGE_RUNS runs into one, each key's place by binary searches (not for a single run)
//   3. sum     EMB_CHUNK sorted positions a group of lanes, however they are spread over tokens: a token's sum that lies inside a
//              chunk is stored, one that crosses a border is left as partial sums
//   4. join    partial sums, in the order of the chunks
// so that neither a token that is every second one nor one that comes once costs more than its rows, without an atomic addition.
#include "common.hpp"

namespace mp {

typedef unsigned u32x4e __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int EMB_THREADS = 256;
constexpr int SORT_RUN    = 2048;   // 11 bits of position beside 21 bits of token
constexpr int SORT_BITS   = 11;
constexpr int MERGE_RUNS  = 32;
constexpr int EMB_CHUNK   = 32;
constexpr int FILL_WGS    = 2048;

// The product rounded to fp32 before it is rounded to fp16: the compiler else makes one instruction of the two in some places,
// which rounds once (an element in 10^4 differs, and a call with `add` from one without).
__device__ __forceinline__ float scaled(float x, float scale) {
    x *= scale;
    asm("" : "+v"(x));
    return x;
}

// VEC elements of a row (8: one 16-byte access, 1: any alignment)
template <int VEC>
struct Part {
    float x[VEC];
    __device__ __forceinline__ void load(const uint16_t* p) {
        if (VEC == 8) {
            const u32x4e q = *reinterpret_cast<const u32x4e*>(p);
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[i] = h2f((uint16_t)(q[i / 2] >> (16 * (i & 1))));
        } else {
            x[0] = h2f(*p);
        }
    }
    __device__ __forceinline__ void store(uint16_t* p) const {
        if (VEC == 8) {
            u32x4e q;
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = (unsigned)f2h(x[2 * i]) | ((unsigned)f2h(x[2 * i + 1]) << 16);
            *reinterpret_cast<u32x4e*>(p) = q;
        } else {
            *p = f2h(x[0]);
        }
    }
};

// ------------------------------------------------------------------------------------------------ forward
template <int VEC>
__global__ __launch_bounds__(EMB_THREADS) void embedding_fwd_kernel(long long pieces, int per_row, int vocab, int d, const int* __restrict__ tokens,
                                                                    const uint16_t* __restrict__ w, float scale, uint16_t* __restrict__ y) {
    for (long long i = (long long)blockIdx.x * EMB_THREADS + threadIdx.x; i < pieces; i += (long long)gridDim.x * EMB_THREADS) {
        const int t = (int)(i / per_row), c = (int)(i - (long long)t * per_row) * VEC;
        const int v = tokens[t];
        Part<VEC> p;
        if ((unsigned)v < (unsigned)vocab) {
            p.load(w + (long long)v * d + c);
#pragma unroll
            for (int k = 0; k < VEC; ++k) p.x[k] = scaled(p.x[k], scale);
        } else {
#pragma unroll
            for (int k = 0; k < VEC; ++k) p.x[k] = 0.f;
        }
        p.store(y + (long long)t * d + c);
    }
}

// ------------------------------------------------------------------------------------------------ sort
// The first `runs` workgroups sort; the others clear dw (or copy add into it), in words and a last half word.
__global__ __launch_bounds__(1024) void embedding_sort_kernel(int rows, int vocab, int runs, const int* __restrict__ tokens, u64* __restrict__ keys,
                                                              uint16_t* __restrict__ dw, const uint16_t* __restrict__ add, size_t n, mp_scale_state* st) {
    __shared__ unsigned s[SORT_RUN];
    if ((int)blockIdx.x >= runs) {
        const size_t step = (size_t)(gridDim.x - runs) * 1024, first = (size_t)(blockIdx.x - runs) * 1024 + threadIdx.x;
        if (!add) {
            const size_t head = min(n, (size_t)((16 - (reinterpret_cast<uintptr_t>(dw) & 15)) & 15) / 2), n8 = (n - head) / 8;
            u32x4e*      q    = reinterpret_cast<u32x4e*>(dw + head);
            for (size_t i = first; i < n8; i += step) q[i] = u32x4e{0u, 0u, 0u, 0u};
            if (first < head) dw[first] = 0;
            if (first < n - head - n8 * 8) dw[head + n8 * 8 + first] = 0;
        } else {
            bool bad = false;
            for (size_t i = first; i < n; i += step) {
                const uint16_t x = add[i];
                bad |= half_nonfinite(x);
                dw[i] = x;
            }
            if (st && __any(bad) && (threadIdx.x & 63) == 0) atomicOr(&st->found_inf, 1);
        }
        return;
    }
    const int base = blockIdx.x * SORT_RUN;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int i = threadIdx.x + 1024 * j, p = base + i;
        unsigned  key = 0xFFFFFFFFu;
        if (p < rows) {
            const int t = tokens[p];
            key         = ((unsigned)t < (unsigned)vocab ? (unsigned)t : (unsigned)vocab) << SORT_BITS | (unsigned)i;
        }
        s[i] = key;
    }
    __syncthreads();
    for (int k = 2; k <= SORT_RUN; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            const int      a = 2 * threadIdx.x - (threadIdx.x & (j - 1)), b = a + j;
            const unsigned x = s[a], y = s[b];
            if ((x > y) == ((a & k) == 0)) {
                s[a] = y;
                s[b] = x;
            }
            __syncthreads();
        }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int i = threadIdx.x + 1024 * j;
        if (base + i < rows) keys[base + i] = (u64)(s[i] >> SORT_BITS) << 32 | (unsigned)(base + (s[i] & (SORT_RUN - 1)));
    }
}

// Groups of MERGE_RUNS sorted runs of `run` keys into one each.  All keys differ.
__global__ __launch_bounds__(EMB_THREADS) void embedding_merge_kernel(int rows, long long run, const u64* __restrict__ in, u64* __restrict__ out) {
    const long long p = (long long)blockIdx.x * EMB_THREADS + threadIdx.x;
    if (p >= rows) return;
    const u64       key   = in[p];
    const long long group = p / (run * MERGE_RUNS) * (run * MERGE_RUNS), own = p / run * run;
    long long       at    = group + (p - own);
    const long long end   = min((long long)rows, group + run * MERGE_RUNS);
    for (long long r = group; r < end; r += run) {
        if (r == own) continue;
        int a = 0, b = (int)min(run, end - r);  // keys below `key` in that run
        while (a < b) {
            const int c = (a + b) >> 1;
            if (in[r + c] < key) a = c + 1; else b = c;
        }
        at += a;
    }
    out[at] = key;
}

// ------------------------------------------------------------------------------------------------ sums
// A group of `lanes` lanes (a power of two) has one chunk of sorted positions and `lanes` x VEC columns.
template <int VEC>
struct SumAt {
    long long chunk, p0, p1;
    int       col;
    bool      in;
    __device__ SumAt(int rows, int d, int lanes, int blocks) {
        const long long id = ((long long)blockIdx.x * EMB_THREADS + threadIdx.x) / lanes;
        chunk              = id / blocks;
        col                = ((int)(id - chunk * blocks) * lanes + (int)(threadIdx.x & (lanes - 1))) * VEC;
        p0                 = chunk * EMB_CHUNK;
        p1                 = min((long long)rows, p0 + EMB_CHUNK);
        in                 = p0 < rows && col < d;
    }
};
__device__ __forceinline__ unsigned token_of(u64 k) { return (unsigned)(k >> 32); }

template <int VEC>
__device__ __forceinline__ bool finish_row(const float (&sum)[VEC], float scale, uint16_t* dw, const uint16_t* add) {
    Part<VEC> r, a;
    if (add) a.load(add);
    bool bad = false;
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        r.x[k] = scaled(sum[k], scale);
        if (add) r.x[k] = round16(r.x[k]) + a.x[k];
        bad |= half_nonfinite(f2h(r.x[k]));
    }
    r.store(dw);
    return bad;
}

template <int VEC>
__global__ __launch_bounds__(EMB_THREADS) void embedding_sum_kernel(int rows, int vocab, int d, int lanes, int blocks, const u64* __restrict__ keys,
                                                                    const uint16_t* __restrict__ dy, float scale, const uint16_t* add,
                                                                    uint16_t* dw, float* __restrict__ part, mp_scale_state* st) {
    const SumAt<VEC> at(rows, d, lanes, blocks);
    bool             bad = false;
    if (at.in) {
        unsigned prev  = at.p0 > 0 ? token_of(keys[at.p0 - 1]) : 0xFFFFFFFFu;  // token of the open sum
        bool     whole = false;                                               // whether that began in this chunk
        float    sum[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) sum[k] = 0.f;
        bool       some  = false;
        const auto close = [&](bool tail) {
            if (!some || prev >= (unsigned)vocab) return;
            if (whole && !tail) {
                bad |= finish_row<VEC>(sum, scale, dw + (long long)prev * d + at.col, add ? add + (long long)prev * d + at.col : nullptr);
            } else {
                float* o = part + (at.chunk * 2 + (whole ? 1 : 0)) * d + at.col;
#pragma unroll
                for (int k = 0; k < VEC; ++k) o[k] = sum[k];
            }
        };
        constexpr int AHEAD = 8;
        for (long long p = at.p0; p < at.p1; p += AHEAD) {
            u64       key[AHEAD];
            Part<VEC> x[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) key[j] = p + j < at.p1 ? keys[p + j] : ~0ull;
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (token_of(key[j]) < (unsigned)vocab) x[j].load(dy + (long long)(unsigned)key[j] * d + at.col);
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                if (p + j >= at.p1) break;
                const unsigned t = token_of(key[j]);
                if (t != prev) {
                    close(false);
                    prev  = t;
                    whole = true;
#pragma unroll
                    for (int k = 0; k < VEC; ++k) sum[k] = 0.f;
                }
                some = true;
                if (t < (unsigned)vocab) {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) sum[k] += x[j].x[k];
                }
            }
        }
        close(at.p1 < rows && token_of(keys[at.p1]) == prev);
    }
    if (st && __any(bad) && (threadIdx.x & 63) == 0) atomicOr(&st->found_inf, 1);
}

// Sums that cross a border, by the chunk they begin in.
template <int VEC>
__global__ __launch_bounds__(EMB_THREADS) void embedding_join_kernel(int rows, int vocab, int d, int lanes, int blocks, const u64* __restrict__ keys,
                                                                     float scale, const uint16_t* add, uint16_t* dw, const float* __restrict__ part,
                                                                     mp_scale_state* st) {
    const SumAt<VEC> at(rows, d, lanes, blocks);
    bool             bad = false;
    if (at.in && at.p1 < rows) {
        const unsigned t      = token_of(keys[at.p1 - 1]);
        const bool     begins = token_of(keys[at.p0]) != t || at.p0 == 0 || token_of(keys[at.p0 - 1]) != t;
        if (t < (unsigned)vocab && begins && token_of(keys[at.p1]) == t) {
            float        sum[VEC];
            const float* o = part + (at.chunk * 2 + 1) * d + at.col;
#pragma unroll
            for (int k = 0; k < VEC; ++k) sum[k] = o[k];
            for (long long c = at.chunk + 1;; ++c) {
                o = part + c * 2 * d + at.col;
#pragma unroll
                for (int k = 0; k < VEC; ++k) sum[k] += o[k];
                const long long next = (c + 1) * EMB_CHUNK;
                if (next >= rows || token_of(keys[next]) != t) break;
            }
            bad = finish_row<VEC>(sum, scale, dw + (long long)t * d + at.col, add ? add + (long long)t * d + at.col : nullptr);
        }
    }
    if (st && __any(bad) && (threadIdx.x & 63) == 0) atomicOr(&st->found_inf, 1);
}

static size_t keys_bytes(int rows) { return ((size_t)rows * sizeof(u64) + 255) / 256 * 256; }
static long long chunks_of(int rows) { return ((long long)rows + EMB_CHUNK - 1) / EMB_CHUNK; }

template <int VEC>
static int launch_sums(int rows, int vocab, int d, const u64* keys, const mp_half* dy, float scale, const mp_half* add, mp_half* dw, float* part,
                       mp_scale_state* st, hipStream_t hs) {
    int lanes = 1;
    while (lanes < 64 && lanes * VEC < d) lanes *= 2;
    const int       blocks = (d + lanes * VEC - 1) / (lanes * VEC);
    const long long wgs    = (chunks_of(rows) * blocks * lanes + EMB_THREADS - 1) / EMB_THREADS;
    MP_REQUIRE(wgs < (1ll << 31), "mp_embedding_bwd: too many rows and columns");
    hipLaunchKernelGGL(embedding_sum_kernel<VEC>, dim3((unsigned)wgs), dim3(EMB_THREADS), 0, hs, rows, vocab, d, lanes, blocks, keys, dy, scale, add, dw,
                       part, st);
    MP_LAUNCH_CHECK("mp_embedding_bwd(sum)");
    hipLaunchKernelGGL(embedding_join_kernel<VEC>, dim3((unsigned)wgs), dim3(EMB_THREADS), 0, hs, rows, vocab, d, lanes, blocks, keys, scale, add, dw, part,
                       st);
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
    const bool      vec    = (d & 7) == 0 && aligned16(w) && aligned16(y);
    const int       per    = vec ? d / 8 : d;
    const long long pieces = (long long)rows * per, wgs = (pieces + EMB_THREADS - 1) / EMB_THREADS;
    const dim3      grid((unsigned)(wgs < (1 << 20) ? wgs : (1 << 20)));
    if (vec)
        hipLaunchKernelGGL(embedding_fwd_kernel<8>, grid, dim3(EMB_THREADS), 0, as_stream(stream), pieces, per, vocab, d, tokens, w, scale, y);
    else
        hipLaunchKernelGGL(embedding_fwd_kernel<1>, grid, dim3(EMB_THREADS), 0, as_stream(stream), pieces, per, vocab, d, tokens, w, scale, y);
    MP_LAUNCH_CHECK("mp_embedding_fwd");
    return MP_OK;
}

extern "C" size_t mp_embedding_bwd_workspace_bytes(int rows, int vocab, int d) {
    if (rows < 0 || vocab <= 0 || d <= 0) return 0;
    return 2 * keys_bytes(rows) + (size_t)chunks_of(rows) * 2 * d * sizeof(float) + 256;
}

extern "C" int mp_embedding_bwd(int rows, int vocab, int d, const int32_t* tokens, const mp_half* dy, float scale, const mp_half* add, mp_half* dw,
                                mp_scale_state* st, void* ws, size_t ws_bytes, mp_stream stream) {
    int rc = embedding_check("mp_embedding_bwd", rows, vocab, d);
    if (rc) return rc;
    MP_REQUIRE(dw && (rows == 0 || (tokens && dy)), "mp_embedding_bwd: NULL argument");
    if (rows > (1 << 24) || vocab >= (1 << (32 - SORT_BITS))) {
        set_error("mp_embedding_bwd: more than 2^24 rows or a vocabulary of 2^21 or more (%d, %d)", rows, vocab);
        return MP_E_UNSUPPORTED;
    }
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
    const bool   fill = add != dw;
    const size_t want = (n + 8191) / 8192;
    const int    wgs  = runs + (fill ? (int)(want < FILL_WGS ? want : FILL_WGS) : 0);
    if (wgs == 0) return MP_OK;
    hipLaunchKernelGGL(embedding_sort_kernel, dim3(wgs), dim3(1024), 0, hs, rows, vocab, runs, tokens, keys, dw, add, n, st);
    MP_LAUNCH_CHECK("mp_embedding_bwd(sort)");
    if (rows == 0) return MP_OK;
    for (long long run = SORT_RUN; run < rows; run *= MERGE_RUNS) {
        hipLaunchKernelGGL(embedding_merge_kernel, dim3((rows + EMB_THREADS - 1) / EMB_THREADS), dim3(EMB_THREADS), 0, hs, rows, run, keys, more);
        MP_LAUNCH_CHECK("mp_embedding_bwd(merge)");
        u64* t = keys;
        keys   = more;
        more   = t;
    }
    const bool vec = (d & 7) == 0 && aligned16(dy) && aligned16(dw) && (!add || aligned16(add));
    return vec ? launch_sums<8>(rows, vocab, d, keys, dy, scale, add, dw, part, st, hs)
               : launch_sums<1>(rows, vocab, d, keys, dy, scale, add, dw, part, st, hs);
}
