// Distillation from a teacher's top logits: fp32 loss and loss-scaled fp16 seed gradient in one pass over the student's logits.
//
// With z = x / temperature, p = softmax z, A the classes that the teacher's list names, q_u its probability of class u (entries of one
// class added up), Q = sum q, and r what is left for all other classes together (0 where lists are renormalised):
//     L = sum_A q_u (ln q_u - ln p_u) + r (ln r - ln p_rest),       dL/dz_j = (Q + r) p_j - (j in A ? q_j : r p_j / p_rest)
//     dx_j = S / rows (weight / temperature dL/dz_j + hard (softmax(x)_j - 1[j = target]))
//
// Bound by HBM: 2 bytes a class read, 2 written.  A workgroup holds a row in registers from its sums to its gradient, and takes the
// next row's pieces into the same registers one by one as the gradient leaves them, so loads and stores run beside each other.
// Outside A the gradient is one factor a row times the exponential.  The classes of A, at most 128, are one wave's work: their
// gradients wait in LDS, and a map from pieces to entries tells each piece which of its elements to replace.  For r the sum over
// "all others" is formed without A, not as a difference of sums, which would lose it where the student is sure of A.
//
// Rows longer than 131064 classes, or too few for the chip, are cut into chunks: one launch for the sums, one for the gradient.
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

struct EntryLds {
    int            id[MP_TOP_MAX + 1], next[MP_TOP_MAX + 1];
    float          q[MP_TOP_MAX];
    unsigned short value[MP_TOP_MAX + 1];
};
struct RowFactors {
    float a, ref, b, ref2;  // gradient outside A: a 2^(c2 x - ref) + b 2^(log2(e) x - ref2)
    int   none;             // a zero row, whatever it holds
};

// One wave's view of a row's entries: lane l has entries l and l + 64.  SHIFT: 2^SHIFT elements share a word of the map.
template <int SHIFT>
struct Entries {
    int   id[2], target;
    float t[2], x[2], xt;
    bool  there[2], listed, twice;  // listed: the target is in A.  twice: some class is named more than once

    __device__ __forceinline__ void load(const DistillArgs& a, long long row) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const bool in = lane + 64 * s < a.top;
            id[s] = in ? a.ids[row * a.top + lane + 64 * s] : -1;
            t[s]  = in ? a.teacher[row * a.top + lane + 64 * s] : 0.f;
        }
        target = a.targets ? a.targets[row] : -1;
    }
    // place of a class in the stretch, or -1
    __device__ __forceinline__ static int place(const DistillArgs& a, const Stretch& z, int first, int c) {
        return c >= first && c < a.vocab && c - first < z.len ? c - first : -1;
    }
    // into the map of the row's pieces, those that lie in the stretch
    __device__ __forceinline__ void insert(const DistillArgs& a, const Stretch& z, int first, unsigned* map, EntryLds& l) {
        const int lane = threadIdx.x & 63;
        bool      eq   = false;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            there[s] = id[s] >= 0 && id[s] < a.vocab;
            eq |= there[s] && id[s] == target;
        }
        listed     = __any(eq);
        bool again = false;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int e = lane + 64 * s, at = place(a, z, first, id[s]);
            if (e < a.top) l.id[e] = id[s];
            if (at >= 0) l.next[e] = (int)atomicExch(&map[(at + z.head) >> SHIFT], (unsigned)e + 1);
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int s = 0; s < 2; ++s)
            if (place(a, z, first, id[s]) >= 0)
                for (int o = l.next[lane + 64 * s]; o; o = l.next[o - 1]) again |= l.id[o - 1] == id[s];
        twice        = a.chunks > 1 || __any(again);  // (the rest of a list may lie in another chunk)
        const int at = place(a, z, first, target);
        if (lane == 0 && !listed && at >= 0) {
            l.id[DI_TARGET]   = target;
            l.next[DI_TARGET] = (int)atomicExch(&map[(at + z.head) >> SHIFT], (unsigned)DI_TARGET + 1);
        }
    }
    __device__ __forceinline__ void remove(const DistillArgs& a, const Stretch& z, int first, unsigned* map) const {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int at = place(a, z, first, id[s]);
            if (at >= 0) map[(at + z.head) >> SHIFT] = 0;
        }
        const int at = place(a, z, first, target);
        if ((threadIdx.x & 63) == 0 && at >= 0) map[(at + z.head) >> SHIFT] = 0;
    }
    // the student's logits of the entries
    __device__ __forceinline__ void gather(const DistillArgs& a, long long row) {
        const uint16_t* z = a.logits + row * a.ld;
#pragma unroll
        for (int s = 0; s < 2; ++s) x[s] = there[s] ? h2f(z[id[s]]) : -INFINITY;
        xt = target >= 0 && target < a.vocab ? h2f(z[target]) : 0.f;
    }
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int far = 32; far; far >>= 1) v += __shfl_xor(v, far, 64);
    return v;
}

// One wave: the row's loss, its factors, and the entries' gradients.  one, two: sums at the temperature and (TWO) at 1, without A if
// TAIL.
template <bool TAIL, bool TWO, int SHIFT>
__device__ __forceinline__ void finish_row(const DistillArgs& a, const Entries<SHIFT>& n, const Sums<false> one, const Sums<false> two, EntryLds& l, RowFactors& out,
                                           float* row_loss) {
    const int  lane   = threadIdx.x & 63;
    const bool some   = __any(n.there[0] || n.there[1]);
    const bool real   = n.target >= 0 && n.target < a.vocab && a.hard != 0.f;
    const float scale = (float)((double)a.st->scale / (double)a.rows), wc = some ? a.weight * a.inv_temperature * scale : 0.f, hs = real ? a.hard * scale : 0.f;
    float      q[2], r = 0.f, sum_q;
    if (TAIL) {
        double w[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            w[s] = n.there[s] ? exp((double)n.t[s]) : 0.0;  // (64 bits: 1 minus their sum is often next to nothing)
            q[s] = (float)w[s];
        }
        const double sum = wave_sum64(w[0] + w[1]);
        sum_q            = (float)sum;
        if (some && one.s > 0.f && sum < 1.0) r = (float)(1.0 - sum);
    } else {
        float m = wave_max(fmaxf(n.there[0] ? n.t[0] : -INFINITY, n.there[1] ? n.t[1] : -INFINITY));
        m       = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int s = 0; s < 2; ++s) q[s] = n.there[s] ? expf(n.t[s] - m) : 0.f;
        const float sum = wave_sum(q[0] + q[1]), inv = sum == 0.f ? 0.f : 1.f / sum;
        q[0] *= inv;
        q[1] *= inv;
        sum_q = sum * inv;
    }
    bool first[2] = {n.there[0], n.there[1]};
    if (n.twice) {  // a class counts once, with the sum of its entries in their order
#pragma unroll
        for (int s = 0; s < 2; ++s)
            if (lane + 64 * s < a.top) l.q[lane + 64 * s] = q[s];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            float sum  = 0.f;
            bool  seen = false;
            for (int j = 0; j < a.top; ++j)
                if (l.id[j] == n.id[s]) {
                    sum += l.q[j];
                    seen |= j < lane + 64 * s;
                }
            if (n.there[s]) {
                q[s]     = sum;
                first[s] = !seen;
            }
        }
    }
    Sums<false> all = one, at1 = two;
    if (TAIL) {
        const float top         = wave_max(fmaxf(n.x[0], n.x[1]));
        const auto  with_listed = [&](Sums<false>& t, float c2) {
            t.move(fmaxf(t.ref, top * c2));
            t.s += wave_sum((first[0] ? __builtin_amdgcn_exp2f(fmaf(n.x[0], c2, -t.ref)) : 0.f) +
                            (first[1] ? __builtin_amdgcn_exp2f(fmaf(n.x[1], c2, -t.ref)) : 0.f));
        };
        with_listed(all, a.c2);
        if (TWO) with_listed(at1, LOG2E);
    }
    const float log_s = log2f(all.s), inv_s = 1.f / all.s, u = sum_q + r, rest = TAIL ? __builtin_amdgcn_exp2f(one.ref - all.ref) : 1.f;
    const float inv_1 = TWO ? 1.f / at1.s : inv_s;
    RowFactors  f;
    f.a    = wc * (u * (rest * inv_s) - (TAIL && r > 0.f ? r / one.s : 0.f)) + (TWO ? 0.f : hs * (rest * inv_s));
    f.ref  = TAIL ? one.ref : all.ref;
    f.b    = TWO ? hs * inv_1 : 0.f;
    f.ref2 = at1.ref;
    f.none = !some && !real;
    float kl = 0.f;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const float y = fmaf(n.x[s], a.c2, -all.ref), p = __builtin_amdgcn_exp2f(y) * inv_s, p1 = TWO ? __builtin_amdgcn_exp2f(fmaf(n.x[s], LOG2E, -at1.ref)) * inv_1 : p;
        if (n.there[s]) l.value[lane + 64 * s] = f2h(wc * (p * u - q[s]) + (real ? hs * (p1 - (n.id[s] == n.target ? 1.f : 0.f)) : 0.f));
        if (first[s] && q[s] != 0.f) kl += q[s] * (logf(q[s]) - LN2 * (y - log_s));
    }
    kl = wave_sum(kl);
    if (TAIL && r > 0.f) kl += r * (logf(r) - LN2 * ((one.ref - all.ref) + (log2f(one.s) - log_s)));
    if (lane == 0) {
        float loss = some ? a.weight * kl : 0.f;
        if (real) {
            loss -= a.hard * (LN2 * (TWO ? fmaf(n.xt, LOG2E, -at1.ref) - log2f(at1.s) : fmaf(n.xt, a.c2, -all.ref) - log_s));
            if (!n.listed)
                l.value[DI_TARGET] =
                    f2h(f.a * __builtin_amdgcn_exp2f(fmaf(n.xt, a.c2, -f.ref)) + (TWO ? f.b * __builtin_amdgcn_exp2f(fmaf(n.xt, LOG2E, -f.ref2)) : 0.f) - hs);
        }
        if (row_loss) *row_loss = loss;
        out = f;
    }
}

// half k of a piece
__device__ __forceinline__ void set_half(u32x4& q, int k, unsigned h) {
#pragma unroll
    for (int w = 0; w < 4; ++w)
        if (w == k >> 1) q[w] = (k & 1) ? (q[w] & 0xFFFFu) | (h << 16) : (q[w] & 0xFFFF0000u) | h;
}

template <int SHIFT>
__host__ __device__ constexpr int map_words(int len) { return (len + 7 + (1 << SHIFT) - 1) >> SHIFT; }

// FUSED: whole rows, in turn.  SUMS, GRADIENT: one chunk of one row, sums out or in through a.sums.
enum { DI_FUSED = 0, DI_SUMS = 1, DI_GRADIENT = 2 };

template <int THREADS, int VECS, bool TAIL, bool TWO, int MODE, int SHIFT>
__global__ __launch_bounds__(THREADS) void distill_kernel(const DistillArgs a) {
    extern __shared__ unsigned map[];  // entry + 1 of each piece, others behind it in EntryLds::next; 0: none
    __shared__ EntryLds        l;
    __shared__ RowFactors      factors;
    __shared__ float           red[THREADS / 64][4];
    constexpr int              NW = THREADS / 64, G = VECS < 4 ? VECS : 4;
    const int                  tid = threadIdx.x, wave = tid >> 6;
    long long                  row   = MODE == DI_FUSED ? blockIdx.x : blockIdx.x / a.chunks;
    const int                  chunk = MODE == DI_FUSED ? 0 : blockIdx.x - (int)row * a.chunks, first = chunk * a.chunk, len = min(a.chunk, a.vocab - first);
    Stretch                    z(a.logits + row * a.ld + first, len);
    Entries<SHIFT>             n, ahead;
    u32x4                      raw[VECS];
#pragma unroll
    for (int i = 0; i < VECS; ++i) raw[i] = z.load(i * THREADS + tid);
    if (wave == 0) n.load(a, row);
    for (int v = tid; v < map_words<SHIFT>(a.chunk); v += THREADS) map[v] = 0;
    const auto replace = [&](u32x4& q, int v, int e, unsigned h) {
        const int at = l.id[e] - first + z.head;
        if (SHIFT == 3 || (at >> 3) == v) set_half(q, at & 7, h);
    };
    lds_barrier();
    for (;;) {
        const long long next = row + gridDim.x;
        int             at   = tid;
        asm("" : "+v"(at));  // (places of the pieces are formed where they are used, not kept in registers from row to row)
        if (wave == 0) {
            n.insert(a, z, first, map, l);
            if (MODE != DI_GRADIENT) n.gather(a, row);
        }
        if (TAIL && MODE != DI_GRADIENT) lds_barrier();
        Sums<false> one(a.c2), two(LOG2E);
        if (MODE != DI_GRADIENT) {
#pragma unroll
            for (int i = 0; i < VECS; i += G) {
                u32x4 q[G];
#pragma unroll
                for (int j = 0; j < G; ++j) {
                    q[j] = raw[i + j];
                    if (TAIL) {
                        const int v = (i + j) * THREADS + at;
                        if (v < z.pieces())
                            for (unsigned e = map[v >> (SHIFT - 3)]; e; e = l.next[e - 1])
                                if (e - 1 != DI_TARGET) replace(q[j], v, e - 1, 0xFC00u);
                    }
                }
                const float m = max_of<G>(q);
                one.template add_pieces<G>(q, a.c2, m);
                if (TWO) two.template add_pieces<G>(q, LOG2E, m);
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
            if (MODE == DI_GRADIENT) {
                for (int c = 0; c < a.chunks; ++c) {
                    const f32x4 v = *reinterpret_cast<const f32x4*>(a.sums + (row * a.chunks + c) * 4);
                    s1.add_sums(v[0], v[1], 0.f);
                    if (TWO) s2.add_sums(v[2], v[3], 0.f);
                }
                const float* x = a.chosen + row * (MP_TOP_MAX + 1);
#pragma unroll
                for (int s = 0; s < 2; ++s) n.x[s] = n.there[s] ? x[(tid & 63) + 64 * s] : -INFINITY;
                n.xt = n.target >= 0 && n.target < a.vocab ? x[DI_TARGET] : 0.f;
            } else {
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    s1.add_sums(red[w][0], red[w][1], 0.f);
                    if (TWO) s2.add_sums(red[w][2], red[w][3], 0.f);
                }
            }
            if (MODE == DI_SUMS) {
                if (tid == 0) *reinterpret_cast<f32x4*>(a.sums + (row * a.chunks + chunk) * 4) = f32x4{s1.ref, s1.s, s2.ref, s2.s};
                float* x = a.chosen + row * (MP_TOP_MAX + 1);
                if (chunk == 0) {
#pragma unroll
                    for (int s = 0; s < 2; ++s)
                        if (n.there[s]) x[(tid & 63) + 64 * s] = n.x[s];
                    if (tid == 0) x[DI_TARGET] = n.xt;
                }
            } else {
                finish_row<TAIL, TWO, SHIFT>(a, n, s1, s2, l, factors, first == 0 ? a.row_loss + row : nullptr);
            }
        }
        if (MODE == DI_SUMS) return;
        lds_barrier();
        const RowFactors f    = factors;
        const bool       more = MODE == DI_FUSED && next < a.rows;
        if (wave == 0 && more) ahead.load(a, next);
        Stretch   zn(a.logits + (more ? next : row) * a.ld + first, len);
        uint16_t* dz = a.dlogits + row * a.ld + first;
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const int v = i * THREADS + at;
            u32x4     o = {0, 0, 0, 0};
            asm("" : "+v"(raw[i]));  // (or the compiler keeps the sums' halves, taken apart, in twice the registers until here)
            if (!f.none) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float d[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float x = (float)as_pair(raw[i][k])[h];
                        d[h]          = f.a * __builtin_amdgcn_exp2f(fmaf(x, a.c2, -f.ref));
                        if (TWO) d[h] = fmaf(f.b, __builtin_amdgcn_exp2f(fmaf(x, LOG2E, -f.ref2)), d[h]);
                    }
                    o[k] = (unsigned)f2h(d[0]) | ((unsigned)f2h(d[1]) << 16);
                }
                if (v < z.pieces())
                    for (unsigned e = map[v >> (SHIFT - 3)]; e; e = l.next[e - 1])
                        replace(o, v, e - 1, l.value[e - 1]);
            }
            z.store(dz, v, o);
            if (more) raw[i] = zn.load(v);
        }
        if (!more) return;
        lds_barrier();  // everyone is done with the map
        if (wave == 0) {
            n.remove(a, z, first, map);
            n = ahead;
        }
        row = next;
        z   = zn;
    }
}

}  // namespace mp

using namespace mp;

namespace {

constexpr int DI_FEW = 256 * 8;      // 16-byte pieces of a chunk
constexpr int DI_MOST = 1024 * 16;   // of a row in registers

struct DistillPlan {
    int chunks, chunk;  // 0 chunks: rows in registers
};
DistillPlan distill_plan(int rows, int vocab, bool even) {
    if ((vocab + (even ? 7 : 14)) / 8 <= DI_MOST && !(rows <= 32 && vocab > 32768)) return {0, vocab};
    int n = (vocab + 8 * DI_FEW - 9) / (8 * DI_FEW - 8);
    while ((long long)rows * n * 2 <= 256 && vocab / (n * 2) >= 4096) n *= 2;
    const int chunk = ((vocab + n - 1) / n + 7) / 8 * 8;
    return {(vocab + chunk - 1) / chunk, chunk};
}
size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t distill_bytes(int rows, const DistillPlan& p) {
    return round256((size_t)rows * sizeof(float)) + (p.chunks ? (size_t)rows * (p.chunks * 16 + (MP_TOP_MAX + 1) * sizeof(float)) : 0);
}
size_t distill_most_bytes(int rows, int vocab) {
    const size_t even = distill_bytes(rows, distill_plan(rows, vocab, true)), any = distill_bytes(rows, distill_plan(rows, vocab, false));
    return even > any ? even : any;
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

template <int THREADS, int VECS, int MODE>
int launch_distill(const DistillArgs& a, const mp_distill_desc* d, long long workgroups, hipStream_t hs) {
    constexpr int SHIFT = THREADS == 1024 ? 4 : 3;  // (a map within 64 KB)
    MP_REQUIRE(grid_fits(workgroups, THREADS), "mp_distill_scaled: too many rows");
    const dim3   grid((unsigned)workgroups), block(THREADS);
    const size_t lds = map_words<SHIFT>(a.chunk) * sizeof(unsigned);
    const bool   two = d->hard_weight != 0.f && d->inv_temperature != 1.f;
    if (d->tail && two) hipLaunchKernelGGL((distill_kernel<THREADS, VECS, true, true, MODE, SHIFT>), grid, block, lds, hs, a);
    else if (d->tail) hipLaunchKernelGGL((distill_kernel<THREADS, VECS, true, false, MODE, SHIFT>), grid, block, lds, hs, a);
    else if (two) hipLaunchKernelGGL((distill_kernel<THREADS, VECS, false, true, MODE, SHIFT>), grid, block, lds, hs, a);
    else hipLaunchKernelGGL((distill_kernel<THREADS, VECS, false, false, MODE, SHIFT>), grid, block, lds, hs, a);
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
        const auto grid   = [&](int resident) { return d->rows < 256 * resident ? d->rows : 256 * resident; };
        if (pieces <= 256) rc = launch_distill<256, 1, DI_FUSED>(a, d, grid(8), hs);
        else if (pieces <= 256 * 4) rc = launch_distill<256, 4, DI_FUSED>(a, d, grid(6), hs);
        else if (pieces <= 256 * 8) rc = launch_distill<256, 8, DI_FUSED>(a, d, grid(4), hs);
        else if (pieces <= 256 * 16) rc = launch_distill<256, 16, DI_FUSED>(a, d, grid(4), hs);
        else if (pieces <= 512 * 16) rc = launch_distill<512, 16, DI_FUSED>(a, d, grid(2), hs);
        else rc = launch_distill<1024, 16, DI_FUSED>(a, d, grid(1), hs);
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
