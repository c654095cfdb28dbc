// Rows of fp16 logits in the registers of a workgroup: loads at any alignment, sums of exponentials against a running reference.
#pragma once
#include "common.hpp"

namespace mp {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4    u32x4_any __attribute__((aligned(2)));  // stores at any element: the hardware takes them

constexpr float    LOG2E    = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr unsigned NEG_INF2 = 0xFC00FC00u;  // a pair of -inf

static __device__ const u32x4 no_piece = {NEG_INF2, NEG_INF2, NEG_INF2, NEG_INF2};

// A stretch of a row, cut into 16-byte pieces of memory (not of the row: rows of an odd length start anywhere, and a load that crosses
// the pieces takes three times as long).  Piece v holds elements 8 v - head + k, k < 8, of which the first and the last piece
// may have some outside [0, len).
struct Stretch {
    const uint16_t* base;  // 16-byte aligned, `head` elements ahead of the first
    int             head, len;
    __device__ __forceinline__ Stretch(const uint16_t* p, int len_) : head((int)((reinterpret_cast<uintptr_t>(p) >> 1) & 7)), len(len_) { base = p - head; }
    __device__ __forceinline__ int  pieces() const { return (head + len + 7) >> 3; }
    __device__ __forceinline__ int  first_whole() const { return head ? 1 : 0; }
    __device__ __forceinline__ int  end_whole() const { return (head + len) >> 3; }
    __device__ __forceinline__ bool whole(int v) const { return v >= first_whole() && v < end_whole(); }
    // a piece at an end of the stretch: what is outside reads as -inf
    __device__ __forceinline__ u32x4 edge(int v) const {
        unsigned x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = 8 * v + k >= head && 8 * v + k < head + len ? base[8u * (unsigned)v + k] : 0xFC00u;
        return u32x4{x[0] | (x[1] << 16), x[2] | (x[3] << 16), x[4] | (x[5] << 16), x[6] | (x[7] << 16)};
    }
    __device__ __forceinline__ u32x4 load(int v) const {
        u32x4 q = {NEG_INF2, NEG_INF2, NEG_INF2, NEG_INF2};
        if (whole(v)) q = *reinterpret_cast<const u32x4*>(base + 8u * (unsigned)v);
        else if (v < pieces()) q = edge(v);
        return q;
    }
    // the whole piece next to v: a load without a branch, so that the waits for it need not wait for later ones
    __device__ __forceinline__ u32x4 load_inside(int v) const {
        const bool      any = end_whole() > first_whole();
        const u32x4*    p   = any ? reinterpret_cast<const u32x4*>(base) : &no_piece;
        const unsigned  at  = any ? (unsigned)max(first_whole(), min(v, end_whole() - 1)) : 0u;
        return p[at];
    }
    // out: where element 0 belongs
    __device__ __forceinline__ void store(uint16_t* out, int v, const u32x4 q) const {
        uint16_t* o = out - head + 8u * (unsigned)v;
        if (whole(v)) {
            *reinterpret_cast<u32x4_any*>(o) = q;
        } else if (v < pieces()) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (8 * v + k >= head && 8 * v + k < head + len) o[k] = (uint16_t)((k & 1) ? q[k >> 1] >> 16 : q[k >> 1] & 0xFFFFu);
        }
    }
};

// The pieces of a stretch that thread tid of THREADS holds, piece i THREADS + tid in raw[i]; `last` is the stretch's last piece where it is not
// whole.  settle() before raw[i] is used for the first time.
template <int THREADS, int VECS>
__device__ __forceinline__ void load_pieces(const Stretch& z, int tid, u32x4 (&raw)[VECS], u32x4& last) {
    const int v = z.pieces() - 1;
    last        = u32x4{NEG_INF2, NEG_INF2, NEG_INF2, NEG_INF2};
    if (VECS > 1 && v >= z.end_whole() && v % THREADS == tid) last = z.edge(v);
    raw[0] = z.load(tid);
#pragma unroll
    for (int i = 1; i < VECS; ++i) raw[i] = z.load_inside(i * THREADS + tid);
}
template <int THREADS>
__device__ __forceinline__ void settle(const Stretch& z, int i, int tid, u32x4& q, const u32x4& last) {
    if (i > 0 && (i + 1) * THREADS > z.end_whole()) {
        const int v = i * THREADS + tid;
        if (v >= z.end_whole()) q = v == z.pieces() - 1 ? last : u32x4{NEG_INF2, NEG_INF2, NEG_INF2, NEG_INF2};
    }
}

__device__ __forceinline__ f16x2 as_pair(unsigned w) { return __builtin_bit_cast(f16x2, w); }
// (the builtin maximum first makes every operand quiet, which is an instruction more each)
__device__ __forceinline__ unsigned pair_max(unsigned a, unsigned b) {
    unsigned d;
    asm("v_pk_max_f16 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
    return d;
}
template <int N>
__device__ __forceinline__ float max_of(const u32x4* q) {
    unsigned m = pair_max(pair_max(q[0][0], q[0][1]), pair_max(q[0][2], q[0][3]));
#pragma unroll
    for (int i = 1; i < N; ++i) m = pair_max(m, pair_max(pair_max(q[i][0], q[i][1]), pair_max(q[i][2], q[i][3])));
    return fmaxf((float)as_pair(m)[0], (float)as_pair(m)[1]);
}

__device__ __forceinline__ float max_of_half(const u32x4 q, int h) {
    const unsigned m = pair_max(q[2 * h], q[2 * h + 1]);
    return fmaxf((float)as_pair(m)[0], (float)as_pair(m)[1]);
}

// Sums over exponentials of base 2, y = c2 x - ref with c2 = log2(e) / temperature:  s = sum 2^y, t = sum 2^y y (for the entropy).
// ref is the largest c2 x so far, rounded: y of the largest is what that left, at most 2^-24 |c2 x| (1 where 1 / temperature is 256 and x near
// 60000, so that its term is 2^y and not 1).  All sums of a row and all that is made of them have the same ref, so that it cancels.  Never below
// the floor, which is below every finite logit, so that a row of -inf makes no NaN of differences.  +inf and NaN make s NaN.
constexpr float REF_FLOOR = -70000.f;
template <bool ENTROPY>
struct Sums {
    float ref, s, t;
    __device__ __forceinline__ explicit Sums(float c2) : ref(REF_FLOOR * c2), s(0.f), t(0.f) {}
    __device__ __forceinline__ void move(float to) {  // to >= ref
        const float d = ref - to, k = __builtin_amdgcn_exp2f(d);
        if (ENTROPY) t = k * (t + d * s);
        s *= k;
        ref = to;
    }
    __device__ __forceinline__ void add(float y) {
        const float e = __builtin_amdgcn_exp2f(y);
        s += e;
        if (ENTROPY) t = fmaf(e, fmaxf(y, -150.f), t);  // (0 x -inf; 2^-150 is 0)
    }
    // N pieces whose largest logit is `top`
    template <int N>
    __device__ __forceinline__ void add_pieces(const u32x4* q, float c2, float top) {
        move(fmaxf(ref, top * c2));
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                add(fmaf((float)as_pair(q[i][k])[0], c2, -ref));
                add(fmaf((float)as_pair(q[i][k])[1], c2, -ref));
            }
    }
    __device__ __forceinline__ void add_sums(float ref2, float s2, float t2) {
        const float to = fmaxf(ref, ref2), d = ref2 - to, k = __builtin_amdgcn_exp2f(d);
        move(to);
        if (ENTROPY) t += k * (t2 + d * s2);
        s += k * s2;
    }
    __device__ __forceinline__ void over_wave() {
        move(wave_max(ref));
        s = wave_sum(s);
        if (ENTROPY) t = wave_sum(t);
    }
};

// As add_pieces of one, and of two with twice its c2: exponentials that are the squares of the others.
template <int N>
__device__ __forceinline__ void add_pieces_and_squares(Sums<false>& one, Sums<false>& two, const u32x4* q, float c2, float top) {
    const float to = fmaxf(one.ref, top * c2), k = __builtin_amdgcn_exp2f(one.ref - to);
    one.s *= k;
    two.s *= k * k;
    one.ref = to;
    two.ref = 2.f * to;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = __builtin_amdgcn_exp2f(fmaf((float)as_pair(q[i][j >> 1])[j & 1], c2, -to));
            one.s += e;
            two.s = fmaf(e, e, two.s);
        }
}

}  // namespace mp
