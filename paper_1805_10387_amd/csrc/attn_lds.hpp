// Row-major matrix tiles in LDS for the masked attention kernels, and the matrix-core fragments that come out of them.
//
// A tile keeps rows the way they lie in memory, 64 or 128 columns of fp16 a row, in 16-byte pieces whose place within the row is
// swizzled by the row number, so that (a) plain fragment reads (16 consecutive rows at one piece) and (b) transposing reads
// (`ds_read_b64_tr_b16`: 4 consecutive rows x 4 consecutive pieces' halves) are free of bank conflicts.
//
// v_mfma_f32_32x32x16_f16, operands A then B: a lane supplies 8 contraction values of row lane % 32 of each, lanes 0-31 and 32-63
// (half hf) two disjoint sets; the result lane holds D[i][j], j = lane % 32, i = 8 (r / 4) + 4 hf + r % 4, r = 0 .. 15.  The order of
// the contraction within an instruction is free as long as both operands agree: the registers of a result, packed in pairs, are
// the second operand of the next product as they are, with contraction indices i0 = 16 s + 4 hf + {0..3} and i0 + 8.
#pragma once
#include "common.hpp"

namespace mp {

typedef unsigned u32x4m __attribute__((ext_vector_type(4)));
typedef unsigned u32x2m __attribute__((ext_vector_type(2)));
typedef short    s16x4m __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f16x8 frag8(u32x4m v) { return __builtin_bit_cast(f16x8, v); }
__device__ __forceinline__ unsigned pack_f16(float a, float b) {  // RNE16 of both
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    typedef float    f2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_convertvector(f2{a, b}, h2));
}
// Packed pairs of columns 8 q + 4 hf + {0,1}, {2,3} for q = 2c (a0, a1) and 2c + 1 (b0, b1): lanes r and r + 32 trade, and each has
// the 8 columns from 16 c + 8 hf on.
__device__ __forceinline__ u32x4m trade8(unsigned a0, unsigned a1, unsigned b0, unsigned b1) {
    const auto s0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);
    const auto s1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
    return u32x4m{s0[0], s1[0], s0[1], s1[1]};
}
// A value of each of lanes r and r + 32, joined: both get the result.
template <typename F>
__device__ __forceinline__ float join_halves(float v, F&& op) {
    const auto     s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    const unsigned a = s[0], b = s[1];
    return op(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

template <int ROWB>  // bytes of a row: 128 or 256
struct LdsTile {
    static constexpr int PIECES = ROWB / 16;
    static __device__ __forceinline__ int swz(int r) {
        return ROWB == 128 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3);
    }
    static __device__ __forceinline__ char* piece(char* X, int row, int c) { return X + row * ROWB + ((c ^ swz(row)) << 4); }
    // columns 16 kk + 8 hf ... of a row
    static __device__ __forceinline__ f16x8 frag(const char* X, int row, int kk, int hf) {
        return frag8(*reinterpret_cast<const u32x4m*>(X + row * ROWB + (((2 * kk + hf) ^ swz(row)) << 4)));
    }
    // rows are the contraction: of column col0 + lane % 32, the rows k0 .. k0 + 3 and k0 + 8 .. k0 + 11
    static __device__ __forceinline__ f16x8 frag_t(const char* X, int col0, int k0, int lane) {
        const int  i16 = lane & 15, c = col0 + 16 * ((lane >> 4) & 1) + 4 * (i16 & 3);
        const int  r0 = k0 + (i16 >> 2), r1 = r0 + 8;
        const auto tr = [&](int r) {
            const char* p = X + r * ROWB + (((c >> 3) ^ swz(r)) << 4) + (c & 4) * 2;
            return __builtin_bit_cast(u32x2m, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                  (__attribute__((address_space(3))) s16x4m*)((__attribute__((address_space(3))) void*)p)));
        };
        const u32x2m lo = tr(r0), hi = tr(r1);
        return frag8(u32x4m{lo.x, lo.y, hi.x, hi.y});
    }
};

}  // namespace mp
