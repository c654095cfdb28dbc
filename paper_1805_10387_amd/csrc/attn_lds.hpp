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

__device__ __forceinline__ unsigned lds_address(const void* p) { return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }

template <int ROWB>  // bytes of a row: 128 or 256, and a tile begins at a multiple of it
struct LdsTile {
    static constexpr int PIECES = ROWB / 16;
    static __device__ __forceinline__ int swz(int r) {
        return ROWB == 128 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3);
    }
    // Fragments are read at a lane's place in the tile, whose address is a register, with the piece exchanged by bits of a constant and
    // whole rows (multiples of 16, after which the swizzle repeats) added: addresses of their own would each take a register.
    // The swizzle of rows 8 further differs in one bit.
    typedef __attribute__((address_space(3))) const char as3_char;
    // row lane % 32, piece hf ...
    static __device__ __forceinline__ unsigned plain(int lane) { return (lane & 31) * ROWB + (((lane >> 5) ^ swz(lane & 31)) << 4); }
    // ... columns 16 kk + 8 hf of row `row` + lane % 32
    static __device__ __forceinline__ f16x8 frag(unsigned at, int row, int kk) {
        return frag8(*reinterpret_cast<__attribute__((address_space(3))) const u32x4m*>((as3_char*)(uintptr_t)(at ^ (unsigned)(kk << 5)) + row * ROWB));
    }
    // rows are the contraction: rows 4 hf + (lane % 16) / 4, columns 16 (lane / 16 % 2) + 4 (lane % 4) ...
    static __device__ __forceinline__ unsigned across(int lane) {
        const int r = 4 * (lane >> 5) + (lane >> 2 & 3);
        return r * ROWB + (((lane >> 4 & 1) * 2 + (lane >> 1 & 1)) ^ swz(r)) * 16 + (lane & 1) * 8;
    }
    // ... of column 32 dt + lane % 32, rows `row` + 4 hf + {0..3} and 8 further
    static __device__ __forceinline__ f16x8 frag_t(unsigned at, int row, int dt) {
        const auto tr = [](unsigned p, int offset) {
            return __builtin_bit_cast(u32x2m, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4m*)((as3_char*)(uintptr_t)p + offset)));
        };
        const u32x2m lo = tr(at ^ (unsigned)(dt << 6), row * ROWB), hi = tr(at ^ (unsigned)(dt << 6 | 32), (row + 8) * ROWB);
        return frag8(u32x4m{lo.x, lo.y, hi.x, hi.y});
    }
};

// 64 rows of a matrix straight into an LDS tile (`buffer_load ... lds`: no staging registers), by NW waves.  A wave load deposits 64
// lanes x 16 bytes side by side, so each lane fetches the piece whose place its own is.  Rows from `rows` on and columns from `d` on
// lie outside the buffer and arrive as zeros.
constexpr unsigned LDS_OUT = 0x80000000u;  // (leading dimensions are below 2^22, so a tile spans less)
template <int ROWB, int NW>
struct TileLoad {
    typedef LdsTile<ROWB> Tile;
    static constexpr int LOADS = 64 * ROWB / 1024, N = LOADS / NW, RPL = 1024 / ROWB;  // of a tile, of a wave; rows of a load
    static constexpr int VAR = RPL * NW % 16 ? 2 : 1;  // a row's swizzle repeats after 16 rows
    unsigned             voff[VAR], step;
    __device__ __forceinline__ void init(int ld, int d, int wave, int lane) {
        step = (unsigned)(RPL * NW) * 2u * (unsigned)ld;
#pragma unroll
        for (int j = 0; j < VAR; ++j) {
            const int row = (wave + NW * j) * RPL + lane / Tile::PIECES, c = (lane % Tile::PIECES) ^ Tile::swz(row);
            voff[j]       = 8 * c < d ? (unsigned)(wave * RPL + lane / Tile::PIECES) * 2u * (unsigned)ld + 16u * c : LDS_OUT;
        }
    }
    // Asks for rows row0 .. row0 + 63 of M (a column block's first element) into X.  (One vmcnt each.)
    __device__ __forceinline__ void issue(const uint16_t* M, int ld, int row0, int rows, int d, char* X, int wave) const {
        const int      left  = min(rows - row0, 64);
        const uint64_t base  = reinterpret_cast<uint64_t>(M + (long long)row0 * ld);
        const unsigned bytes = ((unsigned)(left - 1) * (unsigned)ld + (unsigned)d) * 2u;
        u32x4m         rsrc;
        rsrc.x = __builtin_amdgcn_readfirstlane((unsigned)base);
        rsrc.y = __builtin_amdgcn_readfirstlane((unsigned)(base >> 32) & 0xFFFFu);
        rsrc.z = __builtin_amdgcn_readfirstlane(bytes);
        rsrc.w = 0x00020000u;
        const unsigned to = __builtin_amdgcn_readfirstlane(lds_address(X) + (unsigned)wave * 1024u);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            // (one assembly block: the compiler would wait for every load in flight ahead of any LDS read)
            const unsigned v = voff[j % VAR] + (unsigned)j * step;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to + j * NW * 1024u), "v"(v), "s"(rsrc) : "memory");
        }
    }
    // Zeroes non-finite elements of a tile that has arrived; bad (may be null): per row, NaN if it had one, else 0.
    static __device__ __forceinline__ void clean(char* X, float* bad, int wave, int lane) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            u32x4m* const at = reinterpret_cast<u32x4m*>(X + (wave + NW * j) * 1024 + lane * 16);
            u32x4m        q  = *at;
            unsigned      any = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                // exponent all ones in a half: bit 10 of it is carried out of the mantissa's top when 1 is added there
                const unsigned full = ((q[w] & 0x7C007C00u) + 0x04000400u) & 0x80008000u;
                any |= full;
                q[w] &= ~(full | (full - (full >> 15)));
            }
            if (any) *at = q;
            if (bad) {  // the pieces of a row are with neighbouring lanes
                const unsigned long long m     = __ballot(any != 0);
                const int                first = lane / Tile::PIECES * Tile::PIECES;
                if (lane == first) bad[(wave + NW * j) * RPL + lane / Tile::PIECES] = (m >> first) & ((1ull << Tile::PIECES) - 1) ? NAN : 0.f;
            }
        }
    }
};

// 64 words, or 64 pairs of words, side by side in memory straight into LDS, by one wave (the pairs by half of it: the other half's
// lanes lie outside and write zeros behind them).
__device__ __forceinline__ u32x4m plain_buffer(const void* p, unsigned bytes) {
    const uint64_t base = reinterpret_cast<uint64_t>(p);
    return u32x4m{(unsigned)__builtin_amdgcn_readfirstlane((unsigned)base), (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(base >> 32) & 0xFFFFu), bytes,
                  0x00020000u};
}
__device__ __forceinline__ void load_words(const float* from, float* X, int lane) {
    const unsigned to = __builtin_amdgcn_readfirstlane(lds_address(X));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(4 * lane), "s"(plain_buffer(from, 256)) : "memory");
}
__device__ __forceinline__ void load_ranges(const int2* from, int2* X, int lane) {
    const unsigned to = __builtin_amdgcn_readfirstlane(lds_address(X));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(16 * lane), "s"(plain_buffer(from, 512)) : "memory");
}

}  // namespace mp
