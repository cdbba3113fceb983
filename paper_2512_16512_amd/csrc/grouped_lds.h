// Operands of the grouped and 8-bit products in LDS: their copies from memory,
// their layouts, and the fragments that the matrix instructions take.
//
// A stage holds KB = 128 or 64 bytes of k (128 e4m3 values; 64 or 32 bf16 ones).  An
// operand whose rows run along k lies as rows of KB bytes, its 16-byte chunk c of
// row r at slot c ^ swz_row(r): the fragment reads, 16 rows of two neighbouring
// chunks at a time, then meet every bank once.  An operand with one k a row lies
// as it is in memory, read by the transpose reads, chunk c of row k at
// c ^ swz_k(k).
//
// A fragment is MI rows of an operand's stage, KB bytes of k each: piece q holds
// the 16 bytes of chunk KG q + lane / MI, KG = 64 / MI, for both operands.
#pragma once

#include "grouped.h"
#include "lds_dma.h"

namespace xtc {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int MI = 16;   // rows (or columns) of a fragment

// Chunk swizzle of rows of KB bytes along k.  The reads are served 16 lanes at a
// time, rows 0-3 and 12-15 of one chunk with rows 4-11 of its neighbour: of 128
// bytes two rows fill the banks, of 64 four.
template <int KB>
__device__ __forceinline__ int swz_row(int r) {
    return KB == 128 ? (r >> 1) & 7 : (0x78 >> (2 * ((r >> 2) & 3))) & 3;   // 0, 2, 3, 1
}

// Chunk swizzle of rows of CB chunks with one k each: spreads the four rows that
// a transpose read takes at once, and rows k and k + 8, over the banks (rows of
// 8 chunks fill half of them, so that odd rows are apart by themselves; of 4, where four
// rows fill them, rows 8 apart remain; of 2 those meet).
template <int CB>
__device__ __forceinline__ int swz_k(int k) {
    return CB == 2   ? 0
           : CB == 4 ? (k >> 2) & 2
           : CB == 8 ? (k & 2) | ((k >> 1) & 4)
                     : ((k & 1) * 6) ^ ((k & 2) * 5) ^ (((k >> 3) & 1) * 2);
}

// WIDE: e4m3 operands widened to bf16 (fp32 sums; see mfma_fp8.h).
template <Kind KIND, bool WIDE, int KB = 128>
struct Product {
    static constexpr int PIECES = KB / 16 / (64 / MI);
    // registers of a fragment as the instructions take it
    struct Frag {
        u32x4 v[WIDE ? 2 * PIECES : PIECES];
    };
    // piece q of them, from the 16 bytes read
    static __device__ __forceinline__ void prepare(Frag &f, const u32x4 (&raw)[PIECES], int q) {
        if constexpr (WIDE) {
            f.v[2 * q] = __builtin_bit_cast(u32x4, widen_fp8(raw[q][0], raw[q][1]));
            f.v[2 * q + 1] = __builtin_bit_cast(u32x4, widen_fp8(raw[q][2], raw[q][3]));
        } else {
            f.v[q] = raw[q];
        }
    }
    static __device__ __forceinline__ Frag prepare(const u32x4 (&raw)[PIECES]) {
        Frag f;
#pragma unroll
        for (int q = 0; q < PIECES; ++q) prepare(f, raw, q);
        return f;
    }
    static __device__ __forceinline__ f32x4 mul(const Frag &a, const Frag &b, f32x4 c) {
        if constexpr (KIND == kFp8 && !WIDE) {
#pragma unroll
            for (int s = 0; s < PIECES / 2; ++s) {
                const i32x8 x = __builtin_bit_cast(i32x8, __builtin_shufflevector(a.v[2 * s], a.v[2 * s + 1], 0, 1, 2, 3, 4, 5, 6, 7));
                const i32x8 y = __builtin_bit_cast(i32x8, __builtin_shufflevector(b.v[2 * s], b.v[2 * s + 1], 0, 1, 2, 3, 4, 5, 6, 7));
                c = mma_fp8(x, y, c);
            }
        } else {
#pragma unroll
            for (int s = 0; s < (WIDE ? 2 : 1) * PIECES; ++s)
                c = Bf16Mfma<MI>::mma(__builtin_bit_cast(u16x8, a.v[s]), __builtin_bit_cast(u16x8, b.v[s]), c);
        }
        return c;
    }
};

// One operand's copies: where this lane's 16-byte chunks lie in a stage (kOOB,
// read as zeros, outside the operand), and the buffer of a stage.
template <bool K_ROWS, int ROWS, int PER_WAVE, int KB = 128>
struct Source {
    const unsigned char *base;   // of the stage to copy next
    int64_t ld;                  // bytes
    int rows;                    // rows (or columns of rows along k) that exist
    int off[PER_WAVE];
    int k_at[PER_WAVE];          // rows along k: the chunk's first byte of k

    __device__ __forceinline__ Source(const unsigned char *p, int64_t ld_, int extent, int wave, int lane)
        : base(p), ld(ld_), rows(extent < ROWS ? extent : ROWS) {
#pragma unroll
        for (int q = 0; q < PER_WAVE; ++q) {
            const int blk = wave * PER_WAVE + q;
            if constexpr (K_ROWS) {
                constexpr int CB = ROWS / 8;      // chunks of a row (one k)
                const int byte = blk * 1024 + lane * 16, k = byte / (ROWS * 2), c = (byte / 16 % CB) ^ swz_k<CB>(k);
                off[q] = c * 8 < extent ? (int)(k * ld) + c * 16 : kOOB;
                k_at[q] = 0;
            } else {
                constexpr int CH = KB / 16;           // chunks of a row
                const int row = blk * (64 / CH) + lane / CH, c = (lane % CH) ^ swz_row<KB>(row);
                off[q] = row < extent ? (int)(row * ld) + c * 16 : kOOB;
                k_at[q] = c * 16;
            }
        }
    }
    // The buffer of the next stage, of which `left` values of k exist; steps
    // `stages` on.
    __device__ __forceinline__ i32x4 stage(int left, int elt, int stages = 1) {
        const int bk = KB / elt, ks = left < bk ? left : bk;
        int bytes = 0;
        // (whole chunks: one that holds any value of a row is mapped)
        if (left > 0) bytes = K_ROWS ? (ks - 1) * (int)ld + ((rows * 2 + 15) & ~15) : (rows - 1) * (int)ld + ((ks * elt + 15) & ~15);
        const i32x4 r = make_rsrc(base, bytes);
        base += stages * (K_ROWS ? bk * ld : KB);
        return r;
    }
    // Where this lane's chunk of copy q lies in it.
    __device__ __forceinline__ int offset(int q, int left, int elt) const {
        return K_ROWS || k_at[q] < left * elt ? off[q] : kOOB;
    }
};

// The same for rows at any address, through registers: fetch() starts the loads
// of the next stage, store() writes them where the copies would have.
template <bool K_ROWS, int ROWS, int PER_WAVE, int KB>
struct Carried {
    const unsigned char *base;
    int64_t ld;
    int extent, rows;
    u32x4 r[PER_WAVE];

    __device__ __forceinline__ Carried(const unsigned char *p, int64_t ld_, int extent_)
        : base(p), ld(ld_), extent(extent_), rows(extent_ < ROWS ? extent_ : ROWS) {}

    // 16 bytes at p of which the first `valid` exist (whole elements of ELT bytes).
    template <int ELT>
    static __device__ __forceinline__ u32x4 cut(const unsigned char *p, int valid) {
        u32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 16; i += ELT)
            if (i < valid) v[i / 4] |= (unsigned)(ELT == 2 ? *reinterpret_cast<const unsigned short *>(p + i) : p[i]) << (8 * (i % 4));
        return v;
    }
    // v shifted down by `bytes`, 0 to 15.
    static __device__ __forceinline__ u32x4 shifted(const u32x4 &v, int bytes) {
        // by 8 and by 4 bytes as asked (bitwise selects), then within a dword
        const unsigned m8 = bytes & 8 ? ~0u : 0u, m4 = bytes & 4 ? ~0u : 0u;
        const unsigned a0 = v[0] ^ ((v[0] ^ v[2]) & m8), a1 = v[1] ^ ((v[1] ^ v[3]) & m8), a2 = v[2] & ~m8, a3 = v[3] & ~m8;
        const unsigned b0 = a0 ^ ((a0 ^ a1) & m4), b1 = a1 ^ ((a1 ^ a2) & m4), b2 = a2 ^ ((a2 ^ a3) & m4), b3 = a3 & ~m4;
        const unsigned s = (unsigned)(bytes & 3);
        return u32x4{(unsigned)__builtin_amdgcn_alignbyte(b1, b0, s), (unsigned)__builtin_amdgcn_alignbyte(b2, b1, s),
                     (unsigned)__builtin_amdgcn_alignbyte(b3, b2, s), (unsigned)__builtin_amdgcn_alignbyte(0, b3, s)};
    }
    // `wide`: the operand's rows hold 16 bytes at least.  A chunk that ends past its
    // row (or the last of k) is then read from 16 bytes before that end and
    // shifted; of narrower rows byte by byte.
    template <int ELT>
    __device__ __forceinline__ void fetch(int left, bool wide, int wave, int lane) {
        constexpr int BK = KB / ELT;
        const bool whole = left >= BK && (!K_ROWS || extent >= ROWS);
        const unsigned char *row_at[PER_WAVE];
        int at[PER_WAVE], end[PER_WAVE];       // bytes of the row: the chunk's first, and one past the last
#pragma unroll
        for (int q = 0; q < PER_WAVE; ++q) {
            const int blk = wave * PER_WAVE + q;
            if constexpr (K_ROWS) {
                constexpr int CB = ROWS / 8;
                const int byte = blk * 1024 + lane * 16, k = byte / (ROWS * 2);
                at[q] = ((byte / 16 % CB) ^ swz_k<CB>(k)) * 16;
                end[q] = k < left ? extent * 2 : 0;
                row_at[q] = base + (k < left ? k : 0) * ld;
            } else {
                constexpr int CH = KB / 16;
                // (rows past the last one repeat it: nothing of theirs is kept)
                const int row = blk * (64 / CH) + lane / CH;
                at[q] = ((lane % CH) ^ swz_row<KB>(row)) * 16;
                end[q] = left * ELT;
                row_at[q] = base + (row < rows ? row : rows - 1) * ld;
            }
        }
        if (whole) {
#pragma unroll
            for (int q = 0; q < PER_WAVE; ++q) __builtin_memcpy(&r[q], row_at[q] + at[q], 16);
        } else if (left > 0 && wide) {
            u32x4 v[PER_WAVE];
#pragma unroll
            for (int q = 0; q < PER_WAVE; ++q) {
                // (of a row of k past the last one, whose end is 0, the first row's)
                const int last = (K_ROWS ? extent * 2 : end[q]) - 16;
                __builtin_memcpy(&v[q], row_at[q] + (at[q] < last ? at[q] : last), 16);
            }
#pragma unroll
            for (int q = 0; q < PER_WAVE; ++q) {
                const int over = at[q] - (end[q] - 16);
                const u32x4 none = {0, 0, 0, 0};
                r[q] = over <= 0 ? v[q] : over < 16 ? shifted(v[q], over) : none;
            }
        } else {
#pragma unroll
            for (int q = 0; q < PER_WAVE; ++q) r[q] = cut<ELT>(row_at[q] + at[q], left > 0 ? end[q] - at[q] : 0);
        }
        base += K_ROWS ? BK * ld : KB;
    }
    __device__ __forceinline__ void store(unsigned char *lds, int q, int lane) const {
        *reinterpret_cast<u32x4 *>(lds + q * 1024 + lane * 16) = r[q];
    }
};

// The same for bf16 rows of eight values at least, SETS stages ahead: a load is never waited for before its stage is
// stored, and none stands in a branch, whose end would have to wait for them all.  A chunk that ends past its row
// (or the last of k) is read from 16 bytes before that end and shifted as it is stored.
template <bool K_ROWS, int ROWS, int PER_WAVE, int KB, int SETS>
struct CarriedAhead {
    static constexpr int BK = KB / 2;
    const unsigned char *base;   // of the stage to fetch next, or the last one again
    int64_t ld;
    int extent, left;            // (left: values of k from base on, one at least)
    int64_t off[PER_WAVE];       // of the chunks' rows
    u32x4 r[SETS][PER_WAVE];

    __device__ __forceinline__ CarriedAhead(const unsigned char *p, int64_t ld_, int extent_, int k, int wave, int lane)
        : base(p), ld(ld_), extent(extent_ < ROWS + 8 ? extent_ : ROWS + 8), left(k) {
#pragma unroll
        for (int q = 0; q < PER_WAVE; ++q) {
            // (rows past the last one repeat it, of k past the last one the first: nothing of theirs is kept)
            const int row = row_of(q, wave, lane);
            off[q] = (K_ROWS || row < extent_ ? row : extent_ - 1) * ld;
        }
    }

    // Where this lane's chunk q lies: its row (or k), and its first byte of it.
    static __device__ __forceinline__ int row_of(int q, int wave, int lane) {
        const int blk = wave * PER_WAVE + q;
        return K_ROWS ? (blk * 1024 + lane * 16) / (ROWS * 2) : blk * (1024 / KB) + lane / (KB / 16);
    }
    static __device__ __forceinline__ int byte_of(int q, int wave, int lane) {
        const int row = row_of(q, wave, lane);
        if constexpr (K_ROWS) return (((wave * PER_WAVE + q) * 64 + lane) % (ROWS / 8) ^ swz_k<ROWS / 8>(row)) * 16;
        else return ((lane % (KB / 16)) ^ swz_row<KB>(row)) * 16;
    }
    template <int SET>
    __device__ __forceinline__ void fetch(int wave, int lane) {
        const int last = (K_ROWS ? extent : left < BK + 8 ? left : BK + 8) * 2 - 16;
#pragma unroll
        for (int q = 0; q < PER_WAVE; ++q) {
            const int at = byte_of(q, wave, lane);
            const int64_t o = !K_ROWS || row_of(q, wave, lane) < left ? off[q] : 0;
            __builtin_memcpy(&r[SET][q], base + o + (at < last ? at : last), 16);
        }
        const bool more = left > BK;
        base += more ? (K_ROWS ? BK * ld : KB) : 0;
        left -= more ? BK : 0;
    }
    // `of_k`: values of k from the stage's first on
    template <int SET>
    __device__ __forceinline__ void store(unsigned char *lds, int q, int of_k, int wave, int lane) const {
        u32x4 v = r[SET][q];
        if (of_k < BK || (K_ROWS && extent < ROWS)) {
            const int end = K_ROWS ? (row_of(q, wave, lane) < of_k ? extent * 2 : 0) : of_k * 2;
            const int over = byte_of(q, wave, lane) - (end - 16);
            const u32x4 none = {0, 0, 0, 0};
            v = over <= 0 ? v : over < 16 ? Carried<K_ROWS, ROWS, PER_WAVE, KB>::shifted(v, over) : none;
        }
        *reinterpret_cast<u32x4 *>(lds + q * 1024 + lane * 16) = v;
    }
};

// Fragment of the rows (or columns) first .. first + MI - 1 from an operand's
// stage at s, `ROWS` rows of it in all.
template <bool K_ROWS, int ROWS, int KB>
__device__ __forceinline__ void read_fragment(const unsigned char *s, int first, int lane, u32x4 (&raw)[KB * MI / 1024]) {
    constexpr int KG = 64 / MI;
    const int lrow = lane % MI, lgrp = lane / MI;
    if constexpr (!K_ROWS) {
        const int row = first + lrow, swz = swz_row<KB>(row);
#pragma unroll
        for (int q = 0; q < KB / 16 / KG; ++q)
            raw[q] = *reinterpret_cast<const u32x4 *>(s + row * KB + (((KG * q + lgrp) ^ swz) << 4));
    } else {
        const int rsub = (lane & 15) >> 2, c = first + (lrow & ~15) + 4 * (lane & 3);
#pragma unroll
        for (int q = 0; q < KB / 16 / KG; ++q) {
            // k and k + 4: their swizzle is one
            const int k = 8 * (KG * q + lgrp) + rsub;
            const unsigned char *q0 = s + k * ROWS * 2 + (((c >> 3) ^ swz_k<ROWS / 8>(k)) << 4) + 8 * (lane & 1);
            const u16x4 lo = ds_read_tr16(reinterpret_cast<const unsigned short *>(q0));
            const u16x4 hi = ds_read_tr16(reinterpret_cast<const unsigned short *>(q0 + 4 * ROWS * 2));
            raw[q] = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
}

}  // namespace xtc
