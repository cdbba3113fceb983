// The grouped and 8-bit products on LDS-staged tiles: operands copied straight
// from memory into LDS (dma16), two stages of 128 bytes of k (128 e4m3 or 64 bf16
// values) in a ring.
//
// LDS layouts.  An operand whose rows run along k lies as rows of 128 bytes, its
// 16-byte chunk c of row r at slot c ^ (r >> 1 & 7): the fragment reads, 16 or 32
// rows of one or two chunks at a time, then meet every bank once.  An operand
// with one k a row lies as it is in memory, read by the transpose reads, chunk
// c of row k at c ^ swz_k(k).
//
// A fragment is MI rows of an operand's stage, 128 bytes of k each: piece q holds
// the 16 bytes of chunk KG q + lane / MI, KG = 64 / MI, for both operands.
//
// Loop.  A wave keeps the fragments of its columns (B) of a stage in registers
// and walks through its rows (A), one fragment ahead.  Before the last row
// fragment's products every read of the stage has returned; a wait for the
// next stage's copies and a barrier stand there, after which the copies of the
// stage after it go into the slot just read, and the next stage's
// first fragments are read while the last products run.
#include "grouped.h"
#include "lds_dma.h"
#include "unroll.h"

namespace xtc {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// Chunk swizzle of rows with one k each (see the bf16 matrix product): spreads
// the four rows that a transpose read takes at once, and rows k and k + 8.
__device__ __forceinline__ int swz_k(int k) {
    return ((k & 1) * 6) ^ ((k & 2) * 5) ^ (((k >> 3) & 1) * 2);
}

// WIDE: e4m3 operands widened to bf16 (fp32 sums; see mfma_fp8.h).
template <Kind KIND, bool WIDE, int MI>
struct Product {
    static constexpr int KG = 64 / MI, PIECES = 8 / KG;
    typedef typename Bf16Mfma<MI>::acc_t acc_t;
    static constexpr int NACC = Bf16Mfma<MI>::NACC;
    // registers of a fragment as the instructions take it
    struct Frag {
        u32x4 v[WIDE ? 2 * PIECES : PIECES];
    };
    static __device__ __forceinline__ Frag prepare(const u32x4 (&raw)[PIECES]) {
        Frag f;
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            if constexpr (WIDE) {
                f.v[2 * q] = __builtin_bit_cast(u32x4, widen_fp8(raw[q][0], raw[q][1]));
                f.v[2 * q + 1] = __builtin_bit_cast(u32x4, widen_fp8(raw[q][2], raw[q][3]));
            } else {
                f.v[q] = raw[q];
            }
        }
        return f;
    }
    static __device__ __forceinline__ acc_t mul(const Frag &a, const Frag &b, acc_t c) {
        if constexpr (KIND == kFp8 && !WIDE) {
#pragma unroll
            for (int s = 0; s < PIECES / 2; ++s) {
                const i32x8 x = __builtin_bit_cast(i32x8, __builtin_shufflevector(a.v[2 * s], a.v[2 * s + 1], 0, 1, 2, 3, 4, 5, 6, 7));
                const i32x8 y = __builtin_bit_cast(i32x8, __builtin_shufflevector(b.v[2 * s], b.v[2 * s + 1], 0, 1, 2, 3, 4, 5, 6, 7));
                c = Fp8Mfma<MI>::mma(x, y, c);
            }
        } else {
#pragma unroll
            for (int s = 0; s < (WIDE ? 2 : 1) * PIECES; ++s)
                c = Bf16Mfma<MI>::mma(__builtin_bit_cast(u16x8, a.v[s]), __builtin_bit_cast(u16x8, b.v[s]), c);
        }
        return c;
    }
};

template <Kind KIND, int BM, int BN, int WM, int WN, int MI>
struct TileCfg {
    static constexpr int E = KIND == kFp8 ? 1 : 2, BK = 128 / E;
    static constexpr bool A_K_ROWS = KIND == kWgrad, B_K_ROWS = KIND == kWgrad || KIND == kBf16N;
    static constexpr int NWM = BM / WM, NWN = BN / WN, NWAVES = NWM * NWN, NT = NWAVES * 64;
    static constexpr int TM = WM / MI, TN = WN / MI;
    static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128;
    static constexpr int A_PER_WAVE = A_BYTES / 1024 / NWAVES, B_PER_WAVE = B_BYTES / 1024 / NWAVES;
    static constexpr int S_BYTES = KIND == kFp8 ? NWAVES * 256 : 0;   // scales: 64 values a wave
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + S_BYTES;
    static constexpr int LOADS = A_PER_WAVE + B_PER_WAVE + (KIND == kFp8 ? 1 : 0);
    static_assert(A_PER_WAVE * NWAVES * 1024 == A_BYTES && B_PER_WAVE * NWAVES * 1024 == B_BYTES,
                  "tiles must split into whole 1 KiB blocks per wave");
    static_assert(KIND != kFp8 || NWAVES > BM / 64, "a wave for B's scales");
    static_assert(128 % WN == 0, "the columns of a wave share a scale");
    static_assert(2 * STAGE_BYTES <= 160 * 1024, "LDS budget");
    static_assert(TM >= 2, "a fragment ahead");
};

// Source of one operand's copies.
template <bool K_ROWS, int ROWS, int PER_WAVE>
struct Source {
    const unsigned char *base;   // of the stage to copy next
    int64_t ld;
    int off[PER_WAVE];           // byte offset of this lane's chunk in a stage, kOOB outside the operand
    int k_at[PER_WAVE];          // rows along k: its first byte of k

    __device__ __forceinline__ Source(const unsigned char *p, int64_t ld_, int extent, int wave, int lane, int elt)
        : base(p), ld(ld_) {
        each([&](int q) {
            const int blk = wave * PER_WAVE + q;
            if constexpr (K_ROWS) {
                constexpr int CB = ROWS / 8;      // chunks of a row (one k)
                const int byte = blk * 1024 + lane * 16, k = byte / (ROWS * 2), c = (byte / 16 % CB) ^ swz_k(k);
                off[q] = c * 8 < extent ? (int)(k * ld) + c * 16 : kOOB;
                k_at[q] = 0;
            } else {
                const int row = blk * 8 + lane / 8, c = (lane & 7) ^ ((row >> 1) & 7);
                off[q] = row < extent ? (int)(row * ld) + c * 16 : kOOB;
                k_at[q] = c * 16;
            }
        });
    }
    template <typename F>
    static __device__ __forceinline__ void each(F &&f) {
#pragma unroll
        for (int q = 0; q < PER_WAVE; ++q) f(q);
    }
};

template <Kind KIND, bool WIDE, int BM, int BN, int WM, int WN, int MI>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * 64)
grouped_tile_kernel(GroupedArgs p) {
    typedef TileCfg<KIND, BM, BN, WM, WN, MI> G;
    typedef Product<KIND, WIDE, MI> P;
    typedef typename P::acc_t acc_t;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * G::STAGE_BYTES];

    Tile t;
    if (!find_tile<KIND, BM, BN>(p, t)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / G::NWN, wn = wave % G::NWN;
    const int lrow = lane % MI, lgrp = lane / MI;
    const unsigned smem_base = lds_address(smem);
    const int KT = (t.k + G::BK - 1) / G::BK;

    Source<G::A_K_ROWS, BM, G::A_PER_WAVE> sa(t.A, t.lda, t.m, wave, lane, G::E);
    Source<G::B_K_ROWS, BN, G::B_PER_WAVE> sb(t.B, t.ldb, t.n, wave, lane, G::E);
    const int a_rows = t.m < BM ? t.m : BM, b_rows = t.n < BN ? t.n : BN;

    // this lane's scale of a stage: rows of A, then the blocks of B's columns
    int s_off = kOOB;
    const float *s_base = t.SA;
    int s_bytes = 0;
    if constexpr (KIND == kFp8) {
        const int r = wave * 64 + lane;
        if (wave < BM / 64) {
            s_off = r < a_rows ? r * (int)p.ldsa * 4 : kOOB;
            s_bytes = ((a_rows - 1) * (int)p.ldsa + KT) * 4;
        } else {
            const int nb = r - BM;
            s_off = nb * 128 < b_rows ? nb * (int)p.ldsb * 4 : kOOB;
            s_base = t.SB;
            s_bytes = ((b_rows - 1) / 128 * (int)p.ldsb + KT) * 4;
        }
    }

    // The copies of stage kt into slot kt & 1.  Every stage issues LOADS copies a
    // wave, past the end of k too (they write zeros), so that one count of
    // copies in flight holds throughout.
    auto copy = [&](int kt) {
        const unsigned at = smem_base + (kt & 1) * G::STAGE_BYTES;
        const int left = t.k - kt * G::BK;       // of k
        auto operand = [&](auto &s, bool k_rows, int rows, unsigned lds, int per_wave) {
            int bytes;
            if (k_rows) {
                const int ks = left < G::BK ? left : G::BK;
                // (whole chunks: one that holds any value of a row is mapped)
                bytes = left > 0 ? (ks - 1) * (int)s.ld + ((rows * 2 + 15) & ~15) : 0;
            } else {
                bytes = left > 0 ? (rows - 1) * (int)s.ld + (left < G::BK ? left : G::BK) * G::E : 0;
            }
            const i32x4 r = make_rsrc(s.base, bytes);
            s.each([&](int q) {
                int o = s.off[q];
                if (!k_rows) o = s.k_at[q] < left * G::E ? o : kOOB;
                dma16(r, lds + (wave * per_wave + q) * 1024, o);
            });
            s.base += k_rows ? G::BK * s.ld : 128;
        };
        operand(sa, G::A_K_ROWS, a_rows, at, G::A_PER_WAVE);
        operand(sb, G::B_K_ROWS, b_rows, at + G::A_BYTES, G::B_PER_WAVE);
        if constexpr (KIND == kFp8)
            dma4(make_rsrc(s_base, s_bytes), at + G::A_BYTES + G::B_BYTES + wave * 256,
                 left > 0 ? s_off + (s_off == kOOB ? 0 : kt * 4) : kOOB);
    };

    // Reads of fragment i of the wave's rows, or columns, from slot `slot`.
    auto read = [&](bool k_rows, const unsigned char *s, int rows, int first, u32x4 (&raw)[P::PIECES]) {
        if (!k_rows) {
            const int row = first + lrow;
            const unsigned char *q0 = s + row * 128;
            const int swz = (row >> 1) & 7;
#pragma unroll
            for (int q = 0; q < P::PIECES; ++q)
                raw[q] = *reinterpret_cast<const u32x4 *>(q0 + (((P::KG * q + lgrp) ^ swz) << 4));
        } else {
            const int rsub = (lane & 15) >> 2;
#pragma unroll
            for (int q = 0; q < P::PIECES; ++q) {
                // k = 8 (KG q + lgrp) + rsub (+ 4): four rows of one parity of k / 8
                const int k = 8 * (P::KG * q + lgrp) + rsub;
                const int c = first + (lrow & ~15) + 4 * (lane & 3);
                const unsigned char *q0 = s + k * rows * 2 + (((c >> 3) ^ swz_k(k)) << 4) + 8 * (lane & 1);
                const u16x4 lo = ds_read_tr16(reinterpret_cast<const unsigned short *>(q0));
                const u16x4 hi = ds_read_tr16(reinterpret_cast<const unsigned short *>(q0 + 4 * rows * 2));
                raw[q] = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        }
    };

    acc_t acc[G::TM][G::TN];
#pragma unroll
    for (int i = 0; i < G::TM; ++i)
#pragma unroll
        for (int j = 0; j < G::TN; ++j)
#pragma unroll
            for (int r = 0; r < P::NACC; ++r) acc[i][j][r] = 0.f;

    typename P::Frag b[G::TN], a[2];
    auto read_b = [&](int slot) {
        const unsigned char *s = smem + slot * G::STAGE_BYTES + G::A_BYTES;
#pragma unroll
        for (int j = 0; j < G::TN; ++j) {
            u32x4 raw[P::PIECES];
            read(G::B_K_ROWS, s, BN, wn * WN + j * MI, raw);
            b[j] = P::prepare(raw);
        }
    };
    auto read_a = [&](int slot, int i) {
        u32x4 raw[P::PIECES];
        read(G::A_K_ROWS, smem + slot * G::STAGE_BYTES, BM, wm * WM + i * MI, raw);
        a[i & 1] = P::prepare(raw);
    };
    // scales of the wave's rows in a stage, times that of its columns
    float scale[KIND == kFp8 ? G::TM : 1];
    auto read_scales = [&](int slot) {
        if constexpr (KIND == kFp8) {
            const float *s = reinterpret_cast<const float *>(smem + slot * G::STAGE_BYTES + G::A_BYTES + G::B_BYTES);
            const float c = s[BM + wn * WN / 128];
#pragma unroll
            for (int i = 0; i < G::TM; ++i) scale[i] = s[wm * WM + i * MI + lrow] * c;
        }
    };
    acc_t part[2][G::TN];      // e4m3: sums of a block of k, not yet scaled
    auto products = [&](int i) {
#pragma unroll
        for (int j = 0; j < G::TN; ++j) {
            if constexpr (KIND == kFp8) {
                acc_t z;
#pragma unroll
                for (int r = 0; r < P::NACC; ++r) z[r] = 0.f;
                part[i & 1][j] = P::mul(b[j], a[i & 1], z);
            } else {
                acc[i][j] = P::mul(b[j], a[i & 1], acc[i][j]);
            }
        }
    };
    auto add_scaled = [&](int i) {
        if constexpr (KIND == kFp8) {
#pragma unroll
            for (int j = 0; j < G::TN; ++j)
#pragma unroll
                for (int r = 0; r < P::NACC; ++r) acc[i][j][r] += part[i & 1][j][r] * scale[i];
        }
    };

    copy(0);
    copy(1);
    wait_vmcnt<G::LOADS>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read_scales(0);
    read_b(0);
    read_a(0, 0);
    for (int kt = 0; kt < KT; ++kt) {
        const int slot = kt & 1;
        each_index([&](auto I) {
            constexpr int i = I;
            read_a(slot, i + 1);
            products(i);
            if constexpr (i > 0) add_scaled(i - 1);
        }, std::make_integer_sequence<int, G::TM - 1>());
        // every read of the slot has returned, and stage kt + 1 has landed
        asm volatile("" ::: "memory");
        wait_vmcnt_and_lds<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        copy(kt + 2);
        products(G::TM - 1);
        add_scaled(G::TM - 2);
        add_scaled(G::TM - 1);
        read_scales(slot ^ 1);
        read_b(slot ^ 1);
        read_a(slot ^ 1, 0);
    }
    wait_vmcnt<0>();   // no copy may still be writing LDS when the workgroup ends

#pragma unroll
    for (int i = 0; i < G::TM; ++i) {
        const int m = wm * WM + i * MI + lrow;
        if (m >= t.m) continue;
        unsigned char *c = t.C + (int64_t)m * p.ldc * (p.out_bf16 ? 2 : 4);
#pragma unroll
        for (int j = 0; j < G::TN; ++j)
#pragma unroll
            for (int r = 0; r < P::NACC; r += 4) {
                const int n = wn * WN + j * MI + Bf16Mfma<MI>::row(lane, r);
                float v[4] = {acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]};
                write4(p, c, n, t.n - n, v);
            }
    }
}

template <Kind KIND, bool WIDE, int BM, int BN, int WM, int WN, int MI>
xtc_status launch_as(const GroupedArgs &a, hipStream_t s) {
    const int64_t tiles = tile_count<KIND>(a, BM, BN);
    if (tiles >= kMostGroups / 2) return XTC_ERR_TOO_LARGE;
    grouped_tile_kernel<KIND, WIDE, BM, BN, WM, WN, MI><<<(unsigned)tiles, (BM / WM) * (BN / WN) * 64, 0, s>>>(a);
    return hip_status(hipGetLastError());
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

// 16-byte aligned rows whose k is whole 16-byte chunks where they run along it,
// and strides that keep a tile's offsets within 31 bits.
template <Kind KIND>
bool tile_takes(const GroupedArgs &a) {
    const int64_t e = KIND == kFp8 ? 1 : 2, most = (int64_t(1) << 31) / 257;
    if (!aligned16(a.A) || !aligned16(a.B) || a.lda * e % 16 || a.ldb * e % 16 || a.stride_b * e % 16) return false;
    if (KIND != kWgrad && a.K * e % 16) return false;
    return a.lda * e < most && a.ldb * e < most && a.ldsa * 4 < most && a.ldsb * 4 < most;
}

template <Kind KIND>
xtc_status launch_tile(const GroupedArgs &a, hipStream_t s) {
    if constexpr (KIND == kFp8) {
        if (!a.out_bf16) return launch_as<KIND, true, 128, 128, 32, 64, 16>(a, s);
        if (tile_count<KIND>(a, 256, 256) >= 256) return launch_as<KIND, false, 256, 256, 128, 64, 16>(a, s);
        return launch_as<KIND, false, 128, 128, 64, 32, 16>(a, s);
    } else {
        if (tile_count<KIND>(a, 256, 256) >= 256) return launch_as<KIND, false, 256, 256, 128, 64, 32>(a, s);
        return launch_as<KIND, false, 128, 128, 64, 64, 32>(a, s);
    }
}

template bool tile_takes<kFp8>(const GroupedArgs &);
template bool tile_takes<kBf16N>(const GroupedArgs &);
template bool tile_takes<kBf16T>(const GroupedArgs &);
template bool tile_takes<kWgrad>(const GroupedArgs &);
template xtc_status launch_tile<kFp8>(const GroupedArgs &, hipStream_t);
template xtc_status launch_tile<kBf16N>(const GroupedArgs &, hipStream_t);
template xtc_status launch_tile<kBf16T>(const GroupedArgs &, hipStream_t);
template xtc_status launch_tile<kWgrad>(const GroupedArgs &, hipStream_t);

}  // namespace xtc
