// The grouped, 8-bit and linear products on LDS-staged tiles: operands copied straight
// from memory into LDS (dma16), two to four stages of 128 or 64 bytes of k (128
// e4m3 values; 64 or 32 bf16 ones) in a ring.
//
// Rows at any address (ANY) go through registers instead, one stage further
// ahead, or AHEAD of them.
//
// What bounds it.  Large products the matrix cores: the loop of a 256x256 tile
// runs at 1583 TFLOP/s in bf16 and 2562 in e4m3, with the first data's way and the
// results' (12 to 16 us a tile) 8192 x 8192 x 8192 in e4m3 at 2200.  Grouped ones the
// CUs' shares: 16384 rows over 16 uneven groups are a few rounds of tiles of
// which the last is partly empty (1024 to 2048: 84 us, 813 TFLOP/s).
//
// Loop.  A wave keeps the fragments of its columns (B) of a stage in registers
// and walks through its rows (A), two fragments ahead.  Before the products of
// the last two row fragments every read of the stage has returned: there
// stands the one barrier of a stage, with a wait for the next stage's copies.
// Those last products are taken column by column, and each column's fragment of
// the next stage is read as soon as the old one has been used; the copies of
// the stage STAGES ahead, into the slot just read, are spread between them.
// The sums of a block of e4m3 products are scaled LAG instructions after they were
// begun, beside the matrix cores.
#pragma once

#include "grouped_lds.h"
#include "linear.h"
#include "unroll.h"

namespace xtc {

template <Kind KIND, int BM, int BN, int WM, int WN, int STAGES, int KB>
struct TileCfg {
    static constexpr int E = KIND == kFp8 ? 1 : 2, BK = KB / E;
    static constexpr bool A_K_ROWS = KIND == kWgrad, B_K_ROWS = KIND == kWgrad || KIND == kBf16N;
    static constexpr int NWM = BM / WM, NWN = BN / WN, NWAVES = NWM * NWN, NT = NWAVES * 64;
    static constexpr int TM = WM / MI, TN = WN / MI;
    static constexpr int A_BYTES = BM * KB, B_BYTES = BN * KB;
    static constexpr int A_PER_WAVE = A_BYTES / 1024 / NWAVES, B_PER_WAVE = B_BYTES / 1024 / NWAVES;
    static constexpr int S_BYTES = KIND == kFp8 ? NWAVES * 256 : 0;   // scales: 64 values a wave
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + S_BYTES;
    static constexpr int LOADS = A_PER_WAVE + B_PER_WAVE + (KIND == kFp8 ? 1 : 0);
    static_assert(A_PER_WAVE * NWAVES * 1024 == A_BYTES && B_PER_WAVE * NWAVES * 1024 == B_BYTES,
                  "tiles must split into whole 1 KiB blocks per wave");
    static_assert(KIND != kFp8 || KB == 128, "a stage is a block of scales");
    static_assert(KIND != kFp8 || NWAVES > BM / 64, "a wave for B's scales");
    static_assert(128 % WN == 0, "the columns of a wave share a scale");
    static_assert(STAGES >= 2 && STAGES * STAGE_BYTES <= 160 * 1024, "LDS budget");
    static_assert((STAGES - 1) * LOADS < 64, "vmcnt range");
    static_assert(TM % 4 == 0, "the last two rows and the next stage's first two lie in four places");
};

template <Kind KIND, bool WIDE, int BM, int BN, int WM, int WN, int STAGES, int KB, bool ANY, int AHEAD, typename Args>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * 64, 2)
grouped_tile_kernel(Args p) {
    typedef TileCfg<KIND, BM, BN, WM, WN, STAGES, KB> G;
    typedef Product<KIND, WIDE, KB> P;
    constexpr bool LINEAR = std::is_same<Args, LinearArgs>::value;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[STAGES * G::STAGE_BYTES];

    const OrderOf<Args, KIND, BM, BN> order(p);
    const int id = tile_id<KIND == kWgrad && !LINEAR>(order.total);
    if (id < 0) return;
    const Place place = order.at(id);
    const Tile t = make_tile<KIND>(p, place);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / G::NWN, wn = wave % G::NWN;
    const int lrow = lane % MI, lcol = lane / MI * 4;   // of a fragment's results: the row, the first of four columns
    const unsigned smem_base = lds_address(smem);
    const int KT = (t.k + G::BK - 1) / G::BK;

    constexpr bool FAR = AHEAD > 1;
    static_assert(!FAR || (ANY && KIND != kFp8), "bf16 rows at any address");
    typedef std::conditional_t<ANY, Carried<G::A_K_ROWS, BM, G::A_PER_WAVE, KB>, Source<G::A_K_ROWS, BM, G::A_PER_WAVE, KB>> NearA;
    typedef std::conditional_t<ANY, Carried<G::B_K_ROWS, BN, G::B_PER_WAVE, KB>, Source<G::B_K_ROWS, BN, G::B_PER_WAVE, KB>> NearB;
    typedef std::conditional_t<FAR, CarriedAhead<G::A_K_ROWS, BM, G::A_PER_WAVE, KB, AHEAD>, NearA> FromA;
    typedef std::conditional_t<FAR, CarriedAhead<G::B_K_ROWS, BN, G::B_PER_WAVE, KB, AHEAD>, NearB> FromB;
    FromA sa = [&]() __attribute__((always_inline)) {
        if constexpr (FAR) return FromA(t.A, t.lda, t.m, t.k, wave, lane);
        else if constexpr (ANY) return FromA(t.A, t.lda, t.m);
        else return FromA(t.A, t.lda, t.m, wave, lane);
    }();
    FromB sb = [&]() __attribute__((always_inline)) {
        if constexpr (FAR) return FromB(t.B, t.ldb, t.n, t.k, wave, lane);
        else if constexpr (ANY) return FromB(t.B, t.ldb, t.n);
        else return FromB(t.B, t.ldb, t.n, wave, lane);
    }();
    // this lane's scale of a stage: rows of A, then the blocks of B's columns
    const float *s_base = t.SA;
    int64_t s_off = -1;          // in values; none: -1
    int s_bytes = 0;
    float s_value = 0.f;
    if constexpr (KIND == kFp8) {
        const int r = wave * 64 + lane;
        if (wave < BM / 64) {
            if (r < sa.rows) s_off = r * p.ldsa;
            s_bytes = ((sa.rows - 1) * (int)p.ldsa + KT) * 4;
        } else {
            const int nb = r - BM;
            if (nb * 128 < sb.rows) s_off = nb * p.ldsb;
            s_base = t.SB;
            s_bytes = ((sb.rows - 1) / 128 * (int)p.ldsb + KT) * 4;
        }
    }

    // The copies of stage kt into a slot: LOADS a wave, past the end of k too (they
    // write zeros), so that one count of copies in flight holds throughout.
    // begin() settles the stage, piece(q) issues one of them.  Of rows at any
    // address (ANY) the stage's values are on their way to registers since
    // fetch(), and piece(q) writes them, from the set of registers SET where there are several.
    i32x4 ra, rb;
    int left = 0, next = 0;      // of k from stage `next` on
    unsigned at = 0;
    unsigned char *to = smem;
    auto fetch = [&](int kt, auto SET) __attribute__((always_inline)) {
        if constexpr (FAR) {
            sa.template fetch<SET()>(wave, lane);
            sb.template fetch<SET()>(wave, lane);
        } else if constexpr (ANY) {
            left = t.k - kt * G::BK;
            sa.template fetch<G::E>(left, (KIND == kWgrad ? p.K : t.k) * G::E >= 16, wave, lane);
            sb.template fetch<G::E>(left, (G::B_K_ROWS ? p.N : t.k) * G::E >= 16, wave, lane);
            if constexpr (KIND == kFp8) s_value = left > 0 && s_off >= 0 ? s_base[s_off + kt] : 0.f;
        }
    };
    auto begin = [&](int kt, int slot) __attribute__((always_inline)) {
        if constexpr (ANY) {
            to = smem + slot * G::STAGE_BYTES;
            if constexpr (FAR) left = t.k - kt * G::BK;
        } else {
            at = smem_base + slot * G::STAGE_BYTES;
            left = t.k - kt * G::BK;
            next = kt;
            ra = sa.stage(left, G::E);
            rb = sb.stage(left, G::E);
        }
    };
    auto piece = [&](auto Q, auto SET) __attribute__((always_inline)) {
        constexpr int q = Q;
        constexpr bool of_a = q < G::A_PER_WAVE, of_b = !of_a && q < G::A_PER_WAVE + G::B_PER_WAVE;
        constexpr int qb = q - G::A_PER_WAVE;
        if constexpr (FAR) {
            if constexpr (of_a) sa.template store<SET()>(to + wave * G::A_PER_WAVE * 1024, q, left, wave, lane);
            else sb.template store<SET()>(to + G::A_BYTES + wave * G::B_PER_WAVE * 1024, qb, left, wave, lane);
        } else if constexpr (ANY) {
            if constexpr (of_a) sa.store(to + wave * G::A_PER_WAVE * 1024, q, lane);
            else if constexpr (of_b) sb.store(to + G::A_BYTES + wave * G::B_PER_WAVE * 1024, qb, lane);
            else reinterpret_cast<float *>(to + G::A_BYTES + G::B_BYTES)[wave * 64 + lane] = s_value;
        } else {
            if constexpr (of_a)
                dma16(ra, at + (wave * G::A_PER_WAVE + q) * 1024, sa.offset(q, left, G::E));
            else if constexpr (of_b)
                dma16(rb, at + G::A_BYTES + (wave * G::B_PER_WAVE + qb) * 1024, sb.offset(qb, left, G::E));
            else
                dma4(make_rsrc(s_base, s_bytes), at + G::A_BYTES + G::B_BYTES + wave * 256,
                     left > 0 && s_off >= 0 ? ((int)s_off + next) * 4 : kOOB);
        }
    };

    f32x4 acc[G::TM][G::TN] = {};

    // Fragments: of A four rows as read and, where they have to be widened first, two
    // widened; of B all columns, and two as read.  What is read is widened some
    // products later, so that no product waits for either (818 x 3552 x 4608 widened as
    // soon as read 43 us, so 39; vector instructions set singly between the matrix
    // ones, or two products' chains in turn, gave nothing more).
    typename P::Frag b[G::TN], wide[2];
    u32x4 a[4][P::PIECES], b_read[2][P::PIECES];
    auto read_b = [&](int slot, int j) __attribute__((always_inline)) {
        read_fragment<G::B_K_ROWS, BN, KB>(smem + slot * G::STAGE_BYTES + G::A_BYTES, wn * WN + j * MI, lane, b_read[j & 1]);
    };
    auto prepare_b = [&](int j) __attribute__((always_inline)) { b[j] = P::prepare(b_read[j & 1]); };
    auto read_a = [&](int slot, int i) __attribute__((always_inline)) {
        read_fragment<G::A_K_ROWS, BM, KB>(smem + slot * G::STAGE_BYTES, wm * WM + i * MI, lane, a[i & 3]);
    };
    auto widen_a = [&](int i, int q) __attribute__((always_inline)) {
        if constexpr (WIDE) P::prepare(wide[i & 1], a[i & 3], q);
    };
    auto row_fragment = [&](int i) __attribute__((always_inline)) {
        if constexpr (WIDE) return wide[i & 1];
        else return P::prepare(a[i & 3]);
    };
    // scales of the wave's rows in a stage, times that of its columns
    float scale[2][KIND == kFp8 ? G::TM : 1];
    auto read_scales = [&](int slot, int set) __attribute__((always_inline)) {
        if constexpr (KIND == kFp8) {
            const float *s = reinterpret_cast<const float *>(smem + slot * G::STAGE_BYTES + G::A_BYTES + G::B_BYTES);
            const float c = s[BM + wn * WN / 128];
#pragma unroll
            for (int i = 0; i < G::TM; ++i) scale[set][i] = s[wm * WM + i * MI + lrow] * c;
        }
    };
    // Step n of a stage's products: rows of fragments one after the other, the
    // last two column by column.
    constexpr int STEPS = G::TM * G::TN, HEAD = STEPS - 2 * G::TN;
    constexpr int LAG = KIND == kFp8 ? 4 : 0;
    f32x4 part[LAG + 1];         // e4m3: sums of a block of k, not yet scaled
    auto row_of = [](int n) { return n < HEAD ? n / G::TN : G::TM - 2 + (n - HEAD) % 2; };
    auto column_of = [](int n) { return n < HEAD ? n % G::TN : (n - HEAD) / 2; };
    auto product = [&](auto N) __attribute__((always_inline)) {
        constexpr int n = N, i = row_of(n), j = column_of(n);
        if constexpr (KIND == kFp8) {
            const f32x4 z = {0.f, 0.f, 0.f, 0.f};
            part[n % (LAG + 1)] = P::mul(b[j], row_fragment(i), z);
        } else {
            acc[i][j] = P::mul(b[j], row_fragment(i), acc[i][j]);
        }
    };
    auto add_scaled = [&](auto N) __attribute__((always_inline)) {
        constexpr int n = N, i = row_of(n), j = column_of(n);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[i][j][r] += part[n % (LAG + 1)][r] * scale[0][i];
    };

    // (AHEAD sets of registers: stage n is in the set n % AHEAD, and fetched when the one before in it has been stored)
    if constexpr (FAR)
        each_index([&](auto S) __attribute__((always_inline)) {
            fetch(S, S);
            __builtin_amdgcn_sched_barrier(0);
        }, std::make_integer_sequence<int, AHEAD>());
    each_index([&](auto S) __attribute__((always_inline)) {
        constexpr std::integral_constant<int, S() % AHEAD> SET;
        if constexpr (!FAR) fetch(S, SET);
        begin(S, S);
        each_index([&](auto Q) __attribute__((always_inline)) { piece(Q, SET); }, std::make_integer_sequence<int, G::LOADS>());
        if constexpr (FAR && S() + 1 < STAGES) {
            __builtin_amdgcn_sched_barrier(0);
            fetch(S + AHEAD, SET);
            __builtin_amdgcn_sched_barrier(0);
        }
    }, std::make_integer_sequence<int, STAGES>());
    if constexpr (FAR) {
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
    } else if constexpr (ANY) {
        __syncthreads();
    } else {
        wait_vmcnt<(STAGES - 1) * G::LOADS>();
        __builtin_amdgcn_s_barrier();
    }
    asm volatile("" ::: "memory");
    read_scales(0, 0);
#pragma unroll
    for (int j = 0; j < G::TN; ++j) {
        read_b(0, j);
        prepare_b(j);
    }
    read_a(0, 0);
    read_a(0, 1);
#pragma unroll
    for (int q = 0; q < P::PIECES; ++q) widen_a(0, q);
    int slot = 0;
    auto stage = [&](int kt, auto TURN) __attribute__((always_inline)) {
        constexpr std::integral_constant<int, (TURN() + STAGES) % AHEAD> SET;                  // of stage kt + STAGES
        constexpr std::integral_constant<int, (TURN() + STAGES + AHEAD - 1) % AHEAD> FREE;     // of the one before
        fetch(kt + STAGES + AHEAD - 1, FREE);
        each_index([&](auto N) __attribute__((always_inline)) {
            constexpr int n = N;
            if constexpr (n % G::TN == 0) read_a(slot, n / G::TN + 2);
            product(N);
            if constexpr (KIND == kFp8 && n >= LAG) add_scaled(std::integral_constant<int, n - LAG>());
#pragma unroll
            for (int q = 0; q < P::PIECES; ++q)     // the next row, piece by piece
                if (n % G::TN == (q + 1 < G::TN ? q + 1 : G::TN - 1)) widen_a(n / G::TN + 1, q);
            __builtin_amdgcn_sched_barrier(0);
        }, std::make_integer_sequence<int, HEAD>());
        // every read of the slot has returned, and stage kt + 1 has landed
        asm volatile("" ::: "memory");
        if constexpr (ANY) __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): also what this wave wrote for stage kt + 1
        else wait_vmcnt_and_lds<(STAGES - 2) * G::LOADS>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int after = slot + 1 < STAGES ? slot + 1 : 0;
        begin(kt + STAGES, slot);
        read_scales(after, 1);
        read_a(after, 0);
        read_a(after, 1);
        __builtin_amdgcn_sched_barrier(0);
        each_index([&](auto M) __attribute__((always_inline)) {
            constexpr int m = M, n = HEAD + m, q0 = m * G::LOADS / (2 * G::TN), q1 = (m + 1) * G::LOADS / (2 * G::TN);
            if constexpr (WIDE && m % 2 == 0) read_b(after, m / 2);
            product(std::integral_constant<int, n>());
            if constexpr (KIND == kFp8 && n >= LAG) add_scaled(std::integral_constant<int, n - LAG>());
            if constexpr (WIDE) {
                if constexpr (m % 2 == 1 && m > 1) prepare_b(m / 2 - 1);
                if constexpr (m == 2 * G::TN - 1) prepare_b(m / 2);
#pragma unroll
                for (int q = 0; q < P::PIECES; ++q) {
                    if constexpr (m == 0) widen_a(G::TM - 1, q);
                    if constexpr (m == 2 * G::TN - 1) widen_a(0, q);
                }
            } else if constexpr (m % 2 == 1) {
                read_b(after, m / 2);
                prepare_b(m / 2);
            }
            each_index([&](auto Q) __attribute__((always_inline)) { piece(std::integral_constant<int, q0 + Q>(), SET); },
                       std::make_integer_sequence<int, q1 - q0>());
            __builtin_amdgcn_sched_barrier(0);
        }, std::make_integer_sequence<int, 2 * G::TN>());
        if constexpr (KIND == kFp8) {
            each_index([&](auto N) __attribute__((always_inline)) { add_scaled(std::integral_constant<int, STEPS - LAG + N>()); },
                       std::make_integer_sequence<int, LAG>());
#pragma unroll
            for (int i = 0; i < G::TM; ++i) scale[0][i] = scale[1][i];
        }
        slot = after;
    };
    // AHEAD stages a trip, for constant sets, and the rest behind the loop: another way out of it would pass its head
    // for the compiler, which would then have it wait for loads that only the long way has taken.
    int done = 0;
    for (; done + AHEAD <= KT; done += AHEAD)
        each_index([&](auto TURN) __attribute__((always_inline)) { stage(done + TURN(), TURN); }, std::make_integer_sequence<int, AHEAD>());
    each_index([&](auto TURN) __attribute__((always_inline)) {
        if (done + TURN() < KT) stage(done + TURN(), TURN);
    }, std::make_integer_sequence<int, AHEAD - 1>());
    if constexpr (!ANY) wait_vmcnt<0>();   // no copy may still be writing LDS when the workgroup ends

    if (p.relu) {
#pragma unroll
        for (int i = 0; i < G::TM; ++i)
#pragma unroll
            for (int j = 0; j < G::TN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][r] = acc[i][j][r] < 0.f ? 0.f : acc[i][j][r];
    }
    // Results leave as whole lines past the caches, which the operands then keep, by way
    // of a part of LDS of the wave's own.  16384 rows over 16 groups, 1024 to 2048, bf16:
    // 98 us with ordinary stores of four columns a lane, 104 with those past the caches,
    // half lines each, and 85 this way; e4m3 8192 x 8192 x 8192: 526 and 504.  fp32 results
    // straight from the registers are half lines too, of which 1.4 times the bytes reach
    // memory: weights' gradients of the same rows 105 us, so 95; of 64 groups of 64 rows,
    // 1024 x 1024, 80 and 58.
    int64_t ldc = p.ldc;
    if constexpr (LINEAR) ldc = p.splits > 1 ? p.N : p.ldc;
    __syncthreads();
    auto store = [&](auto ZERO) __attribute__((always_inline)) {
        typedef decltype(ZERO) T;
        constexpr int PART = STAGES * G::STAGE_BYTES / G::NWAVES / 16 * 16;
        constexpr int PITCH = WN * (int)sizeof(T) + 16;                             // (rows a few banks apart)
        constexpr int FIT = PART / PITCH / MI, PASS = FIT < G::TM ? FIT : G::TM;    // fragments' rows at once
        static_assert(PASS > 0, "a fragment's rows fit");
        constexpr int EACH = 16 / (int)sizeof(T), LANES = WN / EACH;                // columns a lane, lanes a row
        unsigned char *own = smem + wave * PART;
        each_index([&](auto I0) __attribute__((always_inline)) {
            constexpr int i0 = I0 * PASS, i1 = i0 + PASS < G::TM ? i0 + PASS : G::TM;
            each_index([&](auto I) __attribute__((always_inline)) {
                constexpr int i = i0 + I;
#pragma unroll
                for (int j = 0; j < G::TN; ++j) {
                    T v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = (T)acc[i][j][e];
                    void *to = own + (I * MI + lrow) * PITCH + (j * MI + lcol) * (int)sizeof(T);
                    __builtin_memcpy(__builtin_assume_aligned(to, sizeof(v)), v, sizeof(v));
                }
            }, std::make_integer_sequence<int, i1 - i0>());
            asm volatile("" ::: "memory");
            const int n = wn * WN + lane % LANES * EACH;
#pragma unroll
            for (int q = 0; q < (i1 - i0) * MI * LANES / 64; ++q) {
                const int row = q * (64 / LANES) + lane / LANES, m = wm * WM + i0 * MI + row;
                T v[EACH];
                __builtin_memcpy(v, __builtin_assume_aligned(own + row * PITCH + lane % LANES * 16, 16), 16);
                if (m < t.m) store_past_caches(reinterpret_cast<T *>(t.C) + m * ldc + n, v, t.n - n);
            }
            asm volatile("" ::: "memory");
        }, std::make_integer_sequence<int, (G::TM + PASS - 1) / PASS>());
    };
    if constexpr (LINEAR) {
        // the sums themselves pass LDS, in fp32; the epilogue stands behind it, at whole 16 bytes of results
        auto finish = [&](auto ZERO) __attribute__((always_inline)) {
            typedef decltype(ZERO) T;
            constexpr int PART = STAGES * G::STAGE_BYTES / G::NWAVES / 16 * 16;
            constexpr int PITCH = WN * 4 + 16;
            constexpr int FIT = PART / PITCH / MI, PASS = FIT < G::TM ? FIT : G::TM;
            static_assert(PASS > 0, "a fragment's rows fit");
            constexpr int EACH = 16 / (int)sizeof(T), LANES = WN / EACH;
            unsigned char *own = smem + wave * PART;
            const int n = wn * WN + lane % LANES * EACH, row0 = KIND == kWgrad ? place.m0 : place.row0;
            const Epilogue<T, EACH> e(p, row0, place.n0 + n);
            each_index([&](auto I0) __attribute__((always_inline)) {
                constexpr int i0 = I0 * PASS, i1 = i0 + PASS < G::TM ? i0 + PASS : G::TM;
                each_index([&](auto I) __attribute__((always_inline)) {
                    constexpr int i = i0 + I;
#pragma unroll
                    for (int j = 0; j < G::TN; ++j) {
                        void *to = own + (I * MI + lrow) * PITCH + (j * MI + lcol) * 4;
                        __builtin_memcpy(__builtin_assume_aligned(to, 16), &acc[i][j], 16);
                    }
                }, std::make_integer_sequence<int, i1 - i0>());
                asm volatile("" ::: "memory");
                constexpr int STEPS_OUT = (i1 - i0) * MI * LANES / 64;
                auto row_at = [&](int q) { return q * (64 / LANES) + lane / LANES; };
                auto m_at = [&](int q) { return wm * WM + i0 * MI + row_at(q); };
                auto there = [&](int q) { return q < STEPS_OUT && m_at(q) < t.m; };
                auto r = e.residual(m_at(0), there(0));
#pragma unroll 1
                for (int q = 0; q < STEPS_OUT; ++q) {
                    const auto next = e.residual(m_at(q + 1), there(q + 1));
                    float v[EACH];
                    __builtin_memcpy(v, __builtin_assume_aligned(own + row_at(q) * PITCH + lane % LANES * EACH * 4, 16), sizeof(v));
                    if (there(q)) e.write(m_at(q), v, r);
                    r = next;
                }
                asm volatile("" ::: "memory");
            }, std::make_integer_sequence<int, (G::TM + PASS - 1) / PASS>());
        };
        if (p.splits > 1) store(0.f);
        else if (p.out_bf16) finish(__bf16());
        else finish(0.f);
    } else {
        if (p.out_bf16) store(__bf16());
        else store(0.f);
    }
}

// (a LinearArgs is launched by its base: the rules of choice are for both)
template <Kind KIND, bool WIDE, int BM, int BN, int WM, int WN, int STAGES, int KB, bool ANY = false, typename Args = GroupedArgs, int AHEAD = 1>
xtc_status launch_tiles(const GroupedArgs &base, hipStream_t s) {
    const Args &a = static_cast<const Args &>(base);
    const int64_t tiles = tile_count<KIND>(a, BM, BN);
    if (tiles >= kMostGroups / 2) return XTC_ERR_TOO_LARGE;
    grouped_tile_kernel<KIND, WIDE, BM, BN, WM, WN, STAGES, KB, ANY, AHEAD, Args>
        <<<(unsigned)tiles, (BM / WM) * (BN / WN) * 64, 0, s>>>(a);
    return hip_status(hipGetLastError());
}

}  // namespace xtc
