// The grouped and 8-bit products on LDS-staged tiles: operands copied straight
// from memory into LDS (dma16), two to four stages of 128 or 64 bytes of k (128
// e4m3 values; 64 or 32 bf16 ones) in a ring.
//
// Rows at any address (ANY) go through registers instead, one stage further
// ahead.
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
#include "grouped_lds.h"
#include "unroll.h"

namespace xtc {
namespace {

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

template <Kind KIND, bool WIDE, int BM, int BN, int WM, int WN, int STAGES, int KB, bool ANY>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * 64, 2)
grouped_tile_kernel(GroupedArgs p) {
    typedef TileCfg<KIND, BM, BN, WM, WN, STAGES, KB> G;
    typedef Product<KIND, WIDE, KB> P;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[STAGES * G::STAGE_BYTES];

    const TileOrder<KIND, BM, BN> order(p);
    const int id = tile_id<KIND>(order.total);
    if (id < 0) return;
    const Tile t = make_tile<KIND>(p, order.at(id));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / G::NWN, wn = wave % G::NWN;
    const int lrow = lane % MI, lcol = lane / MI * 4;   // of a fragment's results: the row, the first of four columns
    const unsigned smem_base = lds_address(smem);
    const int KT = (t.k + G::BK - 1) / G::BK;

    typedef std::conditional_t<ANY, Carried<G::A_K_ROWS, BM, G::A_PER_WAVE, KB>, Source<G::A_K_ROWS, BM, G::A_PER_WAVE, KB>> FromA;
    typedef std::conditional_t<ANY, Carried<G::B_K_ROWS, BN, G::B_PER_WAVE, KB>, Source<G::B_K_ROWS, BN, G::B_PER_WAVE, KB>> FromB;
    FromA sa = [&]() __attribute__((always_inline)) {
        if constexpr (ANY) return FromA(t.A, t.lda, t.m);
        else return FromA(t.A, t.lda, t.m, wave, lane);
    }();
    FromB sb = [&]() __attribute__((always_inline)) {
        if constexpr (ANY) return FromB(t.B, t.ldb, t.n);
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
    // fetch(), and piece(q) writes them.
    i32x4 ra, rb;
    int left = 0, next = 0;      // of k from stage `next` on
    unsigned at = 0;
    unsigned char *to = smem;
    auto fetch = [&](int kt) __attribute__((always_inline)) {
        if constexpr (ANY) {
            left = t.k - kt * G::BK;
            sa.template fetch<G::E>(left, (KIND == kWgrad ? p.K : t.k) * G::E >= 16, wave, lane);
            sb.template fetch<G::E>(left, (G::B_K_ROWS ? p.N : t.k) * G::E >= 16, wave, lane);
            if constexpr (KIND == kFp8) s_value = left > 0 && s_off >= 0 ? s_base[s_off + kt] : 0.f;
        }
    };
    auto begin = [&](int kt, int slot) __attribute__((always_inline)) {
        if constexpr (ANY) {
            to = smem + slot * G::STAGE_BYTES;
        } else {
            at = smem_base + slot * G::STAGE_BYTES;
            left = t.k - kt * G::BK;
            next = kt;
            ra = sa.stage(left, G::E);
            rb = sb.stage(left, G::E);
        }
    };
    auto piece = [&](auto Q) __attribute__((always_inline)) {
        constexpr int q = Q;
        constexpr bool of_a = q < G::A_PER_WAVE, of_b = !of_a && q < G::A_PER_WAVE + G::B_PER_WAVE;
        constexpr int qb = q - G::A_PER_WAVE;
        if constexpr (ANY) {
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

    each_index([&](auto S) __attribute__((always_inline)) {
        fetch(S);
        begin(S, S);
        each_index([&](auto Q) __attribute__((always_inline)) { piece(Q); }, std::make_integer_sequence<int, G::LOADS>());
    }, std::make_integer_sequence<int, STAGES>());
    if constexpr (ANY) {
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
    for (int kt = 0; kt < KT; ++kt) {
        fetch(kt + STAGES);
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
            each_index([&](auto Q) __attribute__((always_inline)) { piece(std::integral_constant<int, q0 + Q>()); },
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
    }
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
                if (m < t.m) store_past_caches(reinterpret_cast<T *>(t.C) + m * p.ldc + n, v, t.n - n);
            }
            asm volatile("" ::: "memory");
        }, std::make_integer_sequence<int, (G::TM + PASS - 1) / PASS>());
    };
    if (p.out_bf16) store(__bf16());
    else store(0.f);
}

template <Kind KIND, bool WIDE, int BM, int BN, int WM, int WN, int STAGES, int KB, bool ANY = false>
xtc_status launch_as(const GroupedArgs &a, hipStream_t s) {
    const int64_t tiles = tile_count<KIND>(a, BM, BN);
    if (tiles >= kMostGroups / 2) return XTC_ERR_TOO_LARGE;
    grouped_tile_kernel<KIND, WIDE, BM, BN, WM, WN, STAGES, KB, ANY>
        <<<(unsigned)tiles, (BM / WM) * (BN / WN) * 64, 0, s>>>(a);
    return hip_status(hipGetLastError());
}

}  // namespace

// Measured: 8-bit products from 512^3 to 8192^3 and 8 to 4096 rows over 8 to 64
// groups, bf16 ones likewise up to 16384 rows over 16.
template <Kind KIND>
const Choice *tile_choices(bool wide, int *count) {
    if constexpr (KIND == kFp8) {
        static const Choice sums[] = {
            // Widening costs about what the products do: the squarer the waves' parts, the
            // less of it (4096 x 4096 x 4096: parts of 64x64 138 us, 64x32 178; tiles of
            // 256x128 of the first 137, but 1531 x 2000 x 4096 58 for 38).
            {128, 128, 2, 1.f, 1.3f, 2.f, 4, false, launch_as<KIND, true, 128, 128, 64, 64, 2, 128>},
            // (4138 x 944 x 896: 13.5 us, the tile above 19; 571 x 1264 x 768: 8.2 and 11)
            {128, 64, 2, .73f, .8f, 1.2f, 4, false, launch_as<KIND, true, 128, 64, 64, 32, 3, 128>},
        };
        static const Choice rounded[] = {
            {256, 256, 1, 1.75f, 1.75f, 1.75f, 9, false, launch_as<KIND, false, 256, 256, 128, 64, 2, 128>},
            {128, 128, 2, .88f, 1.1f, 1.34f, 4, false, launch_as<KIND, false, 128, 128, 64, 64, 2, 128>},
            {128, 128, 1, .75f, .75f, .75f, 4, true, launch_as<KIND, false, 128, 128, 64, 32, 4, 128>},
            {64, 128, 3, .72f, 1.1f, 1.4f, 2, false, launch_as<KIND, false, 64, 128, 64, 32, 2, 128>},
        };
        *count = wide ? 2 : 4;
        return wide ? sums : rounded;
    } else if constexpr (KIND == kWgrad) {
        static const Choice all[] = {
            // Four stages of 64 bytes, of the same LDS as two of 128, wait less for memory.
            {256, 256, 1, 1.1f, 1.1f, 1.1f, 12, false, launch_as<KIND, false, 256, 256, 128, 64, 4, 64>},
            {128, 256, 1, .81f, .81f, .81f, 7.9f, false, launch_as<KIND, false, 128, 256, 64, 64, 3, 128>},
            {128, 128, 2, .7f, .7f, 1.18f, 7.1f, false, launch_as<KIND, false, 128, 128, 64, 64, 2, 128>},
        };
        *count = 3;
        return all;
    } else {
        static const Choice all[] = {
            {256, 256, 1, 1.5f, 1.5f, 1.5f, 8, false, launch_as<KIND, false, 256, 256, 128, 64, 2, 128>},
            // Stages of 64 bytes let a CU hold two workgroups of four 64x128 waves, one of
            // which computes while the other begins or stores (16384 rows over 16 groups,
            // 1024 -> 2048: 87 us, the other tiles 103); rows along k then move half a
            // line at a time, so B's other layout gains less (96 us, 100).
            {128, 256, 2, KIND == kBf16N ? 1.2f : 1.3f, KIND == kBf16N ? 1.2f : 1.3f, KIND == kBf16N ? 2.f : 2.4f, KIND == kBf16N ? 6.f : 4.f, false,
             launch_as<KIND, false, 128, 256, 64, 128, 3, 64>},
            {128, 256, 1, .9f, .9f, .9f, 5, false, launch_as<KIND, false, 128, 256, 64, 64, 3, 128>},
            {128, 128, 2, .7f, 1.05f, 1.7f, 3, false, launch_as<KIND, false, 128, 128, 64, 64, 2, 128>},
            {64, 128, 3, .6f, 1.f, 1.5f, 2, false, launch_as<KIND, false, 64, 128, 64, 32, 2, 128>},
        };
        *count = 5;
        return all;
    }
}

template <Kind KIND>
xtc_status launch_any(const GroupedArgs &a, hipStream_t s) {
    // Slower than aligned rows: 4096 x 4095 x 4097 in e4m3 141 us, 4096^3 66; 7 x 4096 x 4095,
    // of which nothing splits the reduction, 43 us, 7 x 4096 x 4096 5.4.
    // 64 rows for few of them (KIND wgrad: 128 throughout).  (Widened parts of 64x64
    // would not fit the registers beside the values on their way.)
    const bool few = KIND != kWgrad && (a.ends ? a.T / a.G : a.T) <= 64;
    if constexpr (KIND == kFp8) {
        if (!a.out_bf16)
            return few ? launch_as<KIND, true, 64, 128, 64, 32, 2, 128, true>(a, s)
                       : launch_as<KIND, true, 128, 128, 64, 32, 2, 128, true>(a, s);
        return few ? launch_as<KIND, false, 64, 128, 64, 32, 2, 128, true>(a, s)
                   : launch_as<KIND, false, 128, 128, 64, 64, 2, 128, true>(a, s);
    } else if constexpr (KIND == kWgrad) {
        return launch_as<KIND, false, 128, 128, 64, 64, 2, 128, true>(a, s);
    } else {
        return few ? launch_as<KIND, false, 64, 128, 64, 32, 2, 128, true>(a, s)
                   : launch_as<KIND, false, 128, 128, 64, 64, 2, 128, true>(a, s);
    }
}

template xtc_status launch_any<kFp8>(const GroupedArgs &, hipStream_t);
template xtc_status launch_any<kBf16N>(const GroupedArgs &, hipStream_t);
template xtc_status launch_any<kBf16T>(const GroupedArgs &, hipStream_t);
template xtc_status launch_any<kWgrad>(const GroupedArgs &, hipStream_t);
template const Choice *tile_choices<kFp8>(bool, int *);
template const Choice *tile_choices<kBf16N>(bool, int *);
template const Choice *tile_choices<kBf16T>(bool, int *);
template const Choice *tile_choices<kWgrad>(bool, int *);

}  // namespace xtc
