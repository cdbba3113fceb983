// The grouped and 8-bit products of few rows: what they cost is the reading of B,
// so every workgroup takes a narrow strip of B's columns and its waves share
// the reduction, wave w reducing the stages w, w + NW, ... through an LDS ring
// of its own.  No barrier stands before the end, where the waves' sums are
// added in their order; a CU keeps NW x STAGES stages in flight.
//
// Bound by memory: 7 x 4096 x 4096 in e4m3 5.4 us, of which about 2 are a launch's own
// (weights at 3.1 TB/s over the whole); 100 rows over 32 groups, 4096 to 1024, in
// 26.5 us at 5.1 TB/s, as fast as a copy.
#include "grouped_lds.h"

namespace xtc {
namespace {

template <Kind KIND, int BM, int BN, int NW, int STAGES>
struct StreamCfg {
    static constexpr int E = KIND == kFp8 ? 1 : 2, BK = 128 / E;
    static constexpr bool B_K_ROWS = KIND == kBf16N;
    static constexpr int TM = BM / MI, TN = BN / MI;
    static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, S_BYTES = KIND == kFp8 ? 512 : 0;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + S_BYTES;
    static constexpr int LOADS = (A_BYTES + B_BYTES) / 1024 + (KIND == kFp8 ? 2 : 0);
    static constexpr int RING = NW * STAGES * STAGE_BYTES, SUMS = NW * TM * TN * 1024;
    static constexpr int LDS = RING > SUMS ? RING : SUMS;
    static_assert(KIND != kWgrad && BM <= 64 && 128 % BN == 0, "a lane a row's scale, and one for the strip");
    static_assert((STAGES - 1) * LOADS < 64, "vmcnt range");
    static_assert(LDS <= 160 * 1024, "LDS budget");
};

template <Kind KIND, bool WIDE, int BM, int BN, int NW, int STAGES>
__global__ void __launch_bounds__(NW * 64) grouped_stream_kernel(GroupedArgs p) {
    typedef StreamCfg<KIND, BM, BN, NW, STAGES> G;
    typedef Product<KIND, WIDE> P;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[G::LDS];

    const TileOrder<KIND, BM, BN> order(p);
    const int id = tile_id<KIND>(order.total);
    if (id < 0) return;
    const Tile t = make_tile<KIND>(p, order.at(id));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g4 = lane >> 4;
    const int KT = (t.k + G::BK - 1) / G::BK;
    unsigned char *ring = smem + wave * STAGES * G::STAGE_BYTES;
    const unsigned ring_at = lds_address(ring);

    // from this wave's first stage on
    Source<false, BM, G::A_BYTES / 1024> sa(t.A + wave * 128, t.lda, t.m, 0, lane);
    Source<G::B_K_ROWS, BN, G::B_BYTES / 1024> sb(t.B + (G::B_K_ROWS ? wave * G::BK * t.ldb : wave * 128), t.ldb, t.n, 0, lane);
    auto copy = [&](int kt, int slot) {
        const unsigned at = ring_at + slot * G::STAGE_BYTES;
        const int left = t.k - kt * G::BK;
        const i32x4 ra = sa.stage(left, G::E, NW), rb = sb.stage(left, G::E, NW);
#pragma unroll
        for (int q = 0; q < G::A_BYTES / 1024; ++q) dma16(ra, at + q * 1024, sa.offset(q, left, G::E));
#pragma unroll
        for (int q = 0; q < G::B_BYTES / 1024; ++q) dma16(rb, at + G::A_BYTES + q * 1024, sb.offset(q, left, G::E));
        if constexpr (KIND == kFp8) {
            const unsigned s = at + G::A_BYTES + G::B_BYTES;
            dma4(make_rsrc(t.SA, ((sa.rows - 1) * (int)p.ldsa + KT) * 4), s,
                 left > 0 && lane < sa.rows ? (lane * (int)p.ldsa + kt) * 4 : kOOB);
            dma4(make_rsrc(t.SB, KT * 4), s + 256, left > 0 && lane == 0 ? kt * 4 : kOOB);
        }
    };

    f32x4 acc[G::TM][G::TN] = {};
#pragma unroll
    for (int s = 0; s < STAGES; ++s) copy(wave + s * NW, s);
    int slot = 0;
    for (int kt = wave; kt < KT; kt += NW) {
        wait_vmcnt<(STAGES - 1) * G::LOADS>();
        asm volatile("" ::: "memory");
        const unsigned char *s = ring + slot * G::STAGE_BYTES;
        u32x4 ra[G::TM][P::PIECES], rb[G::TN][P::PIECES];
        float scale[G::TM];
#pragma unroll
        for (int i = 0; i < G::TM; ++i) read_fragment<false, BM, 128>(s, i * 16, lane, ra[i]);
#pragma unroll
        for (int j = 0; j < G::TN; ++j) read_fragment<G::B_K_ROWS, BN, 128>(s + G::A_BYTES, j * 16, lane, rb[j]);
        if constexpr (KIND == kFp8) {
            const float *c = reinterpret_cast<const float *>(s + G::A_BYTES + G::B_BYTES);
#pragma unroll
            for (int i = 0; i < G::TM; ++i) scale[i] = c[i * 16 + l16] * c[64];
        }
        // the slot's reads have returned before copies enter it again
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
        asm volatile("" ::: "memory");
        copy(kt + STAGES * NW, slot);
        typename P::Frag a[G::TM], b[G::TN];
#pragma unroll
        for (int i = 0; i < G::TM; ++i) a[i] = P::prepare(ra[i]);
#pragma unroll
        for (int j = 0; j < G::TN; ++j) b[j] = P::prepare(rb[j]);
#pragma unroll
        for (int i = 0; i < G::TM; ++i)
#pragma unroll
            for (int j = 0; j < G::TN; ++j) {
                if constexpr (KIND == kFp8) {
                    const f32x4 z = {0.f, 0.f, 0.f, 0.f}, d = P::mul(b[j], a[i], z);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] += d[r] * scale[i];
                } else {
                    acc[i][j] = P::mul(b[j], a[i], acc[i][j]);
                }
            }
        slot = slot + 1 < STAGES ? slot + 1 : 0;
    }
    wait_vmcnt<0>();   // no copy may still be writing LDS when the sums go there
    __syncthreads();
    f32x4 *sums = reinterpret_cast<f32x4 *>(smem);
#pragma unroll
    for (int i = 0; i < G::TM; ++i)
#pragma unroll
        for (int j = 0; j < G::TN; ++j) sums[((i * G::TN + j) * NW + wave) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int f = wave; f < G::TM * G::TN; f += NW) {
        f32x4 v = sums[f * NW * 64 + lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) v += sums[(f * NW + w) * 64 + lane];
        const int m = f / G::TN * 16 + l16, n = f % G::TN * 16 + 4 * g4;
        if (m < t.m) {
            float o[4] = {relu_if(p.relu, v[0]), relu_if(p.relu, v[1]), relu_if(p.relu, v[2]), relu_if(p.relu, v[3])};
            write4(p, t.C + (int64_t)m * p.ldc * (p.out_bf16 ? 2 : 4), n, t.n - n, o);
        }
    }
}

template <Kind KIND, bool WIDE, int BM, int BN, int NW, int STAGES>
xtc_status launch_as(const GroupedArgs &a, hipStream_t s) {
    const int64_t tiles = tile_count<KIND>(a, BM, BN);
    if (tiles >= kMostGroups / 4) return XTC_ERR_TOO_LARGE;
    grouped_stream_kernel<KIND, WIDE, BM, BN, NW, STAGES><<<(unsigned)tiles, NW * 64, 0, s>>>(a);
    return hip_status(hipGetLastError());
}

}  // namespace

// Measured as the tiles' (`one` and `full` hold four waves' or eight's share of k).
template <Kind KIND>
const Choice *stream_choices(bool wide, int *count) {
    if constexpr (KIND == kFp8) {
        static const Choice sums[] = {
            {16, 16, 2, .065f, .065f, .13f, 1, true, launch_as<KIND, true, 16, 16, 4, 3>},
            {32, 16, 3, .08f, .08f, .22f, 2.2f, true, launch_as<KIND, true, 32, 16, 4, 2>},
            {32, 32, 2, .17f, .17f, .33f, 2.8f, false, launch_as<KIND, true, 32, 32, 4, 2>},
            {32, 64, 1, .2f, .35f, .2f, 3, false, launch_as<KIND, true, 32, 64, 4, 2>},
            {64, 64, 1, .3f, .41f, .3f, 3, false, launch_as<KIND, true, 64, 64, 4, 2>},
        };
        static const Choice rounded[] = {
            {16, 16, 2, .06f, .06f, .125f, 1, true, launch_as<KIND, false, 16, 16, 4, 3>},
            {32, 16, 3, .07f, .07f, .2f, 2.2f, true, launch_as<KIND, false, 32, 16, 4, 2>},
            {32, 32, 2, .15f, .15f, .3f, 2.8f, false, launch_as<KIND, false, 32, 32, 4, 2>},
            {32, 64, 1, .15f, .34f, .15f, 3, false, launch_as<KIND, false, 32, 64, 4, 2>},
            {64, 64, 1, .22f, .39f, .22f, 2.5f, false, launch_as<KIND, false, 64, 64, 4, 2>},
        };
        *count = 5;
        return wide ? sums : rounded;
    } else {
        static const Choice all[] = {{32, 64, 1, .28f, .35f, .28f, 2.5f, false, launch_as<KIND, false, 32, 64, 4, 2>}};
        *count = 1;
        return all;
    }
}

template const Choice *stream_choices<kFp8>(bool, int *);
template const Choice *stream_choices<kBf16N>(bool, int *);
template const Choice *stream_choices<kBf16T>(bool, int *);

}  // namespace xtc
