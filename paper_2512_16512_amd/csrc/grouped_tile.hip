// The grouped and 8-bit products on LDS-staged tiles: the compiled kernels.
#include "grouped_tile.h"

namespace xtc {

// Measured: 8-bit products from 512^3 to 8192^3 and 8 to 4096 rows over 8 to 64
// groups, bf16 ones likewise up to 16384 rows over 16.
template <Kind KIND>
const Choice *tile_choices(bool wide, int *count) {
    if constexpr (KIND == kFp8) {
        static const Choice sums[] = {
            // Widening costs about what the products do: the squarer the waves' parts, the
            // less of it (4096 x 4096 x 4096: parts of 64x64 138 us, 64x32 178; tiles of
            // 256x128 of the first 137, but 1531 x 2000 x 4096 58 for 38).
            {128, 128, 2, 1.f, 1.3f, 2.f, 4, false, launch_tiles<KIND, true, 128, 128, 64, 64, 2, 128>},
            // (4138 x 944 x 896: 13.5 us, the tile above 19; 571 x 1264 x 768: 8.2 and 11)
            {128, 64, 2, .73f, .8f, 1.2f, 4, false, launch_tiles<KIND, true, 128, 64, 64, 32, 3, 128>},
        };
        static const Choice rounded[] = {
            {256, 256, 1, 1.75f, 1.75f, 1.75f, 9, false, launch_tiles<KIND, false, 256, 256, 128, 64, 2, 128>},
            {128, 128, 2, .88f, 1.1f, 1.34f, 4, false, launch_tiles<KIND, false, 128, 128, 64, 64, 2, 128>},
            {128, 128, 1, .75f, .75f, .75f, 4, true, launch_tiles<KIND, false, 128, 128, 64, 32, 4, 128>},
            {64, 128, 3, .72f, 1.1f, 1.4f, 2, false, launch_tiles<KIND, false, 64, 128, 64, 32, 2, 128>},
        };
        *count = wide ? 2 : 4;
        return wide ? sums : rounded;
    } else if constexpr (KIND == kWgrad) {
        static const Choice all[] = {
            // Four stages of 64 bytes, of the same LDS as two of 128, wait less for memory.
            {256, 256, 1, 1.1f, 1.1f, 1.1f, 12, false, launch_tiles<KIND, false, 256, 256, 128, 64, 4, 64>},
            {128, 256, 1, .81f, .81f, .81f, 7.9f, false, launch_tiles<KIND, false, 128, 256, 64, 64, 3, 128>},
            {128, 128, 2, .7f, .7f, 1.18f, 7.1f, false, launch_tiles<KIND, false, 128, 128, 64, 64, 2, 128>},
        };
        *count = 3;
        return all;
    } else {
        static const Choice all[] = {
            {256, 256, 1, 1.5f, 1.5f, 1.5f, 8, false, launch_tiles<KIND, false, 256, 256, 128, 64, 2, 128>},
            // Stages of 64 bytes let a CU hold two workgroups of four 64x128 waves, one of
            // which computes while the other begins or stores (16384 rows over 16 groups,
            // 1024 -> 2048: 87 us, the other tiles 103); rows along k then move half a
            // line at a time, so B's other layout gains less (96 us, 100).
            {128, 256, 2, KIND == kBf16N ? 1.2f : 1.3f, KIND == kBf16N ? 1.2f : 1.3f, KIND == kBf16N ? 2.f : 2.4f, KIND == kBf16N ? 6.f : 4.f, false,
             launch_tiles<KIND, false, 128, 256, 64, 128, 3, 64>},
            {128, 256, 1, .9f, .9f, .9f, 5, false, launch_tiles<KIND, false, 128, 256, 64, 64, 3, 128>},
            {128, 128, 2, .7f, 1.05f, 1.7f, 3, false, launch_tiles<KIND, false, 128, 128, 64, 64, 2, 128>},
            {64, 128, 3, .6f, 1.f, 1.5f, 2, false, launch_tiles<KIND, false, 64, 128, 64, 32, 2, 128>},
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
            return few ? launch_tiles<KIND, true, 64, 128, 64, 32, 2, 128, true>(a, s)
                       : launch_tiles<KIND, true, 128, 128, 64, 32, 2, 128, true>(a, s);
        return few ? launch_tiles<KIND, false, 64, 128, 64, 32, 2, 128, true>(a, s)
                   : launch_tiles<KIND, false, 128, 128, 64, 64, 2, 128, true>(a, s);
    } else if constexpr (KIND == kWgrad) {
        return launch_tiles<KIND, false, 128, 128, 64, 64, 2, 128, true>(a, s);
    } else {
        return few ? launch_tiles<KIND, false, 64, 128, 64, 32, 2, 128, true>(a, s)
                   : launch_tiles<KIND, false, 128, 128, 64, 64, 2, 128, true>(a, s);
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
