// The linear layer's products on LDS-staged tiles: the compiled kernels.
#include "grouped_tile.h"

namespace xtc {

template <Kind KIND>
const Choice *linear_tile_choices(int *count) {
    if constexpr (KIND == kWgrad) {
        static const Choice all[] = {
            {256, 256, 1, 1.5f, 1.5f, 1.5f, 12, false, launch_tiles<KIND, false, 256, 256, 128, 64, 4, 64, false, LinearArgs>},
            {128, 256, 1, .81f, .81f, .81f, 7.9f, false, launch_tiles<KIND, false, 128, 256, 64, 64, 3, 128, false, LinearArgs>},
            {128, 128, 2, .7f, .7f, 1.18f, 7.1f, false, launch_tiles<KIND, false, 128, 128, 64, 64, 2, 128, false, LinearArgs>},
        };
        *count = 3;
        return all;
    } else {
        static const Choice all[] = {
            {256, 256, 1, 1.5f, 1.5f, 1.5f, 8, false, launch_tiles<KIND, false, 256, 256, 128, 64, 2, 128, false, LinearArgs>},
            {128, 256, 2, 1.25f, 1.25f, 2.2f, 5, false, launch_tiles<KIND, false, 128, 256, 64, 128, 3, 64, false, LinearArgs>},
            {128, 256, 1, .9f, .9f, .9f, 5, false, launch_tiles<KIND, false, 128, 256, 64, 64, 3, 128, false, LinearArgs>},
            {128, 128, 2, .7f, 1.05f, 1.7f, 3, false, launch_tiles<KIND, false, 128, 128, 64, 64, 2, 128, false, LinearArgs>},
            {64, 128, 3, .6f, 1.f, 1.5f, 2, false, launch_tiles<KIND, false, 64, 128, 64, 32, 2, 128, false, LinearArgs>},
        };
        *count = 5;
        return all;
    }
}

template <Kind KIND>
xtc_status launch_linear_any(const LinearArgs &a, hipStream_t s) {
    if constexpr (KIND != kWgrad) {
        if (a.T <= 64) return launch_tiles<KIND, false, 64, 128, 64, 32, 2, 128, true, LinearArgs>(a, s);
    }
    return launch_tiles<KIND, false, 128, 128, 64, 64, 2, 128, true, LinearArgs>(a, s);
}

template xtc_status launch_linear_any<kBf16N>(const LinearArgs &, hipStream_t);
template xtc_status launch_linear_any<kBf16T>(const LinearArgs &, hipStream_t);
template xtc_status launch_linear_any<kWgrad>(const LinearArgs &, hipStream_t);
template const Choice *linear_tile_choices<kBf16N>(int *);
template const Choice *linear_tile_choices<kBf16T>(int *);
template const Choice *linear_tile_choices<kWgrad>(int *);

}  // namespace xtc
