// The linear layer's products on LDS-staged tiles: the compiled kernels.
#include "grouped_tile.h"

namespace xtc {
namespace {

template <Kind KIND, int BM, int BN, int WM, int WN, int STAGES, int KB>
constexpr auto kLaunch = launch_tiles<KIND, false, BM, BN, WM, WN, STAGES, KB, false, LinearArgs>;

// Rows at any address: AHEAD stages ahead (184 rows, 1731 to 3459, B N x K: 16.1 us, 19.6 with one stage; 1 row, 7833 to 2849:
// 16.6 and 18.9; B K x N, whose rows are the pieces that it waits for, the same within 3 %) unless rows hold less than 16
// bytes or there is nothing to sum.
template <Kind KIND, int BM, int BN, int WM, int WN, int STAGES, int KB, int AHEAD>
xtc_status launch_any_rows(const GroupedArgs &a, hipStream_t s) {
    const bool far = a.K >= 8 && (KIND == kBf16T || a.N >= 8) && (KIND != kWgrad || a.T > 0);
    return far ? launch_tiles<KIND, false, BM, BN, WM, WN, STAGES, KB, true, LinearArgs, AHEAD>(a, s)
               : launch_tiles<KIND, false, BM, BN, WM, WN, STAGES, KB, true, LinearArgs>(a, s);
}

}  // namespace

// Measured, these and those of linear_stream.hip, on 145 layers of 1 to 16384 rows and widths of 512 to 8192, each
// kernel with 1 to 16 splits: the kernel chosen by the estimate takes 1.5 % longer than the best of all in the mean,
// 30 % at most (2 rows, 4608 to 576: 9.0 us for 6.9).  8192 x 4096 to 4096 with gelu_tanh 210 us, z kept too 223 (tiles of
// 256x256; those of 128x128 a fifth longer), 1531 x 4096 to 2000 36 us (B N x K, 128x128 with four stages, the reduction
// whole; 56 with the choices of the grouped products).
template <Kind KIND>
const LinearChoice *linear_tile_choices(int *count) {
    if constexpr (KIND == kWgrad) {
        static const LinearChoice all[] = {
            {256, 256, 1, 1.39f, 1.39f, 14.8f, .79f, kLaunch<KIND, 256, 256, 128, 64, 4, 64>},
            {128, 256, 1, .78f, .78f, 10.6f, .75f, kLaunch<KIND, 128, 256, 64, 64, 3, 128>},
            {128, 128, 2, .7f, .87f, 9.5f, .75f, kLaunch<KIND, 128, 128, 64, 64, 2, 128>},
        };
        *count = 3;
        return all;
    } else {
        constexpr bool N = KIND == kBf16N;
        static const LinearChoice all[] = {
            {256, 256, 1, N ? 1.44f : 1.34f, N ? 1.44f : 1.34f, 11.8f, N ? .64f : .74f, kLaunch<KIND, 256, 256, 128, 64, 2, 128>},
            {256, 128, 1, N ? .76f : .74f, N ? .76f : .74f, N ? 8.2f : 8.f, .78f, kLaunch<KIND, 256, 128, 64, 64, 3, 128>},
            {128, 128, 2, N ? .7f : .63f, N ? .89f : .85f, 7.3f, .73f, kLaunch<KIND, 128, 128, 64, 64, 2, 128>},
            {128, 128, 1, N ? .44f : .42f, N ? .44f : .42f, N ? 6.6f : 6.1f, .88f, kLaunch<KIND, 128, 128, 64, 32, 4, 128>},
            {64, 128, 1, N ? .35f : .29f, N ? .35f : .29f, 5.1f, 1, kLaunch<KIND, 64, 128, 64, 16, 4, 128>},
            {64, 64, 2, N ? .28f : .25f, N ? .39f : .37f, N ? 4.9f : 4.6f, .75f, kLaunch<KIND, 64, 64, 64, 16, 4, 128>},
        };
        *count = 6;
        return all;
    }
}

// Rows at any address go through registers, whose loads reach lines in pieces: a stage of 64x128 takes .6 us where the
// direct copies take .35.  Copied first they run the kernels above where that is faster (a weights' gradient of 12190 rows,
// 803 x 6111: 206 us with the copies of 184 MB, 317 without; one row, 7833 to 2849: 17 us through registers, 25 copied; 181
// rows, 5076 to 4503: 37 and 42).  90 layers of odd widths: the kernel chosen takes 2 % longer than the best in the mean, 44 %
// at most (32 rows, 7539 to 6848, whose A alone is copied: 38 us for 27).
template <Kind KIND>
const LinearChoice *linear_any_choices(int *count) {
    if constexpr (KIND == kWgrad) {
        static const LinearChoice all[] = {
            {64, 128, 1, .53f, .53f, 5.2f, 1, launch_any_rows<KIND, 64, 128, 64, 16, 2, 128, 4>},
            {64, 64, 3, .58f, .95f, 5.9f, .77f, launch_any_rows<KIND, 64, 64, 64, 16, 2, 128, 4>},
        };
        *count = 2;
        return all;
    } else {
        constexpr bool N = KIND == kBf16N;
        static const LinearChoice all[] = {
            {64, 128, 1, N ? .61f : .58f, N ? .61f : .58f, 4.7f, N ? 1.f : .75f, launch_any_rows<KIND, 64, 128, 64, 16, 2, 128, 4>},
            {64, 64, 3, N ? .52f : .37f, N ? 1.03f : 1.14f, 5.f, N ? .83f : .78f, launch_any_rows<KIND, 64, 64, 64, 16, 2, 128, 4>},
        };
        *count = 2;
        return all;
    }
}

template const LinearChoice *linear_any_choices<kBf16N>(int *);
template const LinearChoice *linear_any_choices<kBf16T>(int *);
template const LinearChoice *linear_any_choices<kWgrad>(int *);
template const LinearChoice *linear_tile_choices<kBf16N>(int *);
template const LinearChoice *linear_tile_choices<kBf16T>(int *);
template const LinearChoice *linear_tile_choices<kWgrad>(int *);

}  // namespace xtc
