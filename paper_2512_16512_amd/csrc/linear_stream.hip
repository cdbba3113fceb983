// The linear layer's products of few rows: the compiled kernels.
#include "grouped_stream.h"

namespace xtc {
namespace {

template <Kind KIND, int BM, int BN, int NW, int STAGES>
constexpr auto kLaunch = launch_streams<KIND, false, BM, BN, NW, STAGES, LinearArgs>;

}  // namespace

template <Kind KIND>
const LinearChoice *linear_stream_choices(int *count) {
    // B that is K x N is read in pieces of 32 bytes by strips of 16 columns, 64 by 32 (1 x 4096 to 4096: 11.2 us,
    // the other layout's whole lines 7.8).
    constexpr bool N = KIND == kBf16N;
    static const LinearChoice all[] = {
        {16, 16, 2, N ? .128f : .045f, N ? .225f : .112f, N ? 3.f : 3.3f, N ? .41f : .8f, kLaunch<KIND, 16, 16, 4, 4>},
        {16, 32, 1, N ? .146f : .058f, N ? .146f : .058f, N ? 3.2f : 3.5f, N ? .5f : .88f, kLaunch<KIND, 16, 32, 4, 4>},
        {32, 32, 1, N ? .139f : .096f, N ? .139f : .096f, 3.7f, .57f, kLaunch<KIND, 32, 32, 4, 4>},
        {32, 64, 1, .168f, .168f, 4.2f, N ? .59f : .53f, kLaunch<KIND, 32, 64, 4, 2>},
        {64, 64, 1, N ? .236f : .222f, N ? .236f : .222f, N ? 5.f : 5.4f, N ? .62f : .52f, kLaunch<KIND, 64, 64, 4, 2>},
    };
    *count = 5;
    return all;
}

template const LinearChoice *linear_stream_choices<kBf16N>(int *);
template const LinearChoice *linear_stream_choices<kBf16T>(int *);

}  // namespace xtc
