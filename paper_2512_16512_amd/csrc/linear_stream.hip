// The linear layer's products of few rows: the compiled kernels.
#include "grouped_stream.h"

namespace xtc {

template <Kind KIND>
const Choice *linear_stream_choices(int *count) {
    static const Choice all[] = {
        {16, 16, 1, .06f, .06f, .06f, 2, false, launch_streams<KIND, false, 16, 16, 8, 3, LinearArgs>},
        {16, 32, 1, .09f, .09f, .09f, 2, false, launch_streams<KIND, false, 16, 32, 8, 3, LinearArgs>},
        {32, 64, 1, .28f, .35f, .28f, 2.5f, false, launch_streams<KIND, false, 32, 64, 4, 2, LinearArgs>},
    };
    *count = 3;
    return all;
}

template const Choice *linear_stream_choices<kBf16N>(int *);
template const Choice *linear_stream_choices<kBf16T>(int *);

}  // namespace xtc
