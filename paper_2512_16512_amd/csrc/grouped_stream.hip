// The grouped and 8-bit products of few rows: the compiled kernels.
#include "grouped_stream.h"

namespace xtc {

// Measured as the tiles' (`one` and `full` hold four waves' or eight's share of k).
template <Kind KIND>
const Choice *stream_choices(bool wide, int *count) {
    if constexpr (KIND == kFp8) {
        static const Choice sums[] = {
            {16, 16, 2, .065f, .065f, .13f, 1, true, launch_streams<KIND, true, 16, 16, 4, 3>},
            {32, 16, 3, .08f, .08f, .22f, 2.2f, true, launch_streams<KIND, true, 32, 16, 4, 2>},
            {32, 32, 2, .17f, .17f, .33f, 2.8f, false, launch_streams<KIND, true, 32, 32, 4, 2>},
            {32, 64, 1, .2f, .35f, .2f, 3, false, launch_streams<KIND, true, 32, 64, 4, 2>},
            {64, 64, 1, .3f, .41f, .3f, 3, false, launch_streams<KIND, true, 64, 64, 4, 2>},
        };
        static const Choice rounded[] = {
            {16, 16, 2, .06f, .06f, .125f, 1, true, launch_streams<KIND, false, 16, 16, 4, 3>},
            {32, 16, 3, .07f, .07f, .2f, 2.2f, true, launch_streams<KIND, false, 32, 16, 4, 2>},
            {32, 32, 2, .15f, .15f, .3f, 2.8f, false, launch_streams<KIND, false, 32, 32, 4, 2>},
            {32, 64, 1, .15f, .34f, .15f, 3, false, launch_streams<KIND, false, 32, 64, 4, 2>},
            {64, 64, 1, .22f, .39f, .22f, 2.5f, false, launch_streams<KIND, false, 64, 64, 4, 2>},
        };
        *count = 5;
        return wide ? sums : rounded;
    } else {
        static const Choice all[] = {{32, 64, 1, .28f, .35f, .28f, 2.5f, false, launch_streams<KIND, false, 32, 64, 4, 2>}};
        *count = 1;
        return all;
    }
}

template const Choice *stream_choices<kFp8>(bool, int *);
template const Choice *stream_choices<kBf16N>(bool, int *);
template const Choice *stream_choices<kBf16T>(bool, int *);

}  // namespace xtc
