// A mixture's router: each token's best experts and their weights, the rows of the grouped products
// sorted by expert, the counts and the balance loss, and the gradient of the scores.
//
//   chosen  the `top` largest scores, the highest first, of equal ones the lowest index first (a NaN
//           is above every number)
//   p       softmax over the chosen,  q  softmax over all E
//   loss    E / (top n^2) sum_e c_e S_e,  c_e the rows of expert e, S_e = sum_t q_te, n tokens
//   ds      at the chosen p_j (dp_j - sum_i p_i dp_i), everywhere dloss E / (top n^2) q_e (c_e - sum_i c_i q_i)
//
// LANES lanes share a token, VPT neighbouring scores each, in registers; its maximum, sums and the next
// best expert pass among them by lane rotations.  Lane j keeps the choice j.
//
// The order of the rows (by expert, then by token) has no atomics in it that could change it: of 64
// tokens each expert has a word of 64 bits, one a token, so that a row's place among them is a count of
// bits; the workgroups' counts go to memory, and a second kernel adds up those before its own.
//
// Bound by latency, not by its few bytes: one token over 64 experts 5.8 us in one launch (top times a chain of
// maxima over the lanes); 16383 over 128 experts, top 8, 17 us in two, a team for each token of a group (16 teams that took
// four in turn 4 us more) and the counts read in one go (one load after the other 4 us more).
#include <type_traits>

#include "activation.h"
#include "operators.h"
#include "values.h"

namespace xtc {
namespace {

constexpr int kThreads = 256, kManyThreads = 1024, kGroup = 64;   // tokens whose bits fill a word
constexpr int kSmallGroup = 16;                                   // of few tokens, for more workgroups to have some

// The value of the lane N places on, around the 16 that share a token.
template <int N>
__device__ __forceinline__ unsigned rotated(unsigned v) {
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xF, 0xF, false);
}
// f over the lanes, in all of them alike: each step joins halves that hold the same values.
template <int LANES, typename V, typename F>
__device__ __forceinline__ V over_lanes(V v, F &&f) {
    static_assert(sizeof(V) == 4, "a register");
    auto step = [&](unsigned u) { return f(v, __builtin_bit_cast(V, u)); };
    v = step(rotated<8>(__builtin_bit_cast(unsigned, v)));
    v = step(rotated<4>(__builtin_bit_cast(unsigned, v)));
    v = step(rotated<2>(__builtin_bit_cast(unsigned, v)));
    v = step(rotated<1>(__builtin_bit_cast(unsigned, v)));
    if constexpr (LANES == 64) {
        // the even rows of 16 lanes and the odd ones, each twice; then the halves
        const unsigned u = __builtin_bit_cast(unsigned, v);
        const auto rows = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        v = f(__builtin_bit_cast(V, (unsigned)rows[0]), __builtin_bit_cast(V, (unsigned)rows[1]));
        const unsigned w = __builtin_bit_cast(unsigned, v);
        const auto halves = __builtin_amdgcn_permlane32_swap(w, w, false, false);
        v = f(__builtin_bit_cast(V, (unsigned)halves[0]), __builtin_bit_cast(V, (unsigned)halves[1]));
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ float team_sum(float v) {
    return over_lanes<LANES>(v, [](float a, float b) { return a + b; });
}

// Scores as whole numbers in their order: NaN highest, -0 and 0 the same; 0 stands below all.
__device__ __forceinline__ unsigned key_of(float v) {
    const unsigned u = __float_as_uint(v + 0.f);
    return v != v ? ~0u : u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float score_of(unsigned key) {
    return __uint_as_float(key >> 31 ? key & 0x7FFFFFFFu : ~key);
}

// VPT scores of a row from e on; -inf past the end.
template <int VPT, typename T>
__device__ __forceinline__ void load_scores(const T *row, int e, int E, float (&v)[VPT]) {
    if (e + VPT <= E) {
        T t[VPT];
        __builtin_memcpy(t, row + e, sizeof(t));
#pragma unroll
        for (int i = 0; i < VPT; ++i) v[i] = widen(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < VPT; ++i) v[i] = e + i < E ? widen(row[e + i]) : -__builtin_inff();
    }
}

// Softmax of a team's scores whose largest is `most`; zeros where that is -inf.
template <int LANES, int VPT>
__device__ __forceinline__ void softmax(const float (&v)[VPT], float most, float (&q)[VPT]) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        q[i] = exp_of(v[i] - most);
        sum += q[i];
    }
    const float inv = 1.f / team_sum<LANES>(sum);
#pragma unroll
    for (int i = 0; i < VPT; ++i) q[i] = most == -__builtin_inff() ? 0.f : q[i] * inv;
}

// What the first half of the work leaves for the second: in memory, or in LDS where one workgroup does both.
struct Halfway {
    int32_t *counts;     // a row of E in whole fours for each workgroup, likewise the sums of q
    float *sums;
    int32_t *expert;     // of each choice of the tokens from `first` on, and its place among the workgroup's
    int32_t *rank;
    int64_t first;
};
__device__ __forceinline__ int fours(int E) { return (E + 3) & ~3; }

// Tokens t0 .. t0 + p.each - 1: their experts and weights, their rows' places among the workgroup's, its counts
// and sums of q.
template <typename T, int LANES, int VPT, int THREADS, int GROUP, bool SMALL>
__device__ __forceinline__ void choose(const RouteArgs &p, const Halfway &h, int block, unsigned char *smem) {
    constexpr int TEAMS = THREADS / LANES, EACH = GROUP / TEAMS, WAVES = THREADS / 64;
    const int E = p.E, top = p.top, tid = threadIdx.x, team = tid / LANES, lane = tid % LANES, e0 = lane * VPT;
    unsigned long long *bits = reinterpret_cast<unsigned long long *>(smem);
    int *before = reinterpret_cast<int *>(bits + E);
    float *sums = reinterpret_cast<float *>(before + E);                    // WAVES x E
    for (int e = tid; e < E; e += THREADS) before[e] = 0;
    float total[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) total[i] = 0.f;
    const int64_t first = (int64_t)block * p.each, end = first + p.each < p.T ? first + p.each : p.T;
    for (int64_t t0 = first; t0 < end; t0 += GROUP) {
        for (int e = tid; e < E; e += THREADS) bits[e] = 0;
        __syncthreads();
        int mine[EACH];              // lane j: the expert of choice j (-1: none)
#pragma unroll
        for (int r = 0; r < EACH; ++r) {
            const int at = r * TEAMS + team;
            const int64_t t = t0 + at;
            const bool there = t < end && (!p.mask || p.mask[t]);
            mine[r] = -1;
            if (there) {
                float v[VPT], q[VPT];
                load_scores<VPT>(static_cast<const T *>(p.scores) + t * p.lds, e0, E, v);
                unsigned key[VPT], chosen = 0;
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    key[i] = key_of(v[i]);
                    if constexpr (sizeof(T) == 2) key[i] = (key[i] & 0xFFFF0000u) | (0xFFFFu - (unsigned)(e0 + i));
                    if (e0 + i >= E) key[i] = 0u;
                }
                float most = 0.f;
                for (int j = 0; j < top; ++j) {
                    unsigned best = key[0];
#pragma unroll
                    for (int i = 1; i < VPT; ++i) best = key[i] > best ? key[i] : best;
                    best = over_lanes<LANES>(best, [](unsigned a, unsigned b) { return a > b ? a : b; });
                    int e;
                    if constexpr (sizeof(T) == 2) {
                        // 16 bits hold a score, the others its expert, the lowest one the largest: no two are equal, and one
                        // maximum finds both
                        e = 0xFFFF - (int)(best & 0xFFFFu);
#pragma unroll
                        for (int i = 0; i < VPT; ++i) key[i] = key[i] == best ? 0u : key[i];
                        best = best >> 31 ? best & 0xFFFF0000u : best | 0xFFFFu;
                    } else {
                        // (the lanes' minimum: their votes and a permutation take 0.2 us longer for one token's eight choices)
                        e = 0x7FFFFFFF;
#pragma unroll
                        for (int i = VPT - 1; i >= 0; --i) e = key[i] == best ? e0 + i : e;
                        e = over_lanes<LANES>(e, [](int a, int b) { return a < b ? a : b; });
#pragma unroll
                        for (int i = 0; i < VPT; ++i) key[i] = e0 + i == e ? 0u : key[i];
                    }
                    if (lane == j) {
                        mine[r] = e;
                        chosen = best;
                    }
                    if (j == 0) most = score_of(best);
                }
                const float w = lane < top ? exp_of(score_of(chosen) - most) : 0.f;
                const float sum = team_sum<LANES>(w);
                if (lane < top) {
                    p.expert[t * top + lane] = mine[r];
                    if constexpr (SMALL) h.expert[(t - h.first) * top + lane] = mine[r];
                    p.p[t * top + lane] = most == -__builtin_inff() ? 0.f : w / sum;
                    atomicOr(&bits[mine[r]], 1ull << at);      // (whichever comes first)
                }
                softmax<LANES>(v, most, q);
#pragma unroll
                for (int i = 0; i < VPT; ++i) total[i] += q[i];
            } else if (t < end && lane < top) {
                p.expert[t * top + lane] = -1;
                if constexpr (SMALL) h.expert[(t - h.first) * top + lane] = -1;
                p.p[t * top + lane] = 0.f;
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < EACH; ++r) {
            const int at = r * TEAMS + team;
            const int64_t t = t0 + at;
            if (t < end && lane < top)
                h.rank[(t - h.first) * top + lane] = mine[r] < 0 ? -1 : before[mine[r]] + __popcll(bits[mine[r]] & ((1ull << at) - 1));
        }
        __syncthreads();
        for (int e = tid; e < E; e += THREADS) before[e] += __popcll(bits[e]);
    }
    // a wave's teams, then the waves
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
#pragma unroll
        for (int d = LANES; d < 64; d *= 2) total[i] += __shfl_xor(total[i], d, 64);
        if (tid % 64 < LANES && e0 + i < E) sums[tid / 64 * E + e0 + i] = total[i];
    }
    __syncthreads();
    for (int e = tid; e < E; e += THREADS) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) s += sums[i * E + e];
        h.counts[block * fours(E) + e] = before[e];
        h.sums[block * fours(E) + e] = s;
    }
}

constexpr int kMostTurns = 64;
// What there is once (block == blocks), or the places of a workgroup's rows: those of all lower experts, of
// this expert in the workgroups before, and the place among its own.
template <int THREADS>
__device__ __forceinline__ void place(const RouteArgs &p, const Halfway &h, int block, int blocks, bool once, bool rows_of, unsigned char *smem) {
    const int E = p.E, top = p.top, tid = threadIdx.x;
    int *start = reinterpret_cast<int *>(smem);          // of this workgroup's rows of each expert
    int *all = start + E;                                // rows of each expert, then up to and with it
    float *part = reinterpret_cast<float *>(all + E);    // 4 x THREADS, and a value a wave
    // (the first trip's choices, on their way beside the counts)
    const int64_t first = (int64_t)block * p.each * top, last = first + (int64_t)p.each * top, end = last < p.T * top ? last : p.T * top;
    int64_t i = first + tid;
    int e = -1, rank = 0;
    auto fetch = [&]() {
        if (i < end) {
            e = h.expert[i - h.first * top];
            rank = h.rank[i - h.first * top];
        }
    };
    if (rows_of) fetch();
    for (int e = tid; e < E; e += THREADS) start[e] = all[e] = 0;
    __syncthreads();
    // the workgroups' counts, four experts a load, the threads taking the workgroups in turn; whole numbers,
    // whose sums do not depend on the order
    // (kMostTurns of them at most: their sums of q are added one after the other)
    const int width = fours(E) / 4, fit = THREADS / width < kMostTurns ? THREADS / width : kMostTurns;
    const int turns = fit < blocks ? fit : blocks, g = tid % width, turn = tid / width;
    if (turn < turns) {
        int sum[4] = {0, 0, 0, 0}, mine[4] = {0, 0, 0, 0};
        float q[4] = {0.f, 0.f, 0.f, 0.f};
        constexpr int AT_ONCE = 8;       // loads on their way together
        for (int b0 = turn; b0 < blocks; b0 += AT_ONCE * turns) {
            int c[AT_ONCE][4];
            float f[AT_ONCE][4];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int b = b0 + k * turns, at = ((b < blocks ? b : turn) * width + g) * 4;
                __builtin_memcpy(c[k], __builtin_assume_aligned(h.counts + at, 16), 16);
                if (once) __builtin_memcpy(f[k], __builtin_assume_aligned(h.sums + at, 16), 16);
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int b = b0 + k * turns;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sum[i] += b < blocks ? c[k][i] : 0;
                    mine[i] += b < block && b < blocks ? c[k][i] : 0;
                    if (once) q[i] += b < blocks ? f[k][i] : 0.f;
                }
            }
        }
        if (once) {
#pragma unroll
            for (int i = 0; i < 4; ++i) part[(turn * width + g) * 4 + i] = q[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (g * 4 + i < E) {
                atomicAdd(&all[g * 4 + i], sum[i]);
                if (rows_of) atomicAdd(&start[g * 4 + i], mine[i]);
            }
    }
    __syncthreads();
    float weighed = 0.f;         // counts times sums of q, the latter over the turns in their order
    if (once) {
        for (int e = tid; e < E; e += THREADS) {
            float q = 0.f;
            for (int i = 0; i < turns; ++i) q += part[i * width * 4 + e];
            weighed += (float)all[e] * q;
        }
        weighed = lanes_sum<64>(weighed);
        if ((tid & 63) == 0) part[4 * THREADS + tid / 64] = weighed;
        __syncthreads();
    }
    // rows up to and with each expert: a wave at a time, 64 experts a step
    if (tid < 64) {
        int before = 0;
        for (int e0 = 0; e0 < E; e0 += 64) {
            const int e = e0 + tid;
            int v = e < E ? all[e] : 0;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int u = __shfl_up(v, d, 64);
                if (tid >= d) v += u;
            }
            v += before;
            if (e < E) {
                start[e] += v - all[e];
                if (once) {
                    p.counts[e] = all[e];
                    p.ends[e] = v;
                }
                all[e] = v;
            }
            before = __shfl(v, 63, 64);
        }
    }
    __syncthreads();
    const int rows = all[E - 1];
    if (once && tid == 0) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) s += part[4 * THREADS + i];
        const float n = (float)(rows / top > 1 ? rows / top : 1);
        *p.loss = rows > 0 ? (float)E / ((float)top * n) * (s / n) : 0.f;
    }
    if (!rows_of) return;
    for (; i < end; i += THREADS, fetch()) {
        int at = -1;
        if (e >= 0) {
            at = start[e] + rank;
            p.token[at] = (int32_t)((unsigned)i / (unsigned)top);      // (T top rows fit 31 bits)
        }
        p.row[i] = at;
        if (i >= rows) p.token[i] = -1;
    }
}

size_t choose_bytes(int E, int threads) { return (size_t)E * 12 + (size_t)(threads / 64) * E * 4; }
size_t place_bytes(int E, int threads) { return (size_t)E * 8 + (size_t)threads * 17; }

__device__ __forceinline__ Halfway in_memory(const RouteArgs &p) { return Halfway{p.counts_of, p.sums_of, p.expert, p.row, 0}; }

template <typename T, int LANES, int VPT, int THREADS, int GROUP>
__global__ void __launch_bounds__(THREADS) route_choose_kernel(RouteArgs p) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    choose<T, LANES, VPT, THREADS, GROUP, false>(p, in_memory(p), blockIdx.x, smem);
}

// (one workgroup more than route_choose_kernel's)
__global__ void __launch_bounds__(kManyThreads) route_place_kernel(RouteArgs p, int blocks) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int block = blockIdx.x;
    place<kManyThreads>(p, in_memory(p), block, blocks, block == blocks, block < blocks, smem);
}

// The few tokens of one workgroup, in one launch; what lies halfway stays in LDS.
constexpr int kMostChoices = 16;
template <typename T, int LANES, int VPT>
__global__ void __launch_bounds__(kThreads) route_small_kernel(RouteArgs p) {
    __shared__ __attribute__((aligned(16))) int32_t counts[LANES * VPT];
    __shared__ __attribute__((aligned(16))) float sums[LANES * VPT];
    __shared__ int32_t expert[kSmallGroup * kMostChoices], rank[kSmallGroup * kMostChoices];
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const Halfway h = {counts, sums, expert, rank, 0};
    choose<T, LANES, VPT, kThreads, kSmallGroup, true>(p, h, 0, smem);
    __syncthreads();
    place<kThreads>(p, h, 0, 1, true, true, smem);
}

// ds of the tokens blockIdx.x, + gridDim.x, ... of each team.  16384 x 64 fp32, top 6: 4.8 us with the launch, of which
// its 9.6 MB are 1.8.
template <typename T, typename O, int LANES, int VPT>
__global__ void __launch_bounds__(kThreads) route_backward_kernel(RouteBackwardArgs p) {
    constexpr int TEAMS = kThreads / LANES;
    const int E = p.E, top = p.top, team = threadIdx.x / LANES, lane = threadIdx.x % LANES, e0 = lane * VPT;
    float c[VPT], rows = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        c[i] = e0 + i < E ? (float)p.counts[e0 + i] : 0.f;
        rows += c[i];
    }
    float n = team_sum<LANES>(rows) / (float)top;
    n = n > 1.f ? n : 1.f;
    const float scale = p.dloss * ((float)E / ((float)top * n)) / n;
    for (int64_t t = (int64_t)blockIdx.x * TEAMS + team; t < p.T; t += (int64_t)gridDim.x * TEAMS) {
        const bool has = lane < top;
        const int e = has ? p.expert[t * top + lane] : -1;
        const bool there = __shfl(e, 0, LANES) >= 0;
        float d[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) d[i] = 0.f;
        if (there) {
            float v[VPT];
            load_scores<VPT>(static_cast<const T *>(p.scores) + t * p.lds, e0, E, v);
            const float w = has ? p.p[t * top + lane] : 0.f, dp = has && p.DP ? p.DP[t * top + lane] : 0.f;
            float most = v[0];
#pragma unroll
            for (int i = 1; i < VPT; ++i) most = fmaxf(most, v[i]);
            most = over_lanes<LANES>(most, [](float a, float b) { return fmaxf(a, b); });
            softmax<LANES>(v, most, d);
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < VPT; ++i) dot += c[i] * d[i];
            dot = team_sum<LANES>(dot);
#pragma unroll
            for (int i = 0; i < VPT; ++i) d[i] = scale * d[i] * (c[i] - dot);
            const float g = w * (dp - team_sum<LANES>(w * dp));
            for (int j = 0; j < top; ++j) {
                const int at = __shfl(e, j, LANES) - e0;
                const float add = __shfl(g, j, LANES);
#pragma unroll
                for (int i = 0; i < VPT; ++i) d[i] += at == i ? add : 0.f;
            }
        }
        O *out = static_cast<O *>(p.DS) + t * p.ldds + e0;
        O o[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) narrow(d[i], &o[i]);
        if (e0 + VPT <= E) {
            __builtin_memcpy(out, o, sizeof(o));
        } else {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (e0 + i < E) out[i] = o[i];
        }
    }
}

// f(lanes, scores a lane) for E experts, as constants.
template <typename F>
void with_lanes(int E, F &&f) {
    typedef std::integral_constant<int, 16> Row;
    if (E <= 16) f(Row(), std::integral_constant<int, 1>());
    else if (E <= 32) f(Row(), std::integral_constant<int, 2>());
    else if (E <= 64) f(Row(), std::integral_constant<int, 4>());
    else if (E <= 128) f(Row(), std::integral_constant<int, 8>());
    else if (E <= 256) f(Row(), std::integral_constant<int, 16>());
    else if (E <= 512) f(std::integral_constant<int, 64>(), std::integral_constant<int, 8>());
    else f(std::integral_constant<int, 64>(), std::integral_constant<int, 16>());
}

// Tokens of a workgroup (whole groups), and the workgroups.  Every one of them reads the counts of all: 128 up to 128 tokens
// each, 256 beyond (16384 tokens, 200 experts 24.7 us, with 256 27.5).  Groups of 16 as long as 128 workgroups hold the
// tokens (1291 tokens, 200 experts 14.1 us, with groups of 64 17.7), and one of them is a single launch (64 tokens in one
// launch 9 us longer than in two, 9.4).
constexpr int kFewBlocks = 128, kManyBlocks = 256;
int64_t each_of(int64_t T) {
    if (T <= kFewBlocks * kSmallGroup) return kSmallGroup;
    const int64_t most = T <= kFewBlocks * 2 * kGroup ? kFewBlocks : kManyBlocks;
    return ((T + kGroup - 1) / kGroup + most - 1) / most * kGroup;
}
int blocks_of(int64_t T) { return T > 0 ? (int)((T + each_of(T) - 1) / each_of(T)) : 1; }

}  // namespace

int64_t route_workspace(int64_t T, int64_t E) { return blocks_of(T) > 1 ? (int64_t)blocks_of(T) * ((E + 3) / 4 * 4) * 8 : 0; }

xtc_status launch_route(const RouteArgs &given, xtc_dtype dtype, void *workspace, hipStream_t s) {
    RouteArgs a = given;
    const int blocks = blocks_of(a.T);
    a.each = (int)each_of(a.T);
    a.counts_of = static_cast<int32_t *>(workspace);
    a.sums_of = workspace ? reinterpret_cast<float *>(a.counts_of + (int64_t)blocks * ((a.E + 3) / 4 * 4)) : nullptr;
    with_lanes(a.E, [&](auto lanes, auto vpt) {
        constexpr int LANES = lanes(), VPT = vpt();
        if (blocks == 1) {
            const size_t one = choose_bytes(a.E, kThreads), two = place_bytes(a.E, kThreads);
            const auto kernel = dtype == XTC_F32 ? route_small_kernel<float, LANES, VPT> : route_small_kernel<Bf16, LANES, VPT>;
            kernel<<<1, kThreads, one > two ? one : two, s>>>(a);
        } else {
            auto run = [&](auto threads, auto group) {
                constexpr int THREADS = threads(), GROUP = group();
                const auto kernel = dtype == XTC_F32 ? route_choose_kernel<float, LANES, VPT, THREADS, GROUP> : route_choose_kernel<Bf16, LANES, VPT, THREADS, GROUP>;
                kernel<<<(unsigned)blocks, THREADS, choose_bytes(a.E, THREADS), s>>>(a);
            };
            if (a.each == kSmallGroup) run(std::integral_constant<int, kThreads>(), std::integral_constant<int, kSmallGroup>());
            else run(std::integral_constant<int, kManyThreads>(), std::integral_constant<int, kGroup>());
            route_place_kernel<<<(unsigned)blocks + 1, kManyThreads, place_bytes(a.E, kManyThreads), s>>>(a, blocks);
        }
    });
    return hip_status(hipGetLastError());
}

xtc_status launch_route_backward(const RouteBackwardArgs &a, xtc_dtype dtype, xtc_dtype out_dtype, hipStream_t s) {
    with_lanes(a.E, [&](auto lanes, auto vpt) {
        constexpr int LANES = lanes(), VPT = vpt(), TEAMS = kThreads / LANES;
        const int64_t groups = (a.T + TEAMS - 1) / TEAMS;
        const auto kernel =
            dtype == XTC_F32 ? (out_dtype == XTC_F32 ? route_backward_kernel<float, float, LANES, VPT> : route_backward_kernel<float, Bf16, LANES, VPT>)
                             : (out_dtype == XTC_F32 ? route_backward_kernel<Bf16, float, LANES, VPT> : route_backward_kernel<Bf16, Bf16, LANES, VPT>);
        kernel<<<(unsigned)(groups < 2048 ? groups : 2048), kThreads, 0, s>>>(a);
    });
    return hip_status(hipGetLastError());
}

}  // namespace xtc
