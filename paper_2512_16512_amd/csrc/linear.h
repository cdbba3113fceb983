// The linear layer on the kernels of the grouped products: which tile of it, and of which part of
// the reduction, a workgroup computes, and the epilogue
//
//   z = sum + bias,  out = act(z) + residual
//
// in fp32, z and out rounded once each.
#pragma once

#include <type_traits>

#include "activation.h"
#include "grouped.h"
#include "values.h"

namespace xtc {

// The tiles of a layer: `splits` times those of the whole, split by split, each over its part of
// the reduction.
template <Kind KIND, int BM, int BN>
struct LinearOrder {
    const LinearArgs &p;
    int tiles_m, tiles_n, total;

    __device__ __forceinline__ LinearOrder(const LinearArgs &p_) : p(p_) {
        tiles_m = ((KIND == kWgrad ? p.K : (int)p.T) + BM - 1) / BM;
        tiles_n = (p.N + BN - 1) / BN;
        total = tiles_m * tiles_n * p.splits;
    }
    __device__ __forceinline__ Place at(int id) const {
        const int each = tiles_m * tiles_n, split = id / each;
        int im, in;
        tile_coords(id - split * each, each, tiles_m, tiles_n, kBand, 0, im, in);
        if constexpr (KIND == kBf16N && BN < 64) {
            // Few rows: the lines of 128 bytes of B's rows, shared by the strips that read pieces of one, go to the XCDs in turn.
            // With a run of neighbours each, rows of 8 KB lie in a quarter of an XCD's L2 channels (1 x 4096 to 4096
            // 11.8 us, so 11.0; 2560 to 2048 6.2 and 5.5).
            constexpr int G = 64 / BN;
            const int lines = tiles_n / G;
            if (tiles_m == 1 && tiles_n % (8 * G) == 0) {
                const int l = in / G, each = lines / 8;
                in = (l % each * 8 + l / each) * G + in % G;
            }
        }
        const int at = split * p.k_each;
        if constexpr (KIND == kWgrad) {
            const int left = (int)p.T - at;
            return Place{split, at, left < p.k_each ? left : p.k_each, im * BM, in * BN};
        } else {
            const int left = (int)p.T - im * BM;
            return Place{split, im * BM, left < BM ? left : BM, 0, in * BN};
        }
    }
};

template <Kind KIND, int BM, int BN>
struct OrderFor<LinearArgs, KIND, BM, BN> {
    typedef LinearOrder<KIND, BM, BN> type;
};

template <Kind KIND>
__device__ __forceinline__ Tile make_tile(const LinearArgs &p, const Place &w) {
    static_assert(KIND != kFp8, "bf16 operands");
    Tile t;
    t.lda = p.lda * 2;
    t.ldb = p.ldb * 2;
    t.SA = t.SB = nullptr;
    t.n = p.N - w.n0;
    t.A = static_cast<const unsigned char *>(p.A) + w.row0 * t.lda;
    t.B = static_cast<const unsigned char *>(p.B);
    int64_t row = w.row0;
    if constexpr (KIND == kWgrad) {
        t.A += (int64_t)w.m0 * 2;
        t.B += w.row0 * t.ldb + (int64_t)w.n0 * 2;
        t.m = p.K - w.m0;
        t.k = w.rows;
        row = w.m0;
    } else {
        const int k0 = w.group * p.k_each, left = p.K - k0;
        t.A += (int64_t)k0 * 2;
        t.B += KIND == kBf16N ? k0 * t.ldb + (int64_t)w.n0 * 2 : w.n0 * t.ldb + (int64_t)k0 * 2;
        t.m = w.rows;
        t.k = left < p.k_each ? left : p.k_each;
    }
    if (p.splits > 1) {
        const int64_t rows = KIND == kWgrad ? p.K : p.T;
        t.C = reinterpret_cast<unsigned char *>(p.part + (w.group * rows + row) * p.N + w.n0);
    } else {
        t.C = static_cast<unsigned char *>(p.C) + (row * p.ldc + w.n0) * (p.out_bf16 ? 2 : 4);
    }
    return t;
}

// EACH columns of a row of results from column n on.
template <typename T, int EACH>
struct Epilogue {
    const LinearArgs &p;
    int64_t row0;
    int n, left;
    float bias[EACH];

    static __device__ __forceinline__ void load(const void *base, int f32, int64_t at, int left, float (&v)[EACH]) {
        if (f32) {
            const float *s = static_cast<const float *>(base) + at;
            if (left >= EACH) {
                __builtin_memcpy(v, s, sizeof(v));
            } else {
#pragma unroll
                for (int i = 0; i < EACH; ++i) v[i] = i < left ? s[i] : 0.f;
            }
        } else {
            const Bf16 *s = static_cast<const Bf16 *>(base) + at;
            Bf16 t[EACH];
            if (left >= EACH) {
                __builtin_memcpy(t, s, sizeof(t));
#pragma unroll
                for (int i = 0; i < EACH; ++i) v[i] = widen(t[i]);
            } else {
#pragma unroll
                for (int i = 0; i < EACH; ++i) v[i] = i < left ? widen(s[i]) : 0.f;
            }
        }
    }

    __device__ __forceinline__ Epilogue(const LinearArgs &p_, int row0_, int n_) : p(p_), row0(row0_), n(n_), left(p_.N - n_) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) bias[i] = 0.f;
        if (p.bias && left > 0) load(p.bias, p.bias_f32, n, left, bias);
    }

    struct Residual {
        float v[EACH];
    };
    __device__ __forceinline__ Residual residual(int m, bool there) const {
        Residual r = {};
        if (p.R && there && left > 0) load(p.R, p.r_f32, (row0 + m) * p.ldr + n, left, r.v);
        return r;
    }

    // Results 16 bytes wide leave past the caches, as whole lines.
    static __device__ __forceinline__ void store(T *c, int left, const float (&v)[EACH]) {
        T t[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) t[i] = (T)v[i];
        if constexpr (sizeof(t) == 16) {
            store_past_caches(c, t, left);
        } else if (left >= EACH) {
            __builtin_memcpy(c, t, sizeof(t));
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (i < left) c[i] = t[i];
        }
    }

    // Row row0 + m: v the sums.
    __device__ __forceinline__ void write(int m, float (&v)[EACH], const Residual &r) const {
        if (left <= 0) return;
#pragma unroll
        for (int i = 0; i < EACH; ++i) v[i] += bias[i];
        if (p.Z) store(static_cast<T *>(p.Z) + (row0 + m) * p.ldz + n, left, v);
        with_activation(p.act, [&](auto ACT) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) v[i] = activated<ACT()>(v[i]);
        });
#pragma unroll
        for (int i = 0; i < EACH; ++i) v[i] += r.v[i];
        store(static_cast<T *>(p.C) + (row0 + m) * p.ldc + n, left, v);
    }
};

template <typename T, int EACH>
__device__ __forceinline__ void finish_at(const LinearArgs &p, int row, int n, float (&v)[EACH]) {
    const Epilogue<T, EACH> e(p, row, n);
    e.write(0, v, e.residual(0, true));
}

// A compiled kernel and what a launch of it takes, in microseconds: with n tiles on 256 CUs
// of per_cu workgroups each, every round costs `fixed` (the launch, the first data's way and the
// results') and for each stage of k (128 bytes) `one` where each CU holds one workgroup, `full`
// where it holds per_cu; a round that leaves CUs empty has fill * one for a stage at the least.
struct LinearChoice {
    int bm, bn, per_cu;
    float one, full, fixed, fill;
    xtc_status (*launch)(const GroupedArgs &, hipStream_t);
};

// The kernels of one file each for bf16 layers; those of linear_any_choices take every call, the
// others such with aligned rows.
template <Kind KIND>
const LinearChoice *linear_any_choices(int *count);
template <Kind KIND>
const LinearChoice *linear_tile_choices(int *count);
template <Kind KIND>
const LinearChoice *linear_stream_choices(int *count);

inline int64_t linear_tiles(const LinearArgs &a, Kind kind, int bm, int bn) {
    return cdiv(kind == kWgrad ? a.K : a.T, bm) * cdiv(a.N, bn) * a.splits;
}
template <Kind KIND>
int64_t tile_count(const LinearArgs &a, int bm, int bn) {
    return linear_tiles(a, KIND, bm, bn);
}

}  // namespace xtc
