// logits.hpp -- what the operators on rows of logits share: a row's chunks, its
// bounds, and how it is split over workgroups.
#pragma once

#include <algorithm>
#include <cmath>

#include "common.hpp"

namespace gp {
namespace {

constexpr float LOG2E = 1.44269504088896341f;
constexpr float NEVER = -1e30f;  // a logit down here is a mask's, its token cannot occur
__host__ __device__ inline float lower_bound(float clip) { return -clip > NEVER ? -clip : NEVER; }
constexpr float NO_REF = -2e30f;  // below every reference
constexpr int SPLIT_MAX = 32;    // workgroups of one row: at most the lanes of the wave that joins them

// A row in chunks of 16 bytes, the last one short where V asks for it.  Global memory
// takes 16-byte accesses at any element's address.
template <typename T> struct Chunks {
    static constexpr int N = Vec16<T>::N;
    typedef typename Vec16<T>::type vec __attribute__((aligned(sizeof(T))));
    static __device__ __forceinline__ vec load(const T* row, int j) {
        return *reinterpret_cast<const vec*>(row + (long)j * N);
    }
    // the values of any chunk of a row of V; `none` behind its end
    static __device__ __forceinline__ void values(const T* row, int V, int j, float none, float (&x)[N]) {
        if (j < V / N) {
            const vec v = load(row, j);
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = to_f32((T)v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = j * N + e < V ? to_f32(row[(long)j * N + e]) : none;
        }
    }
};

int chunk_count(int dtype, int vocab) {
    const int n = dtype == GP_BF16 ? 8 : 4;
    return vocab / n + (vocab % n ? 1 : 0);
}
// Workgroups of a row, joined by a second launch: several for up to 96 rows of 256 KB or
// more, each over 16 KB or more of it and 768 in all, while one workgroup per row
// leaves most CUs without work and takes longer for its row than the joining does.  us,
// split / whole, bf16 with 5 alternatives: one row of 131072 9.1 / 14.8, 32 rows 10.8 / 15.3,
// 64 rows 12.2 / 15.0 (7.4 / 11.6 with none, 16.6 / 16.2 with 20), 96 rows 13.3 / 15.2; but 128
// rows 15.7 / 15.8, one row of 32000 8.4 / 7.4, 64 of 65536 10.6 / 10.3, and 93 of 50021 fp32
// with 20 17.5 / 11.1 (19.2 / 12.9 with one row of masks alone, whose alternatives are all ties).
int row_splits(int dtype, long rows, int vocab) {
    const long chunks = chunk_count(dtype, vocab);
    if (rows < 1 || rows > 96 || chunks < 16384) return 1;
    return (int)std::min<long>(SPLIT_MAX, std::min(768 / rows, chunks / 1024));
}
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Rows of `row` bytes, `pitch` apart, from two starts lie between each other (the columns of one
// buffer) without overlapping.
bool side_by_side(uintptr_t a, uintptr_t b, size_t row, size_t pitch) {
    const size_t off = pitch ? (a < b ? b - a : a - b) % pitch : 0;
    return off >= row && off + row <= pitch;
}

// Rows of a launch at most: a launch holds fewer than 2^32 threads, a workgroup of a row
// up to 1024 of them.
constexpr long LAUNCH_ROWS = 1L << 21;

template <typename P> P* past(P* p, long n) { return p ? p + n : nullptr; }

} // namespace
} // namespace gp
