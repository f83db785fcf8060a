// attention_rows.hpp -- attention on tensors of any strides and lengths: the
// launchers of attention_rows.hip.
#pragma once

#include "common.hpp"

namespace gp {

// Rows [sequence, row, head, feature] with adjacent features; strides in bytes.
struct HeadRows {
    char* p = nullptr;
    long seq = 0, row = 0, head = 0;
    __host__ __device__ __forceinline__ char* at(int b, int i, int h) const { return p + b * seq + i * row + h * head; }
};

struct AttendArgs {
    int dtype = 0, B = 0, H = 0, HK = 0, Sq = 0, Sk = 0, dh = 0, causal = 0;
    float scale = 1.f;
    HeadRows q, k, v, o, dout, dq, dk, dv;
    float* lse = nullptr;           // [B, H, Sq], written by the forward
    const float* lse_in = nullptr;  // the same, read by the backward
    const int *q_lens = nullptr, *k_lens = nullptr, *q_starts = nullptr;
    const float* bias = nullptr;  // [H, buckets]
    const int* bucket_of = nullptr;
    int buckets = 0, max_distance = 0;
    float* dbias = nullptr;
    // set by the launchers
    int waves = 0, pack = 1, blocks = 0, splits = 1, stat_rows = 0;
    float* part = nullptr;   // splits' sums: [splits][B H Sq][width], then their (reference, sum) pairs
    f32x2* stats = nullptr;  // (lse / log 2, delta) of each row: [B, H, stat_rows]
    float* dist = nullptr;   // sums of dS by distance: [H][B blocks][2 max_distance + 1]
};

// Bytes of scratch, and the calls.  exact: delta from the probabilities, not from out.
size_t attend_workspace(const AttendArgs& a);
gp_status attend_forward(AttendArgs a, void* ws, hipStream_t st);
size_t attend_backward_workspace(const AttendArgs& a);
gp_status attend_backward(AttendArgs a, bool exact, void* ws, hipStream_t st);

} // namespace gp
