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
    int keys = 0, pack = 1, blocks = 0, splits = 1, stat_rows = 0;
    float* part = nullptr;   // splits' sums: [splits][B H Sq][width], the forward's then followed by their (reference, sum) pairs
    float* stats = nullptr;  // lse / log 2, then delta, of each row (negative, the first over the scale, where sums start from them): [B, H, 2, stat_rows]
    float* dist = nullptr;   // sums of dS by distance: [H][B blocks splits][2 max_distance + 1]
};

// How a kernel's work is split.
struct Shape {
    bool keys = false;  // few rows: the waves of a workgroup share them and take a part of the keys each
    int pack = 1;       // heads whose rows are packed together
    int blocks = 1;     // of rows
    int splits = 1;     // workgroups of one block
};
// The backward's dQ pass corrects delta for the rounding of out (attend_dq).
template <typename T> constexpr bool refines() { return sizeof(T) == 2; }
// Floats of the sums that n rows of splits of such a pass leave: dQ', R, two of each row; a multiple of 16 bytes.
constexpr size_t refined_floats(size_t n, size_t width) { return 2 * n * width + (2 * n + 3) / 4 * 4; }
constexpr int BW = 4;  // waves of the backward's workgroups
// Features that a kernel is made for: whole matrix blocks (4 x 2048, 16 heads, bf16 forward: 73 us at 32, 95 at 64, 130 at 96).
constexpr int head_bucket(int dh) { return (dh + 31) / 32 * 32; }
// Rows of a tile in LDS: 64 in bf16 (us at 32 / 64: 1000 queries to 50000 keys 455 / 432, backward of 4 x 2048 with a bias
// 367 / 350, of 64 x 256 149 / 143), in fp32 as many bytes.
constexpr int tile_rows(int esize) { return esize == 2 ? 64 : 32; }
// Tiles in LDS at a time: three where two workgroups of them fit a CU (dK and dV with two: 94 us for 85).
constexpr int stages(int width) { return width <= 64 ? 3 : 2; }
// Waves that share few rows, each with two tiles of keys and values of 32 rows in LDS: as many as 128 KB hold.
constexpr int key_waves(int row_bytes) { return row_bytes <= 128 ? 8 : row_bytes <= 256 ? 4 : 2; }

// The kernels for one type.
template <typename T> gp_status attend_forward_as(const AttendArgs& a, hipStream_t st);
template <typename T> gp_status attend_backward_as(const AttendArgs& a, bool exact, const Shape& dq, const Shape& dkv, hipStream_t st);

// Bytes of scratch, and the calls.  exact: delta from the probabilities, not from out.
size_t attend_workspace(const AttendArgs& a);
gp_status attend_forward(AttendArgs a, void* ws, hipStream_t st);
size_t attend_backward_workspace(const AttendArgs& a);
gp_status attend_backward(AttendArgs a, bool exact, void* ws, hipStream_t st);

} // namespace gp
