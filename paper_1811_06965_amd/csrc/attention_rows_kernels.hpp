// attention_rows_kernels.hpp -- attention on the caller's tensors: queries against
// keys of another length, ragged batches, heads that share keys, a learned
// relative position bias by buckets, and the gradients of all of them.
#pragma once

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <type_traits>

#include "attention_rows.hpp"
#include "common.hpp"
#include "gemm_tile.hpp"

namespace gp {

namespace {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
constexpr float NEVER = -1e30f;     // a bias down here is a mask's
constexpr float NO_REF = -FLT_MAX;  // the reference of a row that has seen no score
constexpr float AHEAD = 8.f;        // a row's sums change their reference when a score is 2^8 ahead of it

// 16 bytes of one row: the unit in which rows are staged and multiplied.
template <typename T> struct Elt;
template <> struct Elt<bf16> {
    typedef bf16x8 frag;
    static constexpr int E = 8;    // elements of a chunk
    static constexpr int RC = 64;  // features of a 128-byte row of an LDS tile
};
template <> struct Elt<float> {
    typedef f32x4 frag;
    static constexpr int E = 4, RC = 32;
};

// c += a b over two chunks of features (lanes 0-31 hold the first, 32-63 the second): one
// product of depth 16 in bf16, four of depth 2 in fp32, whose order of features is
// the same on both sides.
__device__ __forceinline__ f32x16 mma(const bf16x8& a, const bf16x8& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const f32x4& a, const f32x4& b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f32x16 splat16(float x) {
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = x;
    return z;
}
__device__ __forceinline__ f32x16 zero16() { return splat16(0.f); }
// The backward's products start from -lse / c and -delta, which saves their subtractions: in bf16, whose vector
// instructions bound it.  fp32's products take long, and each of their many sums would be rounded at the lse's size.
template <typename T> constexpr bool starts_sums() { return sizeof(T) == 2; }
// Row (within a block of 32) of accumulator register r; the column is lane % 32.
__device__ __forceinline__ int acc_row(int r, int lane) { return (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3); }

// An LDS tile of R rows x DH features: DH / RC parts of R rows of 128 bytes without padding.
// The 16-byte chunk c of row r lies at chunk c ^ swizzle(r) of its row: 16 lanes that read the
// same chunk of 16 consecutive rows, and a half-wave that reads four chunks of four
// consecutive rows (the transposing reads), then fall into distinct banks.
__device__ __forceinline__ int swizzle(int r) { return (((r >> 1) & 1) << 2) | ((r >> 2) & 3); }

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename T, int DH, int R> struct Tile {
    typedef Elt<T> X;
    typedef typename X::frag frag;
    static constexpr int PARTS = (DH + X::RC - 1) / X::RC, BYTES = R * PARTS * 128, LOADS = R * PARTS / 8;

    // Loads that one of W waves issues for a tile, 1 KB each straight into LDS: offset of this
    // lane's chunk in each, out of the buffer's range where the head is narrower than DH.
    template <int W> struct Loader {
        static_assert(LOADS % W == 0, "loads of a wave");
        static constexpr int N = LOADS / W;
        uint32_t off[N];
        __device__ __forceinline__ Loader(long row_bytes, int dh, int wave, int lane) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int n = wave * N + i, r = n % (R / 8) * 8 + (lane >> 3);
                const int f = n / (R / 8) * X::RC + ((lane & 7) ^ swizzle(r)) * X::E;
                off[i] = f < dh ? (uint32_t)(r * row_bytes) + f * (int)sizeof(T) : OOB;
            }
        }
        // Rows behind `rows` are filled with zeros (they lie behind the buffer's end).
        __device__ __forceinline__ void operator()(char* s, const char* p, int rows, long row_bytes, int dh, int wave) const {
            const Rsrc rs = make_rsrc(p, rows > 0 ? (uint32_t)((min(rows, R) - 1) * row_bytes) + dh * (int)sizeof(T) : 0u);
#pragma unroll
            for (int i = 0; i < N; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LdsPtr)(s + (wave * N + i) * 1024), 16, (int)off[i], 0, 0, 0);
        }
    };
    // Chunks 2 ks, 2 ks + 1 lie within the head; what lies behind it are zeros, which fp32's slow products leave out.
    static __device__ __forceinline__ bool has(int ks, int dh) { return sizeof(T) == 2 || 2 * ks * X::E < dh; }
    // Operand of 32 rows over the chunks 2 ks, 2 ks + 1 of features.
    static __device__ __forceinline__ frag rows(const char* s, int row0, int ks, int lane) {
        const int r = row0 + (lane & 31);
        return *reinterpret_cast<const frag*>(s + (ks >> 2) * (R * 128) + r * 128 + (((((ks & 3) << 1) | (lane >> 5)) ^ swizzle(r)) << 4));
    }
    // The tile's rows row0 .. row0 + 31 transposed, for acc (32 features x lane's column) += rows^T w, w the accumulator
    // registers whose rows those are.  In bf16 one transposing read gives a lane four rows of its feature.  The reads wait for
    // themselves: as builtins they count as writes, before which the compiler waits for the tiles on their way.
    template <int ND> struct Columns {
        bf16x8 x[2][ND];
        // of the 32 features from 32 first on
        __device__ __forceinline__ Columns(const char* s, int row0, int lane, int first = 0) {
            const int g = lane >> 4, q = lane & 15, r = row0 + 4 * (g >> 1) + (q >> 2), col = 16 * (g & 1) + 4 * (q & 3);
            const uint32_t at = (uint32_t)(size_t)(LdsPtr)s + r * 128 + (col & 7) * 2;
            // rows 8 on: swizzle ^ 2; features 32 on: chunk ^ 4; rows 16 on and parts of 64 features: a constant further
            const uint32_t a0 = (at + (((col >> 3) ^ swizzle(r)) << 4)) ^ ((first & 1) << 6), a1 = (a0 ^ 32) + 1024;
#pragma unroll
            for (int d = 0; d < ND; d += 2) {
                if (d + 1 < ND)
                    read(a0, a1, a0 ^ 64, a1 ^ 64, (first + d) / 2, x[0][d], x[1][d], x[0][d + 1], x[1][d + 1]);
                else
                    read(a0, a1, (first + d) / 2, x[0][d], x[1][d]);
            }
        }
        static __device__ __forceinline__ bf16x8 pair(i32x2 x, i32x2 y) { return __builtin_bit_cast(bf16x8, i32x4{x[0], x[1], y[0], y[1]}); }
        static __device__ __forceinline__ void read(uint32_t a0, uint32_t a1, int part, bf16x8& x0, bf16x8& x1) {
            i32x2 v[4];
            a0 += part * (R * 128);
            a1 += part * (R * 128);
            asm volatile("ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %5\n\tds_read_b64_tr_b16 %2, %4 offset:2048\n\t"
                         "ds_read_b64_tr_b16 %3, %5 offset:2048\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
                         : "v"(a0), "v"(a1));
            x0 = pair(v[0], v[1]);
            x1 = pair(v[2], v[3]);
        }
        static __device__ __forceinline__ void read(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1, int part, bf16x8& x0, bf16x8& x1,
                                                    bf16x8& y0, bf16x8& y1) {
            i32x2 v[8];
            a0 += part * (R * 128);
            a1 += part * (R * 128);
            b0 += part * (R * 128);
            b1 += part * (R * 128);
            asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %9\n\tds_read_b64_tr_b16 %2, %8 offset:2048\n\t"
                         "ds_read_b64_tr_b16 %3, %9 offset:2048\n\tds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %11\n\t"
                         "ds_read_b64_tr_b16 %6, %10 offset:2048\n\tds_read_b64_tr_b16 %7, %11 offset:2048\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
                         : "v"(a0), "v"(a1), "v"(b0), "v"(b1));
            x0 = pair(v[0], v[1]);
            x1 = pair(v[2], v[3]);
            y0 = pair(v[4], v[5]);
            y1 = pair(v[6], v[7]);
        }
    };
    static __device__ __forceinline__ float element(const char* s, int r, int d0, int lane) {
        return *reinterpret_cast<const float*>(s + (d0 >> 5) * (R * 128) + (lane & 3) * 4 + r * 128 +
                                               ((((lane & 31) >> 2) ^ swizzle(r)) << 4));
    }
    // acc += the tile's 32 rows from row0 on, transposed, times w.  In bf16 w is rounded, the matrix unit's type: by up to
    // 2^-8 of each weight, while their sums stay in fp32.
    // CAREFUL: without the pairs marked by a weight of -INFINITY: what a masked row holds, infinities and NaN included,
    // does not reach the sum.  The finite values are multiplied as always; two more products with weights of 1 find
    // where an unmasked pair holds +inf or -inf (a NaN counts as both), which is then added.
    template <bool CAREFUL, int ND>
    static __device__ __forceinline__ void add(const char* s, int row0, const f32x16& w, int lane, f32x16 (&acc)[ND]) {
        if constexpr (sizeof(T) == 2 && CAREFUL) {
#pragma unroll
            for (int d = 0; d < ND; ++d) {  // one by one, in fewer registers
                f32x16 one[1] = {acc[d]};
                add_columns<CAREFUL>(Columns<1>(s, row0, lane, d), w, one);
                acc[d] = one[0];
            }
        } else if constexpr (sizeof(T) == 2)
            add_columns<CAREFUL>(Columns<ND>(s, row0, lane), w, acc);
        else
            add_elements<CAREFUL>(s, row0, w, lane, acc);
    }
    // Two sums from one reading of the rows.  total += the sum of this lane's w as they are rounded.
    template <bool CAREFUL, int ND>
    static __device__ __forceinline__ void add(const char* s, int row0, const f32x16& w, const f32x16& w2, int lane, f32x16 (&acc)[ND],
                                               f32x16 (&acc2)[ND], float& total) {
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const auto rounded = [&](int i) { return (bf16)(CAREFUL && w[i] == -INFINITY ? 0.f : w[i]); };
            total = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{rounded(e), rounded(e + 1)}, bf16x2{(bf16)1.f, (bf16)1.f}, total, false);
        }
        static_assert(sizeof(T) == 2, "fp32 reads its elements one by one");
        if constexpr (CAREFUL) {
            add<CAREFUL>(s, row0, w, lane, acc);
            add<CAREFUL>(s, row0, w2, lane, acc2);
        } else {
            const Columns<ND> c(s, row0, lane);
            add_columns<CAREFUL>(c, w, acc);
            add_columns<CAREFUL>(c, w2, acc2);
        }
    }
    template <bool CAREFUL, int ND>
    static __device__ __forceinline__ void add_columns(const Columns<ND>& c, const f32x16& w, f32x16 (&acc)[ND]) {
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) {
            bf16x8 b, seen;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = w[8 * cc + e];
                b[e] = (bf16)(CAREFUL && x == -INFINITY ? 0.f : x);
                if (CAREFUL) seen[e] = (bf16)(x == -INFINITY ? 0.f : 1.f);
            }
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                if (!CAREFUL) {
                    acc[d] = mma(c.x[cc][d], b, acc[d]);
                    continue;
                }
                bf16x8 f;
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = (bf16)finite((float)c.x[cc][d][e]);
                acc[d] = mma(f, b, acc[d]);
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    const float inf = which ? -INFINITY : INFINITY;
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = (bf16)(infinite((float)c.x[cc][d][e], inf) ? 1.f : 0.f);
                    found(mma(f, seen, zero16()), inf, acc[d]);
                }
            }
        }
    }
    template <bool CAREFUL, int ND>
    static __device__ __forceinline__ void add_elements(const char* s, int row0, const f32x16& w, int lane, f32x16 (&acc)[ND]) {
#pragma unroll
        for (int cc = 0; cc < 2; ++cc)
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = w[8 * cc + e];
                    x[e] = element(s, row0 + acc_row(8 * cc + e, lane), d * 32, lane);
                    acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(CAREFUL ? finite(x[e]) : x[e], CAREFUL && y == -INFINITY ? 0.f : y, acc[d], 0, 0, 0);
                }
                if (!CAREFUL) continue;
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    const float inf = which ? -INFINITY : INFINITY;
                    f32x16 n = zero16();
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        n = __builtin_amdgcn_mfma_f32_32x32x2f32(infinite(x[e], inf) ? 1.f : 0.f, w[8 * cc + e] == -INFINITY ? 0.f : 1.f, n, 0, 0, 0);
                    found(n, inf, acc[d]);
                }
            }
    }
    static __device__ __forceinline__ float finite(float x) { return x - x == 0.f ? x : 0.f; }
    static __device__ __forceinline__ bool infinite(float x, float which) { return x == which || x != x; }
    static __device__ __forceinline__ void found(const f32x16& n, float inf, f32x16& acc) {
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] = n[e] > 0.f ? acc[e] + inf : acc[e];
    }
};

// Operand of 32 rows in memory: the chunk of each feature step of this lane's row (zeros where it has none).
template <typename T, int NK>
__device__ __forceinline__ void load_row(const char* row, bool live, int dh, int lane, typename Elt<T>::frag (&f)[NK]) {
    typedef Elt<T> X;
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) {
        const int c = (2 * ks + (lane >> 5)) * X::E;
        typename X::frag z = {};
        f[ks] = live && c < dh ? *reinterpret_cast<const typename X::frag*>(row + c * (int)sizeof(T)) : z;
    }
}
// This lane's row of a transposed accumulator (features x rows), times f, four features at a time.
template <typename T, int ND>
__device__ __forceinline__ void store_row(char* row, const f32x16 (&acc)[ND], float f, int dh, int lane) {
    typedef T vec __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
            const int d = db * 32 + rg * 8 + (lane >> 5) * 4;
            vec t;
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = to_elt<T>(f == 0.f ? 0.f : acc[db][4 * rg + e] * f);
            if (d < dh) *reinterpret_cast<vec*>(row + d * (int)sizeof(T)) = t;
        }
}

template <int ND> __device__ __forceinline__ bool all_finite(const f32x16 (&x)[ND]) {
    float z = 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) z = __builtin_fmaf(x[d][e], 0.f, z);
    return z == 0.f;
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Of lanes l and l + 32 both: the larger value, the sum.
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, WAVE); }
__device__ __forceinline__ float both_max(float x) { return fmaxf(x, other_half(x)); }
__device__ __forceinline__ float both_sum(float x) { return x + other_half(x); }

// Tiles in LDS at a time, all but one on their way; the ring's next place.
template <int ST> __device__ __forceinline__ int ring(int buf, int by) { return buf + by < ST ? buf + by : buf + by - ST; }

// Every LDS read of this wave has returned, and none is moved across.
__device__ __forceinline__ void lds_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Lengths and the position of the first query of one sequence.
struct Lens {
    int q, k, start;
    __device__ __forceinline__ Lens(const AttendArgs& a, int b) {
        q = a.q_lens ? min(max(a.q_lens[b], 0), a.Sq) : a.Sq;
        k = a.k_lens ? min(max(a.k_lens[b], 0), a.Sk) : a.Sk;
        // beyond 2^29 every key is further than any table reaches, on the same side
        start = a.q_starts ? min(max(a.q_starts[b], -(1 << 29)), 1 << 29) : 0;
    }
    // Keys that the query rows up to `last` may see.
    __device__ __forceinline__ int keys(bool causal, int last) const {
        return causal ? min(k, max(0, last + start + 1)) : k;
    }
};

// The bias of one head by distance, in LDS, in units of log 2: PAD further places on either side hold the outermost
// values, so that a block of 32 x 32 pairs that any distance of the table meets needs no clamping.  A bias of NEVER
// or less is -INFINITY.
constexpr int PAD = 64;
__device__ __forceinline__ int table_size(const AttendArgs& a) { return 2 * (a.max_distance + PAD) + 1; }
__device__ __forceinline__ bool load_table(float* t, const AttendArgs& a, int h, int tid, int threads) {
    bool masks = false;
    for (int i = tid; i < table_size(a); i += threads) {
        const int d = min(max(i - PAD, 0), 2 * a.max_distance);
        const float x = a.bias[(long)h * a.buckets + min(max(a.bucket_of[d], 0), a.buckets - 1)];
        t[i] = x <= NEVER ? -INFINITY : x * LOG2E;
        masks = masks || x <= NEVER;
    }
    return masks;
}
// One block of 32 x 32 pairs whose distances (key - position) go from lo to lo + 62 over the block: where they all lie
// beyond the table on one side, one value.  The branches on that and on masks are of whole blocks.
struct Near {
    bool far;
    float value;       // far: of every pair
    const float* at;   // near: of this lane's register 0; that of register r lies STEP * (row r - row 0) further
    __device__ __forceinline__ Near(const float* t, const AttendArgs& a, int lo, int mine) {
        far = lo >= a.max_distance || lo + 62 <= -a.max_distance;
        value = t[lo >= a.max_distance ? 2 * (a.max_distance + PAD) : 0];
        at = t + (far ? 0 : mine + a.max_distance + PAD);
    }
    // s = s c + bias
    template <int STEP> __device__ __forceinline__ void add(f32x16& s, float c) const {
        if (far) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], c, value);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], c, at[STEP * ((e >> 2) * 8 + (e & 3))]);
        }
    }
    // f(e) for the registers whose bias is a mask's
    template <int STEP, typename F> __device__ __forceinline__ void mask(F f) const {
        if (far) {
            if (value == -INFINITY) {
#pragma unroll
                for (int e = 0; e < 16; ++e) f(e);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (at[STEP * ((e >> 2) * 8 + (e & 3))] == -INFINITY) f(e);
        }
    }
};

// Workgroup -> (sequence, head, block of rows, split); the blocks of a head are neighbours on one XCD, whose L2 then
// serves its keys and values to all of them.  Causal blocks differ in length: each XCD (workgroups go to the eight in
// turn) takes an eighth of the heads, and the longest blocks of all of them first, so that none starts last
// (a bias, 4 x 2048 causal queries: 89 us head by head, 64 so; its backward 309 and 240).
enum Order { EVEN, LAST_LONGEST, FIRST_LONGEST };
struct Work {
    int b, h, blk, split;
    __device__ __forceinline__ Work(int blocks, int heads, int splits, Order order) {
        const int groups = (int)gridDim.x / (blocks * splits);
        if (order != EVEN && splits == 1 && groups % 8 == 0) {
            const int each = groups / 8, at = (int)blockIdx.x >> 3, g = (blockIdx.x & 7) * each + at % each;
            split = 0;
            blk = at / each;
            if (order == LAST_LONGEST) blk = blocks - 1 - blk;
            h = g % heads;
            b = g / heads;
            return;
        }
        int id = xcd_order(blockIdx.x, gridDim.x);
        split = id % splits;
        id /= splits;
        blk = id % blocks;
        if (order == LAST_LONGEST) blk = blocks - 1 - blk;
        id /= blocks;
        h = id % heads;
        b = id / heads;
    }
};

// ------------------------------------------------------------------ forward
// A wave owns 32 query rows and goes through the keys once, in tiles of KT that the workgroup's W waves stage in LDS,
// the next tile on its way while this one is used.  S^T = K Q^T puts a query's scores into one lane and its neighbour
// half a wave on, so that the softmax needs one exchange per tile; P^T is then already the operand of O^T += V^T P^T.
// Each row keeps its sums around a reference score, which follows the largest one only where that is 2^8 ahead: most
// tiles rescale nothing.  Bound by vector instructions and products: 4 x 2048 queries and keys, 16 heads of 64, bf16, 93 to 96 us (723
// TFLOP/s); 1000 queries to 50000 keys, width 128, 420 to 475 us from card to card (865 to 975); short loops by what surrounds them, 64 x 256
// to up to 320 keys 42 to 50 us.
// Few rows (KEYS): the W waves own the same 32 rows and every W-th tile each, without barriers, and join their sums in LDS: one
// token of 4 sequences of up to 200 keys 7.2 us (8.4 by one wave), of 16 of up to 32768 266 us (5.3 TB/s; 276).
template <typename T, int DH, int KT, int W, bool BIAS, bool KEYS>
__global__ void __launch_bounds__(64 * W) attend_fwd(AttendArgs a) {
    typedef Tile<T, DH, KT> Tl;
    constexpr int NK = DH / Elt<T>::E / 2, ND = DH / 32, NB = KT / 32, LW = KEYS ? 1 : W, ST = KEYS ? 2 : stages(DH);
    constexpr int TB = 2 * Tl::BYTES;  // a tile of keys and one of values
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    float* const table = reinterpret_cast<float*>(lds + (KEYS ? W : 1) * ST * TB);
    const int lane = threadIdx.x & 63, wave = uniform_wave_id(threadIdx.x);
    const Work wk(a.blocks, a.H / a.pack, a.splits, a.causal ? LAST_LONGEST : EVEN);
    const Lens len(a, wk.b);
    const int rows = a.Sq * a.pack, row0 = KEYS ? wk.blk * 32 : (wk.blk * W + wave) * 32, r = row0 + (lane & 31);
    const int i = a.pack == 1 ? r : r / a.pack, h = a.pack == 1 ? wk.h : wk.h * a.pack + (r - i * a.pack);
    const int hk = a.pack == 1 ? wk.h / (a.H / a.HK) : wk.h;
    const bool in = r < rows, live = in && i < len.q;
    const int pos = i + len.start, pos0 = row0 / a.pack + len.start;

    typename Elt<T>::frag qf[NK];
    load_row<T>(a.q.at(wk.b, min(i, a.Sq - 1), min(h, a.H - 1)), live, a.dh, lane, qf);

    // keys that any row of the workgroup, and of this wave, may see
    auto reach = [&](int first, int end) {
        return first >= rows || first / a.pack >= len.q ? 0 : len.keys(a.causal, (min(end, rows) - 1) / a.pack);
    };
    const int kw = reach(row0, row0 + 32);
    const int tiles = ((KEYS ? kw : reach(wk.blk * W * 32, (wk.blk + 1) * W * 32)) + KT - 1) / KT;
    const int t0 = (int)((long)tiles * wk.split / a.splits), t1 = (int)((long)tiles * (wk.split + 1) / a.splits);
    const char *kp = a.k.at(wk.b, 0, hk), *vp = a.v.at(wk.b, 0, hk);
    const typename Tl::template Loader<LW> kl(a.k.row, a.dh, KEYS ? 0 : wave, lane), vl(a.v.row, a.dh, KEYS ? 0 : wave, lane);
    const int own = KEYS ? wave : 0, step = KEYS ? W : 1;  // tiles of this wave: from t0 + own on, every step-th
    char* const base = lds + own * ST * TB;
    auto stage = [&](int t, int buf) {
        char* s = base + buf * TB;
        kl(s, kp + (long)t * KT * a.k.row, len.k - t * KT, a.k.row, a.dh, KEYS ? 0 : wave);
        vl(s + Tl::BYTES, vp + (long)t * KT * a.v.row, len.k - t * KT, a.v.row, a.dh, KEYS ? 0 : wave);
    };

    auto first_tiles = [&] {
#pragma unroll
        for (int x = 0; x < ST - 1; ++x)
            if (t0 + own + x * step < t1) stage(t0 + own + x * step, x);
    };
    first_tiles();  // on their way while the table is made
    bool masks = false;
    if (BIAS) masks = __syncthreads_or(load_table(table, a, wk.h, threadIdx.x, 64 * W));
    const float c = a.scale * LOG2E;
    float m, l;
    f32x16 o[ND];
    // A product of a masked pair's weight 0 with an infinity or a NaN is a NaN: where a mask may lie inside a block and
    // something not finite came out, a second, careful pass leaves those products out.
    auto pass = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        m = NO_REF;
        l = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] = zero16();
        for (int t = t0 + own, buf = 0; t < t1; t += step, buf = ring<ST>(buf, 1)) {
            if (ST > 2 && t + step < t1) wait_vmcnt<2 * decltype(kl)::N>(); else wait_vmcnt<0>();
            if (KEYS) lds_reads_done(); else lds_barrier();
            if (t + (ST - 1) * step < t1) stage(t + (ST - 1) * step, ring<ST>(buf, ST - 1));
            if (t * KT >= kw) continue;
            const char *ks = base + buf * TB, *vs = ks + Tl::BYTES;
            f32x16 s[NB];
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                s[kb] = zero16();
#pragma unroll
                for (int x = 0; x < NK; ++x)
                    if (Tl::has(x, a.dh)) s[kb] = mma(Tl::rows(ks, kb * 32, x, lane), qf[x], s[kb]);
            }
            const bool edge = t * KT + KT > len.k || (a.causal && t * KT + KT - 1 > pos0);
            float tm = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                const int k0 = t * KT + kb * 32;
                if (BIAS) {
                    const Near n(table, a, k0 - pos0 - 31, k0 + 4 * (lane >> 5) - pos);
                    n.add<1>(s[kb], c);
                    if (masks) n.mask<1>([&](int e) { s[kb][e] = -INFINITY; });
                }
                if (edge) {
                    const int last = a.causal ? min(len.k - 1, pos) : len.k - 1;
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (k0 + acc_row(e, lane) > last) s[kb][e] = -INFINITY;
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) tm = fmaxf(tm, s[kb][e]);
            }
            tm = both_max(BIAS ? tm : tm * c);
            if (__any(tm > m + AHEAD)) {
                const float mn = fmaxf(m, tm), f = exp2_hw(m - mn);
                m = mn;
                l *= f;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[d][e] *= f;
            }
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float x = s[kb][e], p = exp2_hw(BIAS ? x - m : __builtin_fmaf(x, c, -m));
                    sum[e & 3] += p;
                    s[kb][e] = CAREFUL && x == -INFINITY ? x : p;
                }
                Tl::template add<CAREFUL>(vs, kb * 32, s[kb], lane, o);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        }
    };
    pass(std::false_type{});
    if (a.causal || masks) {
        if (__syncthreads_or(!all_finite(o))) {
            first_tiles();
            pass(std::true_type{});
        }
    }
    l = both_sum(l);
    if constexpr (KEYS) {
        lds_reads_done();
        float* sums = reinterpret_cast<float*>(base);  // [row][DH], in place of this wave's tiles
        f32x2* stat = reinterpret_cast<f32x2*>(lds + W * ST * TB + (BIAS ? table_size(a) * 4 + 4 : 0)) + wave * 32;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int rg = 0; rg < 4; ++rg)
                *reinterpret_cast<f32x4*>(sums + (lane & 31) * DH + d * 32 + rg * 8 + (lane >> 5) * 4) =
                    f32x4{o[d][4 * rg], o[d][4 * rg + 1], o[d][4 * rg + 2], o[d][4 * rg + 3]};
        if (lane < 32) stat[lane] = f32x2{m, l};
        __syncthreads();
        stat -= wave * 32;
        for (int x = threadIdx.x; x < 32 * (DH / 4); x += 64 * W) {
            const int row = x / (DH / 4), d = x % (DH / 4) * 4, rr = row0 + row;
            if (rr >= rows) break;
            float M = NO_REF, L = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) M = fmaxf(M, stat[w * 32 + row][0]);
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const f32x2 y = stat[w * 32 + row];
                const float f = exp2_hw(y[0] - M);
                const f32x4 v = *reinterpret_cast<const f32x4*>(lds + w * ST * TB + (row * DH + d) * 4);
                L = __builtin_fmaf(y[1], f, L);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] = __builtin_fmaf(v[e], f, sum[e]);
            }
            const int qi = rr / a.pack, qh = wk.h * a.pack + rr - qi * a.pack;
            if (a.splits > 1) {
                const long at = ((long)wk.b * (a.H / a.pack) + wk.h) * rows + rr, n = (long)a.B * a.H * a.Sq;
                *reinterpret_cast<f32x4*>(a.part + (wk.split * n + at) * DH + d) = sum;
                if (d == 0) reinterpret_cast<f32x2*>(a.part + a.splits * n * DH)[wk.split * n + at] = f32x2{M, L};
                continue;
            }
            const bool none = L == 0.f || qi >= len.q;
            typedef T vec __attribute__((ext_vector_type(4)));
            vec out;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = to_elt<T>(none ? 0.f : sum[e] / L);
            if (d < a.dh) *reinterpret_cast<vec*>(a.o.at(wk.b, qi, qh) + d * (int)sizeof(T)) = out;
            if (a.lse && d == 0) a.lse[((long)wk.b * a.H + qh) * a.Sq + qi] = none ? -INFINITY : M * LN2 + logf(L);
        }
        return;
    }
    if (!in) return;
    if (a.splits > 1) {
        const long row = ((long)wk.b * (a.H / a.pack) + wk.h) * rows + r, n = (long)a.B * a.H * a.Sq;
        float* p = a.part + (wk.split * n + row) * DH;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int rg = 0; rg < 4; ++rg)
                *reinterpret_cast<f32x4*>(p + d * 32 + rg * 8 + (lane >> 5) * 4) =
                    f32x4{o[d][4 * rg], o[d][4 * rg + 1], o[d][4 * rg + 2], o[d][4 * rg + 3]};
        if (lane < 32) reinterpret_cast<f32x2*>(a.part + a.splits * n * DH)[wk.split * n + row] = f32x2{m, l};
        return;
    }
    const bool none = l == 0.f || !live;
    store_row<T, ND>(a.o.at(wk.b, i, h), o, none ? 0.f : 1.f / l, a.dh, lane);
    if (a.lse && lane < 32) a.lse[((long)wk.b * a.H + h) * a.Sq + i] = none ? -INFINITY : m * LN2 + logf(l);
}

// Joins the splits of a row: out = sum 2^(m_s - m) O_s / sum 2^(m_s - m) l_s.  A wave per row.
template <typename T, int DH>
__global__ void __launch_bounds__(256) attend_join(AttendArgs a) {
    const int lane = threadIdx.x & 63;
    const long n = (long)a.B * a.H * a.Sq, row = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= n) return;
    const f32x2* st = reinterpret_cast<const f32x2*>(a.part + a.splits * n * DH);
    const int rows = a.Sq * a.pack;
    const long group = row / rows;
    const int r = (int)(row - group * rows), i = r / a.pack, heads = a.H / a.pack;
    const int b = (int)(group / heads), h = (int)(group % heads) * a.pack + r % a.pack;
    // a split per lane (there are at most 64)
    const f32x2 x = lane < a.splits ? st[lane * n + row] : f32x2{NO_REF, 0.f};
    const float m = wave_max(x[0]), mine = lane < a.splits ? exp2_hw(x[0] - m) : 0.f, l = wave_sum(x[1] * mine);
    constexpr int N = (DH + 63) / 64;
    float o[N] = {};
    for (int s0 = 0; s0 < a.splits; s0 += 8) {  // eight on their way at a time; lanes behind the last split hold a weight of 0
        float v[8][N];
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int d = 0; d < N; ++d)
                v[u][d] = s0 + u < a.splits && (DH % 64 == 0 || d * 64 + lane < DH) ? a.part[((s0 + u) * n + row) * DH + d * 64 + lane] : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float f = __shfl(mine, s0 + u, WAVE);
#pragma unroll
            for (int d = 0; d < N; ++d) o[d] = __builtin_fmaf(v[u][d], f, o[d]);
        }
    }
    const Lens len(a, b);
    const bool none = l == 0.f || i >= len.q;
    T* out = reinterpret_cast<T*>(a.o.at(b, i, h));
#pragma unroll
    for (int d = 0; d < N; ++d)
        if (d * 64 + lane < a.dh) out[d * 64 + lane] = to_elt<T>(none ? 0.f : o[d] / l);
    if (a.lse && lane == 0) a.lse[((long)b * a.H + h) * a.Sq + i] = none ? -INFINITY : m * LN2 + logf(l);
}

// ----------------------------------------------------------------- backward
// The sums of dS over one distance each, for one wave.  A block's 32 x 32 values go to LDS with each query row one
// place further left than the one before, so that a distance is a column, which one lane adds up from top to bottom:
// no atomics, one order.  Distances beyond the table are added in registers.
constexpr int SKEW = 32 * 64;  // floats of a wave's block
struct Distances {
    float *skew, *sums, low, high;
    int D, lane;
    __device__ __forceinline__ Distances(float* base, int D_, int wave, int waves, int lane_) : D(D_), lane(lane_) {
        skew = base + wave * SKEW;
        sums = base + waves * SKEW + wave * (2 * D + 1);
        low = high = 0.f;
    }
    __device__ __forceinline__ void clear() {
        for (int i = lane; i < SKEW; i += WAVE) skew[i] = 0.f;
        for (int i = lane; i < 2 * D + 1; i += WAVE) sums[i] = 0.f;
        low = high = 0.f;
    }
    // lo: distance of the block's first key from its last query.  MARKED: a pair of -INFINITY is a masked one
    template <bool MARKED> __device__ __forceinline__ void add(const f32x16& ds, int lo) {
#pragma clang fp contract(off)
        const auto value = [](float x) { return MARKED && x == -INFINITY ? 0.f : x; };
        if (lo >= D || lo + 62 <= -D) {
            float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e & 3] += value(ds[e]);
            const float x = (s[0] + s[1]) + (s[2] + s[3]);
            if (lo >= D) high += x; else low += x;
            return;
        }
        float* p = skew + 4 * (lane >> 5) * 63 + 31 + (lane & 31);  // query row r of the block, key lane % 32: row r, place 31 - r + key
#pragma unroll
        for (int e = 0; e < 16; ++e) p[((e >> 2) * 8 + (e & 3)) * 63] = value(ds[e]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int i = 0; i < 32; i += 8)  // in steps: few registers
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j & 3] += skew[(i + j) * 64 + lane];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const float x = (s[0] + s[1]) + (s[2] + s[3]);
        const int rel = lo + lane;  // lane 63 has no pairs
        if (rel <= -D) low += x;
        else if (rel >= D) high += x;
        else sums[rel + D] += x;
    }
    __device__ __forceinline__ void finish() {
        const float a = wave_sum(low), b = wave_sum(high);
        if (lane == 0) {
            sums[0] += a;
            sums[2 * D] += b;
        }
    }
};

// dQ: a wave owns 32 queries and goes through the keys as the forward does:
//   P = 2^(S - lse), dP^T = V dO^T, dS = P (dP - delta), dQ^T += K^T dS^T.
// delta_i = sum_j P_ij dP_ij = dO_i . O_i.  O in bf16 is off by up to 2^-8 of itself, and so would be each row's sum of dS, which all
// the row's pairs share, dQ multiplies by the row's mean key and the bias's gradient adds up.  So delta is made
//   FROM_OUT: by the second form (fp32);
//   FROM_WEIGHTS: by the first, in a pass of its own over the keys (calls without O);
//   REFINED (bf16): by the second, d, and with the sums of dS' = P (dP - d), which are the error e = delta - d (the weights add
//   up to 1), and dQ'^T = K^T dS'^T, R^T = K^T P^T, dQ = dQ' - e R: one product for the three, and the
//   exponential, of a pass of its own.  The sum taken off dQ is that of dS' as it was rounded: the exact dS of a row add up to 0, so what
//   the rounding has in common with the row's mean key R goes too.  Errors against 64 bits, by O / by the weights / refined, of random
//   inputs: dQ 0.0028 / 0.0025 / 0.0023, with 7 keys 0.0038 / 0.0025 / 0.0023; where keys and values have means of 3 and 6 times
//   their spread dQ 0.28 / 0.0056 / 0.0023, dK 0.011 / 0.0023 / 0.0023.  us of a backward, 4 x 2048 queries, 16 heads, by O / by the
//   weights / refined: 192 / 243 / 208 at width 32, 275 / 340 / 301 at 64, 382 / 470 / 418 at 96, 548 / 664 / 681 at 128; with a bias by the
//   weights / refined 298 / 260, 392 / 348, 655 / 592, 768 / 800; 64 x 256 queries to 320 keys 152 / 157 / 157 at 64, 352 / 372 / 404 at
//   128, whose registers leave one wave a SIMD.  Splits of a row's keys leave their sums to attend_refine.
// Writes (lse, delta) of each row for dK and dV.
enum Delta { FROM_OUT, FROM_WEIGHTS, REFINED };
template <typename T, int DH, int KT, int W, bool BIAS, int DELTA>
__global__ void __launch_bounds__(64 * W) attend_dq(AttendArgs a) {
    typedef Tile<T, DH, KT> Tl;
    constexpr int NK = DH / Elt<T>::E / 2, ND = DH / 32, NB = KT / 32, ST = stages(DH), TB = 2 * Tl::BYTES;
    // beyond 64 its registers cost the second wave (592 us for 684 at 96 with a bias)
    constexpr bool INIT = starts_sums<T>() && (BIAS || DELTA == REFINED) && DH <= 64;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    float* const table = reinterpret_cast<float*>(lds + ST * TB);
    const int lane = threadIdx.x & 63, wave = uniform_wave_id(threadIdx.x);
    const Work wk(a.blocks, a.H, a.splits, a.causal ? LAST_LONGEST : EVEN);
    const Lens len(a, wk.b);
    const int row0 = (wk.blk * W + wave) * 32, i = row0 + (lane & 31), hk = wk.h / (a.H / a.HK);
    const bool in = i < a.Sq, live = i < len.q;
    const int pos = i + len.start, pos0 = row0 + len.start;
    const long stat = ((long)wk.b * a.H + wk.h) * 2 * a.stat_rows;

    typename Elt<T>::frag qf[NK], gf[NK];
    const int ic = min(i, a.Sq - 1);
    load_row<T>(a.q.at(wk.b, ic, wk.h), live, a.dh, lane, qf);
    load_row<T>(a.dout.at(wk.b, ic, wk.h), live, a.dh, lane, gf);
    float delta = 0.f;
    if (DELTA != FROM_WEIGHTS) {
        typename Elt<T>::frag of[NK];
        load_row<T>(a.o.at(wk.b, ic, wk.h), live, a.dh, lane, of);
#pragma unroll
        for (int x = 0; x < NK; ++x)
#pragma unroll
            for (int e = 0; e < Elt<T>::E; ++e) delta = __builtin_fmaf(to_f32((T)of[x][e]), to_f32((T)gf[x][e]), delta);
        delta = both_sum(delta);
    }
    // a row that sees nothing has weights of 0: its lse is taken as +inf
    float lse2 = live ? a.lse_in[((long)wk.b * a.H + wk.h) * a.Sq + ic] * LOG2E : INFINITY;
    if (lse2 == -INFINITY) lse2 = INFINITY;

    auto reach = [&](int first, int end) { return first >= len.q ? 0 : len.keys(a.causal, min(end, a.Sq) - 1); };
    const int kw = reach(row0, row0 + 32);
    const int tiles = (reach(wk.blk * W * 32, (wk.blk + 1) * W * 32) + KT - 1) / KT;
    const int t0 = (int)((long)tiles * wk.split / a.splits), t1 = (int)((long)tiles * (wk.split + 1) / a.splits);
    const char *kp = a.k.at(wk.b, 0, hk), *vp = a.v.at(wk.b, 0, hk);
    const typename Tl::template Loader<W> kl(a.k.row, a.dh, wave, lane), vl(a.v.row, a.dh, wave, lane);
    auto stage = [&](int t, int buf) {
        char* s = lds + buf * TB;
        kl(s, kp + (long)t * KT * a.k.row, len.k - t * KT, a.k.row, a.dh, wave);
        vl(s + Tl::BYTES, vp + (long)t * KT * a.v.row, len.k - t * KT, a.v.row, a.dh, wave);
    };
    auto first_tiles = [&](int t, int end) {
#pragma unroll
        for (int x = 0; x < ST - 1; ++x)
            if (t + x < end) stage(t + x, x);
    };
    auto next_tile = [&](int t, int end, int buf) {  // tile t is there; the one ST - 1 on is sent for
        if (ST > 2 && t + 1 < end) wait_vmcnt<2 * decltype(kl)::N>(); else wait_vmcnt<0>();
        lds_barrier();
        if (t + ST - 1 < end) stage(t + ST - 1, ring<ST>(buf, ST - 1));
    };
    if (DELTA == FROM_WEIGHTS) first_tiles(0, tiles); else first_tiles(t0, t1);  // on their way while the table is made
    bool masks = false;
    if (BIAS) masks = __syncthreads_or(load_table(table, a, wk.h, threadIdx.x, 64 * W));
    const float c = a.scale * LOG2E;
    const f32x16 s0 = splat16(INIT ? -lse2 / c : 0.f);
    // the weights of one block (s) and dP from dp0 on (dp); -INFINITY marks a masked pair's weight where `mark` asks for it
    auto block = [&](const char* ks, const char* vs, int k0, int kb, bool edge, bool mark, const f32x16& dp0, f32x16& s, f32x16& dp) {
        s = s0;
        dp = dp0;
#pragma unroll
        for (int x = 0; x < NK; ++x) {
            if (!Tl::has(x, a.dh)) continue;
            s = mma(Tl::rows(ks, kb * 32, x, lane), qf[x], s);
            dp = mma(Tl::rows(vs, kb * 32, x, lane), gf[x], dp);
        }
        const Near n(table, a, BIAS ? k0 - pos0 - 31 : 0, BIAS ? k0 + 4 * (lane >> 5) - pos : 0);
        if (BIAS) n.add<1>(s, c);
#pragma unroll
        for (int e = 0; e < 16; ++e)
            s[e] = exp2_hw(INIT ? (BIAS ? s[e] : s[e] * c) : BIAS ? s[e] - lse2 : __builtin_fmaf(s[e], c, -lse2));
        auto hide = [&](int e) {
            s[e] = mark ? -INFINITY : 0.f;
            dp[e] = 0.f;
        };
        if (edge) {
            const int last = !live ? -1 : a.causal ? min(len.k - 1, pos) : len.k - 1;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (k0 + acc_row(e, lane) > last) hide(e);
        }
        if (BIAS && masks) n.mask<1>(hide);
    };
    const bool short_rows = row0 + 32 > len.q;  // a row that is not in use has no weights, whatever the keys hold
    auto tile_edge = [&](int t) { return short_rows || t * KT + KT > len.k || (a.causal && t * KT + KT - 1 > pos0); };
    if (DELTA == FROM_WEIGHTS) {
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        for (int t = 0, buf = 0; t < tiles; ++t, buf = ring<ST>(buf, 1)) {
            next_tile(t, tiles, buf);
            if (t * KT >= kw) continue;
            const char *ks = lds + buf * TB, *vs = ks + Tl::BYTES;
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                f32x16 s, dp;
                block(ks, vs, t * KT + kb * 32, kb, tile_edge(t), false, zero16(), s, dp);
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[e & 3] = __builtin_fmaf(s[e], dp[e], sum[e & 3]);
            }
        }
        delta = both_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
        lds_barrier();
        first_tiles(t0, t1);
    }
    const f32x16 dp0 = splat16(INIT ? -delta : 0.f);
    f32x16 dq[ND], r[DELTA == REFINED ? ND : 1];
    float error = 0.f, rounded = 0.f;  // sums of dS, and of dS as it is multiplied
    auto pass = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        error = rounded = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d) dq[d] = r[DELTA == REFINED ? d : 0] = zero16();
        for (int t = t0, buf = 0; t < t1; ++t, buf = ring<ST>(buf, 1)) {
            next_tile(t, t1, buf);
            if (t * KT >= kw) continue;
            const char *ks = lds + buf * TB, *vs = ks + Tl::BYTES;
            const bool edge = tile_edge(t);
#pragma unroll 1
            for (int kb = 0; kb < NB; ++kb) {
                f32x16 s, dp;
                block(ks, vs, t * KT + kb * 32, kb, edge, CAREFUL, dp0, s, dp);
                f32x16 ds;
                float sum[2] = {0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    // Sums of dS are of its rounded products in every pass, not fused with them in those that mark nothing: else what a masked
                    // pair holds, by which the careful pass is taken, would change their last bits.
#pragma clang fp contract(off)
                    ds[e] = s[e] * (INIT ? dp[e] : dp[e] - delta);
                    if (CAREFUL) ds[e] = s[e] == -INFINITY ? s[e] : ds[e] == -INFINITY ? NAN : ds[e];
                    if (DELTA == REFINED) sum[e & 1] += CAREFUL && s[e] == -INFINITY ? 0.f : ds[e];
                }
                error += sum[0] + sum[1];
                if constexpr (DELTA == REFINED)
                    Tl::template add<CAREFUL>(ks, kb * 32, ds, s, lane, dq, r, rounded);
                else
                    Tl::template add<CAREFUL>(ks, kb * 32, ds, lane, dq);
            }
        }
    };
    pass(std::false_type{});
    if (a.causal || masks) {
        if (__syncthreads_or(!all_finite(dq))) {
            first_tiles(t0, t1);
            pass(std::true_type{});
        }
    }
    const long n = (long)a.B * a.H * a.Sq, row = ((long)wk.b * a.H + wk.h) * a.Sq + i;  // of the splits' sums
    if constexpr (DELTA == REFINED) {
        error = both_sum(error);
        rounded = both_sum(rounded);
        if (a.splits > 1) {  // attend_refine does the rest
            if (in) {
                store_row<float, ND>(reinterpret_cast<char*>(a.part + ((a.splits + wk.split) * n + row) * DH), r, live ? 1.f : 0.f, DH, lane);
                if (lane < 32) reinterpret_cast<f32x2*>(a.part + 2 * a.splits * n * DH)[wk.split * n + row] = f32x2{live ? error : 0.f, live ? rounded : 0.f};
            }
        } else {
            delta += error;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) dq[d][e] = __builtin_fmaf(-rounded, r[d][e], dq[d][e]);
        }
    }
    if (in && a.splits > 1)
        store_row<float, ND>(reinterpret_cast<char*>(a.part + (wk.split * n + row) * DH), dq, live ? 1.f : 0.f, DH, lane);
    else if (in)
        store_row<T, ND>(a.dq.at(wk.b, i, wk.h), dq, live ? a.scale : 0.f, a.dh, lane);
    if (wk.split == 0 && lane < 32 && i < a.stat_rows) {
        a.stats[stat + i] = starts_sums<T>() ? -lse2 / c : lse2;
        a.stats[stat + a.stat_rows + i] = starts_sums<T>() ? -delta : delta;
    }
}

// The rows of dQ, and their deltas, from the splits' sums of a refined pass: dQ', R = sum P k, and (the error of delta, the sum of the
// rounded dS').  Four features a thread.
template <typename T, int DH> __global__ void __launch_bounds__(256) attend_refine(AttendArgs a) {
    const long n = (long)a.B * a.H * a.Sq, x = (long)blockIdx.x * 256 + threadIdx.x, row = x / (DH / 4);
    const int d = (int)(x % (DH / 4)) * 4;
    if (row >= n || d >= a.dh) return;
    const f32x2* sums = reinterpret_cast<const f32x2*>(a.part + 2 * a.splits * n * DH);
    f32x4 dq = {0.f, 0.f, 0.f, 0.f}, r = {0.f, 0.f, 0.f, 0.f};
    float error = 0.f, rounded = 0.f;
#pragma unroll 4
    for (int i = 0; i < a.splits; ++i) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(a.part + (i * n + row) * DH + d);
        const f32x4 w = *reinterpret_cast<const f32x4*>(a.part + ((a.splits + i) * n + row) * DH + d);
        const f32x2 y = sums[i * n + row];
        error += y[0];
        rounded += y[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            dq[e] += v[e];
            r[e] += w[e];
        }
    }
    typedef T vec __attribute__((ext_vector_type(4)));
    vec t;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = to_elt<T>(__builtin_fmaf(-rounded, r[e], dq[e]) * a.scale);
    const long group = row / a.Sq;
    const int i = (int)(row - group * a.Sq);
    *reinterpret_cast<vec*>(a.dq.at((int)(group / a.H), i, (int)(group % a.H)) + d * (int)sizeof(T)) = t;
    if (d == 0) a.stats[group * 2 * a.stat_rows + a.stat_rows + i] -= error;  // -delta
}

// dK and dV: a wave owns 32 keys and goes through the queries of all the heads that share them, in tiles of QT:
//   S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS,
// and dS by distance for the bias's gradient.  Bound by vector instructions and products, at two waves a SIMD: 4 x 2048, 16 heads of 64,
// bf16, 194 us with a bias, 45 of them for the distances; 64 x 256 queries to up to 320 keys 81 us.  In fp32 at 36 to 64 wide two waves
// keep 5 registers in memory (33 with a bias) that one would not, yet take less: backward of 8 x 512, 16 heads of 64, 249 us for 266, with a bias
// 285 for 304, 2 x 2048 896 for 961; of 2 x 2048 causal ones, whose workgroups are fewer, 695 for 616.
template <typename T, int DH, int QT, int W, bool BIAS>
__global__ void __launch_bounds__(64 * W, DH <= 64 ? 2 : 1) attend_dkv(AttendArgs a) {
    typedef Tile<T, DH, QT> Tl;
    constexpr int NK = DH / Elt<T>::E / 2, ND = DH / 32, NB = QT / 32, ST = BIAS ? 2 : stages(DH), TB = 2 * Tl::BYTES;
    constexpr bool INIT = starts_sums<T>();
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    float* const stats = reinterpret_cast<float*>(lds + ST * TB);  // of the tiles' rows: two planes of 64
    float* const table = stats + ST * 128;
    const int lane = threadIdx.x & 63, wave = uniform_wave_id(threadIdx.x);
    const Work wk(a.blocks, a.HK, a.splits, a.causal ? FIRST_LONGEST : EVEN);
    const Lens len(a, wk.b);
    const int group = a.H / a.HK, k0 = (wk.blk * W + wave) * 32, key = k0 + (lane & 31);
    const bool in = key < a.Sk, live = key < len.k;

    typename Elt<T>::frag kf[NK], vf[NK];
    const int kc = min(key, a.Sk - 1);
    load_row<T>(a.k.at(wk.b, kc, wk.h), live, a.dh, lane, kf);
    load_row<T>(a.v.at(wk.b, kc, wk.h), live, a.dh, lane, vf);

    // query tiles that see any key of the workgroup
    const int first = wk.blk * W * 32, t1 = first < len.k ? (len.q + QT - 1) / QT : 0;
    const int t0 = a.causal ? min(max(first - len.start, 0) / QT, t1) : 0;
    // this split's share of the tiles of all the heads
    const long all = (long)group * (t1 - t0), u0 = all * wk.split / a.splits, u1 = all * (wk.split + 1) / a.splits;
    const typename Tl::template Loader<W> ql(a.q.row, a.dh, wave, lane), gl(a.dout.row, a.dh, wave, lane);
    const float c = a.scale * LOG2E;
    bool masks = false;
    Distances dist(table + (BIAS ? table_size(a) : 0), a.max_distance, wave, W, lane);
    const int distances = 2 * a.max_distance + 1;
    f32x16 dk[ND], dv[ND];
    auto pass = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
#pragma unroll
        for (int d = 0; d < ND; ++d) dk[d] = dv[d] = zero16();
        for (int g = 0; g < group; ++g) {
            const long at = (long)g * (t1 - t0);  // of this head's first tile
            const int ta = t0 + (int)max(0l, u0 - at), tb = t0 + (int)min((long)(t1 - t0), u1 - at);
            const int h = wk.h * group + g;
            float* const dist_out = BIAS ? a.dist + ((((long)h * a.B + wk.b) * a.blocks + wk.blk) * a.splits + wk.split) * distances : nullptr;
            if (ta >= tb) {
                if (BIAS && a.dist)
                    for (int x = threadIdx.x; x < distances; x += 64 * W) dist_out[x] = 0.f;
                continue;
            }
            const char *qp = a.q.at(wk.b, 0, h), *gp = a.dout.at(wk.b, 0, h);
            const float* sp = a.stats + ((long)wk.b * a.H + h) * 2 * a.stat_rows;
            auto stage = [&](int t, int buf) {
                char* s = lds + buf * TB;
                ql(s, qp + (long)t * QT * a.q.row, len.q - t * QT, a.q.row, a.dh, wave);
                gl(s + Tl::BYTES, gp + (long)t * QT * a.dout.row, len.q - t * QT, a.dout.row, a.dh, wave);
                // a plane a load (zeros behind QT rows); each wave issues one, so that all have as many on their way
                const int plane = wave & 1;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(sp + plane * a.stat_rows + t * QT, QT * 4), (LdsPtr)(stats + buf * 128 + plane * 64),
                                                         4, lane * 4, 0, 0, 0);
            };
            __syncthreads();  // the last head's tiles are done with
#pragma unroll
            for (int x = 0; x < ST - 1; ++x)
                if (ta + x < tb) stage(ta + x, x);
            if (BIAS) masks = masks | (__syncthreads_or(load_table(table, a, h, threadIdx.x, 64 * W)) != 0);
            if (BIAS && a.dist) dist.clear();
            for (int t = ta, buf = 0; t < tb; ++t, buf = ring<ST>(buf, 1)) {
                if (ST > 2 && t + 1 < tb) wait_vmcnt<2 * decltype(ql)::N + 1>(); else wait_vmcnt<0>();
                lds_barrier();
                if (t + ST - 1 < tb) stage(t + ST - 1, ring<ST>(buf, ST - 1));
                const int pos0 = t * QT + len.start;
                if (k0 >= len.k || (a.causal && pos0 + QT - 1 < k0)) continue;
                const char *qs = lds + buf * TB, *gs = qs + Tl::BYTES;
                const bool edge = t * QT + QT > len.q || k0 + 32 > len.k || (a.causal && pos0 < k0 + 31);
#pragma unroll 1
                for (int qb = 0; qb < NB; ++qb) {
                    // rows of the registers: (reference, delta) as the dQ kernel left them
                    const float* st = stats + buf * 128 + qb * 32 + 4 * (lane >> 5);
                    f32x16 lse, delta;
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const f32x4 x = *reinterpret_cast<const f32x4*>(st + 2 * e), y = *reinterpret_cast<const f32x4*>(st + 64 + 2 * e);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            lse[e + k] = x[k];
                            delta[e + k] = y[k];
                        }
                    }
                    f32x16 s = INIT ? lse : zero16(), dp = INIT ? delta : zero16();
#pragma unroll
                    for (int x = 0; x < NK; ++x) {
                        if (!Tl::has(x, a.dh)) continue;
                        s = mma(Tl::rows(qs, qb * 32, x, lane), kf[x], s);
                        dp = mma(Tl::rows(gs, qb * 32, x, lane), vf[x], dp);
                    }
                    const int p0 = pos0 + qb * 32;
                    // distances fall with the register here
                    const Near n(table, a, BIAS ? k0 - p0 - 31 : 0, BIAS ? key - p0 - 4 * (lane >> 5) : 0);
                    f32x16 ds;
                    if (BIAS) n.add<-1>(s, c);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        s[e] = exp2_hw(INIT ? (BIAS ? s[e] : s[e] * c) : BIAS ? s[e] - lse[e] : __builtin_fmaf(s[e], c, -lse[e]));
                        ds[e] = s[e] * (INIT ? dp[e] : dp[e] - delta[e]);
                        if (CAREFUL && ds[e] == -INFINITY) ds[e] = NAN;
                    }
                    auto hide = [&](int e) { s[e] = ds[e] = CAREFUL ? -INFINITY : 0.f; };
                    if (edge) {  // rows of the block that see the key
                        const int r0 = a.causal ? key - p0 : 0, r1 = live ? len.q - t * QT - qb * 32 : 0;
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (acc_row(e, lane) < r0 || acc_row(e, lane) >= r1) hide(e);
                    }
                    if (BIAS && masks) n.mask<-1>(hide);
                    // here: behind the products it took more registers, and the second wave
                    if (BIAS && a.dist) dist.template add<CAREFUL>(ds, k0 - p0 - 31);
                    Tl::template add<CAREFUL>(gs, qb * 32, s, lane, dv);
                    Tl::template add<CAREFUL>(qs, qb * 32, ds, lane, dk);
                }
            }
            if (BIAS && a.dist) {
                dist.finish();
                __syncthreads();
                const float* sums = table + table_size(a) + W * SKEW;
                for (int x = threadIdx.x; x < distances; x += 64 * W) {
                    float y = sums[x];
                    for (int w = 1; w < W; ++w) y += sums[w * distances + x];
                    dist_out[x] = y;
                }
            }
        }
    };
    pass(std::false_type{});
    if (a.causal || masks) {
        if (__syncthreads_or(!all_finite(dk) || !all_finite(dv))) pass(std::true_type{});
    }
    if (!in) return;
    if (a.splits > 1) {
        const long n = (long)a.B * a.HK * a.Sk, row = ((long)wk.b * a.HK + wk.h) * a.Sk + key;
        store_row<float, ND>(reinterpret_cast<char*>(a.part + (wk.split * n + row) * DH), dk, live ? 1.f : 0.f, DH, lane);
        store_row<float, ND>(reinterpret_cast<char*>(a.part + ((a.splits + wk.split) * n + row) * DH), dv, live ? 1.f : 0.f, DH, lane);
        return;
    }
    store_row<T, ND>(a.dk.at(wk.b, key, wk.h), dk, live ? a.scale : 0.f, a.dh, lane);
    store_row<T, ND>(a.dv.at(wk.b, key, wk.h), dv, live ? 1.f : 0.f, a.dh, lane);
}

// The gradients' rows from the splits' sums [splits][B][heads][len][DH]: added up in order, times f.  Four features a thread,
// a gradient per blockIdx.y.
struct SumOf {
    const float* part;
    HeadRows out;
    int heads, len, splits;
    float f;
};
struct Sums {
    SumOf of[3];
};
template <typename T, int DH> __global__ void __launch_bounds__(256) attend_sum(Sums sums, int B, int dh) {
    const SumOf& o = sums.of[blockIdx.y];
    const long n = (long)B * o.heads * o.len, x = (long)blockIdx.x * 256 + threadIdx.x, row = x / (DH / 4);
    const int d = (int)(x % (DH / 4)) * 4;
    if (row >= n || d >= dh) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = 0; i < o.splits; ++i) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(o.part + (i * n + row) * DH + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += v[e];
    }
    typedef T vec __attribute__((ext_vector_type(4)));
    vec t;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = to_elt<T>(s[e] * o.f);
    const long group = row / o.len;
    *reinterpret_cast<vec*>(o.out.at((int)(group / o.heads), (int)(row - group * o.len), (int)(group % o.heads)) + d * (int)sizeof(T)) = t;
}

// ---------------------------------------------------------------- launches
// A kernel's dynamic LDS beyond 64 KB is allowed once per device.
template <auto K> gp_status allow_lds(size_t bytes) {
    static std::atomic<uint64_t> allowed{0};
    if (bytes <= 65536) return GP_OK;
    int dev = 0;
    GP_HIP(hipGetDevice(&dev));
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (allowed.load(std::memory_order_relaxed) & bit) return GP_OK;
    GP_HIP(hipFuncSetAttribute((const void*)K, hipFuncAttributeMaxDynamicSharedMemorySize, 159 * 1024));
    allowed.fetch_or(bit, std::memory_order_relaxed);
    return GP_OK;
}
size_t table_bytes(const AttendArgs& a) { return (2 * ((size_t)a.max_distance + PAD) + 1) * 4; }

template <typename T, int DH, int KT, int W, bool BIAS, bool KEYS>
gp_status launch_fwd(const AttendArgs& a, hipStream_t st) {
    const size_t bytes = (KEYS ? 4 * W : 2 * stages(DH)) * Tile<T, DH, KT>::BYTES + (BIAS ? table_bytes(a) + 4 : 0) + (KEYS ? W * 32 * 8 : 0);
    constexpr auto k = attend_fwd<T, DH, KT, W, BIAS, KEYS>;
    GP_TRY(allow_lds<k>(bytes));
    klaunch(k, dim3((unsigned)((long)a.B * (a.H / a.pack) * a.blocks * a.splits)), dim3(64 * W), (uint32_t)bytes, st, a);
    if (a.splits > 1)
        klaunch(attend_join<T, DH>, dim3((unsigned)(((long)a.B * a.H * a.Sq + 3) / 4)), dim3(256), 0, st, a);
    GP_LAUNCH_CHECK();
    return GP_OK;
}
template <typename T, int DH> gp_status forward(const AttendArgs& a, hipStream_t st) {
    constexpr int KT = tile_rows(sizeof(T)), W = key_waves(DH * sizeof(T));
    if (a.keys) return a.bias ? launch_fwd<T, DH, 32, W, true, true>(a, st) : launch_fwd<T, DH, 32, W, false, true>(a, st);
    return a.bias ? launch_fwd<T, DH, KT, 4, true, false>(a, st) : launch_fwd<T, DH, KT, 4, false, false>(a, st);
}

template <typename T, int DH, int W, bool BIAS, int DELTA>
gp_status launch_dq(const AttendArgs& a, hipStream_t st) {
    constexpr int KT = tile_rows(sizeof(T));
    const size_t bytes = 2 * stages(DH) * Tile<T, DH, KT>::BYTES + (BIAS ? table_bytes(a) : 0);
    constexpr auto k = attend_dq<T, DH, KT, W, BIAS, DELTA>;
    GP_TRY(allow_lds<k>(bytes));
    klaunch(k, dim3((unsigned)((long)a.B * a.H * a.blocks * a.splits)), dim3(64 * W), (uint32_t)bytes, st, a);
    GP_LAUNCH_CHECK();
    return GP_OK;
}
template <typename T, int DH, int W, bool BIAS>
gp_status launch_dkv(const AttendArgs& a, hipStream_t st) {
    constexpr int QT = tile_rows(sizeof(T));
    constexpr int ST = BIAS ? 2 : stages(DH);
    const size_t bytes = ST * (2 * Tile<T, DH, QT>::BYTES + 512) + (BIAS ? table_bytes(a) + W * (SKEW + 2 * a.max_distance + 1) * 4 : 0);
    constexpr auto k = attend_dkv<T, DH, QT, W, BIAS>;
    GP_TRY(allow_lds<k>(bytes));
    klaunch(k, dim3((unsigned)((long)a.B * a.HK * a.blocks * a.splits)), dim3(64 * W), (uint32_t)bytes, st, a);
    GP_LAUNCH_CHECK();
    return GP_OK;
}
template <typename T, int DH> gp_status backward(const AttendArgs& a, bool exact, const Shape& dq, const Shape& dkv, hipStream_t st) {
    AttendArgs q = a;
    q.blocks = dq.blocks;
    q.splits = dq.splits;
    constexpr int BY_OUT = refines<T>() ? REFINED : FROM_OUT;
    const bool refined = refines<T>() && !exact;
    if (q.blocks) {
        if (a.bias)
            GP_TRY(exact ? (launch_dq<T, DH, BW, true, FROM_WEIGHTS>(q, st)) : (launch_dq<T, DH, BW, true, BY_OUT>(q, st)));
        else
            GP_TRY(exact ? (launch_dq<T, DH, BW, false, FROM_WEIGHTS>(q, st)) : (launch_dq<T, DH, BW, false, BY_OUT>(q, st)));
        if constexpr (refines<T>())
            if (refined && q.splits > 1) {
                klaunch(attend_refine<T, DH>, dim3((unsigned)(((long)a.B * a.H * a.Sq * (DH / 4) + 255) / 256)), dim3(256), 0, st, q);
                GP_LAUNCH_CHECK();
            }
    }
    AttendArgs k = a;
    k.blocks = dkv.blocks;
    k.splits = dkv.splits;
    const size_t nq = (size_t)a.B * a.H * a.Sq * DH, nk = (size_t)a.B * a.HK * a.Sk * DH;
    if (q.splits > 1) k.part += refined ? refined_floats(nq / DH * q.splits, DH) : q.splits * nq;
    if (k.blocks) GP_TRY(a.bias ? (launch_dkv<T, DH, BW, true>(k, st)) : (launch_dkv<T, DH, BW, false>(k, st)));
    Sums sums;
    int n = 0;
    if (q.blocks && q.splits > 1 && !refined) sums.of[n++] = {q.part, a.dq, a.H, a.Sq, q.splits, a.scale};
    if (k.blocks && k.splits > 1) {
        sums.of[n++] = {k.part, a.dk, a.HK, a.Sk, k.splits, a.scale};
        sums.of[n++] = {k.part + k.splits * nk, a.dv, a.HK, a.Sk, k.splits, 1.f};
    }
    if (n) {
        const size_t most = std::max(q.splits > 1 && !refined ? nq : 0, k.splits > 1 ? nk : 0) / 4;
        klaunch(attend_sum<T, DH>, dim3((unsigned)((most + 255) / 256), n), dim3(256), 0, st, sums, a.B, a.dh);
        GP_LAUNCH_CHECK();
    }
    return GP_OK;
}

} // namespace

// The widths that a head is padded to.
template <typename T> gp_status attend_forward_as(const AttendArgs& a, hipStream_t st) {
    switch (head_bucket(a.dh)) {
    case 32: return forward<T, 32>(a, st);
    case 64: return forward<T, 64>(a, st);
    case 96: return forward<T, 96>(a, st);
    default: return forward<T, 128>(a, st);
    }
}
template <typename T> gp_status attend_backward_as(const AttendArgs& a, bool exact, const Shape& dq, const Shape& dkv, hipStream_t st) {
    switch (head_bucket(a.dh)) {
    case 32: return backward<T, 32>(a, exact, dq, dkv, st);
    case 64: return backward<T, 64>(a, exact, dq, dkv, st);
    case 96: return backward<T, 96>(a, exact, dq, dkv, st);
    default: return backward<T, 128>(a, exact, dq, dkv, st);
    }
}

} // namespace gp
