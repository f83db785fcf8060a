// attention_rows.hip -- attention on the caller's tensors: queries against keys
// of another length, ragged batches, heads that share keys, a learned relative
// position bias by buckets, and the gradients of all of them.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdio>
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
__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}
// Row (within a block of 32) of accumulator register r; the column is lane % 32.
__device__ __forceinline__ int acc_row(int r, int lane) { return (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3); }

// An LDS tile of R rows x DH features: DH / RC parts of R rows of 128 bytes without padding.
// The 16-byte chunk c of row r lies at chunk c ^ swizzle(r) of its row: 16 lanes that read the
// same chunk of 16 consecutive rows, and a half-wave that reads four chunks of four
// consecutive rows (the transposing reads), then fall into distinct banks.
__device__ __forceinline__ int swizzle(int r) { return (((r >> 1) & 1) << 2) | ((r >> 2) & 3); }

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16* LdsV4;

template <typename T, int DH, int R> struct Tile {
    typedef Elt<T> X;
    typedef typename X::frag frag;
    static constexpr int PARTS = DH / X::RC, BYTES = R * PARTS * 128, LOADS = R * PARTS / 8;

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
    // Operand of 32 rows over the chunks 2 ks, 2 ks + 1 of features.
    static __device__ __forceinline__ frag rows(const char* s, int row0, int ks, int lane) {
        const int r = row0 + (lane & 31);
        return *reinterpret_cast<const frag*>(s + (ks >> 2) * (R * 128) + r * 128 + (((((ks & 3) << 1) | (lane >> 5)) ^ swizzle(r)) << 4));
    }
    // acc (32 features from d0 on x lane's column) += the tile's rows row0 + 16 cc .. + 15, transposed, times the
    // accumulator registers 8 cc .. 8 cc + 7 of `w`, whose rows those are.  In bf16 one transposing read gives a lane
    // four rows of its feature, and w is rounded to bf16, the matrix unit's type: by up to 2^-8 of each weight,
    // while their sums stay in fp32.
    static __device__ __forceinline__ bf16x8 column(const char* s, int row0, int cc, int d0, int lane) {
        const int g = lane >> 4, q = lane & 15;
        const int row = row0 + 16 * cc + 4 * (g >> 1) + (q >> 2), col = (d0 & 63) + 16 * (g & 1) + 4 * (q & 3);
        const char* p = s + (d0 >> 6) * (R * 128) + (col & 7) * 2;
        auto at = [&](int r) { return (LdsV4)(p + r * 128 + (((col >> 3) ^ swizzle(r)) << 4)); };
        const bf16x4 x = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(row)));
        const bf16x4 y = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(row + 8)));
        return bf16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    }
    static __device__ __forceinline__ float element(const char* s, int r, int d0, int lane) {
        return *reinterpret_cast<const float*>(s + (d0 >> 5) * (R * 128) + (lane & 3) * 4 + r * 128 +
                                               ((((lane & 31) >> 2) ^ swizzle(r)) << 4));
    }
    static __device__ __forceinline__ f32x16 transposed(const char* s, int row0, int cc, int d0, const f32x16& w, int lane,
                                                        f32x16 acc) {
        if constexpr (sizeof(T) == 2) {
            bf16x8 b;
#pragma unroll
            for (int e = 0; e < 8; ++e) b[e] = (bf16)w[8 * cc + e];
            return mma(column(s, row0, cc, d0, lane), b, acc);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(element(s, row0 + acc_row(8 * cc + e, lane), d0, lane), w[8 * cc + e], acc, 0, 0, 0);
            return acc;
        }
    }
    // The same without the pairs marked by a weight of -INFINITY: what a masked row holds, infinities and NaN included,
    // does not reach the sum.  The finite values are multiplied as above; two more products with weights of 1 find
    // where an unmasked pair holds +inf or -inf (a NaN counts as both), which is then added.
    static __device__ __forceinline__ f32x16 unmasked(const char* s, int row0, int cc, int d0, const f32x16& w, int lane,
                                                      f32x16 acc) {
        const auto infinite = [](float x, float which) { return x == which || x != x; };
        const auto finite = [](float x) { return x - x == 0.f ? x : 0.f; };
        f32x16 found;
        if constexpr (sizeof(T) == 2) {
            const bf16x8 x = column(s, row0, cc, d0, lane);
            bf16x8 f, b, seen;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool m = w[8 * cc + e] == -INFINITY;
                f[e] = (bf16)finite((float)x[e]);
                b[e] = (bf16)(m ? 0.f : w[8 * cc + e]);
                seen[e] = (bf16)(m ? 0.f : 1.f);
            }
            acc = mma(f, b, acc);
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                const float inf = which ? -INFINITY : INFINITY;
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = (bf16)(infinite((float)x[e], inf) ? 1.f : 0.f);
                found = mma(f, seen, zero16());
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[e] = found[e] > 0.f ? acc[e] + inf : acc[e];
            }
        } else {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = element(s, row0 + acc_row(8 * cc + e, lane), d0, lane);
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(finite(x[e]), w[8 * cc + e] == -INFINITY ? 0.f : w[8 * cc + e], acc, 0, 0, 0);
            }
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                const float inf = which ? -INFINITY : INFINITY;
                found = zero16();
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    found = __builtin_amdgcn_mfma_f32_32x32x2f32(infinite(x[e], inf) ? 1.f : 0.f, w[8 * cc + e] == -INFINITY ? 0.f : 1.f, found, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[e] = found[e] > 0.f ? acc[e] + inf : acc[e];
            }
        }
        return acc;
    }
    // acc += the tile's 32 rows from row0 on, transposed, times w.
    template <bool CAREFUL, int ND>
    static __device__ __forceinline__ void add(const char* s, int row0, const f32x16& w, int lane, f32x16 (&acc)[ND]) {
#pragma unroll
        for (int cc = 0; cc < 2; ++cc)
#pragma unroll
            for (int d = 0; d < ND; ++d)
                acc[d] = CAREFUL ? unmasked(s, row0, cc, d * 32, w, lane, acc[d]) : transposed(s, row0, cc, d * 32, w, lane, acc[d]);
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
// beyond the table on one side, one value.
struct Near {
    bool far;
    float value;       // far: of every pair
    const float* at;   // near: of this lane's register 0; register r lies step * (row r - row 0) further
    __device__ __forceinline__ Near(const float* t, const AttendArgs& a, int lo, int mine) {
        far = lo >= a.max_distance || lo + 62 <= -a.max_distance;
        value = t[lo >= a.max_distance ? 2 * (a.max_distance + PAD) : 0];
        at = t + (far ? 0 : mine + a.max_distance + PAD);
    }
};

// Workgroup -> (sequence, head, block of rows, split); the blocks of a head are neighbours on one XCD, whose L2 then
// serves its keys and values to all of them.
struct Work {
    int b, h, blk, split;
    __device__ __forceinline__ Work(int blocks, int heads, int splits, bool reverse) {
        int id = xcd_order(blockIdx.x, gridDim.x);
        split = id % splits;
        id /= splits;
        blk = id % blocks;
        if (reverse) blk = blocks - 1 - blk;  // the longest first
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
// tiles rescale nothing.
template <typename T, int DH, int KT, int W, bool BIAS>
__global__ void __launch_bounds__(64 * W) attend_fwd(AttendArgs a) {
    typedef Tile<T, DH, KT> Tl;
    constexpr int NK = DH / Elt<T>::E / 2, ND = DH / 32, NB = KT / 32;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    float* const table = reinterpret_cast<float*>(lds + 4 * Tl::BYTES);
    const int lane = threadIdx.x & 63, wave = uniform_wave_id(threadIdx.x);
    const Work wk(a.blocks, a.H / a.pack, a.splits, a.causal != 0);
    const Lens len(a, wk.b);
    const int rows = a.Sq * a.pack, row0 = (wk.blk * W + wave) * 32, r = row0 + (lane & 31);
    const int i = a.pack == 1 ? r : r / a.pack, h = a.pack == 1 ? wk.h : wk.h * a.pack + (r - i * a.pack);
    const int hk = a.pack == 1 ? wk.h / (a.H / a.HK) : wk.h;
    const bool in = r < rows, live = in && i < len.q;
    const int pos = i + len.start, pos0 = row0 / a.pack + len.start;

    bool masks = false;
    if (BIAS) masks = __syncthreads_or(load_table(table, a, wk.h, threadIdx.x, 64 * W));
    typename Elt<T>::frag qf[NK];
    load_row<T>(a.q.at(wk.b, min(i, a.Sq - 1), min(h, a.H - 1)), live, a.dh, lane, qf);

    // keys that any row of the workgroup, and of this wave, may see
    auto reach = [&](int first, int end) {
        return first >= rows || first / a.pack >= len.q ? 0 : len.keys(a.causal, (min(end, rows) - 1) / a.pack);
    };
    const int kw = reach(row0, row0 + 32);
    const int tiles = (reach(wk.blk * W * 32, (wk.blk + 1) * W * 32) + KT - 1) / KT;
    const int t0 = (int)((long)tiles * wk.split / a.splits), t1 = (int)((long)tiles * (wk.split + 1) / a.splits);
    const char *kp = a.k.at(wk.b, 0, hk), *vp = a.v.at(wk.b, 0, hk);
    const typename Tl::template Loader<W> kl(a.k.row, a.dh, wave, lane), vl(a.v.row, a.dh, wave, lane);
    auto stage = [&](int t) {
        char* s = lds + (t & 1) * 2 * Tl::BYTES;
        kl(s, kp + (long)t * KT * a.k.row, len.k - t * KT, a.k.row, a.dh, wave);
        vl(s + Tl::BYTES, vp + (long)t * KT * a.v.row, len.k - t * KT, a.v.row, a.dh, wave);
    };

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
        if (t0 < t1) stage(t0);
        for (int t = t0; t < t1; ++t) {
            wait_vmcnt<0>();
            lds_barrier();
            if (t + 1 < t1) stage(t + 1);
            if (t * KT >= kw) continue;
            const char *ks = lds + (t & 1) * 2 * Tl::BYTES, *vs = ks + Tl::BYTES;
            f32x16 s[NB];
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                s[kb] = zero16();
#pragma unroll
                for (int x = 0; x < NK; ++x) s[kb] = mma(Tl::rows(ks, kb * 32, x, lane), qf[x], s[kb]);
            }
            const bool edge = t * KT + KT > len.k || (a.causal && t * KT + KT - 1 > pos0);
            float tm = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                const int k0 = t * KT + kb * 32;
                if (BIAS) {
                    const Near n(table, a, k0 - pos0 - 31, k0 + 4 * (lane >> 5) - pos);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float bias = n.far ? n.value : n.at[(e >> 2) * 8 + (e & 3)];
                        const float x = __builtin_fmaf(s[kb][e], c, bias);
                        s[kb][e] = masks && bias == -INFINITY ? bias : x;
                    }
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
        if (__syncthreads_or(!all_finite(o))) pass(std::true_type{});
    }
    l = both_sum(l);
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
    float m = NO_REF;
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, st[s * n + row][0]);
    float l = 0.f, o[DH / 64] = {};
    for (int s = 0; s < a.splits; ++s) {
        const f32x2 x = st[s * n + row];
        const float f = exp2_hw(x[0] - m);
        l = __builtin_fmaf(x[1], f, l);
#pragma unroll
        for (int d = 0; d < DH / 64; ++d) o[d] = __builtin_fmaf(a.part[(s * n + row) * DH + d * 64 + lane], f, o[d]);
    }
    const Lens len(a, b);
    const bool none = l == 0.f || i >= len.q;
    T* out = reinterpret_cast<T*>(a.o.at(b, i, h));
#pragma unroll
    for (int d = 0; d < DH / 64; ++d)
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
    // lo: distance of the block's first key from its last query
    __device__ __forceinline__ void add(const f32x16& ds, int lo) {
        if (lo >= D || lo + 62 <= -D) {
            float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e & 3] += ds[e];
            const float x = (s[0] + s[1]) + (s[2] + s[3]);
            if (lo >= D) high += x; else low += x;
            return;
        }
        float* p = skew + (lane & 31) * 63 + 31 + 4 * (lane >> 5);
#pragma unroll
        for (int e = 0; e < 16; ++e) p[(e >> 2) * 8 + (e & 3)] = ds[e];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i & 3] += skew[i * 64 + lane];
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
// delta_i = sum_j P_ij dP_ij = dO_i . O_i.  EXACT takes the first form, in a pass of its own over the keys: O in bf16
// is off by up to 2^-8 of itself, and so would each row's sum of dS be, which all the row's pairs share and the bias's
// gradient adds up.  Writes (lse, delta) of each row for dK and dV.
template <typename T, int DH, int KT, int W, bool BIAS, bool EXACT>
__global__ void __launch_bounds__(64 * W) attend_dq(AttendArgs a) {
    typedef Tile<T, DH, KT> Tl;
    constexpr int NK = DH / Elt<T>::E / 2, ND = DH / 32, NB = KT / 32;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    float* const table = reinterpret_cast<float*>(lds + 4 * Tl::BYTES);
    const int lane = threadIdx.x & 63, wave = uniform_wave_id(threadIdx.x);
    const Work wk(a.blocks, a.H, 1, a.causal != 0);
    const Lens len(a, wk.b);
    const int row0 = (wk.blk * W + wave) * 32, i = row0 + (lane & 31), hk = wk.h / (a.H / a.HK);
    const bool in = i < a.Sq, live = i < len.q;
    const int pos = i + len.start, pos0 = row0 + len.start;
    const long stat = ((long)wk.b * a.H + wk.h) * a.stat_rows;

    bool masks = false;
    if (BIAS) masks = __syncthreads_or(load_table(table, a, wk.h, threadIdx.x, 64 * W));
    Distances dist(table + (BIAS ? table_size(a) : 0), a.max_distance, wave, W, lane);

    typename Elt<T>::frag qf[NK], gf[NK];
    const int ic = min(i, a.Sq - 1);
    load_row<T>(a.q.at(wk.b, ic, wk.h), live, a.dh, lane, qf);
    load_row<T>(a.dout.at(wk.b, ic, wk.h), live, a.dh, lane, gf);
    float delta = 0.f;
    if (!EXACT) {
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
    const int t1 = (reach(wk.blk * W * 32, (wk.blk + 1) * W * 32) + KT - 1) / KT;
    const char *kp = a.k.at(wk.b, 0, hk), *vp = a.v.at(wk.b, 0, hk);
    const typename Tl::template Loader<W> kl(a.k.row, a.dh, wave, lane), vl(a.v.row, a.dh, wave, lane);
    auto stage = [&](int t) {
        char* s = lds + (t & 1) * 2 * Tl::BYTES;
        kl(s, kp + (long)t * KT * a.k.row, len.k - t * KT, a.k.row, a.dh, wave);
        vl(s + Tl::BYTES, vp + (long)t * KT * a.v.row, len.k - t * KT, a.v.row, a.dh, wave);
    };
    const float c = a.scale * LOG2E;
    // the weights of one block (s) and dP (dp); -INFINITY marks a masked pair's weight where `mark` asks for it
    auto block = [&](const char* ks, const char* vs, int k0, int kb, bool edge, bool mark, f32x16& s, f32x16& dp) {
        s = zero16();
        dp = zero16();
#pragma unroll
        for (int x = 0; x < NK; ++x) {
            s = mma(Tl::rows(ks, kb * 32, x, lane), qf[x], s);
            dp = mma(Tl::rows(vs, kb * 32, x, lane), gf[x], dp);
        }
        const int last = !live ? -1 : a.causal ? min(len.k - 1, pos) : len.k - 1;
        const Near n(table, a, BIAS ? k0 - pos0 - 31 : 0, BIAS ? k0 + 4 * (lane >> 5) - pos : 0);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float bias = !BIAS ? 0.f : n.far ? n.value : n.at[(e >> 2) * 8 + (e & 3)];
            float p = exp2_hw(BIAS ? __builtin_fmaf(s[e], c, bias) - lse2 : __builtin_fmaf(s[e], c, -lse2));
            if ((edge && k0 + acc_row(e, lane) > last) || (BIAS && masks && bias == -INFINITY)) {
                p = mark ? -INFINITY : 0.f;
                dp[e] = 0.f;
            }
            s[e] = p;
        }
    };
    const bool short_rows = row0 + 32 > len.q;  // a row that is not in use has no weights, whatever the keys hold
    auto tile_edge = [&](int t) { return short_rows || t * KT + KT > len.k || (a.causal && t * KT + KT - 1 > pos0); };
    if (EXACT) {
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        if (t1 > 0) stage(0);
        for (int t = 0; t < t1; ++t) {
            wait_vmcnt<0>();
            lds_barrier();
            if (t + 1 < t1) stage(t + 1);
            if (t * KT >= kw) continue;
            const char *ks = lds + (t & 1) * 2 * Tl::BYTES, *vs = ks + Tl::BYTES;
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                f32x16 s, dp;
                block(ks, vs, t * KT + kb * 32, kb, tile_edge(t), false, s, dp);
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[e & 3] = __builtin_fmaf(s[e], dp[e], sum[e & 3]);
            }
        }
        delta = both_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
        lds_barrier();
    }
    f32x16 dq[ND];
    auto pass = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        if (BIAS && a.dist) dist.clear();
#pragma unroll
        for (int d = 0; d < ND; ++d) dq[d] = zero16();
        if (t1 > 0) stage(0);
        for (int t = 0; t < t1; ++t) {
            wait_vmcnt<0>();
            lds_barrier();
            if (t + 1 < t1) stage(t + 1);
            if (t * KT >= kw) continue;
            const char *ks = lds + (t & 1) * 2 * Tl::BYTES, *vs = ks + Tl::BYTES;
            const bool edge = tile_edge(t);
#pragma unroll 1
            for (int kb = 0; kb < NB; ++kb) {
                f32x16 s, dp;
                block(ks, vs, t * KT + kb * 32, kb, edge, CAREFUL, s, dp);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float d = s[e] * (dp[e] - delta);
                    s[e] = !CAREFUL ? d : s[e] == -INFINITY ? s[e] : d == -INFINITY ? NAN : d;
                }
                Tl::template add<CAREFUL>(ks, kb * 32, s, lane, dq);
                if (CAREFUL) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = s[e] == -INFINITY ? 0.f : s[e];
                }
                if (BIAS && a.dist) dist.add(s, t * KT + kb * 32 - pos0 - 31);
            }
        }
    };
    pass(std::false_type{});
    if (a.causal || masks) {
        if (__syncthreads_or(!all_finite(dq))) pass(std::true_type{});
    }
    if (in) store_row<T, ND>(a.dq.at(wk.b, i, wk.h), dq, live ? a.scale : 0.f, a.dh, lane);
    if (lane < 32 && i < a.stat_rows) a.stats[stat + i] = f32x2{lse2, delta};
    if (wk.blk == a.blocks - 1)  // the rows that a tile of queries may read behind the last one
        for (int x = a.blocks * W * 32 + (int)threadIdx.x; x < a.stat_rows; x += 64 * W) a.stats[stat + x] = f32x2{INFINITY, 0.f};
    if (BIAS && a.dist) {
        dist.finish();
        __syncthreads();
        const int n = 2 * a.max_distance + 1;
        float* out = a.dist + (((long)wk.h * a.B + wk.b) * a.blocks + wk.blk) * n;
        const float* sums = table + table_size(a) + W * SKEW;
        for (int d = threadIdx.x; d < n; d += 64 * W) {
            float x = sums[d];
            for (int w = 1; w < W; ++w) x += sums[w * n + d];
            out[d] = x;
        }
    }
}

// dK and dV: a wave owns 32 keys and goes through the queries of all the heads that share them, in tiles of QT:
//   S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS.
template <typename T, int DH, int QT, int W, bool BIAS>
__global__ void __launch_bounds__(64 * W) attend_dkv(AttendArgs a) {
    typedef Tile<T, DH, QT> Tl;
    constexpr int NK = DH / Elt<T>::E / 2, ND = DH / 32, NB = QT / 32;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    f32x2* const stats = reinterpret_cast<f32x2*>(lds + 4 * Tl::BYTES);  // two tiles' rows
    float* const table = reinterpret_cast<float*>(stats + 2 * QT);
    const int lane = threadIdx.x & 63, wave = uniform_wave_id(threadIdx.x);
    const Work wk(a.blocks, a.HK, 1, false);
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
    const typename Tl::template Loader<W> ql(a.q.row, a.dh, wave, lane), gl(a.dout.row, a.dh, wave, lane);
    const float c = a.scale * LOG2E;
    bool masks = false;
    f32x16 dk[ND], dv[ND];
    auto pass = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
#pragma unroll
        for (int d = 0; d < ND; ++d) dk[d] = dv[d] = zero16();
        for (int g = 0; g < group; ++g) {
            const int h = wk.h * group + g;
            const char *qp = a.q.at(wk.b, 0, h), *gp = a.dout.at(wk.b, 0, h);
            const f32x2* sp = a.stats + ((long)wk.b * a.H + h) * a.stat_rows;
            auto stage = [&](int t) {
                char* s = lds + (t & 1) * 2 * Tl::BYTES;
                ql(s, qp + (long)t * QT * a.q.row, len.q - t * QT, a.q.row, a.dh, wave);
                gl(s + Tl::BYTES, gp + (long)t * QT * a.dout.row, len.q - t * QT, a.dout.row, a.dh, wave);
                if (wave < QT / 32)  // 32 rows' pairs a load
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(sp + t * QT, QT * 8), (LdsPtr)(stats + (t & 1) * QT + wave * 32), 4,
                                                             wave * 256 + lane * 4, 0, 0, 0);
            };
            __syncthreads();  // the last head's tiles are done with
            if (BIAS) masks = masks | (__syncthreads_or(load_table(table, a, h, threadIdx.x, 64 * W)) != 0);
            if (t0 < t1) stage(t0);
            for (int t = t0; t < t1; ++t) {
                wait_vmcnt<0>();
                lds_barrier();
                if (t + 1 < t1) stage(t + 1);
                const int pos0 = t * QT + len.start;
                if (k0 >= len.k || (a.causal && pos0 + QT - 1 < k0)) continue;
                const char *qs = lds + (t & 1) * 2 * Tl::BYTES, *gs = qs + Tl::BYTES;
                const bool edge = t * QT + QT > len.q || (a.causal && pos0 < k0 + 31);
#pragma unroll 1
                for (int qb = 0; qb < NB; ++qb) {
                    f32x16 s = zero16(), dp = zero16();
#pragma unroll
                    for (int x = 0; x < NK; ++x) {
                        s = mma(Tl::rows(qs, qb * 32, x, lane), kf[x], s);
                        dp = mma(Tl::rows(gs, qb * 32, x, lane), vf[x], dp);
                    }
                    const int p0 = pos0 + qb * 32;
                    const int r0 = a.causal ? key - p0 : 0, r1 = len.q - t * QT - qb * 32;  // rows of the block that see the key
                    // distances fall with the register here
                    const Near n(table, a, BIAS ? k0 - p0 - 31 : 0, BIAS ? key - p0 - 4 * (lane >> 5) : 0);
                    const f32x2* st = stats + (t & 1) * QT + qb * 32 + 4 * (lane >> 5);
                    f32x16 ds;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const f32x2 row = st[(e >> 2) * 8 + (e & 3)];
                        const float bias = !BIAS ? 0.f : n.far ? n.value : n.at[-((e >> 2) * 8 + (e & 3))];
                        float p = exp2_hw(BIAS ? __builtin_fmaf(s[e], c, bias) - row[0] : __builtin_fmaf(s[e], c, -row[0]));
                        float d = p * (dp[e] - row[1]);
                        if (CAREFUL && d == -INFINITY) d = NAN;
                        if ((edge && (acc_row(e, lane) < r0 || acc_row(e, lane) >= r1)) || (BIAS && masks && bias == -INFINITY)) {
                            p = CAREFUL ? -INFINITY : 0.f;
                            d = p;
                        }
                        s[e] = p;
                        ds[e] = d;
                    }
                    Tl::template add<CAREFUL>(gs, qb * 32, s, lane, dv);
                    Tl::template add<CAREFUL>(qs, qb * 32, ds, lane, dk);
                }
            }
        }
    };
    pass(std::false_type{});
    if (a.causal || masks) {
        if (__syncthreads_or(!all_finite(dk) || !all_finite(dv))) pass(std::true_type{});
    }
    if (!in) return;
    store_row<T, ND>(a.dk.at(wk.b, key, wk.h), dk, live ? a.scale : 0.f, a.dh, lane);
    store_row<T, ND>(a.dv.at(wk.b, key, wk.h), dv, live ? 1.f : 0.f, a.dh, lane);
}

// Sums of n rows of `width` floats, STEP rows at a time: out row x = rows x STEP .. of head blockIdx.y.
constexpr int STEP = 32;
__global__ void __launch_bounds__(256) distance_rows(const float* __restrict__ in, long n, int width, float* __restrict__ out) {
    const long x = blockIdx.x, y = blockIdx.y, steps = gridDim.x;
    const long r0 = x * STEP, r1 = min(n, r0 + STEP);
    for (int d = threadIdx.x; d < width; d += 256) {
        float s = 0.f;
#pragma unroll 8
        for (long r = r0; r < r1; ++r) s += in[(y * n + r) * width + d];
        out[(y * steps + x) * width + d] = s;
    }
}
// dbias of head blockIdx.x: its n rows of distances added up, then the distances of each bucket, in their order.
__global__ void __launch_bounds__(256) distance_buckets(const float* __restrict__ in, long n, AttendArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int width = 2 * a.max_distance + 1;
    float* sums = reinterpret_cast<float*>(lds);
    int* of = reinterpret_cast<int*>(sums + width);
    for (int d = threadIdx.x; d < width; d += 256) {
        float s = 0.f;
#pragma unroll 8
        for (long r = 0; r < n; ++r) s += in[(blockIdx.x * n + r) * width + d];
        sums[d] = s;
        of[d] = min(max(a.bucket_of[d], 0), a.buckets - 1);
    }
    __syncthreads();
    const int lane = threadIdx.x & 63;
    for (int b = threadIdx.x >> 6; b < a.buckets; b += 4) {  // a wave per bucket
        float s = 0.f;
        for (int d = lane; d < width; d += WAVE) s += of[d] == b ? sums[d] : 0.f;
        s = wave_sum(s);
        if (lane == 0) a.dbias[(long)blockIdx.x * a.buckets + b] = s;
    }
}

// ---------------------------------------------------------------- launches
long up(long n, long m) { return (n + m - 1) / m * m; }
template <typename T> constexpr int tile_rows() { return sizeof(T) == 2 ? 64 : 32; }

struct Shape {
    int waves;   // of a workgroup
    int pack;    // heads whose rows are packed together
    int blocks;  // of 32 waves rows
    int splits;
};
Shape forward_shape(const AttendArgs& a) {
    Shape s{4, 1, 1, 1};
    const int group = a.H / a.HK;
    if (!a.bias && group > 1 && a.Sq < 32) s.pack = group;
    const long rows = (long)a.Sq * s.pack;
    if (rows <= 32) s.waves = 1;
    s.blocks = (int)((rows + 32 * s.waves - 1) / (32 * s.waves));
    const long groups = std::max(1l, (long)a.B * (a.H / s.pack) * s.blocks);
    const int kt = 32, tiles = (a.Sk + kt - 1) / kt;
    if (groups * s.waves < 1024) s.splits = (int)std::max(1l, std::min<long>(std::min(64, tiles / 4), 2048 / (groups * s.waves)));
    return s;
}

template <typename T, int DH, int KT, int W, bool BIAS>
gp_status launch_fwd(const AttendArgs& a, hipStream_t st) {
    const size_t bytes = 4 * Tile<T, DH, KT>::BYTES + (BIAS ? (2 * (a.max_distance + PAD) + 1) * 4 : 0);
    auto* k = attend_fwd<T, DH, KT, W, BIAS>;
    if (bytes > 65536) GP_HIP(hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    klaunch(k, dim3((unsigned)((long)a.B * (a.H / a.pack) * a.blocks * a.splits)), dim3(64 * W), (uint32_t)bytes, st, a);
    if (a.splits > 1)
        klaunch(attend_join<T, DH>, dim3((unsigned)(((long)a.B * a.H * a.Sq + 3) / 4)), dim3(256), 0, st, a);
    GP_LAUNCH_CHECK();
    return GP_OK;
}
template <typename T, int DH>
gp_status forward(AttendArgs& a, hipStream_t st) {
    if (a.waves == 1) return a.bias ? launch_fwd<T, DH, 32, 1, true>(a, st) : launch_fwd<T, DH, 32, 1, false>(a, st);
    constexpr int KT = tile_rows<T>();
    return a.bias ? launch_fwd<T, DH, KT, 4, true>(a, st) : launch_fwd<T, DH, KT, 4, false>(a, st);
}

template <typename T, int DH, int W, bool BIAS, bool EXACT>
gp_status launch_dq(const AttendArgs& a, hipStream_t st) {
    constexpr int KT = tile_rows<T>();
    const size_t bytes = 4 * Tile<T, DH, KT>::BYTES +
                         (BIAS ? (2 * (a.max_distance + PAD) + 1 + W * (SKEW + 2 * a.max_distance + 1)) * 4 : 0);
    auto* k = attend_dq<T, DH, KT, W, BIAS, EXACT>;
    if (bytes > 65536) GP_HIP(hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    klaunch(k, dim3((unsigned)((long)a.B * a.H * a.blocks)), dim3(64 * W), (uint32_t)bytes, st, a);
    GP_LAUNCH_CHECK();
    return GP_OK;
}
template <typename T, int DH, int W, bool BIAS>
gp_status launch_dkv(const AttendArgs& a, hipStream_t st) {
    constexpr int QT = tile_rows<T>();
    const size_t bytes = 4 * Tile<T, DH, QT>::BYTES + 2 * QT * 8 + (BIAS ? (2 * (a.max_distance + PAD) + 1) * 4 : 0);
    auto* k = attend_dkv<T, DH, QT, W, BIAS>;
    if (bytes > 65536) GP_HIP(hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    klaunch(k, dim3((unsigned)((long)a.B * a.HK * a.blocks)), dim3(64 * W), (uint32_t)bytes, st, a);
    GP_LAUNCH_CHECK();
    return GP_OK;
}

constexpr int BW = 4;  // waves of the backward's workgroups
template <typename T, int DH>
gp_status backward(AttendArgs& a, bool exact, hipStream_t st) {
    AttendArgs q = a;
    q.blocks = (a.Sq + 32 * BW - 1) / (32 * BW);
    if (q.blocks) {
        if (a.bias)
            GP_TRY(exact ? (launch_dq<T, DH, BW, true, true>(q, st)) : (launch_dq<T, DH, BW, true, false>(q, st)));
        else
            GP_TRY(exact ? (launch_dq<T, DH, BW, false, true>(q, st)) : (launch_dq<T, DH, BW, false, false>(q, st)));
    }
    AttendArgs k = a;
    k.blocks = (a.Sk + 32 * BW - 1) / (32 * BW);
    if (k.blocks) GP_TRY(a.bias ? (launch_dkv<T, DH, BW, true>(k, st)) : (launch_dkv<T, DH, BW, false>(k, st)));
    return GP_OK;
}

int head_bucket(int dh) { return dh <= 64 ? 64 : 128; }
long stat_rows(int Sq) { return up(Sq, 64); }
// Rows of distances of one head that the dQ kernel writes, and that one addition leaves.
long distance_rows_of(const AttendArgs& a) { return (long)a.B * ((a.Sq + 32 * BW - 1) / (32 * BW)); }

} // namespace

size_t attend_workspace(const AttendArgs& a) {
    const Shape s = forward_shape(a);
    return s.splits > 1 ? (size_t)s.splits * a.B * a.H * a.Sq * (head_bucket(a.dh) + 2) * 4 : 0;
}

gp_status attend_forward(AttendArgs a, void* ws, hipStream_t st) {
    const Shape s = forward_shape(a);
    a.waves = s.waves;
    a.pack = s.pack;
    a.blocks = s.blocks;
    a.splits = s.splits;
    a.part = static_cast<float*>(ws);
    if (a.dtype == GP_BF16) return a.dh <= 64 ? forward<bf16, 64>(a, st) : forward<bf16, 128>(a, st);
    return a.dh <= 64 ? forward<float, 64>(a, st) : forward<float, 128>(a, st);
}

size_t attend_backward_workspace(const AttendArgs& a) {
    size_t n = (size_t)a.B * a.H * stat_rows(a.Sq) * 8;
    if (a.bias) {
        const size_t rows = (size_t)distance_rows_of(a);
        n += a.H * (rows + (rows + STEP - 1) / STEP) * (2 * (size_t)a.max_distance + 1) * 4;
    }
    return n;
}

gp_status attend_backward(AttendArgs a, bool exact, void* ws, hipStream_t st) {
    a.stat_rows = (int)stat_rows(a.Sq);
    a.stats = static_cast<f32x2*>(ws);
    float* dist = reinterpret_cast<float*>(a.stats + (size_t)a.B * a.H * a.stat_rows);
    a.dist = a.bias && a.dbias ? dist : nullptr;
    a.pack = a.splits = 1;
    if (a.B) {
        if (a.dtype == GP_BF16)
            GP_TRY(a.dh <= 64 ? (backward<bf16, 64>(a, exact, st)) : (backward<bf16, 128>(a, exact, st)));
        else
            GP_TRY(a.dh <= 64 ? (backward<float, 64>(a, exact, st)) : (backward<float, 128>(a, exact, st)));
    }
    if (!a.bias || !a.dbias) return GP_OK;
    const int width = 2 * a.max_distance + 1;
    long n = distance_rows_of(a);
    const float* in = dist;
    if (n > STEP) {
        float* out = dist + (size_t)a.H * n * width;
        const long steps = (n + STEP - 1) / STEP;
        klaunch(distance_rows, dim3((unsigned)steps, (unsigned)a.H), dim3(256), 0, st, in, n, width, out);
        in = out;
        n = steps;
    }
    klaunch(distance_buckets, dim3((unsigned)a.H), dim3(256), (uint32_t)(width * 8), st, in, n, a);
    GP_LAUNCH_CHECK();
    return GP_OK;
}

} // namespace gp

// ------------------------------------------------------------------- C ABI
namespace gp {
namespace {

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// A configuration's sizes as arguments of the kernels, or a refusal.
gp_status read_config(const gp_attention_config* c, AttendArgs& a, const char*& why) {
    auto bad = [&](const char* m) {
        why = m;
        return GP_ERR_INVALID_ARG;
    };
    if (!c) return bad("a NULL configuration");
    if (c->dtype != GP_F32 && c->dtype != GP_BF16) return bad("unknown dtype");
    if (c->batch < 0 || c->q_len < 0 || c->k_len < 0 || c->q_len > (1 << 28) || c->k_len > (1 << 28))
        return bad("batch must be >= 0, lengths in [0, 2^28]");
    if (c->heads < 1 || c->kv_heads < 1 || c->heads % c->kv_heads) return bad("heads must be a multiple of kv_heads");
    const int esz = c->dtype == GP_BF16 ? 2 : 4;
    if (c->head_dim < 1 || c->head_dim * esz % 16) return bad("head_dim must fill whole 16 bytes");
    if (!(c->scale > 0.f) || !(c->scale <= FLT_MAX)) return bad("scale must be finite and > 0");
    for (const int* p : {c->q_lens, c->k_lens, c->q_starts})
        if (!aligned(p, 4)) return bad("misaligned lengths or positions");
    if (c->bias) {
        if (!c->bucket_of || c->buckets < 1 || c->max_distance < 1) return bad("a bias needs bucket_of, buckets >= 1 and max_distance >= 1");
        if (!aligned(c->bias, 4) || !aligned(c->bucket_of, 4)) return bad("a misaligned bias or bucket_of");
    } else if (c->bucket_of || c->buckets || c->max_distance) {
        return bad("bucket_of, buckets and max_distance belong to a bias");
    }
    // a launch holds fewer than 2^32 threads, 256 of them take 128 rows; a head's own grid dimension 2^16
    const long groups = (long)c->batch * c->heads;
    if (c->heads > 65535 || groups >= (1l << 24) || groups * (c->q_len / 128 + 1l) >= (1l << 24) ||
        groups * (c->k_len / 128 + 1l) >= (1l << 24))
        return bad("more heads (65535) or rows than a launch holds");
    a = AttendArgs{};
    a.dtype = c->dtype;
    a.B = c->batch;
    a.H = c->heads;
    a.HK = c->kv_heads;
    a.Sq = c->q_len;
    a.Sk = c->k_len;
    a.dh = c->head_dim;
    a.causal = c->causal != 0;
    a.scale = c->scale;
    a.q_lens = c->q_lens;
    a.k_lens = c->k_lens;
    a.q_starts = c->q_starts;
    a.bias = c->bias;
    a.bucket_of = c->bucket_of;
    a.buckets = c->buckets;
    a.max_distance = c->max_distance;
    if (c->head_dim > 128) {
        why = "head_dim must be at most 128";
        return GP_ERR_UNSUPPORTED;
    }
    if (c->bias && (c->buckets > GP_BUCKETS_MAX || c->max_distance > GP_DISTANCE_MAX)) {
        why = "a bias has at most 1024 buckets and a max_distance of 1024";
        return GP_ERR_UNSUPPORTED;
    }
    return GP_OK;
}

// One tensor of rows [batch, len, heads, head_dim] as the kernels take it, and what it spans.
struct Rows {
    HeadRows t;
    struct Dim { long stride, n; } dim[3];  // of more than one step, the widest stride first
    int dims = 0;
    long inner;  // bytes of one row of a head

    // Bytes from the first element to the last one's end over the dimensions whose strides are below `pitch`.
    long span(long pitch) const {
        long n = inner;
        for (int d = 0; d < dims; ++d)
            if (dim[d].stride < pitch) n += dim[d].stride * (dim[d].n - 1);
        return n;
    }
    uintptr_t at() const { return reinterpret_cast<uintptr_t>(t.p); }
    // No two rows share memory (each step passes over all that lies within it).
    bool distinct() const {
        for (int d = 0; d < dims; ++d) {
            long n = inner;
            for (int e = d + 1; e < dims; ++e) n += dim[e].stride * (dim[e].n - 1);
            if (dim[d].stride < n) return false;
        }
        return true;
    }
    // Every row starts at a multiple of `pitch` and something within span(pitch).
    bool pitched(long pitch) const {
        for (int d = 0; d < dims; ++d)
            if (dim[d].stride >= pitch && dim[d].stride % pitch) return false;
        return true;
    }
};
// Two tensors do not touch: they lie apart, or beside each other in every period of a stride that both have
// (the halves of a packed projection).
bool apart(const Rows& x, const Rows& y) {
    if (!x.t.p || !y.t.p) return true;
    const Rows &a = x.at() <= y.at() ? x : y, &b = x.at() <= y.at() ? y : x;
    const long all = 1l << 62, off = (long)(b.at() - a.at());
    if (off >= a.span(all)) return true;
    for (int d = 0; d < a.dims; ++d)
        for (int e = 0; e < b.dims; ++e) {
            const long pitch = a.dim[d].stride;
            if (pitch != b.dim[e].stride || pitch <= 0 || !a.pitched(pitch) || !b.pitched(pitch)) continue;
            const long r = off % pitch;
            if (r >= a.span(pitch) && r + b.span(pitch) <= pitch) return true;
        }
    return false;
}

const char* read_rows(const AttendArgs& a, const gp_head_rows* t, int len, int heads, Rows& out) {
    out = Rows{};
    if (!a.B || !len) return nullptr;
    if (!t || !t->data) return "a NULL tensor";
    const long esz = a.dtype == GP_BF16 ? 2 : 4, most = 1l << 41;
    HeadRows& r = out.t;
    r.p = static_cast<char*>(t->data);
    if (a.B == 1) r.seq = 0; else r.seq = t->seq_stride;
    if (heads == 1) r.head = 0; else r.head = t->head_stride;
    if (len == 1) r.row = a.dh; else r.row = t->row_stride;
    if (r.head < 0 || r.seq < 0 || r.row < 0 || r.head > most || r.seq > most || r.row > most) return "a stride is out of range";
    r.seq *= esz;
    r.row *= esz;
    r.head *= esz;
    if (!aligned(r.p, 16) || r.seq % 16 || r.row % 16 || r.head % 16) return "addresses and strides must be multiples of 16 bytes";
    if (r.row < a.dh * esz || r.row > (1l << 24)) return "rows must not overlap, and lie at most 2^24 bytes apart";
    out.inner = a.dh * esz;
    for (const Rows::Dim& d : {Rows::Dim{r.seq, a.B}, Rows::Dim{r.row, len}, Rows::Dim{r.head, heads}})
        if (d.n > 1) out.dim[out.dims++] = d;
    std::sort(out.dim, out.dim + out.dims, [](const Rows::Dim& x, const Rows::Dim& y) { return x.stride > y.stride; });
    return nullptr;
}

gp_status refuse(gp_status s, const char* entry, const char* why) {
    char m[256];
    snprintf(m, sizeof m, "%s: %s", entry, why);
    return set_error(s, m);
}

} // namespace
} // namespace gp

extern "C" {

using namespace gp;

gp_status gp_relative_buckets(int buckets, int max_distance, int bidirectional, int* bucket_of) {
    auto bad = [](const char* m) { return set_error(GP_ERR_INVALID_ARG, m); };
    if (!bucket_of) return bad("relative_buckets: bucket_of must not be NULL");
    const int n = bidirectional ? buckets / 2 : buckets, half = n / 2;
    if (n < 2 || (bidirectional && buckets % 2)) return bad("relative_buckets: at least two buckets a side, an even number for both");
    if (buckets > GP_BUCKETS_MAX || max_distance <= half || max_distance > GP_DISTANCE_MAX)
        return bad("relative_buckets: at most 1024 buckets, max_distance in (half a side's buckets, 1024]");
    // Bucket half + t of the logarithmic part begins at the least d with
    //   log(d / half) / log(max_distance / half) >= t / (n - half),
    // that is d^(n - half) half^t >= max_distance^t half^(n - half): compared in whole numbers, so that no border is
    // rounded to the wrong side.
    auto reaches = [&](int d, int t) {
        // products of up to 2^10 factors of up to 2^10, as little-endian digits of 32 bits
        uint32_t x[2][344] = {};
        int len[2] = {1, 1};
        x[0][0] = x[1][0] = 1;
        auto times = [&](int k, uint32_t f, int count) {
            for (int c = 0; c < count; ++c) {
                uint64_t carry = 0;
                for (int i = 0; i < len[k]; ++i) {
                    carry += (uint64_t)x[k][i] * f;
                    x[k][i] = (uint32_t)carry;
                    carry >>= 32;
                }
                if (carry) x[k][len[k]++] = (uint32_t)carry;
            }
        };
        const int steps = n - half;
        times(0, (uint32_t)d, steps);  // half^t on one side leaves half^(steps - t) on the other
        times(1, (uint32_t)max_distance, t);
        times(1, (uint32_t)half, steps - t);
        if (len[0] != len[1]) return len[0] > len[1];
        for (int i = len[0] - 1; i >= 0; --i)
            if (x[0][i] != x[1][i]) return x[0][i] > x[1][i];
        return true;
    };
    int t = 0;
    for (int d = 0; d <= max_distance; ++d) {
        int side = d;
        if (d >= half) {
            while (t + 1 < n - half && reaches(d, t + 1)) ++t;
            side = half + t;
        }
        // key - query = -d, and + d
        bucket_of[max_distance - d] = side;
        if (d) bucket_of[max_distance + d] = bidirectional ? n + side : 0;
    }
    return GP_OK;
}

gp_status gp_attention_workspace(const gp_attention_config* cfg, int backward, size_t* bytes) {
    AttendArgs a;
    const char* why = "";
    if (!bytes) return set_error(GP_ERR_INVALID_ARG, "attention_workspace: bytes must not be NULL");
    const gp_status ok = read_config(cfg, a, why);
    if (ok != GP_OK) return refuse(ok, "attention_workspace", why);
    *bytes = !a.B ? 0 : backward ? attend_backward_workspace(a) : attend_workspace(a);
    return GP_OK;
}

gp_status gp_attention(const gp_attention_config* cfg, const gp_head_rows* q, const gp_head_rows* k, const gp_head_rows* v,
                       const gp_head_rows* out, float* lse, void* ws, size_t ws_bytes, gp_stream stream) {
    AttendArgs a;
    const char* why = "";
    auto bad = [](const char* m) { return refuse(GP_ERR_INVALID_ARG, "attention", m); };
    const gp_status ok = read_config(cfg, a, why);
    if (ok != GP_OK) return refuse(ok, "attention", why);
    if (!a.B || !a.Sq) return GP_OK;
    Rows rq, rk, rv, ro;
    for (const char* m : {read_rows(a, q, a.Sq, a.H, rq), read_rows(a, k, a.Sk, a.HK, rk), read_rows(a, v, a.Sk, a.HK, rv),
                          read_rows(a, out, a.Sq, a.H, ro)})
        if (m) return bad(m);
    if (!ro.distinct()) return bad("the rows of out must not overlap");
    for (const Rows* t : {&rq, &rk, &rv})
        if (!apart(*t, ro)) return bad("out must not overlap an input");
    if (!aligned(lse, 4)) return bad("a misaligned lse");
    if (!aligned(ws, 16)) return bad("the workspace must be 16-byte aligned");
    const size_t need = attend_workspace(a);
    if (need && (!ws || ws_bytes < need)) return bad("the workspace is smaller than gp_attention_workspace says");
    a.q = rq.t;
    a.k = rk.t;
    a.v = rv.t;
    a.o = ro.t;
    a.lse = lse;
    return attend_forward(a, ws, (hipStream_t)stream);
}

gp_status gp_attention_backward(const gp_attention_config* cfg, const gp_head_rows* q, const gp_head_rows* k,
                                const gp_head_rows* v, const gp_head_rows* out, const float* lse, const gp_head_rows* dout,
                                const gp_head_rows* dq, const gp_head_rows* dk, const gp_head_rows* dv, float* dbias,
                                void* ws, size_t ws_bytes, gp_stream stream) {
    AttendArgs a;
    const char* why = "";
    auto bad = [](const char* m) { return refuse(GP_ERR_INVALID_ARG, "attention_backward", m); };
    const gp_status ok = read_config(cfg, a, why);
    if (ok != GP_OK) return refuse(ok, "attention_backward", why);
    Rows in[5] = {}, grad[3] = {};  // q, k, v, dout, out; dq, dk, dv
    for (const char* m : {read_rows(a, q, a.Sq, a.H, in[0]), read_rows(a, k, a.Sk, a.HK, in[1]), read_rows(a, v, a.Sk, a.HK, in[2]),
                          read_rows(a, dout, a.Sq, a.H, in[3]), out ? read_rows(a, out, a.Sq, a.H, in[4]) : nullptr,
                          read_rows(a, dq, a.Sq, a.H, grad[0]), read_rows(a, dk, a.Sk, a.HK, grad[1]),
                          read_rows(a, dv, a.Sk, a.HK, grad[2])})
        if (m) return bad(m);
    if (dbias && !a.bias) return bad("dbias needs a bias");
    if (a.B && a.Sq && !lse) return bad("lse must not be NULL");
    if (!aligned(lse, 4) || !aligned(dbias, 4)) return bad("a misaligned address");
    for (int x = 0; x < 3; ++x) {
        if (!grad[x].distinct()) return bad("the rows of a gradient must not overlap");
        for (int y = 0; y < 5; ++y)
            if (!apart(grad[x], in[y])) return bad("a gradient must not overlap an input");
        for (int y = 0; y < x; ++y)
            if (!apart(grad[x], grad[y])) return bad("the gradients must not overlap each other");
    }
    if (!aligned(ws, 16)) return bad("the workspace must be 16-byte aligned");
    const size_t need = a.B ? attend_backward_workspace(a) : 0;
    if (need && (!ws || ws_bytes < need)) return bad("the workspace is smaller than gp_attention_workspace says");
    a.q = in[0].t;
    a.k = in[1].t;
    a.v = in[2].t;
    a.dout = in[3].t;
    a.o = in[4].t;
    a.dq = grad[0].t;
    a.dk = grad[1].t;
    a.dv = grad[2].t;
    a.lse_in = lse;
    a.dbias = dbias;
    return attend_backward(a, !out || (a.bias && a.dtype == GP_BF16), ws, (hipStream_t)stream);
}

} // extern "C"
