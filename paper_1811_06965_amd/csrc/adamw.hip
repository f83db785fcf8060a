// adamw.hip -- the AdamW update of many tensors at once, states in 32 or in 8
// bits, and the global gradient norm that clips it.
//
// The tensors of a call travel in the kernel arguments, BATCH of them per
// launch: no table in device memory, nothing to copy or to keep alive, and a
// captured launch holds its own.  A workgroup takes one chunk of one tensor: the
// lanes of a wave compare its index with the tensors' first chunks, one each, so
// that it is at its data after two reads of the arguments (a binary search, six reads
// one after the other, took 10 of the 13 us of an update of 32 small tensors).
#include <cmath>
#include <type_traits>

#include "adamw.hpp"

namespace gp {

namespace {

constexpr int BATCH = 48;    // tensors per launch: 3.8 KB of the 4 KB of kernel arguments
constexpr int CHUNK = 4096;  // elements a workgroup updates

struct AdamwTensor {
    void* p;
    const void* g;
    void* m;
    void* v;
    float* ms;
    float* vs;
    bf16* c;
    long n;
    float keep;  // 1 - lr weight_decay
};
struct AdamwBatch {
    int n;
    int chunk0[BATCH];  // chunks of the launch's tensors before each
    AdamwTensor t[BATCH];
};
static_assert(sizeof(AdamwBatch) + sizeof(AdamwScalars) <= 4096, "kernel arguments");

// The last of n tensors whose first chunk is not after id.
template <int MOST> __device__ __forceinline__ int tensor_of(const int (&chunk0)[MOST], int n, int id) {
    int l = -1;
#pragma unroll
    for (int i = 0; i < MOST; i += WAVE) {
        const int k = i + (threadIdx.x & 63);
        l += __popcll(__ballot(k < n && chunk0[k < MOST ? k : 0] <= id));
    }
    return __builtin_amdgcn_readfirstlane(l);
}

// Four elements at any element's address, whole or as many as lie before n.
template <typename T> struct Four {
    typedef T vec __attribute__((ext_vector_type(4)));
    typedef vec at_any __attribute__((aligned(sizeof(T))));
    static __device__ __forceinline__ vec load(const void* p, long i, long n, bool whole) {
        const T* t = static_cast<const T*>(p) + i;
        if (whole) return *reinterpret_cast<const at_any*>(t);
        vec r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = i + e < n ? t[e] : (T)0;
        return r;
    }
    static __device__ __forceinline__ void store(void* p, long i, long n, bool whole, vec x) {
        T* t = static_cast<T*>(p) + i;
        if (whole) {
            *reinterpret_cast<at_any*>(t) = x;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < n) t[e] = x[e];
        }
    }
    static __device__ __forceinline__ f32x4 values(vec x) { return f32x4{to_f32(x[0]), to_f32(x[1]), to_f32(x[2]), to_f32(x[3])}; }
    static __device__ __forceinline__ vec rounded(f32x4 x) {
        return vec{to_elt<T>(x[0]), to_elt<T>(x[1]), to_elt<T>(x[2]), to_elt<T>(x[3])};
    }
};
typedef Four<unsigned char> Codes;
// The values of four e4m3 codes.
__device__ __forceinline__ f32x4 e4m3_values(Codes::vec c) {
    const int q = (int)__builtin_bit_cast(unsigned, c);
    return f32x4{__builtin_amdgcn_cvt_f32_fp8(q, 0), __builtin_amdgcn_cvt_f32_fp8(q, 1),
                 __builtin_amdgcn_cvt_f32_fp8(q, 2), __builtin_amdgcn_cvt_f32_fp8(q, 3)};
}
// A block's scale and its inverse from the largest |x| (as bits, so that a NaN, the
// largest of all, reaches the scale; then the codes mean nothing).
__device__ __forceinline__ unsigned largest_bits(f32x4 x) {
    unsigned b[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = __float_as_uint(x[e]) & 0x7FFFFFFFu;
    return wave_max_u(max(max(b[0], b[1]), max(b[2], b[3])));
}
__device__ __forceinline__ void block_scale(float top, float& scale, float& inv) {
    const bool tiny = top < 0x1p-100f;
    // 1 / top rounded to nearest: the device's reciprocal, off by up to a step, and one correction
    const float r = __builtin_amdgcn_rcpf(top), one_over = __builtin_fmaf(__builtin_fmaf(-top, r, 1.f), r, r);
    scale = tiny ? 0.f : top * (1.f / 448.f);
    inv = tiny ? 0.f : one_over * 448.f;
}
// The bits of |x| inv 2^-120, inv the block's: 2^-120 brings the e4m3 exponents (and zero
// and the subnormals) to those of fp32, whose bits 20 and up are then the code.
// FOLDED: inv is that times 2^-120 already (a block below 2^13, where it is no subnormal).
template <bool FOLDED> __device__ __forceinline__ unsigned code_bits(float x, float inv) {
    return __float_as_uint(FOLDED ? fabsf(x) * inv : fabsf(x) * inv * 0x1p-120f);
}
// Rounded up where the 16 random bits exceed what rounding down leaves of a step.
__device__ __forceinline__ unsigned e4m3_code(unsigned bits, unsigned rnd16) {
    return min((bits + (rnd16 << 4) + 8u) >> 20, 126u);
}
// The square root rounded to nearest, of 0 and of what lies from 2^-96 to the largest float:
// the device's, off by up to a step, and one correction from its exact remainder (half the
// instructions of sqrtf).
__device__ __forceinline__ float root_of(float x) {
    const float s = __builtin_amdgcn_sqrtf(x);
    return __builtin_fmaf(__builtin_fmaf(-s, s, x), 0.5f * __builtin_amdgcn_rcpf(fmaxf(s, 1e-30f)), s);
}
// Of four values that are not negative, any of them: below 2^-96, where the device's root
// drops subnormals and the remainder has no bits left, that of 2^64 as much; of an infinity itself.
// Two instructions a value tell the ordinary four: 336M bf16 633 us, 626 without, 652 with every
// value scaled; 2.2M fp32 11.7, 11.2, 11.5.
__device__ __forceinline__ f32x4 roots_of(f32x4 x) {
    unsigned least = ~0u, most = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        least = min(least, __float_as_uint(x[e]) - 1u);  // a zero comes last
        most = max(most, __float_as_uint(x[e]));
    }
    f32x4 r;
    if (least >= 0x0F7FFFFFu && most < 0x7F800000u) {
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = root_of(x[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool low = x[e] < 0x1p-96f;
            const float s = root_of(low ? x[e] * 0x1p64f : x[e]);
            r[e] = x[e] == INFINITY ? x[e] : low ? s * 0x1p-32f : s;
        }
    }
    return r;
}

// What four lanes' worth of memory holds before the update.
template <typename P, typename G, int BITS> struct Quad {
    typename Four<P>::vec p;
    typename Four<G>::vec g;
    typename std::conditional<BITS == 32, f32x4, Codes::vec>::type m, v;
    float sm, sv;
    __device__ __forceinline__ void load(const AdamwTensor& T, long i, bool whole) {
        typedef typename std::conditional<BITS == 32, Four<float>, Codes>::type S;
        p = Four<P>::load(T.p, i, T.n, whole);
        g = Four<G>::load(T.g, i, T.n, whole);
        m = S::load(T.m, i, T.n, whole);
        v = S::load(T.v, i, T.n, whole);
        if (BITS == 8) {
            sm = T.ms[i / GP_STATE_BLOCK];
            sv = T.vs[i / GP_STATE_BLOCK];
        }
    }
};
// The update of four consecutive elements from i on; the 64 lanes of a wave have one
// block of the 8-bit states.
template <typename P, typename G, int BITS>
__device__ __forceinline__ void update4(const AdamwTensor& T, const AdamwScalars& s, const AdamwStep& st,
                                        const Quad<P, G, BITS>& q, long i, bool whole) {
#pragma clang fp contract(off)
    f32x4 pv = Four<P>::values(q.p), mv, vv, root;
    const f32x4 gv = Four<G>::values(q.g);
    if constexpr (BITS == 32) {
        mv = q.m;
        vv = q.v;
    } else {
        mv = e4m3_values(q.m) * q.sm;
        vv = e4m3_values(q.v) * q.sv;
        vv = vv * vv;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float m = mv[e], v = vv[e];
        adamw_moments(gv[e], m, v, s, st);
        mv[e] = m;
        vv[e] = v;
        if constexpr (BITS == 32) pv[e] = adamw_param(pv[e], m, v, T.keep, s, st);
    }
    if constexpr (BITS == 8) {  // the parameter's step by a reciprocal that is off by a step
        root = roots_of(vv);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float den = __builtin_fmaf(root[e], st.inv_root, s.eps);
            pv[e] = __builtin_fmaf(pv[e], T.keep, -st.step_size * mv[e] * __builtin_amdgcn_rcpf(den));
        }
    }
    Four<P>::store(T.p, i, T.n, whole, Four<P>::rounded(pv));
    if (T.c) Four<bf16>::store(T.c, i, T.n, whole, Four<bf16>::rounded(pv));
    if constexpr (BITS == 32) {
        Four<float>::store(T.m, i, T.n, whole, mv);
        Four<float>::store(T.v, i, T.n, whole, vv);
    } else {
        const float tm = __uint_as_float(largest_bits(mv)), tr = __uint_as_float(largest_bits(root));
        float sm, im, sr, ir;
        block_scale(tm, sm, im);
        block_scale(tr, sr, ir);
        unsigned h = (unsigned)(i / 4) + st.key;
        h ^= h >> 16;
        h *= 0x6A3F9B15u;
        h ^= h >> 15;
        h *= 0x5D47C1E3u;
        h ^= h >> 16;
        constexpr unsigned K[4] = {0x4F1BBCDDu, 0x7A6D2C8Bu, 0x35E9A1F7u, 0x1D872B41u};
        unsigned qm = 0, qr = 0;
        // What is not zero in v does not become zero: at least code 1 (told from the root itself, whose
        // scaled bits are 0 from 2^-38 of the block's largest down); 0 in a block stored as zeros.
        // In a block with an infinite v every one becomes infinite (a zero times the scale would be a NaN).
        const unsigned least = sr != 0.f ? 1u : 0u, lost = sr == INFINITY ? 1u : 0u;
        auto codes = [&](auto folded, float am, float ar) {
            constexpr bool F = decltype(folded)::value;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned u = h * K[e], bm = code_bits<F>(mv[e], am), br = code_bits<F>(root[e], ar);
                const unsigned sign = __float_as_uint(mv[e]) >> 24 & 0x80u;
                qm |= (e4m3_code(bm, u & 0xFFFFu) | sign) << (8 * e);
                const unsigned some = __float_as_uint(root[e]) | (F ? 0u : lost);
                qr |= max(e4m3_code(br, u >> 16), min(some, least)) << (8 * e);
            }
        };
        if (tm < 0x1p13f && tr < 0x1p13f)
            codes(std::true_type{}, im * 0x1p-120f, ir * 0x1p-120f);
        else  // (a reciprocal that could be subnormal takes the whole division)
            codes(std::false_type{}, tm < 0x1p-100f ? 0.f : 1.f / tm * 448.f, tr < 0x1p-100f ? 0.f : 1.f / tr * 448.f);
        Codes::store(T.m, i, T.n, whole, __builtin_bit_cast(Codes::vec, qm));
        Codes::store(T.v, i, T.n, whole, __builtin_bit_cast(Codes::vec, qr));
        if ((threadIdx.x & 63) == 0) {
            T.ms[i / GP_STATE_BLOCK] = sm;
            T.vs[i / GP_STATE_BLOCK] = sr;
        }
    }
}

// A workgroup per chunk of 4096 elements, whose loads all come before their first use.
// Bound by HBM: 336M fp32 parameters with bf16 copies 1.90 ms (10.1 GB, 5.3 TB/s); 336M bf16
// with 8-bit states 624 to 646 us by the card (3.4 GB, 5.3 to 5.4 TB/s), where the 67 vector
// instructions a value are near their limit too (1.7 times as many took 920 us).
template <typename P, typename G, int BITS>
__global__ void __launch_bounds__(256) adamw_kernel(const AdamwBatch b, const AdamwScalars s) {
    AdamwStep st;
    if (!adamw_begin(s, st)) return;
    const int at = tensor_of(b.chunk0, b.n, blockIdx.x);
    const AdamwTensor& T = b.t[at];
    const long base = (long)((int)blockIdx.x - b.chunk0[at]) * CHUNK, i = base + (long)threadIdx.x * 4;
    constexpr int U = CHUNK / 1024;
    Quad<P, G, BITS> q[U];
    if (base + CHUNK <= T.n) {  // every load of the chunk before the first use
#pragma unroll
        for (int u = 0; u < U; ++u) q[u].load(T, i + u * 1024, true);
#pragma unroll
        for (int u = 0; u < U; ++u) update4<P, G, BITS>(T, s, st, q[u], i + u * 1024, true);
        return;
    }
    const int lane4 = 4 * (int)(threadIdx.x & 63);
#pragma unroll 1
    for (int u = 0; u < U; ++u) {
        const long k = i + u * 1024;
        if (k - lane4 >= T.n) break;  // the wave's block is behind the end
        q[0].load(T, k, k + 4 <= T.n);
        update4<P, G, BITS>(T, s, st, q[0], k, k + 4 <= T.n);
    }
}

// step_dev of a captured update: one more, unless the update is skipped.
__global__ void advance_kernel(long long* step, const float* factor) {
    if (!factor || factor[0] == factor[0]) step[0] += 1;
}

// ------------------------------------------------------------ gradient norm
constexpr int NORM_BLOCKS = 2048;  // workgroups at most, but for the tensors' ragged ends

struct NormTensor {
    const void* g;
    long n;
};
constexpr int NORM_BATCH = 128;
struct NormBatch {
    int n;
    int chunk0[NORM_BATCH];
    NormTensor t[NORM_BATCH];
};

// Bound by HBM: 336M fp32 gradients 243 us (1.34 GB, 5.5 TB/s), four loads ahead of their
// use; a conversion and a product-sum in fp64 per value, which the vector units do at half
// their fp32 rate, stay hidden.
template <typename G>
__global__ void __launch_bounds__(256) norm_kernel(const NormBatch b, long chunk, double* __restrict__ partial) {
    __shared__ double red[4];
    const int at = tensor_of(b.chunk0, b.n, blockIdx.x);
    const NormTensor& T = b.t[at];
    const long base = (long)((int)blockIdx.x - b.chunk0[at]) * chunk, end = min(T.n, base + chunk);
    double s = 0.0;
    long i = base + (long)threadIdx.x * 4;
    constexpr int U = 4;
    auto add = [&](f32x4 x) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_fma((double)x[e], (double)x[e], s);
    };
    for (; i + (U - 1) * 1024 + 4 <= end; i += U * 1024) {
        typename Four<G>::vec x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = Four<G>::load(T.g, i + u * 1024, end, true);
#pragma unroll
        for (int u = 0; u < U; ++u) add(Four<G>::values(x[u]));
    }
    for (; i < end; i += 1024) add(Four<G>::values(Four<G>::load(T.g, i, end, i + 4 <= end)));
    s = wave_sum_d(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) partial[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// The norm and the factor that clips it: a NaN where the norm, as it is stored, is not finite.
__device__ __forceinline__ void write_norm(double sum, float max_norm, float* __restrict__ out) {
    const double norm = sqrt(sum);
    const double f = norm > (double)max_norm ? (double)max_norm / norm : 1.0;
    out[0] = (float)norm;
    out[1] = isfinite((float)norm) ? (float)f : NAN;
}

__global__ void __launch_bounds__(256) norm_finish_kernel(const double* __restrict__ partial, int n, float max_norm,
                                                          float* __restrict__ out) {
    __shared__ double red[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) s += partial[i];
    s = wave_sum_d(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) write_norm((red[0] + red[1]) + (red[2] + red[3]), max_norm, out);
}

// The whole of a short list in one workgroup and launch: wave w takes the chunks w, w + 16,
// .. of SMALL_CHUNK elements.  A wave's chunks are a chain of reads, so it is for lists whose
// second launch costs the host more than that: up to SMALL_CHUNKS chunks.  us a call, so /
// in two launches: one tensor of 100 7.2 / 9.4, of 100000 6.6 / 9.4, 32 of 1000 6.8 / 9.3, 100 of 64
// 8.5 / 9.5, and the one loss within the limit, 100 of 1000, 10.4 / 9.7; past it, 160 chunks, 8.6 to
// 9.9 / 9.2.
constexpr int SMALL_CHUNK = 1024, SMALL_CHUNKS = 120;
template <typename G>
__global__ void __launch_bounds__(1024) norm_small_kernel(const NormBatch b, int chunks, float max_norm,
                                                          float* __restrict__ out) {
    __shared__ double red[16];
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    double s = 0.0;
    for (int id = w; id < chunks; id += 16) {
        const int at = tensor_of(b.chunk0, b.n, id);
        const NormTensor& T = b.t[at];
        const long base = (long)(id - b.chunk0[at]) * SMALL_CHUNK, i = base + lane * 4;
        constexpr int U = SMALL_CHUNK / 256;
        typename Four<G>::vec x[U];
        if (base + SMALL_CHUNK <= T.n) {
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = Four<G>::load(T.g, i + u * 256, T.n, true);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                x[u] = typename Four<G>::vec{};
                if (base + u * 256 < T.n) x[u] = Four<G>::load(T.g, i + u * 256, T.n, i + u * 256 + 4 <= T.n);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const f32x4 v = Four<G>::values(x[u]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_fma((double)v[e], (double)v[e], s);
        }
    }
    s = wave_sum_d(s);
    if (lane == 0) red[w] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = red[0];
        for (int i = 1; i < 16; ++i) t += red[i];
        write_norm(t, max_norm, out);
    }
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t elt_size(int dtype) { return dtype == GP_BF16 ? 2 : 4; }

// The capture state of a stream; a query that fails counts as none.
bool capturing(hipStream_t st) {
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(st, &cs) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    return cs != hipStreamCaptureStatusNone;
}

gp_status check_adamw(const gp_adamw_tensor* t, int n, const gp_adamw_config* c, long long step,
                      const long long* step_dev, const float* factor) {
    auto bad = [](const char* m) { return set_error(GP_ERR_INVALID_ARG, m); };
    if (n < 0 || (n > 0 && !t) || !c) return bad("adamw: n must be >= 0, tensors and cfg not NULL");
    if ((c->param_dtype != GP_F32 && c->param_dtype != GP_BF16) || (c->grad_dtype != GP_F32 && c->grad_dtype != GP_BF16))
        return bad("adamw: unknown dtype");
    if (c->state_bits != 32 && c->state_bits != 8) return bad("adamw: state_bits must be 32 or 8");
    if (!(c->lr >= 0.0 && std::isfinite(c->lr)) || !(c->beta1 >= 0.0 && c->beta1 < 1.0) ||
        !(c->beta2 >= 0.0 && c->beta2 < 1.0) || !((float)c->eps > 0.f && std::isfinite(c->eps)))
        return bad("adamw: lr must be >= 0, betas in [0, 1), eps > 0, all finite");
    // the 8-bit form's reciprocal of a subnormal is infinite, and 0 times it (no gradient yet) a NaN
    if (c->state_bits == 8 && (float)c->eps < 0x1p-126f) return bad("adamw: 8-bit states need eps >= 2^-126");
    if (step_dev ? step != 0 : step < 1) return bad("adamw: give a step >= 1, or step_dev and step 0");
    if (!aligned(step_dev, 8) || !aligned(factor, 4)) return bad("adamw: misaligned step_dev or factor");
    for (int i = 0; i < n; ++i) {
        const gp_adamw_tensor& x = t[i];
        if (x.count < 0) return bad("adamw: negative count");
        if (x.count > (1LL << 40)) return bad("adamw: a tensor of more than 2^40 elements");
        if (!(x.weight_decay >= 0.0) || !(c->lr * x.weight_decay <= 1.0))
            return bad("adamw: weight_decay must be >= 0 and lr weight_decay <= 1");
        if (x.copy && c->param_dtype != GP_F32) return bad("adamw: a working copy belongs to fp32 parameters");
        const bool scales = x.m_scale || x.v_scale;
        if (c->state_bits == 32 && scales) return bad("adamw: scales belong to 8-bit states");
        if (x.count == 0) continue;
        if (!x.param || !x.grad || !x.m || !x.v) return bad("adamw: a tensor's param, grad, m and v must not be NULL");
        if (c->state_bits == 8 && (!x.m_scale || !x.v_scale)) return bad("adamw: 8-bit states need both scales");
        const size_t sb = c->state_bits == 32 ? 4 : 1;
        if (!aligned(x.param, elt_size(c->param_dtype)) || !aligned(x.grad, elt_size(c->grad_dtype)) ||
            !aligned(x.m, sb) || !aligned(x.v, sb) || !aligned(x.m_scale, 4) || !aligned(x.v_scale, 4) ||
            !aligned(x.copy, 2))
            return bad("adamw: an address is not aligned to its elements");
    }
    return GP_OK;
}

template <typename P, typename G>
void launch_adamw(const AdamwBatch& b, const AdamwScalars& s, int chunks, int bits, hipStream_t st) {
    if (bits == 32)
        klaunch(adamw_kernel<P, G, 32>, chunks, 256, 0, st, b, s);
    else
        klaunch(adamw_kernel<P, G, 8>, chunks, 256, 0, st, b, s);
}

} // namespace

gp_status adamw_advance(long long* step, const float* factor, hipStream_t st) {
    klaunch(advance_kernel, 1, 1, 0, st, step, factor);
    GP_LAUNCH_CHECK();
    return GP_OK;
}

} // namespace gp

using namespace gp;

extern "C" {

gp_status gp_adamw_step(const gp_adamw_tensor* tensors, int n, const gp_adamw_config* cfg, long long step,
                        long long* step_dev, const float* factor, gp_stream stream) {
    const gp_status ok = check_adamw(tensors, n, cfg, step, step_dev, factor);
    if (ok != GP_OK) return ok;
    hipStream_t st = (hipStream_t)stream;
    if (!step_dev && capturing(st))
        return set_error(GP_ERR_STATE, "adamw: a captured update needs step_dev (a replay would repeat its step)");
    const AdamwScalars s =
        adamw_scalars(cfg->lr, cfg->beta1, cfg->beta2, cfg->eps, cfg->seed, step, step_dev, factor);
    if (step_dev) {
        const gp_status advanced = adamw_advance(step_dev, factor, st);
        if (advanced != GP_OK) return advanced;
    }
    for (int i = 0; i < n;) {
        AdamwBatch b;
        b.n = 0;
        long chunks = 0;
        for (; i < n && b.n < BATCH; ++i) {
            const gp_adamw_tensor& x = tensors[i];
            const long more = (long)((x.count + CHUNK - 1) / CHUNK);
            if (more == 0) continue;
            if (chunks + more > 0x7FFFFFFFL) break;
            b.chunk0[b.n] = (int)chunks;
            b.t[b.n++] = {x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, static_cast<bf16*>(x.copy), (long)x.count,
                          (float)(1.0 - cfg->lr * x.weight_decay)};
            chunks += more;
        }
        if (b.n == 0) break;
        const int bits = cfg->state_bits;
        if (cfg->param_dtype == GP_F32 && cfg->grad_dtype == GP_F32)
            launch_adamw<float, float>(b, s, (int)chunks, bits, st);
        else if (cfg->param_dtype == GP_F32)
            launch_adamw<float, bf16>(b, s, (int)chunks, bits, st);
        else if (cfg->grad_dtype == GP_F32)
            launch_adamw<bf16, float>(b, s, (int)chunks, bits, st);
        else
            launch_adamw<bf16, bf16>(b, s, (int)chunks, bits, st);
    }
    GP_LAUNCH_CHECK();
    return GP_OK;
}

gp_status gp_grad_norm_workspace(int n, size_t* bytes) {
    if (n < 0 || !bytes) return set_error(GP_ERR_INVALID_ARG, "grad_norm: n must be >= 0 and bytes not NULL");
    *bytes = ((size_t)NORM_BLOCKS + n) * sizeof(double);
    return GP_OK;
}

gp_status gp_grad_norm(int dtype, const gp_grad_tensor* grads, int n, float max_norm, float* norm_factor, void* ws,
                       size_t ws_bytes, gp_stream stream) {
    auto bad = [](const char* m) { return set_error(GP_ERR_INVALID_ARG, m); };
    if (dtype != GP_F32 && dtype != GP_BF16) return bad("grad_norm: unknown dtype");
    if (n < 0 || (n > 0 && !grads) || !norm_factor) return bad("grad_norm: n must be >= 0, grads and norm_factor not NULL");
    if (!(max_norm > 0.f)) return bad("grad_norm: max_norm must be > 0");
    if (!aligned(norm_factor, 4) || !ws || !aligned(ws, 8) || ws_bytes < ((size_t)NORM_BLOCKS + n) * sizeof(double))
        return bad("grad_norm: misaligned output, or a workspace that is NULL, misaligned or too small");
    const size_t ge = elt_size(dtype);
    long long total = 0;
    for (int i = 0; i < n; ++i) {
        if (grads[i].count < 0 || grads[i].count > (1LL << 40)) return bad("grad_norm: a count out of range");
        if (grads[i].count && (!grads[i].grad || !aligned(grads[i].grad, ge)))
            return bad("grad_norm: a gradient is NULL or not aligned to its elements");
        total += grads[i].count;
    }
    hipStream_t st = (hipStream_t)stream;
    long small = 0;  // chunks, if the list is short enough for one workgroup
    for (int i = 0; i < n && n <= NORM_BATCH && small <= SMALL_CHUNKS; ++i)
        small += (long)((grads[i].count + SMALL_CHUNK - 1) / SMALL_CHUNK);
    if (n <= NORM_BATCH && small <= SMALL_CHUNKS) {
        NormBatch b;
        b.n = 0;
        int chunks = 0;
        for (int i = 0; i < n; ++i) {
            if (grads[i].count == 0) continue;
            b.chunk0[b.n] = chunks;
            b.t[b.n++] = {grads[i].grad, (long)grads[i].count};
            chunks += (int)((grads[i].count + SMALL_CHUNK - 1) / SMALL_CHUNK);
        }
        if (dtype == GP_BF16)
            klaunch(norm_small_kernel<bf16>, 1, 1024, 0, st, b, chunks, max_norm, norm_factor);
        else
            klaunch(norm_small_kernel<float>, 1, 1024, 0, st, b, chunks, max_norm, norm_factor);
        GP_LAUNCH_CHECK();
        return GP_OK;
    }
    // chunks of one size, so many that a tensor's last one is the only short one
    const long chunk = std::max<long>(4096, (long)((total / NORM_BLOCKS + 4096) / 4096 * 4096));
    double* partial = static_cast<double*>(ws);
    int used = 0;
    for (int i = 0; i < n;) {
        NormBatch b;
        b.n = 0;
        int chunks = 0;
        for (; i < n && b.n < NORM_BATCH; ++i) {
            const int more = (int)((grads[i].count + chunk - 1) / chunk);
            if (more == 0) continue;
            b.chunk0[b.n] = chunks;
            b.t[b.n++] = {grads[i].grad, (long)grads[i].count};
            chunks += more;
        }
        if (b.n == 0) break;
        if (dtype == GP_BF16)
            klaunch(norm_kernel<bf16>, chunks, 256, 0, st, b, chunk, partial + used);
        else
            klaunch(norm_kernel<float>, chunks, 256, 0, st, b, chunk, partial + used);
        used += chunks;
    }
    klaunch(norm_finish_kernel, 1, 256, 0, st, partial, used, max_norm, norm_factor);
    GP_LAUNCH_CHECK();
    return GP_OK;
}

} // extern "C"
