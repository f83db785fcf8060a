// adamw.hip -- the AdamW update of many tensors at once, states in 32 or in 8
// bits, and the global gradient norm that clips it.
//
// The tensors of a call travel in the kernel arguments, BATCH of them per
// launch: no table in device memory, nothing to copy or to keep alive, and a
// captured launch holds its own.  A workgroup takes one chunk of one tensor
// (the last tensor whose first chunk is not after the workgroup's index).
#include <cmath>

#include "common.hpp"

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
    int chunk0;  // chunks of the launch's tensors before this one
    int vec;     // every address allows 4-element accesses
};
struct AdamwBatch {
    AdamwTensor t[BATCH];
    int n;
};
struct AdamwScalars {
    float lr, b1, c1, b2, c2, eps;  // c = 1 - b
    float ln_b1, ln_b2;             // step_dev: the bias corrections are computed on the device
    float step_size, inv_root;      // else: lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    unsigned key;                   // of the random bits: the seed's part, and with a host step t's
    const long long* step_dev;
    const float* factor;
};
constexpr unsigned KEY_SEED = 0x3C6EF372u, KEY_STEP = 0x1E3779B1u;

template <typename Batch> __device__ __forceinline__ int tensor_of(const Batch& b, int id) {
    int l = 0;
    for (int hi = b.n; l + 1 < hi;) {
        const int mid = (l + hi) / 2;
        if (b.t[mid].chunk0 <= id)
            l = mid;
        else
            hi = mid;
    }
    return l;
}

template <typename T> __device__ __forceinline__ f32x4 load4(const T* p, long i, long n, int vec) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
    if (vec && i + 4 <= n) {
        const T4 x = *reinterpret_cast<const T4*>(p + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = to_f32(x[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) r[e] = to_f32(p[i + e]);
    }
    return r;
}
template <typename T> __device__ __forceinline__ void store4(T* p, long i, long n, int vec, f32x4 x) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    if (vec && i + 4 <= n) {
        *reinterpret_cast<T4*>(p + i) = T4{to_elt<T>(x[0]), to_elt<T>(x[1]), to_elt<T>(x[2]), to_elt<T>(x[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) p[i + e] = to_elt<T>(x[e]);
    }
}
__device__ __forceinline__ unsigned load_codes(const unsigned char* p, long i, long n, int vec) {
    if (vec && i + 4 <= n) return *reinterpret_cast<const unsigned*>(p + i);
    unsigned r = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (i + e < n) r |= (unsigned)p[i + e] << (8 * e);
    return r;
}
__device__ __forceinline__ void store_codes(unsigned char* p, long i, long n, int vec, unsigned q) {
    if (vec && i + 4 <= n) {
        *reinterpret_cast<unsigned*>(p + i) = q;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) p[i + e] = (unsigned char)(q >> (8 * e));
    }
}
// The four values of packed e4m3 codes.
__device__ __forceinline__ f32x4 e4m3_values(unsigned q) {
    return f32x4{__builtin_amdgcn_cvt_f32_fp8((int)q, 0), __builtin_amdgcn_cvt_f32_fp8((int)q, 1),
                 __builtin_amdgcn_cvt_f32_fp8((int)q, 2), __builtin_amdgcn_cvt_f32_fp8((int)q, 3)};
}
// |y| <= 448 to e4m3, rounded up where the 16 random bits exceed what rounding down
// leaves of a step: 2^-120 brings the e4m3 exponents (and zero and the subnormals) to
// those of fp32, whose bits 20 and up are then the code.
__device__ __forceinline__ unsigned e4m3_code(float y, unsigned rnd16) {
    const unsigned c = (__float_as_uint(fabsf(y) * 0x1p-120f) + (rnd16 << 4) + 8u) >> 20;
    return c < 126u ? c : 126u;
}
// A block's scale and its inverse from the largest |x|; NaN and infinities come through as NaN.
__device__ __forceinline__ void block_scale(float top, float& scale, float& inv) {
    const bool tiny = top < 0x1p-100f;
    scale = tiny ? 0.f : top * (1.f / 448.f);
    inv = tiny ? 0.f : 1.f / top * 448.f;
}
// fmaxf drops a NaN; here it has to reach the scale.
__device__ __forceinline__ float max_nan(float a, float b) { return b > a || b != b ? b : a; }
__device__ __forceinline__ float wave_max_nan(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max_nan(v, __shfl_xor(v, o, WAVE));
    return v;
}

// Four consecutive elements per lane, so that a wave's 256 are one block of the
// 8-bit states.  Every product and sum is rounded by itself, in the order of the
// formulas, so that an update is the same bits wherever it is compiled.
template <typename P, typename G, int BITS>
__global__ void __launch_bounds__(256) adamw_kernel(const AdamwBatch b, const AdamwScalars s) {
#pragma clang fp contract(off)
    const float factor = s.factor ? s.factor[0] : 1.f;
    if (factor != factor) return;
    float step_size = s.step_size, inv_root = s.inv_root;
    unsigned key = s.key;
    if (s.step_dev) {
        const long long t = s.step_dev[0];
        step_size = s.lr / -expm1f((float)t * s.ln_b1);
        inv_root = 1.f / sqrtf(-expm1f((float)t * s.ln_b2));
        key += KEY_STEP * (unsigned)t;
    }
    const AdamwTensor& T = b.t[tensor_of(b, blockIdx.x)];
    const long n = T.n, base = (long)((int)blockIdx.x - T.chunk0) * CHUNK;
    P* p = static_cast<P*>(T.p);
    const G* g = static_cast<const G*>(T.g);
    const int lane = threadIdx.x & 63;
    const unsigned K[4] = {0x4F1BBCDDu, 0x7A6D2C8Bu, 0x35E9A1F7u, 0x1D872B41u};
#pragma unroll
    for (int it = 0; it < CHUNK / 1024; ++it) {
        const long i = base + it * 1024 + (long)threadIdx.x * 4;
        const long block = i / GP_STATE_BLOCK;
        if (i - 4 * lane >= n) return;  // the wave's block is behind the end
        f32x4 pv = load4(p, i, n, T.vec), gv = load4(g, i, n, T.vec), mv, vv;
        if constexpr (BITS == 32) {
            mv = load4(static_cast<const float*>(T.m), i, n, T.vec);
            vv = load4(static_cast<const float*>(T.v), i, n, T.vec);
        } else {
            mv = e4m3_values(load_codes(static_cast<const unsigned char*>(T.m), i, n, T.vec)) * T.ms[block];
            vv = e4m3_values(load_codes(static_cast<const unsigned char*>(T.v), i, n, T.vec)) * T.vs[block];
            vv = vv * vv;
        }
        f32x4 root;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float ge = gv[e] * factor;
            mv[e] = mv[e] * s.b1 + ge * s.c1;
            vv[e] = vv[e] * s.b2 + ge * ge * s.c2;
            root[e] = sqrtf(vv[e]);
            pv[e] = pv[e] * T.keep - step_size * mv[e] / (root[e] * inv_root + s.eps);
        }
        store4(p, i, n, T.vec, pv);
        if (T.c) store4(T.c, i, n, T.vec, pv);
        if constexpr (BITS == 32) {
            store4(static_cast<float*>(T.m), i, n, T.vec, mv);
            store4(static_cast<float*>(T.v), i, n, T.vec, vv);
        } else {
            float tm = 0.f, tr = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                tm = max_nan(tm, fabsf(mv[e]));
                tr = max_nan(tr, root[e]);
            }
            float sm, im, sr, ir;
            block_scale(wave_max_nan(tm), sm, im);
            block_scale(wave_max_nan(tr), sr, ir);
            unsigned h = (unsigned)(i / 4) + key;
            h ^= h >> 16;
            h *= 0x6A3F9B15u;
            h ^= h >> 15;
            h *= 0x5D47C1E3u;
            h ^= h >> 16;
            unsigned qm = 0, qr = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned u = h * K[e];
                const float ym = mv[e] * im, yr = root[e] * ir;
                unsigned cr = e4m3_code(yr, u >> 16);
                cr = yr > 0.f && cr == 0 ? 1u : cr;
                qm |= (e4m3_code(ym, u & 0xFFFFu) | (ym < 0.f ? 128u : 0u)) << (8 * e);
                qr |= cr << (8 * e);
            }
            store_codes(static_cast<unsigned char*>(T.m), i, n, T.vec, qm);
            store_codes(static_cast<unsigned char*>(T.v), i, n, T.vec, qr);
            if (lane == 0) {
                T.ms[block] = sm;
                T.vs[block] = sr;
            }
        }
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
    int chunk0;
    int vec;
};
constexpr int NORM_BATCH = 128;
struct NormBatch {
    NormTensor t[NORM_BATCH];
    int n;
};

template <typename G>
__global__ void __launch_bounds__(256) norm_kernel(const NormBatch b, long chunk, double* __restrict__ partial) {
    __shared__ double red[4];
    const NormTensor& T = b.t[tensor_of(b, blockIdx.x)];
    const long base = (long)((int)blockIdx.x - T.chunk0) * chunk, end = min(T.n, base + chunk);
    const G* g = static_cast<const G*>(T.g);
    double s = 0.0;
    for (long i = base + (long)threadIdx.x * 4; i < end; i += 1024) {
        const f32x4 x = load4(g, i, end, T.vec);
#pragma unroll
        for (int e = 0; e < 4; ++e) s += (double)x[e] * (double)x[e];
    }
    s = wave_sum_d(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) partial[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ void __launch_bounds__(256) norm_finish_kernel(const double* __restrict__ partial, int n, float max_norm,
                                                          float* __restrict__ out) {
    __shared__ double red[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) s += partial[i];
    s = wave_sum_d(s);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        const double norm = sqrt((red[0] + red[1]) + (red[2] + red[3]));
        const double f = norm > (double)max_norm ? (double)max_norm / norm : 1.0;
        out[0] = (float)norm;
        out[1] = isfinite(norm) ? (float)f : NAN;
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
    AdamwScalars s{};
    s.lr = (float)cfg->lr;
    s.b1 = (float)cfg->beta1;
    s.c1 = (float)(1.0 - cfg->beta1);
    s.b2 = (float)cfg->beta2;
    s.c2 = (float)(1.0 - cfg->beta2);
    s.eps = (float)cfg->eps;
    s.key = KEY_SEED * cfg->seed;
    s.step_dev = step_dev;
    s.factor = factor;
    if (step_dev) {
        s.ln_b1 = (float)std::log(cfg->beta1);
        s.ln_b2 = (float)std::log(cfg->beta2);
        klaunch(advance_kernel, 1, 1, 0, st, step_dev, factor);
    } else {
        s.step_size = (float)(cfg->lr / (1.0 - std::pow(cfg->beta1, (double)step)));
        s.inv_root = (float)(1.0 / std::sqrt(1.0 - std::pow(cfg->beta2, (double)step)));
        s.key += KEY_STEP * (unsigned)step;
    }
    const size_t pe = elt_size(cfg->param_dtype), ge = elt_size(cfg->grad_dtype);
    for (int i = 0; i < n;) {
        AdamwBatch b;
        b.n = 0;
        long chunks = 0;
        for (; i < n && b.n < BATCH; ++i) {
            const gp_adamw_tensor& x = tensors[i];
            const long more = (long)((x.count + CHUNK - 1) / CHUNK);
            if (more == 0) continue;
            if (chunks + more > 0x7FFFFFFFL) break;
            const size_t sb = cfg->state_bits == 32 ? 16 : 4;
            const bool vec = aligned(x.param, 4 * pe) && aligned(x.grad, 4 * ge) && aligned(x.m, sb) &&
                             aligned(x.v, sb) && aligned(x.copy, 8);
            b.t[b.n++] = {x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, static_cast<bf16*>(x.copy), (long)x.count,
                          (float)(1.0 - cfg->lr * x.weight_decay), (int)chunks, vec ? 1 : 0};
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
            b.t[b.n++] = {grads[i].grad, (long)grads[i].count, chunks, aligned(grads[i].grad, 4 * ge) ? 1 : 0};
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
