// logprob.hip -- log probabilities of given tokens under rows of logits, the
// rows' entropy and most likely tokens, and the gradient of the first two.
#include <algorithm>
#include <cmath>

#include "common.hpp"

namespace gp {

namespace {

constexpr float LOG2E = 1.44269504088896341f;
constexpr float NEVER = -1e30f;  // a logit down here is a mask's, its token cannot occur

// Partial sums of a row: the largest s, sum exp(s - m), sum exp(s - m) (s - m).
struct Part {
    float m, a, b;
};
// A term of the sums; -inf (a token that cannot occur) adds nothing, NaN and
// +inf make a NaN.
__device__ __forceinline__ void add_term(Part& p, float s) {
    const float m = fmaxf(p.m, s);
    if (m > p.m) {
        const float f = __builtin_amdgcn_exp2f((p.m - m) * LOG2E);  // 0 for the first term
        p.b = f > 0.f ? f * (p.b + p.a * (p.m - m)) : 0.f;
        p.a *= f;
        p.m = m;
    }
    const float d = s - (m == -INFINITY ? 0.f : m);
    const float e = __builtin_amdgcn_exp2f(d * LOG2E);
    p.a += e;
    p.b += e * fmaxf(d, -1e30f);
}
__device__ __forceinline__ Part join(Part x, Part y) {
    const float m = fmaxf(x.m, y.m), mm = m == -INFINITY ? 0.f : m;
    const float dx = fmaxf(x.m - mm, -1e30f), dy = fmaxf(y.m - mm, -1e30f);
    const float fx = __builtin_amdgcn_exp2f(dx * LOG2E), fy = __builtin_amdgcn_exp2f(dy * LOG2E);
    return {m, x.a * fx + y.a * fy, fx * (x.b + x.a * dx) + fy * (y.b + y.a * dy)};
}

// The order of alternatives as one integer: larger logits first (a NaN before all,
// both zeros equal), then the lower index.  No key is 0 or ~0.
constexpr unsigned NAN_ORDER = 0xFFFFFFFEu;
__device__ __forceinline__ unsigned long long rank_key(float x, int v) {
    unsigned u = __float_as_uint(x + 0.f);
    u = (u >> 31) ? ~u : u | 0x80000000u;
    if (x != x) u = NAN_ORDER;
    return ((unsigned long long)u << 32) | (0xFFFFFFFFu - (unsigned)v);
}
__device__ __forceinline__ float key_value(unsigned long long k) {
    const unsigned u = (unsigned)(k >> 32);
    if (u == NAN_ORDER) return NAN;
    return __uint_as_float((u >> 31) ? u & 0x7FFFFFFFu : ~u);
}
__device__ __forceinline__ int key_index(unsigned long long k) { return (int)(0xFFFFFFFFu - (unsigned)k); }

// A workgroup per row: the sums in one pass, then a pass per alternative.
template <typename T>
__global__ void __launch_bounds__(256) logprob_kernel(const T* __restrict__ z, int V, long ld,
                                                      const int* __restrict__ tokens, float scale, float clip,
                                                      float* __restrict__ logp, float* __restrict__ lse_out,
                                                      float* __restrict__ entropy, int top, int* __restrict__ top_ids,
                                                      float* __restrict__ top_logp) {
    __shared__ Part red[4];
    __shared__ unsigned long long best[4];
    const long row = blockIdx.x;
    const T* zr = z + row * ld;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    auto logit = [&](int v) {
        const float x = to_f32(zr[v]);
        return clip > 0.f && x == x ? fminf(fmaxf(x, -clip), clip) : x;
    };
    Part p = {-INFINITY, 0.f, 0.f};
    for (int v = tid; v < V; v += 256) add_term(p, scale * logit(v));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        p = join(p, Part{__shfl_xor(p.m, o, WAVE), __shfl_xor(p.a, o, WAVE), __shfl_xor(p.b, o, WAVE)});
    if (lane == 0) red[w] = p;
    __syncthreads();
    p = join(join(red[0], red[1]), join(red[2], red[3]));
    // the terms of a row of masks alone are those of a constant row, or none
    const bool empty = p.m <= NEVER * scale && p.a == p.a;
    const float la = logf(p.a);
    auto log_prob = [&](float x) { return empty ? -INFINITY : x <= NEVER ? -INFINITY - la : scale * x - p.m - la; };
    if (tid == 0) {
        if (lse_out) lse_out[row] = empty ? -INFINITY : p.m + la;
        if (entropy) entropy[row] = empty ? 0.f : la - p.b / p.a;
        if (logp) {
            const int t = tokens[row];
            float r = NAN;
            if (t == GP_NO_TOKEN)
                r = 0.f;
            else if (t >= 0 && t < V)
                r = log_prob(logit(t));
            logp[row] = r;
        }
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < top; ++k) {
        unsigned long long mine = 0;
        for (int v = tid; v < V; v += 256) {
            const unsigned long long key = rank_key(logit(v), v);
            if (key < last && key > mine) mine = key;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const unsigned long long other = __shfl_xor(mine, o, WAVE);
            mine = other > mine ? other : mine;
        }
        if (lane == 0) best[w] = mine;
        __syncthreads();
        last = std::max(std::max(best[0], best[1]), std::max(best[2], best[3]));
        __syncthreads();
        if (tid == 0) {
            top_ids[row * top + k] = key_index(last);
            top_logp[row * top + k] = log_prob(key_value(last));
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) logprob_grad_kernel(const T* z, int V, long ld, const int* __restrict__ tokens,
                                                           float scale, float clip, const float* __restrict__ lse,
                                                           const float* __restrict__ entropy,
                                                           const float* __restrict__ dlogp,
                                                           const float* __restrict__ dentropy, T* dz, long ldd) {
    const long row = blockIdx.x;
    const T* zr = z + row * ld;
    T* dr = dz + row * ldd;
    const float l = lse[row], lim = clip > 0.f ? clip : INFINITY;
    float a = dlogp ? dlogp[row] : 0.f;
    const float b = dentropy ? dentropy[row] : 0.f, h = dentropy ? entropy[row] : 0.f;
    int t = dlogp ? tokens[row] : GP_NO_TOKEN;
    if (t == GP_NO_TOKEN) {
        a = 0.f;
    } else if (t < 0 || t >= V) {
        a = NAN;
        t = GP_NO_TOKEN;
    }
    const bool empty = l == -INFINITY;
    for (int v = threadIdx.x; v < V; v += 256) {
        const float x = to_f32(zr[v]);
        const float s = scale * (x == x ? fminf(fmaxf(x, -lim), lim) : x);
        const float d = s - l;
        const float p = __builtin_amdgcn_exp2f(d * LOG2E);
        // p is 0 where s is -inf: no product of the two
        float g = -p * (a + b * (fmaxf(d, -1e30f) + h));
        if (v == t) g += a;
        g *= scale;
        const bool stays = empty || (clip > 0.f && fabsf(x) > clip);
        dr[v] = to_elt<T>(stays ? a * 0.f : g);  // a NaN reaches the whole row
    }
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

gp_status check_rows(int dtype, const void* logits, long rows, int vocab, long ld, float scale, float clip) {
    auto bad = [](const char* m) { return set_error(GP_ERR_INVALID_ARG, m); };
    if (dtype != GP_F32 && dtype != GP_BF16) return bad("token_logprobs: unknown dtype");
    if (rows < 0 || rows > 0x7FFFFFFFL) return bad("token_logprobs: rows must be in [0, 2^31 - 1]");
    if (vocab < 1 || ld < vocab) return bad("token_logprobs: vocab must be >= 1 and ld >= vocab");
    if (!(scale > 0.f) || !std::isfinite(scale)) return bad("token_logprobs: scale must be > 0 and finite");
    if (!(clip >= 0.f) || !std::isfinite(clip)) return bad("token_logprobs: clip must be >= 0 and finite");
    if (!logits && rows > 0) return bad("token_logprobs: logits must not be NULL");
    if (!aligned(logits, dtype == GP_BF16 ? 2 : 4)) return bad("token_logprobs: logits not aligned to their elements");
    return GP_OK;
}

} // namespace

} // namespace gp

using namespace gp;

extern "C" {

gp_status gp_token_logprobs_workspace(int dtype, long rows, int vocab, int top, size_t* bytes) {
    if (!bytes || (dtype != GP_F32 && dtype != GP_BF16) || rows < 0 || vocab < 1 || top < 0 || top > GP_TOP_MAX)
        return set_error(GP_ERR_INVALID_ARG, "token_logprobs_workspace: an argument is out of range");
    *bytes = 0;
    return GP_OK;
}

gp_status gp_token_logprobs(int dtype, const void* logits, long rows, int vocab, long ld, const int* tokens,
                            float scale, float clip, float* logp, float* lse, float* entropy, int top, int* top_ids,
                            float* top_logp, void* ws, size_t ws_bytes, gp_stream stream) {
    const gp_status ok = check_rows(dtype, logits, rows, vocab, ld, scale, clip);
    if (ok != GP_OK) return ok;
    auto bad = [](const char* m) { return set_error(GP_ERR_INVALID_ARG, m); };
    if (top < 0 || top > GP_TOP_MAX || top > vocab) return bad("token_logprobs: top must be in [0, min(32, vocab)]");
    if (rows > 0 && top > 0 && (!top_ids || !top_logp)) return bad("token_logprobs: top needs top_ids and top_logp");
    if (rows > 0 && logp && !tokens) return bad("token_logprobs: logp needs tokens");
    for (const void* p : {(const void*)tokens, (const void*)logp, (const void*)lse, (const void*)entropy,
                          (const void*)top_ids, (const void*)top_logp})
        if (!aligned(p, 4)) return bad("token_logprobs: a misaligned address");
    if (!aligned(ws, 16)) return bad("token_logprobs: the workspace must be 16-byte aligned");
    if (rows == 0) return GP_OK;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == GP_BF16)
        klaunch(logprob_kernel<bf16>, (unsigned)rows, 256, 0, st, static_cast<const bf16*>(logits), vocab, ld, tokens,
                scale, clip, logp, lse, entropy, top, top_ids, top_logp);
    else
        klaunch(logprob_kernel<float>, (unsigned)rows, 256, 0, st, static_cast<const float*>(logits), vocab, ld, tokens,
                scale, clip, logp, lse, entropy, top, top_ids, top_logp);
    GP_LAUNCH_CHECK();
    return GP_OK;
}

gp_status gp_token_logprobs_backward(int dtype, const void* logits, long rows, int vocab, long ld, const int* tokens,
                                     float scale, float clip, const float* lse, const float* entropy,
                                     const float* dlogp, const float* dentropy, void* dlogits, long ldd,
                                     gp_stream stream) {
    const gp_status ok = check_rows(dtype, logits, rows, vocab, ld, scale, clip);
    if (ok != GP_OK) return ok;
    auto bad = [](const char* m) { return set_error(GP_ERR_INVALID_ARG, m); };
    if (ldd < vocab) return bad("token_logprobs_backward: ldd must be >= vocab");
    if (rows > 0 && !dlogp && !dentropy) return bad("token_logprobs_backward: dlogp or dentropy must be given");
    if (rows > 0 && (!lse || !dlogits)) return bad("token_logprobs_backward: lse and dlogits must not be NULL");
    if (rows > 0 && ((dlogp && !tokens) || (dentropy && !entropy)))
        return bad("token_logprobs_backward: dlogp needs tokens, dentropy needs entropy");
    const size_t es = dtype == GP_BF16 ? 2 : 4;
    for (const void* p : {(const void*)tokens, (const void*)lse, (const void*)entropy, (const void*)dlogp,
                          (const void*)dentropy})
        if (!aligned(p, 4)) return bad("token_logprobs_backward: a misaligned address");
    if (!aligned(dlogits, es)) return bad("token_logprobs_backward: dlogits not aligned to its elements");
    if (rows == 0) return GP_OK;
    const uintptr_t z0 = reinterpret_cast<uintptr_t>(logits), d0 = reinterpret_cast<uintptr_t>(dlogits);
    const uintptr_t z1 = z0 + ((size_t)(rows - 1) * ld + vocab) * es, d1 = d0 + ((size_t)(rows - 1) * ldd + vocab) * es;
    if (!(z0 == d0 && ld == ldd) && z0 < d1 && d0 < z1)
        return bad("token_logprobs_backward: dlogits overlaps the logits without being them");
    hipStream_t st = (hipStream_t)stream;
    if (dtype == GP_BF16)
        klaunch(logprob_grad_kernel<bf16>, (unsigned)rows, 256, 0, st, static_cast<const bf16*>(logits), vocab, ld,
                tokens, scale, clip, lse, entropy, dlogp, dentropy, static_cast<bf16*>(dlogits), ldd);
    else
        klaunch(logprob_grad_kernel<float>, (unsigned)rows, 256, 0, st, static_cast<const float*>(logits), vocab, ld,
                tokens, scale, clip, lse, entropy, dlogp, dentropy, static_cast<float*>(dlogits), ldd);
    GP_LAUNCH_CHECK();
    return GP_OK;
}

} // extern "C"
