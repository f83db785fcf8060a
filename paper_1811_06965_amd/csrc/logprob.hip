// logprob.hip -- log probabilities of given tokens under rows of logits, the
// rows' entropy and most likely tokens, and the gradient of the first two.
#include <algorithm>
#include <cmath>

#include "common.hpp"

namespace gp {

namespace {

constexpr float LOG2E = 1.44269504088896341f;
constexpr float NEVER = -1e30f;  // a logit down here is a mask's, its token cannot occur
constexpr int ROW_THREADS = 256;
constexpr int SPLIT_MAX = 64;    // workgroups of one row: the lanes of the wave that joins them

__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float min_nan(float a, float b) { return __builtin_elementwise_minimum(a, b); }

// Sums of a row's terms around a reference logit r: with d = x - r, a = sum exp(scale d)
// and b = sum d exp(scale d).  Then lse = scale r + log a and the entropy is
// log a - scale b / a, whatever r is; its term stays within 2^8 of the largest.
// d is finite for every x that is (the reference is subtracted before scaling),
// so a term that vanishes adds no 0 inf.
struct Part {
    float r, a, b;
};
constexpr float NO_REF = -2e30f;  // below every reference
// c2 = scale log2 e
__device__ __forceinline__ Part join(Part x, Part y, float c2) {
    const float r = max_nan(x.r, y.r), dx = x.r - r, dy = y.r - r;
    const float fx = __builtin_amdgcn_exp2f(dx * c2), fy = __builtin_amdgcn_exp2f(dy * c2);
    return {r, x.a * fx + y.a * fy, fx * (x.b + x.a * dx) + fy * (y.b + y.a * dy)};
}
__device__ __forceinline__ Part wave_join(Part p, float c2) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        p = join(p, Part{__shfl_xor(p.r, o, WAVE), __shfl_xor(p.a, o, WAVE), __shfl_xor(p.b, o, WAVE)}, c2);
    return p;
}

// The order of alternatives as one integer: larger logits first (a NaN before all,
// both zeros equal), then the lower index.  No key is 0 or ~0.
typedef unsigned long long u64;
constexpr unsigned NAN_ORDER = 0xFFFFFFFEu;
__device__ __forceinline__ u64 rank_key(float x, int v) {
    unsigned u = __float_as_uint(x + 0.f);
    u = (u >> 31) ? ~u : u | 0x80000000u;
    if (x != x) u = NAN_ORDER;
    return ((u64)u << 32) | (0xFFFFFFFFu - (unsigned)v);
}
__device__ __forceinline__ float key_value(u64 k) {
    const unsigned u = (unsigned)(k >> 32);
    if (u == NAN_ORDER) return NAN;
    return __uint_as_float((u >> 31) ? u & 0x7FFFFFFFu : ~u);
}
__device__ __forceinline__ int key_index(u64 k) { return (int)(0xFFFFFFFFu - (unsigned)k); }
__device__ __forceinline__ u64 wave_max_key(u64 k) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const u64 x = __shfl_xor(k, o, WAVE);
        k = x > k ? x : k;
    }
    return k;
}

// A row in chunks of 16 bytes of memory: chunk j holds the elements N j - mis .. + N - 1
// that lie in [0, V); only the first and the last can be short.
template <typename T> struct Chunks {
    static constexpr int N = Vec16<T>::N;
    typedef typename Vec16<T>::type vec;
    const T* base;  // of chunk 0, 16-byte aligned
    int V, mis, count, f0, f1;  // chunks f0 .. f1 - 1 are whole
    __device__ __forceinline__ Chunks(const T* row, int V_) : V(V_) {
        mis = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        base = row - mis;
        count = (V + mis + N - 1) / N;
        f0 = mis ? 1 : 0;
        f1 = (V + mis) / N;
    }
    __device__ __forceinline__ int first(int j) const { return j * N - mis; }
    __device__ __forceinline__ bool whole(int j) const { return j >= f0 && j < f1; }
    __device__ __forceinline__ vec load(int j) const { return reinterpret_cast<const vec*>(base)[j]; }
    // any chunk; `none` in the places outside the row
    __device__ __forceinline__ void values(int j, float none, float (&x)[N]) const {
        if (whole(j)) {
            const vec v = load(j);
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = to_f32((T)v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int v = first(j) + e;
                x[e] = v >= 0 && v < V ? to_f32(base[(long)j * N + e]) : none;
            }
        }
    }
};

struct RowOut {
    float* logp;
    float* lse;
    float* entropy;
    int* top_ids;
    float* top_logp;
};

// What a row's sums say of one logit: log p.  The reference of a row of masks alone
// is a mask's (the next float up is further off than the 2^8 it may lie above).
struct RowLog {
    float scale, r, la;
    bool empty;
    __device__ __forceinline__ RowLog(Part p, float scale_)
        : scale(scale_), r(p.r), la(logf(p.a)), empty(p.r <= NEVER && p.a == p.a) {}
    __device__ __forceinline__ float operator()(float x) const {
        if (empty) return -INFINITY;
        return x <= NEVER ? -INFINITY - la : scale * (x - r) - la;
    }
};
template <typename T>
__device__ __forceinline__ void write_row(const RowOut& o, long row, Part p, const RowLog& log_p, const T* zr, int V,
                                          const int* tokens, float lo, float hi) {
    if (o.lse) o.lse[row] = log_p.empty ? -INFINITY : log_p.scale * p.r + log_p.la;
    if (o.entropy) o.entropy[row] = log_p.empty ? 0.f : log_p.la - log_p.scale * p.b / p.a;
    if (o.logp) {
        const int t = tokens[row];
        float r = NAN;
        if (t == GP_NO_TOKEN)
            r = 0.f;
        else if (t >= 0 && t < V)
            r = log_p(min_nan(max_nan(to_f32(zr[t]), lo), hi));
        o.logp[row] = r;
    }
}

// A workgroup per row, or `splits` of them, each over `per` chunks of it; thread t
// takes the chunks t, t + 256, ..  One pass gives the sums and each thread's largest
// logit.  Alternatives: the k-th largest of the 256 threads' largest is a bound
// that at least k logits reach, and only the k threads whose largest does hold any
// such logit; those threads' chunks are read a second time and what reaches the
// bound (a few more than k) is ranked.  A row with a NaN, or more than CAND
// such logits, goes through its logits once per alternative instead.
constexpr int CAND = 1024;
template <typename T, bool CLIP, bool TOP>
__global__ void __launch_bounds__(ROW_THREADS) logprob_kernel(const T* __restrict__ z, int V, long ld,
                                                              const int* __restrict__ tokens, float scale, float clip,
                                                              RowOut out, int top, int splits, int per,
                                                              Part* __restrict__ parts, u64* __restrict__ lists) {
    constexpr int N = Chunks<T>::N, U = 4;
    __shared__ Part red[4];
    __shared__ u64 best[TOP ? ROW_THREADS : 1], cand[TOP ? CAND : 1];
    __shared__ int owner[TOP ? GP_TOP_MAX : 1], found;
    const long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits);
    const T* zr = z + row * ld;
    const Chunks<T> ch(zr, V);
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int c0 = min(split * per, ch.count), c1 = min(c0 + per, ch.count);
    const float c2 = scale * LOG2E, near = 8.f / c2, lo = CLIP ? -clip : NEVER, hi = CLIP ? clip : INFINITY;
    auto bounded = [&](float x) { return CLIP ? min_nan(max_nan(x, lo), hi) : max_nan(x, lo); };

    Part p = {NO_REF, 0.f, 0.f};
    float most = -INFINITY;  // this thread's largest logit, and its first chunk that holds it
    int most_j = -1;
    auto add = [&](const float (&x)[N], int j) {
        float cm = x[0];
#pragma unroll
        for (int e = 1; e < N; ++e) cm = max_nan(cm, x[e]);
        if (!(cm <= p.r + near)) {  // NaN too
            const float d = p.r - cm, f = __builtin_amdgcn_exp2f(d * c2);
            p = {cm, p.a * f, f * (p.b + p.a * d)};
        }
        if (TOP && cm > most) {
            most = cm;
            most_j = j;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float d = x[e] - p.r, q = __builtin_amdgcn_exp2f(d * c2);
            p.a += q;
            p.b = __builtin_fmaf(q, d, p.b);
        }
    };
    auto add_any = [&](int j) {  // a chunk that may be short: outside the row, nothing
        float x[N];
        ch.values(j, -INFINITY, x);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int v = ch.first(j) + e;
            x[e] = v >= 0 && v < V ? bounded(x[e]) : NEVER;
        }
        add(x, j);
    };
    if (c0 < ch.f0 && tid == 0 && c0 < c1) add_any(c0);
    int j = c0 + tid;
    if (j < ch.f0) j += ROW_THREADS;
    const int f1 = min(c1, ch.f1);
    for (; j < f1; j += U * ROW_THREADS) {
        typename Chunks<T>::vec v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j + u * ROW_THREADS < f1) v[u] = ch.load(j + u * ROW_THREADS);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j + u * ROW_THREADS >= f1) break;
            float x[N];
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = bounded(to_f32((T)v[u][e]));
            add(x, j + u * ROW_THREADS);
        }
    }
    // the short last chunk, if it is not the first
    if (c1 == ch.count && c1 - 1 >= c0 && ch.f1 < ch.count && c1 - 1 >= ch.f0 && tid == (c1 - 1 - c0) % ROW_THREADS)
        add_any(c1 - 1);

    p = wave_join(p, c2);
    if (lane == 0) red[w] = p;
    if (TOP && tid == 0) found = 0;
    __syncthreads();
    p = join(join(red[0], red[1], c2), join(red[2], red[3], c2), c2);
    const RowLog log_p(p, scale);
    if (splits > 1) {
        if (tid == 0) parts[blockIdx.x] = p;
    } else if (tid == 0) {
        write_row(out, row, p, log_p, zr, V, tokens, lo, hi);
    }
    if constexpr (TOP) {
        auto give = [&](int k, u64 key) {
            if (splits > 1) {
                lists[(long)blockIdx.x * top + k] = key;
            } else {
                out.top_ids[row * top + k] = key_index(key);
                out.top_logp[row * top + k] = log_p(key_value(key));
            }
        };
        // the key of element e of chunk j; 0 outside the row
        auto key_of = [&](float x, int j2, int e) -> u64 {
            const int v = ch.first(j2) + e;
            return v >= 0 && v < V ? rank_key(bounded(x), v) : 0;
        };
        bool slow = p.a != p.a;
        if (!slow) {
            u64 mine = 0;
            if (most_j >= 0) {
                float x[N];
                ch.values(most_j, 0.f, x);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const u64 key = key_of(x[e], most_j, e);
                    mine = key > mine ? key : mine;
                }
            }
            best[tid] = mine;
            __syncthreads();
            int rank = 0;
            for (int i = 0; i < ROW_THREADS; ++i) rank += best[i] > mine ? 1 : 0;
            // fewer than `top` threads hold a logit: then all that do
            if (rank < top && mine) owner[rank] = tid;
            const int owners = min(top, (int)__syncthreads_count(mine != 0));
            const u64 bound = owners == top ? best[owner[top - 1]] : 1;
            const int rounds = (c1 - c0 + ROW_THREADS - 1) / ROW_THREADS;
            for (int i = tid; i < owners * rounds; i += ROW_THREADS) {
                const int j2 = c0 + owner[i % owners] + i / owners * ROW_THREADS;
                if (j2 >= c1) continue;
                float x[N];
                ch.values(j2, 0.f, x);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const u64 key = key_of(x[e], j2, e);
                    if (key >= bound) {
                        const int at = atomicAdd(&found, 1);
                        if (at < CAND) cand[at] = key;
                    }
                }
            }
            __syncthreads();
            const int n = found;
            slow = n > CAND;
            if (!slow) {
                for (int i = tid; i < n; i += ROW_THREADS) {
                    const u64 key = cand[i];
                    int r = 0;
                    for (int k = 0; k < n; ++k) r += cand[k] > key ? 1 : 0;
                    if (r < top) give(r, key);
                }
                for (int k = n + tid; k < top; k += ROW_THREADS) give(k, 0);  // a split of fewer logits
            }
        }
        if (slow) {
            u64 last = ~0ull;
            for (int k = 0; k < top; ++k) {
                u64 mine = 0;
                for (int j2 = c0 + tid; j2 < c1; j2 += ROW_THREADS) {
                    float x[N];
                    ch.values(j2, 0.f, x);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const u64 key = key_of(x[e], j2, e);
                        if (key < last && key > mine) mine = key;
                    }
                }
                mine = wave_max_key(mine);
                __syncthreads();
                if (lane == 0) best[w] = mine;
                __syncthreads();
                last = std::max(std::max(best[0], best[1]), std::max(best[2], best[3]));
                if (tid == 0) give(k, last);
            }
        }
    }
}

// The parts of a row's splits joined by one wave, lane s taking split s; its list of
// alternatives is sorted, so the next one is always the largest of the lists' heads.
template <typename T>
__global__ void __launch_bounds__(64) logprob_join_kernel(const T* __restrict__ z, int V, long ld,
                                                          const int* __restrict__ tokens, float scale, float lo, float hi,
                                                          RowOut out, int top, int splits,
                                                          const Part* __restrict__ parts, const u64* __restrict__ lists) {
    const long row = blockIdx.x;
    const int s = threadIdx.x;
    Part p = {NO_REF, 0.f, 0.f};
    if (s < splits) p = parts[row * splits + s];
    p = wave_join(p, scale * LOG2E);
    const RowLog log_p(p, scale);
    if (s == 0) write_row(out, row, p, log_p, z + row * ld, V, tokens, lo, hi);
    const u64* list = lists + (row * splits + s) * top;
    int at = 0;
    u64 head = s < splits && top > 0 ? list[0] : 0;
    for (int k = 0; k < top; ++k) {
        const u64 key = wave_max_key(head);
        if (s == 0) {
            out.top_ids[row * top + k] = key_index(key);
            out.top_logp[row * top + k] = log_p(key_value(key));
        }
        if (head == key && s < splits) head = ++at < top ? list[at] : 0;
    }
}

// The gradient: with d = s - lse, dz = -p (A + B d) + [v = t] scale a,
// A = scale (a + b H), B = scale b.  d is held above -200, where p is 0 and the product
// with it finite.
template <typename T, bool CLIP>
__global__ void __launch_bounds__(256) logprob_grad_kernel(const T* z, int V, long ld, const int* __restrict__ tokens,
                                                           float scale, float clip, const float* __restrict__ lse,
                                                           const float* __restrict__ entropy,
                                                           const float* __restrict__ dlogp,
                                                           const float* __restrict__ dentropy, T* dz, long ldd,
                                                           int splits, int per) {
    constexpr int N = Chunks<T>::N, U = 4;
    typedef typename Chunks<T>::vec vec;
    const long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits);
    const Chunks<T> ch(z + row * ld, V);
    const Chunks<T> to(dz + row * ldd, V);
    const int c0 = min(split * per, ch.count), c1 = min(c0 + per, ch.count);
    const float l = lse[row];
    float a = dlogp ? dlogp[row] : 0.f;
    const float b = dentropy ? dentropy[row] : 0.f, h = dentropy ? entropy[row] : 0.f;
    int t = dlogp ? tokens[row] : GP_NO_TOKEN;
    bool flat = l == -INFINITY;  // the whole row is `fill`
    float fill = 0.f;
    if (t == GP_NO_TOKEN) {
        a = 0.f;
    } else if (t < 0 || t >= V) {
        flat = true;
        fill = NAN;
    }
    const float A = scale * (a + b * h), B = scale * b, at = scale * a;
    auto grads = [&](const float (&x)[N], int j, float (&g)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float s = CLIP ? min_nan(max_nan(x[e], -clip), clip) : x[e];
            const float d = max_nan(__builtin_fmaf(s, scale, -l), -200.f);
            g[e] = -__builtin_amdgcn_exp2f(d * LOG2E) * __builtin_fmaf(B, d, A);
        }
        const int k = t - ch.first(j);
        if (t >= 0 && k >= 0 && k < N) {
#pragma unroll
            for (int e = 0; e < N; ++e) g[e] += e == k ? at : 0.f;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (CLIP) g[e] = fabsf(x[e]) > clip ? 0.f : g[e];
            if (flat) g[e] = fill;
        }
    };
    const bool same = ch.mis == to.mis;  // both rows lie alike on the 16-byte grid
    auto store = [&](int j, const float (&g)[N]) {
        if (same && ch.whole(j)) {
            vec o;
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = to_elt<T>(g[e]);
            reinterpret_cast<vec*>(dz + row * ldd - to.mis)[j] = o;
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int v = ch.first(j) + e;
                if (v >= 0 && v < V) dz[row * ldd + v] = to_elt<T>(g[e]);
            }
        }
    };
    for (int j = c0 + (int)threadIdx.x; j < c1; j += U * 256) {
        vec v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j + u * 256 < c1 && ch.whole(j + u * 256)) v[u] = ch.load(j + u * 256);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = j + u * 256;
            if (k >= c1) break;
            float x[N], g[N];
            if (ch.whole(k)) {
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = to_f32((T)v[u][e]);
            } else {
                ch.values(k, 0.f, x);
            }
            grads(x, k, g);
            store(k, g);
        }
    }
}

// Workgroups of a row: as many as give 1024 in all (four per CU) while each thread
// still has two chunks or more.
int row_splits(int dtype, long rows, int vocab) {
    const long chunks = vocab / (dtype == GP_BF16 ? 8 : 4);
    const long s = std::min(rows > 0 ? 1024 / rows : 1, chunks / (2 * ROW_THREADS));
    return (int)std::max(1L, std::min<long>(s, SPLIT_MAX));
}
size_t split_bytes(long rows, int splits, int top) { return (size_t)rows * splits * (sizeof(Part) + 8 * (size_t)top); }

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

gp_status check_rows(int dtype, const void* logits, long rows, int vocab, long ld, float scale, float clip) {
    auto bad = [](const char* m) { return set_error(GP_ERR_INVALID_ARG, m); };
    if (dtype != GP_F32 && dtype != GP_BF16) return bad("token_logprobs: unknown dtype");
    if (rows < 0 || rows > 0x7FFFFFFFL) return bad("token_logprobs: rows must be in [0, 2^31 - 1]");
    if (vocab < 1 || ld < vocab) return bad("token_logprobs: vocab must be >= 1 and ld >= vocab");
    if (!(scale >= 1e-6f && scale <= 1e6f)) return bad("token_logprobs: scale must be in [1e-6, 1e6]");
    if (!(clip >= 0.f) || !std::isfinite(clip)) return bad("token_logprobs: clip must be >= 0 and finite");
    if (!logits && rows > 0) return bad("token_logprobs: logits must not be NULL");
    if (!aligned(logits, dtype == GP_BF16 ? 2 : 4)) return bad("token_logprobs: logits not aligned to their elements");
    return GP_OK;
}

template <typename T>
gp_status launch_rows(const T* z, long rows, int V, long ld, const int* tokens, float scale, float clip,
                      const RowOut& out, int top, void* ws, size_t ws_bytes, hipStream_t st) {
    const int dtype = sizeof(T) == 2 ? GP_BF16 : GP_F32, N = 16 / sizeof(T);
    int splits = row_splits(dtype, rows, V);
    if (splits > 1) {
        const size_t fit = ws ? ws_bytes / split_bytes(rows, 1, top) : 0;
        splits = (int)std::min<size_t>(splits, std::max<size_t>(fit, 1));
    }
    const int chunks = (V + 2 * (N - 1)) / N;  // of the worst alignment
    const int per = (chunks + splits - 1) / splits;
    u64* lists = static_cast<u64*>(ws);
    Part* parts = reinterpret_cast<Part*>(lists + (splits > 1 ? (size_t)rows * splits * top : 0));
    const unsigned grid = (unsigned)(rows * splits);
    const bool clipped = clip > 0.f;
#define GP_ROWS(CLIP, TOP) \
    klaunch(logprob_kernel<T, CLIP, TOP>, grid, ROW_THREADS, 0, st, z, V, ld, tokens, scale, clip, out, top, splits, per, \
            parts, lists)
    if (clipped && top) GP_ROWS(true, true);
    else if (clipped) GP_ROWS(true, false);
    else if (top) GP_ROWS(false, true);
    else GP_ROWS(false, false);
#undef GP_ROWS
    if (splits > 1)
        klaunch(logprob_join_kernel<T>, (unsigned)rows, 64, 0, st, z, V, ld, tokens, scale, clipped ? -clip : NEVER,
                clipped ? clip : INFINITY, out, top, splits, parts, lists);
    GP_LAUNCH_CHECK();
    return GP_OK;
}

template <typename T>
gp_status launch_grad(const T* z, long rows, int V, long ld, const int* tokens, float scale, float clip, const float* lse,
                      const float* entropy, const float* dlogp, const float* dentropy, T* dz, long ldd, hipStream_t st) {
    const int N = 16 / sizeof(T), chunks = (V + 2 * (N - 1)) / N;
    // 4096 workgroups in all where the rows have that much to split
    const long want = std::max(1L, std::min<long>((4096 + rows - 1) / rows, chunks / 512));
    const int splits = (int)want, per = (chunks + splits - 1) / splits;
    const unsigned grid = (unsigned)(rows * splits);
    if (clip > 0.f)
        klaunch(logprob_grad_kernel<T, true>, grid, 256, 0, st, z, V, ld, tokens, scale, clip, lse, entropy, dlogp,
                dentropy, dz, ldd, splits, per);
    else
        klaunch(logprob_grad_kernel<T, false>, grid, 256, 0, st, z, V, ld, tokens, scale, clip, lse, entropy, dlogp,
                dentropy, dz, ldd, splits, per);
    GP_LAUNCH_CHECK();
    return GP_OK;
}

} // namespace

} // namespace gp

using namespace gp;

extern "C" {

gp_status gp_token_logprobs_workspace(int dtype, long rows, int vocab, int top, size_t* bytes) {
    if (!bytes || (dtype != GP_F32 && dtype != GP_BF16) || rows < 0 || vocab < 1 || top < 0 || top > GP_TOP_MAX)
        return set_error(GP_ERR_INVALID_ARG, "token_logprobs_workspace: an argument is out of range");
    const int splits = row_splits(dtype, rows, vocab);
    *bytes = splits > 1 ? split_bytes(rows, splits, top) : 0;
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
    const RowOut out = {logp, lse, entropy, top_ids, top_logp};
    if (dtype == GP_BF16)
        return launch_rows(static_cast<const bf16*>(logits), rows, vocab, ld, tokens, scale, clip, out, top, ws, ws_bytes,
                           (hipStream_t)stream);
    return launch_rows(static_cast<const float*>(logits), rows, vocab, ld, tokens, scale, clip, out, top, ws, ws_bytes,
                       (hipStream_t)stream);
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
    if (dtype == GP_BF16)
        return launch_grad(static_cast<const bf16*>(logits), rows, vocab, ld, tokens, scale, clip, lse, entropy, dlogp,
                           dentropy, static_cast<bf16*>(dlogits), ldd, (hipStream_t)stream);
    return launch_grad(static_cast<const float*>(logits), rows, vocab, ld, tokens, scale, clip, lse, entropy, dlogp,
                       dentropy, static_cast<float*>(dlogits), ldd, (hipStream_t)stream);
}

} // extern "C"
