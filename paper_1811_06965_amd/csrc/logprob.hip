// logprob.hip -- log probabilities of given tokens under rows of logits, the
// rows' entropy and most likely tokens, and the gradient of the first two.
#include <algorithm>
#include <cmath>

#include "common.hpp"
#include "logits.hpp"

namespace gp {

namespace {

// Sums of a row's terms around a reference logit r: with d = x - r, a = sum exp(scale d)
// and b = sum d exp(scale d).  Then lse = scale r + log a and the entropy is
// log a - scale b / a, whatever r is; its term stays within 2^8 of the largest.
// d is finite for every x that is (the reference is subtracted before scaling),
// so a term that vanishes adds no 0 inf.
struct Part {
    float r, a, b;
    // The same sums around another reference.  c2 = scale log2 e; f comes before the
    // product with d, which alone could pass the largest float.
    __device__ __forceinline__ Part around(float to, float c2) const {
        const float d = r - to, f = __builtin_amdgcn_exp2f(d * c2), fa = a * f;
        return {to, fa, __builtin_fmaf(fa, d, f * b)};
    }
};
// The parts of 64 lanes as one.
__device__ __forceinline__ Part wave_join(Part p, float c2) {
    const float r = wave_reduce_f(p.r, NO_REF, [](float a, float b) { return max_nan(a, b); });
    p = p.around(r, c2);
    auto add = [](float a, float b) { return a + b; };
    return {r, wave_reduce_f(p.a, 0.f, add), wave_reduce_f(p.b, 0.f, add)};
}

// The order of alternatives as integers: the code of a logit (larger first, a NaN
// before all, both zeros equal), and in the low half of a key its index, lower first.
// No code is 0, no key 0 or ~0.
typedef unsigned long long u64;
constexpr unsigned NAN_CODE = 0xFFFFFFFEu;
__device__ __forceinline__ unsigned code_of(float x) {
    const unsigned u = __float_as_uint(x + 0.f);
    return x != x ? NAN_CODE : (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ u64 key_of(unsigned code, int v) { return ((u64)code << 32) | (0xFFFFFFFFu - (unsigned)v); }
__device__ __forceinline__ float key_value(u64 k) {
    const unsigned u = (unsigned)(k >> 32);
    if (u == NAN_CODE) return NAN;
    return __uint_as_float((u >> 31) ? u & 0x7FFFFFFFu : ~u);
}
__device__ __forceinline__ int key_index(u64 k) { return (int)(0xFFFFFFFFu - (unsigned)k); }
__device__ __forceinline__ u64 wave_max_key(u64 k) {
    const unsigned hi = wave_max_u((unsigned)(k >> 32));
    const unsigned lo = wave_max_u((unsigned)(k >> 32) == hi ? (unsigned)k : 0u);
    return ((u64)hi << 32) | lo;
}

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

// Alternatives of one workgroup's part of a row.  Its threads make GROUPS groups of
// neighbours.  A bound that the largest logits of at least `top` groups reach is
// reached by at least `top` logits, and only by logits of the groups whose largest
// does: those groups' chunks are read a second time and what reaches the bound, a few
// more than `top` logits, is ranked.  One wave finds the bound bit by bit from the
// groups' largest, until a quarter more than `top` reach it.  Where more than
// OWNERS groups do, equal at the last bit, the logits above it come from
// the groups that have any, and those at it from the row's start on, until there are
// enough.  A row with a NaN, or with more than CAND logits that reach the bound, goes
// through its logits once per alternative instead.
constexpr int OWNERS = 48;
template <int NT> struct TopShared {
    static constexpr int GROUPS = NT < 256 ? NT : 256, CAND = 4 * GROUPS, TIE_CHUNKS = GROUPS / 2;
    unsigned most[GROUPS];
    u64 best[NT / WAVE];
    u64 cand[CAND + TIE_CHUNKS * 8];  // ties come in where fewer than `top` are listed
    int owner[GROUPS];
    int owners, found;
    unsigned bound;
};
template <typename T, int NT, typename Bounded, typename Give>
__device__ __forceinline__ void find_top(TopShared<NT>& sh, const T* zr, int V, int c0, int c1, int top, bool has_nan,
                                         Bounded bounded, Give give) {
    typedef Chunks<T> C;
    typedef TopShared<NT> S;
    constexpr int N = C::N, G = NT / S::GROUPS, PER = S::GROUPS / WAVE, ROOM = S::CAND + S::TIE_CHUNKS * 8;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    auto take = [&](int j, auto wanted) {  // lists a chunk's logits whose code is wanted
        float x[N];
        C::values(zr, V, j, 0.f, x);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const unsigned code = code_of(bounded(x[e]));
            if (j * N + e < V && wanted(code)) {
                const int at = atomicAdd(&sh.found, 1);
                if (at < ROOM) sh.cand[at] = key_of(code, j * N + e);
            }
        }
    };
    bool slow = has_nan;
    if (!slow) {
        if (w == 0) {
            unsigned m[PER], bound = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) m[i] = sh.most[lane + WAVE * i];
            auto reach = [&](unsigned t) {
                int c = 0;
#pragma unroll
                for (int i = 0; i < PER; ++i) c += __popcll(__ballot(m[i] >= t));
                return c;
            };
            int n = reach(1);
            if (n < top) {
                bound = 1;  // fewer groups hold a logit: all that do
            } else {
                for (int bit = 31; bit >= 0 && (bound == 0 || n > top + top / 4 + 2); --bit) {
                    const int c = reach(bound | (1u << bit));
                    if (c >= top) {
                        bound |= 1u << bit;
                        n = c;
                    }
                }
            }
            const unsigned least = n > OWNERS && n >= top ? bound + 1 : bound;  // ties: the groups above the bound
            int base = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const u64 mask = __ballot(m[i] >= least);
                if (m[i] >= least) sh.owner[base + __popcll(mask & ((1ull << lane) - 1))] = lane + WAVE * i;
                base += __popcll(mask);
            }
            if (lane == 0) {
                sh.owners = base;
                sh.bound = least;
                sh.found = 0;
            }
        }
        __syncthreads();
        const unsigned least = sh.bound;
        const int rounds = (c1 - c0 + NT - 1) / NT, each = sh.owners * G;
        for (int i = tid; i < each * rounds; i += NT) {
            const int o = i % each, j = c0 + sh.owner[o / G] * G + o % G + i / each * NT;
            if (j < c1) take(j, [&](unsigned code) { return code >= least; });
        }
        __syncthreads();
        int n = sh.found;
        slow = n > S::CAND;
        // too few: the rest equal the bound below
        for (int j0 = c0, step = S::TIE_CHUNKS / 4; !slow && n < top && least > 1 && j0 < c1;
             j0 += step, step = S::TIE_CHUNKS) {
            __syncthreads();
            if (tid < step)
                for (int i = tid; i < step; i += NT)
                    if (j0 + i < c1) take(j0 + i, [&](unsigned code) { return code == least - 1; });
            __syncthreads();
            n = sh.found;
        }
        if (!slow) {
            for (int i = tid; i < n; i += NT) {
                const u64 key = sh.cand[i];
                int r = 0;
                for (int k = 0; k < n; ++k) r += sh.cand[k] > key ? 1 : 0;
                if (r < top) give(r, key);
            }
            for (int k = n + tid; k < top; k += NT) give(k, 0);  // a part of fewer logits
        }
    }
    if (slow) {
        u64 last = ~0ull;
        for (int k = 0; k < top; ++k) {
            u64 mine = 0;
            for (int j = c0 + tid; j < c1; j += NT) {
                float x[N];
                C::values(zr, V, j, 0.f, x);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const u64 key = j * N + e < V ? key_of(code_of(bounded(x[e])), j * N + e) : 0;
                    if (key < last && key > mine) mine = key;
                }
            }
            mine = wave_max_key(mine);
            __syncthreads();
            if (lane == 0) sh.best[w] = mine;
            __syncthreads();
            last = wave_max_key(lane < NT / WAVE ? sh.best[lane] : 0);
            if (tid == 0) give(k, last);
        }
    }
}

// A workgroup of NT threads per row, or `splits` of them, each over `per` chunks of it;
// thread t takes the chunks t, t + NT, .., four loads ahead of their use (eight made
// long rows 3% slower).  Bound by HBM where rows are many: 1024 rows of 32000 bf16
// 14.0 us (4.7 TB/s, the launch included), 4096 of 32000 fp32 91 us (5.8 TB/s) and 95 with 8
// alternatives, 4096 of 128000 bf16 with 8 191 us (5.5 TB/s), close to what its 11 vector
// instructions a logit take; for few rows by the chain of reductions: one row of 32000 4.4 us, with
// 5 alternatives 7.3.
template <typename T, bool CLIP, bool TOP, int NT>
__global__ void __launch_bounds__(NT) logprob_kernel(const T* __restrict__ z, int V, long ld,
                                                     const int* __restrict__ tokens, float scale, float clip, RowOut out,
                                                     int top, int splits, int per, Part* __restrict__ parts,
                                                     u64* __restrict__ lists) {
    typedef Chunks<T> C;
    constexpr int N = C::N, U = 4, NW = NT / WAVE;
    __shared__ Part red[NW];
    const long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits);
    const T* zr = z + row * ld;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int chunks = V / N + (V % N ? 1 : 0), c0 = min(split * per, chunks), c1 = min(c0 + per, chunks);
    const float c2 = scale * LOG2E, near = 8.f / c2, lo = CLIP ? lower_bound(clip) : NEVER, hi = CLIP ? clip : INFINITY;
    auto bounded = [&](float x) { return CLIP ? min_nan(max_nan(x, lo), hi) : max_nan(x, lo); };

    Part p = {NO_REF, 0.f, 0.f};
    float most = -INFINITY;  // this thread's largest logit
    auto add = [&](const float (&x)[N]) {
        float cm = x[0];
#pragma unroll
        for (int e = 1; e < N; ++e) cm = max_nan(cm, x[e]);
        if (!(cm <= p.r + near)) p = p.around(cm, c2);  // NaN too
        if (TOP) most = max_nan(most, cm);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float d = x[e] - p.r, q = __builtin_amdgcn_exp2f(d * c2);
            p.a += q;
            p.b = __builtin_fmaf(q, d, p.b);
        }
    };
    const int f1 = min(c1, V / N);  // whole chunks
    for (int j = c0 + tid; j < f1; j += U * NT) {
        typename C::vec v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j + u * NT < f1) v[u] = C::load(zr, j + u * NT);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j + u * NT >= f1) break;
            float x[N];
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = bounded(to_f32((T)v[u][e]));
            add(x);
        }
    }
    if (f1 < c1 && tid == (f1 - c0) % NT) {  // the short last chunk: a mask behind its end adds nothing
        float x[N];
        C::values(zr, V, f1, 0.f, x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = f1 * N + e < V ? bounded(x[e]) : NEVER;
        add(x);
    }

    p = wave_join(p, c2);
    if (lane == 0) red[w] = p;
    auto sums = [&] { return wave_join(lane < NW ? red[lane] : Part{NO_REF, 0.f, 0.f}, c2); };
    auto write = [&](const RowLog& log_p) {
        if (tid != 0) return;
        if (splits > 1)
            parts[blockIdx.x] = p;
        else
            write_row(out, row, p, log_p, zr, V, tokens, lo, hi);
    };
    if constexpr (TOP) {
        __shared__ TopShared<NT> sh;
        unsigned m = most == -INFINITY ? 0u : code_of(most);  // 0: no logit
        constexpr int G = NT / TopShared<NT>::GROUPS;
#pragma unroll
        for (int o = 1; o < G; o *= 2) m = max(m, __shfl_xor(m, o, WAVE));
        if (tid % G == 0) sh.most[tid / G] = m;
        __syncthreads();
        p = sums();
        const RowLog log_p(p, scale);
        write(log_p);
        find_top<T, NT>(sh, zr, V, c0, c1, top, p.a != p.a, bounded, [&](int k, u64 key) {
            if (splits > 1) {
                lists[(long)blockIdx.x * top + k] = key;
            } else {
                out.top_ids[row * top + k] = key_index(key);
                out.top_logp[row * top + k] = log_p(key_value(key));
            }
        });
    } else {
        __syncthreads();
        p = sums();
        write(RowLog(p, scale));
    }
}

// The parts of a row's splits joined by one wave, lane s taking split s; its list of
// alternatives is sorted, so the next one is always the largest of the lists' heads.
// 2 us, and 0.15 us per alternative.
template <typename T>
__global__ void __launch_bounds__(64) logprob_join_kernel(const T* __restrict__ z, int V, long ld,
                                                          const int* __restrict__ tokens, float scale, float lo, float hi,
                                                          RowOut out, int top, int splits,
                                                          const Part* __restrict__ parts, const u64* __restrict__ lists) {
    __shared__ u64 list[SPLIT_MAX * GP_TOP_MAX];
    const long row = blockIdx.x;
    const int s = threadIdx.x;
    for (int i = s; i < splits * top; i += WAVE) list[i] = lists[row * splits * top + i];
    Part p = {NO_REF, 0.f, 0.f};
    if (s < splits) p = parts[row * splits + s];
    p = wave_join(p, scale * LOG2E);
    const RowLog log_p(p, scale);
    if (s == 0) write_row(out, row, p, log_p, z + row * ld, V, tokens, lo, hi);
    __syncthreads();
    int at = 0;
    u64 head = s < splits && top > 0 ? list[s * top] : 0;
    for (int k = 0; k < top; ++k) {
        const u64 key = wave_max_key(head);
        if (s == 0) {
            out.top_ids[row * top + k] = key_index(key);
            out.top_logp[row * top + k] = log_p(key_value(key));
        }
        if (head == key && s < splits) head = ++at < top ? list[s * top + at] : 0;
    }
}

// The gradient: with d = s - lse, dz = -p (A + B d) + [v = t] scale a,
// A = scale (a + b H), B = scale b.  d is held above -200, where p is 0 and the product
// with it finite.  Rows are split until there are 4096 workgroups or 512 chunks in each.  Bound by
// HBM: 1024 rows of 32000 bf16 24 us (131 MB, 5.45 TB/s), 93 rows of 50021 fp32 between
// strides of 50048 and 50021 7.7 us (4.8 TB/s).
template <typename T, bool CLIP>
__global__ void __launch_bounds__(256) logprob_grad_kernel(const T* z, int V, long ld, const int* __restrict__ tokens,
                                                           float scale, float clip, const float* __restrict__ lse,
                                                           const float* __restrict__ entropy,
                                                           const float* __restrict__ dlogp,
                                                           const float* __restrict__ dentropy, T* dz, long ldd,
                                                           int splits, int per) {
    typedef Chunks<T> C;
    constexpr int N = C::N, U = 4;
    typedef typename C::vec vec;
    const long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits);
    const T* zr = z + row * ld;
    T* dr = dz + row * ldd;
    const int chunks = V / N + (V % N ? 1 : 0), c0 = min(split * per, chunks), c1 = min(c0 + per, chunks);
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
        const int k = t - j * N;
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
    const int f1 = min(c1, V / N);  // whole chunks
    for (int j = c0 + (int)threadIdx.x; j < f1; j += U * 256) {
        vec v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j + u * 256 < f1) v[u] = C::load(zr, j + u * 256);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j + u * 256 >= f1) break;
            float x[N], g[N];
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = to_f32((T)v[u][e]);
            grads(x, j + u * 256, g);
            vec o;
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = to_elt<T>(g[e]);
            *reinterpret_cast<vec*>(dr + (long)(j + u * 256) * N) = o;
        }
    }
    if (f1 < c1 && (int)threadIdx.x == (f1 - c0) % 256) {  // the short last chunk
        float x[N], g[N];
        C::values(zr, V, f1, 0.f, x);
        grads(x, f1, g);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (f1 * N + e < V) dr[(long)f1 * N + e] = to_elt<T>(g[e]);
    }
}

// Threads of a workgroup.  Short rows take one wave, whose joins and rankings wait for
// nobody; few rows, or rows over 128 KB, the most loads in flight, from 32 KB a row on where
// a CU has one row at most, else from 50 KB on; in between many rows
// share a CU, and alternatives are ranked faster by more threads.  us at 64 / 256 / 512 / 1024
// threads: 4096 x 1000 bf16 with 5 alternatives 8.6 / 15.1 / 24.7 / 42.6; 3000 x 4111
// with 1 12.4 / 15.3 / 23.3 / 36.3; 512 x 9000 fp32 with 20 18.0 / 7.8 / 8.1 / 9.3; 93 x
// 50021 fp32 with 20 69 / 15.7 / 11.7 / 10.6; 1024 x 32000 bf16 20.2 / 14.4 / 14.5 / 15.7,
// with 20 46 / 20.0 / 19.1 / 23.0; 4096 x 128000 with 8 319 / 216 / 191 / 193.  At 256 / 1024
// threads, bf16 with 20: 256 x 14000 8.0 / 8.1, 256 x 21000 9.3 / 8.5; 512 x 24000 11.4 / 11.8,
// 512 x 27000 12.6 / 12.2.
int row_threads(long rows, int chunks, int splits, int top) {
    if (chunks <= 256 || (chunks <= 1024 && rows >= 1024)) return 64;
    if (splits > 1 || chunks <= (rows <= 256 ? 2048 : 3200)) return 256;
    if (rows < 768 || chunks > 8192) return 1024;
    return top ? 512 : 256;
}
size_t split_bytes(long rows, int splits, int top) { return (size_t)rows * splits * (sizeof(Part) + 8 * (size_t)top); }

gp_status check_rows(int dtype, const void* logits, long rows, int vocab, long ld, float scale, float clip) {
    auto bad = [](const char* m) { return set_error(GP_ERR_INVALID_ARG, m); };
    if (dtype != GP_F32 && dtype != GP_BF16) return bad("token_logprobs: unknown dtype");
    if (rows < 0 || rows > 0x7FFFFFFFL) return bad("token_logprobs: rows must be in [0, 2^31 - 1]");
    if (vocab < 1 || vocab > (1 << 30) || ld < vocab)
        return bad("token_logprobs: vocab must be in [1, 2^30] and ld >= vocab");
    if (!(scale >= 1e-6f && scale <= 1e6f)) return bad("token_logprobs: scale must be in [1e-6, 1e6]");
    if (!(clip >= 0.f) || !std::isfinite(clip)) return bad("token_logprobs: clip must be >= 0 and finite");
    if (!logits && rows > 0) return bad("token_logprobs: logits must not be NULL");
    if (!aligned(logits, dtype == GP_BF16 ? 2 : 4)) return bad("token_logprobs: logits not aligned to their elements");
    return GP_OK;
}

template <typename T>
gp_status launch_rows(const T* z, long rows, int V, long ld, const int* tokens, float scale, float clip,
                      const RowOut& out, int top, void* ws, size_t ws_bytes, hipStream_t st) {
    const int dtype = sizeof(T) == 2 ? GP_BF16 : GP_F32;
    int splits = row_splits(dtype, rows, V);
    if (splits > 1) {
        const size_t fit = ws ? ws_bytes / split_bytes(rows, 1, top) : 0;
        splits = (int)std::min<size_t>(splits, std::max<size_t>(fit, 1));
    }
    const int chunks = chunk_count(dtype, V), per = (chunks + splits - 1) / splits;
    u64* lists = static_cast<u64*>(ws);
    Part* parts = reinterpret_cast<Part*>(lists + (splits > 1 ? (size_t)rows * splits * top : 0));
    const unsigned grid = (unsigned)(rows * splits);
    const bool clipped = clip > 0.f;
    const int nt = row_threads(rows, chunks, splits, top);
#define GP_ROWS_NT(CLIP, TOP, NT) \
    klaunch(logprob_kernel<T, CLIP, TOP, NT>, grid, NT, 0, st, z, V, ld, tokens, scale, clip, out, top, splits, per, parts, \
            lists)
#define GP_ROWS(CLIP, TOP)                      \
    do {                                        \
        if (nt == 64)                           \
            GP_ROWS_NT(CLIP, TOP, 64);          \
        else if (nt == 256)                     \
            GP_ROWS_NT(CLIP, TOP, 256);         \
        else if (nt == 512 && TOP)              \
            GP_ROWS_NT(CLIP, TOP, (TOP ? 512 : 64)); \
        else                                    \
            GP_ROWS_NT(CLIP, TOP, 1024);        \
    } while (0)
    if (clipped && top)
        GP_ROWS(true, true);
    else if (clipped)
        GP_ROWS(true, false);
    else if (top)
        GP_ROWS(false, true);
    else
        GP_ROWS(false, false);
#undef GP_ROWS
#undef GP_ROWS_NT
    if (splits > 1)
        klaunch(logprob_join_kernel<T>, (unsigned)rows, 64, 0, st, z, V, ld, tokens, scale,
                clipped ? lower_bound(clip) : NEVER, clipped ? clip : INFINITY, out, top, splits, parts, lists);
    GP_LAUNCH_CHECK();
    return GP_OK;
}

template <typename T>
gp_status launch_grad(const T* z, long rows, int V, long ld, const int* tokens, float scale, float clip, const float* lse,
                      const float* entropy, const float* dlogp, const float* dentropy, T* dz, long ldd, hipStream_t st) {
    const int chunks = chunk_count(sizeof(T) == 2 ? GP_BF16 : GP_F32, V);
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
    if (!bytes || (dtype != GP_F32 && dtype != GP_BF16) || rows < 0 || vocab < 1 || vocab > (1 << 30) || top < 0 || top > GP_TOP_MAX)
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
    for (long r = 0; r < rows; r += LAUNCH_ROWS) {
        const long n = std::min(LAUNCH_ROWS, rows - r);
        const RowOut out = {past(logp, r), past(lse, r), past(entropy, r), past(top_ids, r * top), past(top_logp, r * top)};
        const int* t = past(tokens, r);
        if (dtype == GP_BF16)
            GP_TRY(launch_rows(static_cast<const bf16*>(logits) + r * ld, n, vocab, ld, t, scale, clip, out, top, ws,
                               ws_bytes, (hipStream_t)stream));
        else
            GP_TRY(launch_rows(static_cast<const float*>(logits) + r * ld, n, vocab, ld, t, scale, clip, out, top, ws,
                               ws_bytes, (hipStream_t)stream));
    }
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
    const bool same = z0 == d0 && (ld == ldd || rows == 1);
    if (!same && z0 < d1 && d0 < z1 && !side_by_side(z0, d0, (size_t)vocab * es, ld == ldd ? (size_t)ld * es : 0))
        return bad("token_logprobs_backward: dlogits overlaps the logits without being them");
    for (long r = 0; r < rows; r += LAUNCH_ROWS) {
        const long n = std::min(LAUNCH_ROWS, rows - r);
        const int* t = past(tokens, r);
        const float *h = past(entropy, r), *a = past(dlogp, r), *b = past(dentropy, r);
        if (dtype == GP_BF16)
            GP_TRY(launch_grad(static_cast<const bf16*>(logits) + r * ld, n, vocab, ld, t, scale, clip, lse + r, h, a, b,
                               static_cast<bf16*>(dlogits) + r * ldd, ldd, (hipStream_t)stream));
        else
            GP_TRY(launch_grad(static_cast<const float*>(logits) + r * ld, n, vocab, ld, t, scale, clip, lse + r, h, a, b,
                               static_cast<float*>(dlogits) + r * ldd, ldd, (hipStream_t)stream));
    }
    return GP_OK;
}

} // extern "C"
