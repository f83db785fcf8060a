// distill.hip -- the divergence of rows of logits from a teacher that is known
// by its most likely tokens, and its gradient.
#include <algorithm>
#include <cmath>

#include "common.hpp"
#include "logits.hpp"

namespace gp {

namespace {

constexpr float LN2 = 0.693147180559945309f;

// Sums of a row's terms around a reference logit r: a = sum exp(scale (x - r)); lse = scale r + log a.
struct Sum {
    float r, a;
    __device__ __forceinline__ Sum around(float to, float c2) const { return {to, a * __builtin_amdgcn_exp2f((r - to) * c2)}; }
    __device__ __forceinline__ bool empty() const { return r <= NEVER && a == a; }  // masks alone
};
__device__ __forceinline__ Sum wave_join(Sum p, float c2) {
    const float r = wave_reduce_f(p.r, NO_REF, [](float a, float b) { return max_nan(a, b); });
    p = p.around(r, c2);
    return {r, wave_reduce_f(p.a, 0.f, [](float a, float b) { return a + b; })};
}

// A row's tokens in LDS.
typedef int i32x4 __attribute__((ext_vector_type(4)));
struct Named {
    alignas(16) int id[GP_DISTILL_MAX];        // negative: none, or not a token; so are those behind the last, in fours
    alignas(16) float teacher[GP_DISTILL_MAX];
    alignas(16) float x[GP_DISTILL_MAX];       // the student's logit, bounded
    float first[GP_DISTILL_MAX];               // the same where the token is named for the first time, else a mask
    int wrong;                                 // an id that is not a token
};
struct Logits {
    int V;
    long ld;
    const int* ids;
    const float* teacher;
    int top;
    float scale, clip;
};

// Loads a row's tokens; a barrier must follow, then find_first (whose results need another).
template <typename T, bool CLIP>
__device__ __forceinline__ void load_named(Named& s, const T* zr, const Logits& a, long row, int tid, int threads) {
    if (tid == 0) s.wrong = 0;
    const float lo = CLIP ? lower_bound(a.clip) : NEVER, hi = CLIP ? a.clip : INFINITY;
    for (int j = tid; j < (a.top + 3) / 4 * 4; j += threads) {
        if (j >= a.top) {
            s.id[j] = GP_NO_TOKEN;
            continue;
        }
        const int id = a.ids[row * a.top + j];
        const bool is = id >= 0 && id < a.V;
        s.id[j] = is ? id : id == GP_NO_TOKEN ? GP_NO_TOKEN : GP_NO_TOKEN - 1;
        s.teacher[j] = a.teacher[row * a.top + j];
        if (is) s.x[j] = min_nan(max_nan(to_f32(zr[id]), lo), hi);
    }
}
template <bool REST> __device__ __forceinline__ void find_first(Named& s, int top, int tid, int threads) {
    for (int j = tid; j < top; j += threads) {
        const int id = s.id[j];
        if (id < GP_NO_TOKEN) s.wrong = 1;
        if (!REST || id < 0) continue;
        bool again = false;
#pragma unroll 4
        for (int k = 0; k < j; k += 4) {  // four at a time: one by one this took longer than the logits of a row
            const i32x4 v = *reinterpret_cast<const i32x4*>(s.id + k);
#pragma unroll
            for (int e = 0; e < 4; ++e) again = again || (v[e] == id && k + e < j);
        }
        s.first[j] = again ? NEVER : s.x[j];
    }
}

// The teacher's weights of a row, by one wave: with `rest` q = exp(t) as they are and what they leave of 1, else q
// normalised over the named tokens.
struct Teacher {
    float shift;  // log q = t - shift
    float total;  // sum of q, and of what is left
    float left;
    bool any;
    __device__ __forceinline__ Teacher(const Named& s, int top, bool rest, int lane) : shift(0.f), total(0.f), left(0.f) {
        bool some = false;
        float m = -INFINITY;
        for (int j = lane; j < top; j += WAVE)
            if (s.id[j] >= 0) {
                some = true;
                m = max_nan(m, s.teacher[j]);
            }
        any = __any(some);
        m = wave_reduce_f(m, -INFINITY, [](float x, float y) { return max_nan(x, y); });
        const double from = rest || m == -INFINITY ? 0.0 : (double)m;
        double sum = 0.0;
        for (int j = lane; j < top; j += WAVE)
            if (s.id[j] >= 0) sum += exp((double)s.teacher[j] - from);
        sum = wave_sum_d(sum);
        if (rest) {
            left = any && sum < 1.0 ? (float)(1.0 - sum) : 0.f;
            total = sum < 1.0 ? 1.f : (float)sum;
        } else if (sum > 0.0 || sum != sum) {
            shift = (float)(from + log(sum));
            total = 1.f;
        }
    }
};

struct DistillOut {
    float* loss;
    float* lse;
    float* rest_lse;
};

// A row's results from the sum over what is not named (REST) or over everything, by one wave.
template <bool REST>
__device__ __forceinline__ void finish_row(const DistillOut& o, long row, Sum away, const Named& s, const Logits& a, int lane) {
    const float c2 = a.scale * LOG2E;
    Sum all = away;
    if (REST) {
        Sum p = {NO_REF, 0.f};
        for (int j = lane; j < a.top; j += WAVE)
            if (s.id[j] >= 0) p.r = max_nan(p.r, s.first[j]);
        if (lane == 0) p.r = max_nan(p.r, away.r);
        p.r = wave_reduce_f(p.r, NO_REF, [](float x, float y) { return max_nan(x, y); });
        for (int j = lane; j < a.top; j += WAVE)
            if (s.id[j] >= 0) p.a += __builtin_amdgcn_exp2f((s.first[j] - p.r) * c2);
        if (lane == 0) p.a += away.around(p.r, c2).a;
        all = {p.r, wave_reduce_f(p.a, 0.f, [](float x, float y) { return x + y; })};
    }
    const Teacher t(s, a.top, REST, lane);
    const float la = logf(all.a);
    float loss = 0.f;
    for (int j = lane; j < a.top; j += WAVE) {
        if (s.id[j] < 0) continue;
        const float logq = s.teacher[j] - t.shift, q = expf(logq);
        const float logp = all.empty() || s.x[j] <= NEVER ? -INFINITY : a.scale * (s.x[j] - all.r) - la;
        if (!(q == 0.f)) loss += q * (logq - logp);
    }
    loss = wave_reduce_f(loss, 0.f, [](float x, float y) { return x + y; });
    if (lane != 0) return;
    if (REST && t.left > 0.f && !away.empty()) loss += t.left * (logf(t.left) - (a.scale * (away.r - all.r) + logf(away.a) - la));
    o.loss[row] = s.wrong ? NAN : t.any ? loss : 0.f;
    o.lse[row] = all.empty() ? -INFINITY : a.scale * all.r + la;
    if (REST) o.rest_lse[row] = away.empty() ? -INFINITY : a.scale * away.r + logf(away.a);
}

// A workgroup of NT threads per row, or `splits` of them, each over `per` chunks of it; one pass over the logits
// with a running reference, four loads ahead of their use.  REST: the named tokens are left out of the sum, which
// alone keeps the rest's share exact where the student gives it little (the difference of the sums would not): a byte
// in LDS marks them in each chunk, WINDOW chunks at a time.  Bound by HBM where rows are many: 4096 of 128000 bf16 with 64 tokens
// 180 to 192 us (5.5 to 5.8 TB/s), else by a row's chain of tokens, marks, loads and reductions: 93 rows of 50021 fp32 with 100 tokens 13.
// The next loads before these sums, in more registers, made the long rows 7% slower.
constexpr int WINDOW = 16384;
template <typename T, bool CLIP, bool REST, int NT>
__global__ void __launch_bounds__(NT) distill_kernel(const T* __restrict__ z, Logits a, DistillOut out, int splits, int per,
                                                     Sum* __restrict__ parts) {
    typedef Chunks<T> C;
    constexpr int N = C::N, U = 4, NW = NT / WAVE;
    __shared__ Sum red[NW];
    __shared__ Named named;
    extern __shared__ __attribute__((aligned(16))) unsigned marks[];
    const long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits), V = a.V;
    const T* zr = z + row * a.ld;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int chunks = V / N + (V % N ? 1 : 0), c0 = min(split * per, chunks), c1 = min(c0 + per, chunks);
    const float c2 = a.scale * LOG2E, near = 8.f / c2, lo = CLIP ? lower_bound(a.clip) : NEVER, hi = CLIP ? a.clip : INFINITY;
    auto bounded = [&](float x) { return CLIP ? min_nan(max_nan(x, lo), hi) : max_nan(x, lo); };

    Sum p = {NO_REF, 0.f};
    auto add = [&](float (&x)[N], unsigned m) {
        if (REST && m) {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = (m >> e) & 1 ? NEVER : x[e];
        }
        float cm = x[0];
#pragma unroll
        for (int e = 1; e < N; ++e) cm = max_nan(cm, x[e]);
        if (!(cm <= p.r + near)) p = p.around(cm, c2);  // NaN too
#pragma unroll
        for (int e = 0; e < N; ++e) p.a += __builtin_amdgcn_exp2f((x[e] - p.r) * c2);
    };
    load_named<T, CLIP>(named, zr, a, row, tid, NT);
    __syncthreads();
    find_first<REST>(named, a.top, tid, NT);
    const unsigned char* mark = reinterpret_cast<const unsigned char*>(marks);
    for (int w0 = c0; w0 < c1; w0 += WINDOW) {
        const int w1 = min(w0 + WINDOW, c1), f1 = min(w1, V / N);  // f1: whole chunks
        if (REST) {
            __syncthreads();
            for (int i = tid; i < (w1 - w0 + 3) / 4; i += NT) marks[i] = 0;
            __syncthreads();
            for (int j = tid; j < a.top; j += NT) {
                const int id = named.id[j], c = id / N;
                if (id >= 0 && c >= w0 && c < w1) atomicOr(&marks[(c - w0) >> 2], 1u << (8 * ((c - w0) & 3) + id % N));
            }
            __syncthreads();
        }
        for (int j = w0 + tid; j < f1; j += U * NT) {
            typename C::vec v[U];
            unsigned m[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j + u * NT < f1) {
                    v[u] = C::load(zr, j + u * NT);
                    m[u] = REST ? mark[j + u * NT - w0] : 0;
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (j + u * NT >= f1) break;
                float x[N];
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = bounded(to_f32((T)v[u][e]));
                add(x, m[u]);
            }
        }
        if (f1 < w1 && tid == (f1 - w0) % NT) {  // the short last chunk: a mask behind its end adds nothing
            float x[N];
            C::values(zr, V, f1, 0.f, x);
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = f1 * N + e < V ? bounded(x[e]) : NEVER;
            add(x, REST ? mark[f1 - w0] : 0);
        }
    }
    p = wave_join(p, c2);
    if (lane == 0) red[w] = p;
    __syncthreads();
    if (w != 0) return;
    p = wave_join(lane < NW ? red[lane] : Sum{NO_REF, 0.f}, c2);
    if (splits == 1)
        finish_row<REST>(out, row, p, named, a, lane);
    else if (lane == 0)
        parts[blockIdx.x] = p;
}

// The parts of a row's splits joined, and its results, by one wave.
template <typename T, bool CLIP, bool REST>
__global__ void __launch_bounds__(64) distill_join_kernel(const T* __restrict__ z, Logits a, DistillOut out, int splits,
                                                          const Sum* __restrict__ parts) {
    __shared__ Named named;
    const long row = blockIdx.x;
    const int lane = threadIdx.x;
    load_named<T, CLIP>(named, z + row * a.ld, a, row, lane, WAVE);
    __syncthreads();
    find_first<REST>(named, a.top, lane, WAVE);
    __syncthreads();
    const Sum p = wave_join(lane < splits ? parts[row * splits + lane] : Sum{NO_REF, 0.f}, a.scale * LOG2E);
    finish_row<REST>(out, row, p, named, a, lane);
}

// The gradient: with W the sum of the teacher's weights (and of what they leave),
//   dz_v = dloss scale (W p_v - q_v) for a named token,
//   dz_v = dloss scale (W - left / R) p_v else, R = exp(rest_lse - lse): written as
//          (W R - left) exp(s - rest_lse), neither of whose factors passes 1 by much.
// One pass writes the second form everywhere, then the named tokens, each by the thread that holds it.  Bound by HBM: 1024 rows of
// 32000 bf16 28 us (131 MB, 4.6 TB/s).
struct DistillGrad {
    const float* lse;
    const float* rest_lse;
    const float* dloss;
    long ldd;
};
template <typename T, bool CLIP, bool REST>
__global__ void __launch_bounds__(256) distill_grad_kernel(const T* z, Logits a, DistillGrad g, T* dz, int splits, int per) {
    typedef Chunks<T> C;
    typedef typename C::vec vec;
    constexpr int N = C::N, U = 4, NT = 256;
    static_assert(GP_DISTILL_MAX <= NT, "a thread per named token");
    __shared__ Named named;
    __shared__ float base_coef[2];
    const long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits), tid = threadIdx.x, V = a.V;
    const T* zr = z + row * a.ld;
    T* dr = dz + row * g.ldd;
    const int chunks = V / N + (V % N ? 1 : 0), c0 = min(split * per, chunks), c1 = min(c0 + per, chunks);
    const float lse = g.lse[row], dloss = g.dloss[row] * a.scale;

    // the tokens; logits only of those that this workgroup writes (another may have written its own over them)
    if (tid == 0) named.wrong = 0;
    float mine = 0.f;
    bool owner = false;
    if (tid >= a.top && tid < (a.top + 3) / 4 * 4) named.id[tid] = GP_NO_TOKEN;
    if (tid < a.top) {
        const int id = a.ids[row * a.top + tid];
        const bool is = id >= 0 && id < V;
        named.id[tid] = is ? id : id == GP_NO_TOKEN ? GP_NO_TOKEN : GP_NO_TOKEN - 1;
        named.teacher[tid] = a.teacher[row * a.top + tid];
        owner = is && id / N >= c0 && id / N < c1;
        if (owner) mine = to_f32(zr[id]);
        named.x[tid] = mine;  // read before anything is written
    }
    __syncthreads();
    if (tid < a.top && named.id[tid] < GP_NO_TOKEN) named.wrong = 1;
    if (tid < WAVE) {
        const Teacher t(named, a.top, REST, tid);
        if (tid == 0) {
            float base = lse, coef = t.total;
            if (REST) {
                const float r = g.rest_lse[row];
                if (t.left > 0.f && r > -INFINITY) {
                    base = r;
                    coef = expf(r - lse) - t.left;
                } else {
                    coef = t.total - t.left;
                }
            }
            base_coef[0] = base;
            base_coef[1] = t.any ? coef : 0.f;
            named.first[0] = t.shift;
            named.first[1] = REST && !(t.left > 0.f && g.rest_lse[row] > -INFINITY) ? t.total - t.left : t.total;
            named.first[2] = t.any ? 1.f : 0.f;
        }
    }
    __syncthreads();
    if (tid < (a.top + 3) / 4 * 4) named.x[tid] = tid < a.top ? expf(named.teacher[tid] - named.first[0]) : 0.f;  // q
    const float base = base_coef[0], coef = base_coef[1] * dloss, total = named.first[1];
    const bool flat = named.wrong || lse == -INFINITY || named.first[2] == 0.f;  // the whole row is `fill`
    const float fill = named.wrong ? NAN : 0.f;
    auto bounded = [&](float x) { return CLIP ? min_nan(max_nan(x, -a.clip), a.clip) : x; };
    auto grads = [&](const float (&x)[N], float (&d)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            d[e] = coef * __builtin_amdgcn_exp2f(__builtin_fmaf(bounded(x[e]), a.scale, -base) * LOG2E);
            if (CLIP) d[e] = fabsf(x[e]) > a.clip ? 0.f : d[e];
            if (flat) d[e] = fill;
        }
    };
    const int f1 = min(c1, V / N);  // whole chunks
    for (int j = c0 + tid; j < f1; j += U * NT) {
        vec v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j + u * NT < f1) v[u] = C::load(zr, j + u * NT);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j + u * NT >= f1) break;
            float x[N], d[N];
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = to_f32((T)v[u][e]);
            grads(x, d);
            vec o;
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = to_elt<T>(d[e]);
            *reinterpret_cast<vec*>(dr + (long)(j + u * NT) * N) = o;
        }
    }
    if (f1 < c1 && tid == (f1 - c0) % NT) {  // the short last chunk
        float x[N], d[N];
        C::values(zr, V, f1, 0.f, x);
        grads(x, d);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (f1 * N + e < V) dr[(long)f1 * N + e] = to_elt<T>(d[e]);
    }
    if (flat) return;
    __syncthreads();
    if (owner) {
        float q = 0.f;  // a token that is named twice has both its weights
        const int id = named.id[tid];
#pragma unroll 4
        for (int k = 0; k < a.top; k += 4) {
            const i32x4 v = *reinterpret_cast<const i32x4*>(named.id + k);
            const f32x4 w = *reinterpret_cast<const f32x4*>(named.x + k);
#pragma unroll
            for (int e = 0; e < 4; ++e) q += v[e] == id ? w[e] : 0.f;
        }
        float d = dloss * (total * __builtin_amdgcn_exp2f(__builtin_fmaf(bounded(mine), a.scale, -lse) * LOG2E) - q);
        if (CLIP) d = fabsf(mine) > a.clip ? 0.f : d;
        dr[id] = to_elt<T>(d);
    }
}

// Threads of a workgroup: a wave for short rows, whose reductions wait for nobody; for few or long rows the most loads in
// flight.  us at 64 / 256 / 1024 threads, bf16 with 32 tokens unless noted: 4096 x 1000 with 8 8.8 / 11.9 / 34.6; 3000 x 4111 14.3 /
// 17.2 / 42.9; 1024 x 8000 12.0 / 10.1 / 15.3; 512 x 9000 fp32 with 20 12.7 / 8.4 / 8.5; 256 x 14000 13.5 / 8.6 / 8.0; 512 x
// 27000 21.9 / 12.3 / 11.6; 93 x 50021 fp32 with 100 44.3 / 17.7 / 13.2; 1024 x 32000 26.1 / 19.1 / 23.3.
int distill_threads(long rows, int chunks, int splits) {
    if (chunks <= 256 || (chunks <= 700 && rows >= 1024)) return 64;
    if (splits > 1 || chunks <= (rows <= 256 ? 2048 : 3200)) return 256;
    return rows < 768 || chunks > 8192 ? 1024 : 256;
}

// Rows are split, of those that row_splits would, where that saves more than it costs.  A chunk takes a whole row's workgroup 0.52 ns
// (bf16) or 0.30 (fp32), a split one's less by 0.002 ns for each row that shares the bandwidth; the join takes 2 us and 7 ns for
// each token, 40 with a rest and 0.18 for each pair of tokens, whose first places it finds again; and each workgroup reads the tokens
// anew, 0.2 ns for each of them and row.  us, whole / split, with 32 and 128 tokens and a rest, with 32 and 256 without:
//   bf16  1 x 131072 14.1 / 10.3, 18.1 / 19.7, 11.6 / 6.7, 12.9 / 9.5;  96 15.0 / 14.2, 18.8 / 25.2, 12.1 / 10.7, 13.5 / 17.8
//   96 x 262144 25.3 / 19.4, 29.2 / 29.6, 21.7 / 15.8, 23.4 / 22.1;  with 256 and a rest 1 x 262144 32.2 / 39.0, 1 x 524288 49.5 / 40.3
//   fp32  1 x 65536 10.5 / 10.2, 14.0 / 19.3, 7.9 / 6.5, 9.3 / 9.1;  64 11.0 / 11.8, 14.7 / 21.8, 8.5 / 8.2, 9.8 / 13.3
//   96 x 131072 18.4 / 18.1, 21.8 / 27.9, 14.6 / 14.2, 16.1 / 20.6;  96 x 262144 30.1 / 25.4, 33.3 / 34.7, 23.9 / 21.8
int distill_splits(int dtype, long rows, int vocab, int top, bool rest) {
    const int splits = row_splits(dtype, rows, vocab);
    const long saved = chunk_count(dtype, vocab) * ((dtype == GP_BF16 ? 520 : 300) - 2 * rows);  // ps
    return saved > 2000000 + ((rest ? 40000 + 180 * top : 7000) + 200 * rows) * top ? splits : 1;
}

template <typename T, bool CLIP, bool REST>
gp_status launch_rows(const T* z, long rows, const Logits& a, const DistillOut& out, void* ws, size_t ws_bytes, hipStream_t st) {
    const int dtype = sizeof(T) == 2 ? GP_BF16 : GP_F32;
    int splits = distill_splits(dtype, rows, a.V, a.top, REST);
    if (splits > 1) {
        const size_t fit = ws ? ws_bytes / (rows * sizeof(Sum)) : 0;
        splits = (int)std::min<size_t>(splits, std::max<size_t>(fit, 1));
    }
    const int chunks = chunk_count(dtype, a.V), per = (chunks + splits - 1) / splits;
    Sum* parts = static_cast<Sum*>(ws);
    const unsigned grid = (unsigned)(rows * splits);
    const uint32_t lds = REST ? (std::min(per, WINDOW) + 15) / 16 * 16 : 0;
    const int nt = distill_threads(rows, chunks, splits);
    if (nt == 64)
        klaunch(distill_kernel<T, CLIP, REST, 64>, grid, 64, lds, st, z, a, out, splits, per, parts);
    else if (nt == 256)
        klaunch(distill_kernel<T, CLIP, REST, 256>, grid, 256, lds, st, z, a, out, splits, per, parts);
    else
        klaunch(distill_kernel<T, CLIP, REST, 1024>, grid, 1024, lds, st, z, a, out, splits, per, parts);
    if (splits > 1) klaunch(distill_join_kernel<T, CLIP, REST>, (unsigned)rows, 64, 0, st, z, a, out, splits, parts);
    GP_LAUNCH_CHECK();
    return GP_OK;
}
template <typename T, bool CLIP, bool REST>
gp_status launch_grad(const T* z, long rows, const Logits& a, const DistillGrad& g, T* dz, hipStream_t st) {
    const int chunks = chunk_count(sizeof(T) == 2 ? GP_BF16 : GP_F32, a.V);
    // 4096 workgroups in all where the rows have that much to split
    const long want = std::max(1L, std::min<long>((4096 + rows - 1) / rows, chunks / 512));
    const int splits = (int)want, per = (chunks + splits - 1) / splits;
    klaunch(distill_grad_kernel<T, CLIP, REST>, (unsigned)(rows * splits), 256, 0, st, z, a, g, dz, splits, per);
    GP_LAUNCH_CHECK();
    return GP_OK;
}

gp_status check_distill(int dtype, const void* logits, long rows, int vocab, long ld, const int* ids, const float* teacher,
                        int top, float scale, float clip) {
    auto bad = [](const char* m) { return set_error(GP_ERR_INVALID_ARG, m); };
    if (dtype != GP_F32 && dtype != GP_BF16) return bad("distill: unknown dtype");
    if (rows < 0 || rows > 0x7FFFFFFFL) return bad("distill: rows must be in [0, 2^31 - 1]");
    if (vocab < 1 || vocab > (1 << 30) || ld < vocab || ld > (1l << 40)) return bad("distill: vocab must be in [1, 2^30], ld in [vocab, 2^40]");
    if (top < 1 || top > GP_DISTILL_MAX) return bad("distill: top must be in [1, 256]");
    if (!(scale >= 1e-6f && scale <= 1e6f)) return bad("distill: scale must be in [1e-6, 1e6]");
    if (!(clip >= 0.f) || !std::isfinite(clip)) return bad("distill: clip must be >= 0 and finite");
    if (rows > 0 && (!logits || !ids || !teacher)) return bad("distill: logits, ids and teacher must not be NULL");
    if (!aligned(logits, dtype == GP_BF16 ? 2 : 4) || !aligned(ids, 4) || !aligned(teacher, 4)) return bad("distill: a misaligned address");
    return GP_OK;
}

// run(integral constants T, clipped, rest) for the types and flags of a call
template <typename F> gp_status with_flags(bool clipped, bool rest, F run) {
    if (clipped) return rest ? run(std::true_type{}, std::true_type{}) : run(std::true_type{}, std::false_type{});
    return rest ? run(std::false_type{}, std::true_type{}) : run(std::false_type{}, std::false_type{});
}

} // namespace

} // namespace gp

using namespace gp;

extern "C" {

gp_status gp_distill_workspace(int dtype, long rows, int vocab, size_t* bytes) {
    if (!bytes || (dtype != GP_F32 && dtype != GP_BF16) || rows < 0 || vocab < 1 || vocab > (1 << 30))
        return set_error(GP_ERR_INVALID_ARG, "distill_workspace: an argument is out of range");
    const int splits = row_splits(dtype, rows, vocab);
    *bytes = splits > 1 ? rows * splits * sizeof(Sum) : 0;
    return GP_OK;
}

gp_status gp_distill(int dtype, const void* logits, long rows, int vocab, long ld, const int* ids, const float* teacher,
                     int top, float scale, float clip, int rest, float* loss, float* lse, float* rest_lse, void* ws,
                     size_t ws_bytes, gp_stream stream) {
    const gp_status ok = check_distill(dtype, logits, rows, vocab, ld, ids, teacher, top, scale, clip);
    if (ok != GP_OK) return ok;
    auto bad = [](const char* m) { return set_error(GP_ERR_INVALID_ARG, m); };
    if (rows > 0 && (!loss || !lse || (rest && !rest_lse))) return bad("distill: loss, lse and with rest rest_lse must not be NULL");
    if (!aligned(loss, 4) || !aligned(lse, 4) || !aligned(rest_lse, 4)) return bad("distill: a misaligned address");
    if (!aligned(ws, 16)) return bad("distill: the workspace must be 16-byte aligned");
    for (long r = 0; r < rows; r += LAUNCH_ROWS) {
        const long n = std::min(LAUNCH_ROWS, rows - r);
        const Logits a = {vocab, ld, ids + r * top, teacher + r * top, top, scale, clip};
        const DistillOut out = {loss + r, lse + r, past(rest_lse, r)};
        GP_TRY(with_flags(clip > 0.f, rest != 0, [&](auto c, auto w) {
            if (dtype == GP_BF16)
                return launch_rows<bf16, c.value, w.value>(static_cast<const bf16*>(logits) + r * ld, n, a, out, ws, ws_bytes,
                                                           (hipStream_t)stream);
            return launch_rows<float, c.value, w.value>(static_cast<const float*>(logits) + r * ld, n, a, out, ws, ws_bytes,
                                                        (hipStream_t)stream);
        }));
    }
    return GP_OK;
}

gp_status gp_distill_backward(int dtype, const void* logits, long rows, int vocab, long ld, const int* ids,
                              const float* teacher, int top, float scale, float clip, int rest, const float* lse,
                              const float* rest_lse, const float* dloss, void* dlogits, long ldd, gp_stream stream) {
    const gp_status ok = check_distill(dtype, logits, rows, vocab, ld, ids, teacher, top, scale, clip);
    if (ok != GP_OK) return ok;
    auto bad = [](const char* m) { return set_error(GP_ERR_INVALID_ARG, m); };
    if (ldd < vocab || ldd > (1l << 40)) return bad("distill_backward: ldd must be in [vocab, 2^40]");
    if (rows > 0 && (!lse || !dloss || !dlogits || (rest && !rest_lse)))
        return bad("distill_backward: lse, dloss, dlogits and with rest rest_lse must not be NULL");
    const size_t es = dtype == GP_BF16 ? 2 : 4;
    if (!aligned(lse, 4) || !aligned(rest_lse, 4) || !aligned(dloss, 4) || !aligned(dlogits, es))
        return bad("distill_backward: a misaligned address");
    if (rows == 0) return GP_OK;
    const uintptr_t z0 = reinterpret_cast<uintptr_t>(logits), d0 = reinterpret_cast<uintptr_t>(dlogits);
    const uintptr_t z1 = z0 + ((size_t)(rows - 1) * ld + vocab) * es, d1 = d0 + ((size_t)(rows - 1) * ldd + vocab) * es;
    const bool same = z0 == d0 && (ld == ldd || rows == 1);
    if (!same && z0 < d1 && d0 < z1 && !side_by_side(z0, d0, (size_t)vocab * es, ld == ldd ? (size_t)ld * es : 0))
        return bad("distill_backward: dlogits overlaps the logits without being them");
    for (long r = 0; r < rows; r += LAUNCH_ROWS) {
        const long n = std::min(LAUNCH_ROWS, rows - r);
        const Logits a = {vocab, ld, ids + r * top, teacher + r * top, top, scale, clip};
        const DistillGrad g = {lse + r, past(rest_lse, r), dloss + r, ldd};
        GP_TRY(with_flags(clip > 0.f, rest != 0, [&](auto c, auto w) {
            if (dtype == GP_BF16)
                return launch_grad<bf16, c.value, w.value>(static_cast<const bf16*>(logits) + r * ld, n, a, g,
                                                           static_cast<bf16*>(dlogits) + r * ldd, (hipStream_t)stream);
            return launch_grad<float, c.value, w.value>(static_cast<const float*>(logits) + r * ld, n, a, g,
                                                        static_cast<float*>(dlogits) + r * ldd, (hipStream_t)stream);
        }));
    }
    return GP_OK;
}

} // extern "C"
