// attention_rows.hip -- attention on the caller's tensors: how its work is split,
// the bias's gradient by buckets, and the C ABI.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdio>

#include "attention_rows.hpp"
#include "common.hpp"

namespace gp {

namespace {

// Sums of n rows of `width` floats, STEP rows at a time: out row x = rows x STEP .. of head blockIdx.y.
constexpr int STEP = 128;
// rows r0 .. r1 - 1 added up into sums[width]: the 1024 threads make groups that take every n-th row, whose sums are
// added in order.
__device__ __forceinline__ void add_rows(const float* in, long r0, long r1, int width, float* sums, float* groups) {
    const int cols = min(1024, (width + 63) / 64 * 64), n = 1024 / cols, g = threadIdx.x / cols, c = threadIdx.x - g * cols;
    for (int d0 = 0; d0 < width; d0 += cols) {
        const int d = d0 + c;
        float s = 0.f;
        if (d < width && g < n) {
#pragma unroll 8
            for (long r = r0 + g; r < r1; r += n) s += in[r * width + d];
        }
        groups[threadIdx.x] = s;
        __syncthreads();
        if (d < width && g == 0) {
            for (int x = 1; x < n; ++x) s += groups[x * cols + c];
            sums[d] = s;
        }
        __syncthreads();
    }
}
__global__ void __launch_bounds__(1024) distance_rows(const float* __restrict__ in, long n, int width, float* __restrict__ out) {
    __shared__ float groups[1024];
    const long x = blockIdx.x, y = blockIdx.y, steps = gridDim.x;
    add_rows(in + y * n * width, x * STEP, min(n, x * STEP + STEP), width, out + (y * steps + x) * width, groups);
}
// dbias of head blockIdx.x: its n rows of distances added up, then the distances of each bucket by a wave.
__global__ void __launch_bounds__(1024) distance_buckets(const float* __restrict__ in, long n, AttendArgs a) {
    __shared__ float groups[1024], sums[2 * GP_DISTANCE_MAX + 1];
    __shared__ int of[2 * GP_DISTANCE_MAX + 1];
    const int width = 2 * a.max_distance + 1, lane = threadIdx.x & 63;
    for (int d = threadIdx.x; d < width; d += 1024) of[d] = min(max(a.bucket_of[d], 0), a.buckets - 1);
    add_rows(in + blockIdx.x * n * width, 0, n, width, sums, groups);
    for (int b = threadIdx.x >> 6; b < a.buckets; b += 16) {
        float s = 0.f;
        for (int d = lane; d < width; d += WAVE) s += of[d] == b ? sums[d] : 0.f;
        s = wave_sum(s);
        if (lane == 0) a.dbias[(long)blockIdx.x * a.buckets + b] = s;
    }
}

long up(long n, long m) { return (n + m - 1) / m * m; }
long stat_rows(int Sq) { return up(Sq, 64); }
int esize(const AttendArgs& a) { return a.dtype == GP_BF16 ? 2 : 4; }

// Rows of a group's heads share their keys' tiles where they fit into one; up to 32 rows are left to waves that share them.
// Fewer than 1024 waves (one a SIMD) are split into up to 2048, each over 4 tiles or more: 40 queries of 16 heads to 30000 keys 35 us, 2
// of 16 on 4 heads to 60000 34.
Shape forward_shape(const AttendArgs& a) {
    Shape s;
    const int group = a.H / a.HK;
    if (!a.bias && group > 1 && a.Sq < 32) s.pack = group;
    const long rows = (long)a.Sq * s.pack;
    s.keys = rows <= 32;
    s.blocks = (int)((rows + (s.keys ? 31 : 127)) / (s.keys ? 32 : 128));
    const int waves = s.keys ? key_waves(head_bucket(a.dh) * esize(a)) : 4;
    const long groups = std::max(1l, (long)a.B * (a.H / s.pack) * s.blocks);
    const int tiles = (a.Sk + 31) / 32;
    if (groups * waves < 1024)
        s.splits = (int)std::max(1l, std::min<long>(std::min(64, tiles / (s.keys ? 4 * waves : 4)), 2048 / (groups * waves)));
    return s;
}
// Blocks of 128 rows (`rows` of them in each of `groups`), whose work is `tiles` tiles long.  Fewer than one for each CU are split, and
// another launch adds up: fp32 backward of 3 x 77 queries to up to 501 keys 103 us whole, 41 split to two tiles, 31 to one.  A tile
// is 2 to 3 us of fp32's products, but a fraction of one of bf16's.
Shape backward_shape(const AttendArgs& a, long groups, int rows, long tiles) {
    Shape s;
    s.blocks = (rows + 32 * BW - 1) / (32 * BW);
    groups = std::max(1l, groups * s.blocks);
    if (groups < 256) s.splits = (int)std::max(1l, std::min(std::min(32l, a.dtype == GP_BF16 ? tiles / 2 : tiles), 512 / groups));
    return s;
}
Shape dq_shape(const AttendArgs& a) {
    const int kt = tile_rows(esize(a));
    return backward_shape(a, (long)a.B * a.H, a.Sq, (a.Sk + kt - 1) / kt);
}
Shape dkv_shape(const AttendArgs& a) {
    const int qt = tile_rows(esize(a));
    return backward_shape(a, (long)a.B * a.HK, a.Sk, (long)(a.H / a.HK) * ((a.Sq + qt - 1) / qt));
}
// Rows of distances of one head that the dK and dV kernel writes.
long distance_rows_of(const AttendArgs& a) {
    const Shape s = dkv_shape(a);
    return (long)a.B * s.blocks * s.splits;
}
size_t distance_floats(const AttendArgs& a) {
    const size_t rows = (size_t)distance_rows_of(a);
    return a.bias ? a.H * (rows + (rows + STEP - 1) / STEP) * (2 * (size_t)a.max_distance + 1) : 0;
}
// The splits' sums of dQ, dK and dV, and in bf16 those that refine dQ and delta.
size_t part_floats(const AttendArgs& a) {
    const Shape q = dq_shape(a), k = dkv_shape(a);
    const size_t nq = q.splits > 1 ? (size_t)q.splits * a.B * a.H * a.Sq : 0;
    const size_t nk = k.splits > 1 ? (size_t)k.splits * a.B * a.HK * a.Sk * 2 : 0;
    const size_t dh = head_bucket(a.dh);
    return (a.dtype == GP_BF16 ? refined_floats(nq, dh) : nq * dh) + nk * dh;
}

} // namespace

size_t attend_workspace(const AttendArgs& a) {
    const Shape s = forward_shape(a);
    return s.splits > 1 ? (size_t)s.splits * a.B * a.H * a.Sq * (head_bucket(a.dh) + 2) * 4 : 0;
}

gp_status attend_forward(AttendArgs a, void* ws, hipStream_t st) {
    const Shape s = forward_shape(a);
    a.keys = s.keys;
    a.pack = s.pack;
    a.blocks = s.blocks;
    a.splits = s.splits;
    a.part = static_cast<float*>(ws);
    return a.dtype == GP_BF16 ? attend_forward_as<bf16>(a, st) : attend_forward_as<float>(a, st);
}

// Statistics of the rows, the splits' sums, sums by distance: each a multiple of 16 bytes but the last.
size_t attend_backward_workspace(const AttendArgs& a) {
    return (size_t)a.B * a.H * stat_rows(a.Sq) * 8 + (part_floats(a) + distance_floats(a)) * 4;
}

gp_status attend_backward(AttendArgs a, bool exact, void* ws, hipStream_t st) {
    a.stat_rows = (int)stat_rows(a.Sq);
    a.stats = static_cast<float*>(ws);
    a.part = a.stats + (size_t)a.B * a.H * 2 * a.stat_rows;
    float* dist = a.part + part_floats(a);
    a.dist = a.bias && a.dbias ? dist : nullptr;
    if (a.B)
        GP_TRY(a.dtype == GP_BF16 ? attend_backward_as<bf16>(a, exact, dq_shape(a), dkv_shape(a), st)
                                  : attend_backward_as<float>(a, exact, dq_shape(a), dkv_shape(a), st));
    if (!a.bias || !a.dbias) return GP_OK;
    const int width = 2 * a.max_distance + 1;
    long n = distance_rows_of(a);
    const float* in = dist;
    if (n > STEP) {
        float* out = dist + (size_t)a.H * n * width;
        const long steps = (n + STEP - 1) / STEP;
        klaunch(distance_rows, dim3((unsigned)steps, (unsigned)a.H), dim3(1024), 0, st, in, n, width, out);
        in = out;
        n = steps;
    }
    klaunch(distance_buckets, dim3((unsigned)a.H), dim3(1024), 0, st, in, n, a);
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
    if (!(c->scale >= 1e-6f && c->scale <= 1e6f)) return bad("scale must be in [1e-6, 1e6]");
    for (const int* p : {c->q_lens, c->k_lens, c->q_starts})
        if (!aligned(p, 4)) return bad("misaligned lengths or positions");
    if (c->bias) {
        if (!c->bucket_of || c->buckets < 1 || c->max_distance < 1) return bad("a bias needs bucket_of, buckets >= 1 and max_distance >= 1");
        if (!aligned(c->bias, 4) || !aligned(c->bucket_of, 4)) return bad("a misaligned bias or bucket_of");
    } else if (c->bucket_of || c->buckets || c->max_distance) {
        return bad("bucket_of, buckets and max_distance belong to a bias");
    }
    // a launch holds fewer than 2^32 threads, 256 of them take 128 rows and 512 a few; a head's own grid dimension 2^16
    const long groups = (long)c->batch * c->heads;
    if (c->heads > 65535 || groups >= (1l << 23) || groups * (c->q_len / 128 + 1l) >= (1l << 23) ||
        groups * (c->k_len / 128 + 1l) >= (1l << 23))
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
    for (const Rows::Dim& d : {Rows::Dim{r.seq, a.B}, Rows::Dim{r.row, len}, Rows::Dim{r.head, heads}}) {
        if (d.stride > (1l << 47) / d.n) return "a stride is out of range";  // of any address
        if (d.n > 1) out.dim[out.dims++] = d;
    }
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
    return attend_backward(a, !out, ws, (hipStream_t)stream);
}

} // extern "C"
