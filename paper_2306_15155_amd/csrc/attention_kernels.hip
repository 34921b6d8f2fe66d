// Multi-head attention over the stored entries of a pattern, forward and backward: scores scale <q_i, k_j>, optionally capped by a tanh and
// biased by the entry's bucket, softmax over a row's entries, weights optionally dropped; key and value heads may be shared by query heads.
//
// Nothing is stored per entry.  The forward walk keeps a running maximum m, sum l and weighted sum of values per row; the backward forms the
// weights again from the rows' (m, log l):
//     x = bias + cap tanh(scale <q, k> / cap),  p = exp(x - m - log l),  dt = p (keep/(1-p_drop) <dy, v> - D),  D_i = <dy_i, y_i>,
//     dq_i = sum_j ds k_j,  dk_j = sum_i ds q_i,  dv_j = sum_i p keep/(1-p_drop) dy_i,  dbias[h, b] = sum dt,  ds = dt (1 - tanh^2) scale
// as two walks, one over the rows (dq, dbias) and one over the transposed pattern (dk, dv), so that no sum needs an atomic.
//
// What bounds these walks is the gathering of k and v (q and dy) rows from the caches: an entry takes 2 d elements a head for 4 d
// operations.  A head's vector is spread over G lanes, eight elements (four for heads of at most 16) a lane; a group of lanes takes the same
// entry for a few neighbouring heads (a bundle), so that a gather fills a 128-byte line and shared key heads are read once; and every group
// walks a chunk of consecutive entries by itself, four at a time.  Rows that cross chunks leave a piece per chunk in scratch, joined by
// a second kernel in chunk order: results do not depend on scheduling.
#include "element_types.h"
#include "sensei_internal.h"

namespace sensei {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kBatch = 4;

struct WalkPattern {
    const int32_t *row_ptr, *col;
    const uint8_t *bucket;        // in this pattern's order, null: none
    const int32_t *chunk_row;     // row of the first entry of every chunk
    int n_rows, nnz, chunk, n_chunks;
};

struct AttnArgs {
    WalkPattern p;
    const void *Q, *K, *V, *Y, *dY;
    void *O1, *O2;                // outputs: Y, dQ, or dK and dV
    long long ldq, ldk, ldv, ldy, lddy, ldo1, ldo2;
    float2 *stats;                // (m, log l) of every row and query head
    float4 *row_stats;            // (m, log l, D, -) for the walk over the transposed pattern
    int heads, kv_heads, ratio, d, dv;
    float scale, cap, inv_cap;
    const float *bias;
    int n_buckets;
    int bundle_log;               // heads of a bundle: 1 << bundle_log
    DropKey key;                  // threshold 0: nothing is dropped
    float *piece;                 // sums of row pieces: (chunk, first or last piece, head) x G * VEC floats (twice that where two sums are kept)
    float2 *piece_ml;
    float *bias_part;             // a block's share of dbias, null: not asked for
};

// ------------------------------------------------------------------------------------------------------------------ lanes of a head

template <int CTRL> __device__ __forceinline__ float dpp(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true)); }
template <int CTRL> __device__ __forceinline__ int dpp(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, true); }

// sum over the G lanes of a head, in all of them (G neighbouring lanes are always active together)
template <int G> __device__ __forceinline__ float head_sum(float x) {
    x += dpp<0xB1>(x);                       // the neighbour in a pair
    x += dpp<0x4E>(x);                       // the other pair of a quad
    if (G >= 8) x += dpp<0x141>(x);          // mirrored within eight lanes
    if (G >= 16) x += dpp<0x140>(x);         // mirrored within sixteen
    if (G >= 32) x += __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(x), 0x401F));   // sixteen lanes away
    return x;
}

// a lane's share of a head's vector: PIECES pieces of PER elements, piece r at element (r G + t) PER, so that the lanes of a head read side by side
template <class T, int VEC, int G> struct Share {
    static constexpr int PER = VEC < kPerPiece<T> ? VEC : kPerPiece<T>, PIECES = VEC / PER;
    float v[VEC];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] = 0.f;
    }
    __device__ __forceinline__ void load(const T *p, int t, int d) {
#pragma unroll
        for (int r = 0; r < PIECES; ++r) {
            const int at = (r * G + t) * PER;
            if (at + PER <= d) {
                const Piece<T, PER> x = Piece<T, PER>::load(p + at);
#pragma unroll
                for (int k = 0; k < PER; ++k) v[r * PER + k] = to_f32(x.x[k]);
            } else {
#pragma unroll
                for (int k = 0; k < PER; ++k) v[r * PER + k] = 0.f;
                if (at < d) {
#pragma unroll
                    for (int k = 0; k < PER; ++k)
                        if (at + k < d) v[r * PER + k] = to_f32(p[at + k]);
                }
            }
        }
    }
    __device__ __forceinline__ void store(T *p, int t, int d, float by) const {
#pragma unroll
        for (int r = 0; r < PIECES; ++r) {
            const int at = (r * G + t) * PER;
            Piece<T, PER> x;
#pragma unroll
            for (int k = 0; k < PER; ++k) x.x[k] = from_f32<T>(v[r * PER + k] * by);
            if (at + PER <= d) x.store(p + at);
            else if (at < d) {
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (at + k < d) p[at + k] = x.x[k];
            }
        }
    }
    // scratch: VEC floats a lane, lane by lane
    __device__ __forceinline__ void put(float *p, int t) const {
#pragma unroll
        for (int k = 0; k < VEC; k += 4) *reinterpret_cast<float4 *>(p + t * VEC + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
    }
    __device__ __forceinline__ void get(const float *p, int t) {
#pragma unroll
        for (int k = 0; k < VEC; k += 4) {
            const float4 x = *reinterpret_cast<const float4 *>(p + t * VEC + k);
            v[k] = x.x; v[k + 1] = x.y; v[k + 2] = x.z; v[k + 3] = x.w;
        }
    }
    __device__ __forceinline__ float dot(const Share &o) const {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < VEC; ++k) s = fmaf(v[k], o.v[k], s);
        return s;
    }
    __device__ __forceinline__ void add(float w, const Share &o) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] = fmaf(w, o.v[k], v[k]);
    }
    __device__ __forceinline__ void scale(float w) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] *= w;
    }
};

// ------------------------------------------------------------------------------------------------------------------ walk of a chunk

// A group's place in its chunk: the row it is in, and the columns (and buckets) of the next four entries, fetched a batch ahead.
struct Walk {
    int e, end, i, row_end;
    bool goes_on;            // the row began in an earlier chunk
    int col[kBatch];
    unsigned bucket;         // four of eight bits
    __device__ __forceinline__ void fetch(const WalkPattern &p, int at) {
        if (at + kBatch <= p.nnz) {
            const Piece<float, 4>::Raw x = *reinterpret_cast<const Piece<float, 4>::Raw *>(p.col + at);
            col[0] = (int)x.x; col[1] = (int)x.y; col[2] = (int)x.z; col[3] = (int)x.w;
            typedef unsigned Byte4 __attribute__((aligned(1)));
            bucket = p.bucket ? *reinterpret_cast<const Byte4 *>(p.bucket + at) : 0u;
        } else {
            bucket = 0u;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int k = at + u < p.nnz ? at + u : p.nnz - 1;
                col[u] = p.col[k];
                if (p.bucket) bucket |= (unsigned)p.bucket[k] << (8 * u);
            }
        }
    }
    __device__ __forceinline__ void begin(const WalkPattern &p, int chunk) {
        e = chunk * p.chunk;
        end = p.nnz - e < p.chunk ? p.nnz : e + p.chunk;
        i = p.chunk_row[chunk];
        row_end = p.row_ptr[i + 1];
        goes_on = p.row_ptr[i] < e;
        fetch(p, e);
    }
    __device__ __forceinline__ int count() const {
        const int n = (row_end < end ? row_end : end) - e;
        return n < kBatch ? n : kBatch;
    }
    __device__ __forceinline__ bool row_done() const { return e == row_end || e == end; }
    // the row of entry e, which lies behind row i: the next one, or across a run of empty rows by doubling steps and halving
    __device__ __forceinline__ void next_row(const WalkPattern &p) {
        int lo = i, hi = i + 1, step = 1;
        row_end = p.row_ptr[hi + 1];
        if (row_end <= e) {
            do {
                lo = hi;
                hi = hi + step < p.n_rows ? hi + step : p.n_rows - 1;
                step *= 2;
            } while (p.row_ptr[hi + 1] <= e);
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.row_ptr[mid + 1] <= e) lo = mid; else hi = mid;
            }
            row_end = p.row_ptr[hi + 1];
        }
        i = hi;
        goes_on = false;
    }
};

// Where a lane works: t of the G lanes of head h, group `chunk` of the walk.
template <int G> struct Place {
    int t, slot, in_bundle, h, chunk;
    bool live;       // a head and a chunk that there are
    __device__ __forceinline__ Place(int n_heads, int n_chunks, int bundle_log) {
        const int lane = threadIdx.x & 63, groups = (64 / G) >> bundle_log;
        t = lane % G;
        slot = lane / G;
        in_bundle = slot & ((1 << bundle_log) - 1);
        const int head = ((int)blockIdx.y << bundle_log) + in_bundle;
        chunk = ((int)blockIdx.x * kWaves + (int)(threadIdx.x >> 6)) * groups + (slot >> bundle_log);
        live = head < n_heads && chunk < n_chunks;
        h = head < n_heads ? head : n_heads - 1;
    }
};

// tanh(x) and 1 - tanh(x)^2.  From a quarter on by y = exp(-2 |x|): (1 - y) / (1 + y) and 4 y / (1 + y)^2; below, where 1 - y would cancel, by the
// odd series up to x^11 (what is left out is below 3e-10 of the value).
struct Tanh { float value, slope; };
__device__ __forceinline__ Tanh tanh_of(float x) {
    const float a = fabsf(x), y = __builtin_amdgcn_exp2f(a * (-2.f * kLog2E)), r = __builtin_amdgcn_rcpf(1.f + y);
    const float x2 = x * x;
    float s = fmaf(x2, -1382.f / 155925.f, 62.f / 2835.f);
    s = fmaf(x2, s, -17.f / 315.f);
    s = fmaf(x2, s, 2.f / 15.f);
    s = fmaf(x2, s, -1.f / 3.f);
    s = fmaf(x * x2, s, x);
    return a < 0.25f ? Tanh{s, fmaf(-s, s, 1.f)} : Tanh{copysignf((1.f - y) * r, x), 4.f * y * r * r};
}

// the bundle's bias table in LDS; every thread of the workgroup comes here
__device__ __forceinline__ const float *load_bias(const AttnArgs &a, float *lds) {
    if (!a.bias) return nullptr;
    const int n = a.n_buckets << a.bundle_log, first = ((int)blockIdx.y << a.bundle_log) * a.n_buckets, all = a.heads * a.n_buckets;
    for (int k = threadIdx.x; k < n; k += kThreads) lds[k] = first + k < all ? a.bias[first + k] : 0.f;
    __syncthreads();
    return lds;
}
__device__ __forceinline__ int bucket_of(const AttnArgs &a, unsigned four, int u) {
    const int b = (int)(four >> (8 * u) & 255u);
    return b < a.n_buckets ? b : a.n_buckets - 1;
}

// Which of the four entries (row of the pattern: row[u], column: col[u]) keep their weight for query head h.  A quad of lanes works out an entry each
// and hands the answers round: one generator call a lane and batch.
__device__ __forceinline__ void keep_flags(const DropKey &key, unsigned offset, const int *row, const int *col, int h, int t, bool *keep) {
    const int u = t & 3;
    const unsigned r = (unsigned)(u & 2 ? (u & 1 ? row[3] : row[2]) : (u & 1 ? row[1] : row[0]));
    const unsigned c = (unsigned)(u & 2 ? (u & 1 ? col[3] : col[2]) : (u & 1 ? col[1] : col[0]));
    const Words w = philox(c, r, 0x80000000u | (unsigned)(h >> 2), offset, key.k0, key.k1);
    const unsigned mine = h & 2 ? (h & 1 ? w.w[3] : w.w[2]) : (h & 1 ? w.w[1] : w.w[0]);
    const int kept = mine >= key.threshold;
    keep[0] = dpp<0x00>(kept) != 0;
    keep[1] = dpp<0x55>(kept) != 0;
    keep[2] = dpp<0xAA>(kept) != 0;
    keep[3] = dpp<0xFF>(kept) != 0;
}
__device__ __forceinline__ unsigned drop_offset(const DropKey &key) { return key.offset + (key.offset_dev ? *key.offset_dev : 0u); }

// slot of a row piece: first piece of a chunk when the row goes on from the chunk before, else its last
__device__ __forceinline__ size_t piece_at(int chunk, bool goes_on, int heads, int h) { return ((size_t)chunk * 2 + (goes_on ? 0 : 1)) * heads + h; }

// ------------------------------------------------------------------------------------------------------------------ forward

template <class T, int VEC, int G>
__global__ __launch_bounds__(kThreads) void k_attention(AttnArgs a) {
    extern __shared__ float lds[];
    const float *bias = load_bias(a, lds);
    const Place<G> at(a.heads, a.p.n_chunks, a.bundle_log);
    if (!at.live) return;
    const int h = at.h, g = h / a.ratio, t = at.t;
    const T *Q = static_cast<const T *>(a.Q) + (size_t)h * a.d, *K = static_cast<const T *>(a.K) + (size_t)g * a.d, *V = static_cast<const T *>(a.V) + (size_t)g * a.dv;
    T *Y = static_cast<T *>(a.O1) + (size_t)h * a.dv;
    if (bias) bias += at.in_bundle * a.n_buckets;
    const unsigned offset = drop_offset(a.key);
    Walk w;
    w.begin(a.p, at.chunk);
    Share<T, VEC, G> q, acc;
    q.load(Q + (long long)w.i * a.ldq, t, a.d);
    acc.zero();
    float m = -INFINITY, l = 0.f;
    while (w.e < w.end) {
        const int n = w.count();
        int col[kBatch], row[kBatch];
        bool use[kBatch], keep[kBatch];
        float x[kBatch], b[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            col[u] = w.col[u];
            row[u] = w.i;
            use[u] = u < n;
            keep[u] = true;
            b[u] = bias ? bias[bucket_of(a, w.bucket, u)] : 0.f;
            use[u] = use[u] && b[u] != -INFINITY;    // a masked entry has no share, whatever its key and value hold
        }
        if (w.e + n < w.end) w.fetch(a.p, w.e + n);
        if (a.key.threshold) keep_flags(a.key, offset, row, col, h, t, keep);
        Share<T, VEC, G> k[kBatch], v[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            k[u].zero();
            if (use[u]) k[u].load(K + (long long)col[u] * a.ldk, t, a.d);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            v[u].zero();
            if (use[u] && keep[u]) v[u].load(V + (long long)col[u] * a.ldv, t, a.dv);
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            x[u] = head_sum<G>(q.dot(k[u])) * a.scale;
            if (a.cap > 0.f) x[u] = a.cap * tanh_of(x[u] * a.inv_cap).value;
            x[u] = use[u] ? x[u] + b[u] : -INFINITY;
            top = fmaxf(top, x[u]);
        }
        const float base = top > -INFINITY ? top : 0.f;
        const float f = exp_neg(m - base);
        m = top;
        l *= f;
        acc.scale(f);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const float p = exp_neg(x[u] - base);
            l += p;
            acc.add(keep[u] ? p : 0.f, v[u]);
        }
        w.e += n;
        if (w.row_done()) {
            if (!w.goes_on && w.e == w.row_end) {
                acc.store(Y + (long long)w.i * a.ldo1, t, a.dv, l == 0.f ? 0.f : a.key.keep_scale / l);
                if (t == 0) a.stats[(size_t)w.i * a.heads + h] = make_float2(m, logf(l));
            } else {
                const size_t s = piece_at(at.chunk, w.goes_on, a.heads, h);
                acc.put(a.piece + s * (G * VEC), t);
                if (t == 0) a.piece_ml[s] = make_float2(m, l);
            }
            if (w.e < w.end) {
                w.next_row(a.p);
                q.load(Q + (long long)w.i * a.ldq, t, a.d);
                acc.zero();
                m = -INFINITY;
                l = 0.f;
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------------------------ backward, over the rows

template <class T, int VEC, int G>
__global__ __launch_bounds__(kThreads) void k_attention_back_rows(AttnArgs a) {
    extern __shared__ float lds[];
    const float *bias = load_bias(a, lds);
    const Place<G> at(a.heads, a.p.n_chunks, a.bundle_log);
    // dbias: a table of its own for every head of every group, so that its sums have one order
    float *tables = lds + ((a.n_buckets << a.bundle_log) + 3) / 4 * 4, *mine = tables + ((threadIdx.x >> 6) * (64 / G) + at.slot) * a.n_buckets;
    if (a.bias_part) {
        for (int k = threadIdx.x; k < kWaves * (64 / G) * a.n_buckets; k += kThreads) tables[k] = 0.f;
        __syncthreads();
    }
    if (at.live) {
        const int h = at.h, g = h / a.ratio, t = at.t;
        const T *Q = static_cast<const T *>(a.Q) + (size_t)h * a.d, *K = static_cast<const T *>(a.K) + (size_t)g * a.d, *V = static_cast<const T *>(a.V) + (size_t)g * a.dv;
        const T *Y = static_cast<const T *>(a.Y) + (size_t)h * a.dv, *dY = static_cast<const T *>(a.dY) + (size_t)h * a.dv;
        T *dQ = static_cast<T *>(a.O1) + (size_t)h * a.d;
        const float *my_bias = bias ? bias + at.in_bundle * a.n_buckets : nullptr;
        const unsigned offset = drop_offset(a.key);
        Walk w;
        w.begin(a.p, at.chunk);
        Share<T, VEC, G> q, dy, acc;
        float m, log_l, D;
        auto enter = [&]() {
            Share<T, VEC, G> y;
            q.load(Q + (long long)w.i * a.ldq, t, a.d);
            dy.load(dY + (long long)w.i * a.lddy, t, a.dv);
            y.load(Y + (long long)w.i * a.ldy, t, a.dv);
            const float2 ml = a.stats[(size_t)w.i * a.heads + h];
            m = ml.x;
            log_l = ml.y;
            D = head_sum<G>(dy.dot(y));
            if (!w.goes_on && t == 0) a.row_stats[(size_t)w.i * a.heads + h] = make_float4(m, log_l, D, 0.f);
            acc.zero();
        };
        enter();
        while (w.e < w.end) {
            const int n = w.count();
            int col[kBatch], row[kBatch], bin[kBatch];
            bool use[kBatch], keep[kBatch];
            float b[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                col[u] = w.col[u];
                row[u] = w.i;
                keep[u] = true;
                bin[u] = my_bias ? bucket_of(a, w.bucket, u) : 0;
                b[u] = my_bias ? my_bias[bin[u]] : 0.f;
                use[u] = u < n && b[u] != -INFINITY;
            }
            if (w.e + n < w.end) w.fetch(a.p, w.e + n);
            if (a.key.threshold) keep_flags(a.key, offset, row, col, h, t, keep);
            Share<T, VEC, G> k[kBatch], v[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                k[u].zero();
                if (use[u]) k[u].load(K + (long long)col[u] * a.ldk, t, a.d);
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                v[u].zero();
                if (use[u] && keep[u]) v[u].load(V + (long long)col[u] * a.ldv, t, a.dv);
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                float x = head_sum<G>(q.dot(k[u])) * a.scale, slope = 1.f;
                if (a.cap > 0.f) {
                    const Tanh th = tanh_of(x * a.inv_cap);
                    x = a.cap * th.value;
                    slope = th.slope;
                }
                const float p = use[u] ? exp_neg((x + b[u] - m) - log_l) : 0.f;
                const float dp = head_sum<G>(dy.dot(v[u])) * a.key.keep_scale;
                const float dt = use[u] ? p * (dp - D) : 0.f;
                if (a.bias_part && t == 0 && use[u]) __hip_atomic_fetch_add(mine + bin[u], dt, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                acc.add(dt * slope * a.scale, k[u]);
            }
            w.e += n;
            if (w.row_done()) {
                if (!w.goes_on && w.e == w.row_end) acc.store(dQ + (long long)w.i * a.ldo1, t, a.d, 1.f);
                else acc.put(a.piece + piece_at(at.chunk, w.goes_on, a.heads, h) * (G * VEC), t);
                if (w.e < w.end) {
                    w.next_row(a.p);
                    enter();
                }
            }
        }
    }
    if (a.bias_part) {
        __syncthreads();
        const int n = a.n_buckets << a.bundle_log, per_wave = 64 / G;
        for (int k = threadIdx.x; k < n; k += kThreads) {
            const int in_bundle = k / a.n_buckets, b = k % a.n_buckets, h = ((int)blockIdx.y << a.bundle_log) + in_bundle;
            if (h >= a.heads) continue;
            float s = 0.f;
            for (int o = in_bundle; o < kWaves * per_wave; o += 1 << a.bundle_log) s += tables[o * a.n_buckets + b];
            a.bias_part[((size_t)blockIdx.x * a.heads + h) * a.n_buckets + b] = s;
        }
    }
}

// dbias[k] = sum over the blocks of the walk, in their order; sixteen sums a workgroup, 64 threads each
__global__ __launch_bounds__(1024) void k_attention_bias(const float *__restrict__ part, int blocks, int n, float *__restrict__ out) {
    __shared__ double lds[64][16];
    const int k = blockIdx.x * 16 + (threadIdx.x & 15), seg = threadIdx.x >> 4;
    double s = 0.0;
    if (k < n)
        for (int b = seg; b < blocks; b += 64) s += (double)part[(size_t)b * n + k];
    lds[seg][threadIdx.x & 15] = s;
    for (int half = 32; half > 0; half >>= 1) {
        __syncthreads();
        if (seg < half) lds[seg][threadIdx.x & 15] += lds[seg + half][threadIdx.x & 15];
    }
    if (seg == 0 && k < n) out[k] = (float)lds[0][threadIdx.x & 15];
}

// ------------------------------------------------------------------------------------------------------------------ backward, over the columns

// The walk goes over the transposed pattern: its rows are the columns j, its entries the rows i that attend to them.  A lane stays with one key
// head and takes that head's query heads one after the other.
template <class T, int VEC, int G>
__global__ __launch_bounds__(kThreads) void k_attention_back_cols(AttnArgs a) {
    extern __shared__ float lds[];
    const float *bias = nullptr;
    const Place<G> at(a.kv_heads, a.p.n_chunks, a.bundle_log);
    if (a.bias) {   // of all query heads of the bundle's key heads
        const int per = a.ratio * a.n_buckets, n = per << a.bundle_log, first = ((int)blockIdx.y << a.bundle_log) * per, all = a.heads * a.n_buckets;
        for (int k = threadIdx.x; k < n; k += kThreads) lds[k] = first + k < all ? a.bias[first + k] : 0.f;
        __syncthreads();
        bias = lds + at.in_bundle * per;
    }
    if (!at.live) return;
    const int g = at.h, t = at.t;
    const T *Q = static_cast<const T *>(a.Q), *dY = static_cast<const T *>(a.dY);
    const T *K = static_cast<const T *>(a.K) + (size_t)g * a.d, *V = static_cast<const T *>(a.V) + (size_t)g * a.dv;
    T *dK = static_cast<T *>(a.O1) + (size_t)g * a.d, *dV = static_cast<T *>(a.O2) + (size_t)g * a.dv;
    const unsigned offset = drop_offset(a.key);
    Walk w;
    w.begin(a.p, at.chunk);
    Share<T, VEC, G> k, v, dk, dv;
    k.load(K + (long long)w.i * a.ldk, t, a.d);
    v.load(V + (long long)w.i * a.ldv, t, a.dv);
    dk.zero();
    dv.zero();
    while (w.e < w.end) {
        const int n = w.count();
        int col[kBatch], row[kBatch], bin[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            row[u] = w.col[u];
            col[u] = w.i;
            bin[u] = bias ? bucket_of(a, w.bucket, u) : 0;
        }
        if (w.e + n < w.end) w.fetch(a.p, w.e + n);
        for (int r = 0; r < a.ratio; ++r) {
            const int h = g * a.ratio + r;
            bool use[kBatch], keep[kBatch];
            float b[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                keep[u] = true;
                b[u] = bias ? bias[r * a.n_buckets + bin[u]] : 0.f;
                use[u] = u < n && b[u] != -INFINITY;
            }
            if (a.key.threshold) keep_flags(a.key, offset, row, col, h, t, keep);
            Share<T, VEC, G> q[kBatch], dy[kBatch];
            float4 st[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                q[u].zero();
                dy[u].zero();
                st[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (use[u]) {
                    q[u].load(Q + (long long)row[u] * a.ldq + (size_t)h * a.d, t, a.d);
                    st[u] = a.row_stats[(size_t)row[u] * a.heads + h];
                    if (keep[u]) dy[u].load(dY + (long long)row[u] * a.lddy + (size_t)h * a.dv, t, a.dv);
                }
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                float x = head_sum<G>(k.dot(q[u])) * a.scale, slope = 1.f;
                if (a.cap > 0.f) {
                    const Tanh th = tanh_of(x * a.inv_cap);
                    x = a.cap * th.value;
                    slope = th.slope;
                }
                const float p = use[u] ? exp_neg((x + b[u] - st[u].x) - st[u].y) : 0.f;
                const float dp = head_sum<G>(v.dot(dy[u])) * a.key.keep_scale;
                const float dt = use[u] ? p * (dp - st[u].z) : 0.f;
                dk.add(dt * slope * a.scale, q[u]);
                dv.add(keep[u] ? p * a.key.keep_scale : 0.f, dy[u]);
            }
        }
        w.e += n;
        if (w.row_done()) {
            if (!w.goes_on && w.e == w.row_end) {
                dk.store(dK + (long long)w.i * a.ldo1, t, a.d, 1.f);
                dv.store(dV + (long long)w.i * a.ldo2, t, a.dv, 1.f);
            } else {
                float *s = a.piece + piece_at(at.chunk, w.goes_on, a.kv_heads, g) * (2 * G * VEC);
                dk.put(s, t);
                dv.put(s + G * VEC, t);
            }
            if (w.e < w.end) {
                w.next_row(a.p);
                k.load(K + (long long)w.i * a.ldk, t, a.d);
                v.load(V + (long long)w.i * a.ldv, t, a.dv);
                dk.zero();
                dv.zero();
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------------------------ rows in pieces, empty rows

enum { kJoinForward = 0, kJoinOne = 1, kJoinTwo = 2 };

// A wavefront per chunk boundary (and bundle of heads): where a row crosses it that crossed none before, the wavefront joins that row's pieces, its
// groups taking them in turn.  Workgroups behind those (of the first bundle) look over 64 rows a wavefront and write the rows without entries.
template <class T, int VEC, int G, int MODE>
__global__ __launch_bounds__(kThreads) void k_attention_join(AttnArgs a, int n_heads, int join_blocks) {
    const int lane = threadIdx.x & 63, wave = (int)blockIdx.x * kWaves + (int)(threadIdx.x >> 6);
    if ((int)blockIdx.x >= join_blocks) {
        if (blockIdx.y > 0) return;
        const long long r0 = ((long long)((int)blockIdx.x - join_blocks) * kWaves + (threadIdx.x >> 6)) * 64;
        const bool none = r0 + lane < a.p.n_rows && a.p.row_ptr[r0 + lane] == a.p.row_ptr[r0 + lane + 1];
        unsigned long long todo = __ballot(none);
        const int w1 = MODE == kJoinForward ? n_heads * a.dv : n_heads * a.d, w2 = MODE == kJoinTwo ? n_heads * a.dv : 0;
        while (todo) {
            const long long row = r0 + __builtin_ctzll(todo);
            todo &= todo - 1;
            for (int c = lane; c < w1; c += 64) static_cast<T *>(a.O1)[row * a.ldo1 + c] = from_f32<T>(0.f);
            for (int c = lane; c < w2; c += 64) static_cast<T *>(a.O2)[row * a.ldo2 + c] = from_f32<T>(0.f);
            if (MODE == kJoinForward)
                for (int h = lane; h < n_heads; h += 64) a.stats[row * n_heads + h] = make_float2(-INFINITY, -INFINITY);
        }
        return;
    }
    const int c = wave + 1;
    if (c >= a.p.n_chunks) return;
    const int i = a.p.chunk_row[c], start = a.p.row_ptr[i], T0 = a.p.chunk;
    if (start == c * T0 || start / T0 != c - 1) return;
    const int pieces = (a.p.row_ptr[i + 1] - 1) / T0 - (c - 1) + 1;
    const int groups = (64 / G) >> a.bundle_log, t = lane % G, slot = lane / G, group = slot >> a.bundle_log;
    const int head = ((int)blockIdx.y << a.bundle_log) + (slot & ((1 << a.bundle_log) - 1)), h = head < n_heads ? head : n_heads - 1;
    constexpr int W = MODE == kJoinTwo ? 2 * G * VEC : G * VEC;
    Share<T, VEC, G> s1, s2;
    s1.zero();
    s2.zero();
    float m = -INFINITY, l = 0.f;
    auto join = [&](float om, float ol, const Share<T, VEC, G> &o) {
        const float top = fmaxf(m, om), base = top > -INFINITY ? top : 0.f, f = exp_neg(m - base), fo = exp_neg(om - base);
        m = top;
        l = l * f + ol * fo;
        s1.scale(f);
        s1.add(fo, o);
    };
    for (int k = group; k < pieces; k += groups) {
        const size_t at = piece_at(c - 1 + k, k > 0, n_heads, h);
        Share<T, VEC, G> x;
        x.get(a.piece + at * W, t);
        if (MODE == kJoinForward) {
            const float2 ml = a.piece_ml[at];
            join(ml.x, ml.y, x);
        } else {
            s1.add(1.f, x);
            if (MODE == kJoinTwo) {
                x.get(a.piece + at * W + G * VEC, t);
                s2.add(1.f, x);
            }
        }
    }
    for (int dist = G << a.bundle_log; dist < 64; dist <<= 1) {
        Share<T, VEC, G> x;
#pragma unroll
        for (int k = 0; k < VEC; ++k) x.v[k] = __shfl_xor(s1.v[k], dist, 64);
        if (MODE == kJoinForward) join(__shfl_xor(m, dist, 64), __shfl_xor(l, dist, 64), x);
        else {
            s1.add(1.f, x);
            if (MODE == kJoinTwo) {
#pragma unroll
                for (int k = 0; k < VEC; ++k) x.v[k] = __shfl_xor(s2.v[k], dist, 64);
                s2.add(1.f, x);
            }
        }
    }
    if (group != 0 || head >= n_heads) return;
    if (MODE == kJoinForward) {
        s1.store(static_cast<T *>(a.O1) + (long long)i * a.ldo1 + (size_t)h * a.dv, t, a.dv, l == 0.f ? 0.f : a.key.keep_scale / l);
        if (t == 0) a.stats[(size_t)i * n_heads + h] = make_float2(m, logf(l));
    } else {
        s1.store(static_cast<T *>(a.O1) + (long long)i * a.ldo1 + (size_t)h * a.d, t, a.d, 1.f);
        if (MODE == kJoinTwo) s2.store(static_cast<T *>(a.O2) + (long long)i * a.ldo2 + (size_t)h * a.dv, t, a.dv, 1.f);
    }
}

// ------------------------------------------------------------------------------------------------------------------ preparation

// chunk_row[c] = row of entry c * chunk, of up to two patterns; and the buckets in the order of the transposed pattern
struct PrepArgs {
    struct { const int32_t *row_ptr; int32_t *chunk_row; int n_rows, chunk, n_chunks, block0; } plan[2];
    int n_plans, scatter0;
    const uint8_t *bucket;
    const int32_t *t_pos;
    uint8_t *out;
    int nnz;
};
__global__ __launch_bounds__(kThreads) void k_attention_prep(PrepArgs a) {
    if ((int)blockIdx.x >= a.scatter0) {
        const long long k = (long long)((int)blockIdx.x - a.scatter0) * kThreads + threadIdx.x;
        if (k < a.nnz) a.out[a.t_pos[k]] = a.bucket[k];
        return;
    }
    const auto &p = a.n_plans > 1 && (int)blockIdx.x >= a.plan[1].block0 ? a.plan[1] : a.plan[0];
    const int c = ((int)blockIdx.x - p.block0) * kThreads + (int)threadIdx.x;
    if (c >= p.n_chunks) return;
    const int e = c * p.chunk;
    int lo = 0, hi = p.n_rows;     // row_ptr[lo] <= e < row_ptr[hi]
    while (hi - lo > 1) {
        const int mid = lo + ((hi - lo) >> 1);
        if (p.row_ptr[mid] <= e) lo = mid; else hi = mid;
    }
    p.chunk_row[c] = lo;
}

// ------------------------------------------------------------------------------------------------------------------ host side

// Lanes of a head and elements a lane, from the wider of a head's key and value.
struct Shape { int vec, lanes; };
Shape shape_of(int d, int dv) {
    const int w = d > dv ? d : dv;
    return w <= 16 ? Shape{4, 4} : w <= 32 ? Shape{8, 4} : w <= 64 ? Shape{8, 8} : w <= 128 ? Shape{8, 16} : Shape{8, 32};
}
// Heads of a bundle: as many as fill a 128-byte line, and all query heads of a key head
int bundle_log_of(const Shape &s, int n_heads, int together, int bytes) {
    int log = 0;
    while ((s.lanes << (log + 1)) <= 64 && (1 << log) < n_heads && ((bytes << log) < 128 || (1 << log) < together)) ++log;
    return log;
}
int chunk_of(int64_t nnz, int bundles, int groups) {
    int t = 256;
    while (t > 16 && nnz / t * bundles / groups < 16384) t >>= 1;
    return t;
}

struct Layout {
    Shape shape;
    int bundle_log, bundles, groups, chunk, n_chunks, blocks;
    Layout(int64_t nnz, int n_heads, int together, int d, int dv, int elem) {
        shape = shape_of(d, dv);
        bundle_log = bundle_log_of(shape, n_heads, together, (d > dv ? d : dv) * elem);
        bundles = (n_heads + (1 << bundle_log) - 1) >> bundle_log;
        groups = (64 / shape.lanes) >> bundle_log;
        chunk = chunk_of(nnz, bundles, groups);
        n_chunks = (int)((nnz + chunk - 1) / chunk);
        blocks = (n_chunks + kWaves * groups - 1) / (kWaves * groups);
    }
    size_t rows_bytes() const { return align_up((size_t)n_chunks * sizeof(int32_t), 256); }
    size_t piece_bytes(int n_heads, int sums) const { return align_up((size_t)n_chunks * 2 * n_heads * shape.vec * shape.lanes * sums * sizeof(float), 256); }
    size_t ml_bytes(int n_heads) const { return align_up((size_t)n_chunks * 2 * n_heads * sizeof(float2), 256); }
};

struct Room {   // what the backward carves its scratch into
    Layout rows, cols;
    size_t bucket, stats, piece, bias;
    Room(const AttentionCall &c)
        : rows(c.A->nnz, c.heads, c.heads / c.kv_heads, c.d, c.dv, c.elem), cols(c.A->nnz, c.kv_heads, 1, c.d, c.dv, c.elem) {
        bucket = c.n_buckets > 0 ? align_up((size_t)c.A->nnz, 256) : 0;
        stats = align_up((size_t)c.A->n_rows * c.heads * sizeof(float4), 256);
        const size_t p1 = rows.piece_bytes(c.heads, 1), p2 = cols.piece_bytes(c.kv_heads, 2);   // one after the other
        piece = p1 > p2 ? p1 : p2;
        bias = c.n_buckets > 0 && c.dbias ? align_up((size_t)rows.blocks * c.heads * c.n_buckets * sizeof(float), 256) : 0;
    }
    size_t bytes() const { return rows.rows_bytes() + cols.rows_bytes() + bucket + stats + piece + bias; }
};

AttnArgs args_of(const AttentionCall &c) {
    AttnArgs a = {};
    a.Q = c.Q; a.K = c.K; a.V = c.V; a.Y = c.Y; a.dY = c.dY;
    a.ldq = c.ldq; a.ldk = c.ldk; a.ldv = c.ldv; a.ldy = c.ldy; a.lddy = c.lddy;
    a.stats = c.stats;
    a.heads = c.heads; a.kv_heads = c.kv_heads; a.ratio = c.heads / c.kv_heads; a.d = c.d; a.dv = c.dv;
    a.scale = c.scale; a.cap = c.cap; a.inv_cap = c.cap > 0.f ? 1.f / c.cap : 0.f;
    a.bias = c.n_buckets > 0 ? c.bias : nullptr;
    a.n_buckets = c.n_buckets;
    a.key = {(unsigned)c.seed, (unsigned)(c.seed >> 32), c.offset, c.offset_dev, drop_threshold(c.p), (float)(1.0 / (1.0 - c.p))};
    return a;
}

WalkPattern pattern_of(const sensei_csr &A, const Layout &l, const uint8_t *bucket, const int32_t *chunk_row) {
    return {A.row_ptr, A.col_idx, bucket, chunk_row, A.n_rows, (int)A.nnz, l.chunk, l.n_chunks};
}

template <class T, int VEC, int G, int MODE> hipError_t join_and_fill(const AttnArgs &a, const Layout &l, int n_heads, hipStream_t s) {
    const int join_blocks = l.n_chunks > 1 ? (l.n_chunks - 1 + kWaves - 1) / kWaves : 0, fill = (int)((a.p.n_rows + 64ll * kWaves - 1) / (64 * kWaves));
    if (join_blocks + fill == 0) return hipSuccess;
    hipLaunchKernelGGL((k_attention_join<T, VEC, G, MODE>), dim3(join_blocks + fill, l.bundles), dim3(kThreads), 0, s, a, n_heads, join_blocks);
    return hipGetLastError();
}

template <class T, int VEC, int G> hipError_t forward_shape(AttnArgs a, const Layout &l, hipStream_t s) {
    if (a.p.nnz > 0) {
        const size_t lds = a.bias ? (size_t)(a.n_buckets << l.bundle_log) * sizeof(float) : 0;
        hipLaunchKernelGGL((k_attention<T, VEC, G>), dim3(l.blocks, l.bundles), dim3(kThreads), lds, s, a);
    }
    return join_and_fill<T, VEC, G, kJoinForward>(a, l, a.heads, s);
}

template <class T, int VEC, int G> hipError_t backward_shape(const AttentionCall &c, AttnArgs a, const Room &room, const WalkPattern &pr, const WalkPattern &pc, hipStream_t s) {
    hipError_t e;
    a.p = pr;
    a.O1 = c.dQ; a.ldo1 = c.lddq;
    a.bundle_log = room.rows.bundle_log;
    if (pr.nnz > 0) {
        const size_t table = (size_t)(((a.n_buckets << a.bundle_log) + 3) / 4 * 4);
        const size_t lds = a.bias ? (table + (a.bias_part ? (size_t)kWaves * (64 / G) * a.n_buckets : 0)) * sizeof(float) : 0;
        hipLaunchKernelGGL((k_attention_back_rows<T, VEC, G>), dim3(room.rows.blocks, room.rows.bundles), dim3(kThreads), lds, s, a);
        if (a.bias_part) {
            const int n = a.heads * a.n_buckets;
            hipLaunchKernelGGL(k_attention_bias, dim3((n + 15) / 16), dim3(1024), 0, s, a.bias_part, room.rows.blocks, n, c.dbias);
        }
    }
    if ((e = join_and_fill<T, VEC, G, kJoinOne>(a, room.rows, a.heads, s)) != hipSuccess) return e;
    a.p = pc;
    a.O1 = c.dK; a.ldo1 = c.lddk;
    a.O2 = c.dV; a.ldo2 = c.lddv;
    a.bundle_log = room.cols.bundle_log;
    if (pc.nnz > 0) {
        const size_t lds = a.bias ? (size_t)(a.n_buckets * a.ratio << a.bundle_log) * sizeof(float) : 0;
        hipLaunchKernelGGL((k_attention_back_cols<T, VEC, G>), dim3(room.cols.blocks, room.cols.bundles), dim3(kThreads), lds, s, a);
    }
    return join_and_fill<T, VEC, G, kJoinTwo>(a, room.cols, a.kv_heads, s);
}

#define SENSEI_BY_SHAPE(T, shape, CALL)                                                              \
    (shape.vec == 4 ? CALL(T, 4, 4) : shape.lanes == 4 ? CALL(T, 8, 4) : shape.lanes == 8 ? CALL(T, 8, 8) \
     : shape.lanes == 16 ? CALL(T, 8, 16) : CALL(T, 8, 32))
#define SENSEI_BY_TYPE(type, shape, CALL) \
    (type == SENSEI_F32 ? SENSEI_BY_SHAPE(float, shape, CALL) : type == SENSEI_BF16 ? SENSEI_BY_SHAPE(Bf16, shape, CALL) : SENSEI_BY_SHAPE(F16, shape, CALL))

}  // namespace

size_t attention_ws_bytes(const AttentionCall &c) {
    const Layout l(c.A->nnz, c.heads, c.heads / c.kv_heads, c.d, c.dv, c.elem);
    return l.rows_bytes() + l.piece_bytes(c.heads, 1) + l.ml_bytes(c.heads) + 256;
}

hipError_t launch_attention(const AttentionCall &c, char *ws, hipStream_t s) {
    if (c.A->n_rows <= 0) return hipSuccess;
    const Layout l(c.A->nnz, c.heads, c.heads / c.kv_heads, c.d, c.dv, c.elem);
    AttnArgs a = args_of(c);
    int32_t *chunk_row = reinterpret_cast<int32_t *>(ws);
    a.p = pattern_of(*c.A, l, a.bias ? c.bucket : nullptr, chunk_row);
    a.piece = reinterpret_cast<float *>(ws + l.rows_bytes());
    a.piece_ml = reinterpret_cast<float2 *>(ws + l.rows_bytes() + l.piece_bytes(c.heads, 1));
    a.O1 = c.out; a.ldo1 = c.ldo;
    a.bundle_log = l.bundle_log;
    if (c.A->nnz > 0) {
        PrepArgs p = {};
        p.n_plans = 1;
        p.plan[0] = {c.A->row_ptr, chunk_row, c.A->n_rows, l.chunk, l.n_chunks, 0};
        p.scatter0 = (l.n_chunks + kThreads - 1) / kThreads;
        hipLaunchKernelGGL(k_attention_prep, dim3(p.scatter0), dim3(kThreads), 0, s, p);
    }
#define SENSEI_CALL(T, V, G) forward_shape<T, V, G>(a, l, s)
    return SENSEI_BY_TYPE(c.type, l.shape, SENSEI_CALL);
#undef SENSEI_CALL
}

size_t attention_backward_ws_bytes(const AttentionCall &c) { return Room(c).bytes() + 256; }

hipError_t launch_attention_backward(const AttentionCall &c, char *ws, hipStream_t s) {
    const Room room(c);
    AttnArgs a = args_of(c);
    char *at = ws;
    auto take = [&](size_t n) { char *p = at; at += n; return p; };
    int32_t *rows_r = reinterpret_cast<int32_t *>(take(room.rows.rows_bytes())), *rows_c = reinterpret_cast<int32_t *>(take(room.cols.rows_bytes()));
    uint8_t *bucket_t = reinterpret_cast<uint8_t *>(take(room.bucket));
    a.row_stats = reinterpret_cast<float4 *>(take(room.stats));
    a.piece = reinterpret_cast<float *>(take(room.piece));
    a.bias_part = a.bias && c.dbias ? reinterpret_cast<float *>(take(room.bias)) : nullptr;
    const WalkPattern pr = pattern_of(*c.A, room.rows, a.bias ? c.bucket : nullptr, rows_r), pc = pattern_of(*c.At, room.cols, a.bias ? bucket_t : nullptr, rows_c);
    if (c.A->nnz > 0) {
        PrepArgs p = {};
        p.n_plans = 2;
        p.plan[0] = {c.A->row_ptr, rows_r, c.A->n_rows, room.rows.chunk, room.rows.n_chunks, 0};
        p.plan[1] = {c.At->row_ptr, rows_c, c.At->n_rows, room.cols.chunk, room.cols.n_chunks, (room.rows.n_chunks + kThreads - 1) / kThreads};
        p.scatter0 = p.plan[1].block0 + (room.cols.n_chunks + kThreads - 1) / kThreads;
        p.bucket = c.bucket; p.t_pos = c.t_pos; p.out = bucket_t; p.nnz = (int)c.A->nnz;
        hipLaunchKernelGGL(k_attention_prep, dim3(p.scatter0 + (a.bias ? (p.nnz + kThreads - 1) / kThreads : 0)), dim3(kThreads), 0, s, p);
    } else if (a.bias_part) {
        const hipError_t e = launch_zero_matrix(c.dbias, 1, c.heads * c.n_buckets, c.heads * c.n_buckets, false, s);
        if (e != hipSuccess) return e;
    }
#define SENSEI_CALL(T, V, G) backward_shape<T, V, G>(c, a, room, pr, pc, s)
    return SENSEI_BY_TYPE(c.type, room.rows.shape, SENSEI_CALL);
#undef SENSEI_CALL
}

}  // namespace sensei
