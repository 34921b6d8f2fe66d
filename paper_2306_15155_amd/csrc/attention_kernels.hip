// Multi-head attention over the stored entries of a pattern, forward and backward: scores scale <q_i, k_j>, optionally capped by a tanh and
// biased by the entry's bucket, softmax over a row's entries, weights optionally dropped; key and value heads may be shared by query heads.
//
// Nothing is stored per entry.  The forward walk keeps a running maximum m, sum l and weighted sum of values per row; the backward forms the
// weights again from the rows' (m, log l):
//     x = bias + cap tanh(scale <q, k> / cap),  p = exp(x - m - log l),  dt = p (keep/(1-p_drop) <dy, v> - D),  D_i = <dy_i, y_i>,
//     dq_i = sum_j ds k_j,  dk_j = sum_i ds q_i,  dv_j = sum_i p keep/(1-p_drop) dy_i,  dbias[h, b] = sum dt,  ds = dt (1 - tanh^2) scale
// as two walks, one over the rows (dq) and one over the transposed pattern (dk, dv, dbias), so that no sum needs an atomic across wavefronts.
//
// D comes from Y.  Where Y was rounded to 16 bits, the walk over the rows sums what the rounding took from D along (delta = sum dt, 0 with the whole D)
// and takes it out of dq at the row's end; dbias is summed by the walk over the columns, which has the whole D.  (Without: dbias 1.9e-3 of
// its size off, the other gradients 10 % further than their own rounding.)
//
// What bounds these walks is the gathering of k and v (q and dy) rows from the caches, and behind it the instructions around four operations an
// element.  A head's vector is spread over as few lanes as hold 32 bytes of it each (G: one lane for 16 elements of 16 bits); a group of lanes takes
// the same entry for a few neighbouring heads (a bundle), so that a gather takes whole 128-byte lines and shared key heads are read
// once; and every group walks a chunk of consecutive entries by itself, four at a time (a batch).  The four dot products are summed so that
// the lanes of a head share them out: cap, bias, mask and exponential are worked out once an entry and head, and the weights are handed
// round by moves within a quad of lanes; so are the generator's words, of which a call has four heads'.  Rows that cross chunks leave a
// piece per chunk in scratch, joined by a second kernel in chunk order: results do not depend on scheduling.
//
// Walks, us, and what they gather a second (every entry's vectors counted):             forward       over rows     over columns
//     100,000 nodes of 21, 4 heads of 32, fp32, cap, bias, drop                         262, 8.2 TB/s 259, 8.3 TB/s 354, 6.5 TB/s
//     290,000 nodes in graphs of 10 to 60, 8 heads of 16, bf16, bias, drop              515, 12 TB/s  654, 9.2 TB/s 800, 9.4 TB/s
//     233,000 nodes of 87, 8 query on 2 key heads of 64, bf16, cap                      1,650, 6.3 TB/s
// In fp32 that is what lines from L2s and the Infinity Cache come at; in 16 bits half as many lines carry as many operations, and two thirds of
// the time are vector instructions at two or three wavefronts a SIMD (132 to 250 registers).
#include <algorithm>

#include "element_types.h"
#include "sensei_internal.h"

namespace sensei {

namespace {

constexpr int kThreads = 256, kBatch = 4;
__device__ __forceinline__ int waves() { return (int)(blockDim.x >> 6); }

struct WalkPattern {
    const int32_t *row_ptr, *col;
    const uint8_t *bucket;        // in this pattern's order, null: none
    int32_t *chunk_row;           // row of the first entry of every chunk, written by the walk
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
    float2 *piece_ml;             // (m, l) of a row piece; backward over the rows: (delta, -)
    float *bias_part;             // a block's share of dbias, null: not asked for
};

// ------------------------------------------------------------------------------------------------------------------ lanes of a head

// What a head's lanes work out for the four entries of a batch: lane t has entry t % 4, with two lanes a head entries t and t + 2, a lone lane all.
template <int G> struct Own {
    static constexpr int N = G >= 4 ? 1 : 4 / G, SHARERS = G < 4 ? G : 4;
    __device__ __forceinline__ static int entry(int t, int o) { return G >= 4 ? t & 3 : t + G * o; }
    __device__ __forceinline__ static int of(int t, int o, const int (&x)[kBatch]) {
        if (G == 1) return x[o];
        if (G == 2) {
            const int even = x[2 * o], odd = x[2 * o + 1];
            return t ? odd : even;
        }
        const int x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3], lo = t & 1 ? x1 : x0, hi = t & 1 ? x3 : x2;
        return t & 2 ? hi : lo;
    }
    // sums over the head's lanes of four numbers, each to the lane whose it is
    __device__ __forceinline__ static void sums(const float (&s)[kBatch], int t, float (&out)[N]) {
        if constexpr (G == 1) {
#pragma unroll
            for (int o = 0; o < 4; ++o) out[o] = s[o];
        } else if constexpr (G == 2) {
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const float even = s[2 * o], odd = s[2 * o + 1];
                out[o] = (t ? odd : even) + dpp<0xB1>(t ? even : odd);
            }
        } else {
            float a0 = s[0], a1 = s[1], a2 = s[2], a3 = s[3];
            if (G == 8) {
                a0 += dpp<0x141>(a0); a1 += dpp<0x141>(a1); a2 += dpp<0x141>(a2); a3 += dpp<0x141>(a3);
            }
            const bool odd = t & 1, high = t & 2;
            float lo = odd ? a1 : a0, hi = odd ? a3 : a2;
            lo += dpp<0xB1>(odd ? a0 : a1);
            hi += dpp<0xB1>(odd ? a2 : a3);
            float x = high ? hi : lo;
            x += dpp<0x4E>(high ? lo : hi);
            if (G >= 16) {      // quads of a row of sixteen lanes, turned by one and by two
                x += dpp<0x124>(x);
                x += dpp<0x128>(x);
            }
            if (G >= 32) x += from_16_away(x);
            out[0] = x;
        }
    }
    // entry U's number, in all lanes of the head
    template <int U, class X> __device__ __forceinline__ static X get(const X (&own)[N]) {
        if constexpr (G == 1) return own[U];
        else if constexpr (G == 2) return dpp<U & 1 ? 0xF5 : 0xA0>(own[U / 2]);
        else return dpp<U * 0x55>(own[0]);
    }
    // the largest of the four, the sum of what every lane has for its own
    __device__ __forceinline__ static float max(const float (&own)[N]) {
        float x = own[0];
#pragma unroll
        for (int o = 1; o < N; ++o) x = fmaxf(x, own[o]);
        if (G >= 2) x = fmaxf(x, dpp<0xB1>(x));
        if (G >= 4) x = fmaxf(x, dpp<0x4E>(x));
        return x;
    }
    __device__ __forceinline__ static float sum(float x) { return sum_over<SHARERS>(x); }
};

// The number as it is, but worked on here: what follows from it is not kept from outside a loop in registers that are short there.
__device__ __forceinline__ int here(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// A lane's share of a head's vector of d elements: PIECES pieces of PER, piece r from element at(r) = (r G + t) PER on, so that the lanes of a head read
// side by side.  Where the vector ends inside a piece the lane reads the last PER elements instead and leaves those before at(r) to the lane
// whose they are: every gather is a full piece within its row.  GENERIC (vectors shorter than a piece, matrices past 32-bit offsets): elements one by
// one where a piece is not whole, 64-bit offsets.
template <class T, int VEC, int G, bool GENERIC> struct Lanes {
    static constexpr int PER = kPerPiece<T>, PIECES = VEC / PER;
    __device__ __forceinline__ static int at(int r, int t) { return (r * G + t) * PER; }
    __device__ __forceinline__ static int from(int r, int t, int d) { return GENERIC || at(r, t) + PER <= d ? at(r, t) : d - PER; }
};

// gathered elements as they came: packed pairs in 16 bits
template <class T, int VEC> struct Gathered {
    static constexpr int WORDS = VEC * (int)sizeof(T) / 4;
    unsigned w[WORDS];
    __device__ __forceinline__ void mask(int ones) {
#pragma unroll
        for (int k = 0; k < WORDS; ++k) w[k] &= (unsigned)ones;
    }
    __device__ __forceinline__ float get(int k) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
        else return to_f32(T{(unsigned short)(k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xFFFFu)});
    }
};
template <class T, int VEC> __device__ __forceinline__ float dot(const Gathered<T, VEC> &a, const Gathered<T, VEC> &b) {
    float s = 0.f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) s = fmaf(a.get(k), b.get(k), s);
    } else {
#pragma unroll
        for (int k = 0; k < VEC / 2; ++k) {   // products of 16-bit numbers are exact in fp32, sums are held in it
            if constexpr (__is_same(T, Bf16)) {
                typedef __bf16 Pair __attribute__((ext_vector_type(2)));
                s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Pair, a.w[k]), __builtin_bit_cast(Pair, b.w[k]), s, false);
            } else {
                typedef _Float16 Pair __attribute__((ext_vector_type(2)));
                s = __builtin_amdgcn_fdot2(__builtin_bit_cast(Pair, a.w[k]), __builtin_bit_cast(Pair, b.w[k]), s, false);
            }
        }
    }
    return s;
}

// where a lane's pieces of a head lie in a matrix: for gathers by row number
template <class T, int VEC, int G, bool GENERIC> struct Source {
    using L = Lanes<T, VEC, G, GENERIC>;
    const char *base;            // the same in every lane
    unsigned offset[L::PIECES];  // bytes
    unsigned ld24;
    long long ld;
    int t, d;
    __device__ __forceinline__ Source(const void *p, long long ld_, int first, int d_, int t_) : base(static_cast<const char *>(p)), t(t_), d(d_) {
        ld = ld_ * (long long)sizeof(T);
        ld24 = (unsigned)ld;
#pragma unroll
        for (int r = 0; r < L::PIECES; ++r) offset[r] = (unsigned)(first + L::from(r, t, d)) * (unsigned)sizeof(T);
    }
    // `more`: bytes that are the same in every lane
    __device__ __forceinline__ Gathered<T, VEC> row(int i, long long more = 0) const {
        using Raw = typename Piece<T, L::PER>::Raw;
        Gathered<T, VEC> x;
#pragma unroll
        for (int r = 0; r < L::PIECES; ++r) {
            U32x4 raw;
            if constexpr (!GENERIC) raw = *reinterpret_cast<const Raw *>((base + more) + (__umul24((unsigned)i, ld24) + offset[r]));
            else {
                const T *p = reinterpret_cast<const T *>(base + more + (long long)i * ld + offset[r]);
                const int left = d - L::at(r, t);
                Piece<T, L::PER> y;
                if (left >= L::PER) y = Piece<T, L::PER>::load(p);
                else {
#pragma unroll
                    for (int k = 0; k < L::PER; ++k) {
                        y.x[k] = T{};
                        if (k < left) y.x[k] = p[k];
                    }
                }
                raw = __builtin_bit_cast(U32x4, y);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) x.w[4 * r + k] = raw[k];
        }
        return x;
    }
    // 0 in the place of elements that are not this lane's own
    __device__ __forceinline__ void keep_own(Gathered<T, VEC> &x) const {
        if (GENERIC || d == VEC * G) return;
        const int t = here(this->t);
#pragma unroll
        for (int r = 0; r < L::PIECES; ++r) {
            const int skip = L::at(r, t) - L::from(r, t, d);   // of the piece's elements; a lane behind the end has none
#pragma unroll
            for (int k = 0; k < L::PER; ++k) {
                unsigned &w = x.w[(r * L::PER + k) * (int)sizeof(T) / 4];
                if (k < skip) w &= sizeof(T) == 4 ? 0u : k & 1 ? 0xFFFFu : 0xFFFF0000u;
            }
        }
    }
    // row i with nothing but own elements: one side of every product
    __device__ __forceinline__ Gathered<T, VEC> own(int i) const {
        Gathered<T, VEC> x = row(i);
        keep_own(x);
        return x;
    }
};

// sums of a lane's share
template <class T, int VEC, int G, bool GENERIC> struct Sums {
    using L = Lanes<T, VEC, G, GENERIC>;
    float v[VEC];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] = 0.f;
    }
    __device__ __forceinline__ void add(float w, const Gathered<T, VEC> &x) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] = fmaf(w, x.get(k), v[k]);
    }
    // nothing of x where `ones` is 0: a masked entry has no share, whatever its key and value hold
    __device__ __forceinline__ void add(float w, Gathered<T, VEC> x, int ones) {
        x.mask(ones);
        add(w, x);
    }
    __device__ __forceinline__ void add(float w, const Sums &x) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] = fmaf(w, x.v[k], v[k]);
    }
    __device__ __forceinline__ void scale(float w) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] *= w;
    }
    __device__ __forceinline__ void store(T *p, int t_, int d, float by) const {
        const int t = here(t_);
#pragma unroll
        for (int r = 0; r < L::PIECES; ++r) {
            const int first = L::at(r, t), from = L::from(r, t, d);
            Piece<T, L::PER> x;
#pragma unroll
            for (int k = 0; k < L::PER; ++k) x.x[k] = from_f32<T>(v[r * L::PER + k] * by);
            if (from == first && first + L::PER <= d) x.store(p + first);
            else {
#pragma unroll
                for (int k = 0; k < L::PER; ++k)
                    if (from + k >= first && from + k < d) p[from + k] = x.x[k];
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
};

// ------------------------------------------------------------------------------------------------------------------ walk of a chunk

// A group's place in its chunk: the row it is in, and the columns (and buckets) of the next four entries, fetched a batch ahead.
struct Walk {
    int e, end, i, row_end;
    int next_end;            // where the row behind this one ends: fetched while this one is walked
    bool goes_on;            // the row began in an earlier chunk
    int col[kBatch];
    unsigned bucket;         // four of eight bits
    __device__ __forceinline__ void fetch(const WalkPattern &p, int at) {
        if (at <= p.nnz - kBatch) {
            typedef U32x4 Four __attribute__((aligned(4)));
            const U32x4 x = *reinterpret_cast<const Four *>(p.col + at);
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
    __device__ __forceinline__ void look_ahead(const WalkPattern &p) { next_end = p.row_ptr[i < p.n_rows - 2 ? i + 2 : p.n_rows]; }
    // The row of the chunk's first entry is found by the group's lanes together (lane `j` of `lanes`), which narrow the rows down (4 lanes + 1)-fold a
    // look: a launch that did so ahead of the walk cost 9 us.
    __device__ __forceinline__ void begin(const WalkPattern &p, int chunk, int j, int lanes) {
        e = chunk * p.chunk;
        end = p.nnz - e < p.chunk ? p.nnz : e + p.chunk;
        fetch(p, e);
        int lo = 0, hi = p.n_rows;     // row_ptr[lo] <= e < row_ptr[hi]
        const unsigned long long mine = (lanes < 64 ? (1ull << lanes) - 1 : ~0ull) << ((int)(threadIdx.x & 63) - j);
        while (hi - lo > 1) {
            const int step = (hi - lo - 1) / (4 * lanes + 1) + 1;
            int below = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const long long at = lo + (long long)step * (4 * j + q + 1);
                below += __popcll(__ballot(at < hi && p.row_ptr[at < hi ? at : lo] <= e) & mine);
            }
            lo += step * below;
            if (step < hi - lo) hi = lo + step;
        }
        i = lo;
        row_end = p.row_ptr[i + 1];
        look_ahead(p);
        goes_on = p.row_ptr[i] < e;
        if (j == 0 && blockIdx.y == 0) p.chunk_row[chunk] = i;   // for the pass that joins the pieces
    }
    __device__ __forceinline__ int count() const {
        const int n = (row_end < end ? row_end : end) - e;
        return n < kBatch ? n : kBatch;
    }
    // columns of the batch: behind its n entries the first one again, which is there to be read
    __device__ __forceinline__ void columns(int n, int (&c)[kBatch]) const {
        c[0] = col[0];
#pragma unroll
        for (int u = 1; u < kBatch; ++u) c[u] = u < n ? col[u] : col[0];
    }
    __device__ __forceinline__ int bucket_of(int u, int n_buckets) const {
        const int b = (int)(bucket >> (8 * u) & 255u);
        return b < n_buckets ? b : n_buckets - 1;
    }
    __device__ __forceinline__ bool row_done() const { return e == row_end || e == end; }
    // the row of entry e, which lies behind row i: the next one, or across a run of empty rows by doubling steps and halving
    __device__ __forceinline__ void next_row(const WalkPattern &p) {
        i = i + 1;
        row_end = next_end;
        if (row_end <= e) {
            int lo = i, hi = i, step = 1;
            do {
                lo = hi;
                hi = step < p.n_rows - hi ? hi + step : p.n_rows - 1;
                step = step < 1 << 29 ? 2 * step : step;
            } while (p.row_ptr[hi + 1] <= e);
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.row_ptr[mid + 1] <= e) lo = mid; else hi = mid;
            }
            i = hi;
            row_end = p.row_ptr[hi + 1];
        }
        look_ahead(p);
        goes_on = false;
    }
};

// Where a lane works: t of the G lanes of head h, group `chunk` of the walk.  The first workgroups take the last chunks: where node numbers follow
// degrees from the highest down (power-law patterns mostly do), those are the chunks of many short rows, which take longest and would run on
// alone at the end (first / last chunks first, us: training steps, 100,000 nodes of 21 1,108 / 959, 97,000 of 11 994 / 893, forward, 233,000 of 87
// 1,965 / 1,733; uniform patterns alike, 2,210 / 2,196, 614 / 611).  The lanes of a bundle's heads that there are not work along on the last
// head (others want what they work out) and store nothing.
template <int G> struct Place {
    int t, slot, in_bundle, h, chunk;
    int in_group, group_lanes;
    bool live, head_live;
    __device__ __forceinline__ Place(int n_heads, int n_chunks, int bundle_log) {
        const int lane = threadIdx.x & 63, groups = (64 / G) >> bundle_log;
        t = lane % G;
        slot = lane / G;
        group_lanes = G << bundle_log;
        in_group = lane & (group_lanes - 1);
        in_bundle = slot & ((1 << bundle_log) - 1);
        const int head = ((int)blockIdx.y << bundle_log) + in_bundle;
        chunk = ((int)(gridDim.x - 1 - blockIdx.x) * waves() + (int)(threadIdx.x >> 6)) * groups + (slot >> bundle_log);
        live = chunk < n_chunks;
        head_live = head < n_heads;
        h = head_live ? head : n_heads - 1;
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

// a score and what it does to the gradient
struct Score { float x, slope; };
__device__ __forceinline__ Score score_of(const AttnArgs &a, float dot) {
    const float x = dot * a.scale;
    if (!(a.cap > 0.f)) return {x, 1.f};
    const Tanh th = tanh_of(x * a.inv_cap);
    return {a.cap * th.value, th.slope};
}

// Which weights of the lane's own entries stay for query head h: generator at counter (column, row, 2^31 + h / 4, offset), word h % 4.  COLS: the entries
// lie in one column, else in one row.  A lane calls it for its own entries; where lanes of one quad work on the same entries for heads of
// one call (bundles of neighbouring heads, fewer than four lanes a head), each calls it for other entries and hands round four bits.
// Bit r of keep: head h + r, of the R heads (of one call) that the lane works on.
template <int G, bool COLS, int R>
__device__ __forceinline__ void kept(const DropKey &key, unsigned offset, int fixed, const int (&other)[kBatch], int h, int t, int bundle_log, int (&keep)[Own<G>::N]) {
    using O = Own<G>;
    auto words = [&](int x) {
        return COLS ? philox((unsigned)fixed, (unsigned)x, 0x80000000u | (unsigned)(h >> 2), offset, key.k0, key.k1)
                    : philox((unsigned)x, (unsigned)fixed, 0x80000000u | (unsigned)(h >> 2), offset, key.k0, key.k1);
    };
    auto mine = [&](int x) {
        const Words w = words(x);
        const unsigned w0 = w.w[0], w1 = w.w[1], w2 = w.w[2], w3 = w.w[3], lo = h & 1 ? w1 : w0, hi = h & 1 ? w3 : w2;
        return (h & 2 ? hi : lo) >= key.threshold;
    };
    auto bits = [&](int x) {
        const Words w = words(x);
        return (w.w[0] >= key.threshold ? 1 : 0) | (w.w[1] >= key.threshold ? 2 : 0) | (w.w[2] >= key.threshold ? 4 : 0) | (w.w[3] >= key.threshold ? 8 : 0);
    };
    if constexpr (R > 1) {
#pragma unroll
        for (int o = 0; o < O::N; ++o) keep[o] = bits(O::of(t, o, other)) >> (h & 3);
        return;
    }
    if constexpr (G < 4) {
        const int z = threadIdx.x & 3;
        if ((G << bundle_log) >= 4) {
            const int b = bits(Own<4>::of(z, 0, other));
            if constexpr (G == 2) {
                keep[0] = dpp<0x44>(b) >> (h & 3) & 1;
                keep[1] = dpp<0xEE>(b) >> (h & 3) & 1;
            } else {
                keep[0] = dpp<0x00>(b) >> (h & 3) & 1;
                keep[1] = dpp<0x55>(b) >> (h & 3) & 1;
                keep[2] = dpp<0xAA>(b) >> (h & 3) & 1;
                keep[3] = dpp<0xFF>(b) >> (h & 3) & 1;
            }
            return;
        }
        if constexpr (G == 1) {
            if (bundle_log == 1) {
                const int b0 = bits(Own<2>::of(z & 1, 0, other)), b1 = bits(Own<2>::of(z & 1, 1, other));
                keep[0] = dpp<0xA0>(b0) >> (h & 3) & 1;
                keep[1] = dpp<0xF5>(b0) >> (h & 3) & 1;
                keep[2] = dpp<0xA0>(b1) >> (h & 3) & 1;
                keep[3] = dpp<0xF5>(b1) >> (h & 3) & 1;
                return;
            }
        }
    }
#pragma unroll
    for (int o = 0; o < O::N; ++o) keep[o] = mine(O::of(t, o, other)) ? 1 : 0;
}
__device__ __forceinline__ unsigned drop_offset(const DropKey &key) { return key.offset + (key.offset_dev ? *key.offset_dev : 0u); }

// slot of a row piece: first piece of a chunk when the row goes on from the chunk before, else its last
__device__ __forceinline__ size_t piece_at(int chunk, bool goes_on, int heads, int h) { return ((size_t)chunk * 2 + (goes_on ? 0 : 1)) * heads + h; }

// ------------------------------------------------------------------------------------------------------------------ forward

// for every entry of a batch
#define SENSEI_EACH(F) F(0) F(1) F(2) F(3)

// R: query heads of one key head that a lane takes together (R divides their number), from one gathering of the entry
template <class T, int VEC, int G, bool GENERIC, int R>
__global__ __launch_bounds__(kThreads) void k_attention(AttnArgs a) {
    using O = Own<G>;
    const Place<G> at(a.heads / R, a.p.n_chunks, a.bundle_log);
    if (!at.live) return;
    const int h = at.h * R, g = h / a.ratio, t = at.t;
    const Source<T, VEC, G, GENERIC> Q(a.Q, a.ldq, h * a.d, a.d, t), K(a.K, a.ldk, g * a.d, a.d, t), V(a.V, a.ldv, g * a.dv, a.dv, t);
    T *Y = static_cast<T *>(a.O1) + (size_t)h * a.dv;
    const float *bias = a.bias ? a.bias + h * a.n_buckets : nullptr;
    const unsigned offset = drop_offset(a.key);
    Walk w;
    w.begin(a.p, at.chunk, at.in_group, at.group_lanes);
    Gathered<T, VEC> q[R];
    Sums<T, VEC, G, GENERIC> acc[R];
    float m[R], l[R];                // l: the lane's own entries
#pragma unroll
    for (int r = 0; r < R; ++r) {
        acc[r].zero();
        m[r] = -INFINITY;
        l[r] = 0.f;
    }
    bool fresh = true;
    while (w.e < w.end) {
        const int n = w.count();
        int col[kBatch], bin[O::N];
        w.columns(n, col);
        float b[R][O::N];
#pragma unroll
        for (int o = 0; o < O::N; ++o) bin[o] = bias ? w.bucket_of(O::entry(t, o), a.n_buckets) : 0;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int o = 0; o < O::N; ++o) b[r][o] = bias ? bias[r * a.n_buckets + bin[o]] : 0.f;
        if (fresh) {     // a new row's loads go with those of its first entries: waited for where the row changes, they cost a round trip a row
#pragma unroll
            for (int r = 0; r < R; ++r) q[r] = Q.row(w.i, (long long)r * a.d * (int)sizeof(T));
            fresh = false;
        }
        Gathered<T, VEC> k[kBatch], v[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) k[u] = K.row(col[u]);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) v[u] = V.row(col[u]);
        if (w.e + n < w.end) w.fetch(a.p, w.e + n);
        int keep[O::N];              // bit r: head h + r
        if (a.key.threshold) kept<G, false, R>(a.key, offset, w.i, col, h, t, a.bundle_log, keep);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            Q.keep_own(q[r]);
            int use[O::N];               // all ones, or none
            bool masked = false;
#pragma unroll
            for (int o = 0; o < O::N; ++o) {
                const bool there = O::entry(t, o) < n, open = b[r][o] != -INFINITY;
                use[o] = there && open ? -1 : 0;
                masked = masked || (there && !open);
            }
            float s[kBatch], x[O::N];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) s[u] = dot(q[r], k[u]);
            O::sums(s, t, x);
#pragma unroll
            for (int o = 0; o < O::N; ++o) {
                const float y = score_of(a, x[o]).x + b[r][o];
                x[o] = use[o] ? y : -INFINITY;
            }
            const float top = fmaxf(m[r], O::max(x)), base = top > -INFINITY ? top : 0.f, f = exp_weight(m[r] - base);
            m[r] = top;
            l[r] *= f;
#pragma unroll
            for (int o = 0; o < O::N; ++o) {
                const float p = exp_weight(x[o] - base);
                l[r] += p;
                x[o] = a.key.threshold && !(keep[o] >> r & 1) ? 0.f : p;
            }
            acc[r].scale(f);
            if (bias && __any(masked)) {
#define SENSEI_ADD(U) acc[r].add(O::template get<U>(x), v[U], O::template get<U>(use));
                SENSEI_EACH(SENSEI_ADD)
#undef SENSEI_ADD
            } else {
#define SENSEI_ADD(U) acc[r].add(O::template get<U>(x), v[U]);
                SENSEI_EACH(SENSEI_ADD)
#undef SENSEI_ADD
            }
        }
        w.e += n;
        if (w.row_done()) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float sum = O::sum(l[r]);
                if (at.head_live) {
                    if (!w.goes_on && w.e == w.row_end) {
                        acc[r].store(Y + (long long)w.i * a.ldo1 + r * a.dv, t, a.dv, sum == 0.f ? 0.f : a.key.keep_scale / sum);
                        if (t == 0) a.stats[(size_t)w.i * a.heads + h + r] = make_float2(m[r], logf(sum));
                    } else {
                        const size_t at_piece = piece_at(at.chunk, w.goes_on, a.heads, h + r);
                        acc[r].put(a.piece + at_piece * (G * VEC), t);
                        if (t == 0) a.piece_ml[at_piece] = make_float2(m[r], sum);
                    }
                }
                acc[r].zero();
                m[r] = -INFINITY;
                l[r] = 0.f;
            }
            if (w.e < w.end) w.next_row(a.p);
            fresh = true;
        }
    }
}

// ------------------------------------------------------------------------------------------------------------------ backward, over the rows

template <class T, int VEC, int G, bool GENERIC, int R>
__global__ __launch_bounds__(kThreads) void k_attention_back_rows(AttnArgs a) {
    constexpr bool WHOLE_Y = sizeof(T) == 4;     // Y holds what D needs
    using O = Own<G>;
    const Place<G> at(a.heads / R, a.p.n_chunks, a.bundle_log);
    if (!at.live) return;
    const int h = at.h * R, g = h / a.ratio, t = at.t;
    const Source<T, VEC, G, GENERIC> Q(a.Q, a.ldq, h * a.d, a.d, t), K(a.K, a.ldk, g * a.d, a.d, t), V(a.V, a.ldv, g * a.dv, a.dv, t), dY(a.dY, a.lddy, h * a.dv, a.dv, t);
    T *dQ = static_cast<T *>(a.O1) + (size_t)h * a.d;
    const float *bias = a.bias ? a.bias + h * a.n_buckets : nullptr;
    const unsigned offset = drop_offset(a.key);
    Walk w;
    w.begin(a.p, at.chunk, at.in_group, at.group_lanes);
    Gathered<T, VEC> q[R], dy[R];
    Sums<T, VEC, G, GENERIC> acc[R], share[R];   // sum of ds k; of alpha slope scale k, which delta is taken out by
    float4 st[R];
    float delta[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        acc[r].zero();
        share[r].zero();
        delta[r] = 0.f;
    }
    bool fresh = true;
    while (w.e < w.end) {
        const int n = w.count();
        int col[kBatch], bin[O::N];
        w.columns(n, col);
        float b[R][O::N];
#pragma unroll
        for (int o = 0; o < O::N; ++o) bin[o] = bias ? w.bucket_of(O::entry(t, o), a.n_buckets) : 0;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int o = 0; o < O::N; ++o) b[r][o] = bias ? bias[r * a.n_buckets + bin[o]] : 0.f;
        if (fresh) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                q[r] = Q.row(w.i, (long long)r * a.d * (int)sizeof(T));
                dy[r] = dY.row(w.i, (long long)r * a.dv * (int)sizeof(T));
                st[r] = a.row_stats[(size_t)w.i * a.heads + h + r];
            }
            fresh = false;
        }
        Gathered<T, VEC> k[kBatch], v[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) k[u] = K.row(col[u]);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) v[u] = V.row(col[u]);
        if (w.e + n < w.end) w.fetch(a.p, w.e + n);
        int keep[O::N];
        if (a.key.threshold) kept<G, false, R>(a.key, offset, w.i, col, h, t, a.bundle_log, keep);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            Q.keep_own(q[r]);
            dY.keep_own(dy[r]);
            int use[O::N];
            bool masked = false;
#pragma unroll
            for (int o = 0; o < O::N; ++o) {
                const bool there = O::entry(t, o) < n, open = b[r][o] != -INFINITY;
                use[o] = there && open ? -1 : 0;
                masked = masked || (there && !open);
            }
            float s[kBatch], c[kBatch], x[O::N], dv[O::N], pb[O::N];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                s[u] = dot(q[r], k[u]);
                c[u] = dot(dy[r], v[u]);
            }
            O::sums(s, t, x);
            O::sums(c, t, dv);
#pragma unroll
            for (int o = 0; o < O::N; ++o) {
                const Score sc = score_of(a, x[o]);
                const float dp = a.key.threshold && !(keep[o] >> r & 1) ? 0.f : dv[o] * a.key.keep_scale;
                const float p = use[o] ? exp_weight((sc.x + b[r][o] - st[r].x) - st[r].y) : 0.f, dt = use[o] ? p * (dp - st[r].z) : 0.f, by = sc.slope * a.scale;
                delta[r] += dt;
                x[o] = dt * by;
                pb[o] = use[o] ? p * by : 0.f;
                x[o] = use[o] ? x[o] : 0.f;
            }
            if (bias && __any(masked)) {
#define SENSEI_ADD(U)                                                                                        \
    acc[r].add(O::template get<U>(x), k[U], O::template get<U>(use));                                        \
    if constexpr (!WHOLE_Y) share[r].add(O::template get<U>(pb), k[U], O::template get<U>(use));
                SENSEI_EACH(SENSEI_ADD)
#undef SENSEI_ADD
            } else {
#define SENSEI_ADD(U)                                                     \
    acc[r].add(O::template get<U>(x), k[U]);                              \
    if constexpr (!WHOLE_Y) share[r].add(O::template get<U>(pb), k[U]);
                SENSEI_EACH(SENSEI_ADD)
#undef SENSEI_ADD
            }
        }
        w.e += n;
        if (w.row_done()) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float off = WHOLE_Y ? 0.f : O::sum(delta[r]);
                if (at.head_live) {
                    if (!w.goes_on && w.e == w.row_end) {
                        if (!WHOLE_Y) {
                            acc[r].add(-off, share[r]);
                            if (t == 0) a.row_stats[(size_t)w.i * a.heads + h + r].z = st[r].z + off;
                        }
                        acc[r].store(dQ + (long long)w.i * a.ldo1 + r * a.d, t, a.d, 1.f);
                    } else {
                        const size_t at_piece = piece_at(at.chunk, w.goes_on, a.heads, h + r);
                        float *to = a.piece + at_piece * ((WHOLE_Y ? 1 : 2) * G * VEC);
                        acc[r].put(to, t);
                        if (!WHOLE_Y) {
                            share[r].put(to + G * VEC, t);
                            if (t == 0) a.piece_ml[at_piece] = make_float2(off, 0.f);
                        }
                    }
                }
                acc[r].zero();
                if (!WHOLE_Y) share[r].zero();
                delta[r] = 0.f;
            }
            if (w.e < w.end) w.next_row(a.p);
            fresh = true;
        }
    }
}

// ------------------------------------------------------------------------------------------------------------------ backward, over the columns

// The walk goes over the transposed pattern: its rows are the columns j, its entries the rows i that attend to them.  A lane stays with one key
// head and takes that head's query heads one after the other.  dbias is summed in LDS, in a table of their own for every head of every
// group, so that the sums have one order.
template <class T, int VEC, int G, bool GENERIC>
__global__ __launch_bounds__(kThreads) void k_attention_back_cols(AttnArgs a) {
    extern __shared__ float tables[];
    using O = Own<G>;
    const Place<G> at(a.kv_heads, a.p.n_chunks, a.bundle_log);
    const int per = a.ratio * a.n_buckets;
    float *table = tables + ((int)(threadIdx.x >> 6) * (64 / G) + at.slot) * per;
    if (a.bias_part) {
        for (int k = threadIdx.x; k < waves() * (64 / G) * per; k += (int)blockDim.x) tables[k] = 0.f;
        __syncthreads();
    }
    if (at.live) {
        const int g = at.h, t = at.t;
        const Source<T, VEC, G, GENERIC> Q(a.Q, a.ldq, g * a.ratio * a.d, a.d, t), dY(a.dY, a.lddy, g * a.ratio * a.dv, a.dv, t), K(a.K, a.ldk, g * a.d, a.d, t),
            V(a.V, a.ldv, g * a.dv, a.dv, t);
        T *dK = static_cast<T *>(a.O1) + (size_t)g * a.d, *dV = static_cast<T *>(a.O2) + (size_t)g * a.dv;
        const float *bias = a.bias ? a.bias + g * per : nullptr;
        const unsigned offset = drop_offset(a.key);
        const int call_log = a.ratio == 1 ? a.bundle_log : 0;   // heads of one generator call lie side by side
        Walk w;
        w.begin(a.p, at.chunk, at.in_group, at.group_lanes);
        Gathered<T, VEC> k, v;
        Sums<T, VEC, G, GENERIC> dk, dv;
        dk.zero();
        dv.zero();
        bool fresh = true;
        while (w.e < w.end) {
            const int n = w.count();
            int row[kBatch], own[O::N], bin[O::N];
            w.columns(n, row);
#pragma unroll
            for (int o = 0; o < O::N; ++o) {
                own[o] = O::of(t, o, row);
                bin[o] = bias ? w.bucket_of(O::entry(t, o), a.n_buckets) : 0;
            }
            if (fresh) {
                k = K.row(w.i);
                v = V.row(w.i);
                fresh = false;
            }
            for (int r = 0; r < a.ratio; ++r) {
                const int h = g * a.ratio + r;
                float b[O::N];
                float4 st[O::N];
#pragma unroll
                for (int o = 0; o < O::N; ++o) {
                    b[o] = bias ? bias[r * a.n_buckets + bin[o]] : 0.f;
                    st[o] = a.row_stats[(size_t)own[o] * a.heads + h];
                }
                Gathered<T, VEC> q[kBatch], dy[kBatch];
#pragma unroll
                for (int u = 0; u < kBatch; ++u) q[u] = Q.row(row[u], (long long)r * a.d * (int)sizeof(T));
#pragma unroll
                for (int u = 0; u < kBatch; ++u) dy[u] = dY.row(row[u], (long long)r * a.dv * (int)sizeof(T));
                if (r == 0 && w.e + n < w.end) w.fetch(a.p, w.e + n);
                K.keep_own(k);
                V.keep_own(v);
                int keep[O::N];
                if (a.key.threshold) kept<G, true, 1>(a.key, offset, w.i, row, h, t, call_log, keep);
                int use[O::N];
                bool masked = false;
#pragma unroll
                for (int o = 0; o < O::N; ++o) {
                    const bool there = O::entry(t, o) < n, open = b[o] != -INFINITY;
                    use[o] = there && open ? -1 : 0;
                    masked = masked || (there && !open);
                }
                if (bias && __any(masked)) {
#define SENSEI_WIPE(U)                     \
    q[U].mask(O::template get<U>(use));    \
    dy[U].mask(O::template get<U>(use));
                    SENSEI_EACH(SENSEI_WIPE)
#undef SENSEI_WIPE
                }
                float s[kBatch], c[kBatch], x[O::N], pw[O::N];
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {
                    s[u] = dot(k, q[u]);
                    c[u] = dot(v, dy[u]);
                }
                O::sums(s, t, x);
                O::sums(c, t, pw);
#pragma unroll
                for (int o = 0; o < O::N; ++o) {
                    const Score sc = score_of(a, x[o]);
                    const float ks = a.key.threshold && !(keep[o] & 1) ? 0.f : a.key.keep_scale, dp = ks == 0.f ? 0.f : pw[o] * ks;
                    const float p = use[o] ? exp_weight((sc.x + b[o] - st[o].x) - st[o].y) : 0.f, dt = use[o] ? p * (dp - st[o].z) : 0.f;
                    x[o] = dt * sc.slope * a.scale;
                    pw[o] = p * ks;
                    if (a.bias_part) {   // a head's lanes one after the other: two may be in one bucket
#pragma unroll
                        for (int z = 0; z < O::SHARERS; ++z)
                            if (t == z && use[o]) __hip_atomic_fetch_add(table + r * a.n_buckets + bin[o], dt, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                    }
                }
#define SENSEI_ADD(U)                      \
    dk.add(O::template get<U>(x), q[U]);   \
    dv.add(O::template get<U>(pw), dy[U]);
                SENSEI_EACH(SENSEI_ADD)
#undef SENSEI_ADD
            }
            w.e += n;
            if (w.row_done()) {
                if (at.head_live) {
                    if (!w.goes_on && w.e == w.row_end) {
                        dk.store(dK + (long long)w.i * a.ldo1, t, a.d, 1.f);
                        dv.store(dV + (long long)w.i * a.ldo2, t, a.dv, 1.f);
                    } else {
                        float *to = a.piece + piece_at(at.chunk, w.goes_on, a.kv_heads, g) * (2 * G * VEC);
                        dk.put(to, t);
                        dv.put(to + G * VEC, t);
                    }
                }
                dk.zero();
                dv.zero();
                if (w.e < w.end) w.next_row(a.p);
                fresh = true;
            }
        }
    }
    if (a.bias_part) {
        __syncthreads();
        const int n = per << a.bundle_log, slots = waves() * (64 / G);
        for (int k = threadIdx.x; k < n; k += (int)blockDim.x) {
            const int in_bundle = k / per, g = ((int)blockIdx.y << a.bundle_log) + in_bundle;
            if (g >= a.kv_heads) continue;
            float s = 0.f;
            for (int o = in_bundle; o < slots; o += 1 << a.bundle_log) s += tables[o * per + k % per];
            a.bias_part[(size_t)blockIdx.x * a.heads * a.n_buckets + (size_t)g * per + k % per] = s;
        }
    }
}

// dbias[k] = sum over the blocks of the walk, in their order; sixteen sums a workgroup, 64 threads each
__global__ __launch_bounds__(1024) void k_attention_bias(const float *__restrict__ part, int blocks, int n, float *__restrict__ out) {
    __shared__ double lds[64][16];
    const int k = blockIdx.x * 16 + (threadIdx.x & 15), seg = threadIdx.x >> 4;
    double s = 0.0;
    if (k < n) {
        int b = seg;
        for (; b + 7 * 64 < blocks; b += 8 * 64) {   // eight loads under way: one after the other they took 40 us of 5,700 blocks
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = part[(size_t)(b + u * 64) * n + k];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += (double)x[u];
        }
        for (; b < blocks; b += 64) s += (double)part[(size_t)b * n + k];
    }
    lds[seg][threadIdx.x & 15] = s;
    for (int half = 32; half > 0; half >>= 1) {
        __syncthreads();
        if (seg < half) lds[seg][threadIdx.x & 15] += lds[seg + half][threadIdx.x & 15];
    }
    if (seg == 0 && k < n) out[k] = (float)lds[0][threadIdx.x & 15];
}

// ------------------------------------------------------------------------------------------------------------------ rows in pieces, empty rows

enum { kJoinForward = 0, kJoinRows = 1, kJoinCols = 2 };

// Bound by reading the pieces (28 to 70 us where the walks take 500 to 1,700) and, in small calls, by being a launch (4 us).  A group of lanes per chunk boundary and bundle of heads (blockIdx.y): where a row crosses it that crossed none before, the group joins that row's pieces, in their order; a
// row of more than kManyPieces is left to the whole wavefront, whose groups take them in turn.  Workgroups behind those (of the first bundle)
// look over 64 rows a wavefront and write the rows without entries.  (4 rows of 500,000 entries: 5.5 times as slow with every row left to its group; rows
// of 100, and bounds of 4 or 64, made no difference.)
constexpr int kManyPieces = 16;
template <class T, int VEC, int G, int MODE, bool GENERIC>
__global__ __launch_bounds__(kThreads) void k_attention_join(AttnArgs a, int n_heads, int join_blocks) {
    const int lane = threadIdx.x & 63, wave = (int)blockIdx.x * waves() + (int)(threadIdx.x >> 6);
    if ((int)blockIdx.x >= join_blocks) {
        if (blockIdx.y > 0) return;
        const long long r0 = ((long long)((int)blockIdx.x - join_blocks) * waves() + (threadIdx.x >> 6)) * 64;
        const bool none = r0 + lane < a.p.n_rows && a.p.row_ptr[r0 + lane] == a.p.row_ptr[r0 + lane + 1];
        unsigned long long todo = __ballot(none);
        const int w1 = MODE == kJoinForward ? n_heads * a.dv : n_heads * a.d, w2 = MODE == kJoinCols ? n_heads * a.dv : 0;
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
    const int groups = (64 / G) >> a.bundle_log, group_lanes = G << a.bundle_log, t = lane % G, slot = lane / G, group = slot >> a.bundle_log;
    const int head = ((int)blockIdx.y << a.bundle_log) + (slot & ((1 << a.bundle_log) - 1)), h = head < n_heads ? head : n_heads - 1;
    // the first piece's chunk and the number of pieces of the row that first crosses the group's boundary; 0: there is none
    int first = wave * groups + group, pieces = 0, i = 0;
    if (first + 1 < a.p.n_chunks) {
        const int T0 = a.p.chunk, c = first + 1;
        i = a.p.chunk_row[c];
        const int start = a.p.row_ptr[i];
        if (start != c * T0 && start / T0 == first) pieces = (a.p.row_ptr[i + 1] - 1) / T0 - first + 1;
    }
    constexpr bool TWO = MODE == kJoinCols || (MODE == kJoinRows && sizeof(T) == 2);
    constexpr int W = (TWO ? 2 : 1) * G * VEC;
    using S = Sums<T, VEC, G, GENERIC>;
    S s1, s2;
    s1.zero();
    s2.zero();
    float m = -INFINITY, l = 0.f, delta = 0.f;
    auto join = [&](float om, float ol, const S &o) {
        const float top = fmaxf(m, om), base = top > -INFINITY ? top : 0.f, f = exp_weight(m - base), fo = exp_weight(om - base);
        m = top;
        l = l * f + ol * fo;
        s1.scale(f);
        s1.add(fo, o);
    };
    // pieces k, k + by, .. of n, a few at a time: their loads are under way together
    auto take = [&](int from, int k, int by, int n) {
        constexpr int AT_ONCE = VEC == 16 || TWO ? 4 : 8;
        for (; k < n; k += AT_ONCE * by) {
            S x[AT_ONCE], y[TWO ? AT_ONCE : 1];
            float2 ml[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int kk = k + u * by < n ? k + u * by : k;
                const size_t at = piece_at(from + kk, kk > 0, n_heads, h);
                x[u].get(a.piece + at * W, t);
                if (TWO) y[u].get(a.piece + at * W + G * VEC, t);
                ml[u] = MODE == kJoinForward || (MODE == kJoinRows && TWO) ? a.piece_ml[at] : make_float2(0.f, 0.f);
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                if (k + u * by >= n) break;
                if (MODE == kJoinForward) join(ml[u].x, ml[u].y, x[u]);
                else {
                    s1.add(1.f, x[u]);
                    if (TWO) s2.add(1.f, y[u]);
                    delta += ml[u].x;
                }
            }
        }
    };
    auto finish = [&](int row) {
        if (head >= n_heads) return;
        if (MODE == kJoinForward) {
            s1.store(static_cast<T *>(a.O1) + (long long)row * a.ldo1 + (size_t)h * a.dv, t, a.dv, l == 0.f ? 0.f : a.key.keep_scale / l);
            if (t == 0) a.stats[(size_t)row * n_heads + h] = make_float2(m, logf(l));
            return;
        }
        if (MODE == kJoinRows && TWO) {
            s1.add(-delta, s2);
            if (t == 0) a.row_stats[(size_t)row * n_heads + h].z += delta;
        }
        s1.store(static_cast<T *>(a.O1) + (long long)row * a.ldo1 + (size_t)h * a.d, t, a.d, 1.f);
        if (MODE == kJoinCols) s2.store(static_cast<T *>(a.O2) + (long long)row * a.ldo2 + (size_t)h * a.dv, t, a.dv, 1.f);
    };
    const unsigned long long many = __ballot(pieces > kManyPieces);
    if (pieces > 0 && pieces <= kManyPieces) {
        take(first, 0, 1, pieces);
        finish(i);
    }
    for (int o = 0; o < groups; ++o) {
        if (!(many >> (o * group_lanes) & 1)) continue;     // the same for the whole wavefront
        const int from = __shfl(first, o * group_lanes, 64), row = __shfl(i, o * group_lanes, 64), n = __shfl(pieces, o * group_lanes, 64);
        s1.zero();
        s2.zero();
        m = -INFINITY;
        l = delta = 0.f;
        take(from, group, groups, n);
        for (int dist = group_lanes; dist < 64; dist <<= 1) {
            S x;
#pragma unroll
            for (int k = 0; k < VEC; ++k) x.v[k] = __shfl_xor(s1.v[k], dist, 64);
            if (MODE == kJoinForward) join(__shfl_xor(m, dist, 64), __shfl_xor(l, dist, 64), x);
            else {
                s1.add(1.f, x);
                if (TWO) {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) x.v[k] = __shfl_xor(s2.v[k], dist, 64);
                    s2.add(1.f, x);
                }
                if (MODE == kJoinRows && TWO) delta += __shfl_xor(delta, dist, 64);
            }
        }
        if (group == 0) finish(row);
    }
}

// (m, log l, D) of every row and query head, D = <dY, Y>, side by side for the walks; workgroups behind those put the buckets into the order of the
// transposed pattern.  Bound by memory where there are no buckets, else by writing single bytes out of order: 31 us for 100,000 rows of 4 heads of 32 and
// 2.1 M entries, 73 us for 290,000 rows of 8 heads of 16 in bf16 and 11.8 M entries.
template <class T, int VEC, int G, bool GENERIC>
__global__ __launch_bounds__(kThreads) void k_attention_row_stats(AttnArgs a, unsigned blocks, const uint8_t *__restrict__ bucket, const int32_t *__restrict__ t_pos,
                                                                  int nnz, uint8_t *__restrict__ out) {
    if (blockIdx.x >= blocks) {
        const long long k = (long long)(blockIdx.x - blocks) * kThreads + threadIdx.x;
        if (k < nnz) out[t_pos[k]] = bucket[k];
        return;
    }
    const int t = threadIdx.x % G;
    for (long long at = (long long)blockIdx.x * (kThreads / G) + threadIdx.x / G; at < (long long)a.p.n_rows * a.heads; at += (long long)blocks * (kThreads / G)) {
        const int i = (int)(at / a.heads), h = (int)(at % a.heads);
        const Source<T, VEC, G, GENERIC> Y(a.Y, a.ldy, h * a.dv, a.dv, t), dY(a.dY, a.lddy, h * a.dv, a.dv, t);
        const Gathered<T, VEC> y = Y.own(i), dy = dY.own(i);
        const float2 ml = a.stats[at];
        float d = 0.f;
#pragma unroll
        for (int k = 0; k < VEC; ++k) d = fmaf(dy.get(k), y.get(k), d);
        d = sum_over<G>(d);
        if (t == 0) a.row_stats[at] = make_float4(ml.x, ml.y, d, 0.f);
    }
}

// ------------------------------------------------------------------------------------------------------------------ host side

// Lanes of a head, from the wider of a head's key and value: 32 bytes a lane; 8 elements where a lane takes several query heads (16 of them and
// their sums would leave a SIMD one wavefront).  Tables of dbias (`table` floats a head) are kept for every head that a
// wavefront works on: more lanes a head where those would not fit 64 KB.
struct Shape { int vec, lanes; };
Shape shape_of(int d, int dv, int elem, int heads_a_lane, int table) {
    const int w = d > dv ? d : dv;
    Shape s{heads_a_lane > 1 ? 8 : 32 / elem, 1};
    while (s.lanes * s.vec < w || (size_t)(64 / s.lanes) * table * sizeof(float) > 65536) s.lanes *= 2;
    return s;
}
// Heads of a bundle: as many as gather 256 bytes an entry, and all query heads of a key head (`together`).  Bundles of 1, 2, 4, 8 heads, us: 290,000
// nodes of batched graphs, 8 heads of 16 in bf16, forward and backward 12,377 / 5,320 / 2,890 / 2,623; 100,000 nodes of 21, 4 heads of 32 in fp32 1,247 /
// 1,164 / 1,263; 233,000 nodes of 87, 8 heads of 64 on 2 in bf16, forward 4,086 / 2,206 / 1,983 / 1,949.
int bundle_log_of(const Shape &s, int n_heads, int together, int bytes) {
    int log = 0;
    while ((s.lanes << (log + 1)) <= 64 && (1 << log) < n_heads && ((bytes << log) / together < 256 || (1 << log) < together)) ++log;
    return log;
}
// Entries of a chunk: as many as leave 8,192 wavefronts, 32 to 256, so that chunks of many short rows (a batch each, however few their entries) even out
// and pieces of rows stay few; 16 where a SIMD would have less than a wavefront.  4,096 / 8,192 / 16,384 wavefronts, us: power-law patterns, training,
// 100,000 nodes of 21 1,273 / 959 / 933, 97,000 of 11 1,065 / 893 / 866, forward, 212,000 of 22 1,542 / 1,552 / 1,366; uniform ones, training, batched
// graphs of 290,000 nodes 2,405 / 2,196 / 2,279, 51,000 rows of 60 1,555 / 1,639 / 1,743, forward, 123,000 rows of 48 306 / 308 / 339, 172,000 of 16
// 631 / 611 / 654.  Chunks of 16 / 32 entries: 10,000 nodes of 11 21 / 26.
// Rows of thousands of entries are cut no finer than sixteen pieces a row.
int chunk_of(int64_t nnz, int n_rows, int bundles, int groups) {
    int t = 256;
    while (t > 32 && nnz / t * bundles / groups < 8192 && t * 8ll * n_rows > nnz) t >>= 1;
    return t == 32 && nnz / t * bundles / groups < 1024 ? 16 : t;
}

// Gathers by 24-bit products and 32-bit offsets, whole pieces: every number of a row and of bytes a row below 2^24, every matrix below 4 GB, heads
// no narrower than a piece.  These / general ones, us: 10,000 nodes of 11 30 / 32, 100,000 of 21 (fp32, training) 1,031 / 1,147, batched graphs (bf16,
// training) 2,284 / 6,650, 233,000 of 87 (bf16) 1,995 / 7,725.
bool plain_gathers(const AttentionCall &c) {
    const int per = 16 / c.elem;
    if (c.d < per || c.dv < per || c.A->n_rows >= 1 << 24 || c.A->n_cols >= 1 << 24) return false;
    struct { int64_t rows, ld; } m[] = {{c.A->n_cols, c.ldk}, {c.A->n_cols, c.ldv}, {c.A->n_rows, c.ldq}, {c.At ? c.A->n_rows : 0, c.lddy}, {c.At ? c.A->n_rows : 0, c.ldy}};
    for (const auto &x : m)
        if (x.rows && (x.ld * c.elem >= 1 << 24 || x.rows * x.ld * c.elem > 0xFFFFFFFFll)) return false;
    return true;
}

enum Walks { kForward, kRows, kCols };
struct Layout {
    Shape shape;
    int heads_a_lane;                              // R of the walk
    int bundle_log, bundles, groups, chunk, n_chunks;
    int join_log, join_bundles;                    // bundles of the pass that joins the pieces: eight lanes, 256 bytes of the pieces and more
    // A lane takes two query heads of a key head together where heads are wider than 128 bytes: what they gather is the same, and a wavefront has twice as
    // much of different rows under way.  One / two / four heads a lane, us: forward, fp32, 184,000 rows of 15, 16 heads of 96 on 4 2,780 / 2,158 / 2,279;
    // 212,000 nodes of 22, 6 heads of 128 on 3 1,770 / 1,482; training, fp16, 51,000 rows of 60, 4 heads of 96 on 1 1,951 / 1,757 / 1,812.  Narrower heads
    // lose the lanes that would share out their entries: bf16, 233,000 nodes of 87, 8 heads of 64 on 2 1,978 / 2,057 / 2,371.
    static int together_of(const AttentionCall &c, Walks walk, bool plain) {
        return walk != kCols && plain && c.heads / c.kv_heads % 2 == 0 && (c.d > c.dv ? c.d : c.dv) * c.elem > 128 ? 2 : 1;
    }
    Layout(const AttentionCall &c, Walks walk, bool plain) {
        const int64_t nnz = c.A->nnz;
        heads_a_lane = together_of(c, walk, plain);
        const bool cols = walk == kCols;
        const int all = cols ? c.kv_heads : c.heads, n_heads = all / heads_a_lane, together = cols ? 1 : c.heads / c.kv_heads / heads_a_lane, elem = c.elem, d = c.d, dv = c.dv;
        shape = shape_of(d, dv, elem, heads_a_lane, cols && c.dbias ? c.heads / c.kv_heads * c.n_buckets : 0);
        bundle_log = bundle_log_of(shape, n_heads, together, (d > dv ? d : dv) * elem);
        bundles = (n_heads + (1 << bundle_log) - 1) >> bundle_log;
        groups = (64 / shape.lanes) >> bundle_log;
        chunk = chunk_of(nnz, cols ? c.A->n_cols : c.A->n_rows, bundles, groups);
        n_chunks = (int)((nnz + chunk - 1) / chunk);
        join_log = 0;
        while ((shape.lanes << join_log) < 8 && (1 << join_log) < all) ++join_log;
        join_bundles = (all + (1 << join_log) - 1) >> join_log;
    }
    int blocks(int waves) const { return (n_chunks + waves * groups - 1) / (waves * groups); }
    int join_blocks(int waves) const {
        const int per = waves * ((64 / shape.lanes) >> join_log);
        return n_chunks > 1 ? (n_chunks + per - 1) / per : 0;
    }
    size_t rows_bytes() const { return align_up((size_t)n_chunks * sizeof(int32_t), 256); }
    size_t piece_bytes(int n_heads, int sums) const { return align_up((size_t)n_chunks * 2 * n_heads * shape.vec * shape.lanes * sums * sizeof(float), 256); }
    size_t ml_bytes(int n_heads) const { return align_up((size_t)n_chunks * 2 * n_heads * sizeof(float2), 256); }
};

// Wavefronts of a workgroup of the walk over the columns: as many as the tables of dbias leave room for in 64 KB of LDS
int table_waves(const AttentionCall &c, const Shape &s) {
    const size_t wave = (size_t)(64 / s.lanes) * (c.heads / c.kv_heads) * c.n_buckets * sizeof(float);
    return !c.dbias || 4 * wave <= 65536 ? 4 : 2 * wave <= 65536 ? 2 : 1;
}

struct Room {   // what the backward carves its scratch into
    Layout rows, cols;
    int col_waves;
    size_t bucket, stats, piece, ml, bias;
    Room(const AttentionCall &c, bool plain) : rows(c, kRows, plain), cols(c, kCols, plain) {
        col_waves = table_waves(c, cols.shape);
        bucket = c.n_buckets > 0 ? align_up((size_t)c.A->nnz, 256) : 0;
        stats = align_up((size_t)c.A->n_rows * c.heads * sizeof(float4), 256);
        const size_t p1 = rows.piece_bytes(c.heads, c.elem == 4 ? 1 : 2), p2 = cols.piece_bytes(c.kv_heads, 2);   // one after the other
        piece = p1 > p2 ? p1 : p2;
        ml = c.elem == 4 ? 0 : rows.ml_bytes(c.heads);
        bias = c.n_buckets > 0 && c.dbias ? align_up((size_t)cols.blocks(col_waves) * c.heads * c.n_buckets * sizeof(float), 256) : 0;
    }
    size_t bytes() const { return rows.rows_bytes() + cols.rows_bytes() + bucket + stats + piece + ml + bias; }
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

WalkPattern pattern_of(const sensei_csr &A, const Layout &l, const uint8_t *bucket, int32_t *chunk_row) {
    return {A.row_ptr, A.col_idx, bucket, chunk_row, A.n_rows, (int)A.nnz, l.chunk, l.n_chunks};
}

template <class T, int VEC, int G, bool GENERIC, int MODE> hipError_t join_and_fill(AttnArgs a, const Layout &l, int n_heads, hipStream_t s) {
    constexpr int waves = kThreads / 64;
    a.bundle_log = l.join_log;
    const int join_blocks = l.join_blocks(waves), fill = (int)((a.p.n_rows + 64ll * waves - 1) / (64 * waves));
    if (join_blocks + fill == 0) return hipSuccess;
    hipLaunchKernelGGL((k_attention_join<T, VEC, G, MODE, GENERIC>), dim3(join_blocks + fill, l.join_bundles), dim3(kThreads), 0, s, a, n_heads, join_blocks);
    return hipGetLastError();
}

// VEC elements a lane: 8 of fp32 whatever R, of 16 bits 16 with R = 1 and 8 with others
template <class T, int VEC, int R> constexpr bool kShaped = sizeof(T) == 4 || (R == 1) == (VEC == 16);

template <class T, int VEC, int G, bool GENERIC> hipError_t forward_shape(const AttnArgs &a, const Layout &l, hipStream_t s) {
    const dim3 grid(l.blocks(kThreads / 64), l.bundles), block(kThreads);
    if (a.p.nnz > 0) {
        if constexpr (!GENERIC && kShaped<T, VEC, 2>) {
            if (l.heads_a_lane == 2) hipLaunchKernelGGL((k_attention<T, VEC, G, GENERIC, 2>), grid, block, 0, s, a);
        }
        if constexpr (kShaped<T, VEC, 1>) {
            if (l.heads_a_lane == 1) hipLaunchKernelGGL((k_attention<T, VEC, G, GENERIC, 1>), grid, block, 0, s, a);
        }
    }
    return join_and_fill<T, VEC, G, GENERIC, kJoinForward>(a, l, a.heads, s);
}

// (m, log l, D) and dQ
template <class T, int VEC, int G, bool GENERIC> hipError_t rows_shape(const AttentionCall &c, AttnArgs a, const Layout &l, uint8_t *bucket_t, hipStream_t s) {
    a.O1 = c.dQ; a.ldo1 = c.lddq;
    a.bundle_log = l.bundle_log;
    if (a.p.nnz > 0) {
        // 2^22 workgroups at most (a grid's threads are counted in 32 bits): more rows and heads than those take another turn
        const unsigned blocks = (unsigned)std::min<int64_t>(((int64_t)a.p.n_rows * a.heads + kThreads / G - 1) / (kThreads / G), 1 << 22), more = a.bias ? (unsigned)((a.p.nnz + kThreads - 1) / kThreads) : 0;
        hipLaunchKernelGGL((k_attention_row_stats<T, VEC, G, GENERIC>), dim3(blocks + more), dim3(kThreads), 0, s, a, blocks, c.bucket, c.t_pos, a.p.nnz, bucket_t);
        const dim3 grid(l.blocks(kThreads / 64), l.bundles), block(kThreads);
        if constexpr (!GENERIC && kShaped<T, VEC, 2>) {
            if (l.heads_a_lane == 2) hipLaunchKernelGGL((k_attention_back_rows<T, VEC, G, GENERIC, 2>), grid, block, 0, s, a);
        }
        if constexpr (kShaped<T, VEC, 1>) {
            if (l.heads_a_lane == 1) hipLaunchKernelGGL((k_attention_back_rows<T, VEC, G, GENERIC, 1>), grid, block, 0, s, a);
        }
    }
    return join_and_fill<T, VEC, G, GENERIC, kJoinRows>(a, l, a.heads, s);
}

// dK, dV and dbias
template <class T, int VEC, int G, bool GENERIC> hipError_t cols_shape(const AttentionCall &c, AttnArgs a, const Room &room, hipStream_t s) {
    if constexpr (kShaped<T, VEC, 1>) {
        const Layout &l = room.cols;
        a.O1 = c.dK; a.ldo1 = c.lddk;
        a.O2 = c.dV; a.ldo2 = c.lddv;
        a.bundle_log = l.bundle_log;
        if (a.p.nnz > 0) {
            const int blocks = l.blocks(room.col_waves), n = a.heads * a.n_buckets;
            const size_t lds = a.bias_part ? (size_t)room.col_waves * (64 / G) * a.ratio * a.n_buckets * sizeof(float) : 0;
            hipLaunchKernelGGL((k_attention_back_cols<T, VEC, G, GENERIC>), dim3(blocks, l.bundles), dim3(64 * room.col_waves), lds, s, a);
            if (a.bias_part) hipLaunchKernelGGL(k_attention_bias, dim3((n + 15) / 16), dim3(1024), 0, s, a.bias_part, blocks, n, c.dbias);
        }
        return join_and_fill<T, VEC, G, GENERIC, kJoinCols>(a, l, a.kv_heads, s);
    }
    return hipErrorInvalidValue;   // no layout has this shape
}

#define SENSEI_BY_SHAPE(T, VEC, lanes, GEN, CALL)                                                              \
    (lanes == 1 ? CALL(T, VEC, 1, GEN) : lanes == 2 ? CALL(T, VEC, 2, GEN) : lanes == 4 ? CALL(T, VEC, 4, GEN) \
     : lanes == 8 ? CALL(T, VEC, 8, GEN) : lanes == 16 ? CALL(T, VEC, 16, GEN) : CALL(T, VEC, 32, GEN))
#define SENSEI_BY_GATHER(T, VEC, lanes, plain, CALL) (plain ? SENSEI_BY_SHAPE(T, VEC, lanes, false, CALL) : SENSEI_BY_SHAPE(T, VEC, lanes, true, CALL))
#define SENSEI_BY_VEC(T, vec, lanes, plain, CALL) (vec == 16 ? SENSEI_BY_GATHER(T, 16, lanes, plain, CALL) : SENSEI_BY_SHAPE(T, 8, lanes, false, CALL))
#define SENSEI_BY_TYPE(type, shape, plain, CALL)                                                                                                   \
    (type == SENSEI_F32 ? SENSEI_BY_GATHER(float, 8, shape.lanes, plain, CALL) : type == SENSEI_BF16 ? SENSEI_BY_VEC(Bf16, shape.vec, shape.lanes, plain, CALL) \
     : SENSEI_BY_VEC(F16, shape.vec, shape.lanes, plain, CALL))

}  // namespace

// The queries do not know the leading dimensions: room for either kind of gathers.
size_t attention_ws_bytes(const AttentionCall &c) {
    size_t most = 0;
    for (const bool plain : {false, true}) {
        const Layout l(c, kForward, plain);
        const size_t n = l.rows_bytes() + l.piece_bytes(c.heads, 1) + l.ml_bytes(c.heads) + 256;
        most = n > most ? n : most;
    }
    return most;
}

hipError_t launch_attention(const AttentionCall &c, char *ws, hipStream_t s) {
    if (c.A->n_rows <= 0) return hipSuccess;
    const bool plain = plain_gathers(c);
    const Layout l(c, kForward, plain);
    AttnArgs a = args_of(c);
    int32_t *chunk_row = reinterpret_cast<int32_t *>(ws);
    a.p = pattern_of(*c.A, l, a.bias ? c.bucket : nullptr, chunk_row);
    a.piece = reinterpret_cast<float *>(ws + l.rows_bytes());
    a.piece_ml = reinterpret_cast<float2 *>(ws + l.rows_bytes() + l.piece_bytes(c.heads, 1));
    a.O1 = c.out; a.ldo1 = c.ldo;
    a.bundle_log = l.bundle_log;
#define SENSEI_CALL(T, V, G, GEN) forward_shape<T, V, G, GEN>(a, l, s)
    return SENSEI_BY_TYPE(c.type, l.shape, plain, SENSEI_CALL);
#undef SENSEI_CALL
}

size_t attention_backward_ws_bytes(const AttentionCall &c) {
    const size_t a = Room(c, false).bytes(), b = Room(c, true).bytes();
    return (a > b ? a : b) + 256;
}

hipError_t launch_attention_backward(const AttentionCall &c, char *ws, hipStream_t s) {
    const bool plain = plain_gathers(c);
    const Room room(c, plain);
    AttnArgs a = args_of(c);
    char *at = ws;
    auto take = [&](size_t n) { char *p = at; at += n; return p; };
    int32_t *rows_r = reinterpret_cast<int32_t *>(take(room.rows.rows_bytes())), *rows_c = reinterpret_cast<int32_t *>(take(room.cols.rows_bytes()));
    uint8_t *bucket_t = reinterpret_cast<uint8_t *>(take(room.bucket));
    a.row_stats = reinterpret_cast<float4 *>(take(room.stats));
    a.piece = reinterpret_cast<float *>(take(room.piece));
    a.piece_ml = reinterpret_cast<float2 *>(take(room.ml));
    a.bias_part = a.bias && c.dbias ? reinterpret_cast<float *>(take(room.bias)) : nullptr;
    if (c.A->nnz == 0 && a.bias_part) {
        const hipError_t e = launch_zero_matrix(c.dbias, 1, c.heads * c.n_buckets, c.heads * c.n_buckets, false, s);
        if (e != hipSuccess) return e;
    }
    a.p = pattern_of(*c.A, room.rows, a.bias ? c.bucket : nullptr, rows_r);
#define SENSEI_CALL(T, V, G, GEN) rows_shape<T, V, G, GEN>(c, a, room.rows, bucket_t, s)
    const hipError_t e = SENSEI_BY_TYPE(c.type, room.rows.shape, plain, SENSEI_CALL);
#undef SENSEI_CALL
    if (e != hipSuccess) return e;
    a.p = pattern_of(*c.At, room.cols, a.bias ? bucket_t : nullptr, rows_c);
#define SENSEI_CALL(T, V, G, GEN) cols_shape<T, V, G, GEN>(c, a, room, s)
    return SENSEI_BY_TYPE(c.type, room.cols.shape, plain, SENSEI_CALL);
#undef SENSEI_CALL
}

}  // namespace sensei
