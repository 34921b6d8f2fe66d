// What a training step and an answer need around the layers: dropout, and the log probabilities of labels with their entropy, their
// highest alternatives and their gradient.  Elements are fp32, bf16 or fp16; everything is computed in fp32.
#include <cfloat>

#include "element_types.h"
#include "sensei_internal.h"

namespace sensei {

namespace {

// ------------------------------------------------------------------------------------------------------------------------ dropout

// Y = add + keep (x) X / (1 - p).  Whether element (i, c) is kept is word c % 4 of the generator at counter (c / 4, i, 0, offset): it
// depends on the element's place alone, not on leading dimensions or the launch, and the backward pass is the same call on dY.
// A lane takes 16 bytes (one counter's four elements in fp32, two counters' in 16 bits), whose row and column come from one multiplication (FastDiv).
// Bound by memory: 233,000 x 602 in fp32 207 us (5.4 TB/s, a copy of this size 5.0), 2.45 M x 256 in bf16 462 us (5.4 TB/s), with a residual 622 us (6.0).  Four pieces a lane, a
// workgroup apart, took 213 and 522 us.
struct DropArgs {
    const void *X, *add;
    void *Y;
    long long ldx, lda, ldy;
    unsigned row0;             // of this launch
    unsigned units;            // rows * pieces a row
    int cols;
    FastDiv per_row;
    DropKey key;
};
constexpr int kDropThreads = 256;

template <class T, bool ADD>
__global__ __launch_bounds__(kDropThreads) void k_dropout(DropArgs a) {
    constexpr int E = kPerPiece<T>;
    const unsigned at = blockIdx.x * (unsigned)kDropThreads + threadIdx.x;
    if (at >= a.units) return;
    const unsigned offset = a.key.offset + (a.key.offset_dev ? *a.key.offset_dev : 0u);
    const unsigned i = a.per_row.div(at), row = a.row0 + i;
    const int col = (int)(at - i * a.per_row.d) * E, live = a.cols - col < E ? a.cols - col : E;   // fewer than E at a row's end
    const T *px = static_cast<const T *>(a.X) + (long long)row * a.ldx + col;
    const T *pr = ADD ? static_cast<const T *>(a.add) + (long long)row * a.lda + col : nullptr;
    Piece<T, E> x, r, y;
    if (live == E) {
        x = Piece<T, E>::load(px);
        if (ADD) r = Piece<T, E>::load(pr);
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (k < live) {
                x.x[k] = px[k];
                if (ADD) r.x[k] = pr[k];
            }
        }
    }
#pragma unroll
    for (int q = 0; q < E / 4; ++q) {
        const Words w = philox((unsigned)col / 4 + q, row, 0u, offset, a.key.k0, a.key.k1);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int e = 4 * q + k;
            float v = w.w[k] < a.key.threshold ? 0.f : to_f32(x.x[e]) * a.key.keep_scale;
            if (ADD) v += to_f32(r.x[e]);
            y.x[e] = from_f32<T>(v);
        }
    }
    T *py = static_cast<T *>(a.Y) + (long long)row * a.ldy + col;
    if (live == E) y.store(py);
    else {
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (k < live) py[k] = y.x[k];
    }
}

template <class T, bool ADD> hipError_t dropout_typed(DropArgs a, long long rows, hipStream_t s) {
    const unsigned per_row = (unsigned)((a.cols + kPerPiece<T> - 1) / kPerPiece<T>);
    a.per_row = FastDiv::of(per_row);
    const long long slab = (0x7FFFFFFFll - kDropThreads) / per_row;   // piece numbers of a launch stay below 2^31
    for (long long r0 = 0; r0 < rows; r0 += slab) {
        const long long n = rows - r0 < slab ? rows - r0 : slab;
        a.row0 = (unsigned)r0;
        a.units = (unsigned)(n * per_row);
        hipLaunchKernelGGL((k_dropout<T, ADD>), dim3((a.units + kDropThreads - 1) / kDropThreads), dim3(kDropThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// -------------------------------------------------------------------------------------------------------- log probabilities of labels

// One row of C logits z: with its maximum m,
//     s = sum exp(z - m),  t = sum (z - m) exp(z - m);   lse = m + log s,  entropy = log s - t / s,  log p_j = (z_j - m) - log s.
// Classes at -inf have no share (and add 0 to t); a row of nothing else has lse = -inf.
//
// The gradient needs no difference of its own: exp(z - m) = 2^(z L - c) 2^(c - m L), L = log2(e) in fp32, c = m L rounded, is one fused product and one
// instruction an element, and the second factor, the same for a whole row, goes with 1 / s.  Where m L has no room in fp32 (rows of a type's lowest
// value) the difference is formed first.
struct RowBase {
    float m, c;
    bool direct;     // differences
    __device__ __forceinline__ explicit RowBase(float top) {
#pragma clang fp contract(off)   // c is the rounded product wherever it goes
        m = top > -INFINITY ? top : 0.f;
        direct = !(fabsf(m) < 1e30f);      // and an infinite maximum, whose row is NaN whatever is done
        c = direct ? 0.f : m * kLog2E;
    }
    template <bool DIRECT> __device__ __forceinline__ float power(float z) const { return DIRECT ? exp_neg(z - m) : __builtin_amdgcn_exp2f(fmaf(z, kLog2E, -c)); }
    // log of a power over that of exp(z - m)
    __device__ __forceinline__ float shift() const { return direct ? 0.f : fmaf(m, kLog2E, -c) * kLn2; }
};

// Sums of a part of a row whose maximum is known to be at least every element of it.
struct RowSum {
    float m, s, t;   // relative to m
    __device__ __forceinline__ static RowSum empty() { return {-INFINITY, 0.f, 0.f}; }
    __device__ __forceinline__ void raise(float top) {   // top > m
        if (m > -INFINITY) {
            const float f = exp_neg(m - top);
            t = f == 0.f ? 0.f : fmaf(m - top, s, t) * f;   // the difference may be as low as a type's lowest value
            s *= f;
        }
        m = top;
    }
    __device__ __forceinline__ void join(const RowSum &o) {
        RowSum b = o;
        if (b.m > m) raise(b.m);
        else if (m > b.m) b.raise(m);
        s += b.s;
        t += b.t;
    }
    // z - lse, the large numbers first: exact where m is far from 0 (a row of nothing but a type's lowest value)
    __device__ __forceinline__ float log_p(float z, float log_s) const { return s == 0.f ? -INFINITY : (z - m) - log_s; }
};

// Rank of a class: a number that orders logits as unsigned integers do (NaN above all, the two zeros alike), over the class from the
// lowest: equal logits rank the lower class first, and no two classes rank alike.  0 is no class.
__device__ __forceinline__ unsigned order_key(float z) {
    const unsigned b = __float_as_uint(z + 0.f);
    if (z != z) return 0xFFFFFFFFu;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float order_value(unsigned k) {
    if (k == 0xFFFFFFFFu) return NAN;
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
typedef unsigned long long Rank;
__device__ __forceinline__ Rank rank_of(unsigned key, int cls) { return (Rank)key << 32 | (unsigned)~cls; }
__device__ __forceinline__ int rank_class(Rank r) { return (int)~(unsigned)r; }

struct LogArgs {
    const void *Z;
    long long ld, rows;
    int classes, top;
    const int32_t *labels;
    float2 *stats;         // written by the forward (read by the backward)
    float *logp, *entropy;
    long long row0;        // first row of this launch
    int32_t *top_idx;
    float *top_logp;
    // long rows that several workgroups share: classes a part, and what each part leaves
    int parts, part_classes;
    RowSum *part_sum;      // rows * parts
    Rank *part_top;        // rows * parts * top, 0 where a part has fewer classes
    // backward
    const float *g_logp, *g_entropy, *entropy_in;
    void *dZ;
    long long lddz;
};
constexpr int kLogThreads = 256, kMaxParts = 64;

// A lane's R highest classes among those it has seen, in order.
template <int R> struct Highest {
    unsigned key[R];
    int cls[R];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < R; ++i) { key[i] = 0; cls[i] = 0; }
    }
    // classes come in ascending order: an equal one stays behind
    __device__ __forceinline__ void see(unsigned k, int c) {
        if (k <= key[R - 1]) return;
#pragma unroll
        for (int i = R - 1; i > 0; --i) {
            const bool above = k > key[i - 1], here = k > key[i];
            cls[i] = above ? cls[i - 1] : here ? c : cls[i];
            key[i] = above ? key[i - 1] : here ? k : key[i];
        }
        if (k > key[0]) { key[0] = k; cls[0] = c; }
    }
    // what a class has to be above to be seen: NaN (nothing is known to be below it) while the list has room
    __device__ __forceinline__ float least() const { return key[R - 1] ? order_value(key[R - 1]) : NAN; }
    __device__ __forceinline__ Rank head() const { return key[0] ? rank_of(key[0], cls[0]) : 0; }
    __device__ __forceinline__ void pop() {
#pragma unroll
        for (int i = 0; i + 1 < R; ++i) { key[i] = key[i + 1]; cls[i] = cls[i + 1]; }
        key[R - 1] = 0;
    }
};
template <> struct Highest<0> {
    __device__ __forceinline__ void clear() {}
    __device__ __forceinline__ void see(unsigned, int) {}
};

template <int CTRL> __device__ __forceinline__ Rank dpp_rank(Rank r) { return (Rank)(unsigned)dpp<CTRL>((int)(r >> 32)) << 32 | (unsigned)dpp<CTRL>((int)(unsigned)r); }
__device__ __forceinline__ Rank higher(Rank a, Rank b) { return a > b ? a : b; }
// the highest of L lanes' ranks, in all of them (as over_lanes)
template <int L> __device__ __forceinline__ Rank max_over_lanes(Rank r) {
    r = higher(r, dpp_rank<0xB1>(r));
    r = higher(r, dpp_rank<0x4E>(r));
    if (L >= 16) {
        r = higher(r, dpp_rank<0x141>(r));
        r = higher(r, dpp_rank<0x140>(r));
    }
    if (L >= 64) {
        r = higher(r, __shfl_xor(r, 16, 64));
        r = higher(r, __shfl_xor(r, 32, 64));
    }
    return r;
}

template <class T> __device__ __forceinline__ void finish_row(const LogArgs &a, long long row, const RowSum &v, float log_s, const T *z) {
    if (a.stats) a.stats[row] = make_float2(v.m, log_s);
    if (a.entropy) a.entropy[row] = v.s == 0.f ? 0.f : log_s - v.t / v.s;
    if (a.logp) {
        const int y = a.labels[row];
        a.logp[row] = y >= 0 && y < a.classes ? v.log_p(to_f32(z[y]), log_s) : 0.f;
    }
}

// E classes side by side into the sums (whose m is at least their maximum)
template <int E> __device__ __forceinline__ void add_powers(RowSum &v, const float (&f)[E]) {
    const float base = v.m > -INFINITY ? v.m : 0.f;
#pragma unroll
    for (int k = 0; k < E; ++k) {
        const float d = f[k] - base, e = exp_weight(d);
        v.s += e;
        v.t = fmaf(e, fmaxf(d, -FLT_MAX), v.t);   // -inf: 0 times a finite number
    }
}

// The alternatives, one after the other: each the highest head of all lanes' lists.  A lane whose list was drawn empty goes over its classes again for those
// behind the last one drawn: rare (more than R of a row's highest in one lane) and exact.  draw(r): the highest rank of all lanes.
// Classes [c0, c1), `head` single ones (one each of the first lanes) before those that the lanes take by pieces.
template <class T, int L, int R, class Draw, class Put>
__device__ __forceinline__ void draw_alternatives(Highest<R> &best, int top, const T *z, int c0, int head, int c1, int lane, Draw draw, Put put) {
    constexpr int E = kPerPiece<T>;
    int mine = 0;                          // drawn from this lane
    for (int k = 0; k < top; ++k) {
        const Rank r = draw(best.head(), k);
        put(r, k);
        if (r != 0 && best.head() == r) {
            best.pop();
            if (++mine % R == 0 && k + 1 < top) {
                auto again = [&](int c) {
                    const unsigned key = order_key(to_f32(z[c]));
                    if (rank_of(key, c) < r) best.see(key, c);
                };
                if (lane < head) again(c0 + lane);
                for (int cc = c0 + head + lane * E; cc < c1; cc += L * E)
                    for (int e = 0; e < E && cc + e < c1; ++e) again(cc + e);
            }
        }
    }
}

// Rows that L lanes (4, 16, 64) hold in their registers, PIECES 16-byte pieces a lane: the maximum first, then one sum.  Bound by memory once there are
// rows enough: 233,000 x 41 in fp32 10 us (3.9 TB/s), the gradient 18 us (4.2 TB/s); 1,024 x 47 is the launch.
template <class T, int L, int PIECES, int R>
__global__ __launch_bounds__(kLogThreads) void k_logprobs_short(LogArgs a) {
    constexpr int E = kPerPiece<T>;
    const int lane = threadIdx.x % L;
    const long long row = a.row0 + (long long)blockIdx.x * (kLogThreads / L) + threadIdx.x / L;
    const bool live = row < a.rows;      // whole groups of lanes; nobody leaves before the lanes' exchanges
    const T *z = static_cast<const T *>(a.Z) + (live ? row : a.rows - 1) * a.ld;
    Piece<T, E> x[PIECES];
#pragma unroll
    for (int q = 0; q < PIECES; ++q) {
        const int c = (q * L + lane) * E;
        if (c + E <= a.classes) x[q] = Piece<T, E>::load(z + c);
        else {
#pragma unroll
            for (int k = 0; k < E; ++k) x[q].x[k] = c + k < a.classes ? z[c + k] : from_f32<T>(-INFINITY);
        }
    }
    RowSum v = RowSum::empty();
#pragma unroll
    for (int q = 0; q < PIECES; ++q)
#pragma unroll
        for (int k = 0; k < E; ++k) v.m = fmaxf(v.m, to_f32(x[q].x[k]));
    v.m = max_over<L>(v.m);
    Highest<R> best;
    best.clear();
#pragma unroll
    for (int q = 0; q < PIECES; ++q) {
        const int c = (q * L + lane) * E;
        if (q > 0 && q * L * E >= a.classes) break;      // the same in every lane
        float f[E];
#pragma unroll
        for (int k = 0; k < E; ++k) f[k] = to_f32(x[q].x[k]);
        add_powers(v, f);
        if (R > 0) {
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (c + k < a.classes) best.see(order_key(f[k]), c + k);
        }
    }
    v.s = sum_over<L>(v.s);
    v.t = sum_over<L>(v.t);
    const float log_s = logf(v.s);
    if (live && lane == 0) finish_row(a, row, v, log_s, z);
    if constexpr (R > 0)
        draw_alternatives<T, L, R>(best, a.top, z, 0, 0, a.classes, lane, [&](Rank r, int) { return max_over_lanes<L>(r); }, [&](Rank r, int k) {
            if (live && lane == 0) {
                a.top_idx[row * a.top + k] = rank_class(r);
                a.top_logp[row * a.top + k] = v.log_p(order_value((unsigned)(r >> 32)), log_s);
            }
        });
}

// Elements before the first 16-byte address, at most n: rows that begin elsewhere (odd numbers of 16-bit classes) are read and written a quarter
// slower in pieces across those addresses.
template <class T> __device__ __forceinline__ int elements_to_line(const T *p, int n) {
    const int k = (int)((16u - (unsigned)(reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / (int)sizeof(T);
    return k < n ? k : n;
}

// Long rows, a workgroup each or (parts) several: one pass with a running maximum, m raised to m' multiplies s by f = exp(m - m') and turns t into
// (t + (m - m') s) f.  R: classes that a lane keeps for the alternatives (0: none asked for).  A wavefront now and then raises the bar for
// all its lanes to the a.top-th highest of their best: a class that is not above it has that many before it (all of lower numbers),
// so that most classes are looked at no further than their step's maximum.  Bound by memory: 16,384 x 50,021 in fp16 320 us (5.1 TB/s), the gradient
// 637 us (5.1 TB/s); with ten alternatives in bf16 the vector instructions weigh as much: 4,096 x 100,003 187 to 211 us by card (3.9 to 4.4 TB/s; with the
// exponential's argument chosen element by element 226 where this took 209).
template <class T, int R>
__global__ __launch_bounds__(kLogThreads) void k_logprobs_long(LogArgs a) {
    constexpr int E = kPerPiece<T>, U = 4, L = kLogThreads;
    __shared__ RowSum wave_sum[4];
    __shared__ Rank wave_top[2][4];
    const int lane = threadIdx.x, wave = threadIdx.x / 64;
    const long long unit = (long long)blockIdx.x, row = a.row0 + unit / a.parts;
    const int c0 = (int)(unit % a.parts) * a.part_classes, c1 = c0 + a.part_classes < a.classes ? c0 + a.part_classes : a.classes;
    const T *z = static_cast<const T *>(a.Z) + row * a.ld;
    RowSum v = RowSum::empty();
    Highest<R> best;
    best.clear();
    float bar = NAN;
    auto take = [&](const Piece<T, E> &x, int c, int n) {   // n classes from c on, n <= E
        float f[E], top = -INFINITY;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            f[k] = k < n ? to_f32(x.x[k]) : -INFINITY;
            top = fmaxf(top, f[k]);
        }
        if (top > v.m) v.raise(top);
        add_powers(v, f);
        if constexpr (R > 0) {
            if (!(top <= bar) || v.s != v.s) {   // NaN is above all, and once there shows in the sum
#pragma unroll
                for (int k = 0; k < E; ++k)
                    if (k < n && !(f[k] <= bar)) {
                        best.see(order_key(f[k]), c + k);
                        const float least = best.least();
                        if (least == least && !(bar >= least)) bar = least;     // NaN while the list has room and no bar was raised
                    }
            }
        }
    };
    const int head = elements_to_line(z + c0, c1 - c0);
    if (lane < head) {
        Piece<T, E> x;
        x.x[0] = z[c0 + lane];
        take(x, c0 + lane, 1);
    }
    int c = c0 + head + lane * E, step = 0, next = 1;
    for (; c + (U - 1) * L * E + E <= c1; c += U * L * E) {
        Piece<T, E> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = Piece<T, E>::load(z + c + u * L * E);
#pragma unroll
        for (int u = 0; u < U; ++u) take(x[u], c + u * L * E, E);
        if constexpr (R > 0) {
            if (++step == next) {
                next *= 2;
                if (__popcll(__ballot(1)) == 64) {      // the bits of the a.top-th highest (at most one a lane), from the highest on
                    unsigned at = 0;
                    const unsigned head = best.key[0];
#pragma unroll
                    for (int bit = 31; bit >= 0; --bit) {
                        const unsigned with = at | 1u << bit;
                        if (__popcll(__ballot(head >= with)) >= a.top) at = with;
                    }
                    if (at != 0u && at != 0xFFFFFFFFu) {
                        const float raised = order_value(at);
                        if (!(raised <= bar)) bar = raised;
                    }
                }
            }
        }
    }
    for (; c < c1; c += L * E) {
        Piece<T, E> x;
        if (c + E <= c1) x = Piece<T, E>::load(z + c);
        else {
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (c + k < c1) x.x[k] = z[c + k];
        }
        take(x, c, c1 - c < E ? c1 - c : E);
    }
    const float most = max_over<64>(v.m);
    if (most > v.m) v.raise(most);
    v.s = sum_over<64>(v.s);
    v.t = sum_over<64>(v.t);
    if (threadIdx.x % 64 == 0) wave_sum[wave] = v;
    __syncthreads();
    v = wave_sum[0];
    for (int w = 1; w < 4; ++w) v.join(wave_sum[w]);
    const float log_s = logf(v.s);
    if (lane == 0) {
        if (a.parts > 1) a.part_sum[unit] = v;
        else finish_row(a, row, v, log_s, z);
    }
    if constexpr (R > 0)
        draw_alternatives<T, L, R>(best, a.top, z, c0, head, c1, lane,
            [&](Rank r, int k) {
                r = max_over_lanes<64>(r);
                if (threadIdx.x % 64 == 0) wave_top[k & 1][wave] = r;
                __syncthreads();
                r = wave_top[k & 1][0];
                for (int w = 1; w < 4; ++w) r = wave_top[k & 1][w] > r ? wave_top[k & 1][w] : r;
                return r;
            },
            [&](Rank r, int k) {
                if (lane != 0) return;
                if (a.parts > 1) a.part_top[unit * a.top + k] = r;
                else {
                    a.top_idx[row * a.top + k] = rank_class(r);
                    a.top_logp[row * a.top + k] = v.log_p(order_value((unsigned)(r >> 32)), log_s);
                }
            });
}

// Joins what the parts of long rows left: a wavefront a row.
template <class T> __global__ __launch_bounds__(64) void k_logprobs_join(LogArgs a) {
    __shared__ Rank lists[kMaxParts * SENSEI_MAX_TOP];
    const long long row = blockIdx.x;
    const int lane = threadIdx.x, n = a.parts * a.top;
    for (int k = lane; k < n; k += 64) lists[k] = a.part_top[row * n + k];
    RowSum v = RowSum::empty();
    if (lane < a.parts) v = a.part_sum[row * a.parts + lane];
    const float most = max_over<64>(v.m);
    if (most > v.m) v.raise(most);
    v.s = sum_over<64>(v.s);
    v.t = sum_over<64>(v.t);
    const float log_s = logf(v.s);
    if (lane == 0) finish_row(a, row, v, log_s, static_cast<const T *>(a.Z) + row * a.ld);
    __syncthreads();
    int next = 0;
    const Rank *list = lists + lane * a.top;
    Rank head = a.top > 0 && lane < a.parts ? list[0] : 0;
    for (int k = 0; k < a.top; ++k) {
        const Rank r = max_over_lanes<64>(head);
        if (lane == 0) {
            a.top_idx[row * a.top + k] = rank_class(r);
            a.top_logp[row * a.top + k] = v.log_p(order_value((unsigned)(r >> 32)), log_s);
        }
        if (r != 0 && head == r) head = ++next < a.top ? list[next] : 0;
    }
}

// dZ_j = g ([j = label] - p_j) - h p_j (log p_j + entropy),  p_j = exp((z_j - m) - log s): g and h the gradients of the row's log probability and entropy.
// Read once, written once; classes without a share (-inf) and rows of nothing else get 0 from both terms but the label's own.
template <class T> struct RowGradient {
    RowBase base;
    float inv_s, by_g, h, at_max, g;
    int label;      // -1: none
    bool entropy;
    __device__ __forceinline__ RowGradient(const LogArgs &a, long long row) : base(a.stats[row].x) {
        const float log_s = a.stats[row].y;
        label = a.g_logp ? a.labels[row] : -1;
        if (label >= a.classes) label = -1;
        g = label >= 0 ? a.g_logp[row] : 0.f;
        entropy = a.g_entropy != nullptr;
        h = entropy ? a.g_entropy[row] : 0.f;
        const bool empty = log_s == -INFINITY;     // its powers are all 0
        // a power times what is the same for the row: 1 / s, and -g where there is no entropy term
        inv_s = empty ? 0.f : expf(-base.shift() - log_s);
        by_g = empty ? 0.f : -g * inv_s;
        at_max = -g - h * ((entropy ? a.entropy_in[row] : 0.f) - log_s);
    }
    template <bool DIRECT, int E> __device__ __forceinline__ void terms(const Piece<T, E> &x, float (&f)[E]) const {
#pragma unroll
        for (int k = 0; k < E; ++k) f[k] = base.template power<DIRECT>(to_f32(x.x[k]));
        if (entropy) {
#pragma unroll
            for (int k = 0; k < E; ++k) f[k] = f[k] == 0.f ? 0.f : f[k] * inv_s * fmaf(-h, to_f32(x.x[k]) - base.m, at_max);   // -g - h (log p + entropy)
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k) f[k] *= by_g;
        }
    }
    template <int E> __device__ __forceinline__ void piece(Piece<T, E> &x, int c) const {
        float f[E];
        if (base.direct) terms<true, E>(x, f);     // once a piece, not once an element
        else terms<false, E>(x, f);
        if (label >= c && label < c + E) {
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (c + k == label) f[k] += g;
        }
#pragma unroll
        for (int k = 0; k < E; ++k) x.x[k] = from_f32<T>(f[k]);
    }
    // fewer than a piece
    template <int E> __device__ __forceinline__ void some(const T *z, T *dz, int c, int n) const {
        Piece<T, E> x;
#pragma unroll
        for (int k = 0; k < E; ++k) x.x[k] = z[c + (k < n ? k : 0)];
        piece<E>(x, c);
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (k < n) dz[c + k] = x.x[k];
    }
};

template <class T, int L, int PIECES>
__global__ __launch_bounds__(kLogThreads) void k_logprobs_backward_short(LogArgs a) {
    constexpr int E = kPerPiece<T>;
    const int lane = threadIdx.x % L;
    const long long row = a.row0 + (long long)blockIdx.x * (kLogThreads / L) + threadIdx.x / L;
    if (row >= a.rows) return;
    const T *z = static_cast<const T *>(a.Z) + row * a.ld;
    T *dz = static_cast<T *>(a.dZ) + row * a.lddz;
    Piece<T, E> x[PIECES];
#pragma unroll
    for (int q = 0; q < PIECES; ++q) {
        const int c = (q * L + lane) * E;
        if (c + E <= a.classes) x[q] = Piece<T, E>::load(z + c);
    }
    const RowGradient<T> grad(a, row);
#pragma unroll
    for (int q = 0; q < PIECES; ++q) {
        const int c = (q * L + lane) * E;
        if (c + E <= a.classes) {
            grad.template piece<E>(x[q], c);
            x[q].store(dz + c);
        } else if (c < a.classes) grad.template some<E>(z, dz, c, a.classes - c);
    }
}

template <class T>
__global__ __launch_bounds__(kLogThreads) void k_logprobs_backward_long(LogArgs a) {
    constexpr int E = kPerPiece<T>, U = 4, L = kLogThreads;
    const int lane = threadIdx.x;
    const long long unit = (long long)blockIdx.x, row = a.row0 + unit / a.parts;
    const int c0 = (int)(unit % a.parts) * a.part_classes, c1 = c0 + a.part_classes < a.classes ? c0 + a.part_classes : a.classes;
    const T *z = static_cast<const T *>(a.Z) + row * a.ld;
    T *dz = static_cast<T *>(a.dZ) + row * a.lddz;
    const RowGradient<T> grad(a, row);
    const int head = elements_to_line(dz + c0, c1 - c0);
    if (lane < head) grad.template some<E>(z, dz, c0 + lane, 1);
    int c = c0 + head + lane * E;
    for (; c + (U - 1) * L * E + E <= c1; c += U * L * E) {
        Piece<T, E> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = Piece<T, E>::load(z + c + u * L * E);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            grad.template piece<E>(x[u], c + u * L * E);
            x[u].store(dz + c + u * L * E);
        }
    }
    for (; c < c1; c += L * E) {
        if (c + E <= c1) {
            Piece<T, E> x = Piece<T, E>::load(z + c);
            grad.template piece<E>(x, c);
            x.store(dz + c);
        } else grad.template some<E>(z, dz, c, c1 - c);
    }
}

// Lanes a row and pieces a lane: eight pieces at most, on as few lanes as hold the row so (what is done once a row and lane is shared by more rows);
// more than 64 lanes hold is walked.  Forward, us: 2.45 M rows of 47 (fp32) on 4 lanes / 16 114 / 185, with five alternatives 190 / 392; 100,000 of 349
// (bf16) on 16 / 64 21 / 35; 20,000 of 1,800 (fp32) held by 64 lanes / walked by 256 25 / 43, of 3,900 (bf16) 45 / 75.  The gradient hardly
// minds (283 / 265, 29 / 43, 49 / 52).
struct LogShape { int lanes, pieces; };
LogShape log_shape(int classes, int per_piece) {
    const int all = (classes + per_piece - 1) / per_piece;
    LogShape s{all <= 32 ? 4 : all <= 128 ? 16 : all <= 512 ? 64 : 256, 1};
    while (s.lanes < 256 && s.lanes * s.pieces < all) s.pieces *= 2;
    return s;
}

// A launch has 2^22 workgroups at most (a grid's threads are counted in 32 bits): more rows than those take another one.
template <class Launch> hipError_t by_rows(LogArgs a, int L, Launch launch) {
    const long long slab = ((1ll << 22) / a.parts) * (kLogThreads / L);
    for (a.row0 = 0; a.row0 < a.rows; a.row0 += slab) {
        const long long n = a.rows - a.row0 < slab ? a.rows - a.row0 : slab;
        launch(a, dim3((unsigned)((n * a.parts + kLogThreads / L - 1) / (kLogThreads / L))));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, int L, int PIECES> void launch_short(const LogArgs &a, bool backward, dim3 grid, hipStream_t s) {
    const dim3 block(kLogThreads);
    if (backward) hipLaunchKernelGGL((k_logprobs_backward_short<T, L, PIECES>), grid, block, 0, s, a);
    else if (a.top == 0) hipLaunchKernelGGL((k_logprobs_short<T, L, PIECES, 0>), grid, block, 0, s, a);
    else if (a.top == 1) hipLaunchKernelGGL((k_logprobs_short<T, L, PIECES, 1>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_logprobs_short<T, L, PIECES, 4>), grid, block, 0, s, a);
}
template <class T> void launch_long(const LogArgs &a, bool backward, dim3 grid, hipStream_t s) {
    const dim3 block(kLogThreads);
    if (backward) hipLaunchKernelGGL(k_logprobs_backward_long<T>, grid, block, 0, s, a);
    else if (a.top == 0) hipLaunchKernelGGL((k_logprobs_long<T, 0>), grid, block, 0, s, a);
    else if (a.top == 1) hipLaunchKernelGGL((k_logprobs_long<T, 1>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_logprobs_long<T, 4>), grid, block, 0, s, a);
}

template <class T> hipError_t logprobs_typed(const LogArgs &args, bool backward, hipStream_t s) {
    const LogShape shape = log_shape(args.classes, kPerPiece<T>);
    const hipError_t e = by_rows(args, shape.lanes, [&](const LogArgs &a, dim3 grid) {
#define SENSEI_PIECES(L) \
    (shape.pieces == 1 ? launch_short<T, L, 1>(a, backward, grid, s) : shape.pieces == 2 ? launch_short<T, L, 2>(a, backward, grid, s) \
     : shape.pieces == 4 ? launch_short<T, L, 4>(a, backward, grid, s) : launch_short<T, L, 8>(a, backward, grid, s))
        if (shape.lanes == 4) SENSEI_PIECES(4);
        else if (shape.lanes == 16) SENSEI_PIECES(16);
        else if (shape.lanes == 64) SENSEI_PIECES(64);
        else launch_long<T>(a, backward, grid, s);
#undef SENSEI_PIECES
    });
    if (e != hipSuccess || backward || args.parts == 1) return e;
    hipLaunchKernelGGL(k_logprobs_join<T>, dim3((unsigned)args.rows), dim3(64), 0, s, args);
    return hipGetLastError();
}

// Workgroups that share a row: where the rows alone leave the chip short of workgroups, as many as fill it (1,024) while a part keeps 2,048 classes.  Shared /
// one workgroup each, us: 2 rows of 250,000 with five alternatives 21 / 90, 1 row of 50,000 21 / 30; 64 rows of 50,000 18 / 18.
int log_parts(int64_t rows, int classes, int per_piece) {
    if (log_shape(classes, per_piece).lanes < 256 || rows >= 512) return 1;
    const int64_t want = 1024 / rows, most = classes / 2048, parts = want < most ? want : most;
    return parts < 1 ? 1 : parts > kMaxParts ? kMaxParts : (int)parts;
}

}  // namespace

hipError_t launch_dropout(const sensei_tmat &X, const sensei_tmat *add, double p, uint64_t seed, uint32_t offset, const uint32_t *offset_dev, void *Y, int64_t ldy,
                          hipStream_t s) {
    if (X.rows <= 0 || X.cols <= 0) return hipSuccess;
    DropArgs a = {};
    a.X = X.ptr; a.ldx = X.ld; a.Y = Y; a.ldy = ldy; a.cols = (int)X.cols;
    if (add) { a.add = add->ptr; a.lda = add->ld; }
    a.key = {(unsigned)seed, (unsigned)(seed >> 32), offset, offset_dev, drop_threshold(p), (float)(1.0 / (1.0 - p))};
    switch (X.type) {
    case SENSEI_F32: return add ? dropout_typed<float, true>(a, X.rows, s) : dropout_typed<float, false>(a, X.rows, s);
    case SENSEI_BF16: return add ? dropout_typed<Bf16, true>(a, X.rows, s) : dropout_typed<Bf16, false>(a, X.rows, s);
    default: return add ? dropout_typed<F16, true>(a, X.rows, s) : dropout_typed<F16, false>(a, X.rows, s);
    }
}

size_t logprobs_ws_bytes(int64_t rows, int classes, int top, int type) {
    const int parts = rows > 0 ? log_parts(rows, classes, type == SENSEI_F32 ? 4 : 8) : 1;
    if (parts == 1) return 0;
    return align_up((size_t)rows * parts * sizeof(RowSum), 256) + align_up((size_t)rows * parts * top * sizeof(Rank), 256);
}

hipError_t launch_logprobs(const sensei_tmat &Z, const int32_t *labels, int top, float2 *stats, float *logp, float *entropy, int32_t *top_idx, float *top_logp,
                           void *workspace, hipStream_t s) {
    if (Z.rows <= 0) return hipSuccess;
    LogArgs a = {};
    a.Z = Z.ptr; a.ld = Z.ld; a.rows = Z.rows; a.classes = (int)Z.cols; a.top = top; a.labels = labels;
    a.stats = stats; a.logp = logp; a.entropy = entropy; a.top_idx = top_idx; a.top_logp = top_logp;
    a.parts = log_parts(Z.rows, a.classes, Z.type == SENSEI_F32 ? 4 : 8);
    a.part_classes = (a.classes + a.parts - 1) / a.parts;
    if (a.parts > 1) {   // parts begin where a step of the workgroup does
        a.part_classes = (a.part_classes + 2047) / 2048 * 2048;
        a.parts = (a.classes + a.part_classes - 1) / a.part_classes;
        a.part_sum = static_cast<RowSum *>(workspace);
        a.part_top = reinterpret_cast<Rank *>(static_cast<char *>(workspace) + align_up((size_t)Z.rows * a.parts * sizeof(RowSum), 256));
    }
    switch (Z.type) {
    case SENSEI_F32: return logprobs_typed<float>(a, false, s);
    case SENSEI_BF16: return logprobs_typed<Bf16>(a, false, s);
    default: return logprobs_typed<F16>(a, false, s);
    }
}

hipError_t launch_logprobs_backward(const sensei_tmat &Z, const int32_t *labels, const float2 *stats, const float *g_logp, const float *entropy, const float *g_entropy,
                                    void *dZ, int64_t lddz, hipStream_t s) {
    if (Z.rows <= 0) return hipSuccess;
    LogArgs a = {};
    a.Z = Z.ptr; a.ld = Z.ld; a.rows = Z.rows; a.classes = (int)Z.cols; a.labels = labels; a.stats = const_cast<float2 *>(stats); a.g_logp = g_logp;
    a.entropy_in = entropy; a.g_entropy = g_entropy; a.dZ = dZ; a.lddz = lddz; a.parts = 1;
    if (log_shape(a.classes, Z.type == SENSEI_F32 ? 4 : 8).lanes == 256) {   // a workgroup takes 16,384 classes at most: long rows are shared, whatever their number
        a.part_classes = 16384;
        a.parts = (a.classes + a.part_classes - 1) / a.part_classes;
    }
    switch (Z.type) {
    case SENSEI_F32: return logprobs_typed<float>(a, true, s);
    case SENSEI_BF16: return logprobs_typed<Bf16>(a, true, s);
    default: return logprobs_typed<F16>(a, true, s);
    }
}

}  // namespace sensei
