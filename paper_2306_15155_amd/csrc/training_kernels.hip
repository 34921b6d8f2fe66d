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
// A lane takes 16 bytes (one counter's four elements in fp32, two counters' in 16 bits), UNITS of them a block apart so that their loads are
// under way together; a unit's row and column come from one multiplication (FastDiv).
struct DropArgs {
    const void *X, *add;
    void *Y;
    long long ldx, lda, ldy;
    unsigned row0;             // of this launch
    unsigned units;            // rows * units a row
    int cols;
    FastDiv per_row;
    DropKey key;
};
constexpr int kDropThreads = 256;

template <class T, bool ADD, int UNITS>
__global__ __launch_bounds__(kDropThreads) void k_dropout(DropArgs a) {
    constexpr int E = kPerPiece<T>;
    const unsigned first = blockIdx.x * (unsigned)(kDropThreads * UNITS) + threadIdx.x;
    const unsigned offset = a.key.offset + (a.key.offset_dev ? *a.key.offset_dev : 0u);
    Piece<T, E> x[UNITS], r[UNITS];
    unsigned row[UNITS];
    int col[UNITS], live[UNITS];   // elements of the unit: E, fewer at a row's end, none behind the last unit
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const unsigned at = first + u * kDropThreads;
        row[u] = 0; col[u] = 0; live[u] = 0;
        if (at < a.units) {
            const unsigned i = a.per_row.div(at);
            row[u] = a.row0 + i;
            col[u] = (int)(at - i * a.per_row.d) * E;
            live[u] = a.cols - col[u] < E ? a.cols - col[u] : E;
        }
        const T *px = static_cast<const T *>(a.X) + (long long)row[u] * a.ldx + col[u];
        const T *pr = static_cast<const T *>(a.add) + (ADD ? (long long)row[u] * a.lda + col[u] : 0);
        if (live[u] == E) {
            x[u] = Piece<T, E>::load(px);
            if (ADD) r[u] = Piece<T, E>::load(pr);
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k) {
                if (k < live[u]) {
                    x[u].x[k] = px[k];
                    if (ADD) r[u].x[k] = pr[k];
                }
            }
        }
    }
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        if (live[u] == 0) continue;
        Piece<T, E> y;
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {
            const Words w = philox((unsigned)col[u] / 4 + q, row[u], 0u, offset, a.key.k0, a.key.k1);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int e = 4 * q + k;
                float v = w.w[k] < a.key.threshold ? 0.f : to_f32(x[u].x[e]) * a.key.keep_scale;
                if (ADD) v += to_f32(r[u].x[e]);
                y.x[e] = from_f32<T>(v);
            }
        }
        T *py = static_cast<T *>(a.Y) + (long long)row[u] * a.ldy + col[u];
        if (live[u] == E) y.store(py);
        else {
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (k < live[u]) py[k] = y.x[k];
        }
    }
}

template <class T, bool ADD> hipError_t dropout_units(DropArgs a, long long rows, hipStream_t s) {
    const unsigned per_row = (unsigned)((a.cols + kPerPiece<T> - 1) / kPerPiece<T>);
    a.per_row = FastDiv::of(per_row);
    const long long slab = (0x7FFFFFFFll - 4 * kDropThreads) / per_row;   // unit numbers of a launch stay below 2^31
    for (long long r0 = 0; r0 < rows; r0 += slab) {
        const long long n = rows - r0 < slab ? rows - r0 : slab;
        a.row0 = (unsigned)r0;
        a.units = (unsigned)(n * per_row);
        // four units a lane once that still fills the chip several times over
        if (a.units >= 4u * kDropThreads * 2048) hipLaunchKernelGGL((k_dropout<T, ADD, 4>), dim3((a.units + 4 * kDropThreads - 1) / (4 * kDropThreads)), dim3(kDropThreads), 0, s, a);
        else hipLaunchKernelGGL((k_dropout<T, ADD, 1>), dim3((a.units + kDropThreads - 1) / kDropThreads), dim3(kDropThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// -------------------------------------------------------------------------------------------------------- log probabilities of labels

// One row of C logits z, in one pass: with a running maximum m,
//     s = sum exp(z - m),  t = sum (z - m) exp(z - m);   lse = m + log s,  entropy = log s - t / s,  log p_j = z_j - lse,
// m raised to m' multiplies s by f = exp(m - m') and turns t into (t + (m - m') s) f.  Classes at -inf have no share (and add 0 to t); a
// row of nothing else has lse = -inf.
struct RowSum {
    float m, s, t;
    __device__ __forceinline__ static RowSum empty() { return {-INFINITY, 0.f, 0.f}; }
    __device__ __forceinline__ void raise(float top) {   // top >= m, not both -inf
        const float d = m - top;
        if (m > -INFINITY) {
            const float f = exp_neg(d);
            t = f == 0.f ? 0.f : fmaf(d, s, t) * f;   // d may be as low as a type's lowest value
            s *= f;
        }
        m = top;
    }
    __device__ __forceinline__ void join(const RowSum &o) {
        const float top = fmaxf(m, o.m);
        if (top > -INFINITY) {
            RowSum b = o;
            raise(top);
            b.raise(top);
            s += b.s;
            t += b.t;
        } else {   // nothing but -inf and NaN so far
            s += o.s;
            t += o.t;
        }
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
constexpr int kLogThreads = 256;

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

template <int L> __device__ __forceinline__ Rank max_over_lanes(Rank r) {
#pragma unroll
    for (int d = (L < 64 ? L : 64) / 2; d > 0; d >>= 1) {
        const Rank o = __shfl_xor(r, d, 64);
        r = o > r ? o : r;
    }
    return r;
}
template <int L> __device__ __forceinline__ RowSum join_lanes(RowSum v) {
#pragma unroll
    for (int d = (L < 64 ? L : 64) / 2; d > 0; d >>= 1) v.join({__shfl_xor(v.m, d, 64), __shfl_xor(v.s, d, 64), __shfl_xor(v.t, d, 64)});
    return v;
}

template <class T> __device__ __forceinline__ void finish_row(const LogArgs &a, long long row, const RowSum &v, float log_s, const T *z) {
    if (a.stats) a.stats[row] = make_float2(v.m, log_s);
    if (a.entropy) a.entropy[row] = v.s == 0.f ? 0.f : log_s - v.t / v.s;
    if (a.logp) {
        const int y = a.labels[row];
        a.logp[row] = y >= 0 && y < a.classes ? v.log_p(to_f32(z[y]), log_s) : 0.f;
    }
}

// L lanes a row (4, 16, 64, or a workgroup's 256), 16 bytes a lane and step.  R: classes a lane keeps for the alternatives (0: none asked for); the
// alternatives are then drawn one after the other, each the highest head of all lanes' lists.  A lane whose list was drawn empty goes over its
// classes again for those behind the last one drawn: rare (more than R of a row's highest in one lane) and exact.
template <class T, int L, int R>
__global__ __launch_bounds__(kLogThreads) void k_logprobs(LogArgs a) {
    constexpr int E = kPerPiece<T>, U = 4;
    __shared__ RowSum wave_sum[4];
    __shared__ Rank wave_top[2][4];
    const int lane = threadIdx.x % L, wave = threadIdx.x / 64;
    const long long unit = (long long)blockIdx.x * (kLogThreads / L) + threadIdx.x / L;
    const long long row = a.row0 + (L == 256 ? unit / a.parts : unit);
    const int part = L == 256 ? (int)(unit % a.parts) : 0;
    const bool live = row < a.rows;      // whole groups of lanes; nobody leaves before the workgroup's exchanges
    const T *z = static_cast<const T *>(a.Z) + (live ? row : 0) * a.ld;
    const int c0 = L == 256 ? part * a.part_classes : 0;
    const int c1 = !live ? c0 : L == 256 && c0 + a.part_classes < a.classes ? c0 + a.part_classes : a.classes;
    RowSum v = RowSum::empty();
    Highest<R> best;
    best.clear();
    auto take = [&](const T *x, int c, int n) {   // n classes from c on, n <= E
        float f[E], top = -INFINITY;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            f[k] = k < n ? to_f32(x[k]) : -INFINITY;
            top = fmaxf(top, f[k]);
        }
        if (top > v.m) v.raise(top);
        const float base = v.m > -INFINITY ? v.m : 0.f;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const float d = f[k] - base, e = exp_neg(d);
            v.s += e;
            v.t = fmaf(e, fmaxf(d, -FLT_MAX), v.t);
        }
        if (R > 0) {
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (k < n) best.see(order_key(f[k]), c + k);
        }
    };
    int c = c0 + lane * E;
    for (; c + (U - 1) * L * E + E <= c1; c += U * L * E) {
        Piece<T, E> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = Piece<T, E>::load(z + c + u * L * E);
#pragma unroll
        for (int u = 0; u < U; ++u) take(x[u].x, c + u * L * E, E);
    }
    for (; c < c1; c += L * E) {
        if (c + E <= c1) {
            const Piece<T, E> x = Piece<T, E>::load(z + c);
            take(x.x, c, E);
        } else {
            T x[E];
#pragma unroll
            for (int k = 0; k < E; ++k) x[k] = z[c + k < c1 ? c + k : c1 - 1];
            take(x, c, c1 - c);
        }
    }
    v = join_lanes<L>(v);
    if (L == 256) {
        if (threadIdx.x % 64 == 0) wave_sum[wave] = v;
        __syncthreads();
        v = wave_sum[0];
        for (int w = 1; w < 4; ++w) v.join(wave_sum[w]);
    }
    const bool whole = L < 256 || a.parts == 1;
    const float log_s = logf(v.s);
    if (live && lane == 0) {
        if (!whole) a.part_sum[unit] = v;
        else finish_row(a, row, v, log_s, z);
    }
    if constexpr (R > 0) {
        int mine = 0;                          // drawn from this lane
        for (int k = 0; k < a.top; ++k) {
            Rank r = max_over_lanes<L>(best.head());
            if (L == 256) {
                if (threadIdx.x % 64 == 0) wave_top[k & 1][wave] = r;
                __syncthreads();
                r = wave_top[k & 1][0];
                for (int w = 1; w < 4; ++w) r = wave_top[k & 1][w] > r ? wave_top[k & 1][w] : r;
            }
            if (live && lane == 0) {
                if (!whole) a.part_top[unit * a.top + k] = r;
                else {
                    a.top_idx[row * a.top + k] = rank_class(r);
                    a.top_logp[row * a.top + k] = v.log_p(order_value((unsigned)(r >> 32)), log_s);
                }
            }
            if (r != 0 && best.head() == r) {
                best.pop();
                if (++mine % R == 0 && k + 1 < a.top) {
                    for (int cc = c0 + lane * E; cc < c1; cc += L * E)
                        for (int e = 0; e < E && cc + e < c1; ++e) {
                            const unsigned key = order_key(to_f32(z[cc + e]));
                            if (rank_of(key, cc + e) < r) best.see(key, cc + e);
                        }
                }
            }
        }
    }
}

// Joins what the parts of long rows left: a wavefront a row.
template <class T> __global__ __launch_bounds__(64) void k_logprobs_join(LogArgs a) {
    const long long row = blockIdx.x;
    const int lane = threadIdx.x;
    RowSum v = RowSum::empty();
    if (lane < a.parts) v = a.part_sum[row * a.parts + lane];
    v = join_lanes<64>(v);
    const float log_s = logf(v.s);
    if (lane == 0) finish_row(a, row, v, log_s, static_cast<const T *>(a.Z) + row * a.ld);
    int next = 0;
    const Rank *list = a.part_top + (row * a.parts + lane) * a.top;
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
template <class T, int L>
__global__ __launch_bounds__(kLogThreads) void k_logprobs_backward(LogArgs a) {
    constexpr int E = kPerPiece<T>, U = 4;
    const int lane = threadIdx.x % L;
    const long long unit = (long long)blockIdx.x * (kLogThreads / L) + threadIdx.x / L;
    const long long row = a.row0 + (L == 256 ? unit / a.parts : unit);
    if (row >= a.rows) return;
    const int c0 = L == 256 ? (int)(unit % a.parts) * a.part_classes : 0;
    const int c1 = L == 256 && c0 + a.part_classes < a.classes ? c0 + a.part_classes : a.classes;
    const T *z = static_cast<const T *>(a.Z) + row * a.ld;
    T *dz = static_cast<T *>(a.dZ) + row * a.lddz;
    const int y = a.g_logp ? a.labels[row] : -1;
    const bool has = y >= 0 && y < a.classes;
    const float2 st = a.stats[row];
    const float g = has ? a.g_logp[row] : 0.f, h = a.g_entropy ? a.g_entropy[row] : 0.f, ent = a.g_entropy ? a.entropy_in[row] : 0.f;
    const bool empty = st.y == -INFINITY;
    auto one = [&](float f, int c) {
        const float lp = (f - st.x) - st.y, p = empty ? 0.f : exp_neg(lp);
        float d = -g * p;
        if (a.g_entropy) d = fmaf(-h * p, fmaxf(lp, -FLT_MAX) + ent, d);
        if (p == 0.f) d = 0.f;
        return has && c == y ? d + g : d;
    };
    int c = c0 + lane * E;
    for (; c + (U - 1) * L * E + E <= c1; c += U * L * E) {
        Piece<T, E> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = Piece<T, E>::load(z + c + u * L * E);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int k = 0; k < E; ++k) x[u].x[k] = from_f32<T>(one(to_f32(x[u].x[k]), c + u * L * E + k));
            x[u].store(dz + c + u * L * E);
        }
    }
    for (; c < c1; c += L * E) {
        if (c + E <= c1) {
            Piece<T, E> x = Piece<T, E>::load(z + c);
#pragma unroll
            for (int k = 0; k < E; ++k) x.x[k] = from_f32<T>(one(to_f32(x.x[k]), c + k));
            x.store(dz + c);
        } else {
            for (int k = c; k < c1; ++k) dz[k] = from_f32<T>(one(to_f32(z[k]), k));
        }
    }
}

// Lanes a row: the fewest that take it in eight steps at most.
int log_lanes(int classes, int per_piece) {
    const int pieces = (classes + per_piece - 1) / per_piece;
    return pieces <= 8 ? 4 : pieces <= 64 ? 16 : pieces <= 512 ? 64 : 256;
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

template <class T, int L> void launch_log(const LogArgs &a, dim3 grid, hipStream_t s) {
    if (a.top == 0) hipLaunchKernelGGL((k_logprobs<T, L, 0>), grid, dim3(kLogThreads), 0, s, a);
    else if (a.top == 1) hipLaunchKernelGGL((k_logprobs<T, L, 1>), grid, dim3(kLogThreads), 0, s, a);
    else hipLaunchKernelGGL((k_logprobs<T, L, 4>), grid, dim3(kLogThreads), 0, s, a);
}

template <class T> hipError_t logprobs_typed(const LogArgs &args, hipStream_t s) {
    const int L = log_lanes(args.classes, kPerPiece<T>);
    const hipError_t e = by_rows(args, L, [&](const LogArgs &a, dim3 grid) {
        if (L == 4) launch_log<T, 4>(a, grid, s);
        else if (L == 16) launch_log<T, 16>(a, grid, s);
        else if (L == 64) launch_log<T, 64>(a, grid, s);
        else launch_log<T, 256>(a, grid, s);
    });
    if (e != hipSuccess || args.parts == 1) return e;
    hipLaunchKernelGGL(k_logprobs_join<T>, dim3((unsigned)args.rows), dim3(64), 0, s, args);
    return hipGetLastError();
}

template <class T> hipError_t logprobs_backward_typed(LogArgs args, hipStream_t s) {
    const int L = log_lanes(args.classes, kPerPiece<T>);
    if (L == 256) {   // a workgroup takes 16,384 classes at most: long rows are shared, whatever their number
        args.part_classes = 16384;
        args.parts = (args.classes + args.part_classes - 1) / args.part_classes;
    }
    return by_rows(args, L, [&](const LogArgs &a, dim3 grid) {
        const dim3 block(kLogThreads);
        if (L == 4) hipLaunchKernelGGL((k_logprobs_backward<T, 4>), grid, block, 0, s, a);
        else if (L == 16) hipLaunchKernelGGL((k_logprobs_backward<T, 16>), grid, block, 0, s, a);
        else if (L == 64) hipLaunchKernelGGL((k_logprobs_backward<T, 64>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((k_logprobs_backward<T, 256>), grid, block, 0, s, a);
    });
}

// Workgroups that share a row: where the rows alone leave the chip short of workgroups, as many as fill it (1,024) while a part keeps 8,192 classes.
int log_parts(int64_t rows, int classes, int per_piece) {
    if (log_lanes(classes, per_piece) < 256 || rows >= 512) return 1;
    int64_t parts = 1024 / rows, most = classes / 8192;
    if (parts > most) parts = most;
    return parts < 1 ? 1 : parts > 64 ? 64 : (int)parts;
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
    case SENSEI_F32: return add ? dropout_units<float, true>(a, X.rows, s) : dropout_units<float, false>(a, X.rows, s);
    case SENSEI_BF16: return add ? dropout_units<Bf16, true>(a, X.rows, s) : dropout_units<Bf16, false>(a, X.rows, s);
    default: return add ? dropout_units<F16, true>(a, X.rows, s) : dropout_units<F16, false>(a, X.rows, s);
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
    case SENSEI_F32: return logprobs_typed<float>(a, s);
    case SENSEI_BF16: return logprobs_typed<Bf16>(a, s);
    default: return logprobs_typed<F16>(a, s);
    }
}

hipError_t launch_logprobs_backward(const sensei_tmat &Z, const int32_t *labels, const float2 *stats, const float *g_logp, const float *entropy, const float *g_entropy,
                                    void *dZ, int64_t lddz, hipStream_t s) {
    if (Z.rows <= 0) return hipSuccess;
    LogArgs a = {};
    a.Z = Z.ptr; a.ld = Z.ld; a.rows = Z.rows; a.classes = (int)Z.cols; a.labels = labels; a.stats = const_cast<float2 *>(stats); a.g_logp = g_logp;
    a.entropy_in = entropy; a.g_entropy = g_entropy; a.dZ = dZ; a.lddz = lddz; a.parts = 1;
    switch (Z.type) {
    case SENSEI_F32: return logprobs_backward_typed<float>(a, s);
    case SENSEI_BF16: return logprobs_backward_typed<Bf16>(a, s);
    default: return logprobs_backward_typed<F16>(a, s);
    }
}

}  // namespace sensei
