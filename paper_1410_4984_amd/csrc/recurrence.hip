// The gated linear recurrence over packed sequences, and its gradients.
//
//   h_t = a_t h_{t-1} + (1 - a_t) x_t,   a_t = sigmoid(gate_t)        elementwise over D channels
//
// Backwards, with G_t = dL/dh_t as a whole and gamma_t = a_t G_t (what row t hands to the row
// before it):
//   G_t = dh_t + gamma_{t+1},  dx_t = (1 - a_t) G_t,  dgate_t = a_t (1 - a_t) G_t (h_{t-1} - x_t)
// which is the same kind of recurrence, gamma_t = a_t (dh_t + gamma_{t+1}), in the other
// direction.  Both kernels below go through "positions" p = 0, 1, .. in their direction; the
// rows' strides are negative where that is from the last row to the first.
//
// A recurrence y_t = A_t y_{t-1} + B_t is a scan: two neighbouring pieces (A1, B1), (A2, B2) make
// (A1 A2, A2 B1 + B2).  A sequence's first row forgets what came before; its piece has A = -1,
// which stands for that (no product of gates is negative): joined with anything before it, the
// piece stays as it is.  It is a selection and not a product with zero, so that infinities and
// NaN of one sequence never reach the next.
//
// A workgroup takes a tile of rows and channels: a thread holds R rows of 16 bytes (V
// channels), S = 256 / W slices of R rows lie one after the other in time.  The tile is read
// once, each thread joins its rows, the slices are joined in shared memory, and with the state
// before the tile each thread goes through its rows again, in registers.
//
// Short calls: the workgroups of a slab of channels go through the tiles one after the other and
// keep the state in registers (one launch).  Longer ones: a workgroup for each tile, joined by a
// chain in the workspace.  A tile publishes its piece as soon as it has read its rows.  Tiles are
// in groups of 16; the state before a tile is the state after the group before (which that
// group's last tile publishes) joined with the pieces of the tiles before it in its own group, always
// in that order, so the result does not depend on timing.  Every published word
// carries its own validity (it differs from the all-ones pattern that a first kernel writes), so
// no ordering between words is needed.  Tiles are handed out by a counter in the order of the
// rows: a workgroup only waits for tiles with smaller numbers, whose workgroups run already, and
// the first of them waits for none, so every wait ends.
//
// The gate: with s = e / (1 + e), e = exp(-|gate|), the smaller of a and 1 - a is s to full
// relative precision, and h = base + s (other - base) with base the operand of the larger weight.
// A long memory (1 - a of 1e-3) then keeps its digits, which a rounded a times h would lose
// row by row.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "elem.h"
#include "internal.h"

namespace {

using gpps::bf16_t;
using gpps::Elem;

constexpr int kThreads = 256;

template <typename T>
struct RecArgs {
    using A = typename Elem<T>::Acc;
    using S = typename Elem<T>::Store;
    int64_t N, D, B;
    const int64_t *offsets;      // NULL: one sequence of all rows
    int down;                    // positions run from the last row to the first
    // rows at position 0 and their strides from one position to the next
    const S *x, *gate, *h, *dh;
    int64_t sx, sgate, sh, sdh;
    S *out, *dgate;              // forward: h; gradient: dx and dgate
    int64_t sout, sdgate;
    const A *init;               // state before a sequence: h0, or dh_last (NULL: zero)
    const A *h0;                 // gradient: the state before a sequence's first row
    A *fin;                      // state after a sequence: h_last, or dh0 (may be NULL)
    int64_t tiles;               // along the rows
    // the chain, in the workspace: (a, b) of each tile and channel, the state after each group
    unsigned long long *next;    // the next tile to hand out
    A *pieces, *states;
};

constexpr int kGroup = 16;       // tiles of a group

// Words that other workgroups wait for.  A value is never the all-ones pattern (a NaN), which
// stands for "not yet".
template <typename U>
__device__ inline U peek(const U *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename U>
__device__ inline void put(U *p, U v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename U>
__device__ inline U await(const U *p, U v) {
    while (v == ~U(0)) {
        __builtin_amdgcn_s_sleep(1);
        v = peek(p);
    }
    return v;
}

template <typename A> struct Word;
template <> struct Word<float> {
    using U = uint32_t;
    __device__ static U of(float x) {
        const U u = __float_as_uint(x);
        return u == ~U(0) ? 0x7fc00000u : u;
    }
    __device__ static float from(U u) { return __uint_as_float(u); }
};
template <> struct Word<double> {
    using U = unsigned long long;
    __device__ static U of(double x) {
        const U u = (U)__double_as_longlong(x);
        return u == ~U(0) ? 0x7ff8000000000000ull : u;
    }
    __device__ static double from(U u) { return __longlong_as_double((long long)u); }
};

// A piece (a, b): one word of 64 bits in single precision, two in double.
template <typename A> struct Pair;
template <> struct Pair<float> {
    unsigned long long w;
    __device__ void read(const float *p) { w = peek((const unsigned long long *)p); }
    __device__ void wait(const float *p) { w = await((const unsigned long long *)p, w); }
    __device__ float a() const { return __uint_as_float(uint32_t(w)); }
    __device__ float b() const { return __uint_as_float(uint32_t(w >> 32)); }
    __device__ static void write(float *p, float a, float b) {
        put((unsigned long long *)p, (unsigned long long)Word<float>::of(a) | (unsigned long long)Word<float>::of(b) << 32);
    }
};
template <> struct Pair<double> {
    unsigned long long u, v;
    __device__ void read(const double *p) {
        u = peek((const unsigned long long *)p);
        v = peek((const unsigned long long *)p + 1);
    }
    __device__ void wait(const double *p) {
        u = await((const unsigned long long *)p, u);
        v = await((const unsigned long long *)p + 1, v);
    }
    __device__ double a() const { return Word<double>::from(u); }
    __device__ double b() const { return Word<double>::from(v); }
    __device__ static void write(double *p, double a, double b) {
        put((unsigned long long *)p, Word<double>::of(a));
        put((unsigned long long *)p + 1, Word<double>::of(b));
    }
};

__device__ inline float gate_part(float ag) {
    // exp(-|gate|): the product with log2(e) in two parts, so that it keeps its digits
    const float log2e = 1.44269504f, rest = 1.92596299e-8f;
    const float t = -ag * log2e;
    const float lo = ag < 128.0f ? __builtin_fmaf(-ag, log2e, -t) - ag * rest : 0.0f;
    float e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e, lo * 0.693147181f, e);
}
__device__ inline double gate_part(double ag) { return exp(-ag); }

__device__ inline float reciprocal(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ inline double reciprocal(double x) { return 1.0 / x; }

// s = min(a, 1 - a) and r = max(a, 1 - a).
template <typename A>
__device__ inline void gate_of(A g, A &s, A &r) {
    const A e = gate_part(g < A(0) ? -g : g);
    r = reciprocal(A(1) + e);
    s = e * r;
}

template <typename A>
__device__ inline A mix(A g, A s, A h, A x) {
    const A base = g >= A(0) ? h : x, other = g >= A(0) ? x : h;
    return base + s * (other - base);
}
// a times y
template <typename A>
__device__ inline A times_gate(A g, A s, A y) {
    return g >= A(0) ? y - s * y : s * y;
}

// The piece (a1, b1) followed by (a2, b2), into the first.
template <typename A>
__device__ inline void join(A &a1, A &b1, A a2, A b2) {
    const bool fresh = a2 < A(0);
    b1 = fresh ? b2 : a2 * b1 + b2;
    a1 = fresh || a1 < A(0) ? A(-1) : a1 * a2;
}
template <typename A>
__device__ inline A after(A state, A a, A b) {
    return a < A(0) ? b : a * state + b;
}

// Marks, for the positions p0 .. p0 + len - 1 of a tile, which sequence begins or ends there (-1:
// none).  Called by all threads; ends with a barrier.  Offsets that break the contract change
// which rows are marked, never what is accessed.
template <int TR, typename T>
__device__ inline void mark(const RecArgs<T> &a, int64_t p0, int len, int *begins, int *ends, int *found) {
    for (int i = threadIdx.x; i < TR; i += kThreads) begins[i] = ends[i] = -1;
    __syncthreads();
    if (!a.offsets) {
        if (threadIdx.x == 0) {
            if (p0 == 0) begins[0] = 0;
            if (p0 + len == a.N) ends[len - 1] = 0;
        }
        __syncthreads();
        return;
    }
    const int64_t lo = a.down ? a.N - p0 - len : p0, hi = lo + len;      // the tile's rows
    int64_t at = 0;
    if (a.B > kThreads) {
        // the first sequence that begins at `lo` or later, by a wave: 64 places a step
        if (threadIdx.x < 64) {
            int64_t l = 0, r = a.B;                                      // it is in [l, r]
            while (r - l > 0) {
                const int64_t step = (r - l + 63) / 64, i = l + int64_t(threadIdx.x) * step;
                const int below = __popcll(__ballot(i < r && a.offsets[i] < lo));
                const int64_t l2 = below ? l + int64_t(below - 1) * step + 1 : l;
                r = below < 64 && l + int64_t(below) * step < r ? l + int64_t(below) * step : r;
                l = l2 < r ? l2 : r;
            }
            if (threadIdx.x == 0) *found = int(l > 0 ? l - 1 : 0);       // .. and the one before it
        }
        __syncthreads();
        at = *found;
    }
    for (;; at += kThreads) {
        const int64_t b = at + threadIdx.x;
        bool more = false;
        if (b < a.B) {
            const int64_t o = a.offsets[b], e = a.offsets[b + 1];
            if (e > o) {
                const int64_t first = (a.down ? a.N - e : o) - p0, last = (a.down ? a.N - 1 - o : e - 1) - p0;
                if (first >= 0 && first < len) begins[first] = int(b);
                if (last >= 0 && last < len) ends[last] = int(b);
            }
            more = o < hi && threadIdx.x == kThreads - 1 && b + 1 < a.B;
        }
        if (!__syncthreads_or(more)) break;
    }
    __syncthreads();
}

// Empty sequences hand their state on as it is.
template <typename T>
__device__ inline void copy_empty(const RecArgs<T> &a, int64_t b, int64_t c, int n) {
    using A = typename Elem<T>::Acc;
    const int64_t o = a.offsets ? a.offsets[b] : 0, e = a.offsets ? a.offsets[b + 1] : a.N;
    if (e > o) return;
    for (int v = 0; v < n; ++v) a.fin[b * a.D + c + v] = a.init ? a.init[b * a.D + c + v] : A(0);
}

// Before the tiles of a chain: its words, its counter, and the empty sequences.
template <typename T>
__global__ __launch_bounds__(kThreads) void rec_init_kernel(RecArgs<T> a) {
    using A = typename Elem<T>::Acc;
    using U = typename Word<A>::U;
    const int64_t at = int64_t(blockIdx.x) * kThreads + threadIdx.x, all = int64_t(gridDim.x) * kThreads;
    if (at == 0) *a.next = 0;
    const int64_t words = (a.tiles * 2 + (a.tiles + kGroup - 1) / kGroup) * a.D;     // the states lie behind the pieces
    for (int64_t i = at; i < words; i += all) ((U *)a.pieces)[i] = ~U(0);
    if (!a.fin || !a.offsets) return;
    for (int64_t b = at / 64; b < a.B; b += all / 64)
        for (int64_t c = at % 64; c < a.D; c += 64) copy_empty(a, b, c, 1);
}

// The state before tile `tile` of channel c, given by the chain.
template <typename A>
__device__ inline A chain_state(const A *pieces, const A *states, int64_t tile, int64_t D, int64_t c) {
    using U = typename Word<A>::U;
    const int64_t group = tile / kGroup;
    const int before = int(tile % kGroup);
    const U *sp = (const U *)states + (group - 1) * D + c;
    const A *pp = pieces + (group * kGroup * D + c) * 2;
    U w = 0;
    if (group) w = peek(sp);
    Pair<A> q[kGroup - 1];
#pragma unroll
    for (int j = 0; j < kGroup - 1; ++j)
        if (j < before) q[j].read(pp + j * D * 2);
    A state = 0;
    if (group) state = Word<A>::from(await(sp, w));
#pragma unroll
    for (int j = 0; j < kGroup - 1; ++j)
        if (j < before) {
            q[j].wait(pp + j * D * 2);
            state = after(state, q[j].a(), q[j].b());
        }
    return state;
}

template <typename T, bool GRAD, bool CHAIN, int W, int R>
__global__ __launch_bounds__(kThreads) void rec_kernel(RecArgs<T> a) {
    using E = Elem<T>;
    using A = typename E::Acc;
    using S = typename E::Store;
    using Vec = typename gpps::Wide<S, E::V>::type;
    constexpr int V = E::V, kSlices = kThreads / W, kRows = kSlices * R, kCols = W * V;
    __shared__ int begins[kRows], ends[kRows], found;
    __shared__ A piece_a[kSlices][kCols], piece_b[kSlices][kCols], state[kCols];
    __shared__ int64_t ticket;
    const int slice = threadIdx.x / W, lane = threadIdx.x % W;
    const int64_t slabs = (a.D + kCols - 1) / kCols;
    int64_t tile = 0, c0 = int64_t(blockIdx.x) * kCols;
    if (!CHAIN && a.fin) {
        const int64_t c = c0 + lane * V;
        const int n = int(a.D - c < V ? (a.D > c ? a.D - c : 0) : V);
        for (int64_t b = slice; b < a.B; b += kSlices) copy_empty(a, b, c, n);
    }
    A carry = 0;                 // of channel c0 + threadIdx.x, in the first kCols threads
    for (;; ++tile) {
        if (CHAIN) {
            if (threadIdx.x == 0) ticket = (int64_t)atomicAdd(a.next, 1ull);
            __syncthreads();
            tile = ticket / slabs;
            c0 = ticket % slabs * kCols;
        }
        if (tile >= a.tiles) break;
        const int64_t c = c0 + lane * V;
        const int n = int(a.D - c < V ? (a.D > c ? a.D - c : 0) : V);
        const int64_t p0 = tile * kRows;
        const int len = int(a.N - p0 < kRows ? a.N - p0 : kRows);
        // rows of this thread: its part of the tile's, in order
        const int i0 = slice * R;
        const int64_t p = p0 + i0;
        Vec gr[R], ur[R];        // gate, and what it weighs: x, or dh
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int m = i0 + r < len ? n : 0;
            gr[r] = gpps::load_some<S, V>(a.gate + (p + r) * a.sgate + c, m);
            if (!GRAD) ur[r] = gpps::load_some<S, V>(a.x + (p + r) * a.sx + c, m);
            else if (a.dh) ur[r] = gpps::load_some<S, V>(a.dh + (p + r) * a.sdh + c, m);
            else ur[r] = 0;
        }
        mark<kRows>(a, p0, len, begins, ends, &found);
        A pa[V], pb[V];
#pragma unroll
        for (int v = 0; v < V; ++v) pa[v] = 1, pb[v] = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (i0 + r >= len) continue;
            const int q = begins[i0 + r];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const A g = E::up(gr[r][v]), u = E::up(ur[r][v]);
                A s, rr;
                gate_of(g, s, rr);
                if (q >= 0) {
                    pb[v] = a.init && v < n ? a.init[q * a.D + c + v] : A(0);
                    pa[v] = -1;
                }
                pb[v] = GRAD ? times_gate(g, s, u + pb[v]) : mix(g, s, pb[v], u);
                pa[v] = pa[v] < A(0) ? pa[v] : times_gate(g, s, pa[v]);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            piece_a[slice][lane * V + v] = pa[v];
            piece_b[slice][lane * V + v] = pb[v];
        }
        __syncthreads();
        if (threadIdx.x < kCols) {
            // each slice gets the piece before it within the tile
            A ta = 1, tb = 0;
            for (int i = 0; i < kSlices; ++i) {
                const A na = piece_a[i][threadIdx.x], nb = piece_b[i][threadIdx.x];
                piece_a[i][threadIdx.x] = ta;
                piece_b[i][threadIdx.x] = tb;
                join(ta, tb, na, nb);
            }
            const int64_t ch = c0 + threadIdx.x;
            if (!CHAIN) {
                state[threadIdx.x] = carry;
                carry = after(carry, ta, tb);
            } else if (ch < a.D) {
                Pair<A>::write(a.pieces + (tile * a.D + ch) * 2, ta, tb);
                const A y = chain_state(a.pieces, a.states, tile, a.D, ch);
                state[threadIdx.x] = y;
                if (tile % kGroup == kGroup - 1)
                    put((typename Word<A>::U *)a.states + tile / kGroup * a.D + ch, Word<A>::of(after(y, ta, tb)));
            }
        }
        __syncthreads();
        A y[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
            y[v] = after(state[lane * V + v], piece_a[slice][lane * V + v], piece_b[slice][lane * V + v]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = i0 + r;
            if (i >= len) continue;
            const int q = begins[i], z = ends[i];
            Vec o1, o2, xr, hr;
            if (GRAD) {
                xr = gpps::load_some<S, V>(a.x + (p + r) * a.sx + c, n);
                hr = gpps::load_some<S, V>(a.h + (p + r + 1) * a.sh + c, z >= 0 || p + r + 1 >= a.N ? 0 : n);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const A g = E::up(gr[r][v]), u = E::up(ur[r][v]);
                A s, rr;
                gate_of(g, s, rr);
                if (q >= 0) y[v] = a.init && v < n ? a.init[q * a.D + c + v] : A(0);
                if (!GRAD) {
                    y[v] = mix(g, s, y[v], u);
                    o1[v] = E::down(y[v]);
                } else {
                    const A G = u + y[v];
                    A before = E::up(hr[v]);
                    if (z >= 0) before = a.h0 && v < n ? a.h0[z * a.D + c + v] : A(0);
                    o1[v] = E::down((g >= A(0) ? s : rr) * G);
                    o2[v] = E::down(s * rr * G * (before - E::up(xr[v])));
                    y[v] = times_gate(g, s, G);
                }
                if (z >= 0 && a.fin && v < n) a.fin[z * a.D + c + v] = y[v];
            }
            gpps::store_some<S, V>(a.out + (p + r) * a.sout + c, n, o1);
            if (GRAD) gpps::store_some<S, V>(a.dgate + (p + r) * a.sdgate + c, n, o2);
        }
        __syncthreads();         // the marks and pieces are written anew
    }
}

constexpr int kLanes = 16;       // W: 256 bytes of a row
constexpr int kSlicesOf = kThreads / kLanes;
constexpr int kRowsMany = 16, kRowsFew = 4;

// How a call is cut: rows of a thread, tiles along the rows, and whether they are chained.
struct Cut {
    int rows;
    int64_t tiles;
    bool chain;
};

Cut cut(int64_t N, int64_t D, int V) {
    const int64_t slabs = (D + kLanes * V - 1) / (kLanes * V);
    const int64_t few = kSlicesOf * kRowsFew, many = kSlicesOf * kRowsMany;
    if (N <= 2 * few) return Cut{kRowsFew, (N + few - 1) / few, false};
    if ((N + many - 1) / many * slabs < 512) return Cut{kRowsFew, (N + few - 1) / few, true};
    return Cut{kRowsMany, (N + many - 1) / many, true};
}

constexpr size_t kCounterBytes = 256;

template <typename T, bool GRAD>
hipError_t launch(RecArgs<T> a, void *ws, hipStream_t st) {
    using A = typename Elem<T>::Acc;
    constexpr int kCols = kLanes * Elem<T>::V;
    const int64_t slabs = (a.D + kCols - 1) / kCols;
    const Cut k = cut(a.N, a.D, Elem<T>::V);
    a.tiles = k.tiles;
    if (!k.chain) {
        gpps::TimedScope ts(st, GRAD ? "recurrence_grad" : "recurrence_fwd");
        rec_kernel<T, GRAD, false, kLanes, kRowsFew><<<unsigned(slabs), kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
    a.next = static_cast<unsigned long long *>(ws);
    a.pieces = reinterpret_cast<A *>(static_cast<char *>(ws) + kCounterBytes);
    a.states = a.pieces + 2 * a.tiles * a.D;
    {
        gpps::TimedScope ts(st, "recurrence_init");
        const int64_t words = 3 * a.tiles * a.D;
        rec_init_kernel<T><<<unsigned(std::min<int64_t>((words + kThreads * 8 - 1) / (kThreads * 8), 2048)), kThreads, 0, st>>>(a);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    gpps::TimedScope ts(st, GRAD ? "recurrence_grad" : "recurrence_fwd");
    const unsigned blocks = unsigned(std::min<int64_t>(a.tiles * slabs, gpps::kMaxBlocks));
    if (k.rows == kRowsFew)
        rec_kernel<T, GRAD, true, kLanes, kRowsFew><<<blocks, kThreads, 0, st>>>(a);
    else
        rec_kernel<T, GRAD, true, kLanes, kRowsMany><<<blocks, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool valid_dtype(gpps_dtype dt) { return dt == GPPS_F32 || dt == GPPS_F64 || dt == GPPS_BF16; }

bool valid_shape(int64_t N, int64_t B, int64_t D) {
    return N >= 0 && B >= 1 && B <= INT32_MAX && D >= 1 && D <= GPPS_MAX_WIDTH && N <= (int64_t(1) << 40) / D;
}

size_t elem_size(gpps_dtype dt) { return dt == GPPS_F64 ? 8 : dt == GPPS_BF16 ? 2 : 4; }
size_t acc_size(gpps_dtype dt) { return dt == GPPS_F64 ? 8 : 4; }

gpps_status check_common(gpps_dtype dt, int64_t N, int64_t B, int64_t D, const void *offsets, int flags,
                         const void *workspace, size_t workspace_bytes) {
    if (!valid_dtype(dt)) return GPPS_ERR_DTYPE;
    if (!valid_shape(N, B, D) || (!offsets && B != 1)) return GPPS_ERR_SHAPE;
    if (!workspace) return GPPS_ERR_NULL;
    if (!aligned(workspace, 256) || !aligned(offsets, 8)) return GPPS_ERR_ALIGN;
    if (workspace_bytes < gpps_recurrence_workspace_bytes(dt, N, B, D)) return GPPS_ERR_WORKSPACE;
    if (flags & ~GPPS_REVERSE) return GPPS_ERR_PATH;
    return GPPS_OK;
}

// The row at position 0 and the stride between positions.
template <typename S>
void rows(const void *p, int64_t N, int64_t ld, bool down, S *&first, int64_t &stride) {
    first = p ? (S *)const_cast<void *>(p) + (down && N ? (N - 1) * ld : 0) : nullptr;
    stride = down ? -ld : ld;
}

template <typename T>
hipError_t forward(int64_t N, int64_t B, int64_t D, const void *x, int64_t ldx, const void *gate, int64_t ldg,
                   const int64_t *offsets, const void *h0, void *h, int64_t ldh, void *h_last, bool reverse,
                   void *ws, hipStream_t st) {
    using A = typename Elem<T>::Acc;
    RecArgs<T> a{};
    a.N = N, a.D = D, a.B = B, a.offsets = offsets, a.down = reverse;
    rows(x, N, ldx, reverse, a.x, a.sx);
    rows(gate, N, ldg, reverse, a.gate, a.sgate);
    rows(h, N, ldh, reverse, a.out, a.sout);
    a.init = (const A *)h0, a.fin = (A *)h_last;
    return launch<T, false>(a, ws, st);
}

template <typename T>
hipError_t gradient(int64_t N, int64_t B, int64_t D, const void *x, int64_t ldx, const void *gate, int64_t ldg,
                    const void *h, int64_t ldh, const void *dh, int64_t lddh, const int64_t *offsets,
                    const void *h0, const void *dh_last, void *dx, int64_t lddx, void *dgate, int64_t lddg,
                    void *dh0, bool reverse, void *ws, hipStream_t st) {
    using A = typename Elem<T>::Acc;
    RecArgs<T> a{};
    const bool down = !reverse;  // the gradient runs against the recurrence
    a.N = N, a.D = D, a.B = B, a.offsets = offsets, a.down = down;
    rows(x, N, ldx, down, a.x, a.sx);
    rows(gate, N, ldg, down, a.gate, a.sgate);
    rows(h, N, ldh, down, a.h, a.sh);
    rows(dh, N, lddh, down, a.dh, a.sdh);
    rows(dx, N, lddx, down, a.out, a.sout);
    rows(dgate, N, lddg, down, a.dgate, a.sdgate);
    a.init = (const A *)dh_last, a.h0 = (const A *)h0, a.fin = (A *)dh0;
    return launch<T, true>(a, ws, st);
}

}  // namespace

extern "C" {

size_t gpps_recurrence_workspace_bytes(gpps_dtype dt, int64_t N, int64_t B, int64_t D) {
    if (!valid_dtype(dt) || !valid_shape(N, B, D)) return 0;
    const Cut k = cut(N, D, int(16 / elem_size(dt)));
    if (!k.chain) return kCounterBytes;
    const int64_t words = (2 * k.tiles + (k.tiles + kGroup - 1) / kGroup) * D;
    return gpps::align_up(kCounterBytes + size_t(words) * acc_size(dt), 256);
}

gpps_status gpps_recurrence(gpps_dtype dt, int64_t N, int64_t B, int64_t D, const void *x, int64_t ldx,
                            const void *gate, int64_t ldg, const int64_t *offsets, const void *h0, void *h,
                            int64_t ldh, void *h_last, int flags, void *workspace, size_t workspace_bytes,
                            void *stream) {
    if (gpps_status r = check_common(dt, N, B, D, offsets, flags, workspace, workspace_bytes)) return r;
    if (ldx < D || ldg < D || ldh < D) return GPPS_ERR_SHAPE;
    if (N && (!x || !gate || !h)) return GPPS_ERR_NULL;
    for (const void *p : {x, gate, (const void *)h})
        if (!aligned(p, elem_size(dt))) return GPPS_ERR_ALIGN;
    for (const void *p : {h0, (const void *)h_last})
        if (!aligned(p, acc_size(dt))) return GPPS_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool rev = flags & GPPS_REVERSE;
    const hipError_t e =
        dt == GPPS_F32   ? forward<float>(N, B, D, x, ldx, gate, ldg, offsets, h0, h, ldh, h_last, rev, workspace, st)
        : dt == GPPS_F64 ? forward<double>(N, B, D, x, ldx, gate, ldg, offsets, h0, h, ldh, h_last, rev, workspace, st)
                         : forward<bf16_t>(N, B, D, x, ldx, gate, ldg, offsets, h0, h, ldh, h_last, rev, workspace, st);
    return e == hipSuccess ? GPPS_OK : GPPS_ERR_HIP;
}

gpps_status gpps_recurrence_grads(gpps_dtype dt, int64_t N, int64_t B, int64_t D, const void *x, int64_t ldx,
                                  const void *gate, int64_t ldg, const void *h, int64_t ldh, const void *dh,
                                  int64_t lddh, const int64_t *offsets, const void *h0, const void *dh_last,
                                  void *dx, int64_t lddx, void *dgate, int64_t lddg, void *dh0, int flags,
                                  void *workspace, size_t workspace_bytes, void *stream) {
    if (gpps_status r = check_common(dt, N, B, D, offsets, flags, workspace, workspace_bytes)) return r;
    if (ldx < D || ldg < D || ldh < D || (dh && lddh < D) || lddx < D || lddg < D) return GPPS_ERR_SHAPE;
    if (N && (!x || !gate || !h || !dx || !dgate)) return GPPS_ERR_NULL;
    for (const void *p : {x, gate, h, dh, (const void *)dx, (const void *)dgate})
        if (!aligned(p, elem_size(dt))) return GPPS_ERR_ALIGN;
    for (const void *p : {h0, dh_last, (const void *)dh0})
        if (!aligned(p, acc_size(dt))) return GPPS_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool rev = flags & GPPS_REVERSE;
    const hipError_t e =
        dt == GPPS_F32 ? gradient<float>(N, B, D, x, ldx, gate, ldg, h, ldh, dh, lddh, offsets, h0, dh_last, dx,
                                         lddx, dgate, lddg, dh0, rev, workspace, st)
        : dt == GPPS_F64
            ? gradient<double>(N, B, D, x, ldx, gate, ldg, h, ldh, dh, lddh, offsets, h0, dh_last, dx, lddx, dgate,
                               lddg, dh0, rev, workspace, st)
            : gradient<bf16_t>(N, B, D, x, ldx, gate, ldg, h, ldh, dh, lddh, offsets, h0, dh_last, dx, lddx, dgate,
                               lddg, dh0, rev, workspace, st);
    return e == hipSuccess ? GPPS_OK : GPPS_ERR_HIP;
}

}  // extern "C"
