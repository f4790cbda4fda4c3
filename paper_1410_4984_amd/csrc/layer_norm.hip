// Layer norm over the rows of x [N x D] and its gradients.
//
//   mean = sum x / D,  rstd = (sum (x - mean)^2 / D + eps)^-1/2,  y = (x - mean) rstd w + b
//   xh = (x - mean) rstd,  u = dy w
//   dx = rstd (u - sum u / D - xh sum(u xh) / D),  dw = sum_n dy xh,  db = sum_n dy
//
// Both are bound by the rows' bytes: x and y, or x, dy and dx, once each.  A row is kept in
// registers between the sums and the output, so nothing is read twice, and the variance is
// that of the differences from the mean (not a difference of two sums, which loses the digits
// that a row with a large mean shares).
//
// A group of TPR threads takes a row, R vectors of 16 bytes each: 8, 16 or 32 lanes of a wave
// for narrow rows, a wave, four waves or sixteen.  Groups go through the rows with a stride, so
// the weights are loaded once.  In the gradient they also carry their columns' dw and db in
// registers; a workgroup joins its groups' sums in a fixed order and writes one partial row,
// and a second kernel adds those up.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "elem.h"
#include "internal.h"

namespace {

using gpps::bf16_t;
using gpps::Elem;

template <typename T>
struct LnArgs {
    using A = typename Elem<T>::Acc;
    using S = typename Elem<T>::Store;
    int64_t N, D;
    const S *x;
    int64_t ldx;
    const A *w, *b;
    A eps;
    S *y;                        // forward: y; gradient: dx
    int64_t ldy;
    A *mean, *rstd;
    const S *dy;
    int64_t lddy;
    A *dw, *db;                  // gradient: where the sums of workgroup 0, 1, .. go, `step` apart
    int64_t step;
    int accumulate;              // dw, db are added to
};

// Sums over the TPR threads of a row, the same in each.  `turn` alternates between two sets of
// slots, so that one barrier a row is enough.
template <typename A, int TPR, int K>
__device__ inline void row_sum(A (&x)[K], A *slots, int turn) {
    constexpr int kLanes = TPR < 64 ? TPR : 64;
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = gpps::lanes_sum(x[k], kLanes);
    if constexpr (TPR > 64) {
        constexpr int kWaves = TPR / 64;
        A *s = slots + turn * kWaves * K;
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) s[threadIdx.x / 64 * K + k] = x[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            A t = 0;
            for (int i = 0; i < kWaves; ++i) t += s[i * K + k];
            x[k] = t;
        }
    }
}

template <typename T, int TPR, int R>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void ln_fwd_kernel(LnArgs<T> a) {
    using E = Elem<T>;
    using A = typename E::Acc;
    using S = typename E::Store;
    constexpr int V = E::V, kThreads = TPR < 256 ? 256 : TPR, kGroups = kThreads / TPR;
    __shared__ A slots[TPR > 64 ? 4 * (TPR / 64) : 1];
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    A w[R][V], b[R][V];
    int n[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t c = (int64_t(r) * TPR + lane) * V;
        n[r] = int(a.D - c < V ? (a.D > c ? a.D - c : 0) : V);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            w[r][v] = a.w && v < n[r] ? a.w[c + v] : A(1);
            b[r][v] = a.b && v < n[r] ? a.b[c + v] : A(0);
        }
    }
    // the rows' groups of a workgroup run together: the barriers of row_sum (TPR > 64, one
    // group) are met by all threads
    for (int64_t row = int64_t(blockIdx.x) * kGroups + group; row < a.N; row += int64_t(gridDim.x) * kGroups) {
        const S *x = a.x + row * a.ldx;
        A f[R][V], s[1] = {0};
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * TPR + lane) * V;
            const auto raw = gpps::load_some<S, V>(x + c, n[r]);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                f[r][v] = E::up(raw[v]);
                s[0] += f[r][v];
            }
        }
        row_sum<A, TPR>(s, slots, 0);
        const A mean = s[0] / A(a.D);
        A q[1] = {0};
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                f[r][v] = v < n[r] ? f[r][v] - mean : A(0);
                q[0] += f[r][v] * f[r][v];
            }
        row_sum<A, TPR>(q, slots, 1);
        const A rstd = A(1) / sqrt(q[0] / A(a.D) + a.eps);
        S *y = a.y + row * a.ldy;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * TPR + lane) * V;
            typename gpps::Wide<S, V>::type out;
#pragma unroll
            for (int v = 0; v < V; ++v) out[v] = E::down(f[r][v] * rstd * w[r][v] + b[r][v]);
            gpps::store_some<S, V>(y + c, n[r], out);
        }
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

template <typename T, int TPR, int R>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void ln_grad_kernel(LnArgs<T> a) {
    using E = Elem<T>;
    using A = typename E::Acc;
    using S = typename E::Store;
    constexpr int V = E::V, kThreads = TPR < 256 ? 256 : TPR, kGroups = kThreads / TPR;
    constexpr int kCols = TPR * R * V;
    __shared__ A slots[TPR > 64 ? 4 * (TPR / 64) : 1];
    __shared__ A sum_w[kGroups > 1 ? kCols : 1], sum_b[kGroups > 1 ? kCols : 1];
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    A w[R][V], dw[R][V], db[R][V];
    int n[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t c = (int64_t(r) * TPR + lane) * V;
        n[r] = int(a.D - c < V ? (a.D > c ? a.D - c : 0) : V);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            w[r][v] = a.w && v < n[r] ? a.w[c + v] : A(1);
            dw[r][v] = db[r][v] = 0;
        }
    }
    int turn = 0;
    for (int64_t row = int64_t(blockIdx.x) * kGroups + group; row < a.N; row += int64_t(gridDim.x) * kGroups) {
        const S *x = a.x + row * a.ldx, *dy = a.dy + row * a.lddy;
        const A mean = a.mean[row], rstd = a.rstd[row];
        A xh[R][V], u[R][V], s[2] = {0, 0};
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * TPR + lane) * V;
            const auto xr = gpps::load_some<S, V>(x + c, n[r]);
            const auto gr = gpps::load_some<S, V>(dy + c, n[r]);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const A g = E::up(gr[v]);                    // 0 past the row's end
                xh[r][v] = v < n[r] ? (E::up(xr[v]) - mean) * rstd : A(0);
                dw[r][v] += g * xh[r][v];
                db[r][v] += g;
                u[r][v] = g * w[r][v];
                s[0] += u[r][v];
                s[1] += u[r][v] * xh[r][v];
            }
        }
        row_sum<A, TPR>(s, slots, turn);
        turn ^= 1;
        const A m0 = s[0] / A(a.D), m1 = s[1] / A(a.D);
        S *dx = a.y + row * a.ldy;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * TPR + lane) * V;
            typename gpps::Wide<S, V>::type out;
#pragma unroll
            for (int v = 0; v < V; ++v) out[v] = E::down(rstd * (u[r][v] - m0 - xh[r][v] * m1));
            gpps::store_some<S, V>(dx + c, n[r], out);
        }
    }
    // the groups' sums, joined within a wave by its lanes and between waves in their order
    if constexpr (TPR < 64) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v)
                for (int o = TPR; o < 64; o <<= 1) {
                    dw[r][v] += __shfl_xor(dw[r][v], o);
                    db[r][v] += __shfl_xor(db[r][v], o);
                }
    }
    if constexpr (kGroups > 1) {
        for (int wave = 0; wave < kThreads / 64; ++wave) {
            if (int(threadIdx.x) / 64 == wave && int(threadIdx.x) % 64 < TPR) {
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const int c = (r * TPR + lane) * V + v;
                        if (wave) {
                            dw[r][v] += sum_w[c];
                            db[r][v] += sum_b[c];
                        }
                        sum_w[c] = dw[r][v];
                        sum_b[c] = db[r][v];
                    }
            }
            __syncthreads();
        }
    }
    // (the last wave holds the workgroup's sums)
    if (kGroups == 1 || (threadIdx.x / 64 == kThreads / 64 - 1 && int(threadIdx.x) % 64 < TPR)) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int64_t c = (int64_t(r) * TPR + lane) * V + v;
                if (v >= n[r]) continue;
                if (a.dw) {
                    A *to = a.dw + blockIdx.x * a.step + c;
                    *to = a.accumulate ? *to + dw[r][v] : dw[r][v];
                }
                if (a.db) {
                    A *to = a.db + blockIdx.x * a.step + c;
                    *to = a.accumulate ? *to + db[r][v] : db[r][v];
                }
            }
    }
}

// dw and db from `parts` partial rows (dw's D columns, then db's): 16 columns a workgroup, 64
// slices of the rows each, then a tree over the slices.
template <typename A>
__global__ __launch_bounds__(1024) void ln_reduce_kernel(int64_t D, int parts, const A *__restrict__ part,
                                                         A *dw, A *db, int accumulate) {
    __shared__ A sums[64][16];
    const int col = threadIdx.x % 16, slice = threadIdx.x / 16;
    const int64_t c = int64_t(blockIdx.x) * 16 + col;
    A s = 0;
    if (c < 2 * D)
        for (int i = slice; i < parts; i += 64) s += part[int64_t(i) * 2 * D + c];
    sums[slice][col] = s;
    __syncthreads();
    for (int o = 32; o > 0; o >>= 1) {
        if (slice < o) sums[slice][col] += sums[slice + o][col];
        __syncthreads();
    }
    if (slice == 0 && c < 2 * D) {
        A *to = c < D ? (dw ? dw + c : nullptr) : (db ? db + (c - D) : nullptr);
        if (to) *to = accumulate ? *to + sums[0][col] : sums[0][col];
    }
}

template <typename A>
__global__ __launch_bounds__(256) void ln_zero_kernel(int64_t D, A *dw, A *db) {
    const int64_t c = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (c < D && dw) dw[c] = 0;
    if (c < D && db) db[c] = 0;
}

// The threads of a row and the vectors of each: the fewest threads that keep a row in
// `kMost` vectors or fewer a thread.
struct Plan {
    int tpr, r;
};

Plan plan(int64_t D, int V, int most) {
    const int64_t chunks = (D + V - 1) / V;
    for (int tpr : {8, 16, 32, 64, 256, 1024}) {
        const int64_t r = (chunks + tpr - 1) / tpr;
        if (r <= (tpr < 64 ? 1 : most) || tpr == 1024) return Plan{tpr, r <= 1 ? 1 : r <= 2 ? 2 : r <= 4 ? 4 : 8};
    }
    return Plan{1024, 8};
}

// Vectors a thread: four in the forward kernel, two in the gradient's, which holds five values
// for each element against three.
constexpr int kMostFwd = 4, kMostGrad = 2;

template <typename T, template <typename, int, int> class K>
hipError_t dispatch(const Plan &p, const LnArgs<T> &a, unsigned blocks, hipStream_t st) {
    switch (p.tpr) {
        case 8: return K<T, 8, 1>::go(a, blocks, st);
        case 16: return K<T, 16, 1>::go(a, blocks, st);
        case 32: return K<T, 32, 1>::go(a, blocks, st);
        case 64: return p.r == 1 ? K<T, 64, 1>::go(a, blocks, st) : p.r == 2 ? K<T, 64, 2>::go(a, blocks, st) : K<T, 64, 4>::go(a, blocks, st);
        case 256: return p.r == 1 ? K<T, 256, 1>::go(a, blocks, st) : p.r == 2 ? K<T, 256, 2>::go(a, blocks, st) : K<T, 256, 4>::go(a, blocks, st);
        default: return p.r <= 2 ? K<T, 1024, 2>::go(a, blocks, st) : p.r == 4 ? K<T, 1024, 4>::go(a, blocks, st) : K<T, 1024, 8>::go(a, blocks, st);
    }
}

template <typename T, int TPR, int R>
struct Fwd {
    static hipError_t go(const LnArgs<T> &a, unsigned blocks, hipStream_t st) {
        ln_fwd_kernel<T, TPR, R><<<blocks, TPR < 256 ? 256 : TPR, 0, st>>>(a);
        return hipGetLastError();
    }
};
template <typename T, int TPR, int R>
struct Grad {
    static hipError_t go(const LnArgs<T> &a, unsigned blocks, hipStream_t st) {
        ln_grad_kernel<T, TPR, R><<<blocks, TPR < 256 ? 256 : TPR, 0, st>>>(a);
        return hipGetLastError();
    }
};

int64_t groups_of(const Plan &p) { return p.tpr < 256 ? 256 / p.tpr : 1; }

// Workgroups of the gradient: enough rows in flight for the memory, few enough that the partial
// rows stay small beside the data.
int64_t grad_blocks(int64_t N, const Plan &p) {
    const int64_t rows = groups_of(p);
    return std::max<int64_t>(1, std::min<int64_t>((N + 4 * rows - 1) / (4 * rows), 1024));
}

template <typename T>
hipError_t forward(LnArgs<T> a, hipStream_t st) {
    const Plan p = plan(a.D, Elem<T>::V, kMostFwd);
    const int64_t rows = groups_of(p);
    const unsigned blocks = unsigned(std::min<int64_t>((a.N + rows - 1) / rows, 2048));
    gpps::TimedScope ts(st, "layer_norm_fwd");
    return dispatch<T, Fwd>(p, a, blocks, st);
}

template <typename T>
hipError_t gradient(LnArgs<T> a, void *ws, hipStream_t st) {
    using A = typename Elem<T>::Acc;
    A *dw = a.dw, *db = a.db;
    const Plan p = plan(a.D, Elem<T>::V, kMostGrad);
    const int64_t blocks = grad_blocks(a.N, p);
    const int accumulate = a.accumulate;
    if (blocks > 1) {
        a.dw = static_cast<A *>(ws);
        a.db = a.dw + a.D;
        a.step = 2 * a.D;
        a.accumulate = 0;
    }
    {
        gpps::TimedScope ts(st, "layer_norm_grad");
        const hipError_t e = dispatch<T, Grad>(p, a, unsigned(blocks), st);
        if (e != hipSuccess || blocks == 1) return e;
    }
    gpps::TimedScope ts(st, "layer_norm_reduce");
    ln_reduce_kernel<A><<<unsigned((2 * a.D + 15) / 16), 1024, 0, st>>>(a.D, int(blocks), (const A *)ws, dw, db, accumulate);
    return hipGetLastError();
}

bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool valid_dtype(gpps_dtype dt) { return dt == GPPS_F32 || dt == GPPS_F64 || dt == GPPS_BF16; }

bool valid_shape(int64_t N, int64_t D) { return N >= 0 && D >= 1 && D <= GPPS_MAX_WIDTH && N <= (int64_t(1) << 40) / D; }

size_t elem_size(gpps_dtype dt) { return dt == GPPS_F64 ? 8 : dt == GPPS_BF16 ? 2 : 4; }
size_t acc_size(gpps_dtype dt) { return dt == GPPS_F64 ? 8 : 4; }

template <typename T>
hipError_t run_forward(int64_t N, int64_t D, const void *x, int64_t ldx, const void *w, const void *b, double eps,
                       void *y, int64_t ldy, void *mean, void *rstd, hipStream_t st) {
    using A = typename Elem<T>::Acc;
    using S = typename Elem<T>::Store;
    LnArgs<T> a{};
    a.N = N, a.D = D, a.x = (const S *)x, a.ldx = ldx, a.w = (const A *)w, a.b = (const A *)b, a.eps = A(eps);
    a.y = (S *)y, a.ldy = ldy, a.mean = (A *)mean, a.rstd = (A *)rstd;
    return forward<T>(a, st);
}

template <typename T>
hipError_t run_gradient(int64_t N, int64_t D, const void *x, int64_t ldx, const void *w, const void *mean,
                        const void *rstd, const void *dy, int64_t lddy, void *dx, int64_t lddx, void *dw, void *db,
                        int accumulate, void *ws, hipStream_t st) {
    using A = typename Elem<T>::Acc;
    using S = typename Elem<T>::Store;
    LnArgs<T> a{};
    a.N = N, a.D = D, a.x = (const S *)x, a.ldx = ldx, a.w = (const A *)w;
    a.mean = (A *)const_cast<void *>(mean), a.rstd = (A *)const_cast<void *>(rstd);
    a.dy = (const S *)dy, a.lddy = lddy, a.y = (S *)dx, a.ldy = lddx, a.dw = (A *)dw, a.db = (A *)db;
    a.accumulate = accumulate;
    if (N == 0) {
        if (accumulate) return hipSuccess;
        ln_zero_kernel<A><<<unsigned((D + 255) / 256), 256, 0, st>>>(D, a.dw, a.db);
        return hipGetLastError();
    }
    return gradient<T>(a, ws, st);
}

}  // namespace

extern "C" {

gpps_status gpps_layer_norm(gpps_dtype dt, int64_t N, int64_t D, const void *x, int64_t ldx, const void *weight,
                            const void *bias, double eps, void *y, int64_t ldy, void *mean, void *rstd,
                            void *stream) {
    if (!valid_dtype(dt)) return GPPS_ERR_DTYPE;
    if (!valid_shape(N, D) || ldx < D || ldy < D) return GPPS_ERR_SHAPE;
    if (!std::isfinite(eps) || eps < 0.0) return GPPS_ERR_HYPER;
    if (N == 0) return GPPS_OK;
    if (!x || !y) return GPPS_ERR_NULL;
    if (!aligned(x, elem_size(dt)) || !aligned(y, elem_size(dt))) return GPPS_ERR_ALIGN;
    for (const void *p : {weight, bias, (const void *)mean, (const void *)rstd})
        if (p && !aligned(p, acc_size(dt))) return GPPS_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const hipError_t e =
        dt == GPPS_F32   ? run_forward<float>(N, D, x, ldx, weight, bias, eps, y, ldy, mean, rstd, st)
        : dt == GPPS_F64 ? run_forward<double>(N, D, x, ldx, weight, bias, eps, y, ldy, mean, rstd, st)
                         : run_forward<bf16_t>(N, D, x, ldx, weight, bias, eps, y, ldy, mean, rstd, st);
    return e == hipSuccess ? GPPS_OK : GPPS_ERR_HIP;
}

size_t gpps_layer_norm_workspace_bytes(gpps_dtype dt, int64_t N, int64_t D) {
    if (!valid_dtype(dt) || !valid_shape(N, D)) return 0;
    const Plan p = plan(D, int(16 / elem_size(dt)), kMostGrad);
    return gpps::align_up(size_t(grad_blocks(N, p)) * 2 * size_t(D) * acc_size(dt), 256);
}

gpps_status gpps_layer_norm_grads(gpps_dtype dt, int64_t N, int64_t D, const void *x, int64_t ldx,
                                  const void *weight, const void *mean, const void *rstd, const void *dy,
                                  int64_t lddy, void *dx, int64_t lddx, void *dweight, void *dbias, int flags,
                                  void *workspace, size_t workspace_bytes, void *stream) {
    if (!valid_dtype(dt)) return GPPS_ERR_DTYPE;
    if (!valid_shape(N, D) || ldx < D || lddy < D || lddx < D) return GPPS_ERR_SHAPE;
    if (N && (!x || !mean || !rstd || !dy || !dx)) return GPPS_ERR_NULL;
    if (!workspace) return GPPS_ERR_NULL;
    if (!aligned(workspace, 256)) return GPPS_ERR_ALIGN;
    if (workspace_bytes < gpps_layer_norm_workspace_bytes(dt, N, D)) return GPPS_ERR_WORKSPACE;
    for (const void *p : {x, dy, (const void *)dx})
        if (p && !aligned(p, elem_size(dt))) return GPPS_ERR_ALIGN;
    for (const void *p : {weight, mean, rstd, (const void *)dweight, (const void *)dbias})
        if (p && !aligned(p, acc_size(dt))) return GPPS_ERR_ALIGN;
    if (flags & ~GPPS_ACCUMULATE) return GPPS_ERR_PATH;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int acc = flags & GPPS_ACCUMULATE;
    const hipError_t e =
        dt == GPPS_F32 ? run_gradient<float>(N, D, x, ldx, weight, mean, rstd, dy, lddy, dx, lddx, dweight, dbias, acc, workspace, st)
        : dt == GPPS_F64
            ? run_gradient<double>(N, D, x, ldx, weight, mean, rstd, dy, lddy, dx, lddx, dweight, dbias, acc, workspace, st)
            : run_gradient<bf16_t>(N, D, x, ldx, weight, mean, rstd, dy, lddy, dx, lddx, dweight, dbias, acc, workspace, st);
    return e == hipSuccess ? GPPS_OK : GPPS_ERR_HIP;
}

}  // extern "C"
