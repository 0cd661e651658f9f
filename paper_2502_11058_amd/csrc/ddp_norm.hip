// Layer norm and root-mean-square norm, forward and backward.  Memory bound: the forward pass reads and writes a row once, the
// backward pass reads two rows and writes one.
//
// A row belongs to a wavefront or to a workgroup and stays in its registers between the sums and the result; the variance is the
// sum of squared differences from the mean that the first sum gave, not a difference of sums, so a mean far from zero costs no
// digits.  The weight's and bias' gradients are columns' sums over all rows: every workgroup of the backward pass adds up its
// own rows in registers, writes one partial row in fp32, and a second kernel adds the partial rows in their order.
//
// Measured: 16384 x 4096 bf16, 43 us forward (6.2 TB/s), 63 backward (6.4 TB/s), 5 for the partial rows; 8192 x 768 fp32, which the last-level
// cache holds, 11.6, 16.0 and 3.9 us.  A workgroup holds rows of up to 16 KiB.  Longer ones are read again for each sum, and twice more than
// the columns' sums take: 4096 x 8192 fp32, calls of 75 us forward (root mean square 57) and 134 backward, where 8192 x 4096 takes 40 and 67.
// bf16 rows beyond 8 KiB leave the backward kernel one wavefront a SIMD (255 registers and two to six more): 8192 x 8192 in 90 us, 4.5 TB/s.
#include "ddp_operators.h"

namespace ddp {
namespace {

struct NormArgs {
    const void *x, *dy, *w, *b;
    void *y;
    float *mean, *rstd;
    int64_t rows, cols, x_stride, y_stride;
    float eps, inv;
};

// Sum over the GROUP threads that share a row; every thread of them gets it.
template <int GROUP>
__device__ __forceinline__ float group_sum(float v, float *scratch) {
    v = wave_sum(v);
    if constexpr (GROUP > 64) {
        __syncthreads();  // (the scratch may still be read for the sum before)
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < GROUP / 64; ++i) v += scratch[i];
    }
    return v;
}
template <int GROUP>
__device__ __forceinline__ f32x2 group_sum2(f32x2 v, float *scratch) {
    v.x = wave_sum(v.x);
    v.y = wave_sum(v.y);
    if constexpr (GROUP > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
            scratch[threadIdx.x >> 6] = v.x;
            scratch[GROUP / 64 + (threadIdx.x >> 6)] = v.y;
        }
        __syncthreads();
        v = f32x2{0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < GROUP / 64; ++i) {
            v.x += scratch[i];
            v.y += scratch[GROUP / 64 + i];
        }
    }
    return v;
}

// NV groups of 16 bytes a thread hold the row; NV = 0: a row too long for that is read again for each sum.
template <class T, bool RMS, int GROUP, int NV, bool STREAM>
__global__ __launch_bounds__(256) void norm_forward_kernel(const NormArgs a) {
    constexpr int N = Group<T>::n, HELD = NV ? NV : 1;
    __shared__ float scratch[8];
    const int lane = threadIdx.x % GROUP;
    const int cols = (int)a.cols, groups = (cols + N - 1) / N;
    const T *w = static_cast<const T *>(a.w), *b = static_cast<const T *>(a.b);
    for (int64_t row = (int64_t)blockIdx.x * (256 / GROUP) + threadIdx.x / GROUP; row < a.rows; row += (int64_t)gridDim.x * (256 / GROUP)) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        T *y = static_cast<T *>(a.y) + row * a.y_stride;
        Vec<T> held[HELD];
        if constexpr (NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = (lane + k * GROUP) * N;
                held[k] = c < cols ? load_part(x + c, cols - c) : Vec<T>{};
            }
        }
        auto each = [&](auto &&f) {
            if constexpr (NV > 0) {
#pragma unroll
                for (int k = 0; k < NV; ++k) f(held[k], (lane + k * GROUP) * N);
            } else {
                for (int g = lane; g < groups; g += GROUP) f(load_part(x + g * N, cols - g * N), g * N);
            }
        };
        float mean = 0.0f;
        if constexpr (!RMS) {
            float s = 0.0f;
            each([&](Vec<T> v, int c) {
#pragma unroll
                for (int j = 0; j < N; ++j) s += (float)v[j];  // (zeros beyond the row)
            });
            mean = group_sum<GROUP>(s, scratch) * a.inv;
        }
        float s = 0.0f;
        each([&](Vec<T> v, int c) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float d = RMS || c + j < cols ? (float)v[j] - mean : 0.0f;
                s += d * d;
            }
        });
        const float rstd = 1.0f / sqrtf(group_sum<GROUP>(s, scratch) * a.inv + a.eps);
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
        each([&](Vec<T> v, int c) {
            if (c >= cols) return;
            const Vec<T> wv = load_part(w + c, cols - c);
            Vec<T> bv{}, o;
            if (b) bv = load_part(b + c, cols - c);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float h = ((float)v[j] - mean) * rstd;
                o[j] = (T)(h * (float)wv[j] + (b ? (float)bv[j] : 0.0f));
            }
            store_part<STREAM>(y + c, o, cols - c);
        });
    }
}

struct NormBackArgs {
    NormArgs n;
    void *dx;
    int64_t dx_stride;
    float *part_w, *part_b;  // [workgroups][cols], nullable
};

template <class T, bool RMS, int GROUP, int NV, bool STREAM>
__global__ __launch_bounds__(256) void norm_backward_kernel(const NormBackArgs a) {
    constexpr int N = Group<T>::n, ROWS = 256 / GROUP;
    __shared__ float scratch[8];
    __shared__ float fold[GROUP == 64 ? 256 * N : 1];
    const int lane = threadIdx.x % GROUP;
    const int cols = (int)a.n.cols;
    const T *w = static_cast<const T *>(a.n.w);
    float sw[NV * N] = {}, sb[NV * N] = {};
    Vec<T> wv[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (lane + k * GROUP) * N;
        wv[k] = c < cols ? load_part(w + c, cols - c) : Vec<T>{};
    }
    // (the workgroup's threads go round together: the rows' sums meet in LDS)
    // The next row is asked for before this one's sums meet.
    struct Row {
        Vec<T> x[NV], d[NV];
        float mean, rstd;
    };
    auto fetch = [&](int64_t row) {
        Row v;
        const T *x = static_cast<const T *>(a.n.x) + row * a.n.x_stride, *dy = static_cast<const T *>(a.n.dy) + row * a.n.y_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (lane + k * GROUP) * N;
            v.x[k] = c < cols ? load_part(x + c, cols - c) : Vec<T>{};
            v.d[k] = c < cols ? load_part(dy + c, cols - c) : Vec<T>{};  // (zero beyond the row: nothing is added there)
        }
        v.mean = RMS ? 0.0f : a.n.mean[row];
        v.rstd = a.n.rstd[row];
        return v;
    };
    const int64_t mine = threadIdx.x / GROUP, step = (int64_t)gridDim.x * ROWS;
    Row next;
    if ((int64_t)blockIdx.x * ROWS + mine < a.n.rows) next = fetch((int64_t)blockIdx.x * ROWS + mine);
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < a.n.rows; row0 += step) {
        const int64_t row = row0 + mine;
        if (GROUP == 64 && row >= a.n.rows) break;
        const Row now = next;
        if (row + step < a.n.rows) next = fetch(row + step);
        const auto &xv = now.x;
        const auto &dv = now.d;
        const float mean = now.mean, rstd = now.rstd;
        f32x2 s{0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float h = ((float)xv[k][j] - mean) * rstd, d = (float)dv[k][j], g = d * (float)wv[k][j];
                s.x += g;
                s.y += g * h;
                sw[k * N + j] += d * h;
                sb[k * N + j] += d;
            }
        if (!a.dx) continue;
        s = group_sum2<GROUP>(s, scratch);
        const float c1 = RMS ? 0.0f : s.x * a.n.inv, c2 = s.y * a.n.inv;
        T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (lane + k * GROUP) * N;
            if (c >= cols) continue;
            Vec<T> o;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float h = ((float)xv[k][j] - mean) * rstd, g = (float)dv[k][j] * (float)wv[k][j];
                o[j] = (T)(rstd * (g - c1 - h * c2));
            }
            store_part<STREAM>(dx + c, o, cols - c);
        }
    }
    auto put = [&](float *part, const float *sum) {
        if (!part) return;
        part += (int64_t)blockIdx.x * cols;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (lane + k * GROUP) * N;
            float o[N];
            if constexpr (GROUP == 64) {  // the four wavefronts' rows, in their order
                __syncthreads();
#pragma unroll
                for (int j = 0; j < N; ++j) fold[j * 256 + threadIdx.x] = sum[k * N + j];
                __syncthreads();
                if (threadIdx.x >= 64) continue;
#pragma unroll
                for (int j = 0; j < N; ++j) o[j] = fold[j * 256 + lane] + fold[j * 256 + 64 + lane] + fold[j * 256 + 128 + lane] + fold[j * 256 + 192 + lane];
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) o[j] = sum[k * N + j];
            }
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (c + j < cols) part[c + j] = o[j];
        }
    };
    put(a.part_w, sw);
    put(a.part_b, sb);
}

// Rows too long for registers: x and dy are read twice here, for the sums and for the result, and once more by the columns' kernel.
template <class T, bool RMS, bool STREAM>
__global__ __launch_bounds__(256) void norm_backward_long_kernel(const NormBackArgs a) {
    constexpr int N = Group<T>::n;
    __shared__ float scratch[8];
    const int cols = (int)a.n.cols, groups = (cols + N - 1) / N;
    const T *w = static_cast<const T *>(a.n.w);
    for (int64_t row = blockIdx.x; row < a.n.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.n.x) + row * a.n.x_stride, *dy = static_cast<const T *>(a.n.dy) + row * a.n.y_stride;
        T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
        const float mean = RMS ? 0.0f : a.n.mean[row], rstd = a.n.rstd[row];
        f32x2 s{0.0f, 0.0f};
        for (int g = threadIdx.x; g < groups; g += 256) {
            const int c = g * N;
            const Vec<T> xv = load_part(x + c, cols - c), dv = load_part(dy + c, cols - c), wv = load_part(w + c, cols - c);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float e = (float)dv[j] * (float)wv[j];
                s.x += e;
                s.y += e * (((float)xv[j] - mean) * rstd);
            }
        }
        s = group_sum2<256>(s, scratch);
        const float c1 = RMS ? 0.0f : s.x * a.n.inv, c2 = s.y * a.n.inv;
        for (int g = threadIdx.x; g < groups; g += 256) {
            const int c = g * N;
            const Vec<T> xv = load_part(x + c, cols - c), dv = load_part(dy + c, cols - c), wv = load_part(w + c, cols - c);
            Vec<T> o;
#pragma unroll
            for (int j = 0; j < N; ++j) o[j] = (T)(rstd * ((float)dv[j] * (float)wv[j] - c1 - ((float)xv[j] - mean) * rstd * c2));
            store_part<STREAM>(dx + c, o, cols - c);
        }
    }
}
template <class T, bool RMS>
__global__ __launch_bounds__(256) void norm_columns_kernel(const NormBackArgs a) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.n.cols) return;
    float sw = 0.0f, sb = 0.0f;
    for (int64_t row = blockIdx.y; row < a.n.rows; row += gridDim.y) {
        const float mean = RMS ? 0.0f : a.n.mean[row], rstd = a.n.rstd[row];
        const float d = (float)static_cast<const T *>(a.n.dy)[row * a.n.y_stride + c];
        sw += d * (((float)static_cast<const T *>(a.n.x)[row * a.n.x_stride + c] - mean) * rstd);
        sb += d;
    }
    if (a.part_w) a.part_w[(int64_t)blockIdx.y * a.n.cols + c] = sw;
    if (a.part_b) a.part_b[(int64_t)blockIdx.y * a.n.cols + c] = sb;
}

// Column sums of the partial rows: 32 columns and 32 runs of rows a workgroup, joined in order.
template <class T>
__global__ __launch_bounds__(1024) void norm_fold_kernel(const float *part_w, const float *part_b, int parts, int64_t cols, T *dw, T *db) {
    __shared__ float run[32][33];
    const float *part = blockIdx.y ? part_b : part_w;
    T *out = blockIdx.y ? db : dw;
    if (!out) return;
    const int col = threadIdx.x & 31, r = threadIdx.x >> 5;
    for (int64_t c0 = (int64_t)blockIdx.x * 32; c0 < cols; c0 += (int64_t)gridDim.x * 32) {
        const int64_t c = c0 + col;
        float s = 0.0f;
        if (c < cols)
#pragma unroll 8
            for (int i = r; i < parts; i += 32) s += part[i * cols + c];
        run[r][col] = s;
        __syncthreads();
        if (r == 0 && c < cols) {
            s = 0.0f;
#pragma unroll
            for (int i = 0; i < 32; ++i) s += run[i][col];
            out[c] = (T)s;
        }
        __syncthreads();  // (the runs may still be read for these columns)
    }
}

// Workgroups of the backward pass, each with a partial row: as many as keep enough bytes under way, and no more, since partial rows are written
// and read again.  8192 x 768 fp32: 19.3 us with 512, 16.5 with 1024, 17.4 with 2048; 16384 x 4096 bf16: 79 us with 512, 86 with 768, 95 with 1024.
// Rows that are not held have 64 runs of rows a column.
int norm_parts(const ddp_norm &n) {
    const int64_t groups = cdiv(n.cols * (int64_t)element_size(n.dtype), 16), most = groups <= 256 ? 1024 : groups <= 1024 ? 512 : 64;
    const int64_t wgs = groups <= 256 ? cdiv(n.rows, 4) : n.rows;
    return (int)(wgs < most ? wgs : most);
}

int check_norm(const char *who, const ddp_norm *n) {
    if (!n) return bad(who, DDP_EINVAL, "the shape is NULL");
    if (!typed(n->dtype)) return bad(who, DDP_EINVAL, "dtype must be DDP_F32 or DDP_BF16");
    if (n->kind != DDP_NORM_LAYER && n->kind != DDP_NORM_RMS) return bad(who, DDP_EINVAL, "unknown kind");
    if (n->rows < 0 || n->rows > ((int64_t)1 << 40)) return bad(who, DDP_EINVAL, "rows out of range");
    if (n->cols < 1 || n->cols > (1 << 28)) return bad(who, DDP_EINVAL, "cols must be in [1, 2^28]");
    if (!(n->eps >= 0)) return bad(who, DDP_EINVAL, "eps must not be negative");
    if (n->rows > 1 && (n->x_stride < n->cols || n->y_stride < n->cols)) return bad(who, DDP_EINVAL, "rows overlap: a stride is smaller than cols");
    if (reach(n->rows, n->x_stride) < 0 || reach(n->rows, n->y_stride) < 0) return bad(who, DDP_EINVAL, "a stride is too large");
    return DDP_OK;
}

NormArgs norm_args(const ddp_norm &n) {
    NormArgs a{};
    a.rows = n.rows, a.cols = n.cols, a.x_stride = n.x_stride, a.y_stride = n.y_stride, a.eps = n.eps, a.inv = 1.0f / (float)n.cols;
    return a;
}

// f(whether results are written with streaming stores)
template <class F>
void by_size(const ddp_norm &n, int tensors, F &&f) {
    if (streams_past(tensors * n.rows * n.cols * (int64_t)element_size(n.dtype)))
        f(std::true_type{});
    else
        f(std::false_type{});
}
template <class F>
int by_type(const ddp_norm &n, F &&f) {
    if (n.dtype == DDP_BF16) return n.kind == DDP_NORM_RMS ? f(bf16{}, std::true_type{}) : f(bf16{}, std::false_type{});
    return n.kind == DDP_NORM_RMS ? f(float{}, std::true_type{}) : f(float{}, std::false_type{});
}
// By the row's length: f(threads that share a row, groups a thread holds).  A wavefront needs no barrier for its sums: 8192 x 768 fp32 forward
// 14.0 us with a workgroup a row, 11.3 with a wavefront; beyond four groups its registers leave too few rows under way.
template <class T, class F>
void by_length(int64_t cols, F &&f) {
    const int64_t g = cdiv(cols, Group<T>::n);
    typedef std::integral_constant<int, 64> wave;
    typedef std::integral_constant<int, 256> block;
    if (g <= 64) f(wave{}, std::integral_constant<int, 1>{});
    else if (g <= 128) f(wave{}, std::integral_constant<int, 2>{});
    else if (g <= 192) f(wave{}, std::integral_constant<int, 3>{});
    else if (g <= 256) f(wave{}, std::integral_constant<int, 4>{});
    else if (g <= 512) f(block{}, std::integral_constant<int, 2>{});
    else if (g <= 1024) f(block{}, std::integral_constant<int, 4>{});
    else f(block{}, std::integral_constant<int, 0>{});
}

}  // namespace
}  // namespace ddp

extern "C" int ddp_norm_forward(const ddp_norm *norm, const void *x, const void *weight, const void *bias, void *y, float *mean, float *rstd, void *stream) {
    using namespace ddp;
    return guarded(nullptr, [&]() -> int {
        const char *who = "ddp_norm_forward";
        if (int rc = check_norm(who, norm)) return rc;
        const ddp_norm &n = *norm;
        if (n.rows == 0) return DDP_OK;
        if (!x || !weight || !y || !rstd || (!mean && n.kind == DDP_NORM_LAYER)) return bad(who, DDP_EINVAL, "NULL pointer");
        const size_t e = element_size(n.dtype);
        if (misaligned(x, e) || misaligned(weight, e) || misaligned(bias, e) || misaligned(y, e) || misaligned(mean, 4) || misaligned(rstd, 4))
            return bad(who, DDP_EALIGN, "a tensor is not aligned to its element type");
        NormArgs a = norm_args(n);
        a.x = x, a.w = weight, a.b = bias, a.y = y, a.mean = mean, a.rstd = rstd;
        return by_type(n, [&](auto t, auto rms) -> int {
            typedef decltype(t) T;
            by_length<T>(n.cols, [&](auto group, auto nv) {
                const int64_t wgs = cdiv(n.rows, 256 / group.value);
                by_size(n, 2, [&](auto past) {
                    hipLaunchKernelGGL((norm_forward_kernel<T, rms.value, group.value, nv.value, past.value>), dim3((unsigned)(wgs < (1 << 20) ? wgs : 1 << 20)),
                                       dim3(256), 0, static_cast<hipStream_t>(stream), a);
                });
            });
            return launched(who);
        });
    });
}

extern "C" int64_t ddp_norm_backward_workspace(const ddp_norm *norm) {
    using namespace ddp;
    if (int rc = guarded(nullptr, [&]() -> int { return check_norm("ddp_norm_backward_workspace", norm); })) return -rc;
    return up((int64_t)norm_parts(*norm) * norm->cols * 4, 256) * 2;
}

extern "C" int ddp_norm_backward(const ddp_norm *norm, const void *dy, const void *x, const void *weight, const float *mean, const float *rstd, void *dx,
                                 void *dweight, void *dbias, void *workspace, int64_t workspace_bytes, void *stream) {
    using namespace ddp;
    return guarded(nullptr, [&]() -> int {
        const char *who = "ddp_norm_backward";
        if (int rc = check_norm(who, norm)) return rc;
        const ddp_norm &n = *norm;
        const bool columns = dweight || dbias;
        if (n.rows > 0 && (!dy || !x || !weight || !rstd || (!mean && n.kind == DDP_NORM_LAYER))) return bad(who, DDP_EINVAL, "NULL pointer");
        const size_t e = element_size(n.dtype);
        for (const void *p : {dy, x, weight, (const void *)dx, (const void *)dweight, (const void *)dbias})
            if (misaligned(p, e)) return bad(who, DDP_EALIGN, "a tensor is not aligned to its element type");
        if (misaligned(mean, 4) || misaligned(rstd, 4)) return bad(who, DDP_EALIGN, "mean or rstd is not aligned to its element type");
        const int64_t dx_stride = n.dx_stride ? n.dx_stride : n.x_stride;
        if (dx && n.rows > 1 && (dx_stride < n.cols || reach(n.rows, dx_stride) < 0)) return bad(who, DDP_EINVAL, "dx_stride is smaller than cols or too large");
        if (dx == dy && dx && n.rows > 1 && dx_stride != n.y_stride) return bad(who, DDP_EINVAL, "in place, the strides of dx and dy have to be the same");
        const int parts = norm_parts(n);
        const int64_t part = up((int64_t)parts * n.cols * 4, 256);
        if (columns && n.rows > 0) {
            if (!workspace) return bad(who, DDP_EINVAL, "workspace is NULL");
            if (misaligned(workspace, 256)) return bad(who, DDP_EALIGN, "workspace is not 256-byte aligned");
            if (workspace_bytes < 2 * part) return bad(who, DDP_ESHAPE, "workspace is too small");
        }
        if (!dx && !columns) return DDP_OK;
        const hipStream_t st = static_cast<hipStream_t>(stream);
        NormBackArgs a{};
        a.n = norm_args(n);
        a.n.x = x, a.n.dy = dy, a.n.w = weight, a.n.mean = const_cast<float *>(mean), a.n.rstd = const_cast<float *>(rstd), a.dx = dx, a.dx_stride = dx_stride;
        a.part_w = dweight ? static_cast<float *>(workspace) : nullptr;
        a.part_b = dbias ? reinterpret_cast<float *>(static_cast<char *>(workspace) + part) : nullptr;
        return by_type(n, [&](auto t, auto rms) -> int {
            typedef decltype(t) T;
            if (n.rows > 0)
                by_length<T>(n.cols, [&](auto group, auto nv) {
                    if constexpr (nv.value > 0) {
                        by_size(n, 3, [&](auto past) {
                            hipLaunchKernelGGL((norm_backward_kernel<T, rms.value, group.value, nv.value, past.value>), dim3((unsigned)parts), dim3(256), 0, st, a);
                        });
                    } else {
                        // (before dx, which may take the place of dy)
                        if (columns) hipLaunchKernelGGL((norm_columns_kernel<T, rms.value>), dim3((unsigned)cdiv(n.cols, 256), (unsigned)parts), dim3(256), 0, st, a);
                        if (dx)
                            by_size(n, 3, [&](auto past) {
                                hipLaunchKernelGGL((norm_backward_long_kernel<T, rms.value, past.value>), dim3((unsigned)(n.rows < 65536 ? n.rows : 65536)), dim3(256), 0, st, a);
                            });
                    }
                });
            if (columns) {
                const int64_t wgs = cdiv(n.cols, 32);
                hipLaunchKernelGGL((norm_fold_kernel<T>), dim3((unsigned)(wgs < most_groups(1024) ? wgs : most_groups(1024)), dbias ? 2 : 1), dim3(1024), 0, st, a.part_w,
                                   a.part_b, parts, n.cols, static_cast<T *>(dweight), static_cast<T *>(dbias));
            }
            return launched(who);
        });
    });
}
