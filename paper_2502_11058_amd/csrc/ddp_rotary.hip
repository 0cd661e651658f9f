// Rotary positions.  Memory bound: an element is read and written once with two products and a sum, and a token's row of the table
// serves all its heads.  16384 tokens of 32 and 8 heads of 128 in bf16: 59 us a call, 5.7 TB/s.
#include "ddp_operators.h"

namespace ddp {
namespace {

struct RotaryArgs {
    const void *x[2];
    void *y[2];
    int64_t x_token[2], x_head[2], y_token[2], y_head[2];
    int heads[2];
    const float *table;
    const void *positions;
    int64_t tokens, table_rows, sequence;
    int dim, half, position_bytes, inverse;
    int units, turned;     // threads' places in a head, and those of pairs among them
    int64_t tokens_each;   // of a workgroup
};

__device__ __forceinline__ int64_t position_of(const RotaryArgs &a, int64_t t) {
    if (!a.positions) return t % a.sequence;
    return a.position_bytes == 8 ? reinterpret_cast<const int64_t *>(a.positions)[t] : (int64_t) reinterpret_cast<const int32_t *>(a.positions)[t];
}

// One thread has 16 bytes of a head's first halves of pairs and 16 of the second (HALF), 32 bytes of pairs (INTERLEAVED), or as much of
// what is copied, so that every access is of 128 bits: `units` of them a head, the first `turned` of which are pairs.  Consecutive threads go
// over a token's heads, whose row of the table then comes from the cache.  A head whose rotated part ends inside a group takes single
// elements there (load_part).
template <class T, bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a) {
    constexpr int N = Group<T>::n;
    const unsigned per_token = (unsigned)(a.heads[0] + a.heads[1]) * (unsigned)a.units;
    for (int64_t t = (int64_t)blockIdx.x * a.tokens_each + threadIdx.y; t < a.tokens && t < ((int64_t)blockIdx.x + 1) * a.tokens_each; t += blockDim.y) {
        const int64_t p = position_of(a, t);
        const bool known = p >= 0 && p < a.table_rows;
        const float *table = a.table + (known ? p * a.half * 2 : 0);
        for (unsigned in = threadIdx.x; in < per_token; in += blockDim.x) {
            const unsigned head = in / (unsigned)a.units, u = in - head * (unsigned)a.units;
            const int which = head >= (unsigned)a.heads[0], h = (int)head - (which ? a.heads[0] : 0);
            const T *x = static_cast<const T *>(a.x[which]) + t * a.x_token[which] + h * a.x_head[which];
            T *y = static_cast<T *>(a.y[which]) + t * a.y_token[which] + h * a.y_head[which];
            if ((int)u >= a.turned) {
                const int c = 2 * a.half + ((int)u - a.turned) * 2 * N;
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (c + k * N < a.dim) store_part<STREAM>(y + c + k * N, load_part(x + c + k * N, a.dim - c - k * N), a.dim - c - k * N);
                continue;
            }
            const int first = (int)u * N, pairs = a.half - first < N ? a.half - first : N;  // pairs of this thread
            float c[N], s[N];
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                f32x4 v = {__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
                if (known && j < pairs) v = load_part(table + 2 * (first + j), 2 * (pairs - j));
                c[j] = v[0], s[j] = v[1], c[j + 1] = v[2], s[j + 1] = v[3];
            }
            Vec<T> p0, p1, q0, q1;
            const int at0 = INTERLEAVED ? 2 * first : first, at1 = INTERLEAVED ? 2 * first + N : a.half + first;
            const int n0 = INTERLEAVED ? 2 * pairs : pairs, n1 = INTERLEAVED ? 2 * pairs - N : pairs;
            p0 = load_part(x + at0, n0);
            p1 = n1 > 0 ? load_part(x + at1, n1) : Vec<T>{};
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float sn = a.inverse ? -s[j] : s[j];
                // pair j: its two elements' places in the 2 N loaded
                const int e0 = INTERLEAVED ? 2 * j : j, e1 = INTERLEAVED ? 2 * j + 1 : j;
                const float u0 = (float)(INTERLEAVED && e0 >= N ? p1[e0 % N] : p0[e0 % N]);
                const float u1 = (float)(INTERLEAVED ? (e1 >= N ? p1[e1 % N] : p0[e1 % N]) : p1[j]);
                const T r0 = (T)(u0 * c[j] - u1 * sn), r1 = (T)(u0 * sn + u1 * c[j]);
                if (INTERLEAVED) {
                    if (e0 >= N) {
                        q1[e0 % N] = r0;
                        q1[e1 % N] = r1;
                    } else {
                        q0[e0 % N] = r0;
                        q0[e1 % N] = r1;
                    }
                } else {
                    q0[j] = r0;
                    q1[j] = r1;
                }
            }
            store_part<STREAM>(y + at0, q0, n0);
            if (n1 > 0) store_part<STREAM>(y + at1, q1, n1);
        }
    }
}

struct Frequencies {
    double f[DDP_ROTARY_MAX_ROTATED / 2];
};
__global__ __launch_bounds__(256) void table_kernel(const Frequencies f, double amplitude, int64_t n, int half, float *table) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        double s, c;
        sincos((double)(i / half) * f.f[i % half], &s, &c);
        table[2 * i] = (float)(amplitude * c);
        table[2 * i + 1] = (float)(amplitude * s);
    }
}

int check_side(const char *who, const void *x, const void *y, const ddp_rotary_shape &r, int heads, int64_t xt, int64_t xh, int64_t yt, int64_t yh) {
    if (heads == 0) return DDP_OK;
    if (!x || !y) return bad(who, DDP_EINVAL, "a tensor is NULL");
    if (misaligned(x, element_size(r.dtype)) || misaligned(y, element_size(r.dtype))) return bad(who, DDP_EALIGN, "a tensor is not aligned to its element type");
    for (const int64_t a : {reach(r.tokens, xt), reach(heads, xh), reach(r.tokens, yt), reach(heads, yh)})
        if (a < 0) return bad(who, DDP_EINVAL, "a stride is negative or too large");
    if (x == y && (xt != yt || xh != yh)) return bad(who, DDP_EINVAL, "in place, the strides of input and output have to be the same");
    return DDP_OK;
}

template <class T>
int launch_rotary(const ddp_rotary_shape &r, RotaryArgs &a, hipStream_t stream) {
    constexpr int N = Group<T>::n;
    a.turned = (a.half + N - 1) / N;
    a.units = a.turned + (a.dim - 2 * a.half + 2 * N - 1) / (2 * N);
    // 64, 128 or 256 threads lie over a token's places, whichever leaves the fewest idle in the last round, and the rest over other tokens
    const int64_t per_token = (int64_t)(a.heads[0] + a.heads[1]) * a.units;
    int x = 64;
    for (const int wide : {128, 256})
        if (up(per_token, wide) <= up(per_token, x)) x = wide;
    a.tokens_each = 256 / x;
    while (cdiv(a.tokens, a.tokens_each) > most_groups(256)) a.tokens_each *= 2;
    const dim3 grid((unsigned)cdiv(a.tokens, a.tokens_each)), block((unsigned)x, (unsigned)(256 / x));
    const bool past = streams_past(2 * r.tokens * (r.q_heads + r.k_heads) * r.head_dim * (int64_t)sizeof(T));
    auto go = [&](auto interleaved, auto stream_past) {
        hipLaunchKernelGGL((rotary_kernel<T, interleaved.value, stream_past.value>), grid, block, 0, stream, a);
    };
    if (r.layout == DDP_ROTARY_HALF)
        past ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
    else
        past ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
    return launched("ddp_rotary");
}

}  // namespace
}  // namespace ddp

extern "C" int ddp_rotary_frequencies(int scaling, int rotated, double base, double factor, double low, double high, double context, double *freq) {
    using namespace ddp;
    return guarded(nullptr, [&]() -> int {
        const char *who = "ddp_rotary_frequencies";
        if (!freq) return bad(who, DDP_EINVAL, "freq is NULL");
        if (rotated < 2 || rotated > DDP_ROTARY_MAX_ROTATED || rotated % 2) return bad(who, DDP_EINVAL, "rotated must be even and in [2, 256]");
        if (!(base > 0) || !std::isfinite(base)) return bad(who, DDP_EINVAL, "base must be positive");
        if (scaling < DDP_ROTARY_PLAIN || scaling > DDP_ROTARY_BY_WAVELENGTH) return bad(who, DDP_EINVAL, "unknown scaling");
        if (scaling != DDP_ROTARY_PLAIN && (!(factor > 0) || !std::isfinite(factor))) return bad(who, DDP_EINVAL, "factor must be positive");
        if (scaling == DDP_ROTARY_STRETCHED && rotated == 2) return bad(who, DDP_EINVAL, "a stretched base needs more than one pair");
        if (scaling == DDP_ROTARY_BY_WAVELENGTH && (!(context > 0) || !(low < high) || !std::isfinite(low) || !std::isfinite(high) || !std::isfinite(context)))
            return bad(who, DDP_EINVAL, "by wavelength, context must be positive and low < high");
        if (scaling == DDP_ROTARY_STRETCHED) base *= std::pow(factor, (double)rotated / (rotated - 2));
        for (int i = 0; i < rotated / 2; ++i) {
            double f = std::pow(base, -2.0 * i / rotated);
            if (scaling == DDP_ROTARY_LINEAR) f /= factor;
            if (scaling == DDP_ROTARY_BY_WAVELENGTH) {
                const double turns = context * f / (2 * 3.14159265358979323846);
                const double s = turns > high ? 1.0 : turns < low ? 0.0 : (turns - low) / (high - low);
                f = (1 - s) * f / factor + s * f;
            }
            freq[i] = f;
        }
        return DDP_OK;
    });
}

extern "C" int ddp_rotary_table(int rotated, const double *freq, double amplitude, int64_t rows, float *table, void *stream) {
    using namespace ddp;
    return guarded(nullptr, [&]() -> int {
        const char *who = "ddp_rotary_table";
        if (!freq || (!table && rows > 0)) return bad(who, DDP_EINVAL, "NULL pointer");
        if (rotated < 2 || rotated > DDP_ROTARY_MAX_ROTATED || rotated % 2) return bad(who, DDP_EINVAL, "rotated must be even and in [2, 256]");
        if (rows < 0 || rows > ((int64_t)1 << 31)) return bad(who, DDP_EINVAL, "rows must be in [0, 2^31]");
        if (misaligned(table, 4)) return bad(who, DDP_EALIGN, "table is not aligned to its element type");
        if (rows == 0) return DDP_OK;
        Frequencies f{};
        for (int i = 0; i < rotated / 2; ++i) f.f[i] = freq[i];
        const int64_t n = rows * (rotated / 2), wgs = cdiv(n, 256);
        hipLaunchKernelGGL(table_kernel, dim3((unsigned)(wgs < most_groups(256) ? wgs : most_groups(256))), dim3(256), 0, static_cast<hipStream_t>(stream), f, amplitude, n, rotated / 2, table);
        return launched(who);
    });
}

extern "C" int ddp_rotary(const ddp_rotary_shape *shape, const void *q, const void *k, const float *table, const void *positions, void *q_out, void *k_out,
                          void *stream) {
    using namespace ddp;
    return guarded(nullptr, [&]() -> int {
        const char *who = "ddp_rotary";
        if (!shape) return bad(who, DDP_EINVAL, "shape is NULL");
        const ddp_rotary_shape &r = *shape;
        if (!typed(r.dtype)) return bad(who, DDP_EINVAL, "dtype must be DDP_F32 or DDP_BF16");
        if (r.layout != DDP_ROTARY_HALF && r.layout != DDP_ROTARY_INTERLEAVED) return bad(who, DDP_EINVAL, "unknown layout");
        if (r.tokens < 0 || r.tokens > ((int64_t)1 << 40)) return bad(who, DDP_EINVAL, "tokens out of range");
        if (r.q_heads < 1 || r.k_heads < 0 || r.q_heads > 65536 || r.k_heads > 65536) return bad(who, DDP_EINVAL, "heads out of range");
        if (r.head_dim < 2 || r.head_dim > 65536) return bad(who, DDP_EINVAL, "head_dim out of range");
        if (r.rotated < 2 || r.rotated > DDP_ROTARY_MAX_ROTATED || r.rotated % 2 || r.rotated > r.head_dim)
            return bad(who, DDP_EINVAL, "rotated must be even, in [2, 256] and at most head_dim");
        if (r.table_rows < 1 || r.table_rows > ((int64_t)1 << 31)) return bad(who, DDP_EINVAL, "table_rows out of range");
        if (positions ? r.position_bytes != 4 && r.position_bytes != 8 : r.sequence < 1 || r.sequence > r.table_rows)
            return bad(who, DDP_EINVAL, positions ? "position_bytes must be 4 or 8" : "sequence must be in [1, table_rows] without positions");
        if (r.tokens == 0) return DDP_OK;
        if (!table || misaligned(table, 4)) return bad(who, table ? DDP_EALIGN : DDP_EINVAL, "table is NULL or not aligned");
        if (positions && misaligned(positions, (size_t)r.position_bytes)) return bad(who, DDP_EALIGN, "positions are not aligned");
        if (int rc = check_side(who, q, q_out, r, r.q_heads, r.q_token, r.q_head, r.q_out_token, r.q_out_head)) return rc;
        if (int rc = check_side(who, k, k_out, r, r.k_heads, r.k_token, r.k_head, r.k_out_token, r.k_out_head)) return rc;
        RotaryArgs a{};
        a.x[0] = q, a.x[1] = k, a.y[0] = q_out, a.y[1] = k_out;
        a.heads[0] = r.q_heads, a.heads[1] = r.k_heads;
        a.x_token[0] = r.q_token, a.x_head[0] = r.q_head, a.x_token[1] = r.k_token, a.x_head[1] = r.k_head;
        a.y_token[0] = r.q_out_token, a.y_head[0] = r.q_out_head, a.y_token[1] = r.k_out_token, a.y_head[1] = r.k_out_head;
        a.table = table, a.positions = positions, a.tokens = r.tokens, a.table_rows = r.table_rows, a.sequence = positions ? 1 : r.sequence;
        a.dim = r.head_dim, a.half = r.rotated / 2, a.position_bytes = r.position_bytes, a.inverse = r.inverse != 0;
        const hipStream_t st = static_cast<hipStream_t>(stream);
        return r.dtype == DDP_BF16 ? launch_rotary<bf16>(r, a, st) : launch_rotary<float>(r, a, st);
    });
}
