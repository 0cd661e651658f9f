// Cross entropy of a language model's head, from hidden states x [tokens, hidden] and weight [vocab, hidden].
//
// Three matrix products of 2 tokens vocab hidden operations each bound it: the logits z = x weight^T, in the forward call and again in the
// backward call, dx = dz weight and dweight = dz^T x.  All run in one tiled product whose operands lie either with k along their rows or
// with k down them, so nothing is transposed in memory; what is done with a tile of the product differs:
//   forward    a tile's logits stay in registers, and only their maximum and sum of exponentials per token leave it
//   backward   a tile becomes dz in dtype, for a piece of the vocabulary at a time, and two products go over the piece
//
// Measured, 8192 tokens, 128256 words of 4096 in bf16: logits 6.8 to 7.2 ms, and for each of eight pieces dz .89, dx .87, dweight .88 ms: 1.19 to 1.25
// Pflop/s.  fp32, 2048 tokens, 50257 words of 768, six bf16 products each: .89, .99, .80 and 1.0 ms, 1.0 to 1.15 Pflop/s of them.
//
// Registers of the large tiles: the logits kernel keeps 210 scalar ones in lanes of vector registers, dx's product 12 vector ones in scratch memory (52
// bytes a lane), both outside the loop of the products.
#include "ddp_operators.h"

namespace ddp {
namespace {

// ---- the product ---------------------------------------------------------------------------------------------------
// C[M, N] = sum_k A(m, k) B(n, k).  KROW: an operand's rows are its m (n), k along them; KMAJ: its rows are k, m (n) along them.
// A workgroup has TM x TN of C, WM x WN wavefronts of MI x NI accumulators of 32 x 32.  A step takes BK of k, from one of four LDS
// buffers that the loads write directly; three steps' loads are under way while one's products run.
//
// fp32 operands are planes of bf16 (Triple), whose six products are six steps of the same loop.
struct Operand {
    const void *p;
    int64_t stride;  // elements between rows
    int64_t rows;    // that may be read; beyond, the last one is read again
    int64_t groups;  // 16-byte groups of a row that may be read (KMAJ); beyond, the last one is
    int64_t plane;   // elements between the planes
};

constexpr int BK = 32;  // k of a step

template <class T_, int WM_, int WN_, int MI_, int NI_>
struct Shape {
    typedef T_ T;
    static constexpr int WM = WM_, WN = WN_, MI = MI_, NI = NI_, TM = 32 * WM * MI, TN = 32 * WN * NI, THREADS = 64 * WM * WN, STAGE = (TM + TN) * BK * 2;
};

// One operand's part of a tile, BK of k of ROWS rows, on its way to LDS: 16 bytes a lane and load, written where the lane is in
// the wavefront's kilobyte, so that the tile's exchange of groups (swizzle) is one of the addresses read.
template <class T, int ROWS, int THREADS, bool KMAJ>
struct Loader {
    static constexpr int PER_ROW = KMAJ ? ROWS / 8 : BK / 8, EACH = ROWS * BK / 8 / THREADS, ROWB = PER_ROW * 16, BYTES = ROWS * BK * 2;
    static constexpr int STEP = THREADS / PER_ROW;  // rows between a lane's loads
    static_assert(STEP % 16 == 0, "a lane's loads are exchanged alike");
    const char *base;    // of the tile (KROW), or of its columns' row 0 (KMAJ); uniform
    int64_t rows;        // KMAJ: of k
    int64_t plane;       // bytes
    int row_bytes;
    int row, column;
    int last_row;        // KROW: that may be read, counted from the tile's
    __device__ __forceinline__ Loader(const Operand &o, int64_t first) {
        row_bytes = (int)(o.stride * 2);
        rows = o.rows;
        plane = o.plane * 2;
        row = threadIdx.x / PER_ROW;
        int group = (int)(threadIdx.x % PER_ROW) ^ swizzle<ROWB>(row);
        if constexpr (KMAJ) {
            base = static_cast<const char *>(o.p) + first * 2;
            const int last = (int)(o.groups - 1 - first / 8 < PER_ROW ? o.groups - 1 - first / 8 : PER_ROW);
            group = group < last ? group : last;
        } else {
            // (a tile that lies behind the last row, as the padded end of a piece may, has that row)
            if (first > rows - 1) first = rows - 1;
            base = static_cast<const char *>(o.p) + first * row_bytes;
            last_row = (int)(rows - 1 - first < ROWS ? rows - 1 - first : ROWS);
        }
        column = group * 16;
    }
    __device__ __forceinline__ void start(int step, bool b, char *tile) const {
        const char *from = base;
        if constexpr (kTriple<T>) {
            from += plane_of(step % kProducts, b) * plane;
            step /= kProducts;
        }
        // (what lies behind the last row of k is that row again)
        const int64_t k0 = KMAJ ? ((int64_t)step * BK < rows - 1 ? (int64_t)step * BK : rows - 1) : 0;
        from += KMAJ ? k0 * row_bytes : (int64_t)step * (BK * 2);
        const int last = KMAJ ? (int)(rows - 1 - k0 < BK ? rows - 1 - k0 : BK) : last_row;
        DDP_LDS char *to = (DDP_LDS char *)tile + uniform(threadIdx.x & ~63) * 16;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int r = row + i * STEP < last ? row + i * STEP : last;
            const char *x = from + (unsigned)(r * row_bytes + column);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)x, (DDP_LDS void *)(to + i * THREADS * 16), 16, 0, 0);
        }
    }
    // eight elements of k from ks * 16 on of 32 rows
    static __device__ __forceinline__ bf16x8 operand(const char *tile, int row0, int ks, int lane) {
        if constexpr (KMAJ)
            return tile_col<ROWB, true>(tile, ks * 16, row0, lane);
        else
            return tile_row<ROWB>(tile, row0 + (lane & 31), 2 * ks + (lane >> 5));
    }
};

// All but the last `LEFT` of a wavefront's direct loads have arrived, everybody's with the barrier, and everybody's reads before it are done.
template <int LEFT>
__device__ __forceinline__ void arrived() {
    // (by the builtin, so that the compiler knows what has arrived and adds no wait of its own)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | 7 << 4 | LEFT >> 4 << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The products of steps [from, to).  A step's barrier waits for the loads that are read until the next one, and for no others: the rest go
// on while the products run.  The next step's first operands are read with this step's last products, except where both operands are read
// across their rows, whose addresses leave no registers for it (.89 ms for 4096 x 16128 of 8192 instead of 1.2).  Bound by the matrix
// cores at the clock that their power leaves: 8192 x 128256 of 4096 takes 6.9 ms, 1.25 Pflop/s, the cores busy 71 % of the time at 1.6 GHz
// (a large library product of these operands 1.3 Pflop/s, 85 % at 1.5 GHz).  Measured and not taken: steps of 64 of k with two buffers,
// all of whose loads a barrier waited for, 7.3 ms; four wavefronts of 4 x 4 accumulators, 7.4; a raised priority during the products, 7.3.
template <class S, bool AK, bool BKMAJ>
__device__ __forceinline__ void product(f32x16 (&c)[S::MI][S::NI], const Operand &a, const Operand &b, int64_t m0, int64_t n0, int from, int to, char *lds0,
                                        char *lds1, char *lds2, char *lds3) {
    typedef Loader<typename S::T, S::TM, S::THREADS, AK> LA;
    typedef Loader<typename S::T, S::TN, S::THREADS, BKMAJ> LB;
    if (from >= to) return;  // (a split of a short piece)
    const LA la(a, m0);
    const LB lb(b, n0);
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int am = wave / S::WN * (32 * S::MI), bn = wave % S::WN * (32 * S::NI);
    constexpr int LOADS = LA::EACH + LB::EACH;
    constexpr bool AHEAD = !(AK && BKMAJ);
    auto start = [&](int step, char *lds) {
        step = step < to ? step : to - 1;  // (behind the last one: read again, and not used)
        la.start(step, false, lds);
        lb.start(step, true, lds + LA::BYTES);
    };
    bf16x8 av[2][S::MI], bv[2][S::NI];
    auto read = [&](const char *lds, int ks) {
#pragma unroll
        for (int j = 0; j < S::NI; ++j) bv[ks & 1][j] = LB::operand(lds + LA::BYTES, bn + 32 * j, ks, lane);
#pragma unroll
        for (int i = 0; i < S::MI; ++i) av[ks & 1][i] = LA::operand(lds, am + 32 * i, ks, lane);
    };
    constexpr int READS = S::MI * (AK ? 2 : 1) + S::NI * (BKMAJ ? 2 : 1), PRODUCTS = S::MI * S::NI, SLOTS = PRODUCTS > 2 ? PRODUCTS - 2 : 1,
                  EACH = (READS + SLOTS - 1) / SLOTS;
    auto all = [&](int ks, bool reads) {
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int j = 0; j < S::NI; ++j) c[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[ks & 1][i], bv[ks & 1][j], c[i][j], 0, 0, 0);
        // the next operands' reads go between these products, evenly and early
        if (reads)
#pragma unroll
            for (int i = 0; i < PRODUCTS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (i * EACH < READS) __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](const char *lds, const char *next) {
        if constexpr (!AHEAD) read(lds, 0);
        read(lds, 1);
        all(0, true);
        if constexpr (AHEAD) read(next, 0);
        all(1, AHEAD);
    };
    start(from, lds0);
    start(from + 1, lds1);
    start(from + 2, lds2);
    if constexpr (AHEAD) {
        arrived<2 * LOADS>();
        read(lds0, 0);
    }
    int s = from;
    constexpr int LEFT = AHEAD ? LOADS : 2 * LOADS;
    for (; s + 4 <= to; s += 4) {
        arrived<LEFT>();
        start(s + 3, lds3);
        multiply(lds0, lds1);
        arrived<LEFT>();
        start(s + 4, lds0);
        multiply(lds1, lds2);
        arrived<LEFT>();
        start(s + 5, lds1);
        multiply(lds2, lds3);
        arrived<LEFT>();
        start(s + 6, lds2);
        multiply(lds3, lds0);
    }
    // (one to three steps more: they are under way)
    arrived<0>();
    if (s < to) multiply(lds0, lds1);
    if (s + 1 < to) multiply(lds1, lds2);
    if (s + 2 < to) multiply(lds2, lds0);
    __syncthreads();
}

// Workgroups go to the eight XCDs in turn: each XCD takes a run of tiles of its own, in columns of up to eight tiles of m, so that what its
// L2 holds of both operands is used by several tiles.
__device__ __forceinline__ void tile_of(int64_t mt, int64_t nt, int64_t &m, int64_t &n) {
    const int64_t all = mt * nt, per = all / 8, rest = all % 8;
    const int64_t x = blockIdx.x % 8, i = blockIdx.x / 8;
    const int64_t id = x * per + (x < rest ? x : rest) + i;
    const int64_t band = 8 * nt, b = id / band, in = id - b * band, tall = mt - b * 8 < 8 ? mt - b * 8 : 8;
    m = b * 8 + in % tall;
    n = in / tall;
}

// ---- forward -------------------------------------------------------------------------------------------------------
struct LogitArgs {
    Operand x, w;
    int64_t tokens, vocab, steps;
    int64_t v0;       // first word of this launch's weight rows
    int64_t mt, nt;   // tiles of words and of tokens
    const int64_t *targets;
    float2 *part;     // forward: [mt][tokens] maximum (of z * log2 e) and sum
    float *picked;    // forward: [tokens] the target's logit
    const float *lse, *dloss;  // backward
    const float *most;         // backward: the largest |dloss|, which dz is relative to
    void *dz;         // backward: [token rows][piece]
    int64_t piece, token_rows;
};

template <class S>
__global__ __launch_bounds__(S::THREADS) void logits_kernel(const LogitArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds0[S::STAGE], lds1[S::STAGE], lds2[S::STAGE], lds3[S::STAGE];
    __shared__ float2 meet[S::WM][S::TN];
    int64_t mt, nt;
    tile_of(a.mt, a.nt, mt, nt);
    f32x16 c[S::MI][S::NI] = {};
    product<S, false, false>(c, a.w, a.x, mt * S::TM, nt * S::TN, 0, (int)a.steps, lds0, lds1, lds2, lds3);
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5, wm = wave / S::WN, wn = wave % S::WN;
#pragma unroll
    for (int j = 0; j < S::NI; ++j) {
        const int col = wn * 32 * S::NI + 32 * j + (lane & 31);
        const int64_t token = nt * S::TN + col, aim = token < a.tokens ? a.targets[token] : -1;
        const int first = (int)mt * S::TM + wm * 32 * S::MI, vocab = (int)a.vocab, target = aim >= 0 && aim < vocab ? (int)aim : -1;
        float m = -kInf;
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int word = first + 32 * i + acc_row(half, r);
                if (word == target) a.picked[token] = c[i][j][r];
                c[i][j][r] = word < vocab ? c[i][j][r] * kLog2e : -kInf;
                m = fmaxf(m, c[i][j][r]);
            }
        m = fmaxf(m, __shfl_xor(m, 32));
        const float base = m == -kInf ? 0.0f : m;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) s += __builtin_amdgcn_exp2f(c[i][j][r] - base);
        s += __shfl_xor(s, 32);
        if (half == 0) meet[wm][col] = float2{m, s};
    }
    __syncthreads();
    for (int col = threadIdx.x; col < S::TN; col += S::THREADS) {
        const int64_t token = nt * S::TN + col;
        if (token >= a.tokens) continue;
        float m = meet[0][col].x;
#pragma unroll
        for (int i = 1; i < S::WM; ++i) m = fmaxf(m, meet[i][col].x);
        const float base = m == -kInf ? 0.0f : m;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < S::WM; ++i) s += meet[i][col].y * exp2f(meet[i][col].x - base);
        a.part[mt * a.tokens + token] = float2{m, s};
    }
}

// Joins the tiles' maxima and sums: 16 tokens a workgroup, 16 runs of tiles each.
__global__ __launch_bounds__(256) void join_kernel(const float2 *part, int64_t tiles, int64_t tokens, int64_t vocab, const int64_t *targets, const float *picked,
                                                   float *loss, float *lse) {
    __shared__ float2 run[16][16];
    const int col = threadIdx.x & 15, r = threadIdx.x >> 4;
    const int64_t token = (int64_t)blockIdx.x * 16 + col;
    float m = -kInf, s = 0.0f;
    if (token < tokens)
        for (int64_t i = r; i < tiles; i += 16) {
            const float2 p = part[i * tokens + token];
            const float top = fmaxf(m, p.x), base = top == -kInf ? 0.0f : top;
            s = s * exp2f(m - base) + p.y * exp2f(p.x - base);
            m = top;
        }
    run[r][col] = float2{m, s};
    __syncthreads();
    if (r || token >= tokens) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) {
        const float2 p = run[i][col];
        const float top = fmaxf(m, p.x), base = top == -kInf ? 0.0f : top;
        s = s * exp2f(m - base) + p.y * exp2f(p.x - base);
        m = top;
    }
    const float l = m * kLn2 + logf(s);
    lse[token] = l;
    const int64_t t = targets[token];
    loss[token] = t >= 0 && t < vocab ? l - picked[token] : 0.0f;
}

// ---- backward ------------------------------------------------------------------------------------------------------
// dz is rounded relative to the largest |dloss| of the tokens that have a target, which multiplies the results: where all are
// the same, as under a mean, the target's p - 1 is rounded close to 1, where a factor of its own would round all tokens' the same way.
__global__ __launch_bounds__(1024) void most_kernel(const float *dloss, const int64_t *targets, int64_t tokens, int64_t vocab, float *most) {
    __shared__ float meet[16];
    float m = 0.0f;
    for (int64_t t = threadIdx.x; t < tokens; t += 1024) {
        const float g = fabsf(dloss[t]);
        if (targets[t] >= 0 && targets[t] < vocab && g < kInf) m = fmaxf(m, g);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if ((threadIdx.x & 63) == 0) meet[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) m = fmaxf(m, meet[i]);
    *most = m > 0.0f ? m : 1.0f;
}

template <class S>
__global__ __launch_bounds__(S::THREADS) void dlogits_kernel(const LogitArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds0[S::STAGE], lds1[S::STAGE], lds2[S::STAGE], lds3[S::STAGE];
    int64_t mt, nt;
    tile_of(a.mt, a.nt, mt, nt);
    f32x16 c[S::MI][S::NI] = {};
    product<S, false, false>(c, a.w, a.x, mt * S::TM, nt * S::TN, 0, (int)a.steps, lds0, lds1, lds2, lds3);
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5, wm = wave / S::WN, wn = wave % S::WN;
#pragma unroll
    for (int j = 0; j < S::NI; ++j) {
        const int64_t token = nt * S::TN + wn * 32 * S::NI + 32 * j + (lane & 31);
        const int first = (int)mt * S::TM + wm * 32 * S::MI, v0 = (int)a.v0, vocab = (int)a.vocab;
        if (token >= a.token_rows) continue;
        float g = 0.0f, lse2 = 0.0f;
        int target = -1;
        if (token < a.tokens) {
            const int64_t aim = a.targets[token];
            target = aim >= 0 && aim < vocab ? (int)aim : -1;
            g = target < 0 ? 0.0f : a.dloss[token] / *a.most;
            lse2 = a.lse[token] * kLog2e;
        }
        bf16 *row = static_cast<bf16 *>(a.dz) + token * a.piece + first;
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int word = v0 + first + 32 * i + acc_row(half, r);
                const float p = __builtin_amdgcn_exp2f(c[i][j][r] * kLog2e - lse2) - (word == target ? 1.0f : 0.0f);
                c[i][j][r] = target >= 0 && word < vocab ? g * p : 0.0f;
            }
            // (a piece is whole tiles)
            store_acc(row + 32 * i, c[i][j], 1.0f, 32);
            if constexpr (kTriple<typename S::T>)
#pragma unroll
                for (int k = 1; k < 3; ++k) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) c[i][j][r] = left_over(c[i][j][r]);
                    store_acc(row + 32 * i + k * a.token_rows * a.piece, c[i][j], 1.0f, 32);
                }
        }
    }
}

struct GradArgs {
    Operand a, b;
    int64_t rows_m, rows_n;   // of the result: hidden, and tokens or words; of logits in splits, words and tokens
    int64_t steps, mt, nt;
    int splits;               // that the steps are split into, each with sums of its own
    void *out;                // [rows_n][out_stride], m along the rows
    float *acc;               // [splits][rows_n][rows_m], where the result is the sum of several splits or pieces
    int64_t out_stride;
    int first, last;          // whether the sums start here, and whether the result is written here
    const float *most;        // multiplies the result
};

template <class S, bool AK, bool BKMAJ>
__global__ __launch_bounds__(S::THREADS) void grad_kernel(const GradArgs g) {
    typedef typename S::T T;
    __shared__ __attribute__((aligned(1024))) char lds0[S::STAGE], lds1[S::STAGE], lds2[S::STAGE], lds3[S::STAGE];
    int64_t mt, nt;
    tile_of(g.mt, g.nt, mt, nt);
    const int64_t split = blockIdx.y;
    f32x16 c[S::MI][S::NI] = {};
    product<S, AK, BKMAJ>(c, g.a, g.b, mt * S::TM, nt * S::TN, (int)(split * g.steps / g.splits), (int)((split + 1) * g.steps / g.splits), lds0, lds1, lds2, lds3);
    const float most = AK ? *g.most : 1.0f;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5, wm = wave / S::WN, wn = wave % S::WN;
#pragma unroll
    for (int j = 0; j < S::NI; ++j) {
        const int64_t n = nt * S::TN + wn * 32 * S::NI + 32 * j + (lane & 31);
        if (n >= g.rows_n) continue;
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
            const int64_t m = mt * S::TM + wm * 32 * S::MI + 32 * i;
            const int left = (int)(g.rows_m - m < 32 ? g.rows_m - m : 32);
            if (left <= 0) continue;
            float *acc = g.acc + (split * g.rows_n + n) * g.rows_m + m;
            if (!g.first) {
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int at = acc_row(half, r);
                    if (at >= left) continue;
                    const f32x4 v = load_part(acc + at, left - at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[i][j][r + e] += v[e];
                }
            }
            if (g.last)
                store_acc(static_cast<Out<T> *>(g.out) + n * g.out_stride + m, c[i][j], most, left);
            else
                store_acc(acc, c[i][j], 1.0f, left);
        }
    }
}

// The splits' sums, in their order; a thread four elements.
template <class T>
__global__ __launch_bounds__(256) void split_join_kernel(const GradArgs g) {
    const float most = g.most ? *g.most : 1.0f;
    const int64_t per = (g.rows_m + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < g.rows_n * per; i += (int64_t)gridDim.x * 256) {
        const int64_t n = i / per, m = (i - n * per) * 4;
        const int left = (int)(g.rows_m - m < 4 ? g.rows_m - m : 4);
        f32x4 v = {};
        const float *from = g.acc + n * g.rows_m + m;
        const int64_t apart = g.rows_n * g.rows_m;
        if (left == 4) {
#pragma unroll 8
            for (int s = 0; s < g.splits; ++s) v += load_group(from + s * apart);
        } else {
            for (int j = 0; j < left; ++j) {
                float sum = 0.0f;
#pragma unroll 8
                for (int s = 0; s < g.splits; ++s) sum += from[s * apart + j];
                v[j] = sum;
            }
        }
        store4(static_cast<Out<T> *>(g.out) + n * g.out_stride + m, v * most, left);
    }
}

// Few tokens are few tiles, each with all of hidden to go over: their logits are formed in splits of hidden, whose sums these two kernels
// take up where the whole products' kernels would: a token a y of the grid, 1024 words a workgroup, four a thread.
__device__ __forceinline__ f32x4 split_logits(const GradArgs &g, int64_t token, int64_t word, int left) {
    f32x4 v = {};
    for (int s = 0; s < g.splits; ++s) v += load_part(g.acc + (s * g.rows_n + token) * g.rows_m + word, left);
    return v;
}
__global__ __launch_bounds__(256) void split_logits_kernel(const LogitArgs a, const GradArgs g) {
    __shared__ float2 meet[4];
    const int64_t token = blockIdx.y, word = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, aim = a.targets[token];
    float m = -kInf, s = 0.0f;
    f32x4 z = {-kInf, -kInf, -kInf, -kInf};
    if (word < a.vocab) {
        const int left = (int)(a.vocab - word < 4 ? a.vocab - word : 4);
        const f32x4 v = split_logits(g, token, word, left);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) {
                if (word + j == aim) a.picked[token] = v[j];
                z[j] = v[j] * kLog2e;
                m = fmaxf(m, z[j]);
            }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    const float base = m == -kInf ? 0.0f : m;
#pragma unroll
    for (int j = 0; j < 4; ++j) s += __builtin_amdgcn_exp2f(z[j] - base);
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) meet[threadIdx.x >> 6] = float2{m, s};
    __syncthreads();
    if (threadIdx.x) return;
#pragma unroll
    for (int i = 1; i < 4; ++i) m = fmaxf(m, meet[i].x);
    const float top = m == -kInf ? 0.0f : m;
    s *= exp2f(base - top);
#pragma unroll
    for (int i = 1; i < 4; ++i) s += meet[i].y * exp2f(meet[i].x - top);
    a.part[blockIdx.x * a.tokens + token] = float2{m, s};
}
template <class T>
__global__ __launch_bounds__(256) void split_dlogits_kernel(const LogitArgs a, const GradArgs g) {
    const int64_t token = blockIdx.y, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= a.piece) return;
    f32x4 z = {};
    if (token < a.tokens) {
        const int64_t aim = a.targets[token], left = a.vocab - a.v0 - at;
        const bool valid = aim >= 0 && aim < a.vocab;
        const float by = valid ? a.dloss[token] / (a.most ? *a.most : 1.0f) : 0.0f, lse2 = a.lse[token] * kLog2e;
        if (valid && left > 0) {
            const f32x4 v = split_logits(g, token, at, (int)(left < 4 ? left : 4));
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < left) z[j] = by * (__builtin_amdgcn_exp2f(v[j] * kLog2e - lse2) - (a.v0 + at + j == aim ? 1.0f : 0.0f));
        }
    }
    if constexpr (std::is_same_v<T, float>) {
        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.dz) + token * a.piece + at) = z;
        return;
    }
    bf16 *to = static_cast<bf16 *>(a.dz) + token * a.piece + at;
#pragma unroll
    for (int k = 0; k < kPlanes<T>; ++k) {
        *reinterpret_cast<bf16x4 *>(to + k * a.token_rows * a.piece) = __builtin_convertvector(z, bf16x4);
        if (k + 1 < kPlanes<T>)
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] = left_over(z[j]);
    }
}

// ---- fp32 and few tokens -------------------------------------------------------------------------------------------
// Up to 64 tokens a product of fp32 takes less time on the fp32 matrix instruction (64 flop a cycle and SIMD) than planes of the weight
// take to write and read (a pass of 16 tokens, 6787 words of 2590: 280 us with planes, 127 so; 53, 15401 of 3002: 545 and 425; 64, 1302 of 123: 67 and
// 65), so these read the tensors as they lie, each operand straight into registers: four elements of a row a lane, whose places in k
// (or columns) are spread over four instructions; the sum over k has no order to keep.  Lane l of an operand has row (column) l % 32 and k l / 32.
constexpr int kFew = 64;

// A tile's sums of the workgroup's four wavefronts, in the first one's registers.
template <int N>
__device__ __forceinline__ void add_waves(f32x16 (&c)[N], float (*meet)[16][64]) {
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        __syncthreads();
        if (wave)
#pragma unroll
            for (int r = 0; r < 16; ++r) meet[wave - 1][r][lane] = c[n][r];
        __syncthreads();
        if (!wave)
#pragma unroll
            for (int r = 0; r < 16; ++r) c[n][r] += meet[0][r][lane] + meet[1][r][lane] + meet[2][r][lane];
    }
}

// four elements, or as many as are left (no more than four of them)
template <bool WHOLE>
__device__ __forceinline__ f32x4 four(const float *p, int left) {
    if constexpr (WHOLE)
        return load_group(p);
    else
        return load_part(p, left);
}
// f(whether all loads are of four), so that those that are need no branch each, and all are under way at once
template <class F>
__device__ __forceinline__ void by_whole(bool whole, F &&f) {
    if (whole)
        f(std::true_type{});
    else
        f(std::false_type{});
}

struct FewArgs {
    const float *x, *w, *dz;
    int64_t x_stride, w_stride, dz_stride, out_stride;
    int tokens, words, hidden, splits;
    float *out;  // logits [splits][tokens][words], dx [splits][tokens][hidden], dweight [words][out_stride]
};

// Logits of 64 words and a split of hidden, a quarter of it a wavefront, 32 at a time.  23 tokens, 94675 words of 368: 51 us, 2.7 TB/s; 53, 15401
// of 3002: 110 to 125 us, the matrix cores busy 45 % of the time on 180 of 256 compute units.
template <int MT>
__global__ __launch_bounds__(256) void few_logits_kernel(const FewArgs a) {
    __shared__ float meet[3][16][64];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5;
    const float *xr[MT], *wr[2];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int t = 32 * i + (lane & 31);
        xr[i] = a.x + (t < a.tokens ? t : a.tokens - 1) * a.x_stride;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int v = blockIdx.x * 64 + 32 * j + (lane & 31);
        wr[j] = a.w + (v < a.words ? v : a.words - 1) * a.w_stride;
    }
    const int blocks = (a.hidden + 31) / 32, parts = 4 * a.splits, part = blockIdx.y * 4 + wave;
    f32x16 c[2 * MT] = {};
    for (int b = (int)((int64_t)blocks * part / parts); b < (int)((int64_t)blocks * (part + 1) / parts); ++b) {
        f32x4 u[4][MT], v[4][2];
        by_whole(b * 32 + 32 <= a.hidden, [&](auto whole) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int k = b * 32 + g * 8 + half * 4;
#pragma unroll
                for (int i = 0; i < MT; ++i) u[g][i] = four<whole.value>(xr[i] + k, a.hidden - k);
#pragma unroll
                for (int j = 0; j < 2; ++j) v[g][j] = four<whole.value>(wr[j] + k, a.hidden - k);
            }
        });
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) c[2 * i + j] = __builtin_amdgcn_mfma_f32_32x32x2f32(u[g][i][e], v[g][j][e], c[2 * i + j], 0, 0, 0);
    }
    add_waves(c, meet);
    if (wave) return;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int word = blockIdx.x * 64 + 32 * j + (lane & 31);
            if (word >= a.words) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int t = 32 * i + acc_row(half, r);
                if (t < a.tokens) a.out[((int64_t)blockIdx.y * a.tokens + t) * a.words + word] = c[2 * i + j][r];
            }
        }
}

// dx of 128 columns and a split of the words, a quarter of it a wavefront, eight at a time: a lane has four columns.  53 tokens, 15401 words of
// 3002: 123 us with one wavefront a SIMD, 98 with two.
template <int MT>
__global__ __launch_bounds__(256, 2) void few_dx_kernel(const FewArgs a) {
    __shared__ float meet[3][16][64];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5;
    const int col = blockIdx.x * 128 + 4 * (lane & 31), left = a.hidden - col;
    const float *zr[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int t = 32 * i + (lane & 31);
        zr[i] = a.dz + (t < a.tokens ? t : a.tokens - 1) * a.dz_stride;
    }
    const int blocks = (a.words + 7) / 8, parts = 4 * a.splits, part = blockIdx.y * 4 + wave;
    f32x16 c[4 * MT] = {};
    by_whole((int)blockIdx.x * 128 + 128 <= a.hidden, [&](auto whole) {
        const int to = (int)((int64_t)blocks * (part + 1) / parts);
        f32x4 u[2][MT], v[2][4];
        auto load = [&](int b, int at) {  // (behind the last one: read again, and not used)
            const int k = (b < to ? b : to - 1) * 8 + half * 4;
#pragma unroll
            for (int i = 0; i < MT; ++i) u[at][i] = *reinterpret_cast<const f32x4 *>(zr[i] + k);  // (zeros behind the last word)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[at][e] = four<whole.value>(a.w + (int64_t)(k + e < a.words ? k + e : a.words - 1) * a.w_stride + col, left);
        };
        auto multiply = [&](int at) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) c[4 * i + j] = __builtin_amdgcn_mfma_f32_32x32x2f32(u[at][i][e], v[at][e][j], c[4 * i + j], 0, 0, 0);
        };
        int b = (int)((int64_t)blocks * part / parts);
        if (b >= to) return;
        load(b, 0);
        for (; b + 2 <= to; b += 2) {
            load(b + 1, 1);
            multiply(0);
            load(b + 2, 0);
            multiply(1);
        }
        if (b < to) multiply(0);
    });
    add_waves(c, meet);
    if (wave || left <= 0) return;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int t = 32 * i + acc_row(half, r);
            if (t < a.tokens) store_part(a.out + ((int64_t)blockIdx.y * a.tokens + t) * a.hidden + col, Vec<float>{c[4 * i][r], c[4 * i + 1][r], c[4 * i + 2][r], c[4 * i + 3][r]}, left);
        }
}

// dweight of 32 words and 128 columns a wavefront: all of a token's places are two rows an instruction.
__global__ __launch_bounds__(256) void few_dw_kernel(const FewArgs a) {
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5;
    const int col = blockIdx.x * 128 + 4 * (lane & 31), left = a.hidden - col;
    const int64_t word = ((int64_t)blockIdx.y * 4 + wave) * 32;
    if (word >= a.words) return;
    f32x16 c[4] = {};
    by_whole((int)blockIdx.x * 128 + 128 <= a.hidden, [&](auto whole) {
        for (int k0 = 0; k0 < a.tokens; k0 += 8) {
            f32x4 v[4];
            float u[4];
            bool there[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int k = k0 + 2 * e + half, t = k < a.tokens ? k : a.tokens - 1;
                there[e] = k < a.tokens;
                v[e] = four<whole.value>(a.x + t * a.x_stride + col, left);
                u[e] = a.dz[t * a.dz_stride + word + (lane & 31)];  // (zeros behind the last word)
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < 4; ++j) c[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(there[e] ? u[e] : 0.0f, there[e] ? v[e][j] : 0.0f, c[j], 0, 0, 0);
        }
    });
    if (left <= 0) return;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int64_t row = word + acc_row(half, r);
        if (row < a.words) store_part(a.out + row * a.out_stride + col, Vec<float>{c[0][r], c[1][r], c[2][r], c[3][r]}, left);
    }
}

// Rows of `cols` elements into rows of `padded`, zeros behind them: bf16 as it is, fp32 as three planes.  A thread has eight, which it reads
// at once from wherever they lie.
template <class T>
__global__ __launch_bounds__(256) void pad_rows_kernel(const Out<T> *x, int64_t stride, int64_t rows, int64_t cols, int64_t padded, bf16 *y) {
    typedef Out<T> E;
    const int64_t per = padded / 8, n = rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = n >> 32 ? i / per : (unsigned)i / (unsigned)per, c = (i - r * per) * 8;
        const E *from = x + r * stride + c;
        typedef E Eight __attribute__((ext_vector_type(8)));
        Eight v;
        if (c + 8 <= cols)
            __builtin_memcpy(&v, from, sizeof v);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? from[j] : (E)0.0f;
        bf16 *to = y + r * padded + c;
#pragma unroll
        for (int k = 0; k < kPlanes<T>; ++k) {
            bf16x8 o;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                o[j] = (bf16)v[j];
                if (k + 1 < kPlanes<T>) v[j] = (E)left_over((float)v[j]);
            }
            *reinterpret_cast<bf16x8 *>(to + k * rows * padded) = o;
        }
    }
}
template <class T>
__global__ __launch_bounds__(256) void zero_rows_kernel(T *x, int64_t stride, int64_t rows, int64_t cols) {
    const int64_t per = (cols + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * per; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per, c = (i - r * per) * 4;
        store4(x + r * stride + c, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, (int)(cols - c < 4 ? cols - c : 4));
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------
template <class T>
using Large = Shape<T, 2, 4, 4, 2>;  // 256 x 256
template <class T>
using Small = Shape<T, 2, 2, 2, 1>;  // 128 x 64

// How a product of m x n over `steps` steps is cut.  256 x 256 needs half the LDS and cache traffic per operation, 128 x 64 fills the chip with a
// quarter of the work; a gradient's product, whose k is long where the result is small, is also split along k, so that there are
// workgroups for all compute units.
struct Cut {
    bool large;
    int splits;
};
inline Cut cut_of(int64_t m, int64_t n, int64_t steps, bool may_split) {
    const int64_t tiles = cdiv(m, 256) * cdiv(n, 256), small = cdiv(m, 128) * cdiv(n, 64);
    if (tiles >= 192) return {true, 1};
    if (!may_split) return {false, 1};
    const int64_t s = 256 / tiles;  // (one round of workgroups, one a compute unit)
    if (s <= 16 && steps / s >= 32) return {true, (int)s};
    int64_t t = cdiv(512, small);
    t = t < 16 ? t : 16;
    t = t < steps / 32 ? t : steps / 32;  // (a shorter split takes less than its join)
    return {false, (int)(t > 1 ? t : 1)};
}

// Logits have a row of words a token to join, and are split where their tiles would leave half the chip without one: a pass of 100 tokens, 1000 words of
// 1024 in fp32 takes 126 us with whole products, 81 so; of 16 tokens, 6787 words of 2590 in bf16, 115 and 104.
inline Cut logit_cut(int64_t words, int64_t tokens, int64_t steps) {
    if (cut_of(words, tokens, steps, false).large) return {true, 1};
    int64_t t = 512 / (cdiv(words, 128) * cdiv(tokens, 64));
    t = t < 16 ? t : 16;
    t = t < steps / 16 ? t : steps / 16;
    return {false, (int)(t > 1 ? t : 1)};
}
constexpr int64_t kSplitWords = 1024;  // of a workgroup that joins logits' splits

struct Layout {  // of a call's workspace; offsets in bytes
    int64_t padded;         // hidden as the products take it
    bool copy_x, copy_w;
    int64_t x, w, part, picked, most, dz, acc, acc_w, logits, bytes;
    int64_t piece, pieces, token_rows;
};

int check_head(const char *who, const ddp_head *h) {
    if (!h) return bad(who, DDP_EINVAL, "the shape is NULL");
    if (!typed(h->dtype)) return bad(who, DDP_EINVAL, "dtype must be DDP_F32 or DDP_BF16");
    // (16 tokens, or 64 words, are a workgroup of 256 threads)
    if (h->tokens < 0 || h->tokens > 16 * most_groups(256)) return bad(who, DDP_EINVAL, "tokens must be in [0, 2^28 - 16]");
    if (h->vocab < 1 || h->vocab > 64 * most_groups(256)) return bad(who, DDP_EINVAL, "vocab must be in [1, 2^30 - 64]");
    if (h->hidden < 1 || h->hidden > (1 << 20)) return bad(who, DDP_EINVAL, "hidden must be in [1, 2^20]");
    if ((h->tokens > 1 && h->x_stride < h->hidden) || (h->vocab > 1 && h->w_stride < h->hidden)) return bad(who, DDP_EINVAL, "rows overlap: a stride is smaller than hidden");
    if (reach(h->tokens, h->x_stride) < 0 || reach(h->vocab, h->w_stride) < 0) return bad(who, DDP_EINVAL, "a stride is too large");
    // (the large tiles: products of few of them, which take small ones, are far from it)
    const int64_t tokens = cdiv(h->tokens, 256), words = cdiv(h->vocab, 256), columns = cdiv(h->hidden, 256), most = most_groups(512);
    if (tokens * words > most || columns * words > most || columns * tokens > most)
        return bad(who, DDP_EINVAL, "more than 2^23 tiles of 256 x 256: split the tokens over several calls");
    return DDP_OK;
}

// The products read 16-byte groups and whole steps of k: rows that are no multiple of them, or lie elsewhere, are copied into padded ones.
bool is_few(const ddp_head &h) { return h.dtype == DDP_F32 && h.tokens <= kFew; }
// splits of a few tokens' product with `tiles` workgroups and `most` at the longest
int few_splits(int64_t tiles, int64_t most) {
    int64_t n = cdiv(1024, tiles);
    n = n < most ? n : most;
    return (int)(n < 1 ? 1 : n < 64 ? n : 64);
}
int few_logit_splits(const ddp_head &h) { return few_splits(cdiv(h.vocab, 64), h.hidden / 256); }
int few_dx_splits(const ddp_head &h) { return few_splits(cdiv(h.hidden, 128), h.vocab / 128); }

Layout layout_of(const ddp_head &h, bool backward, const void *x, const void *w) {
    if (is_few(h)) {
        Layout l{};
        auto take = [&](int64_t bytes) {
            const int64_t here = l.bytes;
            l.bytes += up(bytes, 1024);
            return here;
        };
        l.logits = take(few_logit_splits(h) * h.tokens * h.vocab * 4);
        if (!backward) {
            l.part = take(cdiv(h.vocab, kSplitWords) * h.tokens * 8);
            l.picked = take(h.tokens * 4);
        } else {
            l.piece = up(h.vocab, 256);
            l.dz = take(h.tokens * l.piece * 4);
            l.acc = take(few_dx_splits(h) * h.tokens * h.hidden * 4);
        }
        return l;
    }
    constexpr int64_t step = 64;
    const bool triple = h.dtype == DDP_F32;
    const int64_t bytes = triple ? 6 : 2, products = triple ? kProducts : 1;  // of an element, and of a step
    Layout l{};
    l.padded = up(h.hidden, step);
    const bool ragged = h.hidden % step != 0;
    // (a tile's 256 rows are addressed with 31 bits)
    const int64_t far = ((int64_t)1 << 30) / (256 * 2);
    l.copy_x = triple || ragged || (h.tokens > 1 && (h.x_stride % 8 || h.x_stride >= far)) || misaligned(x, 16);
    l.copy_w = triple || ragged || (h.vocab > 1 && (h.w_stride % 8 || h.w_stride >= far)) || misaligned(w, 16);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up(bytes, 1024);
        return here;
    };
    if (!backward) {
        const Cut cut = logit_cut(h.vocab, h.tokens, l.padded / BK * products);
        const int64_t tiles = cdiv(h.vocab, cut.splits > 1 ? kSplitWords : cut.large ? 256 : 128);
        l.logits = cut.splits > 1 ? take(cut.splits * h.tokens * h.vocab * 4) : 0;
        l.part = take(tiles * h.tokens * 8);
        l.picked = take(h.tokens * 4);
    } else {
        l.token_rows = up(h.tokens, step);
        const int64_t words = up(h.vocab, 256), most = up(((int64_t)1 << 27) / l.token_rows + 1, 256);
        l.pieces = cdiv(words, most);
        l.piece = up(cdiv(words, l.pieces), 256);
        l.pieces = cdiv(words, l.piece);
        const Cut cut = logit_cut(l.piece, l.token_rows, l.padded / BK * products);
        l.logits = cut.splits > 1 ? take(cut.splits * l.token_rows * l.piece * 4) : 0;
        l.most = take(4);
        l.dz = take(l.token_rows * l.piece * bytes);
        const int of_x = cut_of(h.hidden, h.tokens, l.piece / BK * products, true).splits, of_w = cut_of(h.hidden, l.piece, l.token_rows / BK * products, true).splits;
        l.acc = of_x > 1 || l.pieces > 1 ? take(of_x * h.tokens * h.hidden * 4) : 0;
        l.acc_w = of_w > 1 ? take(of_w * l.piece * h.hidden * 4) : 0;
    }
    l.x = l.copy_x ? take(h.tokens * l.padded * bytes) : 0;
    l.w = l.copy_w ? take(h.vocab * l.padded * bytes) : 0;
    l.bytes = at;
    return l;
}

template <class T>
Operand operand(const ddp_head &h, const Layout &l, bool of_x, const void *p, char *ws, hipStream_t st) {
    const int64_t rows = of_x ? h.tokens : h.vocab, stride = rows > 1 ? (of_x ? h.x_stride : h.w_stride) : l.padded;
    if (!(of_x ? l.copy_x : l.copy_w)) return Operand{p, stride, rows, h.hidden / 8, 0};
    bf16 *to = reinterpret_cast<bf16 *>(ws + (of_x ? l.x : l.w));
    const int64_t n = cdiv(rows * (l.padded / 8), 256);
    hipLaunchKernelGGL((pad_rows_kernel<T>), dim3((unsigned)(n < (1 << 20) ? n : 1 << 20)), dim3(256), 0, st, static_cast<const Out<T> *>(p), stride, rows, h.hidden,
                       l.padded, to);
    return Operand{to, l.padded, rows, l.padded / 8, rows * l.padded};
}

int check_call(const char *who, const ddp_head &h, const void *x, const void *w, const void *targets, const void *a, const void *b, const void *ws, int64_t bytes,
               int64_t need) {
    if (!x || !w || !targets || !a || !b) return bad(who, DDP_EINVAL, "NULL pointer");
    const size_t e = element_size(h.dtype);
    if (misaligned(x, e) || misaligned(w, e) || misaligned(targets, 8) || misaligned(a, 4) || misaligned(b, 4))
        return bad(who, DDP_EALIGN, "a tensor is not aligned to its element type");
    if (!ws && need > 0) return bad(who, DDP_EINVAL, "workspace is NULL");
    if (misaligned(ws, 256)) return bad(who, DDP_EALIGN, "workspace is not 256-byte aligned");
    if (bytes < need) return bad(who, DDP_ESHAPE, "workspace is too small");
    return DDP_OK;
}

// f(Shape) with the tile of a cut
template <class T, class F>
void by_tile(bool large, F &&f) {
    if (large)
        f(Large<T>{});
    else
        f(Small<T>{});
}

// Logits [splits][tokens][words] of each split of hidden.
template <class T>
GradArgs split_logits(const Operand &w, const Operand &x, int64_t words, int64_t tokens, int64_t steps, const Cut &cut, char *to, hipStream_t st) {
    typedef Small<T> S;
    GradArgs g{};
    g.a = w, g.b = x, g.rows_m = words, g.rows_n = tokens, g.steps = steps, g.splits = cut.splits, g.first = 1;
    g.acc = reinterpret_cast<float *>(to), g.mt = cdiv(words, S::TM), g.nt = cdiv(tokens, S::TN);
    hipLaunchKernelGGL((grad_kernel<S, false, false>), dim3((unsigned)(g.mt * g.nt), (unsigned)g.splits), dim3(S::THREADS), 0, st, g);
    return g;
}

// Logits of few tokens, in splits.
GradArgs few_logits(const ddp_head &h, FewArgs &f, char *to, hipStream_t st) {
    GradArgs g{};
    f.splits = g.splits = few_logit_splits(h);
    f.out = g.acc = reinterpret_cast<float *>(to);
    g.rows_m = h.vocab, g.rows_n = h.tokens;
    const dim3 grid((unsigned)cdiv(h.vocab, 64), (unsigned)f.splits);
    if (h.tokens <= 32)
        hipLaunchKernelGGL((few_logits_kernel<1>), grid, dim3(256), 0, st, f);
    else
        hipLaunchKernelGGL((few_logits_kernel<2>), grid, dim3(256), 0, st, f);
    return g;
}
FewArgs few_args(const ddp_head &h, const void *x, const void *w) {
    FewArgs f{};
    f.x = static_cast<const float *>(x), f.w = static_cast<const float *>(w);
    f.x_stride = h.tokens > 1 ? h.x_stride : 0, f.w_stride = h.vocab > 1 ? h.w_stride : 0;
    f.tokens = (int)h.tokens, f.words = (int)h.vocab, f.hidden = (int)h.hidden;
    return f;
}
int few_forward(const ddp_head &h, const void *x, const void *w, const int64_t *targets, float *loss, float *lse, char *ws, hipStream_t st) {
    const Layout l = layout_of(h, false, x, w);
    FewArgs f = few_args(h, x, w);
    const GradArgs g = few_logits(h, f, ws + l.logits, st);
    LogitArgs a{};
    a.tokens = h.tokens, a.vocab = h.vocab, a.targets = targets, a.mt = cdiv(h.vocab, kSplitWords);
    a.part = reinterpret_cast<float2 *>(ws + l.part), a.picked = reinterpret_cast<float *>(ws + l.picked);
    hipLaunchKernelGGL(split_logits_kernel, dim3((unsigned)a.mt, (unsigned)h.tokens), dim3(256), 0, st, a, g);
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)cdiv(h.tokens, 16)), dim3(256), 0, st, a.part, a.mt, h.tokens, h.vocab, targets, a.picked, loss, lse);
    return launched("ddp_cross_entropy_forward");
}
int few_backward(const ddp_head &h, const float *dloss, const void *x, const void *w, const int64_t *targets, const float *lse, void *dx, void *dw, char *ws,
                 hipStream_t st) {
    const Layout l = layout_of(h, true, x, w);
    FewArgs f = few_args(h, x, w);
    const GradArgs z = few_logits(h, f, ws + l.logits, st);
    LogitArgs a{};
    a.tokens = h.tokens, a.vocab = h.vocab, a.targets = targets, a.lse = lse, a.dloss = dloss, a.dz = ws + l.dz, a.piece = l.piece;
    hipLaunchKernelGGL((split_dlogits_kernel<float>), dim3((unsigned)cdiv(l.piece, kSplitWords), (unsigned)h.tokens), dim3(256), 0, st, a, z);
    f.dz = reinterpret_cast<const float *>(ws + l.dz), f.dz_stride = l.piece;
    if (dx) {
        GradArgs g{};
        f.splits = g.splits = few_dx_splits(h);
        f.out = g.acc = reinterpret_cast<float *>(ws + l.acc);
        const dim3 grid((unsigned)cdiv(h.hidden, 128), (unsigned)f.splits);
        if (h.tokens <= 32)
            hipLaunchKernelGGL((few_dx_kernel<1>), grid, dim3(256), 0, st, f);
        else
            hipLaunchKernelGGL((few_dx_kernel<2>), grid, dim3(256), 0, st, f);
        g.rows_m = h.hidden, g.rows_n = h.tokens, g.out = dx, g.out_stride = h.tokens > 1 ? h.dx_stride : h.hidden;
        hipLaunchKernelGGL((split_join_kernel<Triple>), dim3((unsigned)cdiv(h.tokens * cdiv(h.hidden, 4), 256)), dim3(256), 0, st, g);
    }
    if (dw) {
        f.out = static_cast<float *>(dw), f.out_stride = h.vocab > 1 ? h.dw_stride : h.hidden;
        // (grids' y ends at 65535: 8 M words)
        for (int64_t first = 0; first < h.vocab; first += (int64_t)65535 * 128) {
            FewArgs part = f;
            part.dz += first, part.out += first * f.out_stride, part.words = (int)(h.vocab - first < (int64_t)65535 * 128 ? h.vocab - first : (int64_t)65535 * 128);
            hipLaunchKernelGGL(few_dw_kernel, dim3((unsigned)cdiv(h.hidden, 128), (unsigned)cdiv(part.words, 128)), dim3(256), 0, st, part);
        }
    }
    return launched("ddp_cross_entropy_backward");
}

template <class T>
int forward(const ddp_head &h, const void *x, const void *w, const int64_t *targets, float *loss, float *lse, char *ws, hipStream_t st) {
    const Layout l = layout_of(h, false, x, w);
    LogitArgs a{};
    a.x = operand<T>(h, l, true, x, ws, st);
    a.w = operand<T>(h, l, false, w, ws, st);
    a.tokens = h.tokens, a.vocab = h.vocab, a.steps = l.padded / BK * (kTriple<T> ? kProducts : 1), a.targets = targets;
    a.part = reinterpret_cast<float2 *>(ws + l.part);
    a.picked = reinterpret_cast<float *>(ws + l.picked);
    const Cut cut = logit_cut(h.vocab, h.tokens, a.steps);
    if (cut.splits > 1) {
        const GradArgs g = split_logits<T>(a.w, a.x, h.vocab, h.tokens, a.steps, cut, ws + l.logits, st);
        a.mt = cdiv(h.vocab, kSplitWords);
        hipLaunchKernelGGL(split_logits_kernel, dim3((unsigned)a.mt, (unsigned)h.tokens), dim3(256), 0, st, a, g);
    } else {
        by_tile<T>(cut.large, [&](auto s) {
            typedef decltype(s) S;
            a.mt = cdiv(h.vocab, S::TM), a.nt = cdiv(h.tokens, S::TN);
            hipLaunchKernelGGL((logits_kernel<S>), dim3((unsigned)(a.mt * a.nt)), dim3(S::THREADS), 0, st, a);
        });
    }
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)cdiv(h.tokens, 16)), dim3(256), 0, st, a.part, a.mt, h.tokens, h.vocab, targets, a.picked, loss, lse);
    return launched("ddp_cross_entropy_forward");
}

// One gradient's product over a piece; `first`: its sums start here, `last`: they end here.
template <class T, bool BKMAJ>
void gradient(GradArgs &g, bool first, bool last, const Cut &cut, hipStream_t st) {
    g.splits = cut.splits, g.first = first, g.last = last && cut.splits == 1;
    by_tile<T>(cut.large, [&](auto s) {
        typedef decltype(s) S;
        g.mt = cdiv(g.rows_m, S::TM), g.nt = cdiv(g.rows_n, S::TN);
        hipLaunchKernelGGL((grad_kernel<S, true, BKMAJ>), dim3((unsigned)(g.mt * g.nt), (unsigned)g.splits), dim3(S::THREADS), 0, st, g);
    });
    if (!last || cut.splits == 1) return;
    const int64_t n = cdiv(g.rows_n * cdiv(g.rows_m, 4), 256);
    hipLaunchKernelGGL((split_join_kernel<T>), dim3((unsigned)(n < (1 << 20) ? n : 1 << 20)), dim3(256), 0, st, g);
}

template <class T>
int backward(const ddp_head &h, const float *dloss, const void *x, const void *w, const int64_t *targets, const float *lse, void *dx, void *dw, char *ws,
             hipStream_t st) {
    const Layout l = layout_of(h, true, x, w);
    const Operand ox = operand<T>(h, l, true, x, ws, st), ow = operand<T>(h, l, false, w, ws, st);
    constexpr int STEP = BK, PRODUCTS = kTriple<T> ? kProducts : 1;
    bf16 *dz = reinterpret_cast<bf16 *>(ws + l.dz);
    float *most = reinterpret_cast<float *>(ws + l.most);
    hipLaunchKernelGGL(most_kernel, dim3(1), dim3(1024), 0, st, dloss, targets, h.tokens, h.vocab, most);
    // (cuts by the longest piece, so that every piece's sums lie alike)
    const Cut of_x = cut_of(h.hidden, h.tokens, l.piece / STEP * PRODUCTS, true), of_w = cut_of(h.hidden, l.piece, l.token_rows / STEP * PRODUCTS, true);
    const Cut of_logits = logit_cut(l.piece, l.token_rows, l.padded / STEP * PRODUCTS);
    for (int64_t i = 0; i < l.pieces; ++i) {
        const int64_t v0 = i * l.piece, words = h.vocab - v0 < l.piece ? h.vocab - v0 : l.piece;
        // (a last piece that is shorter has dz rows that are)
        const int64_t width = up(words, 256);
        const Operand piece{static_cast<const bf16 *>(ow.p) + v0 * ow.stride, ow.stride, words, ow.groups, ow.plane};
        const int64_t dz_plane = l.token_rows * width;
        LogitArgs a{};
        a.x = ox, a.w = piece, a.tokens = h.tokens, a.vocab = h.vocab, a.steps = l.padded / STEP * PRODUCTS, a.v0 = v0, a.targets = targets, a.lse = lse, a.dloss = dloss, a.most = most;
        a.dz = dz, a.piece = width, a.token_rows = l.token_rows;
        if (of_logits.splits > 1) {  // (then there is one piece)
            const GradArgs z = split_logits<T>(piece, ox, words, h.tokens, a.steps, of_logits, ws + l.logits, st);
            hipLaunchKernelGGL((split_dlogits_kernel<T>), dim3((unsigned)cdiv(width, kSplitWords), (unsigned)l.token_rows), dim3(256), 0, st, a, z);
        } else {
            by_tile<T>(logit_cut(width, l.token_rows, a.steps).large, [&](auto s) {
                typedef decltype(s) S;
                a.mt = cdiv(width, S::TM), a.nt = cdiv(l.token_rows, S::TN);
                hipLaunchKernelGGL((dlogits_kernel<S>), dim3((unsigned)(a.mt * a.nt)), dim3(S::THREADS), 0, st, a);
            });
        }
        GradArgs g{};
        g.rows_m = h.hidden, g.most = most;
        if (dx) {
            g.a = piece, g.b = Operand{dz, width, h.tokens, width / 8, dz_plane}, g.rows_n = h.tokens, g.steps = width / STEP * PRODUCTS;
            g.out = dx, g.out_stride = h.tokens > 1 ? h.dx_stride : h.hidden, g.acc = reinterpret_cast<float *>(ws + l.acc);
            gradient<T, false>(g, i == 0, i == l.pieces - 1, of_x, st);
        }
        if (dw) {
            const int64_t dw_stride = h.vocab > 1 ? h.dw_stride : h.hidden;
            g.a = ox, g.b = Operand{dz, width, l.token_rows, width / 8, dz_plane}, g.rows_n = words, g.steps = l.token_rows / STEP * PRODUCTS;
            g.out = static_cast<Out<T> *>(dw) + v0 * dw_stride, g.out_stride = dw_stride, g.acc = reinterpret_cast<float *>(ws + l.acc_w);
            gradient<T, true>(g, true, true, of_w, st);
        }
    }
    return launched("ddp_cross_entropy_backward");
}

}  // namespace
}  // namespace ddp

extern "C" int64_t ddp_cross_entropy_forward_workspace(const ddp_head *head, const void *x, const void *weight) {
    using namespace ddp;
    if (int rc = guarded(nullptr, [&]() -> int { return check_head("ddp_cross_entropy_forward_workspace", head); })) return -rc;
    return head->tokens ? layout_of(*head, false, x, weight).bytes : 0;
}

extern "C" int ddp_cross_entropy_forward(const ddp_head *head, const void *x, const void *weight, const int64_t *targets, float *loss, float *lse, void *workspace,
                                         int64_t workspace_bytes, void *stream) {
    using namespace ddp;
    return guarded(nullptr, [&]() -> int {
        const char *who = "ddp_cross_entropy_forward";
        if (int rc = check_head(who, head)) return rc;
        const ddp_head &h = *head;
        if (h.tokens == 0) return DDP_OK;
        if (int rc = check_call(who, h, x, weight, targets, loss, lse, workspace, workspace_bytes, layout_of(h, false, x, weight).bytes)) return rc;
        char *ws = static_cast<char *>(workspace);
        const hipStream_t st = static_cast<hipStream_t>(stream);
        if (is_few(h)) return few_forward(h, x, weight, targets, loss, lse, ws, st);
        return h.dtype == DDP_BF16 ? forward<bf16>(h, x, weight, targets, loss, lse, ws, st) : forward<Triple>(h, x, weight, targets, loss, lse, ws, st);
    });
}

extern "C" int64_t ddp_cross_entropy_backward_workspace(const ddp_head *head, const void *x, const void *weight) {
    using namespace ddp;
    if (int rc = guarded(nullptr, [&]() -> int { return check_head("ddp_cross_entropy_backward_workspace", head); })) return -rc;
    return head->tokens ? layout_of(*head, true, x, weight).bytes : 0;
}

extern "C" int ddp_cross_entropy_backward(const ddp_head *head, const float *dloss, const void *x, const void *weight, const int64_t *targets, const float *lse,
                                          void *dx, void *dweight, void *workspace, int64_t workspace_bytes, void *stream) {
    using namespace ddp;
    return guarded(nullptr, [&]() -> int {
        const char *who = "ddp_cross_entropy_backward";
        if (int rc = check_head(who, head)) return rc;
        const ddp_head &h = *head;
        if (dx && h.tokens > 1 && (h.dx_stride < h.hidden || reach(h.tokens, h.dx_stride) < 0)) return bad(who, DDP_EINVAL, "dx_stride is smaller than hidden or too large");
        if (dweight && h.vocab > 1 && (h.dw_stride < h.hidden || reach(h.vocab, h.dw_stride) < 0)) return bad(who, DDP_EINVAL, "dw_stride is smaller than hidden or too large");
        const size_t e = element_size(h.dtype);
        if (misaligned(dx, e) || misaligned(dweight, e)) return bad(who, DDP_EALIGN, "a gradient is not aligned to its element type");
        const hipStream_t st = static_cast<hipStream_t>(stream);
        if (h.tokens == 0) {  // no token: the weight's gradient is zero
            if (!dweight) return DDP_OK;
            const int64_t stride = h.vocab > 1 ? h.dw_stride : h.hidden, n = cdiv(h.vocab * cdiv(h.hidden, 4), 256);
            const dim3 grid((unsigned)(n < (1 << 20) ? n : 1 << 20));
            if (h.dtype == DDP_BF16)
                hipLaunchKernelGGL((zero_rows_kernel<bf16>), grid, dim3(256), 0, st, static_cast<bf16 *>(dweight), stride, h.vocab, h.hidden);
            else
                hipLaunchKernelGGL((zero_rows_kernel<float>), grid, dim3(256), 0, st, static_cast<float *>(dweight), stride, h.vocab, h.hidden);
            return launched(who);
        }
        if (int rc = check_call(who, h, x, weight, targets, dloss, lse, workspace, workspace_bytes, layout_of(h, true, x, weight).bytes)) return rc;
        char *ws = static_cast<char *>(workspace);
        if (is_few(h)) return few_backward(h, dloss, x, weight, targets, lse, dx, dweight, ws, st);
        return h.dtype == DDP_BF16 ? backward<bf16>(h, dloss, x, weight, targets, lse, dx, dweight, ws, st) : backward<Triple>(h, dloss, x, weight, targets, lse, dx, dweight, ws, st);
    });
}
