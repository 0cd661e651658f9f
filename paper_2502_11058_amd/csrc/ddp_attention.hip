// Attention, forward and backward, on the 32x32 matrix instructions.
//
// No product's result passes through LDS on its way to the next product: an accumulator has a column per lane and rows in registers,
// an operand has a row or column per lane and k in registers, so with the scores' k of the second product in registers the
// first product's accumulator is the second's operand as it stands (acc_operand).  So the forward pass and dq form the scores
// with a query per lane, s^T = K Q^T, where a query's maximum, sum and factors are one value a lane, and dk and dv form them with a
// key per lane, s = Q K^T.  What is read down the rows of a tile (V in o = p V, K in dq, Q and dO in dk and dv) is read by the
// transposing LDS load.
//
// The backward pass is two kernels: one owns 128 queries and goes over the keys for dq, one owns 128 keys and goes over the queries for dk
// and dv.  It forms s and dO V^T twice, seven products in place of five, but no gradient is added up in memory by whoever comes first: results
// do not depend on any order, and where nothing is split no fp32 copy of a gradient is needed.
//
// What bounds it, 8192 causal tokens, 32 heads of 128 over 8, bf16: the matrix cores and the exponentials' vector instructions by turns, at the
// 1.6 GHz that their power leaves (forward: matrix cores busy 57 % of the time, vector units 59 %, .57 to .64 ms, .86 to .97 Pflop/s; dq 60 and
// 56 %, 1.06 ms; dk and dv 53 and 40 %, 1.27 ms).  Tiles of 64 keys (32 in fp32, three planes) are what two pairs of buffers, the next pair on its way while one
// is worked on, leave room for beside a second workgroup.
//
// In bf16 the second products' operands, p and ds, are rounded to bf16, which is what the matrix instruction for bf16 takes: planes of them as
// for fp32 would be three times the products.  Results are up to 1.4 times as far from 64 bits for it as their own rounding makes them.
// dO . O of the rounded O is off by as much as a rounding of ds, in every ds of a row alike.  The rows' ds have to sum to zero; what
// they sum to in the dq kernel is that error, and the dk and dv kernel, which runs behind it, has dO . O without.  dq's own ds are
// multiplied with their rounding's remainder too: an eighth product.  Errors of dq and dk against 64 bits, 6001 tokens in 11 documents:
// 2.6e-3 without both, 2.0e-3 and 2.3e-3 with them; 1.7e-3 is the result's own rounding.
#include "ddp_operators.h"

#include <initializer_list>

namespace ddp {
namespace {

constexpr int kRows = 128;  // queries (or keys) of a workgroup, 32 a wavefront

// Wavefronts per SIMD that each kernel's registers leave room for: two wherever 256 registers a lane hold operands and accumulators.
template <class T, int DP>
constexpr int kForwardWaves = !kTriple<T> || DP == 64 ? 2 : 1;
template <class T, int DP>
constexpr int kDqWaves = !kTriple<T> || DP == 64 ? 2 : 1;
template <class T, int DP>
constexpr bool kWideDkdv = !kTriple<T> && DP == 128;
template <class T, int DP>
constexpr int kDkdvThreads = kWideDkdv<T, DP> ? 512 : 256;
template <class T, int DP>
constexpr int kDkdvWaves = kTriple<T> ? 1 : 2;

struct View {
    char *p;
    int64_t batch, token, head;  // strides in elements
    int64_t plane;               // likewise, of an operand's planes
};
struct AttentionArgs {
    View q, k, v, d_o;           // operands: planes of bf16 in 16-byte groups, the caller's tensors or copies of them
    View o;                      // as the caller has it
    View dq, dk, dv;
    const int32_t *cu_q, *cu_k;
    float *lse;            // of the forward pass
    const float *lse_in;   // natural
    float *lse2, *delta;   // workspace: lse * log2 e (0 where there is none), do . o
    float *sums;           // workspace of the portions: o or dq [portions][query rows][q_heads][dim], or dk and dv [portions][2][key rows][k_heads][dim]
    float2 *stats;         // likewise: [portions][query rows x q_heads], what o is relative to and its sum, or the sum of ds
    int portions;          // that a workgroup's tiles are split into
    int64_t q_tokens, k_tokens;
    int q_heads, k_heads, dim, batch;
    float scale;
    int causal;
    int blocks;      // blocks of kRows rows of one head in the call
    unsigned first;  // workgroup of the call that is this launch's first
};

// One sequence's rows.
struct Sequence {
    int b;
    int64_t q0, k0;  // first row, counted in the packed tensor or in the sequence
    int q_len, k_len;
    int block;       // which kRows of it this workgroup has
};

__device__ __forceinline__ int64_t bounded(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }

// Rows of sequence b, the first one's from 0 on.  b = batch: what lies behind the last one, queries without keys, or keys without queries.
template <bool KEYS>
__device__ __forceinline__ void bounds(const AttentionArgs &a, int b, int64_t &q0, int64_t &q1, int64_t &k0, int64_t &k1) {
    q0 = b ? bounded(a.cu_q[b], 0, a.q_tokens) : 0;
    k0 = b ? bounded(a.cu_k[b], 0, a.k_tokens) : 0;
    if (b < a.batch) {
        q1 = bounded(a.cu_q[b + 1], q0, a.q_tokens);
        k1 = bounded(a.cu_k[b + 1], k0, a.k_tokens);
    } else {
        q1 = KEYS ? q0 : a.q_tokens;
        k1 = KEYS ? a.k_tokens : k0;
    }
}

// The sequence that block `block` belongs to, counted over the sequences' blocks of kRows queries (keys); false beyond the last.  The
// wavefront looks at 64 sequences at a time.
template <bool KEYS>
__device__ __forceinline__ bool find_sequence(const AttentionArgs &a, int block, Sequence &s) {
    if (!a.cu_q) {
        // (one block of each sequence after the other, so that causal attention's long ones of all sequences come first)
        s.block = block / a.batch;
        s.b = block - s.block * a.batch;
        s.q0 = s.k0 = 0;
        s.q_len = (int)a.q_tokens;
        s.k_len = (int)a.k_tokens;
        return true;
    }
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int b0 = 0; b0 <= a.batch; b0 += 64) {
        const int b = b0 + lane;
        int64_t q0 = 0, q1 = 0, k0 = 0, k1 = 0;
        if (b <= a.batch) bounds<KEYS>(a, b, q0, q1, k0, k1);
        const int mine = (int)(((KEYS ? k1 - k0 : q1 - q0) + kRows - 1) / kRows);
        int sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(sum, d);
            if (lane >= d) sum += up;
        }
        const unsigned long long hit = __ballot(before + sum > block);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            s.b = b0 + l;
            s.block = uniform(block - before - (__shfl(sum, l) - __shfl(mine, l)));
            bounds<KEYS>(a, s.b, q0, q1, k0, k1);
            s.q0 = uniform((int)q0), s.k0 = uniform((int)k0), s.q_len = uniform((int)(q1 - q0)), s.k_len = uniform((int)(k1 - k0));
            return true;
        }
        before += __shfl(sum, 63);
    }
    return false;
}

template <class T>
__device__ __forceinline__ T *row_of(const View &v, const Sequence &s, bool packed, int64_t first, int head) {
    return reinterpret_cast<T *>(v.p) + (packed ? 0 : s.b * v.batch) + first * v.token + (int64_t)head * v.head;
}

__device__ const u32x4 kZeros = {0u, 0u, 0u, 0u};

// Brings tiles of ROWS rows of DP columns to LDS, zeros from row `rows` and column `dim` on, plane after plane: 16 bytes a lane and load at
// the lane's place in its wavefront's kilobyte, so the tile's exchange of groups is one of the addresses read; what is to be zero is read
// from kZeros.  A tile is there after arrived().
template <class T, int DP, int ROWS, int THREADS = 256>
struct Tiles {
    static constexpr int PER_ROW = DP / 8, EACH = ROWS * PER_ROW / THREADS, ROWB = DP * 2, STEP = THREADS / PER_ROW, PLANE = ROWS * ROWB, BYTES = kPlanes<T> * PLANE;
    unsigned stride;      // bytes
    int row, group, dim;  // of the first of this lane's groups; where the next ones are exchanged differently, it is another one of its row
    int64_t plane;        // bytes
    __device__ __forceinline__ Tiles(const View &v, int dim_) {
        row = threadIdx.x / PER_ROW;
        group = (int)(threadIdx.x % PER_ROW) ^ swizzle<ROWB>(row);
        dim = dim_;
        stride = (unsigned)(v.token * 2);
        plane = v.plane * 2;
    }
    __device__ __forceinline__ void start(const bf16 *base, int rows, char *tile) const {
        const bool whole = rows >= ROWS && dim == DP;
#pragma unroll
        for (int k = 0; k < kPlanes<T>; ++k) {
            const char *from = reinterpret_cast<const char *>(base) + k * plane;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                DDP_LDS void *to = (DDP_LDS void *)(tile + k * PLANE + (i * THREADS + uniform(threadIdx.x & ~63)) * 16);
                const int g = group ^ swizzle<ROWB>(i * STEP);
                const char *x = from + ((unsigned)(row + i * STEP) * stride + (unsigned)g * 16);
                if (!whole && !(g * 8 < dim && row + i * STEP < rows)) x = reinterpret_cast<const char *>(&kZeros);
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)x, to, 16, 0, 0);
            }
        }
    }
};
// an operand from such a tile, by rows or by columns
template <class T, int ROWB, int PLANE>
__device__ __forceinline__ Operand8<T> of_row(const char *tile, int row, int group) {
    Operand8<T> v;
#pragma unroll
    for (int k = 0; k < kPlanes<T>; ++k) v.p[k] = tile_row<ROWB>(tile + k * PLANE, row, group);
    return v;
}
template <class T, int ROWB, int PLANE>
__device__ __forceinline__ Operand8<T> of_col(const char *tile, int k0, int col0, int lane) {
    Operand8<T> v;
#pragma unroll
    for (int k = 0; k < kPlanes<T>; ++k) v.p[k] = tile_col<ROWB>(tile + k * PLANE, k0, col0, lane);
    return v;
}
__device__ __forceinline__ void arrived() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// The two phases of a tile, their operands read one step before the products that take them.
// z[j] += rows of tile[j] (32 from row0 on) times operand(j, i), over the head's channels.
template <class T, int ROWB, int PLANE, int KS, int NZ, class B>
__device__ __forceinline__ void score(f32x16 (&z)[NZ], const char *const (&tile)[NZ], const int (&row0)[NZ], B &&operand) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    Operand8<T> a[2][NZ], b[2][NZ];
    auto read = [&](int i) {
#pragma unroll
        for (int j = 0; j < NZ; ++j) {
            a[i & 1][j] = of_row<T, ROWB, PLANE>(tile[j], row0[j] + (lane & 31), 2 * i + half);
            b[i & 1][j] = operand(j, i);
        }
    };
    read(0);
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        if (i + 1 < KS) read(i + 1);
#pragma unroll
        for (int j = 0; j < NZ; ++j) mma<T>(z[j], a[i & 1][j], b[i & 1][j]);
        __builtin_amdgcn_sched_barrier(0x416);  // products and LDS reads stay where they are; other instructions may move
    }
}
// out[j][d] += columns of tile[j] (rows from row0 on, 32 of them) times x[j], a score tile of those rows; with TWICE, what rounding x to bf16
// leaves over is rounded and multiplied too.
template <class T, int ROWB, int PLANE, int DS, int NZ, bool TWICE = false>
__device__ __forceinline__ void gather(f32x16 (*const (&out)[NZ])[DS], const char *const (&tile)[NZ], int row0, const f32x16 (&x)[NZ]) {
    constexpr int STEPS = 2 * DS;
    const int lane = threadIdx.x & 63;
    Operand8<T> a[2][NZ], p[NZ], rest[NZ];
    auto read = [&](int i) {
#pragma unroll
        for (int j = 0; j < NZ; ++j) a[i & 1][j] = of_col<T, ROWB, PLANE>(tile[j], row0 + i / DS * 16, i % DS * 32, lane);
    };
    read(0);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        if (i + 1 < STEPS) read(i + 1);
#pragma unroll
        for (int j = 0; j < NZ; ++j) {
            if (i % DS == 0) {
                p[j] = acc_operand<T>(x[j], i / DS);
                if constexpr (TWICE)
#pragma unroll
                    for (int e = 0; e < 8; ++e) rest[j].p[0][e] = (bf16)(x[j][i / DS * 8 + e] - (float)p[j].p[0][e]);
            }
            mma<T>((*out[j])[i % DS], a[i & 1][j], p[j]);
            if constexpr (TWICE) mma<T>((*out[j])[i % DS], a[i & 1][j], rest[j]);
        }
        __builtin_amdgcn_sched_barrier(0x416);
    }
}
template <class T, int ROWB, int PLANE, int KS, int NS>
__device__ __forceinline__ void scores_of(f32x16 (&z)[NS], const char *tile, int first, const Operand8<T> (&q)[KS]) {
    const char *tiles[NS];
    int row0[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
        tiles[n] = tile;
        row0[n] = first + 32 * n;
    }
    score<T, ROWB, PLANE, KS, NS>(z, tiles, row0, [&](int, int i) { return q[i]; });
}

// Tile after tile through two pairs of buffers: while body(t, first, second) works on one pair, start(t, first, second) brings the next.
template <class Start, class Body>
__device__ __forceinline__ void in_turn(int tiles, char *a0, char *b0, char *a1, char *b1, Start &&start, Body &&body) {
    if (tiles <= 0) return;
    start(0, a0, b0);
    int t = 0;
    for (; t + 2 <= tiles; t += 2) {
        arrived();
        start(t + 1, a1, b1);
        body(t, a0, b0);
        arrived();
        start(t + 2 < tiles ? t + 2 : tiles - 1, a0, b0);  // (behind the last one: read again, and not used)
        body(t + 1, a1, b1);
    }
    arrived();
    if (t < tiles) body(t, a0, b0);
}

// A portion's tiles.
struct Range {
    int first, n;
};
__device__ __forceinline__ Range range_of(int tiles, int portion, int portions) {
    if (portions == 1) return {0, tiles};
    const int first = (int)((int64_t)tiles * portion / portions);
    return {first, (int)((int64_t)tiles * (portion + 1) / portions) - first};
}

// One row's groups for the operands that stay in registers: lane l has row l % 32 and the groups 2 i + l / 32.
template <class T, int KS>
__device__ __forceinline__ void row_operand(Operand8<T> (&v)[KS], const bf16 *row, int64_t plane, bool valid, int dim) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        const int c = (2 * i + half) * 8;
#pragma unroll
        for (int k = 0; k < kPlanes<T>; ++k) {
            v[i].p[k] = bf16x8{};
            if (valid && c < dim) v[i].p[k] = *reinterpret_cast<const bf16x8 *>(row + k * plane + c);
        }
    }
}

// A lane's row of a result.
template <class T, int DS>
__device__ __forceinline__ void store_row(T *out, const f32x16 (&x)[DS], float factor, int dim) {
#pragma unroll
    for (int d = 0; d < DS; ++d)
        if (d * 32 < dim) store_acc(out + d * 32, x[d], factor, dim - d * 32 < 32 ? dim - d * 32 : 32);
}

template <class T>
constexpr int kTile = kTriple<T> ? 32 : 64;  // rows of a tile in LDS, that a wavefront goes over
// Wavefronts that the forward and the dq kernel give the same 32 queries, each a part of a tile's keys; they add up at the end.  fp32's
// chains of six products leave a SIMD's matrix core idle with one wavefront, and a few hundred workgroups are one a compute unit: 4 x 1024
// tokens, 12 heads of 64, forward 73 and dq (its products alone) 91 us with one part, 59 and 79 with two.  (128 channels: two parts' tiles exceed LDS.)
template <class T, int DP>
constexpr int kParts = kTriple<T> && DP == 64 ? 2 : 1;

// A second part's sums, a value a lane and register, to the first part's wavefront of the same rows.
template <class F, int N>
__device__ __forceinline__ void meet_parts(char *lds, int group, int part, F &&join, f32x16 (&x)[N]) {
    const int lane = threadIdx.x & 63;
    f32x4 *meet = reinterpret_cast<f32x4 *>(lds) + group * 4 * 64 + lane;
#pragma unroll
    for (int d = 0; d < N; ++d) {
        __syncthreads();
        if (part == 1)
#pragma unroll
            for (int r = 0; r < 4; ++r) meet[r * 64] = f32x4{x[d][4 * r], x[d][4 * r + 1], x[d][4 * r + 2], x[d][4 * r + 3]};
        __syncthreads();
        if (part == 0)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const f32x4 v = meet[r * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[d][4 * r + e] = join(x[d][4 * r + e], v[e]);
            }
    }
}

// What a workgroup's 128 queries, and a lane's one, see of the keys.
struct Sight {
    int keys;    // of the workgroup's tiles
    int last;    // this query's last key
    int most;    // this wavefront's
    int edge;    // keys beyond it may be hidden from queries of this wavefront
};
__device__ __forceinline__ Sight sight_of(const AttentionArgs &a, const Sequence &s, int wave, int row) {
    Sight v{s.k_len, s.k_len - 1, s.k_len - 1, s.k_len - 1};
    if (a.causal) {
        const int shift = s.k_len - s.q_len, end = s.block * kRows + kRows - 1, most = end < s.q_len - 1 ? end : s.q_len - 1;
        v.last = row + shift;
        v.edge = s.block * kRows + wave * 32 + shift;
        v.most = v.edge + 31;
        if (most + shift + 1 < v.keys) v.keys = most + shift + 1;
    }
    return v;
}

// Maxima are followed with this much slack, in powers of two: o and its sum are only scaled down when a query's maximum has grown by more,
// which after the first tiles is seldom; what the exponentials are relative to cancels in o / total and lse.
constexpr float kSlack = 8.0f;

// One pass over the keys with the running maximum and sum.  Queries stay in registers, scores and o in accumulators.
template <class T, int DP>
__global__ __launch_bounds__((256 * kParts<T, DP>), (kForwardWaves<T, DP>)) void attention_forward_kernel(const AttentionArgs a) {
    constexpr int PARTS = kParts<T, DP>, OWN = kTile<T>, BN = OWN * PARTS, ROWB = DP * 2, PLANE = BN * ROWB, KS = DP / 16, NS = OWN / 32, DS = DP / 32;
    typedef Tiles<T, DP, BN, 256 * PARTS> Load;
    __shared__ __attribute__((aligned(1024))) char k0_lds[Load::BYTES], v0_lds[Load::BYTES], k1_lds[Load::BYTES], v1_lds[Load::BYTES];
    const unsigned in_call = a.first + blockIdx.x;
    const int head = in_call % a.q_heads, portion = in_call / a.q_heads % a.portions;
    const int order = a.blocks - 1 - in_call / a.q_heads / a.portions;  // the last queries see the most keys: first
    Sequence s;
    if (!find_sequence<false>(a, order, s)) return;
    const bool packed = a.cu_q != nullptr;
    const int kv_head = head / (a.q_heads / a.k_heads);
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5;
    const int group = wave % 4, part = PARTS > 1 ? wave / 4 : 0;  // of the queries, and of a tile's keys
    const int row = s.block * kRows + group * 32 + (lane & 31);
    const bool mine = row < s.q_len;
    const bf16 *k = row_of<const bf16>(a.k, s, packed, s.k0, kv_head), *v = row_of<const bf16>(a.v, s, packed, s.k0, kv_head);
    Operand8<T> q[KS];
    row_operand(q, row_of<const bf16>(a.q, s, packed, s.q0 + (mine ? row : 0), head), a.q.plane, mine, a.dim);
    const Sight sight = sight_of(a, s, group, row);

    f32x16 o[DS] = {};
    float base = -kInf, total = 0.0f;  // what the exponentials are relative to
    // Scores are scaled within the exponential, so the factor has to be positive for -inf to stay what it is: a negative scale turns the queries
    // round, and a scale of zero is the smallest one.
    const float scale2 = a.scale == 0.0f ? 1.17549435e-38f : fabsf(a.scale) * kLog2e;
    if (a.scale < 0.0f)
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int k = 0; k < kPlanes<T>; ++k) q[i].p[k] = -q[i].p[k];
    const Load of_k(a.k, a.dim), of_v(a.v, a.dim);
    const Range tiles = range_of(sight.keys > 0 ? (sight.keys + BN - 1) / BN : 0, portion, a.portions);
    in_turn(tiles.n, k0_lds, v0_lds, k1_lds, v1_lds,
        [&](int t, char *kt, char *vt) {
            t += tiles.first;
            of_k.start(k + (int64_t)t * BN * a.k.token, s.k_len - t * BN, kt);
            of_v.start(v + (int64_t)t * BN * a.v.token, s.k_len - t * BN, vt);
        },
        [&](int t, const char *kt, const char *vt) {
            const int key0 = (tiles.first + t) * BN + part * OWN;
            if (key0 > sight.most) return;
            f32x16 z[NS] = {};
            scores_of<T, ROWB, PLANE, KS, NS>(z, kt, part * OWN, q);
            if (key0 + OWN - 1 > sight.edge) {
#pragma unroll
                for (int n = 0; n < NS; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int key = key0 + n * 32 + acc_row(half, r);
                        if (key > sight.last || key >= s.k_len) z[n][r] = -kInf;
                    }
            }
            float m = z[0][0];
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) m = fmaxf(m, z[n][r]);
            m = fmaxf(m, other_half(m)) * scale2;
            if (__any(m > base + kSlack || (base == -kInf && m != -kInf))) {
                const float top = fmaxf(base, m);
                const float keep = top == -kInf ? 1.0f : __builtin_amdgcn_exp2f(base - top);  // (0 where there was nothing)
                base = top;
                total *= keep;
#pragma unroll
                for (int d = 0; d < DS; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[d][r] *= keep;
            }
            const float from = base == -kInf ? 0.0f : base;
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    z[n][r] = __builtin_amdgcn_exp2f(z[n][r] * scale2 - from);
                    total += z[n][r];
                }
#pragma unroll
            for (int n = 0; n < NS; ++n) gather<T, ROWB, PLANE, DS, 1>({&o}, {vt}, part * OWN + n * 32, {z[n]});
        });
    total += other_half(total);
    if constexpr (PARTS > 1) {
        float2 *meet = reinterpret_cast<float2 *>(v0_lds) + group * 64 + lane;
        __syncthreads();
        if (part == 1) *meet = float2{base, total};
        __syncthreads();
        const float2 there = *meet;
        const float top = fmaxf(base, there.x);
        // (what is relative to -inf is zero)
        const float keep = base == -kInf ? 1.0f : __builtin_amdgcn_exp2f(base - top), take = there.x == -kInf ? 1.0f : __builtin_amdgcn_exp2f(there.x - top);
        meet_parts(k0_lds, group, part, [&](float u, float v) { return u * keep + v * take; }, o);
        total = total * keep + there.y * take;
        base = top;
    }
    if (!mine || part) return;
    const int64_t at = packed ? (int64_t)head * a.q_tokens + s.q0 + row : ((int64_t)s.b * a.q_heads + head) * a.q_tokens + row;
    if (a.portions > 1) {
        const int64_t rows = (packed ? 1 : a.batch) * a.q_tokens, r = (packed ? s.q0 : s.b * a.q_tokens) + row;
        if (half == 0) a.stats[portion * rows * a.q_heads + at] = float2{base, total};
        store_row<float, DS>(a.sums + ((portion * rows + r) * a.q_heads + head) * a.dim, o, 1.0f, a.dim);
        return;
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    if (half == 0) a.lse[at] = total == 0.0f ? -kInf : base * kLn2 + logf(total);
    store_row<Out<T>, DS>(row_of<Out<T>>(a.o, s, packed, s.q0 + row, head), o, inv, a.dim);
}

// o and lse from the portions' sums and statistics, or dq and do . o from theirs; a thread four channels of a query.
template <class T, bool DQ>
__global__ __launch_bounds__(256) void attention_query_join_kernel(const AttentionArgs a) {
    const int64_t rows = (a.cu_q ? 1 : a.batch) * a.q_tokens, n = rows * a.q_heads;
    const int quads = (a.dim + 3) / 4;
    const View &out = DQ ? a.dq : a.o;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n * quads; i += (int64_t)gridDim.x * 256) {
        const int c = (int)(i % quads) * 4, head = (int)(i / quads % a.q_heads), left = a.dim - c;
        const int64_t row = i / quads / a.q_heads, b = a.cu_q ? 0 : row / a.q_tokens, t = row - b * a.q_tokens, at = (b * a.q_heads + head) * a.q_tokens + t;
        float top = -kInf, total = 0.0f;
        for (int p = 0; p < a.portions; ++p) {
            const float2 stat = a.stats[p * n + at];
            if constexpr (DQ)
                total += stat.x;
            else
                top = fmaxf(top, stat.x);
        }
        f32x4 x = {};
        for (int p = 0; p < a.portions; ++p) {
            const f32x4 v = load_part(a.sums + ((p * rows + row) * a.q_heads + head) * a.dim + c, left);
            if constexpr (DQ) {
                x += v;
            } else {
                const float2 stat = a.stats[p * n + at];
                const float take = stat.x == -kInf ? 1.0f : __builtin_amdgcn_exp2f(stat.x - top);  // (what is relative to -inf is zero)
                x += v * take;
                total += stat.y * take;
            }
        }
        if constexpr (!DQ) x *= total == 0.0f ? 0.0f : 1.0f / total;
        store4(reinterpret_cast<T *>(out.p) + b * out.batch + t * out.token + (int64_t)head * out.head + c, x, left);
        if (c) continue;
        if constexpr (DQ)
            a.delta[at] += total;
        else
            a.lse[at] = total == 0.0f ? -kInf : top * kLn2 + logf(total);
    }
}

// do . o of this lane's row, whose do is an operand; both of a row's lanes get it.
template <class T, int KS>
__device__ __forceinline__ float row_product(const Operand8<T> (&dout)[KS], const Out<T> *o, bool valid, int dim) {
    constexpr int N = Group<Out<T>>::n;
    const int half = (threadIdx.x & 63) >> 5;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
#pragma unroll
        for (int e = 0; e < 8; e += N) {
            const int c = (2 * i + half) * 8 + e;
            if (!valid || c >= dim) continue;
            const Vec<Out<T>> v = load_part(o + c, dim - c);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float d = 0.0f;
#pragma unroll
                for (int k = kPlanes<T> - 1; k >= 0; --k) d += (float)dout[i].p[k][e + j];  // (the planes add up to the value)
                s += (float)v[j] * d;
            }
        }
    }
    return s + other_half(s);
}

// One pass over the keys: p from s and lse, ds = p (dO V^T - dO . O), dq += ds K.  Queries and dO stay in registers; dO . O is formed from them
// first and left for the kernel behind (a kernel of its own took 4 to 26 us).
template <class T, int DP>
__global__ __launch_bounds__((256 * kParts<T, DP>), (kDqWaves<T, DP>)) void attention_dq_kernel(const AttentionArgs a) {
    constexpr int PARTS = kParts<T, DP>, OWN = kTile<T>, BN = OWN * PARTS, ROWB = DP * 2, PLANE = BN * ROWB, KS = DP / 16, NS = OWN / 32, DS = DP / 32;
    typedef Tiles<T, DP, BN, 256 * PARTS> Load;
    __shared__ __attribute__((aligned(1024))) char k0_lds[Load::BYTES], v0_lds[Load::BYTES], k1_lds[Load::BYTES], v1_lds[Load::BYTES];
    const unsigned in_call = a.first + blockIdx.x;
    const int head = in_call % a.q_heads, portion = in_call / a.q_heads % a.portions;
    const int order = a.blocks - 1 - in_call / a.q_heads / a.portions;
    Sequence s;
    if (!find_sequence<false>(a, order, s)) return;
    const bool packed = a.cu_q != nullptr;
    const int kv_head = head / (a.q_heads / a.k_heads);
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5;
    const int group = wave % 4, part = PARTS > 1 ? wave / 4 : 0;  // of the queries, and of a tile's keys
    const int row = s.block * kRows + group * 32 + (lane & 31);
    const bool mine = row < s.q_len;
    const bf16 *k = row_of<const bf16>(a.k, s, packed, s.k0, kv_head), *v = row_of<const bf16>(a.v, s, packed, s.k0, kv_head);
    Operand8<T> q[KS], dout[KS];
    row_operand(q, row_of<const bf16>(a.q, s, packed, s.q0 + (mine ? row : 0), head), a.q.plane, mine, a.dim);
    row_operand(dout, row_of<const bf16>(a.d_o, s, packed, s.q0 + (mine ? row : 0), head), a.d_o.plane, mine, a.dim);
    const float delta = row_product<T, KS>(dout, row_of<const Out<T>>(a.o, s, packed, s.q0 + (mine ? row : 0), head), mine, a.dim);
    const int64_t at = packed ? (int64_t)head * a.q_tokens + s.q0 + row : ((int64_t)s.b * a.q_heads + head) * a.q_tokens + row;
    float lse2 = 0.0f;
    if (mine) {
        const float lse = a.lse_in[at];
        lse2 = lse == -kInf ? 0.0f : lse * kLog2e;
    }
    const Sight sight = sight_of(a, s, group, row);

    f32x16 dq[DS] = {};
    float off = 0.0f;  // sum of ds: what do . o of the rounded o is short of sum of p (do . v)
    const float scale2 = a.scale * kLog2e;
    const Load of_k(a.k, a.dim), of_v(a.v, a.dim);
    const Range tiles = range_of(sight.keys > 0 ? (sight.keys + BN - 1) / BN : 0, portion, a.portions);
    in_turn(tiles.n, k0_lds, v0_lds, k1_lds, v1_lds,
        [&](int t, char *kt, char *vt) {
            t += tiles.first;
            of_k.start(k + (int64_t)t * BN * a.k.token, s.k_len - t * BN, kt);
            of_v.start(v + (int64_t)t * BN * a.v.token, s.k_len - t * BN, vt);
        },
        [&](int t, const char *kt, const char *vt) {
            const int key0 = (tiles.first + t) * BN + part * OWN;
            if (key0 > sight.most) return;
            const bool masked = key0 + OWN - 1 > sight.edge;
            constexpr int HALVES = kTriple<T> || DP == 64 ? NS : 1;
            // (128 channels of bf16 leave no registers for two halves of a tile at once: 1212 us with both unrolled, 39 registers in memory, 1112 so)
#pragma unroll HALVES
            for (int n = 0; n < NS; ++n) {
                f32x16 z[2] = {};  // the scores, and do . v
                score<T, ROWB, PLANE, KS, 2>(z, {kt, vt}, {part * OWN + n * 32, part * OWN + n * 32}, [&](int j, int i) { return j ? dout[i] : q[i]; });
#pragma unroll
                for (int r = 0; r < 16; ++r) z[0][r] = __builtin_amdgcn_exp2f(z[0][r] * scale2 - lse2) * (z[1][r] - delta);
                if (masked) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int key = key0 + n * 32 + acc_row(half, r);
                        if (key > sight.last || key >= s.k_len) z[0][r] = 0.0f;
                    }
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) off += z[0][r];
                gather<T, ROWB, PLANE, DS, 1, !kTriple<T>>({&dq}, {kt}, part * OWN + n * 32, {z[0]});
            }
        });
    off += other_half(off);
    if constexpr (PARTS > 1) {
        float *meet = reinterpret_cast<float *>(v0_lds) + group * 64 + lane;
        __syncthreads();
        if (part == 1) *meet = off;
        __syncthreads();
        off += *meet;
        meet_parts(k0_lds, group, part, [](float u, float v) { return u + v; }, dq);
    }
    if (!mine || part) return;
    if (half == 0 && portion == 0) {
        a.lse2[at] = lse2;
        a.delta[at] = a.portions > 1 ? delta : delta + off;
    }
    if (a.portions > 1) {
        const int64_t rows = (packed ? 1 : a.batch) * a.q_tokens, r = (packed ? s.q0 : s.b * a.q_tokens) + row;
        if (half == 0) a.stats[portion * rows * a.q_heads + at] = float2{off, 0.0f};
        store_row<float, DS>(a.sums + ((portion * rows + r) * a.q_heads + head) * a.dim, dq, a.scale, a.dim);
        return;
    }
    store_row<Out<T>, DS>(row_of<Out<T>>(a.dq, s, packed, s.q0 + row, head), dq, a.scale, a.dim);
}

// One pass over the queries of all heads that share the key head: dv += p^T dO, dk += ds^T Q.
// Keys and values stay in registers, or in LDS where they and both gradients' accumulators leave no room for a second wavefront per SIMD: then
// eight wavefronts share the tiles, two of them the same 32 keys, one for each half of a tile's queries, and add up at the end.
template <class T, int DP>
__global__ __launch_bounds__((kDkdvThreads<T, DP>), (kDkdvWaves<T, DP>)) void attention_dkdv_kernel(const AttentionArgs a) {
    constexpr bool WIDE = kWideDkdv<T, DP>;
    constexpr int BM = kTile<T>, ROWB = DP * 2, PLANE = BM * ROWB, KS = DP / 16, MS = BM / 32 / (WIDE ? 2 : 1), DS = DP / 32, THREADS = kDkdvThreads<T, DP>;
    typedef Tiles<T, DP, BM, THREADS> Load;
    __shared__ __attribute__((aligned(1024))) char q0_lds[Load::BYTES], d0_lds[Load::BYTES], q1_lds[Load::BYTES], d1_lds[Load::BYTES];
    __shared__ __attribute__((aligned(1024))) char k_lds[WIDE ? kRows * ROWB : 16], v_lds[WIDE ? kRows * ROWB : 16];
    __shared__ __attribute__((aligned(256))) float stat0[2 * 64], stat1[2 * 64];  // the tile's lse2 and delta
    const unsigned in_call = a.first + blockIdx.x;
    const int kv_head = in_call % a.k_heads, portion = in_call / a.k_heads % a.portions;
    Sequence s;
    if (!find_sequence<true>(a, in_call / a.k_heads / a.portions, s)) return;
    const bool packed = a.cu_q != nullptr;
    const int share = a.q_heads / a.k_heads, first_head = kv_head * share;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5;
    const int group = wave % 4, part = wave / 4;  // of the keys, and of a tile's queries
    const int key = s.block * kRows + group * 32 + (lane & 31);
    const bool mine = key < s.k_len;
    const bf16 *k_rows = row_of<const bf16>(a.k, s, packed, s.k0, kv_head), *v_rows = row_of<const bf16>(a.v, s, packed, s.k0, kv_head);
    Operand8<T> k[WIDE ? 1 : KS], v[WIDE ? 1 : KS];
    if constexpr (WIDE) {  // (there with the first tile)
        Tiles<T, DP, kRows, THREADS>(a.k, a.dim).start(k_rows + (int64_t)s.block * kRows * a.k.token, s.k_len - s.block * kRows, k_lds);
        Tiles<T, DP, kRows, THREADS>(a.v, a.dim).start(v_rows + (int64_t)s.block * kRows * a.v.token, s.k_len - s.block * kRows, v_lds);
    } else {
        row_operand(k, k_rows + (int64_t)(mine ? key : 0) * a.k.token, a.k.plane, mine, a.dim);
        row_operand(v, v_rows + (int64_t)(mine ? key : 0) * a.v.token, a.v.plane, mine, a.dim);
    }
    const int shift = s.k_len - s.q_len;
    // queries from the first that sees the workgroup's first key, in whole tiles
    int from = a.causal ? s.block * kRows - shift : 0;
    from = from < 0 ? 0 : from / BM * BM;
    const int tiles = s.q_len > from ? (s.q_len - from + BM - 1) / BM : 0;
    const int edge = a.causal ? s.block * kRows + group * 32 + 31 - shift : 0;  // queries from it on see all of this wavefront's keys

    f32x16 dk[DS] = {}, dv[DS] = {};
    const float scale2 = a.scale * kLog2e;
    const Load of_q(a.q, a.dim), of_do(a.d_o, a.dim);
    const Range range = range_of(tiles * share, portion, a.portions);
    int head_of = first_head + (tiles ? range.first / tiles : 0), tile_of = tiles ? range.first % tiles : 0;  // of the tile that is brought next
    int at_tile = tile_of;                                                                                 // of the tile that is worked on
    in_turn(range.n, q0_lds, d0_lds, q1_lds, d1_lds,
        [&](int, char *qt, char *dt) {
            const int q0 = from + tile_of * BM;
            if (wave < 2) {  // (64 values from the tile's first on: the workspace ends as many behind the last query)
                const int64_t at = packed ? (int64_t)head_of * a.q_tokens + s.q0 : ((int64_t)s.b * a.q_heads + head_of) * a.q_tokens;
                float *to = (qt == q0_lds ? stat0 : stat1) + wave * 64;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)((wave ? a.delta : a.lse2) + at + q0 + lane), (DDP_LDS void *)to, 4, 0, 0);
            }
            of_q.start(row_of<const bf16>(a.q, s, packed, s.q0 + q0, head_of), s.q_len - q0, qt);
            of_do.start(row_of<const bf16>(a.d_o, s, packed, s.q0 + q0, head_of), s.q_len - q0, dt);
            if (++tile_of == tiles) {
                if (head_of < first_head + share - 1) ++head_of;  // (behind the last one: read again)
                tile_of = 0;
            }
        },
        [&](int, const char *qt, const char *dt) {
            const int q0 = from + at_tile * BM;
            const float *stat = qt == q0_lds ? stat0 : stat1;
            if (++at_tile == tiles) at_tile = 0;
            if (a.causal && q0 + BM <= edge - 31) return;
            const bool masked = q0 + BM > s.q_len || q0 < edge;
#pragma unroll
            for (int mm = 0; mm < MS; ++mm) {
                const int m = WIDE ? part : mm;
                f32x16 z[2] = {};  // the scores, and do . v
                score<T, ROWB, PLANE, KS, 2>(z, {qt, dt}, {m * 32, m * 32}, [&](int j, int i) {
                    if constexpr (WIDE)
                        return of_row<T, ROWB, 0>(j ? v_lds : k_lds, group * 32 + (lane & 31), 2 * i + half);
                    else
                        return j ? v[i] : k[i];
                });
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const f32x4 l4 = *reinterpret_cast<const f32x4 *>(stat + m * 32 + acc_row(half, r));
                    const f32x4 d4 = *reinterpret_cast<const f32x4 *>(stat + 64 + m * 32 + acc_row(half, r));
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        z[0][r + j] = __builtin_amdgcn_exp2f(z[0][r + j] * scale2 - l4[j]);
                        z[1][r + j] = z[0][r + j] * (z[1][r + j] - d4[j]);
                    }
                }
                if (masked) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int i = q0 + m * 32 + acc_row(half, r);
                        if (i >= s.q_len || (a.causal && key > i + shift)) z[0][r] = z[1][r] = 0.0f;
                    }
                }
                gather<T, ROWB, PLANE, DS, 2>({&dv, &dk}, {dt, qt}, m * 32, z);
            }
        });
    if constexpr (WIDE) {
        static_assert(4 * 64 * 16 * 4 <= sizeof k_lds, "a step's sums fit where the keys were");
        arrived();  // (without a tile, nothing has waited for the keys yet)
        const auto sum = [](float u, float v) { return u + v; };
        meet_parts(k_lds, group, part, sum, dk);
        meet_parts(k_lds, group, part, sum, dv);
    }
    if (!mine || part) return;
    if (a.portions > 1) {
        const int64_t rows = packed ? a.k_tokens : a.batch * a.k_tokens, at = (packed ? s.k0 : s.b * a.k_tokens) + key;
        float *sums = a.sums + ((portion * 2 * rows + at) * a.k_heads + kv_head) * a.dim;
        store_row<float, DS>(sums, dk, a.scale, a.dim);
        store_row<float, DS>(sums + rows * a.k_heads * a.dim, dv, 1.0f, a.dim);
        return;
    }
    store_row<Out<T>, DS>(row_of<Out<T>>(a.dk, s, packed, s.k0 + key, kv_head), dk, a.scale, a.dim);
    store_row<Out<T>, DS>(row_of<Out<T>>(a.dv, s, packed, s.k0 + key, kv_head), dv, 1.0f, a.dim);
}

// dk (y = 0) and dv (y = 1) from the portions' sums, in their order; a thread four channels.
template <class T>
__global__ __launch_bounds__(256) void attention_join_kernel(const AttentionArgs a) {
    const int64_t rows = (a.cu_q ? 1 : a.batch) * a.k_tokens;
    const int quads = (a.dim + 3) / 4;
    const View &out = blockIdx.y ? a.dv : a.dk;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * a.k_heads * quads; i += (int64_t)gridDim.x * 256) {
        const int c = (int)(i % quads) * 4, head = (int)(i / quads % a.k_heads), n = a.dim - c;
        const int64_t row = i / quads / a.k_heads, b = a.cu_q ? 0 : row / a.k_tokens, t = row - b * a.k_tokens;
        f32x4 x = {};
        for (int p = 0; p < a.portions; ++p) x += load_part(a.sums + (((2 * p + blockIdx.y) * rows + row) * a.k_heads + head) * a.dim + c, n);
        store4(reinterpret_cast<T *>(out.p) + b * out.batch + t * out.token + (int64_t)head * out.head + c, x, n);
    }
}

// Tensors as operands: rows of heads of `padded` channels in planes of bf16, zeros behind the last channel.  One tensor a y of the grid.
struct Copies {
    View from[4];
    bf16 *to[4];
    int64_t rows[4], tokens[4];  // in all, and of a sequence (packed: in all)
    int heads[4];
    int dim, padded;
};
template <class T>
__global__ __launch_bounds__(256) void attention_copy_kernel(const Copies c) {
    const int w = blockIdx.y, per = c.padded / 8;
    const int64_t n = c.rows[w] * c.heads[w] * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int at = (int)(i % per) * 8, head = (int)(i / per % c.heads[w]);
        const int64_t row = i / per / c.heads[w], b = row / c.tokens[w], t = row - b * c.tokens[w];
        const Out<T> *x = reinterpret_cast<const Out<T> *>(c.from[w].p) + b * c.from[w].batch + t * c.from[w].token + (int64_t)head * c.from[w].head + at;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; j += Group<Out<T>>::n) {
            const Vec<Out<T>> g = at + j < c.dim ? load_part(x + j, c.dim - at - j) : Vec<Out<T>>{};
#pragma unroll
            for (int e = 0; e < Group<Out<T>>::n; ++e) v[j + e] = (float)g[e];
        }
#pragma unroll
        for (int k = 0; k < kPlanes<T>; ++k) {
            bf16x8 o;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                o[j] = (bf16)v[j];
                if (k + 1 < kPlanes<T>) v[j] = left_over(v[j]);
            }
            *reinterpret_cast<bf16x8 *>(c.to[w] + (k * n + i) * 8) = o;
        }
    }
}

int check_attention(const char *who, const ddp_attention *a) {
    if (!a) return bad(who, DDP_EINVAL, "the shape is NULL");
    if (!typed(a->dtype)) return bad(who, DDP_EINVAL, "dtype must be DDP_F32 or DDP_BF16");
    if (a->q_heads < 1 || a->k_heads < 1 || a->q_heads > 65536 || a->q_heads % a->k_heads) return bad(who, DDP_EINVAL, "q_heads must be a multiple of k_heads, both in [1, 65536]");
    if (a->head_dim < 1 || a->head_dim > 128) return bad(who, DDP_EINVAL, "head_dim must be in [1, 128]");
    if (a->batch < 0) return bad(who, DDP_EINVAL, "batch must not be negative");
    if (a->q_tokens < 0 || a->k_tokens < 0 || a->q_tokens > (1 << 30) || a->k_tokens > (1 << 30)) return bad(who, DDP_EINVAL, "tokens must be in [0, 2^30]");
    if (!std::isfinite(a->scale)) return bad(who, DDP_EINVAL, "scale must be finite");
    if (cdiv(a->q_tokens, 32) * (a->q_heads / a->k_heads) > 0x7fffffff) return bad(who, DDP_EINVAL, "too many queries share a key head");
    const int64_t batch = a->packed ? 1 : a->batch;
    for (const int64_t tokens : {a->q_tokens, a->k_tokens}) {
        const int64_t blocks = a->packed ? tokens / kRows + a->batch + 1 : cdiv(tokens, kRows) * batch;
        if (blocks > 0x7fffffff / a->q_heads || batch * tokens > ((int64_t)0x7fffffff * 16) / a->q_heads) return bad(who, DDP_EINVAL, "too many queries or keys");
    }
    return DDP_OK;
}

int take_view(const char *who, const ddp_attention &a, const ddp_heads *h, bool of_q, View &v) {
    const int64_t tokens = of_q ? a.q_tokens : a.k_tokens;
    if (!h) return bad(who, DDP_EINVAL, "a tensor's description is NULL");
    v = View{static_cast<char *>(h->data), a.packed ? 0 : h->batch, h->token, h->head, 0};
    if (tokens == 0 || (a.batch == 0 && !a.packed)) return DDP_OK;
    if (!h->data) return bad(who, DDP_EINVAL, "a tensor is NULL");
    if (misaligned(h->data, element_size(a.dtype))) return bad(who, DDP_EALIGN, "a tensor is not aligned to its element type");
    if (reach(tokens, h->token) < 0 || reach(of_q ? a.q_heads : a.k_heads, h->head) < 0 || (!a.packed && reach(a.batch, h->batch) < 0))
        return bad(who, DDP_EINVAL, "a stride is negative or too large");
    return DDP_OK;
}

int64_t blocks_of(const ddp_attention &a, bool keys) {
    const int64_t tokens = keys ? a.k_tokens : a.q_tokens;
    return a.packed ? tokens / kRows + a.batch + 1 : cdiv(tokens, kRows) * a.batch;
}

AttentionArgs attention_args(const ddp_attention &a, const int32_t *cu_q, const int32_t *cu_k) {
    AttentionArgs g{};
    g.cu_q = cu_q, g.cu_k = cu_k, g.q_tokens = a.q_tokens, g.k_tokens = a.k_tokens, g.q_heads = a.q_heads, g.k_heads = a.k_heads;
    g.dim = a.head_dim, g.batch = a.batch, g.scale = a.scale, g.causal = a.causal != 0, g.portions = 1;
    return g;
}

// Whether a tensor is an operand as it is: bf16 in 16-byte groups, close enough for a tile's offsets to fit 32 bits.
bool is_operand(const ddp_attention &a, const ddp_heads *h) {
    return h && a.dtype == DDP_BF16 && a.head_dim % 8 == 0 && !misaligned(h->data, 16) && h->token % 8 == 0 && h->head % 8 == 0 && (a.packed || h->batch % 8 == 0) &&
           h->token < ((int64_t)1 << 31) / (kRows * 2);
}
int64_t copy_bytes(const ddp_attention &a, bool of_q) {
    const int64_t rows = (a.packed ? 1 : a.batch) * (of_q ? a.q_tokens : a.k_tokens);
    return up(rows * (of_q ? a.q_heads : a.k_heads) * up(a.head_dim, 8) * (a.dtype == DDP_BF16 ? 2 : 6), 256);
}

// The operands of a call, and what copies of those that are none take of its workspace from `at` on.
struct Source {
    const ddp_heads *h;
    bool of_q;
    View *v;
};
template <int N>
int64_t operand_bytes(const ddp_attention &a, const Source (&from)[N]) {
    int64_t n = 0;
    for (const Source &s : from)
        if (!is_operand(a, s.h)) n += copy_bytes(a, s.of_q);
    return n;
}
template <int N>
void make_operands(const ddp_attention &a, const Source (&from)[N], char *at, hipStream_t st) {
    Copies c{};
    c.dim = a.head_dim, c.padded = (int)up(a.head_dim, 8);
    int n = 0;
    int64_t most = 0;
    for (const Source &s : from) {
        if (is_operand(a, s.h)) continue;
        const int64_t tokens = s.of_q ? a.q_tokens : a.k_tokens, rows = (a.packed ? 1 : a.batch) * tokens;
        const int heads = s.of_q ? a.q_heads : a.k_heads;
        c.from[n] = *s.v, c.to[n] = reinterpret_cast<bf16 *>(at), c.rows[n] = rows, c.tokens[n] = tokens > 0 ? tokens : 1, c.heads[n] = heads;
        *s.v = View{at, tokens * heads * c.padded, (int64_t)heads * c.padded, c.padded, rows * heads * c.padded};
        at += copy_bytes(a, s.of_q);
        const int64_t groups = rows * heads * (c.padded / 8);
        most = groups > most ? groups : most;
        ++n;
    }
    if (n == 0 || most == 0) return;
    const dim3 grid((unsigned)(cdiv(most, 256) < (1 << 20) ? cdiv(most, 256) : 1 << 20), (unsigned)n);
    if (a.dtype == DDP_BF16)
        hipLaunchKernelGGL((attention_copy_kernel<bf16>), grid, dim3(256), 0, st, c);
    else
        hipLaunchKernelGGL((attention_copy_kernel<Triple>), grid, dim3(256), 0, st, c);
}

// f(element, padded head_dim)
template <class F>
void by_form(const ddp_attention &a, F &&f) {
    auto wide = [&](auto t) {
        if (a.head_dim <= 64)
            f(t, std::integral_constant<int, 64>{});
        else
            f(t, std::integral_constant<int, 128>{});
    };
    if (a.dtype == DDP_BF16)
        wide(bf16{});
    else
        wide(Triple{});
}

int check_cu(const char *who, const ddp_attention &a, const int32_t *cu_q, const int32_t *cu_k) {
    if ((cu_q != nullptr) != (a.packed != 0) || (cu_k != nullptr) != (a.packed != 0)) return bad(who, DDP_EINVAL, "packed sequences need cu_q and cu_k, others none");
    if (misaligned(cu_q, 4) || misaligned(cu_k, 4)) return bad(who, DDP_EALIGN, "cu_q or cu_k is not aligned");
    return DDP_OK;
}
int check_workspace(const char *who, const void *workspace, int64_t bytes, int64_t need) {
    if (need == 0) return DDP_OK;
    if (!workspace) return bad(who, DDP_EINVAL, "workspace is NULL");
    if (misaligned(workspace, 256)) return bad(who, DDP_EALIGN, "workspace is not 256-byte aligned");
    return bytes < need ? bad(who, DDP_ESHAPE, "workspace is too small") : DDP_OK;
}

// Few heads and blocks leave compute units without a workgroup and the others with one alone: a workgroup's tiles are then split into portions,
// whose fp32 sums another kernel joins in their order.  `least` tiles take about what that kernel does (5 us), by what a tile took: in bf16 .8 us
// forward and 1.3 for dq up to 64 channels, half as much again beyond, 1.8 for dk and dv; three times that in fp32.  2125 tokens after 849, two
// heads of 32, 34 workgroups: forward 46, dq 67, dk and dv 61 us whole, 21, 26 and 22 with their joins in portions.  6001 tokens in 11 documents,
// 32 heads of 64 over 4, 232 workgroups for dk and dv: 401 us whole, 141 in four.  4 x 1024 tokens, 12 heads of 64 in fp32, 384 workgroups:
// dk and dv 112 us whole, 136 in two.
int portions_of(int64_t workgroups, int64_t tiles, int64_t least) {
    if (workgroups >= 256 || workgroups < 1) return 1;
    const int64_t n = cdiv(768, workgroups), most = tiles / least < 16 ? tiles / least : 16;
    return (int)(n < most ? n : most > 1 ? most : 1);
}
// (of a packed call's sequences, which the host does not know, the mean)
int64_t mean_length(const ddp_attention &a, int64_t tokens) { return a.packed && a.batch > 0 ? cdiv(tokens, a.batch) : tokens; }
int query_portions(const ddp_attention &a) {
    const int least = a.dtype == DDP_F32 ? 2 : a.head_dim > 64 ? 5 : 8;
    return portions_of(blocks_of(a, false) * a.q_heads, cdiv(mean_length(a, a.k_tokens), 64), least);
}
int key_portions(const ddp_attention &a) {
    const int64_t tile = a.dtype == DDP_F32 ? 32 : 64;
    return portions_of(blocks_of(a, true) * a.k_heads, cdiv(mean_length(a, a.q_tokens), tile) * (a.q_heads / a.k_heads), 4);
}
// what query portions take of a workspace: sums and statistics
struct QuerySums {
    int64_t sums, stats, bytes;
    QuerySums(const ddp_attention &a, int n) {
        const int64_t rows = (a.packed ? 1 : a.batch) * a.q_tokens * a.q_heads;
        sums = n > 1 ? up(n * rows * a.head_dim * 4, 256) : 0;
        stats = n > 1 ? up(n * rows * 8, 256) : 0;
        bytes = sums + stats;
    }
};
struct BackwardLayout {
    int64_t lse2, delta, sums, stats, copies, bytes;
    BackwardLayout(const ddp_attention &a, int64_t copied) {
        const int64_t rows = a.packed ? 1 : a.batch;
        const int n = key_portions(a);
        const int64_t stat = a.q_tokens > 0 ? up(rows * a.q_tokens * a.q_heads * 4 + 64 * 4, 256) : 0;  // (and a tile: read, not used)
        const QuerySums of_q(a, query_portions(a));
        const int64_t of_k = n > 1 ? up(2 * n * rows * a.k_tokens * a.k_heads * a.head_dim * 4, 256) : 0;
        lse2 = 0, delta = stat, sums = 2 * stat;  // (dq's are joined before dk's and dv's are there)
        stats = sums + of_q.sums;
        copies = sums + (of_q.bytes > of_k ? of_q.bytes : of_k);
        bytes = copies + copied;
    }
};
// f(workgroups): a call's workgroups in as many launches as grids have room for them.
template <class F>
void in_launches(AttentionArgs &a, int heads, int threads, F &&f) {
    const int64_t all = (int64_t)a.blocks * heads * a.portions, most = most_groups(threads);
    for (int64_t at = 0; at < all; at += most) {
        a.first = (unsigned)at;
        f(dim3((unsigned)(all - at < most ? all - at : most)));
    }
}
template <class T, bool DQ>
void join_queries(const ddp_attention &at, const AttentionArgs &a, hipStream_t st) {
    const int64_t n = cdiv((at.packed ? 1 : at.batch) * at.q_tokens * at.q_heads * cdiv(at.head_dim, 4), 256);
    hipLaunchKernelGGL((attention_query_join_kernel<T, DQ>), dim3((unsigned)(n < (1 << 20) ? n : 1 << 20)), dim3(256), 0, st, a);
}

}  // namespace
}  // namespace ddp

extern "C" int64_t ddp_attention_forward_workspace(const ddp_attention *attention, const ddp_heads *q, const ddp_heads *k, const ddp_heads *v) {
    using namespace ddp;
    if (int rc = guarded(nullptr, [&]() -> int { return check_attention("ddp_attention_forward_workspace", attention); })) return -rc;
    return QuerySums(*attention, query_portions(*attention)).bytes + operand_bytes(*attention, {Source{q, true, nullptr}, Source{k, false, nullptr}, Source{v, false, nullptr}});
}

extern "C" int ddp_attention_forward(const ddp_attention *attention, const ddp_heads *q, const ddp_heads *k, const ddp_heads *v, const int32_t *cu_q,
                                     const int32_t *cu_k, const ddp_heads *o, float *lse, void *workspace, int64_t workspace_bytes, void *stream) {
    using namespace ddp;
    return guarded(nullptr, [&]() -> int {
        const char *who = "ddp_attention_forward";
        if (int rc = check_attention(who, attention)) return rc;
        const ddp_attention &at = *attention;
        if (int rc = check_cu(who, at, cu_q, cu_k)) return rc;
        AttentionArgs a = attention_args(at, cu_q, cu_k);
        const Source from[] = {{q, true, &a.q}, {k, false, &a.k}, {v, false, &a.v}};
        for (const Source &s : from)
            if (int rc = take_view(who, at, s.h, s.of_q, *s.v)) return rc;
        if (int rc = take_view(who, at, o, true, a.o)) return rc;
        if (at.q_tokens == 0 || (at.batch == 0 && !at.packed)) return DDP_OK;
        if (!lse) return bad(who, DDP_EINVAL, "lse is NULL");
        if (misaligned(lse, 4)) return bad(who, DDP_EALIGN, "lse is not aligned");
        a.portions = query_portions(at);
        const QuerySums of_q(at, a.portions);
        if (int rc = check_workspace(who, workspace, workspace_bytes, of_q.bytes + operand_bytes(at, from))) return rc;
        char *ws = static_cast<char *>(workspace);
        a.sums = reinterpret_cast<float *>(ws), a.stats = reinterpret_cast<float2 *>(ws + of_q.sums);
        a.lse = lse;
        const hipStream_t st = static_cast<hipStream_t>(stream);
        make_operands(at, from, ws + of_q.bytes, st);
        a.blocks = (int)blocks_of(at, false);
        by_form(at, [&](auto t, auto dp) {
            typedef decltype(t) T;
            constexpr int threads = 256 * kParts<T, dp.value>;
            in_launches(a, a.q_heads, threads, [&](dim3 grid) { hipLaunchKernelGGL((attention_forward_kernel<T, dp.value>), grid, dim3(threads), 0, st, a); });
            if (a.portions > 1) join_queries<Out<T>, false>(at, a, st);
        });
        return launched(who);
    });
}

extern "C" int64_t ddp_attention_backward_workspace(const ddp_attention *attention, const ddp_heads *d_o, const ddp_heads *q, const ddp_heads *k, const ddp_heads *v) {
    using namespace ddp;
    if (int rc = guarded(nullptr, [&]() -> int { return check_attention("ddp_attention_backward_workspace", attention); })) return -rc;
    return BackwardLayout(*attention, operand_bytes(*attention, {Source{d_o, true, nullptr}, Source{q, true, nullptr}, Source{k, false, nullptr}, Source{v, false, nullptr}})).bytes;
}

extern "C" int ddp_attention_backward(const ddp_attention *attention, const ddp_heads *d_o, const ddp_heads *q, const ddp_heads *k, const ddp_heads *v,
                                      const ddp_heads *o, const float *lse, const int32_t *cu_q, const int32_t *cu_k, const ddp_heads *dq,
                                      const ddp_heads *dk, const ddp_heads *dv, void *workspace, int64_t workspace_bytes, void *stream) {
    using namespace ddp;
    return guarded(nullptr, [&]() -> int {
        const char *who = "ddp_attention_backward";
        if (int rc = check_attention(who, attention)) return rc;
        const ddp_attention &at = *attention;
        if (int rc = check_cu(who, at, cu_q, cu_k)) return rc;
        AttentionArgs a = attention_args(at, cu_q, cu_k);
        const Source from[] = {{d_o, true, &a.d_o}, {q, true, &a.q}, {k, false, &a.k}, {v, false, &a.v}};
        for (const Source &s : from)
            if (int rc = take_view(who, at, s.h, s.of_q, *s.v)) return rc;
        for (const Source &s : {Source{o, true, &a.o}, Source{dq, true, &a.dq}, Source{dk, false, &a.dk}, Source{dv, false, &a.dv}})
            if (int rc = take_view(who, at, s.h, s.of_q, *s.v)) return rc;
        if (at.batch == 0 && !at.packed) return DDP_OK;
        const BackwardLayout l(at, operand_bytes(at, from));
        if (!lse && at.q_tokens > 0) return bad(who, DDP_EINVAL, "lse is NULL");
        if (misaligned(lse, 4)) return bad(who, DDP_EALIGN, "lse is not aligned");
        if (int rc = check_workspace(who, workspace, workspace_bytes, l.bytes)) return rc;
        char *ws = static_cast<char *>(workspace);
        a.lse_in = lse;
        a.lse2 = reinterpret_cast<float *>(ws + l.lse2);
        a.delta = reinterpret_cast<float *>(ws + l.delta);
        a.sums = reinterpret_cast<float *>(ws + l.sums), a.stats = reinterpret_cast<float2 *>(ws + l.stats);
        const hipStream_t st = static_cast<hipStream_t>(stream);
        make_operands(at, from, ws + l.copies, st);
        by_form(at, [&](auto t, auto dp) {
            typedef decltype(t) T;
            if (at.q_tokens > 0) {  // (first: it leaves lse and do . o for dk and dv)
                a.blocks = (int)blocks_of(at, false);
                a.portions = query_portions(at);
                constexpr int threads = 256 * kParts<T, dp.value>;
                in_launches(a, a.q_heads, threads, [&](dim3 grid) { hipLaunchKernelGGL((attention_dq_kernel<T, dp.value>), grid, dim3(threads), 0, st, a); });
                if (a.portions > 1) join_queries<Out<T>, true>(at, a, st);
            }
            if (at.k_tokens > 0) {
                a.blocks = (int)blocks_of(at, true);
                a.portions = key_portions(at);
                constexpr int threads = kDkdvThreads<T, dp.value>;
                in_launches(a, a.k_heads, threads, [&](dim3 grid) { hipLaunchKernelGGL((attention_dkdv_kernel<T, dp.value>), grid, dim3(threads), 0, st, a); });
                if (a.portions > 1) {
                    const int64_t n = cdiv((at.packed ? 1 : at.batch) * at.k_tokens * at.k_heads * cdiv(at.head_dim, 4), 256);
                    hipLaunchKernelGGL((attention_join_kernel<Out<T>>), dim3((unsigned)(n < (1 << 20) ? n : 1 << 20), 2), dim3(256), 0, st, a);
                }
            }
        });
        return launched(who);
    });
}
