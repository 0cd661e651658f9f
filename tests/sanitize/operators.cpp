// The operators' entry points with their kernels run on the host: every tensor and workspace is memory of exactly its size, so the sanitizers
// see each access beyond one and each that is not aligned as its type asks; and every element of a result has to be written, nothing else.
#include <cstdio>
#include <cstdlib>
#include <memory>
#include <string>
#include <vector>

#include "hip/hip_runtime.h"

#include "ddp_internal.h"
#include "dreamddp_operators.h"

static std::string last_message;
namespace ddp {
int fail(const ddp_ctx *, int code, const std::string &msg) {
    last_message = msg;
    return code;
}
}  // namespace ddp

static int64_t blocks_run, kMostBlocks = 1 << 30;  // of a launch; of a larger one the first, the last and some between
void host_launch(dim3 grid, dim3 block, void (*thread)(void *), void *f) {
    gridDim = {grid.x, grid.y, grid.z};
    blockDim = {block.x, block.y, block.z};
    const int64_t all = (int64_t)grid.x * grid.y, n = all < kMostBlocks ? all : kMostBlocks;
    for (int64_t i = 0; i < n; ++i) {
        const int64_t b = n == all ? i : i < n / 4 ? i : i >= n - n / 4 ? all - (n - i) : (int64_t)((double)rand() / RAND_MAX * (double)(all - 1));
        blockIdx = {(unsigned)(b % grid.x), (unsigned)(b / grid.x), 0};
        ++blocks_run;
        for (unsigned y = 0; y < block.y; ++y)
            for (unsigned x = 0; x < block.x; ++x) {
                threadIdx = {x, y, 0};
                thread(f);
            }
    }
}

#define CHECK(cond, ...)                                                                                        \
    do {                                                                                                        \
        if (!(cond)) {                                                                                          \
            std::fprintf(stderr, "%s:%d: check failed: %s: %s; ", __FILE__, __LINE__, #cond, last_message.c_str()); \
            std::fprintf(stderr, __VA_ARGS__);                                                                  \
            std::fprintf(stderr, "\n");                                                                         \
            std::exit(1);                                                                                       \
        }                                                                                                       \
    } while (0)

// Memory of `bytes` that starts `past` bytes behind a 256-byte boundary and ends with the allocation.
struct Memory {
    std::unique_ptr<char, void (*)(void *)> all{nullptr, std::free};
    char *p = nullptr;
    int64_t bytes = 0;
    Memory(int64_t n, int64_t past = 0) : bytes(n) {
        if (n <= 0) return;
        void *a = nullptr;
        if (posix_memalign(&a, 256, (size_t)(n + past))) std::abort();
        all.reset(static_cast<char *>(a));
        p = all.get() + past;
        std::memset(a, 0x3c, (size_t)(n + past));  // (small numbers of either type)
    }
};
static const unsigned char kMark = 0xa5;

// A tensor of rows of `cols` elements, [outer][mid][inner] of them with strides.
struct Tensor : Memory {
    int64_t n[3], stride[3], cols, e;
    static int64_t span(const int64_t (&n)[3], const int64_t (&s)[3], int64_t cols) {
        if (!n[0] || !n[1] || !n[2]) return 0;
        return (n[0] - 1) * s[0] + (n[1] - 1) * s[1] + (n[2] - 1) * s[2] + cols;
    }
    Tensor(const int64_t (&n_)[3], const int64_t (&s)[3], int64_t cols_, int64_t e_, int64_t past = 0)
        : Memory(span(n_, s, cols_) * e_, past * e_), n{n_[0], n_[1], n_[2]}, stride{s[0], s[1], s[2]}, cols(cols_), e(e_) {}
    void mark() {
        if (p) std::memset(p, kMark, (size_t)bytes);
    }
    // every element is written, nothing between the rows is
    void written(const char *what) const {
        if (!p) return;
        std::vector<char> seen((size_t)bytes, 0);
        for (int64_t i = 0; i < n[0]; ++i)
            for (int64_t j = 0; j < n[1]; ++j)
                for (int64_t k = 0; k < n[2]; ++k) {
                    const int64_t at = (i * stride[0] + j * stride[1] + k * stride[2]) * e;
                    for (int64_t c = 0; c < cols; ++c) {
                        const unsigned char *x = reinterpret_cast<unsigned char *>(p) + at + c * e;
                        CHECK(!(x[0] == kMark && x[e - 1] == kMark), "%s: row %ld %ld %ld, column %ld is not written", what, i, j, k, c);
                    }
                    std::memset(seen.data() + at, 1, (size_t)(cols * e));
                }
        for (int64_t i = 0; i < bytes; ++i) CHECK(seen[(size_t)i] || (unsigned char)p[i] == kMark, "%s: byte %ld between the rows is written", what, i);
    }
};
static Tensor rows_of(int64_t rows, int64_t cols, int64_t stride, int64_t e, int64_t past) { return Tensor({1, 1, rows}, {0, 0, stride}, cols, e, past); }

#ifdef NORM
static void norm(int kind, int dtype, int64_t rows, int64_t cols, int64_t wider, int64_t past, bool bias) {
    const int64_t e = dtype == DDP_BF16 ? 2 : 4;
    Tensor x = rows_of(rows, cols, cols + wider, e, past), y = rows_of(rows, cols, cols + 2 * wider, e, past), dx = rows_of(rows, cols, cols + 3 * wider, e, past);
    Tensor w = rows_of(1, cols, cols, e, past), b = rows_of(1, cols, cols, e, past + 1), dw = rows_of(1, cols, cols, e, past + 1), db = rows_of(1, cols, cols, e, past);
    Tensor mean = rows_of(1, rows, rows, 4, 0), rstd = rows_of(1, rows, rows, 4, 1);
    for (Tensor *t : {&y, &mean, &rstd}) t->mark();
    ddp_norm n{kind, dtype, rows, cols, cols + wider, cols + 2 * wider, 1e-5f, cols + 3 * wider};
    const bool layer = kind == DDP_NORM_LAYER;
    CHECK(!ddp_norm_forward(&n, x.p, w.p, bias ? b.p : nullptr, y.p, layer ? (float *)mean.p : nullptr, (float *)rstd.p, nullptr), "norm %ld x %ld", rows, cols);
    y.written("y"), rstd.written("rstd");
    if (layer) mean.written("mean");
    std::memset(y.p, 0x3c, (size_t)y.bytes), std::memset(rstd.p, 0x3c, (size_t)rstd.bytes), std::memset(mean.p, 0x3c, (size_t)mean.bytes);
    for (int part = 0; part < 4; ++part) {  // all, dx alone, the columns' sums alone, in the place of dy
        Memory ws(part == 1 ? 0 : ddp_norm_backward_workspace(&n));
        for (Tensor *t : {&dx, &dw, &db}) t->mark();
        if (part == 3) n.dx_stride = n.y_stride;
        CHECK(!ddp_norm_backward(&n, y.p, x.p, w.p, layer ? (float *)mean.p : nullptr, (float *)rstd.p, part == 2 ? nullptr : part == 3 ? y.p : dx.p, part == 1 ? nullptr : dw.p,
                                 bias && part != 1 ? db.p : nullptr, ws.p, ws.bytes, nullptr),
              "norm %ld x %ld", rows, cols);
        if (part < 2) dx.written("dx");
        if (part != 1) dw.written("dw");
        if (part != 1 && bias) db.written("db");
    }
}
static void all(int dtype) {
    for (int kind : {DDP_NORM_LAYER, DDP_NORM_RMS}) {
        const int64_t shapes[][2] = {{1, 1}, {3, 5}, {9, 255}, {5, 256}, {130, 513}, {4100, 24}, {9, 1025}, {2, 2048}, {600, 2049}, {3, 4096}, {5, 4099}, {70, 8200}};
        for (const auto &s : shapes)
            for (int64_t wider : {0, 3}) norm(kind, dtype, s[0], s[1], wider, wider ? 1 : 0, wider == 0);
    }
}
#endif
#ifdef ROTARY
static void rotary(int layout, int dtype, int64_t tokens, int q_heads, int k_heads, int dim, int rotated, int64_t wider, int64_t past, int position_bytes) {
    const int64_t e = dtype == DDP_BF16 ? 2 : 4, head = dim + wider, qt = q_heads * head + wider, kt = k_heads * head + wider;
    Tensor q({1, tokens, q_heads}, {0, qt, head}, dim, e, past), k({1, tokens, k_heads}, {0, kt, head}, dim, e, past);
    Tensor qo({1, tokens, q_heads}, {0, qt + wider, head}, dim, e, past + 1), ko({1, tokens, k_heads}, {0, kt + wider, head}, dim, e, past);
    const int64_t rows = 7;
    Memory table(rows * rotated * 4), positions(tokens * position_bytes);
    for (int64_t t = 0; t < tokens && position_bytes; ++t) {
        const int64_t p = t % 5 == 4 ? (t % 2 ? -7 : rows + 100000) : rows - 1 - t % rows;
        if (position_bytes == 8)
            reinterpret_cast<int64_t *>(positions.p)[t] = t % 10 == 9 ? INT64_MIN : p;
        else
            reinterpret_cast<int32_t *>(positions.p)[t] = (int32_t)p;
    }
    qo.mark(), ko.mark();
    ddp_rotary_shape r{layout, dtype, tokens, q_heads, k_heads, dim, rotated, qt, head, kt, head, qt + wider, head, kt + wider, head, rows, 7, position_bytes ? position_bytes : 4, 1};
    CHECK(!ddp_rotary(&r, q.p, k.p, (float *)table.p, position_bytes ? positions.p : nullptr, qo.p, ko.p, nullptr), "rotary %ld %d %d", tokens, dim, rotated);
    qo.written("q"), ko.written("k");
}
static void all(int dtype) {
    for (int layout : {DDP_ROTARY_HALF, DDP_ROTARY_INTERLEAVED}) {
        const int shapes[][5] = {{1, 1, 1, 2, 2}, {5, 3, 1, 10, 6}, {33, 8, 2, 32, 32}, {7, 12, 12, 64, 32}, {9, 4, 0, 80, 80}, {17, 32, 8, 128, 128}, {3, 2, 1, 300, 256}, {4, 5, 5, 33, 14}, {2, 3, 3, 72, 24}};
        for (const auto &s : shapes)
            for (int bytes : {0, 4, 8})
                for (int64_t wider : {0, 1}) rotary(layout, dtype, s[0], s[1], s[2], s[3], s[4], wider, wider, bytes);
    }
}
#endif
#ifdef ATTENTION
struct Packed {
    std::vector<int32_t> q, k;
};
static void attention(int dtype, int causal, int q_heads, int k_heads, int dim, int batch, int64_t tq, int64_t tk, int64_t wider, int64_t past, const Packed *packed = nullptr,
                      float scale = 0.125f) {
    const int64_t e = dtype == DDP_BF16 ? 2 : 4, head = dim + wider, outer = packed ? 1 : batch;
    auto make = [&](bool of_q, int64_t more) {
        const int64_t heads = of_q ? q_heads : k_heads, tokens = of_q ? tq : tk, token = heads * head + more;
        return Tensor({outer, tokens, heads}, {tokens * token + more, token, head}, dim, e, past);
    };
    Tensor q = make(true, wider), k = make(false, 0), v = make(false, wider), o = make(true, 0), d_o = make(true, wider), dq = make(true, 0), dk = make(false, wider), dv = make(false, 0);
    Tensor lse({outer, q_heads, 1}, {q_heads * tq, tq, 0}, tq, 4, 1);
    auto view = [&](Tensor &t) { return ddp_heads{t.p, t.stride[0], t.stride[1], t.stride[2]}; };
    const ddp_heads hq = view(q), hk = view(k), hv = view(v), ho = view(o), hd = view(d_o), hdq = view(dq), hdk = view(dk), hdv = view(dv);
    ddp_attention a{dtype, causal, q_heads, k_heads, dim, packed ? (int)packed->q.size() - 1 : batch, tq, tk, scale, packed != nullptr};
    // (as the caller's memory, cu ends with the allocation)
    Memory cu_q(packed ? (int64_t)packed->q.size() * 4 : 0), cu_k(packed ? (int64_t)packed->k.size() * 4 : 0);
    if (packed) std::memcpy(cu_q.p, packed->q.data(), (size_t)cu_q.bytes), std::memcpy(cu_k.p, packed->k.data(), (size_t)cu_k.bytes);
    const int32_t *cq = packed ? (int32_t *)cu_q.p : nullptr, *ck = packed ? (int32_t *)cu_k.p : nullptr;
    Memory ws(ddp_attention_forward_workspace(&a, &hq, &hk, &hv));
    o.mark(), lse.mark();
    CHECK(!ddp_attention_forward(&a, &hq, &hk, &hv, cq, ck, &ho, (float *)lse.p, ws.p, ws.bytes, nullptr), "attention %ld %ld %d", tq, tk, dim);
    o.written("o"), lse.written("lse");
    if (lse.p) std::memset(lse.p, 0x3c, (size_t)lse.bytes);
    if (o.p) std::memset(o.p, 0x3c, (size_t)o.bytes);
    Memory bs(ddp_attention_backward_workspace(&a, &hd, &hq, &hk, &hv));
    dq.mark(), dk.mark(), dv.mark();
    CHECK(!ddp_attention_backward(&a, &hd, &hq, &hk, &hv, &ho, (float *)lse.p, cq, ck, &hdq, &hdk, &hdv, bs.p, bs.bytes, nullptr), "attention %ld %ld %d", tq, tk, dim);
    dq.written("dq"), dk.written("dk"), dv.written("dv");
}
static void all(int dtype) {
    const int64_t shapes[][6] = {{1, 1, 1, 1, 1, 8}, {2, 5, 5, 2, 1, 64}, {1, 33, 33, 4, 2, 32}, {1, 129, 129, 3, 3, 80}, {1, 200, 200, 4, 2, 128}, {1, 1, 300, 4, 1, 64}, {2, 70, 391, 2, 2, 128},
                                 {1, 257, 257, 2, 2, 17}, {1, 140, 1, 2, 1, 64}, {2, 5, 0, 2, 1, 40}, {2, 0, 7, 2, 1, 40}, {3, 31, 95, 4, 4, 100}, {1, 300, 129, 2, 2, 1}, {1, 1100, 1100, 1, 1, 64}, {1, 900, 650, 2, 1, 120}};
    for (const auto &s : shapes)
        for (int causal : {0, 1})
            for (int64_t wider : {0, 8, 3}) attention(dtype, causal, (int)s[3], (int)s[4], (int)s[5], (int)s[0], s[1], s[2], wider, wider == 3, nullptr, wider == 8 ? -0.125f : 0.125f);
    const Packed lengths[] = {{{0, 7, 8, 8, 138, 202, 202, 203}, {0, 7, 8, 8, 138, 202, 202, 203}}, {{0, 10, 10, 75, 203}, {0, 31, 40, 90, 150}}, {{0, 40, 100}, {0, 30, 90}}, {{0}, {0}},
                              {{5, 40, 1 << 30}, {9, 20, 1 << 30}}, {{0, 850, 853, 853, 1300}, {0, 900, 900, 905, 1500}}};
    for (const Packed &p : lengths)
        for (int causal : {0, 1})
            for (int dim : {64, 100}) {
                const int64_t tq = p.q.back() > 1 << 20 ? 170 : p.q.back() + 13, tk = p.k.back() > 1 << 20 ? 150 : p.k.back() + 5;
                attention(dtype, causal, 2, 1, dim, 0, tq, tk, dim == 100 ? 4 : 0, 0, &p);
            }
}
#endif
#ifdef ENTROPY
static void entropy(int dtype, int64_t tokens, int64_t vocab, int64_t hidden, int64_t wider, int64_t past, bool whole = true) {
    const int64_t e = dtype == DDP_BF16 ? 2 : 4;
    Tensor x = rows_of(tokens, hidden, hidden + wider, e, past), w = rows_of(vocab, hidden, hidden + 2 * wider, e, past);
    Tensor dx = rows_of(tokens, hidden, hidden + wider, e, past + 1), dw = rows_of(vocab, hidden, hidden + wider, e, past);
    Tensor loss = rows_of(1, tokens, tokens, 4, 1), lse = rows_of(1, tokens, tokens, 4, 0), g = rows_of(1, tokens, tokens, 4, 1);
    Memory targets(tokens * 8);
    for (int64_t t = 0; t < tokens; ++t) reinterpret_cast<int64_t *>(targets.p)[t] = t % 6 == 5 ? (t % 12 == 5 ? -100 : vocab + t) : t % 6 == 4 ? vocab - 1 : t * 7919 % vocab;
    ddp_head h{dtype, tokens, vocab, hidden, hidden + wider, hidden + 2 * wider, hidden + wider, hidden + wider};
    kMostBlocks = whole ? 1 << 30 : 24;
    Memory ws(ddp_cross_entropy_forward_workspace(&h, x.p, w.p));
    loss.mark(), lse.mark();
    CHECK(!ddp_cross_entropy_forward(&h, x.p, w.p, (int64_t *)targets.p, (float *)loss.p, (float *)lse.p, ws.p, ws.bytes, nullptr), "%ld %ld %ld", tokens, vocab, hidden);
    if (whole) loss.written("loss"), lse.written("lse");
    std::memset(lse.p, 0x3c, (size_t)lse.bytes);
    Memory bs(ddp_cross_entropy_backward_workspace(&h, x.p, w.p));
    for (int part = 0; part < 3; ++part) {
        dx.mark(), dw.mark();
        CHECK(!ddp_cross_entropy_backward(&h, (float *)g.p, x.p, w.p, (int64_t *)targets.p, (float *)lse.p, part == 2 ? nullptr : dx.p, part == 1 ? nullptr : dw.p, bs.p, bs.bytes, nullptr),
              "%ld %ld %ld", tokens, vocab, hidden);
        if (whole && part != 2) dx.written("dx");
        if (whole && part != 1) dw.written("dw");
        if (!whole) break;
    }
    kMostBlocks = 1 << 30;
}
static void all(int dtype) {
    const int64_t shapes[][3] = {{1, 1, 1}, {1, 2, 8}, {3, 5, 7}, {64, 128, 64}, {65, 129, 96}, {17, 1000, 33}, {100, 700, 256}, {300, 257, 130}, {5, 3001, 64}, {130, 50, 1000}, {31, 1000, 129},
                                 {64, 300, 257}, {70, 1025, 1100}, {17, 2000, 1030}};
    for (const auto &s : shapes)
        for (int64_t wider : {0, 8, 3}) entropy(dtype, s[0], s[1], s[2], wider, wider == 3);
    entropy(dtype, 3400, 3500, 72, 0, 0, false);     // large tiles
    entropy(dtype, 9000, 20011, 64, 0, 0, false);    // pieces of the vocabulary, the last one shorter
    entropy(dtype, 1100, 12345, 192, 8, 0, false);
}
#endif

int main() {
    for (int dtype : {DDP_F32, DDP_BF16}) all(dtype);
    std::printf("ok, %ld workgroups\n", blocks_run);
}
