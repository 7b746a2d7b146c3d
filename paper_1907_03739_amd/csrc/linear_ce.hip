// Cross entropy of labels with the softmax of a linear layer's outputs, z = x W^T +
// bias, and its gradients, without the logits in memory (pvconv_train.h).
//
// Forward: tiles of the product keep their logits in registers and leave a row's
// maximum and its sum of exponentials for each 64 classes (and the label's logit);
// the rows' statistics are joined in a second launch. Backward: the product again,
// whose epilogue turns a logit into dz = weight (exp(z - lse) - [class = label]), in
// bf16 parts, for a piece of the vocabulary at a time: dx += dz W and dW = dz^T x are
// then plain products, of W, dz and x as they lie (pv_product.h). Up to 64 classes, a
// wave holds whole rows: loss and dz come from one product.
//
// Multiplying twice is cheaper than keeping the logits up to some thousand channels: in 32
// bits, as a difference of logits needs them, they would be written and read at 8 bytes of
// memory for 2 K operations. 4096 x 512, 49999 classes, bf16, us: statistics 259 (0.81
// PFLOP/s), dz 403 (0.52), dx of its two parts 441 (0.95), dw 467 (0.90). The first two are
// bound by their epilogues beside eight slices of products: the matrix cores work 36 and
// 22 % of the time, the vector ones 27 and 29 (some nine instructions a logit, the
// exponential at a quarter of their rate among them), one after the other in most waves.
// The exponential is the hardware's power of two: off by 2^-24 |z - lse| of itself, as a
// rounding of z would make it.
#include "pv_product.h"
#include "pv_wave.h"

namespace {

constexpr int kThreads = 256;
constexpr float kInf = __builtin_huge_valf();

struct DzPanel {  // where dz goes: bf16 parts, rows of a pitch in bytes (p NULL: nowhere)
    uint8_t* p;
    size_t pitch, part_bytes;
    int parts, rows;  // zeros from the last row on
};

struct Ce {
    const float* bias;      // of the piece's first class, or NULL
    const int32_t* labels;
    int v0, V;              // the piece's first class; all classes
    float2* stats;          // [M][nb]: maximum, sum of exponentials about it
    int nb;
    float* zlab;            // [M]: the label's logit
    float* loss;
    float* lse;
    const float* weight;    // [M] or NULL
    DzPanel dz;             // [M][piece]
    float* sums;            // [row blocks][piece]: dz summed over a wave's rows, or NULL
};

__device__ __forceinline__ float lanes_max(float v) {  // over the lanes of a row
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float lanes_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// The next bf16 part of v, which leaves v - part (dz is finite, or NaN whole).
__device__ __forceinline__ uint32_t next_part2(float& a, float& b) {
    const uint32_t w = pv_pack_bf16x2(a, b);
    a -= __uint_as_float(w << 16);
    b -= __uint_as_float(w & 0xffff0000u);
    return w;
}

// a branch of the wave: as one of its lanes, the compiler takes both sides
__device__ __forceinline__ bool any_lane(bool b) { return __builtin_amdgcn_ballot_w64(b) != 0; }

enum Mode { kStats, kWhole, kGrad };

template <int MODE>
struct CeEpi {
    Ce c;

    // one part of dz of a row: two runs of eight classes a lane
    __device__ __forceinline__ void store(int part, int m, int nb, float (&d)[16]) const {
#pragma unroll
        for (int a = 0; a < 2; a++) {
            pv_u32x4 w;
#pragma unroll
            for (int q = 0; q < 4; q++) w[q] = next_part2(d[8 * a + 2 * q], d[8 * a + 2 * q + 1]);
            const size_t at = (size_t)(nb + 32 * a) * 2;
            if (m < c.dz.rows && at < c.dz.pitch)
                *(pv_u32x4*)(c.dz.p + part * c.dz.part_bytes + (size_t)m * c.dz.pitch + at) = w;
        }
    }

    template <int MI>
    __device__ __forceinline__ void tile(const PvProduct& p, int mw, int nw, int lane,
                                         const pv_f32x4 (&acc)[4][MI]) const {
        const int r = lane & 15, h = lane >> 4, nb = nw + 8 * h;
        // a class past the last has the logit -inf, and so takes no part
        float b[16], cs[16];
        pv_load_columns(c.bias, nb, p.N, -kInf, b);
#pragma unroll
        for (int q = 0; q < 16; q++) cs[q] = 0.f;
        const bool grads = MODE == kGrad || (MODE == kWhole && (c.dz.p || c.sums));
        // what the rows need, all of it under way at once
        int labels[MI];
        float lses[MI], weights[MI];
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const int m = min(mw + 16 * i + r, p.M - 1);
            labels[i] = c.labels[m];
            lses[i] = MODE == kGrad ? c.lse[m] : 0.f;
            weights[i] = MODE != kStats && c.weight ? c.weight[m] : 1.f;
        }
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const int m = mw + 16 * i + r, label = labels[i];
            const bool known = label >= 0 && label < c.V;
            // which of the lane's sixteen classes the label is, if any (few lanes have it)
            const unsigned to = (unsigned)label - (unsigned)(c.v0 + nb);
            const int at = to < 8u ? (int)to : to - 32u < 8u ? (int)to - 24 : -1;
            float z[16];
#pragma unroll
            for (int q = 0; q < 16; q++) z[q] = acc[q >> 2][i][q & 3] + b[q];
            float lse = 0.f;
            if constexpr (MODE != kGrad) {
                float top = z[0];
#pragma unroll
                for (int q = 1; q < 16; q++) top = fmaxf(top, z[q]);
                top = lanes_max(top);
                // (every logit -inf, or not a number: fmaxf passes NaN over)
                const float about = top == -kInf ? 0.f : top;
                float sum = 0.f, zl = 0.f;
#pragma unroll
                for (int q = 0; q < 16; q++) sum += __expf(z[q] - about);
                if (any_lane(at >= 0)) {
#pragma unroll
                    for (int q = 0; q < 16; q++) zl = q == at ? z[q] : zl;
                }
                sum = lanes_sum(sum);
                if constexpr (MODE == kStats) {
                    if (m < p.M) {
                        if (h == 0 && nw < p.N)
                            c.stats[(size_t)m * c.nb + (unsigned)nw / 64] = make_float2(top, sum);
                        if (known && at >= 0) c.zlab[m] = zl;
                    }
                } else {
                    lse = sum == 0.f ? -kInf : about + logf(sum);
                    zl = lanes_sum(known && at >= 0 ? zl : 0.f);
                    if (m < p.M && h == 0) {
                        c.lse[m] = lse;
                        c.loss[m] = known && lse != -kInf ? lse - zl : 0.f;
                    }
                }
            } else {
                lse = lses[i];
            }
            if (MODE != kStats && grads) {
                const float g = m < p.M && known && lse != -kInf ? weights[i] : 0.f;
#pragma unroll
                for (int q = 0; q < 16; q++) z[q] = g * __expf(z[q] - lse);
                if (any_lane(at >= 0)) {
#pragma unroll
                    for (int q = 0; q < 16; q++) z[q] -= q == at ? g : 0.f;
                }
                if (any_lane(g == 0.f)) {  // 0, whatever the logits are
#pragma unroll
                    for (int q = 0; q < 16; q++) z[q] = g == 0.f ? 0.f : z[q];
                }
#pragma unroll
                for (int q = 0; q < 16; q++) cs[q] += z[q];
                if (c.dz.p)
                    for (int part = 0; part < c.dz.parts; part++) store(part, m, nb, z);
            }
        }
        if (MODE != kStats && grads && c.sums) {
            // over the 16 rows of lanes: halves of the columns change places, so that
            // lane r is left with the sum of column r
#pragma unroll
            for (int w = 8; w; w >>= 1) {
                // (by masks: of two elements chosen by the lane the compiler makes one
                // that it looks for among all)
                const uint32_t up = r & w ? ~0u : 0u;
#pragma unroll
                for (int q = 0; q < w; q++) {
                    const uint32_t x = __float_as_uint(cs[q]), y = __float_as_uint(cs[q + w]);
                    const float keep = __uint_as_float((y & up) | (x & ~up)),
                                give = __uint_as_float((x & up) | (y & ~up));
                    cs[q] = keep + __shfl_xor(give, w);
                }
            }
            const int block = mw / (16 * MI), n = pv_col(nb, r);
            if (n < p.N) c.sums[(size_t)block * p.N + n] = cs[0];
        }
    }
    __device__ __forceinline__ void one(int, int, float) const {}  // never split
};

// A row's statistics over the piece's blocks (TEAM lanes a row), joined with those of
// the pieces before it (run), and at the last piece lse and loss.
struct Join {
    const float2* stats;
    int nb, M, V;
    float2* run;
    bool first, last;
    const int32_t* labels;
    const float* zlab;
    float* loss;
    float* lse;
};
template <int TEAM>
__global__ __launch_bounds__(kThreads) void pv_ce_join_kernel(Join j) {
    constexpr int kRows = kThreads / TEAM;
    const int lane = threadIdx.x % TEAM;
    for (size_t row0 = (size_t)blockIdx.x * kRows; row0 < (size_t)j.M;
         row0 += (size_t)gridDim.x * kRows) {
        const size_t m = min(row0 + threadIdx.x / TEAM, (size_t)j.M - 1);
        float top = -kInf, sum = 0.f;
        auto add = [&](float t, float s) {
            const float to = fmaxf(top, t);
            const float about = to == -kInf ? 0.f : to;
            // -inf about a finite value: exp gives 0. Sums that are not numbers stay so.
            sum = sum * __expf(top - about) + s * __expf(t - about);
            top = to;
        };
        for (int k0 = 0; k0 < j.nb; k0 += 8 * TEAM) {
            float2 v[8];
#pragma unroll
            for (int u = 0; u < 8; u++)
                v[u] = j.stats[m * j.nb + min(k0 + u * TEAM + lane, j.nb - 1)];
#pragma unroll
            for (int u = 0; u < 8; u++)
                if (k0 + u * TEAM + lane < j.nb) add(v[u].x, v[u].y);
        }
#pragma unroll
        for (int w = 1; w < TEAM; w <<= 1) {
            const float t = __shfl_xor(top, w), s = __shfl_xor(sum, w);
            add(t, s);
        }
        if (lane || row0 + threadIdx.x / TEAM >= (size_t)j.M) continue;
        if (!j.first) add(j.run[m].x, j.run[m].y);
        if (!j.last) {
            j.run[m] = make_float2(top, sum);
            continue;
        }
        const float lse = sum == 0.f ? -kInf : (top == -kInf ? 0.f : top) + logf(sum);
        const int label = j.labels[m];
        j.lse[m] = lse;
        j.loss[m] = label >= 0 && label < j.V && lse != -kInf ? lse - j.zlab[m] : 0.f;
    }
}

// ---- the plan --------------------------------------------------------------
constexpr int kWholeClasses = 64;
// dz of a piece: at most this many bytes of all its parts, at least this many classes
// (each piece reads and writes the 32-bit sums of dx)
constexpr size_t kPieceBytes = (size_t)1 << 29;
constexpr int kLeastClasses = 2048;
// statistics of a piece of the forward
constexpr size_t kStatsBytes = (size_t)1 << 26;

int parts_of(bool bf16) { return bf16 ? 1 : 3; }
// Parts of dz for a gradient: 24 bits for an fp32 one; for a bf16 one two parts, which leave
// 2^-16 of a term where the result's rounding is 2^-8. (One part leaves 2^-8 of a term more,
// which nothing averages: a row's dz at its label scales the row's whole dx, and rows of
// one weight and small probabilities round alike, which scales their whole dw. The steps of
// 4096 x 512, 49999 classes, and 8192 x 2048, 5003, take 1024 and 679 us with it, 1612 and
// 1063 without.) The other factor of a bf16 gradient is rounded to 16 bits too.
int dz_parts_of(bool bf16) { return bf16 ? 2 : 3; }

struct Plan {
    PvPanel x, w;             // what every product takes
    bool pack_x, pack_w;
    bool whole;
    unsigned grad_sizes;
    int forward_classes, classes;  // a piece's
    PvPanel dz;
    PvProduct dx, dw;         // of a piece of `classes`
    int pair;                 // the tile in which the two are one launch, or -1
    float2 *stats, *run;
    float *zlab, *lse, *sums, *acc;
    uint32_t* partial;
    size_t total;
};

// Bytes from a row of dz to the next: whole slices, not a multiple of 4 KB, whose rows would
// lie in few of the memory's channels (4096 x 512, 49999 classes, the first piece's 64 KB
// apart: the step takes 1743 us, 1612 with a slice more).
size_t dz_pitch(int classes) {
    const size_t pitch = pv_up(classes, kDeep) * 2;
    return pitch % 4096 ? pitch : pitch + kSlice;
}

template <class T>
int row_blocks_of(int M) {
    return (int)(pv_up(M, T::TM) / (16 * T::MI));
}
int row_blocks(int M, int size) {  // as many as waves have rows
    switch (size) {
        case kPvL: return row_blocks_of<PvTileL>(M);
        case kPvG: return row_blocks_of<PvTileG>(M);
        case kPvM: return row_blocks_of<PvTileM>(M);
        case kPvP: return row_blocks_of<PvTileP>(M);
        default: return row_blocks_of<PvTileS>(M);
    }
}
// The tiles of an epilogue. A wave that has whole rows has all of 64 columns; beside the
// sums of the largest tiles there are no registers for dz. (dz of 4096 x 512, 32768 classes,
// us: 317 in 256 x 128, 354 in 128 x 128.)
constexpr unsigned sizes_of(int mode) {
    const unsigned narrow = 1u << kPvS | 1u << kPvP;
    if (mode == kWhole) return narrow;
    if (mode == kStats) return kPvAnySize;
    return narrow | 1u << kPvM | 1u << kPvG;
}
// The product of x with n classes from v0 on.
PvProduct logits_of(const PvPanel& x, const PvPanel& w, int M, int K, int v0, int n,
                    unsigned sizes) {
    PvProduct q{};
    q.a = x;
    q.b = w;
    q.b.p += (size_t)v0 * w.pitch;
    q.M = M;
    q.N = n;
    q.slices = pv_slices(K, kDeep);
    pv_pairs(q, x.parts, w.parts);
    pv_plan(q, false, sizes);
    return q;
}

Plan carve(void* base, const PvLinearCe& a, bool forward, bool grads, bool may_direct) {
    PvCarve c{(char*)base, 0};
    Plan p{};
    p.whole = a.V <= kWholeClasses;
    auto operand = [&](const PvRows& r, int rows, PvPanel& to, bool& pack) {
        pack = !(may_direct && pv_in_place(r, a.K));
        if (pack)
            to = pv_take_panel(c, rows, a.K, parts_of(r.bf16));
        else
            to = pv_panel_of(r, rows);
    };
    operand(a.x, a.M, p.x, p.pack_x);
    operand(a.w, a.V, p.w, p.pack_w);
    if (forward) {
        if (!p.whole) {
            const size_t most = kStatsBytes / 8 / (a.M > 0 ? a.M : 1) * 64;
            p.forward_classes =
                most >= (size_t)a.V ? a.V : (int)(most < 4096 ? 4096 : most / 128 * 128);
            if (p.forward_classes > a.V) p.forward_classes = a.V;
            p.stats = (float2*)c.take((size_t)a.M * ((p.forward_classes + 63) / 64) * 8);
            p.run = (float2*)c.take((size_t)a.M * 8);
            p.zlab = (float*)c.take((size_t)a.M * 4);
        }
        p.lse = (float*)c.take((size_t)a.M * 4);
    }
    if (!grads) {
        p.total = c.off;
        return p;
    }
    const bool want_dx = a.dx.p != nullptr, want_dw = a.dw.p != nullptr;
    const int px = dz_parts_of(a.dx.bf16), pw = dz_parts_of(a.dw.bf16);
    // (of both, wanted or not: the workspace of fewer gradients is then no larger)
    const size_t per = pv_up(a.M > 0 ? a.M : 1, 64) * 2 * (px > pw ? px : pw);
    size_t n = kPieceBytes / per / 256 * 256;
    if (n < (size_t)kLeastClasses) n = kLeastClasses;
    p.classes = n >= (size_t)a.V ? a.V : (int)n;
    p.grad_sizes = sizes_of(p.whole ? kWhole : kGrad);
    // (of both, wanted or not: one alone has the same bits)
    auto plan = [&](PvProduct& q, const PvPanel& x, const PvPanel& y, int rows, int cols,
                    int depth) {
        q.a = x;
        q.b = y;
        q.M = rows;
        q.N = cols;
        q.slices = pv_slices(depth, kDeep);
        pv_pairs(q, x.parts, y.parts);
        pv_plan(q, true);
    };
    PvPanel dz{}, w = p.w, x = p.x;
    if (want_dx || want_dw)
        dz = p.dz = pv_take_panel(c, (int)pv_up(a.M, kDeep), (int)(dz_pitch(p.classes) / 2),
                                  want_dx && want_dw ? (px > pw ? px : pw) : want_dx ? px : pw);
    dz.parts = px;
    if (a.dx.bf16 && w.parts > 2) w.parts = 2;  // (of the three that are there)
    plan(p.dx, dz, w, a.M, a.K, p.classes);
    dz.parts = pw;
    if (a.dw.bf16 && x.parts > 2) x.parts = 2;
    plan(p.dw, dz, x, p.classes, a.K, a.M);
    p.pair = p.classes < a.V ? -1 : pv_pair_size(p.dx, p.dw);
    if (p.pair >= 0) {
        pv_take_pair(p.dx, p.pair);
        pv_take_pair(p.dw, p.pair);
    }
    // the splits' sums of a whole piece and of the last one, which may have fewer classes
    size_t partial = 0;
    const int tail = a.V % p.classes;
    auto sums = [&](const PvProduct& q) {
        const size_t b = pv_partial_bytes(q);
        partial = partial > b ? partial : b;
    };
    if (want_dx) {
        sums(p.dx);
        if (tail) {
            PvProduct q = p.dx;
            q.slices = pv_slices(tail, kDeep);
            pv_plan(q, true);
            sums(q);
        }
        if (p.classes < a.V) p.acc = (float*)c.take((size_t)a.M * a.K * 4);
    }
    if (want_dw) {
        sums(p.dw);
        if (tail) {
            PvProduct q = p.dw;
            q.M = tail;
            pv_plan(q, true);
            sums(q);
        }
    }
    p.partial = (uint32_t*)c.take(partial);
    if (a.dbias) {
        // (of a smaller last piece too, whose tiles may be smaller)
        const auto need = [&](int n) {
            const PvProduct q = logits_of(p.x, p.w, a.M, a.K, 0, n, p.grad_sizes);
            return (size_t)row_blocks(a.M, q.size) * n;
        };
        const size_t b = need(p.classes), t = tail ? need(tail) : 0;
        p.sums = (float*)c.take((b > t ? b : t) * 4);
    }
    p.total = c.off;
    return p;
}

template <int MODE>
void run_logits(const PvProduct& p, const Ce& c, hipStream_t s) {
    pv_run_product<false, false, false, sizes_of(MODE)>(p, CeEpi<MODE>{c}, s);
}

}  // namespace

size_t pv_linear_ce_ws_bytes(const PvLinearCe& a, bool forward, bool grads) {
    return carve(nullptr, a, forward, grads, false).total;
}

pvconv_status pv_launch_linear_ce(const PvLinearCe& a, bool forward, void* ws, hipStream_t s) {
    const bool grads = a.dx.p || a.dw.p || a.dbias;
    const Plan p = carve(ws, a, forward, grads, true);
    float* lse = a.lse ? a.lse : p.lse;
    auto kind = [](const PvRows& r) { return r.bf16 ? kPvBf16 : kPvF32; };
    PvPacks packs{};
    if (p.pack_x && a.M > 0) packs.add(pv_pack_of(a.x.p, kind(a.x), a.x.ld, a.M, a.K, p.x));
    if (p.pack_w && a.M > 0) packs.add(pv_pack_of(a.w.p, kind(a.w), a.w.ld, a.V, a.K, p.w));
    pv_launch_packs(packs, s);
    auto logits = [&](int v0, int n, unsigned sizes) {
        return logits_of(p.x, p.w, a.M, a.K, v0, n, sizes);
    };
    Ce c{};
    c.labels = a.labels;
    c.V = a.V;
    c.weight = a.weight;
    c.lse = lse;
    c.loss = a.loss;
    if (forward && !p.whole) {
        for (int v0 = 0; v0 < a.V; v0 += p.forward_classes) {
            const int n = a.V - v0 < p.forward_classes ? a.V - v0 : p.forward_classes;
            c.v0 = v0;
            c.bias = a.bias ? a.bias + v0 : nullptr;
            c.stats = p.stats;
            c.nb = (n + 63) / 64;
            c.zlab = p.zlab;
            run_logits<kStats>(logits(v0, n, sizes_of(kStats)), c, s);
            const Join j{p.stats, c.nb, a.M, a.V, p.run, v0 == 0, v0 + n == a.V, a.labels, p.zlab,
                         a.loss, lse};
            if (a.M > 0) {
                if (c.nb <= 8)
                    hipLaunchKernelGGL((pv_ce_join_kernel<1>), dim3(pv_blocks(a.M, kThreads)),
                                       dim3(kThreads), 0, s, j);
                else
                    hipLaunchKernelGGL((pv_ce_join_kernel<64>), dim3(pv_blocks(a.M, 4)),
                                       dim3(kThreads), 0, s, j);
            }
        }
    } else if (forward && !grads) {
        c.bias = a.bias;
        run_logits<kWhole>(logits(0, a.V, sizes_of(kWhole)), c, s);
    }
    if (!grads) return pv_launch_status();
    for (int v0 = 0; v0 < a.V; v0 += p.classes) {
        const int n = a.V - v0 < p.classes ? a.V - v0 : p.classes;
        c.v0 = v0;
        c.bias = a.bias ? a.bias + v0 : nullptr;
        c.sums = p.sums;
        const size_t pitch = dz_pitch(n);
        c.dz = DzPanel{(uint8_t*)p.dz.p, pitch, p.dz.part_bytes, p.dz.parts, p.dz.rows};
        const PvProduct z = logits(v0, n, p.grad_sizes);
        const PvSums none{nullptr, 0, 0, nullptr},
            sums{p.sums, row_blocks(a.M, z.size), n, a.dbias ? a.dbias + v0 : nullptr};
        const bool dx = a.dx.p && a.M > 0, dw = a.dw.p;
        if (p.whole && forward)
            run_logits<kWhole>(z, c, s);
        else
            run_logits<kGrad>(z, c, s);
        PvProduct to_dx = p.dx, to_dw = p.dw;
        to_dx.a.pitch = to_dw.a.pitch = pitch;
        to_dx.partial = to_dw.partial = p.partial;  // one after the other
        to_dx.b.p += (size_t)v0 * to_dx.b.pitch;
        to_dx.b.rows = n;
        if (n < p.classes) {
            to_dx.slices = pv_slices(n, kDeep);
            pv_plan(to_dx, true);
            to_dw.M = n;
            pv_plan(to_dw, true);
        }
        const PvPlain out_dx{v0 + n == a.V ? a.dx : PvRows{p.acc, false, a.K}, v0 ? p.acc : nullptr},
            out_dw{PvRows{(char*)a.dw.p + (size_t)v0 * a.dw.ld * (a.dw.bf16 ? 2 : 4), a.dw.bf16,
                          a.dw.ld}, nullptr};
        if (dx && dw && p.pair >= 0) {
            pv_launch_pair(to_dx, out_dx, to_dw, out_dw, sums, s);
        } else {
            if (dx) pv_launch_plain(to_dx, false, out_dx, dw ? none : sums, s);
            if (dw) pv_launch_plain(to_dw, true, out_dw, sums, s);
            if (!dx && !dw) pv_launch_sum_runs(sums, s);
        }
    }
    return pv_launch_status();
}
