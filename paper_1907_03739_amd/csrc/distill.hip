// Distillation loss against a teacher's top logits, and its gradient
// (pvconv_train.h).
//
// With m the row's maximum, s_T = sum exp((z - m) / T) and s_1 likewise at
// temperature 1, lse_T = m / T + log s_T: the loss needs z at the stored entries
// and the label beside them, the gradient of a logit is
//   w (alpha T (exp(z / T - lse_T) - p) + (1 - alpha) (exp(z - lse_1) - [label])).
// z is read once and, where the gradient is taken, dz written. A long row's loss is
// bound by vector issue (two exponentials, a guard and a maximum a logit), its gradient
// by memory.
// Rows of up to 2048 classes stay in the registers of 4 to 64 lanes, from the one
// read to the gradient. Rows of more take a workgroup, which goes over them once
// with a running maximum and sums a thread and, for the gradient, a second time,
// when they still lie in the caches.
#include <type_traits>

#include "pv_train.h"

namespace {

__device__ __forceinline__ bool bad_class(int c, int V) { return (unsigned)c >= (unsigned)V; }

struct Max {
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Add {
    __device__ float operator()(float a, float b) const { return a + b; }
};
// Reduction over LANES consecutive lanes; every one gets the result.
template <int LANES, typename Op>
__device__ __forceinline__ float lanes_reduce(float v, Op op) {
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) v = op(v, __shfl_xor(v, m));
    return v;
}

// What a row's terms weigh, and its label.
struct Terms {
    float kl, ce;  // alpha T, 1 - alpha, or 0 for a term that the row lacks
    int label;
};

__device__ __forceinline__ float log_of(float s) { return __logf(s); }

struct Args {
    PvDistill d;
    float tau;            // 1 / T
    bool soft, hard;      // alpha > 0; labels and alpha < 1
    const float* weight;  // row_weight or dloss
    float* loss;
    float* lse;           // out of a forward, or the statistics of the gradient alone
    PvRows dz;
};

// Whether a row has no logit left: its maximum is -inf, or is -inf over T, as the
// saved lse of the row then is too. A NaN stays one.
__device__ __forceinline__ bool is_empty(float m, float s1, float st, const Args& a) {
    return (m == -INFINITY || (a.soft && m * a.tau == -INFINITY)) && !(s1 != s1) && !(st != st);
}

// The gradient of a logit before the entries of its class. The branches are the
// call's, not the row's: a row that lacks a term weighs it 0, and its
// exponential is finite.
__device__ __forceinline__ float soft_grad(float z, const Args& a, const Terms& w, float lse1,
                                           float lset) {
    float g = 0.f;
    if (a.soft) g = w.kl * __expf(fmaf(z, a.tau, -lset));
    if (a.hard) g = fmaf(w.ce, __expf(z - lse1), g);
    return g;
}

// ---------------------------------------------------------------------------
// Few classes: TEAM lanes hold a row, E logits each (class e * TEAM + lane).
// STATS: loss and statistics are computed, else read. GRAD: dz is written.
// 16384 x 50, top 8, fp32, loss and gradient: 7.9 us, of which 1.5 would move the
// bytes: bound by a row's chain of reductions and entries.
// ---------------------------------------------------------------------------
constexpr int kThreads = 256;

template <int TEAM, int E, bool BF16, bool STATS, bool GRAD>
__global__ __launch_bounds__(kThreads) void pv_distill_short_kernel(Args a) {
    // (of gradients: the last entry that signed a class)
    __shared__ uint16_t owner[GRAD ? kThreads / TEAM : 1][GRAD ? TEAM * E : 1];
    const PvDistill& d = a.d;
    const int lane = threadIdx.x % TEAM;
    const size_t step = (size_t)gridDim.x * (kThreads / TEAM);
    // teams of a wave run the same number of rounds: their shuffles stay whole
    const size_t first = (size_t)blockIdx.x * (kThreads / TEAM) + threadIdx.x / TEAM;
    for (size_t row0 = (size_t)blockIdx.x * (kThreads / TEAM); row0 < (size_t)d.M; row0 += step) {
        const size_t at = row0 + (first - (size_t)blockIdx.x * (kThreads / TEAM));
        const bool live = at < (size_t)d.M;
        const size_t row = live ? at : (size_t)d.M - 1;
        float z[E];
#pragma unroll
        for (int e = 0; e < E; e++) {
            const int c = e * TEAM + lane;
            z[e] = c < d.V ? pv_load_one(d.z.p, BF16, row * d.z.ld + c) : -INFINITY;
        }
        Terms w{0.f, 0.f, d.labels ? d.labels[row] : -1};
        if (a.hard && !bad_class(w.label, d.V)) w.ce = 1.f - d.alpha;

        // the teacher's entries: maximum, and sum at temperature T (of differences: an
        // entry over T may be beyond 32 bits)
        float tmax = -INFINITY, tsum = 0.f;
        if (a.soft) {
            for (int j = lane; j < d.top; j += TEAM)
                if (!bad_class(d.t_class[row * d.top + j], d.V))
                    tmax = fmaxf(tmax, d.t_val[row * d.top + j]);
            tmax = lanes_reduce<TEAM>(tmax, Max());
            if (tmax == -INFINITY) tmax = 0.f;
            for (int j = lane; j < d.top; j += TEAM)
                if (!bad_class(d.t_class[row * d.top + j], d.V))
                    tsum += __expf((d.t_val[row * d.top + j] - tmax) * a.tau);
            tsum = lanes_reduce<TEAM>(tsum, Add());
            // 0 only without an entry of weight; a NaN stays
            if (!(tsum == 0.f)) w.kl = d.alpha * d.temperature;
        }
        const float tinv = 1.f / tsum;

        float lse1, lset;
        bool empty;
        if constexpr (STATS) {
            float m = -INFINITY, s1 = 0.f, st = 0.f;
#pragma unroll
            for (int e = 0; e < E; e++) m = fmaxf(m, z[e]);
            m = lanes_reduce<TEAM>(m, Max());
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float u = z[e] == -INFINITY ? -INFINITY : z[e] - m;
                if (a.hard) s1 += __expf(u);
                if (a.soft) st += __expf(u * a.tau);
            }
            if (a.hard) s1 = lanes_reduce<TEAM>(s1, Add());
            if (a.soft) st = lanes_reduce<TEAM>(st, Add());
            empty = is_empty(m, s1, st, a);
            lse1 = a.hard ? m + log_of(s1) : 0.f;
            lset = a.soft ? m * a.tau + log_of(st) : 0.f;
        } else {
            lse1 = a.lse[2 * row];
            lset = a.lse[2 * row + 1];
            empty = lse1 == -INFINITY || lset == -INFINITY;
        }

        const float scale = GRAD ? (a.weight ? a.weight[row] : 1.f) : 0.f;
        const bool zero = scale == 0.f || empty;
        if constexpr (GRAD) {
#pragma unroll
            for (int e = 0; e < E; e++) {
                const int c = e * TEAM + lane;
                if (c < d.V && live)
                    pv_store_one(a.dz.p, a.dz.bf16, row * a.dz.ld + c,
                                 zero ? 0.f : scale * soft_grad(z[e], a, w, lse1, lset));
            }
        }
        // the entries: their part of the loss, and the whole gradient of their
        // classes, stored after the lines above (same wave, same address order)
        float kl = 0.f;
        const int entries = w.kl != 0.f ? d.top : 0;
        volatile uint16_t* own = owner[threadIdx.x / TEAM];
        bool repeated = false;
        if (GRAD && entries) {
            // Each entry signs its class; one that finds another's name there shares
            // its class. Only then is every entry compared with every other.
            for (int j = lane; j < entries; j += TEAM) {
                const int c = d.t_class[row * d.top + j];
                if (!bad_class(c, d.V)) own[c] = (uint16_t)j;
            }
            __builtin_amdgcn_wave_barrier();
            for (int j = lane; j < entries; j += TEAM) {
                const int c = d.t_class[row * d.top + j];
                if (!bad_class(c, d.V)) repeated |= own[c] != (uint16_t)j;
            }
            constexpr uint64_t kMask = TEAM == 64 ? ~0ull : (1ull << (TEAM & 63)) - 1;
            repeated = (__ballot(repeated) >> ((threadIdx.x & 63) / TEAM * TEAM) & kMask) != 0;
        }
        for (int j0 = 0; j0 <= entries; j0 += TEAM) {
            const int j = j0 + lane;
            const int c = j < entries ? d.t_class[row * d.top + j]
                                      : (j == entries && w.ce != 0.f ? w.label : -1);
            const bool have = !bad_class(c, d.V);
            const float zc = have ? pv_load_one(d.z.p, BF16, row * d.z.ld + c) : 0.f;
            const float u = have && j < entries ? (d.t_val[row * d.top + j] - tmax) * a.tau : 0.f;
            float p = have && j < entries ? __expf(u) * tinv : 0.f;
            if (STATS && have && j < entries && !empty && !(p == 0.f))
                kl += p * (u - log_of(tsum) - fmaf(zc, a.tau, -lset));
            if (GRAD && have && !zero && live) {
                bool mine = true;
                if (repeated) {
                    p = 0.f;
                    for (int i = 0; i < entries; i++)
                        if (d.t_class[row * d.top + i] == c)
                            p += __expf((d.t_val[row * d.top + i] - tmax) * a.tau);
                    p *= tinv;
                } else if (j == entries && entries) {
                    // the label's class, unless an entry of that class writes it
                    const int o = own[c];
                    mine = !(o < entries && d.t_class[row * d.top + o] == c);
                }
                float g = soft_grad(zc, a, w, lse1, lset);
                if (entries) g -= w.kl * p;
                if (w.ce != 0.f && c == w.label) g -= w.ce;
                if (mine) pv_store_one(a.dz.p, a.dz.bf16, row * a.dz.ld + c, scale * g);
            }
        }
        if constexpr (STATS) {
            kl = lanes_reduce<TEAM>(kl, Add());
            if (lane == 0 && live) {
                float l = 0.f;
                if (!empty) {
                    l = w.kl * d.temperature * kl;
                    if (w.ce != 0.f)
                        l += w.ce * (lse1 - pv_load_one(d.z.p, BF16, row * d.z.ld + w.label));
                }
                a.loss[row] = l;
                if (a.lse) {
                    a.lse[2 * row] = lse1;
                    a.lse[2 * row + 1] = lset;
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Many classes: a workgroup of T threads a row, 16-byte vectors from the row's
// first 16-byte boundary on, the elements before and after one a thread. Rows
// of z and dz rarely share that boundary (an odd number of classes): the pass
// that reads alone goes by z's, the pass that writes by dz's.
// 4096 x 49999, top 64, bf16: loss 104 us (3.9 TB/s; the SIMDs issue vector
// instructions in 93 % of the cycles), gradient 197 (4.2 TB/s, 50 %); both in one call 226.
// ---------------------------------------------------------------------------
constexpr int kAhead = 4;  // vectors in flight a thread

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));  // at any element

template <bool BF16>
struct Vec {
    static constexpr int N = BF16 ? 8 : 4;
    u32x4 w;
    __device__ __forceinline__ float get(int i) const {
        const uint32_t u = w[BF16 ? i / 2 : i];
        return __uint_as_float(BF16 ? (i & 1 ? u & 0xffff0000u : u << 16) : u);
    }
};

// Where a row's vectors lie: on the 16-byte boundaries of `by` (es bytes an
// element).
template <bool BF16>
struct RowSpan {
    const char* p;
    int head, vecs, tail;  // elements, vectors, elements
    __device__ RowSpan(const PvRows& x, size_t row, int V, const void* by, int es) {
        p = (const char*)x.p + row * x.ld * (BF16 ? 2 : 4);
        head = min((int)((16 - ((uintptr_t)by & 15)) & 15) / es, V);
        vecs = (V - head) / Vec<BF16>::N;
        tail = V - head - vecs * Vec<BF16>::N;
    }
    // OWN: the boundaries are the row's own. ONCE: past the caches' normal order
    // (streams() has the rule).
    template <bool OWN, bool ONCE = false>
    __device__ __forceinline__ Vec<BF16> vec(int i) const {
        const char* q = p + head * (BF16 ? 2 : 4) + (size_t)i * 16;
        if constexpr (OWN && ONCE)
            return {__builtin_nontemporal_load((const u32x4*)q)};
        else if constexpr (OWN)
            return {*(const u32x4*)q};
        else
            return {*(const u32x4_any*)q};
    }
    __device__ __forceinline__ int first(int i) const { return head + i * Vec<BF16>::N; }
    // the element that this thread takes beside the vectors, or -1
    __device__ __forceinline__ int odd(int t) const {
        if (t < head) return t;
        const int u = t - head;
        return u < tail ? head + vecs * Vec<BF16>::N + u : -1;
    }
};

// Running maximum and sums of a thread.
struct Running {
    float m = -INFINITY, s1 = 0.f, st = 0.f;
    __device__ __forceinline__ void raise(float to, const Args& a) {
        if (to > m) {
            const float e = m - to;
            s1 *= __expf(e);
            st *= __expf(e * a.tau);
            m = to;
        }
    }
    __device__ __forceinline__ void add(float z, const Args& a) {
        // -inf - -inf is no number: a row that starts with -inf
        const float e = z == -INFINITY ? -INFINITY : z - m;
        if (a.hard) s1 += __expf(e);
        if (a.soft) st += __expf(e * a.tau);
    }
};

template <int T, typename Op>
__device__ __forceinline__ float group_reduce(float v, Op op, float* lds) {
    v = lanes_reduce<64>(v, op);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < T / 64; w++) v = op(v, lds[w]);
    return v;
}

template <int T, bool BF16, bool STATS, bool GRAD, bool ONCE>
__global__ __launch_bounds__(T) void pv_distill_long_kernel(Args a) {
    __shared__ float lds[T / 64];
    __shared__ float ep[PVCONV_MAX_TOP];  // exp of the entries
    __shared__ int ec[PVCONV_MAX_TOP];    // their classes, -1 for an absent one
    const PvDistill& d = a.d;
    const int t = threadIdx.x;
    for (size_t row = blockIdx.x; row < (size_t)d.M; row += gridDim.x) {
        constexpr int zs = BF16 ? 2 : 4;
        const RowSpan<BF16> r(d.z, row, d.V, (const char*)d.z.p + row * d.z.ld * zs, zs);
        Terms w{0.f, 0.f, d.labels ? d.labels[row] : -1};
        if (a.hard && !bad_class(w.label, d.V)) w.ce = 1.f - d.alpha;
        // a thread an entry (T >= PVCONV_MAX_TOP)
        const bool mine = a.soft && t < d.top && !bad_class(d.t_class[row * d.top + t], d.V);
        const int c_mine = mine ? d.t_class[row * d.top + t] : -1;
        const float v_mine = mine ? d.t_val[row * d.top + t] : -INFINITY;

        float lse1 = 0.f, lset = 0.f;
        bool empty;
        if constexpr (STATS) {
            Running s;
            for (int i = t; i < r.vecs; i += T * kAhead) {
                Vec<BF16> v[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; u++) v[u] = r.template vec<true, ONCE>(min(i + u * T, r.vecs - 1));
                float m = -INFINITY;
#pragma unroll
                for (int u = 0; u < kAhead; u++)
#pragma unroll
                    for (int k = 0; k < Vec<BF16>::N; k++) m = fmaxf(m, v[u].get(k));
                s.raise(m, a);
#pragma unroll
                for (int u = 0; u < kAhead; u++)
                    if (i + u * T < r.vecs) {
#pragma unroll
                        for (int k = 0; k < Vec<BF16>::N; k++) s.add(v[u].get(k), a);
                    }
            }
            const int odd = r.odd(t);
            if (odd >= 0) {
                const float z = pv_load_one(r.p, BF16, odd);
                s.raise(z, a);
                s.add(z, a);
            }
            const float m = group_reduce<T>(s.m, Max(), lds);
            const float e = s.m == -INFINITY ? -INFINITY : s.m - m;
            const float s1 = a.hard ? group_reduce<T>(s.s1 * __expf(e), Add(), lds) : 0.f;
            const float st = a.soft ? group_reduce<T>(s.st * __expf(e * a.tau), Add(), lds) : 0.f;
            empty = is_empty(m, s1, st, a);
            if (a.hard) lse1 = m + log_of(s1);
            if (a.soft) lset = m * a.tau + log_of(st);
        } else {
            lse1 = a.lse[2 * row];
            lset = a.lse[2 * row + 1];
            empty = lse1 == -INFINITY || lset == -INFINITY;
        }

        float p = 0.f, tsum = 0.f, tmax = 0.f;
        if (a.soft) {
            tmax = group_reduce<T>(v_mine, Max(), lds);
            if (tmax == -INFINITY) tmax = 0.f;
            p = mine ? __expf((v_mine - tmax) * a.tau) : 0.f;
            tsum = group_reduce<T>(p, Add(), lds);
            if (!(tsum == 0.f)) w.kl = d.alpha * d.temperature;
        }
        const float tinv = 1.f / tsum;
        if constexpr (STATS) {
            float kl = 0.f;
            if (mine && w.kl != 0.f && !empty && !(p * tinv == 0.f))
                kl = p * tinv * ((v_mine - tmax) * a.tau - log_of(tsum) -
                                 fmaf(pv_load_one(r.p, BF16, c_mine), a.tau, -lset));
            kl = group_reduce<T>(kl, Add(), lds);
            if (t == 0) {
                float l = 0.f;
                if (!empty) {
                    l = w.kl * d.temperature * kl;
                    if (w.ce != 0.f) l += w.ce * (lse1 - pv_load_one(r.p, BF16, w.label));
                }
                a.loss[row] = l;
                if (a.lse) {
                    a.lse[2 * row] = lse1;
                    a.lse[2 * row + 1] = lset;
                }
            }
        }
        if constexpr (GRAD) {
            const float scale = a.weight ? a.weight[row] : 1.f;
            const bool zero = scale == 0.f || empty;
            const int es = a.dz.bf16 ? 2 : 4;
            char* out = (char*)a.dz.p + row * a.dz.ld * es;
            const RowSpan<BF16> o(d.z, row, d.V, out, es);
            for (int i = t; i < o.vecs; i += T * kAhead) {
                Vec<BF16> v[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; u++) v[u] = o.template vec<false>(min(i + u * T, o.vecs - 1));
#pragma unroll
                for (int u = 0; u < kAhead; u++) {
                    if (i + u * T >= o.vecs) continue;
                    float g[Vec<BF16>::N];
#pragma unroll
                    for (int k = 0; k < Vec<BF16>::N; k++)
                        g[k] = scale * soft_grad(v[u].get(k), a, w, lse1, lset);
                    if (zero)
#pragma unroll
                        for (int k = 0; k < Vec<BF16>::N; k++) g[k] = 0.f;
                    char* to = out + (size_t)o.first(i + u * T) * es;
                    if (a.dz.bf16) {
                        uint32_t q[Vec<BF16>::N / 2];
#pragma unroll
                        for (int k = 0; k < Vec<BF16>::N / 2; k++)
                            q[k] = pv_pack_bf16x2(g[2 * k], g[2 * k + 1]);
                        if constexpr (BF16)
                            *(uint4*)to = make_uint4(q[0], q[1], q[2], q[3]);
                        else  // 4 of fp32 logits: 8 bytes
                            *(uint2*)to = make_uint2(q[0], q[1]);
                    } else {
#pragma unroll
                        for (int k = 0; k < Vec<BF16>::N; k += 4)
                            ((float4*)to)[k / 4] = make_float4(g[k], g[k + 1], g[k + 2], g[k + 3]);
                    }
                }
            }
            const int odd = o.odd(t);
            if (odd >= 0)
                pv_store_one(out, a.dz.bf16, odd,
                             zero ? 0.f
                                  : scale * soft_grad(pv_load_one(r.p, BF16, odd), a, w, lse1,
                                                      lset));
            // the classes of the entries and of the label take their whole value
            // from the thread of the entry, after the stores above
            if (t < PVCONV_MAX_TOP) {
                ec[t] = c_mine;
                ep[t] = p;
            }
            __syncthreads();
            const int c = t < d.top ? c_mine : (t == d.top && w.ce != 0.f ? w.label : -1);
            if (!zero && c >= 0) {
                float sum = 0.f;
                if (w.kl != 0.f)
                    for (int i = 0; i < d.top; i++) sum += ec[i] == c ? ep[i] : 0.f;
                float g = soft_grad(pv_load_one(r.p, BF16, c), a, w, lse1, lset);
                if (w.kl != 0.f) g -= w.kl * sum * tinv;
                if (w.ce != 0.f && c == w.label) g -= w.ce;
                pv_store_one(out, a.dz.bf16, c, scale * g);
            }
            // (the next row's first reduction is a barrier before ec is written)
        }
    }
}

// ---------------------------------------------------------------------------
// Rows of up to 2048 classes stay in registers, with as many lanes as leave each
// 4 to 32 logits (the loss over 80 MB of fp32 logits, 16 lanes / the rule: 13
// classes 204 / 72 us, 50 classes 57 / 38; 1500 classes 74 / 27 against a workgroup
// a row). From kLongV on a workgroup owns a row: 256 threads (2500 classes, loss
// and gradient: 76 us with 512, 43), 512 from kMidV on (49999: loss 133 us, 124),
// 1024 where rows are too few to fill the chip.
constexpr int kLongV = 2049, kFewRows = 512, kWideV = 8192, kMidV = 32768;

template <typename F>
void with_bool(bool b, F f) {
    if (b)
        f(std::true_type());
    else
        f(std::false_type());
}

template <int N>
using Int = std::integral_constant<int, N>;

// Whether a loss alone reads z past the caches' normal order: where z is more than
// the Infinity Cache holds, so that neither what wrote it nor the gradient that
// follows shares it (us, streaming / not, of a z that was just written: 8192 x 5000
// bf16, 82 MB, 31 / 27, with the gradient's call 66 / 58; 2048 x 49999, 205 MB, 42 / 38;
// 4096 x 49999, 410 MB, 77 / 100, with the gradient's call 237 / 273).
bool streams(const PvDistill& d) {
    return (size_t)d.M * d.V * (d.z.bf16 ? 2 : 4) >= (size_t)256 << 20;
}

template <bool STATS, bool GRAD>
pvconv_status launch(const Args& a, hipStream_t s) {
    const size_t M = a.d.M;
    auto grid = [](size_t n) { return (unsigned)(n < (1u << 18) ? n : 1u << 18); };
    with_bool(a.d.z.bf16, [&](auto B) {
        constexpr bool BF16 = decltype(B)::value;
        if (a.d.V >= kLongV) {
            auto wide = [&](auto T, auto O) {
                constexpr int THREADS = decltype(T)::value;
                pv_distill_long_kernel<THREADS, BF16, STATS, GRAD, decltype(O)::value>
                    <<<grid(M), THREADS, 0, s>>>(a);
            };
            auto rows = [&](auto T) {
                if constexpr (STATS && !GRAD) {
                    if (streams(a.d)) {
                        wide(T, std::true_type());
                        return;
                    }
                }
                wide(T, std::false_type());
            };
            if (M <= kFewRows && a.d.V >= kWideV)
                rows(Int<1024>());
            else if (a.d.V < kMidV && a.d.top < 256)  // (a thread an entry and one for the label)
                rows(Int<256>());
            else
                rows(Int<512>());
        } else {
            auto rows = [&](auto T, auto E) {
                constexpr int TEAM = decltype(T)::value;
                pv_distill_short_kernel<TEAM, decltype(E)::value, BF16, STATS, GRAD>
                    <<<grid((M + kThreads / TEAM - 1) / (kThreads / TEAM)), kThreads, 0, s>>>(a);
            };
            const int V = a.d.V;
            if (V <= 16)
                rows(Int<4>(), Int<4>());
            else if (V <= 64)
                rows(Int<8>(), Int<8>());
            else if (V <= 128)
                rows(Int<16>(), Int<8>());
            else if (V <= 256)
                rows(Int<16>(), Int<16>());
            else if (V <= 512)
                rows(Int<64>(), Int<8>());
            else if (V <= 1024)
                rows(Int<64>(), Int<16>());
            else
                rows(Int<64>(), Int<32>());
        }
    });
    return pv_launch_status();
}

}  // namespace

pvconv_status pv_launch_distill(const PvDistill& d, const float* row_weight, float* loss,
                                float* lse, const PvRows& dz, hipStream_t s) {
    const Args a{d, 1.f / d.temperature, d.alpha > 0.f, d.labels && d.alpha < 1.f, row_weight, loss,
                 lse, dz};
    return dz.p ? launch<true, true>(a, s) : launch<true, false>(a, s);
}

pvconv_status pv_launch_distill_bwd(const PvDistill& d, const float* lse, const float* dloss,
                                    const PvRows& dz, hipStream_t s) {
    const Args a{d, 1.f / d.temperature, d.alpha > 0.f, d.labels && d.alpha < 1.f, dloss, nullptr,
                 (float*)lse, dz};
    return launch<false, true>(a, s);
}
