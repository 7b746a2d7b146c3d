// Linear layer in 8-bit integers, a scale for each row of x and of the weight, and
// its gradients from the quantised rows (pvconv_train.h).
//
// With s the scale of a row, the smallest bf16 number with 127 s >= its largest
// magnitude, and q = round(v / s): out[m][n] = act(s_m s_n sum_k q[m][k] q[n][k] +
// bias_n). The integer sums are exact, s_m s_n (16 bits) too: a result is rounded
// when the sum becomes a float, by its scale, its bias and its type.
//
// Two launches, the quantiser and the product (pv_product.h), but for few rows. The scale
// of a row needs the whole row before its first product: 32768 x 4928 -> 256, bf16, is 101
// us at 4.8 TB/s and 47 us of product, which reads the 161 MB of bytes twice over its
// columns; x alone would take 51. (One launch whose workgroups keep the bytes of 16 or 32
// such rows in LDS has not been tried.) 32768 x 512 -> 2048: 13 + 57, 134 MB written at 2.3
// TB/s behind four slices of products.
//
// The gradients are products of bf16 parts, from the bytes and scales that the forward
// kept: with bf16 dy, dx takes dy as it lies by the weight times its scales (15 bits, two
// parts), dw takes dy s in the two parts that hold its 16 bits. 32768 x 2304
// -> 512: operands 76 us (4.4 TB/s), dx 185 (two parts: 0.83 PFLOP/s), dw 191 (0.81).
#include "pv_product.h"
#include "pv_wave.h"

namespace {

constexpr int kThreads = 256;

// The row's scale from its largest magnitude's bits; NaN where a value is not finite.
__device__ __forceinline__ float row_scale_of(uint32_t top) {
    if (top >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    const float a = __uint_as_float(top);
    // a / 127 cut to eight bits, the next such number where 127 times it (fifteen
    // bits: exact) falls short
    uint32_t s = __float_as_uint(fmaxf(a / 127.f, 0x1p-126f)) & 0xffff0000u;
    if (127.f * __uint_as_float(s) < a) s += 0x10000u;
    return __uint_as_float(s);
}

// q = the whole number nearest to v / s, ties to even, as the low byte of the result.
// v * inv is off by less than one step; the remainder v - q s is exact (q s has fifteen
// bits), so that comparing it with s / 2 settles every border.
__device__ __forceinline__ uint32_t quantise(float v, float s, float inv, float half) {
    const float t = __builtin_fmaf(v, inv, 0x1.8p23f);  // rounds to a whole number
    const float e = __builtin_fmaf(-(t - 0x1.8p23f), s, v);
    uint32_t q = __float_as_uint(t);
    if (__builtin_fabsf(e) >= half && (__builtin_fabsf(e) > half || (q & 1u)))
        q += e > 0.f ? 1u : ~0u;
    return q & 255u;
}

struct MaxBits {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const {
        return max(a, b);
    }
};

// Eight consecutive values as they lie in memory.
template <bool XB>
struct Raw {
    pv_u32x4 w[XB ? 1 : 2];
    __device__ __forceinline__ float get(int i) const {
        if constexpr (XB)
            return __uint_as_float(i & 1 ? w[0][i / 2] & 0xffff0000u : w[0][i / 2] << 16);
        else
            return __uint_as_float(w[i / 4][i % 4]);
    }
    __device__ __forceinline__ void load(const PvRows& x, size_t row, int c0, int K) {
        const char* p = (const char*)x.p + (row * x.ld + c0) * (XB ? 2 : 4);
        if (c0 + 8 <= K) {
            w[0] = *(const pv_u32x4_any*)p;
            if constexpr (!XB) w[1] = *(const pv_u32x4_any*)(p + 16);
            return;
        }
        uint32_t e[8];
#pragma unroll
        for (int i = 0; i < 8; i++)
            e[i] = c0 + i < K ? (XB ? (uint32_t)((const uint16_t*)p)[i] : ((const uint32_t*)p)[i])
                              : 0u;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if constexpr (XB) {
                w[0][i] = e[2 * i] | (e[2 * i + 1] << 16);
            } else {
                w[0][i] = e[i];
                w[1][i] = e[4 + i];
            }
        }
    }
    // the largest magnitude's bits, as a float's
    __device__ __forceinline__ uint32_t top() const {
        if constexpr (XB) {
            typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
            u16x2 m = {0, 0};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t u = w[0][i] & 0x7fff7fffu;
                u16x2 v;
                __builtin_memcpy(&v, &u, 4);
                m = __builtin_elementwise_max(m, v);
            }
            return (uint32_t)(m[0] > m[1] ? m[0] : m[1]) << 16;
        } else {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; i++) m = max(m, w[i / 4][i % 4] & 0x7fffffffu);
            return m;
        }
    }
    __device__ __forceinline__ uint2 bytes(float s, float inv, float half) const {
        float t[8], far = 0.f;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            t[i] = __builtin_fmaf(get(i), inv, 0x1.8p23f);
            far = fmaxf(far, __builtin_fabsf(__builtin_fmaf(-(t[i] - 0x1.8p23f), s, get(i))));
        }
        uint32_t q[8];
#pragma unroll
        for (int i = 0; i < 8; i++) q[i] = __float_as_uint(t[i]);
        if (far >= half) {  // a border, or a quotient that rounded across one
#pragma unroll
            for (int i = 0; i < 8; i++) q[i] = quantise(get(i), s, inv, half);
        }
        // the low bytes of the eight
        const uint32_t a = __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u),
                       b = __builtin_amdgcn_perm(q[3], q[2], 0x0c0c0400u),
                       c = __builtin_amdgcn_perm(q[5], q[4], 0x0c0c0400u),
                       d = __builtin_amdgcn_perm(q[7], q[6], 0x0c0c0400u);
        return uint2{a | (b << 16), c | (d << 16)};
    }
};

// Where bytes go: rows of whole blocks, or (a product's own copy) block by block, each
// block of all rows, so that the rows which a product reads at a time lie side by side:
// 128 bytes of rows 5 KB apart came from memory at 2.6 TB/s.
struct Layout {
    size_t row, block;
    __device__ __forceinline__ size_t at(size_t r, int c) const {
        return r * row + (size_t)(c / kSlice) * block + c % kSlice;
    }
};

// A row in the registers of a wave or of the workgroup (TEAM lanes, V vectors of eight a
// lane); of a longer one the rest is read twice. Bound by memory, next by some ten
// instructions a value.
template <bool XB, int TEAM, int V>
__global__ __launch_bounds__(kThreads) void pv_int8_quantise_kernel(PvRows x, int M, int K,
                                                                    int8_t* q, float* scale,
                                                                    Layout to) {
    __shared__ uint32_t tops[kThreads / 64];
    const int K128 = (K + kSlice - 1) / kSlice * kSlice, lane = threadIdx.x % TEAM;
    constexpr int kRows = kThreads / TEAM;
    for (size_t row0 = (size_t)blockIdx.x * kRows; row0 < (size_t)M;
         row0 += (size_t)gridDim.x * kRows) {
        const size_t row = row0 + threadIdx.x / TEAM;
        const bool live = row < (size_t)M;
        Raw<XB> v[V];
        uint32_t top = 0;
        if (live) {
#pragma unroll
            for (int u = 0; u < V; u++)
                if (u * TEAM * 8 < K) v[u].load(x, row, (u * TEAM + lane) * 8, K);
#pragma unroll
            for (int u = 0; u < V; u++)
                if (u * TEAM * 8 < K) top = max(top, v[u].top());
            for (int c0 = (V * TEAM + lane) * 8; c0 < K; c0 += TEAM * 8) {
                Raw<XB> w;
                w.load(x, row, c0, K);
                top = max(top, w.top());
            }
        }
        top = wave_reduce(top, MaxBits());
        if constexpr (TEAM > 64) {
            tops[threadIdx.x >> 6] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kThreads / 64; w++) top = max(top, tops[w]);
            __syncthreads();
        }
        if (!live) continue;
        const float s = row_scale_of(top);
        if (lane == 0) scale[row] = s;
        const float inv = 1.f / s, half = 0.5f * s;
        if (!(s == s)) {  // a row that is not finite
            for (int c0 = lane * 8; c0 < K128; c0 += TEAM * 8)
                *(uint2*)(q + to.at(row, c0)) = uint2{0, 0};
            continue;
        }
#pragma unroll
        for (int u = 0; u < V; u++) {
            const int c0 = (u * TEAM + lane) * 8;
            if (c0 < K)
                *(uint2*)(q + to.at(row, c0)) = v[u].bytes(s, inv, half);
            else if (c0 < K128)
                *(uint2*)(q + to.at(row, c0)) = uint2{0, 0};
        }
        for (int c0 = (V * TEAM + lane) * 8; c0 < K128; c0 += TEAM * 8) {
            Raw<XB> w;
            w.load(x, row, c0, K);
            *(uint2*)(q + to.at(row, c0)) = w.bytes(s, inv, half);
        }
    }
}

// act of a layer: what is not a number stays so
__device__ __forceinline__ float activate(float v, float neg, bool relu) {
    return v < 0.f ? (relu ? 0.f : v * neg) : v;
}

struct LinearEpi {
    const float* row_scale;
    const float* col_scale;
    const float* bias;
    PvRows out;
    float neg;
    bool relu;
    // acc s_m s_n + b, the same operations wherever it is formed: kept rows give the
    // bits of the call that quantised them. The scales' product is exact unless it
    // leaves the 32-bit range.
    __device__ __forceinline__ static bool tame(float s) { return s >= 0x1p-60f && s <= 0x1p60f; }
    __device__ __forceinline__ static float value(int acc, float sm, float sn, float b,
                                                  bool fast) {
        if (fast) return __builtin_fmaf((float)acc, sm * sn, b);
        return (float)((double)acc * ((double)sm * (double)sn) + (double)b);
    }
    template <int MI>
    __device__ __forceinline__ void tile(const PvProduct& p, int mw, int nw, int lane,
                                         const pv_i32x4 (&acc)[4][MI]) const {
        const int r = lane & 15, nb = nw + 8 * (lane >> 4);
        float sn[16], b[16], sms[MI];
#pragma unroll
        for (int i = 0; i < MI; i++) sms[i] = row_scale[min(mw + 16 * i + r, p.M - 1)];
        pv_load_columns(col_scale, nb, p.N, 1.f, sn);
        pv_load_columns(bias, nb, p.N, 0.f, b);
        bool fast = true;
#pragma unroll
        for (int q = 0; q < 16; q++) fast = fast && tame(sn[q]);
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const int m = mw + 16 * i + r;
            if (m >= p.M) continue;
            const float sm = sms[i];
            float v[16];
            if (fast && tame(sm)) {
#pragma unroll
                for (int q = 0; q < 16; q++)
                    v[q] = value(acc[q >> 2][i][q & 3], sm, sn[q], b[q], true);
            } else {
#pragma unroll
                for (int q = 0; q < 16; q++)
                    v[q] = value(acc[q >> 2][i][q & 3], sm, sn[q], b[q],
                                 tame(sm) && tame(sn[q]));
            }
#pragma unroll
            for (int q = 0; q < 16; q++) v[q] = activate(v[q], neg, relu);
            pv_store_runs(out, m, nb, p.N, v);
        }
    }
    __device__ __forceinline__ void one(int m, int n, int acc) const {
        const float sm = row_scale[m], sn = col_scale[n];
        const float v = value(acc, sm, sn, bias ? bias[n] : 0.f, tame(sm) && tame(sn));
        pv_store_one(out.p, out.bf16, (size_t)m * out.ld + n, activate(v, neg, relu));
    }
};

// Few rows: a workgroup takes 16 rows by 16 columns. Its 8 or 16 waves take the rows'
// largest values, then a share of the 64-value pieces each, which a wave quantises in
// registers where they are its matrix operand: lane (r, h) holds row r's values 16 h ..
// of a piece. Their sums meet in LDS; one launch, no workspace. Latency: a wave's first
// pieces are under way while the rows' scales are found.
template <bool XB, int THREADS>
__global__ __launch_bounds__(THREADS) void pv_int8_few_kernel(PvRows x, int M, int K, int N,
                                                              const int8_t* w, LinearEpi epi,
                                                              int8_t* keep, float* keep_scale) {
    // pieces under way: as many as registers hold
    constexpr int kWaves = THREADS / 64, kAhead = XB || THREADS < 1024 ? 4 : 3;
    __shared__ uint32_t tops[16];
    __shared__ int part[kWaves][256];
    const int K128 = (K + kSlice - 1) / kSlice * kSlice, pieces = (K + 63) / 64;
    const int nt = (N + 15) / 16;
    const int m0 = (int)(blockIdx.x / nt) * 16, n0 = (int)(blockIdx.x % nt) * 16;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, h = lane >> 4;
    const int rows = min(16, M - m0);
    const size_t row = min(m0 + r, M - 1);
    const int8_t* gw = w + (size_t)min(n0 + r, N - 1) * K128 + h * 16;
    pv_i32x4 fw[kAhead];
    Raw<XB> v[kAhead][2];
    auto load = [&](int k) {
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            const int at = min(k + u * kWaves, pieces - 1) * 64;
            fw[u] = *(const pv_i32x4*)(gw + at);
            v[u][0].load(x, row, at + h * 16, K);
            v[u][1].load(x, row, at + h * 16 + 8, K);
        }
    };
    load(wave);
    if (threadIdx.x < 16) tops[threadIdx.x] = 0;
    __syncthreads();
    const int chunks = (K + 511) / 512;
    for (int u0 = wave; u0 < rows * chunks; u0 += kWaves * kAhead) {
        uint32_t top[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            const int at = u0 + u * kWaves, i = at / chunks, c0 = (at - i * chunks) * 512 + lane * 8;
            top[u] = 0;
            if (i < rows && c0 < K) {
                Raw<XB> t;
                t.load(x, m0 + i, c0, K);
                top[u] = t.top();
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            const int i = (u0 + u * kWaves) / chunks;
            const uint32_t most = wave_reduce(top[u], MaxBits());
            if (lane == 0 && i < rows) atomicMax(&tops[i], most);  // whole numbers: no order
        }
    }
    __syncthreads();
    const float s = row_scale_of(tops[r]);
    const bool finite = s == s;
    const float inv = 1.f / s, half = 0.5f * s;
    // the first workgroup of a row of tiles keeps its rows, if they are wanted
    int8_t* kept = keep && n0 == 0 && r < rows ? keep + row * K128 + h * 16 : nullptr;
    if (kept && wave == 0) {
        if (h == 0) keep_scale[row] = s;
        if (pieces * 64 < K128) *(pv_i32x4*)(kept + pieces * 64) = pv_i32x4{0, 0, 0, 0};
    }
    pv_i32x4 acc = {0, 0, 0, 0};
    for (int k = wave; k < pieces; k += kWaves * kAhead) {
        if (k != wave) load(k);
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            if (k + u * kWaves >= pieces) break;
            pv_i32x4 fx = {0, 0, 0, 0};
            if (finite) {
                const uint2 a = v[u][0].bytes(s, inv, half), b = v[u][1].bytes(s, inv, half);
                fx = pv_i32x4{(int)a.x, (int)a.y, (int)b.x, (int)b.y};
            }
            if (kept) *(pv_i32x4*)(kept + (k + u * kWaves) * 64) = fx;
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u], fx, acc, 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; i++) part[wave][r * 16 + 4 * h + i] = acc[i];
    __syncthreads();
    const int i = threadIdx.x >> 4, c = threadIdx.x & 15;
    if (threadIdx.x < 256 && i < rows && n0 + c < N) {
        int sum = 0;
#pragma unroll
        for (int u = 0; u < kWaves; u++) sum += part[u][threadIdx.x];
        const float sm = row_scale_of(tops[i]), sn = epi.col_scale[n0 + c];
        const float v = LinearEpi::value(sum, sm, sn, epi.bias ? epi.bias[n0 + c] : 0.f,
                                         LinearEpi::tame(sm) && LinearEpi::tame(sn));
        pv_store_one(epi.out.p, epi.out.bf16, (size_t)(m0 + i) * epi.out.ld + n0 + c,
                     activate(v, epi.neg, epi.relu));
    }
}
// Where its one launch is the shorter call. (us, few / quantiser, product and join: a call of
// many; a replay of a graph, which has no launches to wait for. 1 x 4928 -> 256, fp32: 10.3 /
// 18.3; 9.3 / 10.2. 4 x 8192 -> 256: 16 / 18.3; 16.2 / 10.7; x 12000: 20.9 / 18.5. 16 x 2560 -> 256:
// 12 / 18.1; 12.2 / 9.9; x 4928: 20.5 / 18.2. 256 x 2560 -> 256, 256 workgroups: 12.2 / 18.1; 12.5
// / 11.3. Two a CU, 512 x 323 -> 256: 11.6 / 15; 11.7 / 8.5; 512 x 1024: 15.5 / 15.1; x 1536:
// 17.6 / 15; 4 x 2048 -> 8192: 11.6 / 17.6; x 4096: 20.1 / 18.)
bool few(int M, int K, int N) {
    const size_t tiles = (size_t)((M + 15) / 16) * ((N + 15) / 16);
    if (tiles > 512) return false;
    return K <= (tiles <= 256 ? (M <= 4 ? 8192 : 2560) : M <= 4 ? 2560 : 1024);
}

void run_few(const PvRows& x, int M, int K, int N, const int8_t* weight, const LinearEpi& epi,
             int8_t* rows, float* row_scale, hipStream_t s) {
    const unsigned tiles = (unsigned)((M + 15) / 16 * ((N + 15) / 16));
    auto run = [&](auto kernel, int threads) {
        hipLaunchKernelGGL(kernel, dim3(tiles), dim3(threads), 0, s, x, M, K, N, weight, epi,
                           rows, row_scale);
    };
    if (K > 1024 && tiles <= 256) {  // one workgroup a CU: more waves to share the pieces
        if (x.bf16)
            run(pv_int8_few_kernel<true, 1024>, 1024);
        else
            run(pv_int8_few_kernel<false, 1024>, 1024);
    } else {
        if (x.bf16)
            run(pv_int8_few_kernel<true, 512>, 512);
        else
            run(pv_int8_few_kernel<false, 512>, 512);
    }
}

PvProduct product_of(const int8_t* q, const Layout& rows, int M, int K, const int8_t* w, int N) {
    PvProduct p{};
    p.a = PvPanel{(const uint8_t*)q, rows.row, 0, 1, M, rows.block};
    p.b = PvPanel{(const uint8_t*)w, pv_up(K, kSlice), 0, 1, N, kSlice};
    p.M = M;
    p.N = N;
    p.slices = pv_slices(K, kSlice);
    pv_pairs(p, 1, 1);
    pv_plan(p, true);
    return p;
}

struct LinearWs {
    int8_t* q;
    float* scale;
    uint32_t* partial;
    size_t total;
};
LinearWs carve_linear(void* base, int M, int K, int N, bool rows_given) {
    PvCarve c{(char*)base, 0};
    LinearWs w{nullptr, nullptr, nullptr, 0};
    if (!rows_given) {
        w.q = (int8_t*)c.take((size_t)M * pv_up(K, kSlice));
        w.scale = (float*)c.take((size_t)M * 4);
    }
    w.partial = (uint32_t*)c.take(pv_partial_bytes(product_of(nullptr, Layout{}, M, K, nullptr, N)));
    w.total = c.off;
    return w;
}

// Parts of dx's scaled operand (the weight of a bf16 dy, else dy): the two that hold its 15
// bits where dy is bf16; of an fp32 dy three, for a bf16 result two, which leave 2^-16 of a
// term where the result's rounding is 2^-8. (One rounded part leaves 2^-8 of a term more,
// at whatever number of rows: a row's sum has as many as it has channels, and one of
// them may carry it. The step of 32768 x 2304 -> 512 takes 453 us with it, 535 without.)
int parts_of(bool out_bf16, bool dy_bf16) { return out_bf16 || dy_bf16 ? 2 : 3; }

// dx = dy W: of a bf16 dy as it is by the scaled weight, in parts; of an fp32 one in
// parts, scaled, by the weight's whole numbers. dw = (dy s)^T q.
struct BwdWs {
    PvPanel dys, w, dym, q;
    bool pack_dy;
    PvProduct dx, dw;
    bool pair;  // the two in one launch
    float* sums;
    size_t total;
};
BwdWs carve_bwd(void* base, const PvRows& dy, int M, int K, int N, bool dx_bf16, bool want_dx,
                bool want_dw, bool want_db, bool may_direct) {
    PvCarve c{(char*)base, 0};
    BwdWs w{};
    const int parts = parts_of(dx_bf16, dy.bf16);
    auto plan = [&](PvProduct& p, int parts_a, int parts_b, int rows, int cols, int depth) {
        p.a.parts = parts_a;
        p.b.parts = parts_b;
        p.M = rows;
        p.N = cols;
        p.slices = pv_slices(depth, kDeep);
        pv_pairs(p, parts_a, parts_b);
        pv_plan(p, true);
    };
    plan(w.dx, dy.bf16 ? 1 : parts, dy.bf16 ? parts : 1, M, K, N);
    plan(w.dw, dy.bf16 ? 2 : 3, 1, N, K, M);
    // (dw's plan is that of both, with an fp32 dx, whichever is wanted of whatever type: one
    // gradient alone has the same bits)
    PvProduct most{};
    plan(most, dy.bf16 ? 1 : 3, dy.bf16 ? 2 : 1, M, K, N);
    const int pair = pv_pair_size(most, w.dw);
    if (pair >= 0) pv_take_pair(w.dw, pair);
    w.pair = pair >= 0 && (pair != kPvP || w.dx.a.parts == 3);
    if (w.pair) pv_take_pair(w.dx, pair);
    auto take = [&](PvProduct& p, const PvPanel& a, const PvPanel& b) {
        p.a = a;
        p.b = b;
        p.partial = (uint32_t*)c.take(pv_partial_bytes(p));
    };
    if (want_dx && M > 0) {
        w.pack_dy = !(may_direct && pv_in_place(dy, N));
        w.dys = w.pack_dy ? pv_take_panel(c, M, N, dy.bf16 ? 1 : parts) : pv_panel_of(dy, M);
        w.w = pv_take_panel(c, N, K, dy.bf16 ? parts : 1);
        take(w.dx, w.dys, w.w);
    }
    if (want_dw) {  // both operands across k: dy's rows are padded with zeros
        w.dym = pv_take_panel(c, (int)pv_up(M, kDeep), N, dy.bf16 ? 2 : 3);
        w.q = pv_take_panel(c, M, K, 1);
        take(w.dw, w.dym, w.q);
    }
    if (want_db) w.sums = (float*)c.take((size_t)pv_sum_runs(M) * N * 4);
    w.total = c.off;
    return w;
}

template <bool XB>
void run_quantise(const PvRows& x, int M, int K, int8_t* q, float* scale, const Layout& to,
                  hipStream_t s) {
    auto run = [&](auto kernel, int team) {
        hipLaunchKernelGGL(kernel, dim3(pv_blocks(M, kThreads / team)), dim3(kThreads), 0, s, x, M,
                           K, q, scale, to);
    };
    // A wave a row up to 3584 channels, of which it holds as many as the row has, up to 2560; a
    // workgroup a row of more, and where there are few rows. (us, a wave that holds 512,
    // 1024 or 2560 / a workgroup. bf16, 32768 x 512: 13.5, 14.6, 21 / 54; 1000: 21, 21, 27 / 57;
    // 2560: 47, 46, 48 / 67; 3500: -, 86, 80 / 91; 4096: 100, 100, 88 / 83; 4928: 130, 128, 119 /
    // 101. fp32, 32768 x 2560: 103, 94, 83 / 89; 4096: 172, 164, 137 / 124. bf16, 4096 x 2560: -,
    // 9.3, 10.2 / 13; 1024 x 1100: -, 4.9, 5 / 4.7; x 4928: -, 10.2, 10.2 / 6.8; 256 x 2048: 4.9,
    // 4.9, 5.1 / 3.4.)
    if (K > 3584 || (K > 1024 && M <= 1024))
        run(pv_int8_quantise_kernel<XB, 256, 4>, 256);
    else if (K <= 512)
        run(pv_int8_quantise_kernel<XB, 64, 1>, 64);
    else if (K <= 1024)
        run(pv_int8_quantise_kernel<XB, 64, 2>, 64);
    else
        run(pv_int8_quantise_kernel<XB, 64, 5>, 64);
}

}  // namespace

static pvconv_status quantise_to(const PvRows& x, int M, int K, int8_t* q, float* scale,
                                 const Layout& to, hipStream_t s) {
    if (x.bf16)
        run_quantise<true>(x, M, K, q, scale, to, s);
    else
        run_quantise<false>(x, M, K, q, scale, to, s);
    return pv_launch_status();
}
pvconv_status pv_launch_int8_quantize(const PvRows& x, int M, int K, int8_t* q, float* scale,
                                      hipStream_t s) {
    return quantise_to(x, M, K, q, scale, Layout{pv_up(K, kSlice), kSlice}, s);
}

size_t pv_int8_linear_ws_bytes(int M, int K, int N, bool rows_given) {
    if (!rows_given && few(M, K, N)) return 0;
    return carve_linear(nullptr, M, K, N, rows_given).total;
}

static pvconv_status run_rows(const int8_t* q, const Layout& rows, int M, int K, int N,
                              const int8_t* weight, const LinearEpi& epi, uint32_t* partial,
                              hipStream_t s) {
    PvProduct p = product_of(q, rows, M, K, weight, N);
    p.partial = partial;
    pv_run_product<true, false, false>(p, epi, s);
    pv_run_join<true>(p, epi, s);
    return pv_launch_status();
}

static LinearEpi epi_of(const float* row_scale, const float* weight_scale, const float* bias,
                        int act, float slope, const PvRows& y) {
    return LinearEpi{row_scale, weight_scale, bias, y,
                     act == PVCONV_ACT_LEAKY ? slope : 1.f, act == PVCONV_ACT_RELU};
}

pvconv_status pv_launch_int8_linear(const PvRows& x, int M, int K, int N, const int8_t* weight,
                                    const float* scale, const float* bias, int act, float slope,
                                    const PvRows& y, int8_t* rows, float* row_scale, void* ws,
                                    hipStream_t s) {
    LinearEpi epi = epi_of(row_scale, scale, bias, act, slope, y);
    if (few(M, K, N)) {
        run_few(x, M, K, N, weight, epi, rows, row_scale, s);
        return pv_launch_status();
    }
    const LinearWs w = carve_linear(ws, M, K, N, rows != nullptr);
    Layout to{pv_up(K, kSlice), kSlice};
    if (!rows) {
        to = Layout{kSlice, (size_t)M * kSlice};
        rows = w.q;
        row_scale = w.scale;
        epi.row_scale = w.scale;
    }
    const pvconv_status st = quantise_to(x, M, K, rows, row_scale, to, s);
    if (st != PVCONV_OK) return st;
    return run_rows(rows, to, M, K, N, weight, epi, w.partial, s);
}

pvconv_status pv_launch_int8_linear_rows(const int8_t* rows, const float* row_scale, int M, int K,
                                         int N, const int8_t* weight, const float* scale,
                                         const float* bias, int act, float slope, const PvRows& y,
                                         void* ws, hipStream_t s) {
    const LinearWs w = carve_linear(ws, M, K, N, true);
    return run_rows(rows, Layout{pv_up(K, kSlice), kSlice}, M, K, N, weight,
                    epi_of(row_scale, scale, bias, act, slope, y), w.partial, s);
}

size_t pv_int8_linear_bwd_ws_bytes(int M, int K, int N) {
    size_t most = 0;  // that any of the types takes
    for (int types = 0; types < 4; types++) {
        const PvRows dy{nullptr, (types & 1) != 0, N};
        const size_t n = carve_bwd(nullptr, dy, M, K, N, types & 2, true, true, true, false).total;
        most = most > n ? most : n;
    }
    return most;
}

pvconv_status pv_launch_int8_linear_bwd(const PvRows& dy, const int8_t* rows,
                                        const float* row_scale, int M, int K, int N,
                                        const int8_t* weight, const float* scale,
                                        const PvRows& dx, float* dw, float* dbias, void* ws,
                                        hipStream_t s) {
    const BwdWs w = carve_bwd(ws, dy, M, K, N, dx.bf16, dx.p != nullptr, dw != nullptr,
                              dbias != nullptr, true);
    const PvKind kind = dy.bf16 ? kPvBf16 : kPvF32;
    const size_t qk = pv_up(K, kSlice);
    const bool want_dx = dx.p && M > 0;
    PvPacks packs{};
    if (want_dx) {
        PvPack a = pv_pack_of(dy.p, kind, dy.ld, M, N, w.dys),
               b = pv_pack_of(weight, kPvInt8, qk, N, K, w.w);
        if (dy.bf16)
            b.row_scale = scale;
        else
            a.col_scale = scale;
        if (w.pack_dy) packs.add(a);
        packs.add(b);
    }
    if (dw && M > 0) {
        PvPack a = pv_pack_of(dy.p, kind, dy.ld, M, N, w.dym);
        a.row_scale = row_scale;
        packs.add(a);
        packs.add(pv_pack_of(rows, kPvInt8, qk, M, K, w.q));
    }
    // (sums of one run are whole)
    const int runs = pv_sum_runs(M);
    if (dbias && M > 0) packs.add(pv_sums_of(dy, M, N, runs == 1 ? dbias : w.sums));
    pv_launch_packs(packs, s);
    const PvSums none{nullptr, 0, 0, nullptr},
        sums{w.sums, runs, N, dbias && runs != 1 ? dbias : nullptr};
    const PvPlain to_dx{dx, nullptr}, to_dw{PvRows{dw, false, K}, nullptr};
    if (want_dx && dw && w.pair) {
        pv_launch_pair(w.dx, to_dx, w.dw, to_dw, sums, s);
    } else {
        if (want_dx) pv_launch_plain(w.dx, false, to_dx, dw ? none : sums, s);
        if (dw) pv_launch_plain(w.dw, true, to_dw, sums, s);
        if (!want_dx && !dw) pv_launch_sum_runs(sums, s);
    }
    return pv_launch_status();
}
