// Classification head: logits = fc(mean over pixels of ReLU(BN(x))), forward and backward, in two launches each.
//
// Forward: (1) one workgroup per channel takes the channel's statistics and, with its pixels still in registers, every
// plane's mean of ReLU(z), z = x * scale + shift, the number of positive z and the sum of their xhat = (x - mean) * rstd:
// x is read once; (2) the product with the classifier's weights.
// Backward: (1) the two products of the classifier; (2) BN backward.  Every pixel of a plane receives the same derivative
// g = d_pooled / (h*w), so the sums of BN's backward pass need no pass over x:
//     sum dz = sum_n g_n * count_n,   sum dz * xhat = sum_n g_n * xhat_n
// and one pass reads x and writes dx = scale * ((z > 0 ? g_n : 0) - mean(dz) - xhat * mean(dz * xhat)).
// x is bound by memory: 4 bytes an element forward, 8 backward.  The products are small (n up to a few hundred): bound
// by the latency of their loads, hence one 16x16 tile per workgroup and its reduction split over the wavefronts.
#include <algorithm>

#include "fast_div.h"
#include "kernels.h"
#include "quads.h"

namespace rvn {

namespace {

// ---- pooling ---------------------------------------------------------------------------------------------------

// How a channel's planes fall to wavefronts: 2^tshift lanes share a plane of `per` quads, J of them each; a wavefront takes
// 64 >> tshift planes at a time, `steps` times.
struct Planes {
    int N, C, HW, per, tshift, J, steps;
};

// The sum over the workgroup of a value of each thread, in every thread: wavefronts in fp32, their sums in double.
template <int TH>
__device__ __forceinline__ double block_total(float v, double *lds) {
    const float t = wave_total(v);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = t;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < TH / 64; ++w) s += lds[w];
    return s;
}

// HELD > 0: the channel stays in registers, steps * J <= HELD quads of it in each lane; otherwise it is read three times, the
// second and third mostly from the caches (whole forward pass at 256 x 512 x 14 x 14, 100 classes: 42.2 and 53.7 us).  SINGLE: J == 1, a
// lane has the same quad of every plane of its (256 x 512 x 7 x 7, 1000 classes: 27.1 and 30.8).
// With d = x - mean and the positive pixels of a plane (as z = x * scale + shift says, as in the backward pass), its sum of
// ReLU(z) is scale * sum d + beta * count and that of xhat rstd * sum d: one sum and a count a pixel.  (Instructions of this kernel
// took 21 of its 28 us at 128 x 2048 x 7 x 7 while it formed all three sums pixel by pixel; the whole
// forward pass, with 1000 classes, took 41.6 us then, 35.0 now.  32 x 2048 x 7 x 7: 12.8 MB in 8.0 us.)
template <int TH, int HELD, bool WHOLE, bool SINGLE>
__global__ __launch_bounds__(TH) void head_pool_k(const float *__restrict__ x, int64_t sn, int64_t sc, const Planes g, float eps,
                                                  const float *__restrict__ gamma, const float *__restrict__ beta,
                                                  float *__restrict__ stats, float *__restrict__ pooled, float *__restrict__ count,
                                                  float *__restrict__ xhat) {
    __shared__ float lds[TH / 64][3];
    const int ch = channel_of((int)blockIdx.x, g.C), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
    const int T = 1 << g.tshift, sub = lane & (T - 1), planes = 64 >> g.tshift;
    const float *base = x + (int64_t)ch * sc;
    const QuadAt only = quad_at<WHOLE>(sub, g.HW);
    f4 held[HELD > 0 ? HELD : 1];
    // calls visit(value, whether each pixel is one of the item's own, plane, whether the item is the plane's last) for every item
    // of this lane, in order; a plane's items follow each other
    auto each = [&](bool first, auto visit) {
        int step = 0, j = 0;
        auto item = [&](int k) {
            const int n = (step * (TH / 64) + wave) * planes + (lane >> g.tshift), quad = SINGLE ? sub : j * T + sub;
            const bool live = n < g.N && quad < g.per;
            const QuadAt at = SINGLE ? only : quad_at<WHOLE>(quad, g.HW);
            f4 v = {0.f, 0.f, 0.f, 0.f};
            if (HELD > 0 && !first) v = held[k];
            else if (live) v = fetch4<WHOLE>(base + (int64_t)n * sn, at);
            if (HELD > 0 && first) held[k] = v;
            bool own[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) own[e] = live && (WHOLE || at.owns(e));
            visit(v, own, n, SINGLE || j == g.J - 1);
            if (SINGLE || ++j == g.J) j = 0, ++step;
        };
        if constexpr (HELD > 0) {
            if (first) {  // (all requests before the first use)
#pragma unroll
                for (int k = 0; k < HELD; ++k) {
                    if (step >= g.steps) break;
                    const int n = (step * (TH / 64) + wave) * planes + (lane >> g.tshift), quad = SINGLE ? sub : j * T + sub;
                    held[k] = f4{0.f, 0.f, 0.f, 0.f};
                    if (n < g.N && quad < g.per) held[k] = fetch4<WHOLE>(base + (int64_t)n * sn, SINGLE ? only : quad_at<WHOLE>(quad, g.HW));
                    if (SINGLE || ++j == g.J) j = 0, ++step;
                }
                step = j = 0;
                first = false;
            }
#pragma unroll
            for (int k = 0; k < HELD; ++k)
                if (step < g.steps) item(k);
        } else {
            while (step < g.steps) item(0);
        }
    };
    // mean and squared deviations of every wavefront's pixels, joined over the workgroup in double
    int mine = 0;  // planes of this wavefront
    for (int s = 0; s < g.steps; ++s) mine += min(max(g.N - (s * (TH / 64) + wave) * planes, 0), planes);
    const float here = (float)mine * (float)g.HW;
    float sum = 0.f;
    each(true, [&](f4 v, const bool (&own)[4], int, bool) {
        if (!WHOLE) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = own[e] ? v[e] : 0.f;
        }
        sum += (v.x + v.y) + (v.z + v.w);
    });
    const float wave_mean = mine > 0 ? wave_total(sum) / here : 0.f;
    sum = 0.f;
    each(false, [&](f4 v, const bool (&own)[4], int, bool) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float d = own[e] ? v[e] - wave_mean : 0.f;
            sum = fmaf(d, d, sum);
        }
    });
    sum = wave_total(sum);
    if (lane == 0) lds[wave][0] = here, lds[wave][1] = wave_mean, lds[wave][2] = sum;
    __syncthreads();
    const double m = (double)g.N * g.HW;
    double total = 0.0, m2 = 0.0;
#pragma unroll 4
    for (int w = 0; w < TH / 64; ++w) total += (double)lds[w][0] * lds[w][1];
    const double mean_d = total / m;
#pragma unroll 4
    for (int w = 0; w < TH / 64; ++w) {
        const double d = lds[w][1] - mean_d;
        m2 += lds[w][2] + lds[w][0] * d * d;
    }
    const float mean = (float)mean_d, rstd = 1.f / sqrtf((float)(m2 / m) + eps), center = beta[ch];
    const float scale = gamma[ch] * rstd, shift = fmaf(-mean, scale, center);
    if (threadIdx.x == 0) {
        stats[ch] = mean;
        stats[g.C + ch] = rstd;
        stats[2 * g.C + ch] = scale;
        stats[3 * g.C + ch] = shift;
    }
    const float inv_hw = 1.f / (float)g.HW;
    int pos = 0;
    sum = 0.f;
    each(false, [&](f4 v, const bool (&own)[4], int n, bool last) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool positive = own[e] && !(fmaf(v[e], scale, shift) <= 0.f);  // (a NaN is passed on)
            sum += positive ? v[e] - mean : 0.f;
            pos += positive ? 1 : 0;
        }
        if (!last) return;
        float d = sum, c = (float)pos;
        team_totals(d, c, g.tshift);
        if (sub == 0 && n < g.N) {
            pooled[(int64_t)ch * g.N + n] = fmaf(scale, d, center * c) * inv_hw;
            count[(int64_t)ch * g.N + n] = c;
            xhat[(int64_t)ch * g.N + n] = rstd * d;
        }
        sum = 0.f;
        pos = 0;
    });
}

// dx of a share of a channel's quads; every workgroup forms the channel's two sums for itself.  Bound by memory and, small, by
// latency (32 x 2048 x 7 x 7: 25.7 MB in 7.0 us, 3.7 TB/s).
constexpr int kPoolThreads = 256;

template <bool WHOLE>
__global__ __launch_bounds__(kPoolThreads) void head_pool_bwd_k(const float *__restrict__ x, int64_t sn, int64_t sc, int N, int C, int HW,
                                                                FastDiv by_per, int share, const float *__restrict__ stats,
                                                                const float *__restrict__ count, const float *__restrict__ xhat,
                                                                const float *__restrict__ d_pooled, float *dgamma, float *dbeta,
                                                                int accumulate, float *__restrict__ dx, int64_t osn, int64_t osc) {
    __shared__ double lds[2][kPoolThreads / 64];
    const int ch = channel_of((int)blockIdx.y, C), per = (int)by_per.d, total = N * per;
    const float mean = stats[ch], rstd = stats[C + ch], scale = stats[2 * C + ch], shift = stats[3 * C + ch];
    const float inv_hw = 1.f / (float)HW;
    const float *g = d_pooled + (int64_t)ch * N, *cnt = count + (int64_t)ch * N, *hat = xhat + (int64_t)ch * N;
    float a0 = 0.f, a1 = 0.f;
    for (int n = (int)threadIdx.x; n < N; n += kPoolThreads) {
        const float gn = g[n] * inv_hw;
        a0 = fmaf(gn, cnt[n], a0);
        a1 = fmaf(gn, hat[n], a1);
    }
    const double sb = block_total<kPoolThreads>(a0, lds[0]), sg = block_total<kPoolThreads>(a1, lds[1]);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        dbeta[ch] = (accumulate ? dbeta[ch] : 0.f) + (float)sb;
        dgamma[ch] = (accumulate ? dgamma[ch] : 0.f) + (float)sg;
    }
    const double inv_m = 1.0 / ((double)N * HW);
    const float c1 = (float)(sb * inv_m), c2 = (float)(sg * inv_m);
    const int last = min(total, ((int)blockIdx.x + 1) * share);
    for (int e = (int)blockIdx.x * share + (int)threadIdx.x; e < last; e += kPoolThreads) {
        const int n = quotient(e, by_per);
        const QuadAt at = quad_at<WHOLE>(e - n * per, HW);
        const f4 v = fetch4<WHOLE>(x + (int64_t)n * sn + (int64_t)ch * sc, at);
        const float gn = g[n] * inv_hw;
        f4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float dz = fmaf(v[j], scale, shift) > 0.f ? gn : 0.f;
            r[j] = scale * ((dz - c1) - ((v[j] - mean) * rstd) * c2);
        }
        store4<WHOLE>(dx + (int64_t)n * osn + (int64_t)ch * osc, at, r);
    }
}

// ---- products on v_mfma_f32_16x16x4_f32 -----------------------------------------------------------------------
// Lane l holds row (or column) l % 16 of an operand at reduction index l / 16 and, of the result, column l % 16 of rows
// (l / 16) * 4 .. + 3.  Which reduction index stands at which place is free as long as both operands agree.

// An operand of 16 rows (or columns): row r at p + r * ld where its reduction index runs along memory, else index k at
// p + k * ld; rows beyond `count` are taken for the last one.
template <bool ALONG>
struct Operand {
    const float *p;
    int64_t ld;
    // first: the first of the 16 rows of the matrix
    __device__ __forceinline__ Operand(const float *m, int64_t l, int first, int count) : ld(l) {
        const int lane = (int)threadIdx.x & 63;
        p = ALONG ? m + (int64_t)min(first + (lane >> 2), count - 1) * l + (lane & 3) * 4 : m + min(first + (lane & 15), count - 1);
    }
    // What the lane reads for reduction indices k .. k + 15.  Across memory that is its own four values, with 16 lanes side by
    // side; along memory, where the rows are far apart, four lanes read 64 bytes of a row together (lane by lane in the order
    // of the rows each would be an access of its own: 62 cycles an instruction).  FULL: k + 16 <= k1; else what lies at or
    // behind k1 reads as zero.
    template <bool FULL>
    __device__ __forceinline__ f4 fetch(int k, int k1) const {
        const int lane = (int)threadIdx.x & 63;
        f4 v = {0.f, 0.f, 0.f, 0.f};
        if (ALONG) {
            if (FULL) return *reinterpret_cast<const f4_any *>(p + k);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = k + (lane & 3) * 4 + e < k1 ? p[k + e] : 0.f;
        } else {
            const int mine = k + (lane >> 4) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = FULL || mine + e < k1 ? p[(mine + e) * ld] : 0.f;
        }
        return v;
    }
    // The lane's own four values from what was fetched; lds: kTurn floats of the wavefront's own.
    static constexpr int kPitch = 20;
    static __device__ __forceinline__ f4 own(f4 v, float *lds) {
        if (!ALONG) return v;
        const int lane = (int)threadIdx.x & 63;
        *reinterpret_cast<f4 *>(lds + (lane >> 2) * kPitch + (lane & 3) * 4) = v;
        wave_exchange();
        v = *reinterpret_cast<const f4 *>(lds + (lane & 15) * kPitch + (lane >> 4) * 4);
        wave_exchange();
        return v;
    }
};
constexpr int kTurn = 16 * Operand<true>::kPitch;
__device__ __forceinline__ f4 multiply(f4 a, f4 b, f4 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// sum[t] += the product over reduction indices k0 .. k1 - 1 of A and B[t]; the lanes' own sums of A's values are added to *rows.
// The operands of kAhead steps of 16 are requested together.
template <int kAhead, bool A_ALONG, bool B_ALONG, int NT>
__device__ __forceinline__ void accumulate_product(const Operand<A_ALONG> &a, const Operand<B_ALONG> (&b)[NT], int k0, int k1, float *lds,
                                                   f4 (&sum)[NT], float *rows) {
    auto add = [&](f4 va, const f4 (&vb)[NT]) {
        va = a.own(va, lds);
        *rows += (va.x + va.y) + (va.z + va.w);
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[t] = multiply(va, b[t].own(vb[t], lds + kTurn), sum[t]);
    };
    int k = k0;
    for (; k + 16 * kAhead <= k1; k += 16 * kAhead) {
        f4 va[kAhead], vb[kAhead][NT];
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
            va[s] = a.template fetch<true>(k + 16 * s, k1);
#pragma unroll
            for (int t = 0; t < NT; ++t) vb[s][t] = b[t].template fetch<true>(k + 16 * s, k1);
        }
        __builtin_amdgcn_sched_barrier(0);  // (left alone the compiler moves the loads to their uses, two or three in flight)
#pragma unroll
        for (int s = 0; s < kAhead; ++s) add(va[s], vb[s]);
    }
    for (; k < k1; k += 16) {
        const bool full = k + 16 <= k1;
        const f4 va = full ? a.template fetch<true>(k, k1) : a.template fetch<false>(k, k1);
        f4 vb[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) vb[t] = full ? b[t].template fetch<true>(k, k1) : b[t].template fetch<false>(k, k1);
        add(va, vb);
    }
}

template <int WAVES>
struct TileLds {
    union {
        float turn[WAVES][2 * kTurn];  // while a wavefront adds its products
        float part[WAVES * 256];       // afterwards
    };
    float rows[WAVES * 16];
};

// The 16 x 16 tile at (m0, n0) of the product of an M x K and a K x N operand, its K split over the wavefronts of the
// workgroup and added in their order; put(m, n, value) stores an element that exists, put_rows(m, value) the sum of row m of A.
template <int kAhead, bool A_ALONG, bool B_ALONG, typename Lds, typename Put, typename PutRows>
__device__ __forceinline__ void tile(const float *a, int64_t lda, int M, int m0, const float *b, int64_t ldb, int N, int n0, int K,
                                     Lds &lds, Put put, PutRows put_rows) {
    const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63, waves = (int)blockDim.x >> 6;
    const int each = ((K + 15) / 16 + waves - 1) / waves * 16, k0 = wave * each, k1 = min(K, k0 + each);
    const Operand<A_ALONG> oa(a, lda, m0, M);                                   // (rows and columns beyond the edge are computed,
    const Operand<B_ALONG> ob[1] = {Operand<B_ALONG>(b, ldb, n0, N)};  //  not stored)
    f4 sum[1] = {{0.f, 0.f, 0.f, 0.f}};
    float rows = 0.f;
    accumulate_product<kAhead>(oa, ob, k0, k1, lds.turn[wave], sum, &rows);
    __syncthreads();
    rows += __shfl_xor(rows, 16, 64);
    rows += __shfl_xor(rows, 32, 64);
#pragma unroll
    for (int e = 0; e < 4; ++e) lds.part[wave * 256 + ((lane >> 4) * 4 + e) * 16 + (lane & 15)] = sum[0][e];
    if (lane < 16) lds.rows[wave * 16 + lane] = rows;
    __syncthreads();
    for (int o = (int)threadIdx.x; o < 256 + 16; o += (int)blockDim.x) {
        const bool row = o >= 256;
        float t = 0.f;
#pragma unroll 4
        for (int w = 0; w < waves; ++w) t += row ? lds.rows[w * 16 + o - 256] : lds.part[w * 256 + o];
        const int m = m0 + (row ? o - 256 : o / 16), n = n0 + o % 16;
        if (m >= M) continue;
        if (row) put_rows(m, t);
        else if (n < N) put(m, n, t);
    }
}

constexpr int kForwardWaves = 16, kBackwardWaves = 8;  // the most of a workgroup

// A 16 x 16 tile of the logits, its reduction over the channels split over the wavefronts (32 x 2048 x 1000: 7.5 us, bound by the
// latency of the weights' loads; 131 MFLOP).
__global__ __launch_bounds__(kForwardWaves * 64) void head_linear_k(const float *__restrict__ pooled, int n, int c, int classes,
                                                                 const float *__restrict__ w, const float *__restrict__ b,
                                                                 float *__restrict__ logits, int64_t ld) {
    __shared__ TileLds<kForwardWaves> lds;
    tile<8, false, true>(pooled, n, n, (int)blockIdx.y * 16, w, c, classes, (int)blockIdx.x * 16, c, lds,
                     [&](int i, int k, float v) { logits[(int64_t)i * ld + k] = v + b[k]; }, [](int, float) {});
}

// The first `data_blocks` workgroups: d_pooled as [c][n], a tile each.  The others: the weights' gradient and, where the
// channels begin, the bias's -- STRIPS: 16 classes by 64 channels per wavefront, which reads the 16 classes' derivatives once
// for four tiles; else, where that leaves most of the chip idle, a tile per workgroup with the images split over its wavefronts.
// (32 x 2048 x 1000: 10.8 us for 17 MB and 262 MFLOP.)
template <bool STRIPS>
__global__ __launch_bounds__(kBackwardWaves * 64, 4) void head_linear_bwd_k(const float *__restrict__ dl, int64_t ld, const float *__restrict__ pooled,
                                                                     int n, int c, int classes, const float *__restrict__ w,
                                                                     float *__restrict__ d_pooled, float *dw, float *db, int accumulate,
                                                                     int data_blocks) {
    __shared__ TileLds<kBackwardWaves> lds;
    const int tiles_c = (c + 15) / 16;
    if ((int)blockIdx.x < data_blocks) {
        const int tm = (int)blockIdx.x / tiles_c, tc = channel_of((int)blockIdx.x - tm * tiles_c, tiles_c);
        tile<8, true, false>(dl, ld, n, tm * 16, w, c, c, tc * 16, classes, lds,
                          [&](int i, int ch, float v) { d_pooled[(int64_t)ch * n + i] = v; }, [](int, float) {});
        return;
    }
    const int block = (int)blockIdx.x - data_blocks;
    auto put_bias = [&](int k, float v) { db[k] = (accumulate ? db[k] : 0.f) + v; };
    auto put_weight = [&](int k, int ch, float v) {
        float *to = dw + (int64_t)k * c + ch;
        *to = (accumulate ? *to : 0.f) + v;
    };
    if constexpr (!STRIPS) {
        const int tk = block / tiles_c, tc = block - tk * tiles_c;
        tile<4, false, true>(dl, ld, classes, tk * 16, pooled, n, c, tc * 16, n, lds, put_weight, [&](int k, float v) {
            if (tc == 0) put_bias(k, v);
        });
    } else {
        const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63, waves = (int)blockDim.x >> 6;
        const int strips_c = (c + 63) / 64, strip = block * waves + wave;
        if (strip >= strips_c * ((classes + 15) / 16)) return;
        const int sk = strip / strips_c, c0 = (strip - sk * strips_c) * 64, k0 = sk * 16;
        const Operand<false> oa(dl, ld, k0, classes);
        const Operand<true> ob[4] = {{pooled, n, c0, c}, {pooled, n, c0 + 16, c}, {pooled, n, c0 + 32, c}, {pooled, n, c0 + 48, c}};
        f4 sum[4] = {};
        float bias = 0.f;
        accumulate_product<1>(oa, ob, 0, n, lds.turn[wave], sum, &bias);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int k = k0 + (lane >> 4) * 4 + e, ch = c0 + t * 16 + (lane & 15);
                if (k < classes && ch < c) put_weight(k, ch, sum[t][e]);
            }
        bias += __shfl_xor(bias, 16, 64);
        bias += __shfl_xor(bias, 32, 64);
        if (c0 == 0 && lane < 16 && k0 + lane < classes) put_bias(k0 + lane, bias);
    }
}

// Wavefronts that share a reduction of length K: at least two steps of 16 each.
int waves_for(int K, int most) { return std::max(1, std::min(most, (K + 31) / 32)); }

}  // namespace

void head_pool(Ctx &cx, View x, int c, Geo g, float eps, const float *gamma, const float *beta, HeadSaved s) {
    if (!cx.launch(K_HEAD, 4.0 * (double)g.pixels() * c + 12.0 * (double)g.n * c)) return;
    Planes p{g.n, c, g.hw(), quads_of(g.hw()), 0, 0, 0};
    while (p.tshift < 6 && (1 << p.tshift) < p.per) ++p.tshift;
    p.J = (p.per + (1 << p.tshift) - 1) >> p.tshift;
    const int at_once = 64 >> p.tshift;
    auto steps = [&](int waves) { return (g.n + waves * at_once - 1) / (waves * at_once); };
    // As few wavefronts a channel as keep its quads in registers, eight a lane, and fill the chip with eight a SIMD or have one step
    // of planes each.  (Whole forward passes: 32 x 2048 x 7 x 7 with 4: 15.2 us, with 16: 31.2, with 1: 16.5; 32 x 256 x 7 x 7 with 16: 8.3,
    // with 4: 10.0; 8 x 512 x 7 x 7 with 4, a step each: 7.1, with 16: 11.3.)
    int waves = p.J > 1 ? 16 : 1;
    while (waves < 16 && (((int64_t)c * waves < 8192 && steps(waves) > 1) || (int64_t)steps(waves) * p.J > 8)) waves *= 4;
    p.steps = steps(waves);
    const int64_t held = (int64_t)p.steps * p.J;
    const bool whole = g.hw() % 4 == 0;
#define RVN_POOL(TH, HELD, SINGLE)                                                                                                         \
    cx.run(whole ? head_pool_k<TH, HELD, true, SINGLE> : head_pool_k<TH, HELD, false, SINGLE>, dim3((unsigned)c), dim3(TH), 0, x.p, x.sn, x.sc, p, \
           eps, gamma, beta, s.stats, s.pooled, s.count, s.xhat)
    if (held > 16) RVN_POOL(1024, 0, false);
    else if (p.J > 1) RVN_POOL(1024, 16, false);
    else if (held > 8) RVN_POOL(1024, 16, true);
    else if (waves == 1) RVN_POOL(64, 8, true);
    else if (waves == 4 && held > 2) RVN_POOL(256, 8, true);
    else if (waves == 4) RVN_POOL(256, 2, true);
    else RVN_POOL(1024, 8, true);
#undef RVN_POOL
}

void head_linear(Ctx &cx, const float *pooled, int n, int c, int classes, const float *w, const float *b, float *logits, int64_t ld) {
    if (!cx.launch(K_HEAD, 4.0 * ((double)n * c + (double)classes * c + (double)n * classes), 2.0 * n * (double)c * classes)) return;
    cx.run(head_linear_k, dim3((unsigned)((classes + 15) / 16), (unsigned)((n + 15) / 16)),
           dim3((unsigned)(64 * waves_for(c, kForwardWaves))), 0, pooled, n, c, classes, w, b, logits, ld);
}

void head_linear_bwd(Ctx &cx, const float *dl, int64_t ld, const float *pooled, int n, int c, int classes, const float *w,
                     float *d_pooled, float *dw, float *db, bool accumulate) {
    if (!cx.launch(K_HEAD, 4.0 * (2.0 * n * c + 2.0 * classes * (double)c + (double)n * classes), 4.0 * n * (double)c * classes)) return;
    const int tiles_c = (c + 15) / 16, tiles_k = (classes + 15) / 16, data_blocks = tiles_c * ((n + 15) / 16);
    const int strips = ((c + 63) / 64) * tiles_k;
    // Strips read the derivatives a quarter as often, but each goes through all images: where there are strips enough.  (Whole
    // backward passes, by strips and by tiles: 32 x 2048 x 7 x 7, 1000 classes, 2016 strips 17.6 and 36.9 us; 8 x 512, 1000 classes, 504
    // strips 8.4 and 12.8; 128 x 512 21.9 and 22.1; 256 x 512 35.6 and 29.7; 32 x 256, 100 classes, 28 strips 7.7 and 6.2.)
    const bool in_strips = strips >= 256 + n;
    const int waves = waves_for(in_strips ? classes : std::max(classes, n), kBackwardWaves);
    cx.run(in_strips ? head_linear_bwd_k<true> : head_linear_bwd_k<false>,
           dim3((unsigned)(data_blocks + (in_strips ? (strips + waves - 1) / waves : tiles_c * tiles_k))), dim3((unsigned)(64 * waves)), 0, dl, ld,
           pooled, n, c, classes, w, d_pooled, dw, db, accumulate ? 1 : 0, data_blocks);
}

void head_pool_bwd(Ctx &cx, View x, int c, Geo g, HeadSaved s, const float *d_pooled, float *dgamma, float *dbeta, bool accumulate,
                   View dx) {
    if (!cx.launch(K_HEAD, 8.0 * (double)g.pixels() * c + 12.0 * (double)g.n * c)) return;
    const int per = quads_of(g.hw()), total = g.n * per;
    // workgroups a channel: enough to fill the chip, with four quads or more a thread
    int splits = c >= 2048 ? 1 : 2048 / c;
    const int most = (total + 4 * kPoolThreads - 1) / (4 * kPoolThreads);
    splits = splits < most ? splits : most;
    const int share = (total + splits - 1) / splits;
    cx.run(g.hw() % 4 == 0 ? head_pool_bwd_k<true> : head_pool_bwd_k<false>, dim3((unsigned)splits, (unsigned)c), dim3(kPoolThreads), 0, x.p, x.sn, x.sc, g.n, c, g.hw(), fast_div(per), share,
           s.stats, s.count, s.xhat, d_pooled, dgamma, dbeta, accumulate ? 1 : 0, dx.p, dx.sn, dx.sc);
}

}  // namespace rvn
