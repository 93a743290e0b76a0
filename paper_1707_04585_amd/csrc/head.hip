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
#include "fast_div.h"
#include "kernels.h"
#include "quads.h"

namespace rvn {

namespace {

// ---- pooling ---------------------------------------------------------------------------------------------------

constexpr int kHeld = 8;  // quads a lane keeps in registers

// How a channel's planes fall to wavefronts: 2^tshift lanes share a plane of `per` quads, J of them each; a wavefront takes
// 64 >> tshift planes at a time, `steps` times.
struct Planes {
    int N, C, HW, per, tshift, J, steps;
};

// The sum over the workgroup of a value of each thread, in every thread.
template <int TH>
__device__ __forceinline__ double block_total(float v, double *lds) {
    const double t = wave_total((double)v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = t;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < TH / 64; ++w) s += lds[w];
    return s;
}

// HELD: steps * J <= kHeld, and the channel stays in registers; otherwise it is read three times (the second and third
// mostly from the caches).
template <int TH, bool HELD>
__global__ __launch_bounds__(TH) void head_pool_k(const float *__restrict__ x, int64_t sn, int64_t sc, const Planes g, float eps,
                                                  const float *__restrict__ gamma, const float *__restrict__ beta,
                                                  float *__restrict__ stats, float *__restrict__ pooled, float *__restrict__ count,
                                                  float *__restrict__ xhat) {
    __shared__ double lds[TH / 64];
    const int ch = (int)blockIdx.x, wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
    const int T = 1 << g.tshift, sub = lane & (T - 1), planes = 64 >> g.tshift;
    const float *base = x + (int64_t)ch * sc;
    f4 held[kHeld];
    // calls visit(value, plane, pixels left) for every item of this lane, in order; a plane's items follow each other
    auto each = [&](bool first, auto visit) {
        int step = 0, j = 0;
        auto item = [&](int k) {
            const int n = (step * (TH / 64) + wave) * planes + (lane >> g.tshift), quad = j * T + sub;
            const int left = n < g.N && quad < g.per ? g.HW - quad * 4 : 0;
            f4 v = {0.f, 0.f, 0.f, 0.f};
            if (HELD && !first) v = held[k];
            else if (left > 0) v = load4(base + (int64_t)n * sn + quad * 4, left);
            if (HELD && first) held[k] = v;
            visit(v, n, left, j == g.J - 1);
            if (++j == g.J) j = 0, ++step;
        };
        if constexpr (HELD) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k)
                if (step < g.steps) item(k);
        } else {
            while (step < g.steps) item(0);
        }
    };
    float a = 0.f;
    each(true, [&](f4 v, int, int, bool) { a += (v.x + v.y) + (v.z + v.w); });
    const double m = (double)g.N * g.HW;
    const float mean = (float)(block_total<TH>(a, lds) / m);
    a = 0.f;
    each(false, [&](f4 v, int, int left, bool) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float d = e < left ? v[e] - mean : 0.f;
            a = fmaf(d, d, a);
        }
    });
    const float rstd = (float)(1.0 / sqrt(block_total<TH>(a, lds) / m + (double)eps));
    const float scale = gamma[ch] * rstd, shift = fmaf(-mean, scale, beta[ch]);
    if (threadIdx.x == 0) {
        stats[ch] = mean;
        stats[g.C + ch] = rstd;
        stats[2 * g.C + ch] = scale;
        stats[3 * g.C + ch] = shift;
    }
    const float inv_hw = 1.f / (float)g.HW;
    float sum = 0.f, pos = 0.f, hat = 0.f;
    each(false, [&](f4 v, int n, int left, bool last) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float z = fmaf(v[e], scale, shift);
            if (e < left && z > 0.f) {
                sum += z;
                pos += 1.f;
                hat += (v[e] - mean) * rstd;
            }
        }
        if (!last) return;
        for (int o = T >> 1; o > 0; o >>= 1) {
            sum += __shfl_xor(sum, o, 64);
            pos += __shfl_xor(pos, o, 64);
            hat += __shfl_xor(hat, o, 64);
        }
        if (sub == 0 && n < g.N) {
            pooled[(int64_t)n * g.C + ch] = sum * inv_hw;
            count[(int64_t)ch * g.N + n] = pos;
            xhat[(int64_t)ch * g.N + n] = hat;
        }
        sum = pos = hat = 0.f;
    });
}

// dx of a share of a channel's quads; every workgroup forms the channel's two sums for itself.
constexpr int kPoolThreads = 256;

__global__ __launch_bounds__(kPoolThreads) void head_pool_bwd_k(const float *__restrict__ x, int64_t sn, int64_t sc, int N, int C, int HW,
                                                                FastDiv by_per, int share, const float *__restrict__ stats,
                                                                const float *__restrict__ count, const float *__restrict__ xhat,
                                                                const float *__restrict__ d_pooled, float *dgamma, float *dbeta,
                                                                int accumulate, float *__restrict__ dx, int64_t osn, int64_t osc) {
    __shared__ double lds[kPoolThreads / 64];
    const int ch = (int)blockIdx.y, per = (int)by_per.d, total = N * per;
    const float mean = stats[ch], rstd = stats[C + ch], scale = stats[2 * C + ch], shift = stats[3 * C + ch];
    const float inv_hw = 1.f / (float)HW;
    const float *g = d_pooled + (int64_t)ch * N, *cnt = count + (int64_t)ch * N, *hat = xhat + (int64_t)ch * N;
    float a0 = 0.f, a1 = 0.f;
    for (int n = (int)threadIdx.x; n < N; n += kPoolThreads) {
        const float gn = g[n] * inv_hw;
        a0 = fmaf(gn, cnt[n], a0);
        a1 = fmaf(gn, hat[n], a1);
    }
    const double sb = block_total<kPoolThreads>(a0, lds), sg = block_total<kPoolThreads>(a1, lds);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        dbeta[ch] = (accumulate ? dbeta[ch] : 0.f) + (float)sb;
        dgamma[ch] = (accumulate ? dgamma[ch] : 0.f) + (float)sg;
    }
    const double inv_m = 1.0 / ((double)N * HW);
    const float c1 = (float)(sb * inv_m), c2 = (float)(sg * inv_m);
    const int last = min(total, ((int)blockIdx.x + 1) * share);
    for (int e = (int)blockIdx.x * share + (int)threadIdx.x; e < last; e += kPoolThreads) {
        const int n = quotient(e, by_per), i = (e - n * per) * 4, left = HW - i;
        const f4 v = load4(x + (int64_t)n * sn + (int64_t)ch * sc + i, left);
        const float gn = g[n] * inv_hw;
        f4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float dz = fmaf(v[j], scale, shift) > 0.f ? gn : 0.f;
            r[j] = scale * ((dz - c1) - ((v[j] - mean) * rstd) * c2);
        }
        store4(dx + (int64_t)n * osn + (int64_t)ch * osc + i, left, r);
    }
}

// ---- products on v_mfma_f32_16x16x4_f32 -----------------------------------------------------------------------
// Lane l holds row (or column) l % 16 of an operand at reduction index l / 16 and, of the result, column l % 16 of rows
// (l / 16) * 4 .. + 3.  Four instructions take 16 reduction indices: the lanes of group l / 16 the four from (l / 16) * 4.

// Operand whose reduction index runs along memory: row `r` at p + r * ld; what lies at or behind k1 reads as zero.
__device__ __forceinline__ f4 along(const float *p, int64_t ld, int r, int k, int k1) {
    if (k >= k1) return f4{0.f, 0.f, 0.f, 0.f};
    return load4(p + (int64_t)r * ld + k, k1 - k);
}
// Operand whose reduction index runs across it: index k at p + k * ld + r.
__device__ __forceinline__ f4 across(const float *p, int64_t ld, int r, int k, int k1) {
    f4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = k + e < k1 ? p[(int64_t)(k + e) * ld + r] : 0.f;
    return v;
}
__device__ __forceinline__ f4 multiply(f4 a, f4 b, f4 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// The 16x16 tile at (m0, n0) of the product of an M x K and a K x N operand, its K split over the wavefronts of the
// workgroup and added in their order; put(m, n, value) stores an element that exists.
template <bool B_ALONG, typename Put>
__device__ __forceinline__ void tile(const float *a, int64_t lda, int M, int m0, const float *b, int64_t ldb, int N, int n0, int K,
                                     float *lds, Put put) {
    const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63, waves = (int)blockDim.x >> 6;
    const int steps = (K + 15) / 16, each = (steps + waves - 1) / waves;
    const int k0 = wave * each * 16, k1 = min(K, k0 + each * 16);
    const int r = min(m0 + (lane & 15), M - 1), c = min(n0 + (lane & 15), N - 1);  // (beyond the edge: computed, not stored)
    f4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < each; ++s) {
        const int k = k0 + s * 16 + (lane >> 4) * 4;
        const f4 va = along(a, lda, r, k, k1);
        const f4 vb = B_ALONG ? along(b, ldb, c, k, k1) : across(b, ldb, c, k, k1);
        sum = multiply(va, vb, sum);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) lds[wave * 256 + ((lane >> 4) * 4 + e) * 16 + (lane & 15)] = sum[e];
    __syncthreads();
    for (int o = (int)threadIdx.x; o < 256; o += (int)blockDim.x) {
        float t = 0.f;
        for (int w = 0; w < waves; ++w) t += lds[w * 256 + o];
        const int m = m0 + o / 16, n = n0 + o % 16;
        if (m < M && n < N) put(m, n, t);
    }
}

constexpr int kMostWaves = 16;

__global__ __launch_bounds__(kMostWaves * 64) void head_linear_k(const float *__restrict__ pooled, int n, int c, int classes,
                                                                 const float *__restrict__ w, const float *__restrict__ b,
                                                                 float *__restrict__ logits, int64_t ld) {
    __shared__ float lds[kMostWaves * 256];
    tile<true>(pooled, c, n, (int)blockIdx.y * 16, w, c, classes, (int)blockIdx.x * 16, c, lds,
               [&](int i, int k, float v) { logits[(int64_t)i * ld + k] = v + b[k]; });
}

// The first `data_blocks` workgroups: d_pooled as [c][n], a tile each.  The others: the weights' gradient, a strip of 16
// classes by 64 channels per wavefront, and in the strips of the first channels the bias's.
__global__ __launch_bounds__(kMostWaves * 64) void head_linear_bwd_k(const float *__restrict__ dl, int64_t ld, const float *__restrict__ pooled,
                                                                     int n, int c, int classes, const float *__restrict__ w,
                                                                     float *__restrict__ d_pooled, float *dw, float *db, int accumulate,
                                                                     int data_blocks) {
    __shared__ float lds[kMostWaves * 256];
    if ((int)blockIdx.x < data_blocks) {
        const int tiles_c = (c + 15) / 16, tm = (int)blockIdx.x / tiles_c, tc = (int)blockIdx.x - tm * tiles_c;
        tile<false>(dl, ld, n, tm * 16, w, c, c, tc * 16, classes, lds, [&](int i, int ch, float v) { d_pooled[(int64_t)ch * n + i] = v; });
        return;
    }
    const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63, waves = (int)blockDim.x >> 6;
    const int strips_c = (c + 63) / 64, strips = strips_c * ((classes + 15) / 16);
    const int strip = ((int)blockIdx.x - data_blocks) * waves + wave;
    if (strip >= strips) return;
    const int sk = strip / strips_c, c0 = (strip - sk * strips_c) * 64, k0 = sk * 16;
    const int r = min(k0 + (lane & 15), classes - 1);
    f4 sum[4] = {};
    float bias = 0.f;
    for (int i = (lane >> 4) * 4, s = 0; s < (n + 15) / 16; ++s, i += 16) {
        const f4 va = across(dl, ld, r, i, n);
        bias += (va.x + va.y) + (va.z + va.w);
#pragma unroll
        for (int t = 0; t < 4; ++t) sum[t] = multiply(va, across(pooled, c, min(c0 + t * 16 + (lane & 15), c - 1), i, n), sum[t]);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int ch = c0 + t * 16 + (lane & 15);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int k = k0 + (lane >> 4) * 4 + e;
            if (k >= classes || ch >= c) continue;
            float *to = dw + (int64_t)k * c + ch;
            *to = (accumulate ? *to : 0.f) + sum[t][e];
        }
    }
    if (c0 == 0) {
        bias += __shfl_xor(bias, 16, 64);
        bias += __shfl_xor(bias, 32, 64);
        if (lane < 16 && k0 + lane < classes) db[k0 + lane] = (accumulate ? db[k0 + lane] : 0.f) + bias;
    }
}

// Wavefronts that share a reduction of length K: at least two steps of 16 each.
int waves_for(int K) {
    const int w = (K + 31) / 32;
    return w < 1 ? 1 : w < kMostWaves ? w : kMostWaves;
}

}  // namespace

void head_pool(Ctx &cx, View x, int c, Geo g, float eps, const float *gamma, const float *beta, HeadSaved s) {
    if (!cx.launch(K_HEAD, 4.0 * (double)g.pixels() * c + 12.0 * (double)g.n * c)) return;
    Planes p{g.n, c, g.hw(), quads_of(g.hw()), 0, 0, 0};
    while (p.tshift < 6 && (1 << p.tshift) < p.per) ++p.tshift;
    p.J = (p.per + (1 << p.tshift) - 1) >> p.tshift;
    const int at_once = 64 >> p.tshift;
    auto steps = [&](int waves) { return (g.n + waves * at_once - 1) / (waves * at_once); };
    const bool small = steps(4) * p.J <= kHeld;
    p.steps = steps(small ? 4 : 16);
#define RVN_POOL(TH, HELD)                                                                                                     \
    cx.run(head_pool_k<TH, HELD>, dim3((unsigned)c), dim3(TH), 0, x.p, x.sn, x.sc, p, eps, gamma, beta, s.stats, s.pooled, s.count, \
           s.xhat)
    if (small) RVN_POOL(256, true);
    else if ((int64_t)p.steps * p.J <= kHeld) RVN_POOL(1024, true);
    else RVN_POOL(1024, false);
#undef RVN_POOL
}

void head_linear(Ctx &cx, const float *pooled, int n, int c, int classes, const float *w, const float *b, float *logits, int64_t ld) {
    if (!cx.launch(K_HEAD, 4.0 * ((double)n * c + (double)classes * c + (double)n * classes), 2.0 * n * (double)c * classes)) return;
    cx.run(head_linear_k, dim3((unsigned)((classes + 15) / 16), (unsigned)((n + 15) / 16)), dim3((unsigned)(64 * waves_for(c))), 0, pooled, n,
           c, classes, w, b, logits, ld);
}

void head_linear_bwd(Ctx &cx, const float *dl, int64_t ld, const float *pooled, int n, int c, int classes, const float *w,
                     float *d_pooled, float *dw, float *db, bool accumulate) {
    if (!cx.launch(K_HEAD, 4.0 * (2.0 * n * c + 2.0 * classes * (double)c + (double)n * classes), 4.0 * n * (double)c * classes)) return;
    const int waves = waves_for(classes), data_blocks = ((c + 15) / 16) * ((n + 15) / 16);
    const int strips = ((c + 63) / 64) * ((classes + 15) / 16);
    cx.run(head_linear_bwd_k, dim3((unsigned)(data_blocks + (strips + waves - 1) / waves)), dim3((unsigned)(64 * waves)), 0, dl, ld, pooled, n, c,
           classes, w, d_pooled, dw, db, accumulate ? 1 : 0, data_blocks);
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
    cx.run(head_pool_bwd_k, dim3((unsigned)splits, (unsigned)c), dim3(kPoolThreads), 0, x.p, x.sn, x.sc, g.n, c, g.hw(), fast_div(per), share,
           s.stats, s.count, s.xhat, d_pooled, dgamma, dbeta, accumulate ? 1 : 0, dx.p, dx.sn, dx.sc);
}

}  // namespace rvn
