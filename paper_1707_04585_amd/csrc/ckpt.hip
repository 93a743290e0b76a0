// Activation checkpoints in 8 bits: save, load, and the backward pass of BN + ReLU straight from the codes.
//
// A plane's pixels fall into groups of 128 that share a scale (see include/revnet.h for the format).  Everything here
// is a few instructions on every element of a tensor that is read or written once: bound by memory, save at 5 bytes an
// element (4 in, 1 out), load at 5, the backward pass at 9 (13 with a skip tensor) where a channel fits one workgroup's
// registers and 14 (18) where the sums take a launch of their own.
//
// A lane works on four neighbouring pixels (quads.h): 16 bytes of fp32, 4 of codes.  Planes of any size and tensors of
// any alignment take the same path.
#include <algorithm>

#include "fast_div.h"
#include "kernels.h"
#include "prep_filter.h"
#include "quads.h"
#include "wgrad_reduce.h"

namespace rvn {

namespace {

constexpr int kThreads = 256;
constexpr float kTop = 126.f;                          // the largest code that rounding alone gives
constexpr float kLeast = 126.f * 1.17549435e-38f;      // smallest group magnitude: keeps the scale a normal number

typedef uint32_t u32_any __attribute__((aligned(1)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef u16x4 u16x4_any __attribute__((aligned(2)));

template <bool WHOLE>
__device__ __forceinline__ uint32_t load_codes(const int8_t *plane, QuadAt q) {
    if (WHOLE || q.end == 4) return *reinterpret_cast<const u32_any *>(plane + q.i);
    uint32_t v = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j) v |= j < q.end ? (uint32_t)(uint8_t)plane[j] << (8 * j) : 0u;
    return v;
}
// FAR: nothing reads the codes soon, they shall not push what the caches hold out of them (a stack of 12 bottleneck blocks that
// stores, forward: 4.52 ms, 4.67 without)
template <bool WHOLE, bool FAR>
__device__ __forceinline__ void store_codes(int8_t *plane, QuadAt q, uint32_t word) {
    if (WHOLE || (q.from == 0 && q.end == 4)) {
        u32_any *const to = reinterpret_cast<u32_any *>(plane + q.i);
        if (FAR) __builtin_nontemporal_store(word, to);
        else *to = word;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (q.owns(j)) plane[q.i + j] = (int8_t)(word >> (8 * j));
}
__device__ __forceinline__ f4 decode(uint32_t q, float s) {
    f4 v;
    v.x = (float)(int8_t)q * s;
    v.y = (float)(int8_t)(q >> 8) * s;
    v.z = (float)(int8_t)(q >> 16) * s;
    v.w = (float)((int32_t)q >> 24) * s;
    return v;
}

// The tensors of a launch; the workgroups along x from block0 on are a tensor's.
struct Jobs {
    CkptTensor t[3];
    int block0[3];
};
__device__ __forceinline__ CkptTensor job_of(const Jobs &jobs, int &block) {
    const int b = block;
    CkptTensor t = jobs.t[0];
    if (b >= jobs.block0[1]) t = jobs.t[1], block = b - jobs.block0[1];
    if (b >= jobs.block0[2]) t = jobs.t[2], block = b - jobs.block0[2];
    return t;
}

// 2^tshift neighbouring lanes share a group: 16 lanes with two quads each, 64 pixels apart, or, on planes of at most 64
// pixels, as many as the plane has quads with one each.  blockIdx.x counts the groups of an image, blockIdx.y images; a lane
// requests the quads of kFly images before it uses the first.  (64 x 128 x 56 x 56, half the channels of a tensor: 129 MB in 30 us,
// 4.3 TB/s, mostly of reads; 128 x 512 x 13 x 13, with partial words at both ends of a plane, 3.4 TB/s.)
template <bool BN, bool WHOLE, bool FAR>
__global__ __launch_bounds__(kThreads) void ckpt_save_k(const Jobs jobs, int N, int HW, int G, FastDiv by_g, int tshift) {
    int block = (int)blockIdx.x;
    const CkptTensor t = job_of(jobs, block);
    const float *const x = t.x.p, *const stats = t.stats;
    const int64_t sn = t.x.sn, sc = t.x.sc;
    int8_t *const q = t.k.q;
    float *const s = t.k.s;
    const int C = t.c;
    constexpr int kFly = 2;
    const int item = block * (kThreads >> tshift) + ((int)threadIdx.x >> tshift), lane = (int)threadIdx.x & ((1 << tshift) - 1);
    const bool live = item < C * G;
    const int ch = live ? quotient(item, by_g) : 0, group = live ? item - ch * G : 0;
    const int k0 = group * (kCkptGroup / 4) + lane;
    const QuadAt at[2] = {quad_at<WHOLE>(k0, HW), quad_at<WHOLE>(k0 + 16, HW)};
    const bool mine[2] = {live && k0 * 4 < HW, live && tshift == 4 && (k0 + 16) * 4 < HW};
    float scale = 0.f, shift = 0.f;
    if (BN) scale = stats[2 * C + ch], shift = stats[3 * C + ch];
    const float *px = x + (int64_t)ch * sc;
    for (int n0 = (int)blockIdx.y * kFly; n0 < N; n0 += (int)gridDim.y * kFly) {
        f4 v[kFly][2];
#pragma unroll
        for (int u = 0; u < kFly; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v[u][h] = f4{0.f, 0.f, 0.f, 0.f};
                if (n0 + u < N && mine[h]) v[u][h] = fetch4<WHOLE>(px + (int64_t)(n0 + u) * sn, at[h]);
            }
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            if (n0 + u >= N) break;  // (uniform)
#pragma unroll
            for (int h = 0; h < 2; ++h) v[u][h] = own4<WHOLE>(v[u][h], at[h]);
            // magnitudes as bit patterns: these order as the values do, infinities and NaN on top
            uint32_t most = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) most = max(most, __float_as_uint(v[u][h][j]) & 0x7fffffffu);
            most = team_most(most, tshift);
            const bool finite = most < 0x7f800000u;
            const float a = fmaxf(finite ? __uint_as_float(most) : 1.f, kLeast);
            const float step = a / kTop, inverse = finite ? kTop / a : 0.f;
            const int64_t plane = (int64_t)(n0 + u) * C + ch;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!mine[h]) continue;
                uint32_t word = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float c = rintf(v[u][h][j] * inverse);
                    if (BN) {
                        const bool want = fmaf(v[u][h][j], scale, shift) > 0.f, got = fmaf(c * step, scale, shift) > 0.f;
                        if (want != got) c += (scale > 0.f) == want ? 1.f : -1.f;
                    }
                    word |= ((uint32_t)(int)c & 0xffu) << (8 * j);
                }
                if (!finite) word = 0;
                store_codes<WHOLE, FAR>(q + plane * HW, at[h], word);
            }
            if (live && lane == 0) s[plane * G + group] = finite ? step : __uint_as_float(0x7fc00000u);
        }
    }
}

// One lane per four pixels; prep.blocks workgroups convert filters, then come by_blocks.d workgroups (the quads of an image)
// for each of `images` images at a time.  (The same 129 MB in 20.5 us, 6.3 TB/s, mostly of writes, which a fill reaches 6.8 with.)
template <bool WHOLE, bool PREP>
__global__ __launch_bounds__(kThreads) void ckpt_load_k(const Jobs jobs, int N, int HW, int G, FastDiv by_per, FastDiv by_blocks, int images,
                                                        const PrepArgs prep) {
    int block = (int)blockIdx.x;
    if (PREP) {
        if (block < prep.blocks) {
            prep_filter_body(prep, block);
            return;
        }
        block -= prep.blocks;
    }
    const int n0 = quotient(block, by_blocks);
    block -= n0 * (int)by_blocks.d;
    const CkptTensor t = job_of(jobs, block);
    const int8_t *const q = t.k.q;
    const float *const s = t.k.s;
    float *const x = t.x.p;
    const int64_t sn = t.x.sn, sc = t.x.sc;
    const int C = t.c, per = (int)by_per.d, item = block * kThreads + (int)threadIdx.x;
    if (item >= C * per) return;
    const int ch = quotient(item, by_per), k = item - ch * per;
    const QuadAt at = quad_at<WHOLE>(k, HW);
    for (int n = n0; n < N; n += images) {
        const int64_t plane = (int64_t)n * C + ch;
        const uint32_t word = load_codes<WHOLE>(q + plane * HW, at);
        store4<WHOLE>(x + (int64_t)n * sn + (int64_t)ch * sc, at, decode(word, s[plane * G + k / (kCkptGroup / 4)]));
    }
}

// ---- backward pass of BN + ReLU ----------------------------------------------------------------------------

struct BnLayer {
    const int8_t *q;
    const float *s, *stats;
    int N, C, HW, G;
    FastDiv by_per;  // quads of a plane
};

// A channel's constants, and the quads of its planes: quad e of N * per.
struct Channel {
    float mean, rstd, scale, shift;
};
__device__ __forceinline__ Channel channel(const BnLayer &b, int ch) {
    return Channel{b.stats[ch], b.stats[b.C + ch], b.stats[2 * b.C + ch], b.stats[3 * b.C + ch]};
}
struct Place {
    int n, k;
    QuadAt at;
    int64_t plane;
};
template <bool WHOLE>
__device__ __forceinline__ Place place(const BnLayer &b, int ch, int e) {
    const int n = quotient(e, b.by_per), k = e - n * (int)b.by_per.d;
    return Place{n, k, quad_at<WHOLE>(k, b.HW), (int64_t)n * b.C + ch};
}
// What a quad is made of; zeros where `live` is false.
struct Quad {
    uint32_t word;
    float step;
    f4 da;
};
template <bool WHOLE>
__device__ __forceinline__ Quad fetch(const BnLayer &b, const Place &p, int ch, bool live, const float *da, int64_t dsn, int64_t dsc) {
    Quad q{0u, 0.f, f4{0.f, 0.f, 0.f, 0.f}};
    if (live) {
        q.word = load_codes<WHOLE>(b.q + p.plane * b.HW, p.at);
        q.step = b.s[p.plane * b.G + p.k / (kCkptGroup / 4)];
        q.da = fetch4<WHOLE>(da + (int64_t)p.n * dsn + (int64_t)ch * dsc, p.at);
    }
    return q;
}
// dz and x - mean (pixels that are not the quad's own: dz is zero)
template <bool WHOLE>
__device__ __forceinline__ void quad(const Quad &q, QuadAt at, const Channel &c, f4 &dz, f4 &xm) {
    const f4 v = decode(q.word, q.step), da = own4<WHOLE>(q.da, at);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        dz[j] = fmaf(v[j], c.scale, c.shift) > 0.f ? da[j] : 0.f;
        xm[j] = v[j] - c.mean;
    }
}

// r to a quad of the plane at `out` or, rounded to bf16, at `out16` (nearest even: what the convolutions that read it would
// round it to)
template <bool WHOLE>
__device__ __forceinline__ void put_quad(f4 r, QuadAt q, float *out, uint16_t *out16) {
    if (!out16) {
        store4<WHOLE>(out, q, r);
        return;
    }
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    const u16x4 h = __builtin_bit_cast(u16x4, __builtin_convertvector(r, bf16x4));
    if (WHOLE || (q.from == 0 && q.end == 4)) {
        *reinterpret_cast<u16x4_any *>(out16 + q.i) = h;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (q.owns(j)) out16[q.i + j] = h[j];
}

constexpr int kFly = 4;  // quads a thread requests before it uses the first

// sums[ch][split] = (sum dz, sum dz * (x - mean)) over a share of a channel's quads; threads (52 terms at 256 x 64 x 56 x 56) and
// wavefronts add in fp32, everything above in double.  Bound by memory (64 x 128 x 56 x 56: 129 MB in 30.7 us, 4.2 TB/s).
template <bool WHOLE>
__global__ __launch_bounds__(kThreads) void ckpt_bn_reduce_k(const BnLayer b, const float *da, int64_t dsn, int64_t dsc, int share,
                                                             double2 *sums) {
    __shared__ double part[4][2];
    const int ch = (int)blockIdx.x, total = b.N * (int)b.by_per.d;  // (channels first: neighbours in memory)
    const int first = (int)blockIdx.y * share, last = min(total, first + share);
    const Channel c = channel(b, ch);
    float a0 = 0.f, a1 = 0.f;
    for (int e0 = first + (int)threadIdx.x; e0 < last; e0 += kFly * kThreads) {
        Quad q[kFly];
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            const int e = e0 + u * kThreads;
            q[u] = fetch<WHOLE>(b, place<WHOLE>(b, ch, e < last ? e : e0), ch, e < last, da, dsn, dsc);
        }
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            f4 dz, xm;
            const int e = e0 + u * kThreads;
            quad<WHOLE>(q[u], place<WHOLE>(b, ch, e < last ? e : e0).at, c, dz, xm);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a0 += dz[j];
                a1 = fmaf(dz[j], xm[j], a1);
            }
        }
    }
    const float t0 = wave_total(a0), t1 = wave_total(a1);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][0] = t0, part[threadIdx.x >> 6][1] = t1;
    __syncthreads();
    if (threadIdx.x == 0)
        sums[(int64_t)ch * gridDim.y + blockIdx.y] =
            make_double2((part[0][0] + part[1][0]) + (part[2][0] + part[3][0]), (part[0][1] + part[1][1]) + (part[2][1] + part[3][1]));
}

// dx = scale * (dz - mean dz - xh * mean(dz * xh)) as scale * dz - a - (x - mean) * b
struct Coefs {
    float a, b;
};
__device__ __forceinline__ Coefs coefs(const Channel &c, double sum, double sum_xm, double inv_m) {
    const double r = c.rstd, s = c.scale;
    return Coefs{(float)(s * (sum * inv_m)), (float)(s * r * (r * sum_xm * inv_m))};
}
__device__ __forceinline__ f4 gradient(const f4 &dz, const f4 &xm, const Channel &c, const Coefs &k) {
    f4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = fmaf(-xm[j], k.b, fmaf(c.scale, dz[j], -k.a));
    return r;
}

__device__ __forceinline__ void put_sums(const Channel &c, double sum, double sum_xm, float *dgamma, float *dbeta, int ch, int accumulate) {
    dbeta[ch] = (accumulate ? dbeta[ch] : 0.f) + (float)sum;
    dgamma[ch] = (accumulate ? dgamma[ch] : 0.f) + (float)(c.rstd * sum_xm);
}

// The first carry.blocks workgroups sum a filter gradient's partial results; the others take `chunks` shares of every channel.
// (64 x 128 x 56 x 56 with a skip tensor: 335 MB in 54 us, 6.2 TB/s, part of the second read of codes and da from the Infinity Cache.)
template <bool SKIP, bool WHOLE>
__global__ __launch_bounds__(kThreads) void ckpt_bn_apply_k(const BnLayer b, const float *da, int64_t dsn, int64_t dsc,
                                                            const double2 *__restrict__ sums, int S, double inv_m, FastDiv by_c, int chunks,
                                                            float *dgamma, float *dbeta, int accumulate, const float *skip, int64_t ksn,
                                                            int64_t ksc, float *out, int64_t osn, int64_t osc, uint16_t *out16,
                                                            const WgradReduce carry) {
    if ((int)blockIdx.x < carry.blocks) {
        __shared__ float lds[kThreads];
        wgrad_reduce_body(carry, (int)blockIdx.x, lds);
        return;
    }
    // (channels first, as the sums were formed, and from the end: what was read last is in the nearer caches)
    const int bx = (int)blockIdx.x - carry.blocks, back = quotient(bx, by_c), ch = bx - back * b.C, chunk = chunks - 1 - back;
    const int total = b.N * (int)b.by_per.d, e0 = chunk * kFly * kThreads + (int)threadIdx.x;
    const Channel c = channel(b, ch);
    Quad q[kFly];
    f4 kv[kFly];
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
        const int e = e0 + u * kThreads;
        const Place p = place<WHOLE>(b, ch, e < total ? e : 0);
        q[u] = fetch<WHOLE>(b, p, ch, e < total, da, dsn, dsc);
        if (SKIP && e < total) kv[u] = fetch4<WHOLE>(skip + (int64_t)p.n * ksn + (int64_t)ch * ksc, p.at);
    }
    // every wavefront adds the channel's partial sums for itself, in the same order
    const int lane = (int)threadIdx.x & 63;
    double2 part = make_double2(0.0, 0.0);
    if (lane < S) part = sums[(int64_t)ch * S + lane];
    const double sum = wave_total(part.x), sum_xm = wave_total(part.y);
    if (chunk == 0 && threadIdx.x == 0) put_sums(c, sum, sum_xm, dgamma, dbeta, ch, accumulate);
    const Coefs k = coefs(c, sum, sum_xm, inv_m);
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
        const int e = e0 + u * kThreads;
        if (e >= total) return;
        const Place p = place<WHOLE>(b, ch, e);
        f4 dz, xm;
        quad<WHOLE>(q[u], p.at, c, dz, xm);
        f4 r = gradient(dz, xm, c, k);
        if (SKIP) r += kv[u];
        put_quad<WHOLE>(r, p.at, out + (int64_t)p.n * osn + (int64_t)ch * osc, out16 ? out16 + p.plane * b.HW : nullptr);
    }
}

// Both passes in one launch where a channel's quads fit the registers of one workgroup: codes and da are read once.  (128 x 512 x 10 x 12:
// 71 MB in 15.9 us, 4.5 TB/s; 32 x 512 x 7 x 7, 7.3 MB, 5.1 us, bound by latency.)
constexpr int kFusedQuads = 8;

template <int T, bool SKIP, bool WHOLE>
__global__ __launch_bounds__(T) void ckpt_bn_fused_k(const BnLayer b, const float *da, int64_t dsn, int64_t dsc, double inv_m,
                                                     float *dgamma, float *dbeta, int accumulate, const float *skip, int64_t ksn,
                                                     int64_t ksc, float *out, int64_t osn, int64_t osc, uint16_t *out16,
                                                     const WgradReduce carry) {
    if constexpr (T == kThreads) {
        if ((int)blockIdx.x < carry.blocks) {
            __shared__ float lds[kThreads];
            wgrad_reduce_body(carry, (int)blockIdx.x, lds);
            return;
        }
    }
    __shared__ double part[T / 64][2];
    const int ch = channel_of((int)blockIdx.x - carry.blocks, b.C), total = b.N * (int)b.by_per.d;
    const Channel c = channel(b, ch);
    f4 dz[kFusedQuads], xm[kFusedQuads];
    float a0 = 0.f, a1 = 0.f;
#pragma unroll
    for (int u = 0; u < kFusedQuads; ++u) {
        if (u * T >= total) break;  // (uniform)
        const int e = (int)threadIdx.x + u * T;
        const Place p = place<WHOLE>(b, ch, e < total ? e : 0);
        quad<WHOLE>(fetch<WHOLE>(b, p, ch, e < total, da, dsn, dsc), p.at, c, dz[u], xm[u]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a0 += dz[u][j];
            a1 = fmaf(dz[u][j], xm[u][j], a1);
        }
    }
    const float t0 = wave_total(a0), t1 = wave_total(a1);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][0] = t0, part[threadIdx.x >> 6][1] = t1;
    __syncthreads();
    double sum = 0.0, sum_xm = 0.0;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) sum += part[w][0], sum_xm += part[w][1];
    if (threadIdx.x == 0) put_sums(c, sum, sum_xm, dgamma, dbeta, ch, accumulate);
    const Coefs k = coefs(c, sum, sum_xm, inv_m);
#pragma unroll
    for (int u = 0; u < kFusedQuads; ++u) {
        const int e = (int)threadIdx.x + u * T;
        if (e >= total) return;
        const Place p = place<WHOLE>(b, ch, e);
        f4 r = gradient(dz[u], xm[u], c, k);
        if (SKIP) r += fetch4<WHOLE>(skip + (int64_t)p.n * ksn + (int64_t)ch * ksc, p.at);
        put_quad<WHOLE>(r, p.at, out + (int64_t)p.n * osn + (int64_t)ch * osc, out16 ? out16 + p.plane * b.HW : nullptr);
    }
}

unsigned blocks_for(int64_t n, int per) { return (unsigned)((n + per - 1) / per); }

// Workgroups a channel's sums are split over: enough to fill the chip, at most one partial sum per lane.
int ckpt_bn_splits(int c, const Geo &g) {
    const int64_t quads = (int64_t)g.n * quads_of(g.hw());
    int64_t s = c >= 8192 ? 1 : 8192 / c;
    s = s < 64 ? s : 64;
    const int64_t most = (quads + 2 * kThreads - 1) / (2 * kThreads);
    return (int)(s < most ? s : most);
}

}  // namespace

// Job list with `blocks_of(c)` workgroups a tensor; *blocks, *bytes: in all.
template <typename BlocksOf>
static Jobs make_jobs(const CkptTensor *t, int count, Geo g, BlocksOf blocks_of, unsigned *blocks, double *bytes) {
    Jobs j{};
    *blocks = 0;
    *bytes = 0.0;
    for (int i = 0; i < 3; ++i) {
        j.t[i] = t[i < count ? i : 0];
        j.block0[i] = i < count ? (int)*blocks : 0x7fffffff;
        if (i >= count) continue;
        *blocks += blocks_of(t[i].c);
        *bytes += (double)g.n * t[i].c * (5.0 * g.hw() + 4.0 * ckpt_groups(g.hw()));
    }
    return j;
}

void ckpt_save(Ctx &cx, const CkptTensor *t, int count, Geo g, bool far) {
    const int hw = g.hw(), G = ckpt_groups(hw);
    int tshift = 0;  // lanes of a group: 16, or as many as a smaller plane has quads, rounded up to a power of two
    while (tshift < 4 && (4 << tshift) < hw) ++tshift;
    unsigned blocks;
    double bytes;
    const Jobs jobs = make_jobs(t, count, g, [&](int c) { return blocks_for((int64_t)c * G, kThreads >> tshift); }, &blocks, &bytes);
    if (!cx.launch(K_CKPT, bytes)) return;
    const int pairs = (g.n + 1) / 2;
    const bool whole = hw % 4 == 0, bn = t[0].stats != nullptr;  // (of all tensors or of none)
    void (*kernel)(const Jobs, int, int, int, FastDiv, int) = whole ? ckpt_save_k<false, true, false> : ckpt_save_k<false, false, false>;
    if (bn && far) kernel = whole ? ckpt_save_k<true, true, true> : ckpt_save_k<true, false, true>;
    else if (bn) kernel = whole ? ckpt_save_k<true, true, false> : ckpt_save_k<true, false, false>;
    cx.run(kernel,
           dim3(blocks, (unsigned)(pairs < 65535 ? pairs : 65535)), dim3(kThreads), 0, jobs, g.n, hw, G, fast_div(G), tshift);
}

void ckpt_load(Ctx &cx, const CkptTensor *t, int count, Geo g, const PrepArgs *carry, double carry_bytes) {
    const int hw = g.hw(), G = ckpt_groups(hw), per = quads_of(hw);
    unsigned blocks;
    double bytes;
    const Jobs jobs = make_jobs(t, count, g, [&](int c) { return blocks_for((int64_t)c * per, kThreads); }, &blocks, &bytes);
    if (!cx.launch(K_CKPT, bytes + carry_bytes)) return;
    PrepArgs prep{};
    if (carry) prep = *carry;
    // (a launch counts its threads in 32 bits: the workgroups of at most 2^23 / blocks images, which go on to the others)
    const int images = (int)std::max<int64_t>(1, std::min<int64_t>(g.n, (1 << 23) / blocks));
    const dim3 grid((unsigned)images * blocks + (unsigned)prep.blocks);
    const bool whole = hw % 4 == 0;
    cx.run(prep.blocks > 0 ? (whole ? ckpt_load_k<true, true> : ckpt_load_k<false, true>) : (whole ? ckpt_load_k<true, false> : ckpt_load_k<false, false>),
           grid, dim3(kThreads), 0, jobs, g.n, hw, G, fast_div(per), fast_div((int)blocks), images, prep);
}

size_t ckpt_bn_scratch_floats(int c, const Geo &g) { return (size_t)c * ckpt_bn_splits(c, g) * 4; }

void ckpt_bn_relu_bwd(Ctx &cx, Ckpt k, View da, int c, Geo g, const float *stats, float *scratch, float *dgamma, float *dbeta,
                      bool accumulate, const View *skip, View out, const WgradReduce *carry, uint16_t *out16) {
    if (out16 && skip) {  // a caller's mistake: nothing sensible to launch
        cx.fail(hipErrorInvalidValue);
        return;
    }
    const int hw = g.hw(), per = quads_of(hw), total = g.n * per;
    const double elems = (double)g.pixels() * c;
    const BnLayer b{k.q, k.s, stats, g.n, c, hw, ckpt_groups(hw), fast_div(per)};
    const double inv_m = 1.0 / (double)g.pixels();
    WgradReduce red{};
    if (carry) red = *carry;
    if (red.blocks < 0) red.blocks = 0;
    const View kv = skip ? *skip : View{nullptr, 0, 0};
    const int acc = accumulate ? 1 : 0;
    const double out_bytes = out16 ? 2.0 : skip ? 8.0 : 4.0;
    // One launch where a workgroup of 256 threads holds a channel (32 x 512 x 7 x 7: 4.5 us, 8.5 in two passes; 32 x 16 x 14 x 14: 4.8
    // and 5.9).  Of 1024 threads with up to four quads each always (64 x 16 x 14 x 14: 5.0 and 6.1; 64 x 256 x 14 x 14: 7.9 and 12.4), with up
    // to eight from 64 channels on (150 x 64 x 14 x 14: 9.1 and 9.5; 150 x 16 x 14 x 14: 7.6 and 6.3, with most of the chip idle); these
    // carry no other launch's work.
    const bool wide = total > kFusedQuads * kThreads, whole = hw % 4 == 0;
    if (total <= kFusedQuads * 1024 && !(wide && (red.blocks > 0 || (total > 4096 && c < 64)))) {
        if (!cx.launch(K_BN_BWD_APPLY, (5.0 + out_bytes) * elems)) return;
        const dim3 grid((unsigned)(c + red.blocks));
#define RVN_FUSED(T, K)                                                                                                          \
    cx.run(whole ? ckpt_bn_fused_k<T, K, true> : ckpt_bn_fused_k<T, K, false>, grid, dim3(T), 0, b, da.p, da.sn, da.sc, inv_m, dgamma, dbeta, acc, kv.p, kv.sn, kv.sc, out.p, \
           out.sn, out.sc, out16, red)
        if (wide && skip) RVN_FUSED(1024, true);
        else if (wide) RVN_FUSED(1024, false);
        else if (skip) RVN_FUSED(kThreads, true);
        else RVN_FUSED(kThreads, false);
#undef RVN_FUSED
        return;
    }
    const int S = ckpt_bn_splits(c, g), share = (total + S - 1) / S;
    double2 *sums = reinterpret_cast<double2 *>(scratch);
    if (cx.launch(K_BN_BWD_REDUCE, 5.0 * elems))
        cx.run(whole ? ckpt_bn_reduce_k<true> : ckpt_bn_reduce_k<false>, dim3((unsigned)c, (unsigned)S), dim3(kThreads), 0, b, da.p, da.sn, da.sc, share, sums);
    if (cx.launch(K_BN_BWD_APPLY, (5.0 + out_bytes) * elems)) {
        const int chunks = (total + kFly * kThreads - 1) / (kFly * kThreads);
        const dim3 grid((unsigned)(chunks * c + red.blocks));
        cx.run(skip ? (whole ? ckpt_bn_apply_k<true, true> : ckpt_bn_apply_k<true, false>)
                    : (whole ? ckpt_bn_apply_k<false, true> : ckpt_bn_apply_k<false, false>),
               grid, dim3(kThreads), 0, b, da.p, da.sn, da.sc, sums, S, inv_m, fast_div(c), chunks, dgamma, dbeta, acc, kv.p, kv.sn, kv.sc, out.p,
               out.sn, out.sc, out16, red);
    }
}

}  // namespace rvn
