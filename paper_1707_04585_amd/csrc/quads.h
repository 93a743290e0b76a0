// Four neighbouring pixels of a plane as the unit of a streaming kernel: one 16-byte access, whatever the plane's size and
// the tensor's alignment (16-byte accesses need dword alignment only on this hardware).  Where a plane's size is no multiple
// of four its last quad is read from four pixels before the plane's end, and the pixels that belong to the quad before it are
// dropped: no lane goes pixel by pixel to read.  Device code, but for quads_of.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rvn {

inline int quads_of(int hw) { return (hw + 3) / 4; }

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef f4 f4_any __attribute__((aligned(4)));

// Pixels i + from .. i + end - 1 of a plane are the quad's own; i .. i + 3 are in the plane where end is 4.
struct QuadAt {
    int i, from, end;
    __device__ __forceinline__ bool owns(int j) const { return j >= from && j < end; }
};
// Quad k of a plane of hw pixels; WHOLE: hw is a multiple of four, which no quad's end has to be looked at for (32 x 64 x 56 x 56:
// saving a checkpoint 8.5 us, by the general path 10.6; BN backward from codes 17.1 and 17.8, at 128 x 16 x 8 x 8 5.1 and 6.8).
template <bool WHOLE>
__device__ __forceinline__ QuadAt quad_at(int k, int hw) {
    if (WHOLE) return QuadAt{4 * k, 0, 4};
    const int i = max(0, min(4 * k, hw - 4));
    return QuadAt{i, 4 * k - i, min(4, hw - i)};
}

// The four pixels at a quad's place; those that are not its own are dropped afterwards (own4), so that no request waits for
// the values of another.
template <bool WHOLE>
__device__ __forceinline__ f4 fetch4(const float *plane, QuadAt q) {
    if (WHOLE || q.end == 4) return *reinterpret_cast<const f4_any *>(plane + q.i);
    f4 v = {0.f, 0.f, 0.f, 0.f};  // a plane of fewer than four pixels
#pragma unroll
    for (int j = 0; j < 3; ++j) v[j] = j < q.end ? plane[j] : 0.f;
    return v;
}
template <bool WHOLE>
__device__ __forceinline__ f4 own4(f4 v, QuadAt q) {
    if (WHOLE) return v;
#pragma unroll
    for (int j = 0; j < 3; ++j) v[j] = j < q.from ? 0.f : v[j];
    return v;
}
// (pixels that are not the quad's own are not written)
template <bool WHOLE>
__device__ __forceinline__ void store4(float *plane, QuadAt q, f4 v) {
    if (WHOLE || (q.from == 0 && q.end == 4)) {
        *reinterpret_cast<f4_any *>(plane + q.i) = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (q.owns(j)) plane[q.i + j] = v[j];
}

// What the wavefront's lanes wrote to LDS before this, any of them reads after it.  A wavefront's LDS accesses are carried out in
// order, so this costs no instruction and no wait; the fences keep the compiler from moving accesses over the barrier, which by
// itself orders instructions but not memory.
__device__ __forceinline__ void wave_exchange() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// Sum over the 64 lanes, in every lane.
__device__ __forceinline__ double wave_total(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const int lo = __shfl_xor(__double2loint(v), o, 64), hi = __shfl_xor(__double2hiint(v), o, 64);
        v += __hiloint2double(hi, lo);
    }
    return v;
}
// The same in fp32 by lane moves within the register file (about 50 cycles; a shuffle through LDS costs that for each of six
// steps): rows of 16 lanes first, then the rows.
__device__ __forceinline__ float wave_total(float v) {
#define RVN_STEP(ctrl, rows) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xf, false))
    RVN_STEP(0x111, 0xf);  // row_shr 1, 2, 4, 8: the last lane of each row has the row's
    RVN_STEP(0x112, 0xf);
    RVN_STEP(0x114, 0xf);
    RVN_STEP(0x118, 0xf);
    RVN_STEP(0x142, 0xa);  // row_bcast 15 and 31: lane 63 has all
    RVN_STEP(0x143, 0xc);
#undef RVN_STEP
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// combine(v, w) over the 2^shift neighbouring lanes of each team (shift <= 6, the same in all lanes), in every lane: up to 16
// lanes by moves within a row of 16 -- swapped neighbours, swapped pairs, then mirrored halves and rows, whose parts hold one
// value each by then.
template <typename Combine>
__device__ __forceinline__ uint32_t team_combine(uint32_t v, int shift, Combine combine) {
#define RVN_MOVE(ctrl) (uint32_t) __builtin_amdgcn_update_dpp((int)v, (int)v, ctrl, 0xf, 0xf, true)
    if (__builtin_expect(shift >= 1, 1)) v = combine(v, RVN_MOVE(0xb1));   // quad_perm 1 0 3 2
    if (__builtin_expect(shift >= 2, 1)) v = combine(v, RVN_MOVE(0x4e));   // quad_perm 2 3 0 1
    if (__builtin_expect(shift >= 3, 1)) v = combine(v, RVN_MOVE(0x141));  // row_half_mirror
    if (__builtin_expect(shift >= 4, 1)) v = combine(v, RVN_MOVE(0x140));  // row_mirror
#undef RVN_MOVE
    if (shift >= 5) v = combine(v, (uint32_t)__shfl_xor((int)v, 16, 64));
    if (shift >= 6) v = combine(v, (uint32_t)__shfl_xor((int)v, 32, 64));
    return v;
}
// Both values' sums over the team, in one walk through the steps, those of up to 16 lanes in line (the head's forward pass at
// 256 x 512 x 14 x 14, 100 classes: 42.2 us, with two walks and jumps 49.6).
__device__ __forceinline__ void team_totals(float &a, float &b, int shift) {
    auto add = [](float v, uint32_t w) { return v + __uint_as_float(w); };
#define RVN_MOVE(v, ctrl) (uint32_t) __builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), ctrl, 0xf, 0xf, true)
#define RVN_BOTH(ctrl) a = add(a, RVN_MOVE(a, ctrl)), b = add(b, RVN_MOVE(b, ctrl))
    if (__builtin_expect(shift >= 1, 1)) RVN_BOTH(0xb1);
    if (__builtin_expect(shift >= 2, 1)) RVN_BOTH(0x4e);
    if (__builtin_expect(shift >= 3, 1)) RVN_BOTH(0x141);
    if (__builtin_expect(shift >= 4, 1)) RVN_BOTH(0x140);
#undef RVN_BOTH
#undef RVN_MOVE
    if (shift >= 5) a += __shfl_xor(a, 16, 64), b += __shfl_xor(b, 16, 64);
    if (shift >= 6) a += __shfl_xor(a, 32, 64), b += __shfl_xor(b, 32, 64);
}
__device__ __forceinline__ uint32_t team_most(uint32_t v, int shift) {
    return team_combine(v, shift, [](uint32_t a, uint32_t b) { return max(a, b); });
}

}  // namespace

// Channel of workgroup `block` of C: workgroups go to the 8 XCDs in turn, and each XCD's take a run of channels, so that a
// cache line that ends one plane and begins the next is read by one XCD's cache (32 x 512 x 7 x 7: BN backward from codes 6.5 -> 5.5 us;
// 32 x 2048 x 7 x 7: the head's pooling 11.4 -> 10.5 us, its gradient 8.4 -> 7.0).
__device__ __forceinline__ int channel_of(int block, int C) {
    const int xcd = block & 7;
    return xcd * (C >> 3) + min(xcd, C & 7) + (block >> 3);
}

}  // namespace rvn
