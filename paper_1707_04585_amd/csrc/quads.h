// Four neighbouring pixels of a plane as the unit of a streaming kernel: one 16-byte access, whatever the plane's size and
// the tensor's alignment (16-byte accesses need dword alignment only on this hardware); the last quad of a plane whose
// size is no multiple of four goes pixel by pixel.  Device code, but for quads_of.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rvn {

inline int quads_of(int hw) { return (hw + 3) / 4; }

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef f4 f4_any __attribute__((aligned(4)));

// Pixels i .. i+3 of a plane of which `left` > 0 exist; what lies beyond reads as zero and is not written.
__device__ __forceinline__ f4 load4(const float *p, int left) {
    if (left >= 4) return *reinterpret_cast<const f4_any *>(p);
    f4 v = {p[0], left > 1 ? p[1] : 0.f, left > 2 ? p[2] : 0.f, 0.f};
    return v;
}
__device__ __forceinline__ void store4(float *p, int left, f4 v) {
    if (left >= 4) {
        *reinterpret_cast<f4_any *>(p) = v;
        return;
    }
    p[0] = v.x;
    if (left > 1) p[1] = v.y;
    if (left > 2) p[2] = v.z;
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

}  // namespace

}  // namespace rvn
