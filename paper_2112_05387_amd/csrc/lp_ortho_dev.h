// What the kernels of the orthogonalisation share: the polynomial, the scales of what is held in two fp16, access to either type.
#pragma once
#include "lp_gemm.h"
#include "lp_ortho.h"

namespace lp {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kScaleX = 16384.f, kScaleS = 8192.f, kScaleB = 4096.f;

// the last tensor whose first block is not beyond `block`
__device__ __forceinline__ int ns_find(const int* start, int n, int block) {
    const int lane = threadIdx.x & 63;
    int found = 0;
    for (int i = 0; i < n; i += 64) found += __popcll(__ballot(i + lane < n && start[min(i + lane, n)] <= block));
    return __builtin_amdgcn_readfirstlane(found - 1);
}

__device__ __forceinline__ unsigned f16_bits(float x) { return __builtin_bit_cast(unsigned short, (_Float16)x); }
__device__ __forceinline__ float f16_up(unsigned b) { return (float)__builtin_bit_cast(_Float16, (unsigned short)b); }

// two values in two parts each, packed: hi and the rest of it
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void split_f16x2(float a, float b, unsigned& hi, unsigned& lo) {
    const f16x2_t h = __builtin_convertvector(f32x2_t{a, b}, f16x2_t);
    const f32x2_t rest = {fmaf((float)h[0], -1.f, a), fmaf((float)h[1], -1.f, b)};
    hi = __builtin_bit_cast(unsigned, h);
    lo = __builtin_bit_cast(unsigned, __builtin_convertvector(rest, f16x2_t));
}

__device__ __forceinline__ float load_low(const void* p, int low, size_t e) {
    return low ? bf16_bits_to_float(reinterpret_cast<const unsigned short*>(p)[e]) : reinterpret_cast<const float*>(p)[e];
}
__device__ __forceinline__ void store_low(void* p, int low, size_t e, float x) {
    if (low) reinterpret_cast<unsigned short*>(p)[e] = float_to_bf16_bits(x);
    else reinterpret_cast<float*>(p)[e] = x;
}

}  // namespace lp
