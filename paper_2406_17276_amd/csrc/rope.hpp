// Position rotation of a row of a head, shared by the operators that write queries and keys (gfx950 only).
//
// Eight lanes (head_dim 64: four) hold a row, sixteen columns each, in two runs of eight that can be turned against each
// other:
//   pairs (j, j + R/2):  lane t holds columns 8t.. and R/2 + 8t.. while 8t < R/2, the columns from R on in order after that;
//   pairs (2j, 2j + 1):  lane t holds columns 16t.. and 16t + 8..
// Either way its eight angles are those of j = 8t .. 8t + 7, and lanes with 16t >= R turn nothing.
#pragma once

#include "common.hpp"

#if defined(__HIPCC__)
namespace ot {

// Cosine and sine of an angle in fp64, rounded to fp32.  The angle less the nearest multiple k of pi/2 (pi/2 as a double and
// the rest of it as another: the products are exact inside the multiply-add, so the difference is good to 1e-16 for any
// position of 32 bits), then the Taylor sums, whose first terms left out are below 1e-11 (sine, x^13 / 13!) and 5e-13
// (cosine, x^14 / 14!) for |x| <= pi/4.  fp64 multiply-adds run at the fp32 rate on this machine, and the fp32 of a
// 1e-11 accurate value is the correctly rounded one but for one in some thousand.
__device__ __forceinline__ float2 cos_sin(double angle) {
    const double k = rint(angle * 0.63661977236758134308);               // 2 / pi
    double x = fma(-k, 1.57079632679489661923, angle);
    x = fma(-k, 6.123233995736766036e-17, x);
    const double z = x * x;
    double s = fma(z, -1.0 / 39916800.0, 1.0 / 362880.0);
    s = fma(z, s, -1.0 / 5040.0);
    s = fma(z, s, 1.0 / 120.0);
    s = fma(z, s, -1.0 / 6.0);
    s = fma(z * x, s, x);
    double c = fma(z, 1.0 / 479001600.0, -1.0 / 3628800.0);
    c = fma(z, c, 1.0 / 40320.0);
    c = fma(z, c, -1.0 / 720.0);
    c = fma(z, c, 1.0 / 24.0);
    c = fma(z, c, -0.5);
    c = fma(z, c, 1.0);
    const int q = (int)(long long)k & 3;                                  // quadrant
    const double u = q & 1 ? s : c, v = q & 1 ? c : s;
    return float2{(float)(q == 1 || q == 2 ? -u : u), (float)(q >= 2 ? -v : v)};
}

struct Rotary {
    const double* inv_freq;
    int dim;              // R
    int interleaved;
};

// first column of the two runs of lane t
__device__ __forceinline__ int run_a(const Rotary& r, int t) { return r.interleaved || 16 * t >= r.dim ? 16 * t : 8 * t; }
__device__ __forceinline__ int run_b(const Rotary& r, int t) {
    return r.interleaved || 16 * t >= r.dim ? 16 * t + 8 : r.dim / 2 + 8 * t;
}

// The sixteen values of a lane (a: first run, b: second) turned by its eight angles.  Products are rounded before they are added:
// u cos - v sin then has the same bits as in arithmetic that knows no fused multiply-add, such as a tensor library's.
__device__ __forceinline__ void turn(float (&a)[8], float (&b)[8], const float2 (&cs)[8], int interleaved) {
#pragma clang fp contract(off)
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float u = a[2 * i], v = a[2 * i + 1], w = b[2 * i], x = b[2 * i + 1];
            a[2 * i] = u * cs[i].x - v * cs[i].y;
            a[2 * i + 1] = u * cs[i].y + v * cs[i].x;
            b[2 * i] = w * cs[4 + i].x - x * cs[4 + i].y;
            b[2 * i + 1] = w * cs[4 + i].y + x * cs[4 + i].x;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float u = a[i], v = b[i];
            a[i] = u * cs[i].x - v * cs[i].y;
            b[i] = u * cs[i].y + v * cs[i].x;
        }
    }
}

// Where the cosine and sine of angle j of a row sit among the row's R/2 in LDS: the lanes of a row read 16 bytes, two angles,
// side by side.  lanes: R / 16, the lanes that turn.
__device__ __forceinline__ int angle_at(int j, int lanes) { return ((j >> 1 & 3) * lanes + (j >> 3)) * 2 + (j & 1); }
__device__ __forceinline__ void read_angles(const float2* row, int t, int lanes, float2 (&cs)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const f32x4 w = *(const f32x4*)(row + (e * lanes + t) * 2);
        cs[2 * e] = float2{w[0], w[1]};
        cs[2 * e + 1] = float2{w[2], w[3]};
    }
}

// Eight consecutive values of a row in memory <-> fp32
template <int DT> __device__ __forceinline__ void load8(const void* p, long long at, float (&x)[8]) {
    if constexpr (DT == OT_BF16) {
        VecOf<OT_BF16>::unpack(*(const u32x4*)((const unsigned short*)p + at), x);
    } else {
        const f32x4 lo = *(const f32x4*)((const float*)p + at), hi = *(const f32x4*)((const float*)p + at + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = lo[i]; x[4 + i] = hi[i]; }
    }
}
__device__ __forceinline__ unsigned int pack_bf16(float x, float y) {       // to nearest even
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)x, (__bf16)y};
    return __builtin_bit_cast(unsigned int, v);
}
template <int DT> __device__ __forceinline__ void store8(void* p, long long at, const float (&x)[8]) {
    if constexpr (DT == OT_BF16) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        *(u32x4*)((unsigned short*)p + at) = w;
    } else {
        *(f32x4*)((float*)p + at) = f32x4{x[0], x[1], x[2], x[3]};
        *(f32x4*)((float*)p + at + 4) = f32x4{x[4], x[5], x[6], x[7]};
    }
}

}  // namespace ot
#endif
