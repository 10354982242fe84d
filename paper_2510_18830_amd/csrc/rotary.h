// Rotation of columns (i, i + d/2) by position * freq[i], what the append to the cache
// and the rotation by itself share.
#pragma once

#include "common.h"

namespace msparse {

constexpr int kMaxAxes = 4;
// Positions of a call's tokens on several axes.  Pair i of a head turns by the position on
// axis[i] times freq[i]; an axis that is none of them leaves its pairs as they are.
struct Positions {
    const int32_t* at;     // [axes, tokens of the call]
    const int32_t* axis;   // [d / 2], NULL: the first for every pair
    const float* freq;     // [d / 2]
    int32_t axes;
    int64_t tokens;        // of the call, all sequences
};

namespace {

// cos and sin of pos * freq for any position: the angle in revolutions as a sum of
// two doubles, reduced to an eighth of a revolution, then the Taylor series (their
// first missing terms are below 1e-12).
struct Turn {
    double c, s;
};
__device__ __forceinline__ Turn turn_by(double pos, float freq) {
    constexpr double kInv = 0.15915494309189535, kInvLo = -9.839338337591243e-18;   // 1 / (2 pi) in two parts
    const double x = pos * double(freq);
    const double hi = x * kInv;
    const double lo = __builtin_fma(x, kInv, -hi) + x * kInvLo;
    const double r = (hi - __builtin_rint(hi)) + lo;        // revolutions in [-1/2, 1/2]
    const double quarter = __builtin_rint(4.0 * r);
    const double y = (r - 0.25 * quarter) * 6.283185307179586;   // [-pi/4, pi/4]
    const double y2 = y * y;
    double ps = 1.0 / 6227020800.0, pc = 1.0 / 479001600.0;
    ps = __builtin_fma(ps, y2, -1.0 / 39916800.0);
    pc = __builtin_fma(pc, y2, -1.0 / 3628800.0);
    ps = __builtin_fma(ps, y2, 1.0 / 362880.0);
    pc = __builtin_fma(pc, y2, 1.0 / 40320.0);
    ps = __builtin_fma(ps, y2, -1.0 / 5040.0);
    pc = __builtin_fma(pc, y2, -1.0 / 720.0);
    ps = __builtin_fma(ps, y2, 1.0 / 120.0);
    pc = __builtin_fma(pc, y2, 1.0 / 24.0);
    ps = __builtin_fma(ps, y2, -1.0 / 6.0);
    pc = __builtin_fma(pc, y2, -0.5);
    const double fs = __builtin_fma(ps * y2, y, y), fc = __builtin_fma(pc, y2, 1.0);
    const int n = int(quarter) & 3;
    const double a = (n & 1) ? fs : fc, b = (n & 1) ? fc : fs;
    return Turn{(n == 1 || n == 2) ? -a : a, (n & 2) ? -b : b};
}

// x1 c - x2 s and x2 c + x1 s, every product rounded: the same values whichever
// of the two a fused form would leave unrounded
__device__ __forceinline__ void rotate(float& x1, float& x2, float c, float s) {
#pragma clang fp contract(off)
    const float a = x1 * c, b = x2 * s, e = x2 * c, f = x1 * s;
    x1 = a - b;
    x2 = e + f;
}

__device__ __forceinline__ void unpack8(const u32x4& w, float* x) {
    const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = bf16_lo(a[j]);
        x[2 * j + 1] = bf16_hi(a[j]);
    }
}

// In the place of a pair's sine: the pair stays as it is, bit for bit.  (The angle 0 would do for finite values only:
// an infinity or a NaN of one column times the sine 0 makes the other one NaN, and -0 + 0 is +0.)
constexpr float kStays = 2.f;
__device__ __forceinline__ bool stays(float s) { return fabsf(s) == kStays; }

// Eight pairs of bf16, rounded once.  AXES: some may stay.
template <bool AXES>
__device__ __forceinline__ void rotate8(u32x4& w1, u32x4& w2, const float* c, const float* s) {
    float x1[8], x2[8];
    unpack8(w1, x1);
    unpack8(w2, x2);
#pragma unroll
    for (int j = 0; j < 8; ++j) rotate(x1[j], x2[j], c[j], s[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t r1 = pack_bf16x2(x1[2 * j], x1[2 * j + 1]), r2 = pack_bf16x2(x2[2 * j], x2[2 * j + 1]);
        const uint32_t keep = !AXES ? 0 : (stays(s[2 * j]) ? 0xffffu : 0) | (stays(s[2 * j + 1]) ? 0xffff0000u : 0);
        w1[j] = (w1[j] & keep) | (r1 & ~keep);
        w2[j] = (w2[j] & keep) | (r2 & ~keep);
    }
}

// of pair i of token `t` of the call; the sine is kStays where it has no axis
__device__ __forceinline__ Turn turn_at(const Positions& p, int i, int64_t t) {
    const int axis = p.axis ? p.axis[i] : 0;
    if (uint32_t(axis) >= uint32_t(p.axes)) return Turn{1.0, double(kStays)};
    return turn_by(double(p.at[axis * p.tokens + t]), p.freq[i]);
}

}  // namespace

}  // namespace msparse
