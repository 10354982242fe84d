// Rotation of queries and keys by positions on several axes.
#pragma once

#include <algorithm>

#include "rotary.h"

namespace msparse {

constexpr int kRotateTokens = 64;   // of a workgroup
struct RotateArgs {
    Positions pos;
    const void *q, *k;                      // [B, heads, T, d], bf16 or fp32
    void *qout, *kout;
    int64_t qs[3], ks[3], qos[3], kos[3];   // strides: sequence, head, token
    int32_t B, T, Hq, Hkv, d;               // Hkv = 0: no keys
    bool inverse, f32;
    int32_t blocks, shares;                 // of the tokens, of the heads
};
// Workgroups that share a block of tokens, the heads dealt out: enough of them to fill the
// card, as few as that takes since each forms the angles for itself.  Up to 256, 512 and 1536 in
// all (bf16, us): 64 x 1 token, 28 + 4 heads of 128 3.0, 3.1, 5.0; 4096 tokens 23.2, 21.7, 28.7; 16384,
// 32 + 8 heads 96.7, 77.7, 81.6.  512 rounded down and up: 22594, 16 + 2 heads 66.1, 57.7; 17000, 28 + 4
// 102, 79.
inline void share_heads(RotateArgs& a) {
    const int64_t heads = a.Hq + a.Hkv, groups = int64_t(a.B) * a.blocks;
    a.shares = int32_t(std::min(heads, (511 + groups) / groups));
}
hipError_t launch_rotate(const RotateArgs& a, hipStream_t s);

}  // namespace msparse
