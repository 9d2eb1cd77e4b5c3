// Which form the gradient of the head norm and rotation takes, for the host and its tests.
#pragma once

namespace lory {
namespace rope {

// A few tokens with norms take one workgroup of 16 wavefronts, which writes dw itself, and no second launch: at most 16 tokens, a
// wavefront each at least, and at most kAloneValues values of queries and keys (it is bound by its arithmetic, whatever the type).
// us from a graph and called eagerly, one launch against two, over head counts and widths:
//   bf16   1024 values 4.7 and 6.9 against 6.4 and 9.7,  5120 5.3-6.3 and 7.0 against 6.5 and 9.7,  7680 5.9-6.2 and 7.0
//          against 6.5 and 9.8,  8192 in 16 tokens 7.1 and 7.2 against 6.6 and 9.8,  10240 6.5-6.8 and 7.0 against 6.5 and 9.8,
//          15360 6.7-7.8 and 6.9-7.9 against 6.5 and 9.8,  20480 7.6-8.7 and 7.7-8.8 against 6.6 and 9.8
//   fp32   1024 values 3.6 and 6.6 against 5.5 and 9.8,  5120 4.9-5.4 and 6.6 against 5.7 and 9.8,  7680 5.3-6.0 and 6.7
//          against 5.7 and 9.8,  10240 5.9-6.8 and 6.7 against 5.8 and 9.8
// Up to the limit a replay takes at most 0.5 us more and mostly less; behind it replays lose what eager calls gain.
constexpr int kAlone = 16;
constexpr long kAloneValues = 8192;

inline bool alone(long tokens, long values) { return tokens > 0 && tokens <= kAlone && values <= kAloneValues; }

}  // namespace rope
}  // namespace lory
