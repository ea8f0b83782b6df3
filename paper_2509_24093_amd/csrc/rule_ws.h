// Workspace of the gated delta rule: unit = (sequence, head), chunk by chunk.
#pragma once

#include <algorithm>
#include <type_traits>

#include "seq.h"

namespace cgconv {

struct RuleWs {
  float4* token;   // [unit][chunk][64][2]: see Token in rule_common.h
  float* whole;    // [unit][chunk]: decay of the whole chunk
  float4* inv;     // [unit][chunk][10 blocks][64 lanes]: (1 + A)^-1, rows
  float4* inside;  // the same of P, rows; of the backward columns
  float4* invT;    // (1 + A)^-1, columns (backward)
  float* state;    // [unit][chunk][DP][VP]: the state before every chunk (backward)
  float* gstate;   // [unit][chunk][DP][VP]: gradient of the state after every chunk
  float* value;    // [unit][chunk][64][VP]: what the tokens write, V'
  float* gvalue;   // [unit][chunk][64][VP]: its gradient through (1 + A)^-T, dY
  float* start;       // [unit][segment][DP][VP]: the state before every segment (its gradient behind it)
  float* span_state;  // [unit][segment][DP][VP]: what a segment adds to the state
  // and by what it multiplies it, as the join's operand: [unit][segment][DP / 16 tiles of rows]
  // [DP / 32][3 parts][64 lanes]; and its transpose (backward)
  uint4* span_matrix;
  uint4* span_matrixT;
  int units, chunks, KB, V, VP;  // DP = 32 KB; VP: V in whole tiles of 32
  int segments, span;            // the chunks in segments of `span`, walked at once
};

// Chunks of a segment.  A walk takes as many rounds of 256 blocks, one a CU, as its segments'
// blocks of 128 columns make (those of the first span walk have no matrix), a round the
// segment's length; joining takes half a chunk's time a step.  Measured, bf16, heads of 128 x
// 128: 4 prompts of 8192 tokens and 16 heads in 1, 2, 3, 4, 8 segments 970, 851, 627, 659, 714 us;
// 32768 tokens of 8 heads in 16, 24, 32, 64 segments 456, 461, 413, 492; training of 2 x 4096
// tokens of 8 heads in 4, 8, 16 segments 784, 577, 584.
inline int rule_span(int chunks, int units, int KB, int VP) {
  const long long values = (VP + 127) / 128, both = (VP + 32 * KB + 127) / 128;
  const auto rounds = [&](long long blocks) { return (units * blocks + 255) / 256; };
  int best = chunks;
  long long least = 2 * chunks * rounds(values);
  for (int want = 2; want <= std::min(chunks / 4, 64); ++want) {
    const int span = (chunks + want - 1) / want, n = (chunks + span - 1) / span;
    const long long cost = 2 * span * (rounds(values * n) + rounds(values + both * (n - 2))) + n - 2;
    if (cost < least) {
      least = cost;
      best = span;
    }
  }
  return best;
}

inline RuleWs rule_workspace(const RuleSizes& n, bool backward, char* base, size_t* bytes) {
  RuleWs w{};
  w.units = n.B * n.H;
  w.chunks = (n.N + kRuleChunk - 1) / kRuleChunk;
  w.KB = (n.D + 31) / 32;
  w.V = n.K * (n.C / n.H);
  w.VP = (w.V + 31) / 32 * 32;
  const size_t count = (size_t)w.units * w.chunks;
  size_t at = 0;
  const auto take = [&](auto*& p, size_t n) {
    p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + at);
    at += (n * sizeof(*p) + 255) / 256 * 256;
  };
  take(w.token, count * kRuleChunk * 2);
  take(w.whole, count);
  take(w.inv, count * kRuleTriangle * 64);
  take(w.inside, count * kRuleTriangle * 64);
  if (backward) {
    take(w.invT, count * kRuleTriangle * 64);
    take(w.state, count * 32 * w.KB * w.VP);
    take(w.gstate, count * 32 * w.KB * w.VP);
    take(w.value, count * kRuleChunk * w.VP);
    take(w.gvalue, count * kRuleChunk * w.VP);
  }
  w.span = rule_span(w.chunks, w.units, w.KB, w.VP);
  w.segments = (w.chunks + w.span - 1) / w.span;
  if (w.segments > 1) {
    take(w.start, (size_t)w.units * w.segments * 32 * w.KB * w.VP);
    take(w.span_state, (size_t)w.units * w.segments * 32 * w.KB * w.VP);
    const size_t matrix = (size_t)w.units * w.segments * 2 * w.KB * w.KB * 3 * 64;
    take(w.span_matrix, matrix);
    if (backward) take(w.span_matrixT, matrix);
  }
  if (bytes) *bytes = at;
  return w;
}

// (1 + A)^-1, P and the numbers of every token, of all chunks at once.
hipError_t launch_rule_prepare(const RuleArgs& a, const RuleWs& w, bool backward, hipStream_t s);
// The states from chunk to chunk; for the backward they and V' are kept and no output is formed.
hipError_t launch_rule_states(const RuleArgs& a, const RuleWs& w, bool backward, hipStream_t s);
// From what every segment adds and multiplies by, the state before every segment but the
// first, or in reverse the gradient of the state behind every one but the last.
hipError_t launch_rule_join(const RuleWs& w, bool reverse, hipStream_t s);

}  // namespace cgconv
