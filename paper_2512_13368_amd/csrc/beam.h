// Beam search's selection: kernel-side description of a call (gfx950 only).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace blossom {
namespace beam {

constexpr int kMost = 64;      // beams of a history, and continuations chosen
constexpr int kLists = 1024;   // runs of all of a history's rows

struct Args {
  int B, W, K, V, dtype, eos;
  const void *logits;          // [B W, V] rows
  int64_t stride;              // elements from a row to the next
  const float *score;          // [B, W]
  const unsigned char *ended;  // [B, W] or nullptr
  int *parent, *token;         // [B, K]
  float *out_score;
  unsigned char *out_ended;    // or nullptr
  int loads, subs, lists;      // 16-byte loads of a lane and piece, pieces of a run, runs of a row (0: a history is done by one workgroup)
  double2 *stats;              // [B W, lists] largest logit and sum of exponentials, in the workspace
  unsigned long long *lists_of;  // [B W, lists, K] best logits with their items, there too
};

void plan(Args &a);
bool launch(const Args &a, hipStream_t st);

}  // namespace beam
}  // namespace blossom
