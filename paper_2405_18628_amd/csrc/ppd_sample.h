// Sampled acceptance (k_sample.hip).
#pragma once

#include "ppd_internal.h"

struct SamplePart {
  double rest;   // sum of exp((l - top) / temperature) without the node's drafted tokens: 0 or at least 1
  float top;     // the largest logit of those
  float m;       // the largest logit of the part (NaN left out)
  uint32_t nan;  // it holds a NaN
  uint32_t pad;
};

struct SampleNode {
  int taken;  // the accepted child, or -1
  int bonus;  // then the bonus token
  int bad;    // the row holds a NaN, or no weight at all
  int pad;
};

struct SampleLaunch {
  const int32_t *parent, *ids;
  int T, vocab;
  const float *logits, *draft, *u;
  float temperature;
  int32_t *path, *n_path, *next_tok;
  uint32_t *status;
  SamplePart *part;  // without draft: [T][parts]
  SampleNode *node;  // with draft: [T]
};
size_t sample_workspace_bytes(int T, int vocab);
hipError_t launch_sample(const SampleLaunch &p, hipStream_t s);
