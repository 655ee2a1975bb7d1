// The orthogonalised update as lp_step_muon and the stand-alone entry points run it.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>

namespace lp {

struct OrthoProblem {
  int batch, rows, cols;
  bool g_bf16;            // type of g
  bool split;             // operands as high and low parts in all steps (ortho_two_parts); else X in the first ones
  const void* g;
  const long long* off;   // element offset of each matrix from g, momentum and out (host; at most kOrthoMaxOffsets matrices then),
                          // or null: one after another
  float* momentum;        // or null
  float mu;
  bool nesterov;
  int steps;
  float coeffs[3];
  float eps;
  void* out;              // result, or the weights that are updated
  bool out_bf16;
  bool update;            // out <- keep * out + step * O
  float keep, step;
  int* err;               // error word, or null: the first word of the scratch, cleared by the call
};

constexpr int kOrthoMaxOffsets = 64;
extern const float kOrthoCoeffs[3];
bool ortho_two_parts(int dtype, int rows, int cols);
size_t ortho_scratch_bytes(int batch, int rows, int cols, bool split);
// Enqueues the operator; `launches` (nullable) counts its kernels.
int ortho_run(const OrthoProblem& q, void* scratch, cudaStream_t st, long long* launches);

}  // namespace lp
