// The linear layer's three products (forward, input gradient, weight gradient): what the engines have in common.
#pragma once

#include "sc_act8.cuh"

namespace sc {

// What happens to a finished sum before it is stored.
//   kEpiForward   z = acc + bias[col]; z -> checkpoint (if q); y = act(z) + res
//   kEpiInput     acc * act'(value of the checkpoint) (if q), else acc
//   kEpiWeight    acc * scale
enum EpiKind { kEpiForward = 0, kEpiInput = 1, kEpiWeight = 2 };

struct LinEpilogue {
  void* out;                // rows of D, out_f32 ? fp32 : bf16
  const float* bias;        // forward: one per column of D, or null
  const void* res;          // forward: same type as out, or null
  int8_t* q;                // forward: written; input: read; or null
  uint8_t* e;
  int64_t wide;             // columns of D rounded up to 32; the checkpoint's tokens are the rows of D
  int64_t ldo, ldr;
  int out_f32;
  int act;
  float scale;
  const void* dy;           // weight, tensor-core engine: db = column sums of dy (tokens x rows of D), or db null
  float* db;
  int64_t tokens, ld_dy;
};

// D[m x n] = sum_k A(m, k) B(n, k); element (i, k) of an operand is at base[i * s_row + k * s_k], one stride is 1.
struct LinOperand {
  const void* base;
  int64_t s_row, s_k;
};

struct LinProblem {
  LinOperand A, B;
  int64_t M, N, K;
  LinEpilogue epi;
};

// Tensor-core engine: bf16 operands that TMA can describe (16-byte aligned base and row stride).
bool linear_tc_supported(const LinProblem& p);
sc_status linear_tc(int kind, const LinProblem& p, unsigned* status, cudaStream_t s);

sc_status linear_simt(int kind, int operand_f32, const LinProblem& p, cudaStream_t s);

}  // namespace sc
