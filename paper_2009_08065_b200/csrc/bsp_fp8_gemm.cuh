// Products of two 8-bit operands, out[i, j] = act(sum_k A(i, k) B(j, k) + bias[j]) * keep[i / block, j], and the kernels that compute them.
#pragma once

#include "bsp_fp8.cuh"

namespace bsp {
namespace fp8 {

struct Product {
  Operand A, B;
  int contraction;
  uint16_t* Y;               // bf16 [A.rows, B.rows]
  int ldy;
  const uint16_t* bias;      // bf16 [B.rows], or null
  int act;
  const uint8_t* keep;       // flags [A.rows / block, B.rows], or null
  int block;
};

// bsp_gemm_fp8.cu: operands whose rows begin at multiples of 16 bytes.
bool tensor_core_ok(const Product& p);
int launch_tensor_core(const Product& p, cudaStream_t s);

// bsp_fp8_few.cu: the forward product for few tokens, from up to 32 of bf16 and up to 16 of 8-bit ones (of any 16-byte aligned rows).
constexpr int kFewTokens = 32, kFewReady = 16;
bool few_tokens_ok(const void* Wq, int ldw, int tokens);
int launch_few(const void* Wq, int ldw, const uint8_t* WS, int ldws, int n_out, int k_in, const void* X, int tokens, int ldx, const void* bias, int act,
               void* Y, int ldy, cudaStream_t s);
int launch_few_ready(const Product& p, cudaStream_t s);

}  // namespace fp8
}  // namespace bsp
