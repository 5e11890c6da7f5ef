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

}  // namespace fp8
}  // namespace bsp
