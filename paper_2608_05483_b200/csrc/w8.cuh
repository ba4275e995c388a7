// Shared by the translation units of the 8-bit calls (norm8.cu, gemm8.cu).
#pragma once

#include "paged.cuh"

namespace plora {
namespace w8 {

constexpr int kBlock = 128;      // columns (and, of a weight, rows) that share a scale

// The current device and its SMs (looked up once per device).
cudaError_t device(paged::Device& dev);

}  // namespace w8
}  // namespace plora
