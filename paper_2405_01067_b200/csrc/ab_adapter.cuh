// What the entry points of the adapters (ab_adapter.cu) and their tensor-core path (ab_adapter_tc.cu) share.
#pragma once

#include "ab_common.cuh"

namespace ab {

struct AdapterCall {
  const void *x, *W, *A, *B;
  const float* scale;
  const int* ids;
  int64_t N;
  int m, n, r, L;
  int64_t strideA, strideB;
  int dt;
  cudaStream_t st;
};

// dA[i], dB[i] = sum of the slices at p[s * count + i], in their order; a result may be NULL (ab_adapter.cu)
int adapter_add_slices(const float* pA, float* dA, int64_t ea, const float* pB, float* dB, int64_t eb, int slices, cudaStream_t st);
// sizes alone: what the workspace is for
bool adapter_tc_lists_ok(int64_t N, int L);
bool adapter_tc_shape_ok(int64_t N, int m, int n, int r, int L, int dt);
bool adapter_tc_supported(const AdapterCall& c, const void* dY, const void* out, const float* T, const float* dA, const float* dB);
int adapter_tc_form(int64_t N, int P, int K);
size_t adapter_tc_ws(int64_t N, int m, int n, int r, int L);
int adapter_tc_forward(const AdapterCall& c, void* y, float* T_save, void* ws);
int adapter_tc_backward(const AdapterCall& c, const void* dY, const float* T_saved, void* dX, float* dA, float* dB, void* ws);

}  // namespace ab
