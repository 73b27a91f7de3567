// Low-rank adapters of many requests (or of many training groups) beside one shared projection:
//
//   T_i = s_a B_a x_i,  y_i = W x_i + A_a T_i          U_i = s_a A_a^T dY_i,  dX_i = W^T dY_i + B_a^T U_i
//   dA_a = sum of dY_i T_i^T,  dB_a = sum of U_i x_i^T over the rows i with row_adapter[i] = a
//
// with a = row_adapter[i]; a row whose entry is no adapter has T_i = U_i = 0 and the shared projection alone.  This file has the entry
// points and the general path: any size, fp32 or bf16 storage, rows of adapters in any order.  Rows never mix: what one row or one
// adapter holds (infinities, NaN) reaches no other row's result and no other adapter's gradient, because every sum below runs
// over one row, or over the rows of one adapter, and nothing is masked by a multiplication with zero.
#include <string.h>

#include "ab_adapter.cuh"

namespace ab {
namespace {

bool have_device() {
  int n = 0;
  return cudaGetDeviceCount(&n) == cudaSuccess && n > 0;
}

constexpr int kProjThreads = 256;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// T[i][k] = s_a sum_j In[i][j] F_a(k, j), one block a row; F_a(k, j) at F + a strideF + k f_k + j f_j, one of f_k, f_j is 1: the lanes run
// along that one.  Partial sums of a lane in fp32, joined by a tree.
template <typename TI>
__global__ void __launch_bounds__(kProjThreads)
project_kernel(const TI* __restrict__ In, const TI* __restrict__ F, int64_t strideF, int64_t f_k, int64_t f_j,
               const float* __restrict__ scale, const int* __restrict__ ids, float* __restrict__ T, int K, int r, int L, int* status) {
  __shared__ float part[kProjThreads];
  const int64_t row = blockIdx.x;
  if (row == 0 && threadIdx.x == 0) *status = AB_OK;
  const int a = ids[row];
  float* Trow = T + row * r;
  if (a < 0 || a >= L) {
    for (int k = threadIdx.x; k < r; k += kProjThreads) Trow[k] = 0.f;
    return;
  }
  const float s = scale ? scale[a] : 1.f;
  const TI* x = In + row * (int64_t)K;
  const TI* Fa = F + a * strideF;
  if (f_j == 1) {
    for (int k = threadIdx.x >> 5; k < r; k += kProjThreads / 32) {
      const TI* f = Fa + k * f_k;
      float v = 0.f;
      for (int j = threadIdx.x & 31; j < K; j += 32) v = fmaf(to_f32(x[j]), to_f32(f[j]), v);
      v = warp_sum(v);
      if ((threadIdx.x & 31) == 0) Trow[k] = s * v;
    }
    return;
  }
  int kt = 1;
  while (kt < r && kt < kProjThreads) kt <<= 1;
  const int jp = kProjThreads / kt, kk = threadIdx.x % kt, j0 = threadIdx.x / kt;
  for (int k0 = 0; k0 < r; k0 += kt) {
    const int k = k0 + kk;
    float v = 0.f;
    if (k < r)
      for (int j = j0; j < K; j += jp) v = fmaf(to_f32(x[j]), to_f32(Fa[j * f_j + k]), v);
    part[threadIdx.x] = v;
    __syncthreads();
    for (int h = jp >> 1; h > 0; h >>= 1) {
      if (j0 < h) part[threadIdx.x] += part[threadIdx.x + h * kt];
      __syncthreads();
    }
    if (j0 == 0 && k < r) Trow[k] = s * part[kk];
    __syncthreads();
  }
}

// out[i][c] = base[i][c] + sum_k T[i][k] G_a(c, k), rounded once; G_a(c, k) at G + a strideG + c g_c + k g_k.  base may be out itself
// (fp32).  A map entry that is neither an adapter nor -1 is reported.
constexpr int kDeltaRows = 8, kDeltaCols = 256, kDeltaK = 64;
template <typename TI, typename TO>
__global__ void __launch_bounds__(kDeltaCols)
delta_kernel(const float* base, const float* __restrict__ T, const TI* __restrict__ G, int64_t strideG, int64_t g_c, int64_t g_k,
             const int* __restrict__ ids, TO* out, int64_t N, int P, int r, int L, int* status) {
  __shared__ float Ts[kDeltaRows][kDeltaK];
  __shared__ int id[kDeltaRows];
  const int64_t row0 = (int64_t)blockIdx.x * kDeltaRows;
  const int c = blockIdx.y * kDeltaCols + threadIdx.x;
  const int rows = (int)(N - row0 < kDeltaRows ? N - row0 : kDeltaRows);
  if (threadIdx.x < rows) {
    const int a = ids[row0 + threadIdx.x];
    if (a < -1 || a >= L) atomicExch(status, (int)AB_ERR_INVALID_ARG);
    id[threadIdx.x] = a >= 0 && a < L ? a : -1;
  }
  float acc[kDeltaRows];
#pragma unroll
  for (int i = 0; i < kDeltaRows; ++i) acc[i] = 0.f;
  for (int k0 = 0; k0 < r; k0 += kDeltaK) {
    const int kn = r - k0 < kDeltaK ? r - k0 : kDeltaK;
    __syncthreads();
    for (int e = threadIdx.x; e < rows * kDeltaK; e += kDeltaCols)
      if (e % kDeltaK < kn) Ts[e / kDeltaK][e % kDeltaK] = T[(row0 + e / kDeltaK) * r + k0 + e % kDeltaK];
    __syncthreads();
    if (c < P) {
#pragma unroll
      for (int i = 0; i < kDeltaRows; ++i) {
        if (i >= rows || id[i] < 0) continue;
        const TI* g = G + id[i] * strideG + c * g_c + k0 * g_k;
        float v = acc[i];
        for (int k = 0; k < kn; ++k) v = fmaf(Ts[i][k], to_f32(g[k * g_k]), v);
        acc[i] = v;
      }
    }
  }
  if (c >= P) return;
#pragma unroll
  for (int i = 0; i < kDeltaRows; ++i) {
    if (i >= rows) continue;
    const int64_t o = (row0 + i) * P + c;
    if (id[i] >= 0) from_f32(out[o], base[o] + acc[i]);
    else if ((const void*)base != (const void*)out) from_f32(out[o], base[o]);
  }
}

// The rows of each adapter in ascending order: adapter a's are order[start[a] .. start[a] + count[a]).  One block an adapter: it counts the
// rows of the adapters before it, then lists its own.
constexpr int kListThreads = 512;
__global__ void __launch_bounds__(kListThreads)
list_rows_kernel(const int* __restrict__ ids, int64_t N, int L, int* __restrict__ order, int64_t* __restrict__ start,
                 int64_t* __restrict__ count, int* status, int clear_status) {
  __shared__ int warp_cnt[kListThreads / 32];
  __shared__ int64_t before;
  const int a = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long less = 0;
  int bad = 0;
  for (int64_t i = threadIdx.x; i < N; i += kListThreads) {
    const int v = ids[i];
    less += (v >= 0 && v < a) ? 1 : 0;
    bad |= (v < -1 || v >= L) ? 1 : 0;
  }
  if (threadIdx.x == 0) before = 0;
  bad = __syncthreads_or(bad);
  if (a == 0 && threadIdx.x == 0 && (bad || clear_status)) *status = bad ? (int)AB_ERR_INVALID_ARG : (int)AB_OK;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) less += __shfl_xor_sync(0xffffffffu, less, o);
  if (lane == 0) atomicAdd(reinterpret_cast<unsigned long long*>(&before), (unsigned long long)less);
  __syncthreads();
  const int64_t first = before;
  int64_t at = first;
  for (int64_t i0 = 0; i0 < N; i0 += kListThreads) {
    const int64_t i = i0 + threadIdx.x;
    const bool mine = i < N && ids[i] == a;
    const unsigned vote = __ballot_sync(0xffffffffu, mine);
    if (lane == 0) warp_cnt[warp] = __popc(vote);
    __syncthreads();
    int ahead = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kListThreads / 32; ++w) {
      const int c = warp_cnt[w];
      ahead += w < warp ? c : 0;
      all += c;
    }
    if (mine) order[at + ahead + __popc(vote & ((1u << lane) - 1u))] = (int)i;
    at += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) { start[a] = first; count[a] = at - first; }
}

// D_a(f, k) = sum over the rows i of adapter a of In[i][f] S[i][k], at D + a strideD + f d_f + k d_k.  A block has 64 values of f and 32
// of k of one adapter; rows in their order, 32 at a time in fp32, those sums in fp64: a long sum loses nothing that fp32 shows.
constexpr int kGF = 64, kGK = 32, kGR = 32;
template <typename TI>
__global__ void __launch_bounds__(256)
adapter_grad_kernel(const TI* __restrict__ In, int P, const float* __restrict__ S, int r, const int* __restrict__ order,
                    const int64_t* __restrict__ start, const int64_t* __restrict__ count, float* __restrict__ D, int64_t strideD, int64_t d_f,
                    int64_t d_k) {
  __shared__ float Is[kGR][kGF];
  __shared__ float4 Ss[kGR][kGK / 4];
  __shared__ int rows[kGR];
  const int f0 = blockIdx.x * kGF, k0 = blockIdx.y * kGK, a = blockIdx.z;
  const int f = threadIdx.x % kGF, kq = threadIdx.x / kGF;      // this thread: column f, values 8 kq .. 8 kq + 7
  const int64_t n = count[a];
  const int* mine = order + start[a];
  double acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0;
  for (int64_t i0 = 0; i0 < n; i0 += kGR) {
    const int rn = (int)(n - i0 < kGR ? n - i0 : kGR);
    __syncthreads();
    if (threadIdx.x < rn) rows[threadIdx.x] = mine[i0 + threadIdx.x];
    __syncthreads();
    for (int e = threadIdx.x; e < rn * kGF; e += 256) {
      const int q = e / kGF, c = e % kGF;
      Is[q][c] = f0 + c < P ? to_f32(In[(int64_t)rows[q] * P + f0 + c]) : 0.f;
    }
    for (int e = threadIdx.x; e < rn * kGK; e += 256) {
      const int q = e / kGK, c = e % kGK;
      reinterpret_cast<float*>(&Ss[q][0])[c] = k0 + c < r ? S[(int64_t)rows[q] * r + k0 + c] : 0.f;
    }
    __syncthreads();
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
    for (int q = 0; q < rn; ++q) {
      const float xi = Is[q][f];
      const float4 s0 = Ss[q][2 * kq], s1 = Ss[q][2 * kq + 1];
      v[0] = fmaf(xi, s0.x, v[0]); v[1] = fmaf(xi, s0.y, v[1]); v[2] = fmaf(xi, s0.z, v[2]); v[3] = fmaf(xi, s0.w, v[3]);
      v[4] = fmaf(xi, s1.x, v[4]); v[5] = fmaf(xi, s1.y, v[5]); v[6] = fmaf(xi, s1.z, v[6]); v[7] = fmaf(xi, s1.w, v[7]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += (double)v[e];
  }
  if (f0 + f >= P) return;
  float* d = D + a * strideD + (f0 + f) * d_f;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (k0 + 8 * kq + e < r) d[(k0 + 8 * kq + e) * d_k] = (float)acc[e];
}

typedef AdapterCall Call;

// Workspace of the general path: status word, T, U, base of a bf16 result in fp32, the adapters' rows
struct GeneralWs { int* status; float *T, *U, *base; int* order; int64_t *start, *count; size_t bytes; };
GeneralWs general_ws(void* ws, int64_t N, int m, int n, int r, int L, int dt) {
  Arena ar(ws, 0);
  GeneralWs w;
  w.status = ar.take_n<int>(64);
  w.T = ar.take_n<float>((size_t)N * r);
  w.U = ar.take_n<float>((size_t)N * r);
  w.base = dt == AB_BF16 ? ar.take_n<float>((size_t)N * (m > n ? m : n)) : nullptr;
  w.order = ar.take_n<int>((size_t)N);
  w.start = ar.take_n<int64_t>((size_t)L);
  w.count = ar.take_n<int64_t>((size_t)L);
  w.bytes = align_up(ar.used, 256);
  return w;
}

int project(const Call& c, const void* In, int K, const void* F, int64_t strideF, int64_t f_k, int64_t f_j, float* T, int* status) {
  if (c.dt == AB_F32)
    project_kernel<float><<<(unsigned)c.N, kProjThreads, 0, c.st>>>(static_cast<const float*>(In), static_cast<const float*>(F), strideF, f_k, f_j,
                                                                    c.scale, c.ids, T, K, c.r, c.L, status);
  else
    project_kernel<bf16><<<(unsigned)c.N, kProjThreads, 0, c.st>>>(static_cast<const bf16*>(In), static_cast<const bf16*>(F), strideF, f_k, f_j,
                                                                   c.scale, c.ids, T, K, c.r, c.L, status);
  AB_LAUNCH_OK();
  return AB_OK;
}

int add_delta(const Call& c, const float* base, const float* T, const void* G, int64_t strideG, int64_t g_c, int64_t g_k, void* out, int P,
              int* status) {
  const dim3 grid((unsigned)((c.N + kDeltaRows - 1) / kDeltaRows), (unsigned)((P + kDeltaCols - 1) / kDeltaCols));
  if (c.dt == AB_F32)
    delta_kernel<float, float><<<grid, kDeltaCols, 0, c.st>>>(base, T, static_cast<const float*>(G), strideG, g_c, g_k, c.ids, static_cast<float*>(out),
                                                              c.N, P, c.r, c.L, status);
  else
    delta_kernel<bf16, bf16><<<grid, kDeltaCols, 0, c.st>>>(base, T, static_cast<const bf16*>(G), strideG, g_c, g_k, c.ids, static_cast<bf16*>(out),
                                                            c.N, P, c.r, c.L, status);
  AB_LAUNCH_OK();
  return AB_OK;
}

int grad(const Call& c, const GeneralWs& w, const void* In, int P, const float* S, float* D, int64_t strideD, int64_t d_f, int64_t d_k) {
  for (int a0 = 0; a0 < c.L; a0 += 65535) {
    const dim3 grid((unsigned)((P + kGF - 1) / kGF), (unsigned)((c.r + kGK - 1) / kGK), (unsigned)(c.L - a0 < 65535 ? c.L - a0 : 65535));
    if (c.dt == AB_F32)
      adapter_grad_kernel<float><<<grid, 256, 0, c.st>>>(static_cast<const float*>(In), P, S, c.r, w.order, w.start + a0, w.count + a0, D + a0 * strideD,
                                                         strideD, d_f, d_k);
    else
      adapter_grad_kernel<bf16><<<grid, 256, 0, c.st>>>(static_cast<const bf16*>(In), P, S, c.r, w.order, w.start + a0, w.count + a0, D + a0 * strideD,
                                                        strideD, d_f, d_k);
    AB_LAUNCH_OK();
  }
  return AB_OK;
}

int general_forward(const Call& c, void* y, float* T_save, const GeneralWs& w) {
  float* T = T_save ? T_save : w.T;
  AB_TRY(project(c, c.x, c.n, c.B, c.strideB, c.n, 1, T, w.status));
  float* base = c.dt == AB_F32 ? static_cast<float*>(y) : w.base;
  AB_TRY(gemm_simt(c.x, c.dt, c.n, 1, c.W, c.dt, 1, c.n, base, AB_F32, c.m, c.N, c.m, c.n, c.st));
  return add_delta(c, base, T, c.A, c.strideA, c.r, 1, y, c.m, w.status);
}

int general_backward(const Call& c, const void* dY, const float* T_saved, void* dX, float* dA, float* dB, const GeneralWs& w) {
  const bool want_U = dX || dB;
  if (want_U) AB_TRY(project(c, dY, c.m, c.A, c.strideA, 1, c.r, w.U, w.status));
  if (dA && !T_saved) AB_TRY(project(c, c.x, c.n, c.B, c.strideB, c.n, 1, w.T, w.status));
  if (dX) {
    float* base = c.dt == AB_F32 ? static_cast<float*>(dX) : w.base;
    AB_TRY(gemm_simt(dY, c.dt, c.m, 1, c.W, c.dt, c.n, 1, base, AB_F32, c.n, c.N, c.n, c.m, c.st));
    AB_TRY(add_delta(c, base, w.U, c.B, c.strideB, 1, c.n, dX, c.n, w.status));
  }
  if (!dA && !dB) return AB_OK;
  list_rows_kernel<<<(unsigned)c.L, kListThreads, 0, c.st>>>(c.ids, c.N, c.L, w.order, w.start, w.count, w.status,
                                                             !want_U && (!dA || T_saved) ? 1 : 0);
  AB_LAUNCH_OK();
  if (dA) AB_TRY(grad(c, w, dY, c.m, T_saved ? T_saved : w.T, dA, (int64_t)c.m * c.r, c.r, 1));
  if (dB) AB_TRY(grad(c, w, c.x, c.n, w.U, dB, (int64_t)c.r * c.n, 1, c.n));
  return AB_OK;
}

int check_args(const Call& c) {
  if (!dtype_ok(c.dt) || c.N < 0 || c.m <= 0 || c.n <= 0 || c.r <= 0 || c.L <= 0) return AB_ERR_INVALID_ARG;
  if (c.r > c.m || c.r > c.n) return AB_ERR_INVALID_ARG;
  if (!c.A || !c.B || (c.N > 0 && (!c.x || !c.ids))) return AB_ERR_INVALID_ARG;
  if (c.L > 1 && (c.strideA < (int64_t)c.m * c.r || c.strideB < (int64_t)c.r * c.n)) return AB_ERR_INVALID_ARG;
  const size_t e = dtype_size(c.dt);
  if (!aligned(c.x, e) || !aligned(c.W, e) || !aligned(c.A, e) || !aligned(c.B, e) || !aligned(c.ids, 4) || !aligned(c.scale, 4))
    return AB_ERR_INVALID_ARG;
  if (c.N > 0x7fffffffll) return AB_ERR_UNSUPPORTED;      // rows are counted in 32 bits
  return AB_OK;
}

}  // namespace
}  // namespace ab

using namespace ab;

extern "C" {

size_t ab_adapter_workspace_bytes(int64_t N, int m, int n, int r, int L, int dt) {
  if (N < 0 || N > 0x7fffffffll || m <= 0 || n <= 0 || r <= 0 || L <= 0 || !dtype_ok(dt)) return 0;
  const size_t g = general_ws(nullptr, N, m, n, r, L, dt).bytes;
  const size_t t = adapter_tc_shape_ok(N, m, n, r, L, dt) ? adapter_tc_ws(N, m, n, r, L) : 0;
  return (g > t ? g : t) + 256;
}

int ab_adapter_forward(const void* x, const void* W, const void* A, const void* B, const float* scale, const int* row_adapter,
                       void* y, float* T_save, int64_t N, int m, int n, int r, int L, int64_t strideA, int64_t strideB, int dt,
                       void* ws, size_t ws_bytes, void* cuda_stream) {
  const Call c{x, W, A, B, scale, row_adapter, N, m, n, r, L, strideA, strideB, dt, static_cast<cudaStream_t>(cuda_stream)};
  AB_TRY(check_args(c));
  if (!W || (N > 0 && !y) || !aligned(y, dtype_size(dt)) || !aligned(T_save, 4)) return AB_ERR_INVALID_ARG;
  if (!have_device()) return AB_ERR_CUDA;
  if (N == 0) return AB_OK;
  if (!ws || !aligned(ws, 256)) return AB_ERR_WORKSPACE;
  if (adapter_tc_supported(c, nullptr, y, T_save, nullptr, nullptr)) {
    if (adapter_tc_ws(N, m, n, r, L) > ws_bytes) return AB_ERR_WORKSPACE;
    return adapter_tc_forward(c, y, T_save, ws);
  }
  const GeneralWs w = general_ws(ws, N, m, n, r, L, dt);
  if (w.bytes > ws_bytes) return AB_ERR_WORKSPACE;
  return general_forward(c, y, T_save, w);
}

int ab_adapter_backward(const void* x, const void* dY, const void* W, const void* A, const void* B, const float* scale,
                        const int* row_adapter, const float* T_saved, void* dX, float* dA, float* dB, int64_t N, int m, int n, int r,
                        int L, int64_t strideA, int64_t strideB, int dt, void* ws, size_t ws_bytes, void* cuda_stream) {
  const Call c{x, W, A, B, scale, row_adapter, N, m, n, r, L, strideA, strideB, dt, static_cast<cudaStream_t>(cuda_stream)};
  AB_TRY(check_args(c));
  const size_t e = dtype_size(dt);
  if ((N > 0 && !dY) || (dX && !W) || !aligned(dY, e) || !aligned(dX, e) || !aligned(T_saved, 4) || !aligned(dA, 4) || !aligned(dB, 4))
    return AB_ERR_INVALID_ARG;
  if (!have_device()) return AB_ERR_CUDA;
  if (N == 0) {   // empty batch: the sums over the rows are empty
    if (dA) AB_CUDA_OK(cudaMemsetAsync(dA, 0, (size_t)L * m * r * sizeof(float), c.st));
    if (dB) AB_CUDA_OK(cudaMemsetAsync(dB, 0, (size_t)L * r * n * sizeof(float), c.st));
    return AB_OK;
  }
  if (!ws || !aligned(ws, 256)) return AB_ERR_WORKSPACE;
  if (!dX && !dA && !dB) {
    if (ws_bytes < sizeof(int)) return AB_ERR_WORKSPACE;
    AB_CUDA_OK(cudaMemsetAsync(ws, 0, sizeof(int), c.st));
    return AB_OK;
  }
  if (adapter_tc_supported(c, dY, dX, T_saved, dA, dB)) {
    if (adapter_tc_ws(N, m, n, r, L) > ws_bytes) return AB_ERR_WORKSPACE;
    return adapter_tc_backward(c, dY, T_saved, dX, dA, dB, ws);
  }
  const GeneralWs w = general_ws(ws, N, m, n, r, L, dt);
  if (w.bytes > ws_bytes) return AB_ERR_WORKSPACE;
  return general_backward(c, dY, T_saved, dX, dA, dB, w);
}

}  // extern "C"
