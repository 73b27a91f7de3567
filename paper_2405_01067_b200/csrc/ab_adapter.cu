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
#include "ab_tc_ptx.cuh"

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

// T[i][k] = s_a sum_j In[i][j] F_a(k, j), kRB rows a block; F_a(k, j) at F + a strideF + k f_k + j f_j, one of f_k, f_j is 1: the lanes run
// along that one.  Neighbouring rows mostly have the same adapter: F_a is then read once for all of the block's rows (1531 rows, r 12, 777
// wide: 12.8 us a row a block).  Partial sums of a lane in fp32, joined by a tree: the bits of a row do not depend on its neighbours.
template <typename TI, int kRB>
__global__ void __launch_bounds__(kProjThreads)
project_kernel(const TI* __restrict__ In, const TI* __restrict__ F, int64_t strideF, int64_t f_k, int64_t f_j,
               const float* __restrict__ scale, const int* __restrict__ ids, float* __restrict__ T, int64_t N, int K, int r, int L, int first,
               int* status) {
  __shared__ float part[kRB][kProjThreads];
  tc::dep_wait();
  tc::dep_launch();
  const int64_t row0 = (int64_t)blockIdx.x * kRB;
  if (first && row0 == 0 && threadIdx.x == 0) *status = AB_OK;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int id[kRB];
#pragma unroll
  for (int i = 0; i < kRB; ++i) {
    const int a = row0 + i < N ? ids[row0 + i] : -1;
    id[i] = a >= 0 && a < L ? a : -1;
    if (id[i] < 0 && row0 + i < N)
      for (int k = threadIdx.x; k < r; k += kProjThreads) T[(row0 + i) * r + k] = 0.f;
  }
#pragma unroll 1
  for (int h = 0; h < kRB; ++h) {            // a pass for each adapter of the block
    int a = -1;
    unsigned mine = 0;
#pragma unroll
    for (int i = 0; i < kRB; ++i) {
      bool seen = false;
#pragma unroll
      for (int e = 0; e < kRB; ++e) seen |= e < h && id[e] == id[i];
      if (i == h && !seen) a = id[i];
    }
    if (a < 0) continue;
#pragma unroll
    for (int i = 0; i < kRB; ++i) mine |= id[i] == a ? 1u << i : 0u;
    const float s = scale ? scale[a] : 1.f;
    const TI* x = In + row0 * (int64_t)K;
    const TI* Fa = F + a * strideF;
    const int last = (int)(N - row0 < kRB ? N - row0 : kRB) - 1;
    if (f_j == 1) {
      for (int k = warp; k < r; k += kProjThreads / 32) {
        const TI* f = Fa + k * f_k;
        float v[kRB];
#pragma unroll
        for (int i = 0; i < kRB; ++i) v[i] = 0.f;
#pragma unroll 4
        for (int j = lane; j < K; j += 32) {
          const float w = to_f32(f[j]);
#pragma unroll
          for (int i = 0; i < kRB; ++i) v[i] = fmaf(to_f32(x[(int64_t)(i < last ? i : last) * K + j]), w, v[i]);
        }
#pragma unroll
        for (int i = 0; i < kRB; ++i) {
          const float t = warp_sum(v[i]);
          if (lane == 0 && ((mine >> i) & 1u)) T[(row0 + i) * r + k] = s * t;
        }
      }
      continue;
    }
    int kt = 1;
    while (kt < r && kt < kProjThreads) kt <<= 1;
    const int jp = kProjThreads / kt, kk = threadIdx.x % kt, j0 = threadIdx.x / kt;
    for (int k0 = 0; k0 < r; k0 += kt) {
      const int k = k0 + kk;
      float v[kRB];
#pragma unroll
      for (int i = 0; i < kRB; ++i) v[i] = 0.f;
      if (k < r) {
#pragma unroll 4
        for (int j = j0; j < K; j += jp) {
          const float w = to_f32(Fa[j * f_j + k]);
#pragma unroll
          for (int i = 0; i < kRB; ++i) v[i] = fmaf(to_f32(x[(int64_t)(i < last ? i : last) * K + j]), w, v[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < kRB; ++i) part[i][threadIdx.x] = v[i];
      __syncthreads();
      for (int g = jp >> 1; g > 0; g >>= 1) {
        if (j0 < g) {
#pragma unroll
          for (int i = 0; i < kRB; ++i) part[i][threadIdx.x] += part[i][threadIdx.x + g * kt];
        }
        __syncthreads();
      }
      if (j0 == 0 && k < r) {
#pragma unroll
        for (int i = 0; i < kRB; ++i)
          if ((mine >> i) & 1u) T[(row0 + i) * r + k] = s * part[i][kk];
      }
      __syncthreads();
    }
  }
}

// out[i][c] = sum over the slices of base + sum_k T[i][k] G_a(c, k), rounded once; G_a(c, k) at G + a strideG + c g_c + k g_k.  base may be
// out itself (fp32, one slice).  A map entry that is neither an adapter nor -1 is reported.  A thread has a column and kRD rows; sixteen
// of G's values at a time are in registers, and stay there while the next row has the same adapter.  Where G_a's rows run along k
// (g_k 1), they come by way of shared memory: read by column, a warp's load would touch 32 lines.
constexpr int kDeltaCols = 256, kDeltaK = 64;
template <typename TI, typename TO, int kRD>
__global__ void __launch_bounds__(kDeltaCols)
delta_kernel(const float* base, int slices, const float* __restrict__ T, const TI* __restrict__ G, int64_t strideG, int64_t g_c, int64_t g_k,
             const int* __restrict__ ids, TO* out, int64_t N, int P, int r, int L, int* status) {
  __shared__ float Ts[kRD][kDeltaK];
  __shared__ float Gs[kDeltaCols][17];
  __shared__ int id[kRD];
  tc::dep_wait();
  tc::dep_launch();
  const int64_t row0 = (int64_t)blockIdx.x * kRD;
  const int c = blockIdx.y * kDeltaCols + threadIdx.x, cc = c < P ? c : P - 1;
  const int rows = (int)(N - row0 < kRD ? N - row0 : kRD);
  if (threadIdx.x < kRD) {
    const int a = threadIdx.x < rows ? ids[row0 + threadIdx.x] : -1;
    if (a < -1 || a >= L) atomicExch(status, (int)AB_ERR_INVALID_ARG);
    id[threadIdx.x] = a >= 0 && a < L ? a : -1;
  }
  float acc[kRD];
#pragma unroll
  for (int i = 0; i < kRD; ++i) acc[i] = 0.f;
  for (int k0 = 0; k0 < r; k0 += kDeltaK) {
    const int kn = r - k0 < kDeltaK ? r - k0 : kDeltaK;
    __syncthreads();
    for (int e = threadIdx.x; e < rows * kDeltaK; e += kDeltaCols)
      Ts[e / kDeltaK][e % kDeltaK] = e % kDeltaK < kn ? T[(row0 + e / kDeltaK) * r + k0 + e % kDeltaK] : 0.f;
    __syncthreads();
    for (int k1 = 0; k1 < kn; k1 += 16) {
      float g[16];
      int have = -1;
#pragma unroll
      for (int i = 0; i < kRD; ++i) {
        if (i >= rows || id[i] < 0) continue;
        if (id[i] != have) {
          have = id[i];
          if (g_k == 1) {
            const TI* q = G + have * strideG + k0 + k1;
            const int c0 = blockIdx.y * kDeltaCols, e = threadIdx.x & 15;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kDeltaCols / 16; ++u) {
              const int col = u * 16 + (threadIdx.x >> 4);
              Gs[col][e] = c0 + col < P && k1 + e < kn ? to_f32(q[(c0 + col) * g_c + e]) : 0.f;
            }
            __syncthreads();
#pragma unroll
            for (int i2 = 0; i2 < 16; ++i2) g[i2] = Gs[threadIdx.x][i2];
          } else {
            const TI* q = G + have * strideG + cc * g_c + (k0 + k1) * g_k;
#pragma unroll
            for (int e = 0; e < 16; ++e) g[e] = k1 + e < kn ? to_f32(q[e * g_k]) : 0.f;
          }
        }
        float v = acc[i];
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const float4 t = *reinterpret_cast<const float4*>(&Ts[i][k1 + e]);
          v = fmaf(t.x, g[e], v); v = fmaf(t.y, g[e + 1], v); v = fmaf(t.z, g[e + 2], v); v = fmaf(t.w, g[e + 3], v);
        }
        acc[i] = v;
      }
    }
  }
  if (c >= P) return;
  float v[kRD];
#pragma unroll
  for (int i = 0; i < kRD; ++i) v[i] = i < rows ? base[(row0 + i) * P + c] : 0.f;
  for (int s = 1; s < slices; ++s) {
    const float* q = base + s * N * P + row0 * P + c;
#pragma unroll
    for (int i = 0; i < kRD; ++i) v[i] += i < rows ? q[(int64_t)i * P] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < kRD; ++i)
    if (i < rows) from_f32(out[(row0 + i) * P + c], id[i] >= 0 ? v[i] + acc[i] : v[i]);
}

// The rows of each adapter in ascending order: adapter a's are order[start[a] .. start[a] + count[a]).  One block an adapter: it counts the
// rows of the adapters before it, then lists its own.
constexpr int kListThreads = 512;
__global__ void __launch_bounds__(kListThreads)
list_rows_kernel(const int* __restrict__ ids, int64_t N, int L, int* __restrict__ order, int64_t* __restrict__ start,
                 int64_t* __restrict__ count, int* status, int clear_status) {
  __shared__ int warp_cnt[kListThreads / 32];
  __shared__ int64_t before;
  tc::dep_wait();
  tc::dep_launch();
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

// D_a(f, k) = sum over the rows i of adapter a of In[i][f] S[i][k], at D + a strideD + f d_f + k d_k, for one or two such gradients.  A block
// has 64 values of f and 32 of k of one adapter; rows in their order, 64 at a time in fp32, those sums in fp64: a long sum loses
// nothing that fp32 shows.
constexpr int kGF = 64, kGK = 32, kGR = 64;
struct GradSide { const void* In; int P, tiles; const float* S; float* D; int64_t strideD, d_f, d_k, slice; };      // slice: from slice to slice
struct GradSides { GradSide side[2]; };
template <typename TI>
__global__ void __launch_bounds__(256)
adapter_grad_kernel(const __grid_constant__ GradSides sides, int r, const int* __restrict__ order, const int64_t* __restrict__ start,
                    const int64_t* __restrict__ count, int slices) {
  __shared__ float Is[kGR][kGF];
  __shared__ float4 Ss[kGR][kGK / 4];
  __shared__ int rows[kGR];
  tc::dep_wait();
  tc::dep_launch();
  const int second = (int)blockIdx.x >= sides.side[0].tiles ? 1 : 0;
  const GradSide& w = sides.side[second];
  const TI* In = static_cast<const TI*>(w.In);
  const int P = w.P;
  const int f0 = ((int)blockIdx.x - (second ? sides.side[0].tiles : 0)) * kGF, k0 = blockIdx.y * kGK;
  const int a = (int)blockIdx.z / slices, part = (int)blockIdx.z - a * slices;
  const int f = threadIdx.x % kGF, kq = threadIdx.x / kGF;      // this thread: column f, values 8 kq .. 8 kq + 7
  // this slice's rows, whole blocks of kGR
  const int64_t all = count[a], per = ((all + slices - 1) / slices + kGR - 1) / kGR * kGR, from = part * per < all ? part * per : all;
  const int64_t n = all - from < per ? all - from : per;
  const int* mine = order + start[a] + from;
  double acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0;
  for (int64_t i0 = 0; i0 < n; i0 += kGR) {
    const int rn = (int)(n - i0 < kGR ? n - i0 : kGR);
    __syncthreads();
    if (threadIdx.x < rn) rows[threadIdx.x] = mine[i0 + threadIdx.x];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kGR * kGF / 256; ++u) {
      const int e = threadIdx.x + u * 256, q = e / kGF, c = e % kGF;
      Is[q][c] = q < rn && f0 + c < P ? to_f32(In[(int64_t)rows[q] * P + f0 + c]) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < kGR * kGK / 256; ++u) {
      const int e = threadIdx.x + u * 256, q = e / kGK, c = e % kGK;
      reinterpret_cast<float*>(&Ss[q][0])[c] = q < rn && k0 + c < r ? w.S[(int64_t)rows[q] * r + k0 + c] : 0.f;
    }
    __syncthreads();
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll 8
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
  float* d = w.D + part * w.slice + a * w.strideD + (f0 + f) * w.d_f;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (k0 + 8 * kq + e < r) d[(k0 + 8 * kq + e) * w.d_k] = (float)acc[e];
}

// out[i] = sum over the slices, in their order, for one or two results in one launch
struct SliceSide { const float* part; float* out; int64_t count; };
__global__ void __launch_bounds__(256)
add_slices_kernel(SliceSide x, SliceSide y, int slices) {
  tc::dep_wait();
  tc::dep_launch();
  int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const bool second = i >= x.count;
  if (second) i -= x.count;
  const SliceSide& w = second ? y : x;
  if (i >= w.count) return;
  float v = 0.f;
  for (int s0 = 0; s0 < slices; s0 += 8) {
    float u[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) u[s] = s0 + s < slices ? __ldcg(w.part + (s0 + s) * w.count + i) : 0.f;
#pragma unroll
    for (int s = 0; s < 8; ++s) v += u[s];
  }
  w.out[i] = v;
}

typedef AdapterCall Call;

// The shared product in fp32 goes to the tensor cores as six bf16 terms (one where the storage is bf16), which cut their sums off at every
// step: reductions above 768 are cut into slices (777: 7.4e-7 of the result in one, 5e-7 is what fp32 fused multiply-adds lose;
// 3900: 4.2e-6), whose sums delta_kernel adds.  Above that as many slices as leave the busiest SM the fewest slabs of 64, a tile's start
// and end counted as two, a slice's way through memory as one.
int base_slices(int64_t N, int P, int K) {
  const int sms = sm_count() > 0 ? sm_count() : 148;
  const int least = (K + 767) / 768 < kSplitFew ? (K + 767) / 768 : kSplitFew;
  const int64_t tiles = (N + 127) / 128 * ((P + 127) / 128);
  int best = least;
  int64_t best_t = INT64_MAX;
  for (int s = least; s <= kSplitFew && (s == least || s * 128 <= K); ++s) {
    const int64_t t = (tiles * s + sms - 1) / sms * ((K + 64 * s - 1) / (64 * s) + 2) + s;
    if (t < best_t) { best_t = t; best = s; }
  }
  return best;
}
// The slices lie in the workspace for a band of rows at a time, of as many rows as it holds, bands of one length; the bits do not depend on it.  What
// the query asks for is bounded: up to 1 GB for sizes that always come here, 64 MB beside the tensor-core path, whose sizes come here
// for misaligned pointers alone.  (8191 rows, 4096 x 4096, rank 16, fp32, forward and backward: 6.3 ms with all 805 MB of slices at once, 6.6 in bands
// of 256 MB, 6.8 of 128, 7.5 of 64; bf16 4095 x 4097 10.0, 10.7, 11.7, 13.4: a band ends with SMs that have nothing left to do.)
constexpr int64_t kSliceBytes = (int64_t)1 << 30, kSliceBytesBeside = (int64_t)64 << 20;
constexpr int64_t kLeastRows = 128;
// bytes of `rows` rows' slices: none where one slice by itself lies in an fp32 result
int64_t slice_bytes(int64_t N, int64_t rows, int P, int K, int dt) {
  const int s = base_slices(N, P, K);
  const int64_t row = (int64_t)s * P * (int64_t)sizeof(float), n = rows < N ? rows : N;
  return dt == AB_F32 && s == 1 ? 0 : n > INT64_MAX / row ? INT64_MAX : n * row;
}
int64_t band_rows(int64_t N, int P, int slices, int64_t room) {
  const int64_t most = room / ((int64_t)slices * P * (int64_t)sizeof(float));
  if (N <= most) return N;
  const int64_t whole = most / kLeastRows * kLeastRows, bands = (N + whole - 1) / whole;      // kLeastRows fit (general_ws)
  return ((N + bands - 1) / bands + kLeastRows - 1) / kLeastRows * kLeastRows;
}
// Small products stay on the fp32 pipes (128 x 512 x 256: 11.6 us against 12.0, and no slices)
bool base_small(const Call& c, int P, int K) { return c.dt == AB_F32 && gemm_small_pays(c.N, P, K); }

// Slices of the rows where the gradients' tiles are few (4006 rows of one adapter, rank 4, 208 x 656: 15 blocks took 250 us)
int grad_slices(int64_t N, int m, int n, int r, int L) {
  const int sms = sm_count() > 0 ? sm_count() : 148;
  const int64_t blocks = (int64_t)((m + kGF - 1) / kGF + (n + kGF - 1) / kGF) * ((r + kGK - 1) / kGK) * L;
  int64_t s = 2 * sms / blocks;
  if (s > N / (2 * kGR)) s = N / (2 * kGR);
  return (int)(s < 1 ? 1 : s > 32 ? 32 : s);
}

// Workspace of the general path: status word, T, U, the adapters' rows, the gradients' slices, and in what is left (room, bytes) a band of the
// shared product.  bytes: the least that it runs with.
struct GeneralWs { int* status; float *T, *U, *base; int* order; int64_t *start, *count; float *pA, *pB; int slices; int64_t room; size_t bytes; };
GeneralWs general_ws(void* ws, size_t ws_bytes, int64_t N, int m, int n, int r, int L, int dt) {
  Arena ar(ws, 0);
  GeneralWs w;
  w.status = ar.take_n<int>(64);
  w.T = ar.take_n<float>((size_t)N * r);
  w.U = ar.take_n<float>((size_t)N * r);
  w.order = ar.take_n<int>((size_t)N);
  w.start = ar.take_n<int64_t>((size_t)L);
  w.count = ar.take_n<int64_t>((size_t)L);
  w.slices = grad_slices(N, m, n, r, L);
  w.pA = w.slices > 1 ? ar.take_n<float>((size_t)w.slices * L * m * r) : nullptr;
  w.pB = w.slices > 1 ? ar.take_n<float>((size_t)w.slices * L * n * r) : nullptr;
  w.base = ar.take_n<float>(0);
  w.room = ws_bytes > ar.used ? (int64_t)(ws_bytes - ar.used) : 0;
  const int64_t y = slice_bytes(N, kLeastRows, m, n, dt), x = slice_bytes(N, kLeastRows, n, m, dt);
  w.bytes = align_up(ar.used + (size_t)(x > y ? x : y), 256);
  return w;
}
// What the query asks for: the slices of all rows, up to `most` bytes
size_t general_ws_bytes(int64_t N, int m, int n, int r, int L, int dt, int64_t most) {
  const size_t least = general_ws(nullptr, 0, N, m, n, r, L, dt).bytes;
  const int64_t y = slice_bytes(N, N, m, n, dt), x = slice_bytes(N, N, n, m, dt), all = x > y ? x : y;
  const int64_t y0 = slice_bytes(N, kLeastRows, m, n, dt), x0 = slice_bytes(N, kLeastRows, n, m, dt), some = x0 > y0 ? x0 : y0;
  const int64_t more = (all < most ? all : most) - some;
  return align_up(least + (size_t)(more > 0 ? more : 0), 256);
}

template <typename TI, int kRB>
int launch_project(const Call& c, const void* In, int K, const void* F, int64_t strideF, int64_t f_k, int64_t f_j, float* T, bool first, int* status) {
  return launch_after(project_kernel<TI, kRB>, (unsigned)((c.N + kRB - 1) / kRB), (unsigned)kProjThreads, 0, 1, c.st, static_cast<const TI*>(In),
                      static_cast<const TI*>(F), strideF, f_k, f_j, c.scale, c.ids, T, c.N, K, c.r, c.L, first ? 1 : 0, status);
}
int project(const Call& c, const void* In, int K, const void* F, int64_t strideF, int64_t f_k, int64_t f_j, float* T, bool first, int* status) {
  const bool four = c.N >= 1024;             // fewer rows: a block each fills the device better
  if (c.dt == AB_F32)
    return four ? launch_project<float, 4>(c, In, K, F, strideF, f_k, f_j, T, first, status)
                : launch_project<float, 1>(c, In, K, F, strideF, f_k, f_j, T, first, status);
  return four ? launch_project<bf16, 4>(c, In, K, F, strideF, f_k, f_j, T, first, status)
              : launch_project<bf16, 1>(c, In, K, F, strideF, f_k, f_j, T, first, status);
}

// rows [row0, row0 + rows) of the call; base: their slices
template <typename T16, int kRD>
int launch_delta(const Call& c, int64_t row0, int64_t rows, const float* base, int slices, const float* T, const void* G, int64_t strideG, int64_t g_c,
                 int64_t g_k, void* out, int P, int* status) {
  const dim3 grid((unsigned)((rows + kRD - 1) / kRD), (unsigned)((P + kDeltaCols - 1) / kDeltaCols));
  return launch_after(delta_kernel<T16, T16, kRD>, grid, (unsigned)kDeltaCols, 0, 1, c.st, base, slices, T + row0 * c.r, static_cast<const T16*>(G),
                      strideG, g_c, g_k, c.ids + row0, static_cast<T16*>(out) + row0 * P, rows, P, c.r, c.L, status);
}
template <typename T16>
int delta(const Call& c, int64_t row0, int64_t rows, const float* base, int slices, const float* T, const void* G, int64_t strideG, int64_t g_c,
          int64_t g_k, void* out, int P, int* status) {
  // sixteen rows a block where that still gives every SM two blocks
  const int sms = sm_count() > 0 ? sm_count() : 148;
  const int64_t blocks = (rows + 15) / 16 * ((P + kDeltaCols - 1) / kDeltaCols);
  return blocks >= 2 * sms ? launch_delta<T16, 16>(c, row0, rows, base, slices, T, G, strideG, g_c, g_k, out, P, status)
                           : launch_delta<T16, 2>(c, row0, rows, base, slices, T, G, strideG, g_c, g_k, out, P, status);
}

// out = In W^T (W: P x K, row-major) or In W (W: K x P), and T's part
int shared_and_delta(const Call& c, const void* In, int K, bool w_mn, const float* T, const void* G, int64_t strideG, int64_t g_c, int64_t g_k,
                     void* out, int P, const GeneralWs& w) {
  const bool simt = base_small(c, P, K) || !gemm_tc_available() || c.N > 0x3fffffff;
  const int want = base_slices(c.N, P, K);
  const bool in_place = c.dt == AB_F32 && (simt || want == 1);       // the product lies in the result
  const int64_t e = (int64_t)dtype_size(c.dt), band = in_place ? c.N : band_rows(c.N, P, want, w.room);
  for (int64_t row0 = 0; row0 < c.N; row0 += band) {
    const int64_t rows = c.N - row0 < band ? c.N - row0 : band;
    const char* X = static_cast<const char*>(In) + row0 * K * e;
    float* base = in_place ? static_cast<float*>(out) : w.base;
    int slices = 1;
    if (simt) {
      AB_TRY(gemm_simt(X, c.dt, K, 1, c.W, c.dt, w_mn ? P : 1, w_mn ? 1 : K, base, AB_F32, P, rows, P, K, c.st));
    } else {
      const int per = ((K + want - 1) / want + 63) / 64 * 64;
      SplitGemm p[kSplitFew];
      memset(p, 0, sizeof(p));
      int n = 0;
      for (int k0 = 0; k0 < K; k0 += per, ++n) {
        p[n].A = X + k0 * e; p[n].lda = K;
        p[n].B = static_cast<const char*>(c.W) + (w_mn ? (int64_t)k0 * P : (int64_t)k0) * e; p[n].ldb = w_mn ? P : K; p[n].b_mn = w_mn ? 1 : 0;
        p[n].C = base + (int64_t)n * rows * P; p[n].ldc = P;
        p[n].M = (int)rows; p[n].N = P; p[n].K = K - k0 < per ? K - k0 : per;
      }
      slices = n;
      AB_TRY(gemm_split_few(p, n, c.dt == AB_BF16, w.status, c.st));
    }
    AB_TRY(c.dt == AB_F32 ? delta<float>(c, row0, rows, base, slices, T, G, strideG, g_c, g_k, out, P, w.status)
                          : delta<bf16>(c, row0, rows, base, slices, T, G, strideG, g_c, g_k, out, P, w.status));
  }
  return AB_OK;
}

int grads(const Call& c, const GeneralWs& w, const void* dY, const float* T, float* dA, float* dB) {
  const int64_t ea = (int64_t)c.L * c.m * c.r, eb = (int64_t)c.L * c.n * c.r;
  GradSides s;
  memset(&s, 0, sizeof(s));
  int n = 0;
  if (dA) s.side[n++] = GradSide{dY, c.m, (c.m + kGF - 1) / kGF, T, w.slices > 1 ? w.pA : dA, (int64_t)c.m * c.r, c.r, 1, ea};
  if (dB) s.side[n++] = GradSide{c.x, c.n, (c.n + kGF - 1) / kGF, w.U, w.slices > 1 ? w.pB : dB, (int64_t)c.r * c.n, 1, c.n, eb};
  const unsigned tiles = (unsigned)(s.side[0].tiles + s.side[1].tiles);
  const int step = 65535 / w.slices;          // adapters of a launch
  for (int a0 = 0; a0 < c.L; a0 += step) {
    const dim3 grid(tiles, (unsigned)((c.r + kGK - 1) / kGK), (unsigned)((c.L - a0 < step ? c.L - a0 : step) * w.slices));
    const int* order = w.order;
    const int64_t *start = w.start + a0, *count = w.count + a0;
    if (c.dt == AB_F32) AB_TRY(launch_after(adapter_grad_kernel<float>, grid, 256u, 0, 1, c.st, s, c.r, order, start, count, w.slices));
    else AB_TRY(launch_after(adapter_grad_kernel<bf16>, grid, 256u, 0, 1, c.st, s, c.r, order, start, count, w.slices));
    for (int i = 0; i < n; ++i) s.side[i].D += step * s.side[i].strideD;
  }
  if (w.slices == 1) return AB_OK;
  return adapter_add_slices(w.pA, dA, ea, w.pB, dB, eb, w.slices, c.st);
}

int general_forward(const Call& c, void* y, float* T_save, const GeneralWs& w) {
  float* T = T_save ? T_save : w.T;
  AB_TRY(project(c, c.x, c.n, c.B, c.strideB, c.n, 1, T, true, w.status));
  return shared_and_delta(c, c.x, c.n, false, T, c.A, c.strideA, c.r, 1, y, c.m, w);
}

int general_backward(const Call& c, const void* dY, const float* T_saved, void* dX, float* dA, float* dB, const GeneralWs& w) {
  bool first = true;
  if (dX || dB) { AB_TRY(project(c, dY, c.m, c.A, c.strideA, 1, c.r, w.U, first, w.status)); first = false; }
  if (dA && !T_saved) { AB_TRY(project(c, c.x, c.n, c.B, c.strideB, c.n, 1, w.T, first, w.status)); first = false; }
  if (dX) AB_TRY(shared_and_delta(c, dY, c.m, true, w.U, c.B, c.strideB, 1, c.n, dX, c.n, w));
  if (!dA && !dB) return AB_OK;
  AB_TRY(launch_after(list_rows_kernel, (unsigned)c.L, (unsigned)kListThreads, 0, 1, c.st, c.ids, c.N, c.L, w.order, w.start, w.count, w.status,
                      first ? 1 : 0));
  return grads(c, w, dY, T_saved ? T_saved : w.T, dA, dB);
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

int adapter_add_slices(const float* pA, float* dA, int64_t ea, const float* pB, float* dB, int64_t eb, int slices, cudaStream_t st) {
  const SliceSide x{pA, dA, dA ? ea : 0}, y{pB, dB, dB ? eb : 0};
  return launch_after(add_slices_kernel, (unsigned)((x.count + y.count + 255) / 256), 256u, 0, 1, st, x, y, slices);
}

}  // namespace ab

using namespace ab;

extern "C" {

size_t ab_adapter_workspace_bytes(int64_t N, int m, int n, int r, int L, int dt) {
  if (N < 0 || N > 0x7fffffffll || m <= 0 || n <= 0 || r <= 0 || L <= 0 || !dtype_ok(dt)) return 0;
  const bool tc = adapter_tc_shape_ok(N, m, n, r, L, dt);
  const size_t g = general_ws_bytes(N, m, n, r, L, dt, tc ? kSliceBytesBeside : kSliceBytes), t = tc ? adapter_tc_ws(N, m, n, r, L) : 0;
  return (g > t ? g : t) + 256;
}

int ab_selftest_adapter_form(int64_t N, int P, int K) { return N < 1 || P < 1 || K < 1 ? -1 : adapter_tc_form(N, P, K); }

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
  const GeneralWs w = general_ws(ws, ws_bytes, N, m, n, r, L, dt);
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
  if (adapter_tc_supported(c, dY, dX, T_saved, dA, dB) && ((!dA && !dB) || adapter_tc_lists_ok(N, L))) {
    if (adapter_tc_ws(N, m, n, r, L) > ws_bytes) return AB_ERR_WORKSPACE;
    return adapter_tc_backward(c, dY, T_saved, dX, dA, dB, ws);
  }
  const GeneralWs w = general_ws(ws, ws_bytes, N, m, n, r, L, dt);
  if (w.bytes > ws_bytes) return AB_ERR_WORKSPACE;
  return general_backward(c, dY, T_saved, dX, dA, dB, w);
}

}  // extern "C"
