// Global norm of many gradients and their scaling, between a backward pass and the optimizer step:
//
//   norm = sqrt(sum of g^2 over all tensors),  out = g c,  c = max_norm / norm where that is below 1, else 1
//
// Two launches.  The first cuts the tensors into chunks, one CTA at a time each, and leaves one sum of squares a CTA; in the
// second every CTA adds those sums up in the same order (a few KB from L2: no counter, no atomics, the same bits in every
// run), and scales its chunks.  c depends on every value, so what does not stay in L2 (126 MB) between the launches has to be read
// twice: the second launch takes the chunks in the opposite order, so that it meets what the first read last.
//
// Bound by HBM: 1 GB of bf16 540 us, where two readings and a writing take 493 at the copy rate of 6.54 TB/s.
#include "ab_common.cuh"
#include "ab_tc_ptx.cuh"

namespace ab {
namespace {

constexpr int kClipThreads = 512;
// Tensors of one launch: their records are kernel arguments, so nothing is copied in front of the launch and a captured call is whole.  A
// short table where it is enough: arguments are copied at every launch.
constexpr int kClipShort = 160, kClipLong = 1000;
// Bytes of a chunk: the longest with which every CTA still gets three.  Long ones have fewer beginnings and ends (1 GB of bf16: 32 KB
// 597 us, 128 KB 540; the 144 factors of ViT-B/16, 127 MB: 16 KB 100 us, 32 KB 74, by this rule 67), short ones spread evenly over the CTAs
// (one layer of 1 MB: 9.1 us with 8, 16 or 32 KB).
constexpr int kChunkShort = 16384, kChunkLong = 131072;
constexpr int kClipMaxCtas = 148 * 4;

struct ClipRec { const void* g; void* out; int64_t count; };
template <int kCap>
struct ClipTable {
  ClipRec rec[kCap];
  int first[kCap + 1];                      // chunk index at which each tensor begins
  int tensors, chunk;                       // chunk: bytes
};

// The square of a value in fp32 overflows above 1.8e19 and vanishes below 1e-23: four squares are added in fp32 where their sum says that
// neither happened, else each in fp64.
__device__ __forceinline__ void add_squares(double& acc, float a, float b, float c, float d) {
  const float s = fmaf(a, a, b * b) + fmaf(c, c, d * d);
  if (s > 1e-30f && s < 1e37f) {
    acc += (double)s;
  } else if (((__float_as_uint(a) | __float_as_uint(b) | __float_as_uint(c) | __float_as_uint(d)) << 1) != 0u) {
    const double x = a, y = b, z = c, w = d;
    acc += (x * x + y * y) + (z * z + w * w);
  }
}

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void squares(const uint4& u, double& acc) {
    add_squares(acc, __uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
  }
  static __device__ __forceinline__ uint4 scaled(const uint4& u, float c) {
    return make_uint4(__float_as_uint(__uint_as_float(u.x) * c), __float_as_uint(__uint_as_float(u.y) * c),
                      __float_as_uint(__uint_as_float(u.z) * c), __float_as_uint(__uint_as_float(u.w) * c));
  }
};
__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf_scaled(uint32_t v, float c) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(bf_lo(v) * c, bf_hi(v) * c);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <> struct Vec<bf16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void squares(const uint4& u, double& acc) {
    add_squares(acc, bf_lo(u.x), bf_hi(u.x), bf_lo(u.y), bf_hi(u.y));
    add_squares(acc, bf_lo(u.z), bf_hi(u.z), bf_lo(u.w), bf_hi(u.w));
  }
  static __device__ __forceinline__ uint4 scaled(const uint4& u, float c) {
    return make_uint4(bf_scaled(u.x, c), bf_scaled(u.y, c), bf_scaled(u.z, c), bf_scaled(u.w, c));
  }
};

// The tensor that chunk q belongs to.
template <int kCap>
__device__ __forceinline__ int find_tensor(const ClipTable<kCap>& t, int q) {
  int lo = 0, hi = t.tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= q) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// What chunk q covers: elements [from, to) of tensor i.  A chunk's end lies on a 16-byte boundary of g, so that all but the first and the
// last few values of a tensor go by 16-byte loads wherever it starts.
template <typename T, int kCap>
__device__ __forceinline__ void chunk_range(const ClipTable<kCap>& t, int q, int i, int64_t& from, int64_t& to) {
  const int64_t per = t.chunk / (int64_t)sizeof(T), count = t.rec[i].count;
  const int64_t skew = (int64_t)((reinterpret_cast<uintptr_t>(t.rec[i].g) & 15) / sizeof(T));     // values past a 16-byte boundary
  const int64_t c = q - t.first[i];
  from = c == 0 ? 0 : c * per - skew;
  to = (c + 1) * per - skew;
  if (to > count) to = count;
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double part[kClipThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.0;
  for (int w = 0; w < (int)blockDim.x / 32; ++w) s += part[w];
  return s;
}

// Adds the squares of chunk q.
template <typename T, int kCap>
__device__ __forceinline__ void chunk_squares(const ClipTable<kCap>& t, int q, double& acc) {
  const int i = find_tensor(t, q);
  int64_t from, to;
  chunk_range<T>(t, q, i, from, to);
  const T* g = static_cast<const T*>(t.rec[i].g);
  // up to the first 16-byte boundary, whole 16-byte groups, the rest
  int64_t head = ((16 - (reinterpret_cast<uintptr_t>(g + from) & 15)) & 15) / sizeof(T);
  if (head > to - from) head = to - from;
  const int groups = (int)((to - from - head) / Vec<T>::n);
  const int64_t tail = from + head + (int64_t)groups * Vec<T>::n;
  const uint4* v = reinterpret_cast<const uint4*>(g + from + head);
  if (threadIdx.x < head) { const double x = to_f32(g[from + threadIdx.x]); acc += x * x; }
  if (tail + threadIdx.x < to) { const double x = to_f32(g[tail + threadIdx.x]); acc += x * x; }
  for (int k = threadIdx.x; k < groups; k += 8 * kClipThreads) {
    uint4 u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + e * kClipThreads < groups) u[e] = v[k + e * kClipThreads];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + e * kClipThreads < groups) Vec<T>::squares(u[e], acc);
  }
}

// out = g c over chunk q, c = (float)factor.  A factor below what fp32 holds in full (2^-126; gradients near the type's largest value or a tiny
// limit) is applied in 64 bits, by one value a thread: rounded to fp32 it would have few bits left, or none.
template <typename T, int kCap>
__device__ __forceinline__ void chunk_scaled(const ClipTable<kCap>& t, int q, double factor) {
  const int i = find_tensor(t, q);
  int64_t from, to;
  chunk_range<T>(t, q, i, from, to);
  const T* g = static_cast<const T*>(t.rec[i].g);
  T* out = static_cast<T*>(t.rec[i].out);
  const float c = (float)factor;
  if (c == 1.f && g == out) return;                       // nothing to do where it lies
  if (factor > 0.0 && factor < 1.1754943508222875e-38) {
    for (int64_t k = from + threadIdx.x; k < to; k += kClipThreads) from_f32(out[k], (float)((double)to_f32(g[k]) * factor));
    return;
  }
  if (((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(out)) & 15) != 0) {
    for (int64_t k = from + threadIdx.x; k < to; k += kClipThreads) from_f32(out[k], c == 1.f ? to_f32(g[k]) : to_f32(g[k]) * c);
    return;
  }
  int64_t head = ((16 - (reinterpret_cast<uintptr_t>(g + from) & 15)) & 15) / sizeof(T);
  if (head > to - from) head = to - from;
  const int groups = (int)((to - from - head) / Vec<T>::n);
  const int64_t tail = from + head + (int64_t)groups * Vec<T>::n;
  const uint4* v = reinterpret_cast<const uint4*>(g + from + head);
  uint4* w = reinterpret_cast<uint4*>(out + from + head);
  if (threadIdx.x < head) from_f32(out[from + threadIdx.x], to_f32(g[from + threadIdx.x]) * c);
  if (tail + threadIdx.x < to) from_f32(out[tail + threadIdx.x], to_f32(g[tail + threadIdx.x]) * c);
  for (int k = threadIdx.x; k < groups; k += 8 * kClipThreads) {
    uint4 u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + e * kClipThreads < groups) u[e] = v[k + e * kClipThreads];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + e * kClipThreads < groups) __stcs(w + k + e * kClipThreads, Vec<T>::scaled(u[e], c));
  }
}

// The factor; a norm that is infinite or NaN scales nothing: the caller sees it and can drop the step.
__device__ __forceinline__ double clip_factor(double norm, float max_norm) {
  const double big = max_norm;
  return norm > big && norm <= 1.7976931348623157e308 ? big / norm : 1.0;
}

// part[blockIdx.x]: the sum of the squares of this CTA's chunks (q = blockIdx.x, + grid, ...), on top of what an earlier launch left there
template <typename T, int kCap>
__global__ void __launch_bounds__(kClipThreads)
clip_norm_kernel(const __grid_constant__ ClipTable<kCap> t, int chunks, double* __restrict__ part, int add) {
  tc::dep_wait();
  tc::dep_launch();
  double acc = 0.0;
  for (int q = blockIdx.x; q < chunks; q += gridDim.x) chunk_squares<T>(t, q, acc);
  const double s = block_sum(acc);
  if (threadIdx.x == 0) part[blockIdx.x] = add ? part[blockIdx.x] + s : s;
}

template <typename T, int kCap>
__global__ void __launch_bounds__(kClipThreads)
clip_scale_kernel(const __grid_constant__ ClipTable<kCap> t, int chunks, const double* __restrict__ part, int parts, float max_norm,
                  float* __restrict__ norm_out, int write) {
  tc::dep_wait();
  tc::dep_launch();
  double acc = 0.0;
  for (int p = threadIdx.x; p < parts; p += kClipThreads) acc += __ldcg(part + p);
  const double norm = sqrt(block_sum(acc));
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  if (!write) return;
  const double c = clip_factor(norm, max_norm);
  for (int b = blockIdx.x; b < chunks; b += gridDim.x) chunk_scaled<T>(t, chunks - 1 - b, c);
}

// A table from tensor i on; returns the first tensor that is not in it.
template <int kCap>
int fill_table(ClipTable<kCap>& t, const ab_clip_desc* d, int L, int i, int dt, int* chunks) {
  const int64_t esz = (int64_t)dtype_size(dt);
  t.tensors = 0;
  int64_t q = 0;
  for (; i < L && t.tensors < kCap; ++i) {
    if (d[i].count == 0) continue;
    const int64_t skew = (int64_t)(reinterpret_cast<uintptr_t>(d[i].grad) & 15);
    const int64_t n = (d[i].count * esz + skew + t.chunk - 1) / t.chunk;
    if (t.tensors > 0 && q + n > 0x7fffffffll) break;
    t.rec[t.tensors] = ClipRec{d[i].grad, d[i].out, d[i].count};
    t.first[t.tensors++] = (int)q;
    q += n;
  }
  t.first[t.tensors] = (int)q;
  *chunks = (int)q;
  return i;
}

int clip_grid(int chunks) {
  const int sms = sm_count() > 0 ? sm_count() : 148, most = sms * 4 < kClipMaxCtas ? sms * 4 : kClipMaxCtas;
  return chunks < 1 ? 1 : chunks < most ? chunks : most;
}

template <typename T, int kCap>
int clip_run(const ab_clip_desc* d, int L, float max_norm, float* norm_out, double* part, int dt, bool write, cudaStream_t st) {
  ClipTable<kCap> t;
  int chunks, parts = 0, next;
  int64_t bytes = 0;
  for (int i = 0; i < L; ++i) bytes += d[i].count * (int64_t)dtype_size(dt);
  t.chunk = kChunkShort;
  while (t.chunk < kChunkLong && bytes / (2 * t.chunk) >= 3 * clip_grid(kClipMaxCtas)) t.chunk *= 2;
  for (int i = 0; i < L || i == 0; i = next) {
    next = fill_table(t, d, L, i, dt, &chunks);
    // the first launch sets the sums that later ones add to: where there are later ones it has all the CTAs that there can be
    const int grid = clip_grid(i == 0 && next < L ? kClipMaxCtas : chunks);
    if (i == 0) parts = grid;
    AB_TRY(launch_after(clip_norm_kernel<T, kCap>, (unsigned)grid, (unsigned)kClipThreads, 0, 1, st, t, chunks, part, i == 0 ? 0 : 1));
  }
  const double* sums = part;
  for (int i = 0; i < L || i == 0; i = next) {
    next = write ? fill_table(t, d, L, i, dt, &chunks) : L;
    AB_TRY(launch_after(clip_scale_kernel<T, kCap>, (unsigned)(write ? clip_grid(chunks) : 1), (unsigned)kClipThreads, 0, 1, st, t, chunks, sums, parts,
                        max_norm, norm_out, write ? 1 : 0));
  }
  return AB_OK;
}

template <typename T>
int clip_any(const ab_clip_desc* d, int L, float max_norm, float* norm_out, double* part, int dt, bool write, cudaStream_t st) {
  if (L <= kClipShort) return clip_run<T, kClipShort>(d, L, max_norm, norm_out, part, dt, write, st);
  return clip_run<T, kClipLong>(d, L, max_norm, norm_out, part, dt, write, st);
}

}  // namespace
}  // namespace ab

using namespace ab;

extern "C" {

size_t ab_grad_clip_workspace_bytes(int L) { return L <= 0 ? 0 : align_up(kClipMaxCtas * sizeof(double), 256); }

int ab_grad_clip(const ab_clip_desc* descs, int L, float max_norm, float* norm_out, int dt, void* ws, size_t ws_bytes, void* cuda_stream) {
  if (!descs || L <= 0 || !dtype_ok(dt) || !(max_norm >= 0.f) || !norm_out || !aligned(norm_out, 4)) return AB_ERR_INVALID_ARG;
  bool out = false, none = false;
  for (int i = 0; i < L; ++i) {
    if (descs[i].count < 0 || (descs[i].count > 0 && !descs[i].grad)) return AB_ERR_INVALID_ARG;
    if (!aligned(descs[i].grad, dtype_size(dt)) || !aligned(descs[i].out, dtype_size(dt))) return AB_ERR_INVALID_ARG;
    if (descs[i].count > ((int64_t)1 << 40)) return AB_ERR_UNSUPPORTED;
    if (descs[i].count > 0) (descs[i].out ? out : none) = true;
  }
  if (out && none) return AB_ERR_INVALID_ARG;               // all are scaled or none is
  int dev = 0;
  if (cudaGetDeviceCount(&dev) != cudaSuccess || dev <= 0) return AB_ERR_CUDA;
  if (!ws || !aligned(ws, 256) || ws_bytes < ab_grad_clip_workspace_bytes(L)) return AB_ERR_WORKSPACE;
  double* part = static_cast<double*>(ws);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return dt == AB_F32 ? clip_any<float>(descs, L, max_norm, norm_out, part, dt, out, st)
                      : clip_any<bf16>(descs, L, max_norm, norm_out, part, dt, out, st);
}

}  // extern "C"
