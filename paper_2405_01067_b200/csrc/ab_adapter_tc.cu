// Adapters beside a shared projection on the tensor cores (bf16 storage, fp32 accumulation): see ab_adapter.cu for the operator.
//
// Rows are looked at in groups of 16.  A group is uniform when all of its rows have the same adapter (or none): its products with that
// adapter's factors go to the tensor cores, columns of an accumulator of their own.  A mixed group's rows get their adapters' part one by one:
// a product is formed for several rows at a time, and each row takes its own adapter's.  So runs of rows (prompts, training groups)
// cost their products, single tokens of many adapters cost the reading of each adapter's factors, any order works, and no row's result
// ever holds a product with another adapter's factors, not even one with zero.
//
//   rows_kernel     T_i = s_a F_a In_i of rows in mixed groups, or of all rows where they are few, one row a CTA at a time (fp32 pipes)
//   project_kernel  T by tiles: In tile (rows) x factors of the tile's adapters, up to eight; with it what a backward call prepares
//   wide_kernel     Out^T = W In^T + G_a T^T: 128 or 256 output features x up to 256 rows a tile.  Rows are the N side of the MMA, so a
//                   run of groups is a range of accumulator columns: the adapter's product is a few more slabs of the reduction with
//                   fewer columns.  Mixed groups are added in the epilogue, by mma.sync fragments laid out as TMEM hands them over
//   few_kernel      the same for few rows (generation): bound by the reading of W, whose reduction is cut over a cluster
//   adapter_grad    D_a = In^T T over the 64-row slabs that have rows of a; rows of others in such a slab are cleared in shared memory
//
// Measured, us (floor: the bytes or operations a call cannot do without, at 6538 GB/s and 1679 TFLOP/s): one token, 4096 x 4096, rank 16 15, of
// which 10 are the kernels' (5.2); 64 tokens of 64 adapters 17 (7.9); 6173 rows of 16 adapters, 2048 -> 8192, rank 64 214 (128); training, 50,432
// rows of 4 groups, 768 x 768, rank 64 240 (89); 8191 rows of 8, 4096 x 4096, rank 16 515 (331).
//
// T travels as three bf16 pieces (hi = bf16(T), mid = bf16(T - hi), lo the rest: 24 bits): the second product takes two of them (its result
// is rounded to bf16, of whose half step, 2^-8, the 2^-16 of T that is lost at most is nothing), the gradients take all three.
#include <cstring>

#include "ab_adapter.cuh"
#include "ab_tc_ptx.cuh"

namespace ab {
namespace {

using namespace tc;

constexpr int kG = 16;                    // rows of a group

// ------------------------------------------------------------------------------------------------ rows and groups
__device__ __forceinline__ int clean_id(int a, int L) { return a >= 0 && a < L ? a : -1; }

// What lane l < 16 returns for group l of the 256 rows from row0: its adapter, -1 (no adapter, or no rows), -2 (mixed).  Whole warp; lanes
// 2 l and 2 l + 1 read the group's ids (id: of rows 8 lane ..).  bad: an entry that is neither an adapter nor -1.
__device__ __forceinline__ int group_ids(const int* __restrict__ ids, int64_t N, int L, int64_t row0, int lane, bool& bad, int (&id)[8]) {
  int first = -3, same = 1;
  bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int64_t row = row0 + 8 * lane + e;
    id[e] = -1;
    if (row < N) {
      const int raw = ids[row], v = clean_id(raw, L);
      bad |= raw < -1 || raw >= L;
      id[e] = v;
      if (first == -3) first = v;
      same &= v == first;
    }
  }
  const int of = __shfl_xor_sync(0xffffffffu, first, 1), os = __shfl_xor_sync(0xffffffffu, same, 1);
  const int one = first == -3 ? of : first;
  int g = one == -3 ? -1 : one;
  if (!same || !os || (first != -3 && of != -3 && first != of)) g = -2;
  return __shfl_sync(0xffffffffu, g, (2 * lane) & 31);
}

// The three pieces of a value; what is not finite is in the first alone.
__device__ __forceinline__ void cut(float v, bf16& hi, bf16& mid, bf16& lo) {
  hi = __float2bfloat16_rn(v);
  const float h = __bfloat162float(hi);
  const float r1 = isfinite(h) ? v - h : 0.f;
  mid = __float2bfloat16_rn(r1);
  lo = __float2bfloat16_rn(r1 - __bfloat162float(mid));
}

// eight neighbouring values as pieces at P, P + rp, P + 2 rp
__device__ __forceinline__ void put_pieces(bf16* P, int rp, const float* v) {
  uint32_t h[4], m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bf16 hh[2], mm[2], ll[2];
    cut(v[2 * i], hh[0], mm[0], ll[0]);
    cut(v[2 * i + 1], hh[1], mm[1], ll[1]);
    h[i] = (uint32_t)__bfloat16_as_ushort(hh[0]) | ((uint32_t)__bfloat16_as_ushort(hh[1]) << 16);
    m[i] = (uint32_t)__bfloat16_as_ushort(mm[0]) | ((uint32_t)__bfloat16_as_ushort(mm[1]) << 16);
    l[i] = (uint32_t)__bfloat16_as_ushort(ll[0]) | ((uint32_t)__bfloat16_as_ushort(ll[1]) << 16);
  }
  *reinterpret_cast<uint4*>(P) = make_uint4(h[0], h[1], h[2], h[3]);
  *reinterpret_cast<uint4*>(P + rp) = make_uint4(m[0], m[1], m[2], m[3]);
  *reinterpret_cast<uint4*>(P + 2 * rp) = make_uint4(l[0], l[1], l[2], l[3]);
}

__device__ __forceinline__ void dot8(const uint4& u, const float* t, float& acc) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    acc = fmaf(__uint_as_float(w[e] << 16), t[2 * e], acc);
    acc = fmaf(__uint_as_float(w[e] & 0xffff0000u), t[2 * e + 1], acc);
  }
}

__device__ __forceinline__ void raise(int* abort_any, int* status) {
  *reinterpret_cast<volatile int*>(abort_any) = 1;
  atomicExch(status, (int)AB_ERR_TIMEOUT);
}

// ------------------------------------------------------------------------------------------------ what a backward call prepares
// CTAs 0 .. L-1: the 64-row slabs that have rows of adapter `cta`, ascending: (slab, which of its rows are the adapter's: 32 bits and 32 bits,
// 0).  CTAs behind: T (fp32) cut into pieces, eight values a thread.  Reads the call's inputs alone: the lists are made beside the
// projection, in one launch with it, and its tiles' CTAs cut T (a launch of its own found no room before the kernel in front of it had
// ended: 20 us for the ViT groups).
struct PrepParams {
  uint4* list; int* count; int nslab;
  const float* T; bf16* P;
  int ctas;                                 // all of them; 0: nothing to prepare
};
template <int kWarps>
__device__ __forceinline__ void prep_body(const PrepParams& q, const int* __restrict__ ids, int64_t N, int L, int r, int rp, int cta, int tid,
                                          int* warp_cnt) {
  if (cta >= L) {
    const int64_t step = (int64_t)(q.ctas - L) * 32 * kWarps;
    const int oct = rp / 8;
    for (int64_t i = (int64_t)(cta - L) * 32 * kWarps + tid; i < N * oct; i += step) {
      const int64_t row = i / oct;
      const int k = (int)(i - row * oct) * 8;
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (k < r) {
        const float4 t0 = *reinterpret_cast<const float4*>(q.T + row * r + k), t1 = *reinterpret_cast<const float4*>(q.T + row * r + k + 4);
        v[0] = t0.x; v[1] = t0.y; v[2] = t0.z; v[3] = t0.w; v[4] = t1.x; v[5] = t1.y; v[6] = t1.z; v[7] = t1.w;
      }
      put_pieces(q.P + row * 3 * rp + k, rp, v);
    }
    fence_proxy_async_all();
    return;
  }
  const int lane = tid & 31, warp = tid >> 5;
  uint4* mine = q.list + (int64_t)cta * q.nslab;
  int at = 0;
  for (int s0 = 0; s0 < q.nslab; s0 += 32 * kWarps) {
    // a warp looks at 32 slabs, lane e keeps what slab e is
    unsigned lo = 0u, hi = 0u;
    const int w0 = s0 + warp * 32;
#pragma unroll 16
    for (int e = 0; e < 32; ++e) {
      const int64_t row = (int64_t)(w0 + e) * 64 + lane;
      const bool x = row < N && ids[row] == cta, y = row + 32 < N && ids[row + 32] == cta;
      const unsigned vx = __ballot_sync(0xffffffffu, x), vy = __ballot_sync(0xffffffffu, y);
      if (lane == e) { lo = vx; hi = vy; }
    }
    const bool any = (lo | hi) != 0u;
    const unsigned vote = __ballot_sync(0xffffffffu, any);
    if (lane == 0) warp_cnt[warp] = __popc(vote);
    __syncthreads();
    int ahead = 0, sum = 0;
    for (int w = 0; w < kWarps; ++w) {
      const int c = warp_cnt[w];
      ahead += w < warp ? c : 0;
      sum += c;
    }
    if (any) mine[at + ahead + __popc(vote & ((1u << lane) - 1u))] = make_uint4((uint32_t)(w0 + lane), lo, hi, 0u);
    at += sum;
    __syncthreads();
  }
  if (tid == 0) q.count[cta] = at;
}

// By itself where no projection is launched by tiles.
constexpr int kPrepThreads = 512;
__global__ void __launch_bounds__(kPrepThreads)
prep_kernel(const __grid_constant__ PrepParams q, const int* __restrict__ ids, int64_t N, int L, int r, int rp, int first, int* status) {
  __shared__ int warp_cnt[kPrepThreads / 32];
  dep_wait();
  dep_launch();
  if (first && blockIdx.x == 0 && threadIdx.x == 0) *status = AB_OK;
  prep_body<kPrepThreads / 32>(q, ids, N, L, r, rp, blockIdx.x, threadIdx.x, warp_cnt);
}

// ------------------------------------------------------------------------------------------------ T of rows in mixed groups
// The distinct adapters of the rows [row0, row0 + rows), rows 64 or 128, ascending, into ad (by lane 0); returns how many, kMaxAd + 1 if more than
// kMaxAd.  Whole warp.
constexpr int kMaxAd = 8;
__device__ __forceinline__ int tile_adapters(const int* __restrict__ ids, int64_t N, int L, int64_t row0, int rows, int lane, int* ad) {
  unsigned v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t row = row0 + lane + 32 * e;
    v[e] = lane + 32 * e < rows && row < N ? (unsigned)clean_id(ids[row], L) : 0xffffffffu;       // -1 is 0xffffffff: none
  }
  int n = 0;
  unsigned last = 0;
  while (true) {
    unsigned low = 0xffffffffu;
#pragma unroll
    for (int e = 0; e < 4; ++e) if ((n == 0 || v[e] > last) && v[e] < low) low = v[e];
    low = __reduce_min_sync(0xffffffffu, low);
    if (low == 0xffffffffu) return n;
    if (n == kMaxAd) return kMaxAd + 1;
    if (ad && lane == 0) ad[n] = (int)low;
    last = low;
    ++n;
  }
}

struct ProjParams {
  const bf16* In; int64_t N; int K;
  const bf16* F; int64_t strideF;           // f_mn 0: F_a is r x K, row-major; 1: K x r
  int f_mn;
  const float* scale; const int* ids;
  float* T; bf16* P;                        // T: N x r; P: N x 3 rp
  int r, rp, L;
  int want_T;                               // T is wanted in fp32 too
  int all_rows;                             // every row goes by rows_kernel
  int tile_rows;
  int unit;                                 // rows of a CTA of rows_kernel, a divisor of tile_rows
  int first;                                // the call's first kernel
  int* status;
  // project_tc_kernel
  int prep_ctas, tile_ctas;                 // CTAs that prepare, whole clusters (they come first: lists are chains), and that have tiles
  PrepParams prep;                          // ctas: lists alone; T is cut by the CTAs that have the tiles (cut)
  int cut;
  int nk, csize, ns, slot_bytes, in_bytes, f_bytes, q_max, tmem_cols;
};

constexpr int kRowsThreads = 256;

__device__ __forceinline__ void put_T(const ProjParams& p, int64_t row, int k, float v) {
  bf16 h, m, l;
  cut(v, h, m, l);
  bf16* q = p.P + row * 3 * p.rp + k;
  q[0] = h; q[p.rp] = m; q[2 * p.rp] = l;
  if (k < p.r) p.T[row * p.r + k] = v;
}

// Rows that go one by one: `unit` rows from unit * p.unit, of tiles with more adapters than project_tc_kernel takes (the rows of their mixed
// groups), or all rows where they are few.  f_mn 0: a warp a value, lanes along K, every `parts`th round of warps; f_mn 1: a thread has
// eight neighbouring values and every so manieth row of F_a (parts 1).  red: kWarps x 32 x 8 floats.
template <int kWarps>
__device__ __forceinline__ void rows_body(const ProjParams& p, int64_t unit, int part, int parts, int tid, float (*red)[32][8]) {
  const int lane = tid & 31, warp = tid >> 5;
  const int64_t row0 = (int64_t)unit * p.unit;
  const bool work = p.all_rows || tile_adapters(p.ids, p.N, p.L, row0 / p.tile_rows * p.tile_rows, p.tile_rows, lane, nullptr) > kMaxAd;
  if (work) {
    for (int64_t row = row0; row < row0 + p.unit && row < p.N; ++row) {
      if (!p.all_rows) {                       // a uniform group: not here
        const int64_t other = (row & ~(int64_t)(kG - 1)) + (lane & (kG - 1));
        const int v = other < p.N ? clean_id(p.ids[other], p.L) : -3, v0 = __shfl_sync(0xffffffffu, v, 0);
        if (!__any_sync(0xffffffffu, v != -3 && v != v0)) continue;
      }
      const int a = clean_id(p.ids[row], p.L);
      const float s = a < 0 ? 0.f : p.scale ? p.scale[a] : 1.f;
      const uint4* x = reinterpret_cast<const uint4*>(p.In + row * (int64_t)p.K);
      if (a < 0) {
        if (part == 0) for (int k = tid; k < p.rp; k += 32 * kWarps) put_T(p, row, k, 0.f);
      } else if (!p.f_mn) {
        // short rows leave little to load for a value: four values at a time where every warp has eight or more (rank 128, rows of 160: 22
        // rounds of a trip to L2 each; rank 24, rows of 776: 24.7 us one at a time, 25.9 in fours)
        if (p.K <= 1024 && p.r >= 8 * kWarps) {
          for (int k = (part * kWarps + warp) * 4; k < p.rp; k += parts * kWarps * 4) {
            const uint4* f[4];
            float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = reinterpret_cast<const uint4*>(p.F + a * p.strideF + (int64_t)(k + e < p.r ? k + e : p.r - 1) * p.K);
#pragma unroll 2
            for (int j = lane; j < p.K / 8; j += 32) {
              const uint4 w = x[j];
              const uint32_t xs[4] = {w.x, w.y, w.z, w.w};
              float t[8];
#pragma unroll
              for (int i = 0; i < 4; ++i) { t[2 * i] = __uint_as_float(xs[i] << 16); t[2 * i + 1] = __uint_as_float(xs[i] & 0xffff0000u); }
#pragma unroll
              for (int e = 0; e < 4; ++e) dot8(f[e][j], t, v[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
              for (int o = 16; o > 0; o >>= 1) v[e] += __shfl_xor_sync(0xffffffffu, v[e], o);
              if (lane == 0) put_T(p, row, k + e, k + e < p.r ? s * v[e] : 0.f);
            }
          }
        } else
        for (int k = part * kWarps + warp; k < p.rp; k += parts * kWarps) {
          float v = 0.f;
          if (k < p.r) {
            const uint4* f = reinterpret_cast<const uint4*>(p.F + a * p.strideF + (int64_t)k * p.K);
            for (int j = lane; j < p.K / 8; j += 256) {
              uint4 u[8], w[8];
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (j + 32 * e < p.K / 8) { u[e] = f[j + 32 * e]; w[e] = x[j + 32 * e]; }
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (j + 32 * e < p.K / 8) {
                  const uint32_t xs[4] = {w[e].x, w[e].y, w[e].z, w[e].w};
                  float t[8];
#pragma unroll
                  for (int i = 0; i < 4; ++i) { t[2 * i] = __uint_as_float(xs[i] << 16); t[2 * i + 1] = __uint_as_float(xs[i] & 0xffff0000u); }
                  dot8(u[e], t, v);
                }
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
          }
          if (lane == 0) put_T(p, row, k, s * v);
        }
      } else {
        const int oct = p.r / 8;
        int op = 1;
        while (op < oct) op <<= 1;                           // at most 32
        const int o = tid % op, f0 = tid / op, step = 32 * kWarps / op;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (o < oct) {
          const bf16* F = p.F + a * p.strideF + 8 * o;
          const bf16* xr = p.In + row * (int64_t)p.K;
#pragma unroll 4
          for (int f = f0; f < p.K; f += step) {
            const uint4 u = *reinterpret_cast<const uint4*>(F + (int64_t)f * p.r);
            const float xv = __bfloat162float(xr[f]);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[2 * e] = fmaf(__uint_as_float(w[e] << 16), xv, v[2 * e]);
              v[2 * e + 1] = fmaf(__uint_as_float(w[e] & 0xffff0000u), xv, v[2 * e + 1]);
            }
          }
        }
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1)
          if (d >= op) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += __shfl_xor_sync(0xffffffffu, v[e], d);
          }
        if (lane < op) {
#pragma unroll
          for (int e = 0; e < 8; ++e) red[warp][lane][e] = v[e];
        }
        __syncthreads();
        for (int k = tid; k < p.rp; k += 32 * kWarps) {
          float t = 0.f;
          if (k < p.r)
            for (int w = 0; w < kWarps; ++w) t += red[w][k / 8][k % 8];
          put_T(p, row, k, s * t);
        }
        __syncthreads();
      }
    }
  }
}

__global__ void __launch_bounds__(kRowsThreads)
rows_kernel(const __grid_constant__ ProjParams p) {
  __shared__ float red[kRowsThreads / 32][32][8];
  dep_wait();
  dep_launch();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0 && p.first) *p.status = AB_OK;
  rows_body<kRowsThreads / 32>(p, blockIdx.x, blockIdx.y, gridDim.y, threadIdx.x, red);
  fence_proxy_async_all();
}

// ------------------------------------------------------------------------------------------------ clusters
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// ------------------------------------------------------------------------------------------------ T by tiles
// A cluster has a tile of rows and up to 128 of the r values (blockIdx.y), each of its CTAs a part of the reduction.  Every adapter that the
// tile's rows have gets columns of its own in the accumulator, for all rows of the tile; a row takes its own adapter's.  Four slabs
// (16 MMA steps) are summed in TMEM, the rest in registers: the tensor cores cut a sum off at every step (measured: 2e-8 of T a step),
// registers round.  The parts meet in the shared memory of the CTA that finishes a share of the rows, in rank order.
//
// A slab costs a CTA about 500 cycles of issuing whatever its size, so several CTAs share an SM and long reductions are cut.
constexpr int kProjTcThreads = 192;       // 0 = TMA producer, 1 = MMA issuer and TMEM owner, 2..5 = epilogue
constexpr int kMaxStages = 8;
constexpr int kFlush = 4;                 // slabs
struct ProjBars {
  uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int abort_any;
  int nad, whole, ad[kMaxAd];             // adapters of the tile; all of its rows are handled here
  int row_ad[128];                        // a row's adapter, -1 none, -2: not handled here; + 0x40000000: T is wanted in fp32
};

template <int kChunks>                    // up to 16 kChunks values of r a CTA
__global__ void __launch_bounds__(kProjTcThreads, kChunks <= 4 ? 3 : 1)
project_tc_kernel(const __grid_constant__ CUtensorMap tmIn, const __grid_constant__ CUtensorMap tmF, const __grid_constant__ ProjParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  ProjBars* b = reinterpret_cast<ProjBars*>(ring + (size_t)p.ns * p.slot_bytes);
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (p.first) dep_wait();
  dep_launch();
  if (p.first && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.status = AB_OK;
  const int cta = (int)blockIdx.x - p.prep_ctas;
  if (cta < 0 || cta >= p.tile_ctas) {
    if (blockIdx.y == 0) {
      if (cta < 0) {
        if ((int)blockIdx.x < p.prep.ctas)
          prep_body<kProjTcThreads / 32>(p.prep, p.ids, p.N, p.L, p.r, p.rp, blockIdx.x, threadIdx.x, reinterpret_cast<int*>(ring));
      } else if ((int64_t)(cta - p.tile_ctas) * p.unit < p.N) {      // behind the tiles: rows that go one by one
        rows_body<kProjTcThreads / 32>(p, cta - p.tile_ctas, 0, 1, threadIdx.x, reinterpret_cast<float(*)[32][8]>(ring));
      }
    }
    fence_proxy_async_all();
    if (!p.first) dep_wait();
    return;
  }
  const int tile = cta / p.csize, rank = cta - tile * p.csize;
  const int64_t row0 = (int64_t)tile * p.tile_rows;
  const int kc0 = (int)blockIdx.y * 128, cols = p.rp - kc0 < 128 ? p.rp - kc0 : 128;
  const int per = (p.nk + p.csize - 1) / p.csize, i0 = rank * per, i1 = i0 + per < p.nk ? i0 + per : p.nk;
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.ns; ++i) { mbar_init(&b->full[i], 1); mbar_init(&b->empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&b->acc_full[i], 1); mbar_init(&b->acc_empty[i], 4); }
    b->abort_any = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tmIn); tma_prefetch_desc(&tmF);
  }
  if (warp == 0) {
    int n = tile_adapters(p.ids, p.N, p.L, row0, p.tile_rows, lane, b->ad);
    const int whole = n <= kMaxAd;
    if (!whole) {                          // the uniform groups alone
      bool bad;
      int id[8];
      const int g = group_ids(p.ids, p.N, p.L, row0, lane, bad, id);
      n = 0;
      const int ng = p.tile_rows / kG;
      for (int i = 0; i < ng; ++i) {
        const int v = __shfl_sync(0xffffffffu, g, i);
        if (v >= 0 && !__any_sync(0xffffffffu, lane < i && g == v)) { if (lane == 0) b->ad[n] = v; ++n; }
      }
    }
    if (lane == 0) { b->nad = n; b->whole = whole; }
  }
  if (warp == 1) tmem_alloc(&b->tmem_base, p.tmem_cols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(*reinterpret_cast<volatile uint32_t*>(&b->tmem_base));
  const int nad = (int)uniform(*reinterpret_cast<volatile int*>(&b->nad));
  const int qw = warp & 3;                 // quarter of the TMEM lanes this warp may read = its 32 rows of the tile
  float R[kChunks][16];

  if (warp == 0) {
    int slot = 0, ph = 1;
    bool ok = true;
    for (int q0 = 0; q0 < nad && ok; q0 += p.q_max) {
      const int q = nad - q0 < p.q_max ? nad - q0 : p.q_max;
      for (int i = i0; i < i1; ++i) {
        if (!mbar_wait_warp(&b->empty[slot], ph)) { raise(&b->abort_any, p.status); ok = false; break; }
        if (elect_one()) {
          uint8_t* dst = ring + (size_t)slot * p.slot_bytes;
          uint64_t* bar = &b->full[slot];
          mbar_arrive_expect_tx(bar, p.in_bytes + q * p.f_bytes);
          tma_load_2d(dst, &tmIn, bar, i * 64, (int)row0);
          for (int e = 0; e < q; ++e) {
            uint8_t* df = dst + p.in_bytes + e * p.f_bytes;
            const int a = b->ad[q0 + e];
            if (p.f_mn) for (int h = 0; h * 8192 < p.f_bytes; ++h) tma_load_3d(df + h * 8192, &tmF, bar, kc0 + 64 * h, i * 64, a);
            else tma_load_3d(df, &tmF, bar, i * 64, kc0, a);
          }
        }
        __syncwarp();
        if (++slot == p.ns) { slot = 0; ph ^= 1; }
      }
    }
  } else if (warp == 1) {
    const uint32_t idesc = instr_desc_bf16(128, cols, 0, p.f_mn), base = uniform(smem_u32(ring));
    const uint64_t dI = smem_desc_sw128(base, 16), dF = smem_desc_sw128(base + p.in_bytes, p.f_mn ? 8192 : 16);
    const uint64_t f_step = p.f_mn ? 128u : 2u, slot_step = (uint64_t)(p.slot_bytes >> 4), q_step = (uint64_t)(p.f_bytes >> 4);
    int slot = 0, ph = 0, flush = 0;
    bool ok = true;
    for (int q0 = 0; q0 < nad && ok; q0 += p.q_max) {
      const int q = nad - q0 < p.q_max ? nad - q0 : p.q_max;
      for (int i = i0; i < i1; ++i) {
        const int in = (i - i0) % kFlush, buf = flush & 1;
        if (in == 0) {
          if (!mbar_wait_warp(&b->acc_empty[buf], ((flush >> 1) & 1) ^ 1)) { raise(&b->abort_any, p.status); ok = false; break; }
          tc_fence_after();
        }
        if (!mbar_wait_warp(&b->full[slot], ph)) { raise(&b->abort_any, p.status); ok = false; break; }
        tc_fence_after();
        const uint64_t da = dI + slot_step * slot, db = dF + slot_step * slot;
        const uint32_t tacc = tmem + (uint32_t)(buf * (p.tmem_cols >> 1));
        const int ksteps = (p.K - i * 64 + 15) >> 4;
        const bool last = in == kFlush - 1 || i + 1 == i1;
        if (elect_one()) {
          for (int e = 0; e < q; ++e) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              if (kk < ksteps) tc_mma_bf16(tacc + e * cols, da + 2 * kk, db + q_step * e + f_step * kk, idesc, (in | kk) != 0);
          }
          tc_commit(&b->empty[slot]);
          if (last) tc_commit(&b->acc_full[buf]);
        }
        __syncwarp();
        if (last) ++flush;
        if (++slot == p.ns) { slot = 0; ph ^= 1; }
      }
    }
  } else {
    const int lrow = qw * 32 + lane;
    const int64_t row = row0 + lrow;
    const bool live = lrow < p.tile_rows && row < p.N;
    const int a = live ? clean_id(p.ids[row], p.L) : -1;
    {
      const int g0 = (int)__shfl_sync(0xffffffffu, a, lane & 16);
      const unsigned same = __ballot_sync(0xffffffffu, a == g0 || !live);
      const bool mixed = ((same >> (lane & 16)) & 0xffffu) != 0xffffu;
      b->row_ad[lrow] = !live || (mixed && !b->whole) ? -2 : p.want_T ? (a < 0 ? 0x7fffffff : a | 0x40000000) : a;
    }
    // These warps have nothing to do before the first slabs have been multiplied: they cut this CTA's share of the saved T.  (By CTAs of their
    // own in front of the tiles the ViT groups took 241 us, behind them 245, here 237.)
    if (p.cut && blockIdx.y == 0) {
      const int part = p.tile_rows / p.csize, oct = p.rp / 8;
      const int64_t r0 = row0 + rank * part;
      const int n = r0 >= p.N ? 0 : (int)(p.N - r0 < part ? p.N - r0 : part) * oct;
      for (int i0 = threadIdx.x - 64; i0 < n; i0 += 4 * 128) {
        float4 t[4][2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = i0 + e * 128, lr = i / oct, k = (i - lr * oct) * 8;
          t[e][0] = t[e][1] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (i < n && k < p.r) {
            const float4* q = reinterpret_cast<const float4*>(p.prep.T + (r0 + lr) * p.r + k);
            t[e][0] = q[0];
            t[e][1] = q[1];
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = i0 + e * 128, lr = i / oct, k = (i - lr * oct) * 8;
          if (i >= n) break;
          const float v[8] = {t[e][0].x, t[e][0].y, t[e][0].z, t[e][0].w, t[e][1].x, t[e][1].y, t[e][1].z, t[e][1].w};
          put_pieces(p.prep.P + (r0 + lr) * 3 * p.rp + k, p.rp, v);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) R[c][i] = 0.f;
    bool ok = true;
    int flush = 0;
    for (int q0 = 0; q0 < nad && ok; q0 += p.q_max) {
      const int q = nad - q0 < p.q_max ? nad - q0 : p.q_max;
      for (int i = i0; i < i1 && ok; i += kFlush, ++flush) {
        const int buf = flush & 1;
        ok = mbar_wait_warp(&b->acc_full[buf], (flush >> 1) & 1);
        if (!ok) { raise(&b->abort_any, p.status); break; }
        tc_fence_after();
        const uint32_t t = tmem + (uint32_t)(buf * (p.tmem_cols >> 1)) + ((uint32_t)(qw * 32) << 16);
        for (int e = 0; e < q; ++e) {
          const bool take = a >= 0 && a == b->ad[q0 + e];
          if (!__any_sync(0xffffffffu, take)) continue;
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            if (16 * c >= cols) continue;
            float v[16];
            tmem_ld16(t + e * cols + 16 * c, v);
#pragma unroll
            for (int k = 0; k < 16; ++k) R[c][k] += take ? v[k] : 0.f;
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&b->acc_empty[buf]);
      }
    }
  }

  // The ring has been read: it takes the parts, [rank][row of the share][cols], rows 16 bytes apart more than they are long
  const int share = p.tile_rows / p.csize, pitch = cols + 4;
  float* red = reinterpret_cast<float*>(ring);
  if (p.csize > 1) { cluster_arrive(); cluster_wait(); }       // every CTA of the cluster runs, and is through with its ring
  if (warp >= 2) {
    const int lrow = qw * 32 + lane;
    if (lrow < p.tile_rows) {
      const int owner = lrow / share, at = (rank * share + lrow - owner * share) * pitch;
      const uint32_t to = p.csize > 1 ? cluster_addr(smem_u32(red + at), (uint32_t)owner) : 0u;
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        if (16 * c >= cols) continue;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          if (p.csize > 1)
            asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + (uint32_t)(16 * c + i) * 4), "f"(R[c][i]), "f"(R[c][i + 1]),
                         "f"(R[c][i + 2]), "f"(R[c][i + 3])
                         : "memory");
          else
            *reinterpret_cast<float4*>(red + at + 16 * c + i) = make_float4(R[c][i], R[c][i + 1], R[c][i + 2], R[c][i + 3]);
        }
      }
    }
  }
  if (p.csize > 1) { cluster_arrive(); cluster_wait(); }
  if (warp >= 2) {
    if (p.csize == 1) named_bar_sync(1, 128);
    const int oct = cols / 8;
    for (int u = threadIdx.x - 64; u < share * oct; u += 128) {
      const int lr = u / oct, k = (u - lr * oct) * 8, code = b->row_ad[rank * share + lr];
      if (code == -2) continue;
      const int64_t row = row0 + rank * share + lr;
      const int a = code == 0x7fffffff ? -1 : code < 0 ? -1 : code & 0x3fffffff;
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (a >= 0) {
        for (int q = 0; q < p.csize; ++q) {
          const float4* f = reinterpret_cast<const float4*>(red + (q * share + lr) * pitch + k);
          const float4 x = f[0], y = f[1];
          v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w; v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
        }
        const float s = p.scale ? p.scale[a] : 1.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= s;
      }
      put_pieces(p.P + row * 3 * p.rp + kc0 + k, p.rp, v);
      if (code >= 0x40000000 && kc0 + k < p.r) {
        float4* t = reinterpret_cast<float4*>(p.T + row * p.r + kc0 + k);
        t[0] = make_float4(v[0], v[1], v[2], v[3]);
        t[1] = make_float4(v[4], v[5], v[6], v[7]);
      }
    }
    fence_proxy_async_all();
  }

  tc_fence_before();
  __syncthreads();
  if (*reinterpret_cast<volatile int*>(&b->abort_any)) {
    // give loads that are still in flight time to land before the shared memory is released
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) { }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, p.tmem_cols);
  }
  if (!p.first) dep_wait();            // this kernel is done only after the one before it
}

// ------------------------------------------------------------------------------------------------ Out^T = W In^T + G_a T^T
struct OutParams {
  int64_t N; int P, K, nk;                  // rows, output features, reduction of the shared product, its slabs
  int r, rp, L;
  int mn;                                   // 0: W is P x K and G_a P x r; 1: W is K x P and G_a r x P
  const int* ids; const float* T; const bf16* Tp;      // T in fp32 (few_kernel), in pieces (wide_kernel)
  const bf16* G; int64_t strideG;
  bf16* Out;
  int bn, nft, ntiles, ns, slot_bytes, tmem_cols;
  int csize, share, g_slots;                // few_kernel: CTAs of a cluster, rows that each finishes, pieces of G at a time
  int* status;
};

// A warp's 32 features of 32 rows with mixed adapters, as it holds them between TMEM and the result (v[h][4 j + i]: feature 16 h + lane / 4 (+ 8
// for i >= 2), row 8 j + 2 (lane % 4) (+ 1 for odd i), which is how mma.sync lays out a 16 x 8 accumulator): v += G_a T^T for the rows
// of each adapter that occurs.  id: lane l has row l's adapter, -1 where there is nothing to add.  The product is formed for all rows
// of eight that have one of the adapter's, and each row takes its own: nothing is masked by zeros.
//
// Operands come from global memory straight into fragments, for 64 values of r at once.  Beside the tiles' loads a trip to memory takes 2000
// to 3000 cycles, and shared memory is busy with them and the MMAs' operands: sums over the fp32 pipes with T in shared memory
// took 13,000 cycles for 16 rows at rank 64.
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
// A lane's words of G_a for 32 features and 64 values of r: as mma.sync wants them where a feature's values lie together, else (p.mn) by
// 8 x 8 blocks as they lie, a row of r a lane group, to be transposed by turn_g (two 2-byte loads for each word instead: 5625 rows, 72 -> 536,
// rank 72, five adapters in any order, took 207 us in this kernel).
__device__ __forceinline__ void load_g(const OutParams& p, int a, int f0, int k0, int kn, int lane, uint32_t (&u)[2][4][4]) {
  const bf16* g = p.G + a * p.strideG;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int x = 0; x < 2; ++x) {            // a feature past the last one reads what the last ones do (P is a multiple of 8)
      const int f = f0 + 16 * h + 8 * x + (lane >> 2), ff = f < p.P ? f : p.P - 1;
      const int b0 = f0 + 16 * h + 8 * x, fb = b0 < p.P ? b0 : p.P - 8;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int k = k0 + 16 * kk + 8 * y;
          uint32_t w = 0u;
          if (16 * kk + 8 * y < kn) {
            if (!p.mn) w = *reinterpret_cast<const uint32_t*>(g + (int64_t)ff * p.r + k + 2 * (lane & 3));
            else w = *reinterpret_cast<const uint32_t*>(g + (int64_t)(k + (lane >> 2)) * p.P + fb + 2 * (lane & 3));
          }
          u[h][kk][2 * y + x] = w;
        }
    }
}
__device__ __forceinline__ void turn_g(uint32_t (&u)[2][4][4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int i = 0; i < 4; ++i) asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %0;" : "+r"(u[h][kk][i]));
}
__device__ __forceinline__ void add_mixed(const OutParams& p, int64_t row0, int id, int f0, int lane, uint32_t (&v)[2][16]) {
  const unsigned live = __ballot_sync(0xffffffffu, id >= 0);
  if (live == 0u) return;
  const unsigned same = __match_any_sync(0xffffffffu, id);       // every lane, before any condition
  const unsigned heads = __ballot_sync(0xffffffffu, id >= 0 && lane == __ffs(same) - 1);   // an adapter's first row
#pragma unroll 1
  for (int k0 = 0; k0 < p.r; k0 += 64) {
    const int kn = p.r - k0 < 64 ? p.r - k0 : 64;                // a multiple of 8; T's pieces have zeros up to the next 16
    unsigned left = heads;
    int h = __ffs(left) - 1;
    left &= left - 1;
    uint32_t t[2][4][4][2], g[2][4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      int64_t row = row0 + 8 * j + (lane >> 2);
      if (row >= p.N) row = p.N - 1;
      const bf16* q = p.Tp + row * 3 * p.rp + k0 + 2 * (lane & 3);
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
          for (int y = 0; y < 2; ++y)
            t[c][j][kk][y] = 16 * kk < kn ? *reinterpret_cast<const uint32_t*>(q + c * p.rp + 16 * kk + 8 * y) : 0u;
    }
    load_g(p, __shfl_sync(0xffffffffu, id, h), f0, k0, kn, lane, g);
#pragma unroll 1
    while (true) {
      const unsigned rows = __shfl_sync(0xffffffffu, same, h) & live;
      if (p.mn) turn_g(g);
      float c[2][4][4];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) c[m][j][i] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (((rows >> (8 * j)) & 0xffu) == 0u) continue;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          if (16 * kk >= kn) break;
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            mma_16x8x16(c[m][j], g[m][kk], t[1][j][kk]);
            mma_16x8x16(c[m][j], g[m][kk], t[0][j][kk]);
          }
        }
      }
      h = __ffs(left) - 1;
      left &= left - 1;
      if (h >= 0) load_g(p, __shfl_sync(0xffffffffu, id, h), f0, k0, kn, lane, g);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool take = (rows >> (8 * j + 2 * (lane & 3) + (i & 1))) & 1u;
#pragma unroll
          for (int m = 0; m < 2; ++m)
            if (take) v[m][4 * j + i] = __float_as_uint(__uint_as_float(v[m][4 * j + i]) + c[m][j][i]);
        }
      if (h < 0) break;
    }
  }
}

constexpr int kWideThreads = 192;
constexpr int kABytes = 16384;            // 128 features x 64 bf16
struct WideBars {
  uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int abort_any;
};

// The slabs of a tile behind the shared product's: for every run of groups (lane l: group l's adapter) with one adapter, piece by piece.
// body(a, g0, g1, piece, j) returns false to stop.
template <typename F>
__device__ __forceinline__ bool for_runs(int gid, int ngroups, int rp, F&& body) {
  int g = 0;
  while (g < ngroups) {
    const int a = (int)uniform(__shfl_sync(0xffffffffu, gid, g));
    if (a < 0) { ++g; continue; }
    int e = g + 1;
    while (e < ngroups && (int)uniform(__shfl_sync(0xffffffffu, gid, e)) == a) ++e;
    for (int piece = 0; piece < 2; ++piece)
      for (int j = 0; j * 64 < rp; ++j)
        if (!body(a, g, e, piece, j)) return false;
    g = e;
  }
  return true;
}

// kPair: two CTAs have a tile of 256 features x bn rows together, 128 features each, and load half of the rows each: 32 KB a slab and
// CTA instead of 48, which arrive as fast as they are multiplied (512 cycles against 520; alone 768).  An MMA's columns then come in
// 32s, and so do the groups.
//
// The ring is as deep as shared memory lets it be: beside the other SMs' loads a load takes 2000 to 3000 cycles (8191 x 4096 x 4096, four
// slabs of 32 KB 194 us, five 169).
// Eight epilogue warps, two for each quarter of the TMEM lanes, which take the tile's 32-row pieces in turn: a piece is a chain of latencies
// (ViT groups, twelve slabs a tile: four warps were busy for 10,000 of a tile's 12,000 cycles).
constexpr int kWideAll = 320, kEpiWarps = 8;
constexpr int kEpiBytes = 2048;            // of an epilogue warp: a tile of 32 rows x 32 features
template <bool kPair>
__global__ void __launch_bounds__(kWideAll, 1)
wide_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmIn, const __grid_constant__ CUtensorMap tmG,
            const __grid_constant__ CUtensorMap tmT, const __grid_constant__ CUtensorMap tmOut, const __grid_constant__ OutParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* stg = ring + (size_t)p.ns * p.slot_bytes;
  WideBars* b = reinterpret_cast<WideBars*>(stg + kEpiWarps * kEpiBytes);
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  constexpr int kCtas = kPair ? 2 : 1, kGroup = kG * kCtas;       // rows of a group
  const int rank = kPair ? (int)(blockIdx.x & 1) : 0;
  const int first_tile = (int)blockIdx.x / kCtas, tile_step = (int)gridDim.x / kCtas;
  const int half = p.bn / kCtas;                                  // rows that this CTA loads
  dep_launch();
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.ns; ++i) { mbar_init(&b->full[i], 1); mbar_init(&b->empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&b->acc_full[i], 1); mbar_init(&b->acc_empty[i], kEpiWarps * kCtas); }
    b->abort_any = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tmW); tma_prefetch_desc(&tmIn); tma_prefetch_desc(&tmG); tma_prefetch_desc(&tmT); tma_prefetch_desc(&tmOut);
  }
  if (warp == 1) {
    if constexpr (kPair) tmem_alloc_pair(&b->tmem_base, p.tmem_cols); else tmem_alloc(&b->tmem_base, p.tmem_cols);
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (kPair) { cluster_arrive(); cluster_wait(); }      // the other CTA's barriers are there
  tc_fence_after();
  const uint32_t tmem = uniform(*reinterpret_cast<volatile uint32_t*>(&b->tmem_base));
  const int ngroups = p.bn / kGroup;
  // lane g: the adapter of group g, -1 none, -2 mixed
  auto groups = [&](int row0, bool& bad, int (&id)[8]) {
    int gid = group_ids(p.ids, p.N, p.L, row0, lane, bad, id);
    if constexpr (kPair) {
      const int x = __shfl_sync(0xffffffffu, gid, (2 * lane) & 31), y = __shfl_sync(0xffffffffu, gid, (2 * lane + 1) & 31);
      // a second half behind the last row goes with the first
      gid = x == y || (int64_t)row0 + lane * kGroup + kG >= p.N ? x : -2;
    }
    return gid;
  };
  // The kernels before this one started only after all that a caller had in the stream before: x, W, the factors and the map are
  // complete.  T alone comes from them, and is waited for where it is read.

  if (warp == 0) {
    int slot = 0, ph = 1;
    bool ok = true, waited = false;
    const uint32_t tx = kCtas * (kABytes + half * 128);
    const uint32_t full0 = kPair ? cluster_addr(smem_u32(&b->full[0]), 0) : 0u;      // the first CTA's barriers count both CTAs' bytes
    auto load_2d = [&](uint8_t* dst, const CUtensorMap* m, int s, int c0, int c1) {
      if constexpr (kPair) tma_load_2d_pair(dst, m, full0 + (uint32_t)s * 8, c0, c1); else tma_load_2d(dst, m, &b->full[s], c0, c1);
    };
    auto load_3d = [&](uint8_t* dst, const CUtensorMap* m, int s, int c0, int c1, int c2) {
      if constexpr (kPair) tma_load_3d_pair(dst, m, full0 + (uint32_t)s * 8, c0, c1, c2); else tma_load_3d(dst, m, &b->full[s], c0, c1, c2);
    };
    for (int tile = first_tile; tile < p.ntiles && ok; tile += tile_step) {
      const int f0 = ((tile % p.nft) * kCtas + rank) * 128, row0 = (tile / p.nft) * p.bn;
      bool bad;
      int id[8];
      const int gid = groups(row0, bad, id);
      for (int i = 0; i < p.nk; ++i) {
        if (!mbar_wait_warp(&b->empty[slot], ph)) { raise(&b->abort_any, p.status); ok = false; break; }
        if (elect_one()) {
          uint8_t* dst = ring + (size_t)slot * p.slot_bytes;
          if (rank == 0) mbar_arrive_expect_tx(&b->full[slot], tx);
          if (p.mn) { load_2d(dst, &tmW, slot, f0, i * 64); load_2d(dst + 8192, &tmW, slot, f0 + 64, i * 64); }
          else load_2d(dst, &tmW, slot, i * 64, f0);
          load_2d(dst + kABytes, &tmIn, slot, i * 64, row0 + rank * half);
        }
        __syncwarp();
        if (++slot == p.ns) { slot = 0; ph ^= 1; }
      }
      if (!ok) break;
      if (!waited) { dep_wait(); fence_proxy_async_all(); waited = true; }
      ok = for_runs(gid, ngroups, p.rp, [&](int a, int g0, int g1, int piece, int j) {
        if (!mbar_wait_warp(&b->empty[slot], ph)) { raise(&b->abort_any, p.status); return false; }
        if (elect_one()) {
          uint8_t* dst = ring + (size_t)slot * p.slot_bytes;
          if (rank == 0) mbar_arrive_expect_tx(&b->full[slot], tx);
          if (p.mn) { load_3d(dst, &tmG, slot, f0, j * 64, a); load_3d(dst + 8192, &tmG, slot, f0 + 64, j * 64, a); }
          else load_3d(dst, &tmG, slot, j * 64, f0, a);
          // alone: all rows of the tile; a pair: each its half of the run's rows, at the head of the slot
          load_2d(dst + kABytes, &tmT, slot, piece * p.rp + j * 64, kPair ? row0 + g0 * kGroup + rank * (g1 - g0) * kG : row0);
        }
        __syncwarp();
        if (++slot == p.ns) { slot = 0; ph ^= 1; }
        return true;
      });
    }
  } else if (warp == 1) {
    if (rank == 0) {
      int slot = 0, ph = 0, it = 0;
      bool ok = true, waited = false;
      const uint32_t base = uniform(smem_u32(ring)), idesc = instr_desc_bf16(128 * kCtas, p.bn, p.mn, 0);
      const uint64_t dA = smem_desc_sw128(base, p.mn ? 8192 : 16), dB = smem_desc_sw128(base + kABytes, 16);
      const uint64_t a_step = p.mn ? 128u : 2u, slot_step = (uint64_t)(p.slot_bytes >> 4);
      auto mma = [&](uint32_t d, uint64_t da, uint64_t db, uint32_t id, uint32_t acc) {
        if constexpr (kPair) tc_mma_bf16_pair(d, da, db, id, acc); else tc_mma_bf16(d, da, db, id, acc);
      };
      auto commit = [&](uint64_t* bar) {
        if constexpr (kPair) tc_commit_pair(bar); else tc_commit(bar);
      };
      for (int tile = first_tile; tile < p.ntiles && ok; tile += tile_step, ++it) {
        const int row0 = (tile / p.nft) * p.bn, buf = it & 1;
        bool bad;
        int id[8];
        const int gid = groups(row0, bad, id);
        if (!mbar_wait_warp(&b->acc_empty[buf], ((it >> 1) & 1) ^ 1)) { raise(&b->abort_any, p.status); break; }
        tc_fence_after();
        const uint32_t tacc = tmem + (uint32_t)(buf * (p.tmem_cols >> 1));
        for (int i = 0; i < p.nk; ++i) {
          if (!mbar_wait_warp(&b->full[slot], ph)) { raise(&b->abort_any, p.status); ok = false; break; }
          tc_fence_after();
          const uint64_t da = dA + slot_step * slot, db = dB + slot_step * slot;
          const int ksteps = (p.K - i * 64 + 15) >> 4;
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              if (kk < ksteps) mma(tacc, da + a_step * kk, db + 2 * kk, idesc, (i | kk) != 0);
            commit(&b->empty[slot]);
          }
          __syncwarp();
          if (++slot == p.ns) { slot = 0; ph ^= 1; }
        }
        if (!ok) break;
        // What is waited for from here on (the adapters' slabs, accumulators given back) comes only when the kernel in front is done, which may
        // take longer than a bounded wait may.
        if (!waited) { dep_wait(); waited = true; }
        ok = for_runs(gid, ngroups, p.rp, [&](int, int g0, int g1, int, int j) {
          if (!mbar_wait_warp(&b->full[slot], ph)) { raise(&b->abort_any, p.status); return false; }
          tc_fence_after();
          const uint64_t da = dA + slot_step * slot, db = dB + slot_step * slot + (uint64_t)(kPair ? 0 : g0 * (kG * 128 >> 4));
          const uint32_t id = instr_desc_bf16(128 * kCtas, (g1 - g0) * kGroup, p.mn, 0);
          const int ksteps = (p.rp - j * 64 + 15) >> 4;
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              if (kk < ksteps) mma(tacc + g0 * kGroup, da + a_step * kk, db + 2 * kk, id, 1u);
            commit(&b->empty[slot]);
          }
          __syncwarp();
          if (++slot == p.ns) { slot = 0; ph ^= 1; }
          return true;
        });
        if (ok && elect_one()) commit(&b->acc_full[buf]);
        __syncwarp();
      }
    }
  } else {
    const int qw = warp & 3, turn = (warp - 2) >> 2;
    const uint32_t lane_base = (uint32_t)(qw * 32) << 16;
    uint8_t* tile_s = stg + (size_t)(warp - 2) * kEpiBytes;
    const uint32_t acc_empty0 = kPair ? cluster_addr(smem_u32(&b->acc_empty[0]), 0) : 0u;
    auto give_back = [&](int buf) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (kPair) mbar_arrive_cluster(acc_empty0 + (uint32_t)buf * 8); else mbar_arrive(&b->acc_empty[buf]);
      }
    };
    int it = 0;
    bool ok = true;
    dep_wait();                          // T is complete; and this kernel is done only after the ones before it
    for (int tile = first_tile; tile < p.ntiles && ok; tile += tile_step, ++it) {
      const int ftile = (tile % p.nft) * kCtas + rank, f0 = ftile * 128 + qw * 32, row0 = (tile / p.nft) * p.bn, buf = it & 1;
      bool bad;
      int id[8];
      const int gid = groups(row0, bad, id);
      const bool any_bad = __any_sync(0xffffffffu, bad && lane * 8 < p.bn);
      if (ftile == 0 && qw == 0 && any_bad && lane == 0) atomicExch(p.status, (int)AB_ERR_INVALID_ARG);
      // bit g: the adapters' part of the 16 rows from 16 g is added here
      unsigned mixed = __ballot_sync(0xffffffffu, __shfl_sync(0xffffffffu, gid, lane / kCtas) == -2 && lane < p.bn / kG);
      ok = mbar_wait_warp(&b->acc_full[buf], (it >> 1) & 1);
      if (!ok) { raise(&b->abort_any, p.status); break; }
      tc_fence_after();
      const uint32_t tacc = tmem + (uint32_t)(buf * (p.tmem_cols >> 1)) + lane_base;
      const bool live = f0 < p.P;
      const int n16 = p.bn / kG;
      bool given = false;
      for (int g0 = 2 * turn; g0 < n16; g0 += 4) {
        if (!live || (int64_t)row0 + g0 * kG >= p.N) break;
        const bool last = g0 + 4 >= n16 || (int64_t)row0 + (g0 + 4) * kG >= p.N;      // the accumulator's last columns
        uint32_t v[2][16];               // features 0..15 and 16..31 of the warp, 32 rows
        tmem_ld_16x32_nowait(tacc + g0 * kG, v[0]);
        tmem_ld_16x32_nowait(tacc + (16u << 16) + g0 * kG, v[1]);
        tmem_wait_ld();
        if (last) { give_back(buf); given = true; }
        const unsigned halves = (mixed >> g0) & 3u;
        if (halves) {
          int mine = -1;                 // row l of the 32, which lane 2 g0 + l / 8 has
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int x = __shfl_sync(0xffffffffu, id[e], 2 * g0 + (lane >> 3));
            if ((lane & 7) == e && ((halves >> (lane >> 4)) & 1u)) mine = x;
          }
          add_mixed(p, (int64_t)row0 + g0 * kG, mine, f0, lane, v);
        }
        if (elect_one()) tma_store_wait_read<0>();
        __syncwarp();
        // eight rows (columns 8 j ..) of 32 features are four fragments; transposed they are 8 rows of 64 bytes, whose 16-byte pieces
        // lie where the swizzle puts them
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t w[4];
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const __nv_bfloat162 x = __floats2bfloat162_rn(__uint_as_float(v[h >> 1][4 * j + 2 * (h & 1)]),
                                                           __uint_as_float(v[h >> 1][4 * j + 2 * (h & 1) + 1]));
            w[h] = *reinterpret_cast<const uint32_t*>(&x);
          }
          const int r = 8 * j + (lane & 7), piece = (lane >> 3) ^ ((r >> 1) & 3);
          stmatrix_x4_trans(smem_u32(tile_s) + r * 64 + piece * 16, w[0], w[1], w[2], w[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (elect_one()) {
          tma_store_2d(&tmOut, tile_s, f0, row0 + g0 * kG);
          tma_store_commit();
        }
      }
      if (!given) give_back(buf);
    }
    if (elect_one()) tma_store_wait_all();
    __syncwarp();
  }

  tc_fence_before();
  __syncthreads();
  if (*reinterpret_cast<volatile int*>(&b->abort_any)) {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) { }
    __syncthreads();
  }
  if constexpr (kPair) { cluster_arrive(); cluster_wait(); }      // nothing of the other CTA's is on its way to this one's barriers
  if (warp == 1) {
    tc_fence_after();
    if constexpr (kPair) tmem_dealloc_pair(tmem, p.tmem_cols); else tmem_dealloc(tmem, p.tmem_cols);
  }
  if constexpr (kPair) { cluster_arrive(); cluster_wait(); }
}

// ------------------------------------------------------------------------------------------------ the same for few rows
// A tile of 128 features x bn rows a cluster; its CTAs have a part of the reduction each.  Their partial sums meet in the shared memory of
// the CTA that finishes a share of the rows, which adds them in rank order.  The adapters' part goes row by row over the fp32 pipes: the
// tile's piece of G_a is fetched (once for neighbouring rows of one adapter) while W is still arriving and T not yet there.
// Loops are short and not unrolled: the code runs once, and fetching it is part of the latency.
struct FewBars {
  uint64_t full[kMaxStages], empty[kMaxStages], acc_full, g_full;
  uint32_t tmem_base;
  int abort_any;
};
constexpr int kBatch = 16;                // rows whose T and G are in shared memory at a time, at most

__global__ void __launch_bounds__(kWideThreads, 1)
few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmIn, const __grid_constant__ OutParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* gbuf = ring + (size_t)p.ns * p.slot_bytes;                          // g_slots pieces of G: [128][r], or [r][128]
  float* Tb = reinterpret_cast<float*>(gbuf + (size_t)p.g_slots * 256 * p.r);  // [kBatch][r]
  float* dl = Tb + kBatch * p.r;                                               // [share][128]: the adapters' part of this CTA's rows
  const int pitch = p.share + 4;
  float* red = dl + p.share * 128;                                             // [csize][128][pitch]: partial sums of this CTA's rows
  FewBars* b = reinterpret_cast<FewBars*>(red + (size_t)p.csize * 128 * pitch);
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int ft = (int)blockIdx.x / p.csize, rank = (int)blockIdx.x - ft * p.csize, f0 = ft * 128;
  const int64_t row0 = (int64_t)blockIdx.y * p.bn;
  const int rows = (int)(p.N - row0 < p.bn ? p.N - row0 : p.bn);
  const int per = (p.nk + p.csize - 1) / p.csize, i0 = rank * per, i1 = i0 + per < p.nk ? i0 + per : p.nk;
  const int qw = warp & 3, fl = qw * 32 + lane, t0 = rank * p.share;
  const int t1 = t0 + p.share < rows ? t0 + p.share : rows;                    // the rows that this CTA finishes
  dep_launch();
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.ns; ++i) { mbar_init(&b->full[i], 1); mbar_init(&b->empty[i], 1); }
    mbar_init(&b->acc_full, 1);
    mbar_init(&b->g_full, 1);
    b->abort_any = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tmW); tma_prefetch_desc(&tmIn);
  }
  cluster_arrive();                        // paired with the wait before the first access to another CTA's shared memory
  if (warp == 1) tmem_alloc(&b->tmem_base, p.tmem_cols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(*reinterpret_cast<volatile uint32_t*>(&b->tmem_base));
  bool ok = true;

  if (warp == 0) {
    int slot = 0, ph = 1;
    for (int i = i0; i < i1; ++i) {
      if (!mbar_wait_warp(&b->empty[slot], ph)) { raise(&b->abort_any, p.status); break; }
      if (elect_one()) {
        uint8_t* dst = ring + (size_t)slot * p.slot_bytes;
        uint64_t* bar = &b->full[slot];
        mbar_arrive_expect_tx(bar, kABytes + p.bn * 128);
        if (p.mn) { tma_load_2d(dst, &tmW, bar, f0, i * 64); tma_load_2d(dst + 8192, &tmW, bar, f0 + 64, i * 64); }
        else tma_load_2d(dst, &tmW, bar, i * 64, f0);
        tma_load_2d(dst + kABytes, &tmIn, bar, i * 64, (int)row0);
      }
      __syncwarp();
      if (++slot == p.ns) { slot = 0; ph ^= 1; }
    }
  } else if (warp == 1) {
    const uint32_t base = uniform(smem_u32(ring)), idesc = instr_desc_bf16(128, p.bn, p.mn, 0);
    const uint64_t dA = smem_desc_sw128(base, p.mn ? 8192 : 16), dB = smem_desc_sw128(base + kABytes, 16);
    const uint64_t a_step = p.mn ? 128u : 2u, slot_step = (uint64_t)(p.slot_bytes >> 4);
    int slot = 0, ph = 0;
    for (int i = i0; i < i1; ++i) {
      if (!mbar_wait_warp(&b->full[slot], ph)) { raise(&b->abort_any, p.status); break; }
      tc_fence_after();
      const uint64_t da = dA + slot_step * slot, db = dB + slot_step * slot;
      const int ksteps = (p.K - i * 64 + 15) >> 4;
      if (elect_one()) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          if (kk < ksteps) tc_mma_bf16(tmem, da + a_step * kk, db + 2 * kk, idesc, (i > i0 || kk) ? 1u : 0u);
        tc_commit(&b->empty[slot]);
      }
      __syncwarp();
      if (++slot == p.ns) { slot = 0; ph ^= 1; }
    }
    if (elect_one()) tc_commit(&b->acc_full);
    __syncwarp();
  } else {
    const int nf = p.P - f0 < 128 ? p.P - f0 : 128;          // features of the tile
    bool waited = false;
    for (int b0 = t0, turn = 0; b0 < t1;) {
      // the batch: rows up to the one that would want a piece of G too many; a row's piece
      const int id = lane < kBatch && b0 + lane < t1 ? clean_id(p.ids[row0 + b0 + lane], p.L) : -1;
      const int before = __shfl_up_sync(0xffffffffu, id, 1);
      const bool head = id >= 0 && (lane == 0 || id != before);
      const unsigned heads = __ballot_sync(0xffffffffu, head);
      const int piece = __popc(heads & (0xffffffffu >> (31 - lane))) - 1;
      const unsigned over = __ballot_sync(0xffffffffu, head && piece == p.g_slots);
      int n = t1 - b0 < kBatch ? t1 - b0 : kBatch;
      if (over && __ffs(over) - 1 < n) n = __ffs(over) - 1;
      const int pieces = __popc(heads & (n < 32 ? (1u << n) - 1u : 0xffffffffu));
      if (warp == 2 && pieces > 0) {
        if (lane == 0) mbar_arrive_expect_tx(&b->g_full, (uint32_t)(pieces * nf * p.r * 2));
        __syncwarp();
        unsigned left = heads;
        for (int g = 0; g < pieces; ++g) {
          const int e = __ffs(left) - 1;
          left &= left - 1;
          const bf16* G = p.G + __shfl_sync(0xffffffffu, id, e) * p.strideG;
          uint8_t* dst = gbuf + (size_t)g * 256 * p.r;
          if (!p.mn) {
            if (lane == 0) bulk_load(dst, G + (int64_t)f0 * p.r, (uint32_t)(nf * p.r * 2), &b->g_full);
          } else {
            for (int k = lane; k < p.r; k += 32) bulk_load(dst + k * 256, G + (int64_t)k * p.P + f0, (uint32_t)(nf * 2), &b->g_full);
          }
        }
        __syncwarp();
      }
      if (!waited) {
        dep_wait();                        // T is complete; and this kernel is done only after the ones before it
        waited = true;
      }
      const int rq = p.r / 4;
      for (int i = threadIdx.x - 64; i < n * rq; i += 128) {
        const int e = i / rq, c = i - e * rq;
        *reinterpret_cast<float4*>(Tb + e * p.r + 4 * c) = *reinterpret_cast<const float4*>(p.T + (row0 + b0 + e) * p.r + 4 * c);
      }
      if (pieces > 0 && !mbar_wait_warp(&b->g_full, turn & 1)) { raise(&b->abort_any, p.status); ok = false; }
      named_bar_sync(1, 128);
      // four rows at a time, whose sums hide each other's latency; a row without an adapter is summed with whatever lies there, and
      // gets 0
      const int oct = p.r / 8, c0 = fl % oct;
#pragma unroll 1
      for (int e0 = 0; e0 < n; e0 += 4) {
        const uint8_t* G[4];
        const float* T[4];
        float s[4];
        unsigned has = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int a = __shfl_sync(0xffffffffu, id, e0 + e), g = __shfl_sync(0xffffffffu, piece, e0 + e);
          has |= a >= 0 && e0 + e < n ? 1u << e : 0u;
          G[e] = gbuf + (size_t)(a >= 0 && e0 + e < n ? g : 0) * 256 * p.r + (p.mn ? fl * 2 : fl * p.r * 2);
          T[e] = Tb + (e0 + e) * p.r;
          s[e] = 0.f;
        }
        if (!p.mn) {
          // a lane begins at an eighth of its own: lanes a whole number of bank rows apart would meet in one bank
          int c = c0;
#pragma unroll 1
          for (int i = 0; i < oct; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint4 u = *reinterpret_cast<const uint4*>(G[e] + c * 16);
              const float4 x = *reinterpret_cast<const float4*>(T[e] + 8 * c), y = *reinterpret_cast<const float4*>(T[e] + 8 * c + 4);
              const float t[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
              dot8(u, t, s[e]);
            }
            if (++c == oct) c = 0;
          }
        } else {
#pragma unroll 4
          for (int k = 0; k < p.r; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = fmaf(__bfloat162float(*reinterpret_cast<const bf16*>(G[e] + k * 256)), T[e][k], s[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e0 + e < n) dl[(b0 - t0 + e0 + e) * 128 + fl] = ((has >> e) & 1u) ? s[e] : 0.f;
      }
      named_bar_sync(1, 128);              // the pieces and T have been read
      b0 += n;
      turn += pieces > 0 ? 1 : 0;          // a batch without pieces does not use the barrier
    }
    if (!waited) dep_wait();
    if (ft == 0 && rank == 0 && warp == 2) {
      bool bad = false;
      for (int t = lane; t < rows; t += 32) bad |= p.ids[row0 + t] < -1 || p.ids[row0 + t] >= p.L;
      if (__any_sync(0xffffffffu, bad) && lane == 0) atomicExch(p.status, (int)AB_ERR_INVALID_ARG);
    }
    if (!mbar_wait_warp(&b->acc_full, 0)) { raise(&b->abort_any, p.status); ok = false; }
  }
  cluster_wait();                          // every CTA of the cluster runs
  if (warp >= 2) {
    tc_fence_after();
    const uint32_t dst = smem_u32(red) + (uint32_t)((rank * 128 + fl) * pitch * 4);
    int owner = 0, at = 0;
    uint32_t to = cluster_addr(dst, 0);
#pragma unroll 1
    for (int c = 0; c < p.bn; c += kG) {
      float v[kG];
      if (ok && i1 > i0) tmem_ld16(tmem + ((uint32_t)(qw * 32) << 16) + c, v);
      else {
#pragma unroll
        for (int e = 0; e < kG; ++e) v[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < kG; e += 4) {    // a share is a multiple of four rows
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + (uint32_t)at * 4), "f"(v[e]), "f"(v[e + 1]), "f"(v[e + 2]),
                     "f"(v[e + 3])
                     : "memory");
        at += 4;
        if (at == p.share && c + e + 4 < p.bn) { at = 0; to = cluster_addr(dst, ++owner); }
      }
    }
    tc_fence_before();
  }
  cluster_arrive();
  cluster_wait();                          // and has written its sums
  if (warp >= 2 && f0 + fl < p.P) {
    bf16* out = p.Out + (row0 + t0) * p.P + f0 + fl;
    const float* r0 = red + fl * pitch;
#pragma unroll 2
    for (int t = 0; t < t1 - t0; t += 4) {
      float4 v = *reinterpret_cast<const float4*>(r0 + t);
#pragma unroll 3
      for (int q = 1; q < p.csize; ++q) {
        const float4 x = *reinterpret_cast<const float4*>(r0 + q * 128 * pitch + t);
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
      }
      const float y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e, out += p.P)
        if (t0 + t + e < t1) *out = __float2bfloat16_rn(y[e] + dl[(t + e) * 128 + fl]);
    }
  }
  __syncthreads();
  if (*reinterpret_cast<volatile int*>(&b->abort_any)) {
    const uint64_t w0 = globaltimer_ns();
    while (globaltimer_ns() - w0 < 200000ull) { }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, p.tmem_cols);
  }
}

// ------------------------------------------------------------------------------------------------ gradients of the factors
struct GradJob { int P, tiles; float* out; int64_t strideO, o_f, o_k, slice_stride; };
struct GradParams {
  GradJob job[2];
  int64_t N; int r, rp, L, nslab;
  int halves;                               // parts of the r values a CTA has one of (128 each)
  int slices;
  int stacked;                              // the three pieces side by side as columns of one MMA
  int nb;                                   // 64-column boxes of the small operand a slab
  int ns, slot_bytes, tmem_cols;
  const int* ids; const uint4* list; const int* count;
  int check;                                // report bad map entries (no other kernel of the call does)
  int* status;
};
struct GradBars {
  uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int abort_any;
};

// The adapter at place `place` in the order of descending count (ties: the lower first), so that the longest sums start first.  Whole warp.
__device__ __forceinline__ int longest(const int* __restrict__ count, int L, int place, int lane) {
  if (L > 256) return place;               // many adapters: each is a small share of the work
  int mine = -1;
  for (int a0 = 0; a0 < L; a0 += 32) {
    const int a = a0 + lane, c = a < L ? count[a] : -1;
    int ahead = 0;
    for (int x = 0; x < L; ++x) { const int cx = count[x]; ahead += cx > c || (cx == c && x < a) ? 1 : 0; }
    const unsigned hit = __ballot_sync(0xffffffffu, a < L && ahead == place);
    if (hit) mine = a0 + __ffs(hit) - 1;
  }
  return mine;
}

// Four slabs (256 rows) are summed in TMEM, the rest in registers, as in project_tc_kernel.
template <int kChunks>                    // up to 16 kChunks values of r a CTA
__global__ void __launch_bounds__(kWideThreads)
adapter_grad_tc_kernel(const __grid_constant__ CUtensorMap tmAct0, const __grid_constant__ CUtensorMap tmS0,
                       const __grid_constant__ CUtensorMap tmAct1, const __grid_constant__ CUtensorMap tmS1, const __grid_constant__ GradParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  GradBars* b = reinterpret_cast<GradBars*>(ring + (size_t)p.ns * p.slot_bytes);
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  int item = blockIdx.x;
  const int slice = item % p.slices; item /= p.slices;
  const int half = item % p.halves; item /= p.halves;
  const int tiles = p.job[0].tiles + p.job[1].tiles;
  int tile = item % tiles;
  const int place = item / tiles, j = tile < p.job[0].tiles ? 0 : 1;
  if (j) tile -= p.job[0].tiles;
  const int f0 = tile * 128, kc0 = half * 128, kcols = p.rp - kc0 < 128 ? p.rp - kc0 : 128;
  const CUtensorMap* tmA = j ? &tmAct1 : &tmAct0;
  const CUtensorMap* tmS = j ? &tmS1 : &tmS0;
  const int pieces = p.stacked ? 1 : 3;

  if (threadIdx.x == 0) {
    for (int i = 0; i < p.ns; ++i) { mbar_init(&b->full[i], 1); mbar_init(&b->empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&b->acc_full[i], 1); mbar_init(&b->acc_empty[i], 4); }
    b->abort_any = 0;
    fence_barrier_init();
    tma_prefetch_desc(tmA); tma_prefetch_desc(tmS);
  }
  dep_wait();
  if (warp == 1) tmem_alloc(&b->tmem_base, p.tmem_cols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  dep_launch();
  const uint32_t tmem = uniform(*reinterpret_cast<volatile uint32_t*>(&b->tmem_base));
  const int a = longest(p.count, p.L, place, lane);
  const int cnt = (int)uniform(p.count[a]), per = (cnt + p.slices - 1) / p.slices;
  const int e0 = slice * per < cnt ? slice * per : cnt, e1 = e0 + per < cnt ? e0 + per : cnt;
  const uint4* list = p.list + (int64_t)a * p.nslab;
  if (p.check && blockIdx.x == 0) {
    bool bad = false;
    for (int64_t i = threadIdx.x; i < p.N; i += kWideThreads) bad |= p.ids[i] < -1 || p.ids[i] >= p.L;
    if (bad) atomicExch(p.status, (int)AB_ERR_INVALID_ARG);
  }

  if (warp == 0) {
    fence_proxy_async_all();               // the pieces were written by plain stores
    int slot = 0, ph = 1;
    bool ok = true;
    const uint32_t tx = kABytes + p.nb * 8192;
    uint32_t mine = 0;                     // lane l: entry l of the 32 at hand
    for (int e = e0; e < e1 && ok; ++e) {
      if (((e - e0) & 31) == 0) mine = e + lane < e1 ? list[e + lane].x : 0u;
      const int row0 = (int)__shfl_sync(0xffffffffu, mine, (e - e0) & 31) * 64;
      for (int q = 0; q < pieces; ++q) {
        if (!mbar_wait_warp(&b->empty[slot], ph)) { raise(&b->abort_any, p.status); ok = false; break; }
        if (elect_one()) {
          uint8_t* dst = ring + (size_t)slot * p.slot_bytes;
          uint64_t* bar = &b->full[slot];
          mbar_arrive_expect_tx(bar, tx);
          tma_load_2d(dst, tmA, bar, f0, row0);
          tma_load_2d(dst + 8192, tmA, bar, f0 + 64, row0);
          for (int h = 0; h < p.nb; ++h) tma_load_2d(dst + kABytes + h * 8192, tmS, bar, (p.stacked ? 0 : q * p.rp + kc0) + 64 * h, row0);
        }
        __syncwarp();
        if (++slot == p.ns) { slot = 0; ph ^= 1; }
      }
    }
  } else if (warp == 1) {
    const uint32_t base = uniform(smem_u32(ring)), idesc = instr_desc_bf16(128, p.stacked ? 3 * p.rp : kcols, 1, 1);
    const uint64_t dA = smem_desc_sw128(base, 8192), dS = smem_desc_sw128(base + kABytes, 8192), slot_step = (uint64_t)(p.slot_bytes >> 4);
    int slot = 0, ph = 0;
    bool ok = true;
    uint4 mine = make_uint4(0u, 0u, 0u, 0u);
    for (int e = e0, n = 0; e < e1 && ok; ++e, ++n) {
      if ((n & 31) == 0 && e + lane < e1) mine = list[e + lane];
      const unsigned lo = __shfl_sync(0xffffffffu, mine.y, n & 31), hi = __shfl_sync(0xffffffffu, mine.z, n & 31);
      const int flush = n / kFlush, buf = flush & 1, in = n % kFlush, turn = flush >> 1;
      const bool others = (lo & hi) != 0xffffffffu;
      if (in == 0) {
        if (!mbar_wait_warp(&b->acc_empty[buf], (turn & 1) ^ 1)) { raise(&b->abort_any, p.status); break; }
        tc_fence_after();
      }
      const uint32_t tacc = tmem + (uint32_t)(buf * (p.tmem_cols >> 1));
      for (int q = 0; q < pieces; ++q) {
        if (!mbar_wait_warp(&b->full[slot], ph)) { raise(&b->abort_any, p.status); ok = false; break; }
        if (others) {
          // rows that are not this adapter's: cleared in both operands, whatever they hold
          uint8_t* s = ring + (size_t)slot * p.slot_bytes;
          for (int r4 = 0; r4 < 64; r4 += 4) {
            const int rr = r4 + (lane >> 3);
            const bool mine = ((rr < 32 ? lo >> rr : hi >> (rr - 32)) & 1u) != 0;
            if (!mine)
              for (int h = 0; h < 2 + p.nb; ++h)
                *reinterpret_cast<uint4*>(s + h * 8192 + rr * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async_smem();
          __syncwarp();
        }
        tc_fence_after();
        const uint64_t da = dA + slot_step * slot, ds = dS + slot_step * slot;
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) tc_mma_bf16(tacc, da + 128 * kk, ds + 128 * kk, idesc, (in | q | kk) != 0);
          tc_commit(&b->empty[slot]);
        }
        __syncwarp();
        if (++slot == p.ns) { slot = 0; ph ^= 1; }
      }
      if (ok && (in == kFlush - 1 || e + 1 == e1) && elect_one()) tc_commit(&b->acc_full[buf]);
      __syncwarp();
    }
  } else {
    const int qw = warp & 3, f = f0 + qw * 32 + lane;
    const uint32_t lane_base = (uint32_t)(qw * 32) << 16;
    float R[kChunks][16];
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) R[c][i] = 0.f;
    const int flushes = (e1 - e0 + kFlush - 1) / kFlush;
    bool ok = true;
    for (int n = 0; n < flushes && ok; ++n) {
      const int buf = n & 1, turn = n >> 1;
      ok = mbar_wait_warp(&b->acc_full[buf], turn & 1);
      if (!ok) { raise(&b->abort_any, p.status); break; }
      tc_fence_after();
      const uint32_t t = tmem + (uint32_t)(buf * (p.tmem_cols >> 1)) + lane_base;
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        if (16 * c >= kcols) continue;
        uint32_t u[3][16];
        tmem_ld16_nowait(t + 16 * c, u[0]);
        if (p.stacked) { tmem_ld16_nowait(t + p.rp + 16 * c, u[1]); tmem_ld16_nowait(t + 2 * p.rp + 16 * c, u[2]); }
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float v = __uint_as_float(u[0][i]);
          if (p.stacked) v += __uint_as_float(u[1][i]) + __uint_as_float(u[2][i]);
          R[c][i] += v;
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&b->acc_empty[buf]);
    }
    const GradJob& J = p.job[j];
    if (f < J.P) {
      float* out = J.out + slice * J.slice_stride + a * J.strideO + (int64_t)f * J.o_f;
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        if (16 * c >= kcols) continue;
        const int k = kc0 + 16 * c;
        if (J.o_k == 1) {
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            if (k + i < p.r) *reinterpret_cast<float4*>(out + k + i) = make_float4(R[c][i], R[c][i + 1], R[c][i + 2], R[c][i + 3]);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (k + i < p.r) out[(int64_t)(k + i) * J.o_k] = R[c][i];
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*reinterpret_cast<volatile int*>(&b->abort_any)) {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) { }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, p.tmem_cols);
  }
}

// ------------------------------------------------------------------------------------------------ host
// Lets a kernel of little shared memory begin on SMs whose memory is set up for one that takes all of it.
template <typename K>
cudaError_t beside_large(K* kernel) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
}

int pad16(int r) { return (r + 15) / 16 * 16; }
int pow2_cols(int c) { int v = 32; while (v < c) v <<= 1; return v; }

constexpr int kFewRows = 128;
// Whether few_kernel takes the rows: up to 128, and more while tiles of 64 rows leave an SM each for two CTAs of a cluster
bool few_rows(int64_t N, int P) {
  if (N <= kFewRows) return true;
  const int sms = sm_count() > 0 ? sm_count() : 148;
  return N <= 1024 && (N + 63) / 64 * ((P + 127) / 128) * 2 <= sms;
}

// the stride of a lone matrix may be anything
int stack_map(CUtensorMap* m, const AdapterCall& c, const void* F, int rows, int cols, int64_t stride, int box_rows) {
  return make_tensor_map_stack(m, F, c.L, rows, cols, c.L > 1 ? stride : (int64_t)rows * cols, box_rows);
}

// T = s F In of all rows (two launches, or one for few rows); `first`: nothing of the call was launched before
int launch_project(const AdapterCall& c, const void* In, int K, const void* F, int64_t strideF, bool f_mn, float* T, bool want_T, int out_width, bf16* P,
                   bool first, PrepParams* prep, int* status) {
  const int sms = sm_count();
  if (sms <= 0) return AB_ERR_CUDA;
  ProjParams p;
  std::memset(&p, 0, sizeof(p));
  const int rp = pad16(c.r);
  p.In = static_cast<const bf16*>(In); p.N = c.N; p.K = K; p.F = static_cast<const bf16*>(F); p.strideF = strideF; p.f_mn = f_mn ? 1 : 0;
  p.scale = c.scale; p.ids = c.ids; p.T = T; p.P = P; p.r = c.r; p.rp = rp; p.L = c.L; p.first = first ? 1 : 0; p.status = status;
  p.want_T = want_T || few_rows(c.N, out_width) ? 1 : 0;
  p.all_rows = c.N <= 64 ? 1 : 0;
  p.tile_rows = c.N > 1024 ? 128 : 64;
  const int64_t tiles = (c.N + p.tile_rows - 1) / p.tile_rows;
  // about 600 CTAs for the rows that go one by one
  p.unit = 1;
  while (p.unit < p.tile_rows && tiles * p.tile_rows / p.unit > 600) p.unit *= 2;
  const int64_t units = (c.N + p.unit - 1) / p.unit;
  if (p.all_rows) {
    const int ky = f_mn ? 1 : (rp + kRowsThreads / 32 - 1) / (kRowsThreads / 32);
    AB_CUDA_OK(beside_large(rows_kernel));
    return launch_after(rows_kernel, dim3((unsigned)units, (unsigned)ky), (unsigned)kRowsThreads, 0, 1, c.st, p);
  }
  const int cols = rp < 128 ? rp : 128;
  p.nk = (K + 63) / 64;
  p.in_bytes = p.tile_rows * 128;
  p.f_bytes = f_mn ? (cols + 63) / 64 * 8192 : cols * 128;
  p.csize = 8;
  while (p.csize > 1 && (tiles * p.csize > 2 * sms || 2 * p.csize > p.nk)) p.csize >>= 1;
  // Never more CTAs an SM than TMEM has columns for (three of 128, two of 256): one that waited for columns would hold up its cluster, whose
  // others hold theirs.  Up to three CTAs an SM, and no more room than for as many as there are: CTAs fill an SM before they go to the next.  The ring takes the
  // parts at the end.
  const int64_t each = (tiles * p.csize * ((rp + 127) / 128) + (c.N <= 2048 ? units : 0) + sms - 1) / sms;
  // room for the factors of two adapters at once where that leaves as many CTAs their place
  const int least = f_mn && each <= 2 ? 16384 : 8192, room = p.f_bytes > least ? p.f_bytes : least;
  p.q_max = room / p.f_bytes < 128 / cols ? room / p.f_bytes : 128 / cols;       // two accumulators in half of the columns: two CTAs an SM
  if (p.q_max > kMaxAd) p.q_max = kMaxAd;
  p.slot_bytes = p.in_bytes + room;
  if (p.slot_bytes < 16384) p.slot_bytes = 16384;          // an MMA reads 128 rows of In, loaded or not
  const int parts = p.tile_rows * (cols + 4) * 4, budget = each <= 1 ? 120 * 1024 : each == 2 || cols > 64 ? 96 * 1024 : 72 * 1024;
  p.ns = budget / p.slot_bytes < 3 ? 3 : budget / p.slot_bytes < kMaxStages ? budget / p.slot_bytes : kMaxStages;
  if (p.ns * p.slot_bytes < parts) p.ns = (parts + p.slot_bytes - 1) / p.slot_bytes;
  p.tmem_cols = 2 * pow2_cols(p.q_max * cols);
  CUtensorMap tmIn, tmF;
  AB_TRY(make_tensor_map_2d(&tmIn, In, false, (uint64_t)c.N, K, K, 64, p.tile_rows));
  AB_TRY(stack_map(&tmF, c, F, f_mn ? K : c.r, f_mn ? c.r : K, strideF, f_mn ? 64 : cols));
  p.tile_ctas = (int)(tiles * p.csize);
  if (prep && prep->ctas > 0) {             // taken along
    p.prep = *prep;
    p.cut = prep->ctas > c.L ? 1 : 0;
    p.prep.ctas = c.L;
    prep->ctas = 0;
  }
  p.prep_ctas = (p.prep.ctas + p.csize - 1) / p.csize * p.csize;
  const int64_t ctas = p.prep_ctas + tiles * p.csize + (units + p.csize - 1) / p.csize * p.csize;
  if (ctas > 0x7fffffffll) return AB_ERR_UNSUPPORTED;
  size_t smem = 1024 + (size_t)p.ns * p.slot_bytes + sizeof(ProjBars);
  if (smem < (size_t)budget) smem = budget;
  const dim3 grid((unsigned)ctas, (unsigned)((rp + 127) / 128));
  if (cols <= 64) {
    AB_CUDA_OK(allow_smem(project_tc_kernel<4>));
    return launch_after(project_tc_kernel<4>, grid, (unsigned)kProjTcThreads, smem, p.csize, c.st, tmIn, tmF, p);
  }
  AB_CUDA_OK(allow_smem(project_tc_kernel<8>));
  return launch_after(project_tc_kernel<8>, grid, (unsigned)kProjTcThreads, smem, p.csize, c.st, tmIn, tmF, p);
}

// CTAs by themselves or in pairs, and the rows of a tile: cycles of the busiest SM, a slab's operands arriving at 64 bytes a cycle or its
// MMAs, whichever is longer
struct WideForm { int bn; bool pair; };
WideForm wide_form(int64_t N, int P, int K, int sms) {
  const int nk = (K + 63) / 64;
  double best = 1e30;
  WideForm f = {256, false};
  for (int two = 0; two < 2; ++two)
    for (int bn = 32 << two; bn <= 256; bn *= 2) {
      const int64_t tiles = (int64_t)((P + (128 << two) - 1) / (128 << two)) * ((N + bn - 1) / bn);
      const double mma = bn <= 64 ? 300.0 : bn <= 128 ? 330.0 : 560.0, arrive = 2.0 * (128 + (bn >> two));
      const double t = (double)((tiles + (sms >> two) - 1) / (sms >> two)) * (nk + 2) * (arrive > mma ? arrive : mma) + (two ? 4500.0 : 3000.0);
      if (t < best) { best = t; f.bn = bn; f.pair = two != 0; }
    }
  return f;
}

// Out = In W^T + T G^T; mn as in OutParams
int launch_out(const AdapterCall& c, const void* In, int K, bool mn, const void* G, int64_t strideG, void* Out, int P, const float* T, const bf16* Tp,
               int* status) {
  const int sms = sm_count();
  if (sms <= 0) return AB_ERR_CUDA;
  OutParams p;
  std::memset(&p, 0, sizeof(p));
  const int rp = pad16(c.r);
  p.N = c.N; p.P = P; p.K = K; p.nk = (K + 63) / 64; p.r = c.r; p.rp = rp; p.L = c.L; p.mn = mn ? 1 : 0; p.ids = c.ids; p.T = T; p.Tp = Tp;
  p.G = static_cast<const bf16*>(G); p.strideG = strideG; p.Out = static_cast<bf16*>(Out); p.status = status;
  p.nft = (P + 127) / 128;
  CUtensorMap tmW, tmIn, tmG, tmT, tmOut;
  if (mn) AB_TRY(make_tensor_map_2d(&tmW, c.W, false, K, P, P, 64, 64));
  else AB_TRY(make_tensor_map_2d(&tmW, c.W, false, P, K, K, 64, 128));
  if (few_rows(c.N, P)) {
    // As many CTAs as there are SMs, by parts of the reduction, and where that is short by fewer rows a tile (127 rows of 25 adapters, rank
    // 128, 160 x 232: with 64 rows a CTA 13 pieces of G came one after the other)
    p.bn = c.N <= 64 ? (int)((c.N + 15) / 16 * 16) : 64;
    p.csize = 8;
    while (p.csize > 1 && 2 * p.csize > p.nk) p.csize >>= 1;
    while (p.bn % 32 == 0 && p.nft * ((c.N + p.bn / 2 - 1) / (p.bn / 2)) * p.csize <= sms) p.bn /= 2;
    const int64_t tt = (c.N + p.bn - 1) / p.bn;
    while (p.csize > 1 && (p.nft * tt * p.csize > sms || 2 * p.csize > p.nk)) p.csize >>= 1;
    p.share = ((p.bn + p.csize - 1) / p.csize + 3) / 4 * 4;
    p.slot_bytes = kABytes + p.bn * 128;
    // Up to 96 KB for G where a batch of rows with an adapter each then fits, else 48 KB; with 64 rows of rank 256 in one CTA's hands
    // there are 146 KB beside the ring
    const size_t piece = (size_t)256 * c.r;
    p.g_slots = piece * kBatch <= 98304 ? kBatch : (int)(49152 / piece);
    if (p.g_slots < 1) p.g_slots = 1;
    if (p.g_slots > p.share) p.g_slots = p.share;
    const size_t rest = p.g_slots * piece + (size_t)kBatch * c.r * 4 + (size_t)p.share * 512 + (size_t)p.csize * 128 * (p.share + 4) * 4 + sizeof(FewBars);
    p.ns = (int)((kMaxSmem - 2048 - rest) / p.slot_bytes);
    if (p.ns > kMaxStages) p.ns = kMaxStages;
    p.tmem_cols = pow2_cols(p.bn);
    AB_TRY(make_tensor_map_2d(&tmIn, In, false, (uint64_t)c.N, K, K, 64, p.bn));
    AB_CUDA_OK(allow_smem(few_kernel));
    return launch_after(few_kernel, dim3((unsigned)(p.nft * p.csize), (unsigned)tt), (unsigned)kWideThreads,
                        1024 + (size_t)p.ns * p.slot_bytes + rest, p.csize, c.st, tmW, tmIn, p);
  }
  const WideForm f = wide_form(c.N, P, K, sms);
  const bool pair = f.pair;
  p.bn = f.bn;
  const int ctas = pair ? 2 : 1;
  p.nft = (P + 128 * ctas - 1) / (128 * ctas);
  const int64_t tiles = (int64_t)p.nft * ((c.N + p.bn - 1) / p.bn);
  if (tiles > 0x7fffffffll) return AB_ERR_UNSUPPORTED;
  p.ntiles = (int)tiles;
  p.slot_bytes = kABytes + p.bn / ctas * 128;
  const int rest = 1024 + kEpiWarps * kEpiBytes + (int)sizeof(WideBars);
  p.ns = (kMaxSmem - rest) / p.slot_bytes < kMaxStages ? (kMaxSmem - rest) / p.slot_bytes : kMaxStages;
  p.tmem_cols = 2 * pow2_cols(p.bn);
  AB_TRY(make_tensor_map_2d(&tmIn, In, false, (uint64_t)c.N, K, K, 64, p.bn / ctas));
  AB_TRY(make_tensor_map_2d(&tmT, Tp, false, (uint64_t)c.N, 3 * rp, 3 * rp, 64, p.bn / ctas));
  AB_TRY(stack_map(&tmG, c, G, mn ? c.r : P, mn ? P : c.r, strideG, mn ? 64 : 128));
  AB_TRY(make_tensor_map_sw64(&tmOut, Out, (uint64_t)c.N, P, 32, 32));
  const size_t smem = (size_t)p.ns * p.slot_bytes + rest;
  if (pair) {
    AB_CUDA_OK(allow_smem(wide_kernel<true>));
    const int pairs = p.ntiles < sms / 2 ? p.ntiles : sms / 2;
    return launch_after(wide_kernel<true>, (unsigned)(2 * pairs), (unsigned)kWideAll, smem, 2, c.st, tmW, tmIn, tmG, tmT, tmOut, p);
  }
  AB_CUDA_OK(allow_smem(wide_kernel<false>));
  return launch_after(wide_kernel<false>, (unsigned)(p.ntiles < sms ? p.ntiles : sms), (unsigned)kWideAll, smem, 1, c.st, tmW, tmIn, tmG, tmT,
                      tmOut, p);
}

// Slices of an adapter's rows, so that there are CTAs for every SM where adapters and tiles are few
int grad_slices(int64_t N, int m, int n, int r, int L) {
  const int sms = sm_count() > 0 ? sm_count() : 148;
  const int64_t items = (int64_t)L * ((m + 127) / 128 + (n + 127) / 128) * (pad16(r) > 128 ? 2 : 1);
  const int64_t slabs = (N + 63) / 64 / L;
  int64_t s = sms / items;
  if (s > slabs / 8) s = slabs / 8;
  return (int)(s < 1 ? 1 : s > 16 ? 16 : s);
}

struct TcWs { int* status; float *T, *U; bf16 *TP, *UP; uint4* list; int* count; float *pA, *pB; int slices, nslab; size_t bytes; };
TcWs tc_ws(void* ws, int64_t N, int m, int n, int r, int L) {
  Arena ar(ws, 0);
  TcWs w;
  const int rp = pad16(r);
  w.status = ar.take_n<int>(64);
  w.T = ar.take_n<float>((size_t)N * r);
  w.U = ar.take_n<float>((size_t)N * r);
  w.TP = ar.take_n<bf16>((size_t)N * 3 * rp);
  w.UP = ar.take_n<bf16>((size_t)N * 3 * rp);
  w.nslab = (int)((N + 63) / 64);
  w.list = adapter_tc_lists_ok(N, L) ? ar.take_n<uint4>((size_t)L * w.nslab) : nullptr;
  w.count = ar.take_n<int>((size_t)L);
  w.slices = grad_slices(N, m, n, r, L);
  w.pA = w.slices > 1 ? ar.take_n<float>((size_t)w.slices * L * m * r) : nullptr;
  w.pB = w.slices > 1 ? ar.take_n<float>((size_t)w.slices * L * n * r) : nullptr;
  w.bytes = align_up(ar.used, 256);
  return w;
}

int launch_grads(const AdapterCall& c, const void* dY, float* dA, float* dB, const TcWs& w, bool check) {
  GradParams p;
  std::memset(&p, 0, sizeof(p));
  const int rp = pad16(c.r);
  p.N = c.N; p.r = c.r; p.rp = rp; p.L = c.L; p.nslab = w.nslab; p.slices = w.slices; p.ids = c.ids; p.list = w.list; p.count = w.count;
  p.status = w.status; p.check = check ? 1 : 0;
  p.halves = rp > 128 ? 2 : 1;
  p.stacked = 3 * rp <= 256 ? 1 : 0;
  p.nb = p.stacked ? (3 * rp + 63) / 64 : ((rp < 128 ? rp : 128) + 63) / 64;
  p.slot_bytes = kABytes + p.nb * 8192;
  const int acc = pow2_cols(p.stacked ? 3 * rp : rp < 128 ? rp : 128);
  // Two CTAs an SM where two accumulators leave room for another two.  (r = 64, one accumulator each and two CTAs: 58 us for the ViT groups
  // against 45.)
  const int ring = acc <= 128 ? 108 * 1024 : 200 * 1024;
  p.tmem_cols = 2 * acc;
  p.ns = ring / p.slot_bytes < kMaxStages ? ring / p.slot_bytes : kMaxStages;
  CUtensorMap act[2], small[2];
  int nj = 0;
  if (dA) {
    AB_TRY(make_tensor_map_2d(&act[nj], dY, false, (uint64_t)c.N, c.m, c.m, 64, 64));
    AB_TRY(make_tensor_map_2d(&small[nj], w.TP, false, (uint64_t)c.N, 3 * rp, 3 * rp, 64, 64));
    p.job[nj] = GradJob{c.m, (c.m + 127) / 128, w.slices > 1 ? w.pA : dA, (int64_t)c.m * c.r, c.r, 1, (int64_t)c.L * c.m * c.r};
    ++nj;
  }
  if (dB) {
    AB_TRY(make_tensor_map_2d(&act[nj], c.x, false, (uint64_t)c.N, c.n, c.n, 64, 64));
    AB_TRY(make_tensor_map_2d(&small[nj], w.UP, false, (uint64_t)c.N, 3 * rp, 3 * rp, 64, 64));
    p.job[nj] = GradJob{c.n, (c.n + 127) / 128, w.slices > 1 ? w.pB : dB, (int64_t)c.r * c.n, 1, c.n, (int64_t)c.L * c.r * c.n};
    ++nj;
  }
  if (nj == 1) { act[1] = act[0]; small[1] = small[0]; }
  const int64_t grid = (int64_t)c.L * (p.job[0].tiles + p.job[1].tiles) * p.halves * p.slices;
  if (grid > 0x7fffffffll) return AB_ERR_UNSUPPORTED;
  const size_t smem = 1024 + (size_t)p.ns * p.slot_bytes + sizeof(GradBars);
  if (rp <= 64) {
    AB_CUDA_OK(allow_smem(adapter_grad_tc_kernel<4>));
    AB_TRY(launch_after(adapter_grad_tc_kernel<4>, (unsigned)grid, (unsigned)kWideThreads, smem, 1, c.st, act[0], small[0], act[1], small[1], p));
  } else {
    AB_CUDA_OK(allow_smem(adapter_grad_tc_kernel<8>));
    AB_TRY(launch_after(adapter_grad_tc_kernel<8>, (unsigned)grid, (unsigned)kWideThreads, smem, 1, c.st, act[0], small[0], act[1], small[1], p));
  }
  if (w.slices > 1)
    return adapter_add_slices(w.pA, dA, (int64_t)c.L * c.m * c.r, w.pB, dB, (int64_t)c.L * c.n * c.r, w.slices, c.st);
  return AB_OK;
}

}  // namespace

// The gradients' slab lists take 16 bytes an adapter and 64 rows: up to 256 MB.
bool adapter_tc_lists_ok(int64_t N, int L) { return (N + 63) / 64 * L <= ((int64_t)1 << 24); }

bool adapter_tc_shape_ok(int64_t N, int m, int n, int r, int L, int dt) {
  return dt == AB_BF16 && m % 8 == 0 && n % 8 == 0 && r % 8 == 0 && r <= 256 && N <= ((int64_t)1 << 30) && L < (1 << 30);
}

bool adapter_tc_supported(const AdapterCall& c, const void* dY, const void* out, const float* T, const float* dA, const float* dB) {
  if (!adapter_tc_shape_ok(c.N, c.m, c.n, c.r, c.L, c.dt)) return false;
  if (c.L > 1 && (c.strideA % 8 != 0 || c.strideB % 8 != 0)) return false;
  return aligned(c.x, 16) && aligned(c.W, 16) && aligned(c.A, 16) && aligned(c.B, 16) && aligned(dY, 16) && aligned(out, 16) && aligned(T, 16) &&
         aligned(dA, 16) && aligned(dB, 16) && tc_device_ok();
}

// For tests: which kernel forms N x P results over a reduction of K. 0: the one for few rows; else the rows of a tile, + 1 where CTAs go in pairs.
int adapter_tc_form(int64_t N, int P, int K) {
  if (few_rows(N, P)) return 0;
  const WideForm f = wide_form(N, P, K, sm_count() > 0 ? sm_count() : 148);
  return f.bn + (f.pair ? 1 : 0);
}

size_t adapter_tc_ws(int64_t N, int m, int n, int r, int L) { return tc_ws(nullptr, N, m, n, r, L).bytes; }

int adapter_tc_forward(const AdapterCall& c, void* y, float* T_save, void* ws) {
  const TcWs w = tc_ws(ws, c.N, c.m, c.n, c.r, c.L);
  float* T = T_save ? T_save : w.T;
  AB_TRY(launch_project(c, c.x, c.n, c.B, c.strideB, false, T, T_save != nullptr, c.m, w.TP, true, nullptr, w.status));
  return launch_out(c, c.x, c.n, false, c.A, c.strideA, y, c.m, T, w.TP, w.status);
}

int adapter_tc_backward(const AdapterCall& c, const void* dY, const float* T_saved, void* dX, float* dA, float* dB, void* ws) {
  const TcWs w = tc_ws(ws, c.N, c.m, c.n, c.r, c.L);
  bool first = true;
  PrepParams prep = {};
  if (dA || dB) {
    const int64_t values = dA && T_saved ? c.N * (pad16(c.r) / 8) : 0;
    const int64_t blocks = (values + 1023) / 1024;
    prep = PrepParams{w.list, w.count, w.nslab, T_saved, w.TP, c.L + (int)(blocks < 444 ? blocks : 444)};
  }
  if (dX || dB) {
    AB_TRY(launch_project(c, dY, c.m, c.A, c.strideA, true, w.U, false, c.n, w.UP, first, &prep, w.status));
    first = false;
  }
  if (dA && !T_saved) {
    AB_TRY(launch_project(c, c.x, c.n, c.B, c.strideB, false, w.T, false, c.m, w.TP, first, &prep, w.status));
    first = false;
  }
  if (prep.ctas > 0) {                      // no projection took it along
    AB_CUDA_OK(beside_large(prep_kernel));
    AB_TRY(launch_after(prep_kernel, (unsigned)prep.ctas, (unsigned)kPrepThreads, 0, 1, c.st, prep, c.ids, c.N, c.L, c.r, pad16(c.r), first ? 1 : 0,
                        w.status));
  }
  if (dX) AB_TRY(launch_out(c, dY, c.m, true, c.B, c.strideB, dX, c.n, w.U, w.UP, w.status));
  if (dA || dB) AB_TRY(launch_grads(c, dY, dA, dB, w, !dX));
  return AB_OK;
}

}  // namespace ab
