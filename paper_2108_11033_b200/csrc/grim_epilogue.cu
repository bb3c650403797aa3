// The gradient of a product's epilogue: dP = dY act'(P) and, per row, the sum of dP (the bias's gradient).
//
// One pass: two arrays in, one out, and the sums stay in registers until a row is done: warps of a row meet in shared memory, blocks
// of a row (a cluster, where rows are few) in distributed shared memory.  The order of the additions is fixed: no atomics, the same
// bits every time.  4096 x 8192: fp32 62 us (62 for its bytes at 6.54 TB/s), memory; bf16 35 us (31) with relu, 37 with silu, 39 to 41
// with gelu, 44 with its tanh form, whose slopes' instructions fill two thirds of the issue slots.
#include <algorithm>

#include "grim_epilogue.cuh"

namespace grim {
namespace {

constexpr int kThreads = 256, kWarps = 8;

struct GradParams {
  const void *dY, *pre;
  void* dP;
  float* dbias;
  int64_t ldy, ldpre, ldp, M, N;
  int act, wpr, cluster;  // warps that share a row in a block, blocks that share a row
};

template <typename S, int V>
struct __align__(sizeof(S) * V) Piece { S e[V]; };

// Columns at .. at + V - 1 of a row.
template <typename S, int V>
__device__ __forceinline__ float grad_piece(const GradParams& p, const Piece<S, V>& dy, const Piece<S, V>& x, S* out) {
  float v[V], d[V], sum = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = widen(x.e[i]);
  act_slopes<V>(p.act, v, d);
  Piece<S, V> o;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    d[i] *= widen(dy.e[i]);
    sum += d[i];
    narrow(d[i], o.e[i]);
  }
  if (out) *reinterpret_cast<Piece<S, V>*>(out) = o;
  return sum;
}

template <typename S>
__global__ void __launch_bounds__(kThreads) epilogue_grad_kernel(const __grid_constant__ GradParams p) {
  constexpr int E = 16 / (int)sizeof(S);
  __shared__ float part[kWarps], block_sum;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % p.wpr;
  const int64_t b = blockIdx.x / (unsigned)p.cluster, row = b * (kWarps / p.wpr) + warp / p.wpr;
  const int rank = (int)(blockIdx.x - (unsigned)b * (unsigned)p.cluster);
  const int t = sub * 32 + lane, T = p.wpr * 32;
  float sum = 0.f;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (row < p.M) {
    const S* dy = static_cast<const S*>(p.dY) + row * p.ldy;
    const S* x = p.pre ? static_cast<const S*>(p.pre) + row * p.ldpre : dy;
    S* o = p.dP ? static_cast<S*>(p.dP) + row * p.ldp : nullptr;
    // this block's columns
    const int64_t share = ((p.N + p.cluster - 1) / p.cluster + E - 1) / E * E;
    const int64_t c0 = min(p.N, rank * share), c1 = min(p.N, c0 + share);
    // 16-byte pieces where the three rows lie alike; the columns in front of the first boundary and behind the last one by one
    const uintptr_t at = reinterpret_cast<uintptr_t>(dy + c0);
    const bool alike = ((reinterpret_cast<uintptr_t>(x + c0) ^ at) & 15) == 0 && (!o || ((reinterpret_cast<uintptr_t>(o + c0) ^ at) & 15) == 0);
    const int64_t head = alike ? min(c1 - c0, (int64_t)((16 - (at & 15)) & 15) / (int64_t)sizeof(S)) : c1 - c0;
    const int64_t v0 = c0 + head, v1 = v0 + (c1 - v0) / E * E;
    auto single = [&](int64_t c) {
      Piece<S, 1> a, bb;
      a.e[0] = dy[c];
      bb.e[0] = x[c];
      sum += grad_piece<S, 1>(p, a, bb, o ? o + c : nullptr);
    };
    for (int64_t c = c0 + t; c < v0; c += T) single(c);
    int64_t c = v0 + (int64_t)t * E;
    const int64_t step = (int64_t)T * E;
    for (; c + step < v1; c += 2 * step) {  // two pieces' loads in flight
      const auto a0 = *reinterpret_cast<const Piece<S, E>*>(dy + c), x0 = *reinterpret_cast<const Piece<S, E>*>(x + c);
      const auto a1 = *reinterpret_cast<const Piece<S, E>*>(dy + c + step), x1 = *reinterpret_cast<const Piece<S, E>*>(x + c + step);
      sum += grad_piece<S, E>(p, a0, x0, o ? o + c : nullptr);
      sum += grad_piece<S, E>(p, a1, x1, o ? o + c + step : nullptr);
    }
    if (c < v1) {
      const auto a0 = *reinterpret_cast<const Piece<S, E>*>(dy + c), x0 = *reinterpret_cast<const Piece<S, E>*>(x + c);
      sum += grad_piece<S, E>(p, a0, x0, o ? o + c : nullptr);
    }
    for (int64_t c2 = v1 + t; c2 < c1; c2 += T) single(c2);
  }
  if (!p.dbias) return;  // (the same for every block)
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) part[warp] = sum;
  __syncthreads();
  const bool leader = lane == 0 && sub == 0;
  if (leader) {
    sum = 0.f;
    for (int i = 0; i < p.wpr; ++i) sum += part[warp + i];
  }
  if (p.cluster > 1) {  // (a block has one row then)
    if (leader) block_sum = sum;
    __syncwarp();
    ptx::cluster_sync_all();
    if (leader && rank == 0) {
      sum = 0.f;
      for (int i = 0; i < p.cluster; ++i) {
        uint32_t from;
        float v;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(ptx::smem_u32(&block_sum)), "r"(i));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(from) : "memory");
        sum += v;
      }
    }
    __syncwarp();
    ptx::cluster_sync_all();  // no block leaves while its sum may still be read
  }
  if (leader && rank == 0 && row < p.M) p.dbias[row] = sum;
}

}  // namespace
}  // namespace grim

using namespace grim;

extern "C" grim_status_t grim_epilogue_grad(const grim_mat_t* dY, const grim_mat_t* pre, grim_act_t act, grim_mat_t* dP, float* dbias_dev,
                                            grim_stream_t stream) {
  if (!dY || !dY->ptr || (!dP && !dbias_dev) || (dP && !dP->ptr) || (pre && !pre->ptr)) return GRIM_ERR_INVALID_ARG;
  for (const grim_mat_t* m : {dY, pre, static_cast<const grim_mat_t*>(dP)})
    if (m && reinterpret_cast<uintptr_t>(m->ptr) % (m->dtype == GRIM_F32 ? 4 : 2) != 0) return GRIM_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(dbias_dev) % 4 != 0) return GRIM_ERR_INVALID_ARG;
  if ((int)act < GRIM_ACT_NONE || (int)act > GRIM_ACT_TANH || (!pre && act != GRIM_ACT_NONE)) return GRIM_ERR_INVALID_ARG;
  if (dY->rows <= 0 || dY->cols <= 0 || dY->ld < dY->cols) return GRIM_ERR_SHAPE;
  for (const grim_mat_t* m : {pre, static_cast<const grim_mat_t*>(dP)})
    if (m && (m->rows != dY->rows || m->cols != dY->cols || m->ld < m->cols)) return GRIM_ERR_SHAPE;
  if (dY->dtype != GRIM_F32 && dY->dtype != GRIM_BF16) return GRIM_ERR_DTYPE;
  if ((pre && pre->dtype != dY->dtype) || (dP && dP->dtype != dY->dtype)) return GRIM_ERR_DTYPE;
  GradParams p{};
  p.dY = dY->ptr; p.ldy = dY->ld; p.M = dY->rows; p.N = dY->cols; p.act = act; p.dbias = dbias_dev;
  if (pre) { p.pre = pre->ptr; p.ldpre = pre->ld; }
  if (dP) { p.dP = dP->ptr; p.ldp = dP->ld; }
  const int per_warp = 32 * (dY->dtype == GRIM_F32 ? 4 : 8);
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return GRIM_ERR_CUDA; }
  const int64_t sms = sm_count(dev);
  p.wpr = p.cluster = 1;
  // Warps: for bf16, bound by instructions, no more than 48 to an SM (4096 x 8192, gelu: 39.5 us, with eight warps to a row 45.5); for
  // fp32, bound by memory, more (4096 x 8192: 62 against 68.5).  Eight vectors for each lane where there are rows enough (8192 x 1024,
  // bf16: 10.9 against 18.8).
  const int64_t most = sms * (dY->dtype == GRIM_F32 ? 200 : 48);
  while (p.wpr < kWarps && p.N > (int64_t)p.wpr * per_warp && p.M * p.wpr < most &&
         (p.N >= (int64_t)p.wpr * per_warp * 16 || p.M * p.wpr < sms * 16))
    p.wpr *= 2;
  while (p.wpr == kWarps && p.cluster < 8 && p.M * p.cluster < sms * 4 && p.N > (int64_t)p.cluster * kWarps * per_warp) p.cluster *= 2;
  const int64_t per_block = kWarps / p.wpr, blocks = (p.M + per_block - 1) / per_block * p.cluster;
  if (blocks > 0x7fffffff) return GRIM_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)p.cluster, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = p.cluster > 1 ? 2 : 1;
  const cudaError_t e = dY->dtype == GRIM_F32 ? cudaLaunchKernelEx(&cfg, epilogue_grad_kernel<float>, p) : cudaLaunchKernelEx(&cfg, epilogue_grad_kernel<unsigned short>, p);
  count_launch();
  if (e != cudaSuccess) { cudaGetLastError(); return GRIM_ERR_CUDA; }
  return GRIM_OK;
}
