// The second step of attention whose units are cut over CTAs: the parts' states, merged in the order of the positions.
#pragma once
#include <type_traits>

#include "attend.cuh"

namespace stairs {
namespace att {
namespace {

template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if (std::is_same<T, bf16>::value) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float ex2(float x) { return exp2f(x); }

struct Meta { int parts, slot, first, n, qb, h, failed, pad; };   // of the unit that a CTA begins and does not end

// Joins the parts of the unit that CTA blockIdx.x of the kernel above began and did not end: part 0 is where that CTA says,
// the next ones are the first parts of the CTAs behind it.
template <typename T, int ROWS, bool CHECK> __global__ void __launch_bounds__(128) k_attend_join(const __grid_constant__ AttendParams P) {
  __shared__ float sM[ROWS], sInv[ROWS];
  wait_prerequisites();
  const Meta* metas = reinterpret_cast<const Meta*>(P.ws);
  if (CHECK) {
    // a part whose CTA gave up a wait is no part: nothing of the call counts, and every row says so
    int bad = 0;
    for (int i = threadIdx.x; i < gridDim.x; i += 128) bad |= metas[i].failed;
    if (__syncthreads_or(bad)) {
      const long long all = (long long)P.n_rows * P.heads;
      for (long long r = (long long)blockIdx.y * gridDim.x + blockIdx.x; r < all; r += (long long)gridDim.x * gridDim.y) {
        T* dst = reinterpret_cast<T*>(P.o) + (r / P.heads) * P.o_row + (r % P.heads) * P.o_head;
        for (int d = threadIdx.x; d < P.hd; d += 128) dst[d] = from_f32<T>(NAN);
      }
      return;
    }
  }
  const Meta m = metas[blockIdx.x];
  if (m.parts == 0) return;
  const int group = P.heads / P.kv_heads, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const size_t slot = (size_t)ROWS * (P.hd + 2);
  const float* base = reinterpret_cast<const float*>(reinterpret_cast<const unsigned char*>(P.ws) + (size_t)gridDim.x * sizeof(Meta));
  auto part = [&](int p) { return base + (p ? 2 * (blockIdx.x + p) : m.slot) * slot; };
  const int rows = min(ROWS, m.n * group - m.qb * ROWS);
  // this block's rows (grid y)
  const int per = (rows + gridDim.y - 1) / gridDim.y, ra = blockIdx.y * per, rb = min(rows, ra + per);
  for (int r = ra + warp; r < rb; r += 4) {
    float M = -INFINITY, L = 0.f;
    for (int p = lane; p < m.parts; p += 32) {
      const float* s = part(p) + (size_t)ROWS * P.hd;
      const float mp = s[r], lp = s[ROWS + r], n = fmaxf(M, mp);
      if (n != -INFINITY) L = L * ex2(M - n) + lp * ex2(mp - n);
      M = n;
    }
    const float mx = warp_max(M);
    L = warp_sum(M == -INFINITY ? 0.f : L * ex2(M - mx));
    if (lane == 0) { sM[r] = mx; sInv[r] = mx == -INFINITY ? 0.f : 1.f / L; }
  }
  __syncthreads();
  const int q4 = P.hd / 4;
  for (int it = threadIdx.x; it < (rb - ra) * q4; it += 128) {
    const int r = ra + it / q4, c = it % q4 * 4, qi = m.qb * ROWS + r, j = qi / group;
    const float M = sM[r], inv = sInv[r];
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = 0; p < m.parts; ++p) {
      const float* s = part(p);
      const float mp = s[(size_t)ROWS * P.hd + r];
      const float4 v = *reinterpret_cast<const float4*>(s + (size_t)r * P.hd + c);
      const float w = mp == -INFINITY ? 0.f : ex2(mp - M);
      if (w != 0.f) { o.x = fmaf(v.x, w, o.x); o.y = fmaf(v.y, w, o.y); o.z = fmaf(v.z, w, o.z); o.w = fmaf(v.w, w, o.w); }
    }
    T* dst = reinterpret_cast<T*>(P.o) + (m.first + j) * P.o_row + (m.h * group + qi - j * group) * P.o_head + c;
    uint2 u;
    u.x = pack2<T>(o.x * inv, o.y * inv); u.y = pack2<T>(o.z * inv, o.w * inv);
    *reinterpret_cast<uint2*>(dst) = u;
  }
}

template <typename T, int ROWS, bool CHECK = false> int launch_join(const AttendParams& P, int grid, int cut, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid, cut); cfg.blockDim = dim3(128); cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization; at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = 1;
  SCK(cudaLaunchKernelEx(&cfg, k_attend_join<T, ROWS, CHECK>, P));
  return STAIRS_OK;
}

}  // namespace
}  // namespace att
}  // namespace stairs
