// Sampled acceptance on caller-held scores (stairs_sample_static): temperature, min-p, top-k and top-p, a token drawn by a given
// random number, and the stairs walk over the drawn tokens.
//
// A row's filters keep the first n of its tokens in the order (score down, index up), so each filter is a threshold in that order, and
// the drawn token is where a running sum passes u times the whole.  Weights exp((x - max) / temperature) are computed in 64 bits
// and held as whole numbers of 2^-bits: their sums are exact whatever the order of the additions, so neither atomics nor the split of a row over threads
// changes a result, and the token is the one that the formula in 64 bits gives (32-bit weights move a boundary between two of
// 32000 tokens by about 1e-7 of the sum, with 3e-5 between them: one row in some hundreds would draw another token).
#include <algorithm>
#include <type_traits>

#include "static_ops.cuh"

namespace stairs {
namespace {

typedef unsigned long long u64;

struct SampleParams {
  const void* logits; const float* u; const int* draft; int* tokens; int* accept;
  long long ld;
  int vocab, n_req, n_rows, k_max, bits;      // bits: the largest weight is 2^bits
  int off[STAIRS_SAMPLE_MAX_REQ], k[STAIRS_SAMPLE_MAX_REQ];
  stairs_sampling s[STAIRS_SAMPLE_MAX_REQ];
};

constexpr int NB = 2048, SMALL = 256;        // bins of a histogram; most elements of a bin that are ranked one against another

// (larger score, then lower index) as one number
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o); }
__device__ __forceinline__ u64 full_key(uint32_t o, int i) { return ((u64)o << 32) | (uint32_t)~i; }

// 2^bits exp((x - m) / T), rounded to a whole number.  exp by a table of 2^(j/64) and a polynomial of the rest (P. Tang, "Table-driven
// implementation of the exponential function in IEEE floating-point arithmetic", 1989): |r| <= ln 2 / 128, so its fourth-degree
// Taylor polynomial is off by at most 4e-14.
struct Weigher {
  double m, inv_t, min_w;
  float mf, cut;
  const double* tab;                          // 2^(bits + j/64)
  __device__ __forceinline__ bool eligible(float x) const { return x == mf || mf - x <= cut; }   // (never NaN or -infinity; anything else weighs 0)
  __device__ __forceinline__ u64 operator()(float x) const {
    const double t = x == mf ? 0.0 : ((double)x - m) * inv_t;
    constexpr double MAGIC = 6755399441055744.0, LN2 = 0.69314718055994530942;   // 1.5 * 2^52: adding it rounds to a whole number
    const double z = fma(t, 64.0 / LN2, MAGIC);
    const int n = __double2loint(z);
    const double r = fma(z - MAGIC, -LN2 / 64.0, t);
    const double p = fma(fma(fma(fma(r, 1.0 / 24.0, 1.0 / 6.0), r, 0.5), r, 1.0), r, 1.0);
    const double v = p * tab[n & 63];
    const double w = __hiloint2double(__double2hiint(v) + ((n >> 6) << 20), __double2loint(v));
    if (w < min_w) return 0;
    return (u64)(__double_as_longlong(w + 4503599627370496.0) - 0x4330000000000000ll);   // + 2^52: the low bits are the whole number
  }
};

template <int NT> struct BlockOps {
  static constexpr int NW = NT / 32;
  // inclusive running sum over the block's threads, and the sum of all; `red` holds NW + 1 numbers
  static __device__ __forceinline__ u64 scan(u64 v, u64* red, u64& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 x = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += x;
    }
    __syncthreads();
    if (lane == 31) red[warp] = v;
    __syncthreads();
    u64 before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) { const u64 x = red[w]; all += x; if (w < warp) before += x; }
    total = all;
    return v + before;
  }
};

template <typename T, int NT, bool STAGED>
__global__ void __launch_bounds__(NT, STAGED && sizeof(T) == 4 ? 1 : 2) k_sample(const __grid_constant__ SampleParams P) {
  extern __shared__ __align__(16) unsigned char sp_sm[];
  u64* hist = reinterpret_cast<u64*>(sp_sm);
  u64* list = hist + NB;
  u64* list_w = list + SMALL;
  double* tab = reinterpret_cast<double*>(list_w + SMALL);
  T* xs = reinterpret_cast<T*>(tab + 64);
  __shared__ u64 red[NT / 32 + 1];
  __shared__ u64 s_pick[4];
  __shared__ int s_int[4];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.x, V = P.vocab;
  constexpr int NW = NT / 32;
  launch_dependents();
  wait_prerequisites();
  if (tid < 64) tab[tid] = exp2((double)P.bits + tid / 64.0);
  int lo = 0, hi = P.n_req - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (P.off[mid] <= row) lo = mid; else hi = mid - 1;
  }
  const int req = lo, r_in = row - P.off[req];
  const stairs_sampling S = P.s[req];
  const T* logits = reinterpret_cast<const T*>(P.logits) + (size_t)row * P.ld;
  auto clean = [](float x) { return x == x ? x + 0.f : -INFINITY; };   // (-0 counts as 0)
  auto get = [&](int i) { return clean(to_f32(STAGED ? xs[i] : logits[i])); };

  // the row's extent: largest and smallest score above -infinity
  float mx = -INFINITY, mn = INFINITY;
  {
    constexpr int VN = 16 / sizeof(T);
    const int head = min(V, (int)(((16 - (reinterpret_cast<uintptr_t>(logits) & 15)) & 15) / sizeof(T)));   // elements before the first whole vector
    const int vecs = (V - head) / VN;
    auto look = [&](T raw, int i) {
      if (STAGED) xs[i] = raw;
      const float x = clean(to_f32(raw));
      mx = fmaxf(mx, x);
      mn = fminf(mn, x == -INFINITY ? INFINITY : x);
    };
    constexpr int UN = 4;
    for (int v0 = tid; v0 < vecs; v0 += NT * UN) {
      uint4 q[UN];
#pragma unroll
      for (int j = 0; j < UN; ++j) if (v0 + j * NT < vecs) q[j] = __ldg(reinterpret_cast<const uint4*>(logits + head) + v0 + j * NT);
#pragma unroll
      for (int j = 0; j < UN; ++j)
        if (v0 + j * NT < vecs) {
          const T* e = reinterpret_cast<const T*>(&q[j]);
#pragma unroll
          for (int c = 0; c < VN; ++c) look(e[c], head + (v0 + j * NT) * VN + c);
        }
    }
    for (int i = tid; i < head; i += NT) look(logits[i], i);
    for (int i = head + vecs * VN + tid; i < V; i += NT) look(logits[i], i);
  }
  {
    const uint32_t a = __reduce_max_sync(0xffffffffu, ordered(mx)), b = __reduce_min_sync(0xffffffffu, ordered(mn));
    if (lane == 0) red[warp] = ((u64)a << 32) | b;
    __syncthreads();
    uint32_t A = 0u, B = 0xffffffffu;
#pragma unroll
    for (int w = 0; w < NW; ++w) { A = max(A, (uint32_t)(red[w] >> 32)); B = min(B, (uint32_t)red[w]); }
    mx = unordered(A); mn = unordered(B);
    __syncthreads();
  }
  int token = -1;
  if (mx == -INFINITY) {
    // nothing to draw
  } else if (S.temperature == 0.f) {
    int best = 0x7fffffff;
    for (int i = tid; i < V; i += NT) if (get(i) == mx) { best = i; break; }
    best = __reduce_min_sync(0xffffffffu, best);
    if (lane == 0) red[warp] = (u64)best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) best = min(best, (int)red[w]);
    token = best;
  } else {
    Weigher W;
    W.mf = mx; W.m = (double)mx; W.inv_t = 1.0 / (double)S.temperature; W.tab = tab;
    W.min_w = S.min_p > 0.f ? ldexp((double)S.min_p, P.bits) : 0.0;
    // what may weigh anything: scores not much further than this below the largest
    const float nats = S.min_p > 0.f ? fminf(-logf(S.min_p) + 1e-3f, (P.bits + 1.5f) * 0.6931472f) : (P.bits + 1.5f) * 0.6931472f;
    W.cut = nats * S.temperature * 1.00001f;
    u64 thr = 0;                               // kept: keys from here up
    const int seg = ((V + NW - 1) / NW + 31) / 32 * 32;

    // Lowers the list of kept keys to the first ones whose count (mass: weight) reaches a bound: a histogram of the scores, its bin where the bound is
    // passed, then that bin's elements, finer again while they are many.
    auto find = [&](const bool mass) {
      const float range = fminf(mx - mn, W.cut), fscale = range > 1e-30f ? (float)NB / range : 0.f;
      uint32_t kmin = 0u, kmax = 0xffffffffu;   // ordered scores of the current interval
      int shift = -1;                           // < 0: bins are linear in the score
      if (fscale == 0.f) { kmin = ordered(mn); kmax = ordered(mx); shift = max(0, 32 - __clz(kmax - kmin) - 11); }
      u64 base = 0;
      double target = (double)S.top_k;
      for (bool top = true;; top = false) {
        auto bin_of = [&](float x, uint32_t o) { return shift < 0 ? (x == mx ? 0 : min(NB - 1, (int)((mx - x) * fscale))) : (int)((kmax - o) >> shift); };
        for (int b = tid; b < NB; b += NT) hist[b] = 0;
        __syncthreads();
        for (int i0 = warp * seg; i0 < min(V, (warp + 1) * seg); i0 += 32) {
          const int i = i0 + lane;
          const float x = i < V ? get(i) : -INFINITY;
          const uint32_t o = ordered(x);
          if (x > -INFINITY && W.eligible(x) && o >= kmin && o <= kmax && full_key(o, i) >= thr) {
            const u64 w = mass ? W(x) : 1;
            if (w) atomicAdd(hist + bin_of(x, o), w);
          }
        }
        __syncthreads();
        u64 mine[NB / NT], sum = 0, total;
#pragma unroll
        for (int j = 0; j < NB / NT; ++j) { mine[j] = hist[tid * (NB / NT) + j]; sum += mine[j]; }
        u64 incl = BlockOps<NT>::scan(sum, red, total);
        if (top && mass) target = (double)S.top_p * (double)total;
        if (top && !mass && (double)total <= target) return;   // no more than that: all stay
        u64 c = incl - sum;
#pragma unroll
        for (int j = 0; j < NB / NT; ++j) {
          if ((double)(base + c) < target && !((double)(base + c + mine[j]) < target)) { s_int[0] = tid * (NB / NT) + j; s_pick[0] = c; }
          c += mine[j];
        }
        if (tid == 0) { s_int[1] = 0; s_int[2] = -1; s_int[3] = 0; }   // elements of the bin; smallest and largest score (as unsigned)
        __syncthreads();
        const int bin = s_int[0];
        base += s_pick[0];
        uint32_t omin = 0xffffffffu, omax = 0u;
        for (int i0 = warp * seg; i0 < min(V, (warp + 1) * seg); i0 += 32) {
          const int i = i0 + lane;
          const float x = i < V ? get(i) : -INFINITY;
          const uint32_t o = ordered(x);
          if (x > -INFINITY && W.eligible(x) && o >= kmin && o <= kmax && full_key(o, i) >= thr && bin_of(x, o) == bin) {
            const int at = atomicAdd(s_int + 1, 1);
            if (at < SMALL) list[at] = full_key(o, i);
            omin = min(omin, o); omax = max(omax, o);
          }
        }
        omin = __reduce_min_sync(0xffffffffu, omin); omax = __reduce_max_sync(0xffffffffu, omax);
        if (lane == 0 && omin <= omax) { atomicMin(reinterpret_cast<unsigned*>(s_int + 2), omin); atomicMax(reinterpret_cast<unsigned*>(s_int + 3), omax); }
        __syncthreads();
        const int n = s_int[1];
        kmin = (uint32_t)s_int[2]; kmax = (uint32_t)s_int[3];
        if (n <= SMALL) {
          if (tid < n) list_w[tid] = mass ? W(unordered((uint32_t)(list[tid] >> 32))) : 1;
          if (tid == 0) s_pick[1] = ~0ull;
          __syncthreads();
          if (tid < n) {
            const u64 key = list[tid];
            u64 above = 0;
            for (int j = 0; j < n; ++j) above += list[j] > key ? list_w[j] : 0;
            if ((double)(base + above) < target) atomicMin(s_pick + 1, key);
          }
          __syncthreads();
          thr = s_pick[1];
          __syncthreads();
          return;
        }
        if (kmin == kmax) {
          // equal scores: the first of them by index, as many as the bound needs
          const u64 w = mass ? W(unordered(kmin)) : 1;
          u64 keep = w ? (u64)((target - (double)base) / (double)w) : 0;
          if (keep > 0) --keep;
          while ((double)(base + keep * w) < target && keep < (u64)n) ++keep;   // (the division may be off by one)
          if (keep == 0) keep = 1;
          u64 cnt = 0;
          for (int i0 = warp * seg; i0 < min(V, (warp + 1) * seg); i0 += 32) {
            const int i = i0 + lane;
            cnt += __popc(__ballot_sync(0xffffffffu, i < V && ordered(get(i)) == kmin));
          }
          __syncthreads();
          if (lane == 0) red[warp] = cnt;
          __syncthreads();
          u64 before = 0;
          for (int w2 = 0; w2 < warp; ++w2) before += red[w2];
          if (before < keep && keep <= before + cnt)
            for (int i0 = warp * seg; i0 < min(V, (warp + 1) * seg); i0 += 32) {
              const int i = i0 + lane;
              const unsigned tie = __ballot_sync(0xffffffffu, i < V && ordered(get(i)) == kmin);
              if (before < keep && keep <= before + __popc(tie)) {
                if (((tie >> lane) & 1u) && before + __popc(tie & ((2u << lane) - 1u)) == keep) s_pick[1] = full_key(kmin, i);
              }
              before += __popc(tie);
            }
          __syncthreads();
          thr = s_pick[1];
          __syncthreads();
          return;
        }
        shift = max(0, 32 - __clz(kmax - kmin) - 11);
        __syncthreads();
      }
    };
    __syncthreads();                           // (the table)
    if (S.top_k > 0 && S.top_k < V) find(false);
    if (S.top_p < 1.f) find(true);

    // the running sum of the kept weights in the order of the indices: per warp's segment, then within the one that it passes the bound in
    auto kept_weight = [&](int i) -> u64 {
      if (i >= V) return 0;
      const float x = get(i);
      if (!(x > -INFINITY) || !W.eligible(x) || full_key(ordered(x), i) < thr) return 0;
      return W(x);
    };
    u64 sum = 0;
    for (int i0 = warp * seg; i0 < min(V, (warp + 1) * seg); i0 += 32) sum += kept_weight(i0 + lane);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncthreads();
    if (lane == 0) red[warp] = sum;
    __syncthreads();
    u64 total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) total += red[w];
    const float uf = P.u[row];
    const double bound = (double)(uf >= 0.f ? fminf(uf, 0.99999994f) : 0.f) * (double)total;   // (NaN: 0)
    int sw = NW - 1;
    u64 before = 0, run = 0;
    bool found = false;
    for (int w = 0; w < NW; ++w) {
      const u64 next = run + red[w];
      if (!found && (double)next > bound) { sw = w; before = run; found = true; }
      run = next;
    }
    for (int i0 = sw * seg; i0 < min(V, (sw + 1) * seg); i0 += NT) {
      u64 all;
      const u64 w = kept_weight(i0 + tid < (sw + 1) * seg ? i0 + tid : V);
      const u64 incl = BlockOps<NT>::scan(w, red, all);
      if (tid == 0) s_int[0] = -1;
      __syncthreads();
      if ((double)(before + incl) > bound && !((double)(before + incl - w) > bound)) s_int[0] = i0 + tid;
      __syncthreads();
      token = s_int[0];
      if (token >= 0) break;
      before += all;
    }
  }
  if (tid == 0) {
    P.tokens[(size_t)req * (P.k_max + 1) + r_in] = token;
    if (P.k[req] == 0) P.accept[req] = 0;
  }
}

// The stairs walk over the drawn tokens; one thread per request, started while the rows' kernel ends.
__global__ void k_sample_accept(const __grid_constant__ SampleParams P) {
  wait_prerequisites();
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= P.n_req || P.k[i] == 0) return;
  const int k = P.k[i];
  int a = 0;
  while (a < k && P.draft[(size_t)i * P.k_max + a] == P.tokens[(size_t)i * (P.k_max + 1) + a]) ++a;
  P.accept[i] = a;
}

template <typename T, int NT, bool STAGED> int launch_rows(const SampleParams& P, size_t smem, cudaStream_t st) {
  auto kern = k_sample<T, NT, STAGED>;
  if (smem > 48 * 1024) SCK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - 2048));
  kern<<<P.n_rows, NT, smem, st>>>(P);
  SCK(cudaGetLastError());
  return STAIRS_OK;
}

template <typename T> int launch_sample(const SampleParams& P, cudaStream_t st) {
  const size_t fixed = (size_t)NB * 8 + SMALL * 16 + 64 * 8, row = (size_t)P.vocab * sizeof(T);
  const bool staged = fixed + row <= 227 * 1024 - 2048;
  if (staged) return sizeof(T) == 4 ? launch_rows<T, 1024, true>(P, fixed + row, st) : launch_rows<T, 512, true>(P, fixed + row, st);
  return launch_rows<T, 512, false>(P, fixed, st);
}

}  // namespace
}  // namespace stairs

using namespace stairs;

extern "C" int stairs_sample_static(const void* logits_dev, int dtype, int vocab, int64_t ld, int n_req, const int32_t* k_host,
                                    const stairs_sampling* params_host, const float* u_dev, const int32_t* draft_dev, int k_max,
                                    int32_t* target_tokens_dev, int32_t* accept_len_dev, void* stream) {
  const char* who = "stairs_sample_static";
  if (!logits_dev || !k_host || !params_host || !u_dev || !target_tokens_dev || !accept_len_dev) return static_fail(STAIRS_EINVAL, "%s: NULL buffer", who);
  if (dtype < DT_F32 || dtype > DT_F16) return static_fail(STAIRS_EINVAL, "%s: dtype %d", who, dtype);
  if (vocab < 1 || ld < vocab) return static_fail(STAIRS_EINVAL, "%s: vocab=%d, ld=%lld", who, vocab, (long long)ld);
  if (vocab > (1 << 20)) return static_fail(STAIRS_EUNSUPPORTED, "%s: vocab=%d above 2^20", who, vocab);
  if (reinterpret_cast<uintptr_t>(logits_dev) % dtype_bytes(dtype)) return static_fail(STAIRS_EINVAL, "%s: logits_dev is not aligned to its type", who);
  if (n_req < 1 || n_req > STAIRS_SAMPLE_MAX_REQ) return static_fail(STAIRS_ENOSPC, "%s: n_req=%d outside 1..%d", who, n_req, STAIRS_SAMPLE_MAX_REQ);
  if (k_max < 0 || k_max > 63) return static_fail(STAIRS_EINVAL, "%s: k_max=%d outside 0..63", who, k_max);
  SampleParams P{};
  int rows = 0, top = 0;
  for (int i = 0; i < n_req; ++i) {
    const stairs_sampling& s = params_host[i];
    if (k_host[i] < 0 || k_host[i] > k_max) return static_fail(STAIRS_EINVAL, "%s: k[%d]=%d outside 0..k_max=%d", who, i, k_host[i], k_max);
    if (k_host[i] > 0 && !draft_dev) return static_fail(STAIRS_EINVAL, "%s: draft_dev is NULL", who);
    if (!(s.temperature == 0.f || (s.temperature >= 1e-6f && s.temperature <= 1e6f)))
      return static_fail(STAIRS_EINVAL, "%s: temperature[%d]=%g is neither 0 nor within 1e-6..1e6", who, i, s.temperature);
    if (s.top_k < 0) return static_fail(STAIRS_EINVAL, "%s: top_k[%d]=%d is negative", who, i, s.top_k);
    if (!(s.top_p > 0.f && s.top_p <= 1.f)) return static_fail(STAIRS_EINVAL, "%s: top_p[%d]=%g outside (0, 1]", who, i, s.top_p);
    if (!(s.min_p >= 0.f && s.min_p <= 1.f)) return static_fail(STAIRS_EINVAL, "%s: min_p[%d]=%g outside [0, 1]", who, i, s.min_p);
    P.s[i] = s; P.k[i] = k_host[i]; P.off[i] = rows;
    rows += k_host[i] + 1;
    top = std::max(top, k_host[i]);
  }
  if (rows > STAIRS_STATIC_MAX_ROWS) return static_fail(STAIRS_ENOSPC, "%s: %d rows above %d", who, rows, STAIRS_STATIC_MAX_ROWS);
  P.logits = logits_dev; P.u = u_dev; P.draft = draft_dev; P.tokens = target_tokens_dev; P.accept = accept_len_dev;
  P.ld = ld; P.vocab = vocab; P.n_req = n_req; P.n_rows = rows; P.k_max = k_max;
  int lg = 0;
  while ((1 << lg) < vocab) ++lg;
  P.bits = std::min(47, 62 - lg);             // the sum of all weights stays below 2^62
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const int rc = dtype == DT_F32 ? launch_sample<float>(P, st) : dtype == DT_BF16 ? launch_sample<bf16>(P, st) : launch_sample<__half>(P, st);
  if (rc || top == 0) return rc;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((n_req + 63) / 64); cfg.blockDim = dim3(64); cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization; at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = 1;
  SCK(cudaLaunchKernelEx(&cfg, k_sample_accept, P));
  return STAIRS_OK;
}
