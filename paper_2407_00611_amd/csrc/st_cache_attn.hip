// Attention of packed rows against a cache of pages: a workgroup for each row and query head, a thread a key.
#include "st_cache.h"
#include "st_score.h"

namespace st {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ float value(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ float value(const uint8_t* p) { return e4m3_pair<false>(*p).x; }

template <typename T, typename S>
__global__ __launch_bounds__(kThreads) void cache_attn_kernel(const CacheAttnArgs a) {
  __shared__ float q[256], p[kThreads], fold[kThreads];
  __shared__ int found;
  const CacheArgs& c = a.c;
  const int t = blockIdx.x, h = blockIdx.y, hk = h / (a.Hq / c.Hkv), tid = threadIdx.x, D = c.D;
  if (tid == 0) found = -1;
  __syncthreads();
  for (int b = tid; b < c.B; b += kThreads) {
    const SeqRows r = seq_rows(a.starts, b, a.T);
    if (t >= r.first && t < r.first + min(r.n, a.max_rows)) found = b;
  }
  if (tid < D) q[tid] = value((const T*)a.q.ptr + (int64_t)t * a.q.ss + (int64_t)h * a.q.sh + tid);
  __syncthreads();
  const int b = found;
  if (b < 0) return;
  const SeqRows r = seq_rows(a.starts, b, a.T);
  const int len = seq_len(c, b);
  const int64_t pos = (a.q_first ? a.q_first[b] : (int64_t)c.lens[b] - r.n) + (t - r.first);
  const int64_t hi = a.causal ? min((int64_t)len, pos + 1) : len, lo = a.window > 0 ? max((int64_t)0, pos - a.window + 1) : 0;
  float m = -INFINITY, l = 0.f, acc = 0.f;
  bool nan = false;
  for (int64_t k0 = lo; k0 < hi; k0 += kThreads) {
    const int64_t x = k0 + tid;
    const int page = x < hi ? page_of(c, b, (int)(x >> c.shift)) : -1;
    float s = -INFINITY;
    if (page >= 0) {
      const S* k = (const S*)c.k.ptr + (int64_t)page * c.k.sb + (x & ((1 << c.shift) - 1)) * c.k.ss + (int64_t)hk * c.k.sh;
      float u = 0.f;
      for (int d = 0; d < D; ++d) u = fmaf(q[d], value(k + d), u);
      if (c.dtype == ST_E4M3) u *= scale_value(c.k_scale[(int64_t)page * c.Hkv + hk]);
      u *= a.scale;
      s = a.cap > 0.f ? a.cap * tanhf(u / a.cap) : u;
      if (a.slopes) s -= a.slopes[h] * (float)(x > pos ? x - pos : pos - x);
    }
    fold[tid] = s;
    __syncthreads();
    float top = m;
    for (int y = 0; y < kThreads; ++y) top = fmaxf(top, fold[y]);
    const float ref = top == -INFINITY ? 0.f : top;
    p[tid] = expf(s - ref);
    __syncthreads();
    const float alpha = expf(m - ref);
    m = top;
    l *= alpha;
    acc *= alpha;
    for (int y = 0; y < kThreads; ++y) {
      l += p[y];
      nan = nan || fold[y] != fold[y];
    }
    if (tid < D)
      for (int y = 0; y < kThreads && k0 + y < hi; ++y) {
        const int64_t x2 = k0 + y;
        const int page2 = page_of(c, b, (int)(x2 >> c.shift));
        if (page2 < 0) continue;
        float v = value((const S*)c.v.ptr + (int64_t)page2 * c.v.sb + (x2 & ((1 << c.shift) - 1)) * c.v.ss + (int64_t)hk * c.v.sh + tid);
        if (c.dtype == ST_E4M3) v *= scale_value(c.v_scale[(int64_t)page2 * c.Hkv + hk]);
        acc = fmaf(p[y], v, acc);
      }
    __syncthreads();
  }
  const float o = l != 0.f ? acc / l : 0.f;
  const int64_t at = ((int64_t)t * a.Hq + h) * D + tid;
  if (tid < D) {
    if (a.o) a.o[at] = o;
    if (a.o_lowp && sizeof(T) == 2) ((uint16_t*)a.o_lowp)[at] = (uint16_t)pack_bf16(o, o);
    else if (a.o_lowp) ((float*)a.o_lowp)[at] = o;
  }
  if (tid == 0) a.lse[(int64_t)h * a.T + t] = nan ? NAN : l != 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnArgs& a, bool bf16, hipStream_t stream) {
  ProfScope prof("cache_attn", stream);
  const dim3 grid((unsigned)a.T, (unsigned)a.Hq), block(kThreads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
  if (a.c.dtype == ST_E4M3) bf16 ? go(cache_attn_kernel<uint16_t, uint8_t>) : go(cache_attn_kernel<float, uint8_t>);
  else bf16 ? go(cache_attn_kernel<uint16_t, uint16_t>) : go(cache_attn_kernel<float, float>);
  return hipGetLastError();
}

}  // namespace st
