// Attention of drafted tokens over the pages of a cache.
#include "cache.hpp"
#include "values.hpp"

namespace spt {

namespace {

struct Attention {
  Cache c;
  int layer, total, q_heads, group;
  const int32_t* first;
  Pattern tree;  // pos NULL: each token sees those up to itself
  const char* q;
  char* out;
  float* lse;
  int64_t q_token_bytes, q_head_bytes, out_token_bytes, out_head_bytes;
  float scale;
};

__device__ __forceinline__ float wave_max(float v) {
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// A wave for each drafted token and head: 64 tokens of the row at a time, one to a lane for the scores; for the sums of V a lane
// owns values lane, lane + 64, .. of the head.
template <class T>
__global__ void __launch_bounds__(64) attention_kernel(Attention a) {
  __shared__ float q[256];
  const Cache& c = a.c;
  const int i = blockIdx.x, h = blockIdx.y, lane = lane_id(), width = c.width_bytes / sizeof(T);
  const int s = wave_row_of(a.first, c.rows, i);
  if (s < 0) return;
  const Drafted d = drafted(a.first, s, a.total);
  if (i < d.begin || i >= d.begin + d.count) return;
  const int length = row_length(c, s), context = length - d.count, mask = (1 << c.shift) - 1;
  const T* qi = reinterpret_cast<const T*>(a.q + i * a.q_token_bytes + h * a.q_head_bytes);
  for (int e = lane; e < width; e += kWave) q[e] = to_float(qi[e]) * a.scale;
  __syncthreads();
  const int64_t at = a.layer * c.layer_bytes + (h / a.group) * c.head_bytes;
  float m = -INFINITY, l = 0, o[4] = {0, 0, 0, 0};
  for (int base = 0; base < length; base += kWave) {
    const int t = base + lane;
    const int page = t < length ? page_at(c, s, t >> c.shift) : -1;
    bool seen = page >= 0 && t < context;
    if (base + kWave > context) {
      if (a.tree.pos) {
        uint64_t bits = 0;
        for (int e = pattern_begin(a.tree, i) + lane; e < pattern_end(a.tree, i); e += kWave) {
          const int j = a.tree.crd[e];
          const int64_t b = static_cast<int64_t>(context) + j - base;
          if (j >= 0 && j < d.count && b >= 0 && b < kWave) bits |= 1ull << b;
        }
        for (int x = 32; x; x >>= 1) bits |= __shfl_xor(static_cast<unsigned long long>(bits), x);
        seen = seen || (page >= 0 && (bits >> lane & 1));
      } else {
        seen = seen || (page >= 0 && t - context <= i - d.begin);
      }
    }
    const int64_t slot = page * c.page_bytes + (t & mask) * c.slot_bytes + at;
    float z = -INFINITY;
    if (seen) {
      z = 0;
      for (int e = 0; e < width; e += Vec16<T>::n) {
        const Vec16<T> k = *reinterpret_cast<const Vec16<T>*>(c.K + slot + e * sizeof(T));
#pragma unroll
        for (int x = 0; x < Vec16<T>::n; ++x) z += q[e + x] * to_float(k.v[x]);
      }
    }
    const float top = fmaxf(m, wave_max(z)), zero = top == -INFINITY ? 0 : top;
    const float p = seen ? expf(z - zero) : 0, keep = m == -INFINITY ? 0 : expf(m - zero);
    l = l * keep + wave_sum(p);
    m = top;
    for (int x = 0; x < 4; ++x) o[x] *= keep;
    uint64_t todo = __ballot(seen);
    while (todo) {
      const int b = __builtin_ctzll(todo);
      todo &= todo - 1;
      const float pb = __shfl(p, b);
      const T* v = reinterpret_cast<const T*>(c.V + __shfl(static_cast<long long>(slot), b));
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (lane + x * kWave < width) o[x] += pb * to_float(v[lane + x * kWave]);
    }
  }
  T* out = reinterpret_cast<T*>(a.out + i * a.out_token_bytes + h * a.out_head_bytes);
  const bool none = l == 0;
  for (int x = 0; x < 4; ++x)
    if (lane + x * kWave < width) out[lane + x * kWave] = from_float<T>(none ? 0 : o[x] / l);
  if (a.lse && lane == 0) a.lse[static_cast<int64_t>(i) * a.q_heads + h] = none ? -INFINITY : m + logf(l);
}

}  // namespace

size_t cache_attention_workspace(const spt_cache*, int32_t) { return 256; }

spt_status cache_attention_dispatch(const spt_cache* cache, int32_t layer, const int32_t* first, int32_t total,
                                    const spt_tensor* tree, const void* q, int32_t q_heads, int64_t q_token_stride,
                                    int64_t q_head_stride, float scale, void* out, int64_t out_token_stride, int64_t out_head_stride,
                                    float* lse, void* ws, hipStream_t stream) {
  const int64_t b = value_bytes(cache->dtype);
  const Attention a{cache_view(cache), layer, total, q_heads, q_heads / cache->heads, first, pattern_view(tree),
                    static_cast<const char*>(q), static_cast<char*>(out), lse, q_token_stride * b, q_head_stride * b,
                    out_token_stride * b, out_head_stride * b, scale};
  const dim3 grid(total, q_heads);
  if (cache->dtype == SPT_F32) attention_kernel<float><<<grid, kWave, 0, stream>>>(a);
  else if (cache->dtype == SPT_F16) attention_kernel<f16><<<grid, kWave, 0, stream>>>(a);
  else attention_kernel<bf16><<<grid, kWave, 0, stream>>>(a);
  SPT_CHECK_LAUNCH("cache_attention");
  return SPT_OK;
}

}  // namespace spt
