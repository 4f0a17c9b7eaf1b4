// Rules on logits: penalties for repeated tokens, biases, masks.
#include "cache.hpp"
#include "values.hpp"

namespace spt {

namespace {

struct Logits {
  const void* in;
  void* out;
  int64_t in_stride, out_stride, allowed_stride;
  int rows, cols, sequences;
  const int32_t* first;
  Pattern seen, tree, bias;
  const float* bias_vals;
  const int32_t* drafts;
  const float *repetition, *presence, *frequency;
  const uint32_t* allowed;
};

constexpr int kSegment = 8192;  // columns of a workgroup

// A workgroup takes a row and a segment of the columns: the counts and the biases of the segment are collected in LDS, then the
// row's logits go through once.
template <class T>
__global__ void __launch_bounds__(kBlock) logits_kernel(Logits a) {
  __shared__ int count[kSegment];
  __shared__ float bias[kSegment];
  const int r = blockIdx.x, lo = blockIdx.y * kSegment, n = a.cols - lo < kSegment ? a.cols - lo : kSegment;
  int s = r, begin = r;
  if (a.first) {
    s = wave_row_of(a.first, a.sequences, r);
    if (s < 0) return;
    begin = clamped(a.first[s], 0, a.rows);
  }
  for (int v = threadIdx.x; v < n; v += kBlock) count[v] = 0, bias[v] = 0;
  __syncthreads();
  if (a.seen.pos)
    for (int e = pattern_begin(a.seen, s) + threadIdx.x; e < pattern_end(a.seen, s); e += kBlock) {
      const unsigned v = static_cast<unsigned>(a.seen.crd[e]) - lo;
      if (v < static_cast<unsigned>(n)) atomicAdd(&count[v], 1);
    }
  if (a.drafts) {
    const int x0 = a.tree.pos ? pattern_begin(a.tree, r) : begin, x1 = a.tree.pos ? pattern_end(a.tree, r) : r + 1;
    const int end = a.first ? clamped(a.first[s + 1], 0, a.rows) : r + 1;
    for (int e = x0 + threadIdx.x; e < x1; e += kBlock) {
      const int64_t node = a.tree.pos ? static_cast<int64_t>(begin) + a.tree.crd[e] : e;
      if (node < begin || node >= end) continue;
      const unsigned v = static_cast<unsigned>(a.drafts[node]) - lo;
      if (v < static_cast<unsigned>(n)) atomicAdd(&count[v], 1);
    }
  }
  if (a.bias.pos)
    for (int e = pattern_begin(a.bias, s) + threadIdx.x; e < pattern_end(a.bias, s); e += kBlock) {
      const unsigned v = static_cast<unsigned>(a.bias.crd[e]) - lo;
      if (v < static_cast<unsigned>(n)) bias[v] = a.bias_vals[e];
    }
  __syncthreads();
  const float rep = a.repetition ? a.repetition[s] : 1, pres = a.presence ? a.presence[s] : 0, freq = a.frequency ? a.frequency[s] : 0;
  const T* in = static_cast<const T*>(a.in) + r * a.in_stride + lo;
  T* out = static_cast<T*>(a.out) + r * a.out_stride + lo;
  for (int v = threadIdx.x; v < n; v += kBlock) {
    float x = to_float(in[v]);
    if (count[v] > 0) x = (x > 0 ? x / rep : x * rep) - (pres + freq * static_cast<float>(count[v]));
    x += bias[v];
    if (a.allowed && !(a.allowed[r * a.allowed_stride + ((lo + v) >> 5)] >> ((lo + v) & 31) & 1)) x = -INFINITY;
    out[v] = from_float<T>(x);
  }
}

}  // namespace

spt_status adjust_logits_dispatch(int32_t dtype, int64_t R, int64_t V, const void* logits, int64_t logits_stride,
                                  const spt_logit_rules* rules, void* out, int64_t out_stride, hipStream_t stream) {
  const Logits a{logits, out, logits_stride, out_stride, rules->allowed_stride, static_cast<int>(R), static_cast<int>(V),
                 static_cast<int>(rules->sequences), rules->first, pattern_view(rules->seen), pattern_view(rules->tree),
                 pattern_view(rules->bias), rules->bias ? static_cast<const float*>(rules->bias->vals) : nullptr, rules->drafts,
                 rules->repetition, rules->presence, rules->frequency, rules->allowed};
  const dim3 grid(static_cast<unsigned>(R), static_cast<unsigned>((V + kSegment - 1) / kSegment));
  if (dtype == SPT_F32) logits_kernel<float><<<grid, kBlock, 0, stream>>>(a);
  else if (dtype == SPT_F16) logits_kernel<f16><<<grid, kBlock, 0, stream>>>(a);
  else logits_kernel<bf16><<<grid, kBlock, 0, stream>>>(a);
  SPT_CHECK_LAUNCH("adjust_logits");
  return SPT_OK;
}

}  // namespace spt
