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
  int row0;  // of the launch
  const int32_t* first;
  Pattern seen, tree, bias;
  const float* bias_vals;
  const int32_t* drafts;
  const float *repetition, *presence, *frequency;
  const uint32_t* allowed;
};

constexpr int kThreads = 512;

template <class T>
struct Values {
  T v[Vec16<T>::n];
};

// x / d with 1 / d at hand: the product, corrected once by its remainder. Where that is not finite (x or d is an infinity or NaN, d = 0,
// 1 / d or the product is beyond the largest number, which the quotient need not be), the division.
__device__ __forceinline__ float quotient(float x, float d, float by_d) {
  const float q = x * by_d, rest = __builtin_fmaf(-q, d, x);
  return fabsf(rest) < INFINITY ? __builtin_fmaf(rest, by_d, q) : x / d;
}

// Tokens of the sequence that a thread holds in registers; those behind the first 4096 are read again for each segment. 64 rows of 128 000
// logits in bf16, tokens seen: 1000 13 us, 4000 13, 8000 16, 30 000 37, 100 000 123.
constexpr int kKept = 8;
constexpr int kNowhere = -(1 << 30);  // below every segment

// A workgroup takes segments of a row, VECS times 16 bytes a thread, counted from where the row is aligned: blockIdx.y, blockIdx.y +
// gridDim.y, .. In LDS lie the counts of a segment's columns and their biases: integer counts and unique biases, so nothing depends on an
// order. The sequence's tokens are read at once, into registers, and each segment picks its own; the logits of the next segment are
// under way while one is counted. A thread clears the counts that it has read, so a segment takes two barriers. Bound: the logits' bytes,
// 256 rows of 128 000 in bf16 with biases and masks 38 us, 3.7 TB/s (in f32 61, 4.5); as many workgroups as run at once (four of 512 threads to a compute
// unit): with half as many 60 us, with twice as many 46, with longer segments 55; and one row of 32 000 takes 4.6.
template <class T, int VECS, bool BIAS>
__global__ void __launch_bounds__(kThreads, 8) logits_kernel(Logits a) {
  constexpr int n = Vec16<T>::n, kSegment = kThreads * VECS * n;
  __shared__ __attribute__((aligned(16))) int count[kSegment];
  __shared__ __attribute__((aligned(16))) float bias[BIAS ? kSegment : 4];
  const int r = a.row0 + static_cast<int>(blockIdx.x);
  const T* in = static_cast<const T*>(a.in) + r * a.in_stride;
  T* out = static_cast<T*>(a.out) + r * a.out_stride;
  const int ahead = static_cast<int>(-reinterpret_cast<intptr_t>(in) / static_cast<int>(sizeof(T))) & (n - 1);
  int lo = (ahead ? ahead - n : 0) + static_cast<int>(blockIdx.y) * kSegment;  // column of the segment's first value
  if (lo >= a.cols) return;
  int s = r, begin = r, last = r + 1;
  if (a.first) {
    s = wave_row_of(a.first, a.sequences, r);
    if (s < 0) return;
    begin = clamped(a.first[s], 0, a.rows);
    last = clamped(a.first[s + 1], 0, a.rows);
  }
  const bool aligned = (reinterpret_cast<uintptr_t>(out + ahead) & 15) == 0;
  const uint32_t* allowed = a.allowed ? a.allowed + r * a.allowed_stride : nullptr;
  Values<T> x[VECS];
  uint32_t word[VECS][2];  // those with the bits of the first and of the last value
  auto load = [&](int from) {
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
      const int v = from + (k * kThreads + threadIdx.x) * n;
      if (v >= 0 && v + n <= a.cols) {
        x[k] = *reinterpret_cast<const Values<T>*>(__builtin_assume_aligned(in + v, 16));
      } else {
#pragma unroll
        for (int e = 0; e < n; ++e)
          if (v + e >= 0 && v + e < a.cols) x[k].v[e] = in[v + e];
      }
      if (allowed && v < a.cols) {
        word[k][0] = allowed[(v < 0 ? 0 : v) >> 5];
        word[k][1] = allowed[(v + n - 1 < a.cols ? v + n - 1 : a.cols - 1) >> 5];
      }
    }
  };
  load(lo);
  auto column = [&](int v) { return v >= 0 && v < a.cols ? v : kNowhere; };
  auto way_token = [&](int e) {  // of entry e of the row's way
    const int64_t node = a.tree.pos ? static_cast<int64_t>(begin) + a.tree.crd[e] : e;
    return node >= begin && node < last ? column(a.drafts[node]) : kNowhere;
  };
  const int seen0 = a.seen.pos ? pattern_begin(a.seen, s) : 0, seen1 = a.seen.pos ? pattern_end(a.seen, s) : 0;
  const int bias0 = BIAS ? pattern_begin(a.bias, s) : 0, bias1 = BIAS ? pattern_end(a.bias, s) : 0;
  const int way0 = !a.drafts ? 0 : a.tree.pos ? pattern_begin(a.tree, r) : begin;
  const int way1 = !a.drafts ? 0 : a.tree.pos ? pattern_end(a.tree, r) : r + 1;
  const int t = threadIdx.x;
  int token[kKept], way = kNowhere, at_bias = kNowhere;
  float bias_value = 0;
#pragma unroll
  for (int k = 0; k < kKept; ++k) token[k] = k * kThreads + t < seen1 - seen0 ? a.seen.crd[seen0 + k * kThreads + t] : kNowhere;
  if (t < way1 - way0) way = way_token(way0 + t);
  if (BIAS && t < bias1 - bias0) at_bias = column(a.bias.crd[bias0 + t]), bias_value = a.bias_vals[bias0 + t];
  const float rep = a.repetition ? a.repetition[s] : 1, pres = a.presence ? a.presence[s] : 0, freq = a.frequency ? a.frequency[s] : 0;
  const float by_rep = 1 / rep;
  for (int k = t; k < kSegment / 4; k += kThreads) {
    reinterpret_cast<int4*>(count)[k] = int4{0, 0, 0, 0};
    if (BIAS) reinterpret_cast<float4*>(bias)[k] = float4{0, 0, 0, 0};
  }
#pragma unroll
  for (int k = 0; k < kKept; ++k) token[k] = column(token[k]);
  lds_barrier();

  while (true) {
    const unsigned width = a.cols - lo < kSegment ? a.cols - lo : kSegment;
    auto add = [&](int v) {
      if (static_cast<unsigned>(v - lo) < width) atomicAdd(&count[v - lo], 1);
    };
#pragma unroll
    for (int k = 0; k < kKept; ++k) add(token[k]);
    strided(seen0, seen1, kKept * kThreads + t, kThreads, [&](int e) { add(column(a.seen.crd[e])); });
    add(way);
    strided(way0, way1, kThreads + t, kThreads, [&](int e) { add(way_token(e)); });
    if (BIAS) {
      if (static_cast<unsigned>(at_bias - lo) < width) bias[at_bias - lo] = bias_value;
      strided(bias0, bias1, kThreads + t, kThreads, [&](int e) {
        const int v = column(a.bias.crd[e]);
        if (static_cast<unsigned>(v - lo) < width) bias[v - lo] = a.bias_vals[e];
      });
    }
    Values<T> now[VECS];
    uint32_t now_word[VECS][2];
#pragma unroll
    for (int k = 0; k < VECS; ++k) now[k] = x[k], now_word[k][0] = word[k][0], now_word[k][1] = word[k][1];
    const int64_t following = static_cast<int64_t>(lo) + static_cast<int64_t>(gridDim.y) * kSegment;
    const bool more = following < a.cols;
    if (more) load(static_cast<int>(following));
    lds_barrier();
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
      const int at = (k * kThreads + t) * n, v = lo + at;
      if (v >= a.cols) break;
      int c[n], any = 0;
      float y[n];
#pragma unroll
      for (int e = 0; e < n; e += 4) {
        int4* four = reinterpret_cast<int4*>(&count[at + e]);
        c[e] = four->x, c[e + 1] = four->y, c[e + 2] = four->z, c[e + 3] = four->w;
        any |= four->x | four->y | four->z | four->w;
      }
#pragma unroll
      for (int e = 0; e < n; ++e) y[e] = to_float(now[k].v[e]);
      if (any) {
#pragma unroll
        for (int e = 0; e < n; e += 4) *reinterpret_cast<int4*>(&count[at + e]) = int4{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < n; ++e)
          if (c[e]) y[e] = (y[e] > 0 ? quotient(y[e], rep, by_rep) : y[e] * rep) - (pres + freq * static_cast<float>(c[e]));
      }
      if (BIAS)
#pragma unroll
        for (int e = 0; e < n; e += 4) {
          float4* four = reinterpret_cast<float4*>(&bias[at + e]);
          y[e] += four->x, y[e + 1] += four->y, y[e + 2] += four->z, y[e + 3] += four->w;
          *four = float4{0, 0, 0, 0};
        }
      if (allowed) {
        // bit e: value e is allowed; values before the row's first have no bits and do not count
        const int v0 = v < 0 ? 0 : v;
        const uint64_t both = static_cast<uint64_t>(now_word[k][1]) << 32 | now_word[k][0];
        const uint32_t bits = static_cast<uint32_t>(both >> (v0 & 31)) << (v0 - v);
#pragma unroll
        for (int e = 0; e < n; ++e)
          if (!(bits >> e & 1)) y[e] = -INFINITY;
      }
      Values<T> z;
#pragma unroll
      for (int e = 0; e < n; ++e) z.v[e] = from_float<T>(y[e]);
      if (aligned && v >= 0 && v + n <= a.cols) {
        *reinterpret_cast<Values<T>*>(__builtin_assume_aligned(out + v, 16)) = z;
      } else {
#pragma unroll
        for (int e = 0; e < n; ++e)
          if (v + e >= 0 && v + e < a.cols) out[v + e] = z.v[e];
      }
    }
    if (!more) return;
    lo = static_cast<int>(following);
    lds_barrier();
  }
}

// A launch holds fewer than 2^32 threads in a direction: less than 2^23 rows of 512.
constexpr int kRowsAtOnce = 1 << 22;

template <class T, int VECS>
void launch(Logits a, int most, hipStream_t stream) {
  constexpr int segment = kThreads * VECS * Vec16<T>::n;
  // a row that begins in the middle of 16 bytes has up to 15 bytes more
  const int64_t segments = (static_cast<int64_t>(a.cols) + Vec16<T>::n - 1 + segment - 1) / segment;
  const int64_t parts = a.rows < most ? most / a.rows : 1;
  for (; a.row0 < a.rows; a.row0 += kRowsAtOnce) {
    const int rows = a.rows - a.row0 < kRowsAtOnce ? a.rows - a.row0 : kRowsAtOnce;
    const dim3 grid(rows, static_cast<unsigned>(parts < segments ? parts : segments));
    if (a.bias.pos) logits_kernel<T, VECS, true><<<grid, kThreads, 0, stream>>>(a);
    else logits_kernel<T, VECS, false><<<grid, kThreads, 0, stream>>>(a);
  }
}

template <class T>
void dispatch(const Logits& a, hipStream_t stream) {
  launch<T, 1>(a, 1024, stream);
}

}  // namespace

spt_status adjust_logits_dispatch(int32_t dtype, int64_t R, int64_t V, const void* logits, int64_t logits_stride,
                                  const spt_logit_rules* rules, void* out, int64_t out_stride, hipStream_t stream) {
  const Logits a{logits, out, logits_stride, out_stride, rules->allowed_stride, static_cast<int>(R), static_cast<int>(V),
                 static_cast<int>(rules->sequences), 0, rules->first, pattern_view(rules->seen), pattern_view(rules->tree),
                 pattern_view(rules->bias), rules->bias ? static_cast<const float*>(rules->bias->vals) : nullptr, rules->drafts,
                 rules->repetition, rules->presence, rules->frequency, rules->allowed};
  if (dtype == SPT_F32) dispatch<float>(a, stream);
  else if (dtype == SPT_F16) dispatch<f16>(a, stream);
  else dispatch<bf16>(a, stream);
  SPT_CHECK_LAUNCH("adjust_logits");
  return SPT_OK;
}

}  // namespace spt
