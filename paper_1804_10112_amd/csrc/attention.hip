// Attention of drafted tokens over the pages of a cache: the kernel for few rows, the joining of parts, the choice of a kernel.
#include "attention.hpp"

namespace spt {

namespace {

// ROW_BYTES: bytes of a head's values, rounded up to what the matrix instructions take; NQ: 16 rows times it to a tile.
// FULL: a head fills ROW_BYTES.
// The four waves of a workgroup take 16 or 32 tokens of a step each and do not meet until the tile's end.
template <class T, int ROW_BYTES, int NQ, bool FULL>
__global__ void __launch_bounds__(kBlock, (groups_of<ROW_BYTES, sizeof(T)>() / 256)) attention_kernel(Attention a) {
  constexpr int kTokens = sizeof(T) == 4 ? 16 : 32;  // of a wave in a step: what one matrix instruction takes of 16 bytes a lane
  constexpr int kSub = kTokens / 16, kChunks = ROW_BYTES / 64, kWidth = ROW_BYTES / sizeof(T), kTiles = kWidth / 16;
  constexpr int kRows = 16 * NQ, kGroups = groups_of<ROW_BYTES, sizeof(T)>();
  using P = Plan<kRows, kTokens * kWaves>;
  __shared__ __attribute__((aligned(16))) char area[kWaves][64 * kWidth];  // V of a wave's tokens; O of 16 rows when waves meet
  __shared__ float stat[2][kWaves][kRows];
  const Cache& c = a.c;
  const int group = xcd_contiguous_block_id(), lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), i = lane & 15,
            quad = lane >> 4, vecs = c.width_bytes / 16, width = c.width_bytes / sizeof(T);
  Walk<P> at{{a}};
  if (!at.start(group, kGroups)) return;

  do {
    const int row0 = at.tile * kRows, tokens = at.plan.end(at.q, at.tile), common = at.plan.common(at.q, row0);
    const int64_t pool = a.layer * c.layer_bytes + at.head * c.head_bytes;
    // Where the tokens of the lane lie: the table is read two steps ahead, and what it says is looked at one step ahead.
    auto entries = [&](int base, int(&entry)[kSub]) {
#pragma unroll
      for (int u = 0; u < kSub; ++u) entry[u] = table_entry(c, at.s, base + 16 * u + i, tokens);
    };
    auto places = [&](int base, const int(&entry)[kSub], int64_t(&place)[kSub]) {
#pragma unroll
      for (int u = 0; u < kSub; ++u) place[u] = slot_of(c, entry[u], base + 16 * u + i, tokens);
    };
    // For tokens that are nowhere the first slot of the pool is read, behind the width its last 16 bytes again: values that are put
    // aside before they count.
    auto load = [&](const char* from, const int64_t(&place)[kSub], i4(&x)[kSub][kChunks]) {
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        const char* token = from + pool + (place[u] < 0 ? 0 : place[u]);
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
          const int chunk = quad + 4 * j;
          x[u][j] = *reinterpret_cast<const i4*>(token + (FULL || chunk < vecs ? chunk : vecs - 1) * 16);
        }
      }
    };

    char* mine = area[wave];
    constexpr int kApart = kWaves * kTokens;
    int64_t place[kSub];
    int entry[kSub];
    i4 qf[NQ][kChunks], k[kSub][kChunks], v[kSub][kChunks];
    int base = at.step * kApart + wave * kTokens;
    const int limit = at.stop * kApart < tokens ? at.stop * kApart : tokens;
    if (base < limit) {
      entries(base, entry);
      load_queries<16>(a, at.q, at.head, row0, qf);
      places(base, entry, place);
      entries(base + kApart, entry);
      load(c.K, place, k);
      load(c.V, place, v);
      finish_queries<T, FULL>(a, qf);
    }
    f4 o[NQ][kTiles];
    float m[NQ], l[NQ];
    bool vast = false;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      m[n] = -INFINITY;
      l[n] = 0;
#pragma unroll
      for (int d = 0; d < kTiles; ++d) o[n][d] = f4{0, 0, 0, 0};
    }
    for (; base < limit; base += kApart) {
      if (!FULL)
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
          for (int j = 0; j < kChunks; ++j)
            if (quad + 4 * j >= vecs) k[u][j] = i4{0, 0, 0, 0};
      f4 z[NQ][kSub];
#pragma unroll
      for (int u = 0; u < kSub; ++u)
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          z[n][u] = f4{0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < kChunks; ++j) z[n][u] = multiply<T>(k[u][j], qf[n][j], z[n][u]);
        }
      int64_t next[kSub];
      places(base + kApart, entry, next);
      entries(base + 2 * kApart, entry);
      load(c.K, next, k);

      // tokens of the wave that are there, and those that each row sees
      uint32_t there = 0, bad = 0, sight[NQ];
#pragma unroll
      for (int u = 0; u < kSub; ++u) there |= static_cast<uint32_t>(__ballot(place[u] >= 0) & 0xffff) << (16 * u);
      const bool all = base + kTokens <= common && there == low_bits(kTokens);
      if (!all) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) sight[n] = row_sight(a, at.q, row0 + 16 * n + i, base) & there;
        if (base + kTokens > common) {  // tokens that some rows see and others do not
#pragma unroll
          for (int u = 0; u < kSub; ++u) {
            bool odd = false;
#pragma unroll
            for (int j = 0; j < kChunks; ++j) odd |= any_not_finite<T>(v[u][j]);
            const uint64_t b = __ballot(odd);
            bad |= static_cast<uint32_t>((b | b >> 16 | b >> 32 | b >> 48) & 0xffff) << (16 * u);
          }
          bad &= there;
        }
        const uint32_t out = bad | ~there;
#pragma unroll
        for (int u = 0; u < kSub; ++u)
          if (out >> (16 * u + i) & 1)
#pragma unroll
            for (int j = 0; j < kChunks; ++j) v[u][j] = i4{0, 0, 0, 0};
      }
#pragma unroll
      for (int u = 0; u < kSub; ++u)
#pragma unroll
        for (int j = 0; j < kChunks; ++j) *reinterpret_cast<i4*>(mine + swizzled<ROW_BYTES>(16 * u + i, quad + 4 * j)) = v[u][j];
      int64_t here[kSub];
#pragma unroll
      for (int u = 0; u < kSub; ++u) here[u] = place[u];
      load(c.V, next, v);
#pragma unroll
      for (int u = 0; u < kSub; ++u) place[u] = next[u];

      if (!all)
#pragma unroll
        for (int n = 0; n < NQ; ++n) hide(z[n], &sight[n]);
      softmax_step<T>(z, a.scale, m, l, o, vast);
      i4 p[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) p[n] = weights<T>(z[n]);
      wave_lds_order();
#pragma unroll
      for (int d = 0; d < kTiles; ++d) {
        const i4 vf = turned_values<T, ROW_BYTES>(mine, 0, d);
#pragma unroll
        for (int n = 0; n < NQ; ++n) o[n][d] = multiply<T>(vf, p[n], o[n][d]);
      }
      wave_lds_order();
      while (bad) {
        const int b = __builtin_ctz(bad);
        bad &= bad - 1;
#pragma unroll
        for (int u = 0; u < kSub; ++u)
          if ((b >> 4) == u) {
            const int64_t where = __shfl(static_cast<long long>(here[u]), b & 15);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
              float w = 0;
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if ((b & 3) == r) w = __shfl(z[n][u][r], (b & 12) * 4 + i);
              add_token<T>(c.V + pool + where, width, sight[n] >> b & 1, w, o[n]);
            }
          }
      }
    }

    // the waves meet
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      l[n] = sum_of_row(l[n]);
      if (quad == 0) stat[0][wave][16 * n + i] = m[n], stat[1][wave][16 * n + i] = l[n];
    }
    __syncthreads();
    const bool whole = at.step == 0 && at.stop == at.steps;
    float* slot = a.partial + static_cast<int64_t>(2 * group + (at.step == 0)) * kRows * (kWidth + 2);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stat[0][w][16 * n + i]);
      const float f = exp2_of(m[n] - (top == -INFINITY ? 0 : top));
#pragma unroll
      for (int d = 0; d < kTiles; ++d)
        *reinterpret_cast<f4*>(mine + i * kWidth * 4 + ((4 * d + quad) ^ i) * 16) = o[n][d] * f;
      __syncthreads();
      for (int x = threadIdx.x; x < 16 * kWidth / 4; x += kBlock) {
        const int r = x / (kWidth / 4), e = x - r * (kWidth / 4), row = row0 + 16 * n + r;
        float high = -INFINITY, sum = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) high = fmaxf(high, stat[0][w][16 * n + r]);
        f4 y{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          sum += stat[1][w][16 * n + r] * exp2_of(stat[0][w][16 * n + r] - (high == -INFINITY ? 0 : high));
          y += *reinterpret_cast<const f4*>(area[w] + r * kWidth * 4 + (e ^ r) * 16);
        }
        if (!whole) {
          *reinterpret_cast<f4*>(slot + 2 * kRows + (16 * n + r) * kWidth + 4 * e) = y;
          if (e == 0) slot[16 * n + r] = high, slot[kRows + 16 * n + r] = sum;
        } else if (row < at.q.rows) {
          const int token = at.q.d.begin + row / a.by_group, h = at.head * a.group + row - (token - at.q.d.begin) * a.group;
          T* to = reinterpret_cast<T*>(a.out + token * a.out_token_bytes + h * a.out_head_bytes) + 4 * e;
#pragma unroll
          for (int b = 0; b < 4; ++b)
            if (4 * e < width) to[b] = from_float<T>(sum == 0 ? 0.0f : y[b] / sum);
          if (e == 0 && a.lse) a.lse[static_cast<int64_t>(token) * a.q_heads + h] = natural_lse(high, sum);
        }
      }
      __syncthreads();
    }
  } while (at.next());
}

// Joins the parts of tiles that lie in several workgroups. blockIdx.x is a workgroup that began within a tile; those of one tile share
// its rows, and blockIdx.y divides them further. Few parts: 16 lanes take a row, and all their loads are under way at once; many: the
// waves of a workgroup share the parts of a row.
constexpr int kFewParts = 8;
template <class T, int WIDTH, int ROWS>
__global__ void __launch_bounds__(kBlock) attention_join_kernel(Attention a) {
  constexpr int kEach = WIDTH / 16;  // values of a lane
  __shared__ float area[kWaves][WIDTH], sums[kWaves];
  const Part part = a.part[blockIdx.x];
  if (part.parts == 0) return;
  const Drafted d = drafted(a.first, part.s, a.total);
  const int left = d.count * a.group - part.row, rows = left < ROWS ? left : ROWS;
  const int lane = lane_id(), wave = wave_id(), i = lane & 15, quad = lane >> 4;
  constexpr int64_t kSlot = static_cast<int64_t>(ROWS) * (WIDTH + 2);
  const float* second = a.partial + (static_cast<int64_t>(blockIdx.x) - part.place) * 2 * kSlot;  // part p > 0: slot 0 of p - 1 groups on
  auto slot = [&](int p) { return p ? second + (p - 1) * 2 * kSlot : second - kSlot; };
  const int takers = (part.parts - 1) * gridDim.y, taker = part.place * gridDim.y + blockIdx.y;

  // The lane's values 4 i + 64 e .. of row r: those of part p, weighed.
  auto add = [&](int p, int r, float zero, float& sum, f4(&y)[kEach / 4]) {
    const float* from = slot(p);
    const float f = exp2_of(from[r] - zero);
    sum += f * from[ROWS + r];
#pragma unroll
    for (int e = 0; e < kEach / 4; ++e) y[e] += f * *reinterpret_cast<const f4*>(from + 2 * ROWS + r * WIDTH + 64 * e + 4 * i);
  };
  auto write = [&](int r, float top, float sum, const f4(&y)[kEach / 4]) {
    const int row = part.row + r, token = d.begin + row / a.by_group, h = part.head * a.group + row - (token - d.begin) * a.group;
    T* to = reinterpret_cast<T*>(a.out + token * a.out_token_bytes + h * a.out_head_bytes);
    const int width = a.c.width_bytes / static_cast<int>(sizeof(T));
#pragma unroll
    for (int e = 0; e < kEach / 4; ++e)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        if (64 * e + 4 * i < width) to[64 * e + 4 * i + b] = from_float<T>(sum == 0 ? 0.0f : y[e][b] / sum);
    if (i == 0 && a.lse) a.lse[static_cast<int64_t>(token) * a.q_heads + h] = natural_lse(top, sum);
  };

  if (part.parts <= kFewParts) {
    for (int r = (taker * kWaves + wave) * 4 + quad; r < rows; r += takers * kWaves * 4) {
      float top = -INFINITY, sum = 0;
      f4 y[kEach / 4] = {};
      float m[kFewParts], l[kFewParts];
      f4 x[kFewParts / 2][kEach / 4];
      auto load = [&](int p0) {  // of four parts, again the last one where there are fewer
#pragma unroll
        for (int p = 0; p < kFewParts / 2; ++p) {
          const float* from = slot(p0 + p < part.parts ? p0 + p : part.parts - 1);
          m[p0 + p] = from[r];
          l[p0 + p] = from[ROWS + r];
#pragma unroll
          for (int e = 0; e < kEach / 4; ++e) x[p][e] = *reinterpret_cast<const f4*>(from + 2 * ROWS + r * WIDTH + 64 * e + 4 * i);
        }
      };
      auto add_loaded = [&](int p0, float rescale) {
        const float zero = top == -INFINITY ? 0 : top;
        sum *= rescale;
#pragma unroll
        for (int e = 0; e < kEach / 4; ++e) y[e] *= rescale;
#pragma unroll
        for (int p = 0; p < kFewParts / 2; ++p) {
          if (p0 + p >= part.parts) continue;
          const float f = exp2_of(m[p0 + p] - zero);
          sum += f * l[p0 + p];
#pragma unroll
          for (int e = 0; e < kEach / 4; ++e) y[e] += f * x[p][e];
        }
      };
      load(0);
#pragma unroll
      for (int p = 0; p < kFewParts / 2; ++p) top = fmaxf(top, m[p]);
      add_loaded(0, 1);
      if (part.parts > kFewParts / 2) {
        load(kFewParts / 2);
        const float before = top;
#pragma unroll
        for (int p = kFewParts / 2; p < kFewParts; ++p) top = fmaxf(top, m[p]);
        add_loaded(kFewParts / 2, exp2_of(before - (top == -INFINITY ? 0 : top)));
      }
      write(r, top, sum, y);
    }
    return;
  }
  for (int r = taker; r < rows; r += takers) {  // the 16 lanes of each quad take every fourth of the wave's parts
    float top = -INFINITY, sum = 0;
    f4 y[kEach / 4] = {};
    for (int p = lane; p < part.parts; p += kWave) top = fmaxf(top, slot(p)[r]);
    for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    const float zero = top == -INFINITY ? 0 : top;
#pragma unroll 4
    for (int p = wave * 4 + quad; p < part.parts; p += kWaves * 4) add(p, r, zero, sum, y);
    sum = sum_of_row(sum);
#pragma unroll
    for (int e = 0; e < kEach / 4; ++e)
#pragma unroll
      for (int b = 0; b < 4; ++b) y[e][b] = sum_of_row(y[e][b]);
    __syncthreads();
    if (quad == 0)
#pragma unroll
      for (int e = 0; e < kEach / 4; ++e) *reinterpret_cast<f4*>(&area[wave][64 * e + 4 * i]) = y[e];
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    if (wave != 0 || quad != 0) continue;
    for (int w = 1; w < kWaves; ++w) {
      sum += sums[w];
#pragma unroll
      for (int e = 0; e < kEach / 4; ++e) y[e] += *reinterpret_cast<const f4*>(&area[w][64 * e + 4 * i]);
    }
    write(r, top, sum, y);
  }
}

template <class T, int ROW_BYTES, int NQ>
void launch(const Attention& a, hipStream_t stream) {
  constexpr int groups = groups_of<ROW_BYTES, sizeof(T)>();
  if (a.c.width_bytes == ROW_BYTES)
    attention_kernel<T, ROW_BYTES, NQ, true><<<groups, kBlock, 0, stream>>>(a);
  else
    attention_kernel<T, ROW_BYTES, NQ, false><<<groups, kBlock, 0, stream>>>(a);
  launch_join<T>(a, groups, 16 * NQ, ROW_BYTES / sizeof(T), stream);
}

// Heads are padded to the next of 64, 128, 192, 256 values: what a wave multiplies by zeros costs no bytes.
template <class T, int NQ>
void launch_few_rows(const Attention& a, hipStream_t stream) {
  const int width = a.c.width_bytes / sizeof(T);
  if (width <= 64) launch<T, 64 * sizeof(T), NQ>(a, stream);
  else if (width <= 128) launch<T, 128 * sizeof(T), NQ>(a, stream);
  else if (width <= 192) launch<T, 192 * sizeof(T), NQ>(a, stream);
  else launch<T, 256 * sizeof(T), NQ>(a, stream);
}

template <class T, int WIDTH>
void launch_join_width(const Attention& a, int groups, int rows, hipStream_t stream) {
  const dim3 grid(groups, rows / 16);  // a tile of two parts: four rows to each wave
  if (rows == 16) attention_join_kernel<T, WIDTH, 16><<<grid, kBlock, 0, stream>>>(a);
  else if (rows == 32) attention_join_kernel<T, WIDTH, 32><<<grid, kBlock, 0, stream>>>(a);
  else if (rows == 64) attention_join_kernel<T, WIDTH, 64><<<grid, kBlock, 0, stream>>>(a);
  else attention_join_kernel<T, WIDTH, 128><<<grid, kBlock, 0, stream>>>(a);
}

// Rows of a tile by the mean rows of a sequence and head of K and V, empty ones counted in (n may differ; that costs time, nothing else:
// four trees of 116 rows over 2500 tokens each, by themselves or among 16 sequences, take 43 us, among 64, so in tiles of 16, 50). Few rows: K and V are
// read once for 16 of them, waves by themselves; more: once for 64, or for 128 where the products take longer than the loads.
// 16 sequences of 2500 tokens, 8 heads of 128 values in bf16, us with tiles of 16 | 64 | 128 rows: 4 rows 43 | 47 | 59, 16 rows 43 | 47 | 54,
// 20 rows 54 | 49 | 56, 64 rows 83 | 58 | 64, 128 rows 159 | 70 | 78; 4 sequences of 4096: 256 rows - | 59 | 71, 384 rows - | 78 | 71,
// 1024 rows - | 160 | 120, 4096 rows - | 522 | 359. (32-bit values: 16 or 32 rows, waves by themselves; for 16-bit ones 32 rows so
// took 54 to 55 us where 64 took 49 to 52. Their chunks read K and V again for each 32 rows: of 64, 256, 1024 tokens, 2 sequences of
// 2500, 8 heads, 61, 118, 298 us, where the products alone take 9, 32, 108.)
template <class T>
void dispatch(const Attention& a, hipStream_t stream) {
  const int64_t rows = static_cast<int64_t>(a.total) * a.group, sequences = a.c.rows;
  if (rows <= 16 * sequences) {
    launch_few_rows<T, 1>(a, stream);
  } else if constexpr (sizeof(T) == 4) {
    launch_few_rows<T, 2>(a, stream);
  } else {
    launch_many_rows<T>(a, rows > 256 * sequences, stream);
  }
}

}  // namespace

template <class T>
void launch_join(const Attention& a, int groups, int rows, int width, hipStream_t stream) {
  if (width == 64) launch_join_width<T, 64>(a, groups, rows, stream);
  else if (width == 128) launch_join_width<T, 128>(a, groups, rows, stream);
  else if (width == 192) launch_join_width<T, 192>(a, groups, rows, stream);
  else launch_join_width<T, 256>(a, groups, rows, stream);
}
template void launch_join<f16>(const Attention&, int, int, int, hipStream_t);
template void launch_join<bf16>(const Attention&, int, int, int, hipStream_t);

// The largest of the kernels' needs: m, l and O of two tiles of 128 rows (64 of heads of more than 128 values) for each workgroup.
size_t cache_attention_workspace(const spt_cache* c, int32_t) {
  const size_t width = c->width <= 128 ? (c->width + 63) / 64 * 64 : 256;
  const size_t rows = c->dtype == SPT_F32 ? 32 : c->width <= 128 ? 128 : 64;
  return align_up(kMostGroups * sizeof(Part), 256) + align_up(kMostGroups * 2 * rows * (width + 2) * sizeof(float), 256);
}

spt_status cache_attention_dispatch(const spt_cache* cache, int32_t layer, const int32_t* first, int32_t total,
                                    const spt_tensor* tree, const void* q, int32_t q_heads, int64_t q_token_stride,
                                    int64_t q_head_stride, float scale, void* out, int64_t out_token_stride, int64_t out_head_stride,
                                    float* lse, void* ws, hipStream_t stream) {
  const int64_t b = value_bytes(cache->dtype);
  Workspace w(ws, cache_attention_workspace(cache, q_heads));
  Part* part = w.take<Part>(kMostGroups);
  float* partial = w.take<float>(0);
  // a scale of 0 becomes the smallest number, with which hidden scores stay -infinity and the largest ones are 5e-7
  const float factor = scale == 0 ? __FLT_DENORM_MIN__ : fabsf(scale) * 1.4426950408889634f;
  const Attention a{cache_view(cache), layer, total, q_heads, q_heads / cache->heads, divisor(q_heads / cache->heads), first, pattern_view(tree),
                    static_cast<const char*>(q), static_cast<char*>(out), lse, q_token_stride * b, q_head_stride * b,
                    out_token_stride * b, out_head_stride * b, factor, scale < 0, part, partial};
  if (cache->dtype == SPT_F32) dispatch<float>(a, stream);
  else if (cache->dtype == SPT_F16) dispatch<f16>(a, stream);
  else dispatch<bf16>(a, stream);
  SPT_CHECK_LAUNCH("cache_attention");
  return SPT_OK;
}

}  // namespace spt
