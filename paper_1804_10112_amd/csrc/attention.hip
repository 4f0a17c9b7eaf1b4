// Attention of drafted tokens over the pages of a cache.
//
// A tile is up to 16 NQ rows (drafted token, query head) of one sequence that share a head of K and V; rows run token by token, the
// heads of a group side by side. A tile goes through its tokens in steps, once, with the running maximum m and sum l of the softmax:
//   z = scale log2(e) K Q^T,  m' = max(m, z),  P = exp2(z - m'),  l = l exp2(m - m') + sum P,  O^T = O^T exp2(m - m') + V^T P.
// Both products are matrix instructions of 16 x 16 with the tokens as rows of the first result and as the inner dimension of the
// second: a lane then holds, for one row, the tokens 4q .. 4q+3 of each 16 (q = lane / 16), and since the order of an inner dimension
// is free, its P is the operand of the second product as it stands. V is turned round on its way out of LDS.
//
// The work of a call is all steps of all tiles, a number that only the device knows (lengths change between calls of one captured
// graph). Each workgroup of a fixed grid finds its equal share of it from len and first: a range of steps that may begin and end
// within a tile. A tile that lies in one workgroup goes to `out` at once; one that does not leaves m, l and O of each part in the
// workspace, at most two parts a workgroup, and a second kernel joins them.
#include "cache.hpp"
#include "values.hpp"

namespace spt {

namespace {

constexpr int kWaves = kBlock / kWave;
// Workgroups of the grid, as many as run at once on 256 compute units: two each, one where a lane has to hold more than 256 registers.
constexpr int kMostGroups = 512;
template <int ROW_BYTES, int SIZE>
constexpr int groups_of() {
  return ROW_BYTES > (SIZE == 4 ? 512 : 256) ? 256 : 512;
}

typedef int i4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
using LdsQuad = __attribute__((address_space(3))) s4;
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// Which part of the call a workgroup began within a tile, for the joining kernel.
struct Part {
  int parts;  // of the tile, if this workgroup's is the second of them; else 0
  int s, head, row;
};

struct Attention {
  Cache c;
  int layer, total, q_heads, group;
  const int32_t* first;
  Pattern tree;  // pos NULL: each token sees those up to itself
  const char* q;
  char* out;
  float* lse;
  int64_t q_token_bytes, q_head_bytes, out_token_bytes, out_head_bytes;
  float scale;  // times log2(e)
  Part* part;   // of each workgroup
  float* partial;  // two slots for each workgroup: m[rows], l[rows], O[rows][width]
};

template <class T>
__device__ __forceinline__ f4 multiply(i4 a, i4 b, f4 c);  // c += a (16 x 64 bytes of values) times b
template <>
__device__ __forceinline__ f4 multiply<bf16>(i4 a, i4 b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f4 multiply<f16>(i4 a, i4 b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f4 multiply<float>(i4 a, i4 b, f4 c) {
  const f4 x = __builtin_bit_cast(f4, a), y = __builtin_bit_cast(f4, b);
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

// Whether one of the values in 16 bytes is an infinity or a NaN.
template <class T>
__device__ __forceinline__ bool any_not_finite(i4 v) {
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t x = v[e];
    if (sizeof(T) == 4) {
      bad |= (x & 0x7f800000u) == 0x7f800000u;
    } else {
      const uint32_t ones = sizeof(T) == 2 && __is_same(T, f16) ? 0x7c00u : 0x7f80u;
      bad |= (x & ones) == ones || (x >> 16 & ones) == ones;
    }
  }
  return bad;
}

// Tiles of ROWS rows that go through their tokens STEP at a time.
template <int ROWS, int STEP>
struct Plan {
  const Attention& a;

  struct Sequence {
    Drafted d;
    int length, context, rows, tiles;  // context: tokens before the drafted ones, below 0 where some of those are not there
  };
  __device__ __forceinline__ Sequence sequence(int s) const {
    Sequence q;
    q.d = drafted(a.first, s, a.total);
    q.length = a.c.pages ? row_length(a.c, s) : 0;
    q.context = q.length - q.d.count;
    q.rows = q.d.count * a.group;
    q.tiles = (q.rows + ROWS - 1) / ROWS;
    return q;
  }
  // Tokens that the rows of a tile can see.
  __device__ __forceinline__ int end(const Sequence& q, int tile) const {
    if (a.tree.pos) return q.length;
    const int last = (tile + 1) * ROWS < q.rows ? (tile + 1) * ROWS - 1 : q.rows - 1;
    const int e = q.context + last / a.group + 1;
    return e > 0 ? e : 0;
  }
  __device__ __forceinline__ int steps(const Sequence& q, int tile) const {
    const int e = end(q, tile);
    return e > 0 ? (e + STEP - 1) / STEP : 1;  // one for a tile that sees nothing, whose rows have to be written
  }
  __device__ __forceinline__ int64_t head_steps(const Sequence& q) const {
    if (q.tiles == 0) return 0;
    if (a.tree.pos || q.tiles == 1) return static_cast<int64_t>(q.tiles) * steps(q, q.tiles - 1);
    int64_t n = 0;
    for (int t = 0; t < q.tiles; ++t) n += steps(q, t);
    return n;
  }
};

__device__ __forceinline__ int64_t block_inclusive_scan(int64_t v, int64_t* lds) {
  const int lane = lane_id(), wave = wave_id();
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int64_t o = __shfl_up(static_cast<long long>(v), d);
    if (lane >= d) v += o;
  }
  __syncthreads();
  if (lane == kWave - 1) lds[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += lds[w];
  return v;
}

// Finds the sequence that the workgroup's share begins in: `begin` becomes the steps before it within the sequence. All threads of
// the workgroup; false if the share is empty.
template <class P>
__device__ __forceinline__ bool share(const P& plan, int group, int groups, int64_t* lds, int64_t* found, int64_t& per, int64_t& begin, int64_t& end,
                                      int& s) {
  const int rows = plan.a.c.rows, heads = plan.a.c.heads;
  int64_t total = 0, mine = 0, upto = 0;
  for (int base = 0; base < rows; base += kBlock) {
    const int r = base + threadIdx.x;
    mine = r < rows ? plan.head_steps(plan.sequence(r)) * heads : 0;
    upto = total + block_inclusive_scan(mine, lds);
    __syncthreads();
    if (threadIdx.x == kBlock - 1) lds[0] = upto;
    __syncthreads();
    total = lds[0];
    __syncthreads();
  }
  per = (total + groups - 1) / groups;
  begin = group * per;
  end = begin + per < total ? begin + per : total;
  if (begin >= end) return false;
  int64_t before = 0;
  for (int base = 0; base < rows; base += kBlock) {
    const int r = base + threadIdx.x;
    if (rows > kBlock) {
      mine = r < rows ? plan.head_steps(plan.sequence(r)) * heads : 0;
      upto = before + block_inclusive_scan(mine, lds);
    }
    if (upto > begin && upto - mine <= begin) found[0] = r, found[1] = upto - mine;
    __syncthreads();
    if (threadIdx.x == kBlock - 1) lds[0] = upto;
    __syncthreads();
    before = lds[0];
    __syncthreads();
    if (before > begin) break;
  }
  s = __builtin_amdgcn_readfirstlane(static_cast<int>(found[0]));
  const int64_t skipped = found[1];
  begin -= skipped;
  end -= skipped;
  return true;
}

// ROW_BYTES: bytes of a head's values, rounded up to what the matrix instructions take; NQ: 16 rows times it to a tile.
// FULL: a head fills ROW_BYTES.
// The four waves of a workgroup take 16 or 32 tokens of a step each and do not meet until the tile's end.
template <class T, int ROW_BYTES, int NQ, bool FULL>
__global__ void __launch_bounds__(kBlock, (groups_of<ROW_BYTES, sizeof(T)>() / 256)) attention_kernel(Attention a) {
  constexpr int kTokens = sizeof(T) == 4 ? 16 : 32;  // of a wave in a step: what one matrix instruction takes of 16 bytes a lane
  constexpr int kSub = kTokens / 16, kChunks = ROW_BYTES / 64, kWidth = ROW_BYTES / sizeof(T), kTiles = kWidth / 16;
  constexpr int kRows = 16 * NQ, kVecs = ROW_BYTES / 16, kGroups = groups_of<ROW_BYTES, sizeof(T)>();
  using P = Plan<kRows, kTokens * kWaves>;
  __shared__ __attribute__((aligned(16))) char area[kWaves][64 * kWidth];  // V of a wave's tokens; O of 16 rows when waves meet
  __shared__ float stat[2][kWaves][kRows];
  __shared__ int64_t sums[kWaves], found[2];
  const Cache& c = a.c;
  const P plan{a};
  const int group = xcd_contiguous_block_id(), lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), i = lane & 15,
            quad = lane >> 4, vecs = c.width_bytes / 16, width = c.width_bytes / sizeof(T);
  int64_t per, at, end;
  int s;
  const bool some = share(plan, group, kGroups, sums, found, per, at, end, s);
  Part part{0, 0, 0, 0};
  if (!some) {
    if (threadIdx.x == 0) a.part[group] = part;
    return;
  }
  // `at` counts steps within sequence s: head by head, tile by tile
  typename P::Sequence q = plan.sequence(s);
  int64_t in_head = plan.head_steps(q);
  int head = static_cast<int>(at / in_head), tile = 0;
  int64_t rest = at - head * in_head;
  int steps = plan.steps(q, 0);
  while (rest >= steps) rest -= steps, steps = plan.steps(q, ++tile);
  int step = static_cast<int>(rest);
  int64_t left = end - at;
  if (step > 0 && step <= per) part = {static_cast<int>(1 + (steps - step + per - 1) / per), s, head, tile * kRows};
  if (threadIdx.x == 0) a.part[group] = part;

  while (true) {
    const int stop = steps - step <= left ? steps : step + static_cast<int>(left);
    const int row0 = tile * kRows, tokens = plan.end(q, tile);
    i4 qf[NQ][kChunks];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const int row = row0 + 16 * n + i, token = row / a.group;
      const char* from = a.q + static_cast<int64_t>(q.d.begin + token) * a.q_token_bytes +
                         static_cast<int64_t>(head * a.group + row - token * a.group) * a.q_head_bytes;
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        qf[n][j] = i4{0, 0, 0, 0};
        if (row < q.rows && quad + 4 * j < vecs) qf[n][j] = *reinterpret_cast<const i4*>(from + (quad + 4 * j) * 16);
      }
    }
    f4 o[NQ][kTiles];
    float m[NQ], l[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      m[n] = -INFINITY;
      l[n] = 0;
#pragma unroll
      for (int d = 0; d < kTiles; ++d) o[n][d] = f4{0, 0, 0, 0};
    }

    const int64_t pool = a.layer * c.layer_bytes + head * c.head_bytes;
    // Where the tokens of the lane lie, -1: nowhere.
    auto places = [&](int base, int64_t(&place)[kSub]) {
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        const int t = base + 16 * u + i;
        place[u] = -1;
        if (t < tokens) {
          const int page = page_at(c, s, t >> c.shift);
          if (page >= 0) place[u] = page * c.page_bytes + (t & ((1 << c.shift) - 1)) * c.slot_bytes;
        }
      }
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
    // 16 bytes `chunk` of V of a token lie where the reads of four tokens by 16 lanes and the writes of eight tokens by eight lanes
    // both meet all banks.
    auto swizzled = [&](int token, int chunk) {
      const int turn = kVecs % 16 == 0 ? (token & 7) << 1 : (token >> 1 & 3) << 1;
      return token * ROW_BYTES + (chunk ^ turn) * 16;
    };

    char* mine = area[wave];
    int64_t place[kSub], ahead[kSub];
    i4 k[kSub][kChunks], v[kSub][kChunks];
    int base = (step * kWaves + wave) * kTokens;
    const int limit = stop * kWaves * kTokens < tokens ? stop * kWaves * kTokens : tokens;
    if (base < limit) {
      places(base, place);
      load(c.K, place, k);
      load(c.V, place, v);
      places(base + kWaves * kTokens, ahead);
    }
    for (; base < limit; base += kWaves * kTokens) {
      if (!FULL)
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
          for (int j = 0; j < kChunks; ++j)
            if (quad + 4 * j >= vecs) k[u][j] = i4{0, 0, 0, 0};
      f4 z[kSub][NQ];
#pragma unroll
      for (int u = 0; u < kSub; ++u)
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          z[u][n] = f4{0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < kChunks; ++j) z[u][n] = multiply<T>(k[u][j], qf[n][j], z[u][n]);
        }
      load(c.K, ahead, k);

      // tokens of the wave that are there, and those that each row sees
      uint32_t there = 0, bad = 0, sight[NQ];
#pragma unroll
      for (int u = 0; u < kSub; ++u) there |= static_cast<uint32_t>(__ballot(place[u] >= 0) & 0xffff) << (16 * u);
      const bool all = base + kTokens <= q.context && there == low_bits(kTokens);
      if (!all) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          const int row = row0 + 16 * n + i, token = row / a.group;
          uint32_t bits = low_bits(q.context - base);
          if (row >= q.rows) {
            bits = 0;
          } else if (!a.tree.pos) {
            bits = low_bits(q.context + token + 1 - base);
          } else if (base + kTokens > q.context) {
            const int r = q.d.begin + token, e1 = pattern_end(a.tree, r);
            for (int e = pattern_begin(a.tree, r) + quad; e < e1; e += 4) {
              const int j = a.tree.crd[e];
              if (j >= 0 && j < q.d.count) {
                const int b = q.context + j - base;
                if (b >= 0 && b < kTokens) bits |= 1u << b;
              }
            }
          }
          bits |= __shfl_xor(bits, 16);
          bits |= __shfl_xor(bits, 32);
          sight[n] = bits & there;
        }
        // V of drafted tokens that some rows see and others do not: nothing but finite values may be multiplied by 0
        if (base + kTokens > q.context) {
#pragma unroll
          for (int u = 0; u < kSub; ++u) {
            bool odd = false;
#pragma unroll
            for (int j = 0; j < kChunks; ++j) odd |= any_not_finite<T>(v[u][j]);
            const uint64_t b = __ballot(odd);
            const uint32_t rows = (b | b >> 16 | b >> 32 | b >> 48) & 0xffff;
            bad |= rows << (16 * u);
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
        for (int j = 0; j < kChunks; ++j) *reinterpret_cast<i4*>(mine + swizzled(16 * u + i, quad + 4 * j)) = v[u][j];
      int64_t here[kSub];
#pragma unroll
      for (int u = 0; u < kSub; ++u) here[u] = place[u];
      load(c.V, ahead, v);
#pragma unroll
      for (int u = 0; u < kSub; ++u) place[u] = ahead[u];
      places(base + 2 * kWaves * kTokens, ahead);

#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        float top = m[n];
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            z[u][n][r] *= a.scale;
            if (!all && !(sight[n] >> (16 * u + 4 * quad + r) & 1)) z[u][n][r] = -INFINITY;
            top = fmaxf(top, z[u][n][r]);
          }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float zero = top == -INFINITY ? 0 : top;
        if (__any(top != m[n])) {
          const float keep = exp2_of(m[n] - zero);
          l[n] *= keep;
#pragma unroll
          for (int d = 0; d < kTiles; ++d) o[n][d] *= keep;
          m[n] = top;
        }
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            z[u][n][r] = exp2_of(z[u][n][r] - zero);
            l[n] += z[u][n][r];
          }
      }
      i4 p[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        if constexpr (sizeof(T) == 4) {
          p[n] = __builtin_bit_cast(i4, z[0][n]);
        } else {
          // the weights are rounded to the values' type, which the matrix instruction takes: half a step of it (2^-9 or 2^-12 of a
          // weight), as large as the rounding of the result; their sum l is not rounded
          T w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = from_float<T>(z[e >> 2][n][e & 3]);
          p[n] = __builtin_bit_cast(i4, w);
        }
      }
      wave_lds_order();
#pragma unroll
      for (int d = 0; d < kTiles; ++d) {
        i4 vf;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int e = 0; e < 4; ++e) vf[e] = *reinterpret_cast<const int*>(mine + swizzled(4 * quad + e, 4 * d + (i >> 2)) + (i & 3) * 4);
        } else {
          s4 half[2];
#pragma unroll
          for (int u = 0; u < 2; ++u)
            half[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (LdsQuad*)(mine + swizzled(16 * u + 4 * quad + (i >> 2), 2 * d + (i >> 1 & 1)) + (i & 1) * 8));
          vf = __builtin_bit_cast(i4, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n) o[n][d] = multiply<T>(vf, p[n], o[n][d]);
      }
      wave_lds_order();
      while (bad) {  // rows of V with infinities or NaNs, for the rows that see them
        const int b = __builtin_ctz(bad);
        bad &= bad - 1;
        int64_t where = 0;
        float w[NQ];
#pragma unroll
        for (int u = 0; u < kSub; ++u)
          if ((b >> 4) == u) {
            where = __shfl(static_cast<long long>(here[u]), b & 15);
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if ((b & 3) == r) w[n] = __shfl(z[u][n][r], (b & 12) * 4 + i);
          }
#pragma unroll
        for (int d = 0; d < kTiles; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            __builtin_amdgcn_sched_barrier(0);
            const int e = 16 * d + 4 * quad + r;
            if (e >= width) continue;
            const float x = to_float(*reinterpret_cast<const T*>(c.V + pool + where + e * sizeof(T)));
#pragma unroll
            for (int n = 0; n < NQ; ++n)
              if (sight[n] >> b & 1) o[n][d][r] += w[n] * x;
          }
      }
    }

    // the waves meet
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      l[n] += __shfl_xor(l[n], 16);
      l[n] += __shfl_xor(l[n], 32);
      if (quad == 0) stat[0][wave][16 * n + i] = m[n], stat[1][wave][16 * n + i] = l[n];
    }
    __syncthreads();
    const bool whole = step == 0 && stop == steps;
    float* slot = a.partial + static_cast<int64_t>(2 * group + (step == 0)) * kRows * (kWidth + 2);
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
        } else if (row < q.rows) {
          const int token = q.d.begin + row / a.group, h = head * a.group + row % a.group;
          T* to = reinterpret_cast<T*>(a.out + token * a.out_token_bytes + h * a.out_head_bytes) + 4 * e;
#pragma unroll
          for (int b = 0; b < 4; ++b)
            if (4 * e < width) to[b] = from_float<T>(sum == 0 ? 0.0f : y[b] / sum);
          if (e == 0 && a.lse)
            a.lse[static_cast<int64_t>(token) * a.q_heads + h] = sum == 0 ? -INFINITY : (high + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
        }
      }
      __syncthreads();
    }

    left -= stop - step;
    if (left == 0) return;
    step = 0;
    if (++tile == q.tiles) {
      tile = 0;
      if (++head == c.heads) {
        head = 0;
        do q = plan.sequence(++s);
        while (q.tiles == 0);
      }
    }
    steps = plan.steps(q, tile);
  }
}

// Joins the parts of tiles that lie in several workgroups: blockIdx.x is the workgroup that holds a tile's second part, blockIdx.y four
// of the tile's rows; the waves share the parts.
template <class T, int WIDTH, int ROWS>
__global__ void __launch_bounds__(kBlock) attention_join_kernel(Attention a) {
  __shared__ float area[kWaves][4][WIDTH];
  const Part part = a.part[blockIdx.x];
  const Drafted d = part.parts ? drafted(a.first, part.s, a.total) : Drafted{0, 0};
  const int r0 = blockIdx.y * 4, rows = d.count * a.group - part.row - r0;
  if (rows <= 0) return;
  const int lane = lane_id(), wave = wave_id();
  constexpr int64_t kSlot = static_cast<int64_t>(ROWS) * (WIDTH + 2);
  const float* from = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * kSlot;  // part p > 0: slot 0 of workgroup blockIdx.x + p - 1
  auto slot = [&](int p) { return p ? from + (p - 1) * 2 * kSlot : from - kSlot; };
  float top[4], sum[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) top[r] = -INFINITY, sum[r] = 0;
  for (int p = lane; p < part.parts; p += kWave)
#pragma unroll
    for (int r = 0; r < 4; ++r) top[r] = fmaxf(top[r], slot(p)[r0 + r]);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    for (int x = 32; x; x >>= 1) top[r] = fmaxf(top[r], __shfl_xor(top[r], x));
    for (int p = lane; p < part.parts; p += kWave)
      sum[r] += slot(p)[ROWS + r0 + r] * exp2_of(slot(p)[r0 + r] - (top[r] == -INFINITY ? 0 : top[r]));
    for (int x = 32; x; x >>= 1) sum[r] += __shfl_xor(sum[r], x);
  }
  constexpr int kEach = (WIDTH + kWave - 1) / kWave;
  float y[4][kEach] = {};
  for (int p = wave; p < part.parts; p += kWaves) {
    const float* x = slot(p);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float f = exp2_of(x[r0 + r] - (top[r] == -INFINITY ? 0 : top[r]));
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (lane + e * kWave < WIDTH) y[r][e] += f * x[2 * ROWS + (r0 + r) * WIDTH + lane + e * kWave];
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (lane + e * kWave < WIDTH) area[wave][r][lane + e * kWave] = y[r][e];
  __syncthreads();
  if (wave >= rows) return;
  const int row = part.row + r0 + wave, token = d.begin + row / a.group, h = part.head * a.group + row % a.group;
  float total = 0, high = 0;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (r == wave) total = sum[r], high = top[r];
  T* to = reinterpret_cast<T*>(a.out + token * a.out_token_bytes + h * a.out_head_bytes);
  for (int e = lane; e < a.c.width_bytes / static_cast<int>(sizeof(T)); e += kWave) {
    float x = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += area[w][wave][e];
    to[e] = from_float<T>(total == 0 ? 0.0f : x / total);
  }
  if (lane == 0 && a.lse)
    a.lse[static_cast<int64_t>(token) * a.q_heads + h] = total == 0 ? -INFINITY : (high + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
}

template <class T, int ROW_BYTES, int NQ, bool FULL>
void launch(const Attention& a, hipStream_t stream) {
  constexpr int groups = groups_of<ROW_BYTES, sizeof(T)>();
  attention_kernel<T, ROW_BYTES, NQ, FULL><<<groups, kBlock, 0, stream>>>(a);
  attention_join_kernel<T, ROW_BYTES / sizeof(T), 16 * NQ><<<dim3(groups, 4 * NQ), kBlock, 0, stream>>>(a);
}

template <class T, int ROW_BYTES>
void launch_rows(const Attention& a, bool many, hipStream_t stream) {
  if (a.c.width_bytes == ROW_BYTES)
    many ? launch<T, ROW_BYTES, 2, true>(a, stream) : launch<T, ROW_BYTES, 1, true>(a, stream);
  else
    many ? launch<T, ROW_BYTES, 2, false>(a, stream) : launch<T, ROW_BYTES, 1, false>(a, stream);
}

// Heads are padded to the next of 64, 128, 192, 256 values: what a wave multiplies by zeros costs no bytes.
template <class T>
void launch_width(const Attention& a, int width, bool many, hipStream_t stream) {
  if (width <= 64) launch_rows<T, 64 * sizeof(T)>(a, many, stream);
  else if (width <= 128) launch_rows<T, 128 * sizeof(T)>(a, many, stream);
  else if (width <= 192) launch_rows<T, 192 * sizeof(T)>(a, many, stream);
  else launch_rows<T, 256 * sizeof(T)>(a, many, stream);
}

}  // namespace

size_t cache_attention_workspace(const spt_cache* c, int32_t) {
  const size_t width = (c->width + 63) / 64 * 64;
  return align_up(kMostGroups * sizeof(Part), 256) + align_up(static_cast<size_t>(kMostGroups) * 2 * 32 * (width + 2) * sizeof(float), 256);
}

spt_status cache_attention_dispatch(const spt_cache* cache, int32_t layer, const int32_t* first, int32_t total,
                                    const spt_tensor* tree, const void* q, int32_t q_heads, int64_t q_token_stride,
                                    int64_t q_head_stride, float scale, void* out, int64_t out_token_stride, int64_t out_head_stride,
                                    float* lse, void* ws, hipStream_t stream) {
  const int64_t b = value_bytes(cache->dtype);
  Workspace w(ws, cache_attention_workspace(cache, q_heads));
  Part* part = w.take<Part>(kMostGroups);
  float* partial = w.take<float>(0);
  const int group = q_heads / cache->heads;
  const Attention a{cache_view(cache), layer, total, q_heads, group, first, pattern_view(tree), static_cast<const char*>(q),
                    static_cast<char*>(out), lse, q_token_stride * b, q_head_stride * b, out_token_stride * b, out_head_stride * b,
                    scale * 1.4426950408889634f, part, partial};
  const bool many = static_cast<int64_t>(total) * group > static_cast<int64_t>(cache->rows) * 16;
  if (cache->dtype == SPT_F32) launch_width<float>(a, cache->width, many, stream);
  else if (cache->dtype == SPT_F16) launch_width<f16>(a, cache->width, many, stream);
  else launch_width<bf16>(a, cache->width, many, stream);
  SPT_CHECK_LAUNCH("cache_attention");
  return SPT_OK;
}

}  // namespace spt
