// Attention of drafted tokens over the pages of a cache: what its kernels share.
//
// A tile is up to 16, 32, 64 or 128 rows (drafted token, query head) of one sequence that share a head of K and V; rows run token by token, the
// heads of a group side by side. A tile goes through its tokens in steps, once, with the running maximum m and sum l of the softmax:
//   z = scale log2(e) K Q^T,  m' = max(m, z),  P = exp2(z - m'),  l = l exp2(m - m') + sum P,  O^T = O^T exp2(m - m') + V^T P.
// Both products are matrix instructions of 16 x 16 with the tokens as rows of the first result and as the inner dimension of the
// second: a lane then holds, for one row, the tokens 4q .. 4q+3 of each 16 (q = lane / 16), and since the order of an inner dimension
// is free, its P is the operand of the second product as it stands. V is turned round on its way out of LDS.
//
// The work of a call is all steps of all tiles, a number that only the device knows (lengths change between calls of one captured
// graph). Each workgroup of a fixed grid finds its equal share of it from len and first: a range of steps that may begin and end
// within a tile. A tile that lies in one workgroup goes to `out` at once; one that does not leaves m, l and O of each part in the
// workspace, at most two parts a workgroup, and a second kernel joins them. 512 workgroups, all that run at once: 1024, to even out
// which of them end first, took 4 % longer on a decoding batch and 30 % longer on trees, each having its own start and parts.
//
// What bounds it: the reading of K and V, up to some 250 rows a sequence (1.33 GB of a decoding batch of 64 rows: 265 us and 5 for the
// joining, 4.9 TB/s, what a large copy reaches), the matrix products and the softmax beyond (chunks of 1024 tokens: 579 TFLOP/s, half of a
// large matrix product's), and in small calls the way to the first load: some 8 us in a workgroup, 4 for the joining.
#pragma once
#include "cache.hpp"
#include "values.hpp"

namespace spt {

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

// The tile within which a workgroup began, for the joining kernel.
struct Part {
  int parts;  // of the tile; 0: the workgroup began with a tile
  int place;  // its part is number place + 1
  int s, head, row;
};

struct Attention {
  Cache c;
  int layer, total, q_heads, group;
  Divisor by_group;
  const int32_t* first;
  Pattern tree;  // pos NULL: each token sees those up to itself
  const char* q;
  char* out;
  float* lse;
  int64_t q_token_bytes, q_head_bytes, out_token_bytes, out_head_bytes;
  float scale;  // times log2(e), positive: its sign is in the queries
  bool negative;
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
  static constexpr int kRows = ROWS;
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
    const int e = q.context + last / a.by_group + 1;
    return e > 0 ? e : 0;
  }
  // Tokens that every row from `row` on sees.
  __device__ __forceinline__ int common(const Sequence& q, int row) const {
    return a.tree.pos ? q.context : q.context + row / a.by_group + 1;
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

__device__ __forceinline__ int64_t lane_value(int64_t v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(v), lane), hi = __builtin_amdgcn_readlane(static_cast<int>(v >> 32), lane);
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// Finds the sequence that the workgroup's share of `groups` (a power of two) begins in; begin and end count the steps within it. False if
// the share is empty. Every wave does all of it, 64 sequences at a time, so that none waits for another.
template <class P>
__device__ __forceinline__ bool share(const P& plan, int group, int groups, int64_t& per, int64_t& begin, int64_t& end, int& s) {
  const int rows = plan.a.c.rows, heads = plan.a.c.heads, lane = lane_id();
  int64_t total = 0, mine = 0, upto = 0;
  auto count = [&](int base) {
    const int r = base + lane;
    mine = r < rows ? plan.head_steps(plan.sequence(r)) * heads : 0;
    upto = mine;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const int64_t o = __shfl_up(static_cast<long long>(upto), d);
      if (lane >= d) upto += o;
    }
    upto += total;
    total = lane_value(upto, kWave - 1);
  };
  for (int base = 0; base < rows; base += kWave) count(base);
  per = (total + groups - 1) >> (31 - __builtin_clz(groups));
  begin = group * per;
  end = begin + per < total ? begin + per : total;
  if (begin >= end) return false;
  total = 0;
  int base = 0;
  if (rows > kWave) {
    count(0);
    while (total <= begin) {
      base += kWave;
      count(base);
    }
  }
  const int found = __builtin_ctzll(__ballot(upto > begin));
  const int64_t skipped = lane_value(upto - mine, found);
  s = base + found;
  begin -= skipped;
  end -= skipped;
  return true;
}

// A workgroup's way through its share: tile by tile, the steps [step, stop) of each.
template <class P>
struct Walk {
  P plan;
  typename P::Sequence q;
  int s, head, tile, step, steps, stop;
  int64_t left;

  // False if the share is empty. Notes in `part` whether the workgroup begins within a tile.
  __device__ __forceinline__ bool start(int group, int groups) {
    int64_t per = 0, at = 0, end = 0;
    const bool some = share(plan, group, groups, per, at, end, s);
    Part part{0, 0, 0, 0, 0};
    if (some) {  // `at` counts the steps of sequence s, head by head and tile by tile
      q = plan.sequence(s);
      const int64_t in_head = plan.head_steps(q);
      head = (at | in_head) >> 32 ? static_cast<int>(at / in_head) : static_cast<int>(static_cast<uint32_t>(at) / static_cast<uint32_t>(in_head));
      tile = 0;
      int64_t rest = at - head * in_head;
      steps = plan.steps(q, 0);
      while (rest >= steps) rest -= steps, steps = plan.steps(q, ++tile);
      step = static_cast<int>(rest);
      left = end - at;
      limit();
      if (step > 0) {
        const int each = per < steps ? static_cast<int>(per) : steps, place = (step - 1) / each;
        part = {1 + (steps - (step - place * each) + each - 1) / each, place, s, head, tile * P::kRows};
      }
    }
    if (threadIdx.x == 0) plan.a.part[group] = part;
    return some;
  }
  __device__ __forceinline__ void limit() { stop = steps - step <= left ? steps : step + static_cast<int>(left); }
  __device__ __forceinline__ bool next() {
    left -= stop - step;
    if (left == 0) return false;
    step = 0;
    if (++tile == q.tiles) {
      tile = 0;
      if (++head == plan.a.c.heads) {
        head = 0;
        do q = plan.sequence(++s);
        while (q.tiles == 0);
      }
    }
    steps = plan.steps(q, tile);
    limit();
    return true;
  }
};

// Rows row0 + APART n + i of a tile, for those behind the last the last one: 16 bytes of a lane from each 64 of the head.
template <int APART, int NQ, int CHUNKS, class Q>
__device__ __forceinline__ void load_queries(const Attention& a, const Q& q, int head, int row0, i4 (&x)[NQ][CHUNKS]) {
  const int i = lane_id() & 15, quad = lane_id() >> 4, vecs = a.c.width_bytes / 16;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = row0 + APART * n + i, row = r < q.rows ? r : q.rows - 1, token = row / a.by_group;
    const char* from = a.q + (q.d.begin + token) * a.q_token_bytes + (head * a.group + row - token * a.group) * a.q_head_bytes;
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
      const int chunk = quad + 4 * j;
      x[n][j] = *reinterpret_cast<const i4*>(from + (chunk < vecs ? chunk : vecs - 1) * 16);
    }
  }
}
// Before they are used: zeros behind the width, and the sign of the scale.
template <class T, bool FULL, int NQ, int CHUNKS>
__device__ __forceinline__ void finish_queries(const Attention& a, i4 (&x)[NQ][CHUNKS]) {
  const int quad = lane_id() >> 4, vecs = a.c.width_bytes / 16;
#pragma unroll
  for (int n = 0; n < NQ; ++n)
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
      if (!FULL && quad + 4 * j >= vecs) x[n][j] = i4{0, 0, 0, 0};
      if (a.negative) x[n][j] ^= sizeof(T) == 4 ? static_cast<int>(0x80000000u) : static_cast<int>(0x80008000u);
    }
}

// The table's entry for token t of row s, whatever it holds; a token behind the last takes the last one's.
__device__ __forceinline__ int table_entry(const Cache& c, int s, int t, int tokens) {
  return c.table[static_cast<int64_t>(s) * c.row_pages + ((t < tokens ? t : tokens - 1) >> c.shift)];
}
// With it, once it has arrived: where the token's slot begins, -1 if it is nowhere.
__device__ __forceinline__ int64_t slot_of(const Cache& c, int entry, int t, int tokens) {
  if (t >= tokens || static_cast<unsigned>(entry) >= static_cast<unsigned>(c.pages)) return -1;
  return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(entry)) * c.page_vecs +
                              static_cast<uint64_t>(static_cast<uint32_t>(t & ((1 << c.shift) - 1))) * c.slot_vecs) << 4;
}

// Which of the 32 tokens from `base` on a row sees, as bits; the four lanes of a row share the work and get the same. With a pattern a
// row's list is gone through again for each 32 drafted tokens: fine for trees of some 64 (4 sequences of 2500 tokens, 32 query heads,
// bf16: 49 us, 47 without a tree, 52 with a list of half of all), not for hundreds (256: 151, 94, 177; 512: 369, 144, 472).
template <class Q>
__device__ __forceinline__ uint32_t row_sight(const Attention& a, const Q& q, int row, int base) {
  const int quad = lane_id() >> 4, token = row / a.by_group;
  uint32_t bits = low_bits(q.context - base);
  if (row >= q.rows) {
    bits = 0;
  } else if (!a.tree.pos) {
    bits = low_bits(q.context + token + 1 - base);
  } else if (base + 32 > q.context) {
    const int r = q.d.begin + token;
    strided(pattern_begin(a.tree, r), pattern_end(a.tree, r), quad, 4, [&](int e) {
      const int j = a.tree.crd[e];
      if (j >= 0 && j < q.d.count) {
        const int b = q.context + j - base;
        if (b >= 0 && b < 32) bits |= 1u << b;
      }
    });
  }
  bits |= __shfl_xor(bits, 16);
  bits |= __shfl_xor(bits, 32);
  return bits;
}

// 16 bytes `chunk` of a token of K or V lie where reads of four tokens by 16 lanes, reads of eight tokens by eight lanes and writes
// alike meet all banks.
template <int ROW_BYTES>
__device__ __forceinline__ int swizzled(int token, int chunk) {
  const int turn = ROW_BYTES % 256 == 0 ? (token & 7) << 1 : (token >> 1 & 3) << 1;
  return token * ROW_BYTES + (chunk ^ turn) * 16;
}

// V^T of 16 values of the head and 64 bytes' worth of tokens (32, or 16 of float32), out of LDS.
template <class T, int ROW_BYTES>
__device__ __forceinline__ i4 turned_values(char* area, int token, int d) {
  const int i = lane_id() & 15, quad = lane_id() >> 4;
  if constexpr (sizeof(T) == 4) {
    i4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const int*>(area + swizzled<ROW_BYTES>(token + 4 * quad + e, 4 * d + (i >> 2)) + (i & 3) * 4);
    return v;
  } else {
    s4 half[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
      half[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (LdsQuad*)(area + swizzled<ROW_BYTES>(token + 16 * u + 4 * quad + (i >> 2), 2 * d + (i >> 1 & 1)) + (i & 1) * 8));
    return __builtin_bit_cast(i4, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
}

// Scores of tokens that a row does not see become -infinity. seen: bits of 32 tokens each.
template <int SUB>
__device__ __forceinline__ void hide(f4 (&z)[SUB], const uint32_t* seen) {
  const int quad = lane_id() >> 4;
#pragma unroll
  for (int u = 0; u < SUB; ++u)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (!(seen[u / 2] >> (16 * (u & 1) + 4 * quad + r) & 1)) z[u][r] = -INFINITY;
}

// The largest, and the sum, over the four lanes that hold a row (lane, lane ^ 16, lane ^ 32, lane ^ 48): swapping the odd rows of 16
// lanes of one register with the even rows of another leaves both neighbours' values in the two.
__device__ __forceinline__ float max_of_row(float x) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float sum_of_row(float x) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// One step of the softmax of 16 rows each: scores z (16 tokens each, 4q .. 4q+3 of a lane) become weights exp2(scale z - m). What is
// held so far is rescaled, and m raised, only when a weight would pass 2^kMost: most steps leave it, and m cancels in the result. It is
// raised to 2^kBelow below the largest weight. scale > 0.
// f16 holds 2^16, and below 2^-14 with fewer bits, below 2^-25 nothing, while the sum l keeps all: the largest weights lie between 2^11
// and 2^15, so that only those less than 2^-25 of them lose bits. What is lost of a token is less than 2^-36 of the largest weight,
// all together less than half a step of f16 in rows of 2^25 tokens whose values are alike. (With a largest weight of 1, tokens of 2^-26
// were lost altogether, those of 2^-20 off by up to 3 %.) The other types have the range of 32 bits.
template <class T>
struct Weights {
  static constexpr float kBelow = __is_same(T, f16) ? 11 : 0, kMost = __is_same(T, f16) ? 15 : 8;
};
// A weight's exponent is rounded once, in an fma; m is a product that was rounded before. From 2^22 on that rounding is no longer small (at
// 2^30 the largest weight could be 2^64 as well as 2^-64), and m - kBelow not what it says: once an m is so large (vast, alike in all
// lanes) the products are rounded in the exponents too, so that the largest is 0.
constexpr float kVast = 1 << 22;
template <class T, int COUNT, int NQ, int SUB, int TILES>
__device__ __forceinline__ void softmax_step(f4 (&z)[COUNT][SUB], float scale, float (&m)[NQ], float (&l)[NQ], f4 (&o)[NQ][TILES], bool& vast) {
  const float most = vast ? 0 : Weights<T>::kMost;  // which the sum with a vast m would round
  float top[COUNT];
  bool grown = false;
#pragma unroll
  for (int n = 0; n < COUNT; ++n) {
    top[n] = z[n][0][0];
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) top[n] = fmaxf(top[n], z[n][u][r]);
    top[n] = max_of_row(top[n]) * scale;
    grown |= top[n] > m[n] + most;
  }
  if (__any(grown)) {
    bool large = false;
#pragma unroll
    for (int n = 0; n < COUNT; ++n) {
      const float below = fabsf(top[n]) < kVast ? Weights<T>::kBelow : 0;
      const float high = fmaxf(m[n], top[n] - below), keep = exp2_of(m[n] - (high == -INFINITY ? 0 : high));
      l[n] *= keep;
#pragma unroll
      for (int d = 0; d < TILES; ++d) o[n][d] *= keep;
      m[n] = high;
      large |= fabsf(high) >= kVast && high != -INFINITY;
    }
    vast |= __any(large) != 0;
  }
  if (vast) {  // here, rounded (no fma of it and the difference below), with a scale of 1 below
#pragma clang fp contract(off)
#pragma unroll
    for (int n = 0; n < COUNT; ++n)
#pragma unroll
      for (int u = 0; u < SUB; ++u) z[n][u] *= scale;
    scale = 1;
  }
#pragma unroll
  for (int n = 0; n < COUNT; ++n) {
    const float zero = m[n] == -INFINITY ? 0 : m[n];
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        z[n][u][r] = exp2_of(__builtin_fmaf(z[n][u][r], scale, -zero));
        l[n] += z[n][u][r];
      }
  }
}

// The weights of 32 tokens (16 of float32) as an operand. They are rounded to the values' type, which the matrix instruction takes:
// off by at most half a step of it (2^-8 of a weight in bf16, 2^-11 in f16), as the result is; their sum l is not rounded.
template <class T>
__device__ __forceinline__ i4 weights(const f4* z) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(i4, z[0]);
  } else {
    typedef T t8 __attribute__((ext_vector_type(8)));
    t8 w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = from_float<T>(z[e >> 2][e & 3]);
    return __builtin_bit_cast(i4, w);
  }
}

// What a matrix instruction cannot do: a value of V that is not finite is to reach the rows that see its token and no others. Such tokens
// are zeros in LDS; here their values are added one by one. w: the weight of the lane's row.
template <class T, int TILES>
__device__ __forceinline__ void add_token(const char* value, int width, bool seen, float w, f4 (&o)[TILES]) {
  const int quad = lane_id() >> 4;
#pragma unroll
  for (int d = 0; d < TILES; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int e = 16 * d + 4 * quad + r;
      if (e < width && seen) o[d][r] += w * to_float(reinterpret_cast<const T*>(value)[e]);
    }
}

__device__ __forceinline__ float natural_lse(float m, float l) {
  return l == 0 ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// The kernel for many rows (its own translation unit).
template <class T>
void launch_many_rows(const Attention& a, bool most, hipStream_t stream);
// Joins the parts that kernels with tiles of `rows` rows and heads padded to `width` values left.
template <class T>
void launch_join(const Attention& a, int groups, int rows, int width, hipStream_t stream);

}  // namespace spt
