// Attention of drafted tokens over the pages of a cache: the kernel for many rows.
//
// The four waves of a workgroup take 16 rows of each 64 of a tile and the same tokens, 64 a step: K and V come to LDS once for all of them, two
// steps' worth of it; the loads of the next step or two are under way, in registers, meanwhile.
// A tree of 16 drafted tokens (64 rows) over 100 000 tokens, 205 MB: 57 us and 9 for the joining; waves wait for half of it. Chunks of 1024
// tokens: 172 us and 17; the matrix units are busy for 28 % of the 172, the vector units for 50 %, LDS for 22 %, of which conflicts are
// less than a thousandth (by counters). Measured without gain: half of the tokens for twice the rows of a wave (reads of LDS halved), the
// next tile's loads under way while one is written, higher priority for waves that multiply.
#include "attention.hpp"

namespace spt {

namespace {

constexpr int kStep = 64;

// NQ: 64 rows times it to a tile. FULL: a head fills ROW_BYTES.
template <class T, int ROW_BYTES, int NQ, bool FULL>
__global__ void __launch_bounds__(kBlock, (groups_of<ROW_BYTES, sizeof(T)>() / 256)) attention_rows_kernel(Attention a) {
  constexpr int kChunks = ROW_BYTES / 64, kWidth = ROW_BYTES / sizeof(T), kTiles = kWidth / 16, kVecs = ROW_BYTES / 16;
  constexpr int kRows = 16 * NQ * kWaves, kGroups = groups_of<ROW_BYTES, sizeof(T)>(), kSub = kStep / 16;
  // Steps in registers on their way to LDS. Two where there is room for them and the loads are what takes the time (few rows).
  constexpr int kDepth = NQ == 1 && ROW_BYTES <= 256 ? 2 : 1;
  constexpr int kLoads = kStep * kVecs / kBlock, kTokensApart = kBlock / kVecs;  // of a thread: 16 bytes of tokens so far apart
  using P = Plan<kRows, kStep>;
  __shared__ __attribute__((aligned(16))) char area[2][2][kStep * ROW_BYTES];  // K and V of two steps
  __shared__ uint32_t absent[3][2], bad[3][2];  // bits of the tokens of a step that are not there, that hold values not finite
  const Cache& c = a.c;
  const int group = xcd_contiguous_block_id(), lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), i = lane & 15,
            quad = lane >> 4, vecs = c.width_bytes / 16, width = c.width_bytes / sizeof(T);
  const int chunk = threadIdx.x % kVecs, token0 = threadIdx.x / kVecs, chunk_read = FULL || chunk < vecs ? chunk : vecs - 1;
  Walk<P> at{{a}};
  if (!at.start(group, kGroups)) return;

  do {
    const int row0 = at.tile * kRows, tokens = at.plan.end(at.q, at.tile), common = at.plan.common(at.q, row0);
    const int mine = wave * 16;  // rows mine + 64 n + i of the tile
    const int64_t pool = a.layer * c.layer_bytes + at.head * c.head_bytes;
    int entry[kLoads];         // of the table, for the step behind those that are loaded
    uint32_t missing[kDepth];  // of each loaded step, bit x: token x is nowhere
    i4 k[kDepth][kLoads], v[kDepth][kLoads];
    auto entries = [&](int base) {
#pragma unroll
      for (int x = 0; x < kLoads; ++x) entry[x] = table_entry(c, at.s, base + token0 + x * kTokensApart, tokens);
    };
    // As in the kernel for few rows: the pool's first slot for tokens that are nowhere.
    auto load = [&](int base, int stage) {
      missing[stage] = 0;
#pragma unroll
      for (int x = 0; x < kLoads; ++x) {
        const int t = base + token0 + x * kTokensApart;
        const bool there = t < tokens && static_cast<unsigned>(entry[x]) < static_cast<unsigned>(c.pages);
        const uint64_t page = there ? entry[x] : 0, slot = there ? t & ((1 << c.shift) - 1) : 0;
        const int64_t place = static_cast<int64_t>((page * c.page_vecs + slot * c.slot_vecs + chunk_read) << 4) + pool;
        missing[stage] |= there ? 0 : 1u << x;
        k[stage][x] = *reinterpret_cast<const i4*>(c.K + place);
        v[stage][x] = *reinterpret_cast<const i4*>(c.V + place);
      }
    };
    // To LDS, with what the step's flags have to say of these tokens.
    auto store = [&](int base, int buffer, int flag, int stage) {
      if (__any(missing[stage] != 0))
#pragma unroll
        for (int x = 0; x < kLoads; ++x)
          if (missing[stage] >> x & 1) {
            const int t = token0 + x * kTokensApart;
            if (chunk == 0) atomicOr(&absent[flag][t >> 5], 1u << (t & 31));
            v[stage][x] = i4{0, 0, 0, 0};
          }
      if (base + kStep > common)
#pragma unroll
        for (int x = 0; x < kLoads; ++x) {
          const int t = token0 + x * kTokensApart;
          if (any_not_finite<T>(v[stage][x])) atomicOr(&bad[flag][t >> 5], 1u << (t & 31));
        }
#pragma unroll
      for (int x = 0; x < kLoads; ++x) {
        const int to = swizzled<ROW_BYTES>(token0 + x * kTokensApart, chunk);
        if (!FULL && chunk >= vecs) k[stage][x] = i4{0, 0, 0, 0};
        *reinterpret_cast<i4*>(area[0][buffer] + to) = k[stage][x];
        *reinterpret_cast<i4*>(area[1][buffer] + to) = v[stage][x];
      }
    };

    i4 qf[NQ][kChunks];
    if (threadIdx.x < 6) (&absent[0][0])[threadIdx.x] = 0, (&bad[0][0])[threadIdx.x] = 0;
    const int base0 = at.step * kStep, limit = tokens > 0 ? at.stop * kStep : base0;
    if (base0 < limit) {
      entries(base0);
      load_queries<64>(a, at.q, at.head, row0 + mine, qf);
      load(base0, 0);
      entries(base0 + kStep);
      __syncthreads();
      store(base0, 0, 0, 0);
#pragma unroll
      for (int d = 1; d <= kDepth; ++d) {
        load(base0 + d * kStep, d % kDepth);
        entries(base0 + (d + 1) * kStep);
      }
      lds_barrier();
    }
    finish_queries<T, FULL>(a, qf);
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
    int flag = 0, buffer = 0;
    for (int base = base0; base < limit;)
#pragma unroll
      for (int stage = 0; stage < kDepth; ++stage) {
        if (stage && base >= limit) break;
        const int next_flag = flag == 2 ? 0 : flag + 1, free_flag = next_flag == 2 ? 0 : next_flag + 1;
        const uint32_t gone[2] = {absent[flag][0], absent[flag][1]};
        uint32_t odd[2] = {bad[flag][0], bad[flag][1]};
        if (threadIdx.x < 2) absent[free_flag][threadIdx.x] = 0, bad[free_flag][threadIdx.x] = 0;  // read a step ago, written to in the next
        if (odd[0] | odd[1]) {
          for (int x = threadIdx.x; x < kStep * kVecs; x += kBlock)
            if (odd[x / kVecs >> 5] >> (x / kVecs & 31) & 1)
              *reinterpret_cast<i4*>(area[1][buffer] + swizzled<ROW_BYTES>(x / kVecs, x % kVecs)) = i4{0, 0, 0, 0};
          lds_barrier();
        }
        f4 z[NQ][kSub];
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
#pragma unroll
          for (int n = 0; n < NQ; ++n) z[n][u] = f4{0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < kChunks; ++j) {
            const i4 kf = *reinterpret_cast<const i4*>(area[0][buffer] + swizzled<ROW_BYTES>(16 * u + i, quad + 4 * j));
#pragma unroll
            for (int n = 0; n < NQ; ++n) z[n][u] = multiply<T>(kf, qf[n][j], z[n][u]);
          }
        }
        if (base + kStep < limit) {
          store(base + kStep, buffer ^ 1, next_flag, (stage + 1) % kDepth);
          load(base + (kDepth + 1) * kStep, (stage + 1) % kDepth);
          entries(base + (kDepth + 2) * kStep);
        }
        const bool all = base + kStep <= common && (gone[0] | gone[1]) == 0;
        uint32_t sight[NQ][2];
        if (!all)
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
#pragma unroll
            for (int w = 0; w < 2; ++w) sight[n][w] = row_sight(a, at.q, row0 + mine + 64 * n + i, base + 32 * w) & ~gone[w];
            hide(z[n], sight[n]);
          }
        softmax_step<T>(z, a.scale, m, l, o, vast);
        i4 p[NQ][kSub / 2];
#pragma unroll
        for (int w = 0; w < kSub / 2; ++w)
#pragma unroll
          for (int n = 0; n < NQ; ++n) p[n][w] = weights<T>(&z[n][2 * w]);
#pragma unroll
        for (int w = 0; w < kSub / 2; ++w)
#pragma unroll
          for (int d = 0; d < kTiles; ++d) {
            const i4 vf = turned_values<T, ROW_BYTES>(area[1][buffer], 32 * w, d);
#pragma unroll
            for (int n = 0; n < NQ; ++n) o[n][d] = multiply<T>(vf, p[n][w], o[n][d]);
          }
#pragma unroll
        for (int w = 0; w < 2; ++w)
          while (odd[w]) {
            const int b = __builtin_ctz(odd[w]), t = base + 32 * w + b, where = page_at(c, at.s, t >> c.shift);
            odd[w] &= odd[w] - 1;
            if (where < 0) continue;
            const char* value = c.V + pool + where * c.page_bytes + (t & ((1 << c.shift) - 1)) * c.slot_bytes;
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
              float weight = 0;
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if ((b >> 4) * 4 + (b & 3) == e) weight = __shfl(z[n][2 * w + (e >> 2)][e & 3], (b & 12) * 4 + i);
              add_token<T>(value, width, sight[n][w] >> b & 1, weight, o[n]);
            }
          }
        lds_barrier();
        flag = next_flag;
        buffer ^= 1;
        base += kStep;
      }

    const bool whole = at.step == 0 && at.stop == at.steps;
    float* slot = a.partial + static_cast<int64_t>(2 * group + (at.step == 0)) * kRows * (kWidth + 2);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      l[n] = sum_of_row(l[n]);
      const int in_tile = mine + 64 * n + i, row = row0 + in_tile;
      if (row >= at.q.rows) continue;
      if (!whole) {
#pragma unroll
        for (int d = 0; d < kTiles; ++d)
          *reinterpret_cast<f4*>(slot + 2 * kRows + static_cast<int64_t>(in_tile) * kWidth + 16 * d + 4 * quad) = o[n][d];
        if (quad == 0) slot[in_tile] = m[n], slot[kRows + in_tile] = l[n];
        continue;
      }
      const int token = at.q.d.begin + row / a.by_group, h = at.head * a.group + row - (token - at.q.d.begin) * a.group;
      T* to = reinterpret_cast<T*>(a.out + token * a.out_token_bytes + h * a.out_head_bytes);
      const float f = l[n] == 0 ? 0 : 1 / l[n];
#pragma unroll
      for (int d = 0; d < kTiles; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (16 * d + 4 * quad < width) to[16 * d + 4 * quad + r] = from_float<T>(l[n] == 0 ? 0.0f : o[n][d][r] * f);
      if (quad == 0 && a.lse) a.lse[static_cast<int64_t>(token) * a.q_heads + h] = natural_lse(m[n], l[n]);
    }
  } while (at.next());
}

template <class T, int ROW_BYTES, int NQ>
void launch(const Attention& a, hipStream_t stream) {
  constexpr int groups = groups_of<ROW_BYTES, sizeof(T)>();
  if (a.c.width_bytes == ROW_BYTES)
    attention_rows_kernel<T, ROW_BYTES, NQ, true><<<groups, kBlock, 0, stream>>>(a);
  else
    attention_rows_kernel<T, ROW_BYTES, NQ, false><<<groups, kBlock, 0, stream>>>(a);
  launch_join<T>(a, groups, 64 * NQ, ROW_BYTES / sizeof(T), stream);
}

}  // namespace

// most: tiles of 128 rows, but where a head has more than 128 values.
template <class T>
void launch_many_rows(const Attention& a, bool most, hipStream_t stream) {
  const int width = a.c.width_bytes / sizeof(T);
  if (width <= 64) most ? launch<T, 128, 2>(a, stream) : launch<T, 128, 1>(a, stream);
  else if (width <= 128) most ? launch<T, 256, 2>(a, stream) : launch<T, 256, 1>(a, stream);
  else launch<T, 512, 1>(a, stream);
}
template void launch_many_rows<f16>(const Attention&, bool, hipStream_t);
template void launch_many_rows<bf16>(const Attention&, bool, hipStream_t);

}  // namespace spt
