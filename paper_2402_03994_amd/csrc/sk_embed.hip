// sk_embed.hip -- embedding lookup and its gradient (C ABI of
// include/sketch_train.h).
//
// Lookup: a wave copies up to 4 KB of a row (64 lanes x 4 vectors of 16
// bytes), so that a row needs no more waves than its bytes ask for and one id
// is read per wave.  Bound by memory: 32768 rows of 4096 bf16, 268 MB out of
// 98 MB of the table, 71 us; one row of 768 fp32 2 us, all of it latency.
//
// Gradient, in three or four launches, without atomics on floats (and in one,
// k_eg_few, for few tokens):
//   k_eg_rank   sorts each run of up to 4096 tokens of a group by (id,
//               position): an entry's place is how many entries are smaller,
//               counted by brute force (64 entries a workgroup against all of
//               the run, 64 comparisons an instruction: their mask's bits are
//               counted in the scalar unit), which takes the whole chip less
//               time than a sort's barriers take one workgroup.
//               The launch's other workgroups zero the gradient meanwhile.
//   k_eg_merge  joins up to 16 sorted runs: an entry's place is its own plus
//               what a binary search in each other run gives, one lane a run.
//   k_eg_sum    a wave adds up R sorted entries for 64 vectors of columns and
//               writes out every id that begins and ends among them; what
//               crosses the cut is written to the workspace (head: the part of
//               an id that began earlier, tail: of one that goes on).
//   k_eg_join   tail + heads of the ids that cross cuts.
// Every sum has a fixed order: the sorted one within R entries, then piece by
// piece.  Bound by writing the gradient (vocab x width per group); to zero all
// of it costs the named rows a second write and spares the others a look-up.
// 8 examples of 1024 tokens, 50257 x 768 fp32 each: 183 us to rank and zero (6.8
// TB/s), 20 us to sum, 5 us to join.
#include <algorithm>
#include <type_traits>

#include "sk_train.h"

using namespace sk;

namespace {

constexpr int kNoId = 0x7FFFFFFE;    // of a masked token: sorts to the end
constexpr int kBeyond = 0x7FFFFFFF;  // beyond a run: above whatever is compared with it
constexpr int kRun = 4096;               // tokens ranked by brute force
constexpr int kMergeRuns = 16;

__device__ __forceinline__ int64_t id_at(const void *ids, int index, int64_t t) {
  return index == SK_I64 ? ((const int64_t *)ids)[t] : ((const int32_t *)ids)[t];
}

// N elements from floats, at an address aligned to one element
template <typename O, int N>
__device__ __forceinline__ void store_n(O *p, const float *f, bool past = false) {
  if (sizeof(O) == 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) Vec<O>::store(p + i, Vec<O>::pack(f + i), past);
  } else if (N == 8) {
    Vec<O>::store(p, Vec<O>::pack(f), past);
  } else {  // four bf16
    struct __attribute__((packed, aligned(2))) Half {
      uint32_t a, b;
    };
    *(Half *)p = Half{bf16_bits(f[0]) | bf16_bits(f[1]) << 16, bf16_bits(f[2]) | bf16_bits(f[3]) << 16};
  }
}

template <typename W, typename O>
__global__ __launch_bounds__(256) void k_embed(const W *__restrict__ w, int64_t vocab, int width, int64_t ld,
                                               const void *__restrict__ ids, int index, int64_t block0,
                                               int64_t n, int pieces, float scale, bool past, O *__restrict__ out) {
  constexpr int N = Vec<W>::N, NV = 4;
  const int64_t job = (block0 + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = job / pieces;
  if (t >= n) return;
  const int lane = threadIdx.x & 63, nv = width / N, v0 = (int)(job % pieces) * 64 * NV + lane;
  const int64_t v = id_at(ids, index, t);
  const bool live = v >= 0 && v < vocab;
  const W *x = w + (live ? v : 0) * ld;
  O *o = out + t * width;
  u32x4 raw[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    raw[k] = u32x4{0, 0, 0, 0};
    if (live && v0 + 64 * k < nv) raw[k] = Vec<W>::load(x + (int64_t)(v0 + 64 * k) * N);
  }
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (v0 + 64 * k < nv) {
      float f[N];
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = scale * Vec<W>::get(raw[k], i);
      store_n<O, N>(o + (int64_t)(v0 + 64 * k) * N, f, past);
    }
  const int c = nv * N + lane;  // the width % N last columns, by the first piece
  if (v0 == lane && c < width) o[c] = from_f32<O>(live ? scale * to_f32(x[c]) : 0.0f);
}

struct Entry {  // a token of its group: id and position
  int id;
  uint32_t pos;
};

// What is to be zeroed: `bytes` bytes, an even number, from an even address on.
struct Zeros {
  char *p;
  int64_t bytes;
};

// 16 bytes a thread, one workgroup after the other: 8 x 50257 x 768 fp32 at 6.8 TB/s, where workgroups that go through
// stretches of their own reach 4 to 5.5.
__device__ __forceinline__ void zero_part(Zeros z, int64_t block, int64_t blocks) {
  int64_t head = (int64_t)((16 - ((uintptr_t)z.p & 15)) & 15);
  head = head < z.bytes ? head : z.bytes;
  const int64_t nv = (z.bytes - head) / 16;
  u32x4 *v = (u32x4 *)(z.p + head);
  for (int64_t i = block * 512 + threadIdx.x; i < nv; i += blocks * 512) v[i] = u32x4{0, 0, 0, 0};
  if (block == 0 && threadIdx.x < 16) {  // up to 7 pairs of bytes on either side
    const int64_t at = threadIdx.x < 8 ? 2 * threadIdx.x : head + nv * 16 + 2 * (threadIdx.x - 8);
    if (at < (threadIdx.x < 8 ? head : z.bytes)) *(uint16_t *)(z.p + at) = 0;
  }
}

// Ranks 64 entries of a run against the whole run, eight waves taking turns at its blocks of 64: workgroup block0 +
// blockIdx.x of rank_blocks that rank and zero_blocks that zero.
__global__ __launch_bounds__(512) void k_eg_rank(const void *__restrict__ ids, int index, int64_t n, int64_t vocab,
                                                 int runs, int tiles, uint32_t block0, uint32_t rank_blocks,
                                                 uint32_t zero_blocks, Entry *__restrict__ sorted, Zeros z) {
  __shared__ int part[8][64];
  const uint32_t block = block0 + blockIdx.x;
  // those that rank come first: dealt out among those that zero they take longer (65536 tokens: 41 us, 48 to 60)
  if (block >= rank_blocks) {
    zero_part(z, block - rank_blocks, zero_blocks);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t run = block / (unsigned)tiles, b = run / runs, p0 = (run % runs) * kRun;
  const int tile = block % (unsigned)tiles, len = (int)(n - p0 < kRun ? n - p0 : kRun);
  if (tile * 64 >= len) return;
  auto key = [&](int i) -> int {
    if (i >= len) return kBeyond;
    const int64_t v = id_at(ids, index, b * n + p0 + i);
    return v >= 0 && v < vocab ? (int)v : kNoId;
  };
  const int mine = key(tile * 64 + lane);
  // The wave's share of the run: blocks wave, wave + 8, ..  Entries of earlier blocks count where they are not above an
  // entry (one less is below it), so that entries of one id stay in order.
  constexpr int kBlocks = kRun / 64 / 8;
  const int blocks = (len + 63) / 64, own = wave == tile % 8;
  int theirs[kBlocks];
#pragma unroll
  for (int k = 0; k < kBlocks; ++k) {
    const int blk = wave + 8 * k;
    theirs[k] = kBeyond;
    if (blk < blocks && blk != tile) theirs[k] = key(blk * 64 + lane) - (blk < tile);
  }
  int count = 0;
  auto rank = [&](auto some) {
#pragma unroll 8
    for (int i = 0; i < 64; ++i) {
      const int m = __builtin_amdgcn_readlane(mine, i);
      int c = 0;
#pragma unroll
      for (int k = 0; k < decltype(some)::value; ++k) c += __builtin_popcountll(__ballot(theirs[k] < m));
      count = lane == i ? c : count;
    }
  };
  if (blocks <= 8)
    rank(std::integral_constant<int, 1>());
  else if (blocks <= 24)
    rank(std::integral_constant<int, 3>());
  else
    rank(std::integral_constant<int, kBlocks>());
  if (own) {  // the tile against itself
#pragma unroll 8
    for (int j = 0; j < 64; ++j) {
      const int k = __builtin_amdgcn_readlane(mine, j);
      count += k < mine || (k == mine && j < lane);
    }
  }
  part[wave][lane] = count;
  __syncthreads();
  if (wave == 0 && tile * 64 + lane < len) {
    int place = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) place += part[i][lane];
    sorted[b * n + p0 + place] = Entry{mine, (uint32_t)(p0 + tile * 64 + lane)};
  }
}

// Sorted runs of `len` entries, 16 at a time: 16 lanes an entry.
__global__ __launch_bounds__(256) void k_eg_merge(const Entry *__restrict__ in, Entry *__restrict__ out, int64_t n,
                                                  int64_t len, int64_t total, uint32_t block0) {
  const int64_t e = ((int64_t)(block0 + blockIdx.x) * 256 + threadIdx.x) / kMergeRuns;
  const int r = threadIdx.x % kMergeRuns;
  if (e >= total) return;  // all 16 lanes of an entry
  const int64_t b = e / n, i = e % n, g0 = i / (len * kMergeRuns) * (len * kMergeRuns);
  const int own = (int)((i - g0) / len);
  const Entry mine = in[e];
  // lower bound in later runs, upper bound in earlier ones: entries of one id stay in order
  const int64_t r0 = g0 + r * len;
  int64_t lo = 0, hi = r0 >= n ? 0 : (n - r0 < len ? n - r0 : len);
  if (r == own) {
    lo = hi = i - r0;
  }
  const Entry *run = in + b * n + r0;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    const int k = run[mid].id;
    if (r < own ? k <= mine.id : k < mine.id)
      lo = mid + 1;
    else
      hi = mid;
  }
  int64_t rank = lo;
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) rank += __shfl_xor(rank, d, 16);
  if (r == 0) out[b * n + g0 + rank] = mine;
}

// the N columns from c on of a row of sums to out or (accumulate) onto it; WHOLE: all of them are in the row
template <typename O, int N, bool WHOLE>
__device__ __forceinline__ void put(O *row, int c, int width, const float *acc, float scale, int accumulate) {
  if (WHOLE || c + N <= width) {
    float f[N];
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = scale * acc[i];
    if (accumulate)
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] += to_f32(row[c + i]);
    store_n<O, N>(row + c, f);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < width) row[c + i] = from_f32<O>(scale * acc[i] + (accumulate ? to_f32(row[c + i]) : 0.0f));
  }
}

// Few tokens (up to 256 TURNS), in one launch: a workgroup owns `rows` rows of a group's gradient, lists the tokens that
// name them, in order, and writes every row, the named ones as the sum of their tokens and the others as zeros.  Bound by
// the frequent ids: a wave adds up eight of an id's tokens at a time.
// WHOLE: every lane has a whole vector of columns; the last lane's of a width that is no multiple of one begin earlier,
// so that a few columns are added up and written twice, with the same values.  That is not for accumulation, where the
// second of two waves would add to the first one's sum.
constexpr int kFewTokens = 1024;
template <typename G, typename O, bool WHOLE, int TURNS>
__global__ __launch_bounds__(256) void k_eg_few(const G *__restrict__ dy, int64_t ld, const void *__restrict__ ids,
                                                int index, int n, int64_t vocab, int width, int rows, int64_t per,
                                                int64_t block0, float scale, int accumulate, O *__restrict__ out) {
  constexpr int N = Vec<G>::N, U = WHOLE ? 8 : 1;
  __shared__ int counts[TURNS * 4];
  __shared__ int list[TURNS * 256];  // (row << 16) | position
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t block = block0 + blockIdx.x, b = block / per, v0 = block % per * rows;
  int row[TURNS];
  uint64_t mask[TURNS];
#pragma unroll
  for (int j = 0; j < TURNS; ++j) {
    const int i = j * 256 + tid;
    const int64_t v = i < n ? id_at(ids, index, b * n + i) : -1;
    // ids outside the vocabulary are not in [v0, v0 + rows) either, but for the last rows'
    row[j] = v >= v0 && v < v0 + rows && v < vocab ? (int)(v - v0) : -1;
    mask[j] = __ballot(row[j] >= 0);
    if (lane == 0) counts[j * 4 + wave] = __builtin_popcountll(mask[j]);
  }
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int q = 0; q < TURNS * 4; ++q) {
    const int j = q / 4;
    if (q % 4 == wave && row[j] >= 0)
      list[total + __builtin_popcountll(mask[j] & ((1ull << lane) - 1))] = row[j] << 16 | (j * 256 + tid);
    total += counts[q];
  }
  __syncthreads();
  const int live = vocab - v0 < rows ? (int)(vocab - v0) : rows;
  if (total == 0) {
    if (accumulate) return;
    O *o = out + (b * vocab + v0) * width;
    const int64_t n0 = (int64_t)live * width, nv = n0 / Vec<O>::N;
    for (int64_t i = tid; i < nv; i += 256) Vec<O>::store(o + i * Vec<O>::N, u32x4{0, 0, 0, 0});
    if (nv * Vec<O>::N + tid < n0) o[nv * Vec<O>::N + tid] = from_f32<O>(0.0f);
    return;
  }
  const int pieces = (width + 64 * N - 1) / (64 * N);
  for (int t = wave; t < live * pieces; t += 4) {
    const int r = t / pieces;
    int c = (t % pieces) * 64 * N + lane * N;
    const bool idle = c >= width;
    if (WHOLE && c + N > width) c = width - N;
    O *o = out + (b * vocab + v0 + r) * width;
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.0f;
    bool named = false;
    for (int q = 0; q < total; q += 64) {
      const int e = q + lane < total ? list[q + lane] : -1;
      uint64_t hit = __ballot(e >= 0 && e >> 16 == r);
      named |= hit != 0;
      while (hit) {
        u32x4 x[U];
        int count = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (!hit) break;
          const int pos = __builtin_amdgcn_readlane(e, __builtin_ctzll(hit)) & 0xFFFF;
          hit &= hit - 1;
          ++count;
          const G *g = dy + (b * n + pos) * ld;
          if (WHOLE) {
            if (!idle) x[u] = Vec<G>::load(g + c);
          } else {
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] += c + i < width ? to_f32(g[c + i]) : 0.0f;
          }
        }
        if (WHOLE)
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (u < count)
#pragma unroll
              for (int i = 0; i < N; ++i) acc[i] += Vec<G>::get(x[u], i);
      }
    }
    if ((named || !accumulate) && !idle) put<O, N, WHOLE>(o, c, width, acc, scale, accumulate);
  }
}

// What the sums work on: groups of n sorted entries, cut into tiles of R, and columns cut into pieces of 64 vectors.
struct Sums {
  const Entry *sorted;
  int64_t n, vocab, ld, tiles;
  int width, pieces, R, accumulate;
  float scale;
  float *head, *tail;  // [batch, tiles, width]
};

// WHOLE as above (65536 x 767 bf16: 34 us, 71 us with the last columns one by one).
template <typename G, typename O, bool WHOLE>
__global__ __launch_bounds__(256) void k_eg_sum(Sums s, uint32_t jobs, const G *__restrict__ dy,
                                                O *__restrict__ out) {
  constexpr int N = Vec<G>::N, U = WHOLE ? 16 : 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t job = blockIdx.x * 4 + wave;
  if (job >= jobs) return;
  const uint32_t bt = job / (uint32_t)s.pieces, b = bt / (uint32_t)s.tiles, tile = bt % (uint32_t)s.tiles;
  const int64_t e0 = (int64_t)tile * s.R;
  int c = (int)(job % (uint32_t)s.pieces) * 64 * N + lane * N;
  const bool idle = c >= s.width;
  if (WHOLE && c + N > s.width) c = s.width - N;
  const Entry *k = s.sorted + b * s.n;
  Entry e{kNoId, 0};
  if (lane < s.R && e0 + lane < s.n) e = k[e0 + lane];
  const int before = e0 > 0 ? k[e0 - 1].id : kNoId, after = e0 + s.R < s.n ? k[e0 + s.R].id : kNoId;
  float acc[N];
  int cur = kNoId;
  bool began = true;
  O *const o = out + b * s.vocab * s.width;
  auto flush = [&](bool ends) {
    if (cur == kNoId || idle) return;
    if (began && ends) {
      put<O, N, WHOLE>(o + (int64_t)cur * s.width, c, s.width, acc, s.scale, s.accumulate);
    } else {
      float *part = (began ? s.tail : s.head) + (int64_t)bt * s.width + c;
      if (WHOLE) {
#pragma unroll
        for (int i = 0; i < N; i += 4) Vec<float>::store(part + i, Vec<float>::pack(acc + i));
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (c + i < s.width) part[i] = acc[i];
      }
    }
  };
  for (int i0 = 0; i0 < s.R; i0 += U) {
    u32x4 x[U];
    float y[WHOLE ? 1 : U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int id = __builtin_amdgcn_readlane(e.id, i0 + u);
      const uint32_t pos = (uint32_t)__builtin_amdgcn_readlane((int)e.pos, i0 + u);
      if (id == kNoId) continue;  // the rest of the tile is empty
      const G *row = dy + (b * s.n + pos) * s.ld;
      if (WHOLE) {
        if (!idle) x[u] = Vec<G>::load(row + c);
      } else if (c + N <= s.width) {
        const u32x4 v = Vec<G>::load(row + c);
#pragma unroll
        for (int i = 0; i < N; ++i) y[u][i] = Vec<G>::get(v, i);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) y[u][i] = c + i < s.width ? to_f32(row[c + i]) : 0.0f;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int id = __builtin_amdgcn_readlane(e.id, i0 + u);
      if (id == kNoId) continue;
      if (id != cur) {
        flush(true);
        began = i0 + u > 0 || before != id;
        cur = id;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] += WHOLE ? Vec<G>::get(x[u], i) : y[WHOLE ? 0 : u][i];
    }
  }
  flush(after != cur);
}

// An id that begins in a tile and goes on: its tail there and the heads of the tiles that follow, four waves in turn.
template <typename O>
__global__ __launch_bounds__(256) void k_eg_join(Sums s, O *__restrict__ out) {
  constexpr int N = 4;
  __shared__ float part[3][64 * N];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pieces = (s.width + 64 * N - 1) / (64 * N);
  const int64_t bt = blockIdx.x / (unsigned)pieces, b = bt / s.tiles, tile = bt % s.tiles, e1 = (tile + 1) * s.R;
  if (e1 >= s.n) return;
  const Entry *k = s.sorted + b * s.n;
  // all at once: most workgroups only wait for these
  const int id = k[e1 - 1].id, next = k[e1].id, first = k[e1 - s.R].id, before = e1 > s.R ? k[e1 - s.R - 1].id : kNoId;
  if (id == kNoId || next != id || (first == id && before == id)) return;  // ends here, or began earlier
  int64_t heads = 0;
  for (;;) {
    const int64_t at = e1 + (heads + lane) * s.R;
    const uint64_t no = ~__ballot(at < s.n && k[at].id == id);
    if (no) {
      heads += __builtin_ctzll(no);
      break;
    }
    heads += 64;
  }
  const int c = (int)(blockIdx.x % (unsigned)pieces) * 64 * N + lane * N;
  float acc[N] = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](const float *row) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < s.width) acc[i] += row[c + i];
  };
  if (wave == 0) add(s.tail + bt * s.width);
  const float *head = s.head + (bt + 1) * s.width;
  int64_t h = wave;
  for (; h + 28 < heads; h += 32) {  // eight loads at a time: a frequent id has hundreds of heads
    float x[8][N];
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i) x[u][i] = c + i < s.width ? head[(h + 4 * u) * s.width + c + i] : 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] += x[u][i];
  }
  for (; h < heads; h += 4) add(head + h * s.width);
  if (wave)
#pragma unroll
    for (int i = 0; i < N; ++i) part[wave - 1][lane * N + i] = acc[i];
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] += part[w][lane * N + i];
  if (c < s.width) put<O, N, false>(out + (b * s.vocab + id) * s.width, c, s.width, acc, s.scale, s.accumulate);
}

template <typename W, typename O>
void run_embed(const void *w, int64_t vocab, int64_t width, int64_t ld, const void *ids, int index, int64_t n,
               float scale, void *out, hipStream_t st) {
  const int64_t pieces = std::max<int64_t>(1, (width / Vec<W>::N + 255) / 256);
  grid_parts((n * pieces + 3) / 4, [&](uint32_t block0, uint32_t blocks) {
    hipLaunchKernelGGL((k_embed<W, O>), dim3(blocks), dim3(256), 0, st, (const W *)w, vocab, (int)width, ld, ids, index,
                       (int64_t)block0, n, (int)pieces, scale, n * width * (int64_t)sizeof(O) > kPastBytes, (O *)out);
  });
}

// Entries a wave adds up: few while there are few waves (8192 fill the chip), else enough that little is left to join.
int eg_tile(int64_t batch, int64_t n, int64_t width) {
  const int64_t work = batch * n * ((width + 511) / 512);
  return work <= 16384 * 16 ? 16 : work <= 16384 * 32 ? 32 : 64;
}

struct EgWork {
  int64_t tiles, entries, sums, bytes;  // bytes of one list of entries, of one set of partial sums, of all
};
EgWork eg_work(int64_t batch, int64_t n, int64_t width) {
  EgWork w;
  const int R = eg_tile(batch, n, width);
  w.tiles = (n + R - 1) / R;
  w.entries = (batch * n * (int64_t)sizeof(Entry) + 255) / 256 * 256;
  w.sums = w.tiles > 1 ? (batch * w.tiles * width * 4 + 255) / 256 * 256 : 0;
  w.bytes = w.entries * (n > kRun ? 2 : 1) + 2 * w.sums;
  return w;
}

// Returns at the first launch that fails: the kernels after it would take what the workspace happens to hold for
// positions and ids.
template <typename G, typename O>
int run_eg(const void *dy, int64_t ld, const void *ids, int index, int64_t batch, int64_t n, int64_t vocab,
           int64_t width, float scale, O *out, int accumulate, void *work, hipStream_t st) {
  const bool whole = width % Vec<G>::N == 0 || (!accumulate && width >= Vec<G>::N);
  // One launch is sooner done than three (8000 x 256 fp32: 333 tokens 6 us on the device, 1024 tokens 11 us, sorted 19;
  // 10000 x 1000: 1000 tokens 16 us, 22; 4 x 20000 x 64: 1024 tokens 24 us, 20, and 6 us less to launch); where the
  // gradient is large, looking through the tokens in each of its workgroups costs more than sorting them once (8 x 50257
  // x 768 fp32: 128 tokens 236 us, 204 us sorted).
  const int64_t bytes = batch * vocab * width * (int64_t)sizeof(O);
  if (n <= kFewTokens && bytes <= (64 << 20)) {
    // few rows a workgroup where frequent ids are to be dealt out (8 MB, 333 tokens: 4 KB 5.4 us, 8 KB 7.9 us), more where
    // many workgroups look through the tokens (40 MB, 300 tokens: 15 us, 10 us)
    const int64_t share = bytes <= (16 << 20) ? 4096 : 8192;
    const int rows = (int)std::max<int64_t>(1, std::min<int64_t>(16, share / (width * (int64_t)sizeof(O))));
    const int64_t per = (vocab + rows - 1) / rows;
    grid_parts(batch * per, [&](uint32_t block0, uint32_t blocks) {
      auto launch = [&](auto w, auto turns) {
        hipLaunchKernelGGL((k_eg_few<G, O, decltype(w)::value, decltype(turns)::value>), dim3(blocks), dim3(256), 0, st,
                           (const G *)dy, ld, ids, index, (int)n, vocab, (int)width, rows, per, (int64_t)block0, scale,
                           accumulate, out);
      };
      if (whole && n <= 256)
        launch(std::true_type(), std::integral_constant<int, 1>());
      else if (whole && n <= 512)
        launch(std::true_type(), std::integral_constant<int, 2>());
      else if (whole)
        launch(std::true_type(), std::integral_constant<int, 4>());
      else
        launch(std::false_type(), std::integral_constant<int, 4>());
    });
    return train_launched();
  }
  const EgWork w = eg_work(batch, n, width);
  Entry *sorted = (Entry *)work, *other = (Entry *)((char *)work + w.entries);
  Sums s;
  s.head = (float *)((char *)work + w.entries * (n > kRun ? 2 : 1));
  s.tail = s.head + w.sums / 4;
  const int64_t runs = (n + kRun - 1) / kRun, tiles = (std::min<int64_t>(n, kRun) + 63) / 64;  // tiles of a run
  // up to 2^23 workgroups that rank (a run of few tokens takes as many as the longest) and 2^21 that zero: more than one
  // launch of 512 threads each may hold
  const int64_t rank_blocks = batch * runs * tiles;
  const Zeros z{(char *)out, accumulate ? 0 : batch * vocab * width * (int64_t)sizeof(O)};
  const int64_t zero_blocks = std::min<int64_t>((z.bytes + 8191) / 8192, 1 << 21);
  constexpr int64_t kMost = kGridBlocks / 2;
  for (int64_t b = 0; b < rank_blocks + zero_blocks; b += kMost)
    hipLaunchKernelGGL(k_eg_rank, dim3((unsigned)std::min(kMost, rank_blocks + zero_blocks - b)), dim3(512), 0, st, ids,
                       index, n, vocab, (int)runs, (int)tiles, (uint32_t)b, (uint32_t)rank_blocks, (uint32_t)zero_blocks,
                       sorted, z);
  int rc = train_launched();
  for (int64_t len = kRun; rc == SK_OK && len < n; len *= kMergeRuns) {
    grid_parts((batch * n * kMergeRuns + 255) / 256, [&](uint32_t block0, uint32_t blocks) {
      hipLaunchKernelGGL(k_eg_merge, dim3(blocks), dim3(256), 0, st, sorted, other, n, len, batch * n, block0);
    });
    std::swap(sorted, other);
    rc = train_launched();
  }
  if (rc != SK_OK) return rc;
  s.sorted = sorted;
  s.n = n;
  s.vocab = vocab;
  s.ld = ld;
  s.tiles = w.tiles;
  s.width = (int)width;
  s.pieces = (int)((width + 64 * Vec<G>::N - 1) / (64 * Vec<G>::N));
  s.R = eg_tile(batch, n, width);
  s.accumulate = accumulate;
  s.scale = scale;
  const int64_t jobs = batch * w.tiles * s.pieces;
  const dim3 sum_blocks((unsigned)((jobs + 3) / 4));
  if (jobs && whole)
    hipLaunchKernelGGL((k_eg_sum<G, O, true>), sum_blocks, dim3(256), 0, st, s, (uint32_t)jobs, (const G *)dy, out);
  else if (jobs)
    hipLaunchKernelGGL((k_eg_sum<G, O, false>), sum_blocks, dim3(256), 0, st, s, (uint32_t)jobs, (const G *)dy, out);
  if ((rc = train_launched()) != SK_OK || w.tiles <= 1) return rc;
  hipLaunchKernelGGL((k_eg_join<O>), dim3((unsigned)(batch * w.tiles * ((width + 255) / 256))), dim3(256), 0, st, s, out);
  return train_launched();
}

bool dtype_ok(int d) { return d == SK_F32 || d == SK_BF16; }

}  // namespace

extern "C" {

int sketch_embed(const void *weight, sk_dtype dtype, int64_t vocab, int64_t width, int64_t ld, const void *ids,
                 sk_index index, int64_t n, float scale, void *out, sk_dtype out_dtype, int32_t device, void *stream) {
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype)) return train_fail(SK_EDTYPE, "unknown dtype");
  if (index != SK_I32 && index != SK_I64) return train_fail(SK_EDTYPE, "unknown index type");
  if (vocab < 1 || width < 1 || n < 0 || ld < width)
    return train_fail(SK_EINVAL, "need vocab, width >= 1, n >= 0 and ld >= width");
  if (n > INT32_MAX || width > (1 << 24) || n * ((width + 1023) / 1024) > INT32_MAX)
    return train_fail(SK_EUNSUPPORTED, "too many ids, or a width above 2^24");
  if (n == 0) return SK_OK;
  if (!weight || !ids || !out) return train_fail(SK_EINVAL, "NULL argument");
  TrainGuard guard(device);
  if (!guard.ok) return train_no_device();
  hipStream_t st = (hipStream_t)stream;
  if (dtype == SK_F32 && out_dtype == SK_F32)
    run_embed<float, float>(weight, vocab, width, ld, ids, index, n, scale, out, st);
  else if (dtype == SK_F32)
    run_embed<float, bf16>(weight, vocab, width, ld, ids, index, n, scale, out, st);
  else if (out_dtype == SK_F32)
    run_embed<bf16, float>(weight, vocab, width, ld, ids, index, n, scale, out, st);
  else
    run_embed<bf16, bf16>(weight, vocab, width, ld, ids, index, n, scale, out, st);
  return train_launched();
}

int64_t sketch_embed_grad_work_bytes(int64_t batch, int64_t n, int64_t width) {
  if (batch < 1 || n < 0 || width < 1 || batch > (1 << 18) || n >= (1 << 28) || batch * n >= (1 << 28) || width > (1 << 24))
    return 0;
  return std::max<int64_t>(256, eg_work(batch, n, width).bytes);
}

int sketch_embed_grad(const void *dy, sk_dtype dtype, int64_t ld, const void *ids, sk_index index, int64_t batch,
                      int64_t n, int64_t vocab, int64_t width, float scale, void *out, sk_dtype out_dtype,
                      int32_t accumulate, void *work, int64_t work_bytes, int32_t device, void *stream) {
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype)) return train_fail(SK_EDTYPE, "unknown dtype");
  if (index != SK_I32 && index != SK_I64) return train_fail(SK_EDTYPE, "unknown index type");
  if (batch < 1 || vocab < 1 || width < 1 || n < 0 || ld < width)
    return train_fail(SK_EINVAL, "need batch, vocab, width >= 1, n >= 0 and ld >= width");
  // what the launches' grids and 32-bit entries hold
  if (vocab > (1 << 20) || width > (1 << 24) || batch > (1 << 18) || n >= (1 << 28) || batch * n >= (1 << 28) ||
      batch * vocab > (1ll << 40) / width || batch * eg_work(batch, n, width).tiles * ((width + 255) / 256) > kGridBlocks)
    return train_fail(SK_EUNSUPPORTED, "sizes above what the kernels take");
  if (!out || (n && (!dy || !ids || !work))) return train_fail(SK_EINVAL, "NULL argument");
  if (n && work_bytes < sketch_embed_grad_work_bytes(batch, n, width))
    return train_fail(SK_EINVAL, "work is smaller than sketch_embed_grad_work_bytes");
  TrainGuard guard(device);
  if (!guard.ok) return train_no_device();
  hipStream_t st = (hipStream_t)stream;
  if (dtype == SK_F32 && out_dtype == SK_F32)
    return run_eg<float>(dy, ld, ids, index, batch, n, vocab, width, scale, (float *)out, accumulate, work, st);
  if (dtype == SK_F32)
    return run_eg<float>(dy, ld, ids, index, batch, n, vocab, width, scale, (bf16 *)out, accumulate, work, st);
  if (out_dtype == SK_F32)
    return run_eg<bf16>(dy, ld, ids, index, batch, n, vocab, width, scale, (float *)out, accumulate, work, st);
  return run_eg<bf16>(dy, ld, ids, index, batch, n, vocab, width, scale, (bf16 *)out, accumulate, work, st);
}

}  // extern "C"
