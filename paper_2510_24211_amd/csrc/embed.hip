// Token embedding and its gradient:
//   x[r] = scale * W[id_r]                              one rounding, to bf16
//   dW[v] = scale * sum over the rows r with id_r = v of dx[r]
// Both move memory and compute nothing to speak of.
//
// Gradient.  The rows that share an id have to be added up in 32 bits, in a fixed order, and every row of dW is written
// once.  So the row numbers are sorted by id (a stable radix sort: equal ids keep the order of their rows), and a
// wavefront walks a chunk of the sorted rows along 512 columns.  An id whose rows lie in one chunk is done there; one
// that reaches over a chunk's border leaves a partial sum per chunk, and join_kernel adds those up, in order, by several
// wavefronts: one id may hold most of the rows.  Ids that no row has get their zeros in the same launch as the sums,
// from workgroups behind them that look their stretch of ids up in the sorted list.
//   Bound by memory where there is much to move: 25600 rows of 4096 (a fifth in one id) on 64000 ids take 189 us, 150 of them in the sums'
// launch (4.9 TB/s), 31 for sorting and 7.5 for joining; by its three launches where there is not (576 rows of 1280 on 16384 ids, fp32: 33 us,
// 16 of them the zeros' bytes).  The lookup of 25600 rows takes 66 us, of 64 rows 5.4, a launch.
//   In sorting, every block of 2048 rows reads the digits' counts of all blocks: a term that grows with the square of the rows.  It is lost in the
// rest up to some 2^20 rows (all of the gradient for rows of 8 columns: 186 us for 2^20 rows, 0.75 ms for 2^22) and is nearly all there is at the
// limit of 2^25 (21 ms).
#include "scd_device.h"
#include "scd_kernels.h"
#include "tile_loads.h"

namespace scd {
namespace {

typedef float f32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x8 widen(u32x4 v) { return __builtin_convertvector(__builtin_bit_cast(bf16x8, v), f32x8); }
__device__ __forceinline__ u32x4 narrow(f32x8 v) { return __builtin_bit_cast(u32x4, __builtin_convertvector(v, bf16x8)); }

// ---- lookup ------------------------------------------------------------------------------------
// A wavefront per row and 512 pieces of 16 bytes; all of its loads are under way before the first store.
constexpr int kPieces = 8;       // per lane

// scale * W[id] for the wavefront's stretch of one row; zeros where there is no such id
__device__ __forceinline__ void embed_row(const u32x4* __restrict__ W, int64_t id, bool there, int d8, int first, float scale,
                                          u32x4* __restrict__ to) {
  const int lane = threadIdx.x & 63;
  const u32x4* const from = W + (there ? id * d8 : 0);
  u32x4 v[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) v[i] = from[min(first + i * 64 + lane, d8 - 1)];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int at = first + i * 64 + lane;
    if (at < d8) to[at] = there ? narrow(widen(v[i]) * scale) : u32x4{0u, 0u, 0u, 0u};
  }
}

__global__ __launch_bounds__(256) void embed_kernel(const int32_t* __restrict__ ids, const u32x4* __restrict__ W, u32x4* __restrict__ x,
                                                    int rows, int V, int d8, float scale) {
  const int r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // up to 2^25 rows: in range
  if (r >= rows) return;
  const int id = ids[r];
  embed_row(W, id, id >= 0 && id < V, d8, blockIdx.y * (64 * kPieces), scale, x + static_cast<int64_t>(r) * d8);
}

// The drafts of the current windows: row (b, c, s) is position pos[b] + s, zeros behind the sequence's end.
__global__ __launch_bounds__(256) void embed_window_kernel(const EmbedArgs a) {
  const int r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (r >= a.rows) return;
  const int s = r % a.L, b = r / a.L / a.C, pos = a.pos[b];
  const bool live = pos >= 0 && s < a.N - pos;
  const int id = a.v_lo + a.X[static_cast<int64_t>(b) * a.L + (live ? (pos + s) % a.L : 0)];
  embed_row(reinterpret_cast<const u32x4*>(a.W), id, live && id >= 0 && id < a.V, a.d / 8, blockIdx.y * (64 * kPieces), a.scale,
            reinterpret_cast<u32x4*>(a.x) + static_cast<int64_t>(r) * (a.d / 8));
}

// ---- rows sorted by id ---------------------------------------------------------------------------
// Least significant digit first, digits of up to 9 bits.  Rows without an id get the key V, behind all others.  A
// workgroup sorts a block of neighbouring rows stably: its wavefronts take 64 keys at a time in order, lanes with equal
// digits find each other by ballots, and a key's place is the number of equal digits before it.
constexpr int kMaxBins = 512;
struct Digits {
  int shift, bits;
};
struct KeyRow {
  uint32_t key, row;
};

__device__ __forceinline__ uint32_t key_of(const int32_t* ids, uint32_t r, uint32_t V) {
  const uint32_t id = static_cast<uint32_t>(ids[r]);
  return min(id, V);             // negative ids are large ones
}
// lanes of the wavefront (of those in `live`) whose digit is this lane's
__device__ __forceinline__ uint64_t equal_digits(uint32_t digit, int bits, uint64_t live) {
  uint64_t m = live;
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __builtin_amdgcn_ballot_w64((digit >> b) & 1u);
    m &= (digit >> b) & 1u ? set : ~set;
  }
  return m;
}
// One pass over the block's keys in k[] (`rounds` of the ROUNDS per thread in use, `count` of the block exist; a wavefront holds
// rounds * 64 neighbours): their digits' bins are counted per wavefront in `bins` [NW][kMaxBins], and place[] = number of
// equal digits before the key in its wavefront.
template <int NW, int ROUNDS>
__device__ __forceinline__ void count_digits(const uint32_t (&k)[ROUNDS], const Digits g, int rounds, int count, uint32_t* bins,
                                             uint32_t (&place)[ROUNDS]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int b = lane; b < 1 << g.bits; b += 64) bins[wave * kMaxBins + b] = 0u;
  __syncthreads();
  uint32_t* const mine = bins + wave * kMaxBins;
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    if (j >= rounds) break;
    const bool is = wave * rounds * 64 + j * 64 + lane < count;
    const uint64_t live = __builtin_amdgcn_ballot_w64(is);
    const uint32_t digit = (k[j] >> g.shift) & ((1u << g.bits) - 1u);
    const uint64_t same = equal_digits(digit, g.bits, live);
    const uint32_t before = __popcll(same & ((1ull << lane) - 1ull));
    place[j] = mine[digit] + before;
    compiler_fence();                     // LDS operations of a wavefront are performed in order
    if (is && before == 0u) mine[digit] += __popcll(same);
    compiler_fence();
  }
  __syncthreads();
}
// bins [NW][kMaxBins] -> first place of a wavefront's digit in the sorted block, given the first place of every digit in
// `first` (kMaxBins words; the block's totals are added by the caller's scan before)
template <int NW>
__device__ __forceinline__ void spread_bins(uint32_t* bins, const uint32_t* first, int nbins) {
  for (int b = threadIdx.x; b < nbins; b += NW * 64) {
    uint32_t at = first[b], c[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) c[w] = bins[w * kMaxBins + b];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      bins[w * kMaxBins + b] = at;
      at += c[w];
    }
  }
  __syncthreads();
}
// exclusive prefix sums of kMaxBins words, by the first wavefront; all threads call
__device__ __forceinline__ void scan_bins(uint32_t* v) {
  __syncthreads();
  if (threadIdx.x < 64) {
    constexpr int PER = kMaxBins / 64;
    uint32_t c[PER], sum = 0u;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      c[j] = v[threadIdx.x * PER + j];
      sum += c[j];
    }
    uint32_t incl = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t up = __shfl_up(incl, o, 64);
      incl += static_cast<int>(threadIdx.x) >= o ? up : 0u;
    }
    uint32_t at = incl - sum;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      v[threadIdx.x * PER + j] = at;
      at += c[j];
    }
  }
  __syncthreads();
}

// Up to kOneBlock rows: all passes in LDS by one workgroup, one launch.
constexpr int kOneWaves = 16, kOneRounds = 8, kOneBlock = kOneWaves * 64 * kOneRounds;
__global__ __launch_bounds__(kOneWaves * 64) void sort_one_kernel(const int32_t* __restrict__ ids, int rows, uint32_t V, int passes, int bits,
                                                                 KeyRow* __restrict__ out) {
  __shared__ KeyRow block[kOneBlock];
  __shared__ uint32_t bins[kOneWaves * kMaxBins], first[kMaxBins];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t k[kOneRounds], r[kOneRounds], place[kOneRounds];
  const int rounds = (rows + kOneWaves * 64 - 1) / (kOneWaves * 64);
  auto at = [&](int j) { return j < rounds ? wave * rounds * 64 + j * 64 + lane : rows; };
#pragma unroll
  for (int j = 0; j < kOneRounds; ++j) {
    r[j] = at(j);
    k[j] = at(j) < rows ? key_of(ids, r[j], V) : 0u;
  }
  for (int p = 0; p < passes; ++p) {
    const Digits g{p * bits, bits};
    count_digits<kOneWaves, kOneRounds>(k, g, rounds, rows, bins, place);
    for (int b = tid; b < kMaxBins; b += kOneWaves * 64) {
      uint32_t sum = 0u;
      if (b < 1 << bits)
#pragma unroll
      for (int w = 0; w < kOneWaves; ++w) sum += bins[w * kMaxBins + b];
      first[b] = sum;
    }
    scan_bins(first);
    spread_bins<kOneWaves>(bins, first, 1 << bits);
#pragma unroll
    for (int j = 0; j < kOneRounds; ++j)
      if (at(j) < rows) block[bins[wave * kMaxBins + ((k[j] >> g.shift) & ((1u << bits) - 1u))] + place[j]] = KeyRow{k[j], r[j]};
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kOneRounds; ++j)
      if (at(j) < rows) {
        k[j] = block[at(j)].key;
        r[j] = block[at(j)].row;
      }
  }
#pragma unroll
  for (int j = 0; j < kOneRounds; ++j)
    if (at(j) < rows) out[at(j)] = KeyRow{k[j], r[j]};
}

// More rows: per pass, the digits of every block are counted, then each block works out where its keys go and moves them.
constexpr int kWaves = 4, kRounds = 8, kBlock = kWaves * 64 * kRounds;
template <bool FIRST>
__device__ __forceinline__ void load_keys(const int32_t* ids, const KeyRow* in, int rows, uint32_t V, uint32_t (&k)[kRounds],
                                          uint32_t (&r)[kRounds]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int j = 0; j < kRounds; ++j) {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kBlock + wave * kRounds * 64 + j * 64 + lane;
    k[j] = 0u;
    r[j] = static_cast<uint32_t>(at);
    if (at < rows) {
      if (FIRST) {
        k[j] = key_of(ids, r[j], V);
      } else {
        const KeyRow t = in[at];
        k[j] = t.key;
        r[j] = t.row;
      }
    }
  }
}
template <bool FIRST>
__global__ __launch_bounds__(kWaves * 64) void sort_count_kernel(const int32_t* __restrict__ ids, const KeyRow* __restrict__ in, int rows,
                                                                uint32_t V, Digits g, uint32_t* __restrict__ counts) {
  __shared__ uint32_t bins[kMaxBins];
  uint32_t k[kRounds], r[kRounds];
  load_keys<FIRST>(ids, in, rows, V, k, r);
  for (int i = threadIdx.x; i < kMaxBins; i += kWaves * 64) bins[i] = 0u;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kRounds; ++j) {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kBlock + (threadIdx.x >> 6) * kRounds * 64 + j * 64 + (threadIdx.x & 63);
    if (at < rows) atomicAdd(&bins[(k[j] >> g.shift) & ((1u << g.bits) - 1u)], 1u);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kMaxBins; i += kWaves * 64) counts[static_cast<int64_t>(blockIdx.x) * kMaxBins + i] = bins[i];
}
template <bool FIRST>
__global__ __launch_bounds__(kWaves * 64) void sort_move_kernel(const int32_t* __restrict__ ids, const KeyRow* __restrict__ in, int rows,
                                                               uint32_t V, Digits g, const uint32_t* __restrict__ counts,
                                                               KeyRow* __restrict__ out) {
  __shared__ uint32_t bins[kWaves * kMaxBins], first[kMaxBins];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t k[kRounds], r[kRounds], place[kRounds];
  load_keys<FIRST>(ids, in, rows, V, k, r);
  const int count = static_cast<int>(min(static_cast<int64_t>(kBlock), rows - static_cast<int64_t>(blockIdx.x) * kBlock));
  // keys of a digit in the blocks before this one, and in all of them
  uint32_t before[kMaxBins / (kWaves * 64)];
#pragma unroll
  for (int i = 0; i < kMaxBins / (kWaves * 64); ++i) {
    const int b = threadIdx.x + i * kWaves * 64;
    uint32_t all = 0u;
    before[i] = 0u;
    if (b < 1 << g.bits) {
#pragma unroll 16
      for (int blk = 0; blk < static_cast<int>(gridDim.x); ++blk) {
        const uint32_t c = counts[static_cast<int64_t>(blk) * kMaxBins + b];
        before[i] += blk < static_cast<int>(blockIdx.x) ? c : 0u;
        all += c;
      }
    }
    first[b] = all;
  }
  scan_bins(first);
#pragma unroll
  for (int i = 0; i < kMaxBins / (kWaves * 64); ++i) first[threadIdx.x + i * kWaves * 64] += before[i];
  count_digits<kWaves, kRounds>(k, g, kRounds, count, bins, place);
  spread_bins<kWaves>(bins, first, 1 << g.bits);
#pragma unroll
  for (int j = 0; j < kRounds; ++j)
    if (wave * kRounds * 64 + j * 64 + lane < count)
      out[bins[wave * kMaxBins + ((k[j] >> g.shift) & ((1u << g.bits) - 1u))] + place[j]] = KeyRow{k[j], r[j]};
}

// ---- sums ----------------------------------------------------------------------------------------
constexpr int kSlice = 512;      // columns of a wavefront: 8 per lane
constexpr uint32_t kZeroIds = 16;

// dW row `id`, this lane's 8 columns from `col`: one rounding
template <bool F32, bool ACC>
__device__ __forceinline__ void put(void* dW, int64_t id, int d, int col, f32x8 v) {
  if constexpr (F32) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    f32x4* const to = reinterpret_cast<f32x4*>(static_cast<float*>(dW) + id * d + col);
    f32x4 a{v[0], v[1], v[2], v[3]}, b{v[4], v[5], v[6], v[7]};
    if (ACC) {
      a += to[0];
      b += to[1];
    }
    to[0] = a;
    to[1] = b;
  } else {
    u32x4* const to = reinterpret_cast<u32x4*>(static_cast<uint16_t*>(dW) + id * d + col);
    if (ACC) v += widen(*to);
    *to = narrow(v);
  }
}

struct SumArgs {
  const KeyRow* sorted;
  const uint16_t* dx;
  void* dW;
  float* part;          // [chunks][2][d]: sums of the chunk's first id (it began before the chunk) and of its last (it goes on)
  int rows, V, d, chunk, chunks;
  uint32_t sum_blocks, zero_blocks;
  float scale;
};

constexpr uint32_t kNoKey = 0xFFFFFFFFu;
// key of the sorted row at `at`, or one that no row has
__device__ __forceinline__ uint32_t key_at(const SumArgs& a, int64_t at) { return at >= 0 && at < a.rows ? a.sorted[at].key : kNoKey; }

template <bool F32, bool ACC>
__global__ __launch_bounds__(256) void sum_kernel(const SumArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (!ACC && blockIdx.x >= a.sum_blocks) {
    // ---- rows that no id has: a workgroup looks after kZeroIds neighbouring ids of dW at a time --------------------
    __shared__ uint32_t seen[kZeroIds];
    for (uint32_t stretch = blockIdx.x - a.sum_blocks; stretch < (a.V - 1u) / kZeroIds + 1u; stretch += a.zero_blocks) {
      const uint32_t v0 = stretch * kZeroIds, v1 = min(v0 + kZeroIds, static_cast<uint32_t>(a.V));
      __syncthreads();
      if (threadIdx.x < kZeroIds) seen[threadIdx.x] = 0u;
      __syncthreads();
      // the first sorted row with a key of v0 or more, 64 places at a time
      int64_t lo = 0, hi = a.rows;         // in [lo, hi]
      while (hi > lo) {
        const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
        const bool below = at < hi && a.sorted[at].key < v0;
        const int n = __popcll(__builtin_amdgcn_ballot_w64(below));
        if (n == 0) hi = lo;
        else {
          hi = min(hi, lo + n * step);
          lo = lo + (n - 1) * step + 1;
        }
      }
      for (int64_t at = lo + threadIdx.x; at < a.rows; at += 256) {
        const uint32_t key = a.sorted[at].key;
        if (key >= v1) break;
        seen[key - v0] = 1u;
      }
      __syncthreads();
      const f32x8 zero{};
      for (uint32_t v = v0 + wave; v < v1; v += 4) {
        if (seen[v - v0]) continue;
        for (int col = lane * 8; col < a.d; col += kSlice) put<F32, false>(a.dW, v, a.d, col, zero);
      }
    }
    return;
  }
  // ---- a chunk of the sorted rows along 512 columns ------------------------------------------------------
  const int slices = (a.d + kSlice - 1) / kSlice;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + wave;
  if (item >= static_cast<int64_t>(a.chunks) * slices) return;
  const int chunk = static_cast<int>(item / slices), col = static_cast<int>(item % slices) * kSlice + lane * 8;
  const bool mine = col < a.d;
  const int64_t p0 = static_cast<int64_t>(chunk) * a.chunk, p1 = min(p0 + a.chunk, static_cast<int64_t>(a.rows));
  const uint16_t* const dx = a.dx + (mine ? col : 0);
  const uint32_t before = key_at(a, p0 - 1), behind = key_at(a, p1);
  f32x8 sum{};
  uint32_t key = a.sorted[p0].key;
  bool began = before != key;            // the current id's first row is in this chunk
  auto flush = [&](bool ends) {
    if (!mine || key >= static_cast<uint32_t>(a.V)) return;
    if (began && ends) put<F32, ACC>(a.dW, key, a.d, col, sum * a.scale);
    else {
      f32x8* const to = reinterpret_cast<f32x8*>(a.part + (static_cast<int64_t>(chunk) * 2 + (began ? 1 : 0)) * a.d + col);
      *to = sum;
    }
  };
  constexpr int AHEAD = 8;
  for (int64_t p = p0; p < p1; p += AHEAD) {
    uint32_t k[AHEAD];
    u32x4 v[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const KeyRow t = a.sorted[min(p + j, p1 - 1)];
      k[j] = p + j < p1 ? t.key : static_cast<uint32_t>(a.V);
      v[j] = *reinterpret_cast<const u32x4*>(dx + static_cast<int64_t>(t.row) * a.d);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (p + j >= p1) break;
      if (k[j] != key) {
        flush(true);
        key = k[j];
        began = true;
        sum = f32x8{};
      }
      sum += widen(v[j]);
    }
  }
  flush(behind != key);
}

// The ids that reach over chunks' borders: a workgroup for the chunk in which such an id begins and 512 columns adds its partial
// sums up.  They come from other XCDs, 2 to 4 us a round trip, so its wavefronts share them (a fifth of 25600 rows along 4096
// columns in one id: one wavefront in two 56 us, one in eight 14).
constexpr int kJoinWaves = 8;
template <bool F32, bool ACC>
__global__ __launch_bounds__(kJoinWaves * 64) void join_kernel(const SumArgs a) {
  __shared__ f32x8 sums[kJoinWaves][64];
  __shared__ int run[kJoinWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int chunk = blockIdx.x;
  const int64_t p0 = static_cast<int64_t>(chunk) * a.chunk, p1 = p0 + a.chunk;
  if (p1 >= a.rows) return;
  const uint32_t key = a.sorted[p1 - 1].key, behind = a.sorted[p1].key, first_key = a.sorted[p0].key, before = key_at(a, p0 - 1);
  if (key >= static_cast<uint32_t>(a.V) || behind != key) return;       // it ends here
  if (first_key == key && before == key) return;                         // it began before
  // chunks behind this one that begin with the id: all up to the last one, found kJoinWaves * 64 at a time
  int last = chunk + 1;
  for (;;) {
    const int c = last + 1 + wave * 64 + lane;
    const uint64_t same = __builtin_amdgcn_ballot_w64(c < a.chunks && a.sorted[min(static_cast<int64_t>(c) * a.chunk, static_cast<int64_t>(a.rows) - 1)].key == key);
    if (lane == 0) run[wave] = same == ~0ull ? 64 : __builtin_ctzll(~same);
    __syncthreads();
    int n = 0;
    for (int w = 0; w < kJoinWaves; ++w) {
      n += run[w];
      if (run[w] < 64) break;
    }
    __syncthreads();
    last += n;
    if (n < kJoinWaves * 64) break;
  }
  const int first = chunk + 1, count = last - first + 1, per = (count + kJoinWaves - 1) / kJoinWaves;
  const int c0 = first + wave * per, c1 = min(c0 + per, last + 1);
  const int col = blockIdx.y * kSlice + lane * 8;
  const bool mine = col < a.d;
  f32x8 sum{};
  if (mine) {
    const float* const at = a.part + col;
    if (wave == 0) sum = *reinterpret_cast<const f32x8*>(at + (static_cast<int64_t>(chunk) * 2 + 1) * a.d);
#pragma unroll 8
    for (int c = c0; c < c1; ++c) sum += *reinterpret_cast<const f32x8*>(at + static_cast<int64_t>(c) * 2 * a.d);
  }
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || !mine) return;
#pragma unroll
  for (int w = 1; w < kJoinWaves; ++w) sum += sums[w][lane];
  put<F32, ACC>(a.dW, key, a.d, col, sum * a.scale);
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
// Sorted rows of a wavefront: more of them leave fewer partial sums of frequent ids to be joined (25600 rows of 4096, a fifth in one id: chunks
// of 32 join in 14 - 19 us, of 64 in 7.5, and the sums take as long), fewer of them fill the chip when there are few rows.
inline int chunk_rows(int rows) { return rows > (1 << 16) ? 128 : rows > (1 << 14) ? 64 : 32; }

template <bool F32, bool ACC>
hipError_t launch_sums(SumArgs a, hipStream_t s) {
  const int slices = (a.d + kSlice - 1) / kSlice;
  // the sums first: they wait for loads, and the zeros fill the time
  a.sum_blocks = static_cast<uint32_t>((static_cast<int64_t>(a.chunks) * slices + 3) / 4);
  const int64_t blocks = static_cast<int64_t>(a.sum_blocks) + (ACC ? 0 : a.zero_blocks);
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL((sum_kernel<F32, ACC>), dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, s, a);
  if (a.chunks > 1) hipLaunchKernelGGL((join_kernel<F32, ACC>), dim3(a.chunks - 1, slices), dim3(kJoinWaves * 64), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(const EmbedArgs& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const dim3 grid((a.rows + 3) / 4, (a.d / 8 + 64 * kPieces - 1) / (64 * kPieces));
  if (a.X) hipLaunchKernelGGL(embed_window_kernel, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(embed_kernel, grid, dim3(256), 0, s, a.ids, reinterpret_cast<const u32x4*>(a.W), reinterpret_cast<u32x4*>(a.x), a.rows,
                       a.V, a.d / 8, a.scale);
  return hipGetLastError();
}

// two lists of (key, row); the blocks' counts; two partial sums per chunk
size_t embed_backward_bytes(int rows, int d) {
  if (rows == 0) return 256;
  const size_t blocks = (static_cast<size_t>(rows) + kBlock - 1) / kBlock, chunk = chunk_rows(rows);
  return 2 * up256(sizeof(KeyRow) * static_cast<size_t>(rows)) + up256(sizeof(uint32_t) * kMaxBins * blocks) +
         up256(2 * sizeof(float) * d * ((rows + chunk - 1) / chunk));
}

hipError_t launch_embed_backward(const EmbedBackwardArgs& e, hipStream_t s) {
  const int rows = e.rows;
  char* at = static_cast<char*>(e.ws);
  auto take = [&](size_t bytes) {
    char* const p = at;
    at += up256(bytes);
    return p;
  };
  const int blocks = static_cast<int>((static_cast<int64_t>(rows) + kBlock - 1) / kBlock);
  KeyRow* list[2];
  for (KeyRow*& l : list) l = reinterpret_cast<KeyRow*>(take(sizeof(KeyRow) * static_cast<size_t>(rows)));
  uint32_t* const counts = reinterpret_cast<uint32_t*>(take(sizeof(uint32_t) * kMaxBins * static_cast<size_t>(blocks)));
  SumArgs a{};
  a.dx = e.dx; a.dW = e.dW; a.rows = rows; a.V = e.V; a.d = e.d; a.scale = e.scale;
  a.chunk = chunk_rows(rows);
  a.chunks = static_cast<int>((static_cast<int64_t>(rows) + a.chunk - 1) / a.chunk);
  a.part = reinterpret_cast<float*>(at);
  int all = 1;                                      // bits of the keys 0 .. V
  while (all < 32 && (static_cast<uint64_t>(e.V) >> all) != 0) ++all;
  const int passes = (all + 8) / 9, bits = (all + passes - 1) / passes;
  const KeyRow* sorted = list[0];
  if (rows > 0 && rows <= kOneBlock) {
    hipLaunchKernelGGL(sort_one_kernel, dim3(1), dim3(kOneWaves * 64), 0, s, e.ids, rows, static_cast<uint32_t>(e.V), passes, bits, list[0]);
  } else if (rows > 0) {
    for (int p = 0; p < passes; ++p) {
      const Digits g{p * bits, bits};
      KeyRow* const to = list[p & 1];
      if (p == 0) {
        hipLaunchKernelGGL(sort_count_kernel<true>, dim3(blocks), dim3(kWaves * 64), 0, s, e.ids, sorted, rows, static_cast<uint32_t>(e.V), g, counts);
        hipLaunchKernelGGL(sort_move_kernel<true>, dim3(blocks), dim3(kWaves * 64), 0, s, e.ids, sorted, rows, static_cast<uint32_t>(e.V), g, counts, to);
      } else {
        hipLaunchKernelGGL(sort_count_kernel<false>, dim3(blocks), dim3(kWaves * 64), 0, s, e.ids, sorted, rows, static_cast<uint32_t>(e.V), g, counts);
        hipLaunchKernelGGL(sort_move_kernel<false>, dim3(blocks), dim3(kWaves * 64), 0, s, e.ids, sorted, rows, static_cast<uint32_t>(e.V), g, counts, to);
      }
      sorted = to;
    }
  }
  a.sorted = sorted;
  a.zero_blocks = min((e.V - 1u) / kZeroIds + 1u, 1u << 18);
  if (e.f32) return e.accumulate ? launch_sums<true, true>(a, s) : launch_sums<true, false>(a, s);
  return e.accumulate ? launch_sums<false, true>(a, s) : launch_sums<false, false>(a, s);
}

}  // namespace scd
