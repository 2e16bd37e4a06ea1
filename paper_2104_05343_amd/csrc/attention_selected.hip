// Attention over chosen blocks (attention_selected_kernel.hpp): the lists, the forward pass, the sums over a query's blocks, what the
// host decides.
#include <atomic>

#include "attention_selected_kernel.hpp"

namespace optimus {
namespace {

// ---------------------------------------------------------------- lists
// Bound: round trips to memory (the choice read twice, lists and places written once; the table of counts, a row a chunk, see kFewChunks): 17 and 33 us for 8
// (sequence, head)s of 32768 queries with 16 entries each (17 MB), 5 (10 with the backward pass' sums) and 7 for 16 of 4096 with 8.
// Pairs of 256 queries as a bit a (block, query) in LDS: entries that name a block twice, none, or one that the query does not see
// make no pair, and a query's place among a block's is a count of bits.  bits[word of 32 queries][block].
constexpr int kWords = kListChunk / 32;
// Chunks of a sequence up to which list_fill_kernel adds up the counts by itself, which grows with their square.  Fill, or a launch for the sums and fill, us: width
// 128, 16 (sequence, head)s of 4096, 8 blocks of 128 (16 chunks) 7 / 11; 8 of 16384, 16 entries (64) 19 / 21; of 24576 (96) 26 / 26; of 32768 (128) 34 / 32; of
// 65536 (256) 117 / 63; of 131072 (512) 1042 / 157; one of 2^20, 4 of 1024 (4096) 6884 / 135.
constexpr int kFewChunks = 96;
std::atomic<int> g_form{-1};                      // forced by a tuning hook: 1 masked, 0 lists
constexpr size_t kPortion = (size_t)1 << 30;    // bytes of partial results in memory at a time

__device__ __forceinline__ bool sees(const SelectedArgs& a, int len, int t, int v) {
  return v >= 0 && v < a.blocks && v * a.block < len && (!a.causal || v * a.block <= t);
}
// eight of a query's entries from e0 on, -1 behind the last; as found: a choice may start at any element
__device__ __forceinline__ void load_entries(const int* own, int e0, int count, int v[8]) {
  typedef __attribute__((ext_vector_type(4), aligned(4))) int Four;
#pragma unroll
  for (int h = 0; h < 8; h += 4) {
    if (e0 + h + 4 <= count) {
      const Four x = *(const Four*)(own + e0 + h);
#pragma unroll
      for (int u = 0; u < 4; ++u) v[h + u] = x[u];
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) v[h + u] = e0 + h + u < count ? own[e0 + h + u] : -1;
    }
  }
}
// The thread's query's entries into `bits` (zeroed); of the same block the first counts: entry(e, block, counts).
template <class F>
__device__ __forceinline__ void chunk_pairs(const SelectedArgs& a, int mm, int len, int t, unsigned* bits, F entry) {
  const int tid = threadIdx.x;
  if (t >= len) return;
  const int* own = a.selected + ((long long)mm * a.f.s + t) * a.count;
  for (int e0 = 0; e0 < a.count; e0 += 8) {
    int v[8];
    load_entries(own, e0, a.count, v);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      bool counts = false;
      if (sees(a, len, t, v[u])) {
        const unsigned bit = 1u << (tid & 31);
        counts = !(atomicOr(&bits[(tid >> 5) * a.blocks + v[u]], bit) & bit);   // (a query's bits are one thread's: no race for the first)
      }
      entry(e0 + u, v[u], counts);
    }
  }
}
// rowsum(dO * O) of a wavefront's 32 queries from t0 on, 0 past the end of a sequence
template <int D>
__device__ __forceinline__ void delta_rows(const SelectedArgs& a, int mm, int t0) {
  const FusedArgs& f = a.f;
  const int lane = threadIdx.x & 63, g = lane >> 5;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const int t = t0 + (lane & 31), row = min(t, f.s - 1);
  float delta = 0.f;
  if (t < m.len) {
    const bf16_t* G = f.d_attn + m.attn + (long long)row * f.ldo + g * 8;
    const bf16_t* O = f.attn + m.attn + (long long)row * f.ldo + g * 8;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) delta += delta_piece(*(const bf16x8*)(G + ks * 16), *(const bf16x8*)(O + ks * 16));
  }
  delta = halfwave_sum(delta);
  if (g == 0 && t < f.s) f.delta[m.vec + t] = delta;
}

// D > 0, ahead of a backward pass: the queries' delta too.
template <int D>
__global__ __launch_bounds__(kListChunk) void list_count_kernel(SelectedArgs a) {
  extern __shared__ unsigned bits[];
  const int chunk = blockIdx.x, mm = blockIdx.y;
  const int len = selected_matrix<64>(a, mm).len;
  for (int k = threadIdx.x; k < kWords * a.blocks; k += kListChunk) bits[k] = 0;
  __syncthreads();
  chunk_pairs(a, mm, len, chunk * kListChunk + threadIdx.x, bits, [](int, int, bool) {});
  __syncthreads();
  for (int v = threadIdx.x; v < a.blocks; v += kListChunk) {
    int n = 0;
#pragma unroll
    for (int w = 0; w < kWords; ++w) n += __popc(bits[w * a.blocks + v]);
    a.counts[((long long)mm * (a.chunks + 1) + chunk) * a.blocks + v] = n;
  }
  if constexpr (D > 0) {
#pragma unroll
    for (int k = 0; k < 2; ++k) delta_rows<D>(a, mm, chunk * kListChunk + (threadIdx.x >> 6) * 64 + 32 * k);
  }
}

// Counts of many chunks -> each block's pairs in earlier chunks, and behind the last chunk in all of them.  A workgroup has 64 blocks, each of its
// wavefronts a run of chunks.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(64 * kSumWaves) void list_sums_kernel(SelectedArgs a) {
  __shared__ int sums[kSumWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, v = blockIdx.x * 64 + lane;
  const bool mine = v < a.blocks;
  int* c = a.counts + (long long)blockIdx.y * (a.chunks + 1) * a.blocks + v;
  const int each = (a.chunks + kSumWaves - 1) / kSumWaves, from = min(wave * each, a.chunks), to = min(from + each, a.chunks);
  auto load = [&](int k, int x[16]) {   // sixteen in flight
#pragma unroll
    for (int u = 0; u < 16; ++u) x[u] = mine && k + u < to ? c[(long long)(k + u) * a.blocks] : 0;
  };
  int sum = 0;
  for (int k = from; k < to; k += 16) {
    int x[16];
    load(k, x);
#pragma unroll
    for (int u = 0; u < 16; ++u) sum += x[u];
  }
  sums[wave][lane] = sum;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += sums[w][lane];
  if (mine && wave == kSumWaves - 1) c[(long long)a.chunks * a.blocks] = before + sum;
  for (int k = from; k < to; k += 16) {
    int x[16];
    load(k, x);
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      if (mine && k + u < to) c[(long long)(k + u) * a.blocks] = before;
      before += x[u];
    }
  }
}

// exclusive sums of x over the workgroup's threads, the sum of all in *total
__device__ __forceinline__ int exclusive_sum(int x, int* lds, int* total) {
  constexpr int kWaves = kListChunk / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int in = x;
#pragma unroll
  for (int step = 1; step < 64; step <<= 1) {
    const int y = __shfl_up(in, step);
    if (lane >= step) in += y;
  }
  if (lane == 63) lds[wave] = in;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int y = lds[w];
    before += w < wave ? y : 0;
    all += y;
  }
  __syncthreads();
  *total = all;
  return before + in - x;
}

// Places and entries of a chunk.  SUMMED: list_sums_kernel has added up the counts; otherwise every workgroup does so itself, with its matrix' whole
// table.  The first one of a matrix writes the items too.
template <bool SUMMED>
__global__ __launch_bounds__(kListChunk) void list_fill_kernel(SelectedArgs a) {
  extern __shared__ unsigned bits[];
  int* place_of = (int*)(bits + kWords * a.blocks);   // [word][block]: place of a word's first pair
  int* lds = place_of + kWords * a.blocks;            // [kListChunk / 64]
  const int chunk = blockIdx.x, mm = blockIdx.y, tid = threadIdx.x;
  const int len = selected_matrix<64>(a, mm).len;
  const int t = chunk * kListChunk + tid;
  for (int k = tid; k < kWords * a.blocks; k += kListChunk) bits[k] = 0;
  __syncthreads();
  static_assert(kMostCount <= 64, "an entry is a bit");
  unsigned long long counted = 0;
  chunk_pairs(a, mm, len, t, bits, [&](int e, int, bool counts) { counted |= counts ? 1ull << e : 0; });
  __syncthreads();
  int earlier_pairs = 0, earlier_items[2] = {0, 0};   // of the blocks below
  for (int v0 = 0; v0 < a.blocks; v0 += kListChunk) {
    const int v = v0 + tid;
    int pairs = 0, before = 0;   // of the block, in earlier chunks
    if (v < a.blocks) {
      const int* c = a.counts + (long long)mm * (a.chunks + 1) * a.blocks + v;
      if (SUMMED) {
        pairs = c[(long long)a.chunks * a.blocks];
        before = c[(long long)chunk * a.blocks];
      }
      for (int k = 0; !SUMMED && k < a.chunks; k += 16) {   // sixteen loads in flight
        int x[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) x[u] = k + u < a.chunks ? c[(long long)(k + u) * a.blocks] : 0;
#pragma unroll
        for (int u = 0; u < 16; ++u) {
          pairs += x[u];
          before += k + u < chunk ? x[u] : 0;
        }
      }
    }
    int all;
    const int at = earlier_pairs + exclusive_sum(pairs, lds, &all);
    earlier_pairs += all;
    if (v < a.blocks) {
      int n = at + before;
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        place_of[w * a.blocks + v] = n;
        n += __popc(bits[w * a.blocks + v]);
      }
    }
    if (chunk > 0) continue;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      if (!a.items[kind]) continue;
      // equal items of at most 1.25 seg rows, no short one at the end of a list
      const int most = a.seg[kind] * 5 / 4, wanted = max((pairs + most - 1) / most, 1), size = ((pairs + wanted - 1) / wanted + 127) & ~127;
      const int items = pairs > 0 ? (pairs + size - 1) / size : 0, first = earlier_items[kind] + exclusive_sum(items, lds, &all);
      earlier_items[kind] += all;
      int* firsts = a.first_item + ((long long)kind * a.mats + mm) * (a.blocks + 1);
      if (v < a.blocks) firsts[v] = first;
      if (tid == 0) firsts[min(v0 + kListChunk, a.blocks)] = earlier_items[kind];
      for (int k = 0; k < items; ++k)
        a.items[kind][(long long)mm * a.most[kind] + first + k] = i32x4_t{v, at + k * size, min(size, pairs - k * size), 0};
    }
  }
  __syncthreads();
  if (t >= a.f.s) return;
  const long long first = (long long)mm * a.f.s * a.count;
  int* places = a.places + first + (long long)t * a.count;
  const int* own = a.selected + first + (long long)t * a.count;
  const int word = (tid >> 5) * a.blocks;
  for (int e0 = 0; e0 < a.count; e0 += 8) {
    int v[8], place[8];
    load_entries(own, e0, a.count, v);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      place[u] = -1;
      if (counted >> (e0 + u) & 1) {
        place[u] = place_of[word + v[u]] + __popc(bits[word + v[u]] & ((1u << (tid & 31)) - 1));
        a.list[first + place[u]] = t;
      }
    }
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      if (e0 + h + 4 <= a.count) {
        typedef __attribute__((ext_vector_type(4), aligned(4))) int Four;
        *(Four*)(places + e0 + h) = Four{place[h], place[h + 1], place[h + 2], place[h + 3]};
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (e0 + h + u < a.count) places[e0 + h + u] = place[h + u];
      }
    }
  }
}

// ---------------------------------------------------------------- forward
// maxima and sums of a wavefront's 32 rows, `rows` of them (see store_parts)
__device__ __forceinline__ void store_ml(float2* to, float m, float l, int rows, int g, int lane) {
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(to, 0, __builtin_amdgcn_readfirstlane(rows) * 8, 0x00020000);
  __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(m), __float_as_uint(l)}, rsrc, g == 0 ? lane * 8 : 0x7fffffff, 0, 0);
}

// A wavefront has 32 queries of a tile of 128.  KT > 0: the block is at most 32 KT = 64 or 128 keys, stays in LDS for all of the workgroup's
// queries, and a row's scores are all there before the maximum is taken: no barrier behind the loads, no rescaling.  The next tile's
// queries are requested as soon as the products of this one have read theirs, and ahead of its stores: the wait for them is no wait for stores.
// Bound: nothing alone (1.1 GB of rows in 470 us, the matrix units at 24 %, the vector units at 40 %): a wavefront's products, its soft-max and its
// row's scaling follow each other, two wavefronts a SIMD hide part of one behind the other.  Without the stores 330 us, with stores that are
// dropped 413; exponentials left out 480; other cache policies of the stores 0 to 2 % (all of 510).
template <int D, int KT>
__global__ __launch_bounds__(256, 2) void selected_fwd_kernel(SelectedArgs a) {
  constexpr int KS = D / 16, DT = D / 32, STEPS = KT / 2, AHEAD = 2;
  __shared__ __attribute__((aligned(1024))) bf16_t lds[STEPS][2][BLK * D];   // [64 keys][K, V]
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int unit = blockIdx.x / a.portion, matrix = blockIdx.x % a.portion, mm = a.mat0 + matrix;
  ListItem it;
  if (!list_item(a, 0, mm, unit, &it)) return;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const bf16_t* Qp = f.qkv + m.qkv;
  const int key0 = it.block * a.block, last = m.len - 1;
  TileLoader<D, 4, BLK, true> ldr;
  ldr.init(f.ld, wave, lane);
#pragma unroll
  for (int st = 0; st < STEPS; ++st) {   // (keys past the end of the sequence: zeros)
    ldr.issue(Qp + D, key0 + st * BLK, m.len, lds[st][0]);
    ldr.issue(Qp + 2 * D, key0 + st * BLK, m.len, lds[st][1]);
  }
  const unsigned in_rows = lds_address(lds) + lane_rows<D>(lane), in_cols = lds_address(lds) + lane_cols<D>(lane) + BLK * D * 2;
  const long long pairs = (long long)f.s * a.count, first = mm * pairs + it.start, out = matrix * pairs + it.start;
  const int* list = a.list + first;
  // a tile's queries are requested a tile ahead, their numbers two, and past the end too: the last one again
  const int row = wave * 32 + (lane & 31);
  int t = list[min(row, it.pairs - 1)], t_next = list[min(row + kQueries, it.pairs - 1)];
  bf16x8 qf[KS];
  auto load_queries = [&](int q) {
    const bf16_t* p = Qp + (long long)q * f.ld + g * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const bf16x8*)(p + ks * 16);
  };
  load_queries(t);
  wait_loads_and_barrier();
  for (int base = 0; base + wave * 32 < it.pairs; base += kQueries) {
    f32x16 sacc[KT];
#pragma unroll
    for (int t2 = 0; t2 < KT; ++t2) sacc[t2] = zero16();
    pipelined<KT * KS, AHEAD>([&](int n) { return rows_at<D>(in_rows, n / KS / 2 * (2 * BLK) + n / KS % 2 * 32, n % KS); },
                              [&](int n, const bf16x8& x) {
                                sacc[n / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qf[n % KS], sacc[n / KS], 0, 0, 0);
                              });
    const int limit = a.causal ? min(t, last) : last;
    t = t_next;
    load_queries(t);
    t_next = list[min(base + 2 * kQueries + row, it.pairs - 1)];
    if (__builtin_amdgcn_ballot_w64(limit < key0 + 32 * KT - 1) != 0) {
      const int reach = limit - key0 - 4 * g;
#pragma unroll
      for (int t2 = 0; t2 < KT; ++t2)
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[t2][r] = 32 * t2 + slot(r) > reach ? -INFINITY : sacc[t2][r];
    }
    float mx = -INFINITY, sum = 0.f;
#pragma unroll
    for (int t2 = 0; t2 < KT; ++t2) mx = largest(sacc[t2], mx);
    mx = halfwave_max(mx) * f.scale_log2;   // (a listed query sees the block's first key)
    const float weight = score_weight(sacc, f.scale_log2, large_scores(mx));
#pragma unroll
    for (int t2 = 0; t2 < KT; ++t2)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sacc[t2][r], weight, -mx));
        sacc[t2][r] = p;
        sum += p;
      }
    sum = halfwave_sum(sum);
    bf16x8 pf[KT][2];
#pragma unroll
    for (int t2 = 0; t2 < KT; ++t2) {
      pf[t2][0] = pack_acc<0>(sacc[t2]);
      pf[t2][1] = pack_acc<1>(sacc[t2]);
    }
    f32x16 oacc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt] = zero16();
    pipelined<2 * KT * DT, AHEAD>([&](int n) { return cols_at<D>(in_cols, n / DT / 4 * (2 * BLK) + n / DT % 4 * 16, n % DT); },
                                  [&](int n, const bf16x8& x) {
                                    const int k = n / DT;
                                    oacc[n % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, pf[k / 2][k & 1], oacc[n % DT], 0, 0, 0);
                                  });
    const long long at = out + base + wave * 32;
    const int left = min(it.pairs - base - wave * 32, 32);
    store_parts<DT>(a.rows + at * D, a.units + at, oacc, left, g, lane);
    store_ml(a.ml + at, mx, sum, left, g, lane);
  }
}

// Blocks of more than 128 keys: 64 at a time through two stages, running maximum and sum.
template <int D>
__global__ __launch_bounds__(256, 2) void selected_fwd_long_kernel(SelectedArgs a) {
  constexpr int KS = D / 16, DT = D / 32, AHEAD = 2;
  __shared__ __attribute__((aligned(1024))) bf16_t lds[2][2][BLK * D];   // [stage][K, V]
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int unit = blockIdx.x / a.portion, matrix = blockIdx.x % a.portion, mm = a.mat0 + matrix;
  ListItem it;
  if (!list_item(a, 0, mm, unit, &it)) return;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const bf16_t* Qp = f.qkv + m.qkv;
  const int key0 = it.block * a.block, last = m.len - 1;
  const int steps = (min(a.block, m.len - key0) + BLK - 1) / BLK;
  const int rounds = (it.pairs + kQueries - 1) / kQueries;
  TileLoader<D, 4, BLK, true> ldr;
  ldr.init(f.ld, wave, lane);
  auto issue = [&](int step, int st) {
    ldr.issue(Qp + D, key0 + step * BLK, m.len, lds[st][0]);
    ldr.issue(Qp + 2 * D, key0 + step * BLK, m.len, lds[st][1]);
  };
  issue(0, 0);
  const unsigned in_rows = lds_address(lds) + lane_rows<D>(lane), in_cols = lds_address(lds) + lane_cols<D>(lane) + BLK * D * 2;
  const long long pairs = (long long)f.s * a.count, first = mm * pairs + it.start, out = matrix * pairs + it.start;
  const int* list = a.list + first;
  const int row = wave * 32 + (lane & 31);
  wait_loads_and_barrier();
  int stage = 0;
  for (int round = 0; round < rounds; ++round) {
    const int base = round * kQueries, left = min(it.pairs - base - wave * 32, 32);   // (at most 0: the wavefront only keeps the barriers)
    const int t = list[min(base + row, it.pairs - 1)];
    const int limit = a.causal ? min(t, last) : last;
    bf16x8 qf[KS];
    const bf16_t* p = Qp + (long long)t * f.ld + g * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const bf16x8*)(p + ks * 16);
    f32x16 oacc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt] = zero16();
    float m_run = -INFINITY, l_run = 0.f;
    bool large = false;
    for (int step = 0; step < steps; ++step, stage ^= 1) {
      const int next = step + 1 < steps ? step + 1 : 0;
      if (step + 1 < steps || round + 1 < rounds) issue(next, stage ^ 1);
      const int kbase = key0 + step * BLK;
      if (left > 0 && __builtin_amdgcn_ballot_w64(limit >= kbase) != 0) {
        const unsigned kt = in_rows + stage * (2 * BLK * D * 2), vt = in_cols + stage * (2 * BLK * D * 2);
        f32x16 sacc[2];
        sacc[0] = zero16();
        sacc[1] = zero16();
        pipelined<2 * KS, AHEAD>([&](int n) { return rows_at<D>(kt, n / KS * 32, n % KS); },
                                 [&](int n, const bf16x8& x) {
                                   sacc[n / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qf[n % KS], sacc[n / KS], 0, 0, 0);
                                 });
        if (__builtin_amdgcn_ballot_w64(limit < kbase + BLK - 1) != 0) {
          const int reach = limit - kbase - 4 * g;
#pragma unroll
          for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
            for (int r = 0; r < 16; ++r) sacc[t2][r] = 32 * t2 + slot(r) > reach ? -INFINITY : sacc[t2][r];
        }
        const float mx = halfwave_max(largest(sacc[1], largest(sacc[0], -INFINITY))) * f.scale_log2;
        // The maximum follows the step's when that is above it by more than 8: a step's largest term is at most 2^8 then.
        const bool move = __builtin_amdgcn_ballot_w64(mx > m_run + 8.0f) != 0;
        const float m_new = move ? fmaxf(m_run, mx) : m_run;
        if (move) large = large_scores(m_new);
        const float weight = score_weight(sacc, f.scale_log2, large);
        float sum = 0.f;
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float e = __builtin_amdgcn_exp2f(fmaf(sacc[t2][r], weight, -m_new));
            sacc[t2][r] = e;
            sum += e;
          }
        sum = halfwave_sum(sum);
        if (move) {
          const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);   // (m_new is a score: the first step holds a key of every row)
          l_run *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[dt][r] *= alpha;
          m_run = m_new;
        }
        l_run += sum;
        bf16x8 pf[2][2];
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2) {
          pf[t2][0] = pack_acc<0>(sacc[t2]);
          pf[t2][1] = pack_acc<1>(sacc[t2]);
        }
        pipelined<4 * DT, AHEAD>([&](int n) { return cols_at<D>(vt, n / DT * 16, n % DT); },
                                 [&](int n, const bf16x8& x) {
                                   const int k = n / DT;
                                   oacc[n % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, pf[k / 2][k & 1], oacc[n % DT], 0, 0, 0);
                                 });
      }
      wait_loads_and_barrier();
    }
    if (left > 0) {
      const long long at = out + base + wave * 32;
      store_parts<DT>(a.rows + at * D, a.units + at, oacc, left, g, lane);
      store_ml(a.ml + at, m_run, l_run, left, g, lane);
    }
  }
}

// A query's rows to its output, a half-wavefront each.  FORWARD: weighted by their maxima, divided by the sum; the others: added, times
// 1 / sqrt(d), to dQ.  JOINT: 32 columns of a row have a scale.
// A row is 16 bytes of 16 lanes (8 of width 64), so that two or four come at a time, and four times as many are in flight.
// Bound: memory, 4.3 TB/s of scattered rows of 256 bytes forward, 5 and 6.8 TB/s backward (width 128, 64), where the cache still holds some.
template <int D, bool FORWARD, bool JOINT>
__global__ __launch_bounds__(256) void selected_combine_kernel(SelectedArgs a) {
  constexpr int LANES = D / 8, PARTS = 32 / LANES;
  typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
  const FusedArgs& f = a.f;
  const int half = threadIdx.x >> 5, n = threadIdx.x & 31, part = n / LANES, c = n % LANES;
  const int mm = a.mat0 + blockIdx.y;
  const int t = blockIdx.x * 8 + half;
  const bool inside = t < f.s;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const long long rows = (long long)blockIdx.y * f.s * a.count;
  const int* places = a.places + (m.vec + t) * a.count;
  static_assert(kMostCount <= 64, "two entries a lane");
  // entries n and n + 32
  int place[2];
  float weight[2];
  float2 ml[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) place[k] = inside && n + 32 * k < a.count ? places[n + 32 * k] : -1;
  // rows of entries e0 .. e0 + 4 PARTS - 1; the first ones are on their way while the weights are computed
  f16x8 x[4];
  float unit[4];
  auto load_rows = [&](int e0) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int e = e0 + u * PARTS + part;
      const int p0 = __shfl(place[0], e & 31, 32), p1 = __shfl(place[1], e & 31, 32);
      const int p = e < 32 ? p0 : e < 64 ? p1 : -1;
#pragma unroll
      for (int k = 0; k < 8; ++k) x[u][k] = 0;
      if (p >= 0) x[u] = *(const f16x8*)(a.rows + (rows + p) * D + c * 8);
      if (JOINT) unit[u] = p >= 0 ? a.units[(rows + p) * (D / 32) + c / 4] : 0.f;
    }
  };
  load_rows(0);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    weight[k] = !JOINT && place[k] >= 0 ? a.units[rows + place[k]] : 0.f;
    if (FORWARD) ml[k] = place[k] >= 0 ? a.ml[rows + place[k]] : make_float2(-INFINITY, 0.f);
  }
  float total = 0.f, top = -INFINITY;
  if (FORWARD) {
    top = fmaxf(ml[0].x, ml[1].x);
#pragma unroll
    for (int step = 1; step < 32; step <<= 1) top = fmaxf(top, __shfl_xor(top, step));
    const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float w = __builtin_amdgcn_exp2f(ml[k].x - from);   // (of no pair: 0)
      total += w * ml[k].y;
      weight[k] *= w;
    }
#pragma unroll
    for (int step = 1; step < 32; step <<= 1) total += __shfl_xor(total, step);
    const float inverse = total > 0.f ? 1.0f / total : 0.f;
    weight[0] *= inverse;
    weight[1] *= inverse;
  }
  float sum[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) sum[k] = 0.f;
  for (int e0 = 0; e0 < a.count; e0 += 4 * PARTS) {
    if (e0 > 0) load_rows(e0);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int e = e0 + u * PARTS + part;
      const float w0 = __shfl(weight[0], e & 31, 32), w1 = __shfl(weight[1], e & 31, 32);
      const float w = JOINT ? unit[u] : e < 32 ? w0 : w1;
#pragma unroll
      for (int k = 0; k < 8; ++k) sum[k] = fmaf(w, (float)x[u][k], sum[k]);
    }
  }
#pragma unroll
  for (int step = LANES; step < 32; step <<= 1)
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] += __shfl_xor(sum[k], step);
  if (inside && part == 0) {
    bf16_t* to = FORWARD ? f.attn + m.attn + (long long)t * f.ldo : f.d_qkv + m.qkv + (long long)t * f.ld;
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = FORWARD ? pack2_bf16(sum[2 * k], sum[2 * k + 1]) : pack2_bf16(sum[2 * k] * f.scale, sum[2 * k + 1] * f.scale);
    *(u32x4*)(to + 8 * c) = w;
  }
  if (FORWARD && inside && n == 0) f.lse[m.vec + t] = total > 0.f ? (top + __log2f(total)) * LN2 : -INFINITY;
}

SelectedArgs make_args(const AttnSelectedDesc& b) {
  const AttnFusedDesc& d = b.base;
  SelectedArgs a = {};
  FusedArgs& f = a.f;
  f.qkv = (const bf16_t*)d.qkv; f.attn = (bf16_t*)d.attn; f.lse = d.lse;
  f.d_attn = (const bf16_t*)d.d_attn; f.d_qkv = (bf16_t*)d.d_qkv;
  f.s = d.s; f.nh = d.nh; f.ld = d.ld; f.ldo = d.ldo;
  f.dev_qkv = d.dev_qkv; f.dev_attn = d.dev_attn;
  f.scale = 1.0f / sqrtf((float)d.d);
  f.scale_log2 = (float)(1.4426950408889634 / sqrt((double)d.d));
  a.selected = b.selected; a.lengths = b.lengths;
  a.nb = d.nb; a.nmat = d.nb * d.nh; a.q = b.q; a.dev0 = b.dev0; a.causal = d.causal;
  a.block = b.block; a.count = b.count; a.blocks = (d.s + b.block - 1) / b.block;
  a.by_steps = b.block == 64 ? 0u : (unsigned)(((1ull << 32) + b.block / 64 - 1) / (b.block / 64));
  return a;
}

size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }

// the workspace's parts into the arguments
SelectedArgs with_workspace(const AttnSelectedDesc& b, const SelectedPlan& p, bool bwd) {
  SelectedArgs a = make_args(b);
  a.mats = p.mats; a.chunks = p.chunks; a.mask_words = p.mask_words;
  char* at = (char*)b.ws;
  auto take = [&](size_t bytes) {
    char* r = at;
    at += bytes;
    return r;
  };
  a.f.delta = (float*)take(p.delta);
  a.mask = (unsigned*)take(p.mask);
  a.counts = (int*)take(p.counts);
  a.first_item = (int*)take(p.first_item);
  for (int k = 0; k < 2; ++k) {
    a.seg[k] = p.seg[k];
    a.most[k] = p.most[k];
    a.items[k] = (i32x4_t*)take(p.items[k]);
  }
  if (!bwd) a.items[1] = nullptr;
  if (p.joint) a.items[0] = nullptr;
  a.list = (int*)take(p.list);
  a.places = (int*)take(p.places);
  a.rows = (f16_t*)take(p.rows);
  a.units = (float*)take(p.units);
  a.ml = (float2*)take(p.ml);
  a.key_rows = p.joint ? (float*)take(p.keys) : (float*)a.rows;   // (otherwise dK and dV come when the rows of dQ are done with)
  return a;
}

void launch_lists(const SelectedArgs& a, int d, bool bwd, hipStream_t st) {
  const size_t bits = (size_t)kWords * a.blocks * sizeof(unsigned);   // at most 32 KiB
  const dim3 grid(a.chunks, a.mats);
  if (!bwd) list_count_kernel<0><<<grid, kListChunk, bits, st>>>(a);
  else if (d == 64) list_count_kernel<64><<<grid, kListChunk, bits, st>>>(a);
  else list_count_kernel<128><<<grid, kListChunk, bits, st>>>(a);
  const size_t fill = 2 * bits + kListChunk / 64 * sizeof(int);
  const bool summed = a.chunks > kFewChunks;
  if (summed) list_sums_kernel<<<dim3((a.blocks + 63) / 64, a.mats), 64 * kSumWaves, 0, st>>>(a);
  auto kernel = summed ? list_fill_kernel<true> : list_fill_kernel<false>;
  if (fill > 65536) (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)fill);
  kernel<<<grid, kListChunk, fill, st>>>(a);
}

template <int D>
void fwd_launch(const SelectedArgs& a, hipStream_t st) {
  const int portion = a.portion;
  const dim3 grid(a.most[0] * portion);
  if (a.block == 64) selected_fwd_kernel<D, 2><<<grid, 256, 0, st>>>(a);
  else if (a.block == 128) selected_fwd_kernel<D, 4><<<grid, 256, 0, st>>>(a);
  else selected_fwd_long_kernel<D><<<grid, 256, 0, st>>>(a);
  selected_combine_kernel<D, true, false><<<dim3((a.f.s + 7) / 8, portion), 256, 0, st>>>(a);
}

}  // namespace

void launch_selected_dq_combine(const SelectedArgs& a, int d, bool joint, hipStream_t st) {
  const dim3 grid((a.f.s + 7) / 8, a.portion);
  if (joint && d == 64) selected_combine_kernel<64, false, true><<<grid, 256, 0, st>>>(a);
  else if (joint) selected_combine_kernel<128, false, true><<<grid, 256, 0, st>>>(a);
  else if (d == 64) selected_combine_kernel<64, false, false><<<grid, 256, 0, st>>>(a);
  else selected_combine_kernel<128, false, false><<<grid, 256, 0, st>>>(a);
}

// Which form: the one that should take less time, by what both have taken.  The masked one computes all pairs of queries and keys (causal: half of
// them) at a rate, and its longest workgroup walks over all keys.  Lists compute the chosen pairs at more each, as a block's part of a row goes
// through memory once a block, and have a price a call and a query for the lists and the sums.
// Measured, us, masked / lists, causal, 16 (sequence, head)s unless said otherwise; forward, backward:
//   width 128: 8192 queries, blocks of 128, 4 chosen 341 / 125, 1086 / 223; 8 296 / 195, 1068 / 354; 12 285 / 288, 1055 / 471; 16 284 / 348, 1064 / 569;
//   16384, 256, 8 1091 / 610, 4423 / 1283; 4096, 64, 4 79 / 60, 276 / 122; 14 80 / 138, 295 / 226; 4096, 512, 2 76 / 82, 291 / 210;
//   one of 1024, 64, 4 20 / 23, 39 / 48; 8192, 128, 24 112 / 61, 212 / 105; no mask, 4096, 128, 10 142 / 125, 541 / 208
//   width 64: 8192, 128, 8 158 / 111, 609 / 178; 16 162 / 193, 616 / 305; 16384, 256, 8 579 / 324, 2479 / 744; 4096, 64, 8 55 / 59, 175 / 85; 4096, 512, 2
//   51 / 64, 171 / 145; one of 1024, 64, 4 12 / 23, 25 / 36; 8192, 128, 24 66 / 50, 132 / 84
// (104 such pairs: the form taken was never more than 1.08 times the other one's time.  Queries are those of one device's matrices, whatever the
// launch covers: the forms add up in different orders.)
struct FormCost {
  double masked_pair, masked_call, masked_row;          // us: a pair; the longest workgroup's start and each row that it walks over
  double lists_call, lists_query, lists_pair, by_block; // us; a chosen pair, in masked ones, lists_pair + by_block / block
};
constexpr FormCost kFormCost[3][2] = {   // [forward, backward of blocks of 64 and 128, of larger ones][width 64, 128]
    {{2.8e-7, 6, 0.008, 25, 1.2e-4, 1.6, 128}, {5.0e-7, 6, 0.0138, 25, 1.2e-4, 1.55, 137}},
    {{1.1e-6, 10, 0.015, 38, 1.4e-4, 0.82, 18}, {1.9e-6, 12, 0.024, 46, 3.6e-4, 0.62, 56}},
    {{1.1e-6, 10, 0.015, 38, 3e-4, 1.05, 30}, {1.9e-6, 12, 0.024, 46, 4e-4, 0.98, 60}}};
bool attn_selected_masked(const AttnSelectedDesc& b, bool bwd) {
  const AttnFusedDesc& d = b.base;
  const double blocks = (d.s + b.block - 1) / b.block, k = b.count < blocks ? b.count : blocks, B = b.block;
  if (blocks > kMaskedBlocks) return false;
  const int forced = g_form.load(std::memory_order_relaxed);
  if (forced >= 0) return forced != 0;
  FormCost c = kFormCost[!bwd ? 0 : b.block <= 128 ? 1 : 2][d.d == 128];
  if (bwd && d.d == 128 && b.block > 128 && b.block % 128 != 0) c.by_block = 92;   // (dK and dV of 64 keys at a time)
  const double all = d.causal ? blocks * (blocks + 1) / 2 : blocks * blocks;
  const double chosen = d.causal ? k * (k + 1) / 2 + (blocks - k) * k : blocks * k;
  const double matrices = (double)d.nb * d.nh, pairs = matrices * B * (d.s < b.block ? d.s : B);   // of queries and keys, of a pair of blocks
  const double masked = hypot(all * pairs * c.masked_pair, c.masked_call + d.s * c.masked_row);   // (the longest one counts where few run)
  const double lists = c.lists_call + matrices * d.s * c.lists_query + chosen * pairs * c.masked_pair * (c.lists_pair + c.by_block / B);
  return masked <= lists;
}
void attn_selected_set_form(int form) { g_form.store(form, std::memory_order_relaxed); }

void attn_selected_plan(const AttnSelectedDesc& b, bool bwd, SelectedPlan* out) {
  SelectedPlan p = {};
  const AttnFusedDesc& d = b.base;
  const size_t blocks = (d.s + b.block - 1) / b.block, pairs = (size_t)d.s * b.count;
  p.mats = d.ndev * d.nb * d.nh;
  const size_t mats = p.mats;
  p.masked = attn_selected_masked(b, bwd);
  p.delta = round256(mats * d.s * 4);
  if (p.masked) {
    p.mask_words = (d.s + 31) / 32;
    p.mask = round256(mats * blocks * p.mask_words * 4);
    p.total = p.delta + p.mask;
    *out = p;
    return;
  }
  p.chunks = (d.s + kListChunk - 1) / kListChunk;
  p.joint = bwd && b.block <= 128;
  // Pieces of a block's list: longer ones are fewer sums of dK and dV through memory, shorter ones fill the card.  Backward, us, with pieces chosen
  // so that a device's pairs make 256 / 384 / 512 of them and more: width 128, one of 8192 queries, 8 blocks of 128 69 / 63 / 64; 24 104 / 103 / 117; one of
  // 16384, 16 144 / 109 / 117; two of 8192, 8 93 / 79 / 85; width 64, one of 16384, 16 118 / 85 / 94; at most 2048 queries: 16 of 4096 x 128, 8 blocks
  // 215 with 1024, 178, 175 with 4096.  (One device's pairs: sums depend on it.)
  const size_t all_pairs = pairs * d.nb * d.nh;
  p.seg[1] = 256;
  while (p.seg[1] < 2048 && all_pairs / p.seg[1] >= 384) p.seg[1] *= 2;
  const size_t row_bytes = pairs * (d.d * 2 + (p.joint ? d.d / 8 : 12)), key_row = d.d * 8;   // of a matrix; of a key
  // A piece leaves sums of all of its block's keys, whatever its length: where those of one matrix would be more than a portion and more than a
  // block's only piece and its queries' rows take, pieces are longer.  (One of 262144 x 128, 4 of 64 blocks of 4096: workspace 2317 MiB and backward 7.6 ms
  // without this, 777 MiB and 7.0 ms.)
  while ((blocks + pairs / p.seg[1]) * b.block * key_row > kPortion && pairs / p.seg[1] * b.block * key_row > row_bytes) p.seg[1] *= 2;
  p.most[1] = (int)(blocks + pairs / p.seg[1]);
  const size_t key_bytes = p.most[1] * b.block * key_row;
  auto fit = [&](size_t bytes) { return (int)(kPortion / bytes < 1 ? 1 : kPortion / bytes > mats ? mats : kPortion / bytes); };
  p.portion = fit(p.joint ? row_bytes + key_bytes : row_bytes);
  p.key_portion = p.joint ? p.portion : fit(key_bytes);
  // Pieces of a list as long as some 2000 of them leave no compute unit without work, 256 to 1024 rows (no bits depend on it): a launch of 10^6
  // pairs (two matrices of 32768 queries, 16 blocks each) 1006 us with 256 in all, 932 with 1024; 2.4 * 10^6 of width 64 395 with 256, 376 with 512.
  p.seg[0] = 256;
  while (p.seg[0] < 1024 && p.portion * pairs / p.seg[0] >= 4096) p.seg[0] *= 2;
  p.most[0] = (int)(blocks + pairs / p.seg[0]);
  p.counts = round256(mats * (p.chunks + 1) * blocks * 4);
  p.first_item = round256(2 * mats * (blocks + 1) * 4);
  p.items[0] = p.joint ? 0 : round256(mats * p.most[0] * 16);
  p.items[1] = bwd ? round256(mats * p.most[1] * 16) : 0;
  p.list = p.places = round256(mats * pairs * 4);
  const size_t keys = bwd ? p.key_portion * key_bytes : 0;
  p.rows = round256(p.portion * pairs * d.d * 2);
  p.units = round256(p.portion * pairs * (p.joint ? d.d / 32 : 1) * 4);
  if (p.joint) p.keys = round256(keys);
  else if (keys > p.rows + p.units) p.units = round256(keys - p.rows);   // (in the place of both, when dQ is done)
  p.ml = bwd ? 0 : round256(p.portion * pairs * 8);
  p.total = p.delta + p.counts + p.first_item + p.items[0] + p.items[1] + p.list + p.places + p.rows + p.units + p.ml + p.keys;
  *out = p;
}
size_t attn_selected_ws_bytes(const AttnSelectedDesc& b) {
  SelectedPlan fwd, bwd;
  attn_selected_plan(b, false, &fwd);
  attn_selected_plan(b, true, &bwd);
  return fwd.total > bwd.total ? fwd.total : bwd.total;
}

int launch_attn_selected_fwd(const AttnSelectedDesc& b, hipStream_t st) {
  SelectedPlan p;
  attn_selected_plan(b, false, &p);
  SelectedArgs a = with_workspace(b, p, false);
  if (p.masked) {
    launch_selected_masked(a, p.mats, b.base.d, false, st);
    return hip_launch_status();
  }
  launch_lists(a, b.base.d, false, st);
  for (a.mat0 = 0; a.mat0 < p.mats; a.mat0 += p.portion) {
    a.portion = min(p.portion, p.mats - a.mat0);
    if (b.base.d == 64) fwd_launch<64>(a, st);
    else fwd_launch<128>(a, st);
    if (const int rc = hip_launch_status()) return rc;
  }
  return OPTIMUS_OK;
}

int launch_attn_selected_bwd(const AttnSelectedDesc& b, hipStream_t st) {
  SelectedPlan p;
  attn_selected_plan(b, true, &p);
  const SelectedArgs a = with_workspace(b, p, true);
  if (p.masked) {
    launch_selected_masked(a, p.mats, b.base.d, true, st);
    return hip_launch_status();
  }
  launch_lists(a, b.base.d, true, st);
  return launch_selected_bwd_kernels(a, p, b.base.d, st);
}

}  // namespace optimus
