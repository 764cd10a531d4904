// Softmax cross entropy of a microbatch's labelled rows over a vocabulary
// (vocab_loss_forward, vocab_loss_backward of include/flowpool_train.h).
//
// The labelled rows are listed first and gathered into consecutive rows (in a
// vision-language microbatch three rows in four are image rows and have no
// label; every product below would otherwise be four times as large). How many
// there are is known on the device alone: kernels take the count from memory
// and workgroups without a tile end at once.
//
// Forward: one product, 2 n V H operations. The logits of a tile stay in the
// matrix instructions' sums; its epilogue takes each row's maximum and sum of
// exponentials over the tile's 256 classes, and k_lse joins those of all
// tiles. The label's own class is left out of them, so that the loss is
// log(1 + sum of the others' exp(z - z_label)), which keeps its bits where the
// label is nearly certain; lse - z_label would lose them (a loss of 0.005 at
// logits of 16: relative error 1e-4). Tiles have classes along the lane's own values and rows across lanes,
// so the reduction is nearly all within a lane.
//
// Backward: pieces of the vocabulary, each three products: the logits again,
// with the epilogue making exp(z - lse), rounded to 16 bits, and 0 at the label;
// then its products with the piece's weight (added up in f32 over pieces) and
// with the rows (the piece's rows of dweight). A piece has as many classes as
// the labelled rows leave room for, so the fewer rows there are, the fewer
// pieces; the host enqueues as many as all rows would make, and those past the
// vocabulary end at once. The gradient at a row's label is known once all pieces
// are done: then k_finish adds its parts of dx and of the classes that are
// labels, whose sums waited in f32 (a counting sort of the labelled rows says
// which rows a class has).
//
// Measured (bf16): the loss of 4096 labelled rows over 152064 x 4096 3.90 ms, 1310
// TFLOP/s; a step of 4096 over 152064 x 3584 14.6 ms, of 8192 over 128256 x 5120
// 33.3 ms, 1220 and 1290 TFLOP/s of what is multiplied (the logits twice). A large
// library product reaches 1320 to 1520 here. The matrix cores work in 0.71 of the
// cycles, at the 1.7 GHz that the power allows, while the L2s feed the LDS at 10
// TB/s; with the loads left out the loop runs at 1690 to 2000 TFLOP/s.

#include "gemm.h"

#include <algorithm>

namespace fp {
namespace {

constexpr int kMaxHidden = 12288;
constexpr int64_t kMaxRows = 1 << 22;
constexpr int64_t kMaxStride = 1 << 22;         // of weight, so that a tile's rows lie within 32-bit offsets
constexpr int32_t kMaxVocab = 1 << 22;
constexpr int kCUs = 256;
constexpr int kMaxSplits = 16;                   // of dx's sum over a piece's classes
// Elements of a piece's gradient of the logits, about: 1 GiB. With twice as many a
// step of 4096 rows over 152064 x 3584 takes 14.3 ms for 14.5, but one of 8192 over
// 128256 x 5120 33.7 for 33.3 (one machine, in turn); with half, 1 to 2 % more.
constexpr int64_t kPieceElements = 1ll << 29;

__host__ __device__ constexpr int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// ------------------------------------------------------------------ rows

// Lists the labelled rows in order: rows[i] is the i-th one's index, picks[i]
// its label, slot[t] the place of row t or -1. One workgroup, 4096 labels a
// step.
__global__ __launch_bounds__(1024) void k_label_rows(const int32_t* labels, int32_t n_rows, int32_t vocab, int32_t* rows, int32_t* picks,
                                                     int32_t* slot, int32_t* count, int32_t* count_out, float* lse, u32x4* zeros) {
  __shared__ int32_t waves[16];
  __shared__ int32_t total;
  if (threadIdx.x == 0) total = 0;
  if (threadIdx.x < 16) zeros[threadIdx.x] = u32x4{0, 0, 0, 0};
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int32_t base = 0; base < n_rows; base += 4096) {
    const int32_t t0 = base + threadIdx.x * 4;
    int32_t label[4];
    bool has[4];
    int32_t mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      label[e] = t0 + e < n_rows ? labels[t0 + e] : -1;
      has[e] = (uint32_t)label[e] < (uint32_t)vocab;
      mine += has[e];
    }
    int32_t before = mine;                       // inclusive over the wave
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int32_t o = __shfl_up(before, d);
      if (lane >= d) before += o;
    }
    if (lane == 63) waves[wave] = before;
    __syncthreads();
    int32_t at = total + before - mine, sum = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w < wave) at += waves[w];
      sum += waves[w];
    }
    __syncthreads();
    if (threadIdx.x == 0) total += sum;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (t0 + e >= n_rows) break;
      if (slot) slot[t0 + e] = has[e] ? at : -1;
      if (lse && !has[e]) lse[t0 + e] = 0.f;
      if (has[e]) {
        rows[at] = t0 + e;
        picks[at++] = label[e];
      }
    }
  }
  if (threadIdx.x == 0) {
    *count = total;
    if (count_out) *count_out = total;
  }
}

// The labelled rows by class, for the sums of each class's own rows.
struct Classes {
  int32_t* order;               // [labelled rows]: the rows, by class and then by number
  int32_t* many;                // of the class that begins at this place of order: its rows; 0 at the places behind
  int32_t* begin;               // [vocab]: a class's place in order, -1 for one that is no row's label
};

// Orders the rows of the `tile`-th 256 classes: a stable counting sort, whose
// place among all classes is the number of rows below the tile. Each of 16 waves
// has a 16th of the rows, in their order, and loads 8 of a lane at once: few
// classes are few workgroups, whose time is a wave's chain of steps (32768 rows
// over 1000 classes: 100 us with 4 waves).
constexpr int kOrderWaves = 16;
__device__ __forceinline__ void order_classes(const Classes& o, int32_t tile, const int32_t* picks, int32_t n, int32_t vocab) {
  constexpr int kAtOnce = 8;
  __shared__ int32_t at[kOrderWaves][256], first[256], total[256], sums[kOrderWaves], ends[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c0 = threadIdx.x;
#pragma unroll
  for (int k = 0; k < kOrderWaves * 256; k += kOrderWaves * 64) (&at[0][0])[k + threadIdx.x] = 0;
  __syncthreads();
  const int32_t share = (n + kOrderWaves * 64 - 1) / (kOrderWaves * 64) * 64, from = min(wave * share, n), to = min(from + share, n);
  const int32_t v0 = tile * 256;
  int32_t below = 0;
  for (int32_t i = from + lane; i < to; i += 64 * kAtOnce) {
    int32_t c[kAtOnce];
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e) c[e] = i + 64 * e < to ? picks[i + 64 * e] - v0 : 256;
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e) {
      below += c[e] < 0;
      if ((uint32_t)c[e] < 256u) atomicAdd(&at[wave][c[e]], 1);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) below += __shfl_xor(below, d);
  if (lane == 0) sums[wave] = below;
  __syncthreads();
  int32_t mine = 0, before = 0;                  // rows of class c0; of it and the wave's classes before it
  if (c0 < 256) {
#pragma unroll
    for (int w = 0; w < kOrderWaves; ++w) mine += at[w][c0];
    before = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int32_t other = __shfl_up(before, d);
      if (lane >= d) before += other;
    }
    if (lane == 63) ends[wave] = before;
  }
  __syncthreads();
  if (c0 < 256) {
    int32_t place = before - mine;
#pragma unroll
    for (int w = 0; w < kOrderWaves; ++w) place += sums[w];
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (w < wave) place += ends[w];
    first[c0] = place;
    total[c0] = mine;
    if (v0 + c0 < vocab) o.begin[v0 + c0] = mine ? place : -1;
#pragma unroll
    for (int w = 0; w < kOrderWaves; ++w) {
      const int32_t here = at[w][c0];
      at[w][c0] = place;
      place += here;
    }
  }
  __syncthreads();
  for (int32_t base = from; base < to; base += 64 * kAtOnce) {
    int32_t c[kAtOnce];
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e) c[e] = base + 64 * e + lane < to ? picks[base + 64 * e + lane] - v0 : 256;
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e) {
      const bool in = (uint32_t)c[e] < 256u;
      uint64_t same = __ballot(in);              // lanes with this lane's class
      if (!same) continue;
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const bool bit = c[e] >> b & 1;
        const uint64_t set = __ballot(bit);
        same &= bit ? set : ~set;
      }
      const int32_t rank = __popcll(same & ((1ull << lane) - 1));
      if (in) {
        const int32_t to_place = at[wave][c[e]] + rank;
        o.order[to_place] = base + 64 * e + lane;
        o.many[to_place] = to_place == first[c[e]] ? total[c[e]] : 0;
      }
      wave_order();
      if (in && rank == 0) at[wave][c[e]] += __popcll(same);
      wave_order();
    }
  }
}

// Gathers the labelled rows into xc [.., ld], zeros from hidden to ld, and with
// them (backward) their lse. Past the last row nothing is written: those rows
// of a tile are read as the last one, and left out of every result. A workgroup
// has 4 rows, 256 threads each; the first `tiles` order the rows by class, a tile
// of classes each.
template <class T>
__global__ __launch_bounds__(1024) void k_gather_rows(const T* x, int64_t x_stride, const int32_t* rows, const int32_t* count,
                                                      int32_t hidden, int32_t ld, T* xc, const float* lse, float* lses, int32_t tiles,
                                                      const int32_t* picks, int32_t vocab, Classes classes) {
  if ((int32_t)blockIdx.x < tiles) return order_classes(classes, blockIdx.x, picks, *count, vocab);
  const int32_t i = (blockIdx.x - tiles) * 4 + (threadIdx.x >> 8), t = threadIdx.x & 255;
  if (i >= *count) return;
  if (lse && t == 0) lses[i] = lse[rows[i]];
  const T* src = x + (int64_t)rows[i] * x_stride;
  T* dst = xc + (int64_t)i * ld;
  for (int32_t c = t * 8; c < ld; c += 256 * 8) {
    u32x4 v = {0, 0, 0, 0};
    if (c < hidden) v = *(const u32x4*)(src + c);
    *(u32x4*)(dst + c) = v;
  }
}

// ------------------------------------------------------------------ products

struct LossArgs {
  const int32_t* count;
  const int32_t* picks;         // the labelled rows' labels
  const void* zeros;
  const void* xc;               // labelled rows, ld elements apart
  const void* weight;
  int64_t weight_ld;
  int32_t ld;                   // of xc
  int32_t hidden, vocab;
  // forward
  float2* part;                 // [tiles of classes][rows]: maximum, sum of exponentials
  int32_t part_ld;
  float* picked;                // logit of each row's label
  // backward
  const float* lses;            // of the labelled rows
  void* g;                      // the piece's gradient of the logits [rows][classes of a piece]
  int64_t room;                 // elements of g
  float* others;                // [128 classes][rows]: sums of the other classes' gradients
  int32_t others_ld;
  const float* own;             // each row's gradient at its label
  int32_t u;                    // the piece's number
  float* sum;                   // dx's sums [split][rows][ld]
  int64_t sum_rows;             // of all splits
  const int32_t* begin;         // as in Classes
  float* side;                  // dweight's sums of classes that are labels, at their place of order [rows][ld]
};

// Classes of a piece with n labelled rows: whole tiles, pieces as even as that
// allows.
__host__ __device__ inline int32_t piece_of(int64_t n, int32_t vocab, int64_t room) {
  const int64_t rows = up(n < 1 ? 1 : n, kTile), tiles = ((int64_t)vocab + kTile - 1) / kTile;
  const int64_t fit = room / (rows * kTile), most = fit < 1 ? 1 : fit < tiles ? fit : tiles;
  const int64_t pieces = (tiles + most - 1) / most;
  return (int32_t)((tiles + pieces - 1) / pieces * kTile);
}

struct Piece {
  int32_t ld, first, classes;   // of a piece; the piece's first class, and how many it has (0 or less: none)
};
__device__ __forceinline__ Piece piece(const LossArgs& a, int32_t n) {
  const int32_t ld = uniform(piece_of(n, a.vocab, a.room));
  const int64_t first = (int64_t)a.u * ld;
  return first < a.vocab ? Piece{ld, (int32_t)first, min(ld, a.vocab - (int32_t)first)} : Piece{ld, 0, 0};
}

constexpr float kLog2e = 1.4426950408889634f;
// The gradient of the logits is held as 2^kLift times itself: over a large
// vocabulary most probabilities are below 2^-14, where f16 loses its bits.
template <class T>
constexpr int kLift = __is_same(T, f16) ? 12 : 0;

// Combines (maximum, sum of exp(z - maximum)) pairs.
__device__ __forceinline__ void join(float& m, float& s, float om, float os) {
  const float n = fmaxf(m, om);
  const float a = m == n ? 1.f : __builtin_amdgcn_exp2f((m - n) * kLog2e), b = om == n ? 1.f : __builtin_amdgcn_exp2f((om - n) * kLog2e);
  s = s * a + os * b;
  m = n;
}

// Walks over the tiles of a workgroup: begin(id) starts a tile's loads, take()
// keeps what begin() found out for the results of the tile whose sums are
// ready, and finish(id, acc) takes those while the next tile's loads run.
template <class G, class Begin, class Take, class Finish>
__device__ __forceinline__ void walk(int32_t tiles, int32_t lds, G& g, Begin begin, Take take, Finish finish) {
  int32_t id = blockIdx.x;
  if (id >= tiles) return;
  begin(id);
  for (;;) {
    typename G::Sums acc;
    g.run(lds, acc);
    take();
    const int32_t next = id + gridDim.x;
    if (next < tiles) begin(next);
    finish(id, acc);
    if (next >= tiles) return;
    id = next;
  }
}

// The logits' products by narrow tiles of 32 kJ rows, a wave 64 classes; tile
// `id` is classes id % pt, rows id / pt.
template <class T, int kJ>
__device__ __forceinline__ void narrow_forward(const LossArgs& a, int32_t n, char* lds) {
  const Operand16 P{a.weight, a.weight_ld, a.vocab, a.hidden}, Q{a.xc, a.ld, n, a.hidden};
  Narrow<T, false, kJ> g;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t pt = (a.vocab + kTile - 1) / kTile, qt = (n + 32 * kJ - 1) / (32 * kJ);
  int32_t next[kJ], pick[kJ];      // the rows' labels: of the tile whose loads are under way, of the one that is ready
  const auto begin = [&](int32_t id) {
    const int32_t tq = id / pt * (32 * kJ), tp = id % pt;
#pragma unroll
    for (int j = 0; j < kJ; ++j) next[j] = a.picks[min(tq + lane_q() + j * 32, n - 1)];
    g.start(P, Q, a.zeros, tp * kTile, tq, tp, lds_address(lds));
  };
  const auto take = [&] {
#pragma unroll
    for (int j = 0; j < kJ; ++j) pick[j] = next[j];
  };
  const auto finish = [&](int32_t id, NarrowAcc<kJ>& acc) {
    const int32_t tq = id / pt * (32 * kJ), tp = id % pt, v0 = tp * kTile + wave * 64 + lane_p();
    float2* const other = (float2*)(lds + kOwnAt);        // [wave][row]
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      float z[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int32_t v = v0 + i / 4 * 8 + i % 4;
        z[i] = sum_of(acc, i >> 4, j, i & 15);
        if (v == pick[j] && tq + lane_q() + j * 32 < n) a.picked[tq + lane_q() + j * 32] = z[i];
        z[i] = v < a.vocab && v != pick[j] ? z[i] : -__builtin_inff();
      }
      float x = z[0];
#pragma unroll
      for (int i = 1; i < 32; ++i) x = fmaxf(x, z[i]);
      const float lift = x == -__builtin_inff() ? 0.f : -x * kLog2e;
      float y[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 32; ++i) y[i & 1] += __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], kLog2e, lift));
      float m = x, s = y[0] + y[1];
      const float om = __shfl_xor(m, 32), os = __shfl_xor(s, 32);
      join(m, s, om, os);
      if (lane < 32) other[wave * (32 * kJ) + j * 32 + lane] = make_float2(m, s);
    }
    barrier();
    if ((int)threadIdx.x < min(n - tq, 32 * kJ)) {
      float2 o = other[threadIdx.x];
      float m = o.x, s = o.y;
#pragma unroll
      for (int w = 1; w < 4; ++w) {
        o = other[w * (32 * kJ) + threadIdx.x];
        join(m, s, o.x, o.y);
      }
      a.part[(int64_t)tp * a.part_ld + tq + threadIdx.x] = make_float2(m, s);
    }
  };
  walk(pt * qt, lds_address(lds), g, begin, take, finish);
}

// Rows of a tile, with n labelled rows and pt tiles of the other operand: few
// rows take a narrow tile, and so do more of them while narrow tiles leave half
// of the compute units idle. A loss of 762 rows over 1000 x 5120 takes 115 us by
// tiles of 256 rows, 84 of 128, 73 of 64; at the limit, 256 rows over 16000 x
// 4096, 91, 75 and 94; past it, 200 over 32003 x 4096, 96, 103 and 104.
__device__ __forceinline__ int32_t rows_of_tile(int32_t n, int32_t pt) {
  if (n <= 64 || (int64_t)pt * ((n + 63) / 64) <= kCUs / 2) return 64;
  if (n <= 128 || (int64_t)pt * ((n + 127) / 128) <= kCUs / 2) return 128;
  return kTile;
}
// Calls f(kJ) for a narrow tile.
template <class F>
__device__ __forceinline__ bool if_narrow(int32_t rows, F f) {
  if (rows == kTile) return false;
  if (rows == 128)
    f(std::integral_constant<int, 4>{});
  else
    f(std::integral_constant<int, 2>{});
  return true;
}

template <class T>
__global__ __launch_bounds__(kGemmThreads, 1) void k_logits_forward(LossArgs a) {
  __shared__ __align__(1024) char lds[kGemmLds];
  const int32_t n = uniform(*a.count);
  const int32_t pt = (a.vocab + kTile - 1) / kTile;
  if (n == 0 || if_narrow(rows_of_tile(n, pt), [&](auto j) { narrow_forward<T, decltype(j)::value>(a, n, lds); })) return;
  const int32_t qt = (n + kTile - 1) / kTile;
  const Operand16 P{a.weight, a.weight_ld, a.vocab, a.hidden}, Q{a.xc, a.ld, n, a.hidden};
  Gemm<T, false, false> g;
  int32_t pick[4] = {};            // of the tile whose loads are under way
  int32_t at[4], tp, tq, np, nq;   // at: the label's place among this lane's classes
  const auto begin = [&](int32_t id) {
    tile_of(id, pt, qt, &np, &nq);
#pragma unroll
    for (int j = 0; j < 4; ++j) pick[j] = a.picks[min(nq + wave_q() + lane_q() + j * 32, n - 1)];
    g.start(P, Q, a.zeros, np, nq, lds_address(lds));
  };
  const auto take = [&] {
    tp = np, tq = nq;
#pragma unroll
    for (int j = 0; j < 4; ++j) at[j] = tq + wave_q() + lane_q() + j * 32 < n ? pick[j] - (tp + wave_p() + lane_p()) : -1;
  };
  const auto finish = [&](int32_t, Acc& acc) {
    const int lane = threadIdx.x & 63;
    const int32_t v0 = tp + wave_p() + lane_p(), t0 = tq + wave_q() + lane_q();
    float2* const other = (float2*)(lds + kOwnAt);        // [256] of the waves of the upper classes
    float m[4], s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float z[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) z[i] = sum_of(acc, i >> 4, j, i & 15);
      if (tp + kTile > a.vocab) {
#pragma unroll
        for (int i = 0; i < 64; ++i)
          if (v0 + i / 4 * 8 + i % 4 >= a.vocab) z[i] = -__builtin_inff();
      }
      if (at[j] >= 0 && at[j] < 128 && (at[j] & 7) < 4) {
        float picked = 0.f;
#pragma unroll
        for (int i = 0; i < 64; ++i) {
          const bool is = at[j] == i / 4 * 8 + i % 4;
          picked = is ? z[i] : picked;
          z[i] = is ? -__builtin_inff() : z[i];
        }
        a.picked[t0 + j * 32] = picked;
      }
      float x = z[0];
#pragma unroll
      for (int i = 1; i < 64; ++i) x = fmaxf(x, z[i]);
      const float lift = x == -__builtin_inff() ? 0.f : -x * kLog2e;   // a lane may have no class
      float y[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 64; ++i) y[i & 1] += __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], kLog2e, lift));
      m[j] = x;
      s[j] = y[0] + y[1];
      const float om = __shfl_xor(m[j], 32), os = __shfl_xor(s[j], 32);
      join(m[j], s[j], om, os);
      if (wave_p() && lane < 32) other[wave_q() + j * 32 + lane] = make_float2(m[j], s[j]);
      __builtin_amdgcn_sched_barrier(0);
    }
    barrier();
    if (!wave_p() && lane < 32) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 o = other[wave_q() + j * 32 + lane];
        join(m[j], s[j], o.x, o.y);
        if (t0 + j * 32 < n) a.part[(int64_t)(tp / kTile) * a.part_ld + t0 + j * 32] = make_float2(m[j], s[j]);
      }
    }
  };
  walk(pt * qt, lds_address(lds), g, begin, take, finish);
}

// Each labelled row's loss and lse from its label's logit and the other classes'
// parts, one workgroup 16 rows: 64 threads a row, which are consecutive rows'
// while the parts are read (594 tiles' parts of 55 rows: 24 us with 16 threads a
// row).
__global__ __launch_bounds__(1024) void k_lse(const float2* part, int32_t part_ld, int32_t tiles, const int32_t* count,
                                              const int32_t* rows, const float* picked, float* lse, float* row_loss) {
  const int32_t n = *count, t0 = blockIdx.x * 16;
  __shared__ float2 lds[64][17];
  if (t0 >= n) return;
  float m = -__builtin_inff(), s = 0.f;
  if (t0 + (int)(threadIdx.x & 15) < n)
    for (int32_t i = threadIdx.x >> 4; i < tiles; i += 64) {
      const float2 o = part[(int64_t)i * part_ld + t0 + (threadIdx.x & 15)];
      join(m, s, o.x, o.y);
    }
  lds[threadIdx.x >> 4][threadIdx.x & 15] = make_float2(m, s);
  __syncthreads();
  const int32_t t = t0 + (threadIdx.x >> 6);
  const float2 mine = lds[threadIdx.x & 63][threadIdx.x >> 6];
  m = mine.x, s = mine.y;
#pragma unroll
  for (int w = 1; w < 64; w *= 2) {
    const float om = __shfl_xor(m, w), os = __shfl_xor(s, w);
    join(m, s, om, os);
  }
  if ((threadIdx.x & 63) == 0 && t < n) {
    const float z = picked[t], d = m - z;
    float loss, l;
    if (d <= 0.f) {
      loss = log1pf(s * expf(d));
      l = z + loss;
    } else {
      const float r = logf(s + expf(-d));
      loss = d + r;
      l = m + r;
    }
    if (!(fabsf(l) <= 3.4028234e38f)) loss = l - z;       // infinities: what the definition gives
    lse[rows[t]] = l;
    row_loss[t] = loss;
  }
}

__global__ __launch_bounds__(1024) void k_loss_sum(const float* row_loss, const int32_t* count, int32_t mean, float* loss) {
  __shared__ float lds[16];
  const int32_t n = *count;
  float s = 0.f;
  for (int32_t i = threadIdx.x; i < n; i += 1024) s += row_loss[i];
  s = reduce64<Add>(s);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.f;
    for (int i = 0; i < 16; ++i) s += lds[i];
    *loss = mean && n ? s / (float)n : s;
  }
}

template <class T, int kJ>
__device__ __forceinline__ void narrow_backward(const LossArgs& a, const Piece& c, int32_t n, char* lds) {
  const Operand16 P{(const T*)a.weight + c.first * a.weight_ld, a.weight_ld, c.classes, a.hidden}, Q{a.xc, a.ld, n, a.hidden};
  Narrow<T, false, kJ> g;
  const int wave = threadIdx.x >> 6;
  const int32_t pt = (c.classes + kTile - 1) / kTile, qt = (n + 32 * kJ - 1) / (32 * kJ);
  int32_t next[kJ], pick[kJ];
  float l[kJ], lift[kJ];
  const auto begin = [&](int32_t id) {
    const int32_t tq = id / pt * (32 * kJ), tp = id % pt;
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      const int32_t t = min(tq + lane_q() + j * 32, n - 1);
      next[j] = a.picks[t];
      l[j] = a.lses[t];
    }
    g.start(P, Q, a.zeros, tp * kTile, tq, tp, lds_address(lds));
  };
  const auto take = [&] {
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      pick[j] = next[j] - c.first;
      lift[j] = (float)kLift<T> - l[j] * kLog2e;
    }
  };
  const auto finish = [&](int32_t id, NarrowAcc<kJ>& acc) {
    const int32_t tq = id / pt * (32 * kJ), tp = id % pt, v0 = tp * kTile + wave * 64 + lane_p();
    T* const to = (T*)a.g + (int64_t)tq * c.ld + tp * kTile + wave * 64;
    // each wave's sums of a row, behind what narrow_rows_out uses
    const auto sums = [&](int w) { return (float*)(lds + kOwnAt + w * kOwnBytes + kOwnBytes / 2); };
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      uint32_t w[2][8];
      float z[32], y[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int32_t v = v0 + i / 4 * 8 + i % 4;
        z[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sum_of(acc, i >> 4, j, i & 15), kLog2e, lift[j]));
        if (tq + lane_q() + j * 32 >= n || v >= c.classes || v == pick[j]) z[i] = 0.f;
        y[i & 1] += z[i];
      }
      const float s = y[0] + y[1], both = s + __shfl_xor(s, 32);
      sums(wave)[j * 32 + lane_q()] = both;      // the same from both lanes
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i >> 3][i & 7] = pack2<T>(z[2 * i], z[2 * i + 1]);
      narrow_rows_out(w, j, lds + kOwnAt + wave * kOwnBytes, [&](int q, int p, u32x4 v) { *(u32x4*)(to + (int64_t)q * c.ld + p) = v; });
    }
    barrier();
    if ((int)threadIdx.x < min(n - tq, 32 * kJ)) {
      float* const others = a.others + (int64_t)(c.first / kTile + tp) * 2 * a.others_ld + tq + threadIdx.x;
      others[0] = sums(0)[threadIdx.x] + sums(1)[threadIdx.x];
      others[a.others_ld] = sums(2)[threadIdx.x] + sums(3)[threadIdx.x];
    }
  };
  walk(pt * qt, lds_address(lds), g, begin, take, finish);
}

// The piece's gradient of the logits (without dloss / n): exp(z - lse); zeros at
// the label, past the labelled rows and past the classes. The gradient at the
// label, exp(z - lse) - 1, is minus the sum of the row's others, whose parts of
// 128 classes are kept in f32: it is complete with the last piece alone, but has
// the relative accuracy of its terms, where the subtraction would leave nothing
// of it for a label that is nearly certain (an error of 1e-6 at logits of 28,
// where the gradient may be 1e-7). Being as large as all others of its row
// together, it takes no part in the 16-bit products: their results get it in f32.
template <class T>
__global__ __launch_bounds__(kGemmThreads, 1) void k_logits_backward(LossArgs a) {
  __shared__ __align__(1024) char lds[kGemmLds];
  const int32_t n = uniform(*a.count);
  const Piece c = piece(a, n);
  if (c.classes <= 0) return;
  const int32_t pt = (c.classes + kTile - 1) / kTile;
  if (n == 0 || if_narrow(rows_of_tile(n, pt), [&](auto j) { narrow_backward<T, decltype(j)::value>(a, c, n, lds); })) return;
  const int32_t qt = (n + kTile - 1) / kTile;
  const Operand16 P{(const T*)a.weight + c.first * a.weight_ld, a.weight_ld, c.classes, a.hidden}, Q{a.xc, a.ld, n, a.hidden};
  Gemm<T, false, false> g;
  int32_t pick[4] = {};
  float l[4] = {};
  int32_t at[4], tp, tq, np, nq;
  float lift[4];
  const auto begin = [&](int32_t id) {
    tile_of(id, pt, qt, &np, &nq);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int32_t t = min(nq + wave_q() + lane_q() + j * 32, n - 1);
      pick[j] = a.picks[t];
      l[j] = a.lses[t];
    }
    g.start(P, Q, a.zeros, np, nq, lds_address(lds));
  };
  const auto take = [&] {
    tp = np, tq = nq;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      at[j] = tq + wave_q() + lane_q() + j * 32 < n ? pick[j] - c.first - (tp + wave_p() + lane_p()) : -1;
      lift[j] = (float)kLift<T> - l[j] * kLog2e;
    }
  };
  const auto finish = [&](int32_t, Acc& acc) {
    const int32_t v0 = tp + wave_p() + lane_p(), t0 = tq + wave_q() + lane_q();
    char* const own = lds + kOwnAt + (threadIdx.x >> 6) * kOwnBytes;
    const int64_t ld = here(c.ld);
    T* const to = (T*)a.g + (int64_t)tq * ld + tp;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float z[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) z[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sum_of(acc, i >> 4, j, i & 15), kLog2e, lift[j]));
      if (at[j] >= 0 && at[j] < 128 && (at[j] & 7) < 4) {
#pragma unroll
        for (int i = 0; i < 64; ++i)
          if (at[j] == i / 4 * 8 + i % 4) z[i] = 0.f;
      }
      if (tp + kTile > c.classes || tq + kTile > n) {
#pragma unroll
        for (int i = 0; i < 64; ++i)
          if (t0 + j * 32 >= n || v0 + i / 4 * 8 + i % 4 >= c.classes) z[i] = 0.f;
      }
      float y[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 64; ++i) y[i & 1] += z[i];
      const float s = y[0] + y[1], both = s + __shfl_xor(s, 32);
      if ((threadIdx.x & 63) < 32 && t0 + j * 32 < n)
        a.others[(int64_t)((c.first + tp + wave_p()) / 128) * a.others_ld + t0 + j * 32] = both;
      Packed x;
#pragma unroll
      for (int i = 0; i < 32; ++i) x.w[i >> 3][i & 7] = pack2<T>(z[2 * i], z[2 * i + 1]);
      __builtin_amdgcn_sched_barrier(0);
      rows_out(x, j, own, [&](int q, int p, u32x4 v) { *(u32x4*)(to + (int64_t)q * ld + p) = v; });
    }
  };
  walk(pt * qt, lds_address(lds), g, begin, take, finish);
}

// Each labelled row's gradient at its label, from the others' sums: 64 threads a
// row, as in k_lse.
__global__ __launch_bounds__(1024) void k_own_gradient(const float* others, int32_t ld, int32_t parts, const int32_t* count, float* own) {
  const int32_t n = *count, t0 = blockIdx.x * 16;
  __shared__ float lds[64][17];
  if (t0 >= n) return;
  float s = 0.f;
  if (t0 + (int)(threadIdx.x & 15) < n)
    for (int32_t i = threadIdx.x >> 4; i < parts; i += 64) s += others[(int64_t)i * ld + t0 + (threadIdx.x & 15)];
  lds[threadIdx.x >> 4][threadIdx.x & 15] = s;
  __syncthreads();
  s = reduce64<Add>(lds[threadIdx.x & 63][threadIdx.x >> 6]);
  const int32_t t = t0 + (threadIdx.x >> 6);
  if ((threadIdx.x & 63) == 0 && t < n) own[t] = -s;
}

// How many workgroups share a tile of dx, each with a part of the piece's
// classes and sums of its own: the number whose rounds of 256 workgroups take
// the least time, a tile's results counted as 12 pairs of stages; the same for
// all pieces. 16 by 14 tiles leave 32 of 256 compute units idle, in 8 parts
// none.
__device__ __forceinline__ int32_t splits_of(int32_t pt, int32_t qt, int32_t rows_of_tile, int32_t piece, int64_t sum_rows) {
  const int32_t pairs = (piece + kPairK - 1) / kPairK, most = min(kMaxSplits * (kTile / rows_of_tile), pairs);
  const int32_t s = (threadIdx.x & 63) + 1;     // a lane each: there are at most 64
  int64_t time = (int64_t)((pt * qt * s + kCUs - 1) / kCUs) * ((pairs + s - 1) / s + 12);
  if (s > 1 && (s > most || (int64_t)s * qt * rows_of_tile > sum_rows)) time = 1ll << 48;
  int64_t best = time * 64 + (s - 1);
#pragma unroll
  for (int w = 1; w < 64; w *= 2) best = std::min<int64_t>(best, __shfl_xor(best, w));
  return uniform((int32_t)(best & 63) + 1);
}

// Rows of a tile of dx's sums; the classes are split until the tiles fill the
// chip, so narrow tiles are for few rows alone.
__device__ __forceinline__ int32_t rows_of_sum(int32_t n) { return n > 128 ? kTile : n > 64 ? 128 : 64; }

// A split's part of the classes.
__device__ __forceinline__ int32_t part_from(int32_t split, int32_t splits, const Piece& c) {
  const int32_t pairs = (c.classes + kPairK - 1) / kPairK;
  return min((int32_t)((int64_t)pairs * split / splits) * kPairK, c.classes);
}

template <class T, int kJ>
__device__ __forceinline__ void narrow_gradient(const LossArgs& a, const Piece& c, int32_t n, char* lds) {
  const int32_t pt = (a.hidden + kTile - 1) / kTile, splits = splits_of(pt, 1, 32 * kJ, c.ld, a.sum_rows);
  const T* const weight = (const T*)a.weight + c.first * a.weight_ld;
  Narrow<T, true, kJ> gemm;
  const int wave = threadIdx.x >> 6;
  const auto begin = [&](int32_t id) {
    const int32_t split = id / pt, k0 = part_from(split, splits, c), k1 = part_from(split + 1, splits, c);
    gemm.start(Operand16{weight + k0 * a.weight_ld, a.weight_ld, a.hidden, k1 - k0},
               Operand16{(const T*)a.g + k0, c.ld, n, (int32_t)up(k1 - k0, 8)}, a.zeros, (id - split * pt) * kTile, 0, 0, lds_address(lds));
  };
  const auto finish = [&](int32_t id, NarrowAcc<kJ>& acc) {
    const int32_t split = id / pt, tp = (id - split * pt) * kTile + wave * 64;
    float* const to = a.sum + (int64_t)split * (32 * kJ) * a.ld + tp;
    narrow_rows_out(acc, lds + kOwnAt + wave * kOwnBytes, [&](int q, int p, f32x4 v) {
      if (q >= n || tp + p >= a.hidden) return;
      f32x4* const at = (f32x4*)(to + (int64_t)q * a.ld + p);
      *at = a.u ? *at + v : v;
    });
  };
  walk(c.classes > 0 ? pt * splits : 0, lds_address(lds), gemm, begin, [] {}, finish);
}

// dx's sums of a piece: sum[split][row][h] (+)= g weight.
template <class T>
__global__ __launch_bounds__(kGemmThreads, 1) void k_rows_gradient(LossArgs a) {
  __shared__ __align__(1024) char lds[kGemmLds];
  const int32_t n = uniform(*a.count);
  const Piece c = piece(a, n);
  if (n == 0 || if_narrow(rows_of_sum(n), [&](auto j) { narrow_gradient<T, decltype(j)::value>(a, c, n, lds); })) return;
  const int32_t pt = (a.hidden + kTile - 1) / kTile, qt = (n + kTile - 1) / kTile, splits = splits_of(pt, qt, kTile, c.ld, a.sum_rows);
  const T* const weight = (const T*)a.weight + c.first * a.weight_ld;
  Gemm<T, true, false> gemm;
  const auto begin = [&](int32_t id) {
    const int32_t split = id / (pt * qt);
    int32_t p, q;
    tile_of(id - split * pt * qt, pt, qt, &p, &q);
    const int32_t k0 = part_from(split, splits, c), k1 = part_from(split + 1, splits, c);
    gemm.start(Operand16{weight + k0 * a.weight_ld, a.weight_ld, a.hidden, k1 - k0},
               Operand16{(const T*)a.g + k0, c.ld, n, (int32_t)up(k1 - k0, 8)}, a.zeros, p, q, lds_address(lds));
  };
  const auto finish = [&](int32_t id, Acc& acc) {
    const int32_t split = id / (pt * qt);
    int32_t tp, tq;
    tile_of(id - split * pt * qt, pt, qt, &tp, &tq);
    char* const own = lds + kOwnAt + (threadIdx.x >> 6) * kOwnBytes;
    const int64_t ld = here(a.ld);
    float* const to = a.sum + ((int64_t)split * qt * kTile + tq) * ld + tp;
    rows_out(acc, 1.f, own, [&](int, int q, int p, f32x4 v) {
      if (tq + q >= n || tp + p >= a.hidden) return;
      f32x4* const at = (f32x4*)(to + (int64_t)q * ld + p);
      *at = a.u ? *at + v : v;
    });
  };
  walk(c.classes > 0 ? pt * qt * splits : 0, lds_address(lds), gemm, begin, [] {}, finish);
}

// What the sums over a gradient of the logits are multiplied with. Without
// labelled rows they are empty, whatever dloss is.
template <class T>
__device__ __forceinline__ float factor(const float* dloss, const int32_t* count, int32_t mean) {
  if (*count == 0) return 0.f;
  const float d = (dloss ? *dloss : 1.f) * (1.f / (float)(1 << kLift<T>));
  return mean ? d / (float)*count : d;
}

// The piece's rows of dweight: (+)= factor * transposed g x. Classes that are some
// row's label leave their sums in f32 for k_finish.
template <class T, class O>
__global__ __launch_bounds__(kGemmThreads, 1) void k_weight_gradient(LossArgs a, const float* dloss, int32_t mean, O* dweight,
                                                                     int64_t dw_ld, int32_t add) {
  __shared__ __align__(1024) char lds[kGemmLds];
  const int32_t n = uniform(*a.count);
  const Piece c = piece(a, n);
  const int32_t pt = (a.hidden + kTile - 1) / kTile, qt = (c.classes + kTile - 1) / kTile;
  const float f = factor<T>(dloss, a.count, mean);
  const Operand16 P{a.xc, a.ld, a.hidden, n}, Q{a.g, c.ld, qt * kTile, n};
  Gemm<T, true, true> g;
  int32_t next[4] = {}, side[4];   // where the lane's classes leave their sums: of the tile whose loads are under way, of the one that is ready
  const auto begin = [&](int32_t id) {
    int32_t p, q;
    tile_of(id, pt, qt, &p, &q);
#pragma unroll
    for (int j = 0; j < 4; ++j) next[j] = a.begin[c.first + min(q + wave_q() + lane_q() + j * 32, c.classes - 1)];
    g.start(P, Q, a.zeros, p, q, lds_address(lds));
  };
  const auto take = [&] {
#pragma unroll
    for (int j = 0; j < 4; ++j) side[j] = next[j];
  };
  const auto finish = [&](int32_t id, Acc& acc) {
    int32_t tp, tq;
    tile_of(id, pt, qt, &tp, &tq);
    char* const own = lds + kOwnAt + (threadIdx.x >> 6) * kOwnBytes;
    const int64_t ld = here(dw_ld);
    O* const to = dweight + (c.first + (int64_t)tq) * ld + tp;
    uint32_t labels[4];            // which of the wave's 32 classes are
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (tq + wave_q() + lane_q() + j * 32 >= c.classes) side[j] = -1;
      labels[j] = (uint32_t)__ballot(side[j] >= 0);
      if (!labels[j]) continue;
      float* const row = a.side + (int64_t)side[j] * a.ld + tp + wave_p() + lane_p();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = sum_of(acc, i >> 2, j, 4 * (i & 3) + e);
        if (side[j] >= 0 && tp + wave_p() + lane_p() + i * 8 < a.hidden) *(f32x4*)(row + i * 8) = v;
      }
    }
    if constexpr (__is_same(O, float)) {
      rows_out(acc, f, own, [&](int j, int q, int p, f32x4 v) {
        if (tq + q >= c.classes || tp + p >= a.hidden || (labels[j] >> (q & 31) & 1)) return;
        f32x4* const at = (f32x4*)(to + (int64_t)q * ld + p);
        *at = add ? *at + v : v;
      });
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        Packed x;
#pragma unroll
        for (int i = 0; i < 32; ++i)
          x.w[i >> 3][i & 7] = pack2<O>(sum_of(acc, i >> 3, j, 2 * (i & 7)) * f, sum_of(acc, i >> 3, j, 2 * (i & 7) + 1) * f);
        rows_out(x, j, own, [&](int q, int p, u32x4 v) {
          if (tq + q < c.classes && tp + p < a.hidden) *(u32x4*)(to + (int64_t)q * ld + p) = v;
        });
      }
    }
  };
  walk(pt * qt, lds_address(lds), g, begin, take, finish);
}

// A row of dx: the label's gradient times its weight and the splits' sums, times
// the factor; zeros for rows without a label. 2048 columns a workgroup.
template <class T>
__device__ __forceinline__ void finish_row(const LossArgs& a, int32_t t, int32_t i, float f, T* dx, int64_t dx_stride) {
  T* out = dx + (int64_t)t * dx_stride;
  const int32_t n = *a.count, tile = rows_of_sum(n), rows = (n + tile - 1) / tile * tile;
  const int32_t splits = i < 0 ? 0 : splits_of((a.hidden + kTile - 1) / kTile, rows / tile, tile, piece_of(n, a.vocab, a.room), a.sum_rows);
  const int32_t c = (blockIdx.y * 256 + threadIdx.x) * 8;
  if (c < a.hidden) {
    Pack<T, 8> o;
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (i >= 0) {
      const Pack<T, 8> w = load<T, 8>((const T*)a.weight + a.picks[i] * a.weight_ld + c);
      const float own = a.own[i];
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = own * w.get(e);
    }
#pragma unroll 8
    for (int32_t k = 0; k < splits; ++k) {
      const Pack<float, 8> p = load<float, 8>(a.sum + ((int64_t)k * rows + i) * a.ld + c);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += p.get(e);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) o.set(e, i >= 0 ? s[e] * f : 0.f);      // f may be no number
    store<T, 8>(out + c, o);
  }
}

// Adds up the rows at places `from` to `to` of the order, each times its gradient
// at the label, 8 columns a lane from c on: every kWaves-th row from the wave's
// on, 8 under way.
template <class T, int kWaves>
__device__ __forceinline__ void add_rows(const LossArgs& a, const Classes& o, int32_t from, int32_t to, int32_t c, float (&s)[8]) {
  for (int32_t k = from + uniform(threadIdx.x >> 6) % kWaves; k < to; k += 8 * kWaves) {
    int32_t row[8];
    float own[8];
    Pack<T, 8> x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) row[e] = o.order[min(k + kWaves * e, to - 1)];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      own[e] = a.own[row[e]];
      x[e] = load<T, 8>((const T*)a.xc + (int64_t)row[e] * a.ld + c);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + kWaves * e < to)
#pragma unroll
        for (int d = 0; d < 8; ++d) s[d] += own[e] * x[e].get(d);
  }
}
// Adds the 4 waves' sums to the first one's, in order. All of the workgroup.
__device__ __forceinline__ void join_waves(float (&s)[8], float (*parts)[8][64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (wave)
#pragma unroll
    for (int d = 0; d < 8; ++d) parts[wave - 1][d][lane] = s[d];
  __syncthreads();
  if (!wave)
#pragma unroll
    for (int d = 0; d < 8; ++d) s[d] = ((s[d] + parts[0][d][lane]) + parts[1][d][lane]) + parts[2][d][lane];
  __syncthreads();
}

// A class that many rows share is added up by more than one workgroup: the sums
// of each kPart places that are all its own (the order is by class, so the first
// and the last tell) wait in the side row of the second place, which no class
// begins at. Without this 32768 rows of one class take 3.4 ms over 1000 x 1024,
// with it 0.95, as rows of different classes do.
constexpr int32_t kPart = 256;
template <class T>
__global__ __launch_bounds__(256) void k_class_parts(LossArgs a, Classes o) {
  __shared__ float parts[3][8][64];
  const int32_t i = blockIdx.x * kPart;
  if (i + kPart > *a.count || a.picks[o.order[i]] != a.picks[o.order[i + kPart - 1]]) return;
  const int32_t c = blockIdx.y * 512 + (threadIdx.x & 63) * 8;
  float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  add_rows<T, 4>(a, o, i, i + kPart, min(c, a.hidden - 8), s);
  join_waves(s, parts);
  if (threadIdx.x < 64 && c < a.hidden) {
    Pack<float, 8> p;
#pragma unroll
    for (int d = 0; d < 8; ++d) p.set(d, s[d]);
    store<float, 8>(a.side + (int64_t)(i + 1) * a.ld + c, p);
  }
}

// 8 elements of a class's row of dweight: the pieces' sums p and its own rows' s.
template <class O>
__device__ __forceinline__ void finish_vector(O* to, const Pack<float, 8>& p, const float (&s)[8], float f, int32_t add) {
  Pack<O, 8> out;
  Pack<float, 8> old{};
  if constexpr (__is_same(O, float))
    if (add) old = load<float, 8>(to);
#pragma unroll
  for (int d = 0; d < 8; ++d) out.set(d, old.get(d) + f * (p.get(d) + s[d]));
  store<O, 8>(to, out);
}

// The row of dweight of the class whose rows begin at place i: its sums over the
// piece's product, and each of its own rows times that row's gradient at the
// label, 512 columns at a time. The rows of a class that has few are added up by
// each of the 4 waves for its own columns, those of others by all 4 waves for the
// same columns (16384 rows over 8192 x 2048, two a class: 168 us if all were).
constexpr int32_t kFewRows = 16;
template <class T, class O>
__device__ __forceinline__ void finish_class(const LossArgs& a, const Classes& o, int32_t i, float f, O* dweight, int64_t dw_ld,
                                             int32_t add, bool in_parts) {
  __shared__ float parts[3][8][64];
  const int32_t many = uniform(o.many[i]);
  if (!many) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  O* const row = dweight + (int64_t)a.picks[o.order[i]] * dw_ld;
  const float* const side = a.side + (int64_t)i * a.ld;
  const int32_t from = blockIdx.y * 2048, to = min(a.hidden, from + 2048);
  if (many <= kFewRows) {
    const int32_t c = from + wave * 512 + lane * 8;
    if (c >= to) return;
    const Pack<float, 8> p = load<float, 8>(side + c);
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    add_rows<T, 1>(a, o, i, i + many, c, s);
    return finish_vector(row + c, p, s, f, add);
  }
  // places up to the first whole part, whole parts, and places behind the last; without whole parts all are the first
  int32_t whole = (i + kPart - 1) / kPart, end = (i + many) / kPart;
  if (!in_parts || whole >= end) whole = end = (i + many + kPart - 1) / kPart;
  for (int32_t c0 = from; c0 < to; c0 += 512) {
    const int32_t c = c0 + lane * 8, at = min(c, a.hidden - 8);
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    add_rows<T, 4>(a, o, i, min(whole * kPart, i + many), at, s);
#pragma unroll 8
    for (int32_t k = whole + wave; k < end; k += 4) {
      const Pack<float, 8> p = load<float, 8>(a.side + (int64_t)(k * kPart + 1) * a.ld + at);
#pragma unroll
      for (int d = 0; d < 8; ++d) s[d] += p.get(d);
    }
    add_rows<T, 4>(a, o, min(end * kPart, i + many), i + many, at, s);
    join_waves(s, parts);
    if (!wave && c < to) finish_vector(row + c, load<float, 8>(side + c), s, f, add);
  }
}

// What the pieces left: workgroups up to dx_rows have a row of dx each, those
// behind a place in the order of the labelled rows.
template <class T, class O>
__global__ __launch_bounds__(256) void k_finish(LossArgs a, Classes o, const int32_t* slot, const float* dloss, int32_t mean, int32_t dx_rows,
                                                T* dx, int64_t dx_stride, O* dweight, int64_t dw_ld, int32_t add, int32_t in_parts) {
  const float f = factor<T>(dloss, a.count, mean);
  if ((int32_t)blockIdx.x < dx_rows)
    finish_row(a, blockIdx.x, slot[blockIdx.x], f, dx, dx_stride);
  else if ((int32_t)blockIdx.x - dx_rows < *a.count)
    finish_class<T>(a, o, blockIdx.x - dx_rows, f, dweight, dw_ld, add, in_parts);
}

// ------------------------------------------------------------------ host

// Where the parts of the workspace lie (byte offsets).
struct Plan {
  int64_t rows_p;               // rows up to whole tiles
  int32_t ld;                   // hidden up to whole pairs of stages
  int64_t room, sum_rows;       // as in LossArgs
  int64_t zeros, count, rows, picks, slot, lses, picked, row_loss, part, xc, g, sum, own, others, side, order, many, begin;
  int64_t bytes;
};

Plan plan_of(int64_t rows, int32_t hidden, int32_t vocab, bool backward) {
  Plan p{};
  p.rows_p = up(std::max<int64_t>(rows, 1), kTile);
  p.ld = (int32_t)up(hidden, kPairK);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += up(bytes, 256);
    return here;
  };
  p.zeros = take(256);
  p.count = take(4);
  p.rows = take(4 * p.rows_p);
  p.picks = take(4 * p.rows_p);
  p.slot = take(4 * p.rows_p);
  p.lses = take(4 * p.rows_p);
  p.xc = take(p.rows_p * p.ld * 2);
  const int64_t tiles = (vocab + kTile - 1) / kTile;
  const int64_t shared = at;
  p.picked = take(4 * p.rows_p);
  p.row_loss = take(4 * p.rows_p);
  p.part = take(tiles * p.rows_p * 8);
  p.bytes = at;
  if (backward) {
    at = shared;                 // nothing of the forward pass is needed any more
    // room for a tile of classes of all rows, and for all classes at most
    p.room = std::max(p.rows_p * kTile, std::min(kPieceElements, p.rows_p * tiles * kTile));
    p.g = take(p.room * 2);
    p.sum_rows = std::max<int64_t>(2 * p.rows_p, kMaxSplits * kTile);
    p.sum = take(p.sum_rows * p.ld * 4);
    p.own = take(4 * p.rows_p);
    p.others = take(2 * tiles * p.rows_p * 4);
    p.side = take(p.rows_p * p.ld * 4);
    p.order = take(4 * p.rows_p);
    p.many = take(4 * p.rows_p);
    p.begin = take(4 * (int64_t)vocab);
    p.bytes = std::max(p.bytes, at);
  }
  return p;
}

fp_status check(const char* what, int64_t rows, int32_t hidden, int32_t vocab) {
  if (rows < 0 || rows > kMaxRows) return report(FP_EINVAL, "%s: %lld rows", what, (long long)rows);
  if (hidden < 8 || hidden > kMaxHidden || hidden % 8)
    return report(FP_EINVAL, "%s: hidden %d is not a multiple of 8 in [8, %d]", what, hidden, kMaxHidden);
  if (vocab < 1 || vocab > kMaxVocab) return report(FP_EINVAL, "%s: vocab %d outside [1, %d]", what, vocab, kMaxVocab);
  return FP_OK;
}

fp_status check(const char* what, const void* x, int64_t x_stride, const void* weight, int64_t weight_stride, const int32_t* labels,
                int64_t rows, int32_t hidden, int32_t vocab, int32_t type, int32_t reduction, const float* lse, const void* workspace,
                int64_t workspace_bytes, bool backward) {
  const fp_status st = check(what, rows, hidden, vocab);
  if (st != FP_OK) return st;
  if (type != FP_BF16 && type != FP_F16) return report(FP_EINVAL, "%s: type %d", what, type);
  if (reduction != FP_LOSS_MEAN && reduction != FP_LOSS_SUM) return report(FP_EINVAL, "%s: reduction %d", what, reduction);
  if (!weight || !workspace || (rows && (!x || !labels || !lse))) return report(FP_EINVAL, "%s: null x, weight, labels, lse or workspace", what);
  if (x_stride < hidden || weight_stride < hidden || x_stride > (1ll << 40) || weight_stride > kMaxStride)
    return report(FP_EINVAL, "%s: row strides %lld and %lld, hidden is %d", what, (long long)x_stride, (long long)weight_stride, hidden);
  if (!aligned(x, 16) || !aligned(weight, 16) || x_stride % 8 || weight_stride % 8)
    return report(FP_EALIGN, "%s: x, weight or a row stride is not a multiple of 16 bytes", what);
  if (!aligned(labels, 4) || !aligned(lse, 4)) return report(FP_EALIGN, "%s: labels or lse is not aligned", what);
  if (!aligned(workspace, 256)) return report(FP_EALIGN, "%s: workspace is not 256-byte aligned", what);
  const int64_t need = plan_of(rows, hidden, vocab, backward).bytes;
  if (workspace_bytes < need)
    return report(FP_ECAPACITY, "%s: workspace of %lld bytes, %lld needed", what, (long long)workspace_bytes, (long long)need);
  return FP_OK;
}

// What both passes begin with: zeros, the list of labelled rows, their gather, and (with `classes`) their order.
template <class T>
hipError_t begin(const Plan& p, char* ws, const void* x, int64_t x_stride, const int32_t* labels, int64_t rows, int32_t hidden,
                 int32_t vocab, int32_t* slot, int32_t* count_out, float* zero_lse, const float* lse, const Classes& classes, hipStream_t s) {
  int32_t* const count = (int32_t*)(ws + p.count);
  int32_t* const list = (int32_t*)(ws + p.rows);
  hipError_t e = launch(k_label_rows, dim3(1), dim3(1024), 0, s, labels, (int32_t)rows, vocab, list, (int32_t*)(ws + p.picks), slot,
                        count, count_out, zero_lse, (u32x4*)(ws + p.zeros));
  const int32_t tiles = classes.order ? (vocab + 255) / 256 : 0;
  const int64_t groups = tiles + (rows + 3) / 4;
  if (e == hipSuccess && groups)
    e = launch(k_gather_rows<T>, dim3((unsigned)groups), dim3(64 * kOrderWaves), 0, s, (const T*)x, x_stride, (const int32_t*)list,
               (const int32_t*)count, hidden, p.ld, (T*)(ws + p.xc), lse, (float*)(ws + p.lses), tiles,
               (const int32_t*)(ws + p.picks), vocab, classes);
  return e;
}

LossArgs loss_args(const Plan& p, char* ws, const void* weight, int64_t weight_stride, int32_t hidden, int32_t vocab) {
  LossArgs a{};
  a.count = (int32_t*)(ws + p.count), a.picks = (int32_t*)(ws + p.picks), a.zeros = ws + p.zeros;
  a.xc = ws + p.xc, a.ld = p.ld, a.hidden = hidden, a.vocab = vocab;
  a.weight = weight, a.weight_ld = weight_stride;
  return a;
}

int64_t tiles(int64_t n) { return (n + kTile - 1) / kTile; }

// One workgroup a compute unit, which walks over the tiles, or fewer if there
// cannot be as many tiles.
dim3 resident(int64_t tiles) { return dim3((unsigned)std::min<int64_t>(tiles, kCUs)); }

template <class T>
hipError_t forward(const Plan& p, char* ws, const void* x, int64_t x_stride, const void* weight, int64_t weight_stride,
                   const int32_t* labels, int64_t rows, int32_t hidden, int32_t vocab, int32_t reduction, float* loss, float* lse,
                   int32_t* n_labelled, hipStream_t s) {
  hipError_t e = begin<T>(p, ws, x, x_stride, labels, rows, hidden, vocab, nullptr, n_labelled, lse, nullptr, Classes{}, s);
  LossArgs a = loss_args(p, ws, weight, weight_stride, hidden, vocab);
  a.part = (float2*)(ws + p.part), a.part_ld = (int32_t)p.rows_p, a.picked = (float*)(ws + p.picked);
  float* const row_loss = (float*)(ws + p.row_loss);
  if (rows) {
    if (e == hipSuccess)
      e = launch(k_logits_forward<T>, resident(tiles(vocab) * ((rows + 63) / 64)), dim3(kGemmThreads), 0, s, a);
    if (e == hipSuccess)
      e = launch(k_lse, dim3((unsigned)((rows + 15) / 16)), dim3(1024), 0, s, (const float2*)a.part, a.part_ld, (int32_t)tiles(vocab),
                 a.count, (const int32_t*)(ws + p.rows), (const float*)a.picked, lse, row_loss);
  }
  if (e == hipSuccess)
    e = launch(k_loss_sum, dim3(1), dim3(1024), 0, s, (const float*)row_loss, a.count, (int32_t)(reduction == FP_LOSS_MEAN), loss);
  return e;
}

template <class T>
hipError_t backward(const Plan& p, char* ws, const void* x, int64_t x_stride, const void* weight, int64_t weight_stride,
                    const int32_t* labels, const float* lse, const float* dloss, int64_t rows, int32_t hidden, int32_t vocab,
                    int32_t reduction, void* dx, int64_t dx_stride, void* dweight, int64_t dw_stride, bool dw_f32, bool add,
                    hipStream_t s) {
  int32_t* const slot = (int32_t*)(ws + p.slot);
  Classes classes{};
  if (dweight) classes = {(int32_t*)(ws + p.order), (int32_t*)(ws + p.many), (int32_t*)(ws + p.begin)};
  hipError_t e = begin<T>(p, ws, x, x_stride, labels, rows, hidden, vocab, slot, nullptr, nullptr, lse, classes, s);
  LossArgs a = loss_args(p, ws, weight, weight_stride, hidden, vocab);
  const int32_t mean = reduction == FP_LOSS_MEAN;
  a.lses = (float*)(ws + p.lses), a.g = ws + p.g, a.room = p.room, a.sum = (float*)(ws + p.sum), a.sum_rows = p.sum_rows;
  a.others = (float*)(ws + p.others), a.others_ld = (int32_t)p.rows_p, a.own = (float*)(ws + p.own);
  a.begin = classes.begin, a.side = (float*)(ws + p.side);
  // with all rows labelled there are the most pieces
  const int32_t most = piece_of(rows, vocab, p.room);
  const int64_t pieces = ((int64_t)vocab + most - 1) / most;
  for (a.u = 0; a.u < pieces; ++a.u) {
    // piece 0 may be the whole vocabulary: as many workgroups as any piece has use for
    if (rows && e == hipSuccess) e = launch(k_logits_backward<T>, resident(tiles(vocab) * ((rows + 63) / 64)), dim3(kGemmThreads), 0, s, a);
    if (rows && dx && e == hipSuccess) e = launch(k_rows_gradient<T>, dim3(kCUs), dim3(kGemmThreads), 0, s, a);
    if (dweight && e == hipSuccess) {
      const dim3 grid = resident(tiles(hidden) * tiles(vocab));
      if (dw_f32)
        e = launch(k_weight_gradient<T, float>, grid, dim3(kGemmThreads), 0, s, a, dloss, mean, (float*)dweight, dw_stride, (int32_t)add);
      else
        e = launch(k_weight_gradient<T, T>, grid, dim3(kGemmThreads), 0, s, a, dloss, mean, (T*)dweight, dw_stride, 0);
    }
  }
  if (!rows) return e;
  if (e == hipSuccess)
    e = launch(k_own_gradient, dim3((unsigned)((rows + 15) / 16)), dim3(1024), 0, s, (const float*)a.others, a.others_ld,
               (int32_t)(2 * tiles(vocab)), a.count, (float*)(ws + p.own));
  // up to two parts of rows are soon added up by the workgroup that finishes the class
  const bool in_parts = dweight && rows > 2 * kPart;
  if (in_parts && e == hipSuccess)
    e = launch(k_class_parts<T>, dim3((unsigned)(rows / kPart), (unsigned)((hidden + 511) / 512)), dim3(256), 0, s, a, classes);
  const auto finish = [&](auto* dw) {
    using O = std::remove_pointer_t<decltype(dw)>;
    const dim3 grid((unsigned)((dx ? rows : 0) + (dweight ? rows : 0)), (unsigned)((hidden + 2047) / 2048));
    return launch(k_finish<T, O>, grid, dim3(256), 0, s, a, classes, (const int32_t*)slot, dloss, mean, (int32_t)(dx ? rows : 0), (T*)dx,
                  dx_stride, dw, dw_stride, (int32_t)add, (int32_t)in_parts);
  };
  if (e == hipSuccess) e = dw_f32 ? finish((float*)dweight) : finish((T*)dweight);
  return e;
}

}  // namespace
}  // namespace fp

using namespace fp;

extern "C" {

int64_t vocab_loss_workspace(int64_t rows, int32_t hidden, int32_t vocab, int32_t backward) {
  const fp_status st = check("vocab_loss_workspace", rows, hidden, vocab);
  return st == FP_OK ? plan_of(rows, hidden, vocab, backward != 0).bytes : st;
}

fp_status vocab_loss_forward(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride, const int32_t* labels,
                             int64_t rows, int32_t hidden, int32_t vocab, int32_t type, int32_t reduction, float* loss, float* lse,
                             int32_t* n_labelled, void* workspace, int64_t workspace_bytes, void* stream) {
  const char* const what = "vocab_loss_forward";
  const fp_status st = check(what, x, x_stride, weight, weight_stride, labels, rows, hidden, vocab, type, reduction, lse, workspace,
                             workspace_bytes, false);
  if (st != FP_OK) return st;
  if (!loss) return report(FP_EINVAL, "%s: null loss", what);
  if (!aligned(loss, 4) || !aligned(n_labelled, 4)) return report(FP_EALIGN, "%s: loss or n_labelled is not aligned", what);
  const Plan p = plan_of(rows, hidden, vocab, false);
  auto* const go = type == FP_BF16 ? forward<bf16> : forward<f16>;
  return launched(go(p, (char*)workspace, x, x_stride, weight, weight_stride, labels, rows, hidden, vocab, reduction, loss, lse,
                     n_labelled, (hipStream_t)stream),
                  what);
}

fp_status vocab_loss_backward(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride, const int32_t* labels,
                              const float* lse, const float* dloss, int64_t rows, int32_t hidden, int32_t vocab, int32_t type,
                              int32_t reduction, void* dx, int64_t dx_stride, void* dweight, int64_t dweight_stride,
                              int32_t dweight_type, int32_t accumulate, void* workspace, int64_t workspace_bytes, void* stream) {
  const char* const what = "vocab_loss_backward";
  const fp_status st = check(what, x, x_stride, weight, weight_stride, labels, rows, hidden, vocab, type, reduction, lse, workspace,
                             workspace_bytes, true);
  if (st != FP_OK) return st;
  if (!aligned(dloss, 4)) return report(FP_EALIGN, "%s: dloss is not aligned", what);
  if (dx && (dx_stride < hidden || dx_stride > (1ll << 40)))
    return report(FP_EINVAL, "%s: dx has row stride %lld, hidden is %d", what, (long long)dx_stride, hidden);
  if (dx && (!aligned(dx, 16) || dx_stride % 8)) return report(FP_EALIGN, "%s: dx or its row stride is not a multiple of 16 bytes", what);
  if (dweight) {
    if (dweight_type != FP_F32 && dweight_type != type) return report(FP_EINVAL, "%s: dweight type %d with type %d", what, dweight_type, type);
    if (accumulate && dweight_type != FP_F32) return report(FP_EINVAL, "%s: accumulation in 16 bits", what);
    if (dweight_stride < hidden || dweight_stride > (1ll << 40))
      return report(FP_EINVAL, "%s: dweight has row stride %lld, hidden is %d", what, (long long)dweight_stride, hidden);
    if (!aligned(dweight, 16) || dweight_stride % (16 / type_size(dweight_type)))
      return report(FP_EALIGN, "%s: dweight or its row stride is not a multiple of 16 bytes", what);
  }
  if (!dx && !dweight) return FP_OK;
  const Plan p = plan_of(rows, hidden, vocab, true);
  auto* const go = type == FP_BF16 ? backward<bf16> : backward<f16>;
  return launched(go(p, (char*)workspace, x, x_stride, weight, weight_stride, labels, lse, dloss, rows, hidden, vocab, reduction, dx,
                     dx_stride, dweight, dweight_stride, dweight && dweight_type == FP_F32, accumulate != 0, (hipStream_t)stream),
                  what);
}

}  // extern "C"
