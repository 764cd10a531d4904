// Layer norm of a microbatch's rows, forward and backward (norm_forward,
// norm_backward of include/flowpool_train.h).
//
// Both passes move each row once: a row stays in the registers of the threads
// that loaded it between its statistics and its result, so the bound is HBM
// bytes, 2 (forward) or 3 (backward) times the row. The statistics are taken
// in two passes over the registers (the mean first, then the centred squares),
// which loses nothing to cancellation and costs no memory traffic.
//
// A row is spread over WPR waves of one workgroup, VPT accesses of VE elements
// a thread: 32 elements a thread at most going forward, 24 going backward,
// where each also has two sums. One wave a row needs no barrier. Workgroups are
// resident ones that step through the rows, with the next row's loads issued
// before the present one is used, and the weight and bias in registers as f32.
// Rows pass the caches by: they are used once.
//
// Measured: forward 65536 x 5120 in bf16 238 us, 5.6 TB/s (a large copy reaches
// 6.2), in f32 499 us, 5.4 TB/s; backward 16384 x 3584 in bf16 76 us, 4.7 TB/s, of it
// 4 to 5 for the columns' sums; 4099 rows of 1155 f32 in rows of 1160 9.4 us forward
// and 21.6 backward, a wave's rows one after the other; the smallest forward call
// 9.4 us, of it 3.7 in the kernel.

#include "train_internal.h"

#include <algorithm>

namespace fp {
namespace {

constexpr int kMaxHidden = 12288;
constexpr int64_t kMaxRows = (1ll << 31) - 1;
constexpr int kCUs = 256;              // compute units of an MI355X

// Sum over the WPR waves of a row; every thread gets it. `slot` alternates
// between calls, so that one barrier a call is enough: a wave can only be one
// call ahead of another, and writes the other slot then.
template <int WPR>
__device__ __forceinline__ float row_sum(float x, float (*lds)[WPR], int slot) {
  x = reduce64<Add>(x);
  if constexpr (WPR == 1) {
    return x;
  } else {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[slot][wave] = x;
    __syncthreads();
    float s = 0;
#pragma unroll
    for (int w = 0; w < WPR; ++w) s += lds[slot][w];
    return s;
  }
}

struct NormArgs {
  const void* x;
  const void* dy;
  const void* weight;
  const void* bias;
  void* y;             // forward: y; backward: dx
  float* mean;
  float* rstd;
  float* partial;      // backward: [groups][2][hidden]
  int64_t x_stride, y_stride, dy_stride;
  int32_t rows, hidden;
  float eps, elements; // elements = hidden: divided by, not multiplied with its reciprocal,
                       // so that the mean of equal values is that value
  int32_t wide_weight; // weight and bias are f32
};

template <class T, int VE, int VPT, int WPR>
struct Row {
  Pack<T, VE> a[VPT];
  // Loads the thread's part; elements past the row are zeros.
  __device__ __forceinline__ void load(const T* row, int hidden, int t) {
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int at = (k * 64 * WPR + t) * VE;
      if (at < hidden) {
        a[k] = fp::load_once<T, VE>(row + at);
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) a[k].set(e, 0.f);
      }
    }
  }
};

// The thread's part of weight or bias, as f32 (`missing` where there is none).
template <class T, int VE, int VPT, int WPR>
struct Vector {
  float a[VPT][VE];
  __device__ __forceinline__ void load(const void* p, bool f32, float missing, int hidden, int t) {
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int at = (k * 64 * WPR + t) * VE;
#pragma unroll
      for (int e = 0; e < VE; ++e) a[k][e] = missing;
      if (p && at < hidden) {
        if (f32) {
          const Pack<float, VE> v = fp::load<float, VE>((const float*)p + at);
#pragma unroll
          for (int e = 0; e < VE; ++e) a[k][e] = v.get(e);
        } else {
          const Pack<T, VE> v = fp::load<T, VE>((const T*)p + at);
#pragma unroll
          for (int e = 0; e < VE; ++e) a[k][e] = v.get(e);
        }
      }
    }
  }
};

template <class T, int VE, int VPT, int WPR>
__global__ __launch_bounds__(WPR == 1 ? 256 : 64 * WPR) void k_norm_forward(NormArgs a) {
  constexpr int kThreads = 64 * WPR;               // of a row
  constexpr int kRows = WPR == 1 ? 4 : 1;          // rows a workgroup has at once
  __shared__ float lds[2][WPR];
  const int t = threadIdx.x % kThreads;
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t r = (int64_t)blockIdx.x * kRows + (WPR == 1 ? threadIdx.x >> 6 : 0);
  if (r >= a.rows) return;                         // whole rows' waves, so barriers stay whole

  Vector<T, VE, VPT, WPR> w, b;
  w.load(a.weight, a.wide_weight, 1.f, a.hidden, t);
  b.load(a.bias, a.wide_weight, 0.f, a.hidden, t);
  Row<T, VE, VPT, WPR> x;
  x.load((const T*)a.x + r * a.x_stride, a.hidden, t);
  for (; r < a.rows; r += step) {
    Row<T, VE, VPT, WPR> next;
    if (r + step < a.rows) next.load((const T*)a.x + (r + step) * a.x_stride, a.hidden, t);
    float s = 0;
#pragma unroll
    for (int k = 0; k < VPT; ++k)
#pragma unroll
      for (int e = 0; e < VE; ++e) s += x.a[k].get(e);
    const float mean = row_sum<WPR>(s, lds, 0) / a.elements;
    float q = 0;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int at = (k * kThreads + t) * VE;
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float d = x.a[k].get(e) - mean;
        if (at < a.hidden) q += d * d;
      }
    }
    const float var = row_sum<WPR>(q, lds, 1) / a.elements;
    const float rstd = 1.f / sqrtf(var + a.eps);
    T* y = (T*)a.y + r * a.y_stride;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int at = (k * kThreads + t) * VE;
      if (at < a.hidden) {
        Pack<T, VE> o;
#pragma unroll
        for (int e = 0; e < VE; ++e) o.set(e, (x.a[k].get(e) - mean) * rstd * w.a[k][e] + b.a[k][e]);
        store_once<T, VE>(y + at, o);
      }
    }
    if (t == 0) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
    x = next;
  }
}

// Backward: as the forward pass, with the two sums of a row taken together.
// Each thread also adds up dy xhat and dy of its columns over its rows; the sums
// of a workgroup go to `partial`, and k_norm_columns adds those in a fixed
// order.
template <class T, int VE, int VPT, int WPR>
__global__ __launch_bounds__(WPR == 1 ? 256 : 64 * WPR) void k_norm_backward(NormArgs a) {
  constexpr int kThreads = 64 * WPR;
  constexpr int kRows = WPR == 1 ? 4 : 1;
  constexpr bool kAhead = VE > 1 || VPT < 24;      // 24 single elements leave no registers for the next row's
  constexpr int R = VE > 1 && sizeof(T) == 2 && VPT * VE <= 16 ? 2 : 1;      // rows at a time
  __shared__ float lds[2][2 * R][WPR];
  const int t = threadIdx.x % kThreads;
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t r = (int64_t)blockIdx.x * kRows + (WPR == 1 ? threadIdx.x >> 6 : 0);

  Vector<T, VE, VPT, WPR> w;
  w.load(a.weight, a.wide_weight, 1.f, a.hidden, t);
  float dw[VPT][VE], db[VPT][VE];
#pragma unroll
  for (int k = 0; k < VPT; ++k)
#pragma unroll
    for (int e = 0; e < VE; ++e) dw[k][e] = db[k][e] = 0.f;

  // R rows, `step` apart; one past the last counts as zeros.
  struct Rows {
    Row<T, VE, VPT, WPR> x[R], g[R];
    float mean[R], rstd[R];
    __device__ __forceinline__ void load(const NormArgs& a, int64_t r, int64_t step, int t) {
#pragma unroll
      for (int i = 0; i < R; ++i, r += step) {
        const bool some = r < a.rows;
        x[i].load((const T*)a.x + (some ? r : 0) * a.x_stride, some ? a.hidden : 0, t);
        g[i].load((const T*)a.dy + (some ? r : 0) * a.dy_stride, some ? a.hidden : 0, t);
        mean[i] = some ? a.mean[r] : 0.f;
        rstd[i] = some ? a.rstd[r] : 0.f;
      }
    }
  };
  Rows now;
  now.load(a, r, step, t);
  for (int slot = 0; r < a.rows; r += R * step, slot ^= 1) {
    Rows next;
    if (kAhead) next.load(a, r + R * step, step, t);
    float s[R], q[R];                              // sums of a and a xhat
#pragma unroll
    for (int i = 0; i < R; ++i) {
      s[i] = q[i] = 0;
#pragma unroll
      for (int k = 0; k < VPT; ++k)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float gy = now.g[i].a[k].get(e), xh = (now.x[i].a[k].get(e) - now.mean[i]) * now.rstd[i];
          const float p = gy * w.a[k][e];
          dw[k][e] += gy * xh;                     // past the row gy is 0
          db[k][e] += gy;
          s[i] += p;
          q[i] += p * xh;
        }
      s[i] = reduce64<Add>(s[i]);
      q[i] = reduce64<Add>(q[i]);
    }
    if constexpr (WPR > 1) {                       // one barrier for all: the next rows' slots are other ones
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < R; ++i) {
          lds[slot][2 * i][threadIdx.x >> 6] = s[i];
          lds[slot][2 * i + 1][threadIdx.x >> 6] = q[i];
        }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < R; ++i) {
        s[i] = q[i] = 0;
#pragma unroll
        for (int v = 0; v < WPR; ++v) {
          s[i] += lds[slot][2 * i][v];
          q[i] += lds[slot][2 * i + 1][v];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t row = r + i * step;
      if (row >= a.rows) break;
      const float ms = s[i] / a.elements, mq = q[i] / a.elements;
      T* dx = (T*)a.y + row * a.y_stride;
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int at = (k * kThreads + t) * VE;
        if (at < a.hidden) {
          Pack<T, VE> o;
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float xh = (now.x[i].a[k].get(e) - now.mean[i]) * now.rstd[i];
            o.set(e, now.rstd[i] * (now.g[i].a[k].get(e) * w.a[k][e] - ms - xh * mq));
          }
          store_once<T, VE>(dx + at, o);
        }
      }
    }
    if (kAhead)
      now = next;
    else
      now.load(a, r + R * step, step, t);
  }
  if (!a.partial) return;
  if constexpr (WPR == 1) {                        // the waves' sums, added to the first one's in order
    __shared__ float sums[2][64 * VPT * VE];
    for (int w = 3; w > 0; --w) {
      if ((int)(threadIdx.x >> 6) == w)
#pragma unroll
        for (int k = 0; k < VPT * VE; ++k) {
          sums[0][k * 64 + t] = dw[k / VE][k % VE];
          sums[1][k * 64 + t] = db[k / VE][k % VE];
        }
      __syncthreads();
      if ((int)(threadIdx.x >> 6) == w - 1)
#pragma unroll
        for (int k = 0; k < VPT * VE; ++k) {
          dw[k / VE][k % VE] += sums[0][k * 64 + t];
          db[k / VE][k % VE] += sums[1][k * 64 + t];
        }
      __syncthreads();
    }
    if (threadIdx.x >= 64) return;
  }
  float* const p = a.partial + (int64_t)blockIdx.x * 2 * a.hidden;
#pragma unroll
  for (int k = 0; k < VPT; ++k) {
    const int at = (k * kThreads + t) * VE;
    if (at < a.hidden) {
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        p[at + e] = dw[k][e];
        p[a.hidden + at + e] = db[k][e];
      }
    }
  }
}

// Sums of the partial rows: 64 columns a workgroup, its 16 waves each adding
// every 16th row, 32 of their loads in flight (the rows come from other XCDs'
// writes, some 2 us away: with 8 in flight 512 rows took 11.8 us), then the 16
// sums in order.
__global__ __launch_bounds__(1024) void k_norm_columns(const float* partial, int32_t groups, int32_t hidden, float* dweight,
                                                       float* dbias, int32_t accumulate) {
  __shared__ float lds[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t columns = 2 * (int64_t)hidden, column = (int64_t)blockIdx.x * 64 + lane;
  float s = 0;
  if (column < columns)
    for (int g = wave; g < groups; g += 512) {
      float x[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) x[i] = g + 16 * i < groups ? partial[(g + 16 * i) * columns + column] : 0.f;
#pragma unroll
      for (int d = 16; d > 0; d /= 2)
#pragma unroll
        for (int i = 0; i < d; ++i) x[i] += x[i + d];
      s += x[0];
    }
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && column < columns) {
    float sum = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += lds[i][lane];
    float* out = column < hidden ? dweight : dbias;
    const int64_t at = column < hidden ? column : column - hidden;
    if (out) out[at] = accumulate ? out[at] + sum : sum;
  }
}

// How a row of `hidden` elements is laid over threads: elements an access,
// elements a thread, waves a row.
struct Shape {
  int ve, ept, wpr;
};

// The layout that leaves the fewest threads without an element, and of those
// the one of fewest waves. The backward pass has two operands and two sums of
// each element in registers, so it takes fewer elements a thread: 16384 x 3584
// takes 81 us with 16 elements of a thread in 4 waves, 104 with 8 in 8.
Shape shape_of(int32_t hidden, int ve, bool backward) {
  Shape best{ve, 0, 0};
  int least = 1 << 30;
  for (int wpr = 1; wpr <= 8; wpr *= 2)
    for (int ept = wpr == 1 ? 8 : 16; ept <= (backward ? 24 : 32); ept += 8) {
      const int room = 64 * wpr * ept;
      if (room >= hidden && room < least) {
        least = room;
        best.ept = ept;
        best.wpr = wpr;
      }
    }
  return best;
}

// Workgroups: as many as the chip holds at once, but no more than there are
// rows. Those of the backward pass each end in a row of partial sums, so there
// are fewer of them (12 or 16 waves a CU in place of 8 are slower).
int64_t grid_of(const Shape& s, int64_t rows, bool backward) {
  const int64_t per = s.wpr == 1 ? 4 : 1, waves = backward ? 8 : 16;      // waves a CU
  const int64_t resident = kCUs * (waves / (s.wpr == 1 ? 4 : s.wpr));
  return std::min((rows + per - 1) / per, resident);
}

template <class T, int VE, int EPT, int WPR>
hipError_t go(const NormArgs& a, bool backward, int64_t grid, hipStream_t s) {
  const dim3 block(WPR == 1 ? 256 : 64 * WPR);
  if constexpr (EPT <= 24)
    if (backward) return launch(k_norm_backward<T, VE, EPT / VE, WPR>, dim3((unsigned)grid), block, 0, s, a);
  return launch(k_norm_forward<T, VE, EPT / VE, WPR>, dim3((unsigned)grid), block, 0, s, a);
}

template <class T, int VE, int WPR>
hipError_t go(const NormArgs& a, int ept, bool backward, int64_t grid, hipStream_t s) {
  if constexpr (WPR == 1)
    if (ept == 8) return go<T, VE, 8, WPR>(a, backward, grid, s);
  if (ept == 16) return go<T, VE, 16, WPR>(a, backward, grid, s);
  if (ept == 24) return go<T, VE, 24, WPR>(a, backward, grid, s);
  return go<T, VE, 32, WPR>(a, backward, grid, s);
}

template <class T, int VE>
hipError_t go(const NormArgs& a, const Shape& p, bool backward, int64_t grid, hipStream_t s) {
  switch (p.wpr) {
    case 1: return go<T, VE, 1>(a, p.ept, backward, grid, s);
    case 2: return go<T, VE, 2>(a, p.ept, backward, grid, s);
    case 4: return go<T, VE, 4>(a, p.ept, backward, grid, s);
    default: return go<T, VE, 8>(a, p.ept, backward, grid, s);
  }
}

hipError_t go(const NormArgs& a, const Shape& p, int32_t type, bool backward, int64_t grid, hipStream_t s) {
  if (type == FP_F32) return p.ve == 1 ? go<float, 1>(a, p, backward, grid, s) : go<float, 4>(a, p, backward, grid, s);
  if (type == FP_BF16) return p.ve == 1 ? go<bf16, 1>(a, p, backward, grid, s) : go<bf16, 8>(a, p, backward, grid, s);
  return p.ve == 1 ? go<f16, 1>(a, p, backward, grid, s) : go<f16, 8>(a, p, backward, grid, s);
}

fp_status check(const char* what, int64_t rows, int32_t hidden, int32_t type, int32_t wtype) {
  if (rows < 0 || rows > kMaxRows) return report(FP_EINVAL, "%s: %lld rows", what, (long long)rows);
  if (hidden < 1 || hidden > kMaxHidden) return report(FP_EINVAL, "%s: hidden %d outside [1, %d]", what, hidden, kMaxHidden);
  if (type != FP_F32 && type != FP_BF16 && type != FP_F16) return report(FP_EINVAL, "%s: type %d", what, type);
  if (wtype != FP_F32 && wtype != type) return report(FP_EINVAL, "%s: weight type %d with type %d", what, wtype, type);
  return FP_OK;
}

struct Operand {
  const void* p;
  int64_t stride;       // elements; 0 for a vector
  int size;
  const char* name;
};

// Checks pointers and strides, and finds whether all can move 16 bytes a row
// operand's access (and the matching elements of the vectors).
template <int N>
fp_status operands(const char* what, const Operand (&ops)[N], int64_t rows, int32_t hidden, int size, bool* wide) {
  const int ve = 16 / size;
  *wide = hidden % ve == 0;
  for (const Operand& o : ops) {
    if (!o.p) continue;
    if (!aligned(o.p, o.size)) return report(FP_EALIGN, "%s: %s is not aligned to its elements", what, o.name);
    if (o.stride && o.stride < hidden)
      return report(FP_EINVAL, "%s: %s has row stride %lld, hidden is %d", what, o.name, (long long)o.stride, hidden);
    if (o.stride > (1ll << 40)) return report(FP_EINVAL, "%s: %s has row stride %lld", what, o.name, (long long)o.stride);
    const bool rows16 = o.stride == 0 || rows < 2 || o.stride % ve == 0;
    if (!aligned(o.p, 16) || !rows16) *wide = false;
  }
  return FP_OK;
}

}  // namespace
}  // namespace fp

using namespace fp;

extern "C" {

fp_status norm_forward(const void* x, int64_t x_stride, const void* weight, const void* bias, void* y, int64_t y_stride,
                       float* mean, float* rstd, int64_t rows, int32_t hidden, float eps, int32_t type,
                       int32_t weight_type, void* stream) {
  fp_status st = check("norm_forward", rows, hidden, type, weight_type);
  if (st != FP_OK) return st;
  if (!(eps > 0)) return report(FP_EINVAL, "norm_forward: eps is not above 0");
  if (rows == 0) return FP_OK;
  if (!x || !y || !mean || !rstd) return report(FP_EINVAL, "norm_forward: null x, y, mean or rstd");
  const int size = type_size(type), wsize = type_size(weight_type);
  if (x_stride < hidden || y_stride < hidden) return report(FP_EINVAL, "norm_forward: a row stride is below hidden");
  const Operand ops[] = {{x, x_stride, size, "x"}, {y, y_stride, size, "y"}, {weight, 0, wsize, "weight"}, {bias, 0, wsize, "bias"}};
  bool wide;
  if ((st = operands("norm_forward", ops, rows, hidden, size, &wide)) != FP_OK) return st;
  if (!aligned(mean, 4) || !aligned(rstd, 4)) return report(FP_EALIGN, "norm_forward: mean or rstd is not aligned");
  NormArgs a{};
  a.x = x, a.weight = weight, a.bias = bias, a.y = y, a.mean = mean, a.rstd = rstd;
  a.x_stride = x_stride, a.y_stride = y_stride;
  a.rows = (int32_t)rows, a.hidden = hidden, a.eps = eps, a.elements = (float)hidden;
  a.wide_weight = weight_type == FP_F32;
  const Shape p = shape_of(hidden, wide ? 16 / size : 1, false);
  return launched(go(a, p, type, false, grid_of(p, rows, false), (hipStream_t)stream), "norm_forward");
}

int64_t norm_workspace(int64_t rows, int32_t hidden) {
  const fp_status st = check("norm_workspace", rows, hidden, FP_F32, FP_F32);
  if (st != FP_OK) return st;
  return std::min<int64_t>(rows, kCUs * 4) * 2 * hidden * (int64_t)sizeof(float);   // grid_of()'s most, of 2 waves a row
}

fp_status norm_backward(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const void* weight,
                        const float* mean, const float* rstd, void* dx, int64_t dx_stride, float* dweight, float* dbias,
                        int64_t rows, int32_t hidden, int32_t type, int32_t weight_type, int32_t accumulate,
                        void* workspace, int64_t workspace_bytes, void* stream) {
  fp_status st = check("norm_backward", rows, hidden, type, weight_type);
  if (st != FP_OK) return st;
  if (rows && (!dy || !x || !dx || !mean || !rstd)) return report(FP_EINVAL, "norm_backward: null dy, x, dx, mean or rstd");
  const int size = type_size(type), wsize = type_size(weight_type);
  if (rows && (dy_stride < hidden || x_stride < hidden || dx_stride < hidden))
    return report(FP_EINVAL, "norm_backward: a row stride is below hidden");
  const Operand ops[] = {{dy, dy_stride, size, "dy"}, {x, x_stride, size, "x"}, {dx, dx_stride, size, "dx"},
                         {weight, 0, wsize, "weight"}};
  bool wide;
  if ((st = operands("norm_backward", ops, rows, hidden, size, &wide)) != FP_OK) return st;
  if (!aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dweight, 4) || !aligned(dbias, 4))
    return report(FP_EALIGN, "norm_backward: mean, rstd, dweight or dbias is not aligned");
  const bool sums = dweight || dbias;
  const int64_t need = norm_workspace(rows, hidden);
  if (sums && rows) {
    if (workspace_bytes < need)
      return report(FP_ECAPACITY, "norm_backward: workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
    if (!workspace) return report(FP_EINVAL, "norm_backward: null workspace");
    if (!aligned(workspace, 256)) return report(FP_EALIGN, "norm_backward: workspace is not 256-byte aligned");
  }
  const hipStream_t s = (hipStream_t)stream;
  int64_t groups = 0;
  if (rows) {
    NormArgs a{};
    a.x = x, a.dy = dy, a.weight = weight, a.y = dx;
    a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd), a.partial = sums ? (float*)workspace : nullptr;
    a.x_stride = x_stride, a.y_stride = dx_stride, a.dy_stride = dy_stride;
    a.rows = (int32_t)rows, a.hidden = hidden, a.elements = (float)hidden;
    a.wide_weight = weight_type == FP_F32;
    const Shape p = shape_of(hidden, wide ? 16 / size : 1, true);
    const int64_t grid = grid_of(p, rows, true);
    groups = grid;
    if ((st = launched(go(a, p, type, true, grid, s), "norm_backward")) != FP_OK) return st;
  }
  if (!sums || (accumulate && !rows)) return FP_OK;
  const unsigned blocks = (unsigned)((2 * (int64_t)hidden + 63) / 64);
  return launched(launch(k_norm_columns, dim3(blocks), dim3(1024), 0, s, (const float*)workspace, (int32_t)groups, hidden, dweight,
                         dbias, accumulate),
                  "norm_backward");
}

}  // extern "C"
