// One AdamW step over many tensors (adamw_step of include/flowpool_train.h)
// and the values of 8-bit states.
//
// Every element is read and written once: param, grad, two states, and the
// 16-bit copy. The bound is HBM bytes: 30 an element with f32 gradients and
// states and a copy, 16 with 16-bit gradients and 8-bit states.
//
// A launch takes up to kTensors tensors, listed in its arguments, or any number
// listed in a table in device memory, and cuts each into chunks of kChunk
// elements, a workgroup each. (290 tensors of 6690 elements on average took 63
// us in 7 launches of 9, most of it their latency.) A lane has 4
// consecutive elements at a time, so a wave's accesses are whole lines in every
// type, and a run of 256 elements that share 8-bit scales is one wave's: its
// largest values are found with cross-lane exchanges and its new codes are made
// from the values still in registers, so the state is never held in 32 bits in
// memory. A chunk's loads are all issued before the first is used (4 accesses
// of each operand; 2 and 8 are slower), and all pass the caches by (plain loads or
// stores are slower).
//
// Measured at 545 million values: f32 gradients and states with a bf16 copy 2.91
// ms, 5.6 TB/s; bf16 gradients, 8-bit states and a copy 1.59 ms, 5.5 TB/s, where the
// 93 vector instructions of a value take every issue slot, and 0.46 ms for the
// values of each state (a large copy's rate); 290 tensors of 6690 values on
// average (707 chunks, 290 of them ragged) 15.4 us.
//
// The codes have to come out alike wherever they are computed from the same
// inputs, so the state's arithmetic is separate multiplications and additions
// (no fused ones, whose single rounding depends on the compiler), and a code
// is decided by comparing with its exact thresholds; the square roots that
// lead near it need no particular last bit.

#include "train_internal.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace fp {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 4;                        // consecutive elements of a thread
constexpr int kStep = kThreads * kVec;
constexpr int kSteps = 4;
constexpr int kChunk = kSteps * kStep;         // elements of a workgroup
static_assert(FP_ADAMW_BLOCK == 64 * kVec, "a run of shared scales is a wave's");
static_assert(kVec == 4, "a thread's smallest v, and whether any value is NaN, are taken of 4");
constexpr int kTensors = 48;                   // of one launch
// Runs whose scale is below kSmall are worked on times kLift, which is exact: the
// reciprocals that lead to codes would overflow, and what one unit of a level
// stands for would lose bits below the normal numbers.
constexpr float kSmall = 0x1p-64f, kLift = 0x1p84f, kRootLift = 0x1p-42f;   // the last: the root of 1 / kLift
constexpr float kNormal = 0x1p-126f;
constexpr float kNone = 0x1p-80f;              // below any other scale's reciprocal: for runs of zeros
constexpr float kTopM = 127.f * 127.f, kTopV = 65025.f * 65025.f;   // 127^2, 255^4

struct Tensor {
  void* param;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  void* copy;
  int64_t n;
  float weight_decay;
  uint32_t wide;                               // all pointers allow vectors
};
static_assert(sizeof(Tensor) == 72, "Tensor layout");

// What a step does to each element: om = 1 - beta, rate = lr / bc1, far = 1 / sqrt(bc2).
struct Rates {
  double lr;
  float beta1, om1, beta2, om2, rate, far, eps;
  int32_t copy_type;
};

// A table: this, the first workgroup of each tensor, the tensors.
struct TableHead {
  int64_t groups;
  int32_t n, types;                            // types_of() what they were checked for
  int64_t tensors_at;                          // byte offset
};
constexpr int64_t kFirstAt = 64;
static_assert(sizeof(TableHead) <= kFirstAt, "table layout");

struct AdamArgs {
  const float* grad_scale;
  Rates r;
  int32_t n;
  uint32_t first[kTensors];                    // first workgroup of each tensor
  Tensor t[kTensors];
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments stay within 4 KiB");

struct TableArgs {
  char* table;
  TableHead head;
  int32_t at, n;                               // which tensors
  uint32_t first[kTensors];
  Tensor t[kTensors];
};
static_assert(sizeof(TableArgs) <= 4096, "kernel arguments stay within 4 KiB");

// A thread's elements of one operand, as they lie in memory. `left` of them exist
// (all, with kWhole, and then they are one access).
template <class T>
struct Some {
  Pack<T, kVec> a;
  template <bool kWhole>
  __device__ __forceinline__ void read(const T* p, int left) {
    if constexpr (kWhole) {
      a = load_once<T, kVec>(p);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) a.v[e] = e < left ? p[e] : (T)0;
    }
  }
  template <bool kWhole>
  __device__ __forceinline__ void write(T* p, int left) const {
    if constexpr (kWhole) {
      store_once<T, kVec>(p, a);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (e < left) p[e] = a.v[e];
    }
  }
};

// c (c + 1) + 1/4 = (c + 1/2)^2, exact for c up to 255.
__device__ __forceinline__ float above(float c) { return c * (c + 1.f) + 0.25f; }

// The level of t, given its root to within 8 units of its last place: the
// largest c with t at or above c - 1/2 to the same power. The root less kLow
// leads to it or to the one below it, so one comparison decides (NaN: level 0).
// t is at most the top level's by two roundings, so no level is above that. A
// run that holds a NaN has a NaN for its scale, and one that holds an infinity
// that: their levels are 0.
constexpr float kLow = 0x1p-12f;               // 16 units of the last place of 255
// t = |m| 127^2 / scale, r its square root.
__device__ __forceinline__ uint32_t level_m(float t, float r) {
  const float c = fmaxf(rintf(r - kLow), 0.f);
  return (uint32_t)c + (t >= above(c) ? 1u : 0u);
}
// t = v 255^4 / scale, r its fourth root.
__device__ __forceinline__ uint32_t level_v(float t, float r) {
#pragma clang fp contract(off)
  const float c = fmaxf(rintf(r - kLow), 0.f);
  return (uint32_t)c + (t >= above(c) * above(c) ? 1u : 0u);
}

// What a unit of the level's power stands for (times kLift for a small scale).
__device__ __forceinline__ float unit_of(float scale, float top) { return (scale < kSmall ? scale * kLift : scale) * (1.f / top); }
__device__ __forceinline__ float value_m(uint32_t code, float unit) {   // unit = scale / 127^2
#pragma clang fp contract(off)
  const float c = (float)(code & 127u), q = c * c * unit;
  return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, q) ^ (code & 128u) << 24);
}
__device__ __forceinline__ float value_v(uint32_t code, float unit) {   // unit = scale / 255^4
#pragma clang fp contract(off)
  const float c = (float)code, q = c * c;
  return q * q * unit;
}

// A thread's 4 elements of a tensor, from element `at` on.
template <class P, class G, bool kEight, bool kWhole>
struct Step {
  using S = std::conditional_t<kEight, uint8_t, float>;
  Some<P> p;
  Some<G> g;
  Some<S> m, v;
  float sm, sv;                                  // 8 bits: scales

  __device__ __forceinline__ void read(const Tensor& t, int64_t at, int left) {
    p.template read<kWhole>((const P*)t.param + at, left);
    g.template read<kWhole>((const G*)t.grad + at, left);
    m.template read<kWhole>((const S*)t.m + at, left);
    v.template read<kWhole>((const S*)t.v + at, left);
    if constexpr (kEight) {
      // past the tensor there is no scale
      sm = kWhole || left > 0 ? t.m_scale[at / FP_ADAMW_BLOCK] : 0.f;
      sv = kWhole || left > 0 ? t.v_scale[at / FP_ADAMW_BLOCK] : 0.f;
    }
  }

  // All 64 lanes of a run come here together.
  __device__ __forceinline__ void finish(const Rates& a, const Tensor& t, float keep, int64_t at, int left, float gs) {
#pragma clang fp contract(off)
    float np[kVec], nm[kVec], nv[kVec], rv[kVec];
    if constexpr (kEight) {
      const float um = unit_of(sm, kTopM), uv = unit_of(sv, kTopV);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        nm[e] = value_m(m.a.v[e], um);
        nv[e] = value_v(v.a.v[e], uv);
      }
      if (sm < kSmall)                           // all lanes of a run or none, so it costs a test as a rule
#pragma unroll
        for (int e = 0; e < kVec; ++e) nm[e] *= 1.f / kLift;
      if (sv < kSmall)
#pragma unroll
        for (int e = 0; e < kVec; ++e) nv[e] *= 1.f / kLift;
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        nm[e] = m.a.v[e];
        nv[e] = v.a.v[e];
      }
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const float ge = g.a.get(e) * gs;
      nm[e] = nm[e] * a.beta1 + ge * a.om1;
      nv[e] = nv[e] * a.beta2 + ge * ge * a.om2;
      // the update is a small part of the parameter: the hardware's root and reciprocal (1 ulp) serve it
      rv[e] = __builtin_amdgcn_sqrtf(nv[e]);
    }
    // below the normal numbers that root is 0
    if (fminf(fminf(nv[0], nv[1]), fminf(nv[2], nv[3])) < kNormal)
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (nv[e] < kNormal) rv[e] = __builtin_amdgcn_sqrtf(nv[e] * kLift) * kRootLift;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const float away = __builtin_fmaf(rv[e], a.far, a.eps);
      np[e] = __builtin_fmaf(p.a.get(e), keep, -(nm[e] * a.rate * __builtin_amdgcn_rcpf(away)));
      p.a.set(e, np[e]);
    }
    p.template write<kWhole>((P*)t.param + at, left);
    if (a.copy_type == FP_BF16) {
      Some<bf16> c;
#pragma unroll
      for (int e = 0; e < kVec; ++e) c.a.set(e, np[e]);
      c.template write<kWhole>((bf16*)t.copy + at, left);
    } else if (a.copy_type == FP_F16) {
      Some<f16> c;
#pragma unroll
      for (int e = 0; e < kVec; ++e) c.a.set(e, np[e]);
      c.template write<kWhole>((f16*)t.copy + at, left);
    }
    if constexpr (kEight) {
      float hm = 0.f, hv = 0.f;                  // elements past the tensor are zeros
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        hm = fmaxf(hm, fabsf(nm[e]));
        hv = fmaxf(hv, nv[e]);
      }
      hm = reduce64<Max>(hm);
      hv = reduce64<Max>(hv);
      // a maximum passes over a NaN
      if (__ballot(__builtin_isunordered(nm[0], nm[1]) | __builtin_isunordered(nm[2], nm[3]))) hm = __builtin_nanf("");
      if (__ballot(__builtin_isunordered(nv[0], nv[1]) | __builtin_isunordered(nv[2], nv[3]))) hv = __builtin_nanf("");
      float lm = hm, lv = hv;                    // what the codes are made against
      if (hm < kSmall) {
        lm *= kLift;
#pragma unroll
        for (int e = 0; e < kVec; ++e) nm[e] *= kLift;
      }
      if (hv < kSmall) {
        lv *= kLift;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          nv[e] *= kLift;
          rv[e] = __builtin_amdgcn_sqrtf(nv[e]);
        }
      }
      // (a NaN stays one)
      const float im = 1.f / (lm < kNone ? kNone : lm) * kTopM, iv = 1.f / (lv < kNone ? kNone : lv) * kTopV;
      const float riv = __builtin_amdgcn_sqrtf(iv);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float tm = fabsf(nm[e]) * im;
        m.a.v[e] = (uint8_t)(level_m(tm, __builtin_amdgcn_sqrtf(tm)) | (nm[e] < 0.f ? 128u : 0u));
        // a v that is not 0 has a level that is not
        v.a.v[e] = (uint8_t)std::max(level_v(nv[e] * iv, __builtin_amdgcn_sqrtf(rv[e] * riv)), nv[e] > 0.f ? 1u : 0u);
      }
      if (threadIdx.x % 64 == 0 && (kWhole || left > 0)) {
        t.m_scale[at / FP_ADAMW_BLOCK] = hm;
        t.v_scale[at / FP_ADAMW_BLOCK] = hv;
      }
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        m.a.v[e] = nm[e];
        v.a.v[e] = nv[e];
      }
    }
    m.template write<kWhole>((S*)t.m + at, left);
    v.template write<kWhole>((S*)t.v + at, left);
  }
};

// The tensor of workgroup `group`, the last that starts by it: 64 of the starts
// are compared at once, so 4096 tensors take two loads.
__device__ __forceinline__ int tensor_of(const uint32_t* first, int n, uint32_t group) {
  int lo = 0;
  while (n > 1) {
    const int stride = (n + 63) / 64, i = (threadIdx.x & 63) * stride;
    const bool by = i < n && first[lo + i] <= group;
    const int in = (__popcll(__ballot(by)) - 1) * stride;
    lo += in;
    n = min(stride, n - in);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

template <class P, class G, bool kEight>
__device__ __forceinline__ void chunk(const Rates& r, const Tensor& t, int64_t start, const float* grad_scale) {
  const float gs = grad_scale ? *grad_scale : 1.f;
  if (!(fabsf(gs) <= 3.4028234e38f)) return;
  const float keep = (float)(1.0 - r.lr * (double)t.weight_decay);
  const int64_t mine = threadIdx.x * kVec;
  if (t.wide && start + kChunk <= t.n) {
    Step<P, G, kEight, true> s[kSteps];
#pragma unroll
    for (int k = 0; k < kSteps; ++k) s[k].read(t, start + k * kStep + mine, kVec);
#pragma unroll
    for (int k = 0; k < kSteps; ++k) s[k].finish(r, t, keep, start + k * kStep + mine, kVec, gs);
  } else {
    for (int k = 0; k < kSteps; ++k) {
      const int64_t base = start + k * kStep, at = base + mine;
      if (base >= t.n) return;
      const int left = (int)std::min<int64_t>(std::max<int64_t>(t.n - at, 0), kVec);
      Step<P, G, kEight, false> s;
      s.read(t, at, left);
      s.finish(r, t, keep, at, left, gs);
    }
  }
}

template <class P, class G, bool kEight>
__global__ __launch_bounds__(kThreads) void k_adamw(AdamArgs a) {
  const int i = tensor_of(a.first, a.n, blockIdx.x);
  chunk<P, G, kEight>(a.r, a.t[i], (int64_t)(blockIdx.x - a.first[i]) * kChunk, a.grad_scale);
}

template <class P, class G, bool kEight>
__global__ __launch_bounds__(kThreads) void k_adamw_table(const char* table, int64_t groups, int32_t types, const float* grad_scale,
                                                          Rates r) {
  const TableHead h = *(const TableHead*)table;
  if (h.types != types || h.groups != groups) return;           // a table for something else
  const uint32_t* const first = (const uint32_t*)(table + kFirstAt);
  const int i = tensor_of(first, h.n, blockIdx.x);
  const Tensor t = ((const Tensor*)(table + h.tensors_at))[i];
  chunk<P, G, kEight>(r, t, (int64_t)(blockIdx.x - first[i]) * kChunk, grad_scale);
}

__global__ __launch_bounds__(64) void k_table(TableArgs a) {
  if (threadIdx.x == 0 && a.at == 0) *(TableHead*)a.table = a.head;
  if ((int)threadIdx.x < a.n) {
    ((uint32_t*)(a.table + kFirstAt))[a.at + threadIdx.x] = a.first[threadIdx.x];
    ((Tensor*)(a.table + a.head.tensors_at))[a.at + threadIdx.x] = a.t[threadIdx.x];
  }
}

template <int kMoment, bool kWhole>
__device__ __forceinline__ void values(const uint8_t* codes, const float* scales, float* out, int64_t n, int64_t start) {
#pragma clang fp contract(off)
  constexpr float kTop = kMoment == 1 ? kTopM : kTopV;
  Some<uint8_t> c[kSteps];
  float scale[kSteps];
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    const int64_t at = start + k * kStep;
    const int left = kWhole ? kVec : (int)std::min<int64_t>(std::max<int64_t>(n - at, 0), kVec);
    c[k].read<kWhole>(codes + at, left);
    scale[k] = left ? scales[at / FP_ADAMW_BLOCK] : 0.f;
  }
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    const int64_t at = start + k * kStep;
    const float unit = unit_of(scale[k], kTop), lift = scale[k] < kSmall ? 1.f / kLift : 1.f;
    Some<float> f;
#pragma unroll
    for (int e = 0; e < kVec; ++e) f.a.v[e] = (kMoment == 1 ? value_m(c[k].a.v[e], unit) : value_v(c[k].a.v[e], unit)) * lift;
    f.write<kWhole>(out + at, kWhole ? kVec : (int)std::min<int64_t>(std::max<int64_t>(n - at, 0), kVec));
  }
}

template <int kMoment>
__global__ __launch_bounds__(kThreads) void k_state_values(const uint8_t* codes, const float* scales, float* out, int64_t n,
                                                           uint32_t wide) {
  const int64_t start = (int64_t)blockIdx.x * kChunk + threadIdx.x * kVec;
  if (wide && (int64_t)(blockIdx.x + 1) * kChunk <= n)
    values<kMoment, true>(codes, scales, out, n, start);
  else
    values<kMoment, false>(codes, scales, out, n, start);
}

fp_status check(const char* what, const fp_adamw_config* c, int32_t n_tensors) {
  if (!c) return report(FP_EINVAL, "%s: null config", what);
  if (n_tensors < 0) return report(FP_EINVAL, "%s: %d tensors", what, n_tensors);
  if (c->step < 1) return report(FP_EINVAL, "%s: step %lld", what, (long long)c->step);
  if (!(c->lr >= 0 && std::isfinite(c->lr)) || !(c->eps >= 0 && std::isfinite(c->eps)))
    return report(FP_EINVAL, "%s: lr %g or eps %g", what, c->lr, c->eps);
  if (!(c->beta1 >= 0 && c->beta1 < 1) || !(c->beta2 >= 0 && c->beta2 < 1))
    return report(FP_EINVAL, "%s: beta1 %g or beta2 %g outside [0, 1)", what, c->beta1, c->beta2);
  if (c->param_type != FP_F32 && c->param_type != FP_BF16) return report(FP_EINVAL, "%s: param type %d", what, c->param_type);
  if (c->grad_type != FP_F32 && c->grad_type != FP_BF16 && c->grad_type != FP_F16)
    return report(FP_EINVAL, "%s: grad type %d", what, c->grad_type);
  if (c->state_bits != 32 && c->state_bits != 8) return report(FP_EINVAL, "%s: states of %d bits", what, c->state_bits);
  if (c->copy_type != -1 && c->copy_type != FP_BF16 && c->copy_type != FP_F16)
    return report(FP_EINVAL, "%s: copy type %d", what, c->copy_type);
  if (c->copy_type != -1 && c->param_type != FP_F32) return report(FP_EINVAL, "%s: a copy of 16-bit parameters", what);
  return FP_OK;
}

fp_status check(const char* what, const fp_adamw_tensor& t, int32_t i, const fp_adamw_config* c) {
  const bool eight = c->state_bits == 8, copy = c->copy_type != -1;
  if (t.n < 0 || t.n > (1ll << 40) || t.reserved) return report(FP_EINVAL, "%s: tensor %d: n %lld", what, i, (long long)t.n);
  if (!std::isfinite(t.weight_decay)) return report(FP_EINVAL, "%s: tensor %d: weight decay", what, i);
  if ((t.copy != nullptr) != copy && t.n) return report(FP_EINVAL, "%s: tensor %d: copy and its type disagree", what, i);
  if ((t.m_scale || t.v_scale) && !eight) return report(FP_EINVAL, "%s: tensor %d: scales with 32-bit states", what, i);
  if (!t.n) return FP_OK;
  if (!t.param || !t.grad || !t.m || !t.v || (eight && (!t.m_scale || !t.v_scale)))
    return report(FP_EINVAL, "%s: tensor %d: null pointer", what, i);
  if (!aligned(t.param, type_size(c->param_type)) || !aligned(t.grad, type_size(c->grad_type)) || !aligned(t.copy, 2) ||
      !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4) || (!eight && (!aligned(t.m, 4) || !aligned(t.v, 4))))
    return report(FP_EALIGN, "%s: tensor %d: a pointer is not aligned to its elements", what, i);
  return FP_OK;
}

template <class P>
void (*kernel_of(int32_t grad_type, bool eight))(AdamArgs) {
  if (grad_type == FP_F32) return eight ? k_adamw<P, float, true> : k_adamw<P, float, false>;
  if (grad_type == FP_BF16) return eight ? k_adamw<P, bf16, true> : k_adamw<P, bf16, false>;
  return eight ? k_adamw<P, f16, true> : k_adamw<P, f16, false>;
}
template <class P>
void (*table_kernel_of(int32_t grad_type, bool eight))(const char*, int64_t, int32_t, const float*, Rates) {
  if (grad_type == FP_F32) return eight ? k_adamw_table<P, float, true> : k_adamw_table<P, float, false>;
  if (grad_type == FP_BF16) return eight ? k_adamw_table<P, bf16, true> : k_adamw_table<P, bf16, false>;
  return eight ? k_adamw_table<P, f16, true> : k_adamw_table<P, f16, false>;
}

Rates rates_of(const fp_adamw_config* c) {
  Rates r{};
  r.lr = c->lr;
  r.beta1 = (float)c->beta1, r.om1 = (float)(1.0 - c->beta1), r.beta2 = (float)c->beta2, r.om2 = (float)(1.0 - c->beta2);
  r.rate = (float)(c->lr / (1.0 - std::pow(c->beta1, (double)c->step)));
  r.far = (float)(1.0 / std::sqrt(1.0 - std::pow(c->beta2, (double)c->step)));
  // the hardware's reciprocal of what is below the normal numbers is infinite, and 0 times that no number
  r.eps = c->eps > 0 ? std::max((float)c->eps, kNormal) : 0.f;
  r.copy_type = c->copy_type;
  return r;
}

int32_t types_of(const fp_adamw_config* c) {
  return 1 << 24 | c->param_type << 16 | c->grad_type << 12 | c->state_bits << 4 | (c->copy_type + 1);
}

Tensor tensor_of(const fp_adamw_tensor& t, const fp_adamw_config* c) {
  const uintptr_t state = c->state_bits == 8 ? kVec : 4 * kVec;
  const bool wide = aligned(t.param, kVec * type_size(c->param_type)) && aligned(t.grad, kVec * type_size(c->grad_type)) &&
                    aligned(t.m, state) && aligned(t.v, state) && aligned(t.copy, 2 * kVec);
  return Tensor{t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.copy, t.n, t.weight_decay, wide};
}

constexpr uint64_t kMaxGroups = 0x7fffffffu;   // of a launch

fp_status check(const char* what, const fp_adamw_tensor* tensors, int32_t n, const fp_adamw_config* c) {
  for (int32_t i = 0; i < n; ++i) {
    const fp_status st = check(what, tensors[i], i, c);
    if (st != FP_OK) return st;
  }
  return FP_OK;
}

// Hands out checked tensors that have elements in lists of up to kTensors, with
// the first workgroup of each: list(workgroups so far). With `apart` each
// list's workgroups start at 0.
template <class Args, class List>
fp_status lists(const fp_adamw_tensor* tensors, int32_t n, const fp_adamw_config* c, bool apart, Args& a, List list) {
  uint64_t groups = 0;
  for (int32_t i = 0; i <= n; ++i) {
    const bool end = i == n;
    const uint64_t more = end ? 0 : (uint64_t)((tensors[i].n + kChunk - 1) / kChunk);
    if (a.n && (end || a.n == kTensors || (apart && groups + more > kMaxGroups))) {
      const fp_status st = list(groups);
      if (st != FP_OK) return st;
      a.n = 0;
      if (apart) groups = 0;
    }
    if (!more) continue;
    a.first[a.n] = (uint32_t)groups;
    a.t[a.n++] = tensor_of(tensors[i], c);
    groups += more;
  }
  return FP_OK;
}

}  // namespace
}  // namespace fp

using namespace fp;

extern "C" {

fp_status adamw_step(const fp_adamw_tensor* tensors, int32_t n_tensors, const fp_adamw_config* c, const float* grad_scale,
                     void* stream) {
  fp_status st = check("adamw_step", c, n_tensors);
  if (st != FP_OK) return st;
  if (n_tensors && !tensors) return report(FP_EINVAL, "adamw_step: null tensors");
  if (!aligned(grad_scale, 4)) return report(FP_EALIGN, "adamw_step: grad_scale is not aligned");
  AdamArgs a{};
  a.grad_scale = grad_scale;
  a.r = rates_of(c);
  auto* const k = c->param_type == FP_F32 ? kernel_of<float>(c->grad_type, c->state_bits == 8) : kernel_of<bf16>(c->grad_type, c->state_bits == 8);
  if ((st = check("adamw_step", tensors, n_tensors, c)) != FP_OK) return st;
  return lists(tensors, n_tensors, c, true, a, [&](uint64_t groups) {
    return launched(launch(k, dim3((unsigned)groups), dim3(kThreads), 0, (hipStream_t)stream, a), "adamw_step");
  });
}

int64_t adamw_table_bytes(int32_t n_tensors) {
  if (n_tensors < 0) return report(FP_EINVAL, "adamw_table_bytes: %d tensors", n_tensors);
  return kFirstAt + ((int64_t)n_tensors * 4 + 63) / 64 * 64 + (int64_t)n_tensors * (int64_t)sizeof(Tensor);
}

fp_status adamw_table_write(const fp_adamw_tensor* tensors, int32_t n_tensors, const fp_adamw_config* c, void* table,
                            int64_t table_bytes, int64_t* out_groups, void* stream) {
  const char* const what = "adamw_table_write";
  fp_status st = check(what, c, n_tensors);
  if (st != FP_OK) return st;
  if ((n_tensors && !tensors) || !table || !out_groups) return report(FP_EINVAL, "%s: null tensors, table or out_groups", what);
  if (!aligned(table, 256)) return report(FP_EALIGN, "%s: table is not 256-byte aligned", what);
  if (table_bytes < adamw_table_bytes(n_tensors))
    return report(FP_ECAPACITY, "%s: table of %lld bytes, %lld needed", what, (long long)table_bytes, (long long)adamw_table_bytes(n_tensors));
  TableArgs a{};
  a.table = (char*)table;
  a.head.types = types_of(c);
  a.head.tensors_at = kFirstAt + ((int64_t)n_tensors * 4 + 63) / 64 * 64;
  if ((st = check(what, tensors, n_tensors, c)) != FP_OK) return st;
  for (int32_t i = 0; i < n_tensors; ++i) {
    a.head.n += tensors[i].n > 0;
    a.head.groups += (tensors[i].n + kChunk - 1) / kChunk;
    if (a.head.groups > (int64_t)kMaxGroups) return report(FP_EINVAL, "%s: more than 2^31 chunks of %d elements", what, kChunk);
  }
  st = lists(tensors, n_tensors, c, false, a, [&](uint64_t) {
    const fp_status s = launched(launch(k_table, dim3(1), dim3(64), 0, (hipStream_t)stream, a), what);
    a.at += a.n;
    return s;
  });
  if (st == FP_OK) *out_groups = a.head.groups;
  return st;
}

fp_status adamw_table_step(const void* table, int64_t groups, const fp_adamw_config* c, const float* grad_scale, void* stream) {
  const char* const what = "adamw_table_step";
  const fp_status st = check(what, c, 0);
  if (st != FP_OK) return st;
  if (groups < 0 || groups > (int64_t)kMaxGroups) return report(FP_EINVAL, "%s: %lld groups", what, (long long)groups);
  if (!table) return report(FP_EINVAL, "%s: null table", what);
  if (!aligned(table, 256)) return report(FP_EALIGN, "%s: table is not 256-byte aligned", what);
  if (!aligned(grad_scale, 4)) return report(FP_EALIGN, "%s: grad_scale is not aligned", what);
  if (!groups) return FP_OK;
  auto* const k = c->param_type == FP_F32 ? table_kernel_of<float>(c->grad_type, c->state_bits == 8)
                                          : table_kernel_of<bf16>(c->grad_type, c->state_bits == 8);
  return launched(launch(k, dim3((unsigned)groups), dim3(kThreads), 0, (hipStream_t)stream, (const char*)table, groups, types_of(c),
                         grad_scale, rates_of(c)),
                  what);
}

fp_status adamw_state_values(const void* codes, const float* scales, float* out, int64_t n, int32_t moment, void* stream) {
  if (n < 0 || n > (1ll << 40)) return report(FP_EINVAL, "adamw_state_values: n %lld", (long long)n);
  if (moment != 1 && moment != 2) return report(FP_EINVAL, "adamw_state_values: moment %d", moment);
  if (!n) return FP_OK;
  if (!codes || !scales || !out) return report(FP_EINVAL, "adamw_state_values: null pointer");
  if (!aligned(scales, 4) || !aligned(out, 4)) return report(FP_EALIGN, "adamw_state_values: scales or out is not aligned");
  auto* k = moment == 1 ? k_state_values<1> : k_state_values<2>;
  const uint32_t wide = aligned(codes, kVec) && aligned(out, 4 * kVec);
  return launched(launch(k, dim3((unsigned)((n + kChunk - 1) / kChunk)), dim3(kThreads), 0, (hipStream_t)stream, (const uint8_t*)codes,
                         scales, out, n, wide),
                  "adamw_state_values");
}

}  // extern "C"
