// The matrix product of the vocabulary loss: D[p][q] = sum over k of
// P[p][k] Q[q][k] in f32 for 16-bit P and Q, each contiguous in k or (for the
// gradients, whose sums run over classes or rows) across it.
//
// A workgroup of 4 waves makes a 256 x 256 tile of D, 128 x 128 a wave, one
// wave a SIMD: its 256 sums a lane fill half of the registers. Per 64 of k a
// wave reads 32 KiB of LDS for 64 matrix instructions of 32 cycles. The operands
// go from memory to LDS without passing through registers.
//
// A stage is 32 of k, and five stages fit the LDS. While a stage is multiplied
// the next one's fragments are read into the other set of registers, so no
// matrix instruction waits for the LDS; the stage itself is in registers by
// then, and its place free. Stages are loaded in pairs, so that both halves of
// a 128-byte line are asked for together, evenly over a pair's time (loads in a
// burst queue up, and the wave with them) and one to three stages of 1024
// cycles ahead of the barrier behind which they are read. Between two matrix
// instructions stands at most one read and one load: what takes longer to issue
// than an instruction to run leaves the matrix cores idle.
//
// Workgroups are resident and walk over tiles: the first four stages of the next
// tile are asked for before the present one's results are worked on.
//
// In LDS a row's 4 vectors of 16 bytes (32 elements of k) are stored at their
// index exclusive-or a quarter of the row's number modulo 4: 16 lanes that read
// the same vector of 16 consecutive rows touch all 64 banks. A direct load
// writes LDS in lane order, so it is the lanes' global addresses that are
// permuted.
//
// An operand that is contiguous across k needs no transposed copy: its stage is
// 32 k of 256 elements, and the LDS gives it out transposed (4 elements of k of
// one row to a lane, from 4 rows of 32 bytes that 16 lanes address). Its blocks
// of 16 elements b at k are stored at block (b & 8) | ((b & 1) << 2 | (b >> 1 & 3)) ^ (k & 3),
// so that those 4 rows, and the neighbouring 16 lanes' 4, lie in different banks.
#pragma once

#include "train_internal.h"

#include <type_traits>

namespace fp {

constexpr int kTile = 256;                     // rows of P and of Q a workgroup takes
constexpr int kStageK = 32;                    // elements of k a stage
constexpr int kPairK = 2 * kStageK;
constexpr int kPlaces = 5;                     // for stages in LDS
constexpr int kGemmThreads = 256;
constexpr int kOperandBytes = kTile * kStageK * 2;
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kGemmLds = kPlaces * kStageBytes;
// Of LDS each wave has this much for its results: the last place, which the
// loads of the next tile's first two pairs leave free.
constexpr int kOwnBytes = kStageBytes / 4;
constexpr int kOwnAt = (kPlaces - 1) * kStageBytes;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// A value that is the same in all lanes, in a scalar register.
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// c += p q, 32 x 32 sums over 16 of k, in the accumulation registers. As asm,
// because the compiler, left to itself, moves sums between the two halves of the
// register file every time round. It begins with the wait that a matrix
// instruction needs behind a vector instruction that wrote an operand.
template <class T>
__device__ __forceinline__ void mfma(f32x16& c, const u32x4& p, const u32x4& q) {
  if constexpr (__is_same(T, bf16))
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(p), "v"(q));
  else
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+a"(c) : "v"(p), "v"(q));
}

// Behind products: the wait before a vector instruction may read the sums. It
// ends the loop over products, since at a loop's ends the compiler may copy
// sums between registers, and it does not know that an asm block's instruction
// still runs. The next product could not start earlier.
__device__ __forceinline__ void settle() { asm volatile("s_nop 15\n\ts_nop 3"); }

// An operand: `rows` rows (at least 1) of k elements. Contiguous in k: rows are
// `ld` elements apart, and k is a multiple of 8. Across k: elements of k are
// `ld` apart, and `rows` is a multiple of 8. Rows past the last are read as
// some row of it; from k on `zeros` (16 bytes of zeros) is read, so nothing
// outside the operand is touched. 255 ld elements are less than 2^32 bytes.
struct Operand16 {
  const void* p;
  int64_t ld;
  int32_t rows, k;
};

// Addresses in LDS are byte offsets, as scalars where they are the same in all
// lanes.
__device__ __forceinline__ int32_t lds_address(const char* lds) {
  return uniform((int32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)lds);
}

// Loads of 16 bytes a lane that go straight to LDS, to 16 lane from `to` on. As
// asm: the compiler waits for all loads it knows to write LDS before each
// transposed read. They have no result in registers, and what waits for them is
// arrival() below; a wait that the compiler makes for accesses of its own can
// only come out longer for them. m0, which nothing else here uses, holds the
// place.
__device__ __forceinline__ void load_lds(const char* p, int32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(to) : "memory");
}
__device__ __forceinline__ void load_lds(const u32x4& buffer, uint32_t at, int32_t offset, int32_t to) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" : : "v"(at), "s"(buffer), "s"(offset), "s"(to) : "memory");
}

// One operand's loads of a pair of stages: kLoads KiB of each stage by each
// wave, 16 rows of 64 bytes at a time, or (across k) 2 of 512.
template <bool kAcross, int kLoads = 4>
struct Loader {
  static_assert(!kAcross || kLoads == 4, "across k a tile is 256 elements wide");
  const char* tile;           // k 0 (and row 0 of the tile, contiguous in k); uniform
  int64_t pair_bytes;         // from a pair to the next
  uint32_t at[kLoads];        // each lane's vectors, bytes from there
  int32_t k;

  // The lane's first element of k within a stage, at its j-th load.
  __device__ __forceinline__ static int32_t k_of(int j) {
    return kAcross ? (threadIdx.x >> 6) * 8 + j * 2 + (threadIdx.x >> 5 & 1) : ((threadIdx.x & 3) ^ (threadIdx.x >> 4 & 3)) * 8;
  }

  __device__ __forceinline__ void init(const Operand16& o, int32_t first_row) {
    k = o.k;
    pair_bytes = kAcross ? (int64_t)uniform((int32_t)o.ld) * (kPairK * 2) : kPairK * 2;
    const uint64_t t = reinterpret_cast<uint64_t>(o.p) + (kAcross ? 0 : (uint64_t)((int64_t)first_row * o.ld * 2));
    tile = reinterpret_cast<const char*>((uint64_t)(uint32_t)uniform((int32_t)(t >> 32)) << 32 | (uint32_t)uniform((int32_t)t));
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      if constexpr (kAcross) {
        const int32_t v = threadIdx.x & 31, x = (v >> 1 & 7) ^ (k_of(j) & 3), block = (v >> 1 & 8) | (x & 3) << 1 | x >> 2;
        at[j] = (uint32_t)k_of(j) * (uint32_t)(o.ld * 2) + (uint32_t)min(first_row + block * 16 + (v & 1) * 8, o.rows - 8) * 2u;
      } else {
        const int32_t row = (threadIdx.x >> 6) * (16 * kLoads) + (threadIdx.x >> 2 & 15) + j * 16;
        at[j] = (uint32_t)min(row, o.rows - 1 - first_row) * (uint32_t)(o.ld * 2) + (uint32_t)k_of(j) * 2u;
      }
    }
  }

  // A pair as a buffer of so many bytes: -1 for all, 0 for none, whose loads read nothing.
  __device__ __forceinline__ u32x4 buffer(int32_t pair, int32_t bytes) const {
    const uint64_t p = reinterpret_cast<uint64_t>(tile + pair * pair_bytes);
    return u32x4{(uint32_t)uniform((int32_t)p), (uint32_t)uniform((int32_t)(p >> 32)) & 0xffffu, (uint32_t)uniform(bytes), 0x00027000u};
  }

  // The j-th load of stage h of a pair that lies within k, to the stage's place.
  __device__ __forceinline__ void issue(const u32x4& pair, int32_t place, int h, int j) const {
    load_lds(pair, at[j], h * (int32_t)(pair_bytes >> 1), place + uniform(threadIdx.x >> 6) * (kLoads * 1024) + j * 1024);
  }

  // All loads of any pair, to two places.
  __device__ __forceinline__ void issue_all(int32_t place, int32_t pair, const void* zeros, int32_t apart = kStageBytes) const {
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        load_lds((pair * 2 + h) * kStageK + k_of(j) < k ? tile + pair * pair_bytes + h * (pair_bytes >> 1) + at[j] : (const char*)zeros,
                 place + h * apart + uniform(threadIdx.x >> 6) * (kLoads * 1024) + j * 1024);
  }
};

// Sums of the tile's part of a wave: a[i][j][r] holds, in lane l, row
// 128 (wave / 2) + 32 i + 8 (r / 4) + 4 (l / 32) + r % 4 of P and row
// 128 (wave % 2) + 32 j + l % 32 of Q, both within the tile.
struct Acc {
  f32x16 a[4][4];
};
// One sum. As asm, so that it is read where it is used; the compiler would
// first copy all of them, for which there are no registers.
__device__ __forceinline__ float sum_of(const Acc& acc, int i, int j, int r) {
  float x;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(acc.a[i][j][r]));
  return x;
}
__device__ __forceinline__ int wave_p() { return (threadIdx.x >> 7) * 128; }
__device__ __forceinline__ int wave_q() { return (threadIdx.x >> 6 & 1) * 128; }
__device__ __forceinline__ int lane_p() { return (threadIdx.x >> 5 & 1) * 4; }
__device__ __forceinline__ int lane_q() { return threadIdx.x & 31; }

// A stage's fragments: 32 rows at 16 of k, [2 i + h] rows 32 i.. and k 16 h..;
// lane l has row l % 32, elements 8 (l / 32) + 0..7 of the 16.
struct Fragments {
  u32x4 p[8], q[8];
};

// Waits for this wave's LDS accesses, and for all waves.
__device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// ... and for this wave's loads into LDS, but for the last kLater of them. (The
// compiler knows nothing of those loads.)
template <int kLater>
__device__ __forceinline__ void arrival() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(kLater) : "memory");
}
// 4 elements of k of each lane's row, from the rows that its 16 lanes address.
__device__ __forceinline__ u32x2 read_across(int32_t at) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)(uint32_t)at));
}

// Reads one operand's fragments of a stage: kRows / 32 from the first-th 32 rows
// on.
template <bool kAcross, int kRows = 128>
struct Reader {
  int32_t at[kAcross ? kRows / 32 : 2];  // the lane's place in LDS by fragment, or by the half of k

  __device__ __forceinline__ void init(int32_t first) {
    const int lane = threadIdx.x & 63;
    if constexpr (kAcross) {
#pragma unroll
      for (int i = 0; i < kRows / 32; ++i)
        at[i] = ((lane >> 5) * 8 + (lane >> 2 & 3)) * 512 + (first + i) / 4 * 256 + (lane >> 4 & 1) * 128 +
                (((first + i) & 3) ^ (lane >> 2 & 3)) * 32 + (lane & 3) * 8;
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        at[h] = first * 2048 + (lane & 31) * 64 + (((lane >> 5) + 2 * h) ^ (lane >> 2 & 3)) * 16;
    }
  }
  // Rows 32 i.., k 16 h...
  __device__ __forceinline__ u32x4 read(int32_t from, int i, int h) const {
    if constexpr (kAcross) {
      const u32x2 a = read_across(from + at[i] + h * 8192), b = read_across(from + at[i] + h * 8192 + 2048);
      return u32x4{a.x, a.y, b.x, b.y};
    } else {
      return *(__attribute__((address_space(3))) const u32x4*)(uintptr_t)(uint32_t)(from + at[h] + i * 2048);
    }
  }
};

template <class T, bool kAcrossP, bool kAcrossQ>
struct Gemm {
  using Sums = Acc;
  Loader<kAcrossP> lp;
  Loader<kAcrossQ> lq;
  int32_t k;

  // A pair that ends inside k is taken first, the others in order. Without any
  // k there is one pair of zeros.
  __device__ __forceinline__ int32_t pairs() const { return max((k + kPairK - 1) / kPairK, 1); }
  __device__ __forceinline__ int32_t ragged() const { return pairs() - k / kPairK; }

  // Asks for the first two pairs of the tile at rows prow of P and qrow of Q.
  // The LDS up to kOwnAt has to be free.
  __device__ __forceinline__ void start(const Operand16& P, const Operand16& Q, const void* zeros, int32_t prow, int32_t qrow, int32_t lds) {
    k = uniform(min(P.k, Q.k));              // they differ by less than a vector at most
    lp.init(P, prow);
    lq.init(Q, qrow);
    const int32_t first = ragged() ? pairs() - 1 : 0, second = 1 - ragged();
    lp.issue_all(lds, first, zeros);
    lq.issue_all(lds + kOperandBytes, first, zeros);
    const auto bp = lp.buffer(second, (1 - pairs()) >> 31), bq = lq.buffer(second, (1 - pairs()) >> 31);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        lp.issue(bp, lds + (2 + h) * kStageBytes, h, j);
        lq.issue(bq, lds + (2 + h) * kStageBytes + kOperandBytes, h, j);
      }
  }

  // The products. On return every wave has read its last of the LDS, and no
  // load is under way.
  __device__ __forceinline__ void run(int32_t lds, Acc& acc) const {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc.a[i][j][r] = 0.f;
    Reader<kAcrossP> rp;
    Reader<kAcrossQ> rq;
    rp.init((threadIdx.x >> 7) * 4);
    rq.init((threadIdx.x >> 6 & 1) * 4);
    const int32_t n = uniform(pairs()), skip = uniform(ragged());

    // The r-th of a stage's 16 fragments: q's first, since every product of the first P fragment needs one.
    const auto read = [&](Fragments& f, int32_t from, int r) {
      if (r < 8)
        f.q[r] = rq.read(from + kOperandBytes, r >> 1, r & 1);
      else
        f.p[r - 8] = rp.read(from, (r - 8) >> 1, r & 1);
    };
    // A stage's products, with the reads of the next stage and half of the loads
    // of the pair after next.
    const auto stage = [&](const Fragments& f, Fragments& next, int32_t from, auto second, int32_t to0, int32_t to1, int32_t pair,
                           int32_t bytes) {
      const auto bp = lp.buffer(pair, bytes), bq = lq.buffer(pair, bytes);
#pragma unroll
      for (int m = 0; m < 32; ++m) {
        const int h = m >> 4, i = m >> 2 & 3, j = m & 3;
        mfma<T>(acc.a[i][j], f.p[2 * i + h], f.q[2 * j + h]);
        if (!(m & 1)) read(next, from, m >> 1);
        if ((m & 3) == 3) {
          const int l = (m >> 2) + (second ? 8 : 0), h2 = l & 1;      // both stages of each row together, P's and Q's in turn
          if (l & 2)
            lq.issue(bq, (h2 ? to1 : to0) + kOperandBytes, h2, l >> 2);
          else
            lp.issue(bp, h2 ? to1 : to0, h2, l >> 2);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    const auto place = [](int32_t p) { return p >= kPlaces ? p - kPlaces : p; };

    Fragments f0, f1;
    arrival<16>();                   // the first pair is here, the second under way
#pragma unroll
    for (int r = 0; r < 16; ++r) read(f0, lds, r);
    int32_t p0 = 0;                  // place of the pair's first stage
    for (int32_t u = 0; u < n; ++u) {
      const int32_t s0 = lds + p0 * kStageBytes, s1 = lds + place(p0 + 1) * kStageBytes, s4 = lds + place(p0 + 4) * kStageBytes;
      p0 = uniform(place(p0 + 2));
      barrier();                     // the pair's first stage is in everyone's registers
      const int32_t pair = uniform(u + 2 - skip), bytes = uniform((u + 2 - n) >> 31);
      stage(f0, f1, s1, std::false_type{}, s4, s0, pair, bytes);
      arrival<8>();                  // ... and its second; the next pair is here, half of the one after it under way
      // past the last pair this reads what the place holds, and nothing uses it
      stage(f1, f0, lds + p0 * kStageBytes, std::true_type{}, s4, s0, pair, bytes);
      settle();
    }
    arrival<0>();
  }
};

// The same product with few rows of Q (kJ times 32, contiguous in k): a tile is
// 256 x 32 kJ, 64 rows of P a wave. It is bound by reading P, so what counts is
// bytes under way: pairs of stages are loaded up to kDeep - 1 ahead, over 90 KiB
// a CU, and one barrier a pair suffices, behind which the next pair is here and
// the place of the present one free. A tile of 256 rows of Q would multiply
// mostly rows that do not exist, which takes longer than P takes to come from
// memory: 55 rows over 152064 x 8192 take 510 us where P is contiguous in k (4.9
// TB/s) and 410 where it is not (6.1), 600 with tiles of 256.
// Workgroups begin at different places of k: P's rows are a power of two apart
// as a rule, and the same place of k in all of them is in few of the memory's
// channels (3 rows over 152064 x 4096: 250 us, 314 if all begin at 0).
template <int kJ>
struct NarrowAcc {
  f32x16 a[2][kJ];            // as Acc, rows 64 wave + 32 i.. of P
};
template <int kJ>
__device__ __forceinline__ float sum_of(const NarrowAcc<kJ>& acc, int i, int j, int r) {
  float x;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(acc.a[i][j][r]));
  return x;
}

template <class T, bool kAcrossP, int kJ>
struct Narrow {
  using Sums = NarrowAcc<kJ>;
  static constexpr int kStage = kOperandBytes + 32 * kJ * kStageK * 2, kDeep = kGemmLds / (2 * kStage);
  static constexpr int kOfPair = 8 + kJ;       // loads of a wave
  static_assert(kJ % 2 == 0 && kDeep > 2 && (kDeep - 1) * 2 * kStage <= kOwnAt, "the results' LDS is left free");
  Loader<kAcrossP> lp;
  Loader<false, kJ / 2> lq;
  int32_t k, from;            // the whole pairs begin with this one and come round to it

  __device__ __forceinline__ int32_t pairs() const { return max((k + kPairK - 1) / kPairK, 1); }
  __device__ __forceinline__ int32_t ragged() const { return pairs() - k / kPairK; }

  // The u-th pair (u > 0; past the last: nothing) as buffers.
  __device__ __forceinline__ void pair_of(int32_t u, int32_t n, int32_t skip, u32x4& bp, u32x4& bq) const {
    const int32_t bytes = uniform((u - n) >> 31), at = u - skip + from, pair = uniform(at < n - skip ? at : at - (n - skip));
    bp = lp.buffer(pair, bytes), bq = lq.buffer(pair, bytes);
  }
  // The l-th of the kOfPair / 2 loads of its stage h, to the pair's place.
  __device__ __forceinline__ void ask(const u32x4& bp, const u32x4& bq, int32_t place, int h, int l) const {
    if (l < kJ / 2)
      lq.issue(bq, place + h * kStage + kOperandBytes, h, l);
    else
      lp.issue(bp, place + h * kStage, h, l - kJ / 2);
  }

  // As Gemm's. The whole pairs begin with the one that is `turn` % 256 of 256 parts on.
  __device__ __forceinline__ void start(const Operand16& P, const Operand16& Q, const void* zeros, int32_t prow, int32_t qrow,
                                        int32_t turn, int32_t lds) {
    k = uniform(min(P.k, Q.k));
    lp.init(P, prow);
    lq.init(Q, qrow);
    const int32_t n = uniform(pairs()), skip = uniform(ragged());
    from = uniform((int32_t)((int64_t)(turn & 255) * (n - skip) >> 8));
    const int32_t first = skip ? n - 1 : from;
    lp.issue_all(lds, first, zeros, kStage);
    lq.issue_all(lds + kOperandBytes, first, zeros, kStage);
#pragma unroll
    for (int u = 1; u < kDeep - 1; ++u) {
      u32x4 bp, bq;
      pair_of(u, n, skip, bp, bq);
#pragma unroll
      for (int l = 0; l < kOfPair; ++l) ask(bp, bq, lds + u * (2 * kStage), l * 2 / kOfPair, l % (kOfPair / 2));
    }
  }

  __device__ __forceinline__ void run(int32_t lds, Sums& acc) const {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < kJ; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc.a[i][j][r] = 0.f;
    Reader<kAcrossP, 64> rp;
    Reader<false, 32 * kJ> rq;
    rp.init((threadIdx.x >> 6) * 2);
    rq.init(0);
    const int32_t n = uniform(pairs()), skip = uniform(ragged());
    constexpr int kReads = 4 + 2 * kJ, kProducts = 4 * kJ;
    struct Part {
      u32x4 p[4], q[2 * kJ];
    };
    const auto read = [&](Part& f, int32_t from_at, int r) {
      const int h = r * 2 / kReads, e = r % (kReads / 2);
      if (e < 2)
        f.p[2 * e + h] = rp.read(from_at, e, h);
      else
        f.q[2 * (e - 2) + h] = rq.read(from_at + kOperandBytes, e - 2, h);
    };
    // A stage's products, with the reads of the next stage and half of a later pair's loads between them.
    const auto stage = [&](const Part& f, Part& next, int32_t from_at, const u32x4& bp, const u32x4& bq, int32_t to, auto half) {
#pragma unroll
      for (int m = 0; m < kProducts; ++m) {
        const int h = m / (2 * kJ), j = m / 2 % kJ, i = m % 2;
        mfma<T>(acc.a[i][j], f.p[2 * i + h], f.q[2 * j + h]);
#pragma unroll
        for (int r = m * kReads / kProducts; r < (m + 1) * kReads / kProducts; ++r) read(next, from_at, r);
#pragma unroll
        for (int l = m * kOfPair / 2 / kProducts; l < (m + 1) * kOfPair / 2 / kProducts; ++l) ask(bp, bq, to, half, l);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    const auto place = [&](int32_t p) { return lds + uniform(p >= kDeep ? p - kDeep : p) * (2 * kStage); };

    Part f0, f1;
    u32x4 bp, bq;
    arrival<kOfPair * (kDeep - 2)>();              // the first pair is here, and all of the LDS free
    pair_of(kDeep - 1, n, skip, bp, bq);
#pragma unroll
    for (int r = 0; r < kReads; ++r) read(f0, lds, r);
#pragma unroll
    for (int l = 0; l < kOfPair / 2; ++l) ask(bp, bq, place(kDeep - 1), 0, l);
    int32_t at = 0;                                // the pair's place
    for (int32_t u = 0; u < n; ++u) {
      stage(f0, f1, place(at) + kStage, bp, bq, place(at + kDeep - 1), std::integral_constant<int, 1>{});
      arrival<kOfPair * (kDeep - 2)>();            // the pair is in everyone's registers, the next one here
      pair_of(u + kDeep, n, skip, bp, bq);
      stage(f1, f0, place(at + 1), bp, bq, place(at), std::integral_constant<int, 0>{});
      settle();
      at = uniform(at + 1 == kDeep ? 0 : at + 1);
    }
    arrival<0>();
  }
};

// Tile number `id` among pt x qt tiles. The 256 that run at once are 16 tiles of
// P by 16 of Q (where there are as many), so that each row comes from HBM once
// and then from the memory-side cache; and workgroups go round the 8 XCDs, each
// with an L2 of its own, so the 32 of an XCD are 8 by 4 tiles of those, which
// share 12 tiles' rows. Strips of 16 tiles of P are walked down Q.
__device__ __forceinline__ void tile_of(int32_t id, int32_t pt, int32_t qt, int32_t* p, int32_t* q) {
  const int32_t round = id & ~255, here = min(pt * qt - round, 256), xcd = id & 7;
  const int32_t at = round + xcd * (here >> 3) + min(xcd, here & 7) + ((id & 255) >> 3);
  const int32_t s = at / (16 * qt), in = at - s * 16 * qt, width = min(pt - s * 16, 16);
  const int32_t g = in / (4 * width), rows = min(qt - 4 * g, 4), in4 = in - g * 4 * width;
  const int32_t left = min(width, 8), right = in4 >= left * rows;
  const int32_t in8 = in4 - (right ? left * rows : 0), w8 = right ? width - left : left;
  *q = (4 * g + in8 / w8) * kTile;
  *p = (s * 16 + right * left + in8 % w8) * kTile;
}

// A wave's results in 16 bits for one 32 rows of Q, j: w[i][r] holds those of
// a[i][j][2 r] and [2 r + 1].
struct Packed {
  uint32_t w[4][8];
};
template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  Pack<T, 2> o;
  o.set(0, a);
  o.set(1, b);
  return __builtin_bit_cast(uint32_t, o);
}

// Orders a wave's own LDS accesses, which run in the order they are issued.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Keeps what is computed from x inside the loop over tiles: hoisted out of it,
// the addresses of a tile's rows would not fit the registers.
__device__ __forceinline__ int64_t here(int64_t x) {
  asm volatile("" : "+s"(x));
  return x;
}

// Results leave as rows through the wave's own LDS, 8 KiB at a time.

// As rows of Q: sink(q, p, vector) with 8 values of 16 bits at row q, from
// element p on, both within the tile; 16 lanes hold a row's 256 bytes.
template <class Sink>
__device__ __forceinline__ void rows_out(const Packed& x, int j, char* own, Sink sink) {
  const int lane = threadIdx.x & 63;
  // row l % 32; vectors are stored at their index exclusive-or the row modulo 16
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const u32x2 v = {x.w[i][2 * r], x.w[i][2 * r + 1]};
      *(u32x2*)(own + lane_q() * 256 + (((4 * i + r) ^ (lane_q() & 15)) << 4) + lane_p() * 2) = v;
    }
  wave_order();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int q = k * 4 + (lane >> 4), v = lane & 15;
    sink(wave_q() + j * 32 + q, wave_p() + v * 8, *(const u32x4*)(own + q * 256 + ((v ^ (q & 15)) << 4)));
    if (k & 1) __builtin_amdgcn_sched_barrier(0);
  }
  wave_order();
}

// The sums themselves times `scale`, all 128 rows, 32 rows of Q (the j-th) after
// the other: sink(j, q, p, vector) with 4 values of 32 bits at a time.
template <class Sink>
__device__ __forceinline__ void rows_out(const Acc& acc, float scale, char* own, Sink sink) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = sum_of(acc, 2 * half + i, j, 4 * r + e) * scale;
          *(f32x4*)(own + lane_q() * 256 + (((8 * i + 2 * r + (lane_p() >> 2)) ^ (lane_q() & 15)) << 4)) = v;
        }
      wave_order();
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int q = k * 4 + (lane >> 4), v = lane & 15;
        sink(j, wave_q() + j * 32 + q, wave_p() + half * 64 + v * 4, *(const f32x4*)(own + q * 256 + ((v ^ (q & 15)) << 4)));
        if (k & 1) __builtin_amdgcn_sched_barrier(0);
      }
      wave_order();
    }
}

// The same with few rows of Q: sink(q, p, vector), p from the wave's first row
// of P on. 8 lanes hold a row's 128 bytes.
template <class Sink>
__device__ __forceinline__ void narrow_rows_out(const uint32_t (&w)[2][8], int j, char* own, Sink sink) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const u32x2 v = {w[i][2 * r], w[i][2 * r + 1]};
      *(u32x2*)(own + lane_q() * 128 + (((4 * i + r) ^ (lane_q() & 7)) << 4) + lane_p() * 2) = v;
    }
  wave_order();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int q = k * 8 + (lane >> 3), v = lane & 7;
    sink(j * 32 + q, v * 8, *(const u32x4*)(own + q * 128 + ((v ^ (q & 7)) << 4)));
  }
  wave_order();
}
template <int kJ, class Sink>
__device__ __forceinline__ void narrow_rows_out(const NarrowAcc<kJ>& acc, char* own, Sink sink) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < kJ; ++j) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = sum_of(acc, i, j, 4 * r + e);
        *(f32x4*)(own + lane_q() * 256 + (((8 * i + 2 * r + (lane_p() >> 2)) ^ (lane_q() & 15)) << 4)) = v;
      }
    wave_order();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int q = k * 4 + (lane >> 4), v = lane & 15;
      sink(j * 32 + q, v * 4, *(const f32x4*)(own + q * 256 + ((v ^ (q & 15)) << 4)));
    }
    wave_order();
  }
}

}  // namespace fp
