// Log probabilities of given tokens with entropy and top alternatives, and their gradient.
// Part of the translation unit adagc_ops.cu (included there; not compiled on its own).
//
// Forward, one pass over a row.  A thread keeps, against a reference m of its own,
//     s = sum e_j,   t = sum e_j d_j,   d_j = (z_j - m) log2(e),  e_j = 2^d_j
// and when the reference moves from m to M, delta = (m - M) log2(e): s <- s 2^delta, t <- (t + delta s) 2^delta.
// Two such parts join the same way, so threads, warps, and blocks of a cluster that share one row are joined in a fixed
// tree.  Then lse = m + ln(s) and entropy = ln 2 (log2 s - t / s).
// 8192 x 128256 bf16 takes 297 to 321 us in short runs (6.55 TB/s and more, the rate of a plain copy; XU pipe 75 % busy with one
// exponential per entry) and 345 to 367 us back to back, under the power limit (SM clock 1.52 GHz).
// The kernel is bound by HBM only if it spends few instructions (and little power) per entry, so the reference is not the
// running maximum: it is the largest entry of the thread's first batch, and moves only when a batch's sum passes 2^10.
// d_j is one fused multiply-add, z_j log2(e) - c with c = m log2(e) rounded (c is the reference then, nothing is lost), and
// masked entries are not looked for: they make the batch's t a NaN (0 * -inf), and a batch whose sums are out of range is
// taken again, entry by entry, with the reference raised to its maximum and d_j clamped.  A NaN logit reaches s that way.  The price
// of a mask scattered over the row, when nearly every batch is taken again: 8192 x 128256 bf16 with a tenth of the entries at -inf 606
// against 297 us in short runs, 4096 x 128256 fp32 357 against 294.
// References of 2^14 and more in magnitude take that route always, with d_j from the difference z_j - m, so rows of huge
// magnitudes (all entries at the type's lowest value) neither overflow nor lose their differences.
//
// Top k.  Every thread also keeps its largest logit, the batch it lies in, and the largest of its other batches.  The k-th
// largest of the threads' values is a lower bound of the k-th largest logit, and every candidate lies with a thread whose
// value reaches it, as a rule in that one batch: only those batches are read again, usually a few more than k entries pass,
// and they are ranked by counting, on unique keys (value, then lowest index).  Rows built so that more entries pass than
// the buffer holds (all entries tie) fall back to k rounds of a maximum over the same vectors.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <cfloat>
#include <climits>

namespace {

namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kExpFloor = -200.0f;  // 2^-200 is 0 in fp32
constexpr int kTopBuffer = 288;       // candidates ranked by counting; the vectors of 31 threads and the unaligned ends fit
constexpr int kMaxCluster = 8;        // blocks that share one row at most (the portable cluster size)
constexpr int kRowBlock = 128;                                  // threads of a block: one team, or four of a warp each
constexpr int kRowBatch = 4;                                    // vectors of 16 bytes that a thread takes at a time
constexpr int kRowAhead = 2, kRowSlots = kRowAhead + 1;         // batches in flight per thread; the slots they land in
template <int kT, bool kTop>
constexpr int kRowResident = kTop ? (kT == 32 ? 6 : 7) : 8;     // blocks per SM that shared memory has room for

__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xff800000u); }
__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7fc00000u); }
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float exp2_full(float x) {  // with subnormal results
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two fp32 values in one 64-bit register pair: the packed arithmetic of sm_100 takes them in one instruction.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// Read once: no room in L1.  Not through the read-only path: a kernel may be started while the one that writes its inputs still runs
// (griddep_wait comes before the first load), so they are not read-only for as long as it lives.
__device__ __forceinline__ uint4 ld_once(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

__device__ __forceinline__ void copy_async(uint4* dst, const uint4* src) {  // 16 bytes, past L1
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void copy_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory");
}

// Below this a logit's gradient is 0 where |lse| < 1024 (kExtremeLse): p = 2^d with d < -4400.  The gradient's kernel raises smaller
// logits (masked ones) to it, so that d stays small enough for B d to be finite: A + B d with p = 0 has to give 0.
constexpr float kLowestLogit = -4096.0f;

template <bool kBF16>
struct Elem;  // 16-byte vectors of the logits' type
template <>
struct Elem<true> {
  using Type = __nv_bfloat16;
  static constexpr int kBytes = 2, kVec = 8;
  static constexpr uint32_t kMasked = 0xff80ff80u;  // a pair of -inf
  static __device__ __forceinline__ float load(const void* p, int64_t i) { return __bfloat162float(static_cast<const Type*>(p)[i]); }
  static __device__ __forceinline__ void store(void* p, int64_t i, float x) { static_cast<Type*>(p)[i] = __float2bfloat16_rn(x); }
  static __device__ __forceinline__ void expand(const uint4& w, float (&z)[kVec]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) z[2 * i] = bf16_lo(u[i]), z[2 * i + 1] = bf16_hi(u[i]);
  }
  static __device__ __forceinline__ uint4 collect(const float (&z)[kVec]) {
    return make_uint4(pack_bf16_cvt(z[0], z[1]), pack_bf16_cvt(z[2], z[3]), pack_bf16_cvt(z[4], z[5]), pack_bf16_cvt(z[6], z[7]));
  }
  // largest value of the first n of kN vectors; NaN entries are passed over
  template <int kN>
  static __device__ __forceinline__ float largest(const uint4 (&w)[kN], int n) {
    __nv_bfloat162 m = pair(kMasked);
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (i < n) m = __hmax2(__hmax2(m, __hmax2(pair(w[i].x), pair(w[i].y))), __hmax2(pair(w[i].z), pair(w[i].w)));
    return fmaxf(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ uint4 clamped(uint4 w) {  // at least kLowestLogit; a NaN stays
    uint32_t* u = &w.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(u[i]) : "r"(0xc580c580u));
    return w;
  }
  static __device__ __forceinline__ __nv_bfloat162 pair(uint32_t u) { return *reinterpret_cast<__nv_bfloat162*>(&u); }
};
template <>
struct Elem<false> {
  using Type = float;
  static constexpr int kBytes = 4, kVec = 4;
  static __device__ __forceinline__ float load(const void* p, int64_t i) { return static_cast<const float*>(p)[i]; }
  static __device__ __forceinline__ void store(void* p, int64_t i, float x) { static_cast<float*>(p)[i] = x; }
  static __device__ __forceinline__ void expand(const uint4& w, float (&z)[kVec]) {
    z[0] = __uint_as_float(w.x), z[1] = __uint_as_float(w.y), z[2] = __uint_as_float(w.z), z[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ uint4 collect(const float (&z)[kVec]) {
    return make_uint4(__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3]));
  }
  static __device__ __forceinline__ uint4 clamped(uint4 w) {
    uint32_t* u = &w.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+r"(u[i]) : "r"(0xc5800000u));
    return w;
  }
  template <int kN>
  static __device__ __forceinline__ float largest(const uint4 (&w)[kN], int n) {
    float m = neg_inf();
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (i < n)
        m = fmaxf(fmaxf(m, fmaxf(__uint_as_float(w[i].x), __uint_as_float(w[i].y))), fmaxf(__uint_as_float(w[i].z), __uint_as_float(w[i].w)));
    return m;
  }
};

// One part of a row's softmax: the reference (-inf: nothing but masked entries), sum of e, sum of e d.
struct SoftmaxPart {
  float m, s, t;
};
__device__ __forceinline__ SoftmaxPart join(const SoftmaxPart& a, const SoftmaxPart& b) {
  SoftmaxPart r;
  r.m = fmaxf(a.m, b.m);
  if (r.m == neg_inf()) return {r.m, a.s + b.s, a.t + b.t};  // nothing but masked entries (or NaN sums) on either side
  const float da = a.m == r.m ? 0.0f : fmaxf((a.m - r.m) * kLog2e, kExpFloor), db = b.m == r.m ? 0.0f : fmaxf((b.m - r.m) * kLog2e, kExpFloor);
  const float fa = exp2_approx(da), fb = exp2_approx(db);
  r.s = a.s * fa + b.s * fb;
  r.t = (a.t + da * a.s) * fa + (b.t + db * b.s) * fb;
  return r;
}

// The running part of one thread.
struct RowState {
  static constexpr float kFastReference = 16384.0f;  // below this, c is within 2^-10 of m log2(e)
  static constexpr float kBatchLimit = 1024.0f;
  float ref = neg_inf(), c = 0.0f;  // -inf: nothing but masked entries so far
  float s = 0.0f, t = 0.0f;
  __device__ __forceinline__ bool fast() const { return fabsf(ref) < kFastReference; }
  __device__ __forceinline__ void raise(float to) {
    const bool to_fast = fabsf(to) < kFastReference;
    const float to_c = to * kLog2e;
    if (ref != neg_inf()) {
      float delta = fast() ? (to_fast ? c - to_c : fmaf(-to, kLog2e, c)) : (to_fast ? fmaf(ref, kLog2e, -to_c) : (ref - to) * kLog2e);
      delta = fmaxf(delta, kExpFloor);
      const float f = exp2_approx(delta);
      t = fmaf(delta, s, t) * f;
      s *= f;
    }
    ref = to;
    c = to_c;
  }
  __device__ __forceinline__ void add(float z) {  // one entry, whatever it holds
    if (z > ref) raise(z);
    const float d = fast() ? fmaf(z, kLog2e, -c) : (z - (ref == neg_inf() ? 0.0f : ref)) * kLog2e;
    const float e = exp2_approx(d);
    s += e;
    t = fmaf(e, fmaxf(d, kExpFloor), t);
  }
  // Sums of one batch against the present reference; kAll: all kN vectors are there, otherwise the first n.
  template <bool kBF16, bool kAll, int kN>
  __device__ __forceinline__ float2 sums(const uint4 (&w)[kN], int n) {
    using E = Elem<kBF16>;
    const float nc = fast() ? -c : quiet_nan();
    float s0 = 0.0f, s1 = 0.0f, t0 = 0.0f, t1 = 0.0f;
#pragma unroll
    for (int u = 0; u < kN; ++u) {
      if (!kAll && u >= n) break;
      float z[E::kVec];
      E::expand(w[u], z);
#pragma unroll
      for (int j = 0; j < E::kVec; j += 2) {
        const float d0 = fmaf(z[j], kLog2e, nc), d1 = fmaf(z[j + 1], kLog2e, nc), e0 = exp2_approx(d0), e1 = exp2_approx(d1);
        s0 += e0;
        s1 += e1;
        t0 = fmaf(e0, d0, t0);
        t1 = fmaf(e1, d1, t1);
      }
    }
    return make_float2(s0 + s1, t0 + t1);
  }
  // One batch: w holds its first n vectors; again(u) reads vector u once more.
  template <bool kBF16, int kN, typename Again>
  __device__ __forceinline__ void add(const uint4 (&w)[kN], int n, Again again) {
    using E = Elem<kBF16>;
    if (ref == neg_inf()) {
      const float top = E::largest(w, n);
      if (top > ref) raise(top);
    }
    const float2 x = n >= kN ? sums<kBF16, true>(w, n) : sums<kBF16, false>(w, n);
    if (x.x < kBatchLimit && fabsf(x.y) < 1e30f) {  // false for a NaN
      s += x.x;
      t += x.y;
      return;
    }
    float top = neg_inf();
#pragma unroll 1
    for (int u = 0; u < min(n, kN); ++u) {
      const uint4 v[1] = {again(u)};
      top = fmaxf(top, E::largest(v, 1));
    }
    if (top > ref) raise(top);
    const bool near = fast();
    const float base = near || ref == neg_inf() ? 0.0f : ref, shift = near ? -c : 0.0f;
#pragma unroll 1
    for (int u = 0; u < min(n, kN); ++u) {
      float z[E::kVec];
      E::expand(again(u), z);
#pragma unroll
      for (int j = 0; j < E::kVec; ++j) {
        const float d = fmaf(z[j] - base, kLog2e, shift), e = exp2_approx(d);
        s += e;
        t = fmaf(e, fmaxf(d, kExpFloor), t);
      }
    }
  }
  __device__ __forceinline__ SoftmaxPart part() const {  // against m itself instead of c
    if (!fast()) return {ref, s, t};
    const float delta = fmaf(-ref, kLog2e, c), f = exp2_approx(delta);
    return {ref, s * f, fmaf(delta, s, t) * f};
  }
};

// A row of logits as this block sees it: `head` entries up to the first 16-byte boundary and `tail` after the last
// whole vector (both handled by the first block of a cluster), and the vectors [begin, end) of the middle.
template <bool kBF16>
struct RowSlice {
  const void* row;
  const uint4* body;  // vector 0: the first 16-byte boundary
  int index0;         // entry number of its first element
  int head, tail, tail_at, begin, end;
  __device__ __forceinline__ RowSlice(const void* logits, int64_t r, int64_t ld, int vocab, int part, int parts) {
    using E = Elem<kBF16>;
    const char* p = static_cast<const char*>(logits) + r * ld * E::kBytes;
    row = p;
    index0 = min(vocab, static_cast<int>((16u - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / E::kBytes);
    body = reinterpret_cast<const uint4*>(p + index0 * E::kBytes);
    const int n = (vocab - index0) / E::kVec, per = (n + parts - 1) / parts;
    begin = min(n, part * per);
    end = min(n, begin + per);
    tail_at = index0 + n * E::kVec;
    head = part == 0 ? index0 : 0;
    tail = part == 0 ? vocab - tail_at : 0;
  }
};

// A float as an integer of the same order, and back.
__device__ __forceinline__ int ordered(float x) {
  const int i = __float_as_int(x);
  return i < 0 ? i ^ 0x7fffffff : i;
}
__device__ __forceinline__ float from_ordered(int i) { return __int_as_float(i < 0 ? i ^ 0x7fffffff : i); }

// (value, lowest index first) as one ordered 64-bit key; 0 for a masked entry
__device__ __forceinline__ uint64_t top_key(float z, int index) {
  if (z == neg_inf()) return 0;
  uint32_t u = __float_as_uint(z + 0.0f);  // -0 and 0 tie
  u = (u & 0x80000000u) ? ~u : u | 0x80000000u;
  return (static_cast<uint64_t>(u) << 32) | static_cast<uint32_t>(~index);
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t u = static_cast<uint32_t>(k >> 32);
  return __uint_as_float((u & 0x80000000u) ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_index(uint64_t k) { return static_cast<int>(~static_cast<uint32_t>(k)); }

struct LogprobArgs {
  const void* logits;
  const int64_t* targets;
  float *logprob, *lse, *entropy, *top_logprob;
  int32_t* top_index;
  int64_t rows, ld;
  int vocab, top_k;
};

// The threads that share a row inside a block: the whole block, or one warp of it.
template <int kT>
__device__ __forceinline__ void team_sync() {
  if constexpr (kT == 32) __syncwarp();
  else __syncthreads();
}

template <int kT>
struct TopScratch {
  alignas(16) float largest[kT];  // of each thread's vectors
  uint64_t buffer[kTopBuffer];
  uint64_t best[kT / 32];
  float least;   // lower bound of the k-th largest logit
  int count;     // candidates found
};

// What a thread remembers of its vectors for the top-k search: the largest value, the batch that first had it, and the
// largest value of its other batches.
struct RowPeaks {
  float first = neg_inf(), second = neg_inf();
  int at = 0;
  __device__ __forceinline__ void add(float top, int batch) {
    second = fmaxf(second, fminf(first, top));
    if (top > first) first = top, at = batch;
  }
};

// Calls fn(value, index) for every entry of the block's slice that is at least `least`.
template <bool kBF16, int kT, typename F>
__device__ __forceinline__ void each_candidate(const RowSlice<kBF16>& sl, int tid, const RowPeaks& pk, float least, F fn) {
  using E = Elem<kBF16>;
  const auto vector = [&](const uint4& w, int v) {
    const uint4 one[1] = {w};
    if (!(E::largest(one, 1) >= least)) return;
    float z[E::kVec];
    E::expand(w, z);
#pragma unroll
    for (int j = 0; j < E::kVec; ++j)
      if (z[j] >= least) fn(z[j], sl.index0 + v * E::kVec + j);
  };
  // as a rule the candidates of a thread lie in one batch: it reads that again itself
  if (pk.first >= least && pk.second < least) {
    uint4 w[kRowBatch];
#pragma unroll
    for (int u = 0; u < kRowBatch; ++u)
      if (pk.at + u * kT < sl.end) w[u] = ld_once(sl.body + pk.at + u * kT);
#pragma unroll
    for (int u = 0; u < kRowBatch; ++u)
      if (pk.at + u * kT < sl.end) vector(w[u], pk.at + u * kT);
  }
  // the others' vectors are gone through by their warps
  for (uint32_t deep = __ballot_sync(0xffffffffu, pk.second >= least); deep != 0; deep &= deep - 1) {
    const int owner = (tid & ~31) + __ffs(deep) - 1;
#pragma unroll 4
    for (int v = sl.begin + owner + (tid & 31) * kT; v < sl.end; v += 32 * kT) vector(ld_once(sl.body + v), v);
  }
  if (tid < sl.head + sl.tail) {
    const int j = tid < sl.head ? tid : sl.tail_at + tid - sl.head;
    const float z = E::load(sl.row, j);
    if (z >= least) fn(z, j);
  }
}

// The k largest keys of the slice, sorted, into list[0 .. k) (0 where there are fewer).  Every thread of the team takes part;
// the list is complete for the team's first warp.
template <bool kBF16, int kT>
__device__ __forceinline__ void team_top_k(const RowSlice<kBF16>& sl, int tid, const RowPeaks& pk, int k, TopScratch<kT>& sc, uint64_t* list) {
  sc.largest[tid] = pk.first;
  team_sync<kT>();
  if (tid < 32) {  // the k-th largest of the threads' values: take the largest away, with its ties, until k are gone
    constexpr int kEach = kT / 32;
    int v[kEach], low = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) v[i] = ordered(sc.largest[tid * kEach + i]);
    for (int gone = 0; gone < k;) {
      int top = v[0], ties = 0;
#pragma unroll
      for (int i = 1; i < kEach; ++i) top = max(top, v[i]);
      low = top = __reduce_max_sync(0xffffffffu, top);
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (v[i] == top) v[i] = INT_MIN, ++ties;
      if (top == INT_MIN) break;
      gone += __reduce_add_sync(0xffffffffu, ties);
    }
    if (tid == 0) sc.least = low == INT_MIN ? neg_inf() : from_ordered(low);
  }
  team_sync<kT>();
  const float least = fmaxf(sc.least, -FLT_MAX);  // masked entries are no candidates
  each_candidate<kBF16, kT>(sl, tid, pk, least, [&](float z, int index) {
    const int at = atomicAdd(&sc.count, 1);  // in any order: the buffer is ranked below
    if (at < kTopBuffer) sc.buffer[at] = top_key(z, index);
  });
  team_sync<kT>();
  const int n = sc.count;
  if (n <= kTopBuffer) {
    // few enough for one warp as a rule
    const int team = n <= 128 ? 32 : kT;
    if (tid < team) {
      for (int i = tid; i < k; i += team)
        if (i >= n) list[i] = 0;
      for (int i = tid; i < n; i += team) {
        const uint64_t key = sc.buffer[i];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < n; ++j) rank += sc.buffer[j] > key;
        if (rank < k) list[rank] = key;
      }
    }
    if (n > 128) team_sync<kT>();
    else __syncwarp();
    return;
  }
  uint64_t below = ~0ull;
  for (int round = 0; round < k; ++round) {
    uint64_t best = 0;
    each_candidate<kBF16, kT>(sl, tid, pk, least, [&](float z, int index) {
      const uint64_t key = top_key(z, index);
      if (key < below) best = max(best, key);
    });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = max(best, static_cast<uint64_t>(__shfl_xor_sync(0xffffffffu, static_cast<unsigned long long>(best), o)));
    if ((tid & 31) == 0) sc.best[tid >> 5] = best;
    team_sync<kT>();
    best = 0;
    for (int w = 0; w < kT / 32; ++w) best = max(best, sc.best[w]);
    if (tid == 0) list[round] = best;
    below = best;
    team_sync<kT>();
  }
}

__device__ __forceinline__ SoftmaxPart warp_join(SoftmaxPart p, int from) {  // lane 0 holds the join of `from` * 2 lanes
#pragma unroll
  for (int o = from; o > 0; o >>= 1) {
    SoftmaxPart q;
    q.m = __shfl_down_sync(0xffffffffu, p.m, o);
    q.s = __shfl_down_sync(0xffffffffu, p.s, o);
    q.t = __shfl_down_sync(0xffffffffu, p.t, o);
    p = join(p, q);
  }
  return p;
}

struct RowTarget {
  int64_t index;
  float logit;
};

// What a row's joined part says, by one thread.  Returns (reference, ln s): ln p = (z - reference) - ln s, where z - lse
// would lose ln s in rows of huge magnitudes.
__device__ __forceinline__ float2 write_row(const LogprobArgs& a, int64_t r, const SoftmaxPart& p, const RowTarget& t) {
  // p.m is a reference near the maximum and p.s at least about 1; the logarithm is taken in double, once per row
  const bool empty = p.m == neg_inf() && p.s == 0.0f, bad = p.s != p.s;
  const double ln_s = empty ? 0.0 : log(static_cast<double>(p.s));
  a.lse[r] = bad ? quiet_nan() : empty ? neg_inf() : static_cast<float>(static_cast<double>(p.m) + ln_s);
  if (a.entropy) a.entropy[r] = empty ? 0.0f : static_cast<float>(ln_s - static_cast<double>(p.t) / p.s * 0.69314718055994530942);
  if (a.targets) {
    float lp = 0.0f;
    if (t.index >= a.vocab) lp = quiet_nan();
    else if (t.index >= 0) lp = empty ? neg_inf() : bad ? quiet_nan() : static_cast<float>(static_cast<double>(t.logit) - static_cast<double>(p.m) - ln_s);
    a.logprob[r] = lp;
  }
  return make_float2(p.m, static_cast<float>(ln_s));
}

// The row's list of alternatives from sorted keys, by one warp.
__device__ __forceinline__ void write_top(const LogprobArgs& a, int64_t r, const uint64_t* keys, float2 ref_ln_s) {
  const bool bad = ref_ln_s.y != ref_ln_s.y;  // a NaN or +inf in the row
  for (int i = threadIdx.x & 31; i < a.top_k; i += 32) {
    const uint64_t key = keys[i];
    a.top_logprob[r * a.top_k + i] = bad ? quiet_nan() : key == 0 ? neg_inf() : (key_value(key) - ref_ln_s.x) - ref_ln_s.y;
    a.top_index[r * a.top_k + i] = bad || key == 0 ? -1 : key_index(key);
  }
}

// A team of kT threads takes one row, or shares it with the other blocks of a cluster.  Each thread copies its own vectors,
// kRowAhead batches ahead of the arithmetic, into slots that no other thread touches.  One row per team, with as many
// blocks as that takes: resident blocks that went from row to row, copying across the rows' ends, were slower
// (8192 x 128256 bf16 345 against 321 us in short runs, 5000 x 32000 68 against 63 us).
template <bool kBF16, int kT, bool kTop>
__global__ void __launch_bounds__(kRowBlock, kRowResident<kT, kTop>)
adagc_token_logprobs_kernel(LogprobArgs a) {
  using E = Elem<kBF16>;
  constexpr int kTeams = kRowBlock / kT, kWarps = kT / 32;
  __shared__ uint4 ring[kRowSlots][kRowBatch][kRowBlock];
  __shared__ SoftmaxPart warp_part[kWarps];
  __shared__ SoftmaxPart block_part[kMaxCluster];
  __shared__ typename std::conditional<kTop, TopScratch<kT>, int>::type scratch[kTeams];
  __shared__ uint64_t lists[kTop ? kTeams : 1][kTop ? ADAGC_MAX_TOP_K : 1];
  __shared__ uint64_t gathered[kTop ? kMaxCluster * ADAGC_MAX_TOP_K : 1];
  static_assert(kRowResident<kT, kTop> * (1024 + sizeof(ring) + (kTop ? kTeams * (sizeof(TopScratch<kT>) + sizeof(lists[0])) + sizeof(gathered) : 16) + 256) <= 228 * 1024, "blocks per SM");
  griddep_wait();
  griddep_launch_dependents();
  cg::cluster_group cluster = cg::this_cluster();
  const int parts = kT == 32 ? 1 : static_cast<int>(cluster.num_blocks()), part = kT == 32 ? 0 : static_cast<int>(cluster.block_rank());
  const int team = kT == 32 ? threadIdx.x >> 5 : 0, tid = threadIdx.x - team * kT;
  const int64_t r = kT == 32 ? static_cast<int64_t>(blockIdx.x) * kTeams + team : blockIdx.x / parts;
  if (parts > 1) cluster.barrier_arrive();  // waited for before the first access to another block's shared memory
  if (r >= a.rows) return;                  // (whole warps of the one-warp form only)
  const RowSlice<kBF16> sl(a.logits, r, a.ld, a.vocab, part, parts);

  int ahead = sl.begin + tid;  // the first vector of the next batch to be copied
  const auto prefetch = [&](int slot) {
    const uint4* src = sl.body + ahead;
#pragma unroll
    for (int u = 0; u < kRowBatch; ++u)
      if (ahead + u * kT < sl.end) copy_async(&ring[slot][u][threadIdx.x], src + u * kT);
    copy_async_commit();
    ahead += kRowBatch * kT;
  };
#pragma unroll
  for (int i = 0; i < kRowAhead; ++i) prefetch(i);
  if constexpr (kTop)
    if (tid == 0) scratch[team].count = 0;  // (ordered by the search's barriers)
  RowTarget target{-1, 0.0f};
  if (tid == 0 && part == 0 && a.targets) {  // fetched first: two dependent loads that nothing at the end waits for
    target.index = a.targets[r];
    if (target.index >= 0 && target.index < a.vocab) target.logit = E::load(sl.row, target.index);
  }
  float end_logit = 0.0f;
  if (tid < sl.head + sl.tail) end_logit = E::load(sl.row, tid < sl.head ? tid : sl.tail_at + tid - sl.head);

  RowState st;
  RowPeaks peaks;
  int slot = 0;
  for (int at = sl.begin + tid; at < sl.end; at += kRowBatch * kT) {
    copy_async_wait<kRowAhead - 1>();
    uint4 w[kRowBatch];
#pragma unroll
    for (int u = 0; u < kRowBatch; ++u) w[u] = ring[slot][u][threadIdx.x];  // (stale beyond the slice's end, and not used)
    prefetch(slot == 0 ? kRowSlots - 1 : slot - 1);  // into the slot of the batch before
    const int n = (sl.end - at + kT - 1) / kT;
    if constexpr (kTop) peaks.add(E::largest(w, n), at);
    st.template add<kBF16>(w, n, [&](int u) { return ring[slot][u][threadIdx.x]; });
    slot = slot == kRowSlots - 1 ? 0 : slot + 1;
  }
  if (tid < sl.head + sl.tail) st.add(end_logit);

  SoftmaxPart p = warp_join(st.part(), 16);
  if constexpr (kT > 32) {
    if ((tid & 31) == 0) warp_part[tid >> 5] = p;
    if constexpr (!kTop) __syncthreads();  // (the top-k search has barriers of its own)
  }
  if constexpr (kTop) team_top_k<kBF16, kT>(sl, tid, peaks, a.top_k, scratch[team], lists[team]);
  if (parts > 1) cluster.barrier_wait();
  if (tid < 32) {
    if constexpr (kT > 32) p = warp_join(warp_part[tid % kWarps], kWarps / 2);
    if (parts > 1) {
      if (tid == 0) cluster.map_shared_rank(block_part, 0)[part] = p;
      if constexpr (kTop)
        for (int i = tid; i < a.top_k; i += 32) cluster.map_shared_rank(gathered, 0)[part * a.top_k + i] = lists[0][i];
    }
  }
  if (parts > 1) {  // the first block joins the others' parts
    cluster.sync();
    if (part != 0) return;
    if constexpr (kTop) {
      const int n = parts * a.top_k;
      if (tid < a.top_k) lists[0][tid] = 0;
      __syncthreads();
      for (int i = tid; i < n; i += kT) {
        const uint64_t key = gathered[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += gathered[j] > key;
        if (key != 0 && rank < a.top_k) lists[0][rank] = key;
      }
      __syncthreads();
    }
    p = block_part[0];
    for (int b = 1; b < parts; ++b) p = join(p, block_part[b]);
  }
  if (tid >= 32) return;
  float2 ref = make_float2(0.0f, 0.0f);
  if (tid == 0) ref = write_row(a, r, p, target);
  if constexpr (kTop) {
    ref.x = __shfl_sync(0xffffffffu, ref.x, 0);
    ref.y = __shfl_sync(0xffffffffu, ref.y, 0);
    write_top(a, r, lists[team], ref);
  }
}

struct LogprobGradArgs {
  const void* logits;
  const int64_t* targets;
  const float *lse, *entropy, *g_logprob, *g_lse, *g_entropy;
  void* grad;
  int64_t rows, ld, grad_ld;
  int64_t tiles;      // rows * tiles_per_row
  int tiles_per_row;
  int vocab;
};
constexpr int kGradThreads = 256;
constexpr int kGradBatch = 4;
// A tile is a piece of a row that a team of kT threads takes: a block, or a warp where rows are short.
template <int kT>
constexpr int kGradTile = kT * kGradBatch;  // in vectors

// What the gradient needs of a row, as loaded.
struct RowInputs {
  float lse, entropy, a, b, c;
  int64_t target;
};
__device__ __forceinline__ RowInputs row_inputs(const LogprobGradArgs& x, int64_t r) {
  RowInputs i;
  i.lse = x.lse[r];
  i.a = x.g_logprob ? x.g_logprob[r] : 0.0f;
  i.target = x.g_logprob ? x.targets[r] : -1;
  i.b = x.g_lse ? x.g_lse[r] : 0.0f;
  i.c = x.g_entropy ? x.g_entropy[r] : 0.0f;
  i.entropy = x.g_entropy ? x.entropy[r] : 0.0f;
  return i;
}

// A row's gradient is p_j (A + B d_j) + a [j = t] with d_j = (z_j - lse) log2(e), p_j = 2^d_j, A = b - a - c H,
// B = -c ln 2.  The difference is taken first: with z_j log2(e) - lse log2(e) in one step the rounding of the second product
// would stay in every p of the row.
struct RowGrad {
  float a, A, B, lse;
  int target;    // -1: none
  bool zero;     // nothing flows into this row
  bool extreme;  // lse rounded to fp32 has lost too much of ln s
};
// An lse rounded to fp32 is off by half an ulp at most: 2^-15 from 512 on, 2^-14 from 1024 on, and so on, and every p of the row by
// that factor.  From here on the row's sum is taken anew.
constexpr float kExtremeLse = 1024.0f;
static_assert((kLowestLogit + kExtremeLse) * kLog2e < -200.0f, "p of the lowest logit is 0");
__device__ __forceinline__ RowGrad row_grad(const RowInputs& i, int vocab) {
  RowGrad g;
  const bool wild = i.target >= vocab;
  g.a = i.target >= 0 ? i.a : 0.0f;
  g.target = i.target >= 0 && !wild ? static_cast<int>(i.target) : -1;
  g.lse = i.lse;
  g.zero = (g.a == 0.0f && i.b == 0.0f && i.c == 0.0f) || i.lse == neg_inf();
  g.extreme = !g.zero && fabsf(i.lse) >= kExtremeLse;
  g.A = i.b - g.a - (i.c != 0.0f ? i.c * i.entropy : 0.0f);
  g.B = -i.c * kLn2;
  if (wild && g.a != 0.0f) g.A = quiet_nan();
  return g;
}
// Two entries, clamped beforehand to at least kLowestLogit (so |d| < 7400 where p = 0, and B d is finite for any |c| < 6e34); NaN
// entries stay.  fp32 gradients keep probabilities below 2^-126, for which the exponential costs more instructions.
template <bool kBF16>
__device__ __forceinline__ void grad_pair(float& z0, float& z1, const RowGrad& g) {
  const uint64_t d = mul2(add2(pack2(z0, z1), pack2(-g.lse, -g.lse)), pack2(kLog2e, kLog2e));
  float d0, d1;
  unpack2(d, d0, d1);
  const uint64_t p = kBF16 ? pack2(exp2_approx(d0), exp2_approx(d1)) : pack2(exp2_full(d0), exp2_full(d1));
  unpack2(mul2(p, fma2(pack2(g.B, g.B), d, pack2(g.A, g.A))), z0, z1);
}
template <bool kBF16>
__device__ __forceinline__ float grad_one(float z, const RowGrad& g) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(z) : "f"(kLowestLogit));
  float z1 = 0.0f;
  grad_pair<kBF16>(z, z1, g);
  return z;
}

// Elementwise, a tile per team; kVector: the two rows lie alike against 16-byte boundaries.  Plain (coherent) loads: the
// gradient may be written over the logits, each thread writing what it has read.  Blocks of one tile each, as many as there
// are tiles, keep more loads in flight than resident blocks that go through several: 8192 x 128256 bf16 took 657 us against
// 719 us with eight blocks per SM and the rows' inputs fetched a tile ahead.
// A row of extreme magnitudes (all entries at the type's lowest value, say) takes its maximum and sum anew; one team then
// does the whole row, since the gradient may overwrite the logits.
template <bool kBF16, bool kVector, int kT>
__global__ void __launch_bounds__(kGradThreads)
adagc_token_logprobs_grad_kernel(LogprobGradArgs x) {
  using E = Elem<kBF16>;
  constexpr int kTeams = kGradThreads / kT;
  __shared__ SoftmaxPart warp_part[kGradThreads / 32];
  griddep_wait();
  griddep_launch_dependents();
  const int team = threadIdx.x / kT, tid = threadIdx.x % kT;
  for (int64_t tile = static_cast<int64_t>(blockIdx.x) * kTeams + team; tile < x.tiles; tile += static_cast<int64_t>(gridDim.x) * kTeams) {
    const int64_t r = tile / x.tiles_per_row;
    const int piece = static_cast<int>(tile - r * x.tiles_per_row);
    const RowGrad g = row_grad(row_inputs(x, r), x.vocab);
    const char* in = static_cast<const char*>(x.logits) + r * x.ld * E::kBytes;
    char* out = static_cast<char*>(x.grad) + r * x.grad_ld * E::kBytes;

    if (g.extreme) {
      if (piece != 0) continue;
      RowState st;
      for (int j = tid; j < x.vocab; j += kT) st.add(E::load(in, j));
      SoftmaxPart p = warp_join(st.part(), 16);
      if constexpr (kT > 32) {
        if ((tid & 31) == 0) warp_part[tid >> 5] = p;
        __syncthreads();
        p = warp_part[0];
        for (int w = 1; w < kT / 32; ++w) p = join(p, warp_part[w]);
        __syncthreads();
      } else {
        p.m = __shfl_sync(0xffffffffu, p.m, 0);
        p.s = __shfl_sync(0xffffffffu, p.s, 0);
      }
      const float shift = log2f(p.s);
      for (int j = tid; j < x.vocab; j += kT) {
        float d = fmaf(E::load(in, j) - p.m, kLog2e, -shift);
        // p is 0 from there on, and B d stays finite; a NaN, of the row or of A, passes
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(d) : "f"(kExpFloor));
        E::store(out, j, exp2_full(d) * fmaf(g.B, d, g.A) + (j == g.target ? g.a : 0.0f));
      }
      continue;
    }

    if constexpr (kVector) {
      const int head = min(x.vocab, static_cast<int>((16u - (reinterpret_cast<uintptr_t>(in) & 15u)) & 15u) / E::kBytes);
      const int n = (x.vocab - head) / E::kVec;
      const uint4* src = reinterpret_cast<const uint4*>(in + head * E::kBytes);
      uint4* dst = reinterpret_cast<uint4*>(out + head * E::kBytes);
      const int v0 = piece * kGradTile<kT> + tid;
      uint4 w[kGradBatch];
      if (!g.zero) {
#pragma unroll
        for (int u = 0; u < kGradBatch; ++u)
          if (v0 + u * kT < n) w[u] = __ldcs(src + v0 + u * kT);
      }
#pragma unroll
      for (int u = 0; u < kGradBatch; ++u) {
        const int v = v0 + u * kT;
        if (v >= n) break;
        uint4 res = make_uint4(0, 0, 0, 0);
        if (!g.zero) {
          float z[E::kVec];
          E::expand(E::clamped(w[u]), z);
#pragma unroll
          for (int j = 0; j < E::kVec; j += 2) grad_pair<kBF16>(z[j], z[j + 1], g);
          const int at = g.target - head - v * E::kVec;  // the target's place in this vector, if it is here
          if (g.target >= 0 && static_cast<unsigned>(at) < static_cast<unsigned>(E::kVec)) {
#pragma unroll
            for (int j = 0; j < E::kVec; ++j)
              if (j == at) z[j] += g.a;
          }
          res = E::collect(z);
        }
        __stcs(dst + v, res);
      }
      if (piece == 0) {  // the row's unaligned ends
        const int tail_at = head + n * E::kVec, ends = head + x.vocab - tail_at;
        if (tid < ends) {
          const int j = tid < head ? tid : tail_at + tid - head;
          E::store(out, j, g.zero ? 0.0f : grad_one<kBF16>(E::load(in, j), g) + (j == g.target ? g.a : 0.0f));
        }
      }
    } else {
      const int j0 = piece * kGradTile<kT> * E::kVec, j1 = min(x.vocab - j0, kGradTile<kT> * E::kVec);
#pragma unroll 4
      for (int i = tid; i < j1; i += kT) {
        const int j = j0 + i;
        E::store(out, j, g.zero ? 0.0f : grad_one<kBF16>(E::load(in, j), g) + (j == g.target ? g.a : 0.0f));
      }
    }
  }
}

}  // namespace
