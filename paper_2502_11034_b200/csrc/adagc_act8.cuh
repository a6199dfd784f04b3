// Activation checkpoints in 8 bits: encode, decode, and the gated activation that writes and reads them.
// Part of the translation unit adagc_ops.cu (included there; not compiled on its own).
//
// A unit is 8 consecutive elements of a row: one thread.  Four neighbouring lanes hold a group of 32 and find its largest
// magnitude with two shuffles, on the bit patterns (ordered like the magnitudes; infinities and NaN sort above).  With
// max|x| = 1.f * 2^p the exponent is e = p - 6, or p - 5 where 1.f > 127/64: one addition that carries into the exponent
// field.  x 2^-e is exact, so adding 1.5 * 2^23 rounds it once, to nearest even, and leaves the code in the low byte.
// All kernels here stream: each byte is moved once, and the bound is HBM bandwidth as long as an element costs few
// instructions (bf16 moves 3 bytes of it per encode, 8 in the gated activation): dense matrices need no row arithmetic, codes
// are clamped only at the end of the fp32 range, and decoding is one fused multiply-add.  With row arithmetic, clamps and two
// operations per decoded value the gated activation of 8192 x 11008 bf16 took 145 us forward and 165 us backward.
#pragma once

namespace {

constexpr int kUnit = 8;
constexpr int kGroup = 32;
constexpr int kPitchStep = 128;
constexpr int kActThreads = 256;
constexpr float kRoundMagic = 12582912.0f;  // 1.5 * 2^23

// Divides numbers below 2^31 by a constant: q = (n * mul) >> (31 + shift) with 2^shift >= d > 2^(shift-1),
// mul = floor(2^(31+shift) / d) + 1 (Granlund and Montgomery 1994), as the high word of 2n * mul.
struct FastDiv {
  uint32_t d, mul;
  int shift;
  explicit FastDiv(uint32_t div) : d(div) {
    shift = 0;
    while ((1ull << shift) < div) ++shift;
    mul = static_cast<uint32_t>((1ull << (31 + shift)) / div + 1);
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return __umulhi(n << 1, mul) >> shift; }
};

// How the rows of the matrices of a call lie: dense and without padding (a unit is found without its row), on 16-byte
// boundaries, or anywhere.
enum Rows { kDense, kOnBoundaries, kAnywhere };

struct MatrixIn {
  const char* p;
  int64_t ld;
  uintptr_t begin, end;  // of the whole matrix: what may be read
  Rows rows;
};
struct MatrixOut {
  char* p;
  int64_t ld;
  Rows rows;
  bool wide;  // on 32-byte boundaries
};
struct CheckpointPtrs {
  int8_t* codes;
  uint8_t* exps;
};

// The units of rows [0, rows): unit = row * units_per_row + col / 8; units_per_row is a multiple of 16, so a group never
// lies across the end.  A thread takes kU units, a block's threads apart, and loads all of them first.  Measured on B200 with
// 1 / 2 units per thread, the gated activation of 8192 x 11008 bf16: 114 / 117 us forward, 139 / 147 us backward; encode and
// decode of 16384 x 4096 bf16 with 2 / 4: 33.5 / 33.8 and 32.9 / 33.1 us.
struct UnitGrid {
  uint32_t units;  // < 2^31
  int cols;
  FastDiv per_row;
};
template <Rows kRows>
struct UnitPlace {
  uint32_t at, row = 0;  // at: the unit, 0 beyond the end (those lanes stay for the shuffles)
  int col = 0;
  bool valid;
  __device__ __forceinline__ UnitPlace(const UnitGrid& g, uint32_t unit) {
    valid = unit < g.units;
    at = valid ? unit : 0;
    if constexpr (kRows != kDense) {
      row = g.per_row.div(at);
      col = valid ? static_cast<int>(at - row * g.per_row.d) * kUnit : g.cols;
    }
  }
  __device__ __forceinline__ int64_t element(int64_t ld) const {  // the unit's first element in a matrix
    return kRows == kDense ? static_cast<int64_t>(at) * kUnit : row * ld + col;
  }
};
template <int kU>
__device__ __forceinline__ uint32_t unit_of(int u) {
  return (blockIdx.x * kU + u) * kActThreads + threadIdx.x;
}

// The kOut words that begin `bytes` (0 .. 15, a multiple of the element's size) behind the start of w.
template <bool kBF16, int kIn, int kOut>
__device__ __forceinline__ void shift_words(const uint32_t (&w)[kIn], uint32_t bytes, uint32_t (&out)[kOut]) {
  static_assert(kIn >= kOut + (kBF16 ? 4 : 3), "words to shift in");
  uint32_t t[kOut + 2 + (kBF16 ? 1 : 0)];
  constexpr int kTwo = kOut + 1 + (kBF16 ? 1 : 0), kOne = kOut + (kBF16 ? 1 : 0);
#pragma unroll
  for (int i = 0; i < kTwo; ++i) t[i] = (bytes & 8) ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < kOne; ++i) t[i] = (bytes & 4) ? t[i + 1] : t[i];
#pragma unroll
  for (int i = 0; i < kOut; ++i) out[i] = kBF16 ? __funnelshift_r(t[i], t[i + 1], (bytes & 2) * 8) : t[i];
}

// A unit of a row that starts anywhere is cut out of the aligned vectors around it, where all of them lie inside the
// matrix; element by element otherwise, and at a row's end.
template <bool kBF16, Rows kRows>
__device__ __forceinline__ void load_unit(const MatrixIn& a, const UnitPlace<kRows>& at, int cols, float (&v)[kUnit]) {
  using E = Elem<kBF16>;
  constexpr int kVectors = kUnit / E::kVec;
  const int col = at.col;
  const char* p = a.p + at.element(a.ld) * E::kBytes;
  if (kRows == kDense ? at.valid : col + kUnit <= cols) {
    alignas(16) uint32_t w[4 * kVectors];
    bool done = kRows != kAnywhere;
    if constexpr (kRows != kAnywhere) {
#pragma unroll
      for (int i = 0; i < kVectors; ++i) reinterpret_cast<uint4*>(w)[i] = ld_once(reinterpret_cast<const uint4*>(p) + i);
    } else {
      const uint32_t off = reinterpret_cast<uintptr_t>(p) & 15u;
      const uintptr_t from = reinterpret_cast<uintptr_t>(p) - off;
      done = from >= a.begin && from + 16 * (kVectors + 1) <= a.end;
      if (done) {
        alignas(16) uint32_t x[4 * kVectors + 4];
#pragma unroll
        for (int i = 0; i <= kVectors; ++i) reinterpret_cast<uint4*>(x)[i] = reinterpret_cast<const uint4*>(from)[i];  // (an ordinary load: see ld_once)
        shift_words<kBF16>(x, off, w);
      }
    }
    if (done) {
#pragma unroll
      for (int i = 0; i < kVectors; ++i) {
        float part[E::kVec];
        E::expand(reinterpret_cast<const uint4*>(w)[i], part);
#pragma unroll
        for (int j = 0; j < E::kVec; ++j) v[i * E::kVec + j] = part[j];
      }
      return;
    }
  }
#pragma unroll
  for (int j = 0; j < kUnit; ++j) v[j] = kRows != kDense && col + j < cols ? E::load(p, j) : 0.0f;
}

// A warp's 32 whole units of one row that starts anywhere: through shared memory, from which the lanes take aligned vectors;
// the few elements before the first and behind the last one go in one more store.
template <bool kBF16>
__device__ __forceinline__ void store_run(char* base, const uint32_t (&w)[kUnit * Elem<kBF16>::kBytes / 4], uint4* stage) {
  using E = Elem<kBF16>;
  constexpr int kVectors = kUnit / E::kVec, kAll = 32 * kVectors;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < kVectors; ++i) stage[lane * kVectors + i] = reinterpret_cast<const uint4*>(w)[i];
  __syncwarp();
  const uint32_t off = reinterpret_cast<uintptr_t>(base) & 15u, skip = (16u - off) & 15u;
  const int vectors = off == 0 ? kAll : kAll - 1, head = static_cast<int>(skip) / E::kBytes, tail = static_cast<int>(off) / E::kBytes;
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    const int j = lane + 32 * i;
    if (j < vectors) {
      alignas(16) uint32_t x[8];
      alignas(16) uint32_t y[4];
      reinterpret_cast<uint4*>(x)[0] = stage[j];
      reinterpret_cast<uint4*>(x)[1] = stage[min(j + 1, kAll - 1)];
      shift_words<kBF16>(x, skip, y);
      __stcs(reinterpret_cast<uint4*>(base + skip) + j, reinterpret_cast<const uint4*>(y)[0]);
    }
  }
  const bool at_head = lane < head, at_tail = lane >= 16 && lane - 16 < tail;
  if (off != 0 && (at_head || at_tail)) {
    const int e = at_head ? lane : 32 * kUnit - tail + lane - 16;
    reinterpret_cast<typename E::Type*>(base)[e] = reinterpret_cast<const typename E::Type*>(stage)[e];
  }
  __syncwarp();
}

// Stores one unit; all lanes of a warp call this together, with consecutive units.  In a row that starts anywhere, a warp
// inside one row goes through shared memory (`stage`, its own); in others a lane writes the aligned vectors that begin inside
// its unit, the last of them completed from the next lane's unit, and what no lane completes goes element by element.
template <bool kBF16, Rows kRows>
__device__ __forceinline__ void store_unit(const MatrixOut& a, const UnitPlace<kRows>& at, int cols, const float (&v)[kUnit], uint4* stage) {
  using E = Elem<kBF16>;
  constexpr int kVectors = kUnit / E::kVec;
  const int col = at.col;
  const bool valid = at.valid;
  char* p = a.p + at.element(a.ld) * E::kBytes;
  alignas(16) uint32_t w[4 * kVectors];
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    float part[E::kVec];
#pragma unroll
    for (int j = 0; j < E::kVec; ++j) part[j] = v[i * E::kVec + j];
    reinterpret_cast<uint4*>(w)[i] = E::collect(part);
  }
  const bool whole = valid && (kRows == kDense || col + kUnit <= cols);
  int first = 0, last = valid && kRows != kDense ? min(kUnit, cols - col) : 0;  // elements left to be stored one by one
  if constexpr (kRows != kAnywhere) {
    if (whole) {
      if (kVectors == 2 && a.wide) {
        asm volatile("st.global.cs.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4 % (4 * kVectors)]),
                     "r"(w[5 % (4 * kVectors)]), "r"(w[6 % (4 * kVectors)]), "r"(w[7 % (4 * kVectors)])
                     : "memory");
      } else {
#pragma unroll
        for (int i = 0; i < kVectors; ++i) __stcs(reinterpret_cast<uint4*>(p) + i, reinterpret_cast<const uint4*>(w)[i]);
      }
      last = 0;
    }
  } else if (__all_sync(0xffffffffu, whole) && __shfl_sync(0xffffffffu, at.row, 0) == __shfl_sync(0xffffffffu, at.row, 31)) {
    store_run<kBF16>(p - (threadIdx.x & 31) * (kUnit * E::kBytes), w, stage);
    last = 0;
  } else {
    const uint32_t off = reinterpret_cast<uintptr_t>(p) & 15u, skip = (16u - off) & 15u;  // bytes before the first boundary in the unit
    uint32_t x[4 * kVectors + 4];
    alignas(16) uint32_t y[4 * kVectors];
#pragma unroll
    for (int i = 0; i < 4 * kVectors; ++i) x[i] = w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[4 * kVectors + i] = __shfl_down_sync(0xffffffffu, w[i], 1);
    const int lane = threadIdx.x & 31;
    const bool next_whole = __shfl_down_sync(0xffffffffu, static_cast<int>(whole), 1) && lane < 31 && col + 2 * kUnit <= cols;
    const bool prev_whole = __shfl_up_sync(0xffffffffu, static_cast<int>(whole), 1) && lane > 0 && col > 0;
    if (whole) {
      shift_words<kBF16>(x, skip, y);
      const int vectors = next_whole || skip == 0 ? kVectors : kVectors - 1;
      uint4* q = reinterpret_cast<uint4*>(p + skip);
#pragma unroll
      for (int i = 0; i < kVectors; ++i)
        if (i < vectors) __stcs(q + i, reinterpret_cast<const uint4*>(y)[i]);
      const int head = static_cast<int>(skip) / E::kBytes;
      // the elements before the first boundary belong to the previous lane's last vector, if it was completed
      if (!prev_whole)
#pragma unroll
        for (int j = 0; j < E::kVec; ++j)
          if (j < head) E::store(p, j, v[j]);
      first = head + vectors * E::kVec;
    }
  }
  if (kRows != kDense && __any_sync(0xffffffffu, first < last)) {
#pragma unroll
    for (int j = 0; j < kUnit; ++j)
      if (j >= first && j < last) E::store(p, j, v[j]);
  }
}

// Encodes one unit; the four lanes of its group call this together.  Returns the 8 codes, the exponent byte in `byte`.
__device__ __forceinline__ uint2 encode_unit(const float (&v)[kUnit], uint32_t& byte) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kUnit; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  if (top >= 0x7f800000u) {  // an infinity or a NaN in the group
    byte = 255;
    return make_uint2(0, 0);
  }
  // 0x7e0000: the fraction of 127/64; a larger one carries
  const int e = max(static_cast<int>((top + 0x01ffffu) >> 23) - 6, 1);
  byte = static_cast<uint32_t>(min(e, 248));
  const float inv = __uint_as_float((254 - byte) << 23);
  uint32_t c[kUnit];
#pragma unroll
  for (int j = 0; j < kUnit; ++j) c[j] = __float_as_uint(fmaf(v[j], inv, kRoundMagic));
  if (e > 248) {  // the end of the fp32 range: codes saturate
#pragma unroll
    for (int j = 0; j < kUnit; ++j) c[j] = min(max(c[j], __float_as_uint(kRoundMagic - 127.0f)), __float_as_uint(kRoundMagic + 127.0f));
  }
  return make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410));
}
__device__ __forceinline__ void store_codes(const CheckpointPtrs& c, int64_t unit, const uint2& codes, uint32_t byte) {
  __stcs(reinterpret_cast<uint2*>(c.codes) + unit, codes);
  if ((unit & 3) == 0) c.exps[unit >> 2] = static_cast<uint8_t>(byte);
}

struct EncodedUnit {
  uint2 codes;
  uint32_t byte;
};
__device__ __forceinline__ EncodedUnit load_codes(const CheckpointPtrs& c, uint32_t unit) {
  return {__ldcs(reinterpret_cast<const uint2*>(c.codes) + unit), c.exps[unit >> 2]};
}
// The values of 8 codes: a code's byte, offset by 128, becomes the low bits of 2^23 + (code + 128); all steps are exact.
__device__ __forceinline__ void decode_unit(const EncodedUnit& e, float (&v)[kUnit]) {
  const float scale = e.byte == 255u ? quiet_nan() : __uint_as_float(e.byte << 23);
  const uint32_t u[2] = {e.codes.x ^ 0x80808080u, e.codes.y ^ 0x80808080u};
#pragma unroll
  for (int j = 0; j < kUnit; ++j) v[j] = __uint_as_float(__byte_perm(u[j / 4], 0x4b000000u, 0x7440 + j % 4));
  if (e.byte < 228u) {  // 2^24 times the scale is finite
    const float bias = -8388736.0f * scale;
#pragma unroll
    for (int j = 0; j < kUnit; ++j) v[j] = fmaf(v[j], scale, bias);
  } else {
#pragma unroll
    for (int j = 0; j < kUnit; ++j) v[j] = (v[j] - 8388736.0f) * scale;
  }
}

// 1 / (1 + e^-x).  For bfloat16 results the exponential is one multiplication and one instruction: its relative error grows as
// |x| 2^-24 (4e-6 at -80), a thousandth of their rounding.  fp32 results take the accurate exponential and reciprocal.  Measured
// approximate / accurate, gated activation of 8192 x 11008: bf16 110 / 131 us forward, 135 / 150 us backward with h; fp32 189 / 189
// and 201 / 202 us (HBM), and 57 / 62 and 81 / 88 us for 2731 columns.
template <bool kBF16>
__device__ __forceinline__ float sigmoid(float x) {
  if constexpr (!kBF16) return __frcp_rn(1.0f + expf(-x));
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + exp2_approx(-kLog2e * x)));
  return r;
}

constexpr int kEncodeUnits = 2, kDecodeUnits = 2, kSwigluUnits = 1, kSwigluGradUnits = 1;

// This warp's part of the block's staging area.
template <bool kBF16, Rows kRows>
__device__ __forceinline__ uint4* warp_stage() {
  if constexpr (kRows != kAnywhere) return nullptr;
  constexpr int kVectors = 32 * kUnit / Elem<kBF16>::kVec;
  __shared__ uint4 stage[kRows == kAnywhere ? kActThreads / 32 * kVectors : 1];
  return stage + threadIdx.x / 32 * kVectors;
}

template <bool kBF16, Rows kRows>
__global__ void __launch_bounds__(kActThreads)
adagc_act8_encode_kernel(MatrixIn x, CheckpointPtrs out, UnitGrid g) {
  constexpr int kU = kEncodeUnits;
  griddep_wait();
  griddep_launch_dependents();
  float v[kU][kUnit];
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const UnitPlace<kRows> p(g, unit_of<kU>(u));
    load_unit<kBF16, kRows>(x, p, g.cols, v[u]);
  }
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const uint32_t unit = unit_of<kU>(u);
    uint32_t byte;
    const uint2 codes = encode_unit(v[u], byte);
    if (unit < g.units) store_codes(out, unit, codes, byte);
  }
}

template <bool kBF16, Rows kRows>
__global__ void __launch_bounds__(kActThreads)
adagc_act8_decode_kernel(CheckpointPtrs in, MatrixOut x, UnitGrid g) {
  constexpr int kU = kDecodeUnits;
  griddep_wait();
  griddep_launch_dependents();
  EncodedUnit e[kU];
#pragma unroll
  for (int u = 0; u < kU; ++u) e[u] = load_codes(in, UnitPlace<kRows>(g, unit_of<kU>(u)).at);
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const UnitPlace<kRows> p(g, unit_of<kU>(u));
    float v[kUnit];
    decode_unit(e[u], v);
    store_unit<kBF16, kRows>(x, p, g.cols, v, warp_stage<kBF16, kRows>());
  }
}

template <bool kBF16, Rows kRows>
__global__ void __launch_bounds__(kActThreads)
adagc_act8_swiglu_kernel(MatrixIn gate, MatrixIn up, MatrixOut h, CheckpointPtrs gate8, CheckpointPtrs up8, UnitGrid g) {
  constexpr int kU = kSwigluUnits;
  griddep_wait();
  griddep_launch_dependents();
  float a[kU][kUnit], b[kU][kUnit];
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const UnitPlace<kRows> p(g, unit_of<kU>(u));
    load_unit<kBF16, kRows>(gate, p, g.cols, a[u]);
    load_unit<kBF16, kRows>(up, p, g.cols, b[u]);
  }
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const UnitPlace<kRows> p(g, unit_of<kU>(u));
    uint32_t byte_a, byte_b;
    const uint2 codes_a = encode_unit(a[u], byte_a), codes_b = encode_unit(b[u], byte_b);
    if (p.valid) {
      store_codes(gate8, p.at, codes_a, byte_a);
      store_codes(up8, p.at, codes_b, byte_b);
    }
    float y[kUnit];
#pragma unroll
    for (int j = 0; j < kUnit; ++j) y[j] = a[u][j] * sigmoid<kBF16>(a[u][j]) * b[u][j];
    store_unit<kBF16, kRows>(h, p, g.cols, y, warp_stage<kBF16, kRows>());
  }
}

template <bool kBF16, Rows kRows, bool kKeepH>
__global__ void __launch_bounds__(kActThreads)
adagc_act8_swiglu_grad_kernel(MatrixIn grad_h, CheckpointPtrs gate8, CheckpointPtrs up8, MatrixOut grad_gate, MatrixOut grad_up,
                              CheckpointPtrs h8, UnitGrid g) {
  constexpr int kU = kSwigluGradUnits;
  griddep_wait();
  griddep_launch_dependents();
  float dh[kU][kUnit];
  EncodedUnit ea[kU], eb[kU];
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const UnitPlace<kRows> p(g, unit_of<kU>(u));
    load_unit<kBF16, kRows>(grad_h, p, g.cols, dh[u]);
    ea[u] = load_codes(gate8, p.at);
    eb[u] = load_codes(up8, p.at);
  }
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const UnitPlace<kRows> p(g, unit_of<kU>(u));
    float a[kUnit], b[kUnit], h[kUnit];
    decode_unit(ea[u], a);
    decode_unit(eb[u], b);
#pragma unroll
    for (int j = 0; j < kUnit; ++j) {
      const float s = sigmoid<kBF16>(a[j]), as = a[j] * s;
      h[j] = as * b[j];
      b[j] = dh[u][j] * b[j] * s * fmaf(a[j], 1.0f - s, 1.0f);
      a[j] = dh[u][j] * as;
    }
    store_unit<kBF16, kRows>(grad_gate, p, g.cols, b, warp_stage<kBF16, kRows>());
    store_unit<kBF16, kRows>(grad_up, p, g.cols, a, warp_stage<kBF16, kRows>());
    if constexpr (kKeepH) {
      uint32_t byte;
      const uint2 codes = encode_unit(h, byte);
      if (p.valid) store_codes(h8, p.at, codes, byte);
    }
  }
}

}  // namespace
