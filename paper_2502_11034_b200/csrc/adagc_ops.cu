// Training operators next to the optimizer step: the C ABI of include/adagc_ops.h.
// One translation unit in parts: adagc_logprobs.cuh (token log probabilities and their gradient), adagc_act8.cuh (8-bit
// activation checkpoints, gated activation), adagc_wgrad.cuh (weight gradient from a checkpoint, tensor cores); this file
// holds the checks of arguments, the launch rules and the entry points.  Nothing here has state beyond two lookups made
// once per process (SM counts, the driver's tensor-map encoder).
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <mutex>
#include <type_traits>

#include "../../include/adagc_ops.h"

#include "adagc_common.cuh"
#include "adagc_async.cuh"
#include "adagc_logprobs.cuh"
#include "adagc_act8.cuh"
#include "adagc_wgrad.cuh"

namespace {

bool on_boundary(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
bool known_dtype(int32_t d) { return d == ADAGC_F32 || d == ADAGC_BF16; }
int64_t dtype_bytes(int32_t d) { return d == ADAGC_BF16 ? 2 : 4; }

// Bytes a matrix touches: rows of `width` bytes, `pitch` apart.
struct Span {
  uintptr_t begin, end, width, pitch;
  Span(const void* p, int64_t bytes) : Span(p, 1, bytes, bytes, 1) {}
  Span(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t es)
      : begin(reinterpret_cast<uintptr_t>(p)),
        end(begin + static_cast<uintptr_t>(p ? ((rows - 1) * ld + cols) * es : 0)),
        width(static_cast<uintptr_t>(cols * es)),
        pitch(static_cast<uintptr_t>(ld * es)) {}
  bool overlaps(const Span& o) const {
    if (begin >= o.end || o.begin >= end) return false;
    if (pitch != o.pitch || pitch == 0) return true;
    // the same pitch: column ranges of one matrix may lie side by side
    const uintptr_t d = begin <= o.begin ? (o.begin - begin) % pitch : (pitch - (begin - o.begin) % pitch) % pitch;
    return d < width || d + o.width > pitch;
  }
};

// Columns that leave room for a tile in 32 bits, and extents whose products stay far from the end of 64.
constexpr int64_t kMaxColumns = int64_t{1} << 30, kMaxExtent = int64_t{1} << 40;
bool valid_matrix(int64_t rows, int64_t cols, int64_t ld) {
  return rows >= 0 && cols >= 0 && cols <= kMaxColumns && ld >= cols && ld <= kMaxExtent && rows <= kMaxExtent &&
         (ld == 0 || rows <= (kMaxExtent << 10) / ld);
}

struct DeviceInfo {
  std::once_flag once;
  int sms = 0;
  bool wgrad_ready = false;  // the product's kernel may use the shared memory it wants
};
constexpr int kMaxOpsDevices = 64;
DeviceInfo g_device[kMaxOpsDevices];

// The current device, looked up once; NULL if there is none.
const DeviceInfo* current_device() {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxOpsDevices) {
    (void)cudaGetLastError();
    return nullptr;
  }
  std::call_once(g_device[dev].once, [dev] {
    int sms = 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) g_device[dev].sms = sms;
    g_device[dev].wgrad_ready = cudaFuncSetAttribute(adagc_act8_wgrad_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kWgSmem) == cudaSuccess;
    (void)cudaGetLastError();
  });
  return &g_device[dev];
}

// SMs of the current device, 0 if there is none.
int device_sms() {
  const DeviceInfo* d = current_device();
  return d ? d->sms : 0;
}

// Launches with the programmatic-serialization attribute: the kernel may be started while the one before it in the stream
// drains, and waits for it (griddep_wait) before it touches anything.  Between two kernels of this file that hides the second
// one's launch and set-up: a product of 64 x 768 x 768 went from 10.2 to 7.4 us a call, a checkpoint of 16384 x 4096 fp32 out
// and back from 107.2 to 102.8 us.
template <typename... Params, typename... Args>
int launch(void (*kernel)(Params...), int64_t grid, int block, size_t smem, int cluster, cudaStream_t s, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(static_cast<unsigned>(block));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess) return ADAGC_OK;
  (void)cudaGetLastError();
  return ADAGC_E_CUDA;
}

// ------------------------------------------------------------------------------------------------
// token log probabilities
// ------------------------------------------------------------------------------------------------
template <bool kBF16, int kT, bool kTop>
int launch_logprobs(const LogprobArgs& a, int cluster, cudaStream_t s) {
  constexpr int kTeams = kRowBlock / kT;
  return launch(adagc_token_logprobs_kernel<kBF16, kT, kTop>, (a.rows + kTeams - 1) / kTeams * cluster, kRowBlock, 0, cluster, s, a);
}
template <bool kBF16, int kT>
int launch_logprobs(const LogprobArgs& a, int cluster, cudaStream_t s) {
  return a.top_k > 0 ? launch_logprobs<kBF16, kT, true>(a, cluster, s) : launch_logprobs<kBF16, kT, false>(a, cluster, s);
}
template <bool kBF16>
int launch_logprobs(const LogprobArgs& a, int sms, cudaStream_t s) {
  const int64_t batch = static_cast<int64_t>(kRowBatch) * Elem<kBF16>::kVec;  // entries of one thread's batch
  // A warp alone takes a short row: no barriers, but a row's batches come one after the other.  Measured on B200, bf16, warp
  // against block: 16384 rows of 1000 18.4 / 44.2 us, of 8000 49.5 / 69.6 us, 8192 rows of 16000 46.9 / 54.9 us; long rows gain
  // nothing (8192 of 128256 317 / 324 us, with 8 alternatives 433 / 361 us).
  if (a.vocab <= 32 * batch * 16 && a.rows > sms) return launch_logprobs<kBF16, 32>(a, 1, s);
  // Rows share a cluster while that still leaves SMs idle and a block keeps a few batches of its own.
  int cluster = 1;
  while (cluster < kMaxCluster && a.rows * cluster * 2 <= 4 * sms && a.vocab >= 2 * cluster * batch * kRowBlock) cluster *= 2;
  return launch_logprobs<kBF16, kRowBlock>(a, cluster, s);
}

template <bool kBF16, int kT>
int launch_logprobs_grad(LogprobGradArgs a, bool vector, cudaStream_t s) {
  constexpr int kPer = kGradTile<kT> * Elem<kBF16>::kVec, kTeams = kGradThreads / kT;
  a.tiles_per_row = (a.vocab + kPer - 1) / kPer;
  a.tiles = a.rows * a.tiles_per_row;
  const int64_t grid = std::min<int64_t>((a.tiles + kTeams - 1) / kTeams, INT32_MAX);
  const auto kernel = vector ? adagc_token_logprobs_grad_kernel<kBF16, true, kT> : adagc_token_logprobs_grad_kernel<kBF16, false, kT>;
  return launch(kernel, grid, kGradThreads, 0, 1, s, a);
}

// ------------------------------------------------------------------------------------------------
// 8-bit checkpoints
// ------------------------------------------------------------------------------------------------
int64_t pitch_of(int64_t cols) { return (cols + kPitchStep - 1) / kPitchStep * kPitchStep; }

int check_checkpoint(const adagc_act8* c) {
  if (!c || !c->codes || !c->exps) return ADAGC_E_INVALID_ARG;
  return on_boundary(c->codes, 16) && on_boundary(c->exps, 4) ? ADAGC_OK : ADAGC_E_MISALIGNED;
}
Span codes_span(const adagc_act8* c, int64_t rows, int64_t pitch) { return Span(c->codes, rows * pitch); }
Span exps_span(const adagc_act8* c, int64_t rows, int64_t pitch) { return Span(c->exps, rows * (pitch / kGroup)); }

Rows rows_of(const void* p, int64_t cols, int64_t ld, int64_t es) {
  if (!on_boundary(p, 16) || ld * es % 16 != 0) return kAnywhere;
  return ld == cols && cols % kPitchStep == 0 ? kDense : kOnBoundaries;
}
MatrixIn matrix_in(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t es) {
  const Span all(p, rows, cols, ld, es);
  return {static_cast<const char*>(p), ld, all.begin, all.end, rows_of(p, cols, ld, es)};
}
MatrixOut matrix_out(void* p, int64_t cols, int64_t ld, int64_t es) {
  return {static_cast<char*>(p), ld, rows_of(p, cols, ld, es), on_boundary(p, 32) && ld * es % 32 == 0};
}
// Calls launch(dtype, rows) with the two as compile-time values.
template <typename F>
int by_kind(int32_t dtype, Rows rows, F launch) {
  const auto with = [&](auto bf16) {
    switch (rows) {
      case kDense: return launch(bf16, std::integral_constant<Rows, kDense>());
      case kOnBoundaries: return launch(bf16, std::integral_constant<Rows, kOnBoundaries>());
      default: return launch(bf16, std::integral_constant<Rows, kAnywhere>());
    }
  };
  return dtype == ADAGC_BF16 ? with(std::true_type()) : with(std::false_type());
}

// Calls piece(first row, grid, UnitGrid) for pieces of fewer than 2^31 units (less a block's), `per_thread` units a thread.
template <typename F>
int by_units(int64_t rows, int64_t cols, int64_t pitch, int per_thread, F piece) {
  const int64_t block = static_cast<int64_t>(kActThreads) * per_thread;
  const int64_t per_row = pitch / kUnit, most = ((int64_t{1} << 31) - 1 - block) / per_row;
  if (most == 0) return ADAGC_E_INVALID_ARG;
  for (int64_t r0 = 0; r0 < rows; r0 += most) {
    const int64_t units = std::min(most, rows - r0) * per_row;
    UnitGrid g{static_cast<uint32_t>(units), static_cast<int>(cols), FastDiv(static_cast<uint32_t>(per_row))};
    if (int rc = piece(r0, (units + block - 1) / block, g)) return rc;
  }
  return ADAGC_OK;
}
CheckpointPtrs rows_from(const adagc_act8* c, int64_t r0, int64_t pitch) {
  return {c->codes + r0 * pitch, c->exps + r0 * (pitch / kGroup)};
}
template <typename M>
M rows_from(M m, int64_t r0, int64_t es) {
  m.p += r0 * m.ld * es;
  return m;
}

// ------------------------------------------------------------------------------------------------
// weight gradient
// ------------------------------------------------------------------------------------------------
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
std::once_flag g_encode_once;
EncodeTiled g_encode = nullptr;
EncodeTiled tensor_map_encoder() {
  std::call_once(g_encode_once, [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) == cudaSuccess &&
        found == cudaDriverEntryPointSuccess)
      g_encode = reinterpret_cast<EncodeTiled>(f);
    (void)cudaGetLastError();
  });
  return g_encode;
}
bool make_map(CUtensorMap* map, CUtensorMapDataType type, const void* base, int64_t cols, int64_t rows, int64_t row_bytes, int box_cols, int box_rows) {
  EncodeTiled encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(row_bytes)};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows)}, unit[2] = {1, 1};
  return encode(map, type, 2, const_cast<void*>(base), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct WgradPlan {
  int tiles_n, steps, whole, tail, splits, steps_per_split;
  int64_t pitch;  // of the packed dY in elements, 0: dY is read in place
  int64_t pack_bytes, bytes;  // the packed dY, then partial sums: of split tiles, then one block for each pair
};
constexpr int kB200Pairs = 74;  // plans do not depend on the device present: the workspace is sized without one
WgradPlan wgrad_plan(int64_t tokens, int64_t n, int64_t k, const void* dy, int64_t ld) {
  WgradPlan p{};
  p.tiles_n = static_cast<int>((n + kWgTileN - 1) / kWgTileN);
  const int tiles = p.tiles_n * static_cast<int>((k + kWgPairK - 1) / kWgPairK);
  p.steps = static_cast<int>((tokens + kWgStep - 1) / kWgStep);
  // Tiles are dealt out whole while every pair of SMs gets one.  The rest, too few for that, have their steps shared out
  // among the pairs where that is worth the kernel that joins the partial sums: a step takes about 300 ns, the join 5 us
  // and 131 ns per partial tile.  Measured on B200 (whole / shared out, us): 8192 x 4096 x 11008 616 / 603, 4096 x 768 x 768
  // 33.8 / 21.8, 16384 x 256 x 256 113 / 18.4; 1024 x 4096 x 4096 41.9 / 51.4 and 512 x 768 x 768 13.3 / 17.5 stay whole.
  const int rest = tiles % kB200Pairs, most = rest ? std::min(kB200Pairs / rest, p.steps / 4) : 0;
  int64_t best = p.steps * int64_t{300};
  for (int n_splits = 2; n_splits <= most; ++n_splits) {
    const int per = (p.steps + n_splits - 1) / n_splits, used = (p.steps + per - 1) / per;
    const int64_t ns = per * int64_t{300} + 5000 + int64_t{131} * used * rest;
    if (ns < best) best = ns, p.splits = used, p.steps_per_split = per;
  }
  p.tail = p.splits ? rest : 0;
  p.whole = tiles - p.tail;
  p.pitch = on_boundary(dy, 16) && ld % 8 == 0 && ld < (int64_t{1} << 38) ? 0 : (n + 7) / 8 * 8;
  p.pack_bytes = (tokens * p.pitch * 2 + 255) / 256 * 256;
  constexpr int64_t tile_bytes = int64_t{kWgTileN} * kWgPairK * 4;
  p.bytes = p.pack_bytes + (p.splits * p.tail + (p.steps > kWgExactSteps ? std::min(p.whole, kB200Pairs) : 0)) * tile_bytes;
  return p;
}
bool valid_wgrad(int64_t tokens, int64_t n, int64_t k, int64_t ld) {
  constexpr int64_t most = kMaxColumns;
  return tokens >= 0 && n >= 0 && k >= 0 && tokens <= most && n <= most && k <= most && valid_matrix(tokens, n, ld) &&
         ((n + kWgTileN - 1) / kWgTileN) * ((k + kWgPairK - 1) / kWgPairK) < most;
}

}  // namespace

extern "C" {

int adagc_token_logprobs(const void* d_logits, int32_t logits_dtype, int64_t rows, int64_t vocab, int64_t ld, const int64_t* d_targets,
                         float* d_logprob, float* d_lse, float* d_entropy, int32_t top_k, float* d_top_logprob, int32_t* d_top_index,
                         void* cuda_stream) {
  if (!valid_matrix(rows, vocab, ld) || vocab < 1 || rows >= (int64_t{1} << 31) || top_k < 0 || top_k > ADAGC_MAX_TOP_K) return ADAGC_E_INVALID_ARG;
  if (!known_dtype(logits_dtype)) return ADAGC_E_DTYPE;
  if (rows == 0) return ADAGC_OK;
  if (!d_logits || !d_lse || (d_targets == nullptr) != (d_logprob == nullptr) || (top_k > 0 && (!d_top_logprob || !d_top_index))) return ADAGC_E_INVALID_ARG;
  const int64_t es = dtype_bytes(logits_dtype);
  if (!on_boundary(d_logits, es) || !on_boundary(d_targets, 8) || !on_boundary(d_logprob, 4) || !on_boundary(d_lse, 4) || !on_boundary(d_entropy, 4) ||
      !on_boundary(d_top_logprob, 4) || !on_boundary(d_top_index, 4))
    return ADAGC_E_MISALIGNED;
  const Span in[2] = {Span(d_logits, rows, vocab, ld, es), Span(d_targets, rows * 8)};
  const Span out[5] = {Span(d_logprob, rows * 4), Span(d_lse, rows * 4), Span(d_entropy, rows * 4),
                       Span(top_k ? d_top_logprob : nullptr, rows * top_k * 4), Span(top_k ? d_top_index : nullptr, rows * top_k * 4)};
  for (int i = 0; i < 5; ++i) {
    for (const Span& s : in)
      if (out[i].overlaps(s)) return ADAGC_E_OVERLAP;
    for (int j = 0; j < i; ++j)
      if (out[i].overlaps(out[j])) return ADAGC_E_OVERLAP;
  }
  const int sms = device_sms();
  if (sms == 0) return ADAGC_E_CUDA;
  const LogprobArgs a{d_logits, d_targets, d_logprob, d_lse, d_entropy, d_top_logprob, d_top_index, rows, ld, static_cast<int>(vocab), top_k};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return logits_dtype == ADAGC_BF16 ? launch_logprobs<true>(a, sms, s) : launch_logprobs<false>(a, sms, s);
}

int adagc_token_logprobs_backward(const void* d_logits, int32_t logits_dtype, int64_t rows, int64_t vocab, int64_t ld, const int64_t* d_targets,
                                  const float* d_lse, const float* d_entropy, const float* d_grad_logprob, const float* d_grad_lse,
                                  const float* d_grad_entropy, void* d_grad_logits, int64_t grad_ld, void* cuda_stream) {
  if (!valid_matrix(rows, vocab, ld) || !valid_matrix(rows, vocab, grad_ld) || vocab < 1) return ADAGC_E_INVALID_ARG;
  if (!known_dtype(logits_dtype)) return ADAGC_E_DTYPE;
  if (rows == 0) return ADAGC_OK;
  if (!d_logits || !d_lse || !d_grad_logits || (d_grad_logprob && !d_targets) || (d_grad_entropy && !d_entropy)) return ADAGC_E_INVALID_ARG;
  const int64_t es = dtype_bytes(logits_dtype);
  const float* stats[5] = {d_lse, d_entropy, d_grad_logprob, d_grad_lse, d_grad_entropy};
  if (!on_boundary(d_logits, es) || !on_boundary(d_grad_logits, es) || !on_boundary(d_targets, 8)) return ADAGC_E_MISALIGNED;
  const Span out(d_grad_logits, rows, vocab, grad_ld, es);
  for (const float* p : stats) {
    if (!on_boundary(p, 4)) return ADAGC_E_MISALIGNED;
    if (out.overlaps(Span(p, rows * 4))) return ADAGC_E_OVERLAP;
  }
  if (out.overlaps(Span(d_targets, rows * 8))) return ADAGC_E_OVERLAP;
  const bool in_place = d_grad_logits == d_logits && grad_ld == ld;
  if (!in_place && out.overlaps(Span(d_logits, rows, vocab, ld, es))) return ADAGC_E_OVERLAP;
  if (device_sms() == 0) return ADAGC_E_CUDA;
  const LogprobGradArgs a{d_logits, d_targets, d_lse, d_entropy, d_grad_logprob, d_grad_lse, d_grad_entropy, d_grad_logits, rows, ld, grad_ld, 0, 0,
                          static_cast<int>(vocab)};
  const bool vector = (reinterpret_cast<uintptr_t>(d_logits) - reinterpret_cast<uintptr_t>(d_grad_logits)) % 16 == 0 && (ld - grad_ld) * es % 16 == 0;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  // Rows that would leave half of a block's threads without a vector go to warps.  Measured on B200, bf16, warp against block:
  // 16384 rows of 1000 12.3 / 36.8 us, of 4000 46.8 / 53.5 us.
  const bool narrow = vocab * es <= 8192;
  if (logits_dtype == ADAGC_BF16) return narrow ? launch_logprobs_grad<true, 32>(a, vector, s) : launch_logprobs_grad<true, kGradThreads>(a, vector, s);
  return narrow ? launch_logprobs_grad<false, 32>(a, vector, s) : launch_logprobs_grad<false, kGradThreads>(a, vector, s);
}

int64_t adagc_act8_pitch(int64_t cols) { return cols < 0 || cols > kMaxExtent ? 0 : pitch_of(cols); }

int adagc_act8_encode(const void* d_x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, const adagc_act8* out, void* cuda_stream) {
  if (!valid_matrix(rows, cols, ld)) return ADAGC_E_INVALID_ARG;
  if (!known_dtype(dtype)) return ADAGC_E_DTYPE;
  if (rows == 0 || cols == 0) return ADAGC_OK;
  if (!d_x) return ADAGC_E_INVALID_ARG;
  if (int rc = check_checkpoint(out)) return rc;
  const int64_t es = dtype_bytes(dtype), pitch = pitch_of(cols);
  if (!on_boundary(d_x, es)) return ADAGC_E_MISALIGNED;
  const Span x(d_x, rows, cols, ld, es), c = codes_span(out, rows, pitch), e = exps_span(out, rows, pitch);
  if (c.overlaps(x) || e.overlaps(x) || c.overlaps(e)) return ADAGC_E_OVERLAP;
  if (device_sms() == 0) return ADAGC_E_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const MatrixIn m = matrix_in(d_x, rows, cols, ld, es);
  return by_kind(dtype, m.rows, [&](auto bf16, auto kind) {
    return by_units(rows, cols, pitch, kEncodeUnits, [&](int64_t r0, int64_t grid, const UnitGrid& g) {
      return launch(adagc_act8_encode_kernel<bf16(), kind()>, grid, kActThreads, 0, 1, s, rows_from(m, r0, es), rows_from(out, r0, pitch), g);
    });
  });
}

int adagc_act8_decode(const adagc_act8* in, int64_t rows, int64_t cols, void* d_x, int32_t dtype, int64_t ld, void* cuda_stream) {
  if (!valid_matrix(rows, cols, ld)) return ADAGC_E_INVALID_ARG;
  if (!known_dtype(dtype)) return ADAGC_E_DTYPE;
  if (rows == 0 || cols == 0) return ADAGC_OK;
  if (!d_x) return ADAGC_E_INVALID_ARG;
  if (int rc = check_checkpoint(in)) return rc;
  const int64_t es = dtype_bytes(dtype), pitch = pitch_of(cols);
  if (!on_boundary(d_x, es)) return ADAGC_E_MISALIGNED;
  const Span x(d_x, rows, cols, ld, es);
  if (x.overlaps(codes_span(in, rows, pitch)) || x.overlaps(exps_span(in, rows, pitch))) return ADAGC_E_OVERLAP;
  if (device_sms() == 0) return ADAGC_E_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const MatrixOut m = matrix_out(d_x, cols, ld, es);
  return by_kind(dtype, m.rows, [&](auto bf16, auto kind) {
    return by_units(rows, cols, pitch, kDecodeUnits, [&](int64_t r0, int64_t grid, const UnitGrid& g) {
      return launch(adagc_act8_decode_kernel<bf16(), kind()>, grid, kActThreads, 0, 1, s, rows_from(in, r0, pitch), rows_from(m, r0, es), g);
    });
  });
}

int adagc_act8_swiglu(const void* d_gate, int64_t ld_gate, const void* d_up, int64_t ld_up, int32_t dtype, int64_t rows, int64_t cols, void* d_h,
                      int64_t ld_h, const adagc_act8* gate8, const adagc_act8* up8, void* cuda_stream) {
  if (!valid_matrix(rows, cols, ld_gate) || !valid_matrix(rows, cols, ld_up) || !valid_matrix(rows, cols, ld_h)) return ADAGC_E_INVALID_ARG;
  if (!known_dtype(dtype)) return ADAGC_E_DTYPE;
  if (rows == 0 || cols == 0) return ADAGC_OK;
  if (!d_gate || !d_up || !d_h) return ADAGC_E_INVALID_ARG;
  if (int rc = check_checkpoint(gate8)) return rc;
  if (int rc = check_checkpoint(up8)) return rc;
  const int64_t es = dtype_bytes(dtype), pitch = pitch_of(cols);
  if (!on_boundary(d_gate, es) || !on_boundary(d_up, es) || !on_boundary(d_h, es)) return ADAGC_E_MISALIGNED;
  const Span in[2] = {Span(d_gate, rows, cols, ld_gate, es), Span(d_up, rows, cols, ld_up, es)};
  const Span out[5] = {Span(d_h, rows, cols, ld_h, es), codes_span(gate8, rows, pitch), exps_span(gate8, rows, pitch), codes_span(up8, rows, pitch),
                       exps_span(up8, rows, pitch)};
  for (int i = 0; i < 5; ++i) {
    for (const Span& x : in)
      if (out[i].overlaps(x)) return ADAGC_E_OVERLAP;
    for (int j = 0; j < i; ++j)
      if (out[i].overlaps(out[j])) return ADAGC_E_OVERLAP;
  }
  if (device_sms() == 0) return ADAGC_E_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const MatrixIn mg = matrix_in(d_gate, rows, cols, ld_gate, es), mu = matrix_in(d_up, rows, cols, ld_up, es);
  const MatrixOut mh = matrix_out(d_h, cols, ld_h, es);
  return by_kind(dtype, std::max({mg.rows, mu.rows, mh.rows}), [&](auto bf16, auto kind) {
    return by_units(rows, cols, pitch, kSwigluUnits, [&](int64_t r0, int64_t grid, const UnitGrid& g) {
      return launch(adagc_act8_swiglu_kernel<bf16(), kind()>, grid, kActThreads, 0, 1, s, rows_from(mg, r0, es), rows_from(mu, r0, es), rows_from(mh, r0, es),
                    rows_from(gate8, r0, pitch), rows_from(up8, r0, pitch), g);
    });
  });
}

int adagc_act8_swiglu_backward(const void* d_grad_h, int64_t ld_grad_h, int32_t dtype, int64_t rows, int64_t cols, const adagc_act8* gate8,
                               const adagc_act8* up8, void* d_grad_gate, int64_t ld_grad_gate, void* d_grad_up, int64_t ld_grad_up,
                               const adagc_act8* h8, void* cuda_stream) {
  if (!valid_matrix(rows, cols, ld_grad_h) || !valid_matrix(rows, cols, ld_grad_gate) || !valid_matrix(rows, cols, ld_grad_up)) return ADAGC_E_INVALID_ARG;
  if (!known_dtype(dtype)) return ADAGC_E_DTYPE;
  if (rows == 0 || cols == 0) return ADAGC_OK;
  if (!d_grad_h || !d_grad_gate || !d_grad_up) return ADAGC_E_INVALID_ARG;
  if (int rc = check_checkpoint(gate8)) return rc;
  if (int rc = check_checkpoint(up8)) return rc;
  if (h8)
    if (int rc = check_checkpoint(h8)) return rc;
  const int64_t es = dtype_bytes(dtype), pitch = pitch_of(cols);
  if (!on_boundary(d_grad_h, es) || !on_boundary(d_grad_gate, es) || !on_boundary(d_grad_up, es)) return ADAGC_E_MISALIGNED;
  const Span in[5] = {Span(d_grad_h, rows, cols, ld_grad_h, es), codes_span(gate8, rows, pitch), exps_span(gate8, rows, pitch),
                      codes_span(up8, rows, pitch), exps_span(up8, rows, pitch)};
  const Span out[4] = {Span(d_grad_gate, rows, cols, ld_grad_gate, es), Span(d_grad_up, rows, cols, ld_grad_up, es),
                       Span(h8 ? h8->codes : nullptr, rows * pitch), Span(h8 ? h8->exps : nullptr, rows * (pitch / kGroup))};
  for (int i = 0; i < 4; ++i) {
    for (const Span& x : in)
      if (out[i].overlaps(x)) return ADAGC_E_OVERLAP;
    for (int j = 0; j < i; ++j)
      if (out[i].overlaps(out[j])) return ADAGC_E_OVERLAP;
  }
  if (device_sms() == 0) return ADAGC_E_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const MatrixIn mdh = matrix_in(d_grad_h, rows, cols, ld_grad_h, es);
  const MatrixOut mg = matrix_out(d_grad_gate, cols, ld_grad_gate, es), mu = matrix_out(d_grad_up, cols, ld_grad_up, es);
  return by_kind(dtype, std::max({mdh.rows, mg.rows, mu.rows}), [&](auto bf16, auto kind) {
    return by_units(rows, cols, pitch, kSwigluGradUnits, [&](int64_t r0, int64_t grid, const UnitGrid& g) {
      const auto kernel = h8 ? adagc_act8_swiglu_grad_kernel<bf16(), kind(), true> : adagc_act8_swiglu_grad_kernel<bf16(), kind(), false>;
      return launch(kernel, grid, kActThreads, 0, 1, s, rows_from(mdh, r0, es), rows_from(gate8, r0, pitch), rows_from(up8, r0, pitch), rows_from(mg, r0, es),
                    rows_from(mu, r0, es), h8 ? rows_from(h8, r0, pitch) : CheckpointPtrs{nullptr, nullptr}, g);
    });
  });
}

int64_t adagc_act8_linear_wgrad_workspace_bytes(int64_t tokens, int64_t out_features, int64_t in_features, const void* d_grad_y, int64_t ld_grad_y) {
  if (!valid_wgrad(tokens, out_features, in_features, ld_grad_y)) return ADAGC_E_INVALID_ARG;
  if (tokens == 0 || out_features == 0 || in_features == 0) return 0;
  return wgrad_plan(tokens, out_features, in_features, d_grad_y, ld_grad_y).bytes;
}

int adagc_act8_linear_wgrad(const void* d_grad_y, int32_t grad_y_dtype, int64_t ld_grad_y, const adagc_act8* x8, int64_t tokens, int64_t out_features,
                            int64_t in_features, void* d_grad_w, int32_t grad_w_dtype, int64_t ld_grad_w, int32_t accumulate, void* d_workspace,
                            size_t workspace_bytes, void* cuda_stream) {
  const int64_t n = out_features, k = in_features;
  if (!valid_wgrad(tokens, n, k, ld_grad_y) || !valid_matrix(n, k, ld_grad_w) || accumulate < 0 || accumulate > 1) return ADAGC_E_INVALID_ARG;
  if (grad_y_dtype != ADAGC_BF16 || !known_dtype(grad_w_dtype)) return ADAGC_E_DTYPE;
  if (n == 0 || k == 0 || (tokens == 0 && accumulate)) return ADAGC_OK;
  const int64_t es = dtype_bytes(grad_w_dtype);
  if (!d_grad_w) return ADAGC_E_INVALID_ARG;
  if (!on_boundary(d_grad_w, es)) return ADAGC_E_MISALIGNED;
  const int sms = device_sms();
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const bool bf16 = grad_w_dtype == ADAGC_BF16;
  if (tokens == 0) {
    if (sms == 0) return ADAGC_E_CUDA;
    const int64_t wide = std::min<int64_t>((n * k + 255) / 256, static_cast<int64_t>(sms) * 16);
    return launch(bf16 ? adagc_act8_wgrad_zero_kernel<true> : adagc_act8_wgrad_zero_kernel<false>, wide, 256, 0, 1, s, d_grad_w, n, k, ld_grad_w);
  }
  if (!d_grad_y) return ADAGC_E_INVALID_ARG;
  if (int rc = check_checkpoint(x8)) return rc;
  if (!on_boundary(d_grad_y, 2)) return ADAGC_E_MISALIGNED;
  const WgradPlan p = wgrad_plan(tokens, n, k, d_grad_y, ld_grad_y);
  if (p.bytes > 0 && (!d_workspace || workspace_bytes < static_cast<size_t>(p.bytes) || !on_boundary(d_workspace, 256))) return ADAGC_E_WORKSPACE;
  const int64_t pitch = pitch_of(k);
  const Span in[3] = {Span(d_grad_y, tokens, n, ld_grad_y, 2), codes_span(x8, tokens, pitch), exps_span(x8, tokens, pitch)};
  const Span dw(d_grad_w, n, k, ld_grad_w, es), ws(p.bytes ? d_workspace : nullptr, p.bytes);
  for (const Span& x : in)
    if (dw.overlaps(x) || ws.overlaps(x)) return ADAGC_E_OVERLAP;
  if (dw.overlaps(ws)) return ADAGC_E_OVERLAP;
  if (sms == 0) return ADAGC_E_CUDA;

  const void* dy = p.pitch ? d_workspace : d_grad_y;
  CUtensorMap map_codes, map_dy;
  if (!make_map(&map_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, x8->codes, pitch, tokens, pitch, kWgTileK, kWgStep) ||
      !make_map(&map_dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dy, n, tokens, (p.pitch ? p.pitch : ld_grad_y) * 2, 64, kWgStep))
    return ADAGC_E_CUDA;
  (void)cudaGetLastError();
  if (!current_device()->wgrad_ready) return ADAGC_E_CUDA;
  if (p.pitch) {
    const MatrixIn from = matrix_in(d_grad_y, tokens, n, ld_grad_y, 2);
    const MatrixOut to = matrix_out(d_workspace, p.pitch, p.pitch, 2);
    const int rc = by_units(tokens, n, p.pitch, 1, [&](int64_t r0, int64_t grid, const UnitGrid& g) {
      return launch(adagc_act8_wgrad_pack_kernel, grid, kActThreads, 0, 1, s, rows_from(from, r0, 2), rows_from(to, r0, 2), g);
    });
    if (rc) return rc;
  }
  WgradArgs a{};
  a.exps = x8->exps;
  a.exps_pitch = pitch / kGroup;
  a.out = d_grad_w;
  a.partials = reinterpret_cast<float*>(static_cast<char*>(d_workspace) + p.pack_bytes);
  a.ld_out = ld_grad_w;
  a.tokens = static_cast<int>(tokens);
  a.n = static_cast<int>(n);
  a.k = static_cast<int>(k);
  a.tiles_n = p.tiles_n;
  a.whole = p.whole;
  a.tail = p.tail;
  a.splits = p.splits;
  a.steps = p.steps;
  a.steps_per_split = p.steps_per_split;
  const int most = bf16 ? kWgLongSteps : kWgExactSteps, flushes = (p.steps + most - 1) / most;
  a.steps_per_flush = (p.steps + flushes - 1) / flushes;
  a.apart = (accumulate || bf16) && flushes > 1;
  a.out_bf16 = bf16;
  a.accumulate = accumulate;
  const int pairs = std::min({p.whole + p.tail * p.splits, sms / 2, kB200Pairs});
  if (int rc = launch(adagc_act8_wgrad_kernel, 2 * pairs, kWgThreads, kWgSmem, 1, s, map_codes, map_dy, a)) return rc;
  if (!p.tail) return ADAGC_OK;
  return launch(bf16 ? adagc_act8_wgrad_join_kernel<true> : adagc_act8_wgrad_join_kernel<false>, p.tail * kWgTileN, kWgPairK, 0, 1, s, a);
}

}  // extern "C"
