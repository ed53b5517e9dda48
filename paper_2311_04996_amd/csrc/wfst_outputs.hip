// The operators beside the decoder (the second part of include/wfst_decoder.h): checks of arguments and launches.
#include <hip/hip_runtime.h>

#include <climits>
#include <cstdint>
#include <cstdio>

#include "wfst_decoder.h"
#include "wfst_error.h"
#include "wfst_linear.h"
#include "wfst_logprobs.h"

namespace {

using namespace wfst_ops;

int refuse(const char *what, const char *why) {
  char msg[256];
  snprintf(msg, sizeof msg, "%s: %s", what, why);
  return wfst_note_error(WFST_ERR_INVALID_ARG, msg);
}

// hipLaunchKernel's own answer: an error that an earlier call of the program left behind is not taken for this one's
template <class Args>
int launch(const char *what, void (*kernel)(Args), int64_t workgroups, int threads, const Args &a, void *stream) {
  if (workgroups <= 0) return WFST_OK;
  if (workgroups > UINT32_MAX / threads) return refuse(what, "too many rows for one launch");      // (a grid has 2^32 - 1 work items at most)
  Args copy = a;
  void *argv[] = {&copy};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)workgroups), dim3(threads), argv, 0,
                                       static_cast<hipStream_t>(stream));
  if (e == hipSuccess) return WFST_OK;
  (void)hipGetLastError();
  char msg[256];
  snprintf(msg, sizeof msg, "%s: launch failed: %s", what, hipGetErrorString(e));
  return wfst_note_error(WFST_ERR_HIP, msg);
}

bool type_ok(int32_t t) { return t >= 0 && t <= 2; }
int64_t type_size(int32_t t) { return t == 0 ? 4 : 2; }
bool aligned(const void *p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)to == 0; }

// The bytes that rows (s, t) of `cols` elements take up, -1 if that does not fit 2^62.
int64_t span(int64_t seqs, int64_t frames, int64_t cols, int64_t seq_stride, int64_t stride, int64_t size) {
  if (seqs == 0 || frames == 0) return 0;
  const __int128 n = ((__int128)(seqs - 1) * seq_stride + (__int128)(frames - 1) * stride + cols) * size;
  return n > ((__int128)1 << 62) ? -1 : (int64_t)n;
}

bool overlap(const void *p, int64_t np, const void *q, int64_t nq) {
  if (!p || !q || np <= 0 || nq <= 0) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return a < b + (uintptr_t)nq && b < a + (uintptr_t)np;
}

// Rows (s, t) of `cols` written elements: no two of them share one.
bool rows_apart(int64_t seqs, int64_t frames, int64_t cols, int64_t seq_stride, int64_t stride) {
  if (seq_stride < 0 || stride < 0) return false;
  if (frames > 1 && stride < cols) return false;
  if (seqs > 1 && seq_stride < cols) return false;
  if (seqs <= 1 || frames <= 1) return true;
  return (__int128)seq_stride >= (__int128)(frames - 1) * stride + cols || (__int128)stride >= (__int128)(seqs - 1) * seq_stride + cols;
}

// Every row starts at a multiple of 16 bytes and is a whole number of 16-byte chunks, and the 256 rows of a tile are within 2 GB.
bool chunked(const void *p, int64_t stride, int64_t k, int64_t size) {
  return aligned(p, 16) && k * size % 16 == 0 && stride * size % 16 == 0 && stride < ((1 << 30) - k) / size / 128;
}

template <class F> int by_type(int32_t dtype, F f) { return dtype == 0 ? f(F32{}) : dtype == 1 ? f(F16{}) : f(BF16{}); }

int64_t count_tiles(const LinearArgs &a, int bm, int bn) { return ((a.rows - 1) / bm + 1) * (((int64_t)a.n - 1) / bn + 1); }

template <class E, int BM, int BN, int WM, int WN, int ROW, int STAGES, bool DIRECT>
int run_tiles(LinearArgs a, void *stream) {
  a.tiles_n = (a.n - 1) / BN + 1;
  if ((a.rows - 1) / BM + 1 > INT_MAX / a.tiles_n) return refuse("wfst_linear", "too many rows for one launch");
  return launch("wfst_linear", linear_kernel<E, BM, BN, WM, WN, ROW, STAGES, DIRECT>, count_tiles(a, BM, BN), 64 * (BM / WM) * (BN / WN), a, stream);
}

// The largest tile of which there is one for each compute unit: it reads the least per product (256 x 256: 32 bytes per clock and
// compute unit at full rate, 128 x 128: 64, which is what a compute unit can load), but smaller ones fill the GPU earlier.
// bf16, us, inputs in the caches, tiles of 256 x 256 / 256 x 128 / 128 x 128 / 64 x 64 (k x n): 118,417 rows, 512 x 2048: 279 / 300 / 331 / -;
// 16,384, 2048 x 512: 49 / 44 / 47 / 57 (128, 256, 512, 2,048 tiles); 2,048, 2048 x 2048: 44 / 35 / 28 / 39 (64, 128, 256, 1,024);
// 512, 512 x 2048: 18 / 13 / 10 / 6.  Half of a 64 x 64 tile, as long as there is a compute unit for each: 1,024 rows, 2048 x 512, inputs from
// memory: 10.2, whole ones 12.2; behind that (512 x 2048): 13.8, 9.4.  Tiles of 16 x 16 with k shared out over the waves: 33 to 128 rows,
// 2048 x 512: 7.4, 64 x 64: 9.1; 512 rows (1,024 tiles): 19, 64 x 64: 9.3.  By way of registers 256 x 256 gains nothing
// (511 x 2047: 482 / 476 / 531), 64 x 64 loses more (815 where 256 x 128 takes 436).
// In fp32 the matrix instructions take longest, and 128 x 128 gains little and only where they are most of the time: rows of whole chunks, k of
// 512 or more, results whose rows can be stored 32 bytes at a time, and at most a tenth of the last round idle.  64 x 64 / 128 x 128 (tiles of 128 x 128,
// rounds of 256): 512 x 1024: 448: 61 / 66, 480: 67 / 66, 512: 69 / 68, 928: 125 / 127, 1,024: 134 / 128, 1,280: 174 / 159; 1024 x 256: 1,280:
// 329 / 308; but 512 x 1021: 1,024: 136 / 169; 256 x 1024: 74 / 76; 180 x 333: 960: 67 / 86; by way of registers 177 x 1021: 64 / 98.
template <class E> int run_linear(LinearArgs a, bool direct, void *stream) {
  if (count_tiles(a, 16, 16) <= 256) {
    a.tiles_n = (a.n - 1) / 16 + 1;
    return launch("wfst_linear", linear_few_kernel<E>, count_tiles(a, 16, 16), 512, a, stream);
  }
  if constexpr (sizeof(typename E::T) == 4) {
    const int64_t tiles = count_tiles(a, 128, 128), rounds = (tiles + 255) / 256;
    if (direct && a.k >= 512 && a.n % 8 == 0 && tiles >= 256 && tiles * 10 >= rounds * 256 * 9) return run_tiles<E, 128, 128, 64, 64, 64, 3, true>(a, stream);
    return direct ? run_tiles<E, 64, 64, 32, 32, 64, 4, true>(a, stream) : run_tiles<E, 64, 64, 32, 32, 64, 3, false>(a, stream);
  } else {
    if (direct && count_tiles(a, 256, 256) >= 256) return run_tiles<E, 256, 256, 64, 64, 64, 3, true>(a, stream);
    if (count_tiles(a, 256, 128) >= 256)
      return direct ? run_tiles<E, 256, 128, 64, 64, 64, 3, true>(a, stream) : run_tiles<E, 256, 128, 64, 64, 64, 3, false>(a, stream);
    if (count_tiles(a, 128, 128) >= 256)
      return direct ? run_tiles<E, 128, 128, 64, 64, 64, 3, true>(a, stream) : run_tiles<E, 128, 128, 64, 64, 64, 3, false>(a, stream);
    if (direct && count_tiles(a, 32, 64) <= 256) return run_tiles<E, 32, 64, 32, 32, 128, 4, true>(a, stream);
    return direct ? run_tiles<E, 64, 64, 32, 32, 128, 3, true>(a, stream) : run_tiles<E, 64, 64, 32, 32, 128, 3, false>(a, stream);
  }
}

template <class E, int BM, int BN, int WM, int WN, int ROW, int STAGES, int GROUPS, int PER_SIMD>
int run_rows(const LoglikesArgs &a, bool direct, void *stream) {
  const int64_t blocks = ((int64_t)a.seqs * a.frames - 1) / BM + 1;
  constexpr int kThreads = 64 * (BM / WM) * (BN / WN);
  return direct ? launch("wfst_loglikes", loglikes_kernel<E, BM, BN, WM, WN, ROW, STAGES, GROUPS, true, PER_SIMD>, blocks, kThreads, a, stream)
                : launch("wfst_loglikes", loglikes_kernel<E, BM, BN, WM, WN, ROW, STAGES, GROUPS, false, PER_SIMD>, blocks, kThreads, a, stream);
}

// The narrowest tile that has a whole row, 32 rows high for few frames, when a frame's time is a chain of parts of k, and else as high as
// registers allow, since w is read once per tile.  Up to 256 classes the waves of a high tile have 32 rows each; else they lie
// side by side.  us at k 512, 16 bits, low / high tiles, 129 classes: 16 frames 7.0 / 11.7, 4,096: 7.7 / 13.1, 16,384: 11.4 / 15.9,
// 118,000: 115 / 66; 256 classes: 8.5 / 17, 9.9 / 18, 19 / 21, 197 / 86; 500: 12 / 14, 15 / 17, 35 / 27; 1,000: 20 / 24, 24 / 29, 62 / 45.
// Behind 512 classes they go in groups: two of 512 up to 1,024; three of 384, the most that 64 rows leave registers for (of 512 they
// spill), up to 1,152; behind that four of 512 with 32 rows, which read w twice as often.  14,800 frames, 16 bits (fp32): 600 classes: 31 (116), in groups
// of 384: 35 (106); 1,000: 39 (147), 43 (149); 1,100: 48 (166), with 32 rows: 78 (227); 1,153: 83 (231); 1,536: 90 (257); 2,048: 113 (320).  8,192 frames of
// 1,100: 40, with 32 rows 43; 2,048 frames: 31 to 34 both ways.
template <class E> int run_loglikes(const LoglikesArgs &a, bool direct, void *stream) {
  const int64_t rows = (int64_t)a.seqs * a.frames;
  if (rows <= 8192) {
    if (a.v <= 64) return run_rows<E, 32, 64, 32, 32, 128, 4, 1, 1>(a, direct, stream);
    if (a.v <= 160) return run_rows<E, 32, 160, 32, 32, 64, 4, 1, 2>(a, direct, stream);
    if (a.v <= 256) return run_rows<E, 32, 256, 32, 32, 128, 4, 1, 2>(a, direct, stream);
  }
  if (rows <= 4096) {
    if (a.v <= 512) return run_rows<E, 32, 512, 32, 32, 64, 4, 1, 4>(a, direct, stream);
    if (a.v <= 1024) return run_rows<E, 32, 512, 32, 32, 64, 4, 2, 4>(a, direct, stream);
  }
  if (a.v <= 64) return run_rows<E, 128, 64, 32, 64, 64, 2, 1, 4>(a, direct, stream);
  if (a.v <= 160) return run_rows<E, 128, 160, 32, 160, 64, 2, 1, 3>(a, direct, stream);
  if (a.v <= 256) return run_rows<E, 128, 256, 32, 256, 64, 2, 1, 2>(a, direct, stream);
  if (a.v <= 512) return run_rows<E, 64, 512, 64, 64, 64, 2, 1, 4>(a, direct, stream);
  if (a.v <= 1024) return run_rows<E, 64, 512, 64, 64, 64, 4, 2, 2>(a, direct, stream);
  if (a.v <= 1152) return run_rows<E, 64, 384, 64, 32, 64, 4, 3, 3>(a, direct, stream);
  return run_rows<E, 32, 512, 32, 64, 64, 4, 4, 2>(a, direct, stream);
}

// Long rows are cut until there are about 1,024 workgroups, into 64 parts at most, and so that a part has more than about 1,000 scores (up to
// 64 parts: 2,048 at most, of 2,049 scores 1,032 and 1,017).
int row_splits(int64_t rows, int32_t v) {
  if (v <= kShortRow) return 1;
  const int64_t most = (v - 1) / 2048 + 1, want = (1024 - 1) / rows + 1;
  const int64_t n = want < most ? want : most;
  return (int)(n < 64 ? n : 64);
}

template <class E, int LANES, int EACH> int run_short(const LogprobsArgs &a, int64_t rows, void *stream) {
  // One after the other costs a reduction each; a bound and a sorted list cost as much as about six of them, over 64 lanes eight, whatever
  // the number, until most lanes' maxima are in the list.  fp32, us one after the other / by a bound: 118,417 rows of 129: top 4 29 / 31,
  // 6 39 / 33, 12 56 / 40, 16 67 / 69; 14,800 rows of 2,048: top 4 49 / 64, 8 69 / 65, 16 104 / 68, 48 250 / 88.
  const bool many = a.top >= (LANES == 16 ? 6 : 8) && a.top <= LANES * 3 / 4;
  return launch("wfst_token_logprobs", many ? logprobs_short_kernel<E, LANES, EACH, true> : logprobs_short_kernel<E, LANES, EACH, false>,
                (rows - 1) / (256 / LANES) + 1, 256, a, stream);
}

template <class E> int run_logprobs(LogprobsArgs a, void *stream) {
  const char *me = "wfst_token_logprobs";
  const int64_t rows = (int64_t)a.seqs * a.frames;
  if (a.v <= 64) return run_short<E, 16, 4>(a, rows, stream);
  if (a.v <= 160) return run_short<E, 16, 10>(a, rows, stream);
  if (a.v <= 256) return run_short<E, 16, 16>(a, rows, stream);
  if (a.v <= 512) return run_short<E, 64, 8>(a, rows, stream);
  if (a.v <= 1024) return run_short<E, 64, 16>(a, rows, stream);
  if (a.v <= kShortRow) return run_short<E, 64, 32>(a, rows, stream);
  a.splits = row_splits(rows, a.v);
  a.split_size = ((a.v - 1) / a.splits / 8 + 1) * 8;
  const int rc = launch(me, logprobs_long_kernel<E>, rows * a.splits, kLongThreads, a, stream);
  return rc != WFST_OK || a.splits == 1 ? rc : launch(me, logprobs_join_kernel<E>, rows, kLongThreads, a, stream);
}

template <class E> int run_backward(BackwardArgs a, void *stream) {
  const char *me = "wfst_token_logprobs_backward";
  const int64_t rows = (int64_t)a.seqs * a.frames;
  if (a.v <= 64) return launch(me, backward_short_kernel<E, 16, 4>, (rows - 1) / 16 + 1, 256, a, stream);
  if (a.v <= 160) return launch(me, backward_short_kernel<E, 16, 10>, (rows - 1) / 16 + 1, 256, a, stream);
  if (a.v <= 256) return launch(me, backward_short_kernel<E, 16, 16>, (rows - 1) / 16 + 1, 256, a, stream);
  if (a.v <= 512) return launch(me, backward_short_kernel<E, 64, 8>, (rows - 1) / 4 + 1, 256, a, stream);
  if (a.v <= 1024) return launch(me, backward_short_kernel<E, 64, 16>, (rows - 1) / 4 + 1, 256, a, stream);
  if (a.v <= kShortRow) return launch(me, backward_short_kernel<E, 64, 32>, (rows - 1) / 4 + 1, 256, a, stream);
  const int part = kLongThreads * kLongLoads * Chunk<E>::kN;
  a.splits = (a.v - 1) / part + 1;
  return launch(me, backward_long_kernel<E>, rows * a.splits, kLongThreads, a, stream);
}

}  // namespace

extern "C" {

int32_t wfst_linear(const wfst_linear_args *args, void *stream) {
  const char *me = "wfst_linear";
  if (!args) return refuse(me, "null argument");
  const wfst_linear_args &p = *args;
  if (!type_ok(p.dtype) || !type_ok(p.out_dtype) || (p.bias && !type_ok(p.bias_dtype))) return refuse(me, "unknown element type");
  if (p.activation < WFST_ACT_NONE || p.activation > WFST_ACT_GELU) return refuse(me, "unknown activation");
  if (p.rows < 0 || p.k < 1 || p.n < 1) return refuse(me, "rows must be >= 0, k and n >= 1");
  if (p.rows == 0) return WFST_OK;
  if (!p.x || !p.w || !p.y) return refuse(me, "null x, w or y");
  if (p.x_stride < 0 || p.w_stride < 0) return refuse(me, "negative stride");
  if (!rows_apart(1, p.rows, p.n, 0, p.y_stride) || (p.residual && p.rows > 1 && p.residual_stride < p.n))
    return refuse(me, "y_stride and residual_stride must be >= n");
  const int64_t size = type_size(p.dtype), out_size = type_size(p.out_dtype);
  if (!aligned(p.x, size) || !aligned(p.w, size) || !aligned(p.y, out_size) || !aligned(p.residual, out_size) ||
      (p.bias && !aligned(p.bias, type_size(p.bias_dtype))))
    return refuse(me, "an address is not a multiple of its element's size");
  if (p.k > 1 << 28) return refuse(me, "k must be at most 2^28");
  const int64_t nx = span(1, p.rows, p.k, 0, p.x_stride, size), nw = span(1, p.n, p.k, 0, p.w_stride, size);
  const int64_t ny = span(1, p.rows, p.n, 0, p.y_stride, out_size), nr = p.residual ? span(1, p.rows, p.n, 0, p.residual_stride, out_size) : 0;
  if (nx < 0 || nw < 0 || ny < 0 || nr < 0) return refuse(me, "sizes and strides are too large");
  if (overlap(p.y, ny, p.x, nx) || overlap(p.y, ny, p.w, nw) || (p.bias && overlap(p.y, ny, p.bias, p.n * type_size(p.bias_dtype))))
    return refuse(me, "y overlaps what is read");
  if (overlap(p.y, ny, p.residual, nr) && !(p.residual == p.y && (p.residual_stride == p.y_stride || p.rows == 1)))
    return refuse(me, "y overlaps the residual without being it");
  // The stride of a single row is no one's promise: behind it a tile reads that row again, not what lies a stride further on.
  const int64_t x_stride = p.rows == 1 ? 0 : p.x_stride, w_stride = p.n == 1 ? 0 : p.w_stride;
  LinearArgs a{p.x, p.w, p.bias, p.residual, p.y, p.rows, x_stride, w_stride, p.residual_stride, p.y_stride,
               p.k, p.n, p.bias_dtype, p.out_dtype, p.activation, p.scale, 0};
  const bool direct = chunked(p.x, x_stride, p.k, size) && chunked(p.w, w_stride, p.k, size);
  return by_type(p.dtype, [&](auto e) { return run_linear<decltype(e)>(a, direct, stream); });
}

int32_t wfst_loglikes(const wfst_loglikes_args *args, void *stream) {
  const char *me = "wfst_loglikes";
  if (!args) return refuse(me, "null argument");
  const wfst_loglikes_args &p = *args;
  if (!type_ok(p.dtype) || !type_ok(p.out_dtype) || (p.bias && !type_ok(p.bias_dtype))) return refuse(me, "unknown element type");
  if (p.seqs < 0 || p.frames < 0 || p.k < 1) return refuse(me, "seqs and frames must be >= 0, k >= 1");
  if (p.v < 1 || p.v > 2048) return refuse(me, "v must be 1 to 2048");
  if (p.seqs == 0 || p.frames == 0) return WFST_OK;
  if (!p.x || !p.w || !p.out) return refuse(me, "null x, w or out");
  if (p.x_seq_stride < 0 || p.x_stride < 0 || p.w_stride < 0) return refuse(me, "negative stride");
  if (!rows_apart(p.seqs, p.frames, p.v, p.out_seq_stride, p.out_stride)) return refuse(me, "the rows of out overlap");
  const int64_t size = type_size(p.dtype), out_size = type_size(p.out_dtype);
  if (!aligned(p.x, size) || !aligned(p.w, size) || !aligned(p.out, out_size) || !aligned(p.log_prior, 4) || !aligned(p.lengths, 4) ||
      (p.bias && !aligned(p.bias, type_size(p.bias_dtype))))
    return refuse(me, "an address is not a multiple of its element's size");
  if (p.k > 1 << 28) return refuse(me, "k must be at most 2^28");
  if ((int64_t)p.seqs * p.frames > INT_MAX) return refuse(me, "more than 2^31 - 1 frames");
  const int64_t nx = span(p.seqs, p.frames, p.k, p.x_seq_stride, p.x_stride, size), nw = span(1, p.v, p.k, 0, p.w_stride, size);
  const int64_t no = span(p.seqs, p.frames, p.v, p.out_seq_stride, p.out_stride, out_size);
  if (nx < 0 || nw < 0 || no < 0) return refuse(me, "sizes and strides are too large");
  if (overlap(p.out, no, p.x, nx) || overlap(p.out, no, p.w, nw) || (p.bias && overlap(p.out, no, p.bias, p.v * type_size(p.bias_dtype))) ||
      overlap(p.out, no, p.log_prior, (int64_t)p.v * 4) || overlap(p.out, no, p.lengths, (int64_t)p.seqs * 4))
    return refuse(me, "out overlaps what is read");
  LoglikesArgs a{p.x, p.w, p.bias, p.log_prior, p.lengths, p.out, p.x_seq_stride, p.x_stride, p.w_stride, p.out_seq_stride, p.out_stride,
                 p.seqs, p.frames, p.k, p.v, p.bias_dtype, p.out_dtype};
  const bool direct = aligned(p.x, 16) && aligned(p.w, 16) && p.k * size % 16 == 0 && p.x_seq_stride * size % 16 == 0 && p.x_stride * size % 16 == 0 &&
                      p.w_stride * size % 16 == 0 && nx < INT_MAX - 1024 && nw < INT_MAX - 1024 && p.w_stride < (INT_MAX - 1024) / size / 2048;
  return by_type(p.dtype, [&](auto e) { return run_loglikes<decltype(e)>(a, direct, stream); });
}

int64_t wfst_token_logprobs_workspace(int64_t rows, int32_t v, int32_t top) {
  if (rows < 1 || v < 1 || top < 0) return 0;
  const int splits = row_splits(rows, v);
  return splits == 1 ? 0 : rows * splits * (16 + 8 * (int64_t)top);
}

int32_t wfst_token_logprobs(const wfst_token_logprobs_args *args, void *stream) {
  const char *me = "wfst_token_logprobs";
  if (!args) return refuse(me, "null argument");
  const wfst_token_logprobs_args &p = *args;
  if (!type_ok(p.dtype)) return refuse(me, "unknown element type");
  if (p.seqs < 0 || p.frames < 0) return refuse(me, "seqs and frames must be >= 0");
  if (p.v < 1 || p.v > (1 << 30)) return refuse(me, "v must be 1 to 2^30");
  if (p.given < 0 || p.given > kMaxGiven) return refuse(me, "given must be 0 to 256");
  if (p.top < 0 || p.top > kMaxTop || p.top > p.v) return refuse(me, "top must be 0 to 64, and at most v");
  if (p.seqs == 0 || p.frames == 0) return WFST_OK;
  if (!p.scores || (p.given && p.logprobs && !p.tokens)) return refuse(me, "null scores or tokens");
  if (p.seq_stride < 0 || p.stride < 0) return refuse(me, "negative stride");
  const int64_t size = type_size(p.dtype), rows = (int64_t)p.seqs * p.frames;
  if (rows > INT_MAX) return refuse(me, "more than 2^31 - 1 rows");
  if (!aligned(p.scores, size) || !aligned(p.tokens, 4) || !aligned(p.lengths, 4) || !aligned(p.logprobs, 4) || !aligned(p.lse, 4) ||
      !aligned(p.entropy, 4) || !aligned(p.maximum, 4) || !aligned(p.log_sum, 4) || !aligned(p.top_ids, 4) || !aligned(p.top_logprobs, 4))
    return refuse(me, "an address is not a multiple of its element's size");
  const int64_t need = wfst_token_logprobs_workspace(rows, p.v, p.top);
  if (need > 0 && (!p.workspace || p.workspace_bytes < need || !aligned(p.workspace, 16)))
    return refuse(me, "the workspace is missing, too small or not 16-byte aligned");
  const int64_t ns = span(p.seqs, p.frames, p.v, p.seq_stride, p.stride, size);
  if (ns < 0) return refuse(me, "sizes and strides are too large");
  struct Part { const void *p; int64_t n; };
  const Part read[] = {{p.scores, ns}, {p.tokens, rows * p.given * 4}, {p.lengths, (int64_t)p.seqs * 4}};
  const Part wrote[] = {{p.given ? p.logprobs : nullptr, rows * p.given * 4}, {p.lse, rows * 4}, {p.entropy, rows * 4}, {p.maximum, rows * 4}, {p.log_sum, rows * 4},
                        {p.top ? p.top_ids : nullptr, rows * p.top * 4}, {p.top ? p.top_logprobs : nullptr, rows * p.top * 4},
                        {p.workspace, need}};
  for (int i = 0; i < (int)(sizeof(wrote) / sizeof(Part)); ++i) {
    for (const Part &r : read)
      if (overlap(wrote[i].p, wrote[i].n, r.p, r.n)) return refuse(me, "an output overlaps what is read");
    for (int j = 0; j < i; ++j)
      if (overlap(wrote[i].p, wrote[i].n, wrote[j].p, wrote[j].n)) return refuse(me, "two outputs overlap");
  }
  LogprobsArgs a{p.scores, p.tokens, p.lengths, p.given ? p.logprobs : nullptr, p.lse, p.entropy, p.maximum, p.log_sum, p.top ? p.top_ids : nullptr,
                 p.top ? p.top_logprobs : nullptr, p.workspace, p.seq_stride, p.stride, p.seqs, p.frames, p.v, p.given, p.top, 1, 0};
  if (!a.top_ids && !a.top_logprobs) a.top = 0;
  return by_type(p.dtype, [&](auto e) { return run_logprobs<decltype(e)>(a, stream); });
}

int32_t wfst_token_logprobs_backward(const wfst_token_logprobs_backward_args *args, void *stream) {
  const char *me = "wfst_token_logprobs_backward";
  if (!args) return refuse(me, "null argument");
  const wfst_token_logprobs_backward_args &p = *args;
  if (!type_ok(p.dtype)) return refuse(me, "unknown element type");
  if (p.seqs < 0 || p.frames < 0) return refuse(me, "seqs and frames must be >= 0");
  if (p.v < 1 || p.v > (1 << 30)) return refuse(me, "v must be 1 to 2^30");
  if (p.given < 0 || p.given > kMaxGiven) return refuse(me, "given must be 0 to 256");
  if (p.top < 0 || p.top > kMaxTop || p.top > p.v) return refuse(me, "top must be 0 to 64, and at most v");
  if (p.seqs == 0 || p.frames == 0) return WFST_OK;
  if (!p.scores || !p.maximum || !p.log_sum || !p.grad_scores) return refuse(me, "null scores, maximum, log_sum or grad_scores");
  if (p.given && p.grad_logprobs && !p.tokens) return refuse(me, "grad_logprobs without tokens");
  if (p.grad_entropy && !p.entropy) return refuse(me, "grad_entropy without entropy");
  if (p.top && p.grad_top && !p.top_ids) return refuse(me, "grad_top without top_ids");
  if (p.seq_stride < 0 || p.stride < 0) return refuse(me, "negative stride");
  if (!rows_apart(p.seqs, p.frames, p.v, p.grad_seq_stride, p.grad_stride)) return refuse(me, "the rows of grad_scores overlap");
  const int64_t size = type_size(p.dtype), rows = (int64_t)p.seqs * p.frames;
  if (rows > INT_MAX) return refuse(me, "more than 2^31 - 1 rows");
  if (!aligned(p.scores, size) || !aligned(p.grad_scores, size) || !aligned(p.tokens, 4) || !aligned(p.lengths, 4) || !aligned(p.maximum, 4) || !aligned(p.log_sum, 4) ||
      !aligned(p.entropy, 4) || !aligned(p.top_ids, 4) || !aligned(p.grad_logprobs, 4) || !aligned(p.grad_lse, 4) ||
      !aligned(p.grad_entropy, 4) || !aligned(p.grad_top, 4))
    return refuse(me, "an address is not a multiple of its element's size");
  const int64_t ns = span(p.seqs, p.frames, p.v, p.seq_stride, p.stride, size);
  const int64_t ng = span(p.seqs, p.frames, p.v, p.grad_seq_stride, p.grad_stride, size);
  if (ns < 0 || ng < 0) return refuse(me, "sizes and strides are too large");
  const bool same = p.scores == p.grad_scores && (p.seqs == 1 || p.seq_stride == p.grad_seq_stride) && (p.frames == 1 || p.stride == p.grad_stride);
  if (!same && overlap(p.grad_scores, ng, p.scores, ns)) return refuse(me, "grad_scores overlaps the scores without being them");
  if (overlap(p.grad_scores, ng, p.tokens, rows * p.given * 4) || overlap(p.grad_scores, ng, p.lengths, (int64_t)p.seqs * 4) ||
      overlap(p.grad_scores, ng, p.maximum, rows * 4) || overlap(p.grad_scores, ng, p.log_sum, rows * 4) || overlap(p.grad_scores, ng, p.entropy, rows * 4) ||
      overlap(p.grad_scores, ng, p.top_ids, rows * p.top * 4) || overlap(p.grad_scores, ng, p.grad_logprobs, rows * p.given * 4) ||
      overlap(p.grad_scores, ng, p.grad_lse, rows * 4) || overlap(p.grad_scores, ng, p.grad_entropy, rows * 4) ||
      overlap(p.grad_scores, ng, p.grad_top, rows * p.top * 4))
    return refuse(me, "grad_scores overlaps what is read");
  BackwardArgs a{p.scores, p.tokens, p.lengths, p.maximum, p.log_sum, p.entropy, p.top_ids, p.grad_logprobs, p.grad_lse, p.grad_entropy, p.grad_top,
                 p.grad_scores, p.seq_stride, p.stride, p.grad_seq_stride, p.grad_stride, p.seqs, p.frames, p.v, p.given, p.top, 1};
  if (!a.grad_logprobs) a.given = 0;
  if (!a.grad_top) a.top = 0;
  return by_type(p.dtype, [&](auto e) { return run_backward<decltype(e)>(a, stream); });
}

}  // extern "C"
