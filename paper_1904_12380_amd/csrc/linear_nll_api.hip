// C ABI of the loss over a vocabulary: argument checks, workspace and launches.
// Declarations and contract: include/decoder_mi355x.h.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sm_decoder_host.hpp"
#include "sm_linear_nll.hpp"
#include "sm_linear_nll_launch.hpp"

namespace {

using namespace smx;
using namespace smx_host;

constexpr int64_t kTile = 256;  // all tiles' sizes divide it

// The product of `kind` for m x n entries of the result.
NllProduct product(int kind, int64_t m, int64_t n, int dtype) {
  return dtype == SOFTMAX_F32   ? nll_product_f32(kind, m, n)
         : dtype == SOFTMAX_F16 ? nll_product_f16(kind, m, n)
                                : nll_product_bf16(kind, m, n);
}

// The kernels' NllHead, places and tokens, and the packed rows.  Each starts on a
// 256-byte boundary: 128-byte rows of operands that straddle two lines of the L2 take
// two requests each.
constexpr int64_t kAlign = 256;

struct Room {
  int64_t place, token, packed, more;
};

Room room(int64_t rows, int64_t d, int size) {
  const int64_t padded = up_to(rows, kTile);
  Room r;
  r.place = kAlign;
  r.token = r.place + up_to(rows * 4, kAlign);
  r.packed = r.token + up_to(padded * static_cast<int64_t>(sizeof(NllToken)), kAlign);
  r.more = r.packed + up_to(padded * up_to(d * size, kLineBytes), kAlign);
  return r;
}
static_assert(sizeof(NllHead) <= kAlign, "the head's place");

// The piece of the vocabulary whose g is kept at a time: what fits kPieceBytes, in
// whole rounds of dweight's tiles over the CUs (8192 tokens x 50001 x 2048 of bf16: 8
// rounds in two equal pieces, 7 in pieces of 128 and 68 tiles of the vocabulary).
// Pieces of 128 MiB, which the last cache holds, were slower: 1215 against 1254
// TFLOP/s there.
constexpr int64_t kPieceBytes = int64_t(512) << 20;
constexpr int64_t kCus = 256;  // of MI355X: workspaces and orders of sums go by sizes alone

int64_t piece_of(int64_t rows, int64_t vocab, int64_t d, int size) {
  const int64_t most = std::clamp<int64_t>(kPieceBytes / size / up_to(rows, kTile) / kTile, 1, 4096);
  const int64_t tiles = ceil_div(vocab, kTile);
  if (tiles <= most) return tiles * kTile;
  const int64_t round = std::max<int64_t>(kCus / ceil_div(d, kTile), 1);
  return (most > round ? most - most % round : most) * kTile;
}

// Splits of the sums behind a product's tiles: as few as leave at most a tenth of the
// device idle, or else those that leave the least, with all workgroups that a CU holds
// (dx of 512 tokens x 50001 x 2048 of bf16: 208 us with one, 142 with two); a split has
// `least` stages or more.
int64_t splits_of(const NllProduct& p, int64_t m, int64_t n, int64_t k, int dtype,
                  int64_t least = 4) {
  const int64_t tiles = ceil_div(m, p.bm) * ceil_div(n, p.bn);
  const int64_t stages = ceil_div(k * dtype_size(dtype), kLineBytes);
  const int64_t most = std::clamp<int64_t>(stages / least, 1, 64);
  const int64_t slots = kCus * p.resident;
  int64_t best = 1;
  double full = 0.0;
  for (int64_t s = 1; s <= most && full < 0.9; ++s) {
    const double f = static_cast<double>(tiles * s) / (ceil_div(tiles * s, slots) * slots);
    if (f > full) {
      full = f;
      best = s;
    }
  }
  return best;
}

// Splits of d for the logits, the same in both passes, which form equal ones: of fp32,
// whose matrix ops take 16 times as long, where the tiles leave a quarter of the CUs
// without one.  16 stages each pay for the partial logits, or 8 where the tiles are very
// few (fp32 forward calls, not split and split: 30 tokens x 969 x 4096 171 and 31 us, 64 x
// 15000 x 1024 52 and 43; 256 x 3000 x 512 23 and 26 with 8 stages, not split now).
int64_t d_splits_of(int64_t rows, int64_t vocab, int64_t d, int dtype) {
  if (dtype != SOFTMAX_F32) return 1;
  const NllProduct p = nll_product_f32(kPartial, vocab, rows);
  const int64_t tiles = ceil_div(vocab, p.bm) * ceil_div(rows, p.bn);
  return tiles < kCus * 3 / 4 ? splits_of(p, vocab, rows, d, dtype, tiles < kCus / 4 ? 8 : 16) : 1;
}

int64_t logits_bytes(int64_t rows, int64_t vocab, int64_t splits) {
  return splits > 1 ? splits * up_to(rows, kTile) * up_to(vocab, kTile) * 4 : 0;
}

int64_t forward_bytes(int64_t rows, int64_t vocab, int64_t d, int dtype) {
  const int64_t padded = up_to(rows, kTile);
  const int64_t splits = d_splits_of(rows, vocab, d, dtype);
  const int64_t tiles = ceil_div(vocab, product(kLogits, vocab, rows, dtype).bm);
  return room(rows, d, dtype_size(dtype)).more +
         (splits > 1 ? logits_bytes(rows, vocab, splits) : padded * 4 + tiles * padded * 8);
}

// Of the pieces, in whole tiles, the first has `most` rows of the vocabulary.
struct Backward {
  int64_t g, rest, sums, w_sums, logits, end, piece, most, splits, w_splits, d_splits;
};

Backward backward_room(int64_t rows, int64_t vocab, int64_t d, int dtype) {
  const int size = dtype_size(dtype);
  const int64_t padded = up_to(rows, kTile);
  Backward b;
  b.piece = piece_of(rows, vocab, d, size);
  b.most = std::min(b.piece, vocab);
  b.splits = splits_of(product(kInput, d, rows, dtype), d, rows, b.most, dtype);
  // dweight is many tiles, but for a small vocabulary.  Those of fp32 take longer: splits
  // of 16 stages pay there up to a tile for each CU (4096 tokens x 256 x 2048 with
  // gradients, 128 tiles: 291 us, split 238).
  const NllProduct w = product(kWeight, d, b.most, dtype);
  const int64_t w_tiles = ceil_div(d, w.bm) * ceil_div(b.most, w.bn);
  b.w_splits = 1;
  if (w_tiles < kCus / 2) b.w_splits = splits_of(w, d, b.most, rows, dtype);
  else if (dtype == SOFTMAX_F32 && w_tiles < kCus) b.w_splits = splits_of(w, d, b.most, rows, dtype, 16);
  b.g = room(rows, d, size).more;
  b.rest = b.g + padded * b.piece * size;
  b.sums = b.rest + (size == 2 ? kTwoParts * b.piece * size : 0);
  b.w_sums = b.sums + b.splits * padded * up_to(d * size, kLineBytes) / size * 4;
  b.logits = b.w_sums + up_to(b.w_splits > 1 ? b.w_splits * b.piece * d * 4 : 0, kAlign);
  b.d_splits = d_splits_of(rows, vocab, d, dtype);
  b.end = b.logits + logits_bytes(rows, vocab, b.d_splits);
  return b;
}

// Workgroups of tiles of bm x bn, within what a launch takes.
bool sizes_ok(int64_t rows, int64_t vocab, int64_t d, int dtype) {
  if (dtype_size(dtype) == 0 || !count_ok(rows) || !count_ok(vocab) || !width_ok(d)) return false;
  const int64_t tile = dtype == SOFTMAX_F32 ? 128 : 256;
  const int64_t most = (int64_t(1) << 32) / (dtype == SOFTMAX_F32 ? 256 : 512);
  const int64_t t = ceil_div(rows, tile), v = ceil_div(vocab, tile), c = ceil_div(d, tile);
  return std::max({t * v, t * c, v * c}) < most - 64;
}

bool strides_ok(int64_t x_stride, int64_t w_stride) {
  return x_stride >= 0 && w_stride >= 0 && w_stride <= SOFTMAX_MAX_ROW_STRIDE;
}

void set_call(NllArgs* a, const void* x, int64_t x_stride, const void* weight, int64_t w_stride,
              const int64_t* labels, int64_t rows, int64_t vocab, int64_t d, int64_t ignore,
              int size, void* workspace) {
  const Room r = room(rows, d, size);
  char* const at = static_cast<char*>(workspace);
  a->x = x;
  a->x_pitch = x_stride * size;
  a->weight = weight;
  a->w_pitch = w_stride * size;
  a->labels = labels;
  a->ignore = ignore;
  a->rows = static_cast<int>(rows);
  a->vocab = static_cast<int>(vocab);
  a->d = static_cast<int>(d);
  a->padded_rows = static_cast<int>(up_to(rows, kTile));
  a->padded_d = static_cast<int>(up_to(d * size, kLineBytes) / size);
  a->padded_vocab = static_cast<int>(up_to(vocab, kTile));
  a->head = reinterpret_cast<NllHead*>(at);
  a->place = reinterpret_cast<int*>(at + r.place);
  a->token = reinterpret_cast<NllToken*>(at + r.token);
  a->packed = at + r.packed;
}

hipError_t start(const void* fn, int64_t x, int64_t y, int threads, void** args, hipStream_t s) {
  return hipLaunchKernel(fn, dim3(static_cast<uint32_t>(x), static_cast<uint32_t>(y)),
                         dim3(threads), args, 0, s);
}

template <bool BACK>
hipError_t pack(NllArgs* a, int dtype, hipStream_t stream) {
  // At most 1024 workgroups, since each counts the labels before its own.
  int each = static_cast<int>(up_to(std::max<int64_t>(ceil_div(a->rows, 1024), 1), kPackTokens));
  const void* fn = dtype == SOFTMAX_F32   ? reinterpret_cast<const void*>(&k_nll_pack<float, BACK>)
                   : dtype == SOFTMAX_F16 ? reinterpret_cast<const void*>(&k_nll_pack<f16, BACK>)
                                          : reinterpret_cast<const void*>(&k_nll_pack<bf16, BACK>);
  void* args[] = {a, &each};
  return start(fn, ceil_div(a->rows, each), 1, 256, args, stream);
}

// lse and loss from the tiles' statistics.  A launch of 2^32 threads or more wraps
// around without an error: 16 threads for each of at most 2^27 tokens at a time.
hipError_t join(NllArgs a, hipStream_t stream) {
  constexpr int64_t kMost = int64_t(1) << 27;
  const int64_t rows = a.rows;
  hipError_t e = hipSuccess;
  for (int64_t from = 0; from < rows && e == hipSuccess; from += kMost) {
    const int64_t some = std::min(rows - from, kMost);
    a.rows = static_cast<int>(some);
    void* args[] = {&a};
    e = start(reinterpret_cast<const void*>(&k_nll_join<16>), ceil_div(some, kJoinTokens), 1,
              16 * kJoinTokens, args, stream);
    a.place += some;
    a.loss += some;
    a.lse += some;
  }
  return e;
}

hipError_t multiply_tiles(const NllProduct& p, int64_t m, int64_t n, int64_t splits, NllArgs* a,
                          hipStream_t stream) {
  void* args[] = {a};
  return start(p.fn, up_to(ceil_div(m, p.bm) * ceil_div(n, p.bn), kXcds), splits, p.threads, args,
               stream);
}

}  // namespace

extern "C" {

SOFTMAX_API int64_t softmax_linear_nll_fwd_workspace(int64_t rows, int64_t vocab, int64_t d,
                                                     int dtype) {
  if (!sizes_ok(rows, vocab, d, dtype)) return -1;
  return rows == 0 || vocab == 0 ? 0 : forward_bytes(rows, vocab, d, dtype);
}

SOFTMAX_API int softmax_linear_nll_fwd(const void* x, int64_t x_stride, const void* weight,
                                       int64_t w_stride, const int64_t* labels, int64_t rows,
                                       int64_t vocab, int64_t d, int64_t ignore, int dtype,
                                       float* loss, float* lse, void* workspace,
                                       int64_t workspace_bytes, hipStream_t stream) {
  const int size = dtype_size(dtype);
  int64_t xb = 0, wb = 0;
  if (!sizes_ok(rows, vocab, d, dtype) || !strides_ok(x_stride, w_stride) ||
      !rows_ok(x, rows, x_stride, d, size, &xb) ||
      !rows_ok(weight, vocab, w_stride, d, size, &wb) || !aligned16(workspace))
    return SOFTMAX_ERR_INVALID_ARG;
  if (rows == 0) return SOFTMAX_OK;
  const int64_t need = forward_bytes(rows, vocab, d, dtype);
  if (vocab == 0 || workspace_bytes < need) return SOFTMAX_ERR_INVALID_ARG;
  const Range inputs[] = {{x, xb}, {weight, wb}, {labels, rows * 8}};
  const Range outputs[] = {{loss, rows * 4}, {lse, rows * 4}, {workspace, need}};
  const int rc = check_ranges(inputs, outputs);
  if (rc != SOFTMAX_OK) return rc;
  NllArgs a = {};
  set_call(&a, x, x_stride, weight, w_stride, labels, rows, vocab, d, ignore, size, workspace);
  a.loss = loss;
  a.lse = lse;
  const int64_t splits = d_splits_of(rows, vocab, d, dtype);
  if (splits > 1) {
    a.d_splits = static_cast<int>(splits);
    a.logits = reinterpret_cast<float*>(static_cast<char*>(workspace) + room(rows, d, size).more);
    hipError_t e = pack<false>(&a, dtype, stream);
    if (e == hipSuccess)
      e = multiply_tiles(nll_product_f32(kPartial, vocab, rows), vocab, rows, splits, &a, stream);
    void* args[] = {&a};
    if (e == hipSuccess)
      e = start(reinterpret_cast<const void*>(&k_nll_total<256>), rows, 1, 256, args, stream);
    return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
  }
  const NllProduct p = product(kLogits, vocab, rows, dtype);
  a.tiles = static_cast<int>(ceil_div(vocab, p.bm));
  a.at = reinterpret_cast<float*>(static_cast<char*>(workspace) + room(rows, d, size).more);
  a.part = reinterpret_cast<f32x2*>(a.at + a.padded_rows);
  a.piece = static_cast<int>(up_to(vocab, kTile));
  hipError_t e = pack<false>(&a, dtype, stream);
  if (e == hipSuccess) e = multiply_tiles(p, vocab, rows, 1, &a, stream);
  if (e == hipSuccess) e = join(a, stream);
  return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
}

SOFTMAX_API int64_t softmax_linear_nll_bwd_workspace(int64_t rows, int64_t vocab, int64_t d,
                                                     int dtype) {
  if (!sizes_ok(rows, vocab, d, dtype)) return -1;
  return rows == 0 || vocab == 0 ? 0 : backward_room(rows, vocab, d, dtype).end;
}

SOFTMAX_API int softmax_linear_nll_bwd(const float* dloss, const void* x, int64_t x_stride,
                                       const void* weight, int64_t w_stride,
                                       const int64_t* labels, int64_t rows, int64_t vocab,
                                       int64_t d, int64_t ignore, int dtype, const float* loss,
                                       const float* lse, void* dx, void* dweight,
                                       void* workspace, int64_t workspace_bytes,
                                       hipStream_t stream) {
  const int size = dtype_size(dtype);
  int64_t xb = 0, wb = 0;
  if (!sizes_ok(rows, vocab, d, dtype) || !strides_ok(x_stride, w_stride) ||
      !rows_ok(x, rows, x_stride, d, size, &xb) ||
      !rows_ok(weight, vocab, w_stride, d, size, &wb) || !aligned16(workspace) ||
      !aligned16(dx) || !aligned16(dweight))
    return SOFTMAX_ERR_INVALID_ARG;
  const bool some = rows > 0 && vocab > 0;
  if (rows > 0 && vocab == 0) return SOFTMAX_ERR_INVALID_ARG;
  if (rows == 0 && (vocab == 0 || dweight == nullptr)) return SOFTMAX_OK;
  const Backward b = some ? backward_room(rows, vocab, d, dtype) : Backward{};
  if (workspace_bytes < b.end) return SOFTMAX_ERR_INVALID_ARG;
  const Range inputs[] = {{dloss, rows * 4}, {x, xb},       {weight, wb}, {labels, rows * 8},
                          {loss, rows * 4},  {lse, rows * 4}};
  const Range outputs[] = {{dx, dx ? rows * d * size : 0},
                           {dweight, dweight ? vocab * d * size : 0},
                           {workspace, b.end}};
  const int rc = check_ranges(inputs, outputs);
  if (rc != SOFTMAX_OK) return rc;
  if (!some) {
    // No rows: the sums over them are zeros.
    uint4* out = static_cast<uint4*>(dweight);
    int64_t strips = vocab * d * size / 16;
    void* args[] = {&out, &strips};
    const hipError_t e = start(reinterpret_cast<const void*>(&k_nll_clear<0>),
                               std::min<int64_t>(ceil_div(strips, 256), 2048), 1, 256, args, stream);
    return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
  }
  NllArgs a = {};
  set_call(&a, x, x_stride, weight, w_stride, labels, rows, vocab, d, ignore, size, workspace);
  a.dloss = dloss;
  a.loss = const_cast<float*>(loss);
  a.lse = const_cast<float*>(lse);
  a.dx = dx;
  a.dweight = dweight;
  a.g = static_cast<char*>(workspace) + b.g;
  a.g_rest = static_cast<char*>(workspace) + b.rest;
  a.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + b.sums);
  a.w_sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + b.w_sums);
  a.logits = reinterpret_cast<float*>(static_cast<char*>(workspace) + b.logits);
  a.d_splits = static_cast<int>(b.d_splits);
  a.piece = static_cast<int>(b.piece);
  a.splits = static_cast<int>(b.splits);
  a.w_splits = static_cast<int>(b.w_splits);
  if (dx == nullptr && dweight == nullptr) return SOFTMAX_OK;
  hipError_t e = pack<true>(&a, dtype, stream);
  void* args[] = {&a};
  for (int64_t from = 0; from < vocab && e == hipSuccess; from += b.piece) {
    a.from = static_cast<int>(from);
    const int64_t left = std::min(vocab - from, b.piece);
    if (b.d_splits > 1) {  // few tiles are one piece
      e = multiply_tiles(nll_product_f32(kPartial, vocab, rows), vocab, rows, b.d_splits, &a, stream);
      if (e == hipSuccess)
        e = start(reinterpret_cast<const void*>(&k_nll_grad<256>),
                  std::min<int64_t>(ceil_div(rows * ceil_div(vocab, 4), 256), 16 * kCus), 1, 256,
                  args, stream);
    } else {
      e = multiply_tiles(product(kProbs, b.most, rows, dtype), left, rows, 1, &a, stream);
    }
    if (e == hipSuccess && dx != nullptr)
      e = multiply_tiles(product(kInput, d, rows, dtype), d, rows, b.splits, &a, stream);
    if (e == hipSuccess && dweight != nullptr)
      e = multiply_tiles(product(kWeight, d, b.most, dtype), d, left, b.w_splits, &a, stream);
    if (e == hipSuccess && dweight != nullptr && b.w_splits > 1) {
      const void* fn = dtype == SOFTMAX_F32 ? reinterpret_cast<const void*>(&k_nll_weight<float>)
                       : dtype == SOFTMAX_F16 ? reinterpret_cast<const void*>(&k_nll_weight<f16>)
                                              : reinterpret_cast<const void*>(&k_nll_weight<bf16>);
      e = start(fn, std::min<int64_t>(ceil_div(left * d / 4, 256), 16 * kCus), 1, 256, args,
                stream);
    }
  }
  if (e == hipSuccess && dx != nullptr) {
    const void* fn = dtype == SOFTMAX_F32   ? reinterpret_cast<const void*>(&k_nll_input<float>)
                     : dtype == SOFTMAX_F16 ? reinterpret_cast<const void*>(&k_nll_input<f16>)
                                            : reinterpret_cast<const void*>(&k_nll_input<bf16>);
    e = start(fn, std::min<int64_t>(ceil_div(rows * (d / 8), 256), 16 * kCus), 1, 256, args, stream);
  }
  return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
}

}  // extern "C"
