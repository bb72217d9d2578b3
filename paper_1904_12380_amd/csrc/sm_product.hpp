// Tiles of matrix products on the matrix cores, for operands of 16-bit types
// and fp32, as the loss over a vocabulary needs them (sm_linear_nll.hpp):
//
//     C[m][n] = sum_k A(m, k) B(n, k)
//
// of BM x BN by a workgroup of WM x WN wavefronts.  Either operand lies in
// memory with its k entries side by side ("by rows": row m holds k = 0, 1, ..)
// or with its m (n) entries side by side ("by columns": row k holds m = 0, 1,
// ..).  Stages of 128 bytes of k per row (64 entries of 16-bit types, 32 of
// fp32) go from memory to LDS without registers, STAGES of them at a time.
//
// Operands of v_mfma_f32_16x16x32 (fp32: four v_mfma_f32_16x16x4): lane l holds
// row l % 16 and the eight entries 8 (l / 16) + j of a step's 32 (fp32: the four
// entries 4 (l / 16) + j of 16), which is one 16-byte chunk of a tile by rows.
// Tiles by columns give the same entries by the transposing reads
// (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 columns, and each gets one
// column), fp32 by single reads.  D: column (n) l % 16, rows (m) 4 (l / 16) + i, so
// a lane holds four entries side by side.  On random data these operations draw
// less power than v_mfma_f32_32x32x16, and power sets the clock: from registers
// alone 2110 against 1880 TFLOP/s.
//
// A wavefront's load into LDS writes 1024 bytes side by side, a block: whole rows, in
// their order in memory.  Bank conflicts are avoided by which rows share a block, and
// by blocks that lie 1056 bytes apart (Side); a read's address is then one register
// and constants.
//
// What bounds the large tiles is power: on random values the clock is 1.8 to 2.0 GHz,
// with the matrix pipes busy 55 to 72% of the cycles, and the forward product of 4096 x
// 131072 x 4096 of bf16 runs at 1390 TFLOP/s (on zeros, at the full clock, 1700).
#pragma once

#include <utility>

#include "sm_heads_mfma.hpp"

namespace smx {

// f(0), .., f(N - 1) with constants: loops of this many matrix ops are past what the
// compiler unrolls.
template <int... I, typename F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unrolled(F f) {
  each_of(std::make_integer_sequence<int, N>{}, f);
}

constexpr int kLineBytes = 128;  // of k in a stage, per row

template <typename T>
struct Operand {
  typedef typename Vec8<T>::type type;
};
template <>
struct Operand<float> {
  typedef f32x4 type;
};

__device__ __forceinline__ f32x4 multiply(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// 16 bytes per lane from memory at the uniform `base` + `off` (kFar: zeros)
// into LDS at `lds` + 16 * lane (load_lds has the waits).
__device__ __forceinline__ void load_line(const char* base, unsigned off, unsigned lds) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  const s32x4 rsrc = {static_cast<int>(p), static_cast<int>(p >> 32 & 0xffff), 0x7fffffff,
                      0x00027000};
  load_lds(rsrc, off, lds);
}

// One operand of a workgroup's tile: LINES rows of m (n), staged by WAVES
// wavefronts and read by each of them from its own first row on.
template <typename T, bool BY_ROWS, int LINES, int WAVES>
struct Side {
  static constexpr int kSize = sizeof(T);
  static constexpr int kK = kLineBytes / kSize;  // entries of k in a stage
  static constexpr int kBlocks = LINES * kLineBytes / 1024;
  static constexpr int kLoads = kBlocks / WAVES;
  static constexpr int kRowBytes = BY_ROWS ? kLineBytes : LINES * kSize;
  static constexpr int kChunks = kRowBytes / 16;
  static constexpr int kRowsPer = 64 / kChunks;  // rows of a block
  static_assert(kBlocks % WAVES == 0 && 64 % kChunks == 0, "whole loads");
  static_assert(BY_ROWS ? LINES % 64 == 0 : kRowBytes == 512 || kRowBytes == 256,
                "known layouts");

  // Blocks.  The banks repeat every 256 bytes, of which 16 lanes' reads at a time may
  // touch each once, and the blocks' starts move by 32 bytes from one to the next.
  //   by rows      16 rows are read at once, the lanes' chunks even for the rows 0 .. 3
  //                and 12 .. 15 and odd for the others, or the other way round.  Rows
  //                2 b and 2 b + 1 of four such tiles make the block b of eight.
  //   by columns   16 bits: 32 bytes of the rows 0 .. 3 and 8 .. 11 are read at once,
  //                or of these rows + 4, + 16 or + 20.  A block has one (rows of 256
  //                bytes: two) of each.
  //                fp32: 64 bytes of the rows 0, 4, 8 and 12, or the next ones.  A
  //                block has two rows that follow each other, or all four between two
  //                of these.
  __host__ __device__ static constexpr int block_at(int n) { return 1056 * n; }
  static constexpr int kBytes = block_at(kBlocks);
  // Row j of block n.
  __device__ __forceinline__ static constexpr int row_of(int n, int j) {
    return BY_ROWS        ? n / 8 * 64 + j / 2 * 16 + n % 8 * 2 + j % 2
           : kSize == 4   ? (kRowsPer == 2 ? 2 * n + j : n % 2 * 16 + n / 2 * 4 + j)
           : kRowsPer == 2 ? n / 8 * 16 + n / 4 % 2 * 8 + n % 4 + 4 * j
                           : n / 8 * 32 + n / 4 % 2 * 8 + n % 4 + j % 2 * 4 + j / 2 * 16;
  }

  const char* base;       // of the stage to load next
  int64_t step;           // bytes from stage to stage
  unsigned off[kLoads];   // of each load's chunk from the base, or kFar
  bool whole;             // all of the next stage's k is there
  int some;               // or so many entries
  int read_at;

  // Lines `first` .. of a matrix at `data` of rows of `pitch` bytes, from k on;
  // `lines` of them are there (the others are taken as zeros).
  __device__ __forceinline__ Side(const void* data, int64_t pitch, int64_t first, int64_t lines,
                                  int64_t k, int wave) {
    base = static_cast<const char*>(data) +
           (BY_ROWS ? first * pitch + k * kSize : k * pitch + first * kSize);
    step = BY_ROWS ? kLineBytes : kK * pitch;
    const int lane = static_cast<int>(__lane_id());
    const int64_t left = lines - first;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = row_of(wave * kLoads + i, lane / kChunks), chunk = lane % kChunks;
      const bool there = BY_ROWS ? row < left : chunk * (16 / kSize) < left;
      off[i] = there ? static_cast<unsigned>(row * static_cast<int>(pitch) + 16 * chunk) : kFar;
    }
  }

  // Entries of k that are there from the next stage on decide where its loads go:
  // ready() before the stage's loads, load() for each of them, then advance().
  __device__ __forceinline__ void ready(int64_t left) {
    whole = left >= kK;
    some = left < 0 ? 0 : static_cast<int>(left < kK ? left : kK);
  }
  __device__ __forceinline__ void load(unsigned lds, int i, int wave) const {
    unsigned o = off[i];
    if (!whole) {
      const int lane = static_cast<int>(__lane_id());
      const int at = BY_ROWS ? lane % kChunks * (16 / kSize)
                             : row_of(wave * kLoads + i, lane / kChunks);
      o = at < some ? o : kFar;
    }
    load_line(base, o, lds + block_at(wave * kLoads + i));
  }
  __device__ __forceinline__ void advance() { base += step; }

  // Sets up the reads of the lines `first` .. of the tile, a multiple of what the
  // wavefront takes.
  __device__ __forceinline__ void reader(int first) {
    const int lane = static_cast<int>(__lane_id()), q = lane / 16, r = lane % 16;
    if constexpr (BY_ROWS)
      read_at = block_at(first / 64 * 8 + r / 2) + (first % 64 / 8 + r % 2) * kLineBytes + 16 * q;
    else if constexpr (kSize == 4)
      read_at = block_at(2 * q) + (first + r) * 4;
    else  // 16 lanes read four rows of 32 bytes
      read_at = block_at(kRowsPer == 2 ? 4 * q + r / 4 : q % 2 * 4 + r / 4) +
                (kRowsPer == 2 ? 0 : q / 2 * 2 * kRowBytes) + first * 2 + r % 4 * 8;
  }

  // The operand of step s for the lines 16 t .. of the reader's.
  __device__ __forceinline__ typename Operand<T>::type read(const char SMX_LDS* tile, int s,
                                                            int t) const {
    typedef typename Operand<T>::type V;
    const char SMX_LDS* p = tile + read_at;
    if constexpr (BY_ROWS) {
      p += block_at(t / 4 * 8) + t % 4 * 2 * kLineBytes + 64 * s;
      return *reinterpret_cast<const V SMX_LDS*>(p);
    } else if constexpr (kSize == 4) {
      p += block_at(kRowsPer == 2 ? 8 * s : s) + 64 * t;
      V v;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = *reinterpret_cast<const float SMX_LDS*>(
            p + (kRowsPer == 2 ? block_at(j / 2) + j % 2 * kRowBytes : j * kRowBytes));
      return v;
    } else {
      p += block_at(kRowsPer == 2 ? 16 * s : 8 * s) + 32 * t;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 SMX_LDS*)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 SMX_LDS*)(p + kRowBytes));
      return __builtin_bit_cast(V, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// The products of a workgroup's tile over `k` entries: acc[i][j] of a wavefront
// are its rows (m) 16 i .. and columns (n) 16 j .. .
template <typename T, bool A_ROWS, bool B_ROWS, int BM, int BN, int WM, int WN, int STAGES>
struct Product {
  static constexpr int kWaves = WM * WN;
  static constexpr int kMT = BM / WM / 16, kNT = BN / WN / 16;
  typedef Side<T, A_ROWS, BM, kWaves> A;
  typedef Side<T, B_ROWS, BN, kWaves> B;
  static constexpr int kSteps = kLineBytes / 64;  // of a stage
  static constexpr int kStageBytes = A::kBytes + B::kBytes;
  static constexpr int kLds = STAGES * kStageBytes;
  static constexpr int kLoads = A::kLoads + B::kLoads;
  static_assert(kLds <= 160 * 1024, "LDS of a CU");
  // Tiles of 16 rows by rows lie four to a group of blocks.
  static_assert((BM / WM) % 64 == 0 || 64 % (BM / WM) == 0, "a wavefront's tiles, in groups");
  static_assert((BN / WN) % 64 == 0 || 64 % (BN / WN) == 0, "a wavefront's tiles, in groups");
  static_assert(kSteps == 2, "operands for each");

  f32x4 acc[kMT][kNT];

  typedef typename Operand<T>::type V;

  // The matrix ops of one step, and behind the n-th of them `then(n)`: what is read,
  // and loaded, for later steps.  In this order: the compiler by itself reads each
  // operand right before its use.
  template <int NT, typename F>
  __device__ __forceinline__ void step(const V (&x)[kMT], const V (&y)[NT], F then) {
    unrolled<kMT * NT>([&](auto n) {
      // Rows in turn from either end: one operand stays from op to op.
      constexpr int i = n / NT, j = i % 2 == 0 ? n % NT : NT - 1 - n % NT;
      acc[i][j] = multiply(x[i], y[j], acc[i][j]);
      then(n);
      __builtin_amdgcn_sched_barrier(0);
    });
  }

  __device__ __forceinline__ void clear() {
    unrolled<kMT * kNT>([&](auto n) { acc[n / kNT][n % kNT] = f32x4{}; });
  }

  // Adds the products of the next `k` entries of two operands, of the first NT of a
  // wavefront's kNT tiles of columns.
  template <int NT = kNT>
  __device__ __forceinline__ void run(A& a, B& b, char SMX_LDS* lds, int64_t k, int wave) {
    constexpr int kOps = kMT * NT;  // of a step
    const unsigned at = lds_offset(lds);
    int64_t left = k;  // from the next stage to load on
    auto load = [&](int n, int buf) {
      if (n < A::kLoads) a.load(at + buf * kStageBytes, n, wave);
      else b.load(at + buf * kStageBytes + A::kBytes, n - A::kLoads, wave);
    };
    auto ready = [&] {
      a.ready(left);
      b.ready(left);
      left -= A::kK;
    };
    auto advance = [&] {
      a.advance();
      b.advance();
    };
    a.reader(wave % WM * (BM / WM));
    b.reader(wave / WM * (BN / WN));
#pragma unroll
    for (int s = 0; s < STAGES; ++s) {
      ready();
#pragma unroll
      for (int n = 0; n < kLoads; ++n) load(n, s);
      advance();
    }
    staged_but<(STAGES - 1) * kLoads>();
    __builtin_amdgcn_s_barrier();
    V x[2][kMT], y[2][NT];
    const char SMX_LDS* tile = lds;
    // Operands of the next step are read between the first of a step's matrix ops: by
    // its end they have arrived, and nothing waits for them at the barrier.
    auto read = [&](auto n, int to, int s) {
      if constexpr (n < NT) y[to][n] = b.read(tile + A::kBytes, s, n);
      else if constexpr (n < NT + kMT) x[to][n - NT] = a.read(tile, s, n - NT);
    };
    unrolled<kMT + NT>([&](auto n) { read(n, 0, 0); });
    // The op that a read comes behind; a step of few ops takes several at once.
    auto read_at_op = [&](auto n, int to, int s) {
      unrolled<kMT + NT>([&](auto r) {
        if constexpr (n == r * kOps / (kMT + NT) * 3 / 4) read(r, to, s);
      });
    };
    int buf = 0;
    // A step's operands are read during the step before it, across stages too: the
    // last step of a stage runs behind the barrier, by which the next stage's loads
    // have landed for every wavefront, and all have read this one, whose place the
    // loads of the stage STAGES further on take.
    for (int64_t done = 0; done < k; done += A::kK) {
#pragma unroll
      for (int s = 0; s < kSteps - 1; ++s)
        step<NT>(x[s % 2], y[s % 2], [&](auto n) { read_at_op(n, (s + 1) % 2, s + 1); });
      const int next = buf + 1 == STAGES ? 0 : buf + 1;
      tile = lds + next * kStageBytes;
      lds_read();
      staged_but<(STAGES - 2) * kLoads>();
      __builtin_amdgcn_s_barrier();
      ready();
      step<NT>(x[(kSteps - 1) % 2], y[(kSteps - 1) % 2], [&](auto n) {
        read_at_op(n, kSteps % 2, 0);
        // Load l behind the op l kOps / kLoads + 2, or the last one.
        unrolled<kLoads>([&](auto l) {
          constexpr int at = l * kOps / kLoads + 2;
          if constexpr (n == (at < kOps ? at : kOps - 1)) load(l, buf);
        });
      });
      advance();
      buf = next;
    }
    // The last loads (of nothing) have landed and all tiles have been read: the
    // LDS may be used again.
    lds_read();
    staged();
    __builtin_amdgcn_s_barrier();
  }
};

// The tile of workgroup `id` among rows x cols tiles: each XCD takes a run of
// them (workgroups go to the eight XCDs in turn), in columns of kBand rows, so
// that the 32 workgroups that an XCD runs at a time share their operands in its
// L2.  False past the last one.
constexpr int kXcds = 8;
constexpr int kBand = 8;
__device__ __forceinline__ bool tile_of(int64_t id, int rows, int cols, int* row, int* col) {
  const int64_t all = static_cast<int64_t>(rows) * cols;
  const int64_t each = (all + kXcds - 1) / kXcds;
  const int64_t t = id % kXcds * each + id / kXcds;
  if (id / kXcds >= each || t >= all) return false;
  const int band = static_cast<int>(t / (static_cast<int64_t>(kBand) * cols));
  const int in = static_cast<int>(t - static_cast<int64_t>(band) * kBand * cols);
  const int high = min(kBand, rows - band * kBand);
  *row = band * kBand + in % high;
  *col = in / high;
  return true;
}

}  // namespace smx
