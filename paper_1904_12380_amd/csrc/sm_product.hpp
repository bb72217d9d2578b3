// Tiles of matrix products on the matrix cores, for operands of 16-bit types
// and fp32, as the loss over a vocabulary needs them (sm_linear_nll.hpp):
//
//     C[m][n] = sum_k A(m, k) B(n, k)
//
// of BM x BN by a workgroup of WM x WN wavefronts.  Either operand lies in
// memory with its k entries side by side ("by rows": row m holds k = 0, 1, ..)
// or with its m (n) entries side by side ("by columns": row k holds m = 0, 1,
// ..).  Stages of 128 bytes of k per row (64 entries of 16-bit types, 32 of
// fp32) go from memory to LDS without registers, STAGES - 1 of them ahead of
// the one that is multiplied.
//
// Operands of v_mfma_f32_32x32x16 (fp32: four v_mfma_f32_32x32x2): lane l holds
// row l % 32 and the eight entries 8 (l / 32) + j of a step's 16 (fp32: the four
// entries 4 (l / 32) + j of 8), which is one 16-byte chunk of a tile by rows.
// Tiles by columns give the same entries by the transposing reads
// (ds_read_b64_tr_b16), fp32 by single reads.  D: column (n) l % 32, rows (m)
// 8 (i / 4) + 4 (l / 32) + i % 4, so a lane holds four entries side by side.
//
// LDS holds rows in 16-byte chunks, chunk c of row r at place c ^ swz(r)
// (sm_heads_mfma.hpp): all reads are free of bank conflicts.
#pragma once

#include "sm_heads_mfma.hpp"

namespace smx {

constexpr int kLineBytes = 128;  // of k in a stage, per row
constexpr int kSteps = 4;        // of matrix ops in a stage

template <typename T>
struct Operand {
  typedef typename Vec8<T>::type type;
};
template <>
struct Operand<float> {
  typedef f32x4 type;
};

__device__ __forceinline__ f32x16 multiply(f16x8 a, f16x8 b, f32x16 c) { return mfma32(a, b, c); }
__device__ __forceinline__ f32x16 multiply(bf16x8 a, bf16x8 b, f32x16 c) { return mfma32(a, b, c); }
__device__ __forceinline__ f32x16 multiply(f32x4 a, f32x4 b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
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
  static constexpr int kK = kLineBytes / kSize;     // entries of k in a stage
  static constexpr int kBytes = LINES * kLineBytes;  // of a stage
  static constexpr int kLoads = kBytes / 1024 / WAVES;
  static constexpr int kRowBytes = BY_ROWS ? kLineBytes : LINES * kSize;
  static constexpr int kChunks = kRowBytes / 16;
  static constexpr int kRowsPer = 64 / kChunks;  // rows that a load of a wavefront moves
  static_assert(kBytes % (1024 * WAVES) == 0 && 64 % kChunks == 0, "whole loads");

  const char* base;       // of the stage to load next
  int64_t step;           // bytes from stage to stage
  unsigned off[kLoads];   // of each load's chunk from the base, or kFar
  int place;              // by rows: byte of the lane's chunk in its row; by columns: its row
  int read_at[BY_ROWS ? kSteps : LINES >= 128 || kSize == 4 ? 4 : 2][BY_ROWS || kSize == 4 ? 1 : 2];

  // Place of chunk 0 of row r (an exclusive or).
  __device__ __forceinline__ static constexpr int place_of(int r) {
    return BY_ROWS ? swz<64>(r) : kSize == 4 ? (r >> 2 & 1) << 3 : swz<LINES>(r);
  }

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
      const int row = (wave * kLoads + i) * kRowsPer + lane / kChunks;
      const int chunk = lane % kChunks ^ place_of(row);
      const bool there = BY_ROWS ? row < left : chunk * (16 / kSize) < left;
      off[i] = there ? static_cast<unsigned>(row * static_cast<int>(pitch) + 16 * chunk) : kFar;
    }
    place = wave * kLoads * kRowsPer + lane / kChunks;
  }

  // Loads the next stage into `lds`; `left` entries of k are there from it on.
  __device__ __forceinline__ void load(unsigned lds, int64_t left, int wave) {
    lds += wave * kLoads * 1024;
    if (left >= kK) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load_line(base, off[i], lds + i * 1024);
    } else {
      const int lane = static_cast<int>(__lane_id());
      const int some = left < 0 ? 0 : static_cast<int>(left);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = place + i * kRowsPer;
        const int at = BY_ROWS ? (lane % kChunks ^ place_of(row)) * (16 / kSize) : row;
        load_line(base, at < some ? off[i] : kFar, lds + i * 1024);
      }
    }
    base += step;
  }

  // Sets up the reads of the lines `first` (a multiple of 32) .. of the tile.
  __device__ __forceinline__ void reader(int first) {
    const int lane = static_cast<int>(__lane_id()), half = lane / 32, r = lane % 32;
    if constexpr (BY_ROWS) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        read_at[s][0] = (first + r) * kLineBytes + 16 * ((2 * s + half) ^ place_of(r));
    } else if constexpr (kSize == 4) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int col = first + 32 * t + r;
        read_at[t][0] = 4 * half * kRowBytes + 16 * (col / 4 ^ place_of(4 * half)) + 4 * (col % 4);
      }
    } else {
      const int i = lane % 16;
#pragma unroll
      for (int t = 0; t < (LINES >= 128 ? 4 : 2); ++t) {
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          const int row = 8 * half + 4 * hi + i / 4;
          const int chunk = (first + 32 * t) / 8 + 2 * (lane / 16 % 2) + i % 4 / 2;
          read_at[t][hi] = row * kRowBytes + 16 * (chunk ^ place_of(row)) + 8 * (i % 2);
        }
      }
    }
  }

  // The operand of step s for the lines 32 t .. of the reader's.
  __device__ __forceinline__ typename Operand<T>::type read(const char SMX_LDS* tile, int s,
                                                            int t) const {
    typedef typename Operand<T>::type V;
    if constexpr (BY_ROWS) {
      return *reinterpret_cast<const V SMX_LDS*>(tile + read_at[s][0] + 32 * t * kLineBytes);
    } else if constexpr (kSize == 4) {
      V v;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = *reinterpret_cast<const float SMX_LDS*>(tile + read_at[t][0] +
                                                       (8 * s + j) * kRowBytes);
      return v;
    } else {
      const char SMX_LDS* p = tile + 16 * s * kRowBytes;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 SMX_LDS*)(p + read_at[t][0]));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 SMX_LDS*)(p + read_at[t][1]));
      return __builtin_bit_cast(V, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// The products of a workgroup's tile over `k` entries: acc[i][j] of a wavefront
// are its rows (m) 32 i .. and columns (n) 32 j .. .
template <typename T, bool A_ROWS, bool B_ROWS, int BM, int BN, int WM, int WN, int STAGES>
struct Product {
  static constexpr int kWaves = WM * WN;
  static constexpr int kMT = BM / WM / 32, kNT = BN / WN / 32;
  typedef Side<T, A_ROWS, BM, kWaves> A;
  typedef Side<T, B_ROWS, BN, kWaves> B;
  static constexpr int kStageBytes = A::kBytes + B::kBytes;
  static constexpr int kLds = STAGES * kStageBytes;
  static constexpr int kLoads = A::kLoads + B::kLoads;
  static_assert(kLds <= 160 * 1024, "LDS of a CU");

  f32x16 acc[kMT][kNT];

  __device__ __forceinline__ void run(A& a, B& b, char SMX_LDS* lds, int64_t k, int wave) {
    const unsigned at = lds_offset(lds);
    auto load = [&](int64_t from, int buf) {
      a.load(at + buf * kStageBytes, k - from, wave);
      b.load(at + buf * kStageBytes + A::kBytes, k - from, wave);
    };
    a.reader(wave % WM * (BM / WM));
    b.reader(wave / WM * (BN / WN));
#pragma unroll
    for (int i = 0; i < kMT; ++i)
#pragma unroll
      for (int j = 0; j < kNT; ++j) acc[i][j] = f32x16{};
    int64_t from = 0;
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
      load(from, s);
      from += A::kK;
    }
    int buf = 0, next = STAGES - 1;
    // One barrier a stage: behind it the stage's loads have landed for every
    // wavefront, and all have read the stage before it, whose place the next
    // loads take.
    for (int64_t done = 0; done < k; done += A::kK) {
      staged_but<(STAGES - 2) * kLoads>();
      __builtin_amdgcn_s_barrier();
      load(from, next);
      from += A::kK;
      const char SMX_LDS* ta = lds + buf * kStageBytes;
      const char SMX_LDS* tb = ta + A::kBytes;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        typename Operand<T>::type x[kMT], y[kNT];
#pragma unroll
        for (int i = 0; i < kMT; ++i) x[i] = a.read(ta, s, i);
#pragma unroll
        for (int j = 0; j < kNT; ++j) y[j] = b.read(tb, s, j);
#pragma unroll
        for (int i = 0; i < kMT; ++i)
#pragma unroll
          for (int j = 0; j < kNT; ++j) acc[i][j] = multiply(x[i], y[j], acc[i][j]);
      }
      buf = buf + 1 == STAGES ? 0 : buf + 1;
      next = next + 1 == STAGES ? 0 : next + 1;
    }
    // The last loads (of nothing) have landed and all tiles have been read: the
    // LDS may be used again.
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
