// Multi-head attention of 16-bit types: the forward pass.
//
// Scores transposed, as in sm_heads_f32.hpp, on v_mfma_f32_32x32x16: lane l
// holds A at row l % 32, columns 8 (l / 32) + j, B likewise, and D at column
// l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4.  S^T = K Q^T then leaves a lane
// with one row's scores of half of the keys: the softmax is lane-local but for
// one exchange between the halves of the wavefront, and eight consecutive
// registers are the B operand of the value product O^T += V^T P^T over 16
// keys, in the order 4 (l / 32) + j % 4 + 8 (j / 4).  V^T in that order comes
// from row-major V in LDS by the transposing reads (ds_read_b64_tr_b16: 16
// lanes read 4 rows of 16 columns, and each gets one column).
//
// LDS holds rows of the padded head width in 16-byte chunks, chunk c of row r
// at place c ^ swz(r): reads of 16 rows at one chunk (K) and of 4 rows at 4
// consecutive chunks (V, transposed) then touch each of the 64 banks once.
// Tiles go from memory to LDS without registers.
//
// A tile of up to 32 rows (single tokens of grouped heads, ends of chunks) is
// taken by all four wavefronts over different keys; a larger one by one
// wavefront for each 32 rows, over the same keys.
#pragma once

#include "sm_heads.hpp"

namespace smx {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

template <typename T>
struct Vec8;
template <>
struct Vec8<f16> { typedef f16x8 type; };
template <>
struct Vec8<bf16> { typedef bf16x8 type; };

__device__ __forceinline__ f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

#define SMX_LDS __attribute__((address_space(3)))

// Rows of a workgroup's tile and keys of a staged one.
constexpr int kTileRows = 128;
constexpr int kTileKeys = 64;
constexpr int kTileThreads = 256;

// The swizzle of row r's chunks.  Rows of 256 bytes or more start at the same
// bank: 16 rows at one chunk need 16 places, and 4 rows at 4 consecutive chunks
// 4 places that lie 64 bytes apart.  Of rows of 128 bytes two share the banks.
// swz(a ^ b) = swz(a) ^ swz(b).
template <int DP>
__host__ __device__ constexpr int swz(int r) {
  return DP >= 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
}
// Bytes of a row over which places are permuted.
template <int DP>
constexpr int kSwzSpan = DP >= 128 ? 256 : 128;

// LDS of one workgroup: two stages of kTileKeys rows of K and V.
template <int DP>
constexpr int tile_lds_bytes() { return 2 * 2 * kTileKeys * DP * 2; }

// 16 bytes of zeros for rows and columns that are not there.
__device__ const uint4 g_heads_zero = {0, 0, 0, 0};

constexpr unsigned kFar = 0x80000000u;  // past every buffer

// 16 bytes per lane from memory into LDS at `lds` (uniform) + 16 * lane.  In
// asm, since the compiler holds every later read of LDS back until such a load
// has landed; the kernels wait for a stage's loads themselves (staged()) and
// put a barrier between a stage's last read and its next load.  Nor does it see
// what the asm reads: the hardware needs five wait states between a vector
// instruction's write of a scalar register and a load whose resource holds it, and
// one after m0's, and checks neither, so they are a part of the asm.
typedef int s32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void load_lds(s32x4 rsrc, unsigned off, unsigned lds) {
  lds = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :
               : "v"(off), "s"(rsrc), "s"(lds)
               : "memory");
}
__device__ __forceinline__ void load_lds(const char* p, unsigned lds) {
  lds = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(p), "s"(lds)
               : "memory");
}
__device__ __forceinline__ unsigned lds_offset(const char SMX_LDS* p) {
  return static_cast<unsigned>(reinterpret_cast<uintptr_t>(p));
}
// Waits for all loads of this wavefront (vmcnt(0)), in a form that tells the
// compiler that its own have landed too: it would wait for them later, behind
// the next stage's.
__device__ __forceinline__ void staged() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70);
  asm volatile("" ::: "memory");
}
// Waits for all but this wavefront's last N loads.
template <int N>
__device__ __forceinline__ void staged_but() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
  asm volatile("" ::: "memory");
}
// Waits for this wavefront's reads of LDS (lgkmcnt(0)).
__device__ __forceinline__ void lds_read() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  asm volatile("" ::: "memory");
}

// Where keys lie: in packed tensors; in cache blocks of at least kGroup rows,
// so that the rows that one wavefront stages for a group share a block; in
// smaller blocks, where every lane looks its row's block up.
constexpr int kPacked = 0, kBlocks = 1, kSmallBlocks = 2;
constexpr int kGroup = 16;

// What stages rows from memory into LDS.  A wavefront's instruction moves 64
// chunks of 16 bytes: kRows rows, lane l the chunk at place l % kChunks of row
// l / kChunks.
template <int DP>
struct Stager {
  static constexpr int kChunks = DP / 8;
  static constexpr int kRows = 64 / kChunks;  // per instruction

  const char* base;   // row 0 of the head (packed: of the document)
  int64_t ts2, bs2;   // bytes between rows and between blocks
  int lane_row, lane_chunk;

  __device__ __forceinline__ Stager(const HeadsView& v, int64_t bs, int64_t first, int hk) {
    ts2 = v.ts * 2;
    bs2 = bs * 2;
    base = static_cast<const char*>(v.data) + first * ts2 + hk * v.hs * 2;
    const int lane = static_cast<int>(__lane_id());
    lane_row = lane / kChunks;
    lane_chunk = (lane % kChunks) ^ swz<DP>(lane_row);
  }

  // Column byte of the lane's chunk for the instruction whose first row has
  // the low bits `low`.
  __device__ __forceinline__ int column(int low) const {
    return 16 * (lane_chunk ^ swz<DP>(low));
  }

  // N instructions' rows from `at` on into lds (uniform, a row with the low
  // bits `low`), of which `bytes` are there: zeros past them and past column d.  Each instruction has a buffer
  // of its own, from its first row on, so that all share the lanes' offsets:
  // as offsets from one buffer they would take a register each, held across
  // the loop.
  template <int N>
  __device__ __forceinline__ void rows(const char* at, int bytes, char SMX_LDS* lds, int d2,
                                       int low = 0) const {
    const int step = static_cast<int>(ts2);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int skip = n * kRows * step;
      const uint64_t p = reinterpret_cast<uint64_t>(at + skip);
      // Uniform, also where the compiler does not see it.
      const s32x4 rsrc = {__builtin_amdgcn_readfirstlane(static_cast<int>(p)),
                          __builtin_amdgcn_readfirstlane(static_cast<int>(p >> 32 & 0xffff)),
                          __builtin_amdgcn_readfirstlane(max(bytes - skip, 0)), 0x00027000};
      const int col = column(n * kRows) ^ 16 * swz<DP>(low);
      const unsigned off = col < d2 ? lane_row * step + col : kFar;
      load_lds(rsrc, off, lds_offset(lds) + n * 1024);
    }
  }

  // Rows j, j + 1, .. of packed keys that end at `end`.
  template <int N>
  __device__ __forceinline__ void packed(char SMX_LDS* lds, int j, int end, int d2,
                                         int low = 0) const {
    const int64_t left = end - 1 - j;
    const int64_t bytes = left < 0 ? 0 : left * ts2 + d2;
    rows<N>(base + j * ts2, static_cast<int>(bytes < 0x7fffffff ? bytes : 0x7fffffff), lds, d2,
            low);
  }
};

// Keys of one request or document as a wavefront stages them, in groups of
// kGroup rows.  For blocks, the ids of the groups to stage next are looked up
// a stage ahead.
template <int DP, int WHERE, int GROUPS>
struct KeySource {
  static constexpr int kRows = Stager<DP>::kRows;
  static constexpr int kPer = kGroup / kRows;  // instructions of a group
  Stager<DP> k, v;
  int end, d2;
  const int* table;
  int ids[WHERE == kSmallBlocks ? GROUPS * kPer : GROUPS];

  __device__ __forceinline__ KeySource(const HeadsArgs& a, const DocTile& w, int hk, int to)
      : k(a.k, a.k_bs, w.k0, hk), v(a.v, a.v_bs, w.k0, hk), end(to), d2(2 * a.d) {
    table = WHERE == kPacked ? nullptr : a.table + static_cast<int64_t>(w.b) * a.width;
  }

  // Looks the blocks of rows j .. up: -1 past the end and outside the cache.
  __device__ __forceinline__ void look_up(const HeadsArgs& a, int j) {
    if constexpr (WHERE == kBlocks) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int at = j + g * kGroup;
        int id = -1;
        if (at < end) id = table[at >> a.log_block];
        ids[g] = static_cast<unsigned>(id) < static_cast<uint64_t>(a.blocks) ? id : -1;
      }
    } else if constexpr (WHERE == kSmallBlocks) {
#pragma unroll
      for (int n = 0; n < GROUPS * kPer; ++n) {
        const int at = j + n * kRows + k.lane_row;
        int id = -1;
        if (at < end) id = table[at >> a.log_block];
        ids[n] = static_cast<unsigned>(id) < static_cast<uint64_t>(a.blocks) ? id : -1;
      }
    }
  }

  // Rows of the groups that were looked up and are not there, a bit each.
  __device__ __forceinline__ unsigned absent() const {
    unsigned mask = 0;
    if constexpr (WHERE == kBlocks) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g)
        if (ids[g] < 0) mask |= 0xffffu << (g * kGroup);
    } else if constexpr (WHERE == kSmallBlocks) {
#pragma unroll
      for (int n = 0; n < GROUPS * kPer; ++n) {
        const uint64_t lanes = __ballot(ids[n] < 0);
#pragma unroll
        for (int r = 0; r < kRows; ++r)
          mask |= static_cast<unsigned>(lanes >> (r * Stager<DP>::kChunks) & 1)
                  << (n * kRows + r);
      }
    }
    return mask;
  }

  // Rows j .. (looked up before) of K or V.
  __device__ __forceinline__ void stage(const HeadsArgs& a, const Stager<DP>& s,
                                        char SMX_LDS* lds, int j) const {
    if constexpr (WHERE == kPacked) {
      s.template packed<GROUPS * kPer>(lds, j, end, d2);
    } else if constexpr (WHERE == kBlocks) {
      const int mask = (1 << a.log_block) - 1;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int at = j + g * kGroup;
        const int count = ids[g] < 0 ? 0 : min(end - at, kGroup);
        const char* p = s.base + static_cast<int64_t>(max(ids[g], 0)) * s.bs2 +
                        static_cast<int64_t>(at & mask) * s.ts2;
        s.template rows<kPer>(p, count > 0 ? (count - 1) * static_cast<int>(s.ts2) + d2 : 0,
                              lds + g * kGroup * DP * 2, d2);
      }
    } else {
      const int mask = (1 << a.log_block) - 1;
#pragma unroll
      for (int n = 0; n < GROUPS * kPer; ++n) {
        const int at = j + n * kRows + s.lane_row;
        const int col = s.column(n * kRows);
        const char* p = s.base + static_cast<int64_t>(ids[n]) * s.bs2 +
                        static_cast<int64_t>(at & mask) * s.ts2 + col;
        if (ids[n] < 0 || col >= d2) p = reinterpret_cast<const char*>(&g_heads_zero);
        load_lds(p, lds_offset(lds) + n * 1024);
      }
    }
  }
};

// A wavefront's 32 rows from memory to lds, lane r's row at base + its offset in
// bytes (negative: a row of zeros), which whole chunks at a time: a lane's own
// loads of its row would take 32 bytes of each of 32 rows at once.
template <int DP>
__device__ __forceinline__ void stage_rows(const char* base, int64_t offset, char SMX_LDS* lds,
                                           int d2) {
  constexpr int kChunks = DP / 8, kRows = 64 / kChunks;
  const int lane = static_cast<int>(__lane_id()), row0 = lane / kChunks;
#pragma unroll
  for (int n = 0; n < 32 / kRows; ++n) {
    const int row = n * kRows + row0;
    const int col = 16 * (lane % kChunks ^ swz<DP>(row));
    const int64_t off = __shfl(offset, row);
    const char* p = base + off + col;
    if (off < 0 || col >= d2) p = reinterpret_cast<const char*>(&g_heads_zero);
    load_lds(p, lds_offset(lds) + n * 1024);
  }
}

// The lane's row of Q (or of dO) as the B operand of DP / 16 steps: columns 16 s + 8
// (l / 32) + j, 0 past d and for rows that are not there.
template <typename T, int DP>
__device__ __forceinline__ void load_operand(typename Vec8<T>::type (&r)[DP / 16], const T* row,
                                             bool valid, int half, int d) {
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    const int c = 16 * s + 8 * half;
    uint4 x = {0, 0, 0, 0};
    if (valid && c < d) x = *reinterpret_cast<const uint4*>(row + c);
    r[s] = __builtin_bit_cast(typename Vec8<T>::type, x);
  }
}

// x itself, as a value that the compiler cannot see through: what is built
// from it is built where it is used, not held in registers across a loop.
__device__ __forceinline__ int opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Reads of a staged tile: rows as they lie, and columns, transposed.
template <int DP>
struct TileReader {
  static constexpr int kSpan = kSwzSpan<DP>;
  int row_at;   // byte of row l % 32, chunk l / 32
  int col_at;   // byte of the transposed read at rows 4 (l / 32) .., column 0

  __device__ __forceinline__ TileReader() {
    const int lane = static_cast<int>(__lane_id()), half = lane / 32;
    const int r = lane % 32;
    row_at = r * DP * 2 + 16 * (half ^ swz<DP>(r));
    const int i = lane % 16, cr = 4 * half + i / 4;
    const int chunk = 2 * (lane / 16 % 2) + (i % 4) / 2;
    col_at = cr * DP * 2 + 16 * (chunk ^ swz<DP>(cr)) + 8 * (i % 2);
  }

  // The same reader with addresses built anew.
  __device__ __forceinline__ TileReader fresh() const {
    TileReader r = *this;
    r.row_at = opaque(row_at);
    r.col_at = opaque(col_at);
    return r;
  }

  // A operand: rows row0 + l % 32 (row0 a multiple of 32), columns of step s.
  template <typename T>
  __device__ __forceinline__ typename Vec8<T>::type rows(const char SMX_LDS* tile, int row0,
                                                         int s) const {
    typedef typename Vec8<T>::type V;
    return *reinterpret_cast<const V SMX_LDS*>(tile + row0 * DP * 2 + (row_at ^ 32 * s % kSpan) +
                                               32 * s / kSpan * kSpan);
  }

  // A operand: columns 32 t + l % 32 of the rows row0 + 4 (l / 32) + j % 4 + 8
  // (j / 4), row0 a multiple of 16.
  template <typename T>
  __device__ __forceinline__ typename Vec8<T>::type cols(const char SMX_LDS* tile, int row0,
                                                         int t) const {
    const char SMX_LDS* p = tile + row0 * DP * 2 + 64 * t / kSpan * kSpan;
    const int lo_at = col_at ^ 64 * t % kSpan, hi_at = lo_at ^ 16 * swz<DP>(8);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 SMX_LDS*)(p + lo_at));
    const s16x4 hi =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 SMX_LDS*)(p + 8 * DP * 2 + hi_at));
    const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(typename Vec8<T>::type, both);
  }
};

// Eight registers as a B operand, rounded to the type.
template <typename T>
__device__ __forceinline__ typename Vec8<T>::type pack8(const f32x16& x, int i0) {
  typename Vec8<T>::type r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = static_cast<T>(x[i0 + j]);
  return r;
}
// What that rounding left.
template <typename T>
__device__ __forceinline__ typename Vec8<T>::type pack8_rest(const f32x16& x, int i0,
                                                             typename Vec8<T>::type hi) {
  typename Vec8<T>::type r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = static_cast<T>(x[i0 + j] - static_cast<float>(hi[j]));
  return r;
}

// Orders a run of `reads` reads of LDS (`per` for each operand) and `ops`
// matrix ops that take them: AHEAD operands are read ahead, so that the reads'
// latency passes during earlier matrix ops.  (The compiler by itself waits for
// each read right before its use.)
template <int OPS, int PER, int AHEAD = 4>
__device__ __forceinline__ void interleave() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * PER, 0);
#pragma unroll
  for (int i = 0; i < OPS - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, PER, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
}

// How scores are formed (a template argument): scaled, with a bias, with a cap,
// or with both.
constexpr int kPlain = 0, kBias = 1, kCap = 2, kCapBias = 3;

// Scores in powers of two from dot products.  tanh(y) = 1 - 2 r with r = 1 /
// (e^2y + 1), so that the capped score is one fma of r, and the cap's
// derivative 1 - tanh^2 is 4 r (1 - r).  The difference is within 2e-7 of the
// cap, which the weights' rounding to 16 bits covers up to kWideCap; past it
// tanh is formed to 3e-7 of itself, from its series where it is small.
constexpr float kWideCap = 256.0f;

template <int MODE>
struct Scoring {
  float c;        // scale in powers of two (with a cap: of e^2y)
  float cap2;     // the cap in powers of two
  float slope2;   // the slope in powers of two
  bool wide;

  __device__ __forceinline__ Scoring(const HeadsArgs& a, float slope) {
    c = MODE == kPlain ? fabsf(a.scale) * kLog2eF
        : MODE == kBias ? a.scale * kLog2eF : a.scale * a.exp_cap;
    cap2 = a.cap * kLog2eF;
    slope2 = slope * kLog2eF;
    wide = a.cap > kWideCap;
  }

  // tanh(y) for e^2y = 2^z, as 1 - 2 r.  The series' next term is 62 / 2835 y^8,
  // 3e-7 at 1/4.
  __device__ __forceinline__ static float wide_r(float z) {
    const float y = z * (0.5f * kLn2F), s = y * y;
    const float series =
        y * __builtin_fmaf(
                s,
                __builtin_fmaf(s, __builtin_fmaf(s, -17.0f / 315.0f, 2.0f / 15.0f), -1.0f / 3.0f),
                1.0f);
    return fabsf(y) < 0.25f ? series
                            : 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(z) + 1.0f);
  }

  // 16 dot products of a lane to scores, register i at the distance dist + step *
  // (8 (i / 4) + i % 4); with a cap r[i] = 1 / (e^2y + 1).
  __device__ __forceinline__ void scores(f32x16& s, f32x16& r, float dist, float step) const {
    auto bias = [&](int i) {
      return -slope2 * fabsf(__builtin_fmaf(step, static_cast<float>(8 * (i / 4) + i % 4), dist));
    };
    if constexpr (MODE == kBias) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], c, bias(i));
    } else if (!wide) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        r[i] = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[i] * c) + 1.0f);
        s[i] = __builtin_fmaf(r[i], -2.0f * cap2, MODE == kCap ? cap2 : cap2 + bias(i));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float t = wide_r(s[i] * c);
        r[i] = 0.5f - 0.5f * t;
        s[i] = MODE == kCap ? t * cap2 : __builtin_fmaf(t, cap2, bias(i));
      }
    }
  }
  __device__ __forceinline__ static float derivative(float r) {
    return __builtin_fmaf(-4.0f * r, r, 4.0f * r);
  }
  // Powers of two per unit of what scores() (kPlain: the dot product) gives.
  __device__ __forceinline__ float unit() const { return MODE == kPlain ? c : 1.0f; }
};

// Scores below every real one, of keys that a row does not see: finite, so
// that products with the scale stay ordered.
constexpr float kUnseen = -3.0e38f;

// Weights are taken in two 16-bit parts for the first kTileKeys keys of a
// document (in tiles of up to 32 rows these are two wavefronts' first) where rows
// see at most this many keys.  The rule goes by place, not by weight: past it a
// weight is rounded to the type once, whatever its share of the row.
constexpr int kTwoPartKeys = 128;

// A running maximum is moved (and the sums rescaled) when a score passes it by
// kSlack powers of two: weights then stay below 2^kSlack, and most tiles rescale
// nothing.  For fp16 all weights and their sum are 2^kLift times as large, which
// puts its range around them: below 2^15.5, with 11 bits down to 2^-26 of the
// maximum's weight.  Thousands of keys of 2^-24 and less beside a large one would
// otherwise be rounded to denormal numbers or to 0.
template <typename T>
constexpr float kSlack = __is_same(T, f16) ? 3.5f : 8.0f;
template <typename T>
constexpr float kLift = __is_same(T, f16) ? 12.0f : 0.0f;

constexpr float kFarShift = 0x1p14f;

// One wavefront's state for 32 rows, a lane's row at l % 32.
template <typename T, int DP>
struct RowState {
  typename Vec8<T>::type q[DP / 16];
  f32x16 acc[DP / 32];
  float m, l;        // m in units of the scores, times c in powers of two
  float c;           // powers of two per unit of score
  int pos, lim;
  int lim_all, lim_any;  // keys that every row, and any row, of the wavefront sees
};

// Scores of KT * 32 keys from k0, staged at ktile, their softmax and the
// product with the values at vtile.  scored() runs when the keys have been
// read, ready() before the values are.
template <typename T, int DP, int MODE, int KT, typename F, typename G>
__device__ __forceinline__ void attend(const Scoring<MODE>& sc, RowState<T, DP>& w,
                                       const TileReader<DP>& rd, const char SMX_LDS* ktile,
                                       const char SMX_LDS* vtile, int k0, uint64_t absent,
                                       F scored, G ready) {
  typedef typename Vec8<T>::type V;
  const int half = static_cast<int>(__lane_id()) / 32;
  f32x16 s[KT] = {};
#pragma unroll
  for (int st = 0; st < DP / 16; ++st) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
      s[kt] = mfma32(rd.template rows<T>(ktile, 32 * kt, st), w.q[st], s[kt]);
  }
  interleave<KT * DP / 16, 1>();
  scored();
  if constexpr (MODE != kPlain) {
    const float dist = static_cast<float>(w.pos - k0 - 4 * half);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      f32x16 r;
      sc.scores(s[kt], r, dist - 32 * kt, -1.0f);
    }
  }
  if (k0 + 32 * KT > w.lim_all || absent != 0) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = 32 * kt + 8 * (i / 4) + 4 * half + i % 4;
        if (k0 + r >= w.lim || (absent >> r & 1)) s[kt][i] = kUnseen;
      }
  }
  float top = s[0][0];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kt][i]);
  top = fmaxf(top, half32_partner(top));
  if (__any((top - w.m) * w.c > kSlack<T>)) {
    const float next = fmaxf(top, w.m);
    const float alpha = __builtin_amdgcn_exp2f((w.m - next) * w.c);
    w.m = next;
    w.l *= alpha;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) w.acc[t] *= alpha;
  }
  // Past kFarShift the shift's own rounding would scale a row's weights by a part of
  // a power of two, and further on by several (past fp16's range from scores of
  // 10^7): differences are formed first there, which makes them exact.
  float shift = w.m > kUnseen ? kLift<T> - w.m * w.c : 0.0f;
  const bool far = fabsf(shift) > kFarShift;
  if (__any(far)) {  // other rows of the wavefront keep their bits
    const float base = far ? w.m : 0.0f;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kt][i] -= base;
    if (far) shift = kLift<T>;
  }
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    float part[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[kt][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][i], w.c, shift));
      part[i % 2] += s[kt][i];
    }
    w.l += part[0] + part[1];
  }
  ready();
  V p[2 * KT];
#pragma unroll
  for (int u = 0; u < 2 * KT; ++u) p[u] = pack8<T>(s[u / 2], 8 * (u % 2));
#pragma unroll
  for (int u = 0; u < 2 * KT; ++u)
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
      w.acc[t] = mfma32(rd.template cols<T>(vtile, 16 * u, t), p[u], w.acc[t]);
  interleave<2 * KT * DP / 32, 2>();
  // A document's first keys: what the weights' rounding left, where rows see
  // few keys to average it.
  if (k0 < kTileKeys && w.lim_all <= kTwoPartKeys) {
#pragma unroll
    for (int u = 0; u < 2 * KT; ++u) p[u] = pack8_rest<T>(s[u / 2], 8 * (u % 2), p[u]);
#pragma unroll
    for (int u = 0; u < 2 * KT; ++u)
#pragma unroll
      for (int t = 0; t < DP / 32; ++t)
        w.acc[t] = mfma32(rd.template cols<T>(vtile, 16 * u, t), p[u], w.acc[t]);
  }
}

// A wavefront's 32 rows, a lane's at l % 32 in acc (D of transposed products),
// times f: rounded, turned in LDS (32 * DP * 2 bytes of the wavefront's own) and
// written as whole rows, row r at base + index * d for lane r's index (-1: not
// written).  Straight from the lanes every store would write 16 bytes of each of
// 32 rows: 2.4 us of a workgroup's 10 at one or two key tiles.
template <typename T, int DP>
__device__ __forceinline__ void store_rows(char SMX_LDS* lds, const f32x16 (&acc)[DP / 32],
                                           float f, T* base, int index, int d) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  constexpr int kChunks = DP / 8, kRows = 64 / kChunks;
  const int lane = static_cast<int>(__lane_id()), half = lane / 32, r = lane % 32;
#pragma unroll
  for (int t = 0; t < DP / 32; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      t4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = static_cast<T>(acc[t][4 * i + j] * f);
      *(t4 SMX_LDS*)(lds + r * DP * 2 + 16 * ((4 * t + i) ^ swz<DP>(r)) + 8 * half) = x;
    }
  const int row0 = lane / kChunks, chunk = lane % kChunks;
#pragma unroll
  for (int n = 0; n < 32 / kRows; ++n) {
    const int row = n * kRows + row0;
    const s32x4 x =
        *(const s32x4 SMX_LDS*)(lds + row * DP * 2 + 16 * (chunk ^ swz<DP>(row)));
    const int at = __shfl(index, row);
    if (at >= 0 && 8 * chunk < d)
      *reinterpret_cast<s32x4*>(base + static_cast<int64_t>(at) * d + 8 * chunk) = x;
  }
}

// One pass over the keys with a running maximum and sum.  A chunk of 2048 tokens
// over 65536 keys (32 heads of 128 on 8, bf16, a bias): 2.5 ms, 855 TFLOP/s,
// where a product of 8192 x 8192 matrices reaches 1230 on this card: bound by
// the matrix ops and the exponentials between them, which take turns on a
// SIMD; two workgroups per CU let one's products run during the other's
// softmax.  64 single tokens over up to 8192 keys: 235 us, 4.9 TB/s, bound by
// memory.  16384 tokens of one document (16 heads of 128 on 2): 1.07 ms, 1030
// TFLOP/s.
//
// Weights are rounded to the type for the value product, which the matrix ops of
// 16-bit types ask for; their sum is taken before.  Against one rounding of the
// result in all, errors are 1.1 to 1.3 times as large by norm.
template <typename T, int DP, int WHERE, int MODE>
__global__ __launch_bounds__(kTileThreads, DP <= 128 ? 2 : 1) void k_heads_fwd(HeadsArgs a) {
  __shared__ __attribute__((aligned(16))) char lds_bytes[tile_lds_bytes<DP>()];
  // Rows of a stage that no block holds, a bit each, 16 from each wavefront.
  __shared__ __attribute__((aligned(8))) unsigned short absent_rows[2][4];
  constexpr bool PAGED = WHERE != kPacked;
  char SMX_LDS* lds = (char SMX_LDS*)lds_bytes;
  const int hk = blockIdx.x % a.kv_heads;
  const int slot = static_cast<int>(gridDim.x / a.kv_heads - 1 - blockIdx.x / a.kv_heads);
  const int split = blockIdx.y;
  const DocLanes docs = load_docs<PAGED>(a, threadIdx.x % 64);
  const int chunk = PAGED ? split_chunk<kTileRows>(a, docs) : 0;
  const DocTile w = find_tile<kTileRows, PAGED, false>(a, docs, slot);
  const int rows = w.lq * a.group;
  const int row0 = w.tile * kTileRows;
  if (row0 >= rows) return;
  const int tile_rows = min(rows - row0, kTileRows);
  const bool few = tile_rows <= 32;
  const int seen = keys_seen(a, w, (row0 + tile_rows - 1) / a.group);
  int from, to;
  if (!split_range(seen, chunk, split, &from, &to)) return;

  const int lane = threadIdx.x % 64, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int local = (few ? 0 : 32 * wave) + lane % 32;
  const bool valid = local < tile_rows;
  const int row = valid ? row0 + local : rows - 1;
  const int tok = row / a.group, head = hk * a.group + row % a.group;
  const int64_t token = w.q0 + tok;

  RowState<T, DP> st;
  st.pos = tok + w.lk - w.lq;
  st.lim = valid ? min(keys_seen(a, w, tok), to) : 0;
  {
    const int first = row0 + (few ? 0 : 32 * wave), last = min(rows, first + 32) - 1;
    const bool any = first < row0 + tile_rows;
    // Rows that are not there see nothing, but need no mask either.
    st.lim_all = any ? min(keys_seen(a, w, first / a.group), to) : 0;
    st.lim_any = any ? min(keys_seen(a, w, last / a.group), to) : 0;
  }
  const Scoring<MODE> sc(a, MODE != kPlain && a.slopes != nullptr ? a.slopes[head] : 0.0f);
  st.c = sc.unit();
  st.m = kUnseen;
  st.l = 0.0f;
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) st.acc[t] = f32x16{};

  const TileReader<DP> rd;
  constexpr int kRowBytes = DP * 2;
  // The wavefront's rows of Q, by way of its quarter of the second stage.
  auto load_q = [&] {
    char SMX_LDS* at = lds + tile_lds_bytes<DP>() / 2 + wave * 32 * kRowBytes;
    const int64_t offset = 2 * (token * a.q.ts + head * a.q.hs);
    stage_rows<DP>(static_cast<const char*>(a.q.data), valid ? offset : -1, at, 2 * a.d);
    return at;
  };
  auto read_q = [&](const char SMX_LDS* at) {
    staged();
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      st.q[i] = rd.template rows<T>(at, 0, i);
      if (MODE == kPlain && a.scale < 0.0f) st.q[i] = -st.q[i];  // the sign into q
    }
    lds_read();
  };

  if (!few) {
    constexpr int kTile = kTileKeys * kRowBytes;
    static_assert(kTileKeys == 4 * kGroup, "a group for each wavefront");
    KeySource<DP, WHERE, 1> keys(a, w, hk, to);
    const int r0 = wave * kGroup;
    auto stage = [&](int k0, int buf) {
      char SMX_LDS* kt = lds + buf * 2 * kTile + r0 * kRowBytes;
      keys.stage(a, keys.k, kt, k0 + r0);
      keys.stage(a, keys.v, kt + kTile, k0 + r0);
      if constexpr (PAGED) {
        absent_rows[buf][wave] = static_cast<unsigned short>(keys.absent());
        keys.look_up(a, k0 + kTileKeys + r0);
      }
    };
    if (from < to) {
      const char SMX_LDS* q = load_q();
      keys.look_up(a, from + r0);
      stage(from, 0);
      read_q(q);
    }
    int buf = 0;
    for (int k0 = from; k0 < to; k0 += kTileKeys, buf ^= 1) {
      staged();
      __syncthreads();
      uint64_t absent = 0;
      if constexpr (PAGED) {
        const uint2 m = *reinterpret_cast<const uint2*>(absent_rows[buf]);
        absent = static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(m.y)) << 32 |
                 static_cast<unsigned>(__builtin_amdgcn_readfirstlane(m.x));
      }
      if (k0 + kTileKeys < to) stage(k0 + kTileKeys, buf ^ 1);
      if (k0 < st.lim_any)
        attend<T, DP, MODE, 2>(sc, st, PAGED ? rd.fresh() : rd, lds + buf * 2 * kTile, lds + buf * 2 * kTile + kTile,
                               k0, absent, [] {}, [] {});
    }
  } else {
    constexpr int kKeys = 2 * kGroup;
    KeySource<DP, WHERE, 2> keys(a, w, hk, to);
    char SMX_LDS* kt = lds + wave * (2 * kKeys * kRowBytes);
    char SMX_LDS* vt = kt + kKeys * kRowBytes;
    // Each wavefront has one buffer for keys and one for values, and loads
    // each anew as soon as it has been read: the next keys during the softmax
    // and the value product, the next values during the next scores.  Loads
    // past the end read nothing, and keep the count of those in flight.
    constexpr int kLoads = 2 * KeySource<DP, WHERE, 2>::kPer;
    int k0 = from + wave * kKeys;
    unsigned absent = 0;
    if (k0 < to) {
      keys.look_up(a, k0);
      load_operand<T, DP>(st.q, static_cast<const T*>(a.q.data) + token * a.q.ts + head * a.q.hs,
                          valid, half, a.d);
      keys.stage(a, keys.k, kt, k0);
      keys.stage(a, keys.v, vt, k0);
      staged();  // q too
      if (MODE == kPlain && a.scale < 0.0f) {
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) st.q[i] = -st.q[i];
      }
      for (; k0 < to; k0 += 4 * kKeys) {
        const int next = k0 + 4 * kKeys;
        absent = keys.absent();
        if constexpr (WHERE != kSmallBlocks) {
          staged_but<kLoads>();
          attend<T, DP, MODE, 1>(
              sc, st, rd.fresh(), kt, vt, k0, absent,
              [&] {
                lds_read();
                keys.look_up(a, next);
                keys.stage(a, keys.k, kt, next);
              },
              [&] { staged_but<kLoads>(); });
          lds_read();
          keys.stage(a, keys.v, vt, next);
        } else {  // lanes look up blocks: loads between the stages' own
          staged();
          attend<T, DP, MODE, 1>(sc, st, rd.fresh(), kt, vt, k0, absent, [] {}, [] {});
          lds_read();
          keys.look_up(a, next);
          keys.stage(a, keys.k, kt, next);
          keys.stage(a, keys.v, vt, next);
        }
      }
      staged();
    }
  }

  float l = st.l + half32_partner(st.l);
  float m = st.m;
  if (few) {
    // Join the four wavefronts: maxima and sums, then the products, summed by
    // the wavefront that writes their columns.
    __syncthreads();
    float SMX_LDS* stat = (float SMX_LDS*)lds;
    if (half == 0) {
      stat[64 * wave + 2 * (lane % 32)] = m;
      stat[64 * wave + 2 * (lane % 32) + 1] = l;
    }
    __syncthreads();
    float top = kUnseen, sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, stat[64 * i + 2 * (lane % 32)]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      sum += stat[64 * i + 2 * (lane % 32) + 1] *
             __builtin_amdgcn_exp2f((stat[64 * i + 2 * (lane % 32)] - top) * st.c);
    const float alpha = __builtin_amdgcn_exp2f((m - top) * st.c);
    m = top;
    l = sum;
    __syncthreads();
    float SMX_LDS* part = (float SMX_LDS*)lds;  // [wave][column / 4][row][4]
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = st.acc[t][4 * i + j] * alpha;
        const int quad = 8 * t + 2 * i + half;
        *(f32x4 SMX_LDS*)(part + ((wave * (DP / 4) + quad) * 32 + lane % 32) * 4) = x;
      }
    __syncthreads();
    // Wavefront w's columns: the same places of each quarter of the columns.
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int quad = 8 * t + 2 * i + half;
        f32x4 x = {0, 0, 0, 0};
        if (i == wave)
#pragma unroll
          for (int o = 0; o < 4; ++o)
            x += *(const f32x4 SMX_LDS*)(part + ((o * (DP / 4) + quad) * 32 + lane % 32) * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) st.acc[t][4 * i + j] = x[j];
      }
  }
  const bool some = m > kUnseen;
  const int64_t out = token * a.heads + head;
  const bool writes_stats = valid && half == 0 && (!few || wave == 0);
  if (chunk > 0) {
    if (!valid) return;
    const int64_t at = split * static_cast<int64_t>(a.tokens_q) * a.heads + out;
    if (writes_stats)
      a.part_stat[at] = {some ? (m * st.c - kLift<T>) * kLn2F : -INFINITY, l,
                         split_count(seen, chunk), 0};
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = 32 * t + 8 * i + 4 * half;
        if (col < a.d && (!few || i == wave)) {
          f32x4 x;
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = st.acc[t][4 * i + j];
          *reinterpret_cast<f32x4*>(a.part_o + at * a.d + col) = x;
        }
      }
    return;
  }
  const float inv = some ? 1.0f / l : 0.0f;
  if (writes_stats && a.lse != nullptr)
    a.lse[out] = some ? (m * st.c + (__builtin_amdgcn_logf(l) - kLift<T>)) * kLn2F : lse_of_none(l);
  if (!few) {
    __syncthreads();  // the last tile has been read: its place turns the rows
    store_rows<T, DP>(lds + wave * 32 * kRowBytes, st.acc, inv, static_cast<T*>(a.out),
                      valid ? static_cast<int>(out) : -1, a.d);
    return;
  }
  if (!valid) return;
  T* o = static_cast<T*>(a.out) + out * a.d;
#pragma unroll
  for (int t = 0; t < DP / 32; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = 32 * t + 8 * i + 4 * half;
      if (col < a.d && i == wave) {
        typedef T t4 __attribute__((ext_vector_type(4)));
        t4 x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = static_cast<T>(st.acc[t][4 * i + j] * inv);
        *reinterpret_cast<t4*>(o + col) = x;
      }
    }
}

}  // namespace smx
