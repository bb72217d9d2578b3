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
// at place c ^ swz(r): reads of 8 rows at one chunk (K) and of 4 rows at 4
// consecutive chunks (V, transposed) then touch all banks.  Tiles go from
// memory to LDS without registers.
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

// The swizzle of row r's chunks: its low three bits, the lowest on top, so
// that neighbouring rows lie 64 bytes apart.  swz(a ^ b) = swz(a) ^ swz(b).
__host__ __device__ constexpr int swz(int r) { return (r & 1) << 2 | (r >> 1 & 3); }

// LDS of one workgroup: two stages of kTileKeys rows of K and V.
template <int DP>
constexpr int tile_lds_bytes() { return 2 * 2 * kTileKeys * DP * 2; }

// 16 bytes of zeros for rows and columns that are not there.
__device__ const uint4 g_heads_zero = {0, 0, 0, 0};

constexpr unsigned kFar = 0x80000000u;  // past every buffer

// 16 bytes per lane from memory into LDS at `lds` (uniform) + 16 * lane.  In
// asm, since the compiler holds every later read of LDS back until such a load
// has landed; the kernels wait for a stage's loads themselves (staged()) and
// put a barrier between a stage's last read and its next load.
typedef int s32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void load_lds(s32x4 rsrc, unsigned off, unsigned lds) {
  lds = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
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
// Waits for this wavefront's reads of LDS (lgkmcnt(0)).
__device__ __forceinline__ void lds_read() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  asm volatile("" ::: "memory");
}

// What stages rows of K or V from memory into LDS.  A wavefront's instruction
// moves 64 chunks of 16 bytes: kRows rows, lane l the chunk at place l % kChunks
// of row l / kChunks.
template <int DP, bool PAGED>
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
    lane_chunk = (lane % kChunks) ^ swz(lane_row);
  }

  // Column byte of the lane's chunk for the instruction whose first row has
  // the low bits `low` (a constant).
  __device__ __forceinline__ int column(int low) const { return 16 * (lane_chunk ^ swz(low)); }
};

// Rows [r0, r0 + N * kRows) of the packed keys k0 .. into lds (uniform), zeros
// past key `end` and past column d.  Each instruction has a buffer of its own,
// from its first row on, so that all share the lanes' offsets: as offsets from
// one buffer they would take a register each, held across the loop.
template <int DP, int N>
__device__ __forceinline__ void stage_packed(const Stager<DP, false>& s, char SMX_LDS* lds, int k0,
                                             int r0, int end, int d2) {
  constexpr int kRows = Stager<DP, false>::kRows;
  const int64_t left = end - 1 - k0;
  const int64_t bytes = left < 0 ? 0 : left * s.ts2 + d2;
  const int all = static_cast<int>(bytes < 0x7fffffff ? bytes : 0x7fffffff);
  const int step = static_cast<int>(s.ts2);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int skip = (r0 + n * kRows) * step;
    const uint64_t at = reinterpret_cast<uint64_t>(s.base + k0 * s.ts2 + skip);
    // Uniform, also where the compiler does not see it.
    const s32x4 rsrc = {__builtin_amdgcn_readfirstlane(static_cast<int>(at)),
                        __builtin_amdgcn_readfirstlane(static_cast<int>(at >> 32 & 0xffff)),
                        __builtin_amdgcn_readfirstlane(max(all - skip, 0)), 0x00027000};
    const int col = s.column(n * kRows);
    const unsigned off = col < d2 ? s.lane_row * step + col : kFar;
    load_lds(rsrc, off, lds_offset(lds) + n * 1024);
  }
}

// Block ids of the rows that a lane stages: rows r0 + n * kRows + lane_row of
// the keys k0 ..; -1 past `end` and for entries outside the cache.
template <int DP, int N>
__device__ __forceinline__ void page_ids(const HeadsArgs& a, const Stager<DP, true>& s, int b,
                                         int k0, int r0, int end, int (&ids)[N]) {
  const int* table = a.table + static_cast<int64_t>(b) * a.width;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int j = k0 + r0 + n * Stager<DP, true>::kRows + s.lane_row;
    int id = -1;
    if (j < end) id = table[j >> a.log_block];
    ids[n] = static_cast<unsigned>(id) < static_cast<uint64_t>(a.blocks) ? id : -1;
  }
}

template <int DP, int N>
__device__ __forceinline__ void stage_paged(const HeadsArgs& a, const Stager<DP, true>& s,
                                            char SMX_LDS* lds, int k0, int r0, int d2,
                                            const int (&ids)[N]) {
  const int mask = (1 << a.log_block) - 1;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int j = k0 + r0 + n * Stager<DP, true>::kRows + s.lane_row;
    const int col = s.column(n * Stager<DP, true>::kRows);
    const char* p = s.base + static_cast<int64_t>(ids[n]) * s.bs2 +
                    static_cast<int64_t>(j & mask) * s.ts2 + col;
    if (ids[n] < 0 || col >= d2) p = reinterpret_cast<const char*>(&g_heads_zero);
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

// Reads of a staged tile.  `rows`: chunk 2 s + l / 32 of row l % 32, at LDS
// bytes rows.at ^ (32 s); `cols`: transposed reads, of the columns 32 t.
template <int DP>
struct TileReader {
  int row_at;   // byte of row l % 32, chunk l / 32
  int col_at;   // byte of the transposed read at rows 4 (l / 32) .., column 0

  __device__ __forceinline__ TileReader() {
    const int lane = static_cast<int>(__lane_id()), half = lane / 32;
    const int r = lane % 32;
    row_at = r * DP * 2 + 16 * (half ^ swz(r));
    const int i = lane % 16, cr = 4 * half + i / 4;
    const int chunk = 2 * (lane / 16 % 2) + (i % 4) / 2;
    col_at = cr * DP * 2 + 16 * (chunk ^ swz(cr)) + 8 * (i % 2);
  }

  // The same reader with addresses built anew.
  __device__ __forceinline__ TileReader fresh() const {
    TileReader r = *this;
    r.row_at = opaque(row_at);
    r.col_at = opaque(col_at);
    return r;
  }

  // A operand: rows row0 + l % 32 (row0 a multiple of 8), columns of step s.
  template <typename T>
  __device__ __forceinline__ typename Vec8<T>::type rows(const char SMX_LDS* tile, int row0,
                                                         int s) const {
    typedef typename Vec8<T>::type V;
    return *reinterpret_cast<const V SMX_LDS*>(tile + row0 * DP * 2 + (row_at ^ (s % 4 * 32)) +
                                               s / 4 * 128);
  }

  // A operand: columns 32 t + l % 32 of the rows row0 + 4 (l / 32) + j % 4 + 8
  // (j / 4), row0 a multiple of 16.
  template <typename T>
  __device__ __forceinline__ typename Vec8<T>::type cols(const char SMX_LDS* tile, int row0,
                                                         int t) const {
    const char SMX_LDS* p = tile + row0 * DP * 2 + (col_at ^ (t % 2 * 64)) + t / 2 * 128;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 SMX_LDS*)(p));
    const s16x4 hi =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 SMX_LDS*)(p + 8 * DP * 2));
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

// The score of a dot product in units of 1 / log2 e, and the derivative of the
// cap.  tanh(y) = 1 - 2 / (e^2y + 1): within 2e-7, which the weights' rounding
// to 16 bits covers (up to caps of 1000).
__device__ __forceinline__ float score16(const HeadsArgs& a, float dot, float slope, int dist,
                                         float* dcap) {
  float x = dot * a.scale;
  *dcap = 1.0f;
  if (a.cap > 0.0f) {
    const float e = __builtin_amdgcn_exp2f(x * a.exp_cap);  // e^(2 x / cap)
    const float t = 1.0f - 2.0f * __builtin_amdgcn_rcpf(e + 1.0f);
    x = a.cap * t;
    *dcap = 1.0f - t * t;
  }
  return (x - slope * static_cast<float>(abs(dist))) * kLog2eF;
}

// Scores below every real one, of keys that a row does not see: finite, so
// that products with the scale stay ordered.
constexpr float kUnseen = -3.0e38f;

// A running maximum is moved (and the sums rescaled) when a score passes it by
// this many powers of two: weights then stay below 2^8, and most tiles
// rescale nothing.
constexpr float kSlack = 8.0f;

// One wavefront's state for 32 rows, a lane's row at l % 32.
template <typename T, int DP>
struct RowState {
  typename Vec8<T>::type q[DP / 16];
  f32x16 acc[DP / 32];
  float m, l;        // m in units of the scores, times c in powers of two
  float c;           // powers of two per unit of score
  float slope;
  int pos, lim;
  int lim_all, lim_any;  // keys that every row, and any row, of the wavefront sees
};

// Scores of KT * 32 keys from k0, staged at ktile, their softmax and the
// product with the values at vtile.
template <typename T, int DP, bool SCORED, int KT>
__device__ __forceinline__ void attend(const HeadsArgs& a, RowState<T, DP>& w,
                                       const TileReader<DP>& rd, const char SMX_LDS* ktile,
                                       const char SMX_LDS* vtile, int k0,
                                       uint64_t absent) {
  typedef typename Vec8<T>::type V;
  const int half = static_cast<int>(__lane_id()) / 32;
  f32x16 s[KT] = {};
#pragma unroll
  for (int st = 0; st < DP / 16; ++st) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
      s[kt] = mfma32(rd.template rows<T>(ktile, 32 * kt, st), w.q[st], s[kt]);
  }
  if constexpr (SCORED) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int j = k0 + 32 * kt + 8 * (i / 4) + 4 * half + i % 4;
        float dcap;
        s[kt][i] = score16(a, s[kt][i], w.slope, w.pos - j, &dcap);
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
  if (__any((top - w.m) * w.c > kSlack)) {
    const float next = fmaxf(top, w.m);
    const float alpha = __builtin_amdgcn_exp2f((w.m - next) * w.c);
    w.m = next;
    w.l *= alpha;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) w.acc[t] *= alpha;
  }
  const float shift = w.m > kUnseen ? -w.m * w.c : 0.0f;
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
  V p[2 * KT];
#pragma unroll
  for (int u = 0; u < 2 * KT; ++u) p[u] = pack8<T>(s[u / 2], 8 * (u % 2));
#pragma unroll
  for (int u = 0; u < 2 * KT; ++u)
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
      w.acc[t] = mfma32(rd.template cols<T>(vtile, 16 * u, t), p[u], w.acc[t]);
  if (k0 == 0) {  // a document's first keys: what the weights' rounding left
#pragma unroll
    for (int u = 0; u < 2 * KT; ++u) p[u] = pack8_rest<T>(s[u / 2], 8 * (u % 2), p[u]);
#pragma unroll
    for (int u = 0; u < 2 * KT; ++u)
#pragma unroll
      for (int t = 0; t < DP / 32; ++t)
        w.acc[t] = mfma32(rd.template cols<T>(vtile, 16 * u, t), p[u], w.acc[t]);
  }
}

template <typename T, int DP, bool PAGED, bool SCORED>
__global__ __launch_bounds__(kTileThreads, DP <= 128 ? 2 : 1) void k_heads_fwd(HeadsArgs a) {
  __shared__ __attribute__((aligned(16))) char lds_bytes[tile_lds_bytes<DP>()];
  char SMX_LDS* lds = (char SMX_LDS*)lds_bytes;
  const int hk = blockIdx.x % a.kv_heads;
  const int slot = static_cast<int>(gridDim.x / a.kv_heads - 1 - blockIdx.x / a.kv_heads);
  const int split = blockIdx.y;
  DocTile w;
  w.b = find_doc<kTileRows>(a.cu_q, a.n, a.tokens_q, a.group, slot, &w.tile);
  doc_queries(a, &w);
  doc_keys<PAGED>(a, &w);
  const int rows = w.lq * a.group;
  const int row0 = w.tile * kTileRows;
  if (row0 >= rows) return;
  const int chunk = PAGED ? split_chunk<kTileRows>(a) : 0;
  const int tile_rows = min(rows - row0, kTileRows);
  const bool few = tile_rows <= 32;
  int from, to;
  if (!split_range(keys_seen(a, w, (row0 + tile_rows - 1) / a.group), chunk, split, &from, &to))
    return;

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
  st.slope = SCORED && a.slopes != nullptr ? a.slopes[head] : 0.0f;
  st.c = SCORED ? 1.0f : fabsf(a.scale) * kLog2eF;
  st.m = kUnseen;
  st.l = 0.0f;
  load_operand<T, DP>(st.q, static_cast<const T*>(a.q.data) + token * a.q.ts + head * a.q.hs,
                      valid, half, a.d);
  if (!SCORED && a.scale < 0.0f) {  // the sign into q
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) st.q[i] = -st.q[i];
  }
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) st.acc[t] = f32x16{};

  const Stager<DP, PAGED> ks(a.k, a.k_bs, w.k0, hk), vs(a.v, a.v_bs, w.k0, hk);
  const TileReader<DP> rd;
  const int d2 = 2 * a.d;
  constexpr int kRowBytes = DP * 2;
  constexpr int kRows = Stager<DP, PAGED>::kRows;

  if (!few) {
    constexpr int kTile = kTileKeys * kRowBytes;
    constexpr int N = kTileKeys / 4 / kRows;  // instructions of a wavefront per tile
    const int r0 = wave * (kTileKeys / 4);
    int ids[N];
    if constexpr (PAGED) page_ids<DP, N>(a, ks, w.b, from, r0, to, ids);
    auto stage = [&](int k0, int buf) {
      char SMX_LDS* kt = lds + buf * 2 * kTile + r0 * kRowBytes;
      if constexpr (PAGED) {
        stage_paged<DP, N>(a, ks, kt, k0, r0, d2, ids);
        stage_paged<DP, N>(a, vs, kt + kTile, k0, r0, d2, ids);
      } else {
        stage_packed<DP, N>(ks, kt, k0, r0, to, d2);
        stage_packed<DP, N>(vs, kt + kTile, k0, r0, to, d2);
      }
    };
    if (from < to) stage(from, 0);
    int buf = 0;
    for (int k0 = from; k0 < to; k0 += kTileKeys, buf ^= 1) {
      // Rows of this tile that hold no key, from the table.
      uint64_t absent = 0;
      if constexpr (PAGED) {
        const int j = k0 + lane;
        int id = 0;
        if (j < to) id = a.table[static_cast<int64_t>(w.b) * a.width + (j >> a.log_block)];
        absent = __ballot(static_cast<unsigned>(id) >= static_cast<uint64_t>(a.blocks));
        page_ids<DP, N>(a, ks, w.b, k0 + kTileKeys, r0, to, ids);
      }
      staged();
      __syncthreads();
      if (k0 + kTileKeys < to) stage(k0 + kTileKeys, buf ^ 1);
      if (k0 < st.lim_any)
        attend<T, DP, SCORED, 2>(a, st, rd, lds + buf * 2 * kTile, lds + buf * 2 * kTile + kTile, k0,
                                 absent);
    }
  } else {
    constexpr int kKeys = 32;
    constexpr int N = kKeys / kRows;
    char SMX_LDS* kt = lds + wave * (2 * kKeys * kRowBytes);
    char SMX_LDS* vt = kt + kKeys * kRowBytes;
    int ids[N];
    auto stage = [&](const Stager<DP, PAGED>& s, char SMX_LDS* at, int k0) {
      if constexpr (PAGED)
        stage_paged<DP, N>(a, s, at, k0, 0, d2, ids);
      else
        stage_packed<DP, N>(s, at, k0, 0, to, d2);
    };
    int k0 = from + wave * kKeys;
    if constexpr (PAGED) page_ids<DP, N>(a, ks, w.b, k0, 0, to, ids);
    if (k0 < to) {
      stage(ks, kt, k0);
      stage(vs, vt, k0);
    }
    for (; k0 < to; k0 += 4 * kKeys) {
      uint64_t absent = 0;
      if constexpr (PAGED) {
        const int j = k0 + lane % 32;
        int id = 0;
        if (j < to) id = a.table[static_cast<int64_t>(w.b) * a.width + (j >> a.log_block)];
        absent = __ballot(static_cast<unsigned>(id) >= static_cast<uint64_t>(a.blocks)) &
                 0xffffffffu;
      }
      staged();
      attend<T, DP, SCORED, 1>(a, st, rd, kt, vt, k0, absent);
      const int next = k0 + 4 * kKeys;
      if constexpr (PAGED) page_ids<DP, N>(a, ks, w.b, next, 0, to, ids);
      lds_read();
      if (next < to) {
        stage(ks, kt, next);
        stage(vs, vt, next);
      }
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
  if (!valid) return;
  const bool some = m > kUnseen;
  const int64_t out = token * a.heads + head;
  const bool writes_stats = half == 0 && (!few || wave == 0);
  if (chunk > 0) {
    const int64_t at = split * static_cast<int64_t>(a.tokens_q) * a.heads + out;
    if (writes_stats) {
      a.part_ml[2 * at] = some ? m * st.c * kLn2F : -INFINITY;
      a.part_ml[2 * at + 1] = l;
    }
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
    a.lse[out] = some ? (m * st.c + __builtin_amdgcn_logf(l)) * kLn2F : -INFINITY;
  T* o = static_cast<T*>(a.out) + out * a.d;
#pragma unroll
  for (int t = 0; t < DP / 32; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = 32 * t + 8 * i + 4 * half;
      if (col < a.d && (!few || i == wave)) {
        typedef T t4 __attribute__((ext_vector_type(4)));
        t4 x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = static_cast<T>(st.acc[t][4 * i + j] * inv);
        *reinterpret_cast<t4*>(o + col) = x;
      }
    }
}

}  // namespace smx
