// Matrix products with a weight matrix for each group of rows (experts, or learners with
// batches of their own), groups of any size:
//   forward            y[t] = act(W_g x[t] + b_g)            t in [o_g, o_{g+1})
//   gradient of rows   dx[t] = (W_g^T dy[t]) [h[t] > 0]
//   gradient of weights dW_g = sum_t dy[t] x[t]^T,  db_g = sum_t dy[t]
//
// All three are D[128 features x up to 256 columns] tiles on tcgen05, the features (rows of
// the weights, or of dW) in the MMA's M and the ragged side where it costs nothing: for
// the first two the columns are a group's rows of x or dy, and the MMA's N is their count
// rounded up to 16; for the third the rows are what is summed over.  The offsets stay on
// the device: every CTA builds the list of tiles from them.
#include <algorithm>

#include "internal.h"
#include "op_common.cuh"
#include "ptx.cuh"

namespace ha {
namespace {

// A bounded wait of an operator's kernel that ran out (hier_avg_operator_check reads it).
__device__ int g_operator_error;

constexpr int kFwd = 0, kDx = 1, kDw = 2;
constexpr int kM = 128;                 // features of a CTA's tile
constexpr int kK = 64;                  // values summed over in a chunk: one 128-byte line
constexpr int kMaxGroups = 1024;
constexpr int kEpiWarps = 8;            // two groups of four: a group reads half the columns
constexpr int kThreads = (kEpiWarps + 2) * 32;          // results, loads, products
constexpr int kDwThreads = kThreads + 64;               // and the ends of groups
constexpr int kPairCols = 256;          // columns of a tile of two CTAs
constexpr int kMinChunks = 8;           // of each of the CTAs that share a tile
constexpr int kMaxSplit = 8;            // CTAs that share a tile's summed length
// The tensor core's running sum is taken into fp32 registers after this many chunks: its additions
// truncate, so its error grows with the length (of random products, in the result's norm: 512
// values 4.7e-7, 4096 4.4e-6, 16384 1.9e-5; fp32 additions 1.6e-7, 6.1e-7 and 1.5e-6.  Of positive
// ones about 8e-9 a value: 2^18 of them 2.1e-3).
constexpr int kFold32 = 8, kFold16 = 64;        // of fp32 and of 16-bit results
// Results of a pair's tile: 16 bits from one running sum, fp32, or 16 bits from folded sums.
constexpr int kWhole = 0, kWide = 1, kFolded = 2;

struct Args {
  const int* offsets;
  void* out;
  const float* bias;          // forward, or nullptr
  float* db;                  // weights' gradient: the bias's, or nullptr
  const void* h;              // gradient of rows: the mask's activations, or nullptr
  int64_t out_ld, out_gs;     // in elements; out_gs: between groups of dW
  int64_t bias_ld, h_ld;      // bias_ld: db's too
  int groups, rows;
  int split;                  // dW: parts of a group's rows, each a group of its own here
  int m, n, k;                // features; dW: columns; summed length (forward, rows)
  int in_type, out_type;
  int relu;
  int wide_out;               // 16-byte accesses of the output are aligned
  int wide_h;                 // and of h
};

struct Tile {
  int g, m0, c0, cols, r0, k;   // group, first feature, first column, columns, first row, length
  bool bias;                    // the sums of dy instead of a part of dW
};

// Column tiles of a group of n rows: as few as fit, of equal size.
__device__ __forceinline__ int col_tiles(int n, int NT) { return (n + NT - 1) / NT; }

// Instruction descriptor of a kind::f16 MMA with fp32 sums: element types at bits 7-9 and
// 10-12, N >> 3 at bits 17-22, M >> 4 at bits 24-28.
__device__ __forceinline__ uint32_t idesc_of(int type, int M, int N) {
  const uint32_t t = type == HA_TYPE_BF16 ? 1u : 0u;
  return (1u << 4) | (t << 7) | (t << 10) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(M >> 4) << 24);
}

__device__ __forceinline__ uint16_t narrow(float x, int type) {
  if (type == HA_TYPE_BF16) {
    const __nv_bfloat16 b = __float2bfloat16_rn(x);
    return *reinterpret_cast<const uint16_t*>(&b);
  }
  const __half b = __float2half_rn(x);
  return *reinterpret_cast<const uint16_t*>(&b);
}
__device__ __forceinline__ uint32_t narrow_pair(float a, float b, int type) {
  return type == HA_TYPE_BF16 ? narrow2<__nv_bfloat16>(a, b) : narrow2<__half>(a, b);
}
__device__ __forceinline__ bool positive16(uint32_t w, int type) {   // > 0, not NaN
  return w != 0 && w <= (type == HA_TYPE_BF16 ? 0x7F80u : 0x7C00u);
}

struct Table {
  int* off;         // rows of each group, inside [0, rows]
  int* first;       // first tile of each group
};

// The list of tiles, by all threads; ends with a CTA barrier.
template <int MODE, int M, int NT, int THREADS>
__device__ __forceinline__ void make_table(const Table& s, const Args& a) {
  const int tid = threadIdx.x, lane = tid & 31;
  for (int g = tid; g <= a.groups; g += THREADS) {
    const int of = MODE == kDw ? g / a.split : g, part = MODE == kDw ? g - of * a.split : 0;
    int low = min(max(a.offsets[of], 0), a.rows);
    if (part > 0) {
      // the parts are whole chunks of rows, but for the group's last
      const int n = max(0, min(max(a.offsets[of + 1], 0), a.rows) - low);
      const int64_t size = ((n + kK - 1) / kK + a.split - 1) / a.split * static_cast<int64_t>(kK);
      low += static_cast<int>(min(static_cast<int64_t>(n), part * size));
    }
    s.off[g] = low;
  }
  __syncthreads();
  if (tid < 32) {
    if (MODE != kDw) {
      // Offsets that go back would put rows into two groups, whose tiles then write them without
      // order.  Each start is raised to the largest before it, so that a row is its first group's.
      int top = 0;
      for (int g0 = 0; g0 <= a.groups; g0 += 32) {
        const int g = g0 + lane, x = g <= a.groups ? s.off[g] : 0;
        int y = x;
        const int before = __shfl_up_sync(~0u, x, 1);
        if (__any_sync(~0u, g <= a.groups && x < (lane ? before : top))) {
          y = max(y, top);
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) y = max(y, __shfl_up_sync(~0u, y, o));
          if (g <= a.groups) s.off[g] = y;
        }
        top = __shfl_sync(~0u, y, min(31, a.groups - g0));
      }
      __syncwarp();
    }
    const int mt = (a.m + M - 1) / M, nt = (a.n + NT - 1) / NT + (MODE == kDw && a.db ? 1 : 0);
    int run = 0;
    for (int g0 = 0; g0 < a.groups; g0 += 32) {
      const int g = g0 + lane;
      // offsets that go back leave a group empty
      const int n = g < a.groups ? max(0, s.off[g + 1] - s.off[g]) : 0;
      const int tiles = MODE == kDw ? (g < a.groups ? mt * nt : 0) : mt * col_tiles(n, NT);
      int x = tiles;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(~0u, x, o);
        if (lane >= o) x += y;
      }
      if (g < a.groups) s.first[g] = run + x - tiles;
      run += __shfl_sync(~0u, x, 31);
    }
    if (lane == 0) s.first[a.groups] = run;
  }
  __syncthreads();
}

// The tiles of a CTA (or pair), in rising order.  STEP: the columns of a tile are a multiple of
// it (but for the group's end).
template <int MODE, int M, int NT, int STEP>
struct Tiles {
  const Table& s;
  const Args& a;
  const int mt;
  int g = 0;
  __device__ __forceinline__ Tiles(const Table& s, const Args& a) : s(s), a(a), mt((a.m + M - 1) / M) {}
  __device__ __forceinline__ Tile at(int i) {
    if (MODE == kDw)
      g = i / s.first[1];                  // as many tiles in every group
    else
      while (s.first[g + 1] <= i) ++g;
    const int x = i - s.first[g];
    Tile t;
    t.g = g;
    // dW: the columns of a strip of rows one after the other, so that whole rows are written at
    // about the same time; else the features first, which share the rows they read.
    const int per = MODE == kDw ? s.first[1] / mt : mt, q = x / per, rest = x - q * per;
    const int ct = MODE == kDw ? rest : q, low = s.off[g], n = max(0, s.off[g + 1] - low);
    t.m0 = (MODE == kDw ? q : rest) * M;
    t.bias = false;
    if (MODE == kDw) {
      t.c0 = ct * NT;
      t.bias = t.c0 >= a.n;
      t.cols = t.bias ? 32 : min(NT, a.n - t.c0);
      t.r0 = low;
      t.k = n;
    } else {
      const int parts = col_tiles(n, NT), size = ((n + parts - 1) / parts + STEP - 1) / STEP * STEP;
      t.c0 = low + ct * size;
      t.cols = min(size, n - ct * size);
      t.r0 = t.c0;
      t.k = a.k;
    }
    return t;
  }
};

// The rows that no group covers are zero.
__device__ void clear_rows(const Args& a, int64_t begin, int64_t end) {
  for (int64_t r = begin + blockIdx.x; r < end; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < a.m; c += kThreads) {
      if (a.out_type == HA_TYPE_FP32)
        static_cast<float*>(a.out)[r * a.out_ld + c] = 0.0f;
      else
        static_cast<uint16_t*>(a.out)[r * a.out_ld + c] = 0;
    }
}

// ---- results of the forward and of the rows' gradient
// A warp group holds 128 features (one a thread) of up to 32 columns, which are rows of the
// output.  They pass through shared memory, so that a row's features leave as whole 16-byte
// vectors.  Two buffers of 8 KB (32 rows of 16-bit values, 16 of fp32 ones) take turns, so
// that one barrier a buffer is enough.
constexpr int kRowsStage = 16384;
template <int MODE, typename OUT>
__device__ __forceinline__ void emit_rows(const Args& a, const float* v, int row0, int rows, int m0,
                                          int feature, float bias, unsigned char* stage, int bar,
                                          uint32_t& turn) {
  constexpr int R = 8192 / (kM * sizeof(OUT));            // rows of a buffer: 32 or 16
  constexpr int P = 16 / sizeof(OUT), S = kM / P;         // features of a vector, vectors of a row
  const int et = threadIdx.x & 127;
#pragma unroll
  for (int j = 0; j < 32; j += R) {
    if (j >= rows) return;                                // the same for the whole warp group
    unsigned char* buf = stage + (turn++ & 1) * 8192;
    uint4 hv[R * S / 128];
    // the mask's values are asked for before the barrier
    if (MODE == kDx && a.h && !a.wide_out) {
      uint32_t* p = &hv[0].x;                             // two rows' a word
      const uint16_t* h = static_cast<const uint16_t*>(a.h) + static_cast<int64_t>(row0 + j) * a.h_ld + m0 + et;
      const int n = m0 + et < a.m ? rows - j : 0;
#pragma unroll
      for (int x = 0; x < R; x += 2)
        p[x / 2] = (x < n ? h[x * a.h_ld] : 0u) | (x + 1 < n ? static_cast<uint32_t>(h[(x + 1) * a.h_ld]) << 16 : 0u);
    } else if (MODE == kDx && a.h) {
#pragma unroll
      for (int x = 0; x < R * S / 128; ++x) {
        const int i = et + x * 128, r = i / S, e = m0 + i % S * P;
        hv[x] = make_uint4(0, 0, 0, 0);
        if (j + r < rows && e < a.m) {
          const uint16_t* h = static_cast<const uint16_t*>(a.h) + static_cast<int64_t>(row0 + j + r) * a.h_ld + e;
          if (a.wide_h && e + P <= a.m) {
            if (sizeof(OUT) == 2) {
              hv[x] = *reinterpret_cast<const uint4*>(h);
            } else {
              const uint2 w = *reinterpret_cast<const uint2*>(h);
              hv[x].x = w.x;
              hv[x].y = w.y;
            }
          } else {
            uint16_t* q = reinterpret_cast<uint16_t*>(&hv[x]);
#pragma unroll
            for (int y = 0; y < P; ++y)
              if (e + y < a.m) q[y] = h[y];
          }
        }
      }
    }
#pragma unroll
    for (int x = 0; x < R; ++x) {
      float f = v[j + x] + bias;
      if (MODE == kFwd && a.relu && f < 0.0f) f = 0.0f;
      if constexpr (sizeof(OUT) == 4)
        reinterpret_cast<float*>(buf)[x * kM + feature] = f;
      else
        reinterpret_cast<uint16_t*>(buf)[x * kM + feature] = narrow(f, a.out_type);
    }
    named_barrier_sync(bar, 128);
    if (!a.wide_out) {
      // rows that are not aligned for vectors: a thread a feature, so that a row's leave side by
      // side (2 groups, 4249 rows, 258 -> 1087, bf16: 21 us; a vector's features by one thread, 37)
      OUT* o = static_cast<OUT*>(a.out) + static_cast<int64_t>(row0 + j) * a.out_ld + m0 + et;
      const int n = m0 + et < a.m ? rows - j : 0;
      const uint32_t* p = &hv[0].x;
#pragma unroll
      for (int x = 0; x < R; ++x)
        if (x < n) {
          OUT w = reinterpret_cast<const OUT*>(buf)[x * kM + et];
          if (MODE == kDx && a.h && !positive16(p[x / 2] >> (16 * (x & 1)) & 0xFFFFu, a.in_type)) w = 0;
          o[x * a.out_ld] = w;
        }
      continue;
    }
#pragma unroll
    for (int x = 0; x < R * S / 128; ++x) {
      const int i = et + x * 128, r = i / S, e = m0 + i % S * P;
      if (j + r >= rows || e >= a.m) continue;
      uint4 w = *reinterpret_cast<const uint4*>(buf + i * 16);
      if (MODE == kDx && a.h) {
        uint32_t* p = &w.x;
        const uint32_t* q = &hv[x].x;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          if constexpr (sizeof(OUT) == 4) {
            if (!positive16((q[y >> 1] >> (16 * (y & 1))) & 0xFFFFu, a.in_type)) p[y] = 0;
          } else {
            if (!positive16(q[y] & 0xFFFFu, a.in_type)) p[y] &= 0xFFFF0000u;
            if (!positive16(q[y] >> 16, a.in_type)) p[y] &= 0xFFFFu;
          }
        }
      }
      OUT* o = static_cast<OUT*>(a.out) + static_cast<int64_t>(row0 + j + r) * a.out_ld + e;
      if (e + P <= a.m) {
        *reinterpret_cast<uint4*>(o) = w;
      } else {
        const OUT* p = reinterpret_cast<const OUT*>(&w);
#pragma unroll
        for (int y = 0; y < P; ++y)
          if (e + y < a.m) o[y] = p[y];
      }
    }
  }
}

// ---- results of the weights' gradient
// A warp holds 32 features (rows of dW, one a lane) of 32 columns at a time.  Rows of 128
// bytes are put together in shared memory (16-byte pieces swapped by the row, against bank
// conflicts), and eight lanes store a row.  (32 groups of 512 rows, 4096 x 4096, 16 bits: lanes
// storing their own rows 500 us, bulk stores of boxes with 64-byte rows 409, this 376 to 380.)  Rows
// that are not aligned for that leave value by value, side by side.
constexpr int kWarpStage = 4096;
__device__ __forceinline__ void emit_weights(const Args& a, const float* v, int g, int f0, int c, int end,
                                             unsigned char* stage) {
  const int lane = threadIdx.x & 31;
  const bool wide = a.out_type == HA_TYPE_FP32;
  const int half = wide ? 0 : (c >> 5) & 1;               // which 32 of a 16-bit row's 64 columns
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    if (!wide && p >= 4) break;
    uint4 w;
    if (wide)
      w = make_uint4(__float_as_uint(v[4 * p]), __float_as_uint(v[4 * p + 1]), __float_as_uint(v[4 * p + 2]),
                     __float_as_uint(v[4 * p + 3]));
    else
      w = make_uint4(narrow_pair(v[8 * (p & 3)], v[8 * (p & 3) + 1], a.out_type),
                     narrow_pair(v[8 * (p & 3) + 2], v[8 * (p & 3) + 3], a.out_type),
                     narrow_pair(v[8 * (p & 3) + 4], v[8 * (p & 3) + 5], a.out_type),
                     narrow_pair(v[8 * (p & 3) + 6], v[8 * (p & 3) + 7], a.out_type));
    *reinterpret_cast<uint4*>(stage + lane * 128 + (((half * 4 + p) ^ (lane & 7)) << 4)) = w;
  }
  if (!wide && half == 0 && c + 32 < end) return;         // the row's other half comes next
  __syncwarp();
  const int c0 = c - half * 32;
  if (a.wide_out) {
    const int es = wide ? 4 : 2, piece = lane & 7, col = c0 + piece * (16 / es);
    if (col < end) {
      unsigned char* o = static_cast<unsigned char*>(a.out) +
                         (g * a.out_gs + static_cast<int64_t>(f0 + (lane >> 3)) * a.out_ld + col) * es;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = i * 4 + (lane >> 3);
        if (f0 + row < a.m)
          *reinterpret_cast<uint4*>(o + i * 4 * a.out_ld * es) =
              *reinterpret_cast<const uint4*>(stage + row * 128 + ((piece ^ (row & 7)) << 4));
      }
    }
  } else {
    const int rows = min(32, a.m - f0);
    for (int row = 0; row < rows; ++row) {
      const int64_t at = g * a.out_gs + static_cast<int64_t>(f0 + row) * a.out_ld + c0 + lane;
      if (wide) {
        if (c0 + lane < end)
          static_cast<float*>(a.out)[at] =
              *reinterpret_cast<const float*>(stage + row * 128 + (((lane >> 2) ^ (row & 7)) << 4) + (lane & 3) * 4);
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (c0 + h * 32 + lane < end)
            static_cast<uint16_t*>(a.out)[at + h * 32] = *reinterpret_cast<const uint16_t*>(
                stage + row * 128 + (((h * 4 + (lane >> 3)) ^ (row & 7)) << 4) + (lane & 7) * 2);
      }
    }
  }
  __syncwarp();
}

// A warp's wait for sums, by one lane: 32 lanes asking keep the barrier unit from the roles
// that feed the tensor cores.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity) {
  int ok = 1;
  if ((threadIdx.x & 31) == 0) ok = mbar_wait(bar, parity, &g_operator_error);
  ok = __shfl_sync(~0u, ok, 0);
  tc_fence_after();
  return ok != 0;
}

// A place in a ring of stages and the parity of its round.
template <int STAGES>
struct Ring {
  uint32_t st = 0, round = 0;
  __device__ __forceinline__ void next() {
    if (++st == STAGES) {
      st = 0;
      round ^= 1;
    }
  }
  __device__ __forceinline__ void skip(int n) {
    const uint32_t to = st + static_cast<uint32_t>(n);
    st = to % STAGES;
    round ^= (to / STAGES) & 1;
  }
  __device__ __forceinline__ uint32_t next_st() const { return st + 1 == STAGES ? 0 : st + 1; }
  __device__ __forceinline__ uint32_t next_round() const { return st + 1 == STAGES ? round ^ 1 : round; }
};

// Chunks of a summed length.  In the weights' gradient those of whole steps of 16: what is left is
// summed from a place of its own.
template <int MODE>
__device__ __forceinline__ int chunks_of(int k) { return ((MODE == kDw ? k & ~15 : k) + kK - 1) / kK; }
template <int RES>
__device__ __forceinline__ int fold_of(bool bias) {
  return RES == kWide || bias ? kFold32 : RES == kFolded ? kFold16 : 1 << 30;
}

// One tile's results: `half` of its NT columns, from the sums in TMEM, segment by segment.
template <int MODE, int NT, int RES, typename Wait, typename Free>
__device__ __forceinline__ bool finish_tile(const Args& a, const Tile& t, uint32_t tmem,
                                            int cta_m0, unsigned char* stage, uint32_t& seg, uint32_t& turn,
                                            Wait wait, Free release) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = warp >> 2, quad = warp & 3;
  const int nk = chunks_of<MODE>(t.k), fold = fold_of<RES>(t.bias);
  const int segs = MODE == kDw && nk == 0 && t.k > 0 ? 1 : (nk + fold - 1) / fold;
  constexpr int H = NT / 2;
  const int cb = half * H, ce = min(H, t.cols - cb);      // this warp group's columns
  const int f = cta_m0 + quad * 32 + lane;                // this thread's feature
  const float bias = MODE == kFwd && a.bias && f < a.m ? a.bias[t.g * a.bias_ld + f] : 0.0f;
  constexpr int STEP = 32;
  auto emit = [&](const float* v, int j) {
    if (MODE == kDw)
      emit_weights(a, v, t.g, cta_m0 + quad * 32, t.c0 + cb + j, t.c0 + cb + ce, stage + warp * kWarpStage);
    else if (RES == kWide)
      emit_rows<MODE, float>(a, v, t.c0 + cb + j, min(STEP, ce - j), cta_m0, quad * 32 + lane, bias,
                             stage + half * kRowsStage, 1 + half, turn);
    else
      emit_rows<MODE, uint16_t>(a, v, t.c0 + cb + j, min(STEP, ce - j), cta_m0, quad * 32 + lane, bias,
                                stage + half * kRowsStage, 1 + half, turn);
  };
  auto read = [&](float* v, int buf, int j) {
    const uint32_t at = tmem + (static_cast<uint32_t>(quad * 32) << 16) + buf * NT + cb + j;
    tmem_ld32(at, v);
    tmem_ld_wait();
  };
  if (MODE == kDw && t.bias) {
    // every column has the sums of dy
    float sum = 0.0f;
    for (int s = 0; s < segs; ++s) {
      if (!wait(seg)) return false;
      if (half == 0) {
        float v[16];
        tmem_ld16(tmem + (static_cast<uint32_t>(quad * 32) << 16) + (seg & 1) * NT, v);
        tmem_ld_wait();
        sum += v[0];
      }
      release(seg++);
    }
    if (half == 0 && f < a.m) a.db[t.g * a.bias_ld + f] = sum;
    return true;
  }
  if (RES == kWhole) {
    if (segs && !wait(seg)) return false;
    if (MODE == kDw && segs) {
      // all of a half's reads are under way before the first is used
#pragma unroll
      for (int j0 = 0; j0 < H; j0 += 64) {
        if (j0 >= ce) break;
        float v[64];
        const uint32_t at = tmem + (static_cast<uint32_t>(quad * 32) << 16) + (seg & 1) * NT + cb + j0;
        tmem_ld32(at, v);
        tmem_ld32(at + 32, v + 32);
        tmem_ld_wait();
        if (j0 + 64 >= min(H, ce)) release(seg++);
        emit(v, j0);
        if (j0 + 32 < ce) emit(v + 32, j0 + 32);
      }
      if (ce <= 0) release(seg++);
      return true;
    }
#pragma unroll 1
    for (int j = 0; j < H; j += STEP) {
      if (j >= ce) break;
      float v[32];
#pragma unroll
      for (int x = 0; x < 32; ++x) v[x] = 0.0f;
      if (segs) read(v, seg & 1, j);
      emit(v, j);
    }
    if (segs) release(seg++);
    return true;
  }
  float acc[H];
#pragma unroll
  for (int j = 0; j < H; ++j) acc[j] = 0.0f;
  for (int s = 0; s < segs; ++s) {
    if (!wait(seg)) return false;
#pragma unroll
    for (int j = 0; j < H; j += STEP)
      if (j < ce) {
        float v[32];
        read(v, seg & 1, j);
#pragma unroll
        for (int x = 0; x < STEP; ++x) acc[j + x] += v[x];
      }
    release(seg++);
  }
#pragma unroll
  for (int j = 0; j < H; j += STEP)
    if (j < ce) emit(acc + j, j);
  return true;
}

// ---- groups of few rows: one CTA a tile of 128 features and up to NT rows
// The weights' bytes are what counts, so the stages are many and small: a chunk of weights
// is 16 KB, and 9 of them (NT = 64: 6) are in flight.  Where there are fewer tiles than SMs, the
// CTAs of a cluster share a tile: each sums its part of the length and sends each column's sums to
// the CTA whose column it is, which adds them in the CTAs' order (one row, 4096 -> 4096: 10.8 us; the
// first CTA reading and adding all of them 11.5, one CTA a tile 18.2).
template <int NT>
struct One {
  static constexpr int kA = kM * kK * 2, kB = NT * kK * 2, kStages = NT == 32 ? 9 : 6;
  static constexpr int kPart = kM * NT * 4;               // sums from the cluster's CTAs, or for them
  static constexpr int kOut = 2 * kPart;
  static constexpr int kSmem = kStages * (kA + kB) + kOut + 1024;
};

template <int MODE, bool WIDE, int NT>
__global__ void __launch_bounds__(kThreads, 1)
    k_grouped_one(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb,
                  const __grid_constant__ Args a) {
  using S = One<NT>;
  extern __shared__ unsigned char raw[];
  // theirs: the CTAs' sums of this one's columns are there; mine: every CTA is done with its own
  __shared__ uint64_t full[S::kStages], empty[S::kStages], tfull[2], tempty[2], theirs, mine;
  __shared__ uint32_t tmem_at;
  __shared__ int table[2 * (kMaxGroups + 1)];
  const Table tab = {table, table + kMaxGroups + 1};
  unsigned char* As = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  unsigned char* Bs = As + S::kStages * S::kA;
  unsigned char* Out = Bs + S::kStages * S::kB;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = static_cast<int>(cluster_rank()), split = static_cast<int>(cluster_size());
  if (warp == kEpiWarps) {
    tmem_alloc(&tmem_at, 2 * NT);
    tmem_relinquish();
  }
  if (tid == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&tfull[i], 1);
      mbar_init(&tempty[i], kEpiWarps);
    }
    mbar_init(&theirs, 1);
    mbar_init(&mine, split * kEpiWarps / 2);
    fence_barrier_init();
  }
  tc_fence_before();
  make_table<MODE, kM, NT, kThreads>(tab, a);
  if (split > 1) cluster_arrive();                        // the barriers are set up
  Tiles<MODE, kM, NT, 16> list(tab, a);
  tc_fence_after();
  const uint32_t tmem = tmem_at;
  const int tiles = tab.first[a.groups], i0 = blockIdx.x / split, step = gridDim.x / split;
  const int all = (a.k + kK - 1) / kK;                     // chunks of a tile, and this CTA's
  const int c0 = all * rank / split, c1 = all * (rank + 1) / split;
  constexpr int fold = WIDE ? kFold32 : kFold16;
  bool ok = true;                                         // of the results' warps
  uint32_t round = 0;
  clear_rows(a, 0, tab.off[0]);
  clear_rows(a, tab.off[a.groups], a.rows);

  if (warp == kEpiWarps) {
    // ---- loads
    if (elect_one()) {
      Ring<S::kStages> at;
      bool ok = true;
      const uint64_t stream = l2_stream_policy(true), keep = l2_stream_policy(false);
      for (int i = i0; i < tiles && ok; i += step) {
        const Tile t = list.at(i);
        const int boxes = (t.cols + 15) / 16;
        for (int c = c0; c < c1; ++c, at.next()) {
          const int st = at.st;
          if (!mbar_wait_hot(&empty[st], at.round ^ 1, &g_operator_error)) { ok = false; break; }
          uint64_t* bar = &full[st];
          mbar_arrive_expect_tx(bar, S::kA + boxes * 2048);
          unsigned char* A = As + st * S::kA;
          if (MODE == kFwd) {
            tma_load_3d_hint(A, &ta, bar, c * kK, t.m0, t.g, stream);
          } else {
            tma_load_3d_hint(A, &ta, bar, t.m0, c * kK, t.g, stream);
            tma_load_3d_hint(A + 8192, &ta, bar, t.m0 + 64, c * kK, t.g, stream);
          }
          for (int b = 0; b < boxes; ++b)
            tma_load_3d_hint(Bs + st * S::kB + b * 2048, &tb, bar, c * kK, t.r0 + b * 16, 0, keep);
        }
      }
    }
  } else if (warp == kEpiWarps + 1) {
    // ---- matrix products, by one lane
    if (elect_one()) {
      Ring<S::kStages> at;
      uint32_t seg = 0;
      bool ok = true, peek = false;
      for (int i = i0; i < tiles && ok; i += step) {
        const Tile t = list.at(i);
        const uint32_t idesc = idesc_of(a.in_type, kM, (t.cols + 15) / 16 * 16) | (MODE == kFwd ? 0u : 1u << 15);
        int part = 0;                                     // chunks since the last fold
        for (int c = c0; c < c1; ++c, at.next()) {
          const int buf = seg & 1;
          ok = (part != 0 || mbar_wait_hot(&tempty[buf], ((seg >> 1) & 1) ^ 1, &g_operator_error)) &&
               (peek || mbar_wait_hot(&full[at.st], at.round, &g_operator_error));
          if (!ok) break;
          tc_fence_after();
          const int steps = (min(t.k - c * kK, kK) + 15) / 16;
          const uint32_t as = smem_u32(As + at.st * S::kA), bs = smem_u32(Bs + at.st * S::kB);
          const uint64_t da = MODE == kFwd ? umma_desc_sw128(as) : umma_desc_sw128_mn(as, 8192);
          const uint64_t db = umma_desc_sw128(bs);
          constexpr int SA = MODE == kFwd ? 2 : 128;      // 16 values further, in 16 bytes
          if (steps == 4) {
            peek = tc_chunk<SA, 2>(tmem + buf * NT, da, db, idesc, part != 0, &empty[at.st], &full[at.next_st()],
                                   at.next_round());
          } else {
            for (int k = 0; k < steps; ++k)
              tc_mma_bf16(tmem + buf * NT, da + k * SA, db + k * 2, idesc, part || k ? 1u : 0u);
            tc_commit(&empty[at.st]);
            peek = false;
          }
          if (++part == fold || c == c1 - 1) {
            tc_commit(&tfull[buf]);
            ++seg;
            part = 0;
          }
        }
      }
    }
  } else {
    // ---- results
    constexpr int H = NT / 2;                             // columns of a warp group
    const int half = warp >> 2, quad = warp & 3, feature = quad * 32 + lane;
    const int segs = (c1 - c0 + fold - 1) / fold;
    float* got = reinterpret_cast<float*>(Out);           // [CTA][column][feature]
    float* part = reinterpret_cast<float*>(Out + S::kPart);                 // [column][feature]
    uint32_t seg = 0, turn = 0;
    if (split > 1) cluster_wait();
    for (int i = i0; i < tiles; i += step, ++round) {
      const Tile t = list.at(i);
      const int cb = half * H, ce = min(H, t.cols - cb), f = t.m0 + feature;
      float acc[32];
#pragma unroll
      for (int x = 0; x < 32; ++x) acc[x] = 0.0f;
      // this CTA's columns of a shared tile
      const int per = (t.cols + split - 1) / split, own = max(0, min(per, t.cols - rank * per));
      for (int s = 0; s < segs && ok; ++s, ++seg) {
        ok = warp_wait(&tfull[seg & 1], (seg >> 1) & 1);
        if (!ok) break;
        if (ce > 0) {
          float v[32];
          const uint32_t at = tmem + (static_cast<uint32_t>(quad * 32) << 16) + (seg & 1) * NT + cb;
          if (H == 32) tmem_ld32(at, v);
          else tmem_ld16(at, v);
          tmem_ld_wait();
#pragma unroll
          for (int x = 0; x < H; ++x) acc[x] += v[x];
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&tempty[seg & 1]);
      }
      if (!ok) break;
      if (split > 1) {
        if (round > 0) {
          if (lane == 0) ok = mbar_wait_cluster(&mine, (round - 1) & 1, &g_operator_error);
          ok = __all_sync(~0u, ok);
          if (!ok) break;
        }
#pragma unroll
        for (int x = 0; x < H; ++x)
          if (x < ce) part[(cb + x) * kM + feature] = acc[x];
        fence_proxy_async_smem();
        named_barrier_sync(3, kEpiWarps * 32);
        if (tid == 0) mbar_arrive_expect_tx(&theirs, split * own * kM * 4);
        if (tid < split) {
          const int n = min(per, t.cols - tid * per);
          if (n > 0)
            bulk_to_cta(cluster_addr(got + rank * per * kM, tid), part + tid * per * kM, n * kM * 4,
                        cluster_addr(&theirs, tid));
        }
        if (half != 0) continue;                          // one warp group adds
        if (lane == 0) ok = mbar_wait_cluster(&theirs, round & 1, &g_operator_error);
        ok = __all_sync(~0u, ok);
        if (!ok) break;
#pragma unroll
        for (int x = 0; x < H; ++x) acc[x] = 0.0f;
#pragma unroll 2
        for (int q = 0; q < split; ++q) {
#pragma unroll
          for (int x = 0; x < H; ++x)
            if (x < own) acc[x] += got[(q * per + x) * kM + feature];
        }
        named_barrier_sync(1, 128);                       // the rows pass through the same memory
      }
      const float bias = MODE == kFwd && a.bias && f < a.m ? a.bias[t.g * a.bias_ld + f] : 0.0f;
      const int first = split > 1 ? rank * per : cb, n = split > 1 ? own : min(H, ce);
      if (n > 0) {
        if (WIDE)
          emit_rows<MODE, float>(a, acc, t.c0 + first, n, t.m0, feature, bias, Out + half * kRowsStage, 1 + half, turn);
        else
          emit_rows<MODE, uint16_t>(a, acc, t.c0 + first, n, t.m0, feature, bias, Out + half * kRowsStage, 1 + half, turn);
      }
      if (split > 1) {
        __syncwarp();
        if (i + step < tiles && lane < split) mbar_arrive_release_cluster(cluster_addr(&mine, lane));
      }
    }
  }
  if (split > 1 && warp >= kEpiWarps) {
    __syncwarp();
    cluster_wait();
  }
  tc_fence_before();
  __syncthreads();
  if (split > 1) {
    cluster_sync_all();                                   // the CTAs write to one another's memory
    if (!ok && warp < kEpiWarps) warp_wait(&theirs, round & 1);   // after a wait that ran out: what is on its way
  }
  if (warp == kEpiWarps) tmem_dealloc(tmem, 2 * NT);
}

// ---- everything else: two CTAs of a cluster a tile of 256 features and up to 256 columns
// The pair's MMA (cta_group::2) is issued by its first CTA.  Each CTA loads its own 128
// features and half of the columns; the tensor cores read both halves of the columns, so a
// CTA's shared memory takes in and hands out a third less per product than with a tile of
// 128 x 256 of its own, where it would be the bound.  Each CTA has its features' sums in its
// own TMEM, in two buffers, and writes its own results.
struct Pair {
  static constexpr int kA = kM * kK * 2, kB = kPairCols / 2 * kK * 2, kStages = 5;
  static constexpr int kOut = 2 * kRowsStage;             // = kEpiWarps * kWarpStage
  static constexpr int kOnes = 8192;                      // dW: a column block of ones, for the bias
  static constexpr int kEnd = 8192;                       // dW: the last rows of a group, two of them
  static constexpr int kSmem = kStages * (kA + kB) + kOut + kOnes + 2 * kEnd + 1024;
};
static_assert(2 * kRowsStage == kEpiWarps * kWarpStage, "one buffer serves both kinds of results");

// Maps with boxes of 16 rows, for the last rows of groups in the weights' gradient.
template <int MODE> struct Ends {};
template <> struct Ends<kDw> { CUtensorMap a, b; };

template <int MODE, int RES>
__global__ void __launch_bounds__(MODE == kDw ? kDwThreads : kThreads, 1) __cluster_dims__(2, 1, 1)
    k_grouped_pair(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb,
                   const __grid_constant__ Ends<MODE> ends, const __grid_constant__ Args a) {
  extern __shared__ unsigned char raw[];
  // full: the first CTA's, on which both CTAs' loads are counted.  tempty: the first CTA's too.  Of a
  // group's last rows, end_load: they are in this CTA; end_peer: the second CTA's are ready; end_full:
  // both CTAs' are (these two the first CTA's); end_empty: summed.
  __shared__ uint64_t full[Pair::kStages], empty[Pair::kStages], tfull[2], tempty[2];
  __shared__ uint64_t end_load[2], end_peer[2], end_full[2], end_empty[2];
  __shared__ uint32_t tmem_at;
  __shared__ int table[2 * (kMaxGroups + 1)];
  const Table tab = {table, table + kMaxGroups + 1};
  unsigned char* As = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  unsigned char* Bs = As + Pair::kStages * Pair::kA;
  unsigned char* Out = Bs + Pair::kStages * Pair::kB;
  unsigned char* Ones = Out + Pair::kOut;
  unsigned char* End = Ones + Pair::kOnes;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  if (warp == kEpiWarps) {
    tmem_alloc_pair(&tmem_at, 2 * kPairCols);
    tmem_relinquish_pair();
  }
  if (tid == 0) {
    for (int i = 0; i < Pair::kStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&tfull[i], 1);
      mbar_init(&tempty[i], 2 * kEpiWarps);
      mbar_init(&end_load[i], 1);
      mbar_init(&end_peer[i], 1);
      mbar_init(&end_full[i], 1);
      mbar_init(&end_empty[i], 1);
    }
    fence_barrier_init();
  }
  if (MODE == kDw && a.db) {
    const uint32_t one = a.in_type == HA_TYPE_BF16 ? 0x3F803F80u : 0x3C003C00u;
    for (int i = tid; i < Pair::kOnes / 4; i += kDwThreads) reinterpret_cast<uint32_t*>(Ones)[i] = one;
    fence_proxy_async();
  }
  tc_fence_before();
  make_table<MODE, 2 * kM, kPairCols, MODE == kDw ? kDwThreads : kThreads>(tab, a);
  Tiles<MODE, 2 * kM, kPairCols, 32> list(tab, a);
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = tmem_at;
  const int tiles = tab.first[a.groups], pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  if (MODE != kDw) {
    clear_rows(a, 0, tab.off[0]);
    clear_rows(a, tab.off[a.groups], a.rows);
  }

  if (warp == kEpiWarps) {
    // ---- loads, by both CTAs
    if (elect_one()) {
      Ring<Pair::kStages> at;
      bool ok = true, peek = false;
      const uint32_t full0 = cluster_addr(full, 0);
      for (int i = pair; i < tiles && ok; i += pairs) {
        const Tile t = list.at(i);
        const int nk = chunks_of<MODE>(t.k), hcols = (t.cols + 31) / 32 * 16;  // columns of a CTA
        const int m0 = t.m0 + rank * kM, h0 = rank * hcols, boxes = t.bias ? 0 : (hcols + 63) / 64;
        const uint32_t bytes = Pair::kA + boxes * 8192;
        for (int c = 0; c < nk; ++c, at.next()) {
          const int st = at.st, k = c * kK;
          if (!peek && !mbar_wait_hot(&empty[st], at.round ^ 1, &g_operator_error)) { ok = false; break; }
          const uint32_t bar = full0 + st * 8, armed = rank == 0 ? 2 * bytes : 0;
          unsigned char* A = As + st * Pair::kA;
          unsigned char* B = Bs + st * Pair::kB;
          uint64_t* next = &empty[at.next_st()];
          const uint32_t parity = at.next_round() ^ 1;
          if (MODE == kFwd) {
            peek = tma_chunk_pair<false, false>(A, &ta, k, m0, t.g, B, &tb, k, t.r0 + h0, 0, boxes, bar, &full[st], armed,
                                                next, parity);
          } else if (MODE == kDx) {
            peek = tma_chunk_pair<true, false>(A, &ta, m0, k, t.g, B, &tb, k, t.r0 + h0, 0, boxes, bar, &full[st], armed,
                                               next, parity);
          } else {
            peek = tma_chunk_pair<true, true>(A, &ta, m0, t.r0 + k, 0, B, &tb, t.c0 + h0, t.r0 + k, 0, boxes, bar, &full[st],
                                              armed, next, parity);
          }
        }
      }
    }
  } else if (warp == kEpiWarps + 1) {
    // ---- matrix products, by one lane of the first CTA (a wait of all lanes takes the barrier
    // unit 32 times as long)
    if (rank == 0 && elect_one()) {
      Ring<Pair::kStages> at;
      uint32_t seg = 0, end = 0;
      bool ok = true, peek = false;
      for (int i = pair; i < tiles && ok; i += pairs) {
        const Tile t = list.at(i);
        const int nk = chunks_of<MODE>(t.k), N = (t.cols + 31) / 32 * 32;
        const int fold = fold_of<RES>(t.bias);
        const uint32_t idesc = idesc_of(a.in_type, 2 * kM, N) | (MODE == kFwd ? 0u : 1u << 15) |
                               (MODE == kDw ? 1u << 16 : 0u);
        const bool tail = MODE == kDw && t.k % 16 != 0;
        int part = 0;                                       // chunks since the last fold
        for (int c = 0; c < nk; ++c, at.next()) {
          const int st = at.st, buf = seg & 1;
          ok = (part != 0 || mbar_wait_hot(&tempty[buf], ((seg >> 1) & 1) ^ 1, &g_operator_error)) &&
               (peek || mbar_wait_hot(&full[st], at.round, &g_operator_error));
          if (!ok) break;
          tc_fence_after();
          const int left = t.k - c * kK, steps = left >= kK ? 4 : MODE == kDw ? left / 16 : (left + 15) / 16;
          const uint32_t as = smem_u32(As + st * Pair::kA), bs = smem_u32(t.bias ? Ones : Bs + st * Pair::kB);
          const uint32_t d = tmem + buf * kPairCols;
          const uint64_t da = MODE == kFwd ? umma_desc_sw128(as) : umma_desc_sw128_mn(as, 8192);
          const uint64_t db = MODE == kDw ? umma_desc_sw128_mn(bs, 8192) : umma_desc_sw128(bs);
          constexpr int SA = MODE == kFwd ? 2 : 128, SB = MODE == kDw ? 128 : 2;   // 16 values further
          if (steps == 4) {
            peek = tc_chunk_pair<SA, SB>(d, da, db, idesc, part != 0, &empty[st], &full[at.next_st()], at.next_round());
          } else {
            for (int k = 0; k < steps; ++k) tc_mma_pair(d, da + k * SA, db + k * SB, idesc, part || k ? 1u : 0u);
            tc_commit_pair(&empty[st]);
            peek = false;
          }
          if (++part == fold || c == nk - 1) {
            if (tail && c == nk - 1) break;                 // the last sum goes on below
            tc_commit_pair(&tfull[buf]);
            ++seg;
            part = 0;
          }
        }
        if (tail && ok) {
          if (nk > 0) at.next();                            // which the break has left out
          const int buf = seg & 1, e = end & 1;
          ok = (part != 0 || mbar_wait_hot(&tempty[buf], ((seg >> 1) & 1) ^ 1, &g_operator_error)) &&
               mbar_wait_hot(&end_full[e], (end >> 1) & 1, &g_operator_error);
          if (!ok) break;
          tc_fence_after();
          const uint32_t as = smem_u32(End + e * Pair::kEnd);
          const uint64_t db = t.bias ? umma_desc_sw128_mn(smem_u32(Ones), 8192) : umma_desc_sw128_mn(as + 4096, 2048);
          tc_mma_pair(tmem + buf * kPairCols, umma_desc_sw128_mn(as, 2048), db, idesc, part ? 1u : 0u);
          tc_commit_pair(&end_empty[e]);
          tc_commit_pair(&tfull[buf]);
          ++seg;
          ++end;
        }
      }
    }
  } else if (MODE == kDw && warp >= kEpiWarps + 2) {
    // ---- the ends of groups, in both CTAs: the rows that fill no step of 16 are loaded by themselves,
    // and those after them, which are another group's, cleared.  A warp has every second end, up to two
    // tiles ahead of the products, so that there is time to tell the first CTA across the cluster.  (In
    // the ring's own chunks, told to the products' thread by a release and seen by an acquire at cluster
    // scope: 32 groups, 16384 rows, 4096 to 4096, 434 us, this 385; 64 groups of 47 rows, 2048 to 2048,
    // 118 and 125, with fp32 results 255 and 226.)
    if constexpr (MODE == kDw) {
      uint32_t n = 0;
      for (int i = pair; i < tiles; i += pairs) {
        const Tile t = list.at(i);
        const int left = t.k % 16;
        if (!left || (n++ & 1) != static_cast<uint32_t>(warp) - (kEpiWarps + 2)) continue;
        const int e = warp - (kEpiWarps + 2), hcols = (t.cols + 31) / 32 * 16, blocks = 2 + (t.bias ? 0 : (hcols + 63) / 64);
        const uint32_t parity = ((n - 1) >> 1) & 1;
        unsigned char* to = End + e * Pair::kEnd;
        bool ok = true;
        if (lane == 0) {
          // the sum of two tiles before this one's end is waited for, each of up to all rows
          ok = mbar_wait_hot(&end_empty[e], parity ^ 1, &g_operator_error, kWaitLimitCycles + a.rows / kK * 4096ll);
          if (ok) {
            const int m0 = t.m0 + rank * kM, c0 = t.c0 + rank * hcols, row = t.r0 + t.k - left;
            mbar_arrive_expect_tx(&end_load[e], blocks * 2048);
            for (int b = 0; b < blocks; ++b)
              tma_load_3d(to + b * 2048, b < 2 ? &ends.a : &ends.b, &end_load[e], b < 2 ? m0 + b * 64 : c0 + (b - 2) * 64, row, 0);
            ok = mbar_wait_hot(&end_load[e], parity, &g_operator_error);
          }
        }
        if (!__all_sync(~0u, ok)) break;
        for (int x = lane; x < blocks * 8; x += 32)        // 16-byte columns
          for (int r = left; r < 16; ++r)
            *reinterpret_cast<uint4*>(to + (x >> 3) * 2048 + (x & 7) * 16 + r * 128) = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();                          // before the tensor cores' reads
        __syncwarp();
        if (lane == 0) {
          if (rank != 0) {
            mbar_arrive_release_cluster(cluster_addr(&end_peer[e], 0));
          } else {
            ok = mbar_wait_cluster(&end_peer[e], parity, &g_operator_error);
            if (ok) mbar_arrive(&end_full[e]);
          }
        }
        if (!__all_sync(~0u, ok)) break;
      }
    }
  } else {
    // ---- results, by both CTAs
    uint32_t seg = 0, turn = 0;
    bool ok = true;
    for (int i = pair; i < tiles && ok; i += pairs) {
      const Tile t = list.at(i);
      ok = finish_tile<MODE, kPairCols, RES>(
          a, t, tmem, t.m0 + rank * kM, Out, seg, turn,
          [&](uint32_t s) {
            return warp_wait(&tfull[s & 1], (s >> 1) & 1);
          },
          [&](uint32_t s) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(cluster_addr(&tempty[s & 1], 0));
          });
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == kEpiWarps) tmem_dealloc_pair(tmem, 2 * kPairCols);
}

// Rows of 16-bit values to a pitch of whole 16-byte vectors, for operands that a tensor
// map cannot describe (an odd width, stride or address).  A thread makes a vector at a time, from
// loads as wide as the rows' alignment allows, and knows how far on its next is, so that no place is
// divided for again.  One launch for both operands.  Rows of x or dy: the threads go through the
// vectors.  Weights: 2^`log` neighbouring threads take `per` vectors each of one of the `segs` parts of
// a row, and pass over groups without rows of x (57 groups of 1718 -> 3496, one row: 218 us with all
// of them, 21 so).  Small parts keep the threads busy where there are few rows, large ones pass over
// more at a step.
struct Pack {
  const uint16_t* src;
  uint4* dst;
  const int* offsets;                                     // of the weights' groups, or nullptr: one matrix
  int64_t all;                                            // its vectors
  int64_t ld, gs;
  int groups, per_group, sg, sr;                          // a thread's next row: sg groups, sr rows further
  int sv;                                                 // and vectors (weights: parts)
  int segs, per;
  int cols, pitch8, log, bytes;                           // bytes of a load
  int rows;                                               // that the offsets may reach
};
struct Packs {
  Pack of[2];
  int blocks;                                             // of the first
};
template <typename W>
__device__ __forceinline__ uint4 pack_vector(const uint16_t* s, int left) {
  constexpr int N = sizeof(W) / 2;
  uint4 out = make_uint4(0, 0, 0, 0);
  uint16_t* o = reinterpret_cast<uint16_t*>(&out);
#pragma unroll
  for (int e = 0; e < 8; e += N) {
    if (e + N <= left) {
      const W w = *reinterpret_cast<const W*>(s + e);
#pragma unroll
      for (int x = 0; x < N; ++x) o[e + x] = reinterpret_cast<const uint16_t*>(&w)[x];
    } else {
#pragma unroll
      for (int x = 0; x < N; ++x)
        if (e + x < left) o[e + x] = s[e + x];
    }
  }
  return out;
}
__device__ __forceinline__ uint4 pack_of(const Pack& a, const uint16_t* s, int v) {
  const int left = a.cols - v * 8;
  return a.bytes == 8 ? pack_vector<uint2>(s + v * 8, left)
         : a.bytes == 4 ? pack_vector<uint32_t>(s + v * 8, left) : pack_vector<uint16_t>(s + v * 8, left);
}
__device__ __forceinline__ void pack_matrix(const Pack& a, uint32_t block, uint32_t blocks) {
  const uint32_t first = block * 256 + threadIdx.x;
  int r = static_cast<int>(first / static_cast<uint32_t>(a.pitch8));
  int v = static_cast<int>(first - static_cast<uint32_t>(r) * a.pitch8);
  for (int64_t i = first; i < a.all; i += blocks * 256) {
    a.dst[i] = pack_of(a, a.src + r * a.ld, v);
    r += a.sr;
    v += a.sv;
    if (v >= a.pitch8) {
      v -= a.pitch8;
      ++r;
    }
  }
}
__device__ __forceinline__ void pack_weights(const Pack& a, uint32_t block) {
  const uint32_t first = (block * 256 + threadIdx.x) >> a.log, row = first / static_cast<uint32_t>(a.segs);
  const int lane = threadIdx.x & ((1 << a.log) - 1);
  int seg = static_cast<int>(first - row * a.segs), g = static_cast<int>(row / static_cast<uint32_t>(a.per_group));
  int r = static_cast<int>(row - static_cast<uint32_t>(g) * a.per_group);
  while (g < a.groups) {
    if (min(max(a.offsets[g], 0), a.rows) < min(max(a.offsets[g + 1], 0), a.rows)) {
      const uint16_t* s = a.src + g * a.gs + r * a.ld;
      uint4* d = a.dst + (static_cast<int64_t>(g) * a.per_group + r) * a.pitch8;
      const int end = min(a.pitch8, ((seg + 1) * a.per) << a.log);
      int v = ((seg * a.per) << a.log) + lane;
#pragma unroll 1
      do {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int w = v + (x << a.log);
          if (w < end) d[w] = pack_of(a, s, w);
        }
        v += 2 << a.log;
      } while (v < end);
    }
    g += a.sg;
    r += a.sr;
    seg += a.sv;
    if (seg >= a.segs) {
      seg -= a.segs;
      ++r;
    }
    if (r >= a.per_group) {
      r -= a.per_group;
      ++g;
    }
  }
}
__global__ void __launch_bounds__(256) k_pack(const __grid_constant__ Packs both) {
  const uint32_t second = blockIdx.x >= static_cast<uint32_t>(both.blocks);
  const uint32_t block = blockIdx.x - (second ? both.blocks : 0);
  const Pack& a = both.of[second];
  if (a.offsets)
    pack_weights(a, block);
  else
    pack_matrix(a, block, second ? gridDim.x - both.blocks : both.blocks);
}

// A split weights' gradient: dW and db are the sums of their parts, in the parts' order.
struct Join {
  const float *part, *part_db;      // [groups, split, outer, pitch] and [groups, split, outer]
  void* out;
  float* db;
  int64_t out_ld, out_gs, db_ld;
  int groups, split, outer, inner, pitch, type;
};
__global__ void __launch_bounds__(256) k_join(const Join a) {
  const int quads = a.pitch / 4;
  const int64_t all = static_cast<int64_t>(a.groups) * a.outer * quads, step = gridDim.x * 256ll;
  const int64_t slice = static_cast<int64_t>(a.outer) * a.pitch;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < all; i += step) {
    const int64_t row = i / quads, g = row / a.outer;
    const int f = static_cast<int>(row - g * a.outer), c = static_cast<int>(i - row * quads) * 4;
    const float* p = a.part + g * a.split * slice + static_cast<int64_t>(f) * a.pitch + c;
    float4 sum = *reinterpret_cast<const float4*>(p);
#pragma unroll 4
    for (int q = 1; q < a.split; ++q) {
      const float4 w = *reinterpret_cast<const float4*>(p + q * slice);
      sum.x += w.x;
      sum.y += w.y;
      sum.z += w.z;
      sum.w += w.w;
    }
    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
    const int64_t o = g * a.out_gs + f * a.out_ld + c;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (c + x >= a.inner) break;
      if (a.type == HA_TYPE_FP32)
        static_cast<float*>(a.out)[o + x] = v[x];
      else
        static_cast<uint16_t*>(a.out)[o + x] = narrow(v[x], a.type);
    }
  }
  if (!a.db) return;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < static_cast<int64_t>(a.groups) * a.outer; i += step) {
    const int64_t g = i / a.outer, f = i - g * a.outer;
    float sum = 0.0f;
    for (int q = 0; q < a.split; ++q) sum += a.part_db[(g * a.split + q) * a.outer + f];
    a.db[g * a.db_ld + f] = sum;
  }
}

constexpr int kSms = 152;
// Groups of at most this many rows on average (the offsets are on the device: the host knows no more)
// take the tiles for few rows.  32 groups, 4096 to 4096, bf16: 32 rows each 165 us, by pairs 173; 40 rows
// each 222 and 175.
constexpr int kFewRows = 32;
int64_t round8(int64_t x) { return (x + 7) / 8 * 8; }
int64_t round256(int64_t x) { return (x + 255) / 256 * 256; }

// Parts of each group's rows in the weights' gradient: where its tiles are fewer than half of the
// pairs of SMs, as many as give every pair a tile, with at least kMinChunks chunks each on average
// (one group, 30000 rows, 1024 -> 1000, fp32: 151 us with one part, 53 with 4).
int dw_split(int groups, int64_t rows, int inner, int outer) {
  const int64_t tiles = groups * static_cast<int64_t>((outer + 2 * kM - 1) / (2 * kM)) * ((inner + kPairCols - 1) / kPairCols);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kSms / 2 / tiles, rows / groups / (kK * kMinChunks))));
}
struct Parts {
  int split, pitch;
  int64_t dw, db;                   // bytes
  Parts(int groups, int64_t rows, int inner, int outer) : split(dw_split(groups, rows, inner, outer)), pitch(0), dw(0), db(0) {
    if (split == 1) return;
    pitch = (inner + 3) / 4 * 4;
    dw = round256(static_cast<int64_t>(groups) * split * outer * pitch * 4);
    db = round256(static_cast<int64_t>(groups) * split * outer * 4);
  }
  int64_t bytes() const { return dw + db; }
};

// One operand as the tensor maps need it: address, strides and width multiples of 16 bytes (the
// edge of a map is only sure to cut whole 16-byte pieces), and no two entries in one place (what
// a map with overlapping dimensions cuts off is not safe from being touched).
struct Operand {
  const void* p;
  int64_t groups, rows, cols, ld, gs;   // gs: between groups (groups > 1)
  bool apart() const {                  // groups after one another, or their rows in turn
    return gs >= (rows - 1) * ld + cols || (gs >= cols && ld >= (groups - 1) * gs + cols);
  }
  bool fits() const {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0 && cols % 8 == 0 &&
           (groups == 1 || (gs % 8 == 0 && apart()));   // one matrix for all groups is copied
  }
  int64_t packed_bytes() const { return fits() ? 0 : round256(groups * rows * round8(cols) * 2); }
};

// Copies those of two operands that do not fit to ws, which moves on.  Offsets (or nullptr): of the
// second's groups, up to `rows`.
cudaError_t pack(Operand& x, Operand& y, const int* offsets, int rows, unsigned char*& ws, cudaStream_t s) {
  Packs p = {};
  int count = 0;
  unsigned blocks[2] = {0, 0};
  for (Operand* o : {&x, &y}) {
    if (o->fits()) continue;
    const int64_t pitch = round8(o->cols);
    Pack& a = p.of[count];
    a.src = static_cast<const uint16_t*>(o->p);
    a.dst = reinterpret_cast<uint4*>(ws);
    a.cols = static_cast<int>(o->cols);
    a.pitch8 = static_cast<int>(pitch / 8);
    a.ld = o->ld;
    a.gs = o->gs;
    a.groups = static_cast<int>(o->groups);
    a.per_group = static_cast<int>(o->rows);
    a.offsets = o == &y ? offsets : nullptr;
    a.rows = rows;
    const auto grid = [](int64_t threads) { return static_cast<unsigned>(std::min<int64_t>((threads + 255) / 256, 16 * kSms)); };
    if (a.offsets) {
      while (a.log < 5 && 2 << a.log < a.pitch8) ++a.log;
      const int64_t lanes = o->groups * o->rows << a.log;
      a.per = 2;
      while (a.per < 16 && lanes * ((a.pitch8 >> a.log) / a.per) > 64 * kSms * 256) a.per *= 2;
      a.segs = (a.pitch8 + (a.per << a.log) - 1) / (a.per << a.log);
      blocks[count] = grid(o->groups * o->rows * a.segs << a.log);
      const int64_t step = static_cast<int64_t>(blocks[count]) * 256 >> a.log, rows_on = step / a.segs;
      a.sv = static_cast<int>(step % a.segs);
      a.sr = static_cast<int>(rows_on % o->rows);
      a.sg = static_cast<int>(rows_on / o->rows);
    } else {
      a.all = o->rows * a.pitch8;
      blocks[count] = grid(a.all);
      a.sr = static_cast<int>(blocks[count] * 256 / a.pitch8);
      a.sv = static_cast<int>(blocks[count] * 256 % a.pitch8);
    }
    const uintptr_t low = reinterpret_cast<uintptr_t>(o->p) | static_cast<uintptr_t>(o->ld * 2) |
                          static_cast<uintptr_t>(o->groups > 1 ? o->gs * 2 : 0);
    a.bytes = (low & 7) == 0 ? 8 : (low & 3) == 0 ? 4 : 2;
    ++count;
    ws += o->packed_bytes();
    o->p = a.dst;
    o->ld = pitch;
    o->gs = o->rows * pitch;
  }
  if (count == 0) return cudaSuccess;
  p.blocks = static_cast<int>(blocks[0]);
  k_pack<<<blocks[0] + blocks[1], 256, 0, s>>>(p);
  return cudaGetLastError();
}

// Three dimensions always; box {b0, b1, 1}.
bool make_map(CUtensorMap* m, const Operand& o, int type, uint32_t b0, uint32_t b1) {
  const EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  const int es = type_size(type);
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(o.cols), static_cast<cuuint64_t>(o.rows),
                              static_cast<cuuint64_t>(o.groups)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(o.ld * es),
                                 static_cast<cuuint64_t>((o.groups == 1 ? o.rows * o.ld : o.gs) * es)};
  const cuuint32_t box[3] = {b0, b1, 1}, one[3] = {1, 1, 1};
  const CUtensorMapDataType dt = type == HA_TYPE_FP32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                 : type == HA_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                        : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return enc(m, dt, 3, const_cast<void*>(o.p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Clusters of `size` CTAs that the GPU holds at once.
template <typename K>
int clusters_held(K kernel, int threads, int smem, int size) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kSms / size * size);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  return cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess ? n : 0;
}

// `tiles`: about how many there are; `most`: at most.
template <int MODE, bool WIDE, int NT>
int launch_one(const CUtensorMap& ta, const CUtensorMap& tb, const Args& a, int64_t tiles, int64_t most, cudaStream_t s) {
  const auto kernel = k_grouped_one<MODE, WIDE, NT>;
  constexpr int smem = One<NT>::kSmem;
  static bool allowed[kMaxDevices];
  if (allow_smem(kernel, smem, allowed) != cudaSuccess) return HA_ECUDA;
  // CTAs a tile: as many as fill the GPU, with at least kMinChunks chunks each (one row, 4096 ->
  // 4096: 18.2 us with one CTA a tile).
  static int held[kMaxDevices][4];
  int split = 1, log = 0;
  while (split < kMaxSplit && tiles * split * 2 <= kSms && (a.k + kK - 1) / kK >= split * 2 * kMinChunks) {
    split *= 2;
    ++log;
  }
  const int device = device_slot();
  int once = 0, &found = device >= 0 ? held[device][log] : once;
  if (found == 0) found = split == 1 ? kSms : clusters_held(kernel, kThreads, smem, split);
  if (found < 1) return HA_ECUDA;
  const int64_t clusters = std::min<int64_t>(found, std::max<int64_t>(most, 1));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(clusters * split));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = split;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, ta, tb, a) == cudaSuccess ? HA_OK : HA_ECUDA;
}

template <int MODE, int RES>
int launch_pair_of(const CUtensorMap& ta, const CUtensorMap& tb, const Ends<MODE>& ends, const Args& a, int64_t most,
                   cudaStream_t s) {
  static bool allowed[kMaxDevices];
  if (allow_smem(k_grouped_pair<MODE, RES>, Pair::kSmem, allowed) != cudaSuccess) return HA_ECUDA;
  // As many pairs as the GPU holds at once (its clusters of two leave some SMs out): the tiles
  // are dealt out in advance, so a pair that started late would finish late.
  constexpr int threads = MODE == kDw ? kDwThreads : kThreads;
  static int held[kMaxDevices];
  const int device = device_slot();
  int once = 0, &found = device >= 0 ? held[device] : once;
  if (found == 0) found = clusters_held(k_grouped_pair<MODE, RES>, threads, Pair::kSmem, 2);
  if (found < 1) return HA_ECUDA;
  const int64_t pairs = std::min<int64_t>(found, std::max<int64_t>(most, 1));
  k_grouped_pair<MODE, RES><<<static_cast<unsigned>(2 * pairs), threads, Pair::kSmem, s>>>(ta, tb, ends, a);
  return cudaGetLastError() == cudaSuccess ? HA_OK : HA_ECUDA;
}

// A sum of this many values at most stays whole in a 16-bit result: what truncating costs is then an
// eighth of the type's rounding at worst.  (The gradient of weights of 32 groups, 16384
// rows, 4096 to 4096, bf16: 391 us whole, 425 folded; of 8 groups, 65536 rows, 2048 to 2048: 297 and 301.)
int64_t whole_sum(int type) { return type == HA_TYPE_BF16 ? 65536 : 8192; }
template <int MODE>
int launch_pair(const CUtensorMap& ta, const CUtensorMap& tb, const Ends<MODE>& ends, const Args& a, int64_t length,
                int64_t most, cudaStream_t s) {
  if (a.out_type == HA_TYPE_FP32) return launch_pair_of<MODE, kWide>(ta, tb, ends, a, most, s);
  if (length > whole_sum(a.out_type)) return launch_pair_of<MODE, kFolded>(ta, tb, ends, a, most, s);
  return launch_pair_of<MODE, kWhole>(ta, tb, ends, a, most, s);
}

bool half_type(int t) { return t == HA_TYPE_BF16 || t == HA_TYPE_FP16; }
bool out_type_ok(int in, int out) { return out == in || out == HA_TYPE_FP32; }

bool sizes_ok(int type, int groups, int64_t rows, int inner, int outer) {
  return half_type(type) && groups >= 1 && rows >= 0 && rows <= (1 << 30) && inner >= 1 &&
         outer >= 1 && inner <= (1 << 24) && outer <= (1 << 24);
}
bool even(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 1) == 0; }

// y = act(x W^T + b) (kFwd) or dx = dy W, masked (kDx): rows of x.cols values to a.m features.
template <int MODE>
int rows_product(Operand x, Operand w, Args a, void* ws, int64_t ws_bytes, cudaStream_t s) {
  if (x.packed_bytes() + w.packed_bytes() > ws_bytes) return HA_ENOMEM;
  if (ws_bytes > 0 && (!ws || (reinterpret_cast<uintptr_t>(ws) & 15))) return HA_EINVAL;
  unsigned char* p = static_cast<unsigned char*>(ws);
  if (pack(x, w, a.offsets, a.rows, p, s) != cudaSuccess) return HA_ECUDA;
  a.wide_out = (reinterpret_cast<uintptr_t>(a.out) & 15) == 0 && a.out_ld * type_size(a.out_type) % 16 == 0;
  a.wide_h = a.h && (reinterpret_cast<uintptr_t>(a.h) & 15) == 0 && a.h_ld % 8 == 0;
  const bool wide = a.out_type == HA_TYPE_FP32;
  const int64_t rows = a.rows, used = std::min<int64_t>(rows, a.groups);      // groups with rows, about
  const int64_t m1 = (a.m + kM - 1) / kM, m2 = (a.m + 2 * kM - 1) / (2 * kM);
  // Few rows a group: narrow tiles.  So few rows in all that pairs would leave most SMs idle: tiles of
  // one CTA, twice as many and four times as narrow, as long as one for each SM is enough (one group,
  // 512 rows, 4096 to 2304, 144 tiles: 21.2 us, by pairs 25.3; to 2560, 160 tiles: 36.5 and 25.4).
  const bool few = rows <= kFewRows * static_cast<int64_t>(a.groups);
  const int64_t narrow = m1 * used * ((rows + 64 * used - 1) / (64 * used));
  const bool small = narrow <= kSms;
  if (m1 * std::min<int64_t>(rows, a.groups + rows / 32) > 0x7FFFFFFF) return HA_EUNSUPPORTED;    // tiles
  CUtensorMap ta, tb;
  if (!make_map(&ta, w, a.in_type, 64, MODE == kFwd ? 128 : 64) ||
      !make_map(&tb, x, a.in_type, 64, few || small ? 16 : 64))
    return HA_ECUDA;
  if (few) {
    const int64_t tiles = m1 * used, most = m1 * std::min<int64_t>(rows, a.groups + rows / 32);
    return wide ? launch_one<MODE, true, 32>(ta, tb, a, tiles, most, s)
                : launch_one<MODE, false, 32>(ta, tb, a, tiles, most, s);
  }
  if (small) {
    const int64_t most = m1 * std::min<int64_t>(rows, a.groups + rows / 64);
    return wide ? launch_one<MODE, true, 64>(ta, tb, a, narrow, most, s)
                : launch_one<MODE, false, 64>(ta, tb, a, narrow, most, s);
  }
  const int64_t most = m2 * std::min<int64_t>(rows, a.groups + rows / kPairCols);
  return launch_pair<MODE>(ta, tb, {}, a, a.k, most, s);
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" int hier_avg_grouped_product_workspace(int op, const void* a_dev, int64_t a_ld,
                                                  const void* b_dev, int64_t b_ld, int64_t b_gs,
                                                  int groups, int64_t rows, int inner, int outer,
                                                  int64_t* bytes) {
  if (!bytes || !sizes_ok(HA_TYPE_BF16, groups, rows, inner, outer)) return HA_EINVAL;
  const Operand x = {a_dev, 1, rows, op == HA_GROUPED_FORWARD ? inner : outer, a_ld, 0};
  Operand b = {b_dev, groups, outer, inner, b_ld, b_gs};
  if (op == HA_GROUPED_DW)
    b = {b_dev, 1, rows, inner, b_ld, 0};
  else if (op != HA_GROUPED_FORWARD && op != HA_GROUPED_DX)
    return HA_EINVAL;
  *bytes = x.packed_bytes() + b.packed_bytes();
  if (op == HA_GROUPED_DW) *bytes += Parts(groups, rows, inner, outer).bytes();
  return HA_OK;
}

extern "C" int hier_avg_grouped_product(const void* x_dev, int64_t x_ld, const void* w_dev,
                                        int64_t w_ld, int64_t w_gs, int type,
                                        const int32_t* offsets_dev, int groups, int64_t rows,
                                        int inner, int outer, const float* bias_dev, int64_t bias_ld,
                                        int relu, void* y_dev, int64_t y_ld, int y_type,
                                        void* workspace_dev, int64_t workspace_bytes, void* stream) {
  if (!sizes_ok(type, groups, rows, inner, outer) || !out_type_ok(type, y_type)) return HA_EINVAL;
  if (x_ld < inner || w_ld < inner || y_ld < outer || !even(x_dev) || !even(w_dev) ||
      reinterpret_cast<uintptr_t>(y_dev) % type_size(y_type) || workspace_bytes < 0)
    return HA_EINVAL;
  if (groups > kMaxGroups) return HA_EUNSUPPORTED;
  if (rows == 0) return HA_OK;
  if (!x_dev || !w_dev || !offsets_dev || !y_dev) return HA_EINVAL;
  Args a = {};
  a.offsets = offsets_dev;
  a.out = y_dev;
  a.bias = bias_dev;
  a.bias_ld = bias_ld;
  a.out_ld = y_ld;
  a.groups = groups;
  a.rows = static_cast<int>(rows);
  a.m = outer;
  a.k = inner;
  a.in_type = type;
  a.out_type = y_type;
  a.relu = relu != 0;
  return rows_product<kFwd>({x_dev, 1, rows, inner, x_ld, 0}, {w_dev, groups, outer, inner, w_ld, w_gs},
                            a, workspace_dev, workspace_bytes, static_cast<cudaStream_t>(stream));
}

extern "C" int hier_avg_grouped_product_dx(const void* dy_dev, int64_t dy_ld, const void* w_dev,
                                           int64_t w_ld, int64_t w_gs, int type,
                                           const int32_t* offsets_dev, int groups, int64_t rows,
                                           int inner, int outer, const void* h_dev, int64_t h_ld,
                                           void* dx_dev, int64_t dx_ld, int dx_type,
                                           void* workspace_dev, int64_t workspace_bytes,
                                           void* stream) {
  if (!sizes_ok(type, groups, rows, inner, outer) || !out_type_ok(type, dx_type)) return HA_EINVAL;
  if (dy_ld < outer || w_ld < inner || dx_ld < inner || !even(dy_dev) || !even(w_dev) || !even(h_dev) ||
      (h_dev && h_ld < inner) || reinterpret_cast<uintptr_t>(dx_dev) % type_size(dx_type) ||
      workspace_bytes < 0)
    return HA_EINVAL;
  if (groups > kMaxGroups) return HA_EUNSUPPORTED;
  if (rows == 0) return HA_OK;
  if (!dy_dev || !w_dev || !offsets_dev || !dx_dev) return HA_EINVAL;
  Args a = {};
  a.offsets = offsets_dev;
  a.out = dx_dev;
  a.h = h_dev;
  a.h_ld = h_ld;
  a.out_ld = dx_ld;
  a.groups = groups;
  a.rows = static_cast<int>(rows);
  a.m = inner;
  a.k = outer;
  a.in_type = type;
  a.out_type = dx_type;
  return rows_product<kDx>({dy_dev, 1, rows, outer, dy_ld, 0}, {w_dev, groups, outer, inner, w_ld, w_gs},
                           a, workspace_dev, workspace_bytes, static_cast<cudaStream_t>(stream));
}

extern "C" int hier_avg_grouped_product_dw(const void* dy_dev, int64_t dy_ld, const void* x_dev,
                                           int64_t x_ld, int type, const int32_t* offsets_dev,
                                           int groups, int64_t rows, int inner, int outer,
                                           void* dw_dev, int64_t dw_ld, int64_t dw_gs, int dw_type,
                                           float* db_dev, int64_t db_ld, void* workspace_dev,
                                           int64_t workspace_bytes, void* stream) {
  if (!sizes_ok(type, groups, rows, inner, outer) || !out_type_ok(type, dw_type)) return HA_EINVAL;
  if (dy_ld < outer || x_ld < inner || dw_ld < inner || !even(dy_dev) || !even(x_dev) ||
      reinterpret_cast<uintptr_t>(dw_dev) % type_size(dw_type) || (db_dev && db_ld < outer) ||
      workspace_bytes < 0)
    return HA_EINVAL;
  if (groups > kMaxGroups) return HA_EUNSUPPORTED;
  if (!offsets_dev || !dw_dev || (rows > 0 && (!dy_dev || !x_dev))) return HA_EINVAL;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  Operand dy = {dy_dev, 1, rows, outer, dy_ld, 0}, x = {x_dev, 1, rows, inner, x_ld, 0};
  if (rows == 0) {
    // The maps below need an address and a row; nothing is read, since every group is empty.
    const void* p16 = reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(dw_dev) & ~uintptr_t(15));
    dy = x = {p16, 1, 1, 8, 8, 0};
  }
  const Parts parts(groups, rows, inner, outer);
  if (dy.packed_bytes() + x.packed_bytes() + parts.bytes() > workspace_bytes) return HA_ENOMEM;
  if (workspace_bytes > 0 && (!workspace_dev || (reinterpret_cast<uintptr_t>(workspace_dev) & 15)))
    return HA_EINVAL;
  unsigned char* p = static_cast<unsigned char*>(workspace_dev);
  if (pack(dy, x, nullptr, 0, p, s) != cudaSuccess) return HA_ECUDA;
  Args a = {};
  a.offsets = offsets_dev;
  a.out = dw_dev;
  a.db = db_dev;
  a.bias_ld = db_ld;
  a.out_ld = dw_ld;
  a.out_gs = dw_gs;
  a.groups = groups * parts.split;
  a.split = parts.split;
  a.rows = static_cast<int>(rows);
  a.m = outer;
  a.n = inner;
  a.in_type = type;
  a.out_type = dw_type;
  const int es = type_size(dw_type);
  a.wide_out = (reinterpret_cast<uintptr_t>(dw_dev) & 15) == 0 && dw_ld * es % 16 == 0 && inner * es % 16 == 0 &&
               (groups == 1 || dw_gs * es % 16 == 0);
  if (parts.split > 1) {
    a.out = p;
    a.out_ld = parts.pitch;
    a.out_gs = static_cast<int64_t>(outer) * parts.pitch;
    a.out_type = HA_TYPE_FP32;
    a.wide_out = 1;                 // what is past a row's end is not read
    if (db_dev) {
      a.db = reinterpret_cast<float*>(p + parts.dw);
      a.bias_ld = outer;
    }
  }
  CUtensorMap ta, tb;
  Ends<kDw> ends;
  if (!make_map(&ta, dy, type, 64, 64) || !make_map(&tb, x, type, 64, 64) || !make_map(&ends.a, dy, type, 64, 16) ||
      !make_map(&ends.b, x, type, 64, 16))
    return HA_ECUDA;
  const int64_t most = a.groups * static_cast<int64_t>((outer + 2 * kM - 1) / (2 * kM)) *
                       ((inner + kPairCols - 1) / kPairCols + (db_dev ? 1 : 0));
  if (most > 0x7FFFFFFF) return HA_EUNSUPPORTED;
  // the groups' lengths are not known here: one of them may have all rows
  const int status = launch_pair<kDw>(ta, tb, ends, a, rows, most, s);
  if (status != HA_OK || parts.split == 1) return status;
  Join j = {};
  j.part = static_cast<const float*>(a.out);
  j.part_db = a.db;
  j.out = dw_dev;
  j.db = db_dev;
  j.out_ld = dw_ld;
  j.out_gs = dw_gs;
  j.db_ld = db_ld;
  j.groups = groups;
  j.split = parts.split;
  j.outer = outer;
  j.inner = inner;
  j.pitch = parts.pitch;
  j.type = dw_type;
  const int64_t quads = static_cast<int64_t>(groups) * outer * (parts.pitch / 4);
  k_join<<<static_cast<unsigned>(std::min<int64_t>((quads + 255) / 256, 8 * kSms)), 256, 0, s>>>(j);
  return cudaGetLastError() == cudaSuccess ? HA_OK : HA_ECUDA;
}

extern "C" int hier_avg_operator_check(void* stream) {
  if (cudaStreamSynchronize(static_cast<cudaStream_t>(stream)) != cudaSuccess) return HA_ECUDA;
  int word = 0;
  if (cudaMemcpyFromSymbol(&word, g_operator_error, sizeof word) != cudaSuccess) return HA_ECUDA;
  if (!word) return HA_OK;
  const int zero = 0;
  if (cudaMemcpyToSymbol(g_operator_error, &zero, sizeof zero) != cudaSuccess) return HA_ECUDA;
  return HA_ETIMEOUT;
}
