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
constexpr int kM = 128;                 // features of a tile
constexpr int kK = 64;                  // values summed over in a chunk: one 128-byte line
constexpr int kMaxGroups = 1024;
constexpr int kEpiWarps = 8;            // two groups of four: a group reads half the columns
constexpr int kThreads = (kEpiWarps + 2) * 32;
// fp32 results: the tensor core's running sum is taken into fp32 registers after this many
// chunks.  Its additions truncate; over a sum of 4096 random products that cost 4.4e-6 of the
// result's norm, over 16384 1.9e-5, over 512 4.7e-7 (fp32 additions: 6.1e-7, 1.5e-6 and 1.6e-7).
// A 16-bit result does not see it.
constexpr int kFold = 8;

struct Args {
  const int* offsets;
  void* out;
  const float* bias;          // forward, or nullptr
  const void* h;              // gradient of rows: the mask's activations, or nullptr
  int64_t out_ld, out_gs;     // in elements; out_gs: between groups of dW
  int64_t bias_ld, h_ld;
  int groups, rows;
  int m, n, k;                // features; dW: columns; summed length (forward, rows)
  int in_type, out_type;
  int relu;
  int wide_out;               // 16-byte stores of the output are aligned
};

struct Tile {
  int g, m0, c0, cols, r0, k;   // group, first feature, first column, columns, first row, length
};

// Column tiles of a group of n rows: as few as fit, of equal size.
__device__ __forceinline__ int col_tiles(int n, int NT) { return (n + NT - 1) / NT; }

// Element types of a kind::f16 MMA: bits 7-9 and 10-12 of the instruction descriptor.
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
__device__ __forceinline__ bool positive16(uint16_t w, int type) {   // > 0, not NaN
  return w != 0 && w <= (type == HA_TYPE_BF16 ? 0x7F80u : 0x7C00u);
}

template <int NT> struct Shape {
  static constexpr int kA = kM * kK * 2;                 // bytes of a chunk of the weights
  static constexpr int kB = NT * kK * 2;
  static constexpr int kStages = NT == 256 ? 4 : 6;
  static constexpr int kBoxRows = NT == 256 ? 64 : 16;   // rows of a load of x or dy
  static constexpr int kStage = 8192;                    // results on their way out, per warp group
  static constexpr int kTmem = 2 * NT;
  static constexpr int kSmem = kStages * (kA + kB) + 2 * kStage + 1024;
};

struct Shared {
  uint64_t full[8], empty[8], tfull[2], tempty[2];
  uint32_t tmem;
  int off[kMaxGroups + 1];      // rows of each group, inside [0, rows]
  int first[kMaxGroups + 1];    // first tile of each group
};

template <int MODE, int NT>
__device__ __forceinline__ Tile tile_at(const Shared& s, const Args& a, int i) {
  int lo = 0, hi = a.groups;             // first[lo] <= i < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s.first[mid] <= i) lo = mid; else hi = mid;
  }
  const int mt = (a.m + kM - 1) / kM, at = i - s.first[lo];
  Tile t;
  t.g = lo;
  t.m0 = at % mt * kM;
  const int ct = at / mt, n = max(0, s.off[lo + 1] - s.off[lo]);
  if (MODE == kDw) {
    t.c0 = ct * NT;
    t.cols = min(NT, a.n - t.c0);
    t.r0 = s.off[lo];
    t.k = n;
  } else {
    const int parts = col_tiles(n, NT), size = ((n + parts - 1) / parts + 15) / 16 * 16;
    t.c0 = s.off[lo] + ct * size;
    t.cols = min(size, n - ct * size);
    t.r0 = t.c0;
    t.k = a.k;
  }
  return t;
}

// The rows that no group covers are zero.
__device__ void clear_rows(const Args& a, int64_t begin, int64_t end) {
  const int64_t per = a.m;
  for (int64_t r = begin + blockIdx.x; r < end; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < per; c += kThreads) {
      if (a.out_type == HA_TYPE_FP32)
        static_cast<float*>(a.out)[r * a.out_ld + c] = 0.0f;
      else
        static_cast<uint16_t*>(a.out)[r * a.out_ld + c] = 0;
    }
}

template <int MODE, int NT>
__global__ void __launch_bounds__(kThreads, 1)
    k_grouped(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb,
              const __grid_constant__ Args a) {
  using S = Shape<NT>;
  extern __shared__ unsigned char raw[];
  __shared__ Shared sh;
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  unsigned char* As = base;
  unsigned char* Bs = base + S::kStages * S::kA;
  unsigned char* Out = base + S::kStages * (S::kA + S::kB);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  // ---- the list of tiles
  for (int g = tid; g <= a.groups; g += kThreads) sh.off[g] = min(max(a.offsets[g], 0), a.rows);
  if (warp == kEpiWarps) tmem_alloc(&sh.tmem, S::kTmem);
  if (tid == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.tfull[i], 1);
      mbar_init(&sh.tempty[i], kEpiWarps);
    }
    fence_barrier_init();
  }
  __syncthreads();
  if (warp == 0) {
    const int mt = (a.m + kM - 1) / kM, nt = (a.n + NT - 1) / NT;
    int run = 0;
    for (int g0 = 0; g0 < a.groups; g0 += 32) {
      const int g = g0 + lane;
      // offsets that go back leave a group empty
      const int n = g < a.groups ? max(0, sh.off[g + 1] - sh.off[g]) : 0;
      const int tiles = MODE == kDw ? (g < a.groups ? mt * nt : 0) : mt * col_tiles(n, NT);
      int x = tiles;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(~0u, x, o);
        if (lane >= o) x += y;
      }
      if (g < a.groups) sh.first[g] = run + x - tiles;
      run += __shfl_sync(~0u, x, 31);
    }
    if (lane == 0) sh.first[a.groups] = run;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  const int tiles = sh.first[a.groups];
  if (MODE != kDw) {
    clear_rows(a, 0, sh.off[0]);
    clear_rows(a, sh.off[a.groups], a.rows);
  }

  if (warp == kEpiWarps) {
    // ---- loads
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
        const Tile t = tile_at<MODE, NT>(sh, a, i);
        const int nk = (t.k + kK - 1) / kK;
        const int boxes = MODE == kDw ? (t.cols + 63) / 64 : (t.cols + S::kBoxRows - 1) / S::kBoxRows;
        const uint32_t bytes = S::kA + boxes * (MODE == kDw ? 64 : S::kBoxRows) * 128;
        for (int c = 0; c < nk; ++c, ++it) {
          const int st = it % S::kStages;
          if (!mbar_wait(&sh.empty[st], ((it / S::kStages) & 1) ^ 1, &g_operator_error)) { ok = false; break; }
          uint64_t* bar = &sh.full[st];
          mbar_arrive_expect_tx(bar, bytes);
          unsigned char* A = As + st * S::kA;
          unsigned char* B = Bs + st * S::kB;
          if (MODE == kFwd) {
            tma_load_3d(A, &ta, bar, c * kK, t.m0, t.g);
          } else if (MODE == kDx) {
            tma_load_3d(A, &ta, bar, t.m0, c * kK, t.g);
            tma_load_3d(A + 8192, &ta, bar, t.m0 + 64, c * kK, t.g);
          } else {
            tma_load_2d(A, &ta, bar, t.m0, t.r0 + c * kK);
            tma_load_2d(A + 8192, &ta, bar, t.m0 + 64, t.r0 + c * kK);
          }
          for (int b = 0; b < boxes; ++b) {
            if (MODE == kDw)
              tma_load_2d(B + b * 8192, &tb, bar, t.c0 + b * 64, t.r0 + c * kK);
            else
              tma_load_2d(B + b * S::kBoxRows * 128, &tb, bar, c * kK, t.r0 + b * S::kBoxRows);
          }
        }
      }
    }
  } else if (warp == kEpiWarps + 1) {
    // ---- matrix products
    uint32_t it = 0, seg = 0;
    bool ok = true;
    const int fold = a.out_type == HA_TYPE_FP32 ? kFold : 0x7FFFFFFF;
    for (int i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
      const Tile t = tile_at<MODE, NT>(sh, a, i);
      const int nk = (t.k + kK - 1) / kK;
      const int N = (t.cols + 15) / 16 * 16;
      uint32_t idesc = idesc_of(a.in_type, kM, N);
      if (MODE != kFwd) idesc |= 1u << 15;
      if (MODE == kDw) idesc |= 1u << 16;
      for (int c = 0; c < nk && ok; ++c, ++it) {
        const int buf = seg & 1;
        if (c % fold == 0) {
          ok = mbar_wait(&sh.tempty[buf], ((seg >> 1) & 1) ^ 1, &g_operator_error);
          if (!ok) break;
          tc_fence_after();
        }
        const int st = it % S::kStages;
        ok = mbar_wait(&sh.full[st], (it / S::kStages) & 1, &g_operator_error);
        if (!ok) break;
        tc_fence_after();
        const int left = t.k - c * kK, steps = left >= kK ? kK / 16 : (left + 15) / 16;
        unsigned char* A = As + st * S::kA;
        unsigned char* B = Bs + st * S::kB;
        if (MODE == kDw && left < kK && (left & 15)) {
          // The rows after the group's last are another group's: cleared up to the step's end.
          const int blocks = 2 + (t.cols + 63) / 64;
          const int r0 = left, r1 = steps * 16;
          for (int x = lane; x < blocks * (r1 - r0) * 8; x += 32) {
            const int line = x >> 3, b = line / (r1 - r0), r = r0 + line % (r1 - r0);
            unsigned char* p = (b < 2 ? A + b * 8192 : B + (b - 2) * 8192) + r * 128 + (x & 7) * 16;
            *reinterpret_cast<uint4*>(p) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async_smem();
          __syncwarp();
        }
        if (lane == 0) {
          const uint32_t as = smem_u32(A), bs = smem_u32(B);
          for (int k = 0; k < steps; ++k) {
            const uint64_t da = MODE == kFwd ? umma_desc_sw128(as + k * 32) : umma_desc_sw128_mn(as + k * 2048, 8192);
            const uint64_t db = MODE == kDw ? umma_desc_sw128_mn(bs + k * 2048, 8192) : umma_desc_sw128(bs + k * 32);
            tc_mma_bf16(tmem + buf * NT, da, db, idesc, (c % fold) || k ? 1u : 0u);
          }
          tc_commit(&sh.empty[st]);
          if (c % fold == fold - 1 || c == nk - 1) tc_commit(&sh.tfull[buf]);
        }
        __syncwarp();
        if (c % fold == fold - 1 || c == nk - 1) ++seg;
      }
    }
  } else {
    // ---- results
    uint32_t seg = 0;
    bool ok = true;
    const int half = warp >> 2, quad = warp & 3;       // columns' half; TMEM lanes 32 quad ..
    const int et = tid & 127;                          // thread of the warp group
    const int esize = a.out_type == HA_TYPE_FP32 ? 4 : 2;
    unsigned char* stage = Out + half * S::kStage;
    const int tc = a.out_type == HA_TYPE_FP32 ? 16 : 32;   // columns of a stage
    for (int i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
      const Tile t = tile_at<MODE, NT>(sh, a, i);
      const int nk = (t.k + kK - 1) / kK;
      const int segs = a.out_type == HA_TYPE_FP32 ? (nk + kFold - 1) / kFold : (nk > 0 ? 1 : 0);
      const int cb = half * (NT / 2), ce = min(NT / 2, t.cols - cb);   // this group's columns
      float acc[NT / 2];
#pragma unroll
      for (int j = 0; j < NT / 2; ++j) acc[j] = 0.0f;
      for (int s = 0; s < segs && ok; ++s, ++seg) {
        const int buf = seg & 1;
        ok = mbar_wait(&sh.tfull[buf], (seg >> 1) & 1, &g_operator_error);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int j = 0; j < NT / 2; j += 32) {
          if (j < ce) {
            float v[32];
            tmem_ld32(tmem + (static_cast<uint32_t>(quad * 32) << 16) + buf * NT + cb + j, v);
            tmem_ld_wait();
#pragma unroll
            for (int x = 0; x < 32; ++x) acc[j + x] += v[x];
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.tempty[buf]);
      }
      if (!ok) break;
      const int f = t.m0 + quad * 32 + lane;            // this thread's feature
      if (MODE == kDw) {
        if (f < a.m) {
          const int64_t at = t.g * a.out_gs + f * a.out_ld + t.c0 + cb;
#pragma unroll
          for (int j = 0; j < NT / 2; j += 16) {
            if (j >= ce) continue;
            if (a.wide_out && j + 16 <= ce) {
              if (a.out_type == HA_TYPE_FP32) {
                float4* o = reinterpret_cast<float4*>(static_cast<float*>(a.out) + at + j);
#pragma unroll
                for (int x = 0; x < 4; ++x)
                  o[x] = make_float4(acc[j + 4 * x], acc[j + 4 * x + 1], acc[j + 4 * x + 2], acc[j + 4 * x + 3]);
              } else {
                uint32_t w[8];
#pragma unroll
                for (int x = 0; x < 8; ++x)
                  w[x] = narrow(acc[j + 2 * x], a.out_type) | (static_cast<uint32_t>(narrow(acc[j + 2 * x + 1], a.out_type)) << 16);
                uint4* o = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + at + j);
                o[0] = make_uint4(w[0], w[1], w[2], w[3]);
                o[1] = make_uint4(w[4], w[5], w[6], w[7]);
              }
            } else {
#pragma unroll
              for (int x = 0; x < 16; ++x)
                if (j + x < ce) {
                  if (a.out_type == HA_TYPE_FP32)
                    static_cast<float*>(a.out)[at + j + x] = acc[j + x];
                  else
                    static_cast<uint16_t*>(a.out)[at + j + x] = narrow(acc[j + x], a.out_type);
                }
            }
          }
        }
        continue;
      }
      const float bias = MODE == kFwd && a.bias && f < a.m ? a.bias[t.g * a.bias_ld + f] : 0.0f;
      // Through shared memory, so that a row's features leave as whole 16-byte vectors.
#pragma unroll
      for (int j0 = 0; j0 < NT / 2; j0 += 16) {
        if (j0 % tc) continue;
        const bool any = j0 < ce;
        if (!any) continue;                            // the same for the whole warp group
        named_barrier_sync(1 + half, 128);
#pragma unroll
        for (int x = 0; x < 32; ++x) {
          if (x < tc && j0 + x < NT / 2) {
            float v = acc[(j0 + x) % (NT / 2)] + bias;
            if (MODE == kFwd && a.relu && v < 0.0f) v = 0.0f;
            if (a.out_type == HA_TYPE_FP32)
              reinterpret_cast<float*>(stage)[x * kM + quad * 32 + lane] = v;
            else
              reinterpret_cast<uint16_t*>(stage)[x * kM + quad * 32 + lane] = narrow(v, a.out_type);
          }
        }
        named_barrier_sync(1 + half, 128);
        const int per = 16 / esize, segsr = kM / per;   // elements of a vector, vectors of a row
        for (int x = et; x < tc * segsr; x += 128) {
          const int r = x / segsr, e = x % segsr * per;
          if (j0 + r >= ce || t.m0 + e >= a.m) continue;
          const int64_t row = t.c0 + cb + j0 + r;
          const int nf = min(per, a.m - t.m0 - e);
          uint4 w = *reinterpret_cast<const uint4*>(stage + (r * kM + e) * esize);
          if (MODE == kDx && a.h) {
            const uint16_t* h = static_cast<const uint16_t*>(a.h) + row * a.h_ld + t.m0 + e;
            uint16_t hv[8];
            for (int y = 0; y < nf; ++y) hv[y] = h[y];
            if (esize == 4) {
              float* p = reinterpret_cast<float*>(&w);
#pragma unroll
              for (int y = 0; y < 4; ++y)
                if (y < nf && !positive16(hv[y], a.in_type)) p[y] = 0.0f;
            } else {
              uint16_t* p = reinterpret_cast<uint16_t*>(&w);
#pragma unroll
              for (int y = 0; y < 8; ++y)
                if (y < nf && !positive16(hv[y], a.in_type)) p[y] = 0;
            }
          }
          unsigned char* o = static_cast<unsigned char*>(a.out) + (row * a.out_ld + t.m0 + e) * esize;
          if (a.wide_out && nf == per) {
            *reinterpret_cast<uint4*>(o) = w;
          } else if (esize == 4) {
            const float* p = reinterpret_cast<const float*>(&w);
            for (int y = 0; y < nf; ++y) reinterpret_cast<float*>(o)[y] = p[y];
          } else {
            const uint16_t* p = reinterpret_cast<const uint16_t*>(&w);
            for (int y = 0; y < nf; ++y) reinterpret_cast<uint16_t*>(o)[y] = p[y];
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kEpiWarps) {
    tmem_dealloc(tmem, S::kTmem);
    tmem_relinquish();
  }
}

// db_g[f] = sum of dy[t][f] over the group's rows: a CTA has 32 features, its warps take
// the rows in turn and join in a fixed order.
template <typename T>
__global__ void __launch_bounds__(512) k_bias_grad(const T* dy, int64_t ld, const int* offsets,
                                                   int rows, int n, float* db, int64_t db_ld) {
  __shared__ float part[16][33];
  const int g = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int f = blockIdx.x * 32 + lane;
  const int begin = min(max(offsets[g], 0), rows), end = min(max(offsets[g + 1], 0), rows);
  float s = 0.0f;
  if (f < n)
    for (int t = begin + warp; t < end; t += 16) s += Elem<T>::up(dy[t * ld + f]);
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && f < n) {
    for (int w = 1; w < 16; ++w) s += part[w][lane];
    db[g * db_ld + f] = s;
  }
}

// Rows of 16-bit values to a pitch of whole 16-byte vectors, for operands that a tensor
// map cannot describe (an odd width, stride or address).
__global__ void __launch_bounds__(256) k_pack(const uint16_t* src, int64_t rows, int64_t per_group,
                                              int64_t cols, int64_t ld, int64_t gs, uint16_t* dst,
                                              int64_t pitch) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const uint16_t* s = src + r / per_group * gs + r % per_group * ld;
    for (int64_t c = threadIdx.x; c < pitch; c += 256) dst[r * pitch + c] = c < cols ? s[c] : 0;
  }
}

constexpr int kSms = 152;
int64_t round8(int64_t x) { return (x + 7) / 8 * 8; }
int64_t round256(int64_t x) { return (x + 255) / 256 * 256; }

// One operand as the tensor maps need it: address and strides multiples of 16 bytes.
struct Operand {
  const void* p;
  int64_t groups, rows, cols, ld, gs;   // gs: between groups (groups > 1)
  bool fits() const {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0 &&
           (groups == 1 || (gs > 0 && gs % 8 == 0));   // one matrix for all groups is copied
  }
  int64_t packed_bytes() const { return fits() ? 0 : round256(groups * rows * round8(cols) * 2); }
};

cudaError_t pack(Operand& o, unsigned char*& ws, cudaStream_t s) {
  if (o.fits()) return cudaSuccess;
  const int64_t pitch = round8(o.cols), rows = o.groups * o.rows;
  uint16_t* dst = reinterpret_cast<uint16_t*>(ws);
  ws += o.packed_bytes();
  k_pack<<<static_cast<unsigned>(std::min<int64_t>(rows, 8 * kSms)), 256, 0, s>>>(
      static_cast<const uint16_t*>(o.p), rows, o.rows, o.cols, o.ld, o.gs, dst, pitch);
  o.p = dst;
  o.ld = pitch;
  o.gs = o.rows * pitch;
  return cudaGetLastError();
}

bool make_map(CUtensorMap* m, const Operand& o, int type, bool grouped, uint32_t b0, uint32_t b1) {
  const EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(o.cols), static_cast<cuuint64_t>(o.rows),
                              static_cast<cuuint64_t>(o.groups)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(o.ld * 2),
                                 static_cast<cuuint64_t>((o.groups == 1 ? o.rows * o.ld : o.gs) * 2)};
  const cuuint32_t box[3] = {b0, b1, 1}, one[3] = {1, 1, 1};
  return enc(m, type == HA_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
             grouped ? 3 : 2, const_cast<void*>(o.p), dims, strides, box, one,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int MODE, int NT>
int launch(const CUtensorMap& ta, const CUtensorMap& tb, const Args& a, int64_t max_tiles, cudaStream_t s) {
  const int smem = Shape<NT>::kSmem;
  if (cudaFuncSetAttribute(k_grouped<MODE, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
    return HA_ECUDA;
  const int64_t grid = std::min<int64_t>(kSms, std::max<int64_t>(max_tiles, 1));
  k_grouped<MODE, NT><<<static_cast<unsigned>(grid), kThreads, smem, s>>>(ta, tb, a);
  return cudaGetLastError() == cudaSuccess ? HA_OK : HA_ECUDA;
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
  if (pack(x, p, s) != cudaSuccess || pack(w, p, s) != cudaSuccess) return HA_ECUDA;
  a.wide_out = (reinterpret_cast<uintptr_t>(a.out) & 15) == 0 && a.out_ld * type_size(a.out_type) % 16 == 0;
  // Few rows a group: narrow tiles, whose smaller chunks leave room for more in flight.
  const bool few = a.rows <= 64 * static_cast<int64_t>(a.groups);
  CUtensorMap ta, tb;
  if (!make_map(&ta, w, a.in_type, true, 64, MODE == kFwd ? 128 : 64) ||
      !make_map(&tb, x, a.in_type, false, 64, few ? Shape<64>::kBoxRows : Shape<256>::kBoxRows))
    return HA_ECUDA;
  const int64_t mt = (a.m + kM - 1) / kM;
  const int64_t most = mt * std::min<int64_t>(a.rows, a.groups + a.rows / (few ? 64 : 256));
  return few ? launch<MODE, 64>(ta, tb, a, most, s) : launch<MODE, 256>(ta, tb, a, most, s);
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
    dy = {dw_dev, 1, 1, outer, round8(outer), 0};
    x = {dw_dev, 1, 1, inner, round8(inner), 0};
    dy.p = x.p = reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(dw_dev) & ~uintptr_t(15));
  }
  if (dy.packed_bytes() + x.packed_bytes() > workspace_bytes) return HA_ENOMEM;
  if (workspace_bytes > 0 && (!workspace_dev || (reinterpret_cast<uintptr_t>(workspace_dev) & 15)))
    return HA_EINVAL;
  unsigned char* p = static_cast<unsigned char*>(workspace_dev);
  if (db_dev) {
    const dim3 grid((outer + 31) / 32, groups);
    if (type == HA_TYPE_BF16)
      k_bias_grad<__nv_bfloat16><<<grid, 512, 0, s>>>(static_cast<const __nv_bfloat16*>(dy_dev), dy_ld,
                                                      offsets_dev, static_cast<int>(rows), outer, db_dev, db_ld);
    else
      k_bias_grad<__half><<<grid, 512, 0, s>>>(static_cast<const __half*>(dy_dev), dy_ld, offsets_dev,
                                               static_cast<int>(rows), outer, db_dev, db_ld);
    if (cudaGetLastError() != cudaSuccess) return HA_ECUDA;
  }
  if (pack(dy, p, s) != cudaSuccess || pack(x, p, s) != cudaSuccess) return HA_ECUDA;
  Args a = {};
  a.offsets = offsets_dev;
  a.out = dw_dev;
  a.out_ld = dw_ld;
  a.out_gs = dw_gs;
  a.groups = groups;
  a.rows = static_cast<int>(rows);
  a.m = outer;
  a.n = inner;
  a.in_type = type;
  a.out_type = dw_type;
  const int es = type_size(dw_type);
  a.wide_out = (reinterpret_cast<uintptr_t>(dw_dev) & 15) == 0 && dw_ld * es % 16 == 0 &&
               (groups == 1 || dw_gs * es % 16 == 0);
  CUtensorMap ta, tb;
  if (!make_map(&ta, dy, type, false, 64, 64) || !make_map(&tb, x, type, false, 64, 64)) return HA_ECUDA;
  const int64_t most = groups * static_cast<int64_t>((outer + kM - 1) / kM) * ((inner + 255) / 256);
  if (most > 0x7FFFFFFF) return HA_EUNSUPPORTED;
  return launch<kDw, 256>(ta, tb, a, most, s);
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
