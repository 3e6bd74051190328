// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
// Row i of a sequence has p_i = softmax(logits_i / temperature) over the allowed classes and, for i < K, the
// draft x_i, which was drawn from q_i (without draft probabilities q is 1 at x_i).  With uniform numbers u:
//   draft i is accepted while u_i q_i(x_i) < p_i(x_i);  n is the first that is not, or the first row without a draft;
//   the next token is argmax_j r_j / noise_j with r = max(p_n - q_n, 0) after a rejection (p_n where that
//   leaves nothing), else r = p_n.  With exponential noise that is a draw from r.
//
// Few and short rows are one kernel's, a CTA a sequence.  Else two, each over as many CTAs as fill the GPU.  The first takes
// shares of all rows: their largest logit and the sum of the exponentials.  The second joins them, finds n, and takes shares of
// row n's scores; the last CTA of a sequence to end joins those.  Rows behind a rejected draft are summed for nothing, but a row
// waits for no other: 128 sequences of 6 rows of 50021 fp32 logits under a mask take 54 us so, 57 where CTAs ask before they start
// whether a draft has failed, and 95 by a cluster a sequence that takes its rows in turn and stops.  Both kernels wait
// for memory (issue slots 34 and 40 % full, DRAM 67 and 34 %): 53 us against 41 for all the bytes.
// Sums and scores are in fp32, with a bound of what that may be off; a decision within the bound is made
// again by one CTA, in 64 bits but for the sum of the exponentials, which pairs of floats hold to 2^-40.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <type_traits>

#include "op_common.cuh"

namespace ha {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kResident = 8;              // CTAs of an SM
// A CTA of kOneThreads does a sequence by itself, and saves the second launch and its wait, up to so many classes and elements of
// logits; more where enough sequences fill the SMs.  Above kOneSequences the CTAs of few classes are too wide (2000 sequences, 2
// rows of 1001: 34 us, against 19.6 in two kernels).  One CTA against two kernels, bf16, in us:
//   1 sequence, 5 rows of 1001: 5.4, 7.2;  of 8192: 8.1, 8.2;  of 16384: 11.1, 8.3;  8 sequences, 10 rows of 8192: 10.8, 10.3
//   64 sequences, 5 rows of 1001: 6.6, 8.8;  of 16384: 15.0, 16.6;  fp32, of 32001: 24.8, 21.0;  256, 4 rows of 8192: 11.0, 16.4
// Two CTAs an SM, 64 registers, of which 36 bytes spill: the last takes 11.4 us; one (nothing spills) 14.0, three (132 to 224 bytes) 12.2.
constexpr int kOneThreads = 512, kOneResident = 2, kOneSequences = 512, kFilled = 64;
constexpr int kOneClasses = 8192, kOneElements = 5 * 8192;             // of fewer than kFilled sequences
constexpr int kManyClasses = 16384, kManyElements = 8 * 16384;
constexpr int kUnroll = 4;                // 16-byte loads in flight of a sum
constexpr int kScores = 4;                // classes whose scores are in flight
constexpr int kSumParts = 32;             // CTAs of a row, at most
constexpr int kScoreParts = 128;          // CTAs of a sequence's scores, at most

// The relative error of a probability e^((z - m) / t) / S with d = (z - m) log2(e) / t, in steps of 2^-22: the three roundings of d
// (c, the difference, the product) are 0.52 |d| of them, and bound() takes |d|.  The others, from above:
//   S: 1 for its terms' powers and 16 for their d, whose mean |d| is at most log2 of the classes, 31; 1.75 for the additions within
//      a vector and those of a thread's halves and odd element, 1.5 for its rescaling by that; 7.5 for three joins of warps and CTAs, each
//      a rescaling and 5 additions; of a chain of vectors 0.25 for each addition, and 1.25 for each rescaling by a new largest
//      logit, of which a batch of kUnroll vectors has one
//   p, a score, its bound and their comparison: 1 for 2^d, 0.25 for each of ten roundings
float slack(int64_t classes, int threads, int elements_a_load) {
  const int64_t vectors = classes / (static_cast<int64_t>(threads) * elements_a_load) + 1;
  return 32.0f + 0.25f * static_cast<float>(vectors) + 1.25f * static_cast<float>(vectors / kUnroll + 1);
}
__device__ __forceinline__ float bound(float d, float slack) { return 0x1p-22f * (slack + fabsf(d)); }

struct Sum {
  float m, S;                             // largest logit; sum of e^((z - m) / t), 0: no class, NaN: a bad row
};
// What bounds a class's score, r / noise and what that may be off, from above.
struct Best {
  float most, others;                     // the largest, and the largest of all others
  int index, pad;                         // of the largest
};
struct Head {                             // of a row's draft
  float u, q;                             // accepted while u q < p
  float zx;                               // its logit; kNone: no class, or not allowed
  int draft;                              // -1: none, INT_MAX: no class
};
// The workspace; a row is sequence * (K + 1) + i.
struct Work {
  Head* heads;                            // [rows]
  Sum* sums;                              // [rows, kSumParts]
  Best* bests;                            // [sequences, kScoreParts]
  int* done;                              // [sequences] CTAs whose scores are there
};
constexpr int64_t kRowBytes = sizeof(Head) + kSumParts * sizeof(Sum);
constexpr int64_t kSequenceBytes = kScoreParts * sizeof(Best) + sizeof(int);

// A number as the sum of two floats.
struct Two {
  float hi, lo;
};
__host__ __device__ constexpr Two two(double x) {
  return {static_cast<float>(x), static_cast<float>(x - static_cast<double>(static_cast<float>(x)))};
}

struct VerifyArgs {
  const void* logits;
  int64_t z_seq, z_row;
  const void* drafts;
  const float* uniform;
  const float* noise;
  int64_t noise_ld;
  const void* probs;
  int64_t q_seq, q_row;
  const uint8_t* allowed;
  int64_t ok_seq, ok_row;
  int *tokens, *accepted;
  float* logp;
  double inv_temperature;
  float c;                                // log2(e) / temperature
  Two c2;                                 // the same
  Two inv_t2;                             // 1 / temperature
  float slack;                            // of bound()
  int K, classes;
  int64_t sequences;
  int sum_parts, score_parts;
  int per;                                // warps of a row, where one CTA does the sequence
  Work w;
  bool wide_drafts;
  int probs_type;                         // -1: none
};

__device__ __forceinline__ int64_t draft_of(const VerifyArgs& a, int64_t seq, int i) {
  const int64_t e = seq * a.K + i;
  return a.wide_drafts ? static_cast<const int64_t*>(a.drafts)[e] : static_cast<const int*>(a.drafts)[e];
}
__device__ __forceinline__ float prob_at(const VerifyArgs& a, int64_t e) {
  if (a.probs_type == HA_TYPE_FP32) return static_cast<const float*>(a.probs)[e];
  if (a.probs_type == HA_TYPE_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(a.probs)[e]);
  return __half2float(static_cast<const __half*>(a.probs)[e]);
}

// A row's logit, kNone where the class is not allowed.
template <typename T>
__device__ __forceinline__ float logit(const T* z, const uint8_t* ok, int j) {
  const float v = max_nan(Elem<T>::up(z[j]), kNone<T>);
  return ok && !ok[j] ? kNone<T> : v;
}

// Is a row's largest logit so close to a mask's that masked exponentials do not vanish?  (fp32's numbers are 2^76 apart there, so that
// it takes temperatures above 2^69.)  Its sum is then taken again without them, and 64 bits decide its token.
template <typename T>
__device__ __forceinline__ bool near_masked(float m, float c) { return c < 0x1p-68f && (kNone<T> - m) * c > -150.0f; }

__device__ __forceinline__ Sum join(Sum s, float c) {
  const float m = from_ordered(__reduce_max_sync(~0u, ordered(s.m)));
  Sum r = {m, s.S * exp2_fast(max_nan((s.m - m) * c, -200.0f))};
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.S += __shfl_xor_sync(~0u, r.S, o);
  return r;
}

// The coefficients of 2^f = sum over n of (f log 2)^n / n!.
__host__ __device__ constexpr double power_term(int n) {
  double a = 1.0;
  for (int i = 1; i <= n; ++i) a = a * 0.69314718055994530942 / i;
  return a;
}
// 2^((v - m) c) to about 2^-40 of it, c = c.hi + c.lo > 0 and v <= m; 0 below 2^-120.  In 64 bits the sum of 128000 takes a CTA
// 1.1 ms, so 0.23.  The product's integer part n is taken off, f in [-1/2, 1/2] remains; the series' terms from f^8 on are below
// 2^-27 and need one float, the others are added in two (error-free sums and products, Dekker 1971).
__device__ __forceinline__ Two power(float v, float m, Two c) {
  const float d = v - m, p = d * c.hi;
  const float back = d - v, e = (v - (d - back)) + (-m - back);                // d + e = v - m
  const float n = rintf(p), g = fmaf(d, c.lo, fmaf(d, c.hi, -p)) + e * c.hi, w = p - n, f = w + g, fl = g - (f - w);
  float r = static_cast<float>(power_term(12));
#pragma unroll
  for (int i = 11; i >= 8; --i) r = fmaf(r, f, static_cast<float>(power_term(i)));
  Two s = {r, 0.0f};
#pragma unroll
  for (int i = 7; i >= 0; --i) {
    const Two a = two(power_term(i));
    const float h = s.hi * f, l = fmaf(s.lo, f, fmaf(s.hi, fl, fmaf(s.hi, f, -h)));
    s.hi = a.hi + h;
    s.lo = (h - (s.hi - a.hi)) + (l + a.lo);
  }
  const float scale = __int_as_float((static_cast<int>(n) + 127) << 23);
  const bool any = p > -120.0f;                              // no branch, so that several are computed side by side
  return {any ? s.hi * scale : 0.0f, any ? s.lo * scale : 0.0f};
}

// (v - m) / t - log S, rounded once, for v <= m and S >= 1: v - m, its product and the difference are held in two floats, and l, the
// logarithm in fp32, is made exact by what S e^-l differs from 1.
__device__ __forceinline__ float log_prob(const VerifyArgs& a, float v, float m, float S) {
  const float l = logf(S);
  const Two y = power(-l, 0.0f, two(1.4426950408889634));
  const float rest = fmaf(S, y.hi, -1.0f) + S * y.lo;        // log S = l + log(1 + rest)
  const float d = v - m, back = d - v, e = (v - (d - back)) + (-m - back);
  const float h = d * a.inv_t2.hi, s = h - l, from = s - h;
  const float low = fmaf(d, a.inv_t2.hi, -h) + fmaf(d, a.inv_t2.lo, e * a.inv_t2.hi);
  return s + ((h - (s - from)) + (-l - from) + (low - rest));
}

// The sum of e^((z - m) / t) to about 2^-40, by one CTA; every thread has it.
template <typename T, int THREADS>
__device__ __noinline__ double exact_sum(const VerifyArgs& a, const T* z, const uint8_t* ok, float m, double* part) {
  Two s = {0.0f, 0.0f};
  constexpr int kAtOnce = 4;
  for (int j0 = threadIdx.x; j0 < a.classes; j0 += kAtOnce * THREADS) {
    float v[kAtOnce];
    Two x[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) v[u] = logit(z, ok, min(j0 + u * THREADS, a.classes - 1));
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) x[u] = power(v[u], m, a.c2);
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      if (!(v[u] > kNone<T>) || j0 + u * THREADS >= a.classes) x[u] = {0.0f, 0.0f};
      const float h = s.hi + x[u].hi, back = h - s.hi;
      s.lo += ((s.hi - (h - back)) + (x[u].hi - back)) + x[u].lo;
      s.hi = h;
    }
  }
  double t = static_cast<double>(s.hi) + static_cast<double>(s.lo);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(~0u, t, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = t;
  __syncthreads();
  t = 0.0;
  for (int w = 0; w < THREADS / 32; ++w) t += part[w];
  return t;
}
// A class's probability from it, in 64 bits.
__device__ __forceinline__ double exact_prob(const VerifyArgs& a, float v, float m, double sum) {
  return exp((static_cast<double>(v) - m) * a.inv_temperature) / sum;
}

// Two minus infinities of a 16-bit type.
template <typename T> constexpr uint32_t kBits16 = 0xFC00FC00u;
template <> constexpr uint32_t kBits16<__nv_bfloat16> = 0xFF80FF80u;

// The sum of share `rank` of `parts` of a row, by THREADS threads side by side; each warp has its own.  Masked logits stay as
// they are: the largest is kNone at least, so that their distances are no NaN and their exponentials 0 (unless it is near_masked).
template <typename T, bool MASK, int THREADS>
__device__ __forceinline__ Sum scan(const T* z, const uint8_t* ok, int classes, float c, int rank, int parts) {
  constexpr int V = kVec<T>;
  const int tid = threadIdx.x % THREADS;
  // The vectors start at the row's first 16-byte boundary; the entries before and after them are taken one by one.
  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
  int head = shift ? V - shift : 0;
  if (MASK && head < 4) head += V;                           // the words around a vector's mask bytes are the row's own
  head = min(classes, head);
  int vecs = (classes - head) / V;
  if (MASK && vecs > 0 && head + vecs * V + 4 > classes) --vecs;
  const int tail = head + vecs * V;
  const int v0 = static_cast<int>(static_cast<int64_t>(vecs) * rank / parts);
  const int v1 = static_cast<int>(static_cast<int64_t>(vecs) * (rank + 1) / parts);
  const uint4* zv = reinterpret_cast<const uint4*>(z + head);
  const uint32_t ok_shift = MASK ? 8 * static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ok + head) & 3) : 0;
  const uint32_t* okw = MASK ? reinterpret_cast<const uint32_t*>(ok + head - ok_shift / 8) : nullptr;
  float m = kNone<T>;
  Pair S = pair(0.0f, 0.0f);
  int one = -1;
  if (rank == 0 && tid < head) one = tid;
  if (rank == parts - 1 && tid >= 16 && tail + tid - 16 < classes) one = tail + tid - 16;
  const float left = one >= 0 ? logit(z, MASK ? ok : nullptr, one) : kNone<T>;
  // kUnroll vectors, all loads before the first use and one look at the largest; the last ones may be fewer.
  auto batch = [&](int r, auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
    uint4 w[kUnroll];
    uint32_t in[kUnroll][V / 4 + 1];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int i = r + u * THREADS;
      if (kWhole || i < v1) {
        w[u] = __ldg(zv + i);
        if (MASK) {
#pragma unroll
          for (int h = 0; h <= V / 4; ++h) in[u][h] = __ldg(okw + i * (V / 4) + h);
        }
      } else {
        const uint32_t inf = sizeof(T) == 4 ? 0xFF800000u : kBits16<T>;
        w[u] = make_uint4(inf, inf, inf, inf);
#pragma unroll
        for (int h = 0; h <= V / 4; ++h) in[u][h] = 0;
      }
    }
    float v[kUnroll][V];
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      unpack<T>(w[u], v[u]);
      if (MASK) {
#pragma unroll
        for (int h = 0; h < V / 4; ++h) {
          const uint32_t ok4 = __funnelshift_r(in[u][h], in[u][h + 1], ok_shift);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!(ok4 & 0xFFu << 8 * e)) v[u][4 * h + e] = -INFINITY;
        }
      }
#pragma unroll
      for (int e = 0; e < V; e += 2) top = fmaxf(top, fmaxf(v[u][e], v[u][e + 1]));
    }
    if (top > m) {
      const float f = exp2_fast(max_nan((m - top) * c, -200.0f));
      S = mul2(S, pair(f, f));
      m = top;
    }
    if (m > kNone<T>) {
      const Pair minus_m = pair(-m, -m), c2 = pair(c, c);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        Pair sum;
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          float x, y;
          halves(mul2(add2(pair(v[u][e], v[u][e + 1]), minus_m), c2), x, y);
          const Pair p = pair(exp2_fast(x), exp2_fast(y));
          sum = e == 0 ? p : add2(sum, p);
        }
        S = add2(S, sum);
      }
    } else {                                                 // nothing allowed so far, unless it is a NaN
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (v[u][e] != v[u][e]) S = pair(NAN, 0.0f);
    }
  };
  int r = v0 + tid;
  for (; r + (kUnroll - 1) * THREADS < v1; r += kUnroll * THREADS) batch(r, std::true_type());
  if (r < v1) batch(r, std::false_type());
  Sum s = {m, 0.0f};
  float x, y;
  halves(S, x, y);
  s.S = x + y;
  if (left > s.m) {
    s.S = fmaf(s.S, exp2_fast(max_nan((s.m - left) * c, -200.0f)), left < INFINITY ? 1.0f : NAN);
    s.m = left;
  } else if (!(left <= kNone<T>)) {
    s.S += exp2_fast((left - s.m) * c);
  }
  return join(s, c);
}

__device__ __forceinline__ Best better(const Best& a, const Best& b) {
  const bool first = a.most > b.most;
  return {first ? a.most : b.most, fmaxf(fminf(a.most, b.most), fmaxf(a.others, b.others)), first ? a.index : b.index, 0};
}
__device__ __forceinline__ Best warp_best(Best b) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Best x = {__shfl_xor_sync(~0u, b.most, o), __shfl_xor_sync(~0u, b.others, o), __shfl_xor_sync(~0u, b.index, o), 0};
    b = better(b, x);
  }
  return b;
}

__device__ __forceinline__ float rcp_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Scores below this are not told apart in fp32: the reciprocal of a noise above 2^126 is 0 here, and the score, at most 2^-126, is lost
// with its bound; products below 2^-126 lose bits that no bound counts.  Above it, what the bounds say is so.
constexpr float kLowScore = 0x1p-125f;
// A row's scores r / noise, and what they may be off.
struct Scores {
  float m, inv_s, c, slack;
  __device__ __forceinline__ float of(float v, float q, float e, float& off) const {
    const float d = max_nan((v - m) * c, -1e4f), p = exp2_fast(d) * inv_s, rn = rcp_fast(e);
    off = fmaf(fmaf(-d, 0x1p-22f, slack), p, FLT_MIN) * rn;  // bound(d) p, and what is below fp32's range
    return fmaxf(p - q, 0.0f) * rn;
  }
};

// What a row's largest score is at least, if above kLowScore; by one CTA.  hole: a class without a score.
template <typename T, int THREADS>
__device__ __noinline__ float lowest_score(const VerifyArgs& a, const T* z, const uint8_t* ok, const float* noise, const Scores& sc,
                                           int64_t q0, bool minus_q, int hole, double* part) {
  float low = 0.0f;
  constexpr int kAtOnce = 4;
  for (int j0 = threadIdx.x; j0 < a.classes; j0 += kAtOnce * THREADS) {
    float v[kAtOnce], e[kAtOnce], q[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int j = min(j0 + u * THREADS, a.classes - 1);
      v[u] = logit(z, ok, j);
      e[u] = noise[j];
      q[u] = minus_q ? prob_at(a, q0 + j) : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      float off;
      const float s = sc.of(v[u], q[u], e[u], off);
      if (v[u] > kNone<T> && min(j0 + u * THREADS, a.classes - 1) != hole) low = fmaxf(low, s - fabsf(off));
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) low = fmaxf(low, __shfl_xor_sync(~0u, low, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = low;
  __syncthreads();
  for (int w = 0; w < THREADS / 32; ++w) low = fmaxf(low, static_cast<float>(part[w]));
  return low;
}

// The next token, by one CTA, in 64 bits but for the sum.  low: what the largest score is at least.  Not above kLowScore where the
// class that may be the largest is one of a large p next to its q, whose bound is above its score; the others then say more, and 64
// bits are taken for few classes (2000 sequences of 4097 classes, one token decided so: 50 us; 111 by 64 bits for each class).
template <typename T, int THREADS>
__device__ __noinline__ int exact_token(const VerifyArgs& a, const T* z, const uint8_t* ok, const float* noise, const Scores& sc,
                                        float low, int64_t q0, int x, bool rejected, double* part, int* part_index) {
  const double sum = exact_sum<T, THREADS>(a, z, ok, sc.m, part);
  int best = -1;
  for (int pass = rejected ? 0 : 1; pass < 2 && best < 0; ++pass) {
    double score = -1.0;
    bool any = false;
    best = -1;
    const bool minus_q = pass == 0 && a.probs;
    const float least = low > kLowScore
                            ? low : lowest_score<T, THREADS>(a, z, ok, noise, sc, q0, minus_q, pass == 0 && !a.probs ? x : -1, part);
    constexpr int kAtOnce = 4;
    for (int j0 = threadIdx.x; j0 < a.classes; j0 += kAtOnce * THREADS) {
      float v[kAtOnce], e[kAtOnce], q[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int j = min(j0 + u * THREADS, a.classes - 1);
        v[u] = logit(z, ok, j);
        e[u] = noise[j];
        q[u] = minus_q ? prob_at(a, q0 + j) : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int j = j0 + u * THREADS;
        float off;
        const float most = sc.of(v[u], q[u], e[u], off) + off;
        if (j >= a.classes || !(v[u] > kNone<T>) || (least > kLowScore && most < least)) continue;
        double r = exact_prob(a, v[u], sc.m, sum);
        if (pass == 0) r = a.probs ? fmax(r - static_cast<double>(q[u]), 0.0) : j == x ? 0.0 : r;
        const double s = r / static_cast<double>(e[u]);
        any = any || r > 0.0;
        if (r > 0.0 && s >= 0.0 && s > score) {
          score = s;
          best = j;
        }
      }
    }
    const int some = __syncthreads_or(any);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const double s = __shfl_xor_sync(~0u, score, o);
      const int j = __shfl_xor_sync(~0u, best, o);
      if (s > score || (s == score && static_cast<uint32_t>(j) < static_cast<uint32_t>(best))) {
        score = s;
        best = j;
      }
    }
    if ((threadIdx.x & 31) == 0) {
      part[threadIdx.x >> 5] = score;
      part_index[threadIdx.x >> 5] = best;
    }
    __syncthreads();
    score = -1.0;
    best = -1;
    for (int w = 0; w < THREADS / 32; ++w)
      if (part[w] > score || (part[w] == score && static_cast<uint32_t>(part_index[w]) < static_cast<uint32_t>(best))) {
        score = part[w];
        best = part_index[w];
      }
    __syncthreads();
    if (some) break;
  }
  return best;
}

// Whether a row's draft is accepted: 0, 1, or 2 where it takes more bits to say.
__device__ __forceinline__ int decide(const VerifyArgs& a, const Head& h, Sum s, float none) {
  if (!(h.zx > none && s.S > 0.0f)) return 0;                // no class, or a NaN in the row
  const float d = (h.zx - s.m) * a.c, p = exp2_fast(d) / s.S, left = h.u * h.q;
  if (fabsf(left - p) <= fmaf(bound(d, a.slack), p, 0x1p-23f * left) || (p < 1e-30f && left < 1e-30f)) return 2;
  return left < p;
}

template <typename T>
__device__ __forceinline__ const T* logits_of(const VerifyArgs& a, int64_t seq, int i) {
  return static_cast<const T*>(a.logits) + seq * a.z_seq + i * a.z_row;
}
__device__ __forceinline__ const uint8_t* mask_of(const VerifyArgs& a, int64_t seq, int i) {
  return a.allowed ? a.allowed + seq * a.ok_seq + i * a.ok_row : nullptr;
}

// What row i's draft is accepted by.
template <typename T>
__device__ __forceinline__ Head head_of(const VerifyArgs& a, int64_t seq, int i, const T* z, const uint8_t* ok) {
  Head h = {0.0f, 0.0f, kNone<T>, -1};
  const int64_t x = i < a.K ? draft_of(a, seq, i) : -1;
  if (x < 0) return h;
  h.draft = x < a.classes ? static_cast<int>(x) : INT_MAX;
  if (x < a.classes) {
    h.u = a.uniform[seq * a.K + i];
    h.q = a.probs ? prob_at(a, seq * a.q_seq + i * a.q_row + x) : 1.0f;
    h.zx = logit(z, ok, static_cast<int>(x));
  }
  return h;
}

template <typename T, bool MASK>
__global__ void __launch_bounds__(kThreads, kResident) k_verify_sums(const __grid_constant__ VerifyArgs a) {
  __shared__ Sum warp_sum[kWarps];
  const int tid = threadIdx.x, lane = tid & 31, rank = blockIdx.x % a.sum_parts;
  const int64_t row = blockIdx.x / a.sum_parts, seq = row / (a.K + 1);
  const int i = static_cast<int>(row % (a.K + 1));
  let_next_start();
  const T* z = logits_of<T>(a, seq, i);
  const uint8_t* ok = mask_of(a, seq, i);
  if (rank == 0 && tid == 0) {
    a.w.heads[row] = head_of(a, seq, i, z, ok);
    if (i == 0) a.w.done[seq] = 0;
  }
  Sum s = scan<T, MASK, kThreads>(z, ok, a.classes, a.c, rank, a.sum_parts);
  if (lane == 0) warp_sum[tid >> 5] = s;
  __syncthreads();
  if (tid >= 32) return;
  s = join(lane < kWarps ? warp_sum[lane] : Sum{kNone<T>, 0.0f}, a.c);
  if (lane == 0) a.w.sums[row * kSumParts + rank] = s;
}

// What follows the sums; ONE: few and short rows, and their sums too, a CTA a sequence, the rows side by side, a.per warps each.
// Q: the draft probabilities' type, any where there are none.  (One function: cut into several, the scores of 128 sequences of
// 50021 classes took 27 us, not 22, as the registers do not hold all.)
template <typename T, typename Q, bool ONE, bool MASK>
__global__ void __launch_bounds__(ONE ? kOneThreads : kThreads, ONE ? kOneResident : kResident)
    k_verify_next(const __grid_constant__ VerifyArgs a) {
  constexpr int THREADS = ONE ? kOneThreads : kThreads, kRows = ONE ? THREADS / 32 : 32;        // rows that are decided together
  __shared__ Sum row_sum[kRows];
  __shared__ Head row_head[kRows];
  __shared__ int row_state[kRows];
  __shared__ Best warp_bests[THREADS / 32];
  __shared__ double part[THREADS / 32];
  __shared__ int part_index[THREADS / 32];
  __shared__ int last_token;
  __shared__ bool is_last, unsure;
  __shared__ float lowest;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K = a.K, parts = ONE ? 1 : a.score_parts;
  const int rank = ONE ? 0 : blockIdx.x % parts;
  const int64_t seq = ONE ? blockIdx.x : blockIdx.x / parts, row0 = seq * (K + 1);
  const float* noise = a.noise + seq * a.noise_ld;
  // this CTA's classes
  const int c0 = static_cast<int>(static_cast<int64_t>(a.classes) * rank / parts);
  const int c1 = static_cast<int>(static_cast<int64_t>(a.classes) * (rank + 1) / parts);
  if constexpr (ONE) {
    __shared__ Sum warp_sum[THREADS / 32];
    const int per = a.per, mine = warp / per;
    if (mine <= K) {
      const T* z = logits_of<T>(a, seq, mine);
      const uint8_t* ok = mask_of(a, seq, mine);
      if (lane == 0 && warp % per == 0) row_head[mine] = head_of(a, seq, mine, z, ok);
      const Sum s = scan<T, MASK, 32>(z, ok, a.classes, a.c, warp % per, per);
      if (lane == 0) warp_sum[warp] = s;
    }
    __syncthreads();
    if (warp <= K) {
      const Sum s = join(lane < per ? warp_sum[warp * per + lane] : Sum{kNone<T>, 0.0f}, a.c);
      if (lane == 0) {
        row_sum[warp] = s;
        row_state[warp] = decide(a, row_head[warp], s, kNone<T>);
      }
    }
  } else {
    // what does not depend on n may come meanwhile, by lines
    for (int j = c0 + 32 * tid; j < c1; j += 32 * THREADS) asm volatile("prefetch.global.L2 [%0];" ::"l"(noise + j));
    wait_for_previous();
  }

  // ---- the first row whose draft is not accepted, by every CTA of the sequence
  int n = -1, drafted = -1;
  Sum st = {0.0f, 0.0f};
  for (int i0 = 0; n < 0; i0 += kRows) {
    const int rows = min(kRows, K + 1 - i0);
    for (int r = ONE ? rows : warp; r < rows; r += THREADS / 32) {
      Sum s = {kNone<T>, 0.0f};
      if (lane < a.sum_parts) s = a.w.sums[(row0 + i0 + r) * kSumParts + lane];
      const Head h = a.w.heads[row0 + i0 + r];
      s = join(s, a.c);
      if (lane == 0) {
        row_sum[r] = s;
        row_head[r] = h;
        row_state[r] = decide(a, h, s, kNone<T>);
      }
    }
    __syncthreads();
    for (int r = 0; r < rows && n < 0; ++r) {
      const int i = i0 + r;
      const Head h = row_head[r];
      bool accepted = row_state[r] == 1;
      const bool near = row_sum[r].S > 0.0f && near_masked<T>(row_sum[r].m, a.c);
      if (near || row_state[r] == 2) {
        const T* z = logits_of<T>(a, seq, i);
        const uint8_t* ok = mask_of(a, seq, i);
        const double sum = exact_sum<T, THREADS>(a, z, ok, row_sum[r].m, part);
        accepted = h.zx > kNone<T> && static_cast<double>(h.u) * h.q < exact_prob(a, h.zx, row_sum[r].m, sum);
        if (near) {
          __syncthreads();
          if (tid == 0) row_sum[r].S = static_cast<float>(sum);
          __syncthreads();
        }
      }
      if (!accepted) {
        n = i;
        st = row_sum[r];
        drafted = h.draft;
      }
    }
    if (rank == 0 && tid < (n < 0 ? rows : n - i0)) {        // a thread an accepted draft
      a.tokens[row0 + i0 + tid] = row_head[tid].draft;
      a.logp[row0 + i0 + tid] = log_prob(a, row_head[tid].zx, row_sum[tid].m, row_sum[tid].S);
    }
    __syncthreads();
  }

  // ---- the token behind it
  const bool rejected = drafted >= 0;
  const int x = drafted == INT_MAX ? -1 : drafted;
  const T* z = logits_of<T>(a, seq, n);
  const uint8_t* ok = mask_of(a, seq, n);
  const int64_t q0 = seq * a.q_seq + n * a.q_row;
  const bool dead = !(st.S > 0.0f);                          // no class, or a NaN
  const bool minus_q = rejected && a.probs;
  const int hole = rejected && !a.probs ? x : -1;
  const float inv_s = 1.0f / st.S;
  const Q* qs = static_cast<const Q*>(a.probs) + q0;
  const Scores scores = {st.m, inv_s, a.c, a.slack * 0x1p-22f};
  Best best = {0.0f, 0.0f, -1, 0};
  // kScores classes, all loads before the first use.  A class that is masked has p = 0 and a bound next to 0, with which it wins
  // only where no other is sure to be above it, and more bits decide.
  auto batch = [&](int j0, auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
    T v[kScores];
    Q q[kScores];
    float e[kScores];
    uint8_t in[kScores];
#pragma unroll
    for (int u = 0; u < kScores; ++u)
      if (kWhole || j0 + u * THREADS < c1) {
        v[u] = z[j0 + u * THREADS];
        e[u] = noise[j0 + u * THREADS];
      }
    if (minus_q) {
#pragma unroll
      for (int u = 0; u < kScores; ++u)
        if (kWhole || j0 + u * THREADS < c1) q[u] = qs[j0 + u * THREADS];
    }
    if (ok) {
#pragma unroll
      for (int u = 0; u < kScores; ++u)
        if (kWhole || j0 + u * THREADS < c1) in[u] = ok[j0 + u * THREADS];
    }
#pragma unroll
    for (int u = 0; u < kScores; ++u) {
      const int j = j0 + u * THREADS;
      if (!kWhole && j >= c1) break;
      float off, vu = Elem<T>::up(v[u]);
      if ((ok && !in[u]) || j == hole) vu = -INFINITY;
      const float s = scores.of(vu, minus_q ? Elem<Q>::up(q[u]) : 0.0f, e[u], off), most = s + off;
      // (a NaN, of a noise that is none, makes the others as good as the best)
      best.others = fmaxf(best.others, fminf(most, best.most));
      if (most > best.most) {
        best.most = most;
        best.index = j;
      }
    }
  };
  if (!dead && !near_masked<T>(st.m, a.c)) {
    int j0 = c0 + tid;
    for (; j0 + (kScores - 1) * THREADS < c1; j0 += kScores * THREADS) batch(j0, std::true_type());
    if (j0 < c1) batch(j0, std::false_type());
  }
  best = warp_best(best);
  if (lane == 0) warp_bests[warp] = best;
  __syncthreads();
  if (warp == 0) {
    best = warp_best(lane < THREADS / 32 ? warp_bests[lane] : Best{0.0f, 0.0f, -1, 0});
    if (lane == 0) {
      bool last = true;
      if (parts > 1) {
        a.w.bests[seq * kScoreParts + rank] = best;
        __threadfence();
        last = atomicAdd(a.w.done + seq, 1) == parts - 1;
        __threadfence();
      }
      is_last = last;
    }
  }
  __syncthreads();
  if (!is_last) return;
  if (warp == 0) {
    if (parts > 1) {
      best = {0.0f, 0.0f, -1, 0};
      for (int r = lane; r < parts; r += 32) {
        const int4 v = __ldcg(reinterpret_cast<const int4*>(a.w.bests + seq * kScoreParts + r));
        best = better(best, *reinterpret_cast<const Best*>(&v));
      }
      best = warp_best(best);
    }
    if (lane == 0) {
      float off = 0.0f;
      const int j = best.index;
      // as it was scored: a class that is masked, or the draft itself, may have won by its bound
      if (j >= 0) scores.of(j == hole ? -INFINITY : logit(z, ok, j), minus_q ? prob_at(a, q0 + j) : 0.0f, noise[j], off);
      last_token = j;
      lowest = best.most - 2.0f * off;
      unsure = !dead && !(lowest > fmaxf(best.others, kLowScore));
    }
  }
  __syncthreads();
  int token = last_token;
  if (unsure) token = exact_token<T, THREADS>(a, z, ok, noise, scores, lowest, q0, x, rejected, part, part_index);
  for (int i = n + tid; i <= K; i += THREADS) {
    int t = -1;
    float lp = 0.0f;
    if (i == n) {
      t = dead ? -1 : token;
      if (dead) lp = st.S == 0.0f ? -INFINITY : NAN;
      else if (t >= 0) lp = log_prob(a, logit(z, ok, t), st.m, st.S);
    }
    a.tokens[row0 + i] = t;
    a.logp[row0 + i] = lp;
  }
  if (tid == 0) a.accepted[seq] = n;
}

// CTAs a row or sequence: as many as `ctas` allow, as long as each has a few KB.
int parts_for(int64_t n, int64_t bytes, int most, int64_t ctas) {
  const int64_t parts = std::min(std::min<int64_t>(ctas / n, most), bytes / 4096);
  return static_cast<int>(std::max<int64_t>(parts, 1));
}

template <typename T>
cudaError_t verify_type(VerifyArgs a, cudaStream_t s) {
  const int64_t bytes = a.classes * static_cast<int64_t>(sizeof(T)), rows = a.sequences * (a.K + 1);
  const int load = 16 / static_cast<int>(sizeof(T));
  const bool filled = a.sequences >= kFilled;
  if (a.K < kOneThreads / 32 && a.sequences <= kOneSequences && a.classes <= (filled ? kManyClasses : kOneClasses) &&
      (a.K + 1) * a.classes <= (filled ? kManyElements : kOneElements)) {
    a.per = 1;
    while (2 * a.per * (a.K + 1) <= kOneThreads / 32) a.per *= 2;
    a.slack = slack(a.classes, 32 * a.per, load);
    const auto go = [&](auto mask) {
      constexpr bool M = decltype(mask)::value;
      return a.probs_type == HA_TYPE_BF16   ? k_verify_next<T, __nv_bfloat16, true, M>
             : a.probs_type == HA_TYPE_FP16 ? k_verify_next<T, __half, true, M>
                                            : k_verify_next<T, float, true, M>;
    };
    (a.allowed ? go(std::true_type()) : go(std::false_type()))<<<static_cast<unsigned>(a.sequences), kOneThreads, 0, s>>>(a);
    return cudaGetLastError();
  }
  // several rounds of CTAs for the sums, one for the scores, whose CTAs all look for n first
  a.sum_parts = parts_for(rows, bytes, kSumParts, 152 * kResident * 3);
  a.score_parts = parts_for(a.sequences, a.classes * int64_t(8), kScoreParts, 152 * kResident);
  a.slack = slack(a.classes / a.sum_parts + 1, kThreads, load);
  const auto sums = a.allowed ? k_verify_sums<T, true> : k_verify_sums<T, false>;
  sums<<<static_cast<unsigned>(rows * a.sum_parts), kThreads, 0, s>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const auto next = a.probs_type == HA_TYPE_BF16   ? k_verify_next<T, __nv_bfloat16, false, false>
                    : a.probs_type == HA_TYPE_FP16 ? k_verify_next<T, __half, false, false>
                                                   : k_verify_next<T, float, false, false>;
  return launch_early(next, static_cast<unsigned>(a.sequences * a.score_parts), kThreads, 0, s, a);
}

bool misaligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" int hier_avg_verify_workspace(int64_t sequences, int drafts, int64_t* bytes) {
  if (!bytes || sequences < 0 || drafts < 0) return HA_EINVAL;
  if (drafts == 0x7FFFFFFF || sequences > 0x7FFFFFFF / kSumParts / (drafts + int64_t(1)) || sequences > 0x7FFFFFFF / kScoreParts)
    return HA_EUNSUPPORTED;
  *bytes = sequences * ((drafts + int64_t(1)) * kRowBytes + kSequenceBytes);
  return HA_OK;
}

extern "C" int hier_avg_verify_drafts(const void* logits_dev, int type, int64_t sequences, int drafts, int64_t classes,
                                      int64_t logits_seq, int64_t logits_row, const void* drafts_dev, int draft_bytes,
                                      const float* uniform_dev, const float* noise_dev, int64_t noise_ld,
                                      const void* probs_dev, int probs_type, int64_t probs_seq, int64_t probs_row,
                                      const uint8_t* allowed_dev, int64_t allowed_seq, int64_t allowed_row,
                                      double temperature, int32_t* tokens_dev, int32_t* accepted_dev, float* logp_dev,
                                      void* workspace_dev, int64_t workspace_bytes, void* stream) {
  if (!type_ok(type) || sequences < 0 || drafts < 0 || classes < 1 || classes > 0x7FFFFFFF - (1 << 20) || logits_seq < 0 ||
      logits_row < 0 || noise_ld < 0 || (draft_bytes != 4 && draft_bytes != 8) ||
      !(temperature >= FLT_MIN && temperature <= 1e27) || misaligned(logits_dev, type_size(type)) ||
      misaligned(workspace_dev, 16))
    return HA_EINVAL;
  if (probs_dev && (!type_ok(probs_type) || probs_seq < 0 || probs_row < 0 || misaligned(probs_dev, type_size(probs_type))))
    return HA_EINVAL;
  if (allowed_dev && (allowed_seq < 0 || allowed_row < 0)) return HA_EINVAL;
  int64_t need;
  if (const int e = hier_avg_verify_workspace(sequences, drafts, &need)) return e;
  if (sequences == 0) return HA_OK;
  if (!logits_dev || !noise_dev || (drafts > 0 && (!drafts_dev || !uniform_dev)) || !tokens_dev || !accepted_dev || !logp_dev)
    return HA_EINVAL;
  if (!workspace_dev || workspace_bytes < need) return HA_ENOMEM;
  VerifyArgs a = {};
  a.logits = logits_dev;
  a.z_seq = logits_seq;
  a.z_row = logits_row;
  a.drafts = drafts_dev;
  a.uniform = uniform_dev;
  a.noise = noise_dev;
  a.noise_ld = noise_ld;
  a.probs = probs_dev;
  a.q_seq = probs_seq;
  a.q_row = probs_row;
  a.allowed = allowed_dev;
  a.ok_seq = allowed_seq;
  a.ok_row = allowed_row;
  a.tokens = tokens_dev;
  a.accepted = accepted_dev;
  a.logp = logp_dev;
  a.inv_temperature = 1.0 / temperature;
  a.c2 = two(1.4426950408889634 / temperature);
  a.c = a.c2.hi;
  a.inv_t2 = two(1.0 / temperature);
  a.K = drafts;
  a.sequences = sequences;
  const int64_t rows = sequences * (drafts + int64_t(1));
  a.w.heads = static_cast<Head*>(workspace_dev);
  a.w.bests = reinterpret_cast<Best*>(a.w.heads + rows);
  a.w.sums = reinterpret_cast<Sum*>(a.w.bests + sequences * kScoreParts);
  a.w.done = reinterpret_cast<int*>(a.w.sums + rows * kSumParts);
  a.classes = static_cast<int>(classes);
  a.wide_drafts = draft_bytes == 8;
  a.probs_type = probs_dev ? probs_type : -1;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = type == HA_TYPE_FP32   ? verify_type<float>(a, s)
                        : type == HA_TYPE_BF16 ? verify_type<__nv_bfloat16>(a, s)
                                               : verify_type<__half>(a, s);
  return e == cudaSuccess ? HA_OK : HA_ECUDA;
}
