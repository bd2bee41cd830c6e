// Routing by scores: softmax or sigmoid scores of the router logits, a bias
// per expert on the choice alone, expert groups of which only the best
// compete, the k best experts with renormalised weights, and the histogram,
// offsets and stable permutation of the routes. Without a context, as the
// batched routing is.
//
// Of a token with logits l, scores s = 1 / (1 + exp(-l)), or exp(l - max l) /
// sum exp(l - max l); choice values c = s + b, or s where groups are worth sums of
// two (also where all groups compete), or the logits themselves (their order is the
// scores', but for scores that fp32 makes equal) where neither is so. LPT lanes
// take a token, G groups of LPT / G lanes, each lane up to EPL experts of one
// group. A choice value and its expert make one 40-bit key (the ordered bits of
// c, then 255 - id), held as a double 2^52 + key: a larger key is a larger c or,
// among equal ones, a lower id, one v_max_f64 or v_min_f64 orders two of them,
// and no two keys are equal. Each lane sorts its keys into a list of the KP best
// by a network, and lists merge over lanes: the larger of a[i] and b[KP - 1 - i]
// are the KP best of both, bitonic, and log2 KP steps sort them.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kernels.h"
#include "oled.h"

namespace oled {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kGateThreads = 256;
constexpr int kGateChunkMax = 64;    // tokens whose routes one workgroup ranks, at most
constexpr int kGateSolo = 64;        // tokens of the form with one workgroup, at most
constexpr int kSoloThreads = 512;
constexpr int kScanPer = 32;         // chunks of a thread of the scan, at most
constexpr int kSumChunks = 32;       // chunks that the placing workgroups add up themselves
constexpr float kGateEps = 1e-20f;   // added to the sum of a token's scores

struct GateArgs {
  const void* logits;
  const float* bias;       // [E] or null
  const uint8_t* mask;     // [T] or null: 0 leaves a token without routes
  int T, E, k, G, top_groups, best;
  int softmax, renorm, bf16;
  int aligned;             // logits on a 16-byte boundary
  float scale;
  int32_t* idx;
  float* weights;
  int32_t* counts;
  int32_t* offsets;
  int32_t* perm;
  int32_t* inv_perm;       // between the launches: rank of a route in its chunk
  int32_t* bad;            // or null
  int32_t* chunk;          // [chunks][E] routes of each chunk, then those before it
  int32_t* total;          // [E]
  int chunks, per;         // chunks, and tokens of one
};

// 2^52 + 40-bit key of a choice value (not -0) and its expert, 255 - e of it. Infinities
// and NaN rank by their bits, so that k distinct experts are always chosen.
__device__ __forceinline__ double choice_key(float c, int rest) {
  const uint32_t b = __float_as_uint(c);
  const uint32_t u = b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
  return __hiloint2double(static_cast<int>(__builtin_amdgcn_alignbit(0x00433000u, u, 24)),   // 0x43300000 | u >> 24
                          static_cast<int>((u << 8) + static_cast<uint32_t>(rest)));
}
constexpr double kNoKey = 4503599627370496.0;   // 2^52: below every key of a float

__device__ __forceinline__ float key_value(double key) {
  const uint32_t u = (static_cast<uint32_t>(__double2hiint(key)) << 24) |
                     (static_cast<uint32_t>(__double2loint(key)) >> 8);
  return __uint_as_float(u ^ (static_cast<uint32_t>(~(static_cast<int32_t>(u) >> 31)) | 0x80000000u));
}

// Keys are never NaN: fmax would first quiet one.
__device__ __forceinline__ double larger(double a, double b) {
  double r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ double smaller(double a, double b) {
  double r;
  asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ void order(double& a, double& b) {   // the larger first
  const double hi = larger(a, b), lo = smaller(a, b);
  a = hi;
  b = lo;
}

// Batcher's odd-even merge sort, largest first.
template <int N>
__device__ __forceinline__ void sort_keys(double (&v)[N]) {
#pragma unroll
  for (int p = 1; p < N; p *= 2)
#pragma unroll
    for (int q = p; q >= 1; q /= 2)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int d = i - q % p;
        if (d >= 0 && d % (2 * q) < q && i + q < N && i / (2 * p) == (i + q) / (2 * p)) order(v[i], v[i + q]);
      }
}

// a <- the N best of two lists in order, in order.
template <int N>
__device__ __forceinline__ void merge_keys(double (&a)[N], const double (&b)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) a[i] = larger(a[i], b[N - 1 - i]);
#pragma unroll
  for (int d = N / 2; d >= 1; d /= 2)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!(i & d)) order(a[i], a[i + d]);
}

// Expert of list entry j. (The empty asm keeps the compiler from choosing an address
// first and the list in memory for it.)
template <int N>
__device__ __forceinline__ int pick_expert(const double (&v)[N], int j) {
  int r = __double2loint(v[0]);
#pragma unroll
  for (int i = 1; i < N; ++i) {
    int x = __double2loint(v[i]);
    asm("" : "+v"(x));
    r = i == j ? x : r;
  }
  return 255 - (r & 255);
}

// The value of a partner lane in the other half of 2 D lanes (any, where the lanes
// of a half hold the same): DPP quad permutations and mirrors up to 16 lanes.
template <int D>
__device__ __forceinline__ int from_half(int v) {
  if constexpr (D == 1) return __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);    // lanes 1 0 3 2
  else if constexpr (D == 2) return __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true);  // 2 3 0 1
  else if constexpr (D == 4) return __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true); // mirror of 8
  else if constexpr (D == 8) return __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true); // mirror of 16
  else return __shfl_xor(v, D);
}
template <int D>
__device__ __forceinline__ double from_half(double v) {
  return __hiloint2double(from_half<D>(__double2hiint(v)), from_half<D>(__double2loint(v)));
}
template <int D>
__device__ __forceinline__ float from_half(float v) {
  return __int_as_float(from_half<D>(__float_as_int(v)));
}

// Over halves of 1, 2, ... LPT / 2 lanes: f(integral_constant<D>).
template <int LPT, int D = 1, class F>
__device__ __forceinline__ void over_halves(F&& f) {
  if constexpr (D < LPT) {
    f(std::integral_constant<int, D>{});
    over_halves<LPT, 2 * D>(f);
  }
}

// exp(x) by v_exp_f32: within 2 + |x| units of 2^-24.
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

__device__ __forceinline__ float logit_at(const GateArgs& a, size_t i) {
  return a.bf16 ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(a.logits)[i]) << 16)
                : static_cast<const float*>(a.logits)[i];
}

// Where a lane's logits and biases come from: part(p, v) gives the 8 from its p-th on
// (anything past its last).
struct FromMemory {
  template <int EPL>
  struct Source {
    float l[EPL];
    const GateArgs& a;
    int e0;
    __device__ __forceinline__ Source(const GateArgs& args, size_t row, int first, int n) : a(args), e0(first) {
      if (a.bf16) {
        const uint16_t* p = static_cast<const uint16_t*>(a.logits) + row + e0;
#pragma unroll
        for (int i = 0; i < EPL; ++i) l[i] = i < n ? __uint_as_float(static_cast<uint32_t>(p[i]) << 16) : 0.f;
      } else {
        const float* p = static_cast<const float*>(a.logits) + row + e0;
        if (a.aligned && (a.E | e0 | n) % 4 == 0) {
#pragma unroll
          for (int i = 0; i < EPL; i += 4) {
            u32x4_t v{0u, 0u, 0u, 0u};
            if (i < n) v = *reinterpret_cast<const u32x4_t*>(p + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) l[i + j] = __uint_as_float(v[j]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < EPL; ++i) l[i] = i < n ? p[i] : 0.f;
        }
      }
    }
    __device__ __forceinline__ void part(int p, float (&v)[8]) const {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = l[p + i];
    }
    __device__ __forceinline__ void bias(int p, float (&v)[8]) const {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = a.bias[min(e0 + p + i, a.E - 1)];
    }
  };
};

// Routes token t with LPT lanes (`sub` is the lane's number among them, e0 its first
// expert, n its experts, 0 for a token without routes; no lane has more than epl):
// writes its ids and weights; list: its best keys, on all of them. FULL: every lane has
// EPL experts, and what it makes of a token without routes is not used.
template <int LPT, int EPL, int KP, bool FULL, class Source>
__device__ __forceinline__ void route_scored(const GateArgs& a, const Source& src, int t, int sub, int e0,
                                             int n, int epl, bool live, double (&list)[KP], bool* bad) {
  const size_t row = static_cast<size_t>(t) * a.E;
  const int lpg = LPT / a.G, S = a.E / a.G, g = sub / lpg;   // lanes and experts of a group, the lane's group
  float top = -__builtin_inff(), sum = 0.f;
  if (a.softmax || a.bad) {
    float check = 0.f;
#pragma unroll
    for (int p = 0; p < EPL; p += 8) {
      if (!FULL && p > 0 && p >= epl) continue;
      float v[8];
      src.part(p, v);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (FULL || p + i < n) {
          check = fmaf(v[i], 0.f, check);   // NaN where a logit is NaN or infinite
          top = fmaxf(top, v[i]);
        }
    }
    *bad |= live && !(check == 0.f);
  }
  if (a.softmax) {
    over_halves<LPT>([&](auto d) { top = fmaxf(top, from_half<decltype(d)::value>(top)); });
#pragma unroll
    for (int p = 0; p < EPL; p += 8) {
      if (!FULL && p > 0 && p >= epl) continue;
      float v[8];
      src.part(p, v);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (FULL || p + i < n) sum += fast_exp(v[i] - top);
    }
    over_halves<LPT>([&](auto d) { sum += from_half<decltype(d)::value>(sum); });
    sum = 1.f / sum;
  }
  const bool by_score = a.bias != nullptr || a.best == 2;
  auto score = [&](float x) {
    return a.softmax ? fast_exp(x - top) * sum : __builtin_amdgcn_rcpf(1.f + fast_exp(-x));
  };
  // this lane's KP best
#pragma unroll
  for (int i = 0; i < KP; ++i) list[i] = kNoKey;
#pragma unroll
  for (int p = 0; p < EPL; p += 8) {
    if (!FULL && p > 0 && p >= epl) continue;
    float c[8];
    src.part(p, c);
    if (by_score) {
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = score(c[i]);
      if (a.bias) {
        float b[8];
        src.bias(p, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] += b[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] += 0.f;   // -0 becomes +0
    }
    double key[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double v = choice_key(c[i], 255 - e0 - p - i);
      key[i] = FULL || p + i < n ? v : kNoKey;
    }
    sort_keys(key);
    if (p == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) list[i] = key[i];
    } else {
      double part[KP];
#pragma unroll
      for (int i = 0; i < KP; ++i) part[i] = i < 8 ? key[i & 7] : kNoKey;
      merge_keys(list, part);
    }
  }
  auto merge_over = [&](auto d) {
    double other[KP];
#pragma unroll
    for (int i = 0; i < KP; ++i) other[i] = from_half<decltype(d)::value>(list[i]);
    merge_keys(list, other);
  };
  over_halves<LPT>([&](auto d) {
    if (decltype(d)::value < lpg) merge_over(d);
  });
  if (a.top_groups < a.G) {
    // value of this lane's group, then the groups that come before it
    float v = key_value(list[0]);
    if (a.best == 2 && S >= 2) v += key_value(list[1]);
    int before = 0;
    for (int o = 1; o < a.G; ++o) {
      const int og = g ^ o;
      const float ov = __shfl_xor(v, o * lpg);
      before += (ov > v || (ov == v && og < g)) ? 1 : 0;
    }
    if (before >= a.top_groups)
#pragma unroll
      for (int i = 0; i < KP; ++i) list[i] = kNoKey;
  }
  over_halves<LPT>([&](auto d) {
    if (decltype(d)::value >= lpg) merge_over(d);
  });

  // weights: lane `sub` takes slots sub, sub + LPT, ...
  constexpr int PER = (KP + LPT - 1) / LPT;
  float w[PER], s = 0.f;
  int id[PER];
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int j = sub + p * LPT;
    id[p] = min(pick_expert(list, j), a.E - 1);
    w[p] = live && j < a.k ? score(logit_at(a, row + id[p])) : 0.f;
    s += w[p];
  }
  over_halves<LPT>([&](auto d) { s += from_half<decltype(d)::value>(s); });
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int j = sub + p * LPT;
    if (j < a.k && t < a.T) {
      const size_t r = static_cast<size_t>(t) * a.k + j;
      a.idx[r] = live ? id[p] : -1;
      a.weights[r] = live ? (a.renorm ? w[p] / (s + kGateEps) : w[p]) * a.scale : 0.f;
    }
  }
}

// The same with the logits straight from memory.
template <int LPT, int EPL, int KP>
__device__ __forceinline__ void route_direct(const GateArgs& a, int t, int sub, bool live, double (&list)[KP],
                                             bool* bad) {
  const int lpg = LPT / a.G, S = a.E / a.G, epl = (S + lpg - 1) / lpg;
  const int g = sub / lpg, e0 = g * S + (sub - g * lpg) * epl;
  const int n = live ? min(epl, (g + 1) * S - e0) : 0;
  const FromMemory::Source<EPL> src(a, static_cast<size_t>(t) * a.E, e0, n);
  route_scored<LPT, EPL, KP, false>(a, src, t, sub, e0, n, epl, live, list, bad);
}

__device__ __forceinline__ int scan64(int v) {   // inclusive, over a wavefront
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// Offsets of the experts from their counts, by one wavefront: lane l takes experts
// 4l .. 4l + 3.
__device__ __forceinline__ void scan_experts(const int (&n)[4], int E, int* s_off) {
  const int e0 = 4 * (threadIdx.x & 63);
  const int incl = scan64(n[0] + n[1] + n[2] + n[3]);
  int at = incl - (n[0] + n[1] + n[2] + n[3]);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (e0 + i < E) s_off[e0 + i] = at;
    at += n[i];
  }
  if ((threadIdx.x & 63) == 63) s_off[E] = at;
}

// A chunk's routes per expert, and the rank of each (stable: by expert, then token).
// Each expert has a bit per token of the chunk: a route's rank is the number of lower
// bits set.
constexpr int kMaskWords = kGateChunkMax / 32 + 1;   // of an expert, odd for the LDS banks
template <int THREADS>
__device__ __forceinline__ void rank_chunk(const GateArgs& a, const uint32_t* s_mask, int chunk, bool bad) {
  constexpr int W = kMaskWords;
  const int t0 = chunk * a.per;
  if (a.bad && __any(bad) && (threadIdx.x & 63) == 0) atomicOr(a.bad, 1);
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += THREADS)
    a.chunk[static_cast<size_t>(chunk) * a.E + e] = __popc(s_mask[e * W]) + __popc(s_mask[e * W + 1]);
  const int routes = min(a.per, a.T - t0) * a.k;
  for (int i = threadIdx.x; i < routes; i += THREADS) {
    const int c = i / a.k;
    const size_t r = static_cast<size_t>(t0) * a.k + i;
    const int e = a.idx[r];
    int rank = -1;
    if (e >= 0) {
      rank = __popc(s_mask[e * W + (c >> 5)] & ((1u << (c & 31)) - 1u));
      if (c >= 32) rank += __popc(s_mask[e * W]);
    }
    a.inv_perm[r] = rank;
  }
}

template <int LPT, int KP>
__device__ __forceinline__ void mark_routes(const GateArgs& a, const double (&list)[KP], int sub, int c,
                                            uint32_t* s_mask) {
  for (int j = sub; j < a.k; j += LPT)
    atomicOr(&s_mask[min(pick_expert(list, j), a.E - 1) * kMaskWords + (c >> 5)], 1u << (c & 31));
}

template <int LPT, int EPL, int KP, int THREADS>
__global__ __launch_bounds__(THREADS) void k_gate_route(GateArgs a) {
  __shared__ uint32_t s_mask[kMaxExperts * kMaskWords];
  for (int i = threadIdx.x; i < a.E * kMaskWords; i += THREADS) s_mask[i] = 0u;
  __syncthreads();
  const int sub = threadIdx.x % LPT;
  bool bad = false;
  for (int c = threadIdx.x / LPT; c < a.per; c += THREADS / LPT) {
    const int t = blockIdx.x * a.per + c;
    const bool live = t < a.T && (!a.mask || a.mask[t]);
    double list[KP];
    route_direct<LPT, EPL, KP>(a, t, sub, live, list, &bad);
    if (live) mark_routes<LPT>(a, list, sub, c, s_mask);
  }
  rank_chunk<THREADS>(a, s_mask, blockIdx.x, bad);
}

// Many tokens whose 8 lanes have EPL experts each, no more and no fewer: a wavefront's 8
// rows are one piece of memory, copied by LDS DMA in whole lines, from which lane l
// takes its NC 16-byte pieces. Piece c of lane l lies in place c ^ (l * NC / 16) of the
// lane's NC, so that 16 lanes reading a piece hit all banks once. 65535 tokens x 256
// experts in fp32, 8 groups, k = 8: 24.5 us (67 MB, 2.7 TB/s), bound by instructions:
// 32 keys a lane into a list of 8 are some 300 64-bit minima and maxima.
template <int EPL, int KP, bool BF16>
__global__ __launch_bounds__(256) void k_gate_rows(GateArgs a) {
  constexpr int NC = EPL * (BF16 ? 2 : 4) / 16;
  constexpr int LOG = NC == 8 ? 3 : NC == 4 ? 2 : NC == 2 ? 1 : 0;
  __shared__ uint32_t s_mask[kMaxExperts * kMaskWords];
  __shared__ __align__(1024) u32x4_t s_rows[4][64 * NC];
  __shared__ __align__(16) float s_bias[8][EPL + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = lane & 7;
  for (int i = threadIdx.x; i < a.E * kMaskWords; i += 256) s_mask[i] = 0u;
  if (a.bias && static_cast<int>(threadIdx.x) < a.E) s_bias[threadIdx.x / EPL][threadIdx.x % EPL] = a.bias[threadIdx.x];
  __syncthreads();

  struct Source {
    const u32x4_t* rows;   // this lane's NC pieces
    const float* biases;
    int turn;
    __device__ __forceinline__ void part(int p, float (&v)[8]) const {
      if constexpr (BF16) {
        const u32x4_t r = rows[(p / 8) ^ turn];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[2 * j] = __uint_as_float(r[j] << 16);
          v[2 * j + 1] = __uint_as_float(r[j] & 0xFFFF0000u);
        }
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x4_t r = rows[(p / 4 + h) ^ turn];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[4 * h + j] = __uint_as_float(r[j]);
        }
      }
    }
    __device__ __forceinline__ void bias(int p, float (&v)[8]) const {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = biases[p + i];
    }
  };
  auto turn_of = [](int l) { return (l >> (4 - LOG)) & (NC - 1); };
  const Source src{&s_rows[wave][lane * NC], s_bias[sub], turn_of(lane)};
  const int bytes = a.E * (BF16 ? 2 : 4);
  bool bad = false;
  for (int c0 = 8 * wave; c0 < a.per; c0 += 32) {
    const int t0 = blockIdx.x * a.per + c0;
    if (t0 >= a.T) break;
    const uint64_t base = reinterpret_cast<uint64_t>(a.logits) + static_cast<uint64_t>(t0) * bytes;
    const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void*>(base), 0, min(8, a.T - t0) * bytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int p = 64 * i + lane, o = p >> LOG;   // piece p in LDS belongs to lane o
      const int at = o * 16 * NC + 16 * ((p & (NC - 1)) ^ turn_of(o));
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rows, (__attribute__((address_space(3))) void*)&s_rows[wave][64 * i], 16, at, 0, 0, 0);
    }
    const int c = c0 + (lane >> 3), t = blockIdx.x * a.per + c;
    const bool live = t < a.T && (!a.mask || a.mask[t]);
    __builtin_amdgcn_s_waitcnt(0);   // a wavefront reads only what it copied itself
    asm volatile("" ::: "memory");
    double list[KP];
    route_scored<8, EPL, KP, true>(a, src, t, sub, sub * EPL, EPL, EPL, live, list, &bad);
    if (live) mark_routes<8>(a, list, sub, c, s_mask);
  }
  rank_chunk<256>(a, s_mask, blockIdx.x, bad);
}

// Counts of the chunks -> routes before each chunk, and the experts' totals. A
// workgroup takes 8 experts, a thread PER consecutive chunks of one. A launch and a
// latency each way: 5.7 us for 1024 chunks x 256 experts.
constexpr int kScanExperts = 8, kScanParts = 256 / kScanExperts;
template <int PER>
__global__ __launch_bounds__(256) void k_gate_scan(int32_t* __restrict__ chunk, int32_t* __restrict__ total,
                                                   int chunks, int E) {
  __shared__ int s_wave[4][kScanExperts];   // of the parts of each wavefront
  const int e = blockIdx.x * kScanExperts + static_cast<int>(threadIdx.x) % kScanExperts;
  const int part = threadIdx.x / kScanExperts, i0 = part * PER;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int v[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    v[i] = e < E && i0 + i < chunks ? chunk[static_cast<size_t>(i0 + i) * E + e] : 0;
    sum += v[i];
  }
  int incl = sum;
#pragma unroll
  for (int d = kScanExperts; d < 64; d *= 2) {
    const int up = __shfl_up(incl, d);
    if (lane >= d) incl += up;
  }
  if (lane >= 64 - kScanExperts) s_wave[wave][lane % kScanExperts] = incl;
  __syncthreads();
  int at = incl - sum;
#pragma unroll
  for (int w = 0; w < 3; ++w) at += w < wave ? s_wave[w][lane % kScanExperts] : 0;
  if (e >= E) return;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (i0 + i < chunks) chunk[static_cast<size_t>(i0 + i) * E + e] = at;
    at += v[i];
  }
  if (part == kScanParts - 1) total[e] = at;
}

// Offsets of the experts (every workgroup for itself), and the place of each
// route of a chunk: offset + routes of earlier chunks + rank in its chunk. SUM: the
// chunks' counts are as the routing launch left them, and each workgroup adds up
// those of its experts' earlier chunks itself. 65535 tokens x 8 routes: 5.0-5.6 us.
template <bool SUM>
__global__ __launch_bounds__(kGateThreads) void k_gate_place(GateArgs a) {
  __shared__ int s_total[kMaxExperts], s_before[kMaxExperts], s_off[kMaxExperts + 1];
  const int chunk = blockIdx.x, t0 = chunk * a.per;
  static_assert(kGateThreads == kMaxExperts, "a thread an expert");
  if (static_cast<int>(threadIdx.x) < a.E) {
    const int32_t* row = a.chunk + threadIdx.x;
    int before, total;
    if constexpr (SUM) {
      int v[kSumChunks];
      before = total = 0;
#pragma unroll
      for (int i = 0; i < kSumChunks; ++i) v[i] = i < a.chunks ? row[static_cast<size_t>(i) * a.E] : 0;
#pragma unroll
      for (int i = 0; i < kSumChunks; ++i) {
        total += v[i];
        before += i < chunk ? v[i] : 0;
      }
    } else {
      before = row[static_cast<size_t>(chunk) * a.E];
      total = a.total[threadIdx.x];
    }
    s_before[threadIdx.x] = before;
    s_total[threadIdx.x] = total;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    int n[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = 4 * static_cast<int>(threadIdx.x) + i;
      n[i] = e < a.E ? s_total[e] : 0;
    }
    scan_experts(n, a.E, s_off);
  }
  __syncthreads();
  if (chunk == 0) {
    for (int e = threadIdx.x; e <= a.E; e += kGateThreads) {
      a.offsets[e] = s_off[e];
      if (e < a.E) a.counts[e] = s_total[e];
    }
  }
  const int routes = min(a.per, a.T - t0) * a.k;
  const int used = s_off[a.E];
  for (int i = threadIdx.x; i < routes; i += kGateThreads) {
    const size_t r = static_cast<size_t>(t0) * a.k + i;
    const int e = a.idx[r];
    if (e >= 0) {
      const int pos = s_off[e] + s_before[e] + a.inv_perm[r];
      a.inv_perm[r] = pos;
      a.perm[pos] = static_cast<int32_t>(r);
    }
    if (r >= static_cast<size_t>(used)) a.perm[r] = -1;   // places without a route
  }
}

// Up to kGateSolo tokens in one workgroup: routed as above, ranked from the bits and
// placed in the same launch. Bound by latency: 1 token x 256 experts 5.6 us of the
// device, of which an empty launch is 2.3.
template <int LPT, int EPL, int KP, int THREADS>
__global__ __launch_bounds__(THREADS) void k_gate_solo(GateArgs a) {
  constexpr int W = kGateSolo / 32 + 1;
  __shared__ uint32_t s_mask[kMaxExperts * W];
  __shared__ int16_t s_idx[kGateSolo * kMaxTopK];
  __shared__ int s_off[kMaxExperts + 1];
  __shared__ int s_bad;
  for (int i = threadIdx.x; i < a.E * W; i += THREADS) s_mask[i] = 0u;
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();
  const int sub = threadIdx.x % LPT;
  bool bad = false;
  for (int t = threadIdx.x / LPT; t < a.T; t += THREADS / LPT) {
    const bool live = !a.mask || a.mask[t];
    double list[KP];
    route_direct<LPT, EPL, KP>(a, t, sub, live, list, &bad);
    for (int j = sub; j < a.k; j += LPT) {
      const int e = min(pick_expert(list, j), a.E - 1);
      s_idx[t * a.k + j] = static_cast<int16_t>(live ? e : -1);
      if (live) atomicOr(&s_mask[e * W + (t >> 5)], 1u << (t & 31));
    }
  }
  if (__any(bad) && (threadIdx.x & 63) == 0) s_bad = 1;
  __syncthreads();
  if (threadIdx.x < 64) {
    int n[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = 4 * static_cast<int>(threadIdx.x) + i;
      n[i] = 0;
      if (e < a.E) {
#pragma unroll
        for (int w = 0; w < W - 1; ++w) n[i] += __popc(s_mask[e * W + w]);
        a.counts[e] = n[i];
      }
    }
    scan_experts(n, a.E, s_off);
    if (a.bad && threadIdx.x == 0) *a.bad = s_bad;
  }
  __syncthreads();
  for (int e = threadIdx.x; e <= a.E; e += THREADS) a.offsets[e] = s_off[e];
  const int routes = a.T * a.k, used = s_off[a.E];
  for (int r = threadIdx.x; r < routes; r += THREADS) {
    const int e = s_idx[r], t = r / a.k;
    int pos = -1;
    if (e >= 0) {
      pos = s_off[e];
#pragma unroll
      for (int w = 0; w < W - 1; ++w) {
        const uint32_t m = s_mask[e * W + w];
        pos += __popc(w < (t >> 5) ? m : w == (t >> 5) ? m & ((1u << (t & 31)) - 1u) : 0u);
      }
      a.perm[pos] = r;
    }
    a.inv_perm[r] = pos;
    if (r >= used) a.perm[r] = -1;
  }
}

__global__ void k_gate_clear(int32_t* bad) { *bad = 0; }

// Tokens of a chunk: 16 while that gives the chip no more than two workgroups a CU. us of a
// call, 256 experts, 16 against 64: 512 tokens 10.2 : 14.8, 4096 12.3 : 17.0, 8192 16.4 : 18.4.
constexpr int kGateShort = 8192;   // tokens up to which a chunk has 16
int gate_per(int T) { return T <= kGateShort ? 16 : kGateChunkMax; }
int gate_chunks(int T) { return (T + gate_per(T) - 1) / gate_per(T); }
static_assert((65535 + kGateChunkMax - 1) / kGateChunkMax <= kScanParts * kScanPer, "a thread's chunks");

template <int LPT, int EPL, int THREADS>
hipError_t launch_gate_route(const GateArgs& a, hipStream_t s) {
  if (a.k <= 8)
    hipLaunchKernelGGL((k_gate_route<LPT, EPL, 8, THREADS>), dim3(a.chunks), dim3(THREADS), 0, s, a);
  else
    hipLaunchKernelGGL((k_gate_route<LPT, EPL, 16, THREADS>), dim3(a.chunks), dim3(THREADS), 0, s, a);
  return hipGetLastError();
}

template <int LPT, int EPL>
hipError_t launch_gate_solo(const GateArgs& a, hipStream_t s) {
  if (a.k <= 8)
    hipLaunchKernelGGL((k_gate_solo<LPT, EPL, 8, kSoloThreads>), dim3(1), dim3(kSoloThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_gate_solo<LPT, EPL, 16, kSoloThreads>), dim3(1), dim3(kSoloThreads), 0, s, a);
  return hipGetLastError();
}

template <int EPL>
hipError_t launch_gate_rows(const GateArgs& a, hipStream_t s) {
  const dim3 grid(a.chunks), block(256);
  if (a.k <= 8) {
    if (a.bf16)
      hipLaunchKernelGGL((k_gate_rows<EPL, 8, true>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((k_gate_rows<EPL, 8, false>), grid, block, 0, s, a);
  } else {
    if (a.bf16)
      hipLaunchKernelGGL((k_gate_rows<EPL, 16, true>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((k_gate_rows<EPL, 16, false>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

hipError_t launch_gate(const GateArgs& a, hipStream_t s) {
  // experts of a lane with 8 lanes a token (64: more groups than lanes)
  const int dense = a.G <= 8 ? (a.E / a.G + 8 / a.G - 1) / (8 / a.G) : 64;
  // One workgroup against two launches, us of the device: 16 tokens x 256 experts 8.0 :
  // 9.5, 32 x 256 9.5 : 10.0, 48 x 256 15 : 9.9; 64 x 64 6.5 : 8.0, 128 x 64 10.0 : 8.5.
  if (a.T <= kGateSolo && a.T * min(dense, 32) <= 512) {
    // 8 lanes a token against 32: 1 x 64 4.5 : 5.0, 64 x 64 6.5 : 13.8; 1 x 256 9.4 : 6.1
    if (dense <= 8) return launch_gate_solo<8, 8>(a, s);
    if (dense <= 16) return launch_gate_solo<8, 16>(a, s);
    return launch_gate_solo<32, 8>(a, s);
  }
  if (a.bad) {
    hipLaunchKernelGGL(k_gate_clear, dim3(1), dim3(1), 0, s, a.bad);
    if (hipError_t e = hipGetLastError()) return e;
  }
  hipError_t e;
  // us of a call on the device. Rows by LDS DMA against lanes that load their own: 65535 x
  // 256 36 : 49, 65535 x 64 23.6 : 24.5, 4096 x 256 12.3 : 13.4, 128 x 64 7.1 : 7.5. 32 lanes
  // a token against 8: 512 x 200 10.0 : 11.6, 4096 x 200 12.3 : 13.7, 8192 x 200 alike;
  // 512 x 96 9.5 : 8.7, 4096 x 96 11.8 : 10.9.
  if (a.aligned && dense * 8 == a.E && (dense == 8 || dense == 16 || dense == 32))
    e = dense == 8 ? launch_gate_rows<8>(a, s) : dense == 16 ? launch_gate_rows<16>(a, s) : launch_gate_rows<32>(a, s);
  else if (dense > 32 || (dense > 16 && a.T <= 4096))
    e = launch_gate_route<32, 8, 512>(a, s);
  else if (dense <= 8)
    e = launch_gate_route<8, 8, 256>(a, s);
  else if (dense <= 16)
    e = launch_gate_route<8, 16, 256>(a, s);
  else
    e = launch_gate_route<8, 32, 256>(a, s);
  if (e != hipSuccess) return e;
  // Without the scan's launch: 128 x 256 9.6 : 11.4, 512 x 256 10.2 : 11.6; each workgroup
  // adds up all chunks, which past kSumChunks costs what the launch does.
  if (a.chunks <= kSumChunks) {
    hipLaunchKernelGGL(k_gate_place<true>, dim3(a.chunks), dim3(kGateThreads), 0, s, a);
    return hipGetLastError();
  }
  const dim3 scan((a.E + kScanExperts - 1) / kScanExperts);
  if (a.chunks <= 8 * kScanParts)
    hipLaunchKernelGGL(k_gate_scan<8>, scan, dim3(256), 0, s, a.chunk, a.total, a.chunks, a.E);
  else
    hipLaunchKernelGGL(k_gate_scan<kScanPer>, scan, dim3(256), 0, s, a.chunk, a.total, a.chunks, a.E);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(k_gate_place<false>, dim3(a.chunks), dim3(kGateThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace oled

extern "C" size_t oled_route_scored_workspace(int32_t T, int32_t E) {
  if (T < 1 || E < 1) return 0;
  // what T tokens need and any number below T
  int chunks = oled::gate_chunks(T);
  if (T > oled::kGateShort && chunks < oled::gate_chunks(oled::kGateShort))
    chunks = oled::gate_chunks(oled::kGateShort);
  return sizeof(int32_t) * static_cast<size_t>(E) * (chunks + 1);
}

extern "C" oled_status oled_route_scored(const oled_router* router, const void* logits_dev,
                                         const float* bias_dev, const uint8_t* token_mask_dev,
                                         int32_t T, int32_t* topk_idx_dev, float* weights_dev,
                                         int32_t* counts_dev, int32_t* offsets_dev,
                                         int32_t* perm_dev, int32_t* inv_perm_dev,
                                         int32_t* nonfinite_dev, void* workspace_dev,
                                         size_t workspace_bytes, void* stream) {
  if (!router || !logits_dev || !topk_idx_dev || !weights_dev || !counts_dev || !offsets_dev ||
      !perm_dev || !inv_perm_dev || !workspace_dev) {
    oled::set_noctx_error("oled_route_scored: NULL router, input, output or workspace");
    return OLED_ERR_INVALID_ARG;
  }
  const oled_router& r = *router;
  const int E = r.n_experts, k = r.top_k, G = r.n_groups;
  if (T < 1 || E < 1 || k < 1 || G < 1 || E % G != 0 || r.top_groups < 1 || r.top_groups > G ||
      k > r.top_groups * (E / G)) {
    oled::set_noctx_error("oled_route_scored: T, n_experts, top_k and n_groups must be >= 1, "
                          "n_groups must divide n_experts, top_groups be in [1, n_groups] and "
                          "top_k at most the experts of top_groups groups");
    return OLED_ERR_INVALID_ARG;
  }
  if ((r.score != OLED_SCORE_SOFTMAX && r.score != OLED_SCORE_SIGMOID) ||
      (r.dtype != OLED_F32 && r.dtype != OLED_BF16) || (r.group_best != 1 && r.group_best != 2)) {
    oled::set_noctx_error("oled_route_scored: bad score, dtype or group_best");
    return OLED_ERR_INVALID_ARG;
  }
  if (T > 65535 || E > oled::kMaxExperts || k > oled::kMaxTopK || G > 32 || (G & (G - 1)) != 0) {
    oled::set_noctx_error("oled_route_scored: T above 65535, n_experts above 256, top_k above 16, "
                          "or n_groups not a power of two up to 32");
    return OLED_ERR_UNSUPPORTED;
  }
  if (workspace_bytes < oled_route_scored_workspace(T, E)) {
    oled::set_noctx_error("oled_route_scored: workspace smaller than "
                          "oled_route_scored_workspace(T, n_experts)");
    return OLED_ERR_INVALID_ARG;
  }
  oled::GateArgs a{};
  a.logits = logits_dev;
  a.bias = bias_dev;
  a.mask = token_mask_dev;
  a.T = T;
  a.E = E;
  a.k = k;
  a.G = G;
  a.top_groups = r.top_groups;
  a.best = r.group_best;
  a.softmax = r.score == OLED_SCORE_SOFTMAX;
  a.renorm = r.renorm;
  a.bf16 = r.dtype == OLED_BF16;
  a.aligned = (reinterpret_cast<uintptr_t>(logits_dev) & 15) == 0;
  a.scale = r.scale;
  a.idx = topk_idx_dev;
  a.weights = weights_dev;
  a.counts = counts_dev;
  a.offsets = offsets_dev;
  a.perm = perm_dev;
  a.inv_perm = inv_perm_dev;
  a.bad = nonfinite_dev;
  a.per = oled::gate_per(T);
  a.chunks = oled::gate_chunks(T);
  a.chunk = static_cast<int32_t*>(workspace_dev);
  a.total = a.chunk + static_cast<size_t>(E) * a.chunks;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (oled::launch_gate(a, s) != hipSuccess) {
    oled::set_noctx_error("oled_route_scored: launch failed");
    return OLED_ERR_HIP;
  }
  return OLED_OK;
}
