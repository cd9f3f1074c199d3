// Log probabilities of given tokens with entropy and top alternatives, and their gradient.
//   lse = log sum_v exp(x_v);  logprob = x_token - lse;  entropy = lse - sum_v p_v x_v,  p = exp(x - lse);
//   dx_v = p_v (g_lse - g_logprob - g_entropy (log p_v + entropy)) + [v = token] g_logprob.
// Forward: one pass over the logits.  A thread keeps the running maximum m, s = sum 2^y and t = sum y 2^y with
// y = (x - m) log2(e); when m grows by d (in units of log2), s becomes 2^-d s and t becomes 2^-d (t - d s).
// Alternatives: a candidate is an element at least as large as a lower bound of the k-th largest value; candidates
// go to a list in shared memory.  The bound comes from the first round of loads (its exact k-th largest element,
// found by cutting that round's candidates back to k), and again from rounds 4, 16, 64, ...; in between the warps
// of a CTA do not meet.  A row with more candidates than the list holds (rising values, ties) is scanned again for them alone.
// A row is shared by the CTAs of a cluster where there are fewer rows than the GPU has room for.
#include <cooperative_groups.h>

#include "qasg_lm.cuh"

namespace qasg {
namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kTiny = -160.f;  // 2^kTiny is 0 in fp32: stands for every smaller power, so that 0 * y is 0
template <typename T> constexpr int kRoundUnits = sizeof(T) == 4 ? 2 : 4;  // units a thread loads per round: 64 bytes
constexpr int kListSize = 1024;  // candidates a CTA has room for
constexpr int kMaxCluster = 8;

// 2^y within 2 units in the last place; below 2^-126 it is 0.
__device__ __forceinline__ float exp2_fast(float y) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  return r;
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 a, b, r;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 r, a, b;\nmov.b64 {%0, %1}, r;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 a, b, r;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 r, a, b;\nmov.b64 {%0, %1}, r;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n.reg .b64 a, b, c, r;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\n"
      "fma.rn.f32x2 r, a, b, c;\nmov.b64 {%0, %1}, r;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}

// Keys order values, NaN above all, then columns, the lowest first; the two zeros are equal.
__device__ __forceinline__ uint32_t value_order(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ unsigned long long value_key(float x, uint32_t column) {
  return (static_cast<unsigned long long>(value_order(x)) << 32) | (0xffffffffu - column);
}
__device__ __forceinline__ float key_value(unsigned long long key) {
  const uint32_t o = static_cast<uint32_t>(key >> 32);
  return __uint_as_float(o == 0xffffffffu ? 0x7fffffffu : (o >> 31) ? (o ^ 0x80000000u) : ~o);
}

// A unit of row values [i, i + 8) of n, -inf outside the row.
template <typename T> __device__ __forceinline__ Unit<T> load_row_unit(const T* row, int64_t i, int64_t n) {
  if (i >= 0 && i + kUnit <= n) return load_unit(row + i);  // the caller's units lie on 16-byte boundaries
  Unit<T> u;
#pragma unroll
  for (int k = 0; k < kUnit; ++k) {
    const float v = i + k >= 0 && i + k < n ? to_float(row[i + k]) : -INFINITY;
    set_value(u, k, v);
  }
  return u;
}
template <typename T> __device__ __forceinline__ float unit_top(const Unit<T>& u) {
  typedef decltype(pair_of(T())) Pair;
  Pair m = *reinterpret_cast<const Pair*>(&u.w[0]);
#pragma unroll
  for (int i = 1; i < kUnit / 2; ++i) m = __hmax2_nan(m, *reinterpret_cast<const Pair*>(&u.w[i]));
  return max_nan(to_float(m.x), to_float(m.y));
}
template <> __device__ __forceinline__ float unit_top<float>(const Unit<float>& u) {
  float m = __uint_as_float(u.w[0]);
#pragma unroll
  for (int i = 1; i < kUnit; ++i) m = max_nan(m, __uint_as_float(u.w[i]));
  return m;
}

struct RowSums {
  float m, s, t;
};
// Adds o to a; either may be empty (m = -inf, s = t = 0).
__device__ __forceinline__ RowSums join(RowSums a, RowSums o) {
  const float m = max_nan(a.m, o.m), base = m == -INFINITY ? 0.f : m;
  const float da = max_nan((a.m - base) * kLog2e, kTiny), db = max_nan((o.m - base) * kLog2e, kTiny);
  const float ca = exp2_fast(da), cb = exp2_fast(db);
  RowSums r;
  r.m = m;
  r.s = fmaf(ca, a.s, cb * o.s);
  r.t = fmaf(ca, fmaf(a.s, da, a.t), cb * fmaf(o.s, db, o.t));
  return r;
}

struct RowShared {
  unsigned long long list[kListSize];
  unsigned long long best[kMaxTop];
  float group_max[32];
  RowSums warp_sums[32];
  RowSums sums;
  unsigned int count, lost;
  unsigned long long bound;
};

// Cuts the list back to its k best, in order, also in `best`; raises the bound.  Called by all threads; what
// they pushed before is seen.  Keys are distinct, so an element's rank is the number of larger ones.
template <int kThreads>
__device__ __forceinline__ void cut_list(RowShared& sh, uint32_t k) {
  __syncthreads();
  const uint32_t n = min(sh.count, static_cast<unsigned>(kListSize));
  for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
    const unsigned long long key = sh.list[i];
    uint32_t rank = 0;
    for (uint32_t j = 0; j < n; ++j) rank += sh.list[j] > key;
    if (rank < k) sh.best[rank] = key;
  }
  __syncthreads();
  const uint32_t kept = min(n, k);
  for (uint32_t i = threadIdx.x; i < kept; i += kThreads) sh.list[i] = sh.best[i];
  if (threadIdx.x == 0) {
    sh.count = kept;
    if (kept == k) sh.bound = max(sh.bound, sh.best[k - 1] + 1ull);
  }
  __syncthreads();
}

// Puts the candidates among a thread's units (pending: a bit for each element still to be looked at) on the list;
// returns the bits of those that found no room.
template <typename T, int kThreads>
__device__ __forceinline__ uint32_t push_pending(RowShared& sh, const T* x, uint32_t pending, int64_t c0) {
  const unsigned long long limit = sh.bound;
  uint32_t left = 0;
  while (pending) {
    const int b = __ffs(pending) - 1;
    pending &= pending - 1;
    const uint32_t c = static_cast<uint32_t>(c0 + static_cast<int64_t>(b >> 3) * (kThreads * kUnit) + (b & 7));
    const unsigned long long key = value_key(to_float(x[c]), c);
    if (key < limit) continue;
    const uint32_t at = atomicAdd(&sh.count, 1u);
    if (at < kListSize) sh.list[at] = key;
    else left |= 1u << b;
  }
  return left;
}

// One round of units at which all warps meet, so that the list is cut back as often as it fills up.
template <typename T, int kThreads>
__device__ __noinline__ void push_round(RowShared& sh, const T* x, uint32_t k, uint32_t pending, int64_t c0) {
  do {
    pending = push_pending<T, kThreads>(sh, x, pending, c0);
    cut_list<kThreads>(sh, k);
  } while (__syncthreads_or(pending != 0));
}

template <typename T, int kThreads, bool kTop>
__global__ void __launch_bounds__(kThreads, 768 / kThreads)
token_logprob_kernel(LogprobArgs a, uint32_t cluster, unsigned int* __restrict__ status) {
  constexpr int kUnits = kRoundUnits<T>;
  __shared__ RowShared sh;
  const uint64_t row = blockIdx.x / cluster;
  const uint32_t part = blockIdx.x - static_cast<uint32_t>(row) * cluster, tid = threadIdx.x, vocab = a.vocab;
  chain_wait();
  chain_trigger();
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  int64_t token = 0;
  if (a.tokens) {
    token = a.tokens[row];
    if (token < 0 || token >= vocab) {  // the whole cluster leaves: a padding row is not read
      if (part == 0) {
        if (tid == 0) {
          if (a.logprob) a.logprob[row] = 0.f;
          if (a.entropy) a.entropy[row] = 0.f;
          if (a.lse) a.lse[row] = 0.f;
          if (token >= vocab) atomicOr(status, kFlagBadIndex);
        }
        if (kTop && tid < a.k) {
          if (a.top_ids) a.top_ids[row * a.k + tid] = -1;
          if (a.top_logprob) a.top_logprob[row * a.k + tid] = 0.f;
        }
      }
      return;
    }
  }
  if (kTop && tid == 0) sh.count = 0, sh.lost = 0, sh.bound = 0;
  // units on 16-byte boundaries: unit u holds columns 8u - off .. 8u - off + 7
  const uint32_t off = static_cast<uint32_t>((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T));
  const uint32_t units = (vocab + off + kUnit - 1) / kUnit, per_part = (units + cluster - 1) / cluster;
  const uint32_t u0 = part * per_part, u1 = min(units, u0 + per_part);
  RowSums r = {-INFINITY, 0.f, 0.f};
  float2 s2 = {0.f, 0.f}, t2 = {0.f, 0.f};  // s and t of the even and the odd columns
  float base = 0.f;                         // m, 0 while m is -inf
  float bound = -INFINITY;
  uint32_t meet = u0;  // the next round at which the list is cut back: 0, 4, 16, 64, ...
  // Rounds of units: the next one's loads are under way while one is worked on.
  const uint32_t whole = min(u1, (vocab + off) / kUnit);  // units before this one end inside the row; unit 0 may begin before it
  auto is_inside = [&](uint32_t u) { return u > 0 && u + kThreads * kUnits <= whole; };
  auto load = [&](uint32_t u, Unit<T>(&raw)[kUnits]) {
    const int64_t c0 = static_cast<int64_t>(u + tid) * kUnit - off;
    if (is_inside(u)) {
#pragma unroll
      for (int j = 0; j < kUnits; ++j) raw[j] = load_unit(x + c0 + j * kThreads * kUnit);
    } else {
#pragma unroll
      for (int j = 0; j < kUnits; ++j)
        raw[j] = load_row_unit<T>(x, c0 + j * kThreads * kUnit, u + j * kThreads + tid < u1 ? vocab : 0);
    }
  };
  Unit<T> raw[kUnits];
  if (u0 < u1) load(u0, raw);
  for (uint32_t u = u0; u < u1; u += kThreads * kUnits) {
    Unit<T> next[kUnits];
    if (u + kThreads * kUnits < u1) load(u + kThreads * kUnits, next);
    const int64_t c0 = static_cast<int64_t>(u + tid) * kUnit - off;
    float top[kUnits];
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      top[j] = unit_top(raw[j]);
      m = max_nan(m, top[j]);
    }
    if (!(m <= r.m)) {
      const float d = max_nan((r.m - m) * kLog2e, kTiny), c = exp2_fast(d);
      t2 = mul2(make_float2(c, c), fma2(s2, make_float2(d, d), t2));
      s2 = mul2(make_float2(c, c), s2);
      r.m = m;
      base = m;
    }
    if (kTop) {
      if (u == u0) {
        // The smallest of the largest elements of g groups is at most the g-th largest element of all, so with
        // g >= k at most the k-th: g groups of threads, g the power of two from k on (up to 32).
        constexpr int kLanes = kThreads / 32;
        float g = m == m ? m : INFINITY;
#pragma unroll
        for (int s = kLanes / 2; s > 0; s >>= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, s));
        if (tid % kLanes == 0) sh.group_max[tid / kLanes] = g;
        __syncthreads();
        g = sh.group_max[tid & 31];
        const uint32_t wide = 32u >> (32 - __clz(a.k - 1));  // of the 32 groups of kLanes threads in one of the g
        for (uint32_t s = 1; s < 32; s <<= 1) {
          const float o = __shfl_xor_sync(0xffffffffu, g, s);
          g = s < wide ? fmaxf(g, o) : fminf(g, o);
        }
        if (tid == 0) sh.bound = static_cast<unsigned long long>(value_order(g)) << 32;
        bound = g;
        __syncthreads();
      }
      uint32_t pending = 0;
      if (!(m < bound)) {
#pragma unroll
        for (int j = 0; j < kUnits; ++j)
          if (!(top[j] < bound)) {
            float v[kUnit];
            unit_floats(raw[j], v);
            uint32_t bits = 0;
#pragma unroll
            for (int k = 0; k < kUnit; ++k) bits |= v[k] < bound ? 0u : 1u << k;
            if (!is_inside(u)) {  // not what lies outside the row, or in another part
              const int64_t c = c0 + j * kThreads * kUnit;
              if (c < 0) bits &= 0xffu << -c;
              if (c + kUnit > vocab) bits &= c >= vocab ? 0u : 0xffu >> (c + kUnit - vocab);
              if (u + j * kThreads + tid >= u1) bits = 0u;
            }
            pending |= bits << (j * kUnit);
          }
      }
      if (u == meet) {
        push_round<T, kThreads>(sh, x, a.k, pending, c0);
        meet = u0 + max(4u * (u - u0), 4u * kThreads * kUnits);
        bound = key_value(sh.bound);
        if (bound != bound) bound = INFINITY;  // k NaNs: nothing but another NaN passes
      } else if (pending) {
        if (push_pending<T, kThreads>(sh, x, pending, c0)) sh.lost = 1u;
      }
    }
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      float v[kUnit];
      unit_floats(raw[j], v);
#pragma unroll
      for (int k = 0; k < kUnit; k += 2) {
        float2 y = mul2(add2(make_float2(v[k], v[k + 1]), make_float2(-base, -base)), make_float2(kLog2e, kLog2e));
        y.x = max_nan(y.x, kTiny), y.y = max_nan(y.y, kTiny);
        const float2 e = make_float2(exp2_fast(y.x), exp2_fast(y.y));
        s2 = add2(s2, e);
        t2 = fma2(e, y, t2);
      }
    }
#pragma unroll
    for (int j = 0; j < kUnits; ++j) raw[j] = next[j];
  }
  r.s = s2.x + s2.y, r.t = t2.x + t2.y;
  if (kTop) {
    __syncthreads();
    if (sh.lost) {
      // the k-th best of what was kept is a far better bound: once more, from the start, meeting at every round
      cut_list<kThreads>(sh, a.k);
      if (tid == 0) sh.count = 0, sh.bound = sh.best[a.k - 1];
      __syncthreads();
      for (uint32_t u = u0; u < u1; u += kThreads * kUnits) {
        const int64_t c0 = static_cast<int64_t>(u + tid) * kUnit - off;
        uint32_t pending = 0;
        const float limit = key_value(sh.bound);
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
          const uint32_t w = u + j * kThreads + tid;
          float v[kUnit];
          unit_floats(load_row_unit<T>(x, static_cast<int64_t>(w) * kUnit - off, w < u1 ? vocab : 0), v);
#pragma unroll
          for (int k = 0; k < kUnit; ++k) {
            const int64_t c = static_cast<int64_t>(w) * kUnit - off + k;
            if (!(v[k] < limit) && w < u1 && c >= 0 && c < vocab) pending |= 1u << (j * kUnit + k);
          }
        }
        push_round<T, kThreads>(sh, x, a.k, pending, c0);
      }
    }
  }
  const float given = to_float(x[token]);
  // join the threads, then the CTAs
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    RowSums o;
    o.m = __shfl_xor_sync(0xffffffffu, r.m, s);
    o.s = __shfl_xor_sync(0xffffffffu, r.s, s);
    o.t = __shfl_xor_sync(0xffffffffu, r.t, s);
    r = join(r, o);
  }
  if ((tid & 31) == 0) sh.warp_sums[tid >> 5] = r;
  if (kTop) cut_list<kThreads>(sh, a.k);
  else __syncthreads();
  r = sh.warp_sums[0];
#pragma unroll
  for (int i = 1; i < kThreads / 32; ++i) r = join(r, sh.warp_sums[i]);
  if (cluster > 1) {
    cg::cluster_group group = cg::this_cluster();
    if (tid == 0) sh.sums = r;
    group.sync();
    if (part == 0) {
      for (uint32_t o = 1; o < cluster; ++o) {
        const RowShared* other = group.map_shared_rank(&sh, o);
        r = join(r, other->sums);
        if (kTop && tid < other->count) {
          const uint32_t at = atomicAdd(&sh.count, 1u);
          sh.list[at] = other->list[tid];
        }
      }
    }
    group.sync();  // the other CTAs' shared memory has been read
    if (part) return;
    if (kTop) cut_list<kThreads>(sh, a.k);
  }
  const float log_s = logf(r.s);
  const bool empty = r.m == -INFINITY;  // every logit is -inf
  if (tid == 0) {
    if (a.logprob) a.logprob[row] = empty ? -INFINITY : (given - r.m) - log_s;
    if (a.entropy) a.entropy[row] = empty ? 0.f : log_s - r.t * kLn2 / r.s;
    if (a.lse) a.lse[row] = empty ? -INFINITY : r.m + log_s;
    if (!(fabsf(r.s) < INFINITY)) atomicOr(status, kFlagNonFinite);
  }
  if (kTop && tid < a.k) {
    const unsigned long long key = sh.best[tid];
    if (a.top_ids) a.top_ids[row * a.k + tid] = 0xffffffffu - static_cast<uint32_t>(key);
    if (a.top_logprob) a.top_logprob[row * a.k + tid] = empty ? -INFINITY : (key_value(key) - r.m) - log_s;
  }
}

// ------------------------------------------------------------------ gradient
constexpr int kGradThreads = 256, kGradUnits = 4;
template <typename T>
__global__ void __launch_bounds__(kGradThreads)
token_logprob_grad_kernel(LogprobGradArgs a, uint32_t per_row, unsigned int* __restrict__ status) {
  const uint64_t row = blockIdx.x / per_row;
  const uint32_t part = blockIdx.x - static_cast<uint32_t>(row) * per_row, vocab = a.vocab;
  chain_wait();
  chain_trigger();
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  T* dx = static_cast<T*>(a.dlogits) + row * a.ld_d;
  int64_t token = a.tokens ? a.tokens[row] : -1;
  const bool skip = a.tokens && (token < 0 || token >= vocab);
  if (skip && token >= 0 && part == 0 && threadIdx.x == 0) atomicOr(status, kFlagBadIndex);
  const float lse = a.lse[row], g_lp = a.g_logprob && a.tokens ? a.g_logprob[row] : 0.f;
  const float g_h = a.g_entropy ? a.g_entropy[row] : 0.f, g_lse = a.g_lse ? a.g_lse[row] : 0.f;
  const bool zero = skip || lse == -INFINITY;  // a padding row, or one whose logits are all -inf
  // p (c0 - c1 y) with y = log2 p
  const float c0 = g_lse - g_lp - (a.g_entropy ? g_h * a.entropy[row] : 0.f), c1 = g_h * kLn2;
  const uint32_t off = static_cast<uint32_t>((reinterpret_cast<uintptr_t>(dx) & 15u) / sizeof(T));
  const uint32_t u0 = part * (kGradThreads * kGradUnits) + threadIdx.x;
  float v[kGradUnits][kUnit];
  if (!zero) {
#pragma unroll
    for (int j = 0; j < kGradUnits; ++j)
      load_values<T>(x, static_cast<int64_t>(u0 + j * kGradThreads) * kUnit - off, vocab, -INFINITY, v[j]);
  }
#pragma unroll
  for (int j = 0; j < kGradUnits; ++j) {
    const int64_t c = static_cast<int64_t>(u0 + j * kGradThreads) * kUnit - off;
#pragma unroll
    for (int k = 0; k < kUnit; ++k) {
      if (zero) {
        v[j][k] = 0.f;
      } else {
        const float y = max_nan((v[j][k] - lse) * kLog2e, kTiny);
        v[j][k] = exp2_fast(y) * fmaf(-c1, y, c0);
        if (c + k == token) v[j][k] += g_lp;
      }
    }
    store_values<T>(dx, c, vocab, v[j]);
  }
}

// ------------------------------------------------------------------ launchers
constexpr int kWide = 256, kNarrow = 128;
int launch_token_logprob(int dtype, const LogprobArgs& a, unsigned int* status, const LaunchShape& shape,
                         cudaStream_t stream) {
  // Rows are split over a cluster until there are about two CTAs for every SM, as long as a CTA keeps a round.
  const bool narrow = a.vocab <= 4096;
  uint32_t cluster = 1;
  if (!narrow)
    while (cluster < kMaxCluster && a.rows * cluster < static_cast<uint64_t>(shape.sm_count) && a.vocab / cluster > 16384) cluster *= 2;
  with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const dim3 grid(static_cast<unsigned>(a.rows * cluster));
    auto go = [&](auto kernel, unsigned threads) { launch_lm(kernel, grid, threads, 0, cluster, stream, shape.chained, a, cluster, status); };
    if (narrow) a.k ? go(token_logprob_kernel<T, kNarrow, true>, kNarrow) : go(token_logprob_kernel<T, kNarrow, false>, kNarrow);
    else a.k ? go(token_logprob_kernel<T, kWide, true>, kWide) : go(token_logprob_kernel<T, kWide, false>, kWide);
  });
  return 1;
}

int launch_token_logprob_grad(int dtype, const LogprobGradArgs& a, unsigned int* status, const LaunchShape& shape,
                              cudaStream_t stream) {
  // one unit more than the row's: it may begin inside a 16-byte group
  const uint32_t per_row = (a.vocab / kUnit + 2 + kGradThreads * kGradUnits - 1) / (kGradThreads * kGradUnits);
  with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    launch_lm(token_logprob_grad_kernel<T>, dim3(static_cast<unsigned>(a.rows * per_row)), kGradThreads, 0, 1, stream,
              shape.chained, a, per_row, status);
  });
  return 1;
}

}  // namespace qasg
