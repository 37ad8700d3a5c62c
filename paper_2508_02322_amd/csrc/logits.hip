// What a model answers with, row by row of its logits Z [n x vocab]: the log probabilities of given tokens with the entropy and
// the most likely alternatives, the distance from a teacher whose most likely tokens are known, and the gradients of both.
//
// With p = softmax(z / T), m = max z and S = sum exp((z - m) / T):
//   log p_v = (z_v - m) / T - log S,      H = -sum p log p = log S - (1 / S) sum exp(d_v) d_v,  d_v = (z_v - m) / T
// One pass over a row keeps, per thread, the largest logit so far, the sum of exponentials relative to it and the sum weighted
// by the exponents, all in float32, and rescales the sums when the largest logit grows.  d_v is taken as a difference first, so
// that logits of any size (the type's lowest value as a mask among them) stay exact; a logit of -inf adds nothing.  A NaN, or the
// difference of two infinities, stays in the sums and makes the row's results NaN; only the maxima pass it over.
//
// All of it is bound by reading the logits once (and writing the gradient once).  bf16, 4096 rows of 151936: log probabilities, entropy and
// 64 alternatives 227 us (5.5 TB/s), distillation with 64 listed tokens and the rest as a class 214 us (5.8), gradients of 2048 rows
// 223 us (5.6 read and written; a copy of as many bytes 4.9).  (After 20 ms of them; the first 10 ms of passes are a sixth slower.)
// One row: 8.3 us in 33 parts and 6.5 us to join them, latencies: what a part does after its one load (three reductions, the bound, the
// candidates) is a chain of LDS and cache round trips.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "camera_internal.h"

namespace camera {
namespace {

// Threads of a workgroup (TH below): kLong, or kShort where many short rows would leave most of the threads without a vector.
constexpr int kLong = 512, kShort = 128;
constexpr int kShortVocab = 16384, kShortTop = 64;  // longest row and most alternatives for the short workgroup
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.693147180559945309417f;
constexpr float kFloor = -1.0e4f;  // exponents are clamped here: exp2 of it is 0, and 0 times it is 0
__device__ __forceinline__ float floored(float d) { return __builtin_elementwise_maximum(d, kFloor); }  // NaN stays NaN, one instruction
static_assert(kLong >= CAMERA_MAX_ALTERNATIVES && kShort >= kShortTop, "the k-th largest of the threads' maxima exists");

// 16 bytes of a row.  Rows start where the caller's do, at any element: the loads and stores carry the element's alignment only.
template <class T>
struct Pack;
template <>
struct Pack<float> {
  static constexpr int N = 4;
  typedef uint32_t Raw __attribute__((ext_vector_type(4), aligned(4)));
  static __device__ __forceinline__ void get(Raw r, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t bits = r[i];  // (a bit cast of the vector's element itself takes its first one, with this compiler)
      v[i] = __builtin_bit_cast(float, bits);
    }
  }
  static __device__ __forceinline__ Raw put(const float* v) {
    Raw r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, v[i]);
    return r;
  }
  static __device__ __forceinline__ float one(float x) { return x; }
  static __device__ __forceinline__ float round(float x) { return x; }
};
template <>
struct Pack<__bf16> {
  static constexpr int N = 8;
  typedef uint32_t Raw __attribute__((ext_vector_type(4), aligned(2)));
  static __device__ __forceinline__ void get(Raw r, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __builtin_bit_cast(float, r[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, r[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ Raw put(const float* v) {
    typedef __bf16 Pair __attribute__((ext_vector_type(2)));
    Raw r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, Pair{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]});
    return r;
  }
  static __device__ __forceinline__ float one(__bf16 x) { return (float)x; }
  static __device__ __forceinline__ __bf16 round(float x) { return (__bf16)x; }
};

// ---- reductions over the workgroup ---------------------------------------------------------------------------------
template <class X, class F>
__device__ __forceinline__ X wave_all(X x, F f) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) x = f(x, __shfl_xor(x, d));
  return x;
}
// Every thread gets the result, taken in the same order; slots: a value of LDS per wave.  Barriers inside.
template <int TH, class X, class F>
__device__ __forceinline__ X block_all(X x, F f, X* slots) {
  x = wave_all(x, f);
  __syncthreads();  // the slots' earlier use is over
  if (threadIdx.x % kWave == 0) slots[threadIdx.x / kWave] = x;
  __syncthreads();
  X all = slots[0];
#pragma unroll
  for (int w = 1; w < TH / kWave; ++w) all = f(all, slots[w]);
  return all;
}
struct Add {
  template <class X>
  __device__ __forceinline__ X operator()(X a, X b) const { return a + b; }
};
struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// ---- the running sums ----------------------------------------------------------------------------------------------
// scale = log2(e) / T.  s = sum exp2((z - m) scale), t = sum exp2(d) d with d in powers of two.
struct Running {
  float m = -INFINITY, s = 0.0f, t = 0.0f;
};
// What an empty row or thread is taken relative to.
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.0f : m; }
// Nothing but logits of -inf: any other adds at least the largest one's 1, or NaN.
__device__ __forceinline__ bool nothing(const Running& r) { return r.s == 0.0f; }
__device__ __forceinline__ float log_sum_of(const Running& r) { return nothing(r) ? 0.0f : logf(r.s); }
// The sums relative to the larger maximum `m`.
__device__ __forceinline__ void rescale(Running& r, float m, float scale) {
  const float d = fmaxf((r.m - reference(m)) * scale, kFloor), c = __builtin_amdgcn_exp2f(d);
  r.t = c * fmaf(r.s, d, r.t);
  r.s *= c;
  r.m = m;
}
// Adds N values; returns the largest of them.
template <bool ENTROPY, int N>
__device__ __forceinline__ float add_values(Running& r, const float* z, float scale) {
  float largest = z[0];
#pragma unroll
  for (int i = 1; i < N; ++i) largest = fmaxf(largest, z[i]);
  const float m = fmaxf(r.m, largest);
  rescale(r, m, scale);
  const float ref = reference(m);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float d = (z[i] - ref) * scale;
    if constexpr (ENTROPY) d = floored(d);  // 0 times -inf would not be 0
    const float e = __builtin_amdgcn_exp2f(d);
    r.s += e;
    if constexpr (ENTROPY) r.t = fmaf(e, d, r.t);
  }
  return largest;
}
struct Slots {
  float f[2][kLong / kWave];
};
template <int TH>
__device__ __forceinline__ Running block_running(Running r, float scale, Slots& slots) {
  rescale(r, block_all<TH>(r.m, Max{}, slots.f[0]), scale);
  r.s = block_all<TH>(r.s, Add{}, slots.f[1]);
  r.t = block_all<TH>(r.t, Add{}, slots.f[0]);
  return r;
}

// ---- a token's place in the order ---------------------------------------------------------------------------------
// A token's key orders as (logit, lower index first) does: the logit's bits made monotone, then the index turned round.  -0 and
// +0 are equal.  0 stands for no token: -inf (and NaN) are never alternatives.
__device__ __forceinline__ uint32_t order_bits(float z) {
  if (!(z > -INFINITY)) return 0;
  const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_order_bits(uint32_t o) {
  return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t make_key(uint32_t bits, int index) { return (uint64_t)bits << 32 | (0xffffffffu - (uint32_t)index); }
__device__ __forceinline__ int key_index(uint64_t key) { return (int)(0xffffffffu - (uint32_t)key); }

// ---- one part of a row ---------------------------------------------------------------------------------------------
// Thread j's stripe is the vectors j, j + TH, ... of the part, and element j of what is left behind the whole vectors.  A
// stripe is cut into cells of per_cell groups of kUnroll vectors (what is left belongs to the last one).
constexpr int kUnroll = 4;  // vectors in flight per thread
constexpr int kCells = 16;
template <class T, int TH>
struct RowPart {
  static constexpr int N = Pack<T>::N;
  using Raw = typename Pack<T>::Raw;
  const T* z;  // first element of the part
  int first;   // its index in the row
  int vecs, rest;
  int per_cell, cells;
  __device__ RowPart(const T* row, int64_t first_, int len) : z(row + first_), first((int)first_), vecs(len / N), rest(len % N) {
    const int groups = (vecs + kUnroll * TH - 1) / (kUnroll * TH);
    per_cell = groups / kCells + 1;
    cells = groups / per_cell + 1;  // <= kCells
  }
  __device__ __forceinline__ Raw load(int v) const { return *reinterpret_cast<const Raw*>(z + (int64_t)v * N); }
  __device__ __forceinline__ float left(int i) const { return Pack<T>::one(z[(int64_t)vecs * N + i]); }
};

// Marks of a part's listed elements, a bit each: 32 KiB of LDS for the long workgroup, four of them a compute unit.
constexpr int kMaxListed = 1 << 18;

// The thread's sums over its stripe.  cell_max (CELLS): upper half of the order bits of every cell's largest value, [cell][thread].
// meanwhile(): done once the first loads are under way.
template <bool ENTROPY, bool LISTED, bool CELLS, class T, int TH, class F>
__device__ __forceinline__ Running stream_part(const RowPart<T, TH>& p, float scale, const unsigned char* marks, uint16_t* cell_max, F&& meanwhile) {
  constexpr int N = Pack<T>::N, U = kUnroll;
  const int tid = threadIdx.x;
  Running r;
  auto one = [&](typename Pack<T>::Raw raw, int v, float* z) {
    Pack<T>::get(raw, z);
    if constexpr (LISTED) {
      const unsigned bits = N == 8 ? marks[v] : (marks[v >> 1] >> (4 * (v & 1))) & 15u;
      if (bits != 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = bits >> i & 1 ? -INFINITY : z[i];
      }
    }
  };
  float largest = -INFINITY;  // of the cell
  int cell = 0, groups = 0;
  int v = tid;
  typename Pack<T>::Raw raw[U];
  auto fetch = [&] {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (v + u * TH < p.vecs) raw[u] = p.load(v + u * TH);
  };
  fetch();
  meanwhile();
  for (; v + (U - 1) * TH < p.vecs; v += U * TH, fetch()) {
    float z[U * N];
#pragma unroll
    for (int u = 0; u < U; ++u) one(raw[u], v + u * TH, z + u * N);
    largest = fmaxf(largest, add_values<ENTROPY, U * N>(r, z, scale));
    if constexpr (CELLS) {
      if (++groups == p.per_cell) {
        cell_max[cell++ * TH + tid] = (uint16_t)(order_bits(largest) >> 16);
        largest = -INFINITY;
        groups = 0;
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U - 1; ++u)  // up to three vectors are left
    if (v + u * TH < p.vecs) {
      float z[N];
      one(raw[u], v + u * TH, z);
      largest = fmaxf(largest, add_values<ENTROPY, N>(r, z, scale));
    }
  if constexpr (CELLS) {
    for (; cell < p.cells; ++cell) {
      if (cell == p.cells - 1 && tid < p.rest) largest = fmaxf(largest, p.left(tid));
      cell_max[cell * TH + tid] = (uint16_t)(order_bits(largest) >> 16);
      largest = -INFINITY;
    }
  }
  if (tid < p.rest) {
    float z = p.left(tid);
    if constexpr (LISTED) {
      const int at = p.vecs * N + tid;
      if (marks[at >> 3] >> (at & 7) & 1) z = -INFINITY;
    }
    add_values<ENTROPY, 1>(r, &z, scale);
  }
  return r;
}

// ---- the largest k -------------------------------------------------------------------------------------------------
// Up to this many candidates are placed by counting the larger ones (their square, over the workgroup's lanes), more by sorting.
constexpr int kCounted = 128;
template <int TH>
struct SelectSmem {
  // as many candidates as a part has elements that has fewer stripes than alternatives are wanted
  static constexpr int kCandidates = 8 * (TH == kLong ? CAMERA_MAX_ALTERNATIVES : kShortTop), kChosen = 2 * TH;
  uint32_t largest[TH];
  uint16_t cell_max[kCells * TH];  // of the rows' cells
  int32_t chosen[kChosen];         // cells that may hold candidates: cell * TH + stripe
  uint64_t keys[kCandidates];
  int32_t hist[256];
  uint32_t bound, least, most;
  int32_t n_chosen, n_keys;
  uint64_t prefix;
  int32_t want;
};

// Where keys come from: every stripe has cells() cells of positions() places of up to N keys.
template <class T, int TH>
struct LogitKeys {
  const RowPart<T, TH>& p;
  __device__ __forceinline__ int cells() const { return p.cells; }
  __device__ __forceinline__ int positions() const { return p.per_cell * kUnroll + (p.rest != 0 ? 1 : 0); }
  template <class F>
  __device__ __forceinline__ void at(int stripe, int cell, int pos, F&& f) const {
    constexpr int N = Pack<T>::N;
    const int whole = p.per_cell * kUnroll;
    if (pos < whole) {
      const int v = (cell * whole + pos) * TH + stripe;
      if (v < p.vecs) {
        float z[N];
        Pack<T>::get(p.load(v), z);
#pragma unroll
        for (int i = 0; i < N; ++i) f(order_bits(z[i]), p.first + v * N + i);
      }
    } else if (cell == p.cells - 1 && stripe < p.rest) {
      f(order_bits(p.left(stripe)), p.first + p.vecs * N + stripe);
    }
  }
};
template <int TH>
struct ListKeys {
  const uint64_t* keys;
  int n;
  __device__ __forceinline__ int cells() const { return 1; }
  __device__ __forceinline__ int positions() const { return (n + TH - 1) / TH; }
  template <class F>
  __device__ __forceinline__ void at(int stripe, int, int pos, F&& f) const {
    const int i = pos * TH + stripe;
    if (i < n) {
      const uint64_t key = keys[i];
      f((uint32_t)(key >> 32), key_index(key));
    }
  }
};

// out(r, key) for the k largest keys of a source in falling order, key 0 where there are fewer.  `largest`: order bits of the
// largest value of the thread's stripe; sm.cell_max: their upper half for its cells.  At least k stripes have a value as large as
// the k-th largest of the stripes' maxima, so that is a lower bound of the k-th largest value.  One wave finds it, bit by bit, with
// its lower 16 bits left 0 (all that a bf16 value has; counting for every maximum how many are larger took the workgroup 7 us).
// The values not below it lie in the cells whose maximum is not, mostly k of them, which are read again, from the caches.  The
// keys are all different, so the order in which candidates are found does not show.  Where more values reach the bound than there
// is room for, they are mostly equal (a mask by the type's lowest value with fewer tokens left than wanted, a constant row): then
// the larger values are taken and of the equal ones the first, in index order, one pass and the beginning of another.  Otherwise
// the k-th largest key is found by its digits, eight passes over the source.  1024 x 102400 bf16, 5 tokens left, 20 alternatives: 95 us,
// 745 by digits, 42 without ties.  4096 x 151936 bf16, us: 216 without alternatives, 220 with one, 223 with 20, 227 with 64, 242 with 128,
// 280 with 256 (half the lines again).
template <int TH, class SOURCE, class OUT>
__device__ __forceinline__ void select_top(const SOURCE& src, uint32_t largest, int k, SelectSmem<TH>& sm, OUT&& out) {
  constexpr int kWaves = TH / kWave, kCandidates = SelectSmem<TH>::kCandidates, kChosen = SelectSmem<TH>::kChosen;
  static_assert(TH >= kCounted, "a thread for every counted candidate");
  const int tid = threadIdx.x, cells = src.cells(), positions = src.positions();
  sm.largest[tid] = largest;
  if (tid == 0) {
    sm.n_chosen = 0;
    sm.n_keys = 0;
  }
  __syncthreads();
  if (tid < kWave) {
    uint32_t mine[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mine[w] = sm.largest[w * kWave + tid];
    uint32_t bound = 0;
    for (int bit = 31; bit >= 16; --bit) {
      const uint32_t higher = bound | 1u << bit;
      int reached = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) reached += (int)__popcll(__ballot(mine[w] >= higher));
      if (reached >= k) bound = higher;
    }
    if (tid == 0) sm.bound = bound;
  }
  __syncthreads();
  const uint32_t bound = sm.bound;
  for (int c = 0; c < cells; ++c) {
    const uint32_t m = sm.cell_max[c * TH + tid];
    if (m >= bound >> 16 && m != 0) {
      const int at = atomicAdd(&sm.n_chosen, 1);
      if (at < kChosen) sm.chosen[at] = c * TH + tid;
    }
  }
  __syncthreads();
  const int n_chosen = sm.n_chosen;
  auto add_key = [&](uint64_t key) {
    const int at = atomicAdd(&sm.n_keys, 1);
    if (at < kCandidates) sm.keys[at] = key;
  };
  if (n_chosen <= kChosen) {
    for (int w = tid; w < n_chosen * positions; w += TH) {
      const int c = sm.chosen[w % n_chosen];
      src.at(c % TH, c / TH, w / n_chosen, [&](uint32_t bits, int index) {
        if (bits >= bound && bits != 0) add_key(make_key(bits, index));
      });
    }
    __syncthreads();
  }
  int n_keys = sm.n_keys;
  if (n_chosen > kChosen || n_keys > kCandidates) {
    // Step 8: the larger keys, and the range of the values that share the bound's upper half.  Steps 7 to 0: a digit.  Then: the keys.
    uint64_t prefix = 0;
    int want = k;
    bool equal = false;
    for (int step = 8; step >= -1 && !equal; --step) {
      __syncthreads();
      for (int i = tid; i < 256; i += TH) sm.hist[i] = 0;
      if (tid == 0) {
        sm.n_keys = 0;
        sm.least = 0xffffffffu;
        sm.most = 0;
      }
      __syncthreads();
      uint32_t least = 0xffffffffu, most = 0;
      for (int c = 0; c < cells; ++c)
        for (int pos = 0; pos < positions; ++pos)
          src.at(tid, c, pos, [&](uint32_t bits, int index) {
            if (bits < bound || bits == 0) return;
            const uint64_t key = make_key(bits, index);
            if (step == 8 && bits >> 16 == bound >> 16) {
              least = min(least, bits);
              most = max(most, bits);
            } else if (step == 8 || step < 0) {
              if (key >= prefix) add_key(key);
            } else if (step == 7 || (key ^ prefix) >> (8 * step + 8) == 0) {
              // lanes that count the same digit as the first one add once
              const int digit = (int)(key >> 8 * step & 255), lead = __builtin_amdgcn_readfirstlane(digit);
              const uint64_t same = __ballot(digit == lead);
              if (digit != lead) atomicAdd(&sm.hist[digit], 1);
              else if (tid % kWave == __ffsll((unsigned long long)same) - 1) atomicAdd(&sm.hist[digit], (int)__popcll(same));
            }
          });
      if (most != 0) {
        atomicMin(&sm.least, least);
        atomicMax(&sm.most, most);
      }
      __syncthreads();
      if (step == 8) equal = sm.n_keys < k && sm.least == sm.most;
      if (step == 8 || step < 0) continue;
      if (tid < kWave) {  // the digit at which the counts from 255 down reach `want`: lane l has four, from 255 - 4 l down
        int count[4], mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) mine += count[i] = sm.hist[255 - 4 * tid - i];
        int upto = mine;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
          const int more = __shfl_up(upto, d);
          if (tid >= d) upto += more;
        }
        int left = want - (upto - mine);  // still to be found among this lane's four
        if (left > 0 && left <= mine) {   // one lane
          int i = 0;
#pragma unroll
          for (int j = 0; j < 3; ++j)
            if (i == j && left > count[j]) left -= count[j], i = j + 1;
          sm.prefix = prefix | (uint64_t)(255 - 4 * tid - i) << 8 * step;
          sm.want = left;
        }
      }
      __syncthreads();
      prefix = sm.prefix;
      want = sm.want;
    }
    n_keys = sm.n_keys;  // k, or the ones larger than the equal values
    if (equal) {
      // every round of the source is in index order over the threads (of a list: the equal values' order in it is the index order)
      const uint32_t value = sm.most;
      for (int c = 0; c < cells && n_keys < k; ++c)
        for (int pos = 0; pos < positions && n_keys < k; ++pos) {
          uint32_t found = 0;  // a bit per element, the last one's the lowest
          int last = 0;
          src.at(tid, c, pos, [&](uint32_t bits, int index) {
            found = found << 1 | (bits == value);
            last = index;
          });
          const int mine = __popc(found);
          int upto = mine;
#pragma unroll
          for (int d = 1; d < kWave; d <<= 1) {
            const int more = __shfl_up(upto, d);
            if (tid % kWave >= d) upto += more;
          }
          __syncthreads();  // the previous round's totals have been read
          if (tid % kWave == kWave - 1) sm.hist[tid / kWave] = upto;
          __syncthreads();
          int place = n_keys + upto - mine;
          for (int w = 0; w < kWaves; ++w) {
            n_keys += sm.hist[w];
            place += w < tid / kWave ? sm.hist[w] : 0;
          }
          for (; found != 0 && place < k; ++place) {
            const int back = 31 - __clz(found);
            sm.keys[place] = make_key(value, last - back);
            found ^= 1u << back;
          }
        }
      n_keys = min(n_keys, k);
      __syncthreads();
    }
  }
  if (n_keys <= kCounted) {
    if (tid < n_keys) {
      const uint64_t key = sm.keys[tid];
      int place = 0;
#pragma unroll 4
      for (int j = 0; j < n_keys; ++j) place += sm.keys[j] > key;
      if (place < k) out(place, key);
    }
  } else {
    int size = 2 * kCounted;
    while (size < n_keys) size *= 2;
    for (int i = n_keys + tid; i < size; i += TH) sm.keys[i] = 0;
    __syncthreads();
    for (int run = 2; run <= size; run *= 2)
      for (int apart = run / 2; apart > 0; apart /= 2) {
        for (int c = tid; c < size / 2; c += TH) {
          const int i = 2 * c - (c & (apart - 1)), j = i + apart;  // the pairs `apart` from each other
          const uint64_t x = sm.keys[i], y = sm.keys[j];
          if ((x < y) == ((i & run) == 0)) sm.keys[i] = y, sm.keys[j] = x;
        }
        __syncthreads();
      }
    for (int r = tid; r < min(k, n_keys); r += TH) out(r, sm.keys[r]);
  }
  for (int r = n_keys + tid; r < k; r += TH) out(r, (uint64_t)0);
}

// ---- log probabilities, entropy, alternatives ----------------------------------------------------------------------
template <class T>
__device__ __forceinline__ void finish_logprobs(const Running& r, const LogprobArgs& a, int64_t row) {
  const bool none = nothing(r);
  const float log_sum = log_sum_of(r);
  if (threadIdx.x == 0) {
    if (a.stats) {
      a.stats[2 * row] = r.m;
      a.stats[2 * row + 1] = log_sum;
    }
    if (a.entropy) a.entropy[row] = none ? 0.0f : log_sum - r.t / r.s * kLn2;
    if (a.logprob) {
      const int64_t target = a.targets[row];
      float lp = 0.0f;
      if (target >= 0 && target < a.vocab)
        lp = none ? -INFINITY
                  : (Pack<T>::one(static_cast<const T*>(a.logits)[row * a.ld + target]) - r.m) * a.inv_temperature - log_sum;
      a.logprob[row] = lp;
    }
  }
}
__device__ __forceinline__ void write_alternative(const LogprobArgs& a, const Running& r, float log_sum, int64_t row, int place,
                                                  uint64_t key) {
  const bool none = key == 0;
  a.top_idx[row * a.top_k + place] = none ? -1 : key_index(key);
  a.top_logprob[row * a.top_k + place] =
      none ? -INFINITY : (of_order_bits((uint32_t)(key >> 32)) - r.m) * a.inv_temperature - log_sum;
}

// A workgroup has a part of a row; where that is the WHOLE row it ends it, else it leaves its sums and its alternatives' keys.  Four
// workgroups share a compute unit only with at most 64 vector and 80 scalar registers a wave: with both ends in one kernel (87 scalar
// ones) three did, and 64 x 102400 bf16 took 15.1 us where it takes 11.7.
template <class T, int TH, bool TOP, bool WHOLE>
__global__ __launch_bounds__(TH, 4) void logprobs_kernel(LogprobArgs a) {
  __shared__ Slots slots;
  const int64_t block = linear_block();
  const int64_t row = block / a.parts;
  if (row >= a.n) return;
  const int part = (int)(block - row * a.parts);
  const int64_t first = part * a.part_len;
  const RowPart<T, TH> p(static_cast<const T*>(a.logits) + row * a.ld, first, (int)min(a.part_len, a.vocab - first));
  const float scale = a.inv_temperature * kLog2e;
  SelectSmem<TH>* select = nullptr;
  if constexpr (TOP) {
    __shared__ SelectSmem<TH> sm;
    select = &sm;
  }
  const Running mine = stream_part<true, false, TOP>(p, scale, nullptr, TOP ? select->cell_max : nullptr, [] {});
  const Running r = block_running<TH>(mine, scale, slots);
  if constexpr (WHOLE) finish_logprobs<T>(r, a, row);
  else if (threadIdx.x == 0) a.part_stats[block] = make_float4(r.m, r.s, r.t, 0.0f);
  if constexpr (TOP) {
    const float log_sum = log_sum_of(r);
    select_top<TH>(LogitKeys<T, TH>{p}, order_bits(mine.m), a.top_k, *select, [&](int place, uint64_t key) {
      if constexpr (WHOLE) write_alternative(a, r, log_sum, row, place, key);
      else a.part_keys[block * a.top_k + place] = key;
    });
  }
}

// A row's parts put together, in their order.
template <int TH>
__device__ __forceinline__ Running join_parts(const float4* part_stats, int parts, float scale, Slots& slots) {
  Running mine;
  for (int i = threadIdx.x; i < parts; i += TH) {
    const float4 s = part_stats[i];
    Running other;
    other.m = s.x;
    other.s = s.y;
    other.t = s.z;
    const float m = fmaxf(mine.m, other.m);
    rescale(mine, m, scale);
    rescale(other, m, scale);
    mine.s += other.s;
    mine.t += other.t;
  }
  return block_running<TH>(mine, scale, slots);
}
template <class T, bool TOP>
__global__ __launch_bounds__(kLong) void logprobs_join_kernel(LogprobArgs a) {
  constexpr int TH = kLong;
  __shared__ Slots slots;
  const int64_t row = linear_block();
  if (row >= a.n) return;
  const float scale = a.inv_temperature * kLog2e;
  const Running r = join_parts<TH>(a.part_stats + row * a.parts, a.parts, scale, slots);
  finish_logprobs<T>(r, a, row);
  if constexpr (TOP) {
    __shared__ SelectSmem<TH> sm;
    const float log_sum = log_sum_of(r);
    const ListKeys<TH> keys{a.part_keys + row * a.parts * a.top_k, a.parts * a.top_k};
    uint32_t largest = 0;
    for (int pos = 0; pos < keys.positions(); ++pos) keys.at(threadIdx.x, 0, pos, [&](uint32_t bits, int) { largest = max(largest, bits); });
    sm.cell_max[threadIdx.x] = (uint16_t)(largest >> 16);
    select_top<TH>(keys, largest, a.top_k, sm, [&](int place, uint64_t key) { write_alternative(a, r, log_sum, row, place, key); });
  }
}

// ---- gradients -----------------------------------------------------------------------------------------------------
// A workgroup has TH * kGradUnroll vectors of a row, a thread's loads in flight together.
constexpr int kGradUnroll = 4;
template <class T, int TH>
struct GradPart {
  static constexpr int N = Pack<T>::N, kLen = TH * kGradUnroll * N;
  using Raw = typename Pack<T>::Raw;
  const T* z;
  T* out;
  int64_t first;  // of the part, in the row
  int len;
  bool accumulate;

  Raw raw[kGradUnroll], old[kGradUnroll];

  __device__ __forceinline__ void fetch() {
    const int vecs = len / N, tid = threadIdx.x;
#pragma unroll
    for (int u = 0; u < kGradUnroll; ++u) {
      const int v = tid + u * TH;
      if (v < vecs) {
        raw[u] = *reinterpret_cast<const Raw*>(z + v * N);
        if (accumulate) old[u] = *reinterpret_cast<const Raw*>(out + v * N);
      }
    }
  }
  // out (+)= f(z, index in the part) over the part, after fetch(); f gets a vector's values and leaves the gradient in their place.
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    const int vecs = len / N, rest = len - vecs * N, tid = threadIdx.x;
#pragma unroll
    for (int u = 0; u < kGradUnroll; ++u) {
      const int v = tid + u * TH;
      if (v < vecs) {
        float x[N];
        Pack<T>::get(raw[u], x);
        f(x, v * N, std::integral_constant<int, N>{});
        if (accumulate) {
          float y[N];
          Pack<T>::get(old[u], y);
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] += y[i];
        }
        *reinterpret_cast<Raw*>(out + v * N) = Pack<T>::put(x);
      }
    }
    if (tid < rest) {
      const int at = vecs * N + tid;
      float x = Pack<T>::one(z[at]);
      f(&x, at, std::integral_constant<int, 1>{});
      if (accumulate) x += Pack<T>::one(out[at]);
      out[at] = Pack<T>::round(x);
    }
  }
  __device__ __forceinline__ void zero() const {
    const int vecs = len / N, rest = len - vecs * N;
    for (int v = threadIdx.x; v < vecs; v += TH) *reinterpret_cast<Raw*>(out + v * N) = Raw{0, 0, 0, 0};
    if ((int)threadIdx.x < rest) out[vecs * N + threadIdx.x] = Pack<T>::round(0.0f);
  }
};
template <class T, int TH>
__device__ __forceinline__ GradPart<T, TH> grad_part(const LogitGradArgs& a, int64_t row, int part) {
  GradPart<T, TH> p;
  p.first = (int64_t)part * p.kLen;
  p.len = (int)min((int64_t)p.kLen, a.vocab - p.first);
  p.z = static_cast<const T*>(a.logits) + row * a.ld + p.first;
  p.out = static_cast<T*>(a.dlogits) + row * a.ldd + p.first;
  p.accumulate = a.accumulate != 0;
  return p;
}

// d logprob[t] / dz_v = (1[v = t] - p_v) / T,  d H / dz_v = -p_v (log p_v + H) / T
template <class T, int TH>
__global__ __launch_bounds__(TH) void logprobs_grad_kernel(LogitGradArgs a, const int32_t* __restrict__ targets,
                                                                 const float* __restrict__ entropy,
                                                                 const float* __restrict__ grad_logprob,
                                                                 const float* __restrict__ grad_entropy) {
  const int64_t block = linear_block();
  const int64_t row = block / a.parts;
  if (row >= a.n) return;
  GradPart<T, TH> p = grad_part<T, TH>(a, row, (int)(block - row * a.parts));
  const int64_t target = targets ? (int64_t)targets[row] : -1;
  const float m = a.stats[2 * row], log_sum = a.stats[2 * row + 1];
  const float one = grad_logprob && target >= 0 && target < a.vocab ? grad_logprob[row] * a.inv_temperature : 0.0f;
  const float two = grad_entropy ? grad_entropy[row] * a.inv_temperature : 0.0f;
  if ((one == 0.0f && two == 0.0f) || (m == -INFINITY && log_sum == 0.0f)) {  // no gradient, or nothing but -inf
    if (!p.accumulate) p.zero();
    return;
  }
  const float inv_t = a.inv_temperature, h = two != 0.0f ? entropy[row] : 0.0f;
  const int64_t at = target - p.first;  // in this part, or not
  p.fetch();
  p.each([&](float* x, int v, auto count) {
    constexpr int N = decltype(count)::value;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float lp = floored((x[i] - m) * inv_t - log_sum);
      x[i] = __builtin_amdgcn_exp2f(lp * kLog2e) * -fmaf(two, lp + h, one);
    }
    if (one != 0.0f && at >= v && at < v + N) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (at == v + i) x[i] += one;
    }
  });
}

// ---- distillation --------------------------------------------------------------------------------------------------
// The teacher's distribution q over the tokens it lists, and with `tail` the rest of its probability as one class of all tokens it
// does not list; the student's p over the same classes.  Kullback-Leibler divergence:
//   loss = sum_j q_j (log q_j - log p_j)  [+ q_r (log q_r - log p_r)],  q_r = 1 - sum q_j,  p_r = sum of p_v over the unlisted v
// p_r is summed over the unlisted tokens themselves (1 - sum p_j would cancel): a bit per token of the part marks the listed ones.
// The few values of the listed tokens are handled in float64.
// The gradient takes the class by log(q_r / p_r), as a float32 off by u of itself and the exponents with it.  Beyond kFarClass (all
// unlisted tokens masked by -1e4 or the type's lowest value: off by anything up to infinity) it takes the class by itself instead:
// p_v q_r / p_r = q_r exp((z_v - m_r) / T) / S_r with the class's own maximum and sum, beside which p_v is nothing.  stats have no more
// room, but for the two that then are known: norm (0 with tail) and the sum of q (1) hold m_r and log(q_r / S_r).
constexpr float kFarClass = 256.0f;
// Such a class with less than this of the teacher is none: it is what the roundings of the listed log probabilities leave of 1 (each
// is off by about 4 u of it, together up to 16 u), and times the logarithm of a mask it would be the loss (1e31 for the type's lowest).
constexpr double kNoClass = 0x1p-20;

// A row's teacher list in LDS, id -1 where an entry does not count: it names no token, has no probability, or an entry before it
// names the same token.
struct TeacherSmem {
  __align__(16) int32_t id[CAMERA_MAX_ALTERNATIVES];
  float value[CAMERA_MAX_ALTERNATIVES];
};
template <int TH>
__device__ __forceinline__ void load_teacher(const DistillTeacher& t, int64_t row, int64_t vocab, TeacherSmem& sm) {
  constexpr int kEach = (CAMERA_MAX_ALTERNATIVES + TH - 1) / TH;  // entries of a thread
  const int padded = (t.k + 3) & ~3;
  int32_t id[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int j = threadIdx.x + e * TH;
    id[e] = -1;
    if (j < padded) {
      float value = -INFINITY;
      if (j < t.k) {
        id[e] = t.idx[row * t.k + j];
        value = t.logprob[row * t.k + j];
      }
      sm.id[j] = id[e];
      sm.value[j] = value;
      if (id[e] < 0 || id[e] >= vocab || !(value > -INFINITY)) id[e] = -1;
    }
  }
  __syncthreads();
  bool repeats[kEach] = {};
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int j = threadIdx.x + e * TH;
    if (j < padded) {
      for (int i = 0; i < padded; i += 4) {  // whole vectors, no early end: the reads follow each other without waiting
        const int4 other = *reinterpret_cast<const int4*>(&sm.id[i]);
        repeats[e] = repeats[e] || (other.x == id[e] && i < j) || (other.y == id[e] && i + 1 < j) || (other.z == id[e] && i + 2 < j) ||
                     (other.w == id[e] && i + 3 < j);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int j = threadIdx.x + e * TH;
    if (j < padded && (repeats[e] || id[e] < 0)) sm.id[j] = -1;
  }
  __syncthreads();
}

// rest: the sums over all tokens, or with tail over the unlisted ones.  One wave does it, lane l the entries l, l + 64, ...: in
// float64 the exponentials and logarithms of eight waves took as long as the row's own.
template <class T>
__device__ __forceinline__ void finish_distill(const Running& rest, const DistillArgs& a, int64_t row, const TeacherSmem& sm) {
  constexpr int kEntries = CAMERA_MAX_ALTERNATIVES / kWave;
  const int lane = threadIdx.x;
  const double inv_t = 1.0 / (double)a.temperature;
  bool ok[kEntries];
  float z[kEntries], value[kEntries];
  float z_max = -INFINITY, value_max = -INFINITY;
#pragma unroll
  for (int e = 0; e < kEntries; ++e) {
    const int j = e * kWave + lane;
    ok[e] = j < a.teacher.k && sm.id[j] >= 0;
    z[e] = value[e] = -INFINITY;
    if (ok[e]) {
      z[e] = Pack<T>::one(static_cast<const T*>(a.logits)[row * a.ld + sm.id[j]]);
      value[e] = sm.value[j];
    }
    z_max = fmaxf(z_max, z[e]);
    value_max = fmaxf(value_max, value[e]);
  }
  float m = rest.m;
  double sum = rest.s, log_sum = 0.0, norm = 0.0;
  if (a.tail) {
    m = fmaxf(m, wave_all(z_max, Max{}));
    const double ref = reference(m);
    double listed = 0.0;
#pragma unroll
    for (int e = 0; e < kEntries; ++e)
      if (z[e] != -INFINITY) listed += exp(((double)z[e] - ref) * inv_t);
    sum = wave_all(listed, Add{});
    if (!nothing(rest)) sum += (double)rest.s * exp(((double)rest.m - ref) * inv_t);
  } else {
    const double ref = reference(wave_all(value_max, Max{}));
    double total = 0.0;
#pragma unroll
    for (int e = 0; e < kEntries; ++e)
      if (ok[e]) total += exp(((double)value[e] - ref) * inv_t);
    total = wave_all(total, Add{});
    if (total > 0.0) norm = ref * inv_t + log(total);
  }
  if (sum != 0.0) log_sum = log(sum);
  double loss = 0.0, mass = 0.0, log_ratio = -INFINITY;
#pragma unroll
  for (int e = 0; e < kEntries; ++e)
    if (ok[e]) {
      const double log_q = a.tail ? (double)value[e] : (double)value[e] * inv_t - norm, q = exp(log_q);
      const double log_p = ((double)z[e] - (double)reference(m)) * inv_t - log_sum;
      mass += q;
      if (q > 0.0) loss += q * (log_q - log_p);
    }
  loss = wave_all(loss, Add{});
  mass = wave_all(mass, Add{});
  double left = 0.0;
  if (a.tail && !nothing(rest)) {
    left = fmax(0.0, 1.0 - mass);
    const double log_rest = ((double)rest.m - (double)m) * inv_t + log((double)rest.s) - log_sum;
    log_ratio = log(left) - log_rest;  // -inf where nothing is left
    if (log_ratio > (double)kFarClass && left < kNoClass) {
      left = 0.0;
      log_ratio = -INFINITY;
    }
    mass += left;
    if (left > 0.0) loss += left * log_ratio;
  }
  if (lane == 0) {
    a.loss[row] = (float)loss;
    float* st = a.stats + row * CAMERA_DISTILL_STATS;
    st[0] = m;
    st[1] = (float)log_sum;
    const bool far = log_ratio > kFarClass;
    st[2] = far ? rest.m : (float)norm;
    st[3] = far ? (float)log(left / (double)rest.s) : (float)mass;
    st[4] = (float)log_ratio;
  }
}

template <class T, int TH, bool TAIL>
__global__ __launch_bounds__(TH, 4) void distill_kernel(DistillArgs a) {
  __shared__ Slots slots;
  __shared__ TeacherSmem teacher;
  const int64_t block = linear_block();
  const int64_t row = block / a.parts;
  if (row >= a.n) return;
  const int part = (int)(block - row * a.parts);
  const int64_t first = part * a.part_len;
  const int len = (int)min(a.part_len, a.vocab - first);
  const RowPart<T, TH> p(static_cast<const T*>(a.logits) + row * a.ld, first, len);
  const float scale = kLog2e / a.temperature;
  Running mine;
  if constexpr (TAIL) {
    __shared__ __align__(16) uint32_t marks[(TH == kLong ? kMaxListed : kShortVocab) / 32];
    mine = stream_part<false, true, false>(p, scale, reinterpret_cast<const unsigned char*>(marks), nullptr, [&] {
      for (int i = threadIdx.x; i < (len + 31) / 32; i += TH) marks[i] = 0;
      load_teacher<TH>(a.teacher, row, a.vocab, teacher);
      for (int j = threadIdx.x; j < a.teacher.k; j += TH) {
        const int64_t at = teacher.id[j] < 0 ? -1 : teacher.id[j] - first;
        if (at >= 0 && at < len) atomicOr(&marks[at >> 5], 1u << (at & 31));
      }
      __syncthreads();
    });
  } else {
    mine = stream_part<false, false, false>(p, scale, nullptr, nullptr, [&] {
      if (a.parts == 1) load_teacher<TH>(a.teacher, row, a.vocab, teacher);
    });
  }
  const Running r = block_running<TH>(mine, scale, slots);
  if (a.parts == 1) {
    if (threadIdx.x < kWave) finish_distill<T>(r, a, row, teacher);
  } else if (threadIdx.x == 0) a.part_stats[block] = make_float4(r.m, r.s, 0.0f, 0.0f);
}
template <class T>
__global__ __launch_bounds__(kLong) void distill_join_kernel(DistillArgs a) {
  constexpr int TH = kLong;
  __shared__ Slots slots;
  __shared__ TeacherSmem teacher;
  const int64_t row = linear_block();
  if (row >= a.n) return;
  load_teacher<TH>(a.teacher, row, a.vocab, teacher);
  const Running r = join_parts<TH>(a.part_stats + row * a.parts, a.parts, kLog2e / a.temperature, slots);
  if (threadIdx.x < kWave) finish_distill<T>(r, a, row, teacher);
}

// The largest of the values that count, and 1 over the sum of exp((value - that) / T), for a wave of its own accord.  Log q_j is
// value / T - norm, but with the values far from 0 norm as a float32 is off by more than their differences: beyond kNormTrusted (log
// probabilities as a teacher has them are within it; there log q_j is off by 3e-6 at most) q_j is taken from the values alone.  65 x 50021
// float32 with 100 listed: 11.3 us by the norm, 12.4 without it.
constexpr float kNormTrusted = 16.0f;
__device__ __forceinline__ void list_softmax(const TeacherSmem& list, int k, float scale, float& value_max, float& share) {
  constexpr int kEntries = CAMERA_MAX_ALTERNATIVES / kWave;
  const int lane = threadIdx.x % kWave;
  float value[kEntries], most = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int e = 0; e < kEntries; ++e) {
    const int j = e * kWave + lane;
    value[e] = j < k && list.id[j] >= 0 ? list.value[j] : -INFINITY;
    most = fmaxf(most, value[e]);
  }
  most = wave_all(most, Max{});
#pragma unroll
  for (int e = 0; e < kEntries; ++e) sum += __builtin_amdgcn_exp2f((value[e] - most) * scale);  // 0 where there is none
  value_max = most;
  share = 1.0f / wave_all(sum, Add{});
}

// d loss / dz_v = (mass p_v - q_v) / T for a listed v, p_v (mass - q_r / p_r) / T for an unlisted one (mass alone without tail):
// the second for every token of the part, then the first over the listed ones.  A listed token's logit and old gradient
// are read before anything is written (dlogits may be logits), and its value is written after the workgroup's stores are done.
template <class T, int TH>
__global__ __launch_bounds__(TH) void distill_grad_kernel(LogitGradArgs a, DistillTeacher teacher, int tail,
                                                                const float* __restrict__ grad_loss) {
  __shared__ TeacherSmem list;
  const int64_t block = linear_block();
  const int64_t row = block / a.parts;
  if (row >= a.n) return;
  GradPart<T, TH> p = grad_part<T, TH>(a, row, (int)(block - row * a.parts));
  const float* st = a.stats + row * CAMERA_DISTILL_STATS;
  const float m = st[0], log_sum = st[1], norm = st[2], log_ratio = st[4];
  const bool far = log_ratio > kFarClass;
  const float mass = far ? 1.0f : st[3];
  const float inv_t = a.inv_temperature, g = grad_loss[row] * inv_t;
  if (g == 0.0f || (m == -INFINITY && log_sum == 0.0f)) {  // no gradient, or nothing but -inf
    if (!p.accumulate) p.zero();
    return;
  }
  p.fetch();  // in flight while the list is looked through
  load_teacher<TH>(teacher, row, a.vocab, list);
  constexpr int kEach = (CAMERA_MAX_ALTERNATIVES + TH - 1) / TH;  // entries of a thread
  int64_t at[kEach];
  float listed[kEach];
  bool any = false;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int j = threadIdx.x + e * TH;
    at[e] = j < teacher.k && list.id[j] >= 0 ? list.id[j] - p.first : -1;
    if (at[e] >= p.len) at[e] = -1;
    any = any || at[e] >= 0;
  }
  const float scale2 = inv_t * kLog2e;
  const bool by_norm = fabsf(norm) <= kNormTrusted;
  float value_max = 0.0f, share = 0.0f;  // of a norm that is not trusted
  if (!tail && !by_norm && __any(any)) list_softmax(list, teacher.k, scale2, value_max, share);
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    listed[e] = 0.0f;
    if (at[e] >= 0) {
      const float value = list.value[threadIdx.x + e * TH];
      const float lp = floored((Pack<T>::one(p.z[at[e]]) - m) * inv_t - log_sum);
      float q;
      if (tail || by_norm) q = expf(tail ? value : value * inv_t - norm);
      else q = share * __builtin_amdgcn_exp2f((value - value_max) * scale2);
      listed[e] = g * (mass * expf(lp) - q);
      if (p.accumulate) listed[e] += Pack<T>::one(p.out[at[e]]);
    }
  }
  __syncthreads();  // the reads above are done before the part is written
  // p_v (mass - q_r / p_r) as one exponential: the ratio may be as large as p_r is small, and mass is then nothing beside it
  const float factor = mass - expf(log_ratio), c = factor < 0.0f ? -g : g, from = far ? norm : m;
  const float log2_factor = far              ? st[3] * kLog2e
                            : factor == 0.0f ? kFloor
                                             : (log_ratio > 80.0f ? log_ratio : logf(fabsf(factor))) * kLog2e - log_sum * kLog2e;
  p.each([&](float* x, int, auto count) {
    constexpr int N = decltype(count)::value;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = c * __builtin_amdgcn_exp2f(fmaf(x[i] - from, scale2, log2_factor));
  });
  __syncthreads();  // and written before the listed tokens are
#pragma unroll
  for (int e = 0; e < kEach; ++e)
    if (at[e] >= 0) p.out[at[e]] = Pack<T>::round(listed[e]);
}

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

}  // namespace

// Parts of a row: as many as give the chip kLogitParts workgroups, each with at least a vector for every thread.  Many short rows
// are left whole, in short workgroups, which the chip holds four times as many of.  us in long / short ones, 4096 rows, 20
// alternatives: of 1000 31 / 13, of 4000 32 / 17, of 16000 43 / 36; of 32000 (beyond the line) 54 in long ones.
LogitPlan logit_plan(int dtype, int64_t n, int64_t vocab, bool marks, int top_k) {
  const int64_t vec = dtype == CAMERA_BF16 ? 8 : 4, least = kLong * vec;
  LogitPlan plan{1, vocab, kShort};
  if (n >= kLogitParts && vocab <= kShortVocab && top_k <= kShortTop) return plan;
  plan.threads = kLong;
  int64_t parts = std::max<int64_t>(1, kLogitParts / std::max<int64_t>(1, n));
  parts = std::min(parts, std::max<int64_t>(1, vocab / least));
  if (marks) parts = std::max(parts, (vocab + kMaxListed - 1) / kMaxListed);
  parts = std::max(parts, (vocab + (int64_t(1) << 30) - 1) >> 30);  // a part's elements are counted in 31 bits
  plan.part_len = round_up((vocab + parts - 1) / parts, least / 8);
  plan.parts = (int)((vocab + plan.part_len - 1) / plan.part_len);
  return plan;
}

// CALL with T and TH
#define CAMERA_BY_TYPE(dtype, threads, CALL) \
  do {                                       \
    auto call = [&](auto type, auto th) {    \
      using T = decltype(type);              \
      constexpr int TH = decltype(th)::value; \
      CALL;                                  \
    };                                       \
    using Short = std::integral_constant<int, kShort>; \
    using Long = std::integral_constant<int, kLong>;   \
    if ((dtype) == CAMERA_BF16) {            \
      if ((threads) == kShort) call(__bf16{}, Short{}); \
      else call(__bf16{}, Long{});           \
    } else {                                 \
      if ((threads) == kShort) call(float{}, Short{});  \
      else call(float{}, Long{});            \
    }                                        \
  } while (0)

hipError_t launch_token_logprobs(hipStream_t stream, int dtype, const LogprobArgs& a) {
  const int64_t blocks = a.n * a.parts;
  if (blocks <= 0 || blocks >= (int64_t(1) << 31)) return hipErrorInvalidValue;
  if (a.threads == kShort ? a.parts != 1 || a.top_k > kShortTop : a.threads != kLong) return hipErrorInvalidValue;
  CAMERA_BY_TYPE(dtype, a.threads, {
    if (a.parts == 1) {
      if (a.top_k > 0) hipLaunchKernelGGL((logprobs_kernel<T, TH, true, true>), launch_grid(blocks), dim3(TH), 0, stream, a);
      else hipLaunchKernelGGL((logprobs_kernel<T, TH, false, true>), launch_grid(blocks), dim3(TH), 0, stream, a);
    } else if constexpr (TH == kLong) {
      if (a.top_k > 0) {
        hipLaunchKernelGGL((logprobs_kernel<T, TH, true, false>), launch_grid(blocks), dim3(TH), 0, stream, a);
        hipLaunchKernelGGL((logprobs_join_kernel<T, true>), launch_grid(a.n), dim3(TH), 0, stream, a);
      } else {
        hipLaunchKernelGGL((logprobs_kernel<T, TH, false, false>), launch_grid(blocks), dim3(TH), 0, stream, a);
        hipLaunchKernelGGL((logprobs_join_kernel<T, false>), launch_grid(a.n), dim3(TH), 0, stream, a);
      }
    }
  });
  return hipGetLastError();
}

LogitPlan logit_grad_plan(int dtype, int64_t vocab) {
  const int64_t vec = dtype == CAMERA_BF16 ? 8 : 4;
  LogitPlan plan{1, kShort * kGradUnroll * vec, kShort};
  if (vocab > plan.part_len) plan = {1, kLong * kGradUnroll * vec, kLong};
  plan.parts = (int)((vocab + plan.part_len - 1) / plan.part_len);
  return plan;
}

hipError_t launch_token_logprobs_grad(hipStream_t stream, int dtype, const LogitGradArgs& a, const int32_t* targets,
                                      const float* entropy, const float* grad_logprob, const float* grad_entropy) {
  const int64_t blocks = a.n * a.parts;
  if (blocks <= 0 || blocks >= (int64_t(1) << 31)) return hipErrorInvalidValue;
  CAMERA_BY_TYPE(dtype, a.threads, hipLaunchKernelGGL((logprobs_grad_kernel<T, TH>), launch_grid(blocks), dim3(TH), 0, stream, a, targets,
                                                      entropy, grad_logprob, grad_entropy));
  return hipGetLastError();
}

hipError_t launch_distill(hipStream_t stream, int dtype, const DistillArgs& a) {
  const int64_t blocks = a.n * a.parts;
  if (blocks <= 0 || blocks >= (int64_t(1) << 31)) return hipErrorInvalidValue;
  if (a.threads == kShort ? a.parts != 1 || a.vocab > kShortVocab : a.threads != kLong) return hipErrorInvalidValue;
  if (a.tail && a.part_len > kMaxListed) return hipErrorInvalidValue;
  CAMERA_BY_TYPE(dtype, a.threads, {
    if (a.tail) hipLaunchKernelGGL((distill_kernel<T, TH, true>), launch_grid(blocks), dim3(TH), 0, stream, a);
    else hipLaunchKernelGGL((distill_kernel<T, TH, false>), launch_grid(blocks), dim3(TH), 0, stream, a);
    if (a.parts > 1) hipLaunchKernelGGL((distill_join_kernel<T>), launch_grid(a.n), dim3(kLong), 0, stream, a);
  });
  return hipGetLastError();
}

hipError_t launch_distill_grad(hipStream_t stream, int dtype, const LogitGradArgs& a, const DistillTeacher& teacher, int tail,
                               const float* grad_loss) {
  const int64_t blocks = a.n * a.parts;
  if (blocks <= 0 || blocks >= (int64_t(1) << 31)) return hipErrorInvalidValue;
  CAMERA_BY_TYPE(dtype, a.threads, hipLaunchKernelGGL((distill_grad_kernel<T, TH>), launch_grid(blocks), dim3(TH), 0, stream, a, teacher,
                                                      tail, grad_loss));
  return hipGetLastError();
}

}  // namespace camera
