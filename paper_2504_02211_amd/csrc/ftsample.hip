// Choice of the next token from its logits: the kernels and the C ABI of ../include/ftsample.h.
//
// Every logit has a key, a whole number that is ordered as the logits are; what the rules keep is "the keys above one key, and the first of those equal to it".  Weights are
// formed in 64 bits and summed as whole numbers: a sum in 32 bits is off by more than the borders between neighbouring tokens are apart, and one of 64-bit floating-point
// numbers depends on the order of its terms.
//
// A workgroup takes a row, each of its 8 waves a run of neighbouring tokens, in registers where they fit (131,072 of 16 bits, 65,536 of 32).  Rows with a small top_k keep
// what lies at or above the top_k-th largest of the threads' maxima (few more than top_k), sort it and sum it up by rank.  Without top_k all weights are formed; for top_p they are added to a histogram over
// their logarithm, 128 bins an octave, and the bin in which the limit lies is searched by keys.  In all other cases (a large top_k, thousands of equal
// logits) the border is searched by histograms of the keys' bits.  Last, kept weights are summed wave by wave, and the wave in which the random number falls looks for the token.
#include "ftsample.h"
#include "ftserve_device.h"

#include <cmath>
#include <new>
#include <string>

namespace ftsample {
using namespace ftserve;

constexpr int THREADS = 512, WAVES = THREADS / 64;
constexpr int BITS = 11, BINS = 1 << BITS;      // of a level of the search by keys
constexpr int STEPS = 128;                      // bins of the weights' logarithm to an octave
constexpr int OCTAVES = 51;                     // what lies further below the largest weight is 0 in all units
constexpr int LIST = THREADS, MOST_LISTED = THREADS / 2;   // tokens that are sorted; largest top_k that is
constexpr int MOST_WORDS = 32;                  // 16-byte words of a lane in registers

struct Args {
  const void* logits;
  int64_t stride;          // in elements
  int32_t vocab, shift;    // weights are whole multiples of 2^-shift
  const float* uniform;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* tokens;
  float* probability;
};

// Keys are ordered as their logits; both zeros have the same.  -infinity and NaN have 0, which nothing keeps.  (16 bits where the logits have as many.)
template <int DT> struct Keys {
  static constexpr bool WIDE = DT == FTSAMPLE_F32;
  static constexpr int PER = WIDE ? 4 : 8;               // elements of 16 bytes
  static constexpr uint32_t INF = WIDE ? 0x7F800000u : DT == FTSAMPLE_BF16 ? 0x7F80u : 0x7C00u, SIGN = WIDE ? 0x80000000u : 0x8000u, ALL = WIDE ? 0xFFFFFFFFu : 0xFFFFu;
  static constexpr uint32_t KEY_INFINITY = INF | SIGN;
  static __device__ __forceinline__ uint32_t of_bits(uint32_t u) {
    const uint32_t magnitude = u & (ALL ^ SIGN);
    if (magnitude > INF || u == (INF | SIGN)) return 0;
    return u & SIGN ? (magnitude ? ALL ^ u : SIGN) : u | SIGN;
  }
  // A key at or below (above: at or above) those of all logits that are at least (at most) x.
  static __device__ __forceinline__ uint32_t near(float x, bool above) {
    if (!(x == x)) return above ? ALL : 1u;
    const uint32_t u = as_u(x), wide = u & 0x80000000u ? ~u : u | 0x80000000u;
    if constexpr (WIDE) return above ? (wide > 0xFFFFFFF0u ? ALL : wide + 2) : (wide < 3 ? 1u : wide - 2);
    else if constexpr (DT == FTSAMPLE_BF16) return above ? ((wide >> 16) + 1 > ALL ? ALL : (wide >> 16) + 1) : ((wide >> 16) < 2 ? 1u : (wide >> 16) - 1);
    else {
      const uint32_t h = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x), k = h & SIGN ? ALL ^ h : h | SIGN;
      return above ? (k + 1 > ALL ? ALL : k + 1) : (k < 2 ? 1u : k - 1);
    }
  }
  static __device__ __forceinline__ float logit(uint32_t k) {
    const uint32_t u = k & SIGN ? k ^ SIGN : ALL ^ k;
    if constexpr (WIDE) return as_f(u);
    else if constexpr (DT == FTSAMPLE_BF16) return as_f(u << 16);
    else return (float)__builtin_bit_cast(half2v, u)[0];
  }
};

// The rules of a row, as they hold.
struct Rules {
  double per_t;        // 1 / temperature
  double floor;        // least weight that is kept
  double top_p, u;
  int32_t top_k;       // vocab: no limit
  bool cut_p, greedy;
};
__device__ __forceinline__ Rules rules_of(const Args& a, int row) {
  Rules r;
  float t = a.temperature ? a.temperature[row] : 1.f;
  if (t != t) t = 1.f;
  r.greedy = t <= 0.f;
  r.per_t = r.greedy ? 1.0 : 1.0 / (double)t;
  const int32_t k = a.top_k ? a.top_k[row] : 0;
  r.top_k = r.greedy ? 1 : k <= 0 || k > a.vocab ? a.vocab : k;
  const float p = a.top_p ? a.top_p[row] : 1.f, m = a.min_p ? a.min_p[row] : 0.f, u = a.uniform[row];
  r.cut_p = p < 1.f;
  r.top_p = p > 0.f ? (double)p : 0.0;
  r.floor = m > 0.f ? (m < 1.f ? (double)m : 1.0) : 0.0;
  r.u = u > 0.f ? (u < 1.f ? (double)u : 1.0 - 0x1p-24) : 0.0;
  return r;
}

// Weights of keys, given the largest one: w = 2^(n / STEPS) 2^(r / STEPS) with n whole and |r| <= 1/2, the first factor from a table and an exponent, the second
// from its series (the term left out is below 2^-65), in whole multiples of 2^-shift.
struct Weights {
  double scale, most;        // STEPS / (temperature * ln 2); the largest logit
  const double* table;       // 2^(i / STEPS)
  int shift;
  uint32_t infinite;         // the largest key where it stands for +infinity, else 0
  // w, and the number of the bin (0: the largest weights; STEPS * OCTAVES: nothing)
  __device__ __forceinline__ unsigned long long of(float x, uint32_t key, int& bin) const {
    if (__builtin_expect(infinite != 0, 0)) {
      bin = key == infinite ? 0 : STEPS * OCTAVES;
      return key == infinite ? 1ull << shift : 0ull;
    }
    constexpr double ROUND = 6755399441055744.0;      // 1.5 * 2^52
    const double t = __builtin_fmax(((double)x - most) * scale, -(double)(STEPS * OCTAVES));
    const double at = t + ROUND, r = t - (at - ROUND);
    const int n = (int)(uint32_t)__builtin_bit_cast(uint64_t, at);
    constexpr double L = 0.69314718055994530942 / STEPS;
    double p = __builtin_fma(r, L * L * L * L * L / 120, L * L * L * L / 24);
    p = __builtin_fma(r, p, L * L * L / 6);
    p = __builtin_fma(r, p, L * L / 2);
    p = __builtin_fma(r, p, L);
    p = __builtin_fma(r, p, 1.0);
    bin = -n;
    const double w = __builtin_ldexp(p * table[n & (STEPS - 1)], (n >> 7) + shift);
    return __builtin_bit_cast(uint64_t, w + 0x1p52) & ((1ull << 52) - 1);
  }
};
static_assert(STEPS == 128, "the octave is n >> 7");

// Sums over the workgroup of up to and before this thread's value.
template <class T> __device__ __forceinline__ T before_me(T x, T* scratch, T& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T upto = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T y = __shfl_up(upto, d);
    if (lane >= d) upto += y;
  }
  __syncthreads();
  if (lane == 63) scratch[wave] = upto;
  __syncthreads();
  T sum = 0, mine = 0;
  for (int w = 0; w < WAVES; ++w) {
    if (w == wave) mine = sum;
    sum += scratch[w];
  }
  all = sum;
  return mine + upto - x;
}

template <class T> __device__ __forceinline__ T wave_sum(T x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ uint32_t wave_most(uint32_t x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const uint32_t y = __shfl_xor(x, d);
    x = y > x ? y : x;
  }
  return x;
}

struct Shared {
  unsigned long long bins[STEPS * OCTAVES + 1 + (THREADS - (STEPS * OCTAVES + 1) % THREADS) % THREADS];      // whole rounds of all threads
  double table[STEPS];
  unsigned long long sums[WAVES];
  uint32_t words[WAVES];
  unsigned long long above;      // what lies above the bin that was found, and the bin
  uint32_t bin, count;
};

// The first bin, from first_bin on upwards in `order`, before which less than `limit` lies and with which it is reached, or the last that holds anything: s.bin, s.above.
// value(i): what the i-th bin in falling order of keys holds; PER of them a thread.
template <int PER, class F> __device__ __forceinline__ void find_bin(Shared& s, unsigned long long above, unsigned long long limit, F value) {
  unsigned long long mine = 0, all;
  const int first = (int)threadIdx.x * PER;
  for (int i = 0; i < PER; ++i) mine += value(first + i);
  unsigned long long at = above + before_me<unsigned long long>(mine, s.sums, all);
  if (mine)
    for (int i = 0; i < PER; ++i) {
      const unsigned long long n = value(first + i);
      if (n && at < limit && (at + n >= limit || at + n == above + all)) {
        s.bin = (uint32_t)(first + i);
        s.above = at;
      }
      at += n;
    }
  __syncthreads();
}

// The keys of a row, as the waves have them: wave w has neighbouring tokens, lane l of it those of its words l, l + 64, .. of 16 bytes; up to 32 words a lane in
// registers (HELD), or read anew every time.
template <int DT, bool HELD> struct Row {
  typedef Keys<DT> K;
  typedef uint32_t Words __attribute__((ext_vector_type(MOST_WORDS)));
  static constexpr int PER = K::PER;
  const char* x;           // aligned to 16 bytes, `skip` elements before the row
  int skip, vocab, words;  // words of a lane
  int first;               // this lane's first word
  Words held[HELD ? 4 : 1];      // (a register of each word, by its number: read with an index that is the same in all lanes)
  __device__ __forceinline__ Row(const Args& a, int row) : vocab(a.vocab) {
    constexpr int SIZE = K::WIDE ? 4 : 2;
    const char* const at = static_cast<const char*>(a.logits) + (int64_t)row * a.stride * SIZE;
    skip = (int)((uintptr_t)at & 15) / SIZE;
    x = at - skip * SIZE;
    words = ((vocab + skip + PER - 1) / PER + THREADS - 1) / THREADS;
    first = (int)(threadIdx.x >> 6) * words * 64 + (int)(threadIdx.x & 63);
    if constexpr (HELD) {
#pragma unroll
      for (int v = 0; v < MOST_WORDS; ++v) {
        uint4v r = nothing();
        if (v < words && whole(first + 64 * v)) r = load(first + 64 * v);
#pragma unroll
        for (int w = 0; w < 4; ++w) held[w][v] = r[w];
      }
      // the row's first and last word may lie in it only in part
#pragma unroll 1
      for (int v = 0; v < words; ++v) {
        uint4v r = {held[0][v], held[1][v], held[2][v], held[3][v]};
        const int word = first + 64 * v;
        if (__any(!whole(word) && some(word))) {
          const uint4v y = part(word);
          if (!whole(word) && some(word)) r = y;
        }
        r = keys(r);
#pragma unroll
        for (int w = 0; w < 4; ++w) held[w][v] = r[w];
      }
    }
  }
  // 16 bytes that lie in the row; that do in part (what does not is -infinity); that do not
  __device__ __forceinline__ bool whole(int word) const { return word * PER >= skip && word * PER - skip + PER <= vocab; }
  __device__ __forceinline__ bool some(int word) const { return word * PER - skip + PER > 0 && word * PER - skip < vocab; }
  __device__ __forceinline__ uint4v load(int word) const { return *reinterpret_cast<const uint4v*>(x + (int64_t)word * 16); }
  static __device__ __forceinline__ uint4v nothing() {
    constexpr uint32_t none = K::WIDE ? K::INF | K::SIGN : (K::INF | K::SIGN) * 0x10001u;
    return uint4v{none, none, none, none};
  }
  __device__ __forceinline__ uint4v part(int word) const {
    uint4v r = nothing();
    const int i = word * PER - skip;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      if (i + e < 0 || i + e >= vocab) continue;
      if constexpr (K::WIDE) r[e] = reinterpret_cast<const uint32_t*>(x)[(int64_t)word * PER + e];
      else r[e >> 1] = (r[e >> 1] & ~(0xFFFFu << 16 * (e & 1))) | (uint32_t)reinterpret_cast<const uint16_t*>(x)[(int64_t)word * PER + e] << 16 * (e & 1);
    }
    return r;
  }
  static __device__ __forceinline__ uint4v keys(uint4v r) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (K::WIDE) r[w] = K::of_bits(r[w]);
      else r[w] = K::of_bits(r[w] & 0xFFFFu) | K::of_bits(r[w] >> 16) << 16;
    }
    return r;
  }
  static __device__ __forceinline__ uint32_t key(const uint4v& k, int e) {
    if constexpr (K::WIDE) return k[e];
    else return k[e >> 1] >> 16 * (e & 1) & 0xFFFFu;
  }
  // f(v, keys) for every word of this lane
  template <class F> __device__ __forceinline__ void each_word(F f) const {
#pragma unroll 1
    for (int v = 0; v < words; ++v) {
      if constexpr (HELD) f(v, uint4v{held[0][v], held[1][v], held[2][v], held[3][v]});
      else {
        const int word = first + 64 * v;
        f(v, keys(whole(word) ? load(word) : part(word)));
      }
    }
  }
  template <class F> __device__ __forceinline__ void each(F f) const {
    each_word([&](int, const uint4v& k) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < PER; ++e) f(key(k, e));
    });
  }
  __device__ __forceinline__ int token(int v, int e) const { return (first + 64 * v) * PER + e - skip; }
};

// What the rules have left: keys above `border`, and the first `equal` of those that are it; of those, weights of at least `floor`.
struct Kept {
  uint32_t border;
  int equal;
  unsigned long long floor;
};

template <int DT, bool HELD>
__global__ __launch_bounds__(THREADS) void ftsample_row(const Args a) {
  typedef Keys<DT> K;
  __shared__ Shared s;
  __shared__ unsigned long long list[LIST];      // (under top_k) key and place, then weights by place
  __shared__ int listed[LIST];
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Row<DT, HELD> x(a, row);
  if (tid < STEPS) s.table[tid] = exp2((double)tid / STEPS);
  const Rules r = rules_of(a, row);

  uint32_t mine = 0;
  x.each([&](uint32_t k) __attribute__((always_inline)) { mine = k > mine ? k : mine; });
  uint32_t most = wave_most(mine);
  if (lane == 0) s.words[wave] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) most = s.words[w] > most ? s.words[w] : most;
  auto answer = [&](int token, double chance) {
    a.tokens[row] = token;
    if (a.probability) a.probability[row] = (float)chance;
  };
  if (most == 0) {
    if (tid == 0) answer(-1, 0.0);
    return;
  }
  const Weights weights{r.per_t * (STEPS / 0.69314718055994530942), (double)K::logit(most), s.table, a.shift, most == K::KEY_INFINITY ? most : 0u};
  auto weight = [&](uint32_t k) __attribute__((always_inline)) {
    int bin;
    return weights.of(K::logit(k), k, bin);
  };
  const unsigned long long floor = (unsigned long long)__builtin_ceil(__builtin_ldexp(r.floor, a.shift));
  auto limit_of = [&](unsigned long long all) -> unsigned long long {      // the least whole number that is top_p of all, or 1
    const double limit = __builtin_ceil(r.top_p * (double)all);
    return limit >= 1.0 ? (unsigned long long)limit : 1ull;
  };

  // The first place at which the sum of kept weights exceeds u times all: whole numbers exceed it where they reach the next one.  sum: this wave's kept weights without those of the
  // border; ties: how many keys of it are the border.
  auto choose = [&](const Kept& kept, unsigned long long sum, uint32_t ties) {
    const unsigned long long each = kept.equal ? weight(kept.border) : 0, worth = each >= kept.floor || kept.border == most ? each : 0;
    __syncthreads();
    if (lane == 0) {
      s.sums[wave] = sum;
      s.words[wave] = ties;
    }
    __syncthreads();
    unsigned long long before = 0, all = 0, inside = 0;
    int left = kept.equal, allowed = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int n = (int)s.words[w] < left ? (int)s.words[w] : left;
      const unsigned long long here = s.sums[w] + (unsigned long long)n * worth;
      if (w < wave) before += here;
      if (w == wave) {
        allowed = n;
        inside = here;
      }
      left -= n;
      all += here;
    }
    const unsigned long long goal = (unsigned long long)__builtin_floor(r.u * (double)all) + 1;
    if (before >= goal || before + inside < goal) return;      // (another wave)
    bool done = false;
    x.each_word([&](int v, const uint4v& k) {
      if (done) return;
      uint32_t n = 0;
#pragma unroll
      for (int e = 0; e < K::PER; ++e) n += kept.equal && Row<DT, HELD>::key(k, e) == kept.border;
      // ties of lanes before this one
      uint32_t upto = n;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
      }
      int mine = allowed - (int)(upto - n);
      auto one = [&](int e) __attribute__((always_inline)) -> unsigned long long {
        const uint32_t key = Row<DT, HELD>::key(k, e);
        if (key == 0 || key < kept.border) return 0;
        if (key == kept.border) return mine-- > 0 ? worth : 0;
        const unsigned long long w = weight(key);
        return key == most || w >= kept.floor ? w : 0;
      };
      const int held = mine;
      unsigned long long lane_sum = 0;
#pragma unroll
      for (int e = 0; e < K::PER; ++e) lane_sum += one(e);
      unsigned long long lane_upto = lane_sum;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const unsigned long long y = __shfl_up(lane_upto, d);
        if (lane >= d) lane_upto += y;
      }
      unsigned long long at = before + lane_upto - lane_sum;
      if (at < goal && at + lane_sum >= goal) {
        mine = held;
#pragma unroll
        for (int e = 0; e < K::PER; ++e) {
          const unsigned long long w = one(e);
          if (at < goal && at + w >= goal) answer(x.token(v, e), (double)w / (double)all);
          at += w;
        }
      }
      const int n_all = (int)__shfl(upto, 63);
      allowed -= n_all < allowed ? n_all : allowed;
      before += __shfl(lane_upto, 63);
      done = before >= goal;
    });
  };
  auto sum_up = [&](const Kept& kept) {
    unsigned long long sum = 0;
    uint32_t ties = 0;
    x.each([&](uint32_t k) __attribute__((always_inline)) {
      if (k > kept.border) {
        const unsigned long long w = weight(k);
        sum += k == most || w >= kept.floor ? w : 0;
      }
      ties += k == kept.border;
    });
    choose(kept, wave_sum(sum), wave_sum(kept.equal ? ties : 0u));
  };

  // The border moves up to the lowest key above which less than `limit` lies, by counts or by sums of weights; among the keys of lowest .. highest.
  Kept kept{0, 0, floor};
  auto search = [&](unsigned long long limit, bool by_weight, uint32_t lowest, uint32_t highest, unsigned long long above) {
    while (lowest != highest) {
      const uint32_t range = highest - lowest;
      const int bits = 32 - __builtin_clz(range), drop = bits > BITS ? bits - BITS : 0;
      __syncthreads();
      for (int i = tid; i < BINS; i += THREADS) s.bins[i] = 0;
      __syncthreads();
      x.each([&](uint32_t k) __attribute__((always_inline)) {
        if (k < lowest || k > highest || k <= kept.border) return;
        atomicAdd(&s.bins[(highest - k) >> drop], by_weight ? weight(k) : 1ull);
      });
      __syncthreads();
      // (the kept ones of the border that there is)
      if (tid == 0 && kept.equal && kept.border >= lowest && kept.border <= highest) s.bins[(highest - kept.border) >> drop] += (by_weight ? weight(kept.border) : 1ull) * (unsigned)kept.equal;
      __syncthreads();
      find_bin<BINS / THREADS>(s, above, limit, [&](int i) { return s.bins[i]; });
      above = s.above;
      const uint32_t top = highest - (s.bin << drop), least = top - ((1u << drop) - 1);
      lowest = least > lowest && least <= top ? least : lowest;
      highest = top;
      __syncthreads();
    }
    // of the keys that are the border, as many as fit
    const unsigned long long each = by_weight ? weight(lowest) : 1;
    unsigned long long fit = each ? (limit - above + each - 1) / each : 0x7FFFFFFFull;
    if (lowest == kept.border && (unsigned long long)kept.equal < fit) fit = kept.equal;
    kept.border = lowest;
    kept.equal = (int)(fit > 0x7FFFFFFFull ? 0x7FFFFFFFull : fit);
  };

  if (r.top_k < x.vocab) {
    bool sorted = false;
    if (r.top_k <= MOST_LISTED) {
      // The top_k-th largest of the threads' maxima: at least top_k keys are as large.  Its highest bits are enough for a bound: two levels.
      uint32_t lowest = 1, highest = most;
      unsigned long long above = 0;
      for (int level = 0; level < 2 && lowest != highest; ++level) {
        const int bits = 32 - __builtin_clz(highest - lowest), drop = bits > BITS ? bits - BITS : 0;
        __syncthreads();
        for (int i = tid; i < BINS; i += THREADS) s.bins[i] = 0;
        __syncthreads();
        if (mine >= lowest && mine <= highest) atomicAdd(&s.bins[(highest - mine) >> drop], 1ull);
        __syncthreads();
        find_bin<BINS / THREADS>(s, above, (unsigned long long)r.top_k, [&](int i) { return s.bins[i]; });
        above = s.above;
        const uint32_t top = highest - (s.bin << drop), least = top - ((1u << drop) - 1);
        lowest = least > lowest && least <= top ? least : lowest;
        highest = top;
        __syncthreads();
      }
      uint32_t n = 0, maxima;
      before_me<uint32_t>(mine >= lowest ? 1u : 0u, s.words, maxima);
      if (maxima < (uint32_t)r.top_k) lowest = 1;      // (fewer of them that can be chosen)
      x.each([&](uint32_t k) __attribute__((always_inline)) { n += k >= lowest; });
      __syncthreads();
      const uint32_t in_wave = wave_sum(n);
      if (lane == 0) s.words[wave] = in_wave;
      __syncthreads();
      uint32_t at = 0, count = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        if (w < wave) at += s.words[w];
        count += s.words[w];
      }
      if (count <= LIST) {
        sorted = true;
        // the keys in the order of their tokens: (key, place) in the list, tokens by place
        if (in_wave)
          x.each_word([&](int v, const uint4v& k) {
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < K::PER; ++e) m += Row<DT, HELD>::key(k, e) >= lowest;
            if (!__any(m != 0)) return;
            uint32_t upto = m;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
              const uint32_t y = __shfl_up(upto, d);
              if (lane >= d) upto += y;
            }
            uint32_t place = at + upto - m;
#pragma unroll
            for (int e = 0; e < K::PER; ++e) {
              const uint32_t key = Row<DT, HELD>::key(k, e);
              if (key < lowest) continue;
              list[place] = (unsigned long long)key << 32 | (0xFFFFFFFFu - place);
              listed[place] = x.token(v, e);
              ++place;
            }
            at += __shfl(upto, 63);
          });
        __syncthreads();
        // sorted, the largest first: thread i has the i-th.  Distances below 64 stay inside a wave.
        int size = 64;
        while (size < (int)count) size <<= 1;
        unsigned long long e = tid < (int)count ? list[tid] : 0;
        for (int k = 2; k <= size; k <<= 1)
          for (int j = k >> 1; j > 0; j >>= 1) {
            unsigned long long other;
            if (j >= 64) {
              __syncthreads();
              list[tid] = e;
              __syncthreads();
              other = list[tid ^ j];
            } else {
              other = __shfl_xor(e, j);
            }
            const bool larger_first = (tid & k) == 0, lower = (tid & j) == 0;
            const bool take = (lower == larger_first) ? other > e : other < e;
            if (take) e = other;
          }
        const uint32_t key = (uint32_t)(e >> 32);
        unsigned long long w = tid < (int)count && tid < r.top_k ? weight(key) : 0, all;
        unsigned long long before = before_me<unsigned long long>(w, s.sums, all);
        if (r.cut_p && before >= limit_of(all) && tid > 0) w = 0;
        if (w < floor && tid > 0) w = 0;
        __syncthreads();
        list[tid] = 0;
        __syncthreads();
        if (w) list[0xFFFFFFFFu - (uint32_t)e] = w;
        __syncthreads();
        // and summed up in the order of their tokens
        w = list[tid];
        before = before_me<unsigned long long>(w, s.sums, all);
        const unsigned long long goal = (unsigned long long)__builtin_floor(r.u * (double)all) + 1;
        if (before < goal && before + w >= goal) answer(listed[tid], (double)w / (double)all);
      }
    }
    if (sorted) return;
    __syncthreads();
    search((unsigned long long)r.top_k, false, 1, most, 0);
    if (r.cut_p) {
      unsigned long long sum = 0, all;
      uint32_t there = 0, ties;
      x.each([&](uint32_t k) __attribute__((always_inline)) {
        if (k > kept.border) sum += weight(k);
        there += k == kept.border;
      });
      before_me<unsigned long long>(sum, s.sums, all);
      // (where fewer than top_k can be chosen, fewer are equal than there is room for)
      before_me<uint32_t>(there, s.words, ties);
      if ((uint32_t)kept.equal > ties) kept.equal = (int)ties;
      all += (unsigned long long)kept.equal * weight(kept.border);
      search(limit_of(all), true, kept.border, most, 0);
    }
    sum_up(kept);
    return;
  }

  // No top_k: all weights, those of at least the floor, and (top_p) how they are distributed.
  if (r.cut_p) {
    constexpr int N = sizeof(s.bins) / sizeof(s.bins[0]);
    for (int i = tid; i < N; i += THREADS) s.bins[i] = 0;
    __syncthreads();
  }
  unsigned long long sum = 0, high = 0;
  x.each([&](uint32_t k) __attribute__((always_inline)) {
    if (k == 0) return;
    int bin;
    const unsigned long long w = weights.of(K::logit(k), k, bin);
    sum += w;
    high += k == most || w >= floor ? w : 0;
    if (r.cut_p && w) atomicAdd(&s.bins[bin], w);
  });
  high = wave_sum(high);
  if (!r.cut_p) {
    choose(kept, high, 0);
    return;
  }
  unsigned long long all, all_high = 0;
  before_me<unsigned long long>(sum, s.sums, all);
  __syncthreads();
  if (lane == 0) s.sums[wave] = high;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) all_high += s.sums[w];
  const unsigned long long limit = limit_of(all);
  if (all_high <= limit) {      // top_p keeps more than min_p does: what is not below the floor has, before its last, less than the limit
    choose(kept, high, 0);
    return;
  }
  __syncthreads();
  constexpr int PER_THREAD = sizeof(s.bins) / sizeof(s.bins[0]) / THREADS;
  find_bin<PER_THREAD>(s, 0, limit, [&](int i) { return s.bins[i]; });
  const int bin = (int)s.bin;
  const unsigned long long above = s.above;
  // the keys of that bin, and some more: a bin is as wide as 1 / scale
  __syncthreads();
  uint32_t lowest = 0xFFFFFFFFu, highest = 0;
  {
    const double wide = 1.0 / weights.scale, top = weights.most - ((double)bin - 0.5) * wide, margin = wide * 0.01 + __builtin_fabs(weights.most) * 0x1p-40;
    const float lo = (float)(top - wide - margin), hi = (float)(top + margin);
    const uint32_t klo = K::near(lo, false), khi = K::near(hi, true);
    x.each([&](uint32_t k) __attribute__((always_inline)) {
      if (k < klo || k > khi || k == 0) return;
      int b;
      const unsigned long long w = weights.of(K::logit(k), k, b);
      if (b != bin || !w) return;
      lowest = k < lowest ? k : lowest;
      highest = k > highest ? k : highest;
    });
  }
  highest = wave_most(highest);
  lowest = ~wave_most(~lowest);
  if (lane == 0) s.words[wave] = highest;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) highest = s.words[w] > highest ? s.words[w] : highest;
  __syncthreads();
  if (lane == 0) s.words[wave] = lowest;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) lowest = s.words[w] < lowest ? s.words[w] : lowest;
  search(limit, true, lowest, highest, above);      // (no key between these is in another bin)
  sum_up(kept);
}

typedef void (*kernel_fn)(const Args);
// The kernel of a vocabulary: rows in registers where they fit, wherever they begin.
template <int DT> kernel_fn kernel_of(int vocab) {
  const int words = (vocab + 2 * Keys<DT>::PER - 2) / Keys<DT>::PER;
  return words <= MOST_WORDS * THREADS ? ftsample_row<DT, true> : ftsample_row<DT, false>;
}


}  // namespace ftsample

using namespace ftsample;

struct ftsample_ctx {
  ftsample_config cfg;
  kernel_fn fn = nullptr;
  std::string err;
};

static thread_local std::string g_sample_create_err;

static int sfail(ftsample_ctx* c, int code, const char* msg) {
  try {
    (c ? c->err : g_sample_create_err) = msg;
  } catch (...) {
  }
  return code;
}
static int sfail_hip(ftsample_ctx* c, const char* what, hipError_t e) {
  try {
    (c ? c->err : g_sample_create_err) = std::string(what) + ": " + hipGetErrorString(e);
  } catch (...) {
  }
  return e == hipErrorOutOfMemory ? FTSAMPLE_ENOMEM : FTSAMPLE_EHIP;
}

extern "C" int ftsample_create(const ftsample_config* cfg, ftsample_ctx** out) {
  if (!cfg || !out) return sfail(nullptr, FTSAMPLE_EINVAL, "null argument");
  *out = nullptr;
  if (cfg->struct_size != sizeof(ftsample_config)) return sfail(nullptr, FTSAMPLE_EINVAL, "struct_size mismatch");
  if (cfg->vocab < 1) return sfail(nullptr, FTSAMPLE_EINVAL, "vocab must be >= 1");
  if (cfg->vocab > 1 << 20) return sfail(nullptr, FTSAMPLE_EUNSUPPORTED, "vocab above 2^20");
  if (cfg->max_rows < 1 || cfg->max_rows > 65536) return sfail(nullptr, FTSAMPLE_EINVAL, "max_rows must be 1 .. 65536");
  if (cfg->in_dtype != FTSAMPLE_F16 && cfg->in_dtype != FTSAMPLE_BF16 && cfg->in_dtype != FTSAMPLE_F32) return sfail(nullptr, FTSAMPLE_EINVAL, "in_dtype must be F16, BF16 or F32");
  ftsample_ctx* c = new (std::nothrow) ftsample_ctx();
  if (!c) return sfail(nullptr, FTSAMPLE_ENOMEM, "out of host memory");
  c->cfg = *cfg;
  c->fn = cfg->in_dtype == FTSAMPLE_F32 ? kernel_of<FTSAMPLE_F32>(cfg->vocab) : cfg->in_dtype == FTSAMPLE_BF16 ? kernel_of<FTSAMPLE_BF16>(cfg->vocab) : kernel_of<FTSAMPLE_F16>(cfg->vocab);
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess) he = hipSetDevice(cfg->device);
  if (he == hipSuccess) (void)hipSetDevice(before);
  if (he != hipSuccess) {
    const int rc = sfail_hip(nullptr, "device", he);
    delete c;
    return rc;
  }
  *out = c;
  return FTSAMPLE_OK;
}

extern "C" int ftsample_get_config(const ftsample_ctx* ctx, ftsample_config* effective) {
  if (!ctx || !effective) return FTSAMPLE_EINVAL;
  *effective = ctx->cfg;
  return FTSAMPLE_OK;
}

extern "C" int ftsample_choose(ftsample_ctx* c, const void* logits, int64_t row_stride, int32_t rows, const float* uniform, const ftsample_rules* rules, int32_t* tokens,
                               float* probability, void* hip_stream) {
  if (!c) return FTSAMPLE_EINVAL;
  const ftsample_config& e = c->cfg;
  if (rows < 0 || rows > e.max_rows) return sfail(c, FTSAMPLE_EINVAL, "rows must be 0 .. max_rows");
  if (rows == 0) return FTSAMPLE_OK;
  if (!logits || !uniform || !tokens) return sfail(c, FTSAMPLE_EINVAL, "null argument");
  if ((uintptr_t)logits % (e.in_dtype == FTSAMPLE_F32 ? 4 : 2) || ((uintptr_t)uniform | (uintptr_t)tokens | (uintptr_t)probability) % 4) return sfail(c, FTSAMPLE_EINVAL, "arrays must be aligned to their elements");
  if (rules && ((uintptr_t)rules->temperature | (uintptr_t)rules->top_k | (uintptr_t)rules->top_p | (uintptr_t)rules->min_p) % 4) return sfail(c, FTSAMPLE_EINVAL, "arrays must be aligned to their elements");
  if (row_stride < 0 || row_stride > (1ll << 40)) return sfail(c, FTSAMPLE_EUNSUPPORTED, "the row stride must be 0 .. 2^40");
  int bits = 0;
  while ((1 << bits) < e.vocab) ++bits;
  Args a{logits, row_stride, e.vocab, bits <= 12 ? 50 : 62 - bits, uniform, rules ? rules->temperature : nullptr, rules ? rules->top_k : nullptr, rules ? rules->top_p : nullptr,
         rules ? rules->min_p : nullptr, tokens, probability};
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess && before != e.device) he = hipSetDevice(e.device);
  if (he != hipSuccess) return sfail_hip(c, "device", he);
  hipLaunchKernelGGL(c->fn, dim3((uint32_t)rows), dim3(THREADS), 0, (hipStream_t)hip_stream, a);
  he = hipGetLastError();
  if (before != e.device) (void)hipSetDevice(before);
  return he == hipSuccess ? FTSAMPLE_OK : sfail_hip(c, "launch", he);
}

extern "C" int ftsample_destroy(ftsample_ctx* c) {
  delete c;
  return FTSAMPLE_OK;
}

extern "C" const char* ftsample_last_error(const ftsample_ctx* c) { return c ? c->err.c_str() : g_sample_create_err.c_str(); }
