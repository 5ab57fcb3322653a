// Choice of the next token from its logits: the kernels and the C ABI of ../include/ftsample.h.
//
// Every logit has a key, a whole number that is ordered as the logits are; what the rules keep is "the keys above one key, and the first of those equal to it".  Weights are
// formed in 64 bits and summed as whole numbers: a sum in 32 bits is off by more than the borders between neighbouring tokens are apart, and one of 64-bit floating-point
// numbers depends on the order of its terms.
//
// A workgroup takes a row, each of its 8 waves a run of neighbouring tokens, in registers where they fit (131,072 of 16 bits, 65,536 of 32).  Rows with a small top_k keep
// what lies at or above the top_k-th largest of the threads' maxima (few more than top_k), sort it and sum it up by rank.  In all other cases the border that top_k and
// top_p draw comes first, then one pass sums up the weights above it, wave by wave and run by run of words, and the lane of the run in which the random number falls finds the
// token.
//   - bf16 has few values: each has a number, how often it occurs is counted in LDS, and its weight stands there; no weight is formed per logit.  256 rows of 131,072 with a
//     temperature of their own take 30 us, with top_p 49 us; with a weight formed for each logit as below they took 46 and 100 us.
//   - fp16 and fp32: counts or weights are added to a histogram over the weights' logarithm, 128 bins an octave, and the bin in which the limit lies is searched: few logits of
//     32 bits lie there, which are sorted (48 rows of 50,001 with top_p 44 us; 50 when searched by histograms of the keys' bits); of 16 bits many are equal, and one
//     histogram of the keys' bits tells (sorted where they fit, 512 rows of 65,536 took 3 us more).  512 rows of 65,536 in fp16 take 48 us, with top_p 100 us.
// Bound by the row's one CU: reading 67 MB, 131,072 logits a CU, takes 10 of the 49 us (7 TB/s), counting 14, the border 6, the sum 12, where the reads and additions in LDS
// and the instructions that find their addresses take turns; greedy rows take 21 us.  Rows that do not fit in registers are read anew in each pass: one of 262,144 in
// fp32 takes 80 us greedy, 235 with top_p.
#include "ftsample.h"
#include "ftserve_device.h"

#include <cmath>
#include <new>
#include <string>
#include <type_traits>

namespace ftsample {
using namespace ftserve;

constexpr int THREADS = 512, WAVES = THREADS / 64;
constexpr int BITS = 11, BINS = 1 << BITS;      // of a level of the search by keys
constexpr int STEPS = 512;                      // of a weight's logarithm to an octave, for each of which there is a factor in LDS
constexpr int OCTAVES = 51;                     // what lies further below the largest weight is 0 in all units
constexpr int TO_BIN = 2, LAST_BIN = STEPS * OCTAVES >> TO_BIN;      // bins of the logarithm: 128 an octave
constexpr int MOST_BOUNDED = 256;               // largest top_k whose border the threads' maxima bound
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

// Logits of 16 bytes, and their keys: whole numbers that are ordered as they are (both zeros have the same), of as many bits as it takes.
template <int DT> struct Type {
  static constexpr bool WIDE = DT == FTSAMPLE_F32;
  static constexpr int SIZE = WIDE ? 4 : 2, PER = 16 / SIZE, DROP = WIDE ? 0 : DT == FTSAMPLE_BF16 ? 16 : 13;
  static constexpr uint32_t NONE = WIDE ? 0xFF800000u : DT == FTSAMPLE_BF16 ? 0xFF80FF80u : 0xFC00FC00u;      // -infinity
  static __device__ __forceinline__ float logit(const uint4v& r, int e) {
    if constexpr (WIDE) return as_f(r[e]);
    else return e & 1 ? high_of<DT == FTSAMPLE_BF16>(r[e >> 1]) : low_of<DT == FTSAMPLE_BF16>(r[e >> 1]);
  }
  static __device__ __forceinline__ uint32_t key(float x) {
    const uint32_t u = as_u(x + 0.f);
    return (u & 0x80000000u ? ~u : u | 0x80000000u) >> DROP;
  }
  static __device__ __forceinline__ float of_key(uint32_t k) {
    const uint32_t u = k << DROP;
    return as_f(u & 0x80000000u ? u ^ 0x80000000u : ~(u | ((1u << DROP) - 1)));
  }
  // The largest number whose key is at most k.  (The key below that of the zeros would be that of -0, which compares as they do.)
  static __device__ __forceinline__ float upto_key(uint32_t k) {
    const float x = of_key(k);
    return as_u(x) == 0x80000000u ? as_f(0x80000001u) : x;
  }
};
constexpr float NOTHING = -__builtin_inff();

// The rules of a row, as they hold.
struct Rules {
  double per_t;        // 1 / temperature
  double floor;        // least weight that is kept, 0: any
  double top_p, u;
  int32_t top_k;       // vocab: no limit
  bool cut_p, greedy;
};
__device__ __forceinline__ Rules rules_of(const Args& a, int row) {
  Rules r;
  float t = a.temperature ? a.temperature[row] : 1.f;
  if (t != t) t = 1.f;
  r.greedy = t <= 0.f;
  r.per_t = r.greedy ? 1.0 : __builtin_fmax(1.0 / (double)t, 0x1p-200);      // (never 0: the difference to -infinity is multiplied by it)
  const int32_t k = a.top_k ? a.top_k[row] : 0;
  r.top_k = r.greedy ? 1 : k <= 0 || k > a.vocab ? a.vocab : k;
  const float p = a.top_p ? a.top_p[row] : 1.f, m = a.min_p ? a.min_p[row] : 0.f, u = a.uniform[row];
  r.cut_p = p < 1.f;
  r.top_p = p > 0.f ? (double)p : 0.0;
  r.floor = m > 0.f ? (m < 1.f ? (double)m : 1.0) : 0.0;
  r.u = u > 0.f ? (u < 1.f ? (double)u : 1.0 - 0x1p-24) : 0.0;
  return r;
}

// Weights of logits, given the largest one: w = 2^(n / STEPS) 2^(r / STEPS) with n whole and |r| <= 1/2, the first factor from a table and an exponent, the second
// from its series (the term left out is below 2^-46), in whole multiples of 2^-shift.
struct Weights {
  double scale, most, least; // STEPS / (temperature * ln 2); the largest logit; the difference to it from which on all weights are 0
  const double* table;       // 2^(i / STEPS + shift)
  static constexpr double ROUND = 6755399441055744.0;      // 1.5 * 2^52
  // the logarithm in steps, and the nearest whole number of them; -infinity and NaN: as far below as counts
  __device__ __forceinline__ double steps(float x, int& n) const {
    const double d = __builtin_fmax((double)x - most, least), at = __builtin_fma(d, scale, ROUND);
    n = (int)(uint32_t)__builtin_bit_cast(uint64_t, at);
    return __builtin_fma(d, scale, ROUND - at);
  }
  __device__ __forceinline__ int bin(float x) const {
    int n;
    steps(x, n);
    return -n >> TO_BIN;
  }
  // w (of -infinity and NaN: 0), and its bin
  __device__ __forceinline__ unsigned long long of(float x, int& bin) const {
    int n;
    const double r = steps(x, n);
    constexpr double L = 0.69314718055994530942 / STEPS;
    double p = __builtin_fma(r, L * L * L / 6, L * L / 2);
    p = __builtin_fma(r, p, L);
    p = __builtin_fma(r, p, 1.0);
    bin = -n >> TO_BIN;
    const double w = __builtin_ldexp(p * table[n & (STEPS - 1)], n >> 9);
    return __builtin_bit_cast(uint64_t, w + 0x1p52) & ((1ull << 52) - 1);
  }
};
static_assert(STEPS == 512, "the octave is n >> 9");

// Sums over the lanes up to this one: rows of 16 by shifts, then their last lanes handed on.
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t shifted(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false); }
template <int CTRL, int ROWS> __device__ __forceinline__ unsigned long long shifted(unsigned long long x) {
  return (unsigned long long)shifted<CTRL, ROWS>((uint32_t)(x >> 32)) << 32 | shifted<CTRL, ROWS>((uint32_t)x);
}
template <class T> __device__ __forceinline__ T sum_upto(T x) {
  x += shifted<0x111, 0xF>(x);
  x += shifted<0x112, 0xF>(x);
  x += shifted<0x114, 0xF>(x);
  x += shifted<0x118, 0xF>(x);
  x += shifted<0x142, 0xA>(x);
  return x + shifted<0x143, 0xC>(x);
}
// The value of lane ^ J.
template <int J> __device__ __forceinline__ uint32_t across(uint32_t x) {
  if constexpr (J == 1) return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, false);           // quad_perm 1 0 3 2
  else if constexpr (J == 2) return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, false);      // quad_perm 2 3 0 1
  else if constexpr (J == 4) return (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, 4 << 10 | 0x1F);
  else if constexpr (J == 8) return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xF, 0xF, false);     // row_ror 8
  else if constexpr (J == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  }
}
template <int J> __device__ __forceinline__ float across(float x) { return as_f(across<J>(as_u(x))); }
template <int J> __device__ __forceinline__ unsigned long long across(unsigned long long x) {
  return (unsigned long long)across<J>((uint32_t)(x >> 32)) << 32 | across<J>((uint32_t)x);
}
// Steps of a bitonic sort, the largest first, over lanes J, J / 2, .. 1 apart; K: how many are merged in one direction.
template <int J, class T> __device__ __forceinline__ void merge(T& x, int at, int K) {
  const T other = across<J>(x);
  const bool larger = ((at & J) == 0) == ((at & K) == 0);
  x = larger == (other > x) ? other : x;
  if constexpr (J > 1) merge<J / 2>(x, at, K);
}
template <int K = 2, class T> __device__ __forceinline__ void sort_wave(T& x, int at) {
  merge<K / 2>(x, at, K);
  if constexpr (K < 64) sort_wave<2 * K>(x, at);
}
__device__ __forceinline__ uint32_t last_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, 63); }
__device__ __forceinline__ unsigned long long last_lane(unsigned long long x) { return (unsigned long long)last_lane((uint32_t)(x >> 32)) << 32 | last_lane((uint32_t)x); }

// Sums over the workgroup of up to and before this thread's value.
template <class T> __device__ __forceinline__ T before_me(T x, T* scratch, T& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T upto = sum_upto(x);
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

template <class T> __device__ __forceinline__ T wave_sum(T x) { return last_lane(sum_upto(x)); }
__device__ __forceinline__ float wave_most(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = __builtin_fmaxf(x, __shfl_xor(x, d));
  return x;
}

// Logits of bf16 by their value: there are few enough of them.  Those of a magnitude from `base` on, 23 octaves of 128, have a number, that of negative ones below 0; what is smaller
// ("tiny") is taken one by one; what is larger is so far below the largest logit, or NaN, that it has no weight: the numbers at either end.
constexpr int MAGNITUDES = 23 * 128, VALUES = 2 * MAGNITUDES + 2;
constexpr int TIE = 57;                  // (its bit: a lane adds up less than 2^56 and 64 ties)
template <bool KEYED> struct ByValue {};
template <> struct ByValue<true> {
  unsigned long long worth[VALUES];      // what a logit adds to the sum, TIE if it is the border
  uint32_t counts[VALUES];
};
template <bool KEYED> struct Shared : ByValue<KEYED> {
  unsigned long long bins[KEYED ? BINS : (LAST_BIN + THREADS) / THREADS * THREADS];      // whole rounds of all threads
  double table[STEPS];
  unsigned long long sums[WAVES];
  uint32_t words[WAVES];
  unsigned long long above;      // what lies above the bin that was found, and the bin
  uint32_t bin, count;
};

// The first bin in falling order of keys before which less than the limit lies and with which it is reached, or the last that holds anything: s.bin, s.above.
// value(i): what the i-th bin holds; PER of them a thread; above: what lies before all; limit(all): from what all hold.  Gives what all hold.
template <int PER, class S, class L, class F> __device__ __forceinline__ unsigned long long find_bin(S& s, unsigned long long above, L limit, F value) {
  unsigned long long held[PER], mine = 0, all;
  const int first = (int)threadIdx.x * PER;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    held[i] = value(first + i);
    mine += held[i];
  }
  unsigned long long at = above + before_me<unsigned long long>(mine, s.sums, all);
  const unsigned long long reached = limit(all);
  if (mine)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const unsigned long long n = held[i];
      if (n && at < reached && (at + n >= reached || at + n == above + all)) {
        s.bin = (uint32_t)(first + i);
        s.above = at;
      }
      at += n;
    }
  __syncthreads();
  return all;
}

// The logits of a row, as the waves have them: wave w has neighbouring tokens, lane l of it those of its words l, l + 64, .. of 16 bytes; up to 32 words a lane in
// registers (HELD), or read anew every time, 8 at once.
template <int DT, bool HELD> struct Row {
  typedef Type<DT> L;
  static constexpr int N = HELD ? MOST_WORDS : 8;
  typedef uint32_t Words __attribute__((ext_vector_type(N)));
  static constexpr int PER = L::PER;
  const char* x;           // aligned to 16 bytes, `skip` elements before the row
  __amdgpu_buffer_rsrc_t whole_words;      // from there on: what lies behind them is not read
  int skip, vocab, words;  // words of a lane
  int first;               // this lane's first word
  bool flat;               // the largest logit is +infinity: those that are it count as 0, the others as -infinity
  Words held[4];           // (a register of each word, by its number: read with an index that is the same in all lanes)
  float largest;           // of this lane
  __device__ __forceinline__ Row(const Args& a, int row) : vocab(a.vocab) {
    const char* const at = static_cast<const char*>(a.logits) + (int64_t)row * a.stride * L::SIZE;
    skip = (int)((uintptr_t)at & 15) / L::SIZE;
    x = at - skip * L::SIZE;
    whole_words = __builtin_amdgcn_make_buffer_rsrc((void*)x, 0, (vocab + skip) / PER * 16, 0x00027000);
    words = ((vocab + skip + PER - 1) / PER + THREADS - 1) / THREADS;
    first = (int)(threadIdx.x >> 6) * words * 64 + (int)(threadIdx.x & 63);
    flat = false;
    largest = NOTHING;
    if constexpr (HELD) {
      fill(held, 0, largest);
    } else {
      each_word([&](int, const uint4v& k) { larger(largest, k); });
    }
  }
  // This lane's words from v0 on, 8 loads under way at a time.
  static __device__ __forceinline__ void larger(float& most, const uint4v& r) {
#pragma unroll
    for (int e = 0; e < PER; ++e) most = __builtin_fmaxf(most, L::logit(r, e));
  }
  // ...; `most`: the largest of it and them
  __device__ __forceinline__ void fill(Words (&to)[4], int v0, float& most) const {
#pragma unroll
    for (int g = 0; g < N / 8; ++g) {
      uint4v r[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = (uint4v){L::NONE, L::NONE, L::NONE, L::NONE};
      if (v0 + 8 * g < words) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = load(first + 64 * (v0 + 8 * g + i));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          r[i] = v0 + 8 * g + i < words && whole(first + 64 * (v0 + 8 * g + i)) ? r[i] : (uint4v){L::NONE, L::NONE, L::NONE, L::NONE};
          larger(most, r[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) to[w][8 * g + i] = r[i][w];
    }
    // the row's first and last word, where they lie in it only in part
    const int last = (vocab + skip - 1) / PER;
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
      const int word = side ? last : 0, w0 = word / (words * 64), v = word % (words * 64) / 64 - v0;
      if ((int)(threadIdx.x >> 6) != w0 || v < 0 || v >= N || whole(word)) continue;
      const uint4v y = part(word);
      const bool mine = first + 64 * (v + v0) == word;
      if (mine) larger(most, y);
#pragma unroll
      for (int w = 0; w < 4; ++w) to[w][v] = mine ? y[w] : to[w][v];
    }
  }
  // 16 bytes that lie in the row; that do in part (what does not is -infinity); that do not
  __device__ __forceinline__ bool whole(int word) const { return word * PER >= skip && word * PER - skip + PER <= vocab; }
  __device__ __forceinline__ bool some(int word) const { return word * PER - skip + PER > 0 && word * PER - skip < vocab; }
  __device__ __forceinline__ uint4v load(int word) const {      // (zeros where it does not lie in the row, or only its end does not)
    return __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(whole_words, word * PER >= skip ? word * 16 : 1 << 30, 0, 0));
  }
  __device__ __forceinline__ uint4v part(int word) const {
    uint4v r = {L::NONE, L::NONE, L::NONE, L::NONE};
    const int i = word * PER - skip;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      if (i + e < 0 || i + e >= vocab) continue;
      if constexpr (L::WIDE) r[e] = reinterpret_cast<const uint32_t*>(x)[(int64_t)word * PER + e];
      else r[e >> 1] = (r[e >> 1] & ~(0xFFFFu << 16 * (e & 1))) | (uint32_t)reinterpret_cast<const uint16_t*>(x)[(int64_t)word * PER + e] << 16 * (e & 1);
    }
    return r;
  }
  // f(v, word) for every word of this lane
  template <class F> __device__ __forceinline__ void each_word(F f) const {
    if constexpr (HELD) {
#pragma unroll 1
      for (int v = 0; v < words; ++v) f(v, at(v));
    } else {
#pragma unroll 1
      for (int v0 = 0; v0 < words; v0 += N) {
        Words read[4];
        float unused = NOTHING;
        fill(read, v0, unused);
        const int end = words - v0 < N ? words - v0 : N;
#pragma unroll 1
        for (int v = 0; v < end; ++v) f(v0 + v, flattened(uint4v{read[0][v], read[1][v], read[2][v], read[3][v]}));
      }
    }
  }
  // This lane's v-th word, where they are held.
  __device__ __forceinline__ uint4v at(int v) const { return flattened(uint4v{held[0][v], held[1][v], held[2][v], held[3][v]}); }
  // Four words, 64 apart, from memory; those from `end` on are not looked at.
  __device__ __forceinline__ void four_words(int word, int end, uint4v (&k)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) k[i] = load(word + 64 * i);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (word + 64 * i < end && !whole(word + 64 * i)) k[i] = part(word + 64 * i);
      k[i] = flattened(k[i]);
    }
  }
  __device__ __forceinline__ uint4v flattened(uint4v r) const {
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(flat), 0)) {
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const bool is = L::logit(r, e) == -NOTHING;
        if constexpr (L::WIDE) r[e] = is ? 0u : L::NONE;
        else r[e >> 1] = (r[e >> 1] & ~(0xFFFFu << 16 * (e & 1))) | (is ? 0u : L::NONE & 0xFFFFu << 16 * (e & 1));
      }
    }
    return r;
  }
  template <class F> __device__ __forceinline__ void each(F f) const {
    each_word([&](int, const uint4v& r) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < PER; ++e) f(L::logit(r, e));
    });
  }
  __device__ __forceinline__ int token(int v, int e) const { return (first + 64 * v) * PER + e - skip; }
};

// What the rules have left: logits above `border`, and the first `equal` of those that are it.
struct Kept {
  float border;
  int equal;
};
// The number below x, and the least that is not below a number of 64 bits.
__device__ __forceinline__ float below(float x) {
  const uint32_t u = as_u(x + 0.f);
  return as_f(u == 0 ? 0x80000001u : u & 0x80000000u ? u + 1 : u - 1);
}
__device__ __forceinline__ float not_below(double x) {
  const float y = (float)x;
  return (double)y >= x ? y : -below(-y);
}

template <int DT, bool HELD>
__global__ __launch_bounds__(THREADS) void ftsample_row(const Args a) {
  typedef Type<DT> L;
  constexpr bool KEYED = DT == FTSAMPLE_BF16;
  __shared__ Shared<KEYED> s;
  constexpr int LIST = KEYED ? THREADS : 2 * THREADS;      // logits that are sorted
  __shared__ unsigned long long list[LIST];      // (under top_k) key and place, then weights by place
  __shared__ int listed[LIST];
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Rules r = rules_of(a, row);
  Row<DT, HELD> x(a, row);
  for (int i = tid; i < STEPS; i += THREADS) s.table[i] = __builtin_ldexp(exp2((double)i / STEPS), a.shift);

  float mine = x.largest;
  float most = wave_most(mine);
  if (lane == 0) s.words[wave] = as_u(most);
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) most = __builtin_fmaxf(most, as_f(s.words[w]));
  auto answer = [&](int token, double chance) {
    a.tokens[row] = token;
    if (a.probability) a.probability[row] = (float)chance;
  };
  if (!(most > NOTHING)) {
    if (tid == 0) answer(-1, 0.0);
    return;
  }
  if (most == -NOTHING) {
    x.flat = true;
    most = 0.f;
    mine = mine == -NOTHING ? 0.f : NOTHING;
  }
  if (r.top_k == 1) {      // the first that is as large
    int token = 0x7FFFFFFF;
    x.each_word([&](int v, const uint4v& k) __attribute__((always_inline)) {
#pragma unroll
      for (int e = L::PER - 1; e >= 0; --e) {
        const int t = x.token(v, e);
        token = L::logit(k, e) == most && t < token ? t : token;
      }
    });
#pragma unroll
    for (int d = 32; d; d >>= 1) {
      const int y = __shfl_xor(token, d);
      token = y < token ? y : token;
    }
    __syncthreads();
    if (lane == 0) s.words[wave] = (uint32_t)token;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < WAVES; ++w) token = (int)s.words[w] < token ? (int)s.words[w] : token;
      answer(token, 1.0);
    }
    return;
  }
  const double scale = r.per_t * (STEPS / 0.69314718055994530942);
  const Weights weights{scale, (double)most, -(STEPS * OCTAVES + 0.25) / scale, s.table};
  auto weight = [&](float y) __attribute__((always_inline)) {
    int bin;
    return weights.of(y, bin);
  };
  // the least logit that min_p keeps: its weight is at least the floor
  const float least = r.floor >= 1.0 ? most : r.floor > 0.0 ? not_below((double)most + log(r.floor) / r.per_t) : NOTHING;
  auto limit_of = [&](unsigned long long all) -> unsigned long long {      // the least whole number that is top_p of all, or 1
    const double limit = __builtin_ceil(r.top_p * (double)all);
    return limit >= 1.0 ? (unsigned long long)limit : 1ull;
  };

  // Logits of bf16 by their value.
  int base = 0;
  if constexpr (KEYED) {
    const float low = most + (float)weights.least, far = __builtin_fmaxf(__builtin_fabsf(most), __builtin_fabsf(low));
    const int octave = (int)(as_u(far) >> 23) + 2;      // (one more than holds `far`: `low` is rounded)
    base = (octave < 255 ? octave : 255) * 128 - MAGNITUDES;
    base = base > 0 ? base : 0;
  }
  // The numbers of a word's logits, two in a word and times UNIT; whether one is tiny, and (at_ends) whether one is at either end.
  auto numbers_of = [&](auto unit, const uint4v& k, uint32_t (&pair)[4], bool& at_ends) __attribute__((always_inline)) {
    constexpr uint16_t UNIT = decltype(unit)::value;
    ushort2v furthest = {0, 0};
    uint32_t signs = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = k[i];
      const ushort2v at = __builtin_bit_cast(ushort2v, u & 0x7FFF7FFFu) - (ushort2v)(uint16_t)base, in = __builtin_elementwise_min(at, (ushort2v)(uint16_t)MAGNITUDES);
      furthest = __builtin_elementwise_max(furthest, at);
      signs |= __builtin_bit_cast(uint32_t, at);
      const ushort2v number = in ^ __builtin_bit_cast(ushort2v, __builtin_bit_cast(short2v, u) >> (short2v)(short)15);
      pair[i] = __builtin_bit_cast(uint32_t, number * (ushort2v)UNIT + (ushort2v)(uint16_t)((MAGNITUDES + 1) * UNIT));
    }
    at_ends = furthest[0] >= MAGNITUDES || furthest[1] >= MAGNITUDES;
    return (signs & 0x80008000u) != 0;      // (magnitudes and `base` are below 2^15)
  };
  auto tiny = [&](float y) { return (int)(as_u(y) >> 16 & 0x7FFF) < base; };
  auto value_of = [&](int number) {      // (not of those at either end)
    const int at = number - (MAGNITUDES + 1), magnitude = (at < 0 ? -at - 1 : at) + base;
    return as_f((uint32_t)magnitude << 16 | (at < 0 ? 0x80000000u : 0u));
  };
  bool worth_known = false;
  auto know_worth = [&]() {
    if constexpr (KEYED) {
      if (worth_known) return;
#pragma unroll 4
      for (int i = tid; i < VALUES; i += THREADS) s.worth[i] = weight(value_of(i));
      if (tid == 0) s.worth[0] = 0;
      if (tid == (VALUES - 1) % THREADS) s.worth[VALUES - 1] = 0;
      worth_known = true;
    }
  };
  // What the logits of a word that lie above the border add to the sum.
  auto worths = [&](const uint4v& k, float border, unsigned long long (&w)[L::PER]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < L::PER; ++e) {
      const float y = L::logit(k, e);
      w[e] = weight(y);
      w[e] = y > border ? w[e] : 0;
    }
  };

  // The first place at which the sum of kept weights exceeds u times all: whole numbers exceed it where they reach the next one.  Lane g has of this wave's g-th run of `per` words
  // the kept weights without those of the border, and how many logits are the border.
  auto choose = [&](const Kept& kept, int per, unsigned long long sum, uint32_t ties) {
    const unsigned long long worth = kept.equal ? weight(kept.border) : 0, sums = sum_upto(sum);
    const uint32_t tied = sum_upto(ties);
    __syncthreads();
    if (lane == 63) {
      s.sums[wave] = sums;
      s.words[wave] = tied;
    }
    __syncthreads();
    unsigned long long all = 0, before = 0;
    int left = kept.equal, left_here = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      if (w == wave) {
        before = all;
        left_here = left;
      }
      const int n = (int)s.words[w] < left ? (int)s.words[w] : left;
      all += s.sums[w] + (unsigned long long)n * worth;
      left -= n;
    }
    const unsigned long long goal = (unsigned long long)__builtin_floor(r.u * (double)all) + 1;
    // the run in which it lies, of one lane of one wave
    left = left_here - (int)(tied - ties);
    left = left > 0 ? left : 0;
    before += sums - sum + (unsigned long long)(left_here - left) * worth;
    const unsigned long long here = sum + (unsigned long long)((int)ties < left ? (int)ties : left) * worth;
    const uint64_t found = __ballot(before < goal && before + here >= goal);
    if (!found) return;
    const int run = __builtin_ctzll(found), end = (run + 1) * per < x.words ? (run + 1) * per : x.words;
    before = (unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(before >> 32), run) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)before, run);
    left = __builtin_amdgcn_readlane(left, run);
    uint4v ahead[4];
#pragma unroll 1
    for (int v = run * per; v < end; ++v) {
      uint4v k;
      if constexpr (HELD) {
        k = x.at(v);
      } else {
        if ((v - run * per) % 4 == 0) x.four_words(x.first + 64 * v, x.first - lane + 64 * end, ahead);
        k = ahead[0];
        ahead[0] = ahead[1];
        ahead[1] = ahead[2];
        ahead[2] = ahead[3];
      }
      unsigned long long w[L::PER];
      worths(k, kept.border, w);
      sum = 0;
      ties = 0;
#pragma unroll
      for (int e = 0; e < L::PER; ++e) {
        ties += kept.equal && L::logit(k, e) == kept.border;
        sum += w[e];
      }
      if (kept.equal && __any(ties != 0)) {
        // those of the border that are left, in the order of their tokens
        const uint32_t upto = sum_upto(ties);
        int mine = left - (int)(upto - ties);
#pragma unroll
        for (int e = 0; e < L::PER; ++e)
          if (L::logit(k, e) == kept.border && mine-- > 0) {
            w[e] = worth;
            sum += worth;
          }
        const int all_n = (int)last_lane(upto);
        left -= all_n < left ? all_n : left;
      }
      const unsigned long long upto = sum_upto(sum);
      unsigned long long at = before + upto - sum;
      if (at < goal && at + sum >= goal)
#pragma unroll
        for (int e = 0; e < L::PER; ++e) {
          if (at < goal && at + w[e] >= goal) answer(x.token(v, e), (double)w[e] / (double)all);
          at += w[e];
        }
      before += last_lane(upto);
      if (before >= goal) return;
    }
  };
  auto sum_up = [&](Kept kept) {
    if (least > kept.border) kept = Kept{below(least), 0};
    if constexpr (KEYED) {
      know_worth();
      __syncthreads();
      if (kept.border > NOTHING) {
        for (int i = tid; i < VALUES; i += THREADS) {
          const float y = value_of(i);
          if (!(y > kept.border)) s.worth[i] = y == kept.border ? 1ull << TIE : 0;
        }
        __syncthreads();
      }
    }
    const int per = x.words <= 4 * 64 ? 4 : (x.words + 63) / 64;      // of a run
    unsigned long long sum = 0, sum_of_run = 0;
    uint32_t ties = 0, ties_of_run = 0;
    int run = 0, in_run = 0;
    x.each_word([&](int v, const uint4v& k) __attribute__((always_inline)) {
      if constexpr (KEYED) {
        uint32_t pair[4];
        bool at_ends;
        const bool some = numbers_of(std::integral_constant<uint16_t, 8>{}, k, pair, at_ends);
#pragma unroll
        for (int e = 0; e < L::PER; ++e)
          sum += *reinterpret_cast<const unsigned long long*>(reinterpret_cast<const char*>(s.worth) + (e & 1 ? pair[e >> 1] >> 16 : pair[e >> 1] & 0xFFFFu));
        if (__any(some))
#pragma unroll
          for (int e = 0; e < L::PER; ++e) {
            const float y = L::logit(k, e);
            if (tiny(y) && y >= kept.border) sum += y == kept.border ? 1ull << TIE : weight(y);
          }
      } else {
        float largest = NOTHING;
        x.larger(largest, k);
        if (kept.border == NOTHING || __any(largest >= kept.border)) {
          unsigned long long w[L::PER];
          worths(k, kept.border, w);
#pragma unroll
          for (int e = 0; e < L::PER; ++e) sum += w[e];
          if (kept.equal)
#pragma unroll
            for (int e = 0; e < L::PER; ++e) ties += L::logit(k, e) == kept.border;
        }
      }
      if (++in_run == per || v + 1 == x.words) {
        if constexpr (KEYED) {
          ties = (uint32_t)(sum >> TIE);
          sum &= (1ull << TIE) - 1;
        }
        sum = wave_sum(sum);
        sum_of_run = lane == run ? sum : sum_of_run;
        if (kept.equal) {
          ties = wave_sum(ties);
          ties_of_run = lane == run ? ties : ties_of_run;
        }
        ++run;
        sum = 0;
        ties = in_run = 0;
      }
    });
    choose(kept, per, sum_of_run, ties_of_run);
  };

  // The border moves up to the lowest logit above which less than `limit` lies, by counts or by sums of weights; among those with keys lowest .. highest, above which `above` lies.
  Kept kept{NOTHING, 0};
  const uint32_t top_key = L::key(most);
  auto empty_bins = [&]() {
    __syncthreads();
    for (int i = tid; i < BINS; i += THREADS) s.bins[i] = 0;
    __syncthreads();
  };
  // after bins of keys highest - k >> drop are filled; counted: with numbers of logits of one key each, which have a weight
  auto narrow = [&](uint32_t& lowest, uint32_t& highest, int drop, bool counted, unsigned long long& above, unsigned long long limit) {
    __syncthreads();
    if (counted) {
      for (int i = tid; i < BINS; i += THREADS)
        if (s.bins[i]) s.bins[i] *= weight(L::of_key(highest - i));
      __syncthreads();
    }
    if (find_bin<BINS / THREADS>(s, above, [&](unsigned long long) { return limit; }, [&](int i) { return s.bins[i]; }) == 0) return false;
    above = s.above;
    const uint32_t top = highest - (s.bin << drop), least = top - ((1u << drop) - 1);
    lowest = least > lowest && least <= top ? least : lowest;
    highest = top;
    return true;
  };
  auto drop_of = [](uint32_t range) {
    const int bits = 32 - __builtin_clz(range);
    return bits > BITS ? bits - BITS : 0;
  };
  auto search = [&](unsigned long long limit, bool by_weight, uint32_t lowest, uint32_t highest, unsigned long long above) {
    while (lowest != highest) {
      const int drop = drop_of(highest - lowest);
      const float from = L::of_key(lowest), to = L::upto_key(highest);
      empty_bins();
      const bool counted = by_weight && drop == 0;
      auto fill = [&](auto value) __attribute__((always_inline)) {
        x.each_word([&](int, const uint4v& k) __attribute__((always_inline)) {
#pragma unroll
          for (int e = 0; e < L::PER; ++e) {
            const float y = L::logit(k, e);
            if (y >= from && y <= to && y > kept.border) atomicAdd(&s.bins[(highest - L::key(y)) >> drop], value(y));
          }
        });
        __syncthreads();
        // (the kept ones of the border that there is)
        if (tid == 0 && kept.equal && kept.border >= from && kept.border <= to) s.bins[(highest - L::key(kept.border)) >> drop] += value(kept.border) * (unsigned)kept.equal;
      };
      if (by_weight && !counted) fill(weight);
      else fill([](float) { return 1ull; });
      if (!narrow(lowest, highest, drop, counted, above, limit)) return;      // (none lies there)
    }
    // of the logits that are the border, as many as fit
    const float border = L::of_key(lowest);
    const unsigned long long each = by_weight ? weight(border) : 1;
    unsigned long long fit = each ? (limit - above + each - 1) / each : 0x7FFFFFFFull;
    if (border == kept.border && (unsigned long long)kept.equal < fit) fit = kept.equal;
    kept.border = border;
    kept.equal = (int)(fit > 0x7FFFFFFFull ? 0x7FFFFFFFull : fit);
  };
  const uint32_t least_key = L::key(NOTHING) + 1;
  // The list's `count` entries in falling order: e[0] the tid-th, e[1] (`large`: there may be more than 512) the (tid + 512)-th.
  auto sort_list = [&](auto large, int count, unsigned long long (&e)[2]) {
    const bool two = decltype(large)::value && count > THREADS;
    e[0] = tid < count ? list[tid] : 0;
    e[1] = two && tid + THREADS < count ? list[tid + THREADS] : 0;
    auto exchange = [&](int j, int k) {
      __syncthreads();
      list[tid] = e[0];
      if (two) list[tid + THREADS] = e[1];
      __syncthreads();
      const bool first = (tid & j) == 0;
      const unsigned long long other = list[tid ^ j];
      e[0] = (first == ((tid & k) == 0)) == (other > e[0]) ? other : e[0];
      if (two) {
        const unsigned long long above = list[(tid ^ j) + THREADS];
        e[1] = (first == ((tid + THREADS & k) == 0)) == (above > e[1]) ? above : e[1];
      }
    };
    sort_wave(e[0], tid);
    if (two) sort_wave(e[1], tid + THREADS);
    for (int k = 128; k < 2 * count && k <= LIST; k <<= 1) {
      if (two && k == LIST) {
        const unsigned long long larger = e[0] > e[1] ? e[0] : e[1];
        e[1] = e[0] > e[1] ? e[1] : e[0];
        e[0] = larger;
      }
      for (int j = two && k == LIST ? THREADS / 2 : k >> 1; j >= 64; j >>= 1) exchange(j, k);
      merge<32>(e[0], tid, k);
      if (two) merge<32>(e[1], tid + THREADS, k);
    }
  };
  // The same for all that is kept, the bin of the weights' logarithm first; limit: from the sum of all.
  auto by_bins = [&](bool by_weight, auto limit_from) {
    constexpr int N = sizeof(s.bins) / sizeof(s.bins[0]);
    __syncthreads();
    for (int i = tid; i < N; i += THREADS) s.bins[i] = 0;
    __syncthreads();
    uint32_t beyond = 0;
    x.each_word([&](int, const uint4v& k) __attribute__((always_inline)) {
      unsigned long long w[L::PER];
      int bin[L::PER];
      if (by_weight) {
#pragma unroll
        for (int e = 0; e < L::PER; ++e) w[e] = weights.of(L::logit(k, e), bin[e]);
      } else {
#pragma unroll
        for (int e = 0; e < L::PER; ++e) {
          bin[e] = weights.bin(L::logit(k, e));
          w[e] = 1;
          beyond += bin[e] == LAST_BIN && L::logit(k, e) > NOTHING;
        }
      }
#pragma unroll
      for (int e = 0; e < L::PER; ++e)
        if (L::logit(k, e) > kept.border && w[e] && bin[e] < LAST_BIN) atomicAdd(&s.bins[bin[e]], w[e]);
    });
    __syncthreads();
    // (what is in the last bin is not counted there: thousands of logits may lie so far below, and would be added up one after the other)
    if (tid == 0 && kept.equal) s.bins[weights.bin(kept.border)] += (by_weight ? weight(kept.border) : 1ull) * (unsigned)kept.equal;
    __syncthreads();
    unsigned long long limit = 0;
    const unsigned long long all = find_bin<N / THREADS>(s, 0, [&](unsigned long long all) { return limit = limit_from(all); }, [&](int i) { return s.bins[i]; });
    int bin = LAST_BIN;
    unsigned long long above = all;
    if (all < limit && !by_weight) {
      uint32_t beyond_all;
      before_me<uint32_t>(beyond, s.words, beyond_all);
      if (all + beyond_all <= limit) return;      // no more than that can be chosen: all of them are kept
    } else {
      bin = (int)s.bin;
      above = s.above;
    }
    // The keys of that bin: those from the first that lies in it or above on, up to before the first that lies above.  64 keys at a time are tried, one a lane.
    auto first_key = [&](int last) {      // ... whose bin is at most `last`: one of n from `from` on
      uint32_t from = least_key, n = top_key - least_key + 1;      // (top_key's bin is 0)
      while (n > 1) {
        const uint32_t step = (n + 63) >> 6;
        const uint64_t at = (uint64_t)lane * step;
        const int low = __popcll(__ballot(at < n && weights.bin(L::of_key(from + (uint32_t)at)) > last));      // the first `low` of the lanes' keys lie below
        if (low == 0) break;
        const uint32_t passed = (uint32_t)(low - 1) * step + 1;
        from += passed;
        n = n - passed < step ? n - passed : step;
      }
      return from;
    };
    const uint32_t lowest = bin == LAST_BIN ? least_key : first_key(bin), highest = bin == 0 ? top_key : first_key(bin - 1) - 1;
    // Few logits of 32 bits lie there, as a rule: they are sorted.  (Of 16 bits many are equal.)
    const float from = L::of_key(lowest), to = L::upto_key(highest);
    if (L::WIDE && !(kept.equal && kept.border >= from && kept.border <= to)) {
      if (tid == 0) s.count = 0;
      __syncthreads();
      x.each([&](float y) __attribute__((always_inline)) {
        if (y >= from && y <= to && y > kept.border) {
          const uint32_t at = atomicAdd(&s.count, 1u);
          if (at < THREADS) list[at] = (unsigned long long)L::key(y) << 32;
        }
      });
      __syncthreads();
      const int count = (int)s.count;
      if (count > 0 && count <= THREADS) {
        unsigned long long e[2];
        sort_list(std::false_type{}, count, e);
        const uint32_t key = (uint32_t)(e[0] >> 32);
        const unsigned long long each = tid >= count ? 0 : by_weight ? weight(L::of_key(key)) : 1;
        unsigned long long all_here;
        const unsigned long long at = above + before_me<unsigned long long>(each, s.sums, all_here);
        if (at < limit && (at + each >= limit || tid == count - 1)) {
          s.bin = (uint32_t)tid;
          s.words[0] = key;
        }
        __syncthreads();
        const uint32_t border = s.words[0], last = s.bin;
        uint32_t equal;
        before_me<uint32_t>(key == border && tid <= (int)last, s.words, equal);
        kept.border = L::of_key(border);
        kept.equal = (int)equal;
        return;
      }
    }
    search(limit, by_weight, lowest, highest, above);
  };

  // The same for bf16: how many there are of each value tells the border of all limits.
  constexpr int IN_ORDER = ((2 * MAGNITUDES + THREADS) / THREADS | 1) * THREADS;      // (of a thread an odd number: they lie in different banks)
  bool counted = false;
  uint32_t tiny_count = 0;
  unsigned long long tiny_sum = 0;      // of this thread
  auto by_values = [&](bool by_weight, auto limit_from) {
    if constexpr (KEYED) {
      const bool anew = kept.border > NOTHING && tiny(kept.border);
      if (!counted) {
        __syncthreads();
        for (int i = tid; i < VALUES; i += THREADS) s.counts[i] = 0;
        __syncthreads();
      }
      if (!counted || anew) {
        tiny_count = 0;
        tiny_sum = 0;
        x.each_word([&](int, const uint4v& k) __attribute__((always_inline)) {
          uint32_t pair[4];
          bool at_ends;
          const bool some = numbers_of(std::integral_constant<uint16_t, 4>{}, k, pair, at_ends), checked = __any(at_ends);
          if (!counted)
#pragma unroll
            for (int e = 0; e < L::PER; ++e) {
              const uint32_t at = e & 1 ? pair[e >> 1] >> 16 : pair[e >> 1] & 0xFFFFu;
              if (!checked || at - 4 < 4 * (VALUES - 2)) atomicAdd(reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(s.counts) + at), 1u);
            }
          if (__any(some))
#pragma unroll
            for (int e = 0; e < L::PER; ++e) {
              const float y = L::logit(k, e);
              if (tiny(y) && y > kept.border) {
                ++tiny_count;
                tiny_sum += weight(y);
              }
            }
        });
        __syncthreads();
        counted = true;
      }
      // In falling order: positive ones, tiny ones, negative ones.
      auto number_at = [&](int i) { return i < MAGNITUDES ? VALUES - 2 - i : VALUES - 1 - i; };
      unsigned long long all_tiny = 0;
      if (!(kept.border > 0.f && !tiny(kept.border))) before_me<unsigned long long>(by_weight ? tiny_sum : tiny_count, s.sums, all_tiny);
      if (anew) all_tiny += (by_weight ? weight(kept.border) : 1ull) * (unsigned)kept.equal;
      auto at = [&](int i) -> unsigned long long {
        const int number = i > 2 * MAGNITUDES ? 0 : number_at(i);      // (number 0 has no weight, and is not counted)
        const float y = value_of(number);
        uint32_t n = s.counts[number];
        if (base == 0 && number == MAGNITUDES + 1) n += s.counts[MAGNITUDES];      // (both zeros are one)
        n = base == 0 && number == MAGNITUDES ? 0 : y > kept.border ? n : y == kept.border && n ? (uint32_t)kept.equal : 0;
        const unsigned long long all_of_it = by_weight ? s.worth[number] * n : n;
        return i == MAGNITUDES ? all_tiny : all_of_it;
      };
      if (by_weight) know_worth();
      __syncthreads();
      unsigned long long limit = 0;
      const unsigned long long all = find_bin<IN_ORDER / THREADS>(s, 0, [&](unsigned long long all) { return limit = limit_from(all); }, at);
      if (all < limit) return;      // fewer than that have a weight: all of them are kept
      const int bin = (int)s.bin;
      const uint32_t one = bin == MAGNITUDES ? 0 : L::key(value_of(number_at(bin))), far = (uint32_t)(base - 1) << 16;
      search(limit, by_weight, bin == MAGNITUDES ? L::key(as_f(far | 0x80000000u)) : one, bin == MAGNITUDES ? L::key(as_f(far)) : one, s.above);
    } else {
      by_bins(by_weight, limit_from);
    }
  };

  // With top_k all that is left may be few: logits from `from` on, top_k or more of them, are sorted.  False: they are too many.
  auto by_list = [&](auto large, float from) {
    constexpr int ROOM = decltype(large)::value ? 2 * THREADS : THREADS;
    uint32_t n = 0;
    x.each([&](float y) __attribute__((always_inline)) { n += y >= from; });
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
    if (count > ROOM) return false;
    // the logits in the order of their tokens: (key, place) in the list, tokens by place
    if (in_wave)
      x.each_word([&](int v, const uint4v& k) {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < L::PER; ++e) m += L::logit(k, e) >= from;
        if (!__any(m != 0)) return;
        const uint32_t upto = sum_upto(m);
        uint32_t place = at + upto - m;
#pragma unroll
        for (int e = 0; e < L::PER; ++e) {
          const float y = L::logit(k, e);
          if (!(y >= from)) continue;
          list[place] = (unsigned long long)L::key(y) << 32 | (0xFFFFFFFFu - place);
          listed[place] = x.token(v, e);
          ++place;
        }
        at += last_lane(upto);
      });
    __syncthreads();
    unsigned long long e[2], w[2], before[2], all, more = 0;
    sort_list(large, (int)count, e);
    const bool two = decltype(large)::value && count > THREADS;
    // Sums in the order of w; both halves' sums of up to before this thread's.
    auto sum_all = [&]() {
      before[0] = before_me<unsigned long long>(w[0], s.sums, all);
      if (two) {
        before[1] = all + before_me<unsigned long long>(w[1], s.sums, more);
        all += more;
      }
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = tid + i * THREADS < (int)count && tid + i * THREADS < r.top_k ? weight(L::of_key((uint32_t)(e[i] >> 32))) : 0;
    sum_all();
    const unsigned long long limit = limit_of(all);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (tid + i * THREADS > 0 && (L::of_key((uint32_t)(e[i] >> 32)) < least || (r.cut_p && w[i] && before[i] >= limit))) w[i] = 0;
    __syncthreads();
    list[tid] = 0;
    if (two) list[tid + THREADS] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (w[i]) list[0xFFFFFFFFu - (uint32_t)e[i]] = w[i];
    __syncthreads();
    // and summed up in the order of their tokens
    w[0] = list[tid];
    w[1] = two ? list[tid + THREADS] : 0;
    sum_all();
    const unsigned long long goal = (unsigned long long)__builtin_floor(r.u * (double)all) + 1;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (w[i] && before[i] < goal && before[i] + w[i] >= goal) answer(listed[tid + i * THREADS], (double)w[i] / (double)all);
    return true;
  };

  if (r.top_k < x.vocab) {
    float from = NOTHING;
    if (r.top_k <= MOST_BOUNDED) {
      // A bound that at least top_k logits reach (or all that can be chosen): of every wave's 64 maxima the (top_k / 8)-th largest, of these the smallest.
      float sorted = mine;
      sort_wave(sorted, lane);
      const float mine_of_wave = as_f((uint32_t)__builtin_amdgcn_readlane((int)as_u(sorted), (r.top_k + WAVES - 1) / WAVES - 1));
      __syncthreads();
      if (lane == 0) s.words[wave] = as_u(mine_of_wave);
      __syncthreads();
      from = as_f(s.words[0]);
#pragma unroll
      for (int w = 1; w < WAVES; ++w) from = __builtin_fminf(from, as_f(s.words[w]));
      from = __builtin_fmaxf(from, L::of_key(least_key));      // (where fewer can be chosen)
    }
    if (from > NOTHING && by_list(std::false_type{}, from)) return;
    // With a larger top_k, or where too many reach the bound, the border itself comes first.
    by_values(false, [&](unsigned long long) { return (unsigned long long)r.top_k; });
    // (sorted where they are few, not weighed a second time: 48 rows of 50,001 in fp32 with all rules 41 us, else 61; 512 of 65,536 in fp16 68 to 76, 86.  In bf16 values are
    // counted already, and the sort takes 10 us more.)
    if constexpr (!KEYED)
      if (r.cut_p && r.top_k <= LIST && kept.border > NOTHING && by_list(std::true_type{}, kept.border)) return;
  }
  if (r.cut_p) by_values(true, limit_of);
  sum_up(kept);
}

typedef void (*kernel_fn)(const Args);
// The kernel of a vocabulary: rows in registers where they fit; `skip`: most elements between a word of 16 bytes and the row that begins in it.
template <int DT> kernel_fn kernel_of(int vocab, int skip) {
  return (vocab + skip + Type<DT>::PER - 1) / Type<DT>::PER <= MOST_WORDS * THREADS ? ftsample_row<DT, true> : ftsample_row<DT, false>;
}

}  // namespace ftsample

using namespace ftsample;

struct ftsample_ctx {
  ftsample_config cfg;
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
  const int size = e.in_dtype == FTSAMPLE_F32 ? 4 : 2, skip = ((uintptr_t)logits | (uintptr_t)(row_stride * size)) % 16 ? 16 / size - 1 : 0;
  const kernel_fn fn = e.in_dtype == FTSAMPLE_F32 ? kernel_of<FTSAMPLE_F32>(e.vocab, skip) : e.in_dtype == FTSAMPLE_BF16 ? kernel_of<FTSAMPLE_BF16>(e.vocab, skip) : kernel_of<FTSAMPLE_F16>(e.vocab, skip);
  hipLaunchKernelGGL(fn, dim3((uint32_t)rows), dim3(THREADS), 0, (hipStream_t)hip_stream, a);
  he = hipGetLastError();
  if (before != e.device) (void)hipSetDevice(before);
  return he == hipSuccess ? FTSAMPLE_OK : sfail_hip(c, "launch", he);
}

extern "C" int ftsample_destroy(ftsample_ctx* c) {
  delete c;
  return FTSAMPLE_OK;
}

extern "C" const char* ftsample_last_error(const ftsample_ctx* c) { return c ? c->err.c_str() : g_sample_create_err.c_str(); }
