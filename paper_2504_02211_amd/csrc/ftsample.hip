// Choice of the next token from its logits: the kernels and the C ABI of ../include/ftsample.h.
//
// A workgroup takes a row.  Every logit has a key, a whole number that is ordered as the logits are; what the rules keep is "the keys above one key, and the first
// of those equal to it", so top_k and top_p are searches for that key: a histogram of the leading bits of the keys (counts for top_k, weights for top_p), then of
// the next bits of those with the same leading bits, until one key is left.  Then the kept weights are summed in the order of the vocabulary.
// Weights are formed in 64 bits and summed as whole numbers: a sum in 32 bits is off by more than the borders between neighbouring tokens are apart, and one of 64-bit floating-point numbers
// depends on the order of its terms.
#include "ftsample.h"
#include "ftserve_device.h"

#include <cmath>
#include <new>
#include <string>

namespace ftsample {
using namespace ftserve;

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int BITS = 11, BINS = 1 << BITS;      // of a level of the search

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

template <int DT> __device__ __forceinline__ float logit(const void* row, int i) {
  if constexpr (DT == FTSAMPLE_F32) return reinterpret_cast<const float*>(row)[i];
  else if constexpr (DT == FTSAMPLE_BF16) return as_f((uint32_t)reinterpret_cast<const uint16_t*>(row)[i] << 16);
  else return (float)reinterpret_cast<const _Float16*>(row)[i];
}

// Keys are ordered as their logits; both zeros have the same.  -infinity and NaN have 0, which nothing keeps.
__device__ __forceinline__ uint32_t key_of(float x) {
  if (!(x > -__builtin_inff())) return 0;
  const uint32_t u = as_u(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return as_f(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }

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

// The weight of a key that is not 0, given the largest one (whose logit may be +infinity).
constexpr uint32_t KEY_INFINITY = 0xFF800000u;
__device__ __forceinline__ double weight_of(uint32_t key, uint32_t most, double per_t) {
  return key == most ? 1.0 : most == KEY_INFINITY ? 0.0 : exp(((double)of_key(key) - (double)of_key(most)) * per_t);
}
__device__ __forceinline__ uint64_t whole(double w, int shift) { return (uint64_t)__builtin_rint(__builtin_ldexp(w, shift)); }

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

struct Shared {
  unsigned long long bins[BINS];
  unsigned long long sums[WAVES];
  uint32_t words[WAVES];
  unsigned long long above;      // what lies above the bin that was found, and the bin
  uint32_t bin;
  int token;
  double chance;
};

// The lowest bin above which less than `limit` lies (in all, not in the histogram alone): s.bin, s.above.
__device__ __forceinline__ void find_bin(Shared& s, unsigned long long above, unsigned long long limit) {
  constexpr int PER = BINS / THREADS;
  unsigned long long mine = 0, all;
  const int first = (THREADS - 1 - (int)threadIdx.x) * PER;      // thread 0 has the highest bins
  for (int i = 0; i < PER; ++i) mine += s.bins[first + i];
  unsigned long long at = above + before_me<unsigned long long>(mine, s.sums, all);
  for (int i = PER - 1; i >= 0; --i) {
    const unsigned long long n = s.bins[first + i];
    if (n && at < limit && (at + n >= limit || at + n == above + all)) {
      s.bin = (uint32_t)(first + i);
      s.above = at;
    }
    at += n;
  }
  __syncthreads();
}

template <int DT>
__global__ __launch_bounds__(THREADS) void ftsample_row(const Args a) {
  __shared__ Shared s;
  const int row = blockIdx.x, tid = threadIdx.x, vocab = a.vocab;
  const void* const x = static_cast<const char*>(a.logits) + (int64_t)row * a.stride * (DT == FTSAMPLE_F32 ? 4 : 2);
  const Rules r = rules_of(a, row);
  auto key_at = [&](int i) { return key_of(logit<DT>(x, i)); };

  uint32_t most = 0;
  for (int i = tid; i < vocab; i += THREADS) {
    const uint32_t k = key_at(i);
    most = k > most ? k : most;
  }
  for (int d = 32; d; d >>= 1) {
    const uint32_t y = __shfl_xor(most, d);
    most = y > most ? y : most;
  }
  if ((tid & 63) == 0) s.words[tid >> 6] = most;
  __syncthreads();
  for (int w = 0; w < WAVES; ++w) most = s.words[w] > most ? s.words[w] : most;
  if (most == 0) {
    if (tid == 0) {
      a.tokens[row] = -1;
      if (a.probability) a.probability[row] = 0.f;
    }
    return;
  }
  auto weight = [&](uint32_t k) { return weight_of(k, most, r.per_t); };

  // kept: keys above `border`, and the first `equal` of those that are it
  uint32_t border = 0;
  int equal = 0;
  // by_weight: by sums of weights instead of counts.  The border moves up to the lowest key above which less than `limit` lies.
  auto search = [&](unsigned long long limit, bool by_weight) {
    uint32_t prefix = 0;
    unsigned long long above = 0;
    for (int left = 32; left > 0;) {
      const int bits = left < BITS ? left : BITS;
      __syncthreads();
      for (int i = tid; i < BINS; i += THREADS) s.bins[i] = 0;
      __syncthreads();
      for (int i = tid; i < vocab; i += THREADS) {
        const uint32_t k = key_at(i);
        if (k < border || k == 0 || (left < 32 && k >> left != prefix)) continue;
        if (k == border) continue;      // (its kept ones count below)
        const uint32_t bin = k >> (left - bits) & ((1u << bits) - 1);
        atomicAdd(&s.bins[bin], by_weight ? (unsigned long long)whole(weight(k), a.shift) : 1ull);
      }
      __syncthreads();
      if (tid == 0 && equal && (left == 32 || border >> left == prefix))
        s.bins[border >> (left - bits) & ((1u << bits) - 1)] += by_weight ? (unsigned long long)equal * whole(weight(border), a.shift) : (unsigned long long)equal;
      __syncthreads();
      find_bin(s, above, limit);
      above = s.above;
      prefix = prefix << bits | s.bin;
      left -= bits;
      __syncthreads();
    }
    // of the keys that are the border, as many as fit
    const unsigned long long each = by_weight ? whole(weight(prefix), a.shift) : 1;
    unsigned long long fit = each ? (limit - above + each - 1) / each : ~0ull;
    if (prefix == border && (unsigned long long)equal < fit) fit = equal;
    border = prefix;
    equal = (int)(fit > 0x7FFFFFFFull ? 0x7FFFFFFFull : fit);
  };
  if (r.top_k < vocab) search((unsigned long long)r.top_k, false);
  if (r.cut_p) {
    unsigned long long mine = 0, all;
    for (int i = tid; i < vocab; i += THREADS) {
      const uint32_t k = key_at(i);
      if (k > border) mine += whole(weight(k), a.shift);
    }
    __syncthreads();
    before_me<unsigned long long>(mine, s.sums, all);
    if (equal) {
      // (how many of them there are is not known where top_k allows more)
      uint32_t n = 0, there;
      for (int i = tid; i < vocab; i += THREADS) n += key_at(i) == border;
      before_me<uint32_t>(n, s.words, there);
      if ((uint32_t)equal > there) equal = (int)there;
      all += (unsigned long long)equal * whole(weight(border), a.shift);
    }
    const double limit = __builtin_ceil(r.top_p * (double)all);
    search(limit >= 1.0 ? (unsigned long long)limit : 1ull, true);
  }

  // kept weights in the order of the vocabulary: a thread has neighbouring tokens
  const int per = (vocab + THREADS - 1) / THREADS, first = tid * per < vocab ? tid * per : vocab, end = first + per < vocab ? first + per : vocab;
  uint32_t ties = 0, all_ties;
  if (equal)
    for (int i = first; i < end; ++i) ties += key_at(i) == border;
  const uint32_t ties_before = before_me<uint32_t>(ties, s.words, all_ties);
  auto kept = [&](int i, uint32_t& seen) -> uint64_t {
    const uint32_t k = key_at(i);
    if (k == 0 || k < border) return 0;
    if (k == border && seen++ >= (uint32_t)equal) return 0;
    const double w = weight(k);
    return k == most || w >= r.floor ? whole(w, a.shift) : 0;
  };
  uint32_t seen = ties_before;
  unsigned long long mine = 0, all;
  for (int i = first; i < end; ++i) mine += kept(i, seen);
  unsigned long long at = before_me<unsigned long long>(mine, s.sums, all);
  // the first place at which the sum exceeds u times all: whole numbers exceed it where they reach the next one
  const unsigned long long goal = (unsigned long long)__builtin_floor(r.u * (double)all) + 1;
  if (at < goal && at + mine >= goal) {
    seen = ties_before;
    for (int i = first; i < end; ++i) {
      const unsigned long long w = kept(i, seen);
      if (at + w >= goal) {
        a.tokens[row] = i;
        if (a.probability) a.probability[row] = (float)((double)w / (double)all);
        break;
      }
      at += w;
    }
  }
}

typedef void (*kernel_fn)(const Args);

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
  c->fn = cfg->in_dtype == FTSAMPLE_F32 ? ftsample_row<FTSAMPLE_F32> : cfg->in_dtype == FTSAMPLE_BF16 ? ftsample_row<FTSAMPLE_BF16> : ftsample_row<FTSAMPLE_F16>;
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
