// Stands in for the HIP runtime where a kernel is compiled for the host (x86-64): a launch runs its workgroups one after the other, each thread of one a stack of its
// own.  Threads run until they meet a barrier or an instruction that takes values from other lanes, in the order that host_order() sets, which nothing may depend on.
// LDS holds what host_order() fills it with when a workgroup begins.  Only what ftsample.hip uses is here; instructions across lanes are to be met by all 64 of them.
#pragma once
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>

#define __device__
#define __global__
#define __forceinline__ inline __attribute__((always_inline))
#define __launch_bounds__(...)
#define __shared__ static __attribute__((section("lds")))

struct dim3 {
  uint32_t x, y, z;
  dim3(uint32_t x = 1, uint32_t y = 1, uint32_t z = 1) : x(x), y(y), z(z) {}
};

extern char __start_lds[], __stop_lds[];
extern "C" void host_switch(void** from, void* to);      // saves this stack's registers, goes on with those of another
asm(R"(
.text
host_switch:
  push %rbp
  push %rbx
  push %r12
  push %r13
  push %r14
  push %r15
  mov %rsp, (%rdi)
  mov %rsi, %rsp
  pop %r15
  pop %r14
  pop %r13
  pop %r12
  pop %rbx
  pop %rbp
  ret
)");

namespace host {
constexpr int MOST = 1024;
constexpr size_t STACK = 128 << 10;
struct Thread {
  dim3 thread, block;
  void* at = nullptr;
  char* stack = nullptr;
  long steps = 0, barriers = 0;      // instructions across lanes and barriers that it has met
  bool done = false;
};
inline Thread threads[MOST];
inline Thread* now;
inline void* back;
inline int count, order;
inline uint8_t filling;
inline long most_steps = 1 << 17;
inline std::function<void()> body;
inline uint64_t given[MOST][2];      // by the threads, for this instruction and the one before it

inline void wait() { host_switch(&now->at, back); }
inline void entry() {
  body();
  now->done = true;
  wait();
}
[[noreturn]] inline void fail(const char* what) {
  std::fprintf(stderr, "workgroup %u, thread %u: %s\n", now->block.x, now->thread.x, what);
  std::fflush(stderr);
  std::_Exit(3);
}
inline bool waits(const Thread& t) {
  const int wave = t.thread.x / 64 * 64;
  for (int i = wave; i < wave + 64; ++i)
    if (threads[i].steps < t.steps) return true;
  for (int i = 0; i < count; ++i)
    if (!threads[i].done && threads[i].barriers < t.barriers) return true;
  return false;
}
inline void run_workgroup(uint32_t block) {
  std::memset(__start_lds, filling, (size_t)(__stop_lds - __start_lds));
  for (int i = 0; i < count; ++i) {
    Thread& t = threads[i];
    if (!t.stack) t.stack = static_cast<char*>(std::aligned_alloc(64, STACK));
    void** top = reinterpret_cast<void**>(t.stack + STACK) - 2;
    top[0] = reinterpret_cast<void*>(&entry);
    top[1] = nullptr;
    for (int r = 1; r <= 6; ++r) top[-r] = nullptr;
    t.at = top - 6;
    t.thread = dim3((uint32_t)i);
    t.block = dim3(block);
    t.steps = t.barriers = 0;
    t.done = false;
  }
  for (int left = count; left;) {
    bool moved = false;
    for (int n = 0; n < count; ++n) {
      // waves in either order, each as far as it comes, or all side by side
      const int i = order == 1 ? count - 1 - n : n;
      Thread& t = threads[i];
      now = &t;
      if (t.done || waits(t)) continue;
      moved = true;
      host_switch(&back, t.at);
      left -= t.done;
      if (order < 2 && n % 64 == 63) {      // this wave again, if it can go on
        bool can = false;
        for (int w = i / 64 * 64; w < i / 64 * 64 + 64; ++w) can = can || (!threads[w].done && !waits(threads[w]));
        if (can) n -= 64;
      }
    }
    if (!moved) fail("waits for threads that do not come");
  }
}
// This lane's value to all lanes of the wave.
inline uint64_t* give(uint64_t x) {
  Thread& t = *now;
  if (++t.steps > most_steps) fail("does not end");
  given[t.thread.x][t.steps & 1] = x;
  wait();
  return &given[t.thread.x / 64 * 64][t.steps & 1];
}
inline uint64_t of_lane(uint64_t x, int lane) { return give(x)[2 * (lane & 63)]; }
inline int lane() { return (int)now->thread.x & 63; }
inline void barrier() {
  if (++now->barriers > most_steps) fail("does not end");
  wait();
}
template <class T> T shuffled(T x, int lane) {
  uint64_t bits = 0;
  std::memcpy(&bits, &x, sizeof(T));
  bits = of_lane(bits, lane);
  std::memcpy(&x, &bits, sizeof(T));
  return x;
}
inline uint64_t ballot(bool x) {
  const uint64_t* all = give(x);
  uint64_t bits = 0;
  for (int i = 0; i < 64; ++i) bits |= all[2 * i] << i;
  return bits;
}
inline int update_dpp(int old, int x, int ctrl, int rows, int, bool) {
  const uint64_t* all = give((uint32_t)x);
  const int l = lane(), row = l / 16;
  if (!(rows >> row & 1)) return old;
  auto of = [&](int i) { return (int)(uint32_t)all[2 * i]; };
  if (ctrl > 0x110 && ctrl < 0x120) return l % 16 >= ctrl - 0x110 ? of(l - (ctrl - 0x110)) : old;
  if (ctrl > 0x120 && ctrl < 0x130) return of(row * 16 + (l - (ctrl - 0x120) & 15));
  if (ctrl == 0x142) return row ? of(16 * row - 1) : old;
  if (ctrl == 0x143) return row > 1 ? of(31) : old;
  if (ctrl < 0x100) return of((l & ~3) | (ctrl >> 2 * (l & 3) & 3));
  fail("an unknown form of dpp");
}
struct Pair {
  uint32_t r[2];
  uint32_t operator[](int i) const { return r[i]; }
};
// The upper one of two neighbouring groups of N lanes in the first result is the lower one's, the lower one in the second the upper one's.
inline Pair swapped(uint32_t x, int N) {
  const uint64_t* all = give(x);
  const int l = lane();
  return Pair{{l & N ? (uint32_t)all[2 * (l - N)] : x, l & N ? x : (uint32_t)all[2 * (l + N)]}};
}
struct Buffer {
  const char* data;
  uint32_t bytes;
};
struct Words4 {
  uint32_t w[4];
};
inline Words4 load4(const Buffer& b, int at, int more) {
  Words4 r = {{0, 0, 0, 0}};
  if ((uint32_t)at + 16 <= b.bytes) std::memcpy(&r, b.data + at + more, 16);
  return r;
}
template <class F, class A> void launch(F f, dim3 grid, dim3 block, const A& a) {
  count = (int)block.x;
  for (uint32_t b = 0; b < grid.x; ++b) {
    body = [&] { f(a); };
    run_workgroup(b);
  }
}
}  // namespace host
extern "C" inline __attribute__((used)) void host_order(int order, uint8_t filling) {
  host::order = order;
  host::filling = filling;
}

#define threadIdx (host::now->thread)
#define blockIdx (host::now->block)
#define __amdgpu_buffer_rsrc_t host::Buffer
#define __builtin_amdgcn_make_buffer_rsrc(p, stride, bytes, flags) (host::Buffer{(const char*)(p), (uint32_t)(bytes)})
#define __builtin_amdgcn_raw_buffer_load_b128(b, at, more, flags) host::load4(b, at, more)
#define __builtin_amdgcn_readfirstlane(x) ((int)(uint32_t)host::of_lane((uint32_t)(x), 0))
#define __builtin_amdgcn_readlane(x, l) ((int)(uint32_t)host::of_lane((uint32_t)(x), l))
#define __builtin_amdgcn_update_dpp host::update_dpp
#define __builtin_amdgcn_mov_dpp(x, ctrl, rows, banks, bound) host::update_dpp(0, x, ctrl, rows, banks, bound)
#define __builtin_amdgcn_ds_swizzle(x, how) ((int)(uint32_t)host::of_lane((uint32_t)(x), host::lane() ^ (how) >> 10))
#define __builtin_amdgcn_permlane16_swap(x, y, a, b) host::swapped(x, 16)
#define __builtin_amdgcn_permlane32_swap(x, y, a, b) host::swapped(x, 32)
#define __builtin_amdgcn_exp2f exp2f
inline void __syncthreads() { host::barrier(); }
inline uint64_t __ballot(bool x) { return host::ballot(x); }
inline bool __any(bool x) { return host::ballot(x) != 0; }
inline int __popcll(uint64_t x) { return __builtin_popcountll(x); }
template <class T> T __shfl_xor(T x, int d) { return host::shuffled(x, host::lane() ^ d); }
template <class T> T __shfl(T x, int l) { return host::shuffled(x, l); }
template <class T> T atomicAdd(T* to, T x) {
  const T before = *to;
  *to += x;
  return before;
}

enum hipError_t { hipSuccess = 0, hipErrorOutOfMemory = 2 };
typedef struct host_stream* hipStream_t;
inline const char* hipGetErrorString(hipError_t) { return ""; }
inline hipError_t hipGetDevice(int* d) { return *d = 0, hipSuccess; }
inline hipError_t hipSetDevice(int) { return hipSuccess; }
inline hipError_t hipGetLastError() { return hipSuccess; }
#define hipLaunchKernelGGL(f, grid, block, lds, stream, a) host::launch(f, grid, block, a)
