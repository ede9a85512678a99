// One wave of 64 lanes on the host, for device functions that only index: 64 contexts that
// take turns, each running until it exchanges a value with the others. All lanes must
// make the same exchanges. Include it before the device code.
#pragma once

#include <ucontext.h>

#include <algorithm>
#include <cstdint>
#include <functional>
#include <vector>

#define __device__
#define __forceinline__ inline

struct Index3 {
  uint32_t x = 0, y = 0, z = 0;
};
inline Index3 threadIdx, blockIdx, gridDim;

using std::max;
using std::min;

namespace wave {
inline ucontext_t lanes[64], caller;
inline int64_t held[2][64];  // the values of this exchange and of the one before
inline int turn[64];
inline std::function<void()> body;
inline int finished;
inline int64_t exchanges;  // of all lanes

inline void start() {
  body();
  ++finished;
}
// The other lanes run up to the same point.
inline void others() {
  const Index3 me = threadIdx, block = blockIdx;
  swapcontext(&lanes[me.x], &caller);
  threadIdx = me;
  blockIdx = block;
}
template <class T, class F>
T exchange(T v, F pick) {
  const int t = turn[threadIdx.x] ^= 1;
  ++exchanges;
  held[t][threadIdx.x] = (int64_t)v;
  others();
  return (T)pick(held[t]);
}
}  // namespace wave

template <class T>
T __shfl(T v, int lane) {
  return wave::exchange(v, [&](const int64_t* h) { return h[lane % 64]; });
}
template <class T>
T __shfl_xor(T v, int mask) {
  return wave::exchange(v, [&](const int64_t* h) { return h[threadIdx.x ^ (uint32_t)mask]; });
}
template <class T>
T __shfl_up(T v, int d) {
  return wave::exchange(v, [&](const int64_t* h) { return h[(int)threadIdx.x < d ? threadIdx.x : threadIdx.x - d]; });
}
inline uint64_t __ballot(bool p) {
  return wave::exchange((uint64_t)p, [&](const int64_t* h) {
    uint64_t r = 0;
    for (int i = 0; i < 64; ++i) r |= (uint64_t)h[i] << i;
    return r;
  });
}
#define __builtin_amdgcn_readfirstlane(v) __shfl(v, 0)
inline int __ffsll(unsigned long long v) { return __builtin_ffsll((long long)v); }
inline int __clzll(long long v) { return v == 0 ? 64 : __builtin_clzll((unsigned long long)v); }

// body() in every lane of a wave.
inline void run_wave(std::function<void()> body) {
  static std::vector<char> stacks(64 << 17);
  wave::body = std::move(body);
  wave::finished = 0;
  for (int i = 0; i < 64; ++i) {
    wave::turn[i] = 0;
    getcontext(&wave::lanes[i]);
    wave::lanes[i].uc_stack.ss_sp = stacks.data() + ((size_t)i << 17);
    wave::lanes[i].uc_stack.ss_size = 1 << 17;
    wave::lanes[i].uc_link = &wave::caller;
    makecontext(&wave::lanes[i], wave::start, 0);
  }
  while (wave::finished < 64)
    for (uint32_t i = 0; i < 64 && wave::finished < 64; ++i) {
      threadIdx.x = i;
      swapcontext(&wave::caller, &wave::lanes[i]);
    }
}
