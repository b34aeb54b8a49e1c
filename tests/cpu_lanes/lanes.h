// lanes.h -- runs the dense operators' kernels on the CPU from their own
// source: a block's lanes are threads, a wave's exchanges (matrix
// instructions, transposing LDS reads) go through a table of the wave, LDS is
// a static array.  For checks that a sanitizer makes of indexes and of what is
// read of the operands.  Include it before the kernels.
#pragma once

#define __HIP_PLATFORM_AMD__
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <barrier>
#include <memory>
#include <thread>
#include <type_traits>
#include <vector>

namespace lanes {

constexpr int kWaveLanes = 64;
struct Index {
  unsigned x = 0, y = 0, z = 0;
};
inline thread_local Index thread, block, block_dim, grid;

struct Wave {
  std::barrier<> meet{kWaveLanes};
  alignas(16) unsigned char a[kWaveLanes][16], b[kWaveLanes][16];
};
inline std::vector<std::unique_ptr<Wave>> waves;
inline std::unique_ptr<std::barrier<>> all;

inline Wave &wave() { return *waves[thread.x / kWaveLanes]; }
inline int lane() { return thread.x % kWaveLanes; }
inline void wave_meets() { wave().meet.arrive_and_wait(); }
inline void block_meets() { all->arrive_and_wait(); }

// D = A B + C over a wave, I rows and columns, K long: lane l brings K *
// I / 64 consecutive k of row (column) l % I, and holds column l % I of D.
template <int I, int K, class E, class V, class A>
A mfma(V a, V b, A c) {
  constexpr int each = K * I / kWaveLanes;
  static_assert(sizeof(V) == each * sizeof(E), "a lane's piece");
  Wave &w = wave();
  memcpy(w.a[lane()], &a, sizeof(a));
  memcpy(w.b[lane()], &b, sizeof(b));
  wave_meets();
  const int col = lane() % I, group = lane() / I;
  constexpr int groups = kWaveLanes / I;
  for (int r = 0; r < I * I / kWaveLanes; ++r) {
    const int row = r / 4 * 4 * groups + 4 * group + r % 4;
    float sum = c[r];
    for (int k = 0; k < K; ++k) {
      E x, y;
      memcpy(&x, w.a[row + I * (k / each)] + k % each * sizeof(E), sizeof(E));
      memcpy(&y, w.b[col + I * (k / each)] + k % each * sizeof(E), sizeof(E));
      sum += (float)x * (float)y;
    }
    c[r] = sum;
  }
  wave_meets();
  return c;
}

// 16 lanes read 4 lines of 16 two-byte values, four a lane; lane c gets
// column c of the lines.
template <class V>
V read_transposed(const void *p) {
  Wave &w = wave();
  memcpy(w.a[lane()], p, 8);
  wave_meets();
  V v;
  const int c = lane() % 16, first = lane() - c;
  for (int j = 0; j < 4; ++j) {
    short e;
    memcpy(&e, w.a[first + 4 * j + c / 4] + 2 * (c % 4), 2);
    v[j] = e;
  }
  wave_meets();
  return v;
}

inline float exchange(float v, int by) {
  Wave &w = wave();
  memcpy(w.a[lane()], &v, 4);
  wave_meets();
  memcpy(&v, w.a[lane() ^ by], 4);
  wave_meets();
  return v;
}

inline uint32_t byte_permute(uint32_t hi, uint32_t lo, uint32_t select) {
  const uint64_t both = ((uint64_t)hi << 32) | lo;
  uint32_t r = 0;
  for (int i = 0; i < 4; ++i)
    r |= (uint32_t)((both >> (8 * (select >> (8 * i) & 7))) & 255) << (8 * i);
  return r;
}

// Runs `kernel` in blocks of nt lanes, one block after the other.
template <class F>
void launch(unsigned blocks, int nt, F kernel) {
  waves.clear();
  for (int i = 0; i < nt / kWaveLanes; ++i)
    waves.push_back(std::make_unique<Wave>());
  all = std::make_unique<std::barrier<>>(nt);
  std::vector<std::thread> threads;
  for (int t = 0; t < nt; ++t)
    threads.emplace_back([=] {
      thread.x = t;
      block_dim.x = nt;
      grid.x = blocks;
      for (unsigned b = 0; b < blocks; ++b) {
        block.x = b;
        kernel();
        block_meets();
      }
    });
  for (std::thread &t : threads) t.join();
}

}  // namespace lanes

template <class A, class B>
std::common_type_t<A, B> min(A a, B b) {
  return a < b ? a : b;
}
template <class A, class B>
std::common_type_t<A, B> max(A a, B b) {
  return a < b ? b : a;
}
inline float __uint_as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
inline uint32_t __float_as_uint(float v) {
  return __builtin_bit_cast(uint32_t, v);
}
inline int __float_as_int(float v) { return __builtin_bit_cast(int, v); }

// named by the shared headers, called by no kernel that runs here
template <class... A>
int not_here(A...) {
  abort();
}
#define atomicAdd not_here
#define atomicMax not_here
#define atomicOr not_here
#define __builtin_amdgcn_update_dpp not_here
#define __builtin_amdgcn_readlane not_here

#undef __device__
#undef __global__
#undef __shared__
#undef __forceinline__
#undef __launch_bounds__
#undef hipLaunchKernelGGL
#define __device__
#define __global__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define hipLaunchKernelGGL(...) ((void)0)
#define threadIdx lanes::thread
#define blockIdx lanes::block
#define blockDim lanes::block_dim
#define gridDim lanes::grid
#define __syncthreads() lanes::block_meets()
#define __shfl_xor(v, by, width) lanes::exchange(v, by)
#define __builtin_amdgcn_readfirstlane(v) (v)
#define __builtin_amdgcn_wave_barrier() lanes::wave_meets()
#define __builtin_amdgcn_sched_barrier(v) ((void)0)
#define __builtin_amdgcn_exp2f exp2f
#define __builtin_amdgcn_rcpf(v) (1.0f / (v))
#define __builtin_amdgcn_perm lanes::byte_permute
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) \
  lanes::read_transposed<s16x4_t>((const void *)(p))
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) \
  lanes::mfma<32, 16, __bf16>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) \
  lanes::mfma<16, 32, __bf16>(a, b, c)
#define __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, x, y, z) \
  lanes::mfma<32, 2, float>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, x, y, z) \
  lanes::mfma<16, 4, float>(a, b, c)
// instructions written out: only copies that bypass the registers, which the
// forms run here do not use
#define asm
#define volatile(...) ((void)0)
