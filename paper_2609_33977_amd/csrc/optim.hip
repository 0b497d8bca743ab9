// The optimiser's work over many tensors at once: the norm of all their
// gradients, the coefficient that clips it, and one AdamW step over all of them.
//
//   norm = sqrt(sum g^2),  coef = min(1, max_norm / norm)
//   p, m, v <- AdamW(p, coef g, m, v),  p16 <- bf16(p)
//
// Both passes are bound by memory: 4 (or 2) bytes per value for the norm, 30
// for the step with its bf16 copy.  The clipped gradients are never written:
// the step multiplies as it reads.  The tensors are cut into chunks of
// kListChunk values; a list in device memory, written once, holds the
// tensors' addresses and the tensor of every chunk, so that a call is one
// launch however many tensors there are.
#include "gm_adamw.h"
#include "gm_device.h"
#include "gm_launch.h"
#include "gm_list.h"

namespace gm {

// A list as a kernel reads it: nothing of it is followed unless its header and
// its size agree.
struct ListView {
  const ListEntry* entries;
  const int* map;
  int chunks;
  __device__ __forceinline__ ListView(const void* list, size_t bytes) {
    const ListHead h = *static_cast<const ListHead*>(list);
    const bool ok = h.magic == kListMagic && h.n >= 1 && h.chunks >= 0 &&
                    kListHeadBytes + size_t(h.n) * sizeof(ListEntry) + size_t(h.chunks) * 4 <= bytes;
    entries = reinterpret_cast<const ListEntry*>(static_cast<const char*>(list) + kListHeadBytes);
    map = reinterpret_cast<const int*>(entries + (ok ? h.n : 0));
    chunks = ok ? h.chunks : 0;
  }
};

// At most one block per chunk that a list of this size can hold.
static int list_blocks(size_t bytes, int most) {
  const size_t chunks = bytes > kListHeadBytes + sizeof(ListEntry) ? (bytes - kListHeadBytes - sizeof(ListEntry)) / 4 : 1;
  return chunks < size_t(most) ? (chunks ? int(chunks) : 1) : most;
}

struct ListWrite {
  ListEntry e[kListPerLaunch];
  int index[kListPerLaunch];
  int chunks[kListPerLaunch];
};

__global__ __launch_bounds__(256) void tensor_list_kernel(ListWrite w, int total, int n, ListHead* head,
                                                         ListEntry* entries, int* map) {
  const int i = blockIdx.x;
  if (threadIdx.x == 0) {
    entries[w.index[i]] = w.e[i];
    if (w.index[i] == 0) *head = {kListMagic, n, total, 0};
  }
  for (int c = threadIdx.x; c < w.chunks[i]; c += 256) map[w.e[i].first + c] = w.index[i];
}

__device__ __forceinline__ double sum_block(double v) {
  __shared__ double s_w[4];
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) v += __shfl_xor(v, x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = v;
  __syncthreads();
  return (s_w[0] + s_w[1]) + (s_w[2] + s_w[3]);
}

// Squares are summed in fp64: the square of an fp32 value is exact there and
// cannot overflow.
__global__ __launch_bounds__(256) void grad_norm_kernel(const void* list, size_t bytes, double* __restrict__ part) {
  double sum = 0.0;
  const ListView L(list, bytes);
  for (int c = blockIdx.x; c < L.chunks; c += gridDim.x) {
    const ListEntry e = L.entries[L.map[c]];
    const int64_t at = int64_t(c - e.first) * kListChunk;
    const int len = int(min(e.numel - at, int64_t(kListChunk)));
    if (e.flags & kListGradBf16) {
      const uint16_t* g = static_cast<const uint16_t*>(e.g) + at;
      int done = 0;
      if (e.flags & kListVector) {
        done = len / 8 * 8;
        for (int i = 8 * threadIdx.x; i < done; i += 2048) {
          const u32x4 v = ld16(g + i);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const double a = bf16_lo(v[q]), b = bf16_hi(v[q]);
            sum = fma(a, a, sum);
            sum = fma(b, b, sum);
          }
        }
      }
      for (int i = done + threadIdx.x; i < len; i += 256) {
        const double a = bf16_to_f32(g[i]);
        sum = fma(a, a, sum);
      }
    } else {
      const float* g = static_cast<const float*>(e.g) + at;
      int done = 0;
      if (e.flags & kListVector) {
        done = len / 4 * 4;
#pragma unroll 8
        for (int i = 4 * threadIdx.x; i < done; i += 1024) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(g + i);
#pragma unroll
          for (int q = 0; q < 4; ++q) sum = fma(double(v[q]), double(v[q]), sum);
        }
      }
      for (int i = done + threadIdx.x; i < len; i += 256) {
        const double a = g[i];
        sum = fma(a, a, sum);
      }
    }
  }
  const double s = sum_block(sum);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(256) void grad_norm_done_kernel(const double* __restrict__ part, int blocks,
                                                            float max_norm, float* __restrict__ norm,
                                                            float* __restrict__ coef) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < blocks; i += 256) sum += part[i];
  const double n = sqrt(sum_block(sum));
  if (threadIdx.x == 0) {
    norm[0] = float(n);
    coef[0] = !(n < __builtin_huge_val()) ? 0.0f : n > double(max_norm) ? float(double(max_norm) / n) : 1.0f;
  }
}

__global__ __launch_bounds__(256) void adamw_list_kernel(const void* list, size_t bytes, const float* coef, AdamW opt) {
  const float k = coef ? coef[0] : 1.0f;
  if (!(k > 0.0f && k < __builtin_huge_valf())) return;  // no step on a norm that is not finite
  const ListView L(list, bytes);
  for (int c = blockIdx.x; c < L.chunks; c += gridDim.x) {
    const ListEntry e = L.entries[L.map[c]];
    if (!e.p || !e.m || !e.v) continue;
    const int64_t at = int64_t(c - e.first) * kListChunk;
    const int len = int(min(e.numel - at, int64_t(kListChunk)));
    float *p = e.p + at, *m = e.m + at, *v = e.v + at;
    uint16_t* h = e.p16 ? e.p16 + at : nullptr;
    const bool b16 = e.flags & kListGradBf16;
    const float* g = b16 ? nullptr : static_cast<const float*>(e.g) + at;
    const uint16_t* gh = b16 ? static_cast<const uint16_t*>(e.g) + at : nullptr;
    int done = 0;
    if (e.flags & kListVector) {
      done = len / 4 * 4;
      for (int i = 4 * threadIdx.x; i < done; i += 1024) {
        f32x4 pv = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + i));
        f32x4 mv = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(m + i));
        f32x4 vv = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(v + i));
        f32x4 gv;
        if (b16) {
          const uint64_t w = *reinterpret_cast<const uint64_t*>(gh + i);
#pragma unroll
          for (int q = 0; q < 4; ++q) gv[q] = bf16_to_f32(uint16_t(w >> (16 * q)));
        } else {
          gv = *reinterpret_cast<const f32x4*>(g + i);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float mq = mv[q], vq = vv[q];
          pv[q] = opt.step(pv[q], gv[q] * k, mq, vq);
          mv[q] = mq, vv[q] = vq;
        }
        __builtin_nontemporal_store(pv, reinterpret_cast<f32x4*>(p + i));
        __builtin_nontemporal_store(mv, reinterpret_cast<f32x4*>(m + i));
        __builtin_nontemporal_store(vv, reinterpret_cast<f32x4*>(v + i));
        if (h) {
          const uint64_t w = uint64_t(pack_bf16x2(pv[0], pv[1])) | uint64_t(pack_bf16x2(pv[2], pv[3])) << 32;
          *reinterpret_cast<uint64_t*>(h + i) = w;
        }
      }
    }
    for (int i = done + threadIdx.x; i < len; i += 256) {
      float mq = m[i], vq = v[i];
      const float w = opt.step(p[i], (b16 ? bf16_to_f32(gh[i]) : g[i]) * k, mq, vq);
      p[i] = w, m[i] = mq, v[i] = vq;
      if (h) h[i] = uint16_t(f32_to_bf16_bits(w));
    }
  }
}

hipError_t launch_tensor_list(float* const* p, const void* const* g, float* const* m, float* const* v,
                              uint16_t* const* p16, const uint8_t* g_bf16, const int64_t* numel, int n, void* list, hipStream_t s) {
  ListHead* head = static_cast<ListHead*>(list);
  ListEntry* entries = reinterpret_cast<ListEntry*>(static_cast<char*>(list) + kListHeadBytes);
  int* map = reinterpret_cast<int*>(entries + n);
  const auto aligned = [](const void* x, uintptr_t a) { return (reinterpret_cast<uintptr_t>(x) & (a - 1)) == 0; };
  int64_t total = 0;
  for (int i = 0; i < n; ++i) total += list_chunks(numel[i]);
  int first = 0;
  for (int i0 = 0; i0 < n; i0 += kListPerLaunch) {
    ListWrite w = {};
    const int k = n - i0 < kListPerLaunch ? n - i0 : kListPerLaunch;
    for (int i = 0; i < k; ++i) {
      const int t = i0 + i;
      ListEntry& e = w.e[i];
      e.g = g[t];
      e.p = p ? p[t] : nullptr;
      e.m = m ? m[t] : nullptr;
      e.v = v ? v[t] : nullptr;
      e.p16 = p16 ? p16[t] : nullptr;
      e.numel = numel[t];
      e.first = first;
      const bool b16 = g_bf16 && g_bf16[t];
      // Vectors of four values (eight bf16 gradients in the norm) where every address allows them.
      const bool vec = aligned(e.g, 16) && aligned(e.p, 16) && aligned(e.m, 16) && aligned(e.v, 16) && aligned(e.p16, 8);
      e.flags = (b16 ? kListGradBf16 : 0) | (vec ? kListVector : 0);
      w.index[i] = t;
      w.chunks[i] = int(list_chunks(numel[t]));
      first += w.chunks[i];
    }
    hipLaunchKernelGGL(tensor_list_kernel, dim3(k), dim3(256), 0, s, w, int(total), n, head, entries, map);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

hipError_t launch_grad_norm(const void* list, size_t list_bytes, float max_norm, float* norm, float* coef,
                            double* part, hipStream_t s) {
  const int blocks = list_blocks(list_bytes, kNormBlocks);
  hipLaunchKernelGGL(grad_norm_kernel, dim3(blocks), dim3(256), 0, s, list, list_bytes, part);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL(grad_norm_done_kernel, dim3(1), dim3(256), 0, s, part, blocks, max_norm, norm, coef);
  return hipGetLastError();
}

hipError_t launch_adamw_list(const void* list, size_t list_bytes, double lr, double beta1, double beta2, double eps,
                             double weight_decay, int step, const float* coef, hipStream_t s) {
  hipLaunchKernelGGL(adamw_list_kernel, dim3(list_blocks(list_bytes, 16384)), dim3(256), 0, s, list, list_bytes, coef,
                     make_adamw(lr, beta1, beta2, eps, weight_decay, step));
  return hipGetLastError();
}

}  // namespace gm
