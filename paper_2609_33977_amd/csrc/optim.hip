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

// At most one block per chunk that a list of this size can hold.  Only the size is known here, so every entry after the
// first counts as 14 chunks, and so does room that the list does not need by its size.
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

__device__ __forceinline__ double add_squares(double sum, const f32x4& v) {
#pragma unroll
  for (int q = 0; q < 4; ++q) sum = fma(double(v[q]), double(v[q]), sum);
  return sum;
}

__device__ __forceinline__ double add_squares(double sum, const u32x4& v) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const double a = bf16_lo(v[q]), b = bf16_hi(v[q]);
    sum = fma(a, a, sum);
    sum = fma(b, b, sum);
  }
  return sum;
}

// A chunk's values: [start, end), of which those before `body` are the tensor's head.
struct ListRange {
  int64_t start, body, end;
  __device__ __forceinline__ ListRange(const ListEntry& e, int chunk) {
    const int64_t k = chunk - e.first, head = e.flags >> kListHeadShift;
    body = min(head + k * kListChunk, e.numel);
    end = min(head + (k + 1) * kListChunk, e.numel);
    start = k == 0 ? 0 : body;
  }
};

__device__ __forceinline__ double square_of(float g) { return double(g) * double(g); }
__device__ __forceinline__ double square_of(uint16_t g) { return square_of(bf16_to_f32(g)); }

// A chunk's squares, by 16-byte vectors of type V; a whole chunk has all its loads in flight.
template <typename V, typename T>
__device__ __forceinline__ double chunk_squares(double sum, const ListEntry& e, int chunk) {
  constexpr int PER = 16 / sizeof(T), N = kListChunk / (256 * PER);
  const ListRange r(e, chunk);
  const T* g = static_cast<const T*>(e.g) + r.body;
  const int len = int(r.end - r.body);
  if (r.start + threadIdx.x < r.body) sum += square_of(static_cast<const T*>(e.g)[r.start + threadIdx.x]);
  if (len == kListChunk) {
    V v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __builtin_nontemporal_load(reinterpret_cast<const V*>(g) + i * 256 + threadIdx.x);
#pragma unroll
    for (int i = 0; i < N; ++i) sum = add_squares(sum, v[i]);
    return sum;
  }
  const int done = len / PER * PER;
  for (int i = PER * threadIdx.x; i < done; i += 256 * PER) sum = add_squares(sum, *reinterpret_cast<const V*>(g + i));
  if (done + int(threadIdx.x) < len) sum += square_of(g[done + threadIdx.x]);
  return sum;
}

// Squares are summed in fp64: the square of an fp32 value is exact there and
// cannot overflow.  The next chunk's entry is loaded while this one's values are.
__global__ __launch_bounds__(256) void grad_norm_kernel(const void* list, size_t bytes, double* __restrict__ part) {
  double sum = 0.0;
  const ListView L(list, bytes);
  ListEntry next;
  if (int(blockIdx.x) < L.chunks) next = L.entries[L.map[blockIdx.x]];
  for (int c = blockIdx.x; c < L.chunks; c += gridDim.x) {
    const ListEntry e = next;
    if (c + int(gridDim.x) < L.chunks) next = L.entries[L.map[c + gridDim.x]];
    if (e.flags & kListGradBf16)
      sum = chunk_squares<u32x4, uint16_t>(sum, e, c);
    else
      sum = chunk_squares<f32x4, float>(sum, e, c);
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
    // 0 stands for a norm that is not finite as it is returned, and for no other: a finite one gets the least positive
    // fp32 value where its quotient would round to 0.
    const float f = float(n);
    norm[0] = f;
    coef[0] = !(f < __builtin_huge_valf()) ? 0.0f : n > double(max_norm) ? float(fmax(double(max_norm) / n, 0x1p-149)) : 1.0f;
  }
}

// `share` blocks take a chunk together, so that a list of few long tensors fills the chip too (262144 values of one
// tensor: 11.5 us with one block, 3.8 with eight).  Many short tensors count as more chunks than they are (list_blocks) and
// get fewer: 128 of 8192 values 10.5 us with one, a single tensor of as many values 6.5 with eight.
__global__ __launch_bounds__(256) void adamw_list_kernel(const void* list, size_t bytes, const float* coef, int share,
                                                        AdamW opt) {
  const float k = coef ? coef[0] : 1.0f;
  if (!(k > 0.0f && k < __builtin_huge_valf())) return;  // no step on a norm that is not finite
  const ListView L(list, bytes);
  const int tid = blockIdx.x % share * 256 + threadIdx.x, threads = share * 256;
  for (int c = blockIdx.x / share; c < L.chunks; c += gridDim.x / share) {
    const ListEntry e = L.entries[L.map[c]];
    if (!e.p || !e.m || !e.v) continue;
    const ListRange r(e, c);
    const bool b16 = e.flags & kListGradBf16;
    const float* g = static_cast<const float*>(e.g);
    const uint16_t* gh = static_cast<const uint16_t*>(e.g);
    auto one = [&](int64_t i) {
      float mq = e.m[i], vq = e.v[i];
      const float w = opt.step(e.p[i], (b16 ? bf16_to_f32(gh[i]) : g[i]) * k, mq, vq);
      e.p[i] = w, e.m[i] = mq, e.v[i] = vq;
      if (e.p16) e.p16[i] = uint16_t(f32_to_bf16_bits(w));
    };
    if (!(e.flags & kListVector)) {
      for (int64_t i = r.start + tid; i < r.end; i += threads) one(i);
      continue;
    }
    if (r.start + tid < r.body) one(r.start + tid);
    const int64_t done = r.body + (r.end - r.body) / 4 * 4;
    // Plain loads and nontemporal stores: parameters and moments of 2 to 15 M values, which stay in the last-level
    // cache from step to step, at 4.7 to 6.0 TB/s (3.9 to 5.1 with nontemporal loads too), 48 M at 5.1 (5.3).
#pragma unroll 2
    for (int64_t i = r.body + 4 * tid; i < done; i += 4 * threads) {
      f32x4 pv = *reinterpret_cast<const f32x4*>(e.p + i);
      f32x4 mv = *reinterpret_cast<const f32x4*>(e.m + i);
      f32x4 vv = *reinterpret_cast<const f32x4*>(e.v + i);
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
      __builtin_nontemporal_store(pv, reinterpret_cast<f32x4*>(e.p + i));
      __builtin_nontemporal_store(mv, reinterpret_cast<f32x4*>(e.m + i));
      __builtin_nontemporal_store(vv, reinterpret_cast<f32x4*>(e.v + i));
      if (e.p16) {
        const uint64_t w = uint64_t(pack_bf16x2(pv[0], pv[1])) | uint64_t(pack_bf16x2(pv[2], pv[3])) << 32;
        __builtin_nontemporal_store(w, reinterpret_cast<uint64_t*>(e.p16 + i));
      }
    }
    if (done + tid < r.end) one(done + tid);
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
      // Values before the gradient's first 16-byte boundary, and whether the step's vectors of four fit the other
      // addresses there too (tensors cut alike from one buffer per role have them in the same place).
      const uintptr_t size = b16 ? 2 : 4, head = ((16 - reinterpret_cast<uintptr_t>(e.g)) & 15) / size;
      const bool vec = e.p && aligned(e.p + head, 16) && aligned(e.m + head, 16) && aligned(e.v + head, 16) &&
                       (!e.p16 || aligned(e.p16 + head, 8));
      e.flags = (b16 ? kListGradBf16 : 0) | (vec ? kListVector : 0) | int(head) << kListHeadShift;
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
  const int blocks = list_blocks(list_bytes, 16384);
  const int share = blocks <= 256 ? 8 : blocks <= 1024 ? 2 : 1;
  hipLaunchKernelGGL(adamw_list_kernel, dim3(blocks * share), dim3(256), 0, s, list, list_bytes, coef, share,
                     make_adamw(lr, beta1, beta2, eps, weight_decay, step));
  return hipGetLastError();
}

}  // namespace gm
