// Layout of a tensor list in device memory: a header, one entry per tensor,
// and the tensor of every chunk of kListChunk values.  A tensor's chunks begin
// where its gradient is 16-byte aligned; the few values before that (its head)
// belong to the first.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace gm {

constexpr int kListChunk = 8192;
constexpr int kListPerLaunch = 48;  // entries that one launch carries in its arguments
constexpr int32_t kListMagic = 0x4c9e21b7;
constexpr int kListVector = 1, kListGradBf16 = 2, kListHeadShift = 8;  // entry flags, and the head's values from bit 8 up
constexpr int kNormBlocks = 2048;

struct ListHead {
  int32_t magic, n, chunks, spare;
};

struct ListEntry {
  float* p;
  const void* g;
  float* m;
  float* v;
  uint16_t* p16;
  int64_t numel;
  int32_t first;  // the tensor's first chunk
  int32_t flags;
};

constexpr size_t kListHeadBytes = 64;

inline int64_t list_chunks(int64_t numel) { return (numel + kListChunk - 1) / kListChunk; }
inline size_t list_bytes_of(int64_t n, int64_t chunks) {
  return kListHeadBytes + size_t(n) * sizeof(ListEntry) + (size_t(chunks) * 4 + 15) / 16 * 16;
}

}  // namespace gm
