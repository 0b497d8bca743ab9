// Low-rank adapters beside a masked or packed linear: for a token t with
// adapter a (scale c_a, A_a [R, d_in] with R = parts r, B_a [d_out, r])
//
//   P[t] = X[t] A_a^T                       Y[t]  = base[t] + c_a P[t] B_a^T   (part by part)
//   Q[t] = c_a dY[t] B_a                    dX[t] = base[t] + Q[t] A_a
//   dA_a = sum_t Q[t]^T X[t]                dB_a  = c_a sum_t dY[t]^T P[t]
//
// All four tall matrices (X, Y, dY, dX) stream through once per product and the
// adapters are small, so every product is bound by memory (r = 16 does 16
// multiply-adds per byte of X).  The tokens are taken in the plan's order,
// sorted by adapter, so that a tile of tokens shares one adapter wherever its
// tokens lie in the batch; a gathered row is still d_in contiguous values.
//
// P and Q are fp32.  The matrix instructions multiply bf16, so a product with P
// or Q takes them as a sum of bf16 terms: two (16 bits of significand) where
// the result is rounded to bf16, three (all 24 bits) where it stays fp32.
// Every sum over blocks goes through partial sums added in a fixed order.
#include "gm_device.h"
#include "gm_launch.h"
#include "gm_lora.h"
#include "gm_pipe.h"

namespace gm {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// C [16 x 16] += A [16 x 32] B [32 x 16]: lane l supplies A row (l % 16) and B
// column (l % 16), each over k = 8 (l / 16) .. + 7, and holds C rows
// 4 (l / 16) + i of column (l % 16).
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0,
                                                 0, 0);
}

// ---------------------------------------------------------------- plan

struct LoraTile {
  int pos, count, adapter, only;
};

struct LoraPlan {
  const int* head;
  const LoraTile* tiles;
  const int* tokens;
  const LoraTile* gtiles;  // of the length in use
  const int* gstart;
  int glen, T, n;
  // Entry i of a table with head[which] of them, without tokens if there is none: past the last, or in a
  // plan that was made for other sizes.  Header, entry and the tile's tokens do not wait for one another.
  __device__ __forceinline__ LoraTile tile(const LoraTile* table, int i, int which) const {
    const int magic = head[0], hT = head[1], hn = head[2], count = head[which];
    LoraTile t = table[i];
    if (magic != kLoraMagic || hT != T || hn != n || i >= count) t.count = 0;
    return t;
  }
};

static LoraPlan lora_plan(const void* plan, int T, int n, int glen) {
  const LoraPlanLayout L = lora_plan_layout(T, n);
  const int* w = static_cast<const int*>(plan);
  return {w, reinterpret_cast<const LoraTile*>(w + L.tiles), w + L.tokens,
          reinterpret_cast<const LoraTile*>(w + L.gtiles[glen]), w + L.gstart[glen], glen, T, n};
}

// Lanes of the wave with the same key, as a mask; runs of one key are told at once.
__device__ __forceinline__ uint64_t same_key(int key, int bits, bool on) {
  uint64_t m = __ballot(on);
  if ((__ballot(key != __builtin_amdgcn_readfirstlane(key)) & m) == 0) return m;
#pragma unroll 1
  for (int b = 0; b < bits; ++b) {
    const uint64_t one = __ballot((key >> b) & 1);
    m &= (key >> b) & 1 ? one : ~one;
  }
  return m;
}

constexpr int kPlanBatch = 8;  // runs of 64 ids that a wave loads at once

struct LoraPlanOut {
  int* head;
  LoraTile* tiles;
  int* tokens;
  LoraTile* gtiles[kLoraGradLens];
  int* gstart[kLoraGradLens];
};

// Per bucket, scanned together: its first position and tile and its first gradient tile of each length, 14 bits or more each.
struct LoraFirst {
  uint64_t a;  // position, 20 bits | tile << 20 | gradient tiles << 34 and << 48
  uint32_t b;  // gradient tiles, 16 bits each
  __device__ __forceinline__ int pos() const { return int(a & 0xfffff); }
  __device__ __forceinline__ int tile() const { return int(a >> 20) & 0x3fff; }
  __device__ __forceinline__ int gtile(int i) const {
    return i == 0 ? int(a >> 34) & 0x3fff : i == 1 ? int(a >> 48) : i == 2 ? int(b & 0xffff) : int(b >> 16);
  }
  __device__ __forceinline__ void add(const LoraFirst& o) { a += o.a, b += o.b; }
};
static_assert(kLoraGradLens == 4, "fields of LoraFirst");

// A stable counting sort of the tokens by adapter in one block: each wave
// counts and later places a contiguous run of tokens, so that equal adapters
// keep their tokens' order and sums over them do not depend on timing: the lanes
// of one key elect a leader, which adds to its wave's own counter in LDS (an
// atomic only so that the wave need not wait for it; a wave's LDS operations run in
// order).  One launch per batch serves every linear of the model.  Bound by
// latency, of instructions too: they run once, so loops stay rolled (10 KB of
// code took 13 us for 8192 tokens).  The ids of 512 tokens per wave are loaded at a time.
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void lora_plan_kernel(const int* __restrict__ adapter, int T, int n,
                                                              LoraPlanOut out) {
  extern __shared__ int s_count[];  // [WAVES][n + 1], then the buckets' first entries [n + 2] and last tokens [n + 1]
  __shared__ LoraFirst s_sum[WAVES];
  __shared__ int s_ids[WAVES][64 * kPlanBatch];
  constexpr int NT = 64 * WAVES;
  const int nb = n + 1, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  LoraFirst* s_first = reinterpret_cast<LoraFirst*>(s_count + (WAVES * nb + 1) / 2 * 2);
  int* s_last = reinterpret_cast<int*>(s_first + nb + 1);
  const int bits = 32 - __builtin_clz(n);
  const int per = (T + NT - 1) / NT * 64;  // tokens per wave
  const int t0 = min(wave * per, T), t1 = min(t0 + per, T);
  int* mine = s_count + wave * nb;
  auto load_ids = [&](int t) {
    int ids[kPlanBatch];
#pragma unroll
    for (int i = 0; i < kPlanBatch; ++i) ids[i] = adapter[min(t + 64 * i + lane, T - 1)];
#pragma unroll
    for (int i = 0; i < kPlanBatch; ++i) s_ids[wave][64 * i + lane] = unsigned(ids[i]) < unsigned(n) ? ids[i] : n;
  };
  for (int i = tid; i < WAVES * nb; i += NT) s_count[i] = 0;
  __syncthreads();
  // Twice over this wave's tokens: count them, and place them once everybody's counts are known.
  for (int place = 0; place < 2; ++place) {
    for (int t = t0; t < t1; t += 64 * kPlanBatch) {
      if (place == 0 || per > 64 * kPlanBatch) load_ids(t);  // else they are still there
      const int chunks = min((t1 - t + 63) >> 6, kPlanBatch);
#pragma unroll 1
      for (int i = 0; i < chunks; ++i) {
        const int token = t + 64 * i + lane, key = s_ids[wave][64 * i + lane];
        const bool on = token < t1;
        const uint64_t m = same_key(key, bits, on);
        const int before = __popcll(m & ((uint64_t(1) << lane) - 1));
        const int at = on && before == 0 ? atomicAdd(mine + key, __popcll(m)) : 0;
        if (place) {
          const int rank = __shfl(at, __builtin_ctzll(m | (uint64_t(1) << 63))) + before;
          const LoraFirst f = s_first[key];
          if (on) {
            out.tokens[f.tile() * kLoraTile + rank] = token;
            if (rank == s_first[key + 1].pos() - f.pos() - 1) s_last[key] = token;
          }
        }
      }
    }
    __syncthreads();
    if (place) break;
    // Totals of a run of buckets per thread, scanned over the threads that have any; a wave's
    // counts become its first position within the bucket.
    const int run = (nb + NT - 1) / NT, b0 = min(tid * run, nb), b1 = min(b0 + run, nb);
    LoraFirst c = {0, 0};
    for (int b = b0; b < b1; ++b) {
      int tot = 0;
      int k[WAVES];
#pragma unroll
      for (int w = 0; w < WAVES; ++w) k[w] = s_count[w * nb + b];
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        s_count[w * nb + b] = tot;
        tot += k[w];
      }
      s_first[b] = c;
      auto tiles = [&](int len) { return uint64_t((tot + len - 1) / len); };
      LoraFirst f = {uint64_t(tot) | tiles(kLoraTile) << 20, 0};
      if (b < n) {
        f.a |= tiles(kLoraGradTokens) << 34 | tiles(kLoraGradTokens * 2) << 48;
        f.b = uint32_t(tiles(kLoraGradTokens * 4)) | uint32_t(tiles(kLoraGradTokens * 8)) << 16;
      }
      c.add(f);
    }
    LoraFirst e = c;
#pragma unroll 1
    for (int d = 1; d < min(64, nb); d <<= 1) {
      const LoraFirst up = {__shfl_up(e.a, d), uint32_t(__shfl_up(int(e.b), d))};
      if (lane >= d) e.add(up);
    }
    if (lane == 63) s_sum[wave] = e;
    __syncthreads();
    e.a -= c.a, e.b -= c.b;
    if (b0 < b1) {
#pragma unroll 1
      for (int w = 0; w < wave; ++w) e.add(s_sum[w]);
    }
    for (int b = b0; b < b1; ++b) {
      LoraFirst f = s_first[b];
      f.add(e);
      s_first[b] = f;
    }
    if (b0 < b1 && b1 == nb) {
      e.add(c);
      s_first[nb] = e;
      out.head[0] = kLoraMagic, out.head[1] = T, out.head[2] = n, out.head[3] = e.tile();
#pragma unroll
      for (int i = 0; i < kLoraGradLens; ++i) out.head[4 + i] = e.gtile(i);
    }
    __syncthreads();
  }
  // 16 lanes per bucket
  const int l16 = tid & 15;
#pragma unroll 1
  for (int b = tid >> 4; b < nb; b += NT / 16) {
    const LoraFirst f = s_first[b], g = s_first[b + 1];
    const int p = f.pos(), tot = g.pos() - p, nt = g.tile() - f.tile();
#pragma unroll 1
    for (int i = l16; i < nt; i += 16)
      out.tiles[f.tile() + i] = {p + i * kLoraTile, min(kLoraTile, tot - i * kLoraTile), b, 0};
#pragma unroll 1
    for (int i = tot + l16; i < nt * kLoraTile; i += 16) out.tokens[f.tile() * kLoraTile + i] = s_last[b];
#pragma unroll
    for (int l = 0; l < kLoraGradLens; ++l) {
      const int len = kLoraGradTokens << l, first = f.gtile(l), ng = g.gtile(l) - first;
      if (l16 == 0) out.gstart[l][b] = first;
#pragma unroll 1
      for (int i = l16; i < ng; i += 16)
        out.gtiles[l][first + i] = {f.tile() + i * (len / kLoraTile), min(len, tot - i * len), b, ng == 1};
    }
  }
}

// ---------------------------------------------------------------- products with the long axis contracted

struct LoraDown {
  const uint16_t* X;  // rows of the tall matrix
  int64_t ldx;
  const uint16_t* W;  // one adapter's weights: [wrows, K] (A) or [K, wrows] (B, one part)
  int64_t wstride;    // elements from one adapter to the next
  int K, wrows;
  float* part;  // [splits][T][R], rows in the plan's order
  int R;
  int splits;
  int off[kLoraMaxParts], width[kLoraMaxParts];  // B: the parts' columns
  int chunks;                                    // blocks of 16 RT ranks per part
};

// 16 bytes per lane from memory into LDS at lds + 16 lane (uniform), without a register between.
__device__ __forceinline__ void lora_dma16(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds) : "memory");
}

// Fragment of 16 columns with the rows contracted, from rows of `pitch` bytes in LDS: the lane's column is
// col0 + lane % 16 and its k rows 8 (lane / 16) .. + 7.  The 16-lane group q reads rows 8 q + (lane % 16) / 4 and + 4.
__device__ __forceinline__ u32x4 lora_tr_frag(const char* base, int pitch, int col0, int lane) {
  const int row = lane & 15, q = lane >> 4;
  const char* b = base + (8 * q + (row >> 2)) * pitch + col0 * 2 + 8 * (row & 3);
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)b);
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(b + 4 * pitch));
  u32x4 f;
  __builtin_memcpy(&f, &lo, 8);
  __builtin_memcpy(reinterpret_cast<char*>(&f) + 8, &hi, 8);
  return f;
}

constexpr int kDownK = 128;  // contraction length per stage, dealt to the splits in turn

// Stages in LDS, each 16 KiB of tokens and 4 RT KiB of the adapter: two blocks per CU (60, 72 and 64 KiB a block).  With
// two stages of 128 k 8192 tokens of 11008 columns and 64 ranks took 44 us in a loop without plan and stores, with four of
// 64 k 47; the whole kernel takes 48.
template <int RT>
constexpr int kDownStages = RT == 4 ? 2 : 3;
template <int RT>
constexpr int kDownSlots = kDownStages<RT> * (16 + 4 * RT) * 64;  // of 16 bytes

// part[s][p][c] = sum over split s's share of K of X[token p][k] W[c][k], for a
// tile of 17 to 64 tokens: 128 k of the tokens' rows and of the adapter are copied into LDS ahead of their use;
// each wave takes 16 tokens and all ranks.  Splits take every splits-th 128 k, so that
// blocks that run together read neighbouring columns: 4096 tokens of 4096 columns, 16 ranks 10.6 us, 4099 tokens of 12
// adapters 9.1, against 11.4 and 9.4 with a run of columns for each split; 8192 tokens of 11008 columns, 64 ranks 48.0
// against 44.3.  B is contracted over its rows, which come back transposed.
template <int RT, bool BMAJOR>
__device__ __forceinline__ void lora_down_wide(const LoraDown& a, const LoraTile& tile, const int* tokens,
                                               int split, int K, int col0, int r0, int nr, float* out, u32x4* s_mem) {
  constexpr int NS = kDownStages<RT>, COPIES = 16 + 4 * RT, PER = COPIES / 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, q = lane >> 4;
  const uint32_t lds = lds_addr(s_mem);
  const uint16_t* w = a.W + int64_t(tile.adapter) * a.wstride;
  // Copy c < 16: 32 k (quarter c / 4) of 16 tokens, the wave's own; then 32 k of 16 ranks, or 1 KiB of B's rows.
  int tr, tchunk;
  km_dma_target(wave * 64 + lane, tr, tchunk);
  const uint16_t* x = a.X + int64_t(tokens[tr]) * a.ldx + col0;
  auto issue = [&](int step) {
    const uint32_t at = lds + uint32_t(step % NS) * (COPIES * 1024);
    const int k0 = (step * a.splits + split) * kDownK;
    // Past K the last values stand in, against zeros of the adapter.
#pragma unroll
    for (int i = 0; i < 4; ++i)
      lora_dma16(x + min(k0 + 32 * i + 8 * tchunk, K - 8),
                 __builtin_amdgcn_readfirstlane(at + uint32_t(wave + 4 * i) * 1024));
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int f = wave + 4 * i;
      const uint16_t* p;
      if constexpr (BMAJOR) {
        const int e = f * 64 + lane;
        p = w + int64_t(col0 + min(k0 + e / (2 * RT), K - 1)) * a.wrows + r0 + min(8 * (e % (2 * RT)), nr - 8);
      } else {
        int r, chunk;
        km_dma_target((f % RT) * 64 + lane, r, chunk);
        p = w + int64_t(r0 + min(r, nr - 1)) * K + min(k0 + 32 * (f / RT) + 8 * chunk, K - 8);
      }
      lora_dma16(p, __builtin_amdgcn_readfirstlane(at + uint32_t(16 + f) * 1024));
    }
  };
  f32x4 acc[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int steps = ((K + kDownK - 1) / kDownK - split + a.splits - 1) / a.splits;  // at least one
  for (int s = 0; s < NS - 1 && s < steps; ++s) issue(s);
  for (int s = 0; s < steps; ++s) {
    // stage s has landed, and the stage that is filled next has been read by every wave
    wait_stages<PER>(min(steps - 1 - s, NS - 2));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    block_sync();
    if (s + NS - 1 < steps) issue(s + NS - 1);
    const u32x4* st = s_mem + s % NS * (COPIES * 64);
    const int left = K - (s * a.splits + split) * kDownK;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const u32x4 xf = km_frag(st + h * 256, 16 * wave, lane);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        u32x4 f = BMAJOR ? lora_tr_frag(reinterpret_cast<const char*>(st + 1024) + 32 * h * (32 * RT), 32 * RT, 16 * t, lane)
                         : km_frag(st + 1024 + h * 64 * RT, 16 * t, lane);
        if (left < kDownK) f = 32 * h + 8 * q < left ? f : zero16();
        acc[t] = mfma16(xf, f, acc[t]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int tok = 16 * wave + 4 * q + i;
      if (tok < tile.count && t * 16 + row < nr) out[int64_t(tok) * a.R + t * 16 + row] = acc[t][i];
    }
}

// The same for a tile of up to 16 tokens, where the adapter is the operand that
// counts: the waves take 128 of every 512 k and add up through LDS, and
// fragments come straight from memory into registers, four steps of 32 k ahead.
template <int RT, bool BMAJOR>
__device__ __forceinline__ void lora_down_few(const LoraDown& a, const LoraTile& tile, int tok, int split, int K,
                                              int col0, int r0, int nr, float* out, u32x4* s_mem) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, q = lane >> 4;
  const uint16_t* xr = a.X + int64_t(tok) * a.ldx + col0;
  const uint16_t* w = a.W + int64_t(tile.adapter) * a.wstride;
  const int k0 = split * kLoraSlice, next = a.splits * kLoraSlice;
  f32x4 acc[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  u32x4 x[4];
  auto load_x = [&](int kw, int j) { x[j] = ld16(xr + min(kw + 32 * j + 8 * q, K - 8)); };
  if constexpr (!BMAJOR) {
    u32x4 wf[RT][4];
    const uint16_t* wr[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) wr[t] = w + int64_t(r0 + min(t * 16 + row, nr - 1)) * K;
    auto load_w = [&](int kw, int j) {
#pragma unroll
      for (int t = 0; t < RT; ++t) wf[t][j] = ld16(wr[t] + min(kw + 32 * j + 8 * q, K - 8));
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) load_x(k0 + wave * 128, j), load_w(k0 + wave * 128, j);
    for (int kb = k0; kb < K; kb += next) {
      const int kw = kb + wave * 128;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool in = kw + 32 * j + 8 * q < K;
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t] = mfma16(x[j], in ? wf[t][j] : zero16(), acc[t]);
        if (kb + next < K) load_x(kw + next, j), load_w(kw + next, j);
      }
    }
  } else {
    constexpr int CH = 2 * RT;  // 16-byte chunks per row of 16 RT ranks; a wave's 32 rows in LDS at a time
    w += int64_t(col0) * a.wrows + r0;
    u32x4* sw = s_mem + wave * 32 * CH;
    u32x4 v[RT][4];
    auto load_w = [&](int kw, int j) {
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const int e = i * 64 + lane;
        v[i][j] = ld16(w + int64_t(min(kw + 32 * j + e / CH, K - 1)) * a.wrows + min(8 * (e % CH), nr - 8));
      }
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) load_x(k0 + wave * 128, j), load_w(k0 + wave * 128, j);
    for (int kb = k0; kb < K; kb += next) {
      const int kw = kb + wave * 128;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RT; ++i) sw[i * 64 + lane] = v[i][j];
        __syncthreads();
        const bool in = kw + 32 * j + 8 * q < K;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const u32x4 f = lora_tr_frag(reinterpret_cast<const char*>(sw), 32 * RT, 16 * t, lane);
          acc[t] = mfma16(x[j], in ? f : zero16(), acc[t]);
        }
        if (kb + next < K) load_x(kw + next, j), load_w(kw + next, j);
      }
    }
  }
  float* s_red = reinterpret_cast<float*>(s_mem);  // [4 waves][16 tokens][16 RT ranks, 1 spare]
  constexpr int P = 16 * RT + 1;
  __syncthreads();
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) s_red[(wave * 16 + 4 * q + i) * P + t * 16 + row] = acc[t][i];
  __syncthreads();
  for (int e = threadIdx.x; e < 256 * RT; e += 256) {
    const int i = e / (16 * RT), c = e % (16 * RT);
    const float v = (s_red[i * P + c] + s_red[(16 + i) * P + c]) + (s_red[(32 + i) * P + c] + s_red[(48 + i) * P + c]);
    if (i < tile.count && c < nr) out[int64_t(i) * a.R + c] = v;
  }
}

template <int RT, bool BMAJOR>
__global__ __launch_bounds__(256, 2) void lora_down_kernel(LoraDown a, LoraPlan plan) {
  __shared__ u32x4 s_mem[kDownSlots<RT>];
  const int split = blockIdx.x % a.splits, ti = blockIdx.x / a.splits;
  const int* tokens = plan.tokens + ti * kLoraTile;
  const int tok = tokens[threadIdx.x & 15];
  const LoraTile tile = plan.tile(plan.tiles, ti, 3);
  if (tile.count == 0 || tile.adapter >= plan.n) return;
  const int chunk = blockIdx.y % a.chunks, part = BMAJOR ? blockIdx.y / a.chunks : 0;
  const int r0 = chunk * 16 * RT, nr = min(16 * RT, a.wrows - r0);
  const int col0 = BMAJOR ? a.off[part] : 0, K = BMAJOR ? a.width[part] : a.K;
  float* out = a.part + (int64_t(split) * plan.T + tile.pos) * a.R + part * a.wrows + r0;
  // A narrower part than the widest may have nothing for this split: tiles of few tokens deal it in slices, others in stages.
  if (split * (tile.count <= 16 ? kLoraSlice : kDownK) >= K) {
    for (int e = threadIdx.x; e < tile.count * nr; e += 256) out[int64_t(e / nr) * a.R + e % nr] = 0.0f;
  } else if (tile.count <= 16) {
    lora_down_few<RT, BMAJOR>(a, tile, tok, split, K, col0, r0, nr, out, s_mem);
  } else {
    lora_down_wide<RT, BMAJOR>(a, tile, tokens, split, K, col0, r0, nr, out, s_mem);
  }
}

// Sum of the splits' partial sums at p, four values.  Four loads are in flight at a time, since the blocks of Y wait for
// them before they begin (203 tokens of 40 adapters, 22016 columns, 64 ranks: 30.8 us, with one 33.9; 64 tokens of 32
// adapters, 5120 columns, 16 ranks: 6.6 and 8.2).
__device__ __forceinline__ f32x4 sum_splits(const float* p, int splits, int64_t stride) {
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < splits; s += 4) {
    f32x4 u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = *reinterpret_cast<const f32x4*>(p + min(s + i, splits - 1) * stride);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (s + i < splits) v += u[i];
  }
  return v;
}

// ---------------------------------------------------------------- bf16 terms of fp32 values

// The first N >= 2 terms of eight values: each term is what the ones before left, rounded.  The first is held to the
// largest finite bf16 value, which a finite value may round past: what is beyond goes to the second, and so do
// infinities and NaN.  No later term can.
template <int N>
__device__ __forceinline__ void lora_terms(const float (&x)[8], u32x4 (&f)[N]) {
  constexpr float kMost = 0x1.fep127f;
  // What the second term leaves: nothing of an infinity.
  auto rest = [](float v, uint32_t term) { return (term & 0x7f80u) == 0x7f80u ? 0.0f : v - __uint_as_float(term << 16); };
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    float a = x[2 * p], b = x[2 * p + 1];
    f[0][p] = pack_bf16x2(__builtin_amdgcn_fmed3f(a, -kMost, kMost), __builtin_amdgcn_fmed3f(b, -kMost, kMost));
    a -= bf16_lo(f[0][p]), b -= bf16_hi(f[0][p]);
#pragma unroll
    for (int i = 1; i < N; ++i) {
      f[i][p] = pack_bf16x2(a, b);
      a = rest(a, f[i][p] & 0xffffu), b = rest(b, f[i][p] >> 16);
    }
  }
}

struct LoraTerms {
  const float* part;  // [splits][T][R]: Q before its scale
  int splits, R;
  const float* scale;
  const float* P;  // [T, R] in the tokens' order
  int r, parts;
  uint16_t* Qn;  // [tile][64][blocks of 16 ranks][2 terms][16], or nullptr
  uint16_t* Qt;  // [tile][2][blocks][3 terms][64 lanes][8]: fragments over 32 tokens
  uint16_t* Pt;  // the same of P, the parts' blocks one after the other
  int blocksQ, blocksP;  // blocks of 16 ranks (0: not wanted)
};

// Splits Q and P into the bf16 terms that the products below multiply with, once for all columns: of Q
// two terms row by row for dX, and three of both in the order in which a wave's lanes hold them as a
// fragment with the tokens contracted.  Rows past a tile's tokens and ranks past the last are zeros.
__global__ __launch_bounds__(256) void lora_terms_kernel(LoraTerms a, LoraPlan plan) {
  __shared__ float s_v[64 * 17];
  const int blocks = a.blocksQ + a.blocksP, ti = blockIdx.x / blocks, b = blockIdx.x % blocks;
  const int row = threadIdx.x >> 2, c = 4 * (threadIdx.x & 3);
  const int token = plan.tokens[ti * kLoraTile + row];
  const LoraTile tile = plan.tile(plan.tiles, ti, 3);
  if (tile.count == 0 || tile.adapter >= plan.n) return;
  const bool isq = b < a.blocksQ;
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  if (isq) {
    if (row < tile.count && 16 * b + c < a.R)
      v = sum_splits(a.part + int64_t(tile.pos + row) * a.R + 16 * b + c, a.splits, int64_t(plan.T) * a.R) *
          a.scale[tile.adapter];
  } else {
    const int per = a.blocksP / a.parts, part = (b - a.blocksQ) / per, k = 16 * ((b - a.blocksQ) % per) + c;
    if (row < tile.count && k < a.r) v = *reinterpret_cast<const f32x4*>(a.P + int64_t(token) * a.R + part * a.r + k);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) s_v[row * 17 + c + i] = v[i];
  __syncthreads();
  if (isq && a.Qn && threadIdx.x < 128) {
    const int r = threadIdx.x >> 1, h = threadIdx.x & 1;
    float x[8];
    u32x4 f[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s_v[r * 17 + 8 * h + i];
    lora_terms<2>(x, f);
    uint16_t* out = a.Qn + ((int64_t(ti) * kLoraTile + r) * a.blocksQ + b) * 32 + 8 * h;
    st16(out, f[0]);
    st16(out + 16, f[1]);
  }
  uint16_t* frag = isq ? a.Qt : a.Pt;
  if (frag && threadIdx.x >= 128) {
    const int h = (threadIdx.x >> 6) & 1, lane = threadIdx.x & 63, k = lane & 15, q = lane >> 4;
    const int fb = isq ? b : b - a.blocksQ, fblocks = isq ? a.blocksQ : a.blocksP;
    float x[8];
    u32x4 f[3];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s_v[(32 * h + 8 * q + i) * 17 + k];
    lora_terms<3>(x, f);
    uint16_t* out = frag + ((int64_t(ti) * 2 + h) * fblocks + fb) * (3 * 512) + lane * 8;
#pragma unroll
    for (int i = 0; i < 3; ++i) st16(out + 512 * i, f[i]);
  }
}

// ---------------------------------------------------------------- products with the rank contracted

struct LoraUp {
  const float* part;  // [splits][T][R], rows in the plan's order
  int splits, R;
  const float* scale;
  const uint16_t* W;  // one adapter's weights: B [d_out, r] or A [R, d_in]
  int64_t wstride;
  int r;
  const uint16_t* base;
  int64_t ld_base;
  uint16_t* Y;
  int64_t ldy;
  float* P;  // [T, R] in the tokens' order, or nullptr
  const uint16_t* Qn;  // dX: Q's terms instead of `part`
  int blocksQ;
  int parts, span;  // columns per block
  int off[kLoraMaxParts], width[kLoraMaxParts], first[kLoraMaxParts + 1];  // first block of each part
};

// A row of a tile's rank terms in LDS: per 16 ranks the first terms, then the second; 8 spare values.
template <int RT>
constexpr int kUpPitch = 32 * RT + 8;

// Stages the ranks of `rows` rows of the tile, zeros past the tile's tokens
// and past r; with `keep`, the block also stores them to P.
template <int RT>
__device__ __forceinline__ void lora_stage(const LoraUp& a, const LoraPlan& plan, const LoraTile& tile, int ti, int rows,
                                           int col0, bool keep, uint16_t* s_terms) {
  const float c = a.scale[tile.adapter];
  for (int e = threadIdx.x; e < rows * 2 * RT; e += 256) {
    const int row = e / (2 * RT), h = e % (2 * RT), k = 8 * h;
    float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (row < tile.count && k < a.r) {
      const float* src = a.part + int64_t(tile.pos + row) * a.R + col0 + k;
      const int64_t stride = int64_t(plan.T) * a.R;
      const f32x4 lo = sum_splits(src, a.splits, stride), hi = sum_splits(src + 4, a.splits, stride);
      if (keep) {
        float* p = a.P + int64_t(plan.tokens[ti * kLoraTile + row]) * a.R + col0 + k;
        *reinterpret_cast<f32x4*>(p) = lo;
        *reinterpret_cast<f32x4*>(p + 4) = hi;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = lo[i] * c, v[4 + i] = hi[i] * c;
    }
    u32x4 f[2];
    lora_terms<2>(v, f);
    uint16_t* out = s_terms + row * kUpPitch<RT> + (h >> 1) * 32 + 8 * (h & 1);
    st16(out, f[0]);
    st16(out + 16, f[1]);
  }
}

// A tile of tokens without an adapter: columns of base, and zeros in P.
__device__ __forceinline__ void lora_copy(const LoraUp& a, const LoraPlan& plan, const LoraTile& tile, int ti, int col0,
                                          int cols, int rank0, int ranks) {
  const int* tokens = plan.tokens + ti * kLoraTile;
  if (a.base != a.Y) {
    const int cpr = cols / 8;
    for (int e = threadIdx.x; e < tile.count * cpr; e += 256) {
      const int64_t t = tokens[e / cpr];
      const int c = col0 + 8 * (e % cpr);
      st16(a.Y + t * a.ldy + c, ld16(a.base + t * a.ld_base + c));
    }
  }
  for (int e = threadIdx.x; e < tile.count * ranks; e += 256)
    a.P[int64_t(tokens[e / ranks]) * a.R + rank0 + e % ranks] = 0.0f;
}

// Columns whose weights are in LDS at a time.
template <int RT>
constexpr int kUpCols = lora_up_cols(RT);

// B's chunk of 8 ranks c of row o is at c ^ up_swizzle(o): the rows that eight lanes read at once then lie in
// different 16-byte columns.
template <int RT>
__device__ __forceinline__ int up_swizzle(int o) {
  if constexpr (RT == 1)
    return (o >> 3) & 1;
  else if constexpr (RT == 2)
    return ((o >> 1) & 1) | ((o >> 3) & 1) << 1;
  else
    return (o & 3) | ((o >> 3) & 1) << 2;
}

// Swaps a of the upper eight lanes of every 16 with b of the lower eight.
__device__ __forceinline__ void lora_swap8(u32x4& a, u32x4& b, bool lower) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t give = lower ? b[i] : a[i];
    const uint32_t got = uint32_t(__builtin_amdgcn_mov_dpp(int(give), 0x128, 0xf, 0xf, true));  // row_ror:8
    a[i] = lower ? a[i] : got;
    b[i] = lower ? got : b[i];
  }
}

// Y = base + c P B^T, and with TR dX = base + Q A.  The matrix product's rows
// are output columns and its columns tokens, with the columns dealt so that
// two instructions leave eight consecutive ones of one token in each lane.  One
// instruction's 32 k hold the two terms of 16 ranks.  base and Y move between
// memory and registers as 128 bytes of eight tokens at a time, 64 columns of 16
// tokens per unit, and eight lanes of every 16 swap halves on the way: copying
// 8192 rows of 11008 columns took 72 us so (5.0 TB/s) and 98 us as 64 bytes of 16 tokens, and not
// keeping either in the caches pays at 128 bytes only (79 -> 75 us).
//
// A block takes 64 tokens and `span` columns; a wave 16 of the tokens and all
// columns, or a share of the columns where there are fewer tokens.  The weights of kUpCols
// columns at a time are copied into LDS, which all waves share; A's come back transposed.
// base is loaded two units ahead.  More ranks than fit go in several rounds (MULTI),
// with the sums of one round of columns held in registers.
template <int RT, bool TR, bool MULTI>
__device__ __forceinline__ void lora_up_body(const LoraUp& a, const LoraPlan& plan, const LoraTile& tile, int ti,
                                             int part, int cb, bool keep, int subs, u32x4* s_w, uint16_t* s_terms) {
  constexpr int COLS = kUpCols<RT>, UN = 2, CPR = COLS / 8, COPIES = COLS * RT / 32, UNIT = 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, q = lane >> 4;
  const int off = a.off[part], end = min(cb + a.span, a.width[part]), ranks = TR ? a.R : a.r;
  const int share = 4 / subs, first = 16 * (wave % subs), o0 = cb + UNIT * (wave / subs), stride = UNIT * share;
  const int units = (end - cb + stride - 1) / stride, per = COLS / stride;  // of a wave: in all, and per weights in LDS
  const uint16_t* w = a.W + int64_t(tile.adapter) * a.wstride + int64_t(off) * (TR ? 1 : a.r);
  // This lane's 16 bytes of a unit's two moves: tokens row % 8 and row % 8 + 8, columns 32 (row / 8) + 8 q.
  const bool lower = row < 8;
  const int mc = (lower ? 0 : 32) + 8 * q;
  const uint16_t* br[2];
  uint16_t* yr[2];
  bool on[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = first + (row & 7) + 8 * h;
    const int64_t tok = plan.tokens[ti * kLoraTile + i];
    br[h] = a.base + tok * a.ld_base + off;
    yr[h] = a.Y + tok * a.ldy + off;
    on[h] = i < tile.count;
  }
  u32x4 b[UN][2];
  auto load_base = [&](int i, int u) {
    const int o = o0 + stride * i;
    if (o < end) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        b[u][h] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(br[h] + min(o + mc, end - 8)));
    }
  };
  if constexpr (!MULTI) {
#pragma unroll
    for (int u = 0; u < UN; ++u) load_base(u, u);
  }
  const uint32_t lds = lds_addr(s_w);
  // Weights of columns [c, c + COLS) and ranks [k0, k0 + 16 RT); none past the last column, whose products are
  // not stored; past the last rank others stand in, against zero terms.
  auto stage_w = [&](int c, int k0) {
    block_sync();
#pragma unroll
    for (int i = 0; i < COPIES / 4; ++i) {
      const int s = (wave + 4 * i) * 64 + lane;
      const uint32_t at = __builtin_amdgcn_readfirstlane(lds + uint32_t(wave + 4 * i) * 1024);
      if constexpr (TR) {
        const int r = s / CPR, x = s % CPR, chunk = (((x >> 2) ^ (r & 3)) << 2) | (x & 3);
        const uint16_t* p = w + int64_t(min(k0 + r, ranks - 1)) * a.width[0] + c + 8 * chunk;
        if (c + 8 * chunk < end) lora_dma16(p, at);
      } else {
        const int r = s / (2 * RT), chunk = (s % (2 * RT)) ^ up_swizzle<RT>(r);
        const uint16_t* p = w + int64_t(c + r) * a.r + min(8 * chunk, ranks - 8);
        if (c + r < end) lora_dma16(p, at);
      }
    }
  };
  auto weights = [&](int o, int j, int t) {  // o: the run's first column within the weights in LDS
    if constexpr (TR) {
      // The lane reads four columns of a rank; columns of a run are dealt 8 (row % 4) + 4 j.
      const int r = 16 * t + 8 * (q & 1) + (row >> 2), x = o / 8 + (row & 3);
      const char* p = reinterpret_cast<const char*>(s_w + r * CPR + ((((x >> 2) ^ (r & 3)) << 2) | (x & 3))) + 8 * j;
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p);
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p + 4 * CPR * 16));
      u32x4 f;
      __builtin_memcpy(&f, &lo, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&f) + 8, &hi, 8);
      return f;
    } else {
      const int r = o + 8 * (row >> 2) + 4 * j + (row & 3);
      return s_w[r * 2 * RT + ((2 * t + (q & 1)) ^ up_swizzle<RT>(r))];
    }
  };
  u32x4 pf[RT];
  auto load_terms = [&](int k0) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if constexpr (TR) {
        const int block = k0 / 16 + t;
        pf[t] = block < a.blocksQ ? ld16(a.Qn + ((int64_t(ti) * kLoraTile + first + row) * a.blocksQ + block) * 32 + 8 * q)
                                  : zero16();
      } else {
        pf[t] = ld16(s_terms + (first + row) * kUpPitch<RT> + t * 32 + 8 * q);
      }
    }
  };
  // d[g][j]: run g's columns 4 j .. + 3 of this lane's eight.
  auto multiply = [&](int o, f32x4 (&d)[2][2]) {
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int t = 0; t < RT; ++t) d[g][j] = mfma16(weights(o + 32 * g, j, t), pf[t], d[g][j]);
  };
  auto store = [&](int o, u32x4 (&v)[2], const f32x4 (&d)[2][2]) {
    lora_swap8(v[0], v[1], lower);
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int p = 0; p < 4; ++p)
        v[g][p] = pack_bf16x2(bf16_lo(v[g][p]) + d[g][p >> 1][2 * (p & 1)], bf16_hi(v[g][p]) + d[g][p >> 1][2 * (p & 1) + 1]);
    lora_swap8(v[0], v[1], lower);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (on[h] && o + mc < end) __builtin_nontemporal_store(v[h], reinterpret_cast<u32x4*>(yr[h] + o + mc));
  };
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  if constexpr (MULTI) {
    constexpr int MU = COLS / UNIT;
    f32x4 d[MU][2][2];
#pragma unroll
    for (int u = 0; u < MU; ++u) d[u][0][0] = d[u][0][1] = d[u][1][0] = d[u][1][1] = zero;
    for (int k0 = 0; k0 < ranks; k0 += 16 * RT) {
      stage_w(cb, k0);
      load_terms(k0);
      wait_vmcnt<0>();
      block_sync();
#pragma unroll
      for (int u = 0; u < MU; ++u)
        if (u < per) multiply(o0 - cb + stride * u, d[u]);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
#pragma unroll
    for (int u = 0; u < MU; ++u)
      if (u < units) {
        load_base(u, 0);
        store(o0 + stride * u, b[0], d[u]);
      }
  } else {
    stage_w(cb, 0);
    if constexpr (!TR)
      lora_stage<RT>(a, plan, tile, ti, 16 * subs, part * a.r, keep, s_terms);
    else
      load_terms(0);
    wait_vmcnt<0>();
    __syncthreads();
    if constexpr (!TR) load_terms(0);
    for (int i0 = 0; i0 < units; i0 += UN) {
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        const int i = i0 + u;
        if (i >= units) break;  // uniform, in the block too
        if (i > 0 && i % per == 0) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          stage_w(cb + i / per * COLS, 0);
          wait_vmcnt<0>();
          block_sync();
        }
        f32x4 d[2][2] = {{zero, zero}, {zero, zero}};
        multiply(o0 - cb + stride * (i % per), d);
        store(o0 + stride * i, b[u], d);
        load_base(i + UN, u);
      }
    }
  }
}

template <int RT, bool TR, bool MULTI>
__device__ __forceinline__ void lora_up_block(const LoraUp& a, const LoraPlan& plan, int block, u32x4* s_w, uint16_t* s_terms) {
  const int blocks = a.first[a.parts], ti = block / blocks, cbk = block % blocks;
  const LoraTile tile = plan.tile(plan.tiles, ti, 3);
  if (tile.count == 0) return;
  int part = 0;
  while (part + 1 < a.parts && cbk >= a.first[part + 1]) ++part;
  const int cb = (cbk - a.first[part]) * a.span;
  const bool keep = a.P != nullptr && cb == 0;
  if (tile.adapter >= plan.n)
    lora_copy(a, plan, tile, ti, a.off[part] + cb, min(a.span, a.width[part] - cb), part * a.r, keep ? a.r : 0);
  else
    lora_up_body<RT, TR, MULTI>(a, plan, tile, ti, part, cb, keep, tile.count <= 16 ? 1 : tile.count <= 32 ? 2 : 4, s_w,
                                s_terms);
}

// Slots of 16 bytes that the weights take.
template <int RT>
constexpr int kUpSlots = kUpCols<RT> * 2 * RT;

// At 16 ranks registers for six blocks per CU: 4099 tokens of 12 adapters, 11008 columns 43.2 us, 46.1 without.
template <int RT, bool TR, bool MULTI>
__global__ __launch_bounds__(256, RT == 8 && !TR ? 1 : RT == 1 ? 6 : 2) void lora_up_kernel(LoraUp a, LoraPlan plan) {
  __shared__ u32x4 s_w[kUpSlots<RT>];
  __shared__ __align__(16) uint16_t s_terms[TR ? 8 : 64 * kUpPitch<RT>];
  lora_up_block<RT, TR, MULTI>(a, plan, blockIdx.x, s_w, s_terms);
}

// ---------------------------------------------------------------- products with the tokens contracted

struct LoraGrad {
  const uint16_t* X;  // the tall matrix
  int64_t ldx;
  const uint16_t* terms;  // fragments of Q or P (lora_terms_kernel)
  int tblocks;            // their blocks of 16 ranks, all parts
  int pblocks;            // of one part
  int r;                  // ranks of a part (R for dA)
  const float* scale;
  float* out;       // [n, ranks, cols] (dA) or [n, cols, r] (dB)
  int64_t ostride;  // elements per adapter
  int ocols;        // all columns of the tall matrix
  float* part;      // the same, per gradient tile
  int parts, chunks;  // chunks: blocks of 16 RT ranks
  int off[kLoraMaxParts], width[kLoraMaxParts], first[kLoraMaxParts + 1];
};

// Stages in LDS: two blocks per CU at 64 ranks (20 KiB a stage), three at 16 (11 KiB).
template <int RT>
constexpr int kGradStages = RT == 4 ? 3 : 4;

// One block sums the products of up to 2048 tokens of one adapter for 128
// columns and 16 RT ranks.  A stage of the pipeline is 32 tokens: their rows
// of the tall matrix and the terms' fragments are copied into LDS two or three stages ahead, and
// the rows come back transposed, so that the tokens become the contracted
// index.  The waves split ranks and columns, never tokens, so no sum crosses a wave.
// An adapter with one gradient tile is done; others leave partial sums.
template <int RT, bool DB>
__device__ __forceinline__ void lora_grad_body(const LoraGrad& a, const LoraPlan& plan, int block, u32x4* s_mem,
                                               int* s_tok) {
  constexpr int NS = kGradStages<RT>;
  constexpr int NC = 2 * RT;                  // 16-column fragments per wave: 128 RT / 4 columns
  constexpr int COPIES = 8 + 3 * RT;          // 1 KiB each: 4 rows of 128 columns, or one fragment
  constexpr int PER = (COPIES + 3) / 4;       // per wave
  const int chunk = block % a.chunks, cbk = block / a.chunks % a.first[a.parts], gi = block / a.chunks / a.first[a.parts];
  const LoraTile tile = plan.tile(plan.gtiles, gi, 4 + plan.glen);
  if (tile.count == 0) return;
  int part = 0;
  while (part + 1 < a.parts && cbk >= a.first[part + 1]) ++part;
  const int cb = (cbk - a.first[part]) * kLoraGradCols, width = a.width[part];
  const int rb0 = chunk * RT;  // first block of 16 ranks within the part
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, q = lane >> 4;
  const int steps = (tile.count + 31) / 32;
  for (int i = threadIdx.x; i < 32 * steps; i += 256) s_tok[i] = plan.tokens[tile.pos * kLoraTile + i];
  __syncthreads();
  const uint32_t lds = lds_addr(s_mem);
  const uint16_t* x = a.X + a.off[part] + cb;
  const uint16_t* terms = a.terms + (int64_t(tile.pos) * 2 * a.tblocks + part * a.pblocks) * (3 * 512) + lane * 8;
  auto issue = [&](int step) {
    const uint32_t at = lds + uint32_t(step % NS) * (COPIES * 1024);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = min(wave + 4 * i, COPIES - 1);  // uniform; a wave with fewer repeats the last
      const void* p;
      if (c < 8) {
        int r, chunk;
        mn_dma_target<128>(c * 64 + lane, r, chunk);
        p = x + int64_t(s_tok[32 * step + r]) * a.ldx + min(8 * chunk, width - cb - 8);
      } else {
        const int f = c - 8, rb = min(rb0 + f / 3, a.pblocks - 1);
        p = terms + (int64_t(step) * a.tblocks + rb) * (3 * 512) + (f % 3) * 512;
      }
      lora_dma16(p, __builtin_amdgcn_readfirstlane(at + uint32_t(c) * 1024));
    }
  };
  f32x4 acc[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) acc[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int rb = wave % RT, cw = wave / RT * (16 * NC);  // this wave's ranks and columns
  for (int s = 0; s < NS - 1 && s < steps; ++s) issue(s);
  for (int s = 0; s < steps; ++s) {
    // stage s has landed, and the stage that is filled next has been read by every wave
    wait_stages<PER>(min(steps - 1 - s, NS - 2));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    block_sync();
    if (s + NS - 1 < steps) issue(s + NS - 1);
    const u32x4* st = s_mem + s % NS * (COPIES * 64);
    u32x4 f[3];
#pragma unroll
    for (int m = 0; m < 3; ++m) f[m] = st[(8 + 3 * rb + m) * 64 + lane];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const u32x4 xf = mn_frag<128>(st, cw + 16 * c, lane);
#pragma unroll
      for (int m = 0; m < 3; ++m) acc[c] = mfma16(xf, f[m], acc[c]);
    }
  }
  const int rank = 16 * (rb0 + rb) + row;
  if (rank >= a.r) return;
  float* out = tile.only ? a.out + tile.adapter * a.ostride : a.part + gi * a.ostride;
  const float scale = DB ? a.scale[tile.adapter] : 1.0f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = cw + 16 * c + 4 * q;
    if (cb + col >= width) continue;
    const int64_t at = a.off[part] + cb + col;
    if constexpr (DB) {
#pragma unroll
      for (int i = 0; i < 4; ++i) out[(at + i) * a.r + rank] = acc[c][i] * scale;
    } else {
      *reinterpret_cast<f32x4*>(out + rank * int64_t(a.ocols) + at) = acc[c];
    }
  }
}

// Slots of 16 bytes that the stages take.
template <int RT>
constexpr int kGradSlots = kGradStages<RT> * (8 + 3 * RT) * 64;

// Both gradients in one launch: dA's blocks, over all parts' ranks, then dB's, over one part's.
template <int RTA, int RTB>
__global__ __launch_bounds__(256, 2) void lora_grad_kernel(LoraGrad a, int blocksA, LoraGrad b, LoraPlan plan) {
  __shared__ u32x4 s_mem[kGradSlots<RTA> > kGradSlots<RTB> ? kGradSlots<RTA> : kGradSlots<RTB>];
  __shared__ int s_tok[kLoraGradMost];
  if (int(blockIdx.x) < blocksA)
    lora_grad_body<RTA, false>(a, plan, blockIdx.x, s_mem, s_tok);
  else
    lora_grad_body<RTB, true>(b, plan, blockIdx.x - blocksA, s_mem, s_tok);
}

// All that waits for the terms alone in one launch, the gradients, then dX: 15.2 -> 9.9 us for 1000 tokens, 2816 and
// 2056 columns, 24 ranks, and still 102 -> 99 for 8192 tokens, 4096 and 11008 columns, 64 ranks.
template <int RTA, int RTB>
__global__ __launch_bounds__(256, 2) void lora_bwd_kernel(LoraGrad a, int blocksA, LoraGrad b, int blocksB, LoraUp u,
                                                          LoraPlan plan) {
  constexpr int G = kGradSlots<RTA> > kGradSlots<RTB> ? kGradSlots<RTA> : kGradSlots<RTB>;
  __shared__ u32x4 s_mem[G > kUpSlots<RTA> ? G : kUpSlots<RTA>];
  __shared__ int s_tok[kLoraGradMost];
  if (int(blockIdx.x) < blocksA)
    lora_grad_body<RTA, false>(a, plan, blockIdx.x, s_mem, s_tok);
  else if (int(blockIdx.x) < blocksA + blocksB)
    lora_grad_body<RTB, true>(b, plan, blockIdx.x - blocksA, s_mem, s_tok);
  else
    lora_up_block<RTA, true, false>(u, plan, blockIdx.x - blocksA - blocksB, s_mem, nullptr);
}

// The gradients of adapters with several tiles from their partial sums, in the
// tiles' order, and zeros for adapters that no token chose.
__global__ __launch_bounds__(256) void lora_grad_sum_kernel(const float* __restrict__ partA, float* __restrict__ dA,
                                                            int64_t sA, int blocksA, const float* __restrict__ partB,
                                                            float* __restrict__ dB, int64_t sB, LoraPlan plan) {
  const int a = blockIdx.y, g0 = plan.gstart[a], g1 = plan.gstart[a + 1];
  if (plan.head[0] != kLoraMagic || plan.head[1] != plan.T || plan.head[2] != plan.n || g1 - g0 == 1) return;
  const bool second = int(blockIdx.x) >= blocksA;
  const float* part = second ? partB : partA;
  const int64_t stride = second ? sB : sA;
  float* out = (second ? dB : dA) + a * stride;
  const int64_t e = int64_t(second ? blockIdx.x - blocksA : blockIdx.x) * 1024 + 4 * threadIdx.x;
  if (e >= stride) return;
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int g = g0; g < g1; ++g) v += *reinterpret_cast<const f32x4*>(part + g * stride + e);
  *reinterpret_cast<f32x4*>(out + e) = v;
}

// ---------------------------------------------------------------- launchers

hipError_t launch_lora_plan(const int* adapter, int T, int n, void* plan, hipStream_t s) {
  const LoraPlanLayout L = lora_plan_layout(T, n);
  int* w = static_cast<int*>(plan);
  LoraPlanOut out = {w, reinterpret_cast<LoraTile*>(w + L.tiles), w + L.tokens, {}, {}};
  for (int i = 0; i < kLoraGradLens; ++i)
    out.gtiles[i] = reinterpret_cast<LoraTile*>(w + L.gtiles[i]), out.gstart[i] = w + L.gstart[i];
  const int waves = n <= 1024 ? 16 : 8;  // whose counts fit LDS
  const size_t lds = size_t(waves * (n + 1) + 1) * sizeof(int) + size_t(n + 2) * sizeof(LoraFirst) + size_t(n + 1) * sizeof(int);
  if (waves == 16) hipLaunchKernelGGL(lora_plan_kernel<16>, dim3(1), dim3(1024), lds, s, adapter, T, n, out);
  else hipLaunchKernelGGL(lora_plan_kernel<8>, dim3(1), dim3(512), lds, s, adapter, T, n, out);
  return hipGetLastError();
}

static int lora_max_tiles(const LoraShape& z) { return int(lora_plan_layout(z.T, z.n).max_tiles); }

template <bool BMAJOR>
static hipError_t launch_down(const LoraDown& a, const LoraPlan& plan, int tiles, int rt, int blocks_y, hipStream_t s) {
  const dim3 grid(unsigned(tiles) * unsigned(a.splits), unsigned(blocks_y)), block(256);
  switch (rt) {
    case 1: hipLaunchKernelGGL((lora_down_kernel<1, BMAJOR>), grid, block, 0, s, a, plan); break;
    case 2: hipLaunchKernelGGL((lora_down_kernel<2, BMAJOR>), grid, block, 0, s, a, plan); break;
    default: hipLaunchKernelGGL((lora_down_kernel<4, BMAJOR>), grid, block, 0, s, a, plan); break;
  }
  return hipGetLastError();
}

// Deals the parts' columns to blocks; returns how many there are.
template <bool TR>
static int up_blocks(LoraUp& u, int ranks, int tiles, const LoraPlan& plan) {
  u.span = lora_up_span(u.width, u.parts, plan.T, tiles, ranks, TR);
  for (int p = 0, off = 0; p < u.parts; ++p) {
    u.off[p] = off;
    off += u.width[p];
    u.first[p + 1] = u.first[p] + (u.width[p] + u.span - 1) / u.span;
  }
  return tiles * u.first[u.parts];
}

template <bool TR>
static hipError_t launch_up(LoraUp& u, int ranks, int tiles, const LoraPlan& plan, hipStream_t s) {
  const dim3 grid(unsigned(up_blocks<TR>(u, ranks, tiles, plan))), block(256);
  if (ranks <= 16) hipLaunchKernelGGL((lora_up_kernel<1, TR, false>), grid, block, 0, s, u, plan);
  else if (ranks <= 32) hipLaunchKernelGGL((lora_up_kernel<2, TR, false>), grid, block, 0, s, u, plan);
  else if (ranks <= 64) hipLaunchKernelGGL((lora_up_kernel<4, TR, false>), grid, block, 0, s, u, plan);
  else if (ranks <= 128) hipLaunchKernelGGL((lora_up_kernel<8, TR, false>), grid, block, 0, s, u, plan);
  else if constexpr (TR) hipLaunchKernelGGL((lora_up_kernel<8, true, true>), grid, block, 0, s, u, plan);
  return hipGetLastError();
}

hipError_t launch_lora_fwd(const uint16_t* X, int64_t ldx, const uint16_t* A, const uint16_t* B, const float* scale,
                           const void* plan, const LoraShape& z, const uint16_t* base, int64_t ld_base, uint16_t* Y,
                           int64_t ldy, float* P, float* part, int splits, hipStream_t s) {
  const LoraPlan pl = lora_plan(plan, z.T, z.n, 0);
  const int R = z.parts * z.r, tiles = lora_max_tiles(z);
  LoraDown d = {};
  d.X = X, d.ldx = ldx, d.W = A, d.wstride = int64_t(R) * z.d_in, d.K = z.d_in, d.wrows = R;
  d.part = part, d.R = R;
  d.splits = splits;
  const int rt = lora_rank_tiles(R);
  d.chunks = (R + 16 * rt - 1) / (16 * rt);
  if (hipError_t e = launch_down<false>(d, pl, tiles, rt, d.chunks, s)) return e;
  LoraUp u = {};
  u.part = part, u.splits = splits, u.R = R, u.scale = scale;
  u.W = B, u.wstride = int64_t(z.d_out) * z.r, u.r = z.r;
  u.base = base, u.ld_base = ld_base, u.Y = Y, u.ldy = ldy, u.P = P;
  u.parts = z.parts;
  for (int p = 0; p < z.parts; ++p) u.width[p] = z.widths[p];
  return launch_up<false>(u, z.r, tiles, pl, s);
}

// The gradients that are asked for, and dX (unless u is null) in the same launch.
static hipError_t launch_grad(LoraGrad& a, LoraGrad& b, LoraUp* u, int tiles, const LoraPlan& plan, int gtiles,
                              hipStream_t s) {
  const int ra = lora_rank_tiles(a.r), rb = lora_rank_tiles(b.r);
  a.chunks = (a.r + 16 * ra - 1) / (16 * ra), b.chunks = (b.r + 16 * rb - 1) / (16 * rb);
  const int blocksA = gtiles * a.first[a.parts] * a.chunks, blocksB = gtiles * b.first[b.parts] * b.chunks;
  const int blocksU = u ? up_blocks<true>(*u, a.r, tiles, plan) : 0;
  const dim3 grid(unsigned(blocksA) + unsigned(blocksB) + unsigned(blocksU)), block(256);
  // dA has at least as many ranks as dB
#define GM_LORA_GRAD(RA, RB)                                                                                     \
  {                                                                                                              \
    if (u) hipLaunchKernelGGL((lora_bwd_kernel<RA, RB>), grid, block, 0, s, a, blocksA, b, blocksB, *u, plan);    \
    else hipLaunchKernelGGL((lora_grad_kernel<RA, RB>), grid, block, 0, s, a, blocksA, b, plan);                  \
  }
  if (ra == 1) GM_LORA_GRAD(1, 1)
  else if (ra == 2 && rb == 1) GM_LORA_GRAD(2, 1)
  else if (ra == 2) GM_LORA_GRAD(2, 2)
  else if (rb == 1) GM_LORA_GRAD(4, 1)
  else if (rb == 2) GM_LORA_GRAD(4, 2)
  else GM_LORA_GRAD(4, 4)
#undef GM_LORA_GRAD
  return hipGetLastError();
}

int lora_bwd_glen(const LoraShape& z) {
  int64_t blocks = (z.d_in + kLoraGradCols - 1) / kLoraGradCols;
  for (int p = 0; p < z.parts; ++p) blocks += (z.widths[p] + kLoraGradCols - 1) / kLoraGradCols;
  return lora_grad_len(z.T, blocks);
}

hipError_t launch_lora_bwd(const uint16_t* dY, int64_t lddy, const uint16_t* X, int64_t ldx, const uint16_t* A,
                           const uint16_t* B, const float* scale, const void* plan, const float* P,
                           const LoraShape& z, const uint16_t* base, int64_t ld_base, uint16_t* dX, int64_t lddx,
                           float* dA, float* dB, const LoraBwdWs& w, int splits, hipStream_t s) {
  const LoraPlanLayout L = lora_plan_layout(z.T, z.n);
  const int glen = lora_bwd_glen(z);
  const LoraPlan pl = lora_plan(plan, z.T, z.n, glen);
  const int R = z.parts * z.r, tiles = int(L.max_tiles), gtiles = int(L.max_gtiles[glen]);
  int off[kLoraMaxParts] = {}, widest = 0;
  for (int p = 0, at = 0; p < z.parts; ++p) {
    off[p] = at;
    at += z.widths[p];
    widest = z.widths[p] > widest ? z.widths[p] : widest;
  }
  hipError_t e = hipSuccess;
  if (dX || dA) {
    LoraDown d = {};
    d.X = dY, d.ldx = lddy, d.W = B, d.wstride = int64_t(z.d_out) * z.r, d.K = widest, d.wrows = z.r;
    d.part = w.part, d.R = R, d.splits = splits;
    for (int p = 0; p < z.parts; ++p) d.off[p] = off[p], d.width[p] = z.widths[p];
    const int rt = lora_rank_tiles(z.r);
    d.chunks = (z.r + 16 * rt - 1) / (16 * rt);
    if ((e = launch_down<true>(d, pl, tiles, rt, d.chunks * z.parts, s))) return e;
  }
  LoraTerms m = {};
  m.part = w.part, m.splits = splits, m.R = R, m.scale = scale, m.P = P, m.r = z.r, m.parts = z.parts;
  m.Qn = dX ? w.Qn : nullptr, m.Qt = dA ? w.Qt : nullptr, m.Pt = w.Pt;
  m.blocksQ = dX || dA ? (R + 15) / 16 : 0, m.blocksP = dB ? z.parts * ((z.r + 15) / 16) : 0;
  hipLaunchKernelGGL(lora_terms_kernel, dim3(unsigned(tiles) * unsigned(m.blocksQ + m.blocksP)), dim3(256), 0, s, m, pl);
  if ((e = hipGetLastError())) return e;
  LoraUp u = {};
  u.R = R, u.W = A, u.wstride = int64_t(R) * z.d_in, u.base = base, u.ld_base = ld_base, u.Y = dX, u.ldy = lddx;
  u.Qn = w.Qn, u.blocksQ = m.blocksQ, u.parts = 1, u.width[0] = z.d_in;
  const bool together = dX && (dA || dB) && R <= 64;
  if (dX && !together && (e = launch_up<true>(u, R, tiles, pl, s))) return e;
  LoraGrad ga = {}, gb = {};
  ga.r = R, gb.r = z.r;
  if (dA) {
    ga.X = X, ga.ldx = ldx, ga.terms = w.Qt, ga.tblocks = ga.pblocks = m.blocksQ;
    ga.out = dA, ga.ostride = int64_t(R) * z.d_in, ga.ocols = z.d_in, ga.part = w.partA, ga.parts = 1;
    ga.width[0] = z.d_in;
    ga.first[1] = (z.d_in + kLoraGradCols - 1) / kLoraGradCols;
  }
  if (dB) {
    gb.X = dY, gb.ldx = lddy, gb.terms = w.Pt, gb.tblocks = m.blocksP, gb.pblocks = m.blocksP / z.parts;
    gb.scale = scale, gb.out = dB, gb.ostride = int64_t(z.d_out) * z.r, gb.ocols = z.d_out, gb.part = w.partB;
    gb.parts = z.parts;
    for (int p = 0; p < z.parts; ++p) {
      gb.off[p] = off[p], gb.width[p] = z.widths[p];
      gb.first[p + 1] = gb.first[p] + (z.widths[p] + kLoraGradCols - 1) / kLoraGradCols;
    }
  }
  if ((dA || dB) && (e = launch_grad(ga, gb, together ? &u : nullptr, tiles, pl, gtiles, s))) return e;
  if (dA || dB) {
    const int64_t sA = int64_t(R) * z.d_in, sB = int64_t(z.d_out) * z.r;
    const unsigned bA = dA ? unsigned((sA + 1023) / 1024) : 0, bB = dB ? unsigned((sB + 1023) / 1024) : 0;
    hipLaunchKernelGGL(lora_grad_sum_kernel, dim3(bA + bB, unsigned(z.n)), dim3(256), 0, s, w.partA, dA, sA, int(bA),
                       w.partB, dB, sB, pl);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace gm
