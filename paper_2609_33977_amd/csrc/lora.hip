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

namespace gm {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short lora_i16x4 __attribute__((ext_vector_type(4)));

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
  const int* order;
  const int* start;
  const int* gstart;
  const LoraTile* tiles;
  const LoraTile* gtiles;
  const int* head;
  int T, n;
  // A plan made for other sizes is not followed: no tile of it is valid.
  __device__ __forceinline__ bool valid() const { return head[0] == kLoraMagic && head[1] == T && head[2] == n; }
};

static LoraPlan lora_plan(const void* plan, int T, int n) {
  const LoraPlanLayout L = lora_plan_layout(T, n);
  const int* w = static_cast<const int*>(plan);
  return {w + L.order, w + L.start, w + L.gstart, reinterpret_cast<const LoraTile*>(w + L.tiles),
          reinterpret_cast<const LoraTile*>(w + L.gtiles), w, T, n};
}

constexpr int kPlanWaves = 8;

// Lanes of the wave with the same key, as a mask.
__device__ __forceinline__ uint64_t same_key(int key, int bits, bool on) {
  uint64_t m = __ballot(on);
  for (int b = 0; b < bits; ++b) {
    const uint64_t one = __ballot((key >> b) & 1);
    m &= (key >> b) & 1 ? one : ~one;
  }
  return m;
}

// A stable counting sort of the tokens by adapter in one block: each wave
// counts and later places a contiguous run of tokens, so that equal adapters
// keep their tokens' order and sums over them do not depend on timing.  No
// atomics: the lanes of one key elect a leader.  One launch per batch serves
// every linear of the model.
__global__ __launch_bounds__(64 * kPlanWaves) void lora_plan_kernel(const int* __restrict__ adapter, int T, int n,
                                                                    int gtokens, int* __restrict__ head,
                                                                    int* __restrict__ order, int* __restrict__ start,
                                                                    int* __restrict__ gstart,
                                                                    LoraTile* __restrict__ tiles,
                                                                    LoraTile* __restrict__ gtiles) {
  extern __shared__ int s_count[];  // [kPlanWaves][n + 1], then the buckets' totals, first tiles and first gradient tiles
  __shared__ int s_sum[3][64 * kPlanWaves];
  const int nb = n + 1, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, NT = 64 * kPlanWaves;
  int* s_tile = s_count + kPlanWaves * nb;
  int* s_gtile = s_tile + nb + 1;
  int* s_start = s_gtile + nb + 1;
  for (int i = tid; i < kPlanWaves * nb; i += NT) s_count[i] = 0;
  __syncthreads();
  const int bits = 32 - __builtin_clz(n);
  const int per = (T + NT - 1) / NT * 64;  // tokens per wave
  const int t0 = min(wave * per, T), t1 = min(t0 + per, T);
  int* mine = s_count + wave * nb;
  auto key_of = [&](int t) {
    const int a = t < t1 ? adapter[t] : n;
    return unsigned(a) < unsigned(n) ? a : n;
  };
  for (int t = t0; t < t1; t += 64) {
    const bool on = t + lane < t1;
    const int key = key_of(t + lane);
    const uint64_t m = same_key(key, bits, on);
    if (on && (m & ((uint64_t(1) << lane) - 1)) == 0) mine[key] += __popcll(m);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  // Totals of a run of buckets per thread, scanned over the block; a wave's
  // counts become its first position within the bucket.
  const int run = (nb + NT - 1) / NT, b0 = min(tid * run, nb), b1 = min(b0 + run, nb);
  int c = 0, ct = 0, cg = 0;
  for (int b = b0; b < b1; ++b) {
    int tot = 0;
    for (int w = 0; w < kPlanWaves; ++w) {
      const int k = s_count[w * nb + b];
      s_count[w * nb + b] = tot;
      tot += k;
    }
    s_start[b] = c, s_tile[b] = ct, s_gtile[b] = cg;
    c += tot;
    ct += (tot + kLoraTile - 1) / kLoraTile;
    if (b < n) cg += (tot + gtokens - 1) / gtokens;
  }
  s_sum[0][tid] = c, s_sum[1][tid] = ct, s_sum[2][tid] = cg;
  __syncthreads();
  for (int d = 1; d < NT; d <<= 1) {
    int add[3] = {0, 0, 0};
    if (tid >= d)
      for (int q = 0; q < 3; ++q) add[q] = s_sum[q][tid - d];
    __syncthreads();
    for (int q = 0; q < 3; ++q) s_sum[q][tid] += add[q];
    __syncthreads();
  }
  const int e = s_sum[0][tid] - c, et = s_sum[1][tid] - ct, eg = s_sum[2][tid] - cg;
  for (int b = b0; b < b1; ++b) s_start[b] += e, s_tile[b] += et, s_gtile[b] += eg;
  if (tid == NT - 1) {
    s_start[nb] = T;
    s_tile[nb] = s_sum[1][tid];
    s_gtile[nb] = s_sum[2][tid];
    head[0] = kLoraMagic, head[1] = T, head[2] = n, head[3] = s_sum[1][tid], head[4] = s_sum[2][tid];
  }
  __syncthreads();
  for (int b = tid; b <= nb; b += NT) {
    start[b] = s_start[b];
    if (b <= n) gstart[b] = s_gtile[b];
  }
  for (int b = wave; b < nb; b += kPlanWaves) {
    const int p = s_start[b], tot = s_start[b + 1] - p;
    const int nt = s_tile[b + 1] - s_tile[b], ng = s_gtile[b + 1] - s_gtile[b];
    for (int i = lane; i < nt; i += 64)
      tiles[s_tile[b] + i] = {p + i * kLoraTile, min(kLoraTile, tot - i * kLoraTile), b, nt == 1};
    for (int i = lane; i < ng; i += 64)
      gtiles[s_gtile[b] + i] = {p + i * gtokens, min(gtokens, tot - i * gtokens), b, ng == 1};
  }
  for (int t = t0; t < t1; t += 64) {
    const bool on = t + lane < t1;
    const int key = key_of(t + lane);
    const uint64_t m = same_key(key, bits, on);
    const uint64_t before = m & ((uint64_t(1) << lane) - 1);
    const int at = on ? s_start[key] + mine[key] : 0;
    __builtin_amdgcn_wave_barrier();
    if (on) order[at + __popcll(before)] = t + lane;
    if (on && before == 0) mine[key] += __popcll(m);
    __builtin_amdgcn_wave_barrier();
  }
}

// ---------------------------------------------------------------- products with the long axis contracted

struct LoraDown {
  const uint16_t* X;  // rows of the tall matrix
  int64_t ldx;
  const uint16_t* W;  // one adapter's weights: [wrows, K] (A) or [K, wrows] (B, one part)
  int64_t wstride;    // elements from one adapter to the next
  int K, wrows;
  float* part;  // [splits][T][R]
  int R;
  int splits, slice;  // K per split, a multiple of kLoraSlice
  int off[kLoraMaxParts], width[kLoraMaxParts];  // B: the parts' columns
  int chunks;                                    // blocks of 16 RT ranks per part
};

// part[s][p][c] = sum over split s's K range of X[order[p]][k] W[c][k].  A
// block takes a tile of up to 64 tokens; its waves take 128 of every 512 k, so
// that an adapter's fragment is loaded once and used for all four 16-token
// fragments, and add up through LDS.  All fragments of a wave's 128 k are loaded before
// they are used: 16 KiB in flight per wave.  B is contracted over its rows: 128 of them go
// through LDS and come back transposed.
template <int RT, bool BMAJOR, int NSUB>
__device__ __forceinline__ void lora_down_body(const LoraDown& a, const LoraTile& tile, const LoraPlan& plan, int split,
                                               int chunk, int part, float* s_red, u32x4* s_w) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, q = lane >> 4;
  const int r0 = chunk * 16 * RT, nr = min(16 * RT, a.wrows - r0);
  const int col0 = BMAJOR ? a.off[part] : 0, K = BMAJOR ? a.width[part] : a.K;
  const int k0 = split * a.slice, k1 = min(k0 + a.slice, K);
  const uint16_t* xr[NSUB];
#pragma unroll
  for (int s = 0; s < NSUB; ++s)
    xr[s] = a.X + int64_t(plan.order[tile.pos + min(s * 16 + row, tile.count - 1)]) * a.ldx + col0;
  const uint16_t* w = a.W + int64_t(tile.adapter) * a.wstride;
  if (BMAJOR) w += int64_t(col0) * a.wrows;
  f32x4 acc[NSUB][RT];
#pragma unroll
  for (int s = 0; s < NSUB; ++s)
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[s][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int kb = k0; kb < k1; kb += kLoraSlice) {
    const int kw = kb + wave * 128;
    u32x4 x[NSUB][4], wf[RT][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = kw + 32 * j + 8 * q;
      const bool in = k < k1;
#pragma unroll
      for (int s = 0; s < NSUB; ++s) x[s][j] = in ? ld16(xr[s] + k) : zero16();
      if constexpr (!BMAJOR) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
          wf[t][j] = in ? ld16(w + int64_t(r0 + min(t * 16 + row, nr - 1)) * K + k) : zero16();
      }
    }
    if constexpr (BMAJOR) {
      constexpr int CH = 2 * RT;  // 16-byte chunks per row of 16 RT ranks
      u32x4* sw = s_w + wave * 128 * CH;
      u32x4 v[CH * 2];
#pragma unroll
      for (int i = 0; i < CH * 2; ++i) {
        const int e = i * 64 + lane, k = kw + e / CH, c = 8 * (e % CH);
        v[i] = k < k1 && c < nr ? ld16(w + int64_t(k) * a.wrows + r0 + c) : zero16();
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < CH * 2; ++i) sw[i * 64 + lane] = v[i];
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      // the 16-lane group q reads rows 8 q + (row / 4) and + 4 of each 32, columns 4 (row % 4) .. + 3
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const char* b = reinterpret_cast<const char*>(sw) + (32 * j + 8 * q + (row >> 2)) * (CH * 16) + t * 32 + 8 * (row & 3);
          const lora_i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) lora_i16x4*)b);
          const lora_i16x4 hi =
              __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) lora_i16x4*)(b + 4 * CH * 16));
          __builtin_memcpy(&wf[t][j], &lo, 8);
          __builtin_memcpy(reinterpret_cast<char*>(&wf[t][j]) + 8, &hi, 8);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int s = 0; s < NSUB; ++s)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[s][t] = mfma16(x[s][j], wf[t][j], acc[s][t]);
  }
  float* out = a.part + (int64_t(split) * plan.T + tile.pos) * a.R + part * a.wrows + r0;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (t * 16 >= nr) break;  // uniform
    __syncthreads();
#pragma unroll
    for (int s = 0; s < NSUB; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_red[(wave * 64 + s * 16 + 4 * q + i) * 17 + row] = acc[s][t][i];
    __syncthreads();
    for (int e = threadIdx.x; e < NSUB * 256; e += 256) {
      const int tok = e >> 4, c = e & 15;
      const float v = (s_red[tok * 17 + c] + s_red[(64 + tok) * 17 + c]) +
                      (s_red[(128 + tok) * 17 + c] + s_red[(192 + tok) * 17 + c]);
      if (tok < tile.count && t * 16 + c < nr) out[int64_t(tok) * a.R + t * 16 + c] = v;
    }
  }
}

template <int RT, bool BMAJOR>
__global__ __launch_bounds__(256) void lora_down_kernel(LoraDown a, LoraPlan plan) {
  __shared__ float s_red[256 * 17];
  __shared__ u32x4 s_w[BMAJOR ? 4 * 128 * 2 * RT : 1];
  if (!plan.valid()) return;
  const int split = blockIdx.x % a.splits, ti = blockIdx.x / a.splits;
  if (ti >= plan.head[3]) return;
  const LoraTile tile = plan.tiles[ti];
  if (tile.adapter >= plan.n) return;
  const int chunk = blockIdx.y % a.chunks, part = BMAJOR ? blockIdx.y / a.chunks : 0;
  if (tile.count <= 16)
    lora_down_body<RT, BMAJOR, 1>(a, tile, plan, split, chunk, part, s_red, s_w);
  else if (tile.count <= 32)
    lora_down_body<RT, BMAJOR, 2>(a, tile, plan, split, chunk, part, s_red, s_w);
  else
    lora_down_body<RT, BMAJOR, 4>(a, tile, plan, split, chunk, part, s_red, s_w);
}

// Q[p][c] = scale sum_s part[s][p][c]
__global__ __launch_bounds__(256) void lora_sum_kernel(const float* __restrict__ part, int splits, int R,
                                                       const float* __restrict__ scale, LoraPlan plan,
                                                       float* __restrict__ Q) {
  if (!plan.valid()) return;
  const int ti = blockIdx.x;
  if (ti >= plan.head[3]) return;
  const LoraTile tile = plan.tiles[ti];
  if (tile.adapter >= plan.n) return;
  const float c = scale[tile.adapter];
  const int64_t at = int64_t(tile.pos) * R;
  for (int e = 4 * threadIdx.x; e < tile.count * R; e += 1024) {
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(part + int64_t(s) * plan.T * R + at + e);
    *reinterpret_cast<f32x4*>(Q + at + e) = v * c;
  }
}

// ---------------------------------------------------------------- products with the rank contracted

// The first two bf16 terms of eight fp32 values.  An infinity is all in the first.
__device__ __forceinline__ float lora_rest(float x, uint32_t term) {
  const float h = __uint_as_float(term << 16);
  return (term & 0x7f80u) == 0x7f80u ? 0.0f : x - h;
}
__device__ __forceinline__ void lora_terms(const float (&x)[8], u32x4& hi, u32x4& lo) {
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    hi[p] = pack_bf16x2(x[2 * p], x[2 * p + 1]);
    lo[p] = pack_bf16x2(lora_rest(x[2 * p], hi[p] & 0xffffu), lora_rest(x[2 * p + 1], hi[p] >> 16));
  }
}

struct LoraUp {
  const float* low;  // [splits][T][R], rows in the plan's order
  int splits, R;
  const float* scale;  // nullptr: already in `low`
  const uint16_t* W;   // B [d_out, r] or A [R, d_in] of one adapter
  int64_t wstride;
  int r;  // ranks contracted: a part's for B, all for A
  const uint16_t* base;
  int64_t ld_base;
  uint16_t* Y;
  int64_t ldy;
  float* P;  // [T, R] in the tokens' order, or nullptr
  int parts, span;  // columns per block
  int off[kLoraMaxParts], width[kLoraMaxParts], first[kLoraMaxParts + 1];  // first block of each part
};

// A tile's rank terms in LDS: [64 tokens][RT blocks of 16 ranks, 8 spare] bf16, the first terms, then the second.
template <int RT>
constexpr int kUpPitch = 16 * RT + 8;

// Stages ranks [c0, c0 + 16 RT) of rows [t0, t0 + rows) of the tile as bf16
// terms, zeros past the tile's tokens and past `ranks`; with `keep`, the block
// also stores them to P.
template <int RT>
__device__ __forceinline__ void lora_stage(const LoraUp& a, const LoraPlan& plan, const LoraTile& tile, int t0, int rows,
                                           int col0, int c0, int ranks, bool keep, uint16_t* s_hi, uint16_t* s_lo) {
  const float c = a.scale ? a.scale[tile.adapter] : 1.0f;
  for (int e = threadIdx.x; e < rows * 2 * RT; e += 256) {
    const int row = e / (2 * RT), k = 8 * (e % (2 * RT)), tok = t0 + row;
    float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (tok < tile.count && c0 + k < ranks) {
      const float* src = a.low + int64_t(tile.pos + tok) * a.R + col0 + c0 + k;
      for (int s = 0; s < a.splits; ++s) {
        const f32x4 u0 = *reinterpret_cast<const f32x4*>(src + int64_t(s) * plan.T * a.R);
        const f32x4 u1 = *reinterpret_cast<const f32x4*>(src + int64_t(s) * plan.T * a.R + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += u0[i], v[4 + i] += u1[i];
      }
      if (keep) {
        float* p = a.P + int64_t(plan.order[tile.pos + tok]) * a.R + col0 + c0 + k;
        *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= c;
    }
    u32x4 hi, lo;
    lora_terms(v, hi, lo);
    st16(s_hi + row * kUpPitch<RT> + k, hi);
    st16(s_lo + row * kUpPitch<RT> + k, lo);
  }
}

// A tile of tokens without an adapter: columns of base, and zeros in P.
__device__ __forceinline__ void lora_copy(const LoraUp& a, const LoraPlan& plan, const LoraTile& tile, int col0,
                                          int cols, int rank0, int ranks) {
  if (a.base != a.Y) {
    const int cpr = cols / 8;
    for (int e = threadIdx.x; e < tile.count * cpr; e += 256) {
      const int64_t t = plan.order[tile.pos + e / cpr];
      const int c = col0 + 8 * (e % cpr);
      st16(a.Y + t * a.ldy + c, ld16(a.base + t * a.ld_base + c));
    }
  }
  for (int e = threadIdx.x; e < tile.count * ranks; e += 256)
    a.P[int64_t(plan.order[tile.pos + e / ranks]) * a.R + rank0 + e % ranks] = 0.0f;
}

__device__ __forceinline__ u32x4 lora_add8(const u32x4& b, const float (&d)[8]) {
  u32x4 r;
#pragma unroll
  for (int p = 0; p < 4; ++p) r[p] = pack_bf16x2(bf16_lo(b[p]) + d[2 * p], bf16_hi(b[p]) + d[2 * p + 1]);
  return r;
}

// Y = base + c P B^T.  The matrix product's rows are output columns and its
// columns tokens, with B's rows dealt so that two instructions leave eight
// consecutive columns of one token in each lane: base and Y move as 16-byte
// vectors straight between memory and registers, 64 bytes per token.  One
// instruction's 32 k hold the two terms of 16 ranks.
template <int RT, int NSUB>
__device__ __forceinline__ void lora_up_body(const LoraUp& a, const LoraPlan& plan, const LoraTile& tile, int part,
                                             int cb, const uint16_t* s_hi, const uint16_t* s_lo) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, q = lane >> 4;
  const int off = a.off[part], width = a.width[part];
  const uint16_t* w = a.W + int64_t(tile.adapter) * a.wstride + int64_t(off) * a.r + 8 * (q & 1);
  u32x4 pf[NSUB][RT];
  const uint16_t* sp = (q >> 1 ? s_lo : s_hi) + row * kUpPitch<RT> + 8 * (q & 1);
  const uint16_t* br[NSUB];
  uint16_t* yr[NSUB];
#pragma unroll
  for (int s = 0; s < NSUB; ++s) {
#pragma unroll
    for (int t = 0; t < RT; ++t) pf[s][t] = ld16(sp + s * 16 * kUpPitch<RT> + t * 16);
    const int64_t tok = plan.order[tile.pos + min(s * 16 + row, tile.count - 1)];
    yr[s] = a.Y + tok * a.ldy + off + 8 * q;
    br[s] = a.base + tok * a.ld_base + off + 8 * q;
  }
  const int end = min(cb + a.span, width);
  for (int o0 = cb + 32 * wave; o0 < end; o0 += 128) {
    const bool in = o0 + 8 * q < end;
    u32x4 wf[2][RT], b[NSUB];
#pragma unroll
    for (int s = 0; s < NSUB; ++s) b[s] = in ? ld16(br[s] + o0) : zero16();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int o = min(o0 + 8 * (row >> 2) + 4 * j + (row & 3), width - 1);
#pragma unroll
      for (int t = 0; t < RT; ++t)
        wf[j][t] = t * 16 + 8 * (q & 1) < a.r ? ld16(w + int64_t(o) * a.r + t * 16) : zero16();
    }
#pragma unroll
    for (int s = 0; s < NSUB; ++s) {
      f32x4 d[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        d[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < RT; ++t) d[j] = mfma16(wf[j][t], pf[s][t], d[j]);
      }
      const float v[8] = {d[0][0], d[0][1], d[0][2], d[0][3], d[1][0], d[1][1], d[1][2], d[1][3]};
      if (in && s * 16 + row < tile.count) st16(yr[s] + o0, lora_add8(b[s], v));
    }
  }
}

template <int RT>
__global__ __launch_bounds__(256) void lora_up_kernel(LoraUp a, LoraPlan plan) {
  __shared__ __align__(16) uint16_t s_terms[2][64 * kUpPitch<RT>];
  if (!plan.valid()) return;
  const int blocks = a.first[a.parts], ti = blockIdx.x / blocks, cbk = blockIdx.x % blocks;
  if (ti >= plan.head[3]) return;
  const LoraTile tile = plan.tiles[ti];
  int part = 0;
  while (part + 1 < a.parts && cbk >= a.first[part + 1]) ++part;
  const int cb = (cbk - a.first[part]) * a.span;
  const bool keep = a.P != nullptr && cb == 0;
  if (tile.adapter >= plan.n) {
    lora_copy(a, plan, tile, a.off[part] + cb, min(a.span, a.width[part] - cb), part * a.r, keep ? a.r : 0);
    return;
  }
  const int subs = (tile.count + 15) / 16, nsub = subs == 3 ? 4 : subs;
  lora_stage<RT>(a, plan, tile, 0, nsub * 16, part * a.r, 0, a.r, keep, s_terms[0], s_terms[1]);
  __syncthreads();
  if (nsub == 1)
    lora_up_body<RT, 1>(a, plan, tile, part, cb, s_terms[0], s_terms[1]);
  else if (nsub == 2)
    lora_up_body<RT, 2>(a, plan, tile, part, cb, s_terms[0], s_terms[1]);
  else
    lora_up_body<RT, 4>(a, plan, tile, part, cb, s_terms[0], s_terms[1]);
}

// dX = base + Q A.  A's rows are ranks, so a lane loads eight ranks of eight
// columns and transposes them in registers; eight instructions then give a
// lane four runs of eight consecutive columns (32 apart) of one token.
constexpr int kUpTRanks = 64;   // ranks staged at a time
constexpr int kUpTCols = 512;   // columns per block, 128 per wave

__global__ __launch_bounds__(256) void lora_up_t_kernel(LoraUp a, int d_in, LoraPlan plan) {
  constexpr int RT = kUpTRanks / 16, NS = 2;
  __shared__ __align__(16) uint16_t s_terms[2][16 * NS * kUpPitch<RT>];
  if (!plan.valid()) return;
  const int blocks = (d_in + kUpTCols - 1) / kUpTCols, ti = blockIdx.x / blocks, cb = blockIdx.x % blocks * kUpTCols;
  if (ti >= plan.head[3]) return;
  const LoraTile tile = plan.tiles[ti];
  if (tile.adapter >= plan.n) {
    lora_copy(a, plan, tile, cb, min(kUpTCols, d_in - cb), 0, 0);
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, q = lane >> 4;
  const int c0 = cb + 128 * wave;
  const int wc = c0 + 8 * (4 * (row & 3) + (row >> 2));  // row 4 q + i of the products: columns 32 i + 8 q + c
  const uint16_t* w = a.W + int64_t(tile.adapter) * a.wstride + wc;
  for (int t0 = 0; t0 < tile.count; t0 += 16 * NS) {
    uint16_t* yr[NS];
    u32x4 b[NS][4];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int64_t tok = plan.order[tile.pos + min(t0 + s * 16 + row, tile.count - 1)];
      yr[s] = a.Y + tok * a.ldy + c0 + 8 * q;
      const uint16_t* br = a.base + tok * a.ld_base + c0 + 8 * q;
#pragma unroll
      for (int i = 0; i < 4; ++i) b[s][i] = c0 + 32 * i + 8 * q < d_in ? ld16(br + 32 * i) : zero16();
    }
    f32x4 acc[NS][8];
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[s][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int r0 = 0; r0 < a.r; r0 += kUpTRanks) {
      __syncthreads();
      lora_stage<RT>(a, plan, tile, t0, 16 * NS, 0, r0, a.r, false, s_terms[0], s_terms[1]);
      __syncthreads();
      const int nt = (min(a.r - r0, kUpTRanks) + 15) / 16;
      for (int t = 0; t < nt; ++t) {
        const int k = r0 + 16 * t + 8 * (q & 1);
        u32x4 v[8], wf[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = k < a.r && wc < d_in ? ld16(w + int64_t(k + j) * d_in) : zero16();
        transpose8x8_b16(v, wf);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const u32x4 pf = ld16(s_terms[q >> 1] + (s * 16 + row) * kUpPitch<RT> + 16 * t + 8 * (q & 1));
#pragma unroll
          for (int c = 0; c < 8; ++c) acc[s][c] = mfma16(wf[c], pf, acc[s][c]);
        }
      }
    }
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = acc[s][c][i];
        if (c0 + 32 * i + 8 * q < d_in && t0 + s * 16 + row < tile.count) st16(yr[s] + 32 * i, lora_add8(b[s][i], v));
      }
  }
}

// ---------------------------------------------------------------- products with the tokens contracted

struct LoraGrad {
  const uint16_t* X;  // the tall matrix
  int64_t ldx;
  const float* low;  // [T, R]: P in the tokens' order, or Q in the plan's
  int R, r;          // ranks of a part (R for dA)
  const float* scale;
  float* out;     // [n, ranks, cols] (dA) or [n, cols, r] (dB)
  int64_t ostride;  // elements per adapter
  int ocols;        // all columns of the tall matrix
  float* part;    // the same, per gradient tile
  int chunks, parts;
  int off[kLoraMaxParts], width[kLoraMaxParts], first[kLoraMaxParts + 1];
};

// One block sums the products of up to 512 tokens of one adapter for 128
// columns and 16 RT ranks, each wave over 32 of every 128 tokens.  A lane loads eight
// tokens of eight columns and transposes them in registers, so that the tokens become
// the contracted index without a trip through LDS.  An adapter with
// one tile of tokens is done; others leave partial sums.
template <int RT, bool DB>
__global__ __launch_bounds__(256) void lora_grad_kernel(LoraGrad a, LoraPlan plan) {
  __shared__ float s_red[4 * 128 * 17];
  if (!plan.valid()) return;
  const int blocks = a.first[a.parts], gi = blockIdx.x / blocks, cbk = blockIdx.x % blocks;
  if (gi >= plan.head[4]) return;
  const LoraTile tile = plan.gtiles[gi];
  int part = 0;
  while (part + 1 < a.parts && cbk >= a.first[part + 1]) ++part;
  const int cb = (cbk - a.first[part]) * kLoraGradCols, width = a.width[part];
  const int r0 = blockIdx.y * 16 * RT, nr = min(16 * RT, a.r - r0);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, q = lane >> 4;
  const int cols = cb + 8 * row;
  const uint16_t* x = a.X + a.off[part] + cols;
  const float* low = a.low + (DB ? part * a.r : 0) + r0 + row;
  f32x4 acc[8][RT];
#pragma unroll
  for (int c = 0; c < 8; ++c)
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[c][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int tb = 32 * wave; tb < tile.count; tb += 128) {
    u32x4 v[8], xf[8];
    float l[RT][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = tb + 8 * q + j;
      const bool on = t < tile.count;
      const int p = tile.pos + min(t, tile.count - 1);
      const int64_t tok = plan.order[p];
      v[j] = on && cols < width ? ld16(x + tok * a.ldx) : zero16();
      const float* lr = low + (DB ? tok : int64_t(p)) * a.R;
#pragma unroll
      for (int u = 0; u < RT; ++u) l[u][j] = on && 16 * u + row < nr ? lr[16 * u] : 0.0f;
    }
    transpose8x8_b16(v, xf);
#pragma unroll
    for (int u = 0; u < RT; ++u) {
      u32x4 f[3];
      float rest[8];
      lora_terms(l[u], f[0], f[1]);
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        rest[2 * p] = lora_rest(lora_rest(l[u][2 * p], f[0][p] & 0xffffu), f[1][p] & 0xffffu);
        rest[2 * p + 1] = lora_rest(lora_rest(l[u][2 * p + 1], f[0][p] >> 16), f[1][p] >> 16);
        f[2][p] = pack_bf16x2(rest[2 * p], rest[2 * p + 1]);
      }
#pragma unroll
      for (int m = 0; m < 3; ++m)
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[c][u] = mfma16(xf[c], f[m], acc[c][u]);
    }
  }
  float* out = tile.only ? a.out + tile.adapter * a.ostride : a.part + gi * a.ostride;
  const float scale = DB ? a.scale[tile.adapter] : 1.0f;
  for (int u = 0; u < RT; ++u) {
    if (u * 16 >= nr) break;  // uniform
    __syncthreads();
#pragma unroll
    for (int t = 0; t < RT; ++t)
      if (t == u) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) s_red[(wave * 128 + 8 * (4 * q + i) + c) * 17 + row] = acc[c][t][i];
      }
    __syncthreads();
    for (int e = threadIdx.x; e < 128 * 16; e += 256) {
      const int c = DB ? e >> 4 : e & 127, k = DB ? e & 15 : e >> 7;
      const float* p = s_red + c * 17 + k;
      const float g = scale * ((p[0] + p[128 * 17]) + (p[256 * 17] + p[384 * 17]));
      if (cb + c < width && u * 16 + k < nr) {
        const int64_t col = a.off[part] + cb + c, rank = r0 + u * 16 + k;
        out[DB ? col * a.r + rank : rank * a.ocols + col] = g;
      }
    }
  }
}

// The gradients of adapters with several tiles from their partial sums, in the
// tiles' order, and zeros for adapters that no token chose.
__global__ __launch_bounds__(256) void lora_grad_sum_kernel(const float* __restrict__ partA, float* __restrict__ dA,
                                                            int64_t sA, int blocksA, const float* __restrict__ partB,
                                                            float* __restrict__ dB, int64_t sB, LoraPlan plan) {
  if (!plan.valid()) return;
  const int a = blockIdx.y, g0 = plan.gstart[a], g1 = plan.gstart[a + 1];
  if (g1 - g0 == 1) return;
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
  const size_t lds = size_t(kPlanWaves * (n + 1) + 3 * (n + 2)) * sizeof(int);
  hipLaunchKernelGGL(lora_plan_kernel, dim3(1), dim3(64 * kPlanWaves), lds, s, adapter, T, n, lora_grad_tokens(T), w,
                     w + L.order, w + L.start, w + L.gstart, reinterpret_cast<LoraTile*>(w + L.tiles),
                     reinterpret_cast<LoraTile*>(w + L.gtiles));
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

// Blocks of 16, 32 or 64 ranks.
static int rank_tiles(int ranks) { return ranks <= 16 ? 1 : ranks <= 32 ? 2 : 4; }

static int round_slice(int K, int splits) {
  return ((K + splits - 1) / splits + kLoraSlice - 1) / kLoraSlice * kLoraSlice;
}

hipError_t launch_lora_fwd(const uint16_t* X, int64_t ldx, const uint16_t* A, const uint16_t* B, const float* scale,
                           const void* plan, const LoraShape& z, const uint16_t* base, int64_t ld_base, uint16_t* Y,
                           int64_t ldy, float* P, float* part, int splits, hipStream_t s) {
  const LoraPlan pl = lora_plan(plan, z.T, z.n);
  const int R = z.parts * z.r, tiles = lora_max_tiles(z);
  LoraDown d = {};
  d.X = X, d.ldx = ldx, d.W = A, d.wstride = int64_t(R) * z.d_in, d.K = z.d_in, d.wrows = R;
  d.part = part, d.R = R;
  d.slice = round_slice(z.d_in, splits);
  d.splits = splits;
  const int rt = rank_tiles(R);
  d.chunks = (R + 16 * rt - 1) / (16 * rt);
  if (hipError_t e = launch_down<false>(d, pl, tiles, rt, d.chunks, s)) return e;
  LoraUp u = {};
  u.low = part, u.splits = splits, u.R = R, u.scale = scale;
  u.W = B, u.wstride = int64_t(z.d_out) * z.r, u.r = z.r;
  u.base = base, u.ld_base = ld_base, u.Y = Y, u.ldy = ldy, u.P = P, u.parts = z.parts;
  // Blocks of 512 columns where that gives every CU a few; narrower ones below.
  u.span = 512;
  while (u.span > 128 && int64_t(tiles) * (z.d_out / u.span) < 1024) u.span /= 2;
  for (int p = 0, off = 0; p < z.parts; ++p) {
    u.off[p] = off, u.width[p] = z.widths[p];
    off += z.widths[p];
    u.first[p + 1] = u.first[p] + (z.widths[p] + u.span - 1) / u.span;
  }
  const dim3 grid(unsigned(tiles) * unsigned(u.first[z.parts])), block(256);
  if (z.r <= 16) hipLaunchKernelGGL(lora_up_kernel<1>, grid, block, 0, s, u, pl);
  else if (z.r <= 32) hipLaunchKernelGGL(lora_up_kernel<2>, grid, block, 0, s, u, pl);
  else if (z.r <= 64) hipLaunchKernelGGL(lora_up_kernel<4>, grid, block, 0, s, u, pl);
  else hipLaunchKernelGGL(lora_up_kernel<8>, grid, block, 0, s, u, pl);
  return hipGetLastError();
}

template <bool DB>
static hipError_t launch_grad(const LoraGrad& a, const LoraPlan& plan, int gtiles, int rt, hipStream_t s) {
  const dim3 grid(unsigned(gtiles) * unsigned(a.first[a.parts]), unsigned(a.chunks)), block(256);
  switch (rt) {
    case 1: hipLaunchKernelGGL((lora_grad_kernel<1, DB>), grid, block, 0, s, a, plan); break;
    case 2: hipLaunchKernelGGL((lora_grad_kernel<2, DB>), grid, block, 0, s, a, plan); break;
    default: hipLaunchKernelGGL((lora_grad_kernel<4, DB>), grid, block, 0, s, a, plan); break;
  }
  return hipGetLastError();
}

hipError_t launch_lora_bwd(const uint16_t* dY, int64_t lddy, const uint16_t* X, int64_t ldx, const uint16_t* A,
                           const uint16_t* B, const float* scale, const void* plan, const float* P,
                           const LoraShape& z, const uint16_t* base, int64_t ld_base, uint16_t* dX, int64_t lddx,
                           float* dA, float* dB, const LoraBwdWs& w, int splits, hipStream_t s) {
  const LoraPlan pl = lora_plan(plan, z.T, z.n);
  const LoraPlanLayout L = lora_plan_layout(z.T, z.n);
  const int R = z.parts * z.r, tiles = int(L.max_tiles), gtiles = int(L.max_gtiles);
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
    d.part = w.part, d.R = R, d.splits = splits, d.slice = round_slice(widest, splits);
    for (int p = 0; p < z.parts; ++p) d.off[p] = off[p], d.width[p] = z.widths[p];
    const int rt = rank_tiles(z.r);
    d.chunks = (z.r + 16 * rt - 1) / (16 * rt);
    if ((e = launch_down<true>(d, pl, tiles, rt, d.chunks * z.parts, s))) return e;
    hipLaunchKernelGGL(lora_sum_kernel, dim3(tiles), dim3(256), 0, s, w.part, splits, R, scale, pl, w.Q);
    if ((e = hipGetLastError())) return e;
  }
  if (dX) {
    LoraUp u = {};
    u.low = w.Q, u.splits = 1, u.R = R, u.W = A, u.wstride = int64_t(R) * z.d_in, u.r = R;
    u.base = base, u.ld_base = ld_base, u.Y = dX, u.ldy = lddx, u.parts = 1;
    const int blocks = (z.d_in + kUpTCols - 1) / kUpTCols;
    hipLaunchKernelGGL(lora_up_t_kernel, dim3(unsigned(tiles) * unsigned(blocks)), dim3(256), 0, s, u, z.d_in, pl);
    if ((e = hipGetLastError())) return e;
  }
  LoraGrad g = {};
  if (dA) {
    g.X = X, g.ldx = ldx, g.low = w.Q, g.R = R, g.r = R, g.out = dA, g.ostride = int64_t(R) * z.d_in, g.ocols = z.d_in;
    g.part = w.partA, g.parts = 1, g.width[0] = z.d_in;
    g.first[1] = (z.d_in + kLoraGradCols - 1) / kLoraGradCols;
    const int rt = rank_tiles(R);
    g.chunks = (R + 16 * rt - 1) / (16 * rt);
    if ((e = launch_grad<false>(g, pl, gtiles, rt, s))) return e;
  }
  if (dB) {
    g.X = dY, g.ldx = lddy, g.low = P, g.R = R, g.r = z.r, g.scale = scale, g.out = dB;
    g.ostride = int64_t(z.d_out) * z.r, g.ocols = z.d_out, g.part = w.partB, g.parts = z.parts;
    for (int p = 0; p < z.parts; ++p) {
      g.off[p] = off[p], g.width[p] = z.widths[p];
      g.first[p + 1] = g.first[p] + (z.widths[p] + kLoraGradCols - 1) / kLoraGradCols;
    }
    const int rt = rank_tiles(z.r);
    g.chunks = (z.r + 16 * rt - 1) / (16 * rt);
    if ((e = launch_grad<true>(g, pl, gtiles, rt, s))) return e;
  }
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
