// New tokens over a key / value cache: rotary positions with the rows appended, attention of the new rows over a shared prefix
// and their own rows, accumulated attention weights, and eviction by those weights.
//
//   rope_kernel           (a, b) -> m (a cos f - b sin f, b cos f + a sin f) for up to four tensors of the same rows
//   ca_stream_kernel      partial softmax sums of up to 16 stacked query rows over a range of keys, keys and values streamed once
//   ca_tile_kernel        the same for more rows, 256 at a time on the tensor cores
//   ca_join_kernel        partial sums of a row -> output and ln of the sum
//   ca_weight_kernel      probabilities summed over query rows and heads, per key
//   ca_weight_few_kernel  the same for few rows, from the partial sums, without waiting for the join
//   evict_select_kernel   rows kept by rank
//   evict_move_kernel     kept rows of the cache tensors, their weights and positions
//   evict_in_place_kernel the same within the same tensors
//   slot_kernel           the row of every sequence's next token
#pragma once

#include <cuda_fp16.h>
#include <limits.h>

#include <type_traits>

#include "common.cuh"

namespace asap {

enum : uint32_t { STATUS_CACHE_TIMEOUT = 64u };   // a bounded wait ran out in a cache attention kernel

__device__ __forceinline__ void ld_prev8(const void *p, uint4 &v) {
  asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
}
// In place of pdl_enter in a kernel whose predecessor has waited for all that this one reads, before it let this one start.  That lies in L2 by now.
// A processor's L1 may hold older copies, which the wait would have dropped: the fence does (what this thread loads from here on is no older).
__device__ __forceinline__ void pdl_after() {
  pdl_trigger();
  __threadfence();
}
template <bool F16>
__device__ __forceinline__ uint32_t pack2_t(float a, float b) {
  if constexpr (F16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
  } else {
    return pack2_rn(a, b);
  }
}
// ... rounded towards zero
template <bool F16>
__device__ __forceinline__ uint32_t pack2_rz(float a, float b) {
  uint32_t d;
  if constexpr (F16) asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
  else asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
  return d;
}
template <bool F16>
__device__ __forceinline__ float2 unpack2_t(uint32_t w) {
  if constexpr (F16) return __half22float2(*reinterpret_cast<const __half2 *>(&w));
  else return make_float2(bf16_lo(w), bf16_hi(w));
}

// =======================================================================================
// Rotary positions
// =======================================================================================
constexpr int ROPE_THREADS = 256;
constexpr int ROPE_MAX_PAIRS = 128;
constexpr int ROPE_MAX_ROWS = 16;      // rows of a block

struct RopeTensor {
  const uint16_t *src;
  uint16_t *dst;
  int heads, rotate, mapped;
  int rows, first_block;               // rows of a block, and the tensor's first block
  long long src_row, src_head, dst_row, dst_head;
};
struct RopeArgs {
  RopeTensor t[4];
  int n_tensors, n_rows, head_dim, n_pairs, interleaved, dst_rows;
  float magnitude, sign;
  const int *pos, *map;
  unsigned long long turns[ROPE_MAX_PAIRS];
};

// One element pair, or eight elements at a time (VEC) where the pairs allow it: half layout n_pairs % 8 == 0, interleaved
// n_pairs % 4 == 0.  The angles of a row are taken once for all its heads: pos * turns modulo 2^64 is the fraction of a turn, whose
// upper 32 bits, as a signed number, are the angle in [-1/2, 1/2) turns (2^-32 turns off at most); sincospi takes it in fp32.
// What bounds it on prompts is the memory, kept busy by many warps with little in hand: 24531 rows of 32 + 2 x 32 heads 214 us, 87 % of a
// copy's rate.  (Four rows of a piece under way together per thread, 74 registers, 237 us; warps with angles of their own, 94 registers, 315.)
// A block takes about 128 heads of one tensor: four rows of 32 heads, sixteen of 8 or fewer.
template <bool F16, bool VEC>
__global__ void __launch_bounds__(ROPE_THREADS)
rope_kernel(const __grid_constant__ RopeArgs a) {
  __shared__ __align__(16) float cs[ROPE_MAX_ROWS][2][ROPE_MAX_PAIRS];
  __shared__ int dst_of[ROPE_MAX_ROWS];
  pdl_enter();
  int ti = 0;
  while (ti + 1 < a.n_tensors && (int)blockIdx.x >= a.t[ti + 1].first_block) ++ti;
  const RopeTensor &t = a.t[ti];
  const int row0 = (blockIdx.x - t.first_block) * t.rows;
  const int rows = min(t.rows, a.n_rows - row0);
  for (int i = threadIdx.x; t.rotate && i < rows * a.n_pairs; i += ROPE_THREADS) {
    const int r = i / a.n_pairs, p = i - r * a.n_pairs;
    const long long pos = ld_prev(a.pos + row0 + r);
    const unsigned long long turn = (unsigned long long)pos * a.turns[p];
    const float half_turns = (float)(int)(turn >> 32) * 0x1p-31f;      // in units of pi
    float s, c;
    sincospif(half_turns, &s, &c);
    cs[r][0][p] = c * a.magnitude;
    cs[r][1][p] = s * a.magnitude * a.sign;
  }
  if (threadIdx.x < rows) {
    int d = row0 + threadIdx.x;
    if (a.map) {
      d = ld_prev(a.map + d);
      if (d >= a.dst_rows) d = -1;
    }
    dst_of[threadIdx.x] = d;
  }
  __syncthreads();
  const int P = a.n_pairs, rot = 2 * P;
  // tasks of a head: rotated pieces first, then pieces that pass through
  const int n_rot = t.rotate ? (VEC ? (a.interleaved ? P / 4 : P / 8) : P) : 0;
  const int n_pass = VEC ? (a.head_dim - (t.rotate ? rot : 0)) / 8 : a.head_dim - (t.rotate ? rot : 0);
  const int per_head = n_rot + n_pass;
  const int lanes = ROPE_THREADS / per_head * per_head;      // threads at work: whole heads
  const int v = threadIdx.x % per_head;
  if (threadIdx.x >= lanes) return;
  for (int j = threadIdx.x / per_head; j < rows * t.heads; j += ROPE_THREADS / per_head) {
    const int r = j / t.heads, h = j - r * t.heads;
    const int d = t.mapped ? dst_of[r] : row0 + r;
    if (d < 0) continue;
    const uint16_t *src = t.src + (long long)(row0 + r) * t.src_row + (long long)h * t.src_head;
    uint16_t *dst = t.dst + (long long)d * t.dst_row + (long long)h * t.dst_head;
    // (pieces that pass through and rotated ones lie in the same warp: their loads are one instruction)
    const bool turned = v < n_rot;
    const int e0 = turned ? v * 8 : (t.rotate ? rot : 0) + (v - n_rot) * (VEC ? 8 : 1);
    uint4 x, y;
    if constexpr (VEC) {
      ld_prev8(src + e0, x);
      if (turned && !a.interleaved) ld_prev8(src + P + e0, y);
    }
    if (!turned) {
      if constexpr (VEC) *reinterpret_cast<uint4 *>(dst + e0) = x;
      else dst[e0] = *reinterpret_cast<const volatile uint16_t *>(src + e0);
      continue;
    }
    if constexpr (VEC) {
      if (a.interleaved) {
        uint32_t w[4] = {x.x, x.y, x.z, x.w};
        const float4 c = *reinterpret_cast<const float4 *>(&cs[r][0][v * 4]), s = *reinterpret_cast<const float4 *>(&cs[r][1][v * 4]);
        const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 p = unpack2_t<F16>(w[e]);
          w[e] = pack2_t<F16>(p.x * cc[e] - p.y * ss[e], p.y * cc[e] + p.x * ss[e]);
        }
        *reinterpret_cast<uint4 *>(dst + v * 8) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        uint32_t wx[4] = {x.x, x.y, x.z, x.w}, wy[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 p = unpack2_t<F16>(wx[e]), q = unpack2_t<F16>(wy[e]);
          const float2 c = *reinterpret_cast<const float2 *>(&cs[r][0][v * 8 + 2 * e]), s = *reinterpret_cast<const float2 *>(&cs[r][1][v * 8 + 2 * e]);
          wx[e] = pack2_t<F16>(p.x * c.x - q.x * s.x, p.y * c.y - q.y * s.y);
          wy[e] = pack2_t<F16>(q.x * c.x + p.x * s.x, q.y * c.y + p.y * s.y);
        }
        *reinterpret_cast<uint4 *>(dst + v * 8) = make_uint4(wx[0], wx[1], wx[2], wx[3]);
        *reinterpret_cast<uint4 *>(dst + P + v * 8) = make_uint4(wy[0], wy[1], wy[2], wy[3]);
      }
    } else {
      const int ea = a.interleaved ? 2 * v : v, eb = a.interleaved ? 2 * v + 1 : v + P;
      const uint32_t w = *reinterpret_cast<const volatile uint16_t *>(src + ea) | (uint32_t)*reinterpret_cast<const volatile uint16_t *>(src + eb) << 16;
      const float2 p = unpack2_t<F16>(w);
      const float c = cs[r][0][v], s = cs[r][1][v];
      const uint32_t o = pack2_t<F16>(p.x * c - p.y * s, p.y * c + p.x * s);
      dst[ea] = (uint16_t)o;
      dst[eb] = (uint16_t)(o >> 16);
    }
  }
}

// =======================================================================================
// Attention over the cache
// =======================================================================================
// A segment is a run of cache rows with the query rows that look at it: segment g < G is the prefix of group g with all query
// rows of its sequences, segment G + b the own rows of sequence b.  Per key / value head the R = (query rows) * (H / kv_heads)
// stacked rows of a segment are cut into row tiles, the keys that a row tile admits into key tiles.  Segments of up to 16 stacked rows
// are streamed (ca_stream_kernel), the others go to the tensor cores as tiles of 128 rows, two side by side (ca_tile_kernel).  Each of
// the two kernels numbers its key tiles through (all row tiles, heads and segments) and cuts the numbers into equal pieces: lengths may be
// as ragged as they like, and the host needs to know none of them.  A row tile whose key tiles lie in one piece is complete
// there; otherwise each piece leaves a partial result (maximum, sum, weighted values) and the join adds them up in order.
// The streaming kernel takes four or two heads side by side where their rows are few: a tile is then 16 or 32 keys of each, so that short
// segments waste little of their last tile, and fewer warps (or none) have to add up their sums.
// Every row tile counts EXTRA numbers more than it has key tiles, for its queries and its result: pieces of many short row tiles
// and pieces of few long ones then take the same time.  A block's first piece is its own number, further ones are drawn.
struct StreamWork {
  static constexpr int ROWS = 16, KEYS = 64, EXTRA = 2, INDEX = 0;
};
struct TileWork {
  static constexpr int ROWS = 256, KEYS = 128, EXTRA = 4, INDEX = 1;
};
constexpr int CA_CONSUMERS = 4;                           // warps; each takes 16 keys of a tile
constexpr int CA_THREADS = 32 * (CA_CONSUMERS + 1);       // and the copying warp
constexpr int CA_STAGES = 3;
constexpr int CA_BLOCK_BYTES = StreamWork::KEYS * 128;    // 64 keys x 64 columns
constexpr int CA_STAGE_BYTES = 4 * CA_BLOCK_BYTES;        // K and V
constexpr int CA_JOIN_BYTES = 4096;                       // the warps' sums of an item, a piece at a time
constexpr int CA_JOBS = 2;                                // items announced ahead
constexpr int CA_Q_PITCH = 272;                           // a query row of 256 bytes; eight rows side by side meet all banks
constexpr int CA_Q_BYTES = StreamWork::ROWS * CA_Q_PITCH;
constexpr int CA_MAX_SEGMENTS = 1024;
constexpr long long CA_WAIT_LIMIT = 2000000000LL;

// Key / value heads that the streaming kernel takes together for segments of R stacked rows: at most 16 rows in all.  Long segments are taken
// head by head: there is nothing to gain, and the heads of a piece would be spread over as many times more pieces for the join to add
// up (5 sequences of 2000 to 60000 rows, four heads together 109 us, one 104).
constexpr int CA_TOGETHER_KEYS = 4096;
__device__ __forceinline__ int ca_heads(int R, int kv, int keys) {
  return keys > CA_TOGETHER_KEYS ? 1 : R <= 4 && kv % 4 == 0 ? 4 : R <= 8 && kv % 2 == 0 ? 2 : 1;
}

// What the join has to know of a query row: its place in the prefix's and in its own segment.
struct CaRowPart {
  int i0, R;               // stacked row of its first head, stacked rows of the segment (0: no keys there)
  int adm0, causal, keys;
  int off, per_head;       // numbers of the segment and of one of its heads (or of the heads that go together)
};
struct CaRow {
  CaRowPart part[2];
  int valid, pad;
};
static_assert(sizeof(CaRow) == 64, "a row's entry is four 16-byte loads");

struct CacheArgs {
  int B, G, H, kv, rep;                    // rep = H / kv
  int n_q, max_q, max_len, max_prefix, cache_rows;
  long long q_row, q_head, out_row, out_head;
  const int *q_cu, *start, *len, *group_cu, *prefix_start, *prefix_len;
  const uint16_t *q, *v;
  long long kv_row, kv_head;
  uint16_t *out;
  float *lse, *weights;
  float scale_log2;                        // scale * log2(e)
  // scratch
  int *plan;                               // [2][n_seg + 1] first number of every segment, streamed and tiled; the last entry: all of them.  Behind
                                           // them 0 if the call is skipped
  int pieces[2];                           // pieces of the two kernels' work; 0: the kernel is not launched
  unsigned int *work;                      // [2] pieces drawn / blocks done; both zero between launches
  int join_behind;                         // the join runs behind ca_weight_few_kernel, which does not need it
  int q_tiled;                             // rep divides 128: a row tile of query rows is one tiled copy
  int rec_rows;                            // rows of a streamed piece's partial result, those of all heads that go together
  CaRow *rows;                             // [n_q]
  float2 *rec_ml[2], *full_ml;             // partial results: two per piece and row of a row tile; [2][n_q * H] (prefix, own) complete ones
  float *rec_o[2], *full_o;                // 128 values each
  float *lse2;                             // [n_q * H] log2 of a row's sum of 2^x; +inf: the row adds no weight
  float *logits;                           // [n_q * H, pitch] x = scale * log2(e) * q.k; prefix keys first, own keys from own_off on
  long long pitch;
  int own_off;
  uint32_t *status;
  long long wait_limit;
};

struct __align__(16) CaSeg {
  int q0, nq;          // query rows
  int row0, keys;      // cache rows; keys < 0: the segment failed validation
};
__device__ __forceinline__ int ca_qcu(const CacheArgs &a, int b) { return a.q_cu ? ld_prev(a.q_cu + b) : b; }

// Segment s as the caller's arrays have it.  `broken`: the offsets of its query rows, or of a group's sequences, do not ascend within
// their bounds; segments of other sequences may then overlap this one's, and the whole call is skipped.
__device__ __forceinline__ CaSeg ca_segment(const CacheArgs &a, int s, bool &broken) {
  CaSeg g;
  bool valid;
  if (s < a.G) {
    const int b0 = ld_prev(a.group_cu + s), b1 = ld_prev(a.group_cu + s + 1);
    g.row0 = ld_prev(a.prefix_start + s); g.keys = ld_prev(a.prefix_len + s);
    broken = b0 < 0 || b0 > b1 || b1 > a.B;
    valid = !broken && g.keys <= a.max_prefix;
    g.q0 = broken ? 0 : ca_qcu(a, b0);
    g.nq = broken ? 0 : ca_qcu(a, b1) - g.q0;
    valid = valid && (long long)g.nq <= (long long)(b1 - b0) * a.max_q;
  } else {
    const int b = s - a.G;
    g.row0 = ld_prev(a.start + b); g.keys = ld_prev(a.len + b);
    const int q0 = ca_qcu(a, b), q1 = ca_qcu(a, b + 1);
    broken = q0 < 0 || q0 > q1 || q1 > a.n_q;
    g.q0 = q0; g.nq = broken ? 0 : q1 - q0;
    valid = g.keys <= a.max_len && g.nq <= a.max_q;
  }
  valid = valid && !broken && g.keys >= 0 && g.row0 >= 0 && (long long)g.row0 + g.keys <= a.cache_rows && g.q0 >= 0 && g.nq >= 0 &&
          g.q0 <= a.n_q && (long long)g.q0 + g.nq <= a.n_q;
  if (!valid) g.keys = -1;
  return g;
}
// group of a sequence: -1 none
__device__ __forceinline__ int ca_group(const CacheArgs &a, int b) {
  int lo = 0, hi = a.G;                    // the last g with group_cu[g] <= b
  if (a.G == 0 || ld_prev(a.group_cu) > b) return -1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (ld_prev(a.group_cu + mid) <= b) lo = mid;
    else hi = mid;
  }
  return b < ld_prev(a.group_cu + lo + 1) ? lo : -1;
}
// Stacked row i admits the first adm0 + i / rep own keys (causal), or all of them.
__device__ __forceinline__ int ca_admitted(int keys, int adm0, int causal, int t) { return causal ? max(0, min(keys, adm0 + t)) : keys; }
__device__ __forceinline__ bool ca_streamed(int R) { return R <= StreamWork::ROWS; }
template <typename WORK>
__device__ __forceinline__ int ca_together(int R, int kv, int keys) { return WORK::INDEX == 0 ? ca_heads(R, kv, keys) : 1; }
// key tiles of row tile rt; `hg` heads go together.  (A streamed segment has one row tile, whose last row admits every key.)
template <typename WORK>
__device__ __forceinline__ int ca_key_tiles(int R, int keys, int adm0, int causal, int rep, int hg, int rt) {
  if constexpr (WORK::INDEX == 0) return (keys * hg + WORK::KEYS - hg) / WORK::KEYS;
  const int last = min((rt + 1) * WORK::ROWS, R) - 1;
  return (ca_admitted(keys, adm0, causal, causal ? last / rep : 0) + WORK::KEYS - 1) / WORK::KEYS;
}
// numbers of the first `n` row tiles of a head
template <typename WORK>
__device__ __forceinline__ int ca_numbers(int R, int keys, int adm0, int causal, int rep, int hg, int n) {
  if (!causal || WORK::INDEX == 0) return keys > 0 && n > 0 ? n * (ca_key_tiles<WORK>(R, keys, adm0, 0, rep, hg, 0) + WORK::EXTRA) : 0;
  int t = 0;
  for (int rt = 0; rt < n; ++rt) {
    const int kt = ca_key_tiles<WORK>(R, keys, adm0, causal, rep, hg, rt);
    t += kt > 0 ? kt + WORK::EXTRA : 0;
  }
  return t;
}
template <typename WORK>
__device__ __forceinline__ int ca_row_tiles(const CaSeg &g, int rep) {
  const int R = g.nq * rep;
  return g.keys > 0 && ca_streamed(R) == (WORK::INDEX == 0) ? (R + WORK::ROWS - 1) / WORK::ROWS : 0;
}

// An item of a block's work: a range of key tiles of one row tile.
struct __align__(16) CaJob {
  int q0, R, row0, keys;
  int adm0, causal, head, rt;   // head: the first of `together`
  int kt0, n;              // key tiles; n < 0: the block's work is done
  int complete, record;    // the row tile has no other items; where the result goes otherwise
  int n_act[2];            // (tile kernel) key tiles that the two row tiles of the pair look at
  int together, pad;
};
__device__ __forceinline__ int ca_admitted(const CaJob &j, int t) { return ca_admitted(j.keys, j.adm0, j.causal, t); }

// Walks the numbers [t, end) of a piece.
template <typename WORK>
struct CaWalk {
  int t, end, begin_t, piece;
  int seg, head, rt, pos;  // pos: numbers of the row tile that lie before t
  int R, causal, hg;
  CaSeg g;
  __device__ __forceinline__ int key_tiles(const CacheArgs &a) const { return ca_key_tiles<WORK>(R, g.keys, g.keys - g.nq + 1, causal, a.rep, hg, rt); }
  __device__ __forceinline__ void enter(const CacheArgs &a, const CaSeg *segs) {
    g = segs[seg];
    R = g.nq * a.rep;
    causal = seg >= a.G;
    hg = ca_together<WORK>(R, a.kv, g.keys);
  }
  __device__ __forceinline__ void begin(const CacheArgs &a, const int *off, const CaSeg *segs, int n_seg, int number, int t0, int t1) {
    t = begin_t = t0; end = t1; piece = number;
    if (t >= end) return;
    int lo = 0, hi = n_seg;                // off[lo] <= t < off[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (off[mid] <= t) lo = mid;
      else hi = mid;
    }
    seg = lo;
    enter(a, segs);
    int u = t - off[seg];
    if constexpr (WORK::INDEX == 0) {
      const int per_head = key_tiles(a) + WORK::EXTRA, group = u / per_head;
      pos = u - group * per_head;
      head = group * hg;
      rt = 0;
      return;
    }
    const int per_head = (off[seg + 1] - off[seg]) / a.kv;
    head = u / per_head;
    u -= head * per_head;
    for (rt = 0;; ++rt) {
      const int kt = key_tiles(a), n = kt > 0 ? kt + WORK::EXTRA : 0;
      if (u < n) break;
      u -= n;
    }
    pos = u;
  }
  // the next item that has key tiles; false: none is left
  __device__ __forceinline__ bool next(const CacheArgs &a, const int *off, const CaSeg *segs, CaJob &j) {
    while (t < end) {
      if (pos < 0) {                       // the row tile is done: the next one that has keys
        pos = 0;
        do {
          if (++rt >= ca_row_tiles<WORK>(g, a.rep)) {
            rt = 0;
            if ((head += hg) >= a.kv) {
              head = 0;
              do ++seg; while (off[seg + 1] <= t);
              enter(a, segs);
            }
          }
        } while (key_tiles(a) == 0);
      }
      const int kt = key_tiles(a), p1 = min(kt + WORK::EXTRA, pos + (end - t));
      const int k0 = max(0, pos - WORK::EXTRA), k1 = p1 - WORK::EXTRA, first = t - pos + WORK::EXTRA;
      t += p1 - pos;
      pos = -1;
      if (k1 <= k0) continue;
      j.q0 = g.q0; j.R = R; j.row0 = g.row0; j.keys = g.keys; j.adm0 = g.keys - g.nq + 1; j.causal = causal; j.head = head; j.rt = rt; j.together = hg;
      j.kt0 = k0; j.n = k1 - k0; j.complete = k0 == 0 && k1 == kt; j.record = 2 * piece + (first <= begin_t ? 0 : 1);
      return true;
    }
    return false;
  }
};

// Segments into segs[0 .. n_seg) and the first number of each into off[0 .. n_seg] (shared memory); all threads of the block.  True if the
// call is to be skipped.
template <typename WORK, int THREADS>
__device__ __forceinline__ bool ca_plan(const CacheArgs &a, int *off, CaSeg *segs, int n_seg, int *warp_part) {
  const int per = (n_seg + THREADS - 1) / THREADS, s0 = min(n_seg, (int)threadIdx.x * per), s1 = min(n_seg, s0 + per);
  int mine = 0;
  bool broken = (*reinterpret_cast<volatile uint32_t *>(a.status) & STATUS_CACHE_TIMEOUT) != 0, bad = false;
  for (int s = s0; s < s1; ++s) {
    bool b;
    const CaSeg g = ca_segment(a, s, b);
    broken |= b;
    bad |= g.keys < 0;
    const int R = g.nq * a.rep, hg = ca_together<WORK>(R, a.kv, g.keys);
    const int n = a.kv / hg * ca_numbers<WORK>(R, g.keys, g.keys - g.nq + 1, s >= a.G, a.rep, hg, ca_row_tiles<WORK>(g, a.rep));
    segs[s] = g;
    off[s + 1] = n;
    mine += n;
  }
  if (WORK::INDEX == 0 && bad && blockIdx.x == 0) atomicOr(a.status, (uint32_t)STATUS_BAD_SAMPLE);
  int scan = mine;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, scan, o);
    if (lane >= o) scan += v;
  }
  if (lane == 31) warp_part[warp] = scan;
  broken = __syncthreads_or(broken);
  int base = scan - mine;
  for (int w = 0; w < warp; ++w) base += warp_part[w];
  for (int s = s0; s < s1; ++s) {
    base += off[s + 1];
    off[s + 1] = base;                     // (its own entries only)
  }
  if (threadIdx.x == 0) off[0] = 0;
  __syncthreads();
  if (blockIdx.x == 0) {
    for (int s = threadIdx.x; s <= n_seg; s += THREADS) a.plan[WORK::INDEX * (n_seg + 1) + s] = off[s];
    if (WORK::INDEX == 0 && threadIdx.x == 0) a.plan[2 * (n_seg + 1)] = broken ? 0 : 1;
  }
  return broken;
}
__device__ __forceinline__ int ca_chunk(int all, int pieces) { return max(1, (all + pieces - 1) / pieces); }

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// The 8 x 8 matrix of 16-bit values whose row `lane / 4` holds this register's two in columns 2 (lane % 4) and the next, transposed.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <bool F16>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Keys or values as [head][column half][row][64 columns], see make_cache_map: one copy brings the tile of all heads and both halves.
__device__ __forceinline__ void tma_load_cache_w(uint32_t smem_dst, const void *tmap, uint32_t bar, int32_t row, int32_t head, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "@q cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %4, %3, %5}], [%2];\n\t}"
      ::"r"(smem_dst), "l"(tmap), "r"(bar), "r"(0), "r"(row), "r"(head), "r"(leader)
      : "memory");
}
// A row tile of stacked query rows as [column half][query row][head of the key / value head][64 columns].
__device__ __forceinline__ void tma_load_query_w(uint32_t smem_dst, const void *tmap, uint32_t bar, int32_t row, int32_t head, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "@q cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %3, %4, %3, %5}], [%2];\n\t}"
      ::"r"(smem_dst), "l"(tmap), "r"(bar), "r"(0), "r"(row), "r"(head), "r"(leader)
      : "memory");
}

// Non-zero if either half is an infinity or NaN: an exponent of all ones, plus one, carries into the sign's place.
template <bool F16>
__device__ __forceinline__ uint32_t not_finite_bits(uint32_t w) {
  constexpr uint32_t exponent = F16 ? 0x7c007c00u : 0x7f807f80u, one = F16 ? 0x04000400u : 0x00800080u;
  return ((w & exponent) + one) & 0x80008000u;
}

// One arrival for the (converged) warp, which is converged afterwards too: lanes that went on to spin on another barrier while lane 0
// had still to arrive here kept it from ever doing so.
__device__ __forceinline__ void mbar_arrive_lane0(uint32_t bar, int lane) {
  if (lane == 0) mbar_arrive(bar);
  __syncwarp();
}

// The whole (converged) warp waits and knows whether all its lanes saw the phase complete: it goes on as one, or gives up as one.
__device__ __forceinline__ bool mbar_wait_all(uint32_t bar, uint32_t parity, const WaitCtx &w) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, w));
}
// A block's last wait for copies that it issued itself (the abort flag does not end it); giving up is recorded.
__device__ __forceinline__ void mbar_settle(uint32_t bar, uint32_t parity, const WaitCtx &w) {
  if (!mbar_wait_drain(bar, parity, CA_WAIT_LIMIT)) atomicOr(w.status, w.status_bit);
}

// The waits in the streaming kernel's queue of items, by a whole (converged) warp.  The consumers meet in barriers without a limit at every item's
// end, so all of them have to see the same items, after an abort too.  A wait past the limit raises the abort flag, which ends every wait but those
// in the queue, so whoever has to be waited for comes then.  Only should that not happen either, for a second and more of looking, is the wait lost: 0.
// 1: in time.  2: late.  (Bounded mbarriers in place of the barriers at an item's end: 61 sequences under 6 prefixes 90.0 us for 87.9.)
constexpr int CA_QUEUE_LOOKS = 1 << 20;                   // of a microsecond at least
__device__ __forceinline__ int ca_wait_on(uint32_t bar, uint32_t parity, volatile int *abort_flag, uint32_t *status, long long limit) {
  const long long t0 = clock64();
  bool ok;
  while (!(ok = mbar_try_wait(bar, parity)) && clock64() - t0 <= limit) {}
  if (__all_sync(0xffffffffu, ok)) return 1;
  *abort_flag = 1;
  atomicOr(status, (uint32_t)STATUS_CACHE_TIMEOUT);
  for (int i = 0; !(ok = mbar_test_wait(bar, parity)) && i < CA_QUEUE_LOOKS; ++i) __nanosleep(1000);
  return __all_sync(0xffffffffu, ok) ? 2 : 0;
}
// A consumer warp: whether it takes item n.  The first late warp decides for all of them (`decision`: 2 n + 2 none takes it, 2 n + 3 all do), and a
// warp that is in time has seen an item that no other one has given up yet.
__device__ __forceinline__ bool ca_wait_on_item(unsigned int *decision, int n, uint32_t bar, uint32_t parity, volatile int *abort_flag, uint32_t *status,
                                             long long limit) {
  const int how = ca_wait_on(bar, parity, abort_flag, status, limit);
  if (how == 1) return true;
  const unsigned int mine = 2u * n + 2u + (how == 2 ? 1u : 0u);
  unsigned int said = 0u;
  if ((threadIdx.x & 31) == 0) {
    said = *reinterpret_cast<volatile unsigned int *>(decision);
    while (said >> 1 != mine >> 1) {
      const unsigned int before = atomicCAS(decision, said, mine);
      said = before == said ? mine : before;
    }
  }
  if (!(__shfl_sync(0xffffffffu, said, 0) & 1u)) return false;
  mbar_wait_drain(bar, parity, CA_WAIT_LIMIT);            // (complete: another warp has seen it)
  __syncwarp();
  return true;
}
__device__ __forceinline__ bool mbar_try_all(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_try_wait(bar, parity)); }

// Keys and values with a tile's box for one, two and four heads together.
struct CaMaps {
  CUtensorMap k[3], v[3];
};

struct CaBook {
  uint64_t full[CA_STAGES], empty[CA_STAGES], job_full[CA_JOBS], job_empty[CA_JOBS];
  int warp_part[7];
  unsigned int decision;                    // see ca_wait_on_item
  int abort_flag;
  float2 ml[2][StreamWork::ROWS];
  CaJob job[CA_JOBS];
};

// Named barriers of two warps: one arrives, the other waits.
__device__ __forceinline__ void pair_arrive(int id) { asm volatile("bar.arrive %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ void pair_sync(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }

// The entries of the query rows, for the join: a block takes every gridDim.x-th sequence.
__device__ __forceinline__ void ca_describe_rows(const CacheArgs &a, const int *off, const CaSeg *segs, int n_seg, int thread, int threads) {
  for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
    const CaSeg own = segs[a.G + b];
    const int grp = ca_group(a, b);
    CaRow row;
    row.valid = own.keys >= 0 && (grp < 0 || segs[grp].keys >= 0);
    row.pad = 0;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int s = p == 0 ? grp : a.G + b;
      CaRowPart &part = row.part[p];
      part.i0 = part.R = part.adm0 = part.causal = part.keys = part.off = part.per_head = 0;
      if (s < 0 || !row.valid) continue;
      const CaSeg g = segs[s];
      if (g.keys == 0) continue;
      const int R = g.nq * a.rep;
      int o0 = off[s], o1 = off[s + 1];
      if (!ca_streamed(R)) {
        o0 = ld_prev(a.plan + n_seg + 1 + s);
        o1 = ld_prev(a.plan + n_seg + 2 + s);
      }
      part.R = R; part.i0 = (own.q0 - g.q0) * a.rep; part.keys = g.keys; part.adm0 = g.keys - g.nq + 1; part.causal = p;
      part.off = o0; part.per_head = (o1 - o0) * (ca_streamed(R) ? ca_heads(R, a.kv, g.keys) : 1) / a.kv;
    }
    for (int r = thread; r < own.nq; r += threads) {
      CaRow mine = row;
      mine.part[0].i0 += r * a.rep;
      mine.part[1].i0 += r * a.rep;
      a.rows[own.q0 + r] = mine;
    }
  }
}

// One (maximum, sum, values) of a query row and another one: factors of both.  (What has no maximum has sums of zero.)
__device__ __forceinline__ void ca_merge(float &m, float &l, float2 other, float &f, float &g) {
  const float top = fmaxf(m, other.x);
  f = m == -INFINITY ? 0.f : fast_exp2(m - top);
  g = other.x == -INFINITY ? 0.f : fast_exp2(other.x - top);
  l = l * f + other.y * g;
  m = top;
}

// What bounds it is the memory where the cache is long: 64 sequences of 643 to 1100 rows of 32 heads, 0.89 GB, 155 us a call with its join and
// weights (5.7 TB/s), 5 sequences of 2000 to 60000 rows of 8 heads, 0.63 GB, 108 us (5.8 TB/s).  A short call is the sum of its launches'
// latencies: one token over 267 rows 12.8 us.  Two blocks fit on a processor up to 204 sequences and groups, whose list lies in shared memory too; above
// that one does, and the rate falls (32 key / value heads, rows of 400 to 600: 204 sequences 6.38 TB/s, 205 5.95; 8 heads 5.30, 4.44).  S^T = K Q^T and O^T = V^T P^T, with the keys and then the columns as the 16 rows of an
// m16n8k16 instruction and up to 8 query rows as its 8 columns: a tile of 64 keys takes half the instructions, and half the
// accumulators, of the form with (mostly empty) 16 query rows.  Rows 8 .. 15, where there are any, are a second set of columns for the
// same key and value fragments.  A warp's logits of 16 keys x 8 rows become the second product's operand by transposing two 8 x 8
// matrices between the lanes, as two terms of the element type (one request 12.6 -> 12.9 us, the others within 0.7 %; error of bf16 outputs
// against 64 bits 2.0e-3 -> 1.7e-3 of their size, which is their own rounding).  Every warp keeps its own running maximum and sums; the four meet at an item's end.
template <bool F16>
__global__ void __launch_bounds__(CA_THREADS, 2)
ca_stream_kernel(const __grid_constant__ CaMaps maps, const __grid_constant__ CacheArgs a) {
  extern __shared__ __align__(1024) uint8_t ca_smem[];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  float *join = reinterpret_cast<float *>(ca_smem + CA_STAGES * CA_STAGE_BYTES);
  const uint32_t base = smem_u32(ca_smem), q_smem = base + CA_STAGES * CA_STAGE_BYTES + CA_JOIN_BYTES;
  CaBook *bk = reinterpret_cast<CaBook *>(ca_smem + CA_STAGES * CA_STAGE_BYTES + CA_JOIN_BYTES + CA_JOBS * CA_Q_BYTES);
  const int n_seg = a.G + a.B;
  CaSeg *segs = reinterpret_cast<CaSeg *>(bk + 1);
  int *off = reinterpret_cast<int *>(segs + n_seg);
  if (threadIdx.x == 0) {
    for (int s = 0; s < CA_STAGES; ++s) {
      mbar_init(smem_u32(&bk->full[s]), 1);
      mbar_init(smem_u32(&bk->empty[s]), CA_CONSUMERS);
    }
    for (int s = 0; s < CA_JOBS; ++s) {
      mbar_init(smem_u32(&bk->job_full[s]), 1);
      mbar_init(smem_u32(&bk->job_empty[s]), CA_CONSUMERS);
    }
    bk->abort_flag = 0;
    bk->decision = 0u;
    fence_barrier_init();
  }
  if (threadIdx.x < 3) {
    tma_prefetch_desc(&maps.k[threadIdx.x]);
    tma_prefetch_desc(&maps.v[threadIdx.x]);
  }
  __syncthreads();
  WaitCtx wc{&bk->abort_flag, a.status, STATUS_CACHE_TIMEOUT, a.wait_limit};
  // Behind the tile kernel of the same call: nothing but that kernel's plan is needed from it, and its blocks have all waited for what
  // precedes the call before this kernel can start.  So this one fills the processors that it leaves, and waits for its end at its own.
  const bool behind = a.pieces[1] != 0;
  if (behind) pdl_after();
  else pdl_enter();
  const bool stop = ca_plan<StreamWork, CA_THREADS>(a, off, segs, n_seg, bk->warp_part);

  if (warp == CA_CONSUMERS) {
    // ------------------------------------------------------------------ items, query rows, key and value tiles
    // (the whole warp walks the loop and stays converged)
    const int all = stop ? 0 : off[n_seg], chunk = ca_chunk(all, a.pieces[0]), pieces = (all + chunk - 1) / chunk;
    CaWalk<StreamWork> walk;
    int piece = blockIdx.x;
    walk.begin(a, off, segs, n_seg, piece, min(all, piece * chunk), min(all, (piece + 1) * chunk));
    const uint32_t leader = warp_leader();
    RingPos pos;
    int issued = 0, used = 0;
    CaJob j;
    for (int jc = 0;; ++jc) {
      const int slot = jc % CA_JOBS;
      bool more = walk.next(a, off, segs, j);
      while (!more && pieces > (int)gridDim.x && piece < pieces) {       // the next piece (drawn: memory does not serve all blocks alike)
        unsigned int drawn = 0u;
        if (lane == 0) drawn = atomicAdd(a.work, 1u);
        piece = (int)gridDim.x + (int)__shfl_sync(0xffffffffu, drawn, 0);
        if (piece >= pieces) break;
        walk.begin(a, off, segs, n_seg, piece, piece * chunk, min(all, (piece + 1) * chunk));
        more = walk.next(a, off, segs, j);
      }
      if (!more) j.n = -1;
      // (the queue keeps working after an abort: all consumers see the same items, up to the one with -1)
      if (jc >= CA_JOBS && !mbar_try_all(smem_u32(&bk->job_empty[slot]), ((jc / CA_JOBS) - 1) & 1) &&
          !ca_wait_on(smem_u32(&bk->job_empty[slot]), ((jc / CA_JOBS) - 1) & 1, &bk->abort_flag, a.status, a.wait_limit)) {
        // (its consumers may have left too: the query rows on their way land first)
        for (int s = 0; s < CA_JOBS; ++s) mbar_settle(smem_u32(&bk->job_full[s]), ((jc - CA_JOBS + (s < slot ? CA_JOBS : 0)) / CA_JOBS) & 1, wc);
        break;
      }
      const bool going = more && !__shfl_sync(0xffffffffu, bk->abort_flag, 0);
      const uint32_t jbar = smem_u32(&bk->job_full[slot]);
      if (lane == 0) {
        bk->job[slot] = j;
        if (going) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(jbar), "r"(j.R * j.together * 256) : "memory");
        else mbar_arrive(jbar);
      }
      __syncwarp();
      if (!more) break;
      auto load_tile = [&](int kt) {
        if (used >= CA_STAGES) mbar_wait_warp(smem_u32(&bk->empty[pos.slot]), pos.phase ^ 1u, wc);
        if (!__shfl_sync(0xffffffffu, bk->abort_flag, 0)) {
          const uint32_t bar = smem_u32(&bk->full[pos.slot]), dst = base + pos.slot * CA_STAGE_BYTES;
          const int row = j.row0 + kt * (StreamWork::KEYS / j.together), box = j.together >> 1;
          mbar_expect_tx_w(bar, CA_STAGE_BYTES, leader);
          tma_load_cache_w(dst, &maps.k[box], bar, row, j.head, leader);
          tma_load_cache_w(dst + CA_STAGE_BYTES / 2, &maps.v[box], bar, row, j.head, leader);
          issued = used + 1;
        }
        ++used;
        pos.step(CA_STAGES);
      };
      const bool early = used < CA_STAGES;       // (nothing to wait for)
      if (early) load_tile(j.kt0);
      if (going && lane < j.R * j.together) {
        const int sub = lane / j.R, i = lane - sub * j.R, t = i / a.rep;
        const uint16_t *src = a.q + (long long)(j.q0 + t) * a.q_row + (long long)((j.head + sub) * a.rep + (i - t * a.rep)) * a.q_head;
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], 256, [%2];"
                     ::"r"(q_smem + slot * CA_Q_BYTES + lane * CA_Q_PITCH), "l"(src), "r"(jbar) : "memory");
      }
      __syncwarp();
      for (int kt = j.kt0 + (early ? 1 : 0); kt < j.kt0 + j.n; ++kt) load_tile(kt);
    }
    // every copy issued has landed before the block leaves (the consumers wait for the query rows whatever happens)
    for (int s = 0; s < CA_STAGES; ++s) {
      const int fills = issued > s ? (issued - s + CA_STAGES - 1) / CA_STAGES : 0;
      if (fills > 0) mbar_settle(smem_u32(&bk->full[s]), (fills - 1) & 1, wc);
    }
    // the block that leaves last puts the counters back to zero for the next launch (every block has drawn its last piece by then)
    if (pieces > (int)gridDim.x && lane == 0 && atomicAdd(a.work + 1, 1u) == gridDim.x - 1) {
      a.work[0] = 0u;
      a.work[1] = 0u;
      __threadfence();
    }
    if (behind) pdl_wait();
    __syncwarp();
    return;
  }
  // -------------------------------------------------------------------- consumers
  if (!stop && !behind) ca_describe_rows(a, off, segs, n_seg, threadIdx.x, 32 * CA_CONSUMERS);
  const int gq = lane >> 2, tq = lane & 3;       // fragment row / column pair
  const int mi = lane >> 3, mr = lane & 7;       // matrix of an ldmatrix, row in it
  RingPos pos;
  bool handed = false;                           // (warps 2 and 3) the buffer holds something that may not have been read yet
  for (int jc = 0;; ++jc) {
    const int slot = jc % CA_JOBS;
    if (!mbar_try_all(smem_u32(&bk->job_full[slot]), (jc / CA_JOBS) & 1) &&
        !ca_wait_on_item(&bk->decision, jc, smem_u32(&bk->job_full[slot]), (jc / CA_JOBS) & 1, &bk->abort_flag, a.status, a.wait_limit))
      break;
    const CaJob j = bk->job[slot];
    if (j.n < 0) break;
    const bool two = j.R > 8;                    // rows 8 .. 15 are in use
    // Four heads together: a warp each.  Two: warps 0 and 2, 1 and 3 share one's keys.  One: all four do.
    const int hg = j.together, sub = warp & (hg - 1), slice = warp / hg, keys = StreamWork::KEYS / hg, head = j.head + sub;
    const int half_bytes = keys * 128, warp_off = (2 * sub * keys + slice * 16) * 128;       // a column half; this warp's 16 keys in a tile
    uint32_t qb[2][8][2];                        // the query rows as the second operand, a k-step each; [rows 0 .. 7, 8 .. 15]
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int k2 = 0; k2 < 4; ++k2) {
        uint32_t r[4] = {0u, 0u, 0u, 0u};
        if (h == 0 || two) ldsm4(q_smem + slot * CA_Q_BYTES + min(sub * j.R + h * 8 + mr, 15) * CA_Q_PITCH + (k2 * 4 + mi) * 16, r);    // (past the last row: any)
        qb[h][2 * k2][0] = r[0]; qb[h][2 * k2][1] = r[1];
        qb[h][2 * k2 + 1][0] = r[2]; qb[h][2 * k2 + 1][1] = r[3];
      }
    __syncwarp();
    mbar_arrive_lane0(smem_u32(&bk->job_empty[slot]), lane);
    int adm[2][2];                               // admitted keys of query rows 8 h + 2 tq + e (rows past the last: none, whatever the buffer held)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int i = 8 * h + 2 * tq + e;
        adm[h][e] = i < j.R ? ca_admitted(j, i / a.rep) : 0;
      }
    // (query row, head) of row 8 h + 2 tq + e; -1: none
    auto entry_of = [&](int h, int e) -> long long {
      const int i = 8 * h + 2 * tq + e, t = i / a.rep;
      return i < j.R ? (long long)(j.q0 + t) * a.H + head * a.rep + (i - t * a.rep) : -1;
    };
    float o[2][8][4];                            // [][16 columns][column gq or gq + 8, row 2 tq or 2 tq + 1]
    float m[2][2], l[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[h][n][e] = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) { m[h][e] = -INFINITY; l[h][e] = 0.f; }
    }
    float *lrow[2][2];                           // this lane's place in the rows of logits
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const long long entry = a.logits ? entry_of(h, e) : -1;
        lrow[h][e] = entry < 0 ? nullptr : a.logits + entry * a.pitch + (j.causal ? a.own_off : 0) + gq;
      }
    // One tile; TWO: with rows 8 .. 15 (both sets step by step, so that neither waits for the other's latencies).
    auto tile = [&](auto two_sets, int kt) {
      constexpr int SETS = decltype(two_sets)::value;
      const uint32_t ks = base + pos.slot * CA_STAGE_BYTES + warp_off, vs = ks + CA_STAGE_BYTES / 2;
      const int j0 = kt * keys + slice * 16;     // this warp's first key
      // ---- logits of 16 keys x 8 rows: x[][2 c + e] is key gq + 8 c, row 2 tq + e
      float x[SETS][4], y[SETS][4];
#pragma unroll
      for (int h = 0; h < SETS; ++h)
#pragma unroll
        for (int c = 0; c < 4; ++c) x[h][c] = y[h][c] = 0.f;
      {
        const int key = (mi & 1) * 8 + mr;
        const uint32_t row = ks + key * 128;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {         // (two chains)
          const int c = kk * 2 + (mi >> 1);
          uint32_t k[4];
          ldsm4(row + (kk >> 2) * half_bytes + (((c & 7) ^ (key & 7)) << 4), k);
#pragma unroll
          for (int h = 0; h < SETS; ++h) mma16816<F16>(kk & 1 ? y[h] : x[h], k, qb[h][kk][0], qb[h][kk][1]);
        }
      }
#pragma unroll
      for (int h = 0; h < SETS; ++h)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int key = j0 + gq + 8 * (c >> 1);
          x[h][c] = key < adm[h][c & 1] ? (x[h][c] + y[h][c]) * a.scale_log2 : -INFINITY;
        }
#pragma unroll
      for (int h = 0; h < SETS; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (lrow[h][e]) {
            lrow[h][e][j0] = x[h][e];
            lrow[h][e][j0 + 8] = x[h][2 + e];
          }
      // ---- probabilities relative to the running maximum
      float mx[SETS][2];
      bool up = false;
#pragma unroll
      for (int h = 0; h < SETS; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) mx[h][e] = fmaxf(x[h][e], x[h][2 + e]);
#pragma unroll
      for (int s = 4; s < 32; s <<= 1)
#pragma unroll
        for (int h = 0; h < SETS; ++h)
#pragma unroll
          for (int e = 0; e < 2; ++e) mx[h][e] = fmaxf(mx[h][e], __shfl_xor_sync(0xffffffffu, mx[h][e], s));
#pragma unroll
      for (int h = 0; h < SETS; ++h) up = up || mx[h][0] > m[h][0] || mx[h][1] > m[h][1];
      if (__any_sync(0xffffffffu, up)) {
#pragma unroll
        for (int h = 0; h < SETS; ++h) {
          float f[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float top = fmaxf(m[h][e], mx[h][e]);
            f[e] = top == m[h][e] ? 1.f : fast_exp2(m[h][e] - top);
            m[h][e] = top;
            l[h][e] *= f[e];
          }
#pragma unroll
          for (int n = 0; n < 8; ++n) { o[h][n][0] *= f[0]; o[h][n][1] *= f[1]; o[h][n][2] *= f[0]; o[h][n][3] *= f[1]; }
        }
      }
      // Probabilities of keys gq and gq + 8, rows 2 tq and 2 tq + 1, as two terms of the element type: truncated, and what that leaves.  The
      // instructions of the second one fit into the waits for memory, and the output is as exact as one of probabilities in 32 bits.  The
      // remainder of a probability above zero stays above zero, so that an infinite value stays one (0 * inf is NaN).
      constexpr float LEAST = F16 ? 0x1p-24f : 0x1p-126f;
      uint32_t p0[SETS], p1[SETS], r0[SETS], r1[SETS];
#pragma unroll
      for (int h = 0; h < SETS; ++h) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float ref = m[h][e] == -INFINITY ? 0.f : m[h][e];
          p[e] = fast_exp2(x[h][e] - ref);
          p[2 + e] = fast_exp2(x[h][2 + e] - ref);
          l[h][e] += p[e] + p[2 + e];
        }
        p0[h] = pack2_rz<F16>(p[0], p[1]);
        p1[h] = pack2_rz<F16>(p[2], p[3]);
        const float2 a0 = unpack2_t<F16>(p0[h]), a1 = unpack2_t<F16>(p1[h]);
        r0[h] = pack2_t<F16>(fmaxf(p[0] - a0.x, fminf(p[0], LEAST)), fmaxf(p[1] - a0.y, fminf(p[1], LEAST)));
        r1[h] = pack2_t<F16>(fmaxf(p[2] - a1.x, fminf(p[2], LEAST)), fmaxf(p[3] - a1.y, fminf(p[3], LEAST)));
      }
      // ---- values.  Rows that no query row of the tile admits are cleared (0 * NaN is NaN).  A row that only some of them
      // admit may hold infinities or NaN too: then its part is added without the matrix instruction, to the rows that admit it.
      if (j0 + 16 > (j.causal ? j.adm0 : j.keys)) {
        const int r = lane >> 1, half = lane & 1;           // two lanes per key
        const bool dead = j0 + r >= j.keys;
        uint8_t *values = ca_smem + pos.slot * CA_STAGE_BYTES + CA_STAGE_BYTES / 2 + warp_off, *vrow = values + half * half_bytes + r * 128;
        uint32_t hit = 0u;
        if (!dead)
          for (int c = 0; c < 8; ++c) {
            const uint4 v = reinterpret_cast<const uint4 *>(vrow)[c];
            hit |= not_finite_bits<F16>(v.x) | not_finite_bits<F16>(v.y) | not_finite_bits<F16>(v.z) | not_finite_bits<F16>(v.w);
          }
        const uint32_t who = __ballot_sync(0xffffffffu, hit != 0u);
        if (dead)
          for (int c = 0; c < 8; ++c) reinterpret_cast<uint4 *>(vrow)[c] = make_uint4(0u, 0u, 0u, 0u);
        __syncwarp();
        if (who) {
          uint32_t bad = 0u;                     // keys of this warp's 16 to be added apart
#pragma unroll
          for (int e = 0; e < 16; ++e) bad |= ((who >> (2 * e)) & 3u) ? 1u << e : 0u;
          for (uint32_t left = bad; left; left &= left - 1) {
            const int k = __ffs(left) - 1;
#pragma unroll
            for (int h = 0; h < SETS; ++h) {
              float2 pk = unpack2_t<F16>(__shfl_sync(0xffffffffu, (k & 8) ? p1[h] : p0[h], (k & 7) * 4 + tq));
              const float2 rk = unpack2_t<F16>(__shfl_sync(0xffffffffu, (k & 8) ? r1[h] : r0[h], (k & 7) * 4 + tq));
              pk.x += rk.x;
              pk.y += rk.y;
              const bool in0 = j0 + k < adm[h][0], in1 = j0 + k < adm[h][1];
#pragma unroll
              for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {    // column 16 n + 8 c + gq
                  const int chunk = 2 * n + c;
                  const uint16_t w = *reinterpret_cast<const uint16_t *>(values + (chunk >> 3) * half_bytes + k * 128 + (((chunk & 7) ^ (k & 7)) << 4) + 2 * gq);
                  const float v = unpack2_t<F16>(w).x;
                  if (in0) o[h][n][2 * c] += pk.x * v;
                  if (in1) o[h][n][2 * c + 1] += pk.y * v;
                }
            }
          }
          __syncwarp();
          if ((bad >> r) & 1u)
            for (int c = 0; c < 8; ++c) reinterpret_cast<uint4 *>(vrow)[c] = make_uint4(0u, 0u, 0u, 0u);
          __syncwarp();
        }
        fence_proxy_async();                     // these writes come before the next copy into the slot
      }
      uint32_t b0[SETS], b1[SETS];
#pragma unroll
      for (int h = 0; h < SETS; ++h) {
        b0[h] = transpose8x8(p0[h]); b1[h] = transpose8x8(p1[h]);
        r0[h] = transpose8x8(r0[h]); r1[h] = transpose8x8(r1[h]);
      }
      {
        const int key = (mi >> 1) * 8 + mr;
        const uint32_t row = vs + key * 128;
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          const int c = 2 * n + (mi & 1);
          uint32_t v[4];
          ldsm4t(row + (n >> 2) * half_bytes + (((c & 7) ^ (key & 7)) << 4), v);
#pragma unroll
          for (int h = 0; h < SETS; ++h) mma16816<F16>(o[h][n], v, b0[h], b1[h]);
#pragma unroll
          for (int h = 0; h < SETS; ++h) mma16816<F16>(o[h][n], v, r0[h], r1[h]);
        }
      }
    };
    for (int kt = j.kt0; kt < j.kt0 + j.n; ++kt) {
      mbar_wait_warp(smem_u32(&bk->full[pos.slot]), pos.phase, wc);
      if (two) tile(std::integral_constant<int, 2>{}, kt);
      else tile(std::integral_constant<int, 1>{}, kt);
      __syncwarp();
      mbar_arrive_lane0(smem_u32(&bk->empty[pos.slot]), lane);
      pos.step(CA_STAGES);
    }
    // ---- the sums of the warps that share a head: 2 -> 0 and 3 -> 1, then (one head) 1 -> 0; the last one stores.  Values stay in fragment order, and the warps that
    // hand theirs on go on to the next item.  (Through a buffer of whole rows that all four read, with a barrier of all four before and
    // after each piece of it, an item's end took 3700 to 4700 clocks.)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (h == 1 && !two) continue;
#pragma unroll
        for (int s = 4; s < 32; s <<= 1) l[h][e] += __shfl_xor_sync(0xffffffffu, l[h][e], s);
        if (l[h][e] != l[h][e] && m[h][e] == -INFINITY) m[h][e] = 0.f;      // every logit was NaN: not an empty row
      }
    float4 *buf = reinterpret_cast<float4 *>(join) + (warp & 1) * (CA_JOIN_BYTES / 32);
    // Columns 16 N0 .. 16 N1 - 1 of rows 8 h ..; the maxima and sums go with the first.
    float fac[2][4];                             // factors of both sums of either step
    auto pass = [&](auto n0, auto n1, auto hh) {
      constexpr int N0 = decltype(n0)::value, N1 = decltype(n1)::value, h = decltype(hh)::value;
      const int cols = (min(8, j.R - 8 * h) + 1) >> 1;       // values of tq in use
      const bool on = tq < cols;
      auto put = [&]() {
        if (N0 == 0 && gq == 0) {
          bk->ml[warp & 1][8 * h + 2 * tq] = make_float2(m[h][0], l[h][0]);
          bk->ml[warp & 1][8 * h + 2 * tq + 1] = make_float2(m[h][1], l[h][1]);
        }
        if (on)
#pragma unroll
          for (int n = N0; n < N1; ++n) buf[((n - N0) * 8 + gq) * cols + tq] = make_float4(o[h][n][0], o[h][n][1], o[h][n][2], o[h][n][3]);
      };
      auto get = [&](const float4 *from, const float2 *other, int step) {
        if (N0 == 0)
#pragma unroll
          for (int e = 0; e < 2; ++e) ca_merge(m[h][e], l[h][e], other[8 * h + 2 * tq + e], fac[e][2 * step], fac[e][2 * step + 1]);
        if (on)
#pragma unroll
          for (int n = N0; n < N1; ++n) {
            const float4 v = from[((n - N0) * 8 + gq) * cols + tq];
            o[h][n][0] = o[h][n][0] * fac[0][2 * step] + v.x * fac[0][2 * step + 1];
            o[h][n][1] = o[h][n][1] * fac[1][2 * step] + v.y * fac[1][2 * step + 1];
            o[h][n][2] = o[h][n][2] * fac[0][2 * step] + v.z * fac[0][2 * step + 1];
            o[h][n][3] = o[h][n][3] * fac[1][2 * step] + v.w * fac[1][2 * step + 1];
          }
      };
      if (warp >= 2) {
        if (handed) pair_sync(4 + (warp & 1));   // the buffer has been read
        handed = true;
        put();
        pair_arrive(1 + (warp & 1));
        return;
      }
      pair_sync(1 + warp);
      get(buf, bk->ml[warp], 0);
      __syncwarp();
      if (hg == 2) {
        pair_arrive(4 + warp);
      } else if (warp == 0) {
        pair_arrive(4);
        pair_sync(3);
        get(reinterpret_cast<const float4 *>(join) + CA_JOIN_BYTES / 32, bk->ml[1], 1);
        __syncwarp();
        pair_arrive(5);
      } else {
        put();                                   // (the warp's own buffer: warp 3's values are in registers)
        pair_arrive(3);
      }
    };
    using std::integral_constant;
    constexpr integral_constant<int, 0> c0{};
    constexpr integral_constant<int, 1> c1{};
    constexpr integral_constant<int, 4> c4{};
    constexpr integral_constant<int, 8> c8{};
    if (hg == 4) {
    } else if (j.R <= 4) {
      pass(c0, c8, c0);
    } else {
      pass(c0, c4, c0);
      pass(c4, c8, c0);
      if (two) {
        pass(c0, c4, c1);
        pass(c4, c8, c1);
      }
    }
    if (slice == 0 && !bk->abort_flag) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const long long entry = entry_of(h, e);
          if (entry < 0) continue;
          const long long at = j.complete ? (j.causal ? (long long)a.n_q * a.H : 0) + entry : (long long)j.record * a.rec_rows + sub * j.R + 8 * h + 2 * tq + e;
          float *dst = (j.complete ? a.full_o : a.rec_o[0]) + at * 128 + gq;
#pragma unroll
          for (int n = 0; n < 8; ++n) {
            dst[16 * n] = o[h][n][e];
            dst[16 * n + 8] = o[h][n][2 + e];
          }
          if (gq == 0) (j.complete ? a.full_ml : a.rec_ml[0])[at] = make_float2(m[h][e], l[h][e]);
        }
    }
  }
  if (handed) pair_sync(4 + (warp & 1));         // (every arrival is met)
  if (behind) {
    pdl_wait();
    if (!stop) ca_describe_rows(a, off, segs, n_seg, threadIdx.x, 32 * CA_CONSUMERS);
  }
}

// ---------------------------------------------------------------------------------------
// Segments of more than 16 stacked rows.  Persistent blocks; two row tiles of 128 rows share every key and value tile of 128 keys and take
// turns on the tensor pipe: S = Q K^T into tensor memory, one thread per row turns it into probabilities relative to a reference
// maximum, P goes back to tensor memory in the element type, O += P V accumulates there.  (P rounded to the element type: the second product
// takes no other.  A second term would be half as many products again, and tensor memory is full.  Error of bf16 outputs against 64 bits 2.3e-3 of
// their size, 1.7e-3 of which is their own rounding.)
// What bounds it: a pair of key tiles takes 2300 to 2750 clocks, near the products' own rate, but an item's ends cost 8000 to 10000 more (the
// first tile's maximum, 128 KB of results a block, nothing for the tensor pipe to do meanwhile) and a launch 11 us before its first
// product: 13 sequences of 16 to 256 query rows over prefixes of 2915 rows, 32 heads: 142 us of the call's 198, where the
// products alone are 69 at the measured rate; the tensor pipe is active for 49 % of the cycles.  (Results through shared memory, queries gathered and items counted two tiles longer
// than their keys, in place of four: 175.)
// ---------------------------------------------------------------------------------------
constexpr int CT_THREADS = 384;                 // warp 0: key / value copies, 1: MMA issue, 2: value rows to be cleared, 3: query rows, 4-11: softmax
constexpr int CT_TILE_BYTES = 128 * 128 * 2;
constexpr int CT_BLOCK_BYTES = CT_TILE_BYTES / 2;
constexpr int CT_SLOTS = 4;                     // ring of key and value tiles in the order K0 V0 K1 V1 ...
constexpr int CT_BOOK_OFF = (2 + CT_SLOTS) * CT_TILE_BYTES;
constexpr int CT_JOBS = 4;                      // items announced ahead
constexpr uint32_t CT_TMEM_COLS = 512, CT_S_COL = 256, CT_P_COL = 384;   // O of both row tiles, one S that they use in turn, P of both
// A tile's sum relative to the reference at which the reference moves: no probability may leave the element type's range.
constexpr float CT_SUM_LIMIT_BF16 = 1.0995116e12f, CT_SUM_LIMIT_F16 = 32768.f;

struct CtBook {
  uint64_t full[CT_SLOTS], empty[CT_SLOTS], raw[CT_SLOTS];
  uint64_t q_full[2], q_empty[2], s_full[2], s_empty, p_ready[2], pv_done[2], mma_done, job_full[CT_JOBS], job_empty[CT_JOBS];
  CaJob job[CT_JOBS];
  int warp_part[CT_THREADS / 32];
  uint32_t tmem_base;
  int abort_flag;
  int bad[2 * CT_JOBS];    // the item (modulo their number) has value rows with infinities or NaN that not all of its query rows admit.  The softmax warps
                           // read it at the item's end; warp 2 may then be CT_JOBS items further on, where the next one's announcement waits for them
};

// Key tile kt holds rows that not all query rows of the pair admit: its values pass through warp 2.
__device__ __forceinline__ bool ct_passed(const CaJob &j, int rep, int kt) {
  return (kt + 1) * 128 > ca_admitted(j, j.causal ? j.rt * TileWork::ROWS / rep : 0);
}

template <bool F16, bool WEIGHTS>
__global__ void __launch_bounds__(CT_THREADS, 1)
ca_tile_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ CUtensorMap tmap_q,
               const __grid_constant__ CacheArgs a) {
  extern __shared__ __align__(1024) uint8_t ct_smem[];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(ct_smem), q_smem = base, ring = base + 2 * CT_TILE_BYTES;
  CtBook *bk = reinterpret_cast<CtBook *>(ct_smem + CT_BOOK_OFF);
  const int n_seg = a.G + a.B;
  CaSeg *segs = reinterpret_cast<CaSeg *>(bk + 1);
  int *off = reinterpret_cast<int *>(segs + n_seg);
  if (threadIdx.x == 0) {
    for (int s = 0; s < CT_JOBS; ++s) {
      mbar_init(smem_u32(&bk->job_full[s]), 1);
      mbar_init(smem_u32(&bk->job_empty[s]), 11);           // the MMA issuer, warps 2 and 3, every softmax warp
    }
    for (int s = 0; s < CT_SLOTS; ++s) {
      mbar_init(smem_u32(&bk->full[s]), 1);
      mbar_init(smem_u32(&bk->empty[s]), 1);
      mbar_init(smem_u32(&bk->raw[s]), 1);
    }
    for (int g = 0; g < 2; ++g) {
      mbar_init(smem_u32(&bk->q_full[g]), 1);
      mbar_init(smem_u32(&bk->q_empty[g]), 1);
      mbar_init(smem_u32(&bk->s_full[g]), 1);
      mbar_init(smem_u32(&bk->p_ready[g]), 4);            // the row tile's four softmax warps
      mbar_init(smem_u32(&bk->pv_done[g]), 1);
    }
    mbar_init(smem_u32(&bk->s_empty), 4);                 // the softmax warps that have taken an S into registers
    mbar_init(smem_u32(&bk->mma_done), 1);
    bk->abort_flag = 0;
    for (int i = 0; i < 2 * CT_JOBS; ++i) bk->bad[i] = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tmap_k);
    tma_prefetch_desc(&tmap_v);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&bk->tmem_base), CT_TMEM_COLS);
    tmem_relinquish();
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = bk->tmem_base;
  WaitCtx wc{&bk->abort_flag, a.status, STATUS_CACHE_TIMEOUT, a.wait_limit};
  pdl_enter();
  const bool stop = ca_plan<TileWork, CT_THREADS>(a, off, segs, n_seg, bk->warp_part);
  // the next item; false: there is none, or the block gives up
  auto take = [&](int jc, CaJob &j) {
    const int slot = jc % CT_JOBS;
    if (!mbar_wait_all(smem_u32(&bk->job_full[slot]), (jc / CT_JOBS) & 1, wc)) return false;
    j = bk->job[slot];
    __syncwarp();
    mbar_arrive_lane0(smem_u32(&bk->job_empty[slot]), lane);
    return j.n >= 0;
  };

  // The launch gives every thread 168 registers; a softmax thread holds its row's 128 logits and needs more, the first
  // warpgroup needs few: 128 x 72 + 256 x 216 = 384 x 168.
  if (warp < 4) {
    reg_dec<72>();
    if (warp == 0) {
      // ---------------------------------------------------------------- items, key / value tiles
      const uint32_t leader = warp_leader();
      const int all = stop ? 0 : off[n_seg], chunk = ca_chunk(all, a.pieces[1]);        // (a piece per block)
      CaWalk<TileWork> walk;
      walk.begin(a, off, segs, n_seg, blockIdx.x, min(all, (int)blockIdx.x * chunk), min(all, ((int)blockIdx.x + 1) * chunk));
      CaJob j;
      int tc = 0, issued = 0;
      uint32_t raw_any = 0u, raw_odd = 0u, raw_last = 0u;     // per ring slot: copies through `raw`: any, an odd number, the latest one
      for (int jc = 0;; ++jc) {
        const int slot = jc % CT_JOBS;
        const bool more = walk.next(a, off, segs, j);
        if (more) {
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const int i0 = j.rt * TileWork::ROWS + g * 128, last = min(i0 + 128, j.R) - 1;
            j.n_act[g] = i0 < j.R ? max(0, min(j.kt0 + j.n, (ca_admitted(j, j.causal ? last / a.rep : 0) + 127) / 128) - j.kt0) : 0;
          }
        } else {
          j.n = -1;
        }
        // (after an abort nothing more is announced: the flag ends every wait of the consumers)
        if (jc >= CT_JOBS && !mbar_wait_all(smem_u32(&bk->job_empty[slot]), ((jc / CT_JOBS) - 1) & 1, wc)) break;
        if (__shfl_sync(0xffffffffu, bk->abort_flag, 0)) break;
        if (lane == 0) bk->job[slot] = j;
        mbar_arrive_lane0(smem_u32(&bk->job_full[slot]), lane);
        if (!more) break;
#pragma unroll 1
        for (int kt = j.kt0; kt < j.kt0 + j.n; ++kt) {
          const bool passed = ct_passed(j, a.rep, kt);
#pragma unroll
          for (int kv = 0; kv < 2; ++kv, ++tc) {
            const int s = tc % CT_SLOTS;
            if (tc >= CT_SLOTS) mbar_wait_warp(smem_u32(&bk->empty[s]), ((tc / CT_SLOTS) - 1) & 1, wc);
            if (__shfl_sync(0xffffffffu, bk->abort_flag, 0)) continue;
            const bool past = passed && kv == 1;
            const uint32_t bar = smem_u32(past ? &bk->raw[s] : &bk->full[s]), dst = ring + s * CT_TILE_BYTES, bit = 1u << s;
            raw_last = past ? raw_last | bit : raw_last & ~bit;
            if (past) { raw_any |= bit; raw_odd ^= bit; }
            const int row = j.row0 + kt * 128;
            mbar_expect_tx_w(bar, CT_TILE_BYTES, leader);
            tma_load_cache_w(dst, kv ? &tmap_v : &tmap_k, bar, row, j.head, leader);
            issued = tc + 1;
          }
        }
      }
      // every copy issued has landed before the block leaves
      for (int s = 0; s < CT_SLOTS; ++s) {
        const int fills = issued > s ? (issued - s + CT_SLOTS - 1) / CT_SLOTS : 0;
        if ((raw_any >> s) & 1u) mbar_settle(smem_u32(&bk->raw[s]), ((raw_odd >> s) & 1u) ^ 1u, wc);
        if (fills > 0 && !((raw_last >> s) & 1u)) mbar_settle(smem_u32(&bk->full[s]), (fills - 1) & 1, wc);
      }
      __syncwarp();
    } else if (warp == 1) {
      // ---------------------------------------------------------------- MMA issuer
      // Per key tile and row tile: S of this key tile, then P V of the previous one (an S never waits in the pipe behind a P V that could
      // as well run after it).  The whole warp walks the loop and stays converged (see warp_leader).
      const uint32_t leader = warp_leader();
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem_base, 0);
      const uint32_t idesc_s = F16 ? umma_idesc_f16(128, 128) : umma_idesc_bf16(128, 128), idesc_o = idesc_s | UMMA_IDESC_B_MN;
      const uint64_t qdesc = umma_desc_sw128(q_smem), tile0 = umma_desc_sw128(ring), vtile0 = umma_desc_sw128_mn(ring, CT_BLOCK_BYTES);
      int t0 = 0;                                 // first tile of the item in the ring
      int qc[2] = {0, 0}, pc[2] = {0, 0}, sn = 0; // query tiles, P tiles and S so far
      CaJob j;
      for (int jc = 0; take(jc, j); ++jc) {
        auto field = [&](int f) { return __shfl_sync(0xffffffffu, f, 0); };
        const int n[2] = {field(j.n_act[0]), field(j.n_act[1])}, n_max = field(j.n);
        for (int kt = 0; kt <= n_max; ++kt) {
          const int tk = t0 + 2 * kt, tv = tk - 1;            // ring tiles: K of this key tile, V of the previous one
          const int sk = tk & (CT_SLOTS - 1), sv = tv & (CT_SLOTS - 1);
          if (kt < n_max) mbar_wait_warp(smem_u32(&bk->full[sk]), (tk / CT_SLOTS) & 1, wc);
          if (kt > 0) mbar_wait_warp(smem_u32(&bk->full[sv]), (tv / CT_SLOTS) & 1, wc);
          const uint64_t kdesc = tile0 + sk * (CT_TILE_BYTES >> 4), vdesc = vtile0 + sv * (CT_TILE_BYTES >> 4);
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (kt < n[g]) {
              if (kt == 0) {
                mbar_wait_warp(smem_u32(&bk->q_full[g]), qc[g] & 1, wc);
                ++qc[g];
              }
              if (sn > 0) mbar_wait_warp(smem_u32(&bk->s_empty), (sn - 1) & 1, wc);     // the previous S is in registers
              ++sn;
              tc_fence_after();
              tc_mma_bf16_k128_w(tm + CT_S_COL, qdesc + g * (CT_TILE_BYTES >> 4), kdesc, CT_BLOCK_BYTES, CT_BLOCK_BYTES, idesc_s, leader);
              tc_commit_w(smem_u32(&bk->s_full[g]), leader);
              if (kt == n[g] - 1) tc_commit_w(smem_u32(&bk->q_empty[g]), leader);
            }
            if (kt > 0 && kt - 1 < n[g]) {
              mbar_wait_warp(smem_u32(&bk->p_ready[g]), pc[g] & 1, wc);
              ++pc[g];
              tc_fence_after();
#pragma unroll
              for (int kk = 0; kk < 8; ++kk)
                tc_mma_bf16_ta_w(tm + g * 128, tm + CT_P_COL + g * 64 + kk * 8, vdesc + kk * (2048 >> 4), idesc_o,
                                 (kt > 1 || kk > 0) ? 1u : 0u, leader);
              tc_commit_w(smem_u32(&bk->pv_done[g]), leader);
            }
          }
          if (kt < n_max) tc_commit_w(smem_u32(&bk->empty[sk]), leader);
          if (kt > 0) tc_commit_w(smem_u32(&bk->empty[sv]), leader);
        }
        t0 += 2 * n_max;
      }
      // every MMA this warp issued has completed before tensor memory is given back
      tc_commit_w(smem_u32(&bk->mma_done), leader);
      mbar_settle(smem_u32(&bk->mma_done), 0, wc);
      __syncwarp();
    } else if (warp == 2) {
      // ---------------------------------------------------------------- value rows that must not reach every query row
      // Their probabilities are exactly zero there, but 0 * NaN is NaN: rows past the segment are cleared, and elements that are not finite
      // in rows that only some query rows admit are cleared too and added by the softmax warps at the item's end (bk->bad).
      int t0 = 0;
      uint32_t raw_phase = 0u;                    // per ring slot
      CaJob j;
      for (int jc = 0; take(jc, j); ++jc) {
        if (lane == 0) *reinterpret_cast<volatile int *>(&bk->bad[jc % (2 * CT_JOBS)]) = 0;
        __syncwarp();
        for (int k = 0; k < j.n; ++k) {
          const int kt = j.kt0 + k;
          if (!ct_passed(j, a.rep, kt)) continue;
          const int s = (t0 + 2 * k + 1) & (CT_SLOTS - 1);
          const bool landed = mbar_wait(smem_u32(&bk->raw[s]), (raw_phase >> s) & 1u, wc);
          raw_phase ^= 1u << s;
          if (!__all_sync(0xffffffffu, landed)) continue;     // (gave up: the copy may not have been issued)
          uint8_t *tile = ct_smem + (2 + s) * CT_TILE_BYTES;
          const int rows = max(0, min(128, j.keys - kt * 128));             // rows of the segment
          const int free_rows = max(0, min(rows, ca_admitted(j, j.causal ? j.rt * TileWork::ROWS / a.rep : 0) - kt * 128));   // ... that all query rows admit
          uint32_t hit = 0u;
#pragma unroll 8
          for (int i = free_rows * 8 + lane; i < rows * 8; i += 32)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint4 x = reinterpret_cast<const uint4 *>(tile + h * CT_BLOCK_BYTES)[i];
              hit |= not_finite_bits<F16>(x.x) | not_finite_bits<F16>(x.y) | not_finite_bits<F16>(x.z) | not_finite_bits<F16>(x.w);
            }
          for (int i = rows * 8 + lane; i < 128 * 8; i += 32) {
            reinterpret_cast<uint4 *>(tile)[i] = make_uint4(0u, 0u, 0u, 0u);
            reinterpret_cast<uint4 *>(tile + CT_BLOCK_BYTES)[i] = make_uint4(0u, 0u, 0u, 0u);
          }
          if (__any_sync(0xffffffffu, hit != 0u)) {
            for (int i = free_rows * 16 + lane; i < rows * 16; i += 32) {
              uint4 *p = reinterpret_cast<uint4 *>(tile + (i & 1) * CT_BLOCK_BYTES) + (i >> 1);
              uint4 x = *p;
              uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t b = not_finite_bits<F16>(w[e]);
                if (b & 0x8000u) w[e] &= 0xffff0000u;
                if (b & 0x80000000u) w[e] &= 0xffffu;
              }
              *p = make_uint4(w[0], w[1], w[2], w[3]);
            }
            if (lane == 0) *reinterpret_cast<volatile int *>(&bk->bad[jc % (2 * CT_JOBS)]) = 1;
          }
          __threadfence_block();
          fence_proxy_async();
          __syncwarp();
          mbar_arrive_lane0(smem_u32(&bk->full[s]), lane);
        }
        t0 += 2 * j.n;
      }
    } else {
      // ---------------------------------------------------------------- query rows
      // Stacked row i is query row i / rep, head i % rep of the key / value head; rows past the last one hold anything (other sequences' query
      // rows, or what the buffer held), nothing of theirs is used.  One tiled copy where rep divides 128 (see make_query_map); otherwise
      // gathered, a lane working out the addresses of four rows and sixteen lanes copying a row.
      const uint32_t leader = warp_leader();
      int tiled[2] = {0, 0};                      // tiled copies issued
      int qc[2] = {0, 0};
      CaJob j;
      for (int jc = 0; take(jc, j); ++jc) {
#pragma unroll 1
        for (int g = 0; g < 2; ++g) {
          if ((g ? j.n_act[1] : j.n_act[0]) == 0) continue;
          if ((g ? qc[1] : qc[0]) >= 1) mbar_wait_warp(smem_u32(&bk->q_empty[g]), ((g ? qc[1] : qc[0]) - 1) & 1, wc);
          if (g) ++qc[1];
          else ++qc[0];
          const int i0 = j.rt * TileWork::ROWS + g * 128, n = min(128, j.R - i0);
          if (a.q_tiled) {
            if (!__shfl_sync(0xffffffffu, bk->abort_flag, 0)) {
              mbar_expect_tx_w(smem_u32(&bk->q_full[g]), CT_TILE_BYTES, leader);
              tma_load_query_w(q_smem + g * CT_TILE_BYTES, &tmap_q, smem_u32(&bk->q_full[g]), j.q0 + i0 / a.rep, j.head, leader);
              if (g) tiled[1] = qc[1];
              else tiled[0] = qc[0];
            }
            continue;
          }
          const int c = lane & 15;                // 16-byte piece of a row
          long long from[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int i = min(i0 + 32 * k + lane, j.R - 1), t = i / a.rep;
            from[k] = (long long)(j.q0 + t) * a.q_row + (long long)(j.head * a.rep + (i - t * a.rep)) * a.q_head;
          }
          const uint32_t dst = q_smem + g * CT_TILE_BYTES + (c >> 3) * CT_BLOCK_BYTES;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (32 * k >= n) continue;
#pragma unroll 4
            for (int r2 = 0; r2 < 32; r2 += 2) {
              const int r = 32 * k + r2 + (lane >> 4);
              const long long at = __shfl_sync(0xffffffffu, from[k], r2 + (lane >> 4));
              cp_async16(dst + r * 128 + (((c & 7) ^ (r & 7)) << 4), a.q + at + c * 8);
            }
          }
          cp_async_commit();
          cp_async_wait<0>();
          fence_proxy_async();
          __syncwarp();
          mbar_arrive_lane0(smem_u32(&bk->q_full[g]), lane);
        }
      }
      // every copy issued has landed before the block leaves
      for (int g = 0; g < 2; ++g)
        if ((g ? tiled[1] : tiled[0]) > 0) mbar_settle(smem_u32(&bk->q_full[g]), ((g ? tiled[1] : tiled[0]) - 1) & 1, wc);
      __syncwarp();
    }
  } else {
    reg_inc<216>();
    // ------------------------------------------------------------------ softmax: one thread per stacked row
    const int g = (warp - 4) >> 2;                // row tile of this warpgroup
    const int quarter = warp & 3;                 // the TMEM lanes this warp may read
    const int lrow = quarter * 32 + lane;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_addr = lane_addr + CT_S_COL, p_addr = lane_addr + CT_P_COL + g * 64, o_addr = lane_addr + g * 128;
    const float scale = a.scale_log2;
    const uint64_t scale2 = f2_pack(scale, scale);
    int sc = 0;                                   // key tiles so far
    CaJob j;
    for (int jc = 0; take(jc, j); ++jc) {
      const int i = j.rt * TileWork::ROWS + g * 128 + lrow, i_lo = i - lane;
      if (i_lo - quarter * 32 >= j.R) continue;   // no such row tile
      const int n_act = g ? j.n_act[1] : j.n_act[0];
      const bool live = i_lo < j.R;               // the warp has rows
      const int qt = i / a.rep;
      const int adm = i < j.R ? ca_admitted(j, qt) : 0, adm_lo = live ? ca_admitted(j, i_lo / a.rep) : 0;
      const int entry = i < j.R ? (j.q0 + qt) * a.H + j.head * a.rep + (i - qt * a.rep) : -1;
      // p = 2^(x * scale - ref).  The reference is the maximum of the row's first key tile and then stays: one below the running
      // maximum only scales the sums.  Should a tile's sum outgrow the limit in some row of the warp, that tile is done again with the
      // row's true maximum as the new reference (O and the sum so far are rescaled).
      float neg_ref = 0.f, l_run = 0.f;
      bool unset = true;                          // no logit above -inf so far
      for (int t = 0; t < n_act; ++t, ++sc) {
        const int j0 = (j.kt0 + t) * 128;
        mbar_wait_warp(smem_u32(&bk->s_full[g]), sc & 1, wc);    // (no lane may still wait for a phase when lane 0 has arrived for it)
        tc_fence_after();
        if (!live) {                              // (one arrival per phase: the previous P V comes first here too)
          mbar_arrive_lane0(smem_u32(&bk->s_empty), lane);
          if (t > 0) mbar_wait_warp(smem_u32(&bk->pv_done[g]), (sc - 1) & 1, wc);
          mbar_arrive_lane0(smem_u32(&bk->p_ready[g]), lane);
          continue;
        }
        uint32_t xr[128];
#pragma unroll
        for (int c = 0; c < 128; c += 32) tmem_ld32p(s_addr + c, xr + c);
        tmem_wait_ld();
        tc_fence_before();
        __syncwarp();
        mbar_arrive_lane0(smem_u32(&bk->s_empty), lane);
        if (j0 + 128 > adm_lo) {
          const int lim = adm - j0;
#pragma unroll
          for (int c = 0; c < 128; ++c)
            if (c >= lim) xr[c] = __float_as_uint(-INFINITY);
        }
        if constexpr (WEIGHTS) {
          if (entry >= 0) {
            float *row = a.logits + (long long)entry * a.pitch + (j.causal ? a.own_off : 0) + j0;
#pragma unroll
            for (int c = 0; c < 128; c += 8) {
              float v[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(xr[c + e]) * scale;
              asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                           ::"l"(row + c), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
            }
          }
          __syncwarp();
        }
        if (t > 0) {
          mbar_wait(smem_u32(&bk->pv_done[g]), (sc - 1) & 1, wc);      // O is complete up to here, and P may be overwritten
          tc_fence_after();
        }
        bool move = unset, moved = false, again = __any_sync(0xffffffffu, unset && j0 < adm);
        float tile_sum;
#pragma unroll 1
        while (true) {
          if (again) {
            float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};       // four independent chains
#pragma unroll
            for (int c = 0; c < 128; c += 8)
#pragma unroll
              for (int e = 0; e < 4; ++e) mx4[e] = max3(mx4[e], __uint_as_float(xr[c + e]), __uint_as_float(xr[c + 4 + e]));
            const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
            const float neg = mx == -INFINITY ? 0.f : -mx * scale;
            if (t > 0) {
              const float f = move && !unset ? fast_exp2(neg - neg_ref) : 1.0f;
#pragma unroll 1
              for (int c0 = 0; c0 < 128; c0 += 16) {
                uint32_t r[16];
                tmem_ld16(o_addr + c0, r);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * f);
                tmem_st16(o_addr + c0, r);
              }
              l_run *= f;
            }
            if (move) {
              moved = true;
              neg_ref = neg;
              if (mx != -INFINITY) unset = false;
            }
          }
          const uint64_t neg2 = f2_pack(neg_ref, neg_ref);
          uint64_t sum2[2] = {0ull, 0ull};          // even and odd keys apart, two chains
#pragma unroll
          for (int c0 = 0; c0 < 128; c0 += 32) {
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float p0, p1;
              f2_unpack(f2_fma(f2_pack(__uint_as_float(xr[c0 + 2 * e]), __uint_as_float(xr[c0 + 2 * e + 1])), scale2, neg2), p0, p1);
              p0 = fast_exp2(p0);
              p1 = fast_exp2(p1);
              sum2[e & 1] = f2_add(sum2[e & 1], f2_pack(p0, p1));
              w[e] = pack2_t<F16>(p0, p1);
            }
            tmem_st16(p_addr + (c0 >> 1), w);
          }
          float s0, s1;
          f2_unpack(f2_add(sum2[0], sum2[1]), s0, s1);
          tile_sum = s0 + s1;
          move = i < j.R && !moved && !(tile_sum < (F16 ? CT_SUM_LIMIT_F16 : CT_SUM_LIMIT_BF16));     // (relative to the true maximum no sum exceeds 128)
          if (!__any_sync(0xffffffffu, move)) break;
          again = true;
        }
        l_run += tile_sum;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        mbar_arrive_lane0(smem_u32(&bk->p_ready[g]), lane);
      }
      // ---- the item's part of the rows
      if (n_act > 0) {
        mbar_wait_warp(smem_u32(&bk->pv_done[g]), (sc - 1) & 1, wc);
        tc_fence_after();
      }
      if (!live) continue;
      // NaN in every logit leaves no maximum, but the row is not an empty one
      const bool none = n_act == 0 || (unset && l_run == 0.f), complete = j.complete != 0;
      const int at = entry < 0 ? -1 : complete ? (j.causal ? a.n_q * a.H : 0) + entry : j.record * TileWork::ROWS + g * 128 + lrow;
      const bool write = !bk->abort_flag;
      if (at >= 0 && write) (complete ? a.full_ml : a.rec_ml[1])[at] = none ? make_float2(-INFINITY, 0.f) : make_float2(-neg_ref, l_run);
      if (n_act == 0) continue;
      float *dst = complete ? a.full_o : a.rec_o[1];
      const bool bad = *reinterpret_cast<volatile int *>(&bk->bad[jc % (2 * CT_JOBS)]) != 0;
      // (A thread stores its own row, 32 bytes at a time: whole sectors.)
#pragma unroll 1
      for (int c0 = 0; c0 < 128; c0 += 32) {
        uint32_t r[32];
        tmem_ld32(o_addr + c0, r);
        tmem_wait_ld();
        if (bad) {                                  // what warp 2 left out
          const int from = max(j.kt0 * 128, ca_admitted(j, j.causal ? j.rt * TileWork::ROWS / a.rep : 0)), to = min((j.kt0 + j.n) * 128, adm);
          for (int key = from; key < to; ++key) {
            const uint16_t *v = a.v + (long long)(j.row0 + key) * a.kv_row + (long long)j.head * a.kv_head + c0;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              uint32_t w;
              asm volatile("ld.global.u32 %0, [%1];" : "=r"(w) : "l"(v + 2 * e));
              const float2 x = unpack2_t<F16>(w);
              if (!isfinite(x.x)) r[2 * e] = __float_as_uint(__uint_as_float(r[2 * e]) + x.x);
              if (!isfinite(x.y)) r[2 * e + 1] = __float_as_uint(__uint_as_float(r[2 * e + 1]) + x.y);
            }
          }
          __syncwarp();
        }
        if (at >= 0 && write) {
#pragma unroll
          for (int c = 0; c < 32; c += 8)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                         ::"l"(dst + (long long)at * 128 + c0 + c), "r"(r[c]), "r"(r[c + 1]), "r"(r[c + 2]), "r"(r[c + 3]), "r"(r[c + 4]), "r"(r[c + 5]),
                           "r"(r[c + 6]), "r"(r[c + 7])
                         : "memory");
        }
        __syncwarp();
      }
      tc_fence_before();                            // the next item's first P (and so its first P V) comes after these loads
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, CT_TMEM_COLS);
  }
}

// ---------------------------------------------------------------------------------------
// Partial results of a (query row, head) -> output, four of the 128 values a lane.  A thread works out where the partial results of one (head,
// prefix or own rows) lie.  (With the addresses worked out by every warp for itself the kernel was bound by those instructions: 2254
// rows x 32 heads 67 us.)  Many rows: a block takes 32 heads of four, a warp two at a time, small blocks that hide each other's beginnings (2254
// rows x 32 heads: 41 us with a row and 512 threads a block, 35 with four rows, 33 with four rows and 256 threads,
// of which the whole call shows nothing, 193 and 194).  With fewer rows it takes
// 16, 8 or 2 heads, and one, two or eight warps share the partial results of a head, eight of which are under way together; a long sequence has a
// hundred or more.
// ---------------------------------------------------------------------------------------
constexpr int CA_JOIN_THREADS = 512, CA_JOIN_WARPS = CA_JOIN_THREADS / 32;
constexpr int CA_JOIN_HEADS = 32, CA_JOIN_MANY_THREADS = 256;

__device__ __forceinline__ float2 ld_prev2f(const float2 *p) {
  float2 v;
  asm volatile("ld.global.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ float4 ld_prev4f(const float *p) {
  float4 v;
  asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p));
  return v;
}

struct CaSum {
  float top = -INFINITY, sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  __device__ __forceinline__ void add(float2 ml, float4 o) {
    if (ml.x == -INFINITY) return;
    const float t = fmaxf(top, ml.x), f = top == -INFINITY ? 0.f : fast_exp2(top - t), g = fast_exp2(ml.x - t);
    sum = sum * f + ml.y * g;
    acc.x = acc.x * f + o.x * g; acc.y = acc.y * f + o.y * g; acc.z = acc.z * f + o.z * g; acc.w = acc.w * f + o.w * g;
    top = t;
  }
};
// The partial results of one part of a (query row, head): the first at entry `first` of `ml` and `o`, the others every `step` entries from
// `next` on, `n` in all.
struct CaParts {
  const float2 *ml;
  const float *o;
  long long first, next;
  int step, n;
  int pad[2];
  __device__ __forceinline__ long long at(int k) const { return k == 0 ? first : next + (long long)(k - 1) * step; }
};
template <typename WORK>
__device__ __forceinline__ CaParts ca_parts_of(const CacheArgs &a, const CaRowPart &p, int which, int all, long long entry, int kvh, int sub) {
  CaParts out;
  const int hg = ca_together<WORK>(p.R, a.kv, p.keys), i = p.i0 + sub, rt = i / WORK::ROWS;
  const int r = i - rt * WORK::ROWS + (hg > 1 ? (kvh & (hg - 1)) * p.R : 0);
  const int kt = ca_key_tiles<WORK>(p.R, p.keys, p.adm0, p.causal, a.rep, hg, rt);
  const int chunk = ca_chunk(all, a.pieces[WORK::INDEX]), rec_rows = WORK::INDEX == 0 ? a.rec_rows : WORK::ROWS;
  const int first = p.off + kvh / hg * p.per_head + ca_numbers<WORK>(p.R, p.keys, p.adm0, p.causal, a.rep, hg, rt) + WORK::EXTRA;
  const int c0 = first / chunk, c1 = (first + kt - 1) / chunk;
  const bool complete = c0 == c1;
  out.n = kt == 0 ? 0 : c1 - c0 + 1;
  out.step = 2 * rec_rows;
  out.ml = complete ? a.full_ml : a.rec_ml[WORK::INDEX];
  out.o = complete ? a.full_o : a.rec_o[WORK::INDEX];
  out.first = complete ? (long long)which * a.n_q * a.H + entry : (long long)(2 * c0 + (first <= c0 * chunk ? 0 : 1)) * rec_rows + r;
  out.next = (long long)(2 * c0 + 2) * rec_rows + r;
  return out;
}

template <bool F16>
__device__ __forceinline__ void ca_finish_row(const CacheArgs &a, const CaSum &s, int qr, int h, int lane) {
  const long long entry = (long long)qr * a.H + h;
  const float inv = s.sum > 0.f ? 1.f / s.sum : (s.sum == 0.f ? 0.f : s.sum);    // (NaN stays NaN)
  uint16_t *dst = a.out + (long long)qr * a.out_row + (long long)h * a.out_head + lane * 4;
  *reinterpret_cast<uint2 *>(dst) = make_uint2(pack2_t<F16>(s.acc.x * inv, s.acc.y * inv), pack2_t<F16>(s.acc.z * inv, s.acc.w * inv));
  if (lane == 0) {
    const float l2 = s.top + __log2f(s.sum);
    if (a.lse) a.lse[entry] = s.sum == 0.f ? -INFINITY : l2 * 0.6931471805599453f;
    a.lse2[entry] = s.sum == 0.f ? INFINITY : l2;
  }
}

template <bool F16, int HEADS, int ROWS>
__global__ void __launch_bounds__(ROWS > 1 ? CA_JOIN_MANY_THREADS : CA_JOIN_THREADS, ROWS > 1 ? 4 : 2)
ca_join_kernel(const __grid_constant__ CacheArgs a) {
  constexpr int THREADS = ROWS > 1 ? CA_JOIN_MANY_THREADS : CA_JOIN_THREADS, WARPS = THREADS / 32;
  constexpr int SHARE = WARPS / HEADS;           // warps that share a head
  constexpr bool SPLIT = ROWS == 1 && SHARE >= 1;
  __shared__ CaParts sh_parts[ROWS * HEADS][2];
  __shared__ int sh_valid[ROWS];
  __shared__ float4 sh_acc[SPLIT ? CA_JOIN_WARPS : 1][32];
  __shared__ float2 sh_ml[SPLIT ? CA_JOIN_WARPS : 1];
  // Behind the weights' kernel: its blocks have all waited for the partial results before this kernel can start, and nothing of its own is
  // needed.  The wait for its end comes last.
  if (a.join_behind) pdl_after();
  else pdl_enter();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n_seg = a.G + a.B, h0 = blockIdx.y * HEADS;
  // every query row of [q_cu[0], q_cu[B]) has an entry of this call unless the call is skipped
  const uint32_t status = *reinterpret_cast<volatile uint32_t *>(a.status);
  const int q0 = a.q_cu ? ld_prev(a.q_cu) : 0, q1 = a.q_cu ? ld_prev(a.q_cu + a.B) : a.n_q, going = ld_prev(a.plan + 2 * (n_seg + 1));
  static_assert(ROWS * HEADS * 2 <= THREADS, "a thread per (query row, head, part)");
  if (threadIdx.x < ROWS * HEADS * 2) {
    const int qr = blockIdx.x * ROWS + threadIdx.x / (2 * HEADS), h = h0 + (threadIdx.x >> 1) % HEADS, p = threadIdx.x & 1;
    CaParts mine;
    mine.n = 0;
    int valid = -1;                              // not this call's row
    if (qr < a.n_q) {
      const CaRowPart *src = &a.rows[qr].part[p];
      const int entry_valid = ld_prev(&a.rows[qr].valid);
      CaRowPart part;
      part.i0 = ld_prev(&src->i0); part.R = ld_prev(&src->R); part.adm0 = ld_prev(&src->adm0); part.causal = ld_prev(&src->causal);
      part.keys = ld_prev(&src->keys); part.off = ld_prev(&src->off); part.per_head = ld_prev(&src->per_head);
      const int all0 = ld_prev(a.plan + n_seg), all1 = a.pieces[1] ? ld_prev(a.plan + 2 * n_seg + 1) : 0;
      if (going && qr >= q0 && qr < q1 && !(status & STATUS_CACHE_TIMEOUT)) {
        valid = entry_valid;
        if (h < a.H && valid == 1 && part.R > 0) {
          const int kvh = h / a.rep, sub = h - kvh * a.rep;
          const long long entry = (long long)qr * a.H + h;
          mine = ca_streamed(part.R) ? ca_parts_of<StreamWork>(a, part, p, all0, entry, kvh, sub) : ca_parts_of<TileWork>(a, part, p, all1, entry, kvh, sub);
        }
      }
    }
    sh_parts[threadIdx.x >> 1][p] = mine;
    if (threadIdx.x % (2 * HEADS) == 0) sh_valid[threadIdx.x / (2 * HEADS)] = valid;
  }
  __syncthreads();
  // a row of a sequence that is skipped adds no weight
  if (threadIdx.x < ROWS * HEADS) {
    const int r = threadIdx.x / HEADS, h = h0 + threadIdx.x % HEADS;
    if (sh_valid[r] == 0 && h < a.H) a.lse2[(long long)(blockIdx.x * ROWS + r) * a.H + h] = INFINITY;
  }
  if constexpr (SPLIT) {
    const int e = warp / SHARE, w = warp - e * SHARE;
    CaSum s;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const CaParts &c = sh_parts[e][p];
      for (int k0 = w; k0 < c.n; k0 += 8 * SHARE) {
        float2 m8[8];
        float4 o8[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const long long at = c.at(min(k0 + k * SHARE, c.n - 1));
          m8[k] = ld_prev2f(c.ml + at);
          o8[k] = ld_prev4f(c.o + at * 128 + lane * 4);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k0 + k * SHARE < c.n) s.add(m8[k], o8[k]);
      }
    }
    sh_acc[warp][lane] = s.acc;
    if (lane == 0) sh_ml[warp] = make_float2(s.top, s.sum);
    __syncthreads();
    if (w == 0 && h0 + e < a.H && sh_valid[0] == 1) {
      for (int k = 1; k < SHARE; ++k) s.add(sh_ml[warp + k], sh_acc[warp + k][lane]);
      ca_finish_row<F16>(a, s, blockIdx.x, h0 + e, lane);
    }
  } else {
    constexpr int MINE = 2;                      // (query row, head) pairs of a warp whose first loads are under way together
#pragma unroll 1
    for (int e0 = warp * MINE; e0 < ROWS * HEADS; e0 += WARPS * MINE) {
      float2 ml[MINE][2];
      float4 o[MINE][2];
#pragma unroll
      for (int x = 0; x < MINE; ++x)
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const CaParts &c = sh_parts[e0 + x][p];
          if (c.n == 0) continue;
          ml[x][p] = ld_prev2f(c.ml + c.first);
          o[x][p] = ld_prev4f(c.o + c.first * 128 + lane * 4);
        }
#pragma unroll
      for (int x = 0; x < MINE; ++x) {
        const int e = e0 + x, r = e / HEADS, h = h0 + e % HEADS;
        if (h >= a.H || sh_valid[r] != 1) continue;
        CaSum s;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const CaParts &c = sh_parts[e][p];
          if (c.n == 0) continue;
          s.add(ml[x][p], o[x][p]);
          for (int k0 = 1; k0 < c.n; k0 += 4) {
            float2 m4[4];
            float4 o4[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const long long at = c.at(min(k0 + k, c.n - 1));
              m4[k] = ld_prev2f(c.ml + at);
              o4[k] = ld_prev4f(c.o + at * 128 + lane * 4);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (k0 + k < c.n) s.add(m4[k], o4[k]);
          }
        }
        ca_finish_row<F16>(a, s, blockIdx.x * ROWS + r, h, lane);
      }
    }
  }
  if (a.join_behind) pdl_wait();
}

// ---------------------------------------------------------------------------------------
// weights[j] += 1 / H * sum over the segment's query rows and heads of 2^(x - lse2).  A thread takes four keys; `lanes` threads side by side
// on the keys, the others below them share the (row, head) pairs, and their sums are added in order.  Few pairs (own rows of single
// tokens): 64 threads on 256 keys, 8 pairs a thread under way together; many: 16 on 64 keys; more than 512: 4 on 16 keys.  (64 x 870 keys, 32
// pairs: 9 us against 24 with 64 keys a block; a prefix with 320 pairs and 2000 keys is the other way round.)
// ---------------------------------------------------------------------------------------
constexpr int CA_WEIGHT_THREADS = 256;

__global__ void __launch_bounds__(CA_WEIGHT_THREADS)
ca_weight_kernel(const __grid_constant__ CacheArgs a, int prefix_blocks, int prefix_lanes, int own_blocks, int own_lanes) {
  __shared__ float4 part[CA_WEIGHT_THREADS];
  pdl_enter();
  const int n_pre = a.G * prefix_blocks;         // (no blocks for rows that the bounds rule out: then no block divides by that number either)
  const int s = (int)blockIdx.x < n_pre ? blockIdx.x / prefix_blocks : a.G + (blockIdx.x - n_pre) / own_blocks;
  const int kb = (int)blockIdx.x < n_pre ? blockIdx.x % prefix_blocks : (blockIdx.x - n_pre) % own_blocks;
  const uint32_t status = *reinterpret_cast<volatile uint32_t *>(a.status);
  const int going = ld_prev(a.plan + 2 * (a.G + a.B + 1));
  bool broken;
  const CaSeg g = ca_segment(a, s, broken);
  const int lanes = s < a.G ? prefix_lanes : own_lanes, shares = CA_WEIGHT_THREADS / lanes, k0 = kb * lanes * 4;
  if (k0 >= g.keys || going == 0 || (status & STATUS_CACHE_TIMEOUT)) return;
  const int share = threadIdx.x / lanes, j = k0 + (threadIdx.x - share * lanes) * 4;
  const int n = g.nq * a.H, adm0 = g.keys - g.nq + 1, causal = s >= a.G;
  const float *x = a.logits + (long long)g.q0 * a.H * a.pitch + (causal ? a.own_off : 0) + j;
  const float *lse2 = a.lse2 + (long long)g.q0 * a.H;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  for (int e0 = share; e0 < n; e0 += 8 * shares) {
    float l2[8];
    float4 v[8];
    int lim[8];                                  // keys of the thread's four that the row admits
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int e = e0 + k * shares;
      lim[k] = e < n ? ca_admitted(g.keys, adm0, causal, causal ? e / a.H : 0) - j : 0;
      l2[k] = e < n ? ld_prev(lse2 + e) : INFINITY;
      v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (lim[k] > 0) v[k] = ld_prev4f(x + e * a.pitch);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
      for (int c = 0; c < 4; ++c) sum[c] += c < lim[k] && l2[k] != INFINITY ? fast_exp2(w[c] - l2[k]) : 0.f;
    }
  }
  part[threadIdx.x] = make_float4(sum[0], sum[1], sum[2], sum[3]);
  __syncthreads();
  const int key = k0 + (int)threadIdx.x;
  if ((int)threadIdx.x < lanes * 4 && key < g.keys) {
    float t = 0.f;
#pragma unroll 4
    for (int w = 0; w < shares; ++w) t += reinterpret_cast<const float *>(part + w * lanes)[threadIdx.x];
    float *p = a.weights + g.row0 + key;
    *p = ld_prev(p) + t / (float)a.H;
  }
}

// The same for batches without prefixes whose sequences have at most 64 (row, head) pairs each: a block works out ln of their sums itself, from the
// partial results, and so need not wait for the join, which runs beside it (1 x 267 keys: the call 15.7 -> 12.5 us).
constexpr int CA_FEW_PAIRS = 64, CA_FEW_LANES = 64;

__global__ void __launch_bounds__(CA_WEIGHT_THREADS)
ca_weight_few_kernel(const __grid_constant__ CacheArgs a, int own_blocks) {
  constexpr int SHARES = CA_WEIGHT_THREADS / CA_FEW_LANES, MINE = CA_FEW_PAIRS / SHARES;
  __shared__ float4 part[CA_WEIGHT_THREADS];
  __shared__ float sh_lse2[CA_FEW_PAIRS];
  pdl_enter();
  const int b = blockIdx.x / own_blocks, k0 = (blockIdx.x - b * own_blocks) * CA_FEW_LANES * 4, n_seg = a.B;
  const uint32_t status = *reinterpret_cast<volatile uint32_t *>(a.status);
  const int going = ld_prev(a.plan + 2 * (n_seg + 1)), all0 = ld_prev(a.plan + n_seg), all1 = a.pieces[1] ? ld_prev(a.plan + 2 * n_seg + 1) : 0;
  bool broken;
  const CaSeg g = ca_segment(a, b, broken);
  if (k0 >= g.keys || going == 0 || (status & STATUS_CACHE_TIMEOUT)) return;
  const int n = g.nq * a.H, adm0 = g.keys - g.nq + 1;        // n <= CA_FEW_PAIRS: the caller's bound on the query rows holds
  const int share = threadIdx.x / CA_FEW_LANES, j = k0 + (threadIdx.x - share * CA_FEW_LANES) * 4;
  const float *x = a.logits + (long long)g.q0 * a.H * a.pitch + a.own_off + j;
  float4 v[MINE];
  int lim[MINE];                                 // keys of the thread's four that the row admits
#pragma unroll
  for (int k = 0; k < MINE; ++k) {
    const int e = share + k * SHARES;
    lim[k] = e < n ? ca_admitted(g.keys, adm0, 1, e / a.H) - j : 0;
    v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (lim[k] > 0) v[k] = ld_prev4f(x + e * a.pitch);
  }
  {
    // four threads a pair
    const int e = threadIdx.x >> 2, sub = threadIdx.x & 3;
    float top = -INFINITY, sum = 0.f;
    if (e < n) {
      const int t = e / a.H, h = e - t * a.H, kvh = h / a.rep;
      const CaRowPart *src = &a.rows[g.q0 + t].part[1];
      CaRowPart p;
      p.i0 = ld_prev(&src->i0); p.R = ld_prev(&src->R); p.adm0 = ld_prev(&src->adm0); p.causal = ld_prev(&src->causal);
      p.keys = ld_prev(&src->keys); p.off = ld_prev(&src->off); p.per_head = ld_prev(&src->per_head);
      const long long entry = (long long)(g.q0 + t) * a.H + h;
      const CaParts c = ca_streamed(p.R) ? ca_parts_of<StreamWork>(a, p, 1, all0, entry, kvh, h - kvh * a.rep) : ca_parts_of<TileWork>(a, p, 1, all1, entry, kvh, h - kvh * a.rep);
      for (int r0 = sub; r0 < c.n; r0 += 16) {
        float2 ml[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) ml[r] = r0 + 4 * r < c.n ? ld_prev2f(c.ml + c.at(r0 + 4 * r)) : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float f, q;
          ca_merge(top, sum, ml[r], f, q);
        }
      }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      const float2 other = make_float2(__shfl_xor_sync(0xffffffffu, top, o), __shfl_xor_sync(0xffffffffu, sum, o));
      float f, q;
      ca_merge(top, sum, other, f, q);
    }
    if (sub == 0) sh_lse2[e] = sum == 0.f ? INFINITY : top + __log2f(sum);       // (+inf: adds nothing)
  }
  __syncthreads();
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < MINE; ++k) {
    const float l2 = sh_lse2[share + k * SHARES], w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
    for (int c = 0; c < 4; ++c) sum[c] += c < lim[k] && l2 != INFINITY ? fast_exp2(w[c] - l2) : 0.f;
  }
  part[threadIdx.x] = make_float4(sum[0], sum[1], sum[2], sum[3]);
  __syncthreads();
  const int key = k0 + (int)threadIdx.x;
  if (key < g.keys) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < SHARES; ++w) t += reinterpret_cast<const float *>(part + w * CA_FEW_LANES)[threadIdx.x];
    float *p = a.weights + g.row0 + key;
    *p = ld_prev(p) + t / (float)a.H;
  }
}

// =======================================================================================
// Eviction
// =======================================================================================
constexpr int EV_THREADS = 1024;
constexpr int EV_CLUSTER = 8;                    // blocks that share a long sequence
// Rows from which they do, if the device takes all sequences' clusters at once, or per round of them if it does not.  (One block: 7.4 us for 2048
// rows, 12.5 for 8192, 32 for 32768, for 64 sequences as for one.  Clusters: 11 to 14 us for up to 8 sequences, 22 to 29 for 19, 53 to 70
// for 64.)
constexpr int EV_CLUSTER_MIN = 6144, EV_CLUSTER_MIN_ROUND = 12288;
constexpr int EV_KEYS_BYTES = 192 * 1024;        // a block's keys in shared memory, if its rows fit

struct EvictArgs {
  int B, max_len, keep, sink, recent, rows, dst_rows;
  int cached;                                    // rows of a block whose keys it keeps in shared memory; 0: taken again in every pass
  const int *start, *len, *dst_start;
  const float *weights;
  const int *pos;
  int *keep_idx, *new_len;
  uint32_t *status;
};

// A float's order as an unsigned number: -inf .. +inf ascending from 1 up, -0 as +0, NaN 0.
__device__ __forceinline__ uint32_t rank_key(float w) {
  if (!(w == w)) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);           // -0 + 0 = +0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
// ... with the held rows above everything (no float's order is 2^32 - 1)
__device__ __forceinline__ uint32_t row_key(float w, int row, int pos, int sink, int recent, long long newest) {
  return row < sink || (long long)pos > newest - recent ? 0xffffffffu : rank_key(w);
}

// The keep-th largest key by radix selection, eight bits a pass, then every warp writes the kept rows of a range.  A block per sequence, or
// for long ones a cluster of eight that share its rows and add their histograms through each other's shared memory.  A row's weight and
// position are read once, its key stays in shared memory.  (One block that read both again in each of its seven passes: 2 x 30001 to
// 60001 rows, 4096 kept 119 us.)
template <bool CLUSTER>
__global__ void __launch_bounds__(EV_THREADS)
evict_select_kernel(const __grid_constant__ EvictArgs a) {
  extern __shared__ uint32_t ev_keys[];
  __shared__ int hist[2][256];
  __shared__ int warp_gt[32], warp_eq[32];
  __shared__ int sh_pub[4];                      // what the other blocks of the cluster read: largest position, rows above and at the threshold
  __shared__ uint32_t sh_prefix;
  __shared__ int sh_need;
  pdl_enter();
  constexpr int PARTS = CLUSTER ? EV_CLUSTER : 1;
  const int b = blockIdx.y, part = CLUSTER ? (int)cluster_cta_rank() : 0, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto meet = [&]() {
    if constexpr (CLUSTER) cluster_sync_all();
    else __syncthreads();
  };
  auto theirs = [&](const int *p, int rank) {    // the word at p of block `rank`
    if constexpr (CLUSTER) return ld_cluster_s32(cluster_map(smem_u32(p), (uint32_t)rank));
    else return *reinterpret_cast<const volatile int *>(p);
  };
  const int n = ld_prev(a.len + b), row0 = ld_prev(a.start + b), dst0 = a.dst_start ? ld_prev(a.dst_start + b) : row0;
  int *idx = a.keep_idx + (size_t)b * a.keep;
  const int m = min(n, a.keep);
  // (all blocks of a cluster see the same sequence: they leave together)
  if (n < 0 || n > a.max_len || row0 < 0 || (long long)row0 + n > a.rows || dst0 < 0 || (long long)dst0 + m > a.dst_rows) {
    for (int i = part * EV_THREADS + tid; i < a.keep; i += PARTS * EV_THREADS) idx[i] = -1;
    if (tid == 0 && part == 0) atomicOr(a.status, (uint32_t)STATUS_BAD_SAMPLE);
    return;
  }
  for (int i = m + part * EV_THREADS + tid; i < a.keep; i += PARTS * EV_THREADS) idx[i] = -1;
  if (n <= a.keep) {
    for (int i = part * EV_THREADS + tid; i < n; i += PARTS * EV_THREADS) idx[i] = i;
    meet();                                      // (every block has read the length, which may be new_len itself)
    if (tid == 0 && part == 0) a.new_len[b] = m;
    return;
  }
  const float *w = a.weights + row0;
  const int *pos = a.pos ? a.pos + row0 : nullptr;
  const int share = ((n + PARTS - 1) / PARTS + 31) & ~31, first = min(n, part * share), last = min(n, first + share), mine = last - first;
  const bool cached = mine <= a.cached;
  // ---- the largest position; positions wait in the keys' place
  long long newest = n - 1;
  if (pos) {
    int top = INT_MIN;
#pragma unroll 4
    for (int i = tid; i < mine; i += EV_THREADS) {
      const int p = ld_prev(pos + first + i);
      if (cached) ev_keys[i] = (uint32_t)p;
      top = max(top, p);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) warp_gt[warp] = top;
    __syncthreads();
    if (warp == 0) {
      top = __reduce_max_sync(0xffffffffu, warp_gt[lane]);
      if (lane == 0) sh_pub[0] = top;
    }
    meet();
    top = INT_MIN;
#pragma unroll
    for (int r = 0; r < PARTS; ++r) top = max(top, theirs(&sh_pub[0], r));
    newest = top;
  }
  auto fresh = [&](int i) {                      // key of this block's row i from memory
    return row_key(ld_prev(w + first + i), first + i, pos ? ld_prev(pos + first + i) : first + i, a.sink, a.recent, newest);
  };
  auto key = [&](int i) { return cached ? ev_keys[i] : fresh(i); };
  uint32_t prefix = 0u;
  int need = a.keep;                             // rows still to be taken among those that share the prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    int *h = hist[(shift >> 3) & 1];             // (the other one may still be read by other blocks)
    if (tid < 256) h[tid] = 0;
    __syncthreads();
    if (shift == 24) {
#pragma unroll 4
      for (int i = tid; i < mine; i += EV_THREADS) {
        uint32_t k;
        if (cached) {
          k = row_key(ld_prev(w + first + i), first + i, pos ? (int)ev_keys[i] : first + i, a.sink, a.recent, newest);
          ev_keys[i] = k;
        } else {
          k = fresh(i);
        }
        atomicAdd(&h[k >> 24], 1);
      }
    } else {
      for (int i = tid; i < mine; i += EV_THREADS) {
        const uint32_t k = key(i);
        if ((k >> (shift + 8)) == prefix) atomicAdd(&h[(k >> shift) & 255u], 1);
      }
    }
    meet();
    if (warp < 8) {                              // all blocks' counts, thread t has bin 255 - t
      int c = 0;
#pragma unroll
      for (int r = 0; r < PARTS; ++r) c += theirs(&h[255 - tid], r);
      int above = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, above, o);
        if (lane >= o) above += v;
      }
      if (lane == 31) warp_eq[warp] = above;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      for (int v = 0; v < warp; ++v) above += warp_eq[v];
      if (above >= need && above - c < need) {
        sh_prefix = (prefix << 8) | (uint32_t)(255 - tid);
        sh_need = need - (above - c);
      }
    }
    __syncthreads();
    prefix = sh_prefix;
    need = sh_need;
  }
  // ---- rows above the threshold, and the first `need` equal to it; a warp's rows lie side by side
  const int per = ((mine + 1023) / 1024) * 32, lo = min(mine, warp * per), hi = min(mine, lo + per);
  int gt = 0, eq = 0;
  for (int i = lo + lane; i < hi; i += 32) {
    const uint32_t k = key(i);
    gt += k > prefix;
    eq += k == prefix;
  }
  gt = __reduce_add_sync(0xffffffffu, gt);
  eq = __reduce_add_sync(0xffffffffu, eq);
  if (lane == 0) { warp_gt[warp] = gt; warp_eq[warp] = eq; }
  __syncthreads();
  if (warp == 0) {
    const int g = __reduce_add_sync(0xffffffffu, warp_gt[lane]), e = __reduce_add_sync(0xffffffffu, warp_eq[lane]);
    if (lane == 0) { sh_pub[1] = g; sh_pub[2] = e; }
  }
  meet();
  int gt0 = 0, eq0 = 0;
  for (int r = 0; r < part; ++r) { gt0 += theirs(&sh_pub[1], r); eq0 += theirs(&sh_pub[2], r); }
  for (int v = 0; v < warp; ++v) { gt0 += warp_gt[v]; eq0 += warp_eq[v]; }
  int at = gt0 + min(eq0, need);
  for (int i0 = lo; i0 < hi; i0 += 32) {
    const int i = i0 + lane;
    const uint32_t k = i < hi ? key(i) : 0u;
    const uint32_t beq = __ballot_sync(0xffffffffu, i < hi && k == prefix);
    const bool take = i < hi && (k > prefix || (k == prefix && eq0 + __popc(beq & ((1u << lane) - 1u)) < need));
    const uint32_t bt = __ballot_sync(0xffffffffu, take);
    if (take) idx[at + __popc(bt & ((1u << lane) - 1u))] = first + i;
    at += __popc(bt);
    eq0 += __popc(beq);
  }
  if (tid == 0 && part == 0) a.new_len[b] = m;
  if constexpr (CLUSTER) cluster_sync_all();     // nobody's shared memory goes while it may be read
}

constexpr int EV_MAX_TENSORS = 64;
constexpr int EV_MOVE_THREADS = 256;
struct EvictMoveArgs {
  const uint4 *src[EV_MAX_TENSORS];
  uint4 *dst[EV_MAX_TENSORS];
  const int *keep_idx, *start, *dst_start;
  int n_tensors, keep, row_vecs, warp_rows;
  int in_order;                                  // weights or positions move in place
  const float *weights;
  const int *pos;
  float *dst_weights;
  int *dst_pos;
};

// Weights and positions of a sequence, a piece at a time: it is read before it is written, and no later piece has its source where an earlier
// one went.
__device__ __forceinline__ void evict_meta_in_order(const EvictMoveArgs &a, int b, int row0, int dst0) {
  const int *idx = a.keep_idx + (size_t)b * a.keep;
  for (int i0 = 0; i0 < a.keep; i0 += EV_MOVE_THREADS) {
    const int i = i0 + threadIdx.x, k = i < a.keep ? ld_prev(idx + i) : -1;
    float w = 0.f;
    int p = 0;
    if (k >= 0 && a.dst_weights) w = ld_prev(a.weights + row0 + k);
    if (k >= 0 && a.dst_pos) p = a.pos ? ld_prev(a.pos + row0 + k) : k;
    const bool end = __syncthreads_or(k < 0);
    if (k >= 0 && a.dst_weights) a.dst_weights[dst0 + i] = w;
    if (k >= 0 && a.dst_pos) a.dst_pos[dst0 + i] = p;
    if (end) break;
  }
}

// Into other tensors: a warp takes as many kept rows as make up 4 KB, or one long one, eight loads of a lane under way together (19
// sequences, 1875 rows of 1 KB kept: the whole call 54 -> 50 us against a row per warp).  What bounds it is the memory: 24 x 640 rows of 8 KB,
// keys and values, 87 us with the selection, 5.7 TB/s.  The last grid layer moves weights and positions, a thread per row.
__global__ void __launch_bounds__(EV_MOVE_THREADS)
evict_move_kernel(const __grid_constant__ EvictMoveArgs a) {
  pdl_enter();
  const int b = blockIdx.y, t = blockIdx.z, lane = threadIdx.x & 31;
  const int row0 = ld_prev(a.start + b), dst0 = a.dst_start ? ld_prev(a.dst_start + b) : row0;
  const int *idx = a.keep_idx + (size_t)b * a.keep;
  if (t == a.n_tensors) {
    if (a.in_order) {
      if (blockIdx.x == 0) evict_meta_in_order(a, b, row0, dst0);
      return;
    }
    const int i = blockIdx.x * EV_MOVE_THREADS + threadIdx.x, k = i < a.keep ? ld_prev(idx + i) : -1;
    if (k < 0) return;
    if (a.dst_weights) a.dst_weights[dst0 + i] = ld_prev(a.weights + row0 + k);
    if (a.dst_pos) a.dst_pos[dst0 + i] = a.pos ? ld_prev(a.pos + row0 + k) : k;
    return;
  }
  const int i0 = (blockIdx.x * (EV_MOVE_THREADS / 32) + (threadIdx.x >> 5)) * a.warp_rows;
  const int n = min(a.warp_rows, a.keep - i0) * a.row_vecs;      // vectors of this warp's rows
  for (int v0 = 0; v0 < n; v0 += 8 * 32) {
    uint4 x[8];
    long long to[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int f = v0 + 32 * e + lane, r = a.warp_rows == 1 ? 0 : f / a.row_vecs, v = f - r * a.row_vecs;
      to[e] = -1;
      if (f >= n) continue;
      const int k = ld_prev(idx + i0 + r);
      if (k < 0) continue;
      to[e] = (long long)(dst0 + i0 + r) * a.row_vecs + v;
      ld_prev8(a.src[t] + (size_t)(row0 + k) * a.row_vecs + v, x[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (to[e] >= 0) a.dst[t][to[e]] = x[e];
  }
}

// In place: a block per (sequence, tensor, 256 bytes of every row) takes the kept rows in ascending order, 128 at a time, and reads a piece
// before it writes it.  Row i of the kept ones goes to row i <= its own number, so no later piece reads what an earlier one wrote.  Weights
// and positions likewise, by one block of the last grid layer.
__global__ void __launch_bounds__(EV_MOVE_THREADS)
evict_in_place_kernel(const __grid_constant__ EvictMoveArgs a) {
  pdl_enter();
  const int b = blockIdx.y, t = blockIdx.z;
  const int *idx = a.keep_idx + (size_t)b * a.keep;
  const int row0 = ld_prev(a.start + b), dst0 = a.dst_start ? ld_prev(a.dst_start + b) : row0;
  if (t == a.n_tensors) {
    if (blockIdx.x == 0) evict_meta_in_order(a, b, row0, dst0);
    return;
  }
  const int v = blockIdx.x * 16 + (threadIdx.x & 15), r0 = threadIdx.x >> 4;
  uint4 *base = a.dst[t] + v;
  const bool in = v < a.row_vecs;
  for (int i0 = 0; i0 < a.keep; i0 += 128) {
    uint4 x[8];
    int k[8];
    bool end = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = i0 + r0 + 16 * e;
      k[e] = i < a.keep ? ld_prev(idx + i) : -1;
      end = end || k[e] < 0;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (in && k[e] > i0 + r0 + 16 * e) ld_prev8(base + (size_t)(row0 + k[e]) * a.row_vecs, x[e]);
    const bool done = __syncthreads_or(end);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = i0 + r0 + 16 * e;
      if (in && k[e] > i) base[(size_t)(row0 + i) * a.row_vecs] = x[e];
    }
    if (done) break;
  }
}

// The lowest ranked row of a full cache: smallest key, the last row among equals.  A block per sequence reads its weights and positions once; 64 x
// 1152 rows 3.7 us, the call's own cost and one round trip to the memory.
constexpr int SLOT_THREADS = 512;
struct SlotArgs {
  int B, capacity, sink, recent, rows;
  const int *start;
  int *len;
  float *weights;
  int *pos;
  const int *new_pos;
  int *row;
  uint32_t *status;
};
__global__ void __launch_bounds__(SLOT_THREADS)
slot_kernel(const __grid_constant__ SlotArgs a) {
  __shared__ unsigned long long part[SLOT_THREADS / 32];
  pdl_enter();
  const int b = blockIdx.x, tid = threadIdx.x;
  const int n = ld_prev(a.len + b), row0 = ld_prev(a.start + b), np = ld_prev(a.new_pos + b);
  __syncthreads();                               // (every thread has read the length, which the first one writes below)
  if (n < 0 || n > a.capacity || row0 < 0 || (long long)row0 + min(n + 1, a.capacity) > a.rows) {
    if (tid == 0) {
      a.row[b] = -1;
      atomicOr(a.status, (uint32_t)STATUS_BAD_SAMPLE);
    }
    return;
  }
  int slot = n;
  if (n == a.capacity) {
    unsigned long long best = ~0ull;
#pragma unroll 4
    for (int i = tid; i < n; i += SLOT_THREADS) {
      const uint32_t k = row_key(ld_prev(a.weights + row0 + i), i, ld_prev(a.pos + row0 + i), a.sink, a.recent, (long long)np - 1);
      best = min(best, ((unsigned long long)k << 32) | (0xffffffffu - (uint32_t)i));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, o));
    if ((tid & 31) == 0) part[tid >> 5] = best;
    __syncthreads();
    best = part[0];
    for (int w = 1; w < SLOT_THREADS / 32; ++w) best = min(best, part[w]);
    slot = (int)(0xffffffffu - (uint32_t)best);
  }
  if (tid == 0) {
    a.row[b] = row0 + slot;
    if (n < a.capacity) a.len[b] = n + 1;
    a.weights[row0 + slot] = 0.f;
    a.pos[row0 + slot] = np;
  }
}

}  // namespace asap
