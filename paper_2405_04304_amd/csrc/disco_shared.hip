// gfx950 (MI355X) kernels for several sequences that continue one prompt: keys and values appended to a paged cache with head
// norms and rotation on the way, attention that reads the prompt's pages once for all sequences, the beams' next tokens, and
// the reordering of their page tables.
#include "disco_device.h"
#include "disco_shared.h"

#include <climits>
#include <type_traits>

namespace disco {

namespace {

constexpr float LOG2E = 1.44269504088896f, LN2 = 0.693147180559945f;

__device__ __forceinline__ int page_of(const SharedKv& kv, int pos) { return kv.pt_shift >= 0 ? pos >> kv.pt_shift : pos / kv.pt; }

// What the wavefront's lanes have written to LDS is there for all of them (the unit works in order: this only holds the compiler).
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Four consecutive elements of a row as floats, and back.
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const bf16_t* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(bf16_t* p, float4 v) { *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)); }

// ---------------------------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------------------------
//
// y = rotate(norm(x)) for query and key heads, K to [token][channel] blocks, V to [channel][token] blocks, one pass.  Norm and rotation in fp32, one rounding
// to bf16 at the cache's entry (queries: to their own type).  Bytes only: 5999 rows of 3 x 40 heads of 128 in bf16, 372 MB, take 86 us, 4.3 TB/s; what is left to the
// copy's rate (73 us) is the tiles of V, whose loads end at a barrier before their stores begin.  Small calls are three dependent round trips (position,
// page, entry): 2.9 us for four rows, 6.4 us for 192.

// Where row i goes: its sequence's own position and the page that holds it; pos < 0: nowhere (padding, or outside the tables).
struct RowPlace { int seq, pos, page; };
__device__ __forceinline__ RowPlace row_place(const AppendArgs& a, int i) {
  RowPlace r{-1, -1, -1};
  if (i >= a.rows) return r;
  if (a.seq != nullptr) {
    r.seq = a.seq[i];
    r.pos = a.pos[i];
  } else {
    r.seq = i / a.n_tok;
    r.pos = a.kv.lens[r.seq] - a.n_tok + (i - r.seq * a.n_tok);
  }
  if ((unsigned)r.seq >= (unsigned)a.kv.n_seqs || r.pos < 0 || page_of(a.kv, r.pos) >= a.kv.table_ld) { r.seq = r.pos = -1; return r; }
  r.page = a.kv.tables[(size_t)r.seq * a.kv.table_ld + page_of(a.kv, r.pos)];
  if ((unsigned)r.page >= (unsigned)a.kv.n_pages) r.page = -1;
  return r;
}

// N (4 or 8) consecutive elements of a row as floats, and floats as elements of a row.
template <int N, typename T>
__device__ __forceinline__ void load_piece(const T* p, float (&v)[N]) {
  if constexpr (N == 8 && sizeof(T) == 2) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(x[i] << 16); v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u); }
  } else {
    static_assert(N == 4, "16 bytes at most");
    const float4 x = load4(p);
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
  }
}
template <int N, typename T>
__device__ __forceinline__ void store_piece(T* p, const float (&v)[N]) {
  if constexpr (N == 8) *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
  else store4(p, make_float4(v[0], v[1], v[2], v[3]));
}

// Queries and keys: y = rotate(norm(x)).  A lane holds N elements of a row's first half of a head and their rotary partners in the second; its
// (cos, sin) stay in registers over HB heads of the row, whose loads are on their way together.  In calls of few rows the values' heads
// come here as well, one entry at a time into their transposed blocks.
template <typename T, int HB> constexpr int append_piece = HB > 1 && sizeof(T) == 2 ? 8 : 4;      // (16 bytes; few rows take what gives more wavefronts)
template <int DH, typename T, int HB>
__device__ __forceinline__ void append_heads(const AppendArgs& a, const int row_block, const int h0) {
  constexpr int N = append_piece<T, HB>, LPR = DH / 2 / N, RPW = 256 / LPR;
  const SharedKv& kv = a.kv;
  const int i = row_block * RPW + threadIdx.x / LPR, c = threadIdx.x % LPR * N, heads = a.nq + (HB == 1 ? 2 : 1) * kv.nkv;
  float lo[HB][N], hi[HB][N];
  if (i < a.rows) {
    const T* x = static_cast<const T*>(a.qkv) + (size_t)i * a.ld + c;
#pragma unroll
    for (int u = 0; u < HB; ++u) {
      const int h = min(h0 + u, heads - 1);
      load_piece(x + h * DH, lo[u]);
      load_piece(x + h * DH + DH / 2, hi[u]);
    }
  }
  const RowPlace at = row_place(a, i);
  if (at.pos < 0) return;
  float cs[N], sn[N];
  if (a.rope != nullptr) {
    const float* t = a.rope + ((size_t)(kv.prefix_len + at.pos) * (DH / 2) + c) * 2;
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const float4 p = load4(t + 2 * e);
      cs[e] = p.x; sn[e] = p.y; cs[e + 1] = p.z; sn[e + 1] = p.w;
    }
  }
  const int off = at.pos - page_of(kv, at.pos) * kv.pt;
#pragma unroll
  for (int u = 0; u < HB; ++u) {
    const int h = h0 + u;
    if (h >= heads) break;
    if (HB == 1 && h >= a.nq + kv.nkv) {
      if (at.page < 0) break;
      bf16_t* v = kv.pages + ((size_t)at.page * 2 * kv.nkv + (h - a.nq)) * kv.pt * DH + (size_t)c * kv.pt + off;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        v[(size_t)e * kv.pt] = f32_to_bf16(lo[u][e]);
        v[(size_t)(DH / 2 + e) * kv.pt] = f32_to_bf16(hi[u][e]);
      }
      break;
    }
    const float* gain = h < a.nq ? a.q_gain : a.k_gain;
    if (gain != nullptr) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) ss += lo[u][e] * lo[u][e] + hi[u][e] * hi[u][e];
#pragma unroll
      for (int o = 1; o < LPR; o *= 2) ss += __shfl_xor(ss, o);
      const float r = 1.0f / sqrtf(ss * (1.0f / DH) + a.eps);
#pragma unroll
      for (int e = 0; e < N; ++e) { lo[u][e] *= r * gain[c + e]; hi[u][e] *= r * gain[DH / 2 + c + e]; }
    }
    if (a.rope != nullptr) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float x = lo[u][e], y = hi[u][e];
        lo[u][e] = x * cs[e] - y * sn[e];
        hi[u][e] = y * cs[e] + x * sn[e];
      }
    }
    if (h < a.nq) {
      T* q = static_cast<T*>(a.q) + (size_t)i * a.ld_q + (size_t)h * DH + c;
      store_piece(q, lo[u]);
      store_piece(q + DH / 2, hi[u]);
    } else if (at.page >= 0) {
      bf16_t* k = kv.pages + (((size_t)at.page * 2 * kv.nkv + (h - a.nq)) * kv.pt + off) * DH + c;
      store_piece(k, lo[u]);
      store_piece(k + DH / 2, hi[u]);
    }
  }
}

// Values of 64 rows of one head, into blocks [channel][position]: rows G of which are a run of consecutive positions that starts at a multiple of G
// are written G positions at a time (a run belongs to the workgroup of its first row, which reads up to G - 1 rows of the next), others alone.
constexpr int APPEND_RV = 64;        // rows of a workgroup
template <int DH> struct ValueTile {
  bf16_t v[APPEND_RV + 8][DH + 2];
  int seq[APPEND_RV + 16], pos[APPEND_RV + 16], page[APPEND_RV + 16];      // from 8 rows in front on
  unsigned char run[APPEND_RV + 8];                                        // a run starts here (from 8 rows in front on)
  int n_run, n_one;
  unsigned char runs[APPEND_RV], ones[APPEND_RV];                          // rows of this workgroup: first of a run, in none
};
template <int DH, typename T, int G>
__device__ __forceinline__ void append_values(const AppendArgs& a, const int row_block, const int head, ValueTile<DH>& s) {
  constexpr int rv = APPEND_RV, N = append_piece<T, 4>, LPR = DH / N;
  const SharedKv& kv = a.kv;
  const int r0 = row_block * rv, t = threadIdx.x;
  const T* x = static_cast<const T*>(a.qkv) + (size_t)(a.nq + kv.nkv + head) * DH;
  if (t < rv + 16) {
    const int i = r0 - 8 + t;
    const RowPlace p = i >= 0 ? row_place(a, i) : RowPlace{-1, -1, -1};
    s.seq[t] = p.seq; s.pos[t] = p.pos; s.page[t] = p.page;
  }
  if (t == 0) { s.n_run = 0; s.n_one = 0; }
  for (int i = t; i < (rv + G - 1) * LPR; i += 256) {
    const int r = i / LPR, c = i % LPR * N;
    if (r0 + r >= a.rows) break;
    float v[N];
    load_piece(x + (size_t)(r0 + r) * a.ld + c, v);
#pragma unroll
    for (int e = 0; e < N; e += 2) *reinterpret_cast<uint32_t*>(&s.v[r][c + e]) = pack_bf16(v[e], v[e + 1]);
  }
  __syncthreads();
  if (t < rv + 8) {                                             // (pages are multiples of four positions, of G where G is 8)
    bool run = s.page[t] >= 0 && (s.pos[t] & (G - 1)) == 0 && t + G <= rv + 16;
#pragma unroll
    for (int j = 1; j < G; ++j) run = run && s.seq[t + j] == s.seq[t] && s.pos[t + j] == s.pos[t] + j;
    s.run[t] = run;
  }
  __syncthreads();
  if (t < rv) {
    const int u = t + 8, first = u - (s.pos[u] & (G - 1));
    if (s.run[u]) s.runs[atomicAdd(&s.n_run, 1)] = (unsigned char)t;
    else if (s.page[u] >= 0 && !(s.run[first] && s.seq[first] == s.seq[u] && s.pos[first] + (u - first) == s.pos[u])) s.ones[atomicAdd(&s.n_one, 1)] = (unsigned char)t;
  }
  __syncthreads();
  auto place = [&](const int r, const int ch) {
    const int u = r + 8, off = s.pos[u] - page_of(kv, s.pos[u]) * kv.pt;
    return kv.pages + ((size_t)s.page[u] * 2 * kv.nkv + kv.nkv + head) * kv.pt * DH + (size_t)ch * kv.pt + off;
  };
  for (int i = t; i < (s.n_run + 1) / 2 * 2 * DH; i += 256) {   // (two runs side by side: neighbours in a page, mostly)
    const int k = (i & 1) + i / (2 * DH) * 2, ch = (i >> 1) % DH;
    if (k >= s.n_run) continue;
    const int r = s.runs[k];
    uint32_t w[G / 2];
#pragma unroll
    for (int j = 0; j < G / 2; ++j) w[j] = s.v[r + 2 * j][ch] | ((uint32_t)s.v[r + 2 * j + 1][ch] << 16);
    if constexpr (G == 8) *reinterpret_cast<u32x4*>(place(r, ch)) = u32x4{w[0], w[1], w[2], w[3]};
    else *reinterpret_cast<uint2*>(place(r, ch)) = make_uint2(w[0], w[1]);
  }
  for (int i = t; i < s.n_one * DH; i += 256) *place(s.ones[i / DH], i % DH) = s.v[s.ones[i / DH]][i % DH];
}

// Workgroups of queries and keys first (HB heads of a row block side by side), then those of the values (HB == 1: none).
template <int DH, typename T, int HB, int G>
__global__ __launch_bounds__(256) void k_append(AppendArgs a, int n_heads_wgs, int head_groups, int value_blocks) {
  int b = blockIdx.x;
  if (HB == 1 || b < n_heads_wgs) {
    append_heads<DH, T, HB>(a, b / head_groups, b % head_groups * HB);
  } else if constexpr (HB > 1) {
    __shared__ ValueTile<DH> s;
    b -= n_heads_wgs;
    append_values<DH, T, G>(a, b % value_blocks, b / value_blocks, s);
  }
}

// ---------------------------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------------------------
//
// Row r = (sequence * n_tok + token) * group + query head of a K / V head's rows.  A workgroup takes up to 128 rows (k_attn_many) or up to 16 or 32
// (k_attn_few) of one K / V head and a range of positions, of the prompt (then the rows are those of all sequences) or of one sequence's own.
//   S^T[position][row] = K . Q^T,   O^T[channel][row] += V^T . P^T       (32x32x16 or 16x16x32 bf16, fp32 accumulators)
// with a running maximum and sum per row, in fp32.  K rows lie in LDS in the order that gives a lane the scores of consecutive positions, eight at a time: P's
// operand without a move between lanes.  fp32 queries and the probabilities beside them enter as three bf16 terms (24 bits); bf16 queries as they are,
// and the probabilities rounded to bf16 (relative error up to 2^-8 each, independent, so that a row's sum of many errs by less than its own rounding to
// bf16; the sum that divides it is that of the unrounded ones).

struct SoftParts { u32x4 t[3]; };

// Eight floats as bf16 terms.
template <int TERMS>
__device__ __forceinline__ SoftParts split_terms(const float (&x)[8]) {
  SoftParts r;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i];
#pragma unroll
  for (int k = 0; k < TERMS; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = pack_bf16(y[2 * i], y[2 * i + 1]);
      r.t[k][i] = w;
      y[2 * i] -= __uint_as_float(w << 16);
      y[2 * i + 1] -= __uint_as_float(w & 0xffff0000u);
    }
  return r;
}

// Which rows and positions a workgroup takes.
struct AttnItem {
  const bf16_t* pool; const int32_t* table; int n_pages;
  int kvh, row0, rows, part;         // row0: of the K / V head's rows
  int begin, end;                    // positions; begin is a multiple of 32
  int first;                         // own positions: those below it are seen by every token of the call (prompt: end)
};

// A block of 32 positions in LDS, 16-byte chunks.  K: chunk c of the row in place m at m * DH / 8 + (c ^ k_swizzle(m)): a copy of 1 KiB is rows of four
// consecutive positions each, and a fragment read (one chunk column of many rows) meets no bank twice.  Places: a lane's scores have to be those
// of eight consecutive positions (see AttnRows), which are in places four apart from each other.  V: eight positions of a channel, half h of group g
// of sixteen at (g * DH + channel) * 2 + (h ^ channel / 16): a copy takes consecutive bytes of a page of sixteen, and a read meets no bank twice either (a
// 16-byte read of a wavefront goes through LDS in four sets of lanes: 0-3, 12-15, 20-23 and 24-27 are the first).
template <int DH> struct AttnBlock {
  static constexpr int CK = DH / 8, K_CHUNKS = 32 * CK, V_CHUNKS = 4 * DH, COPIES = DH / 16;     // copies (of K, of V) of a wavefront's width
};
template <int DH> __device__ __forceinline__ constexpr int k_swizzle(int m) { return DH == 128 ? m & 15 : (m >> 1) & 7; }
// Which four positions (of a block's eight fours) are in the four places 4 j ..
template <int RB> __device__ __forceinline__ constexpr int four_of(int j) {
  return RB == 32 ? (j & 4) | ((j & 1) << 1) | ((j & 2) >> 1) : ((j & 3) << 1) | (j >> 2);
}

// Copies blocks begin, begin + stride, .. of a range into LDS.  Lane 8 n + f looks up the page of positions 4 f .. of the n-th of eight blocks:
// one table load and one address computation a lane for eight blocks.
template <int DH, int RB>
struct BlockCopy {
  typedef AttnBlock<DH> Bk;
  const AttnItem& it;
  const SharedKv& kv;
  int begin, stride;
  size_t head_elems, page_elems;
  int bad;                           // the first position this lane found in a page outside the pool
  uint64_t k_addr, v_addr;           // of this lane's positions
  int pos, lp, entry;                // of the next eight blocks: positions, page of the sequence, table entry (on its way)

  __device__ __forceinline__ BlockCopy(const AttnItem& i, const SharedKv& k, const int first, const int step) : it(i), kv(k), begin(first), stride(step), head_elems((size_t)k.pt * DH), bad(0x7fffffff) {
    page_elems = 2 * (size_t)k.nkv * head_elems;
    k_addr = v_addr = 0; pos = lp = entry = 0;
  }
  // table entries of blocks i .. i + 7 (beyond the end: the last pieces once more, their scores and values are dropped)
  __device__ __forceinline__ void look_up(const int i) {
    const int lane = threadIdx.x & 63, f = lane & 7, last = (it.end - 1) & ((f & 1) ? ~3 : ~7);
    const long p = (long)begin + (long)(i + (lane >> 3)) * stride + 4 * f;
    pos = p < last ? (int)p : last;
    lp = page_of(kv, pos);
    entry = it.table ? it.table[lp] : lp;
  }
  __device__ __forceinline__ void resolve() {
    int page = entry;
    if ((unsigned)page >= (unsigned)it.n_pages) { page = 0; bad = min(bad, pos); }
    const int off = pos - lp * kv.pt;
    const bf16_t* base = it.pool + (size_t)page * page_elems + it.kvh * head_elems;
    k_addr = reinterpret_cast<uint64_t>(base + (size_t)off * DH);
    v_addr = reinterpret_cast<uint64_t>(base + kv.nkv * head_elems + off);
  }
  // Before block i is copied, in order.
  __device__ __forceinline__ void at_block(const int i) {
    if ((i & 7) == 0) {
      if (i == 0) look_up(0);
      resolve();
      look_up(i + 8);
    }
  }
  static __device__ __forceinline__ uint64_t lane_value(const uint64_t v, const int l) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, l) | ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), l) << 32);
  }
  // copies J0 .. J1 - 1 of block i's K to LDS address lds
  template <int J0, int J1>
  __device__ __forceinline__ void copy_k(const int i, const uint32_t lds) const {
    const int lane = threadIdx.x & 63, n = 8 * (i & 7);
#pragma unroll
    for (int j = J0; j < J1; ++j) {
      if constexpr (DH == 128) {               // four rows
        const uint32_t at = (uint32_t)(lane >> 4) * (DH * 2) + (uint32_t)(((lane & 15) ^ (lane >> 4) ^ (4 * (j & 3))) * 16);
        lds_dma_16(reinterpret_cast<const void*>(lane_value(k_addr, n + four_of<RB>(j))), at, lds + (uint32_t)j * 1024u);
      } else {                                 // eight, of two fours
        const uint64_t b0 = lane_value(k_addr, n + four_of<RB>(2 * j)), b1 = lane_value(k_addr, n + four_of<RB>(2 * j + 1));
        const uint32_t at = (uint32_t)((lane >> 3) & 3) * (DH * 2) + (uint32_t)(((lane & 7) ^ (lane >> 4) ^ (4 * (j & 1))) * 16);
        lds_dma_16(reinterpret_cast<const void*>(((lane & 32) ? b1 : b0) + at), lds + (uint32_t)j * 1024u);
      }
    }
  }
  // ... and of its V, to LDS address lds of chunks v
  template <int J0, int J1>
  __device__ __forceinline__ void copy_v(const int i, const uint32_t lds, u32x4* v) const {
    constexpr int PER_G = DH / 32;             // copies of sixteen positions
    const int lane = threadIdx.x & 63, n = 8 * (i & 7), half = (lane ^ (lane >> 5)) & 1;
    const uint64_t row = (uint64_t)(uint32_t)((lane >> 1) * kv.pt * 2);
    if ((kv.pt & 7) == 0) {
      uint64_t b = 0;
#pragma unroll
      for (int j = J0; j < J1; ++j) {
        if (j == J0 || j % PER_G == 0) {
          const uint64_t b0 = lane_value(v_addr, n + 4 * (j / PER_G)), b1 = lane_value(v_addr, n + 4 * (j / PER_G) + 2);
          b = (half ? b1 : b0) + row;
        }
        lds_dma_16(reinterpret_cast<const void*>(b + (uint64_t)(64 * (j % PER_G)) * kv.pt), lds + (uint32_t)j * 1024u);
      }
    } else {                                   // a page may end after four of the eight: through registers
#pragma unroll
      for (int j = J0; j < J1; ++j) {
        uint64_t b[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) b[u] = lane_value(v_addr, n + 4 * (j / PER_G) + u) + row + (uint64_t)(64 * (j % PER_G)) * kv.pt;
        const uint2 x = *reinterpret_cast<const uint2*>(half ? b[2] : b[0]), y = *reinterpret_cast<const uint2*>(half ? b[3] : b[1]);
        v[j * 64 + lane] = u32x4{x.x, x.y, y.x, y.y};
      }
    }
  }
};

// V chunks i0, i0 + step, .. of a block of positions from base on that not every row sees or that lie beyond the end, put right in LDS: what is beyond
// the end is anything, and 0 * NaN would poison the sum; so would an infinity or NaN among the newest positions, which some tokens do not see.
// Those become 0 as well, and the result says so (add_odd gives them to the rows that do see them).
template <int DH>
__device__ __forceinline__ bool mend_values(const AttnItem& it, const int base, u32x4* vs, const int i0, const int step) {
  bool odd = false;
  for (int i = i0; i < AttnBlock<DH>::V_CHUNKS; i += step) {
    const int ch = (i >> 1) % DH, half = (i ^ (ch >> 4)) & 1, at = base + 16 * (i / (2 * DH)) + 8 * half;
    if (at + 8 <= it.first) continue;
    u32x4 v = vs[i];
    const int n = it.end - at, n_all = it.first - at;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t mask = (e & 1) ? 0xffff0000u : 0xffffu, x = v[e >> 1] & mask, inf = 0x7f807f80u & mask;
      if (e >= n) v[e >> 1] &= ~mask;
      else if (e >= n_all && (x & inf) == inf) { v[e >> 1] &= ~mask; odd = true; }
    }
    vs[i] = v;
  }
  return odd;
}

// RB (16 or 32) rows of a wavefront: queries, running statistics, output.  A lane's scores are those of its row and, eight at a time, of consecutive
// positions: 32 rows, 32x32x16 products: positions 16 n + 8 (lane / 32) + 0 .. 7; 16 rows, 16x16x32 products: positions 8 (lane / 16) + 0 .. 7.
// Those are what the second product wants of the lane, so the probabilities never leave it.
template <int DH, int RB, bool F32>
struct AttnRows {
  typedef typename std::conditional<RB == 32, f32x16, f32x4>::type Acc;
  static constexpr int CK = DH / 8, TERMS = F32 ? 3 : 1;
  static constexpr int STEPS = RB == 32 ? DH / 16 : DH / 32;   // products over the channels
  static constexpr int CB = DH / RB, AV = RB == 32 ? 16 : 4;   // channel tiles of the output, values of one
  static constexpr int NS = RB == 32 ? 16 : 8, SV = NS / 8;    // scores of a lane in a block
  bf16x8 q[STEPS][TERMS];
  Acc O[CB];
  float m_run, l_run, ce;
  int col, hf, tok, see;                                        // row, part of the wavefront, token of the call, positions of the range that the row sees

  // The queries as they lie in memory: requested first, turned into terms (init) when the first copies are on their way.
  struct Raw { u32x4 v[STEPS * (F32 ? 2 : 1)]; };
  static __device__ __forceinline__ Raw request(const SharedAttnArgs& a, const AttnItem& it, const int r, const int grp) {
    Raw q;
    const size_t at = (size_t)(r / grp) * a.ld_q + (size_t)(it.kvh * grp + r % grp) * DH + 8 * ((threadIdx.x & 63) / RB);
    constexpr int W = DH / STEPS;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if constexpr (F32) {
        const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const float*>(a.q) + at + W * s);
        q.v[2 * s] = p[0]; q.v[2 * s + 1] = p[1];
      } else {
        q.v[s] = *reinterpret_cast<const u32x4*>(static_cast<const bf16_t*>(a.q) + at + W * s);
      }
    }
    return q;
  }
  __device__ __forceinline__ void init(const SharedAttnArgs& a, const AttnItem& it, const Raw& raw, const int r, const int grp) {
    const int lane = threadIdx.x & 63;
    col = lane & (RB - 1); hf = lane / RB;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if constexpr (F32) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(raw.v[2 * s + (i >> 2)][i & 3]);
        const SoftParts sp = split_terms<TERMS>(y);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) q[s][k] = as_bf16x8(sp.t[k]);
      } else {
        q[s][0] = as_bf16x8(raw.v[s]);
      }
    }
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int v = 0; v < AV; ++v) O[c][v] = 0.f;
    m_run = -INFINITY; l_run = 0.f;
    ce = a.scale * LOG2E;
    tok = r / grp % a.n_tok;
    see = min(it.end, it.first + tok);
  }
  static __device__ __forceinline__ Acc product(const bf16x8 x, const bf16x8 y, const Acc c) {
    if constexpr (RB == 32) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
  }
  static __device__ __forceinline__ float row_max(float x) { if constexpr (RB == 32) return half_max(x); else return row4_max(x); }
  __device__ __forceinline__ float row_sum() const { if constexpr (RB == 32) return half_sum(l_run); else return row4_sum(l_run); }
  // channel of value v of output tile c
  __device__ __forceinline__ int channel(const int c, const int v) const { return RB == 32 ? 32 * c + 8 * (v >> 2) + 4 * hf + (v & 3) : 16 * c + 4 * hf + v; }

  template <int NB> struct Scores { float s[NB * NS]; };
  // scores of NB blocks of 32 positions in LDS at ks
  template <int NB>
  __device__ __forceinline__ Scores<NB> scores(const u32x4* ks) const {
    Scores<NB> r;
    constexpr int TILES = 32 / RB * NB, AHEAD = 4, N = STEPS * TILES;      // tiles of places; fragments are read AHEAD of their products
    Acc S[TILES];
    auto k_frag = [&](const int i) {
      const int place = i % TILES * RB + col;
      return as_bf16x8(ks[place * CK + ((64 / RB * (i / TILES) + hf) ^ k_swizzle<DH>(place & 31))]);
    };
    bf16x8 kk[AHEAD + 1];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) kk[i] = k_frag(i);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i + AHEAD < N) kk[(i + AHEAD) % (AHEAD + 1)] = k_frag(i + AHEAD);
#pragma unroll
      for (int u = 0; u < TERMS; ++u) {
        if (i < TILES && u == 0) {
          Acc z;
#pragma unroll
          for (int v = 0; v < AV; ++v) z[v] = 0.f;
          S[i % TILES] = product(kk[i % (AHEAD + 1)], q[0][0], z);
        } else {
          S[i % TILES] = product(kk[i % (AHEAD + 1)], q[i / TILES][u], S[i % TILES]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int v = 0; v < NB * NS; ++v) r.s[v] = S[v / AV][v % AV];
    return r;
  }
  // Probabilities (relative to the running maximum) of the positions from base on, in place of their scores.
  template <int NB>
  __device__ __forceinline__ void weigh(const AttnItem& it, const int base, Scores<NB>& S) {
    if (base + 32 * NB > it.first) {                            // some position is not seen by every row (uniform)
#pragma unroll
      for (int v = 0; v < NB * NS; ++v)
        if (base + 32 * (v / NS) + 16 * (v % NS >> 3) + 8 * hf + (v & 7) >= see) S.s[v] = -INFINITY;
    }
    float mx = S.s[0];
#pragma unroll
    for (int v = 1; v < NB * NS; ++v) mx = fmaxf(mx, S.s[v]);
    mx = row_max(mx) * ce;
    // The sums stay relative to an older maximum while the new one is at most 2^8 of it: the largest terms are then below 2^8 and no sum loses
    // precision for it, and after the first blocks almost no block rescales its output.
    if (__builtin_amdgcn_ballot_w64(mx > m_run + 8.f) != 0ull) {
      const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;    // (-inf: the row has seen nothing yet)
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
      l_run *= alpha;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int v = 0; v < AV; ++v) O[c][v] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int v = 0; v < NB * NS; ++v) { S.s[v] = __builtin_amdgcn_exp2f(fmaf(S.s[v], ce, -m_use)); sum[v & 1] += S.s[v]; }
    l_run += sum[0] + sum[1];
  }
  // output += values in LDS at vs, weighted
  template <int NB>
  __device__ __forceinline__ void add(const u32x4* vs, const Scores<NB>& P) {
    constexpr int N = NB * SV;
    u32x4 vv[2][CB];
    auto v_frag = [&](const int s, const int c) {
      const int ch = RB * c + col, g = RB == 32 ? s : 2 * s + (hf >> 1), half = RB == 32 ? hf : hf & 1;
      return vs[(g * DH + ch) * 2 + (half ^ ((ch >> 4) & 1))];
    };
#pragma unroll
    for (int c = 0; c < CB; ++c) vv[0][c] = v_frag(0, c);
#pragma unroll
    for (int s = 0; s < N; ++s) {
      if (s + 1 < N)
#pragma unroll
        for (int c = 0; c < CB; ++c) vv[(s + 1) & 1][c] = v_frag(s + 1, c);
      const float px[8] = {P.s[8 * s], P.s[8 * s + 1], P.s[8 * s + 2], P.s[8 * s + 3], P.s[8 * s + 4], P.s[8 * s + 5], P.s[8 * s + 6], P.s[8 * s + 7]};
      const SoftParts sp = split_terms<TERMS>(px);
#pragma unroll
      for (int u = 0; u < TERMS; ++u)
#pragma unroll
        for (int c = 0; c < CB; ++c) O[c] = product(as_bf16x8(vv[s & 1][c]), as_bf16x8(sp.t[u]), O[c]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Infinities and NaN among the values of the newest positions of this range, to the rows that see them (with whatever weight: they stay
  // infinite); mend_values has kept them out of the sums.  (share w of wt: the blocks that this wavefront takes)
  __device__ __forceinline__ void add_odd(const SharedKv& kv, const AttnItem& it, const int w, const int wt) {
    const int begin = max(max(it.first, it.begin), 0);
    const size_t head_elems = (size_t)kv.pt * DH, page_elems = 2 * (size_t)kv.nkv * head_elems;
    for (int pos = begin; pos < it.end; ++pos) {
      if (((pos - it.begin) >> 5) % wt != w) continue;
      const int lp = page_of(kv, pos), page = it.table ? it.table[lp] : lp;
      if ((unsigned)page >= (unsigned)it.n_pages) continue;
      const bf16_t* v = it.pool + (size_t)page * page_elems + (kv.nkv + it.kvh) * head_elems + (pos - lp * kv.pt);
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < AV; ++i) {
          const uint32_t x = v[(size_t)channel(c, i) * kv.pt];
          if (pos < see && (x & 0x7f80u) == 0x7f80u) O[c][i] += __uint_as_float(x << 16);
        }
    }
  }
};

// Four channels of a row as the next matrix' input (panels of up to sixteen rows).
__device__ __forceinline__ void put_panels(const SharedAttnArgs& a, const int row, const int k, const float4 o) {
  const float v[4] = {o.x, o.y, o.z, o.w};
  xpack_store4(a.panels, (a.nq * a.kv.dh) >> 5, a.kv.n_seqs * a.n_tok, row, k, v);
}

// A row's result: to the output, or as this range's part.
template <int DH, bool F32>
struct AttnPut {
  const SharedAttnArgs& a;
  const AttnItem& it;
  int grp;
  size_t head_rows;
  __device__ __forceinline__ AttnPut(const SharedAttnArgs& x, const AttnItem& i) : a(x), it(i), grp(x.nq / x.kv.nkv), head_rows((size_t)x.kv.n_seqs * x.n_tok * grp) {}
  __device__ __forceinline__ void row(const int r, const int c, float4 o, const float l) const {
    if (a.plan.parts > 1) {
      store4(a.part + (((size_t)it.part * a.kv.nkv + it.kvh) * head_rows + r) * DH + c, o);
      return;
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    o = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (F32 && a.panels != nullptr) {
      put_panels(a, r / grp, (it.kvh * grp + r % grp) * DH + c, o);
      return;
    }
    const size_t at = (size_t)(r / grp) * a.ld_out + (size_t)(it.kvh * grp + r % grp) * DH + c;
    if constexpr (F32) store4(static_cast<float*>(a.out) + at, o);
    else store4(static_cast<bf16_t*>(a.out) + at, o);
  }
  __device__ __forceinline__ void stat(const int r, const float m, const float l) const {
    if (a.plan.parts > 1) a.ml[((size_t)it.part * a.kv.nkv + it.kvh) * head_rows + r] = make_float2(m, l);
    else if (a.lse != nullptr) a.lse[(size_t)(r / grp) * a.nq + it.kvh * grp + r % grp] = l == 0.f ? -INFINITY : (m + __log2f(l)) * LN2;
  }
};

// 128 rows: four wavefronts of 32 that share the positions through LDS, 64 at a time in two buffers.  Bound by the LDS reads of K and V beside the products (each
// wavefront reads all of a tile: 128 KiB at 128 bytes a clock are as long as the products of two workgroups of a compute unit) and, in long prompts whose pages lie in
// random order, by the feed: 96 sequences of 32 heads on 8 behind 65537 positions 122 us, 0.85 PFLOP/s; 4608 rows of one K / V head over 3001 positions 20 us,
// one workgroup a compute unit (2.6 us for a tile, as with two).  Scores of the next tile between the products of this one in a wavefront: 123 to 130 us.
template <int DH, bool F32>
__device__ __forceinline__ void attn_many(const SharedAttnArgs& a, const AttnItem& it, char* lds) {
  typedef AttnBlock<DH> Bk;
  u32x4* ks = reinterpret_cast<u32x4*>(lds);                    // [buffer][block]
  u32x4* vs = ks + 4 * Bk::K_CHUNKS;
  __shared__ int s_bad, s_odd;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = 32 * (w >> 1);
  BlockCopy<DH, 32> cp(it, a.kv, it.begin + mine, 64);
  const uint32_t lds_k = lds_address(ks), lds_v = lds_address(vs);
  auto copy = [&](const int i) {                                // tile i: of block w / 2, half its copies
    const int b = 2 * (i & 1) + (w >> 1);
    constexpr int H = Bk::COPIES / 2;
    cp.at_block(i);
    if (w & 1) {
      cp.template copy_k<H, Bk::COPIES>(i, lds_k + b * Bk::K_CHUNKS * 16);
      cp.template copy_v<H, Bk::COPIES>(i, lds_v + b * Bk::V_CHUNKS * 16, vs + b * Bk::V_CHUNKS);
    } else {
      cp.template copy_k<0, H>(i, lds_k + b * Bk::K_CHUNKS * 16);
      cp.template copy_v<0, H>(i, lds_v + b * Bk::V_CHUNKS * 16, vs + b * Bk::V_CHUNKS);
    }
  };
  if (threadIdx.x == 0) { s_bad = 0x7fffffff; s_odd = 0; }
  const int grp = a.nq / a.kv.nkv, r_in = 32 * w + (threadIdx.x & 31), r_mine = it.row0 + min(r_in, it.rows - 1);    // surplus lanes repeat the last row
  AttnRows<DH, 32, F32> x;
  const auto raw = x.request(a, it, r_mine, grp);
  const int tiles = it.begin < it.end ? (it.end - it.begin + 63) / 64 : 0;
  if (tiles > 0) copy(0);
  x.init(a, it, raw, r_mine, grp);
  const bool idle = 32 * w >= it.rows;
  for (int i = 0; i < tiles; ++i) {
    const int t0 = it.begin + 64 * i, buf = i & 1;
    // the tile has arrived and every wavefront has left the other buffer
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (i + 1 < tiles) copy(i + 1);
    if (t0 + 64 > it.first) {
      if (mend_values<DH>(it, t0 + mine, vs + (2 * buf + (w >> 1)) * Bk::V_CHUNKS, threadIdx.x & 127, 128)) s_odd = 1;
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    if (!idle) {
      auto S = x.template scores<2>(ks + 2 * buf * Bk::K_CHUNKS);
      x.weigh(it, t0, S);
      x.add(vs + 2 * buf * Bk::V_CHUNKS, S);
    }
  }
  __syncthreads();
  if (cp.bad != 0x7fffffff) atomicMin(&s_bad, cp.bad);
  __syncthreads();
  if (s_odd != 0) x.add_odd(a.kv, it, 0, 1);
  if (r_in >= it.rows) return;
  float l = x.row_sum();
  if (s_bad < x.see) l = NAN;
  const AttnPut<DH, F32> put(a, it);
  const int r = it.row0 + r_in;
#pragma unroll
  for (int c = 0; c < x.CB; ++c)
#pragma unroll
    for (int i = 0; i < 16; i += 4) put.row(r, x.channel(c, i), make_float4(x.O[c][i], x.O[c][i + 1], x.O[c][i + 2], x.O[c][i + 3]), l);
  if (x.hf == 0) put.stat(r, x.m_run, l);
}

// Up to RB rows: WT wavefronts take a block of 32 positions each in turn, copied by themselves into a K and a V buffer of their own (no barrier): the
// next block's K is on its way from the scores on, its V from the output on, and other wavefronts of the SIMD cover what is left of the wait.
// Results are put together at the end.  Bound by the feed: own positions of 96 sequences on 8 heads, 1 to 700 each, 137 MB, 49 us, 2.8 TB/s (ranges of equal length, sequences
// of different ones); eight beams of 40 heads over 2048 + 130 positions, 54 MB, 16 us; four of 12 heads over 523 + 37 7 us, round trips.  `also`: a second range for the same rows, walked first (pool == nullptr: none).
template <int DH, int RB, int WT, bool F32> struct FewShape {
  typedef AttnBlock<DH> Bk;
  static constexpr int OLD = DH + 4;                            // a row put together in LDS
  static constexpr size_t stage = (size_t)WT * (Bk::K_CHUNKS + Bk::V_CHUNKS) * 16, merge = WT == 1 ? 0 : (size_t)(WT * RB * (OLD + 2) + 4 * WT) * 4;
  static constexpr size_t lds = stage > merge ? stage : merge;
};
template <int DH, int RB, int WT, bool F32>
__device__ __forceinline__ void attn_few(const SharedAttnArgs& a, const AttnItem& it, const AttnItem& also, char* lds) {
  typedef AttnBlock<DH> Bk;
  constexpr int OLD = FewShape<DH, RB, WT, F32>::OLD;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = threadIdx.x & (RB - 1), lane = threadIdx.x & 63;
  u32x4* ks = reinterpret_cast<u32x4*>(lds) + w * (Bk::K_CHUNKS + Bk::V_CHUNKS);
  u32x4* vs = ks + Bk::K_CHUNKS;
  const uint32_t lds_k = lds_address(ks), lds_v = lds_address(vs);
  const int r_mine = it.row0 + min(col, it.rows - 1);
  AttnRows<DH, RB, F32> x;
  const auto raw = x.request(a, it, r_mine, a.nq / a.kv.nkv);
  bool started = false;
  auto walk = [&](const AttnItem& seg) {                        // the first position of seg in a page outside the pool
    BlockCopy<DH, RB> cp(seg, a.kv, seg.begin + 32 * w, 32 * WT);
    const int n = seg.end > cp.begin ? (seg.end - cp.begin + 32 * WT - 1) / (32 * WT) : 0;    // blocks
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // (reads of the range before)
    if (n > 0) {
      cp.at_block(0);
      cp.template copy_k<0, Bk::COPIES>(0, lds_k);
      cp.template copy_v<0, Bk::COPIES>(0, lds_v, vs);
    }
    if (!started) x.init(a, it, raw, r_mine, a.nq / a.kv.nkv);
    started = true;
    x.see = min(seg.end, seg.first + x.tok);
    bool odd = false;
    for (int i = 0; i < n; ++i) {
      const int t0 = cp.begin + i * cp.stride;
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(Bk::COPIES) : "memory");     // its K (V's copies were sent later)
      auto S = x.template scores<1>(ks);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (i + 1 < n) {
        cp.at_block(i + 1);
        cp.template copy_k<0, Bk::COPIES>(i + 1, lds_k);
      }
      x.weigh(seg, t0, S);
      if (i + 1 < n) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(Bk::COPIES) : "memory");
      else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      if (t0 + 32 > seg.first) {
        odd |= mend_values<DH>(seg, t0, vs, lane, 64);
        wave_lds_fence();
      }
      x.add(vs, S);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (i + 1 < n) cp.template copy_v<0, Bk::COPIES>(i + 1, lds_v, vs);
    }
    odd = __builtin_amdgcn_ballot_w64(odd) != 0ull;
    if (odd) x.add_odd(a.kv, seg, w, WT);
    int bad = cp.bad;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) bad = min(bad, __shfl_xor(bad, o));
    return bad;
  };
  int bad = 0x7fffffff;                                         // of `it`; in front of all positions: one of `also`
  if (also.pool != nullptr && walk(also) != 0x7fffffff) bad = INT_MIN;
  bad = min(bad, walk(it));
  const float l_wave = x.row_sum();
  const AttnPut<DH, F32> put(a, it);
  constexpr int AV = AttnRows<DH, RB, F32>::AV, CB = AttnRows<DH, RB, F32>::CB;
  if constexpr (WT == 1) {
    if (col < it.rows) {
      const float l = bad < x.see ? NAN : l_wave;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < AV; i += 4) put.row(r_mine, x.channel(c, i), make_float4(x.O[c][i], x.O[c][i + 1], x.O[c][i + 2], x.O[c][i + 3]), l);
      if (x.hf == 0) put.stat(r_mine, x.m_run, l);
    }
    return;
  }
  float* sm = reinterpret_cast<float*>(lds);                    // [WT][RB] maxima, sums, first bad positions, then rows
  float* sl = sm + WT * RB;
  int* sb = reinterpret_cast<int*>(sl + WT * RB);
  float* so = sl + WT * RB + 4 * WT;
  __syncthreads();
  if (x.hf == 0) { sm[w * RB + col] = x.m_run; sl[w * RB + col] = l_wave; }
  if (lane == 0) sb[w] = bad;
  __syncthreads();
  float mm = sm[col];
#pragma unroll
  for (int u = 1; u < WT; ++u) mm = fmaxf(mm, sm[u * RB + col]);
  const float f = mm == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.m_run - mm);
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int i = 0; i < AV; i += 4)
      store4(so + (size_t)(w * RB + col) * OLD + x.channel(c, i), make_float4(x.O[c][i] * f, x.O[c][i + 1] * f, x.O[c][i + 2] * f, x.O[c][i + 3] * f));
  __syncthreads();
  int first_bad = sb[0];
#pragma unroll
  for (int u = 1; u < WT; ++u) first_bad = min(first_bad, sb[u]);
  for (int i = threadIdx.x; i < it.rows * (DH / 4); i += 64 * WT) {
    const int row = i / (DH / 4), c = i % (DH / 4) * 4;
    float m = sm[row], l = 0.f;
#pragma unroll
    for (int u = 1; u < WT; ++u) m = fmaxf(m, sm[u * RB + row]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int u = 0; u < WT; ++u) {
      const float4 y = load4(so + (size_t)(u * RB + row) * OLD + c);
      o = make_float4(o.x + y.x, o.y + y.y, o.z + y.z, o.w + y.w);
      l += m == -INFINITY ? 0.f : sl[u * RB + row] * __builtin_amdgcn_exp2f(sm[u * RB + row] - m);
    }
    const int r = it.row0 + row, t = r / put.grp % a.n_tok;
    if (first_bad < min(it.end, it.first + t)) l = NAN;
    put.row(r, c, o, l);
    if (c == 0) put.stat(r, m, l);
  }
}

// Workgroup b of the prompt's: ranges of a K / V head, whose row tiles go to one XCD (ids go round-robin to the eight) and so share its L2.
__device__ __forceinline__ AttnItem prefix_item(const SharedAttnArgs& a, const int b, const int row_tile) {
  const SharedAttnPlan& p = a.plan;
  const SharedKv& kv = a.kv;
  const int units = kv.nkv * p.prefix_splits, block = 8 * p.prefix_tiles, g = b / block, left = min(8, units - 8 * g), r = b - g * block;
  const int tile = r / left, unit = 8 * g + r - tile * left, split = unit / kv.nkv;
  AttnItem it;
  it.kvh = unit - split * kv.nkv;
  it.pool = kv.prefix; it.table = kv.prefix_table; it.n_pages = kv.n_prefix_pages;
  it.row0 = tile * row_tile; it.rows = min(row_tile, kv.n_seqs * a.n_tok * (a.nq / kv.nkv) - it.row0);
  it.begin = split * p.prefix_len; it.end = min(kv.prefix_len, it.begin + p.prefix_len); it.first = it.end;
  it.part = split;
  return it;
}
// Workgroup b of the own positions'.
__device__ __forceinline__ AttnItem own_item(const SharedAttnArgs& a, int b, const int row_tile) {
  const SharedAttnPlan& p = a.plan;
  const SharedKv& kv = a.kv;
  AttnItem it;
  it.kvh = b % kv.nkv; b /= kv.nkv;
  const int split = b % p.own_splits; b /= p.own_splits;
  const int tile = b % p.own_tiles, seq = b / p.own_tiles;
  const int rows = a.n_tok * (a.nq / kv.nkv), len = min(kv.lens[seq], kv.table_ld * kv.pt);
  it.pool = kv.pages; it.table = kv.tables + (size_t)seq * kv.table_ld; it.n_pages = kv.n_pages;
  it.row0 = seq * rows + tile * row_tile; it.rows = min(row_tile, rows - tile * row_tile);
  it.begin = split * p.own_len; it.end = split + 1 == p.own_splits ? len : min(len, it.begin + p.own_len);
  it.first = len - a.n_tok + 1;
  it.part = p.prefix_splits + split;
  return it;
}

template <int DH, bool F32>
__global__ __launch_bounds__(256, F32 && DH == 128 ? 1 : 2) void k_attn_many(SharedAttnArgs a, int n_prefix) {
  __shared__ __align__(16) char lds[4 * (AttnBlock<DH>::K_CHUNKS + AttnBlock<DH>::V_CHUNKS) * 16];
  const int b = blockIdx.x;
  attn_many<DH, F32>(a, b < n_prefix ? prefix_item(a, b, 128) : own_item(a, b - n_prefix, 128), lds);
}
// fused: a workgroup walks the prompt itself before its sequence's own positions
template <int DH, int RB, int WT, bool F32>
__global__ __launch_bounds__(64 * WT, RB == 32 && DH == 128 ? 1 : 2) void k_attn_few(SharedAttnArgs a, int n_prefix) {
  __shared__ __align__(16) char lds[FewShape<DH, RB, WT, F32>::lds];
  const int b = blockIdx.x;
  const AttnItem it = b < n_prefix ? prefix_item(a, b, RB) : own_item(a, b - n_prefix, RB);
  AttnItem also = it;
  also.pool = nullptr;
  if (a.plan.fused) {
    also.pool = a.kv.prefix; also.table = a.kv.prefix_table; also.n_pages = a.kv.n_prefix_pages;
    also.begin = 0; also.end = also.first = a.kv.prefix_len;
  }
  attn_few<DH, RB, WT, F32>(a, it, also, lds);
}

// The parts of a row put together.  DH / 4 lanes a row: first every lane takes statistics of some parts, then its four channels of all of them,
// eight parts on their way at once.  Bound by the round trips: parts come from other XCDs' stores, through the memory-side cache (3.6 us for 48 rows, 5.5 us for 4608 of
// eight parts, 19 MB).
template <int DH, bool F32>
__global__ __launch_bounds__(256) void k_shared_merge(SharedAttnArgs a) {
  constexpr int LPR = DH / 4, RPW = 256 / LPR, PPL = ATTN_MAX_PARTS / LPR;
  __shared__ float s_f[RPW][ATTN_MAX_PARTS];
  const SharedKv& kv = a.kv;
  const int grp = a.nq / kv.nkv, parts = a.plan.parts, me = threadIdx.x % LPR, wr = threadIdx.x / LPR;
  const size_t head_rows = (size_t)kv.n_seqs * a.n_tok * grp, total = head_rows * kv.nkv;
  const size_t i = (size_t)blockIdx.x * RPW + wr;
  if (i >= total) return;                                       // (a row's lanes are of one wavefront)
  float2 st[PPL];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int u = 0; u < PPL; ++u) {
    st[u] = make_float2(-INFINITY, 0.f);
    if (u * LPR + me < parts) st[u] = a.ml[(size_t)(u * LPR + me) * total + i];
  }
#pragma unroll
  for (int u = 0; u < PPL; ++u) m = fmaxf(m, st[u].x);
#pragma unroll
  for (int o = 1; o < LPR; o *= 2) m = fmaxf(m, __shfl_xor(m, o));
#pragma unroll
  for (int u = 0; u < PPL; ++u) {
    // a part of which the row sees nothing has sum 0 and weighs nothing
    const float f = st[u].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(st[u].x - m);
    if (st[u].y != 0.f) l += st[u].y * f;
    if (u * LPR + me < parts) s_f[wr][u * LPR + me] = f;
  }
#pragma unroll
  for (int o = 1; o < LPR; o *= 2) l += __shfl_xor(l, o);
  wave_lds_fence();
  const float* part = a.part + i * DH + me * 4;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p = 0; p < parts; p += 8) {
    float4 x[8];
    float f[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int q = min(p + u, parts - 1);
      x[u] = load4(part + (size_t)q * total * DH);
      f[u] = p + u < parts ? s_f[wr][q] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (f[u] != 0.f) o = make_float4(fmaf(x[u].x, f[u], o.x), fmaf(x[u].y, f[u], o.y), fmaf(x[u].z, f[u], o.z), fmaf(x[u].w, f[u], o.w));
  }
  const int kvh = (int)(i / head_rows), row = (int)(i % head_rows), tr = row / grp, head = kvh * grp + row % grp;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  o = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  if (F32 && a.panels != nullptr) put_panels(a, tr, head * DH + me * 4, o);
  else if constexpr (F32) store4(static_cast<float*>(a.out) + (size_t)tr * a.ld_out + (size_t)head * DH + me * 4, o);
  else store4(static_cast<bf16_t*>(a.out) + (size_t)tr * a.ld_out + (size_t)head * DH + me * 4, o);
  if (me == 0 && a.lse != nullptr) a.lse[(size_t)tr * a.nq + head] = l == 0.f ? -INFINITY : (m + __log2f(l)) * LN2;
}

// ---------------------------------------------------------------------------------------------
// beam selection
// ---------------------------------------------------------------------------------------------
//
// key(b, v) = score_b + x_bv - logsumexp(x_b).  Inside a row the order is that of the logits themselves; between rows the keys are
// compared in 64 bits.  Two launches: a wavefront per unit of 64 E logits of a row holds them in registers and leaves their maximum,
// their sum of exponentials and the k largest in order; a workgroup per group merges the units of each row (a wavefront a row) and
// ranks the rows' k best against each other.  The k largest of many come from a bound (the k-th largest of 256 partial maxima), a
// list of what reaches it, and the rank of each entry of the list: no sort and no rounds of k.
// Units: bound by the instructions of a logit (unpacking, maximum, difference, exponential at a quarter of the rate, sum): 64 groups of sixteen beams over 128001
// bf16 logits, 262 MB, 63 us, 4.2 TB/s.  Merge: one workgroup a group, a chain of round trips (candidates from other XCDs 2 us, the row's list 2 us, logarithm
// and keys 1 us, ranks between the rows 1.5 us): 6 us for one group of four beams, 9 for eight of eight, 11 for the 64 of sixteen.

__device__ __forceinline__ float logit(const float* p) { return *p; }
__device__ __forceinline__ float logit(const bf16_t* p) { return bf16_to_f32(*p); }

// A bound that at least k of the wavefront's 256 values reach (0 where fewer are not 0): the k-th largest but for its last 12 bits (stopping
// once few enough reach the bound makes the list longer: half a microsecond slower).
__device__ __forceinline__ uint32_t kth_bound(const uint32_t (&m)[4], const int k) {
  const uint32_t top = wave_max_u32(max(max(m[0], m[1]), max(m[2], m[3])));
  uint32_t cur = 0;
  for (int bit = 31; bit >= 12; --bit) {
    const uint32_t t = cur | (1u << bit);
    if (t > top) continue;
    const int n = __popcll(__ballot(m[0] >= t)) + __popcll(__ballot(m[1] >= t)) + __popcll(__ballot(m[2] >= t)) + __popcll(__ballot(m[3] >= t));
    if (n >= k) cur = t;
  }
  return cur;
}

constexpr int BEAM_LIST = 256;       // keys of a wavefront's list
constexpr int BEAM_STAGE = 64;       // quarters of lanes' logits that are kept in LDS

// The k largest keys of a wavefront, in order, to out[0 .. k) (0 behind the last).  visit(f): f(whether the lane's e-th entry reaches the bound,
// entry) for every e; narrow(): makes the bound the k-th largest key itself; key(entry): distinct.  At least k entries reach the bound, or all do.
template <typename Visit, typename Narrow, typename Key>
__device__ __forceinline__ void wave_top_k(Visit visit, Narrow narrow, Key key, const int k, unsigned long long* list, unsigned long long* out) {
  const int lane = threadIdx.x & 63;
  int n = 0;
  auto append = [&](const bool mine, auto entry) {
    const unsigned long long hit = __ballot(mine);
    if (hit == 0) return;
    if (mine) {
      const int at = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(hit >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hit, 0));
      if (at < BEAM_LIST) list[at] = entry();
    }
    n += __popcll(hit);
  };
  visit(append);
  if (n > BEAM_LIST) {               // many equal values
    narrow();
    n = 0;
    visit(append);
  }
  wave_lds_fence();
  const int n_pad = (n + 7) & ~7;
  for (int i = lane; i < n_pad; i += 64) list[i] = i < n ? key(list[i]) : 0ull;
  wave_lds_fence();
  for (int i = lane; i < n; i += 64) {
    const unsigned long long mine = list[i];
    int rank = 0;
    for (int j = 0; j < n_pad; j += 8) {                        // (eight reads on their way at once)
      unsigned long long x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = list[j + u];
#pragma unroll
      for (int u = 0; u < 8; ++u) rank += x[u] > mine ? 1 : 0;
    }
    if (rank < k) out[rank] = mine;
  }
  for (int i = n + lane; i < k; i += 64) out[i] = 0;
}
// The same over 64 x 16 keys r in registers.
__device__ __forceinline__ void wave_top_k_keys(const unsigned long long (&r)[16], const uint32_t bound, const int k, unsigned long long* list, unsigned long long* out) {
  unsigned long long least = (unsigned long long)max(bound, 1u) << 32;
  wave_top_k([&](auto f) {
#pragma unroll
    for (int e = 0; e < 16; ++e) f(r[e] >= least, [&]() { return r[e]; });
  }, [&]() {
    least = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long t = least | (1ull << bit);
      int c = 0;
#pragma unroll
      for (int e = 0; e < 16; ++e) c += __popcll(__ballot(r[e] >= t));
      if (c >= k) least = t;
    }
    if (least == 0) least = 1;
  }, [](unsigned long long x) { return x; }, k, list, out);
}
// The same over `total` keys in memory, of which at least k reach the bound, or all that are not 0.  While more than the list holds reach it, the k-th
// largest of those in the list becomes the bound: at least k reach that, and BEAM_LIST - k fewer than before.
__device__ __forceinline__ void wave_top_k_memory(const unsigned long long* src, const int total, const uint32_t bound, const int k, unsigned long long* list, unsigned long long* out) {
  const int lane = threadIdx.x & 63;
  unsigned long long least = (unsigned long long)max(bound, 1u) << 32;
  int n;
  auto rank_of = [&](const unsigned long long mine, const int end) {
    int rank = 0;
    for (int j = 0; j < end; j += 8)
#pragma unroll
      for (int u = 0; u < 8; ++u) rank += list[j + u] > mine ? 1 : 0;
    return rank;
  };
  for (;;) {
    n = 0;
    for (int i = lane; i - lane < total; i += 64 * 8) {
      unsigned long long x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = i + 64 * u < total ? src[i + 64 * u] : 0ull;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const unsigned long long hit = __ballot(x[u] >= least);
        const int at = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(hit >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hit, 0));
        if (x[u] >= least && at < BEAM_LIST) list[at] = x[u];
        n += __popcll(hit);
      }
    }
    wave_lds_fence();
    if (n <= BEAM_LIST) break;
    unsigned long long kth = 0;
    for (int i = lane; i < BEAM_LIST; i += 64)
      if (rank_of(list[i], BEAM_LIST) == k - 1) kth = list[i];
    least = __shfl(kth, __ffsll((unsigned long long)__ballot(kth != 0)) - 1);
    wave_lds_fence();
  }
  const int n_pad = (n + 7) & ~7;
  for (int i = n + lane; i < n_pad; i += 64) list[i] = 0;
  wave_lds_fence();
  for (int i = lane; i < n; i += 64) {
    const unsigned long long mine = list[i];
    const int rank = rank_of(mine, n_pad);
    if (rank < k) out[rank] = mine;
  }
  for (int i = n + lane; i < k; i += 64) out[i] = 0;
}

// E logits of a lane in registers, eight consecutive ones at a time, in 16-byte loads wherever the row starts (rows of an odd vocabulary do not
// start at 16 bytes); -inf beyond the row.  bf16 logits stay packed and are unpacked in every pass over them: half the registers, so that
// six wavefronts share a SIMD instead of three (1024 rows of 128001: 63 us; four 72, five 64, seven, with registers spilled, 71).
template <typename T, int E> struct UnitLogits;
template <int E> struct UnitLogits<float, E> {
  float v[E];
  __device__ __forceinline__ void load(const float* x, const int e0, const int i, const int n) {
    if (i + 8 <= n) {
      f32x4 u[2];
      __builtin_memcpy(u, x + i, 32);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e0 + e] = u[e >> 2][e & 3];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e0 + e] = i + e < n ? x[i + e] : -INFINITY;
    }
  }
  __device__ __forceinline__ float operator[](int e) const { return v[e]; }
  __device__ __forceinline__ void next_pass() {}
  __device__ __forceinline__ void store_quarter(float* to, const int q) const {
#pragma unroll
    for (int e = 0; e < E / 4; e += 4) *reinterpret_cast<f32x4*>(to + e) = f32x4{v[q * E / 4 + e], v[q * E / 4 + e + 1], v[q * E / 4 + e + 2], v[q * E / 4 + e + 3]};
  }
};
template <int E> struct UnitLogits<bf16_t, E> {
  uint32_t v[E / 2];
  __device__ __forceinline__ void load(const bf16_t* x, const int e0, const int i, const int n) {
    if (i + 8 <= n) {
      u32x4 u;
      __builtin_memcpy(&u, x + i, 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e0 / 2 + e] = u[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e0 / 2 + e] = (i + 2 * e < n ? x[i + 2 * e] : 0xff80u) | ((uint32_t)(i + 2 * e + 1 < n ? x[i + 2 * e + 1] : 0xff80u) << 16);
    }
  }
  __device__ __forceinline__ float operator[](int e) const { return __uint_as_float((e & 1) ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16); }
  __device__ __forceinline__ void store_quarter(bf16_t* to, const int q) const {
#pragma unroll
    for (int e = 0; e < E / 4; e += 4) *reinterpret_cast<uint2*>(to + e) = make_uint2(v[(q * E / 4 + e) / 2], v[(q * E / 4 + e) / 2 + 1]);
  }
  __device__ __forceinline__ void next_pass() {                 // what was unpacked is forgotten
#pragma unroll
    for (int e = 0; e < E / 2; ++e) asm volatile("" : "+v"(v[e]));
  }
};

template <typename T, int E>
__global__ __launch_bounds__(256, E == 64 ? (sizeof(T) == 2 ? 6 : 3) : 8) void k_beam_units(BeamSelectArgs a) {
  constexpr int Q = E / 4;
  __shared__ unsigned long long lists[4][BEAM_LIST];
  __shared__ __align__(16) T staged[4][BEAM_STAGE * Q];
  __shared__ unsigned char staged_from[4][BEAM_STAGE];          // quarter * 64 + lane
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int id = blockIdx.x * 4 + w;
  if (id >= a.n_groups * a.n_beams * a.units) return;
  const int row = id / a.units, first = (id - row * a.units) * 64 * E;
  const T* x = static_cast<const T*>(a.logits) + (size_t)row * a.ld;
  UnitLogits<T, E> v;
#pragma unroll
  for (int e = 0; e < E; e += 8) v.load(x, e, first + e * 64 + lane * 8, a.vocab);
  // maxima of a quarter of the lane's values each (a NaN stays out of them, and shows in the sum)
  uint32_t m[4];
  float mx = -INFINITY;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float y = v[q * E / 4];
#pragma unroll
    for (int e = 1; e < E / 4; ++e) y = fmaxf(y, v[q * E / 4 + e]);
    y = fmaxf(y, -INFINITY);
    m[q] = y > -INFINITY ? f32_key(y + 0.f) : 0u;
    mx = fmaxf(mx, y);
  }
  mx = key_f32(wave_max_u32(f32_key(mx)));
  const float m_use = mx == -INFINITY ? 0.f : mx;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  v.next_pass();
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e & 3] += __builtin_amdgcn_exp2f((v[e] - m_use) * LOG2E);
  const float total = wave_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
  if (lane == 0) a.stats[id] = make_float2(mx, total);
  // entries: logits of at least `least` (compared as numbers: a NaN reaches nothing), those equal to `edge` up to index `upto`
  const uint32_t bound = kth_bound(m, a.k);
  float least = bound == 0 ? -3.402823466e38f : key_f32(bound), edge = NAN;
  int upto = 0;
  const int at0 = first + lane * 8;                             // index of e: at0 + 64 (e & ~7) + (e & 7)
  // Only quarters whose maximum reaches the bound hold entries, about k of the 256: those go to LDS, and a pass over what is there takes the place
  // of one over every register (1024 rows of 128001: 63 us against 68).
  int n_staged = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) n_staged += __popcll(__ballot(m[q] >= max(bound, 1u)));
  const bool stage = n_staged <= BEAM_STAGE;
  if (stage) {
    int n = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const bool mine = m[q] >= max(bound, 1u);
      const unsigned long long hit = __ballot(mine);
      if (mine) {
        const int slot = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(hit >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hit, 0));
        v.store_quarter(&staged[w][slot * Q], q);
        staged_from[w][slot] = (unsigned char)(q * 64 + lane);
      }
      n += __popcll(hit);
    }
    wave_lds_fence();
  }
  wave_top_k([&](auto f) {
    if (stage) {
      for (int i0 = 0; i0 < n_staged * Q; i0 += 64) {
        const int i = i0 + lane;
        const bool in = i < n_staged * Q;
        const int from = in ? staged_from[w][i / Q] : 0, e = (from >> 6) * Q + i % Q, at = first + (from & 63) * 8 + (e & ~7) * 64 + (e & 7);
        const float y = in ? logit(&staged[w][i]) : -INFINITY;
        f(y >= least && !(y == edge && at > upto), [&]() { return ((unsigned long long)__float_as_uint(y) << 32) | (uint32_t)at; });
      }
      return;
    }
    v.next_pass();
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int off = (e & ~7) * 64 + (e & 7);
      f(v[e] >= least && !(v[e] == edge && at0 > upto - off),
        [&]() {
          int at = at0;
          asm volatile("" : "+v"(at));                          // (left to itself the compiler keeps 64 sums in registers for the few that are needed)
          return ((unsigned long long)__float_as_uint(v[e]) << 32) | (uint32_t)(at + off);
        });
    }
  }, [&]() {
    uint32_t cur = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const float t = key_f32(cur | (1u << bit));               // (no number: nothing reaches it)
      int c = 0;
      v.next_pass();
#pragma unroll
      for (int e = 0; e < E; ++e) c += __popcll(__ballot(v[e] >= t));
      if (c >= a.k) cur |= 1u << bit;
    }
    least = edge = key_f32(cur);
    int above = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) above += __popcll(__ballot(v[e] > edge));
    int lo = first, hi = first + 64 * E - 1;                    // the lowest index up to which enough are equal
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      int c = above;
      v.next_pass();
#pragma unroll
      for (int e = 0; e < E; ++e) c += __popcll(__ballot(v[e] == edge && at0 <= mid - ((e & ~7) * 64 + (e & 7))));
      if (c >= a.k) hi = mid; else lo = mid + 1;
    }
    upto = lo;
  }, [&](unsigned long long r) {                                // (+ 0: zeros of both signs are equal)
    return ((unsigned long long)f32_key(__uint_as_float((uint32_t)(r >> 32)) + 0.f) << 32) | (uint32_t)~(uint32_t)r;
  }, a.k, lists[w], a.cand + (size_t)id * a.k);
}

struct BeamCand { double s; int token; int rank; };   // of one row; equal keys by the lower token

// LDS: candidates [beam][k], keys [wavefront][k], lists [wavefront][BEAM_LIST].  Workgroup of a wavefront per row, up to sixteen.  LONG: the units'
// candidates of a row are more than the registers hold (1024).
template <bool LONG>
__global__ __launch_bounds__(1024) void k_beam_merge(BeamSelectArgs a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ int s_bad;
  __shared__ int s_n[DISCO_BEAM_MAX_ROWS], s_cut[DISCO_BEAM_MAX_ROWS];         // candidates of a row, and those that can be wanted
  const int g = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6, nw = blockDim.x >> 6, k = a.k;
  const float per_unit = 1.0f / (float)a.units;
  BeamCand* cand = reinterpret_cast<BeamCand*>(smem);
  unsigned long long* keys = reinterpret_cast<unsigned long long*>(cand + a.n_beams * k) + w * k;
  unsigned long long* list = reinterpret_cast<unsigned long long*>(cand + a.n_beams * k) + nw * k + w * BEAM_LIST;
  auto part = [](const int i, const float by) { return (int)(((float)i + 0.5f) * by); };    // i / n for i up to 2^19 and quotients up to 1024: off by less than 0.5 / n
  if (t == 0) s_bad = 0;
  __syncthreads();
  for (int b = w; b < a.n_beams; b += nw) {
    const int row = g * a.n_beams + b, total = a.units * k;
    // What the row needs is requested together: candidates (LONG: the best of every unit, next to each other so that the 256 maxima below are those
    // of the best few), statistics, score.
    const unsigned long long* src = a.cand + (size_t)row * a.units * k;
    unsigned long long r[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int i = e * 64 + lane;
      if constexpr (LONG) {
        const int pos = part(i, per_unit);
        r[e] = pos < 64 * 16 / a.units ? src[(i - pos * a.units) * k + pos] : 0ull;
      } else {
        r[e] = i < total ? src[i] : 0ull;
      }
    }
    const float2* st = a.stats + (size_t)row * a.units;
    const float2 mine = lane < a.units ? st[lane] : make_float2(-INFINITY, 0.f);
    const float score = a.scores[row];
    bool bad = !(score < INFINITY);
    int n = 0;
    if (a.done != nullptr && a.done[row] != 0) {
      n = score > -INFINITY ? 1 : 0;
      if (lane == 0) cand[b * k] = BeamCand{(double)score, a.end_token, 0};
    } else {
      float m = mine.x;
      for (int c = lane + 64; c < a.units; c += 64) m = fmaxf(m, st[c].x);
      m = key_f32(wave_max_u32(f32_key(m)));
      double sum = 0.0;
      for (int c = lane; c < a.units; c += 64) {
        const float2 s = c == lane ? mine : st[c];
        bad |= !(s.y < INFINITY);
        if (s.x > -INFINITY) sum += (double)s.y * exp((double)s.x - (double)m);
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
      bad = __any(bad);
      const double off = (double)score - ((double)m + log(sum));
      if (!bad && score > -INFINITY && m > -INFINITY) {
        uint32_t q[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 16; ++e) q[e & 3] = max(q[e & 3], (uint32_t)(r[e] >> 32));
        const uint32_t bound = kth_bound(q, k);
        bool deep = false;                                      // the last of a unit's in registers reaches the bound: there may be more behind it
        if constexpr (LONG) {
          const int last = 64 * 16 / a.units - 1;
#pragma unroll
          for (int e = 0; e < 16; ++e) deep |= (uint32_t)(r[e] >> 32) >= max(bound, 1u) && part(e * 64 + lane, per_unit) == last;
          deep = __any(deep);
        }
        if (LONG && deep) wave_top_k_memory(src, total, bound, k, list, keys);
        else wave_top_k_keys(r, bound, k, list, keys);
        wave_lds_fence();
        for (int i = lane; i < k; i += 64) {
          const unsigned long long key = keys[i];
          if (key != 0) cand[b * k + i] = BeamCand{off + (double)key_f32((uint32_t)(key >> 32)), (int)~(uint32_t)key, 0};
          n += __popcll(__ballot(key != 0));
        }
        n = __builtin_amdgcn_readfirstlane(n);
      }
    }
    if (lane == 0) { s_n[b] = n; if (bad) s_bad = 1; }
  }
  __syncthreads();
  const bool bad = s_bad != 0;
  int have = 0;
  for (int b = 0; b < a.n_beams; ++b) have += s_n[b];
  // Rank of a candidate: its place in its own row's list and, counted row by row, the better ones of the others (lists in order).  LONG: every eighth of
  // a list first, behind one that has k better ones no other is wanted; neighbouring lanes take the same place of different rows, so that places that
  // are not wanted are skipped by whole wavefronts (32 beams of 64 candidates: 12 us less; four beams of four: 0.1 us more).
  const int n_all = a.n_beams * k;
  const float per_beam = 1.0f / (float)k, per_row = 1.0f / (float)a.n_beams;
  for (int i = t; i < n_all; i += blockDim.x) cand[i].rank = i - part(i, per_beam) * k;
  for (int b = t; b < a.n_beams; b += blockDim.x) s_cut[b] = s_n[b];
  __syncthreads();
  auto count = [&](const int step, const bool rest) {
    const int n_p = (k + step - 1) / step, n_set = n_p * a.n_beams;
    const float per_set = 1.0f / (float)n_set;
    for (int i = t; i < n_set * a.n_beams; i += blockDim.x) {
      const int o = part(i, per_set), x = i - o * n_set;
      int b, p;
      if constexpr (LONG) { const int place = part(x, per_row); b = x - place * a.n_beams; p = place * step; }
      else { b = part(x, per_beam); p = x - b * k; }
      if (o == b || p >= s_cut[b] || (rest && (p & 7) == 0)) continue;
      const int c = b * k + p;
      const double mine = cand[c].s;
      int lo = 0, hi = s_n[o];
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const double y = cand[o * k + mid].s;
        if (y > mine || (y == mine && o < b)) lo = mid + 1; else hi = mid;
      }
      if (lo > 0) atomicAdd(&cand[c].rank, lo);
    }
    __syncthreads();
  };
  if (!bad) {
    if constexpr (LONG) {
      count(8, false);
      for (int i = t; i < n_all; i += blockDim.x) {
        const int b = part(i, per_beam), p = i - b * k;
        if ((p & 7) == 0 && p < s_n[b] && cand[i].rank >= k) atomicMin(&s_cut[b], p);
      }
      __syncthreads();
    }
    count(1, LONG);
  }
  for (int i = t; i < n_all; i += blockDim.x) {
    const int b = part(i, per_beam);
    const BeamCand c = cand[i];
    if (bad || i - b * k >= s_cut[b] || c.rank >= k) continue;
    const size_t at = (size_t)g * k + c.rank;
    a.tokens[at] = c.token; a.parents[at] = b; a.scores_out[at] = (float)c.s;
    if (a.done_out != nullptr) a.done_out[at] = (a.done != nullptr && a.done[g * a.n_beams + b] != 0) || c.token == a.end_token ? 1 : 0;
  }
  for (int i = (bad ? 0 : have) + t; i < k; i += blockDim.x) {
    const size_t at = (size_t)g * k + i;
    a.tokens[at] = -1; a.parents[at] = -1; a.scores_out[at] = bad ? NAN : -INFINITY;
    if (a.done_out != nullptr) a.done_out[at] = 1;
  }
}

// ---------------------------------------------------------------------------------------------
// reordering
// ---------------------------------------------------------------------------------------------

// Sequence b of a group goes on from sequence parents[b].  Pages that are full are shared by reference; of the one being filled
// the first child takes its parent's, further children get those of sequences without a child, with the contents copied.
// Workgroups: `pieces` of every copied page of every layer (a sequence that needs no copy ends at once), then one for the group's tables.
// Bound by the copies: 16 bytes a lane, four at a time (48 pages of 16 positions of 8 heads of 128 in 16 layers, 101 MB: 23 us, 4.3 TB/s; 40 layers of one beam's page of
// 40 heads, 26 MB: 8.7 us).
__global__ __launch_bounds__(256) void k_beam_reorder(BeamReorderArgs a, int pieces) {
  __shared__ int s_par[64], s_dst[64], s_src[64], s_of[64], s_n;
  const int nb = a.n_beams, t = threadIdx.x, g = blockIdx.y;
  const int32_t* old = a.tables + (size_t)g * nb * a.table_ld;
  if (t < 64) {
    int p = t < nb ? a.parents[(size_t)g * nb + t] : -1;
    if (t < nb && (unsigned)p >= (unsigned)nb) p = t;
    s_par[t] = p;
    const int mine = t < nb && a.live ? old[(size_t)t * a.table_ld + a.full] : 0;     // the page being filled
    // (one wavefront: every lane sees all parents)
    bool further = false, childless = t < nb;
    for (int j = 0; j < nb; ++j) {
      const int pj = __builtin_amdgcn_readlane(p, j);
      further |= j < t && pj == p;
      childless &= pj != t;
    }
    further &= t < nb;
    const unsigned long long fm = __ballot(further), em = __ballot(childless);
    const int rank = __popcll(fm & ((1ull << t) - 1));
    unsigned long long rest = em;                               // the rank-th sequence without a child
    for (int j = 0; j < rank; ++j) rest &= rest - 1;
    const int src = __shfl(mine, p < 0 ? 0 : p), dst = __shfl(mine, further ? __ffsll(rest) - 1 : (p < 0 ? 0 : p));   // (all lanes active)
    s_dst[t] = dst;
    s_src[t] = src;
    if (further) s_of[rank] = t;
    if (t == 0) s_n = __popcll(fm);
  }
  __syncthreads();
  const int unit = blockIdx.x, n_units = (int)gridDim.x - 1;
  if (unit < n_units) {
    // unit = (layer, copied page, piece)
    const int per_layer = (nb - 1) * pieces;                    // (at most n_beams - 1 pages are copied)
    const int layer = unit / per_layer, k = unit % per_layer / pieces, piece = unit % pieces;
    if (k >= s_n) return;
    const int b = s_of[k], src = s_src[b], dst = s_dst[b];
    if ((unsigned)src >= (unsigned)a.n_pages || (unsigned)dst >= (unsigned)a.n_pages) return;
    bf16_t* pages = a.pages + (size_t)layer * a.layer_stride;
    const u32x4* from = reinterpret_cast<const u32x4*>(pages + (size_t)src * a.page_elems);
    u32x4* to = reinterpret_cast<u32x4*>(pages + (size_t)dst * a.page_elems);
    const int64_t n = a.page_elems / 8, share = (n + pieces - 1) / pieces, end = min(n, share * (piece + 1));
    for (int64_t i = share * piece + t; i < end; i += 1024) {
      u32x4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) if (i + 256 * u < end) x[u] = from[i + 256 * u];
#pragma unroll
      for (int u = 0; u < 4; ++u) if (i + 256 * u < end) to[i + 256 * u] = x[u];
    }
  } else {                                                      // the tables
    for (int i = t; i < nb * a.table_ld; i += 256) {
      const int b = i / a.table_ld, c = i % a.table_ld;
      int32_t v;
      if (c < a.full) v = old[(size_t)s_par[b] * a.table_ld + c];
      else if (c == a.full && a.live) v = s_dst[b];
      else v = old[(size_t)b * a.table_ld + c];
      a.tables_out[((size_t)g * nb + b) * a.table_ld + c] = v;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// embedding of a step
// ---------------------------------------------------------------------------------------------

// Token of every sequence, all at one position: residual row, its sum of squares (and sum, for a LayerNorm) in the first slot, and the panels of
// gain * row.  A workgroup a row.
__global__ __launch_bounds__(256) void k_beam_embed(BeamEmbedArgs a) {
  __shared__ float red[2][4];
  const int m = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int tok = min(max(a.tokens[m], 0), a.vocab - 1);
  const bf16_t* e = a.tok_emb + (size_t)tok * a.tok_stride;
  float ss = 0.f, sx = 0.f;
  for (int k = t * 4; k < a.d; k += 1024) {
    float4 v = load4(e + k);
    if (a.pos_row != nullptr) { const float4 p = load4(a.pos_row + k); v = make_float4(v.x + p.x, v.y + p.y, v.z + p.z, v.w + p.w); }
    store4(a.h + (size_t)m * a.d + k, v);
    ss += (v.x * v.x + v.y * v.y) + (v.z * v.z + v.w * v.w);
    sx += (v.x + v.y) + (v.z + v.w);
    const float4 g = load4(a.gain + k);
    const float o[4] = {v.x * g.x, v.y * g.y, v.z * g.z, v.w * g.w};
    xpack_store4(a.panels, a.d >> 5, a.rows, m, k, o);
  }
  ss = wave_sum(ss); sx = wave_sum(sx);
  if (lane == 0) { red[0][w] = ss; red[1][w] = sx; }
  __syncthreads();
  for (int i = t; i < a.n_slots; i += 256) {
    a.ssq[i * 16 + m] = i == 0 ? (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]) : 0.f;
    if (a.sum != nullptr) a.sum[i * 16 + m] = i == 0 ? (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]) : 0.f;
  }
}

}  // namespace

hipError_t launch_beam_embed(const BeamEmbedArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_beam_embed, dim3((unsigned)a.rows), dim3(256), 0, s, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------------

// Calls whose rows can be runs (several tokens of a sequence) and whose values are worth 128 workgroups take four heads a workgroup and value
// tiles: 5999 rows of 40 heads of their own 86 us against 150 with a head a workgroup and values written one by one; 192 rows of one token
// 5.9 against 6.5, four rows 2.8 against 3.5 the other way round.
template <int DH, typename T>
static hipError_t launch_append_of(const AppendArgs& a, hipStream_t s) {
  const int value_blocks = (a.rows + APPEND_RV - 1) / APPEND_RV;
  auto row_blocks = [&](int piece) { const int rpw = 256 / (DH / 2 / piece); return (a.rows + rpw - 1) / rpw; };
  if ((a.seq != nullptr || a.n_tok >= 4) && (long)value_blocks * a.kv.nkv >= 128) {
    const int groups = (a.nq + a.kv.nkv + 3) / 4, n = row_blocks(append_piece<T, 4>) * groups;
    const dim3 grid((unsigned)(n + value_blocks * a.kv.nkv));
    if ((a.kv.pt & 7) == 0) hipLaunchKernelGGL((k_append<DH, T, 4, 8>), grid, dim3(256), 0, s, a, n, groups, value_blocks);
    else hipLaunchKernelGGL((k_append<DH, T, 4, 4>), grid, dim3(256), 0, s, a, n, groups, value_blocks);
  } else {
    const int groups = a.nq + 2 * a.kv.nkv, n = row_blocks(append_piece<T, 1>) * groups;
    hipLaunchKernelGGL((k_append<DH, T, 1, 8>), dim3((unsigned)n), dim3(256), 0, s, a, n, groups, 0);
  }
  return hipGetLastError();
}
hipError_t launch_append(const AppendArgs& a, bool fp32, hipStream_t s) {
  if (a.kv.dh == 128) return fp32 ? launch_append_of<128, float>(a, s) : launch_append_of<128, bf16_t>(a, s);
  return fp32 ? launch_append_of<64, float>(a, s) : launch_append_of<64, bf16_t>(a, s);
}

// Which rows share a workgroup, and how the positions are cut into ranges.  Up to 32 rows a K / V head (or a sequence) has: workgroups of that
// many rows and two wavefronts, ranges of at least 128 positions, as many as give every compute unit one workgroup (eight beams of 40 heads, 2048
// positions: 256 wanted 20 us, 512 21, 1024 25; four wavefronts 23, one 25), and two of own positions, whose lengths differ (32 sequences of 8 K / V
// heads with up to 700 own positions: 37 us with one, 33 with two; eight with up to 4000: 29 and 24).  More rows: 128 a workgroup, ranges of at least 256 positions for
// two workgroups a compute unit (one where registers allow no more), but one where a range would then have no more than 512 positions: what is
// gained is less than what the additional parts cost (4608 rows over 3001 positions: 28 us with one, 32 with two; 384 over 65537: 245 and 193).
// A prompt and own positions that four wavefronts walk in two steps take one launch, every sequence reading the prompt by itself: 100 + 20
// positions of 12 heads 7.9 us against 9.9, but 523 + 37 for four sequences 13.2 against 10.4.  Such workgroups have four wavefronts where two fit
// every compute unit, and all have one where they are more than four for each: 71 sequences of 40 heads, 3 positions: 30 us with one, 46 with two, 84
// with four; 32 of 40 heads, 300 + 100 positions: 32 and 38 with one and two, but 8 of them with 2048 + 130: 25 and 20.
SharedAttnPlan shared_attn_plan(int n_seqs, int n_tok, int nq, int nkv, int dh, bool fp32, int prefix_len, int max_len) {
  SharedAttnPlan p{};
  const long grp = nq / nkv, own_rows = n_tok * grp, rows = n_seqs * own_rows;
  auto ranges = [&](bool many, long few_wanted, long tiles, int len, int* splits, int* range) {
    const int least = many ? 256 : 128;
    auto cut = [&](long want) {
      long n = want / tiles;
      const long most = ((long)len + least - 1) / least;
      n = n > most ? most : n;
      return n < 1 ? 1 : (n > ATTN_MAX_PARTS / 2 ? ATTN_MAX_PARTS / 2 : n);
    };
    long n = cut(many ? 256 : few_wanted);
    if (many && !(fp32 && dh == 128) && len > 512 * n) n = cut(512);
    long r = (len + n - 1) / n;
    r = (r + 63) / 64 * 64;
    if (r < 64) r = 64;
    *range = (int)r;
    *splits = (int)((len + r - 1) / r);
    if (*splits < 1) *splits = 1;
  };
  p.own_many = own_rows > 32;
  p.own_tiles = p.own_many ? (int)((own_rows + 127) / 128) : 1;
  p.fused = prefix_len > 0 && !p.own_many && (long)prefix_len + max_len <= 256;
  if (p.fused) {
    p.own_splits = 1; p.own_len = max_len;
  } else {
    if (prefix_len > 0) {
      p.prefix_many = rows > 32;
      p.prefix_tiles = p.prefix_many ? (int)((rows + 127) / 128) : 1;
      ranges(p.prefix_many, 256, (long)p.prefix_tiles * nkv, prefix_len, &p.prefix_splits, &p.prefix_len);
    }
    ranges(p.own_many, 512, (long)p.own_tiles * nkv * n_seqs, max_len, &p.own_splits, &p.own_len);
  }
  const long few = (p.own_many ? 0 : (long)n_seqs * nkv * p.own_splits) + (p.prefix_many ? 0 : (long)p.prefix_tiles * nkv * p.prefix_splits);
  p.few_waves = few > 1024 ? 1 : (p.fused && few <= 512 ? 4 : 2);
  p.few_rows = (p.prefix_tiles > 0 && !p.prefix_many ? rows : own_rows) <= 16 ? 16 : 32;
  p.parts = p.prefix_splits + p.own_splits;
  if (p.parts > 1) p.bytes = (size_t)p.parts * rows * nkv * (dh * sizeof(float) + sizeof(float2));
  return p;
}

template <int DH, bool F32>
static hipError_t launch_attn_all(const SharedAttnArgs& a, hipStream_t s) {
  const SharedAttnPlan& p = a.plan;
  const unsigned n_prefix = (unsigned)(p.prefix_tiles * p.prefix_splits * a.kv.nkv), n_own = (unsigned)(a.kv.n_seqs * p.own_tiles * p.own_splits * a.kv.nkv);
  auto launch = [&](bool many, unsigned n, int prefix) {
    if (many) hipLaunchKernelGGL((k_attn_many<DH, F32>), dim3(n), dim3(256), 0, s, a, prefix);
    else if (p.few_rows == 16 && p.few_waves == 1) hipLaunchKernelGGL((k_attn_few<DH, 16, 1, F32>), dim3(n), dim3(64), 0, s, a, prefix);
    else if (p.few_rows == 16 && p.few_waves == 2) hipLaunchKernelGGL((k_attn_few<DH, 16, 2, F32>), dim3(n), dim3(128), 0, s, a, prefix);
    else if (p.few_rows == 16) hipLaunchKernelGGL((k_attn_few<DH, 16, 4, F32>), dim3(n), dim3(256), 0, s, a, prefix);
    else if (p.few_waves == 1) hipLaunchKernelGGL((k_attn_few<DH, 32, 1, F32>), dim3(n), dim3(64), 0, s, a, prefix);
    else if (p.few_waves == 2) hipLaunchKernelGGL((k_attn_few<DH, 32, 2, F32>), dim3(n), dim3(128), 0, s, a, prefix);
    else hipLaunchKernelGGL((k_attn_few<DH, 32, 4, F32>), dim3(n), dim3(256), 0, s, a, prefix);
    return hipGetLastError();
  };
  hipError_t e;
  if (n_prefix == 0 || p.prefix_many == p.own_many) {
    e = launch(p.own_many, n_prefix + n_own, (int)n_prefix);
  } else {
    e = launch(p.prefix_many, n_prefix, (int)n_prefix);
    if (e == hipSuccess) e = launch(p.own_many, n_own, 0);
  }
  if (e != hipSuccess || p.parts == 1) return e;
  const size_t rows = (size_t)a.kv.n_seqs * a.n_tok * a.nq;
  constexpr int rpw = 256 / (DH / 4);
  hipLaunchKernelGGL((k_shared_merge<DH, F32>), dim3((unsigned)((rows + rpw - 1) / rpw)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_shared_attn(const SharedAttnArgs& a, bool fp32, hipStream_t s) {
  if (a.kv.dh == 128) return fp32 ? launch_attn_all<128, true>(a, s) : launch_attn_all<128, false>(a, s);
  return fp32 ? launch_attn_all<64, true>(a, s) : launch_attn_all<64, false>(a, s);
}

// Logits of a lane: 64 where that leaves every SIMD two wavefronts, else 16.
int beam_unit_logits(int rows, int vocab) { return 64 * ((long)rows * ((vocab + 4095) / 4096) >= 2048 ? 64 : 16); }

hipError_t launch_beam_select(const BeamSelectArgs& a, bool fp32, hipStream_t s) {
  const dim3 grid((unsigned)(((long)a.n_groups * a.n_beams * a.units + 3) / 4));
  const bool wide = beam_unit_logits(a.n_groups * a.n_beams, a.vocab) == 64 * 64;
  if (fp32 && wide) hipLaunchKernelGGL((k_beam_units<float, 64>), grid, dim3(256), 0, s, a);
  else if (fp32) hipLaunchKernelGGL((k_beam_units<float, 16>), grid, dim3(256), 0, s, a);
  else if (wide) hipLaunchKernelGGL((k_beam_units<bf16_t, 64>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_beam_units<bf16_t, 16>), grid, dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  int nw = a.n_beams < 16 ? a.n_beams : 16;
  auto lds_bytes = [&]() { return sizeof(BeamCand) * a.n_beams * a.k + sizeof(unsigned long long) * nw * (a.k + BEAM_LIST); };
  while (nw > 4 && lds_bytes() > (size_t)150 << 10) nw /= 2;    // 64 beams of 128: 128 KiB for the candidates
  const size_t lds = lds_bytes();
  if (a.units * a.k <= 64 * 16) hipLaunchKernelGGL(k_beam_merge<false>, dim3((unsigned)a.n_groups), dim3(64 * nw), lds, s, a);
  else hipLaunchKernelGGL(k_beam_merge<true>, dim3((unsigned)a.n_groups), dim3(64 * nw), lds, s, a);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(const BeamReorderArgs& a, hipStream_t s) {
  // pieces of 64 KiB and more: sixteen loads a lane
  const int pieces = (int)((a.page_elems * 2 + (64 << 10) - 1) >> 16);
  const long units = a.live ? (long)a.n_layers * (a.n_beams - 1) * pieces : 0;
  hipLaunchKernelGGL(k_beam_reorder, dim3((unsigned)(units + 1), (unsigned)a.n_groups), dim3(256), 0, s, a, pieces);
  return hipGetLastError();
}

}  // namespace disco
