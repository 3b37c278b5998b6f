// The paged cache: rows appended with the rotation on the way, and the scores that select pages.
#include <cuda_bf16.h>
#include <limits.h>

#include "rkv_internal.h"
#include "rkv_pick.cuh"
#include "rkv_ptx.cuh"
#include "rkv_rows.cuh"

namespace rkv {
namespace {

// ----------------------------------------------------------------------------------------------------------- append
// Rows of the fused projection become queries [token][head] and keys and values in their pages, queries and keys turned by
// their positions (the angle as in rkv_rope.cu: turns as 64-bit fixed point), and the keys' bounds follow.
//
// HBM-bound for prompts: every channel is read once and written once.  A CTA takes the new rows of kUnit positions (or of
// one page, where that is more) for 8 or more heads, of queries or of keys and values.  Eight threads share a row, each with two
// pieces of eight channels (eight pairs, or channels that are only copied).  Keys and values: a warp takes one head at a time
// over all of those rows, so that a page's bounds stay in the warp's registers until the page ends, and no two CTAs meet at a page
// and head; it works through batches of 16 rows, four of a thread's, all of them requested before the first is used.  Queries: four
// rows to a warp, of which eight threads go through the heads, four at a time.  Sines and cosines of the unit's (row, pair)s
// are worked out once per CTA, in shared memory, each from its own angle, so that rows are those of rkv_rope to the last bit (from the
// angles of every eighth position and of 0 .. 7 positions, by the sum's formula: the prompt 139 us, 16 rows 4.9 instead of 4.2, and 2^-22 off instead of 2^-23).
// With up to kFewRows rows a sequence (tokens of a decode step) eight threads take a head, and a CTA 32 of them.
// Measured (32 + 16 heads): a prompt of 32768 bf16 rows 135 us, 6.0 TB/s (rows requested one by one as others are done with 215, two
// batches in turn 153, three or four CTAs to an SM, which spill, 158 to 231, 512 threads 144); one row 3.1 us.
// Few rows here / in units: 1 row 3.1 / 4.1 us, 64 sequences of 1 row 3.1 / 7.8, of 4 rows 5.3 / 9.2, of 8 rows 8.1 / 9.4, but
// 1 sequence of 8 rows 6.6 / 4.0, of 16 rows 10.9 / 4.2, 64 of 16 rows 16.4 / 10.6.
// fp32 rows hold twice the registers in flight: 128 of them and 28 to 36 bytes spilled; a prompt of 16384 rows 104 us, 5.8 TB/s (interleaved pairs 130).
constexpr int kAppendThreads = 256, kAppendWarps = kAppendThreads / 32;
constexpr int kUnit = 64;                    // positions of a CTA
constexpr int kBatchRows = 16, kAhead = kBatchRows / 4;      // rows of a warp in flight, and of a thread
constexpr int kFewRows = 4;
constexpr int kAppendSpread = 6;
constexpr int kCsRow = kHeadDim / 2 + 8;     // (the four rows of a warp beside each other in the banks)
static_assert(kUnit % kBatchRows == 0, "whole batches");

struct AppendShared {
  float2 cs[kUnit][kCsRow];                  // pair 8 i + j of a row at 8 j + i: the eight threads of a row read side by side
  int sizes[3];
  int page[kUnit / 16];
};

struct NewRows { int start, count; };

// One thread reads the sizes for its CTA; behind the barrier it draws a ticket, the last of which writes the new length:
// a ticket says that nobody in its CTA will read the sizes again.
__device__ __forceinline__ NewRows append_sizes(const PagedAppendParams& p, AppendShared& sm, int b, int tid) {
  if (tid == 0) {
    const int l = __ldcg(p.c.len + b);
    sm.sizes[0] = l;
    sm.sizes[1] = p.start != nullptr ? __ldcg(p.start + b) : l;
    sm.sizes[2] = p.count != nullptr ? __ldcg(p.count + b) : p.n_tok;
  }
  __syncthreads();
  int ticket = -1;
  if (tid == 0) ticket = atomicAdd(p.tickets + b, 1);
  NewRows n;
  n.start = sm.sizes[1];
  n.count = min(max(sm.sizes[2], 0), p.n_tok);
  const int64_t room = min((int64_t)p.c.table_stride << p.c.page_shift, (int64_t)INT_MAX);   // (lengths are 32 bits)
  const bool sound = n.start >= 0 && n.start <= sm.sizes[0] && n.start <= room;
  int flags = 0;
  if (!sound) {
    flags = RKV_DEV_LEN_CLAMPED;
    n.count = 0;
  } else if (n.count > room - n.start) {
    flags = RKV_DEV_APPEND_OVERFLOW;
    n.count = (int)(room - n.start);
  }
  if (tid == 0) {
    if (ticket == (int)(gridDim.x * gridDim.y) - 1) {
      if (sound) p.c.len[b] = n.start + n.count;
      p.tickets[b] = 0;   // ready for the next call on this stream
    }
    if (flags != 0 && blockIdx.x == 0 && blockIdx.y == 0) atomicOr(p.status, flags);
  }
  return n;
}

// (cos, sin) of a position's angle, as rkv_rope forms them.
__device__ __forceinline__ float2 angle(int64_t pos, unsigned long long freq) {
  float s, c;
  sincospif((float)(int)(((unsigned long long)pos * freq) >> 32) * 4.656612873e-10f, &s, &c);   // 2^-31: half turns
  return make_float2(c, s);
}

// Pages and angles of the rows of positions lo .. hi - 1, which lie in the unit (or the half of a page of 128) that begins at
// s0; row r of it at sm.cs[r].
template <bool kFew>
__device__ __forceinline__ void append_part(const PagedAppendParams& p, AppendShared& sm, int b, int64_t s0, int64_t lo, int64_t hi,
                                            int tid) {
  const int most = min(1 << p.c.page_shift, kUnit);       // positions of a page in this part
  if (tid < kUnit / most) {
    const int64_t at = s0 + tid * most;
    int pg = -1;
    if (at < hi && at + most > lo) {
      pg = __ldcg(p.c.table + (int64_t)b * p.c.table_stride + (at >> p.c.page_shift));
      if ((unsigned)pg >= (unsigned)p.c.n_pages) {
        pg = -1;
        if (blockIdx.y == 0) atomicOr(p.status, RKV_DEV_BAD_INDEX);
      }
    }
    sm.page[tid] = pg;
  }
  const int half = p.rot >> 1, r0 = (int)(lo - s0), n = (int)(hi - lo);
  auto put = [&](int r, int j, unsigned long long freq) {
    const float2 e = angle(s0 + r, freq);
    sm.cs[r][8 * (j & 7) + (j >> 3)] = make_float2(e.x * p.amp, e.y * p.amp);
  };
  if constexpr (kFew) {
    for (int i = tid; i < n * half; i += kAppendThreads) put(r0 + i / half, i % half, __ldg(p.freqs + i % half));
  } else {                                                 // a warp per row
    for (int j = tid & 31; j < half; j += 32) {
      const unsigned long long freq = __ldg(p.freqs + j);
      for (int r = r0 + (tid >> 5); r < r0 + n; r += kAppendWarps) put(r, j, freq);
    }
  }
}

// The eight pairs of a thread's two pieces.
template <bool kInterleaved>
__device__ __forceinline__ void turn_pieces(float (&a)[8], float (&w)[8], const float2 (&cs)[8]) {
  if (kInterleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 e = cs[j], f = cs[4 + j];
      const float x = a[2 * j], y = a[2 * j + 1], z = w[2 * j], u = w[2 * j + 1];
      a[2 * j] = x * e.x - y * e.y;
      a[2 * j + 1] = x * e.y + y * e.x;
      w[2 * j] = z * f.x - u * f.y;
      w[2 * j + 1] = z * f.y + u * f.x;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 e = cs[j];
      const float x = a[j], y = w[j];
      a[j] = x * e.x - y * e.y;
      w[j] = x * e.y + y * e.x;
    }
  }
}

// A page's bounds of one head leave, this thread's two pieces of them; joins: it keeps what it had.
__device__ __forceinline__ void store_bounds(const PagedAppendParams& p, Bounds8& ba, Bounds8& bb, int pg, int g, int ca, int cb,
                                             bool joins) {
  const int64_t at = ((int64_t)pg * p.c.n_kv_heads + g) * kHeadDim;
  uint4* lo4 = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.c.k_min) + at);
  uint4* hi4 = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.c.k_max) + at);
  if (joins) {
    ba.join(__ldcg(lo4 + ca / 8), __ldcg(hi4 + ca / 8));
    bb.join(__ldcg(lo4 + cb / 8), __ldcg(hi4 + cb / 8));
  }
  lo4[ca / 8] = ba.lo4();
  lo4[cb / 8] = bb.lo4();
  hi4[ca / 8] = ba.hi4();
  hi4[cb / 8] = bb.hi4();
}

struct Head {   // of the fused projection
  bool is_q, is_k;
  int g;
  __device__ __forceinline__ Head(const PagedAppendParams& p, int h) {
    is_q = h < p.n_q_heads;
    is_k = !is_q && h < p.n_q_heads + p.c.n_kv_heads;
    g = is_q ? h : h - p.n_q_heads - (is_k ? 0 : p.c.n_kv_heads);
  }
  // where the row of position pos (token t) goes; null: its page is not there
  __device__ __forceinline__ __nv_bfloat16* row(const PagedAppendParams& p, int b, int t, int64_t pos, int pg) const {
    if (is_q) return static_cast<__nv_bfloat16*>(p.q) + (((int64_t)b * p.n_tok + t) * p.n_q_heads + g) * kHeadDim;
    return in_page(p, pos, pg);
  }
  __device__ __forceinline__ __nv_bfloat16* in_page(const PagedAppendParams& p, int64_t pos, int pg) const {
    if (pg < 0) return nullptr;
    return static_cast<__nv_bfloat16*>(is_k ? p.c.k : p.c.v) +
           ((((int64_t)pg * p.c.n_kv_heads + g) << p.c.page_shift) + (pos & ((1 << p.c.page_shift) - 1))) * kHeadDim;
  }
};

template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(kAppendThreads, 2) paged_append_kernel(const PagedAppendParams p) {
  __shared__ AppendShared sm;
  const int b = blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int part = tid & 7, octet = lane >> 3;
  const int page = 1 << p.c.page_shift, unit = page > kUnit ? page : kUnit, most = page < kUnit ? page : kUnit;
  const bool turns = part < (p.rot >> 4);
  const int ca = (kInterleaved || !turns) ? 16 * part : 8 * part;          // this thread's pieces of a row
  const int cb = (kInterleaved || !turns) ? 16 * part + 8 : (p.rot >> 1) + 8 * part;
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  const NewRows nr = append_sizes(p, sm, b, tid);
  const int64_t end = (int64_t)nr.start + nr.count;
  const int64_t u0 = ((int64_t)nr.start / unit + blockIdx.x) * unit;       // the CTA's positions
  const int64_t first = u0 > nr.start ? u0 : nr.start, last = u0 + unit < end ? u0 + unit : end;
  if (nr.count <= 0 || first >= last) return;

  const int heads = p.n_q_heads + 2 * p.c.n_kv_heads, y_kv = (int)blockIdx.y - p.q_groups;   // < 0: queries
  const int h0 = p.n_q_heads + max(y_kv, 0) * p.rounds * kAppendWarps + warp;
  const int n_heads = min(p.rounds, (heads - h0 + kAppendWarps - 1) / kAppendWarps);   // of this warp: h0, h0 + 8, ...
  const T* rows = static_cast<const T*>(p.qkv) + (int64_t)b * p.seq_stride - (int64_t)nr.start * p.tok_stride;   // by position
  for (int64_t s0 = u0; s0 < last; s0 += kUnit) {       // (once, but for pages of 128)
    const int64_t lo = s0 > first ? s0 : first, hi = s0 + kUnit < last ? s0 + kUnit : last;
    if (lo >= hi) continue;
    const int r0 = (int)(lo - s0), r1 = (int)(hi - s0);   // rows of this part
    const int c0 = r0 / kBatchRows, c1 = (r1 + kBatchRows - 1) / kBatchRows;   // batches
    if (s0 != u0) __syncthreads();                       // (the sines of the half before are still in use)
    append_part<false>(p, sm, b, s0, lo, hi, tid);
    __syncthreads();
    const T* part_rows = rows + s0 * p.tok_stride;
    if (y_kv < 0) {   // queries: eight threads go through a row's heads
      const int q0 = (int)blockIdx.y * p.q_per, q1 = min(q0 + p.q_per, p.n_q_heads);
      for (int r = r0 + 4 * warp + octet; r < r1; r += 4 * kAppendWarps) {
        float2 cs[8];
        if (turns) {
#pragma unroll
          for (int j = 0; j < 8; ++j) cs[j] = sm.cs[r][part + 8 * j];
        }
        const T* x = part_rows + r * p.tok_stride;
        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.q) +
                            ((int64_t)b * p.n_tok + (s0 + r - nr.start)) * p.n_q_heads * kHeadDim;
        for (int h = q0; h < q1; h += kAhead) {
          Raw8<T> xa[kAhead], xb[kAhead];
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {   // (heads beyond the last are loaded in place of it, and not used)
            const int hh = min(h + i, q1 - 1);
            xa[i].load(x + hh * kHeadDim + ca);
            xb[i].load(x + hh * kHeadDim + cb);
          }
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {
            float a[8], w[8];
            xa[i].get(a);
            xb[i].get(w);
            if (turns) turn_pieces<kInterleaved>(a, w, cs);
            if (h + i < q1) {
              *reinterpret_cast<uint4*>(to + (h + i) * kHeadDim + ca) = pack8(a);
              *reinterpret_cast<uint4*>(to + (h + i) * kHeadDim + cb) = pack8(w);
            }
          }
        }
      }
      continue;
    }
    for (int round = 0; round < n_heads; ++round) {
      const int h = h0 + round * kAppendWarps;
      const Head head(p, h);
      const bool turn = turns && head.is_k, bounds = head.is_k && p.c.k_min != nullptr;
      const T* x = part_rows + h * kHeadDim;
      Bounds8 ba, bb;
      ba.reset();
      bb.reset();
      for (int c = c0; c < c1; ++c) {
        const int at = c * kBatchRows, pg = sm.page[at / most];
        // rows that are not new are loaded in place of others, and not used
        Raw8<T> xa[kAhead], xb[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int r = min(max(at + 4 * i + octet, r0), r1 - 1);
          xa[i].load(x + r * p.tok_stride + ca);
          xb[i].load(x + r * p.tok_stride + cb);
        }
        __nv_bfloat16* to = head.in_page(p, s0 + at + octet, pg);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int r = at + 4 * i + octet;
          const bool live = r >= r0 && r < r1;
          float a[8], w[8];
          xa[i].get(a);
          xb[i].get(w);
          if (turn) {
            float2 cs[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) cs[j] = sm.cs[r][part + 8 * j];
            turn_pieces<kInterleaved>(a, w, cs);
          }
          const uint4 pa = pack8(a), pb = pack8(w);
          if (live) {
            if (bounds) {
              ba.take(pa);
              bb.take(pb);
            }
            if (to != nullptr) {
              *reinterpret_cast<uint4*>(to + 4 * i * kHeadDim + ca) = pa;
              *reinterpret_cast<uint4*>(to + 4 * i * kHeadDim + cb) = pb;
            }
          }
        }
        // The page's last new row: its bounds leave.  A page whose first position is not among the new ones takes in the
        // bounds that it had; one of 128 positions whose first half this warp has just done, those.
        if (bounds && (c + 1 == c1 || (at + kBatchRows) % most == 0)) {
          __syncwarp();
          ba.over_octets();
          bb.over_octets();
          const int64_t begin = s0 + max(at / most * most, r0);           // the page's first new row here
          if (octet == 0 && pg >= 0) store_bounds(p, ba, bb, pg, head.g, ca, cb, (begin & (page - 1)) != 0);
          ba.reset();
          bb.reset();
        }
      }
    }
  }
}

template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(kAppendThreads) paged_append_few_kernel(const PagedAppendParams p) {
  __shared__ AppendShared sm;
  const int b = blockIdx.z, tid = threadIdx.x, part = tid & 7;
  const int page = 1 << p.c.page_shift, unit = page > kUnit ? page : kUnit, most = page < kUnit ? page : kUnit;
  const bool turns = part < (p.rot >> 4);
  const int ca = (kInterleaved || !turns) ? 16 * part : 8 * part;          // this thread's pieces of a row
  const int cb = (kInterleaved || !turns) ? 16 * part + 8 : (p.rot >> 1) + 8 * part;
  const int heads = p.n_q_heads + 2 * p.c.n_kv_heads, h = (int)blockIdx.y * (kAppendThreads / 8) + (tid >> 3);
  const T* rows = static_cast<const T*>(p.qkv) + (int64_t)b * p.seq_stride + h * kHeadDim;   // by token
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  Raw8<T> xa, xb;
  if (h < heads && blockIdx.x == 0) {       // the first token, on its way with the sizes
    xa.load(rows + ca);
    xb.load(rows + cb);
  }
  const NewRows nr = append_sizes(p, sm, b, tid);
  const int64_t end = (int64_t)nr.start + nr.count;
  const int64_t u0 = ((int64_t)nr.start / unit + blockIdx.x) * unit;       // the CTA's positions
  const int64_t first = u0 > nr.start ? u0 : nr.start, last = u0 + unit < end ? u0 + unit : end;
  if (nr.count <= 0 || first >= last) return;
  const Head head(p, h);
  const bool turn = turns && (head.is_q || head.is_k), bounds = h < heads && head.is_k && p.c.k_min != nullptr;
  for (int64_t s0 = u0; s0 < last; s0 += kUnit) {       // (once, but for pages of 128)
    const int64_t lo = s0 > first ? s0 : first, hi = s0 + kUnit < last ? s0 + kUnit : last;
    if (lo >= hi) continue;
    if (s0 != u0) __syncthreads();                       // (the sines of the half before are still in use)
    append_part<true>(p, sm, b, s0, lo, hi, tid);
    __syncthreads();
    if (h >= heads) continue;
    Bounds8 ba, bb;
    ba.reset();
    bb.reset();
    int64_t begin = lo;                                  // the page's first new row
    for (int64_t pos = lo; pos < hi; ++pos) {
      const int r = (int)(pos - s0), t = (int)(pos - nr.start), pg = sm.page[r / most];
      if (t > 0) {
        xa.load(rows + t * p.tok_stride + ca);
        xb.load(rows + t * p.tok_stride + cb);
      }
      float a[8], w[8];
      xa.get(a);
      xb.get(w);
      if (turn) {
        float2 cs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) cs[j] = sm.cs[r][part + 8 * j];
        turn_pieces<kInterleaved>(a, w, cs);
      }
      const uint4 pa = pack8(a), pb = pack8(w);
      __nv_bfloat16* to = head.row(p, b, t, pos, pg);
      if (to != nullptr) {
        *reinterpret_cast<uint4*>(to + ca) = pa;
        *reinterpret_cast<uint4*>(to + cb) = pb;
      }
      if (bounds) {
        ba.take(pa);
        bb.take(pb);
        if (pos + 1 == hi || (r + 1) % most == 0) {      // its last one: the bounds leave (see above)
          if (pg >= 0) store_bounds(p, ba, bb, pg, head.g, ca, cb, (begin & (page - 1)) != 0);
          ba.reset();
          bb.reset();
          begin = pos + 1;
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------------ pages' scores
// score[i] = max_h sum_c max(q[h][c] k_min[i][c], q[h][c] k_max[i][c]): the bound that is taken depends on the sign of
// q[h][c] alone, so a page and head cost 128 products.  They are formed and added in 64 bits: the products of two bf16 are
// then exact and their sums all but exact, and the selection does not depend on the order of the sum.  A bf16 becomes a
// double of 2^-896 its value by moving its bits (subnormals and zeros too), without a conversion; the queries carry 2^512.
//
// Bound by the bounds' bytes and, in the end, by the instructions around the products (a choice and a product each, conversions,
// exchanges).  Up to four heads: sixteen threads share a page, eight channels each, and have four pages in flight.  The sixteen sums
// (page, head) of a thread meet in fifteen exchanges that leave each thread one of them.  More heads: the MMAs below, which need no
// exchanges but twice the products, all eight columns of them.  A CTA of four warps takes 32 pages.  Measured: 2048 pages of
// 8 x 4 heads 6.5 us (MMAs 8.1), sixteen ragged sequences of up to 2048 pages of 4 x 7 heads 22.4 (as two rounds of four heads 28.5).
constexpr int kScoreCtaThreads = 128, kEachPages = 4, kScalarHeads = 4;
constexpr int kCtaPages = kScoreCtaThreads / 16 * kEachPages;

__device__ __forceinline__ double wide_hi(uint32_t top) {   // bf16 in the upper half of `top`, as a double times 2^-896
  return __hiloint2double((int)((top & 0x80000000u) | ((top & 0x7fff0000u) >> 3)), 0);
}

__global__ void __launch_bounds__(kScoreCtaThreads) page_score_kernel(const PageSelectParams p) {
  constexpr int kPages = kEachPages, kCta = kCtaPages, kHeads = kScalarHeads;
  __shared__ double2 sm_q[kHeads][4][16];   // channels 8 l + 2 i, 8 l + 2 i + 1 of head h at [h][i][l]
  const int b = blockIdx.z, g = blockIdx.y, tid = threadIdx.x, lane = tid & 31, l = lane & 15;
  const int n_kv = p.c.n_kv_heads, G = p.group;
  const int32_t* row = p.c.table + (int64_t)b * p.c.table_stride;
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  // sizes, queries and the first pages' numbers (any of the table's): one round trip
  const int act = p.active != nullptr ? __ldcg(p.active + b) : 1;
  const int n = __ldcg(p.c.len + b);
  const int i0 = blockIdx.x * kCta + (tid >> 4) * kPages;    // this thread's pages
  int pg[kPages];
#pragma unroll
  for (int u = 0; u < kPages; ++u) pg[u] = i0 + u < p.c.table_stride ? __ldcg(row + i0 + u) : -1;
  uint4 qw = make_uint4(0u, 0u, 0u, 0u);
  if (tid < G * 16)
    qw = __ldcg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) +
                                               ((int64_t)b * p.n_q_heads + (int64_t)g * G) * kHeadDim) + tid);
  const int64_t room = (int64_t)p.c.table_stride << p.c.page_shift;
  const int lim = room < p.max_len ? (int)room : p.max_len;
  const int pages = (min(max(n, 0), lim) + (1 << p.c.page_shift) - 1) >> p.c.page_shift;
  if (act == 0 || (int)blockIdx.x * kCta >= pages) return;
  if (tid < kHeads * 16) {
    const uint32_t x[4] = {qw.x, qw.y, qw.z, qw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      sm_q[tid >> 4][i][tid & 15] = make_double2(wide_hi(x[i] << 16) * 0x1p1000 * 0x1p408, wide_hi(x[i]) * 0x1p1000 * 0x1p408);
  }
  if (tid == 0 && blockIdx.x == 0 && g == 0 && n > lim) atomicOr(p.status, RKV_DEV_LEN_CLAMPED);
  __syncthreads();
  uint4 least[kPages], most[kPages];
  int bad = 0;
#pragma unroll
  for (int u = 0; u < kPages; ++u) {
    least[u] = most[u] = make_uint4(0u, 0u, 0u, 0u);
    if (i0 + u < pages) {
      if ((unsigned)pg[u] >= (unsigned)p.c.n_pages) {
        bad |= 1 << u;
      } else {
        const int64_t at = ((int64_t)pg[u] * n_kv + g) * (kHeadDim / 8) + l;
        least[u] = __ldcg(static_cast<const uint4*>(p.c.k_min) + at);
        most[u] = __ldcg(static_cast<const uint4*>(p.c.k_max) + at);
      }
    }
  }
  const int u = l / kHeads;                    // this thread's sum: page u, head l % kHeads
  uint64_t key = 0ull;
  double v[16];   // [page][head]
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = 0.0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    double a0[kPages], a1[kPages], z0[kPages], z1[kPages];
#pragma unroll
    for (int w = 0; w < kPages; ++w) {
      const uint32_t a = i == 0 ? least[w].x : i == 1 ? least[w].y : i == 2 ? least[w].z : least[w].w;
      const uint32_t z = i == 0 ? most[w].x : i == 1 ? most[w].y : i == 2 ? most[w].z : most[w].w;
      a0[w] = wide_hi(a << 16);
      a1[w] = wide_hi(a);
      z0[w] = wide_hi(z << 16);
      z1[w] = wide_hi(z);
    }
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      const double2 q = sm_q[h][i][l];
      const bool n0 = __double2hiint(q.x) < 0, n1 = __double2hiint(q.y) < 0;
#pragma unroll
      for (int w = 0; w < kPages; ++w) {
        v[kHeads * w + h] = fma(q.x, n0 ? a0[w] : z0[w], v[kHeads * w + h]);
        v[kHeads * w + h] = fma(q.y, n1 ? a1[w] : z1[w], v[kHeads * w + h]);
      }
    }
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    const bool up = (lane & o) != 0;
#pragma unroll
    for (int j = 0; j < o; ++j) {
      const double keep = up ? v[j + o] : v[j], give = up ? v[j] : v[j + o];
      v[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
  if (l % kHeads < G) key = score_key(v[0]);
#pragma unroll
  for (int o = 1; o < kHeads; o <<= 1) key = max(key, (uint64_t)__shfl_xor_sync(0xffffffffu, (unsigned long long)key, o));
  if (l % kHeads == 0 && i0 + u < pages) {
    if ((bad >> u) & 1) {   // a page that is not there comes after all others
      key = 0ull;
      if (g == 0) atomicOr(p.status, RKV_DEV_BAD_INDEX);
    }
    p.keys[((int64_t)b * n_kv + g) * p.key_stride + i0 + u] = key;
  }
}

// Groups of five to eight heads: the products as m8n8k4 MMAs in 64 bits, eight pages x eight heads, 128 upper bounds with the
// positive parts of the queries and 128 lower ones with the negative parts.  A warp takes eight pages; the four lanes of a
// page have 32 channels each, and since the order of a sum is free they hold page and query alike, in 16-byte pieces as they lie in memory.
__device__ __forceinline__ void mma_f64(double (&c)[2], double a, double b) {
  asm volatile("mma.sync.aligned.m8n8k4.row.col.f64.f64.f64.f64 {%0,%1}, {%2}, {%3}, {%0,%1};" : "+d"(c[0]), "+d"(c[1]) : "d"(a), "d"(b));
}

__global__ void __launch_bounds__(kScoreCtaThreads) page_score_mma_kernel(const PageSelectParams p) {
  const int b = blockIdx.z, g = blockIdx.y, tid = threadIdx.x, lane = tid & 31, r = lane >> 2, t = lane & 3;
  const int n_kv = p.c.n_kv_heads, G = p.group;
  const int page = blockIdx.x * kCtaPages + (tid >> 5) * 8 + r;
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  // sizes, queries and page number (any of the table's): one round trip
  const int act = p.active != nullptr ? __ldcg(p.active + b) : 1;
  const int n = __ldcg(p.c.len + b);
  const int pg = page < p.c.table_stride ? __ldcg(p.c.table + (int64_t)b * p.c.table_stride + page) : -1;
  const int64_t room = (int64_t)p.c.table_stride << p.c.page_shift;
  const int lim = room < p.max_len ? (int)room : p.max_len;
  const int pages = (min(max(n, 0), lim) + (1 << p.c.page_shift) - 1) >> p.c.page_shift;
  if (act == 0 || (int)blockIdx.x * kCtaPages >= pages) return;
  if (tid == 0 && blockIdx.x == 0 && g == 0 && n > lim) atomicOr(p.status, RKV_DEV_LEN_CLAMPED);
  const bool there = page < pages && (unsigned)pg < (unsigned)p.c.n_pages;
  uint4 q[4], least[4], most[4];               // channels 32 j + 8 t .. + 7 of head r, of page r
  const uint4* q_at = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) +
                                                     ((int64_t)b * p.n_q_heads + (int64_t)g * G + min(r, G - 1)) * kHeadDim) + t;
  const int64_t at = ((int64_t)(there ? pg : 0) * n_kv + g) * (kHeadDim / 8) + t;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    q[j] = __ldcg(q_at + 4 * j);
    least[j] = __ldcg(static_cast<const uint4*>(p.c.k_min) + at + 4 * j);
    most[j] = __ldcg(static_cast<const uint4*>(p.c.k_max) + at + 4 * j);
  }
  double c[4][2] = {};                         // chains
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t qw[4] = {q[j].x, q[j].y, q[j].z, q[j].w}, lw[4] = {least[j].x, least[j].y, least[j].z, least[j].w},
                   mw[4] = {most[j].x, most[j].y, most[j].z, most[j].w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t up = (e & 1) != 0 ? 0u : 16u;
      const double x = wide_hi(qw[e >> 1] << up) * 0x1p1000 * 0x1p408;
      const bool neg = __double2hiint(x) < 0;
      mma_f64(c[e & 1], wide_hi(mw[e >> 1] << up), neg ? 0.0 : x);
      mma_f64(c[2 + (e & 1)], wide_hi(lw[e >> 1] << up), neg ? x : 0.0);
    }
  }
  uint64_t key = 0ull;                         // page r, heads 2 t and 2 t + 1
  if (2 * t < G) key = score_key((c[0][0] + c[1][0]) + (c[2][0] + c[3][0]));
  if (2 * t + 1 < G) key = max(key, score_key((c[0][1] + c[1][1]) + (c[2][1] + c[3][1])));
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) key = max(key, (uint64_t)__shfl_xor_sync(0xffffffffu, (unsigned long long)key, o));
  if (t == 0 && page < pages) {
    if (!there) {   // a page that is not there comes after all others
      key = 0ull;
      if (g == 0) atomicOr(p.status, RKV_DEV_BAD_INDEX);
    }
    p.keys[((int64_t)b * n_kv + g) * p.key_stride + page] = key;
  }
}

// -------------------------------------------------------------------------------------------------------- selection
// As a launch of its own, one CTA per (sequence, KV head): for batches, and where the scores do not fit beside the attention's
// buffers (otherwise the CTAs that attend pick for themselves: rkv_paged_attn.cu).
constexpr int kPickThreads = 512;

__global__ void __launch_bounds__(kPickThreads) page_select_kernel(const PageSelectParams p) {
  extern __shared__ uint64_t sm_k[];
  __shared__ PickShared<kPickThreads> sh;
  const int b = blockIdx.y, g = blockIdx.x, tid = threadIdx.x;
  pdl_wait();
  pdl_launch();   // dependents are released only after this kernel's own wait (see launch_ex)
  const int act = p.active != nullptr ? __ldcg(p.active + b) : 1;
  const int64_t room = (int64_t)p.c.table_stride << p.c.page_shift;
  const int lim = room < p.max_len ? (int)room : p.max_len;
  const int n = min(max(__ldcg(p.c.len + b), 0), lim);
  if (act == 0) return;
  const int pages = (n + (1 << p.c.page_shift) - 1) >> p.c.page_shift;
  int32_t* out = p.page_idx + ((int64_t)b * gridDim.x + g) * p.top;
  for (int i = min(p.top, pages) + tid; i < p.top; i += kPickThreads) out[i] = -1;
  pick_pages<kPickThreads>(p.keys + ((int64_t)b * gridDim.x + g) * p.key_stride, pages, p.top, p.first, p.last, sm_k, sh, tid,
                           [&](int k, int page) { out[k] = page; }, [](int) {});
}

}  // namespace

cudaError_t prepare_page_select() {
  return cudaFuncSetAttribute(page_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostPages * 8);
}

cudaError_t launch_page_scores(const PageSelectParams& p, int n_seq, int most_pages, cudaStream_t st) {
  return launch_ex(p.group > kScalarHeads ? page_score_mma_kernel : page_score_kernel,
                   dim3((most_pages + kCtaPages - 1) / kCtaPages, p.c.n_kv_heads, n_seq), dim3(kScoreCtaThreads), 0, st, 1, p);
}

cudaError_t launch_page_select(const PageSelectParams& p, int n_seq, int most_pages, cudaStream_t st) {
  return launch_ex(page_select_kernel, dim3(p.c.n_kv_heads, n_seq), dim3(kPickThreads), (size_t)most_pages * 8, st, 1, p);
}

cudaError_t launch_paged_append(const PagedAppendParams& p0, bool is_bf16, bool interleaved, int n_seq, int sm_count,
                                cudaStream_t st) {
  PagedAppendParams p = p0;
  const int unit = (1 << p.c.page_shift) > kUnit ? (1 << p.c.page_shift) : kUnit;
  const int units = p.n_tok == 1 ? 1 : (p.n_tok - 1) / unit + 2;   // new rows that begin inside a unit may end inside one more
  const int heads = p.n_q_heads + 2 * p.c.n_kv_heads;
  const dim3 block(kAppendThreads);
  if (p.n_tok <= kFewRows) {
    const dim3 grid(units, (heads + kAppendThreads / 8 - 1) / (kAppendThreads / 8), n_seq);
    auto go = [&](auto* kernel) { return launch_ex(kernel, grid, block, 0, st, 1, p); };
    if (is_bf16) return interleaved ? go(paged_append_few_kernel<__nv_bfloat16, true>) : go(paged_append_few_kernel<__nv_bfloat16, false>);
    return interleaved ? go(paged_append_few_kernel<float, true>) : go(paged_append_few_kernel<float, false>);
  }
  // CTAs of a unit: queries in groups of 32 heads or so, keys and values in groups as large (four rounds of the CTA's
  // warps) or, where that leaves less than kAppendSpread CTAs to an SM, smaller ones (sines and cosines are worked out once per CTA).
  // 32 heads a CTA / 8: 1024 rows 21.0 / 10.4 us, 4096 rows 29.0 / 26.7, 32768 rows 134.5 / 143.6, 64 sequences of 256 rows 75.7 / 76.4.
  const int64_t want = kAppendSpread * (int64_t)sm_count, have = (int64_t)units * n_seq;
  int per = 32;
  while (per > 8 && have * ((heads + per - 1) / per) < want) per -= 8;
  p.rounds = per / kAppendWarps;
  p.q_groups = (p.n_q_heads + per - 1) / per;
  p.q_per = (p.n_q_heads + p.q_groups - 1) / p.q_groups;
  const dim3 grid(units, p.q_groups + (2 * p.c.n_kv_heads + per - 1) / per, n_seq);
  auto go = [&](auto* kernel) { return launch_ex(kernel, grid, block, 0, st, 1, p); };
  if (is_bf16) return interleaved ? go(paged_append_kernel<__nv_bfloat16, true>) : go(paged_append_kernel<__nv_bfloat16, false>);
  return interleaved ? go(paged_append_kernel<float, true>) : go(paged_append_kernel<float, false>);
}

}  // namespace rkv
