// Attention of one or a few new rows over a paged key/value cache.
//
// o = softmax(scale q K^T) V over the rows of the pages: every key and value row
// is read once for the G = H_q / H_kv query heads (times new rows) that share it,
// so a single token does 2 G FLOP a byte in bf16 and memory bounds it.  What the
// kernel is built for is bytes in flight and even shares:
//
// * A wave takes 32 keys (fp32: 16) a step, loads the next step's K and V straight into
//   registers while it works on this one, and keeps a softmax of its own; four waves
//   of a workgroup walk neighbouring steps and are joined through LDS at the end.
//   No barrier in the loop, and no LDS (but for values that are not finite).
// * The keys of all sequences are cut into parts of nearly one size (plan below),
//   planned on the device from the lengths, so that ragged batches fill the card
//   evenly; rows whose keys are cut are joined by a second kernel.
//
// Measured: 8 x 32 heads x 32K keys 622 us, 6.9 TB/s of keys and values (a kernel that does
// nothing but read reaches 6.5 to 7.1 here); in 8 bits 325 us, 6.7 TB/s; 64 ragged sequences of up to
// 32K, 8 heads, 8 bits, pages of 16 rows 365 us, 6.0 TB/s (its loads bound it: 368 us with the arithmetic
// of the whole steps left out, 215 with their loads left out).  One token of one 8K sequence takes 7.2 +
// 3.3 us, a chain of loads (arguments, lengths, page numbers, keys) in each workgroup, of which
// every CU has one.
//
// Operand layouts (lane = 16 g + n).  16x16x32 bf16: A holds row n, B column n, both
// at k = 8 g .. 8 g + 7; the result's element e is row 4 g + e of column n.
//   S^T = K Q^T: row = key, column = query row, k = channel.
//   O^T += V^T P^T over 32 keys: k slot 8 g + j is key 4 g + j of the step's first
//     16 keys (j < 4) or 4 g + j - 4 of its second, so the result of S^T is P^T
//     as it stands.  A lane reads E = D / 16 neighbouring channels of its eight keys,
//     16 lanes a whole row; a byte permutation of register pairs turns the
//     8 x E block into the A operands of E products.  Row m of product t is channel base(m) + t,
//     E m + t in bf16.
// 16x16x4 fp32: k = g, one value a lane; four products per 16-byte read, and the
// channels of a read are permuted alike in both operands.
#include <type_traits>

#include "paged_common.h"

namespace pd {

constexpr int kPagedWaves = 4;

int paged_block_keys(bool fp32) { return kPagedWaves * (fp32 ? 16 : 32); }

// Query rows and keys of one workgroup.
struct PagedPart {
  int b, g, rb;          // sequence, KV head, row block
  int len, n_new;        // the sequence's rows and new rows
  int first, last;       // blocks of keys of this part
  int parts, index;      // how many the row block's keys are cut into, and which this is
  int slot;              // where its sums go; a unit's parts lie row_blocks apart
  bool any;
};

// The cut of all sequences' keys.  Sequence b has n_b blocks of keys for each of its
// units (KV head x row block).  With a quota of Q blocks a part, a unit has ceil(n_b / Q)
// parts, the last one shorter; they are numbered by sequence, head and part.  Every
// wave finds its own part from the lengths, 64 sequences at a time (large batches: from sums that a
// launch before has left, paged_plan_kernel).
//
// The quota: units of one size (the longest at most 5/4 of the mean), as many as the CUs or fewer,
// or nearly twice as many, are cut into as few parts as give every CU one.  Otherwise parts of 16
// blocks or more, paged_parts of them where the keys suffice, so that the workgroups of short
// sequences and the ends of long ones fill in.  Measured:
// 8 x 32 heads x 8K keys 160 us, 174 in such finer parts; 16 of them 327 and 326, 15 of them 311
// and 324, 12 of them 296 and 251, 9 of them 271 and 199; 64 ragged sequences in 8 bits 365 us in
// finer parts, 474 in as few as the CUs.
struct PagedSeq {
  int len, n_new, blocks;
};
template <int BK>
__device__ __forceinline__ PagedSeq paged_seq(const PagedAttnArgs& a, int b) {
  const PagedArgs& p = a.c;
  // Both loads in flight at once, also where there is no such sequence.
  const int at = b < p.B ? b : 0;
  const int len = p.kv_len[at], n_new = p.new_rows ? p.new_rows[at] : p.Ln;
  PagedSeq s{min(max(len, 0), p.max_pages << p.log2R), min(max(n_new, 0), p.Ln), 0};
  if (b < p.B && s.len > 0 && s.n_new > 0) s.blocks = ((a.page_idx ? a.top_k << p.log2R : s.len) + BK - 1) / BK;
  return s;
}

// n / d for 0 <= n < 2^27 and quotients below 2^17: the product with the reciprocal is off by
// less than one then.
__device__ __forceinline__ int short_div(int n, int d) {
  int q = (int)((float)n * __builtin_amdgcn_rcpf((float)d));
  const int r = n - q * d;
  q += r >= d ? 1 : 0;
  return r < 0 ? q - 1 : q;
}
// ceil(blocks / quota), at most paged_parts + 1.
__device__ __forceinline__ int parts_of(int blocks, int quota) {
  return blocks <= quota ? 1 : short_div(blocks - 1, quota) + 1;
}

// The quota.  all: the blocks of all units, in fp32, which a quota need not be exact for: an error of 2^-12
// still leaves the number of parts below what the host has made room for.  most: of the longest.
__device__ __forceinline__ int paged_quota(const PagedAttnArgs& a, float all, int most) {
  const float seqs = (float)a.c.B * (float)(a.c.Hkv * a.row_blocks);
  auto ceil_of = [](float x) {
    const int c = (int)fminf(x, 1073741824.f);
    return (float)c < x ? c + 1 : c;
  };
  const int fill = ceil_of(all * (1.f / kNumCu)), fine = ceil_of(all * a.per_part);
  const bool even = 0.8f * (float)most * seqs <= all &&
                    (seqs <= 1.f * kNumCu || (seqs >= 1.8f * kNumCu && seqs <= 2.f * kNumCu));
  return max(1, uniform(even ? fill : max(fine, min(fill, 16))));
}
// Order: the parts of a whole quota, then the shorter ends, which even out when the
// workgroups finish (7 x 32 heads x 8K keys 156 us, with 32 new rows 174; sequence by sequence 232
// and 249, as CUs got two whole parts).  `whole` of the parts of each of a sequence's units come in the first turn.
struct PagedCut {
  int parts, whole;
};
__device__ __forceinline__ PagedCut paged_cut(const PagedAttnArgs& a, int quota, int b, const PagedSeq& s) {
  PagedCut c{0, 0};
  if (b < a.c.B) {
    c.parts = parts_of(s.blocks, quota);
    c.whole = c.parts * quota == s.blocks ? c.parts : c.parts - 1;
  }
  return c;
}
__device__ __forceinline__ int wave_sum(int x) {
  return __builtin_amdgcn_readlane(wave_scan(x, 0, [](int p, int q) { return p + q; }), 63);
}
__device__ __forceinline__ int wave_most(int x) {
  return __builtin_amdgcn_readlane(wave_scan(x, 0, [](int p, int q) { return max(p, q); }), 63);
}

// The sums that every wave needs to find its part, for batches of more than kPlanBatch sequences,
// where walking all lengths would cost each wave more than this launch: quota, parts of the first
// turn; then for every 64 sequences the parts of the first turn, and of both, up to their end.
// One workgroup.
template <int BK>
__global__ __launch_bounds__(1024) void paged_plan_kernel(PagedAttnArgs a) {
  __shared__ float sums[16];
  __shared__ int tops[16], whole[1024], parts[1024], ends[2][16];
  const PagedArgs& p = a.c;
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  const int units = p.Hkv * a.row_blocks, n = (p.B + 63) / 64;   // at most 1024
  float all = 0.f;
  int most = 0;
  for (int i = wave; i < n; i += 16) {
    const int x = paged_seq<BK>(a, 64 * i + lane).blocks;
    all += (float)wave_sum(x);
    most = max(most, wave_most(x));
  }
  sums[wave] = all;
  tops[wave] = most;
  __syncthreads();
  all = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    all += sums[w];
    most = max(most, tops[w]);
  }
  const int quota = paged_quota(a, all * (float)units, most);
  for (int i = wave; i < n; i += 16) {
    const PagedCut c = paged_cut(a, quota, 64 * i + lane, paged_seq<BK>(a, 64 * i + lane));
    const int w = wave_sum(c.whole), x = wave_sum(c.parts);
    if (lane == 0) {
      whole[i] = w;
      parts[i] = x;
    }
  }
  __syncthreads();
  auto add = [](int x, int y) { return x + y; };
  int w = wave_scan(tid < n ? whole[tid] : 0, 0, add), x = wave_scan(tid < n ? parts[tid] : 0, 0, add);
  if (lane == 63) {
    ends[0][wave] = w;
    ends[1][wave] = x;
  }
  __syncthreads();
  int first = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    first += ends[0][i];
    w += i < wave ? ends[0][i] : 0;
    x += i < wave ? ends[1][i] : 0;
  }
  if (tid == 0) {
    a.plan[0] = quota;
    a.plan[1] = first * units;
  }
  if (tid < n) {
    a.plan[2 + 2 * tid] = w * units;
    a.plan[3 + 2 * tid] = x * units;
  }
}

template <int BK>
__device__ __forceinline__ PagedPart paged_find(const PagedAttnArgs& a, int find, int lane) {
  const PagedArgs& p = a.c;
  const int units = p.Hkv * a.row_blocks;
  auto add = [](int x, int y) { return x + y; };
  PagedPart r{};
  // Number i among a sequence's parts of this turn, `each` a unit: head and part, and row block.  Row
  // blocks of the same keys run on one XCD, eight workgroups apart, so that all but the first find
  // them in its L2.
  auto place = [&](int i, int each) {
    int pair = i;
    r.rb = 0;
    if (a.row_blocks > 1) {
      if (i < p.Hkv * each / kNumXcd * kNumXcd * a.row_blocks) {
        const int q = a.by_blocks.quot(i / kNumXcd);
        r.rb = a.by_blocks.rem(i / kNumXcd, q);
        pair = q * kNumXcd + i % kNumXcd;
      } else {
        pair = a.by_blocks.quot(i);
        r.rb = a.by_blocks.rem(i, pair);
      }
    }
    return pair;
  };
  if (a.max_chunks == 1) {   // one part a unit
    r.b = a.by_units.quot(find);
    if (r.b >= p.B) return r;
    const PagedSeq s = paged_seq<BK>(a, r.b);
    r.len = s.len;
    r.n_new = s.n_new;
    r.g = place(a.by_units.rem(find, r.b), 1);
    r.last = s.blocks;
    r.parts = 1;
    r.any = true;
    return r;
  }
  int quota;
  PagedSeq s;
  int first_turn, b0 = 0, before = 0, before_all = 0;   // parts of the turn, and of both, before sequence b0
  bool second;
  if (a.plan) {
    quota = a.plan[0];
    first_turn = a.plan[1];
    second = find >= first_turn;
    if (second) find -= first_turn;
    const int n = (p.B + 63) / 64;
    for (int i0 = 0;; i0 += 64) {
      if (i0 >= n) return r;
      const int i = min(i0 + lane, n - 1), w = a.plan[2 + 2 * i], x = a.plan[3 + 2 * i];
      const int own = second ? x - w : w;
      const uint64_t past = __ballot(own > find);
      const int l = past ? __ffsll((unsigned long long)past) - 1 : 64;   // those before end at or below `find`
      if (l > 0) {
        before = __builtin_amdgcn_readlane(own, l - 1);
        before_all = __builtin_amdgcn_readlane(x, l - 1);
      }
      if (past) {
        b0 = (i0 + l) * 64;
        break;
      }
    }
    s = paged_seq<BK>(a, b0 + lane);
  } else {
    const PagedSeq head = s = paged_seq<BK>(a, lane);
    float all = 0.f;
    int most = 0;
    for (int c0 = 0; c0 < p.B; c0 += 64) {
      const int n = c0 == 0 ? head.blocks : paged_seq<BK>(a, c0 + lane).blocks;
      all += (float)wave_sum(n);
      most = max(most, wave_most(n));
    }
    quota = paged_quota(a, all * (float)units, most);
    first_turn = 0;
    for (int c0 = 0; c0 < p.B; c0 += 64)
      first_turn += wave_sum(paged_cut(a, quota, c0 + lane, c0 == 0 ? head : paged_seq<BK>(a, c0 + lane)).whole);
    first_turn *= units;
    second = find >= first_turn;
    if (second) find -= first_turn;
  }
  for (;;) {
    const PagedCut c = paged_cut(a, quota, b0 + lane, s);
    const int own = (second ? c.parts - c.whole : c.whole) * units;
    const int incl = before + wave_scan(own, 0, add);
    const int incl_all = before_all + wave_scan(c.parts * units, 0, add);
    const uint64_t past = __ballot(incl > find);
    if (past) {
      const int l = __ffsll((unsigned long long)past) - 1;
      const int n = __builtin_amdgcn_readlane(s.blocks, l);
      r.b = b0 + l;
      r.len = __builtin_amdgcn_readlane(s.len, l);
      r.n_new = __builtin_amdgcn_readlane(s.n_new, l);
      r.parts = __builtin_amdgcn_readlane(c.parts, l);
      const int mine = __builtin_amdgcn_readlane(own, l);
      const int each = second ? 1 : __builtin_amdgcn_readlane(c.whole, l);   // of a unit in this turn
      const int pair = place(find - (__builtin_amdgcn_readlane(incl, l) - mine), each);
      r.g = pair;
      r.index = second ? r.parts - 1 : 0;
      if (each > 1) {
        r.g = short_div(pair, each);
        r.index = pair - r.g * each;
      }
      r.first = r.parts > 1 ? r.index * quota : 0;
      r.last = r.parts > 1 ? min(r.first + quota, n) : n;
      r.slot = __builtin_amdgcn_readlane(incl_all, l) - r.parts * units + (r.g * r.parts + r.index) * a.row_blocks + r.rb;
      r.any = true;
      return r;
    }
    before = __builtin_amdgcn_readlane(incl, 63);
    before_all = __builtin_amdgcn_readlane(incl_all, 63);
    b0 += 64;
    if (b0 >= p.B) return r;
    s = paged_seq<BK>(a, b0 + lane);
  }
}

enum { kBf16 = 0, kFp8 = 1, kFp32 = 2 };

template <int D, int CT>
struct PagedShape {
  static constexpr int KS = CT == kFp32 ? 16 : 32;          // keys of a step
  static constexpr int H = KS / 16;                         // groups of 16 keys
  static constexpr int CB = CT == kFp32 ? 4 : CT == kFp8 ? 1 : 2;
  static constexpr int NK = D * CB / 64;                    // 16-byte reads of a lane for 16 keys
  static constexpr int VR = CT == kFp32 ? 4 : 8;            // V rows of a lane
  static constexpr int VW = D * CB / 64;                    // dwords of each
  static constexpr int E = CT == kFp32 ? 4 : D / 16;        // neighbouring channels of a lane
  static constexpr int NT = D / 16;                         // products of P V
  // First channel of result row m (bf16 and E4M3).
  static __device__ __forceinline__ int base(int m) { return CT == kFp8 ? 2 * E * (m & 7) + E * (m >> 3) : E * m; }
  static constexpr int BK = kPagedWaves * KS;
};

// What a wave holds of one step.
template <int D, int CT>
struct PagedStep {
  using S = PagedShape<D, CT>;
  u32x4 k[S::H][S::NK];
  uint32_t v[S::VR][S::VW];      // E4M3: read 2 j + i of 16 keys, rows 2 j and 2 j + 1 in a line
  uint32_t ex;                   // exponent bytes of four keys (see load)
  int pos[S::H];                 // position of the first key of each 16
};

// Over the four lanes n, 16 + n, 32 + n, 48 + n of a query row: halves, then neighbouring rows
// of 16 lanes, exchanged on the vector units.
template <class F>
__device__ __forceinline__ float over_groups(float x, F op) {
  const uint32_t u = __float_as_uint(x);
  const auto h = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t w = __float_as_uint(op(__uint_as_float(h[0]), __uint_as_float(h[1])));
  const auto r = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float group_max(float x) {
  return over_groups(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float group_sum(float x) {
  return over_groups(x, [](float a, float b) { return a + b; });
}

template <int CTRL, int BANKS>
__device__ __forceinline__ uint32_t dpp_bits(uint32_t old, uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, CTRL, 0xf, BANKS, false);
}
// The value of lane L + h of the own row of 16 lanes.
template <int L>
__device__ __forceinline__ uint32_t row_lane(uint32_t x, int h) {
  return h == 0 ? dpp_bits<0x150 + L, 0xf>(x, x) : dpp_bits<0x151 + L, 0xf>(x, x);   // row_newbcast
}

template <bool STREAM, class T>
__device__ __forceinline__ T fetch(const T* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  else return *p;
}

constexpr int kFarPos = 1 << 30;   // the position of keys that are not there

// STREAM: the keys are read by one workgroup alone (non-temporal loads: 8 x 32 heads x 32K keys 648
// against 723 us, 64 ragged sequences in 8 bits 381 against 402); row blocks that share them leave
// them in the caches.  Waves a SIMD: what the registers of each form leave room for (two blocks of 16
// rows in d = 64 use 168 in 8 bits, and more would cost the third wave).
template <int D, int CT, int RT, bool STREAM>
__global__ __launch_bounds__(256, D == 64 && CT != kFp32 ? 3 : D == 64 || (RT == 1 && CT != kFp32) ? 2 : 1) void paged_attn_kernel(PagedAttnArgs a) {
  using S = PagedShape<D, CT>;
  constexpr int H = S::H, CB = S::CB, NK = S::NK, VR = S::VR, VW = S::VW, E = S::E, NT = S::NT, BK = S::BK;
  constexpr int OP = D + 4;
  __shared__ float lds_o[kPagedWaves][16][OP];
  __shared__ float lds_ml[kPagedWaves][RT * 16][2];
  const PagedArgs& p = a.c;
  const int wave = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, n = lane & 15, g4 = lane >> 4;
  const PagedPart part = paged_find<BK>(a, uniform((int)block_id()), lane);
  if (!part.any) return;
  const int b = uniform(part.b), g = uniform(part.g), len = uniform(part.len), n_new = uniform(part.n_new);
  const int rows = n_new * p.G, row0 = uniform(part.rb) * (RT * 16);
  if (a.max_chunks > 1 && part.index == 0 && threadIdx.x == 0) {   // what the join has to know of the unit
    int32_t* u = a.unit + (((long long)b * p.Hkv + g) * a.row_blocks + part.rb) * 4;
    u[0] = part.slot;
    u[1] = part.parts;
    u[2] = rows - row0;
  }
  if (row0 >= rows) return;

  // Query rows: row r is new row r / G, head g G + r % G.
  bf16x8 qb[RT][D / 32];
  f32x4 qf[RT][D / 16];
  int lim[RT];                       // the row sees positions below
  int every = kFarPos;               // positions below which every row of the block sees
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int r = row0 + t * 16 + n;
    const bool real = r < rows;
    const int rr = real ? r : row0, nr = a.by_group.quot(rr);
    const long long q_el = (((long long)b * p.Ln + nr) * p.Hq + (long long)g * p.G + a.by_group.rem(rr, nr)) * D;
    lim[t] = !real ? 0 : p.causal ? len - n_new + 1 + nr : len;
    if constexpr (CT == kFp32) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) qf[t][i] = *(const f32x4*)((const float*)a.q + q_el + 16 * i + 4 * g4);
    } else {
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        // bf16 keys: read i of a lane is channels 32 i + 8 g..; E4M3 keys: 64 (i/2) + 16 g + 8 (i%2)..
        const int ch = CT == kBf16 ? 32 * i + 8 * g4 : 64 * (i / 2) + 16 * g4 + 8 * (i & 1);
        qb[t][i] = *(const bf16x8*)((const uint16_t*)a.q + q_el + ch);
      }
    }
  }
  every = p.causal ? len - n_new + 1 + a.by_group.quot(row0) : len;

  f32x4 o[RT][NT];
  float m[RT], l[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = kNoMax;
    l[t] = 0.f;
#pragma unroll
    for (int i = 0; i < NT; ++i) o[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Where the keys of 64 steps lie, a lane each: page and position of every 16.
  const int32_t* table = p.page_table + (long long)b * p.max_pages;
  const int32_t* chosen = a.page_idx ? a.page_idx + ((long long)b * p.Hkv + g) * a.top_k : nullptr;
  // Blocks behind the last row's own position are in no row's sight.
  const int sight = p.causal ? len - n_new + 1 + a.by_group.quot(min(rows - 1, row0 + RT * 16 - 1)) : len;
  const int n_steps = (chosen ? part.last : min(part.last, (max(sight, 0) + BK - 1) / BK)) - part.first;
  int at_page[H], at_pos[H];
  int bad = kFarPos;                 // the least position on a page outside the pool
  auto locate = [&](int i0) {
    const int i = i0 + lane;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      at_page[h] = 0;
      at_pos[h] = kFarPos;
      if (i < n_steps) {
        const int key = (part.first + i) * BK + wave * S::KS + h * 16;   // among the keys to visit
        int ord = key >> p.log2R;
        if (chosen) ord = ord < a.top_k ? chosen[ord] : -1;
        const int pos = (int)((unsigned)ord << p.log2R) + (key & (p.R - 1));
        if ((unsigned)ord < (unsigned)p.max_pages && pos < len) {
          const int page = table[ord];
          at_pos[h] = pos;
          if ((unsigned)page < (unsigned)p.n_pages) at_page[h] = page;
          else bad = min(bad, pos);
        }
      }
    }
  };

  const uint32_t page_rows = (uint32_t)p.R;
  auto load = [&](PagedStep<D, CT>& s, int i) {
    long long rows_at[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int page = __builtin_amdgcn_readlane(at_page[h], i & 63);
      s.pos[h] = __builtin_amdgcn_readlane(at_pos[h], i & 63);
      const long long row = ((long long)page * p.Hkv + g) * page_rows + (s.pos[h] & (p.R - 1));
      const char* kp = (const char*)p.k_pages + row * (D * CB) + n * (D * CB) + 16 * g4;
#pragma unroll
      for (int j = 0; j < NK; ++j) s.k[h][j] = fetch<STREAM>((const u32x4*)(kp + 64 * j));
      const char* vp = (const char*)p.v_pages + row * (D * CB) + g4 * (4 * D * CB);
      if constexpr (CT == kFp8) {
        // Lanes n and n ^ 8 read twice the channels that they need, of two keys each, and swap
        // halves later: loads of 8 bytes a lane were twice as many (one sequence of 128K keys
        // with 8 heads 50.8 us, now 49.0; 64 ragged ones 380, now 377).
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t* w = s.v[4 * h + 2 * j];
          const char* at = vp + (2 * (n >> 3) + j) * D + (n & 7) * (D / 8);
          if constexpr (VW == 2) *(u32x4*)w = fetch<STREAM>((const u32x4*)at);
          else *(u32x2*)w = fetch<STREAM>((const u32x2*)at);
        }
      } else {
        // fp32: channels 64 u + 4 n.., u = 0..D/64-1; bf16: E n..
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t* w = s.v[4 * h + j];
          if constexpr (CT == kFp32) {
#pragma unroll
            for (int u = 0; u < VW / 4; ++u) *(u32x4*)(w + 4 * u) = fetch<STREAM>((const u32x4*)(vp + j * (D * CB) + 256 * u + 16 * n));
          } else if constexpr (VW == 4) {
            *(u32x4*)w = fetch<STREAM>((const u32x4*)(vp + j * (D * CB) + 16 * n));
          } else {
            *(u32x2*)w = fetch<STREAM>((const u32x2*)(vp + j * (D * CB) + 8 * n));
          }
        }
      }
      rows_at[h] = row;
    }
    // One load of all exponent bytes: keys 4 g.. of K's first 16 in lanes n = 0 (mod 4), of its
    // second in 1, of V's in 2 and 3.
    if constexpr (CT == kFp8)
      s.ex = *(const uint32_t*)((n & 2 ? p.v_exp : p.k_exp) + (n & 1 ? rows_at[H - 1] : rows_at[0]) + 4 * g4);
  };

  // whole: every row sees every key of the step.
  auto compute = [&](PagedStep<D, CT>& s, auto whole_step) {
    constexpr bool whole = decltype(whole_step)::value;
    // Values as bf16 (or fp32), zeros where no key is: a weight of zero does not cancel
    // an infinity or a NaN.
    constexpr int W = CT == kFp32 ? VW : D / 32;
    uint32_t v[VR][W], ke[H], ve[H];
    if constexpr (CT == kFp8) {
#pragma unroll
      for (int h = 0; h < H; ++h) {
        ke[h] = row_lane<0>(s.ex, h);
        ve[h] = row_lane<2>(s.ex, h);
      }
#pragma unroll
      for (int j = 0; j < VR; j += 4)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            // lanes 0..7 hold keys 0 and 1, 8..15 keys 2 and 3; the lower keep the lower channels
            const uint32_t lo = s.v[j + 2 * i][w], hi = s.v[j + 2 * i + 1][w];
            const uint32_t x = dpp_bits<0x128, 0xc>(lo, hi), y = dpp_bits<0x128, 0x3>(hi, lo);
            v[j + i][2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, false));
            v[j + i][2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, true));
            v[j + 2 + i][2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, 1.0f, false));
            v[j + 2 + i][2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, 1.0f, true));
          }
    } else {
#pragma unroll
      for (int j = 0; j < VR; ++j)
#pragma unroll
        for (int w = 0; w < W; ++w) v[j][w] = s.v[j][w];
    }
    if constexpr (!whole) {
#pragma unroll
      for (int j = 0; j < VR; ++j) {
        const bool there = s.pos[j / 4] + 4 * g4 + j % 4 < len;
#pragma unroll
        for (int w = 0; w < W; ++w) v[j][w] = there ? v[j][w] : 0u;
      }
    }
    // A key that some rows see and others do not: its value has to stay out of the others
    // even where it is not finite, which a weight of zero does not achieve.  Such values are
    // zeros in the products, and are added by themselves to the rows that see them, from a
    // copy of the step's values in the wave's part of lds_o.
    bool any_odd = false;
    if (!whole && p.causal && n_new > 1) {
      float z = 0.f;
#pragma unroll
      for (int j = 0; j < VR; ++j)
#pragma unroll
        for (int w = 0; w < W; ++w) {
          if constexpr (CT == kFp32) {
            z = fmaf(0.f, __uint_as_float(v[j][w]), z);
          } else {
            z = fmaf(0.f, __uint_as_float(v[j][w] << 16), z);
            z = fmaf(0.f, __uint_as_float(v[j][w] & 0xffff0000u), z);
          }
        }
      any_odd = __any(z != z);
      if (any_odd) {
        uint32_t* copy = (uint32_t*)&lds_o[wave][0][0];   // [key of the step][channels]
#pragma unroll
        for (int j = 0; j < VR; ++j)
#pragma unroll
          for (int w = 0; w < W; ++w) {
            const int key = 16 * (j / 4) + 4 * g4 + j % 4;
            const int at = CT == kFp32 ? 64 * (w / 4) + 4 * n + w % 4 : (S::base(n) + 2 * w) / 2;
            copy[key * (CT == kFp32 ? D : D / 2) + at] = v[j][w];
            if constexpr (CT == kFp32) {
              if (!(fabsf(__uint_as_float(v[j][w])) < INFINITY)) v[j][w] = 0u;
            } else {
              if ((v[j][w] & 0x7f80u) == 0x7f80u) v[j][w] &= 0xffff0000u;
              if ((v[j][w] & 0x7f800000u) == 0x7f800000u) v[j][w] &= 0xffffu;
            }
          }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      f32x4 sc[H];
#pragma unroll
      for (int h = 0; h < H; ++h) {
        sc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (CT == kFp32) {
#pragma unroll
          for (int i = 0; i < NK; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sc[h] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(s.k[h][i][e]), qf[t][i][e], sc[h], 0, 0, 0);
        } else if constexpr (CT == kBf16) {
#pragma unroll
          for (int i = 0; i < NK; ++i) sc[h] = mfma16x16x32(__builtin_bit_cast(bf16x8, s.k[h][i]), qb[t][i], sc[h]);
        } else {
#pragma unroll
          for (int i = 0; i < NK; ++i)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              u32x4 kk;
#pragma unroll
              for (int w = 0; w < 2; ++w) {
                kk[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(s.k[h][i][2 * z + w], 1.0f, false));
                kk[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(s.k[h][i][2 * z + w], 1.0f, true));
              }
              sc[h] = mfma16x16x32(__builtin_bit_cast(bf16x8, kk), qb[t][2 * i + z], sc[h]);
            }
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = sc[h][e] * p.scale_log2;
          if constexpr (CT == kFp8) x *= exp_to_scale((ke[h] >> (8 * e)) & 255);
          if (!whole) x = s.pos[h] + 4 * g4 + e < lim[t] ? x : -INFINITY;
          sc[h][e] = x;
          top = fmaxf(top, x);
        }
      top = fmaxf(m[t], group_max(top));
      // The sums are brought to a new maximum only where it has risen by more than 8
      // (a factor of 256, far from overflow).
      if (__any(top > m[t] + 8.f)) {
        const float f = fast_exp2(m[t] - top);
        l[t] *= f;
#pragma unroll
        for (int i = 0; i < NT; ++i) o[t][i] *= f;
        m[t] = top;
      }
      float pr[H][4];
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = fast_exp2(sc[h][e] - m[t]);
          l[t] += x;
          if constexpr (CT == kFp8) {
            x *= exp_to_scale((ve[h] >> (8 * e)) & 255);
            if (!whole) x = s.pos[h] + 4 * g4 + e < lim[t] ? x : 0.f;   // bytes that no row wrote
          }
          pr[h][e] = x;
        }
      if constexpr (CT == kFp32) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < NT; ++i)
            o[t][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[j][i]), pr[0][j], o[t][i], 0, 0, 0);
      } else {
        // The weights as bf16; their sum l is taken before.  One tile of rows: two terms, the upper half of
        // the weight's bits and the rest rounded, 15 bits or more, so that the output's rounding is what is left
        // of the error (64 ragged requests in 8 bits 1.95e-3 of the 2-norm with weights of one term, 1.65e-3 with two);
        // memory bounds such calls, and the second product costs nothing there (8 x 32 heads x 32K keys 614.5 and
        // 615.1 us, one token of 8K keys 10.2 and 10.3).  Two tiles: one term, rounded to nearest; the second would be
        // paid for (32 rows of 4 heads over 8 x 8K keys 85.4 us with one, 89.1 with two; in 8 bits 84.4 and 97.9, d = 64
        // 50.3 and 57.4).
        u32x4 pw, pl;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x = pr[j < 2 ? 0 : H - 1][2 * (j & 1)], y = pr[j < 2 ? 0 : H - 1][2 * (j & 1) + 1];
          if constexpr (RT == 1) {
            const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
            pw[j] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            // 2^-24 of the weight more: a second term of zero would turn infinite values into NaN
            pl[j] = pack_bf16x2(fmaf(x, 0x1p-24f, x - __uint_as_float(a & 0xffff0000u)),
                                fmaf(y, 0x1p-24f, y - __uint_as_float(b & 0xffff0000u)));
          } else {
            pw[j] = pack_bf16x2(x, y);
          }
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          u32x4 w;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            w[j] = __builtin_amdgcn_perm(v[2 * j + 1][i / 2], v[2 * j][i / 2], i & 1 ? 0x07060302u : 0x05040100u);
          if constexpr (RT == 1) o[t][i] = mfma16x16x32(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, pl), o[t][i]);
          o[t][i] = mfma16x16x32(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, pw), o[t][i]);
        }
      }
      if (!whole && any_odd) {
        for (int key = 0; key < S::KS; ++key) {
          // The row's weight of the key, from the lane that holds it: a value counts with its weight
          // as in a product, so where this has underflowed an infinity gives NaN here too.
          float w = pr[0][0];
#pragma unroll
          for (int i = 1; i < 4 * H; ++i) w = (key >> 4) * 4 + key % 4 == i ? pr[i / 4][i % 4] : w;
          w = __shfl(w, 16 * (key / 4 % 4) + n);
          if ((key < 16 ? s.pos[0] : s.pos[H - 1]) + key % 16 >= lim[t]) continue;
          const uint32_t* copy = (const uint32_t*)&lds_o[wave][0][0] + key * (CT == kFp32 ? D : D / 2);
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < NT; ++i) {
              const int ch = CT == kFp32 ? 64 * (i / 4) + 4 * (4 * g4 + r) + i % 4 : S::base(4 * g4 + r) + i;
              const uint32_t u = copy[CT == kFp32 ? ch : ch / 2];
              const float x = __uint_as_float(CT == kFp32 ? u : i & 1 ? u & 0xffff0000u : u << 16);
              if (!(fabsf(x) < INFINITY)) o[t][i][r] += w * x;
            }
        }
      }
    }
  };

  // Whole steps first, each with the loads of the next one in flight (there is one: the wait for
  // a step's own loads can only be counted past the next one's where those are always
  // issued).  From the first other step on (the last one, the end of the rows, the new rows'
  // own positions) step by step, with masks.
  if (n_steps > 0) {
    PagedStep<D, CT> s0, s1;
    int i = 0;
    auto whole_before_another = [&]() {
      bool w = i + 1 < n_steps;
#pragma unroll
      for (int h = 0; h < H; ++h) w = w && __builtin_amdgcn_readlane(at_pos[h], i & 63) + 16 <= every;
      return w;
    };
    auto fetch_next = [&](PagedStep<D, CT>& s) {
      if (((i + 1) & 63) == 0) locate(i + 1);
      load(s, i + 1);
      __builtin_amdgcn_sched_barrier(0);
    };
    locate(0);
    load(s0, 0);
    while (whole_before_another()) {
      fetch_next(s1);
      compute(s0, std::true_type{});
      ++i;
      if (!whole_before_another()) {
        s0 = s1;
        break;
      }
      fetch_next(s0);
      compute(s1, std::true_type{});
      ++i;
    }
    for (;;) {
      compute(s0, std::false_type{});
      if (++i >= n_steps) break;
      if ((i & 63) == 0) locate(i);
      load(s0, i);
    }
  }

  // Join of the four waves.  Column n of the results is query row n.
  int spoilt = kFarPos;              // rows that see this position are NaN
  if (__any(bad < kFarPos)) spoilt = __builtin_amdgcn_readlane(wave_scan(bad, kFarPos, [](int x, int y) { return min(x, y); }), 63);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l[t] = group_sum(l[t]);
    if (spoilt < lim[t]) l[t] = NAN;
    if (g4 == 0) {
      lds_ml[wave][t * 16 + n][0] = m[t];
      lds_ml[wave][t * 16 + n][1] = l[t];
    }
  }
  __syncthreads();
  const int rl = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * (D / 16);
  const long long slot = (long long)part.slot * a.part_rows;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float top = lds_ml[0][t * 16 + n][0];
#pragma unroll
    for (int w = 1; w < kPagedWaves; ++w) top = fmaxf(top, lds_ml[w][t * 16 + n][0]);
    const float f = fast_exp2(m[t] - top);
    // fp32: product 4 u + e has channel 64 u + 4 (4 g + r) + e, otherwise t has base(4 g + r) + t.
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < NT; i += 4) {
        const int ch = CT == kFp32 ? 16 * i + 4 * (4 * g4 + r) : S::base(4 * g4 + r) + i;
        *(f32x4*)&lds_o[wave][n][ch] = f32x4{o[t][i][r], o[t][i + 1][r], o[t][i + 2][r], o[t][i + 3][r]} * f;
      }
    __syncthreads();
    const int r = row0 + t * 16 + rl;
    if (r < rows) {
      float M = lds_ml[0][t * 16 + rl][0], L = 0.f;
#pragma unroll
      for (int w = 1; w < kPagedWaves; ++w) M = fmaxf(M, lds_ml[w][t * 16 + rl][0]);
#pragma unroll
      for (int w = 0; w < kPagedWaves; ++w) L += lds_ml[w][t * 16 + rl][1] * fast_exp2(lds_ml[w][t * 16 + rl][0] - M);
      float x[D / 16];
#pragma unroll
      for (int e = 0; e < D / 16; ++e) {
        x[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kPagedWaves; ++w) x[e] += lds_o[w][rl][c0 + e];
      }
      if (part.parts > 1) {
        const long long at = slot + t * 16 + rl;
#pragma unroll
        for (int e = 0; e < D / 16; e += 4) *(f32x4*)(a.o_part + at * D + c0 + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
        if (c0 == 0) {
          a.ml_part[2 * at] = M;
          a.ml_part[2 * at + 1] = L;
        }
      } else {
        const float inv = 1.0f / L;
        const int nr = a.by_group.quot(r), head = g * p.G + a.by_group.rem(r, nr);
        const long long el = (((long long)b * p.Ln + nr) * p.Hq + head) * D + c0;
#pragma unroll
        for (int e = 0; e < D / 16; e += 4) {
          float y[4];
#pragma unroll
          for (int z = 0; z < 4; ++z) y[z] = L == 0.f ? 0.f : x[e + z] * inv;
          if constexpr (CT == kFp32) *(f32x4*)((float*)a.o + el + e) = f32x4{y[0], y[1], y[2], y[3]};
          else *(u32x2*)((uint16_t*)a.o + el + e) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
        }
        if (c0 == 0 && a.lse)
          a.lse[((long long)b * p.Hq + head) * p.Ln + nr] = L == 0.f ? -INFINITY : (M + __log2f(L)) * kLn2;
      }
    }
    __syncthreads();
  }
}

// The join of rows whose keys were cut: o = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s in the
// parts' order.  A thread takes four channels of every SL-th part, with the loads of eight
// parts in flight, and the slices are joined through LDS.  RW rows a workgroup: one where
// there are few rows, which may have many parts each; four where there are many rows and
// so few parts, or one, each (a call of 13 x 16 heads x 33 rows 22.2 us, 23.6 with one row a workgroup).
template <int D, bool BF16, int RW>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a) {
  constexpr int T = D / 4, SL = 256 / T / RW, U = 8;   // threads of a row, slices of the parts
  __shared__ f32x4 lds_o[RW][SL][T];
  __shared__ float lds_m[RW][SL], lds_l[RW][SL];
  const PagedArgs& p = a.c;
  const int rw = threadIdx.x / (T * SL), c = threadIdx.x % T, sl = threadIdx.x / T % SL;
  const int id = uniform((int)block_id()) * RW + rw;
  const int bg = a.by_rows.quot(id), r = a.by_rows.rem(id, bg);
  const int b = a.by_heads.quot(bg), g = a.by_heads.rem(bg, b);
  const int rb = r / kPagedRows, rl = r - rb * kPagedRows;
  int first = 0, parts = 1, rows = 0;
  if (b < p.B) {
    const int32_t* unit = a.unit + ((long long)bg * a.row_blocks + rb) * 4;
    first = unit[0];
    parts = unit[1];
    rows = unit[2];
  }
  const bool live = parts > 1 && rl < rows;
  if constexpr (RW == 1) {
    if (!live) return;
  }
  float M = kNoMax, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = sl; live && s0 < parts; s0 += SL * U) {
    float ms[U], ls[U];
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long at = ((long long)first + (long long)min(s0 + u * SL, parts - 1) * a.row_blocks) * a.part_rows + rl;
      ms[u] = a.ml_part[2 * at];
      ls[u] = a.ml_part[2 * at + 1];
      v[u] = *(const f32x4*)(a.o_part + at * D + 4 * c);
    }
    float top = M;
#pragma unroll
    for (int u = 0; u < U; ++u) top = fmaxf(top, ms[u]);
    const float f = fast_exp2(M - top);
    L *= f;
    acc *= f;
    M = top;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s0 + u * SL < parts) {
        const float w = fast_exp2(ms[u] - M);
        L += w * ls[u];
        acc += w * v[u];
      }
  }
  lds_o[rw][sl][c] = acc;
  if (c == 0) {
    lds_m[rw][sl] = M;
    lds_l[rw][sl] = L;
  }
  __syncthreads();
  if (sl > 0 || !live) return;
#pragma unroll
  for (int s = 0; s < SL; ++s) M = fmaxf(M, lds_m[rw][s]);
  L = 0.f;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < SL; ++s) {
    const float w = fast_exp2(lds_m[rw][s] - M);
    L += w * lds_l[rw][s];
    acc += w * lds_o[rw][s][c];
  }
  const int nr = a.by_group.quot(r), head = g * p.G + a.by_group.rem(r, nr);
  const long long el = (((long long)b * p.Ln + nr) * p.Hq + head) * D + 4 * c;
  const float inv = 1.0f / L;
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = L == 0.f ? 0.f : acc[e] * inv;
  if constexpr (BF16) *(u32x2*)((uint16_t*)a.o + el) = u32x2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
  else *(f32x4*)((float*)a.o + el) = acc;
  if (c == 0 && a.lse) a.lse[((long long)b * p.Hq + head) * p.Ln + nr] = L == 0.f ? -INFINITY : (M + __log2f(L)) * kLn2;
}

template <int D, int CT>
hipError_t paged_attn_of(const PagedAttnArgs& a, hipStream_t s) {
  const dim3 grid = grid_xy(a.grid);
  const int rows = a.c.G * a.c.Ln;
  if (a.plan) {
    hipLaunchKernelGGL((paged_plan_kernel<PagedShape<D, CT>::BK>), dim3(1), dim3(1024), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (rows <= 16) hipLaunchKernelGGL((paged_attn_kernel<D, CT, 1, true>), grid, dim3(256), 0, s, a);
  else if (rows <= kPagedRows) hipLaunchKernelGGL((paged_attn_kernel<D, CT, 2, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_attn_kernel<D, CT, 2, false>), grid, dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.max_chunks == 1) return e;
  const long long all = (long long)a.c.B * a.c.Hkv * rows;
  if (all >= 4 * kNumCu) hipLaunchKernelGGL((paged_join_kernel<D, CT != kFp32, 4>), grid_xy((all + 3) / 4), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_join_kernel<D, CT != kFp32, 1>), grid_xy(all), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  const bool wide = a.c.D == 128;
  if (a.c.fp8) return wide ? paged_attn_of<128, kFp8>(a, s) : paged_attn_of<64, kFp8>(a, s);
  if (a.c.bf16) return wide ? paged_attn_of<128, kBf16>(a, s) : paged_attn_of<64, kBf16>(a, s);
  return wide ? paged_attn_of<128, kFp32>(a, s) : paged_attn_of<64, kFp32>(a, s);
}

}  // namespace pd
