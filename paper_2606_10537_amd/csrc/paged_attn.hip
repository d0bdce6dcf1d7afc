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
//   No barrier and no LDS in the loop.
// * The keys of all sequences are cut into parts of nearly one size (plan below),
//   planned on the device from the lengths, so that ragged batches fill the card
//   evenly; rows whose keys are cut are joined by a second kernel.
//
// Operand layouts (lane = 16 g + n).  16x16x32 bf16: A holds row n, B column n, both
// at k = 8 g .. 8 g + 7; the result's element e is row 4 g + e of column n.
//   S^T = K Q^T: row = key, column = query row, k = channel.
//   O^T += V^T P^T over 32 keys: k slot 8 g + j is key 4 g + j of the step's first
//     16 keys (j < 4) or 4 g + j - 4 of its second, so the result of S^T is P^T
//     as it stands.  A lane reads E = D / 16 neighbouring channels of its eight keys,
//     16 lanes a whole row; a byte permutation of register pairs turns the
//     8 x E block into the A operands of E products.  Row m of product t is channel E m + t.
// 16x16x4 fp32: k = g, one value a lane; four products per 16-byte read, and the
// channels of a read are permuted alike in both operands.
#include "paged_common.h"

namespace pd {

constexpr int kPagedWaves = 4;

int paged_block_keys(bool fp32) { return kPagedWaves * (fp32 ? 16 : 32); }

// Query rows and keys of one workgroup.
struct PagedPart {
  int b, g, rb;          // sequence, KV head, row block
  int first, last;       // its blocks of keys
  int parts;             // how many the row block's keys are cut into
  bool any;
};

// The cut of all sequences' keys.  Sequence b has n_b blocks of keys for each of its
// units (KV head x row block).  With Q blocks a part, Q = ceil(all blocks / target), unit parts
// are ceil(n_b / Q) of nearly one size, numbered by sequence, head, part, row block: at
// most target + units parts in all.  Every wave finds its part with two sweeps over the
// lengths, 64 sequences at a time; `find` is a part number, or, for the join, a unit
// number (by_unit), whose first part comes back in first_part.
__device__ __forceinline__ int paged_blocks(const PagedAttnArgs& a, int b, int block_keys) {
  const PagedArgs& p = a.c;
  const int len = paged_len(p, b);
  if (len == 0 || paged_new(p, b) == 0) return 0;
  return ((a.page_idx ? a.top_k << p.log2R : len) + block_keys - 1) / block_keys;
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x += __shfl_xor(x, m);
  return x;
}

template <int BK>
__device__ __forceinline__ int paged_quota(const PagedAttnArgs& a, int lane) {
  if (a.max_chunks == 1) return 1 << 30;
  const int units = a.c.Hkv * a.row_blocks;
  long long all = 0;
  for (int b0 = 0; b0 < a.c.B; b0 += 64) all += wave_sum(b0 + lane < a.c.B ? paged_blocks(a, b0 + lane, BK) : 0);
  return (int)((all * units + a.target - 1) / a.target);
}

__device__ __forceinline__ int parts_of(int blocks, int quota) {
  return max(1, quota <= 1 ? blocks : (blocks + quota - 1) / quota);
}

template <int BK>
__device__ __forceinline__ PagedPart paged_find(const PagedAttnArgs& a, int find, int lane) {
  const int units = a.c.Hkv * a.row_blocks, quota = paged_quota<BK>(a, lane);
  PagedPart r{};
  int before = 0;
  for (int b0 = 0; b0 < a.c.B; b0 += 64) {
    const int blocks = b0 + lane < a.c.B ? paged_blocks(a, b0 + lane, BK) : 0;
    const int parts = b0 + lane < a.c.B ? parts_of(blocks, quota) * units : 0;
    int incl = parts;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const int y = __shfl_up(incl, m);
      if (lane >= m) incl += y;
    }
    const uint64_t past = __ballot(before + incl > find);
    if (past) {
      const int l = __ffsll((unsigned long long)past) - 1;
      const int n = __shfl(blocks, l);
      r.b = b0 + l;
      r.parts = parts_of(n, quota);
      int i = find - (before + __shfl(incl - parts, l));
      r.rb = i % a.row_blocks;
      i /= a.row_blocks;
      const int c = i % r.parts;
      r.g = i / r.parts;
      r.first = (int)((long long)c * n / r.parts);
      r.last = (int)((long long)(c + 1) * n / r.parts);
      r.any = true;
      return r;
    }
    before += __shfl(incl, 63);
  }
  return r;
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
  static constexpr int BK = kPagedWaves * KS;
};

// What a wave holds of one step.
template <int D, int CT>
struct PagedStep {
  using S = PagedShape<D, CT>;
  u32x4 k[S::H][S::NK];
  uint32_t v[S::VR][S::VW];
  uint32_t ke[S::H], ve[S::H];   // exponent bytes of keys 4 g .. 4 g + 3
  int pos[S::H];                 // position of the first key of each 16
};

__device__ __forceinline__ float group_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float group_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

constexpr int kFarPos = 1 << 30;   // the position of keys that are not there

// MIXED: some rows of a workgroup may see a key that others do not (several new rows, causal).
template <int D, int CT, int RT, bool MIXED>
__global__ __launch_bounds__(256, RT == 1 ? 2 : 1) void paged_attn_kernel(PagedAttnArgs a) {
  using S = PagedShape<D, CT>;
  constexpr int H = S::H, CB = S::CB, NK = S::NK, VR = S::VR, VW = S::VW, E = S::E, NT = S::NT, BK = S::BK;
  constexpr int OP = D + 4;
  __shared__ float lds_o[kPagedWaves][16][OP];
  __shared__ float lds_ml[kPagedWaves][RT * 16][2];
  const PagedArgs& p = a.c;
  const int wave = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, n = lane & 15, g4 = lane >> 4;
  const PagedPart part = paged_find<BK>(a, (int)block_id(), lane);
  if (!part.any) return;
  const int b = uniform(part.b), g = uniform(part.g);
  const int len = uniform(paged_len(p, b)), n_new = uniform(paged_new(p, b));
  const int rows = n_new * p.G, row0 = uniform(part.rb) * (RT * 16);
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
    const int rr = real ? r : row0;
    const long long q_el = (((long long)b * p.Ln + rr / p.G) * p.Hq + (long long)g * p.G + rr % p.G) * D;
    lim[t] = !real ? 0 : p.causal ? len - n_new + 1 + r / p.G : len;
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
  every = p.causal ? len - n_new + 1 + row0 / p.G : len;

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
  const int n_steps = part.last - part.first;
  int at_page[H], at_pos[H];
  bool bad = false;
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
          else bad = true;
        }
      }
    }
  };

  const uint32_t page_rows = (uint32_t)p.R;
  auto load = [&](PagedStep<D, CT>& s, int i) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int page = __builtin_amdgcn_readlane(at_page[h], i & 63);
      s.pos[h] = __builtin_amdgcn_readlane(at_pos[h], i & 63);
      const long long row = ((long long)page * p.Hkv + g) * page_rows + (s.pos[h] & (p.R - 1));
      const char* kp = (const char*)p.k_pages + row * (D * CB) + n * (D * CB) + 16 * g4;
#pragma unroll
      for (int j = 0; j < NK; ++j) s.k[h][j] = *(const u32x4*)(kp + 64 * j);
      const char* vp = (const char*)p.v_pages + row * (D * CB) + g4 * (4 * D * CB);
      // fp32: channels 64 u + 4 n.., u = 0..D/64-1; otherwise E n..
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t* w = s.v[4 * h + j];
        if constexpr (CT == kFp32) {
#pragma unroll
          for (int u = 0; u < VW / 4; ++u) *(u32x4*)(w + 4 * u) = *(const u32x4*)(vp + j * (D * CB) + 256 * u + 16 * n);
        } else if constexpr (VW == 4) {
          *(u32x4*)w = *(const u32x4*)(vp + j * (D * CB) + 16 * n);
        } else if constexpr (VW == 2) {
          *(u32x2*)w = *(const u32x2*)(vp + j * (D * CB) + 8 * n);
        } else {
          *w = *(const uint32_t*)(vp + j * (D * CB) + 4 * n);
        }
      }
      if constexpr (CT == kFp8) {
        s.ke[h] = *(const uint32_t*)(p.k_exp + row + 4 * g4);
        s.ve[h] = *(const uint32_t*)(p.v_exp + row + 4 * g4);
      }
    }
  };

  auto compute = [&](PagedStep<D, CT>& s) {
    bool whole = true, inside = true;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      whole = whole && s.pos[h] + 16 <= every;     // every row sees every key
      inside = inside && s.pos[h] + 16 <= len;     // every key is there
    }
    // Values as bf16 (or fp32), zeros where no key is: a weight of zero does not cancel
    // an infinity or a NaN.
    constexpr int W = CT == kFp32 ? VW : D / 32;
    uint32_t v[VR][W];
#pragma unroll
    for (int j = 0; j < VR; ++j) {
      if constexpr (CT == kFp8) {
#pragma unroll
        for (int w = 0; w < VW; ++w) {
          v[j][2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(s.v[j][w], 1.0f, false));
          v[j][2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(s.v[j][w], 1.0f, true));
        }
      } else {
#pragma unroll
        for (int w = 0; w < W; ++w) v[j][w] = s.v[j][w];
      }
    }
    if (!inside) {
#pragma unroll
      for (int j = 0; j < VR; ++j) {
        const bool there = s.pos[j / 4] + 4 * g4 + j % 4 < len;
#pragma unroll
        for (int w = 0; w < W; ++w) v[j][w] = there ? v[j][w] : 0u;
      }
    }
    // A key that some rows see and others do not: its value has to stay out of the
    // others even where it is not finite, which a weight of zero does not achieve.
    bool odd = false;
    if (MIXED && !whole) {
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
      odd = __any(z != z);
    }
    // Products of P V: value(j, w) gives dword w of the lane's row j, add(i, x) takes
    // product i with the accumulator from(i).
    auto products = [&](const float (&pp)[H][4], auto value, auto from, auto add) {
      if constexpr (CT == kFp32) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          f32x4 x = from(i);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            x = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(value(j, i)), pp[0][j], x, 0, 0, 0);
          add(i, x);
        }
      } else {
        // The weights are rounded to bf16 here, to nearest; their sum l is taken before.
        const u32x4 pw = {pack_bf16x2(pp[0][0], pp[0][1]), pack_bf16x2(pp[0][2], pp[0][3]),
                          pack_bf16x2(pp[H - 1][0], pp[H - 1][1]), pack_bf16x2(pp[H - 1][2], pp[H - 1][3])};
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          u32x4 w;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            w[j] = __builtin_amdgcn_perm(value(2 * j + 1, i / 2), value(2 * j, i / 2), i & 1 ? 0x07060302u : 0x05040100u);
          add(i, mfma16x16x32(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, pw), from(i)));
        }
      }
    };
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
          if constexpr (CT == kFp8) x *= exp_to_scale((s.ke[h] >> (8 * e)) & 255);
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
            x *= exp_to_scale((s.ve[h] >> (8 * e)) & 255);
            if (!whole) x = s.pos[h] + 4 * g4 + e < lim[t] ? x : 0.f;   // bytes that no row wrote
          }
          pr[h][e] = x;
        }
      if (!MIXED || !odd) {
        products(pr, [&](int j, int w) { return v[j][w]; }, [&](int i) { return o[t][i]; },
                 [&](int i, f32x4 x) { o[t][i] = x; });
      } else {
        // Row by row: the values that the row sees, its weights, and its sums alone (what a
        // value that is not finite does to the other rows' is dropped).
        for (int r = 0; r < 16; ++r) {
          const int end = __builtin_amdgcn_readlane(lim[t], r);
          float pp[H][4];
#pragma unroll
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) pp[h][e] = n == r ? pr[h][e] : 0.f;
          products(pp, [&](int j, int w) { return s.pos[j / 4] + 4 * g4 + j % 4 < end ? v[j][w] : 0u; },
                   [&](int i) { return o[t][i]; },
                   [&](int i, f32x4 x) {
#pragma unroll
                     for (int e = 0; e < 4; ++e) o[t][i][e] = n == r ? x[e] : o[t][i][e];
                   });
        }
      }
    }
  };

  if (n_steps > 0) {
    PagedStep<D, CT> s0, s1;
    locate(0);
    load(s0, 0);
    for (int i = 0;;) {
      if (i + 1 < n_steps) {
        if (((i + 1) & 63) == 0) locate(i + 1);
        load(s1, i + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      compute(s0);
      if (++i >= n_steps) break;
      if (i + 1 < n_steps) {
        if (((i + 1) & 63) == 0) locate(i + 1);
        load(s0, i + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      compute(s1);
      if (++i >= n_steps) break;
    }
  }

  // Join of the four waves.  Column n of the results is query row n.
  const bool wave_bad = __any(bad);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l[t] = group_sum(l[t]);
    if (wave_bad) l[t] = NAN;
    if (g4 == 0) {
      lds_ml[wave][t * 16 + n][0] = m[t];
      lds_ml[wave][t * 16 + n][1] = l[t];
    }
  }
  __syncthreads();
  const int rl = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * (D / 16);
  const long long slot = (long long)block_id() * a.part_rows;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float top = lds_ml[0][t * 16 + n][0];
#pragma unroll
    for (int w = 1; w < kPagedWaves; ++w) top = fmaxf(top, lds_ml[w][t * 16 + n][0]);
    const float f = fast_exp2(m[t] - top);
    // fp32: product 4 u + e has channel 64 u + 4 (4 g + r) + e, otherwise t has E (4 g + r) + t.
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < NT; i += 4) {
        const int ch = CT == kFp32 ? 16 * i + 4 * (4 * g4 + r) : E * (4 * g4 + r) + i;
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
        const float inv = L == 0.f ? 0.f : 1.0f / L;
        const int head = g * p.G + r % p.G, nr = r / p.G;
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
// parts' order.  One workgroup a row; its threads take four channels of every
// (1024 / D)-th part each, all loads of eight parts in flight, and are joined through LDS.
template <int BK, int D, bool BF16>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a) {
  constexpr int T = D / 4, SL = 256 / T, U = 8;   // threads of a row, slices of the parts
  __shared__ f32x4 lds_o[SL][T];
  __shared__ float lds_m[SL], lds_l[SL];
  const PagedArgs& p = a.c;
  const int lane = threadIdx.x & 63;
  const int rows_all = p.G * p.Ln;
  const long long id = block_id();
  const int r = (int)(id % rows_all);
  const long long bg = id / rows_all;
  const int g = (int)(bg % p.Hkv), b = (int)(bg / p.Hkv);
  if (b >= p.B || r >= paged_new(p, b) * p.G) return;
  const int quota = paged_quota<BK>(a, lane);
  const int parts = parts_of(paged_blocks(a, b, BK), quota);
  if (parts == 1) return;
  // The number of the row's first part: all parts of the sequences before, then of the heads before.
  int before = 0;
  for (int b0 = 0; b0 < b; b0 += 64)
    before += wave_sum(b0 + lane < b ? parts_of(paged_blocks(a, b0 + lane, BK), quota) : 0);
  const int rb = r / kPagedRows;
  const long long first = ((long long)before * p.Hkv + (long long)g * parts) * a.row_blocks + rb;
  const int rl = r - rb * kPagedRows;
  const int c = threadIdx.x % T, sl = threadIdx.x / T;
  float M = kNoMax, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = sl; s0 < parts; s0 += SL * U) {
    float ms[U], ls[U];
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long at = (first + (long long)min(s0 + u * SL, parts - 1) * a.row_blocks) * a.part_rows + rl;
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
  lds_o[sl][c] = acc;
  if (c == 0) {
    lds_m[sl] = M;
    lds_l[sl] = L;
  }
  __syncthreads();
  if (sl > 0) return;
#pragma unroll
  for (int s = 0; s < SL; ++s) M = fmaxf(M, lds_m[s]);
  L = 0.f;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < SL; ++s) {
    const float w = fast_exp2(lds_m[s] - M);
    L += w * lds_l[s];
    acc += w * lds_o[s][c];
  }
  const int head = g * p.G + r % p.G, nr = r / p.G;
  const long long el = (((long long)b * p.Ln + nr) * p.Hq + head) * D + 4 * c;
  const float inv = 1.0f / L;
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = L == 0.f ? 0.f : acc[e] * inv;
  if constexpr (BF16) *(u32x2*)((uint16_t*)a.o + el) = u32x2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
  else *(f32x4*)((float*)a.o + el) = acc;
  if (c == 0 && a.lse) a.lse[((long long)b * p.Hq + head) * p.Ln + nr] = L == 0.f ? -INFINITY : (M + __log2f(L)) * kLn2;
}

template <int D, int CT, int RT>
void paged_attn_rows(const PagedAttnArgs& a, hipStream_t s) {
  if (a.c.causal && a.c.Ln > 1) hipLaunchKernelGGL((paged_attn_kernel<D, CT, RT, true>), grid_xy(a.grid), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_attn_kernel<D, CT, RT, false>), grid_xy(a.grid), dim3(256), 0, s, a);
}

template <int D, int CT>
hipError_t paged_attn_of(const PagedAttnArgs& a, hipStream_t s) {
  const int rows = a.c.G * a.c.Ln;
  if (rows <= 16) paged_attn_rows<D, CT, 1>(a, s);
  else paged_attn_rows<D, CT, 2>(a, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.max_chunks == 1) return e;
  hipLaunchKernelGGL((paged_join_kernel<PagedShape<D, CT>::BK, D, CT != kFp32>),
                     grid_xy((long long)a.c.B * a.c.Hkv * rows), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  const bool wide = a.c.D == 128;
  if (a.c.fp8) return wide ? paged_attn_of<128, kFp8>(a, s) : paged_attn_of<64, kFp8>(a, s);
  if (a.c.bf16) return wide ? paged_attn_of<128, kBf16>(a, s) : paged_attn_of<64, kBf16>(a, s);
  return wide ? paged_attn_of<128, kFp32>(a, s) : paged_attn_of<64, kFp32>(a, s);
}

}  // namespace pd
