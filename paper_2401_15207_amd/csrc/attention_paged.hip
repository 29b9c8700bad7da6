// Attention of new tokens over a paged cache, forward only: bf16 and fp32, grouped heads, a sliding window, from one token a sequence to chunks.
//
//   s_j = scale q . k_j over the keys j that a row sees (at most its own position, more than position - window, on pages that there are)
//   out = sum_j exp(s_j) v_j / sum_j exp(s_j),  lse = log2 sum_j exp(s_j)
//
// The new rows of a sequence and the query heads that share a key head make one list of rows, m = token * group + head: it is their tile that
// meets a tile of keys, so keys and values are read once for all heads of a group.  One pass over the keys with a running maximum and sum
// per row (log2 domain), as in attention.hip, whose conventions for the matrix instruction's operands and for LDS tiles these kernels share.
//   few_k    32 rows a workgroup: all four wavefronts hold the same rows and take turns at the blocks of 32 keys, each through LDS tiles of its own
//            without any barrier, and their results are joined at the end.  Bound by reading the cache.  Lengths are known on the device only, and
//            differ: the keys of all sequences and heads, one after the other, are cut into equal runs, a workgroup each, wherever that falls.
//            A token each of 64 sequences of up to 8000, 32 / 8 heads of 128 bf16 (1.04 GB): 189 us with its join, 5.5 TB/s (a workgroup a sequence and head 253).
//   few_whole_k  the same, one workgroup a block of rows and key head, where runs would be too short.  One token over 500, 32 / 32 heads: 8.4 us, the chain
//            of its loads, products and joins.
//   mixed_k  128 rows a workgroup, 32 a wavefront, which share tiles of 64 keys.  Its first workgroups take the sequences of few rows.
//            Chunks of 700 to 1024 of 4 sequences over up to 4096, 32 / 32 heads bf16: 188 to 198 us by the card, 770 to 815 TFLOP/s (a large product 1250).  No single unit
//            bounds them: the matrix pipes are busy 41 % of the time; LDS reads (16 KB a wavefront for 16 instructions of 32 cycles) weigh most and the phases overlap in part
//            (an earlier state of 231 us: without loads 198, without exponentials 205, without LDS reads 157).  With at most 256 workgroups (1024 over none 30 us, products 7) a
//            SIMD has one wavefront, which waits out each tile: 1.9 us, products 0.43.  fp32, 1024 over none 152 us of 56: one workgroup a compute unit (131 KB of LDS), the
//            longest with twice the mean work, products and exponentials one after the other.
//   join_k   rows whose keys fell to several workgroups: the parts, weighted by their maxima.
//
// bf16: exponentials are rounded to bf16 for the product with v, which is what the matrix instruction takes, as in attention.hip; their sum, the maxima and all products' sums are
// fp32.  Results are off by 0.0021 of their size instead of 0.0016 (one rounding of the result alone); keeping what that rounding leaves would take the product twice.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "lds_allowed.h"
#include "paged_cache.h"

namespace hift {
namespace {

#define UNIFORM(x) __builtin_amdgcn_readfirstlane(x)

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef short v8i16 __attribute__((ext_vector_type(8)));

constexpr int FEW = 32;    // rows of few_k
constexpr int KB = 32;     // keys of a block
constexpr int GROUP = 16;  // keys that surely lie on one page

struct Args {
  CacheView c;
  int heads, group;     // query heads; those that share a key head
  int64_t rows, ldq, ldo;
  int max_new, window;  // window 0: none
  float scale_log2e;
  const void* q;
  void* out;
  float* lse;           // [rows, heads] or null
  int few_upto;         // sequences of at most so many rows are few_k's, the others mixed_k's
  int few_blocks, many_blocks;  // blocks of rows of the longest sequence
  int runs;             // few_k's workgroups, or 0
  int few_first;        // mixed_k: workgroups that few rows take
  int split, chunk;     // mixed_k: workgroups along the keys of a block of many rows, and keys of each
  int64_t* plan;        // [0]: steps in all; [1 + e]: steps before entry e
  float2* part_ml;      // (maximum, sum of exponentials) of shared rows: few_k [run][2][FEW], a run's first and last block of rows; mixed_k [rows][heads][split]
  float* part;          // [..][HD] their sums
};

// ---- tiles of a type and width ----
// A row of a tile is HD elements without padding; its 16-byte piece c lies at piece position c ^ swizzle(row), which spreads what one LDS
// instruction reads over the banks.  HD: 64 or 128; narrower heads are zeros behind their width, and the blocks of 32 columns behind it, from NB_ on, take no
// part in the products.
template <typename T, int HD, int NB_>
struct Tile {
  static constexpr int ROWB = HD * (int)sizeof(T), PPR = ROWB / 16, RPI = 64 / PPR, NB = NB_;
  static constexpr int IPG = GROUP / RPI;  // load instructions of 16 keys
  static constexpr int BLOCKB = KB * ROWB;
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int NQ = F32 ? NB * 4 : NB * 2;  // fragments of a row
  typedef typename std::conditional<F32, f32x4, bf16x8>::type Frag;  // 16 bytes of a row

  __device__ static __forceinline__ int swizzle(int r) {
    if constexpr (F32) return ((r >> 2) & 1) << 3 | ((r >> 3) & 1) << 2 | (r & 3);
    return PPR == 16 ? (r & 3) << 2 | ((r >> 2) & 3) : (r >> 1) & 7;
  }
  // which row of a 32-key block the score fragments' lane r reads: for bf16 with bits 2 and 3 exchanged, so that scores are operands as they lie
  __device__ static __forceinline__ int key_row(int r) { return F32 ? r : (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }
  // the key of score element e in a lane of half fh
  __device__ static __forceinline__ int key_of(int e, int fh) { return F32 ? 8 * (e >> 2) + 4 * fh + (e & 3) : 16 * (e >> 3) + 8 * fh + (e & 7); }

  // Requests 16 keys from token `key0` on (all on one page) of one of the cache's arrays into LDS; keys from `end` on, and those of a page that is
  // not there, arrive as zeros.  vo: offsets of the lane's pieces within 16 keys (see offsets).
  int64_t page_bytes;
  int head_at, slots, row_bytes;  // the head's first key within a page; slots of a page less one; bytes of a key
  __device__ __forceinline__ Tile(const CacheView& c, int kv_head)
      : page_bytes(c.page_stride * (int64_t)sizeof(T)), head_at(kv_head * c.page), slots(c.page - 1), row_bytes(c.head_dim * (int)sizeof(T)) {}
  // PAST: keys that no other workgroup reads leave the caches first.
  template <bool PAST = false>
  __device__ __forceinline__ void request(const void* array, int key0, int page, int end, const uint32_t (&vo)[IPG], uint32_t lds) const {
    const uint64_t a = reinterpret_cast<uint64_t>(array) + (uint64_t)((int64_t)max(page, 0) * page_bytes + (int64_t)(head_at + (key0 & slots)) * row_bytes);
    const int n = page < 0 ? 0 : min(max(end - key0, 0), GROUP);
    const hift_u32x4 rs = {(uint32_t)UNIFORM((int)(uint32_t)a), (uint32_t)UNIFORM((int)((uint32_t)(a >> 32) & 0xFFFFu)),
                           (uint32_t)UNIFORM(n * row_bytes), 0x00020000u};
#pragma unroll
    for (int i = 0; i < IPG; ++i) load_to_lds_b128<PAST>(rs, lds + i * 1024, vo[i], 0);
  }
  // 32 keys, on one page or two
  template <bool PAST>
  __device__ __forceinline__ void request(const void* array, int key0, int pa, int pb, int end, const uint32_t (&vo)[IPG], uint32_t lds) const {
    request<PAST>(array, key0, pa, end, vo, lds);
    request<PAST>(array, key0 + GROUP, pb, end, vo, lds + GROUP * ROWB);
  }
  __device__ static __forceinline__ void offsets(uint32_t (&vo)[IPG], int lane, int head_dim) {
#pragma unroll
    for (int i = 0; i < IPG; ++i) {
      const int r = i * RPI + lane / PPR, c = (lane % PPR) ^ swizzle(r);
      vo[i] = c * 16 < head_dim * (int)sizeof(T) ? (uint32_t)(r * head_dim * (int)sizeof(T) + c * 16) : 0x80000000u;
    }
  }
  // A row of queries as fragments; piece i of the lane: bytes 32 i + 16 fh
  __device__ static __forceinline__ void load_row(Frag (&f)[NQ], const T* row, bool ok, int head_dim, int fh) {
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      hift_u32x4 t = {0u, 0u, 0u, 0u};
      if (ok && (2 * i + fh) * 16 < head_dim * (int)sizeof(T)) t = *reinterpret_cast<const hift_u32x4*>(reinterpret_cast<const unsigned char*>(row) + (2 * i + fh) * 16);
      f[i] = __builtin_bit_cast(Frag, t);
    }
  }
  struct Address {
    int k[NQ];                  // piece of the lane's key row
    int v[F32 ? 2 : NB][2];     // bf16: transposing reads by column block and half; fp32: see value_of
  };
  __device__ static __forceinline__ void addresses(Address& a, int lane) {
    const int fr = lane & 31, fh = lane >> 5, r = key_row(fr);
#pragma unroll
    for (int i = 0; i < NQ; ++i) a.k[i] = r * ROWB + (((2 * i + fh) ^ swizzle(r)) * 16);
    if constexpr (!F32) {
      const int sl = lane & 15;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const int row = 8 * fh + (sl >> 2) + 4 * hh, col = nb * 32 + 16 * ((lane >> 4) & 1) + 4 * (sl & 3);
          a.v[nb][hh] = row * ROWB + (((col >> 3) ^ swizzle(row)) * 16) + (col & 7) * 2;
        }
    }
  }
  // scores of the lane's query row against the block's keys
  __device__ static __forceinline__ f32x16 scores(const unsigned char* k, const Address& a, const Frag (&q)[NQ]) {
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
    Frag f[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) f[i] = *reinterpret_cast<const Frag*>(k + a.k[i]);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      if constexpr (F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(f[i][j], q[i][j], s, 0, 0, 0);
      } else {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i], q[i], s, 0, 0, 0);
      }
    }
    return s;
  }
  // bf16: values of keys 16 t ..+15 of a block, columns 32 nb ..+31, as the matrix instruction takes them
  __device__ static __forceinline__ bf16x8 value_frag(const unsigned char* v, const Address& a, int t, int nb) {
    const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4i16 __attribute__((address_space(3)))*)(v + t * 16 * ROWB + a.v[nb][0]));
    const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4i16 __attribute__((address_space(3)))*)(v + t * 16 * ROWB + a.v[nb][1]));
    const v8i16 both = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8, both);
  }
  // out += p (of the block's keys) times its values.  Lane: query row lane % 32; element e of out[nb]: column 32 nb + 8 (e / 4) + 4 (lane / 32) + e % 4
  __device__ static __forceinline__ void values(f32x16 (&out)[NB], const unsigned char* v, const Address& a, const f32x16& p, int lane) {
    if constexpr (F32) {
      const int fr = lane & 31, fh = lane >> 5;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = key_of(e, 0) + 4 * fh;
        float f[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) f[nb] = *reinterpret_cast<const float*>(v + key * ROWB + (((nb * 8 + (fr >> 2)) ^ swizzle(key)) * 16) + (fr & 3) * 4);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) out[nb] = __builtin_amdgcn_mfma_f32_32x32x2f32(f[nb], p[e], out[nb], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        bf16x8 pf, vf[NB];
#pragma unroll
        for (int e = 0; e < 8; ++e) pf[e] = static_cast<__bf16>(p[8 * t + e]);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) vf[nb] = value_frag(v, a, t, nb);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) out[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[nb], pf, out[nb], 0, 0, 0);
      }
    }
  }
};

// ---- a row's running softmax (log2 domain) ----
template <int NB>
struct Running {
  float m = -INFINITY, l = 0.f;  // reference of the exponentials, equal in a row's two lanes; sum of the lane's exponentials
  f32x16 o[NB];
  __device__ __forceinline__ Running() {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[nb][e] = 0.f;
  }
  // Turns raw scores into exponentials.  The reference is raised, and the sums rescaled, only where a score exceeds it by more than 2^8: what is
  // left stays below 2^8, which costs bf16, a relative format, nothing.
  template <int N>
  __device__ __forceinline__ void take(f32x16 (&s)[N], float scale_log2e) {
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[b][e]);
    top = fmaxf(top, __shfl_xor(top, 32, 64)) * scale_log2e;
    if (__builtin_amdgcn_ballot_w64(top > m + 8.0f) != 0) {
      const float now = fmaxf(m, top);
      const float by = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
      l *= by;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[nb][e] *= by;
      m = now;
    }
    const float ref = m == -INFINITY ? 0.f : m;  // a row that has seen nothing yet: exp2(-inf - 0) = 0
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[b][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][e], scale_log2e, -ref));
        l += s[b][e];
      }
  }
};

// The keys [from, to) that tokens [t0, t1] of a sequence read; `from` is a multiple of 32.
__device__ __forceinline__ void keys_of(const CacheSeq& of, int t0, int t1, int window, int& from, int& to) {
  to = min(of.total, of.cached + t1 + 1);
  from = window > 0 ? max(0, of.cached + t0 - window + 1) & ~(KB - 1) : 0;
  from = min(from, to & ~(KB - 1));
}

// Where a row of the list m = token * group + head goes
struct RowAt {
  int64_t row;
  int head, pos;
  bool ok;
};
__device__ __forceinline__ RowAt row_at(const Args& p, const CacheSeq& of, int kv_head, int m) {
  RowAt r;
  const int token = m / p.group;
  r.ok = token < of.fresh;
  r.row = of.row0 + (r.ok ? token : 0);
  r.head = kv_head * p.group + (m - token * p.group);
  r.pos = of.cached + token;
  return r;
}

// Scores of keys that the lane's row does not see become -inf.  a, b: whether the pages of the block's halves are there.
template <class L>
__device__ __forceinline__ void mask_scores(f32x16& s, int key0, int fh, int end, int pos, int total, int window, bool a, bool b) {
  const int last = min(min(pos, total - 1), end - 1) - key0, first = window > 0 ? pos - window + 1 - key0 : -1;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int j = L::key_of(e, 0) + (L::key_of(0, 1) - L::key_of(0, 0)) * fh;
    const bool ok = (j <= last) & (j >= first) & (L::key_of(e, 0) < GROUP ? a : b);
    s[e] = ok ? s[e] : -INFINITY;
  }
}

template <typename T>
__device__ __forceinline__ void store_out(const Args& p, const RowAt& r, int c, float v) {
  if (c < p.c.head_dim) ((T*)p.out)[r.row * p.ldo + (int64_t)r.head * p.c.head_dim + c] = from_f32<T>(v);
}

// ---- few rows ----
constexpr int PAGED = 64 * GROUP;  // keys whose page numbers a wavefront holds, a lane each 16
constexpr int STEP = 4 * KB;       // keys that a workgroup of four wavefronts takes at a time

// An entry: a block of 32 rows of a sequence, entry s * few_blocks + block; its key heads take `steps` steps each.
struct Entry {
  CacheSeq of;
  int m0, n_rows, t0, t1, from, to, steps;
  __device__ __forceinline__ Entry(const Args& p, int s, int block) : of(cache_seq(p.c, s, p.rows, p.max_new)), m0(block * FEW) {
    const int all = of.fresh * p.group;
    n_rows = all <= p.few_upto ? min(all - m0, FEW) : 0;
    steps = 0;
    if (n_rows <= 0) return;
    t0 = m0 / p.group;
    t1 = (m0 + n_rows - 1) / p.group;
    keys_of(of, t0, t1, p.window, from, to);
    steps = max(1, (to - from + STEP - 1) / STEP);
  }
};

// Steps [step0, step1) of an entry's key head, by W wavefronts.  shared: -1 where these are all its steps, otherwise the place [..][FEW] its results go to.
template <typename T, int HD, int NB_, int W, bool PAST>
__device__ __forceinline__ void few_rows(const Args& p, const Entry& en, int s, int kv_head, int step0, int step1, int64_t shared, unsigned char* lds, float2 (*ml)[FEW]) {
  typedef Tile<T, HD, NB_> L;
  constexpr int NB = L::NB, IPB = 2 * L::IPG;  // loads of a block of keys
  const int tid = threadIdx.x, lane = tid & 63, wave = UNIFORM(tid >> 6), fr = lane & 31, fh = lane >> 5;
  const int from = UNIFORM(en.from + step0 * STEP), to = UNIFORM(min(en.to, en.from + step1 * STEP)), n_rows = UNIFORM(en.n_rows);
  // page numbers of the keys from `k0` on
  auto pages_from = [&](int k0) { return k0 + lane * GROUP < to ? cache_page_any(p.c, s, k0 + lane * GROUP) : -1; };
  int paged = from, pages = pages_from(paged);
  const RowAt at = row_at(p, en.of, kv_head, en.m0 + fr);
  typename L::Frag q[L::NQ];
  L::load_row(q, (const T*)p.q + at.row * p.ldq + (int64_t)at.head * p.c.head_dim, at.ok, p.c.head_dim, fh);
  uint32_t vo[L::IPG];
  L::offsets(vo, lane, p.c.head_dim);
  typename L::Address ad;
  L::addresses(ad, lane);
  unsigned char* Kb = lds + wave * (2 * L::BLOCKB);
  unsigned char* Vb = Kb + L::BLOCKB;
  const uint32_t lk = (uint32_t)reinterpret_cast<uintptr_t>(Kb), lv = (uint32_t)reinterpret_cast<uintptr_t>(Vb);
  const L head(p.c, kv_head);

  int key0 = from + wave * KB, pa = -1, pb = -1;
  if (key0 < to) {
    const int g = wave * (KB / GROUP);
    pa = __builtin_amdgcn_readlane(pages, g);
    pb = __builtin_amdgcn_readlane(pages, g + 1);
    head.template request<PAST>(p.c.k, key0, pa, pb, to, vo, lk);
    head.template request<PAST>(p.c.v, key0, pa, pb, to, vo, lv);
  }
  Running<NB> run;
  // the compiler waits for the rows here, once, and not in the loop, where it would wait for everything on its way
#pragma unroll
  for (int k = 0; k < L::NQ; ++k) asm volatile("" : "+v"(q[k]));
  const int pos_lo = UNIFORM(en.of.cached + en.t0), pos_hi = UNIFORM(en.of.cached + en.t1);
  for (; key0 < to; key0 += W * KB) {
    const int next = key0 + W * KB;
    const bool more = next < to;
    if (next >= paged + PAGED) {  // PAGED is a multiple of W KB
      paged += PAGED;
      pages = pages_from(paged);
    }
    const int g = (next - paged) / GROUP;
    const int na = more ? __builtin_amdgcn_readlane(pages, g) : -1, nb = more ? __builtin_amdgcn_readlane(pages, g + 1) : -1;
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(IPB) : "memory");  // the keys are there, their values on the way
    f32x16 sc[1];
    sc[0] = L::scores(Kb, ad, q);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) head.template request<PAST>(p.c.k, next, na, nb, to, vo, lk);
    const bool plain = (pa | pb) >= 0 && key0 + KB <= to && key0 + KB - 1 <= pos_lo && (p.window == 0 || key0 > pos_hi - p.window);
    if (!plain) mask_scores<L>(sc[0], key0, fh, to, at.pos, en.of.total, p.window, pa >= 0, pb >= 0);
    run.take(sc, p.scale_log2e);
    if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(IPB) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    L::values(run.o, Vb, ad, sc[0], lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) head.template request<PAST>(p.c.v, next, na, nb, to, vo, lv);
    pa = na; pb = nb;
  }
  run.l += __shfl_xor(run.l, 32, 64);

  // the wavefronts' results, joined
  if (fh == 0) ml[wave][fr] = make_float2(run.m, run.l);
  float* sums = reinterpret_cast<float*>(lds);  // [wave][FEW][HD]
  __syncthreads();
  if (fr < n_rows) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(sums + (wave * FEW + fr) * HD + nb * 32 + 8 * g + 4 * fh) =
            f32x4{run.o[nb][4 * g], run.o[nb][4 * g + 1], run.o[nb][4 * g + 2], run.o[nb][4 * g + 3]};
  }
  __syncthreads();
  for (int i = tid; i < n_rows * (NB * 32); i += 64 * W) {
    const int m = i / (NB * 32), c = i % (NB * 32);
    float top = ml[0][m].x;
#pragma unroll
    for (int w = 1; w < W; ++w) top = fmaxf(top, ml[w][m].x);
    const float ref = top == -INFINITY ? 0.f : top;
    float l = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float by = __builtin_amdgcn_exp2f(ml[w][m].x - ref);
      l = fmaf(by, ml[w][m].y, l);
      o = fmaf(by, sums[(w * FEW + m) * HD + c], o);
    }
    if (shared < 0) {
      const RowAt r = row_at(p, en.of, kv_head, en.m0 + m);
      store_out<T>(p, r, c, l > 0.f || l != l ? o / l : 0.f);
      if (c == 0 && p.lse) p.lse[r.row * p.heads + r.head] = top + __builtin_amdgcn_logf(l);
    } else {
      p.part[(shared + m) * HD + c] = o;
      if (c == 0) p.part_ml[shared + m] = make_float2(top, l);
    }
  }
}

// One workgroup a block of rows and key head
template <typename T, int HD, int NB, int W, bool PAST>
__device__ __forceinline__ void few_whole(const Args& p, int i, unsigned char* lds, float2 (*ml)[FEW]) {
  const int pair = i / p.few_blocks, block = p.few_blocks - 1 - i % p.few_blocks, s = pair / p.c.kv_heads;
  const Entry en(p, s, block);
  if (en.steps > 0) few_rows<T, HD, NB, W, PAST>(p, en, s, pair % p.c.kv_heads, 0, en.steps, -1, lds, ml);
}
template <typename T, int HD, int NB, int W, bool PAST>
__global__ void __launch_bounds__(64 * W) few_whole_k(Args p) {
  extern __shared__ unsigned char lds[];  // [wave][K | V] blocks; at the end of a block of rows [wave][row][HD] sums
  __shared__ float2 ml[W][FEW];
  few_whole<T, HD, NB, W, PAST>(p, (int)blockIdx.x, lds, ml);
}

// Equal runs of steps: run w is [w all / runs, (w + 1) all / runs), rounded down, with no more runs than steps, so that none is empty.
__device__ __forceinline__ int64_t run_start(int w, int64_t all, int runs) { return w * all / runs; }
__device__ __forceinline__ int run_of(int64_t step, int64_t all, int runs) { return (int)(((step + 1) * runs - 1) / all); }
template <typename T, int HD, int NB, bool PAST>
__global__ void __launch_bounds__(256) few_k(Args p) {
  extern __shared__ unsigned char lds[];
  __shared__ float2 ml[4][FEW];
  const int kv_heads = p.c.kv_heads;
  // steps of all entries, and where this run begins
  __shared__ int64_t sums[256];
  __shared__ int64_t found_before;
  __shared__ int found;
  const int tid = threadIdx.x, entries = p.c.sequences * p.few_blocks, each = (entries + 255) / 256;
  const int e0 = min(tid * each, entries), e1 = min(e0 + each, entries);
  int64_t mine = 0, last = 0;
  for (int e = e0; e < e1; ++e) mine += last = (int64_t)Entry(p, e / p.few_blocks, e % p.few_blocks).steps * kv_heads;
  sums[tid] = mine;
  if (tid == 0) found = -1;
  __syncthreads();
  int64_t before = 0, all = 0;
  const int used = each ? (entries + each - 1) / each : 0;
  for (int k = 0; k < used; ++k) {
    const int64_t v = sums[k];
    before += k < tid ? v : 0;
    all += v;
  }
  const int runs = (int)min((int64_t)p.runs, all);
  if (blockIdx.x == 0 && tid == 0) p.plan[0] = all;
  if ((int)blockIdx.x >= runs) return;
  const int64_t at0 = run_start((int)blockIdx.x, all, runs), at1 = run_start((int)blockIdx.x + 1, all, runs);
  if (blockIdx.x == 0 || (before <= at0 && at0 < before + mine)) {
    int64_t b = before;
    for (int e = e0; e < e1; ++e) {
      const int64_t n = each == 1 ? last : (int64_t)Entry(p, e / p.few_blocks, e % p.few_blocks).steps * kv_heads;
      if (blockIdx.x == 0) p.plan[1 + e] = b;
      if (b <= at0 && at0 < b + n) {
        found = e;
        found_before = b;
      }
      b += n;
    }
  }
  __syncthreads();
  int e = UNIFORM(found);
  if (e < 0) return;
  int64_t at = at0, first = found_before;
  for (; at < at1 && e < entries; ++e) {
    const int s = e / p.few_blocks;
    const Entry en(p, s, e % p.few_blocks);
    while (at < at1 && at < first + (int64_t)en.steps * kv_heads) {
      const int in = UNIFORM((int)(at - first)), kv_head = UNIFORM(in / en.steps), step0 = in - kv_head * UNIFORM(en.steps);
      const int n = UNIFORM((int)min((int64_t)(en.steps - step0), at1 - at));
      const bool whole = n == en.steps;
      few_rows<T, HD, NB, 4, PAST>(p, en, s, kv_head, step0, step0 + n, whole ? -1 : ((int64_t)blockIdx.x * 2 + (step0 == 0)) * FEW, lds, ml);
      __syncthreads();  // the next block's keys go where the sums were
      at += n;
    }
    first += (int64_t)en.steps * kv_heads;
  }
}

// ---- many rows ----
// Part `part` of the keys [from, to) of a block of rows; how many parts have keys
__device__ __forceinline__ int part_of(const Args& p, int part, int& from, int& to) {
  const int n = min(p.split, max(1, (to - from + p.chunk - 1) / p.chunk));
  const int last = to;
  from += part * p.chunk;
  if (part + 1 < n) to = from + p.chunk;
  else to = part + 1 == n ? last : from;
  return n;
}
// A row's result: to the output, or as a part.  o: see Tile::values
template <typename T, int HD, int NB>
__device__ __forceinline__ void finish_row(const Args& p, const RowAt& at, const f32x16 (&o)[NB], float m, float l, int part, int parts, int fh) {
  if (!at.ok) return;
  if (parts > 1) {
    const int64_t to = (at.row * p.heads + at.head) * p.split + part;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(p.part + to * HD + nb * 32 + 8 * g + 4 * fh) = f32x4{o[nb][4 * g], o[nb][4 * g + 1], o[nb][4 * g + 2], o[nb][4 * g + 3]};
    if (fh == 0) p.part_ml[to] = make_float2(m, l);
    return;
  }
  const float inv = l > 0.f || l != l ? 1.0f / l : 0.f;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = nb * 32 + 8 * g + 4 * fh;
      if (c < p.c.head_dim) {
        Vec<T, 4> v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v.v[e] = from_f32<T>(o[nb][4 * g + e] * inv);
        *reinterpret_cast<Vec<T, 4>*>((T*)p.out + at.row * p.ldo + (int64_t)at.head * p.c.head_dim + c) = v;
      }
    }
  if (fh == 0 && p.lse) p.lse[at.row * p.heads + at.head] = m + __builtin_amdgcn_logf(l);
}

// ---- many rows, fp32 ----
template <int HD, int NB_>
__device__ __forceinline__ void many_rows_f32(const Args& p, const int index, unsigned char* lds /* [buffer][K | V] tiles of 64 keys */) {
  typedef float T;
  typedef Tile<T, HD, NB_> L;
  constexpr int NB = L::NB, KT = 2 * KB, TILEB = KT * L::ROWB, QB = 128;
  const int tid = threadIdx.x, lane = tid & 63, wave = UNIFORM(tid >> 6), fr = lane & 31, fh = lane >> 5;
  int i = index / p.split;
  const int part = index - i * p.split, kv_head = i % p.c.kv_heads;  // in the order of many_rows_bf16
  i /= p.c.kv_heads;
  const int block = p.many_blocks - 1 - i % p.many_blocks, s = i / p.many_blocks;
  const CacheSeq of = cache_seq(p.c, s, p.rows, p.max_new);
  const int n_rows = of.fresh * p.group;
  if (n_rows <= p.few_upto || block * QB >= n_rows) return;
  const int m0 = block * QB, m_last = min(n_rows, m0 + QB) - 1;
  int from, to;
  keys_of(of, m0 / p.group, m_last / p.group, p.window, from, to);
  const int parts = part_of(p, part, from, to);
  if (part >= parts) return;

  const int w0 = m0 + wave * 32;  // this wavefront's rows; their first and last positions
  const int pos_lo = of.cached + min(w0, m_last) / p.group, pos_hi = of.cached + min(w0 + 31, m_last) / p.group;
  const RowAt at = row_at(p, of, kv_head, w0 + fr);
  typename L::Frag q[L::NQ];
  L::load_row(q, (const T*)p.q + at.row * p.ldq + (int64_t)at.head * p.c.head_dim, at.ok, p.c.head_dim, fh);
  uint32_t vo[L::IPG];
  L::offsets(vo, lane, p.c.head_dim);
  typename L::Address ad;
  L::addresses(ad, lane);
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>(lds);
  const int tiles = (to - from + KT - 1) / KT;
  // every wavefront brings 16 keys of a tile
  auto page = [&](int key) { return UNIFORM(key < to ? cache_page(p.c, s, key) : -1); };
  __shared__ int pages_there[2][4];
  const L head(p.c, kv_head);
  auto request = [&](int tile, int pg) __attribute__((always_inline)) {
    const int key0 = from + tile * KT + wave * GROUP;
    const uint32_t dst = lds0 + (tile & 1) * (2 * TILEB) + wave * (GROUP * L::ROWB);
    head.request(p.c.k, key0, pg, to, vo, dst);
    head.request(p.c.v, key0, pg, to, vo, dst + TILEB);
    if (lane == 0) pages_there[tile & 1][wave] = pg >= 0;
  };
  Running<NB> run;
  int pg = page(from + wave * GROUP);
  if (tiles > 0) request(0, pg);
  for (int t = 0; t < tiles; ++t) {
    const int key0 = from + t * KT;
    pg = t + 1 < tiles ? page(key0 + KT + wave * GROUP) : -1;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // the tile is complete; nobody reads the other buffer any more
    if (t + 1 < tiles) request(t + 1, pg);
    if (key0 > pos_hi || (p.window > 0 && key0 + KT - 1 <= pos_lo - p.window) || w0 > m_last) continue;  // nothing for this wavefront
    const unsigned char* Kb = lds + (t & 1) * (2 * TILEB);
    const int* there = pages_there[t & 1];
    f32x16 sc[2];
    sc[0] = L::scores(Kb, ad, q);
    sc[1] = L::scores(Kb + L::BLOCKB, ad, q);
    const bool plain = (there[0] & there[1] & there[2] & there[3]) && key0 + KT <= to && key0 + KT - 1 <= pos_lo && (p.window == 0 || key0 > pos_hi - p.window);
    if (!plain) {
#pragma unroll
      for (int b = 0; b < 2; ++b) mask_scores<L>(sc[b], key0 + b * KB, fh, to, at.pos, of.total, p.window, there[2 * b] != 0, there[2 * b + 1] != 0);
    }
    run.take(sc, p.scale_log2e);
    L::values(run.o, Kb + TILEB, ad, sc[0], lane);
    L::values(run.o, Kb + TILEB + L::BLOCKB, ad, sc[1], lane);
  }
  run.l += __shfl_xor(run.l, 32, 64);
  finish_row<T, HD, NB>(p, at, run.o, run.m, run.l, part, parts, fh);
}

// ---- many rows, bf16 ----
// 128 rows a workgroup, 32 a wavefront, two workgroups a compute unit (chunks: 188 us; 256 rows in eight wavefronts the same; 64 rows a wavefront would halve the
// LDS reads, but spilled as compiled: 663).  Within a wavefront the products of one block of 32 keys run beside the exponentials of
// the one before:
//   scores of block i (8 MFMAs)     in turn with the exponentials of block i - 1 (products first, then exponentials: 4096 over none, 16 / 2 heads 109 us, in turn 99)
//   P V of block i - 1 (8 MFMAs)    beside the row maxima of block i

// The sequence that has `rank` longer ones before it; with more than 256 of them, which fill the chip in any order, the rank-th.
__device__ __forceinline__ int longest(const Args& p, int rank, int* lengths) {
  const int n = p.c.sequences, tid = threadIdx.x;
  if (n == 1 || n > 256) return rank;
  int mine = 0;
  if (tid < n) {
    const CacheSeq of = cache_seq(p.c, tid, p.rows, p.max_new);
    lengths[tid] = mine = of.fresh ? of.total : -1;
  }
  __syncthreads();
  int before = 0;
  if (tid < n)
    for (int k = 0; k < n; ++k) before += (lengths[k] > mine) | ((lengths[k] == mine) & (k < tid));
  __syncthreads();
  if (tid < n && before == rank) lengths[0] = tid;
  __syncthreads();
  const int s = UNIFORM(lengths[0]);
  __syncthreads();
  return s;
}

template <int HD, int NB_>
__device__ __forceinline__ void many_rows_bf16(const Args& p, const int index, unsigned char* lds /* [2] tiles of K | [3] of V */) {
  typedef Tile<bf16, HD, NB_> L;
  constexpr int NB = L::NB, NQ = L::NQ, KT = 2 * KB, TILEB = KT * L::ROWB, QB = 128;
  const int tid = threadIdx.x, lane = tid & 63, wave = UNIFORM(tid >> 6), fr = lane & 31, fh = lane >> 5;
  // Workgroups start in the order of their index: those with the most keys first.  Neighbours take different heads, so that the workgroups of a head, which read
  // the same keys, are on one of the eight dies where the heads are a multiple of them.
  int i = index / p.split;
  const int part = index - i * p.split, kv_head = i % p.c.kv_heads;
  i /= p.c.kv_heads;
  const int block = p.many_blocks - 1 - i % p.many_blocks, s = longest(p, i / p.many_blocks, reinterpret_cast<int*>(lds));
  const CacheSeq of = cache_seq(p.c, s, p.rows, p.max_new);
  const int n_rows = of.fresh * p.group;
  if (n_rows <= p.few_upto || block * QB >= n_rows) return;
  const int m0 = block * QB, m_last = min(n_rows, m0 + QB) - 1;
  int from, to;
  keys_of(of, m0 / p.group, m_last / p.group, p.window, from, to);
  const int parts = part_of(p, part, from, to);
  if (part >= parts) return;
  const int w0 = m0 + wave * 32, w_last = min(w0 + 31, m_last);  // this wavefront's rows
  const int pos_lo = of.cached + w0 / p.group, pos_hi = of.cached + w_last / p.group;
  const RowAt at = row_at(p, of, kv_head, w0 + fr);
  typename L::Frag q[NQ];
  L::load_row(q, (const bf16*)p.q + at.row * p.ldq + (int64_t)at.head * p.c.head_dim, at.ok, p.c.head_dim, fh);
  uint32_t vo[L::IPG];
  L::offsets(vo, lane, p.c.head_dim);
  typename L::Address ad;
  L::addresses(ad, lane);
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>(lds);
  const L head(p.c, kv_head);
  const int tiles = (to - from + KT - 1) / KT;
  // tiles that this wavefront's rows see
  const int mine = w0 > m_last ? 0 : max(0, min(tiles, (min(to, pos_hi + 1) - from + KT - 1) / KT));

  // whether all pages are there
  bool lane_whole = true;
  for (int key = from + lane * GROUP; key < to; key += 64 * GROUP) lane_whole &= cache_page_any(p.c, s, key) >= 0;
  const bool whole = __builtin_amdgcn_ballot_w64(!lane_whole) == 0;
  // every wavefront brings 16 keys of a tile and their values
  const int own = wave * GROUP;
  auto page = [&](int t) { const int key = from + t * KT + own; return UNIFORM(t < tiles && key < to ? cache_page(p.c, s, key) : -1); };
  int page_next = page(0);
  uint32_t v_last = 0, v_now = 0, v_next = 2 * TILEB;  // LDS offsets of the values of the tile before, of this one and of the next
  auto request = [&](int t) __attribute__((always_inline)) {
    head.request(p.c.k, from + t * KT + own, page_next, to, vo, lds0 + (t & 1) * TILEB + own * L::ROWB);
    head.request(p.c.v, from + t * KT + own, page_next, to, vo, lds0 + v_next + own * L::ROWB);
    page_next = page(t + 1);
  };
  // Tile t is there, and where the next one goes nobody reads any more.
  auto advance = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    v_last = v_now;
    v_now = v_next;
    v_next = v_next == 4 * TILEB ? 2 * TILEB : v_next + TILEB;
  };

  float m = -INFINITY, ref = 0.f, l = 0.f;
  f32x16 o[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[nb][e] = 0.f;
  bf16x8 pr[2];  // probabilities by half of the block

  // of elements [first, last) of a block
  auto exponentials = [&](const f32x16& S, int first, int last) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (e >= first && e < last) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(S[e], p.scale_log2e, -ref));
        l += x;
        pr[e >> 3][e & 7] = static_cast<__bf16>(x);
      }
  };
  auto read_keys = [&](bf16x8 (&f)[NQ], const unsigned char* K) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NQ; ++i) f[i] = *reinterpret_cast<const bf16x8*>(K + ad.k[i]);
  };
  auto read_values = [&](bf16x8 (&f)[NB], const unsigned char* V, int h) __attribute__((always_inline)) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) f[nb] = L::value_frag(V, ad, h, nb);
  };
  auto times_values = [&](const bf16x8 (&f)[NB], int h) __attribute__((always_inline)) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) o[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[nb], pr[h], o[nb], 0, 0, 0);
  };
  auto row_max = [&](const f32x16& S) __attribute__((always_inline)) {
    float top = S[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, S[e]);
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * p.scale_log2e;
  };
  auto mask = [&](f32x16& S, int t, int b) __attribute__((always_inline)) {
    const int key0 = from + t * KT + b * KB;
    if (whole && key0 + KB <= to && key0 + KB - 1 <= pos_lo && (p.window == 0 || key0 > pos_hi - p.window)) return;
    const bool there0 = whole || cache_page(p.c, s, key0) >= 0, there1 = whole || cache_page(p.c, s, key0 + GROUP) >= 0;
    mask_scores<L>(S, key0, fh, to, at.pos, of.total, p.window, there0, there1);
  };
  // The reference is raised, and what was summed against it rescaled, where a score exceeds it by more than 2^8 (see Running).
  auto raise = [&](float top) __attribute__((always_inline)) {
    const float now = fmaxf(m, top), by = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
    l *= by;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[nb][e] *= by;
    m = now;
    ref = now == -INFINITY ? 0.f : now;
  };

  // Scores of block b of tile t into `now` while the block before, its scores in `last` and its values at V, is finished.  What is multiplied has been read from
  // LDS a phase before: keys f by the caller, for the next block of the tile here.
  auto step = [&](int t, int b, const f32x16& last, f32x16& now, const unsigned char* V, bf16x8 (&f)[NQ]) __attribute__((always_inline)) {
    bf16x8 v0[NB], v1[NB];
    read_values(v0, V, 0);
#pragma unroll
    for (int e = 0; e < 16; ++e) now[e] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {  // each product takes as long as the exponentials behind it: left to itself, the compiler puts all products first
      now = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i], q[i], now, 0, 0, 0);
      exponentials(last, i * 16 / NQ, (i + 1) * 16 / NQ);
      __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("" : "+v"(pr[0]), "+v"(pr[1]), "+v"(l));  // here and not behind the branches below
    if (b == 0 && t + 1 < tiles) request(t + 1);
    mask(now, t, b);
    read_values(v1, V, 1);
    times_values(v0, 0);
    if (b == 0) read_keys(f, lds + (t & 1) * TILEB + L::BLOCKB);
    times_values(v1, 1);
    const float top = row_max(now);
    if (__builtin_amdgcn_ballot_w64(top > m + 8.0f) != 0) raise(top);
  };
  if (tiles > 0) request(0);
  int t = 0;
  if (mine > 0) {
    f32x16 S0, S1;
    bf16x8 f[NQ];
    advance();
    if (tiles > 1) request(1);
    S0 = L::scores(lds, ad, q);
    mask(S0, 0, 0);
    raise(row_max(S0));
    read_keys(f, lds + L::BLOCKB);
    step(0, 1, S0, S1, lds + v_now, f);
    for (t = 1; t < mine; ++t) {
      advance();
      read_keys(f, lds + (t & 1) * TILEB);
      step(t, 0, S1, S0, lds + v_last + L::BLOCKB, f);
      step(t, 1, S0, S1, lds + v_now, f);
    }
    exponentials(S1, 0, 16);
    bf16x8 v[NB];
    read_values(v, lds + v_now + L::BLOCKB, 0);
    times_values(v, 0);
    read_values(v, lds + v_now + L::BLOCKB, 1);
    times_values(v, 1);
  }
  for (; t < tiles; ++t) {  // the others' tiles
    advance();
    if (t + 1 < tiles) request(t + 1);
  }

  l += __shfl_xor(l, 32, 64);
  finish_row<bf16, HD, NB>(p, at, o, m, l, part, parts, fh);
}

// Sequences of many rows, and those of few, if there may be any: the first few_first workgroups, one a key head.
template <typename T, int HD, int NB>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) mixed_k(Args p) {
  extern __shared__ unsigned char lds[];
  if ((int)blockIdx.x < p.few_first) few_whole<T, HD, NB, 4, false>(p, (int)blockIdx.x, lds, reinterpret_cast<float2(*)[FEW]>(lds + 4 * 2 * KB * HD * sizeof(T)));
  else if constexpr (sizeof(T) == 2) many_rows_bf16<HD, NB>(p, (int)blockIdx.x - p.few_first, lds);
  else many_rows_f32<HD, NB>(p, (int)blockIdx.x - p.few_first, lds);
}

// ---- rows whose keys fell to several workgroups ----
// W wavefronts, one or four, for each row and head of the first `tokens` tokens of a sequence; they take turns at the parts, four at a time, all their
// loads on the way together.
template <typename T, int HD, bool RUNS, int W>
__global__ void __launch_bounds__(256) join_k(Args p, int tokens) {
  constexpr int P = 4, C = HD / 64;
  __shared__ float sums[W == 1 ? 1 : W][HD];
  __shared__ float2 ml[4];
  const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : UNIFORM(threadIdx.x >> 6);
  const int item = W == 1 ? (int)blockIdx.x * 4 + UNIFORM(threadIdx.x >> 6) : (int)blockIdx.x;
  const int head = (int)((unsigned)item % (unsigned)p.heads), st = (int)((unsigned)item / (unsigned)p.heads);
  const int s = st / tokens, token = st % tokens, kv_head = head / p.group, m = token * p.group + head % p.group;
  if (s >= p.c.sequences) return;
  int n;          // parts
  int64_t first;  // the first one's place; the others follow, every `apart`-th
  int64_t apart;
  int64_t row;
  if constexpr (RUNS) {
    const int block = m / FEW;
    const int64_t all = p.plan[0], before = p.plan[1 + (int64_t)s * p.few_blocks + block];
    const Entry en(p, s, block);
    if (en.steps == 0 || token >= en.of.fresh) return;
    const int64_t step = before + (int64_t)kv_head * en.steps;
    const int runs = (int)min((int64_t)p.runs, all), r0 = run_of(step, all, runs);
    n = run_of(step + en.steps - 1, all, runs) - r0 + 1;
    first = ((int64_t)r0 * 2) * FEW + m % FEW;  // the first part is a run's last block of rows, the others are their run's first
    apart = 2 * FEW;
    row = en.of.row0 + token;
  } else {
    const CacheSeq of = cache_seq(p.c, s, p.rows, p.max_new);
    const int rows = of.fresh * p.group, block = m / 128;
    if (token >= of.fresh || rows <= p.few_upto) return;
    int from, to;
    keys_of(of, block * 128 / p.group, (min(rows, block * 128 + 128) - 1) / p.group, p.window, from, to);
    n = part_of(p, 0, from, to);
    row = of.row0 + token;
    first = (row * p.heads + head) * p.split;
    apart = 1;
  }
  if (n == 1) return;
  float top = -INFINITY, l = 0.f, o[C];
#pragma unroll
  for (int c = 0; c < C; ++c) o[c] = 0.f;
  for (int r = wave * P; r < n; r += W * P) {
    float2 z[P];
    float v[P][C];
#pragma unroll
    for (int k = 0; k < P; ++k) {
      const int i = min(r + k, n - 1);
      const int64_t at = first + i * apart + (RUNS && i == 0 ? FEW : 0);
      z[k] = p.part_ml[at];
#pragma unroll
      for (int c = 0; c < C; ++c) v[k][c] = p.part[at * HD + c * 64 + lane];
    }
    float now = top;
#pragma unroll
    for (int k = 0; k < P; ++k) now = fmaxf(now, z[k].x);
    const float ref = now == -INFINITY ? 0.f : now, by = __builtin_amdgcn_exp2f(top - ref);
    l *= by;
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] *= by;
#pragma unroll
    for (int k = 0; k < P; ++k)
      if (r + k < n) {
        const float w = __builtin_amdgcn_exp2f(z[k].x - ref);
        l = fmaf(w, z[k].y, l);
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] = fmaf(w, v[k][c], o[c]);
      }
    top = now;
  }
  RowAt r;
  r.row = row; r.head = head;
  if constexpr (W == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c) store_out<T>(p, r, c * 64 + lane, l > 0.f || l != l ? o[c] / l : 0.f);
    if (lane == 0 && p.lse) p.lse[row * p.heads + head] = top + __builtin_amdgcn_logf(l);
    return;
  }
#pragma unroll
  for (int c = 0; c < C; ++c) sums[wave][c * 64 + lane] = o[c];
  if (lane == 0) ml[wave] = make_float2(top, l);
  __syncthreads();
  if (threadIdx.x >= HD) return;
  float all_top = ml[0].x, all_l = 0.f, all_o = 0.f;
#pragma unroll
  for (int w = 1; w < W; ++w) all_top = fmaxf(all_top, ml[w].x);
  const float ref = all_top == -INFINITY ? 0.f : all_top;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const float by = __builtin_amdgcn_exp2f(ml[w].x - ref);
    all_l = fmaf(by, ml[w].y, all_l);
    all_o = fmaf(by, sums[w][threadIdx.x], all_o);
  }
  store_out<T>(p, r, threadIdx.x, all_l > 0.f || all_l != all_l ? all_o / all_l : 0.f);
  if (threadIdx.x == 0 && p.lse) p.lse[row * p.heads + head] = all_top + __builtin_amdgcn_logf(all_l);
}

// ---- host ----
struct Plan {
  bool many, past;
  int few_blocks, few_upto, few_first, many_blocks, split, chunk, runs, waves;
  int64_t entries, parts;  // rows of partial sums
};
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
Plan plan_of(int dt, const CacheView& c, int64_t rows, int heads, int max_new, int64_t max_length, int window) {
  Plan p{};
  const int group = heads / c.kv_heads;
  const int64_t most = (int64_t)max_new * group, pairs = (int64_t)c.sequences * c.kv_heads;  // rows of the longest sequence
  int64_t span = std::max<int64_t>(1, std::min<int64_t>(max_length, (int64_t)c.max_pages << c.page_shift));
  // as many workgroups as are on the chip at a time: LDS holds four blocks of rows of 128 bytes, two of 256, one of 512
  const int row_bytes = (c.head_dim <= 64 ? 64 : 128) * (dt == DT_BF16 ? 2 : 4), resident = 256 * 512 / row_bytes;
  // mixed_k shares a tile of keys among more rows, and its parts of the keys need no search for where they begin; few_k has four wavefronts on the same rows, none idle.
  // bf16, us, few_k / mixed_k: 16 sequences, 16 new over 2000, 32 / 8 heads (64 rows) 73 / 33; 1, 256 over 8192, 32 / 8 180 / 57; 1, 128 over 4000, 8 / 8 47 / 21; 1, 40
  // over 200, 16 / 16 of 64 9.3 / 8.8; of at most 32 rows, where three of four wavefronts of mixed_k idle: 4, 4 over 4000, 32 / 8 (32 key heads in all) 31 / 22; 1, 20
  // over 2000, 8 / 8 14.4 / 13.2; 16, 20 over 1000, 8 / 8 (128) 21 / 26; 1, 1 over 16000, 8 / 1 (8 rows) 17 / 21.
  // fp32, where products take eight times as long, and idle wavefronts show: 36, 30 over 1882, 32 / 16 of 64 (60 rows) 241 / 415; 16, 64 over 700, 32 / 32 (64) 177 / 257;
  // 45, 38 over 119, 64 / 32 of 32 (76) 80 / 59; 2, 300 over 300, 16 / 4 (1200 rows, 8 key heads) 64 / 98; 1, 1024, 32 / 32 201 / 152.
  if (dt == DT_BF16) p.many = most > FEW || (most > FEW / 4 && pairs <= 64);
  else p.many = most > 2 * FEW && pairs * up(most, FEW) > 512;
  p.few_upto = p.many ? 0 : INT32_MAX;
  p.few_blocks = (int)(p.many ? 1 : std::max<int64_t>(1, up(most, FEW)));
  p.many_blocks = (int)std::max<int64_t>(1, up(most, 128));
  p.entries = (int64_t)c.sequences * p.few_blocks;
  p.split = 1; p.chunk = INT32_MAX / 2;
  if (p.many) {
    if (window > 0) span = std::min<int64_t>(span, (int64_t)window + 128 / group + KB);
    // The keys are split where a compute unit would not have a workgroup, until it has two, but into parts that cost more than their joining (bf16, us, whole / split:
    // 1, 512 over 4096, 32 / 32 heads (128 workgroups) 99 / 61; 2, 1024 over 8192, 8 / 1 (128) 190 / 97; 8, 64 over 2048, 32 / 32 (256) 52 / 57; 1, 1024 over none, 32 / 32
    // (256) in parts of 512 30 / 45; fp32: 1, 2048 over none, 12 / 12 (192) 264 / 224; 1, 1024 over none, 32 / 32 (256) 152 / 178): 1024 keys (fp32: 512), 256 where
    // workgroups are few (parts of 512 / 256 / 128: 1, 128 over 1000, 8 / 8 18.2 / 16.1 / 15.9; 1, 128 over 4000, 8 / 8
    // 23.5 / 20.9 / 25.5; 1024 / 256: 1, 300 over 3000, 16 / 16 29.6 / 32.4).
    const int64_t blocks = pairs * p.many_blocks;
    const int64_t n = blocks >= 256 ? 1 : std::min<int64_t>({up(512, blocks), up(span, dt != DT_BF16 ? 512 : blocks > 64 ? 1024 : blocks > 32 ? 512 : 256), 64});
    if (n > 1) {
      p.chunk = (int)(up(up(span, n), 64) * 64);
      p.split = (int)up(span, p.chunk);
      p.parts = rows * heads * n;  // of which `split` <= n are used: n does not fall where keys get more, whole tiles may leave fewer parts
    }
    // Without parts, sequences of few rows among the others are few_rows' where there may be any (else none is short where the longest is not, as a rule); parts of
    // their keys are spread over the chip with the others' (11 sequences of up to 36 new, 4 / 4 heads bf16, over up to 6713: 72 us with whole keys, 47 so).
    if (p.split == 1 && rows < (int64_t)c.sequences * max_new) {
      p.few_upto = FEW;
      p.few_first = (int)pairs;
    }
    return p;
  }
  if (window > 0) span = std::min<int64_t>(span, (int64_t)window + FEW + KB);
  // Keys that one workgroup alone reads, of more than the eight L2s hold, go past them.  One token a sequence, us, with / without, each call on another cache of the
  // size as a model's layers are: 8 over 4000, 32 / 8 heads 35.8 / 39.6; 8 over 1000, 32 / 32 23.8 / 26.7; 64 over 2000, 32 / 8 97 / 108; smaller ones that a call
  // before has left in the L2s: 8 over 500, 32 / 8 9.2 / 8.5; several blocks of rows on the same keys: 1, 128 over 8000, 2 / 2 34.9 / 33.0.
  p.past = p.few_blocks == 1 && (int64_t)c.sequences * span * c.kv_heads * 2 * c.head_dim * (dt == DT_BF16 ? 2 : 4) >= int64_t(1) << 25;
  const int64_t items = pairs * p.few_blocks;
  // Eight wavefronts a block of rows where there are no more blocks than compute units (one token, 32 / 32 heads, us, eight / four: 1 over 500 8.1 / 9.9, 1 over 1000
  // 11.2 / 15.1, 8 over 1000 24.0 / 24.2, 32 over 500 47.2 / 42.2).  Runs cost a search for their begin and a second launch, which pays where the longest sequence is
  // long (whole / runs: 1 over 800 9.8 / 11.1, 1 over 1000 11.2 / 11.2, 8 of one length 1000 24.0 / 33.5) -- sequences of one length apart, at 32 x 1500 140 / 152.
  // fp32 steps take longer, so a chip that is not full has runs from two on (1 over 400, 8 / 8 25.4 / 16.2; 8 over 300, 8 / 8 22.2 / 18.7; 4 over 477, 4 / 4 25.7 /
  // 16.5; in one step each 2 x 4 over 228, 4 / 4 of 80 13.8 / 15.0).  Where keys are fewer than the wavefronts' blocks, the others would only take LDS from other
  // workgroups (128 over 20, 32 / 32 bf16, four wavefronts / one 42.5 / 16.5; over 60, fp32, four / two 160 / 94).
  p.waves = items <= 256 && row_bytes <= 256 && span > STEP ? 8 : span <= KB ? 1 : span <= 2 * KB ? 2 : 4;
  if (span > (items >= resident ? 8 : dt == DT_F32 && 2 * items <= resident ? 2 : std::max(p.waves, 4)) * STEP) {
    p.waves = 4;
    p.runs = (int)std::min<int64_t>(resident, items * up(span, STEP));
    p.parts = (int64_t)p.runs * 2 * FEW;
  }
  return p;
}
size_t plan_bytes(const Plan& p) { return p.runs ? (size_t)((1 + p.entries) * 8 + 15) / 16 * 16 : 0; }

template <auto KERNEL, int LDS>
hipError_t allow_lds() {
  static LdsAllowed allowed;  // one an instantiation
  return allowed(reinterpret_cast<const void*>(KERNEL), LDS);
}

template <typename T, int HD, int NB, bool PAST>
hipError_t whole(int waves, dim3 g, const Args& a, hipStream_t st) {
  const auto run = [&](auto w) -> hipError_t {
    constexpr int W = decltype(w)::value, LDS = W * 2 * KB * HD * (int)sizeof(T);
    if constexpr (LDS <= 131072) {
      if (hipError_t e = allow_lds<few_whole_k<T, HD, NB, W, PAST>, LDS>()) return e;
      few_whole_k<T, HD, NB, W, PAST><<<g, 64 * W, LDS, st>>>(a);
    }
    return hipSuccess;
  };
  switch (waves) {
    case 1: return run(std::integral_constant<int, 1>());
    case 2: return run(std::integral_constant<int, 2>());
    case 8: return run(std::integral_constant<int, 8>());
    default: return run(std::integral_constant<int, 4>());
  }
}

template <typename T, int HD, int NB>
hipError_t launch(const Plan& pl, Args a, int max_new, void* workspace, hipStream_t st) {
  a.few_upto = pl.few_upto; a.few_blocks = pl.few_blocks; a.many_blocks = pl.many_blocks; a.runs = pl.runs; a.few_first = pl.few_first; a.split = pl.split; a.chunk = pl.chunk;
  a.plan = (int64_t*)workspace;
  a.part_ml = (float2*)((unsigned char*)workspace + plan_bytes(pl));
  a.part = (float*)(a.part_ml + up(pl.parts, 2) * 2);
  const int64_t pairs = (int64_t)a.c.sequences * a.c.kv_heads, rows = (int64_t)a.c.sequences * max_new * a.heads;
  const int64_t grid = pl.many ? pl.few_first + pairs * pl.many_blocks * pl.split : pl.runs ? pl.runs : pairs * pl.few_blocks;
  if (grid > 0x7FFFFFFF || rows > 0x7FFFFFFF || pl.entries > 0x7FFFFFFF) return hipErrorInvalidValue;
  constexpr int BLOCKB = KB * HD * (int)sizeof(T), FEW_LDS = 4 * 2 * BLOCKB, MANY_LDS = (sizeof(T) == 2 ? 5 : 4) * 2 * BLOCKB;
  constexpr int MIXED_LDS = std::max(MANY_LDS, FEW_LDS + 4 * FEW * 8);
  static_assert(4 * FEW * HD * 4 <= FEW_LDS, "the wavefronts' sums fit where their tiles were");
  const dim3 g((unsigned)grid);
  if (pl.many) {
    if (hipError_t e = allow_lds<mixed_k<T, HD, NB>, MIXED_LDS>()) return e;
    mixed_k<T, HD, NB><<<g, 256, MIXED_LDS, st>>>(a);
    if (pl.split > 1) join_k<T, HD, false, 1><<<(unsigned)up(rows, 4), 256, 0, st>>>(a, max_new);
  } else if (pl.runs) {
    if (pl.past) {
      if (hipError_t e = allow_lds<few_k<T, HD, NB, true>, FEW_LDS>()) return e;
      few_k<T, HD, NB, true><<<g, 256, FEW_LDS, st>>>(a);
    } else {
      if (hipError_t e = allow_lds<few_k<T, HD, NB, false>, FEW_LDS>()) return e;
      few_k<T, HD, NB, false><<<g, 256, FEW_LDS, st>>>(a);
    }
    // Four wavefronts a row where it has more than four parts and one each would not fill the chip's 1024 SIMDs (us, four / one: 1, 1 over 16000, 8 / 1 heads 17.2 /
    // 32.6; 1, 8 over 8000, 32 / 8 32.5 / 41.1; 1, 128 over 4000, 8 / 8 (1024 rows) 46.9 / 48.6; 4, 16 over 4000, 32 / 4 (2048) 40.5 / 38.1; of 4096 and more rows, in 5
    // to 8 parts: 1, 256 over 8192, 32 / 8 64.9 / 55.8).
    if (pl.runs > 4 * pairs * pl.few_blocks && rows <= 1024) join_k<T, HD, true, 4><<<(unsigned)rows, 256, 0, st>>>(a, max_new);
    else join_k<T, HD, true, 1><<<(unsigned)up(rows, 4), 256, 0, st>>>(a, max_new);
  } else if (pl.past) {
    if (hipError_t e = whole<T, HD, NB, true>(pl.waves, g, a, st)) return e;
  } else {
    if (hipError_t e = whole<T, HD, NB, false>(pl.waves, g, a, st)) return e;
  }
  return hipGetLastError();
}
template <typename T>
hipError_t launch_width(const Plan& pl, const Args& a, int max_new, void* workspace, hipStream_t st) {
  switch ((a.c.head_dim + 31) / 32) {
    case 1: return launch<T, 64, 1>(pl, a, max_new, workspace, st);
    case 2: return launch<T, 64, 2>(pl, a, max_new, workspace, st);
    case 3: return launch<T, 128, 3>(pl, a, max_new, workspace, st);
    default: return launch<T, 128, 4>(pl, a, max_new, workspace, st);
  }
}

}  // namespace

size_t attention_paged_bytes(int dt, const CacheView& c, int64_t rows, int heads, int max_new, int64_t max_length, int window) {
  if (rows == 0 || c.sequences == 0 || max_new == 0) return 0;
  const Plan p = plan_of(dt, c, rows, heads, max_new, max_length, window);
  return p.parts ? plan_bytes(p) + (size_t)up(p.parts, 2) * 16 + (size_t)p.parts * (c.head_dim <= 64 ? 64 : 128) * 4 : 0;
}

hipError_t attention_paged(int dt, const CacheView& c, int heads, int64_t rows, int max_new, int64_t max_length, int window, float scale, const void* q, int64_t ldq,
                           void* out, int64_t ldo, float* lse, void* workspace, hipStream_t st) {
  if (rows == 0 || c.sequences == 0 || max_new == 0) return hipSuccess;
  const Plan pl = plan_of(dt, c, rows, heads, max_new, max_length, window);
  Args a{};
  a.c = c; a.heads = heads; a.group = heads / c.kv_heads;
  a.rows = rows; a.ldq = ldq; a.ldo = ldo; a.max_new = max_new; a.window = window;
  a.scale_log2e = scale * 1.4426950408889634f;
  a.q = q; a.out = out; a.lse = lse;
  return dt == DT_BF16 ? launch_width<bf16>(pl, a, max_new, workspace, st) : launch_width<float>(pl, a, max_new, workspace, st);
}

}  // namespace hift
