// Attention of a decode step over the pool in place (sc_decode_attn): few
// query rows per sequence, keys and values read through block lists from
// wherever the blocks are, 16-bit or 8-bit, and a prefix shared by the whole
// batch read once.
//
//     o = sum_j softmax_j(scale * q . k_j) v_j
//
// over the shared keys and the row's own.  A row's keys are cut into chunks;
// every chunk gives a partial (maximum m, sum l = sum 2^(s_j - m), O = sum
// 2^(s_j - m) v_j, all fp32) and decode_merge_kernel joins them: with M the
// largest m, o = sum 2^(m - M) O / sum 2^(m - M) l.  Short sequences and no
// shared prefix: the first kernel writes the result itself, a wave alone or
// the waves of a workgroup joined in LDS.
//
// Narrow (narrow_body): up to 16 rows of one KV head (the tokens and query
// heads of one sequence) against one chunk, bound by reading K and V once:
// 16 rows take the matrix units 16 cycles for 2 KiB (16-bit) that HBM
// delivers to a CU in 230.  K and V go from memory straight into the operand
// registers, with no LDS between, because no two waves share a key:
//   S^T (16 keys x 16 rows) = K . Q^T   lane (m = l % 16, g = l / 16) holds
//       key m's elements of its slots; which elements of the head a slot
//       stands for is free as long as Q^T uses the same, so a lane takes 16
//       contiguous bytes;
//   O^T (16 dims x 16 rows) += V^T . P^T   the slots of lane group g are the
//       8 keys whose scores that group already holds, so P needs no
//       exchange between lanes, and the dims of operand d are D / 16 * m + d:
//       a lane loads D / 16 contiguous elements of 8 keys and the D / 16
//       operands are that square transposed in registers.
// A wave takes 16 KiB of K and V at a time.
//
// Wide (wide_body): more rows than that share the keys (a shared prefix:
// every row of the batch).  A workgroup takes 256 rows through 128-key tiles
// in LDS, where a tile is laid out in operand order, 8-bit codes converted to
// 16 bits (exact in bf16 and fp16) once for all rows.
//
// 8-bit K and V: a key's scales are applied to its score and to its
// probability, in fp32; the codes, exact in either type, go into the products.
// The probabilities are rounded to the element type for the PV product.  With
// 8-bit blocks and fp16 that product 2^(s_j - m) v_scale_j could leave fp16's
// range either way, so there m is the maximum of s_j + log2 v_scale_j (the
// logarithm cut to kMaxLogScale): the rounded factors are then at most 1, and
// what is lost below fp16's normal numbers is 2^-24 of the largest.  The sums
// l, which hold no v_scale, stay in fp32's range: 2^-40 to 2^40 per key.  bf16
// has fp32's range and needs none of this.
//
// Keys past a row's end: scores are replaced by -infinity (never computed
// with), probabilities by 0 after scaling, and where such keys are in a tile
// at all the V operands are zeroed as well, per token of the step where the
// tokens' ends differ, so that nothing a hidden key holds (0 x NaN) arrives.
#include "sc_internal.h"
#include "sc_pool_view.h"
#include "sc_quant.h"

#include <algorithm>
#include <atomic>
#include <type_traits>

namespace sc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;             // of a workgroup without a wide part
constexpr int kWideWaves = 8;
constexpr int kTile = 128;            // keys of a workgroup's tile (wide)
constexpr int kWideRows = 32 * kWideWaves;
constexpr int kMergeThreads = 1024;   // at most
constexpr float kNegInf = -__builtin_inff();

template <int DT>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (DT == SC_DTYPE_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Geometry of one (head_dim, format): a head's row in memory and the pieces
// a lane takes of it.
template <int D, int FMT>
struct Geo {
  static constexpr bool k8 = FMT != SC_KV_16BIT;
  static constexpr int kElem = k8 ? 1 : 2;
  static constexpr int kRow = D * kElem;                 // bytes of one head's row
  static constexpr int kSteps = D / 32;                  // MFMA steps of a score
  static constexpr int kLoads = kRow / 64;               // 16-byte K loads of a lane
  static constexpr int kVd = D / 16;                     // dims a lane takes of a V row
  static constexpr int kVWords = kVd * kElem / 4;        // ... in 32-bit words
  // Keys of a wave's step (narrow): 16 KiB of K and V, 128 registers of a lane's 256.
  static constexpr int kStep = decode_step_keys(D, FMT);
};

// First head element of lane group g's slots in MFMA step c.
template <int D, int FMT>
__device__ __forceinline__ int slot_dim(int c, int g) {
  return Geo<D, FMT>::k8 ? 64 * (c >> 1) + 16 * g + 8 * (c & 1) : 32 * c + 8 * g;
}

// Loads from an address that was computed, which the compiler cannot see to
// be global memory: as flat loads they would also count against, and wait
// for, the LDS accesses between them.
template <class T>
__device__ __forceinline__ T load_global(uint64_t at) {
  return *(const __attribute__((address_space(1))) T *)at;
}

template <int N>
struct Words {
  uint32_t w[N];
};
template <int N>
__device__ __forceinline__ Words<N> load_words(uint64_t at) {
  Words<N> r;
  if constexpr (N == 1) {
    r.w[0] = load_global<uint32_t>(at);
  } else if constexpr (N == 2) {
    const u32x2 v = load_global<u32x2>(at);
    r.w[0] = v.x, r.w[1] = v.y;
  } else {
    const u32x4 v = load_global<u32x4>(at);
    r.w[0] = v.x, r.w[1] = v.y, r.w[2] = v.z, r.w[3] = v.w;
  }
  return r;
}

template <int N>
__device__ __forceinline__ void store_words(uint16_t *p, const Words<N> &w) {
  if constexpr (N == 2)
    *reinterpret_cast<u32x2 *>(p) = u32x2{w.w[0], w.w[1]};
  else
    *reinterpret_cast<u32x4 *>(p) = u32x4{w.w[0], w.w[1], w.w[2], w.w[3]};
}

// K operands of one key: D / 32 steps from its loads.
template <int D, int FMT, int DT>
__device__ __forceinline__ u32x4 k_operand(const u32x4 (&raw)[Geo<D, FMT>::kLoads], int c) {
  if constexpr (!Geo<D, FMT>::k8) {
    return raw[c];
  } else {
    u32x4 r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float f[4];
      codes_to_f32<FMT>(raw[c >> 1][2 * (c & 1) + h], f);
      r[2 * h] = pack16<DT>(f[0], f[1]);
      r[2 * h + 1] = pack16<DT>(f[2], f[3]);
    }
    return r;
  }
}

// V operands of 8 keys: operand d holds dim d of every key.
template <int D, int FMT, int DT>
__device__ __forceinline__ void v_operands(const Words<Geo<D, FMT>::kVWords> (&raw)[8], u32x4 (&op)[D / 16]) {
  using G = Geo<D, FMT>;
  if constexpr (!G::k8) {
#pragma unroll
    for (int w = 0; w < G::kVWords; ++w)
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const uint32_t a = raw[2 * p].w[w], b = raw[2 * p + 1].w[w];
        op[2 * w][p] = __builtin_amdgcn_perm(b, a, 0x05040100u);
        op[2 * w + 1][p] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      }
  } else {
#pragma unroll
    for (int w = 0; w < G::kVWords; ++w)
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        float a[4], b[4];
        codes_to_f32<FMT>(raw[2 * p].w[w], a);
        codes_to_f32<FMT>(raw[2 * p + 1].w[w], b);
#pragma unroll
        for (int i = 0; i < 4; ++i) op[4 * w + i][p] = pack16<DT>(a[i], b[i]);
      }
  }
}

// Whether the reference of a softmax takes in V's scales, and a scale's part.
template <int D, int FMT, int DT>
constexpr bool weigh_scales() {
  return Geo<D, FMT>::k8 && DT == SC_DTYPE_F16;
}
constexpr float kMaxLogScale = 40.f;
__device__ __forceinline__ float log_scale(float s) {          // (finite for a NaN too)
  return fminf(fmaxf(__builtin_amdgcn_logf(s), -kMaxLogScale), kMaxLogScale);
}

// Keys of sequence b in its own blocks; -1 for an empty slot, kBad for a
// length beyond the call's bounds.
constexpr int kBad = -2;
__device__ __forceinline__ int own_len(const DecodeAttnArgs &a, int b) {
  const int len = a.batch.kv_len[b];
  if (len < 0) return -1;
  return len > a.batch.max_len || len > (int64_t)a.batch.max_blocks * a.pool.block_size ? kBad : len;
}

// Whether any lane of the wave says so, as a value the compiler knows to be
// the wave's own: a branch on it then stays a scalar branch.
__device__ __forceinline__ bool wave_any(bool x) { return __builtin_amdgcn_ballot_w64(x) != 0; }

// LDS that only one wave uses: its accesses are executed in order, so only
// the compiler has to keep them so.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Running softmax of one row (one lane column): reference max, this lane's
// part of the sum.
struct RowState {
  float m, l;
};

// p = 2^(x - m) for the lane's N scores of one row, where m is at least the
// largest `key(i)`; the row's four lanes agree on it.  Returns the factor for
// what was accumulated before.
template <int N, class Key>
__device__ __forceinline__ float softmax_step(float (&x)[N], RowState &st, Key key) {
  float top = key(0);
#pragma unroll
  for (int i = 1; i < N; ++i) top = fmaxf(top, key(i));
  top = fmaxf(top, __shfl_xor(top, 16));
  top = fmaxf(top, __shfl_xor(top, 32));
  const float m = fmaxf(st.m, top);
  const float ref = m == kNegInf ? 0.f : m;
  const float alpha = __builtin_amdgcn_exp2f(st.m - ref);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = __builtin_amdgcn_exp2f(x[i] - ref);
    sum += x[i];
  }
  st.l = st.l * alpha + sum;
  st.m = m;
  return alpha;
}

// Writes of one row's 8 (head_dim 64: 4) consecutive dims.
template <int N>
__device__ __forceinline__ void store_f32(float *p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4 *>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}

// ---------------------------------------------------------------------------
// Narrow: a wave takes one chunk of one sequence's own keys (SHARED: of the
// shared ones), one KV head, 16 rows, and writes a partial of its own; the
// waves of a workgroup do not meet.  Consecutive waves take the KV heads of
// one chunk, so that together they read whole token rows: with a workgroup
// per head, the heads' reads of a row came from eight XCDs at different
// times, and HBM delivered 5% less (8-bit rows of 128 bytes a head), and the
// scales of a row were fetched once per XCD.  8 x 65536 e4m3 keys of 8 heads
// of 128: 192 us, 5.7 TB/s, where reading 64 KiB blocks at random places does
// 6.1; 48 sequences of 546 to 8192 fp16 keys of 8 heads of 64: 63 us, 5.3 TB/s.
//
// A wave's step t is pipelined with the next through the registers
// that it frees: K(t + 1) is loaded once the scores of step t are taken and
// arrives during their softmax and the PV product, V(t + 1) once that product
// is done.  Loads return in order, so what a later address needs (the block
// id, two steps ahead, and the scales) is issued before the K and V loads that
// it must not wait for.
// ---------------------------------------------------------------------------
struct NarrowLds {                           // of one wave
  uint64_t addr[64];
  float scale[3][64];                        // K, V, log_scale(V)
};

// A wave's partials that its workgroup joins in LDS.
template <int D>
struct JoinLds {
  float o[16][D + 4];                        // padded against bank conflicts
  float2 ml[16];
};

// Keys [k0, k1) of sequence `seq`, as partial `part` of its rows (`join`:
// the partial goes there instead).
template <int D, int FMT, int DT, bool SHARED>
__device__ __forceinline__ void narrow_keys(const DecodeAttnArgs &a, int seq, int len, int k0, int k1, int kvh, int tile,
                                            int64_t part, NarrowLds &lds, JoinLds<D> *join = nullptr) {
  using G = Geo<D, FMT>;
  constexpr int kStep = G::kStep, kTiles = kStep / 16, kHalves = kStep / 32;
  const PoolView &p = a.pool;
  const int lane = threadIdx.x & 63;
  const int group = a.plan.group;
  const int n_new = a.batch.n_new;
  const int n = lane & 15, g = lane >> 4;
  const int rows = SHARED ? a.plan.tokens * group : n_new * group;
  const int row = tile * 16 + n;             // this lane's column
  const bool has_row = row < rows;
  const int tok_in = has_row ? row / group : 0;              // token of the step (SHARED: of the batch)
  const int token = SHARED ? tok_in : seq * n_new + tok_in;
  const int head = kvh * group + (has_row ? row - tok_in * group : 0);
  const int limit = SHARED ? len : len - n_new + tok_in + 1; // keys below it are the row's

  const int32_t *ids = SHARED ? a.batch.shared_ids : a.batch.block_ids + (int64_t)seq * a.batch.max_blocks;
  const int64_t head_off = (int64_t)kvh * G::kRow;
  const int64_t row_bytes = (int64_t)p.n_kv_heads * G::kRow;
  // Keys from here on are hidden from some row of the tile.
  const int first_tok = tile * 16 / group;
  const int min_limit = SHARED ? len : len - n_new + first_tok + 1;
  bool bad = len == kBad;                    // the rows come out NaN

  uint32_t ks = 0, vs = 0;                   // this lane's key's scales, of the step addressed last
  uint64_t key_at = 0, scale_at = 0;         // addresses of its K row and K scale
  // Addresses of the step at `base`, whose lane's block is `blk_id`.  False
  // if an id is outside the pool: the addresses of the step before then stay
  // (with no branch around the loads) and the sequence's rows come out NaN.
  auto take_addr = [&](int base, int32_t blk_id) {
    const int key = min(base + lane, k1 - 1);
    const char *blk = block_layer(p, blk_id);
    const bool ok = !wave_any(blk == nullptr);
    bad = bad || !ok;
    const int in_block = key - block_of(p, key) * p.block_size;
    if constexpr (G::k8) {
      const int64_t off = p.scale_off + ((int64_t)in_block * p.n_kv_heads + kvh) * 2;
      scale_at = ok ? reinterpret_cast<uint64_t>(blk) + off : scale_at;
    }
    key_at = ok ? reinterpret_cast<uint64_t>(blk) + in_block * row_bytes + head_off : key_at;
    lds.addr[lane] = key_at;
    wave_lds_order();
    return ok;
  };
  auto load_scales = [&] {
    if constexpr (G::k8) {
      ks = load_global<uint16_t>(scale_at);
      vs = load_global<uint16_t>(scale_at + p.half_bytes);
    }
  };
  auto fetch_id = [&](int base) { return ids[block_of(p, min(base + lane, k1 - 1))]; };
  u32x4 kr[kTiles][G::kLoads];
  auto load_k = [&] {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const uint64_t kp = lds.addr[16 * t + n] + 16 * g;
#pragma unroll
      for (int c = 0; c < G::kLoads; ++c) kr[t][c] = load_global<u32x4>(kp + 64 * c);
    }
  };
  Words<G::kVWords> vr[kHalves][8];
  auto load_v = [&] {
#pragma unroll
    for (int u = 0; u < kHalves; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint64_t vp = lds.addr[32 * u + 16 * (j >> 2) + 4 * g + (j & 3)];
        vr[u][j] = load_words<G::kVWords>(vp + p.half_bytes + n * (G::kVd * G::kElem));
      }
  };
  auto write_scales = [&] {
    if constexpr (G::k8) {
      lds.scale[0][lane] = __builtin_bit_cast(float, ks << 16);
      lds.scale[1][lane] = __builtin_bit_cast(float, vs << 16);
      if constexpr (weigh_scales<D, FMT, DT>()) lds.scale[2][lane] = log_scale(__builtin_bit_cast(float, vs << 16));
    }
    wave_lds_order();
  };

  RowState st = {kNegInf, 0.f};
  f32x4 o[G::kVd];
#pragma unroll
  for (int d = 0; d < G::kVd; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};

  int base = k0;
  bool more = base < k1;
  int32_t next_id = 0;                       // block of this lane's key of the step after next
  u32x4 qf[G::kSteps];                       // Q^T operands
  if (more) {
    const int32_t first_id = fetch_id(base);
    if (base + kStep < k1) next_id = fetch_id(base + kStep);
    const uint16_t *qrow = a.q + ((int64_t)token * a.n_q_heads + head) * D;
#pragma unroll
    for (int c = 0; c < G::kSteps; ++c)
      qf[c] = has_row ? *reinterpret_cast<const u32x4 *>(qrow + slot_dim<D, FMT>(c, g)) : u32x4{0, 0, 0, 0};
    more = take_addr(base, first_id);
    if (more) {
      load_scales();
      load_k();
      load_v();
      write_scales();
    }
  }
  // One step; AHEAD: another one follows.
  auto step = [&](auto ahead) {
    constexpr bool kAhead = decltype(ahead)::value;
    // Scores: lane (n, g) gets keys 16 t + 4 g + i of row n.
    float x[4 * kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < G::kSteps; ++c) s = mfma16<DT>(k_operand<D, FMT, DT>(kr[t], c), qf[c], s);
      f32x4 sc = {1.f, 1.f, 1.f, 1.f};
      if constexpr (G::k8) sc = *reinterpret_cast<const f32x4 *>(&lds.scale[0][16 * t + 4 * g]);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * t + i] = s[i] * (G::k8 ? sc[i] * a.scale_log2 : a.scale_log2);
    }
    const int next = base + kStep;
    if constexpr (kAhead) {
      (void)take_addr(next, next_id);
      load_scales();
      next_id = fetch_id(next + kStep);
      load_k();
    }
    const bool edge = base + kStep > min(k1, min_limit);   // the same for the whole wave
    if (edge) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (base + 16 * t + 4 * g + i >= min(limit, k1)) x[4 * t + i] = kNegInf;
    }
    f32x4 lv[kTiles];
    if constexpr (weigh_scales<D, FMT, DT>())
#pragma unroll
      for (int t = 0; t < kTiles; ++t) lv[t] = *reinterpret_cast<const f32x4 *>(&lds.scale[2][16 * t + 4 * g]);
    const float alpha = softmax_step(x, st, [&](int i) {
      if constexpr (weigh_scales<D, FMT, DT>()) return x[i] + lv[i >> 2][i & 3];
      else return x[i];
    });
    if (wave_any(alpha != 1.f)) {
#pragma unroll
      for (int d = 0; d < G::kVd; ++d) o[d] *= alpha;
    }
#pragma unroll
    for (int u = 0; u < kHalves; ++u) {
      u32x4 pf;
      float w[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4 sc = {1.f, 1.f, 1.f, 1.f};
        if constexpr (G::k8) sc = *reinterpret_cast<const f32x4 *>(&lds.scale[1][32 * u + 16 * h + 4 * g]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[4 * h + i] = x[8 * u + 4 * h + i];
          if constexpr (G::k8) w[4 * h + i] *= sc[i];
        }
      }
      if (G::k8 && edge) {                   // 0 x a hidden key's NaN scale
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (base + 32 * u + 16 * (j >> 2) + 4 * g + (j & 3) >= min(limit, k1)) w[j] = 0.f;
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) pf[q] = pack16<DT>(w[2 * q], w[2 * q + 1]);
      u32x4 vo[G::kVd];
      if (!edge) {
        v_operands<D, FMT, DT>(vr[u], vo);
#pragma unroll
        for (int d = 0; d < G::kVd; ++d) o[d] = mfma16<DT>(vo[d], pf, o[d]);
      } else {
        // One pass per distinct end: V without the keys that this token does
        // not see, added to its rows only.
        const int last_tok = SHARED ? first_tok : min(n_new - 1, (tile * 16 + 15) / group);
        for (int tk = first_tok; tk <= last_tok; ++tk) {
          const int end = min(k1, SHARED ? len : len - n_new + tk + 1);
          Words<G::kVWords> cut[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool hidden = base + 32 * u + 16 * (j >> 2) + 4 * g + (j & 3) >= end;
#pragma unroll
            for (int q = 0; q < G::kVWords; ++q) cut[j].w[q] = hidden ? 0u : vr[u][j].w[q];
          }
          v_operands<D, FMT, DT>(cut, vo);
          const bool mine = SHARED || tok_in == tk;
#pragma unroll
          for (int d = 0; d < G::kVd; ++d) {
            const f32x4 add = mfma16<DT>(vo[d], pf, f32x4{0.f, 0.f, 0.f, 0.f});
            if (mine) o[d] += add;
          }
        }
      }
    }
    if constexpr (kAhead) {
      load_v();
      wave_lds_order();
      write_scales();
      base = next;
    }
  };
  // The last step is a copy of its own: a condition around the loads would
  // join ways with and without them at the loop's top, where the compiler
  // would then wait for every load instead of K's.
  if (more) {
    while (base + kStep < k1) step(std::true_type());
    step(std::false_type());
  }

  st.l += __shfl_xor(st.l, 16);
  st.l += __shfl_xor(st.l, 32);
  if (!has_row) return;
  if (bad) st.m = st.l = __builtin_nanf("");
  // o[d][i]: dim G::kVd * (4 g + i) + d of row n.
  if (SHARED || join != nullptr || !a.plan.direct) {
    // `part` is the partial's first row; rows follow tokens, then heads.
    const int64_t at = part + (int64_t)(SHARED ? token : tok_in) * a.n_q_heads + head;
    float *const to = join != nullptr ? join->o[n] : a.part_o + at * D;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[G::kVd];
#pragma unroll
      for (int d = 0; d < G::kVd; ++d) v[d] = o[d][i];
      store_f32(to + G::kVd * (4 * g + i), v);
    }
    if (g == 0) *(join != nullptr ? &join->ml[n] : a.part_ml + at) = float2{st.m, st.l};
    return;
  }
  const int64_t out_row = (int64_t)token * a.n_q_heads + head;
  const bool none = !bad && limit <= 0;      // no key at all: zeros
  const float inv = none ? 0.f : 1.f / st.l;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    Words<G::kVd / 2> w;
#pragma unroll
    for (int d = 0; d < G::kVd; d += 2) w.w[d / 2] = none ? 0u : pack16<DT>(o[d][i] * inv, o[d + 1][i] * inv);
    store_words(a.out + out_row * D + G::kVd * (4 * g + i), w);
  }
  if (g == 0 && a.lse != nullptr)
    a.lse[(int64_t)head * a.plan.tokens + token] = none ? kNegInf : (st.m + __builtin_log2f(st.l)) * 0.6931471805599453f;
}

// Steps of a sequence's own keys.
template <int D, int FMT>
__device__ __forceinline__ int steps_of(int len) {
  return len > 0 ? (len + Geo<D, FMT>::kStep - 1) / Geo<D, FMT>::kStep : 0;
}

// Inclusive sum over the lanes below and at this one.
__device__ __forceinline__ int wave_scan(int x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const int y = __shfl_up(x, s);
    x += lane >= s ? y : 0;
  }
  return x;
}

// Steps of a group's run: ceil(all sequences' steps / groups), at least 1.
// Every lane of the wave calls it.
template <int D, int FMT>
__device__ __forceinline__ int run_steps(const DecodeAttnArgs &a) {
  const int lane = threadIdx.x & 63;
  int mine = 0;
  for (int b = lane; b < a.batch.batch; b += 64) mine += steps_of<D, FMT>(own_len(a, b));
  const int total = __builtin_amdgcn_readlane(wave_scan(mine), 63);
  return max(1, (total + a.plan.groups - 1) / a.plan.groups);
}

// Item `item`: KV head item % n_kv_heads of row tile and chunk (SHARED) or
// group of waves.
template <int D, int FMT, int DT, bool SHARED>
__device__ __forceinline__ void narrow_body(const DecodeAttnArgs &a, int64_t first_item, int row_tiles, char *smem) {
  using G = Geo<D, FMT>;
  // In a scalar register, and with it every condition that only the wave decides.
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  NarrowLds &lds = reinterpret_cast<NarrowLds *>(smem)[wave];
  const int64_t item = first_item + wave;
  int unit = (int)(item / a.pool.n_kv_heads);
  const int kvh = (int)(item - (int64_t)unit * a.pool.n_kv_heads);
  const int tile = unit % row_tiles;
  unit /= row_tiles;
  if constexpr (SHARED) {
    if (unit >= a.plan.shared_chunks) return;                // the last workgroup's waves without an item
    const int k0 = unit * a.plan.shared_chunk, len = a.batch.shared_len;
    narrow_keys<D, FMT, DT, true>(a, 0, len, k0, min(len, k0 + a.plan.shared_chunk), kvh, tile,
                                  (int64_t)unit * a.plan.tokens * a.n_q_heads, lds);
  } else if (a.plan.direct) {
    if (unit >= a.batch.batch) return;
    const int len = own_len(a, unit);
    narrow_keys<D, FMT, DT, false>(a, unit, len, 0, len, kvh, tile, 0, lds);
  } else {
    if (unit >= a.plan.groups) return;
    const int per = run_steps<D, FMT>(a);
    const int first = unit * per;                            // the run's steps [first, first + per); all fit 2^30
    const int64_t rows = (int64_t)a.batch.n_new * a.n_q_heads;
    const int64_t own0 = (int64_t)a.plan.shared_chunks * a.plan.tokens * a.n_q_heads;
    int before = 0;                                          // steps of the sequences before the lanes'
    for (int b0 = 0; b0 < a.batch.batch && before < first + per; b0 += 64) {
      const int len = b0 + lane < a.batch.batch ? own_len(a, b0 + lane) : 0;
      const int steps = steps_of<D, FMT>(len);
      const int upto = wave_scan(steps);
      const int begin = before + upto - steps;
      uint64_t todo = __builtin_amdgcn_ballot_w64(steps > 0 && begin < first + per && begin + steps > first);
      while (todo != 0) {
        const int l = __builtin_ctzll(todo);
        todo &= todo - 1;
        const int n = __builtin_amdgcn_readlane(len, l);
        const int s0 = before + __builtin_amdgcn_readlane(upto - steps, l);
        const int k0 = max(0, first - s0) * G::kStep;
        const int k1 = (int)min((int64_t)n, (int64_t)(first + per - s0) * G::kStep);
        narrow_keys<D, FMT, DT, false>(a, b0 + l, n, k0, k1, kvh, tile, own0 + (int64_t)(unit + b0 + l) * rows, lds);
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
  }
}

// Short sequences (DecodePlan::joined): workgroup `id` takes 16 rows of one KV
// head of a sequence, its waves equal runs of its steps, and joins them in
// LDS: no partials in memory and no second launch.
template <int D, int FMT, int DT>
__device__ __forceinline__ void joined_body(const DecodeAttnArgs &a, int id, int row_tiles, char *smem) {
  constexpr int kStep = Geo<D, FMT>::kStep;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  JoinLds<D> *const join = reinterpret_cast<JoinLds<D> *>(smem + kWaves * sizeof(NarrowLds));
  const int kvh = id % a.pool.n_kv_heads;
  id /= a.pool.n_kv_heads;
  const int tile = id % row_tiles, seq = id / row_tiles;
  const int len = own_len(a, seq);
  const int run = (steps_of<D, FMT>(len) + kWaves - 1) / kWaves * kStep;
  narrow_keys<D, FMT, DT, false>(a, seq, len, wave * run, min(max(len, 0), (wave + 1) * run), kvh, tile, 0,
                                 reinterpret_cast<NarrowLds *>(smem)[wave], join + wave);
  __syncthreads();
  const int group = a.plan.group, n_new = a.batch.n_new;
  // Thread: 4 dims of a row.
  for (int idx = threadIdx.x; idx < 16 * (D / 4); idx += 64 * kWaves) {
    const int r = idx / (D / 4), d0 = 4 * (idx % (D / 4)), row = tile * 16 + r;
    if (row >= n_new * group) break;
    const int tok_in = row / group, token = seq * n_new + tok_in, head = kvh * group + row - tok_in * group;
    float m = kNegInf, l = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, join[w].ml[r].x);
    const float ref = m == kNegInf ? 0.f : m;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 ml = join[w].ml[r];
      const float f = __builtin_amdgcn_exp2f(ml.x - ref);
      l += f * ml.y;
      o += f * *reinterpret_cast<const f32x4 *>(&join[w].o[r][d0]);
    }
    const bool none = len != kBad && len - n_new + tok_in + 1 <= 0;   // no key at all: zeros
    const float inv = 1.f / l;
    u32x2 v;
    v.x = none ? 0u : pack16<DT>(o[0] * inv, o[1] * inv);
    v.y = none ? 0u : pack16<DT>(o[2] * inv, o[3] * inv);
    *reinterpret_cast<u32x2 *>(a.out + ((int64_t)token * a.n_q_heads + head) * D + d0) = v;
    if (d0 == 0 && a.lse != nullptr)
      a.lse[(int64_t)head * a.plan.tokens + token] = none ? kNegInf : (m + __builtin_log2f(l)) * 0.6931471805599453f;
  }
}

// ---------------------------------------------------------------------------
// Wide: one chunk of the shared keys, one KV head, 256 rows of the batch.
//
// Eight waves of 32 rows share 128-key tiles in two LDS buffers with one
// barrier a tile: while tile t is computed, tile t + 1 goes from the loaders'
// registers into the other buffer (waves 0-3 load and lay out V, waves 4-7 K)
// and tile t + 2 is loaded.  LDS holds whole MFMA operands, 16 bytes a lane.
// The two waves of a SIMD (w and w + 4) do their part of that at the opposite
// ends of a tile, so that one takes products while the other is at its
// softmax: 64 x 4 rows of 5 heads over 32768 int8 keys take 246 us (0.70
// PFLOP/s); with both in the middle of a tile, in step from barrier to
// barrier, 275 us.
//
// The vector unit is the bound (per score half a maximum, an FMA, an
// exponential, an add and half a pack, for 8-bit blocks a multiplication by
// each of K's and V's scales, against 32 MFMA cycles for 16 of them), so the
// reference m of a row's softmax, which may be any number, is not its running
// maximum: it moves only when a score (with its part of V's scale, see the top)
// exceeds it by kRefSlack (in the log2
// domain), and only then do lanes exchange anything and the accumulators
// change.  The slack keeps the probabilities inside fp16.
// ---------------------------------------------------------------------------
constexpr float kRefSlack = 12.f;

template <int D>
struct WideLds {
  u32x4 k[2][kTile * D / 8];                 // [buffer][tile of 16 keys][step][lane]
  u32x4 v[2][kTile * D / 8];                 // [buffer][32 keys][operand][lane]
  float scale[2][3][kTile];                  // [buffer][K times the softmax scale, V, log_scale(V)]
  uint64_t addr[2][kTile];
  int bad[2];
};

template <int D, int FMT, int DT>
__device__ __forceinline__ void wide_body(const DecodeAttnArgs &a, int id, int row_tiles, char *smem) {
  using G = Geo<D, FMT>;
  constexpr int kKThreads = 256;
  constexpr int kKPer = kTile * G::kRow / 16 / kKThreads;     // 16-byte K pieces of a loader
  constexpr int kPieces = G::kRow / 16;                       // ... of a key
  static_assert(kKPer <= 8 && kWideWaves == 8, "eight registers of 16 bytes hold a loader's part of a tile");
  WideLds<D> &lds = *reinterpret_cast<WideLds<D> *>(smem);

  const PoolView &p = a.pool;
  const int kvh = id % p.n_kv_heads;
  id /= p.n_kv_heads;
  const int tile = id % row_tiles;
  const int chunk = id / row_tiles;
  const int group = a.plan.group;
  const int k0 = chunk * a.plan.shared_chunk;
  const int k1 = min(a.batch.shared_len, k0 + a.plan.shared_chunk);
  const int tiles = (k1 - k0 + kTile - 1) / kTile;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int rows = a.plan.tokens * group;
  // Fewer rows than eight waves have: row_waves (a power of two) of them
  // cover the rows, and the others share their keys, every key_waves-th
  // 32-key block each.  64 rows over 65536 bf16 keys 68 us, 79 with a wave's
  // keys unshared: two busy waves a CU took longer for a tile than its load.
  const int rows_here = min(kWideRows, rows - tile * kWideRows);
  const int row_waves = rows_here > 128 ? 8 : rows_here > 64 ? 4 : rows_here > 32 ? 2 : 1;
  const int key_waves = kWideWaves / row_waves, key_wave = wave / row_waves;
  const int row0 = tile * kWideRows + (wave & (row_waves - 1)) * 32;
  int64_t out_row[2];
  bool has_row[2];
  u32x4 qf[2][G::kSteps];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int row = row0 + 16 * r + n;
    has_row[r] = row < rows;
    const int token = has_row[r] ? row / group : 0;
    out_row[r] = (int64_t)token * a.n_q_heads + kvh * group + (has_row[r] ? row - token * group : 0);
#pragma unroll
    for (int c = 0; c < G::kSteps; ++c)
      qf[r][c] = has_row[r] ? *reinterpret_cast<const u32x4 *>(a.q + out_row[r] * D + slot_dim<D, FMT>(c, g))
                            : u32x4{0, 0, 0, 0};
  }

  const int64_t head_off = (int64_t)kvh * G::kRow;
  const int64_t row_bytes = (int64_t)p.n_kv_heads * G::kRow;
  const bool loads_v = wave < 4;             // and addresses and scales; the others load K
  const int my_key = tid & (kTile - 1);      // threads 0..127: K's scale, 128..255: V's
  if (tid < 2) lds.bad[tid] = 0;
  __syncthreads();
  int32_t next_id = 0;                       // block of this thread's key of the tile to address next
  auto fetch_id = [&](int t) {
    if (loads_v) next_id = a.batch.shared_ids[block_of(p, min(k0 + t * kTile + my_key, k1 - 1))];
  };
  uint64_t my_scale = 0, next_scale = 0;     // this thread's scale of the tile to load next, and after it
  auto take_addr = [&](int t) {              // address of this thread's key of tile t
    if (!loads_v) return;
    const int key = min(k0 + t * kTile + my_key, k1 - 1);
    const char *base = block_layer(p, next_id);
    if (base == nullptr) {
      lds.bad[t & 1] = 1;
      return;
    }
    const int in_block = key - block_of(p, key) * p.block_size;
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    if (tid < kTile) lds.addr[t & 1][my_key] = at + in_block * row_bytes + head_off;
    if constexpr (G::k8)
      next_scale = at + (tid < kTile ? 0 : p.half_bytes) + p.scale_off + ((int64_t)in_block * p.n_kv_heads + kvh) * 2;
  };
  u32x4 raw[8];                              // the tile in flight: K pieces or V keys
  uint32_t scale_bits = 0;
  auto load_tile = [&](int t) {
    if (loads_v) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const Words<G::kVWords> w =
            load_words<G::kVWords>(lds.addr[t & 1][32 * wave + 16 * (j >> 2) + 4 * g + (j & 3)] + p.half_bytes +
                                   n * (G::kVd * G::kElem));
#pragma unroll
        for (int q = 0; q < G::kVWords; ++q) raw[j][q] = w.w[q];
      }
      if constexpr (G::k8) scale_bits = load_global<uint16_t>(my_scale);
    } else {
#pragma unroll
      for (int i = 0; i < kKPer; ++i) {
        const int idx = tid - kKThreads + kKThreads * i;
        raw[i] = load_global<u32x4>(lds.addr[t & 1][idx / kPieces] + 16 * (idx % kPieces));
      }
    }
  };
  // Position of lane (m, g)'s K operand of step c: rotated among the 16 keys
  // so that the pieces of one key, which consecutive threads write, fall on
  // different banks.
  auto k_slot = [&](int t16, int c, int g_, int m_) {
    return (t16 * G::kSteps + c) * 64 + g_ * 16 + (m_ ^ ((4 * c + g_) & 15));
  };
  auto write_tile = [&](int t) {
    u32x4 *const sk = lds.k[t & 1], *const sv = lds.v[t & 1];
    if (loads_v) {
      if (k0 + (t + 1) * kTile > k1) {       // no value for the keys behind the last: not a copy of its
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (k0 + t * kTile + 32 * wave + 16 * (j >> 2) + 4 * g + (j & 3) >= k1) raw[j] = u32x4{0, 0, 0, 0};
      }
      Words<G::kVWords> vr[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int q = 0; q < G::kVWords; ++q) vr[j].w[q] = raw[j][q];
      u32x4 vo[G::kVd];
      v_operands<D, FMT, DT>(vr, vo);
#pragma unroll
      for (int d = 0; d < G::kVd; ++d) sv[(wave * G::kVd + d) * 64 + lane] = vo[d];
      if constexpr (G::k8) {
        const float s = __builtin_bit_cast(float, scale_bits << 16);
        lds.scale[t & 1][tid / kTile][my_key] = s * (tid < kTile ? a.scale_log2 : 1.f);
        if (weigh_scales<D, FMT, DT>() && tid >= kTile) lds.scale[t & 1][2][my_key] = log_scale(s);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kKPer; ++i) {
        const int idx = tid - kKThreads + kKThreads * i;
        const int key = idx / kPieces, x = idx % kPieces;
        if constexpr (!G::k8) {
          sk[k_slot(key >> 4, x >> 2, x & 3, key & 15)] = raw[i];
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float f0[4], f1[4];
            codes_to_f32<FMT>(raw[i][2 * h], f0);
            codes_to_f32<FMT>(raw[i][2 * h + 1], f1);
            sk[k_slot(key >> 4, 2 * (x >> 2) + h, x & 3, key & 15)] =
                u32x4{pack16<DT>(f0[0], f0[1]), pack16<DT>(f0[2], f0[3]), pack16<DT>(f1[0], f1[1]),
                      pack16<DT>(f1[2], f1[3])};
          }
        }
      }
    }
  };

  float l[2] = {0.f, 0.f};
  float neg_ref[2] = {0.f, 0.f};             // -m, or 0 while there is none
  float limit[2] = {kNegInf, kNegInf};       // a score this much above m moves it; -infinity: no m yet
  f32x4 o[2][G::kVd];
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int d = 0; d < G::kVd; ++d) o[r][d] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto compute = [&](int t, int u) {         // keys 32 u .. 32 u + 31 of tile t
    const u32x4 *const sk = lds.k[t & 1], *const sv = lds.v[t & 1];
    f32x4 s[2][2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      s[0][tt] = s[1][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < G::kSteps; ++c) {
        const u32x4 kf = sk[k_slot(2 * u + tt, c, g, n)];
        s[0][tt] = mfma16<DT>(kf, qf[0][c], s[0][tt]);
        s[1][tt] = mfma16<DT>(kf, qf[1][c], s[1][tt]);
      }
    }
    const int base = k0 + t * kTile + 32 * u;
    const bool edge = base + 32 > k1;
    f32x4 ks[2], vs[2], lv[2];               // scales of the lane's keys
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      ks[tt] = f32x4{a.scale_log2, a.scale_log2, a.scale_log2, a.scale_log2};
      if constexpr (G::k8) {
        ks[tt] = *reinterpret_cast<const f32x4 *>(&lds.scale[t & 1][0][32 * u + 16 * tt + 4 * g]);
        vs[tt] = *reinterpret_cast<const f32x4 *>(&lds.scale[t & 1][1][32 * u + 16 * tt + 4 * g]);
        if constexpr (weigh_scales<D, FMT, DT>())
          lv[tt] = *reinterpret_cast<const f32x4 *>(&lds.scale[t & 1][2][32 * u + 16 * tt + 4 * g]);
      }
    }
    if (edge) {                              // keys behind the last: no score, whatever their scales are
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (base + 16 * tt + 4 * g + i >= k1) {
            s[0][tt][i] = s[1][tt][i] = kNegInf;
            ks[tt][i] = 1.f;
            if constexpr (G::k8) vs[tt][i] = 0.f;
          }
    }
    u32x4 pf[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float x[8], y[8];                      // scores less the reference; y: with V's scale's part
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __builtin_fmaf(s[r][i >> 2][i & 3], ks[i >> 2][i & 3], neg_ref[r]);
        y[i] = weigh_scales<D, FMT, DT>() ? x[i] + lv[i >> 2][i & 3] : x[i];
      }
      float top = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
      if (wave_any(top > limit[r])) {        // a new reference for the rows that need one
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        // (there may be none yet, nothing to scale then, and none stays none
        // while all scores are -infinity)
        const bool none = limit[r] == kNegInf;
        const float up = none ? (top == kNegInf ? 0.f : top) : fmaxf(top, 0.f);
        const float f = none ? 1.f : __builtin_amdgcn_exp2f(-up);
        if (top != kNegInf) limit[r] = kRefSlack;
        neg_ref[r] -= up;
        l[r] *= f;
#pragma unroll
        for (int d = 0; d < G::kVd; ++d) o[r][d] *= f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] -= up;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __builtin_amdgcn_exp2f(x[i]);
        l[r] += x[i];
      }
      if constexpr (G::k8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= vs[i >> 2][i & 3];
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) pf[r][q] = pack16<DT>(x[2 * q], x[2 * q + 1]);
    }
#pragma unroll
    for (int d = 0; d < G::kVd; ++d) {
      const u32x4 vf = sv[(u * G::kVd + d) * 64 + lane];
      o[0][d] = mfma16<DT>(vf, pf[0], o[0][d]);
      o[1][d] = mfma16<DT>(vf, pf[1], o[1][d]);
    }
  };

  // Tile t is addressed in iteration t - 3, loaded in t - 2, written in t - 1;
  // its address slot and its bad flag are those of its parity, and a barrier
  // lies between every use by one tile and the next one's.
  int end = tiles;                           // tiles before the first bad id
  auto check = [&](int t) {
    if (t < end && lds.bad[t & 1] != 0) end = t;
  };
  fetch_id(0);
  take_addr(0);
  if (tiles > 1) fetch_id(1);
  __syncthreads();
  check(0);
  if (end > 0) {
    my_scale = next_scale;
    load_tile(0);
    if (tiles > 1) take_addr(1);
    if (tiles > 2) fetch_id(2);
    write_tile(0);
    __syncthreads();
    check(1);
    my_scale = next_scale;
    if (end > 1) load_tile(1);
    if (end > 1 && tiles > 2) take_addr(2);
    __syncthreads();
    check(2);
  }
  auto move = [&](int t) {                   // the next tile into LDS and the one after it into the registers
    if (t + 1 < end) write_tile(t + 1);
    my_scale = next_scale;
    if (t + 2 < end) load_tile(t + 2);
  };
  for (int t = 0; t < end; ++t) {
    if (t + 3 < end) fetch_id(t + 3);
    if (!loads_v) move(t);
    for (int u = key_wave; u < 4; u += key_waves) compute(t, u);
    if (loads_v) move(t);
    if (t + 3 < end) take_addr(t + 3);
    __syncthreads();
    check(t + 3);
  }
  const bool bad = end < tiles;
  const float nan = __builtin_nanf("");

  const int64_t all_rows = (int64_t)a.plan.tokens * a.n_q_heads;
  // The keys' waves meet in LDS, which no tile needs any more.
  constexpr int kJoinRow = D + 4;            // floats of a row, padded against bank conflicts
  float *const join_o = reinterpret_cast<float *>(smem);
  float2 *const join_ml = reinterpret_cast<float2 *>(&lds.scale[0][0][0]);
  static_assert(sizeof(lds.scale) >= kWideWaves * 32 * sizeof(float2), "one pair a wave and row");
  static_assert(sizeof(lds.k) + sizeof(lds.v) >= kWideWaves * 16 * kJoinRow * sizeof(float), "one half of the rows");
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    float sum_l = l[r];
    sum_l += __shfl_xor(sum_l, 16);
    sum_l += __shfl_xor(sum_l, 32);
    const float m = limit[r] == kNegInf ? kNegInf : -neg_ref[r];
    if (key_waves == 1) {
      if (!has_row[r]) continue;
      const int64_t at = (int64_t)chunk * all_rows + out_row[r];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[G::kVd];
#pragma unroll
        for (int d = 0; d < G::kVd; ++d) v[d] = o[r][d][i];
        store_f32(a.part_o + at * D + G::kVd * (4 * g + i), v);
      }
      if (g == 0) a.part_ml[at] = bad ? float2{nan, nan} : float2{m, sum_l};
      continue;
    }
    if (r == 1) __syncthreads();             // the first half of the rows has been read
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[G::kVd];
#pragma unroll
      for (int d = 0; d < G::kVd; ++d) v[d] = o[r][d][i];
      store_f32(join_o + (wave * 16 + n) * kJoinRow + G::kVd * (4 * g + i), v);
    }
    if (g == 0) join_ml[wave * 16 + n] = float2{m, sum_l};
    __syncthreads();
    // Thread: 4 dims of one of the 16 row_waves rows.
    for (int idx = tid; idx < row_waves * 16 * (D / 4); idx += 64 * kWideWaves) {
      const int jr = idx / (D / 4), d0 = 4 * (idx % (D / 4));          // jr = 16 * row wave + row
      const int row = tile * kWideRows + (jr >> 4) * 32 + 16 * r + (jr & 15);
      if (row >= rows) continue;
      float top = kNegInf, sum = 0.f;
      for (int w = 0; w < key_waves; ++w) top = fmaxf(top, join_ml[w * row_waves * 16 + jr].x);
      const float ref = top == kNegInf ? 0.f : top;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      for (int w = 0; w < key_waves; ++w) {
        const float2 ml = join_ml[w * row_waves * 16 + jr];
        const float f = __builtin_amdgcn_exp2f(ml.x - ref);
        sum += f * ml.y;
        v += f * *reinterpret_cast<const f32x4 *>(join_o + (w * row_waves * 16 + jr) * kJoinRow + d0);
      }
      const int token = row / group;
      const int64_t at = (int64_t)chunk * all_rows + (int64_t)token * a.n_q_heads + kvh * group + (row - token * group);
      *reinterpret_cast<f32x4 *>(a.part_o + at * D + d0) = v;
      if (d0 == 0) a.part_ml[at] = bad ? float2{nan, nan} : float2{top, sum};
    }
  }
}

// One launch for both key lists, the shared one's workgroups first: they are
// the longer ones, and the own keys' loads fill the memory's time beside the
// wide kernel's matrix work.  WIDE: the shared keys have more than 16 rows.
template <int D, int FMT, int DT, bool WIDE>
__global__ __launch_bounds__(64 * (WIDE ? kWideWaves : kWaves), 2) void decode_attn_kernel(DecodeAttnArgs a,
                                                                                          int shared_groups,
                                                                                          int shared_tiles,
                                                                                          int own_tiles) {
  constexpr int kGroupWaves = WIDE ? kWideWaves : kWaves;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int id = blockIdx.x;
  if constexpr (!WIDE)
    if (a.plan.joined) return joined_body<D, FMT, DT>(a, id, own_tiles, smem);
  if (id >= shared_groups)
    narrow_body<D, FMT, DT, false>(a, (int64_t)(id - shared_groups) * kGroupWaves, own_tiles, smem);
  else if constexpr (WIDE)
    wide_body<D, FMT, DT>(a, id, shared_tiles, smem);
  else
    narrow_body<D, FMT, DT, true>(a, (int64_t)id * kGroupWaves, shared_tiles, smem);
}

// ---------------------------------------------------------------------------
// Merge.  D / 4 lanes hold a row's output, 4 dims each; `split` such lane
// groups of a workgroup share one row's partials.  Bound by reading them
// (10240 rows of 5 shared and up to 3 own partials of 128: 11 us) and, for few
// rows, by the way from the lengths to the partials' places (4.4 us).
// ---------------------------------------------------------------------------
template <int D, int FMT, int DT>
__global__ __launch_bounds__(kMergeThreads) void decode_merge_kernel(DecodeAttnArgs a, int split) {
  constexpr int kLanes = D / 4, kSlots = kMergeThreads / kLanes;
  __shared__ __attribute__((aligned(16))) float s_o[kSlots][D];
  __shared__ float s_ml[kSlots][2];
  const int slot = threadIdx.x / kLanes, d0 = 4 * (threadIdx.x % kLanes);
  const int64_t all_rows = (int64_t)a.plan.tokens * a.n_q_heads;
  const int64_t row = ((int64_t)blockIdx.x * blockDim.x / kLanes + slot) / split;
  const bool in = row < all_rows;
  const int token = in ? (int)(row / a.n_q_heads) : 0, head = in ? (int)(row - (int64_t)token * a.n_q_heads) : 0;
  const int seq = token / a.batch.n_new, tok_in = token - seq * a.batch.n_new;
  const int len = own_len(a, seq);
  const int limit = len - a.batch.n_new + tok_in + 1;
  // The sequence's steps and, of the groups' runs, the first and the number
  // that touch them.
  const int steps = steps_of<D, FMT>(len);
  // One pass over the lengths for all rows of the wave (4096 sequences of 200 keys: 26 us; with a scan of every 64 57).
  const int seq0 = __builtin_amdgcn_readfirstlane(seq);      // of its first row
  int sum = 0, begin = 0;                    // steps of all sequences, and of those before
  for (int b = threadIdx.x & 63; b < a.batch.batch; b += 64) {
    const int s = steps_of<D, FMT>(own_len(a, b));
    sum += s;
    begin += b < seq0 ? s : 0;
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    sum += __shfl_xor(sum, s);
    begin += __shfl_xor(begin, s);
  }
  for (int b = seq0; b < seq; ++b) begin += steps_of<D, FMT>(own_len(a, b));   // a wave has 256 / D rows
  const int per = max(1, (sum + a.plan.groups - 1) / a.plan.groups);
  const int r0 = begin / per, own = steps > 0 ? (begin + steps - 1) / per - r0 + 1 : 0;
  const int shared = a.plan.shared_chunks;
  const int parts = in && len >= 0 ? shared + own : 0;
  const int64_t seq_rows = (int64_t)a.batch.n_new * a.n_q_heads;
  const int64_t own0 = shared * all_rows + (int64_t)(r0 + seq) * seq_rows + (int64_t)tok_in * a.n_q_heads + head;
  auto row_of = [&](int p) { return p < shared ? p * all_rows + row : own0 + (p - shared) * seq_rows; };

  float m = kNegInf, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  constexpr int kAhead = 4;
  for (int p = slot % split; p < parts; p += split * kAhead) {
    float2 ml[kAhead];
    f32x4 v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const bool have = p + i * split < parts;
      const int64_t at = row_of(have ? p + i * split : p);
      ml[i] = a.part_ml[at];
      v[i] = *reinterpret_cast<const f32x4 *>(a.part_o + at * D + d0);
      if (!have) ml[i] = float2{kNegInf, 0.f}, v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) top = fmaxf(top, ml[i].x);
    const float ref = top == kNegInf ? 0.f : top;
    const float f = __builtin_amdgcn_exp2f(m - ref);
    l *= f;
    o *= f;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float w = __builtin_amdgcn_exp2f(ml[i].x - ref);
      l += w * ml[i].y;
      o += w * v[i];
    }
    m = top;
  }
  if (split > 1) {
    *reinterpret_cast<f32x4 *>(&s_o[slot][d0]) = o;
    if (d0 == 0) s_ml[slot][0] = m, s_ml[slot][1] = l;
    __syncthreads();
    if (slot % split != 0) return;
    for (int j = 0; j < split; ++j) m = fmaxf(m, s_ml[slot + j][0]);
    const float ref = m == kNegInf ? 0.f : m;
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < split; ++j) {
      const float w = __builtin_amdgcn_exp2f(s_ml[slot + j][0] - ref);
      l += w * s_ml[slot + j][1];
      o += w * *reinterpret_cast<const f32x4 *>(&s_o[slot + j][d0]);
    }
  }
  if (!in) return;
  const bool none = len == -1 || (len >= 0 && limit <= 0 && a.batch.shared_len == 0);
  if (len == kBad) l = __builtin_nanf("");
  const float inv = 1.f / l;
  u32x2 w;
  w.x = none ? 0u : pack16<DT>(o[0] * inv, o[1] * inv);
  w.y = none ? 0u : pack16<DT>(o[2] * inv, o[3] * inv);
  *reinterpret_cast<u32x2 *>(a.out + row * D + d0) = w;
  if (d0 == 0 && a.lse != nullptr)
    a.lse[(int64_t)head * a.plan.tokens + token] = none ? kNegInf : (m + __builtin_log2f(l)) * 0.6931471805599453f;
}

template <int D, int FMT, int DT, bool WIDE>
hipError_t launch_chunks(const DecodeAttnArgs &a, hipStream_t stream) {
  const DecodePlan &pl = a.plan;
  constexpr int waves = WIDE ? kWideWaves : kWaves;
  static_assert(sizeof(WideLds<D>) >= kWideWaves * sizeof(NarrowLds), "both bodies' LDS");
  const size_t lds = WIDE ? sizeof(WideLds<D>) : waves * (sizeof(NarrowLds) + (pl.joined ? sizeof(JoinLds<D>) : 0));
  const void *kernel = reinterpret_cast<const void *>(&decode_attn_kernel<D, FMT, DT, WIDE>);
  if (lds > 64 * 1024) {
    static std::atomic<uint64_t> ready{0};   // devices on which the kernel may use that much LDS
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = (uint64_t)1 << (dev & 63);
    if (!(ready.load(std::memory_order_relaxed) & bit) || dev > 63) {
      e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) return e;
      ready.fetch_or(bit, std::memory_order_relaxed);
    }
  }
  const int heads = a.pool.n_kv_heads;
  const int shared_rows = WIDE ? kWideRows : 16;
  const int shared_tiles = (pl.tokens * pl.group + shared_rows - 1) / shared_rows;
  const int own_tiles = (pl.rows + 15) / 16;
  auto narrow_groups = [&](int64_t units) { return (units * heads + waves - 1) / waves; };
  const int shared_groups = WIDE ? heads * shared_tiles * pl.shared_chunks
                                 : (int)narrow_groups((int64_t)shared_tiles * pl.shared_chunks);
  const int64_t groups =
      pl.joined ? (int64_t)heads * own_tiles * a.batch.batch
                : shared_groups + narrow_groups((int64_t)own_tiles * (pl.direct ? a.batch.batch : pl.groups));
  hipLaunchKernelGGL((decode_attn_kernel<D, FMT, DT, WIDE>), dim3((unsigned)groups), dim3(64 * waves), lds, stream, a,
                     shared_groups, shared_tiles, own_tiles);
  return hipGetLastError();
}

template <int D, int FMT, int DT>
hipError_t launch_all(const DecodeAttnArgs &a, hipStream_t stream) {
  const DecodePlan &pl = a.plan;
  const hipError_t e = pl.shared_wide && pl.shared_chunks > 0 ? launch_chunks<D, FMT, DT, true>(a, stream)
                                                              : launch_chunks<D, FMT, DT, false>(a, stream);
  if (e != hipSuccess || pl.direct || pl.joined) return e;
  // A row's partials: all shared chunks, and the own keys' share of the groups
  // if the sequences were equally long (the rows of longer ones loop).
  const int parts = pl.shared_chunks + (pl.groups + a.batch.batch - 1) / a.batch.batch;
  constexpr int lanes = D / 4;
  int split = 1;
  while (split < kMergeThreads / lanes && 4 * split <= parts) split *= 2;
  const int threads = std::max(256, split * lanes);
  const int64_t per = threads / lanes / split, all_rows = (int64_t)pl.tokens * a.n_q_heads;
  hipLaunchKernelGGL((decode_merge_kernel<D, FMT, DT>), dim3((unsigned)((all_rows + per - 1) / per)), dim3(threads), 0,
                     stream, a, split);
  return hipGetLastError();
}

template <int D, int FMT>
hipError_t launch_dtype(const DecodeAttnArgs &a, hipStream_t stream) {
  return a.pool.dtype == SC_DTYPE_BF16 ? launch_all<D, FMT, SC_DTYPE_BF16>(a, stream)
                                       : launch_all<D, FMT, SC_DTYPE_F16>(a, stream);
}
template <int D>
hipError_t launch_format(const DecodeAttnArgs &a, hipStream_t stream) {
  switch (a.pool.kv_format) {
    case SC_KV_16BIT: return launch_dtype<D, SC_KV_16BIT>(a, stream);
    case SC_KV_INT8: return launch_dtype<D, SC_KV_INT8>(a, stream);
    default: return launch_dtype<D, SC_KV_E4M3>(a, stream);
  }
}

}  // namespace

hipError_t launch_decode_attn(const DecodeAttnArgs &a, hipStream_t stream) {
  return a.pool.head_dim == 128 ? launch_format<128>(a, stream) : launch_format<64>(a, stream);
}

}  // namespace sc
