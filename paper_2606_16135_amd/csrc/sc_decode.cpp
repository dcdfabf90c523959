// Host entry points of rotary positions and decode steps: argument checks,
// the rotary frequencies and the split of a decode step's keys.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>
#include <vector>

#include "sc_internal.h"

struct sc_rope {
  sc_rope_desc desc;
  std::vector<double> theta;     // scaled frequencies, radians per position
  double *d_turns = nullptr;     // theta / (2 pi) on desc.device
  float amplitude = 1.f;
};

namespace sc {
namespace {

constexpr double kPi = 3.14159265358979323846;

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// The scaled frequencies (sc_rope_scaling).
std::vector<double> frequencies(const sc_rope_desc &d) {
  const int half = d.rotary_dim / 2;
  std::vector<double> theta(half);
  auto index_of = [&](double turns) {
    return d.rotary_dim * std::log(d.original_len / (2 * kPi * turns)) / (2 * std::log(d.base));
  };
  double lo = 0, hi = 0;
  if (d.scaling == SC_ROPE_RAMP) {
    lo = std::max(0.0, std::floor(index_of(d.high)));
    hi = std::min(d.rotary_dim - 1.0, std::ceil(index_of(d.low)));
  }
  for (int i = 0; i < half; ++i) {
    const double t = std::pow(d.base, -2.0 * i / d.rotary_dim);
    double w = 1;   // share of the unscaled frequency
    if (d.scaling == SC_ROPE_LINEAR) w = 0;
    if (d.scaling == SC_ROPE_BANDED)
      w = std::clamp((d.original_len * t / (2 * kPi) - d.low) / (d.high - d.low), 0.0, 1.0);
    if (d.scaling == SC_ROPE_RAMP) w = 1 - std::clamp((i - lo) / std::max(hi - lo, 1e-3), 0.0, 1.0);
    theta[i] = w == 1 ? t : (1 - w) * (t / d.factor) + w * t;
  }
  return theta;
}

RopeView view_of(const sc_rope *r) {
  RopeView v{};
  if (r == nullptr) return v;
  v.turns = r->d_turns;
  v.half = r->desc.rotary_dim / 2;
  v.interleaved = r->desc.layout == SC_ROPE_INTERLEAVED;
  v.amplitude = r->amplitude;
  return v;
}

PoolView view_of(const sc_pool *p, int layer) {
  const sc_pool_desc &d = p->desc;
  PoolView v{};
  v.tier[0] = p->dev_base;
  v.tier[1] = p->host_dev;
  v.tier[2] = p->rc_base;
  v.first[0] = d.n_device_blocks;
  v.first[1] = d.n_device_blocks + d.n_host_blocks;
  v.n_ids = v.first[1] + d.n_rc_blocks;
  {
    std::lock_guard<std::mutex> lk(const_cast<sc_pool *>(p)->mu);
    v.lent = p->dev_lent;
  }
  v.block_bytes = (int64_t)p->block_bytes;
  v.layer_off = (int64_t)layer * (int64_t)p->slice_bytes;
  v.half_bytes = (int64_t)(p->slice_bytes / 2);
  v.scale_off = (int64_t)p->scale_off;
  v.block_size = d.block_size;
  while ((1 << v.block_shift) < d.block_size) ++v.block_shift;
  v.block_magic = (uint32_t)(((((uint64_t)1 << (31 + v.block_shift)) - 1) / (uint64_t)d.block_size) + 1);
  v.n_kv_heads = d.n_kv_heads;
  v.head_dim = d.head_dim;
  v.kv_format = p->kv_format;
  v.dtype = d.dtype;
  return v;
}

// What the three decode calls check alike.  `pointers`: the index arrays too.
sc_status check_batch(const sc_pool *pool, const sc_decode_batch *b, bool pointers) {
  if (!pool || !b) return fail(SC_ERR_INVALID, "null argument");
  if (b->batch <= 0 || b->n_new < 1 || b->n_new > 16 || b->max_blocks < 0 || b->max_len < 0 || b->shared_len < 0)
    return fail(SC_ERR_INVALID, "decode batch: batch %d, n_new %d (1..16), max_blocks %d, max_len %d, shared_len %d",
                b->batch, b->n_new, b->max_blocks, b->max_len, b->shared_len);
  if (b->batch > 65536) return fail(SC_ERR_RANGE, "a decode step of %d sequences (at most 65536)", b->batch);
  // The kernels add to a position in 32 bits: up to three tiles, and the rounding of every chunk.
  if ((int64_t)b->max_len + b->shared_len > INT32_MAX - (1 << 18))
    return fail(SC_ERR_RANGE, "%d shared and %d own tokens exceed 32-bit positions", b->shared_len, b->max_len);
  if (!pointers) return SC_OK;
  if (!b->kv_len || (b->max_blocks > 0 && !b->block_ids) || (b->shared_len > 0 && !b->shared_ids))
    return fail(SC_ERR_INVALID, "null index array in the decode batch");
  if (!aligned(b->kv_len, 4) || !aligned(b->block_ids, 4) || !aligned(b->shared_ids, 4))
    return fail(SC_ERR_INVALID, "index arrays of a decode batch must be 4-byte aligned");
  return SC_OK;
}

sc_status no_device(int device) {
  (void)hipGetLastError();
  return fail(SC_ERR_INVALID, "cannot select device %d", device);
}

DecodeView view_of(const sc_decode_batch *b) {
  return DecodeView{b->block_ids, b->kv_len,     b->shared_ids, b->batch,
                    b->n_new,     b->max_blocks, b->max_len,    b->shared_len};
}

constexpr int kDecodeCus = 256;              // MI355X
constexpr int kNarrowRows = 16;
// Waves that read own keys: two per SIMD, what a CU holds of them.
constexpr int kDecodeWaves = 8 * kDecodeCus;
constexpr int kMaxDecodeGroups = 1 << 22;    // workgroups of a launch, whose threads are counted in 32 bits
// Steps of the longest sequence up to which a workgroup takes a sequence alone
// and joins its waves in LDS, instead of waves taking equal runs of all
// sequences and a second launch merging them.  32 / 8 heads of 128, 16-bit,
// joined against apart: 1 sequence of 400 keys 7.4 against 6.0 + 4.5 us, of
// 700 10.0 against 6.0 + 4.4, of 1000 12.8 against 6.4 + 5.2; 32 sequences of
// 700 20.1 against 20.1 + 4.8; 8 of 1000 18.7 against 12.8 + 4.6.  (What bounds
// it is what one CU reads, 22 to 35 KB a us: eight waves instead of four take
// as long.)
constexpr int kJoinedSteps = 24;
// The wide part's tile of rows and keys, and the times a CU takes for one,
// measured: 256 rows 4.8 us (64 x 4 rows of 5 heads over 32768 int8 keys),
// few rows 2.5 us (the tile's loads); and what a CU reads of own keys.
constexpr int kWideRows = 256, kWideKeys = 128;
constexpr double kWideTileUs = 2.5, kWideRowUs = 4.8 / 256, kCuBytesPerUs = 22e3;
// From a workgroup's start to its first tile; writing and reading partials.
constexpr double kStartUs = 8, kPartBytesPerUs = 4e6;
constexpr int64_t kMinOwnCus = 32;

sc_status plan_decode(const sc_pool *pool, const sc_decode_batch *b, int hq, DecodePlan *out) {
  const int hkv = pool->desc.n_kv_heads;
  if (hq <= 0 || hq % hkv != 0)
    return fail(SC_ERR_INVALID, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", hq, hkv);
  if (hq / hkv > 16) return fail(SC_ERR_UNSUPPORTED, "GQA group %d > 16 not supported", hq / hkv);
  if ((int64_t)b->batch * b->n_new * hq > INT32_MAX)
    return fail(SC_ERR_RANGE, "%d x %d tokens of %d heads exceed 32-bit rows", b->batch, b->n_new, hq);
  const int step = decode_step_keys(pool->desc.head_dim, pool->kv_format);
  DecodePlan p{};
  p.group = hq / hkv;
  p.rows = b->n_new * p.group;
  p.tokens = b->batch * b->n_new;
  const int64_t all_rows = (int64_t)p.tokens * p.group;
  p.shared_wide = all_rows > kNarrowRows;
  int64_t shared_items = 0;
  const int64_t heads = (int64_t)hkv * ((p.rows + kNarrowRows - 1) / kNarrowRows);
  int64_t own_waves = kDecodeWaves;
  if (b->shared_len > 0 && p.shared_wide) {
    // A workgroup per CU, a wide one leaves a CU no room for another.  Of the
    // chunk counts that fit, the one whose estimate ends first: the own keys
    // beside the wide workgroups on the CUs those leave, or after them.  (The
    // own keys count in full: their lengths are not known here.)
    const int64_t tiles = (all_rows + kWideRows - 1) / kWideRows;
    const int64_t key_tiles = ((int64_t)b->shared_len + kWideKeys - 1) / kWideKeys;
    const double tile_us = std::max(kWideTileUs, kWideRowUs * (double)std::min<int64_t>(all_rows, kWideRows));
    const double own_us = (double)b->batch * b->max_len * (double)heads * (double)(pool->row_bytes / hkv) * 2 / kCuBytesPerUs;
    const int64_t most = std::max<int64_t>(1, std::min(key_tiles, kDecodeCus / (tiles * hkv)));
    int64_t chunks = 1;
    double best = 0;
    for (int64_t c = 1; c <= most; ++c) {
      const int64_t groups = tiles * hkv * c, free = kDecodeCus - groups;
      const double wide_us = tile_us * (double)((key_tiles + c - 1) / c) * (double)((groups + kDecodeCus - 1) / kDecodeCus);
      const bool beside = free >= kMinOwnCus;
      const double parts_us = (double)(c * p.tokens * hq) * pool->desc.head_dim * 8 / kPartBytesPerUs;
      const double us = parts_us + kStartUs + (beside ? std::max(wide_us, own_us / (double)free)
                                                      : wide_us + kStartUs + own_us / kDecodeCus);
      if (c > 1 && us >= best) continue;
      best = us;
      chunks = c;
      own_waves = beside && own_us / (double)free <= 1.1 * wide_us + 5 ? 8 * free : kDecodeWaves;
    }
    p.shared_chunk = (int32_t)((key_tiles + chunks - 1) / chunks * kWideKeys);
    p.shared_chunks = (b->shared_len + p.shared_chunk - 1) / p.shared_chunk;
    shared_items = tiles * hkv * p.shared_chunks;
  } else if (b->shared_len > 0) {
    // A wave per step, up to two per SIMD.
    const int64_t steps = ((int64_t)b->shared_len + step - 1) / step;
    const int64_t chunks = std::min<int64_t>(steps, std::max(1, kDecodeWaves / hkv));
    p.shared_chunk = (int32_t)((steps + chunks - 1) / chunks * step);
    p.shared_chunks = (b->shared_len + p.shared_chunk - 1) / p.shared_chunk;
    shared_items = (int64_t)hkv * p.shared_chunks;
  }
  // Own keys: as many groups as the device holds waves, but no more than
  // there can be steps.
  const int64_t steps = (int64_t)b->batch * std::max<int64_t>(1, ((int64_t)b->max_len + step - 1) / step);
  if (steps > (1 << 30))   // the device adds the sequences' steps in 32 bits
    return fail(SC_ERR_RANGE, "%d sequences of up to %d tokens are too many keys for a decode step", b->batch, b->max_len);
  p.groups = (int32_t)std::max<int64_t>(1, std::min<int64_t>(own_waves / heads, steps));
  p.direct = b->shared_len == 0 && b->max_len <= step;
  p.joined = b->shared_len == 0 && !p.direct && b->max_len <= kJoinedSteps * step;
  if (heads * std::max<int64_t>(p.groups, p.direct || p.joined ? b->batch : 0) > kMaxDecodeGroups || shared_items > kMaxDecodeGroups ||
      (all_rows + 15) / 16 * hkv > kMaxDecodeGroups)
    return fail(SC_ERR_RANGE, "a decode step of %d sequences x %d KV heads needs too many workgroups", b->batch, hkv);
  *out = p;
  return SC_OK;
}

// Partial outputs, then their (maximum, sum) pairs.
size_t workspace_bytes_of(const DecodePlan &p, const sc_decode_batch *b, int hq, int head_dim, size_t *ml_off) {
  const size_t seq_rows = (size_t)b->n_new * hq;
  const size_t rows =
      p.direct || p.joined ? 0 : (size_t)p.shared_chunks * b->batch * seq_rows + ((size_t)p.groups + b->batch) * seq_rows;
  *ml_off = rows * head_dim * sizeof(float);
  return *ml_off + rows * sizeof(float2);
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" {

sc_status sc_rope_create(const sc_rope_desc *desc, sc_rope **out) {
  clear_error();
  if (!desc || !out) return fail(SC_ERR_INVALID, "null argument");
  *out = nullptr;
  const sc_rope_desc &d = *desc;
  if (d.head_dim != 64 && d.head_dim != 128)
    return fail(SC_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", d.head_dim);
  if (d.rotary_dim < 16 || d.rotary_dim > d.head_dim || d.rotary_dim % 16 != 0)
    return fail(SC_ERR_UNSUPPORTED, "rotary_dim %d not supported (a multiple of 16 up to head_dim %d)", d.rotary_dim,
                d.head_dim);
  if (d.layout != SC_ROPE_HALF && d.layout != SC_ROPE_INTERLEAVED)
    return fail(SC_ERR_INVALID, "unknown rotary layout %d", d.layout);
  if (d.scaling < SC_ROPE_PLAIN || d.scaling > SC_ROPE_RAMP)
    return fail(SC_ERR_INVALID, "unknown rotary scaling %d", d.scaling);
  if (!(d.base > 1) || !std::isfinite(d.base)) return fail(SC_ERR_INVALID, "rotary base must be above 1");
  if (d.scaling != SC_ROPE_PLAIN && (!(d.factor > 0) || !std::isfinite(d.factor)))
    return fail(SC_ERR_INVALID, "rotary factor must be positive");
  if ((d.scaling == SC_ROPE_BANDED || d.scaling == SC_ROPE_RAMP) &&
      (!(d.original_len > 0) || !std::isfinite(d.original_len) || !(d.low > 0) || !(d.high > d.low) ||
       !std::isfinite(d.high)))
    return fail(SC_ERR_INVALID, "rotary scaling needs original_len > 0 and 0 < low < high");
  if (!(d.amplitude >= 0) || !std::isfinite(d.amplitude))
    return fail(SC_ERR_INVALID, "rotary amplitude must not be negative");
  try {
    std::unique_ptr<sc_rope> r(new sc_rope());
    r->desc = d;
    r->theta = frequencies(d);
    double amplitude = d.amplitude;
    if (amplitude == 0) amplitude = d.scaling == SC_ROPE_RAMP ? std::max(1.0, 0.1 * std::log(d.factor) + 1.0) : 1.0;
    r->amplitude = (float)amplitude;
    std::vector<double> turns(r->theta);
    for (double &t : turns) t /= 2 * kPi;
    // (a failed hipSetDevice would be reported again by the process's next launch)
    int devices = 0;
    if (hipGetDeviceCount(&devices) != hipSuccess || d.device < 0 || d.device >= devices) {
      (void)hipGetLastError();
      return fail(SC_ERR_INVALID, "device %d of %d", d.device, devices);
    }
    DeviceGuard guard(d.device);
    const size_t bytes = turns.size() * sizeof(double);
    hipError_t e = hipMalloc(reinterpret_cast<void **>(&r->d_turns), bytes);
    if (e == hipSuccess) {
      e = hipMemcpy(r->d_turns, turns.data(), bytes, hipMemcpyHostToDevice);
      if (e != hipSuccess) (void)hipFree(r->d_turns);
    }
    if (e != hipSuccess) {
      (void)hipGetLastError();
      return fail_hip(e, "rotary frequencies");
    }
    *out = r.release();
  } catch (const std::bad_alloc &) {
    return fail(SC_ERR_OOM, "out of host memory");
  }
  return SC_OK;
}

void sc_rope_destroy(sc_rope *rope) {
  if (!rope) return;
  if (rope->d_turns) {
    DeviceGuard guard(rope->desc.device);
    (void)hipFree(rope->d_turns);
  }
  delete rope;
}

sc_status sc_rope_frequencies(const sc_rope *rope, double *theta, int32_t capacity, int32_t *n) {
  clear_error();
  if (!rope || !n) return fail(SC_ERR_INVALID, "null argument");
  *n = (int32_t)rope->theta.size();
  if (!theta) return SC_OK;
  if (capacity < *n) return fail(SC_ERR_RANGE, "capacity %d < %d frequencies", capacity, *n);
  std::copy(rope->theta.begin(), rope->theta.end(), theta);
  return SC_OK;
}

sc_status sc_rope_apply(const sc_rope *rope, int32_t dtype, int64_t n_tokens, const int32_t *positions,
                        const void *q, int64_t q_stride, int32_t n_q_heads, void *q_out, int64_t q_out_stride,
                        const void *k, int64_t k_stride, int32_t n_kv_heads, void *k_out, int64_t k_out_stride,
                        void *stream) {
  clear_error();
  if (!rope) return fail(SC_ERR_INVALID, "null argument");
  if (dtype != SC_DTYPE_BF16 && dtype != SC_DTYPE_F16) return fail(SC_ERR_INVALID, "unknown dtype %d", dtype);
  if (n_tokens < 0 || n_q_heads < 0 || n_kv_heads < 0) return fail(SC_ERR_INVALID, "negative count");
  if (n_tokens > INT32_MAX) return fail(SC_ERR_RANGE, "%lld tokens", (long long)n_tokens);
  RopeArgs a{};
  a.rope = view_of(rope);
  a.positions = positions;
  a.n_tokens = (int32_t)n_tokens;
  a.dtype = dtype;
  a.dim_shift = rope->desc.head_dim == 128 ? 7 : 6;
  const void *x[2] = {q, k};
  void *y[2] = {q_out, k_out};
  const int64_t xs[2] = {q_stride, k_stride}, ys[2] = {q_out_stride, k_out_stride};
  const int32_t heads[2] = {n_q_heads, n_kv_heads};
  if (n_tokens > 0 && heads[0] + (int64_t)heads[1] > 0 && (!positions || !aligned(positions, 4)))
    return fail(SC_ERR_INVALID, "positions must be a 4-byte aligned device array");
  // A workgroup's units (at most 16 per head of four tokens) are counted in 32 bits.
  if (heads[0] + (int64_t)heads[1] > (1 << 24)) return fail(SC_ERR_RANGE, "too many heads");
  for (int i = 0; i < 2; ++i) {
    if (heads[i] == 0 || n_tokens == 0) continue;
    if (!x[i] || !y[i]) return fail(SC_ERR_INVALID, "null argument");
    if (!aligned(x[i], 16) || !aligned(y[i], 16))
      return fail(SC_ERR_INVALID, "q, k and their outputs must be 16-byte aligned");
    const int64_t row = (int64_t)heads[i] * rope->desc.head_dim;
    if (xs[i] < row || ys[i] < row || xs[i] % 8 != 0 || ys[i] % 8 != 0)
      return fail(SC_ERR_INVALID, "strides (%lld, %lld) must be multiples of 8 of at least %lld elements",
                  (long long)xs[i], (long long)ys[i], (long long)row);
    a.x[i] = static_cast<const uint16_t *>(x[i]);
    a.y[i] = static_cast<uint16_t *>(y[i]);
    a.x_stride[i] = xs[i];
    a.y_stride[i] = ys[i];
    a.heads[i] = heads[i];
    a.in_place[i] = x[i] == y[i];
    if (a.in_place[i] && xs[i] != ys[i]) return fail(SC_ERR_INVALID, "in place needs equal strides");
  }
  DeviceGuard guard(rope->desc.device);
  const hipError_t e = launch_rope(a, (hipStream_t)stream);
  return e == hipSuccess ? SC_OK : fail_hip(e, "rotary launch");
}

sc_status sc_decode_store(sc_pool *pool, int32_t layer, const sc_decode_batch *batch, const void *k_new,
                          const void *v_new, const sc_rope *rope, const void *q, int32_t n_q_heads, void *q_out,
                          void *stream) {
  clear_error();
  sc_status st = check_batch(pool, batch, true);
  if (st != SC_OK) return st;
  const sc_pool_desc &d = pool->desc;
  if (layer < 0 || layer >= d.n_layers) return fail(SC_ERR_RANGE, "layer %d outside [0, %d)", layer, d.n_layers);
  if (!k_new || !v_new) return fail(SC_ERR_INVALID, "null k_new/v_new");
  if (!aligned(k_new, 16) || !aligned(v_new, 16)) return fail(SC_ERR_INVALID, "k_new/v_new not 16-byte aligned");
  if (rope && rope->desc.head_dim != d.head_dim)
    return fail(SC_ERR_UNSUPPORTED, "rotary object for head_dim %d, pool has %d", rope->desc.head_dim, d.head_dim);
  if (rope && rope->desc.device != d.device)
    return fail(SC_ERR_INVALID, "rotary object of device %d, pool of device %d", rope->desc.device, d.device);
  if (q) {
    if (!rope) return fail(SC_ERR_INVALID, "q without a rotary object");
    if (n_q_heads <= 0 || !q_out) return fail(SC_ERR_INVALID, "q needs n_q_heads > 0 and q_out");
    if (!aligned(q, 16) || !aligned(q_out, 16)) return fail(SC_ERR_INVALID, "q and q_out must be 16-byte aligned");
  }
  const int hq = q ? n_q_heads : 0;
  const int64_t units = 2ll * d.n_kv_heads * (d.head_dim / 8) + (int64_t)hq * (d.head_dim / 8);
  if ((int64_t)batch->batch * batch->n_new * std::max(hq, d.n_kv_heads) > INT32_MAX || units > 65535ll * 256)
    return fail(SC_ERR_RANGE, "too many heads in a decode step");
  DecodeStoreArgs a{};
  a.pool = view_of(pool, layer);
  a.batch = view_of(batch);
  a.rope = view_of(rope);
  a.k = static_cast<const uint16_t *>(k_new);
  a.v = static_cast<const uint16_t *>(v_new);
  a.q = static_cast<const uint16_t *>(q);
  a.q_out = static_cast<uint16_t *>(q_out);
  a.n_q_heads = hq;
  a.q_in_place = q == q_out;
  DeviceGuard guard(d.device);
  if (!guard.ok()) return no_device(d.device);
  const hipError_t e = launch_decode_store(a, (hipStream_t)stream);
  return e == hipSuccess ? SC_OK : fail_hip(e, "decode store launch");
}

sc_status sc_decode_workspace(const sc_pool *pool, const sc_decode_batch *batch, int32_t n_q_heads, size_t *bytes) {
  clear_error();
  if (!bytes) return fail(SC_ERR_INVALID, "null argument");
  sc_status st = check_batch(pool, batch, false);
  if (st != SC_OK) return st;
  DecodePlan plan;
  st = plan_decode(pool, batch, n_q_heads, &plan);
  if (st != SC_OK) return st;
  size_t ml;
  *bytes = workspace_bytes_of(plan, batch, n_q_heads, pool->desc.head_dim, &ml);
  return SC_OK;
}

sc_status sc_decode_attn(sc_pool *pool, int32_t layer, const sc_decode_batch *batch, const void *q,
                         int32_t n_q_heads, float scale, void *out, float *lse, void *workspace,
                         size_t workspace_bytes, void *stream) {
  clear_error();
  sc_status st = check_batch(pool, batch, true);
  if (st != SC_OK) return st;
  const sc_pool_desc &d = pool->desc;
  if (layer < 0 || layer >= d.n_layers) return fail(SC_ERR_RANGE, "layer %d outside [0, %d)", layer, d.n_layers);
  DecodeAttnArgs a{};
  st = plan_decode(pool, batch, n_q_heads, &a.plan);
  if (st != SC_OK) return st;
  if (!q || !out) return fail(SC_ERR_INVALID, "null argument");
  if (!aligned(q, 16) || !aligned(out, 16)) return fail(SC_ERR_INVALID, "q and out must be 16-byte aligned");
  if (!aligned(lse, 4)) return fail(SC_ERR_INVALID, "lse must be 4-byte aligned");
  size_t ml_off = 0;
  const size_t need = workspace_bytes_of(a.plan, batch, n_q_heads, d.head_dim, &ml_off);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
    return fail(SC_ERR_INVALID, "the call needs a 256-byte aligned workspace of %zu bytes (got %zu)", need,
                workspace_bytes);
  a.pool = view_of(pool, layer);
  a.batch = view_of(batch);
  a.q = static_cast<const uint16_t *>(q);
  a.out = static_cast<uint16_t *>(out);
  a.lse = lse;
  a.part_o = static_cast<float *>(workspace);
  a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + ml_off);
  a.n_q_heads = n_q_heads;
  if (!(scale > 0.f)) scale = 1.f / std::sqrt((float)d.head_dim);
  a.scale_log2 = scale * 1.4426950408889634f;
  DeviceGuard guard(d.device);
  if (!guard.ok()) return no_device(d.device);
  const hipError_t e = launch_decode_attn(a, (hipStream_t)stream);
  return e == hipSuccess ? SC_OK : fail_hip(e, "decode attention launch");
}

}  // extern "C"
