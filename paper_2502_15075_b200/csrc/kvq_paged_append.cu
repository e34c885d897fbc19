// kvq_paged_append: rotation of queries and keys by position, group-wise quantization of keys and values (App. B.1 quantizer per
// group) and packing into the pages that a block table names.
//
// A row (one head of one token) is spread over D / 8 lanes, eight consecutive channels each: half-split pairs are a shuffle apart, interleaved
// ones sit in a lane, and a group's minimum and maximum are a few shuffles.
#include "kvq_paged.cuh"
#include "kvq_quantize.cuh"

namespace kvq {

namespace {

constexpr int kThreads = 256;

struct AppendArgs {
  const uint16_t *k, *v, *q;
  uint16_t* q_out;
  long long kv_row, kv_head, q_row, q_head;
  RopeArgs rope;
};

template <int DTYPE>
__device__ __forceinline__ void unpack8(const uint4& raw, float (&x)[8]) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bits16_to_f32((uint16_t)(w[i] & 0xFFFF), DTYPE);
    x[2 * i + 1] = bits16_to_f32((uint16_t)(w[i] >> 16), DTYPE);
  }
}

// Rotation of a row, lane l of its D / 8 lanes holding channels 8 l .. 8 l + 7; cos, sin: the position's rows of the table.  All lanes of
// the warp take part (channels from rotary_dim on stay as they are).
template <int D>
__device__ __forceinline__ void rotate_row(float (&x)[8], const RopeArgs& r, const float* cos, const float* sin, int l) {
  if (r.interleaved) {
    if (8 * l < 2 * r.half) {
      const float4 c = *reinterpret_cast<const float4*>(cos + 4 * l), s = *reinterpret_cast<const float4*>(sin + 4 * l);
      const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = x[2 * i], b = x[2 * i + 1];
        x[2 * i] = __fsub_rn(__fmul_rn(a, cc[i]), __fmul_rn(b, ss[i]));
        x[2 * i + 1] = __fadd_rn(__fmul_rn(b, cc[i]), __fmul_rn(a, ss[i]));
      }
    }
  } else {
    const int lh = r.half >> 3;                  // lanes of the first halves of the pairs, then as many of the second
    const bool second = l >= lh, turned = l < 2 * lh;
    const int partner = !turned ? l : second ? l - lh : l + lh;
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = __shfl_sync(FULL, x[i], partner, D / 8);
    if (turned) {
      const int at = 8 * (second ? l - lh : l);
      float cc[8], ss[8];
      *reinterpret_cast<float4*>(cc) = *reinterpret_cast<const float4*>(cos + at);
      *reinterpret_cast<float4*>(cc + 4) = *reinterpret_cast<const float4*>(cos + at + 4);
      *reinterpret_cast<float4*>(ss) = *reinterpret_cast<const float4*>(sin + at);
      *reinterpret_cast<float4*>(ss + 4) = *reinterpret_cast<const float4*>(sin + at + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float own = __fmul_rn(x[i], cc[i]), other = __fmul_rn(o[i], ss[i]);
        x[i] = second ? __fadd_rn(own, other) : __fsub_rn(own, other);
      }
    }
  }
}

// Rows of a token: n_kv_heads keys, as many values, then the query heads; a warp takes 256 / D of them.
template <int D, int DTYPE>
__global__ void __launch_bounds__(kThreads)
paged_append_rows_kernel(Geom g, Paged p, AppendArgs a, int per_token) {
  constexpr int LPR = D / 8, RPW = 32 / LPR;
  const int lane = threadIdx.x & 31, l = lane % LPR;
  const long long task = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  begin_after_predecessor();
  const int row = (int)(task / per_token);
  if (row >= p.n_rows) return;                                           // (whole warps)
  const int part = (int)(task - (long long)row * per_token);
  const int b = sequence_of(p.cu, g.B, row, lane);
  bool bad;
  const int limit = a.rope.half ? min(g.capacity, a.rope.n_positions) : g.capacity;
  const SeqRows s = seq_rows(p, b, limit, p.n_rows, bad);
  if (bad && lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
  if (row < s.first || row >= s.first + s.rows) return;
  const int t = s.n - s.rows + (row - s.first);
  const int slot = part * RPW + lane / LPR, slots = 2 * g.Hkv + (a.q ? g.Hq : 0);
  const bool active = slot < slots;
  const int head = slot < g.Hkv ? slot : slot < 2 * g.Hkv ? slot - g.Hkv : slot - 2 * g.Hkv;
  const bool is_k = slot < g.Hkv, is_v = !is_k && slot < 2 * g.Hkv;
  const uint16_t* src = is_k ? a.k : is_v ? a.v : a.q;
  src += is_k || is_v ? (long long)row * a.kv_row + (long long)head * a.kv_head : (long long)row * a.q_row + (long long)head * a.q_head;
  uint4 raw = make_uint4(0u, 0u, 0u, 0u);
  if (active) raw = *reinterpret_cast<const uint4*>(src + 8 * l);
  const int id = pool_page(p, b, t >> 7);
  if (id < 0 && lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
  float x[8];
  unpack8<DTYPE>(raw, x);
  if (a.rope.half) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
    rotate_row<D>(y, a.rope, a.rope.cos + (long long)t * a.rope.half, a.rope.sin + (long long)t * a.rope.half, l);
    if (!is_v) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = y[i];
    }
  }
  if (active && !is_k && !is_v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bits16(x[2 * i], DTYPE) | ((uint32_t)f32_to_bits16(x[2 * i + 1], DTYPE) << 16);
    *reinterpret_cast<uint4*>(a.q_out + ((long long)row * g.Hq + head) * D + 8 * l) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  if (__all_sync(FULL, !active || (!is_k && !is_v))) return;
  // ---- quantize (queries of a mixed warp go along and are not stored)
  const int bits = is_v ? g.vb : g.kb, gsz = is_v ? g.gv : g.gk, lpg = gsz >> 3;       // lanes per group
  const float qmax = (float)((1 << bits) - 1);
  float mn = fminf(fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), fminf(fminf(x[4], x[5]), fminf(x[6], x[7])));
  float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
#pragma unroll
  for (int off = 1; off < LPR; off <<= 1) {
    const float lo = __shfl_xor_sync(FULL, mn, off), hi = __shfl_xor_sync(FULL, mx, off);
    if (off < lpg) { mn = fminf(mn, lo); mx = fmaxf(mx, hi); }
  }
  const GroupParams gp = group_params(mn, mx, qmax);
  uint32_t n[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) n[i] = code_of_fast(x[i], gp, qmax);
  // fields of a byte: channels 16 apart, that is lanes 2 (and 4) apart; every lane of a byte ends up with all its fields
  const int lf = bits == 8 ? 0 : bits == 4 ? 1 : 2;      // log2 of the fields per byte
  const int rh = l & 1, f = (l >> 1) & ((1 << lf) - 1), mw = l >> (1 + lf);
  uint32_t w[2];
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    w[hh] = (n[4 * hh] | (n[4 * hh + 1] << 8) | (n[4 * hh + 2] << 16) | (n[4 * hh + 3] << 24)) << (bits * f);
    const uint32_t o2 = __shfl_xor_sync(FULL, w[hh], 2);
    if (lf >= 1) w[hh] |= o2;
    const uint32_t o4 = __shfl_xor_sync(FULL, w[hh], 4);
    if (lf == 2) w[hh] |= o4;
  }
  if (!active || id < 0 || (!is_k && !is_v)) return;
  uint8_t* pg = p.pages + ((size_t)id * g.Hkv + head) * g.page_bytes;
  const int tp = t & 127, ng = D / gsz;
  if ((l & (lpg - 1)) == 0) reinterpret_cast<uint32_t*>(pg + (is_v ? g.v_meta_off : g.k_meta_off))[tp * ng + (8 * l) / gsz] = gp.meta;
  if (is_k) {
    const int wpc = D * bits / 128;
    uint8_t* dst = pg + tp * (D * bits / 8);
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
      if (lf == 0 || f == hh) *reinterpret_cast<uint32_t*>(dst + chunk_word_byte(2 * rh + hh, mw, wpc, 4)) = w[hh];
  } else {
    const int tau = tp & 31, kh = tau >> 4, u = tau & 15;
    uint8_t* vb = pg + g.v_codes_off + (tp >> 5) * (4 * D * bits) + mw * 512 + ((u & 7) >> 1) * 16 + 4 * (2 * rh + kh) + 2 * (u & 1) + (u >> 3);
    const uint64_t bytes = (uint64_t)w[0] | ((uint64_t)w[1] << 32);
    for (int i = (8 >> lf) * f; i < (8 >> lf) * (f + 1); ++i) vb[64 * i] = (uint8_t)(bytes >> (8 * i));
  }
}

}  // namespace

int launch_paged_append(const Geom& g, const Paged& p, const void* k, const void* v, int64_t kv_row, int64_t kv_head,
                        const RopeArgs& rope, const void* q, int64_t q_row, int64_t q_head, void* q_out, cudaStream_t stream) {
  const AppendArgs a{static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), static_cast<const uint16_t*>(q),
                     static_cast<uint16_t*>(q_out), kv_row, kv_head, q_row, q_head, rope};
  const int rpw = 256 / g.D, per_token = (2 * g.Hkv + (q ? g.Hq : 0) + rpw - 1) / rpw;
  const long long ctas = ((long long)p.n_rows * per_token + kThreads / 32 - 1) / (kThreads / 32);
  if (ctas > 0x7FFFFFFFll) return KVQ_ERR_INVALID_ARG;
  auto launch = [&](auto kern) { return launch_dependent(kern, dim3((unsigned)ctas), kThreads, 0, stream, 1, g, p, a, per_token); };
  const bool bf = g.in_dtype == KVQ_BF16;
  const cudaError_t e = g.D == 128 ? launch(bf ? paged_append_rows_kernel<128, KVQ_BF16> : paged_append_rows_kernel<128, KVQ_FP16>)
                                   : launch(bf ? paged_append_rows_kernel<64, KVQ_BF16> : paged_append_rows_kernel<64, KVQ_FP16>);
  return e == cudaSuccess ? KVQ_OK : KVQ_ERR_CUDA_LAUNCH;
}

}  // namespace kvq
