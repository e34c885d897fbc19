// kvq_paged_append: rotation of queries and keys by position, group-wise quantization of keys and values (App. B.1 quantizer per
// group) and packing into the pages that a block table names.
//
// A row (one head of one token) is spread over D / 8 lanes, eight consecutive channels each: half-split pairs are a shuffle apart, interleaved
// ones sit in a lane, and a group's minimum and maximum are a few shuffles.
#include "kvq_paged.cuh"
#include "kvq_quantize.cuh"

namespace kvq {

namespace {

constexpr int kThreads = 256, kValueThreads = 128;

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

// A lane's part of a position's rows of the table: cos, sin of its eight channels' pairs (of four pairs, twice, where interleaved).
template <int D>
__device__ __forceinline__ void load_angles(const RopeArgs& r, int t, int l, float (&c)[8], float (&s)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) { c[i] = 1.0f; s[i] = 0.0f; }
  const int lh = r.half >> 3;                    // lanes of the first halves of the pairs, then as many of the second
  if (l >= 2 * lh) return;
  const long long at = (long long)t * r.half + (r.interleaved ? 4 * l : 8 * (l >= lh ? l - lh : l));
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const int j = r.interleaved ? 0 : i;
    *reinterpret_cast<float4*>(c + i) = __ldg(reinterpret_cast<const float4*>(r.cos + at + j));
    *reinterpret_cast<float4*>(s + i) = __ldg(reinterpret_cast<const float4*>(r.sin + at + j));
  }
}

// Rotation of a row, lane l of its D / 8 lanes holding channels 8 l .. 8 l + 7.  All lanes of the warp take part (channels from rotary_dim
// on stay as they are).
template <int D>
__device__ __forceinline__ void rotate_row(float (&x)[8], const RopeArgs& r, const float (&c)[8], const float (&s)[8], int l) {
  const int lh = r.half >> 3;
  const bool turned = l < 2 * lh;
  if (r.interleaved) {
    if (turned) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = x[2 * i], b = x[2 * i + 1];
        x[2 * i] = __fsub_rn(__fmul_rn(a, c[i]), __fmul_rn(b, s[i]));
        x[2 * i + 1] = __fadd_rn(__fmul_rn(b, c[i]), __fmul_rn(a, s[i]));
      }
    }
  } else {
    const bool second = l >= lh;
    const int partner = !turned ? l : second ? l - lh : l + lh;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float o = __shfl_sync(FULL, x[i], partner, D / 8);
      const float own = __fmul_rn(x[i], c[i]), other = __fmul_rn(o, s[i]);
      const float y = second ? __fadd_rn(own, other) : __fsub_rn(own, other);
      x[i] = turned ? y : x[i];
    }
  }
}

// Rows of a token: n_kv_heads keys, as many values where V_ROWS, then the query heads.  A warp takes 256 / D of them at a time and
// `groups` such in a row, the next two's loads in flight: the token's angles stay in registers.
// Long calls are bound by the memory system (8B shape, 32,768 tokens: see launch_paged_append), single tokens by latency.
template <int D, int DTYPE, bool V_ROWS>
__global__ void __launch_bounds__(kThreads, 4)
paged_append_rows_kernel(Geom g, Paged p, AppendArgs a, int per_token, int groups) {
  constexpr int LPR = D / 8, RPW = 32 / LPR;
  const int lane = threadIdx.x & 31, l = lane % LPR;
  const int parts = (per_token + groups - 1) / groups;
  const long long task = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  begin_after_predecessor();
  const int row = (int)(task / parts);
  if (row >= p.n_rows) return;                                           // (whole warps)
  const int g0 = (int)(task - (long long)row * parts) * groups, g1 = min(g0 + groups, per_token);
  const int n_slots = (V_ROWS ? 2 : 1) * g.Hkv + (a.q ? g.Hq : 0), v_end = V_ROWS ? 2 * g.Hkv : g.Hkv;
  struct Slot { int head; bool is_k, is_v, on; };
  auto slot_of = [&](int group) {
    const int i = group * RPW + lane / LPR;
    Slot s;
    s.on = i < n_slots; s.is_k = i < g.Hkv; s.is_v = !s.is_k && i < v_end;
    s.head = s.is_k ? i : s.is_v ? i - g.Hkv : i - v_end;
    return s;
  };
  auto fetch = [&](int group) {
    const Slot s = slot_of(group);
    const uint16_t* src = s.is_k ? a.k : s.is_v ? a.v : a.q;
    src += s.is_k || s.is_v ? (long long)row * a.kv_row + (long long)s.head * a.kv_head : (long long)row * a.q_row + (long long)s.head * a.q_head;
    return s.on ? __ldcs(reinterpret_cast<const uint4*>(src + 8 * l)) : make_uint4(0u, 0u, 0u, 0u);
  };
  // (on their way while the sequence is looked up; rows of padding exist too)
  uint4 next = fetch(g0), after = g0 + 1 < g1 ? fetch(g0 + 1) : make_uint4(0u, 0u, 0u, 0u);
  const int b = sequence_of(p.cu, g.B, row, lane);
  bool bad;
  const int limit = a.rope.half ? min(g.capacity, a.rope.n_positions) : g.capacity;
  const SeqRows s = seq_rows(p, b, limit, p.n_rows, bad);
  if (bad && lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
  if (row < s.first || row >= s.first + s.rows) return;
  const int t = s.n - s.rows + (row - s.first);
  const int id = pool_page(p, b, t >> 7);
  if (id < 0 && lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
  float ac[8], as[8];
  if (a.rope.half) load_angles<D>(a.rope, t, l, ac, as);
#pragma unroll 1
  for (int group = g0; group < g1; ++group) {
  const Slot sl = slot_of(group);
  const bool active = sl.on, is_k = sl.is_k, is_v = sl.is_v;
  const int head = sl.head;
  const uint4 raw = next;
  next = after;
  if (group + 2 < g1) after = fetch(group + 2);
  float x[8];
  unpack8<DTYPE>(raw, x);
  if (a.rope.half) {
    if (V_ROWS) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = x[i];
      rotate_row<D>(y, a.rope, ac, as, l);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = is_v ? x[i] : y[i];
    } else {
      rotate_row<D>(x, a.rope, ac, as, l);
    }
  }
  if (active && !is_k && !is_v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bits16(x[2 * i], DTYPE) | ((uint32_t)f32_to_bits16(x[2 * i + 1], DTYPE) << 16);
    *reinterpret_cast<uint4*>(a.q_out + ((long long)row * g.Hq + head) * D + 8 * l) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  if (__all_sync(FULL, !active || (!is_k && !is_v))) continue;
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
  if (!active || id < 0 || (!is_k && !is_v)) continue;
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
}

// Values of a long call: a warp takes the tokens of one task of 32 (64) of one head, so that the codes of four tokens leave as words.
template <int D, int BITS, int DTYPE>
__global__ void __launch_bounds__(kValueThreads)
paged_append_values_kernel(Geom g, Paged p, AppendArgs a) {
  constexpr int FPB = 8 / BITS, LR = 2 * (D / 16) / FPB, RS = 32 / LR, TT = task_tokens(D, BITS), TK = pass_tokens(BITS, true), NP = TT / RS / TK;
  const int lane = threadIdx.x & 31;
  const long long task = (long long)blockIdx.x * (kValueThreads / 32) + (threadIdx.x >> 5);
  begin_after_predecessor();
  const int h = (int)(task % g.Hkv);
  const BlockTask bt = block_task(p, g.B, (int)(task / g.Hkv), TT, a.rope.half ? min(g.capacity, a.rope.n_positions) : g.capacity, p.n_rows, lane);
  if (bt.lo >= bt.hi) return;
  const int id = pool_page(p, bt.b, bt.t0 >> 7);
  if (id < 0) {
    if (lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
    return;
  }
  uint8_t* pg = p.pages + ((size_t)id * g.Hkv + h) * g.page_bytes;
  const int tp0 = bt.t0 & 127;
  uint8_t* codes = pg + g.v_codes_off + (size_t)(tp0 >> 5) * (4 * D * BITS);
  uint32_t* meta = reinterpret_cast<uint32_t*>(pg + g.v_meta_off) + tp0 * (D / g.gv);
  const int rs = lane / LR, cs = lane % LR;
  const uint16_t* src = a.v + (long long)bt.row0 * a.kv_row + (long long)h * a.kv_head + 16 * FPB * (cs >> 1) + 8 * (cs & 1);
#pragma unroll 1
  for (int pass = 0; pass < NP; ++pass) {
    auto load = [&](int kk, int f) {             // (tokens that are not new: any that is)
      const int tau = token_slot<true, RS>(TK * pass + kk, rs);
      return __ldcs(reinterpret_cast<const uint4*>(src + (long long)(min(max(tau, bt.lo), bt.hi - 1)) * a.kv_row + 16 * f));
    };
    if (!quantize_pass<BITS, true, D, DTYPE, true>(load, [] {}, g.gv, bt.lo, bt.hi, codes, meta, lane, pass))
      quantize_pass<BITS, true, D, DTYPE, false>(load, [] {}, g.gv, bt.lo, bt.hi, codes, meta, lane, pass);
  }
}

}  // namespace

int launch_paged_append(const Geom& g, const Paged& p, const void* k, const void* v, int64_t kv_row, int64_t kv_head,
                        const RopeArgs& rope, const void* q, int64_t q_row, int64_t q_head, void* q_out, cudaStream_t stream) {
  const AppendArgs a{static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), static_cast<const uint16_t*>(q),
                     static_cast<uint16_t*>(q_out), kv_row, kv_head, q_row, q_head, rope};
  // Values go by token rows (their codes then leave byte by byte) in short calls, by blocks of tokens in a launch of their own in long ones.
  const bool blocks = p.n_rows >= 8 * g.B && p.n_rows >= 64;
  const int rpw = 256 / g.D, per_token = ((blocks ? 1 : 2) * g.Hkv + (q ? g.Hq : 0) + rpw - 1) / rpw;
  // enough warps to fill the GPU twice, then longer ones
  const long long warps = (long long)p.n_rows * per_token;
  int groups = (int)(warps / (148 * 64) < 1 ? 1 : warps / (148 * 64) > per_token ? per_token : warps / (148 * 64));
  groups = (per_token + (per_token + groups - 1) / groups - 1) / ((per_token + groups - 1) / groups);      // equal parts
  const long long ctas = ((long long)p.n_rows * ((per_token + groups - 1) / groups) + kThreads / 32 - 1) / (kThreads / 32);
  if (ctas > 0x7FFFFFFFll) return KVQ_ERR_INVALID_ARG;
  auto rows = [&](auto kern) { return launch_dependent(kern, dim3((unsigned)ctas), kThreads, 0, stream, 1, g, p, a, per_token, groups); };
  const bool bf = g.in_dtype == KVQ_BF16;
  cudaError_t e;
#define KVQ_ROWS(D_, V_) rows(bf ? paged_append_rows_kernel<D_, KVQ_BF16, V_> : paged_append_rows_kernel<D_, KVQ_FP16, V_>)
  if (g.D == 128) e = blocks ? KVQ_ROWS(128, false) : KVQ_ROWS(128, true);
  else e = blocks ? KVQ_ROWS(64, false) : KVQ_ROWS(64, true);
#undef KVQ_ROWS
  if (e != cudaSuccess) return KVQ_ERR_CUDA_LAUNCH;
  if (!blocks) return KVQ_OK;
  const long long tasks = block_tasks(p.n_rows, g.B, task_tokens(g.D, g.vb)) * g.Hkv;
  const long long vctas = (tasks + kValueThreads / 32 - 1) / (kValueThreads / 32);
  if (vctas > 0x7FFFFFFFll) return KVQ_ERR_INVALID_ARG;
  auto values = [&](auto kern) { return launch_dependent(kern, dim3((unsigned)vctas), kValueThreads, 0, stream, 1, g, p, a); };
#define KVQ_VALUES(D_, B_) \
  if (g.D == D_ && g.vb == B_) e = values(bf ? paged_append_values_kernel<D_, B_, KVQ_BF16> : paged_append_values_kernel<D_, B_, KVQ_FP16>);
  KVQ_VALUES(128, 2) KVQ_VALUES(128, 4) KVQ_VALUES(128, 8) KVQ_VALUES(64, 2) KVQ_VALUES(64, 4) KVQ_VALUES(64, 8)
#undef KVQ_VALUES
  return e == cudaSuccess ? KVQ_OK : KVQ_ERR_CUDA_LAUNCH;
}

}  // namespace kvq
