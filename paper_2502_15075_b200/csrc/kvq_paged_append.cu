// kvq_paged_append: rotation of queries and keys by position, group-wise quantization of keys and values (App. B.1 quantizer per
// group) and packing into the pages that a block table names.
//
// A row (one head of one token) is spread over D / 8 lanes, eight consecutive channels each: half-split pairs are a shuffle apart, interleaved
// ones sit in a lane, and a group's minimum and maximum are a few shuffles.  8B shape with queries, K4V2: a token each for 64 sequences 3.9 us (a
// replayed graph), prompts of 4 x 8,192 tokens 165 us for 0.70 GB (keys and queries 150 with two thirds of the issue slots, values 22).
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

template <int DTYPE>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if constexpr (DTYPE == KVQ_FP16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}

// A lane's part of a position's rows of the table: cos, sin of its eight channels' pairs (of four pairs, twice, where interleaved); where
// halves are paired the sine carries the sign of the channel's half.  Channels from rotary_dim on get (1, 0), which nobody uses.
template <int D>
__device__ __forceinline__ void load_angles(const RopeArgs& r, int t, int l, float (&c)[8], float (&s)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) { c[i] = 1.0f; s[i] = 0.0f; }
  const int lh = r.half >> 3;                    // lanes of the first halves of the pairs, then as many of the second
  if (l >= 2 * lh) return;
  const long long at = (long long)t * r.half + (r.interleaved ? 4 * l : 8 * (l >= lh ? l - lh : l));
  const bool minus = !r.interleaved && l < lh;
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const int j = r.interleaved ? 0 : i;
    *reinterpret_cast<float4*>(c + i) = __ldg(reinterpret_cast<const float4*>(r.cos + at + j));
    const float4 v = __ldg(reinterpret_cast<const float4*>(r.sin + at + j));
    s[i] = minus ? -v.x : v.x; s[i + 1] = minus ? -v.y : v.y; s[i + 2] = minus ? -v.z : v.z; s[i + 3] = minus ? -v.w : v.w;
  }
}

// Rotation of a row, lane l of its D / 8 lanes holding channels 8 l .. 8 l + 7.  All lanes of the warp take part.  A channel that is not
// turned is its own partner and stays as it is (x 1 + x (+0) would make an infinity NaN).
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
    const int partner = !turned ? l : l >= lh ? l - lh : l + lh;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float o = __shfl_sync(FULL, x[i], partner, D / 8);
      const float y = __fadd_rn(__fmul_rn(x[i], c[i]), __fmul_rn(o, s[i]));
      x[i] = turned ? y : x[i];
    }
  }
}

// Rows of a token: n_kv_heads keys, as many values where V_ROWS, then the query heads.  A warp takes 256 / D of them at a time and
// `groups` such in a row, the next two's loads in flight: the token's angles stay in registers.
// Long calls are bound by issue and by memory, single tokens by latency.
// KB: the keys' width in calls whose values go by blocks (no value rows here), 0: read from the geometry.
template <int D, int DTYPE, int KB>
__global__ void __launch_bounds__(kThreads, 4)
paged_append_rows_kernel(Geom g, Paged p, AppendArgs a, int per_token, int groups) {
  constexpr int LPR = D / 8, RPW = 32 / LPR;
  constexpr bool V_ROWS = KB == 0;
  const int lane = threadIdx.x & 31, l = lane % LPR;
  const int parts = (per_token + groups - 1) / groups;
  const long long task = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  begin_after_predecessor();
  const int row = (int)(task / parts);
  if (row >= p.n_rows) return;                                           // (whole warps)
  const int g0 = (int)(task - (long long)row * parts) * groups, g1 = min(g0 + groups, per_token);
  // groups of rows: of keys, of values, of queries; a group is of one kind
  const int kg = (g.Hkv + RPW - 1) / RPW, vend = V_ROWS ? 2 * kg : kg;
  const uint16_t* k0 = a.k + (long long)row * a.kv_row + 8 * l;
  const uint16_t* v0 = a.v + (long long)row * a.kv_row + 8 * l;
  const uint16_t* q0 = a.q + (long long)row * a.q_row + 8 * l;
  auto fetch = [&](int group) {
    const bool is_q = group >= vend, is_v = V_ROWS && !is_q && group >= kg;
    const int head = (group - (is_q ? vend : is_v ? kg : 0)) * RPW + lane / LPR;
    const uint16_t* src = (is_q ? q0 : is_v ? v0 : k0) + (long long)head * (is_q ? a.q_head : a.kv_head);
    return head < (is_q ? g.Hq : g.Hkv) ? __ldcs(reinterpret_cast<const uint4*>(src)) : make_uint4(0u, 0u, 0u, 0u);
  };
  // (on their way while the sequence is looked up; rows of padding exist too)
  uint4 next = fetch(g0), after = g0 + 1 < g1 ? fetch(g0 + 1) : make_uint4(0u, 0u, 0u, 0u);
  const int b = sequence_of(p.cu, g.B, row, lane);
  bool bad;
  const int limit = a.rope.half ? min(g.capacity, a.rope.n_positions) : g.capacity;
  const SeqRows s = seq_rows(p, b, limit, p.n_rows, bad);
  if (task == 0) report_bad_input(p, g.B, limit, lane);
  if (row < s.first || row >= s.first + s.rows) return;
  const int t = s.n - s.rows + (row - s.first);
  const int id = pool_page(p, b, t >> 7);
  if (id < 0 && lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
  float ac[8], as[8];
  if (a.rope.half) load_angles<D>(a.rope, t, l, ac, as);
  uint16_t* qo = a.q_out + (long long)row * g.Hq * D + 8 * l;
#pragma unroll 1
  for (int group = g0; group < g1; ++group) {
    const uint4 raw = next;
    next = after;
    if (group + 2 < g1) after = fetch(group + 2);
    float x[8];
    unpack8<DTYPE>(raw, x);
    const bool is_v = V_ROWS && group >= kg && group < vend;
    if (a.rope.half && !is_v) rotate_row<D>(x, a.rope, ac, as, l);
    if (group >= vend) {
      const int head = (group - vend) * RPW + lane / LPR;
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = pack16<DTYPE>(x[2 * i], x[2 * i + 1]);
      if (head < g.Hq) *reinterpret_cast<uint4*>(qo + head * D) = make_uint4(w[0], w[1], w[2], w[3]);
      continue;
    }
    const int head = (group - (is_v ? kg : 0)) * RPW + lane / LPR;
    // ---- quantize
    const int bits = KB > 0 ? KB : is_v ? g.vb : g.kb, gsz = is_v ? g.gv : g.gk, lpg = gsz >> 3;       // lanes per group
    const float qmax = (float)((1 << bits) - 1);
    float mn = fminf(fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), fminf(fminf(x[4], x[5]), fminf(x[6], x[7])));
    float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
#pragma unroll
    for (int off = 1; off < LPR; off <<= 1) {
      const float lo = __shfl_xor_sync(FULL, mn, off), hi = __shfl_xor_sync(FULL, mx, off);
      if (off < lpg) { mn = fminf(mn, lo); mx = fmaxf(mx, hi); }
    }
    const GroupParams gp = group_params(mn, mx, qmax);
    // fields of a byte: channels 16 apart, that is lanes 2 (and 4) apart; every lane of a byte ends up with all its fields
    const int lf = bits == 8 ? 0 : bits == 4 ? 1 : 2;      // log2 of the fields per byte
    const int rh = l & 1, f = (l >> 1) & ((1 << lf) - 1), mw = l >> (1 + lf);
    uint32_t w[2];
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const float y[4] = {x[4 * hh], x[4 * hh + 1], x[4 * hh + 2], x[4 * hh + 3]};
      if constexpr (KB > 0) {
        w[hh] = code_word4_packed<KB>(y, gp.z, gp.inv * (1.0f / (float)(1 << KB))) << (KB * f);
      } else {
        w[hh] = (code_of_fast(y[0], gp, qmax) | (code_of_fast(y[1], gp, qmax) << 8) | (code_of_fast(y[2], gp, qmax) << 16) | (code_of_fast(y[3], gp, qmax) << 24)) << (bits * f);
      }
      const uint32_t o2 = __shfl_xor_sync(FULL, w[hh], 2);
      if (lf >= 1) w[hh] |= o2;
      const uint32_t o4 = __shfl_xor_sync(FULL, w[hh], 4);
      if (lf == 2) w[hh] |= o4;
    }
    if (head >= g.Hkv || id < 0) continue;
    uint8_t* pg = p.pages + ((size_t)id * g.Hkv + head) * g.page_bytes;
    const int tp = t & 127, ng = D / gsz;
    if ((l & (lpg - 1)) == 0) reinterpret_cast<uint32_t*>(pg + (is_v ? g.v_meta_off : g.k_meta_off))[tp * ng + (8 * l) / gsz] = gp.meta;
    if (!is_v) {
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
  // Values go by token rows (their codes then leave byte by byte) in short calls, by blocks of tokens in a launch of their own in long ones, where
  // most blocks are full. Measured with 8 heads of each kind, rows | blocks: D 128, 1 x 2 tokens 3.0 | 5.4 us, 8 x 64 tokens 9.5 | 10.7,
  // 64 x 16 tokens 13.2 | 14.1, 8 x 256 tokens 23.3 | 20.0, 64 x 32 tokens 23.5 | 20.8, 64 x 256 tokens 107 | 91; D 64, 8 x 256 tokens 12.4 | 13.5,
  // 64 x 64 tokens 19.7 | 19.1. They meet between one and two million values.
  const bool blocks = (long long)p.n_rows * g.Hkv * g.D >= 3ll << 19 && p.n_rows >= 16ll * g.B;
  const int rpw = 256 / g.D, per_token = (blocks ? 1 : 2) * ((g.Hkv + rpw - 1) / rpw) + (q ? (g.Hq + rpw - 1) / rpw : 0);
  // enough warps to fill the GPU twice, then longer ones
  const long long warps = (long long)p.n_rows * per_token;
  int groups = (int)(warps / (148 * 64) < 1 ? 1 : warps / (148 * 64) > per_token ? per_token : warps / (148 * 64));
  groups = (per_token + (per_token + groups - 1) / groups - 1) / ((per_token + groups - 1) / groups);      // equal parts
  const long long ctas = ((long long)p.n_rows * ((per_token + groups - 1) / groups) + kThreads / 32 - 1) / (kThreads / 32);
  if (ctas > 0x7FFFFFFFll) return KVQ_ERR_INVALID_ARG;
  auto rows = [&](auto kern) { return launch_dependent(kern, dim3((unsigned)ctas), kThreads, 0, stream, 1, g, p, a, per_token, groups); };
  const bool bf = g.in_dtype == KVQ_BF16;
  cudaError_t e = cudaSuccess;
#define KVQ_ROWS(D_, K_) if (g.D == D_ && kb == K_) e = rows(bf ? paged_append_rows_kernel<D_, KVQ_BF16, K_> : paged_append_rows_kernel<D_, KVQ_FP16, K_>);
  const int kb = blocks ? g.kb : 0;
  KVQ_ROWS(128, 0) KVQ_ROWS(128, 2) KVQ_ROWS(128, 4) KVQ_ROWS(128, 8) KVQ_ROWS(64, 0) KVQ_ROWS(64, 2) KVQ_ROWS(64, 4) KVQ_ROWS(64, 8)
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
