// Paged attention in its plainest form: a warp per (row, query head), a lane per token, then a lane per channel.  Online softmax over
// blocks of 32 tokens.
#include "kvq_paged.cuh"

namespace kvq {

namespace {

constexpr int kThreads = 128;

__device__ __forceinline__ float value_of(const uint8_t* pg, const Geom& g, bool is_v, int tp, int d) {
  const int bits = is_v ? g.vb : g.kb, gs = is_v ? g.gv : g.gk;
  const uint32_t m = reinterpret_cast<const uint32_t*>(pg + (is_v ? g.v_meta_off : g.k_meta_off))[tp * (g.D / gs) + d / gs];
  const float2 sz = __half22float2(*reinterpret_cast<const __half2*>(&m));
  return fmaf((float)load_code_any(pg + (is_v ? g.v_codes_off : 0), is_v, tp, d, g.D, bits), sz.x, sz.y);
}

__global__ void __launch_bounds__(kThreads)
paged_plain_kernel(Geom g, Paged p, const uint16_t* __restrict__ q, float c1, void* __restrict__ out, int out_dtype) {
  __shared__ float sq[kThreads / 32][128];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long task = (long long)blockIdx.x * (kThreads / 32) + warp;
  begin_after_predecessor();
  const int row = (int)(task / g.Hq), hq = (int)(task % g.Hq), h = hq / g.G;
  if (row >= p.n_rows) return;
  const int b = sequence_of(p.cu, g.B, row, lane);
  bool bad;
  const SeqRows s = seq_rows(p, b, g.capacity, p.max_rows, bad);
  if (bad && lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
  if (row < s.first || row >= s.first + s.rows) return;
  const int pos = s.n - s.rows + (row - s.first);
  const size_t at = ((size_t)row * g.Hq + hq) * g.D;
  for (int d = lane; d < g.D; d += 32) sq[warp][d] = bits16_to_f32(q[at + d], g.in_dtype) * c1;
  __syncwarp();
  const SeenPages seen = seen_pages(pos, pos, p.window, p.sinks);
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < seen.count; ++i) {
    const int page = seen.logical(i);
    int id = pool_page(p, b, page);
    if (id < 0) {
      if (lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
      id = 0;
    }
    const uint8_t* pg = p.pages + ((size_t)id * g.Hkv + h) * g.page_bytes;
    for (int blk = 0; blk < 4; ++blk) {
      const int tp = 32 * blk + lane, t = 128 * page + tp;
      const bool sees = t <= pos && (p.window == 0 || t > pos - p.window || t < p.sinks);
      float x = -INFINITY;
      if (sees) {
        x = 0.f;
        for (int d = 0; d < g.D; ++d) x = fmaf(sq[warp][d], value_of(pg, g, false, tp, d), x);
      }
      float top = x;
      for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
      if (top == -INFINITY) continue;
      const float nm = fmaxf(m, top), keep = exp2f(m - nm), w = exp2f(x - nm);
      m = nm;
      float sum = w;
      for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      l = l * keep + sum;
      for (int e = 0; e < 4; ++e) o[e] *= keep;
      for (int j = 0; j < 32; ++j) {
        const float wj = __shfl_sync(0xffffffffu, w, j);
        if (wj == 0.f) continue;
        for (int e = 0; e < g.D / 32; ++e) o[e] = fmaf(wj, value_of(pg, g, true, 32 * blk + j, lane + 32 * e), o[e]);
      }
    }
  }
  for (int e = 0; e < g.D / 32; ++e) {
    const float r = l > 0.f ? o[e] / l : 0.f;
    const size_t oi = at + lane + 32 * e;
    if (out_dtype == KVQ_FP32) static_cast<float*>(out)[oi] = r;
    else static_cast<uint16_t*>(out)[oi] = f32_to_bits16(r, out_dtype);
  }
}

}  // namespace

int launch_paged_plain(const Geom& g, const Paged& p, const void* q, void* out, int out_dtype, float c1, cudaStream_t stream) {
  const long long ctas = ((long long)p.n_rows * g.Hq + kThreads / 32 - 1) / (kThreads / 32);
  if (ctas > 0x7FFFFFFFll) return KVQ_ERR_INVALID_ARG;
  const cudaError_t e = launch_dependent(paged_plain_kernel, dim3((unsigned)ctas), kThreads, 0, stream, 1, g, p,
                                         static_cast<const uint16_t*>(q), c1, out, out_dtype);
  return e == cudaSuccess ? KVQ_OK : KVQ_ERR_CUDA_LAUNCH;
}

}  // namespace kvq
