// kvq_paged_dequantize: x^ = fmaf(code, scale, zero) rounded to the 16-bit input type (App. B.1: A^ = scale * Q, here with the group
// minimum as offset), for the rows of a ragged call.
//
// A warp takes one block of 32 tokens of one head and one side.  Keys go from global to global memory: a lane owns a quarter of a
// token's row, whose bytes are four consecutive channels of every 16-channel slice, and four lanes write 32 contiguous bytes.  Values
// are transposed by stmatrix into a padded tile of the warp's own and leave as whole rows.  Code bytes become floats by a byte
// permute and an exact subtraction.  Bound by the 16-bit stores, which are 4 to 8 times what is read: 4 x up to 8,001 tokens of the 8B shape K4V2 27 us
// (element by element 254), 32,768 tokens 36.6 us (161 MB, 0.67 of the copy rate).
#include "kvq_dequantize.cuh"
#include "kvq_paged.cuh"

namespace kvq {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;

__device__ __forceinline__ float2 meta_sz(uint32_t m) { return __half22float2(*reinterpret_cast<const __half2*>(&m)); }

// Keys of tokens lo .. hi - 1 of the block at token tp of its page.  out: the block's first token; stride: of tokens, in elements.
template <int B, int D, int DTYPE>
__device__ __forceinline__ void block_keys(const Geom& g, const uint8_t* __restrict__ pg, int tp, uint16_t* __restrict__ out, long long stride,
                                           int lo, int hi, int lane) {
  constexpr int FPB = 8 / B, ROW = D * B / 8, WPC = D * B / 128, QW = WPC < 4 ? WPC : 4;
  constexpr uint32_t MASK = ((1u << B) - 1u) * 0x01010101u;
  const int chunk = lane & 3, lgk = 31 - __clz(g.gk), ngk = D >> lgk;
  const uint32_t* meta = reinterpret_cast<const uint32_t*>(pg + g.k_meta_off);
#pragma unroll
  for (int pass = 0; pass < 4; ++pass) {
    const int u = 8 * pass + (lane >> 2);
    if (u < lo || u >= hi) continue;
    uint32_t w[WPC];
    const uint8_t* row = pg + (tp + u) * ROW + chunk * (4 * QW);
    if constexpr (WPC == 1) {
      w[0] = __ldcs(reinterpret_cast<const uint32_t*>(row));
    } else if constexpr (WPC == 2) {
      const uint2 v = __ldcs(reinterpret_cast<const uint2*>(row));
      w[0] = v.x; w[1] = v.y;
    } else {
#pragma unroll
      for (int qd = 0; qd < WPC / 4; ++qd) {
        const uint4 v = __ldcs(reinterpret_cast<const uint4*>(row + qd * 64));
        w[4 * qd] = v.x; w[4 * qd + 1] = v.y; w[4 * qd + 2] = v.z; w[4 * qd + 3] = v.w;
      }
    }
    uint16_t* orow = out + (long long)u * stride + 4 * chunk;
    float2 sz = make_float2(0.f, 0.f);
#pragma unroll
    for (int r = 0; r < D / 16; ++r) {           // slice r: channels 16 r + 4 chunk + {0..3}
      if (r == 0 || ((16 * r) & (g.gk - 1)) == 0) sz = meta_sz(__ldg(meta + (tp + u) * ngk + ((16 * r) >> lgk)));       // a new group (the same for all lanes)
      const uint32_t bytes = (w[r / FPB] >> (B * (r % FPB))) & MASK;
      const f32x2 s = pack2(sz.x, sz.x), z = pack2(sz.y, sz.y);
      __stcs(reinterpret_cast<uint2*>(orow + 16 * r), make_uint2(pack16<DTYPE>(fma2(code_pair(bytes, 0, 1), s, z)), pack16<DTYPE>(fma2(code_pair(bytes, 2, 3), s, z))));
    }
  }
}

// Values: lane (channel of eight, tq) has the codes of eight tokens of a channel in every 16 bytes; the pairs of tokens (2 tq, 2 tq + 1) are what
// stmatrix transposes.
template <int B, int D, int DTYPE>
__device__ __forceinline__ void block_values(const Geom& g, const uint8_t* __restrict__ pg, int tp, uint16_t* __restrict__ out, long long stride,
                                             int lo, int hi, uint16_t* tile, int lane) {
  constexpr int FPB = 8 / B, TS = D + 8, NMW = D * B / 128;
  constexpr uint32_t MASK = ((1u << B) - 1u) * 0x01010101u;
  const int tq = lane & 3, lgv = 31 - __clz(g.gv), ngv = D >> lgv;
  const uint4* codes = reinterpret_cast<const uint4*>(pg + g.v_codes_off + (tp >> 5) * (4 * D * B)) + lane;
  const uint32_t* meta = reinterpret_cast<const uint32_t*>(pg + g.v_meta_off) + (tp + 2 * tq) * ngv;
  // the 16-byte row of the tile that this lane's address names: matrix (half, rh) = lane / 8, token lane % 8 of the half
  const uint32_t row0 = (uint32_t)__cvta_generic_to_shared(tile + (8 * (lane >> 4) + (lane & 7)) * TS + 8 * ((lane >> 3) & 1));
  f32x2 sc[2][2], ze[2][2];                      // [kh][half]: tokens 16 kh + 8 half + 2 tq + {0, 1}
#pragma unroll
  for (int mw = 0; mw < NMW; ++mw) {
    const uint4 v = __ldcs(codes + 32 * mw);
    const uint32_t ww[4] = {v.x, v.y, v.z, v.w};           // sub = 2 rh + kh
#pragma unroll
    for (int f = 0; f < FPB; ++f) {
      const int m16 = mw * FPB + f;
      if (m16 == 0 || ((16 * m16) & (g.gv - 1)) == 0) {
        const uint32_t* mt = meta + ((16 * m16) >> lgv);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 a = meta_sz(__ldg(mt + 8 * i * ngv)), b = meta_sz(__ldg(mt + (8 * i + 1) * ngv));
          sc[i >> 1][i & 1] = pack2(a.x, b.x);
          ze[i >> 1][i & 1] = pack2(a.y, b.y);
        }
      }
#pragma unroll
      for (int kh = 0; kh < 2; ++kh) {
        uint32_t r[2][2];                        // [half][rh]
#pragma unroll
        for (int rh = 0; rh < 2; ++rh) {
          const uint32_t bytes = (ww[2 * rh + kh] >> (B * f)) & MASK;       // tokens 2 tq, 2 tq + 8, 2 tq + 1, 2 tq + 9
          r[0][rh] = pack16<DTYPE>(fma2(code_pair(bytes, 0, 2), sc[kh][0], ze[kh][0]));
          r[1][rh] = pack16<DTYPE>(fma2(code_pair(bytes, 1, 3), sc[kh][1], ze[kh][1]));
        }
        asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                     ::"r"(row0 + 2 * (16 * kh * TS + 16 * m16)), "r"(r[0][0]), "r"(r[0][1]), "r"(r[1][0]), "r"(r[1][1]) : "memory");
      }
    }
  }
  __syncwarp();
  constexpr int VPR = D / 8;
  for (int idx = lane; idx < (hi - lo) * VPR; idx += 32) {
    const int u = lo + idx / VPR, v = idx % VPR;
    __stcs(reinterpret_cast<uint4*>(out + (long long)u * stride) + v, reinterpret_cast<const uint4*>(tile + u * TS)[v]);
  }
}

// Tasks: (block, head, side), sides neighbours so that both read a page while it is near.  first_side, sides: 0 keys, 1 values.
template <int D, int DTYPE>
__global__ void __launch_bounds__(kThreads)
paged_dequant_kernel(Geom g, Paged p, uint16_t* k_out, uint16_t* v_out, int first_side, int sides) {
  __shared__ __align__(16) uint16_t tiles[kWarps][32 * (D + 8)];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long task = (long long)blockIdx.x * kWarps + warp;
  begin_after_predecessor();
  if (task == 0) report_bad_input(p, g.B, g.capacity, lane);
  const int side = first_side + (int)(task % sides);
  task /= sides;
  const int h = (int)(task % g.Hkv);
  const BlockTask t = block_task(p, g.B, (int)(task / g.Hkv), 32, g.capacity, p.n_rows, lane);
  if (t.lo >= t.hi) return;
  const int id = pool_page(p, t.b, t.t0 >> 7);
  if (id < 0) {
    if (lane == 0) atomicOr(p.status, KVQ_STATUS_BAD_INPUT);
    return;
  }
  const uint8_t* pg = p.pages + ((size_t)id * g.Hkv + h) * g.page_bytes;
  const int tp = t.t0 & 127;
  const long long stride = (long long)g.Hkv * D;
  uint16_t* out = (side == 0 ? k_out : v_out) + t.row0 * stride + (long long)h * D;
  if (side == 0) {
    if (g.kb == 2) block_keys<2, D, DTYPE>(g, pg, tp, out, stride, t.lo, t.hi, lane);
    else if (g.kb == 4) block_keys<4, D, DTYPE>(g, pg, tp, out, stride, t.lo, t.hi, lane);
    else block_keys<8, D, DTYPE>(g, pg, tp, out, stride, t.lo, t.hi, lane);
  } else {
    if (g.vb == 2) block_values<2, D, DTYPE>(g, pg, tp, out, stride, t.lo, t.hi, tiles[warp], lane);
    else if (g.vb == 4) block_values<4, D, DTYPE>(g, pg, tp, out, stride, t.lo, t.hi, tiles[warp], lane);
    else block_values<8, D, DTYPE>(g, pg, tp, out, stride, t.lo, t.hi, tiles[warp], lane);
  }
}

}  // namespace

int launch_paged_dequantize(const Geom& g, const Paged& p, void* k_out, void* v_out, cudaStream_t stream) {
  const int sides = (k_out ? 1 : 0) + (v_out ? 1 : 0);
  const long long ctas = (block_tasks(p.n_rows, g.B, 32) * g.Hkv * sides + kWarps - 1) / kWarps;
  if (ctas > 0x7FFFFFFFll) return KVQ_ERR_INVALID_ARG;
  auto launch = [&](auto kern) {
    return launch_dependent(kern, dim3((unsigned)ctas), kThreads, 0, stream, 1, g, p, static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out),
                            k_out ? 0 : 1, sides);
  };
  const bool bf = g.in_dtype == KVQ_BF16;
  const cudaError_t e = g.D == 128 ? launch(bf ? paged_dequant_kernel<128, KVQ_BF16> : paged_dequant_kernel<128, KVQ_FP16>)
                                   : launch(bf ? paged_dequant_kernel<64, KVQ_BF16> : paged_dequant_kernel<64, KVQ_FP16>);
  return e == cudaSuccess ? KVQ_OK : KVQ_ERR_CUDA_LAUNCH;
}

}  // namespace kvq
