// Attention of many query rows: prompts, and questions behind a long context.
//
//   S = Q K^T,  P = 2^(scale log2(e) S - m),  O += P V,  out = O / sum(P)
//
// Bound by the tensor cores: 4 D FLOP for every visible (query row, key) pair. A
// block owns 256 flattened query rows of one KV head (two tiles of 128) and walks
// its keys 128 at a time; the two tiles take turns on the tensor core, so that
// one's softmax runs under the other's products.
//
//   warps 0-3, 4-7  softmax of tile 0 and 1: a thread a row.  Scores come from
//                   tensor memory, probabilities go back there as bf16 over them,
//                   as the next product's first operand.  The running maximum
//                   moves only when a score passes it by 2^8; the outputs in tensor
//                   memory are rescaled then, by the same thread.
//   warps 8-11      loaders, into the 128-byte-swizzled layout.  bf16: one warp
//                   brings K and V by tensor copies, a lane a piece of a page (a
//                   step's last rows, where the sequence ends, are cleared: what
//                   lies there must not meet a probability of zero), the others Q;
//                   pages that hold no multiple of eight rows come by cp.async.
//                   4-bit: all four expand the codes to bf16 (exactly).
//   warps 12, 13    issue the products of tile 0 and 1: S = Q K^T from shared
//                   memory, O += P V with P in tensor memory and V as it lies
//                   (its channels contiguous).  A warp a tile: what one spends
//                   on its barriers lies under the other's products.  They take
//                   turns: left to themselves both tiles fall into step, and the
//                   softmaxes run side by side, then the products.
// Tensor memory: S0, S1 (P over them) and O0, O1, 128 columns each.  The
// products of one tile follow each other in issue order, so a tile's new scores
// also say that its last product with V is done.
//
// Every wait is bounded; one that runs out sets HF_CHECK_TIMEOUT and ends the
// block.
#include <algorithm>
#include <string>

#include <cuda.h>

#include "hf_attend.cuh"

namespace hf {
namespace {

constexpr int kTile = 128;       // query rows of a tile, keys of a step
constexpr int kThreads = 512;    // 13 warps work; registers are shared out by warpgroup
constexpr float kStretch = 8.f;  // log2 of what a score may pass the running maximum by

__device__ __forceinline__ void cp_async_16_or_zero(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
template <int N>
__device__ __forceinline__ void regs_more() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_less() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Two fp32 operations an instruction.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float* a, float* b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void mma_bf16_tmem_a(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                                uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Descriptor of an operand whose rows (K) are 128-byte pieces of the other
// dimension, 128-byte swizzle: 1,024 bytes from eight rows of K to the next
// eight, `pitch` bytes from 64 values of the other dimension to the next.
__device__ __forceinline__ uint64_t sw128_mnmajor_desc(uint32_t saddr, uint32_t pitch) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(pitch >> 4) << 16) |
         (static_cast<uint64_t>(1024 >> 4) << 32) | (static_cast<uint64_t>(1) << 46) |
         (static_cast<uint64_t>(2) << 61);
}

// mbar_wait without a call: the registers of a kernel that shares them out anew
// (setmaxnreg) cannot be allocated around one.
__device__ __forceinline__ bool wait_here(uint32_t bar, uint32_t parity) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_timer_ns();
  for (uint32_t i = 1;; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((i & 63u) == 0 && global_timer_ns() - t0 > kWaitLimitNs) return false;
  }
}

#define HF_R4(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3])
#define HF_W4(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3])
// 32 columns of this thread's lane.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : HF_R4(r, 0), HF_R4(r, 4), HF_R4(r, 8), HF_R4(r, 12), HF_R4(r, 16), HF_R4(r, 20), HF_R4(r, 24), HF_R4(r, 28)
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
      "%15};" ::HF_W4(r, 0),
      HF_W4(r, 4), HF_W4(r, 8), HF_W4(r, 12), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Waits for this warp's loads; the registers pass through, so that no use moves above.
#define HF_P4(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3])
__device__ __forceinline__ void tmem_ld_wait32(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : HF_P4(r, 0), HF_P4(r, 4), HF_P4(r, 8), HF_P4(r, 12), HF_P4(r, 16), HF_P4(r, 20), HF_P4(r, 24),
                 HF_P4(r, 28)::"memory");
}

// Eight channels of a 4-bit row lie in an operand as their codes do in a word:
// 0 4 1 5 2 6 3 7; channel k is at place code_place(k).
__host__ __device__ constexpr int code_place(int k) { return k < 4 ? 2 * k : 2 * k - 7; }

// This lane's codes and scales of a row (lane m of the row's four).
template <int D>
struct Q4Words {
  uint32_t w[D / 32], s[D / 64];
};
template <int D>
__device__ __forceinline__ void load_q4(Q4Words<D>& q, const char* codes, const char* scales, int row, int m) {
  constexpr int NG = D / 32;
  if (row < 0) {
#pragma unroll
    for (int i = 0; i < NG; ++i) q.w[i] = 0u;
#pragma unroll
    for (int i = 0; i < NG / 2; ++i) q.s[i] = 0u;
    return;
  }
  const int64_t r = row;
  if constexpr (D == 128) {
    const uint4 u = *reinterpret_cast<const uint4*>(codes + r * 64 + m * 16);
    q.w[0] = u.x, q.w[1] = u.y, q.w[2] = u.z, q.w[3] = u.w;
    const uint2 v = *reinterpret_cast<const uint2*>(scales + r * 8);
    q.s[0] = v.x, q.s[1] = v.y;
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(codes + r * 32 + m * 8);
    q.w[0] = u.x, q.w[1] = u.y;
    q.s[0] = *reinterpret_cast<const uint32_t*>(scales + r * 4);
  }
}
// Their values as bf16, exactly, into row `key` of the operand at `base`: 128 + c
// by masking, - 136, times the scale, two codes at a time.
template <int D>
__device__ __forceinline__ void store_q4_values(const Q4Words<D>& q, uint32_t base, int part, int key, int m) {
  constexpr int NG = D / 32;
  const __nv_bfloat162 off = __floats2bfloat162_rn(136.f, 136.f);
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const uint32_t w = __byte_perm(q.w[g / 2], q.w[NG / 2 + g / 2], g & 1 ? 0x7632 : 0x5410);
    const uint32_t s2 = __byte_perm(q.s[g / 2], q.s[g / 2], g & 1 ? 0x3232 : 0x1010);
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t c = ((w >> (4 * i)) & 0x000f000fu) | 0x43004300u;
      const __nv_bfloat162 x =
          __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&c), off), *reinterpret_cast<const __nv_bfloat162*>(&s2));
      v[i] = *reinterpret_cast<const uint32_t*>(&x);
    }
    const int c = 4 * g + m;
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + (c / 8) * part + key * 128 +
                                                                  (((c % 8) ^ (key & 7)) << 4)),
                 "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3])
                 : "memory");
  }
}

template <int D>
struct Smem {
  static constexpr int kPart = kTile * 128;           // 128 rows of 64 channels
  static constexpr int kOperand = kPart * (D / 64);   // a tile of Q, K or V
  static constexpr int kStages = D == 128 ? 5 : 6;
  static constexpr int kQ = 0;
  static constexpr int kKV = 2 * kOperand;
  static constexpr int kBars = kKV + kStages * kOperand;
  static constexpr int kBytes = kBars + 256;
};

// How a block gets its keys and values.
enum Source { kByTensorCopies, kByCpAsync, kFromCodes };

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* map, int32_t x, int32_t y, int32_t z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}

template <int SRC, int D>
__global__ void __launch_bounds__(kThreads, 1)
    attend_tiles_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                        const CacheArgs C, const AttendArgs A, int ns, int box) {
  using M = Smem<D>;
  constexpr int S = M::kStages;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // ---- the block's rows and keys
  const int h = blockIdx.x % C.H, sp = blockIdx.y;
  const TilePlace place = find_tile(C, A, 2 * kTile, blockIdx.x / C.H);
  if (place.seq >= C.n_seq) return;
  const SeqSpan span = seq_span(C, A, place.seq);
  const int r0 = (place.tiles - 1 - place.at) * 2 * kTile;  // the longest first
  const int n_rows = static_cast<int>(min(static_cast<int64_t>(2 * kTile), static_cast<int64_t>(span.n) * A.G - r0));
  // keys of this part: tiles [t0, t1) of 128; of query tile i: up to its last row's
  const int kv_end = seen(span, A.causal, (r0 + n_rows - 1) / A.G);
  const int all = (kv_end + kTile - 1) / kTile;
  const int t0 = static_cast<int>(static_cast<int64_t>(all) * sp / ns);
  const int t1 = static_cast<int>(static_cast<int64_t>(all) * (sp + 1) / ns);
  int nt[2];
  {
    const int last0 = min(n_rows, kTile) - 1;
    const int end0 = seen(span, A.causal, (r0 + last0) / A.G);
    nt[0] = max(min((end0 + kTile - 1) / kTile, t1) - t0, 0);
    nt[1] = n_rows > kTile ? t1 - t0 : 0;
  }
  const int n_max = max(nt[0], nt[1]);

  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + M::kBars);
  const uint32_t full = smem_addr(bars), empty = full + 8 * S, qfull = empty + 8 * S, sfull = qfull + 8,
                 pfull = sfull + 16, ofull = pfull + 32, turn = ofull + 16, drain = turn + 16, aux = drain + 8;
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(smem + M::kBars + 8 * (2 * S + 13));
  if (smem_addr(smem) & 1023u) {
    if (threadIdx.x == 0) set_status(C, HF_CHECK_INTERNAL);
    return;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(full + 8 * s, SRC == kByTensorCopies ? 1 : 4);
      mbar_init(empty + 8 * s, 2);
    }
    mbar_init(qfull, SRC == kByTensorCopies ? 3 : 4);
    mbar_init(aux, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(sfull + 8 * i, 1);
      mbar_init(pfull + 8 * i, 4);       // first half of the keys
      mbar_init(pfull + 16 + 8 * i, 4);  // second half
      mbar_init(ofull + 8 * i, 1);
      mbar_init(turn + 8 * i, 1);
    }
    mbar_init(drain, 2);
    fence_barrier_init();
  }
  if (SRC == kByTensorCopies && warp == 8 && lane == 0) {
    tma_prefetch_map(&map_k);
    tma_prefetch_map(&map_v);
  }
  if (warp == 12) {
    tmem_alloc(smem_addr(s_tmem), 512);
    tmem_relinquish();
  }
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *s_tmem;
  auto timed_out = [&]() { set_status(C, HF_CHECK_TIMEOUT); };

  // Registers, by warpgroup: 2 x 192 + 72 + 56 = 4 x 128.
  if (warp < 8) {
    // ------------------------------------------------------------ softmax
    regs_more<192>();
    const int i = warp >> 2;
    const int row = (warp & 3) * 32 + lane;
    const int rr = r0 + i * kTile + row;
    const bool live = i * kTile + row < n_rows;
    const int lim = live ? seen(span, A.causal, rr / A.G) : 0;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + i * 128 + lanes, to = tmem + 256 + i * 128 + lanes;
    const uint64_t scale2 = pack2(A.scale_log2, A.scale_log2);
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    const int n = nt[i];
    for (int j = 0; j < n; ++j) {
      if (!wait_here(sfull + 8 * i, j & 1)) {
        timed_out();
        ok = false;
        break;
      }
      tc_fence_after_sync();
      uint32_t s[128];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32(ts + 32 * c, s + 32 * c);
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld_wait32(s + 32 * c);
      const int vis = lim - (t0 + j) * kTile;  // columns that this row sees
      if (__any_sync(0xffffffffu, vis < kTile)) {
#pragma unroll
        for (int c = 0; c < 128; ++c)
          if (c >= vis) s[c] = 0xff800000u;
      }
      float top4[4];  // four chains: one would be 128 latencies long
#pragma unroll
      for (int c = 0; c < 4; ++c) top4[c] = fmaxf(__uint_as_float(s[c]), __uint_as_float(s[c + 4]));
#pragma unroll
      for (int c = 8; c < 128; c += 8)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          top4[e] = fmaxf(top4[e], fmaxf(__uint_as_float(s[c + e]), __uint_as_float(s[c + e + 4])));
      const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])) * A.scale_log2;
      if (__any_sync(0xffffffffu, top > m + kStretch)) {
        const float next = top > m + kStretch ? top : m;
        const float fix = next == m ? 1.f : exp2_approx(m - next);
        m = next;
        l *= fix;
        if (j > 0) {
#pragma unroll
          for (int c = 0; c < D; c += 16) {
            uint32_t o[16];
            tmem_load_16(to + c, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * fix);
            tmem_st16(to + c, o);
          }
        }
      }
      const float base = m == -INFINITY ? 0.f : -m;
      uint64_t sum[2] = {0, 0};
#pragma unroll
      for (int c = 0; c < 128; c += 32) {
        uint32_t p[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          float a, b;
          unpack2(fma2(pack2(__uint_as_float(s[c + e]), __uint_as_float(s[c + e + 1])), scale2, pack2(base, base)), &a, &b);
          a = exp2_approx(a);
          b = exp2_approx(b);
          sum[e / 2 % 2] = add2(sum[e / 2 % 2], pack2(a, b));
          p[e / 2] = pack_bf16(a, b);
        }
        tmem_st16(ts + c / 2, p);
        if (c & 32) {  // 64 keys' probabilities
          tmem_st_wait();
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(pfull + (c > 64 ? 16 : 0) + 8 * i);
        }
      }
      {
        float a, b;
        unpack2(add2(sum[0], sum[1]), &a, &b);
        l += a + b;
      }
    }
    // ---- outputs
    const int64_t tok = span.first + rr / A.G;
    const int hq = h * A.G + rr % A.G;
    if (ok && n > 0 && !wait_here(ofull + 8 * i, 0)) {
      timed_out();
      ok = false;
    }
    if (ok) {
      tc_fence_after_sync();
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int64_t slot = (static_cast<int64_t>(sp) * A.n_tok + tok) * A.H_q + hq;
#pragma unroll
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32];
        if (n > 0) {
          tmem_ld32(to + c, o);
          tmem_ld_wait32(o);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0u;
        }
        if constexpr (SRC == kFromCodes) {
          uint32_t t[8];
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] = o[e + code_place(k)];
#pragma unroll
            for (int k = 0; k < 8; ++k) o[e + k] = t[k];
          }
        }
        if (live) {
          if (ns > 1) {
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<uint4*>(A.part_o + slot * D + c + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          } else {
            __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(A.out) + tok * A.o_row + hq * A.o_head + c;
#pragma unroll
            for (int e = 0; e < 32; e += 8) {
              uint32_t w[4];
#pragma unroll
              for (int k = 0; k < 4; ++k)
                w[k] = pack_bf16(__uint_as_float(o[e + 2 * k]) * inv, __uint_as_float(o[e + 2 * k + 1]) * inv);
              *reinterpret_cast<uint4*>(dst + e) = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
        }
      }
      if (live) {
        if (ns > 1)
          A.part_ml[slot] = make_float2(m, l);
        else if (A.lse)
          A.lse[tok * A.H_q + hq] = (m + log2f(l)) * 0.693147180559945309f;
      }
    }
  } else if (warp < 12) {
    // ------------------------------------------------------------ loaders
    regs_less<72>();
    const int w = warp - 8;
    constexpr int kChunks = D / 8;  // 16-byte pieces of a row
    constexpr int kQWarps = SRC == kByTensorCopies ? 3 : 4;
    if (SRC != kByTensorCopies || w > 0) {
#pragma unroll 1
      for (int k = w + kQWarps - 4; k < 8; k += kQWarps) {  // rows 32 k ..
        int64_t at = -1;
        const int row = 32 * k + lane;
        if (row < n_rows) {
          const int rr = r0 + row;
          at = static_cast<int64_t>(span.first + rr / A.G) * A.q_row + (h * A.G + rr % A.G) * A.q_head;
        }
#pragma unroll 4
        for (int x = 0; x < kChunks; ++x) {
          const int idx = x * 32 + lane, c = idx % kChunks, src = idx / kChunks;
          const int64_t a = __shfl_sync(0xffffffffu, at, src);
          const int qr = 32 * (k & 3) + src;  // row in its tile
          const uint32_t dst = smem_addr(smem) + M::kQ + (k >> 2) * M::kOperand + (c / 8) * M::kPart + qr * 128 +
                               (((c % 8) ^ (qr & 7)) << 4);
          if constexpr (SRC == kFromCodes) {  // channels in the order of the expanded codes
            uint4 u = make_uint4(0, 0, 0, 0);
            if (a >= 0) u = *reinterpret_cast<const uint4*>(A.q + a * 2 + c * 16);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(__byte_perm(u.x, u.z, 0x5410)),
                         "r"(__byte_perm(u.x, u.z, 0x7632)), "r"(__byte_perm(u.y, u.w, 0x5410)),
                         "r"(__byte_perm(u.y, u.w, 0x7632))
                         : "memory");
          } else {
            cp_async_16_or_zero(dst, A.q + (a < 0 ? 0 : a * 2 + c * 16), a >= 0);
          }
        }
      }
      cp_async_commit();
    }
    const int n = 2 * n_max;
    bool ok = true;
    int stage = 0;
    uint32_t phase = 1;
    auto row_of = [&](int j) {  // of key `lane` of this warp's 32 in step j
      const int key = (t0 + j) * kTile + 32 * w + lane;
      return j < n_max && key < kv_end ? cache_row(C, place.seq, key) : -1;
    };
    if constexpr (SRC == kByTensorCopies) {
      if (w > 0) {
        cp_async_wait<0>();
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(qfull);
      } else {
        // Lane b + nb * c: channels 64 c .. of the rows b * box .. of a step.
        const int nb = kTile / box, piece = lane % nb, part = lane / nb;
        const bool active = part < D / 64;
        auto piece_row = [&](int j) {
          const int key = (t0 + j) * kTile + piece * box;
          return active && j < n_max && key < kv_end ? cache_row(C, place.seq, key) : -1;
        };
        uint32_t aux_phase = 0;
        int ahead = piece_row(0), issued = 0;
        for (int j = 0; j < n_max && ok; ++j) {
          const int row = ahead;
          ahead = piece_row(j + 1);
          const int key0 = (t0 + j) * kTile;
          const unsigned there = __ballot_sync(0xffffffffu, row >= 0);
          const bool whole = key0 + kTile <= kv_end && __popc(there) == nb * (D / 64);
#pragma unroll 1
          for (int v = 0; v < 2; ++v) {
            if (!wait_here(empty + 8 * stage, phase)) {
              timed_out();
              ok = false;
              break;
            }
            const uint32_t dst = smem_addr(smem) + M::kKV + stage * M::kOperand;
            const uint32_t bar = whole ? full + 8 * stage : aux;
            if (lane == 0 && there) mbar_arrive_expect_tx(bar, __popc(there) * box * 128);
            __syncwarp();
            ++issued;
            if (row >= 0)
              tma_load_3d(dst + part * M::kPart + piece * box * 128, v ? &map_v : &map_k, 64 * part, row, h, bar);
            if (!whole) {
              if (there) {
                if (!wait_here(aux, aux_phase)) {
                  timed_out();
                  ok = false;
                  break;
                }
                aux_phase ^= 1;
              }
              // rows past the end, and of pages that are not there: zeros
              for (int r = lane / kChunks; r < kTile; r += 32 / kChunks) {
                if (key0 + r >= kv_end || !(there >> (r / box) & 1)) {
                  const int c = lane % kChunks;
                  asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst + (c / 8) * M::kPart + r * 128 +
                                                                                (c % 8) * 16),
                               "r"(0)
                               : "memory");
                }
              }
              fence_proxy_async_smem();
              __syncwarp();
              if (lane == 0) mbar_arrive(full + 8 * stage);
            }
            if (++stage == S) {
              stage = 0;
              phase ^= 1;
            }
          }
        }
        // a block that gives up waits for its copies in flight
        for (int x = max(issued - S, 0); !ok && x < issued; ++x)
          if (!wait_here(full + 8 * (x % S), (x / S) & 1)) break;
      }
    } else if constexpr (SRC == kFromCodes) {
      // the words of the next operand are under way while this one is expanded
      const char* codes[2] = {C.k + static_cast<int64_t>(h) * C.rows * (D / 2), C.v + static_cast<int64_t>(h) * C.rows * (D / 2)};
      const char* scales[2] = {C.ks + static_cast<int64_t>(h) * C.rows * (D / 16),
                               C.vs + static_cast<int64_t>(h) * C.rows * (D / 16)};
      Q4Words<D> q[4];
      const int m = lane & 3;
      int row = row_of(0), next = row_of(1);
#pragma unroll
      for (int p = 0; p < 4; ++p)
        load_q4<D>(q[p], codes[0], scales[0], __shfl_sync(0xffffffffu, row, 8 * p + (lane >> 2)), m);
      for (int x = 0; x < n; ++x) {
        if (!wait_here(empty + 8 * stage, phase)) {
          timed_out();
          break;
        }
        const uint32_t base = smem_addr(smem) + M::kKV + stage * M::kOperand;
        if (x & 1) {
          row = next;
          next = row_of((x >> 1) + 2);
        }
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const int kr = 8 * p + (lane >> 2);
          store_q4_values<D>(q[p], base, M::kPart, 32 * w + kr, m);
          load_q4<D>(q[p], x & 1 ? codes[0] : codes[1], x & 1 ? scales[0] : scales[1],
                     __shfl_sync(0xffffffffu, row, kr), m);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (x == 0) mbar_arrive(qfull);
          mbar_arrive(full + 8 * stage);
        }
        if (++stage == S) {
          stage = 0;
          phase ^= 1;
        }
      }
    } else {
    const char* kb = C.k + h * C.head_stride * 2;
    const char* vb = C.v + h * C.head_stride * 2;
    constexpr int kLag = 2;
    int done = 0;
    int row = -1;
    for (int x = 0; x < n + kLag && ok; ++x) {
      if (x < n) {
        if (!wait_here(empty + 8 * stage, phase)) {
          timed_out();
          ok = false;
          break;
        }
        if ((x & 1) == 0) row = row_of(x >> 1);
        const char* src = x & 1 ? vb : kb;
        const uint32_t base = smem_addr(smem) + M::kKV + stage * M::kOperand;
#pragma unroll 4
        for (int y = 0; y < kChunks; ++y) {
          const int idx = y * 32 + lane, c = idx % kChunks, kr = idx / kChunks;
          const int r = __shfl_sync(0xffffffffu, row, kr);
          const int key = 32 * w + kr;
          cp_async_16_or_zero(base + (c / 8) * M::kPart + key * 128 + (((c % 8) ^ (key & 7)) << 4),
                              src + max(r, 0) * (C.row_stride * 2) + c * 16, r >= 0);
        }
        if (++stage == S) {
          stage = 0;
          phase ^= 1;
        }
      }
      cp_async_commit();
      // Operands land kLag steps after they were issued; Q and the first one,
      // which everything waits for, at once.
      if (x == 1)
        cp_async_wait<1>();
      else
        cp_async_wait<kLag>();
      if (x == 1 || x > kLag) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (x == 1) mbar_arrive(qfull);
          mbar_arrive(full + 8 * done);
        }
        if (++done == S) done = 0;
      }
    }
    }
    cp_async_wait<0>();
  } else {
    // ------------------------------------------------------------ products
    regs_less<56>();
    const int i = warp - 12;
    if (i < 2 && lane == 0 && n_max > 0) {
      constexpr uint32_t idesc_s = make_idesc(1u, kTile, kTile);
      constexpr uint32_t idesc_o = make_idesc(1u, kTile, D) | (1u << 16);
      const uint32_t kv0 = smem_addr(smem) + M::kKV;
      const uint32_t ts = tmem + i * 128, to = tmem + 256 + i * 128;
      const uint64_t q_desc = sw128_kmajor_desc(smem_addr(smem) + M::kQ + i * M::kOperand);
      const int n = nt[i];
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok && !wait_here(bar, parity)) {
          timed_out();
          ok = false;
        }
        return ok;
      };
      auto next = [&]() {
        if (++stage == S) {
          stage = 0;
          phase ^= 1;
        }
      };
      // A stage is released when this tile's products have read it, or, where
      // the tile is done, at once.
      auto release = [&](int st, bool used) {
        if (used)
          tc_commit(empty + 8 * st);
        else
          mbar_arrive(empty + 8 * st);
      };
      auto scores = [&](int st) {
        const uint64_t b = sw128_kmajor_desc(kv0 + st * M::kOperand);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          const uint64_t off = ((c / 4) * M::kPart + (c % 4) * 32) >> 4;
          mma_bf16(ts, q_desc + off, b + off, idesc_s, c > 0);
        }
        tc_commit(sfull + 8 * i);
      };
      // Turns: this tile's products of step j follow the other's of step j (tile
      // 1) or j - 1 (tile 0).
      const uint32_t my_turn = turn + 8 * i, your_turn = turn + 8 * (1 - i);
      if (wait(qfull, 0) && wait(full, 0) && (i == 0 || wait(my_turn, 0))) {
        tc_fence_after_sync();
        if (n > 0) scores(0);
        mbar_arrive(your_turn);
        release(0, n > 0);
      }
      next();
      for (int j = 0; j < n_max && ok; ++j) {
        const int vs = stage;
        if (!wait(full + 8 * vs, phase)) break;
        next();
        const int ks = stage;
        const bool more = j + 1 < n_max;
        if (more) {
          if (!wait(full + 8 * ks, phase)) break;
          next();
        }
        if (!wait(my_turn, (j + i) & 1)) break;
        if (j < n) {
          const uint64_t b = sw128_mnmajor_desc(kv0 + vs * M::kOperand, M::kPart);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            if (!wait(pfull + 16 * half + 8 * i, j & 1)) break;
            tc_fence_after_sync();
#pragma unroll
            for (int c = 4 * half; c < 4 * half + 4; ++c)
              mma_bf16_tmem_a(to, ts + 8 * c, b + ((c * 2048) >> 4), idesc_o, j > 0 || c > 0);
          }
          if (!ok) break;
          if (j + 1 == n) tc_commit(ofull + 8 * i);
          if (j + 1 < n) scores(ks);
        }
        mbar_arrive(your_turn);
        release(vs, j < n);
        if (more) release(ks, j + 1 < n);
      }
      tc_commit(drain);
      if (!wait_here(drain, 0)) timed_out();
    }
    __syncwarp();
  }
  __syncthreads();
  if (warp == 12) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    return cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
                   q == cudaDriverEntryPointSuccess
               ? reinterpret_cast<EncodeTiledFn>(p)
               : nullptr;
  }();
  return fn;
}

// Tensor map of a cache's keys or values: channels, rows, heads; boxes of `box`
// rows of 64 channels.
hf_status cache_map(CUtensorMap* map, const CacheArgs& c, const void* base, int box) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) {
    set_error("cuTensorMapEncodeTiled is not available from the driver");
    return HF_ERR_CUDA;
  }
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(c.D), static_cast<cuuint64_t>(c.rows), static_cast<cuuint64_t>(c.H)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(c.row_stride) * 2, static_cast<cuuint64_t>(c.head_stride) * 2};
  const cuuint32_t boxes[3] = {64, static_cast<cuuint32_t>(box), 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, boxes, estr,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    set_error("cuTensorMapEncodeTiled failed (error " + std::to_string(static_cast<int>(r)) + ")");
    return HF_ERR_CUDA;
  }
  return HF_OK;
}

template <int SRC, int D>
hf_status launch_tiles(const CacheArgs& c, const AttendArgs& a, int max_kv, int box, cudaStream_t stream) {
  const int64_t tiles = most_tiles(a.n_tok, a.G, c.n_seq, 2 * kTile) * c.H;
  // keys are split where the tiles leave SMs idle, in parts of 512 keys at least,
  // as far as the workspace goes
  int64_t ns = std::min<int64_t>(device_sm_count() / tiles, (max_kv + 511) / 512);
  ns = std::min<int64_t>(ns, part_rows(device_sm_count()) / (static_cast<int64_t>(a.n_tok) * a.H_q));
  ns = std::max<int64_t>(1, std::min<int64_t>(ns, 64));
  CUtensorMap maps[2] = {};
  if constexpr (SRC == kByTensorCopies) {
    for (int v = 0; v < 2; ++v) {
      const hf_status st = cache_map(&maps[v], c, v ? c.v : c.k, box);
      if (st != HF_OK) return st;
    }
  }
  auto kern = attend_tiles_kernel<SRC, D>;
  HF_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<D>::kBytes),
              "hf_attend: shared memory size");
  kern<<<dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(ns)), kThreads, Smem<D>::kBytes, stream>>>(
      maps[0], maps[1], c, a, static_cast<int>(ns), box);
  HF_CUDA_TRY(cudaGetLastError(), "hf_attend: launch");
  if (ns > 1) return launch_join(HF_BF16, D, a, static_cast<int>(ns), stream);
  return HF_OK;
}

template <int D>
hf_status attend_tiles_d(const CacheArgs& c, const AttendArgs& a, hf_cache_kind kind, int max_kv, cudaStream_t stream) {
  if (kind == HF_CACHE_Q4) return launch_tiles<kFromCodes, D>(c, a, max_kv, 0, stream);
  // rows that lie together: a page's, in pieces that divide a step
  int box = kTile;
  while (c.table && c.block_size % box) box /= 2;
  if (box < 8 || c.rows == 0) return launch_tiles<kByCpAsync, D>(c, a, max_kv, 0, stream);
  return launch_tiles<kByTensorCopies, D>(c, a, max_kv, box, stream);
}

}  // namespace

bool attend_tiles_takes(hf_cache_kind kind, hf_dtype dtype, int D) {
  return dtype == HF_BF16 && kind != HF_CACHE_F32 && (D == 64 || D == 128);
}

hf_status attend_tiles(const CacheArgs& c, const AttendArgs& a, hf_cache_kind kind, int max_kv, cudaStream_t stream) {
  return c.D == 64 ? attend_tiles_d<64>(c, a, kind, max_kv, stream) : attend_tiles_d<128>(c, a, kind, max_kv, stream);
}

}  // namespace hf
