// RMS norms of queries and keys for each head, rotation by one or several position axes, and the paged append, in one
// pass over the step's new tokens (aspd_qk_norm_append).
//
//     y = x * rsqrt(mean(x^2) + eps) * w;   (y_i, y_{i+d/2}) turned by pos[axis(i)] * theta^(-2i/d)
//
// A unit is one head of q, k_new or v_new: L = d / 2 / VEC neighbouring lanes, each with a 16-byte chunk of the first half of
// the head and its partner chunk in the second half, so that a pair turns inside a thread and a head's sum of squares is
// log2(L) shuffles.  A block takes a run of tokens, all heads of a token at a time (heads beyond what 512 threads hold have
// blocks of their own): a thread's chunks of the next kStages - 1 tokens are on their way to a place of its own in shared
// memory (cp.async; nobody else reads them, so there is no barrier), while the sines and cosines of a group of tokens are made
// by all threads at once, for all heads.
//
// Bound by memory where there are many tokens: 17 069 of 28/4 heads of 128 in bf16 (349 MB) 59 us, 5.9 TB/s, 0.90 of the copy
// bandwidth; by latency where there are few: 4 tokens 2.0 us in a graph, 142 tokens 2.7.  What made the difference on the many:
// a token to a block, loads straight into registers, 94 us; the ring 73; the sines and cosines side by side for a head's lanes
// (11-way bank conflicts before) and packed fp32 pairs 64; positions asked for a group ahead 59.  Three blocks to an SM with
// their registers cut to 64 instead of two with 80: 68.
#include <type_traits>

#include "aspd_internal.cuh"

namespace aspd {
namespace {

constexpr int kMaxNormThreads = 512, kStages = 4, kMaxGroup = 8, kNormThreadsPerSm = 640;

struct NormArgs {
  const void *q, *k_new, *v_new, *q_weight, *k_weight;
  const int32_t* pos;
  void *k_pool, *v_pool, *q_out;
  int64_t q_stride, k_stride, v_stride;
  float eps;
  int n_new, n_q_heads, n_kv_heads, page_size, rotate_q;
  int per_block;               // tokens of a block
  uint8_t axis_of_pair[64];
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t at) {
  uint4 x;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
  return x;
}

__device__ __forceinline__ float2 to_f32x2(__nv_bfloat162 x) { return __bfloat1622float2(x); }
__device__ __forceinline__ float2 to_f32x2(float2 x) { return x; }
__device__ __forceinline__ void from_f32x2(float2 x, __nv_bfloat162* out) { *out = __float22bfloat162_rn(x); }
__device__ __forceinline__ void from_f32x2(float2 x, float2* out) { *out = x; }

template <typename T, int D>
__global__ void __launch_bounds__(kMaxNormThreads) qk_norm_kernel(const __grid_constant__ NormArgs a, PlanDevice pd) {
  using T2 = std::conditional_t<sizeof(T) == 2, __nv_bfloat162, float2>;
  constexpr int VEC = 16 / (int)sizeof(T), HALF = D / 2, L = HALF / VEC, ROW_BYTES = D * (int)sizeof(T);
  extern __shared__ __align__(16) uint8_t ring[];                  // [kStages][2][threads] chunks of 16 bytes
  // two groups: one is made while the other may still be read.  [pairs 2 m, 2 m + 1 of a chunk][chunk]: (cos, cos, sin, sin), so
  // that the lanes of a head read 16 bytes each side by side
  __shared__ float4 cs_sm[2][kMaxGroup][VEC / 2][L];
  __shared__ ulonglong2 place_sm[2][kMaxGroup];                    // byte offset of the row's line in the page's first tile (all ones: none); row % 8
  pdl_launch_dependents();
  const int tid = threadIdx.x, c = tid % L, units = a.n_q_heads + 2 * a.n_kv_heads, u = blockIdx.y * (blockDim.x / L) + tid / L;
  const int t0 = blockIdx.x * a.per_block, n_tok = min(a.per_block, a.n_new - t0);
  const int group = max(1, min(kMaxGroup, (int)blockDim.x / HALF));    // tokens whose sines and cosines are made together
  const int uk = u - a.n_q_heads, uv = uk - a.n_kv_heads;
  const bool is_q = uk < 0, is_v = uv >= 0, active = u < units;
  const bool turn = is_q ? a.rotate_q : !is_v;
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring) + tid * 16u, half_ring = blockDim.x * 16u;
  const size_t tb = tile_bytes(a.page_size, D, sizeof(T));
  // what the thread reads (the next token's chunk to request) and writes
  const size_t stride = is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride;
  const T* src = static_cast<const T*>(is_q ? a.q : is_v ? a.v_new : a.k_new) + t0 * stride + (is_q ? u : is_v ? uv : uk) * D + c * VEC;
  T* q_dst = static_cast<T*>(a.q_out) + ((size_t)t0 * a.n_q_heads + u) * D + c * VEC;
  char* const pool = static_cast<char*>(is_v ? a.v_pool : a.k_pool) + (is_v ? uv : uk) * tb;
  constexpr uint32_t kHalfBytes = HALF * sizeof(T);
  int asked = 0;
  uint32_t ask_at = mine;                          // the ring's next place to fill
  auto request = [&] {
    if (asked < n_tok && active) {
      cp_async16(ask_at, src);
      cp_async16(ask_at + half_ring, src + HALF);
    }
    src += stride;
    ++asked;
    ask_at = asked % kStages == 0 ? mine : ask_at + 2 * half_ring;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  pdl_wait();
#pragma unroll
  for (int j = 0; j < kStages - 1; ++j) request();
  const T* w = static_cast<const T*>(is_q ? a.q_weight : a.k_weight);
  const bool normalise = w != nullptr && !is_v;
  uint4 w0 = make_uint4(0, 0, 0, 0), w1 = w0;
  if (normalise) {
    w0 = *reinterpret_cast<const uint4*>(w + c * VEC);
    w1 = *reinterpret_cast<const uint4*>(w + HALF + c * VEC);
  }
  // positions and places of a group are asked for a group ahead
  auto pos_of = [&](int e, int g0) { return a.pos[(size_t)a.axis_of_pair[e % HALF] * a.n_new + t0 + g0 + e / HALF]; };
  const double freq = pd.inv_freq[tid % HALF];
  int next_pos = 0, next_page = 0, next_row = 0;
  auto ask_group = [&](int g0) {
    const int n = min(group, n_tok - g0);
    if (tid < n * HALF) next_pos = pos_of(tid, g0);
    if (tid < n) { next_page = pd.tok_page[t0 + g0 + tid]; next_row = pd.tok_row[t0 + g0 + tid]; }
  };
  ask_group(0);
  uint32_t at = mine;                              // the ring's next place to read
  for (int g0 = 0, buf = 0; g0 < n_tok; g0 += group, buf ^= 1) {
    // the group's sines and cosines, angle reduced to [-pi, pi] in fp64, then fp32 sincos (as the append kernel); its places
    const int n_group = min(group, n_tok - g0);
    for (int e = tid; e < n_group * HALF; e += blockDim.x) {         // (once, but in blocks of fewer threads than pairs)
      const int k = e / HALF, i = e % HALF;
      double ang = e == tid ? (double)next_pos * freq : (double)pos_of(e, g0) * pd.inv_freq[i];
      ang -= rint(ang * 0.15915494309189535) * 6.283185307179586;
      float sn, cs;
      sincosf((float)ang, &sn, &cs);
      float* to = reinterpret_cast<float*>(&cs_sm[buf][k][i % VEC / 2][i / VEC]) + i % 2;
      to[0] = cs; to[2] = sn;
    }
    if (tid < n_group) {
      const int page = next_page, row = next_row;
      const size_t line = (size_t)page * a.n_kv_heads * tb + (row >> 3) * (8 * ROW_BYTES) + (row & 7) * 128;
      place_sm[buf][tid] = make_ulonglong2(bounds_ok(pd, page, row, a.page_size) ? line : ~0ull, row & 7);
    }
    __syncthreads();                               // (the buffer's readers of two groups ago have passed the one between)
    ask_group(g0 + group);
    for (int k = 0; k < n_group; ++k) {
      request();
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      uint4 x0 = ld_shared16(at), x1 = ld_shared16(at + half_ring);
      at = (g0 + k + 1) % kStages == 0 ? mine : at + 2 * half_ring;
      T2* e0 = reinterpret_cast<T2*>(&x0);
      T2* e1 = reinterpret_cast<T2*>(&x1);
      // (a warp may hold heads of all three kinds, and the shuffles need all of it: the values' lanes go along)
      float2 f0[VEC / 2], f1[VEC / 2], s2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < VEC / 2; ++j) {
        f0[j] = to_f32x2(e0[j]); f1[j] = to_f32x2(e1[j]);
        s2 = __ffma2_rn(f0[j], f0[j], __ffma2_rn(f1[j], f1[j], s2));
      }
      float ss = s2.x + s2.y;
#pragma unroll
      for (int o = L / 2; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (normalise) {
        const float r = rsqrtf(ss * (1.f / D) + a.eps);
        const T2* m0 = reinterpret_cast<const T2*>(&w0);
        const T2* m1 = reinterpret_cast<const T2*>(&w1);
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) {
          f0[j] = __fmul2_rn(__fmul2_rn(f0[j], make_float2(r, r)), to_f32x2(m0[j]));
          f1[j] = __fmul2_rn(__fmul2_rn(f1[j], make_float2(r, r)), to_f32x2(m1[j]));
        }
      }
      if (turn) {
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) {
          // the contractions that the append kernel is compiled to: its keys, bit for bit, where there is no norm
          const float4 cs = cs_sm[buf][k][j][c];
          const float2 t = __fmul2_rn(f1[j], make_float2(cs.z, cs.w)), p = __fmul2_rn(f1[j], make_float2(cs.x, cs.y));
          from_f32x2(__ffma2_rn(f0[j], make_float2(cs.x, cs.y), make_float2(-t.x, -t.y)), &e0[j]);
          from_f32x2(__ffma2_rn(f0[j], make_float2(cs.z, cs.w), p), &e1[j]);
        }
      } else if (normalise) {
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) { from_f32x2(f0[j], &e0[j]); from_f32x2(f1[j], &e1[j]); }
      }
      if (is_q) {
        if (active) {
          *reinterpret_cast<uint4*>(q_dst) = x0;
          *reinterpret_cast<uint4*>(q_dst + HALF) = x1;
        }
        q_dst += (size_t)a.n_q_heads * D;
      } else if (active) {
        const ulonglong2 place = place_sm[buf][k];
        if (place.x == ~0ull) continue;
        // tile_offset with the row's part taken out: the span of the chunk and its place in the line
        const uint32_t r7 = (uint32_t)place.y, b0 = c * 16, b1 = kHalfBytes + c * 16;
        *reinterpret_cast<uint4*>(pool + place.x + (b0 >> 7) * 1024 + ((((b0 & 127) >> 4) ^ r7) << 4)) = x0;
        *reinterpret_cast<uint4*>(pool + place.x + (b1 >> 7) * 1024 + ((((b1 & 127) >> 4) ^ r7) << 4)) = x1;
      }
    }
  }
}

template <typename T, int D>
int launch(const aspd_plan* p, NormArgs& a, cudaStream_t s) {
  constexpr int L = D / 2 / (16 / (int)sizeof(T));
  static bool configured[64] = {};                 // the attribute belongs to the (function, device) pair
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return ASPD_ERR_CUDA;
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    if (cudaFuncSetAttribute(qk_norm_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStages * 2 * kMaxNormThreads * 16) != cudaSuccess)
      return ASPD_ERR_CUDA;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  const int units = a.n_q_heads + 2 * a.n_kv_heads, most = kMaxNormThreads / L, slices = (units + most - 1) / most;
  const int threads = ((units + slices - 1) / slices * L + 31) / 32 * 32;
  // a token to a block while all blocks fit the chip at a time (two of 288 threads to an SM, by their registers); more tokens
  // to a block of a step that fills it
  const int at_a_time = p->sm_count * (kNormThreadsPerSm / threads > 0 ? kNormThreadsPerSm / threads : 1);
  a.per_block = (a.n_new + at_a_time - 1) / at_a_time;
  const dim3 grid((a.n_new + a.per_block - 1) / a.per_block, (units + threads / L - 1) / (threads / L));
  return launch_pdl(qk_norm_kernel<T, D>, grid, dim3(threads), kStages * 2 * threads * 16, s, a, p->dev) == cudaSuccess ? ASPD_OK : ASPD_ERR_CUDA;
}

}  // namespace

int launch_qk_norm(const aspd_plan* p, const aspd_qk_norm_t* nm, const void* q, int64_t q_stride, const void* k_new, int64_t k_stride,
                   const void* v_new, int64_t v_stride, const int32_t* pos, void* k_pool, void* v_pool, void* q_out, cudaStream_t s) {
  const aspd_shape_t& sh = p->shape;
  NormArgs a;
  a.q = q; a.k_new = k_new; a.v_new = v_new; a.q_weight = nm->q_weight; a.k_weight = nm->k_weight;
  a.pos = pos; a.k_pool = k_pool; a.v_pool = v_pool; a.q_out = q_out;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.eps = nm->eps; a.n_new = p->n_new; a.n_q_heads = sh.n_q_heads; a.n_kv_heads = sh.n_kv_heads; a.page_size = sh.page_size; a.rotate_q = nm->rotate_q != 0;
  for (int i = 0; i < 64; ++i) a.axis_of_pair[i] = i < sh.head_dim / 2 ? nm->axis_of_pair[i] : 0;
  if (sh.dtype == ASPD_DTYPE_BF16) return sh.head_dim == 128 ? launch<__nv_bfloat16, 128>(p, a, s) : launch<__nv_bfloat16, 64>(p, a, s);
  return sh.head_dim == 128 ? launch<float, 128>(p, a, s) : launch<float, 64>(p, a, s);
}

}  // namespace aspd
