// RMS norms of queries and keys for each head, rotation by one or several position axes, and the paged append, in one
// pass over the step's new tokens (aspd_qk_norm_append).
//
//     y = x * rsqrt(mean(x^2) + eps) * w;   (y_i, y_{i+d/2}) turned by pos[axis(i)] * theta^(-2i/d)
//
// A block takes one token.  A unit is one head: L = d / 2 / VEC neighbouring lanes, each with a 16-byte chunk of the
// first half of the head and its partner chunk in the second half, so that a pair turns inside a thread and a head's sum
// of squares is log2(L) shuffles.  The units of K carry the head's V chunks along.  All loads of a thread are on their way
// before the token's sines and cosines are made (once per token, by the first d / 2 threads, for all heads), so
// that the two latencies lie beside each other.
#include "aspd_internal.cuh"

namespace aspd {
namespace {

template <typename T> __device__ inline float to_f32(T x);
template <> __device__ inline float to_f32<float>(float x) { return x; }
template <> __device__ inline float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ inline T from_f32(float x);
template <> __device__ inline float from_f32<float>(float x) { return x; }
template <> __device__ inline __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

constexpr int kMaxNormThreads = 512;

struct NormArgs {
  const void *q, *k_new, *v_new, *q_weight, *k_weight;
  const int32_t* pos;
  void *k_pool, *v_pool, *q_out;
  int64_t q_stride, k_stride, v_stride;
  float eps;
  int n_new, n_q_heads, n_kv_heads, page_size, rotate_q;
  uint8_t axis_of_pair[64];
};

template <typename T, int D>
__global__ void __launch_bounds__(kMaxNormThreads) qk_norm_kernel(const __grid_constant__ NormArgs a, PlanDevice pd) {
  constexpr int VEC = 16 / (int)sizeof(T), HALF = D / 2, L = HALF / VEC;
  __shared__ float2 cs_sm[HALF];
  pdl_launch_dependents();
  const int t = blockIdx.x, tid = threadIdx.x, c = tid % L, per_block = blockDim.x / L, n_units = a.n_q_heads + a.n_kv_heads;
  const int page = pd.tok_page[t], row = pd.tok_row[t];            // plan data: may be read before the dependency wait
  const double freq = tid < HALF ? pd.inv_freq[tid] : 0.0;
  const bool placed = bounds_ok(pd, page, row, a.page_size);
  pdl_wait();
  const size_t tb = tile_bytes(a.page_size, D, sizeof(T));
  for (int u0 = 0; u0 < n_units; u0 += per_block) {
    const int u = min(u0 + tid / L, n_units - 1);
    const bool active = u0 + tid / L < n_units, is_k = u >= a.n_q_heads;
    const int h = is_k ? u - a.n_q_heads : u;
    const T* x = static_cast<const T*>(is_k ? a.k_new : a.q) + (size_t)t * (is_k ? a.k_stride : a.q_stride) + h * D + c * VEC;
    const T* w = static_cast<const T*>(is_k ? a.k_weight : a.q_weight);
    uint4 x0 = *reinterpret_cast<const uint4*>(x), x1 = *reinterpret_cast<const uint4*>(x + HALF);
    uint4 w0 = make_uint4(0, 0, 0, 0), w1 = w0, v0 = w0, v1 = w0;
    if (w != nullptr) {
      w0 = *reinterpret_cast<const uint4*>(w + c * VEC);
      w1 = *reinterpret_cast<const uint4*>(w + HALF + c * VEC);
    }
    if (is_k) {
      const T* v = static_cast<const T*>(a.v_new) + (size_t)t * a.v_stride + h * D + c * VEC;
      v0 = *reinterpret_cast<const uint4*>(v);
      v1 = *reinterpret_cast<const uint4*>(v + HALF);
    }
    if (u0 == 0) {
      for (int i = tid; i < HALF; i += blockDim.x) {
        // angle reduced to [-pi, pi] in fp64, then fp32 sincos (as the append kernel)
        double ang = (double)a.pos[(size_t)a.axis_of_pair[i] * a.n_new + t] * (i == tid ? freq : pd.inv_freq[i]);
        ang -= rint(ang * 0.15915494309189535) * 6.283185307179586;
        float sn, cs;
        sincosf((float)ang, &sn, &cs);
        cs_sm[i] = make_float2(cs, sn);
      }
      __syncthreads();
    }
    float f0[VEC], f1[VEC];
    T* e0 = reinterpret_cast<T*>(&x0);
    T* e1 = reinterpret_cast<T*>(&x1);
#pragma unroll
    for (int j = 0; j < VEC; ++j) { f0[j] = to_f32(e0[j]); f1[j] = to_f32(e1[j]); }
    float ss = 0.f;                                // (taken without a weight too: the shuffles need the whole warp)
#pragma unroll
    for (int j = 0; j < VEC; ++j) ss = fmaf(f0[j], f0[j], fmaf(f1[j], f1[j], ss));
#pragma unroll
    for (int o = L / 2; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (w != nullptr) {
      const float r = rsqrtf(ss * (1.f / D) + a.eps);
      const T* g0 = reinterpret_cast<const T*>(&w0);
      const T* g1 = reinterpret_cast<const T*>(&w1);
#pragma unroll
      for (int j = 0; j < VEC; ++j) { f0[j] = f0[j] * r * to_f32(g0[j]); f1[j] = f1[j] * r * to_f32(g1[j]); }
    }
    if (is_k || a.rotate_q) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float2 cs = cs_sm[c * VEC + j];
        e0[j] = from_f32<T>(fmaf(f0[j], cs.x, -(f1[j] * cs.y)));      // the contractions that the append kernel is compiled to:
        e1[j] = from_f32<T>(fmaf(f0[j], cs.y, f1[j] * cs.x));         // its keys, bit for bit, where there is no norm
      }
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) { e0[j] = from_f32<T>(f0[j]); e1[j] = from_f32<T>(f1[j]); }
    }
    if (!active) continue;
    if (is_k) {
      if (!placed) continue;
      const size_t tile = ((size_t)page * a.n_kv_heads + h) * tb;
      const uint32_t o0 = tile_offset(row, c * 16, D * sizeof(T)), o1 = tile_offset(row, HALF * sizeof(T) + c * 16, D * sizeof(T));
      char *kp = static_cast<char*>(a.k_pool) + tile, *vp = static_cast<char*>(a.v_pool) + tile;
      *reinterpret_cast<uint4*>(kp + o0) = x0;
      *reinterpret_cast<uint4*>(kp + o1) = x1;
      *reinterpret_cast<uint4*>(vp + o0) = v0;
      *reinterpret_cast<uint4*>(vp + o1) = v1;
    } else {
      T* out = static_cast<T*>(a.q_out) + ((size_t)t * a.n_q_heads + h) * D + c * VEC;
      *reinterpret_cast<uint4*>(out) = x0;
      *reinterpret_cast<uint4*>(out + HALF) = x1;
    }
  }
}

template <typename T, int D>
int launch(const aspd_plan* p, const NormArgs& a, cudaStream_t s) {
  constexpr int L = D / 2 / (16 / (int)sizeof(T));
  const int want = (a.n_q_heads + a.n_kv_heads) * L;
  const int threads = want < kMaxNormThreads ? (want + 31) / 32 * 32 : kMaxNormThreads;
  return launch_pdl(qk_norm_kernel<T, D>, dim3(p->n_new), dim3(threads), 0, s, a, p->dev) == cudaSuccess ? ASPD_OK : ASPD_ERR_CUDA;
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
