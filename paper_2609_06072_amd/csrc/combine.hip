// The weighted sum of a token's expert outputs and its gradient (Sec. 3.1:
// the layer output is sum over the routed experts of p_e times their output):
//   out[t]      = sum over the routed slots j of w_tj y[t*k + j]
//   dy[t*k + j] = w_tj dout[t],   dw_tj = <dout[t], y[t*k + j]>
// A pair is routed where pair_row >= 0; rows of dropped pairs are neither read
// nor written.  Both are bound by HBM: every row is touched once, and y, out and dy
// stream through (non-temporal; 8192 tokens x 6 of 2048 bf16: forward 48.1 -> 43.8
// us, backward 55.2 -> 40.2 us, with dw 84.8 -> 74.2 us, 5.9 TB/s).
#include "ace_device.hpp"
#include "ace_internal.hpp"

namespace ace {

namespace {

// One 16-byte piece of out per thread; slots in index order (fixed result).
template <typename T>
__global__ __launch_bounds__(kThreads) void combine_fwd_kernel(CombineArgs a) {
  using F = typename Tr<T>::frag;
  constexpr int PER = Tr<T>::PER;
  const uint32_t idx = blockIdx.x * kThreads + threadIdx.x;
  if (idx >= a.pieces) return;
  const uint32_t t = a.per_row.div(idx), pc = (idx - t * a.per_row.d) * PER;
  const T* Y = static_cast<const T*>(a.y);
  T* out = static_cast<T*>(a.out) + (size_t)t * a.d + pc;
  float acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.f;
  bool routed = false;
  for (int j = 0; j < a.k; ++j) {
    const size_t p = (size_t)t * a.k + j;
    if (a.pair_row[p] < 0) continue;
    routed = true;
    const float w = a.pair_w ? a.pair_w[p] : 1.f;
    float v[PER];
    Tr<T>::to_f32(Tr<T>::load_nt(Y + p * a.d + pc), v);
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] += w * v[i];
  }
  if (a.accumulate) {
    if (!routed) return;   // (a sum with 0 would lose a zero's sign)
    float v[PER];
    Tr<T>::to_f32(Tr<T>::load(out), v);
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] += v[i];
  }
  Tr<T>::store_nt(out, Tr<T>::from_f32(acc));
}

// One wave per pair: its row of dy, and the row's dot product with dout[t]
// (lane sums over the row's pieces, then a fixed tree).
template <typename T>
__global__ __launch_bounds__(kThreads) void combine_bwd_kernel(CombineBwdArgs a) {
  using F = typename Tr<T>::frag;
  constexpr int PER = Tr<T>::PER;
  const int lane = threadIdx.x & 63;
  const long p = (long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (p >= a.P) return;
  if (a.pair_row[p] < 0) {
    if (a.dw && lane == 0) a.dw[p] = 0.f;
    return;
  }
  const float w = a.pair_w ? a.pair_w[p] : 1.f;
  const T* dout = static_cast<const T*>(a.dout) + (size_t)(p / a.k) * a.d;
  const T* Y = static_cast<const T*>(a.y) + (size_t)p * a.d;
  T* dy = static_cast<T*>(a.dy) + (size_t)p * a.d;
  float dot = 0.f;
  for (int c = lane * PER; c < a.d; c += 64 * PER) {
    float v[PER], o[PER];
    Tr<T>::to_f32(Tr<T>::load(dout + c), v);
    if (a.dw) {
      float y[PER];
      Tr<T>::to_f32(Tr<T>::load_nt(Y + c), y);
#pragma unroll
      for (int i = 0; i < PER; ++i) dot += v[i] * y[i];
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) o[i] = w * v[i];
    Tr<T>::store_nt(dy + c, Tr<T>::from_f32(o));
  }
  if (a.dw) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o, 64);
    if (lane == 0) a.dw[p] = dot;
  }
}

// One wave per row.
template <typename T>
__global__ __launch_bounds__(kThreads) void zero_dropped_kernel(const int32_t* pair_row, int T_, int d, T* out) {
  const int t = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (t >= T_ || pair_row[t] >= 0) return;
  for (int c = (threadIdx.x & 63) * Tr<T>::PER; c < d; c += 64 * Tr<T>::PER)
    Tr<T>::store(out + (size_t)t * d + c, Tr<T>::zero());
}

}  // namespace

hipError_t launch_zero_dropped(int dtype, const int32_t* pair_row, int T, int d, void* out, hipStream_t stream) {
  const int grid = (T + kThreads / 64 - 1) / (kThreads / 64);
  if (dtype == ACE_BF16) zero_dropped_kernel<__bf16><<<grid, kThreads, 0, stream>>>(pair_row, T, d, static_cast<__bf16*>(out));
  else zero_dropped_kernel<float><<<grid, kThreads, 0, stream>>>(pair_row, T, d, static_cast<float*>(out));
  return hipGetLastError();
}

hipError_t launch_combine_fwd(int dtype, CombineArgs a, int T, hipStream_t stream) {
  const int per = dtype == ACE_BF16 ? 8 : 4;
  a.per_row = FastDiv(a.d / per);
  a.pieces = (uint32_t)((long)T * (a.d / per));
  const unsigned grid = (a.pieces + kThreads - 1) / kThreads;
  if (grid == 0) return hipSuccess;
  if (dtype == ACE_BF16) combine_fwd_kernel<__bf16><<<grid, kThreads, 0, stream>>>(a);
  else combine_fwd_kernel<float><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_combine_bwd(int dtype, const CombineBwdArgs& a, hipStream_t stream) {
  const long grid = (a.P + kThreads / 64 - 1) / (kThreads / 64);
  if (grid == 0) return hipSuccess;
  if (dtype == ACE_BF16) combine_bwd_kernel<__bf16><<<(unsigned)grid, kThreads, 0, stream>>>(a);
  else combine_bwd_kernel<float><<<(unsigned)grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ace
