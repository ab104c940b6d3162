// The weighted sum of a token's expert outputs and its gradient (Sec. 3.1:
// the layer output is sum over the routed experts of p_e times their output):
//   out[t]      = sum over the routed slots j of w_tj y[t*k + j]
//   dy[t*k + j] = w_tj dout[t],   dw_tj = <dout[t], y[t*k + j]>
// A pair is routed where pair_row >= 0; rows of dropped pairs are not used and not
// written.  Both are bound by HBM: every row is touched once, and y, out and dy
// stream through (non-temporal; 8192 tokens x 6 of 2048 bf16: backward 55.2 -> 40.2
// us, with dw 84.8 -> 74.2 us, 5.9 TB/s; forward 37.4 us, 6.3 TB/s).
#include "ace_device.hpp"
#include "ace_internal.hpp"

namespace ace {

namespace {

__device__ const float kOne = 1.f;

// One 16-byte piece of out per thread; slots in index order (fixed result), the
// loads of G slots under way at a time.
template <typename T, int G>
__global__ __launch_bounds__(kThreads) void combine_fwd_kernel(CombineArgs a) {
  using F = typename Tr<T>::frag;
  constexpr int PER = Tr<T>::PER;
  const uint32_t idx = blockIdx.x * kThreads + threadIdx.x;
  if (idx >= a.pieces) return;
  const uint32_t t = a.per_row.div(idx), pc = (idx - t * a.per_row.d) * PER;
  const T* Y = static_cast<const T*>(a.y);
  T* out = static_cast<T*>(a.out) + (size_t)t * a.d + pc;
  const auto W = (const __attribute__((address_space(1))) float*)(uintptr_t)(a.pair_w ? a.pair_w : &kOne);
  float acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.f;
  for (int j0 = 0; j0 < a.k; j0 += G) {
    int row[G];
    float w[G];
    F f[G];
    // (no branches: one would wait for the loads before it)
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const size_t p = (size_t)t * a.k + (G == 1 ? j0 : min(j0 + g, a.k - 1));
      row[g] = a.pair_row[p];
      w[g] = W[a.pair_w ? p : 0];
      f[g] = Tr<T>::load_nt(Y + p * a.d + pc);
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      asm volatile("" : "+v"(f[g]));   // loaded above, not behind the branch
      if (j0 + g >= a.k || row[g] < 0) continue;
      float v[PER];
      Tr<T>::to_f32(f[g], v);
#pragma unroll
      for (int i = 0; i < PER; ++i) acc[i] += w[g] * v[i];
    }
  }
  Tr<T>::store_nt(out, Tr<T>::from_f32(acc));
}

// L lanes per pair: its row of dy, and the row's dot product with dout[t]
// (lane sums over the row's pieces, then a fixed tree).
template <typename T, int L>
__global__ __launch_bounds__(kThreads) void combine_bwd_kernel(CombineBwdArgs a) {
  using F = typename Tr<T>::frag;
  constexpr int PER = Tr<T>::PER;
  const int lane = threadIdx.x % L;
  const long p = (long)blockIdx.x * (kThreads / L) + threadIdx.x / L;
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
  for (int c = lane * PER; c < a.d; c += L * PER) {
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
    for (int o = L / 2; o > 0; o >>= 1) dot += __shfl_xor(dot, o, 64);
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

// Slots under way: as many as the token has, up to eight (bf16 us, one / eight:
// 101 tokens x 16 of 4424 15.4 / 5.7, 4096 x 8 of 2048 29.6 / 26.2, 10744 x 8 of
// 232 14.9 / 9.9; with k = 2, whose other six are the last one over and over, 16384
// x 2 of 4096 two 62, eight 100).
template <typename T>
void combine_fwd(const CombineArgs& a, unsigned grid, hipStream_t stream) {
  if (a.k == 1) combine_fwd_kernel<T, 1><<<grid, kThreads, 0, stream>>>(a);
  else if (a.k == 2) combine_fwd_kernel<T, 2><<<grid, kThreads, 0, stream>>>(a);
  else if (a.k <= 4) combine_fwd_kernel<T, 4><<<grid, kThreads, 0, stream>>>(a);
  else combine_fwd_kernel<T, 8><<<grid, kThreads, 0, stream>>>(a);
}

// Lanes per pair: the fewest of 16, 32 and 64 that hold a row at once (bf16 with
// dw, us with 64 / 32 / 16: 12598 x 8 of 240 38.4 / 23.9 / 26.7, 3000 x 8 of 128
// 9.5 / 7.1 / 5.5, 4096 x 8 of 2048 53 / 62 / 74).
template <typename T>
void combine_bwd(const CombineBwdArgs& a, int lanes, unsigned grid, hipStream_t stream) {
  if (lanes == 16) combine_bwd_kernel<T, 16><<<grid, kThreads, 0, stream>>>(a);
  else if (lanes == 32) combine_bwd_kernel<T, 32><<<grid, kThreads, 0, stream>>>(a);
  else combine_bwd_kernel<T, 64><<<grid, kThreads, 0, stream>>>(a);
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
  if (dtype == ACE_BF16) combine_fwd<__bf16>(a, grid, stream);
  else combine_fwd<float>(a, grid, stream);
  return hipGetLastError();
}

hipError_t launch_combine_bwd(int dtype, const CombineBwdArgs& a, hipStream_t stream) {
  const int pieces = a.d / (dtype == ACE_BF16 ? 8 : 4);
  const int lanes = pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64;
  const long grid = (a.P + kThreads / lanes - 1) / (kThreads / lanes);
  if (grid == 0) return hipSuccess;
  if (dtype == ACE_BF16) combine_bwd<__bf16>(a, lanes, (unsigned)grid, stream);
  else combine_bwd<float>(a, lanes, (unsigned)grid, stream);
  return hipGetLastError();
}

}  // namespace ace
