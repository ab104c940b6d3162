// SwiGLU between the gate/up and the down projections, and 8-bit checkpoints
// of activations for the backward.
//
//   a  = g sigma(g) u
//   dg = da u sigma(g) (1 + g (1 - sigma(g))),   du = da g sigma(g)
//
// Checkpoint (the OCP MXINT8 value): 32 columns of a row share the byte s,
//   s     = exponent field of the block's largest |x| as an fp32 number, plus one
//           where that |x| would round to code 128 (s stays below 255),
//   code  = x 2^(133 - s) rounded to nearest even, at most 127 in size,
//   value = code 2^(s - 133).
// Scaling by a power of two is exact, so the one rounding fixes every bit, and
// a value's seven bits are exact in bf16.  An error is at most half a step,
// 2^(s - 134) <= amax / 127.5 (one step where s would pass 254).  A block that
// holds a NaN or an infinity gets s = 255 and reads back as NaN.
//
// Everything here is bound by HBM.  A thread takes one 16-byte piece (8 bf16 or
// 4 fp32 columns) of a row at a time, so a block's four or eight pieces sit in
// neighbouring lanes: its largest |x| comes from two or three lane exchanges,
// without LDS.  Rows are filled up to whole blocks (lanes past the row's end
// hold zeros and store nothing).
#include <type_traits>

#include "ace_device.hpp"
#include "ace_internal.hpp"

namespace ace {

namespace {

constexpr int kBlockCols = 32;

template <typename T>
struct Pieces {
  static constexpr int PER = Tr<T>::PER, PPB = kBlockCols / PER;   // pieces per block
};

// The codes of one piece: PER bytes.
template <typename T>
struct CodeWord;
template <>
struct CodeWord<__bf16> {
  using type = u32x2;
  __device__ static inline uint32_t word(type c, int i) { return c[i]; }
};
template <>
struct CodeWord<float> {
  using type = uint32_t;
  __device__ static inline uint32_t word(type c, int) { return c; }
};

// s of the block that this lane's PER values belong to (all lanes of the
// block get it).
template <typename T>
__device__ inline uint32_t block_exp(const float* v) {
  uint32_t top = 0;   // |x| as bits: ordered like the numbers, NaN above infinity
#pragma unroll
  for (int i = 0; i < Tr<T>::PER; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < Pieces<T>::PPB; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  const uint32_t s = top >> 23;
  const float m = __uint_as_float(top) * __uint_as_float(s >= 254 ? 0x00400000u : (254u - s) << 23) * 64.f;
  return s < 254 && m >= 127.5f ? s + 1 : s;
}

template <typename T>
__device__ inline typename CodeWord<T>::type encode(const float* v, uint32_t s) {
  // 2^(127 - s), the power of two below the smallest normal number for 254
  const float inv = __uint_as_float(s >= 254 ? 0x00400000u : (254u - s) << 23);
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < Tr<T>::PER; ++i) {
    const float c = fminf(fmaxf(rintf(v[i] * inv * 64.f), -127.f), 127.f);
    w[i / 4] |= (s == 255 ? 0u : (uint32_t)(int)c & 255u) << (8 * (i & 3));
  }
  if constexpr (Tr<T>::PER == 8) return u32x2{w[0], w[1]};
  else return w[0];
}

template <typename T>
__device__ inline void decode(typename CodeWord<T>::type c, uint32_t s, float* v) {
  // 2^(s - 127); in two factors, as 2^(s - 133) may lie below the smallest normal number
  const float scale = __uint_as_float(s == 255 ? 0x7fc00000u : s == 0 ? 0x00400000u : s << 23);
#pragma unroll
  for (int i = 0; i < Tr<T>::PER; ++i)
    v[i] = (float)(int8_t)(CodeWord<T>::word(c, i / 4) >> (8 * (i & 3))) * 0.015625f * scale;
}

// Where a thread's piece lies.  Pieces past the row's end belong to the
// row's last block.
struct Spot {
  bool in;        // inside the row
  size_t elem;    // first element of the piece
  size_t block;   // index of its block's s
  bool first;     // first piece of the block (stores s)
};
template <typename T>
__device__ inline Spot spot(const ActGeom& a, uint32_t idx) {
  constexpr int PER = Pieces<T>::PER, PPB = Pieces<T>::PPB;
  const uint32_t row = a.per_row.div(idx), pc = idx - row * a.per_row.d;
  return Spot{idx < a.pieces && pc * PER < (uint32_t)a.d, (size_t)row * a.d + pc * PER,
              (size_t)row * (a.per_row.d / PPB) + pc / PPB, pc % PPB == 0};
}

// Rows stream through: non-temporal loads and stores (32768 x 1408 bf16, backward
// 83.0 -> 75.0 us, 6.2 TB/s, from checkpoints 66.2 -> 57.9; a whole layer's step,
// whose other calls read and write these rows, takes the same time).  Packing alone
// keeps its loads in the caches (fp32 16000 x 1024 13.3 us, non-temporal 16.8).
template <typename T, bool NT = true>
__device__ inline void load_piece(const void* p, const Spot& s, float* v) {
  typename Tr<T>::frag f = Tr<T>::zero();
  const T* src = static_cast<const T*>(p) + s.elem;
  if (s.in) f = NT ? Tr<T>::load_nt(src) : Tr<T>::load(src);
  Tr<T>::to_f32(f, v);
}
template <typename T>
__device__ inline void store_piece(void* p, const Spot& s, const float* v) {
  Tr<T>::store_nt(static_cast<T*>(p) + s.elem, Tr<T>::from_f32(v));
}

template <typename T>
__device__ inline void store_packed(const ace_packed_act& c, const Spot& s, const float* v) {
  const uint32_t e = block_exp<T>(v);
  if (!s.in) return;
  *reinterpret_cast<typename CodeWord<T>::type*>(c.codes + s.elem) = encode<T>(v, e);
  if (s.first) c.exps[s.block] = (uint8_t)e;
}

// (for pieces inside the row only)
template <typename T>
__device__ inline void load_packed(const ace_packed_act& c, const Spot& s, float* v) {
  decode<T>(*reinterpret_cast<const typename CodeWord<T>::type*>(c.codes + s.elem), c.exps[s.block], v);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void pack_kernel(ActGeom a, const void* x, ace_packed_act c) {
  const Spot s = spot<T>(a, blockIdx.x * kThreads + threadIdx.x);
  float v[Tr<T>::PER];
  load_piece<T, false>(x, s, v);
  store_packed<T>(c, s, v);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void unpack_kernel(ActGeom a, ace_packed_act c, void* x) {
  const Spot s = spot<T>(a, blockIdx.x * kThreads + threadIdx.x);
  if (!s.in) return;
  float v[Tr<T>::PER];
  load_packed<T>(c, s, v);
  store_piece<T>(x, s, v);
}

// sigma(g) = sig * scale^2 and 1 - sigma(g) without overflow or cancellation: with
// t = exp(-|g|), one of them is 1 / (1 + t) and the other t / (1 + t).
// t = 2^n e^(r ln 2): n the product of |g| and -log2 e as rounded and r, its error
// and that of the constant, to first order; with the hardware's 2^n and reciprocal
// (1 ulp each) t is within 2 ulp.  (expf and a division bound the passes that read
// 8-bit codes: a from checkpoints of 32768 x 1408 47.7 us.)
// The hardware's 2^n is 0 below the normal numbers, where sigma u or sigma da need
// not be small.  FAR, for rows with g below kFar: below n = -100 it gives 2^(n + 126)
// (exact: n + 126 is), and scale 2^-63 goes once into the other factor and once into
// the product, so that neither leaves the range while the result is in it.  1 + t is
// 1 there.  sigma below 2^-252 (g < -174.6) is 0.  (FAR for all rows: the three passes
// over 32768 x 1408 with checkpoints 150 -> 158 us.)
constexpr float kFar = -69.f;   // n > -100

template <bool FAR>
__device__ inline void sigmoid2(float g, float& sig, float& one_minus, float& scale) {
#pragma clang fp contract(off)   // (n + 126 of n as rounded, or r is not its error)
  constexpr float kLog2e = 1.44269502f, kLog2eLow = 1.92596303e-8f;   // log2 e in two parts
  const float x = fminf(fabsf(g), 200.f);   // (e^-200 is 0; an infinity has no r)
  const float n = x * -kLog2e;
  const bool far = FAR && n < -100.f;
  const float r = fmaf(x, -kLog2eLow, fmaf(x, -kLog2e, -n));
  const float e = __builtin_amdgcn_exp2f(far ? n + 126.f : n);
  const float t = fmaf(e, r * 0.693147181f, e), p = far ? 1.f : __builtin_amdgcn_rcpf(1.f + t), q = t * p;
  sig = g < 0.f ? q : p;
  one_minus = g < 0.f ? p : far ? 0.f : q;
  scale = far && g < 0.f ? 0x1p-63f : 1.f;
}

// Calls f with whether any of a thread's g is below kFar.
template <int PER, typename F>
__device__ inline void by_range(const float* g, const F& f) {
  float least = g[0];
#pragma unroll
  for (int i = 1; i < PER; ++i) least = fminf(least, g[i]);
  if (least < kFar) f(std::true_type{});
  else f(std::false_type{});
}

// Where g and u come from, and whether their checkpoints are written.
enum { kPlain, kWritePacked, kReadPacked };

template <typename T, int CKPT>
__device__ inline void load_gu(const SwigluArgs& w, const Spot& s, float* g, float* u) {
  if (CKPT == kReadPacked) {
    load_packed<T>(w.g8, s, g);
    load_packed<T>(w.u8, s, u);
  } else {
    load_piece<T>(w.g, s, g);
    load_piece<T>(w.u, s, u);
  }
}

template <typename T, int CKPT>
__global__ __launch_bounds__(kThreads) void swiglu_fwd_kernel(ActGeom a, SwigluArgs w) {
  constexpr int PER = Tr<T>::PER;
  const Spot s = spot<T>(a, blockIdx.x * kThreads + threadIdx.x);
  // (writing checkpoints, lanes past the row's end take part in the exchanges)
  if (CKPT != kWritePacked && !s.in) return;
  float g[PER], u[PER], o[PER];
  load_gu<T, CKPT>(w, s, g, u);
  if (CKPT == kWritePacked) {
    store_packed<T>(w.g8, s, g);
    store_packed<T>(w.u8, s, u);
  }
  if (!s.in) return;
  by_range<PER>(g, [&](auto far) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      float sig, rest, scale;
      sigmoid2<far>(g[i], sig, rest, scale);
      o[i] = g[i] * sig * (u[i] * scale) * scale;
    }
  });
  store_piece<T>(w.a, s, o);
}

template <typename T, int CKPT>
__global__ __launch_bounds__(kThreads) void swiglu_bwd_kernel(ActGeom a, SwigluArgs w) {
  constexpr int PER = Tr<T>::PER;
  const Spot s = spot<T>(a, blockIdx.x * kThreads + threadIdx.x);
  if (!s.in) return;
  float da[PER], g[PER], u[PER], dg[PER], du[PER];
  load_piece<T>(w.da, s, da);
  load_gu<T, CKPT>(w, s, g, u);
  by_range<PER>(g, [&](auto far) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      float sig, rest, scale;
      sigmoid2<far>(g[i], sig, rest, scale);
      dg[i] = da[i] * u[i] * scale * (sig * (1.f + g[i] * rest)) * scale;
      du[i] = da[i] * scale * (g[i] * sig) * scale;
    }
  });
  store_piece<T>(w.dg, s, dg);
  store_piece<T>(w.du, s, du);
}

// Pieces of the rows, filled up to whole blocks.
ActGeom geometry(int dtype, long rows, int d) {
  const int per = dtype == ACE_BF16 ? 8 : 4;
  const int row = (d + kBlockCols - 1) / kBlockCols * (kBlockCols / per);
  return ActGeom{FastDiv(row), (uint32_t)(rows * row), d};
}

template <typename T>
void swiglu_fwd(const ActGeom& a, const SwigluArgs& w, unsigned grid, hipStream_t stream) {
  if (!w.g8.codes) swiglu_fwd_kernel<T, kPlain><<<grid, kThreads, 0, stream>>>(a, w);
  else if (w.g) swiglu_fwd_kernel<T, kWritePacked><<<grid, kThreads, 0, stream>>>(a, w);
  else swiglu_fwd_kernel<T, kReadPacked><<<grid, kThreads, 0, stream>>>(a, w);
}

template <typename T>
void swiglu_bwd(const ActGeom& a, const SwigluArgs& w, unsigned grid, hipStream_t stream) {
  if (w.g) swiglu_bwd_kernel<T, kPlain><<<grid, kThreads, 0, stream>>>(a, w);
  else swiglu_bwd_kernel<T, kReadPacked><<<grid, kThreads, 0, stream>>>(a, w);
}

}  // namespace

hipError_t launch_act_pack(int dtype, long rows, int d, const void* x, const ace_packed_act& c, hipStream_t stream) {
  const ActGeom a = geometry(dtype, rows, d);
  const unsigned grid = (a.pieces + kThreads - 1) / kThreads;
  if (dtype == ACE_BF16) pack_kernel<__bf16><<<grid, kThreads, 0, stream>>>(a, x, c);
  else pack_kernel<float><<<grid, kThreads, 0, stream>>>(a, x, c);
  return hipGetLastError();
}

hipError_t launch_act_unpack(int dtype, long rows, int d, const ace_packed_act& c, void* x, hipStream_t stream) {
  const ActGeom a = geometry(dtype, rows, d);
  const unsigned grid = (a.pieces + kThreads - 1) / kThreads;
  if (dtype == ACE_BF16) unpack_kernel<__bf16><<<grid, kThreads, 0, stream>>>(a, c, x);
  else unpack_kernel<float><<<grid, kThreads, 0, stream>>>(a, c, x);
  return hipGetLastError();
}

hipError_t launch_swiglu_fwd(int dtype, long rows, int d, const SwigluArgs& w, hipStream_t stream) {
  const ActGeom a = geometry(dtype, rows, d);
  const unsigned grid = (a.pieces + kThreads - 1) / kThreads;
  dtype == ACE_BF16 ? swiglu_fwd<__bf16>(a, w, grid, stream) : swiglu_fwd<float>(a, w, grid, stream);
  return hipGetLastError();
}

hipError_t launch_swiglu_bwd(int dtype, long rows, int d, const SwigluArgs& w, hipStream_t stream) {
  const ActGeom a = geometry(dtype, rows, d);
  const unsigned grid = (a.pieces + kThreads - 1) / kThreads;
  dtype == ACE_BF16 ? swiglu_bwd<__bf16>(a, w, grid, stream) : swiglu_bwd<float>(a, w, grid, stream);
  return hipGetLastError();
}

}  // namespace ace
