// Dropout of a branch that joins the residual stream, and its gradient, from a counter-based generator: element i is dropped if 16-bit word first + i of
// the stream of `seed` is below round(p 65536), and the elements that stay are divided by the share that stays.  The mask is never stored: the
// backward draws the same words again.
//
// Words: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) with key seed and counter j gives words 8 j .. 8 j + 7,
// the low half of each of its four results first.  Memory and the generator's 32-bit products (a quarter of the full rate) take about as
// long as each other with a word of 32 bits an element; with 16 bits the generator takes half, and p is a multiple of 2^-16.
#include "dropout.h"

namespace cephalo {
namespace {

struct Words { unsigned v[4]; };
__device__ __forceinline__ Words philox(uint64_t counter, uint64_t seed) {
  unsigned x0 = (unsigned)counter, x1 = (unsigned)(counter >> 32), x2 = 0, x3 = 0, k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)x0 * 0xD2511F53u, b = (uint64_t)x2 * 0xCD9E8D57u;
    x0 = (unsigned)(b >> 32) ^ x1 ^ k0; x1 = (unsigned)b;
    x2 = (unsigned)(a >> 32) ^ x3 ^ k1; x3 = (unsigned)a;
    k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
  }
  return {{x0, x1, x2, x3}};
}
__device__ __forceinline__ bool kept(const Words& w, int i, unsigned drop) { return ((i & 1) ? w.v[i >> 1] >> 16 : w.v[i >> 1] & 0xffffu) >= drop; }

template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; j += Vec<T>::N) {
    float part[Vec<T>::N];
    load_vec<T>(p + j, part);
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) v[j + i] = part[i];
  }
}
template <typename T, bool STREAM> __device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; j += Vec<T>::N) {
    float part[Vec<T>::N];
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) part[i] = v[j + i];
    store_vec_past<T, STREAM>(p + j, part);
  }
}

// ADD: out = resid + dropout(in), fp32;  else out = dropout(in)
template <typename IN, typename OUT, bool ADD, bool STREAM>
__global__ void __launch_bounds__(kDropoutBlock)
dropout_kernel(DropoutArgs d, const IN* __restrict__ in, const float* resid, OUT* out) {
  const int64_t group = (int64_t)blockIdx.x * kDropoutBlock + threadIdx.x, at = group * 8;
  if (at >= d.n) return;
  const uint64_t first = d.first + (d.counter ? *d.counter : 0);
  float x[8], r[8];
  const bool whole = at + 8 <= d.n;
  if (whole) {
    load8<IN>(in + at, x);
    if (ADD) load8<float>(resid + at, r);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = at + i < d.n ? (float)in[at + i] : 0.f;
      if (ADD) r[i] = at + i < d.n ? resid[at + i] : 0.f;
    }
  }
  const Words w = philox((first >> 3) + (uint64_t)group, d.seed);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = kept(w, i, d.drop) ? x[i] * d.scale : 0.f;
    x[i] = ADD ? r[i] + v : v;
  }
  if (whole) {
    store8<OUT, STREAM>(out + at, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at + i < d.n) out[at + i] = (OUT)x[i];
  }
}

template <typename IN, typename OUT, bool ADD>
int launch(const DropoutArgs& d, const IN* in, const float* resid, OUT* out, hipStream_t s) {
  const int64_t blocks = (d.n + kDropoutBlock * 8 - 1) / (kDropoutBlock * 8);
  if (blocks == 0) return CEPHALO_OK;
  // Results beyond 32 MiB, which the L2s together do not hold, go past them: 12288 x 2048, bf16 branch, forward 44 -> 41.7 us (6.0 TB/s), backward 28.2 -> 21.3.
  // (Two or four groups of 8 a thread: no difference, and 131 x 257 3.4 and 4.0 us instead of 2.5.)
  const bool stream = d.n * (int64_t)sizeof(OUT) > (int64_t)32 << 20;
  const auto kern = stream ? dropout_kernel<IN, OUT, ADD, true> : dropout_kernel<IN, OUT, ADD, false>;
  kern<<<(unsigned)blocks, kDropoutBlock, 0, s>>>(d, in, resid, out);
  CEPHALO_CHECK_LAUNCH("dropout");
  return CEPHALO_OK;
}

}  // namespace

template <typename T> int launch_dropout_add(const DropoutArgs& d, const T* branch, const float* resid, float* out, hipStream_t s) {
  return launch<T, float, true>(d, branch, resid, out, s);
}
template <typename T> int launch_dropout_bwd(const DropoutArgs& d, const float* dy, T* dbranch, hipStream_t s) {
  return launch<float, T, false>(d, dy, nullptr, dbranch, s);
}
template int launch_dropout_add<float>(const DropoutArgs&, const float*, const float*, float*, hipStream_t);
template int launch_dropout_add<bf16>(const DropoutArgs&, const bf16*, const float*, float*, hipStream_t);
template int launch_dropout_bwd<float>(const DropoutArgs&, const float*, float*, hipStream_t);
template int launch_dropout_bwd<bf16>(const DropoutArgs&, const float*, bf16*, hipStream_t);

}  // namespace cephalo
