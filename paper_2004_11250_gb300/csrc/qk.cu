// Queries and keys normalised per head and rotated in one pass, keys and values
// stored to the paged cache (pp_qk_rotate, pp_qkv_store).
//
// y = x w / sqrt(mean x^2 + eps) over the D values of a head, then for each pair
// (a, b) -> (a cos - b sin, b cos + a sin).  The angle is position * frequency
// modulo a turn: the frequency in turns is a 64-bit fraction, so the wrapping
// product keeps the exact fraction of a turn whatever the position, and sincospi
// gets a number in [-1, 1).
//
// Bound by device memory (each value read and written once).  A lane holds V
// pairs of one head, both halves of each (two loads of 16 bytes; one run of 2 V
// values when interleaved), so the rotation needs no exchange and the mean one
// butterfly over the group of lanes that share a head.  A group keeps its token
// over a run of heads, whose sines are computed once, and has U heads in flight.
// Rows off 16-byte boundaries, or pairs that do not divide into whole lanes, take
// the form with single elements, pair j in lane j % 32.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "cache.h"
#include "internal.h"

namespace {

using namespace ppc;

constexpr int kThreads = 128;
constexpr int U = 4;       // heads in flight per group of lanes
constexpr int kSingle = 4; // pairs per lane of the form with single elements (D / 2 <= 128)

struct View {
  const void* p;
  int64_t ts, hs;
};

struct QkParams {
  View x[3];          // queries, keys, values
  const float* w[2];  // weights of queries, keys
  void *qo, *ko;      // dense outputs (ko null: the keys are stored)
  void *ck, *cv;      // the cache
  const int *pos, *slots;
  const uint64_t* turn;
  const uint8_t* axis;
  int* status;
  int T, Hq, Hk, Hv, D, pairs;
  int page, H;
  int64_t nslots;
  int run;            // heads per group of lanes
  float eps;
};

template <class T, bool WIDE>
constexpr int kPairs = WIDE ? 16 / (int)sizeof(T) : kSingle;

template <class T, bool WIDE, bool INTER, int GROUP>
__global__ void __launch_bounds__(kThreads) qk_kernel(const QkParams p) {
  constexpr int V = kPairs<T, WIDE>;
  const int64_t group = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / GROUP;
  const int lane = threadIdx.x % GROUP;
  const int heads = p.Hq + p.Hk + p.Hv, runs = (heads + p.run - 1) / p.run;
  if (group >= (int64_t)p.T * runs) return;  // whole groups leave: the butterfly below names its own lanes
  const int t = (int)(group / runs), h0 = (int)(group % runs) * p.run, h1 = min(h0 + p.run, heads);
  const unsigned mask = GROUP == 32 ? 0xFFFFFFFFu : ((1u << (GROUP & 31)) - 1u) << (threadIdx.x % 32 / GROUP * GROUP);
  const int half = p.D / 2, R = half - p.pairs;
  // pair i of the lane; beyond the rotated ones, what is not turned as pairs of its own two halves
  auto pair = [&](int i) { return WIDE ? lane * V + i : lane + 32 * i; };
  auto first = [&](int j) { return INTER ? 2 * j : j < p.pairs ? j : p.pairs + j; };
  auto second = [&](int j) { return INTER ? 2 * j + 1 : j < p.pairs ? p.pairs + j : p.pairs + j + R; };
  const bool on = pair(0) < half;
  const int ia = first(pair(0)), ib = INTER ? ia + V : second(pair(0));  // WIDE: where the lane's two runs begin

  float cs[V], sn[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    cs[i] = 1.f;
    sn[i] = 0.f;
    const int j = pair(i);
    if (h0 < p.Hq + p.Hk && j < p.pairs) {
      const int64_t at = p.pos[(int64_t)p.axis[j] * p.T + t];
      const uint64_t f = (uint64_t)at * p.turn[j];
      sincospif((float)(int32_t)(f >> 32) * 0x1p-31f, &sn[i], &cs[i]);
    }
  }
  int64_t slot = -1;
  if (p.slots) {
    slot = p.slots[t];
    if (slot >= p.nslots || slot < -1) {
      if (lane == 0) atomicOr(p.status, PP_CACHE_BAD_SLOT);
      slot = -1;
    }
  }
  const int64_t cell = slot < 0 ? 0 : (slot / p.page * p.H * p.page + slot % p.page) * p.D;

  for (int hb = h0; hb < h1; hb += U) {
    Vec<T, V> a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = hb + u;
      if (h >= h1 || !on) continue;
      const int part = h < p.Hq ? 0 : h < p.Hq + p.Hk ? 1 : 2;
      const int hh = part == 0 ? h : part == 1 ? h - p.Hq : h - p.Hq - p.Hk;
      const T* x = static_cast<const T*>(p.x[part].p) + t * p.x[part].ts + hh * p.x[part].hs;
      if (WIDE) {
        a[u] = *reinterpret_cast<const Vec<T, V>*>(x + ia);
        b[u] = *reinterpret_cast<const Vec<T, V>*>(x + ib);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int j = pair(i);
          if (j < half) {
            a[u].v[i] = x[first(j)];
            b[u].v[i] = x[second(j)];
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = hb + u;
      if (h >= h1) continue;
      const int part = h < p.Hq ? 0 : h < p.Hq + p.Hk ? 1 : 2;
      const int hh = part == 0 ? h : part == 1 ? h - p.Hq : h - p.Hq - p.Hk;
      if (part < 2) {
        float fa[V], fb[V];  // WIDE and INTER: the first V and the last V of the lane's 2 V values
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const bool in = WIDE ? on : pair(i) < half;
          fa[i] = in ? to_f32(a[u].v[i]) : 0.f;
          fb[i] = in ? to_f32(b[u].v[i]) : 0.f;
        }
        if (p.eps >= 0.f) {
          float s = 0.f;
#pragma unroll
          for (int i = 0; i < V; ++i) s += fa[i] * fa[i] + fb[i] * fb[i];
#pragma unroll
          for (int d = GROUP / 2; d > 0; d >>= 1) s += __shfl_xor_sync(mask, s, d);
          const float r = rsqrtf(s / (float)p.D + p.eps);
          const float* w = p.w[part];
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const bool in = w && (WIDE ? on : pair(i) < half);
            fa[i] *= r * (in ? w[WIDE ? ia + i : first(pair(i))] : 1.f);
            fb[i] *= r * (in ? w[WIDE ? ib + i : second(pair(i))] : 1.f);
          }
        }
        float ra[V], rb[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          // element of a pair in the lane's run of 2 V values
          const float x0 = !(WIDE && INTER) ? fa[i] : 2 * i < V ? fa[(2 * i) % V] : fb[(2 * i) % V];
          const float x1 = !(WIDE && INTER) ? fb[i] : 2 * i < V ? fa[(2 * i + 1) % V] : fb[(2 * i + 1) % V];
          const bool turned = pair(i) < p.pairs;  // the others stay as they are, infinities too
          ra[i] = turned ? x0 * cs[i] - x1 * sn[i] : x0;
          rb[i] = turned ? x1 * cs[i] + x0 * sn[i] : x1;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int k = WIDE && INTER ? 2 * i : i, l = WIDE && INTER ? 2 * i + 1 : i;
          (k < V ? a : b)[u].v[k % V] = from_f32<T>(ra[i]);
          (WIDE && INTER ? (l < V ? a : b) : b)[u].v[l % V] = from_f32<T>(rb[i]);
        }
      }
      T* y;
      if (part == 0)
        y = static_cast<T*>(p.qo) + ((int64_t)t * p.Hq + hh) * p.D;
      else if (part == 1 && p.ko)
        y = static_cast<T*>(p.ko) + ((int64_t)t * p.Hk + hh) * p.D;
      else
        y = slot < 0 ? nullptr : static_cast<T*>(part == 1 ? p.ck : p.cv) + cell + (int64_t)hh * p.page * p.D;
      if (!on || !y) continue;
      if (WIDE) {
        *reinterpret_cast<Vec<T, V>*>(y + ia) = a[u];
        *reinterpret_cast<Vec<T, V>*>(y + ib) = b[u];
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int j = pair(i);
          if (j < half) {
            y[first(j)] = a[u].v[i];
            y[second(j)] = b[u].v[i];
          }
        }
      }
    }
  }
}

template <class T, bool WIDE, bool INTER, int GROUP>
cudaError_t launch(QkParams p, cudaStream_t stream, int sms) {
  // Runs of heads: whole tokens when there are enough of them to fill the GPU (the sines are then computed once per
  // token), else as few heads per group as give every SM about 512 threads.
  const int heads = p.Hq + p.Hk + p.Hv;
  const int64_t want = (int64_t)sms * 512 / GROUP;
  const int64_t runs = std::min<int64_t>(heads, std::max<int64_t>(1, (want + p.T - 1) / p.T));
  p.run = (int)((heads + runs - 1) / runs);
  const int64_t groups = (int64_t)p.T * ((heads + p.run - 1) / p.run);
  const int64_t blocks = (groups * GROUP + kThreads - 1) / kThreads;
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  qk_kernel<T, WIDE, INTER, GROUP><<<(unsigned)blocks, kThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

template <class T, bool INTER>
cudaError_t by_group(const QkParams& p, bool wide, cudaStream_t stream, int sms) {
  if (!wide) return launch<T, false, INTER, 32>(p, stream, sms);
  const int lanes = p.D / 2 / kPairs<T, true>;
  if (lanes <= 4) return launch<T, true, INTER, 4>(p, stream, sms);
  if (lanes <= 8) return launch<T, true, INTER, 8>(p, stream, sms);
  if (lanes <= 16) return launch<T, true, INTER, 16>(p, stream, sms);
  return launch<T, true, INTER, 32>(p, stream, sms);
}

template <class T>
cudaError_t by_order(const QkParams& p, bool inter, bool wide, cudaStream_t stream, int sms) {
  return inter ? by_group<T, true>(p, wide, stream, sms) : by_group<T, false>(p, wide, stream, sms);
}

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

pp_status run(const pp_rope* rope, int dtype, QkParams& p, void* stream) {
  if (p.T == 0 || p.Hq + p.Hk + p.Hv == 0) return PP_OK;
  const size_t e = (size_t)dtype_size(dtype);
  const int n[3] = {p.Hq, p.Hk, p.Hv};
  const int W = 16 / (int)e;
  p.turn = rope->turn;
  p.axis = rope->axis;
  p.D = rope->D;
  p.pairs = rope->pairs;
  bool wide = p.pairs % W == 0 && p.D / 2 % W == 0;
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 0) continue;
    const View& x = p.x[i];
    if (!x.p || x.ts < 0 || x.hs < 0 || !aligned(x.p, e)) return PP_ERR_INVALID_ARG;
    wide = wide && aligned(x.p, 16) && x.ts % W == 0 && x.hs % W == 0;
    if (i < 2 && p.eps < 0.f && p.w[i]) return PP_ERR_INVALID_ARG;
    if (i < 2 && !aligned(p.w[i], 4)) return PP_ERR_INVALID_ARG;
  }
  if (p.Hq > 0 && (!p.qo || !aligned(p.qo, e))) return PP_ERR_INVALID_ARG;
  if (p.ko && !aligned(p.ko, e)) return PP_ERR_INVALID_ARG;
  wide = wide && aligned(p.qo, 16) && aligned(p.ko, 16);
  if (p.pairs > 0 && p.Hq + p.Hk > 0 && !p.pos) return PP_ERR_INVALID_ARG;
  const int sms = device_sms();
  if (sms <= 0) return PP_ERR_CUDA;
  const cudaStream_t s = (cudaStream_t)stream;
  const cudaError_t err = dtype == PP_F32   ? by_order<float>(p, rope->interleaved, wide, s, sms)
                          : dtype == PP_F16 ? by_order<__half>(p, rope->interleaved, wide, s, sms)
                                            : by_order<__nv_bfloat16>(p, rope->interleaved, wide, s, sms);
  return err == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

}  // namespace

extern "C" {

pp_status pp_rope_create(int D, int pairs, const uint8_t* axis, const double* freq, int axes, int interleaved,
                         void* stream, pp_rope** out) {
  if (!out || pairs < 0 || 2 * (int64_t)pairs > D || axes < 1 || axes > 8 || (pairs > 0 && !freq))
    return PP_ERR_INVALID_ARG;
  if (D < 2 || D > 256 || D % 2) return PP_ERR_UNSUPPORTED;
  unsigned char host[128 * 9] = {};  // turns, then axes
  for (int j = 0; j < pairs; ++j) {
    if ((axis && axis[j] >= axes) || !std::isfinite(freq[j])) return PP_ERR_INVALID_ARG;
    double f = std::fmod(freq[j] / 6.283185307179586476925, 1.0);
    if (f < 0) f += 1.0;
    if (f >= 1.0) f = 0.0;  // a negative number too small to move 1
    const double hi = std::floor(std::ldexp(f, 32));  // two steps: 2^64 itself does not fit
    const uint64_t turn = ((uint64_t)hi << 32) | (uint64_t)std::floor(std::ldexp(std::ldexp(f, 32) - hi, 32));
    reinterpret_cast<uint64_t*>(host)[j] = turn;
    host[128 * 8 + j] = axis ? axis[j] : 0;
  }
  pp_rope* r = new (std::nothrow) pp_rope;
  if (!r) return PP_ERR_OOM;
  r->D = D;
  r->pairs = pairs;
  r->axes = axes;
  r->interleaved = interleaved != 0;
  const cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e = cudaMalloc(&r->dmem, sizeof(host));
  if (e != cudaSuccess) {
    cudaGetLastError();
    delete r;
    return e == cudaErrorMemoryAllocation ? PP_ERR_OOM : PP_ERR_CUDA;
  }
  e = cudaMemcpyAsync(r->dmem, host, sizeof(host), cudaMemcpyHostToDevice, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) {
    pp_rope_destroy(r);
    return PP_ERR_CUDA;
  }
  r->turn = static_cast<const uint64_t*>(r->dmem);
  r->axis = static_cast<const uint8_t*>(r->dmem) + 128 * 8;
  *out = r;
  return PP_OK;
}

void pp_rope_destroy(pp_rope* rope) {
  if (!rope) return;
  cudaFree(rope->dmem);
  delete rope;
}

pp_status pp_qk_rotate(const pp_rope* rope, int dtype, int T, const int32_t* pos, float eps, const void* q, int64_t q_ts,
                       int64_t q_hs, int Hq, const float* qw, void* q_out, const void* k, int64_t k_ts, int64_t k_hs,
                       int Hk, const float* kw, void* k_out, void* stream) {
  if (!rope || !dtype_ok(dtype) || T < 0 || Hq < 0 || Hk < 0 || eps != eps || (Hk > 0 && !k_out))
    return PP_ERR_INVALID_ARG;
  QkParams p = {};
  p.x[0] = {q, q_ts, q_hs};
  p.x[1] = {k, k_ts, k_hs};
  p.w[0] = qw;
  p.w[1] = kw;
  p.qo = q_out;
  p.ko = k_out;
  p.pos = pos;
  p.T = T;
  p.Hq = Hq;
  p.Hk = Hk;
  p.page = p.H = 1;
  p.eps = eps;
  return run(rope, dtype, p, stream);
}

pp_status pp_qkv_store(const pp_rope* rope, const pp_cache* cache, int T, const int32_t* pos, const int32_t* slots,
                       float eps, const void* q, int64_t q_ts, int64_t q_hs, int Hq, const float* qw, void* q_out,
                       const void* k, int64_t k_ts, int64_t k_hs, const float* kw, const void* v, int64_t v_ts,
                       int64_t v_hs, void* stream) {
  if (!rope || !cache || T < 0 || Hq < 0 || eps != eps || rope->D != cache->D || (T > 0 && !slots))
    return PP_ERR_INVALID_ARG;
  QkParams p = {};
  p.x[0] = {q, q_ts, q_hs};
  p.x[1] = {k, k_ts, k_hs};
  p.x[2] = {v, v_ts, v_hs};
  p.w[0] = qw;
  p.w[1] = kw;
  p.qo = q_out;
  p.ck = cache->k;
  p.cv = cache->v;
  p.pos = pos;
  p.slots = slots;
  p.status = cache->status;
  p.T = T;
  p.Hq = Hq;
  p.Hk = p.Hv = cache->H;
  p.page = cache->page;
  p.H = cache->H;
  p.nslots = (int64_t)cache->pages * cache->page;
  p.eps = eps;
  return run(rope, cache->dtype, p, stream);
}

}  // extern "C"
