// Queries and keys normalised per head and rotated in one pass, keys and values
// stored to the paged cache (pp_qk_rotate, pp_qkv_store).
//
// y = x w / sqrt(mean x^2 + eps) over the D values of a head, then for each pair
// (a, b) -> (a cos - b sin, b cos + a sin).  The angle is position * frequency
// modulo a turn: the frequency in turns is a 64-bit fraction, so the wrapping
// product is the fraction of a turn to 2^-33 whatever the position, and sincospi
// gets a number in [-1, 1).
//
// Bound by device memory (each value read and written once).  A lane holds V pairs
// of one head, both halves of each (two loads of 16 bytes; one run of 2 V values
// when interleaved), so the rotation needs no exchange and the mean one butterfly
// over the group of lanes that share a head.  A block has up to J heads per group,
// of one token or of neighbours: it asks for all of them at once, and while they
// are under way its threads work out the sines, one each, into shared memory.
// Rows off 16-byte boundaries, or pairs that do not divide into whole lanes, take
// the form with single elements, pair j in lane j % 32.
//
// Measured: 16384 tokens of 48 heads of 128 (f16) normalised, rotated and stored in
// 81 us, 5.0 TB/s (the copy rate is 6.8; the same kernel without norm and rotation
// takes 58 us); 3136 tokens of 16 heads of 64 (fp32) 5.7 us; one token 2.3 us.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "cache.h"
#include "internal.h"
#include "tc_ptx.cuh"

namespace {

using namespace ppc;
using namespace ppc_ptx;

constexpr int kThreads = 256;
constexpr int kSingle = 4;    // pairs per lane of the form with single elements (D / 2 <= 128)
constexpr int kAngles = 4096; // pairs of a block's tokens at most

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
  int page, log_page, H;
  int64_t nslots;
  int64_t items;      // (token, head) pairs
  int span;           // tokens of a block at most
  FastDiv heads;      // by the heads of all three
  float eps, inv_D;
};

template <class T, bool WIDE>
constexpr int kPairs = WIDE ? 16 / (int)sizeof(T) : kSingle;

// Where entry e of n lies in shared memory.  A lane reads V consecutive ones, 16 bytes at a time: with V = 8 the first
// four of all lanes come first, then the other four, so that neighbours read neighbouring words.
template <int V>
__device__ __forceinline__ int place(int e, int n) {
  return V == 8 ? (e >> 2 & 1) * (n / 2) + (e >> 3) * 4 + (e & 3) : e;
}
template <int V>
__device__ __forceinline__ void read_run(const float* from, int e, int n, float* to) {
#pragma unroll
  for (int i = 0; i < V; i += 4) {
    const float4 v = *reinterpret_cast<const float4*>(from + place<V>(e + i, n));
    to[i] = v.x;
    to[i + 1] = v.y;
    to[i + 2] = v.z;
    to[i + 3] = v.w;
  }
}

template <class T, bool WIDE, bool INTER, int GROUP, int J>
__global__ void __launch_bounds__(kThreads) qk_kernel(const QkParams p) {
  constexpr int V = kPairs<T, WIDE>, W = V / 2, GROUPS = kThreads / GROUP;
  extern __shared__ __align__(16) float shared[];  // weights of queries and keys, then the span's cosines and its sines
  float *weights = shared, *cosines = shared + 2 * p.D, *sines = cosines + p.span * p.pairs;
  const int lane = threadIdx.x % GROUP, grp = threadIdx.x / GROUP;
  const unsigned mask = GROUP == 32 ? 0xFFFFFFFFu : ((1u << (GROUP & 31)) - 1u) << (threadIdx.x % 32 / GROUP * GROUP);
  const int half = p.D / 2, R = half - p.pairs;
  // pair i of the lane; beyond the rotated ones, what is not turned as pairs of its own two halves
  auto pair = [&](int i) { return WIDE ? lane * V + i : lane + 32 * i; };
  auto first = [&](int j) { return INTER ? 2 * j : j < p.pairs ? j : p.pairs + j; };
  auto second = [&](int j) { return INTER ? 2 * j + 1 : j < p.pairs ? p.pairs + j : p.pairs + j + R; };
  const bool on = pair(0) < half;
  auto valid = [&](int i) { return WIDE ? on : pair(i) < half; };
  const int ia = first(pair(0)), ib = INTER ? ia + V : second(pair(0));  // WIDE: where the lane's two runs begin
  // element k of pair i in the lane's two vectors: (vector, place)
  auto vec_of = [](int i, int k) { return WIDE && INTER ? (2 * i + k) / V : k; };
  auto place_of = [](int i, int k) { return WIDE && INTER ? (2 * i + k) % V : i; };

  after_previous();
  // ---- the heads' values are asked for
  const int64_t i0 = (int64_t)blockIdx.x * GROUPS * J;
  const int t0 = (int)(i0 / p.heads.d), rest = (int)(i0 - (int64_t)t0 * p.heads.d);  // the first item's token, and its head
  Vec<T, V> ab[J][2];
  T* to[J];
  int tok[J], part[J];
  int head[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    // an item beyond the last is the last once more, and not stored: no conditions around the loads
    const int i = (int)min((int64_t)(rest + grp + j * GROUPS), p.items - 1 - i0 + rest);
    tok[j] = p.heads.div(i);
    const int h = i - tok[j] * p.heads.d;
    part[j] = h < p.Hq ? 0 : h < p.Hq + p.Hk ? 1 : 2;
    head[j] = h - (part[j] == 0 ? 0 : part[j] == 1 ? p.Hq : p.Hq + p.Hk);
    const View& x = p.x[part[j]];
    const T* from = static_cast<const T*>(x.p) + (t0 + tok[j]) * x.ts + head[j] * x.hs;
    if (WIDE) {
      ab[j][0] = *reinterpret_cast<const Vec<T, V>*>(from + (on ? ia : 0));
      ab[j][1] = *reinterpret_cast<const Vec<T, V>*>(from + (on ? ib : 0));
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int e = min(pair(k), half - 1);
        ab[j][0].v[k] = from[first(e)];
        ab[j][1].v[k] = from[second(e)];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int64_t t = t0 + tok[j];
    to[j] = nullptr;
    if (i0 + grp + j * GROUPS >= p.items) continue;
    if (part[j] == 0) {
      to[j] = static_cast<T*>(p.qo) + (t * p.Hq + head[j]) * p.D;
    } else if (part[j] == 1 && p.ko) {
      to[j] = static_cast<T*>(p.ko) + (t * p.Hk + head[j]) * p.D;
    } else {
      const int64_t slot = p.slots[t];
      if (slot >= 0 && slot < p.nslots) {
        const int64_t page = slot >> p.log_page;
        to[j] = static_cast<T*>(part[j] == 1 ? p.ck : p.cv) + (((page * p.H + head[j]) << p.log_page) + (slot & (p.page - 1))) * p.D;
      } else if (slot != -1 && lane == 0) {
        atomicOr(p.status, PP_CACHE_BAD_SLOT);
      }
    }
  }
  // ---- meanwhile the sines of the block's tokens, and the weights
  for (int i = threadIdx.x; i < p.span * p.pairs; i += kThreads) {
    const int tk = i / p.pairs, j = i - tk * p.pairs;
    if (t0 + tk >= p.T) break;
    const int64_t at = p.pos[(int64_t)p.axis[j] * p.T + t0 + tk];
    const uint64_t f = (uint64_t)at * p.turn[j];
    const int to = tk * p.pairs + (WIDE ? place<V>(j, p.pairs) : j);
    sincospif((float)(int32_t)(f >> 32) * 0x1p-31f, &sines[to], &cosines[to]);
  }
  for (int i = threadIdx.x; i < 2 * p.D; i += kThreads) {
    const int k = i >= p.D, d = i - k * p.D;
    weights[k * p.D + (WIDE ? place<V>(d, p.D) : d)] = p.w[k] ? p.w[k][d] : 1.f;
  }
  __syncthreads();
  // ---- each head, its V pairs as packs of two for the two-way fp32 instructions
#pragma unroll
  for (int j = 0; j < J; ++j) {
    if (part[j] < 2) {  // the same for a group
      uint64_t fa[W], fb[W], s2 = 0;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        if (WIDE && INTER) {  // a neighbour pair is a pair of the rotation
          const float2 x = get2(ab[j][4 * i / V], 2 * i % W), y = get2(ab[j][4 * i / V], (2 * i + 1) % W);
          fa[i] = pack2(x.x, y.x);
          fb[i] = pack2(x.y, y.y);
        } else {
          const float2 x = get2(ab[j][0], i), y = get2(ab[j][1], i);
          fa[i] = pack2(x.x, x.y);
          fb[i] = pack2(y.x, y.y);
        }
        if (!valid(2 * i) || !valid(2 * i + 1)) {  // beyond the head: 0
          float v[2];
          unpack2(fa[i], v[0], v[1]);
          fa[i] = pack2(valid(2 * i) ? v[0] : 0.f, valid(2 * i + 1) ? v[1] : 0.f);
          unpack2(fb[i], v[0], v[1]);
          fb[i] = pack2(valid(2 * i) ? v[0] : 0.f, valid(2 * i + 1) ? v[1] : 0.f);
        }
        s2 = fma2(fa[i], fa[i], s2);
        s2 = fma2(fb[i], fb[i], s2);
      }
      if (p.eps >= 0.f) {
        float s, s1, w[2 * V];  // the weights in the order of the lane's two vectors
        unpack2(s2, s, s1);
        s += s1;
#pragma unroll
        for (int d = GROUP / 2; d > 0; d >>= 1) s += __shfl_xor_sync(mask, s, d);
        const float r = rsqrtf(s * p.inv_D + p.eps);
        const uint64_t r2 = pack2(r, r);
        if (WIDE) {
          read_run<V>(weights + part[j] * p.D, on ? ia : 0, p.D, w);
          read_run<V>(weights + part[j] * p.D, on ? ib : 0, p.D, w + V);
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            w[i] = valid(i) ? weights[part[j] * p.D + first(pair(i))] : 1.f;
            w[V + i] = valid(i) ? weights[part[j] * p.D + second(pair(i))] : 1.f;
          }
        }
        auto weight = [&](int i, int k) { return w[vec_of(i, k) * V + place_of(i, k)]; };
#pragma unroll
        for (int i = 0; i < W; ++i) {
          fa[i] = mul2(mul2(fa[i], r2), pack2(weight(2 * i, 0), weight(2 * i + 1, 0)));
          fb[i] = mul2(mul2(fb[i], r2), pack2(weight(2 * i, 1), weight(2 * i + 1, 1)));
        }
      }
      // WIDE: a lane's pairs are turned all or not at all.  Those that are not stay as they are, infinities too
      if (WIDE ? pair(0) < p.pairs : true) {
        float c[V], n[V];
        if (WIDE) {
          read_run<V>(cosines + tok[j] * p.pairs, pair(0), p.pairs, c);
          read_run<V>(sines + tok[j] * p.pairs, pair(0), p.pairs, n);
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            c[i] = pair(i) < p.pairs ? cosines[tok[j] * p.pairs + pair(i)] : 1.f;
            n[i] = pair(i) < p.pairs ? sines[tok[j] * p.pairs + pair(i)] : 0.f;
          }
        }
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const uint64_t c2 = pack2(c[2 * i], c[2 * i + 1]), n2 = pack2(n[2 * i], n[2 * i + 1]);
          const uint64_t ra = fma2(fb[i], pack2(-n[2 * i], -n[2 * i + 1]), mul2(fa[i], c2));
          const uint64_t rb = fma2(fa[i], n2, mul2(fb[i], c2));
          if (WIDE) {
            fa[i] = ra;
            fb[i] = rb;
          } else {
            float v[2][2], o[2][2];
            unpack2(ra, v[0][0], v[0][1]);
            unpack2(rb, v[1][0], v[1][1]);
            unpack2(fa[i], o[0][0], o[0][1]);
            unpack2(fb[i], o[1][0], o[1][1]);
            const bool t0 = pair(2 * i) < p.pairs, t1 = pair(2 * i + 1) < p.pairs;
            fa[i] = pack2(t0 ? v[0][0] : o[0][0], t1 ? v[0][1] : o[0][1]);
            fb[i] = pack2(t0 ? v[1][0] : o[1][0], t1 ? v[1][1] : o[1][1]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < W; ++i) {
        float v[2][2];
        unpack2(fa[i], v[0][0], v[0][1]);
        unpack2(fb[i], v[1][0], v[1][1]);
        if (WIDE && INTER) {
          put2(ab[j][4 * i / V], 2 * i % W, v[0][0], v[1][0]);
          put2(ab[j][4 * i / V], (2 * i + 1) % W, v[0][1], v[1][1]);
        } else {
          put2(ab[j][0], i, v[0][0], v[0][1]);
          put2(ab[j][1], i, v[1][0], v[1][1]);
        }
      }
    }
    if (!on || !to[j]) continue;
    if (WIDE) {
      *reinterpret_cast<Vec<T, V>*>(to[j] + ia) = ab[j][0];
      *reinterpret_cast<Vec<T, V>*>(to[j] + ib) = ab[j][1];
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (pair(i) < half) {
          to[j][first(pair(i))] = ab[j][0].v[i];
          to[j][second(pair(i))] = ab[j][1].v[i];
        }
    }
  }
}

template <class T, bool WIDE, bool INTER, int GROUP, int J>
cudaError_t launch(QkParams p, cudaStream_t stream) {
  const int per = kThreads / GROUP * J;
  p.span = (per - 1) / p.heads.d + 2;
  const int64_t blocks = (p.items + per - 1) / per;
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  const size_t shared = (2 * (size_t)p.D + 2 * (size_t)p.span * p.pairs) * 4;
  return launch_after(qk_kernel<T, WIDE, INTER, GROUP, J>, dim3((unsigned)blocks), kThreads, shared, stream, 1, p);
}

// Two heads per group of lanes where that still gives every SM 8 blocks and the angles fit, else one: more blocks for
// few heads, whose latency counts.
template <class T, bool WIDE, bool INTER, int GROUP>
cudaError_t by_items(const QkParams& p, cudaStream_t stream, int sms) {
  constexpr int J = 2, per = kThreads / GROUP * J;
  const bool many = p.items >= (int64_t)sms * 8 * per && ((per - 1) / p.heads.d + 2) * (int64_t)p.pairs <= kAngles;
  return many ? launch<T, WIDE, INTER, GROUP, J>(p, stream) : launch<T, WIDE, INTER, GROUP, 1>(p, stream);
}

template <class T, bool INTER>
cudaError_t by_group(const QkParams& p, bool wide, cudaStream_t stream, int sms) {
  if (!wide) return by_items<T, false, INTER, 32>(p, stream, sms);
  const int lanes = p.D / 2 / kPairs<T, true>;
  if (lanes <= 4) return by_items<T, true, INTER, 4>(p, stream, sms);
  if (lanes <= 8) return by_items<T, true, INTER, 8>(p, stream, sms);
  if (lanes <= 16) return by_items<T, true, INTER, 16>(p, stream, sms);
  return by_items<T, true, INTER, 32>(p, stream, sms);
}

template <class T>
cudaError_t by_order(const QkParams& p, bool inter, bool wide, cudaStream_t stream, int sms) {
  return inter ? by_group<T, true>(p, wide, stream, sms) : by_group<T, false>(p, wide, stream, sms);
}

// A frequency in radians per position as a 64-bit fraction of a turn, to its last bit while it is below 2^40: 1 / 2 pi is the
// sum of two doubles here, and the product with the first is taken with its rounding error.  (One double would leave 2^-53
// of the frequency, which 2^31 positions make 2^-22 of it.)
uint64_t turn_of(double freq) {
  constexpr double hi = 0x1.45f306dc9c883p-3, lo = -0x1.6b01ec5417056p-57;
  const double f = std::fabs(freq), p = f * hi;
  double whole;
  const uint64_t first = (uint64_t)std::ldexp(std::modf(p, &whole), 64);
  double rest = std::fma(f, hi, -p) + f * lo;
  rest -= std::rint(rest);
  const uint64_t second = (uint64_t)std::rint(std::ldexp(std::fabs(rest), 64));
  const uint64_t turn = rest < 0 ? first - second : first + second;
  return freq < 0 ? 0 - turn : turn;
}

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

pp_status run(const pp_rope* rope, int dtype, QkParams& p, void* stream) {
  if (p.T == 0 || p.Hq + p.Hk + p.Hv == 0) return PP_OK;
  if ((int64_t)p.Hq + p.Hk + p.Hv > 65535) return PP_ERR_UNSUPPORTED;
  const size_t e = (size_t)dtype_size(dtype);
  const int n[3] = {p.Hq, p.Hk, p.Hv};
  const int W = 16 / (int)e;
  p.turn = rope->turn;
  p.axis = rope->axis;
  p.D = rope->D;
  p.inv_D = 1.f / (float)rope->D;
  p.items = (int64_t)p.T * (p.Hq + p.Hk + p.Hv);
  p.heads = FastDiv(p.Hq + p.Hk + p.Hv);
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
    const uint64_t turn = turn_of(freq[j]);
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
  if (cache->scales8[0]) return PP_ERR_UNSUPPORTED;
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
  p.log_page = log2_of(cache->page);
  p.H = cache->H;
  p.nslots = (int64_t)cache->pages * cache->page;
  p.eps = eps;
  return run(rope, cache->dtype, p, stream);
}

}  // extern "C"
