// Rotary positions with several axes, and appending to the paged cache with the rotation on the way.
//
//   angle(t, j) = sum_a pos[t][a] * freq[a][j]
//   (u, w) -> (u cos - w sin, w cos + u sin)   for the pairs j < pairs of a head; the other elements stay
//
// One kernel for both: a workgroup takes a few tokens' heads (queries, keys, values), loads them, forms each
// angle's cosine and sine once for all heads in LDS while those loads are in flight, and stores the turned heads to their
// tensor or to the cache's slot. Nothing of a head is stored before all of it is loaded, so a tensor may be turned in place.
// Bound by memory: every element is read once and written once, 16 bytes a lane (32768 tokens of 16 bf16 heads of 128 out of a packed
// projection: 50 us, 5.4 TB/s; keys and values of 16384 tokens, 4 heads of 64, and 8 of queries: 15 us, 4.5 TB/s); a few tokens are one
// launch's latency (3.8 us on the GPU). That is modes 0 and 1 (below), whose operands stay in registers. Modes 2 and 3 load the partners one by one and
// their builds keep the operands in scratch memory (296 bytes a thread), several times slower: the same 32768 tokens with 60 of 64 pairs 428 us (mode 2,
// fp32 with 62: 795), with rows that begin anywhere 1600 us (mode 3).
// Angles are summed and reduced to a turn in 64 bits (an fp32 product would be off by |angle| * 2^-24), the turn of an
// element in 32 bits, rounded once to the tensor's type.
#include "sc_attend_device.h"
#include "sc_stream.h"

#include <algorithm>

#pragma clang fp contract(off)

namespace sc {

namespace {

constexpr int kThreads = 256;

// Items (see below) a thread holds at once.
template <int MODE> struct Held { static constexpr int kItems = MODE == 0 || MODE == 2 ? 2 : 4; };

template <typename T, int MODE> struct Chunk { static constexpr int kElems = MODE == 3 ? 1 : 16 / (int)sizeof(T); };

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ void narrow(float v, float* o) { *o = v; }
__device__ __forceinline__ void narrow(float v, uint16_t* o) { *o = (uint16_t)(pack2(v, v) & 0xffffu); }

// An item is what one thread turns at a time:
//   MODE 0  two 16-byte chunks a pairing of halves apart (or two neighbours past the pairs)
//   MODE 1  a 16-byte chunk of whole neighbour pairs
//   MODE 2  a 16-byte chunk; the partners are loaded one by one (halves whose distance is no multiple of a chunk)
//   MODE 3  one element and its partner (any size, stride and alignment)
template <typename T, int MODE>
__global__ void __launch_bounds__(kThreads) rotate_kernel(RotateParams p) {
  constexpr int V = Chunk<T, MODE>::kElems, U = Held<MODE>::kItems;
  struct alignas(V * sizeof(T)) Vec { T e[V]; };
  extern __shared__ char lds[];
  floatx2* turn = reinterpret_cast<floatx2*>(lds);  // [token][pair]: cos, sin
  __shared__ int where[8][2];                       // [token]: page (-1: none), slot
  const int group = (int)blockIdx.x / p.head_groups, hg = (int)blockIdx.x - group * p.head_groups;
  const int t0 = group * p.tok_per_wg, h0 = hg * p.heads_per_wg;
  const int heads = p.heads[0] + p.heads[1] + p.heads[2];
  const int nh = min(p.heads_per_wg, heads - h0), nt = min(p.tok_per_wg, p.tokens - t0);
  const int chunks = p.dim / V, far = p.freq ? p.pairs / V : 0;  // MODE 0: chunks of half the pairs
  const int per_head = MODE == 0 ? far + (chunks - 2 * far + 1) / 2 : chunks;
  const int items = nt * nh * per_head;
  const float inv_head = 1.0f / (float)per_head, inv_nh = 1.0f / (float)nh;

  Vec a[U], b[U];
  T other[U][MODE == 2 || MODE == 3 ? V : 1];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int it = (int)threadIdx.x + u * kThreads;
    if (it >= items) break;
    const int row = qdiv(it, inv_head), j = it - row * per_head, tk = qdiv(row, inv_nh);
    int h = h0 + row - tk * nh, which = 0;
    if (h >= p.heads[0]) h -= p.heads[0], which = 1;
    if (which == 1 && h >= p.heads[1]) h -= p.heads[1], which = 2;
    const T* src = reinterpret_cast<const T*>(p.src[which]) + (int64_t)(t0 + tk) * p.src_token[which] + (int64_t)h * p.src_head[which];
    if constexpr (MODE == 0) {
      const int c0 = j < far ? j : 2 * j, c1 = j < far ? j + far : 2 * j + 1;  // past the pairs: 2 far + 2 (j - far)
      a[u] = *reinterpret_cast<const Vec*>(src + c0 * V);
      if (c1 < chunks) b[u] = *reinterpret_cast<const Vec*>(src + c1 * V);
    } else {
      a[u] = *reinterpret_cast<const Vec*>(src + j * V);
      if constexpr (MODE >= 2) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int e = j * V + i;
          if (p.freq && which < 2 && e < 2 * p.pairs)
            other[u][i] = src[p.adjacent ? e ^ 1 : e < p.pairs ? e + p.pairs : e - p.pairs];
        }
      }
    }
  }

  if (p.paged) {
    const int lane = threadIdx.x & 63;
    for (int tk = uniform((int)threadIdx.x >> 6); tk < nt; tk += kThreads / 64) {
      const int s = owner_of(p.cache.row_start, p.cache.batch, t0 + tk);
      int page = -1, slot = 0;
      if (s < p.cache.batch) {
        const Sequence q = sequence_of(p.cache, s);
        const int at = p.cache.kv_len[s] - q.n + (t0 + tk - q.start);
        page = -2;  // its queries turn, its keys and values have no place
        if (t0 + tk >= q.start && at >= 0 && page_of(p.cache, at) < p.cache.width) {
          const int i = page_of(p.cache, at), got = p.cache.table[(int64_t)s * p.cache.width + i];
          slot = at - i * p.cache.page_size;
          if (got >= 0 && got < p.cache.pages) page = got;
        }
      }
      if (lane == 0) where[tk][0] = page, where[tk][1] = slot;
    }
  }
  if (p.freq && h0 < p.heads[0] + p.heads[1]) {
    const float inv_pairs = 1.0f / (float)p.pairs;
    for (int i = threadIdx.x; i < nt * p.pairs; i += kThreads) {
      const int tk = qdiv(i, inv_pairs), j = i - tk * p.pairs;
      double angle = 0.0;
      for (int x = 0; x < p.axes; ++x)
        angle += (double)p.pos[(int64_t)(t0 + tk) * p.axes + x] * (double)p.freq[x * p.pairs + j];
      double turns = angle * 0.15915494309189533577;  // 1 / (2 pi)
      turns -= rint(turns);
      float s, c;
      sincospif(2.0f * (float)turns, &s, &c);
      turn[i] = floatx2{c, p.sign * s};
    }
  }
  __syncthreads();

#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int it = (int)threadIdx.x + u * kThreads;
    if (it >= items) break;
    const int row = qdiv(it, inv_head), j = it - row * per_head, tk = qdiv(row, inv_nh);
    int h = h0 + row - tk * nh, which = 0;
    if (h >= p.heads[0]) h -= p.heads[0], which = 1;
    if (which == 1 && h >= p.heads[1]) h -= p.heads[1], which = 2;
    T* dst;
    if (which == 0) {
      if (p.paged && where[tk][0] == -1) continue;
      dst = reinterpret_cast<T*>(p.dst) + (int64_t)(t0 + tk) * p.dst_token + (int64_t)h * p.dst_head;
    } else {
      const int page = where[tk][0], slot = where[tk][1];
      if (page < 0) continue;
      dst = which == 1 ? reinterpret_cast<T*>(p.cache.k) + page * p.cache.k_page + h * p.cache.k_head + slot * p.cache.k_slot
                       : reinterpret_cast<T*>(p.cache.v) + page * p.cache.v_page + h * p.cache.v_head + slot * p.cache.v_slot;
    }
    const bool turns = p.freq && which < 2;
    const floatx2* tt = turn + tk * p.pairs;
    if constexpr (MODE == 0) {
      const int c0 = j < far ? j : 2 * j, c1 = j < far ? j + far : 2 * j + 1;
      if (turns && j < far) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const floatx2 cs = tt[j * V + i];
          const float x = widen(a[u].e[i]), y = widen(b[u].e[i]);
          narrow(x * cs.x - y * cs.y, &a[u].e[i]);
          narrow(y * cs.x + x * cs.y, &b[u].e[i]);
        }
      }
      *reinterpret_cast<Vec*>(dst + c0 * V) = a[u];
      if (c1 < chunks) *reinterpret_cast<Vec*>(dst + c1 * V) = b[u];
    } else if constexpr (MODE == 1) {
      if (turns) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
          const int pair = (j * V + i) >> 1;
          if (pair < p.pairs) {
            const floatx2 cs = tt[pair];
            const float x = widen(a[u].e[i]), y = widen(a[u].e[i + 1]);
            narrow(x * cs.x - y * cs.y, &a[u].e[i]);
            narrow(y * cs.x + x * cs.y, &a[u].e[i + 1]);
          }
        }
      }
      *reinterpret_cast<Vec*>(dst + j * V) = a[u];
    } else {
      if (turns) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int e = j * V + i;
          if (e < 2 * p.pairs) {
            const int pair = p.adjacent ? e >> 1 : e < p.pairs ? e : e - p.pairs;
            const bool second = p.adjacent ? (e & 1) != 0 : e >= p.pairs;
            const floatx2 cs = tt[pair];
            const float x = widen(a[u].e[i]), y = widen(other[u][i]);
            narrow(second ? x * cs.x + y * cs.y : x * cs.x - y * cs.y, &a[u].e[i]);
          }
        }
      }
      *reinterpret_cast<Vec*>(dst + j * V) = a[u];
    }
  }
}

template <typename T, int MODE>
hipError_t launch(RotateParams p, hipStream_t stream) {
  constexpr int V = Chunk<T, MODE>::kElems, cap = kThreads * Held<MODE>::kItems;
  const int chunks = p.dim / V, far = p.freq ? p.pairs / V : 0;
  const int per_head = MODE == 0 ? far + (chunks - 2 * far + 1) / 2 : chunks;
  const int heads = p.heads[0] + p.heads[1] + p.heads[2];
  // Whole tokens where they fit (their angles are then formed once), up to eight of them, but fewer a workgroup while
  // the launch has under 1024 workgroups (four a compute unit).
  p.heads_per_wg = std::min(heads, cap / per_head);
  p.head_groups = (heads + p.heads_per_wg - 1) / p.heads_per_wg;
  p.tok_per_wg = p.head_groups > 1 ? 1 : std::min(8, cap / (heads * per_head));
  while (p.tok_per_wg > 1 && (int64_t)(p.tokens + p.tok_per_wg - 1) / p.tok_per_wg < 1024) --p.tok_per_wg;
  const int64_t grid = (int64_t)((p.tokens + p.tok_per_wg - 1) / p.tok_per_wg) * p.head_groups;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  const size_t lds = p.freq ? (size_t)p.tok_per_wg * p.pairs * sizeof(floatx2) : 0;
  rotate_kernel<T, MODE><<<dim3((unsigned)grid), dim3(kThreads), lds, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RotateParams& p, int dtype, int mode, hipStream_t stream) {
  if (dtype == 0) {
    switch (mode) {
      case 0: return launch<float, 0>(p, stream);
      case 1: return launch<float, 1>(p, stream);
      case 2: return launch<float, 2>(p, stream);
      default: return launch<float, 3>(p, stream);
    }
  }
  switch (mode) {
    case 0: return launch<uint16_t, 0>(p, stream);
    case 1: return launch<uint16_t, 1>(p, stream);
    case 2: return launch<uint16_t, 2>(p, stream);
    default: return launch<uint16_t, 3>(p, stream);
  }
}

}  // namespace sc
