// Token embedding of M replicas and its gradient.
//
//   y_t = scale E[token_t],   dE[v] = scale sum_{t: token_t = v} dy_t
//
// Both are bound by memory: forward reads a row of the table and writes one of Y a token, backward reads dY and writes dE once.
// The gradient's sums must not depend on the order of atomics, so the tokens are sorted (stable, so that a token's places are in
// order) and every row of dE is summed by one group of threads, or, where a token's places cross from one run of the sorted
// list to the next, from the runs' partial sums in order.  8 x 16384 tokens, 50000 rows of 768, bf16: 68 us forward, 266 backward (5.1 and
// 5.4 TB/s of what has to move).  Rows that are not whole 16-byte pieces are taken in single elements: 4 x 16384 tokens, 50000 rows of
// 766 for 768, bf16 149 us for 35 forward and 325 for 153 backward, fp32 148 for 53 and 328 for 172.
#include "abs_pipeline.cuh"

namespace absk {
namespace {

constexpr int kEmbThreads = 256;
constexpr int kRadixBits = 9, kBinsR = 1 << kRadixBits;
constexpr int kKeysPerThread = 8, kTileKeys = kEmbThreads * kKeysPerThread;      // keys of a CTA in a sorting pass
constexpr int kSmallKeys = 4096;               // as many are sorted by one CTA in one launch
constexpr int kZeroRows = 128;                 // rows of the table that a CTA looks after

struct Embedding {
  const float* E;
  long long e_rs, e_ws;
  const int* tokens;
  long long t_ws;
  void* Y;
  long long y_rs, y_ws;
  long long rows;
  int M, vocab, d;
  float scale;
};
struct EmbeddingGrad {
  const void* dY;
  long long dy_rs, dy_ws;
  const int* tokens;
  long long t_ws;
  float* dE;
  long long e_rs, e_ws;
  int rows, M, vocab, d, accumulate;
  float scale;
  unsigned* key[2];              // [M][rows]
  unsigned* pos[2];
  unsigned* hist;                // [M][kBinsR][tiles]
  int tiles;
  float* part;                   // [M][runs][2][d]
  int runs, run;                 // runs of `run` sorted tokens each
  int sorted;                    // which of the two buffers
};

template <typename T, int V> struct EmbPiece;
template <> struct EmbPiece<float, 4> { typedef uint4 Raw; };
template <> struct EmbPiece<float, 1> { typedef uint32_t Raw; };
template <> struct EmbPiece<__nv_bfloat16, 8> { typedef uint4 Raw; };
template <> struct EmbPiece<__nv_bfloat16, 1> { typedef unsigned short Raw; };

template <typename T, int V>
__device__ __forceinline__ void widen(const typename EmbPiece<T, V>::Raw& r, float (&x)[V]) {
  if constexpr (V == 1) {
    if constexpr (sizeof(T) == 4) x[0] = __uint_as_float(r);
    else x[0] = __uint_as_float(static_cast<uint32_t>(r) << 16);
  } else {
    Vec<T>::unpack(r, x);
  }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T, int V>
__device__ __forceinline__ typename EmbPiece<T, V>::Raw narrow(const float (&x)[V]) {
  if constexpr (V == 1) {
    if constexpr (sizeof(T) == 4) return __float_as_uint(x[0]);
    else return __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
  } else if constexpr (sizeof(T) == 4) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  } else {
    return make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
  }
}
template <int V>
__device__ __forceinline__ void load_row(const float* p, float (&x)[V]) {
  if constexpr (V == 1) {
    x[0] = __ldg(p);
  } else {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const float4 f = __ldg(reinterpret_cast<const float4*>(p + e));
      x[e] = f.x; x[e + 1] = f.y; x[e + 2] = f.z; x[e + 3] = f.w;
    }
  }
}

// A thread has one piece of V elements of kUnroll rows, whose loads all go before the first store.  (8 x 16384 tokens, 50000 rows of 768, bf16:
// 68 us; two rows 79, eight 78, all tokens' numbers before the first row 74.)
template <typename T, int V>
__global__ void __launch_bounds__(kEmbThreads)
embedding_kernel(const Embedding a, int pieces, long long work) {
  constexpr int kUnroll = 4;
  pdl_wait();
  const long long total = a.rows * a.M;
  for (long long i = static_cast<long long>(blockIdx.x) * kEmbThreads + threadIdx.x; i < work;
       i += static_cast<long long>(gridDim.x) * kEmbThreads) {
    const long long block = i / pieces;
    const int c = static_cast<int>(i - block * pieces) * V;
    float x[kUnroll][V];
    long long m = block * kUnroll / a.rows, r = block * kUnroll - m * a.rows, at[kUnroll];
    int token[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      at[u] = -1;
      token[u] = -1;
      if (block * kUnroll + u < total) {
        at[u] = m * a.y_ws + r * a.y_rs + c;
        token[u] = __ldg(a.tokens + m * a.t_ws + r);
        if (token[u] >= a.vocab) token[u] = -1;
        if (token[u] >= 0) load_row<V>(a.E + m * a.e_ws + token[u] * a.e_rs + c, x[u]);
      }
      if (++r == a.rows) {
        r = 0;
        ++m;
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (at[u] < 0) continue;
#pragma unroll
      for (int e = 0; e < V; ++e) x[u][e] = token[u] < 0 ? 0.f : x[u][e] * a.scale;
      __stcs(reinterpret_cast<typename EmbPiece<T, V>::Raw*>(static_cast<T*>(a.Y) + at[u]), narrow<T, V>(x[u]));
    }
  }
}

// ---- sorting ---------------------------------------------------------------------------------------
// Keys are tokens, those outside the table the number behind its last row.  Passes over kRadixBits bits from the lowest on, each
// stable.  A tile's keys keep their order: warp w has the keys 32 (w kKeysPerThread + i) + lane.
__device__ __forceinline__ unsigned token_key(const EmbeddingGrad& a, int m, int i) {
  const int t = __ldg(a.tokens + m * a.t_ws + i);
  return t < 0 || t >= a.vocab ? static_cast<unsigned>(a.vocab) : static_cast<unsigned>(t);
}

// Counts of the digit's values in a tile.
__global__ void __launch_bounds__(kEmbThreads)
emb_count_kernel(const EmbeddingGrad a, int pass) {
  __shared__ unsigned h[kBinsR];
  const int m = blockIdx.y, tile = blockIdx.x;
  for (int b = threadIdx.x; b < kBinsR; b += kEmbThreads) h[b] = 0;
  pdl_wait();
  __syncthreads();
  const unsigned* keys = a.key[(pass + 1) & 1] + static_cast<long long>(m) * a.rows;      // what the pass before wrote
#pragma unroll
  for (int k = 0; k < kKeysPerThread; ++k) {
    const int i = tile * kTileKeys + k * kEmbThreads + threadIdx.x;
    if (i < a.rows) {
      const unsigned key = pass == 0 ? token_key(a, m, i) : keys[i];
      atomicAdd(h + ((key >> (pass * kRadixBits)) & (kBinsR - 1)), 1u);
    }
  }
  __syncthreads();
  for (int b = threadIdx.x; b < kBinsR; b += kEmbThreads) a.hist[(static_cast<long long>(m) * kBinsR + b) * a.tiles + tile] = h[b];
}

// Exclusive sums over values and tiles of one replica.
__global__ void __launch_bounds__(1024)
emb_scan_kernel(const EmbeddingGrad a) {
  __shared__ unsigned red[32];
  unsigned* h = a.hist + static_cast<long long>(blockIdx.x) * kBinsR * a.tiles;
  const long long n = static_cast<long long>(kBinsR) * a.tiles;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  unsigned carry = 0;
  for (long long at = 0; at < n; at += 4096) {
    unsigned v[4], s = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const long long i = at + 4 * threadIdx.x + e;
      v[e] = i < n ? h[i] : 0u;
      s += v[e];
    }
    unsigned x = s;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const unsigned o = __shfl_up_sync(0xffffffffu, x, off);
      if (lane >= off) x += o;
    }
    __syncthreads();
    if (lane == 31) red[warp] = x;
    __syncthreads();
    unsigned before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 32; ++w) {
      if (w < warp) before += red[w];
      all += red[w];
    }
    before += carry + x - s;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const long long i = at + 4 * threadIdx.x + e;
      if (i < n) h[i] = before;
      before += v[e];
    }
    carry += all;
  }
}

// The lanes with the same value of the digit as this one; lanes without a key have values of their own.
__device__ __forceinline__ unsigned same_digit(unsigned digit) { return __match_any_sync(0xffffffffu, digit); }

// A tile's keys, `each` a thread, to their places.  counts: [warps][kBinsR], zero.
__device__ __forceinline__ void place_keys(unsigned short* counts, const unsigned (&digit)[kKeysPerThread], const bool (&live)[kKeysPerThread],
                                           unsigned (&rank)[kKeysPerThread], int each = kKeysPerThread) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned short* mine = counts + warp * kBinsR;
#pragma unroll
  for (int k = 0; k < kKeysPerThread; ++k) {
    if (k >= each) break;
    const unsigned peers = same_digit(live[k] ? digit[k] : kBinsR + lane);
    const unsigned before = __popc(peers & ((1u << lane) - 1u));
    if (live[k]) rank[k] = mine[digit[k]] + before;
    __syncwarp();
    if (live[k] && before == 0) mine[digit[k]] = static_cast<unsigned short>(mine[digit[k]] + __popc(peers));
    __syncwarp();
  }
}

__global__ void __launch_bounds__(kEmbThreads)
emb_scatter_kernel(const EmbeddingGrad a, int pass) {
  __shared__ unsigned short counts[kEmbThreads / 32][kBinsR];
  const int m = blockIdx.y, tile = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int b = threadIdx.x; b < kBinsR * (kEmbThreads / 32); b += kEmbThreads) (&counts[0][0])[b] = 0;
  pdl_wait();
  __syncthreads();
  const long long base = static_cast<long long>(m) * a.rows;
  const unsigned *keys = a.key[(pass + 1) & 1] + base, *from = a.pos[(pass + 1) & 1] + base;
  unsigned key[kKeysPerThread], pos[kKeysPerThread], digit[kKeysPerThread], rank[kKeysPerThread];
  bool live[kKeysPerThread];
#pragma unroll
  for (int k = 0; k < kKeysPerThread; ++k) {
    const int i = tile * kTileKeys + 32 * (warp * kKeysPerThread + k) + lane;
    live[k] = i < a.rows;
    key[k] = pos[k] = 0;
    if (live[k]) {
      key[k] = pass == 0 ? token_key(a, m, i) : keys[i];
      pos[k] = pass == 0 ? static_cast<unsigned>(i) : from[i];
    }
    digit[k] = (key[k] >> (pass * kRadixBits)) & (kBinsR - 1);
  }
  place_keys(&counts[0][0], digit, live, rank);
  __syncthreads();
  for (int b = threadIdx.x; b < kBinsR; b += kEmbThreads) {            // counts of the warps before
    unsigned s = 0;
#pragma unroll
    for (int w = 0; w < kEmbThreads / 32; ++w) {
      const unsigned c = counts[w][b];
      counts[w][b] = static_cast<unsigned short>(s);
      s += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kKeysPerThread; ++k) {
    if (!live[k]) continue;
    const long long to = base + a.hist[(static_cast<long long>(m) * kBinsR + digit[k]) * a.tiles + tile] + counts[warp][digit[k]] + rank[k];
    a.key[pass & 1][to] = key[k];
    a.pos[pass & 1][to] = pos[k];
  }
}

// Few keys: all passes of a replica in one CTA, keys and places in shared memory.
constexpr int kSmallThreads = 512;
__global__ void __launch_bounds__(kSmallThreads)
emb_sort_small_kernel(const EmbeddingGrad a, int passes) {
  static_assert(kSmallKeys == kSmallThreads * kKeysPerThread, "");
  __shared__ unsigned keys[kSmallKeys];
  __shared__ unsigned short places[kSmallKeys], counts[kSmallThreads / 32][kBinsR];
  __shared__ unsigned red[kSmallThreads / 32];
  static_assert(kBinsR == kSmallThreads, "a thread a value");
  const int m = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  unsigned key[kKeysPerThread], pos[kKeysPerThread], digit[kKeysPerThread], rank[kKeysPerThread];
  bool live[kKeysPerThread];
  const int each = (a.rows + kSmallThreads - 1) / kSmallThreads;
  for (int pass = 0; pass < passes; ++pass) {
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
      const int i = 32 * (warp * each + k) + lane;
      live[k] = k < each && i < a.rows;
      key[k] = pos[k] = 0;
      if (live[k]) {
        key[k] = pass == 0 ? token_key(a, m, i) : keys[i];
        pos[k] = pass == 0 ? static_cast<unsigned>(i) : places[i];
      }
      digit[k] = (key[k] >> (pass * kRadixBits)) & (kBinsR - 1);
    }
    for (int b = threadIdx.x; b < kBinsR * (kSmallThreads / 32); b += kSmallThreads) (&counts[0][0])[b] = 0;
    __syncthreads();
    place_keys(&counts[0][0], digit, live, rank, each);
    __syncthreads();
    unsigned s = 0;                                // thread b: value b's keys in all, then in the values before
#pragma unroll
    for (int w = 0; w < kSmallThreads / 32; ++w) {
      const unsigned c = counts[w][threadIdx.x];
      counts[w][threadIdx.x] = static_cast<unsigned short>(s);
      s += c;
    }
    unsigned x = s;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const unsigned o = __shfl_up_sync(0xffffffffu, x, off);
      if (lane >= off) x += o;
    }
    if (lane == 31) red[warp] = x;
    __syncthreads();
    unsigned before = x - s;
    for (int w = 0; w < warp; ++w) before += red[w];
#pragma unroll
    for (int w = 0; w < kSmallThreads / 32; ++w) counts[w][threadIdx.x] = static_cast<unsigned short>(counts[w][threadIdx.x] + before);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kKeysPerThread; ++k) {
      if (!live[k]) continue;
      const unsigned to = counts[warp][digit[k]] + rank[k];
      keys[to] = key[k];
      places[to] = static_cast<unsigned short>(pos[k]);
    }
    __syncthreads();
  }
  const long long base = static_cast<long long>(m) * a.rows;
  for (int i = threadIdx.x; i < a.rows; i += kSmallThreads) {
    a.key[a.sorted][base + i] = keys[i];
    a.pos[a.sorted][base + i] = places[i];
  }
}

// ---- the sums ----------------------------------------------------------------------------------------
template <int V>
__device__ __forceinline__ void store_sum(const EmbeddingGrad& a, float* p, const float (&x)[V]) {
  if constexpr (V == 1) {
    *p = a.accumulate ? *p + x[0] : x[0];
  } else {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      float4* q = reinterpret_cast<float4*>(p + e);
      float4 f = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
      if (a.accumulate) {
        const float4 o = *q;
        f.x += o.x; f.y += o.y; f.z += o.z; f.w += o.w;
      }
      *q = f;
    }
  }
}

// CTAs of blockIdx.x < sum_ctas: a group of `width` threads has a run of sorted tokens and a piece of V columns a thread
// (blockIdx.y: further columns).  A token whose places all lie within the run is written; the first and the last one of a run,
// where they go on beyond it, leave their sums in part[run][0] and [1] (one that fills the run and more: in [0]).
// The other CTAs write zeros into the rows of tokens that do not occur.
template <typename T, int V>
__global__ void __launch_bounds__(kEmbThreads)
emb_sum_kernel(const EmbeddingGrad a, int width, int pieces, int sum_ctas) {
  typedef typename EmbPiece<T, V>::Raw Raw;
  __shared__ unsigned char present[kZeroRows];
  pdl_wait();
  const int groups = blockDim.x / width;
  if (static_cast<int>(blockIdx.x) < sum_ctas) {
    const int group = threadIdx.x / width;
    const long long job = static_cast<long long>(blockIdx.x) * groups + group;
    if (group >= groups || job >= static_cast<long long>(a.M) * a.runs) return;
    const int m = static_cast<int>(job / a.runs), run = static_cast<int>(job - static_cast<long long>(m) * a.runs);
    const long long base = static_cast<long long>(m) * a.rows;
    const unsigned *keys = a.key[a.sorted] + base, *places = a.pos[a.sorted] + base;
    const int first = run * a.run, end = min(first + a.run, a.rows);
    const unsigned none = static_cast<unsigned>(a.vocab);
    // (one turn, but for rows of more than 65535 blocks of columns)
    for (int piece = blockIdx.y * width + threadIdx.x - group * width; piece < pieces; piece += gridDim.y * width) {
      const int c = piece * V;
      const T* dy = static_cast<const T*>(a.dY) + m * a.dy_ws + c;
      float* de = a.dE + m * a.e_ws + c;
      float* part = a.part + job * 2 * a.d + c;
      unsigned now = keys[first];
      bool open = first > 0 && keys[first - 1] == now;      // the token began in a run before
      float sum[V];
#pragma unroll
      for (int e = 0; e < V; ++e) sum[e] = 0.f;
      // kDeep rows at a time; the next ones' numbers are on their way while these are (8 x 16384 tokens: 2, 3, 4, 8 rows 275, 270, 267,
      // 316 us, without looking ahead 283)
      constexpr int kDeep = 4;
      unsigned next[kDeep], place[kDeep];
      auto look = [&](int i) {
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
          const bool in = i + u < end;
          next[u] = in ? keys[i + u] : none;
          place[u] = in ? places[i + u] : 0u;
        }
      };
      look(first);
      for (int i = first; i < end && now != none; i += kDeep) {
        Raw raw[kDeep];
        unsigned k[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
          k[u] = next[u];
          if (k[u] != none) raw[u] = __ldcs(reinterpret_cast<const Raw*>(dy + static_cast<long long>(place[u]) * a.dy_rs));
        }
        look(i + kDeep);
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
          if (i + u >= end) continue;
          if (k[u] != now) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              if (!open) sum[e] *= a.scale;
            }
            if (open) {
#pragma unroll
              for (int e = 0; e < V; ++e) part[e] = sum[e];
            } else if (now != none) {
              store_sum<V>(a, de + now * a.e_rs, sum);
            }
            open = false;
            now = k[u];
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] = 0.f;
          }
          if (k[u] != none) {
            float x[V];
            widen<T, V>(raw[u], x);
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += x[e];
          }
        }
      }
      if (now == none) continue;
      const bool on = end < a.rows && keys[end] == now;     // the token goes on in the next run
      if (open || on) {
        float* p = open ? part : part + a.d;
#pragma unroll
        for (int e = 0; e < V; ++e) p[e] = sum[e];
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] *= a.scale;
        store_sum<V>(a, de + now * a.e_rs, sum);
      }
    }
    return;
  }
  if (blockIdx.y > 0) return;
  const int per = (a.vocab + kZeroRows - 1) / kZeroRows;
  const int z = static_cast<int>(blockIdx.x) - sum_ctas, m = z / per, v0 = (z - m * per) * kZeroRows;
  const int v1 = min(v0 + kZeroRows, a.vocab);
  for (int i = threadIdx.x; i < kZeroRows; i += blockDim.x) present[i] = 0;
  const unsigned* keys = a.key[a.sorted] + static_cast<long long>(m) * a.rows;
  // a row's first place in the sorted list: one search a thread, every row its own
  __syncthreads();
  for (int v = v0 + threadIdx.x; v < v1; v += blockDim.x) {
    int lo = 0, hi = a.rows;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (keys[mid] < static_cast<unsigned>(v)) lo = mid + 1;
      else hi = mid;
    }
    present[v - v0] = lo < a.rows && keys[lo] == static_cast<unsigned>(v);
  }
  __syncthreads();
  const unsigned wide = V == 1 ? 1 : 4, count = a.d / wide;        // (up to 2^31 elements)
  for (unsigned i = threadIdx.x; i < (v1 - v0) * count; i += blockDim.x) {
    const unsigned r = i / count, c = (i - r * count) * wide;
    if (present[r]) continue;
    float* p = a.dE + m * a.e_ws + static_cast<long long>(v0 + r) * a.e_rs + c;
    if (wide == 4) __stcs(reinterpret_cast<float4*>(p), make_float4(0.f, 0.f, 0.f, 0.f));
    else *p = 0.f;
  }
}

// Tokens that cross from one run to the next: the run where one starts adds up what the runs left, in order.
template <int V>
__global__ void __launch_bounds__(kEmbThreads)
emb_join_kernel(const EmbeddingGrad a, int width, int pieces) {
  pdl_wait();
  const int groups = blockDim.x / width, group = threadIdx.x / width;
  const long long job = static_cast<long long>(blockIdx.x) * groups + group;
  if (group >= groups || job >= static_cast<long long>(a.M) * a.runs) return;
  const int m = static_cast<int>(job / a.runs), run = static_cast<int>(job - static_cast<long long>(m) * a.runs);
  const unsigned* keys = a.key[a.sorted] + static_cast<long long>(m) * a.rows;
  const int first = run * a.run, end = min(first + a.run, a.rows);
  if (end >= a.rows) return;
  const unsigned now = keys[end - 1];
  if (now == static_cast<unsigned>(a.vocab) || keys[end] != now) return;               // does not go on
  if (first > 0 && keys[first] == now && keys[first - 1] == now) return;                // did not start here
  for (int piece = blockIdx.y * width + threadIdx.x - group * width; piece < pieces; piece += gridDim.y * width) {
    const int c = piece * V;
    // the last run with the token: every run in between holds nothing else
    const float* part = a.part + job * 2 * a.d + c;
    float sum[V];
    load_row<V>(part + a.d, sum);
    part += 2 * a.d;
    // (four runs at a time: a frequent token's are a long chain; what is loaded of runs that do not have it is not looked at)
    bool on = true;
    for (int r = run + 1; on && r < a.runs; r += 4, part += 8 * a.d) {
      float x[4][V];
      bool has[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        has[u] = r + u < a.runs && keys[(r + u) * a.run] == now;
        if (r + u < a.runs) load_row<V>(part + u * 2 * a.d, x[u]);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        on = on && has[u];
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] = on ? sum[e] + x[u][e] : sum[e];
      }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] *= a.scale;
    store_sum<V>(a, a.dE + m * a.e_ws + c + now * a.e_rs, sum);
  }
}

struct DeviceGuardEmb {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuardEmb(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
    if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    if (prev == dev) prev = -1;
  }
  ~DeviceGuardEmb() { if (prev >= 0) cudaSetDevice(prev); }
};

int validate_shape_emb(abs_ctx* ctx, int M, long long rows, long long vocab, long long d) {
  if (M < 1 || rows < 0 || vocab < 1 || d < 1)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "need M >= 1, rows >= 0, vocab >= 1 and d >= 1 (M=%d rows=%lld vocab=%lld d=%lld)", M, rows,
                     vocab, d);
  if (M > 65535 || rows > (1ll << 28) || vocab >= (1 << 24) || d > (1 << 24) || rows * M > (1ll << 31) || vocab * M > (1ll << 36))
    return set_error(ctx, ABS_ERR_UNSUPPORTED,
                     "M <= 65535, rows <= 2^28, vocab < 2^24, d <= 2^24, M * rows <= 2^31 and M * vocab <= 2^36 (M=%d rows=%lld vocab=%lld d=%lld)", M, rows, vocab, d);
  return ABS_OK;
}
int validate_matrix(abs_ctx* ctx, const char* what, int M, long long rows, long long d, long long rs, long long ws, bool shared) {
  if (rs < d) return set_error(ctx, ABS_ERR_INVALID_ARG, "%s: row_stride %lld < d %lld", what, rs, d);
  if (M > 1 && !(shared && ws == 0) && ws < (rows - 1) * rs + d)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "%s: worker_stride %lld overlaps the previous worker", what, ws);
  return ABS_OK;
}
unsigned long long bits_of(const void* p, int es, int M, long long rs, long long ws) {
  return reinterpret_cast<uintptr_t>(p) | static_cast<unsigned long long>(rs) * es | (M > 1 ? static_cast<unsigned long long>(ws) * es : 0);
}

int key_passes(long long vocab) {
  int bits = 1;
  while ((vocab >> bits) > 0) ++bits;              // keys go up to vocab
  return (bits + kRadixBits - 1) / kRadixBits;
}
// Runs of 32 tokens, longer ones where a frequent token would cross hundreds of them, shorter ones (down to 8) where they would be
// fewer than a few an SM.
int run_length(int M, long long rows) {
  long long r = 8;
  while (r < 32 && M * rows / r > 4 * kSmCountFallback) r *= 2;
  while (r < 1024 && rows / r > 2048) r *= 2;
  return static_cast<int>(r);
}
struct EmbScratch {
  size_t key[2], pos[2], hist, part, bytes;
  int tiles, runs, run;
};
EmbScratch emb_scratch(int M, long long rows, long long d) {
  EmbScratch s;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t r = at;
    at = (at + bytes + 255) & ~static_cast<size_t>(255);
    return r;
  };
  const size_t n = static_cast<size_t>(M) * rows * sizeof(unsigned);
  s.run = run_length(M, rows);
  s.runs = static_cast<int>((rows + s.run - 1) / s.run);
  s.tiles = static_cast<int>((rows + kTileKeys - 1) / kTileKeys);
  const bool small = rows <= kSmallKeys;
  s.key[0] = take(n);
  s.key[1] = small ? s.key[0] : take(n);
  s.pos[0] = take(n);
  s.pos[1] = small ? s.pos[0] : take(n);
  s.hist = take(small ? 0 : static_cast<size_t>(M) * kBinsR * s.tiles * sizeof(unsigned));
  s.part = take(static_cast<size_t>(M) * s.runs * 2 * d * sizeof(float));
  s.bytes = at;
  return s;
}

template <typename T, int V>
int run_embedding(abs_ctx* ctx, const Embedding& a, cudaStream_t st) {
  const int pieces = a.d / V;
  const long long work = (a.rows * a.M + 3) / 4 * pieces;
  long long grid = (work + kEmbThreads - 1) / kEmbThreads;
  const long long most = static_cast<long long>(ctx->sm_count) * 256;
  if (grid > most) grid = most;
  ABS_CUDA_TRY(ctx, launch_dependent(embedding_kernel<T, V>, dim3(static_cast<unsigned>(grid)), dim3(kEmbThreads), 0, st, a, pieces, work));
  return ABS_OK;
}
template <typename T, int V>
int run_sums(abs_ctx* ctx, const EmbeddingGrad& a, cudaStream_t st) {
  const int pieces = a.d / V, width = pieces < kEmbThreads ? pieces : kEmbThreads, groups = kEmbThreads / width;
  const int blocks = (pieces + width - 1) / width, cols = blocks < 65535 ? blocks : 65535;       // (the grid's second dimension)
  const int sum_ctas = static_cast<int>((static_cast<long long>(a.M) * a.runs + groups - 1) / groups);
  const int zero_ctas = a.accumulate ? 0 : a.M * ((a.vocab + kZeroRows - 1) / kZeroRows);
  if (sum_ctas + zero_ctas == 0) return ABS_OK;
  ABS_CUDA_TRY(ctx, launch_dependent(emb_sum_kernel<T, V>, dim3(sum_ctas + zero_ctas, cols), dim3(width * groups), 0, st, a, width, pieces,
                                     sum_ctas));
  if (a.runs > 1)
    ABS_CUDA_TRY(ctx, launch_dependent(emb_join_kernel<V>, dim3(sum_ctas, cols), dim3(width * groups), 0, st, a, width, pieces));
  return ABS_OK;
}

}  // namespace
}  // namespace absk

using namespace absk;

extern "C" int abs_embedding(abs_ctx* ctx, const float* E, int M, long long vocab, long long d, long long e_row_stride,
                             long long e_worker_stride, const int* tokens, long long tokens_stride, long long rows, float scale, void* Y,
                             abs_dtype y_dtype, long long y_row_stride, long long y_worker_stride, void* stream) {
  if (ctx == nullptr) return ABS_ERR_INVALID_ARG;
  if (y_dtype != ABS_F32 && y_dtype != ABS_BF16) return set_error(ctx, ABS_ERR_INVALID_ARG, "unknown dtype %d", (int)y_dtype);
  int rc = validate_shape_emb(ctx, M, rows, vocab, d);
  if (rc != ABS_OK || rows == 0) return rc;
  if (E == nullptr || tokens == nullptr || Y == nullptr) return set_error(ctx, ABS_ERR_INVALID_ARG, "E, tokens or Y is null");
  if ((rc = validate_matrix(ctx, "E", M, vocab, d, e_row_stride, e_worker_stride, true)) != ABS_OK) return rc;
  if ((rc = validate_matrix(ctx, "Y", M, rows, d, y_row_stride, y_worker_stride, false)) != ABS_OK) return rc;
  if (M > 1 && tokens_stride != 0 && tokens_stride < rows)
    return set_error(ctx, ABS_ERR_INVALID_ARG, "tokens_stride %lld < rows %lld", tokens_stride, rows);
  DeviceGuardEmb guard(ctx->device);
  if (!guard.ok) return set_error(ctx, ABS_ERR_CUDA, "cannot select device %d", ctx->device);
  const Embedding a{E, e_row_stride, e_worker_stride, tokens, tokens_stride, Y, y_row_stride, y_worker_stride, rows, M,
                    static_cast<int>(vocab), static_cast<int>(d), scale};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int es = y_dtype == ABS_F32 ? 4 : 2;
  const bool wide = ((bits_of(E, 4, M, e_row_stride, e_worker_stride) | bits_of(Y, es, M, y_row_stride, y_worker_stride) |
                      static_cast<unsigned long long>(d) * es) & 15u) == 0;
  if (y_dtype == ABS_F32) return wide ? run_embedding<float, 4>(ctx, a, st) : run_embedding<float, 1>(ctx, a, st);
  return wide ? run_embedding<__nv_bfloat16, 8>(ctx, a, st) : run_embedding<__nv_bfloat16, 1>(ctx, a, st);
}

extern "C" int abs_embedding_scratch_bytes(int M, long long rows, long long vocab, long long d, size_t* out) {
  if (out == nullptr) return set_error(nullptr, ABS_ERR_INVALID_ARG, "out is null");
  const int rc = validate_shape_emb(nullptr, M, rows, vocab, d);
  if (rc != ABS_OK) return rc;
  *out = emb_scratch(M, rows, d).bytes;
  return ABS_OK;
}

extern "C" int abs_embedding_backward(abs_ctx* ctx, const void* dY, abs_dtype dtype, int M, long long rows, long long d,
                                      long long dy_row_stride, long long dy_worker_stride, const int* tokens, long long tokens_stride,
                                      long long vocab, float scale, float* dE, long long e_row_stride, long long e_worker_stride,
                                      int accumulate, void* scratch, size_t scratch_bytes, void* stream) {
  if (ctx == nullptr) return ABS_ERR_INVALID_ARG;
  if (dtype != ABS_F32 && dtype != ABS_BF16) return set_error(ctx, ABS_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  int rc = validate_shape_emb(ctx, M, rows, vocab, d);
  if (rc != ABS_OK) return rc;
  if (dE == nullptr) return set_error(ctx, ABS_ERR_INVALID_ARG, "dE is null");
  if ((rc = validate_matrix(ctx, "dE", M, vocab, d, e_row_stride, e_worker_stride, false)) != ABS_OK) return rc;
  const EmbScratch s = emb_scratch(M, rows, d);
  if (rows > 0) {
    if (dY == nullptr || tokens == nullptr) return set_error(ctx, ABS_ERR_INVALID_ARG, "dY or tokens is null");
    if ((rc = validate_matrix(ctx, "dY", M, rows, d, dy_row_stride, dy_worker_stride, false)) != ABS_OK) return rc;
    if (M > 1 && tokens_stride != 0 && tokens_stride < rows)
      return set_error(ctx, ABS_ERR_INVALID_ARG, "tokens_stride %lld < rows %lld", tokens_stride, rows);
    if (scratch == nullptr || scratch_bytes < s.bytes)
      return set_error(ctx, ABS_ERR_WORKSPACE, "scratch of %zu bytes needed, %zu given", s.bytes, scratch ? scratch_bytes : 0);
    if (reinterpret_cast<uintptr_t>(scratch) & 255u) return set_error(ctx, ABS_ERR_INVALID_ARG, "scratch must be 256-byte aligned");
  }
  if (rows == 0 && accumulate) return ABS_OK;
  DeviceGuardEmb guard(ctx->device);
  if (!guard.ok) return set_error(ctx, ABS_ERR_CUDA, "cannot select device %d", ctx->device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* mem = static_cast<char*>(scratch);
  const int passes = key_passes(vocab);
  EmbeddingGrad a{dY, dy_row_stride, dy_worker_stride, tokens, tokens_stride, dE, e_row_stride, e_worker_stride, static_cast<int>(rows), M,
                  static_cast<int>(vocab), static_cast<int>(d), accumulate != 0, scale,
                  {reinterpret_cast<unsigned*>(mem + s.key[0]), reinterpret_cast<unsigned*>(mem + s.key[1])},
                  {reinterpret_cast<unsigned*>(mem + s.pos[0]), reinterpret_cast<unsigned*>(mem + s.pos[1])},
                  reinterpret_cast<unsigned*>(mem + s.hist), s.tiles, reinterpret_cast<float*>(mem + s.part), s.runs, s.run, 0};
  if (rows > kSmallKeys) {
    a.sorted = (passes - 1) & 1;
    const dim3 grid(s.tiles, M);
    for (int pass = 0; pass < passes; ++pass) {
      ABS_CUDA_TRY(ctx, launch_dependent(emb_count_kernel, grid, dim3(kEmbThreads), 0, st, a, pass));
      ABS_CUDA_TRY(ctx, launch_dependent(emb_scan_kernel, dim3(M), dim3(1024), 0, st, a));
      ABS_CUDA_TRY(ctx, launch_dependent(emb_scatter_kernel, grid, dim3(kEmbThreads), 0, st, a, pass));
    }
  } else if (rows > 0) {
    ABS_CUDA_TRY(ctx, launch_dependent(emb_sort_small_kernel, dim3(M), dim3(kSmallThreads), 0, st, a, passes));
  }
  const int es = dtype == ABS_F32 ? 4 : 2;
  const bool wide = (((rows > 0 ? bits_of(dY, es, M, dy_row_stride, dy_worker_stride) : 0) | bits_of(dE, 4, M, e_row_stride, e_worker_stride) |
                      static_cast<unsigned long long>(d) * es) & 15u) == 0;
  if (dtype == ABS_F32) return wide ? run_sums<float, 4>(ctx, a, st) : run_sums<float, 1>(ctx, a, st);
  return wide ? run_sums<__nv_bfloat16, 8>(ctx, a, st) : run_sums<__nv_bfloat16, 1>(ctx, a, st);
}
