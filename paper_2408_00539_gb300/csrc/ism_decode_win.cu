// Single tokens under a window in one launch (Section 2.3: a decode step appends
// the new key and value to the cache and attends to what the new row sees).
//
// A window bounds what a step reads, so a step of a few sequences is a matter of
// latency: the cache write, the split attention and the merge of its partials as
// three kernels take 11 us a step whatever they read, most of it launches.  Here a
// thread-block cluster serves one (sequence, KV head): its blocks share out the
// visible keys (the sinks in front of the window, then the window, key by key),
// each with all query heads of the group, and send one another their softmax
// statistics and parts of the outputs through distributed shared memory, where
// each joins its share.  The new key and value are taken
// from the call's own tensors and written to the cache on the side; the lengths
// come from the host's copy in the launch parameters, because no block could tell
// when the others have read the device's, which is advanced here.
//
// CUDA-core arithmetic in fp32: LK lanes hold one row of the head (16 bytes
// each), a block's 8 warps take 8 passes of 8 * (32 / LK) keys at a time with all
// K and V loads of the chunk issued first.  A dot product's partial sums of four
// passes and all heads are added up over the lanes by a butterfly that halves
// the values a lane holds in each step.  P stays in fp32.
#include <atomic>

#include <cooperative_groups.h>

#include "ism_internal.cuh"
#include "ism_tc_common.cuh"

namespace ism {
namespace {

namespace cg = cooperative_groups;

constexpr int kWarps = 8, kThreads = 32 * kWarps, kPasses = 8;
constexpr int kMaxRanks = 8;  // blocks to a cluster

// What every block's first loads wait for comes first: 16 bytes more of fields in
// front of `lens` took 0.2 of 7.3 us a step.
struct WinDecodeArgs {
  const void *q, *k_new, *v_new;
  void *k_cache, *v_cache, *out;
  float* lse;
  const int32_t* table;  // of pages (KvPages), or null
  int32_t page_size, max_pages;
  int64_t cap;
  const float *rope_cos, *rope_sin;
  int32_t* cache_len;
  float scale;
  int32_t batch, hq, hkv, group;
  int32_t page_shift;  // log2 of the page size, or -1
  Window win;
  int32_t lens[kMaxWinDecodeBatch];
  uint32_t* status;
  int32_t num_pages;
};

template <typename T>
struct Row;  // 16 bytes of T as pairs of fp32 values
template <>
struct Row<__nv_bfloat16> {
  static constexpr int N = 8;
  __device__ static void unpack(const uint4& u, float2 (&x)[4]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = make_float2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xFFFF0000u));
  }
  __device__ static uint4 pack(const float2 (&x)[4]) {
    return make_uint4(tc::pack_bf16(x[0].x, x[0].y), tc::pack_bf16(x[1].x, x[1].y), tc::pack_bf16(x[2].x, x[2].y),
                      tc::pack_bf16(x[3].x, x[3].y));
  }
  __device__ static void store(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
};
template <>
struct Row<float> {
  static constexpr int N = 4;
  __device__ static void unpack(const uint4& u, float2 (&x)[2]) {
    x[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
    x[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
  }
  __device__ static uint4 pack(const float2 (&x)[2]) {
    return make_uint4(__float_as_uint(x[0].x), __float_as_uint(x[0].y), __float_as_uint(x[1].x),
                      __float_as_uint(x[1].y));
  }
  __device__ static void store(float* p, float x) { *p = x; }
};

template <typename T, int D, int G>
struct Cfg {
  static constexpr int N = Row<T>::N;          // elements a lane
  static constexpr int LK = D / N;             // lanes a key
  static constexpr int KPW = 32 / LK;          // keys of a warp's pass
  static constexpr int kPass = kWarps * KPW;   // keys of a block's pass
  static constexpr int kChunk = kPasses * kPass;
  // floats of shared memory: scores (then P) of a chunk, each warp's outputs
  static constexpr int SC = G * kChunk, RED = kWarps * G * D;
};

// The rotary encoding of the lane's part of a row (partner coordinates D / 2 away
// are LK / 2 lanes away), rounded to T as the append's rotation is.
template <typename T, int D>
__device__ __forceinline__ uint4 rotated(const uint4& u, const float* cos_row, const float* sin_row, int sub) {
  constexpr int N = Row<T>::N, LK = D / N;
  float2 x[N / 2];
  Row<T>::unpack(u, x);
  const bool high = sub >= LK / 2;
  const int k0 = (sub - (high ? LK / 2 : 0)) * N;
#pragma unroll
  for (int e = 0; e < N / 2; ++e) {
    const float2 y = make_float2(__shfl_xor_sync(0xffffffffu, x[e].x, LK / 2), __shfl_xor_sync(0xffffffffu, x[e].y, LK / 2));
    const float2 c = *reinterpret_cast<const float2*>(cos_row + k0 + 2 * e);
    const float2 s = *reinterpret_cast<const float2*>(sin_row + k0 + 2 * e);
    x[e] = high ? make_float2(x[e].x * c.x + y.x * s.x, x[e].y * c.y + y.y * s.y)
                : make_float2(x[e].x * c.x - y.x * s.x, x[e].y * c.y - y.y * s.y);
  }
  return Row<T>::pack(x);
}

// The value at p where `cond`, else `other`: a predicated load.
__device__ __forceinline__ int32_t ld_gpu_if(const int32_t* p, bool cond, int32_t other) {
  int32_t v;
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.s32 q, %3, 0;\n\tmov.s32 %0, %2;\n\t@q ld.relaxed.gpu.global.s32 %0, [%1];\n\t}"
      : "=&r"(v)
      : "l"(p), "r"(other), "r"((int)cond)
      : "memory");
  return v;
}

// Two blocks an SM where that costs no spills to speak of: the barriers of one leave
// the other running (fp32, 40 sequences of 16 / 4 heads of 64, window 1024: 50.6 us a
// step with one, 32.3 with two).
template <typename T, int D, int G>
__global__ void __launch_bounds__(kThreads, (sizeof(T) == 4 && G <= 4) || G <= 2 ? 2 : 1) decode_window_kernel(const __grid_constant__ WinDecodeArgs a) {
  using C = Cfg<T, D, G>;
  constexpr int N = C::N, LK = C::LK, KPW = C::KPW;
  __shared__ __align__(16) float sm_sc[C::SC];  // [key of the chunk][head]
  __shared__ __align__(16) float sm_red[C::RED];
  // what the cluster's blocks send here: their maxima and sums, and their parts of the outputs that this one joins
  __shared__ __align__(16) float sm_part[G * D];
  __shared__ float sm_pm[kMaxRanks * G], sm_pl[kMaxRanks * G];
  __shared__ float sm_m[G], sm_l[G], sm_alpha[G];
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), ranks = (int)cluster.num_blocks();
  const int item = (int)(blockIdx.x / ranks), b = item / a.hkv, g = item % a.hkv;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane % LK, part = lane / LK;
  const int c = a.lens[b];
  // the new row sees `n` keys: u below `sinks` is key u, from there on u + gap
  const int lo = win_lo(a.win, c), sinks = min(a.win.sinks, lo), gap = lo - sinks, n = c + 1 - gap;
  const int per = (n + ranks - 1) / ranks, u0 = min(rank * per, n), u1 = min(n, u0 + per);
  cluster.barrier_arrive();  // (waited for before anything is sent)
  pdl_wait();

  const int64_t row_elems = (int64_t)a.hkv * D;
  const T* new_k = static_cast<const T*>(a.k_new) + (int64_t)b * row_elems + g * D;
  const T* new_v = static_cast<const T*>(a.v_new) + (int64_t)b * row_elems + g * D;
  // (caches have below 2^31 rows; an entry outside the pool: page_row, *held false)
  auto row_of = [&](int key, bool* held) -> int {
    *held = true;
    if (!a.table) return (int)(b * a.cap) + key;
    const int page = a.page_shift >= 0 ? key >> a.page_shift : key / a.page_size;
    const int32_t entry = a.table[(int64_t)b * a.max_pages + page];
    *held = (uint32_t)entry < (uint32_t)a.num_pages;
    return (int)min((uint32_t)entry, (uint32_t)a.num_pages - 1u) * a.page_size + (key - page * a.page_size);
  };
  bool held;
  auto part_of = [&](const void* cache, int row) {
    return reinterpret_cast<const uint4*>(static_cast<const T*>(cache) + row * row_elems + g * D) + sub;
  };
  // the new key as the cache stores it; the queries, scaled to base 2
  const float *cos_row = nullptr, *sin_row = nullptr;
  if (a.rope_cos) {
    cos_row = a.rope_cos + (int64_t)c * (D / 2);
    sin_row = a.rope_sin + (int64_t)c * (D / 2);
  }
  uint4 k_own = reinterpret_cast<const uint4*>(new_k)[sub];
  if (cos_row) k_own = rotated<T, D>(k_own, cos_row, sin_row, sub);
  float2 q[G][N / 2];
#pragma unroll
  for (int h = 0; h < G; ++h) {
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if (h < a.group)
      u = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + ((int64_t)b * a.hq + g * a.group + h) * D)[sub];
    if (cos_row) u = rotated<T, D>(u, cos_row, sin_row, sub);
    Row<T>::unpack(u, q[h]);
    const float f = a.scale * tc::kLog2e;
#pragma unroll
    for (int e = 0; e < N / 2; ++e) q[h][e] = tc::mul2(q[h][e], make_float2(f, f));
  }
  if (threadIdx.x < G) {  // (read behind the first chunk's barrier, or the one behind the chunks)
    sm_m[threadIdx.x] = -INFINITY;
    sm_l[threadIdx.x] = 0.f;
  }

  float2 o[G][N / 2];
#pragma unroll
  for (int h = 0; h < G; ++h)
#pragma unroll
    for (int e = 0; e < N / 2; ++e) o[h][e] = make_float2(0.f, 0.f);
  // Every K and V row of the first chunk is on its way before any is used; a later
  // chunk's K are loaded while this one's softmax and P V run, its V while its own
  // scores do.  Keys past the range are not loaded.
  uint4 kr[kPasses], vr[kPasses];
  int rows[kPasses];  // of the chunk whose K were loaded last: -1 none, -2 the new key
  auto load_k = [&](int base) {
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int u = base + p * C::kPass + warp * KPW + part, key = u < sinks ? u : u + gap;
      rows[p] = u >= u1 ? -1 : key == c ? -2 : row_of(key, &held);
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      kr[p] = k_own;
      if (rows[p] >= 0) kr[p] = *part_of(a.k_cache, rows[p]);
    }
  };
  auto load_v = [&] {
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      vr[p] = make_uint4(0u, 0u, 0u, 0u);
      if (rows[p] >= 0) vr[p] = *part_of(a.v_cache, rows[p]);
      if (rows[p] == -2) vr[p] = reinterpret_cast<const uint4*>(new_v)[sub];
    }
  };
  // the device's length, which no other block reads, on its way early and without a
  // branch between the loads (read at the end it took 0.3 us a step)
  const bool advances = g == 0 && rank == 0 && threadIdx.x == 0;
  const int32_t found = ld_gpu_if(a.cache_len + b, advances, c);
  if (u0 < u1) {
    load_k(u0);
    load_v();
  }
  for (int base = u0; base < u1; base += C::kChunk) {
    constexpr int kGroup = 4;  // passes whose sums go through the lanes together
#pragma unroll
    for (int p0 = 0; p0 < kPasses; p0 += kGroup) {
      if (base + p0 * C::kPass >= u1) break;
      constexpr int V = kGroup * G;  // values a lane starts with: [pass][head]
      float v[V];
#pragma unroll
      for (int p = 0; p < kGroup; ++p) {
        float2 x[N / 2];
        Row<T>::unpack(kr[p0 + p], x);
#pragma unroll
        for (int h = 0; h < G; ++h) {
          float2 s = tc::mul2(q[h][0], x[0]);
#pragma unroll
          for (int e = 1; e < N / 2; ++e) s = tc::fma2(q[h][e], x[e], s);
          v[p * G + h] = s.x + s.y;
        }
      }
      // after the step of lane bit `sh` a lane keeps the half of its values that the bit selects
      int first = 0;
      int have = V;
#pragma unroll
      for (int sh = LK / 2; sh >= 1; sh >>= 1) {
        if (have > 1) {
          have >>= 1;
          const bool hi = (sub & sh) != 0;
#pragma unroll
          for (int i = 0; i < V / 2; ++i)
            if (i < have) {
              const float send = hi ? v[i] : v[have + i];
              const float keep = hi ? v[have + i] : v[i];
              v[i] = keep + __shfl_xor_sync(0xffffffffu, send, sh);
            }
          first = hi ? first + have : first;
        } else {
          v[0] += __shfl_xor_sync(0xffffffffu, v[0], sh);
        }
      }
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < have) {
          const int at = first + i, p = p0 + at / G, h = at % G;
          sm_sc[(p * C::kPass + warp * KPW + part) * G + h] = v[i];
        }
    }
    if (base + C::kChunk < u1) load_k(base + C::kChunk);
    __syncthreads();
    // softmax of the chunk: a warp a head
    for (int h = warp; h < G; h += kWarps) {
      float* s = sm_sc + h;
      const int m_keys = min(C::kChunk, u1 - base);
      float mx = -INFINITY;
      for (int i = lane; i < m_keys; i += 32) mx = fmaxf(mx, s[i * G]);
#pragma unroll
      for (int sh = 16; sh >= 1; sh >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, sh));
      const float old = sm_m[h], m = fmaxf(old, mx);
      float l = 0.f;
      for (int i = lane; i < C::kChunk; i += 32) {
        const float p = i < m_keys ? tc::ex2(s[i * G] - m) : 0.f;
        s[i * G] = p;
        l += p;
      }
#pragma unroll
      for (int sh = 16; sh >= 1; sh >>= 1) l += __shfl_xor_sync(0xffffffffu, l, sh);
      __syncwarp();
      if (lane == 0) {
        const float f = old == -INFINITY ? 0.f : tc::ex2(old - m);
        sm_alpha[h] = f;
        sm_l[h] = sm_l[h] * f + l;
        sm_m[h] = m;
      }
    }
    __syncthreads();
    if (base > u0) {
#pragma unroll
      for (int h = 0; h < G; ++h) {
        const float f = sm_alpha[h];
#pragma unroll
        for (int e = 0; e < N / 2; ++e) o[h][e] = tc::mul2(o[h][e], make_float2(f, f));
      }
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      if (base + p * C::kPass + warp * KPW >= u1) break;  // (no key of the warp's pass)
      float2 x[N / 2];
      Row<T>::unpack(vr[p], x);
      float w[G];
      const float* ws = sm_sc + (p * C::kPass + warp * KPW + part) * G;
      if constexpr (G % 4 == 0) {
#pragma unroll
        for (int h = 0; h < G; h += 4) {
          const float4 w4 = *reinterpret_cast<const float4*>(ws + h);
          w[h] = w4.x; w[h + 1] = w4.y; w[h + 2] = w4.z; w[h + 3] = w4.w;
        }
      } else {
#pragma unroll
        for (int h = 0; h < G; ++h) w[h] = ws[h];
      }
#pragma unroll
      for (int h = 0; h < G; ++h)
#pragma unroll
        for (int e = 0; e < N / 2; ++e) o[h][e] = tc::fma2(make_float2(w[h], w[h]), x[e], o[h][e]);
    }
    if (base + C::kChunk < u1) {
      load_v();
      __syncthreads();  // the scores are rewritten
    }
  }

  // the block's outputs: over the keys of a pass, then over the warps
  {
    auto add_other = [](const float2& keep, const float2& send, int sh) {
      return make_float2(keep.x + __shfl_xor_sync(0xffffffffu, send.x, sh), keep.y + __shfl_xor_sync(0xffffffffu, send.y, sh));
    };
    int first = 0, have = G;  // heads that the lane adds up
#pragma unroll
    for (int sh = LK; sh < 32; sh <<= 1) {
      const bool hi = (lane & sh) != 0;
      if (have > 1) {
        have >>= 1;
#pragma unroll
        for (int h = 0; h < G / 2; ++h)
          if (h < have)
#pragma unroll
            for (int e = 0; e < N / 2; ++e)
              o[h][e] = add_other(hi ? o[have + h][e] : o[h][e], hi ? o[h][e] : o[have + h][e], sh);
        first = hi ? first + have : first;
      } else {
#pragma unroll
        for (int e = 0; e < N / 2; ++e) o[0][e] = add_other(o[0][e], o[0][e], sh);
      }
    }
#pragma unroll
    for (int h = 0; h < G; ++h)
      if (h < have)
#pragma unroll
        for (int e = 0; e < N / 2; e += 2)
          *reinterpret_cast<float4*>(sm_red + (warp * G + first + h) * D + sub * N + 2 * e) =
              make_float4(o[h][e].x, o[h][e].y, o[h][e + 1].x, o[h][e + 1].y);
  }
  __syncthreads();
  cluster.barrier_wait();
  // every block joins a share of the group's outputs (G * D / ranks of them) and is sent the others' parts of it
  constexpr int total = G * D;
  const int share = total / ranks;
  for (int i = 4 * threadIdx.x; i < total; i += 4 * kThreads) {  // (a share is a multiple of 4)
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 y = *reinterpret_cast<const float4*>(sm_red + w * total + i);
      x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
    }
    *reinterpret_cast<float4*>(cluster.map_shared_rank(sm_part, i / share) + rank * share + i % share) = x;
  }
  if (threadIdx.x < G * ranks) {
    const int h = threadIdx.x % G, to = threadIdx.x / G;
    cluster.map_shared_rank(sm_pm, to)[rank * G + h] = sm_m[h];
    cluster.map_shared_rank(sm_pl, to)[rank * G + h] = sm_l[h];
  }
  cluster.sync();
  for (int j = threadIdx.x; j < share; j += kThreads) {
    const int i = rank * share + j, h = i / D;
    if (h >= a.group) break;
    float m = -INFINITY;
    for (int r = 0; r < ranks; ++r) m = fmaxf(m, sm_pm[r * G + h]);
    float x = 0.f, l = 0.f;
    for (int r = 0; r < ranks; ++r) {  // (a part without keys has maximum -inf)
      const float mr = sm_pm[r * G + h];
      const float f = mr == -INFINITY ? 0.f : tc::ex2(mr - m);
      l = fmaf(f, sm_pl[r * G + h], l);
      x = fmaf(f, sm_part[r * share + j], x);
    }
    Row<T>::store(static_cast<T*>(a.out) + ((int64_t)b * a.hq + g * a.group) * D + i, x / l);
    if (i % D == 0 && a.lse) a.lse[(int64_t)(g * a.group + h) * a.batch + b] = (m + log2f(l)) * tc::kLn2;
  }
  // the cache: the new row, and zeros in the value rows up to the next multiple of 128 (see launch_cache_write); nothing
  // of it is read above
  const int64_t stop = ((int64_t)c + 128) / 128 * 128;
  const int64_t end = a.table || stop < a.cap ? stop : a.cap;
  // (the rows of a page, or of a contiguous cache, follow one another)
  const int own_row = row_of(c, &held);
  uint4* const k_row = const_cast<uint4*>(part_of(a.k_cache, own_row));
  uint4* const v_row = const_cast<uint4*>(part_of(a.v_cache, own_row));
  if (!held && threadIdx.x == 0) atomicOr(a.status, kStatusCache);
  for (int key = c + rank * (kThreads / LK) + threadIdx.x / LK; held && key < end; key += ranks * (kThreads / LK)) {
    if (key == c) *k_row = k_own;
    v_row[(key - c) * (row_elems / N)] = key == c ? reinterpret_cast<const uint4*>(new_v)[sub] : make_uint4(0u, 0u, 0u, 0u);
  }
  if (advances) {
    if (found != c) atomicOr(a.status, kStatusCache);
    a.cache_len[b] = c + 1;
  }
}

template <typename T, int D, int G>
cudaError_t launch_t(const WinDecodeArgs& a, int ranks, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)a.batch * a.hkv * ranks));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ranks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, decode_window_kernel<T, D, G>, a);
}

// Clusters of `ranks` blocks that run at a time on the current device (asked once a
// device, kernel and size, on devices past kMaxDevices each time; 0: unknown).
constexpr int kMaxDevices = 64;
template <typename T, int D, int G>
int active_clusters(int ranks) {
  static std::atomic<int> known[kMaxDevices][kMaxRanks + 1];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
  int n = dev < kMaxDevices ? known[dev][ranks].load(std::memory_order_relaxed) : 0;
  if (n > 0) return n;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(ranks * sm_count()));
  cfg.blockDim = dim3(kThreads);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)ranks;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, decode_window_kernel<T, D, G>, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  if (dev < kMaxDevices) known[dev][ranks].store(n, std::memory_order_relaxed);
  return n;
}

// How a step of `items` (sequence, KV head) pairs that see up to `seen` keys runs:
// the largest cluster that leaves every item one at a time and each block half a
// chunk of keys; and about how long it takes.
struct WinPlan {
  int ranks;
  int64_t ns;
};
template <typename T, int D, int G>
WinPlan plan_t(int64_t items, int64_t seen) {
  constexpr int64_t half = Cfg<T, D, G>::kChunk / 2;
  int ranks = 1;
  while (ranks < kMaxRanks && seen > ranks * half && items <= active_clusters<T, D, G>(2 * ranks)) ranks *= 2;
  const int64_t at_once = active_clusters<T, D, G>(ranks);
  const int64_t waves = at_once > 0 ? (items + at_once - 1) / at_once : 1, per = (seen + ranks - 1) / ranks;
  return WinPlan{ranks, 4500 + waves * ((per + half - 1) / half) * (750 + 200 * G)};
}

template <typename T, int D>
WinPlan plan_g(int group, int64_t items, int64_t seen) {
  return group <= 1   ? plan_t<T, D, 1>(items, seen)
         : group <= 2 ? plan_t<T, D, 2>(items, seen)
         : group <= 4 ? plan_t<T, D, 4>(items, seen)
                      : plan_t<T, D, 8>(items, seen);
}
template <typename T, int D>
cudaError_t launch_g(const WinDecodeArgs& a, int ranks, cudaStream_t st) {
  return a.group <= 1   ? launch_t<T, D, 1>(a, ranks, st)
         : a.group <= 2 ? launch_t<T, D, 2>(a, ranks, st)
         : a.group <= 4 ? launch_t<T, D, 4>(a, ranks, st)
                        : launch_t<T, D, 8>(a, ranks, st);
}

WinPlan plan(const DecodeArgs& d, int64_t seen) {
  const int64_t items = (int64_t)d.batch * d.hkv;
  if (d.dtype == ISM_FP32) return d.d == 64 ? plan_g<float, 64>(d.group, items, seen) : plan_g<float, 128>(d.group, items, seen);
  return d.d == 64 ? plan_g<__nv_bfloat16, 64>(d.group, items, seen) : plan_g<__nv_bfloat16, 128>(d.group, items, seen);
}

int64_t most_seen(const DecodeArgs& d, const int32_t* lens) {
  int64_t most = 0;
  for (int b = 0; b < d.batch; ++b)
    if (lens[b] + (int64_t)1 > most) most = lens[b] + (int64_t)1;
  const int64_t w = (int64_t)d.win.window + d.win.sinks;
  return most < w ? most : w;
}

}  // namespace

// bf16 at head_dim 128 has the tensor-core decode between a cache write and a merge
// (10.8 us, and the 64 KB tiles of the window at some 6.5 TB/s) to choose from, at 64
// the split decode of the CUDA cores (12.5 us, and the 256-byte rows at 3 TB/s); fp32
// only the forward kernel.  Three launches and one, us a step, 32 / 8 heads, window
// 1024: one sequence 11.7 and 8.2, 4 13.6 and 11.5, 8 14.6 and 17.4; one of window
// 4096 12.5 and 16.9; 8 of window 256 12.1 and 8.7; 40 of window 64 21.4 and 16.9, of
// 200 23.6 and 26.0; 4 of 32 / 32 heads, window 512 17.2 and 10.7.  At 64, 16 / 4 heads,
// window 1024: one 12.8 and 6.1, 8 14.8 and 8.4, 40 27.2 and 32.4; fp32 one 49.0 and
// 6.9, 40 601 and 32.3.
bool decode_window_one_launch(const DecodeArgs& d, const int32_t* lens) {
  if (!d.win.window || d.group > 8 || d.batch > kMaxWinDecodeBatch || d.dtype == ISM_E4M3) return false;
  if (knobs().decode_window >= 0) return knobs().decode_window != 0;
  if (d.dtype == ISM_FP32) return true;
  const int64_t seen = most_seen(d, lens), items = (int64_t)d.batch * d.hkv;
  return plan(d, seen).ns < (d.d == 64 ? 12500 + items * seen * 85 / 1000 : 10800 + items * ((seen + 127) / 128 + 1) * 10);
}

cudaError_t launch_decode_window(const DecodeArgs& d, const void* k_new, const void* v_new, const int32_t* lens,
                                 const float* rope_cos, const float* rope_sin, cudaStream_t st) {
  if (!d.win.window || d.group > 8 || d.batch > kMaxWinDecodeBatch || d.dtype == ISM_E4M3) return cudaErrorInvalidValue;
  WinDecodeArgs a;
  a.q = d.q; a.k_new = k_new; a.v_new = v_new;
  a.k_cache = const_cast<void*>(d.k_cache); a.v_cache = const_cast<void*>(d.v_cache);
  a.out = d.out; a.lse = d.lse; a.table = d.pages.table; a.page_size = d.pages.page_size;
  a.max_pages = d.pages.max_pages; a.num_pages = d.pages.num_pages; a.cap = d.cap;
  a.rope_cos = rope_cos; a.rope_sin = rope_sin; a.cache_len = d.cache_len; a.status = d.status; a.scale = d.scale;
  a.batch = d.batch; a.hq = d.hq; a.hkv = d.hkv; a.group = d.group; a.win = d.win;
  a.page_shift = -1;
  if (d.pages.table && (d.pages.page_size & (d.pages.page_size - 1)) == 0)
    for (a.page_shift = 0; (1 << a.page_shift) < d.pages.page_size;) ++a.page_shift;
  for (int b = 0; b < d.batch; ++b) a.lens[b] = lens[b];
  const int ranks = plan(d, most_seen(d, lens)).ranks;
  if (d.dtype == ISM_FP32) return d.d == 64 ? launch_g<float, 64>(a, ranks, st) : launch_g<float, 128>(a, ranks, st);
  return d.d == 64 ? launch_g<__nv_bfloat16, 64>(a, ranks, st) : launch_g<__nv_bfloat16, 128>(a, ranks, st);
}

}  // namespace ism
