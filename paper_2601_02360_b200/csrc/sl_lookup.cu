// Embedding lookup of a flattened batch (sections 2.3 and 2.4: X^(0) = T_S[x] + T_perp[x] + PosEmbed) and its
// gradient.
#include "sl_inner.cuh"

namespace sl {
namespace {

constexpr int kThreads = 256;

constexpr int pieces(int e) { return e == 1 ? 4 : 1; }      // of a thread in the runs kernel

// How the columns of a row are dealt out: threads side by side, rows of a CTA, CTAs (or passes) over the rest of the columns.
// Evenly, so that no CTA of a row has a few columns only; a CTA's threads are whole warps.
struct Columns {
  uint32_t tx, ty, ctas;
  Columns(uint32_t d, int e, int per = 1) {
    const uint32_t parts = (d + e * per - 1) / (e * per);
    ctas = (parts + kThreads - 1) / kThreads;
    tx = (parts + ctas - 1) / ctas;
    const uint32_t step = tx <= 32 ? 8 : tx <= 64 ? 16 : 32;
    tx = (tx + step - 1) / step * step;
    ty = kThreads / tx / (32 / step) * (32 / step);
    if (ty < 1) ty = 1;
  }
};

// E elements of a row, or one where rows are not aligned
template <class T, int E>
__device__ __forceinline__ void load_once(const T* p, float (&f)[E]) {
  if constexpr (E == 1) {
    f[0] = to_f32(*p);
  } else {
    Raw<T, E> r;
    r.load(p);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = r.get(e);
  }
}
// a piece of a row as it is stored, to be looked at later
template <class T, int E>
struct Ring {
  Raw<T, E> r;
  __device__ __forceinline__ void load(const T* p) { r.load(p); }
  __device__ __forceinline__ void load_kept(const T* p) { r.load_kept(p); }
  __device__ __forceinline__ float get(int e) const { return r.get(e); }
};
template <class T>
struct Ring<T, 1> {
  T v;
  __device__ __forceinline__ void load(const T* p) { v = *p; }
  __device__ __forceinline__ void load_kept(const T* p) { v = *p; }
  __device__ __forceinline__ float get(int) const { return to_f32(v); }
};

// partial sums that a later kernel reads soon
template <int E>
__device__ __forceinline__ void store_kept(float* p, const float (&f)[E]) {
  if constexpr (E == 1) {
    *p = f[0];
  } else {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
  }
}
template <class T, int E>
__device__ __forceinline__ void store_once(T* p, const float (&f)[E]) {
  if constexpr (E == 1) {
    *p = from_f32<T>(f[0]);
  } else {
    Raw<T, E> r;
    r.set(f);
    r.store(p);
  }
}

// ---------------------------------------------------------------------------
// Lookup: blockDim.x threads share a row, blockDim.y groups of them to a CTA.
//
// HBM sees the distinct rows of the tables and the output once, but L2 serves every token's rows again.  So the tokens are
// taken position by position (token b L + l for b = 0, 1, ...): a group walks `run` of them in a row and fetches a
// position row once for all that share it (64K tokens, d = 2048, float32, both tables and positions: 170 -> 151 us).  The
// next token's id is on its way while a row is; fetching the next row as well costs more registers than it hides (159 us).
// What bounds it: float32, the rows' latency at the warps that fit, 135 us for 767 MB that HBM has to move (5.7 TB/s);
// bfloat16, instructions:
// 74 us for 384 MB (69 % of the issue slots were taken at 100 us, before a thread had two pieces).
// ---------------------------------------------------------------------------
constexpr uint64_t kSlab = 104ull << 20; // bytes of table rows that stay in L2 beside the output on its way
constexpr uint32_t kSlabColumns = 256;
struct LookupOrder {
  uint32_t B, run;           // sequences; tokens a group takes in a row
  uint32_t width, units;     // columns of a slab; runs of tokens
};

// PER pieces of E consecutive elements to a thread, blockDim.x pieces apart.  Two pieces of 8: the instructions that find a
// row are then shared by twice the elements (64K x 2048 of split bf16 tables: 100 -> 77 us, of f32 ones 151 -> 149 us); four
// cost more in resident warps than they save (98 and 151 us).
template <class TB, class XT, int E, int PER>
__global__ void __launch_bounds__(kThreads, E == 1 || (PER > 1 && sizeof(TB) == 4) ? 3 : 4) embed_lookup_kernel(const LookupArgs a, const LookupOrder o) {
  const TB *ts = static_cast<const TB*>(a.T_S), *tp = static_cast<const TB*>(a.T_perp), *pos = static_cast<const TB*>(a.pos);
  XT* out = static_cast<XT*>(a.X);
  const uint32_t stride = pos ? a.L : 0;                   // from a token to the next sequence's at the same position
  const uint64_t all = (uint64_t)(pos ? a.L : a.n_tok) * o.B;            // places in the order, some behind the last token
  uint32_t slab = 0;                                       // first column of the one at hand
  for (uint32_t unit = blockIdx.x * blockDim.y + threadIdx.y;; unit += gridDim.x * blockDim.y) {
    for (; unit >= o.units && slab < a.d; unit -= o.units) slab += o.width;
    if (slab >= a.d) break;
    const uint32_t end = a.d - slab < o.width ? a.d : slab + o.width;
    const uint64_t j0 = (uint64_t)unit * o.run;
    const uint32_t count = (uint32_t)(j0 + o.run < all ? o.run : all - j0);
    const uint32_t l0 = o.B == 1 ? (uint32_t)j0 : (uint32_t)(j0 / o.B), b0 = (uint32_t)(j0 - (uint64_t)l0 * o.B);
    for (uint32_t c0 = slab + threadIdx.x * E; c0 < end; c0 += blockDim.x * E * PER) {
      // pieces behind the slab's end load its first one, so that no load needs a condition
      uint32_t c[PER];
#pragma unroll
      for (int k = 0; k < PER; ++k) c[k] = c0 + k * blockDim.x * E < end ? c0 + k * blockDim.x * E : slab;
      Ring<TB, E> z[PER];
      uint32_t l = l0, b = b0;
      uint64_t t = (uint64_t)b * stride + l;
      bool fresh = true;                                   // the position row is not here yet
      uint32_t id = t < a.n_tok ? (uint32_t)__ldg(a.ids + t) : ~0u;
      for (uint32_t i = 0; i < count; ++i) {
        const bool wrap = b + 1 == o.B;
        const uint64_t t1 = wrap ? l + 1 : t + stride;
        const uint32_t next = i + 1 < count && t1 < a.n_tok ? (uint32_t)__ldg(a.ids + t1) : ~0u;
        if (t < a.n_tok) {
          const uint64_t row = (uint64_t)(id < a.V ? id : 0) * a.d;
          Ring<TB, E> x[PER], y[PER];
#pragma unroll
          for (int k = 0; k < PER; ++k) x[k].load_kept(ts + row + c[k]);
          if (tp)
#pragma unroll
            for (int k = 0; k < PER; ++k) y[k].load_kept(tp + row + c[k]);
          if (pos && fresh)
#pragma unroll
            for (int k = 0; k < PER; ++k) z[k].load_kept(pos + (uint64_t)l * a.d + c[k]);
          fresh = false;
          float f[PER][E];
#pragma unroll
          for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) f[k][e] = x[k].get(e);
          if (tp)
#pragma unroll
            for (int k = 0; k < PER; ++k)
#pragma unroll
              for (int e = 0; e < E; ++e) f[k][e] = f[k][e] + y[k].get(e);
#pragma unroll
          for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) f[k][e] = a.scale * f[k][e];
          if (pos)
#pragma unroll
            for (int k = 0; k < PER; ++k)
#pragma unroll
              for (int e = 0; e < E; ++e) f[k][e] = f[k][e] + z[k].get(e);
          if (id >= a.V) {
            if (c0 == 0 && a.flags) atomicOr(a.flags, (uint32_t)SL_FLAG_BAD_INDEX);
#pragma unroll
            for (int k = 0; k < PER; ++k)
#pragma unroll
              for (int e = 0; e < E; ++e) f[k][e] = 0.0f;
          }
          XT* to = out + t * a.d;
#pragma unroll
          for (int k = 0; k < PER; ++k)
            if (k == 0 || c[k] != slab) store_once(to + c[k], f[k]);
        }
        if (wrap) {
          ++l;
          b = 0;
          fresh = true;
        } else {
          ++b;
        }
        t = t1;
        id = next;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Gradient.  dT[v] is the sum of the rows of dX whose token is v, in the tokens' order.
//
// Many tokens: the tokens are sorted by id (stable, so a row's tokens stay ascending) and cut into windows of equal
// length, whatever the ids; a part is the runs of equal ids that begin in a window, added up in registers and written where
// they end.  A run that fills a whole window is cut there, and its partial rows are joined in order by a last kernel: one
// id with half of all tokens costs no more than any other batch.  HBM bounds the sums, every row of dX and of the table once:
// 64K x 2048 bf16 into a float32 table of 32,000 rows, 531 MB, in 129 us for the call, of which the sort is 21 and the sums
// 90 (5.9 TB/s).  A few thousand tokens are bound by the chain of the three kernels (4111 x 1535: 38 us).
// Few tokens: one launch, in which the first token of every id finds and sums the others (1000 x 1024: 7.8 us).
// ---------------------------------------------------------------------------

// The one-launch form: rows without a token are set to zero by `slices` CTAs; CTA `slice` marks the ids it finds
// among its own rows in `seen` (kWindow bytes of shared memory).
constexpr uint32_t kWindow = 2048;

template <class DT, bool VEC>
__device__ void zero_absent_rows(const EmbedGradArgs& a, uint32_t slice, uint32_t slices, uint8_t* seen) {
  const uint32_t per = (a.V + slices - 1) / slices, w = per < kWindow ? per : kWindow;
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  for (uint64_t v0 = (uint64_t)slice * w; v0 < a.V; v0 += (uint64_t)slices * w) {
    const uint32_t rows = (uint32_t)(a.V - v0 < w ? a.V - v0 : w);
    for (uint32_t i = threadIdx.x; i < rows; i += blockDim.x) seen[i] = 0;
    __syncthreads();
    const bool quads = (reinterpret_cast<uintptr_t>(a.ids) & 15) == 0;
    const uint32_t nq = quads ? a.n_tok / 4 : 0;
    for (uint32_t q0 = threadIdx.x; q0 < nq; q0 += 4 * blockDim.x) {
      int4 id[4];                                          // on their way together
#pragma unroll
      for (int u = 0; u < 4; ++u) id[u] = q0 + u * blockDim.x < nq ? __ldg(reinterpret_cast<const int4*>(a.ids) + q0 + u * blockDim.x) : make_int4(-1, -1, -1, -1);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t x = (uint32_t)id[u].x - (uint32_t)v0, y = (uint32_t)id[u].y - (uint32_t)v0, z = (uint32_t)id[u].z - (uint32_t)v0,
                       w = (uint32_t)id[u].w - (uint32_t)v0;
        if (x < rows) seen[x] = 1;
        if (y < rows) seen[y] = 1;
        if (z < rows) seen[z] = 1;
        if (w < rows) seen[w] = 1;
      }
    }
    for (uint32_t t = 4 * nq + threadIdx.x; t < a.n_tok; t += blockDim.x) {
      const uint32_t x = (uint32_t)__ldg(a.ids + t) - (uint32_t)v0;
      if (x < rows) seen[x] = 1;
    }
    __syncthreads();
    for (uint32_t r = warp; r < rows; r += warps) {
      if (seen[r]) continue;
      DT* row = static_cast<DT*>(a.dT) + (v0 + r) * a.d;
      if constexpr (VEC) {
        for (uint32_t c = lane; c < a.d * sizeof(DT) / 16; c += 32) __stcs(reinterpret_cast<uint4*>(row) + c, make_uint4(0, 0, 0, 0));
      } else {
        for (uint32_t c = lane; c < a.d; c += 32) row[c] = from_f32<DT>(0.0f);
      }
    }
    __syncthreads();
  }
}

// adds a finished sum to its table row
template <class DT, int E>
__device__ __forceinline__ void finish_row(const EmbedGradArgs& a, uint32_t id, uint32_t c, const float (&sum)[E], const float (&old)[E]) {
  float f[E];
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] = a.acc ? old[e] + a.scale * sum[e] : a.scale * sum[e];
  store_once(static_cast<DT*>(a.dT) + (uint64_t)id * a.d + c, f);
}

constexpr int kDirect = 128;
constexpr uint32_t kDirectMost = 1024;       // tokens up to which the one-launch form is taken
constexpr int kDirectIds = kDirectMost / kDirect;

// CTAs (token, column part) first, then, unless the gradient is accumulated, `slices` CTAs for the absent rows
template <class DX, class DT, int E>
__global__ void __launch_bounds__(kDirect) embed_grad_direct_kernel(const EmbedGradArgs a, uint32_t parts, uint32_t slices) {
  __shared__ uint8_t seen[kWindow];
  __shared__ uint32_t list[kDirectMost], found[kDirectIds * kDirect / 32];
  const uint32_t t = blockIdx.x / parts, part = blockIdx.x - t * parts, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (t >= a.n_tok) {
    zero_absent_rows<DT, (E > 1)>(a, blockIdx.x - a.n_tok * parts, slices, seen);
    return;
  }
  uint32_t ids[kDirectIds];
  const uint32_t id = (uint32_t)__ldg(a.ids + t);
#pragma unroll
  for (int i = 0; i < kDirectIds; ++i) {
    const uint32_t j = i * kDirect + threadIdx.x;
    ids[i] = j < a.n_tok ? (uint32_t)__ldg(a.ids + j) : ~0u;
  }
  if (id >= a.V) {
    if (threadIdx.x == 0 && part == 0 && a.flags) atomicOr(a.flags, (uint32_t)SL_FLAG_BAD_INDEX);
    return;
  }
  const DX* dx = static_cast<const DX*>(a.dX);
  const uint32_t c = (part * kDirect + threadIdx.x) * E;
  float sum[E] = {}, old[E] = {};
  if (a.acc && c < a.d) load_once(static_cast<const DT*>(a.dT) + (uint64_t)id * a.d + c, old);
  // the tokens of this id, ascending; if t is not the first, another CTA has them
  uint32_t hits[kDirectIds];
  bool earlier = false;
#pragma unroll
  for (int i = 0; i < kDirectIds; ++i) {
    hits[i] = __ballot_sync(0xFFFFFFFFu, ids[i] == id);
    earlier |= ids[i] == id && i * kDirect + threadIdx.x < t;
    if (lane == 0) found[i * (kDirect / 32) + warp] = __popc(hits[i]);
  }
  if (__syncthreads_or(earlier)) return;
  uint32_t all = 0;
#pragma unroll
  for (int i = 0; i < kDirectIds; ++i) {
#pragma unroll
    for (uint32_t w = 0; w < kDirect / 32; ++w) {
      if (w == warp && ids[i] == id) list[all + __popc(hits[i] & ((1u << lane) - 1))] = i * kDirect + threadIdx.x;
      all += found[i * (kDirect / 32) + w];
    }
  }
  __syncthreads();
  if (c >= a.d) return;
#pragma unroll 8
  for (uint32_t k = 0; k < all; ++k) {
    float f[E];
    load_once(dx + (uint64_t)list[k] * a.d + c, f);
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] += f[e];
  }
  finish_row<DT, E>(a, id, c, sum, old);
}

// ---- sort by id: one cluster, least significant digit first, up to 9 bits a pass ----
constexpr int kSortCtas = 16, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kDigitBits = 9, kAhead = 8;

struct SortArgs {
  uint2* list[2];                // ids and their tokens: written alternately, the last pass writes [0]
  int passes, bits;              // bits of a digit
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a word of CTA `rank`'s shared memory at the address of this CTA's `p`
__device__ __forceinline__ uint32_t load_cluster(const uint32_t* p, uint32_t rank) {
  uint32_t at = (uint32_t)__cvta_generic_to_shared(p), v;
  asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(at) : "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

// Lanes of the warp with the same digit, by one ballot a bit (the sort of 64K tokens: 37 us, 43 with __match_any_sync).
// A lane that is not `in` matches nobody.
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, int bits, bool in) {
  uint32_t same = __ballot_sync(0xFFFFFFFFu, in);
  for (int b = 0; b < bits; ++b) {
    const uint32_t set = __ballot_sync(0xFFFFFFFFu, (digit >> b) & 1u);
    same &= (digit >> b) & 1u ? set : ~set;
  }
  return same;
}

__device__ void sort_tokens(const EmbedGradArgs& a, const SortArgs& s, uint32_t* smem) {
  uint32_t* hist = smem;                                   // [warps][bins]: counts, then first places
  uint32_t* total = smem + (kSortWarps << s.bits);         // [bins] of this CTA
  uint32_t* wsum = total + (1u << s.bits);                 // [warps]
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = cluster_rank(), bins = 1u << s.bits;
  // the warp's tokens: consecutive, a multiple of 32 of them
  const uint32_t per = (a.n_tok + kSortCtas * kSortThreads - 1) / (kSortCtas * kSortThreads) * 32;
  const uint64_t lo64 = (uint64_t)(rank * kSortWarps + warp) * per;
  const uint32_t lo = lo64 < a.n_tok ? (uint32_t)lo64 : a.n_tok, hi = a.n_tok - lo < per ? a.n_tok : lo + per;
  uint32_t* mine = hist + (warp << s.bits);
  bool bad = false;
  for (int pass = 0; pass < s.passes; ++pass) {
    const uint2* from = s.list[(s.passes - pass) & 1];
    uint2* to = s.list[(s.passes - pass - 1) & 1];
    const int shift = pass * s.bits;
    // kAhead steps of 32 tokens are read together; what lies behind the warp's last token has digit `bins`
    auto read = [&](uint32_t i, uint2(&item)[kAhead]) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const uint32_t j = i + 32 * u + lane;
        item[u] = make_uint2(0, j);
        if (j < hi) {
          if (pass > 0) item[u] = __ldcg(from + j);
          else item[u].x = (uint32_t)__ldg(a.ids + j);
        }
      }
      if (pass == 0)
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          bad |= item[u].x >= a.V;
          item[u].x = item[u].x < a.V ? item[u].x : a.V;   // bad ids go to the end
        }
    };
    for (uint32_t b = lane; b < bins; b += 32) mine[b] = 0;
    __syncwarp();
    const bool once = per <= 32 * kAhead;                  // the warp's tokens are read once a pass
    uint2 item[kAhead];
    uint32_t rank_of[kAhead];                              // of a token among the warp's with its digit
    for (uint32_t i = lo; i < hi; i += 32 * kAhead) {
      read(i, item);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (i + 32 * u >= hi) break;
        const bool in = i + 32 * u + lane < hi;
        const uint32_t digit = (item[u].x >> shift) & (bins - 1), same = same_digit(digit, s.bits, in);
        const uint32_t count = in ? mine[digit] : 0;
        rank_of[u] = count + __popc(same & ((1u << lane) - 1));
        __syncwarp();
        if (in && lane == (uint32_t)(__ffs(same) - 1)) mine[digit] = count + __popc(same);
        __syncwarp();
      }
    }
    __syncthreads();
    uint32_t sum = 0;
    if (threadIdx.x < bins) {
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) sum += hist[(w << s.bits) + threadIdx.x];
      total[threadIdx.x] = sum;
    }
    cluster_barrier();
    // first place of every digit: all smaller digits of all CTAs, then the same digit of the CTAs before
    uint32_t all = 0, before = 0;
    if (threadIdx.x < bins) {
#pragma unroll
      for (uint32_t r = 0; r < kSortCtas; ++r) {
        const uint32_t n = load_cluster(total + threadIdx.x, r);
        all += n;
        before += r < rank ? n : 0;
      }
    }
    uint32_t scan = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, scan, o);
      if (lane >= (uint32_t)o) scan += x;
    }
    if (lane == 31) wsum[warp] = scan;
    __syncthreads();
    if (threadIdx.x < bins) {
      uint32_t place = scan - all + before, n[kSortWarps];
      for (uint32_t w = 0; w < warp; ++w) place += wsum[w];
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) n[w] = hist[(w << s.bits) + threadIdx.x];
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) {
        hist[(w << s.bits) + threadIdx.x] = place;
        place += n[w];
      }
    }
    __syncthreads();
    if (once) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (lo + 32 * u + lane < hi) to[mine[(item[u].x >> shift) & (bins - 1)] + rank_of[u]] = item[u];
    }
    for (uint32_t i = once ? hi : lo; i < hi; i += 32 * kAhead) {
      read(i, item);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (i + 32 * u >= hi) break;
        const bool in = i + 32 * u + lane < hi;
        const uint32_t digit = (item[u].x >> shift) & (bins - 1), same = same_digit(digit, s.bits, in);
        if (in) to[mine[digit] + __popc(same & ((1u << lane) - 1))] = item[u];
        __syncwarp();
        if (in && lane == (uint32_t)(__ffs(same) - 1)) mine[digit] += __popc(same);
        __syncwarp();
      }
    }
    cluster_barrier();                                     // the pass is visible to the whole cluster
  }
  if (__any_sync(0xFFFFFFFFu, bad) && lane == 0 && a.flags) atomicOr(a.flags, (uint32_t)SL_FLAG_BAD_INDEX);
}

// ---- positions: row l is the sum of the tokens l, l + L, l + 2 L, ... ----
// With few positions a row's tokens are cut into `cuts` whose sums go to `part` [cuts][L][d].  The work is dealt out in units
// of one row of one cut and the columns of `tx` threads, PER pieces each; a group of tx threads takes unit after unit.
struct PosArgs {
  float* part;               // NULL: no cuts
  uint32_t cuts, per_cut, tx, column_parts;
};

template <class DX, class DT, int E, int PER>
__device__ void sum_positions(const EmbedGradArgs& a, const PosArgs& q, uint64_t group, uint64_t groups) {
  constexpr int DEPTH = E == 8 && sizeof(DX) == 2 ? 8 : 4; // rows on their way together
  const DX* dX = static_cast<const DX*>(a.dX);
  const uint64_t units = (uint64_t)a.L * q.cuts * q.column_parts;
  for (uint64_t u = group; u < units; u += groups) {
    const uint32_t cp = (uint32_t)(u % q.column_parts), cut = (uint32_t)(u / q.column_parts % q.cuts);
    const uint32_t l = (uint32_t)(u / ((uint64_t)q.column_parts * q.cuts)), c0 = (cp * PER * q.tx + threadIdx.x) * E;
    if (c0 >= a.d) continue;
    uint32_t c[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) c[i] = c0 + i * q.tx * E < a.d ? c0 + i * q.tx * E : 0;
    const uint32_t rows = l < a.n_tok ? (a.n_tok - l + a.L - 1) / a.L : 0;        // tokens at this position
    const uint32_t lo = min(cut * q.per_cut, rows), hi = min(lo + q.per_cut, rows);
    if (a.acc && rows == 0) continue;                // nothing to add
    float sum[PER][E] = {}, old[PER][E] = {};
    DT* out = static_cast<DT*>(a.dpos) + (uint64_t)l * a.d;
    if (!q.part && a.acc)
#pragma unroll
      for (int i = 0; i < PER; ++i) load_once(out + c[i], old[i]);
    for (uint32_t b = lo; b < hi; b += DEPTH) {
      Ring<DX, E> f[DEPTH][PER];
      bool ok[DEPTH];                                // a bad id's row has no position term, whatever it holds
#pragma unroll
      for (int k = 0; k < DEPTH; ++k) {
        const uint64_t t = (uint64_t)min(b + k, hi - 1) * a.L + l;
        ok[k] = b + k < hi && (uint32_t)__ldg(a.ids + t) < a.V;
#pragma unroll
        for (int i = 0; i < PER; ++i) f[k][i].load(dX + t * a.d + c[i]);
      }
#pragma unroll
      for (int k = 0; k < DEPTH; ++k)
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
          for (int e = 0; e < E; ++e) sum[i][e] += ok[k] ? f[k][i].get(e) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (c0 + i * q.tx * E >= a.d) continue;
      if (q.part) {
        store_kept(q.part + ((uint64_t)cut * a.L + l) * a.d + c[i], sum[i]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) sum[i][e] = a.acc ? old[i][e] + sum[i][e] : sum[i][e];
        store_once(out + c[i], sum[i]);
      }
    }
  }
}

template <class DX, class DT, int E, int PER>
__global__ void __launch_bounds__(kThreads) pos_grad_kernel(const EmbedGradArgs a, const PosArgs q) {
  sum_positions<DX, DT, E, PER>(a, q, (uint64_t)blockIdx.x * blockDim.y + threadIdx.y, (uint64_t)gridDim.x * blockDim.y);
}

// Threads of the join kernels side by side in the columns; the CTA's rows of them share a sum's parts.
template <int E>
constexpr int kSide = E == 1 ? 64 : 16;

// joins the cuts of position l
template <class DT, int E>
__device__ void join_positions(const EmbedGradArgs& a, const PosArgs& q, uint32_t l, uint32_t column_part, float* smem) {
  constexpr int X = kSide<E>, Y = kThreads / X;
  const uint32_t x = threadIdx.x % X, y = threadIdx.x / X, c = (column_part * X + x) * E;
  float sum[E] = {}, old[E] = {};
  if (c < a.d) {
#pragma unroll 4
    for (uint32_t k = y; k < q.cuts; k += Y) {
      float f[E];
      load_once(q.part + ((uint64_t)k * a.L + l) * a.d + c, f);
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] += f[e];
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) smem[(y * X + x) * E + e] = sum[e];
  __syncthreads();
  if (y > 0 || c >= a.d) return;
  DT* out = static_cast<DT*>(a.dpos) + (uint64_t)l * a.d + c;
  if (a.acc) load_once(out, old);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    for (int k = 1; k < Y; ++k) sum[e] += smem[(k * X + x) * E + e];
    sum[e] = a.acc ? old[e] + sum[e] : sum[e];
  }
  store_once(out, sum);
}
template <class DT, int E>
__global__ void __launch_bounds__(kThreads) pos_join_kernel(const EmbedGradArgs a, const PosArgs q) {
  __shared__ float smem[kThreads * E];
  join_positions<DT, E>(a, q, blockIdx.x, blockIdx.y, smem);
}

// One cluster.  Other work beside it (absent rows, positions) made the whole longer: the sort is a chain of L2 latencies,
// which double under load.
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(const EmbedGradArgs a, const SortArgs s) {
  extern __shared__ uint32_t smem[];
  let_next_start();
  sort_tokens(a, s, smem);
}

// ---- sums over the sorted tokens ----
// Part p has the runs that begin in its window of `len` tokens, and the whole of them, so that a short run is one CTA's
// alone.  Only a window that one run fills is a part of that run by itself: the run is cut before it.
struct RunArgs {
  const uint2* list;       // ids and tokens
  float *head, *tail;      // [parts][d]: sum of a part that begins inside a run, of the run that goes on behind a part
  uint32_t len, parts;     // tokens to a window
  __device__ __forceinline__ uint32_t key(uint32_t i) const { return __ldg(&list[i].x); }
  // the run that comes into window q fills it (keys are sorted: its two ends tell)
  __device__ __forceinline__ bool cut(const EmbedGradArgs& a, uint32_t q) const {
    if (q == 0 || q >= parts) return false;
    const uint32_t lo = q * len;
    return key(lo - 1) == key(min(lo + len, a.n_tok) - 1);
  }
};

constexpr uint32_t kMaxPart = 64;

// sets the rows of slice `slice` that no token has to zero: one thread looks each row up in the sorted list
constexpr uint32_t kSlice = 64;
template <class DT, bool VEC>
__device__ void zero_slice(const EmbedGradArgs& a, const RunArgs& r, uint64_t slice) {
  __shared__ uint8_t seen[kSlice];
  const uint32_t v0 = (uint32_t)(slice * kSlice), rows = min(kSlice, a.V - v0);
  const uint32_t tid = threadIdx.y * blockDim.x + threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid < rows) {
    uint32_t lo = 0, hi = a.n_tok;                         // key(lo - 1) < row <= key(hi)
    while (lo < hi) {
      const uint32_t mid = (lo + hi) / 2;
      if (r.key(mid) < v0 + tid) lo = mid + 1; else hi = mid;
    }
    seen[tid] = lo < a.n_tok && r.key(lo) == v0 + tid;
  }
  __syncthreads();
  for (uint32_t i = warp; i < rows; i += blockDim.x * blockDim.y / 32) {
    if (seen[i]) continue;
    DT* row = static_cast<DT*>(a.dT) + (uint64_t)(v0 + i) * a.d;
    if constexpr (VEC) {
      for (uint32_t c = lane; c < a.d * sizeof(DT) / 16; c += 32) __stcs(reinterpret_cast<uint4*>(row) + c, make_uint4(0, 0, 0, 0));
    } else {
      for (uint32_t c = lane; c < a.d; c += 32) row[c] = from_f32<DT>(0.0f);
    }
  }
}

// What the CTAs of the runs kernel do, in each column part: the first `pos_ctas` blocks sum positions, which they can while the
// sort still runs; the next `part_ctas` take parts; the rest, counted through all column parts, set `slices` slices of absent
// rows to zero.
struct Roles {
  uint32_t pos_ctas, part_ctas, slices;
};

// blockDim.x threads share the columns of blockIdx.y's part of a row, PER pieces of E consecutive elements each, blockDim.y parts
// of tokens to a CTA.  A thread has DEPTH rows on their way, as they are stored.  With ACC the row that a run is added to is
// asked for when the last of the run's tokens is: single elements into registers; vectors into L2, to be loaded when the run
// is finished while its sum waits in registers until the next run is.
template <class DX, class DT, int E, int PER, bool ACC>
__global__ void __launch_bounds__(kThreads, ACC ? 3 : 4) embed_runs_kernel(const EmbedGradArgs a, const RunArgs r, const PosArgs q, const Roles ro) {
  let_next_start();
  if (blockIdx.x < ro.pos_ctas) {
    sum_positions<DX, DT, E, PER>(a, q, ((uint64_t)blockIdx.y * ro.pos_ctas + blockIdx.x) * blockDim.y + threadIdx.y,
                                  (uint64_t)ro.pos_ctas * gridDim.y * blockDim.y);
    return;
  }
  wait_for_previous();
  const uint32_t block = blockIdx.x - ro.pos_ctas;
  if (block >= ro.part_ctas) {
    const uint32_t slice = block - ro.part_ctas + blockIdx.y * (gridDim.x - ro.pos_ctas - ro.part_ctas);
    if (slice < ro.slices) zero_slice<DT, (E > 1)>(a, r, slice);
    return;
  }
  constexpr int DEPTH = E == 1 ? 4 : sizeof(DX) == 2 ? 8 : 4;
  extern __shared__ uint2 lists[];
  __shared__ uint32_t starts[kThreads / 8][2];
  const uint32_t p = (ro.part_ctas - 1 - block) * blockDim.y + threadIdx.y;     // rare ids, which write most, first
  const uint32_t c0 = (blockIdx.y * PER * blockDim.x + threadIdx.x) * E;
  // two windows and an element on either side: list[1 + i] is token lo + i
  uint2* list = lists + threadIdx.y * (2 * r.len + 2);
  const uint32_t lo = p * r.len;
  const bool here = p < r.parts;
  const uint32_t all = here ? min(2 * r.len, a.n_tok - lo) : 0;
  if (threadIdx.x < 2) starts[threadIdx.y][threadIdx.x] = 2 * r.len + 1;
  if (here)
    for (uint32_t i = threadIdx.x; i < all + 2; i += blockDim.x) {
      const uint32_t j = lo + i - 1;                       // wraps for the element before the first
      list[i] = j < a.n_tok ? __ldg(r.list + j) : make_uint2(a.V + 1, 0);
    }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < all; i += blockDim.x)
    if (list[1 + i].x != list[i].x) atomicMin(&starts[threadIdx.y][i >= r.len], i);
  __syncthreads();
  if (!here || c0 >= a.d) return;
  // tokens [first, end) of the windows; a window without a beginning is cut at its own
  const uint32_t s0 = starts[threadIdx.y][0], s1 = starts[threadIdx.y][1];
  const bool inside = s0 > 2 * r.len;                      // begins inside a run
  const uint32_t first = inside ? 0 : s0, end = all <= r.len ? all : s1 > 2 * r.len ? r.len : s1;
  const bool goes_on = all > r.len && s1 > 2 * r.len;      // the last run goes on in the next part
  uint32_t cnt = end - first;
  list += 1 + first;
  while (cnt > 0 && list[cnt - 1].x >= a.V) --cnt;         // bad ids are last
  if (cnt == 0) return;
  // pieces behind the row's end load its first one, so that no load needs a condition
  uint32_t c[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) c[i] = c0 + i * blockDim.x * E < a.d ? c0 + i * blockDim.x * E : 0;
  auto has = [&](int i) { return c0 + i * blockDim.x * E < a.d; };
  const DX* dx = static_cast<const DX*>(a.dX);
  const DT* dT = static_cast<const DT*>(a.dT);
  Ring<DX, E> ring[DEPTH][PER];
  Ring<DT, 1> before[ACC && E == 1 ? DEPTH : 1][PER];
  auto ask = [&](int k, uint32_t j) {
    const uint2 t = list[j];
    const DX* row = dx + (uint64_t)t.y * a.d;
#pragma unroll
    for (int i = 0; i < PER; ++i) ring[k][i].load(row + c[i]);
    if constexpr (ACC)
      if (j + 1 == cnt || list[j + 1].x != t.x) {
        const DT* to = dT + (uint64_t)t.x * a.d;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          if constexpr (E == 1) before[k][i].load(to + c[i]);
          else asm volatile("prefetch.global.L2 [%0];" ::"l"(to + c[i]));
        }
      }
  };
#pragma unroll
  for (int k = 0; k < DEPTH; ++k)
    if ((uint32_t)k < cnt) ask(k, k);
  float sum[PER][E] = {}, kept[PER][ACC && E > 1 ? E : 1], old[PER][E] = {};
  uint32_t waiting = ~0u;                                  // ACC, vectors: id of the run in `kept`
  bool head = inside;
  for (uint32_t j0 = 0; j0 < cnt; j0 += DEPTH) {
#pragma unroll
    for (int k = 0; k < DEPTH; ++k) {
      const uint32_t j = j0 + k;
      if (j >= cnt) break;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
#pragma unroll
        for (int e = 0; e < E; ++e) sum[i][e] += ring[k][i].get(e);
        if constexpr (ACC && E == 1) old[i][0] = before[k][i].get(0);
      }
      if (j + DEPTH < cnt) ask(k, j + DEPTH);
      const uint32_t id = list[j].x;
      if (j + 1 == cnt || list[j + 1].x != id) {
        const bool cut = goes_on && j + 1 == end - first;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          if (head || cut) {
            if (has(i)) store_kept((head ? r.head : r.tail) + (uint64_t)p * a.d + c[i], sum[i]);
          } else if constexpr (ACC && E > 1) {
            if (waiting != ~0u) finish_row<DT, E>(a, waiting, c[i], kept[i], old[i]);
            load_once(dT + (uint64_t)id * a.d + c[i], old[i]);
#pragma unroll
            for (int e = 0; e < E; ++e) kept[i][e] = sum[i][e];
          } else {
            if (has(i)) finish_row<DT, E>(a, id, c[i], sum[i], old[i]);
          }
#pragma unroll
          for (int e = 0; e < E; ++e) sum[i][e] = 0.0f;
        }
        if (!head && !cut) waiting = id;
        head = false;
      }
    }
  }
  if constexpr (ACC && E > 1)
    if (waiting != ~0u) finish_row<DT, E>(a, waiting, c[0], kept[0], old[0]);
}

// Joins the runs that were cut.  A CTA looks at kJoin parts for runs that begin there and are cut behind, and sums the columns
// of blockIdx.y's part with kSide threads in the columns and the others over the run's parts.  CTAs behind `run_ctas` join
// positions.
constexpr uint32_t kJoin = 8;
template <class DT, int E>
__global__ void __launch_bounds__(kThreads) embed_join_kernel(const EmbedGradArgs a, const RunArgs r, const PosArgs q, uint32_t run_ctas) {
  __shared__ float smem[kThreads * E];
  wait_for_previous();
  if (blockIdx.x >= run_ctas) {
    join_positions<DT, E>(a, q, blockIdx.x - run_ctas, blockIdx.y, smem);
    return;
  }
  constexpr int X = kSide<E>, Y = kThreads / X;
  const uint32_t lane = threadIdx.x & 31, x = threadIdx.x % X, y = threadIdx.x / X, c = (blockIdx.y * X + x) * E;
  const uint32_t mine = blockIdx.x * kJoin + lane % kJoin;
  // in every warp the same
  const bool cut_here = r.cut(a, mine), cut_behind = r.cut(a, mine + 1);
  uint32_t todo = __ballot_sync(0xFFFFFFFFu, lane < kJoin && cut_behind && !cut_here && r.key((mine + 1) * r.len) < a.V);
  for (; todo; todo &= todo - 1) {
    const uint32_t p = blockIdx.x * kJoin + __ffs(todo) - 1, id = r.key((p + 1) * r.len);
    uint32_t end = p + 1;                                  // the last part that begins inside the run
    for (bool more = true; more;) {
      const uint32_t k = end + 1 + lane;
      const uint32_t in = __ballot_sync(0xFFFFFFFFu, r.cut(a, k) && r.key(k * r.len) == id);
      more = in == 0xFFFFFFFFu;
      end += __popc(in);
    }
    float sum[E] = {}, old[E] = {};
    if (c < a.d) {
      if (a.acc && y == 0) load_once(static_cast<const DT*>(a.dT) + (uint64_t)id * a.d + c, old);
#pragma unroll 4
      for (uint32_t k = p + y; k <= end; k += Y) {
        float f[E];
        load_once((k == p ? r.tail : r.head) + (uint64_t)k * a.d + c, f);
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += f[e];
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) smem[(y * X + x) * E + e] = sum[e];
    __syncthreads();
    if (y == 0 && c < a.d) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        for (int k = 1; k < Y; ++k) sum[e] += smem[(k * X + x) * E + e];
      finish_row<DT, E>(a, id, c, sum, old);
    }
    __syncthreads();
  }
}

// ---- host: sizes that depend on n_tok, L and d alone, so that results do not depend on the device ----
// Tokens to a window: 64, fewer (down to 16) while that leaves less than three CTAs for each SM
inline uint32_t part_len(uint64_t n_tok, uint32_t d) {
  const int e = d % 8 == 0 ? 8 : 1;
  const Columns c(d, e, pieces(e));
  uint32_t len = kMaxPart;
  while (len > 16 && n_tok * c.ctas / (len * c.ty) < 444) len /= 2;
  return len;
}
inline uint32_t pos_cuts(uint64_t n_tok, uint64_t L, uint32_t d) {      // enough CTAs for every SM, eight rows to a cut at least
  const uint64_t rows = (n_tok + L - 1) / L, ctas = L * ((d + 2047) / 2048), want = ctas < 256 ? 1024 / ctas : 1, most = (rows + 7) / 8;
  const uint64_t cuts = want < most ? want : most;
  return cuts < 1 ? 1u : (uint32_t)cuts;
}
inline uint64_t up32(uint64_t n) { return (n + 31) / 32 * 32; }

struct Workspace {
  uint64_t list[2], head, tail, pos, bytes;
  Workspace(uint64_t n, uint32_t d) {
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
      const uint64_t p = at;
      at += up32(bytes);
      return p;
    };
    const bool sorted = n > kDirectMost;
    const uint64_t parts = sorted ? (n + part_len(n, d) - 1) / part_len(n, d) : 0;
    for (int i = 0; i < 2; ++i) list[i] = take(sorted ? 8 * n : 0);
    head = take(4 * parts * d);
    tail = take(4 * parts * d);
    pos = take(4 * (n < 1024 ? n : 1024) * (uint64_t)d);   // cuts * L <= 1024, and never more rows than tokens
    bytes = at < 16 ? 16 : at;
  }
};

template <class DX, class DT, int E>
cudaError_t embed_grad_typed(const EmbedGradArgs& a, cudaStream_t st, int sms) {
  const Workspace w(a.n_tok, a.d);
  char* ws = static_cast<char*>(a.ws);
  const Columns cols(a.d, E, pieces(E));
  const uint32_t slice_rows = 16;                          // rows to a CTA at least when absent rows are set to zero
  PosArgs q{nullptr, 1, 0, cols.tx, cols.ctas};
  if (a.dpos) {
    const uint32_t rows = (uint32_t)(((uint64_t)a.n_tok + a.L - 1) / a.L);
    q.cuts = pos_cuts(a.n_tok, a.L, a.d);
    q.per_cut = (rows + q.cuts - 1) / q.cuts;
    if (q.cuts > 1) q.part = reinterpret_cast<float*>(ws + w.pos);
  }
  const uint64_t pos_groups = a.dpos ? (uint64_t)a.L * q.cuts * q.column_parts : 0;
  const dim3 pos_join(a.L, (a.d + kSide<E> * E - 1) / (kSide<E> * E));
  cudaError_t e;
  if (a.n_tok <= kDirectMost) {
    const uint32_t parts = (a.d + kDirect * E - 1) / (kDirect * E), want = (a.V + slice_rows - 1) / slice_rows;
    const uint32_t most = 8u * sms, slices = a.acc ? 0 : (want < most ? want : most);
    embed_grad_direct_kernel<DX, DT, E><<<a.n_tok * parts + slices, kDirect, 0, st>>>(a, parts, slices);
    if ((e = cudaPeekAtLastError()) != cudaSuccess || !a.dpos) return e;
    const uint64_t ctas = (pos_groups + cols.ty - 1) / cols.ty, fit = 8u * sms;
    pos_grad_kernel<DX, DT, E, pieces(E)><<<(uint32_t)(ctas < fit ? ctas : fit), dim3(cols.tx, cols.ty), 0, st>>>(a, q);
    if (q.part) pos_join_kernel<DT, E><<<pos_join, kThreads, 0, st>>>(a, q);
    return cudaPeekAtLastError();
  }
  SortArgs s;
  int bits = 0;
  while (bits < 32 && (a.V >> bits) != 0) ++bits;          // ids and V itself
  s.passes = (bits + kDigitBits - 1) / kDigitBits;
  s.bits = (bits + s.passes - 1) / s.passes;
  for (int i = 0; i < 2; ++i) s.list[i] = reinterpret_cast<uint2*>(ws + w.list[i]);
  auto sort_smem = [](int digit_bits) { return ((size_t)((kSortWarps + 1) << digit_bits) + kSortWarps) * 4; };
  const size_t smem = sort_smem(s.bits);
  // the limit belongs to the process: the same value in every call, so that none lowers it under another thread's launch
  if ((e = cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sort_smem(kDigitBits))) != cudaSuccess)
    return e;
  if ((e = cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) != cudaSuccess) return e;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = kSortCtas;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kSortCtas);
  cfg.blockDim = dim3(kSortThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if ((e = cudaLaunchKernelEx(&cfg, embed_sort_kernel, a, s)) != cudaSuccess) return e;
  RunArgs r;
  r.list = s.list[0];
  r.head = reinterpret_cast<float*>(ws + w.head);
  r.tail = reinterpret_cast<float*>(ws + w.tail);
  r.len = part_len(a.n_tok, a.d);
  r.parts = (a.n_tok + r.len - 1) / r.len;
  Roles ro;
  ro.part_ctas = (r.parts + cols.ty - 1) / cols.ty;
  ro.slices = a.acc ? 0 : (a.V + kSlice - 1) / kSlice;
  const uint64_t pos_ctas = (pos_groups + (uint64_t)cols.ty * cols.ctas - 1) / ((uint64_t)cols.ty * cols.ctas), most = 8u * sms;
  ro.pos_ctas = (uint32_t)(pos_ctas < most ? pos_ctas : most);
  const dim3 grid(ro.pos_ctas + ro.part_ctas + (ro.slices + cols.ctas - 1) / cols.ctas, cols.ctas), block(cols.tx, cols.ty);
  const size_t lists = cols.ty * (2 * r.len + 2) * sizeof(uint2);
  e = a.acc ? launch_behind(embed_runs_kernel<DX, DT, E, pieces(E), true>, grid, block, lists, st, a, r, q, ro)
            : launch_behind(embed_runs_kernel<DX, DT, E, pieces(E), false>, grid, block, lists, st, a, r, q, ro);
  if (e != cudaSuccess) return e;
  const uint32_t run_ctas = (r.parts + kJoin - 1) / kJoin;
  return launch_behind(embed_join_kernel<DT, E>, dim3(run_ctas + (q.part ? a.L : 0), pos_join.y), dim3(kThreads), 0, st, a, r, q, run_ctas);
}

}  // namespace

cudaError_t launch_embed_lookup(const LookupArgs& a, int table_type, int x_type, cudaStream_t st) {
  cudaError_t e;
  const int sms = sm_count(&e);
  if (e != cudaSuccess) return e;
  auto ok = [&](const void* p) { return vector_aligned(p, table_type); };
  const bool vec = a.d % 8 == 0 && ok(a.T_S) && ok(a.T_perp) && ok(a.pos) && vector_aligned(a.X, x_type);
  // Two pieces to a thread from 16 threads a row on (split bf16 tables, 64K x 2048 elements in rows of d: d = 256: 64 against
  // 80 us with one, 1024: 70 against 87; f32 tables: 117 against 127 and 137 against 148, but 153 against 107 at d = 64).
  const bool wide = vec && a.d >= 256;
  // Slabs of columns, each over all tokens, where a token's rows would leave L2 before their next token comes: the rows of one
  // slab stay.  64K x 2048, both tables, float32: 150 -> 135 us with V = 32000, 156 -> 141 us with 50257 (155 with slabs of up
  // to 64 MB, that is with none there); bfloat16 81 -> 74 us.  Widths that leave lanes of a group idle lose it again (384: 154 us),
  // hence powers of two, and rows that are not aligned keep one slab (d = 1537: 236 us, 259 with slabs).
  LookupOrder o;
  const uint64_t rows = a.V < a.n_tok ? a.V : a.n_tok, column = rows * (table_type == SL_F32 ? 4 : 2) * (a.T_perp ? 2 : 1);
  o.width = a.d;
  if (vec && column * a.d > kSlab && column * kSlabColumns <= kSlab)
    for (o.width = kSlabColumns; column * o.width * 2 <= kSlab;) o.width *= 2;
  const uint32_t slabs = (a.d + o.width - 1) / o.width;
  const Columns cols(o.width, vec ? 8 : 1, vec ? (wide ? 2 : 1) : 8);
  const dim3 block(cols.tx, cols.ty);
  o.B = a.pos ? (uint32_t)(((uint64_t)a.n_tok + a.L - 1) / a.L) : 1;
  const uint64_t places = (uint64_t)(a.pos ? a.L : a.n_tok) * o.B, fit = (uint64_t)sms * 5 * block.y;
  // tokens in a row: a position's, while every group still has some
  o.run = 1;
  while (o.run < 16 && places * slabs / (2 * o.run) >= fit) o.run *= 2;
  const uint64_t units = (places + o.run - 1) / o.run, want = (units * slabs + block.y - 1) / block.y, most = (uint64_t)sms * 8;
  const uint32_t grid = (uint32_t)(want < most ? want : most);
  o.units = (uint32_t)units;
  return with_type(table_type, [&](auto tb) {
    return with_type(x_type, [&](auto xt) {
      using TB = decltype(tb);
      using XT = decltype(xt);
      if (wide) embed_lookup_kernel<TB, XT, 8, 2><<<grid, block, 0, st>>>(a, o);
      else if (vec) embed_lookup_kernel<TB, XT, 8, 1><<<grid, block, 0, st>>>(a, o);
      else embed_lookup_kernel<TB, XT, 1, 8><<<grid, block, 0, st>>>(a, o);
      return cudaPeekAtLastError();
    });
  });
}

uint64_t embed_grad_workspace(uint64_t n_tok, uint64_t, uint32_t d) { return Workspace(n_tok, d).bytes; }

static bool embed_grad_vectors(const EmbedGradArgs& a, int dx_type, int dt_type) {
  return a.d % 8 == 0 && vector_aligned(a.dX, dx_type) && vector_aligned(a.dT, dt_type) && vector_aligned(a.dpos, dt_type);
}

// the join kernel of many tokens deals out columns along a grid's second axis, which ends at 65,535 (few tokens' positions are cut
// only where rows are narrow)
bool embed_grad_fits(const EmbedGradArgs& a, int dx_type, int dt_type) {
  if (a.n_tok <= kDirectMost) return true;
  const uint32_t columns = embed_grad_vectors(a, dx_type, dt_type) ? kSide<8> * 8 : kSide<1>;
  return (a.d + columns - 1) / columns <= 65535;
}

cudaError_t launch_embed_grad(const EmbedGradArgs& a, int dx_type, int dt_type, cudaStream_t st) {
  cudaError_t err;
  const int sms = sm_count(&err);
  if (err != cudaSuccess) return err;
  const bool vec = embed_grad_vectors(a, dx_type, dt_type);
  return with_type(dx_type, [&](auto dx) {
    return with_type(dt_type, [&](auto dt) {
      using DX = decltype(dx);
      using DT = decltype(dt);
      return vec ? embed_grad_typed<DX, DT, 8>(a, st, sms) : embed_grad_typed<DX, DT, 1>(a, st, sms);
    });
  });
}

}  // namespace sl
