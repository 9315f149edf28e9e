// mikv_tree.cu — drafted tokens: what the nodes of a tree see of one another, and their attention over the
// mixed-precision cache.
#include <math.h>
#include <string.h>

#include <mutex>

#include "mikv_tree_few.cuh"

namespace mikv {
namespace {

// One block per request: every thread walks from its node up to the root through the parents in shared memory (128 steps
// at most; a chain of 128 takes 4 us, and the masks serve all layers of a step).
__global__ void __launch_bounds__(kTreeNodes) tree_masks_kernel(uint4* masks, int32_t* positions, const int32_t* parents,
                                                                int nodes, const int32_t* first, int start) {
  __shared__ int up[kTreeNodes];
  const int b = blockIdx.x, i = threadIdx.x;
  grid_dependency_wait();
  allow_dependent_launch();
  if (i < nodes) up[i] = parents[(size_t)b * nodes + i];
  __syncthreads();
  if (i >= nodes) return;
  uint32_t m[4] = {0u, 0u, 0u, 0u};
  int depth = -1;
  for (int j = i; j >= 0;) {
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if ((j >> 5) == w) m[w] |= 1u << (j & 31);
    ++depth;
    const int p = up[j];
    if (p < -1 || p >= j) {  // no node, or below one that is none
      depth = -1;
      break;
    }
    j = p;
  }
  const bool node = depth >= 0;
  masks[(size_t)b * nodes + i] = node ? make_uint4(m[0], m[1], m[2], m[3]) : make_uint4(0u, 0u, 0u, 0u);
  if (positions) positions[(size_t)b * nodes + i] = (first ? first[b] : start) + max(depth, 0);
}

using tree::Runs;
using tree::Tiles;

struct TreeMergeArgs {
  TreeArgs a;
  const uint32_t* prefix;
  const float *part_o, *part_lse;
  int m_blocks, log2_G, log2_rows, ctas, lo_blocks;
};

// How an item's units lie in the runs: key tiles by their costs, or the units of few rows, one like another.
struct TileRuns {
  Tiles tl;
  Runs runs;
  __device__ TileRuns(const TreeMergeArgs& m, int b) : tl(m.a.held, b), runs(m.prefix[m.a.batch], m.ctas) {}
  __device__ int cost() const { return tl.cost(); }
  __device__ int last() const { return tl.before(tl.count() - 1); }
  __device__ bool part(int from, int to) const { return tl.first(from) < tl.first(to); }
};
struct FewRuns {
  tree::FewUnits n;
  Runs runs;
  __device__ FewRuns(const TreeMergeArgs& m, int b)
      : n(m.a.held, m.a.nodes, b, m.lo_blocks), runs(m.prefix[m.a.batch], m.ctas, tree::kFewLeast) {}
  __device__ int cost() const { return n.cost(); }
  __device__ int last() const { return n.before(n.count() - 1); }
  __device__ bool part(int from, int to) const { return n.first(from) < n.first(to); }
};

// The parts of an output row, weighted by 2^(lse - largest): a warp to a row. Rows whose item one CTA had are written.
constexpr int kMergeRows = 4;
template <typename R>
__global__ void __launch_bounds__(32 * kMergeRows) tree_merge_kernel(const __grid_constant__ TreeMergeArgs m) {
  const TreeArgs& a = m.a;
  const int lane = threadIdx.x & 31;
  const int b = blockIdx.y, row = blockIdx.x * kMergeRows + (threadIdx.x >> 5);  // node * heads_q + head
  grid_dependency_wait();
  const int node = row / a.heads_q, head = row - node * a.heads_q;
  if (node >= a.nodes) return;
  const int h = head >> m.log2_G, in_head = (node << m.log2_G) + (head & (a.G - 1));
  const int block = in_head >> m.log2_rows, in_item = in_head & ((1 << m.log2_rows) - 1);
  const R item(m, b);
  const Runs& runs = item.runs;
  const uint32_t start = m.prefix[b] + (uint32_t)(h * m.m_blocks + block) * item.cost();
  const int c0 = runs.owner(start), c1 = runs.owner(start + item.last());
  if (c0 == c1) return;
  float top = -INFINITY, sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int first = c0; first <= c1; first += 32) {
    const int c = first + lane;
    const long long at = ((long long)(2 * c + (c == c0)) << m.log2_rows) + in_item;
    bool part = c <= c1;
    if (part) part = item.part((int)(runs.first(c) - start), (int)(runs.first(c + 1) - start));
    const float e = part ? m.part_lse[at] : -INFINITY;
    float next = fmaxf(top, e);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) next = fmaxf(next, __shfl_xor_sync(0xffffffffu, next, o));
    const float old = top == -INFINITY ? 0.f : fast_exp2(top - next);
    sum *= old;
    acc.x *= old, acc.y *= old, acc.z *= old, acc.w *= old;
    top = next;
    const float w = e == -INFINITY ? 0.f : fast_exp2(e - top);
    uint32_t parts = __ballot_sync(0xffffffffu, part && e != -INFINITY);
    while (parts) {
      float wi[8];
      float4 o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {  // (eight loads on their way at a time)
        const int i = __ffs(parts) - 1;
        parts &= parts - 1;
        wi[k] = __shfl_sync(0xffffffffu, w, i & 31);
        o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < 0)
          wi[k] = 0.f;
        else
          o[k] = reinterpret_cast<const float4*>(m.part_o + (((long long)(2 * (first + i) + (first + i == c0)) << m.log2_rows) + in_item) * kHeadDim)[lane];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        sum += wi[k];
        acc.x = fmaf(o[k].x, wi[k], acc.x);
        acc.y = fmaf(o[k].y, wi[k], acc.y);
        acc.z = fmaf(o[k].z, wi[k], acc.z);
        acc.w = fmaf(o[k].w, wi[k], acc.w);
      }
    }
  }
  const float f = sum == 0.f ? 0.f : 1.f / sum;
  const long long to = b * a.out.b + head * a.out.h + node * a.out.t + 4 * lane;
  if (a.out_f32)
    *reinterpret_cast<float4*>(static_cast<float*>(a.out.p) + to) = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
  else
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out.p) + to) =
        make_uint2(pack_bf16(acc.x * f, acc.y * f), pack_bf16(acc.z * f, acc.w * f));
  if (a.lse && lane == 0)
    a.lse[((size_t)b * a.heads_q + head) * a.nodes + node] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * flash::kLn2;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(p);
  });
  return fn;
}

// Map of a bf16 tensor of 128 channels and up to three more dimensions (element strides; 0 where a dimension has one
// entry), box 64 channels x `rows` entries of the next dimension.
bool encode_rows(CUtensorMap* map, const void* data, int dims, const long long (&n)[3], const long long (&stride)[3],
                 int rows = tree::kTile) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  cuuint64_t size[4] = {kHeadDim, 1, 1, 1}, strides[3];
  const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1}, one[4] = {1, 1, 1, 1};
  for (int i = 0; i < 3; ++i) {
    size[i + 1] = (cuuint64_t)n[i];
    strides[i] = stride[i] ? 2 * (cuuint64_t)stride[i] : 2 * kHeadDim;
  }
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dims, const_cast<void*>(data), size, strides, box, one,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Which kernel: few rows stay in registers (mikv_tree_few.cuh), more go through tensor memory. 16 requests of 8192 tokens, 8
// KV heads: 16 rows 89 us against 125, 32 rows (two blocks of 16) 147 against 127. A small cache takes tensor memory for all
// rows, since an item costs the other kernel as much as 100 tokens: 32 KV heads, 8 rows: 512 tokens 18.7 us against 16.0,
// 2048 29.6 against 25.5, 8192 35.1 against 34.9, 16384 47 against 68. (The size is the cache's, not what it holds: the
// workspace depends on it.)
constexpr int kFewMost = 16;
constexpr long long kFewTokens = 1 << 18;

struct Sizes {
  bool few, narrow, pair;
  int rows, item_rows, m_blocks;
  Sizes(int G, int nodes, long long tokens) : rows(G * nodes) {
    few = rows <= kFewMost && tokens > kFewTokens;
    narrow = rows <= 8;
    pair = rows > tree::kTile;
    item_rows = few ? tree::kFewRows : pair ? 2 * tree::kTile : tree::kTile;
    m_blocks = (rows + item_rows - 1) / item_rows;
  }
  int runs(int num_sms) const {
    return num_sms * (!few ? 1 : narrow ? tree::FewShape<true>::kWarps : tree::FewShape<false>::kWarps);
  }
  size_t parts(int num_sms) const { return (size_t)2 * runs(num_sms); }
};

size_t prefix_bytes(int batch) { return ((batch + 1) * sizeof(uint32_t) + 255) / 256 * 256; }

}  // namespace

cudaError_t launch_tree_masks(uint4* masks, int32_t* positions, const int32_t* parents, int batch, int nodes,
                              const int32_t* first, int start, cudaStream_t st) {
  return launch_chained(tree_masks_kernel, dim3(batch), dim3(kTreeNodes), 0, st, masks, positions, parents, nodes, first,
                        start);
}

bool tree_sizes_ok(const mikv_shape& s, int nodes) {
  const Sizes z(s.heads_q / s.heads_kv, nodes, (long long)s.batch * s.heads_kv * (s.hi_stride + (long long)s.lo_cap));
  const long long slots = (long long)s.batch * s.heads_kv * s.hi_stride, rows = (long long)s.batch * s.heads_q * nodes;
  const long long items = (long long)s.batch * s.heads_kv * z.m_blocks;  // of either kernel's costs:
  return slots < 1ll << 31 && rows < 1ll << 31 && items * (32 + ((long long)nodes + s.hi_cap + s.lo_cap) / 16) < 1ll << 32;
}

size_t tree_workspace_bytes(const mikv_shape& s, int nodes, int num_sms) {
  const Sizes z(s.heads_q / s.heads_kv, nodes, (long long)s.batch * s.heads_kv * (s.hi_stride + (long long)s.lo_cap));
  return kWsHeader + prefix_bytes(s.batch) + z.parts(num_sms) * z.item_rows * (kHeadDim + 1) * sizeof(float);
}

cudaError_t launch_tree(const TreeArgs& a, void* ws, int num_sms, cudaStream_t st) {
  const Sizes z(a.G, a.nodes, (long long)a.batch * a.heads_kv * (a.hi_stride + (long long)a.lo_cap));
  const int log2_G = a.G == 1 ? 0 : a.G == 2 ? 1 : a.G == 4 ? 2 : 3;
  char* at = static_cast<char*>(ws) + kWsHeader;
  uint32_t* prefix = reinterpret_cast<uint32_t*>(at);
  float* part_o = reinterpret_cast<float*>(at + prefix_bytes(a.batch));
  float* part_lse = part_o + z.parts(num_sms) * z.item_rows * kHeadDim;
  const long long rows = (long long)a.batch * a.heads_kv * a.hi_stride;
  CUtensorMap k_hi, v_hi;
  memset(&k_hi, 0, sizeof k_hi);
  memset(&v_hi, 0, sizeof v_hi);
  const int box = z.few ? 16 : tree::kTile;
  if (rows > 0 && (!encode_rows(&k_hi, a.k_hi, 2, {rows, 1, 1}, {kHeadDim, 0, 0}, box) ||
                   !encode_rows(&v_hi, a.v_hi, 2, {rows, 1, 1}, {kHeadDim, 0, 0}, box)))
    return cudaErrorInvalidValue;
  TreeMergeArgs m = {a, prefix, part_o, part_lse, z.m_blocks, log2_G, 31 - __builtin_clz(z.item_rows), num_sms, 0};
  const dim3 merge_grid((a.nodes * a.heads_q + kMergeRows - 1) / kMergeRows, a.batch);
  if (z.few) {
    TreeFewArgs p;
    memset(&p, 0, sizeof p);
    p.map_k_hi = k_hi, p.map_v_hi = v_hi;
    p.a = a;
    p.rows = z.rows, p.row_blocks = z.m_blocks, p.log2_G = log2_G;
    p.prefix = prefix, p.part_o = part_o, p.part_lse = part_lse;
    const cudaError_t e = a.bits == 2   ? launch_tree_few<2>(p, z.narrow, num_sms, st)
                          : a.bits == 3 ? launch_tree_few<3>(p, z.narrow, num_sms, st)
                                        : launch_tree_few<4>(p, z.narrow, num_sms, st);
    if (e != cudaSuccess) return e;
    m.ctas = z.runs(num_sms);
    m.lo_blocks = a.bits == 2   ? tree::FewUnit<2>(a.group).blocks
                  : a.bits == 3 ? tree::FewUnit<3>(a.group).blocks
                                : tree::FewUnit<4>(a.group).blocks;
    return launch_chained(tree_merge_kernel<FewRuns>, merge_grid, dim3(32 * kMergeRows), 0, st, m);
  }
  TreeKernelArgs p;
  memset(&p, 0, sizeof p);
  p.map_k_hi = k_hi, p.map_v_hi = v_hi;
  p.a = a;
  p.rows = z.rows;
  p.m_blocks = z.m_blocks;
  p.twin = z.rows <= tree::kTile / 2;
  p.log2_G = log2_G;
  p.prefix = prefix, p.part_o = part_o, p.part_lse = part_lse;
  if (!encode_rows(&p.map_k, a.k.p, 4, {a.nodes, a.heads_kv, a.batch}, {a.k.t, a.k.h, a.k.b}) ||
      !encode_rows(&p.map_v, a.v.p, 4, {a.nodes, a.heads_kv, a.batch}, {a.v.t, a.v.h, a.v.b}))
    return cudaErrorInvalidValue;
  const cudaError_t e = a.bits == 2   ? launch_tree_kernel<2>(p, z.pair, num_sms, st)
                        : a.bits == 3 ? launch_tree_kernel<3>(p, z.pair, num_sms, st)
                                      : launch_tree_kernel<4>(p, z.pair, num_sms, st);
  if (e != cudaSuccess) return e;
  return launch_chained(tree_merge_kernel<TileRuns>, merge_grid, dim3(32 * kMergeRows), 0, st, m);
}

}  // namespace mikv
