// mikv_flash.cu — attention over bf16 / fp16 keys: work plan, tensor maps, merge of split parts and dispatch (the
// kernels are in mikv_flash.cuh).
#include <limits.h>
#include <string.h>

#include <mutex>

#include "mikv_flash.cuh"

namespace mikv {
namespace {

using flash::kTile;

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

// Map of a 16-bit tensor of 128 channels and three more dimensions (element strides; a zero stride makes the
// dimension one entry long: its coordinate is then 0).
bool encode_rows(CUtensorMap* map, bool f16, const void* data, const long long (&n)[3], const long long (&stride)[3],
                 const uint32_t (&box)[3]) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  cuuint64_t dims[4] = {kHeadDim, 1, 1, 1};
  cuuint64_t strides[3];
  cuuint32_t boxes[4] = {64, box[0], box[1], box[2]};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  for (int i = 0; i < 3; ++i) {
    dims[i + 1] = stride[i] ? (cuuint64_t)n[i] : 1;
    strides[i] = stride[i] ? 2 * (cuuint64_t)stride[i] : 2 * kHeadDim;
  }
  return enc(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(data),
             dims, strides, boxes, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Plan {
  int mode;  // flash::Mode
  int m_blocks, item_rows;
  int shares;  // CTAs that share the key tiles out among them; 0: whole row tiles
};

// Row tiles below this number may be shared out: above it a share would hold more than two row tiles' worth of keys, and
// whole row tiles leave little idle. 280 row tiles of few rows with 8000 keys: 170 us shared, 164 whole; 300: 182 and
// 174; 310, where a third round begins: 187 and 217; 400: 238 and 233. With 1000 keys whole tiles win from 200 on (28
// and 27 us; 288: 34 and 29).
long long most_shared(int num_sms) { return 2ll * num_sms; }

// Whole row tiles or shares, and for how many CTAs: what an estimate of the time makes shortest. A CTA has its tiles and
// a start and end per item; shares add the merge, whose time is mostly the traffic of the parts, and its table, which the
// first CTA writes set by set beside its items. The constants are nanoseconds on an idle GB300: those of a tile and of the
// table are measured, kItem is an estimate (2500 and 3500 choose alike). Against fixed numbers of CTAs (0, eighths and
// multiples of the row tiles up to 152) the choice was within 4 % of the best on twenty shapes: 32 requests on 32768
// keys of 8 heads 128 CTAs 32.3 us (whole 223, 152 CTAs 34.1); one request on 4096 keys 128 CTAs 12.0 (whole 30.0, 64
// CTAs 12.4); 160 row tiles of 8000 keys 133 CTAs 103 (whole 138); 240 of 1000 keys whole 27 (152 CTAs 31).
Plan plan_flash(int batch, int heads_kv, int G, int tq, int tk, int num_sms) {
  Plan p;
  const long long rows = (long long)tq * G;
  const bool pair = rows > kTile;
  p.mode = pair ? flash::kPair : rows > flash::Layout<flash::kFew>::kRows ? flash::kOne : flash::kFew;
  p.item_rows = pair ? 2 * kTile : p.mode == flash::kOne ? kTile : flash::Layout<flash::kFew>::kRows;
  p.m_blocks = (int)((rows + p.item_rows - 1) / p.item_rows);
  const long long base = (long long)batch * heads_kv * p.m_blocks;
  const long long tiles = ((long long)tk + kTile - 1) / kTile, units = base * tiles;
  p.shares = 0;
  if (base >= most_shared(num_sms) || units >= INT_MAX - 4 * num_sms) return p;
  // a tile: the products and softmax, or its 64 KB at the SM's share of HBM
  auto tile_ns = [&](double busy) { return pair ? 1600.0 : 9.7 * busy > 1150.0 ? 9.7 * busy : 1150.0; };
  constexpr double kItem = 5000.0;  // start and end of an item
  // 160 sets of one head and 1000 keys: 55 us shared, 26 whole; 40 sets of four: 24 and 26
  const double table = 4000.0 + 350.0 * batch;
  const double rounds = (double)((base + num_sms - 1) / num_sms);
  double best = rounds * (tiles * tile_ns(base < num_sms ? base : num_sms) + kItem);
  const double part_rows = rows < p.item_rows ? rows : p.item_rows;
  auto consider = [&](int c) {
    if (c < 1 || c > num_sms || c <= base / 2 || 2 * (long long)c > units) return;  // (a tile for each stream at least)
    const double items = c % base == 0 ? 1.0 : 2.0 + (double)(base / c);  // the most that a share holds
    const double run = (double)((units + c - 1) / c) * tile_ns(c) + kItem * items;
    const double cost = (run > table ? run : table) + 5000.0 + ((double)c + base) * part_rows * kHeadDim * 4.0 / 3000.0;
    if (cost < best) best = cost, p.shares = c;
  };
  for (int eighths = 1; eighths <= 8; ++eighths) consider(num_sms * eighths / 8);
  for (long long c = 2 * base; c <= num_sms; c += base) consider((int)c);
  return p;
}

struct MergePartsArgs {
  FlashArgs a;
  const int2* table;
  const float* part_o;
  const float* part_lse;
  int rows, m_blocks, log2_item_rows, log2_G, out_kind;  // (out_kind: 0 bf16, 1 fp16, 2 fp32)
};

// The parts of an output row weighted by 2^(lse - largest), then the join with the request's own part. W warps share a
// row (more than eight parts: four), each with up to eight parts at a time; their sums and outputs are asked for
// together (a part that has seen nothing holds anything: it is left out by its sum).
template <int W>
__global__ void __launch_bounds__(128) merge_parts_kernel(const __grid_constant__ MergePartsArgs m) {
  const FlashArgs& a = m.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = W == 1 ? blockIdx.x * 4 + warp : blockIdx.x;  // (set * tq + token) * heads_q + head
  const int first = W == 1 ? 0 : warp;
  __shared__ float s_top[4], s_sum[4];
  __shared__ float4 s_acc[4][32];
  const int bt = row / a.heads_q, head = row - bt * a.heads_q, b = bt / a.tq, token = bt - b * a.tq;
  const int kv = head >> m.log2_G, in_head = (token << m.log2_G) + (head & (a.G - 1));
  const int tile = (b * a.heads_kv + kv) * m.m_blocks + (in_head >> m.log2_item_rows);
  grid_dependency_wait();
  if (W == 1 && row >= m.rows) return;
  const int2 share = m.table[tile];
  const long long at0 = ((long long)(share.x + tile) << m.log2_item_rows) + (in_head & ((1 << m.log2_item_rows) - 1));
  float top = -INFINITY, sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = first; s0 < share.y; s0 += 8 * W) {
    float e[8];
    float4 o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int s = s0 + W * i;
      const long long at = at0 + ((long long)s << m.log2_item_rows);
      e[i] = s < share.y ? m.part_lse[at] : -INFINITY;
      o[i] = s < share.y ? __ldcs(reinterpret_cast<const float4*>(m.part_o + at * kHeadDim) + lane)
                         : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    float next = top;
#pragma unroll
    for (int i = 0; i < 8; ++i) next = fmaxf(next, e[i]);
    const float c = top == -INFINITY ? 0.f : fast_exp2(top - next);
    sum *= c;
    acc.x *= c, acc.y *= c, acc.z *= c, acc.w *= c;
    top = next;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (e[i] == -INFINITY) continue;
      const float w = fast_exp2(e[i] - top);
      sum += w;
      acc.x = fmaf(o[i].x, w, acc.x);
      acc.y = fmaf(o[i].y, w, acc.y);
      acc.z = fmaf(o[i].z, w, acc.z);
      acc.w = fmaf(o[i].w, w, acc.w);
    }
  }
  if constexpr (W > 1) {
    if (lane == 0) s_top[warp] = top, s_sum[warp] = sum;
    s_acc[warp][lane] = acc;
    __syncthreads();
    if (warp > 0) return;
    top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    sum = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if (s_top[i] == -INFINITY && s_sum[i] == 0.f) continue;
      const float w = fast_exp2(s_top[i] - top);
      const float4 o = s_acc[i][lane];
      sum = fmaf(s_sum[i], w, sum);
      acc.x = fmaf(o.x, w, acc.x);
      acc.y = fmaf(o.y, w, acc.y);
      acc.z = fmaf(o.z, w, acc.z);
      acc.w = fmaf(o.w, w, acc.w);
    }
  }
  float lse2 = sum == 0.f ? -INFINITY : top + log2f(sum);
  float f0 = sum == 0.f ? 0.f : 1.f / sum, f1 = 0.f;
  if (a.own_out) flash::join_own(a, row, lse2, f0, f1);
  float v[4] = {acc.x * f0, acc.y * f0, acc.z * f0, acc.w * f0};
  if (f1 != 0.f) {
    const float4 o = reinterpret_cast<const float4*>(a.own_out + row * kHeadDim)[lane];
    v[0] = fmaf(o.x, f1, v[0]);
    v[1] = fmaf(o.y, f1, v[1]);
    v[2] = fmaf(o.z, f1, v[2]);
    v[3] = fmaf(o.w, f1, v[3]);
  }
  const long long at = b * a.o_b + head * a.o_h + token * a.o_t + 4 * lane;
  if (m.out_kind == 2)
    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(v[0], v[1], v[2], v[3]);
  else
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at) =
        m.out_kind == 1 ? make_uint2(pack_f16(v[0], v[1]), pack_f16(v[2], v[3]))
                        : make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  if (lane == 0) flash::store_stat(a, b * a.s_b + head * a.s_h + token * a.s_t, lse2);
}

}  // namespace

// Room for the parts of every plan that keys up to tk may get: it depends on the row tiles alone.
size_t flash_workspace_bytes(int batch, int heads_kv, int G, int tq, int tk, int num_sms) {
  const Plan p = plan_flash(batch, heads_kv, G, tq, 0, num_sms);
  const long long base = (long long)batch * heads_kv * p.m_blocks;
  if (base >= most_shared(num_sms) || tk == 0) return kWsHeader;
  const size_t slots = (size_t)(base + num_sms);
  return kWsHeader + (base * sizeof(int2) + 255) / 256 * 256 + slots * p.item_rows * (kHeadDim + 1) * sizeof(float);
}

bool flash_fits(int batch, int heads_kv, int G, int tq) {
  const double blocks = ((double)tq * G + 2 * kTile - 1) / (2 * kTile);
  return (double)batch * heads_kv * blocks < 2.0e9 && (double)batch * tq * heads_kv * G < 8.0e9;
}

cudaError_t launch_flash(const FlashArgs& a, bool f16, bool out_f32, void* ws, int num_sms, cudaStream_t st) {
  const Plan plan = plan_flash(a.batch, a.heads_kv, a.G, a.tq, a.tk, num_sms);
  FlashKernelArgs p;
  memset(&p, 0, sizeof p);
  p.a = a;
  p.out_f32 = out_f32;
  const int heads = a.batch * a.heads_kv;
  const int base = heads * plan.m_blocks;
  p.m_blocks = plan.m_blocks;
  p.n_items = base;
  p.log2_G = a.G == 1 ? 0 : a.G == 2 ? 1 : a.G == 4 ? 2 : 3;
  if (plan.shares) {
    const size_t slots = (size_t)base + num_sms;
    p.shares = plan.shares;
    p.by_length = a.lens && !a.spans && !a.causal;
    p.units = (int)(((long long)a.tk + kTile - 1) / kTile);
    p.share_each = (int)((long long)base * p.units / p.shares);
    p.share_extra = (int)((long long)base * p.units % p.shares);
    p.inv_units = 1.f / (float)p.units;
    p.by_units.set(p.units);
    p.by_set.set(a.heads_kv * plan.m_blocks);
    p.by_block.set(plan.m_blocks);
    char* at = static_cast<char*>(ws) + kWsHeader;
    p.part_table = reinterpret_cast<int2*>(at);
    p.part_o = reinterpret_cast<float*>(at + ((size_t)base * sizeof(int2) + 255) / 256 * 256);
    p.part_lse = p.part_o + slots * plan.item_rows * kHeadDim;
  }
  if (a.tk > 0) {
    p.k_batch = a.k_b != 0, p.k_head = a.k_h != 0, p.v_batch = a.v_b != 0, p.v_head = a.v_h != 0;
    const uint32_t box_q[3] = {(uint32_t)a.G, (uint32_t)((plan.mode == flash::kFew ? flash::Layout<flash::kFew>::kRows : kTile) / a.G), 1},
                   box_k[3] = {(uint32_t)kTile, 1, 1};
    if (!encode_rows(&p.map_q, f16, a.q, {a.heads_q, a.tq, a.batch}, {a.q_h, a.q_t, a.q_b}, box_q) ||
        !encode_rows(&p.map_k, f16, a.k, {a.tk, a.heads_kv, a.batch}, {a.k_t, a.k_h, a.k_b}, box_k) ||
        !encode_rows(&p.map_v, f16, a.v, {a.tk, a.heads_kv, a.batch}, {a.v_t, a.v_h, a.v_b}, box_k))
      return cudaErrorInvalidValue;
  }
  // heads worked on together: as many as have their keys and values in half of L2, and enough to occupy every SM
  const long long l2_heads = (64ll << 20) / ((long long)a.tk * kHeadDim * 4 + 1) + 1;
  const long long busy_heads = (num_sms + (long long)plan.m_blocks - 1) / plan.m_blocks;
  const long long group = l2_heads > busy_heads ? l2_heads : busy_heads;
  p.group_heads = group < heads ? (int)group : heads;
  const int over = heads % p.group_heads;
  p.by_group.set(p.group_heads * plan.m_blocks);
  p.by_rank.set(p.group_heads);
  p.by_last.set(over ? over : p.group_heads);
  p.by_head.set(a.heads_kv);
  const int grid = p.shares ? p.shares : p.n_items < num_sms ? p.n_items : num_sms;
  cudaError_t e = f16 ? launch_flash_kernel<true>(p, plan.mode, grid, st) : launch_flash_kernel<false>(p, plan.mode, grid, st);
  if (e != cudaSuccess || !p.shares) return e;
  MergePartsArgs m = {a, p.part_table, p.part_o, p.part_lse, a.batch * a.tq * a.heads_q, plan.m_blocks, 0, p.log2_G, out_f32 ? 2 : f16 ? 1 : 0};
  while ((1 << m.log2_item_rows) < plan.item_rows) ++m.log2_item_rows;
  // Four warps to a row where parts are many and rows few (one warp / four warps, whole call): 4 rows of 32 parts 14.7 /
  // 12.0 us, 1024 rows of 16 parts 33.9 / 32.1, 2048 rows of 19 parts 44.1 / 42.4; but 4096 rows of 9 parts 60.9 / 64.3,
  // and 240 rows of 4 parts 44.8 / 46.0.
  if (p.shares > 8 * base && m.rows <= 2048)
    return launch_chained(merge_parts_kernel<4>, dim3(m.rows), dim3(128), 0, st, m);
  return launch_chained(merge_parts_kernel<1>, dim3((m.rows + 3) / 4), dim3(128), 0, st, m);
}

}  // namespace mikv
