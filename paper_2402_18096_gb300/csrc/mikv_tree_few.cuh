// mikv_tree_few.cuh — attention of drafted tokens over the mixed-precision cache where a KV head has few query rows: codes
// go from shared memory through registers into mma.sync, without a tile of dequantized keys in between.
// mikv_tree_f2.cu, mikv_tree_f3.cu and mikv_tree_f4.cu instantiate it for one code width each.
//
// Why not the tensor-memory kernel: its tiles have 128 rows, its codes are written to and read from shared memory as
// fp16 (ten times their size), and 16 rows of 128 are an eighth of what its products cost.
//
// Work. Rows r = node * G + head in blocks of 8 or 16 (FewShape); an item is a row block of one KV head. Its units are 16
// nodes, 16 important slots, or as many blocks of 16 retained rows as fit a stage of 8 KB. All items' units are laid
// end to end and every warp of the grid takes an equal run of them, as the CTAs do in mikv_tree_kernel.cuh; the same
// second kernel merges what lies in several runs. A warp shares nothing with the others: its own two or three stages,
// filled by copies (bulk copies of code rows, swizzled boxes of bf16 rows) that it asks for one or two units ahead.
//
// A block of 16 tokens. Codes enter both products as they lie: a field's bits under a zero exponent are the fp16 number
// code 2^(s - 24), s the field's place, exactly; one LOP3 makes a pair of operands.
//   S = sum over the groups of alpha_g (sum over the group's channels of q^ code) + beta_g (sum of q^), q^ = q / balancer:
//       a chain of MMAs per group, alpha and beta in fp32 afterwards. The keys are never rounded. q^ stands in two fp16
//       terms (22 bits; rounded to one it would be off alike for all keys, 1e-5 of lse), scaled by 2^-s per field.
//   O += (P alpha_g) code: P = 2^(x - r) in fp16 times the tokens' alpha, per group; what beta adds is P beta_g, one more MMA
//       whose other side are the groups, added to the group's channels at the end. O of channels 16 m .. is kept in units of
//       2^(s_m - 24) meanwhile, and of 2^ev for alphas far from 1.
// With alpha and beta applied to every key and value in fp16 (two more instructions a pair) the same kernel took 182 us where
// this one took 149, 16 requests of 205 .. 8192 tokens, 40 heads, 3 bits. Now 128 (3.6 TB/s, 53 % of a copy): bound by the
// instructions of a block (390, with three warps a scheduler that wait for their own results).
// Tokens 2 t and 2 t + 1 of an operand are rows t and t + 4 of their eight, so that eight lanes read four rows of codes from
// different banks.
#pragma once

#include "mikv_tree_kernel.cuh"

namespace mikv {

struct TreeFewArgs {
  CUtensorMap map_k_hi, map_v_hi;  // bf16 [batch * heads * hi_stride][128], box 64 channels x 16 rows, 128B swizzle
  TreeArgs a;
  int rows, row_blocks, log2_G;
  uint32_t* prefix;
  float* part_o;    // [2 * warps][16][128]
  float* part_lse;  // [2 * warps][16], log2
};

template <int BITS>
cudaError_t launch_tree_few(const TreeFewArgs& p, bool narrow, int grid, cudaStream_t st);

namespace tree {

constexpr int kFewRows = 16, kFewStage = 8192;  // rows of a part; bytes of a stage
constexpr int kFewItem = 6;  // cost of an item beside its units (its queries, its output)

// Narrow: up to 8 rows, which are the N side of the MMAs, and the tokens (scores) or channels (output) the M side. Half
// the MMAs and half the registers of 16 rows as the M side, hence 12 warps on an SM and not 8.
template <bool NARROW>
struct FewShape {
  static constexpr int kRows = NARROW ? 8 : 16, kWarps = NARROW ? 12 : 8, kStages = NARROW ? 2 : 3;
};
constexpr int kFewLeast = 2;  // units of a run at least

// Blocks of 16 retained rows in a unit, and where its arrays lie in a stage.
template <int BITS>
struct FewUnit {
  int blocks, v, kp, vp, row_bytes;
  __host__ __device__ explicit FewUnit(int group) : row_bytes(4 * kHeadDim / group) {
    const int block = 2 * 16 * (16 * BITS + row_bytes);
    blocks = kFewStage / block < 5 ? kFewStage / block : 5;
    v = blocks * 16 * 16 * BITS;
    kp = 2 * v;
    vp = kp + blocks * 16 * row_bytes;
  }
};

// Units of a request's items: nodes, slots, retained rows; and their costs for the runs, one for 16 tokens of any kind (a
// block of codes takes as many instructions as two of slots, which take three times its bytes from HBM).
struct FewUnits {
  int nodes, hi, lo, blocks;  // blocks: cost of a unit of retained rows
  __device__ FewUnits(const HeldArgs& held, int n_nodes, int b, int lo_blocks)
      : nodes((n_nodes + 15) / 16), hi((held.hi(b) + 15) / 16), lo((held.lo(b) + 16 * lo_blocks - 1) / (16 * lo_blocks)),
        blocks(lo_blocks) {}
  __device__ int count() const { return nodes + hi + lo; }
  __device__ int before(int u) const {
    return u == 0 ? 0 : kFewItem + min(u, nodes + hi) + blocks * max(0, u - nodes - hi);
  }
  __device__ int cost() const { return before(count()); }
  // the first unit that begins at x or later
  __device__ int first(int x) const {
    if (x <= 0) return 0;
    x = max(1, x - kFewItem);
    return min(count(), x <= nodes + hi ? x : nodes + hi + (x - nodes - hi + blocks - 1) / blocks);
  }
};

__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 r;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(addr));
  return r;
}
__device__ __forceinline__ uint32_t lds32v(uint32_t addr) {
  uint32_t r;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r) : "r"(addr));
  return r;
}

// Code fields m of both 16-bit halves of a word: the fp16 numbers code 2^(place(m) - 24). A field has to lie in the 10 bits
// of the mantissa, so the upper ones are read from the words shifted.
template <int BITS>
struct FieldOf {
  static constexpr int kWords = BITS == 2 ? 1 : 2;
  uint32_t lo[kWords], up[kWords];
  // x, y: the word, and for 4 bits the second word (fields 4 ..), for 3 bits the word of the high bits (at bit 2 m): even
  // and odd fields are brought together with their high bits, 4 bits to a field
  __device__ __forceinline__ FieldOf(uint32_t x, uint32_t y) {
    lo[0] = x;
    if constexpr (BITS == 4) lo[1] = y;
    if constexpr (BITS == 3) lo[0] = merge(x, y << 2), lo[1] = merge(x >> 2, y);
#pragma unroll
    for (int i = 0; i < kWords; ++i) up[i] = lo[i] >> 8;
  }
  static __device__ __forceinline__ uint32_t merge(uint32_t low, uint32_t high) { return (low & 0x33333333u) | (high & ~0x33333333u); }
  static __host__ __device__ constexpr int field(int m) { return BITS == 2 ? m : BITS == 3 ? m >> 1 : m & 3; }  // in its word
  static __host__ __device__ constexpr int place(int m) { return (BITS == 2 ? 2 : 4) * field(m) & 7; }
  __device__ __forceinline__ uint32_t code(int m) const {
    const int i = BITS == 2 ? 0 : BITS == 3 ? m & 1 : m >> 2, at = (BITS == 2 ? 2 : 4) * field(m);
    return (at >= 8 ? up[i] : lo[i]) & (((1u << BITS) - 1u) * 0x10001u << place(m));
  }
};
// 1 / x to 2^-22: the queries stand in 22 bits beside it
__device__ __forceinline__ float fast_inverse(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float fast_log2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// The parameters of a token.
template <int PAIRS>
__device__ __forceinline__ void load_pairs(uint32_t addr, uint32_t (&p)[PAIRS]) {
  if constexpr (PAIRS == 4) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(p[0]), "=r"(p[1]), "=r"(p[2]), "=r"(p[3]) : "r"(addr));
  } else if constexpr (PAIRS == 2) {
    const uint2 x = lds64(addr);
    p[0] = x.x, p[1] = x.y;
  } else {
    p[0] = lds32v(addr);
  }
}

template <int BITS, int PAIRS, bool NARROW>
__global__ void __launch_bounds__(32 * FewShape<NARROW>::kWarps, 1) tree_few_kernel(const __grid_constant__ TreeFewArgs p) {
  constexpr int kFewWarps = FewShape<NARROW>::kWarps, kFewStages = FewShape<NARROW>::kStages, kRows = FewShape<NARROW>::kRows;
  const TreeArgs& a = p.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t s_bar[kFewWarps][kFewStages];
  __shared__ float s_rel[kFewWarps][4][kRows];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const uint32_t stages = ((smem_u32(smem_raw) + 1023u) & ~1023u) + warp * (kFewStages * kFewStage);
  const uint32_t bars = smem_u32(&s_bar[warp][0]);
  if (lane < kFewStages) mbar_init(bars + 8 * lane, 1);
  fence_mbar_init();
  __syncwarp();
  if (lane == 0) {
    prefetch_tensormap(&p.map_k_hi);
    prefetch_tensormap(&p.map_v_hi);
  }
  grid_dependency_wait();
  allow_dependent_launch();
  const FewUnit<BITS> U(kHeadDim / PAIRS);
  constexpr int kOf = 8 / PAIRS;  // fields of 16 channels to a pair of parameters
  const int lo_rows = 16 * U.blocks, per_set = a.heads_kv * p.row_blocks;
  auto units_of = [&](int b) { return FewUnits(a.held, a.nodes, b, U.blocks); };

  // This warp's run of all units.
  auto scan = [&](int b0, uint32_t& mine) {
    mine = b0 + lane < a.batch ? units_of(b0 + lane).cost() * per_set : 0;
    uint32_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    return sum;
  };
  const int me = warp * gridDim.x + blockIdx.x;  // (few runs: on all SMs)
  uint32_t all = 0, mine;
#pragma unroll 1
  for (int b0 = 0; b0 < a.batch; b0 += 32) {
    const uint32_t sum = scan(b0, mine);
    if (me == 0 && b0 + lane < a.batch) p.prefix[b0 + lane] = all + sum - mine;
    all += __shfl_sync(0xffffffffu, sum, 31);
  }
  if (me == 0 && lane == 0) p.prefix[a.batch] = all;
  const Runs runs(all, gridDim.x * kFewWarps, kFewLeast);
  if (me >= runs.n) return;
  const uint32_t from = runs.first(me);
  uint32_t begin = 0;  // costs before the item
  int b = 0, in_set = 0;
#pragma unroll 1
  for (int b0 = 0; b0 < a.batch; b0 += 32) {
    const uint32_t sum = scan(b0, mine), total = __shfl_sync(0xffffffffu, sum, 31);
    if (from < begin + total) {
      const int at = __ffs(__ballot_sync(0xffffffffu, begin + sum > from)) - 1;
      b = b0 + at;
      begin += __shfl_sync(0xffffffffu, sum - mine, at);
      const uint32_t cost = units_of(b).cost();
      in_set = (int)((from - begin) / cost);
      begin += in_set * cost;
      break;
    }
    begin += total;
  }

  int start = (int)(begin - from);  // from here on relative to the run's begin
  const int to = (int)(runs.first(me + 1) - from);
  // The unit that is asked for next: its place, and the stage it goes to.
  struct Place {
    int b, in_set, u;
    FewUnits n;
  };
  int ask_start = start;  // costs before its item
  Place ask = {b, in_set, 0, units_of(b)};
  ask.u = ask.n.first(-start);
  bool more = ask_start + ask.n.before(ask.u) < to;
  int ask_stage = 0, stage = 0;    // of the unit asked for next, of the one worked on next
  uint32_t parity = 0, copies = 0; // per stage: of the copy taken next; whether the unit in it was copied
  auto next_ask_item = [&]() {
    ask_start += ask.n.cost();
    ask.u = 0;
    if (++ask.in_set == per_set) {
      ask.in_set = 0;
      if (++ask.b < a.batch) ask.n = units_of(ask.b);
    }
  };
  auto ask_next = [&]() {
    if (!more) return;
    const int s = ask_stage, bh = ask.b * a.heads_kv + ask.in_set / p.row_blocks;
    ask_stage = s + 1 == kFewStages ? 0 : s + 1;
    const uint32_t at = stages + s * kFewStage, bar = bars + 8 * s;
    copies = (copies & ~(1u << s)) | (ask.u >= ask.n.nodes ? 1u << s : 0u);
    if (lane == 0 && ask.u >= ask.n.nodes) {
      if (ask.u < ask.n.nodes + ask.n.hi) {
        const int row = bh * a.hi_stride + 16 * (ask.u - ask.n.nodes);
        mbar_arrive_expect_tx(bar, kFewStage);
        tma_load_2d(at, &p.map_k_hi, 0, row, bar);
        tma_load_2d(at + 2048, &p.map_k_hi, 64, row, bar);
        tma_load_2d(at + 4096, &p.map_v_hi, 0, row, bar);
        tma_load_2d(at + 6144, &p.map_v_hi, 64, row, bar);
      } else {
        const int r0 = (ask.u - ask.n.nodes - ask.n.hi) * lo_rows;
        const int rows = min(lo_rows, (a.held.lo(ask.b) - r0 + 15) & ~15);  // (a multiple of 16: lo_cap is one)
        const size_t row = (size_t)bh * a.lo_cap + r0;
        const uint32_t codes = rows * 16 * BITS, params = rows * U.row_bytes;
        mbar_arrive_expect_tx(bar, 2 * (codes + params));
        bulk_load(at, a.k_codes + row * 16 * BITS, codes, bar);
        bulk_load(at + U.v, a.v_codes + row * 16 * BITS, codes, bar);
        bulk_load(at + U.kp, reinterpret_cast<const char*>(a.k_params) + row * U.row_bytes, params, bar);
        bulk_load(at + U.vp, reinterpret_cast<const char*>(a.v_params) + row * U.row_bytes, params, bar);
      }
    }
    if (++ask.u == ask.n.count()) next_ask_item();
    more = ask.b < a.batch && ask_start + ask.n.before(ask.u) < to;
  };
  if (ask.u == ask.n.count()) {  // (the run begins within the item's last unit)
    next_ask_item();
    more = ask.b < a.batch && ask_start < to;
  }
#pragma unroll 1
  for (int i = 1; i < kFewStages; ++i) ask_next();

  constexpr float kDrop = flash::ref_drop<true>(), kSlack = flash::ref_slack<true>();
  const float scale = a.sm_scale * kLog2e;
  bool ok = true;
#pragma unroll 1
  for (; ok && start < to; ) {  // an item
    const FewUnits n = units_of(b);
    const int count = n.count(), u0 = n.first(-start), u1 = n.first(to - start);
    if (u0 == u1) {  // (none of its units begins in this run)
      start += n.cost();
      if (++in_set == per_set) in_set = 0, ++b;
      continue;
    }
    const int h = in_set / p.row_blocks, block = in_set - h * p.row_blocks, bh = b * a.heads_kv + h;
    const int n_hi = a.held.hi(b), n_lo = a.held.lo(b), free_slot = a.held.free_slot(bh, n_hi);
    // The lane's rows: g and g + 8, or (narrow) 2 t and 2 t + 1; the queries that it holds are those of rows g and g + 8, or
    // (narrow) of row g alone.
    int node[2], head[2];
    bool there[2], real[2];
    const __nv_bfloat16* query[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int R = block * kRows + (NARROW ? 2 * t + r : g + 8 * r);
      there[r] = R < p.rows;
      node[r] = there[r] ? R >> p.log2_G : 0;
      head[r] = h * a.G + (R & (a.G - 1));
      const uint32_t word = reinterpret_cast<const uint32_t*>(a.masks + (size_t)b * a.nodes + node[r])[node[r] >> 5];
      real[r] = there[r] && (word >> (node[r] & 31) & 1);
      query[r] = static_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.b + head[r] * a.q.h + node[r] * a.q.t;
    }
    bool asks[2] = {real[0], real[1]};
    if constexpr (NARROW) {
      const int R = block * kRows + g, i = R < p.rows ? R >> p.log2_G : 0;
      const uint32_t word = reinterpret_cast<const uint32_t*>(a.masks + (size_t)b * a.nodes + i)[i >> 5];
      asks[0] = R < p.rows && (word >> (i & 31) & 1), asks[1] = false;
      query[0] = static_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.b + (h * a.G + (R & (a.G - 1))) * a.q.h + i * a.q.t;
    }
    constexpr int kHeld = NARROW ? 1 : 2, kO = NARROW ? 8 : 16;
    float ob[4] = {0.f, 0.f, 0.f, 0.f};  // P beta: by groups g (narrow), or rows by groups 2 t, 2 t + 1
    float qs[PAIRS][2];                  // sums of the groups' q^, in units of 2^24 products
    bool spread = false;                 // 32 channels of q^ have a scale of their own (s_rel, beside the row's)
    float alpha_most = -1.f;             // 2^(ev + 6): O is in units of 2^ev (retained rows)
    __half2 unit = u32_as_h2(0u);        // 2^-ev, 2^6 at most
    float o[kO][4], ref[2], sum[2] = {0.f, 0.f}, scale_lo[2] = {0.f, 0.f};
    bool poisoned[2] = {false, false};
#pragma unroll
    for (int i = 0; i < kO; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
    ref[0] = real[0] ? -INFINITY : 0.f, ref[1] = real[1] ? -INFINITY : 0.f;
    uint32_t q[8][2 * kHeld], q2[8][2 * kHeld];  // the queries as operands; the second terms (retained rows)
    int form = -1;               // what q holds: 0 bf16 for nodes and slots, 1 fp16 for retained rows

    // Weights of a block's scores s[half of the tokens][register], packed as the operand of the second product; see(half,
    // parity, row): whether the row sees the token. The lane's tokens are 2 t + parity of a half, or (narrow) row g of a
    // half. A reference that is missing or too low moves, and O with it.
    auto weigh = [&](float (&s)[2][4], const float (&sc)[2], bool masked, auto see, uint32_t (&pk)[4], auto f16) {
      // (narrow: registers 0 and 1 are token g of the first half, rows 2 t and 2 t + 1; 2 and 3 token g of the second)
      auto row_of = [](int half, int e) { return NARROW ? e & 1 : e >> 1; };
      if (masked) {
#pragma unroll
        for (int i = 0; i < (NARROW ? 1 : 2); ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!see(NARROW ? e >> 1 : i, e & 1, row_of(i, e))) s[i][e] = -INFINITY;
      }
      float top[2];
#pragma unroll
      for (int r = 0; r < 2; ++r)
        top[r] = (NARROW ? fmaxf(s[0][r], s[0][2 + r])
                         : fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]))) * sc[r];
      if (__any_sync(0xffffffffu, top[0] > ref[0] + kSlack || top[1] > ref[1] + kSlack)) {
        float f[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float x = top[r];
#pragma unroll
          for (int off = NARROW ? 4 : 1; off < (NARROW ? 32 : 4); off <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
          const float next = x > ref[r] + kSlack ? x - kDrop : ref[r];
          f[r] = ref[r] == -INFINITY ? 0.f : fast_exp2(ref[r] - next);
          sum[r] *= f[r];
          ref[r] = next;
        }
#pragma unroll
        for (int i = 0; i < kO; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][e] *= f[row_of(0, e)];
#pragma unroll
        for (int e = 0; e < 4; ++e) ob[e] *= f[row_of(0, e)];
      }
      float w[2][4];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float less = ref[r] == -INFINITY ? 0.f : -ref[r];
        if constexpr (NARROW) {
          w[0][r] = fast_exp2(fmaf(s[0][r], sc[r], less)), w[0][2 + r] = fast_exp2(fmaf(s[0][2 + r], sc[r], less));
          sum[r] += w[0][r] + w[0][2 + r];
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[r][i] = fast_exp2(fmaf(s[i >> 1][2 * r + (i & 1)], sc[r], less));
          sum[r] += (w[r][0] + w[r][1]) + (w[r][2] + w[r][3]);
          pk[r] = flash::pack16<decltype(f16)::value>(w[r][0], w[r][1]);
          pk[2 + r] = flash::pack16<decltype(f16)::value>(w[r][2], w[r][3]);
        }
      }
      if constexpr (NARROW) {  // tokens g by rows 2 t, 2 t + 1, turned into rows g by tokens 2 t, 2 t + 1
        pk[0] = movmatrix_t(flash::pack16<decltype(f16)::value>(w[0][0], w[0][1]));
        pk[1] = movmatrix_t(flash::pack16<decltype(f16)::value>(w[0][2], w[0][3]));
      }
    };

#pragma unroll 1
    for (int u = u0; ok && u < u1; ++u) {
      ask_next();
      const int s = stage;
      stage = s + 1 == kFewStages ? 0 : s + 1;
      const uint32_t at = stages + s * kFewStage;
      if (copies >> s & 1) {
        ok = mbar_wait(bars + 8 * s, parity >> s & 1);
        ok = __all_sync(0xffffffffu, ok);
        parity ^= 1u << s;
        if (!ok) break;
      }
      if (u < n.nodes + n.hi) {  // bf16 keys and values: [K | V][64 channels][16 rows of 128 bytes], swizzled
        const bool is_node = u < n.nodes;
        if (form != 0) {
          form = 0;
#pragma unroll
          for (int r = 0; r < kHeld; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // 16 bytes: steps 2 i and 2 i + 1
              uint4 x = make_uint4(0u, 0u, 0u, 0u);
              if (asks[r]) x = __ldg(reinterpret_cast<const uint4*>(query[r] + 64 * (i >> 1) + 8 * (2 * t + (i & 1))));
              q[2 * i][r] = x.x, q[2 * i][kHeld + r] = x.y, q[2 * i + 1][r] = x.z, q[2 * i + 1][kHeld + r] = x.w;
            }
        }
        const int first = 16 * (is_node ? u : u - n.nodes);
        uint32_t seen[2] = {0xffffu, 0xffffu};  // of the 16 keys, by rows g and g + 8
        bool masked = false;
        if (is_node) {  // staged here: rows of padding as zeros, and those that hold an infinity or NaN
          uint32_t bad = 0;
          const int row = lane >> 1;  // two lanes to a node, eight chunks of 16 bytes of its key and of its value each
          const int j = first + row;
          bool node_real = false;
          if (j < a.nodes)
            node_real = reinterpret_cast<const uint32_t*>(a.masks + (size_t)b * a.nodes + j)[j >> 5] >> (j & 31) & 1;
          uint4 x[8];
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const TreeView& view = kv ? a.v : a.k;
            const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(view.p) + b * view.b + h * view.h + j * view.t) + 8 * (lane & 1);
            bool is_bad = false;
#pragma unroll
            for (int c = 0; c < 8; ++c) x[c] = node_real ? __ldg(src + c) : make_uint4(0u, 0u, 0u, 0u);
            if (kv) {
#pragma unroll
              for (int c = 0; c < 8; ++c) is_bad |= flash::any_nonfinite<false>(x[c]);
              is_bad |= __shfl_xor_sync(0xffffffffu, (int)is_bad, 1) != 0;
              bad = __ballot_sync(0xffffffffu, is_bad);  // two bits to a node
            }
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const uint4 y = is_bad ? make_uint4(0u, 0u, 0u, 0u) : x[c];
              sts128(at + 4096 * kv + 2048 * (lane & 1) + row * 128 + ((c ^ (row & 7)) << 4), y.x, y.y, y.z, y.w);
            }
          }
          asm volatile("" ::: "memory");
          masked = true;
          uint32_t bad16 = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) bad16 |= (bad >> (2 * i) & 1u) << i;
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const uint32_t word = reinterpret_cast<const uint32_t*>(a.masks + (size_t)b * a.nodes + node[r])[u >> 1];
            seen[r] = real[r] ? (word >> (16 * (u & 1))) & 0xffffu : 0u;
            poisoned[r] |= (seen[r] & bad16) != 0u;
          }
        } else {
          const int left = n_hi - first;
          uint32_t live = left >= 16 ? 0xffffu : (1u << left) - 1u;
          if (free_slot >= first && free_slot < first + 16) live &= ~(1u << (free_slot - first));
          seen[0] = seen[1] = live;
          masked = live != 0xffffu;
          if (masked) {  // values of slots that hold nothing: any bits
            const int row = lane >> 1;
            if (!(live >> row & 1)) {
#pragma unroll
              for (int c = 0; c < 8; ++c) flash::sts128_zero(at + 4096 + 2048 * (lane & 1) + row * 128 + (c << 4));
            }
          }
        }
        __syncwarp();
        float sc[2][4] = {}, sc2[2][4] = {};  // (chains of MMAs: an MMA waits 30 clocks for the one it adds to)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t k[2][4];
#pragma unroll
          for (int half = 0; half < 2; ++half)
            lds_vec(at + 2048 * (i >> 1) + (8 * half + g) * 128 + (((2 * t + (i & 1)) ^ g) << 4), k[half]);
          if constexpr (NARROW) {
            const uint32_t k0[4] = {k[0][0], k[1][0], k[0][1], k[1][1]}, k1[4] = {k[0][2], k[1][2], k[0][3], k[1][3]};
            mma_bf16(sc[0], k0, q[2 * i][0], q[2 * i][1]);
            mma_bf16(sc2[0], k1, q[2 * i + 1][0], q[2 * i + 1][1]);
          } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              mma_bf16(sc[half], q[2 * i], k[half][0], k[half][1]);
              mma_bf16(sc2[half], q[2 * i + 1], k[half][2], k[half][3]);
            }
          }
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[half][e] += sc2[half][e];
        uint32_t pk[4];
        const float c2[2] = {scale, scale};
        weigh(sc, c2, masked, [&](int half, int parity, int r) { return seen[r] >> (8 * half + (NARROW ? g : 2 * t + parity)) & 1; }, pk,
              std::false_type{});
#pragma unroll
        for (int i = 0; i < 8; ++i) {  // 16 channels: two n-blocks
          uint32_t v[4];
          const int row = (lane & 7) + 8 * ((lane >> 3) & 1), c = 2 * i + (lane >> 4);
          ldsm_x4_t(at + 4096 + 2048 * (c >> 3) + row * 128 + (((c & 7) ^ (row & 7)) << 4), v);
          if constexpr (NARROW) {
            const uint32_t vt[4] = {v[0], v[2], v[1], v[3]};
            mma_bf16(o[i], vt, pk[0], pk[1]);
          } else {
            mma_bf16(o[2 * i], pk, v[0], v[1]);
            mma_bf16(o[2 * i + 1], pk, v[2], v[3]);
          }
        }
        if (masked) fence_async();  // (the stage was written here; a copy comes next)
      } else {  // codes
        if (form != 1) {
          form = 1;
          float x[kHeld][8][4], top[kHeld][4] = {};  // (by 32 channels)
#pragma unroll
          for (int m = 0; m < 8; ++m) {
            float4 inv = make_float4(1.f, 1.f, 1.f, 1.f);
            if (a.balancer) {
              const float4 bal = __ldg(reinterpret_cast<const float4*>(a.balancer + h * kHeadDim + 16 * m + 4 * t));
              inv = make_float4(fast_inverse(bal.x), fast_inverse(bal.y), fast_inverse(bal.z), fast_inverse(bal.w));
            }
#pragma unroll
            for (int r = 0; r < kHeld; ++r) {
              uint2 raw = make_uint2(0u, 0u);
              if (asks[r]) raw = __ldg(reinterpret_cast<const uint2*>(query[r] + 16 * m + 4 * t));
              x[r][m][0] = __uint_as_float(raw.x << 16) * inv.x, x[r][m][1] = __uint_as_float(raw.x & 0xffff0000u) * inv.y;
              x[r][m][2] = __uint_as_float(raw.y << 16) * inv.z, x[r][m][3] = __uint_as_float(raw.y & 0xffff0000u) * inv.w;
#pragma unroll
              for (int e = 0; e < 4; ++e) top[r][m >> 1] = fmaxf(top[r][m >> 1], fabsf(x[r][m][e]));
            }
          }
          // Their powers of two, 2^e for the row: the terms of a channel 2^-8 below the largest are as good as its own, so the
          // row's is used for all 128 until 32 channels lie lower; then each 32 take their own.
          auto exponent = [](float y) { return min(max((int)(__float_as_uint(y) >> 23) - 127, -100), 100) - 14; };
          bool low = false;
          float most[kHeld];
#pragma unroll
          for (int r = 0; r < kHeld; ++r) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              top[r][j] = fmaxf(top[r][j], __shfl_xor_sync(0xffffffffu, top[r][j], 1));
              top[r][j] = fmaxf(top[r][j], __shfl_xor_sync(0xffffffffu, top[r][j], 2));
            }
            most[r] = fmaxf(fmaxf(top[r][0], top[r][1]), fmaxf(top[r][2], top[r][3]));
            low |= fminf(fminf(top[r][0], top[r][1]), fminf(top[r][2], top[r][3])) < 0x1p-8f * most[r];
          }
          spread = __any_sync(0xffffffffu, low);
          __syncwarp();
#pragma unroll
          for (int r = 0; r < kHeld; ++r) {
            const int e2 = exponent(most[r]);
            scale_lo[r] = scale * power2(e2) * 0x1p24f;
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
              float all = 0.f;
#pragma unroll
              for (int m = kOf * i; m < kOf * (i + 1); ++m) all += (x[r][m][0] + x[r][m][1]) + (x[r][m][2] + x[r][m][3]);
              all += __shfl_xor_sync(0xffffffffu, all, 1);
              all += __shfl_xor_sync(0xffffffffu, all, 2);
              qs[i][r] = all * power2(-e2) * 0x1p-24f;
            }
#pragma unroll
            for (int m = 0; m < 8; ++m) {
              const int ej = spread ? max(exponent(top[r][m >> 1]), e2 - 100) : e2;
              if (spread && !(m & 1) && t == 0) s_rel[warp][m >> 1][g + 8 * r] = power2(ej - e2);
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float d = power2(-ej) * power2(-FieldOf<BITS>::place(m)), y0 = x[r][m][2 * e] * d, y1 = x[r][m][2 * e + 1] * d;
                const __half2 near = __floats2half2_rn(y0, y1);
                const float2 f = __half22float2(near);
                q[m][kHeld * e + r] = h2_as_u32(near);
                q2[m][kHeld * e + r] = pack_f16(y0 - f.x, y1 - f.y);
              }
            }
          }
          __syncwarp();
          if constexpr (NARROW) {
            auto turn = [&](float mine, float& r0, float& r1) {
              r0 = __shfl_sync(0xffffffffu, mine, 8 * t), r1 = __shfl_sync(0xffffffffu, mine, 8 * t + 4);
            };
            turn(scale_lo[0], scale_lo[0], scale_lo[1]);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) turn(qs[i][0], qs[i][0], qs[i][1]);
          }
#pragma unroll
          for (int i = 0; i < kO; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] *= power2(FieldOf<BITS>::place(NARROW ? i : i >> 1) - 24);
        }
        const int r0 = (u - n.nodes - n.hi) * lo_rows, blocks = min(U.blocks, (n_lo - r0 + 15) >> 4);
        constexpr int kPitch = 16 * BITS;
        // rows of a block in the order of the operand's columns: 2 t and 2 t + 1 are t and t + 4
        const int krow = (g >> 1) + 4 * (g & 1);
#pragma unroll 1
        for (int blk = 0; blk < blocks; ++blk) {
          const int valid = n_lo - (r0 + 16 * blk);  // rows of the block
          const uint32_t kc = at + blk * 16 * kPitch, kp = at + U.kp + blk * 16 * U.row_bytes;
          const uint32_t vc = at + U.v + blk * 16 * kPitch, vp = at + U.vp + blk * 16 * U.row_bytes;
          const bool masked = valid < 16;
          // scores: codes of rows krow of both halves, channels 16 m + 4 t .. 4 t + 3
          float sc[2][4] = {};
          {
            float part[NARROW ? 1 : 2][4][4] = {};  // by 32 channels
            uint2 x[2], y[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const int row = 8 * half + krow;
              x[half] = lds64(kc + row * kPitch + 8 * t);
              y[half] = make_uint2(0u, 0u);
              if constexpr (BITS == 4) y[half] = lds64(kc + row * kPitch + 32 + 8 * t);
              if constexpr (BITS == 3) {
                y[half] = lds64(kc + row * kPitch + 32 + 8 * (t & 1));
                y[half].x >>= t >> 1, y[half].y >>= t >> 1;
              }
            }
            const FieldOf<BITS> f[2][2] = {{FieldOf<BITS>(x[0].x, y[0].x), FieldOf<BITS>(x[0].y, y[0].y)},
                                           {FieldOf<BITS>(x[1].x, y[1].x), FieldOf<BITS>(x[1].y, y[1].y)}};
#pragma unroll
            for (int odd = 0; odd < 2; ++odd)
#pragma unroll
              for (int term = 0; term < 2; ++term)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const int m = 2 * j + odd;
                  const uint32_t k[2][2] = {{f[0][0].code(m), f[0][1].code(m)}, {f[1][0].code(m), f[1][1].code(m)}};
                  if constexpr (NARROW) {
                    const uint32_t kt[4] = {k[0][0], k[1][0], k[0][1], k[1][1]};
                    mma_f16(part[0][j], kt, term ? q2[m][0] : q[m][0], term ? q2[m][1] : q[m][1]);
                  } else {
#pragma unroll
                    for (int half = 0; half < 2; ++half) mma_f16(part[half][j], term ? q2[m] : q[m], k[half][0], k[half][1]);
                  }
                }
            // alpha and beta of the lane's tokens: row krow of both halves, or (16 rows) the columns 2 t and 2 t + 1
            if (spread) {
#pragma unroll
              for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                  const float f = s_rel[warp][j][NARROW ? 2 * t + r : g + 8 * r];
#pragma unroll
                  for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int half = 0; half < (NARROW ? 1 : 2); ++half) part[half][j][NARROW ? 2 * i + r : 2 * r + i] *= f;
                }
            }
            if constexpr (PAIRS < 4) {
#pragma unroll
              for (int half = 0; half < (NARROW ? 1 : 2); ++half)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  part[half][0][e] += part[half][1][e];
                  part[half][1][e] = part[half][2][e] + part[half][3][e];
                  if constexpr (PAIRS == 1) part[half][0][e] += part[half][1][e];
                }
            }
#pragma unroll
            for (int i = 0; i < (NARROW ? 2 : 4); ++i) {  // token: half i (narrow), or half i >> 1 and column 2 t + (i & 1)
              uint32_t pr[PAIRS];
              load_pairs(kp + (NARROW ? 8 * i + krow : 8 * (i >> 1) + t + 4 * (i & 1)) * U.row_bytes, pr);
#pragma unroll
              for (int j = 0; j < PAIRS; ++j) {
                const float2 ab = __half22float2(u32_as_h2(pr[j]));
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                  const int half = NARROW ? 0 : i >> 1, e = NARROW ? 2 * i + r : 2 * r + (i & 1);
                  sc[half][e] = fmaf(ab.x, part[half][j][e], fmaf(ab.y, qs[j][r], sc[half][e]));
                }
              }
            }
          }
          uint32_t pk[4];
          weigh(sc, scale_lo, masked, [&](int half, int parity, int) { return 8 * half + (NARROW ? krow : t + 4 * parity) < valid; }, pk,
                std::true_type{});
          // values: the parameters of tokens 2 t and 2 t + 1 of both halves; beta of group g to every lane g
          __half2 al[2][PAIRS], most = u32_as_h2(0u);
          uint32_t be[2];
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint32_t pa[PAIRS], pb[PAIRS];
            const int ra = 8 * half + t, rb = ra + 4, j = min(g, PAIRS - 1);
            load_pairs(vp + ra * U.row_bytes, pa);
            load_pairs(vp + rb * U.row_bytes, pb);
            uint32_t ba = lds32v(vp + ra * U.row_bytes + 4 * j), bb = lds32v(vp + rb * U.row_bytes + 4 * j);
            if (masked) {  // (rows behind the last: any bits)
#pragma unroll
              for (int i = 0; i < PAIRS; ++i) pa[i] = ra < valid ? pa[i] : 0u, pb[i] = rb < valid ? pb[i] : 0u;
              ba = ra < valid ? ba : 0u, bb = rb < valid ? bb : 0u;
            }
            be[half] = g < PAIRS ? prmt(ba, bb, 0x7632u) : 0u;
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
              al[half][i] = u32_as_h2(prmt(pa[i], pb[i], 0x5410u));
              most = __hmax2(most, __habs2(al[half][i]));
            }
          }
          // P alpha 2^-ev enters, P up to 2^8.5 and alpha up to 2^(ev + 6); the first block chooses ev. The power has to lie
          // on the factor that stays inside fp16: on P it brings P alpha down where ev > 0, and up to P 2^6 = 2^14.5; what is
          // left of it goes to alpha, which stays below 1. Powers upwards are exact, and the product is rounded once.
          const float top_alpha = fmaxf(__low2float(most), __high2float(most));
          if (__any_sync(0xffffffffu, top_alpha > alpha_most)) {
            float x = top_alpha;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
            const int ev = min(max((int)(__float_as_uint(x) >> 23) - 127, -14), 15);
            const float f = alpha_most < 0.f ? power2(-ev) : alpha_most * power2(-6 - ev);
#pragma unroll
            for (int i = 0; i < kO; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[i][e] *= f;
            alpha_most = power2(ev + 6), unit = __float2half2_rn(power2(-max(ev, -6)));
          }
          if (alpha_most < 1.f) {  // 2^(-6 - ev), for all of the warp
            const __half2 up = __float2half2_rn(__uint_as_float(0x7f000000u - __float_as_uint(alpha_most)));
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int i = 0; i < PAIRS; ++i) al[half][i] = __hmul2(al[half][i], up);
          }
          // The codes of both tokens of an operand register, channels 16 m + 8 jj + g: 16-bit units 8 jj + g of their rows,
          // transposed. The lane's address is that of row lane & 7 of matrix (half, jj).
          uint32_t word[4], more[4] = {};
          const uint32_t in8 = ((lane & 7) >> 1) + 4 * (lane & 1), from = vc + (8 * (lane >> 4) + in8) * kPitch + 16 * (lane >> 3 & 1);
          ldsm_x4_t(from, word);
          if constexpr (BITS == 4) ldsm_x4_t(from + 32, more);
          if constexpr (BITS == 3) ldsm_x2_t(vc + (8 * (lane >> 3 & 1) + in8) * kPitch + 32, more[0], more[2]);
          auto words = [&](int half, int jj) {
            return FieldOf<BITS>(word[2 * half + jj], BITS == 3 ? more[2 * half] >> jj : more[2 * half + jj]);
          };
          if constexpr (NARROW) {
            const uint32_t bt[4] = {be[0], 0u, be[1], 0u};
            mma_f16(ob, bt, pk[0], pk[1]);
            uint32_t pa[PAIRS][2];  // P alpha
#pragma unroll
            for (int i = 0; i < PAIRS; ++i)
#pragma unroll
              for (int half = 0; half < 2; ++half)
                pa[i][half] = h2_as_u32(__hmul2(__hmul2(u32_as_h2(pk[half]), unit), al[half][i]));
            const FieldOf<BITS> f00 = words(0, 0), f01 = words(0, 1), f10 = words(1, 0), f11 = words(1, 1);
#pragma unroll
            for (int m = 0; m < 8; ++m) {
              const uint32_t vt[4] = {f00.code(m), f01.code(m), f10.code(m), f11.code(m)};
              mma_f16(o[m], vt, pa[m / kOf][0], pa[m / kOf][1]);
            }
          } else {
            mma_f16(ob, pk, be[0], be[1]);
            uint32_t pa[PAIRS][4];
#pragma unroll
            for (int i = 0; i < PAIRS; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) pa[i][e] = h2_as_u32(__hmul2(__hmul2(u32_as_h2(pk[e]), unit), al[e >> 1][i]));
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
              const FieldOf<BITS> f0 = words(0, jj), f1 = words(1, jj);
#pragma unroll
              for (int m = 0; m < 8; ++m) mma_f16(o[2 * m + jj], pa[m / kOf], f0.code(m), f1.code(m));
            }
          }
        }
      }
      __syncwarp();  // (the stage may be filled again)
    }
    if (!ok) break;

    // Output: channels 8 i + 2 t and the next of every n-block i, or (narrow) 16 i + g and 8 on.
    if (form == 1) {
      float add[PAIRS][2];  // P beta of the groups, for the lane's rows
#pragma unroll
      for (int i = 0; i < PAIRS; ++i)
#pragma unroll
        for (int r = 0; r < 2; ++r)
          add[i][r] = NARROW ? __shfl_sync(0xffffffffu, ob[r], 4 * i + t) : __shfl_sync(0xffffffffu, ob[2 * r + (i & 1)], (lane & 28) + (i >> 1));
#pragma unroll
      for (int i = 0; i < kO; ++i) {
        const int m = NARROW ? i : i >> 1;
        const float f = alpha_most * power2(18 - FieldOf<BITS>::place(m));
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] = fmaf(o[i][e], f, add[m / kOf][NARROW ? e & 1 : e >> 1]);
      }
    }
    const bool whole = u0 == 0 && u1 == count, f32 = !whole || a.out_f32;
    const int slot = 2 * me + (u0 == 0);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float total = sum[r];
#pragma unroll
      for (int off = NARROW ? 4 : 1; off < (NARROW ? 32 : 4); off <<= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
      const bool blank = !real[r] || total == 0.f;
      const float lse2 = blank ? -INFINITY : ref[r] + fast_log2(total);
      const float f = poisoned[r] ? __int_as_float(0x7fffffff) : fast_inverse(total);
#pragma unroll
      for (int i = 0; i < kO; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float& x = o[i][NARROW ? r + 2 * e : 2 * r + e];
          x = blank ? 0.f : x * f;
        }
      const int row = NARROW ? 2 * t + r : g + 8 * r;
      const long long out = b * a.out.b + head[r] * a.out.h + node[r] * a.out.t;
      const int c = NARROW ? g : 2 * t;  // and from there 16 (8) on; two channels that are 8 (one) apart
      if (!there[r]) {
      } else if (f32) {
        float* at = (whole ? static_cast<float*>(a.out.p) + out : p.part_o + ((size_t)slot * kFewRows + row) * kHeadDim) + c;
#pragma unroll
        for (int i = 0; i < kO; ++i)
          if constexpr (NARROW)
            at[16 * i] = o[i][r], at[16 * i + 8] = o[i][r + 2];
          else
            *reinterpret_cast<float2*>(at + 8 * i) = make_float2(o[i][2 * r], o[i][2 * r + 1]);
      } else {
        __nv_bfloat16* at = static_cast<__nv_bfloat16*>(a.out.p) + out + c;
#pragma unroll
        for (int i = 0; i < kO; ++i)
          if constexpr (NARROW)
            at[16 * i] = __float2bfloat16(o[i][r]), at[16 * i + 8] = __float2bfloat16(o[i][r + 2]);
          else
            *reinterpret_cast<uint32_t*>(at + 8 * i) = pack_bf16(o[i][2 * r], o[i][2 * r + 1]);
      }
      if (there[r] && (NARROW ? g == 0 : t == 0)) {
        if (!whole)
          p.part_lse[(size_t)slot * kFewRows + row] = lse2;
        else if (a.lse)
          a.lse[((size_t)b * a.heads_q + head[r]) * a.nodes + node[r]] = lse2 * kLn2;
      }
    }
    start += n.cost();
    if (++in_set == per_set) in_set = 0, ++b;
  }
  if (!ok && lane == 0) {
    record_error(a.status, kErrFullTimeout);
    // no copy may outlive the CTA
    for (int s = 0; s < kFewStages; ++s)
      if (copies >> s & 1) mbar_wait(bars + 8 * s, parity >> s & 1);
  }
}

template <int BITS, int PAIRS, bool NARROW>
cudaError_t launch_few_shape(const TreeFewArgs& p, int grid, cudaStream_t st) {
  using F = FewShape<NARROW>;
  constexpr int kSmem = 1024 + F::kWarps * F::kStages * kFewStage;
  static std::atomic<uint64_t> configured;  // one bit per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  auto kernel = tree_few_kernel<BITS, PAIRS, NARROW>;
  if (dev > 63 || !(configured.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    configured.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_chained(kernel, dim3(grid), dim3(32 * F::kWarps), kSmem, st, p);
}

template <int BITS, bool NARROW>
cudaError_t launch_few_variant(const TreeFewArgs& p, int grid, cudaStream_t st) {
  return p.a.group == 32   ? launch_few_shape<BITS, 4, NARROW>(p, grid, st)
         : p.a.group == 64 ? launch_few_shape<BITS, 2, NARROW>(p, grid, st)
                           : launch_few_shape<BITS, 1, NARROW>(p, grid, st);
}

}  // namespace tree
}  // namespace mikv
