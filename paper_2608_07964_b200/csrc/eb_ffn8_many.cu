// eb_expert_ffn_grouped_fp8 for contexts of many rows per expert: the grouped SwiGLU pass on e4m3 rows and weights with a scale per block of 128.
//
//   gate[r, i] = sum_b xs[r, b] sg[i / 128, b] (sum over the 128 h of block b of xq[r, h] Wg[i, h]);  up likewise
//   a = silu(gate) * up;  as[r, j] = max |a| over block j of 128 outputs / 448;  aq = a / as as e4m3
//   yp[r, h] = sum_j as[r, j] sd[h / 128, j] (sum over block j of aq[r, i] Wd[h, i])                        (bf16 out)
//
// The walk over tiles is that of ffn_kernel (eb_ffn.cu): CTA pairs, a list of gate/up tiles and then down tiles, dealt out as pairs
// come free, down tiles behind the counts of their rows.  What differs is the accumulation.  Scales are arbitrary fp32 values that change
// every 128 elements of the sum, so the tensor cores sum one such block (a k-block: 128 bytes, four MMAs of K = 32) and the epilogue warps
// add it, times both scales, to fp32 sums in registers, while the next block goes into the other half of TMEM.
//
// That is why the TOKENS are the M operand here (256 rows a pair, 128 a CTA; a tile holds up to 256 rows) and 256 weight rows the N
// operand: a TMEM lane is a token, so the product of both scales is one number per thread and block, the largest magnitude of a token's
// outputs is found within threads, and a thread's outputs are neighbours in memory.  With the weights as M (eb_ffn8_few.cu) every
// column has a scale of its own, which each thread reads from shared memory, and twice the MMAs have to be issued: in bursts of eight passes 65536
// rows over 66 matrices of 3 x 2048 x 1408 take 807 us here and 1434 there, 8192 rows over 32 of 3 x 4096 x 14336 2342 and 3544; but 2048 rows
// over 191 of 3 x 2048 x 1408 342 and 281, since a k-block costs much the same here however few its rows.  (eb_enable_fp8 has the border.)
//
// A gate/up tile makes 128 outputs: each CTA brings 64 rows of W_gate and the same 64 of W_up as its half of the N operand, so
// that columns 0..63 | 64..127 of accumulator half c are gate | up of outputs 64 c ..; a down tile makes 256.  A thread
// holds up to 128 sums, which is why the epilogue warps take registers over from the others (setmaxnreg).
//
// Per CTA: warp 0 = weights by TMA, 1 = MMA issuer (leader CTA) or tile dealer (the other), 2 = token rows by TMA, 3 = publisher of
// finished rows, 4 = gate of the epilogue, 5 and 6 = scales, 8..15 = epilogue, two per lane quadrant; those whose lanes hold no rows only pass
// the accumulators on.  A stage is 32 KB per CTA (weights | up to 128 token rows of one k-block); six stages.  One commit per k-block
// frees its stage and hands its accumulator over.
//
// What bounds it: a k-block of 256 rows takes 1230 cycles, of which the MMAs need 512.  TMEM holds two such accumulators, and each goes round a
// chain: MMAs 512 (and 350 until their end is seen), read and added by the epilogue 610, handed back 400.  To keep that chain short the
// epilogue loop has nothing but one barrier, two words of scales, loads and multiply-adds in it; waits, scales and hand-overs are other
// warps' work.  Measured on the way: waits by all lanes of all warps 170 cycles each, a wait with cluster scope by 32 lanes 6000, scales
// fetched one block ahead 1000 a block, sixteen epilogue warps or waits within them no better, 32 columns a load worse (spills).
// Multiply-adds are what the epilogue spends its time on: without them (wrong results) 65536 rows that took 924 us, pass after pass, took 684.
//
// A TMA box costs its issuing thread about 110 cycles, so token rows are one box (rounded up to a power of two: lanes without rows may hold
// anything) or, in a merged tile, a box per lane.  The 128 outputs of a gate/up tile are a block of the intermediate: its largest magnitude per
// token is exchanged between the warps that hold parts of the row.
//
// Every wait on a barrier in memory is bounded as in ffn_kernel.
#include <cstddef>
#include <type_traits>

#include "eb_mma.cuh"
#include "eb_quant.cuh"
#include "eb_silu.cuh"
#include "eb_tiles.cuh"

namespace {

constexpr int BK = 128;                                        // e4m3 elements of one k-block = one scale block
constexpr int kStages = 6;
constexpr int kWBytes = 128 * BK;                              // 128 weight rows of one k-block
constexpr int kTBytes = 128 * BK;                              // up to 128 token rows of one k-block
constexpr int kStageBytes = kWBytes + kTBytes;
constexpr int kRingBytes = kStages * kStageBytes;
constexpr int kEpiWarp0 = 8, kEpiWarps = 8;                    // two per TMEM lane quadrant
constexpr int kThreads = 32 * (kEpiWarp0 + kEpiWarps);
constexpr int kRegsOther = 48, kRegsEpi = 208;                 // registers a thread after the split
static_assert(32 * kEpiWarp0 * kRegsOther + 32 * kEpiWarps * kRegsEpi <= kThreads * 128, "the split draws on what the block was launched with");
constexpr int kTmemCols = 512, kTmemQuarter = 128;
constexpr int kCtaRows = 128;                                  // token rows of a CTA at most
constexpr int kItems = 2, kParts = 4, kAskAhead = 8;           // as in eb_ffn.cu; k-blocks are twice as long here
static_assert(kParts > kItems, "a barrier of the publisher is free again before it comes round");

// shared memory behind the ring
constexpr int kBarOff = kRingBytes;                            // 512 bytes: barriers, TMEM address, abort flag, mailbox
constexpr int kMaxOff = kBarOff + 512;                         // [512] largest magnitudes: per row, of every part of the columns
constexpr int kScaleWarps = 2;
constexpr int kScaleSlots = 12;                                // k-blocks whose scales may lie ready
constexpr int kScaleOff = kMaxOff + 512 * 4;                   // [slots][128 rows] products of both scales, for either half of a warp's columns
constexpr int kTileOff = kScaleOff + kScaleSlots * kCtaRows * 8;                // 2 KB an epilogue warp: rows on their way out
constexpr size_t kSmemBytes = (size_t)kTileOff + kEpiWarps * 2048 + 1024 /*alignment slack*/;
static_assert(kSmemBytes <= 232448, "shared memory of one CTA");

// D[tmem of both CTAs] (+)= A * B^T on e4m3 with M (half of its rows per CTA) and N from the descriptor, K = 32
__device__ __forceinline__ void umma_pair_e4m3(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, {%5, %5, %5, %5, %5, %5, %5, %5}, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(0u)
      : "memory");
}
// Instruction descriptor: fp32 accumulate, e4m3 A and B (format 0), both K-major; N = 256.
__device__ __forceinline__ uint32_t instr_desc_e4m3(int m) { return (1u << 4) | ((256u >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

// Which part of TMEM a k-block's accumulator takes: two of four quarters (128 columns each), or one in a short tile, in turn.  The MMA warp
// and the epilogue walk the same k-blocks and so reach the same placement and the same barrier phases.
struct QuarterTurn {
  uint32_t next = 0, at = 0, phases = 15;   // phases, bit q: parity of the current use of quarter q (the first use has parity 0)
  __device__ __forceinline__ void take(bool is_short) {
    at = is_short ? next : ((next + 1) & 2u);
    phases ^= (is_short ? 1u : 3u) << at;
    next = (at + (is_short ? 1u : 2u)) & 3u;
  }
  __device__ __forceinline__ uint32_t parity(uint32_t q) const { return (phases >> q) & 1u; }
};

// Barriers between the gate warp and the epilogue warps of a CTA, and among the latter.  Nothing bounds these, so every warp of a group comes to each of
// them whatever happens: waits that may give up are the gate warp's alone, which tells the others behind the next barrier.
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
// The gate warp only arrives at kBarTile and kBarReady: one of either may be on its way at a time, so each is followed by a kBarRead, at which it
// waits for all.
constexpr int kBarReady = 1, kBarRead = 2, kBarTile = 3, kBarMax = 4;   // .. + 3
constexpr int kGateThreads = 32 * (kEpiWarps + 1);

__device__ __forceinline__ uint64_t pack2(uint32_t lo, uint32_t hi) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(lo), "r"(hi));
  return v;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  uint32_t lo, hi;
  asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(v));
  return make_float2(__uint_as_float(lo), __uint_as_float(hi));
}
// two fp32 multiply-adds; volatile: they stay in their order among the loads
__device__ __forceinline__ void fma2(uint64_t& acc, uint64_t a, uint64_t b) { asm volatile("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(a), "l"(b)); }

struct TokenMaps8 {
  CUtensorMap box[5];   // 128 / 64 / 32 / 16 / 8 rows
};
struct ManyParams {
  TokenMaps8 xq, act;
  CUtensorMap gate, up, down;        // weight boxes of 64 rows; with the above kMaps tensor maps in a row
  const float *xs, *s_gate, *s_up, *s_down;
  float* act_scale;                  // [ceil(I / 128)][rows_cap]
  const Tile* work;
  const int2* slots;
  const int32_t* work_count;
  int32_t* next;
  int32_t* ready;
  uint8_t* act_out;
  bf16* yp;
  int H, I, rows_cap;
  int part;
  int* status;
};
constexpr int kMaps = 13;
static_assert(offsetof(ManyParams, down) == (kMaps - 1) * sizeof(CUtensorMap), "the maps are prefetched as an array");

// A tile of at most 128 rows is multiplied with M = 128: each CTA then holds 64 of them, in lanes 0..63 with columns 0..127 of the N operand and
// again in lanes 64..127 with columns 128..255, in half the TMEM columns and half the time.
__device__ __forceinline__ bool short_tile(const Tile& it) { return it.rows < 0 ? -it.rows * kSlotRows <= kCtaRows : it.rows <= kCtaRows; }
// Token rows that CTA 0 of the pair takes before CTA 1 takes any.
__device__ __forceinline__ int rows_per_cta(const Tile& it) { return short_tile(it) ? kCtaRows / 2 : kCtaRows; }
// Rows (of 16-row slots of a merged tile: their full 16) that CTA `rank` of the pair holds.
__device__ __forceinline__ int cta_rows(const Tile& it, int rank) {
  const int n = it.rows < 0 ? -it.rows * kSlotRows : it.rows, most = rows_per_cta(it);
  return rank == 0 ? min(n, most) : max(n - most, 0);
}
// Rows that are loaded for them: one box of 8, 16, .. or 128 rows, or the slots of a merged tile.
__device__ __forceinline__ int box_rows(const Tile& it, int rank) {
  const int n = cta_rows(it, rank);
  return n == 0 || it.rows < 0 ? n : n <= 8 ? 8 : 1 << (32 - __clz(n - 1));
}

// sums of 16 columns += TMEM columns * f
__device__ __forceinline__ void add_columns(uint64_t* sum, const uint32_t* r, uint64_t f) {
#pragma unroll
  for (int k = 0; k < 8; ++k) fma2(sum[k], pack2(r[2 * k], r[2 * k + 1]), f);
}

// 32 bytes of a thread's own; whole sectors where the row's place allows it.
__device__ __forceinline__ void store32(void* at, const uint32_t (&v)[8], bool whole) {
  if (whole) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]),
                 "r"(v[6]), "r"(v[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(at)[0] = make_uint4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<uint4*>(at)[1] = make_uint4(v[4], v[5], v[6], v[7]);
  }
}

__global__ void __launch_bounds__(kThreads, 1)
ffn8_many_kernel(const __grid_constant__ ManyParams p) {
  EB_GRID_DEP_SYNC();
  constexpr int NS = kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (base - raw);
  const uint32_t bar0 = base + kBarOff;
  auto w_addr = [&](int s) { return base + s * kStageBytes; };
  auto t_addr = [&](int s) { return base + s * kStageBytes + kWBytes; };
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto done_bar = [&](int s) { return bar0 + 8u * (NS + s); };   // the stage's MMAs are through: it is free, its accumulator full
  auto tempty_bar = [&](int q) { return bar0 + 8u * (2 * NS + q); };
  auto item_full = [&](int i) { return bar0 + 8u * (2 * NS + 4 + i); };
  auto item_empty = [&](int i) { return bar0 + 8u * (2 * NS + 4 + kItems + i); };
  const uint32_t want_bar = bar0 + 8u * (2 * NS + 4 + 2 * kItems);
  auto part_bar = [&](int i) { return bar0 + 8u * (2 * NS + 5 + 2 * kItems + i); };
  auto scale_bar = [&](int i) { return bar0 + 8u * (2 * NS + 5 + 2 * kItems + kParts + i); };
  auto scale_free = [&](int i) { return bar0 + 8u * (2 * NS + 5 + 2 * kItems + kParts + kScaleSlots + i); };
  constexpr int kBarBytes = 8 * (2 * NS + 5 + 2 * kItems + kParts + 2 * kScaleSlots), kMailbox = 512 - kItems * (int)sizeof(Tile);
  static_assert(kBarBytes + 16 <= kMailbox, "512 bytes of barriers and mailbox");
  volatile uint32_t* s_tmem = reinterpret_cast<volatile uint32_t*>(smem + kBarOff + kBarBytes);
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem + kBarOff + kBarBytes + 4);
  volatile int* s_stop = reinterpret_cast<volatile int*>(smem + kBarOff + kBarBytes + 8);   // the gate warp's word to the epilogue warps: no tile, no accumulator
  const uint32_t items = bar0 + kMailbox;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();   // CTA 0 of a pair is the leader
  int* const status = p.status;
  if (threadIdx.x == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(full_bar(s), 3);    // the leader's weight warp, both token warps, and all bytes of the stage of both CTAs
      mbar_init(done_bar(s), 1);
    }
    for (int q = 0; q < 4; ++q) mbar_init(tempty_bar(q), 2);   // the epilogues of both CTAs (leader's barrier)
    for (int i = 0; i < kItems; ++i) {
      mbar_init(item_full(i), 1);
      mbar_init(item_empty(i), 9 + 2 * kScaleWarps);   // every reader of both CTAs (CTA 1's barrier)
    }
    for (int i = 0; i < kParts; ++i) mbar_init(part_bar(i), kEpiWarps);
    for (int i = 0; i < kScaleSlots; ++i) {
      mbar_init(scale_bar(i), kScaleWarps);
      mbar_init(scale_free(i), 1);          // the gate warp
    }
    mbar_init(want_bar, 1);
    *s_abort = 0;
    s_stop[0] = s_stop[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2 && lane < kMaps) prefetch_tmap(&p.xq.box[0] + lane);
  // the pair's first tile, claimed like all others (see ffn_kernel)
  int4 first_a = make_int4(0, 0, -1, 0), first_b = make_int4(0, 0, 0, 0);
  const bool claims_first = rank == 1 && threadIdx.x == 96;
  if (claims_first) {
    const int cnt1 = p.work_count[0], cnt2 = p.work_count[1];
    const int idx = (p.part == 2 ? cnt1 : 0) + atomicAdd(p.next + (p.part == 2 ? 1 : 0), 1);
    if (idx < (p.part == 1 ? cnt1 : cnt1 + cnt2)) {
      const int4* e = reinterpret_cast<const int4*>(p.work + idx);
      first_a = __ldg(e);
      first_b = __ldg(e + 1);
    }
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32((const void*)s_tmem), kTmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *s_tmem;
  const int num_kb1 = ebi_blocks(p.H), num_kb2 = ebi_blocks(p.I);

  auto deal = [&](int i, const int4& a, const int4& b) {
    for (uint32_t r = 0; r < 2; ++r) {
      const uint32_t dst = map_to_cta(items + i * (uint32_t)sizeof(Tile), r);
      st_cluster(dst, a);
      st_cluster(dst + 16, b);
      mbar_arrive_release_cluster(map_to_cta(item_full(i), r));
    }
  };
  if (claims_first) deal(0, first_a, first_b);
  auto take_item = [&](int seq, Tile* it) {
    const int i = seq % kItems;
    if (!mbar_wait_cluster(item_full(i), (uint32_t)(seq / kItems) & 1u, s_abort, status)) return false;
    const int4 a = ld_shared(items + i * (uint32_t)sizeof(Tile)), b = ld_shared(items + i * (uint32_t)sizeof(Tile) + 16);
    *it = Tile{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    return true;
  };
  // The same for a whole warp: one lane takes it (a wait with cluster scope by all 32 takes 6000 cycles) and may free the slot.
  auto take_item_warp = [&](int seq, Tile* it, bool frees) {
    int ok = 1;
    if (lane == 0) {
      ok = take_item(seq, it) ? 1 : 0;
      if (ok && frees && it->w >= 0) mbar_arrive_cluster(map_to_cta(item_empty(seq % kItems), 1));
    }
    it->row = __shfl_sync(0xffffffffu, it->row, 0);
    it->rows = __shfl_sync(0xffffffffu, it->rows, 0);
    it->w = __shfl_sync(0xffffffffu, it->w, 0);
    it->out = __shfl_sync(0xffffffffu, it->out, 0);
    it->phase = __shfl_sync(0xffffffffu, it->phase, 0);
    it->done = __shfl_sync(0xffffffffu, it->done, 0);
    it->need = __shfl_sync(0xffffffffu, it->need, 0);
    return __shfl_sync(0xffffffffu, ok, 0) != 0;
  };
  auto free_item = [&](int seq) { mbar_arrive_cluster(map_to_cta(item_empty(seq % kItems), 1)); };

  // A down tile's rows are all written (a whole warp asks; false: gave up).
  auto rows_ready = [&](const Tile& it) {
    if (it.phase != 2 || it.need <= 0) return true;
    const int* flag = p.ready + it.done;
    int ok = 1;
    if (lane == 0) ok = bounded_wait([&] { return ld_acquire(flag) >= it.need; }, s_abort, status) ? 1 : 0;
    ok = __shfl_sync(0xffffffffu, ok, 0);
    __syncwarp();
    return ok != 0;
  };

  if (warp < kEpiWarp0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == 0) {
      // ---------------- weights (each CTA loads its own half) ----------------
      if (lane == 0) {
        uint64_t stream_policy, keep_policy;   // as in ffn_kernel: weights with one reader leave L2 first
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(stream_policy));
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(keep_policy));
        int stage = 0;
        uint32_t phase = 0;
        for (int seq = 0;; ++seq) {
          Tile it;
          if (!take_item(seq, &it)) goto done;
          if (it.w < 0) break;
          free_item(seq);
          const uint64_t w_policy = it.once ? stream_policy : keep_policy;
          const bool down = it.phase == 2;
          const CUtensorMap* tmW0 = down ? &p.down : &p.gate;
          const CUtensorMap* tmW1 = down ? &p.down : &p.up;
          const int num_kb = down ? num_kb2 : num_kb1;
          // down: this CTA's 128 of the 256 rows; gate/up: its 64 rows of either matrix
          const int wrow0 = down ? it.out * kFeat2Many + (int)rank * 128 : it.out * kFeat1Many + (int)rank * 64;
          const int wrow1 = down ? wrow0 + 64 : wrow0;
          const uint32_t tx = 2u * kWBytes + (uint32_t)(box_rows(it, 0) + box_rows(it, 1)) * BK;   // of both CTAs, tokens included
          const int ask = num_kb > kAskAhead ? num_kb - kAskAhead : 0;
          for (int kb = 0; kb < num_kb; ++kb) {
            if (rank == 0 && kb == ask) mbar_arrive_cluster(map_to_cta(want_bar, 1));
            if (!mbar_wait(done_bar(stage), phase ^ 1u, s_abort, status)) goto done;
            const uint32_t fb = map_to_cta(full_bar(stage), 0);   // both CTAs' copies are counted on the leader's barrier
            if (rank == 0) mbar_expect_tx(full_bar(stage), tx);
            tma_pair_load_3d(w_addr(stage), tmW0, kb * BK, wrow0, it.w, fb, w_policy);
            tma_pair_load_3d(w_addr(stage) + kWBytes / 2, tmW1, kb * BK, wrow1, it.w, fb, w_policy);
            if (++stage == NS) {
              stage = 0;
              phase ^= 1u;
            }
          }
        }
      }
    } else if (warp == 1) {
      if (lane == 0 && rank == 0) {
        // ---------------- MMA issuer (leader CTA only) ----------------
        int stage = 0;
        uint32_t phase = 0;
        QuarterTurn turn;
        for (int seq = 0;; ++seq) {
          Tile it;
          if (!take_item(seq, &it)) goto done;
          if (it.w < 0) break;
          free_item(seq);
          const int num_kb = it.phase == 2 ? num_kb2 : num_kb1;
          const bool is_short = short_tile(it);
          const uint32_t idesc = instr_desc_e4m3(is_short ? 128 : 256);
          for (int kb = 0; kb < num_kb; ++kb) {
            turn.take(is_short);
            if (!mbar_wait(tempty_bar(turn.at), turn.parity(turn.at) ^ 1u, s_abort, status)) goto done;
            if (!is_short && !mbar_wait(tempty_bar(turn.at + 1), turn.parity(turn.at + 1) ^ 1u, s_abort, status)) goto done;
            if (!mbar_wait(full_bar(stage), phase, s_abort, status)) goto done;
            tc_fence_after();
            const uint64_t dw = smem_desc(w_addr(stage)), dt = smem_desc(t_addr(stage));
#pragma unroll
            for (int k = 0; k < BK / 32; ++k) umma_pair_e4m3(tmem_base + turn.at * kTmemQuarter, dt + 2 * k, dw + 2 * k, idesc, k != 0 ? 1u : 0u);
            umma_pair_commit(done_bar(stage));
            if (++stage == NS) {
              stage = 0;
              phase ^= 1u;
            }
          }
        }
      } else if (lane == 0) {
        // ---------------- tile dealer (CTA 1's otherwise idle MMA warp) ----------------
        const int part_first = p.part == 2 ? p.work_count[0] : 0;
        const int part_end = p.part == 1 ? p.work_count[0] : p.work_count[0] + p.work_count[1];
        Tile it;
        if (!take_item(0, &it)) goto done;
        for (int seq = 1; it.w >= 0; ++seq) {
          const int i = seq % kItems;
          if (!mbar_wait_cluster(want_bar, (uint32_t)(seq - 1) & 1u, s_abort, status)) goto done;
          if (seq >= kItems && !mbar_wait_cluster(item_empty(i), (uint32_t)(seq / kItems - 1) & 1u, s_abort, status)) goto done;
          const int idx = part_first + atomicAdd(p.next + (p.part == 2 ? 1 : 0), 1);
          int4 a = make_int4(0, 0, -1, 0), b = make_int4(0, 0, 0, 0);
          if (idx < part_end) {
            const int4* e = reinterpret_cast<const int4*>(p.work + idx);
            a = __ldg(e);
            b = __ldg(e + 1);
            if (b.x == 2 && ld_acquire(p.ready + b.y) >= b.z) b.z = 0;
          }
          deal(i, a, b);
          if (idx >= part_end) break;
        }
      }
    } else if (warp == 2) {
      // ---------------- token rows ----------------
      int stage = 0;
      uint32_t phase = 0;
      for (int seq = 0;; ++seq) {
        Tile it = {};
        if (!take_item_warp(seq, &it, true)) goto done;
        if (it.w < 0) break;
        const bool down = it.phase == 2, merged = it.rows < 0;
        const int num_kb = down ? num_kb2 : num_kb1;
        const int rows = box_rows(it, rank);
        const TokenMaps8* const maps = down ? &p.act : &p.xq;
        // the box of this lane: a slot's 16 rows in a merged tile, all rows by lane 0 otherwise
        const bool loads = merged ? lane * kSlotRows < rows : lane == 0 && rows > 0;
        const CUtensorMap* const tm = &maps->box[merged ? 3 : rows == 128 ? 0 : rows == 64 ? 1 : rows == 32 ? 2 : rows == 16 ? 3 : 4];
        const int row_of_box = merged ? (loads ? __ldg(p.slots + it.row + (int)rank * (rows_per_cta(it) / kSlotRows) + lane).x : 0) : it.row + (int)rank * rows_per_cta(it);
        const uint32_t box_at = merged ? (uint32_t)lane * kSlotRows * BK : 0u;
        if (!rows_ready(it)) goto done;
        if (down) fence_proxy_async();
        for (int kb = 0; kb < num_kb; ++kb) {
          int ok = 1;
          if (lane == 0) ok = mbar_wait(done_bar(stage), phase ^ 1u, s_abort, status) ? 1 : 0;
          if (!__shfl_sync(0xffffffffu, ok, 0)) goto done;
          if (loads) tma_pair_load_2d(t_addr(stage) + box_at, tm, kb * BK, row_of_box, map_to_cta(full_bar(stage), 0));
          // also without rows: no stage comes round twice while this warp is still waiting for it
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(map_to_cta(full_bar(stage), 0));
          if (++stage == NS) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
    } else if (warp == 5 || warp == 6) {
      // ---------------- scales: of rows 64 (warp - 5) + lane and 32 further on, times the weight blocks' ----------------
      // Those of four k-blocks are on their way at a time: with one, a block took as long as its trip to L2 (1000 cycles).
      uint32_t block = 0;
      for (int seq = 0;; ++seq) {
        Tile it = {};
        if (!take_item_warp(seq, &it, true)) goto done;
        if (it.w < 0) break;
        const bool down = it.phase == 2;
        const int num_kb = down ? num_kb2 : num_kb1, mine = cta_rows(it, rank);
        // weight blocks of columns 0..127 and 128..255 of a down tile, of gate and up of a gate/up tile.  A block beyond the matrix: the last one's,
        // for sums that nobody stores.
        const size_t mat = (size_t)it.w * num_kb1 * num_kb2;
        const float* const sw0 = down ? p.s_down + mat + (size_t)min(it.out * 2, num_kb1 - 1) * num_kb2 : p.s_gate + mat + (size_t)it.out * num_kb1;
        const float* const sw1 = down ? p.s_down + mat + (size_t)min(it.out * 2 + 1, num_kb1 - 1) * num_kb2 : p.s_up + mat + (size_t)it.out * num_kb1;
        const float* sx[2];
        bool there[2];
        const int step = down ? p.rows_cap : 1;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int tok = (warp - 5) * 64 + 32 * i + lane;
          there[i] = tok < mine;
          int row = it.row + (int)rank * rows_per_cta(it) + tok;
          if (it.rows < 0 && there[i]) row = __ldg(p.slots + it.row + ((int)rank * rows_per_cta(it) + tok) / kSlotRows).x + tok % kSlotRows;
          row = min(row, p.rows_cap - 1);
          sx[i] = !there[i] ? p.xs : down ? p.act_scale + row : p.xs + (size_t)row * num_kb1;
        }
        if (!rows_ready(it)) goto done;
        float x[4][2], w0[4], w1[4];
        auto load = [&](int kb, float (&xk)[2], float& w0k, float& w1k) {   // the intermediate's scales were written by this launch: from L2
          if (kb >= num_kb) return;
          w0k = __ldg(sw0 + kb);
          w1k = __ldg(sw1 + kb);
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (there[i]) xk[i] = down ? __ldcg(sx[i] + (size_t)kb * step) : __ldg(sx[i] + kb);
        };
#pragma unroll
        for (int j = 0; j < 4; ++j) load(j, x[j], w0[j], w1[j]);
        for (int kb0 = 0; kb0 < num_kb; kb0 += 4) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (kb0 + j >= num_kb) break;
            const uint32_t slot = block % kScaleSlots;
            int ok = 1;
            if (lane == 0) ok = mbar_wait(scale_free(slot), ((block / kScaleSlots) & 1u) ^ 1u, s_abort, status) ? 1 : 0;
            if (!__shfl_sync(0xffffffffu, ok, 0)) goto done;
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (there[i]) reinterpret_cast<float2*>(smem + kScaleOff)[slot * kCtaRows + (warp - 5) * 64 + 32 * i + lane] = make_float2(x[j][i] * w0[j], x[j][i] * w1[j]);
            __syncwarp();
            if (lane == 0) mbar_arrive_release(scale_bar(slot));
            ++block;
            load(kb0 + j + 4, x[j], w0[j], w1[j]);
          }
        }
      }
    } else if (warp == 4) {
      // ---------------- gate of the epilogue: waits for tiles, accumulators and scales, hands accumulators back ----------------
      // One warp for all: a wait by every epilogue warp, and the branches around it in their loop, took several hundred cycles a k-block.
      const uint32_t tempty0 = map_to_cta(tempty_bar(0), 0);
      uint32_t block = 0, phase = 0;
      int stage = 0;
      QuarterTurn turn;
      for (int seq = 0;; ++seq) {
        Tile it = {};
        if (!take_item_warp(seq, &it, false)) s_stop[0] = 1;
        __syncwarp();
        bar_arrive(kBarTile, kGateThreads);
        if (s_stop[0]) goto done;
        if (it.w < 0) break;
        const bool is_short = short_tile(it);
        const int num_kb = it.phase == 2 ? num_kb2 : num_kb1;
        for (int kb = 0; kb < num_kb; ++kb, ++block) {
          turn.take(is_short);
          if (lane == 0 && !(mbar_wait(scale_bar(block % kScaleSlots), (block / kScaleSlots) & 1u, s_abort, status) &&
                             mbar_wait(done_bar(stage), phase, s_abort, status)))
            s_stop[1] = 1;
          __syncwarp();
          bar_arrive(kBarReady, kGateThreads);
          if (s_stop[1]) goto done;
          bar_sync(kBarRead, kGateThreads);
          if (lane == 0) {
            mbar_arrive_cluster(tempty0 + 8 * turn.at);
            if (!is_short) mbar_arrive_cluster(tempty0 + 8 * turn.at + 8);
            mbar_arrive_release(scale_free(block % kScaleSlots));
            if (kb == 0) free_item(seq);   // all have read it
          }
          if (++stage == NS) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
    } else if (warp == 3) {
      if (lane == 0) {
        // ---------------- publisher: counts the CTA's share of a finished gate/up tile on its token tile ----------------
        uint32_t uses = 0;
        for (int seq = 0;; ++seq) {
          Tile it;
          if (!take_item(seq, &it)) goto done;
          if (it.w < 0) break;
          free_item(seq);
          if (it.phase != 1) continue;
          const int i = seq % kParts;
          if (!mbar_wait(part_bar(i), (uses >> i) & 1u, s_abort, status)) goto done;
          uses ^= 1u << i;
          red_publish(p.ready + it.done);
        }
      }
    }
  } else {
    // ---------------- epilogue warps ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsEpi));
    const int q = warp & 3, part = (warp - kEpiWarp0) >> 2;   // lane quadrant; which of its two warps
    uint32_t* const s_max = reinterpret_cast<uint32_t*>(smem + kMaxOff);
    const bool act_whole = (p.I & 31) == 0;   // 32-byte pieces of its rows lie on 32-byte boundaries
    uint32_t block = 0;   // k-blocks so far
    QuarterTurn turn;
    for (int seq = 0;; ++seq) {
      Tile it;
      bar_sync(kBarTile, kGateThreads);
      if (s_stop[0]) goto done;
      {
        const uint32_t at = items + seq % kItems * (uint32_t)sizeof(Tile);
        const int4 a = ld_shared(at), b = ld_shared(at + 16);
        it = Tile{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      }
      if (it.w < 0) break;
      const bool down = it.phase == 2, is_short = short_tile(it);
      const int num_kb = down ? num_kb2 : num_kb1;
      // half: of the N operand's columns, the 64 + 64 (gate and up, or one run of 128) that come from CTA `half`.  Wide: the two warps of a quadrant
      // take a half each; is_short: lanes 64.. hold the second half of the rows in lanes 0.., the warps take 32 + 32 columns.
      const int half = is_short ? q >> 1 : part, tok = is_short ? (q & 1) * 32 + lane : q * 32 + lane;
      const int mine = cta_rows(it, rank);
      const bool busy = tok - lane < mine;   // else no rows in these lanes: the accumulators pass by
      if (!busy) {
        for (int kb = 0; kb < num_kb; ++kb, ++block) {
          turn.take(is_short);
          bar_sync(kBarReady, kGateThreads);
          if (s_stop[1]) goto done;
          bar_arrive(kBarRead, kGateThreads);
        }
        if (!down && lane == 0) mbar_arrive_release(part_bar(seq % kParts));
        continue;
      }
      // sums over the k-blocks of NC columns twice, 64 apart, from column `col` of the accumulator on
      auto run = [&](auto nc) -> bool {
        constexpr int NC = decltype(nc)::value, kEach = NC / 16;
        const int col_half = NC == 64 ? 0 : part * 32;             // within the half's first 64 columns
        const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (NC == 64 ? half * 128 : 0) + col_half;
        uint64_t sum[2][NC / 2];
#pragma unroll
        for (int i = 0; i < NC / 2; ++i) sum[0][i] = sum[1][i] = 0;
        const uint32_t my_scales = base + kScaleOff + 8 * tok + (down && half ? 4u : 0u), second = down ? 0u : 4u;
        uint32_t r[2][16];
        for (int kb = 0; kb < num_kb; ++kb, ++block) {
          turn.take(NC == 32);
          const uint32_t at = taddr + turn.at * kTmemQuarter;
          bar_sync(kBarReady, kGateThreads);
          tc_fence_after();
          tmem_ld16(at, r[0]);
          const bool stop = s_stop[1] != 0;   // the same for all: the gate warp writes it ahead of this barrier only
          uint32_t a, b;                      // scales of the first and the second NC columns
          const uint32_t scale_at = my_scales + block % kScaleSlots * (kCtaRows * 8);
          asm volatile("ld.shared.b32 %0, [%1];" : "=r"(a) : "r"(scale_at));
          asm volatile("ld.shared.b32 %0, [%1];" : "=r"(b) : "r"(scale_at + second));
          const uint64_t f0 = pack2(a, a), f1 = pack2(b, b);
          // 16 columns at a time, the next ones on their way while they are added; the last ones are added when the accumulator has been handed back
#pragma unroll
          for (int i = 0; i < 2 * kEach - 1; ++i) {
            tmem_ld_wait(r[i & 1]);
            tmem_ld16(at + ((i + 1) / kEach) * 64 + ((i + 1) % kEach) * 16, r[(i + 1) & 1]);
            add_columns(sum[i / kEach] + i % kEach * 8, r[i & 1], i < kEach ? f0 : f1);
          }
          tmem_ld_wait(r[1]);
          tc_fence_before();
          if (stop) return false;
          bar_arrive(kBarRead, kGateThreads);
          add_columns(sum[1] + NC / 2 - 8, r[1], f1);
        }
        int row = -1;   // this thread's; -1: none
        if (tok < mine) {
          row = it.row + (int)rank * rows_per_cta(it) + tok;
          if (it.rows < 0) {
            const int2 sl = __ldg(p.slots + it.row + ((int)rank * rows_per_cta(it) + tok) / kSlotRows);
            row = tok % kSlotRows < sl.y ? sl.x + tok % kSlotRows : -1;
          }
        }
        if (!down) {
          {
            // the first NC columns are gate, the others up of outputs 64 half + col_half .. of block it.out
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < NC / 2; ++i) {
              const float2 g = unpack2(sum[0][i]), u = unpack2(sum[1][i]);
              float h0, h1;
              silu_mul2(g.x, u.x, g.y, u.y, &h0, &h1);
              const uint32_t lo = __float_as_uint(h0), hi = __float_as_uint(h1);
              sum[0][i] = pack2(lo, hi);
              most = max(most, max(lo & 0x7fffffffu, hi & 0x7fffffffu));
            }
            // a row's two parts (wide) or four (is_short); the barriers of the next tile keep its writes behind these reads
            constexpr int kRows = NC == 64 ? 128 : 64, kAll = NC == 64 ? 2 : 4;
            uint32_t* const mx = s_max + tok;
            mx[(NC == 64 ? part : half * 2 + part) * kRows] = most;
            if (NC == 64) bar_sync(kBarMax + q, 64);
            else bar_sync(kBarMax + (q & 1), 128);
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < kAll; ++i) m = max(m, mx[i * kRows]);
            const float top = __uint_as_float(m);
            const bool none = top < 7.70371978e-34f;   // 2^-110
            const float inv = none ? 0.f : __fdiv_rn(kE4M3Max, top);
            if (row >= 0) {
              if (part == 0 && half == 0) p.act_scale[(size_t)it.out * p.rows_cap + row] = m >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : none ? 0.f : __fdiv_rn(top, kE4M3Max);
              const int col = it.out * kFeat1Many + half * 64 + col_half;
              uint8_t* const at = p.act_out + (size_t)row * p.I + col;
#pragma unroll
              for (int c = 0; c < NC; c += 32) {
                uint32_t v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  const float2 a = unpack2(sum[0][c / 2 + 2 * k]), b = unpack2(sum[0][c / 2 + 2 * k + 1]);
                  v[k] = pack_e4m3(a.x * inv, a.y * inv) | pack_e4m3(b.x * inv, b.y * inv) << 16;
                }
                if (act_whole) {
                  if (col + c < p.I) store32(at + c, v, true);
                } else {   // I is a multiple of 16
                  if (col + c < p.I) *reinterpret_cast<uint4*>(at + c) = make_uint4(v[0], v[1], v[2], v[3]);
                  if (col + c + 16 < p.I) *reinterpret_cast<uint4*>(at + c + 16) = make_uint4(v[4], v[5], v[6], v[7]);
                }
              }
            }
          }
          // this warp's part of the intermediate is written: the publisher counts the CTA's share of the tile
          __syncwarp();
          if (lane == 0) mbar_arrive_release(part_bar(seq % kParts));
        } else {
          // A thread's outputs are a piece of one row; stored as they are, every store of a warp touches 32 lines (a tile's end took 4700 cycles).
          // By way of shared memory eight (four) lanes write 128 (64) bytes of a row: NC columns at a time, of 16 (32) rows.
          constexpr int kLanes = NC / 8, kRowsAtOnce = 32 * 64 / (2 * NC), kRowBytes = 2 * NC;
          const uint32_t mine_at = base + kTileOff + (warp - kEpiWarp0) * 2048;
          const int col = it.out * kFeat2Many + half * 128 + col_half;
#pragma unroll
          for (int a = 0; a < 2; ++a) {
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += kRowsAtOnce) {
              const int lr = lane - r0;   // this lane's row of those
              if (lr >= 0 && lr < kRowsAtOnce) {
#pragma unroll
                for (int ch = 0; ch < kLanes; ++ch) {
                  uint32_t v[4];
#pragma unroll
                  for (int k = 0; k < 4; ++k) {
                    const float2 f = unpack2(sum[a][4 * ch + k]);
                    v[k] = pack_bf16(f.x, f.y);
                  }
                  // 16-byte pieces in an order of their own in every row, so that neither side meets in a bank
                  const uint32_t to = mine_at + lr * kRowBytes + ((ch ^ (NC == 64 ? lr : lr >> 1)) & (kLanes - 1)) * 16;
                  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                }
              }
              __syncwarp();
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const int rr = j * (32 / kLanes) + lane / kLanes, ch = lane % kLanes;
                const int4 v = ld_shared(mine_at + rr * kRowBytes + ((ch ^ (NC == 64 ? rr : rr >> 1)) & (kLanes - 1)) * 16);
                const int to_row = __shfl_sync(0xffffffffu, row, r0 + rr);
                const int c = col + 64 * a + 8 * ch;
                if (to_row >= 0 && c < p.H) *reinterpret_cast<int4*>(p.yp + (size_t)to_row * p.H + c) = v;   // H is a multiple of 16
              }
              __syncwarp();
            }
          }
        }
        return true;
      };
      if (!(is_short ? run(std::integral_constant<int, 32>()) : run(std::integral_constant<int, 64>()))) goto done;
    }
  }

done:
  if (*s_abort) {
    // give copies and MMAs in flight time to land before shared memory and TMEM go away
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, kTmemCols);
  }
}

cudaError_t launch_many(eb_ctx* c, cudaStream_t st, const ManyParams& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(c->pair_grid8);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  ++g_ebi_launches;
  return cudaLaunchKernelEx(&cfg, ffn8_many_kernel, p);
}

}  // namespace

eb_status ebi_ffn8_many_bind(eb_ctx* c) {
  if (eb_status ds = ebi_check_device(c)) return ds;
  const eb_config& g = c->cfg;
  const uint64_t nw = (uint64_t)g.L * (g.E + g.S);
  if (!make_map(&c->tm8_gate, c->w8_gate, g.H, g.I, nw, BK, 64, true) || !make_map(&c->tm8_up, c->w8_up, g.H, g.I, nw, BK, 64, true) ||
      !make_map(&c->tm8_down, c->w8_down, g.I, g.H, nw, BK, 64, true))
    return ebi_fail(c, EB_ERR_CUDA, "cuTensorMapEncodeTiled failed for the weights");
  cudaError_t e = cudaFuncSetAttribute(ffn8_many_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
  if (e != cudaSuccess) return ebi_check_cuda(c, e, "cudaFuncSetAttribute");
  c->pair_grid8 = ebi_pair_grid(c, (const void*)ffn8_many_kernel, kThreads, kSmemBytes);
  if (!c->pair_grid8) return ebi_fail(c, EB_ERR_CUDA, "the device cannot hold a 2-CTA cluster of the 8-bit expert kernel");
  return EB_OK;
}

eb_status ebi_ffn8_many_run(eb_ctx* c, cudaStream_t st, const void* xq, const float* xs, const int32_t* group_off, const int32_t* group_w,
                       const int32_t* step_meta, void* yp, int32_t device, bool planned) {
  if (!xq || !xs || !group_off || !group_w || !step_meta || !yp) return ebi_fail(c, EB_ERR_INVALID_ARG, "null pointer");
  if (eb_status ds = ebi_check_device(c)) return ds;
  if (!ebi_aligned16(xq) || !ebi_aligned16(xs) || !ebi_aligned16(yp)) return ebi_fail(c, EB_ERR_INVALID_ARG, "xq / xs / yp must be 16-byte aligned");
  if (!c->w8_gate) return ebi_fail(c, EB_ERR_INVALID_ARG, "8-bit weights not bound");
  if (!c->ws) return ebi_fail(c, EB_ERR_WORKSPACE, "no workspace set");
  const eb_config& g = c->cfg;
  const int rows = ebi_rows_cap(c);
  ManyParams p;
  const int box_rows[5] = {128, 64, 32, 16, 8};
  for (int i = 0; i < 5; ++i)
    if (!make_map(&p.xq.box[i], xq, g.H, rows, 0, BK, box_rows[i], true) || !make_map(&p.act.box[i], c->act, g.I, rows, 0, BK, box_rows[i], true))
      return ebi_fail(c, EB_ERR_CUDA, "cuTensorMapEncodeTiled failed for the activations");
  p.gate = c->tm8_gate;
  p.up = c->tm8_up;
  p.down = c->tm8_down;
  p.xs = xs;
  p.s_gate = c->s8_gate;
  p.s_up = c->s8_up;
  p.s_down = c->s8_down;
  p.act_scale = c->act_scale;
  p.work = (const Tile*)c->work;
  p.slots = c->slots;
  p.work_count = c->work_count;
  p.next = c->work_count + 6;
  p.ready = c->tile_ready;
  p.act_out = (uint8_t*)c->act;
  p.yp = (bf16*)yp;
  p.H = g.H;
  p.I = g.I;
  p.rows_cap = rows;
  p.status = c->d_status;
  if (!planned)
    if (eb_status s = ebi_ffn_plan(c, st, group_off, group_w, step_meta, device, EB_PASS_FP8_MANY)) return s;
  if (!c->timing) {
    p.part = 0;
    EB_LAUNCH(c, "expert_ffn_fp8", launch_many(c, st, p));
  } else {   // the same tiles in two launches, so that each phase gets a time of its own
    {
      KernelTimer timer(c, EBK_FFN_GATEUP, st);
      p.part = 1;
      EB_LAUNCH(c, "expert_ffn_fp8", launch_many(c, st, p));
    }
    KernelTimer timer(c, EBK_FFN_DOWN, st);
    p.part = 2;
    EB_LAUNCH(c, "expert_ffn_fp8", launch_many(c, st, p));
  }
  EB_LAUNCH_CHECK(c, "expert_ffn_fp8");
  return EB_OK;
}
