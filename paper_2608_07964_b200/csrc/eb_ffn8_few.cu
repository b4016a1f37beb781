// eb_expert_ffn_grouped_fp8 for contexts of few rows per expert (eb_ffn8_many.cu: the others): the grouped SwiGLU pass on e4m3 rows and weights with a scale per block of 128.
//
//   gate[r, i] = sum_b xs[r, b] sg[i / 128, b] (sum over the 128 h of block b of xq[r, h] Wg[i, h]);  up likewise
//   a = silu(gate) * up;  as[r, j] = max |a| over block j of 128 outputs / 448;  aq = a / as as e4m3
//   yp[r, h] = sum_j as[r, j] sd[h / 128, j] (sum over block j of aq[r, i] Wd[h, i])                        (bf16 out)
//
// The walk over tiles is that of ffn_kernel (eb_ffn.cu): CTA pairs, the weights as the M operand (256 rows, 128 a CTA), the tile's token
// rows as the N operand, W0 and W1 sharing it, a list of gate/up tiles and then down tiles, dealt out as pairs come free, down tiles
// behind the counts of their rows.  What differs is the accumulation.  Scales are arbitrary fp32 values that change every 128
// elements of the sum, so the tensor cores sum one such block (a k-block: 128 bytes, four MMAs of K = 32) and the
// epilogue warps add it, times both scales, to fp32 sums in registers: two 256-column halves of TMEM go back and forth
// between the MMA warp and the epilogue warps, one k-block of a wide tile or several of a narrow one at a time ("a turn").
// The sums of a tile take 128 lanes x 2 x its columns: 128 registers a thread at 128 columns, which is what limits tiles to 128
// token rows and why the epilogue warps take registers over from the others (setmaxnreg).
//
// A token's scale times a weight block's is the same for all 128 outputs of a CTA: the scale warp multiplies them a turn at a time
// into shared memory, so that an element costs its epilogue thread half a packed multiply-add and nothing else.
//
// Per CTA: warp 0 = TMA producer, 1 = MMA issuer (leader CTA) or tile dealer (the other), 2 = scales, 3 = publisher of finished rows,
// 4..11 = epilogue.  A stage is 40 KB per CTA (W0 | W1 | up to 64 token rows of one k-block); five stages.
//
// The outputs of a CTA in a gate/up tile are one block of 128: its largest magnitudes per token are found by warp reductions and one
// exchange between the four lane quadrants.  A down tile takes the scales that way from the workspace.
//
// What bounds it: with few rows the stream of weights (2048 rows over 191 matrices of 3 x 2048 x 1408, 1.65 GB: 297 to 318 us pass after pass, 5.2
// to 5.6 TB/s; 281 in bursts); with many the issue of its MMAs, eight a k-block, and the ends of its tiles.
//
// Every wait is bounded as in ffn_kernel.
#include <cstddef>
#include <type_traits>

#include "eb_mma.cuh"
#include "eb_quant.cuh"
#include "eb_silu.cuh"
#include "eb_tiles.cuh"

namespace {

constexpr int BK = 128;                                        // e4m3 elements of one k-block = one scale block
constexpr int kStages = 5;
constexpr int kWBytes = 128 * BK;                              // 128 weight rows of one k-block
constexpr int kTBytes = 64 * BK;                               // up to 64 token rows of one k-block
constexpr int kStageBytes = 2 * kWBytes + kTBytes;             // W0 | W1 | token rows
constexpr int kRingBytes = kStages * kStageBytes;
constexpr int kEpiWarp0 = 4, kEpiWarps = 8;                    // two per TMEM lane quadrant
constexpr int kThreads = 32 * (kEpiWarp0 + kEpiWarps);
constexpr int kRegsOther = 72, kRegsEpi = 216;                 // registers a thread after the split
static_assert(128 * kRegsOther + 256 * kRegsEpi <= kThreads * 168, "the split draws on what the block was launched with");
constexpr int kTmemCols = 512, kTmemHalf = 256;
constexpr int kMaxCols = 128;                                  // token columns of a tile
constexpr int kScaleSlots = 4;                                 // turns whose scales may lie ready
constexpr int kScaleFloats = 2 * kMaxCols;                     // of a turn: per k-block those of W0 and of W1
constexpr int kItems = 2, kParts = 4, kAskAhead = 8;           // as in eb_ffn.cu; k-blocks are twice as long here
static_assert(kParts > kItems, "a barrier of the publisher is free again before it comes round");

// shared memory behind the ring
constexpr int kBarOff = kRingBytes;                            // 512 bytes: barriers, TMEM address, abort flag, mailbox
constexpr int kScaleOff = kBarOff + 512;
constexpr int kMaxOff = kScaleOff + kScaleSlots * kScaleFloats * 4;      // [2][4 quadrants][128 columns] largest magnitudes
constexpr int kInvOff = kMaxOff + 2 * 4 * kMaxCols * 4;                  // [warps][64] factors of a warp's columns
constexpr int kTileOff = kInvOff + kEpiWarps * 64 * 4;                   // 1 KB a warp: transposes
constexpr size_t kSmemBytes = (size_t)kTileOff + kEpiWarps * 1024 + 1024 /*alignment slack*/;
static_assert(kSmemBytes <= 232448, "shared memory of one CTA");

// D[tmem of both CTAs] (+)= A * B^T on e4m3 with M = 256 (128 rows of A per CTA), N from the descriptor, K = 32
__device__ __forceinline__ void umma_pair_e4m3(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, {%5, %5, %5, %5, %5, %5, %5, %5}, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(0u)
      : "memory");
}
// Instruction descriptor: fp32 accumulate, e4m3 A and B (format 0), both K-major; M = 256, N token columns.
__device__ __forceinline__ uint32_t instr_desc_e4m3(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((256u >> 4) << 24); }

// Columns that a k-block of a tile takes per accumulator: 32, 64 or 128; a turn is 128 / width k-blocks.
__device__ __forceinline__ int turn_width(int cols) { return cols <= 32 ? 32 : cols <= 64 ? 64 : 128; }

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
// two fp32 multiply-adds
__device__ __forceinline__ void fma2(uint64_t& acc, uint64_t a, uint64_t b) { asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(a), "l"(b)); }
__device__ __forceinline__ ulonglong2 ld_shared2(uint32_t addr) {
  ulonglong2 v;
  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v.x), "=l"(v.y) : "r"(addr));
  return v;
}
__device__ __forceinline__ void st_shared4(uint32_t addr, float a, float b, float c, float d) {
  asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
}

struct TokenMaps8 {
  CUtensorMap box[4];   // 64 / 32 / 16 / 8 rows
};
struct FewParams {
  TokenMaps8 xq, act;
  CUtensorMap gate, up, down;        // weight boxes of 128 rows; with the above kMaps tensor maps in a row
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
constexpr int kMaps = 11;
static_assert(offsetof(FewParams, down) == (kMaps - 1) * sizeof(CUtensorMap), "the maps are prefetched as an array");

// The 32 columns a quadrant's two warps share go to them as 16-column chunks in turn: chunk i of a warp starts at column
// first + 32 i.  acc[a][..]: sums of accumulator a, two columns a word.
template <int NC>
struct Sums {
  uint64_t v[2][NC * 8];
};

// One k-block: acc += TMEM columns * scales.  The next chunk is on its way while one is added.
template <int NC>
__device__ __forceinline__ void add_block(Sums<NC>& s, uint32_t tmem, uint32_t scales, int width) {
  uint32_t r[2][16];
  tmem_ld16(tmem, r[0]);
#pragma unroll
  for (int j = 0; j < 2 * NC; ++j) {
    const int a = j / NC, i = j % NC;
    tmem_ld_wait(r[j & 1]);
    if (j + 1 < 2 * NC) tmem_ld16(tmem + ((j + 1) / NC) * width + 32 * ((j + 1) % NC), r[(j + 1) & 1]);
    const uint32_t at = scales + 4u * (a * width + 32 * i);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const ulonglong2 f = ld_shared2(at + 16 * k);
      fma2(s.v[a][i * 8 + 2 * k], pack2(r[j & 1][4 * k], r[j & 1][4 * k + 1]), f.x);
      fma2(s.v[a][i * 8 + 2 * k + 1], pack2(r[j & 1][4 * k + 2], r[j & 1][4 * k + 3]), f.y);
    }
  }
}

__global__ void __launch_bounds__(kThreads, 1)
ffn8_few_kernel(const __grid_constant__ FewParams p) {
  EB_GRID_DEP_SYNC();
  constexpr int NS = kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (base - raw);
  const uint32_t bar0 = base + kBarOff;
  auto w0_addr = [&](int s) { return base + s * kStageBytes; };
  auto w1_addr = [&](int s) { return base + s * kStageBytes + kWBytes; };
  auto t_addr = [&](int s) { return base + s * kStageBytes + 2 * kWBytes; };
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (NS + s); };
  auto tfull_bar = [&](int h) { return bar0 + 8u * (2 * NS + h); };
  auto tempty_bar = [&](int h) { return bar0 + 8u * (2 * NS + 2 + h); };
  auto item_full = [&](int i) { return bar0 + 8u * (2 * NS + 4 + i); };
  auto item_empty = [&](int i) { return bar0 + 8u * (2 * NS + 4 + kItems + i); };
  const uint32_t want_bar = bar0 + 8u * (2 * NS + 4 + 2 * kItems);
  auto part_bar = [&](int i) { return bar0 + 8u * (2 * NS + 5 + 2 * kItems + i); };
  auto sfull_bar = [&](int i) { return bar0 + 8u * (2 * NS + 5 + 2 * kItems + kParts + i); };
  auto sempty_bar = [&](int i) { return bar0 + 8u * (2 * NS + 5 + 2 * kItems + kParts + kScaleSlots + i); };
  auto max_bar = [&](int i) { return bar0 + 8u * (2 * NS + 5 + 2 * kItems + kParts + 2 * kScaleSlots + i); };
  constexpr int kBarBytes = 8 * (2 * NS + 5 + 2 * kItems + kParts + 2 * kScaleSlots + 2), kMailbox = 512 - kItems * (int)sizeof(Tile);
  static_assert(kBarBytes + 8 <= kMailbox, "512 bytes of barriers and mailbox");
  volatile uint32_t* s_tmem = reinterpret_cast<volatile uint32_t*>(smem + kBarOff + kBarBytes);
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem + kBarOff + kBarBytes + 4);
  const uint32_t items = bar0 + kMailbox;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();   // CTA 0 of a pair is the leader
  int* const status = p.status;
  if (threadIdx.x == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int h = 0; h < 2; ++h) {
      mbar_init(tfull_bar(h), 1);
      mbar_init(tempty_bar(h), 2 * kEpiWarps);   // leader's barrier
      mbar_init(max_bar(h), kEpiWarps / 2);      // the four quadrants' warps of every other chunk
    }
    for (int i = 0; i < kItems; ++i) {
      mbar_init(item_full(i), 1);
      mbar_init(item_empty(i), 7 + 2 * kEpiWarps);   // every reader of both CTAs (CTA 1's barrier)
    }
    for (int i = 0; i < kParts; ++i) mbar_init(part_bar(i), kEpiWarps);
    for (int i = 0; i < kScaleSlots; ++i) {
      mbar_init(sfull_bar(i), 1);
      mbar_init(sempty_bar(i), kEpiWarps);
    }
    mbar_init(want_bar, 1);
    *s_abort = 0;
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
  // The same for a whole warp: one lane takes it and frees the slot (a wait with cluster scope by all 32 takes 6000 cycles).
  auto take_item_warp = [&](int seq, Tile* it) {
    int ok = 1;
    if (lane == 0) {
      ok = take_item(seq, it) ? 1 : 0;
      if (ok && it->w >= 0) mbar_arrive_cluster(map_to_cta(item_empty(seq % kItems), 1));
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

  if (warp < kEpiWarp0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == 0) {
      // ---------------- TMA producer (each CTA loads its own halves) ----------------
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
          const bool merged = it.rows < 0;
          const int half = entry_cols(it.rows) >> 1;   // token rows this CTA loads: 8 .. 64 (of 16 each in a merged tile)
          const int tok0 = it.row + (int)rank * half;
          int slot_row[kMaxCols / kSlotRows / 2];
#pragma unroll
          for (int i = 0; i < kMaxCols / kSlotRows / 2; ++i) {
            const int sl = (int)rank * (half / kSlotRows) + i;
            slot_row[i] = (merged && i < half / kSlotRows) ? __ldg(p.slots + it.row + (sl < -it.rows ? sl : 0)).x : 0;
          }
          const bool down = it.phase == 2;
          const CUtensorMap* tmW0 = down ? &p.down : &p.gate;
          const CUtensorMap* tmW1 = down ? &p.down : &p.up;
          const TokenMaps8* tmT = down ? &p.act : &p.xq;
          const int num_kb = down ? num_kb2 : num_kb1;
          const int wrow0 = it.out * (down ? kFeat2 : kFeat1) + (int)rank * 128;
          const int wrow1 = down ? wrow0 + 256 : wrow0;
          const uint32_t tx = 2u * (2u * kWBytes + (uint32_t)half * BK);
          auto load_weights = [&](int st, int kb) {
            const uint32_t fb = map_to_cta(full_bar(st), 0);
            if (rank == 0) mbar_expect_tx(full_bar(st), tx);
            tma_pair_load_3d(w0_addr(st), tmW0, kb * BK, wrow0, it.w, fb, w_policy);
            tma_pair_load_3d(w1_addr(st), tmW1, kb * BK, wrow1, it.w, fb, w_policy);
          };
          auto load_tokens = [&](int st, int kb) {
            const uint32_t fb = map_to_cta(full_bar(st), 0), ta = t_addr(st);
            if (merged) {
#pragma unroll
              for (int i = 0; i < kMaxCols / kSlotRows / 2; ++i)
                if (i < half / kSlotRows) tma_pair_load_2d(ta + i * (kSlotRows * BK), &tmT->box[2], kb * BK, slot_row[i], fb);
            } else if (half == 64) {
              tma_pair_load_2d(ta, &tmT->box[0], kb * BK, tok0, fb);
            } else {
              int r2 = 0;   // rows placed so far; every box starts on a multiple of 8 rows (1 KB), which keeps the swizzle phase
              if (half & 32) {
                tma_pair_load_2d(ta, &tmT->box[1], kb * BK, tok0, fb);
                r2 = 32;
              }
              if (half & 16) {
                tma_pair_load_2d(ta + r2 * BK, &tmT->box[2], kb * BK, tok0 + r2, fb);
                r2 += 16;
              }
              if (half & 8) tma_pair_load_2d(ta + r2 * BK, &tmT->box[3], kb * BK, tok0 + r2, fb);
            }
          };
          const int ask = num_kb > kAskAhead ? num_kb - kAskAhead : 0;
          int kb = 0;
          if (down) {
            const int* flag = p.ready + it.done;
            if (it.need > 0 && ld_acquire(flag) < it.need) {
              // the rows are still being made: the weights of the stages at hand go ahead of them
              const int lead = num_kb < NS ? num_kb : NS;
              int st = stage;
              uint32_t ph = phase;
              for (int i = 0; i < lead; ++i) {
                if (!mbar_wait(empty_bar(st), ph ^ 1u, s_abort, status)) goto done;
                load_weights(st, i);
                if (++st == NS) {
                  st = 0;
                  ph ^= 1u;
                }
              }
              if (!bounded_wait([&] { return ld_acquire(flag) >= it.need; }, s_abort, status)) goto done;
              fence_proxy_async();
              if (rank == 0 && ask < lead) mbar_arrive_cluster(map_to_cta(want_bar, 1));
              for (; kb < lead; ++kb) {
                load_tokens(stage, kb);
                if (++stage == NS) {
                  stage = 0;
                  phase ^= 1u;
                }
              }
            } else {
              fence_proxy_async();
            }
          }
          for (; kb < num_kb; ++kb) {
            if (rank == 0 && kb == ask) mbar_arrive_cluster(map_to_cta(want_bar, 1));
            if (!mbar_wait(empty_bar(stage), phase ^ 1u, s_abort, status)) goto done;
            load_weights(stage, kb);
            load_tokens(stage, kb);
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
        uint32_t phase = 0, turn = 0;
        for (int seq = 0;; ++seq) {
          Tile it;
          if (!take_item(seq, &it)) goto done;
          if (it.w < 0) break;
          free_item(seq);
          const int num_kb = it.phase == 2 ? num_kb2 : num_kb1;
          const int cols = entry_cols(it.rows), width = turn_width(cols), per = kMaxCols / width;
          const uint32_t idesc = instr_desc_e4m3(cols);
          for (int kb0 = 0; kb0 < num_kb; kb0 += per, ++turn) {
            const int h = turn & 1u, n = min(per, num_kb - kb0);
            if (!mbar_wait(tempty_bar(h), ((turn >> 1) & 1u) ^ 1u, s_abort, status)) goto done;
            tc_fence_after();
            for (int g = 0; g < n; ++g) {
              if (!mbar_wait(full_bar(stage), phase, s_abort, status)) goto done;
              tc_fence_after();
              const uint32_t acc0 = tmem_base + h * kTmemHalf + g * 2 * width, acc1 = acc0 + width;
              const uint64_t d0 = smem_desc(w0_addr(stage)), d1 = smem_desc(w1_addr(stage)), dt = smem_desc(t_addr(stage));
#pragma unroll
              for (int k = 0; k < BK / 32; ++k) {
                umma_pair_e4m3(acc0, d0 + 2 * k, dt + 2 * k, idesc, k != 0 ? 1u : 0u);
                umma_pair_e4m3(acc1, d1 + 2 * k, dt + 2 * k, idesc, k != 0 ? 1u : 0u);
              }
              umma_pair_commit(empty_bar(stage));
              if (++stage == NS) {
                stage = 0;
                phase ^= 1u;
              }
            }
            umma_pair_commit(tfull_bar(h));
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
      // ---------------- scales: token's times weight block's, a turn at a time ----------------
      uint32_t turn = 0;
      for (int seq = 0;; ++seq) {
        Tile it = {};
        if (!take_item_warp(seq, &it)) goto done;
        if (it.w < 0) break;
        const bool down = it.phase == 2;
        const int num_kb = down ? num_kb2 : num_kb1;
        const int width = turn_width(entry_cols(it.rows)), per = kMaxCols / width;
        // this lane: four token columns of k-block g of the turn
        const int g = lane / (width / 4), tok = lane % (width / 4) * 4;
        int row = it.row + tok;
        if (it.rows < 0) row = __ldg(p.slots + it.row + min(tok / kSlotRows, -it.rows - 1)).x + tok % kSlotRows;
        const float *sw0, *sw1;   // of this CTA's 128 rows of W0 and W1; blocks beyond the matrix: the last one's, for sums that nobody stores
        const float* sx[4];
        int step;
        if (down) {
          const size_t mat = (size_t)it.w * num_kb1 * num_kb2;
          sw0 = p.s_down + mat + (size_t)min(it.out * 4 + (int)rank, num_kb1 - 1) * num_kb2;
          sw1 = p.s_down + mat + (size_t)min(it.out * 4 + 2 + (int)rank, num_kb1 - 1) * num_kb2;
          step = p.rows_cap;
        } else {
          const size_t at = (size_t)it.w * num_kb1 * num_kb2 + (size_t)min(it.out * 2 + (int)rank, num_kb2 - 1) * num_kb1;
          sw0 = p.s_gate + at;
          sw1 = p.s_up + at;
          step = 1;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = min(row + i, p.rows_cap - 1);
          sx[i] = down ? p.act_scale + r : p.xs + (size_t)r * num_kb1;
        }
        if (down && it.need > 0) {
          const int* flag = p.ready + it.done;
          int ok = 1;   // one lane asks
          if (lane == 0) ok = bounded_wait([&] { return ld_acquire(flag) >= it.need; }, s_abort, status) ? 1 : 0;
          if (!__shfl_sync(0xffffffffu, ok, 0)) goto done;
          __syncwarp();
        }
        // Those of two turns are on their way at a time: with one, a turn takes as long as its trip to L2 (1000 cycles); four cost spills (2 % at
        // 2048 rows over 191 matrices)
        float x[2][4], w0[2], w1[2];
        auto load = [&](int kb, float (&xk)[4], float& w0k, float& w1k) {
          if (kb >= num_kb) return;
          w0k = __ldg(sw0 + kb);
          w1k = __ldg(sw1 + kb);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            // the intermediate's scales were written by this launch: from L2
            xk[i] = down ? __ldcg(sx[i] + (size_t)kb * step) : __ldg(sx[i] + kb);
          }
        };
#pragma unroll
        for (int j = 0; j < 2; ++j) load(j * per + g, x[j], w0[j], w1[j]);
        for (int kb0 = 0; kb0 < num_kb; kb0 += 2 * per) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int kb = kb0 + j * per;
            if (kb >= num_kb) break;
            const int slot = turn % kScaleSlots;
            int ok = 1;
            if (lane == 0) ok = mbar_wait(sempty_bar(slot), ((turn / kScaleSlots) & 1u) ^ 1u, s_abort, status) ? 1 : 0;
            if (!__shfl_sync(0xffffffffu, ok, 0)) goto done;
            if (kb + g < num_kb) {
              const uint32_t at = base + kScaleOff + 4u * (slot * kScaleFloats + g * 2 * width + tok);
              st_shared4(at, x[j][0] * w0[j], x[j][1] * w0[j], x[j][2] * w0[j], x[j][3] * w0[j]);
              st_shared4(at + 4u * width, x[j][0] * w1[j], x[j][1] * w1[j], x[j][2] * w1[j], x[j][3] * w1[j]);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive_release(sfull_bar(slot));
            ++turn;
            load(kb + 2 * per + g, x[j], w0[j], w1[j]);
          }
        }
      }
    } else {
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
    const int ew = warp - kEpiWarp0, q = warp & 3, side = ew >> 2;   // lane quadrant; which of two 16-column chunks in turn
    const int first = side * 16;
    const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + first;
    const uint32_t scale0 = base + kScaleOff + 4u * first;
    uint32_t* const s_max = reinterpret_cast<uint32_t*>(smem + kMaxOff);
    float* const s_inv = reinterpret_cast<float*>(smem + kInvOff) + ew * 64;
    uint8_t* const tile = smem + kTileOff + ew * 1024;
    uint32_t turn = 0, made = 0;   // made: gate/up tiles so far
    for (int seq = 0;; ++seq) {
      Tile it = {};
      if (!take_item_warp(seq, &it)) goto done;
      if (it.w < 0) break;
      const int cols = entry_cols(it.rows), num_kb = it.phase == 2 ? num_kb2 : num_kb1;
      const bool merged = it.rows < 0;
      const int n_cols = merged ? -it.rows * kSlotRows : it.rows;   // columns that may hold rows to store
      // rows of the 16 columns from c on: first row, how many
      auto chunk_rows = [&](int c, int* row0) {
        if (c >= n_cols) return 0;
        if (merged) {
          const int2 sl = __ldg(p.slots + it.row + (c >> 4));
          *row0 = sl.x;
          return sl.y;
        }
        *row0 = it.row + c;
        return min(16, it.rows - c);
      };
      auto run = [&](auto nc) -> bool {
        constexpr int NC = decltype(nc)::value;
        constexpr int W = NC * 32, PER = kMaxCols / W;
        Sums<NC> s;
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int i = 0; i < NC * 8; ++i) s.v[a][i] = 0;
        for (int kb0 = 0; kb0 < num_kb; kb0 += PER, ++turn) {
          const int h = turn & 1u, slot = turn % kScaleSlots, n = min(PER, num_kb - kb0);
          int ok = 1;   // one lane waits: a wait by all 32 takes 170 cycles
          if (lane == 0) ok = mbar_wait(sfull_bar(slot), (turn / kScaleSlots) & 1u, s_abort, status) && mbar_wait(tfull_bar(h), (turn >> 1) & 1u, s_abort, status) ? 1 : 0;
          if (!__shfl_sync(0xffffffffu, ok, 0)) return false;
          tc_fence_after();
          for (int g = 0; g < n; ++g)
            add_block<NC>(s, taddr + h * kTmemHalf + g * 2 * W, scale0 + 4u * (slot * kScaleFloats + g * 2 * W), W);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive_cluster(map_to_cta(tempty_bar(h), 0));
            mbar_arrive_release(sempty_bar(slot));
          }
        }
        if (it.phase == 1) {
          const int block = it.out * 2 + (int)rank;   // of 128 outputs
          // values, and the largest magnitude of every column over the warp's 32 outputs, left in lane (column % 32)
          uint32_t most[(NC + 1) / 2] = {};
#pragma unroll
          for (int i = 0; i < NC * 8; ++i) {
            const float2 gt = unpack2(s.v[0][i]), up = unpack2(s.v[1][i]);
            float h0, h1;
            silu_mul2(gt.x, up.x, gt.y, up.y, &h0, &h1);
            const uint32_t lo = __float_as_uint(h0), hi = __float_as_uint(h1);
            s.v[0][i] = pack2(lo, hi);
            const uint32_t ml = __reduce_max_sync(0xffffffffu, lo & 0x7fffffffu), mh = __reduce_max_sync(0xffffffffu, hi & 0x7fffffffu);
            if (lane == ((2 * i) & 31)) most[i / 16] = ml;
            if (lane == ((2 * i + 1) & 31)) most[i / 16] = mh;
          }
          uint32_t* const mx = s_max + (made & 1u) * 4 * kMaxCols + side * 64;
#pragma unroll
          for (int k = 0; k < (NC + 1) / 2; ++k) mx[q * kMaxCols + 32 * k + lane] = most[k];
          __syncwarp();
          if (lane == 0) mbar_arrive_release(max_bar(side));
          int ok = 1;
          if (lane == 0) ok = mbar_wait(max_bar(side), made & 1u, s_abort, status) ? 1 : 0;
          if (!__shfl_sync(0xffffffffu, ok, 0)) return false;
          ++made;
#pragma unroll
          for (int k = 0; k < (NC + 1) / 2; ++k) {
            const int c = 32 * k + lane;   // of this warp's columns
            uint32_t m = 0;
#pragma unroll
            for (int r = 0; r < 4; ++r) m = max(m, mx[r * kMaxCols + c]);
            const float top = __uint_as_float(m);
            const bool none = top < 7.70371978e-34f;   // 2^-110
            s_inv[c] = none ? 0.f : __fdiv_rn(kE4M3Max, top);
            if (q == 0 && block < num_kb2 && c < NC * 16) {
              int row0 = 0;
              const int at = (c >> 4) * 32 + first, n = chunk_rows(at, &row0);
              if ((c & 15) < n)
                p.act_scale[(size_t)block * p.rows_cap + row0 + (c & 15)] = m >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : none ? 0.f : __fdiv_rn(top, kE4M3Max);
            }
          }
          __syncwarp();
#pragma unroll
          for (int i = 0; i < NC; ++i) {
            int row0 = 0;
            const int n_here = chunk_rows(first + 32 * i, &row0);
            if (n_here > 0) {
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const float2 v = unpack2(s.v[0][i * 8 + k]), f = *reinterpret_cast<const float2*>(s_inv + 16 * i + 2 * k);
                const unsigned b = pack_e4m3(v.x * f.x, v.y * f.y);
                tile[(2 * k) * 32 + lane] = (uint8_t)b;
                tile[(2 * k + 1) * 32 + lane] = (uint8_t)(b >> 8);
              }
              __syncwarp();
              const int tok = lane >> 1, col = block * 128 + q * 32 + (lane & 1) * 16;
              if (tok < n_here && col < p.I)
                *reinterpret_cast<uint4*>(p.act_out + (size_t)(row0 + tok) * p.I + col) = *reinterpret_cast<const uint4*>(tile + lane * 16);
              __syncwarp();
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive_release(part_bar(seq % kParts));
        } else {
          const int f0 = it.out * kFeat2 + (int)rank * 128 + q * 32;
#pragma unroll
          for (int i = 0; i < NC; ++i) {
            int row0 = 0;
            const int n_here = chunk_rows(first + 32 * i, &row0);
            if (n_here > 0) {
              bf16* const t16 = reinterpret_cast<bf16*>(tile);
#pragma unroll
              for (int a = 0; a < 2; ++a) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  const float2 v = unpack2(s.v[a][i * 8 + k]);
                  const uint32_t b = pack_bf16(v.x, v.y);
                  t16[(2 * k) * 32 + lane] = low_half(b);
                  t16[(2 * k + 1) * 32 + lane] = high_half(b);
                }
                __syncwarp();
                const int col = f0 + 256 * a + (lane & 3) * 8;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const int tok = (lane >> 2) + 8 * h;
                  if (tok < n_here && col < p.H)
                    *reinterpret_cast<uint4*>(p.yp + (size_t)(row0 + tok) * p.H + col) = *reinterpret_cast<const uint4*>(t16 + tok * 32 + (lane & 3) * 8);
                }
                __syncwarp();
              }
            }
          }
        }
        return true;
      };
      bool ok;
      if (cols <= 32) ok = run(std::integral_constant<int, 1>());
      else if (cols <= 64) ok = run(std::integral_constant<int, 2>());
      else ok = run(std::integral_constant<int, 4>());
      if (!ok) goto done;
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

cudaError_t launch_few(eb_ctx* c, cudaStream_t st, const FewParams& p) {
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
  return cudaLaunchKernelEx(&cfg, ffn8_few_kernel, p);
}

}  // namespace

eb_status ebi_ffn8_few_bind(eb_ctx* c) {
  if (eb_status ds = ebi_check_device(c)) return ds;
  const eb_config& g = c->cfg;
  const uint64_t nw = (uint64_t)g.L * (g.E + g.S);
  if (!make_map(&c->tm8_gate, c->w8_gate, g.H, g.I, nw, BK, 128, true) || !make_map(&c->tm8_up, c->w8_up, g.H, g.I, nw, BK, 128, true) ||
      !make_map(&c->tm8_down, c->w8_down, g.I, g.H, nw, BK, 128, true))
    return ebi_fail(c, EB_ERR_CUDA, "cuTensorMapEncodeTiled failed for the weights");
  cudaError_t e = cudaFuncSetAttribute(ffn8_few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
  if (e != cudaSuccess) return ebi_check_cuda(c, e, "cudaFuncSetAttribute");
  c->pair_grid8 = ebi_pair_grid(c, (const void*)ffn8_few_kernel, kThreads, kSmemBytes);
  if (!c->pair_grid8) return ebi_fail(c, EB_ERR_CUDA, "the device cannot hold a 2-CTA cluster of the 8-bit expert kernel");
  return EB_OK;
}

eb_status ebi_ffn8_few_run(eb_ctx* c, cudaStream_t st, const void* xq, const float* xs, const int32_t* group_off, const int32_t* group_w,
                       const int32_t* step_meta, void* yp, int32_t device, bool planned) {
  if (!xq || !xs || !group_off || !group_w || !step_meta || !yp) return ebi_fail(c, EB_ERR_INVALID_ARG, "null pointer");
  if (eb_status ds = ebi_check_device(c)) return ds;
  if (!ebi_aligned16(xq) || !ebi_aligned16(xs) || !ebi_aligned16(yp)) return ebi_fail(c, EB_ERR_INVALID_ARG, "xq / xs / yp must be 16-byte aligned");
  if (!c->w8_gate) return ebi_fail(c, EB_ERR_INVALID_ARG, "8-bit weights not bound");
  if (!c->ws) return ebi_fail(c, EB_ERR_WORKSPACE, "no workspace set");
  const eb_config& g = c->cfg;
  const int rows = ebi_rows_cap(c);
  FewParams p;
  const int box_rows[4] = {64, 32, 16, 8};
  for (int i = 0; i < 4; ++i)
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
    if (eb_status s = ebi_ffn_plan(c, st, group_off, group_w, step_meta, device, EB_PASS_FP8_FEW)) return s;
  if (!c->timing) {
    p.part = 0;
    EB_LAUNCH(c, "expert_ffn_fp8", launch_few(c, st, p));
  } else {   // the same tiles in two launches, so that each phase gets a time of its own
    {
      KernelTimer timer(c, EBK_FFN_GATEUP, st);
      p.part = 1;
      EB_LAUNCH(c, "expert_ffn_fp8", launch_few(c, st, p));
    }
    KernelTimer timer(c, EBK_FFN_DOWN, st);
    p.part = 2;
    EB_LAUNCH(c, "expert_ffn_fp8", launch_few(c, st, p));
  }
  EB_LAUNCH_CHECK(c, "expert_ffn_fp8");
  return EB_OK;
}
