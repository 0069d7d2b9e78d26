// The passes of the softmax operators over tiles of scores, on tensor cores.
//
// One block per SM holds one or two tiles (128 rows) of A and streams tiles of B.  One
// warp loads, one issues the matrix instructions, and two groups of eight warps take
// the tiles of scores out of tensor memory by turns, half a row of a tile per thread.
// For the gradients the probabilities go back in place of their scores, in 16 bits, and
// are the first operand of the second product, whose other operand is the tile of B
// that gave the scores, read along its other dimension.  So the n x V scores and
// probabilities exist only as tiles in tensor memory, and B is loaded once for both.
//
// fp32 (PARTS = 2): S = lo hi + hi lo + hi hi of the operands' halves, and the same for
// p B.  The tensor core's additions round towards zero, so a long sum loses in
// proportion to its length; sums run over at most `run` tiles and are then added in fp32.
//
// Rows and cols pass, 2048 x 120k, GB300 (tensor pipe active / instruction issue /
// exponentials, of their peaks): bf16, K = 64: 67 and 81 us (40/54/44%, 32/43/36%): no one
// of them is full; K = 256: 193 and 208 us (54/21/15%, 50/20/14%) and fp32, K = 100: 258 and
// 224 us (56/23/11%, 65/30/13%): the products, and their waits for loads (a tile of B is 64
// KB at both).  Maxima by high halves, fp32, K = 64: 40 us (33/46/0%): the chain from a
// tile's products to its maxima and back to the buffer.
#include <type_traits>

#include "ptx.cuh"
#include "softmax_mma.cuh"

namespace esspt {

namespace {

// Consecutive tiles of B for one group, all for one slot, cut into runs of a.run.
struct Run {
  int64_t slot, group, first;
  int32_t len;
  bool begins, ends;  // the slot's first run, its last
};

// The block's runs in order, the same for every warp.
struct Walk {
  Ranges r;
  int64_t u, begin, end;
  int run;
  __device__ Walk(const Ranges& r_, int run_) : r(r_), run(run_) {
    begin = u = blockIdx.x < r.blocks ? r.begin(blockIdx.x) : 0;
    end = blockIdx.x < r.blocks ? r.begin(blockIdx.x + 1) : 0;
  }
  __device__ bool next(Run& s) {
    if (u >= end) return false;
    if (u == begin || s.ends) {
      s.group = u / r.n_b;
      s.first = u - s.group * r.n_b;
      s.slot = blockIdx.x + s.group;
      s.begins = true;
    } else {
      s.first += s.len;
      s.begins = false;
    }
    const int64_t left = min(r.n_b - s.first, end - u);
    s.len = (int32_t)min(left, (int64_t)run);
    s.ends = s.len == left;
    u += s.len;
    return true;
  }
};

struct Bars {  // shared addresses
  uint32_t full, empty;             // [stages]
  uint32_t a_full, a_empty;
  uint32_t s_full, s_done;          // [4]: scores are there; scores read, or probabilities written
  uint32_t o_full, o_empty;
};
constexpr int kBarBytes = 8 * (2 * kUnits + 2 + 8 + 2);

template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  uint32_t r;
  if (BF16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// What the two halves of p leave of (lo, hi).
__device__ __forceinline__ uint32_t pack16_rest(uint32_t p, float lo, float hi) {
  const __half2 h = *reinterpret_cast<const __half2*>(&p);
  const float2 f = __half22float2(h);
  float x, y;
  unpack2(fma2(pack2(f.x, f.y), pack2(-1.f, -1.f), pack2(lo, hi)), x, y);
  return pack16<false>(x, y);
}

// Sums: the 128 probabilities of every row (half `part`) times units of B.  They lie in
// the place of their scores, 16 words for 32 values, of halves 8 and 8 for 16 values.
template <int PARTS>
__device__ __forceinline__ void sums_mma(uint32_t d, uint32_t p, int part, uint32_t b, uint32_t idesc, uint32_t add,
                                         uint32_t leader) {
#pragma unroll
  for (int k = 0; k < 8; ++k)
    mma_ts(d, p + (PARTS == 2 ? 16 * k + 8 * part : 32 * (k >> 1) + 8 * (k & 1)), b + 128 * k, idesc, k > 0 ? 1u : add, leader);
}

// A place in the ring of stages, with what is used of it.
struct Ring {
  uint32_t at, bar, phase;  // address, full barrier (the empty one lies kEmpty further), parity
  uint32_t at0, bar0, bytes, end;
  __device__ __forceinline__ Ring(uint32_t at_, uint32_t bar_, uint32_t bytes_, int stages)
      : at(at_), bar(bar_), phase(0), at0(at_), bar0(bar_), bytes(bytes_), end(bar_ + 8 * stages) {}
  __device__ __forceinline__ void next() {
    at += bytes, bar += 8;
    if (bar == end) at = at0, bar = bar0, phase ^= 1;
  }
};
constexpr uint32_t kEmpty = 8 * kUnits;

// The warp that issues the matrix instructions, for rows of NK units.  Everything that
// can be is known at compile time: this one warp works through a chain of instructions
// of a few cycles each, and with the loops and addresses left to run time it took longer
// for them than the tensor cores for the products (K = 256, bf16, scores alone: 2500
// cycles per tile, 1020 of them products).
template <Pass PASS, bool BF16, int PARTS, int NK>
struct Issue {
  static constexpr bool STATS = only_scores(PASS);
  static constexpr MmaShape S = mma_shape(PASS, 64 * NK, PARTS);
  static constexpr uint32_t kIdesc = mma_desc(BF16, 128, false);
  static constexpr uint32_t kUnit = kUnitBytes >> 4;  // in descriptors
  const Bars& bar;
  volatile uint32_t* dead;
  const uint32_t leader, tmem, a_base;
  const int last_steps;  // of a row's last unit
  const int out_cols, out_units;
  Ring ring, kept;       // stages for scores (and for sums, where B is loaded again); for sums of what was kept
  uint32_t done_phase = STATS ? 0xfu : 0u;  // parity to wait for on s_done, a bit per buffer
  uint32_t a_phase = 0, o_phase = 1;

  __device__ __forceinline__ Issue(const Bars& bar_, volatile uint32_t* dead_, uint32_t tmem_, uint32_t a_base_, uint32_t b_base,
                                   int steps, int out_cols_, int out_units_)
      : bar(bar_), dead(dead_), leader(elect_one()), tmem(tmem_), a_base(desc_k(a_base_)), last_steps(steps - 4 * (NK - 1)),
        out_cols(out_cols_), out_units(out_units_), ring(b_base, bar_.full, S.stage_units * kUnitBytes, S.stages), kept(ring) {}

  __device__ __forceinline__ void take(const Ring& r) {  // wait for a stage's loads
    warp_wait(r.bar, r.phase, dead);
    fence_after();
  }
  __device__ __forceinline__ void free(Ring& r) {
    mma_commit(r.bar + kEmpty, leader);
    r.next();
  }
  __device__ __forceinline__ void done(uint32_t buf) {  // wait until its scores were read (or made probabilities)
    warp_wait(bar.s_done + 8 * buf, (done_phase >> buf) & 1, dead);
    done_phase ^= 1u << buf;
    fence_after();
  }
  // Products of one unit of A and of B; STEPS of 16 values.
  template <int STEPS>
  __device__ __forceinline__ void steps(uint32_t d, uint32_t a, uint32_t b, uint32_t add) {
#pragma unroll
    for (int k = 0; k < STEPS; ++k) mma_ss(d, a + 2 * k, b + 2 * k, kIdesc, k > 0 ? 1u : add, leader);
  }
  // All products of a pair of units: of halves in the order of their size, W's lo first
  // whichever operand it is, so that a score is the same number in every pass; lo lies
  // a_lo and b_lo further.
  template <int STEPS>
  __device__ __forceinline__ void pair(uint32_t d, uint32_t a, uint32_t b, uint32_t a_lo, uint32_t b_lo, uint32_t add) {
    if constexpr (PARTS == 2) {
      constexpr bool kItems = items_first(PASS);
      steps<STEPS>(d, kItems ? a + a_lo : a, kItems ? b : b + b_lo, add);
      steps<STEPS>(d, kItems ? a : a + a_lo, kItems ? b + b_lo : b, 1);
      steps<STEPS>(d, a, b, 1);
    } else {
      steps<STEPS>(d, a, b, add);
    }
  }
  __device__ __forceinline__ void pair_last(uint32_t d, uint32_t a, uint32_t b, uint32_t a_lo, uint32_t b_lo, uint32_t add) {
    switch (last_steps) {
      case 1: return pair<1>(d, a, b, a_lo, b_lo, add);
      case 2: return pair<2>(d, a, b, a_lo, b_lo, add);
      case 3: return pair<3>(d, a, b, a_lo, b_lo, add);
      default: return pair<4>(d, a, b, a_lo, b_lo, add);
    }
  }
  // Scores of the next tile of B with NT tiles of A, to buffers at d, d + 128.
  template <int NT>
  __device__ __forceinline__ void scores(uint32_t d) {
    if constexpr (S.stage_units == NK * PARTS) {  // a stage is the tile, as it lies in memory: parts, then units
      take(ring);
      const uint32_t b = desc_k(ring.at);
#pragma unroll
      for (int tile = 0; tile < NT; ++tile) {
#pragma unroll
        for (int kc = 0; kc < NK - 1; ++kc)
          pair<4>(d + 128 * tile, a_base + tile * NK * PARTS * kUnit + kc * kUnit, b + kc * kUnit, NK * kUnit, NK * kUnit, kc > 0);
        pair_last(d + 128 * tile, a_base + tile * NK * PARTS * kUnit + (NK - 1) * kUnit, b + (NK - 1) * kUnit, NK * kUnit, NK * kUnit, NK > 1);
      }
      if (STATS) free(ring);
      else ring.next();
    } else if constexpr (S.stage_units == 2) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        take(ring);
        const uint32_t b = desc_k(ring.at);
        if constexpr (PARTS == 2) {
          if (k == 0) pair<4>(d, a_base, b, NK * kUnit, kUnit, 0);
          else pair_last(d, a_base + kUnit, b, NK * kUnit, kUnit, 1);
        } else {
          pair<4>(d, a_base + 2 * k * kUnit, b, 0, 0, k > 0);
          if (k == 0) pair<4>(d, a_base + kUnit, b + kUnit, 0, 0, 1);
          else pair_last(d, a_base + 3 * kUnit, b + kUnit, 0, 0, 1);
        }
        ring.next();
      }
    } else {
      auto unit = [&](Ring& r) {
        take(r);
        const uint32_t at = desc_k(r.at);
        r.next();
        return at;
      };
#pragma unroll
      for (int kc = 0; kc < NK; ++kc) {
        Ring r = ring;
        uint32_t ua[2] = {a_base + kc * kUnit, a_base + (NK + kc) * kUnit}, ub[2] = {0, 0};
        if constexpr (!S.res) {
#pragma unroll
          for (int p = 0; p < PARTS; ++p) ua[p] = unit(r);
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) ub[p] = unit(r);
#pragma unroll
        for (int tile = 0; tile < NT; ++tile) {
          if (kc < NK - 1)
            pair<4>(d + 128 * tile, ua[0] + tile * NK * PARTS * kUnit, ub[0], ua[1] - ua[0], ub[1] - ub[0], kc > 0);
          else
            pair_last(d + 128 * tile, ua[0] + tile * NK * PARTS * kUnit, ub[0], ua[1] - ua[0], ub[1] - ub[0], kc > 0);
        }
        if constexpr (!STATS && S.keep) {
          ring = r;
        } else {
#pragma unroll
          for (int i = 0; i < (S.res ? 1 : 2) * PARTS; ++i) free(ring);
        }
      }
    }
  }
  // Sums of the next tile of B from the probabilities in buffer `buf`.
  __device__ __forceinline__ void sums(uint32_t buf, uint32_t more) {
    done(buf);
    const uint32_t p = tmem + 128 * buf, d = tmem + 128 * S.buffers;
    if constexpr (S.cross) {
      // hi (hi | lo) and lo hi: a stage is the two halves of a unit, 128 columns, and so are
      // the sums of the products of halves hi hi, and of hi lo and lo hi.
#pragma unroll
      for (int kc = 0; kc < NK; ++kc) {
        const uint32_t b = desc_mn(kept.at), to = d + 128 * kc;
        sums_mma<PARTS>(to, p, 0, b, mma_desc(BF16, 128, true), more, leader);
        sums_mma<PARTS>(to + 64, p, 1, b, mma_desc(BF16, min(64, out_cols - 64 * kc), true), 1, leader);
        free(kept);
      }
    } else if constexpr (S.stage_units == 2 && NK == 4) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (k == 1 && out_cols <= 128) break;
        sums_mma<PARTS>(d + 128 * k, p, 0, desc_mn(kept.at), mma_desc(BF16, min(128, out_cols - 128 * k), true), more, leader);
        free(kept);
      }
    } else if constexpr (S.stage_units == NK * PARTS) {
      sums_mma<PARTS>(d, p, 0, desc_mn(kept.at), mma_desc(BF16, out_cols, true), more, leader);
      free(kept);
    } else {
      Ring& from = S.keep ? kept : ring;
      constexpr int kMost = NK < 4 ? NK : 4;
#pragma unroll
      for (int kc = 0; kc < kMost; ++kc) {
        if (kc >= out_units) break;
        const uint32_t idesc = mma_desc(BF16, min(64, out_cols - 64 * kc), true);
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          if (!S.keep) take(from);
          const uint32_t b = desc_mn(from.at);
          if (PARTS == 2 && part == 0) sums_mma<PARTS>(d + 64 * kc, p, 1, b, idesc, more, leader);
          sums_mma<PARTS>(d + 64 * kc, p, 0, b, idesc, PARTS == 2 ? 1 : more, leader);
          free(from);
        }
      }
    }
  }
  __device__ __forceinline__ void run(int nt, const Run& g) {
    const int32_t len = g.len;
    if (S.res && g.begins) {
      warp_wait(bar.a_full, a_phase, dead);
      a_phase ^= 1;
    }
    if constexpr (STATS) {
      for (int32_t j = 0; j < len; ++j) {
        if (S.tiles == 2 && nt == 2) {
          const uint32_t buf = (j & 1) * 2;
          done(buf), done(buf + 1);
          scores<2>(tmem + 128 * buf);
          mma_commit(bar.s_full + 8 * buf, leader), mma_commit(bar.s_full + 8 * buf + 8, leader);
        } else {
          const uint32_t buf = j & 3;
          done(buf);
          scores<1>(tmem + 128 * buf);
          mma_commit(bar.s_full + 8 * buf, leader);
        }
      }
      if (S.res) mma_commit(bar.a_empty, leader);
    } else {
      // Scores run ahead of the sums by all buffers but one, so that the exponentials
      // of the next tiles need not wait for them.
      constexpr uint32_t kAhead = S.buffers - 1;
      uint32_t buf = 0, next = 0;  // of the next sums and scores
      auto ahead = [&](bool last) {
        scores<1>(tmem + 128 * next);
        mma_commit(bar.s_full + 8 * next, leader);
        if (last && S.res && g.ends) mma_commit(bar.a_empty, leader);
        if (++next == S.buffers) next = 0;
      };
      for (int32_t j = 0; j < (int32_t)kAhead && j < len; ++j) ahead(j == len - 1);
      warp_wait(bar.o_empty, o_phase, dead);  // the last run's sums have been read
      o_phase ^= 1;
      fence_after();
      for (int32_t j = 0; j < len; ++j) {
        if (j + (int32_t)kAhead < len) ahead(j + (int32_t)kAhead == len - 1);
        sums(buf, j > 0);
        if (++buf == S.buffers) buf = 0;
      }
      mma_commit(bar.o_full, leader);
    }
  }
};

__device__ __forceinline__ float max3(float x, float y, float z) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}

// x y + z rounded after each operation.  (The intrinsics are never contracted; the packed
// instructions are.)
__device__ __forceinline__ float mul_then_add(float x, float y, float z) { return __fadd_rn(__fmul_rn(x, y), z); }

// Scores of columns from `left` on become -infinity.  Only a tile at the end of B has
// any: a branch of its own (as selects these were most of the instructions).
__device__ __forceinline__ void mask_scores(uint32_t (&r)[32], int left) {
  if (left >= 32) return;
  asm volatile("");
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (i >= left) r[i] = 0xff800000u;
}

// PARTS of the STORED parts of the operands, which come first in memory.
template <Pass PASS, bool BF16, int PARTS, int STORED>
__device__ __forceinline__ void mma_pass(const MmaArgs& a, const MmaShape& sh) {
  extern __shared__ __align__(1024) char smem[];
  __shared__ uint32_t tmem_at;
  __shared__ uint32_t dead_flag;
  constexpr bool STATS = only_scores(PASS);
  constexpr int kColBytes = PARTS == 2 && PASS == Pass::kCols ? 1024 : 512;  // of a tile's columns
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int64_t rows_h = a.words->rows;
  const bool looking = PASS == Pass::kMaxCols && a.low != nullptr;
  const int64_t rows_a = items_first(PASS) ? a.V : rows_h, rows_b = !items_first(PASS) ? a.V : looking ? min(rows_h, (int64_t)128) : rows_h;
  const Ranges ranges(rows_a, rows_b, sh.tiles, gridDim.x);
  if (blockIdx.x >= ranges.blocks || (a.if_redo && a.words->redo == 0u)) return;
  if (PASS == Pass::kMaxCols && ((a.if_apart && !weights_apart(*a.words)) || (a.if_low && a.words->low == 0u))) return;

  const uint32_t base = (smem_addr(smem) + 1023u) & ~1023u;
  const uint32_t a_base = base, b_base = base + (sh.res ? sh.tiles * sh.nk * PARTS : 0) * kUnitBytes;
  const uint32_t col_base = base + kUnits * kUnitBytes;  // [col_slots] of the columns' data
  const char* col_data = smem + (col_base - smem_addr(smem));
  const int col_slots = sh.stages + (PASS == Pass::kMaxCols ? kTopSlots : 0);
  const uint32_t bar0 = col_base + kUnits * 1024;
  Bars bar;
  bar.full = bar0, bar.empty = bar.full + kEmpty, bar.a_full = bar.empty + 8 * kUnits, bar.a_empty = bar.a_full + 8;
  bar.s_full = bar.a_empty + 8, bar.s_done = bar.s_full + 32, bar.o_full = bar.s_done + 32, bar.o_empty = bar.o_full + 8;
  volatile uint32_t* dead = &dead_flag;

  if (threadIdx.x == 0) {
    dead_flag = 0;
    for (int i = 0; i < sh.stages; ++i) mbar_init(bar.full + 8 * i, 1), mbar_init(bar.empty + 8 * i, 1);
    mbar_init(bar.a_full, 1), mbar_init(bar.a_empty, 1);
    for (int i = 0; i < 4; ++i) mbar_init(bar.s_full + 8 * i, 1), mbar_init(bar.s_done + 8 * i, 8);
    mbar_init(bar.o_full, 1), mbar_init(bar.o_empty, 16);
    mbar_init_fence();
  }
  if (warp == 1) tmem_alloc(&tmem_at, 512);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_at;
  const int out_unit = blockIdx.y * 4;  // first unit of the columns summed here
  const int out_units = min(4, sh.nk - out_unit);
  const int out_cols = min(256, sh.steps * 16 - (int)blockIdx.y * 256);
  Walk walk(ranges, a.run);
  Run g;
  // A group's last tile may lie outside: then the groups of warps share the first.
  auto tiles_of = [&](const Run& s) { return sh.tiles == 2 && (s.group * 2 + 1) * 128 < rows_a ? 2 : 1; };
  const int64_t tile_bytes = (int64_t)sh.nk * STORED * kUnitBytes;  // from a tile to the next

  if (warp == 0) {
    // ---- loads ----
    if (lane == 0) {
      Ring ring(b_base, bar.full, sh.stage_units * kUnitBytes, sh.stages);
      int col = 0;  // slot of the column data
      uint32_t a_phase = 1, loads = 0, segs = 0;
      const uint32_t stage_bytes = sh.stage_units * kUnitBytes;
      // A stage of what lies at `from`, or its second unit `apart` further on.
      auto load = [&](const char* from, const char* cols, uint32_t apart = 0) {
        mbar_wait(ring.bar + kEmpty, ring.phase ^ 1, dead);
        if (*dead) return;
        mbar_expect(ring.bar, stage_bytes + (cols ? kColBytes : 0));
        bulk_load(ring.at, from, apart ? kUnitBytes : stage_bytes, ring.bar);
        if (apart) bulk_load(ring.at + kUnitBytes, from + apart, kUnitBytes, ring.bar);
        if (cols) bulk_load(col_base + col * kColBytes, cols, kColBytes, ring.bar);
        ring.next();
        ++loads;
      };
      auto scores_units = [&](int64_t tile, const char* from_a) {
        const char* from = a.B + tile * tile_bytes;
        const char* cols = items_first(PASS) ? reinterpret_cast<const char*>(a.col) + tile * kColBytes : nullptr;
        if (sh.stage_units == sh.nk * PARTS) {
          load(from, cols);
        } else if (sh.stage_units == 2) {  // two units of a row's, or the halves of one
          for (int k = 0; k < 2; ++k)
            load(from + k * (PARTS == 2 ? 1 : 2) * kUnitBytes, k == 0 ? cols : nullptr, PARTS == 2 ? sh.nk * kUnitBytes : 0);
        } else {
          for (int kc = 0; kc < sh.nk; ++kc) {
            if (!sh.res)
              for (int p = 0; p < PARTS; ++p) load(from_a + (p * sh.nk + kc) * (int64_t)kUnitBytes, nullptr);
            for (int p = 0; p < PARTS; ++p)
              load(from + (p * sh.nk + kc) * (int64_t)kUnitBytes, kc == 0 && p == 0 ? cols : nullptr);
          }
        }
        if (++col == col_slots) col = 0;
      };
      auto sums_units = [&](int64_t tile) {
        const char* from = a.B + tile * tile_bytes;
        for (int kc = out_unit; kc < out_unit + out_units; ++kc)
          for (int p = 0; p < PARTS; ++p) load(from + (p * sh.nk + kc) * (int64_t)kUnitBytes, nullptr);
      };
      while (walk.next(g)) {
        const int nt = tiles_of(g);
        const char* from_a = a.A + g.group * sh.tiles * tile_bytes;
        if (sh.res && g.begins) {
          mbar_wait(bar.a_empty, a_phase, dead);
          a_phase ^= 1;
          if (*dead) break;
          ++segs;
          const uint32_t kept = sh.nk * PARTS * kUnitBytes;
          mbar_expect(bar.a_full, nt * kept);
          for (int i = 0; i < nt; ++i) bulk_load(a_base + i * kept, from_a + i * tile_bytes, kept, bar.a_full);
        }
        for (int32_t j = 0; j < g.len; ++j) {
          scores_units(g.first + j, from_a);
          if (!STATS && !sh.keep && j > 0) sums_units(g.first + j - 1);
        }
        if (!STATS && !sh.keep) sums_units(g.first + g.len - 1);
      }
      if (*dead) {  // copies in flight land before the block ends
        for (uint32_t i = 0; i < (uint32_t)sh.stages && i < loads; ++i) {
          const uint32_t n = loads - 1 - i;
          for (int k = 0; k < (1 << 16) && !mbar_try(bar.full + 8 * (n % sh.stages), (n / sh.stages) & 1); ++k) {
          }
        }
        for (int k = 0; k < (1 << 16) && segs > 0 && !mbar_try(bar.a_full, (segs - 1) & 1); ++k) {
        }
      }
    }
  } else if (warp == 1) {
    // ---- matrix instructions ----
    auto issue = [&](auto nk) {
      Issue<PASS, BF16, PARTS, decltype(nk)::value> m(bar, dead, tmem, a_base, b_base, sh.steps, out_cols, out_units);
      while (walk.next(g)) m.run(tiles_of(g), g);
    };
    using std::integral_constant;
    switch (sh.nk) {
      case 1: issue(integral_constant<int, 1>{}); break;
      case 2: issue(integral_constant<int, 2>{}); break;
      case 3: issue(integral_constant<int, 3>{}); break;
      case 4: issue(integral_constant<int, 4>{}); break;
      case 5: issue(integral_constant<int, 5>{}); break;
      case 6: issue(integral_constant<int, 6>{}); break;
      case 7: issue(integral_constant<int, 7>{}); break;
      default: issue(integral_constant<int, 8>{});
    }
    if (*dead) {  // what was issued ends before tensor memory is freed
      const long long begin = clock64();
      while (clock64() - begin < 2'000'000) {
      }
    }
  } else if (warp >= 4) {
    // ---- exponentials ----
    const int pair = (warp - 4) >> 3, half = ((warp - 4) >> 2) & 1, quarter = warp & 3;
    const int row = quarter * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    const int shift_h = half_shift_of(a.words->max_h), shift_w = half_shift_of(a.words->max_w);  // (16-bit rows: 0)
    const float scale_all = ldexpf(a.b * kLog2e, -(shift_h + shift_w));
    float scale = 0.f;  // of this thread's row
    const bool negative = PASS == Pass::kCols && a.words->negative != 0u;
    // Tiles of what is rare (rows past kHuge, rows of B with powers of their own) go a way of
    // their own, by vote: the control flow of a warp stays one.
    const bool slow_cols = __any_sync(0xffffffffu, (items_first(PASS) && a.words->huge != 0u) ||
                                                       (PARTS == 2 && (items_first(PASS) ? a.words->spread_h : a.words->spread_w) != 0u));
    uint32_t phase = 0, o_phase = 0;  // parities of s_full's next turn, a bit per buffer
    int col0 = 0;  // slot of the run's first column data
    float up = 0.f;  // kCols: item_up
    float m = 0.f, l = 0.f, at = 0.f;  // kStats, kMax: maximum (without the scale), sum, and m scale; kRows: sum
    while (walk.next(g)) {
      const int nt = tiles_of(g);
      const int32_t jobs = nt * g.len;
      if (g.begins) {
        m = -INFINITY, l = 0.f, at = 0.f;
        // (Kept off 0 and infinity: scores that far are 0 or overflow in any case, and
        // masked ones stay -infinity.)
        const int64_t r = (g.group * sh.tiles + (nt == 2 ? pair : 0)) * 128 + row;
        scale = fminf(fmaxf(PARTS == 2 ? scale_all * a.scale_a[r].c : scale_all, 1.1754944e-38f), 3.4028235e38f);
      }
      const u64 scale2 = pack2(scale, scale);
      float minus_m = 0.f;
      bool slow = slow_cols;
      if (PASS == Pass::kRows) {
        const int64_t r = g.group * 128 + row;
        minus_m = r < rows_a ? -a.row_max[r] : -1e30f;
        slow |= __any_sync(0xffffffffu, r < rows_a && fabsf(minus_m) > kHuge);
      }
      const float offset = minus_m + a.up;
      if (PASS == Pass::kCols && !BF16 && g.begins) {
        const int64_t item = g.group * 128 + row;
        up = item < rows_a ? item_up<BF16, PARTS>(*a.words, a.item_top, item) : 0.f;
      }
      // Jobs go to the pairs by turns, and to the buffers by turns: with three buffers
      // both pairs come by each, so a pair counts the other's turns too.
      int col = col0, buf = 0;
      for (int32_t n = 0; n < jobs; ++n) {
        const int at_buf = buf, at_col = col;
        if (++buf == sh.buffers) buf = 0;
        if (nt == 1 || (n & 1)) col = col + 1 == col_slots ? 0 : col + 1;
        const uint32_t parity = (phase >> at_buf) & 1;
        phase ^= 1u << at_buf;
        if ((n & 1) != pair) continue;
        const int32_t j = nt == 2 ? n >> 1 : n;
        warp_wait(bar.s_full + 8 * at_buf, parity, dead);
        fence_after();
        const int left = (int)min((int64_t)64, rows_b - (g.first + j) * 128 - 64 * half);  // of this half's columns
        const uint32_t s_at = lanes + 128 * at_buf + 64 * half;
        if (PARTS == 2 || !only_scores(PASS) || PASS == Pass::kMaxCols) {
          if (slow) {
            // 16 columns at a time, scores rounded before maxima come off, column data by
            // ordinary loads.
            const int64_t from = (g.first + j) * 128 + 64 * half;
            const float times_up = exp2f(up);
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              uint32_t x[16], hi[8];
              tmem_load(x, s_at + 16 * c);
              float p[16];
              float m2 = m;
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int64_t col = from + 16 * c + i;
                const bool on = 16 * c + i < left;
                const RowScale k = PARTS == 2 ? a.scale_b[col] : RowScale{1.f, 0.f};
                const float s = __uint_as_float(x[i]) * k.c;
                if (PASS == Pass::kStats) {
                  p[i] = on ? s : -INFINITY;
                  m2 = fmaxf(m2, p[i]);
                } else if (PASS == Pass::kMax) {
                  m2 = on ? fmaxf(m2, mul_then_add(s, scale, k.log2_c)) : m2;
                } else if (PASS == Pass::kRows) {
                  const float q = on ? exp2_fast(mul_then_add(s, scale, minus_m) + a.up) : 0.f;
                  l += q;
                  p[i] = q * k.c;
                } else {
                  const float q = mul_then_add(s, scale, a.col_m[col]);
                  if (PASS == Pass::kMaxCols) m2 = fmaxf(m2, q + log2f(fabsf(a.col_f[col])));
                  else p[i] = exp2_fast(q) * (a.col_f[col] * times_up);
                }
              }
              if (PASS == Pass::kStats) {
                const float at2 = m2 == -INFINITY ? 0.f : m2 * scale;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) sum += exp2_fast(mul_then_add(p[i], scale, -at2));
                l = fmaf(l, m2 == m ? 1.f : m == -INFINITY ? 0.f : exp2_fast(at - at2), sum);
                at = at2;
              }
              if (PASS == Pass::kMax) at = m2;
              if (STATS) {
                m = m2;
                continue;
              }
#pragma unroll
              for (int i = 0; i < 8; ++i) hi[i] = pack16<BF16>(p[2 * i], p[2 * i + 1]);
              if constexpr (PARTS == 2) {
                uint32_t out[16];
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = hi[i], out[8 + i] = pack16_rest(hi[i], p[2 * i], p[2 * i + 1]);
                tmem_store16(s_at + 16 * c, out);
              } else {
                tmem_store8(s_at + 32 * (c >> 1) + 8 * (c & 1), hi);
              }
            }
            if (!STATS) tmem_wait_store();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar.s_done + 8 * at_buf);
            continue;
          }
        }
        // (fp32 rows: 32 columns at a time, for the registers.)
        constexpr bool kBoth = STATS || PARTS == 1;
        uint32_t r[kBoth ? 2 : 1][32];
        if constexpr (kBoth) tmem_load(r[0], s_at, r[1], s_at + 32);
        else tmem_load(r[0], s_at);
        if constexpr (STATS && PASS != Pass::kMaxCols) {
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar.s_done + 8 * at_buf);
        }
        if constexpr (PASS == Pass::kMaxCols) {
          // (Columns after the last: the column data says -infinity.)
          const ulonglong2* cols = reinterpret_cast<const ulonglong2*>(col_data + at_col * kColBytes + kColBytes / 2 * half);
          float top[4] = {m, m, m, m};
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              const ulonglong2 q = cols[8 * c + i / 4];
              float x, y;
              unpack2(fma2(pack2(__uint_as_float(r[c][i]), __uint_as_float(r[c][i + 1])), scale2, q.x), x, y);
              top[(i >> 1) & 3] = max3(top[(i >> 1) & 3], x, y);
              unpack2(fma2(pack2(__uint_as_float(r[c][i + 2]), __uint_as_float(r[c][i + 3])), scale2, q.y), x, y);
              top[(i >> 1 & 3) + 1] = max3(top[(i >> 1 & 3) + 1], x, y);
            }
          m = fmaxf(max3(top[0], top[1], top[2]), top[3]);
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar.s_done + 8 * at_buf);
        } else if constexpr (STATS) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            mask_scores(r[c], left - 32 * c);
            float top[4] = {m, m, m, m};
#pragma unroll
            for (int i = 0; i < 32; i += 2)
              top[(i >> 1) & 3] = max3(top[(i >> 1) & 3], __uint_as_float(r[c][i]), __uint_as_float(r[c][i + 1]));
            const float m2 = fmaxf(max3(top[0], top[1], top[2]), top[3]);
            if constexpr (PASS == Pass::kMax) {
              m = m2, at = m2 * scale;
              continue;
            }
            const float at2 = m2 == -INFINITY ? 0.f : m2 * scale;
            const u64 minus = pack2(-at2, -at2);
            u64 sum[2] = {0ull, 0ull};
            if (__any_sync(0xffffffffu, fabsf(at2) > kHuge)) {
              float e = 0.f;
#pragma unroll
              for (int i = 0; i < 32; ++i) e += exp2_fast(mul_then_add(__uint_as_float(r[c][i]), scale, -at2));
              sum[0] = pack2(e, 0.f);
            } else {
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                float x, y;
                unpack2(fma2(pack2(__uint_as_float(r[c][i]), __uint_as_float(r[c][i + 1])), scale2, minus), x, y);
                sum[(i >> 1) & 1] = add2(sum[(i >> 1) & 1], pack2(exp2_fast(x), exp2_fast(y)));
              }
            }
            // (The same maximum again has to leave l as it is: a factor off by its rounding
            // drifted by 7e-6 over 800 tiles.)
            const float keep = m2 == m ? 1.f : m == -INFINITY ? 0.f : exp2_fast(at - at2);
            l = fmaf(l, keep, sum2(add2(sum[0], sum[1])));
            m = m2, at = at2;
          }
        } else {
          const ulonglong2* cols = reinterpret_cast<const ulonglong2*>(col_data + at_col * kColBytes + kColBytes / 2 * half);
          const u64 offset2 = pack2(offset, offset);
          const float times_up = PARTS == 2 ? exp2f(up) : 0.f;
          const u64 up2 = PARTS == 2 ? pack2(times_up, times_up) : pack2(up, up);
          u64 sum[2] = {0ull, 0ull};
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            if (!kBoth && c == 1) tmem_load(r[0], s_at + 32);
            if (PASS == Pass::kRows) mask_scores(r[kBoth ? c : 0], left - 32 * c);
            // 16 words at a time: 32 values, or the halves of 16.
#pragma unroll
            for (int i0 = 0; i0 < 32; i0 += 32 / PARTS) {
              uint32_t out[16];
#pragma unroll
              for (int i = i0; i < i0 + 32 / PARTS; i += 2) {
                const u64 s2 = pack2(__uint_as_float(r[kBoth ? c : 0][i]), __uint_as_float(r[kBoth ? c : 0][i + 1]));
                float p[2];
                if (PASS == Pass::kRows) {
                  unpack2(fma2(s2, scale2, offset2), p[0], p[1]);
                  p[0] = exp2_fast(p[0]), p[1] = exp2_fast(p[1]);
                  sum[(i >> 1) & 1] = add2(sum[(i >> 1) & 1], pack2(p[0], p[1]));
                } else if (PARTS == 2) {
                  const ulonglong2 q = cols[16 * c + i / 2];
                  unpack2(fma2(s2, scale2, q.x), p[0], p[1]);
                  unpack2(mul2(pack2(exp2_fast(p[0]), exp2_fast(p[1])), mul2(q.y, up2)), p[0], p[1]);
                } else {
                  const ulonglong2 q = cols[8 * c + i / 4];
                  const u64 k = i & 2 ? q.y : q.x;
                  unpack2(fma2(s2, scale2, BF16 ? k : add2(k, up2)), p[0], p[1]);
                  p[0] = exp2_fast(p[0]), p[1] = exp2_fast(p[1]);
                  if (negative) {  // a factor's sign is the lowest bit of its logarithm
                    p[0] = __uint_as_float(__float_as_uint(p[0]) ^ ((uint32_t)k << 31));
                    p[1] = __uint_as_float(__float_as_uint(p[1]) ^ ((uint32_t)(k >> 32) << 31));
                  }
                }
                const int o = (i - i0) / 2;
                out[o] = pack16<BF16>(p[0], p[1]);
                if constexpr (PARTS == 2) out[8 + o] = pack16_rest(out[o], p[0], p[1]);
              }
              tmem_store16(s_at + 32 * c + i0, out);
            }
          }
          tmem_wait_store();
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar.s_done + 8 * at_buf);
          if (PASS == Pass::kRows) l += sum2(add2(sum[0], sum[1]));
        }
      }
      if (PASS == Pass::kRows && a.sums && g.ends && blockIdx.y == 0) a.sums[(g.slot * 4 + 2 * pair + half) * 128 + row] = l;
      if (items_first(PASS)) col0 = (col0 + g.len) % col_slots;
      if (PASS == Pass::kMaxCols) {
        const int64_t item = (g.group * sh.tiles + (nt == 2 ? pair : 0)) * 128 + row;
        if (looking) {  // (each half of a tile for itself; a single tile is one pair's alone)
          if (item < rows_a && jobs > pair && !(m - log2f(__uint_as_float(a.words->max_weight)) >= kLow)) *a.low = 1u;
        } else if (item < rows_a && m != -INFINITY) {
          atomicMax(a.item_top + item, top_key(m));
        }
        continue;
      }
      if (STATS) {
        a.stat[(g.slot * 4 + 2 * pair + half) * 128 + row] = make_float2(m == -INFINITY ? m : at, l);
        continue;
      }
      warp_wait(bar.o_full, o_phase, dead);
      o_phase ^= 1;
      fence_after();
      float* to = a.out + (g.slot * 128 + row) * (int64_t)a.ld + blockIdx.y * 256;
      const uint32_t o_at = lanes + 128 * sh.buffers;
      for (int c = 2 * pair + half; 16 * c < out_cols; c += 4) {
        // (What is added to is on its way while tensor memory is read.)
        float4* p = reinterpret_cast<float4*>(to + 16 * c);
        float4 y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = g.begins ? make_float4(0.f, 0.f, 0.f, 0.f) : p[i];
        uint32_t v[16];
        if (PARTS == 2 && sh.cross) {
          uint32_t x[16];
          const uint32_t at16 = o_at + 128 * (c >> 2) + 16 * (c & 3);
          tmem_load(v, at16, x, at16 + 64);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(x[i]));
        } else {
          tmem_load(v, o_at + 16 * c);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          p[i] = make_float4(y[i].x + __uint_as_float(v[4 * i]), y[i].y + __uint_as_float(v[4 * i + 1]),
                             y[i].z + __uint_as_float(v[4 * i + 2]), y[i].w + __uint_as_float(v[4 * i + 3]));
      }
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar.o_empty);
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && dead_flag) atomicOr(a.status, kErrStuck);
  if (warp == 1) tmem_free(tmem, 512);
}

template <Pass PASS, bool BF16, int PARTS>
__global__ void __launch_bounds__(kMmaThreads, 1) mma_kernel(const __grid_constant__ MmaArgs a) {
  if constexpr (PARTS == 2 && (PASS == Pass::kMax || PASS == Pass::kMaxCols)) {
    if (a.try_high && high_halves_do(*a.words, a.b)) {
      mma_pass<PASS, BF16, 1, 2>(a, a.high);
      return;
    }
  }
  mma_pass<PASS, BF16, PARTS, PARTS>(a, a.s);
}

template <Pass PASS, bool BF16, int PARTS>
cudaError_t launch(const MmaArgs& a, int blocks, int out_chunks, cudaStream_t st) {
  constexpr int kSmem = 1024 + kUnits * (kUnitBytes + 1024) + kBarBytes;
  auto kernel = mma_kernel<PASS, BF16, PARTS>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (e != cudaSuccess) return e;
  kernel<<<dim3(blocks, out_chunks), kMmaThreads, kSmem, st>>>(a);
  return cudaGetLastError();
}

template <Pass PASS>
cudaError_t launch_type(bool bf16, int parts, const MmaArgs& a, int blocks, int out_chunks, cudaStream_t st) {
  if (parts == 2) return launch<PASS, false, 2>(a, blocks, out_chunks, st);
  if (bf16) return launch<PASS, true, 1>(a, blocks, out_chunks, st);
  return launch<PASS, false, 1>(a, blocks, out_chunks, st);
}

}  // namespace

cudaError_t launch_mma(Pass pass, bool bf16, int parts, const MmaArgs& a, int blocks, int out_chunks, cudaStream_t st) {
  if (pass == Pass::kStats) return launch_type<Pass::kStats>(bf16, parts, a, blocks, 1, st);
  if (pass == Pass::kMax) return launch_type<Pass::kMax>(bf16, parts, a, blocks, 1, st);
  if (pass == Pass::kMaxCols)  // (bf16 rows have none)
    return parts == 2 ? launch<Pass::kMaxCols, false, 2>(a, blocks, 1, st) : launch<Pass::kMaxCols, false, 1>(a, blocks, 1, st);
  if (pass == Pass::kRows) return launch_type<Pass::kRows>(bf16, parts, a, blocks, out_chunks, st);
  return launch_type<Pass::kCols>(bf16, parts, a, blocks, out_chunks, st);
}

}  // namespace esspt
