// The products of a linear layer held in 8 bits by blocks of 128 (include/falqon_dense.h), on the tensor cores:
//   D[M][N] = sum over k of  a[i][k] * 2^(ea[i][k / 128] - 127) * b[j][k] * 2^(eb[j][k / 128] - 127)
// The scales are powers of two, so the tensor core applies them itself (tcgen05.mma kind::mxf8f6f4.block_scale, whose blocks of 32
// take the same byte four times) and a tile is accumulated in fp32 over all of K without leaving tensor memory; scales that are
// not powers of two would have to be applied to every partial tile of 128 on its way through registers.
//
// Two CTAs of a cluster compute a tile of 256 x block_n (one tcgen05.mma cta_group::2), a persistent pair walking its tiles (tile_walk.cuh):
//   warp 0        TMA producer: up to 128 rows of A and block_n / 2 rows of B per CTA and stage of 128 values of K
//   warp 1        (leader) issues the MMAs
//   warps 2..9    epilogue: tensor memory -> registers -> shared memory -> full 128-byte lines     (4..11 where sums are held in registers)
//   warps 10..13  (12..15) scales: global memory -> tensor memory (tcgen05.st), four blocks of K at a time, the four bytes of a word
// Tensor memory: the scales' ring takes 64 of the 512 columns, which leaves 448 for two accumulators of up to 256.  They overlap in
// columns 192..255, and the epilogue reads those first: the next tile's MMAs start as soon as they are in registers, so that the
// rest of the epilogue runs beside them.
// The three products differ in how the codes lie (K-major or MN-major, no transposed copies) and in the strides of their scales.
// Few tiles and a long contraction: a cluster of four or eight CTAs shares a tile, its pairs' parts added up in order through shared memory.
// What bounds it: 4096 x 4096 x 11008 forward, 145 to 163 us (2.3 to 2.55 PFLOP/s), has the MMAs running 73 % of the time at 1.54 GHz (135 us
// under the profiler; 79 % while an SM has work), the rest being the last of 9.3 waves and the pipeline's ends; with few rows the MMAs, which
// take 0.22 us a block of K however narrow the tile is.
// fp32 results: the tensor cores' additions cut off instead of rounding, so sums are taken out of tensor memory every 2048 terms and added up in
// registers, 128 of them a thread (kSums), to which the other warps hand theirs.  Of the norm, with scales that differ from block to
// block: 4096 terms 1.9e-6 in one sum, 9.7e-7 in two (a plain fp32 product 7.8e-7); 16384 terms 3.8e-6 in parts of 8192 and 9.8e-7 (1.6e-6).  A part more costs
// 0.8 us, in which the MMAs wait: 4096^3 61 -> 65 us, in parts of 1024 terms 72.
// Every wait is bounded; on a timeout the CTA records it, drains and frees its tensor memory.
#include <cuda.h>

#include <algorithm>
#include <atomic>

#include "../../include/falqon_dense.h"
#include "block_linear.h"
#include "gemm_common.cuh"
#include "internal.h"
#include "ptx.cuh"
#include "tile_walk.cuh"

namespace falqon {
namespace {

constexpr int kEpiWarps = 8, kScaleWarps = 4;
// Warps: TMA producer, MMA issuer, (kSums: two that fill up their group,) epilogue, scales.  kSums' epilogue holds 128 sums a thread: the groups of
// four warps hand registers over (sum of the shares: what the CTA is launched with).
template <bool kSums>
struct Roles {
  static constexpr int kEpi = kSums ? 4 : 2, kScale = kEpi + kEpiWarps, kThreads = 32 * (kScale + kScaleWarps);
};
constexpr int kRegsAtLaunch = 128, kRegsLight = 56, kRegsEpi = 176, kRegsScale = 96;
static_assert(128 * kRegsLight + 32 * kEpiWarps * kRegsEpi + 32 * kScaleWarps * kRegsScale <= Roles<true>::kThreads * kRegsAtLaunch, "register pool of the CTA");
static_assert(Roles<true>::kThreads * kRegsAtLaunch <= 65536, "registers of an SM");
// A stage is 128 values of K of this CTA's rows of A (of which only as many as there are: the MMA reads 128 whatever lies behind
// them, and the results of rows that are not there are not stored) and its half of B's: 32 KB at the most, and as many stages as fit.
constexpr uint32_t kRingBytes = 6 * 32 * 1024;
constexpr int kMostStages = 16;
constexpr uint32_t kAccStride = 192;                 // the second accumulator's first column
constexpr uint32_t kScaleCol0 = 448;                 // ring of kGroups entries of 4 (A) + 8 (B) columns
constexpr int kGroups = 5;
constexpr uint32_t kGroupCols = 12;
constexpr int kGroupBlocks = 4;                      // blocks of K per entry: the bytes of a word
constexpr int kPassBlocks = 16;                      // fp32 results: 2048 terms
constexpr double kPassUs = 0.8;                      // what a pass more costs: the MMAs wait until the overlap has been read
constexpr uint32_t kStagingOff = kRingBytes;             // (the last stage's MMA may read into it)
constexpr uint32_t kWordsOff = kStagingOff + kEpiWarps * 32 * 128;
constexpr uint32_t kWordsBytes = 12 * 32 * 4;        // an entry's scale words, passed between the scale warps
constexpr uint32_t kBarsOff = kWordsOff + kWordsBytes;
constexpr uint32_t kSmem = kBarsOff + 512 + 1024;

struct Scales {               // byte of row i and block kb: p[(i >> shift) * row + kb * block]
  const uint8_t* p;
  long long row, block;
  int shift, rows;            // rows: how many i there are
  bool words;                 // four blocks of a row are an aligned 32-bit word
};

struct ProductArgs {
  int M, N, kblocks;
  int m_tiles;
  TileWalk walk;
  bool a_mn, b_mn;
  int split, split_blocks;    // pairs of a cluster that share a tile's contraction, and how many of its blocks each takes (1: all)
  int pass_blocks;            // blocks of K summed in tensor memory, a multiple of kGroupBlocks
  int stages;
  uint32_t a_bytes, b_off, stage_bytes;      // of A in a stage, where B starts, stride
  uint32_t idesc;             // without N and the scale bytes
  Scales sa, sb;
  void* out;
  bool bf16;
  int* status;
};

// The four bytes of a row on their way: together in [0] where they are an aligned word, else one in each.  Nothing touches them
// before they are needed -- putting them together at once would wait for each load.
struct Bytes { uint32_t v[kGroupBlocks]; };

__device__ __forceinline__ const uint8_t* scale_row(const Scales& s, int i) {
  return i < s.rows ? s.p + static_cast<long long>(i >> s.shift) * s.row : nullptr;     // null: a row that is not there
}
__device__ __forceinline__ void scale_fetch(Bytes& w, const Scales& s, const uint8_t* row, int kb, int kblocks) {
  if (row == nullptr) {
#pragma unroll
    for (int b = 0; b < kGroupBlocks; ++b) w.v[b] = 0u;          // its codes are zero, any scale that is not 255 will do
    return;
  }
  const uint8_t* p = row + kb * s.block;
  if (s.words) {
    w.v[0] = ld_stream(reinterpret_cast<const uint32_t*>(p));
    return;
  }
#pragma unroll
  for (int b = 0; b < kGroupBlocks; ++b, p += s.block) w.v[b] = kb + b < kblocks ? ld_stream(p) : 0u;
}
__device__ __forceinline__ uint32_t scale_word(const Bytes& w, const Scales& s) {
  return s.words ? w.v[0] : w.v[0] | w.v[1] << 8 | w.v[2] << 16 | w.v[3] << 24;
}

constexpr int kPartPitch = 256 + 4;           // of a part's rows in fp32: 128 of them fit into the ring
__device__ __forceinline__ float* part_of(uint8_t* gen) { return reinterpret_cast<float*>(gen); }

// kSums: fp32 results of contractions longer than a pass, summed up in registers.
template <bool kSums>
__global__ void __launch_bounds__(Roles<kSums>::kThreads, 1)
block_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const ProductArgs p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const int n_stages = p.stages;
  const uint32_t stage_bytes = p.stage_bytes;
  const uint32_t bars = base + kBarsOff;
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (n_stages + s); };
  auto sf_full_bar = [&](int g) { return bars + 8u * (2 * n_stages + g); };
  auto sf_empty_bar = [&](int g) { return bars + 8u * (2 * n_stages + kGroups + g); };
  const uint32_t acc_full_bar = bars + 8u * (2 * n_stages + 2 * kGroups), acc_empty_bar = acc_full_bar + 8u;
  const uint32_t slot = acc_empty_bar + 8u;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // rank: in the pair.  With split > 1 a cluster is that many pairs, and they have one tile.
  const uint32_t cluster_rank = cluster_ctarank(), rank = cluster_rank & 1u, first_rank = cluster_rank & ~1u;
  const bool leader = rank == 0;
  const uint16_t both = static_cast<uint16_t>(3u << first_rank);

  if (threadIdx.x == 0) {
    prefetch_tensor_map(&map_a);
    prefetch_tensor_map(&map_b);
    for (int s = 0; s < n_stages; ++s) {
      mbar_init(full_bar(s), 1);                       // the leader's expect_tx; the bytes of both CTAs
      mbar_init(empty_bar(s), 1);                      // one commit to both CTAs
    }
    for (int g = 0; g < kGroups; ++g) {
      mbar_init(sf_full_bar(g), 2 * kScaleWarps);      // the scale warps of both CTAs
      mbar_init(sf_empty_bar(g), 1);
    }
    mbar_init(acc_full_bar, 1);
    mbar_init(acc_empty_bar, 2 * kEpiWarps);
    mbar_fence_init();
  }
  if (warp == 1) {
    tmem_alloc_pair(slot, kTmemCols);
    tmem_relinquish_pair();
  }
  pdl_trigger();
  tc_fence_before_sync();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  tc_fence_after_sync();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(gen + (slot - base));
  pdl_wait();

  const int pairs = gridDim.x / (2 * p.split), pair = blockIdx.x / (2 * p.split);      // that have tiles of their own
  const int kb_begin = static_cast<int>(cluster_rank >> 1) * p.split_blocks, kb_end = min(p.kblocks, kb_begin + p.split_blocks);
  const int items = p.walk.items;
  bool aborted = false;
  struct Piece { int row0, n0, width; };           // of this CTA: rows, columns; no columns: a piece behind the right edge, of which there is nothing
  auto piece = [&](int item) {
    int first, width;
    const int tile = walk_tile(p.walk, item, &first, &width), n_idx = tile / p.m_tiles, n0 = n_idx * p.walk.block_n + first;
    return Piece{(tile - n_idx * p.m_tiles) * 256 + static_cast<int>(rank) * kBlockM, n0, n0 < p.N ? min(width, p.N - n0) : 0};
  };
  const int gran = p.b_mn ? 32 : 16;               // columns of the instruction: what half of them may be
  auto inst_n = [&](const Piece& t) { return (t.width + gran - 1) / gran * gran; };

  if (warp < Roles<kSums>::kEpi) {
  if constexpr (kSums) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsLight));
  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    int stage = 0;
    uint32_t phase = 0;
    const uint32_t bytes = p.a_bytes + (p.b_mn ? kMnChunkBytes : static_cast<uint32_t>(p.walk.block_n >> 1) * kBlockKBytes);
    for (int item = pair; item < items && !aborted; item += pairs) {
      const Piece t = piece(item);
      if (t.width == 0) continue;
      const int row0 = t.row0, bn0 = t.n0 + static_cast<int>(rank) * (inst_n(t) >> 1);
      for (int kb = kb_begin; kb < kb_end; ++kb) {
        if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, p.status)) { aborted = true; break; }
        if (elect_one()) {
          if (leader) mbar_expect_tx(full_bar(stage), 2 * bytes);
          const uint32_t fb = map_to_cta(full_bar(stage), first_rank);
          const uint32_t a_dst = base + static_cast<uint32_t>(stage) * stage_bytes, b_dst = a_dst + p.b_off;
          if (p.a_mn) tma_load_2d_pair(a_dst, &map_a, fb, row0, kb * kBlockKBytes);
          else        tma_load_2d_pair(a_dst, &map_a, fb, kb * kBlockKBytes, row0);
          if (p.b_mn) tma_load_2d_pair(b_dst, &map_b, fb, bn0, kb * kBlockKBytes);
          else        tma_load_2d_pair(b_dst, &map_b, fb, kb * kBlockKBytes, bn0);
        }
        __syncwarp();
        if (++stage == n_stages) { stage = 0; phase ^= 1u; }
      }
    }
    for (int i = 0; i < n_stages && !aborted; ++i) {   // the MMAs have let go of every stage before this CTA may leave
      if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, p.status)) aborted = true;
      if (++stage == n_stages) { stage = 0; phase ^= 1u; }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    if (leader) {
      int stage = 0, group = 0, acc = 0;
      uint32_t phase = 0, sf_phase = 0, acc_phase = 0;
      bool first = true;
      const uint64_t a_desc0 = p.a_mn ? make_smem_desc(base, kMnChunkBytes, 1024) : make_smem_desc(base, 16, 1024);
      const uint64_t b_desc0 = p.b_mn ? make_smem_desc(base + p.b_off, kMnChunkBytes, 1024) : make_smem_desc(base + p.b_off, 16, 1024);
      const uint32_t a_step = (p.a_mn ? kUmmaK * 128 : kUmmaK) >> 4, b_step = (p.b_mn ? kUmmaK * 128 : kUmmaK) >> 4;
      for (int item = pair; item < items && !aborted; item += pairs) {
        const Piece t = piece(item);
        if (t.width == 0) continue;
        const uint32_t idesc_n = p.idesc | (static_cast<uint32_t>(inst_n(t) >> 3) << 17);
        for (int pass = kb_begin; pass < kb_end && !aborted; pass += p.pass_blocks) {
          if (!first) {   // the pass or tile before: its part of the overlap is in registers, everything older is stored
            if (!mbar_wait_warp(acc_empty_bar, acc_phase, p.status)) { aborted = true; break; }
            acc_phase ^= 1u;
            tc_fence_after_sync();
          }
          first = false;
          const uint32_t d = tmem + static_cast<uint32_t>(acc) * kAccStride;
          const int end = min(kb_end, pass + p.pass_blocks);
          for (int kb = pass; kb < end; ++kb) {
            const int byte = kb % kGroupBlocks;
            if (byte == 0 && !mbar_wait_warp(sf_full_bar(group), sf_phase, p.status)) { aborted = true; break; }
            if (!mbar_wait_warp(full_bar(stage), phase, p.status)) { aborted = true; break; }
            tc_fence_after_sync();
            const uint32_t off = (static_cast<uint32_t>(stage) * stage_bytes) >> 4;
            const uint32_t sfa = tmem + kScaleCol0 + static_cast<uint32_t>(group) * kGroupCols;
            const uint32_t idesc = idesc_n | (static_cast<uint32_t>(byte) << 29) | (static_cast<uint32_t>(byte) << 4);
            const bool last = byte == kGroupBlocks - 1 || kb == end - 1;
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < kBlockKBytes / kUmmaK; ++k)
                umma_mx8_pair(d, a_desc0 + off + k * a_step, b_desc0 + off + k * b_step, idesc, sfa, sfa + 4, (kb > pass || k > 0) ? 1u : 0u);
              umma_commit_pair(empty_bar(stage), both);
              if (last) umma_commit_pair(sf_empty_bar(group), both);
            }
            __syncwarp();
            if (++stage == n_stages) { stage = 0; phase ^= 1u; }
            if (last && ++group == kGroups) { group = 0; sf_phase ^= 1u; }
          }
          if (aborted) break;
          if (elect_one()) umma_commit_pair(acc_full_bar, both);
          __syncwarp();
          acc ^= 1;
        }
      }
    }
  }   // (warps 2 and 3 of kSums have no work)
  } else if (warp >= Roles<kSums>::kScale) {
    // ------------------------------------------------------------ scales
    if constexpr (kSums) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsScale));
    const int q = warp & 3;                                   // this warp's quadrant of tensor memory
    const uint32_t lane_base = static_cast<uint32_t>(q * 32) << 16;
    uint32_t* words = reinterpret_cast<uint32_t*>(gen + kWordsOff);
    // Each warp fetches a quarter of an entry's words (rows 32 q .. of A, two columns of B), all four write all of them.  kAhead
    // entries' words are on their way, in registers that no copy touches before they are needed (a queue that moved them waited for
    // each load: 4096 x 16384 x 4096 333 us).
    constexpr int kAhead = 3;
    struct Entry { Bytes a, b0, b1; };
    int next_item = pair, next_kb = kb_begin;
    const uint8_t *row_a = nullptr, *row_b0 = nullptr, *row_b1 = nullptr;
    auto fetch = [&](Entry& w) {
      if (next_item >= items) return;
      if (next_kb == kb_begin) {
        const Piece t = piece(next_item);
        row_a = scale_row(p.sa, t.row0 + 32 * q + lane);
        row_b0 = scale_row(p.sb, t.n0 + 32 * q + lane);
        row_b1 = t.width > 128 ? scale_row(p.sb, t.n0 + 128 + 32 * q + lane) : nullptr;
      }
      scale_fetch(w.a, p.sa, row_a, next_kb, p.kblocks);
      scale_fetch(w.b0, p.sb, row_b0, next_kb, p.kblocks);
      scale_fetch(w.b1, p.sb, row_b1, next_kb, p.kblocks);
      next_kb += kGroupBlocks;
      if (next_kb >= kb_end) {
        next_kb = kb_begin;
        do next_item += pairs; while (next_item < items && piece(next_item).width == 0);
      }
    };
    int group = 0;
    uint32_t phase = 0;
    while (next_item < items && piece(next_item).width == 0) next_item += pairs;
    int steps = 0;
    for (int item = pair; item < items; item += pairs) steps += piece(item).width != 0;
    steps *= (kb_end - kb_begin + kGroupBlocks - 1) / kGroupBlocks;
    Entry ahead[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) fetch(ahead[j]);
    for (int step0 = 0; step0 < steps && !aborted; step0 += kAhead) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (step0 + j >= steps || aborted) break;
        words[q * 32 + lane] = scale_word(ahead[j].a, p.sa);
        words[(4 + q) * 32 + lane] = scale_word(ahead[j].b0, p.sb);
        words[(8 + q) * 32 + lane] = scale_word(ahead[j].b1, p.sb);
        fetch(ahead[j]);
        asm volatile("bar.sync 1, %0;" ::"n"(kScaleWarps * 32) : "memory");
        uint32_t va[4], vb[8];
#pragma unroll
        for (int c = 0; c < 4; ++c) va[c] = words[c * 32 + lane];
#pragma unroll
        for (int c = 0; c < 8; ++c) vb[c] = words[(4 + c) * 32 + lane];
        aborted = !mbar_wait_warp(sf_empty_bar(group), phase ^ 1u, p.status);
        if (!aborted) {
          tc_fence_after_sync();
          const uint32_t t = tmem + lane_base + kScaleCol0 + static_cast<uint32_t>(group) * kGroupCols;
          tmem_st_32x32b_x4(t, va);
          tmem_st_32x32b_x8(t + 4, vb);
          tmem_st_wait();
          tc_fence_before_sync();
          __syncwarp();
          // (a release at cluster scope would wait for the loads ahead, too: 281 us instead of 253)
          if (lane == 0) mbar_arrive_remote(map_to_cta(sf_full_bar(group), first_rank));
        }
        // the words have been read; and all four warps leave together, or the barriers would be waited for in vain
        uint32_t any;
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                     : "=r"(any) : "r"(static_cast<uint32_t>(aborted)), "n"(kScaleWarps * 32) : "memory");
        aborted = any != 0;
        if (aborted) break;
        if (++group == kGroups) { group = 0; phase ^= 1u; }
      }
    }
    // the MMAs have let go of every entry before this CTA may leave
    for (int i = 0; i < kGroups && !aborted; ++i) {
      if (!mbar_wait_warp(sf_empty_bar(group), phase ^ 1u, p.status)) aborted = true;
      if (++group == kGroups) { group = 0; phase ^= 1u; }
    }
  } else {
    // ------------------------------------------------------------ epilogue
    if constexpr (kSums) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsEpi));
    const int quad = warp & 3, half = (warp - Roles<kSums>::kEpi) >> 2;
    uint8_t* stage_out = gen + kStagingOff + (warp - Roles<kSums>::kEpi) * 32 * 128;
    uint8_t* my = stage_out + lane * 128;
    const int sw = lane & 7;
    const uint32_t lane_base = static_cast<uint32_t>(quad * 32) << 16;
    int acc = 0;
    uint32_t full_phase = 0;
    for (int item = pair; item < items && !aborted; item += pairs) {
      const Piece of = piece(item);
      if (of.width == 0) continue;
      const int chunks = (of.width + 63) / 64, low = (chunks + 1) / 2;        // chunks of 64 columns: half 0 takes [0, low) upwards,
      const int count = half == 0 ? low : chunks - low;                       // half 1 [low, chunks) downwards: the overlap first
      auto column = [&](int i) { return 64 * (half == 0 ? i : chunks - 1 - i); };
      const int row0 = of.row0 + quad * 32, n0 = of.n0, end = of.width;
      auto let_go = [&]() {     // what overlaps the other accumulator has been read (the rest will be before this one's next turn)
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(map_to_cta(acc_empty_bar, first_rank));
      };
      // 128 bytes of a row through shared memory: four rows, or eight pieces of 16 bytes, to an instruction; N is a multiple of 16,
      // so a piece lies inside or outside as a whole
      auto flush = [&](int col, int per_piece, int esize) {
        __syncwarp();
        const int piece = lane & 7;
        const bool in = col + piece * per_piece < end;
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += 4) {
          const int r = r0 + (lane >> 3);
          const uint4 val = *reinterpret_cast<const uint4*>(stage_out + r * 128 + ((piece ^ (r & 7)) << 4));
          if (in && row0 + r < p.M)
            *reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.out) + (static_cast<long long>(row0 + r) * p.N + n0 + col + piece * per_piece) * esize) = val;
        }
        __syncwarp();
      };
      auto store32 = [&](int col, const uint32_t* v) {       // 32 columns of fp32
#pragma unroll
        for (int j = 0; j < 8; ++j) *reinterpret_cast<uint4*>(my + ((j ^ sw) << 4)) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        flush(col, 4, 4);
      };
      auto share32 = [&](int col, const uint32_t* v) {       // to be added up: this CTA's rows of the tile as fp32, where the stages were
        if (row0 + lane >= p.M) return;                      // (every copy has been multiplied)
        uint4* row = reinterpret_cast<uint4*>(part_of(gen) + (row0 + lane - of.row0) * kPartPitch + col);
#pragma unroll
        for (int j = 0; j < 8; ++j) row[j] = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
      };
      if constexpr (kSums) {
        uint32_t sum[2][64];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 64; ++j) sum[i][j] = 0u;
        for (int pass = kb_begin; pass < kb_end; pass += p.pass_blocks) {
          if (!mbar_wait_warp(acc_full_bar, full_phase, p.status)) { aborted = true; break; }
          full_phase ^= 1u;
          tc_fence_after_sync();
          const uint32_t t = tmem + lane_base + static_cast<uint32_t>(acc) * kAccStride;
          if (count == 0) let_go();
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (i < count) {
#pragma unroll
              for (int h = 0; h < 64; h += 32) {
                uint32_t v[32];
                __syncwarp();
                tmem_ld_32x32b_x32(t + column(i) + h, v);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) sum[i][h + j] = __float_as_uint(__uint_as_float(sum[i][h + j]) + __uint_as_float(v[j]));
              }
              if (i == 0) let_go();
            }
          }
          acc ^= 1;
        }
        if (aborted) break;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (i < count) {
#pragma unroll
            for (int h = 0; h < 64; h += 32) {
              if (p.split > 1) share32(column(i) + h, sum[i] + h);
              else store32(column(i) + h, sum[i] + h);
            }
          }
        }
      } else {
        if (!mbar_wait_warp(acc_full_bar, full_phase, p.status)) { aborted = true; break; }
        full_phase ^= 1u;
        tc_fence_after_sync();
        const uint32_t t = tmem + lane_base + static_cast<uint32_t>(acc) * kAccStride;
        if (count == 0) let_go();
        for (int i = 0; i < count; ++i) {
          const int c0 = column(i);
          uint32_t v0[32], v1[32];
          __syncwarp();
          tmem_ld_32x32b_x32(t + c0, v0);
          tmem_ld_32x32b_x32(t + c0 + 32, v1);
          tmem_ld_wait();
          if (i == 0) let_go();
          if (p.split > 1) {
            share32(c0, v0);
            share32(c0 + 32, v1);
          } else if (p.bf16) {
            auto put = [&](const uint32_t (&v)[32], int first_piece) {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                uint4 o;
                o.x = pack_bf16x2(__uint_as_float(v[8 * j]), __uint_as_float(v[8 * j + 1]));
                o.y = pack_bf16x2(__uint_as_float(v[8 * j + 2]), __uint_as_float(v[8 * j + 3]));
                o.z = pack_bf16x2(__uint_as_float(v[8 * j + 4]), __uint_as_float(v[8 * j + 5]));
                o.w = pack_bf16x2(__uint_as_float(v[8 * j + 6]), __uint_as_float(v[8 * j + 7]));
                *reinterpret_cast<uint4*>(my + (((first_piece + j) ^ sw) << 4)) = o;
              }
            };
            put(v0, 0);
            put(v1, 4);
            flush(c0, 8, 2);
          } else {
            store32(c0, v0);
            store32(c0 + 32, v1);
          }
        }
        acc ^= 1;
      }
    }
  }

  if (p.split > 1) {
    // ------------------------------------------------------------ the pairs' parts of the tile, added up in order, a strip of columns a pair
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    const Piece t = piece(pair);
    const int rows = max(0, min(kBlockM, p.M - t.row0)), strip = t.width > 0 ? (t.width / 4 + p.split - 1) / p.split : 0;   // in groups of four columns
    const int first = static_cast<int>(cluster_rank >> 1) * strip, count = max(0, min(strip, t.width / 4 - first));
    // (kSums: by the epilogue's threads, which have the registers)
    constexpr int kFirst = kSums ? 32 * Roles<kSums>::kEpi : 0, kAdders = kSums ? 32 * kEpiWarps : Roles<kSums>::kThreads;
    for (int u = static_cast<int>(threadIdx.x) - kFirst; u >= 0 && threadIdx.x < kFirst + kAdders && u < rows * count; u += kAdders) {
      const int r = u / count, c = 4 * (first + u - r * count);
      const uint32_t at = smem_u32(part_of(gen) + r * kPartPitch + c);
      float4 v = ld_shared_cluster_f32x4(map_to_cta(at, rank));
      for (int s = 1; s < p.split; ++s) {
        const float4 w = ld_shared_cluster_f32x4(map_to_cta(at, rank + 2 * s));
        v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
      }
      const long long o = static_cast<long long>(t.row0 + r) * p.N + t.n0 + c;
      if (p.bf16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + o) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
      else *reinterpret_cast<float4*>(static_cast<float*>(p.out) + o) = v;
    }
  }

  // ------------------------------------------------------------ common exit
  if (aborted) {
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < 200000ull) { }
  }
  tc_fence_before_sync();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem, kTmemCols);
  }
}

struct Operand {
  const uint8_t* codes;
  int64_t rows, cols;     // as the codes lie
  bool mn;                // contracted along its rows
  int fmt;
  Scales s;
};

// How many clusters of four or eight CTAs, one CTA to an SM, the current device holds at once: a matter of its groups of SMs, which are not
// all whole.  Asked once per device; 0 where it cannot be told (no tile is split then).
int resident_clusters(int size) {
  static std::atomic<int> known[2][kMaxDevices];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0;
  std::atomic<int>& at = known[size == 8][dev];
  if ((n = at.load(std::memory_order_acquire)) != 0) return n < 0 ? 0 : n;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(sm_count() / size * size));
  cfg.blockDim = dim3(Roles<false>::kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(size);
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, block_product_kernel<false>, &cfg) != cudaSuccess || n < 1) n = -1;
  at.store(n, std::memory_order_release);
  return n < 0 ? 0 : n;
}

// How a product is run, and how long that should take.
struct Way {
  TileWalk walk;
  int split, split_blocks, pass_blocks;
  double us;
};
// The tiles' width: what takes the least time (4096 x 16384 x 4096: five waves of 192 columns 280 us, four of 256 243); or so few tiles that two
// or four pairs can share each one's contraction (a cluster's parts are added up through its shared memory).  Measured: a block of K
// takes 0.16 us and 0.9 ns a column, or its copies' time at 80 GB/s to an SM (128 columns of an MN-major B whatever the width); adding up
// 1.5 to 3.5 us with the rows (weight gradient of 16384 rows, 256 x 1024: 50 us unsplit, 19.6; 8 rows 11008 -> 4096 30.6 and 20.5, 4096 ->
// 4096 15.1 and 12.3; 512 rows 4096 -> 4096 15.8 and 17.1, which stays unsplit).
Way pick_way(int64_t M, int64_t N, int64_t kblocks, int64_t a_rows, bool b_mn, bool f32) {
  const int64_t pairs = sm_count() / 2, m_tiles = (M + 255) / 256;
  Way best{};
  for (int w = 256; w >= 64; w -= 32) {
    const int64_t tiles = m_tiles * ((N + w - 1) / w);
    const double copies = static_cast<double>((std::min<int64_t>(M, a_rows) + (b_mn ? 128 : w / 2)) * kBlockKBytes) / 80e3;
    auto block_us = [&](int width) { return std::max(0.16 + 0.0009 * width, copies); };
    for (int s = 1; s <= 4; s *= 2) {
      const int64_t per = s == 1 ? kblocks : round_up((kblocks + s - 1) / s, kGroupBlocks);
      if (s > 1 && (tiles > resident_clusters(2 * s) || per * (s - 1) >= kblocks)) continue;
      int64_t cost;
      const TileWalk walk = plan_walk(tiles, s == 1 ? pairs : tiles, w, 178, &cost);
      const double waves = s == 1 ? static_cast<double>(tiles / pairs) : 1.0;
      double us = static_cast<double>(per) * (waves * block_us(w) + (walk.items > walk.full ? block_us(walk.part_n) : 0.0));
      const int pass = static_cast<int>(f32 ? std::min<int64_t>(per, kPassBlocks) : per);
      us += kPassUs * (waves + (walk.items > walk.full ? 1.0 : 0.0)) * static_cast<double>((per - 1) / pass);
      if (s > 1) us += 1.5 + 2.0 * static_cast<double>(M < 256 ? M : 256) / 256.0;
      if (best.us == 0.0 || us < best.us) best = Way{walk, s, static_cast<int>(per), pass, us};
    }
  }
  return best;
}
int64_t rows_of_a(const Operand& a, int64_t M) { return a.mn || M >= 128 ? 128 : round_up(M, 8); }

cudaError_t launch_product(Operand a, const Operand& b, int64_t M, int64_t N, int64_t K, void* out, int out_dt, cudaStream_t st) {
  static DeviceMask configured{0}, configured_sums{0};
  cudaError_t e = set_max_dynamic_smem(block_product_kernel<false>, static_cast<int>(kSmem), configured);
  if (e == cudaSuccess) e = set_max_dynamic_smem(block_product_kernel<true>, static_cast<int>(kSmem), configured_sums);
  if (e != cudaSuccess) return e;
  const int64_t kblocks = (K + kBlockKBytes - 1) / kBlockKBytes;
  const bool f32 = out_dt == FALQON_F32;
  Way way = pick_way(M, N, kblocks, rows_of_a(a, M), b.mn, f32);
  // Rows that do not fill a tile of 256 may cost a wave of their own: they go into a second launch where that is less by what a launch costs
  // more than its blocks (8.5 us measured) and a little.  Both sides, one launch and two: 777 rows forward 13824 -> 5120 79.9 and 73.7 us, input
  // gradient of 5120 -> 13824 82 and 82 to 84; 1030 rows, input gradient of 4096 -> 11008 71.7 and 65.5 to 67.6, of 4096 -> 4096 37 and 39 (stays one).
  const int64_t whole = M / 256 * 256;
  if (!a.mn && whole > 0 && whole < M) {
    const Way first = pick_way(whole, N, kblocks, 128, b.mn, f32), rest = pick_way(M - whole, N, kblocks, rows_of_a(a, M - whole), b.mn, f32);
    if (first.us + rest.us + 8.5 < 0.98 * way.us) {
      Operand tail = a;
      tail.codes += whole * a.cols, tail.rows = M - whole;
      tail.s.p += whole * a.s.row, tail.s.rows = static_cast<int>(M - whole);
      e = launch_product(tail, b, M - whole, N, K, static_cast<uint8_t*>(out) + whole * N * (out_dt == FALQON_BF16 ? 2 : 4), out_dt, st);
      if (e != cudaSuccess) return e;
      M = whole, a.rows = whole, a.s.rows = static_cast<int>(whole);
      way = first;
    }
  }
  ProductArgs g{};
  g.M = static_cast<int>(M);
  g.N = static_cast<int>(N);
  g.kblocks = static_cast<int>(kblocks);
  g.m_tiles = static_cast<int>((M + 255) / 256);
  g.walk = way.walk, g.split = way.split, g.split_blocks = way.split_blocks, g.pass_blocks = way.pass_blocks;
  const int64_t pairs_all = sm_count() / 2, a_rows = rows_of_a(a, M);
  g.a_bytes = static_cast<uint32_t>(a_rows) * kBlockKBytes;
  g.b_off = static_cast<uint32_t>(round_up(g.a_bytes, 1024));
  g.stage_bytes = g.b_off + (b.mn ? kMnChunkBytes : static_cast<uint32_t>(g.walk.block_n / 2) * kBlockKBytes);
  g.stages = static_cast<int>(kRingBytes / g.stage_bytes);
  if (g.stages > kMostStages) g.stages = kMostStages;
  g.a_mn = a.mn;
  g.b_mn = b.mn;
  // instruction descriptor of the block-scaled kinds: formats at 7 and 10, majors at 15 and 16, N / 8 at 17, E8M0 scales at 23,
  // M / 16 at 24; the scale bytes of B at 4 and of A at 29
  g.idesc = (static_cast<uint32_t>(a.fmt) << 7) | (static_cast<uint32_t>(b.fmt) << 10) | ((a.mn ? 1u : 0u) << 15) | ((b.mn ? 1u : 0u) << 16) |
            (1u << 23) | (static_cast<uint32_t>(256 >> 4) << 24);
  g.sa = a.s;
  g.sb = b.s;
  g.out = out;
  g.bf16 = out_dt == FALQON_BF16;
  g.status = device_status_ptr();
  if (g.status == nullptr) return cudaErrorInvalidValue;
  CUtensorMap ma, mb;
  if (!make_tensor_map(&ma, a.codes, a.rows, a.cols, a.cols, 128, static_cast<uint32_t>(a_rows))) return cudaErrorInvalidValue;
  if (!make_tensor_map(&mb, b.codes, b.rows, b.cols, b.cols, 128, b.mn ? 128 : static_cast<uint32_t>(g.walk.block_n / 2))) return cudaErrorInvalidValue;
  const int64_t pairs = (g.walk.items < pairs_all ? g.walk.items : pairs_all) * g.split;
  const dim3 grid(static_cast<unsigned>(2 * pairs));
  return g.pass_blocks < g.split_blocks ? launch_pdl(block_product_kernel<true>, grid, dim3(Roles<true>::kThreads), kSmem, st, 2 * g.split, ma, mb, g)
                                        : launch_pdl(block_product_kernel<false>, grid, dim3(Roles<false>::kThreads), kSmem, st, 2 * g.split, ma, mb, g);
}

Scales scales_of(const uint8_t* p, int along, int64_t rows, int64_t cols, bool over_rows) {
  // over_rows: the blocks of the contraction run down the rows and i counts columns; else they run along a row and i counts rows
  const int64_t nb = (cols + 127) / 128;
  Scales s{};
  s.p = p;
  s.rows = static_cast<int>(over_rows ? cols : rows);
  if (along == FALQON_ALONG_ROW) s.row = nb, s.block = 1;
  else if (along == FALQON_ALONG_COL) s.row = 1, s.block = cols;
  else s.row = over_rows ? 1 : nb, s.block = over_rows ? nb : 1, s.shift = 7;
  s.words = s.block == 1 && s.row % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & 3) == 0;
  return s;
}

bool ok16(const void* p) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool fmt_ok(int f) { return f == FALQON_E4M3 || f == FALQON_E5M2; }
// n and m multiples of 16; no dimension so long that a count of tiles or a coordinate leaves 31 bits
bool layer_ok(int64_t T, int64_t n, int64_t m) {
  constexpr int64_t kMost = int64_t{1} << 30;
  return T >= 1 && n >= 16 && m >= 16 && n % 16 == 0 && m % 16 == 0 && T <= kMost && n <= kMost && m <= kMost;
}
bool tiles_ok(int64_t M, int64_t N) { return ((M + 255) / 256) <= (int64_t{1} << 29) / ((N + 63) / 64); }
int finish(cudaError_t e) { return e == cudaSuccess ? FALQON_OK : FALQON_ERR_CUDA; }

}  // namespace
}  // namespace falqon

using namespace falqon;

extern "C" {

int falqon_block_forward(const uint8_t* x_codes, const uint8_t* x_scales, falqon_fp8 x_fmt, const uint8_t* w_codes, const uint8_t* w_scales,
                         falqon_fp8 w_fmt, int64_t T, int64_t n, int64_t m, void* y, int y_dtype, falqon_stream stream) {
  if (!ok16(x_codes) || !ok16(w_codes) || !ok16(y) || x_scales == nullptr || w_scales == nullptr || !fmt_ok(x_fmt) || !fmt_ok(w_fmt) ||
      (y_dtype != FALQON_BF16 && y_dtype != FALQON_F32) || !layer_ok(T, n, m) || !tiles_ok(T, m))
    return FALQON_ERR_INVALID_ARG;
  if (block_linear_takes(T, n, m))
    return finish(launch_block_linear_codes(x_codes, x_scales, x_fmt, w_codes, w_scales, w_fmt, T, n, m, y, y_dtype == FALQON_BF16,
                                            static_cast<cudaStream_t>(stream)));
  const Operand a{x_codes, T, n, false, x_fmt, scales_of(x_scales, FALQON_ALONG_ROW, T, n, false)};
  const Operand b{w_codes, m, n, false, w_fmt, scales_of(w_scales, FALQON_TILE, m, n, false)};
  return finish(launch_product(a, b, T, m, n, y, y_dtype, static_cast<cudaStream_t>(stream)));
}

int falqon_block_input_grad(const uint8_t* dy_codes, const uint8_t* dy_scales, falqon_fp8 dy_fmt, const uint8_t* w_codes,
                            const uint8_t* w_scales, falqon_fp8 w_fmt, int64_t T, int64_t n, int64_t m, void* dx, int dx_dtype,
                            falqon_stream stream) {
  if (!ok16(dy_codes) || !ok16(w_codes) || !ok16(dx) || dy_scales == nullptr || w_scales == nullptr || !fmt_ok(dy_fmt) || !fmt_ok(w_fmt) ||
      (dx_dtype != FALQON_BF16 && dx_dtype != FALQON_F32) || !layer_ok(T, n, m) || !tiles_ok(T, n))
    return FALQON_ERR_INVALID_ARG;
  const Operand a{dy_codes, T, m, false, dy_fmt, scales_of(dy_scales, FALQON_ALONG_ROW, T, m, false)};
  const Operand b{w_codes, m, n, true, w_fmt, scales_of(w_scales, FALQON_TILE, m, n, true)};
  return finish(launch_product(a, b, T, n, m, dx, dx_dtype, static_cast<cudaStream_t>(stream)));
}

int falqon_block_weight_grad(const uint8_t* dy_codes, const uint8_t* dy_scales, falqon_fp8 dy_fmt, const uint8_t* x_codes,
                             const uint8_t* x_scales, falqon_fp8 x_fmt, int64_t T, int64_t n, int64_t m, void* dw, int dw_dtype,
                             falqon_stream stream) {
  if (!ok16(dy_codes) || !ok16(x_codes) || !ok16(dw) || dy_scales == nullptr || x_scales == nullptr || !fmt_ok(dy_fmt) || !fmt_ok(x_fmt) ||
      (dw_dtype != FALQON_BF16 && dw_dtype != FALQON_F32) || !layer_ok(T, n, m) || !tiles_ok(m, n))
    return FALQON_ERR_INVALID_ARG;
  const Operand a{dy_codes, T, m, true, dy_fmt, scales_of(dy_scales, FALQON_ALONG_COL, T, m, true)};
  const Operand b{x_codes, T, n, true, x_fmt, scales_of(x_scales, FALQON_ALONG_COL, T, n, true)};
  return finish(launch_product(a, b, m, n, T, dw, dw_dtype, static_cast<cudaStream_t>(stream)));
}

size_t falqon_block_linear_scratch_bytes(int64_t T, int64_t n, int64_t m) {
  if (!layer_ok(T, n, m) || !tiles_ok(T, m) || block_linear_takes(T, n, m)) return 0;
  return static_cast<size_t>(T * n + round_up(T * ((n + 127) / 128), 16));
}

int falqon_block_linear(const void* x, int x_dtype, const uint8_t* w_codes, const uint8_t* w_scales, falqon_fp8 w_fmt, int64_t T, int64_t n,
                        int64_t m, void* y, int y_dtype, void* scratch, size_t scratch_bytes, falqon_stream stream) {
  if (!ok16(x) || (x_dtype != FALQON_BF16 && x_dtype != FALQON_F32) || !ok16(w_codes) || !ok16(y) || w_scales == nullptr || !fmt_ok(w_fmt) ||
      (y_dtype != FALQON_BF16 && y_dtype != FALQON_F32) || !layer_ok(T, n, m) || !tiles_ok(T, m))
    return FALQON_ERR_INVALID_ARG;
  if (block_linear_takes(T, n, m))
    return finish(launch_block_linear_plain(x, x_dtype == FALQON_BF16, w_codes, w_scales, w_fmt, T, n, m, y, y_dtype == FALQON_BF16,
                                            static_cast<cudaStream_t>(stream)));
  if (!ok16(scratch) || scratch_bytes < falqon_block_linear_scratch_bytes(T, n, m)) return FALQON_ERR_WORKSPACE;
  uint8_t* codes = static_cast<uint8_t*>(scratch);
  uint8_t* scales = codes + T * n;
  const int rc = falqon_block_quantize(x, x_dtype, T, n, n, FALQON_E4M3, FALQON_ALONG_ROW, codes, scales, stream);
  if (rc != FALQON_OK) return rc;
  return falqon_block_forward(codes, scales, FALQON_E4M3, w_codes, w_scales, w_fmt, T, n, m, y, y_dtype, stream);
}

}  // extern "C"
