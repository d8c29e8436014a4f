// Attention, backward: the probabilities are made again from q, k and lse, tile by tile.
//
//   P = 2^(c s - lse2),  c = scale log2(e),  lse2 = lse log2(e);  delta_i = do_i . o_i;  dS = P (do v^T - delta)
//   dq = scale dS k;  dk = scale dS^T q;  dv = P^T do
//
// Two passes of one kernel.  With the queries' tiles staying (Q: q, do stay, k, v stream by) dS is the A operand of the product with
// k; with the keys' staying (KV: k, v stay, q, do stream by) P^T and dS^T are the A operands of those with do and q.  In both a
// thread has a row of s and of do v^T from tensor memory and leaves P and dS there as bf16: neither is ever in shared memory, the sums
// stay in tensor memory over all blocks, and nothing is added up between CTAs by atomics.  Against one pass that makes P and dS
// once, s and do v^T are made twice: seven products instead of five.
// Keys' tiles with many queries are shared by several CTAs, each of which takes a part of the queries; their fp32
// sums are added in a fixed order by a kernel of its own.
#include "attention.cuh"

namespace surgeon {

namespace {

using namespace tc;
using namespace att;

constexpr int kBlock = 64;                       // rows that stream by at a time
constexpr int kThreads = 384;                    // 2 x 4 warps with a thread a row, one that copies, one that issues products, two that idle
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;               // 2 x 208 + 88 = 3 x 168, what 384 threads are launched with
constexpr int kMaxStages = 8;

template <int DP, bool KV> struct Shape {
  static constexpr int kSlabs = DP / kSlabCols;
  static constexpr int kTiles = KV && DP == 128 ? 1 : 2;         // tiles that stay; the two halves of the warps have one each, or every other block of one
  static constexpr int kTileBytes = kTile * DP * 2, kBlockBytes = kBlock * DP * 2;
  static constexpr int kHold = DP == 64 ? 2 : 1;                 // places for what stays
  static constexpr int kStages = DP == 64 ? 5 : KV ? 4 : 3;
  static constexpr int kRowBytes = KV ? kBlock * 8 : 0;          // lse2 and delta of a block
  static constexpr int kStageBytes = 2 * kBlockBytes;
  static constexpr int kHoldBytes = kTiles * 2 * kTileBytes;     // [tile][first, second]
  static constexpr int kSmem = 1024 + kHold * kHoldBytes + kStages * (kStageBytes + kRowBytes);
  static constexpr bool kOwn = !KV && DP == 64;  // dS has columns of its own, else P and dS take the places of s and do v^T
  // columns of tensor memory
  static constexpr uint32_t kStep = KV && DP == 128 ? 128 : 256; // from one half's to the other's
  static constexpr uint32_t kS = 0, kD = 64, kDs = kOwn ? 128 : KV ? 64 : 0, kAcc1 = KV ? (DP == 64 ? 128 : 256) : (DP == 64 ? 192 : 128),
                            kAcc2 = DP == 64 ? 192 : 384, kAccStep = KV && DP == 128 ? 0 : 256;
};

struct Args {
  int batch, heads, kv_heads, group, q_len, kv_len, head_dim, causal;
  int tiles, items, splits, q_pad;
  float scale;
  const int* q_lengths;
  const int* kv_lengths;
  const float2* rows;                            // lse2 and delta, [batch][heads][q_pad]
  surgeon_heads out1, out2;                      // dq; or dk and dv
  float* partial;                                // [split][2][batch][kv_heads][kv_len][head_dim], where there are several
};

template <int DP, bool KV>
struct Item {
  using S = Shape<DP, KV>;
  int b, h, row0, q_valid, kv_valid, off;        // h: of the tiles that stay
  int first, blocks, from, steps;                // blocks of the rows that stream by: first, ..., first + blocks - 1 of each head; steps from, ... are this item's
  int split, valid;                              // valid: rows of the tiles
  bool active[2];
  __device__ __forceinline__ Item(const Args& p, int item) {
    const int heads = KV ? p.kv_heads : p.heads, pairs = p.batch * heads;
    split = 0;
    if (KV && p.splits > 1) {
      split = item % p.splits;
      item /= p.splits;
    }
    int bh, tile;
    if (p.causal) {                              // the longest first
      tile = KV ? item / pairs : p.tiles - 1 - item / pairs;
      bh = item % pairs;
    } else {
      bh = item / p.tiles;
      tile = item % p.tiles;
    }
    b = bh / heads;
    h = bh % heads;
    row0 = tile * S::kTiles * kTile;
    q_valid = length_of(p.q_lengths, b, p.q_len);
    kv_valid = length_of(p.kv_lengths, b, p.kv_len);
    off = kv_valid - q_valid;
    valid = KV ? kv_valid : q_valid;
    first = 0;
    if (KV) {
      int start = p.causal ? max(0, row0 - off) : 0;
      if (row0 >= kv_valid) start = q_valid;
      first = min(start, q_valid) / kBlock;
      blocks = start >= q_valid ? 0 : (q_valid + kBlock - 1) / kBlock - first;
      const int total = blocks * p.group;
      from = static_cast<int>(static_cast<long long>(total) * split / p.splits);
      steps = static_cast<int>(static_cast<long long>(total) * (split + 1) / p.splits) - from;
    } else {
      const int last = min(row0 + S::kTiles * kTile, q_valid) - 1;
      const int keys = row0 >= q_valid ? 0 : p.causal ? max(0, min(kv_valid, last + off + 1)) : kv_valid;
      blocks = (keys + kBlock - 1) / kBlock;
      from = 0;
      steps = blocks;
    }
    active[0] = steps > 0;
    active[1] = steps > 0 && (S::kTiles == 1 || row0 + kTile < valid);
  }
  // Head and first row of the n-th step's block, and how many rows of it count.
  __device__ __forceinline__ void block(const Args& p, int n, int* head, int* row, int* left) const {
    if (KV) {
      const int at = from + n, g = at / blocks;
      *head = h * p.group + g;
      *row = (first + at - g * blocks) * kBlock;
      *left = q_valid - *row;
    } else {
      *head = h / p.group;
      *row = n * kBlock;
      *left = kv_valid - *row;
    }
    if (*left > kBlock) *left = kBlock;
  }
};

template <int DP, bool KV>
__global__ void __launch_bounds__(kThreads, 1)
attention_grad_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap y_map, const __grid_constant__ CUtensorMap u_map,
                      const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap o1_map, const __grid_constant__ CUtensorMap o2_map,
                      const __grid_constant__ Args p) {
  using S = Shape<DP, KV>;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  unsigned char* ring = smem + S::kHold * S::kHoldBytes;
  unsigned char* row_ring = ring + S::kStages * S::kStageBytes;
  __shared__ __align__(8) unsigned long long bars[2 * kMaxStages + 4 + 8 + 3];
  __shared__ uint32_t tmem_slot;

  const int warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x) >> 5, 0);
  const bool leader = elected();
  const uint32_t full = smem_u32(bars), empty = full + 8 * kMaxStages;
  const uint32_t hold_full = empty + 8 * kMaxStages, hold_empty = hold_full + 16;
  const uint32_t s_full = hold_empty + 16, s_free = s_full + 16, p_full = s_free + 16, acc_done = p_full + 16;     // of each half
  const uint32_t item_done = acc_done + 16, acc_free = item_done + 8, fixed = acc_free + 8;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, KV ? 1 + 4 * S::kTiles : 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(hold_full + 8 * i, 1);
      mbar_init(hold_empty + 8 * i, 8);
      mbar_init(s_full + 8 * i, 1);
      mbar_init(s_free + 8 * i, 4);
      mbar_init(p_full + 8 * i, 4);
      mbar_init(acc_done + 8 * i, 1);
    }
    mbar_init(item_done, 1);
    mbar_init(acc_free, 8);
    mbar_init(fixed, 1);
    fence_barrier_init();
  }
  if (warp == 9) tmem_alloc(smem_u32(&tmem_slot), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_trigger();
  pdl_wait();

  if (warp >= 8) {
    set_registers<false, kOtherRegs>();
    if (warp == 8) {
      // ---- copies ----
      int s = 0, it = 0;
      uint32_t phase = 1, fix_phase = 0;         // (a fresh barrier counts as passed in its phase before)
      bool ok = true;
      for (int item = blockIdx.x; item < p.items && ok; item += gridDim.x, ++it) {
        const Item<DP, KV> w(p, item);
        const int hs = S::kHold == 2 ? it & 1 : 0;
        ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(hold_empty + 8 * hs, (S::kHold == 2 ? (it >> 1) & 1 : it & 1) ^ 1));
        if (!ok) break;
        if (leader) {
          if (w.steps) {
            const int tiles = S::kTiles == 2 && !w.active[1] ? 1 : S::kTiles;
            mbar_arrive_expect_tx(hold_full + 8 * hs, tiles * 2 * S::kTileBytes);
            for (int t = 0; t < tiles; ++t)
              for (int c = 0; c < S::kSlabs; ++c) {
                const uint32_t to = smem_u32(smem) + hs * S::kHoldBytes + t * 2 * S::kTileBytes + c * kTile * 128;
                tma_load_4d(to, &x_map, c * kSlabCols, w.row0 + t * kTile, w.h, w.b, hold_full + 8 * hs);
                tma_load_4d(to + S::kTileBytes, &y_map, c * kSlabCols, w.row0 + t * kTile, w.h, w.b, hold_full + 8 * hs);
              }
          } else {
            mbar_arrive(hold_full + 8 * hs);
          }
        }
        for (int n = 0; n < w.steps && ok; ++n) {
          ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(empty + 8 * s, phase));
          if (!ok) break;
          int head, row, left;
          w.block(p, n, &head, &row, &left);
          // Rows behind the last meet zeros in P and dS: they must not hold a NaN.  Behind the tensor's end they are zeros anyway.
          const bool fix = left < kBlock && row + left < (KV ? p.q_len : p.kv_len);
          unsigned char* to = ring + s * S::kStageBytes;
          if (leader) {
            const uint32_t bar = fix ? fixed : full + 8 * s;
            mbar_arrive_expect_tx(bar, S::kStageBytes + S::kRowBytes);
            for (int c = 0; c < S::kSlabs; ++c) {
              tma_load_4d(smem_u32(to) + c * kBlock * 128, &u_map, c * kSlabCols, row, head, w.b, bar);
              tma_load_4d(smem_u32(to) + S::kBlockBytes + c * kBlock * 128, &w_map, c * kSlabCols, row, head, w.b, bar);
            }
            if (KV)
              bulk_load(smem_u32(row_ring) + s * S::kRowBytes, p.rows + (static_cast<long long>(w.b) * p.heads + head) * p.q_pad + row, S::kRowBytes, bar);
          }
          if (fix) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(fixed, fix_phase));
            fix_phase ^= 1;
            zero_rows<S::kSlabs>(to, kBlock, left, round_up(left, 16));
            zero_rows<S::kSlabs>(to + S::kBlockBytes, kBlock, left, round_up(left, 16));
            fence_proxy_async();
            __syncwarp();
            if (leader) mbar_arrive(full + 8 * s);
          }
          if (++s == S::kStages) { s = 0; phase ^= 1; }
        }
      }
      if (!ok)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);         // copies in flight land
    } else if (warp == 9) {
      // ---- products ----
      if (leader) {
        const int k_steps = (p.head_dim + 15) / 16;
        const uint32_t idesc_acc = make_idesc(kTile, round_up(p.head_dim, 16)) | kRowsB;
        int it = 0;
        int ss = 0, as = 0;                      // the ring's next place for s and do v^T, and for the sums
        uint32_t s_phase = 0, seen[2] = {0, 0};  // seen: blocks of each half that have gone into the sums
        bool ok = true;
        for (int item = blockIdx.x; item < p.items && ok; item += gridDim.x, ++it) {
          const Item<DP, KV> w(p, item);
          const int hs = S::kHold == 2 ? it & 1 : 0;
          if (!mbar_wait_suspend(hold_full + 8 * hs, S::kHold == 2 ? (it >> 1) & 1 : it & 1)) break;
          if (!mbar_wait_suspend(acc_free, (it & 1) ^ 1)) break;
          tc_fence_after();
          const uint32_t hold = smem_u32(smem) + hs * S::kHoldBytes;
          // s and do v^T of half t, the n-th step's block in stage st; number: of this block among the half's
          const auto scores = [&](int t, int n, int st, uint32_t number) {
            if (!mbar_wait_suspend((S::kOwn ? s_free : acc_done) + 8 * t, (number & 1) ^ 1)) return false;
            tc_fence_after();
            int head, row, left;
            w.block(p, n, &head, &row, &left);
            const uint32_t idesc = make_idesc(kTile, round_up(left, 16));
            const uint32_t x = hold + (S::kTiles == 2 ? t * 2 * S::kTileBytes : 0), u = smem_u32(ring) + st * S::kStageBytes;
            const uint64_t xd = make_desc(x), yd = make_desc(x + S::kTileBytes), ud = make_desc(u), wd = make_desc(u + S::kBlockBytes);
            const uint32_t d = tmem + S::kStep * t;
            for (int k = 0; k < k_steps; ++k) {
              const uint64_t a = static_cast<uint64_t>((k >> 2) * (kTile * 128 >> 4) + (k & 3) * 2), b = static_cast<uint64_t>((k >> 2) * (kBlock * 128 >> 4) + (k & 3) * 2);
              umma_bf16(d + S::kS, xd + a, ud + b, idesc, k > 0);
            }
            for (int k = 0; k < k_steps; ++k) {
              const uint64_t a = static_cast<uint64_t>((k >> 2) * (kTile * 128 >> 4) + (k & 3) * 2), b = static_cast<uint64_t>((k >> 2) * (kBlock * 128 >> 4) + (k & 3) * 2);
              umma_bf16(d + S::kD, yd + a, wd + b, idesc, k > 0);
            }
            umma_commit(s_full + 8 * t);
            return true;
          };
          const auto sums = [&](int t, int n, int st, bool fresh) {
            if (!mbar_wait_suspend(p_full + 8 * t, seen[t] & 1)) return false;
            tc_fence_after();
            int head, row, left;
            w.block(p, n, &head, &row, &left);
            const int steps = (left + 15) / 16;
            const uint32_t u = smem_u32(ring) + st * S::kStageBytes, d = tmem + S::kStep * t;
            const uint64_t ud = make_desc_rows(u, kBlock * 128), wd = make_desc_rows(u + S::kBlockBytes, kBlock * 128);
            if (KV)
              for (int k = 0; k < steps; ++k)
                umma_bf16_ta(tmem + S::kAcc2 + S::kAccStep * t, d + S::kS + 8 * k, wd + 128 * k, idesc_acc, !fresh || k > 0);
            for (int k = 0; k < steps; ++k)
              umma_bf16_ta(tmem + S::kAcc1 + S::kAccStep * t, d + S::kDs + 8 * k, ud + 128 * k, idesc_acc, !fresh || k > 0);
            umma_commit(acc_done + 8 * t);
            ++seen[t];
            return true;
          };
          const auto forward = [&](int& st) {
            if (++st == S::kStages) st = 0;
          };
          if (S::kTiles == 2) {
            // step n of both halves; s of the step after goes ahead of the sums where it has room
            const auto all_scores = [&](int n, int t) {          // (the first half waits for the block)
              if (t == 0 && !mbar_wait_suspend(full + 8 * ss, s_phase)) return false;
              const bool fine = !w.active[t] || scores(t, n, ss, seen[t] + (S::kOwn && n > 0 ? 1 : 0));
              if (t == 1) {
                forward(ss);
                if (ss == 0) s_phase ^= 1;
              }
              return fine;
            };
            for (int t = 0; t < 2 && ok && w.steps; ++t) ok = all_scores(0, t);
            for (int n = 0; n < w.steps && ok; ++n) {
              for (int t = 0; t < 2 && ok; ++t) {
                if (S::kOwn && n + 1 < w.steps) ok = all_scores(n + 1, t);
                if (ok && w.active[t]) ok = sums(t, n, as, n == 0);
                if (!S::kOwn && ok && n + 1 < w.steps) ok = all_scores(n + 1, t);
              }
              if (ok) umma_commit(empty + 8 * as);
              forward(as);
            }
          } else {
            const auto next_scores = [&](int n) {
              if (!mbar_wait_suspend(full + 8 * ss, s_phase)) return false;
              const bool fine = scores(n & 1, n, ss, seen[n & 1]);
              forward(ss);
              if (ss == 0) s_phase ^= 1;
              return fine;
            };
            for (int n = 0; n < 2 && n < w.steps && ok; ++n) ok = next_scores(n);
            for (int n = 0; n < w.steps && ok; ++n) {
              ok = sums(n & 1, n, as, n == 0);
              if (ok) umma_commit(empty + 8 * as);
              forward(as);
              if (ok && n + 2 < w.steps) ok = next_scores(n + 2);
            }
          }
          if (ok) umma_commit(item_done);
        }
      }
    }
  } else {
    // ---- a thread a row of s ----
    set_registers<true, kSoftmaxRegs>();
    const int t = warp >> 2, quarter = warp & 3, lane = static_cast<int>(lane_id()), row_in_tile = quarter * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(quarter) << 21, mine_at = tmem + S::kStep * t + lanes;
    const float c = p.scale * kLog2E;
    uint32_t seen = 0, before = 0;               // before: steps of the items so far
    int it = 0;
    bool ok = true;
    for (int item = blockIdx.x; item < p.items; item += gridDim.x, ++it) {
      const Item<DP, KV> w(p, item);
      const int row = w.row0 + (S::kTiles == 2 ? t * kTile : 0) + row_in_tile;
      float lse2 = 0.0f, delta = 0.0f;
      if (!KV && w.active[t]) {
        const float2 r = row < p.q_pad ? p.rows[(static_cast<long long>(w.b) * p.heads + w.h) * p.q_pad + row] : make_float2(INFINITY, 0.0f);
        lse2 = r.x;
        delta = r.y;
      }
      // columns [lo, hi) of a block count: Q: hi by the row; KV: lo by the row
      const int edge = KV ? (p.causal ? row - w.off : 0) : (p.causal ? min(w.kv_valid, row + w.off + 1) : w.kv_valid);
      const int tile0 = row - row_in_tile;
      for (int n = S::kTiles == 2 ? 0 : t; n < w.steps && ok; n += S::kTiles == 2 ? 1 : 2) {
        int head, col0, left;
        w.block(p, n, &head, &col0, &left);
        const uint32_t turn = (before + n) / S::kStages, at = before + n - turn * S::kStages;     // this step's place in the ring
        if (KV && !w.active[t]) {                // the block's rows are given back all the same
          ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(full + 8 * at, turn & 1));
          if (!ok) break;
          if (leader) mbar_arrive(empty + 8 * at);
          __syncwarp();
          continue;
        }
        if (!w.active[t]) break;
        ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(s_full + 8 * t, seen & 1));
        // (its lse2 and delta are there: the products have waited for them.  With a single tile this half sees every other block alone; behind
        // s_full the parity is that of this block all the same, whose place is not given back before this warp says so)
        if (KV) ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait_suspend(full + 8 * at, turn & 1));
        if (!ok) break;
        tc_fence_after();
        uint32_t sv[kBlock], dv[kBlock];
        tmem_ld32(mine_at + S::kS, sv);
        tmem_ld32(mine_at + S::kD, dv);
        if (left > 32) {
          tmem_ld32(mine_at + S::kS + 32, sv + 32);
          tmem_ld32(mine_at + S::kD + 32, dv + 32);
        }
        tmem_wait_ld();
        if (S::kOwn) {
          tc_fence_before();
          __syncwarp();
          if (leader) mbar_arrive(s_free + 8 * t);
        }
        const float4* rows = reinterpret_cast<const float4*>(row_ring + at * S::kRowBytes);
        int lo = 0, hi = kBlock;
        bool masked;
        if (KV) {
          lo = edge - col0;
          hi = left;
          masked = left < kBlock || (p.causal && tile0 + kTile - 1 - w.off > col0);
        } else {
          hi = edge - col0;
          masked = (p.causal ? min(w.kv_valid, tile0 + w.off + 1) : w.kv_valid) < col0 + kBlock;
        }
        uint32_t pw[KV ? kBlock / 2 : 1], sw[kBlock / 2];
#pragma unroll
        for (int i = 0; i < kBlock; i += 2) {
          if (i >= 32 && left <= 32) break;
          float4 r = make_float4(lse2, delta, lse2, delta);
          if (KV) r = rows[i >> 1];
          float p0 = exp2_approx(fmaf(c, __uint_as_float(sv[i]), -r.x)), p1 = exp2_approx(fmaf(c, __uint_as_float(sv[i + 1]), -r.z));
          float d0 = p0 * (__uint_as_float(dv[i]) - r.y), d1 = p1 * (__uint_as_float(dv[i + 1]) - r.w);
          if (masked) {
            const bool on0 = i >= lo && i < hi, on1 = i + 1 >= lo && i + 1 < hi;
            p0 = on0 ? p0 : 0.0f;
            d0 = on0 ? d0 : 0.0f;
            p1 = on1 ? p1 : 0.0f;
            d1 = on1 ? d1 : 0.0f;
          }
          if (KV) pw[KV ? i >> 1 : 0] = to_bf16x2(p0, p1);
          sw[i >> 1] = to_bf16x2(d0, d1);
        }
        if (KV) {                                // (its rows have been read)
          __syncwarp();
          if (leader) mbar_arrive(empty + 8 * at);
        }
        if (S::kOwn) {                           // the sums before have read dS
          ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(acc_done + 8 * t, (seen & 1) ^ 1));
          if (!ok) break;
        }
        if (KV) tmem_st16(mine_at + S::kS, pw);
        tmem_st16(mine_at + S::kDs, sw);
        if (left > 32) {
          if (KV) tmem_st16(mine_at + S::kS + 16, pw + (KV ? 16 : 0));
          tmem_st16(mine_at + S::kDs + 16, sw + 16);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (leader) mbar_arrive(p_full + 8 * t);
        ++seen;
      }
      before += w.steps;
      if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(hold_full + 8 * (S::kHold == 2 ? it & 1 : 0), S::kHold == 2 ? (it >> 1) & 1 : it & 1));
      if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(item_done, it & 1));
      // ---- the sums of this half's tile; of a single tile the first half takes the first sums, the second the others ----
      const int hs = S::kHold == 2 ? it & 1 : 0;
      const bool live = S::kTiles == 1 ? w.steps > 0 : w.active[t];
      const int rows_all = KV ? p.kv_len : p.q_len;
      if (ok && live) tc_fence_after();
      for (int part = 0; part < 2; ++part) {
        if (S::kTiles == 1 ? part != t : !KV && part == 1) continue;
        const surgeon_heads& out = part ? p.out2 : p.out1;
        const uint32_t acc = tmem + (part ? S::kAcc2 : S::kAcc1) + S::kAccStep * t + lanes;
        const float f = part ? 1.0f : p.scale;
        if (!ok) {                               // a wait ran out: this warp's rows are NaN, here and from here on
          if (row < rows_all) {
            if (KV && p.splits > 1) {
              float* to = p.partial + (((static_cast<long long>(w.split) * 2 + part) * p.batch + w.b) * p.kv_heads + w.h) * static_cast<long long>(p.kv_len) * p.head_dim +
                          static_cast<long long>(row) * p.head_dim;
              for (int i = 0; i < p.head_dim; ++i) to[i] = __uint_as_float(0x7FC00000u);
            } else {
              unsigned short* to = static_cast<unsigned short*>(out.data) + w.b * out.batch_stride + static_cast<long long>(row) * out.row_stride + w.h * out.head_stride;
              for (int i = 0; i < p.head_dim; ++i) to[i] = 0x7FC0u;
            }
          }
          continue;
        }
        const bool some = live && row < w.valid;
        unsigned char* stage = smem + hs * S::kHoldBytes + (S::kTiles == 2 ? t * 2 + part : part) * S::kTileBytes;
#pragma unroll 1
        for (int q = 0; q < DP / 32; ++q) {
          uint32_t o[32];
          if (live) {
            tmem_ld32(acc + 32 * q, o);
            tmem_wait_ld();
          }
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = some ? __float_as_uint(__uint_as_float(o[i]) * f) : 0u;
          if (KV && p.splits > 1) {
            if (row < p.kv_len) {
              float* to = p.partial + (((static_cast<long long>(w.split) * 2 + part) * p.batch + w.b) * p.kv_heads + w.h) * static_cast<long long>(p.kv_len) * p.head_dim +
                          static_cast<long long>(row) * p.head_dim + 32 * q;
#pragma unroll
              for (int i = 0; i < 8; ++i)
                if (32 * q + 4 * i < p.head_dim) *reinterpret_cast<uint4*>(to + 4 * i) = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const auto two = [&](int e) { return to_bf16x2(__uint_as_float(o[8 * i + e]), __uint_as_float(o[8 * i + e + 1])); };
              *reinterpret_cast<uint4*>(stage + (q >> 1) * kTile * 128 + tile_off(row_in_tile, (q & 1) * 4 + i)) = make_uint4(two(0), two(2), two(4), two(6));
            }
          }
        }
        if (!(KV && p.splits > 1)) {
          fence_proxy_async();
          __syncwarp();
          if (leader) {
            const int first = tile0 + quarter * 32;
            if (first < rows_all)
              for (int i = 0; i < S::kSlabs; ++i)
                tma_store_4d(part ? &o2_map : &o1_map, smem_u32(stage) + i * kTile * 128 + quarter * 32 * 128, i * kSlabCols, first, w.h, w.b);
            bulk_commit();
          }
          __syncwarp();
        }
      }
      tc_fence_before();
      __syncwarp();
      if (leader && ok) {
        mbar_arrive(acc_free);
        bulk_wait_read();
        mbar_arrive(hold_empty + 8 * hs);
      }
      __syncwarp();
    }
  }
  __syncwarp();                                  // (the roles of one lane end here; the barriers take whole warps)
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// lse2 and delta of every row; +infinity and 0 for rows that see nothing and for those that fill the last block up.
// 16 lanes a row, 16 bytes each.
__global__ void __launch_bounds__(256)
attention_rows_kernel(const surgeon_heads o, const surgeon_heads dout, const float* lse, const int* q_lengths, int heads, int q_len, int q_pad,
                      int head_dim, long long total, float2* rows) {
  pdl_trigger();
  pdl_wait();
  const long long at = (static_cast<long long>(blockIdx.x) * 256 + threadIdx.x) >> 4;    // ((b * q_pad) + row) * heads + h: neighbours in memory
  const int part = threadIdx.x & 15;
  if (at >= total) return;                       // (sixteen lanes at a time)
  const int h = static_cast<int>(at % heads);
  const long long br = at / heads;
  const int row = static_cast<int>(br % q_pad), b = static_cast<int>(br / q_pad);
  const bool on = row < length_of(q_lengths, b, q_len);
  float sum = 0.0f;
  if (on && part * 8 < head_dim) {
    float a[8], d[8];
    load_elems<1, 8>(o.data, b * o.batch_stride + static_cast<long long>(row) * o.row_stride + h * o.head_stride + part * 8, a);
    load_elems<1, 8>(dout.data, b * dout.batch_stride + static_cast<long long>(row) * dout.row_stride + h * dout.head_stride + part * 8, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf(a[i], d[i], sum);
  }
  const uint32_t mask = 0xFFFFu << (threadIdx.x & 16);
#pragma unroll
  for (int i = 8; i > 0; i >>= 1) sum += __shfl_xor_sync(mask, sum, i);
  if (part == 0) {
    const float l = on ? lse[(static_cast<long long>(b) * heads + h) * q_len + row] : -INFINITY;
    rows[(static_cast<long long>(b) * heads + h) * q_pad + row] = l == -INFINITY ? make_float2(INFINITY, 0.0f) : make_float2(l * kLog2E, sum);
  }
}

// dk and dv from the parts' sums, in the order of the parts.
__global__ void __launch_bounds__(256)
attention_join_kernel(const float* partial, const surgeon_heads dk, const surgeon_heads dv, int splits, int kv_heads, int kv_len, int head_dim,
                      long long vectors, long long part_size) {
  pdl_trigger();
  pdl_wait();
  const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;    // of 8 elements, of dk then dv
  if (i >= 2 * vectors) return;
  const int which = i >= vectors;
  const long long e = (i - which * vectors) * 8;
  float sum[8] = {};
  for (int s = 0; s < splits; ++s) {
    float f[8];
    load_elems<0, 8>(partial + (static_cast<long long>(s) * 2 + which) * part_size, e, f);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] += f[k];
  }
  const surgeon_heads& out = which ? dv : dk;
  const int d = static_cast<int>(e % head_dim);
  const long long r = e / head_dim;
  const int row = static_cast<int>(r % kv_len);
  const long long bh = r / kv_len;
  store_elems<1, 8>(out.data, bh / kv_heads * out.batch_stride + static_cast<long long>(row) * out.row_stride + bh % kv_heads * out.head_stride + d, sum);
}

// Parts of the queries that the keys' tiles are shared out in: enough for two items an SM (they differ in length), eight blocks each at least.
int splits_of(const surgeon_attention_desc& d) {
  const int rows = kTile * (d.head_dim <= 64 ? 2 : 1);
  const long long items = static_cast<long long>(d.batch) * d.kv_heads * ((d.kv_len + rows - 1) / rows);
  const long long steps = static_cast<long long>(d.heads / d.kv_heads) * ((d.q_len + kBlock - 1) / kBlock);
  if (items <= 0 || items >= 2 * 148) return 1;
  long long splits = (2 * 148 + items - 1) / items;
  if (splits > steps / 8) splits = steps / 8;
  return splits < 1 ? 1 : static_cast<int>(splits);
}
int padded(int q_len) { return round_up(q_len, 128); }
size_t rows_bytes(const surgeon_attention_desc& d) {
  return (static_cast<size_t>(d.batch) * d.heads * padded(d.q_len) * sizeof(float2) + 255) & ~static_cast<size_t>(255);
}
size_t part_elems(const surgeon_attention_desc& d) { return static_cast<size_t>(d.batch) * d.kv_heads * d.kv_len * d.head_dim; }

template <int DP, bool KV>
cudaError_t launch_pass(const surgeon_attention_desc& d, const surgeon_heads& x, const surgeon_heads& y, const surgeon_heads& u, const surgeon_heads& w,
                        Args a, cudaStream_t stream) {
  using S = Shape<DP, KV>;
  const int stay = KV ? d.kv_len : d.q_len, go = KV ? d.q_len : d.kv_len;
  if (stay == 0) return cudaSuccess;
  const int stay_heads = KV ? d.kv_heads : d.heads, go_heads = KV ? d.heads : d.kv_heads;
  a.tiles = (stay + S::kTiles * kTile - 1) / (S::kTiles * kTile);
  if (!KV) a.splits = 1;
  a.items = a.tiles * d.batch * stay_heads * a.splits;
  CUtensorMap maps[6];
  memset(maps, 0, sizeof(maps));
  bool ok = encode(&maps[0], x, d.batch, stay, stay_heads, d.head_dim, kTile) && encode(&maps[1], y, d.batch, stay, stay_heads, d.head_dim, kTile) &&
            encode(&maps[2], u, d.batch, go, go_heads, d.head_dim, kBlock) && encode(&maps[3], w, d.batch, go, go_heads, d.head_dim, kBlock) &&
            encode(&maps[4], a.out1, d.batch, stay, stay_heads, d.head_dim, 32);
  if (KV) ok = ok && encode(&maps[5], a.out2, d.batch, stay, stay_heads, d.head_dim, 32);
  if (!ok) return cudaErrorInvalidValue;
  const auto kernel = attention_grad_kernel<DP, KV>;
  cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), S::kSmem);
  if (e != cudaSuccess) return e;
  const int grid = a.items < sm_count() ? a.items : sm_count();
  e = launch_kernel(kernel, dim3(grid), dim3(kThreads), S::kSmem, stream, true, maps[0], maps[1], maps[2], maps[3], maps[4], maps[5], a);
  note_launches(1);
  return e;
}

template <int DP>
cudaError_t launch_as(const surgeon_attention_desc& d, const surgeon_heads& q, const surgeon_heads& k, const surgeon_heads& v, const surgeon_heads& dout,
                      const surgeon_heads* dq, const surgeon_heads* dk, const surgeon_heads* dv, Args a, cudaStream_t stream) {
  cudaError_t e = cudaSuccess;
  if (dq) {
    a.out1 = *dq;
    e = launch_pass<DP, false>(d, q, dout, k, v, a, stream);
    if (e != cudaSuccess) return e;
  }
  if (!dk || d.kv_len == 0) return e;
  a.out1 = *dk;
  a.out2 = *dv;
  e = launch_pass<DP, true>(d, k, v, q, dout, a, stream);
  if (e != cudaSuccess || a.splits == 1) return e;
  const long long size = static_cast<long long>(part_elems(d)), vectors = size / 8;
  e = launch_kernel(attention_join_kernel, dim3(static_cast<unsigned>((2 * vectors + 255) / 256)), dim3(256), 0, stream, true,
                    static_cast<const float*>(a.partial), *dk, *dv, a.splits, d.kv_heads, d.kv_len, d.head_dim, vectors, size);
  note_launches(1);
  return e;
}

}  // namespace

size_t attention_grad_workspace(const surgeon_attention_desc& d) {
  const int splits = splits_of(d);
  const size_t n = rows_bytes(d) + (splits > 1 ? splits * 2 * part_elems(d) * sizeof(float) : 0);
  return n < 16 ? 16 : n;
}

cudaError_t launch_attention_grad(const surgeon_attention_desc& d, const surgeon_heads& q, const surgeon_heads& k, const surgeon_heads& v,
                                  const surgeon_heads& o, const surgeon_heads& dout, const float* lse, const int* q_lengths,
                                  const int* kv_lengths, const surgeon_heads* dq, const surgeon_heads* dk, const surgeon_heads* dv,
                                  void* workspace, cudaStream_t stream) {
  if (!dq && !dk) return cudaSuccess;
  float2* rows = static_cast<float2*>(workspace);
  const int q_pad = padded(d.q_len);
  if (d.q_len > 0) {
    const long long total = static_cast<long long>(d.batch) * d.heads * q_pad;
    const cudaError_t e = launch_kernel(attention_rows_kernel, dim3(static_cast<unsigned>((total + 15) / 16)), dim3(256), 0, stream, true, o, dout, lse,
                                        q_lengths, d.heads, d.q_len, q_pad, d.head_dim, total, rows);
    note_launches(1);
    if (e != cudaSuccess) return e;
  }
  Args a = {};
  a.batch = d.batch; a.heads = d.heads; a.kv_heads = d.kv_heads; a.group = d.heads / d.kv_heads;
  a.q_len = d.q_len; a.kv_len = d.kv_len; a.head_dim = d.head_dim; a.causal = d.causal != 0;
  a.q_pad = q_pad;
  a.splits = splits_of(d);
  a.scale = static_cast<float>(d.scale);
  a.q_lengths = q_lengths; a.kv_lengths = kv_lengths;
  a.rows = rows;
  a.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + rows_bytes(d));
  return d.head_dim <= 64 ? launch_as<64>(d, q, k, v, dout, dq, dk, dv, a, stream) : launch_as<128>(d, q, k, v, dout, dq, dk, dv, a, stream);
}

}  // namespace surgeon
