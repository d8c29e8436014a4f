// Attention, forward: o = softmax(scale q k^T) v of every sequence and head, one pass over the keys with the running maximum and sum.
//
//   m' = max(m, max_j s_j);  l' = l 2^(c (m - m')) + sum_j 2^(c (s_j - m'));  o' = o 2^(c (m - m')) + sum_j 2^(c (s_j - m')) v_j,
//   c = scale log2(e);  in the end o / l and lse = scale m + log l
//
// A CTA takes 256 queries of a head, two tiles of 128, and walks the keys in blocks of 128.  s = q k^T goes to tensor memory (lane = query),
// four warps a tile read it back, a thread a row, and leave 2^(c (s - m)) as bf16 in tensor memory, where it is the A operand
// of the product with v: neither s nor p is ever in shared memory.  o stays in tensor memory over all blocks; it is multiplied by
// 2^(c (m - m')) only when a row's maximum grew by more than 2^8, so hardly ever after the first block (p then is at most 2^8, as
// exact in bf16 as below 1).  While the four warps of one tile compute, the products of the other run.
// Persistent CTAs: the next item's queries, keys and values are on their way while this one's end.
#include "attention.cuh"

namespace surgeon {

namespace {

using namespace tc;
using namespace att;

constexpr int kBlock = 128;                      // keys of a block
constexpr int kThreads = 384;                    // 2 x 4 softmax warps, one that copies, one that issues products, two that idle
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;               // 2 x 208 + 88 = 3 x 168, what 384 threads are launched with
constexpr int kMaxStages = 8;
constexpr float kGrowth = 8.0f;                  // log2 of what p may grow to before o is scaled

template <int DP> struct Shape {                 // DP: head_dim, padded to 64 or 128
  static constexpr int kSlabs = DP / kSlabCols, kTileBytes = kTile * DP * 2;
  static constexpr bool kOwnP = DP == 64;        // p has columns of its own, else it takes the place of s
  static constexpr int kQStages = DP == 64 ? 2 : 1, kStages = DP == 64 ? 8 : 4;
  static constexpr uint32_t kS = 0, kP = DP == 64 ? 256 : 0, kPStep = DP == 64 ? 64 : 128, kO = DP == 64 ? 384 : 256;  // columns; tile 1's s: + 128
  static constexpr int kSmem = 1024 + (2 * kQStages + kStages) * kTileBytes;
};

struct Args {
  int batch, heads, group, q_len, kv_len, head_dim, causal;     // group: heads that share keys
  int tiles, items;                              // pairs of tiles of a head
  float scale;
  const int* q_lengths;
  const int* kv_lengths;
  surgeon_heads o;
  float* lse;
};

struct Item {
  int b, h, row0, q_valid, kv_valid, off;
  int keys[2], blocks[2], most;                  // of each tile
  __device__ __forceinline__ Item(const Args& p, int item) {
    const int pairs = p.batch * p.heads;
    int bh, qt;
    if (p.causal) {                              // the longest first
      qt = p.tiles - 1 - item / pairs;
      bh = item % pairs;
    } else {
      bh = item / p.tiles;
      qt = item % p.tiles;
    }
    b = bh / p.heads;
    h = bh % p.heads;
    row0 = qt * 2 * kTile;
    q_valid = length_of(p.q_lengths, b, p.q_len);
    kv_valid = length_of(p.kv_lengths, b, p.kv_len);
    off = kv_valid - q_valid;
    most = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r0 = row0 + t * kTile, last = min(r0 + kTile, q_valid) - 1;
      keys[t] = r0 >= q_valid ? 0 : p.causal ? max(0, min(kv_valid, last + off + 1)) : kv_valid;
      blocks[t] = (keys[t] + kBlock - 1) / kBlock;
      most = max(most, blocks[t]);
    }
  }
};

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
attention_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                 const __grid_constant__ CUtensorMap o_map, const __grid_constant__ Args p) {
  using S = Shape<DP>;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  unsigned char* ring = smem + 2 * S::kQStages * S::kTileBytes;
  __shared__ __align__(8) unsigned long long bars[2 * kMaxStages + 8 + 8 + 1];
  __shared__ uint32_t tmem_slot;

  const int warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x) >> 5, 0);
  const bool leader = elected();
  const uint32_t full = smem_u32(bars), empty = full + 8 * kMaxStages;
  const uint32_t q_full = empty + 8 * kMaxStages, q_empty = q_full + 32;         // [stage][tile]
  const uint32_t s_full = q_empty + 32, s_free = s_full + 16, p_full = s_free + 16, o_done = p_full + 16;   // [tile]
  const uint32_t fixed = o_done + 16;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(q_full + 8 * i, 1);
      mbar_init(q_empty + 8 * i, 4);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(s_full + 8 * t, 1);
      mbar_init(s_free + 8 * t, 4);
      mbar_init(p_full + 8 * t, 4);
      mbar_init(o_done + 8 * t, 1);
    }
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
    uint32_t phase = 1, fix_phase = 0;           // (a fresh barrier counts as passed in its phase before)
    bool ok = true;
    for (int item = blockIdx.x; item < p.items && ok; item += gridDim.x, ++it) {
      const Item w(p, item);
      const int qs = S::kQStages == 2 ? it & 1 : 0;
      const uint32_t q_phase = (S::kQStages == 2 ? (it >> 1) & 1 : it & 1) ^ 1;
      for (int t = 0; t < 2 && ok; ++t) {
        const int at = 2 * qs + t;
        ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(q_empty + 8 * at, q_phase));
        if (!ok) break;
        if (leader) {
          if (w.blocks[t]) {
            mbar_arrive_expect_tx(q_full + 8 * at, S::kTileBytes);
            for (int c = 0; c < S::kSlabs; ++c)
              tma_load_4d(smem_u32(smem) + at * S::kTileBytes + c * kTile * 128, &q_map, c * kSlabCols, w.row0 + t * kTile, w.h, w.b, q_full + 8 * at);
          } else {
            mbar_arrive(q_full + 8 * at);
          }
        }
      }
      for (int j = 0; j < 2 * w.most && ok; ++j) {               // k and v in turn
        ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(empty + 8 * s, phase));
        if (!ok) break;
        const int row = (j >> 1) * kBlock, left = w.kv_valid - row;
        // Rows of v behind the last key meet probabilities of zero: they must not hold a NaN.  Behind the tensor's end they are zeros anyway.
        const bool fix = (j & 1) && left < kBlock && w.kv_valid < p.kv_len;
        unsigned char* to = ring + s * S::kTileBytes;
        if (leader) {
          const uint32_t bar = fix ? fixed : full + 8 * s;
          mbar_arrive_expect_tx(bar, S::kTileBytes);
          for (int c = 0; c < S::kSlabs; ++c)
            tma_load_4d(smem_u32(to) + c * kBlock * 128, j & 1 ? &v_map : &k_map, c * kSlabCols, row, w.h / p.group, w.b, bar);
        }
        if (fix) {
          ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(fixed, fix_phase));
          fix_phase ^= 1;
          zero_rows<S::kSlabs>(to, kBlock, left, round_up(left, 16));
          fence_proxy_async();
          __syncwarp();
          if (leader) mbar_arrive(full + 8 * s);
        }
        if (++s == S::kStages) { s = 0; phase ^= 1; }
      }
    }
    if (!ok)
      for (int i = 0; i < 1000; ++i) __nanosleep(1000);           // copies in flight land
  } else if (warp == 9) {
    // ---- products ----
    if (leader) {
      const int k_steps = (p.head_dim + 15) / 16, n_o = round_up(p.head_dim, 16);
      const uint32_t idesc_o = make_idesc(kTile, n_o) | kRowsB;
      int s = 0, it = 0;                         // the ring's next tile
      uint32_t phase = 0;
      uint32_t seen[2] = {0, 0};                 // blocks of each tile so far
      bool ok = true;
      for (int item = blockIdx.x; item < p.items && ok; item += gridDim.x, ++it) {
        const Item w(p, item);
        const int qs = S::kQStages == 2 ? it & 1 : 0;
        const uint32_t q_phase = S::kQStages == 2 ? (it >> 1) & 1 : it & 1;
        for (int t = 0; t < 2 && ok; ++t) ok = mbar_wait_suspend(q_full + 8 * (2 * qs + t), q_phase);
        if (!ok) break;
        if (!w.most) continue;
        // s of tile t and block j from the keys in stage ks
        const auto scores = [&](int t, int j, int ks) {
          if (!mbar_wait_suspend((S::kOwnP ? s_free : o_done) + 8 * t, (seen[t] & 1) ^ 1)) return false;
          tc_fence_after();
          const uint32_t idesc = make_idesc(kTile, round_up(min(kBlock, w.keys[t] - j * kBlock), 16));
          const uint64_t a = make_desc(smem_u32(smem) + (2 * qs + t) * S::kTileBytes), b = make_desc(smem_u32(ring) + ks * S::kTileBytes);
          for (int k = 0; k < k_steps; ++k) {
            const uint64_t step = static_cast<uint64_t>((k >> 2) * (kTile * 128 >> 4) + (k & 3) * 2);
            umma_bf16(tmem + S::kS + 128 * t, a + step, b + step, idesc, k > 0);
          }
          umma_commit(s_full + 8 * t);
          return true;
        };
        const auto values = [&](int t, int j, int vs) {
          if (!mbar_wait_suspend(p_full + 8 * t, seen[t] & 1)) return false;
          tc_fence_after();
          const int steps = (min(kBlock, w.keys[t] - j * kBlock) + 15) / 16;
          const uint64_t b = make_desc_rows(smem_u32(ring) + vs * S::kTileBytes, kBlock * 128);
          for (int k = 0; k < steps; ++k)
            umma_bf16_ta(tmem + S::kO + DP * t, tmem + S::kP + S::kPStep * t + 8 * k, b + 128 * k, idesc_o, j > 0 || k > 0);
          umma_commit(o_done + 8 * t);
          ++seen[t];
          return true;
        };
        const auto next = [&](int& stage, uint32_t& ph) {
          if (++stage == S::kStages) { stage = 0; ph ^= 1; }
        };
        // stage of k of block j: s; of v: the one behind it; of k of the block after: the one behind that
        if (!mbar_wait_suspend(full + 8 * s, phase)) break;
        for (int t = 0; t < 2 && ok; ++t)
          if (w.blocks[t]) ok = scores(t, 0, s);
        for (int j = 0; j < w.most && ok; ++j) {
          const int ks = s;
          next(s, phase);
          umma_commit(empty + 8 * ks);           // (its products have been issued)
          const int vs = s;
          const uint32_t v_phase = phase;
          next(s, phase);
          bool v_there = false, k_there = false;
          for (int t = 0; t < 2 && ok; ++t) {
            if (j >= w.blocks[t]) continue;
            const bool more = j + 1 < w.blocks[t];
            const auto ahead = [&]() {
              if (!more) return true;
              if (!k_there && !mbar_wait_suspend(full + 8 * s, phase)) return false;
              k_there = true;
              if (S::kOwnP) ++seen[t];           // (that block's number, for its own wait)
              const bool fine = scores(t, j + 1, s);
              if (S::kOwnP) --seen[t];
              return fine;
            };
            if (S::kOwnP) ok = ahead();
            if (ok && !v_there) ok = v_there = mbar_wait_suspend(full + 8 * vs, v_phase);
            ok = ok && values(t, j, vs);
            if (!S::kOwnP) ok = ok && ahead();
          }
          if (ok) umma_commit(empty + 8 * vs);
        }
      }
    }
  }
  } else {
    // ---- softmax: a thread a row ----
    set_registers<true, kSoftmaxRegs>();
    const int t = warp >> 2, quarter = warp & 3, lane = static_cast<int>(lane_id()), row_in_tile = quarter * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(quarter) << 21;
    const uint32_t s_at = tmem + S::kS + 128 * t + lanes, p_at = tmem + S::kP + S::kPStep * t + lanes, o_at = tmem + S::kO + DP * t + lanes;
    const float c = p.scale * kLog2E, grown = kGrowth / c;
    uint32_t seen = 0;
    int it = 0;
    bool ok = true;
    for (int item = blockIdx.x; item < p.items; item += gridDim.x, ++it) {
      const Item w(p, item);
      const int row = w.row0 + t * kTile + row_in_tile;
      const int mine = p.causal ? min(w.kv_valid, row + w.off + 1) : w.kv_valid;         // keys that this row sees
      const int all = p.causal ? min(w.kv_valid, w.row0 + t * kTile + w.off + 1) : w.kv_valid;    // that every row of the tile sees
      float m = -INFINITY, l = 0.0f;
      const int blocks = w.blocks[t], qs = S::kQStages == 2 ? it & 1 : 0;
      for (int j = 0; j < blocks && ok; ++j, ++seen) {
        ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(s_full + 8 * t, seen & 1));
        if (!ok) break;
        tc_fence_after();
        const int cols = min(kBlock, w.keys[t] - j * kBlock);
        uint32_t v[kBlock];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q * 32 < cols) tmem_ld32(s_at + 32 * q, v + 32 * q);
        tmem_wait_ld();
        if (S::kOwnP) {
          tc_fence_before();
          __syncwarp();
          if (leader) mbar_arrive(s_free + 8 * t);
        }
        const bool masked = (j + 1) * kBlock > all;
        const int limit = mine - j * kBlock;
        float top = -INFINITY;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (q * 32 >= cols) break;
          if (masked) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (q * 32 + i >= limit) v[q * 32 + i] = 0xFF800000u;
          }
          float a[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < 32; ++i) a[i & 3] = fmaxf(a[i & 3], __uint_as_float(v[q * 32 + i]));
          top = fmaxf(top, fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])));
        }
        if (j > 0) {
          // the block before has gone into o, and p may be written
          ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(o_done + 8 * t, (seen & 1) ^ 1));
          if (!ok) break;
          if (__any_sync(0xFFFFFFFFu, top > m + grown)) {
            tc_fence_after();
            const float to = fmaxf(m, top), f = m == to ? 1.0f : exp2_approx(c * (m - to));
            m = to;
            l *= f;
#pragma unroll 1
            for (int q = 0; q < DP / 32; ++q) {
              uint32_t o[32];
              tmem_ld32(o_at + 32 * q, o);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_st32(o_at + 32 * q, o);
            }
          }
        } else {
          m = top;
        }
        const float mc = m == -INFINITY ? 0.0f : c * m;          // (no key so far: all p are 0)
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (q * 32 >= cols) break;
          uint32_t w16[16];
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float x = exp2_approx(fmaf(c, __uint_as_float(v[q * 32 + i]), -mc)), y = exp2_approx(fmaf(c, __uint_as_float(v[q * 32 + i + 1]), -mc));
            sum[i & 3] += x;
            sum[(i & 3) + 1] += y;
            w16[i >> 1] = to_bf16x2(x, y);
          }
          tmem_st16(p_at + 16 * q, w16);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (leader) mbar_arrive(p_full + 8 * t);
      }
      if (ok && blocks) ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(o_done + 8 * t, (seen & 1) ^ 1));
      // the queries' place takes the outputs: they are not read any more
      if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait_suspend(q_full + 8 * (2 * qs + t), S::kQStages == 2 ? (it >> 1) & 1 : it & 1));
      if (!ok) {                                 // a wait ran out: this warp's rows are NaN, here and from here on
        if (row < p.q_len) {
          unsigned short* to = static_cast<unsigned short*>(p.o.data) + w.b * p.o.batch_stride + static_cast<long long>(row) * p.o.row_stride + w.h * p.o.head_stride;
          for (int i = 0; i < p.head_dim; ++i) to[i] = 0x7FC0u;
          if (p.lse) p.lse[(static_cast<long long>(w.b) * p.heads + w.h) * p.q_len + row] = __uint_as_float(0x7FC00000u);
        }
        continue;
      }
      const bool none = l == 0.0f || row >= w.q_valid;
      const float inv = 1.0f / l;
      if (blocks) tc_fence_after();
      unsigned char* stage = smem + (2 * qs + t) * S::kTileBytes;
#pragma unroll 1
      for (int q = 0; q < DP / 32; ++q) {
        uint32_t o[32];
        if (blocks) {
          tmem_ld32(o_at + 32 * q, o);
          tmem_wait_ld();
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint4 u = make_uint4(0u, 0u, 0u, 0u);
          if (blocks && !none) {
            const auto two = [&](int e) { return to_bf16x2(__uint_as_float(o[8 * i + e]) * inv, __uint_as_float(o[8 * i + e + 1]) * inv); };
            u = make_uint4(two(0), two(2), two(4), two(6));
          }
          *reinterpret_cast<uint4*>(stage + (q >> 1) * kTile * 128 + tile_off(row_in_tile, (q & 1) * 4 + i)) = u;
        }
      }
      if (p.lse && row < p.q_len)
        p.lse[(static_cast<long long>(w.b) * p.heads + w.h) * p.q_len + row] = none ? -INFINITY : fmaf(m, p.scale, logf(l));
      tc_fence_before();
      fence_proxy_async();
      __syncwarp();
      if (leader) {
        const int first = w.row0 + t * kTile + quarter * 32;
        if (first < p.q_len)
          for (int i = 0; i < S::kSlabs; ++i)
            tma_store_4d(&o_map, smem_u32(stage) + i * kTile * 128 + quarter * 32 * 128, i * kSlabCols, first, w.h, w.b);
        bulk_commit();
        bulk_wait_read();
        mbar_arrive(q_empty + 8 * (2 * qs + t));
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

template <int DP>
cudaError_t launch_as(const surgeon_attention_desc& d, const surgeon_heads& q, const surgeon_heads& k, const surgeon_heads& v, const surgeon_heads& o,
                      Args& a, cudaStream_t stream) {
  CUtensorMap maps[4];
  if (!encode(&maps[0], q, d.batch, d.q_len, d.heads, d.head_dim, kTile) || !encode(&maps[1], k, d.batch, d.kv_len, d.kv_heads, d.head_dim, kBlock) ||
      !encode(&maps[2], v, d.batch, d.kv_len, d.kv_heads, d.head_dim, kBlock) || !encode(&maps[3], o, d.batch, d.q_len, d.heads, d.head_dim, 32))
    return cudaErrorInvalidValue;
  const auto kernel = attention_kernel<DP>;
  const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), Shape<DP>::kSmem);
  if (e != cudaSuccess) return e;
  const int grid = a.items < sm_count() ? a.items : sm_count();
  const cudaError_t l = launch_kernel(kernel, dim3(grid), dim3(kThreads), Shape<DP>::kSmem, stream, true, maps[0], maps[1], maps[2], maps[3], a);
  note_launches(1);
  return l;
}

}  // namespace

size_t attention_workspace(const surgeon_attention_desc&) { return 0; }

cudaError_t launch_attention(const surgeon_attention_desc& d, const surgeon_heads& q, const surgeon_heads& k, const surgeon_heads& v,
                             const int* q_lengths, const int* kv_lengths, const surgeon_heads& o, float* lse, void*, cudaStream_t stream) {
  Args a = {};
  a.batch = d.batch; a.heads = d.heads; a.group = d.heads / d.kv_heads;
  a.q_len = d.q_len; a.kv_len = d.kv_len; a.head_dim = d.head_dim; a.causal = d.causal != 0;
  a.tiles = (d.q_len + 2 * kTile - 1) / (2 * kTile);
  a.items = a.tiles * d.batch * d.heads;
  a.scale = static_cast<float>(d.scale);
  a.q_lengths = q_lengths; a.kv_lengths = kv_lengths;
  a.o = o;
  a.lse = lse;
  return d.head_dim <= 64 ? launch_as<64>(d, q, k, v, o, a, stream) : launch_as<128>(d, q, k, v, o, a, stream);
}

}  // namespace surgeon
