// Matrix product of a linear layer on the tensor cores, bias, activation and residual in its epilogue.
//
//   z[m, n] = sum_k a[m, k] b[n, k] + bias[n];  y = act(z) + residual;  z itself, rounded to bf16, where it is kept
//
// Persistent CTAs (or CTA pairs, cta_group::2: 256 rows, each CTA its 128 and half of the columns' operand) walk the output
// tiles, columns fastest.  Warp 0 fetches operands by TMA into a ring, warp 1 issues the MMAs into one of two accumulators
// in tensor memory, sixteen or eight warps (EPI) take the other one: lane = row, 32 columns at a time.  A piece of
// 32 x 32 goes through shared memory, where the residual has been fetched by TMA before, and leaves by TMA.
// b is K-major (weights [n, k], forward) or N-major (weights [k, n], the input's gradient): both are read as they lie.
//
// What bounds it: wide layers the tensor pipe (16384 x 2048 x 2048 with a residual 112-116 us under the power cap, 1185-1225 TFLOP/s, 0.87 of
// a library product's sustained rate; 98 in short runs); few columns of reduction the epilogue (16384 x 128 -> 512 with GELU and z kept:
// 27 instructions an element, 13 us for 38 MB); the input's gradient an SM's intake of operands (12608 x 768 <- 2304: 38 us, 1170
// TFLOP/s; the call with dz and its sums written from the tiles 57, in long runs under the power cap 65-68).
#include <cuda.h>
#include <string.h>

#include "linear.cuh"
#include "tc_common.cuh"

namespace surgeon {

namespace {

using namespace tc;

constexpr int kTileK = 64;                       // 128 bytes of bf16
constexpr int kTileM = 128;                      // rows of a CTA
constexpr int kABytes = kTileM * 128;
constexpr int kMaxStages = 8;
constexpr int kCols = 32;                        // columns (and rows) of a piece
constexpr int kPrePiece = 32 * kCols * 2;
constexpr int kCopyWarps = 4;
template <int COPY, int EPI> constexpr int kThreads = (2 + EPI + (COPY ? kCopyWarps : 0)) * 32;
template <int DT> constexpr int kPiece = 32 * kCols * (DT ? 2 : 4);

struct TileArgs {
  int m, n, k;
  int tile_n;                                    // columns of a tile
  int tiles_n, tiles;
  int step_m, step_n;                            // from a CTA's tile to its next: rows and columns of tiles
  int stages, stage_bytes, ktiles;
  int tmem_cols;
  int vec_y, vec_pre;                            // rows of y (and the residual), of pre, start at 16-byte boundaries: TMA
  const float* bias;
  const void* residual;
  void* y;
  unsigned short* pre;
  uint32_t* status;
  ColumnSums sums;
  CopyOut copy;
};

__device__ __forceinline__ void tma_store_2d(const void* tmap, uint32_t smem_src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(tmap), "r"(x), "r"(y),
               "r"(smem_src)
               : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void bulk_wait_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Descriptor of an N-major operand: rows of 64 elements per k, slabs of 64 k-rows (8 KB) along n.
__device__ __forceinline__ uint64_t make_desc_rows(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>((kTileK * 128) >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}

// Byte offset of 16-byte chunk `j` of row `r` in a piece of rows of 128 (64) bytes, as TMA lays it out.
template <int ROW>
__device__ __forceinline__ uint32_t piece_at(int r, int j) {
  return ROW == 128 ? static_cast<uint32_t>(r * 128 + ((j ^ (r & 7)) << 4)) : static_cast<uint32_t>(r * 64 + ((j ^ ((r >> 1) & 3)) << 4));
}

// Column `c` of row `r` in a piece of 32 columns of type T.
template <typename T>
__device__ __forceinline__ uint32_t piece_elem(int r, int c) {
  constexpr int kPer = 16 / sizeof(T);
  return piece_at<32 * static_cast<int>(sizeof(T))>(r, c / kPer) + (c % kPer) * static_cast<uint32_t>(sizeof(T));
}
// A lane's column of a piece whose rows TMA cannot reach, from and to global memory: eight rows on their way at a time.
template <typename T, typename F>
__device__ __forceinline__ void copy_piece(const T* from, long long pitch, int rows, bool on, F&& place) {
#pragma unroll 1
  for (int q = 0; q < 32; q += 8) {
    T v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = on && q + i < rows ? from[(q + i) * pitch] : T(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) *place(q + i) = v[i];
  }
}
template <typename T, typename F>
__device__ __forceinline__ void copy_out(T* to, long long pitch, int rows, bool on, F&& value) {
#pragma unroll 1
  for (int q = 0; q < 32; q += 8) {
    T v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = value(q + i);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (on && q + i < rows) to[(q + i) * pitch] = v[i];
  }
}

__device__ __forceinline__ void mbar_arrive_many(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

// One of four warps' 32 rows of an operand tile (128 x 64 bf16 at `tile`, as TMA laid it out; rows m0 ..., columns k0 ... of [m, k],
// whose tile row is `slab`): to fp32 in c.out, and the columns' sums of all 128 rows.  The rows are taken into registers and the
// ring's stage given back at `bar` before the copy is written: held until then, it kept the MMAs waiting (12608 x 768 <- 2304 with both
// 77 us against 67 with four stages; a pass of its own over dy before the product took 80).  Given back only with all words arrived:
// an issued load may stand behind the stores of the tile before for longer than the stage's next copy takes, and then
// finds that copy.  Every lane's sum takes all of its words and is stored before the fence, which orders the reads before the
// refill by TMA (another proxy).
// `buf`: [4][64], another one than the call before had.  `there`: false once a wait of this warp ran out.  It goes on all the same, since
// the other three wait for it at the barrier: its rows and their sums are NaN.
__device__ __forceinline__ void copy_tile(const CopyOut& c, const unsigned char* tile, uint32_t bar, bool there, bool leader, int warp, int m0,
                                          int m, int k0, int k, int slab, float (&buf)[4][64]) {
  const int lane = static_cast<int>(lane_id()), col = k0 + 2 * lane;
  uint32_t v[32];
#pragma unroll
  for (int i = 0; i < 32; ++i)                   // (row & 7 = i & 7)
    v[i] = there ? *reinterpret_cast<const uint32_t*>(tile + (warp * 32 + i) * 128 + (((lane >> 2) ^ (i & 7)) << 4) + (lane & 3) * 4) : 0x7FC07FC0u;
  float2 sum = make_float2(0.0f, 0.0f);          // (rows and columns behind the last are zeros)
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    sum.x += bf16_lo(v[i]);
    sum.y += bf16_hi(v[i]);
  }
  *reinterpret_cast<float2*>(&buf[warp][2 * lane]) = sum;
  fence_proxy_async();
  __syncwarp();
  if (leader && there) mbar_arrive(bar);
  if (c.out && col < k) {
    float* to = c.out + static_cast<long long>(m0 + warp * 32) * k + col;
    const int rows = m - m0 - warp * 32;
    if (rows >= 32) {
#pragma unroll
      for (int i = 0; i < 32; ++i) *reinterpret_cast<float2*>(to + static_cast<long long>(i) * k) = make_float2(bf16_lo(v[i]), bf16_hi(v[i]));
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i < rows) *reinterpret_cast<float2*>(to + static_cast<long long>(i) * k) = make_float2(bf16_lo(v[i]), bf16_hi(v[i]));
    }
  }
  if (!c.partial && !c.sums) return;
  named_barrier(2, 32 * kCopyWarps);
  const int at = warp * 32 + lane;               // two warps finish the 64 columns
  if (at < 64 && k0 + at < k) {
    const float t = buf[0][at] + buf[1][at] + buf[2][at] + buf[3][at];
    if (c.sums) c.sums[k0 + at] = c.accumulate ? c.sums[k0 + at] + t : t;
    else c.partial[static_cast<long long>(slab) * k + k0 + at] = t;
  }
}

// DT: type of y and of the residual.  An N-major b comes with no bias, activation or residual (the input's gradient); COPY (single
// CTAs only: a pair's second CTA has no barrier that tells it of its tiles) passes a on as CopyOut says, each of its tiles
// by one of the CTAs that read it.
template <int PAIR, int B_MN, int DT, int ACT, int COPY, int EPI>
__global__ void __launch_bounds__(kThreads<COPY, EPI>, 1)
linear_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
              const __grid_constant__ CUtensorMap y_map, const __grid_constant__ CUtensorMap r_map,
              const __grid_constant__ CUtensorMap p_map, const __grid_constant__ TileArgs p) {
  constexpr int kWarps = EPI, kSlots = kWarps / 4, kRow = kCols * (DT ? 2 : 4), kPreRow = kCols * 2;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  __shared__ __align__(8) unsigned long long bars[2 * kMaxStages + 4 + 2 * kWarps + (COPY ? kMaxStages : 0)];
  __shared__ __align__(16) float s_bias[B_MN ? 1 : kWarps][kCols];
  __shared__ float s_slices[B_MN && !COPY ? kSumSlices : 1][32];
  __shared__ __align__(16) float s_copy[COPY ? 2 : 1][4][COPY ? 64 : 1];
  __shared__ uint32_t tmem_slot;

  const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);      // (uniform for the compiler too)
  const uint32_t lane = lane_id();
  const bool leader = elected();
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * kMaxStages, acc_full = full + 16 * kMaxStages, acc_empty = acc_full + 16;
  const uint32_t res_bar = acc_empty + 16;       // two per epilogue warp
  const uint32_t copy_bar = res_bar + 16 * kWarps;              // a stage's tile is there, and to be copied
  const int b_rows = PAIR ? p.tile_n / 2 : p.tile_n;            // columns' operand: rows that this CTA fetches
  const int tile_step = PAIR ? static_cast<int>(gridDim.x >> 1) : static_cast<int>(gridDim.x);
  const int tile_first = PAIR ? static_cast<int>(blockIdx.x >> 1) : static_cast<int>(blockIdx.x);
  const int first_m = tile_first / p.tiles_n, first_n = tile_first - first_m * p.tiles_n;
  constexpr int kTileRows = PAIR ? 2 * kTileM : kTileM;
  // the tile behind (tm, tn)
  const auto advance = [&](int& tm, int& tn) {
    tm += p.step_m;
    tn += p.step_n;
    if (tn >= p.tiles_n) { tn -= p.tiles_n; ++tm; }
  };

  if (PAIR) cluster_sync_all();                  // (both CTAs are there: tmem_alloc_pair)
  if (tid == 0) {
    tma_prefetch_desc(&a_map);
    tma_prefetch_desc(&b_map);
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, COPY ? 1 + kCopyWarps : 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full + 8 * a, 1);
      mbar_init(acc_empty + 8 * a, (PAIR ? 2 : 1) * kWarps);
    }
    for (int w = 0; w < 2 * kWarps; ++w) mbar_init(res_bar + 8 * w, 1);
    if (COPY)
      for (int s = 0; s < p.stages; ++s) mbar_init(copy_bar + 8 * s, 1);
    fence_barrier_init();
  }
  if (warp == 1) {
    if (PAIR) tmem_alloc_pair(smem_u32(&tmem_slot), p.tmem_cols);
    else tmem_alloc(smem_u32(&tmem_slot), p.tmem_cols);
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0 && tid == 0) *p.status = 0u;              // (a wait gives up after seconds, long behind this)

  const auto give_up = [&]() { atomicMax(p.status, static_cast<uint32_t>(SURGEON_ERR_TIMEOUT)); };

  if (warp == 0) {
    // ---- operands ----
    if (leader) {
      int s = 0, tm = first_m, tn = first_n;
      uint32_t phase = 1;                        // (a fresh barrier counts as passed in its phase before)
      bool ok = true, free = true;
      for (int t = tile_first; t < p.tiles && ok; t += tile_step, advance(tm, tn)) {
        const int m0 = tm * kTileRows + static_cast<int>(rank) * kTileM;
        const int n0 = tn * p.tile_n + static_cast<int>(rank) * b_rows;
        for (int kt = 0; kt < p.ktiles; ++kt) {
          if (!free && !mbar_wait_suspend(empty + 8 * s, phase)) { give_up(); ok = false; break; }
          const uint32_t a_at = smem_u32(smem) + s * p.stage_bytes, b_at = a_at + kABytes, bar = full + 8 * s;
          if (rank == 0) mbar_arrive_expect_tx(bar, (PAIR ? 2u : 1u) * static_cast<uint32_t>(p.stage_bytes));
          if (PAIR) tma_load_2d_pair(a_at, &a_map, kt * kTileK, m0, bar);
          else tma_load_2d(a_at, &a_map, kt * kTileK, m0, bar);
          if (B_MN) {
            for (int g = 0; g < b_rows / 64; ++g) {
              if (PAIR) tma_load_2d_pair(b_at + g * (kTileK * 128), &b_map, n0 + g * 64, kt * kTileK, bar);
              else tma_load_2d(b_at + g * (kTileK * 128), &b_map, n0 + g * 64, kt * kTileK, bar);
            }
          } else if (PAIR) {
            tma_load_2d_pair(b_at, &b_map, kt * kTileK, n0, bar);
          } else {
            tma_load_2d(b_at, &b_map, kt * kTileK, n0, bar);
          }
          if (++s == p.stages) { s = 0; phase ^= 1; }
          free = mbar_test(empty + 8 * s, phase);
        }
      }
      if (!ok)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);       // copies in flight land
    }
  } else if (warp == 1) {
    // ---- MMAs ----
    if (leader && rank == 0) {
      const uint32_t idesc = make_idesc(kTileRows, p.tile_n) | (B_MN ? 1u << 16 : 0u);
      const uint64_t a_base = make_desc(smem_u32(smem));
      const uint64_t b_base = B_MN ? make_desc_rows(smem_u32(smem) + kABytes) : make_desc(smem_u32(smem) + kABytes);
      constexpr int kStepB = B_MN ? 128 : 2;
      int s = 0, it = 0, tm = first_m, tn = first_n;
      uint32_t phase = 0;
      bool ok = true, there = false;
      for (int t = tile_first; t < p.tiles && ok; t += tile_step, ++it, advance(tm, tn)) {
        int copied = tn;                         // the next of this tile's steps whose operand tile the copying warps take
        const int acc = it & 1;
        if (!(PAIR ? mbar_wait_suspend_cluster(acc_empty + 8 * acc, ((it >> 1) & 1) ^ 1)
                   : mbar_wait_suspend(acc_empty + 8 * acc, ((it >> 1) & 1) ^ 1))) { give_up(); break; }
        tc_fence_after();
        const uint32_t d = tmem_base + acc * (p.tmem_cols >> 1);
        for (int kt = 0; kt < p.ktiles; ++kt) {
          if (!there && !mbar_wait_suspend(full + 8 * s, phase)) { give_up(); ok = false; break; }
          tc_fence_after();
          if (COPY) {                            // tell them, or give the stage back for them
            if (kt == copied) {
              mbar_arrive(copy_bar + 8 * s);
              copied += p.tiles_n;
            } else {
              mbar_arrive_many(empty + 8 * s, kCopyWarps);
            }
          }
          const uint64_t off = static_cast<uint64_t>((s * p.stage_bytes) >> 4);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            const uint64_t da = a_base + off + 2 * kk, db = b_base + off + kStepB * kk;
            if (PAIR) umma_bf16_pair(d, da, db, idesc, kt > 0 || kk > 0 ? 1u : 0u);
            else umma_bf16(d, da, db, idesc, kt > 0 || kk > 0 ? 1u : 0u);
          }
          const uint32_t done = empty + 8 * s;
          if (++s == p.stages) { s = 0; phase ^= 1; }
          there = mbar_test(full + 8 * s, phase);
          if (PAIR) umma_commit_pair(done);
          else umma_commit(done);
        }
        if (PAIR) umma_commit_pair(acc_full + 8 * acc);
        else umma_commit(acc_full + 8 * acc);
      }
    }
  } else if (COPY && warp >= 2 + kWarps) {
    // ---- operand tiles on to global memory: every tiles_n-th of the row of tiles, from the one that is the tile's column ----
    if constexpr (COPY) {
      int at = 0, tm = first_m, tn = first_n, turn = 0;         // at: the stage of the tile's first step
      uint32_t phases = 0;                       // of each stage's copy_bar
      bool ok = true;
      for (int t = tile_first; t < p.tiles; t += tile_step, advance(tm, tn)) {
        int s = (at + tn) % p.stages;
        for (int kt = tn; kt < p.ktiles; kt += p.tiles_n) {
          if (ok && !__all_sync(0xFFFFFFFFu, mbar_wait_suspend(copy_bar + 8 * s, (phases >> s) & 1))) { give_up(); ok = false; }
          phases ^= 1u << s;
          copy_tile(p.copy, smem + s * p.stage_bytes, empty + 8 * s, ok, leader, warp - 2 - kWarps, tm * kTileRows, p.m, kt * kTileK, p.k, tm,
                    s_copy[turn]);
          turn ^= 1;
          s = (s + p.tiles_n) % p.stages;
        }
        at = (at + p.ktiles) % p.stages;
      }
    }
  } else {
    // ---- epilogue: rows of tensor memory's quarter `warp % 4`, every kSlots-th piece of columns ----
    const int w = warp - 2, quarter = warp & 3, slot = w >> 2;
    const bool has_bias = !B_MN && p.bias, has_res = !B_MN && p.residual, tma_res = has_res && p.vec_y, keep = !B_MN && p.pre;
    // y's places, two of them where a residual comes early, then pre's
    const int y_places = has_res ? 2 : 1;
    unsigned char* stage = smem + p.stages * p.stage_bytes + w * (y_places * kPiece<DT> + (keep ? kPrePiece : 0));
    unsigned char* pre_stage = stage + y_places * kPiece<DT>;
    const uint32_t stage_at = smem_u32(stage), my_res = res_bar + 16 * w;
    const int r = static_cast<int>(lane);        // this lane's row of a piece
    const int row_in_tile = static_cast<int>(rank) * kTileM + quarter * 32;
    // pieces of columns of tile (tm, tn), none where its rows lie behind the last
    const auto pieces_of = [&](int tm, int tn) {
      if (tm * kTileRows + row_in_tile >= p.m) return 0;
      const int left = p.n - tn * p.tile_n;
      return ((left < p.tile_n ? left : p.tile_n) + kCols - 1) / kCols;
    };
    // A warp's first piece of its it-th tile: the slots go round, so that two tiles of two pieces, or of six, keep all warps busy.
    const auto first_of = [&](int it) { return (slot + it * (p.tile_n / kCols)) % kSlots; };
    // the warp's next piece whose residual is to be fetched
    int ft = tile_first, fm = first_m, fn = first_n, fi = 0, fc = slot;
    uint32_t fetched = 0;
    const auto fetch_next = [&]() {              // (the leader)
      while (ft < p.tiles && fc >= pieces_of(fm, fn)) { ft += tile_step; advance(fm, fn); fc = first_of(++fi); }
      if (ft >= p.tiles) return;
      const uint32_t buf = fetched & 1;
      mbar_arrive_expect_tx(my_res + 8 * buf, kPiece<DT>);
      tma_load_2d(stage_at + buf * kPiece<DT>, &r_map, fn * p.tile_n + fc * kCols, fm * kTileRows + row_in_tile, my_res + 8 * buf);
      ++fetched;
      fc += kSlots;
    };
    if constexpr (B_MN && !COPY) {
      if (p.sums.out) add_columns<kWarps>(p.sums, blockIdx.x, gridDim.x, w, s_slices);
    }
    if (tma_res && leader) fetch_next();
    int it = 0, tm = first_m, tn = first_n;
    uint32_t piece = 0;
    bool ok = true;
    for (int t = tile_first; t < p.tiles && ok; t += tile_step, ++it, advance(tm, tn)) {
      const int n0 = tn * p.tile_n, m0 = tm * kTileRows + row_in_tile, pieces = pieces_of(tm, tn);
      const int acc = it & 1;
      const uint32_t tmem_at = tmem_base + acc * (p.tmem_cols >> 1) + (static_cast<uint32_t>(quarter) << 21);
      bool waited = false;
      for (int c = first_of(it); c < pieces; c += kSlots) {
        const uint32_t buf = y_places == 2 ? piece & 1 : 0;
        unsigned char* mine = stage + buf * kPiece<DT>;
        const int x = n0 + c * kCols;
        if (leader) {
          bulk_wait_read<0>();                   // what left the places has been read
          if (tma_res) fetch_next();
        }
        if (has_bias) s_bias[B_MN ? 0 : w][r] = x + r < p.n ? __ldg(p.bias + x + r) : 0.0f;       // the piece's, for every lane to read
        __syncwarp();
        if (has_res && !tma_res) {
          using T = typename Elem<DT>::type;
          copy_piece<T>(static_cast<const T*>(p.residual) + static_cast<long long>(m0) * p.n + x + r, p.n, p.m - m0, x + r < p.n,
                        [&](int q) { return reinterpret_cast<T*>(mine + piece_elem<T>(q, r)); });
          __syncwarp();
        }
        if (!waited) {
          // (all lanes go the same way: behind are instructions of the whole warp)
          if (!__all_sync(0xFFFFFFFFu, mbar_wait_suspend(acc_full + 8 * acc, (it >> 1) & 1))) { give_up(); ok = false; break; }
          tc_fence_after();
          waited = true;
        }
        if (tma_res && !__all_sync(0xFFFFFFFFu, mbar_wait_suspend(my_res + 8 * buf, (piece >> 1) & 1))) {
          give_up();
          ok = false;
          break;
        }
        uint32_t v[kCols];
        tmem_ld32(tmem_at + c * kCols, v);
        tmem_ld_wait();
        if (c + kSlots >= pieces) {              // the accumulator has been read: it may be written again
          tc_fence_before();
          __syncwarp();
          if (leader) {
            if (PAIR) mbar_arrive_rank0(acc_empty + 8 * acc);
            else mbar_arrive(acc_empty + 8 * acc);
          }
        }
#pragma unroll
        for (int j = 0; j < kCols / 8; ++j) {
          float f[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[8 * j + i]);
          if (has_bias) {
            const float4 b0 = *reinterpret_cast<const float4*>(&s_bias[B_MN ? 0 : w][8 * j]), b1 = *reinterpret_cast<const float4*>(&s_bias[B_MN ? 0 : w][8 * j + 4]);
            f[0] += b0.x; f[1] += b0.y; f[2] += b0.z; f[3] += b0.w;
            f[4] += b1.x; f[5] += b1.y; f[6] += b1.z; f[7] += b1.w;
          }
          if (keep)
            *reinterpret_cast<uint4*>(pre_stage + piece_at<kPreRow>(r, j)) =
                make_uint4(to_bf16x2(f[0], f[1]), to_bf16x2(f[2], f[3]), to_bf16x2(f[4], f[5]), to_bf16x2(f[6], f[7]));
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = activate<ACT>(f[i]);
          if constexpr (DT == 1) {
            uint4* at = reinterpret_cast<uint4*>(mine + piece_at<kRow>(r, j));
            if (has_res) {
              const uint4 q = *at;
              f[0] += bf16_lo(q.x); f[1] += bf16_hi(q.x); f[2] += bf16_lo(q.y); f[3] += bf16_hi(q.y);
              f[4] += bf16_lo(q.z); f[5] += bf16_hi(q.z); f[6] += bf16_lo(q.w); f[7] += bf16_hi(q.w);
            }
            *at = make_uint4(to_bf16x2(f[0], f[1]), to_bf16x2(f[2], f[3]), to_bf16x2(f[4], f[5]), to_bf16x2(f[6], f[7]));
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float4* at = reinterpret_cast<float4*>(mine + piece_at<kRow>(r, 2 * j + h));
              if (has_res) {
                const float4 q = *at;
                f[4 * h] += q.x; f[4 * h + 1] += q.y; f[4 * h + 2] += q.z; f[4 * h + 3] += q.w;
              }
              *at = make_float4(f[4 * h], f[4 * h + 1], f[4 * h + 2], f[4 * h + 3]);
            }
          }
        }
        fence_proxy_async();
        __syncwarp();
        if (leader) {
          if (p.vec_y) tma_store_2d(&y_map, stage_at + buf * kPiece<DT>, x, m0);
          if (keep && p.vec_pre) tma_store_2d(&p_map, smem_u32(pre_stage), x, m0);
          bulk_commit();
        }
        if (!p.vec_y || (keep && !p.vec_pre)) {
          using T = typename Elem<DT>::type;
          const long long at = static_cast<long long>(m0) * p.n + x + r;
          if (!p.vec_y)
            copy_out<T>(static_cast<T*>(p.y) + at, p.n, p.m - m0, x + r < p.n,
                        [&](int q) { return *reinterpret_cast<const T*>(mine + piece_elem<T>(q, r)); });
          if (keep && !p.vec_pre)
            copy_out<unsigned short>(p.pre + at, p.n, p.m - m0, x + r < p.n, [&](int q) {
              return *reinterpret_cast<const unsigned short*>(pre_stage + piece_elem<unsigned short>(q, r));
            });
          __syncwarp();                          // before the next piece takes the place
        }
        ++piece;
      }
      if (ok && !waited) {                       // no piece of this tile: pass the accumulator on
        if (!__all_sync(0xFFFFFFFFu, mbar_wait_suspend(acc_full + 8 * acc, (it >> 1) & 1))) { give_up(); ok = false; break; }
        if (leader) {
          if (PAIR) mbar_arrive_rank0(acc_empty + 8 * acc);
          else mbar_arrive(acc_empty + 8 * acc);
        }
      }
    }
    if (leader) {
      if (!ok)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);       // copies in flight land
      bulk_wait_read<0>();                       // the pieces have left shared memory
    }
    __syncwarp();
    if (!ok) {                                   // a wait ran out: all of this warp's part is NaN
      using T = typename Elem<DT>::type;
      it = 0; tm = first_m; tn = first_n;
      for (int t = tile_first; t < p.tiles; t += tile_step, ++it, advance(tm, tn)) {
        const int m0 = tm * kTileRows + row_in_tile, pieces = pieces_of(tm, tn);
        for (int c = first_of(it); c < pieces; c += kSlots) {
          const int x = tn * p.tile_n + c * kCols + r;
          if (x >= p.n) continue;
#pragma unroll 1
          for (int q = m0; q < m0 + 32 && q < p.m; ++q) {
            const long long at = static_cast<long long>(q) * p.n + x;
            static_cast<T*>(p.y)[at] = static_cast<T>(DT ? 0x7FC0u : 0x7FC00000u);
            if (keep) p.pre[at] = 0x7FC0u;
          }
        }
      }
    }
  }
  __syncwarp();                                  // (the roles of one lane end here; the barriers take whole warps)
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    if (PAIR) tmem_dealloc_pair(tmem_base, p.tmem_cols);
    else tmem_dealloc(tmem_base, p.tmem_cols);
  }
}

// ---- few tiles: the reduction is split over the CTAs of a cluster ----
//
// An SM takes in some 100 to 130 GB/s of operands (24 KB per 64 of k in 0.19 us for tiles of 64 columns, 48 KB in 0.50 for 256: the
// steps of choose_tile), so a product of few tiles goes by how many SMs fetch them.  Each CTA
// of a cluster of S sums its share of k for the same tile of 128 x tile_n, puts its sums into its shared memory, and after
// a cluster barrier finishes 128 / S of the rows: the S sums of an element are added in the order of the CTAs' ranks.

constexpr int kSplitThreads = 256;

struct SplitArgs {
  int m, n, k;
  int tile_n, tiles_n;
  int splits, stages, stage_bytes, ktiles;
  int act, dt;
  const float* bias;
  const void* residual;
  void* y;
  unsigned short* pre;
  uint32_t* status;
  ColumnSums sums;
  CopyOut copy;
};

__device__ __forceinline__ float4 load_cluster(uint32_t addr, uint32_t rank) {
  float4 v;
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}

template <int B_MN, int COPY>
__global__ void __launch_bounds__(kSplitThreads)
linear_split_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                    const __grid_constant__ SplitArgs p) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  __shared__ __align__(8) unsigned long long bars[2 * kMaxStages + 1 + (COPY ? kMaxStages : 0)];
  __shared__ float s_slices[B_MN && !COPY ? kSumSlices : 1][32];
  __shared__ __align__(16) float s_copy[COPY ? 2 : 1][4][COPY ? 64 : 1];
  __shared__ uint32_t tmem_slot, s_gave_up;
  const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
  const uint32_t lane = lane_id();
  const bool leader = elected();
  const uint32_t rank = cluster_ctarank();
  const int tile = static_cast<int>(blockIdx.x) / p.splits;
  const int m0 = tile / p.tiles_n * kTileM, n0 = tile % p.tiles_n * p.tile_n;
  const int kt_begin = static_cast<int>(static_cast<long long>(p.ktiles) * rank / p.splits);
  const int kt_end = static_cast<int>(static_cast<long long>(p.ktiles) * (rank + 1) / p.splits);
  const uint32_t full = smem_u32(bars), empty = full + 8 * kMaxStages, acc_full = full + 16 * kMaxStages, copy_bar = acc_full + 8;
  const int tn = tile % p.tiles_n;               // COPY: the steps kt with kt % tiles_n = tn are copied by this tile's CTAs
  if (tid == 0) {
    s_gave_up = 0u;
    tma_prefetch_desc(&a_map);
    tma_prefetch_desc(&b_map);
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, COPY ? 1 + kCopyWarps : 1);
    }
    mbar_init(acc_full, 1);
    if (COPY)
      for (int s = 0; s < p.stages; ++s) mbar_init(copy_bar + 8 * s, 1);
    fence_barrier_init();
  }
  if (warp == 1) tmem_alloc(smem_u32(&tmem_slot), p.tile_n);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0 && tid == 0) *p.status = 0u;              // (a wait gives up after seconds, long behind this)
  const auto give_up = [&]() {
    atomicMax(p.status, static_cast<uint32_t>(SURGEON_ERR_TIMEOUT));
    *static_cast<volatile uint32_t*>(&s_gave_up) = 1u;
  };
  if (warp == 0) {
    if (leader) {
      int s = 0;
      uint32_t phase = 1;
      bool ok = true, free = true;
      for (int kt = kt_begin; kt < kt_end; ++kt) {
        if (!free && !mbar_wait_suspend(empty + 8 * s, phase)) { give_up(); ok = false; break; }
        const uint32_t a_at = smem_u32(smem) + s * p.stage_bytes, b_at = a_at + kABytes, bar = full + 8 * s;
        mbar_arrive_expect_tx(bar, static_cast<uint32_t>(p.stage_bytes));
        tma_load_2d(a_at, &a_map, kt * kTileK, m0, bar);
        if (B_MN) {
          for (int g = 0; g < p.tile_n / 64; ++g) tma_load_2d(b_at + g * (kTileK * 128), &b_map, n0 + g * 64, kt * kTileK, bar);
        } else {
          tma_load_2d(b_at, &b_map, kt * kTileK, n0, bar);
        }
        if (++s == p.stages) { s = 0; phase ^= 1; }
        free = mbar_test(empty + 8 * s, phase);
      }
      if (!ok)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);       // copies in flight land
    }
  } else if (warp == 1) {
    if (leader) {
      const uint32_t idesc = make_idesc(kTileM, p.tile_n) | (B_MN ? 1u << 16 : 0u);
      const uint64_t a_base = make_desc(smem_u32(smem));
      const uint64_t b_base = B_MN ? make_desc_rows(smem_u32(smem) + kABytes) : make_desc(smem_u32(smem) + kABytes);
      constexpr int kStepB = B_MN ? 128 : 2;
      int s = 0;
      uint32_t phase = 0;
      bool there = false;
      for (int kt = kt_begin; kt < kt_end; ++kt) {
        if (!there && !mbar_wait_suspend(full + 8 * s, phase)) { give_up(); break; }
        tc_fence_after();
        if (COPY) {
          if (kt % p.tiles_n == tn) mbar_arrive(copy_bar + 8 * s);
          else mbar_arrive_many(empty + 8 * s, kCopyWarps);
        }
        const uint64_t off = static_cast<uint64_t>((s * p.stage_bytes) >> 4);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          umma_bf16(tmem_base, a_base + off + 2 * kk, b_base + off + kStepB * kk, idesc, kt > kt_begin || kk > 0 ? 1u : 0u);
        const uint32_t done = empty + 8 * s;
        if (++s == p.stages) { s = 0; phase ^= 1; }
        there = mbar_test(full + 8 * s, phase);
        umma_commit(done);
      }
      umma_commit(acc_full);
    }
  }
  if constexpr (COPY) {
    if (warp >= 2 && warp < 2 + kCopyWarps) {
      int turn = 0;
      uint32_t phases = 0;
      bool ok = true;
      for (int kt = kt_begin; kt < kt_end; ++kt) {
        if (kt % p.tiles_n != tn) continue;
        const int s = (kt - kt_begin) % p.stages;
        if (ok && !__all_sync(0xFFFFFFFFu, mbar_wait_suspend(copy_bar + 8 * s, (phases >> s) & 1))) { give_up(); ok = false; }
        phases ^= 1u << s;
        copy_tile(p.copy, smem + s * p.stage_bytes, empty + 8 * s, ok, leader, warp - 2, m0, p.m, kt * kTileK, p.k, tile / p.tiles_n, s_copy[turn]);
        turn ^= 1;
      }
    }
    // (the sums below take the place of the ring, which the copies have read)
    named_barrier(3, kSplitThreads);
  }
  if constexpr (B_MN && !COPY) {
    if (p.sums.out && warp >= 2) add_columns<kSplitThreads / 32 - 2>(p.sums, blockIdx.x, gridDim.x, warp - 2, s_slices);
  }
  __syncwarp();
  // all MMAs of this CTA are done, and with them the ring: the sums take its place, rows of tile_n + 4
  if (!__all_sync(0xFFFFFFFFu, mbar_wait_suspend(acc_full, 0))) give_up();
  tc_fence_after();
  const int pitch = p.tile_n + 4;
  float* sums = reinterpret_cast<float*>(smem);
  {
    const int quarter = warp & 3, row = quarter * 32 + static_cast<int>(lane);
#pragma unroll 1
    for (int c = (warp >> 2) * 16; c < p.tile_n; c += 32) {
      uint32_t v[8], u[8];
      tmem_ld8(tmem_base + (static_cast<uint32_t>(quarter) << 21) + c, v);
      tmem_ld8(tmem_base + (static_cast<uint32_t>(quarter) << 21) + c + 8, u);
      tmem_ld_wait();
      *reinterpret_cast<uint4*>(sums + row * pitch + c) = make_uint4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<uint4*>(sums + row * pitch + c + 4) = make_uint4(v[4], v[5], v[6], v[7]);
      *reinterpret_cast<uint4*>(sums + row * pitch + c + 8) = make_uint4(u[0], u[1], u[2], u[3]);
      *reinterpret_cast<uint4*>(sums + row * pitch + c + 12) = make_uint4(u[4], u[5], u[6], u[7]);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, p.tile_n);
  }
  if (s_gave_up) {                               // a wait ran out: this CTA's share is NaN, and with it the cluster's tile
#pragma unroll 1
    for (int i = tid; i < kTileM * pitch; i += kSplitThreads) sums[i] = __int_as_float(0x7FC00000);
  }
  cluster_sync_all();
  const int rows = kTileM / p.splits, across = p.tile_n / 4;
#pragma unroll 1
  for (int i = tid; i < rows * across; i += kSplitThreads) {
    const int row = static_cast<int>(rank) * rows + i / across, c = i % across * 4;
    const int m = m0 + row, n = n0 + c;
    if (m >= p.m || n >= p.n) continue;
    const uint32_t at = smem_u32(sums + row * pitch + c);
    float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < p.splits; ++k) {
      const float4 q = load_cluster(at, static_cast<uint32_t>(k));
      f[0] += q.x; f[1] += q.y; f[2] += q.z; f[3] += q.w;
    }
    const long long out = static_cast<long long>(m) * p.n + n;
    const bool vec = (p.n & 3) == 0;             // four columns are one aligned vector of every array
    const int left = p.n - n < 4 ? p.n - n : 4;
    if (p.bias) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < left) f[e] += __ldg(p.bias + n + e);
    }
    if (p.pre) {
      if (vec) store_elems<1, 4>(p.pre, out, f);
      else
        for (int e = 0; e < left; ++e) { const float g[1] = {f[e]}; store_elems<1, 1>(p.pre, out + e, g); }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = activate(f[e], p.act);
    if (p.residual) {
      float q[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (vec) {
        if (p.dt) load_elems<1, 4>(p.residual, out, q);
        else load_elems<0, 4>(p.residual, out, q);
      } else {
        for (int e = 0; e < left; ++e) {
          float g[1];
          if (p.dt) load_elems<1, 1>(p.residual, out + e, g);
          else load_elems<0, 1>(p.residual, out + e, g);
          q[e] = g[0];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] += q[e];
    }
    if (vec) {
      if (p.dt) store_elems<1, 4>(p.y, out, f);
      else store_elems<0, 4>(p.y, out, f);
    } else {
      for (int e = 0; e < left; ++e) {
        const float g[1] = {f[e]};
        if (p.dt) store_elems<1, 1>(p.y, out + e, g);
        else store_elems<0, 1>(p.y, out + e, g);
      }
    }
  }
  cluster_sync_all();                            // the others may still read this CTA's sums
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// A row-major matrix [rows][cols], rows `pitch` elements apart, in boxes of box_cols x box_rows.
bool encode(CUtensorMap* map, const void* base, int dt, long long rows, long long cols, long long pitch, int box_rows, int box_cols) {
  const EncodeFn fn = reinterpret_cast<EncodeFn>(tensor_map_encode_fn());
  if (!fn) return false;
  const int size = dt == 0 ? 4 : 2;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(pitch) * size};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t step[2] = {1, 1};
  return fn(map, dt == 0 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims,
            strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            box_cols * size == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Shape {
  int pair, tile_n, splits;                      // splits > 0: the kernel for few tiles
};

// The tile with the shortest estimate, from measured times in us: `step` per 64 of k, while operands arrive from L2 as fast as
// an SM takes them in (the widest tile: while the tensor cores are the bound); `tile` for a tile's epilogue, which runs beside
// the next tile's products; `once` for a launch.  Waves of tiles take the longer of the two each, the last one both.
Shape choose_tile(const Product& p) {
  struct Cost {
    Shape shape;
    double step, tile, once;
  };
  static const Cost all[] = {{{1, 256, 0}, 0.42, 3.0, 2.3}, {{1, 128, 0}, 0.26, 2.0, 2.3}, {{0, 256, 0}, 0.50, 2.3, 1.5},
                             {{0, 192, 0}, 0.40, 2.0, 1.5}, {{0, 128, 0}, 0.28, 1.25, 1.5}, {{0, 64, 0}, 0.19, 0.75, 1.5},
                             {{1, 192, 0}, 0.34, 3.0, 2.3}};
  constexpr int kKMajorOnly = 6;                 // half a tile's columns are no whole slabs of 64
  const int sms = sm_count();
  const int ktiles = (p.k + kTileK - 1) / kTileK;
  const double heavy = p.act == kActGelu ? 1.5 : 1.0;            // a GELU's share of the epilogue
  Shape best = all[2].shape;
  double least = 1e30;
  for (int i = 0; i < static_cast<int>(sizeof(all) / sizeof(all[0])); ++i) {
    const Cost& c = all[i];
    if (p.b_mn && i >= kKMajorOnly) break;
    if (p.copy_a && c.shape.pair) continue;
    const long long rows = c.shape.pair ? 2 * kTileM : kTileM;
    const long long tiles = ((p.m + rows - 1) / rows) * ((p.n + c.shape.tile_n - 1) / c.shape.tile_n);
    const long long at_once = c.shape.pair ? sms / 2 : sms;
    const double waves = static_cast<double>((tiles + at_once - 1) / at_once), loop = ktiles * c.step, tile = c.tile * heavy;
    const double cost = c.once + waves * (loop > tile ? loop : tile) + (loop > tile ? tile : loop);
    if (cost < least) {
      least = cost;
      best = c.shape;
    }
  }
  // Few tiles: the reduction over the CTAs of a cluster, where all clusters run at once (some SMs are left over by clusters
  // of four and eight).  64 x 2048 x 1000: 8.8 us by one CTA per tile, 6.1 by eight.
  for (int tile_n = 64; tile_n <= 128; tile_n *= 2) {
    const long long tiles = ((p.m + kTileM - 1) / kTileM) * static_cast<long long>((p.n + tile_n - 1) / tile_n);
    for (int splits = 2; splits <= 8 && splits <= ktiles && tiles * splits <= sms - 4 * (splits - 2); splits *= 2) {
      const double cost = (ktiles + splits - 1) / splits * (tile_n == 64 ? 0.19 : 0.28) + (tile_n == 64 ? 4.0 : 6.0) + 0.1 * splits;
      if (cost < least) {
        least = cost;
        best = {0, tile_n, splits};
      }
    }
  }
  return best;
}

template <int PAIR, int B_MN, int DT, int ACT, int COPY, int EPI>
cudaError_t launch_as(const Product& p, int tile_n, uint32_t* status, cudaStream_t stream) {
  TileArgs t = {};
  t.m = p.m; t.n = p.n; t.k = p.k;
  t.tile_n = tile_n;
  const int rows = PAIR ? 2 * kTileM : kTileM;
  t.tiles_n = (p.n + tile_n - 1) / tile_n;
  t.tiles = (p.m + rows - 1) / rows * t.tiles_n;
  t.ktiles = (p.k + kTileK - 1) / kTileK;
  const int b_rows = PAIR ? tile_n / 2 : tile_n;
  t.stage_bytes = kABytes + b_rows * 128;
  const int staging = EPI * ((p.residual ? 2 : 1) * kPiece<DT> + (p.pre ? kPrePiece : 0));
  t.stages = (227 * 1024 - 8192 - staging) / t.stage_bytes;       // (8 KB: alignment, and what is not dynamic)
  if (t.stages > kMaxStages) t.stages = kMaxStages;
  t.tmem_cols = 128;                             // two accumulators; an allocation is a power of two
  while (t.tmem_cols < 2 * tile_n) t.tmem_cols *= 2;
  const int size = DT ? 2 : 4;
  t.vec_y = (static_cast<long long>(p.n) * size) % 16 == 0;
  t.vec_pre = p.n % 8 == 0;
  t.bias = p.bias;
  t.residual = p.residual;
  t.y = p.y;
  t.pre = static_cast<unsigned short*>(p.pre);
  t.status = status;
  t.sums = p.sums;
  t.copy = p.copy;
  CUtensorMap maps[5];
  memset(maps, 0, sizeof(maps));
  bool ok = encode(&maps[0], p.a, 1, p.m, p.k, p.lda, kTileM, kTileK);
  ok = ok && (B_MN ? encode(&maps[1], p.b, 1, p.k, p.n, p.ldb, kTileK, 64) : encode(&maps[1], p.b, 1, p.n, p.k, p.ldb, b_rows, kTileK));
  if (t.vec_y) {
    ok = ok && encode(&maps[2], p.y, DT, p.m, p.n, p.n, 32, kCols);
    if (p.residual) ok = ok && encode(&maps[3], p.residual, DT, p.m, p.n, p.n, 32, kCols);
  }
  if (p.pre && t.vec_pre) ok = ok && encode(&maps[4], p.pre, 1, p.m, p.n, p.n, 32, kCols);
  if (!ok) return cudaErrorInvalidValue;
  const int smem = 1024 + t.stages * t.stage_bytes + staging;
  const auto kernel = linear_kernel<PAIR, B_MN, DT, ACT, COPY, EPI>;
  cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), smem);
  if (e != cudaSuccess) return e;
  const int at_once = PAIR ? sm_count() / 2 : sm_count();
  const int groups = t.tiles < at_once ? t.tiles : at_once;
  t.step_m = groups / t.tiles_n;
  t.step_n = groups % t.tiles_n;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(PAIR ? 2 * groups : groups);
  cfg.blockDim = dim3(kThreads<COPY, EPI>);
  cfg.dynamicSmemBytes = static_cast<size_t>(smem);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = PAIR ? 2 : 1;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, kernel, maps[0], maps[1], maps[2], maps[3], maps[4], t);
  note_launches(1);
  return e;
}

template <int B_MN, int COPY>
cudaError_t launch_split(const Product& p, int tile_n, int splits, uint32_t* status, cudaStream_t stream) {
  SplitArgs t = {};
  t.m = p.m; t.n = p.n; t.k = p.k;
  t.tile_n = tile_n;
  t.tiles_n = (p.n + tile_n - 1) / tile_n;
  t.splits = splits;
  t.ktiles = (p.k + kTileK - 1) / kTileK;
  if (splits > t.ktiles) return cudaErrorInvalidValue;           // (a CTA without a share would never be done)
  t.stage_bytes = kABytes + tile_n * 128;
  const int share = (t.ktiles + splits - 1) / splits;
  t.stages = (200 * 1024) / t.stage_bytes;
  if (t.stages > kMaxStages) t.stages = kMaxStages;
  if (t.stages > share) t.stages = share;
  t.act = p.act; t.dt = p.dt;
  t.bias = p.bias; t.residual = p.residual; t.y = p.y;
  t.pre = static_cast<unsigned short*>(p.pre);
  t.status = status;
  t.sums = p.sums;
  t.copy = p.copy;
  CUtensorMap maps[2];
  memset(maps, 0, sizeof(maps));
  bool ok = encode(&maps[0], p.a, 1, p.m, p.k, p.lda, kTileM, kTileK);
  ok = ok && (B_MN ? encode(&maps[1], p.b, 1, p.k, p.n, p.ldb, kTileK, 64) : encode(&maps[1], p.b, 1, p.n, p.k, p.ldb, tile_n, kTileK));
  if (!ok) return cudaErrorInvalidValue;
  int smem = t.stages * t.stage_bytes;
  const int sums = kTileM * (tile_n + 4) * 4;
  smem = 1024 + (smem > sums ? smem : sums);
  const auto kernel = linear_split_kernel<B_MN, COPY>;
  cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), smem);
  if (e != cudaSuccess) return e;
  const int tiles = (p.m + kTileM - 1) / kTileM * t.tiles_n;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles * splits);
  cfg.blockDim = dim3(kSplitThreads);
  cfg.dynamicSmemBytes = static_cast<size_t>(smem);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, kernel, maps[0], maps[1], t);
  note_launches(1);
  return e;
}

}  // namespace

cudaError_t launch_product(const Product& p, uint32_t* status, cudaStream_t stream) {
  const Shape s = choose_tile(p);
  if (s.splits)
    return p.copy_a ? launch_split<1, 1>(p, s.tile_n, s.splits, status, stream)
           : p.b_mn ? launch_split<1, 0>(p, s.tile_n, s.splits, status, stream)
                    : launch_split<0, 0>(p, s.tile_n, s.splits, status, stream);
  if (p.copy_a)
    return p.dt ? launch_as<0, 1, 1, kActNone, 1, 8>(p, s.tile_n, status, stream) : launch_as<0, 1, 0, kActNone, 1, 8>(p, s.tile_n, status, stream);
  // Sixteen epilogue warps where the epilogue counts, eight where their places in shared memory are better a stage of the ring (us, sixteen and
  // eight: 16384 x 256 -> 1024 with GELU 21 and 27, 12608 x 768 -> 2304 36 and 41; 4096 x 1024 -> 1024 with all 18.5 and 15.4, 16384 x
  // 2048 -> 2048 101 and 96; a residual doubles the places: 16384 x 512 -> 512 16.9 and 15.9).  The input's gradient has
  // a light epilogue: 12608 x 768 <- 2304 41.7 and 38.9, with dz and its sums 65 and 57; 65536 x 64 <- 64 the same.
  const bool wide = p.dt == 1 && !p.b_mn && p.k < (p.residual ? 512 : 1024);
#define SURGEON_FORWARD(PAIR, DT, EPI)                                                                     \
  (p.act == kActNone       ? launch_as<PAIR, 0, DT, kActNone, 0, EPI>(p, s.tile_n, status, stream)          \
   : p.act == kActRelu     ? launch_as<PAIR, 0, DT, kActRelu, 0, EPI>(p, s.tile_n, status, stream)          \
                           : launch_as<PAIR, 0, DT, kActGelu, 0, EPI>(p, s.tile_n, status, stream))
#define SURGEON_PRODUCT(PAIR)                                                                              \
  (p.b_mn   ? (p.dt ? launch_as<PAIR, 1, 1, kActNone, 0, 8>(p, s.tile_n, status, stream)                   \
                    : launch_as<PAIR, 1, 0, kActNone, 0, 8>(p, s.tile_n, status, stream))                  \
   : wide   ? SURGEON_FORWARD(PAIR, 1, 16)                                                                 \
   : p.dt   ? SURGEON_FORWARD(PAIR, 1, 8)                                                                  \
            : SURGEON_FORWARD(PAIR, 0, 8))
  return s.pair ? SURGEON_PRODUCT(1) : SURGEON_PRODUCT(0);
#undef SURGEON_FORWARD
#undef SURGEON_PRODUCT
}

}  // namespace surgeon
