// Block attention over the 8-bit cache on tcgen05: the whole pages' part for 9 to 128 query rows per KV head (head size 128).
// The finish kernel of k_attn_kv8.cu adds the tail and merges.
//
// With 64 query rows (block 16, four heads a group) a key takes 32 KFLOP for its 256 bytes: beyond what mma.sync reaches
// while HBM delivers, and close to what the shared memory ports carry. So both products are laid out to read as little of
// it as possible:
//   S^T = K Q^T  M = 128 keys, K straight from the TMA ring as e4m3 (kind::f8f6f4), no conversion. Q is two e4m3 terms,
//                q * 2^k = q1 + q2 with a k for each row, so that its largest element lies in [2^7, 2^8): eight significant
//                bits, as in bf16, or 2^-18 of the row's largest where that is more. Both products go into one accumulator; the
//                row's 2^-k multiplies the score, next to the K scale. (One k for all rows of the block would be 2 to 4 % faster, but
//                then a row's precision depends on the other tokens and heads, and one that is 2^20 larger takes it all.)
//   O^T = V^T P^T  M = 128 columns, N = rows; V converted once to f16 (exact) and P in f16, both "MN-major": the rows of
//                their tiles are keys, as V comes from memory and as P leaves the threads, nothing is transposed.
// One thread holds one key of a tile and all of its rows: the K scale is one factor per thread, and so is the V scale, since
// P' = 2^(s k - r) s_V. The row references r are shared by the tile's 128 keys; they are moved (and O and the sums rescaled)
// only when a P' passes f16's range, which a vote of the tile's four warps finds out, and then to give 2^10 in every row whose
// largest passes 2^15: P' is a normal f16
// number down to 2^-24 of the largest contribution at least. The sums are of the weights 2^(s k - r) themselves, per thread,
// and are added across threads once per segment.
//
// One block per SM. Two groups of four soft-max warps take the tiles in turn, each with its own S, P, V and O buffer, its own
// references and sums: one group's trip through tensor memory, its vote and its waits are covered by the other group's
// exponentials. Four warps turn V from its ring into f16, a warp copies K, one V and the pages' scales, and one each issues
// the MMAs of either product (an MMA costs its issuer some 60 cycles to set up: twelve per tile from one warp held the others
// up). More than 64 rows are two row groups: blocks 2 i and 2 i + 1 walk the same stretch of keys, so the second read of a
// page finds it in L2.
// Measured, with the finish kernel, captured in a graph at 1965 MHz: batch 32 of 512 to 8192 tokens, block 16: 94.7 us (285 MB:
// 3.0 TB/s); 4 x 32K, block 32: 129.6 us; one request of 2048 tokens, block 16: 16.3 us. (Repeated for a second and more the card
// reaches its power limit, the clock falls to 1860 and 1815 MHz and the first two take 100 and 141 us.) A tile of 128 keys takes about
// 2100 cycles, and as many wavefronts of shared memory (1062 of loads and stores, 768 of MMA operands, 256 of copies; V's way
// through f16 is the largest part); a segment costs about six tiles more to begin and end.
// Work is cut as in k_attn_kv8.cu, in tiles of eight pages. Pages behind the end of a segment, and bad ones, are masked.
#include "kv8_common.cuh"
#include "tc_common.cuh"

namespace {

using namespace kv8;
using namespace tc;

constexpr int HD = 128, TILE = 128, TPAGES = TILE / PAGE, NROW = 64;
constexpr int WORKERS = 256, WARPS = WORKERS / 32, CONV = 4, THREADS = 512;
constexpr int WARP_K = WARPS + CONV, WARP_QK = WARP_K + 1, WARP_V = WARP_K + 2;
constexpr int SLOTS = 2;                                   // tiles of K, and of V, on their way
constexpr int PBUF = 4;                                    // tiles of weights: a group begins its next one while the last is multiplied
constexpr uint32_t T_BYTES = TILE * HD;                    // 16 KB: a tile's K, or V, as it comes
constexpr uint32_t V_HALF = TILE * 128, V_BYTES = 2 * V_HALF, P_BYTES = TILE * 128;
constexpr uint32_t OFF_Q = 0;                              // [2 * npad rows][128 bytes]
constexpr uint32_t OFF_K = OFF_Q + 2 * NROW * HD;          // [SLOTS]
constexpr uint32_t OFF_R = OFF_K + SLOTS * T_BYTES;       // [SLOTS] V as it comes
constexpr uint32_t OFF_V = OFF_R + SLOTS * T_BYTES;       // [2][two halves of the columns][128 keys][64 f16]
constexpr uint32_t OFF_P = OFF_V + 2 * V_BYTES;            // [PBUF][128 keys][64 rows f16]
constexpr uint32_t OFF_CTL = OFF_P + PBUF * P_BYTES;
constexpr uint32_t SMEM = OFF_CTL + 4608 + 1024;
constexpr int SBUF = 3;
constexpr uint32_t COL_S = 0, COL_O = SBUF * NROW, TMEM_COLS = 512;   // S [3][64 columns], O [2][64]
// setmaxnreg: the soft-max warps' budget and the others' add up to what the block is launched with (the host checks that)
constexpr int REGS_LAUNCH = 128, REGS_SOFTMAX = 160, REGS_OTHER = 96;
static_assert(WORKERS * REGS_SOFTMAX + (THREADS - WORKERS) * REGS_OTHER <= THREADS * REGS_LAUNCH, "setmaxnreg budgets exceed the block's registers");
__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// The bounded wait of tc_common, asleep until the phase completes (or 10 us have passed) instead of polling: fourteen warps
// that wait would take issue slots from those that work.
__device__ __forceinline__ bool wait_asleep(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t* status) {
  long long t0 = 0;
  for (int i = 0;; ++i) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity), "r"(10000u) : "memory");
    if (ok) return true;
    if (*abort_flag) return false;
    if (i == 0) t0 = clock64();
    else if (clock64() - t0 > WAIT_LIMIT_CYCLES) {
      *abort_flag = 1;
      atomicOr(status, COD_DEV_TIMEOUT);
      return false;
    }
  }
}
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
// the 128 threads of a group agree whether one of them says yes
__device__ __forceinline__ bool vote_group(int grp, bool mine) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r) : "r"(static_cast<uint32_t>(mine)), "r"(1 + grp) : "memory");
  return r != 0;
}
__device__ __forceinline__ void sync_group(int grp) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(1 + grp) : "memory"); }
__device__ __forceinline__ void sync_workers() { asm volatile("barrier.cta.sync 3, 256;" ::: "memory"); }
__device__ __forceinline__ void tmem_ld16_nowait(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr) : "memory");
}
// (the registers pass through it, so that nothing that uses them moves ahead of the wait)
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                 "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]) :: "memory");
}
__device__ __forceinline__ void tmem_ld8_nowait(uint32_t taddr, uint32_t (&v)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
      : "r"(taddr));
}
// (these two order nothing but each other and the barriers' waits: arithmetic and stores of one step may pass the next one's)
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&v)[8]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]));
}
// two floats at a time
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
        "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void unpack_bf16(const float4& four, float* v) {
  const float w[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(__float_as_uint(w[e]) << 16); v[2 * e + 1] = __uint_as_float(__float_as_uint(w[e]) & 0xFFFF0000u); }
}
// column-wise sum over the 32 lanes of a warp for 16 columns: afterwards lane L (and L + 16) holds column L & 15
__device__ __forceinline__ float warp_sum16(float (&e)[16], int lane) {
#pragma unroll
  for (int c = 0; c < 16; ++c) e[c] += __shfl_xor_sync(0xffffffffu, e[c], 16);
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) {
    const bool hi = (lane & off) != 0;
#pragma unroll
    for (int c = 0; c < off; ++c) {
      const float send = hi ? e[c] : e[c + off], mine = hi ? e[c + off] : e[c];
      e[c] = mine + __shfl_xor_sync(0xffffffffu, send, off);
    }
  }
  return e[0];
}
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}

__global__ void __launch_bounds__(THREADS, 1)
k_attn_kv8_tc(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_zero, const Kv8Params p) {
  cod_pdl_prologue();
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const sm = smem_raw + (base - raw);
  uint64_t* const bars = reinterpret_cast<uint64_t*>(sm + OFF_CTL);
  uint64_t* const k_full = bars;              // [SLOTS]  the tile's K has landed
  uint64_t* const k_empty = k_full + SLOTS; // [SLOTS]  its product has been taken
  uint64_t* const v_full = k_empty + SLOTS; // [SLOTS]  the tile's V has landed
  uint64_t* const v_empty = v_full + SLOTS; // [SLOTS]  (4 warps) and has been read
  uint64_t* const s_full = v_empty + SLOTS; // [SBUF]  S of the tile is in tensor memory, its pages' scales in page_s
  uint64_t* const s_free = s_full + SBUF;     // [SBUF]  (4 warps) and is not needed any more
  uint64_t* const p_full = s_free + SBUF;     // [PBUF]  (4 + 4 warps) P and V of the tile are in shared memory
  uint64_t* const o_done = p_full + PBUF;     // [PBUF]  their product has been added to O
  uint64_t* const q_ready = o_done + PBUF;    // (8 warps) Q of the segment is in shared memory
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(q_ready + 1);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* const nr_s = reinterpret_cast<float*>(sm + OFF_CTL + 256);  // [2][64] row references of the groups, negated
  float* const none_s = nr_s + 2 * NROW;                             // [64] -inf: the references that a masked key sees
  float* const f_s = none_s + NROW;                                  // [2][64] factors of a change of reference
  float* const x_s = f_s + 2 * NROW;                                 // [2][4][64] maxima or sums of a group's four key quarters
  float* const q_s = x_s + 8 * NROW;                                 // [64] each row's score factor: 2^-k of its q
  float4* const page_s = reinterpret_cast<float4*>(q_s + NROW);      // [SBUF][8] K scale, V scale, log2 of it; 0, 0, -inf: no page
  int* const scan_s = reinterpret_cast<int*>(page_s + SBUF * TPAGES);       // [THREADS / 32 + 2]
  Segment* const seg_s = reinterpret_cast<Segment*>(scan_s + THREADS / 32 + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int M = p.W * p.rep, groups = (M + NROW - 1) / NROW;
  const int rg = blockIdx.x % groups, row0 = rg * NROW, rows = min(NROW, M - row0);
  const int npad = (rows + 31) / 32 * 32;
  uint32_t flags = 0;

  if (threadIdx.x == 0) {
    for (int i = 0; i < SLOTS; ++i) { mbar_init(smem_u32(k_full + i), 1); mbar_init(smem_u32(k_empty + i), 1); mbar_init(smem_u32(v_full + i), 1); mbar_init(smem_u32(v_empty + i), CONV); }
    for (int i = 0; i < SBUF; ++i) { mbar_init(smem_u32(s_full + i), 2); mbar_init(smem_u32(s_free + i), 4); }
    for (int i = 0; i < PBUF; ++i) {
      mbar_init(smem_u32(p_full + i), 4 + CONV); mbar_init(smem_u32(o_done + i), 1);
    }
    mbar_init(smem_u32(q_ready), WARPS);
    *abort_flag = 0;
    mbar_init_fence();
  }
  Stretch line;
  if (!cut_line<THREADS / 32>(p, TPAGES, blockIdx.x / groups, gridDim.x / groups, blockIdx.x == 0, scan_s, line, flags)) return;
  if (warp == WARP_QK) tmem_alloc(smem_u32(tmem_slot), TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp >= WARPS) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_OTHER));
    if (warp == WARP_K || warp == WARP_V) {
      // ------------------------------------------------ K and V: eight boxes of a page per tile
      const int kv = warp == WARP_K ? 0 : 1;
      const uint64_t pol = l2_evict_first();
      uint64_t* const full = kv ? v_full : k_full;
      uint64_t* const empty = kv ? v_empty : k_empty;
      const uint32_t ring = base + (kv ? OFF_R : OFF_K);
      int n = 0;
      bool ok = true;
      for (Segment k = first_segment(p, line, TPAGES); k.any && ok; next_segment(p, line, TPAGES, k)) {
        const int pages = min(k.L / PAGE, k.u1 * TPAGES);
        const int* table = p.block_table + static_cast<size_t>(k.s) * p.max_pages;
        const float* const scales = p.scale + (static_cast<size_t>(p.layer) * p.n_pages * p.n_kv + k.h) * 2;
        // this lane's page of a tile. No load stands under a condition (its value would be waited for where the branches meet
        // again): indices are clamped, what came is looked at later.
        auto load_id = [&](int t) -> int { return ld_now(table + min(t * TPAGES + (lane & 7), pages - 1)); };
        int next = load_id(k.u0);               // one tile ahead
        for (int t = k.u0; t < k.u1; ++t, ++n) {
          const int pg = next;
          next = load_id(t + 1);
          const bool in = t * TPAGES + (lane & 7) < pages, valid = in && pg >= 0 && pg < p.n_pages;
          if (in && !valid) flags |= COD_DEV_BAD_PAGE;
          const float2 sc = ld_now(reinterpret_cast<const float2*>(scales + static_cast<size_t>(valid ? pg : 0) * p.n_kv * 2));
          // (a page that is not there comes as zeros: finite scores, which the workers mask)
          const int row = valid ? (((p.layer * p.n_pages + pg) * p.n_kv + k.h) * 2 + kv) * PAGE : -1;
          const int slot = n % SLOTS, use = n / SLOTS;
          if (use > 0) ok = __all_sync(0xffffffffu, wait_asleep(smem_u32(empty + slot), (use - 1) & 1, abort_flag, p.status));
          if (!ok) break;
          const uint32_t fb = smem_u32(full + slot), dst = ring + slot * T_BYTES;
          if (elect_one()) mbar_expect_tx(fb, T_BYTES);
          __syncwarp();
#pragma unroll
          for (int i = 0; i < TPAGES; ++i) {
            const int r = __shfl_sync(0xffffffffu, row, i);
            if (elect_one()) tma_page(dst + i * PAGE * HD, r < 0 ? &map_zero : &map_k, max(r, 0), fb, pol);
          }
          if (kv) {                              // the pages' scales, once the tile that had the buffer before is done with it
            const int buf = n % SBUF;
            if (n >= SBUF) ok = __all_sync(0xffffffffu, wait_asleep(smem_u32(s_free + buf), (n / SBUF - 1) & 1, abort_flag, p.status));
            if (!ok) break;
            // (the references see V's scale as no less than 2^-90, so that the weights stay below 2^106 next to a page of zeros)
            if (lane < TPAGES)
              page_s[buf * TPAGES + lane] = valid ? make_float4(sc.x, sc.y, fmaxf(lg2(fmaxf(sc.y, 1.1754944e-38f)), -90.f), 0.f)
                                                  : make_float4(0.f, 0.f, -INFINITY, 0.f);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(s_full + buf));
          }
        }
      }
    } else if (warp < WARP_K) {
      // ------------------------------------------------ V of each tile to f16
      // This thread has columns 8 c .. of both halves (c = lane & 7) of keys vkey + 16 j. The eight lanes of a key store its
      // 128 bytes of one half, all banks at once; the two keys that sixteen lanes read 8 bytes each of lie four rows apart, so
      // that the copy's swizzle puts them on different banks. All reads stand before the stores: the compiler moves none across.
      const int w4 = warp - WARPS;
      const int vkey = (w4 >> 1) * 8 + ((lane >> 3) & 1) * 4 + (lane >> 4) + 2 * (w4 & 1);
      const uint32_t v_src = vkey * HD + ((((lane & 7) >> 1) ^ (vkey & 7)) << 4) + 8 * (lane & 1), v_dst = vkey * 128 + (((lane & 7) ^ (vkey & 7)) << 4);
      int n = 0;
      bool ok = true;
      for (Segment k = first_segment(p, line, TPAGES); k.any && ok; next_segment(p, line, TPAGES, k)) {
        for (int t = k.u0; t < k.u1; ++t, ++n) {
          const int slot = n % SLOTS;
          ok = wait_asleep(smem_u32(v_full + slot), (n / SLOTS) & 1, abort_flag, p.status);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          uint2 v[8][2];
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
              v[j][hf] = *reinterpret_cast<const uint2*>(sm + OFF_R + slot * T_BYTES + (v_src ^ (hf << 6)) + j * 16 * HD);
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(v_empty + slot));
          if (n > 1) ok = wait_asleep(smem_u32(o_done + (n - 2) % PBUF), ((n - 2) / PBUF) & 1, abort_flag, p.status);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              uint4 w;
              e4m3x4_to_f16x4(v[j][hf].x, w.x, w.y);
              e4m3x4_to_f16x4(v[j][hf].y, w.z, w.w);
              *reinterpret_cast<uint4*>(sm + OFF_V + (n & 1) * V_BYTES + hf * V_HALF + v_dst + j * 16 * 128) = w;
            }
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(p_full + n % PBUF));
        }
      }
    } else if (warp == WARP_QK) {
      // ------------------------------------------------ issuer of S^T = K Q^T. The warp stays together; one lane issues
      const uint32_t id_qk = (1u << 4) | (static_cast<uint32_t>(npad >> 3) << 17) | (static_cast<uint32_t>(TILE >> 4) << 24);
      const uint64_t rest = npad * HD >> 4, q_desc = desc_kmajor_sw128(base + OFF_Q), k_desc0 = desc_kmajor_sw128(base + OFF_K);
      int n = 0, seg = 0;
      bool ok = true;
      for (Segment k = first_segment(p, line, TPAGES); k.any && ok; next_segment(p, line, TPAGES, k), ++seg) {
        ok = __all_sync(0xffffffffu, wait_asleep(smem_u32(q_ready), seg & 1, abort_flag, p.status));
        for (int t = k.u0; t < k.u1 && ok; ++t, ++n) {
          const int slot = n % SLOTS, buf = n % SBUF;
          ok = wait_asleep(smem_u32(k_full + slot), (n / SLOTS) & 1, abort_flag, p.status) &&
               (n < SBUF || wait_asleep(smem_u32(s_free + buf), (n / SBUF - 1) & 1, abort_flag, p.status));
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          const uint64_t k_desc = k_desc0 + slot * (T_BYTES >> 4);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < HD / 32; ++kk) umma_e4m3(tmem + COL_S + buf * NROW, k_desc + kk * 2, q_desc + kk * 2, id_qk, kk ? 1u : 0u);
#pragma unroll
            for (int kk = 0; kk < HD / 32; ++kk) umma_e4m3(tmem + COL_S + buf * NROW, k_desc + kk * 2, q_desc + rest + kk * 2, id_qk, 1u);
            umma_commit(smem_u32(s_full + buf));
            umma_commit(smem_u32(k_empty + slot));
          }
          __syncwarp();
        }
      }
    } else {
      // ------------------------------------------------ issuer of O^T = V^T P^T
      const uint32_t id_pv = (1u << 4) | (1u << 15) | (1u << 16) | (static_cast<uint32_t>(npad >> 3) << 17) | (static_cast<uint32_t>(HD >> 4) << 24);
      const uint64_t v_desc0 = desc_mnmajor_sw128(base + OFF_V, V_HALF), p_desc0 = desc_mnmajor_sw128(base + OFF_P, 1024);
      int n = 0;
      bool ok = true;
      for (Segment k = first_segment(p, line, TPAGES); k.any && ok; next_segment(p, line, TPAGES, k)) {
        for (int t = k.u0; t < k.u1; ++t, ++n) {
          ok = __all_sync(0xffffffffu, wait_asleep(smem_u32(p_full + n % PBUF), (n / PBUF) & 1, abort_flag, p.status));
          if (!ok) break;
          tc_fence_after();
          const uint64_t v_desc = v_desc0 + (n & 1) * (V_BYTES >> 4), p_desc = p_desc0 + n % PBUF * (P_BYTES >> 4);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < TILE / 16; ++kk)
              umma_bf16(tmem + COL_O + (n & 1) * NROW, v_desc + kk * (2048 >> 4), p_desc + kk * (2048 >> 4), id_pv, (t > k.u0 + 1 || kk) ? 1u : 0u);
            umma_commit(smem_u32(o_done + n % PBUF));
          }
          __syncwarp();
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SOFTMAX));
    // ------------------------------------------------ soft-max
    // A failed wait lets the loops run on without waiting (every barrier stays matched); what they store is meaningless then
    // and the status word says so.
    const int grp = warp >> 2, key = 32 * (warp & 3) + lane, tid = threadIdx.x;
    const uint32_t t_lane = tmem + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
    const float sl2 = rsqrtf(static_cast<float>(HD)) * 1.4426950408889634f;
    const bool rotate = p.inv_freq != nullptr;
    float* const nr = nr_s + grp * NROW;
    float* const xs = x_s + grp * 4 * NROW;
    float* const fs = f_s + grp * NROW;
    bool ok = true;
    auto wait_done = [&](int m) {                                             // the product of tile m
      if (ok) ok = wait_asleep(smem_u32(o_done + m % PBUF), (m / PBUF) & 1, abort_flag, p.status);
      __syncwarp();
    };
    if (tid < NROW) none_s[tid] = -INFINITY;
    int n = 0;
    for (Segment k = first_segment(p, line, TPAGES); k.any;) {
      const int first = (grp ^ n) & 1;         // this group's first tile of the segment

      // ---- Q of the segment: four threads a row, each 16 columns of both halves (rotary partners)
      {
        const int i0 = row0 / p.rep, nt = (row0 + rows - 1) / p.rep - i0 + 1;            // tokens of this row group
        float* const tab = reinterpret_cast<float*>(sm + OFF_P);                         // no tile's P is on its way
        const int r = tid >> 2, c = tid & 3;
        const int row = row0 + min(r, rows - 1), tok = row / p.rep, hq = k.h * p.rep + row - tok * p.rep;
        const float4* const src = reinterpret_cast<const float4*>(p.q + (static_cast<size_t>(k.s * p.W + tok) * p.n_kv * p.rep + hq) * HD + 16 * c);
        const float4 raw[4] = {ld_now(src), ld_now(src + 1), ld_now(src + HD / 16), ld_now(src + HD / 16 + 1)};   // on their way meanwhile
        if (rotate) {
          for (int e = tid; e < nt * (HD / 2); e += WORKERS) {
            const int i = e / (HD / 2), j = e - i * (HD / 2);
            cod_sincos_at(k.L + i0 + i, p.inv_freq[j], tab[i * HD + HD / 2 + j], tab[i * HD + j]);
          }
          sync_workers();
        }
        float lo[16], hi[16], a = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) { lo[e] = 0.f; hi[e] = 0.f; }
        if (r < rows) {
#pragma unroll
          for (int e = 0; e < 2; ++e) { unpack_bf16(raw[e], lo + 8 * e); unpack_bf16(raw[2 + e], hi + 8 * e); }
          if (rotate) rotate_chunk<16>(lo, hi, tab + (tok - i0) * HD + 16 * c, HD / 2);
#pragma unroll
          for (int e = 0; e < 16; ++e) { lo[e] *= sl2; hi[e] *= sl2; }       // the products are log2-scores
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) a = fmaxf(a, fmaxf(fabsf(lo[e]), fabsf(hi[e])));
        a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
        a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
        // each row scaled by a power of two of its own so that its largest lies in [2^7, 2^8): a row's precision does not depend on
        // the other tokens and heads of the block. A row with an infinity, which e4m3 does not have, gets no score at all.
        int E = static_cast<int>(__float_as_uint(a) >> 23) - 127;
        E = a > 0.f ? max(E, -100) : 7;
        const float up = __uint_as_float(static_cast<uint32_t>(7 - E + 127) << 23);
        if (tid == 0) *seg_s = k;                // not kept in registers through the tiles
        if (c == 0) q_s[r] = a < INFINITY ? __uint_as_float(static_cast<uint32_t>(E - 7 + 127) << 23) : __uint_as_float(0x7FFFFFFFu);
        if (r < npad) {
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            uint32_t w1[4], w2[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              w1[e] = 0u; w2[e] = 0u;
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const float x = (hf ? hi : lo)[4 * e + 2 * u] * up, y = (hf ? hi : lo)[4 * e + 2 * u + 1] * up;
                const uint32_t q1 = __nv_cvt_float2_to_fp8x2(make_float2(x, y), __NV_SATFINITE, __NV_E4M3);
                const float2 back = e4m3x2_to_float2(q1);
                const uint32_t q2 = __nv_cvt_float2_to_fp8x2(make_float2(x - back.x, y - back.y), __NV_SATFINITE, __NV_E4M3);
                w1[e] |= q1 << (16 * u);
                w2[e] |= q2 << (16 * u);
              }
            }
            const uint32_t at = ((hf * 4 + c) ^ (r & 7)) << 4;
            *reinterpret_cast<uint4*>(sm + OFF_Q + r * HD + at) = make_uint4(w1[0], w1[1], w1[2], w1[3]);
            *reinterpret_cast<uint4*>(sm + OFF_Q + (npad + r) * HD + at) = make_uint4(w2[0], w2[1], w2[2], w2[3]);
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(q_ready));
        sync_workers();                        // q_s is set, the table has been read
      }
      float2 l[NROW / 2];
#pragma unroll
      for (int e = 0; e < NROW / 2; ++e) l[e] = make_float2(0.f, 0.f);
      const int tiles = k.u1 - k.u0;

      for (int i = first; i < tiles; i += 2) {
        const int m = n + i;                   // number of the tile; (m & 1) == grp
        const int buf = m % SBUF;
        if (ok) ok = wait_asleep(smem_u32(s_full + buf), (m / SBUF) & 1, abort_flag, p.status);
        __syncwarp();
        tc_fence_after();
        const uint32_t s_at = t_lane + COL_S + buf * NROW;
        const float4 pg = page_s[buf * TPAGES + (key >> 4)];
        const float kf = pg.x, vs = pg.y, lv = pg.z;
        // log2-score of row q, and more; the factor is a power of two, so the score itself is exact and the weights see the same one
        auto score = [&](uint32_t s, int q, float add) { return fmaf(__uint_as_float(s), q_s[q] * kf, add); };
        const float* const ref = lv > -INFINITY ? nr : none_s;               // a masked key: 2^-inf
        const bool starts = i < 2;             // the group's first tile of the segment sets the references
        if (m >= PBUF) wait_done(m - PBUF);    // the product of the weights that had the buffer before
        uint8_t* const prow = sm + OFF_P + m % PBUF * P_BYTES + key * 128;
        // P, eight rows at a time, the scores of the next eight on their way. The largest P' tells whether the references still
        // serve: f16 infinity if not.
        __half2 big = __half2half2(__ushort_as_half(0));
        auto weights = [&]() {
          const float2 k2 = make_float2(kf, kf), v2 = make_float2(vs, vs);
          uint32_t s[2][8];
          float4 r[2][2], f[2][2];
          tmem_ld8_nowait(s_at, s[0]);
          r[0][0] = *reinterpret_cast<const float4*>(ref);
          r[0][1] = *reinterpret_cast<const float4*>(ref + 4);
          f[0][0] = *reinterpret_cast<const float4*>(q_s);
          f[0][1] = *reinterpret_cast<const float4*>(q_s + 4);
#pragma unroll
          for (int c = 0; c < NROW; c += 8) {
            uint32_t (&a)[8] = s[(c >> 3) & 1];
            if (c == NROW / 2 && c >= npad) {  // (rows are padded to 32 or 64)
              tmem_wait_ld(a);                 // what was asked for lands before its registers serve for something else
              break;
            }
            const float4 (&rc)[2] = r[(c >> 3) & 1];
            const float4 (&fc)[2] = f[(c >> 3) & 1];
            float2 u[4] = {make_float2(rc[0].x, rc[0].y), make_float2(rc[0].z, rc[0].w), make_float2(rc[1].x, rc[1].y), make_float2(rc[1].z, rc[1].w)};
            const float2 kq[4] = {mul2(make_float2(fc[0].x, fc[0].y), k2), mul2(make_float2(fc[0].z, fc[0].w), k2),
                                  mul2(make_float2(fc[1].x, fc[1].y), k2), mul2(make_float2(fc[1].z, fc[1].w), k2)};
            tmem_wait_ld(a);
            if (c + 8 < NROW) {
              const int d = c + 8 == NROW / 2 ? min(c + 8, npad - 8) : c + 8;      // (behind the last row: not used)
              tmem_ld8_nowait(s_at + d, s[((c >> 3) + 1) & 1]);
              r[((c >> 3) + 1) & 1][0] = *reinterpret_cast<const float4*>(ref + d);        // (before the stores: the compiler moves no read across one)
              r[((c >> 3) + 1) & 1][1] = *reinterpret_cast<const float4*>(ref + d + 4);
              f[((c >> 3) + 1) & 1][0] = *reinterpret_cast<const float4*>(q_s + d);
              f[((c >> 3) + 1) & 1][1] = *reinterpret_cast<const float4*>(q_s + d + 4);
            }
            uint32_t pk[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              u[e] = fma2(make_float2(__uint_as_float(a[2 * e]), __uint_as_float(a[2 * e + 1])), kq[e], u[e]);
              const float2 w = make_float2(ex2(u[e].x), ex2(u[e].y));
              l[c / 2 + e] = add2(l[c / 2 + e], w);
              const float2 y = mul2(w, v2);
              const __half2 h = __floats2half2_rn(y.x, y.y);
              big = __hmax2(big, h);
              pk[e] = *reinterpret_cast<const uint32_t*>(&h);
            }
            *reinterpret_cast<uint4*>(prow + (((c >> 3) ^ (key & 7)) << 4)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
          }
        };
        // pass 0: with the references as they are (the group's first tile of the segment has none); 1: with new ones
#pragma unroll 1
        for (int pass = starts ? 1 : 0;; pass = 1) {
          if (pass) {
            // some weight times V's scale outgrows f16: new references where they are needed, O and the sums scaled to them (less
            // what this tile has just added; a sum that became infinite starts again from zero: the row's new reference is more
            // than 2^100 above everything that was in it), P again
            if (!starts) {
#pragma unroll
              for (int c = 0; c < NROW; c += 16) {
                if (c >= npad) break;
                uint32_t s[16];
                tmem_ld16_nowait(s_at + c, s);
                tmem_wait_ld(s);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  float& sum = e & 1 ? l[(c + e) / 2].y : l[(c + e) / 2].x;
                  const float before = sum - ex2(score(s[e], c + e, ref[c + e]));
                  sum = fabsf(before) < INFINITY ? before : 0.f;
                }
              }
            }
            // (scores beyond 2^22 leave no room beside them for log2 s_V: there the row's largest score itself is the reference)
            const int q = tid & 127;
            float mx = 0.f, raw = 0.f;
            bool huge = false;
#pragma unroll 1
            for (int kind = 0;; kind = 1) {
              const float add = kind == 0 || lv == -INFINITY ? lv : 0.f;
#pragma unroll 1
              for (int c = 0; c < npad; c += 16) {
                uint32_t s[16];
                tmem_ld16_nowait(s_at + c, s);
                tmem_wait_ld(s);
                float cm = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const float m = warp_max(score(s[e], c + e, add));
                  cm = lane == e ? m : cm;
                }
                if (lane < 16) xs[(warp & 3) * NROW + c + lane] = cm;
              }
              sync_group(grp);
              if (q < npad) {
                raw = fmaxf(fmaxf(xs[q], xs[NROW + q]), fmaxf(xs[2 * NROW + q], xs[3 * NROW + q]));
                if (kind == 0) { mx = raw; huge = fabsf(mx) >= 4194304.f && mx > -INFINITY; }
              }
              if (kind == 1 || !vote_group(grp, huge)) break;
            }
            if (q < npad) {
              const float old = starts ? -INFINITY : -nr[q];
              const bool up = huge ? raw > old : mx - old > 15.f;
              // (a first tile of bad pages alone leaves the row without a reference: the first key that counts overflows, and sets it)
              const float to = !up ? old : huge ? raw : mx - 10.f;
              fs[q] = starts ? 0.f : up ? ex2(old - to) : 1.f;
              nr[q] = -to;
            }
            sync_group(grp);
            if (!starts) {                       // O of these rows (columns), this warp's 32 lanes of it, once it is complete
              wait_done(m - 2);
              tc_fence_after();
#pragma unroll
              for (int c = 0; c < NROW; c += 16) {
                if (c >= npad) break;
#pragma unroll
                for (int e = 0; e < 8; ++e) l[c / 2 + e] = make_float2(l[c / 2 + e].x * fs[c + 2 * e], l[c / 2 + e].y * fs[c + 2 * e + 1]);
                uint32_t o[16];
                tmem_ld16(t_lane + COL_O + grp * NROW + c, o);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * fs[c + e]);
                tmem_st16(t_lane + COL_O + grp * NROW + c, o);
              }
            }
          }
          weights();
          // (a weight itself may be infinite where V's scale is tiny)
          if (pass || !vote_group(grp, __hisinf(__low2half(big)) != 0 || __hisinf(__high2half(big)) != 0)) break;
        }
        fence_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(smem_u32(s_free + buf));
          mbar_arrive(smem_u32(p_full + m % PBUF));
        }
      }

      // ---- the segment's partial: the two groups' outputs on a common reference
      k = *seg_s;
      const bool have_0 = tiles > 1 || (n & 1) == 0, have_1 = tiles > 1 || (n & 1) == 1;
      const bool have = grp ? have_1 : have_0;
      n += tiles;
      if (have) wait_done(((n - 1) & 1) == grp ? n - 1 : n - 2);
      tc_fence_after();
#pragma unroll
      for (int c = 0; c < NROW; c += 16) {
        if (c >= npad) break;
        float w[16];
#pragma unroll
        for (int e = 0; e < 8; ++e) { w[2 * e] = l[c / 2 + e].x; w[2 * e + 1] = l[c / 2 + e].y; }
        const float sum = warp_sum16(w, lane);
        if (lane < 16) xs[(warp & 3) * NROW + c + lane] = sum;
      }
      sync_workers();
      if ((tid & 127) < NROW && tid < 2 * 128) {           // the groups' factors
        const int q = tid & 127;
        const float r0 = have_0 ? -nr_s[q] : -INFINITY, r1 = have_1 ? -nr_s[NROW + q] : -INFINITY;
        const float top = fmaxf(r0, r1);         // -inf: not a key in the whole segment
        fs[q] = top == -INFINITY ? 0.f : ex2((grp ? r1 : r0) - top);
      }
      sync_workers();
      // each group writes half of the rows: it takes the other's contribution from shared memory and leaves there its own to the
      // other half
      float* const obuf = reinterpret_cast<float*>(sm + OFF_P);       // [64 rows][128 columns]
      const int half = npad / 2;
#pragma unroll 1
      for (int c = grp ? 0 : half; c < (grp ? half : npad) && have; c += 16) {
        uint32_t o[16];
        tmem_ld16(t_lane + COL_O + grp * NROW + c, o);
#pragma unroll
        for (int e = 0; e < 16; ++e) obuf[(c + e) * HD + key] = __uint_as_float(o[e]) * fs[c + e];
      }
      sync_workers();
      const size_t slot = static_cast<size_t>(blockIdx.x / groups) + static_cast<size_t>(k.s) * p.n_kv + k.h;
      float* const po = p.part_o + (slot * M + row0) * HD + key;
#pragma unroll 1
      for (int c = grp ? half : 0; c < (grp ? npad : half); c += 16) {
        float y[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = (grp ? have_0 : have_1) ? obuf[(c + e) * HD + key] : 0.f;
        if (have) {
          uint32_t o[16];
          tmem_ld16(t_lane + COL_O + grp * NROW + c, o);
#pragma unroll
          for (int e = 0; e < 16; ++e) y[e] = fmaf(__uint_as_float(o[e]), fs[c + e], y[e]);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (c + e < rows) po[(c + e) * HD] = y[e];
      }
      if (tid < rows) {
        const int q = tid;
        float sum = 0.f, r = -INFINITY;
        if (have_0) {
          sum = ((x_s[q] + x_s[NROW + q]) + (x_s[2 * NROW + q] + x_s[3 * NROW + q])) * f_s[q];
          r = -nr_s[q];
        }
        if (have_1) {
          const float* const y = x_s + 4 * NROW;
          sum += ((y[q] + y[NROW + q]) + (y[2 * NROW + q] + y[3 * NROW + q])) * f_s[NROW + q];
          r = fmaxf(r, -nr_s[NROW + q]);
        }
        *reinterpret_cast<float4*>(p.part_ml + (slot * M + row0 + q) * 4) = make_float4(0.f, r, sum, 0.f);
      }
      tc_fence_before();
      sync_workers();                          // references, sums and the buffer have been read
      next_segment(p, line, TPAGES, k);
    }
  }

  // ---------------------------------------------------- teardown
  if (flags) atomicOr(p.status, flags);
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == WARP_QK) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, TMEM_COLS);
  }
}

}  // namespace

// The register form has one row tile of eight in its MMAs and is nearer to the memory's rate with that (8 rows: 61 against
// 78 us at batch 32, 55 against 66 at 4 x 32K, 14 against 16 for one request); with a second tile it falls behind, be it full or not
// (9 rows: 111 against 80, 94 against 67, equal for one request; 12: 110 against 78, 94 against 66; 16: 113 against 78, 94 against 67;
// 32: 180 against 80, 168 against 68, 20 against 16).
bool cod_attn_kv8_tc_fits(const cod_ctx* c) {
  const int M = c->cfg.block * (c->cfg.n_q_heads / c->cfg.n_kv_heads);
  return c->cfg.head_dim == HD && M > 8 && M <= 2 * NROW;
}

int cod_attn_kv8_tc_unit() { return TPAGES; }
// Beginning a segment (Q, the first references, the partial) takes as long as six tiles. At batch 32, block 16: 150 us without
// it on the line, 120 with 4, 110 with 6 and with 8, 111 with 10.
int cod_attn_kv8_tc_setup() { return 6; }
// groups of query rows, each with blocks of its own that walk the same line
int cod_attn_kv8_tc_groups(const cod_ctx* c) {
  const int M = c->cfg.block * (c->cfg.n_q_heads / c->cfg.n_kv_heads);
  return (M + NROW - 1) / NROW;
}

int cod_launch_attn_kv8_tc(cod_ctx* c, const Kv8Params& p, int blocks, cudaStream_t st) {
  const cod_config& f = c->cfg;
  CUtensorMap map;
  if (!make_map_pages8(&map, p.pool, static_cast<uint64_t>(f.n_layers) * f.n_pages * f.n_kv_heads * 2 * PAGE, HD, PAGE)) return COD_ERR_CUDA;
  CUtensorMap zero;
  if (!make_map_pages8(&zero, c->zero_page, 2 * PAGE, HD, PAGE)) return COD_ERR_CUDA;
  static bool configured_dev[64] = {};          // the attribute belongs to (kernel, device)
  if (!configured_dev[c->device & 63]) {
    cudaFuncAttributes fa;
    if (cudaFuncGetAttributes(&fa, k_attn_kv8_tc) != cudaSuccess) return COD_ERR_CUDA;
    if (fa.numRegs < REGS_LAUNCH) return COD_ERR_UNSUPPORTED;   // the block's registers would not cover the budgets
    if (cudaFuncSetAttribute(k_attn_kv8_tc, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(SMEM)) != cudaSuccess) return COD_ERR_CUDA;
    configured_dev[c->device & 63] = true;
  }
  cod_launch_pdl(c, k_attn_kv8_tc, dim3(blocks), THREADS, SMEM, st, map, zero, p);
  COD_CHECK_LAUNCH(c);
  return COD_OK;
}
