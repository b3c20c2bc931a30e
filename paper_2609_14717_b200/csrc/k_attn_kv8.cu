// Block attention over an 8-bit committed cache, register form: softmax(Q K^T / sqrt(hd)) V over [C_l; U_l; block] with
// C_l in e4m3 pages of 16 tokens, one scale per (page, head, K|V). bf16 contexts, head size 64, or 128 with up to eight query
// rows per KV head; the finish kernel below serves the tcgen05 form, too.
//
// With few query rows per KV head (a token, a short block) the work is the bytes of the cache. Each warp streams its own
// pages through a ring of its own (one TMA box per page: K and V of a head are adjacent), two pages ahead, and no barrier
// ties the warps together in the loop. From shared memory the bytes go into MMA fragments with 16-byte reads and no
// transpose. Both products are computed transposed, S^T = K Q^T and O^T = V^T P^T, so that the 16 rows of mma.m16n8k16 are
// keys resp. columns and the query rows are its 8 columns: a token's 4 or 8 rows fill them, where they would leave half of
// the 16 rows empty. A permutation of the contracted index and of the output columns puts the fragments on contiguous
// bytes (the same permutation on both operands of a product changes nothing). Lane 4 g + t of a warp:
//   K Q^T:   takes, of keys g and g + 8 of the page, bytes [CH t, CH t + CH) of both halves of the row (CH = hd / 8). The
//            k-th MMA contracts over four of those bytes per lane; Q is laid out the same way once. The two halves are the
//            rotary embedding's partners, so rotating q (and block keys) is local to the lane, too.
//   P^T:     leaves the first product as (key g, rows 2t, 2t+1) and is turned by movmatrix into (row g, keys 2t, 2t+1).
//   V^T P^T: takes bytes [CH g, CH g + CH) of V rows 2t, 2t+1, 2t+8, 2t+9; MMA i covers columns CH g + 2i, CH g + 2i + 1,
//            so a lane ends up with CH contiguous columns of two rows of the output.
// Scores are accumulated in float from f16 operands: an e4m3 byte is exact in f16, and q is scaled by a power of two per
// row, after which bf16 q is exact, too (down to 2^-38 of the row's largest). The K scale multiplies the score; the V scale
// enters the weights: with x = log2-scores, w = 2^(x - r) is what the sum takes and P' = w 2^(log2 s_V - d) what multiplies the
// raw V bytes. A row's r, one of its scores, is moved when a score passes it by 60 (the sum is a plain float), its d when P' would
// pass 2^15, and then to give 2^10, so P' is a normal f16 number (11 bits) down to 2^-24 of the largest contribution at least.
// A page of zeros (scale 2^-100) next to pages of large values keeps its share of the sum however far the scales lie apart, and
// as x - r is exact near the largest score and d small, scores of any size lose nothing here but their own rounding.
//
// Work of the paged kernel: the whole pages of all (sequence, KV head) pairs lie one behind the other on a line, which is cut
// into as many equal stretches as blocks fit on the machine at once, whatever the lengths are: one wave, no block waits for
// a longer one, and the cost of starting up (dependent trips to memory for lengths, table, scales and the first copy) is
// paid once per block. At a segment's end the ring already fills with the next segment's pages. The block's four warps share
// the row tiles of the query rows and, between them, the pages; their results are joined in shared memory and leave as one
// unnormalised partial (o; d, r, l, -) per segment. Block i's partial of pair j is slot i + j: along the line each segment
// moves on by a block, a pair or both, so no two meet.
// The finish kernel takes the rest: the rows of the last, partial page, the carried rows and the block's own rows, in bf16
// MMAs, and merges them with the partials.
// Measured, both kernels, captured in a graph: one token for each of 32 requests of 512 to 8192 tokens (285 MB) 57.6 us =
// 4.9 TB/s, where this grid with its rings of boxes and nothing else (every warp only waits for each box and asks for the next)
// takes 52 to 58; one token of one request 10.6 us, three dependent trips to memory in each kernel. The pages' copies leave
// L2 first (evict-first): 4 us more without.
#include "kv8_common.cuh"
#include "tc_common.cuh"

namespace {

using namespace kv8;

constexpr int NW = 4;                        // warps of a block
constexpr int STAGES = 2;                    // pages in flight per warp (three: 2.7 us more for one token at batch 32: more in flight than
                                             // HBM needs only makes the queues longer)

// Offset of byte `col` of row `row` in a box as the copy swizzles it: 16-byte chunks XORed with the row (128-byte rows),
// or with the pair of rows (64-byte rows), so that the reads below meet few bank conflicts.
template <int HD>
__device__ __forceinline__ uint32_t swizzled(int row, int col) {
  return HD == 128 ? row * 128 + (col ^ ((row & 7) << 4)) : row * 64 + (col ^ (((row >> 1) & 3) << 4));
}
template <int N>
__device__ __forceinline__ void lds_row(const uint8_t* p, uint32_t (&w)[N]) {      // N = 4 or 8 words
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const uint4 u = *reinterpret_cast<const uint4*>(p + 4 * i);
    w[i] = u.x; w[i + 1] = u.y; w[i + 2] = u.z; w[i + 3] = u.w;
  }
}
template <int N>
__device__ __forceinline__ void lds_words(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    w[0] = u.x; w[1] = u.y;
  }
}

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// over the lanes that share t (the eight g), resp. over the lanes that share g
__device__ __forceinline__ float max_over_g(float v) {
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float sum_over_g(float v) {
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float max_over_t(float v) {
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
  return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

// Soft-max state of rows 8 n + 2 t + e (n < NR, e < 2) and the lane's share of the output: o[n][i] = (column CH g + 2 i,
// rows e = 0, 1), (column CH g + 2 i + 1, rows e = 0, 1). The lane's own sums l and lc are relative to r, o to r + d (log2 units).
template <int HD, int NR>
struct RowState {
  static constexpr int NT = HD / 16;
  float o[NR][NT][4];
  float r[NR][2], d[NR][2], l[NR][2], lc[NR][2];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][i][e] = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) { r[n][e] = -INFINITY; d[n][e] = -INFINITY; l[n][e] = 0.f; lc[n][e] = 0.f; }
    }
  }
  // Moves the references where one of the warp's scores asks for it; ml: the lane's largest per row, lv: log2 of V's scale.
  __device__ __forceinline__ void refer(const float (&ml)[NR][2], float lv) {
    bool over = false;
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) over = over || ml[n][e] - r[n][e] > 60.f || (ml[n][e] - r[n][e]) + lv - d[n][e] > 15.f;
    if (!__any_sync(0xffffffffu, over)) return;
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float k = max_over_g(ml[n][e]);
        if (k - r[n][e] > 60.f) {
          const float step = r[n][e] - k, f = ex2(step);        // ex2(-inf) = 0 the first time
          r[n][e] = k;
          d[n][e] += step;
          l[n][e] *= f;
          lc[n][e] *= f;
        }
        const float x = (k - r[n][e]) + lv;
        if (x - d[n][e] > 15.f) {
          const float to = x - 10.f, f = ex2(d[n][e] - to);
          d[n][e] = to;
#pragma unroll
          for (int i = 0; i < NT; ++i) { o[n][i][e] *= f; o[n][i][2 + e] *= f; }
        }
      }
  }
  // what turns a weight of the sum into one of raw V bytes (a weight that is not zero is 2^-126 at least: 2^120 passes no P' by)
  __device__ __forceinline__ float factor(int n, int e, float lv) const { return ex2(fminf(lv - d[n][e], 120.f)); }
};

template <int HD, int NR>
__global__ void __launch_bounds__(NW * 32, NR == 1 ? 3 : 2)
k_attn_kv8(const __grid_constant__ CUtensorMap map_pool, const Kv8Params p) {
  cod_pdl_prologue();
  constexpr int CH = HD / 8;                 // bytes of a lane's chunk
  constexpr int CW = CH / 4;                 // its words
  constexpr int KS = HD / 16;                // contraction steps of K Q^T
  constexpr int NT = HD / 16;                // column tiles of V^T P^T
  constexpr int RT = 8 * NR;                 // query rows of a warp's tile
  constexpr uint32_t PGB = 2 * PAGE * HD;    // bytes of a page's K and V of one head
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const sm0 = smem_raw + ((1024u - (tc::smem_u32(smem_raw) & 1023u)) & 1023u);
  // [NW][STAGES][PGB] pages on their way, [NW][RT][HD] floats of the join, the cos | sin table
  float* const join = reinterpret_cast<float*>(sm0 + NW * STAGES * PGB);
  float* const tab = join + NW * RT * HD;
  __shared__ uint64_t bars[NW][STAGES];
  __shared__ float4 ml_s[NW][RT];            // d, r, l, lc
  __shared__ int scan_s[NW + 4];
  __shared__ int abort_s;
  volatile int& abort_flag = abort_s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int M = p.W * p.rep, mtiles = (M + RT - 1) / RT;
  const int mw = mtiles >= 3 ? 4 : mtiles;                  // warps side by side over the row tiles
  const int kg = warp / mw, KG = NW / mw;                   // and over the pages
  uint32_t flags = 0;
  uint64_t* const full = bars[warp];
  const uint8_t* const ring = sm0 + warp * STAGES * PGB;
  const uint32_t ring_u32 = tc::smem_u32(ring);
  if (threadIdx.x == 0) abort_s = 0;
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i) tc::mbar_init(tc::smem_u32(full + i), 1);
    tc::mbar_init_fence();
  }

  Stretch line;
  if (!cut_line<NW>(p, 1, blockIdx.x, gridDim.x, blockIdx.x == 0, scan_s, line, flags)) return;
  Segment cur = first_segment(p, line, 1), nxt;
  int my_pg = -1, nx_pg = -1;                               // pages of the current and of the next batch, one per lane
  float2 my_sc = make_float2(0.f, 0.f);
  int step = 0;                                             // pages this warp has been through: slot and phase of the ring
  bool ok = true;
  const uint64_t pol = l2_evict_first();
  // K and V of a page: one box of 32 rows (page 0, unused, in the place of a bad one) into the slot of page number `n` of this warp
  auto request = [&](int pg, int h, int n) {
    if (lane == 0) {
      const uint32_t bar = tc::smem_u32(full + n % STAGES);
      tc::mbar_expect_tx(bar, PGB);
      tma_page(ring_u32 + n % STAGES * PGB, &map_pool, ((p.layer * p.n_pages + (pg < 0 || pg >= p.n_pages ? 0 : pg)) * p.n_kv + h) * 2 * PAGE, bar, pol);
    }
  };
  // a batch: up to 32 of this warp's pages of a segment, from number b on; their table entries, checked
  auto count_of = [&](const Segment& k, int b) { return k.any ? max(0, min(32, (k.u1 - k.u0 - kg + KG - 1) / KG - b)) : 0; };
  auto load_ids = [&](const Segment& k, int b, int nb) -> int {
    return lane < nb ? p.block_table[static_cast<size_t>(k.s) * p.max_pages + k.u0 + kg + (b + lane) * KG] : -1;
  };
  auto checked = [&](int pg, int nb) -> int {
    if (lane < nb && (pg < 0 || pg >= p.n_pages)) { flags |= COD_DEV_BAD_PAGE; return -1; }
    return pg;
  };
  auto load_scales = [&](int pg, int h) -> float2 {
    return pg < 0 ? make_float2(0.f, 0.f)
                  : __ldg(reinterpret_cast<const float2*>(p.scale + ((static_cast<size_t>(p.layer) * p.n_pages + pg) * p.n_kv + h) * 2));
  };
  const float sl2 = rsqrtf(static_cast<float>(HD)) * 1.4426950408889634f;           // raw score -> log2 units
  const bool rotate = p.inv_freq != nullptr;

  for (int mt0 = 0; mt0 < mtiles; mt0 += mw) {              // (more than one pass only beyond four row tiles)
    const int mt = mt0 + warp % mw;
    if (mt0 > 0) cur = first_segment(p, line, 1);
    int b = 0, nb = count_of(cur, 0), ready = 0;            // current batch; how many of its pages have been asked for
    if (mt >= mtiles) nb = 0;
    my_pg = checked(load_ids(cur, 0, nb), nb);
    for (; ready < min(nb, STAGES); ++ready) request(__shfl_sync(0xffffffffu, my_pg, ready), cur.h, step + ready);
    my_sc = load_scales(my_pg, cur.h);
    int tab_s = -1;
    while (cur.any) {
      if (rotate && tab_s != cur.s) {                       // cos | sin of this sequence's block rows
        __syncthreads();
        const int half = HD / 2;
        for (int e = threadIdx.x; e < p.W * half; e += NW * 32) {
          const int i = e / half, j = e - i * half;
          cod_sincos_at(cur.L + i, p.inv_freq[j], tab[i * HD + half + j], tab[i * HD + j]);
        }
        __syncthreads();
        tab_s = cur.s;
      }
      // the lane's elements of query row 8 n + g: chunk t of both halves of the row, rotated if need be
      auto load_q = [&](int n, float (&qf)[2][CH]) {
        const int row = mt * RT + 8 * n + g;
#pragma unroll
        for (int k = 0; k < CH; ++k) { qf[0][k] = 0.f; qf[1][k] = 0.f; }
        if (row < M) {
          const int i = row / p.rep, hq = cur.h * p.rep + row - i * p.rep;
          const __nv_bfloat16* src = p.q + (static_cast<size_t>(cur.s * p.W + i) * p.n_kv * p.rep + hq) * HD + CH * t;
          load_chunk<CH>(src, qf[0]);
          load_chunk<CH>(src + HD / 2, qf[1]);
          if (rotate) rotate_chunk<CH>(qf[0], qf[1], tab + i * HD + CH * t, HD / 2);
        }
      };
      RowState<HD, NR> st;
      uint32_t qb[NR][KS][2];
      float rowfac[NR][2];
      {
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          float qf[2][CH], a = 0.f;
          load_q(n, qf);
#pragma unroll
          for (int k = 0; k < CH; ++k) a = fmaxf(a, fmaxf(fabsf(qf[0][k]), fabsf(qf[1][k])));
          a = max_over_t(a);                   // f16: scaled so that the row's largest lies in [2^14, 2^15)
          int E = static_cast<int>(__float_as_uint(a) >> 23) - 127;
          E = a > 0.f ? max(E, -100) : 14;
          const float fac = __uint_as_float(static_cast<uint32_t>(E - 14 + 127) << 23) * sl2;
          const float up = __uint_as_float(static_cast<uint32_t>(14 - E + 127) << 23);
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int w = 0; w < CW; ++w)
#pragma unroll
              for (int k = 0; k < 2; ++k) qb[n][hf * CW + w][k] = pack_f16(qf[hf][4 * w + 2 * k] * up, qf[hf][4 * w + 2 * k + 1] * up);
#pragma unroll
          for (int e = 0; e < 2; ++e) rowfac[n][e] = __shfl_sync(0xffffffffu, fac, 4 * (2 * t + e));   // of row 8 n + 2 t + e
        }
      }

      st.clear();

      // ------------------------------------------------------------------ whole pages, batch by batch
      bool more = true;
      while (more && ok) {
        // the batch after this one: of the same segment, or the first of the next
        nxt = cur;
        const int left = mt < mtiles ? (cur.u1 - cur.u0 - kg + KG - 1) / KG - (b + nb) : 0;
        more = left > 0;
        int nx_b = more ? b + nb : 0;
        if (!more) next_segment(p, line, 1, nxt);
        const int nx_nb = mt < mtiles ? count_of(nxt, nx_b) : 0;
        nx_pg = load_ids(nxt, nx_b, nx_nb);
        int nx_ready = 0;
        for (int i = 0; i < nb; ++i) {
          const int slot = (step + i) % STAGES;
          ok = __all_sync(0xffffffffu, ok && tc::mbar_wait(tc::smem_u32(full + slot), ((step + i) / STAGES) & 1, &abort_flag, p.status));
          if (!ok) break;
          const uint8_t* pk = ring + slot * PGB;
          const bool bad = __shfl_sync(0xffffffffu, my_pg, i) < 0;
          const float2 sc = make_float2(__shfl_sync(0xffffffffu, my_sc.x, i), __shfl_sync(0xffffffffu, my_sc.y, i));
          uint32_t kr[2][2][CW], vr[4][CW];    // raw bytes: K [key g | g + 8][half], V [key 2t | 2t+1 | 2t+8 | 2t+9]
#pragma unroll
          for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int e = 0; e < 2; ++e) lds_words<CW>(pk + swizzled<HD>(g + 8 * a, CH * t + e * (HD / 2)), kr[a][e]);
#pragma unroll
          for (int a = 0; a < 4; ++a) lds_words<CW>(pk + PAGE * HD + swizzled<HD>(2 * t + (a >> 1) * 8 + (a & 1), CH * g), vr[a]);
          __syncwarp();                        // the slot has been read by every lane: it may be filled again
          if (i + STAGES < nb) {
            request(__shfl_sync(0xffffffffu, my_pg, i + STAGES), cur.h, step + i + STAGES);
          } else {                             // pages up to number i + STAGES have a free slot: the next batch's follow this one's
            for (; nx_ready < nx_nb && nb + nx_ready <= i + STAGES; ++nx_ready)
              request(__shfl_sync(0xffffffffu, nx_pg, nx_ready), nxt.h, step + nb + nx_ready);
          }
          if (bad) continue;                   // its keys do not count (all lanes agree)
          float sv[NR][4], sw[NR][4];          // two chains of dependent MMAs
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) { sv[n][e] = 0.f; sw[n][e] = 0.f; }
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int w = 0; w < CW; ++w) {
              uint32_t a[4];
              e4m3x4_to_f16x4(kr[0][hf][w], a[0], a[2]);
              e4m3x4_to_f16x4(kr[1][hf][w], a[1], a[3]);
#pragma unroll
              for (int n = 0; n < NR; ++n) mma_f16(w & 1 ? sw[n] : sv[n], a[0], a[1], a[2], a[3], qb[n][hf * CW + w][0], qb[n][hf * CW + w][1]);
            }
          const float lv = lg2(fmaxf(sc.y, 1.1754944e-38f));
          float ml[NR][2];
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float f = rowfac[n][e] * sc.x;
              sv[n][e] = (sv[n][e] + sw[n][e]) * f;
              sv[n][2 + e] = (sv[n][2 + e] + sw[n][2 + e]) * f;
              ml[n][e] = fmaxf(sv[n][e], sv[n][2 + e]);
            }
          st.refer(ml, lv);
          uint32_t pb[NR][2];
#pragma unroll
          for (int n = 0; n < NR; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sv[n][e] = ex2(sv[n][e] - st.r[n][e & 1]);
#pragma unroll
            for (int e = 0; e < 2; ++e) st.l[n][e] += sv[n][e] + sv[n][2 + e];
            const float f0 = st.factor(n, 0, lv), f1 = st.factor(n, 1, lv);
            pb[n][0] = transpose8x8(pack_f16(sv[n][0] * f0, sv[n][1] * f1));
            pb[n][1] = transpose8x8(pack_f16(sv[n][2] * f0, sv[n][3] * f1));
          }
#pragma unroll
          for (int w = 0; w < CW; ++w) {
            // bytes of two keys interleaved: (a0 b0 a1 b1), (a2 b2 a3 b3)
            uint32_t a[4];
            e4m3x4_to_f16x4(__byte_perm(vr[0][w], vr[1][w], 0x5140), a[0], a[1]);
            e4m3x4_to_f16x4(__byte_perm(vr[2][w], vr[3][w], 0x5140), a[2], a[3]);
#pragma unroll
            for (int n = 0; n < NR; ++n) mma_f16(st.o[n][2 * w], a[0], a[1], a[2], a[3], pb[n][0], pb[n][1]);
            e4m3x4_to_f16x4(__byte_perm(vr[0][w], vr[1][w], 0x7362), a[0], a[1]);
            e4m3x4_to_f16x4(__byte_perm(vr[2][w], vr[3][w], 0x7362), a[2], a[3]);
#pragma unroll
            for (int n = 0; n < NR; ++n) mma_f16(st.o[n][2 * w + 1], a[0], a[1], a[2], a[3], pb[n][0], pb[n][1]);
          }
        }
        if (!ok) break;
        step += nb;
        my_pg = checked(nx_pg, nx_nb);
        for (; nx_ready < min(nx_nb, STAGES); ++nx_ready) request(__shfl_sync(0xffffffffu, my_pg, nx_ready), nxt.h, step + nx_ready);
        my_sc = load_scales(my_pg, nxt.h);
        b = nx_b;
        nb = nx_nb;
      }
      ok = !__syncthreads_or(!ok);                          // one warp's failure ends the block
      if (!ok) break;

#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) st.l[n][e] = sum_over_g(st.l[n][e]);

      // this warp's rows: alone straight to the partial, else joined with the warps that shared the segment's keys
      const size_t slot = static_cast<size_t>(blockIdx.x) + static_cast<size_t>(cur.s) * p.n_kv + cur.h;
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int lr = 8 * n + 2 * t + e, row = mt * RT + lr;
          const float4 ml = make_float4(st.d[n][e], st.r[n][e], st.l[n][e], st.lc[n][e]);
          float* dst = KG > 1 ? join + (warp * RT + lr) * HD + CH * g : p.part_o + (slot * M + row) * HD + CH * g;
          if (KG == 1 && row >= M) continue;
#pragma unroll
          for (int i = 0; i < NT; i += 2)
            *reinterpret_cast<float4*>(dst + 2 * i) = make_float4(st.o[n][i][e], st.o[n][i][2 + e], st.o[n][i + 1][e], st.o[n][i + 1][2 + e]);
          if (g == 0) {
            if (KG > 1) ml_s[warp][lr] = ml;
            else *reinterpret_cast<float4*>(p.part_ml + (slot * M + row) * 4) = ml;
          }
        }
      if (KG > 1) {
        __syncthreads();
        for (int idx = threadIdx.x; idx < mw * RT * (HD / 4); idx += NW * 32) {
          const int tile = idx / (RT * (HD / 4)), rem = idx - tile * RT * (HD / 4), r = rem / (HD / 4), d4 = (rem - r * (HD / 4)) * 4;
          const int row = (mt0 + tile) * RT + r;
          if (row >= M) continue;
          float lg = -INFINITY, mg = -INFINITY;
          for (int k = 0; k < KG; ++k) lg = fmaxf(lg, ml_s[k * mw + tile][r].y);
          const float lb = lg == -INFINITY ? 0.f : lg;
          for (int k = 0; k < KG; ++k) mg = fmaxf(mg, ml_s[k * mw + tile][r].y - lb + ml_s[k * mw + tile][r].x);
          const float mb = mg == -INFINITY ? 0.f : mg;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          float l = 0.f, lc = 0.f;
          for (int k = 0; k < KG; ++k) {
            const int w = k * mw + tile;
            const float4 ml = ml_s[w][r];
            const float fl = ex2(ml.y - lb), f = ex2(ml.y - lb + ml.x - mb);
            const float4 v = *reinterpret_cast<const float4*>(join + (w * RT + r) * HD + d4);
            acc.x = fmaf(f, v.x, acc.x); acc.y = fmaf(f, v.y, acc.y); acc.z = fmaf(f, v.z, acc.z); acc.w = fmaf(f, v.w, acc.w);
            l = fmaf(fl, ml.z, l);
            lc = fmaf(fl, ml.w, lc);
          }
          *reinterpret_cast<float4*>(p.part_o + (slot * M + row) * HD + d4) = acc;
          if (d4 == 0) *reinterpret_cast<float4*>(p.part_ml + (slot * M + row) * 4) = make_float4(mg, lg, l, lc);
        }
        // (the next segment's join writes come after the block-wide vote that ends its pages)
      }
      cur = nxt;
    }
    if (!ok) break;
  }
  if (flags) atomicOr(p.status, flags);
  if (abort_flag)                                          // a copy did not come: let what is in flight land
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
}

// The tail of one (sequence, KV head) and the merge with the whole pages' partials: one block for `tpb` tiles of eight query
// rows (all of them where the batch fills the machine), eight warps over the tiles and, where there are fewer, over the
// tail's keys. ROWS rows and PARTS partials are merged at a time by a warp: one row of many parts, or four rows of few. The keys come into shared memory once
// per block, as bf16, with all loads in flight at once (what bounds this kernel is its chain of dependent trips to memory).
// All of that needs only what was there before the paged kernel, so it runs ahead of the wait for that kernel, on whatever
// SMs its last blocks leave free.
// Keys and values are bf16 (a block's keys are rounded to it after their rotation); q and the weights enter as two bf16 terms
// each, so that of a short context no more is lost than the keys' and the output's rounding (one term each: 0.0026 relative
// instead of 0.0020, where rounding the output alone is 0.0017; 1 us at batch 32, block 16). The 128-wide forms spill 8 to 16
// bytes at the 128 registers that two blocks per SM leave.
constexpr int FW = 8, FKEYS = 64;              // warps; keys staged at a time
__device__ __forceinline__ uint32_t rest_bf16(float x, float y, uint32_t hi) {      // what packing x and y into `hi` left
  return pack_bf16(x - __uint_as_float(hi << 16), y - __uint_as_float(hi & 0xFFFF0000u));
}

template <int HD, int ROWS, int PARTS>
__global__ void __launch_bounds__(FW * 32, 2)
k_attn_kv8_finish(const Kv8Params p, int tpb, __nv_bfloat16* __restrict__ out, float* __restrict__ tap, float* __restrict__ mass) {
  if (!p.run_ahead) cod_pdl_prologue();
  constexpr int CH = HD / 8, CW = CH / 4, KS = HD / 16, NT = HD / 16;
  constexpr int KROW = HD * 2 + 16;          // bytes of a staged row (the pad spreads a fragment's rows over the banks)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int h = blockIdx.x, s = blockIdx.y, M = p.W * p.rep, row0 = blockIdx.z * tpb * 8;
  const int rows = min(M - row0, tpb * 8), mtiles = (rows + 7) / 8;          // this block's
  const int MT = mtiles > 4 ? 8 : mtiles > 2 ? 4 : mtiles, KG = FW / MT;      // warps over the row tiles, and over the keys
  const int jrows = max(FW, mtiles) * 8;
  extern __shared__ uint8_t smf[];
  float* const join = reinterpret_cast<float*>(smf);                          // [jrows][HD]: row tile mt of key group kg at mt + MT kg
  uint8_t* const stage = smf + static_cast<size_t>(jrows) * HD * sizeof(float);   // [2][FKEYS][KROW]
  float* const tab = reinterpret_cast<float*>(stage + 2 * FKEYS * KROW);      // cos | sin of the block rows
  __shared__ float4 ml_s[16 * 8];            // [jrows] d, r, l, lc
  __shared__ float4 row_s[128];              // per row: o's reference against the sum's, factor of o, share of the carried keys, the sum's reference
  __shared__ int place_s[2 * FW];
  uint32_t flags = 0;
  const int L = clamped_len(p, s), Lr = L % PAGE;
  int c = p.use_carry ? p.carry_len[s] : 0;
  if (c < 0 || c > p.cap) { flags |= COD_DEV_BAD_LEN; c = max(0, min(c, p.cap)); }
  const int n_tail = Lr + c + p.W;
  size_t u_last = 0;                         // the partial page's K of this head
  bool have_last = false;                    // false with Lr > 0: a bad page, its keys do not count
  float2 sc = make_float2(0.f, 0.f);
  if (Lr > 0) {
    const int pg = p.block_table[static_cast<size_t>(s) * p.max_pages + L / PAGE];
    if (pg < 0 || pg >= p.n_pages) flags |= COD_DEV_BAD_PAGE;
    else {
      have_last = true;
      u_last = ((static_cast<size_t>(p.layer) * p.n_pages + pg) * p.n_kv + h) * 2;
      sc = *reinterpret_cast<const float2*>(p.scale + u_last);
    }
  }
  const bool rotate = p.inv_freq != nullptr;
  if (rotate) {
    const int half = HD / 2;
    for (int e = threadIdx.x; e < p.W * half; e += FW * 32) {
      const int i = e / half, j = e - i * half;
      cod_sincos_at(L + i, p.inv_freq[j], tab[i * HD + half + j], tab[i * HD + j]);
    }
    __syncthreads();
  }
  const float sl2 = rsqrtf(static_cast<float>(HD)) * 1.4426950408889634f;     // raw score -> log2 units

  for (int mt0 = 0; mt0 < mtiles; mt0 += MT) {
    const int mt = mt0 + warp % MT, kg = warp / MT;
    RowState<HD, 1> st;
    st.clear();
    uint32_t qb[KS][2], qc[KS][2];           // q, and what its rounding to bf16 leaves
    {
      const int row = row0 + mt * 8 + g;
      float qf[2][CH];
#pragma unroll
      for (int k = 0; k < CH; ++k) { qf[0][k] = 0.f; qf[1][k] = 0.f; }
      if (mt < mtiles && row < M) {
        const int i = row / p.rep, hq = h * p.rep + row - i * p.rep;
        const __nv_bfloat16* src = p.q + (static_cast<size_t>(s * p.W + i) * p.n_kv * p.rep + hq) * HD + CH * t;
        load_chunk<CH>(src, qf[0]);
        load_chunk<CH>(src + HD / 2, qf[1]);
        if (rotate) rotate_chunk<CH>(qf[0], qf[1], tab + i * HD + CH * t, HD / 2);
      }
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int w = 0; w < CW; ++w)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float x = qf[hf][4 * w + 2 * k], y = qf[hf][4 * w + 2 * k + 1];
            qb[hf * CW + w][k] = pack_bf16(x, y);
            qc[hf * CW + w][k] = rest_bf16(x, y, qb[hf * CW + w][k]);
          }
    }
    for (int f0 = 0; f0 < n_tail; f0 += FKEYS) {
      const int nf = min(FKEYS, n_tail - f0), nf16 = (nf + 15) & ~15;
      if (f0 > 0 || mt0 > 0) __syncthreads();                // the chunk before has been read
      if (mt0 == 0 || n_tail > FKEYS) {
        constexpr int CPR = HD / 16;                         // pieces of eight columns of the lower half, with their partners
        for (int e = threadIdx.x; e < nf16 * 2 * CPR; e += FW * 32) {
          const int col = (e % CPR) * 8, zz = e / CPR % nf16, kv = e / CPR / nf16, z = f0 + zz;
          float lo[8], hi[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) { lo[k] = 0.f; hi[k] = 0.f; }
          if (z < Lr) {
            if (have_last) {
              const uint8_t* src = p.pool + ((u_last + kv) * PAGE + z) * HD + col;
              const float f = kv ? sc.y : sc.x;
              load_bytes<8>(src, f, lo);
              load_bytes<8>(src + HD / 2, f, hi);
            }
          } else if (z < n_tail) {
            const bool blk = z >= Lr + c;
            const int i = blk ? z - Lr - c : z - Lr;
            const __nv_bfloat16* src = blk ? (kv ? p.vb : p.kb) + (static_cast<size_t>(s * p.W + i) * p.n_kv + h) * HD + col
                                           : p.carry + ((((static_cast<size_t>(p.layer) * p.max_batch + s) * p.n_kv + h) * 2 + kv) * p.cap + i) * HD + col;
            load_chunk<8>(src, lo);
            load_chunk<8>(src + HD / 2, hi);
            if (blk && !kv && rotate) rotate_chunk<8>(lo, hi, tab + i * HD + col, HD / 2);
          }
          uint8_t* const dst = stage + (kv * FKEYS + zz) * KROW + col * 2;
          *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(lo[4], lo[5]), pack_bf16(lo[6], lo[7]));
          *reinterpret_cast<uint4*>(dst + HD) = make_uint4(pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3]), pack_bf16(hi[4], hi[5]), pack_bf16(hi[6], hi[7]));
        }
      }
      __syncthreads();
      if (mt < mtiles) {
        for (int z0 = kg * 16; z0 < nf; z0 += KG * 16) {
          float sv[1][4], ml[1][2];
#pragma unroll
          for (int e = 0; e < 4; ++e) sv[0][e] = 0.f;
          const uint8_t* const k0 = stage + (z0 + g) * KROW + CH * t * 2;
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            uint32_t a0[CW * 2], a1[CW * 2];                 // word 2w: columns 4w, 4w + 1; word 2w + 1: 4w + 2, 4w + 3
            lds_row<CW * 2>(k0 + hf * HD, a0);
            lds_row<CW * 2>(k0 + 8 * KROW + hf * HD, a1);
#pragma unroll
            for (int w = 0; w < CW; ++w)
              mma_bf16(sv[0], a0[2 * w], a1[2 * w], a0[2 * w + 1], a1[2 * w + 1], qb[hf * CW + w][0], qb[hf * CW + w][1]);
            if (rotate)                        // (q that comes rotated is bf16)
#pragma unroll
              for (int w = 0; w < CW; ++w)
                mma_bf16(sv[0], a0[2 * w], a1[2 * w], a0[2 * w + 1], a1[2 * w + 1], qc[hf * CW + w][0], qc[hf * CW + w][1]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {        // (the tail's first 16 keys hold one that counts: Lr < 16, and the block's own follow)
            const int zz = z0 + g + (e >> 1) * 8;
            sv[0][e] = zz < nf && (have_last || f0 + zz >= Lr) ? sv[0][e] * sl2 : -INFINITY;
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) ml[0][e] = fmaxf(sv[0][e], sv[0][2 + e]);
          st.refer(ml, 0.f);
          const float g0 = st.factor(0, 0, 0.f), g1 = st.factor(0, 1, 0.f);
          uint32_t pb[2], pc[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {                      // key z0 + g + 8 k, rows 2 t and 2 t + 1
            const int z = f0 + z0 + g + 8 * k;
            const float w[2] = {ex2(sv[0][2 * k] - st.r[0][0]), ex2(sv[0][2 * k + 1] - st.r[0][1])};
            const float x = w[0] * g0, y = w[1] * g1;
            const uint32_t hi = pack_bf16(x, y);
            pb[k] = transpose8x8(hi);
            pc[k] = transpose8x8(rest_bf16(x, y, hi));
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              st.l[0][e] += w[e];
              if (z >= Lr && z < Lr + c) st.lc[0][e] += w[e];
            }
          }
          const uint8_t* const v0 = stage + (FKEYS + z0 + 2 * t) * KROW + CH * g * 2;
          uint32_t va[4][NT];
#pragma unroll
          for (int a = 0; a < 4; ++a) lds_row<NT>(v0 + ((a >> 1) * 8 + (a & 1)) * KROW, va[a]);
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            const uint32_t v0 = __byte_perm(va[0][i], va[1][i], 0x5410), v1 = __byte_perm(va[0][i], va[1][i], 0x7632);
            const uint32_t v2 = __byte_perm(va[2][i], va[3][i], 0x5410), v3 = __byte_perm(va[2][i], va[3][i], 0x7632);
            mma_bf16(st.o[0][i], v0, v1, v2, v3, pb[0], pb[1]);
            mma_bf16(st.o[0][i], v0, v1, v2, v3, pc[0], pc[1]);
          }
        }
      }
    }
    if (mt < mtiles) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int at = (mt + MT * kg) * 8 + 2 * t + e;
        const float l = sum_over_g(st.l[0][e]), lc = sum_over_g(st.lc[0][e]);
        float* dst = join + at * HD + CH * g;
#pragma unroll
        for (int i = 0; i < NT; i += 2)
          *reinterpret_cast<float4*>(dst + 2 * i) = make_float4(st.o[0][i][e], st.o[0][i][2 + e], st.o[0][i + 1][e], st.o[0][i + 1][2 + e]);
        if (g == 0) ml_s[at] = make_float4(st.d[0][e], st.r[0][e], l, lc);
      }
    }
  }
  if (flags) atomicOr(p.status, flags);
  // the partials of this pair: those of the blocks whose stretches hold some of its pages
  int n_parts = 0;
  size_t first_part = 0;
  {
    int base, per;
    place_of<FW>(p, s, place_s, base, per);              // (its barrier also publishes the tail's partials)
    if (L >= PAGE) {
      const int units = units_of(p, L, p.unit), P0 = base + h * units, first = (P0 + p.setup) / per;
      n_parts = (P0 + units - 1) / per - first + 1;
      first_part = static_cast<size_t>(first) + static_cast<size_t>(s) * p.n_kv + h;
    }
  }
  if (p.run_ahead) cod_pdl_prologue();

  // ---- merge, references and sums: eight lanes a row, each with one key group of the tail and parts lane, lane + 8, ...
  const float4* const recs = reinterpret_cast<const float4*>(p.part_ml) + first_part * M + row0;
  for (int r0 = warp * 4; r0 < rows; r0 += FW * 4) {
    const int r = r0 + (lane >> 3), k0 = lane & 7;
    const bool there = r < rows;
    const float4 none = make_float4(-INFINITY, -INFINITY, 0.f, 0.f);
    const float4 own = there && k0 < KG ? ml_s[((r >> 3) + MT * k0) * 8 + (r & 7)] : none;
    float lg = own.y;
    for (int k = k0; there && k < n_parts; k += 8) lg = fmaxf(lg, recs[static_cast<size_t>(k) * M + r].y);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) lg = fmaxf(lg, __shfl_xor_sync(0xffffffffu, lg, o));
    const float lb = lg == -INFINITY ? 0.f : lg, wl = ex2(own.y - lb);
    float l = own.z * wl, lc = own.w * wl, mg = own.y - lb + own.x;
    for (int k = k0; there && k < n_parts; k += 8) {
      const float4 ml = recs[static_cast<size_t>(k) * M + r];
      l = fmaf(ex2(ml.y - lb), ml.z, l);
      mg = fmaxf(mg, ml.y - lb + ml.x);
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
      l += __shfl_xor_sync(0xffffffffu, l, o);
      lc += __shfl_xor_sync(0xffffffffu, lc, o);
      mg = fmaxf(mg, __shfl_xor_sync(0xffffffffu, mg, o));
    }
    const float mb = mg == -INFINITY ? 0.f : mg, inv_l = 1.f / l, half = ex2(0.5f * mb);     // (2^mb alone may pass float's range)
    if (there && k0 == 0) row_s[r] = make_float4(mb, inv_l * half * half, lc * inv_l, lb);
  }
  __syncthreads();

  // ---- merge, outputs: a warp takes rows warp, warp + 8, ..., ROWS at a time and PARTS partials of each, all their loads in
  // flight; hd / 32 columns per lane. (The code is kept short on purpose: it runs once per block, and comes from memory too.
  // Unrolled over eight rows, with every load ahead of everything else, the merge took 24 us at batch 32, block 16.)
  constexpr int V = HD / 32;
  const float* const parts = p.part_o + (first_part * M + row0) * HD + lane * V;
#pragma unroll 1
  for (int r0 = warp; r0 < rows; r0 += FW * ROWS) {
    float acc[ROWS][V], mb[ROWS], lb[ROWS];
    int rr[ROWS];
#pragma unroll
    for (int b = 0; b < ROWS; ++b) {
      rr[b] = min(r0 + FW * b, rows - 1);
      mb[b] = row_s[rr[b]].x;
      lb[b] = row_s[rr[b]].w;
#pragma unroll
      for (int e = 0; e < V; ++e) acc[b][e] = 0.f;
    }
#pragma unroll 1
    for (int k0 = 0; k0 < n_parts; k0 += PARTS) {
      float v[ROWS][PARTS][V];
      float2 x[ROWS][PARTS];                 // d, r
#pragma unroll
      for (int b = 0; b < ROWS; ++b)
#pragma unroll
        for (int u = 0; u < PARTS; ++u) {
          const size_t at = static_cast<size_t>(min(k0 + u, n_parts - 1)) * M + rr[b];
          x[b][u] = *reinterpret_cast<const float2*>(recs + at);
          if constexpr (V == 4) { const float4 f = ld_now(reinterpret_cast<const float4*>(parts + at * HD)); v[b][u][0] = f.x; v[b][u][1] = f.y; v[b][u][2] = f.z; v[b][u][3] = f.w; }
          else { const float2 f = ld_now(reinterpret_cast<const float2*>(parts + at * HD)); v[b][u][0] = f.x; v[b][u][1] = f.y; }
        }
#pragma unroll
      for (int b = 0; b < ROWS; ++b)
#pragma unroll
        for (int u = 0; u < PARTS; ++u) {
          const float w = k0 + u < n_parts ? ex2(x[b][u].y - lb[b] + x[b][u].x - mb[b]) : 0.f;
#pragma unroll
          for (int e = 0; e < V; ++e) acc[b][e] = fmaf(w, v[b][u][e], acc[b][e]);
        }
    }
#pragma unroll 1
    for (int k = 0; k < KG; ++k)
#pragma unroll
      for (int b = 0; b < ROWS; ++b) {
        const int at = ((rr[b] >> 3) + MT * k) * 8 + (rr[b] & 7);
        const float f = ex2(ml_s[at].y - lb[b] + ml_s[at].x - mb[b]);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[b][e] = fmaf(f, join[at * HD + lane * V + e], acc[b][e]);
      }
#pragma unroll
    for (int b = 0; b < ROWS; ++b) {
      if (r0 + FW * b >= rows) break;
      const float4 st = row_s[rr[b]];
      const int row = row0 + rr[b], i = row / p.rep, gq = h * p.rep + row - i * p.rep;
      const size_t item = static_cast<size_t>(s * p.W + i) * p.n_kv * p.rep + gq;
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        *reinterpret_cast<uint32_t*>(out + item * HD + lane * V + e) = pack_bf16(acc[b][e] * st.y, acc[b][e + 1] * st.y);
        if (tap) *reinterpret_cast<float2*>(tap + item * HD + lane * V + e) = make_float2(acc[b][e] * st.y, acc[b][e + 1] * st.y);
      }
      if (mass && lane == 0) mass[item] = st.z;
    }
  }
}

template <int HD>
int launch(cod_ctx* c, int layer, const void* q, const void* kb, const void* vb, const cod_state* stt, int S, int use_carry, int rotate,
           void* out, float* tap, float* mass, cudaStream_t st) {
  const cod_config& f = c->cfg;
  const int rep = f.n_q_heads / f.n_kv_heads, M = f.block * rep;
  Kv8Params p{};
  p.q = static_cast<const __nv_bfloat16*>(q); p.kb = static_cast<const __nv_bfloat16*>(kb); p.vb = static_cast<const __nv_bfloat16*>(vb);
  p.pool = static_cast<const uint8_t*>(stt->kv_pool); p.scale = stt->kv_scale; p.carry = static_cast<const __nv_bfloat16*>(stt->carry_kv);
  p.block_table = stt->block_table; p.committed_len = stt->committed_len; p.carry_len = stt->carry_len;
  p.inv_freq = rotate ? c->inv_freq_d : nullptr;
  p.use_carry = use_carry; p.layer = layer; p.W = f.block; p.rep = rep; p.n_kv = f.n_kv_heads; p.n_pages = f.n_pages;
  p.max_pages = f.max_pages_per_seq; p.max_batch = f.max_batch; p.cap = c->carry_cap;
  p.S = S;
  p.part_o = c->attn_o; p.part_ml = c->attn_ml; p.status = c->status;
  // row tiles per warp (more than eight rows of head size 128: the other kernel). Head size 64 has this form for every row count,
  // the tcgen05 tile being 128 columns wide: 4, 16, 64, 128 rows take 43, 75, 186, 368 us at batch 32, 12, 14, 21, 35 for one
  // request of 2048 tokens; the plain-FMA kernel 319 to 2988 and 61 to 191.
  const int nr = HD == 128 || M <= 8 ? 1 : 2;
  const bool tcgen = cod_attn_kv8_tc_fits(c);
  p.unit = tcgen ? cod_attn_kv8_tc_unit() : 1;
  p.setup = tcgen ? cod_attn_kv8_tc_setup() : 0;
  p.line_blocks = cod_attn_kv8_blocks(c) / (tcgen ? cod_attn_kv8_tc_groups(c) : 1);
  if (tcgen) {
    const int rc = cod_launch_attn_kv8_tc(c, p, cod_attn_kv8_blocks(c), st);
    if (rc != COD_OK) return rc;
  } else {
    const size_t smem = 1024 + static_cast<size_t>(NW) * STAGES * 2 * PAGE * HD + static_cast<size_t>(NW) * 8 * nr * HD * sizeof(float) +
                        (rotate ? static_cast<size_t>(f.block) * HD * sizeof(float) : 0);
    CUtensorMap map;
    if (!tc::make_map_pages8(&map, stt->kv_pool, static_cast<uint64_t>(f.n_layers) * f.n_pages * f.n_kv_heads * 2 * PAGE, HD, 2 * PAGE)) return COD_ERR_CUDA;
    auto kern = k_attn_kv8<HD, 1>;
    if constexpr (HD == 64)
      if (nr == 2) kern = k_attn_kv8<HD, 2>;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess) return COD_ERR_CUDA;
    cod_launch_pdl(c, kern, cod_attn_kv8_blocks(c), NW * 32, smem, st, map, p);
    COD_CHECK_LAUNCH(c);
  }
  // the finish kernel follows the paged one at once; that one has itself waited for everything before it
  p.run_ahead = c->pdl ? 1 : 0;
  // small batches: the row tiles of a pair go to several blocks (each stages the short tail again), until the machine is full
  const int mtiles = (M + 7) / 8, pairs = S * f.n_kv_heads;
  const int groups = pairs >= c->n_sm ? 1 : (c->n_sm + pairs - 1) / pairs;
  const int tpb = (mtiles + groups - 1) / groups;
  const size_t fsm = static_cast<size_t>(tpb > FW ? tpb : FW) * 8 * HD * sizeof(float) + 2 * FKEYS * (HD * 2 + 16) +
                     (rotate ? static_cast<size_t>(f.block) * HD * sizeof(float) : 0);
  auto fin = tpb == 1 ? k_attn_kv8_finish<HD, 1, 8> : k_attn_kv8_finish<HD, 4, 2>;
  if (cudaFuncSetAttribute(fin, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(fsm)) != cudaSuccess) return COD_ERR_CUDA;
  cod_launch_pdl(c, fin, dim3(f.n_kv_heads, S, (mtiles + tpb - 1) / tpb), FW * 32, fsm, st, p, tpb, static_cast<__nv_bfloat16*>(out), tap, mass);
  COD_CHECK_LAUNCH(c);
  return COD_OK;
}

}  // namespace

// Blocks of the attention kernel: what stays resident at once (registers bound it), so that the work line is cut into equal
// stretches that all run together. Partial slots: one per block and one per (sequence, head) at most.
int cod_attn_kv8_blocks(const cod_ctx* c) {
  const int M = c->cfg.block * (c->cfg.n_q_heads / c->cfg.n_kv_heads);
  return c->n_sm * (cod_attn_kv8_tc_fits(c) ? 1 : M <= 8 ? 3 : 2);
}

bool cod_attn_kv8_supported(const cod_ctx* c) {
  return c->kv8 && c->cfg.dtype == COD_BF16 && c->cfg.max_batch <= 65535 && !c->force_simt && tc::encode_fn() != nullptr &&
         static_cast<long long>(c->cfg.max_batch) * c->cfg.n_kv_heads * (c->cfg.max_pages_per_seq + 16ll) < (1ll << 30) &&   // the work line and
         c->cfg.max_pages_per_seq < (1 << 26) &&                                                      // the lengths are counted in ints,
         static_cast<long long>(c->cfg.n_layers) * c->cfg.n_pages * c->cfg.n_kv_heads * 2 * PAGE < (1ll << 31);   // so are the copies' rows
}

// rotate: q and kb are not rotated yet
int cod_launch_attn_kv8(cod_ctx* c, int layer, const void* q, const void* kb, const void* vb, const cod_state* stt, int S,
                        int use_carry, int rotate, void* out, float* tap, float* mass, cudaStream_t st) {
  return c->cfg.head_dim == 128 ? launch<128>(c, layer, q, kb, vb, stt, S, use_carry, rotate, out, tap, mass, st)
                                : launch<64>(c, layer, q, kb, vb, stt, S, use_carry, rotate, out, tap, mass, st);
}
