// The 8-bit committed cache: rows of K and V quantised into pages through a slot map.
//
// A page holds 16 tokens of one (layer, KV head, K|V) as e4m3 bytes b with one scale s = 2^e; the element is b * s.
// With a the largest finite magnitude appended to the page so far, e is the least integer >= -100 with a <= 448 * 2^e.
// Appending rows x to a page that holds o rows:
//     s' = max(o > 0 ? s : 0, 2^e(max |x|)),   held bytes b -> e4m3(b * (s / s')),   new bytes = e4m3(min(|x| / s', 448)).
// Scales are powers of two so that s / s' and x / s' are exact: a byte written again differs from the one written at
// once only where it falls into e4m3's subnormals, however many times the scale grows, and no precision is lost for it
// (e4m3 is a floating format: a scale of amax / 448 instead would only shift where its 2^-9 floor lies, by less than 2x).
//
// One warp owns one (page, layer, head, K|V) of the call: it finds the rows of the page in the slot map, keeps them in
// registers between the maximum and the rounding (one read), and is the only one to touch the page's bytes and scale,
// so no atomics and no order dependence. The maximum is taken on packed bits: with floats the ALU pipe was busy for 73 % of
// the time and prompts of 24 requests took 158 us instead of 142.
#include "kv8_common.cuh"

namespace {

using namespace kv8;

constexpr int MIN_EXP = -100;          // scale of a page of zeros, and the floor of every scale
constexpr int APPEND_WARPS = 8;

__device__ __forceinline__ uint32_t float2_to_e4m3x2(float a, float b) {     // saturates at 448, keeps NaN
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
// 2^e as above from the largest finite magnitude: 448 = 1.75 * 2^8, so e = k - 8 for a = f * 2^k with f in [1, 1.75], else k - 7
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t u = __float_as_uint(amax);
  int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = e < MIN_EXP ? MIN_EXP : e;
  return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}

// eight consecutive elements
struct Row8 { float v[8]; };
__device__ __forceinline__ void unpack8(const uint4& u, Row8& r) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.v[2 * i] = __uint_as_float(w[i] << 16);
    r.v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void get(Row8& r) const { unpack8(a, r); }
  // the largest magnitude as the upper bits of a float (order of bits is order of magnitudes; infinity and NaN lie above)
  __device__ __forceinline__ uint32_t peak() const {
    const uint32_t m = 0x7FFF7FFFu, two = __vmaxu2(__vmaxu2(a.x & m, a.y & m), __vmaxu2(a.z & m, a.w & m));
    return max(two & 0xFFFF0000u, two << 16);
  }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __ldg(reinterpret_cast<const float4*>(p));
    b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void get(Row8& r) const {
    r.v[0] = a.x; r.v[1] = a.y; r.v[2] = a.z; r.v[3] = a.w; r.v[4] = b.x; r.v[5] = b.y; r.v[6] = b.z; r.v[7] = b.w;
  }
  __device__ __forceinline__ uint32_t peak() const {
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    return m;
  }
};

// Block (x, y) = (chunk of `chunk` rows, layer). A row is a leader if it opens its page's run of rows: the first row,
// offset 0, or a row that does not follow its predecessor. Leaders x (head, K|V) are dealt to the block's warps.
// (A page that occurs again after another page's rows would have two owners unseen: finding those takes a pass over the whole map.)
// LONG: what bounds a long map is how many rows are on their way, so registers give way to a fourth block per SM (bf16; 25,000
// rows of five layers: 142 us, with three blocks 152, with five, which spill, 147; its bytes at the rate of a plain copy: 132).
// A short map fits the machine at once and keeps them (a round's rows at batch 32: 7.5 us). Four blocks spill 8 bytes.
template <typename T, int HD, bool LONG>
__global__ void __launch_bounds__(APPEND_WARPS * 32, !LONG ? 1 : sizeof(T) == 2 ? 4 : 2)
k_kv8_append(const T* __restrict__ J, const int* __restrict__ slot, int n_rows, int n_kv, int n_pages, int chunk,
             uint8_t* __restrict__ pool, float* __restrict__ scale, uint32_t* status) {
  cod_pdl_prologue();
  __shared__ int lead[32], n_lead_s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row0 = blockIdx.x * chunk, layer = blockIdx.y;
  const long long n_slots = static_cast<long long>(n_pages) * PAGE;
  if (warp == 0) {
    const int r = row0 + lane, w = row0 - 32 + lane;
    const int sl = lane < chunk && r < n_rows ? slot[r] : -1, old = w >= 0 ? slot[w] : -1;
    const unsigned here = __ballot_sync(0xffffffffu, sl >= 0), past = __ballot_sync(0xffffffffu, old >= 0);
    const unsigned below = here & ((1u << lane) - 1u);
    const int in_chunk = __shfl_sync(0xffffffffu, sl, below ? 31 - __clz(below) : 0);
    const int in_past = __shfl_sync(0xffffffffu, old, past ? 31 - __clz(past) : 0);
    int before = below ? in_chunk : past ? in_past : -1;     // the nearest earlier row that goes somewhere
    const bool next_to_it = lane ? (here >> (lane - 1)) & 1u : past >> 31;
    bool opens = sl >= 0 && !(next_to_it && before == sl - 1 && (sl & (PAGE - 1)) != 0);
    if (past == 0 && __any_sync(0xffffffffu, opens)) {       // rows that go nowhere, more than 32 of them: further back
      int found = -1;
      for (int end = row0 - 32; found < 0 && end > 0; end -= 256) {
        int v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) { const int at = end - 256 + 32 * u + lane; v[u] = at >= 0 ? slot[at] : -1; }
#pragma unroll
        for (int u = 7; u >= 0; --u) {
          const unsigned some = __ballot_sync(0xffffffffu, v[u] >= 0);
          const int last = __shfl_sync(0xffffffffu, v[u], some ? 31 - __clz(some) : 0);
          if (found < 0 && some) found = last;
        }
      }
      if (!below) before = found;
    }
    // a row of its predecessor's page that does not follow it would be a second owner of that page
    if (opens && (sl >= n_slots || (before >= 0 && before / PAGE == sl / PAGE))) {
      if (layer == 0) atomicOr(status, COD_DEV_BAD_SLOT);
      opens = false;
    }
    const unsigned m = __ballot_sync(0xffffffffu, opens);
    if (opens) lead[__popc(m & ((1u << lane) - 1u))] = r;
    if (lane == 0) n_lead_s = __popc(m);
  }
  __syncthreads();
  const int n_task = n_lead_s * 2 * n_kv;
  constexpr int LPR = HD / 8;              // lanes per row, eight elements each
  constexpr int RPS = 32 / LPR;            // rows per step
  constexpr int STEPS = PAGE / RPS;
  const int sub = lane / LPR, col = (lane % LPR) * 8;
  for (int task = warp; task < n_task; task += APPEND_WARPS) {
    const int r0 = lead[task / (2 * n_kv)], hk = task % (2 * n_kv);   // K and V of a head next to each other in the page
    const int h = hk >> 1, kv = hk & 1;
    const int sl0 = slot[r0], pg = sl0 / PAGE, off = sl0 & (PAGE - 1);
    // rows of the run: up to the end of the page, of the map, or of the increasing slots
    const bool in = lane < PAGE - off && r0 + lane < n_rows && slot[r0 + lane] == sl0 + lane;
    const unsigned run = __ballot_sync(0xffffffffu, in);
    const int n = __ffs(~run) - 1;
    const T* src = J + ((static_cast<size_t>(layer) * n_rows + r0) * 2 + kv) * n_kv * HD + h * HD + col;
    const size_t row_stride = static_cast<size_t>(2) * n_kv * HD;
    Raw8<T> x[STEPS];
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      const int i = t * RPS + sub;
      if (i < n) x[t].load(src + i * row_stride);
    }
    const size_t unit = ((static_cast<size_t>(layer) * n_pages + pg) * n_kv + h) * 2 + kv;
    uint8_t* page = pool + unit * PAGE * HD;
    const float s_old = off > 0 ? scale[unit] : 0.f;
    uint32_t bits = 0;
#pragma unroll
    for (int t = 0; t < STEPS; ++t)
      if (t * RPS + sub < n) bits = max(bits, x[t].peak());
    bits = __reduce_max_sync(0xffffffffu, bits);
    float amax = __uint_as_float(bits);
    if (bits >= 0x7F800000u) {             // something is not finite: the largest of the others
      amax = 0.f;
#pragma unroll
      for (int t = 0; t < STEPS; ++t) {
        if (t * RPS + sub < n) {
          Row8 f;
          x[t].get(f);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float a = fabsf(f.v[e]);
            amax = fmaxf(amax, a < INFINITY ? a : 0.f);
          }
        }
      }
      amax = cod_warp_max(amax);
    }
    const float s_new = fmaxf(s_old, scale_for(amax));
    if (off > 0 && s_new != s_old) {       // the page's scale grows: its held rows, 16 bytes per lane
      const float f = s_old / s_new;       // powers of two: exact (0 where the page never had a scale)
      for (int b = lane * 16; b < off * HD; b += 512) {
        uint4 w = *reinterpret_cast<const uint4*>(page + b);
        uint32_t* u = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 lo = e4m3x2_to_float2(u[e] & 0xFFFFu), hi = e4m3x2_to_float2(u[e] >> 16);
          u[e] = float2_to_e4m3x2(lo.x * f, lo.y * f) | (float2_to_e4m3x2(hi.x * f, hi.y * f) << 16);
        }
        *reinterpret_cast<uint4*>(page + b) = w;
      }
    }
    const float inv = 1.f / s_new;
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      const int i = t * RPS + sub;
      if (i < n) {
        Row8 f;
        x[t].get(f);
        uint2 o;
        o.x = float2_to_e4m3x2(f.v[0] * inv, f.v[1] * inv) | (float2_to_e4m3x2(f.v[2] * inv, f.v[3] * inv) << 16);
        o.y = float2_to_e4m3x2(f.v[4] * inv, f.v[5] * inv) | (float2_to_e4m3x2(f.v[6] * inv, f.v[7] * inv) << 16);
        *reinterpret_cast<uint2*>(page + static_cast<size_t>(off + i) * HD + col) = o;
      }
    }
    __syncwarp();                          // every lane has read the old scale
    if (lane == 0) scale[unit] = s_new;
  }
}

template <typename T, int HD>
int launch_append(cod_ctx* c, const void* J, const int32_t* slot, int n_rows, const cod_state* ds, cudaStream_t st) {
  const cod_config& f = c->cfg;
  // Rows per block: a page's rows are one task per (head, K|V), so blocks of 16 rows give the warps of a long prompt their
  // pages with few empty blocks; short maps are dealt finer, so that the machine fills. Five layers, 16 against 4 rows per block:
  // 2048 rows 14.8 and 19.3 us, 1024 rows 9.0 and 10.2, 512 rows 6.5 and 6.6, but 13.3 and 7.2 for 272 rows of 32 requests. Floats
  // agree (2048 rows: 19.4 and 35.0). The bounds are those of five layers: with one, prompts of 512 to 2048 rows take 7.5 to 8.2 us
  // (floats 9 to 12) where blocks of 16 rows took 6.2, and 272 rows of 32 requests 6.2 where those took 10.3.
  const long long work = static_cast<long long>(n_rows) * f.n_layers;
  const bool is_long = work > 24ll * c->n_sm;
  const int chunk = is_long ? 16 : work > 8ll * c->n_sm ? 4 : 1;
  const dim3 grid((n_rows + chunk - 1) / chunk, f.n_layers);
  cod_launch_pdl(c, is_long ? k_kv8_append<T, HD, true> : k_kv8_append<T, HD, false>, grid, APPEND_WARPS * 32, 0, st, static_cast<const T*>(J), slot, n_rows, f.n_kv_heads,
                 f.n_pages, chunk, static_cast<uint8_t*>(ds->kv_pool), ds->kv_scale, c->status);
  COD_CHECK_LAUNCH(c);
  return COD_OK;
}

}  // namespace

int cod_launch_kv8_append(cod_ctx* c, const void* J, const int32_t* slot, int n_rows, const cod_state* ds, cudaStream_t st) {
  ProfScope prof(c, COD_K_ROWOPS, st);
  if (c->cfg.dtype == COD_BF16)
    return c->cfg.head_dim == 128 ? launch_append<__nv_bfloat16, 128>(c, J, slot, n_rows, ds, st)
                                  : launch_append<__nv_bfloat16, 64>(c, J, slot, n_rows, ds, st);
  return c->cfg.head_dim == 128 ? launch_append<float, 128>(c, J, slot, n_rows, ds, st)
                                : launch_append<float, 64>(c, J, slot, n_rows, ds, st);
}
