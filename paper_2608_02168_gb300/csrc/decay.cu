// Causal linear attention with a decay for each head: entry points, the CUDA-core scan (fp32 storage), the
// join of segments, and the step of one snapshot.
//
//   S_t = gamma S_(t-1) + k_t v_t^T,  o_t = c q_t S_t;  the gradients are three scans of the same form
//   (decay_kernels.cuh).
//
// CUDA-core scan: a lane owns one value feature of a head, so its column of the state (d_h numbers) stays in registers
// and o_t needs no exchange; the keys and queries of a few positions are laid in shared memory for their warp, where
// all lanes read the same 16 bytes at once.  2 d_h FMA a position and lane.  Bound by latency: nothing is loaded ahead,
// and the positions of a lane follow one another (300 histories of 300 positions, 4 heads: 81, 154, 487 and 1672 us at
// d_h = 16, 32, 64 and 128, 4.5 to 14 TFLOP/s of 80 and 0.06 to 0.18 of HBM), so the three scans of a gradient run side
// by side (133, 354, 1004, 4917 us).
// Long histories of few sequences: the histories are cut into segments; a first pass finds each segment's own
// state, a join runs through them, and the scan then starts each segment from its true state.
//
// The step reads and writes the state once (16-byte rows of it across the lanes): bound by HBM (200000 nodes, 4 heads
// of 32, 6.8 GB: 990 us, 0.98 of the measured rate).
#include <algorithm>
#include <initializer_list>

#include "decay_kernels.cuh"
#include "row_sets.cuh"

namespace hg {

namespace {

constexpr int kMaxHeads = 64;
constexpr int kWarps = 4;
constexpr int kSms = 152;

template <int DH>
struct SimtCfg {
  static constexpr int W = DH < 32 ? 32 : DH;     // values of a staged row: the heads of 32 columns
  static constexpr int TC = DH <= 32 ? 16 : 8;    // positions staged at a time
};

// blockIdx.x * kWarps + warp = ((sequence * nseg) + segment) * column blocks + column block, blockIdx.y the scan
template <int DH, bool kLocal>
__global__ void __launch_bounds__(32 * kWarps) scan_simt(const __grid_constant__ ScanBatch b) {
  pdl_begin();
  const ScanArgs& a = b.s[blockIdx.y];
  using T = float;
  using C = SimtCfg<DH>;
  constexpr int W = C::W, TC = C::TC, VEC = VecTraits<T>::kElems;
  __shared__ __align__(16) float sk[kWarps][TC][W];
  __shared__ __align__(16) float sq[kLocal ? 1 : kWarps][kLocal ? 1 : TC][W];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int width = a.heads * DH;
  const int ncb = (width + 31) / 32;
  const int64_t item = (int64_t)blockIdx.x * kWarps + warp;
  const int64_t seq = item / (ncb * a.nseg);
  if (seq >= a.n) return;
  const int cb = (int)(item % ncb), segi = (int)(item / ncb % a.nseg);
  const int col = cb * 32 + lane;
  const bool on = col < width;
  const int head = on ? col / DH : a.heads - 1, j = col % DH;
  const int row0 = cb * 32 / DH * DH;                 // first staged value of a row
  const int rw = min(W, width - row0);                // staged values of a row (a multiple of 16)
  const int hoff = on ? (head * DH - row0) : 0;       // this lane's head within them
  const int64_t len = scan_len(a, seq);
  const int64_t t0 = segi * a.seg_len;
  const int64_t tend = min(t0 + a.seg_len, a.T);
  const int64_t t1 = min(tend, len);
  if (kLocal && segi == a.nseg - 1) return;
  const float ld = clamp_ld(a.ld[head]);
  float S[DH];
#pragma unroll
  for (int i = 0; i < DH; ++i) S[i] = 0.f;
  const int64_t st0 = (seq * a.heads + head) * (int64_t)DH * DH;
  if (!kLocal && on) {
    if (a.nseg > 1) {
      const float* src = a.seg + ((seq * a.heads + head) * a.nseg + segi) * (int64_t)DH * DH + j;
#pragma unroll
      for (int i = 0; i < DH; ++i) S[i] = src[i * DH];
    } else if (a.init) {
#pragma unroll
      for (int i = 0; i < DH; ++i) S[i] = a.init[st0 + (a.init_t ? j * DH + i : i * DH + j)];
    }
  }
  int base = 0;  // frame base, in positions from t0
  const T* qp = static_cast<const T*>(a.q.p) + seq * a.q.sn + row0;
  const T* kp = static_cast<const T*>(a.k.p) + seq * a.k.sn + row0;
  const T* vp = static_cast<const T*>(a.v.p) + seq * a.v.sn;
  T* op = static_cast<T*>(const_cast<void*>(a.o.p)) + seq * a.o.sn;
  for (int64_t tc = t0; tc < t1; tc += TC) {
    const int m = (int)min((int64_t)TC, t1 - tc);
    __syncwarp();
    for (int x = lane; x < m * (rw / VEC); x += 32) {
      const int r = x / (rw / VEC), c = x % (rw / VEC) * VEC;
      const int64_t t = a.reverse ? len - 1 - (tc + r) : tc + r;
      float f[VEC];
      unpack(ld16(kp + t * a.k.st + c), f, T());
#pragma unroll
      for (int e = 0; e < VEC; ++e) sk[warp][r][c + e] = f[e];
      if (!kLocal) {
        unpack(ld16(qp + t * a.q.st + c), f, T());
#pragma unroll
        for (int e = 0; e < VEC; ++e) sq[warp][r][c + e] = f[e];
      }
    }
    float v[TC];
#pragma unroll
    for (int r = 0; r < TC; ++r) {
      const int64_t t = a.reverse ? len - 1 - (tc + r) : tc + r;
      v[r] = on && r < m ? to_f32(vp[t * a.v.st + col]) : 0.f;
    }
    __syncwarp();
#pragma unroll
    for (int r = 0; r < TC; ++r) {
      if (r >= m) break;
      const int64_t t = tc + r;
      const int tau = (int)(t - t0) + a.shift;
      const bool move = (float)(base - tau) * ld > kFrame;
      if (__any_sync(0xffffffffu, move)) {
        const float g = move ? expf(ld * (float)(tau - base)) : 1.f;
#pragma unroll
        for (int i = 0; i < DH; ++i) S[i] *= g;
        if (move) base = tau;
      }
      const float vin = a.c_in * expf(ld * (float)(base - tau)) * v[r];
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int i = 0; i < DH; i += 4) {
        const float4 k4 = *reinterpret_cast<const float4*>(&sk[warp][r][hoff + i]);
        S[i] = fmaf(k4.x, vin, S[i]);
        S[i + 1] = fmaf(k4.y, vin, S[i + 1]);
        S[i + 2] = fmaf(k4.z, vin, S[i + 2]);
        S[i + 3] = fmaf(k4.w, vin, S[i + 3]);
        if (!kLocal) {
          const float4 q4 = *reinterpret_cast<const float4*>(&sq[warp][r][hoff + i]);
          s0 = fmaf(q4.x, S[i], s0);
          s1 = fmaf(q4.y, S[i + 1], s1);
          s0 = fmaf(q4.z, S[i + 2], s0);
          s1 = fmaf(q4.w, S[i + 3], s1);
        }
      }
      if (!kLocal && on) {
        const int64_t row = a.reverse ? len - 1 - t : t;
        op[row * a.o.st + col] = from_f32<T>(a.c_out * expf(ld * (float)(tau - base)) * (s0 + s1));
      }
    }
  }
  if (!kLocal && on)
    for (int64_t t = max(t0, len); t < tend; ++t) op[t * a.o.st + col] = from_f32<T>(0.f);
  if (!on) return;
  const float g = expf(ld * (float)((int)(max(t1, t0) - t0) - base));
  if (kLocal) {
    float* dst = a.seg + ((seq * a.heads + head) * a.nseg + segi) * (int64_t)DH * DH + j;
#pragma unroll
    for (int i = 0; i < DH; ++i) dst[i * DH] = S[i] * g;
  } else if (a.last && segi == (len > 0 ? (len - 1) / a.seg_len : 0)) {
#pragma unroll
    for (int i = 0; i < DH; ++i) a.last[st0 + i * DH + j] = S[i] * g;
  }
}

// seg[s] (segment s's own state, for s < nseg - 1) -> the state at segment s's start: one thread an element,
// blockIdx.y the scan.
__global__ void __launch_bounds__(256) scan_join(const __grid_constant__ ScanBatch b, int dh) {
  pdl_begin();
  const ScanArgs& a = b.s[blockIdx.y];
  const int64_t dd = (int64_t)dh * dh, total = a.n * a.heads * dd;
  const int64_t x = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (x >= total) return;
  const int64_t sh = x / dd, e = x % dd, i = e / dh, j = e % dh;
  const int64_t len = scan_len(a, sh / a.heads);
  const float ld = clamp_ld(a.ld[sh % a.heads]);
  // in a frame, as in the scans: a multiplication for each segment would gather the rounding of its factor
  int base = 0;
  float F = a.init ? a.init[sh * dd + (a.init_t ? j * dh + i : e)] : 0.f;
  float* seg = a.seg + sh * a.nseg * dd + e;
  constexpr int U = 8;  // the next states are loaded while these are joined
  float own[U];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) own[u] = s0 + u + 1 < a.nseg ? seg[(s0 + u) * dd] : 0.f;
  };
  fetch(0);
  for (int s0 = 0; s0 < a.nseg; s0 += U) {
    float now[U];
#pragma unroll
    for (int u = 0; u < U; ++u) now[u] = own[u];
    if (s0 + U < a.nseg) fetch(s0 + U);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + u;
      if (s >= a.nseg) break;
      const int t = (int)min(s * a.seg_len, len), t1 = (int)min((s + 1) * a.seg_len, len);
      seg[s * dd] = F * expf(ld * (float)(t - base));
      if ((float)(base - t1) * ld > kFrame) {
        F *= expf(ld * (float)(t1 - base));
        base = t1;
      }
      F = fmaf(now[u], expf(ld * (float)(base - t1)), F);
    }
  }
}

// One row a node.  A warp takes one head: DH / 4 lanes (32 of them hold 4 columns each at DH = 128) span a row
// of the state, the others the next rows, and the rows' sums meet by shuffles.
template <typename T, int DH>
__global__ void __launch_bounds__(256) decay_step_kernel(const T* __restrict__ q, int64_t sq, const T* __restrict__ k,
                                                         int64_t sk, const T* __restrict__ v, int64_t sv,
                                                         const int32_t* __restrict__ live, const float* __restrict__ ld,
                                                         int64_t n, int heads, float scale, const float* S_in, T* o,
                                                         int64_t so, float* S_out) {
  pdl_begin();
  constexpr int LR = DH / 4;       // lanes of a row
  constexpr int RW = 32 / LR;      // rows at a time
  constexpr int NR = DH / RW;      // rounds
  constexpr int U = NR < 8 ? NR : 8;
  const int lane = threadIdx.x & 31;
  const int64_t item = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  if (item >= n * heads) return;
  const int64_t i = item / heads;
  const int h = (int)(item % heads);
  const int c = lane % LR * 4, r0 = lane / LR;
  const float* src = S_in + item * (DH * DH) + c;
  float* dst = S_out + item * (DH * DH) + c;
  T* orow = o + i * so + h * DH;
  if (live && live[i] <= 0) {
    if (S_in != S_out)
      for (int r = r0; r < DH; r += RW)
        *reinterpret_cast<float4*>(dst + r * DH) = *reinterpret_cast<const float4*>(src + r * DH);
    for (int x = lane; x < DH; x += 32) orow[x] = from_f32<T>(0.f);
    return;
  }
  const float g = expf(clamp_ld(ld[h]));
  const T* qr = q + i * sq + h * DH;
  const T* kr = k + i * sk + h * DH;
  const T* vr = v + i * sv + h * DH + c;
  const float4 vv = make_float4(to_f32(vr[0]), to_f32(vr[1]), to_f32(vr[2]), to_f32(vr[3]));
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int b = 0; b < NR; b += U) {
    float4 s[U];
    float kk[U], qq[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = (b + u) * RW + r0;
      s[u] = *reinterpret_cast<const float4*>(src + r * DH);
      kk[u] = to_f32(kr[r]);
      qq[u] = to_f32(qr[r]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = (b + u) * RW + r0;
      float4 y = s[u];
      y.x = fmaf(kk[u], vv.x, g * y.x);
      y.y = fmaf(kk[u], vv.y, g * y.y);
      y.z = fmaf(kk[u], vv.z, g * y.z);
      y.w = fmaf(kk[u], vv.w, g * y.w);
      *reinterpret_cast<float4*>(dst + r * DH) = y;
      acc.x = fmaf(qq[u], y.x, acc.x);
      acc.y = fmaf(qq[u], y.y, acc.y);
      acc.z = fmaf(qq[u], y.z, acc.z);
      acc.w = fmaf(qq[u], y.w, acc.w);
    }
  }
#pragma unroll
  for (int x = LR; x < 32; x <<= 1) {
    acc.x += __shfl_xor_sync(0xffffffffu, acc.x, x);
    acc.y += __shfl_xor_sync(0xffffffffu, acc.y, x);
    acc.z += __shfl_xor_sync(0xffffffffu, acc.z, x);
    acc.w += __shfl_xor_sync(0xffffffffu, acc.w, x);
  }
  if (lane < LR) {
    orow[c] = from_f32<T>(scale * acc.x);
    orow[c + 1] = from_f32<T>(scale * acc.y);
    orow[c + 2] = from_f32<T>(scale * acc.z);
    orow[c + 3] = from_f32<T>(scale * acc.w);
  }
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
// Segments: as many as fill the GPU with warps, of at least 64 (bf16) or 32 positions, where that pays.  A scan in
// segments takes as long as about 2.5 T / segments + 300 (bf16) or 2 T / segments + 60 positions of one without: keys
// and values are read twice, a state is written and joined for each segment, and there are two more launches.
// Measured (us, whole | segments; 4 heads): bf16, d_h 64, T = 2000, room for 2 segments 209 | 244, 3: 209 | 191, 4:
// 208 | 152; T = 600, 4: 70 | 76; d_h 32, 10 histories of 400: 29 | 27, 700: 45 | 28; fp32, d_h 32, T = 600, room for
// 2: 305 | 327, 3: 301 | 231; 10 histories of 100: 42 | 46, 128: 52 | 38.  fp32 was measured at d_h = 32 alone, and its
// 16 warps an SM are taken for every width (registers leave room for 20, 16, 12 and 8 at d_h = 16 to 128).
void plan_segments(const hg_decay_params* p, int64_t n, int64_t T, int scans, int* nseg, int64_t* seg_len) {
  const bool mma = p->dtype == HG_BF16;
  const int64_t each = mma ? scan_mma_warps(p->heads, p->d_h) : (p->heads * p->d_h + 31) / 32;
  const int64_t full = kSms * (mma ? scan_mma_resident(p->d_h) : 16);
  const int64_t want = std::min<int64_t>(full / (std::max<int64_t>(n, 1) * each * scans), T / (mma ? 64 : 32));
  *nseg = 1;
  *seg_len = std::max<int64_t>(T, 1);
  if (want < 2 || (mma ? 5 * T / want + 600 >= 2 * T : 2 * T / want + 60 >= T)) return;
  *seg_len = (int64_t)align_up((size_t)ceil_div(T, want), 16);
  *nseg = (int)ceil_div(T, *seg_len);
}

template <int DH>
hg_status scan_simt_t(const ScanBatch& b, bool local, cudaStream_t s) {
  const ScanArgs& a = b.s[0];
  const int64_t items = a.n * a.nseg * (int64_t)((a.heads * DH + 31) / 32);
  const dim3 grid((unsigned)ceil_div(items, kWarps), (unsigned)b.count);
  if (local) return launch("decay_scan_local", scan_simt<DH, true>, grid, dim3(32 * kWarps), 0, s, b);
  return launch("decay_scan", scan_simt<DH, false>, grid, dim3(32 * kWarps), 0, s, b);
}

hg_status scan_pass(const ScanBatch& b, const hg_decay_params* p, bool local, cudaStream_t s) {
  if (p->dtype == HG_BF16) return scan_mma(b, p->d_h, local, s);
  if (p->d_h == 16) return scan_simt_t<16>(b, local, s);
  if (p->d_h == 32) return scan_simt_t<32>(b, local, s);
  if (p->d_h == 64) return scan_simt_t<64>(b, local, s);
  return scan_simt_t<128>(b, local, s);
}

// Scratch: counters of the claimed items, one for each launch of a call, then the segments' states.
constexpr int kClaims = 8;
// Ragged histories of this length on are claimed by the warps instead of dealt out (us, dealt | claimed; 4 heads): 400
// of up to 515, d_h 64: 116 | 94; 2000 of up to 200, d_h 32: 71 | 61; 2000 of up to 100: 39.6 | 39.2, and shorter ones
// gain from the lengths that are asked for ahead.
constexpr int64_t kClaimT = 128;
bool scan_claims(const hg_decay_params* p, int64_t T) { return p->dtype == HG_BF16 && T >= kClaimT; }

// The scans [first, first + count) of a call, side by side.
hg_status scan(const ScanArgs* first, int count, uint32_t*& claims, const hg_decay_params* p, cudaStream_t s) {
  ScanBatch b{};
  b.count = count;
  auto pass = [&](bool local) -> hg_status {
    for (int i = 0; i < count; ++i) b.s[i].claims = claims;
    if (claims) ++claims;
    return scan_pass(b, p, local, s);
  };
  for (int i = 0; i < count; ++i) b.s[i] = first[i];
  const ScanArgs& a = b.s[0];
  if (a.nseg > 1) {
    HG_TRY(pass(true));
    const unsigned blocks = (unsigned)ceil_div(a.n * a.heads * (int64_t)p->d_h * p->d_h, 256);
    HG_TRY(launch("decay_scan_join", scan_join, dim3(blocks, (unsigned)count), dim3(256), 0, s, b, p->d_h));
  }
  return pass(false);
}

hg_status check_params(const hg_decay_params* p, int64_t n, int64_t T) {
  HG_REQUIRE(p != nullptr, "params must be non-null");
  if (!(p->d_h == 16 || p->d_h == 32 || p->d_h == 64 || p->d_h == 128) ||
      !(p->dtype == HG_F32 || p->dtype == HG_BF16)) {
    set_error("unsupported d_h=%d / dtype=%d", p->d_h, (int)p->dtype);
    return HG_ERR_UNSUPPORTED;
  }
  HG_REQUIRE(p->heads >= 1 && p->heads <= kMaxHeads, "heads must be in [1, %d]", kMaxHeads);
  HG_REQUIRE(n >= 0 && n < (int64_t(1) << 28) && n * p->heads < (int64_t(1) << 28), "n * heads must be in [0, 2^28)");
  HG_REQUIRE(T >= 0 && T < (int64_t(1) << 30), "T must be in [0, 2^30)");
  return HG_OK;
}

// Rows that are written meet none of the others.
hg_status check_apart(const hg_seq* out, const char* name, int64_t n, int64_t T, int64_t width, size_t esz,
                      std::initializer_list<const hg_seq*> others) {
  for (const hg_seq* r : others)
    HG_TRY(check_apart(seq_set(out, n, T, width, esz), name, {seq_set(r, n, T, width, esz)}));
  return HG_OK;
}

// A state that is written is another one itself, or shares nothing with it.
hg_status check_state(const hg_decay_params* p, int64_t n, const float* out, const float* in, const char* names) {
  const size_t bytes = sizeof(float) * (size_t)n * p->heads * p->d_h * p->d_h;
  HG_REQUIRE(!shifted(out, in, bytes), "%s must not overlap", names);
  return HG_OK;
}

hg_status check_buffers(const hg_decay_params* p, const void* scratch, bool needed) {
  HG_REQUIRE(p->log_decay != nullptr, "log_decay must be non-null");
  HG_REQUIRE(!needed || scratch != nullptr, "scratch must be non-null");
  HG_REQUIRE(((uintptr_t)scratch & 255) == 0, "scratch must be 256-byte aligned");
  return HG_OK;
}

ScanRows rows_of(const hg_seq* r, int64_t n, int64_t T) {
  return {r->p, n < 2 ? 0 : r->stride_n, T < 2 ? 0 : r->stride_t};
}

// Scratch of a call's scans: the counters, then each scan's states.
struct ScanLayout {
  int nseg;
  int64_t seg_len;
  uint32_t* claims;
  float* seg[3];
};
size_t carve_scans(void* scratch, const hg_decay_params* p, int64_t n, int64_t T, int scans, ScanLayout* L) {
  *L = ScanLayout{};
  plan_segments(p, n, T, scans, &L->nseg, &L->seg_len);
  if (n == 0) return 0;
  Carve c(scratch);
  if (scan_claims(p, T)) L->claims = c.take<uint32_t>(kClaims);
  const size_t states = L->nseg > 1 ? (size_t)n * p->heads * L->nseg * p->d_h * p->d_h : 0;
  for (int i = 0; i < scans && states; ++i) L->seg[i] = c.take<float>(states);
  return c.used;
}

// The scans' part of a call: counters zeroed where the lengths are ragged.
hg_status lay_out(ScanArgs* a, int scans, uint32_t** claims, const hg_decay_params* p, void* scratch, cudaStream_t s) {
  ScanLayout L;
  carve_scans(scratch, p, a->n, a->T, scans, &L);
  for (int i = 0; i < scans; ++i) {
    a[i].seg = L.seg[i];
    a[i].nseg = L.nseg;
    a[i].seg_len = L.seg_len;
  }
  *claims = a->lens ? L.claims : nullptr;
  if (*claims) HG_CUDA(cudaMemsetAsync(*claims, 0, sizeof(uint32_t) * kClaims, s));
  return HG_OK;
}

}  // namespace
}  // namespace hg

using namespace hg;

extern "C" hg_status hg_decay_workspace_size(const hg_decay_params* params, int64_t n, int64_t T, size_t* fwd_bytes,
                                             size_t* bwd_bytes) {
  clear_error();
  HG_REQUIRE(fwd_bytes && bwd_bytes, "fwd_bytes and bwd_bytes must be non-null");
  HG_TRY(check_params(params, n, T));
  ScanLayout L;
  *fwd_bytes = carve_scans(nullptr, params, n, T, 1, &L);
  *bwd_bytes = carve_scans(nullptr, params, n, T, 3, &L);
  return HG_OK;
}

extern "C" hg_status hg_decay_fwd(const hg_decay_params* params, const hg_seq* q, const hg_seq* k, const hg_seq* v,
                                  const int32_t* lens, int64_t n, int64_t T, const float* S_in, const hg_seq* o,
                                  float* S_out, void* scratch, hg_stream stream) {
  clear_error();
  HG_TRY(device_guard());
  HG_TRY(check_params(params, n, T));
  ScanLayout L;
  const size_t need = carve_scans(nullptr, params, n, T, 1, &L);
  HG_TRY(check_buffers(params, scratch, need > 0));
  if (n == 0) return HG_OK;
  const size_t esz = params->dtype == HG_BF16 ? 2 : 4;
  const int64_t w = (int64_t)params->heads * params->d_h;
  ScanArgs a{};
  if (T > 0) {
    HG_TRY(check_seq(q, "q", n, T, w, esz, false));
    HG_TRY(check_seq(k, "k", n, T, w, esz, false));
    HG_TRY(check_seq(v, "v", n, T, w, esz, false));
    HG_TRY(check_seq(o, "o", n, T, w, esz, true));
    HG_TRY(check_apart(o, "o", n, T, w, esz, {q, k, v}));
    a.q = rows_of(q, n, T);
    a.k = rows_of(k, n, T);
    a.v = rows_of(v, n, T);
    a.o = rows_of(o, n, T);
  }
  HG_TRY(check_state(params, n, S_out, S_in, "S_out and S_in"));
  a.lens = lens;
  a.ld = params->log_decay;
  a.init = S_in;
  a.last = S_out;
  a.n = n;
  a.T = T;
  a.heads = params->heads;
  a.shift = 1;
  a.c_in = 1.f;
  a.c_out = params->scale;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  uint32_t* claims;
  HG_TRY(lay_out(&a, 1, &claims, params, scratch, s));
  return scan(&a, 1, claims, params, s);
}

extern "C" hg_status hg_decay_bwd(const hg_decay_params* params, const hg_seq* q, const hg_seq* k, const hg_seq* v,
                                  const int32_t* lens, int64_t n, int64_t T, const float* S_in, const hg_seq* d_o,
                                  const float* dS_out, const hg_seq* dq, const hg_seq* dk, const hg_seq* dv,
                                  float* dS_in, void* scratch, hg_stream stream) {
  clear_error();
  HG_TRY(device_guard());
  HG_TRY(check_params(params, n, T));
  ScanLayout L;
  const size_t need = carve_scans(nullptr, params, n, T, 3, &L);
  HG_TRY(check_buffers(params, scratch, need > 0));
  if (n == 0) return HG_OK;
  const size_t esz = params->dtype == HG_BF16 ? 2 : 4;
  const int64_t w = (int64_t)params->heads * params->d_h;
  ScanArgs a{};
  ScanRows rq{}, rk{}, rv{}, ro{}, gq{}, gk{}, gv{};
  if (T > 0) {
    HG_TRY(check_seq(q, "q", n, T, w, esz, false));
    HG_TRY(check_seq(k, "k", n, T, w, esz, false));
    HG_TRY(check_seq(v, "v", n, T, w, esz, false));
    HG_TRY(check_seq(d_o, "d_o", n, T, w, esz, false));
    HG_TRY(check_seq(dq, "dq", n, T, w, esz, true));
    HG_TRY(check_seq(dk, "dk", n, T, w, esz, true));
    HG_TRY(check_seq(dv, "dv", n, T, w, esz, true));
    HG_TRY(check_apart(dq, "dq", n, T, w, esz, {q, k, v, d_o, dk, dv}));
    HG_TRY(check_apart(dk, "dk", n, T, w, esz, {q, k, v, d_o, dv}));
    HG_TRY(check_apart(dv, "dv", n, T, w, esz, {q, k, v, d_o}));
    rq = rows_of(q, n, T);
    rk = rows_of(k, n, T);
    rv = rows_of(v, n, T);
    ro = rows_of(d_o, n, T);
    gq = rows_of(dq, n, T);
    gk = rows_of(dk, n, T);
    gv = rows_of(dv, n, T);
  }
  a.lens = lens;
  a.ld = params->log_decay;
  a.n = n;
  a.T = T;
  a.heads = params->heads;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  HG_REQUIRE(!dS_in || dS_in != S_in, "dS_in must not overlap S_in");
  HG_TRY(check_state(params, n, dS_in, S_in, "dS_in and S_in"));
  HG_TRY(check_state(params, n, dS_in, dS_out, "dS_in and dS_out"));
  ScanArgs g[3] = {a, a, a};
  ScanArgs &aq = g[0], &ak = g[1], &av = g[2];
  aq.q = ro;  // dq
  aq.k = rv;
  aq.v = rk;
  aq.o = gq;
  aq.init = S_in;
  aq.init_t = 1;
  aq.shift = 1;
  aq.c_in = 1.f;
  aq.c_out = params->scale;
  ak.q = rv;  // dk
  ak.k = ro;
  ak.v = rq;
  ak.o = gk;
  ak.init = dS_out;
  ak.init_t = 1;
  ak.reverse = 1;
  ak.c_in = params->scale;
  ak.c_out = 1.f;
  av.q = rk;  // dv
  av.k = rq;
  av.v = ro;
  av.o = gv;
  av.init = dS_out;
  av.last = dS_in;
  av.reverse = 1;
  av.c_in = params->scale;
  av.c_out = 1.f;
  uint32_t* claims;
  HG_TRY(lay_out(g, 3, &claims, params, scratch, s));
  if (T == 0) return scan(&av, 1, claims, params, s);
  // side by side (three launches: 306 us for 400 histories of up to 515 events, d_h = 64), but dv by itself where it
  // leaves dS_in in the place of dS_out, which dk reads
  const int together = dS_in && dS_in == dS_out ? 2 : 3;
  HG_TRY(scan(g, together, claims, params, s));
  return together == 3 ? HG_OK : scan(&av, 1, claims, params, s);
}

namespace hg {
namespace {

template <typename T, int DH>
hg_status step_t(const hg_decay_params* p, const hg_rows* q, const hg_rows* k, const hg_rows* v, const int32_t* live,
                 int64_t n, const float* S_in, const hg_rows* o, float* S_out, cudaStream_t s) {
  return launch("decay_step", decay_step_kernel<T, DH>, dim3((unsigned)ceil_div(n * p->heads, 8)), dim3(256), 0, s,
                (const T*)q->p, q->stride, (const T*)k->p, k->stride, (const T*)v->p, v->stride, live, p->log_decay, n,
                p->heads, p->scale, S_in, (T*)o->p, o->stride, S_out);
}

template <typename T>
hg_status step_w(const hg_decay_params* p, const hg_rows* q, const hg_rows* k, const hg_rows* v, const int32_t* live,
                 int64_t n, const float* S_in, const hg_rows* o, float* S_out, cudaStream_t s) {
  if (p->d_h == 16) return step_t<T, 16>(p, q, k, v, live, n, S_in, o, S_out, s);
  if (p->d_h == 32) return step_t<T, 32>(p, q, k, v, live, n, S_in, o, S_out, s);
  if (p->d_h == 64) return step_t<T, 64>(p, q, k, v, live, n, S_in, o, S_out, s);
  return step_t<T, 128>(p, q, k, v, live, n, S_in, o, S_out, s);
}

}  // namespace
}  // namespace hg

extern "C" hg_status hg_decay_step(const hg_decay_params* params, const hg_rows* q, const hg_rows* k, const hg_rows* v,
                                   const int32_t* live, int64_t n, const float* S_in, const hg_rows* o, float* S_out,
                                   hg_stream stream) {
  clear_error();
  HG_TRY(device_guard());
  HG_TRY(check_params(params, n, 1));
  HG_REQUIRE(params->log_decay != nullptr, "log_decay must be non-null");
  if (n == 0) return HG_OK;
  const size_t esz = params->dtype == HG_BF16 ? 2 : 4;
  const int64_t w = (int64_t)params->heads * params->d_h;
  const hg_rows* in[4] = {q, k, v, o};
  const char* names[4] = {"q", "k", "v", "o"};
  for (int x = 0; x < 4; ++x) {
    HG_REQUIRE(in[x] != nullptr, "%s must be non-null", names[x]);
    const hg_seq r{in[x]->p, in[x]->stride, 0};
    HG_TRY(check_seq(&r, names[x], n, 1, w, esz, x == 3));
  }
  const hg_seq out{o->p, o->stride, 0};
  for (int x = 0; x < 3; ++x) {
    const hg_seq r{in[x]->p, in[x]->stride, 0};
    HG_TRY(check_apart(&out, "o", n, 1, w, esz, {&r}));
  }
  HG_REQUIRE(S_in && S_out, "S_in and S_out must be non-null");
  HG_REQUIRE((((uintptr_t)S_in | (uintptr_t)S_out) & 15) == 0, "S_in and S_out must be 16-byte aligned");
  HG_TRY(check_state(params, n, S_out, S_in, "S_out and S_in"));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (params->dtype == HG_F32) return step_w<float>(params, q, k, v, live, n, S_in, o, S_out, s);
  return step_w<__nv_bfloat16>(params, q, k, v, live, n, S_in, o, S_out, s);
}
