// Scan of the linear attention with decay for bf16 rows on the warp-level tensor instructions.
//
// Chunks of 16 positions.  With F the state in its frame (decay_kernels.cuh), r, j positions of a chunk:
//   rows    o_r = sum_(j <= r) gamma^(r - j) c (q_r . k_j) v_j  +  c_out gamma^(tau_r - b) q_r F
//   state   F += sum_j c_in gamma^(b - tau_j) k_j v_j^T
// A warp owns one head of one sequence (or of one segment of it) and a slice of DS value features (all of them up to
// d_h = 64: 2000 histories of 400 positions, 4 heads, 432 us with two slices of 32 against 398 us, since q k^T and the
// loads are not done twice; at 128, where a state has no place in registers, four slices), and keeps F^T (DS x d_h,
// fp32) in registers as the accumulator of m16n8k16 products: the accumulator's layout is the
// layout in which the next product wants its second operand, so the state goes from sum to operand without
// leaving the registers; likewise the chunk's weights from q k^T to the product with v.  No warp waits for
// another.  Two roundings to bf16 lie inside a row: the chunk's weights, and the state as an operand; the state itself
// stays fp32.  A row is off by 2.3e-3 of itself with them and by 1.7e-3 with its own rounding alone; a second term of
// both would take 40 products more than a chunk's 144 at d_h = 64.  The scaled values that are added to the state are
// split into three bf16 numbers, since a state is an fp32 result that gathers them (two left it 2.5e-6 off; 4e-7).
//
// Why not tcgen05: its tiles are 64 or 128 rows high, while the state of a head is d_h high, histories are often
// shorter than one tile, and the state would go through shared memory between its sum and the next product.  The
// segments' own states (kLocal) are hundreds of positions long and would suit it; they run on this kernel so far.
//
// Bound by instruction issue and latency at the warps that registers leave (16 an SM at d_h = 32, 8 above): 40001
// histories of up to 12 positions, 4 heads of 32, with their states, 188 us (0.74 of the HBM rate); 6 of 32768
// positions, 4 heads of 64, 99 us and 63 us for the segments' own states (0.6 and 0.47 of it).  At d_h = 128 the four
// slices of a head load q and k and form q k^T each for itself: 300 histories of 300, 4 heads, 181 us (0.30 of HBM; at
// d_h = 64 51 us, 0.53).  The gradients' launch at d_h = 32 keeps 24 bytes of a lane in local memory, those of the
// other widths none.
//
// Loads: cp.async, 16 bytes a lane, into a ring of chunks that runs ahead across the warp's items, so short
// histories follow one another without a pause.  Pieces of a row are XORed with the row so that ldmatrix is
// free of bank conflicts.
#include <algorithm>

#include "decay_kernels.cuh"
#include "tc_util.cuh"

namespace hg {

using namespace tc;

namespace {

constexpr int kC = 16;  // positions of a chunk
constexpr int kSms = 152;

template <int DH>
struct Cfg {
  static constexpr int DS = DH <= 64 ? DH : 32;       // value features of a warp
  static constexpr int SL = DH / DS;                 // slices of a head
  static constexpr int ST = DH == 128 ? 2 : 3;       // chunks in the ring
  static constexpr int W = 4;                        // warps of a CTA
  static constexpr int kRow = DH * 2, kVRow = DS * 2;
  static constexpr int kQ = kC * kRow, kV = kC * kVRow;
  static constexpr int kStage = 2 * kQ + kV;
  static constexpr int kSmem = W * (ST * kStage + 16);
  static constexpr int kBlocks = DH == 16 ? 5 : DH == 32 ? 4 : DH == 64 ? 2 : 2;  // resident CTAs of an SM
};

// Byte offset of 16-byte piece c of row r, N pieces a row.
// 2 x pieces further on is an XOR with 32 x, for rows' places that begin at a multiple of their size.
template <int N>
__device__ __forceinline__ uint32_t piece(int r, int c) {
  constexpr int sh = N == 2 ? 2 : N == 4 ? 1 : 0;
  constexpr int mask = (N < 8 ? N : 8) - 1;
  return (uint32_t)(r * N + (c ^ ((r >> sh) & mask))) * 16u;
}

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// d += A (16 x 16) B (16 x 8)
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
      "%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// One warp's piece of work: positions [t0, t1) of the scan of a head (segment segi), value features slice * DS on.
struct Item {
  uint32_t id;  // at or past the number of items: none
  uint32_t seq, unit;
  int set, head, slice, segi;
  int len, t0, t1;
};

template <int DH, bool kMany>
__device__ __forceinline__ void locate(const ScanArgs& a, uint32_t items, uint32_t each, uint32_t segs, Item& it) {
  if (it.id >= items) {
    it.t0 = it.t1 = 0;
    return;
  }
  constexpr uint32_t SL = Cfg<DH>::SL;
  it.set = kMany ? (int)(it.id / each) : 0;
  const uint32_t id = kMany ? it.id % each : it.id;
  it.slice = (int)(id % SL);
  uint32_t x = id / SL;
  it.head = (int)(x % (uint32_t)a.heads);
  x /= (uint32_t)a.heads;
  it.segi = 0;
  if (segs > 1) {
    it.segi = (int)(x % segs);
    x /= segs;
  }
  it.seq = x;
  it.len = (int)scan_len(a, x);
  it.t0 = it.segi * (int)a.seg_len;
  it.t1 = max(it.t0, min(it.t0 + (int)a.seg_len, it.len));
}

// Where a lane's 16-byte pieces of an array's rows start and how far apart the rows of the scan lie, in bytes
// (negative in reverse).  P pieces a row: the lane takes piece lane % P of rows lane / P + i (32 / P).
template <int P>
__device__ __forceinline__ const uint8_t* lane_rows(const ScanRows& r, const ScanArgs& a, const Item& it, int t,
                                                    int col, int lane) {
  const int row = a.reverse ? it.len - 1 - t - lane / P : t + lane / P;
  return static_cast<const uint8_t*>(r.p) + 2 * ((int64_t)it.seq * r.sn + row * r.st + col + lane % P * 8);
}
__device__ __forceinline__ int64_t row_step(const ScanRows& r, const ScanArgs& a) {
  return a.reverse ? -2 * r.st : 2 * r.st;
}

// The lane's pieces of kC rows, m of them in use (the others are not read and become zero), to dst.
template <int P>
__device__ __forceinline__ void load_rows(uint8_t* dst, const uint8_t* src, int64_t step, int m, int lane) {
  constexpr int RS = 32 / P;
#pragma unroll
  for (int i = 0; i < kC / RS; ++i) {
    const int r = lane / P + i * RS;
    uint8_t* at = dst + piece<P>(r, lane % P);
    if (r < m)
      cp_async16(at, src + i * (RS * step), true);
    else
      st16(at, make_uint4(0u, 0u, 0u, 0u));
  }
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// two products, two differences
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 c;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "mul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(c.x), "=f"(c.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return c;
}
__device__ __forceinline__ float2 sub2(float2 a, float2 b) {
  float2 c;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "sub.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(c.x), "=f"(c.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return c;
}
__device__ __forceinline__ float2 wide(uint32_t x) {
  return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}

// z (zeros), NaN in the half where x is not finite
__device__ __forceinline__ uint32_t times_zero(uint32_t x, uint32_t z) {
  asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(z) : "r"(x), "r"(0u));
  return z;
}

// x (a pair of bf16) times f as a sum of three bf16 pairs
__device__ __forceinline__ void scale_split(uint32_t x, float2 f, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  float2 y = mul2(wide(x), f);
  hi = pack2_bf16(y.x, y.y);
  y = sub2(y, wide(hi));
  mid = pack2_bf16(y.x, y.y);
  y = sub2(y, wide(mid));
  lo = pack2_bf16(y.x, y.y);
}

// kMany: the items of several scans over the same sequences, scan by scan.
template <int DH, bool kLocal, bool kMany>
__global__ void __launch_bounds__(32 * Cfg<DH>::W, Cfg<DH>::kBlocks)
    scan_mma_kernel(const __grid_constant__ ScanBatch batch) {
  pdl_begin();
  const ScanArgs& all = batch.s[0];  // what the scans have in common
  auto scan_of = [&](const Item& it) -> const ScanArgs& { return batch.s[kMany ? it.set : 0]; };
  using C = Cfg<DH>;
  constexpr int DS = C::DS, MT = DS / 16, NT = DH / 8, KS = DH / 16, NV = DS / 8, N = DH / 8, ST = C::ST;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  uint8_t* ring = smem + warp * (ST * C::kStage);
  const uint32_t segs = kLocal ? all.nseg - 1 : all.nseg;
  const uint32_t each = (uint32_t)all.n * segs * all.heads * C::SL, items = kMany ? each * batch.count : each;
  const uint32_t stride = gridDim.x * C::W;
  // lane addresses inside a tile of 16 x 16 for ldmatrix: rows by lane & 15 / pieces by lane >> 4, and the other order
  const int r16 = lane & 15, c16 = lane >> 4;
  const int r8 = (lane & 7) + ((lane >> 4) << 3), c8 = (lane >> 3) & 1;

  // Items by turns, or, where a counter is given, as they are claimed: the loads run ahead, so the claimed numbers (or,
  // by turns, the lengths) wait in a queue for the arithmetic.
  uint32_t* queue = reinterpret_cast<uint32_t*>(smem + C::W * ST * C::kStage) + warp * 4;
  uint32_t queued = 0, taken = 0;
  auto enqueue = [&](uint32_t x) {
    if (lane == 0) queue[queued & 3] = x;
    ++queued;
    __syncwarp();
  };
  auto next_id = [&](uint32_t id) -> uint32_t {
    if (!all.claims) return id + stride;
    uint32_t x = 0;
    if (lane == 0) x = atomicAdd(all.claims, 1u);
    x = __shfl_sync(0xffffffffu, x, 0) + stride;
    enqueue(x);
    return x;
  };
  auto follow = [&](uint32_t id) -> uint32_t { return all.claims ? queue[taken++ & 3] : id + stride; };
  // Items dealt out without segments follow each other by steps in (scan, sequence, unit = head and slice): carries
  // replace divisions, and the length of the item after the next is asked for early (40001 histories of up to 12
  // positions, 4 heads of 32: 188 us, with divisions and lengths asked for when needed 222 us).
  const bool steps = !kLocal && !all.claims && segs == 1;
  const uint32_t units = all.heads * C::SL, step_seq = stride / units, step_unit = stride % units;
  auto bump = [&](int& set, uint32_t& seq, uint32_t& unit) {
    seq += step_seq;
    unit += step_unit;
    if (unit >= units) {
      unit -= units;
      ++seq;
    }
    if (kMany)
      for (; seq >= (uint32_t)all.n && set < batch.count; ++set) seq -= (uint32_t)all.n;
  };
  auto use = [&](Item& x, int len) {
    x.t1 = 0;
    if (x.id >= items) return;
    x.head = (int)(x.unit / C::SL);
    x.slice = (int)(x.unit % C::SL);
    x.len = x.t1 = min(max(len, 0), (int)all.T);
  };
  int far_set = 0, far_len = 0;
  uint32_t far_seq = 0, far_unit = 0;
  auto look = [&]() { far_len = !all.lens ? (int)all.T : far_seq < (uint32_t)all.n ? all.lens[far_seq] : 0; };
  Item it{}, nx{};
  it.id = blockIdx.x * C::W + warp;
  locate<DH, kMany>(all, items, each, segs, it);
  // The loads run ahead: position nc of item nx is the next chunk to ask for.  An item without positions passes as one
  // empty chunk, so the loads are at most a ring ahead of the arithmetic.
  const uint8_t *qp = nullptr, *kp = nullptr, *vp = nullptr;
  int nc = 0;
  int64_t qs = row_step(all.q, all), ks = row_step(all.k, all), vs = row_step(all.v, all);
  auto begin = [&]() {
    nc = nx.t0;
    if (nx.id >= items || nx.t0 >= nx.t1) return;
    const ScanArgs& a = scan_of(nx);
    if (kMany) {
      qs = row_step(a.q, a);
      ks = row_step(a.k, a);
      vs = row_step(a.v, a);
    }
    if (!kLocal) qp = lane_rows<N>(a.q, a, nx, nc, nx.head * DH, lane);
    kp = lane_rows<N>(a.k, a, nx, nc, nx.head * DH, lane);
    vp = lane_rows<NV>(a.v, a, nx, nc, nx.head * DH + nx.slice * DS, lane);
  };
  if (steps) {
    it.unit = it.id % units;
    far_set = it.set;
    far_seq = it.seq;
    far_unit = it.unit;
    bump(far_set, far_seq, far_unit);
    look();
  }
  nx = it;
  begin();
  auto advance = [&](uint8_t* stage) {
    if (nx.id < items && nc >= max(nx.t1, nx.t0 + 1)) {
      if (steps) {
        nx.id += stride;
        nx.set = far_set;
        nx.seq = far_seq;
        nx.unit = far_unit;
        use(nx, far_len);
        enqueue((uint32_t)nx.t1);
        bump(far_set, far_seq, far_unit);
        look();
      } else {
        nx.id = next_id(nx.id);
        locate<DH, kMany>(all, items, each, segs, nx);
      }
      begin();
    }
    if (nx.id < items) {
      const int m = min(kC, nx.t1 - nc);
      nc += kC;
      if (m > 0) {
        if (!kLocal) load_rows<N>(stage, qp, qs, m, lane);
        load_rows<N>(stage + C::kQ, kp, ks, m, lane);
        load_rows<NV>(stage + 2 * C::kQ, vp, vs, m, lane);
        qp += kC * qs;
        kp += kC * ks;
        vp += kC * vs;
      }
    }
    cp_async_commit();
  };
  int put = 0, get = 0;
#pragma unroll
  for (int s = 0; s < ST - 1; ++s) {
    advance(ring + put * C::kStage);
    put = put + 1 == ST ? 0 : put + 1;
  }
  auto go_on = [&]() {
    if (steps) {
      it.id += stride;
      bump(it.set, it.seq, it.unit);
      use(it, (int)queue[taken++ & 3]);
    } else {
      it.id = follow(it.id);
      locate<DH, kMany>(all, items, each, segs, it);
    }
  };
  for (; it.id < items; go_on()) {
    const ScanArgs& a = scan_of(it);
    const int64_t os = row_step(a.o, a);
    const float ld = clamp_ld(a.ld[it.head]), ld2 = ld * 1.4426950408889634f;
    const int64_t sh = (int64_t)it.seq * a.heads + it.head;
    float F[MT][NT][4];
    // element e of F[x][y]: value feature 16 x + g + 8 (e / 2) of the slice, key feature 8 y + 2 t4 + e % 2
    const int v0 = it.slice * DS + g, k0 = 2 * t4;
    bool some = false;  // the state is not zero
    if (!kLocal && (a.nseg > 1 || a.init)) {
      const float* src = a.nseg > 1 ? a.seg + (sh * a.nseg + it.segi) * (int64_t)(DH * DH) : a.init + sh * (DH * DH);
      const bool tr = a.nseg > 1 ? false : a.init_t != 0;
      some = true;
#pragma unroll
      for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int y = 0; y < NT; ++y)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int vi = v0 + 16 * x + 8 * (e >> 1), ki = k0 + 8 * y + (e & 1);
            F[x][y][e] = tr ? src[vi * DH + ki] : src[ki * DH + vi];
          }
    } else {
#pragma unroll
      for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int y = 0; y < NT; ++y)
#pragma unroll
          for (int e = 0; e < 4; ++e) F[x][y][e] = 0.f;
    }
    // weights gamma^(r - j) of the chunk's products: rows g, g + 8, columns 2 t4, 2 t4 + 1 (+ 8)
    float w[4];
    const bool keep0 = g >= 2 * t4, keep1 = g >= 2 * t4 + 1;  // the column is not past row g
    if (!kLocal) {
      const float cc = a.c_in * a.c_out;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float gap = (float)(g - 2 * t4 - e);
        w[e] = (e ? keep1 : keep0) ? ex2(ld2 * gap) * cc : 0.f;  // row g, column j; row g + 8, column j + 8
        w[2 + e] = ex2(ld2 * (gap + 8.f)) * cc;                  // row g + 8, column j
      }
    }
    int base = 0;  // positions from t0
    const bool leave = kLocal || (a.last && it.segi == (it.len > 0 ? (it.len - 1) / (int)a.seg_len : 0));
    uint8_t* op = nullptr;
    if (!kLocal) op = const_cast<uint8_t*>(lane_rows<NV>(a.o, a, it, it.t0, it.head * DH + it.slice * DS, lane));
    const int count = it.t1 - it.t0;
    for (int c0 = 0; c0 < max(count, 1); c0 += kC) {
      cp_async_wait<ST - 2>();
      __syncwarp();
      advance(ring + put * C::kStage);
      put = put + 1 == ST ? 0 : put + 1;
      uint8_t* stage = ring + get * C::kStage;
      get = get + 1 == ST ? 0 : get + 1;
      const uint32_t sq = smem_u32(stage), sk = sq + C::kQ, sv = sk + C::kQ;
      const int m = min(kC, count - c0);
      if (m <= 0) break;
      const int tau0 = c0 + a.shift;
      uint32_t vt[MT][4];  // v, positions by pairs: [0], [2] positions 0..7 / 8..15 of features 0..7; [1], [3] of 8..15
#pragma unroll
      for (int x = 0; x < MT; ++x) {
        uint32_t b[4];
        ldsm4t((sv + piece<NV>(r16, c16)) ^ (x * 32), b);
        vt[x][0] = b[0];
        vt[x][2] = b[1];
        vt[x][1] = b[2];
        vt[x][3] = b[3];
      }
      if (!kLocal) {
        float o[NV][4], p0[4] = {0.f, 0.f, 0.f, 0.f}, p1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < NV; ++y)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[y][e] = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          uint32_t qa[4], kb[4];
          ldsm4((sq + piece<N>(r16, c16)) ^ (s * 32), qa);
          ldsm4((sk + piece<N>(r8, c8)) ^ (s * 32), kb);
          mma(p0, qa[0], qa[1], qa[2], qa[3], kb[0], kb[1]);
          mma(p1, qa[0], qa[1], qa[2], qa[3], kb[2], kb[3]);
          if (some) {
#pragma unroll
            for (int y = 0; y < NV; ++y) {
              const float* f0 = F[y >> 1][2 * s];
              const float* f1 = F[y >> 1][2 * s + 1];
              const int e = (y & 1) * 2;
              mma(o[y], qa[0], qa[1], qa[2], qa[3], pack2_bf16(f0[e], f0[e + 1]), pack2_bf16(f1[e], f1[e + 1]));
            }
          }
        }
        if (some) {
          const float x = (float)(tau0 + g - base);
          const float f0 = a.c_out * ex2(ld2 * x), f1 = a.c_out * ex2(ld2 * (x + 8.f));
#pragma unroll
          for (int y = 0; y < NV; ++y) {
            const float2 u = mul2(make_float2(o[y][0], o[y][1]), make_float2(f0, f0));
            const float2 v = mul2(make_float2(o[y][2], o[y][3]), make_float2(f1, f1));
            o[y][0] = u.x;
            o[y][1] = u.y;
            o[y][2] = v.x;
            o[y][3] = v.y;
          }
        }
        const uint32_t a0 = pack2_bf16(keep0 ? p0[0] * w[0] : 0.f, keep1 ? p0[1] * w[1] : 0.f);
        const uint32_t a1 = pack2_bf16(p0[2] * w[2], p0[3] * w[3]);
        const uint32_t a3 = pack2_bf16(keep0 ? p1[2] * w[0] : 0.f, keep1 ? p1[3] * w[1] : 0.f);
        // The product multiplies later positions with zeros, which an infinity or NaN would turn into NaN: a chunk that
        // holds one goes position by position, each row as far as its own.  (To look for one costs 1 to 3 %: 2000
        // histories of 400 positions, 4 heads of 64, 381 -> 385 us; 4000 of 100, 4 of 32, 82 -> 84 us.)
        uint32_t odd[2] = {0u, 0u};
#pragma unroll
        for (int x = 0; x < MT; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) odd[e & 1] = times_zero(vt[x][e], odd[e & 1]);
        if (!__any_sync(0xffffffffu, (odd[0] | odd[1]) != 0u)) {
#pragma unroll
          for (int y = 0; y < NV; ++y) mma(o[y], a0, a1, 0u, a3, vt[y >> 1][y & 1], vt[y >> 1][2 + (y & 1)]);
        } else {
#pragma unroll 1
          for (int j = 0; j < kC; ++j) {
            // this lane's rows are g and g + 8; the weights of column j are with lane j % 8 / 2 of its four
            const int from = (lane & 28) | ((j & 7) >> 1);
            const uint32_t u = __shfl_sync(0xffffffffu, j < 8 ? a0 : 0u, from);
            const uint32_t l = __shfl_sync(0xffffffffu, j < 8 ? a1 : a3, from);
            const float w0 = j & 1 ? wide(u).y : wide(u).x, w1 = j & 1 ? wide(l).y : wide(l).x;
#pragma unroll
            for (int y = 0; y < NV; ++y) {
              const float2 v = wide(*reinterpret_cast<const uint32_t*>(stage + 2 * C::kQ + piece<NV>(j, y) + t4 * 4));
              if (j <= g) {
                o[y][0] = fmaf(w0, v.x, o[y][0]);
                o[y][1] = fmaf(w0, v.y, o[y][1]);
              }
              if (j <= g + 8) {
                o[y][2] = fmaf(w1, v.x, o[y][2]);
                o[y][3] = fmaf(w1, v.y, o[y][3]);
              }
            }
          }
        }
        // rows out through the place of q, 16 bytes a lane
        __syncwarp();
#pragma unroll
        for (int y = 0; y < NV; ++y) {
          *reinterpret_cast<uint32_t*>(stage + piece<NV>(g, y) + t4 * 4) = pack2_bf16(o[y][0], o[y][1]);
          *reinterpret_cast<uint32_t*>(stage + piece<NV>(g + 8, y) + t4 * 4) = pack2_bf16(o[y][2], o[y][3]);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kC * NV / 32; ++i) {
          const int r = lane / NV + i * (32 / NV);
          if (r < m) st16(op + i * (32 / NV) * os, ld16(stage + piece<NV>(r, lane % NV)));
        }
        op += kC * os;
      }
      if (leave || c0 + kC < count) {
        const int target = tau0 + m - 1;
        if (c0 + kC >= count || (float)(base - target) * ld > kFrame) {  // a state that leaves ends its frame
          if (some) {
            const float f = ex2(ld2 * (float)(target - base));
#pragma unroll
            for (int x = 0; x < MT; ++x)
#pragma unroll
              for (int y = 0; y < NT; ++y)
#pragma unroll
                for (int e = 0; e < 4; ++e) F[x][y][e] *= f;
          }
          base = target;
        }
        float2 f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = 2 * t4 + 8 * e;
          f[e].x = r < m ? a.c_in * ex2(ld2 * (float)(base - tau0 - r)) : 0.f;
          f[e].y = r + 1 < m ? a.c_in * ex2(ld2 * (float)(base - tau0 - r - 1)) : 0.f;
        }
        constexpr int XB = MT < 2 ? MT : 2;  // groups of 16 value features at a time: registers for their terms
#pragma unroll
        for (int x0 = 0; x0 < MT; x0 += XB) {
          uint32_t hi[XB][4], mid[XB][4], lo[XB][4];
#pragma unroll
          for (int x = 0; x < XB; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) scale_split(vt[x0 + x][e], f[e >> 1], hi[x][e], mid[x][e], lo[x][e]);
#pragma unroll
          for (int y = 0; y < NT; y += 2) {
            uint32_t kb[4];
            ldsm4t((sk + piece<N>(r16, c16)) ^ (y * 16), kb);
#pragma unroll
            for (int x = 0; x < XB; ++x) {
              auto& f0 = F[x0 + x][y];
              auto& f1 = F[x0 + x][y + 1];
              mma(f0, hi[x][0], hi[x][1], hi[x][2], hi[x][3], kb[0], kb[1]);
              mma(f1, hi[x][0], hi[x][1], hi[x][2], hi[x][3], kb[2], kb[3]);
              mma(f0, mid[x][0], mid[x][1], mid[x][2], mid[x][3], kb[0], kb[1]);
              mma(f1, mid[x][0], mid[x][1], mid[x][2], mid[x][3], kb[2], kb[3]);
              mma(f0, lo[x][0], lo[x][1], lo[x][2], lo[x][3], kb[0], kb[1]);
              mma(f1, lo[x][0], lo[x][1], lo[x][2], lo[x][3], kb[2], kb[3]);
            }
          }
        }
        some = true;
      }
    }
    if (!kLocal) {
      const int tend = min(it.t0 + (int)a.seg_len, (int)a.T), first = max(it.t0, it.len);
      uint8_t* zp = static_cast<uint8_t*>(const_cast<void*>(a.o.p)) +
                    2 * ((int64_t)it.seq * a.o.sn + (first + lane / NV) * a.o.st + it.head * DH + it.slice * DS +
                         lane % NV * 8);
      for (int t = first + lane / NV; t < tend; t += 32 / NV, zp += (32 / NV) * 2 * a.o.st)
        st16(zp, make_uint4(0u, 0u, 0u, 0u));
    }
    if (leave) {
      if (base != count) {  // shift 0
        const float f = ex2(ld2 * (float)(count - base));
#pragma unroll
        for (int x = 0; x < MT; ++x)
#pragma unroll
          for (int y = 0; y < NT; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e) F[x][y][e] *= f;
      }
      float* dst = kLocal ? a.seg + (sh * a.nseg + it.segi) * (int64_t)(DH * DH) : a.last + sh * (DH * DH);
#pragma unroll
      for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int y = 0; y < NT; ++y)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            dst[(k0 + 8 * y + (e & 1)) * DH + v0 + 16 * x + 8 * (e >> 1)] = F[x][y][e];
    }
  }
  cp_async_wait<0>();
}

template <int DH, bool kLocal, bool kMany>
hg_status scan_mma_t(const ScanBatch& b, cudaStream_t s) {
  using C = Cfg<DH>;
  static bool done = false;
  if (!done) {
    HG_CUDA(cudaFuncSetAttribute(scan_mma_kernel<DH, kLocal, kMany>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 C::kSmem));
    done = true;
  }
  const ScanArgs& a = b.s[0];
  const int64_t items = a.n * (kLocal ? a.nseg - 1 : a.nseg) * a.heads * C::SL * b.count;
  const int64_t grid = std::min<int64_t>(ceil_div(items, C::W), kSms * C::kBlocks);
  return launch(kLocal ? "decay_scan_local_mma" : "decay_scan_mma", scan_mma_kernel<DH, kLocal, kMany>,
                dim3((unsigned)grid), dim3(32 * C::W), C::kSmem, s, b);
}

template <int DH>
hg_status scan_mma_d(const ScanBatch& b, bool local, cudaStream_t s) {
  if (b.count > 1) return local ? scan_mma_t<DH, true, true>(b, s) : scan_mma_t<DH, false, true>(b, s);
  return local ? scan_mma_t<DH, true, false>(b, s) : scan_mma_t<DH, false, false>(b, s);
}

}  // namespace

hg_status scan_mma(const ScanBatch& b, int d_h, bool local, cudaStream_t s) {
  if (d_h == 16) return scan_mma_d<16>(b, local, s);
  if (d_h == 32) return scan_mma_d<32>(b, local, s);
  if (d_h == 64) return scan_mma_d<64>(b, local, s);
  return scan_mma_d<128>(b, local, s);
}

int scan_mma_warps(int heads, int d_h) { return heads * (d_h <= 64 ? 1 : d_h / 32); }

int scan_mma_resident(int d_h) {
  if (d_h == 16) return Cfg<16>::W * Cfg<16>::kBlocks;
  if (d_h == 32) return Cfg<32>::W * Cfg<32>::kBlocks;
  if (d_h == 64) return Cfg<64>::W * Cfg<64>::kBlocks;
  return Cfg<128>::W * Cfg<128>::kBlocks;
}

}  // namespace hg
