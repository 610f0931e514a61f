// Tree attention over a cache held in 4 bits (sp_fp4.h): softmax(q K^T / sqrt(d_head) + tree mask) V per (request, query head),
// K and V as the values that the cache holds, q and the result in bf16, scores and sums in float32.
//
// Work is split as in the bf16 kernel: a workgroup owns (request, KV head, block of query rows, chunk of slots), its waves cut
// the chunk into runs of 32-slot tiles, keep an online softmax each and are folded through LDS; chunks of one range are joined
// by a second kernel.  What is different is the way of a tile, which goes from memory to the matrix cores without LDS (as bf16
// tiles through LDS, a tile written once and read once by its wave, LDS set the time: 2200 cycles for a tile of each of eight
// waves):
//   S^T = K Q^T : lane (slot l % 16, kg = l / 16) takes the quarter kg of a slot's row as it lies in memory; at d_head = 128 that
//                 is the operand of v_mfma_scale, codes and scale as they are.
//   O^T = V^T P^T: needs eight slots of a column side by side.  A lane loads the same DH / 16 columns of eight slots, as many as
//                 its share of P^T holds, converts pairs of columns of a slot (one instruction, the group's scale in it), and
//                 exchanges halves of registers of neighbouring slots.
//
// What bounds it: few rows behind a short range, latencies one after the other (one row behind 500 slots 7.1-7.9 us; how they
// divide was not measured); many rows, the issue of vector instructions, the conversions of V above all, which every block of 16
// rows makes for itself (128 rows behind 8000 slots 26.1-28.0 us, 70 MB of it out of L2; 32 requests of 16-32 nodes behind 500-1000
// slots 34); few rows behind a long range, memory and the second launch (one row behind 30000 slots, 32.6 MB, 14.5 us; as a forward
// call's launches 10.6-12.8 and 4.1-4.8).
#include "sp_attn.h"
#include "sp_fp4.h"

struct Fp4AttnArgs {
  const bf16_t* q;          // [M][n_q][DH]
  const ReqTables* tables;
  KvGeom g;
  int layer, n_q, n_kv, group;
  float* part_o;            // [units][DH], followed by [units][2] (running max, sum)
  bf16_t* out;              // rows of n_q * DH columns, in fragment order or (frag false) row-major
  bool frag;
  const AttnPlan* plan;     // device copy of the call's plan; unused where the plan is an argument of the launch
};
struct NoPlan { int unused; };
template <bool VAL> struct PlanArg { typedef NoPlan type; };
template <> struct PlanArg<true> { typedef AttnPlan type; };
static_assert(sizeof(Fp4AttnArgs) + sizeof(AttnPlan) <= 4096, "kernel arguments");

// Eight values of a query row as fp8 (e4m3) pieces: hi = x / scale rounded, lo = what is left of x, 16 times as fine.
__device__ __forceinline__ void split_fp8(u32x4_t x, float scale, uint32_t (&hi)[2], uint32_t (&lo)[2]) {
  typedef __attribute__((ext_vector_type(2))) short s16x2_t;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    s16x2_t h = {0, 0}, l = {0, 0};
    const float v[4] = {bf16_lo(x[2 * i]), bf16_hi(x[2 * i]), bf16_lo(x[2 * i + 1]), bf16_hi(x[2 * i + 1])};
    h = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(h, v[0], v[1], scale, false);
    h = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(h, v[2], v[3], scale, true);
    hi[i] = __builtin_bit_cast(uint32_t, h);
    const f32x2_t b0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi[i], scale, false), b1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi[i], scale, true);
    l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, v[0] - b0[0], v[1] - b0[1], scale * 0.0625f, false);
    l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, v[2] - b1[0], v[3] - b1[1], scale * 0.0625f, true);
    lo[i] = __builtin_bit_cast(uint32_t, l);
  }
}

// The block's 16 query rows as matrix operands, and the scores of 16 slots with them.
//
// Heads of 128: v_mfma_scale takes the 4-bit codes and the groups' scales of K as they are, against 8-bit floats.  A bf16 row
// is two of those: hi, with three mantissa bits, and lo, the rest, at a sixteenth of the scale.  With the row's largest value
// in [128, 256) the two are the bf16 value exactly from 2^-13 of that value on, and off by less than 2^-21 of it below; two
// products of 128 columns then stand for four of 32 and sixteen conversions.  Lane (l15, kg) of the 8-bit operand holds columns
// kg * 16 .. + 15 and 64 + kg * 16 .. + 15.
// Heads of 64: K as bf16, four conversions a product.
template <int DH> struct Queries;
template <> struct Queries<128> {
  typedef u32x4_t codes_t;
  typedef __attribute__((ext_vector_type(8))) int i32x8_t;
  u32x4_t x[4];
  i32x8_t hi, lo;
  int scale;                                        // stored exponents: hi's in the low byte, lo's in the next
  __device__ __forceinline__ void ask(const bf16_t* row, int kg) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const u32x4_t*>(row + (i >> 1) * 64 + kg * 16 + (i & 1) * 8);
  }
  __device__ __forceinline__ void take() {
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) amax = fmaxf(amax, fmaxf(fabsf(bf16_lo(x[i][j])), fabsf(bf16_hi(x[i][j]))));
    amax = quad_rows_max(amax);
    // a row with an infinity in it has no finite weights: NaN, as its softmax is
    if (amax == INFINITY) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (u32x4_t){0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
    }
    const int e = max((int)(__float_as_uint(amax) >> 23) - 7, 5);
    const float sc = __uint_as_float((uint32_t)e << 23);
    scale = e | ((e - 4) << 8);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t h[2], l[2];
      split_fp8(x[i], sc, h, l);
#pragma unroll
      for (int j = 0; j < 2; ++j) { hi[2 * i + j] = (int)h[j]; lo[2 * i + j] = (int)l[j]; }
    }
  }
  __device__ __forceinline__ f32x4_t scores(codes_t c, uint32_t biased) const {
    const i32x8_t k = {(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0};
    const f32x4_t s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, hi, (f32x4_t){0.f, 0.f, 0.f, 0.f}, 4, 0, 0, (int)biased, 0, scale);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, lo, s, 4, 0, 0, (int)biased, 1, scale);
  }
};
template <> struct Queries<64> {
  typedef __attribute__((ext_vector_type(2))) uint32_t codes_t;
  u32x4_t q[2];
  __device__ __forceinline__ void ask(const bf16_t* row, int kg) {
#pragma unroll
    for (int s = 0; s < 2; ++s) q[s] = *reinterpret_cast<const u32x4_t*>(row + kg * 16 + s * 8);
  }
  __device__ __forceinline__ void take() {}
  __device__ __forceinline__ f32x4_t scores(codes_t c, uint32_t biased) const {
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2; ++i)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, fp4_to_bf16x8(c[i], fp4_scale(biased))),
                                                  __builtin_bit_cast(bf16x8_t, q[i]), s, 0, 0, 0);
    return s;
  }
};

__device__ __forceinline__ uint32_t lds_address(const void* p) {
#ifdef __HIP_DEVICE_COMPILE__
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
#else
  return 0u;
#endif
}
// A lane's scales out of a tile's in LDS, [K | V][32 slots][4 bytes]: K's of slots l15 and 16 + l15 at byte `k`, the words of
// V's slots kg * 4 .. + 3 and 16 + kg * 4 .. + 3 at byte `v`.  In assembly, with its wait: the words are then read, and the next
// tile's scales may take their place.
__device__ __forceinline__ void read_scales(const uint32_t* tile, int k, int v, uint32_t (&ks)[2], u32x4_t (&vs)[2]) {
  asm volatile("ds_read_u8 %0, %4\n\tds_read_u8 %1, %4 offset:64\n\tds_read_b128 %2, %5 offset:128\n\tds_read_b128 %3, %5 offset:192\n\t"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(ks[0]), "=&v"(ks[1]), "=&v"(vs[0]), "=&v"(vs[1])
               : "v"(k + lds_address(tile)), "v"(v + lds_address(tile)) : "memory");
}

// (fmaxf would first quiet NaNs, an instruction for each operand)
__device__ __forceinline__ float max_of(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// Bits 0 .. n-1 (none below 0, all from 32 on).
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

#define NW 8              // waves per workgroup
#define QR 16             // query rows per workgroup

// Four waves on a SIMD need 128 registers: a tile is a chain of dependent steps, and it is the other waves that fill it (8B shape,
// 32 requests of 16-32 nodes behind 500-1000 slots 47.0 us with three, 35.8 with four; two tiles of query rows per wave, which
// share the conversions of V, but leave room for two waves, 43.5).
template <int DH, bool PAGED>
__device__ __forceinline__ void attn_fp4(const Fp4AttnArgs& a, const AttnPlan& plan) {
  constexpr int RB = DH / 2, CW = DH / 16;         // bytes of a row's codes; columns of V in a lane
  constexpr float SC = (DH == 128 ? 0.08838834764831845f : 0.125f) * 1.4426950408889634f;    // 1 / sqrt(DH) * log2(e)
  __shared__ __attribute__((aligned(16))) float s_fold[NW * QR * DH];   // the waves' states
  __shared__ __attribute__((aligned(16))) uint32_t s_sc[NW][64];        // a tile's scales of K and V, a word per slot
  __shared__ float s_m[NW][QR];
  __shared__ float s_l[NW][QR];
  __shared__ uint32_t s_anc[QR][10];               // ancestor masks of the query rows, a word of zeros on either side

  auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int wave = uni((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l15 = lane & 15, kg = lane >> 4;
  // KV head fastest: the blocks and chunks of a head share one XCD's L2
  const int kvh = blockIdx.x, item = blockIdx.y;
  int seg = 0;
  const int n_seg = plan.n_seg, units_total = plan.units_total;
  if (n_seg > 1)                                   // each lane looks at a segment
    seg = uni(__popcll(__builtin_amdgcn_ballot_w64(lane < n_seg && item >= plan.seg_item0[lane])) - 1);
  const int chunks = plan.seg_chunks[seg], seg_rows = plan.seg_rows[seg], row0 = plan.seg_row0[seg];
  const int P = plan.seg_P[seg], span = P + plan.seg_T[seg], clen = plan.seg_clen[seg], req = plan.seg_req[seg];
  const int seg_first = plan.seg_first[seg], unit0 = plan.seg_unit0[seg];
  const int local = item - plan.seg_item0[seg];
  // (x + 0.5) / y truncates to x / y for these small integers (a range is cut only where items are fewer than CUs)
  const int qb = chunks == 1 ? local : uni((int)(((float)local + 0.5f) * __builtin_amdgcn_rcpf((float)chunks)));
  const int ch = local - qb * chunks;
  const int g = a.group;
  const int nqrows = seg_rows * g;                 // query rows of this (request, KV head): node * g + head of the group
  const int c0 = ch * clen, c1 = min(c0 + clen, span);
  const int ntiles = (c1 - c0 + 31) >> 5;
  // Waves 4 to 7 share their SIMDs with waves 0 to 3, which go first: where blocks share a range and nothing else is waited for,
  // tiles take them 0.85 us and 0.6, and they get 14 for every 18 (64 rows behind 16000 slots 33.2 -> 31.8 us, 128 behind 8000
  // 27.5 -> 26.1; ranges that a block streams for itself 18.6 -> 19.4, even shares).  Tiles left over go to the first waves.
  const int share = plan.seg_qblocks[seg] > 1 ? 18 : 16;
  auto first_tile = [&](int w) { return (ntiles * (w <= 4 ? w * share : 4 * share + (w - 4) * (32 - share)) + 127) >> 7; };
  const int w0 = c0 + 32 * first_tile(wave), w1 = min(c0 + 32 * first_tile(wave + 1), c1);

  // The query rows are asked for first, then the first tile: what is waited for comes in this order.
  const float inv_g = __uint_as_float(uni(__float_as_uint(__builtin_amdgcn_rcpf((float)g))));               // (qi + 0.5) * inv_g truncates to qi / g for these small integers
  auto node_of = [&](int qi) { return (int)(((float)qi + 0.5f) * inv_g); };
  Queries<DH> q;
  {
    const int qi = min(qb * QR + l15, nqrows - 1), nl = node_of(qi);  // (behind the last row: that row again, for nobody)
    q.ask(a.q + ((size_t)(row0 + nl) * a.n_q + (size_t)kvh * g + qi - nl * g) * DH, kg);
  }
  // ancestor masks, where the chunk has tree slots: four threads have a row's words
  unsigned long long mask_word = 0ull;
  static_assert(SP_W == 4, "a thread per word of a mask");
  if (c1 > P) {
    const int qi = qb * QR + (threadIdx.x >> 2);
    if ((int)threadIdx.x < QR * 4 && qi < nqrows) mask_word = a.tables[req].anc[seg_first + node_of(qi)][threadIdx.x & 3];
  }

  // The head's planes (at most 2 GB each: kv_slots is limited).  Slots behind the data are masked, but their values have to be
  // finite: they take the last slot's scales, and any codes are finite then.
  const int head_plane = a.layer * 2 * a.n_kv + kvh, plane_bytes = (int)a.g.plane_bytes;
  char* const k_plane = a.g.kv + (size_t)head_plane * a.g.plane_bytes;
  char* const v_plane = a.g.kv + (size_t)(head_plane + a.n_kv) * a.g.plane_bytes;
  const auto ksb = buffer_at(a.g.scales + (size_t)head_plane * a.g.scale_plane_bytes, true);
  const auto vsb = buffer_at(a.g.scales + (size_t)(head_plane + a.n_kv) * a.g.scale_plane_bytes, true);
  typedef const __attribute__((address_space(4))) int* const_int_p;
  const const_int_p pt = PAGED ? (const_int_p)(uintptr_t)(a.g.page_table + (size_t)req * a.g.pt_stride) : nullptr;
  const int pg_sh = PAGED ? a.g.pg_shift : 0, pg_mask = (1 << pg_sh) - 1;
  const int base = PAGED ? 0 : (int)plan.seg_base[seg];
  int k_at = l15 * RB + kg * (RB / 4), v_at = kg * 4 * RB + l15 * (CW / 2);
  typename Queries<DH>::codes_t kc[2];
  uint32_t vc[8];
  auto fetch = [&](int s0) {
    const int t0 = uni(min(s0, w1 - 1) & ~31);      // (past the run: its last tile again)
    const int phys = PAGED ? (pt[t0 >> pg_sh] << pg_sh) + (t0 & pg_mask) : base + t0;
    const int scale_at = (phys + min(lane & 31, span - 1 - t0)) * 4;
    if (lane < 32) load_dword_to_lds(ksb, reinterpret_cast<char*>(s_sc[wave]), scale_at);
    if (lane < 32) load_dword_to_lds(vsb, reinterpret_cast<char*>(s_sc[wave] + 32), scale_at);
    // (buffers that begin at the tile and end with the plane; what is added to the lane's offsets belongs into the loads, and not
    // into registers of its own)
    asm volatile("" : "+v"(k_at), "+v"(v_at));
    const auto kb = __builtin_amdgcn_make_buffer_rsrc(k_plane + (size_t)phys * RB, (short)0, plane_bytes - phys * RB, 0x00020000);
    const auto vb = __builtin_amdgcn_make_buffer_rsrc(v_plane + (size_t)phys * RB, (short)0, plane_bytes - phys * RB, 0x00020000);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (DH == 128) kc[h] = __builtin_amdgcn_raw_buffer_load_b128(kb, k_at + h * 16 * RB, 0, 0);
      else kc[h] = __builtin_bit_cast(Queries<64>::codes_t, __builtin_amdgcn_raw_buffer_load_b64(kb, k_at + h * 16 * RB, 0, 0));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int at = v_at + ((j >> 2) * 16 + (j & 3)) * RB;
      if constexpr (CW == 8) vc[j] = __builtin_amdgcn_raw_buffer_load_b32(vb, at, 0, 0);
      else vc[j] = __builtin_amdgcn_raw_buffer_load_b16(vb, at, 0, 0);
    }
  };
  if (w0 < w1) fetch(w0);

  q.take();
  if (c1 > P) {
    const int r = threadIdx.x >> 2, w = threadIdx.x & 3;
    if (r < QR) {
      s_anc[r][2 * w + 1] = (uint32_t)mask_word;
      s_anc[r][2 * w + 2] = (uint32_t)(mask_word >> 32);
      if (w < 2) s_anc[r][w * 9] = 0u;
    }
    __syncthreads();
  }

  // Online softmax.  The weight of a score s is exp2(s * SC + shift), -shift being a past maximum of the row's s * SC (none yet:
  // shift is the largest float, and a masked score weighs exp2(-inf) = 0 under it too).  The sums of the (rounded) weights come
  // out of the matrix cores as well: l, four times the same.
  f32x4_t o[CW], l = {0.f, 0.f, 0.f, 0.f};
  float shift = 3.4028234663852886e38f;
#pragma unroll
  for (int c = 0; c < CW; ++c) o[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  const u32x4_t ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
  int ks_at = l15 * 4 + kg * (DH / 4) / FP4_GROUP, vs_at = kg * 16;
  asm("" : "+v"(ks_at), "+v"(vs_at));
  const int v_turn = (l15 * CW / FP4_GROUP * 8 + 9) & 31;            // turns a word's byte of the lane's columns into the exponent field

  for (int s0 = w0; s0 < w1; s0 += 32) {
    SP_WAIT_VMEM(0);
    uint32_t ks[2];
    u32x4_t vs[2], vf[CW];
    read_scales(s_sc[wave], ks_at, vs_at, ks, vs);
    f32x4_t s[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) s[h] = q.scores(kc[h], ks[h]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {                   // slots 2j and 2j + 1 of the lane's eight
      const uint32_t e0 = vs[j >> 1][(j & 1) * 2], e1 = vs[j >> 1][(j & 1) * 2 + 1];
      const u32x4_t v0 = fp4_to_bf16x8(vc[2 * j], __uint_as_float(__builtin_amdgcn_alignbit(e0, e0, v_turn)));
      const u32x4_t v1 = fp4_to_bf16x8(vc[2 * j + 1], __uint_as_float(__builtin_amdgcn_alignbit(e1, e1, v_turn)));
#pragma unroll
      for (int c = 0; c < CW / 2; ++c) {
        vf[2 * c][j] = __builtin_amdgcn_perm(v1[c], v0[c], 0x05040100);
        vf[2 * c + 1][j] = __builtin_amdgcn_perm(v1[c], v0[c], 0x07060302);
      }
    }
    // Nothing uses the tile's registers any more, and the compiler is to see that: with their old contents alive it takes others
    // for the next tile, and waits for its loads at the end of the loop to move them over.
    asm volatile("" : "+v"(s[0]), "+v"(s[1]));
#pragma unroll
    for (int c = 0; c < CW; ++c) asm volatile("" : "+v"(vf[c]));
    fetch(s0 + 32);
    // A tile with tree slots, or with the end of the run: of the committed slots a row sees all, of the tree's those in its mask.
    if (s0 + 32 > P || s0 + 32 > w1) {
      const int n0 = s0 - P;
      uint32_t seen = low_bits(-n0);
      if (n0 > -32) {                               // bits of the mask from the tile's first tree index on
        asm volatile("" : "+v"(ks_at));
        const uint32_t* w = &s_anc[ks_at >> 2][(n0 >> 5) + 1];        // l15 (kept, it costs a register)
        seen |= __builtin_amdgcn_alignbit(w[1], w[0], n0 & 31);
      }
      const int bits = (int)((seen & low_bits(w1 - s0)) >> (kg * 4));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t keep = (uint32_t)((bits << (31 - ((j >> 2) * 16 + (j & 3)))) >> 31);
        s[j >> 2][j & 3] = __uint_as_float((__float_as_uint(s[j >> 2][j & 3]) & keep) | (0xff800000u & ~keep));
      }
    }
    // The shift only has to keep the weights in range: it is changed (and the sums rescaled) when some lane's would pass 2^8.
    // Changed for every larger score, it was in most of a wave's first sixteen tiles.
    const float mx = max_of(max_of(max_of(s[0][0], s[0][1], s[0][2]), s[0][3], s[1][0]), max_of(s[1][1], s[1][2], s[1][3]), s[1][3]);
    if (__builtin_amdgcn_ballot_w64(__builtin_fmaf(mx, SC, shift) > 8.f)) {
      const float top = quad_rows_max(mx) * SC;     // (its lanes see the same row)
      const float lower = fminf(shift, -top);
      const float alpha = __builtin_amdgcn_exp2f(lower - shift);
      l *= alpha;
#pragma unroll
      for (int c = 0; c < CW; ++c) o[c] *= alpha;
      shift = lower;
    }
    // The weights are rounded to bf16 here, as those over a bf16 cache are, and their sum is that of the rounded ones: each is off
    // by half a step, 2^-8 of itself, at most.  Results are 0.213-0.231 % from 64-bit ones (root mean squares, normal inputs), of
    // which 0.166 is their own rounding to bf16.  Weights as two bf16 numbers each leave those 0.166, but take every product below
    // twice: 64 rows behind 2048 slots 11.6 -> 12.6 us, 32 requests of 1-8 rows 21.9 -> 25.3, 128 rows of 64 heads 27.6 -> 32.1.
    u32x4_t pb;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      pb[j] = pack_bf16x2(__builtin_amdgcn_exp2f(__builtin_fmaf(s[j >> 1][(j & 1) * 2], SC, shift)),
                          __builtin_amdgcn_exp2f(__builtin_fmaf(s[j >> 1][(j & 1) * 2 + 1], SC, shift)));
    l = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ones), __builtin_bit_cast(bf16x8_t, pb), l, 0, 0, 0);
#pragma unroll
    for (int c = 0; c < CW; ++c)
      o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vf[c]), __builtin_bit_cast(bf16x8_t, pb), o[c], 0, 0, 0);
  }

  // The loop has asked for a tile that nobody reads: its scales have to be in LDS before the workgroup gives that away.  (Its ten
  // loads of codes came after them, and go to registers.)
  SP_WAIT_VMEM(10);

  // ---- fold the waves' states (fixed order, so results do not depend on timing) ----
  // (the lane's number is asked for again: carried through the loop, it and what comes of it cost registers)
  const int again = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), row = again & 15, part = again >> 4;
  if (part == 0) { s_m[wave][row] = -shift; s_l[wave][row] = l[0]; }
  __syncthreads();                                  // maxima and sums are posted
  // rows of DH floats, 16-byte units exchanged by the row's number
  auto fold_at = [&](int w, int unit) { return reinterpret_cast<f32x4_t*>(s_fold + (w * QR + row) * DH) + (unit ^ row); };
  {
    float top = s_m[0][row];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, s_m[w][row]);
    const float f = __builtin_amdgcn_exp2f(-shift - top);
    if (part == 0) s_l[wave][row] *= f;
    // o[c][i] is column (part * 4 + i) * CW + c of the row
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < CW; c += 4)
        *fold_at(wave, ((part * 4 + i) * CW + c) / 4) = (f32x4_t){o[c][i] * f, o[c + 1][i] * f, o[c + 2][i] * f, o[c + 3][i] * f};
  }
  __syncthreads();
  const int qi = qb * QR + row;
  if (wave >= DH / 32 || qi >= nqrows) return;      // one wave for 32 columns
  float top = s_m[0][row], lsum = 0.f;
  f32x4_t e0 = {0.f, 0.f, 0.f, 0.f}, e1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    e0 += *fold_at(w, wave * 8 + part * 2);
    e1 += *fold_at(w, wave * 8 + part * 2 + 1);
    lsum += s_l[w][row];
    top = fmaxf(top, s_m[w][row]);
  }
  // columns wave * 32 + part * 8 .. + 7 of the row
  const int nl = node_of(qi), head = kvh * g + qi - nl * g, col = wave * 32 + part * 8;
  if (chunks == 1) {
    const float inv = 1.f / lsum;
    *reinterpret_cast<u32x4_t*>(a.out + row_at(a.frag, row0 + nl, head * DH + col, a.n_q * DH)) =
        (u32x4_t){pack_bf16x2(e0[0] * inv, e0[1] * inv), pack_bf16x2(e0[2] * inv, e0[3] * inv),
                  pack_bf16x2(e1[0] * inv, e1[1] * inv), pack_bf16x2(e1[2] * inv, e1[3] * inv)};
  } else {
    const size_t unit = (size_t)unit0 + (size_t)ch * seg_rows * a.n_q + (size_t)nl * a.n_q + head;
    float* po = a.part_o + unit * DH + col;
    *reinterpret_cast<f32x4_t*>(po) = e0;
    *reinterpret_cast<f32x4_t*>(po + 4) = e1;
    if (col == 0) {
      float* ml = a.part_o + (size_t)units_total * DH + unit * 2;
      ml[0] = top; ml[1] = lsum;
    }
  }
}

template <int DH, bool PAGED, bool VAL>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(4)))
k_attn_fp4(Fp4AttnArgs a, typename PlanArg<VAL>::type plan) {
  if constexpr (VAL) attn_fp4<DH, PAGED>(a, plan);
  else attn_fp4<DH, PAGED>(a, *a.plan);
}
template <int DH, bool VAL>
__global__ void __launch_bounds__(256) k_attn_fp4_merge(Fp4AttnArgs a, int M, typename PlanArg<VAL>::type plan) {
  if constexpr (VAL) attn_merge<DH>(plan, a.part_o, a.out, a.frag, a.n_q, M);
  else attn_merge<DH>(*a.plan, a.part_o, a.out, a.frag, a.n_q, M);
}

template <int DH, bool VAL>
static hipError_t launch(const Fp4AttnArgs& a, const typename PlanArg<VAL>::type& arg, const AttnPlan& plan, int M, hipStream_t st) {
  const dim3 grid(a.n_kv, plan.total_items), block(64 * NW);
  if (a.g.page_table) hipLaunchKernelGGL((k_attn_fp4<DH, true, VAL>), grid, block, 0, st, a, arg);
  else hipLaunchKernelGGL((k_attn_fp4<DH, false, VAL>), grid, block, 0, st, a, arg);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !plan.any_split) return e;
  hipLaunchKernelGGL((k_attn_fp4_merge<DH, VAL>), dim3(((M + 7) / 8 * a.n_q + 7) / 8 * 16), dim3(256), 0, st, a, M, arg);
  return hipGetLastError();
}

hipError_t sp_launch_attn_fp4(const bf16_t* q, const ReqTables* tables, KvGeom g, int layer, const AttnPlan& plan,
                              const AttnPlan* plan_dev, float* part, bf16_t* out, bool frag, int M, int n_q, int n_kv, int d_head,
                              hipStream_t st) {
  if (!g.scales || g.row_bytes != d_head / 2 || plan.qt != 1) return hipErrorInvalidValue;
  Fp4AttnArgs a;
  a.q = q; a.tables = tables; a.g = g; a.layer = layer; a.n_q = n_q; a.n_kv = n_kv; a.group = n_q / n_kv;
  a.part_o = part; a.out = out; a.frag = frag; a.plan = plan_dev;
  if (d_head == 128) return plan_dev ? launch<128, false>(a, NoPlan{0}, plan, M, st) : launch<128, true>(a, plan, plan, M, st);
  if (d_head == 64) return plan_dev ? launch<64, false>(a, NoPlan{0}, plan, M, st) : launch<64, true>(a, plan, plan, M, st);
  return hipErrorInvalidValue;
}
