// Kernels of a key / value cache kept in pages: rows written in place, rows laid out densely, and the attention of one new
// token per sequence over the rows it holds.
//
// A pool is [pages, key heads, slots, channels]: the rows of one head in one page lie one behind another, so a workgroup
// that walks a head's keys reads runs of slots * channels elements.  Position p of sequence b is slot p % S of page
// table[b][p / S].  Rows are numbered (page * HK + h) * S + slot in 32 bits (checked when the graph is finalised); their
// elements are addressed in 64.  What the run-time tables say is bounded in the kernels: a table entry outside the pool is
// a page that is not there (its rows are neither written nor seen), positions and counts are clamped to what the table and
// the operands hold.
//
// Pools of 8 bits keep a row as whole numbers of a step of its own: step = max |x| / 127 in fp32, value = step * n with
// n = x / step rounded to the nearest whole number, halves to even - at most half a step off.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <sstream>

#include "lower_ctx.hpp"

namespace dnnf {

namespace {

// ------------------------------------------------------------------------------------------------ CacheWrite
// Pages of all sequences together that a call may write and still have every workgroup look through them: the work is their
// square, in rounds of 256.  Above, three kernels whose work is the tokens'.  Looked through and settled first, twelve heads of 64
// channels, bfloat16: one token of 2048 sequences 4.8 and 10.4 us; in pages of 16, 32 x 1024 tokens (2080 pages) 32.2 and 33.8, 64 x 1024
// 87.3 and 88.0, 64 x 2048 179 and 167.  51 x 3525 tokens of one head of 32 channels in pages of one slot would be 1.2e10 looks: 16.7 us.
constexpr int64_t kSearchedPages = 4096;

// Rows of new keys and values on their way into the pools: LANES lanes a row.
const char* kWriteRows = R"KRN(
#define VEC (16 / (int)sizeof(elem_t))
#define VECTORS(D) ((D) / VEC)
#define NEW(seq) (HAS_COUNT ? count[seq] : TOKENS)
typedef elem_t in_t __attribute__((ext_vector_type(VEC)));
typedef pool_t out_t __attribute__((ext_vector_type(VEC)));

template <int D> DEV in_t take(const elem_t* __restrict__ x, const long long src, const int lane) {
  in_t v = 0;
  if (VECTORS(D) == LANES || lane < VECTORS(D)) v = *(const in_t*)(x + src * D + lane * VEC);
  return v;
}
template <int D> DEV void put(pool_t* __restrict__ pool, float* __restrict__ scale, const in_t v, const long long dst, const int lane) {
  const bool on = VECTORS(D) == LANES || lane < VECTORS(D);
#if EIGHT_BITS
  float f[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) f[e] = cvt_in(v[e]);
  // the largest magnitude, by bits: infinities and NaN lie above all others
#if ELEM_BYTES == 2
  const u16x8 m = __builtin_bit_cast(u16x8, v) & (u16)0x7fff;
  const u16x4 m4 = __builtin_elementwise_max((u16x4){m[0], m[1], m[2], m[3]}, (u16x4){m[4], m[5], m[6], m[7]});
  const u16x2 m2 = __builtin_elementwise_max((u16x2){m4[0], m4[1]}, (u16x2){m4[2], m4[3]});
  u32 top = max((u32)m2[0], (u32)m2[1]);
#else
  u32 top = 0;
#pragma unroll
  for (int e = 0; e < VEC; ++e) top = max(top, __builtin_bit_cast(u32, f[e]) & 0x7fffffffu);
#endif
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, (u32)__shfl_xor((int)top, o, 64));
#if ELEM_BYTES == 2
  top = __builtin_bit_cast(u32, cvt_in(__builtin_bit_cast(elem_t, (u16)top)));
#endif
  // a row with an infinity or NaN reads back as NaN; one that lies wholly below 2^-119 (where the step would leave the
  // normal numbers) as zeros
  float step = __builtin_bit_cast(float, top) / 127.0f;
  if (top < 0x04000000u) step = 0.0f;
  if (top >= 0x7f800000u) step = __builtin_nanf("");
  out_t q;
  if (__builtin_amdgcn_ballot_w64(!(step >= 7.9e-31f)) != 0) {     // (rows of zeros, tiny ones, infinities and NaN)
#pragma unroll
    for (int e = 0; e < VEC; ++e) q[e] = (pool_t)(step > 0.0f ? __builtin_rintf(f[e] / step) : 0.0f);
  } else {
    // the correctly rounded quotient all the same: from the correctly rounded reciprocal, one correction by the exact
    // remainder is enough (Markstein) where that is a normal number
    const float inv = 1.0f / step;
    u32 n[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float y = f[e] * inv, z = __builtin_fmaf(__builtin_fmaf(-y, step, f[e]), inv, y);
      n[e] = __builtin_bit_cast(u32, z + 12582912.0f);          // (behind 3 * 2^22 a float's low bits are the nearest whole number)
    }
    u32 w[VEC / 4];
#pragma unroll
    for (int e = 0; e < VEC; e += 4)
      w[e / 4] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(n[e + 3], n[e + 2], 0x0c0c0400u), __builtin_amdgcn_perm(n[e + 1], n[e], 0x0c0c0400u), 0x05040100u);
    __builtin_memcpy(&q, w, sizeof q);
  }
  if (on) *(out_t*)(pool + dst * D + lane * VEC) = q;
  if (lane == 0) scale[dst] = step;
#else
  if (on) *(out_t*)(pool + dst * D + lane * VEC) = v;
#endif
}
)KRN";

const char* kWriteBody = R"KRN(
// positions [lo, hi) that a sequence writes whose operands are `f` and `n`
DEV void written(const int f, const int n, int& lo, int& hi) {
  lo = min(max(f, 0), TABLE * SLOTS);
  hi = (int)min((long long)f + min(max(n, 0), TOKENS), (long long)TABLE * SLOTS);
}
// the page that entry e of all sequences' written pages lies in, whose first position is p0; -1: nothing is written there
DEV int written_page(const int e, const int f, const int n, const int* __restrict__ table, int& lo, int& hi, int& p0) {
  written(f, n, lo, hi);
  const int lp = min(lo / SLOTS + e % SPANS, TABLE - 1);
  const int page = table[(long long)(e / SPANS) * TABLE + lp];
  p0 = lp * SLOTS;
  return lo < hi && p0 < hi && lp == lo / SLOTS + e % SPANS ? page : -1;
}
// which of the CHUNK slots from s0 on are among positions [lo, hi) of a page whose first position is p0
DEV u32 slots_of(const int lo, const int hi, const int p0, const int s0) {
  const int a = max(lo - p0 - s0, 0), z = min(hi - p0 - s0, CHUNK);
  return a < z ? (1u << z) - (1u << a) : 0u;
}

// Bound by memory for long prompts (4 x up to 1024 tokens of twelve heads of 64 channels, bfloat16: 20 MB in 5.1 us; 8 x 2048 of eight
// heads of 128: 134 MB in 20.5 us), by the chain of loads - numbers, pages, rows - for a few (2.2 us for one token of four
// sequences).  To 8 bits the quantising comes behind the loads: 2 x 37 tokens of twelve heads of 64 take 2.6 us in bfloat16 and 3.4 to
// 8 bits (3.7 behind another kernel), 8 x 2048 tokens of eight heads of 128 22.6 us for 102 MB.
// A workgroup writes CHUNK positions that lie in one page, counted from the first written one there (a page may hold a whole
// sequence: its other slots need no workgroups), for HEADS_EACH heads; LANES lanes a row.  Where one slot is written
// twice in a call the last write stays (sequences in order, then tokens): a workgroup looks through the written pages behind
// its own for its slots, 256 pages at a time.
extern "C" __global__ __launch_bounds__(256) void KNAME(KPARAMS) {
  __shared__ u32 clash;                                          // bit i: the i-th of this workgroup's positions is written again
  const int tid = threadIdx.x, unit = blockIdx.x, head0 = blockIdx.y * HEADS_EACH;
  const int entry = unit / SUBS, b = entry / SPANS;
  // (of the entry that this thread looks through as well: two rounds of loads in all, the numbers and then pages and rows)
  const int other = entry + 1 + tid, ob = min(other, SEQUENCES * SPANS - 1) / SPANS, f = first[b], n = NEW(b), of = first[ob], on = NEW(ob);
  int lo, hi;
  written(f, n, lo, hi);
  if (lo >= hi) return;
  const int lp = lo / SLOTS + entry % SPANS;
  if (lp >= TABLE) return;
  const int p0 = max(lo, lp * SLOTS) + unit % SUBS * CHUNK, p1 = min(hi, min(p0 + CHUNK, (lp + 1) * SLOTS));
  if (p0 >= p1) return;
  const int page = table[(long long)b * TABLE + lp];
  const int lane = tid % LANES, rows = (p1 - p0) * HEADS_EACH;
  in_t kx[PASSES], vx[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int r = min(tid / LANES + i * (256 / LANES), rows - 1), h = min(head0 + r % HEADS_EACH, HEADS - 1);
    const long long src = ((long long)b * TOKENS + (p0 + r / HEADS_EACH - f)) * HEADS + h;
    kx[i] = take<DK>(k, src, lane);
    vx[i] = take<DV>(v, src, lane);
  }
  int l, h, q;
  u32 later = written_page(min(other, SEQUENCES * SPANS - 1), of, on, table, l, h, q) == page && other < SEQUENCES * SPANS ? slots_of(l, h, q, p0 % SLOTS) : 0u;
  if ((u32)page >= (u32)PAGES) return;
  if (tid == 0) clash = 0;
  __syncthreads();
  for (int e = other + 256; e < SEQUENCES * SPANS; e += 256)
    if (written_page(e, first[e / SPANS], NEW(e / SPANS), table, l, h, q) == page) later |= slots_of(l, h, q, p0 % SLOTS);
  if (later) atomicOr(&clash, later);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int r = tid / LANES + i * (256 / LANES), p = p0 + r / HEADS_EACH, head = head0 + r % HEADS_EACH;
    if (r >= rows || head >= HEADS || (clash >> (p - p0) & 1u)) continue;
    const long long dst = ((long long)page * HEADS + head) * SLOTS + p % SLOTS;
    put<DK>(k_pool, k_scale, kx[i], dst, lane);
    put<DV>(v_pool, v_scale, vx[i], dst, lane);
  }
}
)KRN";

// The same for calls that write many pages, where looking through all of them from every workgroup would be work in the square of
// their number.  Which token has a slot is settled first, in an array with a place for every slot of the pool, by two kernels over the
// tokens: each token stores its number in its slot's place, then numbers above the stored one are raised into it.  Every place that
// counts has been stored to by a token of this call, so the array needs no clearing, and the largest number, the last
// token, stays whatever the order.
const char* kWriteClaimBody = R"KRN(
extern "C" __global__ __launch_bounds__(256) void KNAME(KPARAMS) {
  const u32 i = blockIdx.x * 256u + threadIdx.x, b = i / TOKENS;
  if (b >= SEQUENCES) return;
  const int t = (int)(i % TOKENS);
  const long long p = (long long)first[b] + t;
  if (t >= NEW(b) || p < 0 || p >= TABLE * SLOTS) return;
  const int page = table[(long long)b * TABLE + (int)p / SLOTS];
  if ((u32)page >= (u32)PAGES) return;
  u32* __restrict__ own = owner + ((long long)page * SLOTS + (int)p % SLOTS);
#if RAISE
  if (__hip_atomic_load(own, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < i) __hip_atomic_fetch_max(own, i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#else
  __hip_atomic_store(own, i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#endif
}
)KRN";

// The rows of the tokens that their slots belong to; a row wherever it lies, so that pages of any size fill the workgroups.
const char* kWriteOwnedBody = R"KRN(
extern "C" __global__ __launch_bounds__(256) void KNAME(KPARAMS) {
  const int lane = threadIdx.x % LANES;
  const idx_t base = (idx_t)blockIdx.x * (256 / LANES * PASSES) + threadIdx.x / LANES;
  in_t kx[PASSES], vx[PASSES];
  long long dst[PASSES];
  bool mine[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const idx_t r = base + i * (256 / LANES);
    mine[i] = false;
    dst[i] = 0;
    kx[i] = 0;
    vx[i] = 0;
    if (r >= (idx_t)SEQUENCES * TOKENS * HEADS) continue;
    const idx_t token = r / HEADS;
    const int b = (int)(token / TOKENS), t = (int)(token % TOKENS);
    const long long p = (long long)first[b] + t;
    if (t >= NEW(b) || p < 0 || p >= TABLE * SLOTS) continue;
    kx[i] = take<DK>(k, r, lane);
    vx[i] = take<DV>(v, r, lane);
    const int page = table[(long long)b * TABLE + (int)p / SLOTS];
    if ((u32)page >= (u32)PAGES) continue;
    mine[i] = owner[(long long)page * SLOTS + (int)p % SLOTS] == (u32)token;
    dst[i] = ((long long)page * HEADS + (int)(r % HEADS)) * SLOTS + (int)p % SLOTS;
  }
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    if (!mine[i]) continue;
    put<DK>(k_pool, k_scale, kx[i], dst[i], lane);
    put<DV>(v_pool, v_scale, vx[i], dst[i], lane);
  }
}
)KRN";

// ------------------------------------------------------------------------------------------------ CacheRead
const char* kReadBody = R"KRN(
#define VEC (16 / (int)sizeof(elem_t))
// Bound by memory: a thread has PER vectors on their way (8 x up to 2048 positions of eight heads of 128 channels, float16: 113 MB in
// 17 us; as much from 8 bits in 16 us).  The result is written past the caches, which it does not fit.
#define PER 4
typedef elem_t out_t __attribute__((ext_vector_type(VEC)));
typedef pool_t in_t __attribute__((ext_vector_type(VEC)));

template <int D> DEV void get(elem_t* __restrict__ out, const pool_t* __restrict__ pool, const float* __restrict__ scale,
                              const int* __restrict__ table, const int* __restrict__ held) {
  const idx_t total = (idx_t)SEQUENCES * LENGTH * HEADS * (D / VEC);
  const idx_t base = (idx_t)blockIdx.x * (256 * PER) + threadIdx.x;
  if (base >= total) return;
  in_t x[PER];
  float s[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const idx_t i = base + u * 256;
    x[u] = 0;
    s[u] = 0.0f;
    if (i >= total) continue;
    const idx_t row = i / (D / VEC);
    const int v = (int)(i % (D / VEC)), h = (int)(row % HEADS), t = (int)(row / HEADS % LENGTH), b = (int)(row / HEADS / LENGTH);
    if (t >= min(held[b], TABLE * SLOTS)) continue;
    const int page = table[(long long)b * TABLE + t / SLOTS];
    if ((u32)page >= (u32)PAGES) continue;
    const long long r = ((long long)page * HEADS + h) * SLOTS + t % SLOTS;
    x[u] = *(const in_t*)(pool + r * D + v * VEC);
#if EIGHT_BITS
    s[u] = scale[r];
#endif
  }
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const idx_t i = base + u * 256;
    if (i >= total) continue;
    out_t o;
#if EIGHT_BITS
#pragma unroll
    for (int e = 0; e < VEC; ++e) { elem_t y; cvt_out(&y, (float)x[u][e] * s[u]); o[e] = y; }
#else
    o = x[u];
#endif
    dn_store_stream((out_t*)out + i, o);
  }
}

extern "C" __global__ __launch_bounds__(256) void KNAME(KPARAMS) {
  if (blockIdx.y == 0) get<DK>(k_out, k_pool, k_scale, table, held);
  else get<DV>(v_out, v_pool, v_scale, table, held);
}
)KRN";

// ------------------------------------------------------------------------------------------------ CacheAttention
// For a query q of a head: o = sum_j p_j v_j / sum_j p_j with p_j = 2^(s_j - m), s_j = q . k_j * scale * log2(e), over the keys j
// that its sequence holds.  The keys are read once for up to sixteen query heads that share them; each further sixteen are a workgroup
// of their own that reads them again, at the same time and so mostly from the caches (131072 keys of one head of 128 channels,
// bfloat16: 21.2 us for 16 query heads, 21.6 for 24).  m may be any reference (see below).
//
// Bound by memory: one sequence of 131072 keys (eight key heads of 128 channels, bfloat16) takes 92.7 us for 537 MB, 5.8 TB/s of the
// 5.9 that a plain reading kernel reaches; sixteen sequences of 1000 to 4001 keys 39.6 us for 174 MB, 64 of 512 to 2048 in
// 8 bits 45.2 us for 174 MB - each sequence is cut into the same number of splits, so the longest is what the others wait for,
// and the first loads (numbers, pages, rows, one behind another) are not hidden.  Dealing the steps of all sequences out evenly over
// the workgroups cost more in sequences begun than it gave (43.5 -> 46 us and 47 -> 56 us with the joining); splits of one length
// for all sequences were not tried.  Elsewhere, a pass with the joining: 32768 keys of eight heads of 256 channels, bfloat16, 52.6 us
// (5.1 TB/s), in fp32 127 us (4.2 TB/s); of 128 channels in fp32 53.0 us (5.1 TB/s); 131072 keys of one head 3.2 TB/s, the 128
// splits being all of its workgroups.
//
// Four wavefronts, each with 32 keys per step.  S = K . Q^T by 16x16 MFMA: keys are the rows, the (up to 16) query heads of a
// key head the columns, so that a lane holds eight scores of one query and the softmax needs two exchanges.  Those scores,
// rounded, lie as the right operand of O^T = V^T . P^T needs them if the contraction takes the keys in the order
// 4 h .. 4 h + 3, 16 + 4 h .. (h: a lane's quarter of the wavefront); the left operand, V transposed, is the same order of keys in
// a lane's registers: every lane loads its channels of its eight keys and picks one channel of each.  Nothing but the final sums
// goes through LDS.  Each wavefront has its own maximum and sums; they are joined at the end of a workgroup's keys, and a
// second kernel joins the workgroups among which a sequence's keys were split.
const char* kAttendBody = R"KRN(
#define MASK_ALL 0xffffffffu
#define SHARE (HQ / HEADS)
#if POOL == 0
#define KV 4
#elif POOL == 1
#define KV 8
#else
#define KV (DK % 64 == 0 ? 16 : 8)
#endif
#define NC ((DK + 4 * KV - 1) / (4 * KV))          // steps along a key's channels: four quarters of KV each
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef pool_t krow_t __attribute__((ext_vector_type(KV)));

// ---- operands of the two products
#if POOL == 0
typedef float qfrag_t;
typedef float pfrag_t;
#else
typedef qelem_t qfrag_t __attribute__((ext_vector_type(8)));
typedef pelem_t pfrag_t __attribute__((ext_vector_type(8)));
#endif
DEV qelem_t to_q(float v) { return (qelem_t)v; }

// keys [begin, end) that sequence b attends over, the first step of this split and the step behind its last
DEV void span_of(const int b, const int split, const int* __restrict__ held, int& begin, int& end, int& s0, int& s1, int& splits) {
  end = min(max(held[b], 0), TABLE * SLOTS);
  begin = WINDOW > 0 ? max(0, end - WINDOW) : 0;
  const int tiles = (end + 31) / 32 - begin / 32, steps = end > begin ? (tiles + 3) / 4 : 0;
  const int per = max(1, (steps + NSPLIT - 1) / NSPLIT);
  splits = (steps + per - 1) / per;
  s0 = min(split * per, steps);
  s1 = min(s0 + per, steps);
}

// Rows that wait for their turn are held as 32-bit words (as vectors of small elements the compiler would give each element of
// a loop-carried value a register of its own).
template <int BYTES> struct words { typedef u32 t __attribute__((ext_vector_type(BYTES / 4))); };
template <> struct words<4> { typedef u32 t; };
template <> struct words<2> { typedef u16 t; };
template <> struct words<1> { typedef unsigned char t; };
template <int VW> struct vvec { typedef typename words<VW * (int)sizeof(pool_t)>::t t; typedef pool_t e __attribute__((ext_vector_type(VW))); };
template <> struct vvec<1> { typedef typename words<(int)sizeof(pool_t)>::t t; typedef pool_t e __attribute__((ext_vector_type(1))); };

// the channels BASE + VW n .. of a lane's eight keys
template <int BASE, int VW> DEV void load_values(typename vvec<VW>::t (&x)[8], const pool_t* __restrict__ vp, const long long (&vrow)[8], const int n) {
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = *(const typename vvec<VW>::t*)(vp + vrow[j] * DV + BASE + n * VW);
}
// O^T += V^T . P^T for these channels
#if POOL == 2
// (whole numbers moved to 0 .. 255 as for K; `bias`, 128 sum p below zero, is where the sums begin, and `unit` what a probability
// of the step stands for)
template <int VW, int T0> DEV void values(f32x4* o, typename vvec<VW>::t (&x)[8], const pfrag_t (&p)[PN], const f32x4 bias, const float unit) {
  u32 y[8][(VW + 3) / 4];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (VW == 8) { y[j][0] = x[j][0] ^ 0x80808080u; y[j][1] = x[j][1] ^ 0x80808080u; }
    else y[j][0] = (u32)x[j] ^ 0x80808080u;
  }
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    u32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(y[2 * i + 1][e / 4], y[2 * i][e / 4], 0x0c040c00u + 0x00010001u * (e % 4));
    f32x4 z = bias;
#pragma unroll
    for (int i = 0; i < PN; ++i) z = PV_MFMA(__builtin_bit_cast(pfrag_t, a), p[i], z, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[T0 + e][i] = __builtin_fmaf(unit, z[i], o[T0 + e][i]);
  }
}
#else
template <int VW, int T0> DEV void values(f32x4* o, typename vvec<VW>::t (&x)[8], const u32 seen, const pfrag_t (&p)[PN], const int h) {
  // a masked key's probability is zero, but zero times what its slot happens to hold (an infinity, NaN) need not be
  if (seen != MASK_ALL) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = seen >> (j / 4 * 16 + 4 * h + j % 4) & 1u ? x[j] : (typename vvec<VW>::t)0;
  }
  typename vvec<VW>::e y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = __builtin_bit_cast(typename vvec<VW>::e, x[j]);
#pragma unroll
  for (int e = 0; e < VW; ++e) {
#if POOL == 0
#pragma unroll
    for (int j = 0; j < 8; ++j) o[T0 + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[j][e], p[j], o[T0 + e], 0, 0, 0);
#else
    pfrag_t a;
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = __builtin_bit_cast(pelem_t, (u16)y[j][e]);
#pragma unroll
    for (int i = 0; i < PN; ++i) o[T0 + e] = PV_MFMA(a, p[i], o[T0 + e], 0, 0, 0);
#endif
  }
}
#endif

// what a wavefront reads in one step: 32 keys and their values
struct tile_t {
  typename words<KV * (int)sizeof(pool_t)>::t k[2][NC];
  V_MEMBERS
#if POOL == 2
  f32x4 ks[2], vs[2];
#endif
  u32 seen;                                                      // bit i: key i takes part
};

extern "C" __global__ __launch_bounds__(256, OCCUPANCY) void KNAME(KPARAMS) {
  __shared__ float Ms[4][16], Ls[4][16];
  __shared__ __attribute__((aligned(16))) float Os[4][GQ][DV + 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, h = lane >> 4;
  const int split = blockIdx.x % NSPLIT, rest = blockIdx.x / NSPLIT, q0 = rest % QTILES * 16, head = rest / QTILES % HEADS, b = rest / QTILES / HEADS;
  int begin, end, s0, s1, splits;
  span_of(b, split, held, begin, end, s0, s1, splits);
  if (NSPLIT > 1 && s0 >= s1) return;
  const int* __restrict__ row_of = table + (long long)b * TABLE;

  // this lane's query; filled while the first rows are on their way
  float q_unit = SCALE, q_bias = 0.0f;                           // (pools of 8 bits: what the scores take back, and the offset of K's rows)
  bool endless = false, any_endless = false;                     // (and: an infinity or NaN is in this lane's query, in one of the wavefront's)
#if POOL == 0
  float rq[NC][4];
#else
  qfrag_t rq[NC][KV / 8][QN];
#endif
  f32x4 o[DV / 16];
#pragma unroll
  for (int t = 0; t < DV / 16; ++t) o[t] = 0.0f;
  float m_run = -__builtin_inff(), l_run = 0.0f;

  auto page_at = [&](const int step) {
    const int lp = ((begin / 32 + step * 4 + wave) * 32 + (lane & 31)) / SLOTS;
    const int page = row_of[min(lp, TABLE - 1)];
    return step < s1 && lp < TABLE ? page : -1;
  };
  auto fetch = [&](tile_t& t, const int step, const int page) {
    const int key = (begin / 32 + step * 4 + wave) * 32 + (lane & 31);
    const bool there = (u32)page < (u32)PAGES;
    const int row = there ? (page * HEADS + head) * SLOTS + key % SLOTS : 0;
    t.seen = (u32)__builtin_amdgcn_ballot_w64(there && key >= begin && key < end);
    // rows of this lane's keys: as a row of K, and as the eight keys of its scores
    long long krow[2], vrow[8];
    krow[0] = (u32)__shfl(row, n, 64);
    krow[1] = (u32)__shfl(row, 16 + n, 64);
#if SLOTS % 4 == 0
    const long long g0 = (u32)__shfl(row, 4 * h, 64), g1 = (u32)__shfl(row, 16 + 4 * h, 64);      // (four consecutive keys share a page)
#pragma unroll
    for (int j = 0; j < 4; ++j) { vrow[j] = g0 + j; vrow[4 + j] = g1 + j; }
#else
#pragma unroll
    for (int j = 0; j < 8; ++j) vrow[j] = (u32)__shfl(row, j / 4 * 16 + 4 * h + j % 4, 64);
#endif
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int d = (c * 4 + h) * KV;
        t.k[u][c] = *(const typename words<KV * (int)sizeof(pool_t)>::t*)(k_pool + krow[u] * DK + (DK % (4 * KV) == 0 || d < DK ? d : 0));
      }
#if POOL == 2 && SLOTS % 4 == 0
    t.ks[0] = *(const f32x4*)(k_scale + g0); t.ks[1] = *(const f32x4*)(k_scale + g1);
    t.vs[0] = *(const f32x4*)(v_scale + g0); t.vs[1] = *(const f32x4*)(v_scale + g1);
#elif POOL == 2
#pragma unroll
    for (int j = 0; j < 8; ++j) { t.ks[j / 4][j % 4] = k_scale[vrow[j]]; t.vs[j / 4][j % 4] = v_scale[vrow[j]]; }
#endif
    LOAD_VALUES
  };
  auto attend = [&](tile_t& t) {
    const u32 seen = t.seen;
    if (seen == 0) return;
    // ---- scores: element i of tile u is key 16 u + 4 h + i of query n
    float s[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4 acc = 0.0f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (DK % (4 * KV) != 0 && (c * 4 + h) * KV >= DK) t.k[u][c] = 0;
        const krow_t kr = __builtin_bit_cast(krow_t, t.k[u][c]);
#if POOL == 2
        // whole numbers as they lie, moved to 0 .. 255: the low bits of a float16, n 2^-24 (the matrix units keep such numbers)
#pragma unroll
        for (int f = 0; f < KV / 8; ++f) {
          const u32 lo = t.k[u][c][f * 2] ^ 0x80808080u, hi = t.k[u][c][f * 2 + 1] ^ 0x80808080u;
          const u32x4 a = {__builtin_amdgcn_perm(0u, lo, 0x0c010c00u), __builtin_amdgcn_perm(0u, lo, 0x0c030c02u),
                           __builtin_amdgcn_perm(0u, hi, 0x0c010c00u), __builtin_amdgcn_perm(0u, hi, 0x0c030c02u)};
#pragma unroll
          for (int i = 0; i < QN; ++i) acc = QK_MFMA(__builtin_bit_cast(qfrag_t, a), rq[c][f][i], acc, 0, 0, 0);
        }
#elif POOL == 0
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[e], rq[c][e], acc, 0, 0, 0);
#else
#pragma unroll
        for (int f = 0; f < KV / 8; ++f) {
          qfrag_t a;
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] = __builtin_bit_cast(qelem_t, (u16)kr[f * 8 + e]);
#pragma unroll
          for (int i = 0; i < QN; ++i) acc = QK_MFMA(a, rq[c][f][i], acc, 0, 0, 0);
        }
#endif
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[u * 4 + i] = POOL == 2 ? __builtin_fmaf(acc[i], 16777216.0f, q_bias) * q_unit : acc[i] * SCALE;
    }
#if POOL == 2
    if (__builtin_expect(any_endless, 0)) {
      // Infinities do not stand the offset (infinity times n + 128, less infinity times 128): for such queries, whose other channels
      // do not count, the whole numbers as they are.  (64 sequences in 8 bits: 42.7 us a pass, 42.3 without this branch.)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 acc = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const krow_t kr = __builtin_bit_cast(krow_t, t.k[u][c]);
#pragma unroll
          for (int f = 0; f < KV / 8; ++f) {
            qfrag_t a;
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] = (qelem_t)(float)kr[f * 8 + e];
            acc = QK_MFMA(a, rq[c][f][0], acc, 0, 0, 0);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[u * 4 + i] = endless ? acc[i] * SCALE : s[u * 4 + i];
      }
    }
#endif
    float mx = -__builtin_inff();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
#if POOL == 2
      s[j] *= t.ks[j / 4][j % 4];
#endif
    }
    if (seen != MASK_ALL) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (!(seen >> (j / 4 * 16 + 4 * h + j % 4) & 1u)) {
          s[j] = -__builtin_inff();
#if POOL == 2
          t.vs[j / 4][j % 4] = 0.0f;
#endif
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) mx = fmaxf(mx, s[j]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    // The reference of the exponentials moves only when a row's maximum has grown by more than 2^8: until then the
    // probabilities reach at most 256, harmless in fp32 sums and in the operand, and nothing has to be rescaled.
    const float cand = fmaxf(m_run, mx);
    const bool move = cand - m_run > 8.0f;                       // (also for the first finite maximum, m_run = -inf)
    if (__builtin_amdgcn_ballot_w64(move) != 0) {
      const float m_next = move ? cand : m_run;
      const float alpha = m_next == m_run ? 1.0f : dn_exp2(m_run - m_next);
      m_run = m_next;
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < DV / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] *= alpha;
    }
    // (pools of 8 bits: 2^7 up, towards the middle of float16's range; it cancels in the quotient)
    const float m2 = (m_run == -__builtin_inff() ? 0.0f : m_run) - (POOL == 2 ? 7.0f : 0.0f);
#if POOL == 2
    // a value's step goes to its probability, relative to the largest step of these keys (float16 has the range for nothing else)
    float unit = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) unit = fmaxf(unit, __builtin_fabsf(t.vs[j / 4][j % 4]));
    unit = fmaxf(unit, __shfl_xor(unit, 16, 64));
    unit = fmaxf(unit, __shfl_xor(unit, 32, 64));
    const float per_unit = unit >= 1.17549435e-38f ? dn_rcp(unit) : 0.0f;      // (below the normal numbers it would be infinite)
#endif
    pfrag_t p[PN];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float x = dn_exp2(s[j] - m2);
      l_run += x;                                                // the sum keeps fp32
#if POOL == 2
      x *= t.vs[j / 4][j % 4] * per_unit;
#endif
#if POOL == 0
      p[j] = x;
#else
#pragma unroll
      for (int i = 0; i < PN; ++i) { p[i][j] = (pelem_t)x; x -= (float)p[i][j]; }
#endif
    }
#if POOL == 2
    f32x4 bias = 0.0f;
    pfrag_t ones;
#pragma unroll
    for (int j = 0; j < 8; ++j) ones[j] = (pelem_t)(-128.0f * 5.9604644775390625e-8f);
#pragma unroll
    for (int i = 0; i < PN; ++i) bias = PV_MFMA(ones, p[i], bias, 0, 0, 0);
#endif
    VALUES
  };
  auto query = [&] {
    // the query (behind the last one: that again, computed and not stored)
    const qin_t* __restrict__ qp = q + ((long long)b * HQ + head * SHARE + min(q0 + n, SHARE - 1)) * DK;
#if POOL == 0
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const f32x4 t = *(const f32x4*)(qp + c * 16 + h * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) rq[c][e] = t[e];
    }
#else
    float q_scale = 1.0f;
#if POOL == 2
    // queries as float16 of 2^14 at most, whatever their type's range: multiplied by a power of two, which the scores take back
    {
      u32 top = 0;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < KV; ++e)
          if (DK % (4 * KV) == 0 || (c * 4 + h) * KV < DK) top = max(top, __builtin_bit_cast(u32, cvt_in(qp[(c * 4 + h) * KV + e])) & 0x7fffffffu);
      top = max(top, (u32)__shfl_xor((int)top, 16, 64));
      top = max(top, (u32)__shfl_xor((int)top, 32, 64));
      endless = top >= 0x7f800000u;
      any_endless = __builtin_amdgcn_ballot_w64(endless) != 0;
      const int up = top == 0 || endless ? 0 : 127 + 14 - (int)(top >> 23);
      q_scale = __builtin_ldexpf(1.0f, min(up, 127));
      q_unit = __builtin_ldexpf(SCALE, -min(up, 127));
    }
#endif
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int f = 0; f < KV / 8; ++f) {
        const int d = (c * 4 + h) * KV + f * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float x = DK % (4 * KV) == 0 || d < DK ? cvt_in(qp[DK % (4 * KV) == 0 || d < DK ? d + e : 0]) * q_scale : 0.0f;
#pragma unroll
          for (int i = 0; i < QN; ++i) {
            if (endless && (i > 0 || __builtin_isfinite(x))) x = 0.0f;
            rq[c][f][i][e] = to_q(x);
            x -= (float)rq[c][f][i][e];
            q_bias += (float)rq[c][f][i][e];
          }
        }
      }
    q_bias += __shfl_xor(q_bias, 16, 64);                          // the rows of K lie 128 too high
    q_bias = -128.0f * (q_bias + __shfl_xor(q_bias, 32, 64));
#endif
  };
  int page = page_at(s0);
  tile_t t0;
  fetch(t0, s0, page);
  page = page_at(max(min(s0 + 2, s1 - 1), s0));
  int page1 = page_at(s0 + 1);
  query();
#if AHEAD
  if (s1 - s0 > 1) {
    // The next step's rows are on their way while this one's are worked on, their page numbers one step before that: all
    // wavefronts begin together, and without it they would all wait together and then all compute.  (The last step is
    // fetched once more at the end, from the caches, rather than not at all: loads behind a branch make the next wait one for
    // all of them.)
    tile_t t1;
    for (int step = s0; step < s1; step += 2) {
      fetch(t1, min(step + 1, s1 - 1), page1);
      page1 = page_at(min(step + 3, s1 - 1));
      __builtin_amdgcn_sched_barrier(0);
      attend(t0);
      fetch(t0, min(step + 2, s1 - 1), page);
      page = page_at(min(step + 4, s1 - 1));
      __builtin_amdgcn_sched_barrier(0);
      if (step + 1 < s1) attend(t1);
    }
  } else if (s0 < s1) attend(t0);
#else
  for (int step = s0; step < s1;) {
    attend(t0);
    if (++step == s1) break;
    fetch(t0, step, page1);
    page1 = page_at(step + 1);
  }
#endif

  // ---- the workgroup's four wavefronts joined
  l_run += __shfl_xor(l_run, 16, 64);
  l_run += __shfl_xor(l_run, 32, 64);
  if (h == 0) { Ms[wave][n] = m_run; Ls[wave][n] = l_run; }
  if (n < GQ) {
    OUT_TO_LDS
  }
  __syncthreads();
  for (int i = tid; i < GQ * DV; i += 256) {
    const int r = i / DV, d = i % DV;
    if (q0 + r >= SHARE) break;
    const float m = fmaxf(fmaxf(Ms[0][r], Ms[1][r]), fmaxf(Ms[2][r], Ms[3][r]));
    float l = 0.0f, x = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a = m == -__builtin_inff() ? 0.0f : dn_exp2(Ms[w][r] - m);
      l += a * Ls[w][r];
      x += a * Os[w][r][d];
    }
    if (POOL == 2) x *= 16777216.0f;                            // (the rows were in numbers of 2^-24)
    const long long at = (long long)b * HQ + head * SHARE + q0 + r;
#if NSPLIT > 1
    scratch[PART_AT + (at * NSPLIT + split) * DV + d] = x;
    if (d == 0) { scratch[(at * NSPLIT + split) * 2] = m; scratch[(at * NSPLIT + split) * 2 + 1] = l; }
#else
    qin_t y;
    cvt_out(&y, l == 0.0f ? 0.0f : x / l);                      // (no key, or all of them at -infinity: zeros)
    out[at * DV + d] = y;
#endif
  }
}
)KRN";

// (A kernel of its own, 2.8 to 4.8 us: joined by the workgroup that arrives last, the fences that make the others' sums visible
// across the eight dies' caches cost more - 9.0 -> 13.7 us for twelve heads of 1024 keys, 43 -> 162 us for the sixteen sequences.)
// Joins the splits of one query: weights 2^(m_s - m) / l, l = sum_s 2^(m_s - m) l_s.  The threads are DV / 4 vectors wide and share the
// splits among the rest.
const char* kJoinBody = R"KRN(
#define WIDE (DV / 4)
#define ROWS (256 / WIDE)
DEV void span_of(const int b, const int* __restrict__ held, int& splits) {
  const int end = min(max(held[b], 0), TABLE * SLOTS), begin = WINDOW > 0 ? max(0, end - WINDOW) : 0;
  const int tiles = (end + 31) / 32 - begin / 32, steps = end > begin ? (tiles + 3) / 4 : 0;
  const int per = max(1, (steps + NSPLIT - 1) / NSPLIT);
  splits = (steps + per - 1) / per;
}
extern "C" __global__ __launch_bounds__(256) void KNAME(KPARAMS) {
  __shared__ float w[NSPLIT], inv;
  __shared__ f32x4 part[ROWS][WIDE];
  const int tid = threadIdx.x, r = tid / WIDE, d = tid % WIDE;
  const long long at = blockIdx.x;
  // everything is asked for before it is known how many splits there are (what the others' places hold is not used)
  const f32x4* __restrict__ p = (const f32x4*)(scratch + PART_AT + at * NSPLIT * DV) + d;
  f32x4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = 0.0f; if (r < ROWS && r + i * ROWS < NSPLIT) x[i] = p[(r + i * ROWS) * WIDE]; }
  const f32x2* __restrict__ ml = (const f32x2*)(scratch + at * NSPLIT * 2);
  f32x2 both[2];                                                 // (at most 128 splits)
#pragma unroll
  for (int i = 0; i < 2; ++i) { both[i] = 0.0f; if (tid < 64 && tid + i * 64 < NSPLIT) both[i] = ml[tid + i * 64]; }
  int splits;
  span_of((int)(at / HQ), held, splits);
  if (tid < 64) {
    float m = -__builtin_inff(), ms[2], ls[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool on = tid + i * 64 < splits;
      ms[i] = on ? both[i][0] : -__builtin_inff();
      ls[i] = on ? both[i][1] : 0.0f;
      m = fmaxf(m, ms[i]);
    }
    m = dn_wave_max(m);
    float l = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float a = m == -__builtin_inff() ? 0.0f : dn_exp2(ms[i] - m);
      if (tid + i * 64 < splits) { w[tid + i * 64] = a; l += a * ls[i]; }
    }
    l = dn_wave_sum(l);
    if (tid == 0) inv = l == 0.0f ? 0.0f : 1.0f / l;             // (no key, or all of them at -infinity: zeros)
  }
  __syncthreads();
  if (r < ROWS) {
    f32x4 y = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) if (r + i * ROWS < splits) y += x[i] * w[r + i * ROWS];
    for (int s = r + 4 * ROWS; s < splits; s += 4 * ROWS) {
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[i] = 0.0f; if (s + i * ROWS < splits) x[i] = p[(s + i * ROWS) * WIDE]; }
#pragma unroll
      for (int i = 0; i < 4; ++i) if (s + i * ROWS < splits) y += x[i] * w[s + i * ROWS];
    }
    part[r][d] = y;
  }
  __syncthreads();
  if (tid < DV) {
    float y = 0.0f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) y += ((const float*)part[i])[tid];
    qin_t e;
    cvt_out(&e, y * inv);
    out[at * DV + tid] = e;
  }
}
)KRN";

Launch make_launch(const std::string& prefix, const std::string& head, const char* body, std::vector<int> params, int64_t blocks) {
  // (a launch has fewer than 2^32 threads along an axis)
  DNNF_CHECK(blocks >= 1 && blocks < ((int64_t)1 << 32) / 256, DNNF_UNSUPPORTED_OP, "cache operator: more workgroups than one launch takes");
  Launch L;
  std::string src = std::string(device_preamble()) + head + body;
  L.name = fnv_name(prefix, src);
  size_t pos;
  while ((pos = src.find("KNAME")) != std::string::npos) src.replace(pos, 5, L.name);
  L.source = src;
  L.params = std::move(params);
  L.grid[0] = (unsigned)blocks;
  L.block[0] = 256;
  return L;
}

}  // namespace

Lowered lower_cache(LowerCtx& c) {
  const Graph& g = c.g;
  DNNF_CHECK(c.blk.ops.size() == 1, DNNF_UNSUPPORTED_OP, "a cache operator is a block of its own");
  const Op& op = g.ops[c.blk.ops[0]];
  check_decode_op(g, op);
  const CacheOperands o = cache_operands(g, op);
  const OpClass cls = op.info->cls;
  // (16-bit rows that are attended over go to the matrix units as they are: plain bits)
  const int stored = g.tensors[o.pool[0]].dtype;
  const std::string pool = o.eight_bits ? "signed char" : cls == OC_CACHE_ATTN && dtype_bytes(stored) == 2 ? "u16" : c.ctype(stored);
  Lowered L;
  L.family = FAM_CACHE;
  L.ext_in = op.in;
  L.ext_out = op.out;
  std::ostringstream k;
  k << "typedef " << pool << " pool_t;\n#define EIGHT_BITS " << (int)o.eight_bits << "\n#define PAGES " << o.P << "\n#define HEADS " << o.HK << "\n#define SLOTS "
    << o.S << "\n#define DK " << o.D[0] << "\n#define DV " << o.D[1] << "\n#define SEQUENCES " << o.B << "\n#define TABLE " << o.M << "\n";
  auto scales = [&](bool written) {      // the parameters of the scales, or what stands for them in a pool without
    const std::string cst = written ? "" : "const ";
    return o.eight_bits ? ", " + cst + "float* __restrict__ k_scale, " + cst + "float* __restrict__ v_scale" : std::string();
  };
  if (!o.eight_bits) k << "#define k_scale ((float*)0)\n#define v_scale ((float*)0)\n";
  std::vector<int> params;

  if (cls == OC_CACHE_WRITE) {
    const std::string elem = c.ctype(g.tensors[o.fresh[0]].dtype);
    const int64_t vec = 16 / dtype_bytes(g.tensors[o.fresh[0]].dtype), chunk = std::min<int64_t>(o.S, 16);
    const int64_t spans = (o.T + o.S - 2) / o.S + 1, subs = (std::min(o.S, o.T) + chunk - 1) / chunk;
    int64_t lanes = 1;
    while (lanes * vec < std::max(o.D[0], o.D[1])) lanes *= 2;
    const int64_t at_once = 256 / lanes;
    k << "typedef " << elem << " elem_t;\n#define ELEM_BYTES " << 16 / vec << "\n#define TOKENS " << o.T << "\n#define LANES " << lanes << "\n#define HAS_COUNT " << (int)(o.count >= 0) << "\n";
    if (o.count < 0) k << "#define count ((const int*)0)\n";
    const std::string where = std::string("const int* __restrict__ table, const int* __restrict__ first") + (o.count >= 0 ? ", const int* __restrict__ count" : "");
    const std::string rows = "pool_t* __restrict__ k_pool, pool_t* __restrict__ v_pool" + scales(true) + ", const elem_t* __restrict__ k, const elem_t* __restrict__ v, " + where;
    params = op.out;
    params.push_back(o.fresh[0]);
    params.push_back(o.fresh[1]);
    std::vector<int> where_params = {o.table, o.first};
    if (o.count >= 0) where_params.push_back(o.count);
    params.insert(params.end(), where_params.begin(), where_params.end());
    for (size_t i = 0; i < op.out.size(); i++) L.in_place.push_back({op.out[i], op.in[i]});
    if (o.B * spans > kSearchedPages) {
      DNNF_CHECK(o.B <= (((int64_t)1 << 32) - 256) / o.T, DNNF_UNSUPPORTED_OP, "CacheWrite: 2^32 tokens or more in one call");
      const int64_t total = o.B * o.T * o.HK, passes = 4;
      k << "#define PASSES " << passes << "\ntypedef " << (total < ((int64_t)1 << 31) - at_once * passes ? "int" : "long long") << " idx_t;\n";
      for (int raise = 0; raise < 2; raise++)
        L.launches.push_back(make_launch("dnnf_cache_claim", k.str() + "#define RAISE " + std::to_string(raise) + "\n#define NEW(seq) (HAS_COUNT ? count[seq] : TOKENS)\n#define KPARAMS " + where +
                                         ", u32* __restrict__ owner\n", kWriteClaimBody, where_params, (o.B * o.T + 255) / 256));
      L.launches.push_back(make_launch("dnnf_cache_write", k.str() + "#define KPARAMS " + rows + ", const u32* __restrict__ owner\n" + kWriteRows, kWriteOwnedBody, params,
                                       (total + at_once * passes - 1) / (at_once * passes)));
      for (auto& launch : L.launches) launch.scratch = true;
      L.scratch_bytes = o.P * o.S * 4;
      L.variant = std::string("cache_write_owned") + (o.eight_bits ? "_i8" : "");
      return L;
    }
    // rows a lane: four where that leaves two workgroups per compute unit, else two or one (against all heads of sixteen tokens in a
    // workgroup: 4 x 1024 tokens of twelve heads of 64 channels, bfloat16, 5.2 and 5.1 us, to 8 bits 6.9 and 9.8; 2 x 512 of 32 heads
    // of 128 6.6 and 10.5, to 8 bits 9.6 and 39.7)
    const int64_t tokens = std::min(chunk, o.T), passes_of = o.B * o.T * o.HK / at_once;
    const int64_t want = passes_of >= 4 * 512 ? 4 : passes_of >= 2 * 512 ? 2 : 1;
    const int64_t heads = std::min(o.HK, std::max<int64_t>(1, want * at_once / tokens)), passes = (tokens * heads + at_once - 1) / at_once;
    k << "#define SPANS " << spans << "\n#define SUBS " << subs << "\n#define CHUNK " << chunk << "\n#define HEADS_EACH " << heads << "\n#define PASSES " << passes << "\n";
    k << "#define KPARAMS " << rows << "\n" << kWriteRows;
    L.launches.push_back(make_launch("dnnf_cache_write", k.str(), kWriteBody, params, o.B * spans * subs));
    L.launches[0].grid[1] = (unsigned)((o.HK + heads - 1) / heads);
    DNNF_CHECK(L.launches[0].grid[1] < 65536, DNNF_UNSUPPORTED_OP, "CacheWrite: too many heads");
    L.variant = "cache_write_chunk" + std::to_string(chunk) + (o.eight_bits ? "_i8" : "");
    return L;
  }

  params = {o.pool[0], o.pool[1]};
  if (o.eight_bits) { params.push_back(o.scale[0]); params.push_back(o.scale[1]); }
  params.push_back(o.table);
  params.push_back(o.held);
  const std::string pools = "const pool_t* __restrict__ k_pool, const pool_t* __restrict__ v_pool" + scales(false) + ", const int* __restrict__ table, const int* __restrict__ held";
  if (cls == OC_CACHE_READ) {
    const int dt = g.tensors[op.out[0]].dtype;
    const int64_t vec = 16 / dtype_bytes(dt), most = o.B * o.T * o.HK * (std::max(o.D[0], o.D[1]) / vec);
    k << "typedef " << c.ctype(dt) << " elem_t;\ntypedef " << (most < ((int64_t)1 << 31) - 1024 ? "int" : "long long") << " idx_t;\n#define LENGTH " << o.T << "\n";
    k << "#define KPARAMS " << pools << ", elem_t* __restrict__ k_out, elem_t* __restrict__ v_out\n";
    params.push_back(op.out[0]);
    params.push_back(op.out[1]);
    L.launches.push_back(make_launch("dnnf_cache_read", k.str(), kReadBody, params, (most + 1023) / 1024));
    L.launches[0].grid[1] = 2;
    L.variant = std::string("cache_read") + (o.eight_bits ? "_i8" : "");
    return L;
  }

  // ---- attention
  const int dt = g.tensors[o.q].dtype;
  const int64_t share = o.HQ / o.HK, qtiles = (share + 15) / 16;
  const int64_t window = op.i("window", 0), most = window > 0 ? std::min(window + 31, o.M * o.S) : o.M * o.S;
  const double scale = op.has("scale") ? op.f("scale", 1) : 1.0 / std::sqrt((double)o.D[0]);
  const int form = o.eight_bits ? 2 : dt == DNNF_F32 ? 0 : 1;
  const int qn = form == 2 && dt == DNNF_F32 ? 3 : 1, pn = form == 0 ? 8 : dt == DNNF_F32 ? 3 : 2;
  // A step's rows take (channels of a key + channels of a value) / 8 registers for every byte of their type, beside queries, sums
  // and the work in between; a SIMD unit has 512 for its wavefronts.  Two steps of rows where that leaves two wavefronts.
  const int64_t rows_regs = (o.D[0] + o.D[1]) * dtype_bytes(stored) / 8 + (form == 2 ? 16 : 0), other = o.D[1] / 4 + o.D[0] / 8 * (form == 0 ? 2 : qn) + 46;
  const bool ahead = 2 * rows_regs + other <= 256;
  const int64_t resident = std::max<int64_t>(1, std::min<int64_t>(4, 512 / ((ahead ? 2 : 1) * rows_regs + other)));
  // As many workgroups as the chip holds at once, with one step (128 keys) each at least at the table's capacity.  Pools of 8 bits,
  // 64 sequences of 2048, eight key heads of 128 channels: 57 us with two workgroups per compute unit, 65 with three or four (a
  // second, partly filled round); two sequences of 32768 in bfloat16 53 and 58 us.  Splits that shorter sequences do not need
  // end at once.
  const int64_t units = o.B * o.HK * qtiles, steps = (most + 127) / 128;
  const int64_t nsplit = std::max<int64_t>(1, std::min<int64_t>({steps, (256 * resident + units - 1) / units, 128}));
  k << "#define AHEAD " << (int)ahead << "\n#define OCCUPANCY " << resident << "\n";
  char num[40];
  snprintf(num, sizeof num, "%.9gf", scale * 1.4426950408889634);
  std::string sc = num;
  if (sc.find_first_of(".e") == std::string::npos) sc.insert(sc.size() - 1, ".0");
  const int64_t rows = o.B * o.HQ, part_at = (rows * nsplit * 2 + 3) / 4 * 4;
  k << "typedef " << c.ctype(dt) << " qin_t;\n#define POOL " << form << "\n#define HQ " << o.HQ << "\n#define WINDOW " << window << "\n#define NSPLIT " << nsplit
    << "\n#define QTILES " << qtiles << "\n#define GQ " << std::min<int64_t>(share, 16) << "\n#define SCALE " << sc << "\n#define PART_AT " << part_at << "\n";
  // Types of the products' operands.  Pools of 16 bits: queries and rows as they are.  Pools of 8 bits: float16, which holds the
  // rows' bytes without any arithmetic.  Probabilities are given in two parts (three for fp32 results): rounded once to
  // 8 bits they would add as much error as the rounding of the result (1.4 times its error in all), and the matrix units have
  // time for the second part.
  const std::string h16 = form == 2 || dt == DNNF_F16 ? "_Float16" : "__bf16", mf = std::string("__builtin_amdgcn_mfma_f32_16x16x32_") + (form == 2 || dt == DNNF_F16 ? "f16" : "bf16");
  k << "typedef " << (form == 0 ? "float" : h16) << " qelem_t;\ntypedef " << (form == 0 ? "float" : h16) << " pelem_t;\n#define QN " << qn << "\n#define PN " << pn
    << "\n#define QK_MFMA " << mf << "\n#define PV_MFMA " << mf << "\n";
  // a value's channels in runs of 128, 64, 32 and 16: 8, 4, 2 or 1 for each of the sixteen lanes of a quarter (fp32: 64 at most,
  // 16-byte loads)
  std::string members, loads, values, to_lds;
  int tile = 0;
  for (int64_t at = 0; at < o.D[1];) {
    int64_t w = form == 0 ? 4 : 8;
    while (w * 16 > o.D[1] - at) w /= 2;
    const std::string W = std::to_string(w), v = "v" + std::to_string(at);
    members += "  vvec<" + W + ">::t " + v + "[8]; \\\n";
    loads += "    load_values<" + std::to_string(at) + ", " + W + ">(t." + v + ", v_pool, vrow, n); \\\n";
    values += "    values<" + W + ", " + std::to_string(tile) + ">(o, t." + v + (form == 2 ? ", p, bias, unit); \\\n" : ", seen, p, h); \\\n");
    for (int64_t e = 0; e < w; e++)
      for (int i = 0; i < 4; i++)
        to_lds += "    Os[wave][n][" + std::to_string(at + e + i * w) + " + h * " + std::to_string(4 * w) + "] = o[" + std::to_string(tile + e) + "][" + std::to_string(i) + "]; \\\n";
    tile += (int)w;
    at += 16 * w;
  }
  const std::string head = k.str();
  params.insert(params.begin(), o.q);
  if (nsplit == 1) params.push_back(op.out[0]);
  const std::string main_params = "#define KPARAMS const qin_t* __restrict__ q, " + pools + (nsplit > 1 ? ", float* __restrict__ scratch" : ", qin_t* __restrict__ out") + "\n";
  L.launches.push_back(make_launch("dnnf_cache_attend", head + main_params + "#define V_MEMBERS \\\n" + members + "\n#define LOAD_VALUES \\\n" + loads + "\n#define VALUES \\\n" + values + "\n#define OUT_TO_LDS \\\n" + to_lds + "\n", kAttendBody, params, units * nsplit));
  if (nsplit > 1) {
    L.launches[0].scratch = true;
    L.scratch_bytes = (part_at + rows * nsplit * o.D[1]) * 4;
    L.launches.push_back(make_launch("dnnf_cache_join", head + "#define KPARAMS const int* __restrict__ held, qin_t* __restrict__ out, const float* __restrict__ scratch\n",
                                     kJoinBody, {o.held, op.out[0]}, rows));
    L.launches[1].scratch = true;
  }
  L.variant = "cache_attend_split" + std::to_string(nsplit) + (form == 2 ? "_i8" : form == 0 ? "_f32" : "_16");
  return L;
}

}  // namespace dnnf
