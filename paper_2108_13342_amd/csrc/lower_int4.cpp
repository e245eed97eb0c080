// Products with weights of four bits: y[m, n] = sum_k x[m, k] * (code[n, k] - zero[n, k / G]) * scale[n, k / G], for the few rows of
// single-token inference.  The block may hold One-to-One operators, Reshapes and Splits behind the product, as behind MatMul.
//
// What bounds it: the weights, half a byte each and read once; everything else has to stay out of their way.  (Sizes here are rows of x,
// then K x N; groups of 128 with zero points, bfloat16, where nothing else is said.)
//   - A code becomes an operand of the matrix units by two instructions for two codes: shifted into the mantissa of 16 it is the
//     number 16 + code, exactly, in float16 and bfloat16 alike.  The product of a group is then taken as
//     sum x (16 + code) - (16 + zero) sum x; the row sums of x come from the matrix units too (a column of ones), in the layout
//     that the results have, so that a group costs two fp32 instructions per result.  (Infinite or NaN x: the row is NaN.)
//   - The order of k within a contraction step is free as long as both operands have the same: a lane takes the codes in the order
//     in which they leave a 32-bit word (0, 4, 1, 5, 2, 6, 3, 7), and x is picked in that order.
//   - A wavefront reads 16 weight rows, 16 bytes a lane: 128 codes a row.  In groups of 128 and more, x in LDS, a lane's 32
//     codes go into four steps as they are (each step meets all four quarters of the run).  Smaller groups have to meet 32 successive
//     codes in a step: four exchanges between the wavefront's quarters turn the 4 x 4 words around.  So they do where x comes from
//     memory: a load then touches 64 bytes of each of its rows and not 16 of every 64 (16 rows, 11008 x 4096: 17.2 us, 20.7 unturned).
//   - Scales and zeros lie a row of groups apart: a load of theirs touches sixteen lines, and such loads, not bytes, are what a
//     compute unit runs out of.  Where groups fill a chunk evenly, one vector holds all that the chunk needs.  Elsewhere (groups of
//     96, an odd count) each quarter of the wavefront loads the group of its own quarter of the chunk, and exchanges give it to all: 16 rows,
//     4096 x 11008 in groups of 96: 13.8 us, 39.5 with a load for every part.  (In groups of 32, 4096 x 4096, the vector takes 7.8 us, the
//     exchanges 8.6.)
//   - fp32 x is taken in three bfloat16 parts, which hold all of its 24 bits; weights are exact in either case.
// One row of 4096 x 11008: 23.6 MB in 8.8 us, 2.7 TB/s; 16 rows of 768 x 50257 without zero points 21.5 MB in 9.3 us.  A compute unit holds two
// workgroups of sixteen wavefronts, and what does not fit the 512 places waits for a second round that begins with its loads
// again: one row of 4096 x 4096 takes 4.1 us, x 8192 (512 workgroups) 6.5, x 8208 8.1, x 11008 8.8, x 12288 9.1.  With weights that come from
// memory, not from the memory-side cache: 9.4 us for x 11008, 10.3 for the 16 rows.
// From 17 rows on every tile of sixteen rows decodes the weights again: 4096 x 4096 takes 13.4 us for 64 rows, 94 for 512, 360 for 2048 (191 TFLOP/s).
// The wavefronts of a workgroup share its columns and split K among them; sums are joined in LDS in a fixed order.
#include <algorithm>
#include <sstream>

#include "lower_ctx.hpp"

namespace dnnf {

namespace {

const char* kInt4Body = R"KRN(
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_any __attribute__((aligned(4)));
typedef u32x4 u32x4_byte __attribute__((aligned(1)));
typedef elem_t xvec_t __attribute__((ext_vector_type(8), aligned(ELEM_BYTES)));
typedef part_t frag_t __attribute__((ext_vector_type(8)));
#define CHUNK 128                                  // codes of a row that a wavefront reads at once
#define CHUNKS ((GK + CHUNK - 1) / CHUNK)
#define ROW_BYTES ((GK + 1) / 2)
#define PARTS_OF_CHUNK (4 / STEPS)                 // groups, or pieces of one, in a chunk
#define ROWS (GM < 16 ? GM : 16)

// what a lane reads of a chunk's scales and zeros: those of all its parts or, to SPREAD, those of quarter h's group
#define READ (SPREAD ? 1 : PARTS_OF_CHUNK)
typedef elem_t scales_t __attribute__((ext_vector_type(READ), aligned(ELEM_BYTES)));
typedef unsigned char zeros_t __attribute__((ext_vector_type(READ), aligned(1)));

struct run_t {
  u32x4 w[NT];
  scales_t s[NT];
  zeros_t z[NT];
};

// 16 bytes from any address: the five words around them, moved together (vector loads off a word's boundary are taken apart by the
// hardware).  Reads up to 4 bytes behind them.
DEV u32x4 load_16(const void* p) {
  const unsigned long long at = (unsigned long long)p;
  const u32* __restrict__ q = (const u32*)(at & ~3ull);
  const u32x4 w = *(const u32x4_any*)q;
  const u32 last = q[4], off = (u32)at & 3u;
  return (u32x4){__builtin_amdgcn_alignbyte(w[1], w[0], off), __builtin_amdgcn_alignbyte(w[2], w[1], off), __builtin_amdgcn_alignbyte(w[3], w[2], off),
                 __builtin_amdgcn_alignbyte(last, w[3], off)};
}
// 16 bytes moved down by some of them; zeros follow
DEV u32x4 move_down(const u32x4 v, const int bytes) {
  typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
  const u64x2 w = __builtin_bit_cast(u64x2, v);
  const int s = bytes * 8;
  u64x2 r;
  r[0] = s == 0 ? w[0] : s < 64 ? w[0] >> s | w[1] << (64 - s) : s < 128 ? w[1] >> (s & 63) : 0;
  r[1] = s < 64 ? w[1] >> (s & 63) : 0;
  return __builtin_bit_cast(u32x4, r);
}

// Whether all of a chunk of x lies inside K: then no vector of it needs a look.  (A branch of the whole wavefront, once a chunk.)
struct whole_t { static constexpr bool whole = true; };
struct cut_t { static constexpr bool whole = false; };

#if SPREAD
// the values that the quarters of a chunk's parts hold, for all lanes
DEV void spread(const u32 v, u32 (&r)[PARTS_OF_CHUNK]) {
  const u32x2 a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
#if STEPS == 2
  r[0] = a[0];
  r[1] = a[1];
#else
  const u32x2 p = __builtin_amdgcn_permlane16_swap(a[0], a[0], false, false), q = __builtin_amdgcn_permlane16_swap(a[1], a[1], false, false);
  r[0] = p[0];
  r[1] = p[1];
  r[2] = q[0];
  r[3] = q[1];
#endif
}
#endif

// x[row, k .. k + 8) in the order of a word's codes, in XP parts
template <typename T> DEV void load_x(const elem_t* __restrict__ xr, const int k, frag_t (&f)[XP], T) {
  float v[8];
  elem_t e[8];
#if XP == 1
  u32x4 t;
  if (T::whole) t = X_WORDS ? *(const u32x4_any*)(xr + k) : load_16(xr + k);
  else if (GK >= 8) {                                            // the last eight of the row, moved to where they belong
    const int at = min(k, GK - 8);
    t = move_down(__builtin_bit_cast(u32x4, *(const xvec_t*)(xr + at)), min(k - at, 8) * 2);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) { const elem_t y = xr[min(k + j, GK - 1)]; e[j] = k + j < GK ? y : (elem_t)0; }
    t = __builtin_bit_cast(u32x4, (xvec_t){e[0], e[1], e[2], e[3], e[4], e[5], e[6], e[7]});
  }
  const xvec_t all = __builtin_bit_cast(xvec_t, t);
#pragma unroll
  for (int j = 0; j < 8; ++j) e[j] = all[j];
#else
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (T::whole) e[j] = xr[k + j];
    else { const elem_t y = xr[min(k + j, GK - 1)]; e[j] = k + j < GK ? y : (elem_t)0; }
  }
#endif
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int slot = j < 4 ? 2 * j : 2 * (j - 4) + 1;
#if XP == 1
    f[0][slot] = __builtin_bit_cast(part_t, e[j]);
#else
    v[j] = e[j];
#pragma unroll
    for (int i = 0; i < XP; ++i) { f[i][slot] = (part_t)v[j]; v[j] -= (float)f[i][slot]; }
#endif
  }
}

// eight codes of a word as 16 + code
DEV frag_t decode(const u32 w) {
  u32x4 r;
#if F16_PARTS
  r[0] = (w << 6 & 0x03c003c0u) | 0x4c004c00u;
  r[1] = (w << 2 & 0x03c003c0u) | 0x4c004c00u;
  r[2] = (w >> 2 & 0x03c003c0u) | 0x4c004c00u;
  r[3] = (w >> 6 & 0x03c003c0u) | 0x4c004c00u;
#else
  r[0] = (w << 3 & 0x00780078u) | 0x41804180u;
  r[1] = (w >> 1 & 0x00780078u) | 0x41804180u;
  r[2] = (w >> 5 & 0x00780078u) | 0x41804180u;
  r[3] = (w >> 9 & 0x00780078u) | 0x41804180u;
#endif
  return __builtin_bit_cast(frag_t, r);
}

extern "C" __global__ __launch_bounds__(64 * WAVES) void KNAME(KPARAMS SCRATCH) {
  __shared__ __attribute__((aligned(16))) float part[WAVES][ROWS][16 * NT + 1];
#if STAGED
  // its part of x once per workgroup in the order of the codes (rows 16 bytes apart in their banks, zeros behind K)
  __shared__ __attribute__((aligned(16))) part_t xs[XP][ROWS][RANGE * CHUNK + 8];
#endif
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, h = lane >> 4;
  // The tiles of one column range, which read the same weights, lie eight workgroups apart: on one die, one after another.
  const int group = blockIdx.x / (8 * ROW_TILES), member = blockIdx.x % (8 * ROW_TILES);
  const idx_t c0 = (idx_t)(group * 8 + member % 8) * (16 * NT), r0 = (idx_t)(member / 8) * 16;
  if (c0 >= GN) return;
  const int base = SPLITS > 1 ? blockIdx.y * RANGE : 0;              // this workgroup's part of K, in chunks
  const unsigned char* __restrict__ wr[NT];
  const elem_t* __restrict__ sr[NT];
  const unsigned char* __restrict__ zr[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const idx_t col = min(c0 + t * 16 + n, (idx_t)(GN - 1));         // (behind the last column: that again, not stored)
    wr[t] = PW + (long long)col * ROW_BYTES;
    sr[t] = PS + (long long)col * GROUPS;
#if HAS_ZERO
    zr[t] = PZ + (long long)col * GROUPS;
#endif
  }
#if !STAGED
  const elem_t* __restrict__ xr = PX + offX_batch(0) + offX_row(min(r0 + n, (idx_t)(GM - 1)));
#endif

  auto load = [&](run_t& r, const int c) {
    // (load_16, for rows that begin off a word's boundary, reads a word too much)
    const int more = ROW_BYTES % 4 == 0 ? 0 : 4;
    const bool whole = ROW_BYTES % 64 == 0 || (c + 1) * (CHUNK / 2) + more <= ROW_BYTES;
    const int at = c * (CHUNK / 2) + h * 16;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (whole) r.w[t] = ROW_BYTES % 4 == 0 ? *(const u32x4_any*)(wr[t] + at) : load_16(wr[t] + at);
      else if ((long long)GN * ROW_BYTES >= 16) {
        // The end of a row, and what lies behind it: the next row's codes, which meet zeros of x.  Behind the last row there is
        // nothing: the last bytes of all, moved to where they belong.
        const long long want = wr[t] - PW + at, from = min(want, (long long)GN * ROW_BYTES - 16);
        r.w[t] = move_down(*(const u32x4_byte*)(PW + from), (int)min(want - from, 16ll));
      } else {
        r.w[t] = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (at + i < ROW_BYTES) r.w[t][i / 4] |= (u32)wr[t][at + i] << (i % 4 * 8);
      }
#if SPREAD || STEPS == 4
      const int g = (c * CHUNK + (SPREAD ? h * 32 : 0)) / GROUP, at_g = SPREAD ? min(g, GROUPS - 1) : g;
#else
      const int at_g = c * PARTS_OF_CHUNK;
#endif
      r.s[t] = *(const scales_t*)(sr[t] + at_g);
#if HAS_ZERO
      r.z[t] = *(const zeros_t*)(zr[t] + at_g);
#endif
    }
  };

  f32x4 acc[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u) acc[u] = 0.0f;
  frag_t ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = (part_t)1.0f;

  auto multiply = [&](run_t& r, const int c, auto reach) {
#if TURNED
    // words (quarter q, register i) -> (quarter i, register q)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const u32x2 a = __builtin_amdgcn_permlane32_swap(r.w[t][0], r.w[t][2], false, false), b = __builtin_amdgcn_permlane32_swap(r.w[t][1], r.w[t][3], false, false);
      const u32x2 p = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), q = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
      r.w[t] = (u32x4){p[0], p[1], q[0], q[1]};
    }
#endif
#if SPREAD
    u32 scale[NT][PARTS_OF_CHUNK], zero[NT][PARTS_OF_CHUNK];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      spread(__builtin_bit_cast(u32, cvt_in(r.s[u][0])), scale[u]);
#if HAS_ZERO
      spread(__builtin_bit_cast(u32, 16.0f + (float)r.z[u][0]), zero[u]);
#endif
    }
#endif
#pragma unroll
    for (int p = 0; p < PARTS_OF_CHUNK; ++p) {
      f32x4 sum[NT], sx = 0.0f;
#pragma unroll
      for (int u = 0; u < NT; ++u) sum[u] = 0.0f;
#pragma unroll
      for (int i = p * STEPS; i < (p + 1) * STEPS; ++i) {
        const int k = c * CHUNK + (TURNED ? i * 32 + h * 8 : h * 32 + i * 8);
        frag_t x[XP];
#if STAGED
#pragma unroll
        for (int q = 0; q < XP; ++q) x[q] = *(const frag_t*)&xs[q][min(n, ROWS - 1)][k - base * CHUNK];
#else
        load_x(xr, k, x, reach);
#endif
#pragma unroll
        for (int q = 0; q < XP; ++q) sx = MFMA(x[q], ones, sx, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          const frag_t w = decode(r.w[u][i]);
#pragma unroll
          for (int q = 0; q < XP; ++q) sum[u] = MFMA(x[q], w, sum[u], 0, 0, 0);
        }
      }
#pragma unroll
      for (int u = 0; u < NT; ++u) {
#if SPREAD
        const float s = __builtin_bit_cast(float, scale[u][p]), z = HAS_ZERO ? __builtin_bit_cast(float, zero[u][p]) : 24.0f;
#else
        const float s = cvt_in(r.s[u][p]), z = HAS_ZERO ? 16.0f + (float)r.z[u][p] : 24.0f;
#endif
#pragma unroll
        for (int e = 0; e < (ROWS < 4 ? ROWS : 4); ++e) acc[u][e] = __builtin_fmaf(s, __builtin_fmaf(-z, sx[e], sum[u][e]), acc[u][e]);
      }
    }
  };

  // this wavefront's chunks: EACH successive ones, so that it reads runs of EACH * 64 bytes of a row; AHEAD of them on their way
  const int first = base + wave * EACH, last = min(first + EACH, min(base + RANGE, CHUNKS));
  run_t ring[AHEAD];
#pragma unroll
  for (int p = 0; p < AHEAD; ++p) load(ring[p], max(min(first + p, last - 1), 0));
#if STAGED
  for (int i = tid; i < ROWS * (RANGE * 16); i += 64 * WAVES) {
    const int r = i / (RANGE * 16), k = i % (RANGE * 16) * 8;
    frag_t x[XP];
    load_x(PX + offX_batch(0) + offX_row(min(r0 + r, (idx_t)(GM - 1))), base * CHUNK + k, x, cut_t());
#pragma unroll
    for (int q = 0; q < XP; ++q) *(frag_t*)&xs[q][r][k] = x[q];
  }
  __syncthreads();
#endif
  for (int c = first; c < last; c += AHEAD) {
#pragma unroll
    for (int p = 0; p < AHEAD; ++p) {
      if (c + p < last) {
        if ((X_WORDS && GK % CHUNK == 0) || (c + p + 1) * CHUNK + (X_WORDS ? 0 : 2) <= GK) multiply(ring[p], c + p, whole_t());
        else multiply(ring[p], c + p, cut_t());
      }
      if (EACH > AHEAD) load(ring[p], min(c + p + AHEAD, last - 1));      // (unconditional: loads behind a branch make the next wait one for all)
    }
  }

  // ---- the wavefronts' sums, joined; result (4 h + e, n) of a 16x16 tile is element e
#pragma unroll
  for (int u = 0; u < NT; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (4 * h + e < ROWS) part[wave][4 * h + e][u * 16 + n] = acc[u][e];
  __syncthreads();
  for (int i = tid; i < ROWS * 16 * NT; i += 64 * WAVES) {
    const int rl = i / (16 * NT), cl = i % (16 * NT);
    if (r0 + rl >= GM || c0 + cl >= GN) continue;
    float v = part[0][rl][cl];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += part[w][rl][cl];
#if SPLITS > 1
    scratch[((idx_t)blockIdx.y * GM + r0 + rl) * GN + c0 + cl] = v;
#else
    float cv[NCOLV > 0 ? NCOLV : 1];
    col_loads(c0 + cl, cv, KARGS);
    epilogue(0, r0 + rl, c0 + cl, v, cv, KARGS);
#endif
  }
}
)KRN";

// the sums of the parts of K, joined
const char* kInt4JoinBody = R"KRN(
extern "C" __global__ __launch_bounds__(256) void KNAME(KPARAMS SCRATCH) {
  const idx_t at = (idx_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (idx_t)GM * GN) return;
  float part[SPLITS], v = 0.0f;
#pragma unroll
  for (int i = 0; i < SPLITS; ++i) part[i] = scratch[(idx_t)i * GM * GN + at];
#pragma unroll
  for (int i = 0; i < SPLITS; ++i) v += part[i];
  float cv[NCOLV > 0 ? NCOLV : 1];
  col_loads(at % GN, cv, KARGS);
  epilogue(0, at / GN, at % GN, v, cv, KARGS);
}
)KRN";

}  // namespace

Lowered lower_int4(LowerCtx& c) {
  const Graph& g = c.g;
  const Op& A = g.ops[c.anchor_op];
  check_decode_op(g, A);
  const Tensor &X = g.tensors[A.in[0]], &C = g.tensors[A.out[0]];
  const int64_t K = X.dims.back(), N = C.dims.back(), M = C.n() / N, G = A.i("group_size", 0), groups = (K + G - 1) / G;
  const bool has_zero = A.in.size() == 4;

  // ---- index space: the result's axes and the contraction
  TIdx oi = c.fresh_index(C.dims);
  const int katom = c.new_atom(K);
  TIdx xi = oi;
  xi.back() = DimIdx();
  if (K > 1) xi.back().atoms = {katom};
  c.tidx[c.anchor_out] = oi;
  std::vector<int> ein, eout, removed;
  block_io(g, c.blk, ein, eout, removed);
  c.forward_all();
  for (int t : eout) DNNF_CHECK(c.tidx.count(t), DNNF_UNSUPPORTED_OP, "block output " + g.tensors[t].name + " does not follow the contraction");
  c.collect_stores(eout);
  const int xn = c.value(A.in[0], xi);
  DNNF_CHECK(c.nodes[xn].kind == ENode::LOAD && c.nodes[xn].addr.indirect.empty() && g.tensors[c.nodes[xn].tensor].dtype == X.dtype, DNNF_UNSUPPORTED_OP,
             "arithmetic in front of a product with 4-bit weights has no kernel template");
  const int tx = c.nodes[xn].tensor;
  const Affine xa = c.resolved(c.nodes[xn].addr);
  std::vector<int> katoms, cols, rows;
  c.resolve({katom}, katoms);
  DNNF_CHECK(katoms.size() <= 1 && (katoms.empty() || stride_of(xa, katoms[0]) == 1), DNNF_UNSUPPORTED_OP, "x is not contiguous along the contraction");
  c.resolve(oi.back().atoms, cols);
  for (size_t d = 0; d + 1 < oi.size(); d++) c.resolve(oi[d].atoms, rows);
  DNNF_CHECK(c.extent_of(rows) == M && c.extent_of(cols) == N, DNNF_UNSUPPORTED_OP, "axes of a product with 4-bit weights");

  // ---- parameters
  std::vector<int> params = {tx, A.in[1], A.in[2]};
  if (has_zero) params.push_back(A.in[3]);
  std::map<int, int> pslot;
  std::set<int> written;
  {
    std::set<int> seen;
    std::vector<int> stack;
    for (auto& s : c.stores) stack.push_back(s.value);
    while (!stack.empty()) {
      const int n = stack.back();
      stack.pop_back();
      if (!seen.insert(n).second) continue;
      for (int a : c.nodes[n].args) stack.push_back(a);
      if (c.nodes[n].kind == ENode::LOAD) {
        DNNF_CHECK(c.nodes[n].addr.indirect.empty(), DNNF_UNSUPPORTED_OP, "gathered operand behind a product with 4-bit weights");
        if (!pslot.count(c.nodes[n].tensor)) { pslot[c.nodes[n].tensor] = (int)params.size(); params.push_back(c.nodes[n].tensor); }
      }
    }
  }
  const size_t n_in = params.size();
  for (auto& s : c.stores) {
    DNNF_CHECK(!pslot.count(s.tensor) && std::find(params.begin(), params.begin() + n_in, s.tensor) == params.begin() + n_in, DNNF_UNSUPPORTED_OP,
               "block reads and writes the same tensor");
    pslot[s.tensor] = (int)params.size();
    params.push_back(s.tensor);
    written.insert(s.tensor);
  }
  bool wide = false;
  const int64_t far = ((int64_t)1 << 31) - (1 << 16);      // (tiles reach up to 511 columns behind the last one, and 15 rows)
  for (int t : params) wide = wide || g.tensors[t].n() >= far;
  wide = wide || M * N >= far;

  // ---- tile: sixteen rows; K split among up to sixteen wavefronts.  A product of one row is over before a long loop could settle:
  // what counts is that all of its weights are asked for at once (one row with sixteen wavefronts, eight, four: 4096 x 4096 4.1 us, 5.9
  // and 5.4; 4096 x 11008 8.9, 14.6 and 12.9; 11008 x 4096 9.2, 9.1 and 9.7).
  // Up to four rows x goes through LDS (one row, 4096 x 11008: 8.8 us, 9.3 with x read by every wavefront for itself; sixteen rows,
  // 768 x 50257: 11.7 and 9.3) and a workgroup takes as many columns as leave two of them per compute unit.  With more rows
  // it is x that the wavefronts wait for, and wide tiles read it less often: as many columns as leave 160 workgroups (16 rows,
  // 4096 x 11008: 13.3 us with 64 columns, 18.6 with 16; 64 rows, 4096 x 4096: 13.4 and 24.2; but 16 rows, 4096 x 4096, where that
  // would be 64 workgroups: 12.8 and 7.4, and 11008 x 4096: 39.4 and 17.3).  Without zero points each takes a tenth less.  Two or four
  // row tiles a wavefront, for one pass over the codes, were no faster (64 rows, 4096 x 4096: 20.9 and 22.6 us).
  const int64_t row_tiles = (M + 15) / 16, chunks = (K + 127) / 128, xp = X.dtype == DNNF_F32 ? 3 : 1;
  // Few tiles of a long contraction: K is split among workgroups too, a chunk or more a wavefront, as far as the compute units go, and a
  // second kernel (2 us) joins the sums: 2 rows, 32000 x 1024: 10.3 us, 29.8 in one; 4 rows, 8896 x 841: 6.9 and 10.5; 16 rows,
  // 8320 x 1024: 6.8 and 12.0.  More than one workgroup a unit, or shorter K, gains nothing (one row, 4096 x 4096: 6.7 us, 4.1 in
  // one; 16 rows, 11008 x 4096: 21.4 and 17.2; 16 rows, 4096 x 1024: 7.1 and 7.1).
  const int64_t tiles = (N + 15) / 16 * row_tiles;
  int64_t splits = tiles <= 128 && chunks > (xp * M <= 4 ? 64 : 32) ? std::min<int64_t>({256 / tiles, (chunks + 15) / 16, 32}) : 1;
  const int64_t range = (chunks + splits - 1) / splits;
  splits = (chunks + range - 1) / range;
  const bool staged = xp * M <= 4 && xp * M * (range * 128 + 8) * 2 <= 40 * 1024;
  int64_t NT = 4;
  while (NT > 1 && (N + 16 * NT - 1) / (16 * NT) * row_tiles < (staged ? 512 : 160)) NT /= 2;
  const int64_t most = std::min<int64_t>(16, range), each = (range + most - 1) / most, waves = (range + each - 1) / each, ahead = std::min<int64_t>(each, 2);
  const int steps = G % 128 == 0 || G >= K ? 4 : G % 64 == 0 ? 2 : 1;

  std::ostringstream k;
  const std::string part = X.dtype == DNNF_F16 ? "_Float16" : "__bf16";
  k << "typedef " << (wide ? "long long" : "int") << " idx_t;\ntypedef " << c.ctype(X.dtype) << " elem_t;\ntypedef " << part << " part_t;\n";
  k << "#define ELEM_BYTES " << dtype_bytes(X.dtype) << "\n#define XP " << xp << "\n#define F16_PARTS " << (int)(X.dtype == DNNF_F16) << "\n";
  k << "#define MFMA __builtin_amdgcn_mfma_f32_16x16x32_" << (X.dtype == DNNF_F16 ? "f16" : "bf16") << "\n";
  k << "#define GM " << M << "\n#define GN " << N << "\n#define GK " << K << "\n#define GROUP " << G << "\n#define GROUPS " << groups << "\n#define HAS_ZERO " << (int)has_zero << "\n";
  k << "#define NT " << NT << "\n#define WAVES " << waves << "\n#define AHEAD " << ahead << "\n#define ROW_TILES " << row_tiles << "\n#define EACH " << each << "\n#define STAGED " << (int)staged << "\n#define STEPS " << steps << "\n";
  // (the parts of chunk c have groups c * parts and on where the row is a whole number of such runs: no run leaves its row then)
  const bool spread = steps < 4 && (128 % G != 0 || groups % (4 / steps) != 0);
  // x's rows, and what they are a part of, begin on words' boundaries
  bool x_words = xa.offset % 2 == 0;
  for (int a : rows) x_words = x_words && stride_of(xa, a) % 2 == 0;
  k << "#define X_WORDS " << (int)(x_words || X.dtype == DNNF_F32) << "\n";
  k << "#define TURNED " << (int)(steps < 4 || !staged) << "\n#define SPREAD " << (int)spread << "\n";
  k << "#define PX p0\n#define PW p1\n#define PS p2\n#define PZ p3\n";
  k << gemm_offset_fn(c, "offX_row", rows, xa) << gemm_offset_fn(c, "offX_batch", {}, xa);
  const std::string kparams = c.param_list(params, written);
  std::string kargs;
  for (size_t i = 0; i < params.size(); i++) kargs += (i ? ", p" : "p") + std::to_string(i);
  k << gemm_epilogue_source(c, {}, rows, cols, pslot, kparams, N, -1);
  k << "#define KPARAMS " << kparams << "\n#define KARGS " << kargs << "\n#define SPLITS " << splits << "\n#define RANGE " << range << "\n";
  k << "#define SCRATCH " << (splits > 1 ? ", float* __restrict__ scratch" : "") << "\n";

  Lowered L;
  L.family = FAM_INT4;
  L.ext_in.assign(params.begin(), params.begin() + n_in);
  L.ext_out.assign(params.begin() + n_in, params.end());
  const int64_t blocks = ((N + 16 * NT - 1) / (16 * NT) + 7) / 8 * 8 * row_tiles;
  DNNF_CHECK(blocks * 64 * waves < (int64_t)1 << 32, DNNF_UNSUPPORTED_OP, "MatMulInt4: more workgroups than one launch takes");
  auto launch = [&](const char* stem, const char* body, int64_t gx, int64_t gy, int64_t threads) {
    Launch Kn;
    Kn.params = params;
    Kn.grid[0] = (unsigned)gx;
    Kn.grid[1] = (unsigned)gy;
    Kn.block[0] = (unsigned)threads;
    Kn.scratch = splits > 1;
    std::string src = std::string(device_preamble()) + k.str() + body;
    Kn.name = fnv_name(stem, src);
    size_t pos;
    while ((pos = src.find("KNAME")) != std::string::npos) src.replace(pos, 5, Kn.name);
    Kn.source = src;
    L.launches.push_back(Kn);
  };
  launch("dnnf_int4", kInt4Body, blocks, splits, 64 * waves);
  if (splits > 1) {
    L.scratch_bytes = splits * M * N * 4;
    launch("dnnf_int4_join", kInt4JoinBody, (M * N + 255) / 256, 1, 256);
  }
  L.variant = "int4_16x" + std::to_string(16 * NT) + "_w" + std::to_string(waves) + "_g" + std::to_string(32 * steps) + (splits > 1 ? "_k" + std::to_string(splits) : "");
  return L;
}

}  // namespace dnnf
