// Operands, shapes and checks of the operators of single-token inference: a key / value cache kept in pages (CacheWrite,
// CacheRead, CacheAttention) and products with weights of four bits (MatMulInt4).
#include <algorithm>

#include "ir.hpp"

namespace dnnf {

bool is_decode_op(const Op& op) {
  const OpClass c = op.info->cls;
  return c == OC_CACHE_WRITE || c == OC_CACHE_READ || c == OC_CACHE_ATTN || c == OC_MATMUL_INT4;
}

// An attribute that counts something; -1 where it is no whole number below 2^31.
static int64_t whole_attr(const Op& op, const char* name) {
  const double v = op.f(name, 0);
  return v >= 0 && v < 2147483648.0 && v == (double)(int64_t)v ? (int64_t)v : -1;
}

// Operand order
//   CacheWrite      k_pool, v_pool, [k_scale, v_scale,] k, v, table, first [, count]  ->  k_pool, v_pool [, k_scale, v_scale]
//   CacheRead       k_pool, v_pool, [k_scale, v_scale,] table, held                   ->  k, v
//   CacheAttention  q, k_pool, v_pool, [k_scale, v_scale,] table, held                ->  o
// with the scales where the pools hold 8 bits.
CacheOperands cache_operands(const Graph& g, const Op& op) {
  CacheOperands c;
  const OpClass cls = op.info->cls;
  const std::string& kind = op.kind;
  size_t at = 0;
  auto dims = [&](int t) -> const Dims& { return g.tensors[t].dims; };
  auto take = [&](const char* what) {
    DNNF_CHECK(at < op.in.size(), DNNF_INVALID_ARG, kind + ": no operand for " + what);
    return op.in[at++];
  };
  auto agree = [&](bool ok, const std::string& what) { DNNF_CHECK(ok, DNNF_SHAPE_MISMATCH, kind + ": " + what); };

  if (cls == OC_CACHE_ATTN) c.q = take("q");
  for (int i = 0; i < 2; i++) c.pool[i] = take(i ? "v_pool" : "k_pool");
  c.eight_bits = g.tensors[c.pool[0]].dtype == DNNF_I8;
  if (c.eight_bits) for (int i = 0; i < 2; i++) c.scale[i] = take(i ? "v_scale" : "k_scale");
  if (cls == OC_CACHE_WRITE) for (int i = 0; i < 2; i++) c.fresh[i] = take(i ? "v" : "k");
  c.table = take("table");
  if (cls == OC_CACHE_WRITE) {
    c.first = take("first");
    if (at < op.in.size()) c.count = take("count");
  } else c.held = take("held");
  DNNF_CHECK(at == op.in.size(), DNNF_INVALID_ARG, kind + ": too many operands");

  const Dims& kp = dims(c.pool[0]);
  agree(kp.size() == 4 && dims(c.pool[1]).size() == 4, "a pool is [pages, key heads, slots of a page, channels]");
  c.P = kp[0]; c.HK = kp[1]; c.S = kp[2];
  for (int i = 0; i < 2; i++) {
    const Dims& d = dims(c.pool[i]);
    c.D[i] = d[3];
    agree(d[0] == c.P && d[1] == c.HK && d[2] == c.S, "the pools differ in pages, heads or slots");
    if (c.eight_bits) agree(dims(c.scale[i]) == Dims{c.P, c.HK, c.S}, "a scale tensor is [pages, key heads, slots of a page]");
  }
  agree(dims(c.table).size() == 2, "the table is [sequences, pages of a sequence]");
  c.B = dims(c.table)[0]; c.M = dims(c.table)[1];
  for (int t : {c.first, c.count, c.held})
    if (t >= 0) agree(dims(t) == Dims{c.B}, "positions and counts are one number per sequence");
  if (cls == OC_CACHE_WRITE) {
    agree(dims(c.fresh[0]).size() == 4 && dims(c.fresh[1]).size() == 4, "new keys and values are [sequences, tokens, key heads, channels]");
    c.T = dims(c.fresh[0])[1];
    for (int i = 0; i < 2; i++) agree(dims(c.fresh[i]) == Dims{c.B, c.T, c.HK, c.D[i]}, "new keys / values differ from the pools or the table");
  }
  if (cls == OC_CACHE_READ) {
    c.T = whole_attr(op, "length");
    DNNF_CHECK(c.T >= 1, DNNF_INVALID_ARG, "CacheRead needs \"length\", the positions laid out");
  }
  if (cls == OC_CACHE_ATTN) {
    const Dims& q = dims(c.q);
    agree(q.size() == 3 && q[0] == c.B && q[2] == c.D[0], "queries are [sequences, heads, channels of a key]");
    c.HQ = q[1];
    agree(c.HK >= 1 && c.HQ >= 1 && c.HQ % c.HK == 0, "the query heads are no multiple of the key heads");
  }
  return c;
}

int64_t cache_positions(const Op& op, const CacheOperands& c) {
  if (op.info->cls != OC_CACHE_ATTN) return std::min(c.T, c.M * c.S);
  const int64_t window = whole_attr(op, "window");
  return window > 0 ? std::min(window, c.M * c.S) : c.M * c.S;
}

double cache_bytes(const Graph& g, const Op& op) {
  const CacheOperands c = cache_operands(g, op);
  // (sequences may share pages, whose rows are then read once)
  const int64_t all = c.B * cache_positions(op, c), rows = op.info->cls == OC_CACHE_WRITE ? all : std::min(all, c.P * c.S);
  double bytes = (double)(rows * c.HK) * (double)((c.D[0] + c.D[1]) * dtype_bytes(g.tensors[c.pool[0]].dtype) + (c.eight_bits ? 8 : 0));
  for (int t : {c.q, c.fresh[0], c.fresh[1], c.table, c.first, c.count, c.held})
    if (t >= 0) bytes += (double)g.tensors[t].bytes();
  if (op.info->cls != OC_CACHE_WRITE)
    for (int t : op.out) bytes += (double)g.tensors[t].bytes();
  return bytes;
}

Dims infer_decode_shape(const Graph& g, const Op& op, int oi) {
  if (op.info->cls == OC_MATMUL_INT4) {
    DNNF_CHECK(op.in.size() == 3 || op.in.size() == 4, DNNF_INVALID_ARG, "MatMulInt4 takes x, weights, scales and, where weights are not centred on 8, zero points");
    DNNF_CHECK(op.out.size() == 1, DNNF_INVALID_ARG, "MatMulInt4 has one result");
    const Dims &x = g.tensors[op.in[0]].dims, &w = g.tensors[op.in[1]].dims;
    DNNF_CHECK(x.size() >= 2 && w.size() == 2, DNNF_SHAPE_MISMATCH, "MatMulInt4: x is [.., rows, K], weights [N, K / 2]");
    const int64_t K = x.back(), G = whole_attr(op, "group_size");
    DNNF_CHECK(G >= 32 && G % 32 == 0, DNNF_INVALID_ARG, "MatMulInt4 needs \"group_size\", a multiple of 32");
    DNNF_CHECK(w[1] == (K + 1) / 2, DNNF_SHAPE_MISMATCH, "MatMulInt4: a row of weights is (K + 1) / 2 bytes");
    for (size_t i = 2; i < op.in.size(); i++)
      DNNF_CHECK((g.tensors[op.in[i]].dims == Dims{w[0], (K + G - 1) / G}), DNNF_SHAPE_MISMATCH, "MatMulInt4: scales and zero points are [N, groups of K]");
    Dims out = x;
    out.back() = w[0];
    return out;
  }
  const CacheOperands c = cache_operands(g, op);
  const size_t want = op.info->cls == OC_CACHE_WRITE ? (c.eight_bits ? 4 : 2) : op.info->cls == OC_CACHE_READ ? 2 : 1;
  DNNF_CHECK(op.out.size() == want, DNNF_INVALID_ARG, op.kind + " has " + std::to_string(want) + " results");
  if (op.info->cls == OC_CACHE_WRITE) return g.tensors[op.in[oi]].dims;
  if (op.info->cls == OC_CACHE_READ) return {c.B, c.T, c.HK, c.D[oi]};
  return {c.B, c.HQ, c.D[1]};
}

void check_decode_op(const Graph& g, const Op& op) {
  auto type = [&](int t) { return g.tensors[t].dtype; };
  auto plain = [&](int t) { DNNF_CHECK(g.tensors[t].perm.empty(), DNNF_UNSUPPORTED_OP, op.kind + ": operand in another storage order"); };
  for (int t : op.in) plain(t);
  for (int t : op.out) plain(t);
  if (op.info->cls == OC_MATMUL_INT4) {
    DNNF_CHECK(is_float(type(op.in[0])) && type(op.in[2]) == type(op.in[0]) && type(op.out[0]) == type(op.in[0]), DNNF_INVALID_ARG,
               "MatMulInt4: x, scales and result share a float type");
    DNNF_CHECK(type(op.in[1]) == DNNF_U8 && (op.in.size() < 4 || type(op.in[3]) == DNNF_U8), DNNF_INVALID_ARG, "MatMulInt4: weights and zero points are U8");
    for (int t : {op.in[0], op.in[1], op.out[0]})
      for (int64_t d : g.tensors[t].dims) DNNF_CHECK(d >= 1, DNNF_SHAPE_MISMATCH, "MatMulInt4: empty operand");
    // positions along K, up to the end of the chunk behind the last, are counted in 32 bits
    DNNF_CHECK(g.tensors[op.in[0]].dims.back() < ((int64_t)1 << 31) - 256, DNNF_UNSUPPORTED_OP, "MatMulInt4: a contraction of 2^31 or more");
    return;
  }
  const CacheOperands c = cache_operands(g, op);
  for (int64_t d : {c.P, c.HK, c.S, c.D[0], c.D[1], c.B, c.M}) DNNF_CHECK(d >= 1, DNNF_SHAPE_MISMATCH, op.kind + ": empty operand");
  DNNF_CHECK(op.info->cls != OC_CACHE_WRITE || c.T >= 1, DNNF_SHAPE_MISMATCH, "CacheWrite: no new tokens");
  for (int i = 0; i < 2; i++)
    DNNF_CHECK(c.D[i] % 16 == 0 && c.D[i] <= 256, DNNF_UNSUPPORTED_OP, op.kind + ": the channels of a key or value are a multiple of 16, at most 256");
  // rows are numbered in 32 bits (their elements in 64)
  DNNF_CHECK(c.P <= ((int64_t)1 << 31) / c.HK && c.P * c.HK <= (((int64_t)1 << 31) - 1) / c.S, DNNF_UNSUPPORTED_OP, op.kind + ": a pool of 2^31 rows or more");
  DNNF_CHECK(c.M <= (((int64_t)1 << 30) - 1) / c.S && c.T < (int64_t)1 << 30, DNNF_UNSUPPORTED_OP, op.kind + ": sequences of 2^30 positions or more");
  DNNF_CHECK(c.B < (int64_t)1 << 20 && c.HQ < (int64_t)1 << 16, DNNF_UNSUPPORTED_OP, op.kind + ": too many sequences or heads");
  for (int t : {c.table, c.first, c.count, c.held})
    DNNF_CHECK(t < 0 || type(t) == DNNF_I32, DNNF_INVALID_ARG, op.kind + ": tables, positions and counts are I32");
  const int pooled = type(c.pool[0]);
  DNNF_CHECK(type(c.pool[1]) == pooled && (c.eight_bits || is_float(pooled)), DNNF_INVALID_ARG, op.kind + ": the pools share one type, I8 or a float type");
  for (int t : {c.scale[0], c.scale[1]}) DNNF_CHECK(t < 0 || type(t) == DNNF_F32, DNNF_INVALID_ARG, op.kind + ": scales are F32");
  // what is stored or computed with is of the pools' type, any float type with pools of 8 bits
  std::vector<int> rows;
  if (op.info->cls == OC_CACHE_WRITE) rows = {c.fresh[0], c.fresh[1]};
  else if (op.info->cls == OC_CACHE_READ) rows = op.out;
  else rows = {c.q, op.out[0]};
  DNNF_CHECK(is_float(type(rows[0])) && type(rows[1]) == type(rows[0]) && (c.eight_bits || type(rows[0]) == pooled), DNNF_INVALID_ARG,
             op.kind + ": its float operands share one type, which is the pools' unless those are I8");
  if (op.info->cls == OC_CACHE_ATTN) {
    const double s = op.f("scale", 1);
    DNNF_CHECK(whole_attr(op, "window") >= 0, DNNF_INVALID_ARG, "CacheAttention: \"window\" is a number of keys, 0 for all");
    DNNF_CHECK(s >= -1e38 && s <= 1e38, DNNF_INVALID_ARG, "CacheAttention: \"scale\" is no finite number");
  }
  if (op.info->cls != OC_CACHE_WRITE) return;
  // The pools are updated where they are: a result is its operand's buffer.  Nobody else may read the operand (which
  // rows such a reader saw would depend on the order of the blocks).
  for (size_t i = 0; i < op.out.size(); i++) {
    const Tensor &X = g.tensors[op.in[i]], &R = g.tensors[op.out[i]];
    DNNF_CHECK(R.dtype == X.dtype, DNNF_INVALID_ARG, "CacheWrite: result " + R.name + " differs in type from " + X.name);
    DNNF_CHECK(X.kind == DNNF_INPUT && R.kind == DNNF_OUTPUT, DNNF_INVALID_ARG,
               "CacheWrite updates a graph input in place: " + X.name + " must be an INPUT and its result " + R.name + " an OUTPUT");
    DNNF_CHECK(X.consumers.size() == 1, DNNF_INVALID_ARG, "CacheWrite updates " + X.name + " in place: other operators read its result " + R.name);
  }
}

}  // namespace dnnf
