// Plane family: score products that meet in a plane [.., N, M], elementwise
// primitives on the plane, and products of the plane with streamed operands,
// in one kernel that never stores the plane: attention of any length with its
// score chain (caps, biases, masks) and a softmax in one pass, and attention's
// gradients, which evaluate the scores again (redundant execution, Korch
// Section 4.2).
//
// A kernel is accepted when
//   * every product without another product among its ancestors in the kernel
//     is a score product A . B^T whose operands are stored tensors seen through
//     layout primitives (or a select with zero along their rows);
//   * the other products are output products P . W (the plane's rows are owned,
//     its columns streamed) or P^T . W (columns owned, rows streamed), all of
//     one kind, W stored like the scores' operands;
//   * at most one softmax: m = max over a row, e = exp(s - m) (or 0 where a mask
//     is false), l = sum of e; then P is e or e / l;
//   * row vectors may be products of two stored tensors summed along their rows
//     (the gradients' rowsum(dO O)), with rows owned;
//   * every output is an elementwise function of one output product and of row
//     statistics, a row statistic of the softmax, such a sum, or a sum by bins of
//     the plane.
#include <algorithm>
#include <cmath>
#include <memory>
#include <set>

#include "families.h"

namespace korch {

extern const char* k_device_plane;

namespace {

enum PlaneCls { CONSTV, ROWV, COLV, FULLP };

// An operand stored in memory: rows of `width` consecutive elements.
struct Operand {
  int node = -1;            // node as read by the product
  int mask = -1;            // select's condition along the rows (or -1)
  int source = -1;          // node below the select
  bool transposed = false;  // read as [.., k, row]
  Shape shape;              // of `source`
  std::string key;          // identity of the address map
  std::string off;          // element offset of a row (variables b*, r)
  int root = -1;
  int64_t stride = 0;       // elements from row to row
};

struct PlaneGen {
  const KInfo& ki;
  const Graph& g;
  std::map<int, int> slot;
  Shape PS;                 // plane shape [batch.., N, M]
  int R = 0;                // its rank
  int64_t N = 0, M = 0;
  bool rows_owned = true;
  int dtype = KORCH_F16;
  std::vector<int> scores, outs_p;    // score products, output products
  std::vector<Operand> sc_own, sc_str, out_w;
  std::vector<Operand> streamed;      // distinct streamed tensors
  std::vector<int> sst, ost;          // score / output product -> streamed tensor
  std::vector<int> xnodes, ox;        // distinct plane operands of output products (and bins)
  int xbin = -1, bin_node = -1, bin_out = -1;
  int nm = -1, nl = -1, ne = -1, nexp = -1, nsfinal = -1;  // softmax
  int nfactor = -1;                   // exponential that all plane operands are multiples of (fp16: it carries their scale)
  int cond = -1;                      // mask
  double low = -INFINITY;
  std::vector<int> ovs, tvs, rvs;     // owned vectors, streamed vectors, streamed vectors whose range is read
  // A gather whose table varies from batch entry to batch entry only, by an index
  // computed on the plane (or a gather of such a gather): the values over the
  // innermost index are a table of the workgroup's own, kept in LDS.
  struct Lut {
    int node, index;  // gather, plane node that indexes (innermost)
    int64_t size;
    int at;           // first element
    // Index = base + step * streamed index with whole numbers and step 1 or -1 (a
    // distance): a lane's indices in a subtile are its first one's and its
    // registers', so one clamped base and constant offsets address them all, with
    // the ends repeated over `pad` more elements on both sides.
    int step = 0;
    int64_t pad = 0;
    std::string base;
  };
  std::vector<Lut> luts;
  int64_t lut_size = 0;
  std::map<int, int> prod_of;         // output -> output product index
  std::set<int> ranged;               // owned vectors whose range is read
  std::vector<int> rowdots;           // sums of x y along the rows of stored tensors
  std::map<int, bool> has_score_memo;

  explicit PlaneGen(const KInfo& k) : ki(k), g(k.g) {}

  [[noreturn]] void bad(const std::string& m) const { fail(KORCH_E_UNSUPPORTED, "plane: " + m); }
  bool in(int v) const { return ki.in.count(v) > 0; }
  const Node& nd(int v) const { return g.nodes[v]; }

  bool depends(int v, int on) const { return v == on || ki.ancestor(on, v); }
  bool has_score(int v) const {
    if (!in(v)) return false;
    for (int s : scores)
      if (depends(v, s)) return true;
    return false;
  }

  PlaneCls cls(int v) const {
    const Shape& s = nd(v).shape;
    const int r = (int)s.size();
    if (r > R) return FULLP;
    const bool col = r >= 1 && s[r - 1] > 1, row = r >= 2 && s[r - 2] > 1;
    if (has_score(v) || (row && col)) return FULLP;
    return row ? ROWV : col ? COLV : CONSTV;
  }
  bool is_owned(PlaneCls c) const { return c == CONSTV || c == (rows_owned ? ROWV : COLV); }
  bool is_streamed(PlaneCls c) const { return c == (rows_owned ? COLV : ROWV); }

  // ---- analysis ------------------------------------------------------------

  // Follows a product's operand to a stored tensor.  `batch` are the product's
  // batch dims; the operand is read at [batch, r, k] (or [batch, k, r]).
  Operand operand(int v, bool kfirst, const Shape& batch, const char* what) {
    Operand o;
    o.node = v;
    const Shape& vs = nd(v).shape;
    const int rk = (int)vs.size();
    std::vector<Ix> idx(rk);
    const int nb = (int)batch.size();
    for (int d = 0; d < rk - 2; ++d) {
      const int j = d + nb - (rk - 2);
      idx[d] = vs[d] == 1 ? Ix::k(0) : Ix::var("b.c[" + std::to_string(j) + "]");
    }
    const int VL = 16 / dtype_bytes(nd(v).dtype);
    idx[rk - (kfirst ? 1 : 2)] = Ix::var("r");
    idx[rk - (kfirst ? 2 : 1)] = Ix::var("0", 1, VL);
    idx[rk - (kfirst ? 2 : 1)].konst = true;
    const int64_t width = vs[rk - (kfirst ? 2 : 1)];
    if (width % VL) bad(std::string(what) + ": the contraction or output width is not a multiple of 16 bytes");
    // VL consecutive elements are read as one vector: layout maps must keep
    // them together, so indices split with the vector's lanes in mind
    int cur = v;
    while (in(cur)) {
      const Node& n = nd(cur);
      if (n.op == KORCH_TRANSPOSE) {
        std::vector<Ix> src(idx.size());
        for (size_t d = 0; d < idx.size(); ++d) src[n.attrs.perm[d]] = idx[d];
        idx = src;
        cur = n.in[0];
      } else if (n.op == KORCH_SELECT && n.attrs.has_scalar && n.attrs.scalar == 0.0 && o.mask < 0 && nd(n.in[1]).shape == n.shape) {
        // the condition must not vary along the contraction
        const Shape& cs = nd(n.in[0]).shape;
        const Shape& ns = n.shape;
        std::vector<Ix> ci = broadcast_index(cs, ns, idx);
        for (auto& x : ci)
          if (x.c != 0) bad(std::string(what) + ": a select varies along the contraction");
        o.mask = n.in[0];
        mask_idx[v] = ci;
        cur = n.in[1];
      } else if (n.op == KORCH_RESHAPE || n.op == KORCH_SLICE || n.op == KORCH_BROADCAST) {
        bad(std::string(what) + ": layout primitive not folded");
      } else {
        bad(std::string(what) + ": computed inside the kernel");
      }
    }
    o.root = cur;
    const Node& n = nd(cur);
    auto st = strides_of(n.shape);
    Ix off = Ix::k(0);
    for (size_t d = 0; d < n.shape.size(); ++d) {
      off = ix_add(off, ix_mulk(idx[d], st[d], VL));
      if (idx[d].b == "r") o.stride = st[d];
    }
    if (!off.affine || off.c != 1 || off.al % VL) {
      // alignment is known when every other stride is a multiple of the vector
      bool ok = off.affine && off.c == 1;
      for (size_t d = 0; ok && d < n.shape.size(); ++d)
        if (idx[d].c == 0 && n.shape[d] > 1 && st[d] % VL) ok = false;
      if (!ok) bad(std::string(what) + ": rows are not 16-byte aligned runs of elements");
    }
    o.off = off.b;
    o.key = std::to_string(cur) + ":" + off.b + ":" + std::to_string(o.mask);
    o.shape = {width};
    return o;
  }
  std::map<int, std::vector<Ix>> mask_idx;

  int add_streamed(const Operand& o) {
    for (size_t i = 0; i < streamed.size(); ++i)
      if (streamed[i].key == o.key && streamed[i].shape == o.shape) return (int)i;
    streamed.push_back(o);
    return (int)streamed.size() - 1;
  }

  int strip_identity(int v) const {
    while (in(v) && nd(v).op == KORCH_IDENTITY) v = nd(v).in[0];
    return v;
  }
  // x = select(cond, y, 0): cond, else -1
  int zero_select(int v) const {
    v = strip_identity(v);
    if (!in(v)) return -1;
    const Node& n = nd(v);
    if (n.op != KORCH_SELECT || !n.attrs.has_scalar || n.attrs.scalar != 0.0 || !in(n.in[0])) return -1;
    return n.in[0];
  }

  void analyze() {
    if (ki.linear.empty()) bad("no product");
    for (int v : ki.linear)
      if (nd(v).op != KORCH_MATMUL) bad("a product is not a matrix product");
    for (int v : ki.linear) {
      bool inner = false;
      for (int u : ki.linear)
        if (u != v && ki.ancestor(u, v)) inner = true;
      (inner ? outs_p : scores).push_back(v);
    }
    for (int v : ki.k.prims)
      if (nd(v).op == KORCH_BIN_SUM) {
        if (bin_node >= 0) bad("more than one sum by bins");
        bin_node = v;
      }
    if (outs_p.empty() && bin_node < 0) bad("no product reads the plane");
    if (scores.size() > 2) bad("more than two score products");
    if (outs_p.size() > 2) bad("more than two output products");
    PS = nd(scores[0]).shape;
    R = (int)PS.size();
    N = PS[R - 2], M = PS[R - 1];
    for (int s : scores)
      if (nd(s).shape != PS) bad("score products differ in shape");
    // orientation and plane operands
    std::vector<int> xs;
    bool first = true;
    for (int o : outs_p) {
      int x = nd(o).in[0];
      if (!in(x) || in(nd(o).in[1])) {
        // the right operand may be a layout view or a select of a stored tensor
        if (!in(x)) bad("an output product's left operand is not the plane");
      }
      bool tr = false;
      if (nd(x).op == KORCH_TRANSPOSE && nd(nd(x).in[0]).shape == PS && in(nd(x).in[0])) {
        const korch_attrs& a = nd(x).attrs;
        bool last2 = a.perm[R - 2] == R - 1 && a.perm[R - 1] == R - 2;
        for (int d = 0; d < R - 2; ++d) last2 = last2 && a.perm[d] == d;
        if (!last2) bad("the plane's transpose must swap its last two axes");
        tr = true;
        x = nd(x).in[0];
      }
      if (nd(x).shape != PS) bad("an output product's left operand is not the plane");
      if (!first && tr == rows_owned) bad("output products contract different axes");
      rows_owned = !tr;
      first = false;
      if (nd(x).dtype != nd(nd(o).in[1]).dtype) bad("the plane's dtype differs from the operand it is multiplied with");
      xs.push_back(x);
    }
    dtype = nd(nd(scores[0]).in[0]).dtype;
    const Shape batch(PS.begin(), PS.end() - 2);
    for (int s : scores) {
      const Node& n = nd(s);
      if (nd(n.in[0]).dtype != dtype || nd(n.in[1]).dtype != dtype) bad("operand dtypes differ");
      Operand a = operand(n.in[0], false, batch, "left score operand");
      Operand b = operand(n.in[1], true, batch, "right score operand");
      sc_own.push_back(rows_owned ? a : b);
      sc_str.push_back(rows_owned ? b : a);
      sst.push_back(add_streamed(rows_owned ? b : a));
    }
    for (size_t i = 0; i < outs_p.size(); ++i) {
      const Node& n = nd(outs_p[i]);
      if (nd(n.in[1]).dtype != dtype) bad("operand dtypes differ");
      Shape os = batch;
      os.push_back(rows_owned ? N : M);
      os.push_back(n.shape.back());
      if (n.shape != os) bad("output products differ in batch dims");
      Operand w = operand(n.in[1], false, batch, "output operand");
      out_w.push_back(w);
      ost.push_back(add_streamed(w));
    }
    std::vector<int> stats;
    for (int r : ki.reduces) (is_rowdot(r) ? rowdots : stats).push_back(r);
    if (!rowdots.empty() && !rows_owned) bad("a row sum where columns are owned");
    // softmax
    if (!stats.empty()) {
      if (stats.size() != 2 || !rows_owned || scores.size() != 1) bad("reductions other than one row softmax");
      for (int r : stats) {
        const Node& n = nd(r);
        if (n.axis != R - 1 || !n.attrs.keepdim || nd(n.in[0]).shape != PS) bad("a reduction is not along the plane's rows");
        if (n.op == KORCH_REDUCE_MAX) nm = r;
        if (n.op == KORCH_REDUCE_SUM) nl = r;
      }
      if (nm < 0 || nl < 0) bad("the softmax needs a row maximum and a row sum");
      ne = nd(nl).in[0];
      int c2 = zero_select(ne);
      nexp = c2 >= 0 ? nd(strip_identity(ne)).in[1] : ne;
      if (!in(nexp) || nd(nexp).op != KORCH_EXP) bad("the row sum is not over exponentials");
      int z = nd(nexp).in[0];
      if (!in(z) || nd(z).op != KORCH_SUB || nd(z).attrs.has_scalar || nd(z).in[1] != nm) bad("the exponent is not s - max");
      nsfinal = nd(z).in[0];
      int top = nd(nm).in[0];
      if (c2 >= 0) {
        const Node& t = nd(top);
        if (!in(top) || t.op != KORCH_SELECT || !t.attrs.has_scalar || t.in[0] != c2 || t.in[1] != nsfinal)
          bad("the row maximum must be over select(mask, s, low)");
        low = t.attrs.scalar;
        // rows' maxima start from it, masked pair or not: no score may lie below
        if (low > (nd(nsfinal).dtype == KORCH_F16 ? -6e4 : -1e9)) bad("a masked score that others may lie below");
        cond = c2;
      } else if (top != nsfinal) {
        bad("the row maximum is not over the exponent's scores");
      }
      for (size_t i = 0; i < xs.size(); ++i) {
        int x = strip_identity(xs[i]);
        if (in(x) && nd(x).op == KORCH_DIV && !nd(x).attrs.has_scalar && nd(x).in[1] == nl) {
          divided = true;
          x = strip_identity(nd(x).in[0]);
        }
        if (x != ne) bad("the softmax's product must read its exponentials");
      }
      if (outs_p.size() != 1 || bin_node >= 0) bad("a softmax kernel has one output product");
      ox.push_back(0);
    } else {
      std::vector<int> all = xs;
      if (bin_node >= 0) all.push_back(nd(bin_node).in[0]);
      bool same = true;
      for (size_t i = 0; i < all.size(); ++i) {
        if (!in(all[i]) || nd(all[i]).shape != PS) bad("plane operand outside the kernel");
        const int c = zero_select(all[i]);
        if (i == 0) cond = c;
        if (c != cond) same = false;
        int k = (int)(std::find(xnodes.begin(), xnodes.end(), all[i]) - xnodes.begin());
        if (k == (int)xnodes.size()) xnodes.push_back(all[i]);
        if (i < xs.size())
          ox.push_back(k);
        else
          xbin = k;
      }
      if (!same) cond = -1;
      if (dtype == KORCH_F16 && !outs_p.empty())
        for (int v : ki.k.prims)
          if (nd(v).op == KORCH_EXP && nd(v).shape == PS && has_score(v)) {
            bool all_by = true;
            for (int x : xnodes) all_by = all_by && times(x, v);
            if (all_by) nfactor = v;
          }
    }
    if (bin_node >= 0) {
      if (!rows_owned && !outs_p.empty()) bad("a sum by bins goes with row-owned products");
      const Node& n = nd(bin_node);
      const int tr = (int)n.shape.size();
      // result dims [.., 1, 1, T] or fewer leading ones: rows and columns are summed
      for (int d = 0; d < tr - 1; ++d) {
        const int j = d + R - (tr - 1);
        if (j >= R - 2 && n.shape[d] != 1) bad("bins along a plane axis");
      }
      if (!in(n.in[1]) || has_score(n.in[1])) bad("the bins are not computed in the kernel, or from the scores");
    }
    for (auto& w : streamed)
      if (w.shape[0] > 256) bad("an operand is wider than 256");
    // registers of a lane that live through the walk: accumulators and owned operands
    int64_t regs = 0;
    for (auto& w : out_w) regs += (w.shape[0] + 31) / 32 * 16;
    for (auto& o : sc_own) regs += (o.shape[0] + 31) / 32 * 32 * dtype_bytes(dtype) / 8;
    if (regs > 384) bad("owned operands and output products fill the registers");
    // outputs
    for (int o : ki.k.outs) {
      if (below(o) == bin_node) {
        bin_out = o;
        continue;
      }
      if (std::find(rowdots.begin(), rowdots.end(), below(o)) != rowdots.end()) continue;
      int p = -1;
      for (size_t i = 0; i < outs_p.size(); ++i)
        if (depends(o, outs_p[i])) {
          if (p >= 0) bad("an output reads two output products");
          p = (int)i;
        }
      if (p >= 0) {
        prod_of[o] = p;
      } else {
        if (nm < 0 || !(depends(o, nm) || depends(o, nl))) bad("an output is neither a product's nor a row statistic");
        const Shape& s = nd(below(o)).shape;
        Shape want(PS.begin(), PS.end() - 1);
        want.push_back(1);
        if (s != want) bad("a row statistic's shape");
      }
    }
    if (cond >= 0 && has_score(cond)) bad("a mask computed from scores");
    if (bin_node >= 0 && bin_out < 0) bad("a sum by bins that is not an output");
    for (size_t i = 0; i < outs_p.size(); ++i) {
      bool used = false;
      for (auto& [o, p] : prod_of) used = used || p == (int)i;
      if (!used) bad("an output product without an output");
    }
  }
  bool divided = false;

  // v = f times what does not depend on f (sums of such values too).
  bool times(int v, int f) const {
    if (v == f) return true;
    if (!in(v) || !depends(v, f) || nd(v).shape != PS) return false;
    const Node& n = nd(v);
    const bool one = n.in.size() == 1 || n.attrs.has_scalar;
    switch (n.op) {
      case KORCH_IDENTITY: case KORCH_NEG: return times(n.in[0], f);
      case KORCH_MUL: return one ? times(n.in[0], f) : depends(n.in[0], f) ? times(n.in[0], f) && !depends(n.in[1], f) : times(n.in[1], f);
      case KORCH_DIV: return times(n.in[0], f) && (one || !depends(n.in[1], f));
      case KORCH_ADD: case KORCH_SUB: return !one && times(n.in[0], f) && times(n.in[1], f);
      case KORCH_SELECT: return n.attrs.has_scalar && n.attrs.scalar == 0.0 && !depends(n.in[0], f) && times(n.in[1], f);
      default: return false;
    }
  }

  // sum over the last axis of x y, stored, one row for each row of the plane
  bool is_rowdot(int r) const {
    const Node& n = nd(r);
    const int x = n.in[0];
    if (n.op != KORCH_REDUCE_SUM || !n.attrs.keepdim || !in(x) || nd(x).op != KORCH_MUL || nd(x).attrs.has_scalar) return false;
    const Shape& s = nd(x).shape;
    if (n.axis != (int)s.size() - 1 || numel(n.shape) * M != numel(PS)) return false;
    for (int u : nd(x).in)
      if (in(u) || nd(u).shape != s || nd(u).dtype != dtype || s.back() * dtype_bytes(dtype) % 16) return false;
    return true;
  }
  // The rowdot that a vector is (its elements are in the plane's row order), or -1.
  int rowdot_of(int v) const {
    v = below(v);
    return std::find(rowdots.begin(), rowdots.end(), v) != rowdots.end() ? v : -1;
  }
  int rowdot_slot(int rd) const {
    for (size_t i = 0; i < ovs.size(); ++i)
      if (rowdot_of(ovs[i]) == rd) return (int)i;
    bad("a row sum that the plane does not read");
  }
  // Index of the plane's row `r`, over the whole batch.
  std::string flat_row(const char* r) const {
    std::string f = "(i64)0";
    for (int d = 0; d < R - 2; ++d) f = "(" + f + " * " + std::to_string(PS[d]) + " + b.c[" + std::to_string(d) + "])";
    return "(" + f + " * " + std::to_string(N) + "LL + " + r + ")";
  }

  // Node below the reshapes that end an output (its elements are stored in the same order).
  int below(int o) const {
    while (in(o) && nd(o).op == KORCH_RESHAPE) o = nd(o).in[0];
    return o;
  }

  // ---- emission --------------------------------------------------------------

  std::vector<Ix> plane_index() const {
    std::vector<Ix> it(R);
    for (int d = 0; d < R - 2; ++d) it[d] = Ix::var("b.c[" + std::to_string(d) + "]");
    it[R - 2] = Ix::var(rows_owned ? "ro" : "rs");
    it[R - 1] = Ix::var(rows_owned ? "rs" : "ro");
    return it;
  }
  int vec_id(std::vector<int>& list, int v) {
    auto f = std::find(list.begin(), list.end(), v);
    if (f == list.end()) {
      list.push_back(v);
      return (int)list.size() - 1;
    }
    return (int)(f - list.begin());
  }
  std::string std_key(int node, const std::vector<Ix>& it) const {
    return Emitter::key(node, broadcast_index(nd(node).shape, PS, it));
  }

  std::unique_ptr<Emitter> emitter() const {
    auto e = std::make_unique<Emitter>(g);
    e->inset = ki.in;
    e->argslot = slot;
    e->vec = 1;
    return e;
  }

  // node = c tanh(a x) on the plane, each product optional.
  bool tanh_chain(int node, int* x, double* a, double* c) const {
    *a = *c = 1.0;
    auto scaled = [&](int v) { return in(v) && nd(v).op == KORCH_MUL && nd(v).attrs.has_scalar && nd(v).shape == PS; };
    int v = node;
    if (scaled(v)) *c = nd(v).attrs.scalar, v = nd(v).in[0];
    if (!in(v) || nd(v).op != KORCH_TANH || nd(v).shape != PS) return false;
    v = nd(v).in[0];
    if (scaled(v)) *a = nd(v).attrs.scalar, v = nd(v).in[0];
    *x = v;
    return true;
  }

  static constexpr int64_t kLutMost = 4096;  // floats of all tables: 16 KiB of LDS
  static constexpr int64_t kLutPad = 32;     // a subtile

  // The table for gather `node`, or null.
  const Lut* lut_for(int node) {
    for (auto& l : luts)
      if (l.node == node) return &l;
    int v = node;
    int64_t size = 0;
    while (in(v) && nd(v).op == KORCH_GATHER) {
      const int t = nd(v).in[0];
      const Shape& ts = nd(t).shape;
      if (in(t)) return nullptr;
      // the table's leading dims: batch only (they align with the plane's, below its last axis)
      const int lr = (int)ts.size() - 1;
      if (lr > R || (lr >= 1 && ts[lr - 1] != 1) || (lr >= 2 && ts[lr - 2] != 1)) return nullptr;
      size = ts.back();
      v = nd(v).in[1];
    }
    if (v == node || cls(v) != FULLP || has_score(v) || lut_size + size + 2 * kLutPad > kLutMost) return nullptr;
    Lut l{node, v, size, (int)lut_size};
    const size_t no = ovs.size();
    if (!stepped(v, &l.step, &l.base) || l.step * l.step != 1) {
      ovs.resize(no);
      l.step = 0;
    }
    l.pad = l.step ? kLutPad : 0;
    lut_size += size + 2 * l.pad;
    luts.push_back(l);
    return &luts.back();
  }
  // node = *expr (at streamed index rs) + *step * (streamed index - rs).
  bool stepped(int v, int* step, std::string* expr) {
    const Node& n = nd(v);
    const PlaneCls c = cls(v);
    *step = 0;
    if (c != FULLP && is_owned(c)) return *expr = "ov[" + std::to_string(vec_id(ovs, v)) + "]", true;
    if (!in(v)) return false;
    if (n.op == KORCH_IOTA && is_streamed(c) && (int)n.shape.size() - n.axis == (rows_owned ? 1 : 2)) return *step = 1, *expr = "(float)(int)rs", true;
    if (n.op == KORCH_IDENTITY) return stepped(n.in[0], step, expr);
    if (n.op != KORCH_ADD && n.op != KORCH_SUB) return false;
    int s2 = 0;
    std::string x, y;
    if (!stepped(n.in[0], step, &x)) return false;
    if (n.attrs.has_scalar)
      y = flit(n.attrs.scalar);
    else if (!stepped(n.in[1], &s2, &y))
      return false;
    *step += n.op == KORCH_ADD ? s2 : -s2;
    *expr = "(" + x + (n.op == KORCH_ADD ? " + " : " - ") + y + ")";
    return true;
  }

  // Whether a mask's values are 0 and 1 only: comparisons, and their products,
  // maxima and minima.
  bool truth(int v) const {
    if (!in(v)) return false;
    const Node& n = nd(v);
    if (n.op >= KORCH_LT && n.op <= KORCH_EQ) return true;
    if (n.op == KORCH_IDENTITY) return truth(n.in[0]);
    if ((n.op == KORCH_MUL || n.op == KORCH_MAX || n.op == KORCH_MIN) && !n.attrs.has_scalar) return truth(n.in[0]) && truth(n.in[1]);
    return false;
  }

  // Body of a function that evaluates plane nodes `want` into `dst`; `full`:
  // where the mask holds (one of other values than 0 and 1 is evaluated, as its
  // value may be read beside its truth).
  std::string plane_body(const std::vector<std::pair<int, std::string>>& want, bool full) {
    auto it = plane_index();
    auto e = emitter();
    int x0 = -1;
    double ca = 1, cc = 1;
    e->provide = [&](int node, const std::vector<Ix>& idx, std::string* out) {
      for (size_t s = 0; s < scores.size(); ++s)
        if (node == scores[s]) {
          if (Emitter::key(node, idx) != std_key(node, it)) bad("a score is read at another index");
          *out = "xs[" + std::to_string(s) + "]";
          return true;
        }
      if (full && node == cond && truth(cond)) {
        *out = "(1.0f)";
        return true;
      }
      if (node == nfactor) {
        const int z = nd(node).in[0];
        const std::string x = e->value(z, broadcast_index(nd(z).shape, PS, it));
        *out = e->fresh("t");
        e->body << "    const float " << *out << " = pl_exp_by(" << x << ", sx);\n";
        return true;
      }
      if (fast_math() && tanh_chain(node, &x0, &ca, &cc)) {
        const std::string x = e->value(x0, broadcast_index(nd(x0).shape, PS, it));
        *out = e->fresh("t");
        if (std::abs(cc) <= 256)
          e->body << "    const float " << *out << " = pl_ctanh(" << x << ", " << flit(ca) << ", " << flit(cc) << ");\n";
        else  // a wide cap leaves small arguments, whose relative error counts
          e->body << "    const float " << *out << " = " << flit(cc) << " * tanhf(" << x << " * " << flit(ca) << ");\n";
        return true;
      }
      const PlaneCls c = cls(node);
      if (c == FULLP) {
        if (!in(node) || nd(node).op != KORCH_GATHER) return false;
        if (Emitter::key(node, idx) != std_key(node, it)) return false;
        const Lut* l = lut_for(node);
        if (!l) return false;
        if (l->step) {
          *out = "lb[" + std::to_string(l - luts.data()) + (l->step > 0 ? "][kk]" : "][-kk]");
          return true;
        }
        const int at = l->at, index = l->index;
        const int64_t size = l->size;
        const std::string x = e->value(index, broadcast_index(nd(index).shape, PS, it));
        *out = e->fresh("t");
        e->body << "    const float " << *out << " = lut[" << at << " + (int)k_min(k_max(" << x << ", 0.0f), " << flit((double)(size - 1)) << ")];\n";
        return true;
      }
      if ((int)nd(node).shape.size() > R) return false;
      std::string k;
      try {
        k = std_key(node, it);
      } catch (Error&) {
        return false;
      }
      if (Emitter::key(node, idx) != k) return false;
      if (in(node) && nd(node).op == KORCH_FILL) return false;
      if (is_owned(c))
        *out = "ov[" + std::to_string(vec_id(ovs, node)) + "]";
      else
        *out = "tv[" + std::to_string(vec_id(tvs, node)) + "]";
      return true;
    };
    std::string res;
    for (auto& [node, dst] : want) {
      const std::string v = e->value(node, broadcast_index(nd(node).shape, PS, it));
      e->body << "    " << dst << " = " << v << ";\n";
    }
    std::string code = e->pre.str() + e->body.str();
    // the exponential and tanh of scores: fewer instructions than the shared ones
    for (auto& [from, to] : {std::pair<std::string, std::string>{" f_tanh(", " pl_tanh("}, {" f_exp(", " pl_exp("}})
      for (size_t at = code.find(from); at != std::string::npos; at = code.find(from, at + to.size())) code.replace(at, from.size(), to);
    return code;
  }

  // Value of a vector node at owned / streamed index variable `r`.
  std::string vector_value(int node, bool owned, std::string* stmts) {
    const int rd = rowdot_of(node);
    if (rd >= 0) {
      const Node& x = nd(nd(rd).in[0]);
      if (!owned) bad("a row sum that is streamed");
      const std::string D = std::to_string(x.shape.back()), at = flat_row("r") + " * " + D;
      auto p = [&](int u) { return "(const " + ctype(dtype) + "*)a.p[" + std::to_string(slot.at(u)) + "] + " + at; };
      return "row_dot<" + D + ">(" + p(x.in[0]) + ", " + p(x.in[1]) + ")";
    }
    std::vector<Ix> it(R);
    for (int d = 0; d < R - 2; ++d) it[d] = Ix::var("b.c[" + std::to_string(d) + "]");
    const bool rows = owned == rows_owned;
    it[R - 2] = rows ? Ix::var("r") : Ix::k(0);
    it[R - 1] = rows ? Ix::k(0) : Ix::var("r");
    auto e = emitter();
    // The other axis' index is not used by a vector (its size there is 1).
    const Shape& s = nd(node).shape;
    std::vector<Ix> idx(s.size());
    for (size_t d = 0; d < s.size(); ++d) {
      const size_t j = d + R - s.size();
      idx[d] = s[d] == 1 ? Ix::k(0) : it[j];
    }
    const std::string v = e->value(node, idx);
    *stmts = e->pre.str() + e->body.str();
    return v;
  }

  // Range of a node over a tile: expression of Range functions.
  std::string range(int v) {
    const Node& n = nd(v);
    const PlaneCls c = cls(v);
    if (in(v) && n.op == KORCH_FILL) return "r_pt(" + flit(n.attrs.scalar) + ")";
    if (c != FULLP && is_owned(c)) {
      const int k = vec_id(ovs, v);
      ranged.insert(k);
      return "ow[" + std::to_string(k) + "]";
    }
    if (in(v)) {
      auto two = [&](const char* f) {
        return std::string(f) + "(" + range(n.in[0]) + ", " + (n.attrs.has_scalar ? "r_pt(" + flit(n.attrs.scalar) + ")" : range(n.in[1])) +
               ")";
      };
      auto swapped = [&](const char* f) {
        return std::string(f) + "(" + (n.attrs.has_scalar ? "r_pt(" + flit(n.attrs.scalar) + ")" : range(n.in[1])) + ", " + range(n.in[0]) +
               ")";
      };
      switch (n.op) {
        case KORCH_ADD: return two("r_add");
        case KORCH_SUB: return two("r_sub");
        case KORCH_MUL: return two("r_mul");
        case KORCH_MAX: return two("r_max");
        case KORCH_MIN: return two("r_min");
        case KORCH_LT: return two("r_lt");
        case KORCH_LE: return two("r_le");
        case KORCH_GT: return swapped("r_lt");
        case KORCH_GE: return swapped("r_le");
        case KORCH_EQ: return two("r_eq");
        case KORCH_NEG: return "r_neg(" + range(n.in[0]) + ")";
        case KORCH_ABS: return "r_abs(" + range(n.in[0]) + ")";
        case KORCH_IDENTITY: return range(n.in[0]);
        default: break;
      }
    }
    if (c == FULLP) return "r_all()";
    // a streamed vector: an index along the streamed axis is known, others are read
    if (in(v) && n.op == KORCH_IOTA && (int)n.shape.size() - n.axis == (rows_owned ? 1 : 2)) return "Range{s0, s1}";
    return "rv[" + std::to_string(vec_id(rvs, v)) + "]";
  }

  // Splits of the streamed axis and geometry.
  int NW = 4, TS = 64, SPLIT = 1, STAGES = 2, WPE = 1, OCC = 1;
  bool WSPLIT = false, DMA = true;
  int64_t OTILES = 1, NB = 1, TP = 1, SEG = 1;

  size_t lds_bytes() const {
    const int es = dtype_bytes(dtype);
    size_t tile = 0;
    int nreg = 0;
    for (auto& w : streamed) tile += (size_t)TS * ((w.shape[0] + 31) / 32 * 32) * es;
    for (auto& w : out_w) nreg += (int)((w.shape[0] + 31) / 32 * 32) / 2;
    tile += (size_t)tvs.size() * TS * 4;
    size_t tiles = tile * STAGES * (WSPLIT ? NW : 1);
    size_t merge = WSPLIT ? (size_t)NW * (nreg + 2) * 256 : 0;
    size_t bins = bin_node >= 0 ? (size_t)NW * nd(bin_node).shape.back() * 256 : 0;
    return std::max(tiles, merge) + 4096 + (NW * ovs.size() * 2 + 8) * 4 + 80 + (lut_size + 3) / 4 * 16 + bins;
  }

  // A vector that depends on a stored tensor (positions do not).
  bool reads_data(int v) const {
    if (!in(v)) return true;
    for (int u : nd(v).in)
      if (reads_data(u)) return true;
    return false;
  }

  // Tiles, waves and LDS for workgroups whose waves share tiles or (ws) split the streamed axis.
  void layout(bool ws, int waves) {
    const bool f32 = dtype == KORCH_F32;
    // Registers that live through the walk.  With up to 160 of them two waves fit
    // a SIMD; one computes while the other loads, reduces or waits (2x16 heads of
    // 4096 x 4096, width 128, bf16: 275 us against 343 with one, the queries'
    // gradients 374 against 511).  Gradients of the keys at width 128 hold 192:
    // one wave per SIMD (two spill and gain nothing: 720 to 800 us either way).
    int live = 0;
    for (auto& w : out_w) live += (int)((w.shape[0] + 31) / 32 * 16);
    for (auto& o : sc_own) live += (int)((o.shape[0] + 31) / 32 * 32 * dtype_bytes(dtype) / 8);
    WPE = live > 160 || reg_relief() > 0 ? 1 : 2;
    WSPLIT = ws;
    // Streamed rows of a tile: 64, or 32 where registers are short (two score
    // planes at two waves per SIMD: 372 us against 398; a wave's own tiles, whose
    // rows it loads alone: 62 us against 64 for 16 caches of up to 8192, width 128).
    TS = f32 || WSPLIT || (nm < 0 && WPE == 2) ? 32 : 64;
    NW = waves;
    // Tiles go straight to LDS, into a second stage while the first is read.  A
    // wave's own tiles pass through its registers instead, as long as it has
    // them: with one stage two workgroups fit a compute unit's LDS, and their
    // loads keep twice the bytes in flight (those caches: 62 us, straight to LDS 245).
    int staging = 0;
    for (auto& w : streamed) staging += (int)(TS * w.shape[0] * dtype_bytes(dtype) / 256);
    DMA = !WSPLIT || live + staging > 224;
    STAGES = DMA ? 2 : 1;
    const size_t lds_most = 160 * 1024;
    while (lds_bytes() > lds_most && TS > 32) TS /= 2;
    while (lds_bytes() > lds_most && NW > 1) NW /= 2;
    while (lds_bytes() > lds_most && STAGES > 1) STAGES = 1;
    if (lds_bytes() > lds_most) bad("operands exceed the 160 KiB of LDS");
    OCC = (int)std::max<int64_t>(1, std::min<int64_t>(WPE * 4 / NW, (int64_t)(lds_most / lds_bytes())));
  }

  void geometry() {
    NB = 1;
    for (int d = 0; d < R - 2; ++d) NB *= PS[d];
    const int64_t nown = rows_owned ? N : M, nstr = rows_owned ? M : N;
    // (Times of fp16 gradients below are without their values' scale, which adds 3 to
    // 9 % on either side.)
    // Few owned indices: the waves of a workgroup share 32 of them and split the
    // streamed axis, joined through LDS (more waves at work, no barrier between
    // tiles; every wave loads its own tiles).  Up to one and a half such
    // workgroups for each that the chip holds: 4 heads of 2048 x 2048, width 64,
    // fp16, half as many, forward 15 us, gradients 17 and 20 (shared tiles 20, 24
    // and 33); 12 heads, one and a half times, 33, 38 and 45 (31, 40 and 57); 8
    // heads of width 128, whose gradients take a compute unit each, twice as many
    // 63 and 67 (47 and 74).
    const int64_t own32 = (nown + 31) / 32 * NB;
    bool data = false;  // the mask reads data along the streamed axis: nobody knows which tiles have work
    for (int v : rvs) data = data || (cond >= 0 && reads_data(v));
    int64_t pcols = 0, acols = 0;
    for (auto& o : sc_own) pcols += o.shape[0];
    for (auto& w : out_w) pcols += w.shape[0], acols += (w.shape[0] + 31) / 32 * 32;
    layout(true, 4);
    // Gradients of packed documents: the longest walks decide, and two waves that
    // split one halve it.  12 heads of 4000 rows, width 64, fp16 (rows / columns
    // owned, without rowsum(dO O)): 11 documents 25.6 / 34.7 us, shared tiles 30.5 / 39; 3 documents 44 /
    // 55 (60 / 87); 200 documents 20 / 25 (18 / 23).  Width 128 loads too much that
    // way (50 us, 40), and so do twice as many heads of 8000 (97, 83).
    if (own32 > 384 * OCC && data && nm < 0 && pcols <= 256) layout(true, 2);
    // Shared tiles: four waves, or two where a mask along the diagonal cuts short
    // walks (64 owned rows see fewer masked pairs): causal 8x12 heads of 512 rows,
    // width 64, fp16, forward 12.9 us, gradients 18.9 and 21.8 (four waves 15.1, 21.0
    // and 24.3); 16x12 heads of 1000 60.7, 84 and 107 (61.6, 88 and 112).  Width 128
    // (65 us, two waves 89) and masks without a diagonal (25, 26) keep four.
    bool diagonal = false;
    for (int k : ranged) diagonal = diagonal || cls(ovs[k]) != CONSTV;
    int64_t widest = 0;
    for (auto& w : streamed) widest = std::max(widest, w.shape[0]);
    if (own32 > 384 * OCC) layout(false, diagonal && nstr <= 1024 && widest <= 64 ? 2 : 4);
    const int OT = WSPLIT ? 32 : 32 * NW;
    // Positions repeat along the rows when the heads of a group share them.  With a
    // mask no tile holds the end of one head and the start of the next (it would
    // see every key): each head starts a tile, where that adds a quarter at most
    // (16 heads on 4 of 4000 rows, eleven documents, width 64, fp16: 25 us, 130).
    SEG = nown;
    for (int v : ki.k.prims) {
      const Node& n = nd(v);
      if (n.op != KORCH_IOTA || numel(n.shape) != nown || !rows_owned || cond < 0) continue;
      const int64_t period = n.shape[n.axis];
      if (period < nown && nown % period == 0 && (period + OT - 1) / OT * OT * 4 <= period * 5) SEG = period;
    }
    TP = (SEG + OT - 1) / OT;
    OTILES = nown / SEG * TP;
    const int64_t wgs = OTILES * NB, tiles = (nstr + TS - 1) / TS, per = WSPLIT ? NW : 1;
    // The streamed axis is split over workgroups where that shortens the walk by
    // more than the hand-over takes: about 1.5 us, and the partial results, which
    // pass the device's point of coherence at about 0.8 TB/s (written and read).
    // A tile of 32 takes a wave about 0.3 us and 3.3 ns per column of all products
    // (16-bit; 20 ns in fp32).  Splits beyond the workgroups that are resident at
    // once gain nothing (2048 x 2048, one head of 128, fp16: 13.0 us in 4 splits,
    // 19.5 in one, 18.7 in 8), unless a mask of positions makes them unequal: then
    // up to twice as many (keys' gradient of 8 key heads of 2048 causal positions
    // with four query heads each, width 128: 143 us in 4 splits, 192 in 2).  Where
    // waves split the axis too, for owned columns only, and where the model sees a
    // clear gain (16 heads on 4 of 2800, width 40, fp16: 73 us in two splits, 116 in
    // one; owned rows lose: one token over 16 x 8192 keys 80 us, 62).
    SPLIT = 1;
    const bool uneven = cond >= 0 && !data;
    const double t_tile = (0.3 + (dtype == KORCH_F32 ? 0.02 : 0.0033) * (double)pcols) * TS / 32;
    const double t_part = (double)(wgs * OT * acols) * 4 / 0.8e6;
    if (workgroup_splits()) {
      const int64_t walk = (tiles + per - 1) / per, slots = 256 * OCC * (uneven && !(WSPLIT && rows_owned) ? 2 : 1);
      double best = (double)walk * t_tile;
      for (int64_t q = 2; q <= std::min<int64_t>({walk, 32, slots / std::max<int64_t>(1, wgs)}); ++q) {
        const double t = (double)((walk + q - 1) / q) * t_tile + 1.5 + (double)q * t_part;
        if (t < best * (WSPLIT && wgs * q > 256 * OCC ? 0.85 : 1.0)) best = t, SPLIT = (int)q;
      }
      // Shared tiles that fill the chip once and are long: 16 heads of 4096 causal
      // rows of width 128 take 116 us in two splits, 123 in one; 32 of 2048 rows
      // 75 and 67.  (A mask that reads data, as documents do, leaves few tiles: 12
      // heads of 4000 rows 33 us in two splits, 24.5 in one.)
      if (!WSPLIT && uneven && wgs >= 256) SPLIT = wgs <= 256 * OCC && nstr >= 2560 ? 2 : 1;
    }
    if (wgs * SPLIT * NW * 64 >= (int64_t)1 << 32) bad("more threads than a launch holds");
  }

  GenKernel generate(int index) {
    const bool f32 = dtype == KORCH_F32;
    set_fast_math(!f32);
    GenKernel gk;
    gk.family = KORCH_FAM_PLANE;
    gk.name = kernel_name(index, "plane");
    ki.assign_args(gk, slot);
    const std::string T = ctype(dtype);
    const bool softmax = nm >= 0;
    // The mask, the bins and the vectors that they read round after every
    // primitive: a fused multiply-add could lie outside the range that the same
    // primitives give for a tile.
    const std::string apart = "#pragma clang fp contract(off)\n";
    // functions on the plane where the mask holds, and the mask
    std::vector<std::pair<int, std::string>> want;
    // Scores that are only a product with a constant > 0: the maximum is taken of
    // the products as they are and the constant enters the exponent's.
    double fold = 1.0;
    if (softmax && nsfinal != scores[0] && nd(nsfinal).op == KORCH_MUL && nd(nsfinal).attrs.has_scalar && nd(nsfinal).in[0] == scores[0] &&
        nd(nsfinal).attrs.scalar > 1e-3 && nd(nsfinal).attrs.scalar < 1e3)
      fold = nd(nsfinal).attrs.scalar;
    if (softmax)
      want.push_back({fold != 1.0 ? scores[0] : nsfinal, "const float v_"});
    else
      for (size_t i = 0; i < xnodes.size(); ++i) want.push_back({xnodes[i], "out[" + std::to_string(i) + "]"});
    const std::string fn = plane_body(want, true) + (softmax ? "    return v_;\n" : "");
    const std::string keep_fn = cond >= 0 ? plane_body({{cond, "const float k_"}}, false) + "    return k_ != 0.0f;\n" : "    return true;\n";
    std::string bin_fn;
    if (bin_node >= 0) bin_fn = plane_body({{nd(bin_node).in[1], "const float id_"}}, false);
    std::string mask_expr = cond >= 0 ? range(cond) : "";
    geometry();
    // vectors
    std::ostringstream p;
    const int64_t nown = rows_owned ? N : M, nstr = rows_owned ? M : N;
    p << "struct Pol {\n  typedef " << T << " T;\n  struct B {\n    i64 c[" << std::max(1, R - 2) << "];\n  };\n";
    p << "  static constexpr bool SOFTMAX = " << softmax << ", MASK = " << (cond >= 0) << ", WSPLIT = " << WSPLIT << ", DMA = " << DMA << ", SCALED = " << (nfactor >= 0)
      << ";\n";
    p << "  static constexpr i64 SEG = " << SEG << "LL, NSTR = " << nstr << "LL;\n";
    p << "  static constexpr int NW = " << NW << ", TS = " << TS << ", STAGES = " << STAGES << ", SPLIT = " << SPLIT << ", OTILES = " << OTILES
      << ", NB = " << NB << ", TP = " << TP << ", OCC = " << OCC << ", WPE = " << WPE << ";\n  static constexpr bool LAST_FIRST = " << rows_owned << ";\n";
    const int64_t nbin = bin_node >= 0 ? nd(bin_node).shape.back() : 0;
    p << "  static constexpr int NSP = " << scores.size() << ", NST = " << streamed.size() << ", NOP = " << outs_p.size() << ", NX = "
      << std::max<size_t>(1, xnodes.size()) << ", NBIN = " << nbin << ", XBIN = " << std::max(0, xbin) << ";\n";
    p << "  static constexpr int NTAB = " << tvs.size() << ", NOV = " << ovs.size() << ", NRV = " << rvs.size() << ";\n";
    p << "  static constexpr float MINIT = " << flit(softmax && cond >= 0 ? low / fold : -INFINITY)
      << ", LOW = " << flit(softmax && cond >= 0 ? low : -INFINITY) << ", FOLD = " << flit(fold) << ";\n";
    auto table = [&](const char* name, const std::vector<int>& v) {
      p << "  static constexpr int " << name << "(int i) {\n    constexpr int t[] = {";
      for (int x : v) p << x << ", ";
      p << "0};\n    return t[i];\n  }\n";
    };
    std::vector<int> sw;
    for (auto& w : streamed) sw.push_back((int)w.shape[0]);
    table("sw", sw);
    std::vector<int> rs;
    for (auto& w : streamed) {
      if (w.stride * TS * dtype_bytes(dtype) >= (int64_t)1 << 30) bad("rows too far apart");
      rs.push_back((int)w.stride);
    }
    table("srs", rs);
    table("sst", sst);
    table("ost", ost);
    table("ox", ox);
    std::vector<int> rm, om;
    for (auto& w : streamed) rm.push_back(w.mask >= 0);
    for (auto& w : sc_own) om.push_back(w.mask >= 0);
    p << "  static constexpr bool row_mask(int i) {\n    constexpr bool t[] = {";
    for (int x : rm) p << x << ", ";
    p << "0};\n    return t[i];\n  }\n  static constexpr bool own_mask(int i) {\n    constexpr bool t[] = {";
    for (int x : om) p << x << ", ";
    p << "0};\n    return t[i];\n  }\n";
    // batch coordinates
    p << "  static __device__ __forceinline__ B batch(int l) {\n    B b;\n    i64 q = l;\n";
    for (int d = R - 3; d >= 0; --d)
      p << "    b.c[" << d << "] = q % " << PS[d] << "; q /= " << PS[d] << ";\n";
    if (R == 2) p << "    b.c[0] = q;\n";
    p << "    return b;\n  }\n";
    // operand rows
    auto rows = [&](const char* fnn, const std::vector<Operand>& v, const char* okn) {
      p << "  template <int t> static __device__ __forceinline__ const T* " << fnn << "(const KArgs& a, const B& b, i64 r) {\n";
      for (size_t i = 0; i < v.size(); ++i)
        p << "    if constexpr (t == " << i << ") return (const T*)a.p[" << slot.at(v[i].root) << "] + " << v[i].off << ";\n";
      p << "  }\n";
      p << "  template <int t> static __device__ __forceinline__ bool " << okn << "(const KArgs& a, const B& b, i64 r) {\n" << apart;
      for (size_t i = 0; i < v.size(); ++i) {
        if (v[i].mask < 0) continue;
        auto e = emitter();
        const std::string x = e->value(v[i].mask, mask_idx.at(v[i].node));
        p << "    if constexpr (t == " << i << ") {\n" << e->pre.str() << e->body.str() << "    return " << x << " != 0.0f;\n    }\n";
      }
      p << "    return true;\n  }\n";
    };
    rows("srow", streamed, "srow_ok");
    rows("orow", sc_own, "orow_ok");
    auto vectors = [&](const char* name, const std::vector<int>& v, bool owned) {
      p << "  static __device__ __forceinline__ float " << name << "(const KArgs& a, const B& b, int k, i64 r) {\n" << apart;
      for (size_t i = 0; i < v.size(); ++i) {
        std::string st;
        const std::string x = vector_value(v[i], owned, &st);
        p << "    if (k == " << i << ") {\n" << st << "    return " << x << ";\n    }\n";
      }
      p << "    return 0.0f;\n  }\n";
    };
    vectors("own", ovs, true);
    vectors("tab", tvs, false);
    vectors("rvec", rvs, false);
    p << "  static __device__ __forceinline__ Range mask_range(const KArgs& a, const B& b, const Range* ow, const Range* rv, float s0, float s1) {\n" << apart;
    p << "    return " << (cond >= 0 ? mask_expr : "r_pt(1.0f)") << ";\n  }\n";
    const std::string sig = "(const KArgs& a, const B& b, const float* ov, const float* tv, const float* lut, const LdsFloat* lb, int kk, i64 ro, i64 rs";
    p << "  static __device__ __forceinline__ " << (softmax ? "float logit" : "void plane") << sig << ", const float* xs" << (softmax ? "" : ", float sx, float* out")
      << ") {\n" << fn << "  }\n";
    p << "  static __device__ __forceinline__ bool keep" << sig << ") {\n" << apart << "    const float xs[2] = {};\n" << keep_fn << "  }\n";
    if (bin_node >= 0)
      p << "  static __device__ __forceinline__ float bin" << sig << ") {\n" << apart
        << "    const float xs[2] = {};\n" << bin_fn << "    return k_min(k_max(id_, 0.0f), " << flit((double)(nbin - 1)) << ");\n  }\n";
    // where the tables of stepped indices are read from a subtile's first streamed index on
    p << "  static constexpr int NLUT = " << luts.size() << ";\n";
    p << "  static __device__ __forceinline__ void bases(const float* ov, const float* lut, i64 rs, LdsFloat* lb) {\n" << apart;
    for (size_t i = 0; i < luts.size(); ++i)
      if (luts[i].step)
        p << "    lb[" << i << "] = lds_base(lut + " << luts[i].at + luts[i].pad << " + (int)floorf(k_min(k_max(" << luts[i].base << ", "
          << flit(luts[i].step > 0 ? -(double)luts[i].pad : 0) << "), " << flit((double)(luts[i].size - 1 + (luts[i].step > 0 ? 0 : luts[i].pad))) << ")));\n";
    p << "  }\n";
    p << "  static constexpr int LUT = " << lut_size << ";\n  static __device__ __forceinline__ float lut_value(const KArgs& a, const B& b, int k) {\n" << apart;
    for (auto& l : luts) {
      auto e = emitter();
      e->provide = [&](int node, const std::vector<Ix>&, std::string* out) { return node == l.index ? (*out = "kf", true) : false; };
      std::vector<Ix> it = plane_index();
      it[R - 2] = it[R - 1] = Ix::k(0);  // the tables do not vary along them
      std::vector<Ix> idx(nd(l.node).shape.size());
      for (size_t d = 0; d < idx.size(); ++d) idx[d] = nd(l.node).shape[d] == 1 ? Ix::k(0) : it[d + R - idx.size()];
      const std::string x = e->value(l.node, idx);
      p << "    if (k < " << l.at + l.size + 2 * l.pad << ") {\n    const float kf = k_min(k_max((float)(k - " << l.at + l.pad << "), 0.0f), "
        << flit((double)(l.size - 1)) << ");\n" << e->pre.str() << e->body.str() << "    return " << x
        << ";\n    }\n";
    }
    p << "    return 0.0f;\n  }\n";
    if (bin_node >= 0) {
      // range of the index whose table gives the bins, and the bins at the table's ends
      const int id = nd(bin_node).in[1];
      const Lut* l = nullptr;
      for (auto& x : luts)
        if (x.node == id) l = &x;
      std::string r = "r_all()", first = "0.0f", last = "0.0f";
      if (l) {
        const size_t nr = rvs.size(), no = ovs.size();
        std::string e = range(l->index);
        if (rvs.size() == nr && ovs.size() == no) {
          r = e;
          first = "lut[" + std::to_string(l->at + l->pad) + "]";
          last = "lut[" + std::to_string(l->at + l->pad + l->size - 1) + "]";
        } else {  // its range needs a vector that the kernel does not hold
          rvs.resize(nr);
          ovs.resize(no);
        }
      }
      p << "  static constexpr int BIN_T = " << (l ? l->size : 1) << ";\n";
      p << "  static __device__ __forceinline__ Range bin_range(const KArgs& a, const B& b, const Range* ow, float s0, float s1) {\n" << apart << "    return "
        << r << ";\n  }\n";
      p << "  static __device__ __forceinline__ float bin_end(const float* lut, bool high) { return k_min(k_max(high ? " << last << " : " << first
        << ", 0.0f), " << flit((double)(nbin - 1)) << "); }\n";
    }
    p << "  static constexpr bool ranged(int k) {\n    constexpr bool t[] = {";
    for (size_t k = 0; k < ovs.size(); ++k) p << (ranged.count((int)k) > 0) << ", ";
    p << "0};\n    return t[k];\n  }\n";
    // results
    p << "  template <int o> static __device__ __forceinline__ void store(const KArgs& a, const B& b, i64 ro, int dim, float m, float l, f32x4 v) {\n";
    for (size_t i = 0; i < outs_p.size(); ++i) {
      p << "    if constexpr (o == " << i << ") {\n";
      for (auto& [o, pi] : prod_of)
        if (pi == (int)i) p << store_code(o, (int)i);
      p << "    }\n";
    }
    p << "  }\n";
    p << "  static constexpr bool ROWOUT = " << !rowdots.empty() << ";\n  static __device__ __forceinline__ void row_out(const KArgs& a, const B& b, i64 ro, const float* ov) {\n";
    for (int o : ki.k.outs)
      if (rowdot_of(o) >= 0)
        p << "    st1((" << ctype(nd(o).dtype) << "*)a.p[" << ki.out_slot(o) << "] + " << flat_row("ro") << ", ov[" << rowdot_slot(below(o)) << "]);\n";
    p << "  }\n";
    p << "  static __device__ __forceinline__ void stats(const KArgs& a, const B& b, i64 ro, float m, float l) {\n";
    for (int o : ki.k.outs) {
      if (o == bin_out || prod_of.count(o) || rowdot_of(o) >= 0) continue;
      auto e = emitter();
      std::vector<Ix> it(R);
      for (int d = 0; d < R - 2; ++d) it[d] = Ix::var("b.c[" + std::to_string(d) + "]");
      it[R - 2] = Ix::var("ro");
      it[R - 1] = Ix::k(0);
      e->provide = [&](int node, const std::vector<Ix>&, std::string* out) {
        if (node == nm) return *out = "m", true;
        if (node == nl) return *out = "l", true;
        return false;
      };
      const std::string v = e->value(below(o), it);
      auto st = strides_of(nd(below(o)).shape);
      Ix off = Ix::k(0);
      for (int d = 0; d < R; ++d) off = ix_add(off, ix_mulk(it[d], st[d], 1));
      p << "    {\n" << e->pre.str() << e->body.str() << "    st1((" << ctype(nd(o).dtype) << "*)a.p[" << ki.out_slot(o) << "] + " << off.b
        << ", " << v << ");\n    }\n";
    }
    p << "  }\n";
    if (bin_node >= 0) {
      const Node& n = nd(bin_node);
      const int tr = (int)n.shape.size();
      std::string row = "0", member = "0";
      int64_t members = 1, rows_n = 1;
      for (int d = 0; d < R - 2; ++d) {
        const int j = d - (R - (tr - 1));
        const bool kept = j >= 0 && n.shape[j] != 1;
        std::string c = "b.c[" + std::to_string(d) + "]";
        if (kept)
          row = "(" + row + " * " + std::to_string(PS[d]) + " + " + c + ")", rows_n *= PS[d];
        else
          member = "(" + member + " * " + std::to_string(PS[d]) + " + " + c + ")", members *= PS[d];
      }
      p << "  static constexpr int BIN_MEMBERS = " << members << ";\n";
      p << "  static __device__ __forceinline__ int bin_row(const B& b) { return (int)" << row << "; }\n";
      p << "  static __device__ __forceinline__ int bin_member(const B& b) { return (int)" << member << "; }\n";
      p << "  static __device__ __forceinline__ void store_bin(const KArgs& a, int row, int k, float v) { st1((" << ctype(nd(bin_out).dtype) << "*)a.p["
        << ki.out_slot(bin_out) << "] + (i64)row * " << nbin << " + k, v); }\n";
      ArgRef scr;
      scr.kind = ArgRef::Scratch;
      scr.bytes = (size_t)(rows_n * members * OTILES * SPLIT * nbin) * 4;
      p << "  static constexpr int BSCR = " << gk.args.size() << ";\n";
      gk.args.push_back(scr);
      ArgRef cnt;
      cnt.kind = ArgRef::Counter;
      cnt.bytes = (size_t)rows_n * 128;
      p << "  static constexpr int BCNT = " << gk.args.size() << ";\n";
      gk.args.push_back(cnt);
    }
    gk.wg_split = SPLIT > 1;
    if (SPLIT > 1 && !outs_p.empty()) {
      int nreg = 0;
      for (auto& w : out_w) nreg += (int)((w.shape[0] + 31) / 32 * 32) / 2;
      ArgRef scr;
      scr.kind = ArgRef::Scratch;
      scr.bytes = (size_t)(NB * OTILES) * SPLIT * (WSPLIT ? 1 : NW) * (nreg / 4 + 1) * 1024;
      p << "  static constexpr int SCR = " << gk.args.size() << ";\n";
      gk.args.push_back(scr);
      ArgRef cnt;
      cnt.kind = ArgRef::Counter;
      cnt.bytes = (size_t)(NB * OTILES) * 128;
      p << "  static constexpr int CNT = " << gk.args.size() << ";\n";
      gk.args.push_back(cnt);
    }
    p << "};\n";
    std::ostringstream src;
    src << source_header((int)gk.args.size()) << k_device_plane << "\n" << p.str();
    src << "extern \"C\" __global__ void __launch_bounds__(" << NW * 64 << ") __attribute__((amdgpu_waves_per_eu(" << WPE << ", " << WPE << "))) " << gk.name << "(KArgs a) {\n";
    src << "  __shared__ __attribute__((aligned(16))) char smem[Geo<Pol>::bytes];\n  Plane<Pol> k(a, smem);\n  k.run();\n}\n";
    gk.source = src.str();
    gk.grid[0] = (int)(OTILES * NB * SPLIT);
    gk.block[0] = NW * 64;
    gk.lds_bytes = (int)lds_bytes();
    ki.fill_cost(gk);
    return gk;
  }

  // Epilogue of output `o` (product i): four consecutive elements of a row.
  std::string store_code(int o, int i) {
    const Shape& os = nd(outs_p[i]).shape;  // [batch.., own, width]
    const int r = (int)os.size();
    std::vector<Ix> it(r);
    for (int d = 0; d < r - 2; ++d) it[d] = Ix::var("b.c[" + std::to_string(d) + "]");
    it[r - 2] = Ix::var("ro");
    it[r - 1] = Ix::var("dim", 1, 4);
    // a transpose that ends the output changes where its elements are stored
    const int top = below(o);
    int v = top;
    std::vector<int> perm(r);
    for (int d = 0; d < r; ++d) perm[d] = d;
    while (in(v) && nd(v).op == KORCH_TRANSPOSE && v != outs_p[i]) {
      std::vector<int> q(r);
      if (nd(v).attrs.rank != r) bad("an output's transpose changes its rank");
      for (int d = 0; d < r; ++d) q[d] = nd(v).attrs.perm[perm[d]];
      perm = q;
      v = nd(v).in[0];
    }
    if (nd(v).shape != os) bad("an output's shape differs from its product's");
    auto e = emitter();
    e->vec = 4;
    const std::string key = Emitter::key(outs_p[i], it);
    e->provide = [&](int node, const std::vector<Ix>& idx, std::string* out) {
      if (node == outs_p[i]) {
        if (Emitter::key(node, idx) != key) bad("an output product is read at another index");
        *out = divided ? binary_expr(KORCH_DIV, "v[e]", "l") : "v[e]";
        return true;
      }
      if (node == nm && nm >= 0) return *out = "m", true;
      if (node == nl && nl >= 0) return *out = "l", true;
      return false;
    };
    const std::string x = e->value(v, it);
    auto st = strides_of(nd(top).shape);
    Ix off = Ix::k(0);
    // stored element [i_0, ..] of o is v's element with index it[perm]
    for (int d = 0; d < r; ++d) off = ix_add(off, ix_mulk(it[perm[d]], st[d], 4));
    if (!off.affine || off.c != 1) bad("an output's rows are not consecutive");
    bool al = true;
    for (int d = 0; d < r; ++d)
      if (perm[d] != r - 1 && nd(top).shape[d] > 1 && st[d] % 4) al = false;
    std::ostringstream s;
    s << "      {\n" << e->pre.str() << "      float y[4];\n#pragma unroll\n      for (int e = 0; e < 4; ++e) {\n" << e->body.str()
      << "      y[e] = " << x << ";\n      }\n";
    const std::string P = "((" + ctype(nd(o).dtype) + "*)a.p[" + std::to_string(ki.out_slot(o)) + "])";
    if (!al) bad("an output's rows are not aligned");
    s << "      " << out_store(g, o, P, off.b, 4, "y") << ";\n      }\n";
    return s.str();
  }
};

}  // namespace

bool match_plane(const KInfo& ki, std::string* why) {
  if (ki.linear.size() < 2) {
    *why = "plane: fewer than two products";
    bool bins = false;
    for (int v : ki.k.prims) bins = bins || ki.g.nodes[v].op == KORCH_BIN_SUM;
    if (!bins || ki.linear.empty()) return false;
  }
  try {
    PlaneGen p(ki);
    p.analyze();
    p.generate(0);
  } catch (Error& e) {
    *why = e.what();
    return false;
  }
  return true;
}

GenKernel gen_plane(const KInfo& ki, int index) {
  PlaneGen p(ki);
  p.analyze();
  return p.generate(index);
}

}  // namespace korch
