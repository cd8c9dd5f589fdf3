// Rotary positions: heads [B, H, N, D] whose first 2 P dims turn in pairs by
// angles that all heads of a token share,
//   (x1, x2) -> (x1 c - x2 s, x2 c + x1 s)   (the turn back: s negated),
// the rest copied; several such tensors, and tensors that are only copied, in one
// kernel, read and written through slices, transposes and concatenations of
// whole heads (a projection's packed product on one side, heads before tokens
// on the other).
//
// HBM bound: every head is read and written once.  A workgroup takes a few
// tokens and a range of heads, evaluates each (token, pair)'s cosine and sine
// once, by one thread, and keeps them in LDS for all its heads; so the angles
// (in 64 bits, some hundred cycles) cost little beside the 2 x H x 2 elements
// that they turn.
#include <algorithm>

#include "families.h"

namespace korch {

namespace {

struct Src {
  int ext = -1;
  int64_t off = 0;
  std::vector<int64_t> st;
};

struct Piece {
  bool turned = false, back = false;
  Src x;                        // first element of a head: strides of image, head, token (and 1 along a head)
  int64_t heads = 0, D = 0;
  int out = -1;
  int64_t off = 0;
  std::vector<int64_t> st;      // of the output, likewise
};

struct RotaryGen {
  const KInfo& ki;
  const Graph& g;
  int64_t B = 0, N = 0, pairs = 0;
  int co = -1, si = -1;
  bool interleaved = false;
  std::vector<Piece> pieces;

  RotaryGen(const KInfo& k) : ki(k), g(k.g) {}
  [[noreturn]] static void bad(const std::string& m) { fail(KORCH_E_UNSUPPORTED, "rotary: " + m); }
  const Node& nd(int v) const { return g.nodes[v]; }
  bool in(int v) const { return ki.in.count(v) > 0; }

  // Where the elements of a layout chain lie in its stored tensor.
  Src source(int v) const {
    if (!in(v)) {
      Src s;
      s.ext = v;
      s.st = strides_of(nd(v).shape);
      return s;
    }
    const Node& n = nd(v);
    if (n.op == KORCH_SLICE || n.op == KORCH_TRANSPOSE || n.op == KORCH_RESHAPE) {
      if (n.dtype != nd(n.in[0]).dtype) bad("a layout primitive that rounds");
      Src s = source(n.in[0]);
      if (n.op == KORCH_SLICE) {
        for (size_t d = 0; d < s.st.size(); ++d) s.off += n.attrs.begin[d] * s.st[d];
      } else if (n.op == KORCH_TRANSPOSE) {
        std::vector<int64_t> t(s.st.size());
        for (size_t d = 0; d < t.size(); ++d) t[d] = s.st[n.attrs.perm[d]];
        s.st = t;
      } else {
        // the last dim split in two
        const Shape& a = nd(n.in[0]).shape;
        const Shape& b = n.shape;
        if (b.size() != a.size() + 1 || !std::equal(a.begin(), a.end() - 1, b.begin())) bad("a reshape that is not a split of the last dim");
        const int64_t last = s.st.back();
        s.st.back() = last * b.back();
        s.st.push_back(last);
      }
      return s;
    }
    bad(std::string("a head is read through ") + op_name(n.op));
  }

  int strip(int v) const {
    return in(v) && nd(v).op == KORCH_RESHAPE ? nd(v).in[0] : v;
  }

  // mul(x, angle's cosine or sine), in either order; the factor has one head
  bool product(int v, int& x, int& f) const {
    if (!in(v) || nd(v).op != KORCH_MUL || nd(v).attrs.has_scalar) return false;
    for (int side = 0; side < 2; ++side) {
      x = nd(v).in[side], f = nd(v).in[1 - side];
      const Shape& xs = nd(x).shape;
      const Shape& fs = nd(f).shape;
      if (xs == nd(v).shape && fs.size() == xs.size() && fs.size() >= 4 && fs[1] == 1 && (xs[1] > 1 || side == 0)) return true;
    }
    return false;
  }

  bool same(const Src& a, const Src& b, int64_t apart) const { return a.ext == b.ext && a.st == b.st && b.off == a.off + apart; }

  // Is v a turned tensor [B, H, N, D]?  Fills p.
  bool turned(int v, Piece& p) {
    if (!in(v)) return false;
    const Shape& sh = nd(v).shape;
    if (sh.size() != 4) return false;
    int ab = v, rest = -1;
    bool inter = false;
    if (nd(v).op == KORCH_RESHAPE) {
      ab = nd(v).in[0], inter = true;
    } else if (nd(v).op == KORCH_CONCAT && nd(v).axis == 3) {
      if (nd(v).in.size() == 3) {
        rest = nd(v).in[2];
      } else if (nd(v).in.size() == 2 && in(nd(v).in[0]) && nd(nd(v).in[0]).op == KORCH_RESHAPE) {
        rest = nd(v).in[1], ab = nd(nd(v).in[0]).in[0], inter = true;
      } else if (nd(v).in.size() != 2) {
        return false;
      }
    } else {
      return false;
    }
    if (!in(ab) || nd(ab).op != KORCH_CONCAT || nd(ab).axis != (inter ? 4 : 3) || (inter && nd(ab).in.size() != 2)) return false;
    const int a = nd(ab).in[0], b = nd(ab).in[1];
    if (!in(a) || !in(b)) return false;
    p.back = nd(a).op == KORCH_ADD;
    if (nd(a).op != (p.back ? KORCH_ADD : KORCH_SUB) || nd(b).op != (p.back ? KORCH_SUB : KORCH_ADD) || nd(a).attrs.has_scalar || nd(b).attrs.has_scalar) return false;
    int x1, c1, x2, s1, y2, c2, y1, s2;
    if (!product(nd(a).in[0], x1, c1) || !product(nd(a).in[1], x2, s1) || !product(nd(b).in[0], y2, c2) || !product(nd(b).in[1], y1, s2)) return false;
    if (x1 != y1 || x2 != y2 || c1 != c2 || s1 != s2) return false;
    for (int x : {a, b, ab})
      if (dtype_bytes(nd(x).dtype) < dtype_bytes(nd(v).dtype) || (nd(x).dtype != nd(v).dtype && nd(x).dtype != KORCH_F32)) bad("rounding inside a turn");
    const int64_t P = nd(x1).shape[3];
    const int c = inter ? strip(c1) : c1, s = inter ? strip(s1) : s1;
    for (int f : {c, s}) {
      const Shape& fs = nd(f).shape;
      if (fs.size() != 4 || fs[1] != 1 || (fs[0] != 1 && fs[0] != sh[0]) || fs[2] != sh[2] || fs[3] != P) bad("angles of another shape than [images, 1, tokens, pairs]");
    }
    if (inter)
      for (int f : {c1, s1})
        if (nd(f).shape.size() != 5 || nd(f).shape[3] != P || nd(f).shape[4] != 1) bad("angles of another shape than [images, 1, tokens, pairs, 1]");
    if (co < 0) {
      co = c, si = s, pairs = P, interleaved = inter;
    } else if (co != c || si != s || pairs != P || interleaved != inter) {
      bad("tensors turned by different angles");
    }
    const Src one = source(x1), two = source(x2);
    if (!same(one, two, inter ? 1 : P) || one.st[3] != (inter ? 2 : 1)) bad("the pairs of a head lie otherwise than in halves or neighbours");
    if (rest >= 0) {
      const Src r = source(rest);
      if (r.ext != one.ext || r.off != one.off + 2 * P || r.st[3] != 1) bad("what is left of a head is from elsewhere");
      for (int d = 0; d < 3; ++d)
        if (r.st[d] != one.st[d]) bad("what is left of a head is from elsewhere");
    }
    if (sh[3] != 2 * P + (rest >= 0 ? nd(rest).shape[3] : 0)) return false;
    p.turned = true;
    p.x = one;
    p.x.st.resize(3);
    p.heads = sh[1], p.D = sh[3];
    return true;
  }

  void place(int v, int out, int64_t off, const std::vector<int64_t>& st) {
    const Shape& sh = nd(v).shape;
    if (sh.size() != 4) bad("a tensor that is not [images, heads, tokens, dims]");
    Piece p;
    if (turned(v, p)) {
      p.out = out, p.off = off, p.st = {st[0], st[1], st[2]};
      if (st[3] != 1) bad("an output whose heads are not consecutive");
      add(p, sh);
      return;
    }
    if (in(v) && nd(v).dtype == nd(out).dtype && nd(v).op == KORCH_TRANSPOSE && in(nd(v).in[0])) {
      bool layout = true;  // (a transpose of a stored tensor's slices is a source)
      for (int u = nd(v).in[0]; layout && in(u);) {
        layout = nd(u).op == KORCH_SLICE || nd(u).op == KORCH_TRANSPOSE;
        u = nd(u).in[0];
      }
      if (!layout) {
        std::vector<int64_t> t(4);
        for (int d = 0; d < 4; ++d) t[nd(v).attrs.perm[d]] = st[d];
        place(nd(v).in[0], out, off, t);
        return;
      }
    }
    if (in(v) && nd(v).dtype == nd(out).dtype && nd(v).op == KORCH_CONCAT && nd(v).axis != 3) {
      int64_t at = 0;
      for (int u : nd(v).in) {
        place(u, out, off + at * st[nd(v).axis], st);
        at += nd(u).shape[nd(v).axis];
      }
      return;
    }
    // copied; heads are the dim that is not the tokens': whichever order the
    // dims are in, the copy runs over (image, head, token)
    Src s = source(v);
    if (nd(s.ext).dtype != nd(out).dtype || s.st[3] != 1 || st[3] != 1) bad("a copy that changes the type or whose heads are not consecutive");
    p.x = s;
    p.out = out, p.off = off;
    int h = 1, t = 2;
    if (sh[2] != N && sh[1] == N) std::swap(h, t);
    p.x.st = {s.st[0], s.st[h], s.st[t]};
    p.st = {st[0], st[h], st[t]};
    p.heads = sh[h], p.D = sh[3];
    Shape as = {sh[0], sh[h], sh[t], sh[3]};
    add(p, as);
  }

  void add(const Piece& p, const Shape& sh) {
    if (nd(p.x.ext).dtype != nd(p.out).dtype) bad("a turn between types");
    if (sh[0] != B || sh[2] != N) bad("tensors of different images or tokens");
    pieces.push_back(p);
  }

  int eb = 2, VEC = 1, T = 256;
  int64_t TOK = 1, HB = 1, HT = 0, tiles = 1, hblk = 1;

  void analyze() {
    if (!ki.linear.empty() || !ki.reduces.empty()) bad("products or reductions");
    // a first look for images and tokens: the shape of the angles
    for (int v : ki.k.prims) {
      int x, f;
      if (nd(v).shape.size() >= 4 && product(v, x, f)) {
        const Shape& s = nd(x).shape;
        B = s[0], N = s[2];
        break;
      }
    }
    if (!B) bad("nothing is turned");
    for (int o : ki.k.outs) place(o, o, 0, nd(o).shape.size() == 4 ? strides_of(nd(o).shape) : std::vector<int64_t>(4, 0));
    if (co < 0) bad("nothing is turned");
    eb = dtype_bytes(nd(pieces[0].out).dtype);
    VEC = 16 / eb;
    auto fit = [&](int64_t x) {
      while (VEC > 1 && x % VEC) VEC /= 2;
    };
    for (const Piece& p : pieces) {
      if (dtype_bytes(nd(p.out).dtype) != eb) bad("tensors of different types");
      for (int64_t x : {p.x.off, p.off, p.D}) fit(x);
      for (int d = 0; d < 3; ++d) fit(p.x.st[d]), fit(p.st[d]);
      HT += p.heads;
    }
    fit(interleaved ? 2 * pairs : pairs);
    if (B * N >= ((int64_t)1 << 31)) bad("more tokens than the kernel counts");
    // a workgroup's tokens: one (token, pair) to a thread
    TOK = std::max<int64_t>(1, std::min<int64_t>(T / pairs, B * N));
    if (TOK * pairs * 8 > 64 * 1024) bad("more pairs than LDS holds");
    tiles = (B * N + TOK - 1) / TOK;
    // heads are split over workgroups until 1024 run, as long as every thread has a vector
    const int64_t units = std::max<int64_t>(1, pieces[0].D / (2 * VEC));
    HB = HT;
    while (HB > 1 && tiles * ((HT + HB - 1) / HB) < 1024 && TOK * ((HB + 1) / 2) * units >= T) HB = (HB + 1) / 2;
    hblk = (HT + HB - 1) / HB;
    if (tiles * hblk * T >= ((int64_t)1 << 32)) bad("more threads than a launch holds");
  }

  static std::string id(int64_t v) { return std::to_string(v); }

  GenKernel generate(int index) {
    analyze();
    GenKernel gk;
    gk.family = KORCH_FAM_ROTARY;
    gk.name = kernel_name(index, "rotary");
    std::map<int, int> slot;
    ki.assign_args(gk, slot);
    std::ostringstream s;
    s << source_header((int)gk.args.size());
    s << "extern \"C\" __global__ void __launch_bounds__(" << T << ") " << gk.name << "(KArgs a) {\n";
    s << "  __shared__ __attribute__((aligned(16))) float co_[" << TOK * pairs << "], si_[" << TOK * pairs << "];\n";
    s << "  const unsigned tid = threadIdx.x, tile = blockIdx.x / " << hblk << ", h0 = blockIdx.x % " << hblk << " * " << HB << ", h1 = h0 + " << HB << ";\n";
    s << "  const unsigned t0 = tile * " << TOK << ", nt = " << B * N << "u - t0 < " << TOK << "u ? " << B * N << "u - t0 : " << TOK << "u;\n";
    // the angles
    Emitter em(g);
    em.inset = ki.in;
    em.argslot = slot;
    em.vec = 1;
    em.force_gather = true;
    const Shape AS = {B, 1, N, pairs};
    std::vector<Ix> it = {Ix::var("b_"), Ix::k(0), Ix::var("n_"), Ix::var("p_")};
    const std::string c = em.value(co, broadcast_index(nd(co).shape, AS, it)), sn = em.value(si, broadcast_index(nd(si).shape, AS, it));
    s << "  for (unsigned q = tid; q < nt * " << pairs << "; q += " << T << ") {\n    const unsigned tk_ = t0 + q / " << pairs << ";\n    const i64 b_ = tk_ / " << N << "u, n_ = tk_ % " << N
      << "u, p_ = q % " << pairs << ";\n    (void)b_;\n" << em.pre.str() << em.body.str() << "    co_[q] = " << c << ";\n    si_[q] = " << sn << ";\n  }\n  __syncthreads();\n";
    int64_t first = 0;
    for (const Piece& p : pieces) {
      const std::string T1 = ctype(nd(p.out).dtype), V = id(VEC), VT = "vec_t<" + V + ", " + T1 + ">";
      const std::string X = "((const " + T1 + "*)a.p[" + id(slot.at(p.x.ext)) + "])", Y = "((" + T1 + "*)a.p[" + id(ki.out_slot(p.out)) + "])";
      const bool halves = p.turned && !interleaved;
      // vectors of a head: pairs of vectors (halves) or vectors of neighbours, then what is copied
      const int64_t nturn = !p.turned ? 0 : interleaved ? 2 * pairs / VEC : pairs / VEC;
      const int64_t units = nturn + (p.turned ? (p.D - 2 * pairs) / VEC : p.D / VEC);
      const int U = units * TOK * HB >= 4 * T ? 4 : units * TOK * HB >= 2 * T ? 2 : 1;
      s << "  {\n    const unsigned lo = h0 > " << first << "u ? h0 - " << first << "u : 0u, hi_ = h1 > " << first << "u ? h1 - " << first << "u : 0u, hi = hi_ < " << p.heads << "u ? hi_ : "
        << p.heads << "u;\n    const unsigned count = hi > lo ? (hi - lo) * " << TOK * units << "u : 0u;\n";
      s << "    for (unsigned q0 = tid; q0 < count; q0 += " << U * T << ") {\n      " << VT << " x[" << U << "]" << (halves ? ", y[" + id(U) + "]" : std::string()) << ";\n";
      const std::string where = "        const unsigned q_ = q0 + u * " + id(T) + ", q = q_ < count ? q_ : count - 1, k = q % " + id(units) + "u, r = q / " + id(units) +
                                "u, tk_ = r % " + id(TOK) + "u, tk = tk_ < nt ? tk_ : nt - 1, hd = lo + r / " + id(TOK) + "u;\n        const unsigned at_ = t0 + tk;\n        const i64 b = at_ / " + id(N) + "u, n = at_ % " + id(N) + "u;\n";
      auto offset = [&](int64_t off, const std::vector<int64_t>& st) {
        return "b * " + id(st[0]) + "LL + (i64)hd * " + id(st[1]) + "LL + n * " + id(st[2]) + "LL + " + id(off) + "LL";
      };
      // element of vector k in its head (halves: the first half's vector, then the copied ones)
      const std::string el = halves && p.D > 2 * pairs ? "(k < " + id(nturn) + "u ? k * " + V + "u : k * " + V + "u + " + id(pairs) + "u)" : "k * " + V + "u";
      s << "#pragma unroll\n      for (int u = 0; u < " << U << "; ++u) {\n" << where << "        const " << T1 << "* s = " << X << " + (" << offset(p.x.off, p.x.st) << ") + " << el << ";\n        x[u] = *(const "
        << VT << "*)s;\n";
      if (halves) s << "        y[u] = *(const " << VT << "*)(s + " << (p.D > 2 * pairs ? "(k < " + id(nturn) + "u ? " + id(pairs) + " : 0)" : id(pairs)) << ");\n";
      s << "      }\n#pragma unroll\n      for (int u = 0; u < " << U << "; ++u) {\n" << where << "        if (q_ >= count || tk_ >= nt) continue;\n        const i64 o = " << offset(p.off, p.st) << " + " << el << ";\n";
      const std::string e = VEC > 1 ? "[e]" : "";
      auto copy = [&]() { s << "          float f[" << V << "];\n#pragma unroll\n          for (int e = 0; e < " << V << "; ++e) f[e] = tof(x[u]" << e << ");\n          " << out_store(g, p.out, Y, "o", VEC, "f") << ";\n"; };
      if (!p.turned) {
        s << "        {\n";
        copy();
        s << "        }\n";
      } else {
        const bool rest = units > nturn;
        if (rest) s << "        if (k >= " << nturn << "u) {\n", copy(), s << "          continue;\n        }\n";
        if (halves) {
          s << "        const float* cp = co_ + tk * " << pairs << " + k * " << V << ";\n        const float* sp = si_ + tk * " << pairs << " + k * " << V << ";\n        float f[" << V << "], h[" << V
            << "];\n#pragma unroll\n        for (int e = 0; e < " << V << "; ++e) {\n          const float c = cp[e], sn = " << (p.back ? "-sp[e]" : "sp[e]") << ", x1 = tof(x[u]" << e << "), x2 = tof(y[u]" << e
            << ");\n          f[e] = x1 * c - x2 * sn;\n          h[e] = x2 * c + x1 * sn;\n        }\n        " << out_store(g, p.out, Y, "o", VEC, "f") << ";\n        "
            << out_store(g, p.out, Y, "o + " + id(pairs), VEC, "h") << ";\n";
        } else {
          const std::string pv = id(VEC / 2);
          s << "        const float* cp = co_ + tk * " << pairs << " + k * " << pv << ";\n        const float* sp = si_ + tk * " << pairs << " + k * " << pv << ";\n        float f[" << V
            << "];\n#pragma unroll\n        for (int e = 0; e < " << pv << "; ++e) {\n          const float c = cp[e], sn = " << (p.back ? "-sp[e]" : "sp[e]")
            << ", x1 = tof(x[u][2 * e]), x2 = tof(x[u][2 * e + 1]);\n          f[2 * e] = x1 * c - x2 * sn;\n          f[2 * e + 1] = x2 * c + x1 * sn;\n        }\n        "
            << out_store(g, p.out, Y, "o", VEC, "f") << ";\n";
        }
      }
      s << "      }\n    }\n  }\n";
      first += p.heads;
    }
    s << "}\n";
    gk.source = s.str();
    gk.grid[0] = (int)(tiles * hblk);
    gk.block[0] = T;
    ki.fill_cost(gk);
    return gk;
  }
};

}  // namespace

bool match_rotary(const KInfo& ki, std::string* why) {
  try {
    RotaryGen r(ki);
    r.analyze();
    if (r.interleaved && r.VEC < 2) RotaryGen::bad("pairs of neighbours that no vector holds");
  } catch (Error& e) {
    *why = e.what();
    return false;
  }
  return true;
}

GenKernel gen_rotary(const KInfo& ki, int index) { return RotaryGen(ki).generate(index); }

}  // namespace korch
