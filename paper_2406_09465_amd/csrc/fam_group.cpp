// Group norm, channels last, and its gradient: kernels over a map
// [B, P, G, K] (images, positions, groups, channels of a group; C = G K
// channels are consecutive) whose nodes are
//   * full: elementwise primitives on the map;
//   * per channel, group or image: elementwise primitives on what does not
//     vary along P ([B, 1, G, K], [B, 1, G, 1], [G, K] ..);
//   * sums or means over P (full -> [B, 1, G, K]), over a group's channels
//     ([B, 1, G, K] -> [B, 1, G, 1]) and over the images ([B, 1, G, K] -> [1, 1, G, K]);
//   * reshapes that rename such tensors.
//
// 10 to 30 operations per element: what applies statistics to a large map is
// bound by HBM, what sums by HBM, the vector units (busy 64 to 73 % of the time
// at 8x64x64x320 bf16 with silu) and the hand-over together, a small map by its
// launch and its exchanges.  A thread keeps one vector of channels for every row
// it visits, so what belongs to a channel or its group is loaded and computed
// once per thread, and consecutive threads read consecutive memory.  Kinds of kernels:
//   * slab: a workgroup owns whole groups of one image, whose rows stay in its
//     registers in their own type: every pass over the positions (mean, then
//     variance, then the result) after the first reads registers, and the map
//     is read once.  One launch;
//   * sums: one pass over the positions, split over workgroups; the last
//     workgroup of an image adds the partial sums in order and computes what
//     follows from them;
//   * moments: means and variances of groups in one pass (per thread, rows in
//     batches of up to eight whose mean and centred squares merge into the running
//     ones; then mean and M2 of threads and of workgroups merge likewise), so
//     a mean far from zero costs the variance no bits;
//   * apply: no sum over positions; rows are spread over the chip.
// Every sum is fp32 in a fixed order (no floating-point atomics).
#include <algorithm>
#include <cmath>

#include "families.h"

namespace korch {

namespace {

int64_t pow2floor(int64_t x) {
  int64_t p = 1;
  while (2 * p <= x) p *= 2;
  return p;
}

constexpr int64_t kHandOver = 16;    // partial results that one workgroup adds where there are two levels
constexpr int64_t kOneLevel = 64;    // and at most with one
constexpr int64_t kLds = 160 * 1024; // of a workgroup

struct GroupGen {
  const KInfo& ki;
  const Graph& g;
  int64_t B = 0, P = 0, G = 0, K = 0, C = 0;
  Shape full;
  enum Kind { Slab, Sums, Moments, Apply } kind = Apply;
  std::map<int, int> root;           // reshape -> the node it renames
  std::map<int, bool> is_full;       // nodes of the kernel (not reshapes)
  std::map<int, int> gen;            // passes over the positions that a node needs
  std::vector<int> r1, r3, r0;       // reductions over positions, a group's channels, images
  std::vector<int> xfull;            // external maps
  std::vector<int> full_outs, inv_outs;
  int npass = 0;
  int eb = 2;
  // moments: the node of the mean, of the variance and the map
  int mo_mu = -1, mo_var = -1, mo_x = -1;
  std::set<int> mo_nodes;
  // geometry
  int VEC = 1, T = 256, NJ = 1, LY = 1, NR = 1;
  int U = 1;                         // rows that a thread loads together
  int64_t CT = 0, CVT = 0, tiles = 1, S = 1, chunk = 0;

  GroupGen(const KInfo& k) : ki(k), g(k.g) {}

  [[noreturn]] static void bad(const std::string& m) { fail(KORCH_E_UNSUPPORTED, "group: " + m); }
  const Node& nd(int v) const { return g.nodes[v]; }
  bool in(int v) const { return ki.in.count(v) > 0; }
  int rt(int v) const {
    auto f = root.find(v);
    return f == root.end() ? v : f->second;
  }

  // Dims of a shape against the map's, right-aligned; false when it does not broadcast to it.
  bool aligned(const Shape& s, Shape& d) const {
    if (s.size() > 4) return false;
    d.assign(4 - s.size(), 1);
    d.insert(d.end(), s.begin(), s.end());
    for (int i = 0; i < 4; ++i)
      if (d[i] != 1 && d[i] != full[i]) return false;
    return true;
  }

  void find_shape() {
    for (int v : ki.reduces) {
      const Shape& s = nd(nd(v).in[0]).shape;
      if (nd(v).axis != 1 || s.size() != 4) continue;
      if (!full.empty() && full != s) bad("sums over the positions of different maps");
      full = s;
    }
    if (full.empty()) {
      // no sum over positions: the map whose statistics [B, 1, G, 1] are read
      int elementwise = 0;
      for (int v : ki.k.prims) {
        if (!is_elementwise(nd(v).op)) continue;
        ++elementwise;
        const Shape& s = nd(v).shape;
        if (s.size() != 4 || (!full.empty() && numel(s) <= numel(full))) continue;
        full = s;
      }
      if (full.empty() || elementwise < 2) bad("no map");
      bool stat = false;
      for (int u : ki.ext) stat = stat || (full[1] * full[3] > 1 && nd(u).shape == Shape{full[0], 1, full[2], 1});
      if (!stat) bad("no statistics of groups are read");
    }
    B = full[0], P = full[1], G = full[2], K = full[3], C = G * K;
    if (P >= ((int64_t)1 << 30) || C >= ((int64_t)1 << 20)) bad("more positions or channels than the kernels count");
  }

  void classify() {
    std::set<int> outs(ki.k.outs.begin(), ki.k.outs.end());
    for (int u : ki.ext) {
      Shape d;
      if (!aligned(nd(u).shape, d)) bad("an operand does not broadcast to the map");
      if ((d[1] > 1 || P == 1) && nd(u).shape == full) {
        // (with one position, a tensor that only sums over images read is theirs)
        bool map = P > 1;
        for (int c : g.consumers[u])
          if (in(c) && !(op_kind(nd(c).op) == korch::Kind::Reduce && nd(c).axis == 0)) map = true;
        if (map) {
          xfull.push_back(u);
          eb = std::max(eb, dtype_bytes(nd(u).dtype));
        }
      } else if (d[1] > 1) {
        bad("an operand varies along the positions but is no map");
      }
    }
    auto full_of = [&](int u) {
      if (!in(u)) return std::find(xfull.begin(), xfull.end(), u) != xfull.end();
      return (bool)is_full.at(rt(u));
    };
    auto gen_of = [&](int u) { return in(u) ? gen.at(rt(u)) : 0; };
    for (int v : ki.k.prims) {
      const Node& n = nd(v);
      if (n.op == KORCH_RESHAPE) {
        if (!in(n.in[0])) bad("a view of a stored tensor needs no kernel");
        root[v] = rt(n.in[0]);
        // an operand keeps the layout of what it renames
        bool read = false;
        for (int c : g.consumers[v]) read = read || (in(c) && nd(c).op != KORCH_RESHAPE);
        if (read && n.shape != nd(root[v]).shape) bad("a reshaped operand");
        if (dtype_bytes(n.dtype) < dtype_bytes(nd(root[v]).dtype) && !outs.count(v)) bad("a reshape that rounds");
        continue;
      }
      Shape d;
      if (op_kind(n.op) == korch::Kind::Reduce) {
        if (n.op == KORCH_REDUCE_MAX || !n.attrs.keepdim || nd(n.in[0]).shape.size() != 4) bad("a reduction that is no sum or mean of the map with its axes kept");
        const int u = n.in[0];
        is_full[v] = false;
        if (n.axis == 1) {
          if (!full_of(u)) bad("a sum over positions of something that has none");
          r1.push_back(v);
          gen[v] = gen_of(u) + 1;
          npass = std::max(npass, gen[v]);
        } else if (n.axis == 3) {
          if (full_of(u) || nd(u).shape != Shape{B, 1, G, K}) bad("a sum over a group's channels of something else than sums over positions");
          if (gen_of(u) == 0) bad("a sum over a group's channels of stored values");
          r3.push_back(v);
          gen[v] = gen_of(u);
        } else if (n.axis == 0) {
          if (nd(u).shape != Shape{B, 1, G, K} || full_of(u)) bad("a sum over images of something else than per-channel values");
          for (int c : g.consumers[v])
            if (in(c) && nd(c).op != KORCH_RESHAPE) bad("a sum over images is read in the kernel");
          r0.push_back(v);
          gen[v] = gen_of(u);
        } else {
          bad("a sum over groups");
        }
        continue;
      }
      if (!is_elementwise(n.op)) bad(std::string("unsupported primitive ") + op_name(n.op));
      if (!aligned(n.shape, d)) bad("a node does not broadcast to the map");
      bool f = false;
      int gn = 0;
      for (int u : n.in) {
        if (in(u) && std::find(r0.begin(), r0.end(), rt(u)) != r0.end()) bad("a sum over images is read in the kernel");
        f = f || full_of(u), gn = std::max(gn, gen_of(u));
      }
      if (f && n.shape != full) bad("a node of the map in another shape");
      if (!f && d[1] > 1) bad("a node varies along the positions without a map");
      is_full[v] = f;
      gen[v] = gn;
    }
    for (int o : ki.k.outs) {
      const int v = rt(o);
      if (std::find(r0.begin(), r0.end(), v) != r0.end()) continue;
      if (is_full.at(v)) {
        full_outs.push_back(o);
        eb = std::max(eb, dtype_bytes(nd(o).dtype));
      } else {
        // one value per channel or per group of an image
        const Shape& s = nd(v).shape;
        if (s != Shape{B, 1, G, K} && s != Shape{B, 1, G, 1}) bad("an output that is neither a map nor per channel or group");
        inv_outs.push_back(o);
      }
    }
    for (int v : r0) {
      bool out = false;
      for (int o : ki.k.outs) out = out || rt(o) == v;
      if (!out) bad("a sum over images that is not an output");
    }
    for (int v : r1) {
      if (nd(v).shape != Shape{B, 1, G, K}) bad("sum over positions");
      for (int w : r1)
        if (gen[w] == gen[v] && nd(w).op != nd(v).op) bad("sums and means of one pass");
    }
  }

  // mean over the positions (and the group), then the mean of the centred squares
  bool find_moments() {
    if (r1.size() != 2 || npass != 2 || xfull.size() != 1 || !full_outs.empty() || !r0.empty()) return false;
    mo_x = xfull[0];
    auto group = [&](int v) -> int {
      if (K == 1) return v;
      for (int r : r3)
        if (nd(r).in[0] == v && nd(r).op == KORCH_REDUCE_MEAN) return r;
      return -1;
    };
    const int a = r1[0], b = r1[1];
    if (nd(a).op != KORCH_REDUCE_MEAN || nd(b).op != KORCH_REDUCE_MEAN || nd(a).in[0] != mo_x) return false;
    mo_mu = group(a), mo_var = group(b);
    if (mo_mu < 0 || mo_var < 0 || (K > 1 && r3.size() != 2)) return false;
    const int q = nd(b).in[0];
    if (!in(q) || !(nd(q).op == KORCH_SQUARE || (nd(q).op == KORCH_MUL && !nd(q).attrs.has_scalar && nd(q).in[0] == nd(q).in[1]))) return false;
    const int d = nd(q).in[0];
    if (!in(d) || nd(d).op != KORCH_SUB || nd(d).attrs.has_scalar || nd(d).in[0] != mo_x || nd(d).in[1] != mo_mu) return false;
    mo_nodes = {a, b, mo_mu, mo_var, q, d};
    for (int v : mo_nodes) {
      if (v == mo_mu || v == mo_var) continue;
      for (int c : g.consumers[v])
        if (in(c) && !mo_nodes.count(c)) return false;
      for (int o : ki.k.outs)
        if (rt(o) == v) return false;
    }
    return true;
  }

  // Threads over a tile of CT channels.
  void lanes(int threads) {
    T = threads;
    CVT = CT / VEC;
    NJ = (int)((CVT + T - 1) / T);
    LY = NJ == 1 ? (int)(T / CVT) : 1;
  }

  // Workgroups of 1024 threads have 128 registers for each, half of what smaller
  // ones have: fewer rows and partial results in flight, loops as they are written
  // (spilling, the statistics of 1x64x64x5120 f32 took 48.7 us instead of 20.0, the
  // gradient's sums of 1x64x65x7680 f32 72.3 instead of 69.5).
  bool few_registers() const { return T > 512; }
  std::string as_written() const { return few_registers() ? "#pragma unroll 1\n" : ""; }
  // Rows of the maps in `words` registers.
  int64_t rows_in(int64_t words) const { return std::max<int64_t>(1, words / (NJ * std::max(1, VEC * eb / 4) * std::max<int64_t>(1, xfull.size()))); }

  // Whether `nr` rows of `words` maps stay in a thread's registers beside the
  // fp32 values of a row and the channels' own (256 registers; 1024 threads have 128 each).
  bool slab_fits(int threads, int64_t nr, int vec, int words) const {
    const int64_t raw = nr * std::max(1, vec * eb / 4) * words, own = (int64_t)vec * (words > 1 ? 8 : 5);
    if (threads < 256) return nr == 1;  // (maps of a few positions: no more threads than vectors)
    return threads <= 256 ? raw <= 24 && nr <= 24 : threads == 512 ? raw <= 48 && nr <= 48 : raw + own <= 64 && nr <= 24;
  }

  // A slab of whole groups in a workgroup's registers: the fewest groups whose
  // channels make runs of 64 bytes, so that half of each line a load touches is
  // used; where all groups of all images are 64 at most, of 16 bytes (few
  // workgroups wait for few loads: 1x16x16x320 f16 with runs of 20 bytes 4.2 us, of
  // 80 bytes 6.6).  Where those do not fit, the most groups that do.
  bool slab_geometry() {
    if (P > 65536 || xfull.empty()) return false;
    const int words = std::max<int>(1, (int)xfull.size());
    bool found = false;
    int64_t best = 0;
    for (int64_t gt = 1; gt <= G; ++gt) {
      if (G % gt) continue;
      int vec = 16 / eb;
      while ((gt * K) % vec) vec /= 2;
      const int64_t ct = gt * K;
      bool fits = false;
      for (int t : {64, 128, 256, 512, 1024}) {
        if (ct / vec > t) continue;
        const int64_t ly = t / (ct / vec), nr = (P + ly - 1) / ly;
        if (slab_fits(t, nr, vec, words)) {
          fits = true;
          break;
        }
      }
      if (!fits) continue;
      found = true;
      best = gt;
      if (ct * eb >= (B * G <= 64 ? 16 : 64)) break;
    }
    if (!found) return false;
    // Past about a thousand cache lines of a map (64 bytes; runs that are no whole
    // part of a line touch one more), one compute unit's loads take longer than a second launch: forward
    // 2x32x32x512 f16 (1024 lines) 6.2 us, 10.0 in two kernels; 1x64x64x128 f16 (4096) 12.2 and 9.6;
    // 8x32x32x640 bf16 (runs of 80 bytes, 2304) 12.9 and 11.8.
    const int64_t run = best * K * eb;
    if ((double)P * (run % 64 == 0 ? run / 64.0 : 64 % run == 0 ? 1.0 : run / 64.0 + 1.0) > 1024.0) return false;
    CT = best * K;
    tiles = G / best;
    VEC = 16 / eb;
    while (CT % VEC) VEC /= 2;
    for (int t : {64, 128, 256, 512, 1024}) {
      if (CT / VEC > t) continue;
      lanes(t);
      NR = (int)((P + LY - 1) / LY);
      if (slab_fits(t, NR, VEC, words)) break;
    }
    U = NR;
    if (!r0.empty()) {
      // the sums over images are handed over
      const int64_t lines = B <= kOneLevel ? 1 : (B + kHandOver - 1) / kHandOver + 1;  // counters of a tile (allocation-free execution has 64 KiB of them)
      if (B > kHandOver * 32 || tiles * lines > 256 || B * tiles * ((int64_t)r0.size() * ((CT + 3) / 4 * 4)) * 4 * 17 / 16 > ((int64_t)16 << 20)) return false;
    }
    kind = Slab;
    return lds().bytes() <= kLds && B * tiles * T < ((int64_t)1 << 32);
  }

  void stream_geometry(int threads, int64_t channels) {
    CT = channels;
    tiles = C / CT;
    VEC = 16 / eb;
    while (CT % VEC) VEC /= 2;
    while (threads < 1024 && CT / VEC > threads) threads *= 2;
    while (threads > 64 && threads / 2 >= P * (CT / VEC)) threads /= 2;  // (maps of a few positions)
    lanes(threads);
    if ((int64_t)NJ * VEC > 16 || CT > 8192) bad("more channels than a workgroup keeps");
  }

  void analyze() {
    if (!ki.linear.empty()) bad("has linear primitives");
    for (int v : ki.k.prims)
      if (nd(v).op == KORCH_BIN_SUM || nd(v).op == KORCH_FILL || nd(v).op == KORCH_IOTA) bad("constants or bins");
    find_shape();
    classify();
    for (int v : r0)
      if (npass == 0 ? in(nd(v).in[0]) : !in(nd(v).in[0])) bad("a sum over images beside other sums");
    if (npass == 0 && !inv_outs.empty()) bad("an output per channel without a sum");
    if (npass == 0 && full_outs.empty()) bad("no map among the outputs");
    for (int v : r0)
      if (npass > 0 && std::find(r1.begin(), r1.end(), nd(v).in[0]) == r1.end()) bad("a sum over images of computed values");
    if (npass == 0) {
      kind = Apply;
      stream_geometry(256, C);
      // about eight workgroups to a compute unit, sixteen for maps from 64 MiB on, whose
      // last workgroups would end apart (the gradient's of 8x128x128x256 bf16, 134 MB:
      // 30.1 us, 32.3 with eight; of 4x416x416x64 f16, 89 MB: 41.2, 43.0; of 8x64x64x320,
      // 21 MB: 11.6, 11.3); a thread's rows in whole batches, so that the channels'
      // values are loaded for several rows
      const int64_t want = std::max<int64_t>(1, ((double)B * P * C * eb >= 67108864.0 ? 4096 : 2048) / B);
      chunk = std::max<int64_t>((P + want - 1) / want, 1);
      U = (int)std::min<int64_t>({4, (chunk + LY - 1) / LY, few_registers() ? rows_in(16) : 4});
      chunk = (chunk + (int64_t)LY * U - 1) / ((int64_t)LY * U) * ((int64_t)LY * U);
      S = (P + chunk - 1) / chunk;
      if (B * S * T + (((int64_t)C + 16) * 4 * T) >= ((int64_t)1 << 32) || S >= ((int64_t)1 << 31)) bad("more threads than a launch holds");
      return;
    }
    if (slab_geometry()) return;
    if (!full_outs.empty() || !r0.empty()) bad("a map and sums over it that do not fit the registers of a workgroup");
    if (find_moments())
      kind = Moments;
    else if (npass == 1)
      kind = Sums;
    else
      bad("sums that depend on sums over the same positions");
    // The sums of few wide maps are split into tiles of whole groups (runs of two
    // cache lines or more) as well: a tile's partial sums are a fraction of the channels', and
    // the tiles' last workgroups add theirs side by side.  It pays past 128 KiB of
    // partial sums per image (1x64x64x320 bf16, the gradient's sums: 9.1 us, 10.4 without;
    // 4x32x32x320, 107 KiB: 8.7 and 7.6).
    stream_geometry(512, C);
    int64_t tile = C;
    if (kind == Sums && (double)B * P * C * eb * xfull.size() <= 16777216.0 &&
        std::min<int64_t>(kOneLevel, P / ((int64_t)LY * 2)) * (int64_t)r1.size() * C * 4 > 131072)
      for (int64_t gt = G; gt >= 1; --gt)
        if (G % gt == 0 && gt * K * eb >= 128 && B * (G / gt) <= 32) tile = gt * K;
    stream_geometry(512, tile);
    // A workgroup of eight waves to a compute unit, each thread with a batch of
    // rows at least; batches of few rows, as a workgroup of few rows runs its code
    // once and waits for its instructions (batches of 8 and 4, one set loading
    // while the other is summed: 13.9 us instead of 11.0 for the gradient's sums of
    // 8x32x32x640 bf16, 41.6 instead of 34.7 at 4x416x416x64 f16).
    U = kind == Moments ? P * B >= (int64_t)256 * LY * 32 ? 8 : 4 : 2;
    S = std::max<int64_t>(1, std::min<int64_t>((256 + B * tiles - 1) / (B * tiles), P / ((int64_t)LY * U * (tiles > 1 ? 2 : 1))));
    // one level of hand-over as long as a thread's rows stay few
    if (S > kOneLevel && P <= kOneLevel * LY * 16) S = kOneLevel;
    chunk = (P + S - 1) / S;
    chunk = (chunk + LY - 1) / LY * LY;
    S = (P + chunk - 1) / chunk;
    // few rows: in as few batches as hold them evenly, one where it can be
    const int64_t rows = chunk / LY, most = kind == Moments ? 8 : 4;
    // (as far as they fit registers beside the sums, and the sums' operands)
    const int64_t room = rows_in(few_registers() && kind == Sums ? 16 : 32);
    U = (int)std::min<int64_t>(U, room);
    if (rows <= 2 * most && most <= room) U = (int)((rows + (rows + most - 1) / most - 1) / ((rows + most - 1) / most));
    if (B * tiles * S * T >= ((int64_t)1 << 32)) bad("more threads than a launch holds");
    if (lds().bytes() > kLds) bad("sums of more channels than LDS holds");
  }

  // ---- code ------------------------------------------------------------------

  GenKernel gk;
  std::map<int, int> slot;
  std::ostringstream s;
  std::set<int> inv_done;      // per-channel nodes and operands already in registers

  std::string ptr(int u) const { return "((const " + ctype(nd(u).dtype) + "*)a.p[" + std::to_string(slot.at(u)) + "])"; }
  std::string outp(int o) const { return "((" + ctype(nd(o).dtype) + "*)a.p[" + std::to_string(ki.out_slot(o)) + "])"; }
  static std::string id(int v) { return std::to_string(v); }
  std::string jdecl(const std::string& name) const {
    return "  float " + name + "[" + std::to_string(NJ) + "][" + std::to_string(VEC) + "];\n";
  }
  // `stmt` for every channel of the thread: j (vector), e (element), ch(j) + e the channel
  std::string each(const std::string& stmt) const {
    return "#pragma unroll\n  for (int j = 0; j < " + std::to_string(NJ) + "; ++j)\n#pragma unroll\n    for (int e = 0; e < " + std::to_string(VEC) + "; ++e) { " +
           stmt + " }\n";
  }

  std::string elem_expr(int v, const std::function<std::string(int)>& operand) const {
    const Node& n = nd(v);
    switch (op_kind(n.op)) {
      case korch::Kind::Unary: return unary_expr(n.op, operand(n.in[0]));
      case korch::Kind::Binary: return binary_expr(n.op, operand(n.in[0]), n.attrs.has_scalar ? flit(n.attrs.scalar) : operand(n.in[1]));
      default:
        return "(" + operand(n.in[0]) + " != 0.0f ? " + operand(n.in[1]) + " : " + (n.attrs.has_scalar ? flit(n.attrs.scalar) : operand(n.in[2])) + ")";
    }
  }

  // A per-channel value (the thread's channels in registers); emits it and what it needs.
  std::string inv(int v) {
    if (in(v)) v = rt(v);
    const std::string name = "n" + id(v);
    if (inv_done.count(v)) return name + "[j][e]";
    if (!in(v)) {
      Shape d;
      aligned(nd(v).shape, d);
      const int64_t sk = d[3] > 1 ? 1 : 0, sg = d[2] > 1 ? d[3] : 0, sb = d[0] > 1 ? d[2] * d[3] : 0;
      s << jdecl(name);
      const bool run = (sk || K == 1) && (sg == K || G == 1);  // consecutive over the channels
      const std::string base = ptr(v) + (sb ? " + (i64)b * " + std::to_string(sb) : "");
      if (run)
        s << "#pragma unroll\n  for (int j = 0; j < " << NJ << "; ++j) ldv<" << VEC << ">(" << name << "[j], " << base << " + c0[j]);\n";
      else if (!sk && !sg)
        s << "  {\n    const float x_ = ld1(" << base << ");\n  " << each(name + "[j][e] = x_;") << "  }\n";
      else
        s << each("const int c_ = c0[j] + e; " + name + "[j][e] = ld1(" + base + " + (c_ / " + std::to_string(K) + ") * " + std::to_string(sg) +
                  (sk ? " + c_ % " + std::to_string(K) : std::string()) + ");");
      inv_done.insert(v);
      return name + "[j][e]";
    }
    if (op_kind(nd(v).op) == korch::Kind::Reduce) bad("internal: a sum that is not there yet");
    const std::string ex = elem_expr(v, [&](int u) { return inv(u); });
    s << jdecl(name) << each(name + "[j][e] = " + ex + ";");
    inv_done.insert(v);
    return name + "[j][e]";
  }

  // Statements for one element of the map; per-channel operands must be in registers.
  struct Body {
    std::ostringstream o;
    std::set<int> done;
  };
  std::string full_value(int v, Body& b) {
    if (in(v)) v = rt(v);
    if (!in(v) && std::find(xfull.begin(), xfull.end(), v) != xfull.end()) {
      if (b.done.insert(v).second) b.o << "        const float f" << id(v) << " = tof(x" << id(v) << "[i][j]" << (VEC > 1 ? "[e]" : "") << ");\n";
      return "f" + id(v);
    }
    if (!in(v) || !is_full.at(v)) return inv(v);
    if (b.done.insert(v).second) {
      const std::string ex = elem_expr(v, [&](int u) { return full_value(u, b); });
      b.o << "        const float f" << id(v) << " = " << ex << ";\n";
    }
    return "f" + id(v);
  }
  // Maps of 16 bits take the hardware's approximations of the exponential and the
  // quotient, also where only their sums are stored, in fp32: those are off by a
  // few 2^-24 (and the exponent's rounding, |Z| 2^-24), the maps' own values by 2^-11 or 2^-8.
  bool fast_full() const { return eb == 2; }

  // Rows in registers in their own type.
  std::string raw_decl() const {
    std::ostringstream o;
    for (int u : xfull) o << "  vec_t<" << VEC << ", " << ctype(nd(u).dtype) << "> x" << id(u) << "[" << U << "][" << NJ << "];\n";
    return o.str();
  }
  // Loads rows row0 + i LY (i < U), clamped to the last row `end` - 1.
  std::string raw_load(const std::string& row0, const std::string& end) const {
    std::ostringstream o;
    o << "#pragma unroll\n    for (int i = 0; i < " << U << "; ++i) {\n      const int r_ = " << row0 << " + i * " << LY << ", row = r_ < " << end << " ? r_ : "
      << end << " - 1;\n";
    // within an image of less than 2 GiB, a 32-bit offset from a base that is the same for all lanes
    const bool narrow = (double)P * C * 4 < 2147483648.0;
    o << "      const " << (narrow ? "unsigned" : "i64") << " at = " << (narrow ? "(unsigned)" : "(i64)") << "row * " << C << ";\n";
    for (int u : xfull)
      o << "#pragma unroll\n      for (int j = 0; j < " << NJ << "; ++j) x" << id(u) << "[i][j] = *(const vec_t<" << VEC << ", " << ctype(nd(u).dtype) << ">*)(" << ptr(u)
        << " + (i64)b * " << P * C << "LL + (at + c0[j]));\n";
    o << "    }\n";
    return o.str();
  }
  // The raw rows pass through an empty statement: a pass converts them anew, and
  // the compiler does not keep the fp32 values of one pass for the next one
  // (which took twice the registers, and spilled).
  std::string raw_again() const {
    const int words = VEC * 2 / 4;  // (of 16-bit rows; fp32 rows need no conversion)
    std::ostringstream o;
    for (int u : xfull)
      if (dtype_bytes(nd(u).dtype) == 2 && words >= 1) {
        const std::string w = words == 1 ? "unsigned" : "u32_" + std::to_string(words);
        o << "  {\n";
        if (words > 1) o << "    typedef unsigned " << w << " __attribute__((ext_vector_type(" << words << ")));\n";
        o << "#pragma unroll\n    for (int i = 0; i < " << U << "; ++i)\n#pragma unroll\n      for (int j = 0; j < " << NJ << "; ++j) {\n        " << w << " w_ = __builtin_bit_cast(" << w
          << ", x" << id(u) << "[i][j]);\n        asm volatile(\"\" : \"+v\"(w_));\n        x" << id(u) << "[i][j] = __builtin_bit_cast(vec_t<" << VEC << ", " << ctype(nd(u).dtype)
          << ">, w_);\n      }\n  }\n";
      }
    return o.str();
  }
  // The loop over the rows in registers.
  std::string row_loop(const std::string& row0, const std::string& end, const std::string& elem, const std::string& after_j) const {
    std::ostringstream o;
    o << "#pragma unroll\n    for (int i = 0; i < " << U << "; ++i) {\n      const int row = " << row0 << " + i * " << LY << ";\n      const bool live = row < " << end
      << ";\n#pragma unroll\n      for (int j = 0; j < " << NJ << "; ++j) {\n";
    for (int v : full_outs) o << "        float o" << id(v) << "[" << VEC << "];\n";
    o << "#pragma unroll\n        for (int e = 0; e < " << VEC << "; ++e) {\n" << elem << "        }\n" << after_j << "      }\n    }\n";
    return o.str();
  }
  // Maps past half of the 256 MiB that the device's last cache holds go by it:
  // their reader would not find them there, and what the next kernel reads again
  // stays (32x128x128x256 bf16 trained 366 us, 405 through the cache; 8x64x64x320 44.5 and 43.9).
  bool stream_out() const {
    double bytes = 0;
    for (int v : full_outs) bytes += (double)numel(nd(v).shape) * dtype_bytes(nd(v).dtype);
    return bytes >= 134217728.0;
  }
  std::string store_rows() const {
    std::ostringstream o;
    for (int v : full_outs) {
      const std::string at = "((i64)b * " + std::to_string(P) + " + row) * " + std::to_string(C) + " + c0[j]";
      o << "        if (live && act" << (NJ > 1 ? "[j]" : "") << ") "
        << (stream_out() ? "st_stream<" + std::to_string(VEC) + ">(" + outp(v) + " + " + at + ", o" + id(v) + ")" : out_store(g, v, outp(v), at, VEC, "o" + id(v))) << ";\n";
    }
    return o.str();
  }

  // Per-channel sums of the threads' values acc (nodes `vs`), into chan[i][CT4].
  int64_t CT4() const { return (CT + 3) / 4 * 4; }
  void channel_sums(const std::vector<std::string>& acc) {
    const int n = (int)acc.size();
    const std::string A = NJ > 1 ? "act[j]" : "act";
    if (LY == 1) {
      for (int i = 0; i < n; ++i) s << each("if (" + A + ") chan[" + std::to_string(i * CT4()) + " + c0[j] - ct0 + e] = " + acc[i] + "[j][e];");
      s << "  __syncthreads();\n";
      return;
    }
    const int64_t slab = (int64_t)LY * CT;
    // (whole vectors: element by element, lanes VEC floats apart would share LDS banks)
    for (int i = 0; i < n; ++i) {
      if (VEC >= 4)
        s << "  if (act) {\n#pragma unroll\n    for (int e = 0; e < " << VEC << "; e += 4) *(f32x4*)(red + " << i * slab << " + ly * " << CT << " + c0[0] - ct0 + e) = f32x4{" << acc[i] << "[0][e], "
          << acc[i] << "[0][e + 1], " << acc[i] << "[0][e + 2], " << acc[i] << "[0][e + 3]};\n  }\n";
      else
        s << each("if (act) red[" + std::to_string(i * slab) + " + ly * " + std::to_string(CT) + " + c0[j] - ct0 + e] = " + acc[i] + "[j][e];");
    }
    s << "  __syncthreads();\n";
    int64_t L = 1;
    if (CT < T) L = std::min<int64_t>(std::min<int64_t>(16, pow2floor(T / CT)), pow2floor(LY));
    if (L > 1) {
      // a thread per channel and slice of the rows of lanes; then the slices
      s << "  if (tid < " << L * CT << ") {\n    const int c = tid % " << CT << ", l = tid / " << CT << ";\n";
      for (int i = 0; i < n; ++i)
        s << "    float t" << i << "_ = 0.0f;\n";
      s << "#pragma unroll 8\n    for (int y = l; y < " << LY << "; y += " << L << ") {\n";
      for (int i = 0; i < n; ++i) s << "      t" << i << "_ += red[" << i * slab << " + y * " << CT << " + c];\n";
      s << "    }\n";
      for (int i = 0; i < n; ++i) s << "    part[" << i * L * CT << " + tid] = t" << i << "_;\n";
      s << "  }\n  __syncthreads();\n  if (tid < " << CT << ") {\n";
      for (int i = 0; i < n; ++i) {
        s << "    float t" << i << "_ = part[" << i * L * CT << " + tid];\n#pragma unroll\n    for (int l = 1; l < " << L << "; ++l) t" << i << "_ += part[" << i * L * CT
          << " + l * " << CT << " + tid];\n    chan[" << i * CT4() << " + tid] = t" << i << "_;\n";
      }
      s << "  }\n  __syncthreads();\n";
      return;
    }
    s << "  for (int c = tid; c < " << CT << "; c += " << T << ") {\n";
    for (int i = 0; i < n; ++i) s << "    float t" << i << "_ = 0.0f;\n";
    s << "#pragma unroll 8\n    for (int y = 0; y < " << LY << "; ++y) {\n";
    for (int i = 0; i < n; ++i) s << "      t" << i << "_ += red[" << i * slab << " + y * " << CT << " + c];\n";
    s << "    }\n";
    for (int i = 0; i < n; ++i) s << "    chan[" << i * CT4() << " + c] = t" << i << "_;\n";
    s << "  }\n  __syncthreads();\n";
  }
  // Sums over a group's channels of chan[base ..]: grp[at + g - g0].  (The caller waits for the others.)
  void group_sums(int64_t base, int64_t at = 0) {
    const int64_t gt = CT / K;
    const int64_t L = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(64, pow2floor(K)), pow2floor(std::max<int64_t>(1, T / gt))));
    s << "  for (int q = tid; q < " << (gt * L + T - 1) / T * T << "; q += " << T << ") {\n    const int gr = q / " << L << ", l = q % " << L << ";\n    float t_ = 0.0f;\n";
    s << "    if (gr < " << gt << ")\n#pragma unroll 4\n      for (int k = l; k < " << K << "; k += " << L << ") t_ += chan[" << base << " + gr * " << K << " + k];\n";
    if (L > 1) s << "    t_ = group_sum<" << L << ">(t_);\n";
    s << "    if (l == 0 && gr < " << gt << ") grp[" << at << " + gr] = t_;\n  }\n";
  }
  // Sums over a tile's groups of the threads' values acc, straight into grp[i * groups ..]:
  // a thread adds what of a vector lies in one group, a group's lanes the rest.
  // (The caller waits before and after; by way of the channels' sums it takes
  // twice the barriers.)
  int group_piece() const {
    int sv = VEC;
    while (K % sv) sv /= 2;
    return sv;
  }
  int64_t direct_floats(int n) const { return (int64_t)n * LY * (CT / group_piece()); }
  void group_sums_of(const std::vector<std::string>& acc) {
    const int SV = group_piece();
    const int64_t gt = CT / K, row = CT / SV, KS = K / SV;
    for (size_t i = 0; i < acc.size(); ++i) {
      // (consecutive pieces as vectors: one by one, the lanes' pieces would share LDS banks)
      const int NQ = VEC / SV, W = NQ % 4 == 0 ? 4 : NQ % 2 == 0 ? 2 : 1;
      s << "#pragma unroll\n  for (int j = 0; j < " << NJ << "; ++j)\n    if (" << (NJ > 1 ? "act[j]" : "act") << ") {\n      float t_[" << NQ << "];\n#pragma unroll\n      for (int q = 0; q < " << NQ
        << "; ++q) {\n        t_[q] = " << acc[i] << "[j][q * " << SV << "];\n#pragma unroll\n        for (int e = 1; e < " << SV << "; ++e) t_[q] += " << acc[i] << "[j][q * " << SV
        << " + e];\n      }\n#pragma unroll\n      for (int q = 0; q < " << NQ << "; q += " << W << ") {\n        vec_t<" << W << ", float> w_;\n";
      if (W == 1)
        s << "        w_ = t_[q];\n";
      else
        for (int k = 0; k < W; ++k) s << "        w_[" << k << "] = t_[q + " << k << "];\n";
      s << "        *(vec_t<" << W << ", float>*)(red + " << i * LY * row << " + ly * " << row << " + (c0[j] - ct0) / " << SV << " + q) = w_;\n      }\n    }\n";
    }
    s << "  __syncthreads();\n";
    const int64_t L = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(64, pow2floor(LY * KS)), pow2floor(std::max<int64_t>(1, T / gt))));
    for (size_t i = 0; i < acc.size(); ++i) {
      s << "  for (int q = tid; q < " << (gt * L + T - 1) / T * T << "; q += " << T << ") {\n    const int gr = q / " << L << ", l = q % " << L << ";\n    float t_ = 0.0f;\n    if (gr < " << gt
        << ")\n#pragma unroll 4\n      for (int k = l; k < " << LY * KS << "; k += " << L << ") t_ += red[" << i * LY * row << " + k / " << KS << " * " << row << " + gr * " << KS << " + k % " << KS << "];\n";
      if (L > 1) s << "    t_ = group_sum<" << L << ">(t_);\n";
      s << "    if (l == 0 && gr < " << gt << ") grp[" << i * gt << " + gr] = t_;\n  }\n";
    }
  }
  // Sums of pass `k` that only sums over groups read.
  bool only_groups(const std::vector<int>& sums) const {
    if (K == 1) return false;
    for (int v : sums) {
      for (int c : g.consumers[v])
        if (in(c) && std::find(r3.begin(), r3.end(), c) == r3.end()) return false;
      for (int o : ki.k.outs)
        if (rt(o) == v) return false;
    }
    return true;
  }
  void after_group_pass(const std::vector<int>& sums) {
    s << "  __syncthreads();\n";
    for (size_t i = 0; i < sums.size(); ++i)
      for (int v : r3)
        if (nd(v).in[0] == sums[i]) {
          s << jdecl("n" + id(v)) << each("n" + id(v) + "[j][e] = grp[" + std::to_string(i * (CT / K)) + " + (c0[j] - ct0 + e) / " + std::to_string(K) + "]" +
                                          (nd(v).op == KORCH_REDUCE_MEAN ? " / " + flit((double)K) : std::string()) +
                                          (nd(sums[i]).op == KORCH_REDUCE_MEAN ? " / " + flit((double)P) : std::string()) + ";");
          inv_done.insert(v);
        }
    s << "  __syncthreads();\n";
  }

  // Sums over positions of pass `k` are in chan: they and what follows from
  // them become per-channel values.
  void after_pass(int k, const std::vector<int>& sums) {
    const int64_t gt = CT / K;
    std::vector<int> left, direct;
    for (int v : ki.k.prims)
      if (std::find(r3.begin(), r3.end(), v) != r3.end() && gen.at(v) == k && !inv_done.count(v))
        (std::find(sums.begin(), sums.end(), nd(v).in[0]) != sums.end() ? direct : left).push_back(v);
    auto take = [&](const std::vector<int>& vs, const std::string& scale) {
      s << "  __syncthreads();\n";
      for (size_t i = 0; i < vs.size(); ++i) {
        const int v = vs[i];
        s << jdecl("n" + id(v)) << each("n" + id(v) + "[j][e] = grp[" + std::to_string(i * gt) + " + (c0[j] - ct0 + e) / " + std::to_string(K) + "]" +
                                        (nd(v).op == KORCH_REDUCE_MEAN ? " / " + flit((double)K) : std::string()) + scale + ";");
        inv_done.insert(v);
      }
    };
    // sums over groups of the sums themselves, as they lie
    for (size_t i = 0; i < direct.size(); ++i)
      group_sums((std::find(sums.begin(), sums.end(), nd(direct[i]).in[0]) - sums.begin()) * CT4(), i * gt);
    for (size_t i = 0; i < sums.size(); ++i) {
      const int v = sums[i];
      s << jdecl("n" + id(v)) << each("n" + id(v) + "[j][e] = chan[" + std::to_string(i * CT4()) + " + c0[j] - ct0 + e]" +
                                      (nd(v).op == KORCH_REDUCE_MEAN ? " / " + flit((double)P) : std::string()) + ";");
      inv_done.insert(v);
    }
    if (sums.empty() && left.empty()) return;
    if (!direct.empty()) take(direct, nd(nd(direct[0]).in[0]).op == KORCH_REDUCE_MEAN ? " / " + flit((double)P) : std::string());
    // of values that follow from them, as many together as do not wait for each other
    std::function<bool(int)> ready = [&](int v) {
      if (!in(v)) return true;
      v = rt(v);
      if (inv_done.count(v)) return true;
      if (op_kind(nd(v).op) == korch::Kind::Reduce) return false;
      for (int u : nd(v).in)
        if (!ready(u)) return false;
      return true;
    };
    while (!left.empty()) {
      std::vector<int> now, later;
      for (int v : left) (ready(nd(v).in[0]) ? now : later).push_back(v);
      if (now.empty()) bad("sums over groups that wait for each other");
      std::vector<std::string> x;
      for (int v : now) x.push_back(inv(nd(v).in[0]));
      s << "  __syncthreads();\n";
      for (size_t i = 0; i < now.size(); ++i)
        s << each("if (" + std::string(NJ > 1 ? "act[j]" : "act") + " && ly == 0) chan[" + std::to_string(i * CT4()) + " + c0[j] - ct0 + e] = " + x[i] + ";");
      s << "  __syncthreads();\n";
      for (size_t i = 0; i < now.size(); ++i) group_sums(i * CT4(), i * gt);
      take(now, "");
      left = later;
    }
    s << "  __syncthreads();\n";
  }
  // Per-channel outputs by the first row of lanes, as vectors; per-group outputs by
  // the threads whose vectors begin a group, or, where a vector may begin many, by a
  // thread each, by way of chan.
  void store_inv() {
    const std::string A = NJ > 1 ? "act[j]" : "act";
    std::vector<int> of_group;
    for (int o : inv_outs) {
      const int v = rt(o);
      if (nd(v).shape[3] != K || K == 1) {
        of_group.push_back(o);
        continue;
      }
      const std::string x = inv(v);
      s << "#pragma unroll\n  for (int j = 0; j < " << NJ << "; ++j)\n    if (" << A << " && ly == 0) {\n      float o_[" << VEC << "];\n#pragma unroll\n      for (int e = 0; e < " << VEC
        << "; ++e) o_[e] = " << x << ";\n      " << out_store(g, o, outp(o), "(i64)b * " + std::to_string(C) + " + c0[j]", VEC, "o_") << ";\n    }\n";
    }
    for (int o : of_group) {
      const std::string x = inv(rt(o));
      if (VEC / group_piece() <= 2) {
        const std::string SV = std::to_string(group_piece());
        s << "#pragma unroll\n  for (int j = 0; j < " << NJ << "; ++j)\n#pragma unroll\n    for (int e = 0; e < " << VEC << "; e += " << SV << ")\n      if (" << A << " && ly == 0 && (c0[j] + e) % " << K
          << " == 0) " << out_store(g, o, outp(o), "(i64)b * " + std::to_string(G) + " + (c0[j] + e) / " + std::to_string(K), 0, x) << ";\n";
        continue;
      }
      s << "  __syncthreads();\n" << each("if (" + A + " && ly == 0) chan[c0[j] - ct0 + e] = " + x + ";") << "  __syncthreads();\n  for (int q = tid; q < " << CT / K << "; q += " << T << ") "
        << out_store(g, o, outp(o), "(i64)b * " + std::to_string(G) + " + ct0 / " + std::to_string(K) + " + q", 0, "chan[q * " + std::to_string(K) + "]") << ";\n";
    }
  }

  // Outputs that depend on the groups' means and variances alone: a thread per
  // group evaluates and stores them (eight channels to a thread, each of which may
  // begin a group, took 2 us).  False where a node varies along a group's channels.
  bool store_groups(int64_t G4) {
    std::function<bool(int)> per_group = [&](int v) {
      if (in(v)) v = rt(v);
      if (v == mo_mu || v == mo_var) return true;
      Shape d;
      if (!aligned(nd(v).shape, d) || (d[3] > 1 && K > 1) || d[1] > 1) return false;
      if (!in(v)) return true;
      for (int u : nd(v).in)
        if (!per_group(u)) return false;
      return true;
    };
    for (int o : inv_outs)
      if (!per_group(o)) return false;
    std::set<int> done;
    std::function<std::string(int)> value = [&](int v) -> std::string {
      if (in(v)) v = rt(v);
      const std::string name = "h" + id(v);
      if (!done.insert(v).second) return name;
      if (v == mo_mu) {
        s << "    const float " << name << " = chan[q];\n";
      } else if (v == mo_var) {
        s << "    const float " << name << " = chan[" << G4 << " + q] / " << flit((double)P * (double)K) << ";\n";
      } else if (!in(v)) {
        Shape d;
        aligned(nd(v).shape, d);
        s << "    const float " << name << " = ld1(" << ptr(v) << (d[0] > 1 ? " + (i64)b * " + std::to_string(d[2]) : std::string()) << (d[2] > 1 ? " + gr" : "") << ");\n";
      } else {
        const std::string ex = elem_expr(v, value);
        s << "    const float " << name << " = " << ex << ";\n";
      }
      return name;
    };
    s << "  for (int q = tid; q < " << CT / K << "; q += " << T << ") {\n    const int gr = ct0 / " << K << " + q;\n";
    for (int o : inv_outs) {
      const std::string x = value(o);
      s << "    " << out_store(g, o, outp(o), "(i64)b * " + std::to_string(G) + " + gr", 0, x) << ";\n";
    }
    s << "  }\n";
    return true;
  }

  // Hands `rowf` floats of chan (a multiple of four) from workgroup to
  // workgroup: `units` of them make a set; the last to arrive has their sum in
  // chan and goes on, the others end.  Past 64 units in two levels, groups of
  // 16 first.  `merge` joins partial rows m of the array at row `from` instead
  // of adding them.
  void hand_over(int64_t sets, const std::string& set, int64_t units, const std::string& unit, int64_t rowf, int64_t one,
                 const std::function<void(const std::string& from, const std::string& m, int64_t maxm, int level)>& merge) {
    const int64_t GS = units <= one ? units : kHandOver, NG = (units + GS - 1) / GS;
    const int64_t rows = units + (NG > 1 ? NG : 0);
    ArgRef a;
    a.kind = ArgRef::Scratch;
    a.bytes = (size_t)(sets * rows * rowf) * 4;
    const int scr = (int)gk.args.size();
    gk.args.push_back(a);
    a.kind = ArgRef::Counter;
    a.bytes = (size_t)(sets * (NG > 1 ? NG + 1 : 1)) * 128;
    const int cnt = (int)gk.args.size();
    gk.args.push_back(a);
    s << "  __shared__ int last_;\n  float* const hand = (float*)a.p[" << scr << "] + (i64)(" << set << ") * " << rows * rowf << ";\n";
    s << "  int* const cnt = (int*)a.p[" << cnt << "] + (" << set << ") * " << (NG > 1 ? NG + 1 : 1) * 32 << ";\n";
    auto put = [&](const std::string& row) {
      s << "  {\n    const __amdgpu_buffer_rsrc_t r_ = __builtin_amdgcn_make_buffer_rsrc(hand + (i64)(" << row << ") * " << rowf << ", 0, 0x7fffffff, 0x00020000);\n";
      s << "    for (int q = tid; q < " << rowf / 4 << "; q += " << T << ") coherent_store4(r_, (unsigned)q * 16, *(const float4*)(chan + q * 4));\n  }\n";
      s << "  __builtin_amdgcn_s_waitcnt(0);  // this wave's partial stores are performed\n  __syncthreads();\n";
    };
    auto arrive = [&](const std::string& c, const std::string& n) {
      s << "  if (tid == 0) {\n    int* c_ = cnt + (" << c << ") * 32;\n";
      s << "    last_ = __hip_atomic_fetch_add(c_, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (" << n << ") - 1;\n";
      s << "    if (last_) __hip_atomic_store(c_, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);\n  }\n  __syncthreads();\n  if (!last_) return;\n";
    };
    put(unit);
    if (NG > 1) {
      s << "  const int grp_ = (" << unit << ") / " << GS << ", gsz_ = " << units << " - grp_ * " << GS << " < " << GS << " ? " << units << " - grp_ * " << GS << " : " << GS
        << ";\n";
      arrive("1 + grp_", "gsz_");
      merge("grp_ * " + std::to_string(GS), "gsz_", GS, 1);
      s << "  __syncthreads();\n";
      put(std::to_string(units) + " + grp_");
      arrive("0", std::to_string(NG));
      merge(std::to_string(units), std::to_string(NG), NG, 2);
    } else {
      arrive("0", std::to_string(units));
      merge("0", std::to_string(units), units, 0);
    }
    s << "  __syncthreads();\n";
  }
  int64_t slices(int64_t rowf, int64_t maxm) const {
    int64_t z = 1;
    while (z < 8 && z * 2 <= maxm && 2 * z * (rowf / 4) <= T) z *= 2;
    return z;
  }
  // LDS that adding the partial rows of `units` workgroups takes (floats).
  int64_t slice_floats(int64_t rowf, int64_t units) const {
    int64_t most = 0;
    for (int64_t m : {units <= kOneLevel ? units : kHandOver, units <= kOneLevel ? (int64_t)1 : (units + kHandOver - 1) / kHandOver}) {
      const int64_t z = slices(rowf, m);
      if (z > 1) most = std::max(most, z * rowf);
    }
    return most;
  }
  // Adds partial rows in order: a thread per 16-byte vector and slice of the
  // rows, up to sixteen loads of a thread in flight together, then the slices.
  void add_rows(int64_t rowf, const std::string& from, const std::string& m, int64_t maxm) {
    const int64_t CQ = rowf / 4, ZS = slices(rowf, maxm);
    const int64_t per = (maxm + ZS - 1) / ZS, step = std::min<int64_t>(CQ, T / ZS);
    s << "  {\n    const __amdgpu_buffer_rsrc_t r_ = __builtin_amdgcn_make_buffer_rsrc(hand + (i64)(" << from << ") * " << rowf << ", 0, 0x7fffffff, 0x00020000);\n"
      << "    const int m_ = " << m << ", zs = tid / " << step << ";\n";
    const int64_t RD = std::min<int64_t>(per, 16);
    s << "    if (zs < " << ZS << ")\n" << as_written() << "      for (int v = tid % " << step << "; v < " << CQ << "; v += " << step << ") {\n        f32x4 t_ = {};\n";
    s << (per > RD ? "#pragma unroll 1\n" : "") << "        for (int z0 = 0; z0 < " << per << "; z0 += " << RD << ") {\n          float4 q_[" << RD << "];\n#pragma unroll\n          for (int z = 0; z < " << RD
      << "; ++z) {\n            const int zz = zs * " << per << " + z0 + z;\n            q_[z] = coherent_load4(r_, (unsigned)((zz < m_ ? zz : m_ - 1) * " << rowf * 4
      << " + v * 16));\n          }\n#pragma unroll\n          for (int z = 0; z < " << RD << "; ++z)\n            if (zs * " << per << " + z0 + z < m_" << (per % RD ? " && z0 + z < " + std::to_string(per) : std::string())
      << ") t_ += f32x4{q_[z].x, q_[z].y, q_[z].z, q_[z].w};\n        }\n";
    if (ZS == 1) {
      s << "        *(f32x4*)(chan + v * 4) = t_;\n      }\n  }\n";
      return;
    }
    s << "        *(f32x4*)(red + (zs * " << CQ << " + v) * 4) = t_;\n      }\n    __syncthreads();\n    for (int v = tid; v < " << CQ << "; v += " << T
      << ") {\n      f32x4 t_ = *(const f32x4*)(red + v * 4);\n#pragma unroll\n      for (int z = 1; z < " << ZS << "; ++z) t_ += *(const f32x4*)(red + (z * " << CQ
      << " + v) * 4);\n      *(f32x4*)(chan + v * 4) = t_;\n    }\n  }\n";
  }

  // What a kernel of the kind takes of LDS (floats).
  struct Lds {
    int64_t red = 0, part = 0, chan = 0, grp = 0, mean = 0;
    int64_t bytes() const { return (red + part + chan + grp + mean) * 4 + 64; }  // (and the flag of a hand-over, and what aligns)
  };
  Lds lds() const {
    Lds l;
    const int n = (int)r1.size();
    switch (kind) {
      case Slab: {
        int64_t widest = 1;
        for (const auto& p : passes()) {
          widest = std::max<int64_t>(widest, p.size());
          if (only_groups(p)) l.red = std::max(l.red, direct_floats((int)p.size()));
        }
        l.red = std::max({l.red, red_floats((int)widest), r0.empty() || B == 1 ? 0 : slice_floats((int64_t)r0.size() * CT4(), B)});
        l.part = part_floats((int)widest);
        l.chan = std::max<int64_t>({widest, (int64_t)r0.size(), (int64_t)r3.size()}) * CT4();
        break;
      }
      case Sums:
        l.red = std::max(red_floats(n), S > 1 ? slice_floats(n * CT4(), S) : 0);
        l.part = part_floats(n);
        l.chan = std::max<int64_t>(n, r3.size()) * CT4();
        break;
      case Moments:
        // (chan is written when red has been read for the last time)
        l.red = std::max({direct_floats(1), CT4(), 2 * ((CT / K + 3) / 4 * 4)});
        l.mean = CT / K;
        l.grp = CT / K;
        break;
      case Apply: return l;
    }
    if (kind != Moments) l.grp = std::max<int64_t>(1, r3.size()) * (CT / K);
    return l;
  }

  void head() {
    const Lds l = lds();
    if (l.red) s << "  __shared__ __attribute__((aligned(16))) float red[" << l.red << "];\n";
    if (l.part) s << "  __shared__ float part[" << l.part << "];\n";
    if (l.chan) s << "  __shared__ __attribute__((aligned(16))) float chan[" << l.chan << "];\n";
    if (l.mean) s << "  __shared__ float gmean[" << l.mean << "];\n  float* const chan = red;\n";
    if (l.grp) s << "  __shared__ float grp[" << l.grp << "];\n";
    s << "  const int tid = threadIdx.x;\n";
    if (NJ == 1) {
      s << "  const int ly = tid / " << CVT << ";\n  const bool act = ly < " << LY << ";\n";
      s << "  const int c0[1] = {ct0 + (tid - ly * " << CVT << ") * " << VEC << "};\n";
    } else {
      s << "  const int ly = 0;\n  int c0[" << NJ << "];\n  bool act[" << NJ << "];\n#pragma unroll\n  for (int j = 0; j < " << NJ << "; ++j) {\n    const int v = tid + j * " << T
        << ";\n    act[j] = v < " << CVT << ";\n    c0[j] = ct0 + (act[j] ? v : 0) * " << VEC << ";\n  }\n";
    }
  }
  // Lanes past the last whole row of lanes do no work of their own; they take part in the barriers.
  std::string first_row() const { return NJ == 1 ? "(act ? ly : " + std::to_string(LY - 1) + ")" : "0"; }

  int64_t red_floats(int n) const { return LY > 1 ? (int64_t)n * LY * CT : 0; }
  int64_t part_floats(int n) const {
    if (LY == 1 || CT >= T) return 0;
    const int64_t L = std::min<int64_t>(std::min<int64_t>(16, pow2floor(T / CT)), pow2floor(LY));
    return L > 1 ? n * L * CT : 0;
  }

  void load_invariants(const std::vector<int>& targets) {
    // per-channel operands of the nodes that the targets need, before the row loops
    std::set<int> seen;
    std::function<void(int)> walk = [&](int v) {
      if (in(v)) v = rt(v);
      if (!seen.insert(v).second) return;
      if (!in(v)) {
        if (std::find(xfull.begin(), xfull.end(), v) == xfull.end()) inv(v);
        return;
      }
      if (!is_full.at(v)) {
        inv(v);
        return;
      }
      for (int u : nd(v).in) walk(u);
    };
    for (int v : targets) walk(v);
  }

  // A thread's rows of its workgroup's part in batches, the first of which is loaded already.
  std::string stream(const std::string& work) const {
    std::ostringstream o;
    // (where registers are few, the compiler is not to know how often the loop runs: it unrolls
    // up to 32 rounds, whatever the loop's own pragma says, and spills)
    if (few_registers()) o << "  asm volatile(\"\" : \"+" << (NJ == 1 ? "v" : "s") << "\"(lim));\n";
    o << "  while (row0 < lim) {\n" << work << "    row0 += " << (int64_t)U * LY << ";\n    if (row0 >= lim) break;\n" << raw_load("row0", "p1") << "  }\n";
    return o.str();
  }

  // One pass's accumulation: `sums` over the rows in registers.
  std::string accumulate(const std::vector<int>& sums) {
    Body b;
    std::ostringstream acc;
    for (int v : sums) {
      const std::string x = full_value(nd(v).in[0], b);
      acc << "        a" << id(v) << "[j][e] += live ? " << x << " : 0.0f;\n";
    }
    return b.o.str() + acc.str();
  }
  std::string results() {
    Body b;
    std::ostringstream st;
    for (int o : full_outs) {
      const std::string x = full_value(o, b);
      st << "        o" << id(o) << "[e] = " << x << ";\n";
    }
    return b.o.str() + st.str();
  }

  // The sums over positions of each pass.
  std::vector<std::vector<int>> passes() const {
    std::vector<std::vector<int>> pass(npass);
    for (int v : r1) pass[gen.at(v) - 1].push_back(v);
    return pass;
  }

  void gen_slab() {
    const std::vector<std::vector<int>> pass = passes();
    const int64_t rowf = (int64_t)r0.size() * CT4();
    s << "  const int b = blockIdx.x / " << tiles << ", ct0 = (int)(blockIdx.x % " << tiles << ") * " << CT << ";\n";
    head();
    s << raw_decl() << "  const int row0 = " << first_row() << ";\n  {\n" << raw_load("row0", std::to_string(P)) << "  }\n";
    const std::string end = NJ == 1 ? "(act ? " + std::to_string(P) + " : 0)" : std::to_string(P);
    for (int k = 0; k < npass; ++k) {
      std::vector<int> targets;
      for (int v : pass[k]) targets.push_back(nd(v).in[0]);
      set_fast_math(false);
      load_invariants(targets);
      set_fast_math(fast_full());
      const std::string body = accumulate(pass[k]);
      std::vector<std::string> acc;
      for (int v : pass[k]) {
        s << "  float a" << id(v) << "[" << NJ << "][" << VEC << "] = {};\n";
        acc.push_back("a" + id(v));
      }
      s << "  {\n" << row_loop("row0", end, body, "") << "  }\n";
      set_fast_math(false);
      if (only_groups(pass[k])) {
        group_sums_of(acc);
        after_group_pass(pass[k]);
        after_pass(k + 1, {});
      } else {
        channel_sums(acc);
        after_pass(k + 1, pass[k]);
      }
      s << raw_again();
    }
    if (!full_outs.empty()) {
      set_fast_math(false);
      load_invariants(full_outs);
      set_fast_math(fast_full());
      const std::string body = results();
      s << "  {\n" << row_loop("row0", end, body, store_rows()) << "  }\n";
    }
    set_fast_math(false);
    store_inv();
    if (!r0.empty()) {
      // sums over the images, image by image
      s << "  __syncthreads();\n";
      for (size_t i = 0; i < r0.size(); ++i) {
        const std::string x = inv(nd(r0[i]).in[0]);
        s << each("if (" + std::string(NJ > 1 ? "act[j]" : "act") + " && ly == 0) chan[" + std::to_string(i * CT4()) + " + c0[j] - ct0 + e] = " + x + ";");
        if (CT4() > CT) s << "  if (tid < " << CT4() - CT << ") chan[" << i * CT4() + CT << " + tid] = 0.0f;\n";
      }
      s << "  __syncthreads();\n";
      if (B > 1)
        hand_over(tiles, "blockIdx.x % " + std::to_string(tiles), B, "b", rowf, kOneLevel,
                  [&](const std::string& from, const std::string& m, int64_t maxm, int) { add_rows(rowf, from, m, maxm); });
      store_r0("chan", "ct0");
    }
    gk.grid[0] = (int)(B * tiles);
  }
  // The sums over images in chan[i][..], channels c0 .. c0 + CT - 1.
  void store_r0(const std::string& arr, const std::string& first) {
    for (size_t i = 0; i < r0.size(); ++i)
      for (int o : ki.k.outs)
        if (rt(o) == r0[i]) {
          std::string x = arr + "[" + std::to_string(i * CT4()) + " + c]";
          if (nd(r0[i]).op == KORCH_REDUCE_MEAN) x += " / " + flit((double)B);
          s << "  for (int c = tid; c < " << CT << "; c += " << T << ") " << out_store(g, o, outp(o), "(" + first + " + c)", 0, x) << ";\n";
        }
  }

  void gen_sums() {
    const int64_t rowf = (int64_t)r1.size() * CT4();
    s << "  const int set = blockIdx.x / " << S << ", sp = blockIdx.x % " << S << ", b = set / " << tiles << ", ct0 = (set % " << tiles << ") * " << CT << ";\n";
    head();
    std::vector<int> targets;
    for (int v : r1) targets.push_back(nd(v).in[0]);
    s << raw_decl() << "  const int p1 = (sp + 1) * " << chunk << " < " << P << " ? (sp + 1) * " << chunk << " : " << P << ";\n  int lim = " << (NJ == 1 ? "act ? p1 : 0" : "p1") << ";\n";
    s << "  int row0 = sp * " << chunk << " + " << first_row() << ";\n" << raw_load("row0", "p1");
    load_invariants(targets);
    set_fast_math(fast_full());
    const std::string body = accumulate(r1);
    set_fast_math(false);
    std::vector<std::string> acc;
    for (int v : r1) {
      s << "  float a" << id(v) << "[" << NJ << "][" << VEC << "] = {};\n";
      acc.push_back("a" + id(v));
    }
    s << stream(row_loop("row0", "lim", body, ""));
    channel_sums(acc);
    if (CT4() > CT) {
      for (size_t i = 0; i < r1.size(); ++i) s << "  if (tid < " << CT4() - CT << ") chan[" << i * CT4() + CT << " + tid] = 0.0f;\n";
      s << "  __syncthreads();\n";
    }
    if (S > 1)
      hand_over(B * tiles, "set", S, "sp", rowf, kOneLevel, [&](const std::string& from, const std::string& m, int64_t maxm, int) { add_rows(rowf, from, m, maxm); });
    after_pass(1, r1);
    store_inv();
    gk.grid[0] = (int)(B * tiles * S);
  }

  void gen_moments() {
    const int64_t G = CT / K, G4 = (G + 3) / 4 * 4, rowf = 2 * G4;  // of the tile
    s << "  const int set = blockIdx.x / " << S << ", sp = blockIdx.x % " << S << ", b = set / " << tiles << ", ct0 = (set % " << tiles << ") * " << CT << ";\n";
    head();
    s << raw_decl() << "  const int p1 = (sp + 1) * " << chunk << " < " << P << " ? (sp + 1) * " << chunk << " : " << P << ";\n  int lim = " << (NJ == 1 ? "act ? p1 : 0" : "p1") << ";\n";
    s << "  int row0 = sp * " << chunk << " + " << first_row() << ";\n" << raw_load("row0", "p1");
    s << "  float mean[" << NJ << "][" << VEC << "] = {}, m2[" << NJ << "][" << VEC << "] = {}, cnt_ = 0.0f;\n";
    const std::string x = "tof(x" + id(mo_x) + "[i][j]" + (VEC > 1 ? "[e]" : "") + ")";
    std::ostringstream o;
    o << "    const int left = (p1 - row0 + " << LY - 1 << ") / " << LY << ";\n    const float n = (float)(left < " << U << " ? left : " << U
      << "), nn = cnt_ + n, w = n / nn, w2 = cnt_ * w, ni = 1.0f / n;\n    cnt_ = nn;\n";
    o << "#pragma unroll\n    for (int j = 0; j < " << NJ << "; ++j)\n#pragma unroll\n      for (int e = 0; e < " << VEC << "; ++e) {\n        float t = 0.0f, q = 0.0f;\n";
    // (whole batches without the selects where there are many: 22.4 us with them at 4x416x416x64 f16)
    if (U == 8)
      o << "        if (left >= " << U << ") {\n#pragma unroll\n          for (int i = 0; i < " << U << "; ++i) t += " << x << ";\n          t *= " << flit(1.0 / U) << ";\n#pragma unroll\n          for (int i = 0; i < "
        << U << "; ++i) { const float d = " << x << " - t; q = __builtin_fmaf(d, d, q); }\n        } else {\n";
    o << "#pragma unroll\n        for (int i = 0; i < " << U << "; ++i) t += i < left ? " << x << " : 0.0f;\n        t *= ni;\n#pragma unroll\n        for (int i = 0; i < " << U
      << "; ++i) { const float d = i < left ? " << x << " - t : 0.0f; q = __builtin_fmaf(d, d, q); }\n" << (U == 8 ? "        }\n" : "");
    o << "        const float d = t - mean[j][e];\n        mean[j][e] = __builtin_fmaf(d, w, mean[j][e]);\n        m2[j][e] += __builtin_fmaf(d * w2, d, q);\n      }\n";
    s << stream(o.str());
    // the workgroup's group means, then its sums of centred squares about them
    s << "  float nm[" << NJ << "][" << VEC << "];\n" << each("nm[j][e] = cnt_ * mean[j][e];");
    group_sums_of({"nm"});
    s << "  __syncthreads();\n  const float rows_ = (float)(p1 - sp * " << chunk << ");\n  for (int q = tid; q < " << G << "; q += " << T << ") gmean[q] = grp[q] / (rows_ * " << flit((double)K)
      << ");\n  __syncthreads();\n";
    s << each("const float d = mean[j][e] - gmean[(c0[j] - ct0 + e) / " + std::to_string(K) + "]; nm[j][e] = __builtin_fmaf(cnt_ * d, d, m2[j][e]);");
    group_sums_of({"nm"});
    s << "  __syncthreads();\n  for (int q = tid; q < " << G4 << "; q += " << T << ") {\n    chan[q] = q < " << G << " ? gmean[q] : 0.0f;\n    chan[" << G4 << " + q] = q < " << G
      << " ? grp[q] : 0.0f;\n  }\n  __syncthreads();\n";
    if (S > 1) {
      // (sixteen means and squares of a lane in flight, 32 where a lane has a group to itself and registers allow)
      const int64_t one = std::max<int64_t>(few_registers() ? 16 : 32, std::min(kOneLevel, 16 * std::min<int64_t>(16, pow2floor(std::max<int64_t>(1, T / G)))));
      const int64_t GS = S <= one ? S : kHandOver;
      hand_over(B * tiles, "set", S, "sp", rowf, one, [&](const std::string& from, const std::string& m, int64_t maxm, int level) {
        // rows (positions) of partial z: a split's, or those of a whole group of splits
        const int64_t per = level == 2 ? chunk * GS : chunk;
        const std::string first = level == 1 ? "(" + from + " + z)" : "z";
        const int64_t L = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(16, pow2floor(maxm)), pow2floor(std::max<int64_t>(1, T / G))));
        const int64_t nz = (maxm + L - 1) / L;
        s << as_written() << "  for (int q = tid; q < " << (G * L + T - 1) / T * T << "; q += " << T << ") {\n    const int gr_ = q / " << L << ", gr = gr_ < " << G << " ? gr_ : " << G - 1
          << ", l = q % " << L << ", m_ = " << m << ";\n    float a_[" << nz << "], b_[" << nz << "], n_[" << nz << "], t = 0.0f, n = 0.0f, v = 0.0f;\n";
        s << "    float* const p_ = hand + (i64)(" << from << ") * " << rowf << " + gr;\n";
        s << "#pragma unroll\n    for (int i = 0; i < " << nz << "; ++i) {\n      const int z_ = l + i * " << L << ", z = z_ < m_ ? z_ : m_ - 1;\n      a_[i] = coherent_load(p_ + (i64)z * " << rowf
          << ");\n      b_[i] = coherent_load(p_ + (i64)z * " << rowf << " + " << G4 << ");\n      const int lo = " << first << " * " << per << ", hi = lo + " << per << " < " << P
          << " ? lo + " << per << " : " << P << ";\n      n_[i] = z_ < m_ ? (float)(hi - lo) : 0.0f;\n    }\n";
        s << "#pragma unroll\n    for (int i = 0; i < " << nz << "; ++i) { t = __builtin_fmaf(n_[i], a_[i], t); n += n_[i]; }\n";
        if (L > 1) s << "    t = group_sum<" << L << ">(t);\n    n = group_sum<" << L << ">(n);\n";
        s << "    t /= n;\n#pragma unroll\n    for (int i = 0; i < " << nz << "; ++i) {\n      const float d = a_[i] - t;\n      v += n_[i] > 0.0f ? __builtin_fmaf(n_[i] * " << flit((double)K)
          << " * d, d, b_[i]) : 0.0f;\n    }\n";
        if (L > 1) s << "    v = group_sum<" << L << ">(v);\n";
        s << "    if (l == 0 && gr_ < " << G << ") { chan[gr] = t; chan[" << G4 << " + gr] = v; }\n  }\n";
        if (G4 > G) s << "  if (tid < " << G4 - G << ") { chan[" << G << " + tid] = 0.0f; chan[" << G4 + G << " + tid] = 0.0f; }\n";
      });
    }
    gk.grid[0] = (int)(B * tiles * S);
    if (store_groups(G4)) return;
    for (int v : {mo_mu, mo_var}) {
      s << jdecl("n" + id(v)) << each("n" + id(v) + "[j][e] = chan[" + (v == mo_var ? std::to_string(G4) + " + " : std::string()) + "(c0[j] - ct0 + e) / " + std::to_string(K) + "]" +
                                      (v == mo_var ? " / " + flit((double)P * (double)K) : std::string()) + ";");
      inv_done.insert(v);
    }
    store_inv();
  }

  void gen_apply() {
    const int64_t nblk = r0.empty() ? 0 : (C + 15) / 16;
    int64_t rblk = 0;
    if (nblk) {
      // sums over the images: 16 channels to a workgroup (a cache line of an
      // image's), the images over its groups of 16 lanes, sixteen loads in flight, and
      // many images over up to 64 workgroups (100000 images of 64 channels in one: 1.2 ms)
      const int GR = T / 16;
      const int64_t RS = nblk > 256 ? 1 : std::max<int64_t>(1, std::min<int64_t>(kOneLevel, B / (GR * 16))), per = (B + RS - 1) / RS, rowf = (int64_t)r0.size() * 16;
      rblk = nblk * RS;
      const int64_t red = RS > 1 ? slice_floats(rowf, RS) : 0;
      s << "  if (blockIdx.x >= " << B * S << ") {\n    __shared__ __attribute__((aligned(16))) float sum_[" << T << "], chan[" << rowf << "]";
      if (red) s << ", red[" << red << "]";
      s << ";\n    const int tid = threadIdx.x, k_ = (int)(blockIdx.x - " << B * S << "), set = k_ / " << RS << ", rs = k_ % " << RS << ", c = set * 16 + (tid & 15);\n    const int i1 = (rs + 1) * " << per
        << " < " << B << " ? (rs + 1) * " << per << " : " << B << ";\n";
      for (size_t k = 0; k < r0.size(); ++k) s << "    float x" << k << "_ = 0.0f;\n";
      s << "    if (c < " << C << ")\n#pragma unroll " << (r0.size() > 1 ? 8 : 16) << "\n      for (int i = rs * " << per << " + (tid >> 4); i < i1; i += " << GR << ") {\n";
      for (size_t k = 0; k < r0.size(); ++k) s << "        x" << k << "_ += ld1(" << ptr(nd(r0[k]).in[0]) << " + (i64)i * " << C << " + c);\n";
      s << "      }\n";
      for (size_t k = 0; k < r0.size(); ++k)
        s << "    " << (k ? "__syncthreads();\n    " : "") << "sum_[tid] = x" << k << "_;\n    __syncthreads();\n    if (tid < 16) {\n#pragma unroll\n      for (int w = 1; w < " << GR << "; ++w) x" << k
          << "_ += sum_[w * 16 + tid];\n      chan[" << k * 16 << " + tid] = x" << k << "_;\n    }\n";
      s << "    __syncthreads();\n";
      if (RS > 1)
        hand_over(nblk, "set", RS, "rs", rowf, kOneLevel, [&](const std::string& from, const std::string& m, int64_t maxm, int) { add_rows(rowf, from, m, maxm); });
      for (size_t k = 0; k < r0.size(); ++k)
        for (int o : ki.k.outs)
          if (rt(o) == r0[k])
            s << "    if (tid < 16 && c < " << C << ") " << out_store(g, o, outp(o), "c", 0, "chan[" + std::to_string(k * 16) + " + tid]" + (nd(r0[k]).op == KORCH_REDUCE_MEAN ? " / " + flit((double)B) : std::string()))
              << ";\n";
      s << "    return;\n  }\n";
    }
    s << "  const int b = blockIdx.x / " << S << ", sp = blockIdx.x % " << S << ", ct0 = 0;\n";
    head();
    set_fast_math(false);
    load_invariants(full_outs);
    set_fast_math(fast_full());
    const std::string body = results();
    s << raw_decl() << "  const int p1 = (sp + 1) * " << chunk << " < " << P << " ? (sp + 1) * " << chunk << " : " << P << ";\n";
    s << as_written() << "  for (int row0 = sp * " << chunk << " + " << (NJ == 1 ? "ly" : "0") << "; row0 < " << (NJ == 1 ? "(act ? p1 : 0)" : "p1") << "; row0 += " << (int64_t)U * LY << ") {\n"
      << raw_load("row0", "p1") << row_loop("row0", "p1", body, store_rows()) << "  }\n";
    gk.grid[0] = (int)(B * S + rblk);
  }

  GenKernel generate(int index) {
    analyze();
    gk.family = KORCH_FAM_GROUP;
    gk.name = kernel_name(index, "group");
    ki.assign_args(gk, slot);
    const bool was = fast_math();
    set_fast_math(false);
    switch (kind) {
      case Slab: gen_slab(); break;
      case Sums: gen_sums(); break;
      case Moments: gen_moments(); break;
      case Apply: gen_apply(); break;
    }
    set_fast_math(was);
    gk.block[0] = T;
    const char* const streamed =
        "template <int V, typename T> __device__ __forceinline__ void st_stream(T* p, const float* s) {\n  vec_t<V, T> v;\n  if constexpr (V == 1) {\n    v = fromf<T>(s[0]);\n  } else {\n"
        "#pragma unroll\n    for (int i = 0; i < V; ++i) v[i] = fromf<T>(s[i]);\n  }\n  __builtin_nontemporal_store(v, (vec_t<V, T>*)p);\n}\n";
    gk.source = source_header((int)gk.args.size()) + (stream_out() ? streamed : "") + "extern \"C\" __global__ void __launch_bounds__(" + std::to_string(T) + ") " + gk.name + "(KArgs a) {\n" + s.str() + "}\n";
    ki.fill_cost(gk);
    return gk;
  }
};

}  // namespace

bool match_group(const KInfo& ki, std::string* why) {
  try {
    GroupGen(ki).analyze();
  } catch (Error& e) {
    *why = e.what();
    return false;
  }
  return true;
}

GenKernel gen_group(const KInfo& ki, int index) { return GroupGen(ki).generate(index); }

}  // namespace korch
