// Row programs with column sums: a kernel whose nodes are full rows [R, L] and
// row statistics [R, 1], as in the row family, and that also sums full rows
// over axis 0 (LayerNorm's gradient: the input's gradient needs two row means,
// the weight's and the bias's are sums over the rows; one pass reads the rows
// once for all of them).  Also the sum by bins on its own.
//
// HBM bound: every row tensor is read once and every row output written once.
// A workgroup walks over rows (the next row's loads go out before the current
// row's arithmetic), keeps the column sums of its lanes' columns in fp32
// registers, and hands its sums over through scratch; the last workgroup of a
// group adds the group's partial sums in order, the last group's those of the
// groups (deterministic; no floating-point atomics).  Row programs without
// column sums come here when a row is longer than a wavefront's registers: the
// waves of a workgroup share it.
#include <algorithm>

#include "families.h"

namespace korch {

namespace {

struct RowCol {
  int64_t R = 0, L = 0;
  std::vector<int> cols;      // column reductions
  std::map<int, int> cls;     // 0 full row, 1 row statistic
};

bool analyze_rowcol(const KInfo& ki, RowCol& rc, std::string* why) {
  const Graph& g = ki.g;
  auto bad = [&](const char* m) {
    *why = std::string("rowcol: ") + m;
    return false;
  };
  if (!ki.linear.empty()) return bad("has linear primitives");
  Shape F;
  for (int r : ki.reduces) {
    const Node& n = g.nodes[r];
    const Shape& s = g.nodes[n.in[0]].shape;
    if (s.size() != 2) return bad("a reduced tensor is not [rows, columns]");
    if (F.empty()) F = s;
    if (F != s) return bad("reductions over different shapes");
    if (n.axis == 0) {
      if (n.op == KORCH_REDUCE_MAX) return bad("a column maximum");
      rc.cols.push_back(r);
    } else if (!n.attrs.keepdim) {
      return bad("a row reduction without keepdim");
    }
  }
  if (ki.reduces.empty()) return bad("no reduction");
  rc.R = F[0], rc.L = F[1];
  if (rc.L < 2) return bad("rows shorter than 2");
  const Shape S = {F[0], 1};
  for (int v : ki.k.prims) {
    const Node& n = g.nodes[v];
    const Kind kd = op_kind(n.op);
    if (kd != Kind::Unary && kd != Kind::Binary && kd != Kind::Reduce) return bad("a primitive that is neither elementwise nor a reduction");
    if (std::find(rc.cols.begin(), rc.cols.end(), v) != rc.cols.end()) {
      if (std::find(ki.k.outs.begin(), ki.k.outs.end(), v) == ki.k.outs.end()) return bad("a column sum that is not an output");
      for (int c : g.consumers[v])
        if (ki.in.count(c)) return bad("a column sum is read in the kernel");
      continue;
    }
    if (kd != Kind::Reduce && n.shape == F)
      rc.cls[v] = 0;
    else if (n.shape == S)
      rc.cls[v] = 1;
    else
      return bad("a node is neither a row nor a row statistic");
    if (kd == Kind::Binary && !n.attrs.has_scalar)
      for (int u : n.in)
        if (ki.in.count(u) && rc.cls.count(u) && rc.cls[u] == 0 && rc.cls[v] == 1) return bad("incompatible operands");
  }
  for (int v : ki.k.prims)
    if (op_kind(g.nodes[v].op) == Kind::Reduce) {
      const int u = g.nodes[v].in[0];
      if (ki.in.count(u) && (!rc.cls.count(u) || rc.cls[u] != 0)) return bad("a reduction's operand is not a full row");
    }
  return true;
}

// Lanes per row G, vector VEC, vectors per lane NC; false when a row is too long.
bool rowcol_geometry(int64_t L, int eb, int& G, int& VEC, int& NC) {
  VEC = 16 / eb;
  while (L % VEC) VEC /= 2;
  const int64_t n = L / VEC;
  // up to 16 elements of every row tensor per lane: two row tensors, their
  // sums and the weights then leave two workgroups of eight waves per compute unit
  G = 1;
  while (G < 1024 && (n + G - 1) / G * VEC > 16) G *= 2;
  NC = (int)((n + G - 1) / G);
  return NC * VEC <= 64;
}

}  // namespace

bool match_rowcol(const KInfo& ki, std::string* why) {
  RowCol rc;
  if (!analyze_rowcol(ki, rc, why)) return false;
  int G, VEC, NC;
  if (!rowcol_geometry(rc.L, 2, G, VEC, NC) || !rowcol_geometry(rc.L, 4, G, VEC, NC)) {
    *why = "rowcol: rows longer than the registers of a workgroup";
    return false;
  }
  return true;
}

GenKernel gen_rowcol(const KInfo& ki, int index) {
  const Graph& g = ki.g;
  RowCol rc;
  std::string why;
  if (!analyze_rowcol(ki, rc, &why)) fail(KORCH_E_UNSUPPORTED, why);
  GenKernel gk;
  gk.family = KORCH_FAM_ROWCOL;
  gk.name = kernel_name(index, "rowcol");
  std::map<int, int> slot;
  ki.assign_args(gk, slot);
  const Shape F = {rc.R, rc.L}, S = {rc.R, 1};
  int eb = 2;
  for (int u : ki.ext)
    if (g.nodes[u].shape == F) eb = std::max(eb, dtype_bytes(g.nodes[u].dtype));
  for (int o : ki.k.outs)
    if (g.nodes[o].shape == F) eb = std::max(eb, dtype_bytes(g.nodes[o].dtype));
  int G, VEC, NC;
  if (!rowcol_geometry(rc.L, eb, G, VEC, NC)) fail(KORCH_E_UNSUPPORTED, "rowcol: rows too long");
  // Eight waves per workgroup and a workgroup per compute unit (16384 x 4096
  // bf16, three row tensors: 84 us, four waves and 512 workgroups 96; sixteen
  // waves 97).  Rows past 4096 take sixteen waves, whose hand-over of the sums
  // is the wider one (500 x 8192 fp16: 32 us, with eight 55), although a lane then
  // has 128 registers and the row loop spills some (28 to 38 at bf16 4608 to 12288,
  // 43 to 52 at f32 7168 and 8192; 4096 x 5120 bf16: 57 us, its bytes 26).
  const int NT = std::max(rc.L > 4096 ? 1024 : 512, G);
  const int RPB = NT / G, WR = G > 64 ? G / 64 : 1;
  const int64_t blocks = (rc.R + RPB - 1) / RPB;
  const int64_t NS = (int64_t)rc.cols.size(), LQ = (rc.L + 3) / 4 * 4, C = NS * LQ;  // partial sums, rows of whole 16-byte vectors
  int64_t NWG = std::min<int64_t>(blocks, 256);
  // allocation-free execution has little scratch: fewer workgroups hand over 16 MiB
  const int64_t NWG_small = std::max<int64_t>(1, ((int64_t)16 << 20) / std::max<int64_t>(1, C * 4));
  gk.wg_split = NWG > NWG_small;
  if (!workgroup_splits()) NWG = std::min(NWG, NWG_small);
  const bool ragged = (rc.L / VEC) % G != 0;  // the last vector of some lanes is past the row
  auto guard = [&](int j) { return j == NC - 1 && ragged ? "c" + std::to_string(j) + "_ok" : std::string(); };
  // Row tensors are loaded one row ahead in their own type, into the registers
  // that the conversion to fp32 has just freed (two or three rows ahead gained
  // nothing: 84.9 and 87.2 us against 83.8).
  std::ostringstream decl, raw, load, conv;
  std::map<int, std::string> full;  // external tensors: value in `for e` at chunk j
  auto ext_full = [&](int u) -> std::string {
    auto f = full.find(u);
    if (f != full.end()) return f->second;
    const Node& n = g.nodes[u];
    const std::string T = ctype(n.dtype), P = "((const " + T + "*)a.p[" + std::to_string(slot.at(u)) + "])";
    const std::string id = std::to_string(u);
    const Shape s2 = n.shape.size() == 2 ? n.shape : n.shape.size() == 1 ? Shape{1, n.shape[0]} : Shape{1, 1};
    if (n.shape.size() > 2) fail(KORCH_E_UNSUPPORTED, "rowcol: operand rank");
    const bool byrow = s2[0] > 1, bycol = s2[1] > 1;
    if (!bycol) {  // one value per row, or one value
      if (byrow) {
        raw << "    " << T << " r" << id << ";\n";
        load << "    q.r" << id << " = " << P << "[row];\n";
        conv << "    const float e" << id << " = tof(q_.r" << id << ");\n";
      } else {
        decl << "  const float e" << id << " = ld1(" << P << ");\n";
      }
      return full[u] = "e" + id;
    }
    if (byrow) {
      const std::string VT = "vec_t<" + std::to_string(VEC) + ", " + T + ">";
      raw << "    " << VT << " r" << id << "[" << NC << "];\n";
      for (int j = 0; j < NC; ++j)
        load << "    q.r" << id << "[" << j << "] = *(const " << VT << "*)(" << P << " + row * " << rc.L << "LL + c" << j << ");\n";
      conv << "    float e" << id << "[" << NC << "][" << VEC << "];\n#pragma unroll\n    for (int j = 0; j < " << NC << "; ++j)\n#pragma unroll\n"
           << "      for (int e = 0; e < " << VEC << "; ++e) e" << id << "[j][e] = tof(" << (VEC == 1 ? "q_.r" + id + "[j]" : "q_.r" + id + "[j][e]")
           << ");\n";
    } else {
      decl << "  float e" << id << "[" << NC << "][" << VEC << "];\n";
      for (int j = 0; j < NC; ++j) decl << "  ldv<" << VEC << ">(e" << id << "[" << j << "], " << P << " + c" << j << ");\n";
    }
    return full[u] = "e" + id + "[j][e]";
  };
  std::vector<int> pending;  // row reductions whose lanes are not yet summed
  std::ostringstream body;
  auto flush = [&]() {
    if (pending.empty()) return;
    for (int v : pending) {
      const bool mx = g.nodes[v].op == KORCH_REDUCE_MAX;
      body << "    s" << v << " = " << (mx ? "group_max<" : "group_sum<") << std::min(G, 64) << ">(s" << v << ");\n";
    }
    if (G > 64) {
      // one barrier per exchange: buffers alternate
      const int NP = (int)pending.size();
      body << "    {\n      float* x_ = xch + (par & 1) * " << 8 * NT / 64 << ";\n      par ^= 1;\n";
      for (int i = 0; i < NP; ++i) body << "      if ((tid & 63) == 0) x_[" << i * (NT / 64) << " + (tid >> 6)] = s" << pending[i] << ";\n";
      body << "      __syncthreads();\n";
      for (int i = 0; i < NP; ++i) {
        const int v = pending[i];
        const bool mx = g.nodes[v].op == KORCH_REDUCE_MAX;
        body << "      s" << v << " = x_[" << i * (NT / 64) << " + w0_];\n#pragma unroll\n      for (int w = 1; w < " << WR << "; ++w) s" << v << " = "
             << (mx ? "k_max(s" + std::to_string(v) + ", " : "s" + std::to_string(v) + " + (") << "x_[" << i * (NT / 64) << " + w0_ + w]);\n";
      }
      body << "    }\n";
    }
    for (int v : pending)
      if (g.nodes[v].op == KORCH_REDUCE_MEAN) body << "    s" << v << " = s" << v << " / " << flit((double)rc.L) << ";\n";
    pending.clear();
  };
  auto operand = [&](int u, bool row) -> std::string {
    if (!ki.in.count(u)) {
      const Node& n = g.nodes[u];
      if (!row && n.shape != S && numel(n.shape) != 1) fail(KORCH_E_UNSUPPORTED, "rowcol: a statistic reads a row");
      return ext_full(u);
    }
    if (rc.cls.at(u) == 0) return "v" + std::to_string(u) + "[j][e]";
    if (std::find(pending.begin(), pending.end(), u) != pending.end()) flush();
    return "s" + std::to_string(u);
  };
  auto each = [&](const std::string& stmt, bool guarded) {
    for (int j = 0; j < NC; ++j) {
      const std::string gd = guarded ? guard(j) : "";
      body << "    " << (gd.empty() ? "" : "if (" + gd + ") ") << "{\n      constexpr int j = " << j << ";\n#pragma unroll\n      for (int e = 0; e < "
           << VEC << "; ++e) " << stmt << ";\n    }\n";
    }
  };
  for (int v : ki.k.prims) {
    const Node& n = g.nodes[v];
    const Kind kd = op_kind(n.op);
    const std::string V = std::to_string(v);
    if (std::find(rc.cols.begin(), rc.cols.end(), v) != rc.cols.end()) {
      const std::string x = operand(n.in[0], true);
      each("k" + V + "[j][e] += live ? " + x + " : 0.0f", true);
      continue;
    }
    if (kd == Kind::Reduce) {
      const bool mx = n.op == KORCH_REDUCE_MAX;
      const std::string x = operand(n.in[0], true);
      body << "    float s" << V << " = " << (mx ? "-__builtin_huge_valf()" : "0.0f") << ";\n";
      each("s" + V + " = " + (mx ? "k_max(s" + V + ", " + x + ")" : "s" + V + " + " + x), true);
      pending.push_back(v);
      if (pending.size() == 8) flush();
      continue;
    }
    const bool row = rc.cls.at(v) == 0;
    const std::string x = operand(n.in[0], row);
    const std::string y = kd == Kind::Unary ? "" : n.attrs.has_scalar ? flit(n.attrs.scalar) : operand(n.in[1], row);
    const std::string ex = kd == Kind::Unary ? unary_expr(n.op, x) : binary_expr(n.op, x, y);
    if (row) {
      body << "    float v" << V << "[" << NC << "][" << VEC << "];\n";
      each("v" + V + "[j][e] = " + ex, false);
    } else {
      body << "    const float s" << V << " = " << ex << ";\n";
    }
  }
  flush();
  for (int o : ki.k.outs) {
    if (std::find(rc.cols.begin(), rc.cols.end(), o) != rc.cols.end()) continue;
    const Node& on = g.nodes[o];
    const std::string P = "((" + ctype(on.dtype) + "*)a.p[" + std::to_string(ki.out_slot(o)) + "])";
    if (rc.cls.at(o) == 0) {
      for (int j = 0; j < NC; ++j) {
        const std::string gd = guard(j);
        body << "    if (live" << (gd.empty() ? "" : " && " + gd) << ") "
             << out_store(g, o, P, "row * " + std::to_string(rc.L) + "LL + c" + std::to_string(j), VEC, "v" + std::to_string(o) + "[" + std::to_string(j) + "]")
             << ";\n";
      }
    } else {
      body << "    if (live && lane == 0) " << out_store(g, o, P, "row", 0, "s" + std::to_string(o)) << ";\n";
    }
  }
  // hand-over of the column sums
  int64_t GS = 1, NG = 1;
  int scr = -1, cnt = -1;
  const bool hand = NWG > 1 && NS > 0;
  if (hand) {
    GS = NWG <= 32 ? NWG : 16;
    NG = (NWG + GS - 1) / GS;
    ArgRef a;
    a.kind = ArgRef::Scratch;
    a.bytes = (size_t)((NWG + (NG > 1 ? NG : 0)) * C) * 4;
    scr = (int)gk.args.size();
    gk.args.push_back(a);
    a.kind = ArgRef::Counter;
    a.bytes = (size_t)(NG + 1) * 128;
    cnt = (int)gk.args.size();
    gk.args.push_back(a);
  }
  std::ostringstream s;
  s << source_header((int)gk.args.size());
  s << "extern \"C\" __global__ void __launch_bounds__(" << NT << ") " << gk.name << "(KArgs a) {\n";
  const int64_t LP = (int64_t)G * NC * VEC;  // columns that the lanes of a row cover
  const int64_t CQ = C / 4;                  // 16-byte vectors of a partial row
  // slices of the partial rows that a workgroup adds side by side
  int64_t ZS = 1;
  while (ZS < 16 && 2 * ZS * CQ <= NT) ZS *= 2;
  const int64_t red_floats = std::max(RPB > 1 && NS > 0 ? RPB * LP : 0, hand && ZS > 1 ? ZS * C : 0);
  if (red_floats) s << "  __shared__ __attribute__((aligned(16))) float red[" << red_floats << "];\n";
  if (G > 64) s << "  __shared__ float xch[" << 2 * 8 * NT / 64 << "];\n  int par = 0;\n";
  if (hand) s << "  __shared__ int last_;\n";
  s << "  const int tid = threadIdx.x, lane = tid % " << G << ", sub = tid / " << G << ";\n";
  if (G > 64) s << "  const int w0_ = sub * " << WR << ";\n";
  for (int j = 0; j < NC; ++j) {
    s << "  const i64 cc" << j << " = ((i64)" << j << " * " << G << " + lane) * " << VEC << ";\n";
    s << "  const bool c" << j << "_ok = cc" << j << " < " << rc.L << "LL;\n";
    // lanes past the row read its first elements (their values are not used)
    s << "  const i64 c" << j << " = c" << j << "_ok ? cc" << j << " : 0;\n";
  }
  s << "  struct Raw {\n" << raw.str() << "  };\n  Raw q_;\n";
  s << "  auto fetch = [&](Raw& q, i64 blk) {\n    const i64 w_ = blk * " << RPB << " + sub, row = w_ < " << rc.R << "LL ? w_ : " << rc.R - 1
    << "LL;\n" << load.str() << "  };\n";
  s << decl.str();
  for (int v : rc.cols) s << "  float k" << v << "[" << NC << "][" << VEC << "] = {};\n";
  s << "  fetch(q_, blockIdx.x);\n";
  s << "#pragma unroll 1\n  for (i64 blk = blockIdx.x; blk < " << blocks << "LL; blk += " << NWG << ") {\n";
  s << "    const i64 w_ = blk * " << RPB << " + sub;\n    const bool live = w_ < " << rc.R << "LL;\n    const i64 row = live ? w_ : " << rc.R - 1
    << "LL;\n";
  s << conv.str() << "    fetch(q_, blk + " << NWG << "LL);\n" << body.str() << "  }\n";
  auto final_value = [&](int v, const std::string& x) {
    return g.nodes[v].op == KORCH_REDUCE_MEAN ? "(" + x + ") / " + flit((double)rc.R) : x;
  };
  auto out_ptr = [&](int v) { return "((" + ctype(g.nodes[v].dtype) + "*)a.p[" + std::to_string(ki.out_slot(v)) + "])"; };
  // the workgroup's rows: groups of lanes with the same columns, in order
  if (hand) s << "  float* part = (float*)a.p[" << scr << "] + (i64)blockIdx.x * " << C << "LL;\n";
  for (size_t i = 0; i < rc.cols.size(); ++i) {
    const int v = rc.cols[i];
    const std::string V = std::to_string(v);
    auto put = [&](const std::string& col, const std::string& x) {
      if (hand) return "coherent_store(&part[" + std::to_string(i * LQ) + "LL + " + col + "], " + x + ")";
      return "st1(" + out_ptr(v) + " + " + col + ", " + final_value(v, x) + ")";
    };
    if (RPB > 1) {
      if (i) s << "  __syncthreads();\n";
      for (int j = 0; j < NC; ++j)
        s << "#pragma unroll\n  for (int e = 0; e < " << VEC << "; ++e) red[sub * " << LP << " + " << j * G * VEC << " + lane * " << VEC
          << " + e] = k" << V << "[" << j << "][e];\n";
      s << "  __syncthreads();\n";
      s << "  for (int c = tid; c < " << rc.L << "; c += " << NT << ") {\n    float x_ = red[c];\n#pragma unroll\n    for (int q = 1; q < " << RPB
        << "; ++q) x_ += red[q * " << LP << " + c];\n    " << put("c", "x_") << ";\n  }\n";
    } else {
      for (int j = 0; j < NC; ++j)
        s << "  if (c" << j << "_ok)\n#pragma unroll\n    for (int e = 0; e < " << VEC << "; ++e) " << put("c" + std::to_string(j) + " + e", "k" + V + "[" + std::to_string(j) + "][e]")
          << ";\n";
    }
  }
  if (hand) {
    s << "  __builtin_amdgcn_s_waitcnt(0);  // this wave's partial stores are performed\n  __syncthreads();\n";
    s << "  int* cnt = (int*)a.p[" << cnt << "];\n";
    const std::string base = "((float*)a.p[" + std::to_string(scr) + "])";
    auto arrive = [&](const std::string& c, const std::string& n) {
      s << "  if (tid == 0) {\n    int* c_ = cnt + (" << c << ") * 32;\n";
      s << "    const int n_ = " << n << ";\n";
      s << "    last_ = __hip_atomic_fetch_add(c_, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == n_ - 1;\n";
      s << "    if (last_) __hip_atomic_store(c_, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);\n  }\n  __syncthreads();\n  if (!last_) return;\n";
    };
    // Adds partial rows 0 .. m-1 (m <= maxn) of `from`: a thread per 16-byte
    // vector and slice of the rows, every load of a thread in flight together;
    // then the slices, in order.
    auto add_up = [&](const std::string& from, const std::string& count, int64_t maxn, const std::function<void(const std::string&, const std::string&)>& sink) {
      const int64_t per = (maxn + ZS - 1) / ZS, step = std::min<int64_t>(CQ * ZS, NT) / ZS;
      s << "  {\n    const __amdgpu_buffer_rsrc_t r_ = __builtin_amdgcn_make_buffer_rsrc(" << from << ", 0, 0x7fffffff, 0x00020000);\n    const int m_ = "
        << count << ";\n";
      s << "    const int zs = tid / " << step << ";\n    for (int v = tid % " << step << "; v < " << CQ << " && zs < " << ZS << "; v += " << step << ") {\n";
      s << "      float4 q_[" << per << "];\n#pragma unroll\n      for (int z = 0; z < " << per << "; ++z) {\n        const int zz = zs * " << per
        << " + z;\n        q_[z] = coherent_load4(r_, (unsigned)((zz < m_ ? zz : m_ - 1) * " << C * 4 << " + v * 16));\n      }\n";
      s << "      f32x4 x_ = {};\n#pragma unroll\n      for (int z = 0; z < " << per << "; ++z)\n        if (zs * " << per
        << " + z < m_) x_ += f32x4{q_[z].x, q_[z].y, q_[z].z, q_[z].w};\n";
      if (ZS > 1) {
        s << "      *(f32x4*)(red + zs * " << C << " + v * 4) = x_;\n    }\n    __syncthreads();\n";
        s << "    for (int v = tid; v < " << CQ << "; v += " << NT << ") {\n      f32x4 x_ = *(const f32x4*)(red + v * 4);\n#pragma unroll\n      for (int z = 1; z < "
          << ZS << "; ++z) x_ += *(const f32x4*)(red + z * " << C << " + v * 4);\n";
      }
      sink("v", "x_");
      s << "    }\n  }\n";
    };
    auto outputs = [&](const std::string& v, const std::string& x) {
      for (size_t i = 0; i < rc.cols.size(); ++i) {
        s << "      if (" << v << " >= " << i * LQ / 4 << " && " << v << " < " << (i + 1) * LQ / 4 << ")\n#pragma unroll\n        for (int e = 0; e < 4; ++e)\n";
        s << "          if ((" << v << " - " << i * LQ / 4 << ") * 4 + e < " << rc.L << ") st1(" << out_ptr(rc.cols[i]) << " + ((" << v << " - " << i * LQ / 4
          << ") * 4 + e), " << final_value(rc.cols[i], x + "[e]") << ");\n";
      }
    };
    if (ZS > 1) s << "  __syncthreads();\n";
    if (NG > 1) {
      s << "  const int grp = blockIdx.x / " << GS << ";\n  const int gsz = " << NWG << " - grp * " << GS << " < " << GS << " ? " << NWG << " - grp * " << GS << " : " << GS
        << ";\n";
      arrive("1 + grp", "gsz");
      const std::string to = "(" + base + " + " + std::to_string(NWG * C) + "LL)";
      add_up("(" + base + " + (i64)grp * " + std::to_string(GS * C) + "LL)", "gsz", GS, [&](const std::string& v, const std::string& x) {
        s << "      coherent_store4(__builtin_amdgcn_make_buffer_rsrc(" << to << " + (i64)grp * " << C << "LL, 0, 0x7fffffff, 0x00020000), (unsigned)(" << v
          << " * 16), float4{" << x << "[0], " << x << "[1], " << x << "[2], " << x << "[3]});\n";
      });
      s << "  __builtin_amdgcn_s_waitcnt(0);\n  __syncthreads();\n";
      arrive("0", std::to_string(NG));
      add_up(to, std::to_string(NG), NG, outputs);
    } else {
      arrive("0", std::to_string(NWG));
      add_up(base, std::to_string(NWG), NWG, outputs);
    }
  }
  s << "}\n";
  gk.source = s.str();
  gk.grid[0] = (int)NWG;
  gk.block[0] = NT;
  ki.fill_cost(gk);
  return gk;
}

// ---------------------------------------------------------------------------
// A sum by bins on its own (a plan that stores the summed tensor): a workgroup
// per result element adds the matching values in a fixed order, and so reads all
// values once per bin (only plans of one kernel per primitive come here).
// ---------------------------------------------------------------------------

bool match_binsum(const KInfo& ki, std::string* why) {
  int b = -1;
  for (int v : ki.k.prims) {
    const Kind kd = op_kind(ki.g.nodes[v].op);
    if (kd == Kind::BinSum) {
      if (b >= 0) return *why = "binsum: more than one sum by bins", false;
      b = v;
    } else if (kd == Kind::Reduce || kd == Kind::Linear) {
      return *why = "binsum: a reduction or a product", false;
    }
  }
  if (b < 0 || ki.k.outs.size() != 1 || ki.k.outs[0] != b) return *why = "binsum: the only output must be the sum by bins", false;
  for (int v : ki.k.prims)
    if (v != b && !ki.ancestor(v, b)) return *why = "binsum: a node that the sum does not read", false;
  if (numel(ki.g.nodes[b].shape) * 256 >= (int64_t)1 << 32) return *why = "binsum: more threads than a launch holds", false;
  return true;
}

GenKernel gen_binsum(const KInfo& ki, int index) {
  const Graph& g = ki.g;
  GenKernel gk;
  gk.family = KORCH_FAM_BINSUM;
  gk.name = kernel_name(index, "binsum");
  std::map<int, int> slot;
  ki.assign_args(gk, slot);
  const int o = ki.k.outs[0];
  const Node& n = g.nodes[o];
  const Shape& X = g.nodes[n.in[0]].shape;
  const int R = (int)X.size(), tr = (int)n.shape.size();
  const int64_t T = n.shape.back();
  Emitter em(g);
  em.inset = ki.in;
  em.argslot = slot;
  em.vec = 1;
  em.force_gather = true;
  std::vector<Ix> it(R);
  for (int d = 0; d < R; ++d) it[d] = Ix::var("i" + std::to_string(d));
  const std::string x = em.value(n.in[0], it);
  const std::string k = em.value(n.in[1], broadcast_index(g.nodes[n.in[1]].shape, X, it));
  int64_t inner = 1;
  std::ostringstream kept, summed;
  for (int d = R - 1; d >= 0; --d) {
    const int j = d - (R - (tr - 1));
    const bool keep = j >= 0 && n.shape[j] != 1;
    std::ostringstream& to = keep ? kept : summed;
    to << (keep ? "  " : "    ") << "const i64 i" << d << " = " << (keep ? "w_" : "q_") << " % " << X[d] << "LL; " << (keep ? "w_" : "q_") << " /= " << X[d]
       << "LL;\n";
    if (!keep) inner *= X[d];
  }
  std::ostringstream s;
  s << source_header((int)gk.args.size());
  s << "extern \"C\" __global__ void __launch_bounds__(256) " << gk.name << "(KArgs a) {\n  __shared__ float red[4];\n";
  s << "  const float bin = (float)(blockIdx.x % " << T << ");\n  i64 w_ = blockIdx.x / " << T << ";\n" << kept.str();
  s << "  float sum = 0.0f;\n  for (i64 t = threadIdx.x; t < " << inner << "LL; t += 256) {\n    i64 q_ = t;\n" << summed.str() << em.pre.str() << em.body.str();
  s << "    sum += k_min(k_max(" << k << ", 0.0f), " << flit((double)(T - 1)) << ") == bin ? " << x << " : 0.0f;\n  }\n";
  s << "  sum = group_sum<64>(sum);\n  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;\n  __syncthreads();\n";
  s << "  if (threadIdx.x == 0) st1((" << ctype(n.dtype) << "*)a.p[" << ki.out_slot(o) << "] + (i64)blockIdx.x, ((red[0] + red[1]) + red[2]) + red[3]);\n}\n";
  gk.source = s.str();
  gk.grid[0] = (int)numel(n.shape);
  ki.fill_cost(gk);
  return gk;
}

}  // namespace korch
