// Many tensors in one kernel: the sum of the squares of all of them with what
// follows from it (the global norm of gradients and the factor that clips
// them), and each of them times one number.
//
// HBM bound: one read, and one read and one write, of every element.  The
// tensors are cut into chunks of 16-byte vectors; each workgroup takes a
// contiguous range of the chunks of all tensors and looks up once in which
// tensor it starts.  The scaling kernel walks each range backwards: what the
// norm's kernel read last is what the caches still hold.
//
// Squares are added in 64 bits (the square of an fp32 number is exact there), so
// gradients of 1e30 or 1e-30 keep the norm in range; matrix or vector rates do
// not bound a kernel that reads 16 bytes for eight such additions.  The order
// of the sum is fixed: threads, then the waves of a workgroup, then the
// workgroups by their index (past 32 in groups of 32).
#include <algorithm>

#include "families.h"

namespace korch {

namespace {

constexpr int kT = 256;          // threads
constexpr int kV = 8;            // vectors that a thread loads together
constexpr int kGroup = 32;       // workgroups whose sums one workgroup adds
constexpr int kMaxWG = 1024;     // four workgroups to a compute unit

struct MultiGen {
  const KInfo& ki;
  const Graph& g;
  bool scale = false;
  std::vector<int> in_, out_;      // tensors read (and, scaling, written)
  int factor = -1;                 // scaling: the number
  int total = -1;                  // norm: the node of the sum
  std::vector<int> tail;           // norm: one-element nodes after it
  std::set<int> sums;              // norm: nodes up to the sum

  MultiGen(const KInfo& k) : ki(k), g(k.g) {}
  [[noreturn]] static void bad(const std::string& m) { fail(KORCH_E_UNSUPPORTED, "multi: " + m); }
  const Node& nd(int v) const { return g.nodes[v]; }
  bool in(int v) const { return ki.in.count(v) > 0; }

  void analyze_scale() {
    scale = true;
    for (int o : ki.k.outs) {
      const Node& n = nd(o);
      if (n.op != KORCH_MUL || n.attrs.has_scalar) bad("an output that is not a tensor times a number");
      int x = -1;
      for (int side = 0; side < 2; ++side)
        if (!in(n.in[0]) && !in(n.in[1]) && numel(nd(n.in[1 - side]).shape) == 1 && nd(n.in[side]).shape == n.shape && (factor < 0 || factor == n.in[1 - side])) {
          x = n.in[side], factor = n.in[1 - side];
          break;
        }
      if (x < 0) bad("an output that is not a stored tensor times one stored number");
      in_.push_back(x);
      out_.push_back(o);
      if (nd(x).dtype != n.dtype) bad("a product of another type than its tensor's");
    }
    if (ki.k.prims.size() != ki.k.outs.size()) bad("other primitives");
    if (in_.size() < 2) bad("one tensor");
  }

  void analyze_norm() {
    std::vector<int> parts;
    int cat = -1;
    std::set<int> used;
    for (int r : ki.reduces) {
      const Node& n = nd(r);
      if (n.op != KORCH_REDUCE_SUM || n.axis != 0 || nd(n.in[0]).shape.size() != 2 || nd(n.in[0]).shape[1] != 1) bad("a reduction that is no sum of a column");
      const int q = n.in[0];
      if (in(q) && nd(q).op == KORCH_SQUARE && !in(nd(q).in[0])) {
        parts.push_back(r);
        in_.push_back(nd(q).in[0]);
        used.insert(q);
        used.insert(r);
      } else if (in(q) && nd(q).op == KORCH_RESHAPE && in(nd(q).in[0]) && nd(nd(q).in[0]).op == KORCH_CONCAT && cat < 0) {
        cat = nd(q).in[0];
        used.insert(q);
        used.insert(r);
        used.insert(cat);
        total = r;
      } else {
        bad("a sum of something else than squares of stored tensors");
      }
    }
    if (parts.empty()) bad("no squares");
    if (cat >= 0) {
      std::vector<int> a = nd(cat).in, b = parts;
      std::sort(a.begin(), a.end());
      std::sort(b.begin(), b.end());
      if (a != b) bad("the total is not over every sum once");
    } else {
      if (parts.size() != 1) bad("sums that are not added");
      total = parts[0];
    }
    sums = used;
    sums.erase(total);
    for (int v : ki.k.prims) {
      if (used.count(v)) continue;
      const Node& n = nd(v);
      const Kind k = op_kind(n.op);
      if (numel(n.shape) != 1 || !(k == Kind::Unary || k == Kind::Binary || k == Kind::Select || n.op == KORCH_FILL || n.op == KORCH_RESHAPE)) bad("a node beside the sum that is not one number");
      for (int u : n.in)
        if (sums.count(u) || (!in(u) && numel(nd(u).shape) != 1)) bad("a node reads more than the sum");
      tail.push_back(v);
    }
    for (int o : ki.k.outs)
      if (sums.count(o)) bad("a part of the sum is an output");
  }

  void analyze() {
    if (!ki.linear.empty()) bad("products");
    if (ki.reduces.empty())
      analyze_scale();
    else
      analyze_norm();
    if (ki.k.prims.empty() || in_.size() > 240) bad("more tensors than a launch passes");
    // (their addresses, in and out, within 4 KiB of arguments)
    if (ki.ext.size() + ki.k.outs.size() > 480) bad("more tensors than a launch passes");
    for (int u : in_)
      if (numel(nd(u).shape) >= ((int64_t)1 << 40)) bad("a tensor larger than the memory");
  }

  static std::string id(int64_t v) { return std::to_string(v); }
  int64_t chunk_of(int u) const { return (int64_t)kT * kV * (16 / dtype_bytes(nd(u).dtype)); }

  std::string one_expr(int v) const {
    const Node& n = nd(v);
    auto val = [&](int u) { return in(u) ? "n" + id(u) : "ld1((const " + ctype(nd(u).dtype) + "*)a.p[" + id(slot.at(u)) + "])"; };
    if (n.op == KORCH_FILL) return flit(n.attrs.scalar);
    if (n.op == KORCH_RESHAPE) return val(n.in[0]);
    switch (op_kind(n.op)) {
      case Kind::Unary: return n.op == KORCH_SQRT && n.in[0] == total ? "(float)__builtin_sqrt(sum)" : unary_expr(n.op, val(n.in[0]));
      case Kind::Binary: return binary_expr(n.op, val(n.in[0]), n.attrs.has_scalar ? flit(n.attrs.scalar) : val(n.in[1]));
      default: return "(" + val(n.in[0]) + " != 0.0f ? " + val(n.in[1]) + " : " + (n.attrs.has_scalar ? flit(n.attrs.scalar) : val(n.in[2])) + ")";
    }
  }

  std::map<int, int> slot;

  GenKernel generate(int index) {
    analyze();
    GenKernel gk;
    gk.family = KORCH_FAM_MULTI;
    gk.name = kernel_name(index, "multi");
    ki.assign_args(gk, slot);
    const int n = (int)in_.size();
    int64_t chunks = 0;
    std::vector<int64_t> first;
    for (int u : in_) {
      first.push_back(chunks);
      chunks += (numel(nd(u).shape) + chunk_of(u) - 1) / chunk_of(u);
    }
    first.push_back(chunks);
    const int64_t W = std::min<int64_t>(chunks, kMaxWG);
    int scr = -1, cnt = -1;
    const int64_t NG = (W + kGroup - 1) / kGroup;
    if (!scale && W > 1) {
      ArgRef r;
      r.kind = ArgRef::Scratch;
      r.bytes = (size_t)(W + NG) * 8;
      scr = (int)gk.args.size();
      gk.args.push_back(r);
      r.kind = ArgRef::Counter;
      r.bytes = (size_t)(NG + 1) * 128;
      cnt = (int)gk.args.size();
      gk.args.push_back(r);
    }
    std::ostringstream s;
    s << source_header((int)gk.args.size());
    // tables of the tensors: first chunk, elements, place of the address among the arguments, type
    s << "__device__ const i64 first_[] = {";
    for (int64_t f : first) s << f << ", ";
    s << "};\n__device__ const i64 size_[] = {";
    for (int u : in_) s << numel(nd(u).shape) << ", ";
    s << "};\n__device__ const int in_[] = {";
    for (int u : in_) s << slot.at(u) << ", ";
    s << "};\n__device__ const int type_[] = {";
    bool types[3] = {false, false, false};
    for (int u : in_) s << nd(u).dtype << ", ", types[nd(u).dtype] = true;
    s << "};\n";
    if (scale) {
      s << "__device__ const int out_[] = {";
      for (int o : out_) s << ki.out_slot(o) << ", ";
      s << "};\n";
    }
    // one chunk of one tensor
    s << "template <typename T> __device__ __forceinline__ void chunk_" << (scale ? "(const T* x, T* y, i64 left, float f)" : "(const T* x, i64 left, double& sum)")
      << " {\n  constexpr int V = 16 / (int)sizeof(T);\n  typedef vec_t<V, T> VT;\n  const int tid = threadIdx.x;\n";
    s << "  if (left >= " << kT * kV << " * V) {\n    VT q[" << kV << "];\n#pragma unroll\n    for (int i = 0; i < " << kV << "; ++i) q[i] = *(const VT*)(x + ((i * " << kT << " + tid) * V));\n";
    // Results past half of the 256 MiB that the device's last cache holds go by it:
    // their reader would not find them there, and the gradients that the norm's
    // kernel has just read stay (204 M bf16 gradients: norm and product 208 us, 233 through the cache).
    double written = 0;
    for (int o : out_) written += (double)numel(nd(o).shape) * dtype_bytes(nd(o).dtype);
    const bool stream = written > 134217728.0;
    auto one = [&](const std::string& q, const std::string& at) {
      if (scale) return "VT r_;\n#pragma unroll\n      for (int e = 0; e < V; ++e) r_[e] = fromf<T>(tof(" + q + "[e]) * f);\n      " + (stream ? "__builtin_nontemporal_store(r_, (VT*)(y + " + at + "));\n" : "*(VT*)(y + " + at + ") = r_;\n");
      return "#pragma unroll\n      for (int e = 0; e < V; ++e) { const double d = (double)tof(" + q + "[e]); sum = __builtin_fma(d, d, sum); }\n";
    };
    s << "#pragma unroll\n    for (int i = 0; i < " << kV << "; ++i) {\n      " << one("q[i]", "((i * " + id(kT) + " + tid) * V)") << "    }\n    return;\n  }\n";
    s << "  for (i64 at = tid * V; at < left; at += " << kT << " * V) {\n    if (at + V <= left) {\n      const VT q = *(const VT*)(x + at);\n      " << one("q", "at")
      << "    } else {\n      for (i64 k = at; k < left; ++k) {\n";
    if (scale)
      s << "        y[k] = fromf<T>(tof(x[k]) * f);\n";
    else
      s << "        const double d = (double)tof(x[k]); sum = __builtin_fma(d, d, sum);\n";
    s << "      }\n    }\n  }\n}\n";
    s << "extern \"C\" __global__ void __launch_bounds__(" << kT << ") " << gk.name << "(KArgs a) {\n  const int tid = threadIdx.x, w = blockIdx.x;\n";
    s << "  const i64 c0 = " << chunks << "LL * w / " << W << ", c1 = " << chunks << "LL * (w + 1) / " << W << ";\n";
    if (scale)
      s << "  const float f = ld1((const " << ctype(nd(factor).dtype) << "*)a.p[" << slot.at(factor) << "]);\n";
    else
      s << "  double sum = 0.0;\n";
    const std::string start = scale ? "c1 - 1" : "c0";
    s << "  int t = 0;\n  for (int step = " << (n > 1 ? id(1 << (31 - __builtin_clz(n - 1))) : std::string("0")) << "; step > 0; step >>= 1)\n    if (t + step < " << n << " && first_[t + step] <= "
      << start << ") t += step;\n";
    if (scale)
      s << "  for (i64 c = c1 - 1; c >= c0; --c) {\n    while (first_[t] > c) --t;\n";
    else
      s << "  for (i64 c = c0; c < c1; ++c) {\n    while (first_[t + 1] <= c) ++t;\n";
    s << "    const int ty = type_[t];\n    const i64 k = c - first_[t];\n";
    for (int ty = 0; ty < 3; ++ty) {
      if (!types[ty]) continue;
      const std::string T1 = ctype(ty);
      const int64_t ch = (int64_t)kT * kV * (16 / dtype_bytes(ty));
      s << "    if (ty == " << ty << ") chunk_<" << T1 << ">((const " << T1 << "*)a.p[in_[t]] + k * " << ch << ", " << (scale ? "(" + T1 + "*)a.p[out_[t]] + k * " + id(ch) + ", " : std::string())
        << "size_[t] - k * " << ch << ", " << (scale ? "f" : "sum") << ");\n";
    }
    s << "  }\n";
    if (!scale) {
      s << "  __shared__ double red[" << kT / 64 << "];\n#pragma unroll\n  for (int m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m, 64);\n";
      s << "  if ((tid & 63) == 0) red[tid >> 6] = sum;\n  __syncthreads();\n";
      std::string all = "red[0]";
      for (int i = 1; i < kT / 64; ++i) all = "(" + all + " + red[" + id(i) + "])";
      s << "  if (tid >= 64) return;\n  sum = " << all << ";\n";
      if (W > 1) {
        // one wave goes on: the workgroup's sum to the last of its group of 32, the groups' to the last of those
        s << "  double* part = (double*)a.p[" << scr << "];\n  int* cnt = (int*)a.p[" << cnt << "];\n";
        auto level = [&](const std::string& put, const std::string& from, const std::string& count, const std::string& counter) {
          s << "  {\n    int last = 0;\n    if (tid == 0) {\n      __hip_atomic_store(part + (" << put << "), sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);\n"
            << "      __builtin_amdgcn_s_waitcnt(0);  // the sum is stored\n      int* c_ = cnt + (" << counter << ") * 32;\n"
            << "      last = __hip_atomic_fetch_add(c_, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (" << count << ") - 1;\n"
            << "      if (last) __hip_atomic_store(c_, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);\n    }\n    if (!__shfl(last, 0, 64)) return;\n";
          s << "    const int m_ = " << count << ", z = tid < m_ ? tid : m_ - 1;\n    const double v = __hip_atomic_load(part + (" << from
            << ") + z, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);\n    sum = tid < m_ ? v : 0.0;\n#pragma unroll\n    for (int m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m, 64);\n  }\n";
        };
        if (NG > 1) {
          s << "  const int gr = w / " << kGroup << ", gs = " << W << " - gr * " << kGroup << " < " << kGroup << " ? " << W << " - gr * " << kGroup << " : " << kGroup << ";\n";
          level("w", "gr * " + id(kGroup), "gs", "1 + gr");
          level(id(W) + " + gr", id(W), id(NG), "0");
        } else {
          level("w", "0", id(W), "0");
        }
      }
      s << "  if (tid != 0) return;\n";
      set_fast_math(false);
      bool read_total = false;
      for (int v : tail)
        for (int u : nd(v).in) read_total = read_total || (u == total && nd(v).op != KORCH_SQRT);
      for (int o : ki.k.outs) read_total = read_total || o == total;
      if (read_total) s << "  const float n" << total << " = (float)sum;\n";
      for (int v : tail) s << "  const float n" << v << " = " << one_expr(v) << ";\n";
      for (int o : ki.k.outs) s << "  st1((" << ctype(nd(o).dtype) << "*)a.p[" << ki.out_slot(o) << "], n" << o << ");\n";
    }
    s << "}\n";
    gk.source = s.str();
    gk.grid[0] = (int)W;
    gk.block[0] = kT;
    ki.fill_cost(gk);
    return gk;
  }
};

}  // namespace

bool match_multi(const KInfo& ki, std::string* why) {
  try {
    MultiGen(ki).analyze();
  } catch (Error& e) {
    *why = e.what();
    return false;
  }
  return true;
}

GenKernel gen_multi(const KInfo& ki, int index) { return MultiGen(ki).generate(index); }

}  // namespace korch
