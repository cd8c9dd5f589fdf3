"""Primitive graphs of the five workloads, built through the C ABI, with their plans.

Operator fission is applied by hand (Korch, Section 3): softmax becomes a row
max, a subtraction, an exponential, a row sum and a division; LayerNorm
becomes mean, subtraction, square, mean, add-eps, reciprocal square root,
scaling and the affine pair; Mish becomes exp, add 1, log, tanh and a product.
Broadcast is implicit in binary primitives (ONNX style, Section 5.1).

Each builder returns a ``Workload`` with the graph handle, a name -> node map,
and named plans:
  * "fused":   the recommended orchestration (fewest kernels, redundant
               recomputation where it saves traffic: Section 4.2);
  * "layered": a plan that keeps each dense product in its own kernel;
  * "unfused": one kernel per primitive (korch_plan_unfused).
"""

from __future__ import annotations

import math
from dataclasses import dataclass, field

from ._abi import Graph, Plan


@dataclass
class Workload:
    name: str
    dtype: str
    graph: Graph
    ids: dict
    input_names: list
    output_names: list
    plans: dict = field(default_factory=dict)  # name -> list of (prim names, out names)
    sizes: dict = field(default_factory=dict)

    def node(self, name):
        return self.ids[name]

    def kernels(self, plan_name):
        ks = []
        for prims, outs in self.plans[plan_name]:
            ks.append(([self.ids[p] for p in prims], [self.ids[o] for o in outs]))
        return ks

    def plan(self, plan_name):
        if plan_name == "unfused":
            return Plan(self.graph)
        return Plan(self.graph, self.kernels(plan_name))


class _B:
    """Small helper that names nodes as they are created."""

    def __init__(self, dtype):
        self.g = Graph()
        self.dtype = dtype
        self.ids = {}
        self.inputs = []

    def inp(self, name, shape, dtype=None):
        self.ids[name] = self.g.input(dtype or self.dtype, shape)
        self.inputs.append(name)
        return self.ids[name]

    def op(self, name, op, ins, dtype=None, **attrs):
        self.ids[name] = self.g.op(op, [self.ids[i] for i in ins], dtype or self.dtype, **attrs)
        return self.ids[name]


def _finish(b, name, outputs, sizes, extra_outputs=()):
    """Marks the outputs (then any extra named nodes, so that a test can read
    an intermediate tensor of the unfused plan) and finalizes the graph."""
    names = list(outputs) + [x for x in extra_outputs if x not in outputs]
    for o in names:
        b.g.output(b.ids[o])
    b.g.finalize()
    return Workload(name, b.dtype, b.g, b.ids, b.inputs, names, sizes=sizes)


def _softmax(b, s):
    b.op("m", "reduce_max", [s], axis=-1, keepdim=True)
    b.op("Z", "sub", [s, "m"])
    b.op("E", "exp", ["Z"])
    b.op("s", "reduce_sum", ["E"], axis=-1, keepdim=True)
    b.op("P", "div", ["E", "s"])


def _layernorm(b, x, eps, p=""):
    b.op(p + "mu", "reduce_mean", [x], axis=-1, keepdim=True)
    b.op(p + "D", "sub", [x, p + "mu"])
    b.op(p + "D2", "square", [p + "D"])
    b.op(p + "var", "reduce_mean", [p + "D2"], axis=-1, keepdim=True)
    b.op(p + "ve", "add", [p + "var"], scalar=eps)
    b.op(p + "r", "rsqrt", [p + "ve"])
    b.op(p + "Xh", "mul", [p + "D", p + "r"])
    b.op(p + "Yg", "mul", [p + "Xh", "gamma"])
    b.op(p + "Y", "add", [p + "Yg", "beta"])
    return p + "Y"


def attention(n=128, d=64, nk=None, dtype="f32", extra_outputs=()):
    nk = n if nk is None else nk
    b = _B(dtype)
    b.inp("Q", (n, d))
    b.inp("K", (nk, d))
    b.inp("V", (nk, d))
    b.op("KT", "transpose", ["K"], perm=(1, 0))
    b.op("S0", "matmul", ["Q", "KT"])
    b.op("S", "mul", ["S0"], scalar=1.0 / math.sqrt(d))
    _softmax(b, "S")
    b.op("O", "matmul", ["P", "V"])
    w = _finish(b, "attention", ["O"], dict(n=n, d=d, nk=nk), extra_outputs)
    w.plans["fused"] = [(["KT", "S0", "S", "m", "Z", "E", "s", "P", "O"], ["O"])]
    w.plans["layered"] = [(["KT", "S0", "S"], ["S"]), (["m", "Z", "E", "s", "P"], ["P"]), (["O"], ["O"])]
    return w


def mlp(m=4096, d=768, h=3072, dtype="f16", eps=1e-5, extra_outputs=()):
    b = _B(dtype)
    b.inp("X", (m, d))
    b.inp("W1", (d, h))
    b.inp("W2", (h, d))
    b.inp("gamma", (d,))
    b.inp("beta", (d,))
    _layernorm(b, "X", eps)
    b.op("H0", "matmul", ["Y", "W1"])
    b.op("Hg", "gelu_tanh", ["H0"])
    b.op("Zo", "matmul", ["Hg", "W2"])
    b.op("out", "add", ["Zo", "X"])
    w = _finish(b, "mlp", ["out"], dict(m=m, d=d, h=h), extra_outputs)
    # The statistics kernel materializes the centred rows D and the row scale
    # r (two outputs); normalization and affine run in the first product's
    # operand prologue, GELU in its epilogue, the residual in the second
    # product's epilogue.  (mu cannot be an output of a kernel that also holds
    # its only consumer D: Definition 3.)
    w.plans["fused"] = [
        (["mu", "D", "D2", "var", "ve", "r"], ["D", "r"]),
        (["Xh", "Yg", "Y", "H0", "Hg"], ["Hg"]),
        (["Zo", "out"], ["out"]),
    ]
    w.plans["layered"] = [
        (["mu", "D", "D2", "var", "ve", "r", "Xh", "Yg", "Y"], ["Y"]),
        (["H0", "Hg"], ["Hg"]),
        (["Zo", "out"], ["out"]),
    ]
    return w


def sra(hh=128, ww=128, c=64, r=8, dtype="f16", eps=1e-5, extra_outputs=()):
    b = _B(dtype)
    b.inp("X", (hh, ww, c))
    b.inp("Wsr", (r * r * c, c))
    b.inp("gamma", (c,))
    b.inp("beta", (c,))
    b.op("Xr", "reshape", ["X"], shape=(hh // r, r, ww // r, r, c))
    b.op("Xt", "transpose", ["Xr"], perm=(0, 2, 1, 3, 4))
    b.op("A", "reshape", ["Xt"], shape=((hh // r) * (ww // r), r * r * c))
    b.op("KVp", "matmul", ["A", "Wsr"])
    kv = _layernorm(b, "KVp", eps, p="ln_")
    b.op("Qv", "reshape", ["X"], shape=(hh * ww, c))
    b.op("KT", "transpose", [kv], perm=(1, 0))
    b.op("S0", "matmul", ["Qv", "KT"])
    b.op("S", "mul", ["S0"], scalar=1.0 / math.sqrt(c))
    _softmax(b, "S")
    b.op("O", "matmul", ["P", kv])
    w = _finish(b, "sra", ["O"], dict(hh=hh, ww=ww, c=c, r=r), extra_outputs)
    ln = ["ln_mu", "ln_D", "ln_D2", "ln_var", "ln_ve", "ln_r", "ln_Xh", "ln_Yg", "ln_Y"]
    w.plans["fused"] = [
        (["Xt", "A", "KVp"] + ln, ["ln_Y"]),
        (["KT", "S0", "S", "m", "Z", "E", "s", "P", "O"], ["O"]),
    ]
    w.plans["layered"] = [
        (["Xt", "A", "KVp"], ["KVp"]),
        (ln, ["ln_Y"]),
        (["KT", "S0", "S"], ["S"]),
        (["m", "Z", "E", "s", "P"], ["P"]),
        (["O"], ["O"]),
    ]
    return w


def conv(hh=416, ww=416, cin=32, cout=64, k=3, dtype="f16", extra_outputs=()):
    b = _B(dtype)
    b.inp("X", (hh, ww, cin))
    b.inp("W", (k, k, cin, cout))
    b.inp("scale", (cout,))
    b.inp("shift", (cout,))
    b.op("C", "conv2d", ["X", "W"], stride=1, pad=k // 2)
    b.op("B1", "mul", ["C", "scale"])
    b.op("B", "add", ["B1", "shift"])
    b.op("E", "exp", ["B"])
    b.op("E1", "add", ["E"], scalar=1.0)
    b.op("SP", "log", ["E1"])
    b.op("T", "tanh", ["SP"])
    b.op("Y", "mul", ["B", "T"])
    w = _finish(b, "conv", ["Y"], dict(hh=hh, ww=ww, cin=cin, cout=cout, k=k), extra_outputs)
    w.plans["fused"] = [(["C", "B1", "B", "E", "E1", "SP", "T", "Y"], ["Y"])]
    w.plans["layered"] = [(["C", "B1", "B"], ["B"]), (["E", "E1", "SP", "T", "Y"], ["Y"])]
    return w


def linattn(heads=16, n=4096, d=16, dtype="bf16", eps=1e-6, extra_outputs=()):
    b = _B(dtype)
    b.inp("Q", (heads, n, d))
    b.inp("K", (heads, n, d))
    b.inp("V", (heads, n, d))
    b.op("Qr", "relu", ["Q"])
    b.op("Kr", "relu", ["K"])
    b.op("KrT", "transpose", ["Kr"], perm=(0, 2, 1))
    b.op("KVm", "matmul", ["KrT", "V"])
    b.op("sK", "reduce_sum", ["Kr"], axis=1, keepdim=True)
    b.op("num", "matmul", ["Qr", "KVm"])
    b.op("sKT", "transpose", ["sK"], perm=(0, 2, 1))
    b.op("den0", "matmul", ["Qr", "sKT"])
    b.op("den", "add", ["den0"], scalar=eps)
    b.op("out", "div", ["num", "den"])
    w = _finish(b, "linattn", ["out"], dict(heads=heads, n=n, d=d), extra_outputs)
    w.plans["fused"] = [
        (["Kr", "KrT", "KVm", "sK"], ["KVm", "sK"]),
        (["Qr", "num", "sKT", "den0", "den", "out"], ["out"]),
    ]
    w.plans["layered"] = [
        (["Kr", "KrT", "KVm"], ["KVm"]),
        (["Kr", "sK"], ["sK"]),
        (["Qr", "num", "sKT", "den0", "den", "out"], ["out"]),
    ]
    return w


def instnorm(hh=224, ww=224, c=32, dtype="f16", eps=1e-5, extra_outputs=()):
    b = _B(dtype)
    b.inp("X", (hh, ww, c))
    b.inp("gamma", (c,))
    b.inp("beta", (c,))
    b.op("Xp", "reshape", ["X"], shape=(hh * ww, c))
    b.op("mu", "reduce_mean", ["Xp"], axis=0, keepdim=True)
    b.op("D", "sub", ["Xp", "mu"])
    b.op("D2", "square", ["D"])
    b.op("var", "reduce_mean", ["D2"], axis=0, keepdim=True)
    b.op("ve", "add", ["var"], scalar=eps)
    b.op("r", "rsqrt", ["ve"])
    b.op("Xh", "mul", ["D", "r"])
    b.op("Yg", "mul", ["Xh", "gamma"])
    b.op("Y", "add", ["Yg", "beta"])
    b.op("R", "relu", ["Y"])
    b.op("Ri", "reshape", ["R"], shape=(hh, ww, c))
    b.op("out", "pad", ["Ri"], begin=(1, 1, 0), end=(1, 1, 0))
    w = _finish(b, "instnorm", ["out"], dict(hh=hh, ww=ww, c=c), extra_outputs)
    # operator per kernel (InstanceNorm as mean, variance and normalize; ReLU; Pad).
    # D feeds both the variance and the normalization, and a kernel holding D
    # and Xh but not the variance chain would not be convex, so the variance
    # kernel materializes D.
    w.plans["layered"] = [(["mu"], ["mu"]), (["D", "D2", "var", "ve", "r"], ["D", "r"]),
                          (["Xh", "Yg", "Y"], ["Y"]), (["R"], ["R"]), (["out"], ["out"])]
    # norm fission fused into the following ReLU and Pad (Section 6 case study)
    w.plans["fused"] = [(["mu"], ["mu"]), (["D", "D2", "var", "ve", "r"], ["D", "r"]),
                        (["Xh", "Yg", "Y", "R", "Ri", "out"], ["out"])]
    return w


def layernorm(m=4096, d=768, dtype="f16", eps=1e-5, extra_outputs=()):
    """LayerNorm of the rows of X that keeps what its gradient needs: the row
    means ``mu`` and reciprocal deviations ``r`` (fp32)."""
    if not 0 <= eps < math.inf:
        raise ValueError("eps must be finite and not negative")
    b = _B(dtype)
    b.inp("X", (m, d))
    b.inp("gamma", (d,))
    b.inp("beta", (d,))
    b.op("mu", "reduce_mean", ["X"], "f32", axis=-1, keepdim=True)
    b.op("D", "sub", ["X", "mu"], "f32")
    b.op("D2", "square", ["D"], "f32")
    b.op("var", "reduce_mean", ["D2"], "f32", axis=-1, keepdim=True)
    b.op("ve", "add", ["var"], "f32", scalar=eps)
    b.op("r", "rsqrt", ["ve"], "f32")
    b.op("Xh", "mul", ["D", "r"], "f32")
    b.op("Yg", "mul", ["Xh", "gamma"], "f32")
    b.op("Y", "add", ["Yg", "beta"])
    w = _finish(b, "layernorm", ["Y", "mu", "r"], dict(m=m, d=d), extra_outputs)
    w.plans["fused"] = [(["mu", "D", "D2", "var", "ve", "r", "Xh", "Yg", "Y"], ["Y", "mu", "r"])]
    return w


def layernorm_grad(m=4096, d=768, dtype="f16", eps=1e-5, extra_outputs=()):
    """LayerNorm's gradient from dY and the saved row statistics: dX, and the
    sums over the rows dgamma = sum dY Xh and dbeta = sum dY.  With
    g = dY gamma and Xh = (X - mu) r,  dX = r (g - mean(g) - Xh mean(g Xh)).
    (``eps`` is in the saved r.)"""
    b = _B(dtype)
    b.inp("X", (m, d))
    b.inp("gamma", (d,))
    b.inp("mu", (m, 1), "f32")
    b.inp("r", (m, 1), "f32")
    b.inp("dY", (m, d))
    b.op("D", "sub", ["X", "mu"], "f32")
    b.op("Xh", "mul", ["D", "r"], "f32")
    b.op("dYXh", "mul", ["dY", "Xh"], "f32")
    b.op("dgamma", "reduce_sum", ["dYXh"], axis=0, keepdim=False)
    b.op("dbeta", "reduce_sum", ["dY"], axis=0, keepdim=False)
    b.op("g", "mul", ["dY", "gamma"], "f32")
    b.op("gXh", "mul", ["dYXh", "gamma"], "f32")
    b.op("c1", "reduce_mean", ["g"], "f32", axis=-1, keepdim=True)
    b.op("c2", "reduce_mean", ["gXh"], "f32", axis=-1, keepdim=True)
    b.op("G1", "sub", ["g", "c1"], "f32")
    b.op("Xc", "mul", ["Xh", "c2"], "f32")
    b.op("G2", "sub", ["G1", "Xc"], "f32")
    b.op("dX", "mul", ["G2", "r"])
    w = _finish(b, "layernorm_grad", ["dX", "dgamma", "dbeta"], dict(m=m, d=d), extra_outputs)
    w.plans["fused"] = [(["D", "Xh", "dYXh", "dgamma", "dbeta", "g", "gXh", "c1", "c2", "G1", "Xc", "G2", "dX"],
                         ["dX", "dgamma", "dbeta"])]
    # the row program and the two column sums apart
    w.plans["layered"] = [(["D", "Xh", "dYXh", "g", "gXh", "c1", "c2", "G1", "Xc", "G2", "dX"], ["dX"]),
                          (["D", "Xh", "dYXh", "dgamma"], ["dgamma"]), (["dbeta"], ["dbeta"])]
    return w


LOW = -1e30   # the score of a masked pair in a row's maximum
TINY = 1e-30  # the divisor of a row whose mask leaves nothing: its result is 0


class _Attention:
    """The score plane that attention and its gradient share: operands, scores,
    caps, biases and the mask, as primitives of a builder.

    Query heads that share a key head are rows of one product: Q [batch, heads,
    n, d] is read as [batch, kv_heads, group * n, d] (a view), so the sums over
    a group in the gradients are the products' own.  With a bias table, which
    differs from head to head, a group is a batch axis instead."""

    def __init__(self, b, batch, heads, kv_heads, n, m, d, cap, slopes, causal, prefix, documents, lengths, radius, buckets):
        kv_heads = heads if kv_heads is None else kv_heads
        m = n if m is None else m
        if min(batch, heads, kv_heads, n, m, d) < 1 or heads % kv_heads:
            raise ValueError("heads must be a positive multiple of kv_heads, and every size positive")
        if n > m:
            raise ValueError("the queries are the last n of m positions: n must not exceed m")
        if prefix and not causal:
            raise ValueError("a prefix extends a causal mask: causal must be set")
        if bool(buckets) != bool(radius) or buckets < 0 or radius < 0:
            raise ValueError("radius and buckets go together")
        if not (cap == 0 or 1e-30 <= cap < math.inf):  # (scores are divided by it in fp32)
            raise ValueError("cap must be 0 (none) or finite and at least 1e-30")
        self.b, self.sizes = b, dict(batch=batch, heads=heads, kv_heads=kv_heads, n=n, m=m, d=d, cap=cap, slopes=slopes,
                                     causal=causal, prefix=prefix, documents=documents, lengths=lengths, radius=radius,
                                     buckets=buckets)
        group = heads // kv_heads
        self.batch, self.heads, self.kv, self.group, self.n, self.m, self.d = batch, heads, kv_heads, group, n, m, d
        self.cap, self.scale = cap, 1.0 / math.sqrt(d)
        self.apart = bool(buckets) and group > 1  # a group as a batch axis
        self.fold = group > 1 and not self.apart
        self.rows = group * n if self.fold else n
        # leading dims of query-side and key-side tensors
        self.qlead = (batch, kv_heads, group) if self.apart else (batch, kv_heads)
        self.klead = (batch, kv_heads, 1) if self.apart else (batch, kv_heads)
        self.prims = []
        b.inp("Q", (batch, heads, n, d))
        b.inp("K", (batch, kv_heads, m, d))
        b.inp("V", (batch, kv_heads, m, d))

    def op(self, name, op, ins, dtype="f32", **attrs):
        """A primitive of the plane, part of every kernel that evaluates it."""
        self.b.op(name, op, ins, dtype, **attrs)
        self.prims.append(name)
        return name

    def view(self, name, src, shape, dtype=None):
        """A view of a stored tensor (no kernel computes it)."""
        if self.b.g.node_info(self.b.ids[src])[2] == tuple(shape):
            return src
        self.b.op(name, "reshape", [src], dtype, shape=shape)
        return name

    def per_row(self, name, src, lead, dtype="f32"):
        """[.., n] -> [.., rows, 1]: one value per row of the plane, repeated for the heads of a group."""
        b = self.b
        if self.fold:
            self.op(name + "_g", "broadcast", [src], dtype, shape=lead + (self.group, self.n))
            return self.op(name, "reshape", [name + "_g"], dtype, shape=lead + (self.rows, 1))
        return self.op(name, "reshape", [src], dtype, shape=lead + (self.n, 1))

    def vectors(self, slopes, causal, prefix, documents, lengths, radius, buckets):
        """The inputs beside Q, K and V."""
        b, ones = self.b, (1,) * (len(self.qlead) - 1)
        if slopes:
            b.inp("slopes", (self.heads,), "f32")
        if lengths:
            b.inp("lengths", (self.batch,), "f32")
        if prefix:
            b.inp("prefix", (self.batch,), "f32")
        if documents:
            b.inp("documents", (self.batch, self.m), "f32")
        if buckets:
            b.inp("bucket", (2 * radius + 1,), "f32")
            b.inp("table", (self.heads, buckets))
        # positions of keys and queries (the last n positions in use)
        if causal or slopes or buckets or lengths:
            self.op("key", "iota", [], shape=(1, self.m), axis=1)
        if lengths:
            end = self.view("end", "lengths", (self.batch,) + ones + (1, 1), "f32")
            # rows of K and V past a sequence's length are read as zeros
            self.op("key_r", "iota", [], shape=(self.m, 1), axis=0)
            self.op("used", "lt", ["key_r", end])
        if causal or slopes or buckets or documents:
            pos = "row" if self.m == self.n and not lengths and not self.fold else "row_i"
            if self.fold:
                self.op("row", "iota", [], shape=(self.group, self.n), axis=1)
                self.op("row_i", "reshape", ["row"], shape=(self.rows, 1))
            else:
                self.op(pos, "iota", [], shape=(self.n, 1), axis=0)
            if lengths:
                self.op("first", "sub", [end], scalar=float(self.n))
                self.op("pos", "add", [pos, "first"])
            elif self.m != self.n:
                self.op("pos", "add", [pos], scalar=float(self.m - self.n))
            else:
                self.b.ids["pos"] = self.b.ids[pos]
        if slopes or buckets:
            self.op("rel", "sub", ["key", "pos"])
        mask = None

        def both(x):
            nonlocal mask
            mask = x if mask is None else self.op(f"mask{len(self.prims)}", "mul", [mask, x])

        if causal:
            self.op("seen", "le", ["key", "pos"])
            if prefix:
                pre = self.view("pre", "prefix", (self.batch,) + ones + (1, 1), "f32")
                self.op("inpre", "lt", ["key", pre])
                self.op("seenp", "max", ["seen", "inpre"])
            both("seenp" if prefix else "seen")
        if documents:
            doc = self.view("doc", "documents", (self.batch,) + ones + (1, self.m), "f32")
            tab = self.view("doc_t", "documents", (self.batch,) + ones + (1, 1, self.m), "f32")
            self.op("docq", "gather", [tab, "pos"])
            both(self.op("samedoc", "eq", ["docq", doc]))
        if lengths:
            both(self.op("inuse", "lt", ["key", end]))
        self.mask = mask
        self.lengths, self.slopes, self.buckets = lengths, slopes, buckets

    def operands(self):
        b = self.b
        self.q = self.view("Q4", "Q", self.qlead + (self.rows, self.d))
        self.k = self.view("K4", "K", self.klead + (self.m, self.d))
        self.v = self.view("V4", "V", self.klead + (self.m, self.d))
        if self.lengths:
            self.k = self.op("Km", "select", ["used", self.k], b.dtype, scalar=0.0)
            self.v = self.op("Vm", "select", ["used", self.v], b.dtype, scalar=0.0)

    def swap(self):
        r = len(self.qlead) + 2
        return tuple(range(r - 2)) + (r - 1, r - 2)

    def scores(self):
        """S [.., rows, m] (fp32); with a cap, ``t`` = tanh(scale Q K^T / cap)."""
        b = self.b
        self.op("KT", "transpose", [self.k], b.dtype, perm=self.swap())
        self.op("S0", "matmul", [self.q, "KT"])
        if self.cap:
            self.op("Sx", "mul", ["S0"], scalar=self.scale / self.cap)
            self.op("t", "tanh", ["Sx"])
            s = self.op("Sc", "mul", ["t"], scalar=self.cap)
        else:
            s = self.op("Sc", "mul", ["S0"], scalar=self.scale)
        if self.slopes:
            if self.fold:
                lead = self.view("slope_h", "slopes", (self.kv, self.group, 1), "f32")
                self.op("slope_g", "broadcast", [lead], shape=(self.kv, self.group, self.n))
                self.op("slope", "reshape", ["slope_g"], shape=(self.kv, self.rows, 1))
            else:
                self.view("slope", "slopes", self.qlead[1:] + (1, 1), "f32")
            self.op("dist", "abs", ["rel"])
            self.op("bias_d", "mul", ["dist", "slope"])
            s = self.op("Sd", "sub", [s, "bias_d"])
        if self.buckets:
            self.op("at", "add", ["rel"], scalar=float(self.sizes["radius"]))
            self.op("which", "gather", ["bucket", "at"])
            tab = self.view("table_h", "table", self.qlead[1:] + (1, 1, self.buckets))
            self.op("bias_b", "gather", [tab, "which"])
            s = self.op("Sb", "add", [s, "bias_b"])
        self.s = s

    def masked(self, name, x, value=0.0):
        return x if self.mask is None else self.op(name, "select", [self.mask, x], scalar=value)

    def out(self, name, src, shape, dtype=None):
        """A result in the caller's shape (the last primitive of its kernel)."""
        self.b.op(name, "reshape", [src], dtype, shape=shape)
        return name


def mha(batch=1, heads=8, kv_heads=None, n=1024, m=None, d=64, dtype="bf16", cap=0.0, slopes=False, causal=False, prefix=False,
        documents=False, lengths=False, radius=0, buckets=0, extra_outputs=()):
    """Attention of any length in one kernel: O = softmax(S) V and the row's
    log-sum-exp L (fp32, 0 for a row whose mask leaves nothing; its O is 0).

      S = scale Q K^T, capped by cap tanh(S / cap) if ``cap``,
        - slopes[h] |j - i|           if ``slopes``   (input ``slopes`` [heads], fp32)
        + table[h, bucket[j - i]]     if ``buckets``  (inputs ``table`` [heads, buckets] and ``bucket``
                                                       [2 radius + 1], fp32 whole numbers: the bucket of
                                                       distances -radius .. radius; farther ones take the ends')

    Q is [batch, heads, n, d], K and V are [batch, kv_heads, m, d]; query head h
    reads key head h // (heads / kv_heads).  The queries are the last n of m
    positions (n = 1: the next token over a cache of m - 1).  Masks, all of
    which must hold: ``causal`` (j <= i; with ``prefix`` [batch] also j <
    prefix), ``documents`` [batch, m] (equal document numbers), ``lengths``
    [batch] (the first lengths[b] >= n of the m positions are in use, the
    queries are the last n of those; K and V past them are never used and may hold
    anything).  Numbers are fp32 whole numbers below 2^24.  The fused plan takes
    widths d of whole 16-byte vectors up to 256."""
    b = _B(dtype)
    a = _Attention(b, batch, heads, kv_heads, n, m, d, cap, slopes, causal, prefix, documents, lengths, radius, buckets)
    a.vectors(slopes, causal, prefix, documents, lengths, radius, buckets)
    a.operands()
    a.scores()
    top = a.masked("Sm", a.s, LOW)
    a.op("mx", "reduce_max", [top], axis=-1, keepdim=True)
    a.op("Z", "sub", [a.s, "mx"])
    a.op("Ex", "exp", ["Z"])
    e = a.masked("E", "Ex")
    a.op("l", "reduce_sum", [e], axis=-1, keepdim=True)
    # the exponentials are rounded to the operands' type for the product (half a
    # step of that type each; the fused kernel's, in fp16, times 2^7); their sum is fp32
    ec = e if dtype == "f32" else a.op("Ec", "identity", [e], dtype)
    a.op("Ov", "matmul", [ec, a.v])
    a.op("lt", "max", ["l"], scalar=TINY)
    a.op("On", "div", ["Ov", "lt"], dtype)
    a.op("lg", "log", ["lt"])
    a.op("ml", "add", ["mx", "lg"])
    a.op("some", "gt", ["l"], scalar=0.0)
    a.op("Ln", "select", ["some", "ml"], scalar=0.0)
    a.out("O", "On", (batch, heads, n, d))
    a.out("L", "Ln", (batch, heads, n, 1), "f32")
    w = _finish(b, "mha", ["O", "L"], a.sizes, extra_outputs)
    w.plans["fused"] = [(a.prims + ["O", "L"], ["O", "L"])]
    return w


def mha_grad(batch=1, heads=8, kv_heads=None, n=1024, m=None, d=64, dtype="bf16", cap=0.0, slopes=False, causal=False, prefix=False,
             documents=False, lengths=False, radius=0, buckets=0, extra_outputs=()):
    """The gradient of ``mha`` (same arguments) from dO and the forward pass's O
    and L: dQ, dK, dV, and with ``buckets`` the table's gradient dT.

      P = exp(S - L), dP = dO V^T, delta = rowsum(dO O), dS = P (dP - delta),
      dX = dS (1 - t^2) scale,  dQ = dX K, dK = dX^T Q, dV = P^T dO,
      dT[h, k] = sum of dS over the batch and the pairs of bucket k.

    The scores are evaluated again by the kernel that owns the queries (dQ, dT)
    and by the one that owns the keys (dK, dV): every sum is taken in a fixed
    order.  The fused plan takes as many buckets as their sums fit LDS beside the
    tiles (about 400 for 16-bit heads of 64); in fp16 it scales P and dX by powers of
    two, so that a small dO keeps its bits and a large one stays finite (the
    unfused plan stores both as they are).  Allocation-free execution has 32 MiB for
    the buckets' partial sums."""
    b = _B(dtype)
    a = _Attention(b, batch, heads, kv_heads, n, m, d, cap, slopes, causal, prefix, documents, lengths, radius, buckets)
    b.inp("dO", (batch, heads, n, d))
    b.inp("O", (batch, heads, n, d))
    b.inp("L", (batch, heads, n, 1), "f32")
    a.vectors(slopes, causal, prefix, documents, lengths, radius, buckets)
    b.op("dOO", "mul", ["dO", "O"], "f32")
    b.op("delta", "reduce_sum", ["dOO"], "f32", axis=-1, keepdim=True)
    a.operands()
    a.scores()
    lse = a.view("L4", "L", a.qlead + (a.rows, 1), "f32")
    # delta as the kernel that sums it reads it, and as it is stored
    delta = a.view("delta4", "delta", a.qlead + (a.rows, 1), "f32")
    head = ["dOO", "delta"] + (["delta4"] if delta != "delta" else [])
    a.view("delta_s", "delta", (batch, heads, n), "f32")
    a.view("delta_s4", "delta_s", a.qlead + (a.rows, 1), "f32")
    do = a.view("dO4", "dO", a.qlead + (a.rows, d))
    a.op("Z", "sub", [a.s, lse])
    a.op("Ex", "exp", ["Z"])
    p = a.masked("P", "Ex")
    rest = list(a.prims)
    a.prims.clear()
    a.op("VT", "transpose", [a.v], dtype, perm=a.swap())
    a.op("dP", "matmul", [do, "VT"])
    pre = list(a.prims)

    def score_gradient(delta, c):
        """dS and dX for one of the two kernels.  P and dX are rounded to the operands' type for
        the products, half a step each, as every sum over them averages such errors out (two parts
        of dX would keep it, for one product more in either kernel).  In fp16 the fused kernels
        round them times a power of two, which keeps them among its normal numbers."""
        a.prims.clear()
        a.op("dD" + c, "sub", ["dP", delta])
        a.op("dS" + c, "mul", [p, "dD" + c])
        ds = dx = a.masked("dSm" + c, "dS" + c)
        if cap:
            if not c:
                b.op("t2", "square", ["t"], "f32")
                b.op("nt2", "neg", ["t2"], "f32")
                b.op("dt", "add", ["nt2"], "f32", scalar=1.0)
            a.prims += ["t2", "nt2", "dt"]
            a.op("dU" + c, "mul", [ds, "dt"])
            dx = a.masked("dX" + c, "dU" + c)
        xc = dx if dtype == "f32" else a.op("Xc" + c, "identity", [dx], dtype)
        return ds, xc, pre + list(a.prims)

    ds, xc, plane = score_gradient(delta, "")
    b.op("dQ0", "matmul", [xc, a.k], "f32")
    b.op("dQ1", "mul", ["dQ0"], scalar=a.scale)
    a.out("dQ", "dQ1", (batch, heads, n, d))
    rows, rows_out = ["dQ0", "dQ1", "dQ"], ["dQ"]
    if buckets:
        b.op("dT0", "bin_sum", [ds, "which"], shape=a.qlead[1:] + (1, 1, buckets))
        a.out("dT", "dT0", (heads, buckets))
        rows, rows_out = rows + ["dT0", "dT"], rows_out + ["dT"]
    _, xk, plane_k = score_gradient("delta_s4", "_k")
    b.op("XT", "transpose", [xk], perm=a.swap())
    b.op("dK0", "matmul", ["XT", a.q], "f32")
    pc = p
    cols_p = []
    if dtype != "f32":
        b.op("Pc", "identity", [p])
        pc, cols_p = "Pc", ["Pc"]
    b.op("PT", "transpose", [pc], perm=a.swap())
    cols_p += ["PT"]
    b.op("dV0", "matmul", ["PT", do], "f32")
    after = []
    if a.apart:
        for x in ("K", "V"):
            b.op(f"d{x}g", "reduce_sum", [f"d{x}0"], "f32", axis=2, keepdim=False)
            b.op(f"d{x}", "mul" if x == "K" else "identity", [f"d{x}g"], **(dict(scalar=a.scale) if x == "K" else {}))
            after.append(([f"d{x}g", f"d{x}"], [f"d{x}"]))
        ko, vo = ["dK0"], ["dV0"]
    else:
        b.op("dK1", "mul", ["dK0"], scalar=a.scale)
        b.op("dV1", "identity", ["dV0"])
        a.out("dK", "dK1", (batch, a.kv, a.m, d))
        a.out("dV", "dV1", (batch, a.kv, a.m, d))
        ko, vo = ["dK0", "dK1", "dK"], ["dV0", "dV1", "dV"]
    outs = ["dQ", "dK", "dV"] + (["dT"] if buckets else [])
    w = _finish(b, "mha_grad", outs, a.sizes, extra_outputs)
    kout, vout = ko[-1:], vo[-1:]
    dk = rest + plane_k + ["XT"] + ko
    dv = rest + cols_p + vo
    # dK and dV share their scores in one kernel as far as the registers go (2x16
    # causal capped heads of 2048, width 128: 141 us, two kernels 206; 4096 without
    # a mask 780 and 740)
    cols = [(sorted(set(dk + dv)), kout + vout)] if d <= 128 else [(dk, kout), (dv, vout)]
    # the kernel that owns the queries also sums delta, which the keys' reads (as a
    # node of its own: a kernel's output has a reader that is not in the kernel)
    w.plans["fused"] = [(head + rest + plane + rows, ["delta"] + rows_out)] + cols + after
    return w


# The least normal and the largest fp32 number (eps and limits of a norm are fp32 in the kernels).
_F32_MIN, _F32_MAX = 2.0 ** -126, (2.0 - 2.0 ** -23) * 2.0 ** 127

# Activations after a group norm.
ACTIVATIONS = ("none", "relu", "silu")


class _GroupNorm:
    """The sizes and views that group norm and its gradient share: a map
    [batch, hh, ww, c] is read as [batch, positions, groups, channels of a group]."""

    def __init__(self, b, batch, hh, ww, c, groups, eps, act):
        if min(batch, hh, ww, c, groups) < 1 or c % groups:
            raise ValueError("c must be a positive multiple of groups, and every size positive")
        if hh * ww * (c // groups) < 2:
            raise ValueError("a group needs two elements")
        if not 0 <= eps <= _F32_MAX:
            raise ValueError("eps must be finite in fp32 and not negative")
        if act not in ACTIVATIONS:
            raise ValueError(f"act must be one of {', '.join(ACTIVATIONS)}")
        self.b, self.act, self.eps = b, act, eps
        self.batch, self.groups, self.per, self.positions = batch, groups, c // groups, hh * ww
        self.map, self.sizes = (batch, hh, ww, c), dict(batch=batch, hh=hh, ww=ww, c=c, groups=groups, act=act)
        self.full = (batch, self.positions, groups, self.per)
        self.stat = (batch, 1, groups, 1)
        self.prims = []

    def view(self, name, src, shape, dtype=None):
        """A view of a stored tensor (no kernel computes it)."""
        self.b.op(name, "reshape", [src], dtype, shape=shape)
        return name

    def op(self, name, op, ins, dtype="f32", **attrs):
        """A primitive that kernels compute."""
        self.b.op(name, op, ins, dtype, **attrs)
        self.prims.append(name)
        return name

    def relu(self, name, z, dtype="f32"):
        """max(z, 0), and NaN where z is (the relu primitive is a maximum instruction, which drops it)."""
        self.op(name + "_off", "le", [z], scalar=0.0)
        self.op(name + "_on", "eq", [name + "_off"], scalar=0.0)
        return self.op(name, "select", [name + "_on", z], dtype, scalar=0.0)

    def over_group(self, name, op, src):
        """A reduction over the positions and the channels of a group."""
        src = self.op(name + "_p" if self.per > 1 else name, op, [src], axis=1, keepdim=True)
        return self.op(name, op, [src], axis=3, keepdim=True) if self.per > 1 else src


def groupnorm(batch=1, hh=64, ww=64, c=320, groups=32, dtype="f16", eps=1e-5, act="silu", extra_outputs=()):
    """Group norm of a map X [batch, hh, ww, c] (channels last) with an activation,
    that keeps what its gradient needs: per image and group of c / groups
    channels the mean ``mu`` and the reciprocal deviation ``r`` over all
    positions and the group's channels (fp32 [batch, groups]).

      Xh = (X - mu) r,  Z = Xh gamma + beta,  Y = Z, relu(Z) or silu(Z) = Z / (1 + exp(-Z))

    The "fused" plan is one kernel where an image's group fits the registers of
    a workgroup, else the statistics and the rest ("layered"), which take up to
    8192 channels."""
    b = _B(dtype)
    m = _GroupNorm(b, batch, hh, ww, c, groups, eps, act)
    b.inp("X", m.map)
    b.inp("gamma", (c,))
    b.inp("beta", (c,))
    m.view("X4", "X", m.full)
    m.view("gamma4", "gamma", m.full[2:])
    m.view("beta4", "beta", m.full[2:])
    mu = m.over_group("mu4", "reduce_mean", "X4")
    m.op("mu", "reshape", [mu], shape=(batch, groups))
    m.op("D", "sub", ["X4", mu])
    m.op("D2", "square", ["D"])
    var = m.over_group("var", "reduce_mean", "D2")
    m.op("ve", "add", [var], scalar=eps)
    m.op("r4", "rsqrt", ["ve"])
    m.op("r", "reshape", ["r4"], shape=(batch, groups))
    stats = list(m.prims)
    # the statistics as what comes after them reads them, stored or not
    m.op("mu_s", "reshape", ["mu"], shape=m.stat)
    m.op("r_s", "reshape", ["r"], shape=m.stat)
    views = m.prims[len(stats):]
    m.op("Dn", "sub", ["X4", "mu_s"])
    m.op("Xh", "mul", ["Dn", "r_s"])
    m.op("Yg", "mul", ["Xh", "gamma4"])
    if act == "none":
        last = m.op("Z", "add", ["Yg", "beta4"], dtype)
    else:
        m.op("Z", "add", ["Yg", "beta4"])
        if act == "relu":
            last = m.relu("Ya", "Z", dtype)
        else:
            m.op("nZ", "neg", ["Z"])
            m.op("eZ", "exp", ["nZ"])
            m.op("eZ1", "add", ["eZ"], scalar=1.0)
            last = m.op("Ya", "div", ["Z", "eZ1"], dtype)
    m.op("Y", "reshape", [last], dtype, shape=m.map)
    w = _finish(b, "groupnorm", ["Y", "mu", "r"], m.sizes, extra_outputs)
    rest = [p for p in m.prims if p not in stats and p not in views]
    whole = (list(m.prims), ["Y", "mu", "r"])
    w.plans["layered"] = [(stats, ["mu", "r"]), (rest, ["Y"])]
    w.plans["fused"] = [whole] if _one_kernel(w, whole) else w.plans["layered"]
    return w


def _one_kernel(w, kernel):
    """Whether a family takes the kernel (names) as one."""
    prims, outs = kernel
    return w.graph.family([w.ids[p] for p in prims], [w.ids[o] for o in outs]) != "none"


def groupnorm_grad(batch=1, hh=64, ww=64, c=320, groups=32, dtype="f16", eps=1e-5, act="silu", extra_outputs=()):
    """The gradient of ``groupnorm`` (same arguments) from dY and the saved
    statistics: dX, dgamma and dbeta.  The activation's input is evaluated again
    (so ``beta`` is an input where there is an activation).

      dZ = dY act'(Z),  dbeta = sum dZ,  dgamma = sum dZ Xh  over images and positions,
      g = dZ gamma,  dX = r (g - mean(g) - Xh mean(g Xh))   means over a group's positions and channels,

    with relu'(Z) = [Z > 0] (NaN where Z is) and silu'(Z) = s (1 + Z (1 - s)), s = 1 / (1 + exp(-Z)).
    The means come from the sums over the positions that dgamma and dbeta need
    anyway.  (``eps`` is in the saved r.)"""
    b = _B(dtype)
    m = _GroupNorm(b, batch, hh, ww, c, groups, eps, act)
    b.inp("X", m.map)
    b.inp("gamma", (c,))
    if act != "none":
        b.inp("beta", (c,))
    b.inp("mu", (batch, groups), "f32")
    b.inp("r", (batch, groups), "f32")
    b.inp("dY", m.map)
    m.view("X4", "X", m.full)
    m.view("dY4", "dY", m.full)
    m.view("gamma4", "gamma", m.full[2:])
    m.view("mu4", "mu", m.stat, "f32")
    m.view("r4", "r", m.stat, "f32")
    if act != "none":
        m.view("beta4", "beta", m.full[2:])

    def plane(c):
        """Xh and dZ (the kernel of the sums and the one of dX evaluate them each)."""
        m.prims.clear()
        m.op("D" + c, "sub", ["X4", "mu4"])
        m.op("Xh" + c, "mul", ["D" + c, "r4"])
        if act == "none":
            return "dY4"
        m.op("Yg" + c, "mul", ["Xh" + c, "gamma4"])
        m.op("Z" + c, "add", ["Yg" + c, "beta4"])
        if act == "relu":
            m.op("on" + c, "gt", ["Z" + c], scalar=0.0)
            return m.op("dZ" + c, "select", ["on" + c, "dY4", m.relu("Zp" + c, "Z" + c)])
        m.op("nZ" + c, "neg", ["Z" + c])
        m.op("eZ" + c, "exp", ["nZ" + c])
        m.op("eZ1" + c, "add", ["eZ" + c], scalar=1.0)
        m.op("s" + c, "recip", ["eZ1" + c])
        m.op("ns" + c, "neg", ["s" + c])
        m.op("s1" + c, "add", ["ns" + c], scalar=1.0)
        m.op("Zs" + c, "mul", ["Z" + c, "s1" + c])
        m.op("Zs1" + c, "add", ["Zs" + c], scalar=1.0)
        m.op("slope" + c, "mul", ["s" + c, "Zs1" + c])
        return m.op("dZ" + c, "mul", ["dY4", "slope" + c])

    dz = plane("")
    m.op("dZx", "mul", [dz, "Xh"])
    m.op("sb", "reduce_sum", [dz], axis=1, keepdim=True)
    m.op("sg", "reduce_sum", ["dZx"], axis=1, keepdim=True)

    def mean(name, src):
        m.op(name + "_g", "mul", [src, "gamma4"])
        if m.per > 1:
            m.op(name + "_s", "reduce_sum", [name + "_g"], axis=3, keepdim=True)
        return m.op(name, "mul", [name + ("_s" if m.per > 1 else "_g")], scalar=1.0 / (m.positions * m.per))

    mean("c1", "sb")
    mean("c2", "sg")
    sums = list(m.prims)
    dz = plane("_x")
    m.op("g", "mul", [dz, "gamma4"])
    m.op("G1", "sub", ["g", "c1"])
    m.op("Xc", "mul", ["Xh_x", "c2"])
    m.op("G2", "sub", ["G1", "Xc"])
    m.op("dX4", "mul", ["G2", "r4"], dtype)
    m.op("dX", "reshape", ["dX4"], dtype, shape=m.map)
    m.op("dgamma4", "reduce_sum", ["sg"], dtype, axis=0, keepdim=True)
    m.op("dgamma", "reshape", ["dgamma4"], dtype, shape=(c,))
    m.op("dbeta4", "reduce_sum", ["sb"], dtype, axis=0, keepdim=True)
    m.op("dbeta", "reshape", ["dbeta4"], dtype, shape=(c,))
    outs = ["dX", "dgamma", "dbeta"]
    w = _finish(b, "groupnorm_grad", outs, m.sizes, extra_outputs)
    whole = (sums + m.prims, outs)
    w.plans["layered"] = [(sums, ["sb", "sg", "c1", "c2"]), (list(m.prims), outs)]
    w.plans["fused"] = [whole] if _one_kernel(w, whole) else w.plans["layered"]
    return w


class _Rotary:
    """The angles and the turn that ``rotary`` and its gradient share."""

    def __init__(self, b, batch, heads, kv_heads, n, d, rot, axes, interleaved, packed):
        kv_heads = heads if kv_heads is None else kv_heads
        rot = d if rot is None else rot
        if min(batch, heads, kv_heads, n, d, axes) < 1 or heads % kv_heads:
            raise ValueError("heads must be a positive multiple of kv_heads, and every size positive")
        if rot < 2 or rot % 2 or rot > d:
            raise ValueError("rot must be even, at least 2 and at most d")
        self.b, self.batch, self.heads, self.kv, self.n, self.d, self.rot = b, batch, heads, kv_heads, n, d, rot
        self.pairs, self.axes, self.interleaved, self.packed = rot // 2, axes, interleaved, packed
        self.sizes = dict(batch=batch, heads=heads, kv_heads=kv_heads, n=n, d=d, rot=rot, axes=axes, interleaved=interleaved, packed=packed)
        self.prims, self.reads = [], {}

    def op(self, name, op, ins, dtype="f32", **attrs):
        self.b.op(name, op, ins, dtype, **attrs)
        self.prims.append(name)
        self.reads[name] = ins
        return name

    def fused(self, w, outs):
        """One kernel; where no family takes the results together (neighbouring
        pairs in heads of odd width, which no vector of the rotary kernel holds,
        and results whose heads differ), one for each with what it needs."""
        whole = (list(self.prims), outs)
        if _one_kernel(w, whole):
            return [whole]
        kernels = []
        for o in outs:
            need = {o}
            for p in reversed(self.prims):
                if p in need:
                    need.update(self.reads[p])
            kernels.append(([p for p in self.prims if p in need], [o]))
        return kernels

    def angles(self):
        b = self.b
        b.inp("positions", (self.batch, self.n, self.axes), "f32")
        if self.axes > 1:
            b.inp("axis", (self.pairs,), "f32")
        b.inp("freq", (self.pairs,), "f32")
        if self.axes > 1:
            b.op("places", "reshape", ["positions"], "f32", shape=(self.batch, 1, self.n, 1, self.axes))
            at = self.op("place", "gather", ["places", "axis"])
        else:
            at = "place"
            b.op(at, "reshape", ["positions"], "f32", shape=(self.batch, 1, self.n, 1))
        self.op("co", "cos_mul", [at, "freq"])
        self.op("si", "sin_mul", [at, "freq"])
        if self.interleaved:
            for x in ("co", "si"):
                self.op(x + "_i", "reshape", [x], shape=(self.batch, 1, self.n, self.pairs, 1))

    def _part(self, name, src, first, last):
        """[.., first:last] of the last axis."""
        shape = self.b.g.node_info(self.b.ids[src])[2]
        if (first, last) == (0, shape[-1]):
            return src
        return self.op(name, "slice", [src], self.b.dtype, begin=(0,) * (len(shape) - 1) + (first,), end=shape[:-1] + (last,))

    def turn(self, name, src, heads, back):
        """``name`` = src [batch, heads, n, d] turned by the angles, or by their negatives."""
        p, t = self.pairs, self.b.dtype
        if self.interleaved:
            x = self._part(name + "_t", src, 0, 2 * p)
            x = self.op(name + "_x", "reshape", [x], t, shape=(self.batch, heads, self.n, p, 2))
            one, two, co, si = self._part(name + "_1", x, 0, 1), self._part(name + "_2", x, 1, 2), "co_i", "si_i"
        else:
            one, two, co, si = self._part(name + "_1", src, 0, p), self._part(name + "_2", src, p, 2 * p), "co", "si"
        self.op(name + "_1c", "mul", [one, co])
        self.op(name + "_2s", "mul", [two, si])
        self.op(name + "_a", "add" if back else "sub", [name + "_1c", name + "_2s"], t)
        self.op(name + "_2c", "mul", [two, co])
        self.op(name + "_1s", "mul", [one, si])
        self.op(name + "_b", "sub" if back else "add", [name + "_2c", name + "_1s"], t)
        rest = [self._part(name + "_r", src, 2 * p, self.d)] if self.rot < self.d else []
        ab = [name + "_a", name + "_b"]
        if not self.interleaved:
            return self.op(name, "concat", ab + rest, t, axis=-1)
        both = self.op(name + "_ab", "concat", ab, t, axis=-1)
        flat = self.op(name + "_f" if rest else name, "reshape", [both], t, shape=(self.batch, heads, self.n, 2 * p))
        return self.op(name, "concat", [flat] + rest, t, axis=-1) if rest else flat


def rotary(batch=1, heads=8, kv_heads=None, n=1024, d=64, rot=None, axes=1, interleaved=False, packed=False, dtype="bf16", extra_outputs=()):
    """Rotary positions of queries and keys along one or several axes (time,
    height, width), in one kernel (neighbouring pairs in heads of odd width: one
    for each result).  Pair p of a token's head turns by the angle
    a = positions[b, i, axis[p]] freq[p]:

      (x1, x2) -> (x1 cos a - x2 sin a, x2 cos a + x1 sin a)

    The first ``rot`` (default d) of a head's d dims turn, in rot / 2 pairs:
    dims p and p + rot / 2, or with ``interleaved`` dims 2 p and 2 p + 1; the
    rest stays.  Inputs ``positions`` [batch, n, axes] (any fp32 numbers),
    ``axis`` [rot / 2] (fp32 whole numbers; left out where there is one axis)
    and ``freq`` [rot / 2], radians per position (fp32).  The angle is the exact
    product of its two fp32 factors (up to 2^50), so far positions keep theirs.

    Q [batch, heads, n, d] and K [batch, kv_heads, n, d] give ``Qr`` and ``Kr``;
    ``packed`` takes QKV [batch, n, heads + 2 kv_heads, d] as a projection's
    product leaves it and gives Qr, Kr and V in the layout that ``mha`` reads
    (heads before tokens).  n = 1 is the next token of each sequence."""
    b = _B(dtype)
    a = _Rotary(b, batch, heads, kv_heads, n, d, rot, axes, interleaved, packed)
    if packed:
        b.inp("QKV", (batch, n, a.heads + 2 * a.kv, d))
    else:
        b.inp("Q", (batch, a.heads, n, d))
        b.inp("K", (batch, a.kv, n, d))
    a.angles()
    src, outs = ("Q", "K"), ["Qr", "Kr"]
    if packed:
        first = 0
        for x, h in (("Q", a.heads), ("K", a.kv), ("V", a.kv)):
            a.op(x + "p", "slice", ["QKV"], dtype, begin=(0, 0, first, 0), end=(batch, n, first + h, d))
            a.op(x + "t" if x != "V" else "V", "transpose", [x + "p"], dtype, perm=(0, 2, 1, 3))
            first += h
        src, outs = ("Qt", "Kt"), ["Qr", "Kr", "V"]
    a.turn("Qr", src[0], a.heads, False)
    a.turn("Kr", src[1], a.kv, False)
    w = _finish(b, "rotary", outs, a.sizes, extra_outputs)
    w.plans["fused"] = a.fused(w, outs)
    return w


def rotary_grad(batch=1, heads=8, kv_heads=None, n=1024, d=64, rot=None, axes=1, interleaved=False, packed=False, dtype="bf16", extra_outputs=()):
    """The gradient of ``rotary`` (same arguments): dQr and dKr turned back by the
    same angles, dQ and dK; ``packed`` takes dV too and gives dQKV in the
    projection's layout.  (The turn is orthogonal: its transpose is the turn back.)"""
    b = _B(dtype)
    a = _Rotary(b, batch, heads, kv_heads, n, d, rot, axes, interleaved, packed)
    b.inp("dQr", (batch, a.heads, n, d))
    b.inp("dKr", (batch, a.kv, n, d))
    if packed:
        b.inp("dV", (batch, a.kv, n, d))
    a.angles()
    a.turn("dQ", "dQr", a.heads, True)
    a.turn("dK", "dKr", a.kv, True)
    outs = ["dQ", "dK"]
    if packed:
        for x in ("dQ", "dK", "dV"):
            a.op(x + "t", "transpose", [x], dtype, perm=(0, 2, 1, 3))
        a.op("dQKV", "concat", ["dQt", "dKt", "dVt"], dtype, axis=2)
        outs = ["dQKV"]
    w = _finish(b, "rotary_grad", outs, a.sizes, extra_outputs)
    w.plans["fused"] = a.fused(w, outs)
    return w


# Tensors that one kernel of grad_clip takes: their addresses are kernel
# arguments (8 bytes each, in and out, of the 4 KiB that a launch passes safely).
CLIP_TENSORS = 200


def grad_clip(shapes=((768,), (768, 768)), dtype="bf16", dtypes=None, max_norm=1.0, eps=1e-6, extra_outputs=()):
    """The global norm of many gradients and the gradients clipped by it:

      norm = sqrt(sum over all tensors and elements of G^2),   C_i = G_i min(1, max_norm / (norm + eps))

    Inputs G0, G1, .. of ``shapes`` (and ``dtypes``, default ``dtype`` for all);
    outputs ``norm`` [1] (fp32) and C0, C1, .. of the inputs' shapes and types.
    C_i may share the memory of its own G_i (every kernel reads an element before
    it writes it), as long as no two gradients lie in one memory.  Every tensor
    begins on a multiple of 16 bytes, as for every plan (``KORCH_E_ALIGN``
    otherwise): in one flat buffer of many gradients, pad their sizes to that.  The sum of
    squares is held in 64 bits by the fused plan, so neither 1e30 nor 1e-30
    leaves its range, and taken in a fixed order.
    A norm that is not a number leaves none in any gradient; an infinite one
    leaves zeros, and NaN where the gradient itself is infinite."""
    shapes = [tuple(int(x) for x in s) for s in shapes]
    dtypes = [dtype] * len(shapes) if dtypes is None else list(dtypes)
    if not shapes or len(dtypes) != len(shapes):
        raise ValueError("one shape at least, and a type for each")
    if not (_F32_MIN <= max_norm <= _F32_MAX and 0 <= eps <= _F32_MAX):
        raise ValueError("max_norm must be a positive normal fp32 number, eps finite in fp32 and not negative")
    b = _B(dtype)
    k = len(shapes)
    for i, (s, t) in enumerate(zip(shapes, dtypes)):
        if not s or min(s) < 1 or len(s) > 8:
            raise ValueError(f"shape {s} of gradient {i}: one to eight positive sizes")
        b.inp(f"G{i}", s, t)
    parts = [list(range(i, min(i + CLIP_TENSORS, k))) for i in range(0, k, CLIP_TENSORS)]

    def root_of_squares(name, tensors, c):
        """``name`` [1] = the root of the sum of the squares of tensors (name, type, elements); the kernel's primitives."""
        prims = []
        for x, t, count in tensors:
            b.op(f"{x}_f{c}", "reshape", [x], t, shape=(count, 1))
            b.op(f"{x}_q{c}", "square", [f"{x}_f{c}"], "f32")
            b.op(f"{x}_s{c}", "reduce_sum", [f"{x}_q{c}"], "f32", axis=0, keepdim=False)
            prims += [f"{x}_q{c}", f"{x}_s{c}"]
        total = prims[-1]
        if len(tensors) > 1:
            b.op(name + "_c", "concat", prims[1::2], "f32", axis=0)
            b.op(name + "_r", "reshape", [name + "_c"], "f32", shape=(len(tensors), 1))
            b.op(name + "_t", "reduce_sum", [name + "_r"], "f32", axis=0, keepdim=False)
            prims += [name + "_c", name + "_r", name + "_t"]
            total = name + "_t"
        b.op(name, "sqrt", [total], "f32")
        return prims + [name]

    tensors = [(f"G{i}", t, math.prod(s)) for i, (s, t) in enumerate(zip(shapes, dtypes))]
    kernels = []
    if len(parts) > 1:  # norms of parts, whose norm is the whole one
        for j, part in enumerate(parts):
            kernels.append((root_of_squares(f"norm{j}", [tensors[i] for i in part], ""), [f"norm{j}"]))
        tensors = [(f"norm{j}", "f32", 1) for j in range(len(parts))]
    tail = root_of_squares("norm", tensors, "")
    b.op("norm_e", "add", ["norm"], "f32", scalar=eps)
    b.op("limit", "fill", [], "f32", shape=(1,), scalar=max_norm)
    b.op("ratio", "div", ["limit", "norm_e"], "f32")
    b.op("below", "gt", ["ratio"], "f32", scalar=1.0)
    b.op("one", "fill", [], "f32", shape=(1,), scalar=1.0)
    b.op("factor", "select", ["below", "one", "ratio"], "f32")
    tail += ["norm_e", "limit", "ratio", "below", "one", "factor"]
    for i in range(k):
        b.op(f"C{i}", "mul", [f"G{i}", "factor"], dtypes[i])
    w = _finish(b, "grad_clip", ["norm"] + [f"C{i}" for i in range(k)], dict(shapes=shapes, dtypes=dtypes, max_norm=max_norm), extra_outputs)
    kernels.append((tail, ["norm", "factor"]))
    w.plans["fused"] = kernels + [([f"C{i}" for i in part], [f"C{i}" for i in part]) for part in parts]
    return w


def layout_probe(op, dtype, shapes, **attrs):
    """A graph of one layout primitive (transpose, slice, pad or concat) on
    graph inputs of the given shapes; a concat whose ``fill`` attribute is set
    appends a constant operand of that value (as the product-merging
    transformation does).  Its unfused plan is one kernel per primitive, the
    same generated kernels as the layout nodes of a workload's unfused plan."""
    b = _B(dtype)
    names = []
    for i, sh in enumerate(shapes):
        b.inp(f"in{i}", sh)
        names.append(f"in{i}")
    fill = attrs.pop("fill", None)
    if fill is not None:
        last = list(shapes[-1])
        last[attrs.get("axis", -1)] = 1
        b.op("ones", "fill", [], shape=tuple(last), scalar=fill)
        names.append("ones")
    if op == "pad":
        attrs = dict(begin=attrs["lo"], end=attrs["hi"], pad_value=attrs.get("value", 0.0))
    b.op("out", op, names, **attrs)
    return _finish(b, f"layout_{op}", ["out"], dict(shapes=[tuple(s) for s in shapes]))


BUILDERS = {"attention": attention, "mlp": mlp, "sra": sra, "conv": conv, "linattn": linattn, "instnorm": instnorm}
# Operators of a transformer layer's training and serving, built by name like the workloads.
OPERATORS = {"layernorm": layernorm, "layernorm_grad": layernorm_grad, "mha": mha, "mha_grad": mha_grad, "groupnorm": groupnorm,
             "groupnorm_grad": groupnorm_grad, "rotary": rotary, "rotary_grad": rotary_grad, "grad_clip": grad_clip}


def rewritten(w: Workload, rules=None):
    """The workload's graph after the primitive-graph transformations
    (korch_graph_rewrite), with the same input and output names; returns
    (workload, number of rule applications).  It has no hand-written plans."""
    from ._abi import RW_ALL
    g2, n = w.graph.rewrite(RW_ALL if rules is None else rules)
    ids = dict(zip(w.input_names, g2.inputs()))
    ids.update(zip(w.output_names, g2.outputs()))
    return Workload(w.name, w.dtype, g2, ids, list(w.input_names), list(w.output_names), sizes=dict(w.sizes)), n


def moments_plan(w: Workload):
    """Two kernels for an InstanceNorm whose graph went through the
    split-moments transformation (its variance squares m - X, a node of its
    own): the column moments {mean, m - X, square, variance, + eps, rsqrt}
    exporting the mean and the reciprocal deviation (one pass over X), then
    everything else (X - m recomputed, the normalization and what follows).
    None when the graph has no such variance."""
    g = w.graph
    n = g.num_nodes()
    op = {v: g.node_info(v)[0] for v in range(n)}
    ins = {v: g.node_inputs(v) for v in range(n) if op[v] != "input"}
    cons = {v: [c for c in ins if v in ins[c]] for v in range(n)}
    for var in (v for v in range(n) if op[v] == "reduce_mean"):
        sq = ins[var][0]
        if op[sq] != "square" or op[ins[sq][0]] != "sub":
            continue
        dc = ins[sq][0]
        mu, x = ins[dc]
        if op[mu] != "reduce_mean" or ins[mu][0] != x:
            continue
        k0 = {mu, dc, sq, var}
        if op[x] == "reshape":
            k0.add(x)
        last = var
        while len(cons[last]) == 1 and op[cons[last][0]] in ("add", "rsqrt") and g.node_info(cons[last][0])[2] == g.node_info(var)[2]:
            last = cons[last][0]
            k0.add(last)
        prims = [v for v in range(n) if op[v] != "input"]
        return [(sorted(k0), sorted([mu, last])),
                (sorted(v for v in prims if v not in k0), sorted(o for o in g.outputs() if o not in k0))]
    return None


def plan_record(w: Workload, kernels, rules=0):
    """JSON-able record of a plan of ``w`` (or of its rewritten graph when
    ``rules`` is non-zero): node ids, plus names where the workload names them."""
    from ._abi import RW_LAYOUT_VARIANTS
    names = {v: k for k, v in w.ids.items()} if not rules else {}
    label = "original" if not rules else "layout variants" if rules == RW_LAYOUT_VARIANTS else "rewritten"
    return {"graph": label, "rules": int(rules),
            "kernel_ids": [[list(map(int, p)), list(map(int, o))] for p, o in kernels],
            "kernels": [[[names.get(v, f"#{v}") for v in p], [names.get(v, f"#{v}") for v in o]] for p, o in kernels]}


def plan_from_record(w: Workload, rec):
    """(workload, kernels) of a record written by plan_record."""
    if rec.get("rules"):
        w, _ = rewritten(w, rec["rules"])
    return w, [(list(p), list(o)) for p, o in rec["kernel_ids"]]


def build(workload: str, **sizes) -> Workload:
    return (BUILDERS.get(workload) or OPERATORS[workload])(**sizes)
