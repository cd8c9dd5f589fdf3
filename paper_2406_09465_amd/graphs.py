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
OPERATORS = {"layernorm": layernorm, "layernorm_grad": layernorm_grad, "mha": mha, "mha_grad": mha_grad}


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
