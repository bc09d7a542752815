"""Stacked-layer decode: L sparse-FFN layers chained by pre-norm residuals,

    u_l = bf16(RMSNorm(x_l))   (eps 1e-5, norm weight 1)
    x_{l+1} = x_l + FFN_l(u_l)  (fp32 residual stream)

as in the 32-layer LLaMA-3-8B-shaped decode workload.  With `norms` the norm
is layer norm with each layer's weight and bias (GELU-MLP blocks); with `topk`
every token takes a fixed number of experts by the handles' routers
(prunepath_route_topk) instead of the budget tau.  This module only allocates
the buffers and enqueues the C-ABI calls (prunepath_residual_rmsnorm or
prunepath_residual_layernorm, prunepath_ffn_decode or prunepath_route_topk and
prunepath_ffn_decode_routed) on one stream; every step of the computation runs
in the HIP library.  One step can be captured once in a HIP graph and replayed.

Buffers kept per layer (so that each layer can be checked on its own):
  xs  [L+1, T, d] fp32   residual entering layer l (xs[L] = step output)
  us  [L, T, d]   bf16   normalised layer inputs
  ys  [L, T, d]   fp32   FFN outputs
  idx [L, T, E], cnt [L, T]  selections; with `topk` idx [L, T, k] and
  gate_w [L, T, k] fp32, and no cnt
"""
from . import _lib as pp


class DecodeStack:
    """norms: one pair (weight, bias) per layer, each a [d] fp32 tensor or None (1 and 0),
    or None for RMSNorm.  topk: a dict of prunepath_route_topk's k and, unless the defaults
    do, n_groups, top_groups, scale, flags, and sel_bias, a list of one [E] fp32 tensor (or
    None) per layer, or None for no biases; tau is not used then."""

    def __init__(self, handles, d, E, T, tau, eps=1e-5, norms=None, topk=None):
        self.handles = list(handles)
        self.L = len(self.handles)
        self.d, self.E, self.T, self.tau, self.eps = d, E, T, float(tau), float(eps)
        self.norms = None if norms is None else list(norms)
        if self.norms is not None and len(self.norms) != self.L:
            raise ValueError("norms: %d pairs for %d layers" % (len(self.norms), self.L))
        for n in self.norms or ():
            if n is None or len(n) != 2:
                raise ValueError("norms: a layer's entry that is not a pair (weight, bias)")
            if any(a is not None and a.numel() != d for a in n):
                raise ValueError("norms: a weight or bias that is not [%d]" % d)
        self.topk = None
        if topk is not None:
            self.topk = dict(n_groups=1, top_groups=1, scale=1.0, flags=0,
                             sel_bias=[None] * self.L)
            unknown = set(topk) - set(self.topk) - {"k"}
            if unknown or "k" not in topk:
                raise ValueError("topk: %s" % (sorted(unknown) or "no k"))
            self.topk.update(topk)
            if self.topk["sel_bias"] is None:
                self.topk["sel_bias"] = [None] * self.L
            if len(self.topk["sel_bias"]) != self.L:
                raise ValueError("topk: %d selection biases for %d layers"
                                 % (len(self.topk["sel_bias"]), self.L))
            if any(b is not None and b.numel() != E for b in self.topk["sel_bias"]):
                raise ValueError("topk: a selection bias that is not [%d]" % E)
        import torch
        dev = "cuda"
        self.x_in = torch.zeros((T, d), dtype=torch.float32, device=dev)
        self.xs = torch.zeros((self.L + 1, T, d), dtype=torch.float32, device=dev)
        self.us = torch.zeros((self.L, T, d), dtype=torch.int16, device=dev)
        self.ys = torch.zeros((self.L, T, d), dtype=torch.float32, device=dev)
        if self.topk is None:
            self.idx = torch.zeros((self.L, T, E), dtype=torch.int32, device=dev)
            self.cnt = torch.zeros((self.L, T), dtype=torch.int32, device=dev)
        else:
            k = self.topk["k"]
            self.idx = torch.zeros((self.L, T, k), dtype=torch.int32, device=dev)
            self.gate_w = torch.zeros((self.L, T, k), dtype=torch.float32, device=dev)
        self.graph = None

    def set_input(self, x0):
        """x0: [T, d] fp32 tensor (any device) -> the first residual."""
        self.x_in.copy_(x0)

    def _norm(self, x, y, x_out, l, stream):
        """x_out = x + y and layer l's input (none behind the last layer)."""
        if l == self.L or self.norms is None:
            pp.prunepath_residual_rmsnorm(x, y, x_out, self.T, self.d, self.eps,
                                          None if l == self.L else self.us[l], stream=stream)
        else:
            w, b = self.norms[l]
            pp.prunepath_residual_layernorm(x, y, x_out, self.T, self.d, self.eps, w, b,
                                            self.us[l], stream=stream)

    def _ffn(self, h, l, stream):
        if self.topk is None:
            pp.prunepath_ffn_decode(h, self.us[l], self.T, self.tau, None, self.ys[l],
                                    self.idx[l], self.cnt[l], stream=stream)
            return
        t = self.topk
        pp.prunepath_route_topk(h, self.us[l], self.T, None, t["k"], t["n_groups"],
                                t["top_groups"], t["sel_bias"][l], t["scale"], t["flags"],
                                self.idx[l], self.gate_w[l], stream=stream)
        pp.prunepath_ffn_decode_routed(h, self.us[l], self.T, t["k"], self.idx[l], self.gate_w[l],
                                       self.ys[l], stream=stream)

    def enqueue(self, stream=None):
        """Enqueue one step (all L layers) on `stream` (default: current)."""
        self._norm(self.x_in, None, self.xs[0], 0, stream)
        for l, h in enumerate(self.handles):
            self._ffn(h, l, stream)
            self._norm(self.xs[l], self.ys[l], self.xs[l + 1], l + 1, stream)

    def capture(self):
        """Capture one step in a HIP graph (call after an eager warm-up step)."""
        import torch
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            self.enqueue()
        self.graph = g
        return g

    def replay(self):
        self.graph.replay()

    @property
    def output(self):
        return self.xs[self.L]
