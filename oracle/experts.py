"""Decoder whose MLP is a mixture of experts: the oracle's definition (test
infrastructure only).

From layer ``moe.first_layer`` on, a row h of the normalised MLP input goes
through the experts its router chooses:

    l = Wr h;  s = softmax(l) or sigmoid(l);  c = s + bias
    a group of experts counts the sum of its two best c; the top_groups best
    groups stay, and of their experts the top_k best c are chosen (lower index
    on ties);  w = s of the chosen, over their sum if renorm, times scale
    mlp(h) = out_scale * N(sum_e w_e Wd_e (silu(Wg_e h) * (Wu_e h)))

with N the RMSNorm with the layer's own gain if post_norm, else nothing.
"""

import numpy as np

from .model import OracleModel, rms_norm, silu


class OracleExpertsModel(OracleModel):
    """``moe``: an object with the fields of workloads.configs.MoeConfig.
    ``margin[t]`` is, for row t of the last forward, the smallest distance over
    its layers from the last chosen expert (or group) to the first one left
    out: implementations whose scores differ by less choose alike."""

    def __init__(self, cfg, weights, moe, dtype=np.float64):
        super().__init__(cfg, weights, dtype=dtype)
        self.moe = moe
        self.margin = None

    def choose(self, l, bias):
        """(expert, weight) pairs of one row of router logits, and its margin."""
        m = self.moe
        E = m.n_experts
        if m.score == "softmax":
            z = np.exp(l - l.max())
            s = z / z.sum()
        else:
            s = 1.0 / (1.0 + np.exp(-l))
        c = s + bias
        S = E // m.n_groups
        value = [np.sort(c[g * S:(g + 1) * S])[-2:].sum() for g in range(m.n_groups)]
        best = sorted(value, reverse=True)
        margin = best[m.top_groups - 1] - best[m.top_groups] if m.top_groups < m.n_groups else np.inf
        keep = sorted(range(m.n_groups), key=lambda g: (-value[g], g))[:m.top_groups]
        order = sorted((e for e in range(E) if e // S in keep), key=lambda e: (-c[e], e))
        if len(order) > m.top_k:
            margin = min(margin, c[order[m.top_k - 1]] - c[order[m.top_k]])
        chosen = order[:m.top_k]
        total = sum(s[e] for e in chosen) if m.renorm else 1.0
        return [(e, m.scale * s[e] / total) for e in chosen], margin

    def mlp(self, h, layer):
        if layer < self.moe.first_layer:
            return super().mlp(h, layer)
        p = f"layers.{layer}."
        logits = self.linear(h, p + "router")
        bias = self.w(p + "router_bias") if p + "router_bias" in self.weights else np.zeros(self.moe.n_experts)
        g, u, d = self.w(p + "experts_gate"), self.w(p + "experts_up"), self.w(p + "experts_down")
        out = np.zeros_like(h)
        if layer == self.moe.first_layer:
            self.margin = np.full(h.shape[0], np.inf)
        for t in range(h.shape[0]):
            chosen, margin = self.choose(logits[t], bias)
            self.margin[t] = min(self.margin[t], margin)
            for e, w in chosen:
                out[t] += w * (d[e] @ (silu(g[e] @ h[t]) * (u[e] @ h[t])))
        if self.moe.post_norm:
            out = rms_norm(out, self.w(p + "post_norm"), self.cfg.rms_eps)
        return self.moe.out_scale * out
