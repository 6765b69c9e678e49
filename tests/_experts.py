"""Decoders with expert layers for the tests (not collected by pytest)."""

import numpy as np

from workloads import ModelConfig, make_weights
from workloads.configs import MoeConfig
from workloads.weights import f32_to_bf16_bits

# widths of the tiny decoder; a dense layer, then two with experts
SMALL = ModelConfig("experts-small", 3, 256, 4, 4, 64, 512, 4096, 1.0e4, max_pos=4096)
SMALL_MOE = MoeConfig(n_experts=16, top_k=4, ffn_dim=96, first_layer=1)
# grouped queries; every layer with experts in groups, sigmoid scores, a balance bias, a post norm
GROUPED = ModelConfig("experts-grouped", 2, 512, 8, 2, 128, 1024, 4096, 5.0e5, max_pos=4096)
GROUPED_MOE = MoeConfig(n_experts=40, top_k=6, ffn_dim=160, score="sigmoid", n_groups=5, top_groups=3, scale=2.5,
                        out_scale=0.5, post_norm=True)


def weights(cfg, moe, seed=7, bias=False):
    """Canonical tensors; routers and experts are larger than the other matrices
    so that the choice is clear and the experts count."""
    w = make_weights(cfg, seed=seed, gain_std=0.1)
    rng = np.random.default_rng([seed, 99])
    D, F, E = cfg.d_model, moe.ffn_dim, moe.n_experts
    bits = lambda std, *s: f32_to_bf16_bits(std * rng.standard_normal(s, dtype=np.float32))
    for l in range(moe.first_layer, cfg.n_layers):
        p = f"layers.{l}."
        for n in ("wg", "wu", "wd"):
            del w[p + n]
        w[p + "router"] = bits(0.1, E, D)
        w[p + "experts_gate"], w[p + "experts_up"] = bits(0.06, E, F, D), bits(0.06, E, F, D)
        w[p + "experts_down"] = bits(0.06, E, D, F)
        if bias:
            w[p + "router_bias"] = bits(0.1, E)
        if moe.post_norm:
            w[p + "post_norm"] = f32_to_bf16_bits(0.3 + 0.1 * rng.standard_normal(D, dtype=np.float32))
    return w
