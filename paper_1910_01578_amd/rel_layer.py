"""A placement layer with positions, from the layer operators of gdp.py.

The layer of Section 3.2 has no positional terms; this one adds a learned
relative position bias (the node order is the order of the sequence) and may be
causal:
  Z  = LN1(X + MHA(X W_qkv^T + b_qkv; memory, bias) W_o^T + b_o)
  X' = LN2(Z + W_2 ReLU(W_1 Z + b_1) + b_2)
The cached memory passes a gradient here (all of a graph's rows are inputs of
one call).  Every step runs in the library's kernels.
"""
from __future__ import annotations

from typing import Dict

from . import gdp

#: The layer's weights: gdp_placer_layer's without FiLM, and the bias table
#: [heads, buckets].  w_qkv stacks q [heads * d_head], k and v [kv_heads * d_head].
FIELDS = ("w_qkv", "b_qkv", "w_o", "b_o", "ln1_g", "ln1_b", "w_1", "b_1", "w_2", "b_2", "ln2_g", "ln2_b", "rel_table")


class RelPlacerLayer:
    """One layer for the batch of graphs of `attention` (a gdp.RelAttention whose queries are all positions) and
    `weights` (a tensor per name of FIELDS, in the activations' dtype)."""

    def __init__(self, attention: gdp.RelAttention, weights: Dict):
        missing = [n for n in FIELDS if n not in weights]
        if missing:
            raise gdp.GdpError(gdp.GDP_E_INVALID_ARG, f"the layer has no {', '.join(missing)}")
        if attention.queries is not None or (attention.starts != attention.lengths.cumsum() - attention.lengths).any():
            raise gdp.GdpError(gdp.GDP_E_INVALID_ARG, "the attention's queries and keys are not the same rows")
        self.attention, self.w = attention, dict(weights)

    def _split(self, qkv):
        a = self.attention.heads * self.attention.d_head
        b = a + self.attention.kv_heads * self.attention.d_head
        return qkv[:, :a], qkv[:, a:b], qkv[:, b:]

    def forward(self, x, key_mask=None, stream=None):
        """x [rows, d]; returns (X' [rows, d], what backward needs)."""
        w = self.w
        qkv = gdp.fc(x, w["w_qkv"], w["b_qkv"], stream=stream)
        o, lse = self.attention.forward(*self._split(qkv), w["rel_table"], key_mask=key_mask, stream=stream)
        y = gdp.fc(o, w["w_o"], w["b_o"], stream=stream)
        z, h1 = gdp.layer_norm(y, w["ln1_g"], w["ln1_b"], residual=x, keep_sum=True, stream=stream)
        a = gdp.fc(z, w["w_1"], w["b_1"], act="relu", stream=stream)
        y = gdp.fc(a, w["w_2"], w["b_2"], stream=stream)
        out, h2 = gdp.layer_norm(y, w["ln2_g"], w["ln2_b"], residual=z, keep_sum=True, stream=stream)
        return out, {"x": x, "qkv": qkv, "o": o, "lse": lse, "h1": h1, "z": z, "a": a, "h2": h2, "key_mask": key_mask}

    def backward(self, dout, kept, stream=None):
        """(dx, {name: gradient in fp32}) for dL/dX'."""
        w, g, k = self.w, {}, kept
        dh2, g["ln2_g"], g["ln2_b"] = gdp.layer_norm_backward(k["h2"], w["ln2_g"], dout, stream=stream)
        da, g["w_2"], g["b_2"] = gdp.fc_backward(dh2, k["a"], w["w_2"], stream=stream)
        dz, g["w_1"], g["b_1"] = gdp.fc_backward(da, k["z"], w["w_1"], act="relu", act_out=k["a"], dx_add=dh2,
                                                 stream=stream)
        dh1, g["ln1_g"], g["ln1_b"] = gdp.layer_norm_backward(k["h1"], w["ln1_g"], dz, stream=stream)
        do, g["w_o"], g["b_o"] = gdp.fc_backward(dh1, k["o"], w["w_o"], stream=stream)
        dqkv = gdp._placed(k["x"], stream, lambda _: gdp._t.empty_like(k["qkv"]))
        *_, g["rel_table"] = self.attention.backward(do, *self._split(k["qkv"]), w["rel_table"], k["o"], k["lse"],
                                                     key_mask=k["key_mask"], out=self._split(dqkv), stream=stream)
        dx, g["w_qkv"], g["b_qkv"] = gdp.fc_backward(dqkv, k["x"], w["w_qkv"], dx_add=dh1, stream=stream)
        return dx, g
