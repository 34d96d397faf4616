"""The example of a decoder with a dense and a latent layer over one page table, against the dense layer's plain form in 64 bits."""
import math
import os
import sys

import pytest
import torch

from dense_ref import F64, attend_fast, rotate

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def test_dense_and_latent_layers_share_a_page_table():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import dense_and_latent_layers as example
    finally:
        sys.path.pop(0)
    r = example.run()
    dense, hq, hkv, d = r["dense"], r["dense"].hq, r["dense"].hkv, r["dense"].d
    w, inv = dense.w_qkv.cpu().to(F64), dense.inv_freq.cpu()
    steps, a1, a2 = len(r["tokens"]), 0, 0
    for b, (n1, n2) in enumerate(zip(r["first"], r["second"])):
        x = torch.cat([r["x1"][a1:a1 + n1], r["x2"][a2:a2 + n2]] + [t[b:b + 1] for t in r["tokens"]]).cpu().to(F64)
        y = (x @ w).view(-1, hq + 2 * hkv, d)
        pos = torch.arange(y.shape[0])
        q, k, v = rotate(y[:, :hq], pos, inv), rotate(y[:, hq:hq + hkv], pos, inv), y[:, hq + hkv:]
        want, size = attend_fast(q, k, v, pos, 1.0 / math.sqrt(d))
        got = torch.cat([r["prompt"][a1:a1 + n1], r["more"][a2:a2 + n2]] + [t[b].reshape(1, -1) for t in r["dense_outs"]]).cpu().to(F64).view(-1, hq, d)
        # q, k, v and the output are rounded to bf16, scores of about 1 then carry 2 * 2^-8 relative and the weights as much: 2^-5 of
        # the mean of |v| is eight half steps
        assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -5 * size + 2.0 ** -8).all(), b
        a1, a2 = a1 + n1, a2 + n2
    assert dense.lens.tolist() == [n1 + n2 + steps for n1, n2 in zip(r["first"], r["second"])]
    # the latent layer: a step's output is the weighted mean of reconstructed values, never zero or a non-number, and differs by token
    for t in r["latent_outs"]:
        assert torch.isfinite(t).all() and (t != 0).any(-1).all()
    assert not torch.equal(r["latent_outs"][0], r["latent_outs"][1])
    example.close(r)
