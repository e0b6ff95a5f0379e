"""examples/answer.py, small: the compression loop, pages and attention together, checked step by step."""
import importlib.util
import os

import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import paged as R

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("answer", os.path.join(ROOT, "examples", "answer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("fmt,step", [("bf16", 2.0**-7), ("fp8", 2.0**-4), ("fp4", 2.0**-2)])
def test_runs_and_reads_back(fmt, step):
    m = example()
    outputs, back, kept = m.run(fmt, layers=2, kv_heads=2, q_heads=6, D=64, grid=(4, 4), cap=128, budget=64, recent=1, frames=20,
                                question=9, tokens=3, page_rows=12)
    assert all(bool(torch.isfinite(o).all()) and float(o.abs().max()) > 0 for o in outputs) and len(outputs) == 4
    # an element comes back within the format's half steps of its block's largest (both roundings, a turn there and back)
    for x, y in zip(back, kept):
        y = y.float()
        assert float((x.float() - y).abs().max()) <= step * 2 ** 0.5 * float(y.abs().max()) * 2


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_a_layer_is_plain_attention_over_what_was_written(fmt):
    """The example's layer step against attention in 64 bits over the pool's stored rows, question and tokens."""
    m = example()
    L, H, A, D, n = 2, 2, 6, 64, 45
    a = m.Answers(1, L, H, A, D, 80, 12, m.FORMATS[fmt], 9, "cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    K, V = (torch.randn((1, L, H, 60, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    a.fill(K, V, n)
    at = n
    for M in (9, 1, 1):
        q, k, v = (torch.randn((1, h, M, D), generator=g, device="cuda").bfloat16() for h in (A, H, H))
        out = a.layer(1, q, k, v, at, torch.empty_like(q))
        qr = m.rotated(q, a.rotary, at)
        want, _, spread, size = R.attend(a.pool, fmt, a.table, [at + M], [at], 1, qr, D ** -0.5)
        assert bool(((out.double() - want).abs() <= R.tolerance(fmt, D, spread, size)).all())
        at += M
    assert a.errors() == 0
    # the new tokens' own rows are in the pages: the last key, turned
    last = R.rows_of(a.pool, fmt, a.table, 0, 1, 0)[at - 1]
    turned = R.turned(k[:, None].double(), a.rotary, torch.tensor([[at - 1]], device="cuda"))[0, 0, 0, 0]
    assert float((last - turned).abs().max()) <= {"bf16": 2.0**-7, "fp8": 2.0**-3}[fmt] * float(turned.abs().max())
    assert ipv.ipv_read_device_errors(a.write_ws) == 0
