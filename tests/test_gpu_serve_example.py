"""The example that serves a fitted block: every step's output against the same steps in float64, from the codes on."""
import math
import os
import subprocess
import sys

import pytest
import torch

import serve_ref as R
from workloads import GPT2_SMALL, MISTRAL_7B

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("shape,bits,cache_bits,prefix,prompts,window", [
    (GPT2_SMALL, 4, 8, 128, [5, 1, 40], 0),
    (GPT2_SMALL, 8, 4, 0, [9, 64, 1, 2], 30),
    (MISTRAL_7B, 3, 8, 64, [3, 17], 0),
])
def test_steps(shape, bits, cache_bits, prefix, prompts, window):
    from examples.serve_block import serve

    n_seqs, steps = len(prompts), 5
    block, seqs, log, _ = serve(shape, bits, cache_bits, n_seqs, prefix, prompts, steps, window=window, keep=True)
    assert len(log) == steps + 1 + (prefix > 0)
    hq, hkv, dh = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    past = [[] for _ in range(n_seqs)]  # (k, v) of every step, float64 [n, hkv, dh]
    for at, (x, starts, lens, out) in enumerate(log):
        qkv = R.linear(x, block.codes, block.scales, torch.float16).float().view(-1, hq + 2 * hkv, dh)
        n = [starts[i + 1] - starts[i] for i in range(len(starts) - 1)]
        pos = torch.cat([torch.arange(e - m, e) for m, e in zip(n, lens)]).cuda()
        turned = R.rotate(qkv[:, :hq + hkv], block.rope[0][pos], block.rope[1][pos]) if block.rope else qkv[:, :hq + hkv]
        q = turned[:, :hq].half().double()
        (kc, ks), (vc, vs) = R.quantize_rows(turned[:, hq:], cache_bits), R.quantize_rows(qkv[:, hq + hkv:], cache_bits)
        k, v = kc * ks.double()[..., None], vc * vs.double()[..., None]
        for b, (m, length) in enumerate(zip(n, lens)):
            rows = slice(starts[b], starts[b] + m)
            # (the prefix is one sequence's step: all have it)
            for keep in (past if prefix and at == 0 else [past[b]]):
                keep.append((k[rows], v[rows]))
            kk, vv = (torch.cat([t[i] for t in past[b]]) for i in (0, 1))
            assert kk.shape[0] == length
            o, _, mag = R.attention(q[rows], kk, vv, window, 1 / math.sqrt(dh))
            # a weight's fp16 rounding (2^-11) and exponent, sums of `length` terms, the output's half ulp
            tol = (2.0 ** -11 + 2.0 ** -16) * mag + length * 2.0 ** -25 * vv.abs().max() + 2.0 ** -11 * o.abs() + 2.0 ** -25
            err = (out[rows].double() - o).abs()
            assert bool((err <= tol).all()), (at, b, (err / tol).max().item())


def test_runs_as_a_command():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "serve_block.py"), "--shape", "gpt2", "--seqs", "3",
                        "--prefix", "64", "--steps", "3", "--cache-bits", "4"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "decode step" in r.stdout and "finite: True" in r.stdout
