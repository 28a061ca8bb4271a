"""A fitted attention block as a server runs it: prompts behind a shared prefix, then one token a step.

    python examples/serve_block.py [--shape mistral|gpt2] [--bits 4] [--cache-bits 8] [--seqs 64] [--prefix 1024] [--steps 64]

The joint weight [W_Q | W_K | W_V] is quantised with one scale per output channel (group_size = d_model), as the
scale fit leaves it. From then on the block lives on its codes: a step is the projection in 8-bit integers, the
rotation with the new keys and values into a paged quantised cache, and attention over that cache. The steps of
single tokens are captured in one CUDA graph: page tables, lengths, slots and positions are device buffers that the
host fills between two replays.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_34866_gb300 as J  # noqa: E402
from workloads import GPT2_SMALL, MISTRAL_7B, make_w  # noqa: E402


class Sequences:
    """Pages and lengths of a batch of sequences that begin with the same prefix (host bookkeeping)."""

    def __init__(self, n_seqs: int, prefix: int, max_len: int, page_tokens: int):
        if prefix % page_tokens:
            raise ValueError("the shared prefix must fill whole pages")
        self.page, self.prefix = page_tokens, prefix
        same, per = prefix // page_tokens, -(-max_len // page_tokens)
        own = torch.arange(n_seqs * (per - same), dtype=torch.int32).view(n_seqs, -1) + same
        self.pages = torch.cat((torch.arange(same, dtype=torch.int32).expand(n_seqs, same), own), 1).contiguous()
        self.n_pages = same + n_seqs * (per - same)
        self.lens = torch.full((n_seqs,), prefix, dtype=torch.int32)

    def append(self, counts):
        """The next counts[b] tokens of every sequence: (slots int64, positions int32), sequence by sequence."""
        counts = torch.as_tensor(counts, dtype=torch.int64)
        b = torch.repeat_interleave(torch.arange(counts.numel()), counts)
        pos = torch.arange(b.numel()) - (counts.cumsum(0) - counts)[b] + self.lens[b]
        self.lens += counts.int()
        return self.pages[b, pos // self.page].long() * self.page + pos % self.page, pos.int()


class ServedBlock:
    """Codes, scales, cache and workspaces of one block. `calls`: the kinds of steps it will take, each as (sequences,
    rows, the longest sequence's rows, shared tokens)."""

    def __init__(self, shape, W, bits: int, cache_bits: int, page_tokens: int, n_pages: int, calls, max_len: int,
                 shared_len: int = 0, window: int = 0):
        self.shape, self.max_len, self.shared_len, self.window = shape, max_len, shared_len, window
        desc = J.desc_from_shape(shape, shape.d_model)
        scales = torch.empty((shape.d_out, 1), device=W.device)
        self.codes = torch.empty((shape.d_out, shape.d_model), dtype=torch.int8, device=W.device)
        J.jab_init_scales(desc, bits, 1, W, scales)
        J.jab_quantize(desc, bits, W, scales, codes=self.codes)
        self.scales = scales.view(-1)
        self.cache = J.KvCache(shape.n_kv_heads, shape.head_dim, cache_bits, page_tokens, n_pages, device=W.device)
        self.rope = None
        if shape.use_rope:
            self.rope = tuple(torch.empty((max_len, shape.head_dim // 2), device=W.device) for _ in range(2))
            J.jab_rope_table(*self.rope, shape.rope_theta)
        hq, dh, max_tokens = shape.n_q_heads, shape.head_dim, max(call[1] for call in calls)
        self.qkv = torch.empty((max_tokens, shape.d_out), dtype=torch.float16, device=W.device)
        self.q = torch.empty((max_tokens, hq * dh), dtype=torch.float16, device=W.device)
        self.out = torch.empty_like(self.q)
        self.ws_linear = torch.empty(J.jab_quantized_linear_workspace_size(max_tokens, shape.d_out, shape.d_model),
                                     dtype=torch.uint8, device=W.device)
        sizes = [J.jab_kv_attention_workspace_size(self.cache, n_seqs, n_tokens, hq, max_q, max_len, shared)
                 for n_seqs, n_tokens, max_q, shared in calls]
        self.ws_attn = torch.empty(max(sizes), dtype=torch.uint8, device=W.device)

    def step(self, x, slots, positions, q_start, pages, seq_lens, max_q_len: int, shared_len=None):
        """Attention output [n, n_q_heads, head_dim] of the rows x [n, d_model] (fp16 or bf16), whose keys and
        values go to `slots` first."""
        n, hq, dh = x.shape[0], self.shape.n_q_heads, self.shape.head_dim
        qkv, q, out = self.qkv[:n], self.q[:n], self.out[:n].view(n, hq, dh)
        J.jab_quantized_linear(x, self.codes, self.scales, qkv, self.ws_linear)
        J.jab_kv_write(self.cache, qkv, hq, slots, q_out=q, positions=positions if self.rope else None, rope=self.rope)
        J.jab_kv_attention(self.cache, q.view(n, hq, dh), q_start, pages, seq_lens, out, self.ws_attn, max_q_len,
                           self.max_len, shared_len=self.shared_len if shared_len is None else shared_len, window=self.window)
        return out


class Decoder:
    """Steps of one token a sequence, as one captured graph over static buffers."""

    def __init__(self, block: ServedBlock, seqs: Sequences, device):
        n = seqs.lens.numel()
        self.block, self.seqs = block, seqs
        self.x = torch.zeros((n, block.shape.d_model), dtype=torch.float16, device=device)
        self.q_start = torch.arange(n + 1, dtype=torch.int32, device=device)
        self.pages = seqs.pages.to(device)
        # slots, positions, lengths: a pinned side that the host fills and a device side that the graph reads
        self.host = (torch.full((n,), -1, dtype=torch.int64).pin_memory(), torch.zeros(n, dtype=torch.int32).pin_memory(),
                     seqs.lens.clone().pin_memory())
        self.slots, self.positions, self.seq_lens = (t.to(device) for t in self.host)
        self.copied = torch.cuda.Event()
        self._run()  # (once outside the capture; its slots are padding, nothing is written)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.out = self._run()

    def _run(self):
        return self.block.step(self.x, self.slots, self.positions, self.q_start, self.pages, self.seq_lens, 1)

    def step(self, x):
        self.copied.synchronize()  # the last step's copies have left the pinned buffers
        new = (*self.seqs.append([1] * self.x.shape[0]), self.seqs.lens)
        for host, device, values in zip(self.host, (self.slots, self.positions, self.seq_lens), new):
            host.copy_(values)
            device.copy_(host, non_blocking=True)
        self.copied.record()
        self.x.copy_(x)
        self.graph.replay()
        return self.out


def serve(shape, bits, cache_bits, n_seqs, prefix, prompts, steps, window=0, page_tokens=64, seed=0, keep=False):
    """Prefix, ragged prompts, then `steps` decode steps on random rows. Returns (block, sequences, the rows in the
    order of their steps as [(x, q_start, lens, out)] if keep, else [], milliseconds per decode step)."""
    device = torch.device("cuda")
    g = torch.Generator(device=device).manual_seed(seed)
    max_len = prefix + max(prompts) + steps
    seqs = Sequences(n_seqs, prefix, max_len, page_tokens)
    calls = [(n_seqs, sum(prompts), max(prompts), prefix), (n_seqs, n_seqs, 1, prefix)]
    if prefix:
        calls.append((1, prefix, prefix, 0))
    block = ServedBlock(shape, make_w(shape, 0.02, device, seed), bits, cache_bits, page_tokens, seqs.n_pages, calls, max_len, prefix, window)
    log = []

    def rows(n):
        return torch.randn((n, shape.d_model), generator=g, device=device).to(torch.float16)

    def note(x, starts, lens, out):
        if keep:
            log.append((x.clone(), list(starts), lens.tolist(), out.clone()))

    # the prefix, once for all: one sequence's worth of rows
    if prefix:
        one = Sequences(1, 0, max_len, page_tokens)
        one.pages = seqs.pages[:1]
        slots, positions = one.append([prefix])
        x, starts = rows(prefix), [0, prefix]
        out = block.step(x, slots.to(device), positions.to(device), torch.tensor(starts, dtype=torch.int32, device=device),
                         one.pages.to(device), one.lens.to(device), prefix, shared_len=0)
        note(x, starts, one.lens, out)
    # prompts of different lengths in one call
    slots, positions = seqs.append(prompts)
    starts = [0] + torch.tensor(prompts).cumsum(0).tolist()
    x = rows(starts[-1])
    out = block.step(x, slots.to(device), positions.to(device), torch.tensor(starts, dtype=torch.int32, device=device),
                     seqs.pages.to(device), seqs.lens.to(device), max(prompts))
    note(x, starts, seqs.lens, out)
    decoder = Decoder(block, seqs, device)
    xs = rows(steps * n_seqs).view(steps, n_seqs, -1)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for x in xs:
        out = decoder.step(x)
        note(x, range(n_seqs + 1), seqs.lens, out)
    end.record()
    end.synchronize()
    if J.jab_get_device_status() != 0:
        raise RuntimeError("a kernel reported an error")
    return block, seqs, log, start.elapsed_time(end) / max(1, steps)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--shape", choices=("mistral", "gpt2"), default="mistral")
    p.add_argument("--bits", type=int, default=4, help="of the weights (2 to 8)")
    p.add_argument("--cache-bits", type=int, choices=(4, 8), default=8)
    p.add_argument("--seqs", type=int, default=64)
    p.add_argument("--prefix", type=int, default=1024, help="shared tokens, a multiple of 64")
    p.add_argument("--steps", type=int, default=64)
    p.add_argument("--window", type=int, default=0)
    a = p.parse_args()
    shape = MISTRAL_7B if a.shape == "mistral" else GPT2_SMALL
    prompts = [1 + (37 * b) % 200 for b in range(a.seqs)]
    block, seqs, _, ms = serve(shape, a.bits, a.cache_bits, a.seqs, a.prefix, prompts, a.steps, a.window)
    # what the cache holds of the first sequence's last page, as numbers
    n = int(seqs.lens[0])
    start = (n - 1) // 64 * 64
    k, v = (torch.empty((1, 64, shape.n_kv_heads, shape.head_dim), dtype=torch.float16, device="cuda") for _ in range(2))
    J.jab_kv_read(block.cache, seqs.pages[:1].cuda(), torch.tensor([n - start], dtype=torch.int32, device="cuda"), k, v,
                  starts=torch.tensor([start], dtype=torch.int32, device="cuda"))
    held = sum(t.numel() * t.element_size() for t in (block.cache.k_codes, block.cache.v_codes, block.cache.k_scales, block.cache.v_scales))
    print(f"{a.shape} block, weights in {a.bits} bits, cache in {a.cache_bits} ({held / 2**20:.0f} MiB), {a.seqs} sequences of "
          f"{int(seqs.lens.min())} to {int(seqs.lens.max())} tokens, {a.prefix} of them shared")
    print(f"decode step: {ms * 1e3:.1f} us ({a.seqs / ms * 1e3:.0f} tokens/s); rms of cached keys {float(k[0, :n - start].float().pow(2).mean().sqrt()):.3f}, "
          f"values {float(v[0, :n - start].float().pow(2).mean().sqrt()):.3f}; finite: {math.isfinite(float(block.out[:a.seqs].float().sum()))}")


if __name__ == "__main__":
    main()
