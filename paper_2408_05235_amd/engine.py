"""The serving engine's iterations that a scoreboard projects, run on the paged
cache: what an iteration costs at a batch size and a number of KV blocks.

    python -m paper_2408_05235_amd.engine [--config c0] [--iterations 64]

The projection (Sec. 4.2, Eq. 1-2) says how many requests and KV blocks
are in the batch at every future iteration; the performance model (Sec. 4.3.1) is
trained on what the engine does at such points.  ``Engine`` serves one scenario's
in-flight requests through attention layers over a ``api.KVCache``: their
prompts first, then one token per request and iteration, finished requests
leaving.  The pages in use are the projection's blocks, iteration by iteration; a
request that the pool has no room for stops where it is (``Engine.stopped``).
The layers are random; the times are those of the attention part alone.
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import _lib, api, configs, synth


class Engine:
    """One scenario's in-flight requests (``prompt``, ``generated``,
    ``remaining`` as in tl_project) in as many slots, ``n_layers`` layers of
    ``n_heads`` query heads over ``n_kv_heads`` of ``head_dim``, a window and
    sinks as in tl_attend."""

    def __init__(self, prompt, generated, remaining, block_tokens, kv_capacity, n_layers=2, n_heads=8, n_kv_heads=2,
                 head_dim=128, window=0, sinks=0, dtype=torch.bfloat16, seed=0, device="cuda"):
        self.tokens = np.asarray(prompt, np.int64) + np.asarray(generated, np.int64)
        self.remaining = np.asarray(remaining, np.int64)
        self.n_heads, self.n_kv_heads, self.head_dim = n_heads, n_kv_heads, head_dim
        self.window, self.sinks = window, sinks
        self.max_tokens = int((self.tokens + self.remaining).max())
        self.cache = api.KVCache(n_layers, kv_capacity, n_kv_heads, block_tokens, head_dim, len(self.tokens),
                                 self.max_tokens, dtype, device)
        g = torch.Generator(device=device).manual_seed(seed)
        width = n_heads * head_dim
        weight = lambda a, b: torch.randn(a, b, generator=g, device=device).mul_(a ** -0.5).to(dtype)
        self.qkv = [weight(width, (n_heads + 2 * n_kv_heads) * head_dim) for _ in range(n_layers)]
        self.proj = [weight(width, width) for _ in range(n_layers)]
        self.inputs = lambda n: torch.randn(n, width, generator=g, device=device).to(dtype)
        self.left = torch.from_numpy(self.remaining).to(device, torch.int32)
        self.stopped = torch.zeros(len(self.tokens), dtype=torch.bool, device=device)
        self.iteration = 0

    def _extend(self, add):
        """Room for ``add`` tokens.  A request that is refused keeps the pages and
        tokens that it has until its time is over, and asks for no more: the tokens
        behind a missing one would not be its own."""
        self.stopped |= self.cache.extend(add) != _lib.PAGES_OK

    def forward(self, x, q_offset=None):
        """The new tokens' hidden states [T, n_heads * head_dim] through the
        layers; the slots have room for them already."""
        T, H, G = x.shape[0], self.n_heads, self.n_kv_heads
        for layer, (wq, wo) in enumerate(zip(self.qkv, self.proj)):
            qkv = (x @ wq).view(T, H + 2 * G, self.head_dim)
            self.cache.append(layer, qkv[:, H:H + G], qkv[:, H + G:], q_offset)
            y = self.cache.attend(layer, qkv[:, :H], q_offset, window=self.window, sinks=self.sinks,
                                  max_length=self.max_tokens)
            x = x + y.view(T, -1) @ wo
        return x

    def prefill(self):
        """Iteration 0: every request's prompt and what it has generated.  Rows
        of a request that has stopped are no token's."""
        dev = self.left.device
        self._extend(torch.from_numpy(self.tokens).to(dev, torch.int32))
        off = torch.from_numpy(np.concatenate([[0], np.cumsum(self.tokens)])).to(dev)
        return self.forward(self.inputs(int(self.tokens.sum())), off)

    def step(self):
        """The next iteration: finished requests leave, the others get a
        token.  Returns the hidden states, one row per slot (of a request that
        has left or stopped, no token's)."""
        self.iteration += 1
        gone = np.flatnonzero(self.remaining == self.iteration)
        if len(gone):
            self.cache.free(torch.from_numpy(gone).to(self.left.device, torch.int32))
        self._extend(((self.left > self.iteration) & ~self.stopped).to(torch.int32))
        return self.forward(self.inputs(len(self.tokens)))


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--config", default="c0")
    ap.add_argument("--iterations", type=int, default=64)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--sinks", type=int, default=0)
    a = ap.parse_args(argv)
    cfg = synth.scaled(configs.get_config(a.config), n_scenarios=1)
    inp = synth.make_inputs(cfg)
    flight = inp["arrival"] < 0
    d = api.upload(inp)
    H = min(a.iterations, d["horizon"])
    board = [d[k][torch.from_numpy(np.flatnonzero(flight)).cuda()] for k in ("prompt", "generated", "remaining", "arrival")]
    off = torch.tensor([0, int(flight.sum())], device="cuda")
    proj = api.tl_project(off, *board, d["kv_capacity"], H, d["block_tokens"])
    e = Engine(*(inp[k][flight] for k in ("prompt", "generated", "remaining")), int(inp["block_tokens"]),
               int(inp["kv_capacity"][0]), n_layers=a.layers, n_heads=a.heads, n_kv_heads=a.kv_heads, window=a.window,
               sinks=a.sinks)
    kv, batch = proj["kv"][0].cpu().numpy(), proj["batch"][0].cpu().numpy()
    e.prefill()
    print(f"{'iteration':>9} {'batch':>6} {'blocks':>7} {'in use':>7} {'iterations/s of ' + str(a.layers) + ' layers':>26}")
    for j in range(H):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        if j:
            e.step()
        end.record()
        used = int(e.cache.pages_used())
        if bool(e.stopped.any()):
            raise SystemExit(f"iteration {j}: no room for {int(e.stopped.sum())} of the requests in "
                             f"{int(inp['kv_capacity'][0])} pages ({kv[j]} blocks projected)")
        if used != kv[j]:
            raise SystemExit(f"iteration {j}: {used} pages in use, {kv[j]} blocks projected")
        if j and (j & (j - 1) == 0 or j == H - 1):
            print(f"{j:9d} {batch[j]:6d} {kv[j]:7d} {used:7d} {1e3 / start.elapsed_time(end):26.1f}", flush=True)


if __name__ == "__main__":
    main()
