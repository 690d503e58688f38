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
The layers are random; the times are those of the attention part alone, with
``--norm``, ``--quantize``, ``--select`` and ``--vocabulary`` also of what stands
around it: norms before the products, those in 8 bits, attention over the pages that
score best, and tokens drawn from logits, whose embeddings are the next inputs.
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
    sinks as in tl_attend.

    ``norm``: a norm before each product, the residual's sum in the same call.
    ``quantize``: the products behind a norm in e4m3, a scale a row (implies ``norm``;
    widths and the vocabulary are multiples of 16).
    ``select``: single tokens attend over so many pages, their choice by score (0: all).
    ``vocabulary``: inputs are the embeddings of tokens, drawn from the last hidden
    states' logits (0: random inputs); ``sampling`` holds tl_sample's settings, and
    ``token`` the slots' last tokens."""

    def __init__(self, prompt, generated, remaining, block_tokens, kv_capacity, n_layers=2, n_heads=8, n_kv_heads=2,
                 head_dim=128, window=0, sinks=0, dtype=torch.bfloat16, seed=0, device="cuda", norm=False,
                 quantize=False, select=0, vocabulary=0):
        if select and (window or sinks):
            raise ValueError("select has no window")
        if not 0 <= select <= _lib.MAX_SELECTED:
            raise ValueError(f"select {select} outside [0, {_lib.MAX_SELECTED}]")
        if select and n_heads > n_kv_heads * _lib.MAX_GROUP:
            raise ValueError(f"select takes up to {_lib.MAX_GROUP} query heads per KV head, not {n_heads // n_kv_heads} query heads")
        if not 0 <= vocabulary <= _lib.MAX_COLUMNS:
            raise ValueError(f"vocabulary {vocabulary} outside [0, {_lib.MAX_COLUMNS}]")
        # (what the library's product in 8 bits takes)
        sizes = (("width", n_heads * head_dim), ("width of queries, keys and values", (n_heads + 2 * n_kv_heads) * head_dim),
                 ("vocabulary", vocabulary))
        for name, n in sizes if quantize else ():
            if n % 16:
                raise ValueError(f"quantize needs multiples of 16, not a {name} of {n}")
        self.tokens = np.asarray(prompt, np.int64) + np.asarray(generated, np.int64)
        self.remaining = np.asarray(remaining, np.int64)
        self.n_heads, self.n_kv_heads, self.head_dim = n_heads, n_kv_heads, head_dim
        self.window, self.sinks = window, sinks
        self.max_tokens = int((self.tokens + self.remaining).max())
        self.cache = api.KVCache(n_layers, kv_capacity, n_kv_heads, block_tokens, head_dim, len(self.tokens),
                                 self.max_tokens, dtype, device, summaries=select > 0)
        g = torch.Generator(device=device).manual_seed(seed)
        width = n_heads * head_dim
        weight = lambda a, b: torch.randn(a, b, generator=g, device=device).mul_(a ** -0.5).to(dtype)
        self.qkv = [weight(width, (n_heads + 2 * n_kv_heads) * head_dim) for _ in range(n_layers)]
        self.proj = [weight(width, width) for _ in range(n_layers)]
        self.inputs = lambda n: torch.randn(n, width, generator=g, device=device).to(dtype)
        self.left = torch.from_numpy(self.remaining).to(device, torch.int32)
        self.select, self.norms = select, None
        self.quantize = [None] * (n_layers + 1)
        if norm or quantize:
            self.norms = [(1 + 0.1 * torch.randn(width, generator=g, device=device)).to(dtype) for _ in range(n_layers + 1)]
        self.embedding, self.sampling = None, {}
        if vocabulary:
            self.head = weight(width, vocabulary)
            self.embedding = torch.randn(vocabulary, width, generator=g, device=device).to(dtype)
            self.token = torch.zeros(len(self.tokens), dtype=torch.int32, device=device)
            self.inputs = lambda n: self.embedding[torch.randint(vocabulary, (n,), generator=g, device=device)]
            self.numbers = lambda n: torch.rand(n, generator=g, device=device)
        if quantize:
            self.one = torch.ones((), device=device)
            self.quantize = [self._eight_bits(w) for w in self.qkv + ([self.head] if vocabulary else [])]
        self.stopped = torch.zeros(len(self.tokens), dtype=torch.bool, device=device)
        self.iteration = 0

    def _extend(self, add):
        """Room for ``add`` tokens.  A request that is refused keeps the pages and
        tokens that it has until its time is over, and asks for no more: the tokens
        behind a missing one would not be its own."""
        self.stopped |= self.cache.extend(add) != _lib.PAGES_OK

    @staticmethod
    def _eight_bits(w):
        """A weight [in, out] as e4m3, a scale a column."""
        scale = w.float().abs().amax(0, keepdim=True).clamp(min=2.0 ** -100) / 448
        return (w.float() / scale).T.contiguous().to(torch.float8_e4m3fn).T, scale

    def _product(self, at, x, weight, residual=None):
        """norm(x + residual) @ weight, and the sum (x itself without residual)."""
        eight = self.quantize[at]
        r = api.tl_norm(x, self.norms[at], residual=residual, group=None if eight is None else 0)
        r = r if isinstance(r, tuple) else (r,)
        total = x if residual is None else r[-1]
        if eight is None:
            return r[0] @ weight, total
        if x.dtype == torch.bfloat16:
            return torch._scaled_mm(r[0], eight[0], scale_a=r[1][:, None], scale_b=eight[1], out_dtype=x.dtype), total
        # (the library scales rows in bf16 alone, three bits short of f16: here in fp32, rounded once)
        y = torch._scaled_mm(r[0], eight[0], scale_a=self.one, scale_b=self.one, out_dtype=torch.float32)
        return y.mul_(r[1][:, None]).mul_(eight[1]).to(x.dtype), total

    def _draw(self, x):
        """A token for each slot from its hidden state."""
        logits = x @ self.head if self.norms is None else self._product(len(self.qkv), x, self.head)[0]
        return api.tl_sample(logits, self.numbers(x.shape[0]), **self.sampling)

    def _attend(self, layer, query, q_offset):
        if self.select and q_offset is None:
            # (the last page always, and of two or more the first one)
            pages = self.cache.select(layer, query, self.select, q_offset, first=min(1, self.select - 1))
            return self.cache.attend_pages(layer, query, pages, q_offset)
        return self.cache.attend(layer, query, q_offset, window=self.window, sinks=self.sinks, max_length=self.max_tokens)

    def forward(self, x, q_offset=None):
        """The new tokens' hidden states [T, n_heads * head_dim] through the
        layers; the slots have room for them already."""
        T, H, G = x.shape[0], self.n_heads, self.n_kv_heads
        y = None
        for layer, (wq, wo) in enumerate(zip(self.qkv, self.proj)):
            if self.norms is None:
                qkv = x @ wq
            elif y is None:
                qkv, x = self._product(layer, x, wq)
            else:               # the last layer's output joins the hidden states on the way
                qkv, x = self._product(layer, y, wq, x)
            qkv = qkv.view(T, H + 2 * G, self.head_dim)
            self.cache.append(layer, qkv[:, H:H + G], qkv[:, H + G:], q_offset)
            y = self._attend(layer, qkv[:, :H], q_offset).view(T, -1) @ wo
            if self.norms is None or layer + 1 == len(self.qkv):
                x = x + y
        return x

    def prefill(self):
        """Iteration 0: every request's prompt and what it has generated.  Rows
        of a request that has stopped are no token's."""
        dev = self.left.device
        self._extend(torch.from_numpy(self.tokens).to(dev, torch.int32))
        off = torch.from_numpy(np.concatenate([[0], np.cumsum(self.tokens)])).to(dev)
        x = self.forward(self.inputs(int(self.tokens.sum())), off)
        if self.embedding is not None and len(x):
            self.token = self._draw(x[(off[1:] - 1).clamp(min=0)])
        return x

    def step(self):
        """The next iteration: finished requests leave, the others get a
        token.  Returns the hidden states, one row per slot (of a request that
        has left or stopped, no token's)."""
        self.iteration += 1
        gone = np.flatnonzero(self.remaining == self.iteration)
        if len(gone):
            self.cache.free(torch.from_numpy(gone).to(self.left.device, torch.int32))
        self._extend(((self.left > self.iteration) & ~self.stopped).to(torch.int32))
        if self.embedding is None:
            return self.forward(self.inputs(len(self.tokens)))
        x = self.forward(self.embedding[self.token.clamp(min=0).long()])
        self.token = self._draw(x)
        return x


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--config", default="c0")
    ap.add_argument("--iterations", type=int, default=64)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--sinks", type=int, default=0)
    ap.add_argument("--norm", action="store_true", help="norms before the products")
    ap.add_argument("--quantize", action="store_true", help="the products behind the norms in 8 bits")
    ap.add_argument("--select", type=int, default=0, help="pages that single tokens attend over (0: all)")
    ap.add_argument("--vocabulary", type=int, default=0, help="tokens that the next inputs are drawn from (0: none)")
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
               sinks=a.sinks, norm=a.norm, quantize=a.quantize, select=a.select, vocabulary=a.vocabulary)
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
