"""Several continuations of one prompt, sampled from a small decoder whose projections are mixed-precision SFMP matrices
(random ones: there is no checkpoint here) and whose keys and values live in the 8-bit paged cache.

    python examples/sample_continuations.py [--steps 64] [--continuations 8] [--eager] [--share] [--window 0] [--sinks 0]

The prompt's tokens are reserved, appended and attended to once; the continuations are forked off it and share its pages.
A decoding step reserves one token for each (a shared, partly filled page is copied then), runs the layers, and chooses the next
tokens.  With --share the attention of a step reads the pages that the continuations share once for all of them, as planned once for all layers; with
--window every token sees the last of the tokens before it alone, and the first ones (--sinks).  Nothing in a step asks the host, so it is captured once as a graph and replayed.  At the end half of the continuations
are given back and the pool is compacted."""
import argparse
import math
import os
import sys
import time
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2602_01027_amd as S  # noqa: E402
import sfmp_workloads as W  # noqa: E402


@dataclass
class Shape:
    layers: int = 2
    hidden: int = 4096
    q_heads: int = 32
    kv_heads: int = 8
    head_dim: int = 128
    ffn: int = 14336
    vocab: int = 32000
    theta: float = 500000.0


class Matrix:
    """One packed projection: Y = X W^T."""

    def __init__(self, K, N, seed, device):
        p = W.make_problem("example", K, N, 1, seed, fast_codes=True)
        layout, s2, s3, s4, index = S.sfmp_pack(p.codes, p.bitmap)
        self.problem = p
        self.packed = S.upload_packed(layout, s2, s3, s4, index, p.scales, p.zeros, p.bitmap, device)
        self.col_perm = torch.from_numpy(p.col_perm).to(device)
        self.row_perm = torch.from_numpy(p.row_perm).to(device)
        self.workspaces = {}

    def __call__(self, X):
        M, d = X.shape[0], self.packed
        if M not in self.workspaces:
            self.workspaces[M] = torch.empty(S.sfmp_gemm_workspace(d.layout, M), dtype=torch.uint8, device=X.device)
        Y = torch.empty((M, d.layout.N), dtype=torch.float16, device=X.device)
        S.sfmp_gemm(X, self.col_perm, d.layout, d.s2, d.s3, d.s4, d.index, d.scales, d.zeros, d.bitmap, self.row_perm, Y, self.workspaces[M])
        return Y


def norm(x):
    x = x.float()
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)).half()


class Decoder:
    def __init__(self, shape: Shape, pages: int, sequences: int, table_pages: int, seed: int = 0, device="cuda:0", format="int8",
                 window: int = 0, sinks: int = 0):
        s = self.shape = shape
        self.device = device
        self.window, self.sinks = window, sinks
        width = (s.q_heads + 2 * s.kv_heads) * s.head_dim
        seeds = iter(range(1000 * seed, 1000 * seed + 1000))
        make = lambda K, N: Matrix(K, N, next(seeds), device)  # noqa: E731
        self.layers = [dict(qkv=make(s.hidden, width), out=make(s.q_heads * s.head_dim, s.hidden), up=make(s.hidden, 2 * s.ffn),
                            down=make(s.ffn, s.hidden)) for _ in range(s.layers)]
        self.head = make(s.hidden, s.vocab)
        g = torch.Generator().manual_seed(seed)
        self.embedding = torch.randn((s.vocab, s.hidden), generator=g).half().to(device)
        self.frequency = (s.theta ** (-torch.arange(0, s.head_dim, 2, dtype=torch.float64) / s.head_dim)).float().to(device)
        self.layout = S.sfmp_kv_query(pages, s.kv_heads, s.head_dim, format, s.layers)
        self.cache = S.make_kv_cache(self.layout, device)
        self.tables = S.make_kv_tables(self.layout, sequences, table_pages, device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.pages_workspace = torch.empty(S.sfmp_kv_pages_workspace(self.layout), dtype=torch.uint8, device=device)

    def turn(self, x, positions):
        """Rotary positions, on the pairs (i, i + head_dim / 2)."""
        angle = positions.float()[:, None, None] * self.frequency
        a, b = x.float().chunk(2, -1)
        return torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1).half()

    def attention(self, slots, row_start, rows, max_rows, max_tokens, groups):
        """What attends to the cache, (layer, queries, output), in a step; groups: the first sequence of every group that shares its pages, and their
        end, or None."""
        s, scale, masks = self.shape, 1.0 / math.sqrt(self.shape.head_dim), dict(window=self.window, sinks=self.sinks)
        new = lambda size: torch.empty(size, dtype=torch.uint8, device=self.device)  # noqa: E731
        sizes = (s.q_heads, max_rows, max_tokens)
        if groups is None:
            workspace = new(S.sfmp_kv_attention_workspace(self.layout, slots.shape[0], rows, *sizes))
            return lambda i, q, out: S.sfmp_kv_attention_sinks(self.cache, i, self.tables, slots, row_start, q, out, max_rows, max_tokens, scale,
                                                               workspace, **masks)
        sizes = (self.layout, slots.shape[0], rows, groups.shape[0] - 1, *sizes)
        plan, workspace = new(S.sfmp_kv_share_plan(*sizes)), new(S.sfmp_kv_attention_shared_workspace(*sizes))
        S.sfmp_kv_share(self.cache, self.tables, slots, row_start, groups, rows, s.q_heads, max_rows, max_tokens, plan, **masks)
        return lambda i, q, out: S.sfmp_kv_attention_shared(self.cache, i, self.tables, slots, row_start, groups, q, out, max_rows, max_tokens, scale,
                                                            plan, workspace, **masks)

    def run(self, tokens, positions, slots, row_start, max_rows, max_tokens, groups=None):
        """Hidden states of new tokens, whose places in their sequences have been reserved."""
        s, rows = self.shape, tokens.shape[0]
        x = self.embedding[tokens]
        attend = self.attention(slots, row_start, rows, max_rows, max_tokens, groups)
        for i, m in enumerate(self.layers):
            heads = m["qkv"](norm(x)).unflatten(1, (-1, s.head_dim))
            q, k, v = heads.split((s.q_heads, s.kv_heads, s.kv_heads), 1)
            S.sfmp_kv_append(self.cache, i, self.tables, slots, row_start, self.turn(k, positions), v, max_rows)
            attended = torch.empty((rows, s.q_heads, s.head_dim), dtype=torch.float16, device=self.device)
            attend(i, self.turn(q, positions), attended)
            x = x + m["out"](attended.flatten(1))
            gate, up = m["up"](norm(x)).float().chunk(2, -1)
            x = x + m["down"]((torch.nn.functional.silu(gate) * up).half())
        return x

    def logits(self, x):
        return self.head(norm(x))

    def reserve(self, slots, counts=None):
        S.sfmp_kv_reserve(self.cache, self.tables, slots, counts, self.status, self.pages_workspace)

    def prefill(self, slot, prompt):
        """Puts a prompt into the empty sequence `slot`; the logits of the token after it."""
        n = prompt.shape[0]
        one = lambda v: torch.tensor(v, dtype=torch.int32, device=self.device)  # noqa: E731
        slots = one([slot])
        self.reserve(slots, one([n]))
        x = self.run(prompt, torch.arange(n, device=self.device), slots, one([0, n]), n, n)
        return self.logits(x[-1:])


@dataclass
class Sampling:
    temperature: float = 0.8
    top_k: int = 50
    top_p: float = 0.95
    min_p: float = 0.0

    def on(self, n, device):
        f = lambda v: torch.full((n,), v, dtype=torch.float32, device=device)  # noqa: E731
        return f(self.temperature), torch.full((n,), self.top_k, dtype=torch.int32, device=device), f(self.top_p), f(self.min_p)


def room(status):
    return "the page table is too short" if int(status) < 0 else f"{int(status)} pages are missing"


def sample_continuations(decoder, prompt, n, steps, sampling, seed=0, graph=True, share=False):
    """tokens int32 and their log-probabilities [steps, n].  Sequence 0 of the decoder and 1 .. n have to be empty; the
    continuations are left in 1 .. n.  share: their attention reads the pages that they share once."""
    device, vocab = decoder.device, decoder.shape.vocab
    numbers = lambda a, b: torch.arange(a, b, dtype=torch.int32, device=device)  # noqa: E731
    slots = numbers(1, n + 1)
    uniform = torch.rand((steps, n), generator=torch.Generator().manual_seed(seed)).to(device)
    filters = sampling.on(n, device)
    tokens, logprobs, u = numbers(0, n), torch.empty(n, dtype=torch.float32, device=device), torch.empty(n, dtype=torch.float32, device=device)
    workspace = torch.empty(S.sfmp_sample_workspace(n, vocab), dtype=torch.uint8, device=device)
    failed = torch.zeros(1, dtype=torch.int32, device=device)
    max_tokens = prompt.shape[0] + steps
    groups = torch.tensor([0, n], dtype=torch.int32, device=device) if share else None

    def choose(logits):
        S.sfmp_sample(logits, *filters, u, tokens, logprobs, workspace)

    def step():
        decoder.reserve(slots)
        failed.copy_(torch.where(failed == 0, decoder.status, failed))
        positions = decoder.tables.lengths[1:n + 1] - 1
        choose(decoder.logits(decoder.run(tokens, positions, slots, None, 1, max_tokens, groups)))

    first = decoder.prefill(0, prompt)
    if int(decoder.status):  # (a prompt without room: nothing was reserved, and nothing may be appended for good)
        raise RuntimeError(f"no room for the prompt: {room(decoder.status)}")
    S.sfmp_kv_fork(decoder.cache, decoder.tables, torch.zeros(n, dtype=torch.int32, device=device), slots)
    S.sfmp_kv_free(decoder.cache, decoder.tables, numbers(0, 1))  # (its pages are the continuations' now)
    u.copy_(uniform[0])
    choose(first.expand(n, vocab).contiguous())
    chosen, how = [tokens.clone()], [logprobs.clone()]
    captured = None
    for i in range(1, steps):
        u.copy_(uniform[i])
        if captured is not None:
            captured.replay()
        else:
            step()
            if graph:  # (the eager step has loaded every kernel; recording runs nothing)
                captured = torch.cuda.CUDAGraph()
                with torch.cuda.graph(captured):
                    step()
        chosen.append(tokens.clone())
        how.append(logprobs.clone())
    if int(failed):  # (a step without room changes no length: the steps after it wrote over the last token)
        raise RuntimeError(f"no room for a token: {room(failed)}")
    return torch.stack(chosen), torch.stack(how)


def give_back(decoder, slots):
    """Frees sequences and moves the pages that are left to the low end of the pool; their number."""
    S.sfmp_kv_free(decoder.cache, decoder.tables, torch.tensor(slots, dtype=torch.int32, device=decoder.device))
    S.sfmp_kv_compact(decoder.cache, decoder.tables, decoder.status, decoder.pages_workspace)
    return int(decoder.status)


def main():
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--prompt", type=int, default=1000, help="tokens of the prompt")
    a.add_argument("--continuations", type=int, default=8)
    a.add_argument("--steps", type=int, default=64)
    a.add_argument("--layers", type=int, default=2)
    a.add_argument("--eager", action="store_true", help="launch every step instead of replaying a graph")
    a.add_argument("--share", action="store_true", help="read shared pages once for all continuations")
    a.add_argument("--window", type=int, default=0, help="tokens that a token sees (0: all before it)")
    a.add_argument("--sinks", type=int, default=0, help="first tokens that it sees too")
    a = a.parse_args()
    shape = Shape(layers=a.layers)
    each = (a.prompt + a.steps) // 64 + 2
    decoder = Decoder(shape, pages=each * (a.continuations + 1), sequences=a.continuations + 1, table_pages=each,
                      window=a.window, sinks=a.sinks)
    prompt = torch.randint(0, shape.vocab, (a.prompt,), generator=torch.Generator().manual_seed(1)).to(decoder.device)
    for turn in range(2):  # (the first turn loads the kernels)
        torch.cuda.synchronize()
        start = time.perf_counter()
        tokens, logprobs = sample_continuations(decoder, prompt, a.continuations, a.steps, Sampling(), seed=turn, graph=not a.eager,
                                                share=a.share)
        torch.cuda.synchronize()
        took = time.perf_counter() - start
        live = give_back(decoder, list(range(1, a.continuations + 1, 2)))
        print(f"{a.continuations} continuations x {a.steps} tokens after {a.prompt}: {took * 1e3:.1f} ms, mean log-probability "
              f"{logprobs.mean().item():.3f}, {live} of {decoder.layout.pages} pages held after half were given back")
        print("  first tokens:", tokens[:6].T[:4].tolist())
        give_back(decoder, list(range(2, a.continuations + 1, 2)))


if __name__ == "__main__":
    main()
