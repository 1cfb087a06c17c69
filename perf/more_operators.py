"""The operators of many sequences over one prompt, and of endless ones - attention that reads the pages which forked sequences
share once for all of them, attention over a sliding window and the first tokens, the choice of a beam search and the
reordering of its sequences - as measurable cases.

Fields of a case
  call    "shared"   what the sequences of each group share is found and their attention planned once, then the attention
                     of their last rows in every layer
          "sinks"    attention of the last rows of every sequence over a sliding window and the first tokens
          "select"   one step of a beam search: the best continuations of every request over its beams and the vocabulary
          "reorder"  the sequences of a batch become what their parents were, as a beam search goes on with them
  groups  requests, or prompts ("sinks": 1)
  each    sequences of a group, beams of a request
  rows    new rows per sequence, or rows_lo ... rows, spread over the logarithm of that range ("sinks")
  prefix_lo, prefix_hi  tokens of the prompts, spread likewise over the groups
  tokens_lo, tokens_hi  tokens of the sequences behind their prompt ("sinks", "reorder": in all), spread likewise
  q_heads, kv_heads, head_dim, window (0: none), sinks
  format  of the cache: "int8" or "fp8", with one scale for each page of 64 tokens and head
  dtype   of activations or logits: "fp16", "bf16", "fp32" (logits alone)
  layers  that share the page table, all of them attended to
  vocab, choices        tokens to choose from, continuations wanted per request
  ended_percent         of the beams that have ended
  weighted              continuations are ranked by a weight of their beam times their score
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
PAGE = 64
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}

MOST_GATHERED = 64 * 33768 * 2 * 8 * 128     # values of keys and values, a sequence at a time, of the longest listed batch
MOST_PAIRS = 32 * 2048 * 6144 * 128          # query rows x keys x dimensions of the listed prompt
MOST_SHARED_PAIRS = 64 * 32 * 33768 * 128    # ... of the longest listed batch
MOST_LOGITS = 32 * 8 * 131072


def _case(call, **more):
    c = dict(call=call, groups=1, each=1, rows_lo=0, rows=1, prefix_lo=0, prefix_hi=0, tokens_lo=1, tokens_hi=1, q_heads=32,
             kv_heads=8, head_dim=128, window=0, sinks=0, format="int8", dtype="fp16", layers=1, vocab=0, choices=0,
             ended_percent=0, weighted=False)
    c.update(more)
    c["rows_lo"] = c["rows_lo"] or c["rows"]
    return c


def listed():
    named = [
        # four beams over a prompt of a page and a bit each, two layers: launches and latency
        ("shared_beams", _case("shared", each=4, prefix_lo=1000, prefix_hi=1000, tokens_lo=9, tokens_hi=24, layers=2)),
        # a serving batch: eight prompts, eight samples of each, of different lengths
        ("shared_samples", _case("shared", groups=8, each=8, prefix_lo=1000, prefix_hi=7001, tokens_lo=20, tokens_hi=900,
                                 format="fp8", dtype="bf16", layers=2)),
        # one long document, many questions about it
        ("shared_document", _case("shared", each=64, prefix_lo=32768, prefix_hi=32768, tokens_lo=50, tokens_hi=1000)),
        # speculative decoding of samples: four drafted tokens of each checked at once; small heads
        ("shared_drafts", _case("shared", groups=3, each=12, rows=4, prefix_lo=3001, prefix_hi=9001, tokens_lo=30, tokens_hi=700,
                                q_heads=16, kv_heads=4, head_dim=64, dtype="bf16")),
        # one endless stream: a token after 20000, of which a window and the first page's tokens are seen
        ("sinks_token", _case("sinks", tokens_lo=20000, tokens_hi=20000, window=1024, sinks=4)),
        # a batch of streams of very different lengths
        ("sinks_batch", _case("sinks", each=48, tokens_lo=100, tokens_hi=16000, window=2048, sinks=100, format="fp8",
                              dtype="bf16")),
        # the last part of a long prompt
        ("sinks_prompt", _case("sinks", rows=2048, tokens_lo=6144, tokens_hi=6144, window=1000, sinks=65)),
        # four beams of a small decoder
        ("select_beams", _case("select", each=4, vocab=32000, choices=8)),
        # many requests, a large vocabulary
        ("select_batch", _case("select", groups=32, each=8, vocab=131072, choices=16, dtype="bf16")),
        # an odd vocabulary, beams that have ended among the others, ranked by their lengths
        ("select_ended", _case("select", groups=5, each=5, vocab=100003, choices=5, dtype="fp32", ended_percent=30, weighted=True)),
        # the beams of one request
        ("reorder_beams", _case("reorder", each=4, tokens_lo=1024, tokens_hi=1024)),
        # those of many
        ("reorder_batch", _case("reorder", groups=64, each=8, tokens_lo=200, tokens_hi=8190)),
    ]
    return [dict(c, name=n) for n, c in named]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """Another case of the same ranges: few to many sequences, short to long prompts, every head layout and format."""
    call = rng.choice(("shared", "shared", "shared", "sinks", "sinks", "select", "select", "reorder"))
    heads = rng.choice((1, 2, 4, 8, 16))
    group = rng.choice((1, 2, 4, 5, 7, 8, 16))
    c = _case(call, kv_heads=heads, q_heads=heads * group, head_dim=rng.choice((64, 128, 128, 128, 256)),
              format=rng.choice(("int8", "fp8")), dtype=rng.choice(("fp16", "bf16")))
    row = 2 * c["kv_heads"] * c["head_dim"]  # cached values of a token
    if call == "shared":
        c["each"] = _log_int(rng, 2, 64)
        c["groups"] = _log_int(rng, 1, max(1, 96 // c["each"]))
        c["rows"] = c["rows_lo"] = rng.choice((1, 1, 1, rng.randint(2, 6)))
        batch = c["each"] * c["groups"]
        per_row = c["q_heads"] * c["head_dim"] * c["rows"] * batch
        most = max(128, min(32768, MOST_GATHERED // (row * batch), MOST_SHARED_PAIRS // per_row))
        c["prefix_hi"] = _log_int(rng, 40, most - most // 16)
        c["prefix_lo"] = _log_int(rng, 20, c["prefix_hi"])
        c["tokens_hi"] = max(c["rows"], _log_int(rng, 1, max(1, min(1500, most // 16))))
        c["tokens_lo"] = max(c["rows"], _log_int(rng, 1, c["tokens_hi"]))
        c["layers"] = rng.choice((1, 2)) if c["prefix_hi"] <= most // 4 else 1
        if rng.random() < 0.2:
            c["window"], c["sinks"] = _log_int(rng, 16, 8192), rng.choice((0, 4, 100))
    elif call == "sinks":
        c["each"] = _log_int(rng, 1, 96)
        most = max(64, min(65536, MOST_GATHERED // (row * c["each"])))
        c["tokens_hi"] = _log_int(rng, 16, most)
        c["tokens_lo"] = _log_int(rng, 1, c["tokens_hi"])
        c["window"], c["sinks"] = _log_int(rng, 16, 4096), _log_int(rng, 1, 300)
        if rng.random() < 0.3:
            per_row = c["q_heads"] * c["head_dim"] * c["tokens_hi"] * c["each"]
            c["rows"] = _log_int(rng, 2, max(2, min(2048, c["tokens_hi"], MOST_PAIRS // per_row)))
            c["rows_lo"] = _log_int(rng, 1, c["rows"])
    elif call == "select":
        c["vocab"] = _log_int(rng, 1000, 200000)
        c["each"] = rng.choice((1, 2, 3, 4, 5, 8, 16))
        c["groups"] = _log_int(rng, 1, max(1, min(64, MOST_LOGITS // (c["vocab"] * c["each"]))))
        c["choices"] = rng.choice((c["each"], 2 * c["each"]))
        c["dtype"] = rng.choice(("fp16", "bf16", "fp32"))
        if c["groups"] * c["each"] * c["vocab"] > MOST_LOGITS // 2:
            c["dtype"] = "bf16"
        c["ended_percent"], c["weighted"] = rng.choice(((0, False), (0, False), (25, True)))
    else:
        c["each"] = rng.choice((2, 3, 4, 5, 8, 16))
        c["groups"] = _log_int(rng, 1, 512 // c["each"])
        c["tokens_hi"] = _log_int(rng, 1, 8190)
        c["tokens_lo"] = _log_int(rng, 1, c["tokens_hi"])
    return c


def _spread(lo, hi, n):
    """n whole numbers over the logarithm of [lo, hi]."""
    if n == 1:
        return [hi]
    return [int(round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * i / (n - 1)))) for i in range(n)]


def _lengths(case):
    """Tokens of every group's prompt, new rows and all tokens of every sequence: the same numbers for every seed."""
    n = case["groups"] * case["each"]
    prompts = _spread(case["prefix_lo"], case["prefix_hi"], case["groups"]) if case["prefix_hi"] else [0] * case["groups"]
    rows = _spread(case["rows_lo"], case["rows"], n)
    if case["call"] == "reorder":  # (the beams of a request are of one length)
        tokens = [t for t in _spread(case["tokens_lo"], case["tokens_hi"], case["groups"]) for _ in range(case["each"])]
    else:
        tokens = _spread(case["tokens_lo"], case["tokens_hi"], n)
        random.Random(97).shuffle(tokens)
    return prompts, rows, [max(t, r) + prompts[i // case["each"]] for i, (t, r) in enumerate(zip(tokens, rows))]


def _pages_of(tokens):
    return -(-tokens // PAGE)


def _codes(case, pages, gen):
    """Codes of a pool [layers, pages, kv heads, 2, 64 * head_dim], and a scale for each page, head and of K and V."""
    shape = (case["layers"], pages, case["kv_heads"], 2, PAGE * case["head_dim"])
    codes = torch.empty(shape, dtype=torch.uint8, device=DEVICE)
    flat = codes.view(-1)
    for i in range(0, flat.numel(), 1 << 26):  # a bounded piece of the pool at a time
        part = flat[i:i + (1 << 26)]
        x = torch.empty(part.numel(), dtype=torch.float32, device=DEVICE).normal_(generator=gen)
        if case["format"] == "int8":
            part.copy_(x.mul_(32.0).round_().clamp_(-127, 127).add_(128))
        else:
            part.copy_(x.mul_(64.0).to(torch.float8_e4m3fn).view(torch.uint8))
    scales = torch.empty(shape[:4], dtype=torch.float32, device=DEVICE).normal_(0.0, 0.5, generator=gen)
    scales = scales.exp_() / 32.0 if case["format"] == "int8" else torch.exp2(scales.round_() - 6.0)
    return codes, scales


def _up(a):
    return torch.from_numpy(a).to(DEVICE)


def _tables(case, order):
    """Page table, lengths and holders of every page: whole pages of a prompt are held by all sequences of its group, the
    others by one each, in no order; a few pages to spare."""
    prompts, _, tokens = _lengths(case)
    each = case["each"]
    shared = [p // PAGE for p in prompts]
    used = sum(shared) + sum(_pages_of(t) - shared[i // each] for i, t in enumerate(tokens))
    pages = used + used // 8 + 3
    ids = order.permutation(pages)[:used].astype(np.int32)
    table = np.full((len(tokens), max(_pages_of(t) for t in tokens) + 2), -1, dtype=np.int32)
    refs = np.zeros(pages, dtype=np.int32)
    at = 0
    for g, n in enumerate(shared):
        table[g * each:(g + 1) * each, :n] = ids[at:at + n]
        refs[ids[at:at + n]] = each
        at += n
    for b, t in enumerate(tokens):
        n = _pages_of(t) - shared[b // each]
        table[b, shared[b // each]:_pages_of(t)] = ids[at:at + n]
        refs[ids[at:at + n]] = 1
        at += n
    return pages, table, np.array(tokens, dtype=np.int32), refs


def _starts(counts):
    return _up(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))


def _activations(shape, dtype, gen, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device=DEVICE).normal_(0.0, std, generator=gen).to(DTYPES[dtype])


def _prepare_attention(s, gen, order):
    c = s["case"]
    h, d = c["kv_heads"], c["head_dim"]
    _, rows, tokens = _lengths(c)
    pages, table, lengths, refs = _tables(c, order)
    codes, scales = _codes(c, pages, gen)
    last = _up(np.array([table[b, _pages_of(t) - 1] for b, t in enumerate(tokens)])).long()
    # what no sequence has written: left by an earlier one, for fp8 the pattern that stands for no number
    past = (torch.arange(PAGE, device=DEVICE)[None, :] >= torch.tensor([(t - 1) % PAGE + 1 for t in tokens], device=DEVICE)[:, None])
    stale = 0x7F if c["format"] == "fp8" else 0xFF
    for layer in range(c["layers"]):
        kv = codes[layer, last]
        k, v = kv[:, :, 0].view(-1, h, PAGE, d), kv[:, :, 1].view(-1, h, d, PAGE)
        k.masked_fill_(past[:, None, :, None], stale)
        v.masked_fill_(past[:, None, None, :], stale)
        codes[layer, last] = kv
    s.update(codes=codes, scales=scales, table=_up(table), lengths=_up(lengths), refs=_up(refs), total=sum(rows),
             max_rows=max(rows), max_tokens=max(tokens))
    s["slots"] = torch.arange(len(tokens), dtype=torch.int32, device=DEVICE)
    s["row_start"] = _starts(rows)
    s["group_start"] = _starts([c["each"]] * c["groups"])
    s["prefix"] = torch.zeros(c["groups"], dtype=torch.int32, device=DEVICE)
    # the query part of a fused projection's output: rows lie further apart than they are long
    qkv = _activations((c["layers"], s["total"], (c["q_heads"] + 2 * h) * d), c["dtype"], gen, 1.6)
    s["q"] = [x[:, :c["q_heads"] * d].view(s["total"], c["q_heads"], d) for x in qkv]
    shape = (s["total"], c["q_heads"], d)
    s["out"] = [torch.empty(shape, dtype=DTYPES[c["dtype"]], device=DEVICE) for _ in range(c["layers"])]
    s["lse"] = [torch.empty(shape[:2], dtype=torch.float32, device=DEVICE) for _ in range(c["layers"])]


def _prepare_select(s, gen, order):
    c = s["case"]
    requests, beams, vocab, n = c["groups"], c["each"], c["vocab"], c["groups"] * c["each"]
    x = torch.empty((n, vocab), dtype=torch.float32, device=DEVICE).normal_(0.0, 2.0, generator=gen)
    # a few hundred tokens that the context makes likely, for all beams of a request much the same ones
    likely = torch.rand((requests, vocab), generator=gen, device=DEVICE) < min(0.25, 300 / vocab)
    boost = torch.empty((requests, vocab), device=DEVICE).exponential_(0.3, generator=gen).masked_fill_(~likely, 0.0)
    x.view(requests, beams, vocab).add_(boost[:, None])
    x.masked_fill_(torch.rand((n, vocab), generator=gen, device=DEVICE) < 0.01, -math.inf)  # (what a grammar forbids)
    s["logits"] = x.to(DTYPES[c["dtype"]])
    # log-probabilities that have been added up over some thirty tokens, the best first
    scores = torch.empty((requests, beams), device=DEVICE).normal_(0.0, 3.0, generator=gen) - 40.0
    s["scores"] = scores.sort(dim=1, descending=True).values.reshape(n).contiguous()
    lengths = _up(order.integers(10, 40, n).astype(np.float32))
    s["weights"] = (1.0 / lengths) if c["weighted"] else None
    s["ended"] = None
    if c["ended_percent"]:
        s["ended"] = (torch.rand(n, generator=gen, device=DEVICE) * 100 < c["ended_percent"]).int()
    s["end_token"] = 2
    shape = (requests, c["choices"])
    s["next_scores"] = torch.empty(shape, dtype=torch.float32, device=DEVICE)
    s["parents"] = torch.empty(shape, dtype=torch.int32, device=DEVICE)
    s["tokens"] = torch.empty(shape, dtype=torch.int32, device=DEVICE)


def _prepare_reorder(s, order):
    c = s["case"]
    n = c["groups"] * c["each"]
    # beams have parted since their prompts: half of their pages are still the same
    _, _, tokens = _lengths(c)
    half = dict(c, prefix_lo=1, prefix_hi=1)
    pages, table, lengths, refs = _tables(half, order)
    lengths[:] = tokens
    for g in range(c["groups"]):
        first = g * c["each"]
        common = tokens[first] // PAGE // 2
        refs[table[first + 1:first + c["each"], :common]] = 0
        table[first:first + c["each"], :common] = table[first, :common]
        refs[table[first, :common]] = c["each"]
    held = np.arange(table.shape[1])[None, :] < -(-lengths[:, None] // PAGE)
    refs[:] = np.bincount(table[held], minlength=pages)
    table[~held] = -1
    # the best beams have several children, the worst have none
    beam = np.sort((order.random((c["groups"], c["each"])) ** 1.5 * c["each"]).astype(np.int32), axis=1)
    s["parent_rows"] = _up((beam + c["each"] * np.arange(c["groups"], dtype=np.int32)[:, None]).reshape(-1).astype(np.int32))
    # the three tables in one buffer, and as they are before a step
    s["before"] = _up(np.concatenate([table.reshape(-1), lengths, refs]).astype(np.int32))
    s["now"] = s["before"].clone()
    s["table"] = s["now"][:table.size].view(table.shape)
    s["lengths"], s["refs"] = s["now"][table.size:table.size + n], s["now"][table.size + n:]
    s["slots"] = torch.arange(n, dtype=torch.int32, device=DEVICE)
    s["pages"] = pages
    # (a pool is never touched by this call)
    s["codes"] = torch.empty((1, pages, 1, 2, PAGE * 64), dtype=torch.uint8, device=DEVICE)
    s["scales"] = torch.empty((1, pages, 1, 2), dtype=torch.float32, device=DEVICE)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    order = np.random.default_rng([seed, 0x5348])
    s = dict(case=dict(case), call=case["call"])
    if case["call"] in ("shared", "sinks"):
        _prepare_attention(s, gen, order)
    elif case["call"] == "select":
        _prepare_select(s, gen, order)
    else:
        _prepare_reorder(s, order)
    return s


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _handles(s):
    """What a program makes once beside its buffers: the descriptions of cache and tables, and workspaces."""
    import paper_2602_01027_amd as S
    c, made = s["case"], {}
    new = lambda size: torch.empty(size, dtype=torch.uint8, device=DEVICE)  # noqa: E731
    if s["call"] == "select":
        made["workspace"] = new(S.sfmp_beam_select_workspace(c["groups"], c["each"], c["vocab"], c["choices"]))
        return made
    heads, dim = s["codes"].shape[2], s["codes"].shape[4] // PAGE
    layout = S.sfmp_kv_query(s["codes"].shape[1], heads, dim, c["format"], c["layers"])
    made["cache"] = S.DeviceKvCache(layout, s["codes"], s["scales"])
    made["tables"] = S.DeviceKvTables(s["table"], s["lengths"], s["refs"])
    if s["call"] == "reorder":
        return made
    sizes = (c["q_heads"], s["max_rows"], s["max_tokens"])
    batch = c["groups"] * c["each"]
    if s["call"] == "shared":
        made["plan"] = new(S.sfmp_kv_share_plan(layout, batch, s["total"], c["groups"], *sizes))
        made["workspace"] = new(S.sfmp_kv_attention_shared_workspace(layout, batch, s["total"], c["groups"], *sizes))
    else:
        made["workspace"] = new(S.sfmp_kv_attention_workspace(layout, batch, s["total"], *sizes))
    return made


def _run_own(s):
    import paper_2602_01027_amd as S
    if "handles" not in s:
        s["handles"] = _handles(s)
    m, c = s["handles"], s["case"]
    scale = 1.0 / math.sqrt(c["head_dim"])
    if s["call"] == "shared":
        masks = dict(window=c["window"], sinks=c["sinks"])
        S.sfmp_kv_share(m["cache"], m["tables"], s["slots"], s["row_start"], s["group_start"], s["total"], c["q_heads"],
                        s["max_rows"], s["max_tokens"], m["plan"], prefix=s["prefix"], **masks)
        for i in range(c["layers"]):
            S.sfmp_kv_attention_shared(m["cache"], i, m["tables"], s["slots"], s["row_start"], s["group_start"], s["q"][i],
                                       s["out"][i], s["max_rows"], s["max_tokens"], scale, m["plan"], m["workspace"],
                                       lse=s["lse"][i], **masks)
        return {"prefix": s["prefix"], "out": s["out"], "lse": s["lse"]}
    if s["call"] == "sinks":
        S.sfmp_kv_attention_sinks(m["cache"], 0, m["tables"], s["slots"], s["row_start"], s["q"][0], s["out"][0], s["max_rows"],
                                  s["max_tokens"], scale, m["workspace"], c["window"], c["sinks"], lse=s["lse"][0])
        return {"out": s["out"], "lse": s["lse"]}
    if s["call"] == "select":
        S.sfmp_beam_select(s["logits"], c["each"], s["scores"], s["weights"], s["ended"], s["end_token"], s["next_scores"],
                           s["parents"], s["tokens"], m["workspace"])
        return {"next_scores": s["next_scores"], "parents": s["parents"], "tokens": s["tokens"]}
    s["now"].copy_(s["before"])
    S.sfmp_kv_reorder(m["cache"], m["tables"], s["slots"], s["parent_rows"])
    return {"table": s["table"], "lengths": s["lengths"], "refs": s["refs"]}


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _values(case, codes):
    if case["format"] == "int8":
        return codes.to(torch.float32) - 128.0
    return codes.view(torch.float8_e4m3fn).to(torch.float32)


def _attend(s, layer):
    """Rows of all sequences over keys and values that are read for each of them."""
    c = s["case"]
    d, h, g = c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    length = s["lengths"].long()[s["slots"].long()]
    n, p = length.numel(), _pages_of(s["max_tokens"])
    ids = s["table"].long()[s["slots"].long()][:, :p].clamp(min=0)
    key = torch.arange(p * PAGE, device=DEVICE)
    written = (key[None, :] < length[:, None])[:, None, :, None]

    def dense(which):
        x = _values(c, s["codes"][layer, :, :, which][ids]) * s["scales"][layer, :, :, which][ids][..., None]  # [n, p, h, 64 d]
        x = x.view(n, p, h, PAGE, d) if which == 0 else x.view(n, p, h, d, PAGE).transpose(3, 4)
        return x.permute(0, 2, 1, 3, 4).reshape(n, h, p * PAGE, d).masked_fill_(~written, 0.0)

    rows = s["row_start"].diff().long()
    b = torch.repeat_interleave(torch.arange(n, device=DEVICE), rows, output_size=s["total"])
    i = torch.arange(s["total"], device=DEVICE) - s["row_start"].long()[b]
    q = torch.zeros((n, s["max_rows"], c["q_heads"], d), dtype=torch.float32, device=DEVICE)
    q[b, i] = s["q"][layer].to(torch.float32)
    place = torch.full((n, s["max_rows"]), -1, dtype=torch.long, device=DEVICE)
    place[b, i] = (length - rows)[b] + i
    q = q.view(n, -1, h, g, d).permute(0, 2, 1, 3, 4).reshape(n, h, -1, d)
    scores = torch.matmul(q, dense(0).transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    seen = key[None, None, :] <= place[:, :, None]
    if c["window"]:
        seen &= (key[None, None, :] > place[:, :, None] - c["window"]) | (key < c["sinks"])[None, None, :]
    scores.masked_fill_(~seen.repeat_interleave(g, dim=1)[:, None], -math.inf)
    m = scores.amax(dim=3, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    scores = scores.sub_(m).exp_()
    total = scores.sum(dim=3, keepdim=True)
    out = torch.where(total > 0, torch.matmul(scores, dense(1)) / total, 0.0)
    lse = (m + total.log())[..., 0]
    out = out.view(n, h, -1, g, d).permute(0, 2, 1, 3, 4).reshape(n, -1, c["q_heads"], d)
    lse = lse.view(n, h, -1, g).permute(0, 2, 1, 3).reshape(n, -1, c["q_heads"])
    return out[b, i].to(DTYPES[c["dtype"]]), lse[b, i].contiguous()


def _common(s):
    """Tokens in the whole pages that all sequences of a group hold first."""
    groups, each = s["case"]["groups"], s["case"]["each"]
    table = s["table"].view(groups, each, -1)
    whole = (s["lengths"].view(groups, each) // PAGE).amin(dim=1)
    same = (table == table[:, :1]).all(dim=1) & (torch.arange(table.shape[2], device=DEVICE)[None, :] < whole[:, None])
    return (PAGE * same.int().cumprod(dim=1).sum(dim=1)).int()


def _shared(s):
    made = [_attend(s, layer) for layer in range(s["case"]["layers"])]
    return {"prefix": _common(s), "out": [x[0] for x in made], "lse": [x[1] for x in made]}


def _sinks(s):
    out, lse = _attend(s, 0)
    return {"out": [out], "lse": [lse]}


def _select(s):
    c = s["case"]
    requests, beams, vocab = c["groups"], c["each"], c["vocab"]
    x = s["logits"].to(torch.float64)  # (ranks lie closer together than 32 bits tell apart)
    x = torch.where(torch.isnan(x), -math.inf, x)
    m = x.amax(dim=1, keepdim=True)
    y = torch.where(x == m, 0.0, x - m)
    y -= y.exp().sum(dim=1, keepdim=True).log()
    y = torch.where(x == -math.inf, -math.inf, y)
    value = s["scores"].double()[:, None] + y
    if s["ended"] is not None:
        stays = torch.full_like(value[:1], -math.inf)
        stays[0, s["end_token"]] = 0.0
        value = torch.where(s["ended"][:, None] != 0, s["scores"].double()[:, None] + stays, value)
    key = value if s["weights"] is None else value * s["weights"].double()[:, None]
    order = torch.sort(key.view(requests, beams * vocab), dim=1, descending=True, stable=True).indices[:, :c["choices"]]
    best = value.view(requests, -1).gather(1, order)
    none = best == -math.inf
    row = order // vocab + beams * torch.arange(requests, device=DEVICE)[:, None]
    return {"next_scores": best.float(), "parents": torch.where(none, -1, row).int(),
            "tokens": torch.where(none, -1, order % vocab).int()}


def _reorder(s):
    s["now"].copy_(s["before"])
    table, lengths, refs = s["table"], s["lengths"], s["refs"]
    parents, place = s["parent_rows"].long(), torch.arange(table.shape[1], device=DEVICE)[None, :]
    held = place < _pages_of(lengths)[:, None]
    taken = held[parents]
    rows = torch.where(taken, table[parents], table)
    refs += torch.bincount(rows[taken].long(), minlength=refs.numel()).int() - torch.bincount(table[held].long(), minlength=refs.numel()).int()
    table.copy_(rows)
    lengths.copy_(lengths[parents])
    return {"table": table, "lengths": lengths, "refs": refs}


def run(state):
    if own:
        return _run_own(state)
    return {"shared": _shared, "sinks": _sinks, "select": _select, "reorder": _reorder}[state["call"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def _keys_read(case):
    """Cached tokens that a pass has to read (common pages once for their group), and pairs of row and key."""
    prompts, rows, tokens = _lengths(case)
    read = pairs = 0
    for g, p in enumerate(prompts):
        common = p // PAGE * PAGE if case["each"] > 1 else 0
        members = range(g * case["each"], (g + 1) * case["each"])
        lowest = []  # the first token that a sequence's window reaches back to
        for b in members:
            w, k = case["window"] or tokens[b], case["sinks"] if case["window"] else 0
            first = max(0, tokens[b] - rows[b] - w + 1)
            lowest.append(first)
            read += max(0, tokens[b] - max(first, common)) + max(0, min(k, first) - common)
            at = np.arange(tokens[b] - rows[b], tokens[b])
            pairs += int((np.minimum(at + 1, w) + np.minimum(np.maximum(at + 1 - w, 0), k)).sum())
        first = min(lowest)
        k = case["sinks"] if case["window"] else 0
        read += max(0, common - first) + min(k, first, common)
    return read, pairs


def work(case):
    h, d, size = case["kv_heads"], case["head_dim"], 4 if case["dtype"] == "fp32" else 2
    if case["call"] in ("shared", "sinks"):
        read, pairs = _keys_read(case)
        rows = sum(_lengths(case)[1])
        nbytes = read * h * 2 * d + _pages_of(read) * h * 2 * 4 + rows * case["q_heads"] * (2 * d * size + 4)
        return {"bytes": nbytes * case["layers"], "flops": 4 * pairs * case["q_heads"] * d * case["layers"]}
    if case["call"] == "select":
        n = case["groups"] * case["each"] * case["vocab"]
        return {"bytes": n * size, "flops": 4 * n}
    tokens = _lengths(case)[2]
    # rows read and written, lengths, and the holders of the pages that change hands
    return {"bytes": 4 * sum(3 * _pages_of(t) + 3 for t in tokens), "flops": 0}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _held(case, codes):
    if case["format"] == "int8":
        return codes.double() - 128
    return codes.view(torch.float8_e4m3fn).double()


def _exact_attend(s, layer):
    c = s["case"]
    d, h, group, start = c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"], s["row_start"].tolist()
    outs, lses = [], []
    for b in range(len(start) - 1):
        t, n = int(s["lengths"][b]), start[b + 1] - start[b]
        ids = s["table"][b, :_pages_of(t)].long()
        q = s["q"][layer][start[b]:start[b + 1]].double()
        at = torch.arange(t - n, t, device=DEVICE)[:, None]
        key = torch.arange(t, device=DEVICE)[None, :]
        seen = key <= at
        if c["window"]:
            seen = seen & ((at - key < c["window"]) | (key < c["sinks"]))
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float64, device=DEVICE)
        for head in range(h):
            block, scale = s["codes"][layer, ids, head], s["scales"][layer, ids, head].double()
            k = (_held(c, block[:, 0].contiguous()).view(-1, PAGE, d) * scale[:, 0, None, None]).reshape(-1, d)[:t]
            v = (_held(c, block[:, 1].contiguous()).view(-1, d, PAGE) * scale[:, 1, None, None]).transpose(1, 2).reshape(-1, d)[:t]
            for i in range(head * group, (head + 1) * group):
                z = q[:, i] @ k.t().contiguous() / math.sqrt(d)
                z = torch.where(seen, z, -math.inf)
                lse[:, i] = torch.logsumexp(z, dim=1)
                out[:, i] = torch.exp(z - lse[:, i:i + 1]) @ v.contiguous()
        outs.append(out)
        lses.append(lse)
    return torch.cat(outs), torch.cat(lses)


def _exact_select(s):
    c = s["case"]
    best = []
    for r in range(c["groups"]):
        values, keys = [], []
        for b in range(r * c["each"], (r + 1) * c["each"]):
            z = torch.log_softmax(s["logits"][b].double(), dim=0) + float(s["scores"][b])
            if s["ended"] is not None and int(s["ended"][b]):
                z = s["scores"][b:b + 1].double()
            values.append(z)
            keys.append(z if s["weights"] is None else z * float(s["weights"][b]))
        top = torch.cat(keys).topk(c["choices"]).indices
        best.append(torch.cat(values)[top])
    return {"next_scores": torch.stack(best), "parents": None, "tokens": None}


def exact(case, seed):
    if case["call"] == "reorder":
        return None  # (rows are moved, nothing is computed)
    s = prepare(case, seed)
    if case["call"] == "select":
        return _exact_select(s)
    made = [_exact_attend(s, layer) for layer in range(case["layers"])]
    found = {"out": [x[0] for x in made], "lse": [x[1] for x in made]}
    return dict(found, prefix=None) if case["call"] == "shared" else found
