"""Operator cases: the calls that a program serving decoder models makes around the linears, over the sizes it makes them
at.  Four operators, in seven kinds of case:

  attend   one `window_attention` call: a sliding window and a few first tokens that stay visible, over a paged cache.  One
           new token per sequence (a decoding step), several (a chunk of a prompt, a mixed batch), or whole prompts.
  append   one `cache_append` call: the keys and values of new tokens, as they lie in the QKV projection's output, into the
           pages of their sequences.
  fork     one `cache_free` and one `cache_fork` call: a beam search's step, which drops the beams that lost and forks the
           ones that won, over the caches of all layers.
  admit    one `cache_free` and one `cache_reserve` call: finished sequences leave a batch and new ones take their places.
  compact  one `cache_compact` call: the pages in use move to the lowest numbers, in the caches of all layers.
  copy     one `cache_copy_pages` call: a list of pages copied in the caches of all layers.
  logits   one `process_logits` call: penalties for repeated tokens, biases, a grammar's mask and the best token.

Head layouts are those of the 3B- and 8B-class decoders that the tests and the benchmark use, and generic ones.  `draw`
spreads sizes, ragged ones among them, over the same ranges.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One conversation's decoding step in a small model with a short window: latency is all there is.
        dict(name="attend_step_1", kind="attend", seqs=1, min_len=700, max_len=700, min_new=1, max_new=1, q_heads=8, kv_heads=2,
             dim=64, page=16, window=512, sinks=4, dtype="f16"),
        # A server's decoding step: 48 conversations, up to 30000 tokens long, 3B-class heads, a window of 4096 tokens.
        dict(name="attend_step_48", kind="attend", seqs=48, min_len=300, max_len=30000, min_new=1, max_new=1, q_heads=24, kv_heads=8,
             dim=128, page=16, window=4096, sinks=4, dtype="f16"),
        # A mixed batch: decoding sequences beside chunks of prompts, 8B-class heads, bfloat16.
        dict(name="attend_mixed_12", kind="attend", seqs=12, min_len=200, max_len=6000, min_new=1, max_new=1500, q_heads=32, kv_heads=8,
             dim=128, page=32, window=1024, sinks=4, dtype="bf16"),
        # The largest: a whole 8192-token prompt, 8B-class heads, a window of 4096 tokens.
        dict(name="attend_prompt_8192", kind="attend", seqs=1, min_len=8192, max_len=8192, min_new=8192, max_new=8192, q_heads=32,
             kv_heads=8, dim=128, page=16, window=4096, sinks=4, dtype="f16"),
        # One layer's new keys and values in a decoding step of 48 sequences.
        dict(name="append_step_48", kind="append", seqs=48, min_len=300, max_len=6000, min_new=1, max_new=1, q_heads=24, kv_heads=8,
             dim=128, page=16, dtype="f16"),
        # One layer's keys and values of five prompts.
        dict(name="append_prompt_5", kind="append", seqs=5, min_len=700, max_len=9001, min_new=700, max_new=9001, q_heads=32,
             kv_heads=8, dim=128, page=16, dtype="bf16"),
        # A beam search's step: 12 prompts with 4 beams each, in the key and value caches of 16 layers.
        dict(name="fork_12x4", kind="fork", seqs=12, beams=4, min_len=150, max_len=2000, kv_heads=8, dim=128, page=16, caches=32,
             dtype="f16"),
        # 40 of 256 sequences end and 40 new ones take their places.
        dict(name="admit_40_of_256", kind="admit", seqs=256, change=40, min_len=100, max_len=4000, page=16),
        # A fragmented cache of 2048 pages, 55% in use, in the key and value caches of 8 layers.
        dict(name="compact_2048", kind="compact", pages=2048, use=0.55, kv_heads=8, dim=128, page=16, caches=16, dtype="f16"),
        # One sequence's next token from a 128256-word vocabulary, under a grammar.
        dict(name="logits_1", kind="logits", rows=1, vocab=128256, history=600, bias=8, allow=0.02, dtype="f16"),
        # A batch of 48 sequences with longer histories.
        dict(name="logits_48", kind="logits", rows=48, vocab=128256, history=6000, bias=32, allow=0.4, dtype="f16"),
        # A large batch in 32 bits, with a vocabulary whose rows do not fall on 16-byte boundaries.
        dict(name="logits_256_f32", kind="logits", rows=256, vocab=100277, history=2000, bias=0, allow=0.9, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["attend"] * 5 + ["append"] * 2 + ["fork", "admit", "compact", "copy"] + ["logits"] * 3)
    while True:
        kv = rng.choice([1, 2, 4, 8])
        heads = dict(q_heads=kv * rng.randint(1, 8), kv_heads=kv, dim=rng.choice([64, 128, 128]))
        half = rng.choice(["f16", "bf16"])
        page = rng.choice([8, 16, 16, 32, 64])
        if kind == "attend":
            form = rng.choice(["step", "step", "mixed", "prompt"])
            top = _log_int(rng, 40, 32768) if form == "step" else _log_int(rng, 40, 8192)
            case = dict(kind=kind, seqs=_log_int(rng, 1, 64) if form == "step" else _log_int(rng, 1, 16),
                        min_len=max(1, top // rng.randint(1, 30)), max_len=top, min_new=1, max_new=1, page=page, dtype=half,
                        window=rng.choice([_log_int(rng, 32, 8192), _log_int(rng, 32, 8192), top]),
                        sinks=rng.choice([0, 4, rng.randint(1, 70)]), **heads)
            if form == "mixed":
                case["max_new"] = rng.choice([rng.randint(2, 8), _log_int(rng, 8, 2048)])
            elif form == "prompt":
                case["min_new"], case["max_new"] = case["min_len"], case["max_len"]
        elif kind == "append":
            top = _log_int(rng, 40, 16384)
            case = dict(kind=kind, seqs=_log_int(rng, 1, 64), min_len=max(1, top // rng.randint(1, 30)), max_len=top, min_new=1,
                        max_new=rng.choice([1, _log_int(rng, 2, 8192)]), page=page, dtype=half, **heads)
        elif kind == "fork":
            top = _log_int(rng, 20, 4000)
            case = dict(kind=kind, seqs=_log_int(rng, 1, 24), beams=rng.randint(2, 6), min_len=max(1, top // rng.randint(1, 20)), max_len=top,
                        kv_heads=kv, dim=heads["dim"], page=page, caches=2 * rng.randint(1, 32), dtype=half)
        elif kind == "admit":
            seqs, top = _log_int(rng, 2, 1024), _log_int(rng, 40, 8192)
            case = dict(kind=kind, seqs=seqs, change=rng.randint(1, seqs), min_len=max(1, top // rng.randint(1, 30)), max_len=top, page=page)
        elif kind == "compact":
            case = dict(kind=kind, pages=_log_int(rng, 50, 8192), use=round(rng.uniform(0.1, 0.95), 2), kv_heads=kv, dim=heads["dim"], page=page,
                        caches=2 * rng.randint(1, 32), dtype=half)
        elif kind == "copy":
            pages = _log_int(rng, 50, 8192)
            case = dict(kind=kind, pages=pages, count=_log_int(rng, 1, pages // 2), kv_heads=kv, dim=heads["dim"], page=page,
                        caches=2 * rng.randint(1, 32), dtype=half)
        else:
            case = dict(kind=kind, rows=_log_int(rng, 1, 256), vocab=_log_int(rng, 500, 200000), history=_log_int(rng, 1, 16000),
                        bias=rng.choice([0, rng.randint(1, 300)]), allow=round(rng.uniform(0.001, 1.0), 3), dtype=rng.choice(["f16", "bf16", "f32"]))
        if _bounded(case):
            return case


def _bounded(case):
    """Whether a drawn case costs no more than the largest listed one, and its inputs and the plain form's intermediates stay small."""
    w = work(case)
    if max(w["bytes"] / 4e12, w["flops"] / 4e14) > 1e-3:
        return False
    kind = case["kind"]
    if kind == "attend":
        lens, new = _lens(case)
        keys = min(max(lens), case["sinks"] + case["window"] + max(new))
        return (case["seqs"] * max(new) * case["q_heads"] * keys <= 5 << 29 and case["seqs"] * keys * case["kv_heads"] * case["dim"] <= 1 << 30
                and sum(lens) * case["kv_heads"] * case["dim"] <= 1 << 29)
    if kind == "append":
        return sum(_lens(case)[0]) * case["kv_heads"] * case["dim"] <= 1 << 28
    if kind in ("fork", "compact", "copy"):
        pages = case["pages"] if kind != "fork" else _fork_pages(case)
        return pages * case["caches"] * case["kv_heads"] * case["page"] * case["dim"] <= 1 << 29
    return True


# ------------------------------------------------------------------ inputs


def _lens(case):
    """Tokens in the cache, the new ones among them, and new tokens of every sequence; the longest of each is the bound.  The same
    for every seed, as the case's work is."""
    rng = random.Random(case["seqs"] * 1000003 + case["max_len"])
    lens = [min(case["max_len"], max(case["min_len"], _log_int(rng, case["min_len"], case["max_len"]))) for _ in range(case["seqs"])]
    lens[rng.randrange(len(lens))] = case["max_len"]
    low, high = case["min_new"], case["max_new"]
    if (low, high) == (case["min_len"], case["max_len"]):
        return lens, list(lens)
    return lens, [min(n, max(low, _log_int(rng, low, high))) for n in lens]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, dtype, *shape):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for at in range(0, flat.numel(), 1 << 28):
        part = flat[at:at + (1 << 28)]
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda"))
    return out


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _visible_pages(case, length, new):
    """The table entries of a sequence that hold a token which one of its new tokens sees."""
    page, first = case["page"], max(0, length - new - case.get("window", length) + 1)
    return [e for e in range(-(-length // page)) if e * page < case.get("sinks", 0) or e * page + page > first]


def _table(case, g, lens, new):
    """Pages in a random order, as in a cache that has served and freed many sequences; -1 where a sequence has no page, in a
    window's case also where its page has been freed because no new token sees it."""
    used = [_visible_pages(case, n, m) for n, m in zip(lens, new)]
    pages = sum(map(len, used))
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(-(-n // case["page"]) for n in lens)), -1, dtype=torch.int32, device="cuda")
    rows = _int32([i for i, e in enumerate(used) for _ in e]).long()
    table[rows, _int32([x for e in used for x in e]).long()] = order
    return table, pages


def _starts(new):
    at = [0]
    for n in new:
        at.append(at[-1] + n)
    return at


def _fork_pages(case):
    lens = _lens(dict(case, min_new=1, max_new=1))[0]
    return sum(-(-n // case["page"]) + case["beams"] for n in lens) + 8


def prepare(case, seed):
    g = _generator(seed)
    kind = case["kind"]
    d = dict(kind=kind)
    dtype = DTYPES[case.get("dtype", "f16")]
    if kind in ("attend", "append"):
        lens, new = _lens(case)
        table, pages = _table(case, g, lens, new)
        shape = (pages, case["kv_heads"], case["page"], case["dim"])
        starts = _starts(new)
        d.update(k_cache=_normal(g, dtype, *shape), v_cache=_normal(g, dtype, *shape), table=table, lens=_int32(lens),
                 starts=_int32(starts) if max(new) > 1 else None, max_new=max(new), max_len=max(lens))
        # The queries, keys and values of a token lie side by side, as the QKV projection leaves them.
        hq, hkv, dim = case["q_heads"], case["kv_heads"], case["dim"]
        qkv = _normal(g, dtype, starts[-1], hq + 2 * hkv, dim)
        if kind == "attend":
            d.update(q=qkv[:, :hq], window=case["window"], sinks=case["sinks"], scale=1.0 / math.sqrt(dim),
                     out=torch.empty((starts[-1], hq, dim), dtype=dtype, device="cuda"))
            if own:
                from paper_2412_15803_amd import wq

                d["workspace"] = wq.window_workspace(d["q"], hkv, len(lens), d["max_len"], d["window"], d["sinks"], d["max_new"])
        else:
            d.update(k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:])
    elif kind in ("fork", "compact", "copy"):
        pages = _fork_pages(case) if kind == "fork" else case["pages"]
        shape = (pages, case["kv_heads"], case["page"], case["dim"])
        d["caches"] = [_normal(g, dtype, *shape) for _ in range(case["caches"])]
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        if kind == "copy":
            d.update(src=order[:case["count"]].contiguous(), dst=order[case["count"]:2 * case["count"]].contiguous())
        elif kind == "fork":
            # Sequence i's row is followed by those of its other beams, each with the first one's full pages and a last page of its own.
            beams, page = case["beams"], case["page"]
            lens = _lens(dict(case, min_new=1, max_new=1))[0]
            table = torch.full((len(lens) * beams, -(-max(lens) // page)), -1, dtype=torch.int32)
            refs = torch.zeros(pages, dtype=torch.int32)
            host, at = order.cpu(), 0
            for i, n in enumerate(lens):
                full, need = n // page, -(-n // page)
                rows = table[i * beams:(i + 1) * beams]
                rows[:, :full] = host[at:at + full]
                refs[host[at:at + full].long()] = beams
                at += full
                if need > full:
                    rows[:, full] = host[at:at + beams]
                    refs[host[at:at + beams].long()] = 1
                    at += beams
            d.update(table=table.cuda(), refs=refs.cuda(), lens=_int32([n for n in lens for _ in range(beams)]))
            d.update(src=_int32([i * beams for i in range(len(lens)) for _ in range(beams - 1)]),
                     dst=_int32([i * beams + b for i in range(len(lens)) for b in range(1, beams)]))
        else:
            live = max(1, int(pages * case["use"]))
            width = max(1, live // 24)
            refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
            refs[order[:live].long()] = 1
            table = torch.full((-(-live // width), width), -1, dtype=torch.int32, device="cuda")
            table.view(-1)[:live] = order[:live]
            # Some sequences share their first page.
            if table.shape[0] > 2:
                refs[table[0, 0].long()] += 1
                refs[table[1, 0].long()] -= 1
                table[1, 0] = table[0, 0]
            d.update(table=table, refs=refs, new_table=torch.empty_like(table), new_refs=torch.empty_like(refs), live=_int32([0]))
        if own:
            from paper_2412_15803_amd import wq

            d["cache_set"] = wq.cache_set(d["caches"])
            if kind != "copy":
                d["workspace"] = wq.page_workspace(pages, d["table"].shape[0], "cuda")
        d["shortfall"] = _int32([0])
    elif kind == "admit":
        rng = random.Random(case["seqs"] * 1000003 + case["change"])
        page, seqs = case["page"], case["seqs"]
        lens = _lens(dict(case, min_new=1, max_new=1))[0]
        after = list(lens)
        changed = sorted(rng.sample(range(seqs), case["change"]))
        for i in changed:
            after[i] = min(case["max_len"], max(case["min_len"], _log_int(rng, case["min_len"], case["max_len"])))
        need = [-(-n // page) for n in lens]
        pages = sum(max(a, -(-b // page)) for a, b in zip(need, after)) + 64
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        table = torch.full((seqs, -(-case["max_len"] // page)), -1, dtype=torch.int32, device="cuda")
        rows, entries = _int32([i for i, n in enumerate(need) for _ in range(n)]).long(), _int32([e for n in need for e in range(n)]).long()
        table[rows, entries] = order[:sum(need)]
        refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
        refs[order[:sum(need)].long()] = 1
        d.update(table=table, refs=refs, page=page, lens=_int32(lens), after=_int32(after), shortfall=_int32([0]), ended=_int32(changed),
                 before=_int32([0 if i in set(changed) else n for i, n in enumerate(lens)]))
        if own:
            from paper_2412_15803_amd import wq

            d["workspace"] = wq.page_workspace(pages, seqs, "cuda")
    else:
        rows, vocab, top = case["rows"], case["vocab"], case["history"]
        rng = random.Random(rows * 1000003 + top)
        lens = [min(top, max(1, _log_int(rng, max(1, top // 20), top))) for _ in range(rows)]
        # Words of a text come by a power law: few make up most of it.
        words = torch.rand((rows, top), generator=g, device="cuda").pow_(4).mul_(vocab).to(torch.int32).clamp_(max=vocab - 1)
        bits = torch.rand((rows, -(-vocab // 32), 32), generator=g, device="cuda").lt_(case["allow"]).to(torch.int64)
        packed = (bits << torch.arange(32, device="cuda")).sum(-1)
        d.update(logits=_normal(g, dtype, rows, vocab).mul_(3.0), history=words, history_lens=_int32(lens),
                 prompt_lens=_int32([n // 3 for n in lens]), mask=torch.where(packed >= 1 << 31, packed - (1 << 32), packed).to(torch.int32),
                 repetition=torch.rand(rows, generator=g, device="cuda").mul_(0.3).add_(1.0), frequency=torch.rand(rows, generator=g, device="cuda").mul_(0.5),
                 presence=torch.rand(rows, generator=g, device="cuda").mul_(0.5), out=torch.empty((rows, vocab), dtype=dtype, device="cuda"),
                 token=torch.empty(rows, dtype=torch.int32, device="cuda"), bias_ids=None, bias_values=None)
        if case["bias"]:
            # Distinct words of a row, a stride apart from a place of the row's own.
            count = min(case["bias"], vocab)
            first = torch.randint(vocab, (rows, 1), generator=g, device="cuda")
            d["bias_ids"] = ((first + torch.arange(count, device="cuda") * max(1, vocab // count)) % vocab).to(torch.int32)
            d["bias_values"] = torch.randn((rows, count), generator=g, device="cuda").mul_(5.0)
        if own:
            from paper_2412_15803_amd import wq

            d["workspace"] = wq.logits_workspace(d["logits"])
    return d


# --------------------------------------------------------------------- run


def run(d):
    return (_run_own if own else _PLAIN[d["kind"]])(d)


def _run_own(d):
    from paper_2412_15803_amd import wq

    kind = d["kind"]
    if kind == "attend":
        wq.window_attention(d["q"], d["k_cache"], d["v_cache"], d["table"], d["lens"], d["out"], d["scale"], d["max_len"], d["window"],
                            sinks=d["sinks"], q_starts=d["starts"], max_query_len=d["max_new"], workspace=d["workspace"])
        return d["out"]
    if kind == "append":
        wq.cache_append(d["k"], d["v"], d["k_cache"], d["v_cache"], d["table"], d["lens"], q_starts=d["starts"])
        return dict(k_cache=d["k_cache"], v_cache=d["v_cache"])
    if kind == "fork":
        page = d["caches"][0].shape[2]
        wq.cache_free(d["table"], d["refs"], d["lens"], d["dst"], page)
        wq.cache_fork(d["cache_set"], d["table"], d["refs"], d["lens"], d["src"], d["dst"], d["shortfall"], workspace=d["workspace"])
        return dict(caches=d["caches"], table=d["table"], refs=d["refs"], lens=d["lens"], shortfall=d["shortfall"])
    if kind == "admit":
        wq.cache_free(d["table"], d["refs"], d["lens"], d["ended"], d["page"])
        wq.cache_reserve(d["table"], d["refs"], d["before"], d["after"], d["page"], d["shortfall"], workspace=d["workspace"])
        return dict(table=d["table"], refs=d["refs"], shortfall=d["shortfall"])
    if kind == "compact":
        wq.cache_compact(d["cache_set"], d["table"], d["refs"], d["new_table"], d["new_refs"], d["live"], workspace=d["workspace"])
        return dict(caches=d["caches"], table=d["new_table"], refs=d["new_refs"], live=d["live"])
    if kind == "copy":
        wq.cache_copy_pages(d["cache_set"], d["src"], d["dst"])
        return d["caches"]
    wq.process_logits(d["logits"], d["out"], token=d["token"], mask=d["mask"], history=d["history"], history_lens=d["history_lens"],
                      prompt_lens=d["prompt_lens"], repetition=d["repetition"], frequency=d["frequency"], presence=d["presence"],
                      bias_ids=d["bias_ids"], bias_values=d["bias_values"], workspace=d["workspace"])
    return dict(out=d["out"], token=d["token"])


# ------------------------------------------------------------- plain forms


def _token_places(d, total):
    """Sequence and place in it of every new token."""
    lens = d["lens"].long()
    if d["starts"] is None:
        return torch.arange(total, device="cuda"), lens - 1, torch.zeros(total, dtype=torch.long, device="cuda"), torch.ones_like(lens)
    starts = d["starts"].long()
    token = torch.arange(total, device="cuda")
    seq = torch.searchsorted(starts, token, right=True) - 1
    new = starts[1:] - starts[:-1]
    nth = token - starts[seq]
    return seq, (lens - new)[seq] + nth, nth, new


def _plain_attend(d):
    q, table, page = d["q"], d["table"], d["k_cache"].shape[2]
    total, hq, dim = q.shape
    hkv, window, sinks = d["k_cache"].shape[1], d["window"], d["sinks"]
    seq, place, nth, new = _token_places(d, total)
    lens = d["lens"].long()
    # The tokens of each sequence that any of its new tokens can see: the sinks, then the rest from the oldest's window on.
    first = (lens - new - window + 1).clamp(min=sinks)
    count = min(d["max_len"], sinks + window + d["max_new"])
    tokens = torch.arange(sinks + count, device="cuda").expand(len(lens), -1)
    tokens = torch.where(tokens < sinks, tokens, tokens - sinks + first[:, None])
    held = tokens < lens[:, None]
    at = tokens.clamp(max=table.shape[1] * page - 1)
    pages = table.long().gather(1, at // page).clamp(min=0)
    k = d["k_cache"][pages, :, at % page].float().permute(0, 2, 1, 3)  # [sequence, kv head, token, dim]
    v = d["v_cache"][pages, :, at % page].float().permute(0, 2, 1, 3).contiguous()
    rows = torch.zeros((len(lens), d["max_new"], hq, dim), device="cuda")
    rows[seq, nth] = q.float()
    rows = rows.view(len(lens), d["max_new"], hkv, hq // hkv, dim).permute(0, 2, 3, 1, 4).reshape(len(lens), hkv, -1, dim)
    s = torch.matmul(rows, k.transpose(2, 3)).mul_(d["scale"]).view(len(lens), hkv, hq // hkv, d["max_new"], -1)
    p = (lens - new)[:, None] + torch.arange(d["max_new"], device="cuda")
    seen = held[:, None] & (tokens[:, None] <= p[:, :, None]) & ((tokens[:, None] < sinks) | (tokens[:, None] > p[:, :, None] - window))
    s.masked_fill_(~seen[:, None, None], -math.inf)
    s = s.sub_(s.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(s.view(len(lens), hkv, -1, s.shape[-1]), v).view(s.shape[:-1] + (dim,)).div_(s.sum(-1, keepdim=True))
    return o.permute(0, 3, 1, 2, 4).reshape(len(lens), d["max_new"], hq, dim)[seq, nth].to(q.dtype)


def _plain_append(d):
    page = d["k_cache"].shape[2]
    seq, place, _, _ = _token_places(d, d["k"].shape[0])
    pages = d["table"].long()[seq, place // page]
    d["k_cache"][pages, :, place % page] = d["k"]
    d["v_cache"][pages, :, place % page] = d["v"]
    return dict(k_cache=d["k_cache"], v_cache=d["v_cache"])


def _plain_free_all(table, refs, seqs):
    rows = table[seqs.long()]
    refs.index_add_(0, rows.clamp(min=0).view(-1).long(), -(rows >= 0).view(-1).to(torch.int32))
    table[seqs.long()] = -1


def _plain_fork(d):
    table, refs, lens, src, dst = d["table"], d["refs"], d["lens"], d["src"].long(), d["dst"].long()
    page = d["caches"][0].shape[2]
    _plain_free_all(table, refs, dst)
    length = lens[src].long()
    full, part = length // page, length % page
    entry = torch.arange(table.shape[1], device="cuda")
    tail = table[src].gather(1, full.clamp(max=table.shape[1] - 1)[:, None]).squeeze(1).long()
    own_page = (part > 0) & (tail >= 0)
    free = torch.nonzero(refs == 0).squeeze(1)
    rank = own_page.long().cumsum(0) - 1
    missing = own_page.sum() - len(free)
    d["shortfall"].copy_(missing.clamp(min=0))
    if missing <= 0:
        fresh = free[rank.clamp(min=0)]
        rows = torch.where(entry < full[:, None], table[src], -1)
        refs.index_add_(0, rows.clamp(min=0).view(-1).long(), (rows >= 0).view(-1).to(torch.int32))
        rows = torch.where((entry == full[:, None]) & own_page[:, None], fresh[:, None].to(torch.int32), rows)
        table[dst] = rows
        lens[dst] = lens[src]
        fresh, tail, part = fresh[own_page], tail[own_page], part[own_page]
        refs[fresh] = 1
        slot = (torch.arange(page, device="cuda") < part[:, None])[:, None, :, None]
        for cache in d["caches"]:
            cache[fresh] = torch.where(slot, cache[tail], cache[fresh])
    return dict(caches=d["caches"], table=table, refs=refs, lens=lens, shortfall=d["shortfall"])


def _plain_admit(d):
    table, refs, page = d["table"], d["refs"], d["page"]
    _plain_free_all(table, refs, d["ended"])
    entry = torch.arange(table.shape[1], device="cuda")
    low, high = -(-d["before"] // page), -(-d["after"] // page)
    want = (entry >= low[:, None]) & (entry < high[:, None]) & (table < 0)
    free = torch.nonzero(refs == 0).squeeze(1)
    count = want.sum()
    d["shortfall"].copy_((count - len(free)).clamp(min=0))
    if count <= len(free):
        rank = (want.view(-1).long().cumsum(0) - 1).clamp(min=0).view(want.shape)
        table.copy_(torch.where(want, free[rank].to(torch.int32), table))
        refs[free[:count]] = 1
    return dict(table=table, refs=refs, shortfall=d["shortfall"])


def _plain_compact(d):
    table, refs = d["table"], d["refs"]
    number = torch.arange(len(refs), device="cuda")
    live = refs > 0
    count = live.sum()
    src, dst = number[live & (number >= count)], number[~live & (number < count)]
    moved = number.clone()
    moved[src] = dst
    d["live"].copy_(count)
    d["new_table"].copy_(torch.where(table >= 0, moved[table.clamp(min=0).long()].to(torch.int32), table))
    d["new_refs"].copy_(refs)
    d["new_refs"][dst] = refs[src]
    d["new_refs"][src] = 0
    for cache in d["caches"]:
        cache[dst] = cache[src]
    return dict(caches=d["caches"], table=d["new_table"], refs=d["new_refs"], live=d["live"])


def _plain_copy(d):
    src, dst = d["src"].long(), d["dst"].long()
    for cache in d["caches"]:
        cache[dst] = cache[src]
    return d["caches"]


def _plain_logits(d):
    x = d["logits"].float()
    rows, vocab = x.shape
    place = torch.arange(d["history"].shape[1], device="cuda")
    known = place < d["history_lens"][:, None]
    words = d["history"].long()
    seen = torch.zeros_like(x).scatter_add_(1, words, known.float()) > 0
    count = torch.zeros_like(x).scatter_add_(1, words, (known & (place >= d["prompt_lens"][:, None])).float())
    r = d["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - d["frequency"][:, None] * count
    x = x - d["presence"][:, None] * (count > 0)
    if d["bias_ids"] is not None:
        x = x.scatter_add(1, d["bias_ids"].long(), d["bias_values"])
    word = torch.arange(vocab, device="cuda")
    allowed = (d["mask"][:, word // 32] >> (word % 32).to(torch.int32)) & 1 != 0
    x = torch.where(allowed, x, -math.inf)
    first = torch.where(allowed & (x == x.amax(-1, keepdim=True)), word, vocab).amin(-1)
    return dict(out=x.to(d["out"].dtype), token=torch.where(first < vocab, first, -1).to(torch.int32))


_PLAIN = dict(attend=_plain_attend, append=_plain_append, fork=_plain_fork, admit=_plain_admit, compact=_plain_compact, copy=_plain_copy,
              logits=_plain_logits)


# -------------------------------------------------------------------- work


def _seen(place, window, sinks):
    """Tokens that the token at `place` sees."""
    return min(place + 1, window) + max(0, min(sinks, place - window + 1))


def work(case):
    kind = case["kind"]
    if kind == "attend":
        lens, new = _lens(case)
        window, sinks, per = case["window"], case["sinks"], case["q_heads"] * case["dim"]
        pairs = sum(_seen(p, window, sinks) for n, m in zip(lens, new) for p in range(n - m, n))
        first = [max(0, n - m - window + 1) for n, m in zip(lens, new)]
        keys = sum(n - f + min(sinks, f) for n, f in zip(lens, first))
        return dict(bytes=4 * keys * case["kv_heads"] * case["dim"] + 4 * sum(new) * per + 4 * (keys // case["page"] + 3 * len(lens)),
                    flops=4 * pairs * per)
    if kind == "append":
        lens, new = _lens(case)
        return dict(bytes=8 * sum(new) * case["kv_heads"] * case["dim"] + 4 * (sum(new) // case["page"] + 3 * len(lens)), flops=0)
    if kind in ("fork", "copy", "compact"):
        one = case["caches"] * case["kv_heads"] * case["dim"] * 4  # a token copied in every cache
        if kind == "copy":
            return dict(bytes=case["count"] * (case["page"] * one + 8), flops=0)
        if kind == "compact":
            # A share of the pages in use lies above their number: as many as lie free below it.
            live = max(1, int(case["pages"] * case["use"]))
            return dict(bytes=int(live * (1 - live / case["pages"])) * case["page"] * one + 8 * case["pages"] + 8 * live, flops=0)
        lens = _lens(dict(case, min_new=1, max_new=1))[0]
        entries = sum(-(-n // case["page"]) for n in lens) * (case["beams"] - 1)
        return dict(bytes=sum(n % case["page"] for n in lens) * (case["beams"] - 1) * one + 24 * entries, flops=0)
    if kind == "admit":
        pages = sum(-(-n // case["page"]) for n in _lens(dict(case, min_new=1, max_new=1))[0])
        return dict(bytes=4 * pages + 24 * pages * case["change"] // case["seqs"], flops=0)
    rows, vocab, size = case["rows"], case["vocab"], DTYPES[case["dtype"]].itemsize
    return dict(bytes=rows * (2 * vocab * size + vocab // 8 + 4 * case["history"] // 2 + 8 * case["bias"]), flops=4 * rows * vocab)


# ----------------------------------------------------------------- 64 bits


def exact(case, seed):
    d = prepare(case, seed)
    if case["kind"] == "attend":
        return _exact_attend(case, d)
    return _exact_logits(d) if case["kind"] == "logits" else _exact_pages(case, d)


def _exact_pages(case, d):
    """Tables and counts walked entry by entry on the host; page by page copies."""
    kind = case["kind"]
    if kind == "append":
        out = dict(k_cache=d["k_cache"].double(), v_cache=d["v_cache"].double())
        table, page, at = d["table"].tolist(), case["page"], 0
        for row, n, m in zip(table, *_lens(case)):
            for t in range(n - m, n, 1):
                if t % page == 0 or t == n - m:
                    size = min(page - t % page, n - t)
                    src = slice(at + t - (n - m), at + t - (n - m) + size)
                    out["k_cache"][row[t // page], :, t % page:t % page + size] = d["k"][src].transpose(0, 1).double()
                    out["v_cache"][row[t // page], :, t % page:t % page + size] = d["v"][src].transpose(0, 1).double()
            at += m
        return out
    caches = [c.double() for c in d.get("caches", [])]
    if kind == "copy":
        for a, b in zip(d["src"].tolist(), d["dst"].tolist()):
            for c in caches:
                c[b] = c[a]
        return caches
    table, refs, page = d["table"].tolist(), d["refs"].tolist(), case["page"]
    lowest = lambda: next(i for i, r in enumerate(refs) if r == 0)  # noqa: E731
    if kind == "compact":
        live = [i for i, r in enumerate(refs) if r]
        holes = [i for i, r in enumerate(refs) if not r and i < len(live)]
        moved = dict(zip([i for i in live if i >= len(live)], holes))
        for a, b in moved.items():
            refs[a], refs[b] = 0, refs[a]
        at = torch.tensor([list(moved), list(moved.values())], device="cuda").view(2, -1)
        for c in caches:
            c[at[1]] = c[at[0]]
        return dict(caches=caches, table=_int32([[moved.get(e, e) for e in row] for row in table]), refs=_int32(refs), live=_int32([len(live)]))
    for s in (d["dst"] if kind == "fork" else d["ended"]).tolist():
        for e, x in enumerate(table[s]):
            if x >= 0:
                refs[x] -= 1
            table[s][e] = -1
    if kind == "admit":
        for row, a, b in zip(table, d["before"].tolist(), d["after"].tolist()):
            for e in range(-(-a // page), -(-b // page)):
                if row[e] < 0:
                    row[e] = lowest()
                    refs[row[e]] = 1
        return dict(table=_int32(table), refs=_int32(refs), shortfall=_int32([0]))
    lens = d["lens"].tolist()
    for s, t in zip(d["src"].tolist(), d["dst"].tolist()):
        full, part = divmod(lens[s], page)
        for e in range(full):
            table[t][e] = table[s][e]
            refs[table[s][e]] += 1
        if part:
            table[t][full] = lowest()
            refs[table[t][full]] = 1
            for c in caches:
                c[table[t][full], :, :part] = c[table[s][full], :, :part]
        lens[t] = lens[s]
    return dict(caches=caches, table=_int32(table), refs=_int32(refs), lens=_int32(lens), shortfall=_int32([0]))


def _exact_attend(case, d):
    """Sequence by sequence, the new tokens in blocks, each against the stretch of the cache that its block sees."""
    lens, new = _lens(case)
    page, hkv, dim, window, sinks = case["page"], case["kv_heads"], case["dim"], case["window"], case["sinks"]
    group = case["q_heads"] // hkv
    out = torch.empty(d["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for i, (n, m) in enumerate(zip(lens, new)):
        block = max(1, min(m, (1 << 27) // (n * group)))
        for b in range(0, m, block):
            size = min(block, m - b)
            place = torch.arange(n - m + b, n - m + b + size, device="cuda")
            low = max(0, n - m + b - window + 1)
            tokens = torch.arange(n, device="cuda")
            tokens = tokens[(tokens < sinks) | (tokens >= low)]
            tokens = tokens[tokens < n - m + b + size]
            pages = d["table"][i].long()[tokens // page]
            hidden = (tokens > place[:, None]) | ((tokens >= sinks) & (tokens <= place[:, None] - window))
            for h in range(hkv):
                q = d["q"][at + b:at + b + size, h * group:(h + 1) * group].double()
                a = torch.matmul(q.reshape(-1, dim), d["k_cache"][pages, h, tokens % page].double().t()).view(size, group, -1) / math.sqrt(dim)
                w = torch.softmax(a.masked_fill(hidden[:, None], -math.inf), -1)
                out[at + b:at + b + size, h * group:(h + 1) * group] = torch.matmul(w, d["v_cache"][pages, h, tokens % page].double())
        at += m
    return out


def _exact_logits(d):
    """Row by row, the tokens of its history counted first."""
    outs, tokens = [], []
    lens, prompts = d["history_lens"].tolist(), d["prompt_lens"].tolist()
    for i, (n, m) in enumerate(zip(lens, prompts)):
        x = d["logits"][i].double()
        words = d["history"][i, :n].long()
        count = torch.bincount(words[m:], minlength=len(x)).double()
        seen = torch.bincount(words, minlength=len(x)) > 0
        r = d["repetition"][i].double()
        x[seen] = torch.where(x[seen] > 0, x[seen] / r, x[seen] * r)
        x = x - count * d["frequency"][i].double() - (count > 0).double() * d["presence"][i].double()
        if d["bias_ids"] is not None:
            x[d["bias_ids"][i].long()] += d["bias_values"][i].double()
        bits = (d["mask"][i][:, None] >> torch.arange(32, dtype=torch.int32, device="cuda")).view(-1)[:len(x)] & 1
        x[bits == 0] = -math.inf
        best = torch.nonzero((bits == 1) & (x == x.max())).view(-1)
        outs.append(x)
        tokens.append(int(best[0]) if len(best) else -1)
    return dict(out=torch.stack(outs), token=_int32(tokens))
