"""Generation with several hypotheses a text over paged caches of bf16 / fp32 rows: one step selects, forks, appends and attends.

  attn      attention of the new rows (single tokens, a few drafted ones, pieces of prompts) over every page of their sequences, or over page lists
  fork      the sequences of the next step from those of this one: full pages shared, partly filled ones copied, room for the next
            tokens taken from the free pages, pages of sequences that end given back; then the copies themselves
  compact   the used pages moved to the front of the pools, tables renumbered
  beam      the best continuations of every group of hypotheses over beams and vocabulary

A case is a dict of op and name, and

  attn      dtype, q_heads, kv_heads, head_dim, page; seqs, rows, tokens: sequences, most rows of one, most tokens of one; ragged: the
            sequences differ in both; top_k: past pages listed per sequence and KV head, 0: every page
  fork      dtype, kv_heads, head_dim, page; seqs, tokens: sequences, most tokens of one; width: hypotheses of a text (they share their
            beginning); pools: K and V of how many layers; serve: texts end, begin and go on, else every text's hypotheses are drawn anew
  compact   dtype, kv_heads, head_dim, page, pools; seqs, tokens; idle: share of the pool's pages that is free, anywhere
  beam      dtype, groups, beams, vocab, n_out; pad: elements between the rows; start: only the first hypothesis of a group is alive
"""
import math
import random

import torch

own = False

NOTHING, BEGINS = -1, -2   # parents of a sequence that holds nothing, and of one that begins


def _attn(name, dtype, heads, head_dim, page, seqs, rows, tokens, ragged=False, top_k=0):
    return dict(name=name, op="attn", dtype=dtype, q_heads=heads[0], kv_heads=heads[1], head_dim=head_dim, page=page, seqs=seqs, rows=rows, tokens=tokens,
                ragged=ragged, top_k=top_k)


def _fork(name, dtype, kv_heads, head_dim, page, seqs, width, tokens, pools, serve=False):
    return dict(name=name, op="fork", dtype=dtype, kv_heads=kv_heads, head_dim=head_dim, page=page, seqs=seqs, width=width, tokens=tokens, pools=pools, serve=serve)


def _compact(name, dtype, kv_heads, head_dim, page, seqs, tokens, pools, idle):
    return dict(name=name, op="compact", dtype=dtype, kv_heads=kv_heads, head_dim=head_dim, page=page, seqs=seqs, tokens=tokens, pools=pools, idle=idle)


def _beam(name, dtype, groups, beams, vocab, n_out, pad=0, start=False):
    return dict(name=name, op="beam", dtype=dtype, groups=groups, beams=beams, vocab=vocab, n_out=n_out, pad=pad, start=start)


def listed():
    return [
        # one short conversation: latency
        _attn("attn_short", "bf16", (28, 4), 128, 128, 1, 1, 1000),
        # a batch in generation, lengths from one to 32K tokens
        _attn("attn_batch", "bf16", (28, 4), 128, 128, 32, 1, 32768, ragged=True),
        # one token against a million
        _attn("attn_1m", "bf16", (28, 4), 128, 128, 1, 1, 1048001),
        # single tokens over the pages that they retrieved from long texts
        _attn("attn_listed", "bf16", (28, 4), 128, 128, 16, 1, 60000, ragged=True, top_k=64),
        # a few rows each (drafted tokens, short prompts), fp32, small heads and pages
        _attn("attn_few_fp32", "f32", (14, 2), 64, 16, 6, 9, 5000, ragged=True),
        # pieces of prompts of odd lengths over what stands in front of them
        _attn("attn_prompts", "bf16", (28, 4), 128, 128, 3, 1021, 16000, ragged=True),
        # eight texts of eight hypotheses, four layers at a time
        _fork("fork_beams", "bf16", 4, 128, 128, 64, 8, 4096, 8),
        # a small model's server: texts end, begin and go on, small pages
        _fork("fork_serve", "f32", 2, 64, 16, 24, 1, 2000, 2, serve=True),
        # a cache that is to shrink: a third of the pages is free, anywhere
        _compact("compact_pools", "bf16", 4, 128, 128, 32, 20000, 4, 0.33),
        # a small model's cache after many short texts
        _compact("compact_small", "f32", 1, 64, 16, 5, 700, 2, 0.5),
        # the first step of one text: one live hypothesis, logits in fp32
        _beam("beam_start", "f32", 1, 4, 32000, 8, start=True),
        # many texts, a large vocabulary of odd size in padded rows
        _beam("beam_batch", "bf16", 32, 8, 130999, 16, pad=73),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def spread(lo, hi):   # over the logarithm, ends included
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {}
    for c in listed():
        w = work(c)
        b, f = most.get(c["op"], (0, 0))
        most[c["op"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    while True:
        op = rng.choice(["attn", "attn", "attn", "fork", "compact", "beam", "beam"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        heads, head_dim, page = rng.choice([(28, 4), (14, 2), (8, 2), (6, 2), (2, 1), (4, 4), (16, 1)]), rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128, 128])
        if op == "attn":
            kind = rng.choice(["decode", "decode", "few", "prompt"])
            seqs = {"decode": spread(1, 64), "few": spread(1, 32), "prompt": spread(1, 4)}[kind]
            rows = {"decode": 1, "few": spread(2, 16), "prompt": spread(17, 2048)}[kind]
            tokens = rows + spread(1, 1048000 if seqs == 1 and kind == "decode" else 32768)
            c = _attn("", dtype, heads, head_dim, page, seqs, rows, tokens, ragged=seqs > 1, top_k=spread(1, 64) if rng.random() < 0.3 else 0)
            pairs = c["rows"] * seqs * heads[0] * min(tokens, (c["top_k"] + 1) * page + rows if c["top_k"] else tokens)
            if seqs * (tokens + page) * heads[1] * head_dim * 4 > 3e9 or pairs > 1.6e9:
                continue
        elif op == "fork":
            width = rng.choice([1, 2, 4, 5, 8, 16])
            c = _fork("", dtype, heads[1], head_dim, page, width * spread(1, max(1, 256 // width)), width, spread(20, 32768), 2 * spread(1, 4), serve=rng.random() < 0.4)
            if c["seqs"] * (c["tokens"] + 2 * page) * heads[1] * head_dim * 4 * c["pools"] > 1.2e9:
                continue
        elif op == "compact":
            c = _compact("", dtype, heads[1], head_dim, page, spread(1, 64), spread(20, 32768), 2 * spread(1, 4), round(rng.uniform(0.0, 0.9), 2))
            if c["seqs"] * (c["tokens"] + 2 * page) * heads[1] * head_dim * 4 * c["pools"] / (1.05 - c["idle"]) > 1.2e9:
                continue
        else:
            c = _beam("", dtype, spread(1, 64), spread(1, 16), spread(50, 200000), spread(1, 32), pad=rng.choice([0, 0, 1, 8, 73]), start=rng.random() < 0.2)
        del c["name"]
        w = work(c)
        if w["bytes"] <= most[op][0] and w["flops"] <= most[op][1]:
            return c


def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _spans(case):
    """attn: (rows, tokens) of every sequence: the case's own, or drawn from its sizes: the first has the most of both, now and then
    one is idle (no rows)."""
    c = case
    if not c["ragged"]:
        return [(c["rows"], c["tokens"])] * c["seqs"]
    rng = random.Random("%(seqs)d %(rows)d %(tokens)d" % c)
    spans = [(c["rows"], c["tokens"])]
    for b in range(1, c["seqs"]):
        n = rng.randint(1, c["rows"]) if rng.random() < 0.9 else 0
        spans.append((n, max(n, int(round(math.exp(rng.uniform(0.0, math.log(c["tokens"]))))))))
    return spans


def _list_stride(case):
    """attn: row stride of the page lists: the listed past pages and the pages of the new rows."""
    return case["top_k"] + (case["rows"] + 2 * case["page"] - 2) // case["page"] if case["top_k"] else 0


def _texts(case):
    """fork: (pages of every sequence as numbers 0 .. n - 1, lengths, parents, growth, n), drawn from the case's sizes: the
    hypotheses of a text share its full pages up to where they parted."""
    c = case
    rng = random.Random("%(seqs)d %(width)d %(tokens)d %(page)d %(serve)d" % c)
    P, W = c["page"], c["width"]
    names, lens, n = [], [], 0
    for text in range(c["seqs"] // W):
        length = c["tokens"] if text == 0 else int(round(math.exp(rng.uniform(0.0, math.log(c["tokens"])))))
        full = length // P
        common = list(range(n, n + full - (rng.randint(0, min(full, 3)) if W > 1 else 0)))
        n += len(common)
        for _ in range(W):
            mine = common + list(range(n, n + -(-length // P) - len(common)))
            n += len(mine) - len(common)
            names.append(mine)
            lens.append(length)
    parents, grow = [], []
    for b in range(c["seqs"]):
        kind = rng.random()
        if c["serve"] and kind < 0.1:
            parents.append(NOTHING)
            grow.append(0)
        elif c["serve"] and kind < 0.2:
            parents.append(BEGINS)
            grow.append(int(round(math.exp(rng.uniform(0.0, math.log(max(2, c["tokens"] // 4)))))))
        else:
            parents.append(b // W * W + rng.randrange(W))
            grow.append(1)
    return names, lens, parents, grow, n


def _fork_sizes(case):
    """fork: (entries of a row of the tables, pages of the pools): room for the longest after its growth, and for every child's needs."""
    c = case
    names, lens, parents, grow, n = _texts(c)
    room = max((lens[s] if s >= 0 else 0) + g for s, g in zip(parents, grow))
    room = max([room] + lens)
    need = sum(1 + -(-g // c["page"]) for g in grow)
    return -(-room // c["page"]) + 1, n + need + 5


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    """N(0, 1) values, pages at random places of the pools.  The buffers that a loop keeps are kept here."""
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    s = dict(case=case, dev=dev, gen=gen)
    {"attn": _prepare_attn, "fork": _prepare_fork, "compact": _prepare_compact, "beam": _prepare_beam}[case["op"]](s, case)
    del s["gen"]
    return s


def _normal(s, dtype, *shape):
    out = torch.empty(shape, dtype=dtype, device=s["dev"])
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 26):
        n = min(1 << 26, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=s["gen"], device=s["dev"]).to(dtype)
    return out


def _ints(s, values):
    return torch.tensor(values, dtype=torch.int32, device=s["dev"])


def _prepare_attn(s, c):
    dt, D, P, Hq, Hkv, B, dev, gen = _dtype(c["dtype"]), c["head_dim"], c["page"], c["q_heads"], c["kv_heads"], c["seqs"], s["dev"], s["gen"]
    spans = _spans(c)
    most_pages = -(-c["tokens"] // P)
    R = sum(n for n, _ in spans) + (3 if c["ragged"] and c["rows"] > 1 else 0)   # a batch with room for a few more rows
    pages = [-(-t // P) for _, t in spans]
    n_phys = sum(pages) + 3
    order = torch.randperm(n_phys, generator=gen, device=dev).to(torch.int32)
    s["tables"] = torch.zeros((B, most_pages), dtype=torch.int32, device=dev)
    at = 0
    for b in range(B):
        s["tables"][b, :pages[b]] = order[at:at + pages[b]]
        at += pages[b]
    s["lens"] = _ints(s, [t for _, t in spans])
    starts = [0]
    for n, _ in spans:
        starts.append(starts[-1] + n)
    s["starts"] = _ints(s, starts)
    s["q"] = _normal(s, dt, R, Hq, D)
    s["k_pool"], s["v_pool"] = _normal(s, dt, n_phys, Hkv, P, D), _normal(s, dt, n_phys, Hkv, P, D)
    s["o"] = torch.zeros((R, Hq, D), dtype=dt, device=dev)
    s["lse"] = torch.zeros((Hq, R), dtype=torch.float32, device=dev)
    s["sel"] = s["cnt"] = None
    if c["top_k"]:
        width = _list_stride(c)
        s["sel"] = torch.full((B, Hkv, width), -1, dtype=torch.int32, device=dev)
        s["cnt"] = torch.zeros((B, Hkv), dtype=torch.int32, device=dev)
        for b, (n, t) in enumerate(spans):
            past = (t - n) // P   # pages before the first new row's
            for g in range(Hkv):
                k = min(c["top_k"], past)
                old = torch.randperm(max(past, 1), generator=gen, device=dev)[:k].sort().values
                ids = torch.cat([old, torch.arange(past, pages[b], device=dev)]).to(torch.int32)[:width]
                s["sel"][b, g, :len(ids)] = ids
                s["cnt"][b, g] = len(ids)
    if own:
        from paper_2602_02108_amd import api
        desc = api.make_rows_desc(s["q"], s["k_pool"], s["tables"], c["tokens"], 1.0 / math.sqrt(D), max_rows=c["rows"])
        s["ws"] = torch.empty(max(256, api.rows_workspace_bytes(desc, _list_stride(c) if c["top_k"] else -1)), dtype=torch.uint8, device=dev)


def _pools(s, c, n_phys):
    s["pools"] = [_normal(s, _dtype(c["dtype"]), n_phys, c["kv_heads"], c["page"], c["head_dim"]) for _ in range(c["pools"])]


def _prepare_fork(s, c):
    dev = s["dev"]
    names, lens, parents, grow, _ = _texts(c)
    stride, n_phys = _fork_sizes(c)
    order = torch.randperm(n_phys, generator=s["gen"], device=dev).tolist()
    s["tables"] = _ints(s, [[order[x] for x in mine] + [-1] * (stride - len(mine)) for mine in names])
    s["lens"], s["parents"], s["grow"] = _ints(s, lens), _ints(s, parents), _ints(s, grow)
    refs = [0] * n_phys
    for mine in names:
        for x in mine:
            refs[order[x]] += 1
    s["refs"] = _ints(s, refs)
    _pools(s, c, n_phys)
    s["tables_out"], s["lens_out"], s["refs_out"] = torch.zeros_like(s["tables"]), torch.zeros_like(s["lens"]), torch.zeros_like(s["refs"])
    s["copies"] = torch.zeros((c["seqs"], 3), dtype=torch.int32, device=dev)
    s["status"] = torch.zeros(2, dtype=torch.int32, device=dev)
    if own:
        from paper_2602_02108_amd import api
        s["ws"] = torch.empty(max(256, api.page_fork_workspace_bytes(c["seqs"], c["seqs"], n_phys)), dtype=torch.uint8, device=dev)


def _compact_lens(c):
    rng = random.Random("%(seqs)d %(tokens)d" % c)
    return [c["tokens"]] + [int(round(math.exp(rng.uniform(0.0, math.log(c["tokens"]))))) for _ in range(c["seqs"] - 1)]


def _compact_pages(c):
    used = sum(-(-t // c["page"]) for t in _compact_lens(c))
    return used, int(math.ceil(used / (1.0 - c["idle"])))


def _prepare_compact(s, c):
    dev, lens = s["dev"], _compact_lens(c)
    used, n_phys = _compact_pages(c)
    stride = -(-c["tokens"] // c["page"])
    order = torch.randperm(n_phys, generator=s["gen"], device=dev).to(torch.int32)
    s["tables"] = torch.full((c["seqs"], stride), -1, dtype=torch.int32, device=dev)
    at = 0
    for b, t in enumerate(lens):
        n = -(-t // c["page"])
        s["tables"][b, :n] = order[at:at + n]
        at += n
    s["lens"] = _ints(s, lens)
    s["refs"] = torch.zeros(n_phys, dtype=torch.int32, device=dev)
    s["refs"][order[:used].long()] = 1
    _pools(s, c, n_phys)
    s["tables_out"], s["refs_out"] = torch.zeros_like(s["tables"]), torch.zeros_like(s["refs"])
    s["moves"] = torch.zeros((n_phys // 2 + 1, 3), dtype=torch.int32, device=dev)
    s["map"] = torch.zeros(n_phys, dtype=torch.int32, device=dev)
    s["status"] = torch.zeros(2, dtype=torch.int32, device=dev)
    if own:
        from paper_2602_02108_amd import api
        s["ws"] = torch.empty(max(256, api.page_compact_workspace_bytes(n_phys)), dtype=torch.uint8, device=dev)


def _prepare_beam(s, c):
    dev, gen, R = s["dev"], s["gen"], c["groups"] * c["beams"]
    rows = _normal(s, _dtype(c["dtype"]), R, c["vocab"] + c["pad"])
    rows *= 4.0   # logits are wider than N(0, 1)
    s["logits"] = rows[:, :c["vocab"]]
    score = -20.0 * torch.rand((c["groups"], c["beams"]), generator=gen, device=dev)
    ended = torch.rand((c["groups"], c["beams"]), generator=gen, device=dev) < 0.1
    if c["start"]:
        score[:, 0], score[:, 1:], ended[:] = 0.0, -math.inf, False
    s["scores"], s["done"] = score, ended.to(torch.int32)
    s["parents"], s["tokens"] = (torch.zeros((c["groups"], c["n_out"]), dtype=torch.int32, device=dev) for _ in range(2))
    s["best"] = torch.zeros((c["groups"], c["n_out"]), dtype=torch.float32, device=dev)
    if own:
        from paper_2602_02108_amd import api
        s["ws"] = torch.empty(max(256, api.beam_workspace_bytes(s["logits"], c["groups"], c["n_out"])), dtype=torch.uint8, device=dev)


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"attn": _attn_own, "fork": _fork_own, "compact": _compact_own, "beam": _beam_own}[op](state)
    return {"attn": _attn_plain, "fork": _fork_plain, "compact": _compact_plain, "beam": _beam_plain}[op](state)


def _attn_own(s):
    from paper_2602_02108_amd import api
    c = s["case"]
    desc = api.make_rows_desc(s["q"], s["k_pool"], s["tables"], c["tokens"], 1.0 / math.sqrt(c["head_dim"]), max_rows=c["rows"])
    api.paged_attn_fwd_rows(desc, s["q"], s["k_pool"], s["v_pool"], s["tables"], sel_pages=s["sel"], sel_count=s["cnt"], o=s["o"], lse=s["lse"],
                            workspace=s["ws"], seq_lens=s["lens"], row_starts=s["starts"])
    return dict(o=s["o"], lse=s["lse"])


def _fork_own(s):
    from paper_2602_02108_amd import api
    api.page_fork(s["tables"], s["lens"], s["parents"], s["refs"], s["case"]["page"], grow=s["grow"], tables_out=s["tables_out"], lens_out=s["lens_out"],
                  refs_out=s["refs_out"], copies=s["copies"], status=s["status"], workspace=s["ws"])
    api.page_copy(s["pools"], s["copies"])
    return dict(tables=s["tables_out"], lens=s["lens_out"], refs=s["refs_out"], copies=s["copies"], status=s["status"], pools=s["pools"])


def _compact_own(s):
    from paper_2602_02108_amd import api
    api.page_compact(s["tables"], s["lens"], s["refs"], s["case"]["page"], tables_out=s["tables_out"], refs_out=s["refs_out"], moves=s["moves"],
                     page_map=s["map"], status=s["status"], workspace=s["ws"])
    api.page_copy(s["pools"], s["moves"], count=s["status"][1:])
    return dict(tables=s["tables_out"], refs=s["refs_out"], map=s["map"], status=s["status"], pools=s["pools"])


def _beam_own(s):
    from paper_2602_02108_amd import api
    c = s["case"]
    api.beam_topk(s["logits"], s["scores"], c["n_out"], done=s["done"], pad_token=1, parents=s["parents"], tokens=s["tokens"], scores_out=s["best"],
                  workspace=s["ws"])
    return dict(parents=s["parents"], tokens=s["tokens"], scores=s["best"])


def _attn_plain(s):
    c = s["case"]
    P, D, Hq, Hkv, B, n = c["page"], c["head_dim"], c["q_heads"], c["kv_heads"], c["seqs"], c["rows"]
    G, dev = Hq // Hkv, s["dev"]
    starts, lens = s["starts"].long(), s["lens"].long()
    r = torch.arange(s["q"].shape[0], device=dev)
    seq = (r[:, None] >= starts[None, 1:]).sum(1)
    live = torch.nonzero(seq < B)[:, 0]   # the rows that belong to a sequence
    seq = seq[live]
    row, pos = live - starts[seq], lens[seq] - starts[seq + 1] + live
    q = torch.zeros((B, n, Hq, D), dtype=torch.float32, device=dev)
    q[seq, row] = s["q"][live].float()
    at = torch.full((B, n), -1, dtype=torch.int64, device=dev)   # positions, -1 where there is no row
    at[seq, row] = pos
    o = torch.empty((B, n, Hq, D), dtype=torch.float32, device=dev)
    lse = torch.empty((B, n, Hq), dtype=torch.float32, device=dev)
    every = torch.arange(s["tables"].shape[1], device=dev).expand(B, -1)
    for g in range(Hkv):
        ids = every if s["sel"] is None else s["sel"][:, g].long()
        held = torch.ones_like(ids, dtype=torch.bool) if s["sel"] is None else torch.arange(ids.shape[1], device=dev) < s["cnt"][:, g, None]
        tiles = s["tables"].gather(1, ids.clamp(min=0)).long()
        k, v = (pool[tiles, g].flatten(1, 2).float() for pool in (s["k_pool"], s["v_pool"]))   # [B][tokens][D]
        token = torch.where(held, ids * P, 1 << 40)[..., None] + torch.arange(P, device=dev)
        hidden = token.flatten(1)[:, None] > at[..., None]   # [B][n][tokens]
        x = q[:, :, g * G:(g + 1) * G].flatten(1, 2) @ k.transpose(1, 2).contiguous() * (1.0 / math.sqrt(D))
        x = x.unflatten(1, (n, G)).masked_fill_(hidden[:, :, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        p = x.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        y = p.flatten(1, 2) @ v
        o[:, :, g * G:(g + 1) * G] = y.unflatten(1, (n, G)) / torch.where(total == 0, 1.0, total)
        lse[:, :, g * G:(g + 1) * G] = (top + total.log())[..., 0]
    s["o"][live] = o[seq, row].to(s["o"].dtype)
    s["lse"][:, live] = lse[seq, row].t()
    return dict(o=s["o"], lse=s["lse"])


def _copy_plain(pools, src, dst, tokens):
    """The first tokens of pages, from src to dst."""
    page = pools[0].shape[2]
    new = (torch.arange(page, device=src.device) < tokens[:, None])[:, None, :, None]
    for pool in pools:
        pool[dst] = torch.where(new, pool[src], pool[dst])


def _fork_plain(s):
    P, dev = s["case"]["page"], s["dev"]
    tables, lens, parents, grow, refs = (s[k].long() for k in ("tables", "lens", "parents", "grow", "refs"))
    S, stride = tables.shape
    n_phys = refs.numel()
    of = parents >= 0
    src = parents.clamp(min=0)
    was = torch.where(of, lens[src], 0)
    now = torch.where(parents == NOTHING, 0, (was + grow).clamp(max=stride * P))
    held, part = was // P, was % P
    child = torch.arange(S, device=dev)
    earlier = ((parents[:, None] == parents[None]) & (child[None] < child[:, None])).any(1)
    last = tables[src, held.clamp(max=stride - 1)].clamp(min=0)   # the partly filled page
    copied = of & (part > 0) & (earlier | (refs[last] > 1))
    need = copied.long() + ((now + P - 1) // P - (was + P - 1) // P)
    first = need.cumsum(0) - need
    free = torch.nonzero(refs == 0)[:, 0]
    l = torch.arange(stride, device=dev)[None]
    kept = held[:, None] + ((part > 0) & ~copied)[:, None]
    new = free[(first[:, None] + l - kept).clamp(0, free.numel() - 1)]
    out = torch.where(l < kept, tables[src], torch.where(l < ((now + P - 1) // P)[:, None], new, -1))
    count = refs.clone()
    old = tables[torch.arange(stride, device=dev)[None] < ((lens + P - 1) // P)[:, None]]
    count.index_add_(0, old, torch.full_like(old, -1))
    named = out[out >= 0]
    count.index_add_(0, named, torch.ones_like(named))
    to = free[first.clamp(max=free.numel() - 1)]
    copies = torch.where(copied[:, None], torch.stack([last, to, part], 1), torch.tensor([-1, -1, 0], device=dev))
    _copy_plain(s["pools"], last[copied], to[copied], part[copied])
    s["tables_out"].copy_(out)
    s["lens_out"].copy_(now)
    s["refs_out"].copy_(count)
    s["copies"].copy_(copies)
    s["status"].copy_(torch.stack([need.sum(), torch.zeros_like(need[0])]))
    return dict(tables=s["tables_out"], lens=s["lens_out"], refs=s["refs_out"], copies=s["copies"], status=s["status"], pools=s["pools"])


def _compact_plain(s):
    P, dev = s["case"]["page"], s["dev"]
    refs, tables = s["refs"], s["tables"].long()
    n_phys = refs.numel()
    used = refs > 0
    n = used.sum()
    at = torch.arange(n_phys, device=dev)
    src, dst = torch.nonzero(used & (at >= n))[:, 0], torch.nonzero(~used & (at < n))[:, 0]
    new = torch.where(used, at, -1)
    new[src] = dst
    mine = torch.arange(tables.shape[1], device=dev)[None] < ((s["lens"] + P - 1) // P)[:, None]
    s["tables_out"].copy_(torch.where(mine, new[tables.clamp(min=0)], -1))
    s["refs_out"].zero_()
    s["refs_out"][new[used]] = refs[used]
    s["map"].copy_(new)
    s["status"].copy_(torch.stack([n, torch.full_like(n, src.numel())]))
    _copy_plain(s["pools"], src, dst, torch.full_like(src, P))
    return dict(tables=s["tables_out"], refs=s["refs_out"], map=s["map"], status=s["status"], pools=s["pools"])


def _beam_plain(s):
    c = s["case"]
    V, W = c["vocab"], c["beams"]
    # 64 bits: which of two candidates is the better one is decided by what 32 bits round away
    x = s["logits"].double().unflatten(0, (c["groups"], W))
    top = x.amax(-1, keepdim=True)
    cand = s["scores"].double()[..., None] + (x - (top + (x - top).exp().sum(-1, keepdim=True).log()))
    only = torch.where(torch.arange(V, device=s["dev"]) == 1, s["scores"].double()[..., None], -math.inf)
    cand = torch.where(s["done"][..., None] != 0, only, cand).flatten(1)
    best, at = cand.sort(dim=-1, descending=True, stable=True)   # (ties go to the lowest index)
    k = min(c["n_out"], best.shape[1])
    best, at = best[:, :k], at[:, :k]
    alive = best > -math.inf
    row = torch.arange(c["groups"], device=s["dev"])[:, None] * W + at // V
    s["parents"].fill_(-1)
    s["tokens"].fill_(-1)
    s["best"].fill_(-math.inf)
    s["parents"][:, :k] = torch.where(alive, row, -1)
    s["tokens"][:, :k] = torch.where(alive, at % V, -1)
    s["best"][:, :k] = best
    return dict(parents=s["parents"], tokens=s["tokens"], scores=s["best"])


# ------------------------------------------------------------------------------------------------ from the definitions, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _attn_exact, "fork": _fork_exact, "compact": _compact_exact, "beam": _beam_exact}[case["op"]](s, case)


def _attn_exact(s, c):
    P, D, Hkv, G = c["page"], c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    starts = s["starts"].tolist()
    o, lse = s["o"].double(), s["lse"].double()
    for b, (n, t) in enumerate(_spans(c)):
        for g in range(Hkv) if n else ():
            ids = torch.arange(-(-t // P), device=s["dev"]) if s["sel"] is None else s["sel"][b, g, :int(s["cnt"][b, g])].long()
            tiles = s["tables"][b, ids].long()
            token = (ids[:, None] * P + torch.arange(P, device=ids.device)).flatten()
            k, v = (pool[tiles, g].double().flatten(0, 1) for pool in (s["k_pool"], s["v_pool"]))
            for i in range(0, n, 256):
                m = min(256, n - i)
                q = s["q"][starts[b] + i:starts[b] + i + m, g * G:(g + 1) * G].double()
                x = torch.tensordot(q, k, dims=([2], [1])) / math.sqrt(D)
                hidden = token[None] > (t - n + i + torch.arange(m, device=ids.device))[:, None]
                x = x.masked_fill(hidden[:, None], -math.inf)
                z = torch.logsumexp(x, -1)
                p = torch.where(torch.isinf(z)[..., None], 0.0, (x - z[..., None]).exp())
                o[starts[b] + i:starts[b] + i + m, g * G:(g + 1) * G] = torch.tensordot(p, v, dims=([2], [0]))
                lse[g * G:(g + 1) * G, starts[b] + i:starts[b] + i + m] = z.t()
    return dict(o=o, lse=lse)


def _fork_exact(s, c):
    """Child by child."""
    P = c["page"]
    tables, lens, parents, grow, refs = (s[k].tolist() for k in ("tables", "lens", "parents", "grow", "refs"))
    stride = len(tables[0])
    free = [i for i, r in enumerate(refs) if r == 0]
    count, taken, seen, out, lens_out, copies = list(refs), 0, set(), [], [], []
    for row, t in zip(tables, lens):
        for x in row[:-(-t // P)]:
            count[x] -= 1
    for s_, more in zip(parents, grow):
        mine, t, copy = [], 0, [-1, -1, 0]
        if s_ >= 0:
            t = lens[s_]
            mine = tables[s_][:-(-t // P)]
            if t % P and (s_ in seen or refs[mine[-1]] > 1):
                copy = [mine[-1], free[taken], t % P]
                mine[-1] = free[taken]
                taken += 1
            seen.add(s_)
        if s_ != NOTHING:
            t = min(t + more, stride * P)
        while len(mine) < -(-t // P):
            mine.append(free[taken])
            taken += 1
        for x in mine:
            count[x] += 1
        out.append(mine + [-1] * (stride - len(mine)))
        lens_out.append(t)
        copies.append(copy)
    pools = [pool.double() for pool in s["pools"]]
    for a, b, t in copies:
        for pool in pools if t else ():
            pool[b, :, :t] = pool[a, :, :t]
    return dict(tables=_ints(s, out), lens=_ints(s, lens_out), refs=_ints(s, count), copies=_ints(s, copies), status=_ints(s, [taken, 0]), pools=pools)


def _compact_exact(s, c):
    P = c["page"]
    tables, lens, refs = (s[k].tolist() for k in ("tables", "lens", "refs"))
    n = sum(1 for r in refs if r > 0)
    holes = [i for i in range(n) if refs[i] == 0]
    movers = [i for i in range(n, len(refs)) if refs[i] > 0]
    new = [i if r > 0 else -1 for i, r in enumerate(refs)]
    count = [r if i < n else 0 for i, r in enumerate(refs)]
    pools = [pool.double() for pool in s["pools"]]
    for a, b in zip(movers, holes):
        new[a], count[b] = b, refs[a]
    if movers:
        a, b = torch.tensor(movers, device=s["dev"]), torch.tensor(holes, device=s["dev"])
        for pool in pools:
            pool[b] = pool[a]
    out = [[new[x] if l < -(-t // P) else -1 for l, x in enumerate(row)] for row, t in zip(tables, lens)]
    return dict(tables=_ints(s, out), refs=_ints(s, count), map=_ints(s, new), status=_ints(s, [n, len(movers)]), pools=pools)


def _beam_exact(s, c):
    """Row by row the best tokens, then the best of a group's rows."""
    parents, tokens, best = [], [], []
    x = s["logits"].double()
    z = torch.logsumexp(x, 1).tolist()
    scores, done = s["scores"].flatten().tolist(), s["done"].flatten().tolist()
    V, W, k = c["vocab"], c["beams"], min(c["n_out"], c["vocab"])
    edge = x.topk(k, 1).values[:, -1:]
    for g in range(c["groups"]):
        offers = []
        for r in range(g * W, (g + 1) * W):
            if scores[r] == -math.inf:
                continue
            if done[r]:
                offers.append((-scores[r], r, 1))
                continue
            for v in torch.nonzero(x[r] >= edge[r])[:, 0].tolist():
                offers.append((-(scores[r] + (float(x[r, v]) - z[r])), r, v))
        offers = sorted(offers)[:c["n_out"]]
        offers += [(math.inf, -1, -1)] * (c["n_out"] - len(offers))
        best.append([-y for y, _, _ in offers])
        parents.append([r for _, r, _ in offers])
        tokens.append([v for _, _, v in offers])
    return dict(parents=_ints(s, parents), tokens=_ints(s, tokens), scores=torch.tensor(best, dtype=torch.float64, device=s["dev"]))


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """Bytes: every input read once, every output written once (of the pools: what is copied, read and written).  Operations: attention 4 D for
    each pair of a query and a token that it sees; fork and compact one per table entry; beam four per logit."""
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "attn":
        D, P, Hq, Hkv = c["head_dim"], c["page"], c["q_heads"], c["kv_heads"]
        spans = _spans(c)
        R = sum(n for n, _ in spans)
        pairs = held = 0
        for n, t in spans:
            if n == 0:
                continue
            past = (t - n) // P
            hidden = 0 if not c["top_k"] else (past - min(c["top_k"], past)) * P   # past tokens in no list
            held += t - hidden
            pairs += n * (t - n - hidden) + n * (n + 1) // 2
        return {"bytes": held * Hkv * 2 * D * es + 2 * R * Hq * D * es + 4 * R * Hq, "flops": 4.0 * D * pairs * Hq}
    if c["op"] == "beam":
        R = c["groups"] * c["beams"]
        alive = c["groups"] if c["start"] else R
        return {"bytes": alive * c["vocab"] * es + 8 * R + 12 * c["groups"] * c["n_out"], "flops": 4.0 * alive * c["vocab"]}
    P, token = c["page"], c["kv_heads"] * c["head_dim"] * es * c["pools"]
    if c["op"] == "compact":
        used, n_phys = _compact_pages(c)
        entries = sum(-(-t // P) for t in _compact_lens(c))
        table = c["seqs"] * -(-c["tokens"] // P)
        moved = used * (n_phys - used) // n_phys   # (on average over random places)
        return {"bytes": 4 * (entries + table + 3 * n_phys) + 2 * moved * P * token, "flops": float(entries + n_phys)}
    names, lens, parents, grow, _ = _texts(c)
    stride, n_phys = _fork_sizes(c)
    copied, seen = 0, set()
    for s in parents:
        if s >= 0:
            copied += lens[s] % P if s in seen else 0
            seen.add(s)
    entries = sum(len(mine) for mine in names)
    return {"bytes": 4 * (entries + c["seqs"] * (stride + 8) + 2 * n_phys) + 2 * copied * token, "flops": float(entries + c["seqs"] * stride)}
