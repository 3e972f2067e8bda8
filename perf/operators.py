"""Rows of keys and values on their way into the paged cache, and attention over a cache held in 4 bits.

  append        Q and K of the new rows rotated by their positions, K / V written to their pages, the means of the pages they fill
  append_grad   its backward: dQ rotated back, dK / dV of the rows taken from the paged gradient pools, dK rotated back
  kv4_append    the same append into a cache of 4-bit codes with a power-of-two scale per 32 dims, and what the cache then holds
  kv4_attn      attention of the new rows over such a cache, over every page or over page lists

Rows are packed: [rows of all sequences][heads][head_dim].  Sequence b has the rows starts[b] .. starts[b + 1] - 1, which are the
last of its lens[b] tokens.  A case is a dict of

  op, dtype, q_heads, kv_heads, head_dim, page
  seqs, rows, tokens  sequences, most rows of one, most tokens of one; ragged: the sequences differ in both
  rot, interleaved    rotated dims, and whether the pairs are neighbours or halves (append*, kv4_append)
  grad_dtype          of the gradient pools (append_grad)
  top_k               past pages listed per sequence and KV head, 0: every page (kv4_attn)
"""
import math
import random

import torch

own = False

_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # of a 4-bit code, sign apart


def _case(name, op, dtype, heads, head_dim, page, seqs, rows, tokens, ragged=False, rot=0, interleaved=False, grad_dtype="f32", top_k=0):
    return dict(name=name, op=op, dtype=dtype, q_heads=heads[0], kv_heads=heads[1], head_dim=head_dim, page=page, seqs=seqs, rows=rows,
                tokens=tokens, ragged=ragged, rot=rot, interleaved=interleaved, grad_dtype=grad_dtype, top_k=top_k)


def listed():
    return [
        # one new token for each of a few sequences in generation: launches and latency
        _case("append_decode", "append", "bf16", (28, 4), 128, 128, 8, 1, 4096, ragged=True, rot=128),
        # a training chunk of a full-width layer, its projections packed in one tensor
        _case("append_chunk", "append", "bf16", (28, 4), 128, 128, 1, 4096, 65536, rot=128),
        # fp32 prompts of odd lengths, small pages, half of the dims rotated in neighbouring pairs (toy models, reference runs)
        _case("append_ragged_fp32", "append", "f32", (2, 1), 64, 16, 5, 333, 2100, ragged=True, rot=32, interleaved=True),
        # the backward of the training chunk, fp32 gradient pools
        _case("append_grad_chunk", "append_grad", "bf16", (28, 4), 128, 128, 1, 4096, 65536, rot=128),
        # small heads and pages, bf16 gradients, several texts of odd lengths
        _case("append_grad_ragged", "append_grad", "bf16", (14, 2), 64, 16, 3, 1088, 4000, ragged=True, rot=64, grad_dtype="bf16"),
        # generation over many sequences: one token each
        _case("kv4_append_decode", "kv4_append", "bf16", (28, 4), 128, 128, 64, 1, 8192, ragged=True, rot=128),
        # a long prompt's chunk
        _case("kv4_append_chunk", "kv4_append", "bf16", (28, 4), 128, 128, 1, 8192, 16384, rot=128),
        # one short conversation: latency
        _case("kv4_decode_short", "kv4_attn", "bf16", (28, 4), 128, 128, 1, 1, 1000),
        # a batch in generation, lengths from one to 32K tokens
        _case("kv4_decode_batch", "kv4_attn", "bf16", (28, 4), 128, 128, 32, 1, 32768, ragged=True),
        # one token against a million
        _case("kv4_decode_1m", "kv4_attn", "bf16", (28, 4), 128, 128, 1, 1, 1048001),
        # a few rows each (drafted tokens, short prompts), fp32, small heads and pages
        _case("kv4_few_rows_fp32", "kv4_attn", "f32", (14, 2), 64, 16, 6, 9, 5000, ragged=True),
        # a prompt's chunk over the pages that it retrieved
        _case("kv4_chunk_sparse", "kv4_attn", "bf16", (28, 4), 128, 128, 1, 2048, 131072, top_k=64),
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
        op = rng.choice(["append", "append_grad", "kv4_append", "kv4_attn", "kv4_attn", "kv4_attn"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        heads, head_dim, page = rng.choice([(28, 4), (14, 2), (8, 2), (6, 2), (2, 1), (4, 4)]), rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128, 128])
        kind = rng.choice(["decode", "few", "chunk"])
        seqs = {"decode": spread(1, 64), "few": spread(1, 32), "chunk": spread(1, 4)}[kind]
        rows = {"decode": 1, "few": spread(2, 64), "chunk": spread(64, 8192)}[kind]
        tokens = rows + spread(1, 1048000 if seqs == 1 and kind == "decode" else 32768)
        rot = rng.choice([head_dim, head_dim, head_dim // 2, 16])
        top_k = spread(1, 64) if op == "kv4_attn" and rng.random() < 0.4 else 0
        c = _case("", op, dtype, heads, head_dim, page, seqs, rows, tokens, ragged=seqs > 1, rot=0 if op == "kv4_attn" else rot,
                  interleaved=op != "kv4_attn" and rng.random() < 0.3, grad_dtype=rng.choice(["f32", "bf16"]) if op == "append_grad" else "f32", top_k=top_k)
        del c["name"]
        w = work(c)
        held = seqs * (tokens + page) * heads[1] * head_dim * 2 * (4 if op.startswith("append") else 1)
        if w["bytes"] <= most[op][0] and w["flops"] <= most[op][1] and held <= 3e9 and c["rows"] * seqs * heads[0] * min(tokens, (top_k + 1) * page + rows if top_k else tokens) <= 8e8:
            return c


def _spans(case):
    """(rows, tokens) of every sequence: the case's own, or drawn from its sizes: the first has the most of both, now and then
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


def _lists(case):
    """Row stride of the page lists: the listed past pages and the pages of the new rows."""
    return case["top_k"] + (case["rows"] + 2 * case["page"] - 2) // case["page"] if case["top_k"] else 0


def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


# ------------------------------------------------------------------------------------------------ the 4-bit cache
# A pool is uint8 [pages][kv_heads][page * (head_dim / 2 + head_dim / 32)]: the codes [page][head_dim / 2] of a page's tokens (dim 2 i
# in the low half of byte i), then the scale bytes [head_dim / 32][page].  A byte s stands for 2^(s - 127), 255 for NaN.

def _quantise(x):
    """x [..., D] float32 or float64 -> (codes [..., D] uint8, scale bytes [..., D / 32] uint8)."""
    blocks = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    top = blocks.abs().amax(-1)
    if x.dtype == torch.float32:   # the smallest power of two with top <= 7 of it
        byte = ((top.view(torch.int32).long() + 0x1FFFFF) >> 23) - 2
    else:
        byte = ((top.view(torch.int64) + 0x3FFFFFFFFFFFF) >> 52) - (1023 - 127) - 2
    byte = byte.clamp(2, 252)
    a = (blocks.abs() * torch.ldexp(torch.ones_like(top), (127 - byte).int()).unsqueeze(-1))
    code = (a > 0.25).to(torch.uint8)
    for k, edge in enumerate((0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):   # halves go to the even code
        code += (a >= edge) if k % 2 == 0 else (a > edge)
    code += 8 * torch.signbit(blocks).to(torch.uint8)
    byte = torch.where(torch.isfinite(top), byte, 255)
    return code.reshape(x.shape), byte.to(torch.uint8)


def _values(code, byte):
    """The float32 values of codes [..., D] and scale bytes [..., D / 32]."""
    level = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), dtype=torch.float32, device=code.device)
    scale = torch.ldexp(torch.ones(byte.shape, dtype=torch.float32, device=code.device), byte.int() - 127)
    scale = torch.where(byte == 255, math.nan, scale)
    return level[code.int()] * scale.repeat_interleave(32, -1)


def _pack(code, byte, page, head_dim):
    """Tiles of a pool from codes [..., page, D] and scale bytes [..., page, D / 32]."""
    pairs = code[..., 0::2] | (code[..., 1::2] << 4)
    return torch.cat([pairs.flatten(-2), byte.transpose(-1, -2).flatten(-2)], -1)


def _unpack(tiles, page, head_dim):
    """(codes [..., page, D], scale bytes [..., page, D / 32]) of tiles."""
    cut = page * head_dim // 2
    pairs = tiles[..., :cut].unflatten(-1, (page, head_dim // 2))
    code = torch.stack([pairs & 15, pairs >> 4], -1).flatten(-2)
    return code, tiles[..., cut:].unflatten(-1, (head_dim // 32, page)).transpose(-1, -2)


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    """Rows, pools with a shuffled page table and the tables of angles, N(0, 1) values.  The buffers that a loop keeps are kept here."""
    c = case
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt, D, P, Hq, Hkv, B = _dtype(c["dtype"]), c["head_dim"], c["page"], c["q_heads"], c["kv_heads"], c["seqs"]
    spans = _spans(c)
    most_pages = -(-c["tokens"] // P)
    total = sum(n for n, _ in spans)
    R = total + (3 if c["ragged"] and c["rows"] > 1 else 0)   # a batch with room for a few more rows
    s = dict(case=c, max_len=c["tokens"])
    pages = [-(-t // P) for _, t in spans]
    n_phys = sum(pages) + 3
    order = torch.randperm(n_phys, generator=gen, device=dev).to(torch.int32)
    table = torch.zeros((B, most_pages), dtype=torch.int32, device=dev)
    at = 0
    for b in range(B):
        table[b, :pages[b]] = order[at:at + pages[b]]
        at += pages[b]
    s["tables"] = table
    s["lens"] = torch.tensor([t for _, t in spans], dtype=torch.int32, device=dev)
    starts = [0]
    for n, _ in spans:
        starts.append(starts[-1] + n)
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device=dev)

    def normal(*shape, dtype=dt):
        out = torch.empty(shape, dtype=dtype, device=dev)
        flat = out.view(-1)
        for i in range(0, flat.numel(), 1 << 26):
            n = min(1 << 26, flat.numel() - i)
            flat[i:i + n] = torch.randn(n, generator=gen, device=dev).to(dtype)
        return out

    def pool4():
        tile = P * (D // 2 + D // 32)
        out = torch.empty((n_phys, Hkv, tile), dtype=torch.uint8, device=dev)
        step = max(1, (1 << 25) // (Hkv * P * D))
        for i in range(0, n_phys, step):
            n = min(step, n_phys - i)
            out[i:i + n] = _pack(*_quantise(torch.randn((n, Hkv, P, D), generator=gen, device=dev)), P, D)
        return out

    if c["op"] == "kv4_attn":
        s["q"] = normal(R, Hq, D)
        s["k_pool"], s["v_pool"] = pool4(), pool4()
        s["o"] = torch.zeros((R, Hq, D), dtype=dt, device=dev)
        s["lse"] = torch.zeros((Hq, R), dtype=torch.float32, device=dev)
        s["sel"] = s["cnt"] = None
        if c["top_k"]:
            width = _lists(c)
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
    else:
        if c["op"] == "append_grad":
            gdt = _dtype(c["grad_dtype"])
            s["dq"] = normal(R, Hq, D)
            s["dk_pool"], s["dv_pool"] = normal(n_phys, Hkv, P, D, dtype=gdt), normal(n_phys, Hkv, P, D, dtype=gdt)
            grads = torch.zeros((R, (Hq + 2 * Hkv) * D), dtype=dt, device=dev)   # of the packed projections
            s["dq_out"], s["dk"], s["dv"] = _split(grads, Hq, Hkv, D)
        else:
            s["q"], s["k"], s["v"] = _split(normal(R, (Hq + 2 * Hkv) * D), Hq, Hkv, D)
            s["q_out"] = torch.zeros((R, Hq, D), dtype=dt, device=dev)
            s["kbar"] = torch.zeros((B, most_pages, Hkv, D), dtype=torch.float32, device=dev)
            if c["op"] == "append":
                s["k_pool"], s["v_pool"] = normal(n_phys, Hkv, P, D), normal(n_phys, Hkv, P, D)
            else:
                s["k_pool"], s["v_pool"] = pool4(), pool4()
                s["k_held"], s["v_held"] = (torch.zeros((R, Hkv, D), dtype=dt, device=dev) for _ in range(2))
        half = c["rot"] // 2
        angle = torch.arange(c["tokens"], dtype=torch.float64, device=dev)[:, None] * \
            10000.0 ** (-torch.arange(half, dtype=torch.float64, device=dev) / half)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    if own:
        from paper_2602_02108_amd import api
        if c["op"] == "kv4_attn":
            desc = api.make_rows_desc(s["q"], s["k_pool"], table, s["max_len"], 1.0 / math.sqrt(D), max_rows=c["rows"])
            s["ws"] = torch.empty(max(256, api.kvq_workspace_bytes(desc, _lists(c) if c["top_k"] else -1)), dtype=torch.uint8, device=dev)
        else:
            s["rope"] = api.Rope(s["cos"], s["sin"], interleaved=c["interleaved"])
    return s


def _split(packed, Hq, Hkv, D):
    """The views of Q, K and V in packed rows."""
    q, k, v = packed.split([Hq * D, Hkv * D, Hkv * D], 1)
    return q.unflatten(1, (Hq, D)), k.unflatten(1, (Hkv, D)), v.unflatten(1, (Hkv, D))


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2602_02108_amd import api
    c = s["case"]
    op, where = c["op"], dict(seq_lens=s["lens"], row_starts=s["starts"])
    if op == "append_grad":
        desc = api.make_rows_desc(s["dq"], s["dk_pool"], s["tables"], s["max_len"], max_rows=c["rows"])
        api.kv_append_rope_bwd(desc, s["dk_pool"], s["dv_pool"], s["tables"], d_q=s["dq"], rope=s["rope"], d_q_out=s["dq_out"], d_k=s["dk"],
                               d_v=s["dv"], **where)
        return dict(dq=s["dq_out"], dk=s["dk"], dv=s["dv"])
    if op == "kv4_attn":
        desc = api.make_rows_desc(s["q"], s["k_pool"], s["tables"], s["max_len"], 1.0 / math.sqrt(c["head_dim"]), max_rows=c["rows"])
        api.paged_attn_fwd_kvq(desc, s["q"], s["k_pool"], s["v_pool"], s["tables"], sel_pages=s["sel"], sel_count=s["cnt"], o=s["o"], lse=s["lse"],
                               workspace=s["ws"], **where)
        return dict(o=s["o"], lse=s["lse"])
    desc = api.make_rows_desc(s["q"], s["k_pool"], s["tables"], s["max_len"], max_rows=c["rows"])
    append = api.kv_append_rope if op == "append" else api.kvq_append_rope
    append(desc, s["k"], s["v"], s["tables"], s["k_pool"], s["v_pool"], q=s["q"], q_out=s["q_out"], rope=s["rope"], kbar_cache=s["kbar"], **where)
    out = dict(q=s["q_out"], kbar=s["kbar"])
    if op == "append":
        return dict(out, k_pool=s["k_pool"], v_pool=s["v_pool"])
    api.kvq_read(desc, s["k_pool"], s["v_pool"], s["tables"], k_out=s["k_held"], v_out=s["v_held"], **where)
    return dict(out, k=s["k_held"], v=s["v_held"])


def _rows(s, n):
    """Of the n packed rows: which belong to a sequence, their sequence and their position (of those)."""
    starts, lens = s["starts"].long(), s["lens"].long()
    r = torch.arange(n, device=starts.device)
    seq = (r[:, None] >= starts[None, 1:]).sum(1)
    live = torch.nonzero(seq < lens.numel())[:, 0]
    seq = seq[live]
    return live, seq, lens[seq] - starts[seq + 1] + live


def _rotate(x, cos, sin, interleaved, back=False):
    """x [rows][heads][D], cos / sin [rows][half]: the first 2 half dims rotated."""
    half = cos.shape[-1]
    cos, sin = cos[:, None], (-sin if back else sin)[:, None]
    part = x[..., :2 * half]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :half], part[..., half:])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, x[..., 2 * half:]], -1)


def _run_plain(s):
    c = s["case"]
    if c["op"] == "kv4_attn":
        return _attend_plain(s)
    dt, P, D, inter = _dtype(c["dtype"]), c["page"], c["head_dim"], c["interleaved"]
    if c["op"] == "append_grad":
        live, seq, pos = _rows(s, s["dq"].shape[0])
        cos, sin = s["cos"][pos], s["sin"][pos]
        page, slot = s["tables"][seq, pos // P].long(), pos % P
        s["dq_out"][live] = _rotate(s["dq"][live].float(), cos, sin, inter, back=True).to(dt)
        s["dk"][live] = _rotate(s["dk_pool"][page, :, slot].float(), cos, sin, inter, back=True).to(dt)
        s["dv"][live] = s["dv_pool"][page, :, slot].to(dt)
        return dict(dq=s["dq_out"], dk=s["dk"], dv=s["dv"])

    live, seq, pos = _rows(s, s["q"].shape[0])
    cos, sin = s["cos"][pos], s["sin"][pos]
    page, slot = s["tables"][seq, pos // P].long(), pos % P
    s["q_out"][live] = _rotate(s["q"][live].float(), cos, sin, inter).to(dt)
    full = slot == P - 1   # the rows that fill a page
    filled = page[full]
    # 64 bits: codes change where a value crosses an edge, and what the means sum are keys rounded to their type
    k = _rotate(s["k"][live].double(), cos.double(), sin.double(), inter)
    if c["op"] == "append":
        s["k_pool"][page, :, slot] = k.to(dt)
        s["v_pool"][page, :, slot] = s["v"][live]
        s["kbar"][seq[full], pos[full] // P] = s["k_pool"][filled].float().sum(2) * (1.0 / P)
        return dict(q=s["q_out"], kbar=s["kbar"], k_pool=s["k_pool"], v_pool=s["v_pool"])
    lane = torch.arange(D // 2, device=page.device)
    block = torch.arange(D // 32, device=page.device)
    for pool, x, held in ((s["k_pool"], k, s["k_held"]), (s["v_pool"], s["v"][live].float(), s["v_held"])):
        code, byte = _quantise(x)
        pool[page[:, None], :, slot[:, None] * (D // 2) + lane] = (code[..., 0::2] | (code[..., 1::2] << 4)).transpose(1, 2)
        pool[page[:, None], :, P * D // 2 + block * P + slot[:, None]] = byte.transpose(1, 2)
        held[live] = _values(code, byte).to(dt)
    s["kbar"][seq[full], pos[full] // P] = _values(*_unpack(s["k_pool"][filled], P, D)).sum(2) * (1.0 / P)
    return dict(q=s["q_out"], kbar=s["kbar"], k=s["k_held"], v=s["v_held"])


def _attend_plain(s):
    c = s["case"]
    P, D, Hq, Hkv, B, n = c["page"], c["head_dim"], c["q_heads"], c["kv_heads"], c["seqs"], c["rows"]
    G, dev = Hq // Hkv, s["q"].device
    live, seq, pos = _rows(s, s["q"].shape[0])
    row = live - s["starts"].long()[seq]
    q = torch.zeros((B, n, Hq, D), dtype=torch.float32, device=dev)
    q[seq, row] = s["q"][live].float()
    at = torch.full((B, n), -1, dtype=torch.int64, device=dev)   # positions, -1 where there is no row
    at[seq, row] = pos
    o = torch.empty((B, n, Hq, D), dtype=torch.float32, device=dev)
    lse = torch.empty((B, n, Hq), dtype=torch.float32, device=dev)
    every = torch.arange(s["tables"].shape[1], device=dev).expand(B, -1)
    for g in range(Hkv):
        ids = every if s["sel"] is None else s["sel"][:, g].long()
        held = torch.ones_like(ids, dtype=torch.bool) if s["sel"] is None else \
            torch.arange(ids.shape[1], device=dev) < s["cnt"][:, g, None]
        tiles = s["tables"].gather(1, ids.clamp(min=0)).long()
        k, v = (_values(*_unpack(pool[tiles, g], P, D)).flatten(1, 2) for pool in (s["k_pool"], s["v_pool"]))   # [B][tokens][D]
        token = torch.where(held, ids * P, 1 << 40)[..., None] + torch.arange(P, device=dev)
        seen = token.flatten(1)[:, None] <= at[..., None]   # [B][n][tokens]
        x = q[:, :, g * G:(g + 1) * G].flatten(1, 2) @ k.transpose(1, 2).contiguous() * (1.0 / math.sqrt(D))
        x = x.unflatten(1, (n, G)).masked_fill(~seen[:, :, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        p = (x - top).exp()
        total = p.sum(-1, keepdim=True)
        y = p.flatten(1, 2) @ v
        o[:, :, g * G:(g + 1) * G] = y.unflatten(1, (n, G)) / torch.where(total == 0, 1.0, total)
        lse[:, :, g * G:(g + 1) * G] = (top + total.log())[..., 0]
    s["o"][live] = o[seq, row].to(s["o"].dtype)
    s["lse"][:, live] = lse[seq, row].t()
    return dict(o=s["o"], lse=s["lse"])


# ------------------------------------------------------------------------------------------------ in 64 bits, sequence by sequence

def _level_of(x):
    """x [..., 32] float64 -> the nearest value of the 4-bit grid under the block's scale."""
    top = x.abs().amax(-1, keepdim=True)
    frac, e = torch.frexp(top)                       # top = frac 2^e, frac in [0.5, 1)
    e = torch.where(frac <= 0.875, e - 3, e - 2).clamp(-125, 125)
    unit = torch.ldexp(torch.ones_like(top), e)
    grid = torch.tensor(_LEVELS, dtype=torch.float64, device=x.device)
    a = (x.abs() / unit).clamp(max=6.0)
    above = torch.searchsorted(grid, a).clamp(max=7)
    below = (above - 1).clamp(min=0)
    up, down = grid[above] - a, a - grid[below]
    take = torch.where(up == down, torch.where(above % 2 == 0, above, below), torch.where(up < down, above, below))
    return torch.copysign(grid[take], x) * unit


def _turn(x, angle_cos, angle_sin, interleaved, sign):
    """The rotation as a product with a complex number per pair."""
    half = angle_cos.shape[-1]
    x = x.double()
    if interleaved:
        first, second = torch.arange(0, 2 * half, 2, device=x.device), torch.arange(1, 2 * half, 2, device=x.device)
    else:
        first, second = torch.arange(half, device=x.device), torch.arange(half, 2 * half, device=x.device)
    z = torch.complex(x[..., first], x[..., second]) * torch.complex(angle_cos.double(), sign * angle_sin.double())[:, None]
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    P, D, Hkv, G = c["page"], c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    spans, starts = _spans(c), s["starts"].tolist()
    if c["op"] == "kv4_attn":
        o, lse = s["o"].double(), s["lse"].double()
        for b, (n, t) in enumerate(spans):
            for g in range(Hkv) if n else ():
                ids = torch.arange(-(-t // P), device=s["q"].device)
                if s["sel"] is not None:
                    ids = s["sel"][b, g, :int(s["cnt"][b, g])].long()
                tiles = s["tables"][b, ids].long()
                token = (ids[:, None] * P + torch.arange(P, device=ids.device)).flatten()
                k, v = (_values(*_unpack(pool[tiles, g], P, D)).double().flatten(0, 1) for pool in (s["k_pool"], s["v_pool"]))
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

    names = {"append": ("q_out", "kbar", "k_pool", "v_pool"), "append_grad": ("dq_out", "dk", "dv"), "kv4_append": ("q_out", "kbar", "k_held", "v_held")}
    out = {name: s[name].double() for name in names[c["op"]]}
    for b, (n, t) in enumerate(spans):
        if not n:
            continue
        rows, pos = slice(starts[b], starts[b] + n), torch.arange(t - n, t, device=s["tables"].device)
        cos, sin = s["cos"][pos], s["sin"][pos]
        page, slot = s["tables"][b, pos // P].long(), pos % P
        if c["op"] == "append_grad":
            out["dq_out"][rows] = _turn(s["dq"][rows], cos, sin, c["interleaved"], -1.0)
            out["dk"][rows] = _turn(s["dk_pool"][page, :, slot], cos, sin, c["interleaved"], -1.0)
            out["dv"][rows] = s["dv_pool"][page, :, slot].double()
            continue
        out["q_out"][rows] = _turn(s["q"][rows], cos, sin, c["interleaved"], 1.0)
        k, v = _turn(s["k"][rows], cos, sin, c["interleaved"], 1.0), s["v"][rows].double()
        if c["op"] == "append":
            out["k_pool"][page, :, slot] = k
            out["v_pool"][page, :, slot] = v
            k = k.to(s["k_pool"].dtype).double()   # the mean is that of the keys as they are kept
        else:
            k, v = (_level_of(x.unflatten(-1, (D // 32, 32))).flatten(-2) for x in (k, v))
            out["k_held"][rows], out["v_held"][rows] = k, v
        for l in range((t - n) // P, t // P):      # pages that these rows fill
            tile = s["k_pool"][int(s["tables"][b, l])]
            keys = (tile.double() if c["op"] == "append" else _values(*_unpack(tile, P, D)).double()).clone()
            first = max(0, t - n - l * P)
            keys[:, first:] = k[l * P + first - (t - n):(l + 1) * P - (t - n)].transpose(0, 1)
            out["kbar"][b, l] = keys.mean(1)
    if c["op"] == "append_grad":
        return dict(dq=out["dq_out"], dk=out["dk"], dv=out["dv"])
    if c["op"] == "append":
        return dict(q=out["q_out"], kbar=out["kbar"], k_pool=out["k_pool"], v_pool=out["v_pool"])
    return dict(q=out["q_out"], kbar=out["kbar"], k=out["k_held"], v=out["v_held"])


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """Bytes: every input read once, every output written once.  Operations: 4 D for each pair of a query and a token that it sees,
    6 for each rotated pair of dims (two products and a sum each), one per value that is quantised or summed."""
    c = case
    es, gs = (2 if c["dtype"] == "bf16" else 4), (2 if c["grad_dtype"] == "bf16" else 4)
    D, P, Hq, Hkv = c["head_dim"], c["page"], c["q_heads"], c["kv_heads"]
    tile = D / 2 + D / 32
    spans = _spans(c)
    R = sum(n for n, _ in spans)
    if c["op"] == "kv4_attn":
        pairs = held = 0
        for n, t in spans:
            if n == 0:
                continue
            past = (t - n) // P
            hidden = 0 if not c["top_k"] else (past - min(c["top_k"], past)) * P   # past tokens in no list
            held += t - hidden
            pairs += n * (t - n - hidden) + n * (n + 1) // 2
        return {"bytes": held * Hkv * 2 * tile + 2 * R * Hq * D * es + 4 * R * Hq, "flops": 4.0 * D * pairs * Hq}
    turned = 3.0 * c["rot"] * R * (Hq + Hkv)
    size = 2 * R * Hq * D * es + R * c["rot"] * 4
    if c["op"] == "append_grad":
        return {"bytes": size + 2 * R * Hkv * D * (es + gs), "flops": turned}
    fills = sum(t // P - (t - n) // P for n, t in spans)   # pages that the new rows fill
    size += 2 * R * Hkv * D * es + fills * Hkv * D * 4
    size += 2 * R * Hkv * (D * es if c["op"] == "append" else tile + D * es)
    return {"bytes": size, "flops": turned + fills * P * Hkv * D + (2.0 * R * Hkv * D if c["op"] != "append" else 0.0)}
