"""Performance cases of the operators of decoding on a shared cache.

``beam``    the best continuations of every group of beams, over beams and
            vocabulary (``binding.hs_beam_select``);
``copy``    pages of a key/value cache copied within it, in every layer: forks of
            a partly filled page, moves of whole pages (``binding.hs_cache_copy``);
``prefix``  attention of one row a sequence over a paged cache whose sequences
            share their first positions in groups (``binding.hs_prefix_attention``).

With ``own`` false, ``run`` computes them in elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
TILE = 32   # positions of a value tile of the cache

# Query heads, key/value heads and head size of the stacks that the caches belong to.
HEADS = {"tiny": (4, 2, 64), "talker": (16, 16, 64), "thinker": (28, 4, 128), "mixed": (32, 8, 128)}


def _beam(name, groups, beams, vocab, select, dtype, masked=0.0, done=0.0, pad=0):
    """masked: share of masked tokens; done: share of beams that have ended (as many are empty)."""
    return dict(name=name, op="beam", groups=groups, beams=beams, vocab=vocab, select=select, dtype=dtype,
                masked=masked, done=done, pad=pad)


def _copy(name, heads, layers, page, slots, copies, fill):
    """fill: the most positions that a copied page holds; every copy has its own number, or all whole pages."""
    return dict(name=name, op="copy", heads=heads, layers=layers, page=page, slots=slots, copies=copies, fill=fill)


def _prefix(name, heads, seqs, groups, prefix, rest, page, dtype, pad=0):
    """prefix: shared positions of the largest group; rest: most positions that a sequence has to itself."""
    return dict(name=name, op="prefix", heads=heads, seqs=seqs, groups=groups, prefix=prefix, rest=rest, page=page,
                dtype=dtype, pad=pad)


def listed():
    return [
        # One request's four beams: the smallest step, as many candidates as beams.
        _beam("beam_one", 1, 4, 32000, 4, "f32"),
        # A decode batch of eight requests, logits as the head leaves them; twice the beams are kept,
        # so that ended candidates leave enough others.
        _beam("beam_decode", 8, 4, 65536, 8, "f32", done=0.1),
        # A large batch of wide beams.
        _beam("beam_wide", 64, 8, 131072, 16, "bf16"),
        # Constrained decoding: most of an odd vocabulary masked, odd row starts, ended and empty beams.
        _beam("beam_masked", 17, 5, 50001, 10, "f16", masked=0.9, done=0.2, pad=3),
        # One beam leaves its parent: the filled part of its last page.
        _copy("copy_one", "thinker", 4, 512, 8, 1, 64),
        # A downstream decode batch after a selection: every other beam takes a copy of its parent's last page.
        _copy("copy_fork", "talker", 16, 512, 48, 16, 512),
        # Small pages, ragged fills.
        _copy("copy_ragged", "mixed", 1, 64, 700, 301, 63),
        # A cache made dense again: whole pages move.
        _copy("copy_compact", "mixed", 1, 1024, 256, 120, 0),
        # Two beams of a short prompt: the smallest call.
        _prefix("prefix_short", "talker", 2, 1, 200, 9, 64, "f16"),
        # One request's beams behind a long prompt.
        _prefix("prefix_beams", "thinker", 8, 1, 8192, 128, 512, "f16"),
        # Requests with several system prompts of odd lengths, small pages.
        _prefix("prefix_ragged", "mixed", 45, 5, 1501, 700, 64, "bf16", pad=8),
        # A full decode batch behind one document.
        _prefix("prefix_batch", "mixed", 128, 1, 16384, 512, 512, "f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes over their logarithm, every type, aligned and odd strides."""
    op = rng.choice(("beam", "copy", "prefix"))
    if op == "beam":
        v, dtype = _log(rng, 1000, 160000), rng.choice(("f32", "bf16", "f16"))
        if rng.random() < 0.5:
            v = v // 8 * 8
        beams = _log(rng, 1, 16)
        c = _beam("", _log(rng, 1, max(1, min(256, 130_000_000 // (v * beams * SIZE[dtype])))), beams, v,
                  beams * rng.choice((1, 2, 2, 4)), dtype, rng.choice((0.0, 0.0, 0.5, 0.99)),
                  rng.choice((0.0, 0.0, 0.2)), rng.choice((0, 0, 0, 1, 8, 24)))
    elif op == "copy":
        heads, page = rng.choice(sorted(HEADS)), 64 * _log(rng, 1, 32)
        _, hkv, dh = HEADS[heads]
        layers = rng.choice((1, 2, 4, 16, 28))
        most = 120_000_000 // (layers * page * hkv * dh)     # pages that a copy may move in all
        copies = _log(rng, 1, max(1, min(700, most)))
        c = _copy("", heads, layers, page, 2 * copies + _log(rng, 1, 20), copies,
                  rng.choice((0, page, _log(rng, 1, page))))
    else:
        heads = rng.choice(sorted(HEADS))
        seqs = _log(rng, 1, 96)
        groups = rng.choice((1, 1, _log(rng, 1, seqs)))
        rest = rng.choice((1, _log(rng, 1, 512)))
        prefix = rng.choice((0, _log(rng, 32, 16384), _log(rng, 32, 16384), _log(rng, 32, 16384)))
        c = _prefix("", heads, seqs, groups, prefix // max(1, groups // 4), rest, 64 * _log(rng, 1, 32),
                    rng.choice(("f16", "f16", "bf16")), rng.choice((0, 0, 8, 64)))
    del c["name"]
    return c


def _fills(case):
    """Positions of each copy: the widths of a linear spread from 1 to `fill`, whole pages where fill is 0."""
    if not case["fill"]:
        return [case["page"]] * case["copies"]
    return [1 + (case["fill"] - 1) * (i + 1) // case["copies"] for i in range(case["copies"])]


def _lengths(case):
    """(rows of each group, its prefix, positions that each sequence has to itself): spread over their ranges."""
    n, g = case["seqs"], case["groups"]
    rows = [n * (i + 1) // g - n * i // g for i in range(g)]
    prefix = [case["prefix"] * (g - i) // g for i in range(g)]
    rest = [(case["rest"] * ((37 * i) % n + 1) + n - 1) // n for i in range(n)]
    return rows, prefix, rest


def work(case):
    if case["op"] == "beam":
        rows = case["groups"] * case["beams"]
        n = rows * case["vocab"]
        return {"bytes": n * SIZE[case["dtype"]] + 4 * rows + 12 * case["groups"] * case["select"], "flops": 4 * n}
    hq, hkv, dh = HEADS[case["heads"]]
    if case["op"] == "copy":
        whole = sum((f + TILE - 1) // TILE * TILE for f in _fills(case))
        return {"bytes": 2 * 2 * 2 * case["layers"] * whole * hkv * dh, "flops": 0}
    rows, prefix, rest = _lengths(case)
    shared, keys = sum(p for p in prefix), sum(r * p for r, p in zip(rows, prefix)) + sum(rest)
    return {"bytes": 2 * 2 * (shared + sum(rest)) * hkv * dh + 2 * 2 * case["seqs"] * hq * dh,
            "flops": 4 * keys * hq * dh}


# ---------------------------------------------------------------------------- inputs

def _wide(rows, cols, pad, dtype):
    """[rows, cols] view of a matrix with `pad` more columns."""
    return torch.empty((rows, cols + pad), dtype=dtype, device="cuda")[:, :cols]


def _cache(gen, layers, slots, hkv, page, dh):
    """Keys [slots, hkv, page, dh] and values [slots, hkv, page / 32, dh, 32] of every layer."""
    def new(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float16)
    return ([new(slots, hkv, page, dh) for _ in range(layers)],
            [new(slots, hkv, page // TILE, dh, TILE) for _ in range(layers)])


def _prepare_beam(case, gen, st):
    groups, beams, v = case["groups"], case["beams"], case["vocab"]
    rows = groups * beams
    z = torch.randn((rows, v), generator=gen, device="cuda").mul_(2.5)
    # What a model is sure of: one token stands out, by little in some rows and far in others.
    at = torch.randint(0, v, (rows, 1), generator=gen, device="cuda")
    z.scatter_add_(1, at, 12 * torch.rand((rows, 1), generator=gen, device="cuda"))
    if case["masked"]:
        z.masked_fill_(torch.rand((rows, v), generator=gen, device="cuda") < case["masked"], -math.inf)
    st["logits"] = _wide(rows, v, case["pad"], TYPES[case["dtype"]])
    st["logits"].copy_(z)
    # Beams of a request lie close together, and far from zero after some steps.
    score = -60 * torch.rand((groups, 1), generator=gen, device="cuda") - 5 * torch.rand(
        (groups, beams), generator=gen, device="cuda")
    st["end"], st["finished"] = 2, None
    if case["done"]:
        u = torch.rand((groups, beams), generator=gen, device="cuda")
        st["finished"] = (u < case["done"]).to(torch.uint8)
        score.masked_fill_(u > 1 - case["done"], -math.inf)
    st["scores"] = score


def _prepare_copy(case, gen, st):
    _, hkv, dh = HEADS[case["heads"]]
    st["k"], st["v"] = _cache(gen, case["layers"], case["slots"], hkv, case["page"], dh)
    order = torch.randperm(case["slots"], generator=gen, device="cuda").tolist()
    n = case["copies"]
    # Forks: two children of a parent in places.
    st["dst"] = order[:n]
    parents = order[n:]
    st["src"] = [parents[(i // 2 if i % 5 < 2 else i) % len(parents)] for i in range(n)]
    st["fill"] = _fills(case)


def _prepare_prefix(case, gen, st):
    hq, hkv, dh = HEADS[case["heads"]]
    page, n = case["page"], case["seqs"]
    rows, prefix, rest = _lengths(case)
    offsets = [0]
    for r in rows:
        offsets.append(offsets[-1] + r)
    lens = [p + rest[i] for g, p in enumerate(prefix) for i in range(offsets[g], offsets[g + 1])]
    per_seq = max(1, (max(lens) + page - 1) // page)
    # A group's pages up to the end of its prefix, then each sequence's own; a page that the prefix ends in
    # is a copy of its own in every sequence but read from the first one's.
    whole = [p // page for p in prefix]
    slots = sum(whole) + sum((m + page - 1) // page - whole[g] for g in range(len(rows))
                             for m in lens[offsets[g]:offsets[g + 1]]) + 3
    order = torch.randperm(slots, generator=gen, device="cuda").tolist()
    table = [[0] * per_seq for _ in range(n)]
    for g in range(len(rows)):
        shared = [order.pop() for _ in range(whole[g])]
        for i in range(offsets[g], offsets[g + 1]):
            pages = shared + [order.pop() for _ in range((lens[i] + page - 1) // page - whole[g])]
            table[i][:len(pages)] = pages
    (st["k"],), (st["v"],) = _cache(gen, 1, slots, hkv, page, dh)
    # Heads that look at a few positions and heads that look at many.
    q = torch.randn((n, hq, dh), generator=gen, device="cuda")
    q *= torch.exp(torch.linspace(-1, 1.2, hq, device="cuda"))[:, None]
    st["q"] = _wide(n, hq * dh, case["pad"], TYPES[case["dtype"]])
    st["q"].copy_(q.view(n, hq * dh))

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")
    st.update(table=ints(table), lens=ints(lens), offsets=ints(offsets), prefix=ints(prefix), host_offsets=offsets,
              max_prefix=max(prefix), max_rest=max(rest))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case=case)
    {"beam": _prepare_beam, "copy": _prepare_copy, "prefix": _prepare_prefix}[case["op"]](case, gen, st)
    return st


# ---------------------------------------------------------------------------- plain forms

def _plain_beam(logits, scores, finished, end, select):
    groups, beams = scores.shape
    z = logits.float() + 0.0
    rows, v = z.shape
    k = min(select, v)
    # Candidates next to each other at the border need 64 bits.
    m = z.amax(-1, keepdim=True).double()
    m = torch.where(m > -math.inf, m, 0)
    log_s = torch.log(torch.exp((z - m.float())).sum(-1, keepdim=True, dtype=torch.float64)) + m
    # A row's own order: the value's, then the lower token.
    bits = z.view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32
    best = (order + torch.arange(v - 1, -1, -1, device=z.device)).topk(k, -1).values
    token = v - 1 - (best & 0xFFFFFFFF)
    value = z.gather(1, token).double() - log_s + scores.view(rows, 1).double()
    value = torch.where(z.gather(1, token) > -math.inf, value, -math.inf)
    if finished is not None:
        over = finished.view(rows, 1) != 0
        first = torch.arange(k, device=z.device) == 0
        value = torch.where(over, torch.where(first, scores.view(rows, 1).double(), -math.inf), value)
        token = torch.where(over, end, token)
    value, token = value.view(groups, beams * k), token.view(groups, beams * k)
    value, at = value.sort(dim=-1, descending=True, stable=True)
    value, at = value[:, :select], at[:, :select]
    none = value == -math.inf
    parent = torch.where(none, -1, at // k)
    token = torch.where(none, -1, token.gather(1, at))
    done = token == end
    if finished is not None:
        done = done | (finished.gather(1, parent.clamp(min=0)) != 0) & ~none
    out = {"scores": value.float(), "parents": parent.int(), "tokens": token.int(), "finished": done.to(torch.uint8)}
    if value.shape[1] < select:   # fewer candidates than asked for
        pad = select - value.shape[1]
        for name, fill in (("scores", -math.inf), ("parents", -1), ("tokens", -1), ("finished", 0)):
            out[name] = torch.nn.functional.pad(out[name], (0, pad), value=fill)
    return out


def _plain_copy(ks, vs, src, dst, fill):
    # Copies of one length at a time: a tensor index cannot say how much of a page it means.
    lengths = {}
    for s, d, f in zip(src, dst, fill):
        lengths.setdefault((f + TILE - 1) // TILE, []).append((s, d))
    for tiles, pairs in lengths.items():
        at = torch.tensor(pairs, device=ks[0].device)
        s, d = at[:, 0], at[:, 1]
        for k, v in zip(ks, vs):
            k[d, :, :tiles * TILE] = k[s, :, :tiles * TILE]
            v[d, :, :tiles] = v[s, :, :tiles]


def _positions(cache, slots, at, page, value):
    """fp32 rows [hkv, dh] of positions `at` in the pages `slots` (same shape each)."""
    if value:
        p = at % page
        return cache[slots, :, p // TILE, :, p % TILE].float()
    return cache[slots, :, at % page].float()


def _plain_prefix(q, k, v, table, lens, prefix, offsets, heads, dtype):
    hq, hkv, dh = heads
    n, page, dev = q.shape[0], k.shape[2], q.device
    scale = 1 / math.sqrt(dh)
    qh = q.float().view(n, hkv, hq // hkv, dh)
    lens, starts, out = lens.long(), [], torch.empty((n, hq, dh), dtype=dtype, device=dev)
    for g in range(len(offsets) - 1):
        starts += [prefix[g].long().expand(offsets[g + 1] - offsets[g])]
    start = torch.cat(starts)
    most = int((lens - start).max())
    # What each sequence has to itself, padded to the longest.
    at = start[:, None] + torch.arange(most, device=dev)
    there = at < lens[:, None]
    at = torch.where(there, at, 0)
    slots = table.long().gather(1, at // page)
    own_k, own_v = _positions(k, slots, at, page, False), _positions(v, slots, at, page, True)
    own_s = torch.matmul(qh, own_k.permute(0, 2, 3, 1).contiguous()) * scale        # [n, hkv, G, most]
    own_s = own_s.masked_fill(~there[:, None, None], -math.inf)
    own_v = torch.where(there[:, :, None, None], own_v, 0).permute(0, 2, 1, 3).contiguous()
    for g in range(len(offsets) - 1):
        lo, hi = offsets[g], offsets[g + 1]
        if lo == hi:
            continue
        p = torch.arange(int(prefix[g]), device=dev)
        slots = table[lo].long()[p // page]
        pk = _positions(k, slots, p, page, False).permute(1, 2, 0).contiguous()      # [hkv, dh, P]
        pv = _positions(v, slots, p, page, True).permute(1, 0, 2).contiguous()       # [hkv, P, dh]
        rows = qh[lo:hi].permute(1, 0, 2, 3).reshape(hkv, (hi - lo) * (hq // hkv), dh)
        s = (torch.matmul(rows, pk) * scale).view(hkv, hi - lo, hq // hkv, len(p))
        s = torch.cat((s, own_s[lo:hi].permute(1, 0, 2, 3)), -1)
        m = s.amax(-1, keepdim=True)
        e = torch.exp(s - torch.where(m > -math.inf, m, 0))
        total = e.sum(-1, keepdim=True)
        e = torch.where(total > 0, e / total, 0)
        o = torch.matmul(e[..., :len(p)].reshape(hkv, rows.shape[1], len(p)), pv).view(hkv, hi - lo, hq // hkv, dh)
        o = o + torch.matmul(e[..., len(p):], own_v[lo:hi].permute(1, 0, 2, 3))
        out[lo:hi] = o.permute(1, 0, 2, 3).reshape(hi - lo, hq, dh).to(dtype)
    return out.view(n, hq * dh)


# ---------------------------------------------------------------------------- one pass

_context = None


def _ctx():
    """The program's one context."""
    global _context
    if _context is None:
        from paper_2608_01785_amd import binding
        _context = binding.hs_context_create(0, (256,))
    return _context


def _buffers(st):
    """The outputs and the workspace that a program keeps from call to call."""
    if "out" in st:
        return st["out"]
    from paper_2608_01785_amd import binding
    case = st["case"]

    def new(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if case["op"] == "beam":
        shape = (case["groups"], case["select"])
        st["out"] = {"scores": new(shape, torch.float32), "parents": new(shape, torch.int32),
                     "tokens": new(shape, torch.int32), "finished": new(shape, torch.uint8)}
        size = binding.hs_beam_select_workspace_size(case["groups"], case["beams"], case["vocab"], case["select"])
    elif case["op"] == "copy":
        st["out"], size = {"k": st["k"], "v": st["v"]}, 0
    else:
        hq, hkv, dh = HEADS[case["heads"]]
        st["out"] = new((case["seqs"], hq * dh), TYPES[case["dtype"]])
        size = binding.hs_prefix_attention_workspace_size(hq, hkv, dh, case["seqs"], st["max_prefix"],
                                                          st["max_rest"])
    st["ws"] = new(max(1, size), torch.uint8)
    torch.cuda.synchronize()
    return st["out"]


def run(st):
    case = st["case"]
    if own:
        from paper_2608_01785_amd import binding
        out = _buffers(st)
        if case["op"] == "beam":
            binding.hs_beam_select(_ctx(), st["logits"], st["scores"], out["scores"], out["parents"], out["tokens"],
                                   finished=st["finished"], out_finished=out["finished"], end_token=st["end"],
                                   workspace=st["ws"])
        elif case["op"] == "copy":
            binding.hs_cache_copy(_ctx(), (st["k"], st["v"], case["slots"], case["page"]), st["src"], st["dst"],
                                  st["fill"])
        else:
            binding.hs_prefix_attention(_ctx(), st["q"], out, st["k"], st["v"], st["table"], st["lens"],
                                        st["offsets"], st["prefix"], st["max_prefix"], st["max_rest"],
                                        workspace=st["ws"])
        return out
    if case["op"] == "beam":
        return _plain_beam(st["logits"], st["scores"], st["finished"], st["end"], case["select"])
    if case["op"] == "copy":
        _plain_copy(st["k"], st["v"], st["src"], st["dst"], st["fill"])
        return {"k": st["k"], "v": st["v"]}
    return _plain_prefix(st["q"], st["k"], st["v"], st["table"], st["lens"], st["prefix"], st["host_offsets"],
                         HEADS[case["heads"]], TYPES[case["dtype"]])


# ---------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "beam":
        groups, beams, v, select = case["groups"], case["beams"], case["vocab"], case["select"]
        out = torch.full((groups, select), -math.inf, dtype=torch.float64, device="cuda")
        for g in range(groups):
            lp = torch.log_softmax(st["logits"][g * beams:(g + 1) * beams].to(torch.float64), -1)
            total = torch.nan_to_num(lp, nan=-math.inf, neginf=-math.inf) + st["scores"][g].to(torch.float64)[:, None]
            if st["finished"] is not None:
                ended = st["finished"][g].bool()
                total[ended] = -math.inf
                total[ended, 0] = st["scores"][g][ended].to(torch.float64)
            top = torch.topk(total.view(-1), min(select, beams * v)).values
            out[g, :len(top)] = top
        return {"scores": out, "parents": None, "tokens": None, "finished": None}
    if case["op"] == "copy":
        # One copy after the other: no page is both written and read.
        tiles = [-(-f // TILE) for f in st["fill"]]
        for k, v in zip(st["k"], st["v"]):
            by_tile = k.view(k.shape[0], k.shape[1], -1, TILE, k.shape[3])
            for s, d, n in zip(st["src"], st["dst"], tiles):
                by_tile[d, :, :n].copy_(by_tile[s, :, :n])
                v[d, :, :n].copy_(v[s, :, :n])
        return {"k": st["k"], "v": st["v"]}
    hq, hkv, dh = HEADS[case["heads"]]
    page = case["page"]
    if case["seqs"] * max(st["lens"].tolist()) > 5_000_000:
        return None
    out = torch.zeros((case["seqs"], hq, dh), dtype=torch.float64, device="cuda")
    offsets, prefix, lens = st["host_offsets"], st["prefix"].tolist(), st["lens"].tolist()
    table = st["table"].tolist()
    for g in range(len(prefix)):
        for i in range(offsets[g], offsets[g + 1]):
            # The sequence's pages end to end: whole pages of the first sequence's table under the prefix.
            def line(owner, lo, hi):
                slots = [table[owner][j] for j in range(lo // page, (hi + page - 1) // page)]
                keys = torch.cat([st["k"][s].transpose(0, 1) for s in slots])
                values = torch.cat([st["v"][s].permute(1, 3, 0, 2).reshape(page, hkv, dh) for s in slots])
                part = slice(lo - lo // page * page, hi - lo // page * page)
                return keys[part].to(torch.float64), values[part].to(torch.float64)
            parts = []
            if prefix[g]:
                parts.append(line(offsets[g], 0, prefix[g]))
            if lens[i] > prefix[g]:
                parts.append(line(i, prefix[g], lens[i]))
            if not parts:
                continue
            keys, values = (torch.cat(x) for x in zip(*parts))
            qi = st["q"][i].to(torch.float64).view(hkv, hq // hkv, dh)
            w = torch.softmax(torch.einsum("hgd,phd->hgp", qi, keys) / math.sqrt(dh), -1)
            out[i] = torch.einsum("hgp,phd->hgd", w, values).reshape(hq, dh)
    return out.view(case["seqs"], hq * dh)
