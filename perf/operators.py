"""The paged prefix cache's operators, as a user of the library calls them, over the sizes they come in.

Kinds of case (key "kind"):
  extend  dopr.cache_extend: block tables, slot map, positions and packed offsets of a step's new tokens, from the
          lengths that the sequences have and get
  rotate  dopr.rope_apply: rotary positions on the query and key heads of packed rows (inverse: their gradient)
  append  dopr.cache_append: rotary positions on a layer's new rows, keys and values into the cache's pages
  attend  dopr.shared_attention: sequences that share stored prefixes attend to the prefix, read once for all of
          them, then causally to their own keys

Head counts are those of the Qwen3 shapes the repository is configured for (32 / 8 and 16 / 8 heads of 128), and
generic ones in drawn cases.  Lengths and shapes of attend cases go by the case, everything else by the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"


# ------------------------------------------------------------------ cases
def _extend(name, rows, prefixes, page, held_lo, held_hi, new_lo, new_hi, release=0.0):
    return dict(name=name, kind="extend", rows=rows, prefixes=prefixes, page=page, held_lo=held_lo, held_hi=held_hi,
                new_lo=new_lo, new_hi=new_hi, release=release)


def _rows(name, kind, tokens, hq, hkv, d, dtype, **more):
    return dict(name=name, kind=kind, tokens=tokens, hq=hq, hkv=hkv, d=d, dtype=dtype, rotary=more.get("rotary", d),
                interleaved=more.get("interleaved", False), scaling=more.get("scaling", "plain"),
                factor=more.get("factor", 1.0), far=more.get("far", 8192), inverse=more.get("inverse", False),
                page=more.get("page", 64))


def _attend(name, hq, hkv, d, dtype, page, docs, m_lo, m_hi, reqs, own_lo, own_hi, new_lo, new_hi, **more):
    return dict(name=name, kind="attend", hq=hq, hkv=hkv, d=d, dtype=dtype, page=page, docs=docs, m_lo=m_lo, m_hi=m_hi,
                reqs=reqs, own_lo=own_lo, own_hi=own_hi, new_lo=new_lo, new_hi=new_hi, lens=more.get("lens", 1))


def listed():
    return [
        # a step of 64 running sequences, a token each: what every step begins with
        _extend("extend 64 sequences by a token", 65, 1, 64, 20, 400, 1, 1),
        # a batch of 2,000 queries arrives for 100 stored documents, in small pages
        _extend("extend 2000 queries", 2100, 100, 16, 0, 0, 8, 64),
        # documents of up to 8,192 tokens enter while finished sequences hand their pages back
        _extend("extend documents, some released", 64, 0, 32, 0, 3000, 0, 8192, release=0.3),
        # one new token's heads
        _rows("rotate one token", "rotate", 1, 32, 8, 128, "bf16"),
        # gradient of interleaved rotary positions on half of each head, at far positions of a stretched range
        _rows("rotate gradient, interleaved half heads", "rotate", 4097, 16, 8, 128, "f32", rotary=64, interleaved=True,
              scaling="ramp", factor=8.0, far=250000, inverse=True),
        # a step of 64 sequences: a row each into the cache
        _rows("append 64 rows", "append", 64, 32, 8, 128, "bf16"),
        # a whole scoring chunk's rows into the cache
        _rows("append a chunk", "append", 26800, 32, 8, 128, "f16", page=32),
        # one query's next token on a short document
        _attend("attend one token", 32, 8, 128, "bf16", 64, 1, 512, 512, 1, 24, 24, 1, 1),
        # 64 queries' next tokens on one long document
        _attend("attend 64 queries, one long document", 32, 8, 128, "bf16", 64, 1, 32768, 32768, 64, 8, 64, 1, 1),
        # next tokens over many documents, ragged, small pages, arrival order
        _attend("attend ragged documents", 16, 8, 128, "bf16", 16, 64, 1, 1024, 256, 1, 256, 1, 1, lens=3),
        # queries scored over whole documents: every query token is new
        _attend("attend queries of 16 documents", 32, 8, 128, "f16", 32, 16, 256, 2048, 200, 8, 64, 8, 64, lens=5),
        # long queries over one long document: the largest call
        _attend("attend 2048 rows, one long document", 32, 8, 128, "bf16", 128, 1, 16384, 16384, 32, 64, 64, 64, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["extend", "rotate", "append", "attend", "attend"])
    page = rng.choice([16, 32, 64, 128])
    if kind == "extend":
        rows = _log(rng, 2, 2100)
        hi = min(_log(rng, 1, 8192), max(1, 150000 // rows))
        held = min(_log(rng, 1, 4000), 400000 // rows)
        return {k: v for k, v in _extend("", rows, rng.choice([0, 1, max(1, rows // 20)]) if rows > 2 else 0, page, 0,
                                         held, rng.choice([0, 1, hi // 2]) if hi > 1 else 1, hi,
                                         rng.choice([0.0, 0.3])).items() if k != "name"}
    hkv = rng.choice([1, 2, 4, 8, 8])
    hq = hkv * rng.choice([1, 2, 4, 4, 5, 8])
    d = rng.choice([64, 128, 128])
    if kind in ("rotate", "append"):
        scaling = rng.choice(["plain", "linear", "ntk", "bands", "ramp"])
        c = _rows("", kind, min(_log(rng, 1, 26800), 26800 * 48 * 128 // ((hq + 2 * hkv) * d)), hq, hkv, d,
                  rng.choice(["f16", "bf16", "f32"] if kind == "rotate" else ["f16", "bf16"]),
                  rotary=rng.choice([d, d, d // 2, d // 4]), interleaved=rng.choice([False, True]), scaling=scaling,
                  factor=1.0 if scaling == "plain" else rng.choice([2.0, 4.0, 8.5]), far=_log(rng, 2000, 300000),
                  inverse=kind == "rotate" and rng.choice([False, True]), page=page)
        return {k: v for k, v in c.items() if k != "name"}
    m = _log(rng, 16, 32768)
    docs = rng.choice([1, 1, max(1, min(64, 16384 // m))])
    reqs = max(docs, _log(rng, 1, 256))
    new = rng.choice([1, 1, 1, min(64, max(1, 2048 // reqs))])
    own_hi = max(new, _log(rng, 1, 256))
    if reqs * new * m > 2048 * 16384:
        reqs = max(1, 2048 * 16384 // (new * m))
    c = _attend("", hq, hkv, d, rng.choice(["f16", "bf16"]), page, docs, max(1, m // rng.choice([1, 4])), m, reqs,
                min(own_hi, max(1, new // 2)), own_hi, max(1, new // 2), new, lens=rng.randrange(1, 1000))
    return {k: v for k, v in c.items() if k != "name"}


# ------------------------------------------------------------------ rotary frequencies, in 64 bits
def _rope_more(c):
    """Ranges of the scaled forms: the length the plain positions were made for and the two ends of the blend."""
    return dict(original=4096, low=1.0, high=4.0) if c["scaling"] == "bands" else dict(original=4096, low=1.0, high=32.0)


def _frequencies(c):
    """(d/2 angles per position, factor on cos and sin), numpy in 64 bits."""
    d, theta, s = c["rotary"], 1e6, c["factor"]
    more = _rope_more(c)
    i = np.arange(d // 2, dtype=np.float64)
    f, gain = theta ** (-2.0 * i / d), 1.0
    if c["scaling"] == "linear":
        f = f / s
    elif c["scaling"] == "ntk":
        f = (theta * s ** (d / (d - 2.0))) ** (-2.0 * i / d)
    elif c["scaling"] == "bands":
        turns = more["original"] * f / (2 * math.pi)
        t = np.clip((turns - more["low"]) / (more["high"] - more["low"]), 0, 1)
        f = (1 - t) * f / s + t * f
    elif c["scaling"] == "ramp":
        at = lambda r: d * math.log(more["original"] / (r * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
        lo, hi = max(math.floor(at(more["high"])), 0), min(math.ceil(at(more["low"])), d - 1)
        t = np.clip((i - lo) / max(hi - lo, 1e-3), 0, 1)
        f, gain = f / s * t + f * (1 - t), 0.1 * math.log(s) + 1.0
    return f, gain


# ------------------------------------------------------------------ prepare
def _gen(seed, more=0):
    g = torch.Generator(DEV)
    g.manual_seed(seed * 1000003 + more)
    return g


def _prepare_extend(c, seed):
    r = np.random.default_rng(seed)
    rows, pre, page = c["rows"], c["prefixes"], c["page"]
    held = r.integers(c["held_lo"], c["held_hi"] + 1, rows)
    new = r.integers(c["new_lo"], c["new_hi"] + 1, rows)
    if pre:
        held[:pre], new[:pre] = r.integers(64, 2049, pre), 0
    gone = r.random(rows) < c["release"]
    new[gone] = -1
    prefix = np.full(rows, -1)
    if pre:
        prefix[pre:] = r.integers(0, pre, rows - pre)
    max_blocks = max(-(-(c["held_hi"] + c["new_hi"]) // page), -(-2048 // page) if pre else 0)
    had = -(-held // page)
    total = pre * -(-2048 // page) + (rows - pre) * -(-(c["held_hi"] + c["new_hi"]) // page) + 64
    order = r.permutation(total)
    tables = r.integers(0, total, (rows, max_blocks))
    at = 0
    for i in range(rows):
        tables[i, :had[i]] = order[at:at + had[i]]
        at += had[i]
    free = r.integers(0, total, total)
    free[:total - at] = order[at:]
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)  # noqa: E731
    s = dict(c=c, seq_lens=i32(held), new_lens=i32(new), prefix=i32(prefix), tables=i32(tables), free=i32(free),
             n_free=i32([total - at]), max_tokens=max(1, (rows - pre) * c["new_hi"]), total=total)
    if own:
        from paper_2609_03311_gb300 import dopr

        s["layout"] = dopr.make_cache_layout(total, page, 8, 128, torch.bfloat16, rows, max_blocks)
        s["out"] = dopr.cache_batch(s["layout"], s["max_tokens"], DEV)
    return s


def _prepare_rows(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    T, hq, hkv, d = c["tokens"], c["hq"], c["hkv"], c["d"]
    # the packed q | k | v rows that a projection leaves
    qkv = torch.randn(T, (hq + 2 * hkv) * d, generator=g, device=DEV).to(dt)
    s = dict(c=c, qkv=qkv, positions=torch.randint(0, c["far"], (T,), generator=g, device=DEV, dtype=torch.int32))
    f, gain = _frequencies(c)
    s["freq"], s["gain"] = torch.from_numpy(f).to(DEV), gain
    if c["kind"] == "append":
        page = c["page"]
        blocks = -(-T // page) + 3
        s["slots"] = torch.randperm(blocks * page, generator=g, device=DEV)[:T]
        s["k_pool"] = torch.randn(blocks, hkv, page, d, generator=g, device=DEV).to(dt)
        s["v_pool"] = torch.randn(blocks, hkv, page, d, generator=g, device=DEV).to(dt)
    if own:
        from paper_2609_03311_gb300 import dopr

        more = _rope_more(c)
        s["rope"] = dopr.Rope(c["far"], c["rotary"], theta=1e6,
                              layout=dopr.ROPE_INTERLEAVED if c["interleaved"] else dopr.ROPE_HALF,
                              scaling=getattr(dopr, "ROPE_" + c["scaling"].upper()), factor=c["factor"],
                              original_max_position=more["original"], low=more["low"], high=more["high"])
        s["q_out"] = torch.empty(T, hq, d, device=DEV, dtype=dt)
        if c["kind"] == "rotate":
            s["k_out"] = torch.empty(T, hkv, d, device=DEV, dtype=dt)
        else:
            s["layout"] = dopr.make_cache_layout(blocks, page, hkv, d, dt, 1, blocks)
    return s


def _lengths(c):
    """Documents' lengths, requests' documents (arrival order), own lengths and new tokens: fixed by the case."""
    r = np.random.default_rng(c["lens"])
    m = r.integers(c["m_lo"], c["m_hi"] + 1, c["docs"])
    doc = r.integers(0, c["docs"], c["reqs"])
    held = r.integers(c["own_lo"], c["own_hi"] + 1, c["reqs"])
    new = np.minimum(r.integers(c["new_lo"], c["new_hi"] + 1, c["reqs"]), held)
    if c["own_lo"] == c["new_lo"] and c["own_hi"] == c["new_hi"]:
        new = held.copy()
    return m, doc, held, new


def _padded(lists, width):
    out = np.full((len(lists), width), -1)
    for i, v in enumerate(lists):
        out[i, :len(v)] = v
    return out


def _prepare_attend(c, seed):
    m, doc, held, new = _lengths(c)
    docs, reqs, page = c["docs"], c["reqs"], c["page"]
    lens = np.concatenate([m, held])
    rows = docs + reqs
    pages = -(-lens // page)
    max_blocks, blocks = int(pages.max()), int(pages.sum()) + 2
    order = np.random.default_rng(seed).permutation(blocks)
    tables = np.zeros((rows, max_blocks), dtype=np.int32)
    at = 0
    for i in range(rows):
        tables[i, :pages[i]] = order[at:at + pages[i]]
        at += pages[i]
    off = np.concatenate([np.zeros(docs + 1, dtype=np.int64), np.cumsum(new)])
    T = int(off[-1])
    g, dt = _gen(seed, 1), DTYPES[c["dtype"]]
    rand = lambda *shape: torch.randn(*shape, generator=g, device=DEV).to(dt)  # noqa: E731
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    s = dict(c=c, q=rand(T, c["hq"], c["d"]), k_pool=rand(blocks, c["hkv"], page, c["d"]),
             v_pool=rand(blocks, c["hkv"], page, c["d"]), tables=dev(tables), seq_lens=dev(lens.astype(np.int32)),
             tok_off=dev(off.astype(np.int32)), prefix=dev(np.concatenate([np.full(docs, -1), doc]).astype(np.int32)))
    # the plain form's plan: each document's and each request's tokens, padded with -1
    toks = [np.arange(off[docs + i], off[docs + i + 1]) for i in range(reqs)]
    by_doc = [np.concatenate([toks[i] for i in np.nonzero(doc == k)[0]] + [np.zeros(0, dtype=np.int64)])
              for k in range(docs)]
    s["doc_tok"] = dev(_padded(by_doc, max(len(v) for v in by_doc)))
    s["req_tok"] = dev(_padded(toks, int(new.max())))
    s["doc_len"], s["req_len"], s["req_new"] = dev(m), dev(held), dev(new)
    if own:
        from paper_2609_03311_gb300 import dopr

        s["layout"] = dopr.make_cache_layout(blocks, page, c["hkv"], c["d"], dt, rows, max_blocks)
        s["plan"] = dopr.shared_attention_plan(s["layout"], c["hq"], s["tok_off"], s["seq_lens"], s["prefix"], T)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(T, c["hq"], device=DEV)
        s["workspace"] = dopr.shared_attention_workspace(s["layout"], c["hq"], T, DEV)
    return s


def prepare(case, seed):
    kind = case["kind"]
    return (_prepare_extend if kind == "extend" else _prepare_attend if kind == "attend" else _prepare_rows)(case, seed)


# ------------------------------------------------------------------ the plain forms
def _plain_extend(s):
    c, page = s["c"], s["c"]["page"]
    held, new, prefix = s["seq_lens"].long(), s["new_lens"].long(), s["prefix"].long()
    gone = new < 0
    grow = new.clamp(min=0)
    had = (held + page - 1) // page
    # released pages go onto the stack first, in row and page order
    tables, free = s["tables"].clone(), s["free"].clone()
    col = torch.arange(tables.shape[1], device=DEV)
    back = gone[:, None] & (col < had[:, None])
    n_free = s["n_free"].long()
    given = tables[back]
    free[n_free + torch.arange(given.numel(), device=DEV)] = given
    top = n_free + given.numel()
    # then every row takes its new pages from the top
    lens = torch.where(gone, 0, held + grow)
    need = torch.where(gone, 0, (lens + page - 1) // page - had)
    before = torch.cumsum(need, 0) - need
    fresh = (col >= had[:, None]) & (col < (had + need)[:, None]) & ~gone[:, None]
    nth = before[:, None] + col - had[:, None]
    tables = torch.where(fresh, free[(top - 1 - nth).clamp(0, free.numel() - 1)], tables)
    off = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), torch.cumsum(grow, 0)])
    t = torch.arange(s["max_tokens"], device=DEV)
    row = torch.searchsorted(off[1:], t, right=True).clamp(max=held.numel() - 1)
    live = t < off[-1]
    at = held[row] + t - off[row]
    block = tables[row, (at // page).clamp(0, tables.shape[1] - 1)].long()
    base = torch.where(prefix < 0, 0, lens[prefix.clamp(min=0)])
    return dict(seq_lens=lens.int(), n_free=(top - need.sum()).int(), block_tables=tables, free_blocks=free,
                tok_off=off.int(), slots=torch.where(live, block * page + at % page, -1),
                positions=torch.where(live, base[row] + at, -1).int())


def _turn(x, s):
    """Rotary positions on x [tokens, heads, d] in 32 bits; angles in 64."""
    c, r = s["c"], s["c"]["rotary"]
    a = s["positions"].double()[:, None] * s["freq"]
    cos, sin = (torch.cos(a) * s["gain"]).float()[:, None], (torch.sin(a) * s["gain"]).float()[:, None]
    if c["inverse"]:
        sin = -sin
    x = x.float()
    if c["interleaved"]:
        u, w = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([u * cos - w * sin, w * cos + u * sin], -1).flatten(-2)
    else:
        u, w = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([u * cos - w * sin, w * cos + u * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _heads(s):
    c, qkv = s["c"], s["qkv"]
    heads = qkv.view(qkv.shape[0], -1, c["d"])
    return heads[:, :c["hq"]], heads[:, c["hq"]:c["hq"] + c["hkv"]], heads[:, c["hq"] + c["hkv"]:]


def _plain_rotate(s):
    q, k, _ = _heads(s)
    return dict(q=_turn(q, s).to(q.dtype), k=_turn(k, s).to(k.dtype))


def _plain_append(s):
    q, k, v = _heads(s)
    page = s["c"]["page"]
    block, at = s["slots"] // page, s["slots"] % page
    s["k_pool"][block, :, at] = _turn(k, s).to(k.dtype)
    s["v_pool"][block, :, at] = v
    return dict(q=_turn(q, s).to(q.dtype), k_pool=s["k_pool"], v_pool=s["v_pool"])


def _keys(pool, tables, width):
    """Rows of the cache's pages as [sequences, kv heads, width, d] in 32 bits."""
    page = pool.shape[2]
    t = pool[tables[:, :(width + page - 1) // page].long()]  # [n, pages, kv heads, page, d]
    return t.permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :width].float()


def _part(q, toks, seen, k, v, scale):
    """Softmax parts (maximum, sum, weighted values) of the tokens toks [n, w] over their sequence's keys; seen [n, w]
    keys each; returned by token, as [tokens, heads(, d)]."""
    n, w = toks.shape
    T, hq, d = q.shape
    hkv = k.shape[1]
    x = q[toks.clamp(min=0)].float().view(n, w, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).flatten(2, 3)
    a = (x @ k.transpose(-1, -2)).mul_(scale).view(n, hkv, w, hq // hkv, -1)
    hide = torch.arange(k.shape[2], device=DEV) >= seen[:, :, None]
    a.masked_fill_(hide[:, None, :, None], -math.inf)
    top = a.amax(-1)
    p = a.sub_(torch.where(top == -math.inf, 0.0, top)[..., None]).exp_()
    total = p.sum(-1)
    o = p.flatten(2, 3) @ v
    back = lambda z, tail: z.view((n, hkv, w, hq // hkv) + tail).transpose(1, 2).reshape((n, w, hq) + tail)  # noqa: E731
    live = toks >= 0
    at = toks[live]
    out = (torch.full((T, hq), -math.inf, device=DEV), torch.zeros(T, hq, device=DEV), torch.zeros(T, hq, d, device=DEV))
    out[0][at], out[1][at], out[2][at] = back(top, ())[live], back(total, ())[live], back(o, (d,))[live]
    return out


def _plain_attend(s):
    c, q, docs = s["c"], s["q"], s["c"]["docs"]
    scale = 1 / math.sqrt(c["d"])
    m, held = int(c["m_hi"]), int(c["own_hi"])
    m, held = min(m, s["tables"].shape[1] * c["page"]), min(held, s["tables"].shape[1] * c["page"])
    pre = _part(q, s["doc_tok"], s["doc_len"][:, None].expand_as(s["doc_tok"]), _keys(s["k_pool"], s["tables"][:docs], m),
                _keys(s["v_pool"], s["tables"][:docs], m), scale)
    j = torch.arange(s["req_tok"].shape[1], device=DEV)
    seen = (s["req_len"] - s["req_new"])[:, None] + j + 1
    mine = _part(q, s["req_tok"], torch.minimum(seen, s["req_len"][:, None]),
                 _keys(s["k_pool"], s["tables"][docs:], held), _keys(s["v_pool"], s["tables"][docs:], held), scale)
    top = torch.maximum(pre[0], mine[0])
    wa, wb = torch.exp(pre[0] - top), torch.exp(mine[0] - top)
    total = pre[1] * wa + mine[1] * wb
    o = (pre[2] * wa[..., None] + mine[2] * wb[..., None]) / total[..., None]
    return dict(out=o.to(q.dtype), lse=top + torch.log(total))


# ------------------------------------------------------------------ run
def run(state):
    s, c = state, state["c"]
    kind = c["kind"]
    if own:
        from paper_2609_03311_gb300 import dopr

        if kind == "extend":
            b = dopr.cache_extend(s["layout"], s["seq_lens"], s["tables"], s["free"], s["n_free"], s["new_lens"],
                                  s["max_tokens"], prefix=s["prefix"], out=s["out"])
            return dict(seq_lens=b.seq_lens, n_free=b.n_free, block_tables=s["tables"], free_blocks=s["free"],
                        tok_off=b.tok_off, slots=b.slots, positions=b.positions)
        if kind == "rotate":
            q, k, _ = _heads(s)
            dopr.rope_apply(s["rope"], s["positions"], q, k, q_out=s["q_out"], k_out=s["k_out"], inverse=c["inverse"])
            return dict(q=s["q_out"], k=s["k_out"])
        if kind == "append":
            q, k, v = _heads(s)
            dopr.cache_append(s["layout"], s["slots"], k, v, s["k_pool"], s["v_pool"], rope=s["rope"],
                              positions=s["positions"], q=q, q_out=s["q_out"])
            return dict(q=s["q_out"], k_pool=s["k_pool"], v_pool=s["v_pool"])
        dopr.shared_attention(s["layout"], s["plan"], s["q"], s["k_pool"], s["v_pool"], s["tables"], out=s["out"],
                              lse=s["lse"], workspace=s["workspace"])
        return dict(out=s["out"], lse=s["lse"])
    return {"extend": _plain_extend, "rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend}[kind](s)


# ------------------------------------------------------------------ work
def work(case):
    c = case
    if c["kind"] == "extend":
        new = (c["new_lo"] + c["new_hi"]) / 2 * (c["rows"] - c["prefixes"]) * (1 - c["release"])
        # lengths in and out, offsets; new tokens' slots and positions; new pages on the stack and in the tables
        return {"bytes": 20 * c["rows"] + 12 * new + 8 * new / c["page"], "flops": 0}
    if c["kind"] in ("rotate", "append"):
        size = 4 if c["dtype"] == "f32" else 2
        heads = c["hq"] + c["hkv"] * (1 if c["kind"] == "rotate" else 2)
        turned = (c["hq"] + c["hkv"]) * c["rotary"] / 2
        return {"bytes": c["tokens"] * (2 * heads * c["d"] * size + (4 if c["kind"] == "rotate" else 12)),
                "flops": 6.0 * c["tokens"] * turned}
    m, doc, held, new = _lengths(c)
    used = np.unique(doc)
    T = int(new.sum())
    seen = float((new * (m[doc] + held) - new * (new - 1) / 2).sum())
    kv = 2 * 2 * c["hkv"] * c["d"] * (int(m[used].sum()) + int(held.sum()))
    return {"bytes": 2 * 2 * T * c["hq"] * c["d"] + 4 * T * c["hq"] + kv, "flops": 4.0 * c["d"] * c["hq"] * seen}


# ------------------------------------------------------------------ from the definitions, in 64 bits
def _exact_extend(s):
    c, page = s["c"], s["c"]["page"]
    lens, new = s["seq_lens"].tolist(), s["new_lens"].tolist()
    prefix, tables = s["prefix"].tolist(), s["tables"].cpu().numpy().copy()
    free, top = s["free"].cpu().numpy().copy(), int(s["n_free"])
    for i, n in enumerate(new):
        if n < 0:
            for p in range(-(-lens[i] // page)):
                free[top] = tables[i, p]
                top += 1
            lens[i] = 0
    slots, where, off = [], [], [0]
    for i, n in enumerate(new):
        for j in range(max(n, 0)):
            if lens[i] % page == 0:
                top -= 1
                tables[i, lens[i] // page] = free[top]
            slots.append(int(tables[i, lens[i] // page]) * page + lens[i] % page)
            where.append((i, lens[i]))
            lens[i] += 1
        off.append(len(slots))
    pos = [p + (lens[prefix[i]] if prefix[i] >= 0 else 0) for i, p in where]
    rest = [-1] * (s["max_tokens"] - len(slots))
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)  # noqa: E731
    return dict(seq_lens=i32(lens), n_free=i32([top]), block_tables=i32(tables), free_blocks=i32(free), tok_off=i32(off),
                slots=torch.tensor(slots + rest, dtype=torch.int64, device=DEV), positions=i32(pos + rest))


def _exact_turn(x, s):
    c, r = s["c"], s["c"]["rotary"]
    f, gain = _frequencies(c)
    a = torch.outer(s["positions"].double(), torch.from_numpy(f).to(DEV))
    z = torch.polar(torch.full_like(a, gain), -a if c["inverse"] else a)[:, None]
    y = x.double().clone()
    pairs = (y[..., 0:r:2], y[..., 1:r:2]) if c["interleaved"] else (y[..., :r // 2], y[..., r // 2:r])
    w = torch.complex(pairs[0].contiguous(), pairs[1].contiguous()) * z
    pairs[0].copy_(w.real)
    pairs[1].copy_(w.imag)
    return y


def _exact_rows(s):
    c = s["c"]
    q, k, v = _heads(s)
    if c["kind"] == "rotate":
        return dict(q=_exact_turn(q, s), k=_exact_turn(k, s))
    kp, vp = s["k_pool"].double(), s["v_pool"].double()
    flat = lambda p: p.transpose(1, 2).reshape(-1, c["hkv"], c["d"])  # noqa: E731
    kf, vf = flat(kp), flat(vp)
    kf[s["slots"]], vf[s["slots"]] = _exact_turn(k, s), v.double()
    paged = lambda p: p.view(kp.shape[0], c["page"], c["hkv"], c["d"]).transpose(1, 2).contiguous()  # noqa: E731
    return dict(q=_exact_turn(q, s), k_pool=paged(kf), v_pool=paged(vf))


def _exact_attend(s):
    c = s["c"]
    m, doc, held, new = _lengths(c)
    docs, G, page = c["docs"], c["hq"] // c["hkv"], c["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    off = np.concatenate([[0], np.cumsum(new)])

    def rows(pool, row, n):
        t = s["tables"][row, :-(-n // page)].long()
        return torch.cat([pool[b].double() for b in t], 1)[:, :n]  # [kv heads, n, d]

    for k in np.unique(doc):
        kd, vd = rows(s["k_pool"], k, int(m[k])), rows(s["v_pool"], k, int(m[k]))
        for i in np.nonzero(doc == k)[0]:
            n, L = int(new[i]), int(held[i])
            keys = torch.cat([kd, rows(s["k_pool"], docs + i, L)], 1)
            vals = torch.cat([vd, rows(s["v_pool"], docs + i, L)], 1)
            at = torch.arange(keys.shape[1], device=DEV)
            last = int(m[k]) + L - n + torch.arange(n, device=DEV)
            for h in range(c["hq"]):
                a = s["q"][off[i]:off[i + 1], h].double() @ keys[h // G].T / math.sqrt(c["d"])
                a = a.masked_fill(at > last[:, None], -math.inf)
                out[off[i]:off[i + 1], h] = torch.softmax(a, -1) @ vals[h // G]
                lse[off[i]:off[i + 1], h] = torch.logsumexp(a, -1)
    return dict(out=out, lse=lse)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "extend":
        return _exact_extend(s)
    if case["kind"] == "attend":
        if case["reqs"] * case["hq"] > 10000:  # a loop over sequences and heads: too long
            return None
        return _exact_attend(s)
    return _exact_rows(s)
