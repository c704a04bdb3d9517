"""Head norms with rotary positions, and the paged cache in 4 bits, as a user of the library calls them, over the sizes they
come in.

Kinds of case (key "kind"):
  norm      dopr.head_norm_rope: RMSNorm of each query and key head with a gain, then rotary positions
  backward  dopr.head_norm_rope_backward: the gradients of that for q, k and both gains
  store     dopr.cache_append_4bit, then dopr.cache_read_4bit: a layer's new keys and values into the pages, then what the
            pool's pages stand for, in the rows' type
  attend    dopr.shared_attention_4bit: sequences that share stored prefixes attend to them, then causally to their own keys

Head counts are those of the Qwen3 shapes the repository is configured for (32 / 8 and 16 / 8 heads of 128), and generic ones
in drawn cases.  Lengths and shapes of attend cases go by the case, everything else by the seed.

The 4-bit pages: 32 elements of a head that follow one another share a scale s, the smallest of the scales there are that is
at least max |x| / 7; each is held as c + 8, c = x / s to the nearest whole number, ties away from zero.  A scale is a byte,
five bits of exponent above three of mantissa: the upper bits of the fp16 number; 0xe1 (9216) is the largest.  A page of a kv
head holds its rows' codes, then their scales.  Of 8 codes in a word element 2 i is at bits 4 i, element 2 i + 1 at 16 + 4 i.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"
EPS = 1e-6
GROUP = 32


# ------------------------------------------------------------------ cases
def _rows(name, kind, tokens, hq, hkv, d, dtype, **more):
    return dict(name=name, kind=kind, tokens=tokens, hq=hq, hkv=hkv, d=d, dtype=dtype, gain=more.get("gain", "bf16"),
                rotary=more.get("rotary", d), interleaved=more.get("interleaved", False), scaling=more.get("scaling", "plain"),
                factor=more.get("factor", 1.0), far=more.get("far", 8192))


def _store(name, tokens, hkv, d, dtype, page, spread):
    return dict(name=name, kind="store", tokens=tokens, hkv=hkv, d=d, dtype=dtype, page=page, spread=spread)


def _attend(name, hq, hkv, d, dtype, page, docs, m_lo, m_hi, reqs, own_lo, own_hi, new_lo, new_hi, lens=1):
    return dict(name=name, kind="attend", hq=hq, hkv=hkv, d=d, dtype=dtype, page=page, docs=docs, m_lo=m_lo, m_hi=m_hi,
                reqs=reqs, own_lo=own_lo, own_hi=own_hi, new_lo=new_lo, new_hi=new_hi, lens=lens)


def listed():
    return [
        # one new token's heads
        _rows("norm one token", "norm", 1, 32, 8, 128, "bf16"),
        # a whole scoring chunk's heads
        _rows("norm a chunk", "norm", 26800, 32, 8, 128, "bf16"),
        # a step that trains on a few documents, in 32 bits: interleaved positions on half of each head, far ones
        _rows("gradient of 1021 rows, interleaved", "backward", 1021, 16, 8, 128, "f32", gain="f32", rotary=64,
              interleaved=True, scaling="ramp", factor=8.0, far=250000),
        # a training batch
        _rows("gradient of 8192 rows", "backward", 8192, 32, 8, 128, "bf16", gain="f32"),
        # a step of 64 running sequences: a row each into the page that each has begun
        _store("store 64 rows", 64, 8, 128, "bf16", 16, 64),
        # stored documents' rows, a whole chunk of them, in full pages
        _store("store a chunk", 26800, 8, 128, "f16", 64, 0),
        # one query's next token on a short document
        _attend("attend one token", 32, 8, 128, "bf16", 64, 1, 512, 512, 1, 24, 24, 1, 1),
        # 64 conversations' next tokens, no two of which share anything
        _attend("attend 64 conversations", 32, 8, 128, "bf16", 64, 0, 0, 0, 64, 2000, 6000, 1, 1, lens=2),
        # 64 queries' next tokens on one long document
        _attend("attend 64 queries, one long document", 32, 8, 128, "bf16", 64, 1, 32768, 32768, 64, 8, 64, 1, 1),
        # next tokens over many documents, ragged, small pages, arrival order
        _attend("attend ragged documents", 16, 8, 128, "f16", 16, 64, 1, 1024, 256, 1, 256, 1, 1, lens=3),
        # queries scored over whole documents: every query token is new
        _attend("attend queries of 16 documents", 32, 8, 128, "f16", 32, 16, 256, 2048, 200, 8, 64, 8, 64, lens=5),
        # long queries over one long document: the largest call
        _attend("attend 2048 rows, one long document", 32, 8, 128, "bf16", 128, 1, 16384, 16384, 32, 64, 64, 64, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "backward", "store", "attend", "attend"])
    hkv = rng.choice([1, 2, 4, 8, 8])
    hq = hkv * rng.choice([1, 2, 4, 4, 5, 8])
    d = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    half = rng.choice(["f16", "bf16"])
    if kind == "store":
        tokens = _log(rng, 1, 26800)
        c = _store("", tokens, hkv, d, half, page, rng.choice([0, tokens]) if tokens <= 512 else 0)
    elif kind in ("norm", "backward"):
        d = rng.choice([64, 80, 96, 128, 128, 128, 256])
        most = (26800 if kind == "norm" else 8192) * 40 * 128 // ((hq + hkv) * d)
        scaling = rng.choice(["plain", "linear", "ntk", "bands", "ramp"])
        dtype = rng.choice(["f16", "bf16", "f32"])
        c = _rows("", kind, min(_log(rng, 1, 26800), most // 2 if dtype == "f32" else most), hq, hkv, d, dtype,
                  gain=rng.choice(["bf16", "f32", dtype]), rotary=rng.choice([d, d, d // 2]),
                  interleaved=rng.choice([False, True]), scaling=scaling,
                  factor=1.0 if scaling == "plain" else rng.choice([2.0, 4.0, 8.5]), far=_log(rng, 2000, 300000))
    else:
        m = _log(rng, 16, 32768)
        docs = rng.choice([0, 1, 1, max(1, min(64, 16384 // m))])
        reqs = max(docs, _log(rng, 1, 256))
        new = rng.choice([1, 1, 1, min(64, max(1, 2048 // reqs))])
        own_hi = max(new, _log(rng, 1, 256) if docs else min(m, 65536 // reqs))
        if docs and reqs * new * m > 2048 * 16384:
            reqs = max(1, 2048 * 16384 // (new * m))
        c = _attend("", hq, hkv, d, half, page, docs, max(1, m // rng.choice([1, 4])) if docs else 0, m if docs else 0, reqs,
                    min(own_hi, max(1, new // 2)), own_hi, max(1, new // 2), new, lens=rng.randrange(1, 1000))
    del c["name"]
    return c


# ------------------------------------------------------------------ rotary frequencies, in 64 bits
def _rope_more(c):
    """Ranges of the scaled forms: the length the plain positions were made for and the two ends of the blend."""
    return dict(original=4096, low=1.0, high=4.0) if c["scaling"] == "bands" else dict(original=4096, low=1.0, high=32.0)


def _frequencies(c):
    """(radians a position of each pair, factor on cos and sin)."""
    d, theta, s, more = c["rotary"], 1e6, c["factor"], _rope_more(c)
    i = np.arange(d // 2, dtype=np.float64)
    if c["scaling"] == "ntk":
        theta *= s ** (d / (d - 2.0))
    f = theta ** (-2.0 * i / d)
    if c["scaling"] == "linear":
        f = f / s
    elif c["scaling"] == "bands":
        t = np.clip((more["original"] * f / (2 * math.pi) - more["low"]) / (more["high"] - more["low"]), 0, 1)
        f = (1 - t) * f / s + t * f
    elif c["scaling"] == "ramp":
        at = lambda turns: d * math.log(more["original"] / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
        lo, hi = max(math.floor(at(more["high"])), 0), min(math.ceil(at(more["low"])), d - 1)
        t = np.clip((i - lo) / max(hi - lo, 1e-3), 0, 1)
        return f / s * t + f * (1 - t), 0.1 * math.log(s) + 1.0
    return f, 1.0


# ------------------------------------------------------------------ the 4-bit pages
def _codes(x):
    """c and s [..., groups, 32] / [..., groups, 1] of x [..., d], in 32 bits: every step but the two divisions is exact, and
    neither of those rounds to or across a border (a division by a plain number would be a product with its inverse)."""
    g = x.float().unflatten(-1, (-1, GROUP))
    most = g.abs().amax(-1, keepdim=True)
    want = most / torch.full_like(most, 7)
    step = (((torch.frexp(want)[1] - 4).clamp(min=-17) + 127) << 23).view(torch.float32)  # a power of two
    s = (torch.ceil(want / step) * step).clamp(max=9216.0)
    c = torch.where(s > 0, torch.sign(g) * torch.floor(g.abs() / s + 0.5), 0.0)
    return c, s


def _held(x):
    """What the pages hold of x, in 32 bits."""
    c, s = _codes(x)
    return (c * s).flatten(-2)


def _pack(x):
    """Pages [blocks, kv heads, page, d] as bytes [blocks, kv heads, page * (d / 2 + d / 32)]."""
    c, s = _codes(x)
    n = (c + 8).to(torch.uint8).flatten(-2).unflatten(-1, (-1, 2, 2, 2))  # word, pair of i, i of the pair, parity
    n = n.permute(*range(n.dim() - 3), -1, -3, -2)
    codes = n[..., 0] | (n[..., 1] << 4)  # word, parity, pair of i: four bytes
    scales = (s.squeeze(-1).half().view(torch.int16) >> 7).to(torch.uint8)
    return torch.cat([codes.flatten(2), scales.flatten(2)], -1)


def _unpack(b, page, d):
    """Bytes [..., page * (d / 2 + d / 32)] as the values [..., page, d] they stand for, in 32 bits."""
    codes, scales = b[..., :page * (d // 2)], b[..., page * (d // 2):]
    n = torch.stack([codes & 15, codes >> 4], -1).unflatten(-2, (page, d // 8, 2, 2))  # row, word, parity, pair of i, i
    n = n.flatten(-2).transpose(-1, -2).flatten(-3).float() - 8
    s = (scales.to(torch.int16) << 7).view(torch.float16).float().unflatten(-1, (page, d // GROUP))
    return (n.unflatten(-1, (-1, GROUP)) * s[..., None]).flatten(-2)


# ------------------------------------------------------------------ prepare
def _gen(seed, more=0):
    g = torch.Generator(DEV)
    g.manual_seed(seed * 1000003 + more)
    return g


def _prepare_norm(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    T, hq, hkv, d = c["tokens"], c["hq"], c["hkv"], c["d"]
    rand = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    # the packed q | k | v rows that a projection leaves, gains near one as trained ones are
    s = dict(c=c, qkv=rand(T, (hq + 2 * hkv) * d).to(dt),
             positions=torch.randint(0, c["far"], (T,), generator=g, device=DEV, dtype=torch.int32))
    s["q_gain"], s["k_gain"] = ((1 + 0.2 * rand(d)).to(DTYPES[c["gain"]]) for _ in range(2))
    f, s["factor"] = _frequencies(c)
    s["freq"] = torch.from_numpy(f).to(DEV)
    if c["kind"] == "backward":
        s["dq_out"], s["dk_out"] = rand(T, hq, d).to(dt), rand(T, hkv, d).to(dt)
    if own:
        from paper_2609_03311_gb300 import dopr

        more = _rope_more(c)
        s["rope"] = dopr.Rope(c["far"], c["rotary"], theta=1e6,
                              layout=dopr.ROPE_INTERLEAVED if c["interleaved"] else dopr.ROPE_HALF,
                              scaling=getattr(dopr, "ROPE_" + c["scaling"].upper()), factor=c["factor"],
                              original_max_position=more["original"], low=more["low"], high=more["high"])
        s["q_new"], s["k_new"] = torch.empty(T, hq, d, device=DEV, dtype=dt), torch.empty(T, hkv, d, device=DEV, dtype=dt)
        if c["kind"] == "backward":
            s["workspace"] = dopr.head_norm_rope_workspace(d, DEV)
    return s


def _prepare_store(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    T, hkv, d, page = c["tokens"], c["hkv"], c["d"], c["page"]
    blocks = c["spread"] or -(-T // page) + 3
    rand = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    s = dict(c=c, k=rand(T, hkv, d).to(dt), v=rand(T, hkv, d).to(dt), blocks=blocks,
             k_pool=_pack(rand(blocks, hkv, page, d)), v_pool=_pack(rand(blocks, hkv, page, d)))
    if c["spread"]:  # a row in each sequence's last page
        s["slots"] = torch.randperm(blocks, generator=g, device=DEV)[:T] * page
        s["slots"] += torch.randint(0, page, (T,), generator=g, device=DEV)
    else:  # rows of documents: page after page, the pages anywhere
        at = torch.arange(T, device=DEV)
        s["slots"] = torch.randperm(blocks, generator=g, device=DEV)[at // page] * page + at % page
    s["all"] = torch.arange(blocks * page, device=DEV)
    if own:
        from paper_2609_03311_gb300 import dopr

        s["layout"] = dopr.make_cache_layout(blocks, page, hkv, d, dt, 1, blocks)
        s["k_held"], s["v_held"] = (torch.empty(blocks * page, hkv, d, device=DEV, dtype=dt) for _ in range(2))
    return s


def _lengths(c):
    """Documents' lengths, requests' documents (arrival order; -1: none), own lengths and new tokens: fixed by the case."""
    r = np.random.default_rng(c["lens"])
    m = r.integers(c["m_lo"], c["m_hi"] + 1, c["docs"])
    doc = r.integers(0, c["docs"], c["reqs"]) if c["docs"] else np.full(c["reqs"], -1)
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
    rows, pages = docs + reqs, -(-lens // page)
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
    rand = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    # elements of a key differ in size, as they do behind norms with gains
    size = torch.exp(0.3 * rand(c["hkv"], 1, c["d"]))
    s = dict(c=c, q=rand(T, c["hq"], c["d"]).to(dt), k_pool=_pack(rand(blocks, c["hkv"], page, c["d"]) * size),
             v_pool=_pack(rand(blocks, c["hkv"], page, c["d"])), tables=dev(tables), seq_lens=dev(lens.astype(np.int32)),
             tok_off=dev(off.astype(np.int32)), prefix=dev(np.concatenate([np.full(docs, -1), doc]).astype(np.int32)))
    # the plain form's plan: each document's and each request's tokens, padded with -1
    toks = [np.arange(off[docs + i], off[docs + i + 1]) for i in range(reqs)]
    if docs:
        by_doc = [np.concatenate([toks[i] for i in np.nonzero(doc == k)[0]] + [np.zeros(0, dtype=np.int64)])
                  for k in range(docs)]
        s["doc_tok"] = dev(_padded(by_doc, max(len(v) for v in by_doc)))
    s["req_tok"] = dev(_padded(toks, int(new.max())))
    s["doc_len"], s["req_len"], s["req_new"] = dev(m), dev(held), dev(new)
    s["most_doc"], s["most_req"] = int(m.max()) if docs else 0, int(held.max())
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
    return (_prepare_store if kind == "store" else _prepare_attend if kind == "attend" else _prepare_norm)(case, seed)


# ------------------------------------------------------------------ the plain forms
def _heads(s):
    c, qkv = s["c"], s["qkv"]
    heads = qkv.view(qkv.shape[0], -1, c["d"])
    return heads[:, :c["hq"]], heads[:, c["hq"]:c["hq"] + c["hkv"]]


def _turn(x, s, back):
    """Rotary positions on x [tokens, heads, d] in 32 bits; angles in 64."""
    c, r = s["c"], s["c"]["rotary"]
    a = s["positions"].double()[:, None] * s["freq"]
    cos, sin = (torch.cos(a) * s["factor"]).float()[:, None], (torch.sin(a) * s["factor"]).float()[:, None]
    if back:
        sin = -sin
    if c["interleaved"]:
        u, w = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([u * cos - w * sin, w * cos + u * sin], -1).flatten(-2)
    else:
        u, w = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([u * cos - w * sin, w * cos + u * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_norm(s):
    def one(x, gain):
        x = x.float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
        return _turn(y, s, False)

    q, k = _heads(s)
    return dict(q=one(q, s["q_gain"]).to(q.dtype), k=one(k, s["k_gain"]).to(k.dtype))


def _plain_backward(s):
    def one(x, gain, dz):
        dt, x = x.dtype, x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        dy = _turn(dz.float(), s, True)
        n = x * r
        w = dy * gain.float()
        dx = r * (w - n * (w * n).mean(-1, keepdim=True))
        return dx.to(dt), (dy * n).sum((0, 1), dtype=torch.float64).float()

    q, k = _heads(s)
    dq, dq_gain = one(q, s["q_gain"], s["dq_out"])
    dk, dk_gain = one(k, s["k_gain"], s["dk_out"])
    return dict(dq=dq, dk=dk, dq_gain=dq_gain, dk_gain=dk_gain)


def _plain_store(s):
    c, out = s["c"], {}
    page, d = c["page"], c["d"]
    block, at = s["slots"] // page, s["slots"] % page
    held = _unpack(s["k_pool"], page, d), _unpack(s["v_pool"], page, d)
    held[0][block, :, at] = _held(s["k"])
    held[1][block, :, at] = _held(s["v"])
    out["k"], out["v"] = (x.transpose(1, 2).flatten(0, 1).to(s["k"].dtype) for x in held)
    return out


def _keys(pool, tables, width, page, d):
    """Rows of the cache's pages as [sequences, kv heads, width, d] in 32 bits."""
    t = _unpack(pool[tables[:, :(width + page - 1) // page].long()], page, d)  # [n, pages, kv heads, page, d]
    return t.permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :width]


def _part(q, toks, seen, k, v, scale):
    """Softmax parts (maximum, sum, weighted values) of the tokens toks [n, w] over their sequence's keys; seen [n, w] keys
    each; returned by token, as [tokens, heads(, d)]."""
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
    page, d, scale = c["page"], c["d"], 1 / math.sqrt(c["d"])
    keys = lambda pool, tables, width: _keys(s[pool], tables, width, page, d)  # noqa: E731
    j = torch.arange(s["req_tok"].shape[1], device=DEV)
    seen = (s["req_len"] - s["req_new"])[:, None] + j + 1
    top, total, o = _part(q, s["req_tok"], torch.minimum(seen, s["req_len"][:, None]),
                          keys("k_pool", s["tables"][docs:], s["most_req"]), keys("v_pool", s["tables"][docs:], s["most_req"]),
                          scale)
    if docs:
        pre = _part(q, s["doc_tok"], s["doc_len"][:, None].expand_as(s["doc_tok"]),
                    keys("k_pool", s["tables"][:docs], s["most_doc"]), keys("v_pool", s["tables"][:docs], s["most_doc"]), scale)
        both = torch.maximum(pre[0], top)
        wa, wb = torch.exp(pre[0] - both), torch.exp(top - both)
        top, total, o = both, pre[1] * wa + total * wb, pre[2] * wa[..., None] + o * wb[..., None]
    return dict(out=(o / total[..., None]).to(q.dtype), lse=top + torch.log(total))


# ------------------------------------------------------------------ run
def run(state):
    s, c = state, state["c"]
    kind = c["kind"]
    if own:
        from paper_2609_03311_gb300 import dopr

        if kind == "norm":
            q, k = _heads(s)
            dopr.head_norm_rope(q, k, q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS, rope=s["rope"],
                                positions=s["positions"], q_out=s["q_new"], k_out=s["k_new"])
            return dict(q=s["q_new"], k=s["k_new"])
        if kind == "backward":
            q, k = _heads(s)
            dq, dk, dq_gain, dk_gain = dopr.head_norm_rope_backward(
                s["dq_out"], q, s["dk_out"], k, q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS, rope=s["rope"],
                positions=s["positions"], dq=s["q_new"], dk=s["k_new"], workspace=s["workspace"])
            return dict(dq=dq, dk=dk, dq_gain=dq_gain, dk_gain=dk_gain)
        if kind == "store":
            dopr.cache_append_4bit(s["layout"], s["slots"], s["k"], s["v"], s["k_pool"], s["v_pool"])
            dopr.cache_read_4bit(s["layout"], s["all"], s["k_pool"], s["v_pool"], k_out=s["k_held"], v_out=s["v_held"])
            return dict(k=s["k_held"], v=s["v_held"])
        dopr.shared_attention_4bit(s["layout"], s["plan"], s["q"], s["k_pool"], s["v_pool"], s["tables"], out=s["out"],
                                   lse=s["lse"], workspace=s["workspace"])
        return dict(out=s["out"], lse=s["lse"])
    return {"norm": _plain_norm, "backward": _plain_backward, "store": _plain_store, "attend": _plain_attend}[kind](s)


# ------------------------------------------------------------------ work
def work(case):
    c = case
    d, hkv = c["d"], c["hkv"]
    size = 4 if c["dtype"] == "f32" else 2
    row = hkv * (d // 2 + d // GROUP)  # bytes of a token's keys, or values, in the pages
    if c["kind"] in ("norm", "backward"):
        elements = c["tokens"] * (c["hq"] + hkv) * d
        backward = c["kind"] == "backward"
        gains = 2 * d * (4 if c["gain"] == "f32" else 2) + (8 * d if backward else 0)
        return {"bytes": elements * size * (3 if backward else 2) + 4 * c["tokens"] + gains,
                "flops": elements * (12.0 if backward else 6.0)}
    if c["kind"] == "store":
        slots = (c["spread"] or -(-c["tokens"] // c["page"]) + 3) * c["page"]
        written = c["tokens"] * (2 * hkv * d * size + 2 * row + 8)
        return {"bytes": written + slots * (2 * hkv * d * size + 2 * row + 8), "flops": 4.0 * c["tokens"] * hkv * d}
    m, doc, held, new = _lengths(c)
    used = np.unique(doc) if c["docs"] else np.zeros(0, dtype=np.int64)
    before = m[doc] if c["docs"] else 0
    T = int(new.sum())
    seen = float((new * (before + held) - new * (new - 1) / 2).sum())
    return {"bytes": 2 * 2 * T * c["hq"] * d + 4 * T * c["hq"] + 2 * row * (int(m[used].sum()) + int(held.sum())),
            "flops": 4.0 * d * c["hq"] * seen}


# ------------------------------------------------------------------ from the definitions, in 64 bits
def _exact_turn(y, s, back):
    c, r = s["c"], s["c"]["rotary"]
    f, factor = _frequencies(c)
    a = torch.outer(s["positions"].double(), torch.from_numpy(f).to(DEV))
    z = torch.polar(torch.full_like(a, factor), -a if back else a)[:, None]
    y = y.clone()
    pairs = (y[..., 0:r:2], y[..., 1:r:2]) if c["interleaved"] else (y[..., :r // 2], y[..., r // 2:r])
    w = torch.complex(pairs[0].contiguous(), pairs[1].contiguous()) * z
    pairs[0].copy_(w.real)
    pairs[1].copy_(w.imag)
    return y


def _exact_norm(s):
    def unit(x):
        return x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / x.shape[-1] + EPS)

    out = {}
    for name, x in zip("qk", _heads(s)):
        x, gain = x.double(), s[name + "_gain"].double()
        if s["c"]["kind"] == "norm":
            out[name] = _exact_turn(unit(x) * gain, s, False)
            continue
        # the turn's transpose, then the norm's: with n = x / rms, d n / d x = (1 - n n^T / d) / rms
        dy = _exact_turn(s[f"d{name}_out"].double(), s, True)
        n = unit(x)
        rms = torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
        w = dy * gain
        out["d" + name] = (w - n * torch.einsum("thd,thd->th", w, n)[..., None] / x.shape[-1]) / rms
        out[f"d{name}_gain"] = torch.einsum("thd,thd->d", dy, n)
    return {k: out[k] for k in (("q", "k") if s["c"]["kind"] == "norm" else ("dq", "dk", "dq_gain", "dk_gain"))}


def _exact_scales():
    """The number that each scale byte stands for."""
    return torch.tensor([math.ldexp(8 + i % 8, i // 8 - 18) if i >= 8 else math.ldexp(i, -17) for i in range(0xe2)],
                        dtype=torch.float64, device=DEV)


def _exact_values(b, page, d):
    """Pages' bytes as values [..., page, d]: byte by byte, element by element of a word."""
    table = _exact_scales()
    codes = b[..., :page * d // 2].unflatten(-1, (page, d // 8, 4))
    x = torch.empty(codes.shape[:-1] + (8,), dtype=torch.float64, device=DEV)
    for i in range(8):
        bit = 4 * (i // 2) + 16 * (i % 2)
        x[..., i] = ((codes[..., bit // 8] >> (bit % 8)) & 15).double() - 8
    s = table[b[..., page * d // 2:].long()].unflatten(-1, (page, d // 32))
    return x.flatten(-2) * s.repeat_interleave(32, -1)


def _exact_held(x):
    """The nearest that the format has: the smallest scale s with 7 s >= max |x|, found in the list of all scales."""
    scales = _exact_scales()
    g = x.double().unflatten(-1, (-1, 32))
    s = scales[torch.searchsorted(7 * scales, g.abs().amax(-1)).clamp(max=0xe1)][..., None]
    a = g.abs() / torch.where(s > 0, s, 1.0)
    return (torch.sign(g) * torch.floor(a + 0.5) * s).flatten(-2)


def _exact_store(s):
    c = s["c"]
    out = {}
    for name in "kv":
        pool = _exact_values(s[name + "_pool"], c["page"], c["d"]).transpose(1, 2).reshape(-1, c["hkv"], c["d"])
        pool[s["slots"]] = _exact_held(s[name])
        out[name] = pool
    return out


def _exact_attend(s):
    c = s["c"]
    m, doc, held, new = _lengths(c)
    docs, G, page, d = c["docs"], c["hq"] // c["hkv"], c["page"], c["d"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    off = np.concatenate([[0], np.cumsum(new)])

    def rows(pool, row, n):
        t = _exact_values(s[pool][s["tables"][row, :-(-n // page)].long()], page, d)  # [pages, kv heads, page, d]
        return t.transpose(0, 1).flatten(1, 2)[:, :n]

    for k in np.unique(doc):
        pre = [rows(p, k, int(m[k])) for p in ("k_pool", "v_pool")] if docs else None
        for i in np.nonzero(doc == k)[0]:
            n, L = int(new[i]), int(held[i])
            keys, vals = rows("k_pool", docs + i, L), rows("v_pool", docs + i, L)
            if docs:
                keys, vals = torch.cat([pre[0], keys], 1), torch.cat([pre[1], vals], 1)
            last = keys.shape[1] - n + torch.arange(n, device=DEV)
            hide = torch.arange(keys.shape[1], device=DEV) > last[:, None]
            for h in range(c["hq"]):
                a = s["q"][off[i]:off[i + 1], h].double() @ keys[h // G].T / math.sqrt(d)
                a = a.masked_fill(hide, -math.inf)
                out[off[i]:off[i + 1], h] = torch.softmax(a, -1) @ vals[h // G]
                lse[off[i]:off[i + 1], h] = torch.logsumexp(a, -1)
    return dict(out=out, lse=lse)


def exact(case, seed):
    if case["kind"] == "attend" and case["reqs"] * case["hq"] > 10000:  # a loop over sequences and heads: too long
        return None
    s = prepare(case, seed)
    if case["kind"] == "attend":
        return _exact_attend(s)
    return _exact_store(s) if case["kind"] == "store" else _exact_norm(s)
