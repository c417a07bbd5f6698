"""A step that takes several tokens of a sequence, as a serving program uses it: its operators as measurable cases.

  rotate     ``rotate_store``: queries and keys of new tokens normed head by head and turned by their positions, keys and values into
             their pages
  attend     ``dense_attend`` over every page, ``sparse_attend`` over lists of pages: every new token is a query of its own; scores with a
             cap, a bias by distance, a window, a prefix, documents
  verify     ``verify``: drafted tokens against the target's probabilities, then ``trim_pages``: the pages of refused ones

Projections N(0, I); keys of the cache a topic + N(0, I), queries a topic + N(0, I); logits 3 N(0, I), the draft's a noisy copy.
Pages lie in the pools in random order."""
import math
import random

import torch

own = False

HEAD_DIM = 128
SINK, WINDOW = 1, 4                 # pages a list always has: the first, the last
EPS = 1e-6
VOCAB = 151936                      # probabilities a row, as in the benchmark of the monitor
HEADS = (((8, 8), 16), ((32, 8), 16), ((32, 8), 32), ((28, 4), 16), ((28, 4), 32))


def _case(name, kind, **more):
    c = {"name": name, "kind": kind, "batch": 1, "lo": 0, "hi": 0, "new_lo": 1, "new_hi": 1, "n_q_heads": 32, "n_kv_heads": 8, "page_size": 16}
    c.update({"rotate": {"axes": 1, "turned": HEAD_DIM, "beside": False, "norms": True},
              "attend": {"listed": 0, "cap": 0.0, "slopes": False, "window": 0, "prefix": 0, "document": 0},
              "verify": {"vocab": VOCAB, "given": True}}[kind])
    c.update(more)
    return c


def listed():
    return [
        # one conversation takes its next token: latency only
        _case("rotate_b1_token", "rotate", lo=4096, hi=4096),
        # a serving batch with four drafted tokens a sequence
        _case("rotate_b32_drafts", "rotate", batch=32, lo=1, hi=32768, new_lo=5, new_hi=5),
        # a chunk of prompts with images among them (time, height, width), of odd lengths, behind what their rows hold already
        _case("rotate_b12_prompts", "rotate", batch=12, lo=0, hi=4099, new_lo=131, new_hi=4099, axes=3),
        # one long prompt, pages of 32, seven query heads to a KV head, half of a head turned, no norms
        _case("rotate_b1_64k_page32", "rotate", new_lo=65531, new_hi=65531, n_q_heads=28, n_kv_heads=4, page_size=32, turned=64, beside=True, norms=False),
        # four drafted tokens of one short conversation over its list of pages
        _case("attend_b1_drafts_listed", "attend", lo=4096, hi=4096, new_lo=5, new_hi=5, n_q_heads=8, listed=21),
        # a serving batch with drafted tokens over its lists
        _case("attend_b32_drafts_listed", "attend", batch=32, lo=16384, hi=32768, new_lo=2, new_hi=8, listed=108),
        # drafted tokens over every page of ragged contexts, capped scores
        _case("attend_b16_drafts_every", "attend", batch=16, lo=8200, hi=65531, new_lo=5, new_hi=5, cap=30.0),
        # a chunk of a long prompt
        _case("attend_b1_chunk", "attend", lo=31237, hi=31237, new_lo=1531, new_hi=1531),
        # whole prompts packed of documents, a bias by distance
        _case("attend_b12_prompts", "attend", batch=12, new_lo=131, new_hi=2051, slopes=True, document=1203),
        # one sequence's four drafted tokens
        _case("verify_b1", "verify", lo=4096, hi=4096, new_lo=5, new_hi=5),
        # a serving batch, as many drafts as each row's drafter had
        _case("verify_b32", "verify", batch=32, lo=1, hi=32768, new_lo=1, new_hi=8),
        # a large batch
        _case("verify_b128", "verify", batch=128, lo=1, hi=16384, new_lo=4, new_hi=4),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("rotate", "rotate", "attend", "attend", "attend", "attend", "verify", "verify"))
    (hq, h), page = rng.choice(HEADS)
    c = {"kind": kind, "n_q_heads": hq, "n_kv_heads": h, "page_size": page}
    if kind == "rotate":
        new = spread(1, 65536)
        c.update(batch=max(1, min(spread(1, 256), (1 << 16) // new)), lo=0, hi=spread(1, 8192), new_lo=max(1, new // 3), new_hi=new, axes=rng.choice((1, 1, 2, 3)),
                 turned=rng.choice((128, 128, 64, 96)), beside=rng.random() < 0.3, norms=rng.random() < 0.7)
    elif kind == "verify":
        new = spread(1, 16)
        c.update(batch=max(1, min(spread(1, 256), 640 // new)), lo=1, hi=spread(1, 16384), new_lo=rng.choice((1, new)), new_hi=new, vocab=spread(32000, VOCAB),
                 given=rng.random() < 0.7)
    else:
        new = rng.choice((spread(1, 16), spread(1, 16), spread(16, 256), spread(256, 2048)))
        hi = spread(16, 131072)
        # no more scores, and no more keys, than the largest listed cases have
        batch = max(1, min(spread(1, 48), (1 << 20) // (hi + new), (1 << 25) // (new * (hi + new))))
        hi = max(1, min(hi, (1 << 25) * 3 // (2 * new) - new))
        c.update(batch=batch, lo=spread(max(1, hi // 8), hi) - (1 if rng.random() < 0.5 else 0), hi=hi, new_lo=rng.choice((new, max(1, new // 4))), new_hi=new,
                 listed=0, cap=rng.choice((0.0, 0.0, 20.0, 50.0)), slopes=rng.random() < 0.25, window=0, prefix=0, document=0)
        what = rng.choice(("", "", "window", "prefix", "document"))
        if what:
            c[what] = spread(3, 4096)
        pages = -(-(hi + new) // page)
        if new <= 16:
            c.update(listed=rng.choice((0, min(pages, spread(8, 600)))))
    return c


# ---- sizes that follow from a case
def _between(r, lo, hi, n):
    """n whole numbers between lo and hi, both among them."""
    got = [hi] + [lo + r.randrange(hi - lo + 1) for _ in range(n - 1)]
    if n > 1:
        got[-1] = lo
    return got


def _rows(case):
    """(tokens a sequence holds, tokens it takes) of every sequence."""
    r = random.Random(case["batch"] * 7 + case["hi"] * 3 + case["new_hi"])
    return _between(r, case["lo"], case["hi"], case["batch"]), _between(r, case["new_lo"], case["new_hi"], case["batch"])


def _interval(case, held, new):
    """First and last key that each new token of a sequence sees, as lists."""
    lo, hi = [], []
    for p in range(held, held + new):
        first = p // case["document"] * case["document"] if case["document"] else 0
        lo.append(max(first, p - case["window"] + 1 if case["window"] else 0))
        hi.append(min(held + new - 1, max(p, case["prefix"] - 1)))
    return lo, hi


# ---- inputs
def _table(pages, width, order, dev):
    """Block table of rows that hold so many pages, dealt out of `order`; behind them -1."""
    pages = torch.tensor(pages, device=dev)
    table = torch.full((len(pages), width), -1, dtype=torch.int32, device=dev)
    there = torch.arange(width, device=dev)[None, :] < pages[:, None]
    table[there] = order[: int(pages.sum())].to(torch.int32)
    return table


def _ints(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _starts(new):
    at = [0]
    for n in new:
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    kind, B, H, Hq, d, batch = case["kind"], case["page_size"], case["n_kv_heads"], case["n_q_heads"], HEAD_DIM, case["batch"]
    held, new = _rows(case)
    width = max(-(-(h + n) // B) for h, n in zip(held, new)) + 1
    tokens = sum(new)
    s = {"case": dict(case), "width": width, "tokens": tokens, "lens": _ints([h + n for h, n in zip(held, new)], dev), "starts": _ints(_starts(new), dev)}
    if own:
        import paper_2602_20732_amd as pk
        s["lib"] = pk.Chess(pk.Config(Hq, H, B, batch, width, min(case.get("listed", 0) or width, width)))
        s["ws"] = s["lib"].new_workspace(dev)
    n_phys = sum(-(-(h + n) // B) for h, n in zip(held, new)) + 1
    order = torch.randperm(n_phys, generator=g, device=dev)
    s["table"] = _table([-(-(h + n) // B) for h, n in zip(held, new)], width, order, dev)
    return {"rotate": _prepare_rotate, "attend": _prepare_attend, "verify": _prepare_verify}[kind](s, g, held, new, n_phys)


def _prepare_rotate(s, g, held, new, n_phys):
    c, dev, tokens = s["case"], s["table"].device, s["tokens"]
    B, H, Hq, d = c["page_size"], c["n_kv_heads"], c["n_q_heads"], HEAD_DIM
    # the projection's output: queries, keys and values of a token side by side
    s["rows"] = torch.empty((tokens, Hq + 2 * H, d), dtype=torch.bfloat16, device=dev).normal_(generator=g)
    s["q"], s["k_new"], s["v_new"] = s["rows"][:, :Hq], s["rows"][:, Hq:Hq + H], s["rows"][:, Hq + H:]
    s["k"] = torch.empty((n_phys, H, B, d), dtype=torch.bfloat16, device=dev).normal_(generator=g)
    s["v"] = torch.empty((n_phys, H, d, B), dtype=torch.bfloat16, device=dev).normal_(generator=g)
    s["q_out"] = torch.zeros((tokens, Hq, d), dtype=torch.bfloat16, device=dev)
    place = torch.cat([torch.arange(h, h + n) for h, n in zip(held, new)])
    row = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new))
    s["slots"] = (s["table"].cpu().long()[row, place // B] * B + place % B).to(dev)
    # where a token stands: text moves every axis alike, a patch of an image by its row and column
    place = place.to(dev)
    patch = (place // 256) % 2 == 1
    axes = [place, torch.where(patch, place - place % 256 + place % 256 // 16, place), torch.where(patch, place - place % 256 + place % 16, place)]
    s["positions"] = torch.stack(axes[: c["axes"]]).to(torch.int32).contiguous()
    pairs = c["turned"] // 2
    s["inv_freq"] = (1e6 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float().to(dev)
    s["axis"] = [i % c["axes"] for i in range(pairs)]
    s["norm"] = [1 + 0.2 * torch.randn(d, generator=g, device=dev) if c["norms"] else None for _ in range(2)]
    writes, at = [], 0
    table = s["table"].cpu()
    for b, (h, n) in enumerate(zip(held, new)):
        t = h
        while t < h + n:
            take = min(h + n, (t // B + 1) * B) - t
            writes.append([int(table[b, t // B]), at, t % B, take])
            t, at = t + take, at + take
    s["writes"] = torch.zeros((min(tokens, tokens // B + 2 * len(new)), 4), dtype=torch.int32, device=dev)
    s["writes"][: len(writes)] = _ints(writes, dev)
    s["counts"] = _ints([tokens, len(writes), 0, 0], dev)
    if own:
        import paper_2602_20732_amd as pk
        s["rotary"] = pk.Rotary(s["inv_freq"], axis=s["axis"], interleaved=c["beside"], q_norm=s["norm"][0], k_norm=s["norm"][1], eps=EPS)
    return s


def _prepare_attend(s, g, held, new, n_phys):
    c, dev, tokens = s["case"], s["table"].device, s["tokens"]
    B, H, Hq, d, batch = c["page_size"], c["n_kv_heads"], c["n_q_heads"], HEAD_DIM, c["batch"]
    topics = torch.randn((64, H, d), generator=g, device=dev)
    about = torch.randint(0, 64, (n_phys,), generator=g, device=dev)
    s["k"] = torch.empty((n_phys, H, B, d), dtype=torch.bfloat16, device=dev)
    at = max(1, (1 << 26) // (B * H * d))
    for p in range(0, n_phys, at):
        q = min(n_phys, p + at)
        s["k"][p:q] = (torch.randn((q - p, H, B, d), generator=g, device=dev) + topics[about[p:q]][:, :, None]).to(torch.bfloat16)
    s["v"] = torch.empty((n_phys, H, d, B), dtype=torch.bfloat16, device=dev).normal_(generator=g)
    # a token's queries look for the topics of pages that its sequence holds
    row = torch.repeat_interleave(torch.arange(batch, device=dev), torch.tensor(new, device=dev))
    pick = (torch.rand((tokens, Hq), generator=g, device=dev) * (s["lens"][row] // B).clamp(min=1)[:, None]).long()
    page = s["table"].long()[row[:, None], pick]
    head = torch.arange(Hq, device=dev) // (Hq // H)
    s["q"] = (topics[about[page], head[None, :]] + torch.randn((tokens, Hq, d), generator=g, device=dev)).to(torch.bfloat16)
    s["out"] = torch.zeros((tokens, Hq, d), dtype=torch.bfloat16, device=dev)
    s["slopes"] = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=dev) / Hq) if c["slopes"] else None
    s["prefix"] = _ints([min(c["prefix"], h + n) for h, n in zip(held, new)], dev) if c["prefix"] else None
    s["first"] = _ints([p // c["document"] * c["document"] for h, n in zip(held, new) for p in range(h, h + n)], dev) if c["document"] else None
    if c["listed"]:
        # sink, window and pages from between, ascending, as a selection leaves them
        width, room = s["width"], min(c["listed"], s["width"])
        pages = -(-s["lens"].long() // B)
        score = torch.rand((batch, H, width), generator=g, device=dev)
        at = torch.arange(width, device=dev)
        score = torch.where((at < SINK) | (at >= (pages - WINDOW)[:, None, None]), 2.0, score)
        score = torch.where(at < pages[:, None, None], score, -1.0)
        ids = score.topk(room, dim=2).indices
        n = pages.clamp(max=room)[:, None].expand(batch, H)
        kept = torch.arange(room, device=dev) < n[:, :, None]
        ids = torch.where(kept, ids, width).sort(2).values
        s["ids"] = torch.where(kept, ids, -1).to(torch.int32).contiguous()
        s["n"] = n.to(torch.int32).contiguous()
    if own:
        import paper_2602_20732_amd as pk
        s["rule"] = pk.Scores(cap=c["cap"], slopes=s["slopes"], window=c["window"], prefix_lens=s["prefix"], first_keys=s["first"])
        s["most"] = max(new)
        s["scratch"] = s["lib"].new_attend_scratch(tokens, s["most"], batch, dev)
    return s


def _prepare_verify(s, g, held, new, n_phys):
    c, dev, tokens, batch = s["case"], s["table"].device, s["tokens"], s["case"]["batch"]
    V, most = c["vocab"], max(new) - 1
    starts = s["starts"].long()
    s["target"] = torch.empty((tokens, V), device=dev)
    s["draft"] = torch.zeros((batch, max(most, 1), V), device=dev) if c["given"] else None
    s["ids"] = torch.randint(0, V, (tokens,), generator=g, device=dev)
    for b, n in enumerate(new):
        at = int(sum(new[:b]))
        z = 3 * torch.randn((n, V), generator=g, device=dev)
        s["target"][at:at + n] = torch.softmax(z, 1)
        if n > 1:
            q = torch.softmax(z[: n - 1] + 0.7 * torch.randn((n - 1, V), generator=g, device=dev), 1)
            if c["given"]:
                s["draft"][b, : n - 1] = q
                s["ids"][at + 1:at + n] = torch.multinomial(q, 1, generator=g)[:, 0]
            else:
                s["ids"][at + 1:at + n] = torch.where(torch.rand(n - 1, generator=g, device=dev) < 0.7, s["target"][at:at + n - 1].argmax(1), s["ids"][at + 1:at + n])
    s["ids"] = s["ids"].to(torch.int32)
    s["uniforms"] = torch.rand((batch, most + 1), generator=g, device=dev)
    s["n_accepted"] = torch.zeros(batch, dtype=torch.int32, device=dev)
    s["out"] = torch.zeros((batch, most + 1), dtype=torch.int32, device=dev)
    s["lens_after"] = torch.zeros(batch, dtype=torch.int32, device=dev)
    s["free"] = torch.full((n_phys + 7,), -1, dtype=torch.int32, device=dev)
    s["n_free"], s["n_left"] = _ints([5], dev), _ints([0], dev)
    s["free"][:5] = torch.arange(5, dtype=torch.int32, device=dev) + n_phys
    return s


# ---- the pass
def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"rotate": _plain_rotate, "attend": _plain_attend, "verify": _plain_verify}[kind](s)
    lib = s["lib"]
    if kind == "rotate":
        lib.rotate_store(s["rotary"], s["q"], s["k_new"], s["v_new"], s["positions"], s["writes"], s["counts"], s["q_out"], s["k"], s["v"])
        return [s["q_out"], s["k"], s["v"]]
    if kind == "attend":
        if s["case"]["listed"]:
            lib.sparse_attend(s["q"], s["starts"], s["most"], s["k"], s["v"], s["table"], s["lens"], s["ids"], s["n"], s["out"], s["ws"], s["scratch"], s["rule"])
        else:
            lib.dense_attend(s["q"], s["starts"], s["most"], s["k"], s["v"], s["table"], s["lens"], s["out"], s["ws"], s["scratch"], s["rule"])
        return s["out"]
    lib.verify(s["target"], s["draft"], s["ids"], s["starts"], s["uniforms"], s["lens"], s["n_accepted"], s["out"], s["lens_after"], s["ws"])
    lib.trim_pages(s["lens"], s["lens_after"], s["table"], s["free"], s["n_free"], s["n_left"], s["ws"])
    return {k: s[k] for k in ("n_accepted", "out", "lens_after", "free", "n_left")}


def _plain_turned(s, x, weight, turn):
    c = s["case"]
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + EPS) * weight
    cos, sin = turn
    n = c["turned"]
    y = x.clone()
    a, b = (x[..., 0:n:2], x[..., 1:n:2]) if c["beside"] else (x[..., :n // 2], x[..., n // 2:n])
    first, second = a * cos - b * sin, a * sin + b * cos
    if c["beside"]:
        y[..., 0:n:2], y[..., 1:n:2] = first, second
    else:
        y[..., :n // 2], y[..., n // 2:n] = first, second
    return y.to(torch.bfloat16)


def _plain_rotate(s):
    B, dev = s["case"]["page_size"], s["q"].device
    # angles of far positions need 64 bits
    angle = s["positions"].double()[torch.tensor(s["axis"], device=dev)].t() * s["inv_freq"].double()
    turn = angle.cos().float()[:, None], angle.sin().float()[:, None]
    s["q_out"].copy_(_plain_turned(s, s["q"], s["norm"][0], turn))
    page, offset = s["slots"] // B, s["slots"] % B
    s["k"].transpose(1, 2)[page, offset] = _plain_turned(s, s["k_new"], s["norm"][1], turn)
    s["v"].permute(0, 3, 1, 2)[page, offset] = s["v_new"]
    return [s["q_out"], s["k"], s["v"]]


def _plain_attend(s):
    c = s["case"]
    B, H, G, dev = c["page_size"], c["n_kv_heads"], c["n_q_heads"] // c["n_kv_heads"], s["k"].device
    batch, lens, table, starts = c["batch"], s["lens"].long(), s["table"].long(), s["starts"].long()
    if c["listed"]:
        ids, there = s["ids"].long(), torch.arange(s["ids"].shape[2], device=dev) < s["n"][:, :, None]
    else:
        ids = torch.arange(s["width"] - 1, device=dev).expand(batch, H, -1)
        there = ids * B < lens[:, None, None]
    ids = torch.where(there, ids, 0)
    phys = table[torch.arange(batch, device=dev)[:, None, None], ids].clamp(min=0)           # [batch, H, pages]
    head = torch.arange(H, device=dev)[None, :, None]
    key = (ids[..., None] * B + torch.arange(B, device=dev)).flatten(2)                      # [batch, H, keys]
    there = there.repeat_interleave(B, 2) & (key < lens[:, None, None])
    # the new tokens of a sequence, padded to the most that any has
    n = starts[1:] - starts[:-1]
    i = torch.arange(c["new_hi"], device=dev)
    row = (starts[:-1, None] + i).clamp(max=s["tokens"] - 1)
    p = (lens - n)[:, None] + i                                                              # [batch, new]
    hi = p if s["prefix"] is None else torch.maximum(p, s["prefix"].long()[:, None] - 1)
    lo = torch.zeros_like(p) if s["first"] is None else s["first"].long()[row]
    if c["window"]:
        lo = torch.maximum(lo, p - c["window"] + 1)
    k = s["k"][phys, head].flatten(2, 3).float()
    z = (s["q"][row].view(batch, -1, H, G, HEAD_DIM).float().permute(0, 2, 1, 3, 4).reshape(batch, H, -1, HEAD_DIM) @ k.transpose(2, 3)).mul_(1 / math.sqrt(HEAD_DIM))
    del k
    z = z.view(batch, H, c["new_hi"], G, -1)
    if c["cap"]:
        z = z.div_(c["cap"]).tanh_().mul_(c["cap"])
    if s["slopes"] is not None:
        z -= s["slopes"].view(H, 1, G, 1) * (p[:, None, :, None] - key[:, :, None]).abs().float()[:, :, :, None]
    seen = there[:, :, None] & (key[:, :, None] >= lo[:, None, :, None]) & (key[:, :, None] <= hi[:, None, :, None])
    z = z.masked_fill_(~seen[:, :, :, None], -math.inf)
    z = z.sub_(z.amax(4, keepdim=True).clamp(min=torch.finfo(torch.float32).min)).exp_()
    z = z.div_(z.sum(4, keepdim=True).clamp(min=torch.finfo(torch.float32).tiny)).view(batch, H, c["new_hi"] * G, -1)
    v = s["v"][phys, head].transpose(3, 4).flatten(2, 3).float()
    o = (z @ v).view(batch, H, c["new_hi"], G, HEAD_DIM).permute(0, 2, 1, 3, 4).reshape(batch, c["new_hi"], H * G, HEAD_DIM)
    s["out"].copy_(o[i < n[:, None]])
    return s["out"]


def _plain_verify(s):
    c, dev, B = s["case"], s["ids"].device, s["case"]["page_size"]
    starts, lens, most = s["starts"].long(), s["lens"].long(), s["uniforms"].shape[1] - 1
    batch, n = len(lens), (starts[1:] - starts[:-1]) - 1
    b, j = torch.arange(batch, device=dev), torch.arange(most, device=dev)
    row = (starts[:-1, None] + j).clamp(max=s["tokens"] - 2 if s["tokens"] > 1 else 0)
    x = s["ids"].long()[(row + 1).clamp(max=s["tokens"] - 1)]
    p = s["target"][row, x].double()
    q = s["draft"][b[:, None], j, x].double() if c["given"] else torch.ones_like(p)
    fine = (s["uniforms"][:, :most].double() * q < p) & (j < n[:, None])
    accepted = fine.long().cumprod(1).sum(1)
    # the token behind them: what the target has over the draft, or the target's own where nothing was refused
    w = s["target"][starts[:-1] + accepted].double()
    refused = accepted < n
    at = accepted.clamp(max=max(most - 1, 0))
    if c["given"]:
        w = torch.where(refused[:, None], (w - s["draft"][b, at].double()).clamp(min=0), w)
    elif most:
        w[b, x[b, at]] = torch.where(refused, 0.0, w[b, x[b, at]])
    upto = w.cumsum(1)
    level = s["uniforms"][:, most].double() * upto[:, -1]
    token = (upto <= level[:, None]).sum(1)
    at = torch.arange(most + 1, device=dev)
    drafted = s["ids"].long()[(starts[:-1, None] + 1 + at).clamp(max=s["tokens"] - 1)]
    out = torch.where(at < accepted[:, None], drafted, torch.where(at == accepted[:, None], token[:, None], -1))
    s["n_accepted"].copy_(accepted)
    s["out"].copy_(out)
    after = lens - (n - accepted)
    s["lens_after"].copy_(after)
    # the pages behind, in row and page order
    kept, had = -(-after // B), -(-lens // B)
    page = torch.arange(s["width"], device=dev)
    back = s["table"][(page >= kept[:, None]) & (page < had[:, None])]
    first = s["n_free"].long()
    s["free"].scatter_(0, first + torch.arange(len(back), device=dev), back)
    s["n_left"].copy_(first + len(back))
    return {k: s[k] for k in ("n_accepted", "out", "lens_after", "free", "n_left")}


def work(case):
    kind, B, H, Hq, d = case["kind"], case["page_size"], case["n_kv_heads"], case["n_q_heads"], HEAD_DIM
    held, new = _rows(case)
    if kind == "rotate":
        touched = sum(-(-(h + n) // B) - h // B for h, n in zip(held, new))
        return {"bytes": sum(new) * ((Hq + 2 * H) * d * 4 + 4 * case["axes"]) + 16 * touched, "flops": sum(new) * (Hq + H) * d * 8}
    if kind == "verify":
        rows = 8 if case["given"] else 4
        return {"bytes": case["batch"] * (rows * case["vocab"] + 4 * (new[0] + 8)) + sum(new) * 16, "flops": case["batch"] * 2 * case["vocab"]}
    nbytes = flops = 0
    for h, n in zip(held, new):
        lo, hi = _interval(case, h, n)
        pages = -(-(h + n) // B)
        share = min(1.0, case["listed"] / pages) if case["listed"] else 1.0
        seen = sum(max(0, b - a + 1) for a, b in zip(lo, hi)) * share
        keys = max(0, max(hi) - min(lo) + 1) * share
        nbytes += H * (keys * d * 4 + keys / B * (8 if case["listed"] else 4)) + n * Hq * d * 4
        flops += 4 * Hq * d * seen
    return {"bytes": int(nbytes), "flops": int(flops)}


# ---- the same in 64 bits, sequence by sequence
def exact(case, seed):
    if case["kind"] == "verify":
        return None                                                                          # whole numbers
    s = prepare(case, seed)
    B, H, G, d = case["page_size"], case["n_kv_heads"], case["n_q_heads"] // case["n_kv_heads"], HEAD_DIM
    held, new = _rows(case)
    dev = s["table"].device
    if case["kind"] == "rotate":
        return _exact_rotate(s, case)
    out, at = torch.zeros((s["tokens"], H * G, d), dtype=torch.float64, device=dev), 0
    for b, (before, n) in enumerate(zip(held, new)):
        lo, hi = (torch.tensor(v, device=dev)[:, None] for v in _interval(case, before, n))
        p = torch.arange(before, before + n, device=dev)[:, None]
        for h in range(H):
            ids = s["ids"][b, h, : int(s["n"][b, h])].long() if case["listed"] else torch.arange(-(-(before + n) // B), device=dev)
            t = (ids[:, None] * B + torch.arange(B, device=dev)).reshape(-1)
            live = t < before + n
            t, phys = t[live], s["table"].long()[b, ids]
            k = s["k"][phys, h].reshape(-1, d)[live].double()
            v = s["v"][phys, h].transpose(1, 2).reshape(-1, d)[live].double()
            for i in range(h * G, h * G + G):
                z = s["q"][at:at + n, i].double() @ k.t() / math.sqrt(d)
                if case["cap"]:
                    z = case["cap"] * torch.tanh(z / case["cap"])
                if case["slopes"]:
                    z = z - s["slopes"][i].double() * (p - t).abs()
                z[(t < lo) | (t > hi)] = -math.inf
                out[at:at + n, i] = torch.nan_to_num(torch.softmax(z, 1)) @ v
        at += n
    return out


def _exact_rotate(s, case):
    """By complex numbers; the pools elsewhere as they are."""
    B, n = case["page_size"], case["turned"]
    at = torch.tensor(s["axis"], device=s["q"].device)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=at.device), s["positions"][at].t().double() * s["inv_freq"].double())[:, None]

    def of(x, weight):
        x = x.double()
        if weight is not None:
            x = x / ((x ** 2).sum(2, keepdim=True) / HEAD_DIM + EPS).sqrt() * weight.double()
        turned, kept = x[..., :n], x[..., n:]
        if case["beside"]:
            y = torch.view_as_real(torch.complex(turned[..., 0::2].contiguous(), turned[..., 1::2].contiguous()) * turn).flatten(2)
        else:
            z = torch.complex(turned[..., :n // 2].contiguous(), turned[..., n // 2:].contiguous()) * turn
            y = torch.cat([z.real, z.imag], 2)
        return torch.cat([y, kept], 2)

    k, v = s["k"].double(), s["v"].double()
    k_rows = of(s["k_new"], s["norm"][1])
    flat_k, flat_v = k.transpose(1, 2).reshape(-1, *k_rows.shape[1:]), v.permute(0, 3, 1, 2).reshape(-1, *k_rows.shape[1:])
    flat_k[s["slots"]], flat_v[s["slots"]] = k_rows, s["v_new"].double()
    k = flat_k.view(-1, B, *k_rows.shape[1:]).transpose(1, 2)
    v = flat_v.view(-1, B, *k_rows.shape[1:]).permute(0, 2, 3, 1)
    return [of(s["q"], s["norm"][0]), k, v]
