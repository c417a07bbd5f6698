"""The 8-bit paged cache as a serving program uses it: its operators as measurable cases.

  pages      ``release_pages`` for the requests that ended, then ``map_tokens``: pages for the tokens of the next step,
             block tables, token starts, slot map and write list
  store      ``quant_store``: keys and values of new tokens (slices of a fused projection) into 8-bit pages, one scale
             a page and head
  summarize  ``quant_summarize``: key summaries from 8-bit pages, whole prompts or the pages of the last steps
  attend     ``quant_sparse_decode`` over lists of pages, ``quant_dense_decode`` over every page

Keys: one topic vector for every page or so + N(0, I), a few channels eight times as large as the others; values N(0, I); queries
a topic of the sequence + N(0, I).  Pages lie in the pools in random order."""
import math
import random

import torch

own = False

HEAD_DIM = 128
FP8 = torch.float8_e4m3fn
E_MIN, E_MAX = -64, 119            # exponents a scale can have
SINK, WINDOW = 1, 4
RECENT = 10                        # pages generated between two selections
FAN = 8                            # pages of a chunk, chunks of a grid


def _case(name, kind, **more):
    c = {"name": name, "kind": kind, "batch": 1, "lo": 0, "hi": 0, "n_q_heads": 32, "n_kv_heads": 8, "page_size": 16}
    c.update(more)
    return c


def listed():
    return [
        # one conversation takes its next token: the smallest call
        _case("pages_b1_token", "pages", lo=4096, hi=4096, new_lo=1, new_hi=1, fresh=0.0),
        # a serving batch between two steps: most rows take a token, one in eight has ended and its row takes a prompt
        _case("pages_b256_mixed", "pages", batch=256, lo=1, hi=16384, new_lo=100, new_hi=2000, fresh=0.125),
        # a prefill of many prompts at once
        _case("pages_b64_prompts", "pages", batch=64, lo=0, hi=0, new_lo=1000, new_hi=8192, fresh=1.0),
        # a decode step: one token of every sequence joins a page, begun or new
        _case("store_b32_token", "store", batch=32, lo=1, hi=32768, new_lo=1, new_hi=1),
        # a chunk of prompts behind what their rows hold already, of odd lengths
        _case("store_b12_chunk", "store", batch=12, lo=0, hi=4099, new_lo=131, new_hi=4099),
        # one long prompt, pages of 32
        _case("store_b1_64k_page32", "store", lo=0, hi=0, new_lo=65531, new_hi=65531, n_q_heads=28, n_kv_heads=4, page_size=32),
        # the end of a prefill: summaries of whole prompts
        _case("summarize_b8_prompts", "summarize", batch=8, lo=30011, hi=131063, recent=0, vectors="fp32"),
        # the catch-up before a reselection
        _case("summarize_b96_recent", "summarize", batch=96, lo=4001, hi=21001, recent=RECENT, vectors="bf16"),
        # attention over the list of one short conversation: latency only
        _case("sparse_b1_4k", "attend", lo=4096, hi=4096, n_q_heads=8, listed=21),
        # a serving batch over its lists
        _case("sparse_b32_ragged", "attend", batch=32, lo=16384, hi=32768, listed=108),
        # full attention over ragged contexts (layers or requests that are not sparsified)
        _case("dense_b16_ragged", "attend", batch=16, lo=8200, hi=65536, listed=0),
        # one very long context, pages of 32 and seven query heads to a KV head
        _case("dense_b1_256k_page32", "attend", lo=262139, hi=262139, n_q_heads=28, n_kv_heads=4, page_size=32, listed=0),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("pages", "store", "store", "summarize", "summarize", "attend", "attend", "attend"))
    heads, page = rng.choice((((8, 8), 16), ((32, 8), 16), ((32, 8), 32), ((28, 4), 16), ((28, 4), 32)))
    c = {"kind": kind, "n_q_heads": heads[0], "n_kv_heads": heads[1], "page_size": page}
    if kind == "pages":
        new = spread(1, 8192)
        c.update(batch=spread(1, 512), lo=1, hi=spread(1, 16384), new_lo=max(1, new // 4), new_hi=new, fresh=rng.choice((0.0, 0.1, 0.5)))
        c["batch"] = max(1, min(c["batch"], (1 << 18) // new, (1 << 22) // c["hi"]))
    elif kind == "store":
        new = spread(1, 65536)
        c.update(batch=max(1, min(spread(1, 256), (1 << 16) // new)), lo=0, hi=spread(1, 8192), new_lo=max(1, new // 3), new_hi=new)
    else:
        hi = spread(512, 262144)
        c.update(batch=max(1, min(spread(1, 96), (1 << 19) // hi)), lo=spread(max(1, hi // 8), hi), hi=hi)
        if kind == "summarize":
            c.update(recent=rng.choice((0, 0, 1, spread(1, 40))), vectors=rng.choice(("fp32", "bf16")))
        else:
            pages = -(-hi // page)
            c.update(listed=rng.choice((0, 0, min(pages, spread(5, 600)))))
    return c


# ---- sizes that follow from a case
def _between(r, lo, hi, n):
    """n whole numbers between lo and hi, both among them."""
    got = [hi] + [lo + r.randrange(hi - lo + 1) for _ in range(n - 1)]
    if n > 1:
        got[-1] = lo
    return got


def _rows(case):
    """(tokens a row holds, tokens it takes, whether its request has ended) of every row."""
    r = random.Random(case["batch"] * 7 + case["hi"] * 3 + case.get("new_hi", 0))
    n = case["batch"]
    held = _between(r, case["lo"], case["hi"], n)
    if case["kind"] == "pages":
        fresh = [r.random() < case["fresh"] for _ in range(n)]
        prompts = _between(r, case["new_lo"], case["new_hi"], n)
        return held, [p if f else 1 for p, f in zip(prompts, fresh)], fresh
    if case["kind"] == "store":
        return held, _between(r, case["new_lo"], case["new_hi"], n), [False] * n
    return held, [0] * n, [False] * n


def _touched(held, new, B):
    """Pages that `new` tokens behind `held` ones lie in."""
    return -(-(held + new) // B) - held // B if new else 0


def _most_writes(tokens, batch, B):
    return min(tokens, tokens // B + 2 * batch)


# ---- the 8-bit form
def _power(e):
    """2^e in fp32, for whole e in the normal range."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(a):
    """The smallest e with a 2^-e <= 448 (a >= 0 and finite), within what a scale can have."""
    m, x = torch.frexp(a)
    e = x - 9 + (m > 0.875).to(x.dtype)
    return torch.where(a > 0, e, E_MIN).clamp(E_MIN, E_MAX)


def _exponent_of(scale):
    return ((scale.view(torch.int32) >> 23) & 255) - 127


def _to_fp8(x, e):
    y = (x * _power(-e)).clamp(-448.0, 448.0)
    return torch.where(torch.isfinite(x), y, torch.nan).to(FP8)


def _page_amax(x, dims):
    return torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dims)


# ---- inputs
def _gains(g, H, dev):
    gain = torch.ones((H, HEAD_DIM), device=dev)
    for h in range(H):
        gain[h, torch.randperm(HEAD_DIM, generator=g, device=dev)[:3]] = 8.0
    return gain


def _pools(case, n_phys, g, dev):
    """K pool, V pool, scales of n_phys full pages, and the topic that each page's keys are about."""
    B, H, d = case["page_size"], case["n_kv_heads"], HEAD_DIM
    topics, gain = torch.randn((64, H, d), generator=g, device=dev), _gains(g, H, dev)
    about = torch.randint(0, 64, (n_phys,), generator=g, device=dev)
    k = torch.empty((n_phys, H, B, d), dtype=FP8, device=dev)
    v = torch.empty((n_phys, H, d, B), dtype=FP8, device=dev)
    scales = torch.empty((n_phys, H, 2), dtype=torch.float32, device=dev)
    at = max(1, (1 << 25) // (B * H * d))
    for p in range(0, n_phys, at):
        q = min(n_phys, p + at)
        x = torch.randn((q - p, H, B, d), generator=g, device=dev)
        x = (x + topics[about[p:q]][:, :, None]) * gain[:, None]
        e = _exponent(_page_amax(x, (2, 3)))
        k[p:q] = _to_fp8(x, e[:, :, None, None])
        scales[p:q, :, 0] = _power(e)
        x = torch.randn((q - p, H, d, B), generator=g, device=dev)
        e = _exponent(_page_amax(x, (2, 3)))
        v[p:q] = _to_fp8(x, e[:, :, None, None])
        scales[p:q, :, 1] = _power(e)
    return k, v, scales, (topics, about)


def _table(pages, width, order, dev):
    """Block table of rows that hold so many pages, dealt out of `order`; behind them -1."""
    pages = torch.tensor(pages, device=dev)
    table = torch.full((len(pages), width), -1, dtype=torch.int32, device=dev)
    there = torch.arange(width, device=dev)[None, :] < pages[:, None]
    table[there] = order[: int(pages.sum())].to(torch.int32)
    return table


def _ints(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    kind, B, H, Hq, d, batch = case["kind"], case["page_size"], case["n_kv_heads"], case["n_q_heads"], HEAD_DIM, case["batch"]
    held, new, ended = _rows(case)
    width = max(-(-(h + n) // B) for h, n in zip(held, new)) + 1
    s = {"case": dict(case), "lens": _ints(held, dev), "width": width}
    most_listed = case.get("listed", 0) or width
    if own:
        import paper_2602_20732_amd as pk
        s["lib"] = pk.Chess(pk.Config(Hq, H, B, batch, width, min(most_listed, width), FAN, FAN,
                                      summary_dtype=pk.SUMMARY_BF16 if case.get("vectors") == "bf16" else pk.SUMMARY_F32))
        s["ws"] = s["lib"].new_workspace(dev)

    if kind == "pages":
        pages = [-(-h // B) for h in held]
        n_phys = sum(pages) + sum(-(-n // B) + 1 for n in new)
        order = torch.randperm(n_phys, generator=g, device=dev)
        tokens = sum(new)
        free = n_phys - sum(pages)
        s.update(table=_table(pages, width, order, dev), done=_ints([int(e) for e in ended], dev), new=_ints(new, dev),
                 free=torch.full((n_phys,), -1, dtype=torch.int32, device=dev), n_free=_ints([free], dev), tokens=tokens,
                 lens_kept=torch.zeros(batch, dtype=torch.int32, device=dev), n_kept=_ints([0], dev),
                 lens_after=torch.zeros(batch, dtype=torch.int32, device=dev), n_left=_ints([0], dev),
                 starts=torch.zeros(batch + 1, dtype=torch.int32, device=dev),
                 slots=torch.full((tokens,), -1, dtype=torch.int64, device=dev),
                 writes=torch.full((_most_writes(tokens, batch, B), 4), -1, dtype=torch.int32, device=dev),
                 counts=torch.zeros(4, dtype=torch.int32, device=dev))
        s["free"][:free] = order[sum(pages):].to(torch.int32)
        return s

    n_phys = sum(-(-(h + n) // B) for h, n in zip(held, new)) + 1
    order = torch.randperm(n_phys, generator=g, device=dev)
    s["table"] = _table([-(-(h + n) // B) for h, n in zip(held, new)], width, order, dev)
    s["k"], s["v"], s["scales"], (topics, about) = _pools(case, n_phys, g, dev)

    if kind == "store":
        tokens = sum(new)
        # the projection's output: queries, keys and values of a token side by side
        rows = torch.randn((tokens, Hq + 2 * H, d), generator=g, device=dev)
        rows[:, Hq:Hq + H] = (rows[:, Hq:Hq + H] + topics[torch.randint(0, 64, (tokens,), generator=g, device=dev)]) * _gains(g, H, dev)
        rows = rows.to(torch.bfloat16)
        table, writes, row = s["table"].cpu(), [], 0
        for b, (h, n) in enumerate(zip(held, new)):
            at = h
            while at < h + n:
                take = min(h + n, (at // B + 1) * B) - at
                writes.append([int(table[b, at // B]), row, at % B, take])
                at, row = at + take, row + take
        s.update(k_new=rows[:, Hq:Hq + H], v_new=rows[:, Hq + H:], counts=_ints([tokens, len(writes), 0, 0], dev),
                 writes=torch.zeros((_most_writes(tokens, batch, B), 4), dtype=torch.int32, device=dev))
        s["writes"][: len(writes)] = _ints(writes, dev)
        return s

    if kind == "summarize":
        vec = torch.bfloat16 if case["vectors"] == "bf16" else torch.float32
        chunks = -(-width // FAN)
        s["units"] = [torch.zeros((batch, H, n, d), dtype=vec, device=dev) for n in (width, chunks, -(-chunks // FAN))]
        if case["recent"]:
            _plain_summaries(s, 0)
        if own:
            s["summaries"] = s["lib"].new_summaries(dev)
            for mine, theirs in zip(s["lib"].summary_views(s["summaries"]), s["units"]):
                mine.copy_(theirs)
            s["units"] = list(s["lib"].summary_views(s["summaries"]))
        return s

    # a query looks for the topics of a page that its sequence holds
    pick = (torch.rand((batch, Hq), generator=g, device=dev) * (s["lens"] // B).clamp(min=1)[:, None]).long()
    page = s["table"].long().gather(1, pick)
    head = torch.arange(Hq, device=dev) // (Hq // H)
    s["q"] = (topics[about[page], head[None, :]] + torch.randn((batch, Hq, d), generator=g, device=dev)).to(torch.bfloat16)
    s["out"] = torch.empty((batch, Hq, d), dtype=torch.float32, device=dev)
    if case["listed"]:
        # sink, window and pages from between, ascending, as a selection leaves them
        pages, room = -(-s["lens"].long() // B), s["case"]["listed"]
        score = torch.rand((batch, H, width), generator=g, device=dev)
        at = torch.arange(width, device=dev)
        score = torch.where((at < SINK) | (at >= (pages - WINDOW)[:, None, None]), 2.0, score)
        score = torch.where(at < pages[:, None, None], score, -1.0)
        ids = score.topk(min(room, width), dim=2).indices
        n = pages.clamp(max=room)[:, None].expand(batch, H)
        kept = torch.arange(ids.shape[2], device=dev) < n[:, :, None]
        ids = torch.where(kept, ids, width).sort(2).values
        s["ids"] = torch.where(kept, ids, -1).to(torch.int32).contiguous()
        s["n"] = n.to(torch.int32).contiguous()
    return s


# ---- the pass
def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"pages": _plain_pages, "store": _plain_store, "summarize": lambda s: _plain_summaries(s, s["case"]["recent"]),
                "attend": _plain_attend}[kind](s)
    lib = s["lib"]
    if kind == "pages":
        lib.release_pages(s["lens"], s["done"], s["table"], s["free"], s["n_free"], s["lens_kept"], s["n_kept"], s["ws"])
        lib.map_tokens(s["lens_kept"], s["new"], s["table"], s["free"], s["n_kept"], s["lens_after"], s["n_left"], s["starts"], s["slots"],
                       s["writes"], s["counts"], s["ws"])
        return {k: s[k] for k in ("table", "free", "lens_after", "n_left", "starts", "slots", "writes", "counts")}
    if kind == "store":
        lib.quant_store(s["k_new"], s["v_new"], s["writes"], s["counts"], s["k"], s["v"], s["scales"])
        return [s["k"], s["v"], s["scales"]]
    if kind == "summarize":
        lib.quant_summarize(s["k"], s["scales"], s["table"], s["lens"], s["summaries"], recent_pages=s["case"]["recent"])
        return s["units"]
    if s["case"]["listed"]:
        lib.quant_sparse_decode(s["q"], s["k"], s["v"], s["scales"], s["table"], s["lens"], s["ids"], s["n"], s["out"], s["ws"])
    else:
        lib.quant_dense_decode(s["q"], s["k"], s["v"], s["scales"], s["table"], s["lens"], s["out"], s["ws"])
    return s["out"]


def _plain_pages(s):
    B, width, table, free, dev = s["case"]["page_size"], s["width"], s["table"], s["free"], s["table"].device
    at = torch.arange(width, device=dev)
    # the requests that ended give their pages back, in row and page order
    n_free = s["n_free"].long()
    ended, lens = s["done"] != 0, s["lens"].long()
    back = torch.where(ended, -(-lens // B), 0)
    first = n_free + back.cumsum(0) - back
    pushed = at[None, :] < back[:, None]
    spot = torch.where(pushed, first[:, None] + at[None, :], free.numel())
    longer = torch.cat([free, free[:1]])
    longer[spot.reshape(-1)] = table.reshape(-1)
    free.copy_(longer[:-1])
    n_free = n_free + back.sum()
    lens = torch.where(ended, 0, lens)
    # in row order, as long as tokens and pages last
    new = s["new"].long()
    new = torch.where((new >= 0) & (lens + new <= width * B), new, 0)
    had, need = -(-lens // B), -(-(lens + new) // B) - (-(-lens // B))
    fits = (new.cumsum(0) <= s["tokens"]) & (need.cumsum(0) <= n_free)
    refused = ((s["new"] > 0) & ~(fits & (new > 0))).sum()
    new, need = torch.where(fits, new, 0), torch.where(fits, need, 0)
    upto, taken = new.cumsum(0), need.cumsum(0)
    # the pages they take, from the end of the free list
    gained = (at >= had[:, None]) & (at < (had + need)[:, None])
    source = n_free - 1 - ((taken - need)[:, None] + at[None, :] - had[:, None])
    table.copy_(torch.where(gained, free[source.clamp(0, free.numel() - 1)], table))
    # token by token
    t = torch.arange(s["slots"].numel(), device=dev)
    row = torch.searchsorted(upto, t, right=True).clamp(max=len(upto) - 1)
    place = lens[row] + t - (upto - new)[row]
    slot = table[row, (place // B).clamp(0, width - 1)].long() * B + place % B
    s["slots"].copy_(torch.where(t < upto[-1], slot, s["slots"]))
    # page by page
    pages = torch.where(new > 0, (lens + new - 1) // B - lens // B + 1, 0)
    w_upto = pages.cumsum(0)
    w = torch.arange(s["writes"].shape[0], device=dev)
    row = torch.searchsorted(w_upto, w, right=True).clamp(max=len(upto) - 1)
    page = lens[row] // B + w - (w_upto - pages)[row]
    begin = torch.maximum(lens[row], page * B)
    end = torch.minimum((lens + new)[row], page * B + B)
    entry = torch.stack([table[row, page.clamp(0, width - 1)].long(), (upto - new)[row] + begin - lens[row], begin - page * B, end - begin], 1)
    s["writes"].copy_(torch.where((w < w_upto[-1])[:, None], entry.to(torch.int32), s["writes"]))
    s["lens_after"].copy_(lens + new)
    s["n_left"].copy_(n_free - taken[-1])
    s["starts"].copy_(torch.cat([upto.new_zeros(1), upto]))
    s["counts"].copy_(torch.stack([upto[-1], w_upto[-1], taken[-1], refused]))
    return {k: s[k] for k in ("table", "free", "lens_after", "n_left", "starts", "slots", "writes", "counts")}


def _plain_store(s):
    B, dev = s["case"]["page_size"], s["k"].device
    # (entries behind the last one repeat the first, which stores the same twice)
    live = torch.arange(s["writes"].shape[0], device=dev) < s["counts"][1]
    entry = torch.where(live[:, None], s["writes"], s["writes"][:1]).long()
    phys, row, first, count = entry.unbind(1)
    t = torch.arange(B, device=dev)
    is_new = (t >= first[:, None]) & (t < (first + count)[:, None])
    is_old = t < first[:, None]
    source = (row[:, None] + t - first[:, None]).clamp(0, s["k_new"].shape[0] - 1)
    _plain_store_one(s["k"], s["scales"], 0, s["k_new"][source].float().permute(0, 2, 1, 3), is_new[:, None, :, None], is_old[:, None, :, None], phys, first)
    _plain_store_one(s["v"], s["scales"], 1, s["v_new"][source].float().permute(0, 2, 3, 1), is_new[:, None, None, :], is_old[:, None, None, :], phys, first)
    return [s["k"], s["v"], s["scales"]]


def _plain_store_one(pool, scales, which, x, is_new, is_old, phys, first):
    stored = pool.view(torch.uint8)[phys]
    e_old = torch.where((first > 0)[:, None], _exponent_of(scales[phys, :, which]), E_MIN)
    e = torch.maximum(_exponent(_page_amax(torch.where(is_new, x, 0.0), (2, 3))), e_old)
    fresh = _to_fp8(x, e[:, :, None, None]).view(torch.uint8)
    moved = (stored.view(FP8).float() * _power((e_old - e).clamp(min=-126))[:, :, None, None]).to(FP8).view(torch.uint8)
    pool.view(torch.uint8)[phys] = torch.where(is_new, fresh, torch.where(is_old, moved, stored))
    scales[phys, :, which] = _power(e)




def _plain_summaries(s, recent):
    B, table, lens = s["case"]["page_size"], s["table"].long(), s["lens"].long()
    pages, chunks, grids = s["units"]
    dev, width = table.device, s["width"]
    held = -(-lens // B)
    most = min(recent, width) if recent else width
    first = (held - most).clamp(min=0)
    # pages, then the chunks and the grids that hold them; an index behind a row's last unit repeats that unit
    row = torch.arange(len(lens), device=dev)[:, None]
    j = torch.minimum(first[:, None] + torch.arange(most, device=dev), held[:, None] - 1)
    phys = table.gather(1, j)
    x = s["k"].view(torch.uint8)[phys].view(FP8).float()
    x *= s["scales"][phys, :, 0][..., None, None]
    there = j[:, :, None] * B + torch.arange(B, device=dev) < lens[:, None, None]
    x = x.masked_fill_(~there[:, :, None, :, None], 0.0).sum(3) / there.sum(2)[:, :, None, None]
    pages[row, :, j] = x.to(pages.dtype)
    below, n = pages, held
    for units in (chunks, grids):
        first, n_up = first // FAN, -(-n // FAN)
        most = min((most + FAN - 2) // FAN + 1, units.shape[2])
        j = torch.minimum(first[:, None] + torch.arange(most, device=dev), n_up[:, None] - 1)
        member = j[:, :, None] * FAN + torch.arange(FAN, device=dev)
        there = member < n[:, None, None]
        x = below[row[:, :, None], :, member.clamp(max=below.shape[2] - 1)].float()          # [batch, units, members, H, d]
        x = torch.where(there[..., None, None], x, 0.0).sum(2) / there.sum(2)[:, :, None, None]
        units[row, :, j] = x.to(units.dtype)
        below, n = units, n_up
    return s["units"]


def _plain_attend(s):
    c = s["case"]
    B, H, G, dev = c["page_size"], c["n_kv_heads"], c["n_q_heads"] // c["n_kv_heads"], s["k"].device
    batch, lens, table = c["batch"], s["lens"].long(), s["table"].long()
    if c["listed"]:
        ids, there = s["ids"].long(), torch.arange(s["ids"].shape[2], device=dev) < s["n"][:, :, None]
    else:
        ids = torch.arange(s["width"], device=dev).expand(batch, H, -1)
        there = ids * B < lens[:, None, None]
    ids = torch.where(there, ids, 0)
    phys = table[torch.arange(batch, device=dev)[:, None, None], ids].clamp(min=0)           # [batch, H, pages]
    head = torch.arange(H, device=dev)[None, :, None]
    token = ids[..., None] * B + torch.arange(B, device=dev)
    there = (there[..., None] & (token < lens[:, None, None, None])).flatten(2)              # [batch, H, tokens]
    k = s["k"].view(torch.uint8)[phys, head].view(FP8).float()
    k *= s["scales"][phys, head, 0][..., None, None]
    q = s["q"].float().view(batch, H, G, HEAD_DIM)
    z = (q @ k.flatten(2, 3).transpose(2, 3)) / math.sqrt(HEAD_DIM)
    del k
    z = torch.where(there[:, :, None], z, -math.inf)
    p = torch.exp(z - z.amax(3, keepdim=True))
    p = p / p.sum(3, keepdim=True)
    v = s["v"].view(torch.uint8)[phys, head].view(FP8).float()
    v *= s["scales"][phys, head, 1][..., None, None]
    s["out"].copy_((p @ v.transpose(3, 4).flatten(2, 3)).reshape(batch, H * G, HEAD_DIM))
    return s["out"]


def work(case):
    kind, B, H, Hq, d = case["kind"], case["page_size"], case["n_kv_heads"], case["n_q_heads"], HEAD_DIM
    held, new, ended = _rows(case)
    if kind == "pages":
        back = sum(-(-h // B) for h, e in zip(held, ended) if e)
        kept = [0 if e else h for h, e in zip(held, ended)]
        touched = sum(_touched(h, n, B) for h, n in zip(kept, new))
        gained = sum(-(-(h + n) // B) - (-(-h // B)) for h, n in zip(kept, new))
        return {"bytes": 8 * back + 8 * sum(new) + 16 * touched + 8 * gained + 20 * case["batch"], "flops": 0}
    if kind == "store":
        touched = sum(_touched(h, n, B) for h, n in zip(held, new))
        return {"bytes": sum(new) * H * d * 2 * (2 + 1) + touched * (16 + H * 8), "flops": sum(new) * H * d * 2 * 2}
    nbytes = flops = 0
    for n in held:
        pages = -(-n // B)
        if kind == "summarize":
            recent = min(pages, case["recent"] or pages)
            chunks = -(-pages // FAN) - (pages - recent) // FAN
            grids = -(-(-(-pages // FAN)) // FAN) - (pages - recent) // FAN // FAN
            rows = n - (pages - recent) * B
            nbytes += H * (rows * d + recent * 8 + (recent + chunks + grids) * d * (2 if case["vectors"] == "bf16" else 4))
            flops += H * rows * d
        else:
            taken = min(pages, case["listed"]) if case["listed"] else pages
            tokens = min(n, taken * B)
            nbytes += H * (tokens * d * 2 + taken * (8 + 4 + (4 if case["listed"] else 0))) + Hq * d * (2 + 4)
            flops += 4 * Hq * tokens * d
    return {"bytes": nbytes, "flops": flops}


# ---- the same in 64 bits, sequence by sequence
def exact(case, seed):
    if case["kind"] == "pages":
        return None                                                                          # whole numbers
    s = prepare(case, seed)
    B, H, G = case["page_size"], case["n_kv_heads"], case["n_q_heads"] // case["n_kv_heads"]
    if case["kind"] == "store":
        return _exact_store(s)
    table, lens = s["table"].long(), s["lens"].tolist()
    if case["kind"] == "summarize":
        return _exact_summaries(s)
    out = torch.zeros((case["batch"], H * G, HEAD_DIM), dtype=torch.float64, device=table.device)
    for b, n in enumerate(lens):
        for h in range(H):
            ids = s["ids"][b, h, : int(s["n"][b, h])].long() if case["listed"] else torch.arange(-(-n // B), device=table.device)
            phys = table[b, ids]
            live = (ids[:, None] * B + torch.arange(B, device=table.device) < n).reshape(-1)
            k = (s["k"].view(torch.uint8)[phys, h].view(FP8).double() * s["scales"][phys, h, 0].double()[:, None, None]).reshape(-1, HEAD_DIM)[live]
            v = (s["v"].view(torch.uint8)[phys, h].view(FP8).double() * s["scales"][phys, h, 1].double()[:, None, None]).transpose(1, 2).reshape(-1, HEAD_DIM)[live]
            q = s["q"][b, h * G:(h + 1) * G].double()
            out[b, h * G:(h + 1) * G] = torch.softmax(q @ k.t() / math.sqrt(HEAD_DIM), 1) @ v
    return out


def _exact_store(s):
    """What the bytes would be without rounding, and the scales."""
    k, v, scales = s["k"].double(), s["v"].double(), s["scales"].double()
    for phys, row, first, count in s["writes"][: int(s["counts"][1])].tolist():
        for which, pool, rows in ((0, k[phys], s["k_new"]), (1, v[phys].transpose(1, 2), s["v_new"])):   # [H, B, d] views
            x = rows[row:row + count].double().transpose(0, 1)
            scale = torch.exp2((x.abs().amax((1, 2)) / 448).log2().ceil())
            # (log2 next to a whole number: settled by the definition itself)
            scale = torch.where(x.abs().amax((1, 2)) <= 448 * scale / 2, scale / 2, scale)
            scale = torch.where(x.abs().amax((1, 2)) > 448 * scale, scale * 2, scale)
            if first > 0:
                scale = torch.maximum(scale, scales[phys, :, which])
                pool[:, :first] *= (scales[phys, :, which] / scale)[:, None, None]
            pool[:, first:first + count] = x / scale[:, None, None]
            scales[phys, :, which] = scale
    return [k, v, scales]


def _exact_summaries(s):
    """Every unit of every sequence; units older than the recent pages' are what they were."""
    B, table, recent = s["case"]["page_size"], s["table"].long(), s["case"]["recent"]
    got = [u.double() for u in s["units"]]
    for b, n in enumerate(s["lens"].tolist()):
        held = -(-n // B)
        start = max(0, held - recent) if recent else 0
        phys = table[b, start:held]
        x = s["k"].view(torch.uint8)[phys].view(FP8).double() * s["scales"][phys, :, 0].double()[:, :, None, None]
        count = torch.full((held - start,), B, dtype=torch.float64, device=table.device)
        count[-1] = n - (held - 1) * B
        live = torch.arange(B, device=table.device) < count[:, None]
        below = (x * live[:, None, :, None]).sum(2) / count[:, None, None]
        got[0][b, :, start:held] = below.transpose(0, 1)
        for level in (1, 2):
            start, had = start // FAN, held
            held = -(-held // FAN)
            x = torch.zeros((s["case"]["n_kv_heads"], (held - start) * FAN, HEAD_DIM), dtype=torch.float64, device=table.device)
            x[:, : had - start * FAN] = got[level - 1][b, :, start * FAN:had].to(s["units"][0].dtype).double()
            count = torch.full((held - start,), FAN, dtype=torch.float64, device=table.device)
            count[-1] = had - (held - 1) * FAN
            got[level][b, :, start:held] = x.view(x.shape[0], held - start, FAN, HEAD_DIM).sum(2) / count[None, :, None]
    return got
