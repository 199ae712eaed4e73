"""The operators of a block-sparse attention layer over a paged cache, as measurable cases.

A layer's step is a chain of five calls: new queries and keys are rotated to their positions (`vpp_rope` by itself, or
`vpp_kv_append_rope`, which writes the rotated keys and the values to the cache on the way), the mean keys of the pages that the
chunk completes are formed (`vpp_block_means`), every token's cheap score against those means selects pages
(`vpp_block_select`), and attention runs over the selected pages alone (`vpp_block_attn_fwd`).  The listed cases are each call
for decode batches, where latency counts, and for chunks of long prompts; `draw` gives more of the same ranges, with mixed
batches among them.  A case holds sizes only; ragged lengths follow from its `lens` number, values from the seed.
"""
import math

import numpy as np
import torch

own = False

HALF, INTERLEAVED = "half", "interleaved"


def listed():
    return [
        # queries of a small decode batch, all features rotated (the smallest call: one launch)
        dict(name="rope_few", kind="rope", rows=16, reqs=0, budget=0, longest=131072, heads=64, dim=128, rot=128, offset=0,
             layout=HALF, amplitude=1.0, lens=1),
        # rope part of a chunk's absorbed-MLA queries, far into a prompt, written beside the latent part; scaled for long contexts
        dict(name="rope_chunk", kind="rope", rows=0, reqs=1, budget=8192, longest=524288, heads=128, dim=64, rot=64, offset=0,
             layout=INTERLEAVED, amplitude=1.1386, lens=2),
        # a decode batch's queries, keys and values straight from the fused projection, GQA 64/8
        dict(name="append_few", kind="append", rows=32, reqs=0, budget=0, longest=32768, hq=64, hkv=8, dim=128, rot=128, offset=0,
             layout=HALF, amplitude=1.0, page=16, lens=3),
        # the same for a full-size chunk near the end of a prompt of a million tokens
        dict(name="append_chunk", kind="append", rows=0, reqs=1, budget=16384, longest=1048576, hq=64, hkv=8, dim=128, rot=128,
             offset=0, layout=HALF, amplitude=1.0, page=128, lens=4),
        # continuous batching on one rank's heads: the pages that 256 decode rows complete (about one row in sixteen)
        dict(name="means_few", kind="means", rows=256, reqs=0, budget=0, longest=32768, hkv=8, page=16, lens=5),
        # the pages of a full-size chunk at an unaligned place
        dict(name="means_chunk", kind="means", rows=0, reqs=1, budget=16384, longest=131000, hkv=8, page=128, lens=6),
        # page selection for a decode batch at long contexts
        dict(name="select_few", kind="select", rows=16, reqs=0, budget=0, longest=131072, hq=64, hkv=8, page=64, topk=32, first=1,
             last=2, lens=7),
        # page selection for a chunk deep in a long prompt (GQA 64/4)
        dict(name="select_chunk", kind="select", rows=0, reqs=1, budget=8192, longest=73728, hq=64, hkv=4, page=64, topk=32, first=1,
             last=2, lens=8),
        # attention over the selected pages: four decode rows
        dict(name="blocks_few", kind="blocks", rows=4, reqs=0, budget=0, longest=65536, hq=64, hkv=8, page=64, topk=32, spread=0.5,
             lens=9),
        # a decode batch, ragged contexts
        dict(name="blocks_decode", kind="blocks", rows=64, reqs=0, budget=0, longest=65536, hq=64, hkv=8, page=64, topk=32, spread=0.5,
             lens=10),
        # an ordinary chunk of one rank's heads of a GQA 64/8 model sharded eight ways, unaligned, smaller pages
        dict(name="blocks_shard", kind="blocks", rows=0, reqs=1, budget=1999, longest=30011, hq=8, hkv=1, page=32, topk=48, spread=0.3,
             lens=11),
        # a chunk deep in a long prompt (GQA 64/4): the largest
        dict(name="blocks_chunk", kind="blocks", rows=0, reqs=1, budget=4096, longest=69632, hq=64, hkv=4, page=64, topk=32, spread=0.3,
             lens=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    kind = rng.choice(["rope", "append", "append", "means", "select", "select", "blocks", "blocks", "blocks"])
    form = rng.choice(["rows", "chunk", "mixed"])
    most = {"rope": 8192, "append": 16384, "means": 16384, "select": 8192, "blocks": 4096}[kind]
    case = dict(kind=kind, rows=0, reqs=0, budget=0, longest=_log(rng, 2000, 131072 if kind in ("rope", "append", "select") else 65536),
                lens=rng.randrange(1 << 20))
    if form != "chunk":
        case["rows"] = _log(rng, 1, 256 if kind in ("rope", "append", "means") else 64)
    if form == "chunk":
        case.update(reqs=1, budget=_log(rng, 100, most))
    if form == "mixed":
        case["reqs"] = _log(rng, 2, 8)
        case["budget"] = max(8 * case["reqs"], _log(rng, 100, most // 4))
    hq, hkv = rng.choice([(64, 4), (64, 8), (32, 8), (32, 32), (16, 2), (8, 1), (15, 5)])
    if kind in ("rope", "append"):
        dim = rng.choice([64, 128, 128]) if kind == "rope" else 128
        rot = rng.choice([dim, dim, dim // 2])
        case.update(dim=dim, rot=rot, offset=rng.choice([0, dim - rot]), layout=rng.choice([HALF, INTERLEAVED]),
                    amplitude=rng.choice([1.0, 1.0, 1.2079]))
    if kind == "rope":
        case["heads"] = rng.choice([1, 5, 8, 40, 64, 128])
        return case
    case.update(hkv=hkv, page=rng.choice([16, 32, 64, 128]))
    if kind == "means":
        return case
    case["hq"] = hq
    if kind in ("select", "blocks"):
        case["topk"] = _log(rng, 4, 64)
    if kind == "select":
        case.update(first=rng.choice([0, 1, 2]), last=rng.choice([1, 1, 2]))
    if kind == "blocks":
        case["spread"] = rng.choice([0.1, 0.3, 0.5])
    return case


def draw(rng):
    """One more case of these ranges that costs no more than the largest listed one."""
    def cost(case):
        w = work(case)
        return max(w["bytes"], w["flops"] / 200)      # (about the ratio of the card's matrix rate to its memory rate)
    def held(case):
        """Values that the plain form holds at a time: keys of every token's list, scores of every token against every request's pages."""
        pre, chk = lengths(case)
        if case["kind"] == "blocks":
            return sum(chk) * case["hkv"] * case["topk"] * case["page"] * 128
        if case["kind"] == "select":
            return sum(chk) * case["hkv"] * len(pre) * (max(p + c for p, c in zip(pre, chk)) // case["page"] + 1)
        return 0
    most = max(cost(c) for c in listed())
    while True:
        case = _draw(rng)
        if cost(case) <= most and held(case) <= (1 << 32 if case["kind"] == "blocks" else 1 << 28):
            return case


def lengths(case):
    """(prefix, chunk) lengths of the case's requests: `reqs` chunks of together `budget` tokens, `rows` decode rows."""
    n, rows, longest = case["reqs"], case["rows"], case["longest"]
    if n == 1 and rows == 0:
        return [max(0, longest - case["budget"])], [case["budget"]]
    rng = np.random.default_rng(case["lens"])
    pre, chk = [], []
    if n:
        c = 1 + np.floor(rng.dirichlet(np.full(n, 2.0)) * (case["budget"] - n)).astype(int)
        c[0] += case["budget"] - int(c.sum())
        total = np.exp(rng.uniform(math.log(longest / 64), math.log(longest), size=n)).astype(int)
        pre += [int(rng.integers(0, max(1, t - k) + 1)) for t, k in zip(total, c)]
        chk += [int(k) for k in c]
    if rows:
        # contexts from a sixteenth of the longest to the longest, one of them the longest
        p = np.exp(rng.uniform(math.log(longest / 16), math.log(longest), size=rows)).astype(int)
        p[0] = longest
        pre += [int(x) - 1 for x in p]
        chk += [1] * rows
    order = rng.permutation(len(pre))
    return [pre[i] for i in order], [chk[i] for i in order]


# ---- inputs -------------------------------------------------------------------------------------------------------------------

def _paged(gen, pre, chk, page, every):
    """Block table into a pool a quarter larger than needed, in random order.  every = False: only the pages that the chunks touch
    have places of their own (the call touches no others)."""
    ends = [p + c for p, c in zip(pre, chk)]
    width = max(-(-e // page) for e in ends)
    need = [(r, j) for r, e in enumerate(ends) for j in range(0 if every else pre[r] // page, -(-e // page))]
    pool = len(need) + len(need) // 4 + 1
    place = torch.randperm(pool, generator=gen, device="cuda")[:len(need)].to(torch.int32)
    table = torch.zeros((len(ends), width), dtype=torch.int32, device="cuda")
    at = torch.tensor([r * width + j for r, j in need], dtype=torch.int64).to("cuda")
    table.view(-1)[at] = place
    return table, pool


def _frequencies(rot, longest):
    """Rotary frequencies, base 10000, interpolated between their own and a sixteenth for contexts past 65536 tokens."""
    i = np.arange(rot // 2, dtype=np.float64)
    f = 10000.0 ** (-2.0 * i / rot)
    if longest > 65536:
        f *= 1.0 - (1.0 - 1.0 / 16) * np.clip((i / (rot // 2) - 0.25) / 0.5, 0.0, 1.0)
    return torch.tensor(f, dtype=torch.float32, device="cuda")


def prepare(case, seed):
    pre, chk = lengths(case)
    tokens = sum(chk)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    s = dict(case=case, tokens=tokens, prefix_len=ints(pre), chunk_len=ints(chk), max_seq_len=max(p + c for p, c in zip(pre, chk)),
             status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    kind = case["kind"]
    if kind in ("rope", "append"):
        s["inv_freq"] = _frequencies(case["rot"], case["longest"])
    if kind == "rope":
        s["x"] = randn(tokens, case["heads"], case["dim"])
        # the rotated features stand behind others in a wider row
        s["out"] = torch.zeros((tokens, case["heads"], 4 * case["dim"]), dtype=torch.bfloat16, device="cuda")[..., 3 * case["dim"]:]
        return s
    hkv, page = case["hkv"], case["page"]
    s["table"], pool = _paged(gen, pre, chk, page, every=kind in ("select", "blocks"))
    if kind == "append":
        dim, hq = case["dim"], case["hq"]
        qkv = randn(tokens, hq + 2 * hkv, dim)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["q_out"] = torch.empty((tokens, hq, dim), dtype=torch.bfloat16, device="cuda")
        s["k_cache"], s["v_cache"] = randn(pool, page, hkv, dim), randn(pool, page, hkv, dim)
    elif kind == "means":
        s["k_cache"] = randn(pool, page, hkv, 128)
        s["k_cache"] += randn(pool, 1, hkv, 128)          # keys of a page resemble one another
        s["means"] = torch.zeros((pool, hkv, 128), dtype=torch.bfloat16, device="cuda")
    elif kind == "select":
        hq, group = case["hq"], case["hq"] // hkv
        s["means"] = randn(pool, hkv, 128)
        topic = randn(-(-tokens // 64), hkv, 1, 128).repeat_interleave(64, dim=0)[:tokens]   # neighbours ask for much the same
        s["q"] = (randn(tokens, hkv, group, 128) + topic).reshape(tokens, hq, 128)
        s["indices"] = torch.empty((tokens, hkv, case["topk"]), dtype=torch.int32, device="cuda")
    else:
        hq = case["hq"]
        s["q"] = randn(tokens, hq, 128)
        s["k_cache"], s["v_cache"] = randn(pool, page, hkv, 128), randn(pool, page, hkv, 128)
        s["out"] = torch.empty((tokens, hq, 128), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty((tokens, hq), dtype=torch.float32, device="cuda")
        # lists that neighbouring tokens mostly share, the first page and the own one always among them, as a selection gives them
        _, pos = _tokens(s)
        width, topk = s["table"].shape[1], case["topk"]
        score = torch.randn((-(-tokens // 64), hkv, width), generator=gen, device="cuda").repeat_interleave(64, dim=0)[:tokens]
        score = score + case["spread"] * torch.randn(score.shape, generator=gen, device="cuda")
        last = (pos // page)[:, None, None]
        b = torch.arange(width, device="cuda")
        score = torch.where((b == 0) | (b == last), math.inf, torch.where(b > last, -math.inf, score))
        got, idx = score.topk(min(topk, width), dim=-1)
        idx = torch.where(got == -math.inf, width, idx).sort(dim=-1).values
        lists = torch.full((tokens, hkv, topk), -1, dtype=torch.int32, device="cuda")
        lists[..., :idx.shape[-1]] = torch.where(idx == width, -1, idx).to(torch.int32)
        s["lists"] = lists
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------------------

def _tokens(s):
    """Request and position of every token of the packed chunk."""
    ends = s["chunk_len"].cumsum(0)
    t = torch.arange(s["tokens"], device="cuda")
    req = torch.searchsorted(ends, t, right=True)
    return req, s["prefix_len"][req] + t - (ends - s["chunk_len"])[req]


def _rotated(x, pos, inv_freq, case):
    """x [T, H, dim]: features offset .. offset + rot rotated by the angles pos * inv_freq, the others as they are."""
    angle = pos.double()[:, None] * inv_freq.double()          # (far positions: 32 bits would lose the angle)
    c = (angle.cos() * case["amplitude"]).float()[:, None]
    n = (angle.sin() * case["amplitude"]).float()[:, None]
    o, r = case["offset"], case["rot"]
    y = x.float().clone()
    part = x[..., o:o + r].float()
    if case["layout"] == HALF:
        a, b = part[..., :r // 2], part[..., r // 2:]
        y[..., o:o + r] = torch.cat([a * c - b * n, b * c + a * n], dim=-1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        y[..., o:o + r] = torch.stack([a * c - b * n, b * c + a * n], dim=-1).flatten(-2)
    return y.to(torch.bfloat16)


def _plain_append(s):
    case, page = s["case"], s["case"]["page"]
    req, pos = _tokens(s)
    block, slot = s["table"][req, pos // page].long(), pos % page
    s["k_cache"][block, slot] = _rotated(s["k_new"], pos, s["inv_freq"], case)
    s["v_cache"][block, slot] = s["v_new"]
    s["q_out"].copy_(_rotated(s["q"], pos, s["inv_freq"], case))


def _plain_means(s):
    page, table = s["case"]["page"], s["table"]
    j = torch.arange(table.shape[1], device="cuda")
    begin, end = s["prefix_len"][:, None], (s["prefix_len"] + s["chunk_len"])[:, None]
    done = ((j + 1) * page > begin) & ((j + 1) * page <= end)      # pages whose last position is in the chunk
    block = table[done].long()
    s["means"][block] = s["k_cache"][block].float().mean(dim=1).to(torch.bfloat16)


def _plain_select(s):
    case, table = s["case"], s["table"]
    page, topk, hkv, width = case["page"], case["topk"], case["hkv"], s["table"].shape[1]
    req, pos = _tokens(s)
    asks = s["q"].double().view(s["tokens"], hkv, -1, 128).sum(dim=2)     # (64 bits: which page comes last decides)
    every = torch.einsum("tgd,rbgd->tgrb", asks, s["means"][table.long()].double())
    score = every.gather(2, req[:, None, None, None].expand(-1, hkv, 1, width)).squeeze(2)
    last = (pos // page)[:, None, None]
    b = torch.arange(width, device="cuda")
    score = torch.where((b < case["first"]) | (b > last - case["last"]), math.inf, score)
    score = torch.where(b > last, -math.inf, score)
    got, idx = score.sort(dim=-1, descending=True, stable=True)         # (ties: the lowest index)
    idx = torch.where(got == -math.inf, width, idx)[..., :topk].sort(dim=-1).values
    s["indices"].fill_(-1)
    s["indices"][..., :idx.shape[-1]] = torch.where(idx == width, -1, idx).to(torch.int32)


def _plain_blocks(s):
    case, lists = s["case"], s["lists"].long()
    page, hkv, topk = case["page"], case["hkv"], case["topk"]
    req, pos = _tokens(s)
    pos = pos.long()[:, None, None]
    again = (lists[..., :, None] == lists[..., None, :]).tril(-1).any(-1)       # a page listed twice counts once
    take = (lists >= 0) & (lists <= pos // page) & ~again
    block = s["table"].long()[req[:, None, None], torch.where(take, lists, 0)]
    head = torch.arange(hkv, device="cuda")[None, :, None]
    k = s["k_cache"][block, :, head].flatten(2, 3).float()                      # [T, Hkv, topk * page, 128]
    q = s["q"].view(s["tokens"], hkv, -1, 128).float()
    score = torch.einsum("tghd,tgkd->tghk", q, k) / math.sqrt(128.0)
    del k
    at = lists[..., None] * page + torch.arange(page, device="cuda")
    seen = (take[..., None] & (at <= pos[..., None])).flatten(2)[:, :, None]
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(dim=-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    weight = (score - top).exp()
    total = weight.sum(dim=-1, keepdim=True)
    v = s["v_cache"][block, :, head].flatten(2, 3).float()
    out = torch.einsum("tghk,tgkd->tghd", weight, v) / torch.where(total == 0, 1.0, total)
    s["out"].copy_(out.flatten(1, 2))
    s["lse"].copy_((top + total.log()).flatten(1))


# ---- one pass -----------------------------------------------------------------------------------------------------------------

def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if own:
        from paper_2608_26523_b200 import api
        if kind == "rope":
            api.vpp_rope(s["x"], s["out"], s["prefix_len"], s["chunk_len"], s["inv_freq"], layout=case["layout"],
                         rot_offset=case["offset"], amplitude=case["amplitude"], status=s["status"])
        elif kind == "append":
            api.vpp_kv_append_rope(s["k_new"], s["v_new"], s["k_cache"], s["v_cache"], s["table"], s["prefix_len"], s["chunk_len"],
                                   case["page"], s["max_seq_len"], s["inv_freq"], q=s["q"], q_out=s["q_out"], layout=case["layout"],
                                   rot_offset=case["offset"], amplitude=case["amplitude"], status=s["status"])
        elif kind == "means":
            api.vpp_block_means(s["k_cache"], s["means"], s["table"], s["prefix_len"], s["chunk_len"], case["page"], s["tokens"],
                                status=s["status"])
        elif kind == "select":
            if "workspace" not in s:      # (laid out once, as a user's program does)
                n = api.vpp_block_select_workspace_size(s["tokens"], s["prefix_len"].numel(), case["hq"], case["hkv"], case["page"],
                                                        s["max_seq_len"])
                s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
            api.vpp_block_select(s["q"], s["means"], s["table"], s["prefix_len"], s["chunk_len"], case["page"], s["max_seq_len"],
                                 s["indices"], s["workspace"], num_first=case["first"], num_last=case["last"], status=s["status"])
        else:
            if "args" not in s:
                s["args"] = api.make_args(s["q"], s["k_cache"], s["v_cache"], s["table"], s["prefix_len"], s["chunk_len"], case["page"],
                                          s["max_seq_len"], 1.0 / math.sqrt(128.0), out=s["out"], lse=s["lse"], status=s["status"])
                s["workspace"] = torch.empty(api.vpp_block_attn_workspace_size(s["args"], case["topk"]), dtype=torch.uint8, device="cuda")
                s["args"].workspace, s["args"].workspace_bytes = s["workspace"].data_ptr(), s["workspace"].numel()
            api.vpp_block_attn_fwd(s["args"], s["lists"])
    elif kind == "rope":
        s["out"].copy_(_rotated(s["x"], _tokens(s)[1], s["inv_freq"], case))
    elif kind == "append":
        _plain_append(s)
    elif kind == "means":
        _plain_means(s)
    elif kind == "select":
        _plain_select(s)
    else:
        _plain_blocks(s)
    if kind == "rope":
        return s["out"]
    if kind == "append":
        return [s["q_out"], s["k_cache"], s["v_cache"]]
    return {"means": s.get("means")} if kind == "means" else {"indices": s["indices"]} if kind == "select" else [s["out"], s["lse"]]


def work(case):
    """What a call cannot do without: inputs read once, results written once; a multiplication and an addition each count."""
    pre, chk = lengths(case)
    tokens, kind = sum(chk), case["kind"]
    if kind == "rope":
        n = tokens * case["heads"]
        return {"bytes": 4 * n * case["dim"], "flops": 3 * n * case["rot"]}
    if kind == "append":
        n = tokens * (case["hq"] + case["hkv"])
        return {"bytes": 4 * (n + tokens * case["hkv"]) * case["dim"], "flops": 3 * n * case["rot"]}
    page, hkv = case["page"], case["hkv"]
    if kind == "means":
        done = sum((p + c) // page - p // page for p, c in zip(pre, chk))
        return {"bytes": max(1, done) * hkv * 256 * (page + 1), "flops": done * hkv * 128 * page}
    own_page = [np.arange(p, p + c) // page for p, c in zip(pre, chk)]
    if kind == "select":
        # every query once, the means of every page before the request's last one once; the heads of a kv-head add up first
        pages = sum(int(o[-1]) for o in own_page)
        pairs = sum(int(o.sum()) for o in own_page)
        return {"bytes": 256 * (tokens * case["hq"] + pages * hkv) + 4 * tokens * hkv * case["topk"],
                "flops": tokens * case["hq"] * 128 + 256 * hkv * pairs}
    topk, keys, pages = case["topk"], 0, 0
    for p, c, o in zip(pre, chk, own_page):
        pos = np.arange(p, p + c)
        keys += int(np.where(o < topk, pos + 1, (topk - 1) * page + pos % page + 1).sum())
        pages += min(int(o[-1]) + 1, min(topk, int(o[-1]) + 1) * -(-c // 64))      # neighbours' lists are mostly the same ones
    return {"bytes": tokens * case["hq"] * 516 + pages * page * hkv * 512 + 4 * tokens * hkv * topk, "flops": 512 * case["hq"] * keys}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------

def _by_hand(case):
    """(request, position, row) of every token, by walking over the requests."""
    pre, chk = lengths(case)
    return [(r, p + i) for r, (p, c) in enumerate(zip(pre, chk)) for i in range(c)]


def _turned(x, positions, inv_freq, case):
    """The rotation as a product of complex numbers."""
    y = x.double() * 1.0
    o, r = case["offset"], case["rot"]
    turns = torch.outer(torch.tensor(positions, dtype=torch.float64, device=x.device), inv_freq.double())
    unit = torch.polar(torch.full_like(turns, case["amplitude"]), turns)[:, None]
    p = y[..., o:o + r]
    pairs = (p.reshape(*p.shape[:-1], 2, r // 2).transpose(-1, -2) if case["layout"] == HALF else p.reshape(*p.shape[:-1], r // 2, 2)).contiguous()
    z = torch.view_as_real(torch.view_as_complex(pairs) * unit)
    y[..., o:o + r] = (z.transpose(-1, -2) if case["layout"] == HALF else z).reshape(p.shape)
    return y


def exact(case, seed):
    if case["kind"] == "select":
        return None                # (indices)
    s = prepare(case, seed)
    where = _by_hand(case)
    kind = case["kind"]
    if kind == "rope":
        return _turned(s["x"], [p for _, p in where], s["inv_freq"], case)
    page, table = case["page"], s["table"].cpu().numpy()
    pre, chk = lengths(case)
    if kind == "append":
        positions = [p for _, p in where]
        rows = torch.tensor([int(table[r, p // page]) * page + p % page for r, p in where], device="cuda")
        k, v = s["k_cache"].double(), s["v_cache"].double()
        k.view(-1, *k.shape[2:]).index_copy_(0, rows, _turned(s["k_new"], positions, s["inv_freq"], case))
        v.view(-1, *v.shape[2:]).index_copy_(0, rows, s["v_new"].double())
        return [_turned(s["q"], positions, s["inv_freq"], case), k, v]
    if kind == "means":
        means = s["means"].double()
        for r, (p, c) in enumerate(zip(pre, chk)):
            for j in range(p // page, (p + c) // page):
                b = int(table[r, j])
                means[b] = s["k_cache"][b].double().sum(0) / page
        return {"means": means}
    # every key of the context with a mask, a kv-head and a run of tokens at a time
    hq, hkv = case["hq"], case["hkv"]
    group, scale = hq // hkv, 128.0 ** -0.5
    out = torch.zeros((len(where), hq, 128), dtype=torch.float64, device="cuda")
    lse = torch.full((len(where), hq), -math.inf, dtype=torch.float64, device="cuda")
    t0 = 0
    for r, (p, c) in enumerate(zip(pre, chk)):
        used = -(-(p + c) // page)
        at = torch.tensor(table[r, :used], dtype=torch.int64, device="cuda")
        for g in range(hkv):
            keys = s["k_cache"][at, :, g].reshape(-1, 128).double()
            values = s["v_cache"][at, :, g].reshape(-1, 128).double()
            step = max(1, (1 << 28) // (keys.shape[0] * group))
            for a in range(0, c, step):
                b = min(c, a + step)
                lists = s["lists"][t0 + a:t0 + b, g].long()
                pages = torch.zeros((b - a, used + 1), dtype=torch.bool, device="cuda")
                pages.scatter_(1, torch.where((lists < 0) | (lists >= used), used, lists), True)
                pos = torch.arange(p + a, p + b, device="cuda")
                seen = pages[:, :used].repeat_interleave(page, dim=1) & (torch.arange(used * page, device="cuda")[None] <= pos[:, None])
                q = s["q"][t0 + a:t0 + b, g * group:(g + 1) * group].double()
                score = (q.reshape(-1, 128) @ keys.T).mul_(scale).view(b - a, group, -1).masked_fill_(~seen[:, None], -math.inf)
                total = score.logsumexp(dim=-1, keepdim=True)
                lse[t0 + a:t0 + b, g * group:(g + 1) * group] = total[..., 0]
                weight = score.sub_(torch.where(total == -math.inf, 0.0, total)).exp_()
                # (a slot past the end holds no key: its weight is zero)
                out[t0 + a:t0 + b, g * group:(g + 1) * group] = (weight.view(-1, keys.shape[0]) @ values).view(b - a, group, 128)
        t0 += c
    return [out, lse]
