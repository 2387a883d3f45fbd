"""Measured cases of the operators that read less of a long paged cache than the verify attention does: bounds of every
page's keys, selection of pages by a score on these bounds, attention over the selected pages, and attention of a batch
whose sequences share a long prefix.

``own = False`` runs the plain form (elementary torch operations), ``own = True`` the library's entry points."""
import math

import torch

own = False

DEV = "cuda"
PAGE = 16


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one sequence's draft block behind its context, 64-dim heads: nothing but latency
        dict(name="bounds_single", op="bounds", batch=1, hkv=12, dim=64, ctx_lo=133, ctx_hi=133, new=5),
        # prompts admitted, every page of them new, the last ones partly filled
        dict(name="bounds_prompt", op="bounds", batch=16, hkv=8, dim=128, ctx_lo=7000, ctx_hi=8192, new=8192),
        # a single token of one long conversation
        dict(name="select_single", op="select", batch=1, hkv=8, group=4, dim=128, ctx_lo=32768, ctx_hi=32768, gamma_max=0, n_select=64, n_first=1, n_last=8),
        # a verify step of ragged blocks
        dict(name="select_verify", op="select", batch=16, hkv=8, group=4, dim=128, ctx_lo=1024, ctx_hi=8192, gamma_max=10, n_select=32, n_first=1, n_last=2),
        # the largest verify step: 17 rows of 64 heads for each of 128 sequences
        dict(name="select_batch", op="select", batch=128, hkv=8, group=8, dim=128, ctx_lo=512, ctx_hi=16384, gamma_max=16, n_select=64, n_first=1, n_last=4),
        # a single token over 64 selected pages
        dict(name="pages_single", op="pages", batch=1, hkv=8, group=4, dim=128, ctx_lo=32768, ctx_hi=32768, gamma_max=0, n_select=64, n_first=1, n_last=8),
        # heads that share no keys, blocks of up to 13 rows
        dict(name="pages_mha", op="pages", batch=64, hkv=40, group=1, dim=128, ctx_lo=4096, ctx_hi=4096, gamma_max=12, n_select=32, n_first=1, n_last=2),
        # a decoding batch, single tokens
        dict(name="pages_decode", op="pages", batch=128, hkv=8, group=8, dim=128, ctx_lo=512, ctx_hi=16384, gamma_max=0, n_select=128, n_first=1, n_last=8),
        # the largest verify step, each row with its own pages
        dict(name="pages_verify", op="pages", batch=128, hkv=8, group=8, dim=128, ctx_lo=512, ctx_hi=16384, gamma_max=16, n_select=64, n_first=1, n_last=4),
        # two requests behind one system prompt, a small draft-sized model
        dict(name="prefix_small", op="prefix", batch=2, hkv=12, group=1, dim=64, prefix=2048, groups=1, tail=100, gamma_max=4),
        # many samples of one long prompt, single tokens
        dict(name="prefix_decode", op="prefix", batch=64, hkv=8, group=4, dim=128, prefix=8192, groups=1, tail=1024, gamma_max=0),
        # a large batch over three long documents (some requests over none of them), verify blocks
        dict(name="prefix_verify", op="prefix", batch=128, hkv=8, group=8, dim=128, prefix=12000, groups=3, tail=2048, gamma_max=16),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["bounds", "select", "select", "pages", "pages", "prefix", "prefix"])
    hkv = rng.choice([1, 2, 4, 8, 12])
    dim = rng.choice([64, 128, 128])
    if op == "bounds":
        batch = _log(rng, 1, 128)
        hi = _log(rng, 20, min(16384, 131072 // batch))
        return dict(op=op, batch=batch, hkv=min(hkv, 8), dim=dim, ctx_lo=_log(rng, 1, hi), ctx_hi=hi, new=rng.choice([1, rng.randint(1, 17), hi]))
    group = rng.choice([1, 2, 3, 4, 7, 8])
    gamma_max = rng.choice([0, 0, rng.randint(1, 16), rng.randint(1, 16)])
    if op == "prefix":
        batch = _log(rng, 2, 128)
        return dict(op=op, batch=batch, hkv=min(hkv, 8), group=group, dim=dim, prefix=_log(rng, 40, 12000), groups=rng.randint(1, 4),
                    tail=_log(rng, 20, 2048), gamma_max=gamma_max)
    batch = _log(rng, 1, 128)
    hi = _log(rng, 100, min(65536, 1081344 // batch))
    first, last = rng.choice([0, 1, 4]), rng.choice([1, 2, 8])
    return dict(op=op, batch=batch, hkv=min(hkv, 8), group=group, dim=dim, ctx_lo=max(20, hi // rng.choice([1, 2, 16])), ctx_hi=hi, gamma_max=gamma_max,
                n_select=_log(rng, first + last, 128), n_first=first, n_last=last)


# ------------------------------------------------------------------------------------------------ inputs
class _Gen:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, shape, std=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=self.g, device=DEV, dtype=dtype) * std).to(dtype)

    def uniform(self, shape, lo=0.0, hi=1.0):
        return torch.rand(shape, generator=self.g, device=DEV) * (hi - lo) + lo

    def ints(self, lo, hi, shape):                             # lo <= x < hi
        return torch.randint(int(lo), int(hi), shape, generator=self.g, device=DEV, dtype=torch.int64).to(torch.int32)

    def perm(self, n):
        return torch.randperm(n, generator=self.g, device=DEV).to(torch.int32)


def _prefix(n):
    out = torch.zeros(n.numel() + 1, dtype=torch.int32, device=n.device)
    out[1:] = torch.cumsum(n, 0).to(torch.int32)
    return out


def _table(g, lengths, most, shared=None):
    """Block table of sequences of `lengths` tokens (`most` at most) over pages in any order; shared = (group of each
    sequence, pages of each group's prefix)."""
    need = (lengths.long() + PAGE - 1) // PAGE
    stride = (most + PAGE - 1) // PAGE
    col = torch.arange(stride, device=DEV)
    owned, base = need, 0
    if shared is not None:
        group, pages = shared
        mine = torch.where(group >= 0, pages[group.clamp(min=0)], torch.zeros_like(need))
        owned, base = need - mine, int(pages.sum())
    n_pages = (int(owned.sum()) if shared is not None else len(need) * stride) + base + 3
    ids = g.perm(n_pages)
    at = base + (torch.cumsum(owned, 0) - owned)[:, None] + col
    if shared is not None:
        first = (torch.cumsum(pages, 0) - pages)[group.clamp(min=0)]
        at = torch.where(col < mine[:, None], first[:, None] + col, at - mine[:, None])
    table = torch.where(col < need[:, None], ids[at.clamp(max=n_pages - 1)], torch.full_like(at, -1, dtype=torch.int32))
    return table.to(torch.int32).contiguous(), n_pages


def prepare(case, seed):
    return {"bounds": _prepare_bounds, "select": _prepare_select, "pages": _prepare_pages, "prefix": _prepare_prefix}[case["op"]](case, _Gen(seed))


def _keys(g, n_pages, hkv, dim):
    """Keys as rotated projections have them: some channels much larger than others, neighbours in a page alike."""
    k = g.normal((n_pages, hkv, PAGE, dim), 0.7, torch.bfloat16)
    k += g.normal((n_pages, hkv, 1, dim), 0.7, torch.bfloat16)
    k *= (0.5 + g.uniform((1, hkv, 1, dim)) ** 4 * 3.0).to(torch.bfloat16)
    return k


def _rows(c, g, lengths):
    B, gmax = c["batch"], c["gamma_max"]
    gamma = torch.minimum(g.ints(0, gmax + 1, (B,)) if B < 100 else torch.full((B,), gmax, dtype=torch.int32, device=DEV), lengths - 1)
    return gamma, _prefix(gamma + 1)


def _prepare_bounds(c, g):
    B, hkv, D = c["batch"], c["hkv"], c["dim"]
    lengths = g.ints(c["ctx_lo"], c["ctx_hi"] + 1, (B,))
    table, n_pages = _table(g, lengths, c["ctx_hi"])
    k = _keys(g, n_pages, hkv, D)
    s = dict(op="bounds", k=k, table=table, lengths=lengths, first=torch.clamp(lengths - c["new"], min=0), new=c["new"],
             bounds=torch.zeros((n_pages, hkv, 2, D), dtype=torch.int8, device=DEV), scales=torch.zeros((n_pages, hkv), device=DEV), pool=None)
    if own:
        from paper_2504_00030_b200 import binding as sv
        s["pool"] = sv.spec_kv_pool_register(k, k)               # the values play no part
    return s


def _prepare_select(c, g):
    B, hkv, D, gmax = c["batch"], c["hkv"], c["dim"], c["gamma_max"]
    lengths = g.ints(c["ctx_lo"], c["ctx_hi"] + 1, (B,))
    gamma, cu_q = _rows(c, g, lengths)
    table, n_pages = _table(g, lengths, c["ctx_hi"])
    lo, hi = g.ints(-127, 128, (n_pages, hkv, 1, D)), g.ints(-127, 128, (n_pages, hkv, 1, D))
    bounds = torch.cat((torch.maximum(lo, hi), torch.minimum(lo, hi)), 2).to(torch.int8).contiguous()
    width = min(table.shape[1], (gmax + 1) * c["n_select"])
    s = dict(op="select", q=g.normal((B * (gmax + 1), hkv * c["group"], D), 1.0, torch.bfloat16), bounds=bounds, scales=g.uniform((n_pages, hkv), 0.01, 0.03),
             table=table, lengths=lengths, gamma=gamma, cu_q=cu_q, gamma_max=gmax, most=c["ctx_hi"], n_select=c["n_select"], n_first=c["n_first"],
             n_last=c["n_last"], page_list=torch.full((B, hkv, width), -1, dtype=torch.int32, device=DEV),
             row_mask=torch.zeros((B, hkv, width), dtype=torch.int64, device=DEV), n_list=torch.zeros((B, hkv), dtype=torch.int32, device=DEV), workspace=None)
    if own:
        from paper_2504_00030_b200 import binding as sv
        s["workspace"] = torch.empty(sv.spec_page_select_workspace_bytes(B, gmax, hkv, c["ctx_hi"]), dtype=torch.uint8, device=DEV)
    return s


def _attention_inputs(c, g, lengths, most, shared=None):
    B, hkv, hq, D, gmax = c["batch"], c["hkv"], c["hkv"] * c["group"], c["dim"], c["gamma_max"]
    gamma, cu_q = _rows(c, g, lengths)
    table, n_pages = _table(g, lengths, most, shared)
    q = g.normal((B * (gmax + 1), hq, D), 1.5, torch.bfloat16)
    s = dict(op=c["op"], q=q, o=torch.zeros_like(q), lse=torch.zeros((B * (gmax + 1), hq), device=DEV), k=g.normal((n_pages, hkv, PAGE, D), 1.0, torch.bfloat16),
             v=g.normal((n_pages, hkv, PAGE, D), 1.0, torch.bfloat16), table=table, lengths=lengths, gamma=gamma, cu_q=cu_q, gamma_max=gmax, pool=None, workspace=None, most=most)
    if own:
        from paper_2504_00030_b200 import binding as sv
        s["pool"] = sv.spec_kv_pool_register(s["k"], s["v"])
    return s


def _prepare_pages(c, g):
    B, hkv, gmax = c["batch"], c["hkv"], c["gamma_max"]
    lengths = g.ints(c["ctx_lo"], c["ctx_hi"] + 1, (B,))
    s = _attention_inputs(c, g, lengths, c["ctx_hi"])
    P, R = s["table"].shape[1], gmax + 1
    width = min(P, R * c["n_select"])
    page_list = torch.full((B, hkv, width), -1, dtype=torch.int32, device=DEV)
    row_mask = torch.zeros((B, hkv, width), dtype=torch.int64, device=DEV)
    n_list = torch.zeros((B, hkv), dtype=torch.int32, device=DEV)
    page, row = torch.arange(P, device=DEV), torch.arange(R, device=DEV)
    power = (2 ** row.long())[:, None]
    for b0 in range(0, B, 16):                                   # neighbouring rows of a block look for much the same pages
        sl = slice(b0, min(B, b0 + 16))
        score = g.uniform((sl.stop - sl.start, hkv, 1, P)) + 0.1 * g.uniform((sl.stop - sl.start, hkv, R, P))
        last = ((lengths[sl].long() - 1 - s["gamma"][sl].long())[:, None] + row).div(PAGE, rounding_mode="floor")[:, None, :, None]
        score = torch.where((page < c["n_first"]) | (page > last - c["n_last"]), 2.0 + score, score)
        score = torch.where((page <= last) & (row[:, None] <= s["gamma"][sl][:, None, None, None]), score, torch.full_like(score, -1.0))
        top = torch.topk(score, min(P, c["n_select"]), dim=-1)
        chosen = torch.zeros(score.shape, dtype=torch.bool, device=DEV).scatter_(3, top.indices, top.values >= 0)
        mask = (chosen.long() * power).sum(2)
        n = (mask != 0).sum(-1)
        order = torch.argsort((mask == 0).to(torch.int8), dim=-1, stable=True)[..., :width]
        use = torch.arange(width, device=DEV) < n[..., None]
        page_list[sl] = torch.where(use, order, torch.full_like(order, -1)).to(torch.int32)
        row_mask[sl] = torch.where(use, torch.gather(mask, 2, order), torch.zeros_like(order))
        n_list[sl] = n.to(torch.int32)
    s.update(page_list=page_list, row_mask=row_mask, n_list=n_list)
    if own:
        from paper_2504_00030_b200 import binding as sv
        s["workspace"] = torch.empty(sv.spec_verify_attn_pages_workspace_bytes(B, gmax, s["q"].shape[1], hkv, c["dim"]), dtype=torch.uint8, device=DEV)
    return s


def _prepare_prefix(c, g):
    B, G = c["batch"], c["groups"]
    length = g.ints(max(1, c["prefix"] // 2), c["prefix"] + 1, (G,)) if G > 1 else torch.full((1,), c["prefix"], dtype=torch.int32, device=DEV)
    group = g.ints(0, G, (B,)) if G == 1 else g.ints(-1, G, (B,))           # with several prefixes some requests have none
    pages = length.long() // PAGE
    mine = torch.where(group >= 0, pages[group.long().clamp(min=0)] * PAGE, torch.zeros(B, dtype=torch.int64, device=DEV))
    lengths = (mine + c["gamma_max"] + g.ints(1, c["tail"] + 1, (B,))).to(torch.int32)
    most = c["prefix"] + c["gamma_max"] + c["tail"]
    s = _attention_inputs(c, g, lengths, most, (group.long(), pages))
    s.update(group=group, prefix_len=length)
    if own:
        from paper_2504_00030_b200 import binding as sv
        s["workspace"] = torch.empty(sv.spec_verify_attn_prefix_workspace_bytes(B, c["gamma_max"], s["q"].shape[1], c["hkv"], c["dim"], G), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return {"bounds": _run_bounds, "select": _run_select, "pages": _run_pages, "prefix": _run_prefix}[s["op"]](s)


def _run_bounds(s):
    if own:
        from paper_2504_00030_b200 import binding as sv
        sv.spec_page_bounds_update(s["pool"], s["bounds"], s["scales"], s["table"], s["lengths"], first=s["first"], max_new=s["new"])
    else:
        col = torch.arange(s["table"].shape[1], device=DEV)
        seq, page = torch.nonzero((col >= s["first"][:, None] // PAGE) & (col * PAGE < s["lengths"][:, None]), as_tuple=True)
        at = s["table"][seq, page].long()
        filled = (s["lengths"][seq] - page * PAGE)[:, None, None, None] > torch.arange(PAGE, device=DEV)[:, None]
        k = s["k"][at].float()
        high = torch.where(filled, k, torch.full_like(k, -math.inf)).amax(2)
        low = torch.where(filled, k, torch.full_like(k, math.inf)).amin(2)
        both = torch.stack((high, low), 2)
        scale = both.abs().amax((2, 3)) / 127.0
        whole = torch.where(scale[..., None, None] > 0, both / scale[..., None, None], torch.zeros_like(both))
        s["bounds"][at] = torch.clamp(torch.round(whole), -127, 127).to(torch.int8)
        s["scales"][at] = scale
    return {"bounds": s["bounds"], "scales": s["scales"]}


def _run_select(s):
    if own:
        from paper_2504_00030_b200 import binding as sv
        sv.spec_page_select(s["q"], s["bounds"], s["scales"], s["table"], s["lengths"], s["gamma"], s["cu_q"], s["gamma_max"], s["most"], s["n_select"],
                            s["n_first"], s["n_last"], s["page_list"], s["row_mask"], s["n_list"], s["workspace"])
    else:
        hkv, D = s["bounds"].shape[1], s["bounds"].shape[3]
        length, gamma, cu = s["lengths"].tolist(), s["gamma"].tolist(), s["cu_q"].tolist()
        for b in range(len(length)):
            R, P = gamma[b] + 1, (length[b] + PAGE - 1) // PAGE
            at = s["table"][b, :P].long()
            q = s["q"][cu[b]:cu[b] + R].float().unflatten(1, (hkv, -1))                       # [rows, kv head, head of the group, dim]
            scale = q.abs().amax((2, 3), keepdim=True) / 127.0
            q = torch.where(scale > 0, torch.clamp(torch.round(q / scale), -127, 127), torch.zeros_like(q)).permute(1, 0, 2, 3).flatten(1, 2)
            both = s["bounds"][at].float().permute(1, 2, 3, 0)                                # [kv head, max / min, dim, page]
            n = torch.clamp(q, min=0) @ both[:, 0] + torch.clamp(q, max=0) @ both[:, 1]       # whole numbers below 2^24
            score = n.unflatten(1, (R, -1)).amax(2) * s["scales"][at].t()[:, None]
            page = torch.arange(P, device=DEV)
            last = ((length[b] - R + torch.arange(R, device=DEV)) // PAGE)[:, None]
            score = torch.where((page < s["n_first"]) | (page > last - s["n_last"]), torch.full_like(score, math.inf), score)
            score = torch.where(page <= last, score, torch.full_like(score, -math.inf))
            order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :s["n_select"]]
            chosen = torch.zeros(score.shape, dtype=torch.bool, device=DEV).scatter_(2, order, True) & (page <= last)
            mask = (chosen.long() * (2 ** torch.arange(R, device=DEV))[:, None]).sum(1)
            count = (mask != 0).sum(-1)
            head, page = torch.nonzero(mask, as_tuple=True)
            place = torch.arange(page.numel(), device=DEV) - (torch.cumsum(count, 0) - count)[head]
            s["page_list"][b, head, place] = page.to(torch.int32)
            s["row_mask"][b, head, place] = mask[head, page]
            s["n_list"][b] = count.to(torch.int32)
    return {k: s[k] for k in ("page_list", "row_mask", "n_list")}


def _plain_softmax(s, b, rows, q, k, v, seen):
    """Rows of one sequence: q [kv head, rows * group, dim], k and v [kv head, keys, dim], seen [kv head or 1, rows, keys]."""
    hkv, _, D = q.shape
    score = (q @ k.transpose(1, 2)).unflatten(1, (rows.stop - rows.start, -1)) * D ** -0.5
    score = torch.where(seen[:, :, None], score, torch.full_like(score, -math.inf))
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = weight.sum(-1, keepdim=True)
    o = (weight.flatten(1, 2) @ v).unflatten(1, (rows.stop - rows.start, -1)) / torch.where(total > 0, total, torch.ones_like(total))
    s["o"][rows] = o.permute(1, 0, 2, 3).flatten(1, 2).to(torch.bfloat16)
    s["lse"][rows] = (torch.log(total) + top).squeeze(-1).permute(1, 0, 2).flatten(1)


def _run_pages(s):
    if own:
        from paper_2504_00030_b200 import binding as sv
        sv.spec_verify_attn_pages(s["q"], s["o"], s["pool"], s["table"], s["lengths"], s["gamma"], s["cu_q"], s["gamma_max"], s["most"], s["page_list"],
                                  s["row_mask"], s["n_list"], s["workspace"], lse=s["lse"])
    else:
        hkv = s["k"].shape[1]
        head, slot = torch.arange(hkv, device=DEV)[:, None], torch.arange(PAGE, device=DEV)
        length, gamma, cu, most = s["lengths"].tolist(), s["gamma"].tolist(), s["cu_q"].tolist(), s["n_list"].amax(1).tolist()
        for b in range(len(length)):
            R, n = gamma[b] + 1, most[b]
            rows = slice(cu[b], cu[b] + R)
            page = s["page_list"][b, :, :n].long()
            listed = torch.arange(n, device=DEV) < s["n_list"][b][:, None]
            page = torch.where(listed, page, torch.zeros_like(page))
            at = s["table"][b].long()[page]
            row = torch.arange(R, device=DEV)
            chosen = listed[:, None] & (((s["row_mask"][b, :, :n][:, None] >> row[:, None]) & 1) == 1)         # [kv head, rows, listed page]
            key = (page[:, :, None] * PAGE + slot).flatten(1)
            seen = chosen.repeat_interleave(PAGE, 2) & (key[:, None] <= length[b] - R + row[:, None])
            q = s["q"][rows].float().unflatten(1, (hkv, -1)).permute(1, 0, 2, 3).flatten(1, 2)
            _plain_softmax(s, b, rows, q, s["k"][at, head].float().flatten(1, 2), s["v"][at, head].float().flatten(1, 2), seen)
    return {"o": s["o"], "lse": s["lse"]}


def _run_prefix(s):
    if own:
        from paper_2504_00030_b200 import binding as sv
        sv.spec_verify_attn_prefix(s["q"], s["o"], s["pool"], s["table"], s["lengths"], s["gamma"], s["cu_q"], s["gamma_max"], s["most"], s["group"],
                                   s["prefix_len"], s["workspace"], lse=s["lse"])
    else:
        hkv = s["k"].shape[1]
        length, gamma, cu = s["lengths"].tolist(), s["gamma"].tolist(), s["cu_q"].tolist()
        for b in range(len(length)):
            R = gamma[b] + 1
            rows = slice(cu[b], cu[b] + R)
            at = s["table"][b, :(length[b] + PAGE - 1) // PAGE].long()
            k, v = (s[x][at].float().transpose(0, 1).flatten(1, 2) for x in ("k", "v"))
            seen = torch.arange(k.shape[1], device=DEV) <= (length[b] - R + torch.arange(R, device=DEV))[:, None]
            q = s["q"][rows].float().unflatten(1, (hkv, -1)).permute(1, 0, 2, 3).flatten(1, 2)
            _plain_softmax(s, b, rows, q, k, v, seen[None])
    return {"o": s["o"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(c):
    B, hkv, D = c["batch"], c["hkv"], c["dim"]
    if c["op"] == "bounds":
        keys = min(c["new"], (c["ctx_lo"] + c["ctx_hi"]) / 2)
        pages = keys / PAGE + (PAGE - 1) / PAGE                          # a page in part is read up to its last key
        return {"bytes": B * hkv * ((keys + (PAGE - 1) / 2) * D * 2 + pages * (2 * D + 4)), "flops": B * hkv * D * (2 * keys + 4 * pages)}
    hq = hkv * c["group"]
    rows = B * (c["gamma_max"] + 1 if B >= 100 else c["gamma_max"] / 2 + 1)
    if c["op"] == "prefix":
        member = 1 if c["groups"] == 1 else c["groups"] / (c["groups"] + 1)
        length = c["prefix"] if c["groups"] == 1 else 0.75 * c["prefix"]
        held = c["groups"] * length + B * (c["tail"] / 2 + c["gamma_max"])            # tokens of the cache, each once
        seen = rows * (member * length + c["tail"] / 2 + c["gamma_max"] / 2)
        return {"bytes": held * hkv * D * 4 + rows * hq * (D * 4 + 4), "flops": 4.0 * seen * hq * D}
    pages = (c["ctx_lo"] + c["ctx_hi"]) / 2 / PAGE
    each = min(c["n_select"], pages)
    union = min(pages, each * (1 + 0.05 * rows / B))
    if c["op"] == "select":
        return {"bytes": B * hkv * (pages * (2 * D + 4) + union * 12) + rows * hq * D * 2 + B * pages * 4, "flops": 4.0 * rows * hq * pages * D}
    return {"bytes": B * hkv * union * (PAGE * D * 4 + 12) + rows * hq * (D * 4 + 4), "flops": 4.0 * rows * hq * each * PAGE * D}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    if case["op"] == "select":
        return None                                                      # whole numbers: equal or wrong
    s = prepare(case, seed)
    if case["op"] == "bounds":
        return {"bounds": None, "scales": _exact_scales(s)}
    o, lse = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEV), torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    for b, (length, gamma, first) in enumerate(zip(s["lengths"].tolist(), s["gamma"].tolist(), s["cu_q"].tolist())):
        _exact_sequence(s, b, length, gamma, first, o, lse)
    return {"o": o, "lse": lse}


def _exact_scales(s):
    out = s["scales"].double()
    for b, (length, first) in enumerate(zip(s["lengths"].tolist(), s["first"].tolist())):
        lo, hi = first // PAGE, (length + PAGE - 1) // PAGE
        at = s["table"][b, lo:hi].long()
        size = s["k"][at].double().abs().amax(-1)                        # [page, kv head, slot]
        size[-1, :, length - (hi - 1) * PAGE:] = 0
        out[at] = size.amax(-1) / 127
    return out


def _exact_sequence(s, b, length, gamma, first, o, lse):
    """Row by row and kv head by kv head over the keys that the row sees."""
    hkv = s["k"].shape[1]
    group, D = s["q"].shape[1] // hkv, s["q"].shape[2]
    token = torch.arange(length, device=DEV)
    at, slot = s["table"][b, :(length + PAGE - 1) // PAGE].long()[token // PAGE], token % PAGE
    for h in range(hkv):
        mine = slice(h * group, (h + 1) * group)
        visible = token <= length - 1 - gamma + torch.arange(gamma + 1, device=DEV)[:, None]
        pick = token
        if s["op"] == "pages":
            n = int(s["n_list"][b, h])
            mask = torch.zeros(s["table"].shape[1], dtype=torch.int64, device=DEV)
            mask[s["page_list"][b, h, :n].long()] = s["row_mask"][b, h, :n]
            pick = token[(mask != 0)[token // PAGE]]                     # tokens of any listed page
            bit = torch.bitwise_right_shift(mask[pick // PAGE], torch.arange(gamma + 1, device=DEV)[:, None])
            visible = visible[:, pick] & (bit % 2 != 0)
        k, v = s["k"][at[pick], h, slot[pick]].double(), s["v"][at[pick], h, slot[pick]].double()
        score = torch.einsum("rgd,kd->rgk", s["q"][first:first + gamma + 1, mine].double(), k) / math.sqrt(D)
        score = score.masked_fill(~visible[:, None], -math.inf)
        lse[first:first + gamma + 1, mine] = torch.logsumexp(score, -1)
        o[first:first + gamma + 1, mine] = torch.einsum("rgk,kd->rgd", torch.softmax(score, -1), v)
