"""Measured cases of the operators around the verify step: page tables and slot maps on the device, query / key norm with
rotation and cache append, penalties / biases / grammar masks on logits, and the token counts that the penalties read.

``own = False`` runs the plain form (elementary torch operations), ``own = True`` the library's entry points."""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
PAGE = 16


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one request being decoded with a short draft block: nothing but latency
        dict(name="pages_single", op="pages", batch=1, ctx_lo=2048, ctx_hi=2048, gamma_max=8, retire=0.0),
        # a decoding batch with long contexts: every sequence moves by a block, a few pages change hands
        dict(name="pages_decode", op="pages", batch=128, ctx_lo=512, ctx_hi=16384, gamma_max=16, retire=0.0),
        # a large batch of which half is retired and as many prompts are admitted
        dict(name="pages_admit", op="pages", batch=1024, ctx_lo=64, ctx_hi=16384, gamma_max=4, retire=0.5),
        # one small sequence without norms, 64-dim heads
        dict(name="rope_single", op="rope", rows=5, hq=12, hkv=12, dim=64, rot=64, norm=False, interleaved=False, axes=1, far=2048, pad=0.0),
        # one layer of a verify step, grouped heads with query / key norms, ragged blocks in fixed row slabs
        dict(name="rope_verify", op="rope", rows=176, hq=32, hkv=8, dim=128, rot=128, norm=True, interleaved=False, axes=1, far=8192, pad=0.3),
        # one layer of the largest verify step
        dict(name="rope_batch", op="rope", rows=2176, hq=64, hkv=8, dim=128, rot=128, norm=True, interleaved=False, axes=1, far=16384, pad=0.0),
        # prompts of a model for images and video: three position axes, half of the dims rotated in neighbouring pairs, far positions
        dict(name="rope_prompt", op="rope", rows=16381, hq=32, hkv=8, dim=128, rot=64, norm=True, interleaved=True, axes=3, far=1000000, pad=0.0),
        # one sequence's verify rows
        dict(name="logits_single", op="logits", batch=1, gamma_max=4, vocab=32000, bf16=False, penal=True, bias=16, mask=False, draft=False, inplace=False),
        # a drafting step under a grammar: one row per sequence, masked in place
        dict(name="logits_draft", op="logits", batch=64, gamma_max=12, vocab=128256, bf16=True, penal=False, bias=0, mask=True, draft=True, inplace=True),
        # all verify rows of the largest step, penalties, biases and grammar masks together
        dict(name="logits_verify", op="logits", batch=128, gamma_max=16, vocab=128256, bf16=False, penal=True, bias=300, mask=True, draft=False, inplace=False),
        # the tokens that an accept call emitted
        dict(name="counts_step", op="counts", batch=128, vocab=128256, tokens=17, admit=False),
        # prompts of a newly admitted batch (rows cleared, prompt tokens marked)
        dict(name="counts_admit", op="counts", batch=128, vocab=128256, tokens=8192, admit=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["pages", "rope", "rope", "logits", "logits", "counts"])
    if op == "pages":
        lo = _log(rng, 40, 2048)
        return dict(op=op, batch=_log(rng, 1, 1024), ctx_lo=lo, ctx_hi=_log(rng, lo, 16384), gamma_max=rng.randint(0, 16),
                    retire=rng.choice([0.0, 0.25, 0.5]))
    if op == "rope":
        hkv = rng.choice([1, 2, 4, 8, 12])
        hq = hkv * rng.choice([1, 2, 3, 4])
        dim = rng.choice([64, 96, 128, 128])
        rot = rng.choice([dim, dim, dim // 2, 32])
        return dict(op=op, rows=_log(rng, 1, 16381), hq=hq, hkv=hkv, dim=dim, rot=rot, norm=rng.random() < 0.7,
                    interleaved=rng.random() < 0.3, axes=rng.choice([1, 1, 3]), far=_log(rng, 128, 1000000),
                    pad=rng.choice([0.0, 0.3]))
    if op == "logits":
        draft = rng.random() < 0.3
        inplace = rng.random() < 0.3
        return dict(op=op, batch=_log(rng, 1, 100), gamma_max=rng.randint(0, 16), vocab=rng.choice([4099, 32000, 50257, 128256, rng.randint(1000, 128256)]),
                    bf16=rng.random() < 0.5, penal=not inplace, bias=0 if inplace else rng.choice([0, 0, 5, 300]), mask=inplace or rng.random() < 0.5,
                    draft=draft, inplace=inplace)
    admit = rng.random() < 0.5
    return dict(op=op, batch=_log(rng, 1, 128), vocab=rng.choice([4099, 32000, 50257, 128256, rng.randint(1000, 128256)]),
                tokens=_log(rng, 1, 8192) if admit else rng.randint(1, 65), admit=admit)


# ------------------------------------------------------------------------------------------------ inputs
class _Gen:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, shape, std=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=self.g, device=DEV) * std).to(dtype)

    def uniform(self, shape, lo=0.0, hi=1.0, dtype=torch.float32):
        return torch.rand(shape, generator=self.g, device=DEV, dtype=dtype) * (hi - lo) + lo

    def ints(self, lo, hi, shape, dtype=torch.int32):          # lo <= x < hi
        return torch.randint(int(lo), int(hi), shape, generator=self.g, device=DEV, dtype=torch.int64).to(dtype)

    def perm(self, n):
        return torch.randperm(n, generator=self.g, device=DEV).to(torch.int32)


def _prefix(n):
    out = torch.zeros(n.numel() + 1, dtype=torch.int32, device=n.device)
    out[1:] = torch.cumsum(n, 0).to(torch.int32)
    return out


def _skewed_tokens(g, shape, vocab):
    """Token ids as text has them: few of them often, many rarely."""
    return torch.clamp((g.uniform(shape) ** 4 * vocab).to(torch.int32), max=vocab - 1)


def prepare(case, seed):
    g = _Gen(seed)
    return {"pages": _prepare_pages, "rope": _prepare_rope, "logits": _prepare_logits, "counts": _prepare_counts}[case["op"]](case, g)


def _prepare_pages(c, g):
    B, gmax = c["batch"], c["gamma_max"]
    len_b = g.ints(c["ctx_lo"], c["ctx_hi"] + 1, (B,))                   # where a pass ends (and where the first begins)
    move = g.ints(-gmax, gmax + 2, (B,))                                 # a block further, or a shorter block
    len_a = torch.clamp(len_b + move, min=gmax + 1).to(torch.int32)
    len_a = torch.where(g.uniform((B,)) < c["retire"], torch.zeros_like(len_a), len_a)
    len_b = torch.clamp(len_b, min=gmax + 1).to(torch.int32)
    gamma_a, gamma_b = g.ints(0, gmax + 1, (B,)), g.ints(0, gmax + 1, (B,))
    stride = (c["ctx_hi"] + 2 * gmax + 2 + PAGE - 1) // PAGE + 1
    n_rows = B * (gmax + 1)
    held = (len_b + PAGE - 1) // PAGE
    # every sequence could grow by its block at once
    n_pages = B * ((c["ctx_lo"] + c["ctx_hi"]) // (2 * PAGE) + 4) + B * (c["ctx_hi"] - c["ctx_lo"]) // (2 * PAGE)
    ids = g.perm(n_pages)
    col = torch.arange(stride, device=DEV)
    first = torch.cumsum(held, 0) - held
    used = first[:, None] + col
    table = torch.where(col < held[:, None], ids[torch.clamp(used, max=n_pages - 1)], torch.full_like(used, -1, dtype=torch.int32)).to(torch.int32)
    total = held.sum()
    at = torch.arange(n_pages, device=DEV)
    free_list = torch.where(at < n_pages - total, ids[torch.clamp(at + total, max=n_pages - 1)], torch.full_like(ids, -1))
    return dict(op="pages", steps=[(len_a, gamma_a, _prefix(gamma_a + 1)), (len_b, gamma_b, _prefix(gamma_b + 1))], gamma_max=gmax,
                table=table.contiguous(), held=held.to(torch.int32), free_list=free_list.contiguous(), n_free=(n_pages - total).to(torch.int32).reshape(1),
                slot_map=torch.full((n_rows,), -7, dtype=torch.int64, device=DEV), positions=torch.full((n_rows,), -7, dtype=torch.int32, device=DEV))


def _prepare_rope(c, g):
    n, hq, hkv, D, rot = c["rows"], c["hq"], c["hkv"], c["dim"], c["rot"]
    width = (hq + 2 * hkv) * D
    qkv = g.normal((n, width), 1.5, torch.bfloat16)                      # the projection's output, one row per position
    q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([hq * D, hkv * D, hkv * D], 1))
    n_pages = (n + PAGE - 1) // PAGE + 4
    k_pool, v_pool = (g.normal((n_pages, hkv, PAGE, D), 1.0, torch.bfloat16) for _ in range(2))
    slots = torch.randperm(n_pages * PAGE, generator=g.g, device=DEV)[:n].contiguous()
    if c["pad"]:
        slots = torch.where(g.uniform((n,)) < c["pad"], torch.full_like(slots, -1), slots)
    shape = (n,) if c["axes"] == 1 else (c["axes"], n)
    s = dict(op="rope", q=q, k=k, v=v, q_out=torch.zeros((n, hq, D), dtype=torch.bfloat16, device=DEV), k_pool=k_pool, v_pool=v_pool, slots=slots,
             positions=g.ints(0, c["far"], shape), inv_freq=10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=DEV) / (rot // 2)),
             q_weight=None, k_weight=None, eps=1e-6, interleaved=c["interleaved"], freq_axis=None, pool=None)
    if c["norm"]:
        s["q_weight"], s["k_weight"] = (1.0 + g.normal((D,), 0.2)).to(torch.bfloat16), (1.0 + g.normal((D,), 0.2)).to(torch.bfloat16)
    if c["axes"] > 1:
        s["freq_axis"] = (torch.arange(rot // 2, device=DEV) % c["axes"]).to(torch.uint8)
    if own:
        from paper_2504_00030_b200 import binding as sv
        s["pool"] = sv.spec_kv_pool_register(k_pool, v_pool)
    return s


def _prepare_logits(c, g):
    B, gmax, V = c["batch"], c["gamma_max"], c["vocab"]
    dt = torch.bfloat16 if c["bf16"] else torch.float32
    gamma = g.ints(max(0, gmax - 4), gmax + 1, (B,)) if c["batch"] < 100 else torch.full((B,), gmax, dtype=torch.int32, device=DEV)
    cu_q, cu_d = _prefix(gamma + 1), _prefix(gamma)
    n_rows = B if c["draft"] else B * (gmax + 1)                         # verify rows: a buffer for the longest blocks
    stride = (V + 7) // 8 * 8
    s = dict(op="logits", logits=g.normal((n_rows, V), 2.5, dt), gamma=gamma, cu_q=cu_q, cu_d=cu_d, gamma_max=gmax, vocab=V, draft=c["draft"],
             n_drafted=(g.uniform((B,)) * (gamma + 1)).to(torch.int32) if c["draft"] else None,
             draft_tokens=_skewed_tokens(g, (max(1, B * gmax),), V), counts=None, repetition=None, frequency=None, presence=None,
             bias_tokens=None, bias_values=None, n_bias=None, mask=None)
    s["out"] = s["logits"] if c["inplace"] else torch.zeros_like(s["logits"])
    if c["penal"]:
        counts = torch.zeros((B, stride), dtype=torch.int16, device=DEV)
        one = torch.ones((B, 1024), dtype=torch.int16, device=DEV)
        counts.scatter_add_(1, _skewed_tokens(g, (B, 1024), V).long(), one)                       # 1024 generated tokens
        seen = _skewed_tokens(g, (B, 2048), V).long()                                             # and a prompt of 2048
        counts.scatter_(1, seen, torch.gather(counts, 1, seen) | -32768)
        s["counts"] = counts
        s["repetition"], s["frequency"], s["presence"] = g.uniform((B,), 1.0, 1.4), g.uniform((B,), 0.0, 0.5), g.uniform((B,), 0.0, 0.6)
    if c["bias"]:
        n = min(c["bias"], V)
        s["bias_tokens"] = torch.stack([g.perm(V)[:n] for _ in range(min(B, 4))])[torch.arange(B, device=DEV) % min(B, 4)].contiguous()
        s["bias_values"] = g.uniform((B, n), -20.0, 20.0)
        s["n_bias"] = g.ints(0, n + 1, (B,))
    if c["mask"]:
        words = (V + 31) // 32
        a, b = (g.ints(-2**31, 2**31, (n_rows, words)) for _ in range(2))
        kind = g.ints(0, 3, (n_rows, 1))                                 # a free row, a loose grammar, a tight one
        s["mask"] = torch.where(kind == 0, torch.full_like(a, -1), torch.where(kind == 1, a, a & b & torch.roll(a, 1, 1) & torch.roll(b, 1, 1))).contiguous()
    return s


def _prepare_counts(c, g):
    B, V, n = c["batch"], c["vocab"], c["tokens"]
    counts = torch.zeros((B, (V + 7) // 8 * 8), dtype=torch.int16, device=DEV)
    old = _skewed_tokens(g, (B, 512), V).long()
    counts.scatter_add_(1, old, torch.ones_like(old, dtype=torch.int16))
    tokens = _skewed_tokens(g, (B, n), V)
    if c["admit"]:                                                       # prompts of all lengths, packed
        length = g.ints(max(1, n // 2), n + 1, (B,))
        keep = torch.arange(n, device=DEV) < length[:, None]
        return dict(op="counts", counts=counts, vocab=V, tokens=tokens[keep].contiguous(), cu=_prefix(length), most=n,
                    reset=torch.ones(B, dtype=torch.int32, device=DEV), prompt=True)
    emitted = g.ints(1, n + 1, (B,))
    tokens = torch.where(torch.arange(n, device=DEV) < emitted[:, None], tokens, torch.full_like(tokens, -1)).contiguous()
    return dict(op="counts", counts=counts, vocab=V, tokens=tokens, cu=None, most=n, reset=None, prompt=False)


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return {"pages": _run_pages, "rope": _run_rope, "logits": _run_logits, "counts": _run_counts}[s["op"]](s)


def _run_pages(s):
    """Two updates: to the lengths of the next step (retired sequences at 0), and on to the lengths of the one after it."""
    (len_a, gamma_a, cu_a), (len_b, gamma_b, cu_b) = s["steps"]
    if own:
        from paper_2504_00030_b200 import binding as sv
        sv.spec_kv_pages_update(len_a, s["table"], s["held"], s["free_list"], s["n_free"], gamma_a, cu_a, s["gamma_max"], s["slot_map"], s["positions"])
        sv.spec_kv_pages_update(len_b, s["table"], s["held"], s["free_list"], s["n_free"], gamma_b, cu_b, s["gamma_max"], s["slot_map"], s["positions"])
    else:
        _plain_pages(s, len_a, gamma_a, cu_a)
        _plain_pages(s, len_b, gamma_b, cu_b)
    return {k: s[k] for k in ("table", "held", "free_list", "n_free", "slot_map", "positions")}


def _plain_pages(s, length, gamma, cu_q):
    table, free_list = s["table"], s["free_list"]
    held, n_free = s["held"].long(), s["n_free"].long()
    need = (length.long() + PAGE - 1) // PAGE
    released, wanted = torch.clamp(held - need, min=0), torch.clamp(need - held, min=0)
    col = torch.arange(table.shape[1], device=table.device)
    gone = (col >= need[:, None]) & (col < held[:, None])
    to = n_free + (torch.cumsum(released, 0) - released)[:, None] + (col - need[:, None])
    free_list[to[gone]] = table[gone]
    table[gone] = -1
    have = n_free + released.sum()
    until = torch.cumsum(wanted, 0)
    served = until <= have                                               # in the order of the batch, all of a sequence's pages or none
    new = (col >= held[:, None]) & (col < need[:, None]) & served[:, None]
    at = have - 1 - (until - wanted)[:, None] - (col - held[:, None])
    table[new] = free_list[at[new]]
    s["n_free"].copy_(have - torch.where(served, wanted, torch.zeros_like(wanted)).sum())
    held = torch.where(served, need, torch.minimum(held, need))
    s["held"].copy_(held)
    row = torch.arange(s["slot_map"].numel(), device=table.device)
    seq = torch.clamp(torch.searchsorted(cu_q.long(), row, right=True) - 1, min=0, max=length.numel() - 1)
    i = row - cu_q.long()[seq]
    pos = length.long()[seq] - gamma.long()[seq] - 1 + i
    ok = (i <= gamma.long()[seq]) & (pos >= i) & (need[seq] <= held[seq])
    at = torch.where(ok, pos, torch.zeros_like(pos))
    slot = table[seq, at // PAGE].long() * PAGE + at % PAGE
    s["slot_map"].copy_(torch.where(ok, slot, torch.full_like(slot, -1)))
    s["positions"].copy_(torch.where(ok, pos, torch.full_like(pos, -1)))


def _run_rope(s):
    if own:
        from paper_2504_00030_b200 import binding as sv
        sv.spec_rope_append(s["q"], s["k"], s["v"], s["q_out"], s["pool"], s["positions"], s["slots"], s["inv_freq"], q_weight=s["q_weight"],
                            k_weight=s["k_weight"], eps=s["eps"], interleaved=s["interleaved"], freq_axis=s["freq_axis"])
    else:
        row = torch.nonzero(s["slots"] >= 0).reshape(-1)
        slot = s["slots"][row]
        positions = s["positions"].double()
        if s["freq_axis"] is not None:
            positions = positions[s["freq_axis"].long()].t()             # [rows, frequencies]
        else:
            positions = positions[:, None]
        angle = (positions * s["inv_freq"])[row]                         # far positions: in 64 bits
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        s["q_out"][row] = _plain_norm_rotate(s["q"][row], s["q_weight"], s["eps"], cos, sin, s["interleaved"])
        page, at = slot // PAGE, slot % PAGE
        s["k_pool"][page, :, at] = _plain_norm_rotate(s["k"][row], s["k_weight"], s["eps"], cos, sin, s["interleaved"])
        s["v_pool"][page, :, at] = s["v"][row]
    return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}


def _plain_norm_rotate(x, weight, eps, cos, sin, interleaved):
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + eps) * weight.float()
    rot = 2 * cos.shape[-1]
    turned, rest = y[..., :rot], y[..., rot:]
    if interleaved:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = turned[..., :rot // 2], turned[..., rot // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, rest), -1).to(torch.bfloat16)


def _run_logits(s):
    if own:
        from paper_2504_00030_b200 import binding as sv
        sv.spec_logits_adjust(s["logits"], s["out"], s["gamma"], s["cu_q"], s["cu_d"], s["gamma_max"], draft_tokens=s["draft_tokens"], token_counts=s["counts"],
                              repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"], bias_tokens=s["bias_tokens"],
                              bias_values=s["bias_values"], n_bias=s["n_bias"], mask=s["mask"], n_drafted=s["n_drafted"])
        return s["out"]
    V, B = s["vocab"], s["gamma"].numel()
    n_rows = s["logits"].shape[0]
    row = torch.arange(n_rows, device=DEV)
    if s["draft"]:
        seq, before, used = row, s["n_drafted"].long(), row >= 0
    else:
        cu = s["cu_q"].long()
        seq = torch.clamp(torch.searchsorted(cu, row, right=True) - 1, max=B - 1)
        before = row - cu[seq]
        used = before <= s["gamma"].long()[seq]
    x = s["logits"].float()
    if s["counts"] is not None:
        mine = s["counts"][:, :V][seq].int()
        prompt, count = mine < 0, mine & 0x7FFF
        j = torch.arange(max(1, s["gamma_max"]), device=DEV)
        drafted = (j < before[:, None]) & used[:, None]
        token = s["draft_tokens"][torch.where(drafted, s["cu_d"].long()[seq][:, None] + j, torch.zeros_like(j))].long()
        count.scatter_add_(1, token, drafted.int())
        r = s["repetition"][seq][:, None]
        x = torch.where(prompt | (count > 0), torch.where(x > 0, x / r, x * r), x)
        x = x - s["frequency"][seq][:, None] * count - torch.where(count > 0, s["presence"][seq][:, None], torch.zeros_like(r))
    if s["n_bias"] is not None:
        n = s["bias_tokens"].shape[1]
        value = torch.where(torch.arange(n, device=DEV) < s["n_bias"][:, None], s["bias_values"], torch.zeros_like(s["bias_values"]))
        x = x + torch.zeros((B, V), device=DEV).scatter_add_(1, s["bias_tokens"].long(), value)[seq]
    if s["mask"] is not None:
        bit = torch.arange(V, device=DEV)
        allowed = (s["mask"][:, bit // 32] >> (bit % 32)) & 1
        x = torch.where(allowed == 1, x, torch.full_like(x, -math.inf))
    x = x.to(s["out"].dtype)
    if s["draft"]:
        s["out"].copy_(x)
    else:
        s["out"].copy_(torch.where(used[:, None], x, s["out"]))          # rows of no sequence stay as they are
    return s["out"]


def _run_counts(s):
    counts, V = s["counts"], s["vocab"]
    if own:
        from paper_2504_00030_b200 import binding as sv
        sv.spec_token_counts_update(counts, V, s["tokens"], cu_tokens=s["cu"], max_tokens=s["most"], reset=s["reset"], prompt=s["prompt"])
        return counts
    if s["cu"] is not None:
        at = torch.arange(s["tokens"].numel(), device=DEV)
        seq = torch.searchsorted(s["cu"].long(), at, right=True) - 1
        token = s["tokens"].long()
    else:
        B, n = s["tokens"].shape
        seq = torch.arange(B, device=DEV).repeat_interleave(n)
        token = s["tokens"].reshape(-1).long()
        seq, token = seq[token >= 0], token[token >= 0]
    if s["reset"] is not None:
        counts.copy_(torch.where(s["reset"][:, None] != 0, torch.zeros_like(counts), counts))
    if s["prompt"]:
        counts[seq, token] = counts[seq, token] | -32768
    else:
        more = torch.zeros(counts.shape, dtype=torch.int32, device=DEV).index_put_((seq, token), torch.ones_like(token, dtype=torch.int32), accumulate=True)
        count = torch.clamp((counts.int() & 0x7FFF) + more, max=0x7FFF)
        counts.copy_(torch.where(counts < 0, count - 32768, count).to(torch.int16))
    return counts


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(c):
    if c["op"] == "pages":
        B, rows = c["batch"], c["batch"] * (c["gamma_max"] + 1)
        pages = B * (c["ctx_lo"] + c["ctx_hi"]) / 2 / PAGE * c["retire"] + B * (1 - c["retire"]) * c["gamma_max"] / 2 / PAGE
        # two updates: length, held pages (in and out), block length and offset of each sequence; the rows' slots and positions;
        # each page that changes hands read and written
        return {"bytes": 2 * (B * 20 + rows * 12 + pages * 8), "flops": 2 * (B * 10 + rows * 4)}
    if c["op"] == "rope":
        n = c["rows"] * (1 - c["pad"])
        width = (c["hq"] + 2 * c["hkv"]) * c["dim"]
        return {"bytes": n * width * 4 + c["rows"] * (8 + 4 * c["axes"]), "flops": n * (c["hq"] + c["hkv"]) * (4.0 * c["dim"] * c["norm"] + 3.0 * c["rot"])}
    if c["op"] == "logits":
        rows = c["batch"] if c["draft"] else c["batch"] * (max(0, c["gamma_max"] - 4) + c["gamma_max"] + 2) / 2
        if c["batch"] >= 100 and not c["draft"]:
            rows = c["batch"] * (c["gamma_max"] + 1)
        n = rows * c["vocab"]
        # in place and masked alone: what is allowed stays where it is, and what is forbidden is written only
        logits = n * (2 if c["bf16"] else 4) * ((0.0 + 1 / 2 + 15 / 16) / 3 if c["inplace"] and not c["penal"] else 2)
        return {"bytes": logits + n / 8 * c["mask"] + c["batch"] * c["vocab"] * 2 * c["penal"] + c["batch"] * 8 * c["bias"], "flops": n * (4 * c["penal"] + (c["bias"] > 0))}
    if c["admit"]:
        return {"bytes": c["batch"] * (c["vocab"] * 2 + c["tokens"] * 3), "flops": c["batch"] * c["tokens"]}
    return {"bytes": c["batch"] * (c["tokens"] * 4 + c["tokens"] / 2 * 4), "flops": c["batch"] * c["tokens"]}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    if case["op"] == "rope":
        return _exact_rope(prepare(case, seed))
    if case["op"] == "logits":
        return _exact_logits(prepare(case, seed))
    return None                                                          # whole numbers: equal or wrong


def _exact_rope(s):
    n, hq, D = s["q"].shape
    nf = s["inv_freq"].numel()
    axis = torch.zeros(nf, dtype=torch.int64, device=DEV) if s["freq_axis"] is None else s["freq_axis"].long()
    where = s["positions"].reshape(-1, n)
    turn = torch.polar(torch.ones((n, nf), dtype=torch.float64, device=DEV), torch.stack([where[int(a)].double() * s["inv_freq"][f] for f, a in enumerate(axis.tolist())], 1))

    def heads(x, weight):
        y = x.double()
        if weight is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / D + s["eps"]) * weight.double()
        if s["interleaved"]:
            first, second = torch.arange(0, 2 * nf, 2, device=DEV), torch.arange(1, 2 * nf, 2, device=DEV)
        else:
            first, second = torch.arange(nf, device=DEV), torch.arange(nf, 2 * nf, device=DEV)
        z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        return y

    used = (s["slots"] >= 0).tolist()
    q = torch.where(torch.tensor(used, device=DEV)[:, None, None], heads(s["q"], s["q_weight"]), s["q_out"].double())
    rows = torch.tensor([r for r, u in enumerate(used) if u], dtype=torch.int64, device=DEV)
    page, at = torch.div(s["slots"][rows], PAGE, rounding_mode="floor"), torch.remainder(s["slots"][rows], PAGE)
    k, v = s["k_pool"].double().transpose(1, 2).contiguous(), s["v_pool"].double().transpose(1, 2).contiguous()     # [page, slot, head, dim]
    k[page, at], v[page, at] = heads(s["k"], s["k_weight"])[rows], s["v"].double()[rows]
    return {"q": q, "k": k.transpose(1, 2).contiguous(), "v": v.transpose(1, 2).contiguous()}


def _exact_logits(s):
    V, out = s["vocab"], s["out"].double()
    cu_q, cu_d, gamma = s["cu_q"].tolist(), s["cu_d"].tolist(), s["gamma"].tolist()
    drafted = s["n_drafted"].tolist() if s["draft"] else None
    power = 2 ** torch.arange(32, device=DEV, dtype=torch.int64)
    for b in range(len(gamma)):
        rows = [(b, drafted[b])] if s["draft"] else [(cu_q[b] + i, i) for i in range(gamma[b] + 1)]
        lo, hi = rows[0][0], rows[-1][0] + 1
        x = s["logits"][lo:hi].double()
        if s["counts"] is not None:
            stored = s["counts"][b, :V].to(torch.int64) % 65536
            prompt, base = torch.div(stored, 32768, rounding_mode="floor") > 0, torch.remainder(stored, 32768)
            history = torch.stack([base + torch.bincount(s["draft_tokens"][cu_d[b]:cu_d[b] + n].long(), minlength=V) for _, n in rows])
            r, f, p = (float(s[k][b]) for k in ("repetition", "frequency", "presence"))
            seen = (history > 0) | prompt
            x[seen] = torch.where(x[seen] > 0, x[seen] / r, x[seen] * r)
            x = x - f * history.double() - p * (history > 0).double()
        if s["n_bias"] is not None:
            m = int(s["n_bias"][b])
            x[:, s["bias_tokens"][b, :m].long()] += s["bias_values"][b, :m].double()
        if s["mask"] is not None:
            bits = (s["mask"][lo:hi].to(torch.int64)[:, :, None] & power) != 0
            x[~bits.flatten(1)[:, :V]] = -math.inf
        out[lo:hi] = x
    return out
