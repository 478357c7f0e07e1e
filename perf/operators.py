"""Timing cases of the operators for long contexts on a paged cache: rotary positions written into the cache, attention over a
sliding window and a few first positions (sinks), and the pages themselves (growing and sliding, forking, compacting).

`listed()` names the cases, `draw(rng)` makes more of the same ranges, `prepare` builds what a serving program holds before the call
(cache, tables, new rows), `run` makes ONE pass: the library's call where `own` is set, else the same result in elementary torch
operations in 32 bits.  `exact` states computed numbers in 64 bits, in an arrangement of its own.

Lengths within a case are spread between the case's bounds by a fixed rule, so that `work` follows from the case alone; values, pages'
places and the order of sequences come from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one new token of a 1B-class decoder: latency is all of it
        {"name": "rope_step_1b", "kind": "rope", "tokens": 1, "hq": 32, "hkv": 8, "dh": 64, "rot": 64, "interleaved": False,
         "scaling": "by_parts", "in": "f32", "cache": "bf16", "page": 16, "context": 40000},
        # a long prompt's chunk of an 8B-class decoder that turns three quarters of a head, rows as a 16-bit projection leaves them
        {"name": "rope_prompt_8b", "kind": "rope", "tokens": 8192, "hq": 32, "hkv": 8, "dh": 128, "rot": 96, "interleaved": True,
         "scaling": "ramp", "in": "bf16", "cache": "bf16", "page": 16, "context": 8192},
        # one conversation of a 1B-class decoder past its window
        {"name": "attn_step_1b_r1", "kind": "attn", "seqs": 1, "new_lo": 1, "new_hi": 1, "hist_lo": 1499, "hist_hi": 1499, "hq": 32, "hkv": 8,
         "dh": 64, "window": 1024, "sinks": 4, "dtype": "bf16", "page": 16},
        # a serving batch of an 8B-class decoder with a long window, conversations between half a window and several
        {"name": "attn_step_8b_r128", "kind": "attn", "seqs": 128, "new_lo": 1, "new_hi": 1, "hist_lo": 4000, "hist_hi": 40000, "hq": 32,
         "hkv": 8, "dh": 128, "window": 8192, "sinks": 16, "dtype": "bf16", "page": 16},
        # follow-up prompts of unequal length behind unequal histories, three query heads to a KV head, a short window
        {"name": "attn_prompts_ragged", "kind": "attn", "seqs": 5, "new_lo": 17, "new_hi": 333, "hist_lo": 0, "hist_hi": 1111, "hq": 24,
         "hkv": 8, "dh": 128, "window": 200, "sinks": 20, "dtype": "f16", "page": 32},
        # a long prompt of an 8B-class decoder in one pass
        {"name": "attn_prompt_8b", "kind": "attn", "seqs": 1, "new_lo": 8192, "new_hi": 8192, "hist_lo": 0, "hist_hi": 0, "hq": 32, "hkv": 8,
         "dh": 128, "window": 4096, "sinks": 4, "dtype": "bf16", "page": 16},
        # four beams of one prompt on the 1B shape
        {"name": "reorder_beams_1b", "kind": "reorder", "seqs": 4, "groups": 1, "layers": 16, "hkv": 8, "dh": 64, "page": 16, "len_lo": 500,
         "len_hi": 500, "pages": 256, "dtype": "bf16"},
        # 64 prompts with four beams each on the 8B shape
        {"name": "reorder_beams_8b", "kind": "reorder", "seqs": 256, "groups": 64, "layers": 32, "hkv": 8, "dh": 128, "page": 16, "len_lo": 100,
         "len_hi": 400, "pages": 2048, "dtype": "bf16"},
        # a small pool after a few conversations have ended
        {"name": "compact_1b", "kind": "compact", "layers": 16, "hkv": 8, "dh": 64, "page": 16, "pages": 100, "used": 0.5, "seqs": 4,
         "dtype": "bf16"},
        # a serving pool of the 8B shape, a third in use, to be given back in part
        {"name": "compact_8b", "kind": "compact", "layers": 32, "hkv": 8, "dh": 128, "page": 16, "pages": 2048, "used": 0.35, "seqs": 64,
         "dtype": "bf16"},
        # one more token of one conversation
        {"name": "advance_r1", "kind": "advance", "seqs": 1, "width": 256, "page": 16, "pages": 256, "window": 1024, "sinks": 4, "len_lo": 1999,
         "len_hi": 1999, "new_lo": 1, "new_hi": 1},
        # the next chunks of 256 prompts of up to 32 K positions on a large pool
        {"name": "advance_r256", "kind": "advance", "seqs": 256, "width": 2048, "page": 16, "pages": 65536, "window": 2048, "sinks": 16,
         "len_lo": 1000, "len_hi": 30000, "new_lo": 0, "new_hi": 512},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    kind = rng.choice(["rope", "attn", "attn", "reorder", "compact", "advance"])
    hkv = rng.choice([1, 2, 4, 8])
    dh, page, dtype = rng.choice([64, 128]), rng.choice([16, 32, 64]), rng.choice(["bf16", "bf16", "f16"])
    if kind == "rope":
        rot = rng.choice([dh, dh, dh // 2, dh * 3 // 4, dh // 4 + 2])
        return {"kind": kind, "tokens": _log(rng, 1, 8192), "hq": hkv * rng.choice([1, 3, 4, 8]) if hkv < 8 else hkv * rng.choice([1, 3, 4]),
                "hkv": hkv, "dh": dh, "rot": rot, "interleaved": rng.random() < 0.5, "scaling": rng.choice(["none", "linear", "by_parts", "ramp"]),
                "in": rng.choice([dtype, "f32"]), "cache": dtype, "page": page, "context": _log(rng, 8192, 131072)}
    if kind == "attn":
        g = rng.choice([1, 2, 3, 4, 4, 7, 8, 12])
        if rng.random() < 0.5:  # steps
            seqs, window = _log(rng, 1, 128), _log(rng, 16, 8192)
            new_lo = new_hi = 1
        else:
            new_hi = _log(rng, 2, 4096)
            seqs, window = _log(rng, 1, max(1, 4096 // new_hi)), _log(rng, 16, 4096)
            new_lo = rng.randint(1, new_hi)
        hist_hi = _log(rng, 1, 32768)
        return {"kind": kind, "seqs": seqs, "new_lo": new_lo, "new_hi": new_hi, "hist_lo": rng.randint(0, hist_hi), "hist_hi": hist_hi,
                "hq": min(hkv * g, 32) // hkv * hkv, "hkv": hkv, "dh": dh, "window": window, "sinks": rng.choice([0, 1, 4, 16, 33, 64]),
                "dtype": dtype, "page": page}
    if kind == "reorder":
        groups, beams = _log(rng, 1, 64), rng.choice([2, 3, 4])
        len_hi = _log(rng, 20, 400)
        return {"kind": kind, "seqs": groups * beams, "groups": groups, "layers": rng.choice([4, 16, 32]), "hkv": hkv, "dh": dh, "page": page,
                "len_lo": rng.randint(1, len_hi), "len_hi": len_hi, "pages": groups * (-(-len_hi // page) + 2 * beams), "dtype": dtype}
    if kind == "compact":
        return {"kind": kind, "layers": rng.choice([4, 16, 32]), "hkv": hkv, "dh": dh, "page": page, "pages": _log(rng, 33, 2048 * 16 // page),
                "used": rng.choice([0.05, 0.2, 0.35, 0.5, 0.8, 0.97]), "seqs": rng.randint(1, 64), "dtype": dtype}
    seqs, len_hi = _log(rng, 1, 256), _log(rng, 100, 30000)
    new_hi = _log(rng, 1, 512)
    return {"kind": kind, "seqs": seqs, "width": -(-(len_hi + new_hi) // page) + rng.randint(0, 40), "page": page,
            "pages": seqs * -(-(len_hi + new_hi) // page) + rng.randint(0, 999), "window": _log(rng, 16, 8192), "sinks": rng.choice([0, 1, 4, 16, 33]),
            "len_lo": rng.randint(0, len_hi), "len_hi": len_hi, "new_lo": rng.randint(0, new_hi), "new_hi": new_hi}


def _spread(n, lo, hi, step=0.6180339887498949):
    """n whole numbers between lo and hi, the first one hi."""
    return [lo + int((hi - lo) * ((1.0 - i * step) % 1.0 if i else 1.0) + 0.5) for i in range(n)]


def _attn_lens(case):
    new = _spread(case["seqs"], case["new_lo"], case["new_hi"])
    hist = _spread(case["seqs"], case["hist_lo"], case["hist_hi"], 0.7548776662466927)
    return new, hist


def work(case):
    kind = case["kind"]
    if kind == "rope":
        t, rows = case["tokens"], case["hq"] + 2 * case["hkv"]
        b = t * rows * case["dh"] * (DTYPES[case["in"]].itemsize + 2) + t * 8 + 2 * case["rot"]
        return {"bytes": b, "flops": 3.0 * t * (case["hq"] + case["hkv"]) * case["rot"]}
    if kind == "attn":
        w, sk = case["window"], case["sinks"]
        pairs = keys = tokens = 0
        for n, h in zip(*_attn_lens(case)):
            seen = lambda p: min(p + 1, w) + min(sk, max(0, p + 1 - w))  # noqa: E731
            tokens += n
            pairs += sum(seen(h + i) for i in range(n))
            low = max(0, h - w + 1)
            keys += h + n - low + min(sk, low)
        return {"bytes": 4.0 * tokens * case["hq"] * case["dh"] + 4.0 * keys * case["hkv"] * case["dh"] + 4.0 * keys / case["page"],
                "flops": 4.0 * pairs * case["hq"] * case["dh"]}
    if kind == "advance":
        return {"bytes": 8.0 * (case["seqs"] * case["width"] + case["pages"] + case["seqs"]), "flops": 0}
    per_pos = 2 * case["hkv"] * case["dh"] * 2 * case["layers"]
    if kind == "reorder":
        lens = _spread(case["groups"], case["len_lo"], case["len_hi"])
        # a group's beams come from two of them: all but two copy the tail that is filled in part
        copied = sum(n % case["page"] for n in lens) * (case["seqs"] // case["groups"] - min(2, case["seqs"] // case["groups"]))
        return {"bytes": 2.0 * copied * per_pos + 8.0 * case["seqs"] * (_width(case) + 1) + 8.0 * case["pages"], "flops": 0}
    moved = _moved(case)
    return {"bytes": 2.0 * moved * case["page"] * per_pos + 12.0 * case["pages"], "flops": 0}


def _width(case):
    return -(-case["len_hi"] // case["page"]) + 1


def _used(case):
    return max(1, min(case["pages"], int(case["pages"] * case["used"])))


def _moved(case):
    """Pages in use behind the first _used(case): every second page is in use as far as that goes, then the last ones."""
    n, u = case["pages"], _used(case)
    return sum(1 for p in _used_ids(n, u) if p >= u)


def _used_ids(n, u):
    return sorted({(i * n) // u for i in range(u)})


# ---------------------------------------------------------------- inputs
def _frequencies(case):
    """Radians per position of each pair of dims, and the factor on the turned values."""
    r = case["rot"]
    f = 10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
    if case["scaling"] == "linear":  # all positions drawn together
        f, c = f / 4.0, 1.0
    elif case["scaling"] == "by_parts":  # slow pairs eight times slower, fast ones as they were, in between by their wavelength
        wave = 2 * math.pi / f
        mix = ((8192 / wave - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        f, c = f * (mix + (1 - mix) / 8.0), 1.0
    elif case["scaling"] == "ramp":  # a ramp over the pairs between those that turn 32 times and once in the original context
        at = lambda turns: r * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))  # noqa: E731
        lo, hi = max(math.floor(at(32)), 0), min(math.ceil(at(1)), r - 1)
        ramp = ((torch.arange(r // 2, dtype=torch.float64) - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f, c = f * (1 - ramp) + f / 16.0 * ramp, 0.1 * math.log(16.0) + 1.0
    else:
        c = 1.0
    return f.to(torch.float32), c


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    rand = lambda *shape, dt=torch.bfloat16: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    st = {"case": case}
    if kind == "rope":
        t, hq, hkv, dh, ps = case["tokens"], case["hq"], case["hkv"], case["dh"], case["page"]
        dt = DTYPES[case["in"]]
        # the rows of one product: q, k and v side by side; the tokens are the next ones of up to 64 sequences, a run of positions each
        qkv = rand(t, (hq + 2 * hkv) * dh, dt=dt)
        st["q"], st["k"], st["v"] = (x.unflatten(-1, (-1, dh)) for x in qkv.split([hq * dh, hkv * dh, hkv * dh], -1))
        seqs = min(t, 64) if t <= 256 else max(1, t // 2048)
        run_ = -(-t // seqs)
        width = -(-(case["context"]) // ps)
        pages = seqs * (run_ // ps + 2)
        start = torch.randint(0, case["context"] - run_ + 1, (seqs,), generator=g, device="cuda")
        tok = torch.arange(t, device="cuda")
        st["seqs"], st["positions"] = (tok // run_).int(), (start[tok // run_] + tok % run_).int()
        col = torch.arange(width, device="cuda")[None, :] - (start // ps)[:, None]
        ids = torch.randperm(pages, generator=g, device="cuda")[: seqs * (run_ // ps + 2)].view(seqs, -1)
        held = (col >= 0) & (col < ids.shape[1])
        st["table"] = torch.where(held, ids.gather(1, col.clamp(0, ids.shape[1] - 1)), -1).int()
        st["pool"] = torch.zeros(1, pages, 2, hkv, ps, dh, device="cuda", dtype=DTYPES[case["cache"]])
        st["q_out"] = torch.empty(t, hq, dh, device="cuda", dtype=DTYPES[case["cache"]])
        f, st["scale"] = _frequencies(case)
        st["inv_freq"] = f.cuda()
    elif kind == "attn":
        new, hist = _attn_lens(case)
        hq, hkv, dh, ps, dt = case["hq"], case["hkv"], case["dh"], case["page"], DTYPES[case["dtype"]]
        lens = [a + b for a, b in zip(new, hist)]
        st["lens"], st["q_start"] = ints(lens), ints([0] + torch.tensor(new).cumsum(0).tolist())
        st["max_q"], t = max(new), sum(new)
        st["q"], st["out"] = rand(t, hq, dh, dt=dt) * 1.5, torch.empty(t, hq, dh, device="cuda", dtype=dt)
        # only the pages that the window and the sinks need are held
        width = -(-max(lens) // ps)
        col, n = torch.arange(width, device="cuda")[None, :], st["lens"][:, None]
        first = (n - ints(new)[:, None] - case["window"] + 1).clamp(min=0) // ps
        held = ((col >= first) | (col < -(-case["sinks"] // ps))) & (col < (n + ps - 1) // ps)
        rank = held.flatten().cumsum(0).view(held.shape) - 1
        pages = int(rank.max()) + 1
        st["table"] = torch.where(held, torch.randperm(pages, generator=g, device="cuda")[rank.clamp(min=0)], -1).int()
        st["pool"] = torch.empty(1, pages, 2, hkv, ps, dh, device="cuda", dtype=dt).normal_(generator=g)
    elif kind == "reorder":
        groups, beams, ps, n = case["groups"], case["seqs"] // case["groups"], case["page"], case["pages"]
        lens = ints(_spread(groups, case["len_lo"], case["len_hi"])).repeat_interleave(beams)
        width, seqs = _width(case), case["seqs"]
        # a group's beams share the whole pages of their prompt but the last one, and have one or two of their own
        col, own_from = torch.arange(width, device="cuda")[None, :], ((lens // ps - 1).clamp(min=0))[:, None]
        held, lead = col < ((lens + ps - 1) // ps)[:, None], (torch.arange(seqs, device="cuda") % beams == 0)[:, None]
        mine = held & (lead | (col >= own_from))
        rank = mine.flatten().cumsum(0).view(seqs, width) - 1
        ids = torch.randperm(n, generator=g, device="cuda")[rank.clamp(0, n - 1)]
        shared = ids.view(groups, beams, width)[:, :1].expand(-1, beams, -1).reshape(seqs, width)
        st["table"] = torch.where(held, torch.where(mine, ids, shared), -1).int()
        st["refs"] = torch.zeros(n + 1, dtype=torch.int32, device="cuda").index_add_(
            0, torch.where(held, st["table"], n).flatten().long(), torch.ones(seqs * width, dtype=torch.int32, device="cuda"))[:n].clone()
        st["lens"] = lens
        # of a group's beams two go on: the first ones of a random order, so many children each
        order = torch.rand(groups, beams, generator=g, device="cuda").argsort(1)
        pick = torch.arange(beams, device="cuda") * min(2, beams) // beams
        st["parents"] = (order[:, pick] + torch.arange(groups, device="cuda")[:, None] * beams).flatten().int()
        st["pool"] = torch.empty(case["layers"], n, 2, case["hkv"], ps, case["dh"], device="cuda", dtype=DTYPES[case["dtype"]]).normal_(generator=g)
        st["table_out"], st["lens_out"], st["refs_out"] = (torch.empty_like(st[k]) for k in ("table", "lens", "refs"))
        st["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    elif kind == "compact":
        n, u, seqs = case["pages"], _used(case), case["seqs"]
        ids = ints(_used_ids(n, u))
        width = -(-u // seqs)
        table = torch.full((seqs * width,), -1, dtype=torch.int32, device="cuda")
        table[:u] = ids[torch.randperm(u, generator=g, device="cuda")]
        st["table"] = table.view(seqs, width)
        st["refs"] = torch.zeros(n, dtype=torch.int32, device="cuda")
        st["refs"][ids.long()] = torch.randint(1, 4, (u,), generator=g, device="cuda", dtype=torch.int32)
        st["pool"] = torch.empty(case["layers"], n, 2, case["hkv"], case["page"], case["dh"], device="cuda", dtype=DTYPES[case["dtype"]]).normal_(generator=g)
        st["table_out"], st["refs_out"], st["remap"] = torch.empty_like(st["table"]), torch.empty_like(st["refs"]), torch.empty_like(st["refs"])
        st["n_used"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    else:
        seqs, width, ps, n = case["seqs"], case["width"], case["page"], case["pages"]
        lens, w = ints(_spread(seqs, case["len_lo"], case["len_hi"])), case["window"]
        # what the window needed a chunk ago is held still
        col, c = torch.arange(width, device="cuda")[None, :], (lens[:, None] + ps - 1) // ps
        first = (lens[:, None] - 512 - w + 1).clamp(min=0) // ps
        held = ((col >= first) | (col < -(-case["sinks"] // ps))) & (col < c)
        rank = held.flatten().cumsum(0).view(seqs, width) - 1
        ids = torch.randperm(n, generator=g, device="cuda")[rank.clamp(0, n - 1)]
        st["table"], st["lens"] = torch.where(held, ids, -1).int(), lens
        st["refs"] = torch.zeros(n + 1, dtype=torch.int32, device="cuda").index_add_(
            0, torch.where(held, st["table"], n).flatten().long(), torch.ones(seqs * width, dtype=torch.int32, device="cuda"))[:n].clone()
        st["n_new"] = ints(_spread(seqs, case["new_lo"], case["new_hi"], 0.7548776662466927))[torch.randperm(seqs, generator=g, device="cuda")]
        st["n_new"] = st["n_new"].minimum((width * ps - lens).clamp(min=0).int())
        st["table_out"], st["lens_out"], st["refs_out"] = (torch.empty_like(st[k]) for k in ("table", "lens", "refs"))
        st["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        return _OWN[kind](st, st["case"])
    return _PLAIN[kind](st, st["case"])


def _own_rope(st, case):
    from paper_2604_18396_b200 import rope_append
    rope_append(st["q"], st["k"], st["v"], st["positions"], st["seqs"], st["inv_freq"], st["pool"], 1, st["table"], st["q_out"],
                interleaved=case["interleaved"], scale=st["scale"])
    return {"q": st["q_out"], "pool": st["pool"]}


def _own_attn(st, case):
    from paper_2604_18396_b200 import window_attention
    window_attention(st["q"], st["out"], st["q_start"], st["pool"], 1, st["table"], st["lens"], window=case["window"], sinks=case["sinks"],
                     max_q=st["max_q"])
    return st["out"]


def _own_reorder(st, case):
    from paper_2604_18396_b200 import pages_reorder
    pages_reorder(st["pool"], st["table"], st["lens"], st["refs"], st["parents"], st["table_out"], st["lens_out"], st["refs_out"], st["status"])
    return {k: st[k] for k in ("pool", "table_out", "lens_out", "refs_out", "status")}


def _own_compact(st, case):
    from paper_2604_18396_b200 import pages_compact
    pages_compact(st["pool"], st["table"], st["refs"], st["table_out"], st["refs_out"], st["remap"], st["n_used"])
    return {k: st[k] for k in ("pool", "table_out", "refs_out", "remap", "n_used")}


def _own_advance(st, case):
    from paper_2604_18396_b200 import pages_advance
    pages_advance(st["table"], st["lens"], st["refs"], st["n_new"], st["table_out"], st["lens_out"], st["refs_out"], st["status"],
                  page_size=case["page"], window=case["window"], sinks=case["sinks"])
    return {k: st[k] for k in ("table_out", "lens_out", "refs_out", "status")}


def _plain_rope(st, case):
    r, ps = case["rot"], case["page"]
    angle = st["positions"].float()[:, None] * st["inv_freq"]
    cos, sin = (angle.cos() * st["scale"])[:, None], (angle.sin() * st["scale"])[:, None]

    def turn(x):
        x = x.float()
        a, b = (x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., : r // 2], x[..., r // 2: r])
        a, b = a * cos - b * sin, b * cos + a * sin
        y = torch.stack((a, b), -1).flatten(-2) if case["interleaved"] else torch.cat((a, b), -1)
        return torch.cat((y, x[..., r:]), -1)

    pool, pos = st["pool"], st["positions"].long()
    page, at = st["table"][st["seqs"].long(), pos // ps].long(), pos % ps
    pool[0, page, 0, :, at] = turn(st["k"]).to(pool.dtype)
    pool[0, page, 1, :, at] = st["v"].to(pool.dtype)
    return {"q": turn(st["q"]).to(pool.dtype), "pool": pool}


def _plain_attn(st, case):
    w, sinks, ps, g = case["window"], case["sinks"], case["page"], case["hq"] // case["hkv"]
    q, pool, start, lens, mq = st["q"], st["pool"][0], st["q_start"].long(), st["lens"].long(), st["max_q"]
    new, i = start.diff(), torch.arange(mq, device=q.device)
    row = (start[:-1, None] + i).clamp(max=q.shape[0] - 1)  # [sequences, max_q]
    pos = torch.where(i < new[:, None], (lens - new)[:, None] + i, -1)
    # the positions that some query of a sequence may see: sinks before the first window, then the windows' union
    low = (lens - new - w + 1).clamp(min=0)
    first = torch.arange(sinks, device=q.device).expand(len(lens), -1)
    n = min(w + mq - 1, int(st["table"].shape[1]) * ps)
    span = low[:, None] + torch.arange(n, device=q.device)
    key = torch.cat((torch.where(first < low[:, None], first, -1), torch.where(span < lens[:, None], span, -1)), 1)
    at = key.clamp(min=0)
    page = st["table"].long().gather(1, at // ps).clamp(min=0)
    k, v = (pool[page, x, :, at % ps].float().permute(0, 2, 1, 3) for x in (0, 1))  # [sequences, Hkv, keys, dh]
    s, p = key[:, None, :], pos[:, :, None]
    seen = (s >= 0) & (s <= p) & ((s < sinks) | (s > p - w))
    seen = seen[:, None, None]
    x = q[row].float().unflatten(2, (-1, g)).permute(0, 2, 3, 1, 4)  # [sequences, Hkv, g, max_q, dh]
    shape = x.shape
    score = torch.matmul(x.flatten(2, 3), k.transpose(-1, -2)).view(*shape[:-1], -1) / math.sqrt(case["dh"])
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    e = (score - torch.where(top.isinf(), 0.0, top)).exp()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.flatten(2, 3), v).view(shape) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3)  # [sequences, max_q, Hq, dh]
    t = torch.arange(q.shape[0], device=q.device)
    of = torch.searchsorted(start[1:].contiguous(), t, right=True)
    st["out"].copy_(o[of, t - start[of]])
    return st["out"]


def _lowest_free(refs):
    return torch.argsort((refs > 0).to(torch.int8), stable=True), (refs == 0).sum()


def _plain_reorder(st, case):
    ps, pool, table, lens, refs, parents = case["page"], st["pool"], st["table"], st["lens"], st["refs"], st["parents"].long()
    n, seqs, width = refs.shape[0], table.shape[0], table.shape[1]
    col, i, live, par = torch.arange(width, device=table.device), torch.arange(seqs, device=table.device), parents >= 0, parents.clamp(min=0)
    ln = torch.where(live, lens[par], 0)
    held = lambda x: col < ((x + ps - 1) // ps)[:, None]  # noqa: E731
    tab = torch.where(held(ln), table[par], -1)
    elder = torch.full((seqs,), seqs, device=table.device).scatter_reduce(0, par, torch.where(live, i, seqs), "amin")
    copies = live & (ln % ps != 0) & (elder[par] != i)
    last = (ln // ps).clamp(max=width - 1)[:, None].long()
    src = tab.gather(1, last)
    tab = torch.where(copies[:, None] & (col == last), -1, tab)
    count = lambda t: torch.zeros(n + 1, dtype=torch.int32, device=t.device).index_add_(  # noqa: E731
        0, torch.where(t >= 0, t, n).flatten().long(), torch.ones(t.numel(), dtype=torch.int32, device=t.device))[:n]
    rf = refs + count(tab) - count(torch.where(held(lens), table, -1))
    free, n_free = _lowest_free(rf)
    ok = copies.sum() <= n_free
    dst = free[(copies.cumsum(0) - 1).clamp(0, n - 1)]
    tab = torch.where(copies[:, None] & (col == last), dst[:, None], tab).int()
    rf = rf.scatter_add(0, dst, copies.int())
    j = (copies & ok).nonzero().flatten()
    if j.numel():
        fill = (torch.arange(ps, device=pool.device)[None, :] < (ln[j] % ps)[:, None])[None, :, None, None, :, None]
        pool[:, dst[j]] = torch.where(fill, pool[:, src[j, 0].long()], pool[:, dst[j]])
    st["table_out"].copy_(torch.where(ok, tab, table))
    st["lens_out"].copy_(torch.where(ok, ln, lens))
    st["refs_out"].copy_(torch.where(ok, rf, refs))
    st["status"].copy_(torch.where(ok, 0, -4))
    return {k: st[k] for k in ("pool", "table_out", "lens_out", "refs_out", "status")}


def _plain_compact(st, case):
    pool, table, refs = st["pool"], st["table"].long(), st["refs"]
    n = refs.shape[0]
    i, used = torch.arange(n, device=refs.device), refs > 0
    n_used = used.sum()
    holes, movers = (~used & (i < n_used)).nonzero().flatten(), (used & (i >= n_used)).nonzero().flatten()
    remap = torch.where(used, i, -1).scatter(0, movers, holes)
    pool[:, holes] = pool[:, movers]
    st["table_out"].copy_(torch.where(table >= 0, remap[table.clamp(min=0)], -1))
    st["refs_out"].copy_(refs.scatter(0, holes, refs[movers]).scatter(0, movers, 0))
    st["remap"].copy_(remap)
    st["n_used"].copy_(n_used)
    return {k: st[k] for k in ("pool", "table_out", "refs_out", "remap", "n_used")}


def _plain_advance(st, case):
    ps, w, sinks, table, lens, refs, new = case["page"], case["window"], case["sinks"], st["table"], st["lens"], st["refs"], st["n_new"]
    n, (seqs, width) = refs.shape[0], table.shape
    col = torch.arange(width, device=table.device)[None, :]
    past = (col >= -(-sinks // ps)) & (col < torch.div(lens - w + 1, ps, rounding_mode="floor")[:, None])
    gone = past & (table < 0)
    drop = past & (gone.flip(1).cumsum(1).flip(1) == 0)
    tab = torch.where(drop, -1, table)
    count = lambda t, m: torch.zeros(n + 1, dtype=torch.int32, device=t.device).index_add_(  # noqa: E731
        0, torch.where(m, t, n).flatten().long(), torch.ones(t.numel(), dtype=torch.int32, device=t.device))[:n]
    rf = refs - count(table, drop)
    need = (col >= ((lens + ps - 1) // ps)[:, None]) & (col < ((lens + new + ps - 1) // ps)[:, None])
    free, n_free = _lowest_free(rf)
    ok = (need.sum() <= n_free) & (lens + new <= width * ps).all()
    rank = need.flatten().cumsum(0).view(seqs, width) - 1
    need = need & ok
    tab = torch.where(need, free[rank.clamp(0, n - 1)], tab).int()
    st["table_out"].copy_(tab)
    st["refs_out"].copy_(rf + count(tab, need))
    st["lens_out"].copy_(torch.where(ok, lens + new, lens))
    st["status"].copy_(torch.where(ok, 0, -4))
    return {k: st[k] for k in ("table_out", "lens_out", "refs_out", "status")}


_OWN = {"rope": _own_rope, "attn": _own_attn, "reorder": _own_reorder, "compact": _own_compact, "advance": _own_advance}
_PLAIN = {"rope": _plain_rope, "attn": _plain_attn, "reorder": _plain_reorder, "compact": _plain_compact, "advance": _plain_advance}


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    if case["kind"] == "rope":
        st = prepare(case, seed)
        r = case["rot"]
        # a pair is one complex number, turned by a factor of modulus `scale`
        turned = torch.polar(torch.full((case["tokens"], 1, r // 2), float(st["scale"]), dtype=torch.float64, device="cuda"),
                             (st["positions"].double()[:, None, None] * st["inv_freq"].double()))

        def turn(x):
            x = x.double().clone()
            a = x[..., :r].unflatten(-1, (r // 2, 2)) if case["interleaved"] else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
            b = torch.view_as_real(torch.view_as_complex(a.contiguous()) * turned)
            x[..., :r] = (b if case["interleaved"] else b.transpose(-1, -2)).flatten(-2)
            return x

        pool, ps = st["pool"].double(), case["page"]
        flat = pool.permute(0, 2, 1, 4, 3, 5)[0].contiguous()  # [K / V][page][position][Hkv][dh]
        pos = st["positions"].long()
        slot = st["table"].long()[st["seqs"].long()].gather(1, (pos // ps)[:, None])[:, 0] * ps + pos % ps
        flat = flat.flatten(1, 2)
        flat[0].index_copy_(0, slot, turn(st["k"]))
        flat[1].index_copy_(0, slot, st["v"].double())
        flat = flat.unflatten(1, (-1, ps))
        return {"q": turn(st["q"]), "pool": flat.permute(1, 0, 3, 2, 4)[None].contiguous()}
    if case["kind"] == "attn":
        st = prepare(case, seed)
        new, hist = _attn_lens(case)
        g, ps, w, sinks = case["hq"] // case["hkv"], case["page"], case["window"], case["sinks"]
        out, at = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda"), 0
        for b, (n, h) in enumerate(zip(new, hist)):
            low = max(0, h - w + 1)
            keys = torch.cat((torch.arange(min(sinks, low)), torch.arange(low, h + n))).cuda()
            kv = st["pool"][0, st["table"][b].long()[keys // ps], :, :, keys % ps]  # [keys][K / V][Hkv][dh]
            pos = torch.arange(h, h + n, device="cuda")[:, None]
            hidden = (keys > pos) | ((keys >= sinks) & (keys <= pos - w))
            for head in range(case["hq"]):
                a = st["q"][at:at + n, head].double() @ kv[:, 0, head // g].double().T / math.sqrt(case["dh"])
                out[at:at + n, head] = torch.softmax(a.masked_fill_(hidden, -math.inf), -1) @ kv[:, 1, head // g].double()
            at += n
        return out
    return None  # (whole numbers, and pages moved as they are)
