"""Timing cases of the operators for requests that share prefixes on a paged cache: attention that reads a shared prefix once for its group,
the groups found from the page table, the maps from new tokens to their places, and the page tables of requests from their lengths.

`listed()` names the cases, `draw(rng)` makes more of the same ranges, `prepare` builds what a serving program holds before the call
(cache, tables, new rows), `run` makes ONE pass: the library's call where `own` is set, else the same result in elementary torch
operations in 32 bits.  `exact` states computed numbers in 64 bits, in an arrangement of its own.

Lengths within a case are spread between the case's bounds by a fixed rule, so that `work` follows from the case alone (but those of the prefixes
that `prefix_groups` is to find); values and pages' places come from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # four beams of one prompt on the 1B shape, a dozen to a hundred tokens apart: latency
        {"name": "attn_beams_1b", "kind": "attn", "groups": 1, "members": 4, "shared_lo": 1500, "shared_hi": 1500, "hist_lo": 11, "hist_hi": 99,
         "new_lo": 1, "new_hi": 1, "hq": 32, "hkv": 8, "dh": 64, "dtype": "bf16", "page": 16},
        # 64 requests behind one long instruction, an 8B-class decoder
        {"name": "attn_step_8b_r64", "kind": "attn", "groups": 1, "members": 64, "shared_lo": 8200, "shared_hi": 8200, "hist_lo": 20, "hist_hi": 600,
         "new_lo": 1, "new_hi": 1, "hq": 32, "hkv": 8, "dh": 128, "dtype": "bf16", "page": 16},
        # a full serving batch over four long documents
        {"name": "attn_step_8b_r256", "kind": "attn", "groups": 4, "members": 64, "shared_lo": 9000, "shared_hi": 16400, "hist_lo": 50, "hist_hi": 1000,
         "new_lo": 1, "new_hi": 1, "hq": 32, "hkv": 8, "dh": 128, "dtype": "bf16", "page": 16},
        # 40 prompts with five samples each, three query heads to a KV head, large pages
        {"name": "attn_samples_r200", "kind": "attn", "groups": 40, "members": 5, "shared_lo": 100, "shared_hi": 2100, "hist_lo": 1, "hist_hi": 300,
         "new_lo": 1, "new_hi": 1, "hq": 24, "hkv": 8, "dh": 128, "dtype": "f16", "page": 64},
        # questions of unequal length about two documents
        {"name": "attn_prompts_ragged", "kind": "attn", "groups": 2, "members": 4, "shared_lo": 700, "shared_hi": 2300, "hist_lo": 0, "hist_hi": 311,
         "new_lo": 17, "new_hi": 333, "hq": 24, "hkv": 8, "dh": 128, "dtype": "f16", "page": 32},
        # 16 prompts of 512 tokens behind a long instruction, an 8B-class decoder
        {"name": "attn_prompts_8b", "kind": "attn", "groups": 1, "members": 16, "shared_lo": 8192, "shared_hi": 8192, "hist_lo": 0, "hist_hi": 0,
         "new_lo": 512, "new_hi": 512, "hq": 32, "hkv": 8, "dh": 128, "dtype": "bf16", "page": 16},
        # the groups of a small batch
        {"name": "groups_r8", "kind": "groups", "groups": 2, "members": 4, "width": 256, "page": 16, "shared_lo": 500, "shared_hi": 1500, "hist_hi": 300},
        # the groups of a large batch with tables of 32 K positions
        {"name": "groups_r1000", "kind": "groups", "groups": 20, "members": 50, "width": 2048, "page": 16, "shared_lo": 1000, "shared_hi": 20000,
         "hist_hi": 3000},
        # one new token of each of a few sequences
        {"name": "slots_step_r8", "kind": "slots", "seqs": 8, "width": 256, "page": 16, "len_lo": 100, "len_hi": 3000, "new_lo": 1, "new_hi": 1, "pad": 0},
        # the next chunks of 256 prompts, rows padded to a fixed number
        {"name": "slots_chunks_r256", "kind": "slots", "seqs": 256, "width": 2048, "page": 16, "len_lo": 600, "len_hi": 30000, "new_lo": 0, "new_hi": 512,
         "pad": 1000},
        # a small batch in which half of the requests are new
        {"name": "admit_r8", "kind": "admit", "seqs": 8, "width": 256, "page": 16, "pages": 2048, "len_lo": 100, "len_hi": 2000, "new_hi": 200},
        # a large one on a large pool
        {"name": "admit_r512", "kind": "admit", "seqs": 512, "width": 2048, "page": 16, "pages": 262144, "len_lo": 100, "len_hi": 8000, "new_hi": 2000},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    kind = rng.choice(["attn", "attn", "attn", "groups", "slots", "admit"])
    page = rng.choice([16, 16, 32, 64])
    if kind == "attn":
        hkv, dh, dtype = rng.choice([1, 2, 4, 8]), rng.choice([64, 128]), rng.choice(["bf16", "bf16", "f16"])
        hq = hkv * rng.choice([1, 2, 3, 4, 4, 7, 8, 12])
        hq = min(hq, 32) // hkv * hkv
        if rng.random() < 0.6:  # steps
            members = _log(rng, 1, 64)
            new_lo, new_hi, shared_hi, hist_hi = 1, 1, _log(rng, 16, 16400), _log(rng, 1, 1000)
            groups = _log(rng, 1, max(1, min(48, 256 // members, 130000 // (members * hist_hi), 50000 // shared_hi)))
        else:
            new_hi = _log(rng, 2, 1024)
            members = _log(rng, 1, max(1, min(32, 6000 // new_hi)))
            groups = _log(rng, 1, max(1, min(8, 6000 // (new_hi * members))))
            new_lo, shared_hi, hist_hi = rng.randint(1, new_hi), _log(rng, 16, 8000), _log(rng, 1, 500)
        return {"kind": kind, "groups": groups, "members": members, "shared_lo": rng.randint(1, shared_hi), "shared_hi": shared_hi,
                "hist_lo": rng.randint(0, hist_hi), "hist_hi": hist_hi, "new_lo": new_lo, "new_hi": new_hi, "hq": hq, "hkv": hkv, "dh": dh,
                "dtype": dtype, "page": page}
    if kind == "groups":
        members, shared_hi, hist_hi = _log(rng, 2, 64), _log(rng, 500, 20000), _log(rng, 1, 3000)
        return {"kind": kind, "groups": _log(rng, 1, max(1, 1000 // members)), "members": members, "page": page,
                "width": -(-(shared_hi + hist_hi) // page) + rng.randint(1, 300), "shared_lo": rng.randint(1, shared_hi // 2), "shared_hi": shared_hi,
                "hist_hi": hist_hi}
    if kind == "slots":
        len_hi, new_hi = _log(rng, 100, 30000), _log(rng, 1, 512)
        new_hi = min(new_hi, len_hi)
        return {"kind": kind, "seqs": _log(rng, 1, 256), "width": -(-len_hi // page) + rng.randint(0, 300), "page": page, "len_lo": rng.randint(new_hi, len_hi),
                "len_hi": len_hi, "new_lo": rng.randint(0, new_hi), "new_hi": new_hi, "pad": rng.choice([0, 0, 1, 77, 1000])}
    seqs, len_hi, new_hi = _log(rng, 1, 512), _log(rng, 100, 8000), _log(rng, 1, 2000)
    return {"kind": kind, "seqs": seqs, "width": -(-(len_hi + new_hi) // page) + rng.randint(0, 300), "page": page,
            "pages": seqs * -(-(2 * len_hi + new_hi) // page) + rng.randint(0, 9999), "len_lo": rng.randint(1, len_hi), "len_hi": len_hi, "new_hi": new_hi}


def _spread(n, lo, hi, step=0.6180339887498949):
    """n whole numbers between lo and hi, the first one hi."""
    return [lo + int((hi - lo) * ((1.0 - i * step) % 1.0 if i else 1.0) + 0.5) for i in range(n)]


def _attn_lens(case):
    """Per sequence: positions of whole pages that its group shares, those of its own before the new ones, new ones."""
    g, m, ps = case["groups"], case["members"], case["page"]
    shared = [n // ps * ps for n in _spread(g, case["shared_lo"], case["shared_hi"])]
    hist = _spread(g * m, case["hist_lo"], case["hist_hi"], 0.7548776662466927)
    new = _spread(g * m, case["new_lo"], case["new_hi"])
    return [shared[i // m] for i in range(g * m)], hist, new


def _admit_lens(case):
    """Per sequence: positions held, and of its request those beyond what it begins with."""
    return _spread(case["seqs"], case["len_lo"], case["len_hi"]), _spread(case["seqs"], min(1, case["new_hi"]), case["new_hi"], 0.7548776662466927)


def work(case):
    kind = case["kind"]
    if kind == "attn":
        shared, hist, new = _attn_lens(case)
        m = case["members"]
        keys = sum(shared[::m]) + sum(hist) + sum(new)
        pairs = sum(n * (s + h) + n * (n + 1) // 2 for s, h, n in zip(shared, hist, new))
        return {"bytes": 4.0 * sum(new) * case["hq"] * case["dh"] + 4.0 * keys * case["hkv"] * case["dh"] + 4.0 * keys / case["page"],
                "flops": 4.0 * pairs * case["hq"] * case["dh"]}
    if kind == "groups":
        shared = (case["shared_lo"] + case["shared_hi"]) / 2 / case["page"] + 0.5  # (on average: the lengths come from the seed)
        return {"bytes": (4.0 * shared + 16.0) * case["groups"] * case["members"], "flops": 0}
    if kind == "slots":
        new = _spread(case["seqs"], case["new_lo"], case["new_hi"], 0.7548776662466927)
        return {"bytes": 12.0 * case["seqs"] + 16.0 * (sum(new) + case["pad"]) + 4.0 * sum(-(-n // case["page"]) for n in new), "flops": 0}
    return {"bytes": 8.0 * (case["seqs"] * case["width"] + case["pages"]) + 28.0 * case["seqs"], "flops": 0}


# ---------------------------------------------------------------- inputs
def _shared_table(shared, own_pages, members, width, ids, device):
    """[sequences, width]: `shared` pages of a sequence's group (the group's first sequence's), then its own; -1 behind them.  ids: distinct pages."""
    i = torch.arange(len(shared), device=device)
    col, sh, ow = torch.arange(width, device=device)[None, :], shared[:, None], own_pages[:, None]
    lead = (i % members == 0)[:, None]
    mine = ((col >= sh) & (col < sh + ow)) | (lead & (col < sh))
    rank = mine.flatten().cumsum(0).view(mine.shape) - 1
    first = ids[rank.clamp(min=0)].view(-1, members, width)[:, :1].expand(-1, members, -1).reshape(mine.shape)
    table = torch.where(mine, ids[rank.clamp(min=0)], torch.where(col < sh, first, -1))
    return table.int()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, ps = case["kind"], case["page"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    empty = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")  # noqa: E731
    perm = lambda n: torch.randperm(n, generator=g, device="cuda")  # noqa: E731
    st = {"case": case}
    if kind == "attn":
        shared, hist, new = _attn_lens(case)
        hq, hkv, dh, dt, m = case["hq"], case["hkv"], case["dh"], DTYPES[case["dtype"]], case["members"]
        own_len = [h + n for h, n in zip(hist, new)]
        own_pages = [-(-n // ps) for n in own_len]
        pages = sum(shared[::m]) // ps + sum(own_pages) + 5
        width = max(s // ps + p for s, p in zip(shared, own_pages)) + 1
        st["table"] = _shared_table(ints(shared) // ps, ints(own_pages), m, width, perm(pages), "cuda")
        st["lens"], st["q_start"] = ints(shared) + ints(own_len), ints([0] + torch.tensor(new).cumsum(0).tolist())
        i = torch.arange(len(new), device="cuda", dtype=torch.int32)
        st["lead"], st["shared"] = (i - i % m, ints(shared)) if m > 1 else (i, torch.zeros_like(i))
        st["max_q"], st["max_own"], t = max(new), max(n + (0 if m > 1 else s) for n, s in zip(own_len, shared)), sum(new)
        st["q"] = (torch.randn(t, hq, dh, generator=g, device="cuda") * 1.5).to(dt)
        st["out"] = torch.empty(t, hq, dh, device="cuda", dtype=dt)
        st["pool"] = torch.empty(1, pages, 2, hkv, ps, dh, device="cuda", dtype=dt).normal_(generator=g)
    elif kind == "groups":
        groups, m, width = case["groups"], case["members"], case["width"]
        shared = (torch.randint(case["shared_lo"], case["shared_hi"] + 1, (groups,), generator=g, device="cuda") // ps).repeat_interleave(m).tolist()
        hist = _spread(groups * m, 0, case["hist_hi"], 0.7548776662466927)
        own_pages = [-(-(h + 1) // ps) for h in hist]
        st["table"] = _shared_table(ints(shared), ints(own_pages), m, width, perm(sum(shared[::m]) + sum(own_pages) + 5), "cuda")
        st["lens"] = ints(shared) * ps + ints(hist) + 1
        st["q_start"] = torch.arange(groups * m + 1, device="cuda", dtype=torch.int32)
        st["lead"], st["shared"] = empty(groups * m), empty(groups * m)
    elif kind == "slots":
        seqs, width = case["seqs"], case["width"]
        order = perm(seqs)
        new = _spread(seqs, case["new_lo"], case["new_hi"], 0.7548776662466927)
        st["lens"], st["n_new"] = ints(_spread(seqs, case["len_lo"], case["len_hi"]))[order], ints(new)[order]
        st["lens"] = st["lens"].maximum(st["n_new"])
        held = torch.arange(width, device="cuda")[None, :] < ((st["lens"] + ps - 1) // ps)[:, None]
        st["table"] = torch.where(held, perm(seqs * width).view(seqs, width), -1).int()
        t = sum(new) + case["pad"]
        st["q_start"], st["positions"], st["seqs"] = empty(seqs + 1), empty(t), empty(t)
        st["slots"] = torch.empty(t, dtype=torch.int64, device="cuda")
    else:
        seqs, width, n = case["seqs"], case["width"], case["pages"]
        lens, new = _admit_lens(case)
        i = torch.arange(seqs, device="cuda")
        st["lens"], new = ints(lens), ints(new)[perm(seqs)]
        held = torch.arange(width, device="cuda")[None, :] < ((st["lens"] + ps - 1) // ps)[:, None]
        rank = held.flatten().cumsum(0).view(seqs, width) - 1
        st["table"] = torch.where(held, perm(n)[rank.clamp(0, n - 1)], -1).int()
        st["refs"] = torch.zeros(n + 1, dtype=torch.int32, device="cuda").index_add_(
            0, torch.where(held, st["table"], n).flatten().long(), torch.ones(seqs * width, dtype=torch.int32, device="cuda"))[:n].clone()
        # of four sequences two go on, one makes room for a request that begins like another sequence, one for a request by itself
        other = torch.randint(0, seqs, (seqs,), generator=g, device="cuda")
        st["like"] = torch.where(i % 4 < 2, i, torch.where(i % 4 == 2, other, -1)).int()
        part = (torch.rand(seqs, generator=g, device="cuda") * st["lens"][other]).int()
        st["begin"] = torch.where(i % 4 < 2, st["lens"], torch.where(i % 4 == 2, part, 0)).int()
        st["total"] = (st["begin"] + new).int()
        st["table_out"], st["lens_out"], st["refs_out"], st["n_new"] = empty(seqs, width), empty(seqs), empty(n), empty(seqs)
        st["status"] = ints([0])
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        return _OWN[kind](st, st["case"])
    return _PLAIN[kind](st, st["case"])


def _own_attn(st, case):
    from paper_2604_18396_b200 import prefix_attention
    prefix_attention(st["q"], st["out"], st["q_start"], st["pool"], 1, st["table"], st["lens"], st["lead"], st["shared"], max_q=st["max_q"],
                     max_own=st["max_own"])
    return st["out"]


def _own_groups(st, case):
    from paper_2604_18396_b200 import prefix_groups
    prefix_groups(st["table"], st["lens"], st["q_start"], st["lead"], st["shared"], page_size=case["page"])
    return {k: st[k] for k in ("lead", "shared")}


def _own_slots(st, case):
    from paper_2604_18396_b200 import pages_slots
    pages_slots(st["table"], st["lens"], st["n_new"], st["q_start"], st["positions"], st["seqs"], st["slots"], page_size=case["page"])
    return {k: st[k] for k in ("q_start", "positions", "seqs", "slots")}


def _own_admit(st, case):
    from paper_2604_18396_b200 import pages_admit
    pages_admit(st["table"], st["lens"], st["refs"], st["like"], st["begin"], st["total"], st["table_out"], st["lens_out"], st["refs_out"], st["n_new"],
                st["status"], page_size=case["page"])
    return {k: st[k] for k in ("table_out", "lens_out", "refs_out", "n_new", "status")}


def _plain_attn(st, case):
    hkv, ps, g = case["hkv"], case["page"], case["hq"] // case["hkv"]
    shared, hist, new = _attn_lens(case)
    q, pool, out, at = st["q"], st["pool"][0], st["out"], 0
    for s, (sh, h, n) in enumerate(zip(shared, hist, new)):
        length = sh + h + n
        pages = st["table"][s, : -(-length // ps)].long()
        k, v = (pool[pages, x].transpose(0, 1).reshape(hkv, -1, case["dh"])[:, :length].float() for x in (0, 1))
        x = q[at:at + n].float().unflatten(1, (hkv, g)).permute(1, 2, 0, 3).flatten(1, 2)  # [Hkv, g n, dh]
        score = torch.matmul(x, k.transpose(1, 2)) / math.sqrt(case["dh"])
        if n > 1:
            pos = torch.arange(sh + h, length, device=q.device)
            score.view(hkv, g, n, length).masked_fill_(torch.arange(length, device=q.device) > pos[:, None], -math.inf)
        e = (score - score.amax(-1, keepdim=True)).exp()
        o = torch.matmul(e, v) / e.sum(-1, keepdim=True)
        out[at:at + n] = o.unflatten(1, (g, n)).permute(2, 0, 1, 3).flatten(1, 2).to(out.dtype)
        at += n
    return out


def _plain_groups(st, case):
    ps, table, lens = case["page"], st["table"], st["lens"]
    seqs, width = table.shape
    whole = (lens - st["q_start"].diff()).clamp(min=0) // ps
    col = torch.arange(width, device=table.device)
    same = (table[1:] == table[:-1]) & (table[1:] >= 0) & (col < torch.minimum(whole[1:], whole[:-1])[:, None])
    c = torch.cat((torch.zeros_like(lens[:1]), same.int().cumprod(1).sum(1).int()))  # equal first pages of a sequence and the one before it
    i = torch.arange(seqs, device=table.device)
    lead = torch.where(c > 0, 0, i).cummax(0).values
    least = torch.full((seqs,), 1 << 30, dtype=torch.int32, device=table.device).scatter_reduce(0, lead, torch.where(c > 0, c, 1 << 30).int(), "amin")[lead]
    st["lead"].copy_(lead)
    st["shared"].copy_(torch.where(least < 1 << 30, least * ps, 0))
    return {k: st[k] for k in ("lead", "shared")}


def _plain_slots(st, case):
    ps, new = case["page"], st["n_new"].long()
    start = torch.cat((torch.zeros_like(new[:1]), new.cumsum(0)))
    t = torch.arange(st["positions"].shape[0], device=new.device)
    real = t < start[-1]
    s = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp(max=new.shape[0] - 1)
    pos = st["lens"].long()[s] - new[s] + t - start[s]
    page = st["table"][s, torch.where(real, pos, 0) // ps].long()
    st["q_start"].copy_(start)
    st["positions"].copy_(torch.where(real, pos, -1))
    st["seqs"].copy_(torch.where(real, s, -1))
    st["slots"].copy_(torch.where(real, page * ps + pos % ps, -1))
    return {k: st[k] for k in ("q_start", "positions", "seqs", "slots")}


def _plain_admit(st, case):
    ps, table, lens, refs = case["page"], st["table"], st["lens"], st["refs"]
    (seqs, width), n = table.shape, refs.shape[0]
    col, i = torch.arange(width, device=table.device)[None, :], torch.arange(seqs, device=table.device)
    like, total, up = st["like"].long(), st["total"], ps - 1
    held = torch.where(like >= 0, lens[like.clamp(min=0)], 0)
    s = torch.minimum(torch.minimum(st["begin"], held), total)
    keep = torch.where((like == i) & (s == lens), s, s // ps * ps)  # what a request begins with: all that was held, or whole pages
    old = col < ((lens + up) // ps)[:, None]
    kept = col < ((keep + up) // ps)[:, None]
    tab = torch.where(kept, table[like.clamp(min=0)], -1)
    count = lambda t, m: torch.zeros(n + 1, dtype=torch.int32, device=t.device).index_add_(  # noqa: E731
        0, torch.where(m & (t >= 0), t, n).flatten().long(), torch.ones(t.numel(), dtype=torch.int32, device=t.device))[:n]
    rf = refs + count(tab, kept) - count(table, old)
    want = ~kept & (col < ((total + up) // ps)[:, None])
    free = torch.argsort((rf > 0).to(torch.int8), stable=True)
    ok = (want.sum() <= (rf == 0).sum()) & (total <= width * ps).all()
    rank = want.flatten().cumsum(0).view(seqs, width) - 1
    tab = torch.where(want, free[rank.clamp(0, n - 1)], tab).int()
    st["table_out"].copy_(torch.where(ok, tab, table))
    st["refs_out"].copy_(torch.where(ok, rf + count(tab, want), refs))
    st["lens_out"].copy_(torch.where(ok, total, lens))
    st["n_new"].copy_(torch.where(ok, total - keep, 0))
    st["status"].copy_(torch.where(ok, 0, -4))
    return {k: st[k] for k in ("table_out", "lens_out", "refs_out", "n_new", "status")}


_OWN = {"attn": _own_attn, "groups": _own_groups, "slots": _own_slots, "admit": _own_admit}
_PLAIN = {"attn": _plain_attn, "groups": _plain_groups, "slots": _plain_slots, "admit": _plain_admit}


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    if case["kind"] != "attn":
        return None  # (whole numbers)
    st = prepare(case, seed)
    ps, group = case["page"], case["hq"] // case["hkv"]
    start, lens = st["q_start"].tolist(), st["lens"].tolist()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        j = torch.arange(n, device="cuda")
        kv = st["pool"][0, st["table"][b].long()[j // ps], :, :, j % ps].double()  # [positions][K / V][Hkv][dh]
        rows = slice(start[b], start[b + 1])
        m = start[b + 1] - start[b]
        hidden = j[None, :] >= n - m + 1 + torch.arange(m, device="cuda")[:, None]
        x = st["q"][rows].double().unflatten(1, (-1, group))
        for h in range(case["hkv"]):
            a = torch.einsum("tgd,jd->gtj", x[:, h], kv[:, 0, h]) / math.sqrt(case["dh"])
            out[rows, h * group:(h + 1) * group] = torch.einsum("gtj,jd->tgd", torch.softmax(a.masked_fill_(hidden, -math.inf), -1), kv[:, 1, h])
    return out
