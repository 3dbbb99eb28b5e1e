"""Latent attention under the persistence table, as measurable cases.

A latent-attention model keeps one vector a token and layer in place of keys
and values per head: a latent c [rank] and a rotary key r [rope].  Four kinds
of calls:

  write_read  an emptied cache takes a prompt (the table decides each token:
              HIGH bf16, LOW int4 with an fp16 scale per 32 elements, DROP),
              and the kept entries are read back as dense rows in position
              order, as the expansion of the next prompt chunk needs them;
  read        the read-back of a resident mixed history;
  decode      one token's attention over the resident history in the absorbed
              form, with or without the step's own token persisted first;
  prompt      causal attention of a packed ragged batch in the expanded form,
              after a resident history or from the start.

A LOW latent stands for the bf16 value nearest to code x scale; every reader
of the cache uses that value.
"""

from __future__ import annotations

import math
import random
import struct

import numpy as np
import torch

own = False

N_TAGS = 16
DROP, LOW, HIGH = 0, 1, 2


# ---- cases -----------------------------------------------------------------------------------------------------------
# hi, lo: how many of the 16 tags the table keeps HIGH and LOW; the others are dropped.
_CACHE = dict(batch=1, rank=512, rope=64, nmin=64, nmax=64, hi=6, lo=6, sink=0)


def _write_read(name=None, **kw):
    return _named(name, dict(_CACHE, op="write_read", keep_all=False, **kw))


def _read(name=None, **kw):
    return _named(name, dict(_CACHE, op="read", **kw))


def _decode(name=None, **kw):
    return _named(name, dict(_CACHE, op="decode", heads=16, step=False, **kw))


def _prompt(name=None, **kw):
    return _named(name, dict(dict(op="prompt", batch=1, heads=8, nope=128, rope=64, v=128, nmin=64, nmax=64, past=0),
                             **kw))


def _named(name, case):
    if name:
        case["name"] = name
    return case


def _over(case, **kw):
    case.update(kw)
    return case


def listed():
    return [
        # One short tool reply of an odd length, entered and read back between two turns: latency.
        _write_read("write_read_b1_37", nmin=37, nmax=37),
        # A serving batch's labelled prompts: most of the context int4 or released, first 16 tokens kept.
        _write_read("write_read_b32_labelled", batch=32, nmin=500, nmax=8000, hi=3, lo=9, sink=16),
        # A batch of prompts that the table does not govern, all kept.
        _over(_write_read("write_read_b16_kept", batch=16, nmin=900, nmax=8192), keep_all=True),
        # One user's conversation read back for its next turn.
        _read("read_b1_1500", nmin=1500, nmax=1500),
        # Every resident conversation of a batch read back, most of it int4, smaller latents.
        _read("read_b64_mixed_r256", batch=64, rank=256, nmin=100, nmax=12000, hi=3, lo=10),
        # One user's first steps: the token is persisted, then attends a short history.
        _over(_decode("decode_step_b1_200", nmin=200, nmax=200), step=True),
        # One long context with few heads on the device, a history of kept prompt tokens; odd head count.
        _over(_decode("decode_b1_64k_h20", nmin=64001, nmax=64001, hi=14, lo=1), heads=20),
        # A serving batch split over devices (16 heads here): each step persists its token.
        _over(_decode("decode_step_b64_h16", batch=64, nmin=1000, nmax=8192), step=True),
        # All heads on one device: the matrix cores and the memory are both busy.
        _over(_decode("decode_b128_h128", batch=128, nmin=1024, nmax=8192, hi=14, lo=1), heads=128),
        # Prompts of a few tokens each, as short chat turns come, smaller heads.
        _prompt("prompt_b4_tiny", batch=4, heads=20, nope=64, v=64, nmin=1, nmax=60),
        # A chunk of each prompt after what came before it, ragged.
        _prompt("prompt_b8_chunk", batch=8, heads=20, nmin=200, nmax=1024, past=2500),
        # One long prompt with all heads of the device.
        _prompt("prompt_b1_8k_h32", heads=32, nmin=8192, nmax=8192),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        b, f = most.get(c["op"], (0, 0))
        most[c["op"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    while True:
        op = rng.choice(["write_read", "read", "decode", "decode", "prompt"])
        if op == "prompt":
            nmax = _log_int(rng, 1, 8192)
            c = _prompt(batch=_log_int(rng, 1, 64), heads=_log_int(rng, 1, 128), nope=rng.choice([64, 128, 128]),
                        rope=rng.choice([32, 64, 64]), v=rng.choice([64, 128, 128]),
                        nmin=max(1, int(nmax * rng.uniform(0.05, 1.0))), nmax=nmax,
                        past=rng.choice([0, _log_int(rng, 1, 8192)]))
        else:
            nmax = _log_int(rng, 1, 65536)
            hi = rng.randint(0, 16)
            kw = dict(batch=_log_int(rng, 1, 256), rank=rng.choice([128, 256, 512, 512]),
                      rope=rng.choice([32, 64, 64]), nmin=max(1, int(nmax * rng.uniform(0.05, 1.0))), nmax=nmax,
                      hi=hi, lo=rng.randint(0, 16 - hi), sink=rng.choice([0, 0, 4, 16]))
            if op == "decode":
                c = _over(_decode(**kw), heads=_log_int(rng, 1, 128), step=rng.random() < 0.5)
            elif op == "read":
                c = _read(**kw)
            else:
                c = _over(_write_read(**kw), keep_all=rng.random() < 0.3)
        w = work(c)
        if 1e4 < w["bytes"] <= most[op][0] and w["flops"] <= most[op][1] and _resident(c) < 12e9:
            return c


def _resident(case):
    """Bytes of the padded inputs of a case's cache."""
    if case["op"] == "prompt":
        return 0
    return case["batch"] * (case["nmax"] + 1) * (case["rank"] + case["rope"]) * 2


def _lengths(case):
    """Tokens of each sequence: between nmin and nmax, the same for every seed."""
    r = random.Random(case["nmin"] * 1000003 + case["nmax"] * 101 + case["batch"])
    n = [r.randint(case["nmin"], case["nmax"]) for _ in range(case["batch"])]
    n[r.randrange(len(n))] = case["nmax"]
    return n


def _kept(case):
    """HIGH and LOW entries that the prompts leave: tags come equally often behind the sinks (_history)."""
    table = _table(case)
    n_hi = n_lo = 0
    for n in _lengths(case):
        s = n if case.get("keep_all") else min(n, case["sink"])
        n_hi += s
        for z, a in enumerate(table):
            m = (n - s) // N_TAGS + (z < (n - s) % N_TAGS)
            n_hi += m * (a == HIGH)
            n_lo += m * (a == LOW)
    return n_hi, n_lo


def _pasts(case):
    """Resident tokens before each prompt chunk: between none and `past`."""
    r = random.Random(case["past"] * 7919 + case["batch"])
    return [r.randint(0, case["past"]) if case["past"] else 0 for _ in range(case["batch"])]


def work(case):
    if case["op"] == "prompt":
        H, D, P, V = case["heads"], case["nope"], case["rope"], case["v"]
        nq, nk, pairs = 0, 0, 0
        for n, m in zip(_lengths(case), _pasts(case)):
            nq, nk = nq + n, nk + n + m
            pairs += n * m + n * (n + 1) // 2
        return {"bytes": nq * H * (D + P) * 2 + nk * (H * (D + V) + P) * 2 + nq * H * (V * 2 + 4),
                "flops": 2 * H * pairs * (D + P + V)}
    R, P = case["rank"], case["rope"]
    hi_row, lo_row = 2 * (R + P), R // 2 + R // 16 + 2 * P
    n_hi, n_lo = _kept(case)
    kept, stored = n_hi + n_lo, n_hi * hi_row + n_lo * lo_row
    if case["op"] == "write_read":
        return {"bytes": sum(_lengths(case)) + 2 * kept * hi_row + stored + 4 * kept, "flops": 6 * n_lo * R}
    if case["op"] == "read":
        return {"bytes": stored + kept * (hi_row + 4), "flops": 2 * n_lo * R}
    B, H = case["batch"], case["heads"]
    step = B * (1 + 2 * hi_row) if case["step"] else 0
    return {"bytes": stored + step + B * H * ((R + P) * 2 + R * 2 + 4), "flops": 2 * H * kept * (2 * R + P)}


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _table(case):
    """Action of each tag: the table keeps `hi` tags HIGH, `lo` LOW and drops the rest, in a mixed order."""
    acts = [HIGH] * case["hi"] + [LOW] * case["lo"] + [DROP] * (N_TAGS - case["hi"] - case["lo"])
    return [acts[(5 * z + 3) % N_TAGS] for z in range(N_TAGS)]


def _blob(case):
    """The table as a policy blob: one layer, one group, no controller."""
    body = bytes([0]) + bytes(_table(case)) + bytes(N_TAGS)
    body += bytes(-len(body) % 4) + struct.pack("<%df" % (2 * N_TAGS), *([0.5] * (2 * N_TAGS)))
    blob = b"PASK" + struct.pack("<HHIIIIII", 1, 32, N_TAGS, 1, 1, case["sink"], 0, len(body)) + body
    h = 0x811C9DC5
    for x in blob:
        h = ((h ^ x) * 0x01000193) & 0xFFFFFFFF
    return blob + struct.pack("<I", h)


def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed((seed * 2654435761 + salt) % (1 << 62))


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _rows(case, seed, n, salt):
    """n rows of latents and rotary keys: normalised latents whose channels differ in scale, larger rotary keys."""
    g = _gen(seed, salt)
    gain = torch.exp(0.4 * _normal(g, case["rank"]))
    c = torch.empty(n, case["rank"], device="cuda", dtype=torch.bfloat16)
    r = torch.empty(n, case["rope"], device="cuda", dtype=torch.bfloat16)
    for i in range(0, n, 1 << 18):
        m = min(n, i + (1 << 18)) - i
        c[i:i + m] = (_normal(g, m, case["rank"]) * gain).to(torch.bfloat16)
        r[i:i + m] = (2.0 * _normal(g, m, case["rope"])).to(torch.bfloat16)
    return c, r


def _history(case, seed):
    """Padded prompts: c [B, nmax, rank], r [B, nmax, rope], tags u8 [B, nmax], lengths i32 [B] on the GPU."""
    B, n = case["batch"], case["nmax"]
    c, r = _rows(case, seed, B * n, 1)
    # Tags in a random order, each as often as the others behind the sinks, so that every seed keeps as many rows.
    lens = torch.tensor(_lengths(case), device="cuda", dtype=torch.int32)
    pos = torch.arange(n, device="cuda")[None]
    key = torch.rand(B, n, generator=_gen(seed, 2), device="cuda")
    key = torch.where(pos < case["sink"], -1.0, torch.where(pos < lens[:, None], key, 2.0))
    place = torch.argsort(torch.argsort(key, dim=1), dim=1)
    tags = ((place - case["sink"]) % N_TAGS).to(torch.uint8)
    return c.view(B, n, -1), r.view(B, n, -1), tags, lens


def _queries(case, seed):
    g = _gen(seed, 3)
    q = _normal(g, case["batch"], case["heads"], case["rank"] + case["rope"])
    return (q * (0.5 + torch.rand(case["batch"], case["heads"], 1, generator=g, device="cuda"))).to(torch.bfloat16)


def _scale(case):
    if case["op"] == "prompt":
        return 1.0 / math.sqrt(case["nope"] + case["rope"])
    return 1.0 / math.sqrt(128 + case["rope"])       # heads of 128 + rope before the absorption


def _session(case):
    from paper_2608_28276_amd.session import PaskLatentSession
    pages = sum((n + 16) // 16 for n in _lengths(case))
    all_high = case.get("keep_all") or case["hi"] == N_TAGS
    return PaskLatentSession(_blob(case), max_batch=case["batch"], n_layers=1, n_q_heads=case.get("heads", 1),
                             rank=case["rank"], rope_dim=case["rope"], max_tokens_per_seq=case["nmax"] + 1,
                             hi_pages=pages, lo_pages=0 if all_high else pages, softmax_scale=_scale(case))


def prepare(case, seed):
    s = {"case": case, "scale": _scale(case)}
    if case["op"] == "prompt":
        nq, past = _lengths(case), _pasts(case)
        cq, ck = np.cumsum([0] + nq), np.cumsum([0] + [a + b for a, b in zip(nq, past)])
        g, H = _gen(seed, 5), case["heads"]
        s["q"] = _normal(g, int(cq[-1]), H, case["nope"] + case["rope"]).to(torch.bfloat16)
        s["kv"] = _normal(g, int(ck[-1]), H, case["nope"] + case["v"]).to(torch.bfloat16)
        s["r"] = (1.5 * _normal(g, int(ck[-1]), case["rope"])).to(torch.bfloat16)
        s["lens"] = (nq, past)
        s["cu_q"], s["cu_k"] = (torch.tensor(x, device="cuda", dtype=torch.int32) for x in (cq, ck))
        s["max_q"] = max(nq)
        s["out"] = torch.empty(int(cq[-1]), H, case["v"], device="cuda", dtype=torch.bfloat16)
        s["lse"] = torch.empty(int(cq[-1]), H, device="cuda", dtype=torch.float32)
        return s
    c, r, tags, lens = _history(case, seed)
    if case["op"] in ("write_read", "read"):
        rows = sum(_kept(case))                      # a program has it from the cache's counts
        s["c_out"] = torch.empty(rows, case["rank"], device="cuda", dtype=torch.bfloat16)
        s["r_out"] = torch.empty(rows, case["rope"], device="cuda", dtype=torch.bfloat16)
        s["pos"] = torch.empty(rows, device="cuda", dtype=torch.int32)
        s["cu"] = torch.empty(case["batch"] + 1, device="cuda", dtype=torch.int32)
    if case["op"] == "decode":
        s["q"] = _queries(case, seed)
        s["out"] = torch.empty(case["batch"], case["heads"], case["rank"], device="cuda", dtype=torch.bfloat16)
        s["lse"] = torch.empty(case["batch"], case["heads"], device="cuda", dtype=torch.float32)
        if case["step"]:
            s["c_new"], s["r_new"] = _rows(case, seed, case["batch"], 4)
            s["tags_new"] = torch.randint(0, N_TAGS, (case["batch"],), generator=_gen(seed, 6), device="cuda",
                                          dtype=torch.uint8)
    if own:
        s["cache"] = _session(case)
    if case["op"] == "write_read":
        s.update(c=c, r=r, tags=tags, lens=lens)
    elif own:
        s["cache"].append(0, tags, c, r, n_new=lens)
        s["saved"] = s["cache"].save()
    else:
        s["held"] = _plain_write(case, c, r, tags, lens)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _plain_quantise(x):
    """int4 codes and fp16 scales of rows [n, rank], a scale per 32 elements."""
    x = x.float().unflatten(1, (-1, 32))
    s = torch.clamp(x.abs().amax(-1, keepdim=True) / 7.0, max=65504.0).half()
    q = torch.round(x / s.float().clamp_min(2.0 ** -40)).clamp(-7, 7)
    return torch.where(s > 0, q, torch.zeros_like(q)).to(torch.int8).flatten(1), s[:, :, 0]


def _plain_value(q, s):
    return (q.float().unflatten(1, (-1, 32)) * s.float()[:, :, None]).flatten(1).bfloat16()


def _plain_actions(case, tags, pos):
    a = torch.tensor(_table(case), device=tags.device, dtype=torch.int32)[tags.long()]
    forced = (pos < case["sink"]) | bool(case.get("keep_all"))
    return torch.where(forced, torch.full_like(a, HIGH), a)


def _plain_write(case, c, r, tags, lens):
    """The cache as plain tensors: per store the entries of all sequences, by sequence and position."""
    B, n = tags.shape
    pos = torch.arange(n, device=tags.device, dtype=torch.int32)[None].expand(B, n)
    act = torch.where(pos < lens[:, None], _plain_actions(case, tags, pos), torch.zeros_like(pos))
    held = {"counts": torch.stack([(act == HIGH).sum(1), (act == LOW).sum(1)]).tolist(), "lens": lens}
    for name, a in (("hi", HIGH), ("lo", LOW)):
        at = (act == a).reshape(-1).nonzero()[:, 0]
        rows = c.reshape(B * n, -1)[at]
        held[name] = ((rows,) if a == HIGH else _plain_quantise(rows)) + (r.reshape(B * n, -1)[at],)
        held[name + "_at"] = at
    return held


def _plain_read(case, held):
    """Kept rows in (sequence, position) order."""
    at = torch.cat([held["hi_at"], held["lo_at"]])
    order = torch.argsort(at)
    c = torch.cat([held["hi"][0], _plain_value(held["lo"][0], held["lo"][1])])[order]
    r = torch.cat([held["hi"][1], held["lo"][2]])[order]
    per = torch.tensor(held["counts"], device=at.device).sum(0)
    cu = torch.cat([per.new_zeros(1), per.cumsum(0)]).int()
    return c, r, (at[order] % case["nmax"]).int(), cu


def _plain_decode(s):
    case, held = s["case"], s["held"]
    B, R = case["batch"], case["rank"]
    counters = torch.zeros(B, 6, device="cuda", dtype=torch.int32)
    counters[:, :2] = torch.tensor(held["counts"], device="cuda", dtype=torch.int32).t()
    counters[:, 2] = held["lens"]
    counters[:, 3] = held["lens"] - counters[:, 0] - counters[:, 1]
    counters[:, 4] = torch.clamp(held["lens"], max=case["sink"])
    new = None
    if case["step"]:
        act = _plain_actions(case, s["tags_new"], held["lens"])
        counters[:, 0] += (act == HIGH).int()
        counters[:, 1] += (act == LOW).int()
        counters[:, 3] += (act == DROP).int()
        counters[:, 4] += (held["lens"] < case["sink"]).int()
        counters[:, 2] += 1
        low = _plain_value(*_plain_quantise(s["c_new"]))
        new = torch.where((act == LOW)[:, None], low, s["c_new"]).float()
    outs, lses, h, l = [], [], 0, 0
    for b, (n, m) in enumerate(zip(*held["counts"])):
        c = [held["hi"][0][h:h + n].float(),
             _plain_value(held["lo"][0][l:l + m], held["lo"][1][l:l + m]).float()]
        r = [held["hi"][1][h:h + n].float(), held["lo"][2][l:l + m].float()]
        if new is not None:
            c.append(new[b:b + 1])
            r.append(s["r_new"][b:b + 1].float())
        c, r = torch.cat(c), torch.cat(r)
        q = s["q"][b].float()
        sc = (q[:, :R] @ c.t() + q[:, R:] @ r.t()) * s["scale"]
        if new is not None:
            sc[:, -1] = torch.where(act[b] == DROP, -torch.inf, sc[:, -1])
        o, lse = _plain_softmax(sc, c)
        outs.append(o)
        lses.append(lse)
        h, l = h + n, l + m
    return [torch.stack(outs).bfloat16(), torch.stack(lses), counters]


def _plain_softmax(sc, v):
    """Rows of softmax(sc) v and their ln sum exp; a row that sees nothing gives 0 and -inf."""
    if sc.shape[-1] == 0:
        return sc.new_zeros(*sc.shape[:-1], v.shape[-1]), sc.new_full(sc.shape[:-1], -torch.inf)
    top = sc.amax(-1, keepdim=True)
    seen = top > -torch.inf
    p = torch.exp(sc - torch.where(seen, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(seen, total, torch.ones_like(total))
    return o, (torch.log(total) + top)[..., 0]


def _plain_prompt(s):
    case = s["case"]
    D, H = case["nope"], case["heads"]
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    a = b = 0
    for n, m in zip(*s["lens"]):
        nk = n + m
        hidden = torch.arange(nk, device="cuda")[None] > torch.arange(n, device="cuda")[:, None] + m
        step = max(1, min(H, (1 << 28) // (n * nk)))
        for h in range(0, H, step):
            e = min(H, h + step)
            q = s["q"][a:a + n, h:e].float().transpose(0, 1).contiguous()
            kv = s["kv"][b:b + nk, h:e].float().transpose(0, 1).contiguous()
            sc = torch.matmul(q[:, :, :D].contiguous(), kv[:, :, :D].transpose(1, 2).contiguous())
            sc += torch.matmul(q[:, :, D:], s["r"][b:b + nk].float().t())
            sc = (sc * s["scale"]).masked_fill(hidden, -torch.inf)
            o, x = _plain_softmax(sc, kv[:, :, D:].contiguous())
            out[a:a + n, h:e] = o.transpose(0, 1).bfloat16()
            lse[a:a + n, h:e] = x.t()
        a, b = a + n, b + nk
    return [out, lse]


def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if op == "prompt":
        if not own:
            return _plain_prompt(s)
        from paper_2608_28276_amd.latent import prompt_attn
        prompt_attn(s["q"], s["kv"], s["r"], s["out"], s["lse"], s["cu_q"], s["cu_k"], s["max_q"], s["scale"])
        return [s["out"], s["lse"]]
    if not own:
        if op == "decode":
            return _plain_decode(s)
        return list(_plain_read(case, s["held"] if op == "read" else
                                _plain_write(case, s["c"], s["r"], s["tags"], s["lens"])))
    cache = s["cache"]
    if op == "decode":
        if case["step"]:                             # the same step again, as after a rejected draft
            cache.restore(s["saved"])
            cache.decode(0, s["q"], s["out"], s["lse"], s["tags_new"], s["c_new"], s["r_new"])
        else:
            cache.decode(0, s["q"], s["out"], s["lse"])
        return [s["out"], s["lse"], cache.counters()[:, 0, :6]]
    if op == "write_read":
        cache.reset()
        cache.append(0, s["tags"], s["c"], s["r"], n_new=s["lens"], keep_all=case["keep_all"])
    cache.read(0, s["c_out"], s["r_out"], s["pos"], s["cu"])
    return [s["c_out"], s["r_out"], s["pos"], s["cu"]]


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------
def _exact_entries(case, c, r, tags, n, p0=0):
    """One sequence's kept entries: float64 latents and rotary keys, positions, and (HIGH, LOW, DROP, sink) counts."""
    table = np.array(_table(case))
    action = table[tags.cpu().numpy()[:n].astype(np.int64)]
    pos = np.arange(p0, p0 + n)
    first = pos < case["sink"]
    if case.get("keep_all"):
        first = np.ones(n, bool)
    action = np.where(first, HIGH, action)
    keep = torch.from_numpy(np.flatnonzero(action != DROP)).cuda()
    x = c[keep].double()
    g = x.reshape(len(keep), case["rank"] // 32, 32)
    scale = (g.abs().max(-1).values / 7.0).clamp(max=65504.0).to(torch.float16).double()[..., None]
    ratio = torch.where(scale > 0, g / scale.clamp(min=1e-30), torch.zeros_like(g))
    coded = (torch.clamp(torch.round(ratio), -7.0, 7.0) * scale).to(torch.bfloat16).double().reshape(x.shape)
    is_low = torch.from_numpy(action == LOW).cuda()[keep]
    counts = [int((action == a).sum()) for a in (HIGH, LOW, DROP)] + [int(first.sum())]
    return torch.where(is_low[:, None], coded, x), r[keep].double(), pos[action != DROP], counts


def _exact_attention(logits, values):
    if logits.shape[-1] == 0:
        return logits.new_zeros(logits.shape[0], values.shape[-1]), logits.new_full(logits.shape[:1], -math.inf)
    lse = torch.logsumexp(logits, -1)
    weights = torch.where(torch.isinf(lse)[:, None], torch.zeros_like(logits), torch.exp(logits - lse[:, None]))
    return weights @ values, lse


def exact(case, seed):
    if case["op"] == "prompt":
        global own
        was, own = own, False
        s = prepare(case, seed)
        own = was
        return _exact_prompt(case, s)
    c, r, tags, lens = _history(case, seed)
    B = case["batch"]
    if case["op"] == "decode":
        q = _queries(case, seed).double()
        o = torch.empty(B, case["heads"], case["rank"], device="cuda", dtype=torch.float64)
        lse = torch.empty(B, case["heads"], device="cuda", dtype=torch.float64)
        counters = torch.zeros(B, 6, dtype=torch.int32)
        if case["step"]:
            c_new, r_new = _rows(case, seed, B, 4)
            tags_new = torch.randint(0, N_TAGS, (B,), generator=_gen(seed, 6), device="cuda", dtype=torch.uint8)
        for b, n in enumerate(_lengths(case)):
            x, y, _, k = _exact_entries(case, c[b], r[b], tags[b], n)
            if case["step"]:
                x1, y1, _, k1 = _exact_entries(case, c_new[b:b + 1], r_new[b:b + 1], tags_new[b:b + 1], 1, n)
                x, y, k, n = torch.cat([x, x1]), torch.cat([y, y1]), [i + j for i, j in zip(k, k1)], n + 1
            logits = torch.cat([x, y], 1) @ q[b].t() * _scale(case)
            o[b], lse[b] = _exact_attention(logits.t(), x)
            counters[b] = torch.tensor([k[0], k[1], n, k[2], k[3], 0])
        return [o, lse, counters]
    parts = [_exact_entries(case, c[b], r[b], tags[b], n) for b, n in enumerate(_lengths(case))]
    cu = np.cumsum([0] + [len(p[2]) for p in parts]).astype(np.int32)
    return [torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts]),
            torch.from_numpy(np.concatenate([p[2] for p in parts]).astype(np.int32)), torch.from_numpy(cu)]


def _exact_prompt(case, s):
    H, D, V = case["heads"], case["nope"], case["v"]
    out = torch.zeros(s["q"].shape[0], H, V, device="cuda", dtype=torch.float64)
    lse = torch.zeros(s["q"].shape[0], H, device="cuda", dtype=torch.float64)
    cq, ck = s["cu_q"].tolist(), s["cu_k"].tolist()
    for b in range(case["batch"]):
        nq, nk = cq[b + 1] - cq[b], ck[b + 1] - ck[b]
        r = s["r"][ck[b]:ck[b + 1]].double()
        for h in range(H):
            kv = s["kv"][ck[b]:ck[b + 1], h].double()
            keys = torch.cat([kv[:, :D], r], 1)
            for i in range(0, nq, 4096):
                rows = torch.arange(i, min(nq, i + 4096), device="cuda")
                logits = s["q"][cq[b] + i:cq[b] + i + len(rows), h].double() @ keys.t() * s["scale"]
                seen = torch.arange(nk, device="cuda")[None] <= rows[:, None] + (nk - nq)
                logits = torch.where(seen, logits, torch.full_like(logits, -math.inf))
                a = cq[b] + i
                out[a:a + len(rows), h], lse[a:a + len(rows), h] = _exact_attention(logits, kv[:, D:])
    return [out, lse]

