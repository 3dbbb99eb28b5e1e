"""Rotary positions and attention of many query tokens over the mixed cache,
as measurable cases.

A turn or a prompt chunk goes through a grouped-query layer in three calls: its
queries and keys are rotated at the positions that its tokens take, keys and
values are appended (the table keeps a token bf16, int4 with an fp16 scale per
32 elements, or drops it; the last `window` positions stay bf16), and every
query attends what the cache keeps at its position and before.  Two of those
are measured here:

  rope    rotation of a chunk's queries and keys: half or interleaved pairs, the
          whole head or a part, frequencies scaled for long contexts, rows of a
          fused projection's output;
  prompt  attention of the last n tokens of each sequence over the resident
          history, those tokens included: a draft's few, a turn's, a prompt's.
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
def _rope(name=None, **kw):
    case = dict(op="rope", batch=1, nmin=1, nmax=1, q_heads=32, k_heads=8, head_dim=128, rot_first=0, rot_dim=128,
                interleaved=False, base=1e6, scaling="plain", factor=1.0, original=4096, far=32768, fused=True,
                explicit=False)
    case.update(kw)
    return _named(name, case)


# hi, lo: how many of the 16 tags the table keeps HIGH and LOW; the others are dropped.  nmin .. nmax queries of a
# sequence come after pmin .. pmax tokens.
def _prompt(name=None, **kw):
    case = dict(op="prompt", batch=1, nmin=4, nmax=4, pmin=0, pmax=0, q_heads=32, kv_heads=8, head_dim=128, hi=6, lo=6,
                sink=0, window=0)
    case.update(kw)
    return _named(name, case)


def _named(name, case):
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # One user's next token: latency.
        _rope("rope_step_b1"),
        # A serving batch's step at far positions, frequencies scaled by parts.
        _rope("rope_step_b64_far", batch=64, q_heads=64, scaling="parts", factor=4.0, original=32768, far=131072),
        # Chunks of a layer with latent attention: the rotary part at the end of each query head, interleaved.
        _rope("rope_latent_b8_chunk", batch=8, nmin=200, nmax=1024, q_heads=20, k_heads=0, head_dim=192, rot_first=128,
              rot_dim=64, interleaved=True, base=1e4, fused=False),
        # A packed batch whose rows come with their positions; an odd number of pairs in a part of the head.
        _rope("rope_packed_odd", nmin=5003, nmax=5003, q_heads=24, k_heads=3, head_dim=128, rot_dim=54,
              scaling="linear", factor=2.5, explicit=True),
        # Prompts of a serving batch.
        _rope("rope_prompt_b16", batch=16, nmin=500, nmax=8192, scaling="base", factor=8.0),
        # One user's draft of four tokens, verified: latency.
        _prompt("prompt_draft_b1", pmin=2048, pmax=2048),
        # A serving batch's drafts: reading the cache is all the work.
        _prompt("prompt_draft_b64", batch=64, nmin=5, nmax=5, pmin=1024, pmax=8192),
        # Short ragged turns over small heads.
        _prompt("prompt_b4_small", batch=4, nmin=1, nmax=256, pmin=0, pmax=300, q_heads=8, kv_heads=2, head_dim=64),
        # One long labelled context, most of it int4 or dropped, and a turn of an odd length.
        _prompt("prompt_turn_b1_32k", nmin=333, nmax=333, pmin=32000, pmax=32000, q_heads=64, hi=3, lo=9, sink=16),
        # A batch's turns with a recent window, some of them the sequence's first.
        _prompt("prompt_turn_b8_window", batch=8, nmin=16, nmax=700, pmin=0, pmax=6000, hi=4, lo=7, window=64),
        # Chunks of labelled prompts behind earlier chunks, most of them int4 or dropped.
        _prompt("prompt_chunk_b4_labelled", batch=4, nmin=1000, nmax=4096, pmin=500, pmax=8192, hi=3, lo=9, sink=16),
        # One long prompt that the table does not govern.
        _prompt("prompt_b1_8k", nmin=8192, nmax=8192, hi=16, lo=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _range(rng, lo, hi):
    most = _log_int(rng, lo, hi)
    return max(lo, int(most * rng.uniform(0.05, 1.0))), most


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        b, f = most.get(c["op"], (0, 0))
        most[c["op"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    while True:
        nmin, nmax = _range(rng, 1, 8192)
        batch = _log_int(rng, 1, 256)
        if rng.random() < 0.4:
            head_dim = rng.choice([64, 96, 128, 128, 192, 256])
            rot_dim = rng.choice([head_dim, head_dim, head_dim // 2, 2 * rng.randint(2, head_dim // 2)])
            explicit = rng.random() < 0.25
            c = _rope(batch=1 if explicit else batch, nmin=nmax if explicit else nmin, nmax=nmax,
                      q_heads=_log_int(rng, 1, 64), k_heads=rng.choice([0, 1, 2, 3, 8]), head_dim=head_dim,
                      rot_first=rng.choice([0, 0, head_dim - rot_dim]), rot_dim=rot_dim,
                      interleaved=rng.random() < 0.5, base=rng.choice([1e4, 5e5, 1e6]),
                      scaling=rng.choice(["plain", "linear", "base", "parts"]), factor=rng.uniform(1.0, 16.0),
                      original=rng.choice([2048, 4096, 32768]), far=_log_int(rng, 1, 1 << 20),
                      fused=rng.random() < 0.5, explicit=explicit)
        else:
            hi = rng.randint(0, 16)
            kv_heads = rng.choice([1, 2, 3, 4, 8, 8])
            pmin, pmax = _range(rng, 1, 65536) if rng.random() < 0.8 else (0, 0)
            c = _prompt(batch=batch, nmin=nmin, nmax=nmax, pmin=pmin, pmax=pmax, q_heads=kv_heads * rng.choice([1, 2, 4, 8]),
                        kv_heads=kv_heads, head_dim=rng.choice([64, 128, 128]), hi=hi, lo=rng.randint(0, 16 - hi),
                        sink=rng.choice([0, 0, 4, 16]), window=rng.choice([0, 0, 0, _log_int(rng, 1, 512)]))
        w = work(c)
        if 1e4 < w["bytes"] <= most[c["op"]][0] and w["flops"] <= most[c["op"]][1] and _resident(c) < 8e9:
            return c


def _resident(case):
    """Bytes of the padded inputs of a case."""
    if case["op"] == "rope":
        return case["batch"] * case["nmax"] * (case["q_heads"] + 2 * case["k_heads"]) * case["head_dim"] * 2
    return case["batch"] * (case["pmax"] + case["nmax"]) * case["kv_heads"] * case["head_dim"] * 4


def _spread(case, lo, hi, salt):
    """One size of each sequence: between lo and hi, the same for every seed."""
    r = random.Random(lo * 1000003 + hi * 101 + case["batch"] * 7 + salt)
    n = [r.randint(lo, hi) for _ in range(case["batch"])]
    n[r.randrange(len(n))] = hi
    return n


def _news(case):
    return _spread(case, case["nmin"], case["nmax"], 1)


def _pasts(case):
    return _spread(case, case["pmin"], case["pmax"], 2)


def _kept(case, n):
    """HIGH (the window's among them) and LOW entries of n tokens: tags come equally often behind the sinks."""
    w = min(n, case["window"])
    s = min(n - w, case["sink"])
    rest = n - w - s
    return s + w + rest * case["hi"] / N_TAGS, rest * case["lo"] / N_TAGS


def work(case):
    if case["op"] == "rope":
        rows = sum(_news(case)) * (case["q_heads"] + case["k_heads"])
        return {"bytes": rows * case["head_dim"] * 4, "flops": rows * case["rot_dim"] * 3}
    D, H, KV = case["head_dim"], case["q_heads"], case["kv_heads"]
    n_bytes, pairs, nq = 0.0, 0.0, 0
    for n, m in zip(_news(case), _pasts(case)):
        hi, lo = _kept(case, n + m)
        n_bytes += KV * (hi * 4 * D + lo * (D + D / 8))
        before, after = sum(_kept(case, m)) if m else 0.0, hi + lo
        pairs += n * (before + after + 1) / 2
        nq += n
    return {"bytes": int(n_bytes) + nq * H * (4 * D + 4), "flops": int(4 * D * H * pairs)}


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed((seed * 2654435761 + salt) % (1 << 62))


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _bf16(g, n, *shape, gain=1.0):
    """bf16 [n, *shape], normal with the given gains, made in pieces."""
    x = torch.empty(n, *shape, device="cuda", dtype=torch.bfloat16)
    step = max(1, (1 << 26) // math.prod(shape))
    for i in range(0, n, step):
        m = min(n, i + step) - i
        x[i:i + m] = (_normal(g, m, *shape) * gain).to(torch.bfloat16)
    return x


def _table(case):
    """Action of each tag: the table keeps `hi` tags HIGH, `lo` LOW and drops the rest, in a mixed order."""
    acts = [HIGH] * case["hi"] + [LOW] * case["lo"] + [DROP] * (N_TAGS - case["hi"] - case["lo"])
    return [acts[(5 * z + 3) % N_TAGS] for z in range(N_TAGS)]


def _blob(case):
    """The table as a policy blob: one layer, one group, no controller."""
    body = bytes([0]) + bytes(_table(case)) + bytes(N_TAGS)
    body += bytes(-len(body) % 4) + struct.pack("<%df" % (2 * N_TAGS), *([0.5] * (2 * N_TAGS)))
    blob = b"PASK" + struct.pack("<HHIIIIII", 1, 32, N_TAGS, 1, 1, case["sink"], case["window"], len(body)) + body
    h = 0x811C9DC5
    for x in blob:
        h = ((h ^ x) * 0x01000193) & 0xFFFFFFFF
    return blob + struct.pack("<I", h)


def _history(case, seed):
    """Padded tokens, the queries' own at the end: k, v [B, n, KV, D], tags u8 [B, n], lengths i32 [B] on the GPU."""
    B, KV, D = case["batch"], case["kv_heads"], case["head_dim"]
    lens = [a + b for a, b in zip(_news(case), _pasts(case))]
    n, g = max(lens), _gen(seed, 1)
    gain = torch.exp(0.4 * _normal(g, KV, D))        # channels differ in scale, keys' more than values'
    k = _bf16(g, B * n, KV, D, gain=gain).view(B, n, KV, D)
    v = _bf16(g, B * n, KV, D, gain=gain.sqrt()).view(B, n, KV, D)
    # Tags in a random order, each as often as the others behind the sinks, so that every seed keeps as many entries.
    lens = torch.tensor(lens, device="cuda", dtype=torch.int32)
    pos = torch.arange(n, device="cuda")[None]
    key = torch.rand(B, n, generator=_gen(seed, 2), device="cuda")
    key = torch.where(pos < case["sink"], -1.0, torch.where(pos < lens[:, None], key, 2.0))
    place = torch.argsort(torch.argsort(key, dim=1), dim=1)
    return k, v, ((place - case["sink"]) % N_TAGS).to(torch.uint8), lens


def _queries(case, seed):
    g = _gen(seed, 3)
    shape = (case["batch"] * case["nmax"], case["q_heads"], case["head_dim"])
    return _bf16(g, *shape, gain=0.5 + torch.rand(case["q_heads"], 1, generator=g, device="cuda"))


def _rope_inputs(case, seed):
    B, n, Hq, Hk, D = (case[x] for x in ("batch", "nmax", "q_heads", "k_heads", "head_dim"))
    s, g = {}, _gen(seed, 4)
    if case["fused"]:                                # rows of one projection: queries, keys, values
        rows = _bf16(g, B * n, (Hq + 2 * Hk) * D).view(B, n, -1)
        s["q"] = rows[:, :, :Hq * D].unflatten(2, (Hq, D))
        s["k"] = rows[:, :, Hq * D:(Hq + Hk) * D].unflatten(2, (Hk, D)) if Hk else None
    else:
        s["q"] = _bf16(g, B * n, Hq, D).view(B, n, Hq, D)
        s["k"] = _bf16(g, B * n, Hk, D).view(B, n, Hk, D) if Hk else None
    s["q_out"] = torch.zeros(B, n, Hq, D, device="cuda", dtype=torch.bfloat16)
    s["k_out"] = torch.zeros(B, n, Hk, D, device="cuda", dtype=torch.bfloat16) if Hk else None
    s["n_new"] = torch.tensor(_news(case), device="cuda", dtype=torch.int32)
    s["first"] = torch.randint(0, case["far"], (B,), generator=g, device="cuda", dtype=torch.int32)
    s["pos"] = None
    if case["explicit"]:                             # several sequences' rows behind each other, each from its start on
        cut = torch.rand(B, n, generator=g, device="cuda") < 0.01
        row = torch.arange(n, device="cuda", dtype=torch.int32)[None]
        start = torch.where(cut, row, torch.zeros_like(row)).cummax(1).values
        s["pos"] = (row - start + torch.where(start > 0, start * 37 % case["far"], s["first"][:, None])).int().contiguous()
    return s


def _frequencies(case):
    """Angle of one position, per pair, in 64 bits."""
    R = case["rot_dim"]
    base = case["base"]
    if case["scaling"] == "base" and R > 2:
        base *= case["factor"] ** (R / (R - 2))
    f = base ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    if case["scaling"] == "linear":
        f = f / case["factor"]
    elif case["scaling"] == "parts":
        keep = ((case["original"] * f / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f * keep + f / case["factor"] * (1.0 - keep)
    return f.cuda()


def _magnitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "parts" else 1.0


def _make_rope(case):
    from paper_2608_28276_amd import prompt
    kind = {"plain": prompt.PASK_ROPE_PLAIN, "linear": prompt.PASK_ROPE_LINEAR, "base": prompt.PASK_ROPE_BASE,
            "parts": prompt.PASK_ROPE_PARTS}[case["scaling"]]
    return prompt.make_rope(case["head_dim"], case["base"], rot_first=case["rot_first"], rot_dim=case["rot_dim"],
                            layout=prompt.PASK_ROPE_INTERLEAVED if case["interleaved"] else prompt.PASK_ROPE_HALF,
                            scaling=kind, factor=case["factor"], original_len=case["original"], low_turns=1.0,
                            high_turns=32.0, magnitude=_magnitude(case))


def _session(case):
    from paper_2608_28276_amd.session import PaskSession
    lens = [a + b for a, b in zip(_news(case), _pasts(case))]
    pages = sum((n + 15) // 16 for n in lens)
    return PaskSession(_blob(case), max_batch=case["batch"], n_layers=1, n_q_heads=case["q_heads"],
                       n_kv_heads=case["kv_heads"], head_dim=case["head_dim"],
                       max_tokens_per_seq=max(lens + [case["window"]]), hi_pages=pages,
                       lo_pages=pages if case["lo"] else 0)


def prepare(case, seed):
    if case["op"] == "rope":
        s = _rope_inputs(case, seed)
        if own:
            s["rope"] = _make_rope(case)
        else:
            s["freq"] = _frequencies(case)
        s["case"] = case
        return s
    k, v, tags, lens = _history(case, seed)
    B, n, H, D = case["batch"], case["nmax"], case["q_heads"], case["head_dim"]
    s = {"case": case, "q": _queries(case, seed).view(B, n, H, D), "scale": 1.0 / math.sqrt(D)}
    s["n_q"] = torch.tensor(_news(case), device="cuda", dtype=torch.int32)
    s["out"] = torch.zeros(B, n, H, D, device="cuda", dtype=torch.bfloat16)
    s["lse"] = torch.zeros(B, n, H, device="cuda", dtype=torch.float32)
    if own:
        s["cache"] = _session(case)
        s["cache"].append(0, tags, k, v, n_new=lens)
    else:
        s["held"] = _plain_cache(case, k, v, tags)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _plain_rope(s):
    case = s["case"]
    f, R, at = s["freq"], case["rot_dim"], case["rot_first"]
    row = torch.arange(case["nmax"], device="cuda")
    b, i = (row[None] < s["n_new"][:, None]).nonzero(as_tuple=True)
    p = s["pos"][b, i].double() if s["pos"] is not None else s["first"][b].double() + i.double()
    a = p[:, None] * f[None]
    cos, sin = ((t * _magnitude(case)).float()[:, None] for t in (torch.cos(a), torch.sin(a)))
    outs = []
    for x, out in ((s["q"], s["q_out"]), (s["k"], s["k_out"])):
        if x is None:
            continue
        y = x[b, i].float()
        r = y[:, :, at:at + R]
        if case["interleaved"]:
            u, w = r[:, :, 0::2], r[:, :, 1::2]
            r = torch.stack([u * cos - w * sin, u * sin + w * cos], -1).flatten(2)
        else:
            u, w = r[:, :, :R // 2], r[:, :, R // 2:]
            r = torch.cat([u * cos - w * sin, u * sin + w * cos], -1)
        out[b, i] = torch.cat([y[:, :, :at], r, y[:, :, at + R:]], -1).to(torch.bfloat16)
        outs.append(out)
    return outs


def _plain_quantise(x):
    """int4 codes and fp16 scales of rows [n, KV, D], a scale per 32 elements."""
    x = x.float().unflatten(2, (-1, 32))
    s = torch.clamp(x.abs().amax(-1, keepdim=True) / 7.0, max=65504.0).half()
    q = torch.round(x / s.float().clamp_min(2.0 ** -40)).clamp(-7, 7)
    return torch.where(s > 0, q, torch.zeros_like(q)).to(torch.int8).flatten(2), s[..., 0]


def _plain_cache(case, k, v, tags):
    """Per sequence the bf16 entries (the window's last), the int4 ones, and their positions."""
    table = torch.tensor(_table(case), device="cuda")
    held = []
    for b, (n, m) in enumerate(zip(_news(case), _pasts(case))):
        pos = torch.arange(n + m, device="cuda")
        act = torch.where((pos < case["sink"]) | (pos >= n + m - case["window"]), HIGH, table[tags[b, :n + m].long()])
        hi, lo = (act == HIGH).nonzero()[:, 0], (act == LOW).nonzero()[:, 0]
        held.append((k[b, hi], v[b, hi], _plain_quantise(k[b, lo]), _plain_quantise(v[b, lo]), torch.cat([hi, lo])))
    return held


def _plain_values(q, s):
    return (q.float().unflatten(2, (-1, 32)) * s.float()[..., None]).flatten(2)


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
    KV, G = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    for b, (n, m) in enumerate(zip(_news(case), _pasts(case))):
        kh, vh, kl, vl, pos = s["held"][b]
        k = torch.cat([kh.float(), _plain_values(*kl)]).permute(1, 2, 0).contiguous()          # [KV, D, entries]
        v = torch.cat([vh.float(), _plain_values(*vl)]).transpose(0, 1).contiguous()
        step = max(1, (1 << 29) // max(1, KV * G * len(pos)))
        for i in range(0, n, step):
            e = min(n, i + step)
            q = s["q"][b, i:e].float().unflatten(1, (KV, G)).permute(1, 0, 2, 3).flatten(1, 2).contiguous()
            sc = torch.matmul(q, k) * s["scale"]                                               # [KV, rows * G, entries]
            hidden = pos[None] > torch.arange(m + i, m + e, device="cuda")[:, None]
            sc = sc.masked_fill(hidden.repeat_interleave(G, 0)[None], -torch.inf)
            o, lse = _plain_softmax(sc, v)
            s["out"][b, i:e] = o.unflatten(1, (e - i, G)).transpose(0, 1).flatten(1, 2).to(torch.bfloat16)
            s["lse"][b, i:e] = lse.unflatten(1, (e - i, G)).transpose(0, 1).flatten(1, 2)
    return [s["out"], s["lse"]]


def run(state):
    s, case = state, state["case"]
    if case["op"] == "rope":
        if not own:
            return _plain_rope(s)
        from paper_2608_28276_amd.prompt import rotate
        first = None if case["explicit"] else s["first"]
        rotate(s["rope"], s["q"], s["q_out"], s["k"], s["k_out"], first=first, pos=s["pos"], n_new=s["n_new"])
        return [s["q_out"]] + ([] if s["k_out"] is None else [s["k_out"]])
    if not own:
        return _plain_prompt(s)
    s["cache"].prompt(0, s["q"], s["out"], s["lse"], n_q=s["n_q"])
    return [s["out"], s["lse"]]


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------
def exact(case, seed):
    return _exact_rope(case, seed) if case["op"] == "rope" else _exact_prompt(case, seed)


def _exact_rope(case, seed):
    s, R, at = _rope_inputs(case, seed), case["rot_dim"], case["rot_first"]
    i = np.arange(R // 2, dtype=np.float64)
    base = case["base"]
    if case["scaling"] == "base" and R > 2:
        base = base * math.pow(case["factor"], R / (R - 2.0))
    theta = np.power(base, -2.0 * i / R)
    if case["scaling"] == "linear":
        theta /= case["factor"]
    if case["scaling"] == "parts":
        turns = case["original"] / (2 * math.pi / theta)               # over the original length
        g = np.clip((turns - 1.0) / 31.0, 0.0, 1.0)
        theta = (1 - g) * theta / case["factor"] + g * theta
    theta = torch.from_numpy(theta).cuda()
    first, second = (at + 2 * torch.arange(R // 2), at + 2 * torch.arange(R // 2) + 1) if case["interleaved"] else \
        (at + torch.arange(R // 2), at + R // 2 + torch.arange(R // 2))
    first, second = first.cuda(), second.cuda()
    outs = []
    for x in (s["q"], s["k"]):
        if x is None:
            continue
        out = torch.zeros(x.shape, device="cuda", dtype=torch.float64)
        for b, n in enumerate(_news(case)):
            p = s["pos"][b, :n] if s["pos"] is not None else s["first"][b] + torch.arange(n, device="cuda")
            turn = torch.polar(torch.full((n, R // 2), _magnitude(case), device="cuda", dtype=torch.float64),
                               torch.outer(p.double(), theta))[:, None]
            for h in range(0, x.shape[2], 8):
                y = x[b, :n, h:h + 8].double()
                z = torch.complex(y[..., first], y[..., second]) * turn
                y[..., first], y[..., second] = z.real, z.imag
                out[b, :n, h:h + 8] = y
        outs.append(out)
    return outs


def _exact_prompt(case, seed):
    k, v, tags, _ = _history(case, seed)
    B, N, H, KV, D = (case[x] for x in ("batch", "nmax", "q_heads", "kv_heads", "head_dim"))
    q = _queries(case, seed).view(B, N, H, D)
    out = torch.zeros(B, N, H, D, device="cuda", dtype=torch.float64)
    lse = torch.zeros(B, N, H, device="cuda", dtype=torch.float64)
    table = np.array(_table(case))
    for b, (n, m) in enumerate(zip(_news(case), _pasts(case))):
        position = np.arange(n + m)
        action = table[tags[b, :n + m].cpu().numpy().astype(np.int64)]
        action[:case["sink"]] = HIGH
        action[max(0, n + m - case["window"]):] = HIGH
        keep = np.flatnonzero(action != DROP)
        low = torch.from_numpy(action[keep] == LOW).cuda()[:, None, None]
        at = torch.from_numpy(position[keep]).cuda()
        kd, vd = (torch.where(low, _exact_coded(x[b, at].double()), x[b, at].double()) for x in (k, v))
        for h in range(H):
            keys, values = kd[:, h * KV // H], vd[:, h * KV // H]
            for i in range(0, n, 4096):
                rows = torch.arange(i, min(n, i + 4096), device="cuda")
                logits = q[b, rows, h].double() @ keys.t() / math.sqrt(D)
                logits = torch.where(at[None] <= rows[:, None] + m, logits, torch.full_like(logits, -math.inf))
                if logits.shape[1] == 0:
                    lse[b, rows, h] = -math.inf
                    continue
                total = torch.logsumexp(logits, -1)
                weights = torch.where(torch.isinf(total)[:, None], torch.zeros_like(logits),
                                      torch.exp(logits - total[:, None]))
                out[b, rows, h], lse[b, rows, h] = weights @ values, total
    return [out, lse]


def _exact_coded(x):
    """What int4 codes stand for: clamp(round(x / s)) s, s = fp16(absmax / 7) of each 32 elements."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    scale = (g.abs().amax(-1, keepdim=True) / 7.0).clamp(max=65504.0).to(torch.float16).double()
    ratio = torch.where(scale > 0, g / scale.clamp(min=1e-30), torch.zeros_like(g))
    return (torch.clamp(torch.round(ratio), -7.0, 7.0) * scale).reshape(x.shape)
