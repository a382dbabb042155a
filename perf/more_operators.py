"""Operators of a cache of pages and of the rows on their way into it, as cases that can be timed and compared.

* ``rotate``   rows of queries, keys and values as a projection leaves them (token by token, all heads of a token side by side): queries
               and keys are normed per head (root mean square) where the model does that, rotated by their positions on one
               axis or several, and laid out head by head.
* ``append``   rows of keys and values into a cache of pages.  Rotated ones come from a projection as above and the queries of the same
               pass are returned too; in 8 bits (int8 or e4m3, a scale per row) they come ready, and what the cache now holds is read back.
* ``read``     a cache of pages read back into one array of rows per KV head.
* ``attend``   attention of one new token of every sequence over a cache of pages.

A page holds `page` slots of one KV head (``per_head``: every KV head of a sequence has a table and a length of its own, as eviction per head
leaves them) or of all KV heads of a sequence, which then share a table and a length.  Pages lie anywhere in the pool.
"""
import math

import torch

own = False   # False: plain torch; True: the framework's entry points

DEVICE = "cuda:0"
QMAX = {"i8": 127.0, "e4m3": 448.0}
LEAST = 2.0 ** -100     # a row whose largest magnitude is below is held as zeros
EPS = 1e-6


def _case(name, kind, B, Hq, Hkv, d, dtype, P=0, ragged=0, n=0, page=16, per_head=False, code="", norm=False, rot=0, pairing="halves",
          axes=1, in_turn=False, far=0):
    c = dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, P=P, ragged=ragged, n=n, page=page, per_head=per_head, code=code,
             norm=norm, rot=rot, pairing=pairing, axes=axes, in_turn=in_turn, far=far)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token of eight conversations that are far into their contexts: latency
        _case("rotate_token", "rotate", 8, 32, 8, 128, "bf16", n=1, norm=True, rot=128, far=100000),
        # images and text in one prompt: positions in time, height and width, pairs of channels dealt to the axes in blocks
        _case("rotate_prompt_axes", "rotate", 4, 32, 8, 128, "bf16", n=4096, norm=True, rot=128, axes=3),
        # a small fp32 model that rotates half of its channels, neighbours as pairs; nothing a multiple of a tile
        _case("rotate_odd_f32", "rotate", 3, 24, 3, 64, "f32", n=701, norm=True, rot=32, pairing="neighbours"),
        # the new token of 64 sequences that are served together
        _case("append_token", "append", 64, 32, 8, 128, "bf16", P=2048, ragged=1000, n=1, norm=True, rot=128),
        # the prompts of a batch, padded to the longest, straight from the projection into the pages
        _case("append_prompt", "append", 8, 32, 8, 128, "bf16", P=0, ragged=1500, n=4096, norm=True, rot=128),
        # prompts of a 7B model into int8, and the rows as the cache has them for the prompt's own attention
        _case("append_prompt_i8", "append", 16, 32, 32, 128, "bf16", P=0, ragged=1500, n=4096, page=64, code="i8"),
        # one short evicted conversation, fp32 rows from e4m3: latency
        _case("read_small_f32", "read", 1, 16, 8, 64, "f32", P=701, ragged=300, per_head=True, code="e4m3"),
        # a batch of them back into the arrays that an evicting state works on
        _case("read_7b_b16", "read", 16, 32, 32, 128, "bf16", P=4352, ragged=2000, page=32, per_head=True, code="i8"),
        # a small fp32 model, three short sequences, eight query heads per KV head: latency
        _case("attend_odd_f32", "attend", 3, 24, 3, 64, "f32", P=1531, ragged=300),
        # grouped queries at 8k, a batch of 16 prompts of different lengths
        _case("attend_gqa_8k", "attend", 16, 32, 8, 128, "bf16", P=8192, ragged=4000, page=32),
        # one long conversation, its cache in int8: few units, split over the length
        _case("attend_1seq_i8", "attend", 1, 32, 8, 128, "bf16", P=131072, page=64, code="i8"),
        # a batch of 16 of a 7B model whose heads were evicted apart: the largest read
        _case("attend_7b_b16", "attend", 16, 32, 32, 128, "bf16", P=4352, ragged=1000, per_head=True),
    ]


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(["rotate", "rotate", "append", "append", "append", "read", "attend", "attend", "attend"])
        G = rng.choice([1, 2, 4, 4, 8])
        Hkv = rng.choice([1, 2, 3, 4, 8, 8, 16, 32])
        B = size(1, 64)
        d = rng.choice([64, 128, 128])
        dtype = rng.choice(["f32", "bf16", "bf16"])
        code = rng.choice(["", "i8", "e4m3"]) if kind != "rotate" else ""
        page = rng.choice([16, 16, 32, 64, 128, 256])
        per_head = rng.choice([False, True])
        P, n = size(60, 131072), 0
        ragged = rng.choice([0, P // 3, P])
        c = _case(None, kind, B, G * Hkv, Hkv, d, dtype, P, ragged, n, page, per_head, code)
        if kind in ("rotate", "append"):
            c["n"] = rng.choice([1, size(2, 8192)])
            c["P"] = rng.choice([0, size(1, 8192)]) if kind == "append" else 0
            c["ragged"] = 0 if kind == "rotate" else rng.choice([0, max(c["P"], c["n"]) // 3, max(c["P"], c["n"])])
            if not code:
                c["norm"] = rng.choice([False, True])
                c["rot"] = rng.choice([16, d // 4, d // 2, d, d, d])
                c["pairing"] = rng.choice(["halves", "halves", "neighbours"])
                c["axes"] = rng.choice([1, 1, 2, 3])
                c["in_turn"] = rng.choice([False, True])
                c["far"] = rng.choice([0, 0, size(1, 1000000)])
        if G * Hkv > 64 or work(c)["bytes"] > 1.1e9:
            continue
        if B * Hkv * (c["P"] + c["n"]) * d * (1 if code else 4) > 1.2e9:
            continue
        return c


# ---------------------------------------------------------------- inputs

def _spread(top, span, i, of):
    """A length between top - span and top, another one for every unit; span = top reaches 0."""
    return max(0, top - span * ((i * 37) % of) // max(of - 1, 1))


def _lens(case):
    """Slots in use before the call, [B][tables]"""
    H = case["Hkv"] if case["per_head"] else 1
    return [[_spread(case["P"], case["ragged"], b * H + h, case["B"] * H) for h in range(H)] for b in range(case["B"])]


def _rows(case):
    """Rows that a call brings per sequence."""
    if case["kind"] != "append" or case["n"] == 1:
        return [case["n"]] * case["B"]
    return [_spread(case["n"], min(case["ragged"], case["n"]), b, case["B"]) for b in range(case["B"])]


def _cap(case):
    most = case["P"] + (case["n"] if case["kind"] == "append" else 0)
    return max(1, (most + case["page"] - 1) // case["page"]) * case["page"]


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _sections(case):
    """Pairs of channels per axis: the first has what an equal split leaves over."""
    each = case["rot"] // 2 // (case["axes"] + 1) if case["axes"] > 1 else 0
    return [case["rot"] // 2 - each * (case["axes"] - 1)] + [each] * (case["axes"] - 1)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    B, Hq, Hkv, d, n, page, kind = (case[k] for k in ("B", "Hq", "Hkv", "d", "n", "page", "kind"))
    dt = _dtype(case)
    s = {"case": dict(case)}

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    def keys(*shape):
        # channels of different magnitude: what trained models' keys look like
        return normal(*shape) * (0.6 + 1.6 * torch.rand(shape[-1], generator=g, device=DEVICE) ** 4)

    if kind in ("rotate", "append"):
        if case["rot"]:
            x = normal(B, n, Hq + 2 * Hkv, d)
            x[:, :, :Hq + Hkv] *= 0.6 + 1.6 * torch.rand(d, generator=g, device=DEVICE) ** 4
            s["qkv"] = x.to(dt).view(B, n, (Hq + 2 * Hkv) * d)           # as a projection leaves it
            s["inv_freq"] = (10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"])).float().to(DEVICE)
            # token by token on the first axis; rows and columns of pictures 48 wide on the others
            at = torch.arange(n, device=DEVICE) + (torch.arange(B, device=DEVICE) * 11 + case["far"]).unsqueeze(-1)
            s["positions"] = torch.stack([at, at % 2304 // 48, at % 48][:case["axes"]]).to(torch.int32)
            if case["norm"]:
                s["q_norm"], s["k_norm"] = ((1.0 + 0.2 * normal(d)).to(dt) for _ in range(2))
            s["q_out"] = torch.zeros(B, Hq, n, d, dtype=dt, device=DEVICE)
            if kind == "rotate":
                s["k_out"], s["v_out"] = (torch.zeros(B, Hkv, n, d, dtype=dt, device=DEVICE) for _ in range(2))
        else:
            s["k_new"], s["v_new"] = keys(B, Hkv, n, d).to(dt), normal(B, Hkv, n, d).to(dt)
    if kind == "rotate":
        return s
    # the pool, its pages dealt at random
    H, cap = (Hkv if case["per_head"] else 1), _cap(case)
    lens = torch.tensor(_lens(case), dtype=torch.int32, device=DEVICE)
    s["lens"] = lens
    most = lens.long()
    if kind == "append":
        s["n_new"] = torch.tensor(_rows(case), dtype=torch.int32, device=DEVICE)
        s["lens_out"] = torch.zeros_like(lens)
        most = most + s["n_new"].view(B, 1)
    used = ((most + page - 1) // page).flatten()
    pool = max(1, int(used.sum())) + 3
    at = torch.arange(cap // page, device=DEVICE)
    order = torch.randperm(pool, generator=g, device=DEVICE)
    spot = (used.cumsum(0) - used).unsqueeze(-1) + at
    table = torch.where(at < used.unsqueeze(-1), order[spot.clamp(max=pool - 1)], -1)
    s["table"] = table.to(torch.int32).view(B, H, cap // page)
    shape = (pool,) + (() if case["per_head"] else (Hkv,)) + (page, d)
    if case["code"]:
        cdt = torch.int8 if case["code"] == "i8" else torch.float8_e4m3fn
        if kind == "append":
            s["K"], s["V"] = (torch.zeros(shape, dtype=torch.int8, device=DEVICE).view(cdt) for _ in range(2))
            s["ks"], s["vs"] = (torch.zeros(shape[:-1], device=DEVICE) for _ in range(2))
        else:
            (s["K"], s["ks"]), (s["V"], s["vs"]) = _quantise(keys(*shape), case["code"]), _quantise(normal(*shape), case["code"])
    elif kind == "append":
        s["K"], s["V"] = (torch.zeros(shape, dtype=dt, device=DEVICE) for _ in range(2))       # a pool as it was allocated: what is written stands out
    else:
        s["K"], s["V"] = keys(*shape).to(dt), normal(*shape).to(dt)
    if kind == "attend":
        s["q"] = (1.5 * normal(B, Hq, d)).to(dt)
        s["out"] = torch.zeros(B, Hq, d, device=DEVICE)
    elif kind == "read" or case["code"]:
        s["K_rows"], s["V_rows"] = (torch.zeros(B, Hkv, cap, d, dtype=dt, device=DEVICE) for _ in range(2))
    return s


# ---------------------------------------------------------------- one pass, in plain torch

def _quantise(x, code):
    """x [..., d] -> codes and scales [...]"""
    amax = x.float().abs().amax(-1)
    some = amax >= LEAST
    top = torch.full_like(amax, QMAX[code])
    scale = torch.where(some, amax / top, torch.zeros_like(amax))
    y = x.float() * torch.where(some, top / amax, torch.zeros_like(amax)).unsqueeze(-1)
    return (y.round().clamp_(-127, 127).to(torch.int8) if code == "i8" else y.to(torch.float8_e4m3fn)), scale


def _axis_of(case):
    """The axis of each pair of channels."""
    half, axes, sec = case["rot"] // 2, case["axes"], _sections(case)
    if case["in_turn"]:
        return [i % axes if i % axes and i < axes * sec[i % axes] else 0 for i in range(half)]
    return [a for a in range(axes) for _ in range(sec[a])]


def _angles(s):
    """[B, n, rot / 2], in 64 bits: cos and sin of far positions"""
    pos = s["positions"][torch.tensor(_axis_of(s["case"]), device=DEVICE)].double()      # [rot / 2, B, n]
    return (pos * s["inv_freq"].double().view(-1, 1, 1)).permute(1, 2, 0)


def _turn(x, weight, cos, sin, case):
    """x [B, n, H, d] fp32, cos and sin [B, n, 1, rot / 2] -> normed and rotated"""
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    rot = case["rot"]
    y = x[..., :rot].unflatten(-1, (2, rot // 2) if case["pairing"] == "halves" else (rot // 2, 2))
    a, b = y.unbind(-2 if case["pairing"] == "halves" else -1)
    y = torch.stack([a * cos - b * sin, b * cos + a * sin], -2 if case["pairing"] == "halves" else -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _turned(s):
    """q, k, v of a projection, normed and rotated: [B, H, n, d] in the KV type"""
    case = s["case"]
    B, Hq, Hkv, d, n = (case[k] for k in ("B", "Hq", "Hkv", "d", "n"))
    q, k, v = s["qkv"].view(B, n, Hq + 2 * Hkv, d).split([Hq, Hkv, Hkv], 2)
    a = _angles(s).unsqueeze(2)
    cos, sin = a.cos().float(), a.sin().float()
    q = _turn(q.float(), s.get("q_norm"), cos, sin, case).to(v.dtype)
    k = _turn(k.float(), s.get("k_norm"), cos, sin, case).to(v.dtype)
    return q.transpose(1, 2), k.transpose(1, 2), v.transpose(1, 2)


def _plain_rotate(s):
    q, k, v = _turned(s)
    s["q_out"].copy_(q)
    s["k_out"].copy_(k)
    s["v_out"].copy_(v)
    return {k: s[k] for k in ("q_out", "k_out", "v_out")}


def _spots(s, slots):
    """Row of the pool (its pages one behind the other) of slots [B, tables, m], for every KV head: [B, Hkv, m].  Slots whose table has no page: any."""
    case = s["case"]
    page, Hkv = case["page"], case["Hkv"]
    ids = s["table"].gather(2, (slots // page).clamp(max=s["table"].shape[2] - 1)).long().clamp(min=0)
    if case["per_head"]:
        return ids * page + slots % page
    return (ids * Hkv + torch.arange(Hkv, device=DEVICE).view(1, Hkv, 1)) * page + slots % page


def _plain_append(s):
    case = s["case"]
    B, Hkv, d, n = (case[k] for k in ("B", "Hkv", "d", "n"))
    if case["rot"]:
        q, k, v = _turned(s)
        q_live = (torch.arange(n, device=DEVICE) < s["n_new"].view(B, 1)).view(B, 1, n, 1)
        s["q_out"].copy_(torch.where(q_live, q, s["q_out"]))
    else:
        k, v = s["k_new"], s["v_new"]
    at = torch.arange(n, device=DEVICE)
    spots = _spots(s, s["lens"].long().unsqueeze(-1) + at).expand(B, Hkv, n)
    live = (at < s["n_new"].view(B, 1, 1)).expand(B, Hkv, n)
    for x, pool, sc in ((k, "K", "ks"), (v, "V", "vs")):
        x = x[live]
        if case["code"]:
            x, scale = _quantise(x, case["code"])
            s[sc].view(-1)[spots[live]] = scale
            s[pool].view(torch.int8).view(-1, d)[spots[live]] = x.view(torch.int8)
        else:
            s[pool].view(-1, d)[spots[live]] = x
    s["lens_out"].copy_(s["lens"] + s["n_new"].view(B, 1))
    return _appended(s, lambda: _read_into(s, s["lens_out"]))


def _appended(s, read):
    """What an append leaves: the pool and the queries, or the values that its codes stand for."""
    if s["case"]["code"]:
        read()
        return {k: s[k] for k in ("K_rows", "V_rows", "ks", "vs", "lens_out")}
    return {k: s[k] for k in ("K", "V", "q_out", "lens_out")}


def _gather(s):
    """K and V [B, Hkv, cap, d] fp32"""
    case = s["case"]
    spots = _spots(s, torch.arange(_cap(case), device=DEVICE).expand(*s["table"].shape[:2], -1)).expand(-1, case["Hkv"], -1)
    rows = []
    for pool, sc in (("K", "ks"), ("V", "vs")):
        if case["code"]:
            x = s[pool].view(torch.int8).view(-1, case["d"])[spots].view(s[pool].dtype).float()
            rows.append(x * s[sc].view(-1)[spots].unsqueeze(-1))
        else:
            rows.append(s[pool].view(-1, case["d"])[spots].float())
    return rows


def _read_into(s, lens):
    K, V = _gather(s)
    live = (torch.arange(K.shape[2], device=DEVICE) < lens.unsqueeze(-1)).unsqueeze(-1)
    s["K_rows"].copy_(torch.where(live, K.to(s["K_rows"].dtype), s["K_rows"]))
    s["V_rows"].copy_(torch.where(live, V.to(s["V_rows"].dtype), s["V_rows"]))


def _plain_read(s):
    _read_into(s, s["lens"])
    return {"K_rows": s["K_rows"], "V_rows": s["V_rows"]}


def _plain_attend(s):
    case = s["case"]
    B, Hq, Hkv, d = (case[k] for k in ("B", "Hq", "Hkv", "d"))
    K, V = _gather(s)
    seen = torch.arange(K.shape[2], device=DEVICE) < s["lens"].unsqueeze(-1)
    x = torch.matmul(s["q"].float().view(B, Hkv, Hq // Hkv, d), K.transpose(-2, -1).contiguous()) * (1.0 / math.sqrt(d))
    x = x.masked_fill(~seen.unsqueeze(2), float("-inf"))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    s["out"].copy_(torch.matmul(p, V).view(B, Hq, d))
    return {"out": s["out"]}


# ---------------------------------------------------------------- one pass, by the framework

def _call(s):
    from paper_2404_15949_amd import corm
    case, kind = s["case"], s["case"]["kind"]
    B, Hq, Hkv, d, n = (case[k] for k in ("B", "Hq", "Hkv", "d", "n"))
    if "desc" not in s:                    # what a program makes once: the descriptor, the pages', the model's rotation, a workspace
        cap = _cap(case)
        s["desc"] = corm.make_desc(B, Hq, Hkv, d, cap, cap, 1, 1, case["dtype"])
        if kind != "rotate":
            s["pages"] = corm.Pages(s["desc"], s["K"], s["V"], s["table"], s.get("ks"), s.get("vs"))
        if case["rot"]:
            s["rotation"] = corm.Rotation(s["inv_freq"], q_norm=s.get("q_norm"), k_norm=s.get("k_norm"), eps=EPS, pairing=case["pairing"],
                                          sections=_sections(case), in_turn=case["in_turn"])
        if kind == "attend":
            s["ws"] = torch.empty(corm.corm_paged_workspace_bytes(s["desc"]), dtype=torch.uint8, device=DEVICE)
    desc = s["desc"]
    if kind == "attend":
        corm.corm_paged_attend(desc, s["pages"], s["q"], s["lens"], s["out"], s["ws"])
        return {"out": s["out"]}
    if kind == "read":
        corm.corm_paged_read(desc, s["pages"], s["lens"], s["K_rows"], s["V_rows"])
        return {"K_rows": s["K_rows"], "V_rows": s["V_rows"]}
    if case["rot"]:
        q, k, v = s["qkv"].view(B, n, Hq + 2 * Hkv, d).transpose(1, 2).split([Hq, Hkv, Hkv], 1)
    else:
        k, v = s["k_new"], s["v_new"]
    if kind == "rotate":
        corm.corm_rotate(desc, q, k, v, s["rotation"], s["positions"], s["q_out"], s["k_out"], s["v_out"])
        return {k: s[k] for k in ("q_out", "k_out", "v_out")}
    if case["rot"]:
        corm.corm_paged_append(desc, s["pages"], k, v, s["lens"], s["lens_out"], n_new=s["n_new"], q=q, q_out=s["q_out"],
                               rotation=s["rotation"], positions=s["positions"])
    else:
        corm.corm_paged_append(desc, s["pages"], k, v, s["lens"], s["lens_out"], n_new=s["n_new"])
    return _appended(s, lambda: corm.corm_paged_read(desc, s["pages"], s["lens_out"], s["K_rows"], s["V_rows"]))


_PLAIN = {"rotate": _plain_rotate, "append": _plain_append, "read": _plain_read, "attend": _plain_attend}


def run(s):
    if own:
        return _call(s)
    return _PLAIN[s["case"]["kind"]](s)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    kind, B, Hq, Hkv, d = (case[k] for k in ("kind", "B", "Hq", "Hkv", "d"))
    esz = 4 if case["dtype"] == "f32" else 2
    slot = 2 * d * (1 if case["code"] else esz) + (8 if case["code"] else 0)         # bytes of a slot of a KV head
    slots = sum(sum(row) for row in _lens(case)) * (1 if case["per_head"] else Hkv)
    rows = sum(_rows(case))
    if kind == "attend":
        return {"bytes": slots * slot + B * Hq * d * (esz + 4), "flops": 4.0 * d * slots * (Hq // Hkv)}
    if kind == "read":
        return {"bytes": slots * (slot + 2 * d * esz), "flops": 2.0 * d * slots if case["code"] else 0.0}
    heads = Hq + Hkv if case["rot"] else 0
    flops = rows * heads * (3.0 * case["rot"] + (4.0 * d if case["norm"] else 0.0)) + rows * 4.0 * case["rot"]
    if kind == "rotate":
        return {"bytes": rows * ((Hq + 2 * Hkv) * d * esz * 2 + 4 * case["axes"]), "flops": flops}
    if case["code"]:
        return {"bytes": rows * Hkv * (2 * d * esz + slot) + (slots + rows * Hkv) * (slot + 2 * d * esz), "flops": 8.0 * d * rows * Hkv + 2.0 * d * slots}
    return {"bytes": rows * (Hq * d * esz * 2 + Hkv * (2 * d * esz + slot) + 4 * case["axes"]), "flops": flops}


# ---------------------------------------------------------------- the definitions in 64 bits

def _rotated_exact(s, x, weight):
    """x [B, H, n, d] in 64 bits, channel pair by channel pair"""
    case = s["case"]
    x, rot = x.double(), case["rot"]
    if weight is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / case["d"] + EPS) * weight.double()
    out = x.clone()
    for i, axis in enumerate(_axis_of(case)):
        a, b = (i, i + rot // 2) if case["pairing"] == "halves" else (2 * i, 2 * i + 1)
        angle = s["positions"][axis].double().unsqueeze(1) * float(s["inv_freq"][i])
        c, t = torch.cos(angle), torch.sin(angle)
        out[..., a] = x[..., a] * c - x[..., b] * t
        out[..., b] = x[..., a] * t + x[..., b] * c
    return out


def _held(s, pool, sc, b, h, n):
    """The rows that slots 0 .. n-1 of a KV head hold, page by page, in 64 bits"""
    case, per = s["case"], s["case"]["per_head"]
    x, scale = s[pool], s.get(sc)
    if not per:
        x, scale = x[:, h], None if scale is None else scale[:, h]
    ids = s["table"][b, h if per else 0, :(n + case["page"] - 1) // case["page"]].long()
    if scale is None:
        return x[ids].reshape(-1, case["d"])[:n].double()
    rows = x.view(torch.int8)[ids].view(s[pool].dtype).double() * scale[ids].double().unsqueeze(-1)
    return rows.reshape(-1, case["d"])[:n]


def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    B, Hq, Hkv, d, n, page = (case[k] for k in ("B", "Hq", "Hkv", "d", "n", "page"))
    if case["rot"]:
        x = s["qkv"].view(B, n, Hq + 2 * Hkv, d).transpose(1, 2)
        q, k = _rotated_exact(s, x[:, :Hq], s.get("q_norm")), _rotated_exact(s, x[:, Hq:Hq + Hkv], s.get("k_norm"))
        v = x[:, Hq + Hkv:].double()
        if kind == "rotate":
            return {"q_out": q, "k_out": k, "v_out": v}
    lens = s["lens"].tolist()
    of = (lambda b, h: lens[b][h]) if case["per_head"] else (lambda b, h: lens[b][0])
    if kind == "attend":
        out = torch.zeros(B, Hq, d, dtype=torch.float64, device=DEVICE)
        G = Hq // Hkv
        for b in range(B):
            for h in range(Hkv):
                if of(b, h):
                    K, V = _held(s, "K", "ks", b, h, of(b, h)), _held(s, "V", "vs", b, h, of(b, h))
                    p = torch.softmax(torch.mm(s["q"][b, h * G:(h + 1) * G].double(), K.t()) / math.sqrt(d), dim=-1)
                    out[b, h * G:(h + 1) * G] = torch.mm(p, V)
        return {"out": out}
    new = _rows(case)
    if kind == "append" and not case["code"]:
        K, V = s["K"].double(), s["V"].double()
        for b in range(B):
            for h in range(Hkv):
                at = of(b, h) + torch.arange(new[b], device=DEVICE)
                ids = s["table"][b, h if case["per_head"] else 0].long()[at // page]
                where = (ids, at % page) if case["per_head"] else (ids, torch.full_like(ids, h), at % page)
                K[where], V[where] = k[b, h, :new[b]], v[b, h, :new[b]]
            q[b, :, new[b]:] = 0
        return {"K": K, "V": V, "q_out": q, "lens_out": None}
    rows = {}
    for pool, sc, src in (("K", "ks", "k_new"), ("V", "vs", "v_new")):
        to = s[pool + "_rows"].double()
        scales = s[sc].double() if case["code"] else None
        for b in range(B):
            for h in range(Hkv):
                to[b, h, :of(b, h)] = _held(s, pool, sc, b, h, of(b, h))
                if kind == "append" and new[b]:
                    # the codes are settled in 32 bits, by the definition; what they stand for is exact
                    x = s[src][b, h, :new[b]].float()
                    amax = x.abs().amax(-1)
                    top = torch.full_like(amax, QMAX[case["code"]])
                    y = x * (top / amax).unsqueeze(-1)
                    y = y.round() if case["code"] == "i8" else y.to(torch.float8_e4m3fn)
                    step = amax.double() / QMAX[case["code"]]
                    at = of(b, h) + torch.arange(new[b], device=DEVICE)
                    to[b, h, at] = y.double() * step.unsqueeze(-1)
                    ids = s["table"][b, h if case["per_head"] else 0].long()[at // page]
                    scales[(ids, at % page) if case["per_head"] else (ids, torch.full_like(ids, h), at % page)] = step
        rows[pool + "_rows"] = to
        rows[sc] = scales
    if kind == "read":
        return {"K_rows": rows["K_rows"], "V_rows": rows["V_rows"]}
    return {"K_rows": rows["K_rows"], "V_rows": rows["V_rows"], "ks": rows["ks"], "vs": rows["vs"], "lens_out": None}
