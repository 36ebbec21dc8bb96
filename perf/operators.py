"""The step from a projection's heads to attention over a cache held in 4 bits, as measurable cases.

Kinds:

  norm_rope   rmm_qk_norm_rope: RMS norm of every query and key head and the position rotation, in one pass
  append      rmm_kv4_append: keys (norm and rotation applied on the way) and values quantised into a paged cache; decode steps are
              read back with rmm_kv4_read, prompts return the values that the cache now holds (what the prompt's own attention uses)
  attn        rmm_kv4_attn: attention of a few query rows over that cache, with feature selection where rho_d < 1
  read        rmm_kv4_read: the cached keys and values of the last rows of every sequence, back in bf16 or fp32

The cache: a pool of pages, uint8 [pages, Hkv, page / 16, 18 Dh]; 18 Dh bytes hold 16 tokens of one head: codes of K, codes of V, then
per token the (step, least value) pairs of every 64 columns of K and those of V, in bf16.  A value is least + step * code.
"""
import math

import torch

own = False

BLOCK, GROUP = 16, 64   # tokens of a block; columns that share a step


def listed():
    return [
        # one decode step of eight sequences: a layer's query and key heads, little else than a launch
        {"name": "norm_rope_token", "kind": "norm_rope", "B": 8, "L": 1, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128, "dtype": "bf16",
         "norm": True, "interleaved": False},
        # prompts of 4096 tokens
        {"name": "norm_rope_prompt", "kind": "norm_rope", "B": 2, "L": 4096, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128, "dtype": "bf16",
         "norm": True, "interleaved": False},
        # fp32 heads of 80 columns, 48 of them rotated in neighbouring pairs, an odd number of tokens
        {"name": "norm_rope_fp32", "kind": "norm_rope", "B": 3, "L": 1001, "Hq": 12, "Hkv": 12, "D": 80, "rot": 48, "dtype": "fp32",
         "norm": True, "interleaved": True},
        # a decode step of 32 sequences: one token each goes into the cache
        {"name": "append_token", "kind": "append", "B": 32, "L": 1, "past": 2000, "Hkv": 8, "D": 128, "rot": 128, "page": 64,
         "dtype": "bf16", "norm": True, "interleaved": False},
        # four prompts of 4096 tokens
        {"name": "append_prompt", "kind": "append", "B": 4, "L": 4096, "past": 0, "Hkv": 8, "D": 128, "rot": 128, "page": 64,
         "dtype": "bf16", "norm": False, "interleaved": False},
        # ragged chunks behind what is there, wide fp32 heads, small pages
        {"name": "append_ragged", "kind": "append", "B": 7, "L": 999, "past": 300, "Hkv": 2, "D": 256, "rot": 128, "page": 16,
         "dtype": "fp32", "norm": True, "interleaved": True},
        # one sequence, one token, a short cache: launch latency
        {"name": "attn_short", "kind": "attn", "B": 1, "L": 1, "low": 700, "high": 700, "Hq": 32, "Hkv": 8, "D": 128, "page": 64,
         "rho_d": 1.0, "causal": True},
        # a decode step of 16 sequences with 8192 tokens each
        {"name": "attn_batch", "kind": "attn", "B": 16, "L": 1, "low": 8192, "high": 8192, "Hq": 32, "Hkv": 8, "D": 128, "page": 64,
         "rho_d": 1.0, "causal": True},
        # sequences of very different lengths, wide heads, half of the features kept
        {"name": "attn_ragged", "kind": "attn", "B": 24, "L": 1, "low": 5, "high": 16384, "Hq": 16, "Hkv": 4, "D": 256, "page": 32,
         "rho_d": 0.5, "causal": True},
        # drafts of five tokens checked at once, heads of 64
        {"name": "attn_draft", "kind": "attn", "B": 8, "L": 5, "low": 3000, "high": 5000, "Hq": 32, "Hkv": 8, "D": 64, "page": 16,
         "rho_d": 1.0, "causal": True},
        # a chunk's attention by rmm_reduced_attn wants its prefixes in bf16
        {"name": "read_prefix", "kind": "read", "B": 4, "low": 4096, "high": 4096, "Hkv": 8, "D": 128, "page": 64, "dtype": "bf16"},
        # ragged prefixes in fp32
        {"name": "read_ragged", "kind": "read", "B": 9, "low": 3, "high": 2500, "Hkv": 4, "D": 64, "page": 32, "dtype": "fp32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm_rope", "append", "attn", "attn", "attn", "read"])
    if kind == "norm_rope":
        B = _log(rng, 1, 64)
        D = rng.choice([64, 80, 96, 128, 128, 256])
        Hkv, dtype = rng.choice([1, 2, 4, 8]), rng.choice(["bf16", "bf16", "fp32"])
        L = rng.choice([1, _log(rng, 1, max(1, min(8192, 8192 * 40 * 128 // (B * Hkv * 5 * D))))])
        return {"kind": kind, "B": B, "L": L, "Hq": Hkv * rng.choice([1, 2, 4]), "Hkv": Hkv, "D": D, "rot": rng.choice([D, D, D // 32 * 16]),
                "dtype": dtype, "norm": rng.random() < 0.7, "interleaved": rng.random() < 0.3}
    page = rng.choice([16, 32, 64, 64, 128])
    D = rng.choice([64, 128, 128, 256])
    Hkv = rng.choice([1, 2, 4, 8])
    if kind == "append":
        B = _log(rng, 1, 64)
        L = rng.choice([1, _log(rng, 1, max(1, 16384 * 8 * 128 // (2 * B * Hkv * D)))])
        return {"kind": kind, "B": B, "L": L, "past": rng.choice([0, _log(rng, 1, 5000)]), "Hkv": Hkv, "D": D, "rot": rng.choice([0, D, D, D // 2]),
                "page": page, "dtype": rng.choice(["bf16", "bf16", "fp32"]), "norm": rng.random() < 0.5, "interleaved": rng.random() < 0.3}
    if kind == "attn":
        high = _log(rng, 16, 65536)
        B = _log(rng, 1, max(1, min(128, 16 * 8192 * 8 * 128 // (high * Hkv * D))))
        return {"kind": kind, "B": B, "L": rng.choice([1, 1, 1, rng.randint(2, 8)]), "low": rng.choice([high, max(1, high // 50)]), "high": high,
                "Hq": Hkv * rng.choice([1, 4, 4, 8, 6]), "Hkv": Hkv, "D": D, "page": page, "rho_d": rng.choice([1.0, 1.0, 0.5, round(rng.uniform(0.2, 0.9), 2)]),
                "causal": rng.random() < 0.9}
    high = _log(rng, 1, 8192)
    return {"kind": kind, "B": _log(rng, 1, max(1, min(64, 4 * 4096 * 8 * 128 // (high * Hkv * D)))), "low": rng.choice([high, max(1, high // 50)]),
            "high": high, "Hkv": Hkv, "D": D, "page": page, "dtype": rng.choice(["bf16", "bf16", "fp32"])}


def _spread(n, low, high):
    """n whole numbers from low to high, even over their logarithm, in no order."""
    if low >= high:
        return [high] * n
    return [int(round(low * (high / low) ** ((0.5 + 0.6180339887498949 * i) % 1.0))) for i in range(n)]


def _lengths(case):
    """(tokens that each sequence holds, rows of it that the call is about)"""
    B = case["B"]
    if case["kind"] == "append":
        new = _spread(B, max(1, case["L"] // 4), case["L"])
        new[0] = case["L"]
        return [case["past"] + 7 * b % 61 + n if case["past"] else n for b, n in enumerate(new)], new
    n = _spread(B, case["low"], case["high"])
    return n, [case["L"]] * B if case["kind"] == "attn" else n


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _keys(g, b, h, t, d):
    """Keys of cached heads: normal, a few channels of every head larger than the rest, around means of their own"""
    gain = torch.where(_normal(g, h, 1, d).abs() > 2.2, 5.0, 1.0)
    return _normal(g, b, h, t, d) * gain + _normal(g, h, 1, d)


def _rope(length, rot):
    """cos and sin of every position's angles, fp32 [length, rot], the cosines first"""
    inv = 500000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    angles = torch.arange(length, device="cuda", dtype=torch.float64)[:, None] * inv
    return torch.cat([angles.cos(), angles.sin()], 1).float()


def _cache_of(case, seed, b, n):
    """One sequence's keys and values as they came, bf16 [Hkv, n, D]"""
    g = _gen(1000003 * seed + b)
    return _keys(g, 1, case["Hkv"], n, case["D"])[0].bfloat16(), _normal(g, case["Hkv"], n, case["D"]).bfloat16()


def _pack(K, V):
    """bf16 [H, blocks * 16, D] twice -> uint8 [H, blocks, 18 D]"""
    parts, steps = [], []
    H, T, D = K.shape
    for x in (K, V):
        code, s, low = _quantise(x.float())
        byte = (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8)                      # [H, T, D / 2]
        if x is K:
            byte = byte.view(H, T // 16, 16, D // 32, 4, 4).transpose(3, 4)
        else:  # tokens 8 h + 2 q + e, bytes of the columns 128 j + 64 i + 8 g ..
            i = min(2, D // 64)
            byte = byte.view(H, T // 16, 2, 4, 2, D // 64 // i, i, 8, 4).permute(0, 1, 5, 2, 7, 3, 4, 6, 8)
        parts.append(byte.reshape(H, T // 16, 8 * D))
        steps.append(torch.stack([s, low], -1).bfloat16().view(torch.uint8).reshape(H, T // 16, D))
    return torch.cat(parts + steps, -1)


def _unpack(blocks):
    """uint8 [..., 18 D] -> K, V fp32 [..., 16, D]"""
    D, lead = blocks.shape[-1] // 18, blocks.shape[:-1]
    k, v, sk, sv = (x.contiguous() for x in blocks.split([8 * D, 8 * D, D, D], -1))
    i = min(2, D // 64)
    n = len(lead)
    k = k.view(*lead, 16, 4, D // 32, 4).transpose(-3, -2)
    v = v.view(*lead, D // 64 // i, 2, 8, 4, 2, i, 4).permute(*range(n), n + 1, n + 3, n + 4, n, n + 5, n + 2, n + 6)
    out = []
    for byte, st in ((k, sk), (v, sv)):
        byte = byte.reshape(*lead, 16, D // 2)
        code = torch.stack([byte & 15, byte >> 4], -1).view(*lead, 16, D // 64, 64).float()
        st = st.view(torch.bfloat16).view(*lead, 16, D // 64, 2).float()
        out.append((code * st[..., :1] + st[..., 1:]).view(*lead, 16, D))
    return out


def prepare(case, seed):
    kind = case["kind"]
    st = {"kind": kind, "case": case}
    dt = torch.float32 if case.get("dtype") == "fp32" else torch.bfloat16
    g = _gen(7919 * seed + 1)
    if kind == "norm_rope":
        B, L, Hq, Hkv, D = (case[x] for x in ("B", "L", "Hq", "Hkv", "D"))
        # heads as a projection writes them: a token's query heads, its key heads behind them
        both = (_normal(g, B, L, Hq + Hkv, D) * (1 + 3 * _normal(g, D).abs())).to(dt)
        st.update(Q=both[:, :, :Hq].transpose(1, 2), K=both[:, :, Hq:].transpose(1, 2),
                  qw=1 + 0.2 * _normal(g, D) if case["norm"] else None, kw=1 + 0.2 * _normal(g, D) if case["norm"] else None,
                  rope=_rope(8192, case["rot"]))
        start = torch.randint(0, 8192 - L + 1, (B, 1), generator=g, device="cuda")
        st["positions"] = (start + torch.arange(L, device="cuda")).int()
        return st
    B, Hkv, D, page = (case[x] for x in ("B", "Hkv", "D", "page"))
    total, new = _lengths(case)
    need = [-(-n // page) for n in total]
    order = torch.randperm(sum(need) + 3, generator=g, device="cuda").int()     # pages are handed out in no order
    pages = torch.full((B, max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        pages[b, :n] = order[at:at + n]
        at += n
    pool = torch.zeros(sum(need) + 3, Hkv, page // 16, 18 * D, dtype=torch.uint8, device="cuda")
    st.update(pool=pool, pages=pages, lengths=torch.tensor(total, dtype=torch.int32, device="cuda"),
              new=torch.tensor(new, dtype=torch.int32, device="cuda"))
    if kind == "append":
        L = case["L"]
        K, V = _normal(g, B, L, Hkv, D) * (1 + 3 * _normal(g, D).abs()), _normal(g, B, L, Hkv, D)
        st.update(K=K.to(dt).transpose(1, 2), V=V.to(dt).transpose(1, 2), kw=1 + 0.2 * _normal(g, D) if case["norm"] else None,
                  rope=_rope(max(total), case["rot"]) if case["rot"] else None)
        return st
    for b, n in enumerate(total):
        blocks = _pack(*(torch.nn.functional.pad(x, (0, 0, 0, need[b] * page - n)) for x in _cache_of(case, seed, b, n)))
        pool[pages[b, :need[b]].long()] = blocks.view(Hkv, need[b], page // 16, 18 * D).transpose(0, 1)
    if kind == "attn":
        st["Q"] = _normal(g, B, case["L"], case["Hq"], D).bfloat16().transpose(1, 2)
        st["rho_d"], st["causal"] = case["rho_d"], case["causal"]
    else:
        st["dtype"] = dt
        st["rows"] = max(total)
    return st


def _to_bf16(z):
    """64-bit numbers rounded once to bf16"""
    m, e = torch.frexp(z)
    return torch.ldexp(torch.round(m * 256), e - 8).to(torch.bfloat16)


def _norm_rope(x, weight, rope, eps, interleaved):
    """x [..., L, D] with rope [..., L, rot] (or None), in x's precision"""
    if weight is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * weight.to(x.dtype)
    if rope is None:
        return x
    rot = rope.shape[-1]
    cos, sin = rope[..., :rot // 2].to(x.dtype), rope[..., rot // 2:].to(x.dtype)
    head, rest = x[..., :rot], x[..., rot:]
    a, b = (head[..., 0::2], head[..., 1::2]) if interleaved else (head[..., :rot // 2], head[..., rot // 2:])
    u, v = a * cos - b * sin, b * cos + a * sin
    return torch.cat([torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1), rest], -1)


def _quantise(x):
    """codes, steps and least values of groups of 64 columns of fp32 x (bf16 numbers): integers [..., D], fp32 [..., D / 64] twice"""
    y = x.unflatten(-1, (-1, GROUP))
    low, high = y.amin(-1), y.amax(-1)
    step = ((high - low) / 15).bfloat16().float()
    code = torch.where(step[..., None] > 0, torch.round((y - low[..., None]) / step[..., None]), 0.0).clamp(0, 15)
    return code.flatten(-2).to(torch.int32), step, low


def _held(x):
    code, step, low = _quantise(x)
    return (code.float().unflatten(-1, (-1, GROUP)) * step[..., None] + low[..., None]).flatten(-2)


def _gathered(st):
    """Every sequence's cache, fp32 [B, Hkv, tokens, D] twice"""
    blocks = st["pool"][st["pages"].clamp(min=0).long()]                         # [B, pages, Hkv, blocks, 18 D]
    K, V = _unpack(blocks.transpose(1, 2))
    return K.flatten(2, 4), V.flatten(2, 4)


def _attention(st):
    K, V = _gathered(st)
    Q = st["Q"].float()
    B, Hq, L, D = Q.shape
    Hkv, T = K.shape[1], K.shape[2]
    if st["rho_d"] < 1:
        kept = math.ceil(round(st["rho_d"] * D, 9))
        order = torch.sort(st["Q"].double().square().sum(2, keepdim=True), dim=-1, descending=True, stable=True).indices
        Q = Q * torch.zeros(B, Hq, 1, D, device="cuda").scatter_(3, order[..., :kept], 1.0)
    S = (Q.reshape(B, Hkv, Hq // Hkv * L, D) @ K.transpose(-1, -2)).view(B, Hq, L, T) / math.sqrt(D)
    t, n = torch.arange(T, device="cuda"), st["lengths"][:, None, None, None]
    seen = n - L + 1 + torch.arange(L, device="cuda")[:, None] if st["causal"] else n
    S = torch.where(t < seen, S, -math.inf)
    P = torch.exp(S - S.amax(-1, keepdim=True).clamp(min=-3e38))
    P = P / P.sum(-1, keepdim=True).clamp(min=1e-30)
    P = torch.where(t < seen, P, 0.0).view(B, Hkv, Hq // Hkv * L, T)
    return (P @ V).view(B, Hq, L, D).bfloat16()


def run(state):
    st, kind = state, state["kind"]
    if own:
        import paper_2608_13426_b200 as rmm

        if kind == "norm_rope":
            return rmm.rmm_qk_norm_rope(st["Q"], st["K"], st["qw"], st["kw"], st["rope"], st["positions"], interleaved=st["case"]["interleaved"])
        if kind == "append":
            prompt = st["case"]["L"] > 16
            held = rmm.rmm_kv4_append(st["K"], st["V"], st["pool"], st["pages"], st["lengths"], st["new"], st["kw"], st["rope"],
                                      interleaved=st["case"]["interleaved"], want_values=prompt)
            return held if prompt else rmm.rmm_kv4_read(st["pool"], st["pages"], st["lengths"], st["new"], rows=st["case"]["L"])
        if kind == "attn":
            return rmm.rmm_kv4_attn(st["Q"], st["pool"], st["pages"], st["lengths"], causal=st["causal"], rho_d=st["rho_d"])
        return rmm.rmm_kv4_read(st["pool"], st["pages"], st["lengths"], st["lengths"], rows=st["rows"], out_dtype=st["dtype"])
    if kind == "norm_rope":
        rope = st["rope"][st["positions"].long()][:, None]
        return tuple(_norm_rope(st[x].float(), st[w], rope, 1e-6, st["case"]["interleaved"]).to(st[x].dtype) for x, w in (("Q", "qw"), ("K", "kw")))
    if kind == "append":
        K, V, L = st["K"], st["V"], st["case"]["L"]
        i = torch.arange(L, device="cuda")
        at = (st["lengths"] - st["new"])[:, None].long() + i
        rope = st["rope"][at.clamp(max=st["rope"].shape[0] - 1)][:, None] if st["rope"] is not None else None
        # rotated keys are rounded to bf16 before they are quantised: 64 bits, so that no value falls to the wrong side of a border
        K = _to_bf16(_norm_rope(K.double(), st["kw"], rope, 1e-6, st["case"]["interleaved"])).float()
        there = (i < st["new"][:, None])[:, None, :, None]
        K, V = (torch.where(there, _held(x), 0.0).bfloat16() for x in (K, V.bfloat16().float()))
        return K, V
    if kind == "attn":
        return _attention(st)
    there = (torch.arange(st["rows"], device="cuda") < st["lengths"][:, None])[:, None, :, None]
    return tuple(torch.where(there, x[:, :, :st["rows"]], 0.0).to(st["dtype"]) for x in _gathered(st))


def work(case):
    kind, B, D, Hkv = case["kind"], case["B"], case["D"], case["Hkv"]
    size = 4 if case.get("dtype") == "fp32" else 2
    if kind == "norm_rope":
        values = B * case["L"] * (case["Hq"] + Hkv) * D
        return {"bytes": 2 * values * size + 4 * B * case["L"] * (case["rot"] + 1), "flops": 8 * values}
    total, new = _lengths(case)
    if kind == "append":
        # K and V in, their codes and steps into the cache, the held values out in bf16
        values = 2 * sum(new) * Hkv * D
        out = 2 * B * case["L"] * Hkv * D
        return {"bytes": values * (size + 0.5625) + 2 * out + 4 * sum(new) * case["rot"], "flops": 12 * values}
    values = 2 * sum(total) * Hkv * D
    if kind == "attn":
        return {"bytes": 0.5625 * values + 4 * B * case["Hq"] * case["L"] * D, "flops": 2 * values * case["Hq"] // Hkv * case["L"]}
    return {"bytes": 0.5625 * values + 2 * size * B * max(total) * Hkv * D, "flops": 2 * values}


def _exact_held(z):
    """What a cache holds for z (64-bit numbers that are bf16 numbers)."""
    shape = z.shape
    z = z.reshape(-1, GROUP)
    low = z.min(1, keepdim=True).values
    spread = z.max(1, keepdim=True).values - low
    step = (spread / 15).to(torch.float32).to(torch.bfloat16).double()
    n = torch.floor((z - low) / torch.where(step == 0, 1.0, step) + 0.5)
    q = (z - low) - (n - 0.5) * step
    n = n - ((q == 0) & (n % 2 == 1)).double()                # halves go to the even code
    return (low + n.clamp(0, 15) * step).reshape(shape)


def _exact_rows(x, weight, cos_sin, interleaved):
    """Norm and rotation of rows by their definition, in complex numbers."""
    x = x.double()
    if weight is not None:
        x = x * weight.double() * (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6).pow(-0.5)
    if cos_sin is None:
        return x
    half = cos_sin.shape[-1] // 2
    turn = torch.complex(cos_sin[..., :half].double(), cos_sin[..., half:].double())
    pairs = x[..., :2 * half]
    pairs = pairs.unflatten(-1, (half, 2)) if interleaved else pairs.unflatten(-1, (2, half)).transpose(-1, -2)
    z = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * turn)
    z = z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., 2 * half:]], -1)


def exact(case, seed):
    kind = case["kind"]
    st = prepare(case, seed) if kind in ("norm_rope", "append") else None
    if kind == "norm_rope":
        cs = st["rope"][st["positions"].long()].unsqueeze(1)
        return tuple(_exact_rows(st[x], st[w], cs, case["interleaved"]) for x, w in (("Q", "qw"), ("K", "kw")))
    total, new = _lengths(case)
    if kind == "append":
        K, V = torch.zeros(st["K"].shape, dtype=torch.float64, device="cuda"), torch.zeros(st["V"].shape, dtype=torch.float64, device="cuda")
        for b in range(case["B"]):
            n, first = new[b], total[b] - new[b]
            z = _exact_rows(st["K"][b, :, :n], st["kw"], st["rope"][first:first + n] if case["rot"] else None, case["interleaved"])
            c = z * (2.0 ** 45 + 1)                             # the leading 8 bits of z, rounded to nearest
            K[b, :, :n] = _exact_held(c - (c - z))
            V[b, :, :n] = _exact_held(st["V"][b, :, :n].to(torch.bfloat16).double())
        return K, V
    if kind == "read":
        out = [torch.zeros(case["B"], case["Hkv"], max(total), case["D"], dtype=torch.float64, device="cuda") for _ in range(2)]
        for b, n in enumerate(total):
            for o, x in zip(out, _cache_of(case, seed, b, n)):
                o[b, :, :n] = _exact_held(x.double())
        return tuple(out)
    Q = prepare(case, seed)["Q"]
    B, Hq, L, D = Q.shape
    O = torch.zeros(B, Hq, L, D, dtype=torch.float64, device="cuda")
    kept = D if case["rho_d"] >= 1 else math.ceil(round(case["rho_d"] * D, 9))
    for b, n in enumerate(total):
        K, V = (_exact_held(x.double()) for x in _cache_of(case, seed, b, n))
        group = Hq // case["Hkv"]
        for h in range(Hq):
            q = Q[b, h].double()
            idx = torch.sort(q.square().sum(0), descending=True, stable=True).indices[:kept]
            logits = q[:, idx] @ K[h // group][:, idx].T / math.sqrt(D)
            if case["causal"]:
                logits = logits.masked_fill(torch.ones(L, n, dtype=torch.bool, device="cuda").triu(1 + n - L), -math.inf)
            O[b, h] = torch.nan_to_num(torch.softmax(logits, -1), nan=0.0) @ V[h // group]
    return O
