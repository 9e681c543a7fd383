"""Operators of a decoding loop over a cache of 4-bit groups, as cases that can be timed, each with a plain form in torch.

  norm      new rows go into the paged cache, the heads of q and k normalised and rotated on the way (``owl_append_kv_norm``)
  append    the same into a cache of 4-bit groups, with or without the norms (``owl_append_kv_groups``)
  verify    the verify-step attention over such a cache (``owl_verify_attn_groups``)
  commit    the accepted rows of such a cache move behind the context (``owl_commit_kv_groups``)
  gather    cached rows are read back as 16-bit numbers (``owl_gather_kv_groups``)

A group is 32 neighbouring channels of one token and KV head, of K or of V: 32 e2m1 codes (0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign), two
a byte, the lower channel in the lower half, and one scale byte s; a value is e2m1 * 2^(s - 127), and s = 255 says that the group
is no numbers.  Codes and scale bytes are integers that have to be equal, so the calls that write a cache return the bytes that it
holds.  ``own`` chooses between the plain forms and the library's calls.
"""
import math

import torch

own = False

PAGE, GROUP = 16, 32
DEV = "cuda:0"
_TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_ENDS = {"bf16": (-125, 125), "f16": (-23, 13)}                      # exponents of a group
_MOST_BYTES, _MOST_FLOPS = 6.0e8, 1.72e11                            # of a drawn case
_EPS = 1e-6


# ----------------------------------------------------------------------------------------------------------- cases
def _append(name, kind, dtype, hq, hkv, d, batch, ctx_lo, ctx_hi, n, tree=False, rot_dim=None, interleaved=False, norm=True, lens_seed=0):
    case = {"kind": kind, "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "batch": batch, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "n": n,
            "tree": tree, "rot_dim": d if rot_dim is None else rot_dim, "interleaved": interleaved, "norm": norm, "lens_seed": lens_seed}
    return dict(case, name=name) if name else case


def _verify(name, dtype, hq, hkv, d, batch, ctx_lo, ctx_hi, n, tree="tree", ragged=False, outliers=False, lens_seed=0):
    case = {"kind": "verify", "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "batch": batch, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "n": n, "tree": tree, "ragged": ragged, "outliers": outliers, "lens_seed": lens_seed}
    return dict(case, name=name) if name else case


def _commit(name, hkv, d, batch, ctx_lo, ctx_hi, n, depth, lens_seed=0):
    case = {"kind": "commit", "dtype": "bf16", "hkv": hkv, "d": d, "batch": batch, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "n": n,
            "depth": depth, "lens_seed": lens_seed}
    return dict(case, name=name) if name else case


def _gather(name, dtype, hkv, d, first, n):
    case = {"kind": "gather", "dtype": dtype, "hkv": hkv, "d": d, "batch": 1, "ctx_lo": first, "ctx_hi": first, "n": n, "lens_seed": 0}
    return dict(case, name=name) if name else case


def listed():
    return [
        # the drafted tree of one sequence, heads normalised, into a 16-bit cache at 64K: a few hundred KB, latency
        _append("norm_tree60_64k", "norm", "bf16", 32, 8, 128, 1, 65001, 65001, 60, tree=True),
        # a prompt of 8K tokens from its start, fp16, queries with it: bound by memory
        _append("norm_prompt_8k_f16", "norm", "f16", 32, 8, 128, 1, 0, 0, 8192),
        # sixteen users' trees into a 4-bit cache, each beginning somewhere inside a page
        _append("append_4bit_batch16_tree26", "append", "bf16", 32, 8, 128, 16, 8192, 65536, 26, tree=True, lens_seed=5),
        # four prompts' next chunks, odd lengths, neighbouring channels, half of a head rotated, heads as they come
        _append("append_4bit_chunk4x2501", "append", "bf16", 64, 8, 128, 4, 0, 9001, 2501, rot_dim=64, interleaved=True, norm=False, lens_seed=3),
        # one token after a short prompt, fp16: launches and latency
        _verify("verify_4bit_decode1_5k_f16", "f16", 32, 8, 128, 1, 5003, 5003, 1, tree="chain"),
        # sequence verification of six tokens at 32K: a quarter of the bytes of a 16-bit cache
        _verify("verify_4bit_chain6_32k", "bf16", 32, 8, 128, 1, 32768, 32768, 6, tree="chain"),
        # tree and chain in one draft of a 70B-shaped layer at the 128K limit, keys with outliers: bound by the products
        _verify("verify_4bit_hybrid40_128k", "bf16", 64, 8, 128, 1, 131072, 131072, 40, tree="hybrid", outliers=True),
        # serving: sixteen sequences of very different lengths with drafts of different sizes, fp16
        _verify("verify_4bit_batch16_tree26_f16", "f16", 32, 8, 128, 16, 8192, 65536, 26, ragged=True, lens_seed=5),
        # the accepted path of one tree of 60
        _commit("commit_4bit_tree60", 8, 128, 1, 65001, 65001, 60, 6),
        # the accepted paths of 64 users' trees
        _commit("commit_4bit_batch64", 8, 128, 64, 1000, 32768, 40, 8, lens_seed=7),
        # the rows of one drafted tree are looked at
        _gather("gather_4bit_60", "bf16", 8, 128, 65001, 60),
        # a whole context becomes a 16-bit cache again (a chunk of a prompt attends over it with another kernel, or it moves to another pool)
        _gather("gather_4bit_64k", "bf16", 8, 128, 0, 65536),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "append", "append", "verify", "verify", "verify", "commit", "gather"])
    hq, hkv = rng.choice([(32, 8), (64, 8), (32, 8), (16, 4), (8, 2), (4, 1), (32, 4), (8, 1), (12, 3)])
    d, dtype = rng.choice([128, 128, 128, 64]), rng.choice(["bf16", "bf16", "f16"])
    seed = rng.randrange(1 << 20)
    if kind == "commit":
        batch, hi, n = _log_int(rng, 1, 100), _log_int(rng, 1, 100000), rng.randint(1, 64)
        case = _commit(None, hkv, d, batch, _log_int(rng, 1, hi), hi, n, rng.randint(1, min(n, 12)), seed)
    elif kind == "gather":
        first = rng.choice([0, _log_int(rng, 1, 60000)])
        case = _gather(None, dtype, hkv, d, first, _log_int(rng, 1, 70000))
    elif kind in ("norm", "append"):
        if kind == "norm" and rng.random() < 0.2:
            dtype = "f32"
        tree = rng.random() < 0.5
        n = rng.randint(1, 64) if tree else _log_int(rng, 1, 9000)
        hi = _log_int(rng, 1, 120000)
        lo = rng.choice([0, hi, _log_int(rng, 1, hi)])
        case = _append(None, kind, dtype, hq, hkv, d, _log_int(rng, 1, 24), lo, hi, n, tree, rng.choice([d, d, d // 2, 48, 0]),
                       rng.random() < 0.3, kind == "norm" or rng.random() < 0.5, seed)
    else:
        tree = rng.choice(["chain", "tree", "tree", "hybrid"])
        n = _log_int(rng, 1, 16) if tree == "chain" else rng.randint(4, 64)
        batch = 1 if rng.random() < 0.6 else _log_int(rng, 2, 24)
        hi = _log_int(rng, 20, 131072)
        lo = hi if batch == 1 else rng.choice([0, _log_int(rng, 1, hi)])
        case = _verify(None, dtype, hq, hkv, d, batch, lo, hi, n, tree, rng.random() < 0.3, dtype == "bf16" and rng.random() < 0.25, seed)
    while (w := work(case))["bytes"] > _MOST_BYTES or w["flops"] > _MOST_FLOPS:
        key = "batch" if case["batch"] > 1 else "n" if kind in ("norm", "append") else "ctx_hi"
        case[key] = max(1, case[key] * 3 // 4)
        case["ctx_lo"] = case["ctx_hi"] if case["batch"] == 1 and kind == "verify" else min(case["ctx_lo"], case["ctx_hi"])
    return case


def _lens(case):
    """Context lengths: the two ends, and seeded ones between them."""
    lo, hi, b = case["ctx_lo"], case["ctx_hi"], case["batch"]
    gen = torch.Generator().manual_seed(case["lens_seed"])
    lens = torch.randint(lo, hi + 1, (b,), generator=gen)
    lens[0] = hi
    if b > 1:
        lens[1] = lo
        lens = lens[torch.randperm(b, generator=gen)]
    return [int(x) for x in lens]


def _counts(case):
    """Drafted tokens of each sequence."""
    if not case.get("ragged"):
        return [case["n"]] * case["batch"]
    gen = torch.Generator().manual_seed(case["lens_seed"] + 1)
    return [int(x) for x in torch.randint(max(1, case["n"] // 2), case["n"] + 1, (case["batch"],), generator=gen)]


def work(case):
    kind, size, hkv, d = case["kind"], 4 if case["dtype"] == "f32" else 2, case["hkv"], case["d"]
    held = d // 2 + d // GROUP                                                   # bytes of a cached row of one head, 4 bits
    if kind in ("norm", "append"):
        n, hq = case["batch"] * case["n"], case["hq"]
        return {"bytes": n * (size * (2 * hq + 2 * hkv) * d + 2 * hkv * (held if kind == "append" else size * d)),
                "flops": n * (hq + hkv) * (3 * case["rot_dim"] + 4 * d * case["norm"])}
    if kind == "commit":
        rows = 2 * case["batch"] * case["depth"]                                 # read once, written once, of K and of V
        return {"bytes": 2 * rows * hkv * held + 4 * case["batch"] * case["n"], "flops": 0}
    if kind == "gather":
        return {"bytes": 2 * case["n"] * hkv * (held + size * d), "flops": 2 * case["n"] * hkv * d}
    lens, counts = _lens(case), _counts(case)
    cached = [l + c for l, c in zip(lens, counts)]
    return {"bytes": sum(cached) * hkv * 2 * held + 2 * size * sum(counts) * case["hq"] * d + sum(cached) // 4,
            "flops": sum(4 * t * c for t, c in zip(cached, counts)) * case["hq"] * d}


# ---------------------------------------------------------------------------------------------------------- inputs
def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _parents(kind, n, depth, gen):
    """Parent array: a chain, a random tree, or a random tree with a chain of a fifth of its nodes under its deepest leaf."""
    if kind == "chain":
        return list(range(-1, n - 1))
    tail = n // 5 if kind == "hybrid" else 0
    parent, level = [], []
    for i in range(n - tail):
        up = [-1] + [j for j in range(i) if level[j] < depth]
        p = up[int(torch.randint(0, len(up), (1,), generator=gen))]
        parent.append(p)
        level.append(1 if p < 0 else level[p] + 1)
    leaf = max(range(n - tail), key=lambda j: level[j]) if n > tail else -1
    for i in range(tail):
        parent.append(leaf if i == 0 else n - tail + i - 1)
    return parent


def _depths(parent):
    level = []
    for p in parent:
        level.append(1 if p < 0 else level[p] + 1)
    return level


def _two_to(e):
    """2^e in 64 bits, made of its bits: a power by exp or pow need not be exact."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantise(x, dtype):
    """Rows [..., D] -> (bytes [..., D / 2], scale bytes [..., D / 32])."""
    low, high = _ENDS[dtype]
    x = x.unflatten(-1, (-1, GROUP))
    fine = torch.isfinite(x).all(-1)
    x = torch.where(fine[..., None], x, 0.0)
    big = x.abs().amax(-1)
    mantissa, exponent = torch.frexp(big)                                        # big = mantissa 2^exponent, mantissa in [1/2, 1)
    e = torch.where(mantissa > 0.875, exponent - 2, exponent - 3)                # least with big <= 7 * 2^e
    e = torch.where(big > 0, e, low).clamp(low, high)
    y = x.double().abs() * _two_to(-e)[..., None]                                # exact: a power of two
    code = (y > 0.25).byte() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)       # ties to the even code
    code = torch.where(fine[..., None], code + 8 * torch.signbit(x), 0).byte().flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, torch.where(fine, e + 127, 255).byte()


def _pages_of(case, lens, n, gen, whole):
    """A page table whose pages are scattered over a pool: of the whole context, or of the rows from the last page of the
    context on (the entries before that name page 0, which nothing of the case touches)."""
    first = [0 if whole else l // PAGE for l in lens]
    last = [(l + n + PAGE - 1) // PAGE for l in lens]
    total = sum(b - a for a, b in zip(first, last)) + 1
    order = (torch.randperm(total - 1, generator=gen, device=DEV) + 1).to(torch.int32)
    table = torch.zeros((len(lens), max(last)), dtype=torch.int32, device=DEV)
    at = 0
    for b, (a, z) in enumerate(zip(first, last)):
        table[b, a:z] = order[at:at + z - a]
        at += z - a
    return table, total


def _pools(case, pages, gen, hot=None):
    """Quantised K, its channels of different magnitude as keys have them, and V: bytes [pages][Hkv][16][D / 2], scales [pages][Hkv][16][D / 32]."""
    shape, pools = (PAGE, case["d"]), []
    spread = torch.exp(0.5 * torch.randn((case["hkv"], 1, case["d"]), generator=gen, device=DEV))
    for t in range(2):
        parts = []
        for first in range(0, pages, 2048):
            count = min(2048, pages - first)
            x = torch.randn((count, case["hkv"], *shape), generator=gen, device=DEV)
            if t == 0:
                x *= spread
                if hot is not None:
                    x *= 1.0 + 7.0 * hot[first:first + count]
            parts.append(_quantise(x, case["dtype"]))
        pools += [torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])]
    return dict(zip(("k", "k_scale", "v", "v_scale"), pools))


def prepare(case, seed):
    gen, cpu = torch.Generator(DEV).manual_seed(seed), torch.Generator().manual_seed(seed)
    kind = case["kind"]
    s = {"case": case, "kind": kind, "status": torch.zeros(1, dtype=torch.int32, device=DEV)}
    dt = _TORCH[case["dtype"]]
    lens, n, b = _lens(case), case["n"], case["batch"]
    s["lens"], s["most"] = _i32(lens), max(lens)
    hq, hkv, d = case.get("hq"), case["hkv"], case["d"]
    if kind in ("norm", "append"):
        s["table"], pages = _pages_of(case, lens, n, gen, False)
        if kind == "append":
            s.update(_pools(case, pages, gen))
        else:
            s["k"], s["v"] = (torch.randn((pages, hkv, PAGE, d), generator=gen, device=DEV).to(dt) for _ in range(2))
        s["qkv"] = torch.randn((b, n, (hq + 2 * hkv) * d), generator=gen, device=DEV).to(dt)    # what a fused projection leaves
        s["q_gain"], s["k_gain"] = (1.0 + 0.2 * torch.randn((d,), generator=gen, device=DEV) for _ in range(2)) if case["norm"] else (None, None)
        half = case["rot_dim"] // 2
        s["inv_freq"] = (500000.0 ** (-torch.arange(half, dtype=torch.float64) / max(1, half))).float().to(DEV)
        ahead = [[x - 1 for x in _depths(_parents("tree", n, 8, cpu))] if case["tree"] else list(range(n)) for _ in lens]
        s["pos"] = _i32(ahead) + s["lens"][:, None]
        return s
    if kind == "commit":
        s["table"], pages = _pages_of(case, lens, n, gen, False)
        s.update(_pools(case, pages, gen))
        taken = torch.rand((b, n), generator=cpu).argsort(1)[:, :case["depth"]].sort(1).values  # a path: increasing nodes
        count = torch.randint(0 if b > 1 else case["depth"], case["depth"] + 1, (b,), generator=cpu)
        accepted = torch.full((b, n), -1, dtype=torch.int32)
        accepted[:, :case["depth"]] = torch.where(torch.arange(case["depth"]) < count[:, None], taken, -1).int()
        s["accepted"], s["count"] = accepted.to(DEV), count.int().to(DEV)
        return s
    s["table"], pages = _pages_of(case, lens, n, gen, kind == "verify")
    hot = None
    if case.get("outliers"):                                                     # one cached position in twenty has keys eight times as large
        hot = torch.rand((pages, 1, PAGE, 1), generator=gen, device=DEV) < 0.05
        for i, l in enumerate(lens):                                             # (the drafted tokens' own rows have not)
            own_rows = torch.arange(l, l + n, device=DEV)
            hot[s["table"][i, own_rows // PAGE].long(), 0, own_rows % PAGE, 0] = False
    s.update(_pools(case, pages, gen, hot))
    if kind == "verify":
        s["q"] = torch.randn((b, n, hq, d), generator=gen, device=DEV).to(dt)
        s["parent"] = _i32([_parents(case["tree"], n, 6, cpu) for _ in lens])
        s["counts"] = _i32(_counts(case)) if case["ragged"] else None
    return s


# ----------------------------------------------------------------------------------------------------- plain forms
def _values(raw, scale):
    """What rows of bytes [..., D / 2] with scale bytes [..., D / 32] stand for, in 32 bits."""
    code = torch.stack([raw & 15, raw >> 4], -1).flatten(-2)
    a = (code & 7).float()
    a = torch.where(a < 4, 0.5 * a, torch.where(a < 6, a - 2.0, 2.0 * a - 8.0))  # 0 1/2 1 3/2, 2 3, 4 6
    x = torch.where(code > 7, -a, a).unflatten(-1, (-1, GROUP))
    e = torch.where(scale == 255, torch.nan, _two_to(scale.int() - 127).float())
    return (x * e[..., None]).flatten(-2)


def _normalised(x, gain):
    """x [..., D] times its gain over its root mean square, in 64 bits."""
    x = x.double()
    if gain is None:
        return x
    eps = torch.tensor(_EPS, dtype=torch.float32).double().item()
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * gain.double()


def _rotated(y, cos, sin, case):
    """y [b, n, heads, d] in 64 bits, rotated by the angles whose cosines and sines [b, n, rot_dim / 2] are given."""
    r = case["rot_dim"]
    y, c, s = y.clone(), cos[:, :, None], sin[:, :, None]
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if case["interleaved"] else (y[..., :r // 2], y[..., r // 2:r])
    first, second = a * c - b * s, b * c + a * s
    if case["interleaved"]:
        y[..., 0:r:2], y[..., 1:r:2] = first, second
    else:
        y[..., :r // 2], y[..., r // 2:r] = first, second
    return y


def _rounded(y, dtype):
    """64 bits -> dtype in one rounding: by way of 32 bits rounded to odd, which a second rounding does not see."""
    f = y.float()
    if dtype == torch.float32:
        return f
    past = f.double().abs() > y.abs()
    bits = f.view(torch.int32) - past.int()                                      # towards zero
    bits = torch.where(f.double() == y, bits, bits | 1)
    return bits.view(torch.float32).to(dtype)


def _plain_append(s):
    case = s["case"]
    hq, hkv, d, n = case["hq"], case["hkv"], case["d"], case["n"]
    q, k, v = (x.unflatten(-1, (-1, d)) for x in s["qkv"].split([hq * d, hkv * d, hkv * d], dim=-1))
    angle = s["pos"].double()[..., None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle), torch.sin(angle)
    q, k = (_rounded(_rotated(_normalised(x, gain), cos, sin, case), x.dtype) for x, gain in ((q, s["q_gain"]), (k, s["k_gain"])))
    at = s["lens"].long()[:, None] + torch.arange(n, device=DEV)
    page, slot = s["table"].gather(1, at // PAGE).long(), at % PAGE
    if case["kind"] == "norm":
        s["k"][page, :, slot] = k
        s["v"][page, :, slot] = v
        return {"q": q, "k": s["k"], "v": s["v"]}
    s["k"][page, :, slot], s["k_scale"][page, :, slot] = _quantise(k.float(), case["dtype"])
    s["v"][page, :, slot], s["v_scale"][page, :, slot] = _quantise(v.float(), case["dtype"])
    return {"q": q, "k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _ancestors(parent):
    """[b, n] parents -> [b, n, n] whether node j is on the path from node i to its root."""
    b, n = parent.shape
    step = torch.zeros((b, n, n + 1), device=DEV).scatter_(2, torch.where(parent < 0, n, parent).long()[..., None], 1.0)[..., :n]
    reach = torch.eye(n, device=DEV).expand(b, n, n) + step
    for _ in range(6):                                                           # paths of 1, 2, 4, ... 64 steps
        reach = (reach @ reach).clamp(max=1.0)
    return reach > 0


def _plain_verify(s):
    case = s["case"]
    b, n, hq, hkv, d = (case[x] for x in ("batch", "n", "hq", "hkv", "d"))
    g, long = hq // hkv, s["table"].shape[1] * PAGE
    page = s["table"].long()
    k, v = (_values(pool[page], scale[page]).transpose(1, 2).reshape(b * hkv, long, d) for pool, scale in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])))
    q = s["q"].float().view(b, n, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(b * hkv, n * g, d)
    scores = (torch.bmm(q, k.transpose(1, 2)) / math.sqrt(d)).view(b, hkv, n, g, long)
    node = torch.arange(long, device=DEV) - s["lens"][:, None]                   # [b, long]: the drafted token of a position
    known = _ancestors(s["parent"]).gather(2, node.clamp(0, n - 1)[:, None].expand(b, n, long))
    seen = (node < 0)[:, None] | ((node < n)[:, None] & known)
    scores.masked_fill_(~seen[:, None, :, None], -torch.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    past = (node >= n)[:, None, :, None].expand(b, hkv, long, 1).reshape(b * hkv, long, 1)
    out = torch.bmm(p.view(b * hkv, n * g, long), v.masked_fill(past, 0.0)).view(b, hkv, n, g, d) / p.sum(-1, keepdim=True)
    out = out.permute(0, 2, 1, 3, 4).reshape(b, n, hq, d).to(_TORCH[case["dtype"]])
    if s["counts"] is not None:                                                  # rows of absent nodes are zeros
        out = out * (torch.arange(n, device=DEV) < s["counts"][:, None])[..., None, None]
    return {"out": out}


def _plain_commit(s):
    case = s["case"]
    n, depth, long = case["n"], case["depth"], s["table"].shape[1]
    lens, count = s["lens"].long()[:, None], s["count"].long()[:, None]
    i = torch.arange(depth, device=DEV)
    to = lens + i
    source = torch.where(i < count, lens + s["accepted"][:, :depth].clamp(0, n - 1).long(), to)        # the others stay where they are
    from_page, to_page = (s["table"].gather(1, (x // PAGE).clamp(max=long - 1)).long() for x in (source, to))
    for pool in (s["k"], s["v"], s["k_scale"], s["v_scale"]):
        pool[to_page, :, to % PAGE] = pool[from_page, :, source % PAGE]
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "lens": s["lens"] + s["count"]}


def _plain_gather(s):
    case = s["case"]
    at = case["ctx_lo"] + torch.arange(case["n"], device=DEV)
    page, slot = s["table"][0, at // PAGE].long(), at % PAGE
    return {x: _values(s[x][page, :, slot], s[x + "_scale"][page, :, slot]).to(_TORCH[case["dtype"]]) for x in ("k", "v")}


# ------------------------------------------------------------------------------------------------- the library's calls
def _kept(s):
    """What a program makes once for a shape and keeps: descriptors, output buffers, workspace."""
    from paper_2510_07535_amd import binding as B

    case = s["case"]
    kind, hkv, d, n = case["kind"], case["hkv"], case["d"], case["n"]
    code = {"bf16": B.OWL_BF16, "f16": B.OWL_F16, "f32": B.OWL_F32}[case["dtype"]]
    row = d if kind == "norm" else d // 2                                        # of a cache of 4-bit groups strides count bytes
    desc = B.make_desc(batch=case["batch"], n_draft=min(n, 64), n_q_heads=case.get("hq", hkv), n_kv_heads=hkv, head_dim=d,
                       max_pages_per_seq=s["table"].shape[1], max_ctx_len=s["most"], qkv_dtype=code, scale=1.0 / math.sqrt(d),
                       kv_stride_page=hkv * PAGE * row, kv_stride_head=PAGE * row, kv_stride_token=row, n_pool_pages=s["k"].shape[0],
                       out_dtype=code)
    if kind in ("norm", "append"):
        wide = (case["hq"] + 2 * hkv) * d
        app = B.AppendDesc(n_tokens=n, rot_dim=case["rot_dim"], rot_style=B.OWL_ROT_PAIRS if case["interleaved"] else B.OWL_ROT_HALVES,
                           q_stride=wide, k_stride=wide, v_stride=wide, rot_scale=1.0)
        norm = B.NormDesc(eps=_EPS) if case["norm"] else None
        return B, desc, app, norm, torch.empty((case["batch"], n, case["hq"], d), dtype=s["qkv"].dtype, device=DEV)
    if kind == "commit":
        return B, desc, torch.empty_like(s["lens"])
    if kind == "gather":
        return B, desc, *(torch.empty((n, hkv, d), dtype=_TORCH[case["dtype"]], device=DEV) for _ in range(2))
    return B, desc, torch.empty_like(s["q"]), torch.empty(B.owl_verify_attn_groups_workspace_size(desc), dtype=torch.uint8, device=DEV)


def _own_run(s):
    if "kept" not in s:
        s["kept"] = _kept(s)
    case = s["case"]
    kind, hkv, d = case["kind"], case["hkv"], case["d"]
    if kind in ("norm", "append"):
        B, desc, app, norm, q_out = s["kept"]
        hq = case["hq"]
        q, k, v = s["qkv"].split([hq * d, hkv * d, hkv * d], dim=-1)
        freq = s["inv_freq"] if case["rot_dim"] else None
        if kind == "norm":
            B.owl_append_kv_norm(desc, app, norm, q, k, v, s["q_gain"], s["k_gain"], freq, s["pos"], q_out, s["k"], s["v"], None, None,
                                 s["table"], s["lens"], None, s["status"])
            return {"q": q_out, "k": s["k"], "v": s["v"]}
        B.owl_append_kv_groups(desc, app, norm, q, k, v, s["q_gain"], s["k_gain"], freq, s["pos"], q_out, s["k"], s["v"], s["k_scale"],
                               s["v_scale"], s["table"], s["lens"], None, s["status"])
        return {"q": q_out, "k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if kind == "commit":
        B, desc, new_lens = s["kept"]
        B.owl_commit_kv_groups(desc, s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], s["lens"], s["accepted"], s["count"], new_lens, s["status"])
        return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "lens": new_lens}
    if kind == "gather":
        B, desc, k, v = s["kept"]
        B.owl_gather_kv_groups(desc, s["k"], s["k_scale"], s["table"], 0, case["ctx_lo"], case["n"], k, s["status"])
        B.owl_gather_kv_groups(desc, s["v"], s["v_scale"], s["table"], 0, case["ctx_lo"], case["n"], v, s["status"])
        return {"k": k, "v": v}
    B, desc, out, workspace = s["kept"]
    B.owl_verify_attn_groups(desc, s["q"], s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], s["lens"], s["parent"], s["counts"], out,
                             workspace, s["status"])
    return {"out": out}


def run(s):
    if own:
        return _own_run(s)
    return {"norm": _plain_append, "append": _plain_append, "verify": _plain_verify, "commit": _plain_commit, "gather": _plain_gather}[s["kind"]](s)


# --------------------------------------------------------------------------------------------------- in 64 bits
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _numbers(raw, scale):
    """Cached rows in 64 bits."""
    table = torch.tensor(_E2M1, dtype=torch.float64, device=DEV)
    x = torch.empty((*raw.shape, 2), dtype=torch.float64, device=DEV)
    x[..., 0], x[..., 1] = table[(raw % 16).long()], table[(raw // 16).long()]
    e = scale.double() - 127.0
    return x.flatten(-2) * torch.exp2(e).repeat_interleave(GROUP, -1)


def _exact_append(case, s):
    b, n, hq, hkv, d = (case[x] for x in ("batch", "n", "hq", "hkv", "d"))
    if b * n > 20000:
        return None
    lens, freq = _lens(case), s["inv_freq"].double()
    out_q = torch.empty((b, n, hq, d), dtype=torch.float64, device=DEV)
    pools = [s[x].double() for x in ("k", "v")] if case["kind"] == "norm" else [None, None]
    tokens, table, r = s["qkv"].double(), s["table"].tolist(), case["rot_dim"]
    for i in range(b):
        heads = hq + hkv
        x = tokens[i, :, :heads * d].reshape(n, heads, d).clone()
        if case["norm"]:                                                         # a head's rows have length sqrt(d) without eps and gain
            length = torch.sqrt((x * x).sum(-1, keepdim=True) / d + torch.tensor(_EPS).double().item())
            gain = torch.cat([s["q_gain"].expand(hq, d), s["k_gain"].expand(hkv, d)]).double()
            x = gain * (x / length)
        if r:
            turn = torch.polar(torch.ones((n, 1, r // 2), dtype=torch.float64, device=DEV), (s["pos"][i].double()[:, None] * freq)[:, None])
            pairs = x[..., :r].reshape(n, heads, r // 2, 2) if case["interleaved"] else torch.stack([x[..., :r // 2], x[..., r // 2:r]], -1)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            z = z.reshape(n, heads, r) if case["interleaved"] else torch.cat([z[..., 0], z[..., 1]], -1)
            x = torch.cat([z, x[..., r:]], -1)
        out_q[i] = x[:, :hq]
        if case["kind"] == "norm":
            page, slot = torch.tensor([(table[i][(lens[i] + t) // PAGE], (lens[i] + t) % PAGE) for t in range(n)], device=DEV).T
            pools[0][page, :, slot] = x[:, hq:]
            pools[1][page, :, slot] = tokens[i, :, heads * d:].reshape(n, hkv, d)
    return {"q": out_q, "k": pools[0], "v": pools[1], **({} if case["kind"] == "norm" else {"k_scale": None, "v_scale": None})}


def _exact_verify(case, s):
    b, n, hq, hkv, d = (case[x] for x in ("batch", "n", "hq", "hkv", "d"))
    g, lens, counts, out = hq // hkv, _lens(case), _counts(case), torch.zeros((b, n, hq, d), dtype=torch.float64, device=DEV)
    parents = s["parent"].tolist()
    for i in range(b):
        l, c = lens[i], counts[i]
        seen = torch.ones((c, l + c), dtype=torch.bool)
        seen[:, l:] = False
        for node in range(c):
            at = node
            while at >= 0:
                seen[node, l + at] = True
                at = parents[i][at]
        seen = seen.to(DEV)[:, None]
        where = torch.arange(l + c, device=DEV)
        page = s["table"][i, where // PAGE].long()
        for h in range(hkv):
            k, v = (_numbers(s[x][page, h, where % PAGE], s[x + "_scale"][page, h, where % PAGE]) for x in ("k", "v"))
            x = (s["q"][i, :c, h * g:(h + 1) * g].double().reshape(c * g, d) @ k.T).view(c, g, l + c) * d ** -0.5
            w = torch.softmax(x.masked_fill(~seen, -torch.inf), -1)
            out[i, :c, h * g:(h + 1) * g] = (w.view(c * g, l + c) @ v).view(c, g, d)
    return {"out": out}


def _exact_gather(case, s):
    rows = range(case["ctx_lo"], case["ctx_lo"] + case["n"])
    pages = s["table"][0].tolist()
    page = torch.tensor([pages[t // PAGE] for t in rows], device=DEV)
    slot = torch.tensor([t % PAGE for t in rows], device=DEV)
    return {x: _numbers(s[x][page, :, slot], s[x + "_scale"][page, :, slot]) for x in ("k", "v")}


def exact(case, seed):
    if case["kind"] == "commit":                                                 # bytes move, nothing is computed
        return None
    return {"norm": _exact_append, "append": _exact_append, "verify": _exact_verify, "gather": _exact_gather}[case["kind"]](case, prepare(case, seed))
