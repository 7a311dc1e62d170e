"""What a model's layer does around the attention calls, and the draw of the next tokens, as timed cases.

Four operators, each with the calls that a user's program makes of it:

  rows    `rms_norm`: the residual's addition and the root-mean-square norm of token rows, as bf16 or as E4M3 codes
          with a scale for every 128 values of a row; `quantize`: codes and scales of rows alone, or of the gated
          product silu(a) * b of a row's two halves.
  linear  `linear_fp8`: the product of such rows with a weight matrix in E4M3 that has a scale for every block of
          128 x 128, as bf16 or fp32.
  rotary  `rotate`: the position rotation of the new tokens' queries and keys (decode steps and draft trees, whose
          attention takes the new keys itself); `Pool.kv_write_rotated`: queries and keys of packed tokens are
          rotated, and the keys and values enter one layer of the caches (fp8 pools quantise on the way).
  sample  `sample`: one token a row of logits from a given random number, with temperature, top-k, top-p and min-p.

Sizes are those of the repository's own layers (32/8/128 bf16 and 64/8/128 fp8 heads, rows of 4096 values, populations
of 8 to 512 traces, prompts of 256 to 8192 tokens) with generic feed-forward widths and vocabularies, and what lies
between and around them.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
BS, D = 16, 128
E4M3 = torch.float8_e4m3fn
LEAST = 2.0 ** -60  # least scale of a group of 128 values
FLOOR_FULL, FLOOR_OPEN = 2.0 ** -20, 2.0 ** -6  # least fp8 scale of a cache block that a write fills, and of one it leaves open


def listed():
    return [
        # The step of eight traces: the residual's addition and the norm before a product.  The smallest call.
        dict(name="norm_8", kind="rows", op="norm", n=8, heads=0, dim=4096, x32=False, res="bf16", out="fp8", sizes=1),
        # The query heads of a prompt of 2048 tokens, normed a head at a time out of the packed q, k, v rows.
        dict(name="norm_heads_2048", kind="rows", op="norm", n=2048, heads=32, dim=128, x32=False, res="", out="bf16", sizes=2),
        # A prompt of 8192 tokens between the feed-forward layer's two products: silu(a) * b, quantised.
        dict(name="gate_8192", kind="rows", op="gate", n=8192, heads=0, dim=12288, x32=False, res="", out="fp8", sizes=3),
        # Queries, keys and values of eight traces' next tokens: the smallest product, bound by the weights.
        dict(name="linear_8", kind="linear", m=8, k=4096, n=6144, f32=False, sizes=4),
        # The logits of a 64-trace step, fp32: the largest weights.
        dict(name="linear_logits_64", kind="linear", m=64, k=4096, n=151936, f32=True, sizes=5),
        # The second product of the feed-forward layer for an odd number of packed prompt tokens.
        dict(name="linear_777", kind="linear", m=777, k=12288, n=4096, f32=False, sizes=6),
        # The first product of the feed-forward layer for 8192 tokens: the most arithmetic.
        dict(name="linear_8192", kind="linear", m=8192, k=4096, n=24576, f32=False, sizes=7),
        # The decode step of 64 traces: queries and keys out of the packed q, k, v rows, each at its trace's position.
        dict(name="rotate_64", kind="rotary", write=False, hq=32, hkv=8, fp8=False, layers=1, n=64, lo=1, hi=1, pre=8191, rot=128, pairs=False, sizes=8),
        # Sixteen prompts of 256 to 1024 tokens enter an fp8 layer.
        dict(name="write_16_fp8", kind="rotary", write=True, hq=64, hkv=8, fp8=True, layers=1, n=16, lo=256, hi=1024, pre=0, rot=128, pairs=False, sizes=9),
        # Eight long segments behind what the traces hold already, in the second of two layers; half of a head is rotated, in adjacent pairs.
        dict(name="write_segments_8", kind="rotary", write=True, hq=32, hkv=8, fp8=False, layers=2, n=8, lo=1024, hi=4096, pre=37, rot=64, pairs=True, sizes=10),
        # Eight traces draw their next tokens, each with its own temperature, top-k, top-p and min-p, from bf16 logits.
        dict(name="sample_8", kind="sample", n=8, vocab=151936, f32=False, mode="each", sizes=11),
        # A population of 512 traces, fp32 logits, the nucleus of 0.95 at one temperature.
        dict(name="sample_512", kind="sample", n=512, vocab=151936, f32=True, mode="top_p", sizes=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        b = most.setdefault(c["kind"], {"bytes": 0, "flops": 0})
        for k in b:
            b[k] = max(b[k], w[k])
    while True:
        kind = rng.choice(["rows", "linear", "linear", "rotary", "sample"])
        c = dict(kind=kind, sizes=rng.randrange(1 << 20))
        if kind == "rows":
            c.update(op=rng.choice(["norm", "norm", "norm", "gate", "plain"]), n=_log(rng, 1, 16384), heads=0, dim=16 * _log(rng, 1, 1024),
                     x32=rng.random() < 0.3, res="", out="fp8")
            if c["op"] == "norm":
                c.update(res=rng.choice(["", "bf16", "f32"]), out=rng.choice(["bf16", "f32", "fp8"]))
                if not c["res"] and rng.random() < 0.4:
                    c.update(heads=rng.randint(1, 64), n=_log(rng, 1, 2048), dim=16 * _log(rng, 1, 32))
        elif kind == "linear":
            c.update(m=_log(rng, 1, 8192), k=16 * _log(rng, 8, 1024), n=_log(rng, 16, 32768), f32=rng.random() < 0.3)
        elif kind == "rotary":
            g, hkv = rng.choice([1, 2, 4, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 8, 8])
            c.update(write=rng.random() < 0.6, hq=g * hkv, hkv=hkv, fp8=rng.random() < 0.4, layers=rng.choice([1, 1, 2, 3]), n=_log(rng, 1, 128),
                     pre=rng.choice([0, _log(rng, 1, 30000)]), rot=rng.choice([128, 128, 128, 16 * rng.randint(1, 8)]), pairs=rng.random() < 0.4)
            c["hi"] = _log(rng, 1, 4096 if c["write"] else 64)
            c["lo"] = rng.choice([0, 1, max(1, c["hi"] // 4)])
            if not c["write"]:
                c.update(fp8=False, layers=1)
            elif c["n"] * (c["pre"] + c["hi"]) * hkv > 4 << 20:
                continue
        else:
            c.update(n=_log(rng, 1, 512), vocab=_log(rng, 20, 200000), f32=rng.random() < 0.5, mode=rng.choice(["all", "top_k", "top_p", "each", "each"]))
        w, m = work(c), most[kind]
        if w["bytes"] > m["bytes"] or w["flops"] > m["flops"]:
            continue
        return c


def _counts(case):
    r = random.Random(case["sizes"])
    new = [r.randint(case["lo"], case["hi"]) for _ in range(case["n"])]
    if not any(new):
        new[0] = 1
    return new


def work(case):
    if case["kind"] == "rows":
        n, dim = case["n"] * max(1, case["heads"]), case["dim"]
        b = n * dim * ((4 if case["x32"] else 2) * (2 if case["op"] == "gate" else 1) + {"bf16": 2, "f32": 4, "fp8": 1}[case["out"]])
        if case["res"]:
            b += 2 * n * dim * {"bf16": 2, "f32": 4}[case["res"]]
        if case["out"] == "fp8":
            b += 4 * n * -(-dim // 128)
        return {"bytes": b + (2 * dim if case["op"] == "norm" else 0), "flops": 0}
    if case["kind"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        kb = -(-k // 128)
        return {"bytes": m * k + n * k + 4 * kb * (m + -(-n // 128)) + m * n * (4 if case["f32"] else 2), "flops": 2 * m * n * k}
    if case["kind"] == "rotary":
        N, row = sum(_counts(case)), D * 2
        b = N * (2 * case["hq"] + 2 * case["hkv"]) * row + 4 * case["rot"] * min(N, max(_counts(case)))
        if case["write"]:
            b += N * case["hkv"] * D * (1 if case["fp8"] else 2) * 2
        return {"bytes": b, "flops": 0}
    return {"bytes": case["n"] * case["vocab"] * (4 if case["f32"] else 2), "flops": 0}


# ---- inputs ------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)


def _rows_inputs(case, seed):
    gen, n, dim = _gen(seed), case["n"], case["dim"]
    dt = torch.float32 if case["x32"] else torch.bfloat16
    if case["heads"]:  # the first heads of rows that hold half as many again
        x = _normal(gen, n, case["heads"] + case["heads"] // 2, dim).to(dt)[:, : case["heads"]]
    else:
        x = _normal(gen, n, dim * (2 if case["op"] == "gate" else 1)).to(dt)
    s = dict(case=case, x=x, weight=(1 + 0.2 * _normal(gen, dim)).to(torch.bfloat16), eps=1e-6)
    if case["res"]:
        # a residual stream has a few columns that are far larger than the others
        r = 4 * _normal(gen, n, dim) * (1 + 30 * (torch.rand(dim, generator=gen, device=DEV) < 0.004))
        s["res"] = r.to(torch.float32 if case["res"] == "f32" else torch.bfloat16)
        s["res_out"] = torch.empty_like(s["res"])
    return s


def _linear_inputs(case, seed):
    gen, m, k, n = _gen(seed), case["m"], case["k"], case["n"]
    kb, nb = -(-k // 128), -(-n // 128)
    ws = 0.02 / 100 * (0.5 + torch.rand((nb, kb), generator=gen, device=DEV))
    xs = 1 / 150 * (0.5 + torch.rand((kb, m), generator=gen, device=DEV))
    x = (100 * _normal(gen, m, k)).clamp_(-448, 448).to(E4M3)
    w = torch.empty(n, k, dtype=E4M3, device=DEV)
    for a in range(0, n, 32768):
        w[a:a + 32768] = (100 * _normal(gen, min(32768, n - a), k)).clamp_(-448, 448).to(E4M3)
    return dict(case=case, x=x, xs=xs, w=w, ws=ws)


def _table(n_pos, rot):
    """cos and sin of every position's angles, [n_pos][rot]: the angles in 64 bits."""
    angle = torch.arange(n_pos, device=DEV, dtype=torch.float64)[:, None] * 1e6 ** (-2 * torch.arange(rot // 2, device=DEV, dtype=torch.float64) / rot)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _rotary_inputs(case, seed):
    gen, new = _gen(seed), _counts(case)
    N, hq, hkv = sum(new), case["hq"], case["hkv"]
    qkv = _normal(gen, N, hq + 2 * hkv, D).to(torch.bfloat16)
    q, k, v = qkv.split([hq, hkv, hkv], 1)
    pos = np.concatenate([np.arange(case["pre"], case["pre"] + c) for c in new])
    s = dict(case=case, new=new, q=q, k=k, v=v, pos=torch.from_numpy(pos).to(DEV, torch.int32), table=_table(int(pos.max()) + 1, case["rot"]))
    if case["write"]:
        nb = [-(-(case["pre"] + c) // BS) for c in new]
        first = np.concatenate([[0], np.cumsum(nb)])
        end = np.repeat([case["pre"] + c for c in new], new)
        dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(DEV, t)  # noqa: E731
        s.update(blocks=int(first[-1]), block=dev(np.repeat(first[:-1], new) + pos // BS, torch.int64), slot=dev(pos % BS, torch.int64),
                 started=dev(pos // BS * BS >= case["pre"], torch.bool),
                 floor=dev(np.where((pos // BS + 1) * BS <= end, FLOOR_FULL, FLOOR_OPEN), torch.float32))
    return s


def _sample_inputs(case, seed):
    gen, n, V = _gen(seed), case["n"], case["vocab"]
    # a broad bulk, and a few tokens far above it: how far differs from row to row
    z = 2.5 * _normal(gen, n, V)
    tops = min(V, 40)
    at = torch.randint(0, V, (n, tops), generator=gen, device=DEV)
    z.scatter_(1, at, 8 + (2 + 6 * torch.rand((n, 1), generator=gen, device=DEV)) * torch.rand((n, tops), generator=gen, device=DEV))
    s = dict(case=case, z=z if case["f32"] else z.to(torch.bfloat16), u=torch.rand(n, generator=gen, device=DEV))
    r = random.Random(case["sizes"])
    if case["mode"] == "each":
        dev = lambda f, t: torch.tensor([f() for _ in range(n)], dtype=t, device=DEV)  # noqa: E731
        s.update(temperature=dev(lambda: r.choice([0.0, 0.6, 0.7, 0.8, 1.0, 1.3]), torch.float32), top_k=dev(lambda: r.choice([0, 1, 20, 40, 1000]), torch.int32),
                 top_p=dev(lambda: r.choice([1.0, 0.95, 0.9, 0.5]), torch.float32), min_p=dev(lambda: r.choice([0.0, 0.0, 0.05, 0.1]), torch.float32))
    else:
        s.update(temperature=r.choice([0.6, 0.8, 1.0]), top_k=r.choice([20, 50, 400]) if case["mode"] == "top_k" else 0,
                 top_p=0.95 if case["mode"] == "top_p" else 1.0, min_p=0.0)
    return s


INPUTS = {"rows": _rows_inputs, "linear": _linear_inputs, "rotary": _rotary_inputs, "sample": _sample_inputs}


def prepare(case, seed):
    s = INPUTS[case["kind"]](case, seed)
    if case["kind"] == "rotary" and case["write"]:
        layers = case["layers"]
        if own:
            from paper_2608_08020_amd import gambit

            pool = gambit.Pool(num_blocks=s["blocks"], num_q_heads=case["hq"], num_kv_heads=case["hkv"], max_traces=case["n"],
                               max_blocks_per_trace=max(1, -(-(case["pre"] + max(s["new"])) // BS)),
                               kv_dtype="fp8_e4m3" if case["fp8"] else "bf16", num_layers=layers, max_splits=8, device=DEV)
            pool.k_cache.zero_()
            pool.v_cache.zero_()
            ids = np.arange(case["n"], dtype=np.int32)
            pool.kv_alloc(ids, np.array([case["pre"] + c for c in s["new"]], np.int32))
            s.update(pool=pool, ids=ids, at=np.full(case["n"], case["pre"], np.int32), count=np.array(s["new"], np.int32))
        else:
            es = torch.uint8 if case["fp8"] else torch.bfloat16
            s["caches"] = [torch.zeros(s["blocks"], case["hkv"], BS, D, dtype=es, device=DEV) for _ in range(2)]
            s["scale"] = torch.ones(s["blocks"], 2, device=DEV)
    if case["kind"] == "sample" and not own:
        for k, t in (("temperature", torch.float32), ("top_k", torch.int32), ("top_p", torch.float32), ("min_p", torch.float32)):
            if not isinstance(s[k], torch.Tensor):
                s[k] = torch.full((case["n"],), s[k], dtype=t, device=DEV)
    return s


# ---- one pass ----------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return _call(s)
    return {"rows": _plain_rows, "linear": _plain_linear, "rotary": _plain_rotary, "sample": _plain_sample}[case["kind"]](s)


def _call(s):
    from paper_2608_08020_amd import gambit

    case = s["case"]
    if case["kind"] == "rows":
        if case["op"] != "norm":
            return list(gambit.quantize(s["x"], gated=case["op"] == "gate"))
        od = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": E4M3}[case["out"]]
        y = gambit.rms_norm(s["x"], s["weight"], s["eps"], residual=s.get("res"), residual_out=s.get("res_out"), out_dtype=od)
        return [*(y if case["out"] == "fp8" else [y]), *([s["res_out"]] if case["res"] else [])]
    if case["kind"] == "linear":
        return gambit.linear_fp8(s["x"], s["xs"], s["w"], s["ws"], out_dtype=torch.float32 if case["f32"] else torch.bfloat16)
    if case["kind"] == "sample":
        return gambit.sample(s["z"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    if not case["write"]:
        return list(gambit.rotate(s["q"], s["k"], s["pos"], s["table"], pairs=case["pairs"]))
    layer, pool = case["layers"] - 1, s["pool"]
    q = pool.kv_write_rotated(layer, s["ids"], s["at"], s["count"], s["k"], s["v"], s["table"], q=s["q"], pairs=case["pairs"])
    at = (lambda t: t[layer]) if case["layers"] > 1 else (lambda t: t)
    kc, vc = at(pool.k_cache), at(pool.v_cache)
    if case["fp8"]:
        return [q, kc.view(E4M3), vc.view(E4M3), at(pool.kv_scale)]
    return [q, kc, vc]


def _plain_rows(s):
    case, x = s["case"], s["x"].float()
    dim, out = case["dim"], []
    if case["op"] == "gate":
        x = x[:, :dim] / (1 + torch.exp(-x[:, :dim])) * x[:, dim:]
    if case["op"] == "norm":
        if case["res"]:
            x = x + s["res"].float()
            s["res_out"].copy_(x)
            out.append(s["res_out"])
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * s["weight"].float()
    if case["out"] != "fp8":
        return [x if case["out"] == "f32" else x.to(torch.bfloat16)] + out
    x = x.reshape(-1, dim)
    pad = -dim % 128
    y = torch.cat([x, x.new_zeros(x.shape[0], pad)], 1) if pad else x
    y = y.view(x.shape[0], -1, 128)
    scale = torch.clamp_min(y.abs().amax(2) / 448.0, LEAST)
    code = (y / scale[..., None]).clamp(-448.0, 448.0).to(E4M3).view(x.shape[0], -1)[:, :dim]
    return [code.reshape(s["x"].shape[:-1] + (dim,)), scale.T.contiguous()] + out


def _plain_linear(s):
    case, k, n = s["case"], s["case"]["k"], s["case"]["n"]
    x = s["x"].float() * s["xs"].T.repeat_interleave(128, 1)[:, :k]
    y = torch.empty(case["m"], n, dtype=torch.float32 if case["f32"] else torch.bfloat16, device=DEV)
    ws = s["ws"].repeat_interleave(128, 1)[:, :k]
    for a in range(0, n, 65536):  # the weights in 32 bits a part at a time
        b = min(n, a + 65536)
        w = s["w"][a:b].float() * ws[a // 128:-(-b // 128)].repeat_interleave(128, 0)[: b - a]
        y[:, a:b] = x @ w.T
    return y


def _turned(x, cs, pairs):
    """Rows x [N][heads][128], the first 2 r values of a head rotated by cs [N][2 r], in 32 bits."""
    r = cs.shape[1] // 2
    x, c, z = x.float(), cs[:, None, :r], cs[:, None, r:]
    a, b = (x[..., 0:2 * r:2], x[..., 1:2 * r:2]) if pairs else (x[..., :r], x[..., r:2 * r])
    a, b = a * c - b * z, b * c + a * z
    y = torch.stack([a, b], -1).flatten(2) if pairs else torch.cat([a, b], 2)
    return torch.cat([y, x[..., 2 * r:]], 2)


def _swap(t):
    """Row of token t in a K tile: bits 2 and 3 swapped."""
    return (t & 3) | ((t >> 1) & 4) | ((t << 1) & 8)


def _plain_rotary(s):
    case = s["case"]
    cs = s["table"][s["pos"].long()]
    q, k = _turned(s["q"], cs, case["pairs"]).to(torch.bfloat16), _turned(s["k"], cs, case["pairs"])
    if not case["write"]:
        return [q, k.to(torch.bfloat16)]
    v, (kc, vc) = s["v"], s["caches"]
    C = 16 if case["fp8"] else 8
    if case["fp8"]:
        most = torch.stack([x.float().abs().amax((1, 2)) for x in (k, v)], 1)
        most = torch.where(s["started"][:, None], torch.maximum(most / 448.0, s["floor"][:, None]), torch.zeros_like(most))
        least = torch.zeros_like(s["scale"]).scatter_reduce(0, s["block"][:, None].expand(-1, 2), most, "amax")
        s["scale"] = torch.where(least > 0, least, s["scale"])
        sc = s["scale"][s["block"]]
        code = lambda x, f: (x.float() / f.view(-1, 1, 1)).clamp(-448.0, 448.0).to(E4M3).view(torch.uint8)  # noqa: E731
        k, v = code(k, sc[:, 0]), code(v, sc[:, 1])
    else:
        k = k.to(torch.bfloat16)
    kc.view(-1, case["hkv"], D // C, BS, C)[s["block"], :, :, _swap(s["slot"])] = k.reshape(-1, case["hkv"], D // C, C)
    vc.view(-1, case["hkv"], D, BS)[s["block"], :, :, s["slot"]] = v
    return [q, kc.view(E4M3), vc.view(E4M3), s["scale"]] if case["fp8"] else [q, kc, vc]


def _plain_sample(s):
    z = s["z"].double()
    V = z.shape[1]
    t, k = s["temperature"].double()[:, None], s["top_k"].long()[:, None]
    z = z - z.amax(1, keepdim=True)
    greedy = t <= 0
    w = torch.where(greedy, (z == 0).double(), torch.exp(z / torch.where(greedy, 1.0, t)))
    order = torch.sort(z, dim=1, descending=True, stable=True).indices
    w = w.gather(1, order)
    rank = torch.arange(V, device=DEV)
    w = w * (rank < torch.where(greedy, 1, torch.where((k > 0) & (k < V), k, V)))
    before = torch.cumsum(w, 1) - w
    p, least = s["top_p"].double()[:, None], s["min_p"].double()[:, None]
    w = w * (((p >= 1) | (before < p * w.sum(1, keepdim=True)) | (rank == 0)) & (w >= least))
    w = torch.zeros_like(w).scatter_(1, order, w)
    upto = torch.cumsum(w, 1)
    return (upto <= s["u"].double()[:, None] * upto[:, -1:]).sum(1).to(torch.int32)


# ---- from the definition, in 64 bits -------------------------------------------
def _in_groups(y):
    """Values over their group's scale, and the scales, of rows y."""
    n, dim = y.shape
    scale = torch.stack([y[:, a:a + 128].abs().max(1).values for a in range(0, dim, 128)]) / 448
    scale = scale.clamp(min=LEAST)
    return y / scale.T[:, torch.arange(dim, device=DEV) // 128], scale


def exact(case, seed):
    s = INPUTS[case["kind"]](case, seed)
    if case["kind"] == "rows":
        x, dim, more = s["x"].double(), case["dim"], []
        if case["op"] == "gate":
            x = x[:, dim:] * x[:, :dim] * torch.sigmoid(x[:, :dim])
        elif case["op"] == "norm":
            if case["res"]:
                x = x + s["res"]
                more = [x]
            x = x * s["weight"].double() * (x.square().sum(-1, keepdim=True) / dim + s["eps"]) ** -0.5
        if case["out"] != "fp8":
            return [x] + more
        code, scale = _in_groups(x.reshape(-1, dim))
        return [code.view(x.shape), scale] + more
    if case["kind"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        y = torch.zeros(m, n, dtype=torch.float64, device=DEV)
        for a in range(0, k, 1024):  # whole blocks of the sum at a time
            j = torch.arange(a, min(k, a + 1024), device=DEV)
            x = s["x"][:, a:a + 1024].double() * s["xs"].double()[j // 128].T
            w = s["w"][:, a:a + 1024].double() * s["ws"].double()[torch.arange(n, device=DEV) // 128][:, j // 128]
            y.addmm_(x, w.T)
        return y
    if case["kind"] == "rotary":
        r = case["rot"] // 2
        d = torch.arange(r, device=DEV)
        first, second = (2 * d, 2 * d + 1) if case["pairs"] else (d, d + r)
        turn = torch.complex(s["table"][:, :r].double(), s["table"][:, r:].double())[s["pos"].long()][:, None]

        def turned(x):
            x = x.double()
            y = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = y.real, y.imag
            return x

        q, k = turned(s["q"]), turned(s["k"])
        if not case["write"]:
            return [q, k]
        C, d = 16 if case["fp8"] else 8, torch.arange(D, device=DEV)
        row = torch.tensor([0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15], device=DEV)[s["slot"]]
        place = [(torch.div(d, C, rounding_mode="floor") * BS + row[:, None]) * C + d % C, d * BS + s["slot"][:, None]]
        out = [torch.zeros(s["blocks"], case["hkv"], BS * D, dtype=torch.float64, device=DEV) for _ in range(2)]
        scale = torch.ones(s["blocks"], 2, dtype=torch.float64, device=DEV)
        h = torch.arange(case["hkv"], device=DEV)
        for i, y in enumerate((k, s["v"].double())):
            if case["fp8"]:
                st = s["started"]
                size = torch.maximum(y.abs().flatten(1).max(1).values / 448, s["floor"].double())[st]
                found = torch.zeros_like(scale[:, i]).scatter_reduce(0, s["block"][st], size, "amax")
                scale[:, i] = torch.where(found > 0, found, scale[:, i])
                y = (y / scale[s["block"], i].view(-1, 1, 1)).clamp(-448, 448)
            out[i][s["block"][:, None, None], h[:, None], place[i][:, None]] = y
        out = [q] + [t.view(-1, case["hkv"], BS, D) for t in out]
        return out + [scale] if case["fp8"] else out
    get = lambda k: (s[k].tolist() if isinstance(s[k], torch.Tensor) else [s[k]] * case["n"])  # noqa: E731
    got = []
    for z, u, t, k, p, least in zip(s["z"], s["u"].tolist(), get("temperature"), get("top_k"), get("top_p"), get("min_p")):
        z = z.double()
        down = torch.sort(z, dim=0, descending=True, stable=True).indices  # likeliest first, of equal ones the earlier
        if t <= 0:
            got.append(down[:1])
            continue
        if 0 < k < len(z):
            down = down[:k]
        prob = torch.softmax(z[down] / t, 0)
        if p < 1:
            mass = prob.cumsum(0)
            down = down[:1 + int((mass[:-1] < p).sum())]
        down = down[torch.softmax(z[down] / t, 0) >= least * torch.softmax(z[down] / t, 0)[0]]
        down = down.sort().values
        mass = torch.softmax(z[down] / t, 0).cumsum(0)
        got.append(down[torch.searchsorted(mass, u * mass[-1], right=True).clamp(max=len(down) - 1)].view(1))
    return torch.cat(got).to(torch.int32)
