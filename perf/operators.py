"""Low-rank adapters beside the shared projection and the optimiser step that trains them, as cases that can be timed.

Three operators: the adapters of many tenants at once (`lora`: forward, one matrix or a group that reads one x), their
gradients (`grad`), and AdamW over many tensors at once with states in 32 bits or in 8 (`adamw`).  `run` computes them in
plain torch operations, or, where `own` is true, through the library's entry points.  Sizes are the layer shapes, batches and
tenant counts that the library's other cases have, and generic ones of the same ranges.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
BLOCK = 256            # elements of a tensor that share a scale where states are held in 8 bits
M_TOP, V_TOP = 1984.0, 4032.0   # the largest code values: 31 * 2^6 and 63 * 2^6
BETA1, BETA2, EPS, DECAY = 0.9, 0.999, 1e-8, 0.01


# ---- the cases -------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one token of one tenant behind one projection: the smallest call there is, all latency
        {"name": "lora_decode_one", "kind": "lora", "out": 4096, "in": 4096, "mats": 1, "tokens": 1, "tenants": 1, "rank": 16,
         "mixed": False, "order": "mixed"},
        # a decode step of 16 tenants, one token each: the adapters of q, k and v together
        {"name": "lora_decode_qkv_16", "kind": "lora", "out": 4096, "in": 4096, "mats": 3, "tokens": 16, "tenants": 16, "rank": 16,
         "mixed": False, "order": "mixed"},
        # a continuous batch: decode tokens and drafted ones of 40 tenants with ranks of every kind, some without an adapter,
        # rows of y that are not a multiple of anything
        {"name": "lora_mixed_200", "kind": "lora", "out": 5003, "in": 4096, "mats": 1, "tokens": 200, "tenants": 40, "rank": 64,
         "mixed": True, "order": "mixed"},
        # long prompts: 8 tenants, 4096 tokens, the up projection
        {"name": "lora_prefill_4096", "kind": "lora", "out": 11008, "in": 4096, "mats": 1, "tokens": 4096, "tenants": 8, "rank": 16,
         "mixed": False, "order": "grouped"},
        # a short training step of three tenants' adapters
        {"name": "grad_short", "kind": "grad", "out": 4096, "in": 4096, "tokens": 96, "tenants": 3, "rank": 8, "mixed": False,
         "order": "grouped"},
        # sequences of uneven length, ranks of every kind, odd sizes
        {"name": "grad_ragged", "kind": "grad", "out": 2999, "in": 5024, "tokens": 1237, "tenants": 7, "rank": 24, "mixed": True,
         "order": "grouped"},
        # a training step of 8 tenants at once, 512 tokens each or so
        {"name": "grad_4096", "kind": "grad", "out": 4096, "in": 4096, "tokens": 4096, "tenants": 8, "rank": 16, "mixed": False,
         "order": "grouped"},
        # two tenants with wide adapters on the up projection and long sequences: the largest
        {"name": "grad_wide_8192", "kind": "grad", "out": 11008, "in": 4096, "tokens": 8192, "tenants": 2, "rank": 64,
         "mixed": False, "order": "grouped"},
        # the 14 adapter matrices of one tenant in one layer
        {"name": "adamw_layer_adapter", "kind": "adamw", "shape": "adapters", "tenants": 1, "hidden": 4096, "ffn": 11008, "rank": 16,
         "bits": 32, "grad": "f32"},
        # the adapters of 16 tenants in one layer, states in 8 bits, odd ranks
        {"name": "adamw_8bit_adapters", "kind": "adamw", "shape": "adapters", "tenants": 16, "hidden": 4096, "ffn": 11008, "rank": 13,
         "bits": 8, "grad": "f32"},
        # a dense fine-tune of one layer's seven matrices, whose fp16 weights the compressor takes next
        {"name": "adamw_dense_layer", "kind": "adamw", "shape": "dense", "tenants": 1, "hidden": 4096, "ffn": 11008, "rank": 0,
         "bits": 32, "grad": "f16"},
        # the same with states in 8 bits
        {"name": "adamw_8bit_dense_layer", "kind": "adamw", "shape": "dense", "tenants": 1, "hidden": 4096, "ffn": 11008, "rank": 0,
         "bits": 8, "grad": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lora", "lora", "lora", "grad", "grad", "adamw"])
    if kind == "adamw":
        shape = rng.choice(["adapters", "adapters", "dense"])
        c = {"kind": kind, "shape": shape, "tenants": _log(rng, 1, 24) if shape == "adapters" else 1, "hidden": 32 * _log(rng, 16, 120),
             "ffn": 32 * _log(rng, 32, 300), "rank": rng.choice([1, 4, 7, 8, 16, 30, 64]) if shape == "adapters" else 0,
             "bits": rng.choice([8, 32]), "grad": rng.choice(["f32", "f16"])}
        return c
    rank = rng.choice([1, 4, 8, 12, 16, 20, 32, 64, 128])
    c = {"kind": kind, "out": _log(rng, 200, 11008), "in": 32 * _log(rng, 8, 344)}
    tokens = _log(rng, 1, 8192)
    if kind == "lora":
        c["mats"] = rng.choice([1, 2, 3]) if tokens <= 64 else 1
    # many tenants in small batches, fewer where the batch is long
    tenants = rng.randint(1, max(1, min(tokens, 64 if tokens <= 512 else 12)))
    while tokens * (2 * c["in"] + 2 * c["out"]) > 8192 * 2 * (4096 + 11008):
        tokens = tokens * 3 // 4
    while tokens > 512 and rank * tenants > 512:
        tenants = max(1, tenants // 2)
    c.update(tokens=tokens, tenants=min(tenants, tokens), rank=rank, mixed=rng.random() < 0.4,
             order=rng.choice(["grouped", "grouped", "mixed"]) if tokens > 64 else "mixed")
    return c


def _ranks(case):
    """Rank of every tenant's adapter; 0: the tenant has none."""
    r, n = case["rank"], case["tenants"]
    if not case["mixed"]:
        return [r] * n
    kinds = [r, max(1, r // 2), max(1, r // 4), max(1, r - 3), 0, max(1, r // 8), r]
    return [kinds[e % len(kinds)] for e in range(n)]


def _tenant_of_token(case):
    """Uneven counts (tenant e has about 1 + e % 5 shares), every tenant at least one token; grouped or dealt out in turn."""
    T, n = case["tokens"], case["tenants"]
    share = [1 + (3 * e) % 5 for e in range(n)]
    total, rest = sum(share), T - n
    count = [1 + rest * s // total for s in share]
    count[0] += T - sum(count)
    grouped = [e for e in range(n) for _ in range(count[e])]
    if case["order"] == "grouped":
        return grouped
    step = next(s for s in range(max(1, int(T * 0.618)), T + 2) if math.gcd(s, T) == 1)
    return [grouped[(i * step) % T] for i in range(T)]


def _adamw_sizes(case):
    h, f, r = case["hidden"], case["ffn"], case["rank"]
    mats = [(h, h)] * 4 + [(f, h)] * 2 + [(h, f)]
    if case["shape"] == "dense":
        return [o * i for o, i in mats]
    return [n for _ in range(case["tenants"]) for o, i in mats for n in (r * i, o * r)]


def work(case):
    if case["kind"] == "adamw":
        n = sum(_adamw_sizes(case))
        blocks = sum(-(-k // BLOCK) for k in _adamw_sizes(case))
        grad = 2 if case["grad"] == "f16" else 4
        state = 16 * n if case["bits"] == 32 else 4 * n + 16 * blocks
        return {"bytes": n * (4 + 4 + 2 + grad) + state, "flops": 16 * n}
    T, out, inn, ranks, tok = case["tokens"], case["out"], case["in"], _ranks(case), _tenant_of_token(case)
    weights = sum(ranks[e] * (inn + out) for e in set(tok))
    rank_of_tokens = sum(ranks[e] for e in tok)
    if case["kind"] == "lora":
        m = case["mats"]
        return {"bytes": 2 * T * inn + m * (4 * T * out + 2 * weights), "flops": 2 * m * rank_of_tokens * (inn + out)}
    # dy, x and dx0 read, dx written; h; A and B read in fp16, their gradients written in binary32
    return {"bytes": 2 * T * (out + 3 * inn) + 4 * rank_of_tokens + 6 * weights, "flops": 4 * rank_of_tokens * (inn + out)}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _normal(shape, std, gen, dtype=torch.float16):
    return torch.empty(shape, dtype=torch.float32, device=DEVICE).normal_(0.0, std, generator=gen).to(dtype)


def _prepare_adapters(case, gen):
    out, inn, T, ranks = case["out"], case["in"], case["tokens"], _ranks(case)
    tok = _tenant_of_token(case)
    s = {"tok": torch.tensor(tok, dtype=torch.int32), "ranks": ranks, "x": _normal((T, inn), 1.0, gen), "out": out}
    s["mats"] = []
    for _ in range(case.get("mats", 1)):
        s["mats"].append({
            "a": [_normal((r, inn), inn ** -0.5, gen) if r else None for r in ranks],
            "b": [_normal((out, r), 0.02, gen) if r else None for r in ranks],
            "scale": torch.tensor([16.0 / r if r else 0.0 for r in ranks], dtype=torch.float32, device=DEVICE),
            # what the shared projection gave
            "y0": _normal((T, out), 1.0, gen) if case["kind"] == "lora" else None,
        })
    # which row of all adapters' ranks put together belongs to which tenant, and its place within that tenant's adapter
    s["owner"] = torch.tensor([e for e, r in enumerate(ranks) for _ in range(r)], dtype=torch.int64, device=DEVICE)
    s["place"] = torch.tensor([j for r in ranks for j in range(r)], dtype=torch.int64, device=DEVICE)
    s["tok_dev"] = s["tok"].to(DEVICE).long()
    return s


def _m_code(u):
    """Code of |m| / scale: 3 exponent bits, 4 fraction bits."""
    step = torch.exp2((torch.floor(torch.log2(u.clamp(min=1.0))) - 4).clamp(min=0.0))
    return torch.round(u / step) * step


def _v_code(u, r):
    """Code of sqrt(v) / scale: 3 exponent bits, 5 fraction bits, rounded up where the fraction of a step and r in [0, 1) together
    pass 1; what is not zero stays so."""
    step = torch.exp2((torch.floor(torch.log2(u.clamp(min=1.0))) - 5).clamp(min=0.0))
    return torch.where(u > 0, (torch.floor(u / step + r) * step).clamp(1.0, V_TOP), torch.zeros_like(u))


def _dither(places, lengths, step):
    """The r of every element, from its index in its tensor and the number of the step: multiplications and shifts in 32 bits."""
    at = torch.arange(int(lengths.sum()), dtype=torch.int64, device=DEVICE) - torch.repeat_interleave(places, lengths)
    k = ((at + step * 0x9E3779B9) & 0xFFFFFFFF) * 0xD1B54A33 & 0xFFFFFFFF
    k = ((k ^ (k >> 15)) * 0xB5297A4D) & 0xFFFFFFFF
    return (((k ^ (k >> 16)) * 0x9E3779B9 & 0xFFFFFFFF) >> 14).float() * 2.0 ** -18


def _table(fraction_bits):
    top = 1 << fraction_bits
    return [float(f) if e == 0 else float((top + f) << (e - 1)) for e in range(8) for f in range(top)]


def _byte_of(value, fraction_bits):
    """The byte (without a sign) that stands for a code value."""
    top = float(1 << fraction_bits)
    e = (torch.floor(torch.log2(value.clamp(min=1.0))) - (fraction_bits - 1)).clamp(min=0.0)
    low = value < top
    f = torch.where(low, value, value / torch.exp2(e - 1) - top)
    return (torch.where(low, torch.zeros_like(e), e) * top + f).to(torch.uint8)


def _prepare_adamw(case, gen):
    sizes = _adamw_sizes(case)
    places, at = [], 0
    for n in sizes:
        places.append(at)
        at += -(-n // BLOCK) * BLOCK
    valid = torch.zeros(at, dtype=torch.float32, device=DEVICE)
    for p, n in zip(places, sizes):
        valid[p:p + n] = 1.0
    grad_type = torch.float16 if case["grad"] == "f16" else torch.float32
    s = {"sizes": sizes, "places": places, "total": at, "bits": case["bits"]}
    s["p"] = _normal((at,), 0.02, gen, torch.float32) * valid
    s["p16"] = s["p"].to(torch.float16)
    s["g"] = (_normal((at,), 1e-3, gen, torch.float32) * valid).to(grad_type)
    m = _normal((at,), 3e-4, gen, torch.float32) * valid
    v = (_normal((at,), 1e-3, gen, torch.float32) * valid).square() * 0.5 + 2e-7 * valid
    del valid
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
        ms, vs = m.abs().amax(1) / M_TOP, v.amax(1).sqrt() / V_TOP
        one = torch.ones((), device=DEVICE)
        mv = _m_code(m.abs() / torch.where(ms > 0, ms, one)[:, None])
        s["m"] = (_byte_of(mv, 4).int() + 128 * (m < 0).int()).to(torch.uint8).view(-1)
        s["v"] = _byte_of(_v_code(v.sqrt() / torch.where(vs > 0, vs, one)[:, None], 0.5), 5).view(-1)
        s["ms"], s["vs"] = ms, vs
    s["place"] = torch.tensor(places, dtype=torch.int64, device=DEVICE)
    s["length"] = torch.tensor([-(-n // BLOCK) * BLOCK for n in sizes], dtype=torch.int64, device=DEVICE)
    s["m_table"] = torch.tensor(_table(4) + [-t for t in _table(4)], dtype=torch.float32, device=DEVICE)
    s["v_table"] = torch.tensor(_table(5), dtype=torch.float32, device=DEVICE)
    s["lr"] = torch.full((1,), 1e-4, dtype=torch.float32, device=DEVICE)
    s["step"] = torch.full((1,), 25, dtype=torch.int64, device=DEVICE)
    s["grad_scale"] = torch.full((1,), 0.5, dtype=torch.float32, device=DEVICE)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    if case["kind"] == "adamw":
        return {"kind": "adamw", **_prepare_adamw(case, gen)}
    s = {"kind": case["kind"], **_prepare_adapters(case, gen)}
    if case["kind"] == "grad":
        T, out, inn, ranks = case["tokens"], case["out"], case["in"], s["ranks"]
        s["dy"] = _normal((T, out), 1e-2, gen)
        s["dx0"] = _normal((T, inn), 1e-2, gen)   # the gradient through the shared projection
        # what the forward pass kept: A x of every token, in rows as wide as the widest adapter
        s["h"] = torch.zeros((T, max(ranks)), dtype=torch.float32, device=DEVICE)
        for e, a in enumerate(s["mats"][0]["a"]):
            if a is not None:
                rows = (s["tok_dev"] == e).nonzero()[:, 0]
                s["h"][rows, :a.shape[0]] = s["x"][rows].float() @ a.float().t()
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------
# All adapters' ranks side by side: A [R, in] and B [out, R] with R the sum of the ranks; a token takes part with the rows of
# its own tenant only.

def _mine(s):
    return s["tok_dev"][:, None] == s["owner"][None, :]


def _all_a(m):
    return torch.cat([a for a in m["a"] if a is not None]).float()


def _all_b(m):
    return torch.cat([b for b in m["b"] if b is not None], dim=1).float()


def _plain_lora(s, m):
    h = s["x"].float() @ _all_a(m).t()
    h = torch.where(_mine(s), h * m["scale"][s["owner"]], torch.zeros_like(h))
    return (m["y0"].float() + h @ _all_b(m).t()).to(torch.float16)


def _plain_grad(s):
    m, dy, mine = s["mats"][0], s["dy"].float(), _mine(s)
    scale = m["scale"][s["owner"]]
    g = dy @ _all_b(m)
    g = torch.where(mine, g * scale, torch.zeros_like(g))
    h = s["h"][:, s["place"]]
    h = torch.where(mine, h * scale, torch.zeros_like(h))
    a, x = _all_a(m), s["x"].float()
    db = torch.split(dy.t() @ h, [r for r in s["ranks"] if r], dim=1)
    return {"dx": (s["dx0"].float() + g @ a).to(torch.float16), "da": (g.t() @ x).reshape(-1),
            "db": torch.cat([d.reshape(-1) for d in db])}


def _decoded(s):
    m = s["m_table"][s["m"].long()].view(-1, BLOCK) * s["ms"][:, None]
    v = (s["v_table"][s["v"].long()].view(-1, BLOCK) * s["vs"][:, None]).square()
    return m.view(-1), v.view(-1)


def _states_of(s):
    """The states: as they are, or of those held in 8 bits the code values and, beside them, the scales."""
    if s["bits"] == 32:
        return {"m": s["m"], "v": s["v"]}
    return {"m": s["m_table"][s["m"].long()].half(), "v": s["v_table"][s["v"].long()].half(), "ms": s["ms"], "vs": s["vs"]}


def _plain_adamw(s):
    m, v = (s["m"], s["v"]) if s["bits"] == 32 else _decoded(s)
    g = s["g"].float() * s["grad_scale"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    t, lr = s["step"].double(), s["lr"]
    c1 = (lr / (1 - BETA1 ** t)).float()
    c2 = (1 - BETA2 ** t).sqrt().float()
    s["p"].copy_(s["p"] * (1 - lr * DECAY) - c1 * m / (v.sqrt() / c2 + EPS))
    s["p16"].copy_(s["p"])
    if s["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
        s["ms"].copy_(m.abs().amax(1) / M_TOP)
        s["vs"].copy_(v.amax(1).sqrt() / V_TOP)
        one = torch.ones_like(s["ms"])
        code = _byte_of(_m_code(m.abs() / torch.where(s["ms"] > 0, s["ms"], one)[:, None]), 4)
        s["m"].copy_((code.int() + 128 * (m < 0).int()).view(-1))
        r = _dither(s["place"], s["length"], s["step"]).view(-1, BLOCK)
        s["v"].copy_(_byte_of(_v_code(v.sqrt() / torch.where(s["vs"] > 0, s["vs"], one)[:, None], r), 5).view(-1))
    return {"p": s["p"], "p16": s["p16"], **_states_of(s)}


# ---- the library's calls ---------------------------------------------------------------------------------------------

def _own_lora(s):
    from paper_2402_10193_amd import binding as bd
    if "group" not in s:   # what a server keeps: the tables of the adapters it has loaded, buffers, the workspace
        tables = [bd.LoraTable(m["a"], m["b"], m["scale"]) for m in s["mats"]]
        s["group"] = bd.LoraGroup(tables, [s["out"]] * len(tables)) if len(tables) > 1 else tables[0]
        T = s["x"].shape[0]
        s["ys"] = [torch.empty_like(m["y0"]) for m in s["mats"]]
        s["ws"] = bd.new_workspace(bd.lora_workspace_bytes(T, len(tables), max(s["ranks"])), DEVICE)
    if len(s["mats"]) == 1:
        return [bd.lora_multitenant(s["x"], s["group"], s["tok"], y0=s["mats"][0]["y0"], y=s["ys"][0], workspace=s["ws"])]
    return bd.lora_multitenant_group(s["x"], s["group"], s["tok"], y0s=[m["y0"] for m in s["mats"]], ys=s["ys"], workspace=s["ws"])


def _own_grad(s):
    from paper_2402_10193_amd import binding as bd
    m = s["mats"][0]
    if "table" not in s:   # what a training program keeps
        T, inn = s["x"].shape
        s["table"] = bd.LoraTable(m["a"], m["b"], m["scale"])
        s["da"] = torch.empty(sum(s["ranks"]) * inn, dtype=torch.float32, device=DEVICE)
        s["db"] = torch.empty(sum(s["ranks"]) * s["out"], dtype=torch.float32, device=DEVICE)
        da = iter(torch.split(s["da"], [r * inn for r in s["ranks"] if r]))
        db = iter(torch.split(s["db"], [r * s["out"] for r in s["ranks"] if r]))
        s["grads"] = bd.LoraGrads(s["table"], [next(da) if r else None for r in s["ranks"]], [next(db) if r else None for r in s["ranks"]])
        s["dx"] = torch.empty_like(s["dx0"])
        s["ws"] = bd.new_workspace(bd.lora_backward_workspace_bytes(T, s["out"], inn, len(s["ranks"]), max(s["ranks"])), DEVICE)
    dx = bd.lora_multitenant_backward(s["dy"], s["x"], s["h"], s["table"], s["tok"], s["grads"], dx0=s["dx0"], dx=s["dx"],
                                      workspace=s["ws"])
    return {"dx": dx, "da": s["da"], "db": s["db"]}


def _own_adamw(s):
    from paper_2402_10193_amd import binding as bd
    if "group" not in s:   # what a training program keeps: the tensors' addresses and sizes, marshalled once
        cut = lambda t: [t[p:p + n] for p, n in zip(s["places"], s["sizes"])]
        scales = lambda t: [t[p // BLOCK:p // BLOCK - (-n // BLOCK)] for p, n in zip(s["places"], s["sizes"])]
        more = {} if s["bits"] == 32 else {"exp_avg_scales": scales(s["ms"]), "exp_avg_sq_scales": scales(s["vs"])}
        s["group"] = bd.AdamWGroup(cut(s["p"]), cut(s["g"]), cut(s["m"]), cut(s["v"]), params_f16=cut(s["p16"]), **more)
    bd.adamw(s["group"], s["lr"], s["step"], beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY, grad_scale=s["grad_scale"])
    states = {"m": s["m"], "v": s["v"]}
    if s["bits"] == 8:
        states = {"m": bd.adamw_values(s["m"], False), "v": bd.adamw_values(s["v"], True), "ms": s["ms"], "vs": s["vs"]}
    return {"p": s["p"], "p16": s["p16"], **states}


def run(state):
    if state["kind"] == "lora":
        return _own_lora(state) if own else [_plain_lora(state, m) for m in state["mats"]]
    if state["kind"] == "grad":
        return _own_grad(state) if own else _plain_grad(state)
    return _own_adamw(state) if own else _plain_adamw(state)


# ---- in 64 bits ------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(s)
    tok, ranks, x = s["tok"].tolist(), s["ranks"], s["x"].double()
    rows_of = [torch.tensor([t for t, e in enumerate(tok) if e == k], dtype=torch.int64, device=DEVICE) for k in range(len(ranks))]
    if case["kind"] == "lora":
        ys = []
        for m in s["mats"]:
            y = m["y0"].double()
            for e, rows in enumerate(rows_of):
                if ranks[e]:
                    y[rows] += float(m["scale"][e]) * ((x[rows] @ m["a"][e].double().t()) @ m["b"][e].double().t())
            ys.append(y)
        return ys
    m, dx, da, db = s["mats"][0], s["dx0"].double(), [], []
    for e, rows in enumerate(rows_of):
        if not ranks[e]:
            continue
        dy, scale = s["dy"][rows].double(), float(m["scale"][e])
        g = scale * (dy @ m["b"][e].double())
        dx[rows] += g @ m["a"][e].double()
        da.append((g.t() @ x[rows]).reshape(-1))
        db.append((scale * (dy.t() @ s["h"][rows, :ranks[e]].double())).reshape(-1))
    return {"dx": dx, "da": torch.cat(da), "db": torch.cat(db)}


def _drawn(n, step):
    """The numbers in [0, 1) that decide how v is rounded, of elements 0 .. n - 1 of a tensor in this step."""
    k = np.arange(n, dtype=np.uint32) + np.uint32(step * 0x9E3779B9 % 2 ** 32)
    for shift, factor in ((0, 0xD1B54A33), (15, 0xB5297A4D), (16, 0x9E3779B9)):
        if shift:
            k = k ^ (k >> np.uint32(shift))
        k = k * np.uint32(factor)
    return (k >> np.uint32(14)).astype(np.float64) / 2 ** 18


def _exact_adamw(s):
    """One tensor after the other, the 8-bit states by search in the sorted code values."""
    out = {"p": torch.zeros_like(s["p"], dtype=torch.float64), "m": torch.zeros(s["total"], dtype=torch.float64, device=DEVICE),
           "v": torch.zeros(s["total"], dtype=torch.float64, device=DEVICE)}
    blocks = s["total"] // BLOCK
    if s["bits"] == 8:
        out["ms"], out["vs"] = (torch.zeros(blocks, dtype=torch.float64, device=DEVICE) for _ in range(2))
    t, lr = int(s["step"]), float(s["lr"])
    for at, n in zip(s["places"], s["sizes"]):
        whole, b0, b1 = -(-n // BLOCK) * BLOCK, at // BLOCK, at // BLOCK - (-n // BLOCK)
        part = slice(at, at + whole)
        g = s["g"][part].double() * float(s["grad_scale"])
        if s["bits"] == 32:
            m, v = s["m"][part].double(), s["v"][part].double()
        else:
            m = s["m_table"].double()[s["m"][part].long()] * s["ms"][b0:b1].double().repeat_interleave(BLOCK)
            v = (s["v_table"].double()[s["v"][part].long()] * s["vs"][b0:b1].double().repeat_interleave(BLOCK)) ** 2
        m.mul_(BETA1).add_(g, alpha=1 - BETA1)
        v.mul_(BETA2).addcmul_(g, g, value=1 - BETA2)
        root = v.sqrt()
        out["p"][part] = s["p"][part].double() * (1 - lr * DECAY) - lr / (1 - BETA1 ** t) * m / (root / math.sqrt(1 - BETA2 ** t) + EPS)
        if s["bits"] == 32:
            out["m"][part], out["v"][part] = m, v
            continue
        for name, value, table, top in (("m", m, s["m_table"][:128], M_TOP), ("v", root, s["v_table"], V_TOP)):
            table = table.double()
            size = value.abs().view(-1, BLOCK)
            scale = size.amax(1) / top
            out[name + "s"][b0:b1] = scale
            u = (size / torch.where(scale > 0, scale, torch.ones_like(scale))[:, None]).reshape(-1).contiguous()
            up = torch.searchsorted(table, u, right=True).clamp(1, table.numel() - 1)   # the first code value above u
            low, high = table[up - 1], table[up]
            if name == "m":   # the nearer one, of two as near the one with the even byte
                near = torch.where((u - low < high - u) | ((u - low == high - u) & (up % 2 == 1)), low, high)
            else:             # the upper one where the part of the way to it and a drawn number reach 1
                low, high = torch.where(u >= table[-1], table[-1], low), torch.where(u >= table[-1], table[-1], high)
                r = torch.from_numpy(_drawn(whole, t)).to(DEVICE)
                near = torch.where(u - low >= (1.0 - r) * (high - low), high, low).clamp(min=1.0)
            near = torch.where(u > 0, near, torch.zeros_like(near))
            out[name][part] = near * torch.sign(value)
    return {"p16": out["p"], **out}
