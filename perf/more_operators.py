"""Operators around the experts and the attention of a block on packed tokens: what is measured.

Kinds of a case:
  to_experts  branches sorted by expert (offsets, places, lists) and the tokens' rows copied in that order
  back        the experts' rows back to their tokens: residual + weighted sum
  grad        the gradients of both: of the experts' rows, of the weights and of the tokens
  qk          RMS norm of every query and key head and its position rotation, read from a fused projection
  attention   softmax(q k^T) v over packed sequences of different lengths, grouped heads, causal or not

Types: bf16, or fp32 (the debug path).  Sums are fp32 in both.
"""
import math
import random

import torch

own = False

VALUES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(kind, name=None, **kw):
    base = {
        "to_experts": dict(tokens=4096, slots=2, experts=16, width=1152, dtype="bf16", empty=0.0),
        "back": dict(tokens=4096, slots=2, experts=16, width=1152, dtype="bf16", empty=0.0),
        "grad": dict(tokens=4096, slots=2, experts=16, width=1152, dtype="bf16", empty=0.0),
        "qk": dict(tokens=4096, heads=16, kv_heads=16, dim=72, rot=72, pairs=False, dtype="bf16"),
        "attention": dict(seqs=16, queries=4096, keys=4096, heads=16, kv_heads=16, dim=72, causal=False, even=True,
                          dtype="bf16"),
    }[kind]
    c = dict(base, kind=kind, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One token's two branches: the latency of the calls.
        _case("to_experts", "to_experts_one_token", tokens=1),
        # Fine-grained experts at the largest batch; some branches are served from the cache and not sorted.
        _case("to_experts", "to_experts_k8", tokens=32768, slots=8, experts=64, empty=0.2),
        # Two routed experts of the widest model's layer (1024px images).
        _case("back", "back_d2560", width=2560, experts=4),
        # Many short samples, a width that is no multiple of 16 bytes, half of the branches elsewhere.
        _case("back", "back_ragged", tokens=20011, slots=3, experts=37, width=1001, empty=0.5),
        # A training step of the 28-layer model's layer.
        _case("grad", "grad_d1152"),
        # The same in fp32 with eight branches a token.
        _case("grad", "grad_k8_f32", tokens=8191, slots=8, experts=64, width=768, dtype="f32", empty=0.1),
        # One token through the norms and the rotation.
        _case("qk", "qk_one_token", tokens=1, heads=12, kv_heads=12, dim=64, rot=64),
        # Four 1024px images, shared key heads, rotation over part of the head, interleaved pairs.
        _case("qk", "qk_images", tokens=16384, heads=20, kv_heads=4, dim=128, rot=96, pairs=True),
        # 16 images of 256 tokens, heads of 72 channels.
        _case("attention", "attention_images"),
        # Prompts of different lengths in one batch, causal, four query heads to a key head: the largest.
        _case("attention", "attention_prompts", seqs=5, queries=16384, keys=16384, heads=32, kv_heads=8, dim=128,
              causal=True, even=False),
        # One new token for each of four long sequences of different lengths.
        _case("attention", "attention_one_token", seqs=4, queries=4, keys=131072, heads=32, kv_heads=8, dim=128,
              causal=True, even=False),
        # Short texts in fp32.
        _case("attention", "attention_texts_f32", seqs=4, queries=300, keys=300, heads=12, kv_heads=12, dim=64,
              even=False, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["to_experts", "back", "grad", "qk", "attention", "attention", "attention"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("to_experts", "back", "grad"):
        tokens, slots, width = _log_int(rng, 1, 32768), rng.randint(1, 8), _log_int(rng, 64, 2560)
        while tokens * slots * width > 150_000_000:
            tokens = tokens * 2 // 3
        return _case(kind, tokens=tokens, slots=slots, experts=_log_int(rng, max(2, slots), 256), width=width,
                     dtype=dtype, empty=rng.choice([0.0, 0.0, 0.3]))
    heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 1, 2, 3, 4, 5, 8])
    if kind == "qk":
        dim = rng.choice([32, 64, 72, 80, 96, 100, 128, 192])
        tokens = _log_int(rng, 1, 32768)
        while tokens * heads * (1 + group) * dim > 60_000_000:
            tokens = tokens * 2 // 3
        return _case(kind, tokens=tokens, heads=heads * group, kv_heads=heads, dim=dim, dtype=dtype,
                     rot=rng.choice([dim, dim, dim // 2]), pairs=rng.random() < 0.5)
    c = dict(heads=heads * group, kv_heads=heads, dim=rng.choice([64, 72, 80, 96, 128]), dtype=dtype)
    form = rng.choice(["images", "prompts", "rows", "tokens"])
    if dtype == "f32":  # the debug path: short sequences
        seqs = rng.randint(1, 8)
        keys = seqs * _log_int(rng, 1, 256)
        queries = seqs if form == "tokens" else keys
        return _case(kind, seqs=seqs, queries=queries, keys=keys, causal=form == "prompts", even=form == "images", **c)
    if form == "tokens":
        seqs = _log_int(rng, 1, 64)
        keys = seqs * _log_int(rng, 1, 65536)
        while keys * heads * c["dim"] > 130_000_000:
            keys = max(seqs, keys // 2 // seqs * seqs)
        return _case(kind, seqs=seqs, queries=seqs, keys=keys, causal=True, even=rng.random() < 0.3, **c)
    seqs = _log_int(rng, 1, 32)
    each = _log_int(rng, 1, 8192)
    while seqs * each > 16384 or 4 * seqs * each * each * c["heads"] * c["dim"] > 3e11:
        each = each * 2 // 3
    each = max(each, 1)
    if form == "images":
        return _case(kind, seqs=seqs, queries=seqs * each, keys=seqs * each, **c)
    if form == "prompts":
        return _case(kind, seqs=seqs, queries=seqs * each, keys=seqs * each, causal=True, even=False, **c)
    # A cache step: only some rows of each sample are computed anew, against all of its keys.
    queries = max(1, int(seqs * each * rng.uniform(0.05, 0.6)))
    return _case(kind, seqs=seqs, queries=queries, keys=seqs * each, even=False, **c)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------


def _parts(rng, total, parts):
    """`total` split into uneven parts."""
    share = [rng.uniform(0.1, 1.0) for _ in range(parts)]
    cuts, acc = [0], 0.0
    for s in share[:-1]:
        acc += s
        cuts.append(int(total * acc / sum(share)))
    cuts.append(total)
    return [b - a for a, b in zip(cuts, cuts[1:])]


def _lengths(case):
    """Query and key lengths of the sequences: of the case, not of the seed."""
    n, Q, K = case["seqs"], case["queries"], case["keys"]
    if case["even"]:
        return [Q // n] * n, [K // n] * n
    rng = random.Random(f"{n} {Q} {K} {case['heads']} {case['dim']}")
    if Q == n:  # a new token sees itself
        return [1] * n, [1 + x for x in _parts(rng, K - n, n)]
    if Q == K:
        k = _parts(rng, K, n)
        return k, k
    k = _parts(rng, K, n)
    q = [min(a, b) for a, b in zip(_parts(rng, Q, n), k)]
    left = Q - sum(q)
    for i in range(n):
        more = min(left, k[i] - q[i])
        q[i] += more
        left -= more
    return q, k


def _even_queries(case):
    return case["even"] or case["queries"] == case["seqs"]


def _ids(g, case):
    """Distinct experts for a token's slots, some experts liked more; -1: a branch that is not sorted."""
    T, k, E = case["tokens"], case["slots"], case["experts"]
    like = torch.randn(E, device="cuda", generator=g)
    noise = -torch.log(-torch.log(torch.rand((T, E), device="cuda", generator=g).clamp(1e-7, 1 - 1e-6)))
    ids = (noise + 0.5 * like).topk(k, -1).indices
    drop = torch.rand((T, k), device="cuda", generator=g) < case["empty"]
    return torch.where(drop, -1, ids).to(torch.int32)


def _rows(g, rows, width, dtype):
    x = torch.randn((rows, width), device="cuda", generator=g)
    x *= torch.exp(0.5 * torch.randn((rows, 1), device="cuda", generator=g))
    return x.to(VALUES[dtype])


def _plan(ids, experts):
    """offsets [E + 1], place [T, k], slot [T k] and token [T k], all int32."""
    T, k = ids.shape
    flat = ids.flatten().long()
    key = torch.where((flat >= 0) & (flat < experts), flat, experts)
    order = key.argsort(stable=True)
    row = torch.arange(T * k, device=ids.device)
    count = (key[:, None] == torch.arange(experts, device=ids.device)).sum(0) if T * k * experts <= 1 << 24 else \
        torch.bincount(key, minlength=experts + 1)[:experts]
    offsets = torch.nn.functional.pad(count.cumsum(0), (1, 0))
    place = torch.empty_like(row)
    place[order] = row
    place = torch.where(key < experts, place, -1).view(T, k)
    slot = torch.where(row < offsets[-1], order, -1)
    token = torch.where(slot >= 0, slot // k, -1)
    return [t.to(torch.int32) for t in (offsets, place, slot, token)]


def _table(g, positions, rot):
    """cos and sin [P, rot / 2, 2] of a square image's positions: half of the pairs turn with y, half with x."""
    side = max(1, math.isqrt(positions))
    at = torch.arange(positions, device="cuda", dtype=torch.float64)
    yx = torch.stack([at // side, at % side], -1) + torch.rand(2, device="cuda", dtype=torch.float64, generator=g)
    pair = torch.arange(rot // 2, device="cuda")
    freq = 10000.0 ** (-(pair // 2).double() / max(1, rot // 4))
    angle = yx[:, pair % 2] * freq
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 1_000_003 + 29)
    kind, dtype = case["kind"], case["dtype"]
    s = dict(case=case)
    if kind in ("to_experts", "back", "grad"):
        T, k, D = case["tokens"], case["slots"], case["width"]
        s["ids"] = _ids(g, case)
        s["x"] = _rows(g, T, D, dtype)
        plan = _plan(s["ids"], case["experts"])
        if kind == "to_experts":
            s["plan"] = [torch.empty_like(t) for t in plan]
        else:
            s["plan"] = plan
            n = int(plan[0][-1])
            s["weights"] = torch.randn((T, k), device="cuda", generator=g).softmax(-1)
            s["rows"] = _rows(g, T * k, D, dtype)
            s["rows"][n:] = 0
            if kind == "grad":
                s["drows"] = _rows(g, T * k, D, dtype)
                s["drows"][n:] = 0
    elif kind == "qk":
        T, H, Hk, d = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
        qkv = _rows(g, T, (H + 2 * Hk) * d, dtype).view(T, H + 2 * Hk, d)
        s["q"], s["k"] = qkv[:, :H], qkv[:, H:H + Hk]
        s["q_weight"], s["k_weight"] = 1 + 0.2 * torch.randn((2, d), device="cuda", generator=g)
        each = 256 if T % 256 == 0 else T
        s["table"] = _table(g, each, case["rot"])
        s["pos"] = (torch.arange(T, device="cuda") % each).to(torch.int32)
    else:
        q_len, k_len = _lengths(case)
        s["q_len"], s["k_len"] = q_len, k_len
        H, Hk, d = case["heads"], case["kv_heads"], case["dim"]
        # Normalised queries and keys, as they leave the norm; queries are a part of their own buffer.
        s["q"] = torch.randn((sum(q_len), H, d), device="cuda", generator=g).to(VALUES[dtype])
        kv = torch.randn((sum(k_len), 2, Hk, d), device="cuda", generator=g)
        kv[:, 0] *= torch.exp(0.3 * torch.randn((sum(k_len), 1, 1), device="cuda", generator=g))
        kv = kv.to(VALUES[dtype])
        s["k"], s["v"] = kv[:, 0], kv[:, 1]

        def offsets(n):
            return torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device="cuda")

        s["q_off"] = None if _even_queries(case) else offsets(q_len)
        s["k_off"] = None if case["even"] else offsets(k_len)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------


def _branches(rows, place):
    """The rows of each token's slots in fp32 [T, k, D], zeros for a slot without one."""
    h = rows[place.clamp(min=0).long()].float()
    return torch.where(place[..., None] >= 0, h, 0.0)


def _rotate(y, table, pos, rot, pairs):
    """y [T, H, d] fp32, the first `rot` channels of each head turned."""
    cs = table[pos.long()][:, None]
    c, s = cs[..., 0], cs[..., 1]
    if pairs:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([turned, y[..., rot:]], -1)


def _attend(q, k, v, causal):
    """q [Lq, H, d], k and v [Lk, Hk, d] in fp32: [Lq, H, d]."""
    Lq, H, d = q.shape
    Lk, Hk, _ = k.shape
    if Lq == 0 or Lk == 0:
        return torch.zeros_like(q)
    qt = q.permute(1, 0, 2).reshape(Hk, H // Hk * Lq, d)
    kt, vt = k.permute(1, 2, 0), v.permute(1, 0, 2)
    hidden = None
    if causal:
        hidden = torch.arange(Lk, device=q.device) > (torch.arange(Lq, device=q.device) + (Lk - Lq))[:, None]
        hidden = hidden.repeat(H // Hk, 1)
    out = []
    step = max(1, (1 << 29) // (H // Hk * Lq * Lk))
    for h in range(0, Hk, step):
        z = qt[h:h + step] @ kt[h:h + step] / math.sqrt(d)
        if hidden is not None:
            z = z.masked_fill(hidden, -math.inf)
        z = z - z.amax(-1, keepdim=True).clamp(min=-3e38)
        p = z.exp()
        total = p.sum(-1, keepdim=True)
        out.append(torch.where(total > 0, (p @ vt[h:h + step]) / total, 0.0))
    return torch.cat(out).view(H, Lq, d).permute(1, 0, 2)


def _plain(s, case):
    kind = case["kind"]
    if kind == "to_experts":
        plan = _plan(s["ids"], case["experts"])
        token = plan[3][:, None]
        rows = torch.where(token >= 0, s["x"][token[:, 0].clamp(min=0).long()], 0.0).to(s["x"].dtype)
        return (*plan, rows)
    if kind == "back":
        h = _branches(s["rows"], s["plan"][1])
        return (s["x"].float() + (h * s["weights"][..., None]).sum(1)).to(s["x"].dtype)
    if kind == "grad":
        place, slot, token = s["plan"][1], s["plan"][2], s["plan"][3]
        dy = s["x"].float()
        w = s["weights"].flatten()[slot.clamp(min=0).long()]
        drows = torch.where(token[:, None] >= 0, w[:, None] * dy[token.clamp(min=0).long()], 0.0)
        dw = (_branches(s["rows"], place) * dy[:, None]).sum(-1)
        return drows.to(s["x"].dtype), dw, _branches(s["drows"], place).sum(1).to(s["x"].dtype)
    if kind == "qk":
        out = []
        for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
            y = x.float()
            y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
            out.append(_rotate(y, s["table"], s["pos"], case["rot"], case["pairs"]).to(x.dtype))
        return tuple(out)
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    out, i, j = [], 0, 0
    for m, n in zip(s["q_len"], s["k_len"]):
        out.append(_attend(q[i:i + m], k[j:j + n], v[j:j + n], case["causal"]))
        i, j = i + m, j + n
    return torch.cat(out).to(s["q"].dtype)


def _own(s, case):
    from paper_2606_15615_gb300 import moeca

    kind = case["kind"]
    if kind == "to_experts":
        plan = moeca.expert_sort(s["ids"], case["experts"], plan=moeca.ExpertPlan(*s["plan"]))
        return (*plan, moeca.expert_rows(s["x"], plan))
    if kind == "back":
        return moeca.expert_combine(s["rows"], moeca.ExpertPlan(*s["plan"]), s["weights"], x=s["x"])
    if kind == "grad":
        plan = moeca.ExpertPlan(*s["plan"])
        drows, dw = moeca.expert_combine_grad(s["x"], s["rows"], plan, s["weights"])
        return drows, dw, moeca.expert_rows_grad(s["drows"], plan)
    if kind == "qk":
        return moeca.qk_norm_rope(s["q"], s["k"], s["table"], q_weight=s["q_weight"], k_weight=s["k_weight"], pos=s["pos"],
                                  eps=1e-6, pairs=case["pairs"])
    return moeca.attention(s["q"], s["k"], s["v"], q_offsets=s["q_off"], k_offsets=s["k_off"], n_seqs=case["seqs"],
                           causal=case["causal"], max_q=max(s["q_len"]))


def run(state):
    return _own(state, state["case"]) if own else _plain(state, state["case"])


# ---------------------------------------------------------------------------
# What a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------


def work(case):
    kind = case["kind"]
    size = 2 if case["dtype"] == "bf16" else 4
    if kind in ("to_experts", "back", "grad"):
        T, k, D = case["tokens"], case["slots"], case["width"]
        n = T * k * (1 - case["empty"])
        if kind == "to_experts":
            return {"bytes": 16 * T * k + 4 * case["experts"] + (T + T * k) * D * size, "flops": T * k}
        if kind == "back":
            return {"bytes": 8 * T * k + (n + 2 * T) * D * size, "flops": 2 * n * D}
        return {"bytes": 12 * T * k + (2 * n + T * k + 2 * T) * D * size, "flops": 4 * n * D}
    if kind == "qk":
        n = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        each = 256 if case["tokens"] % 256 == 0 else case["tokens"]
        return {"bytes": 2 * n * size + each * case["rot"] * 4 + 4 * case["tokens"], "flops": 8 * n}
    q_len, k_len = _lengths(case)
    seen = 0
    for m, n in zip(q_len, k_len):
        lo = max(0, m - n)  # the first rows of a longer query see nothing
        seen += (m - lo) * n - (m - lo) * (m - lo - 1) // 2 if case["causal"] else m * n
    bytes_ = (2 * case["heads"] * sum(q_len) + 2 * case["kv_heads"] * sum(k_len)) * case["dim"] * size
    return {"bytes": bytes_, "flops": 4 * seen * case["heads"] * case["dim"]}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "to_experts":
        ids, E = s["ids"].cpu(), case["experts"]
        T, k = ids.shape
        flat = ids.flatten().tolist()
        lists = [[] for _ in range(E)]
        for i, e in enumerate(flat):
            if 0 <= e < E:
                lists[e].append(i)
        offsets, slot = [0], []
        for each in lists:
            slot += each
            offsets.append(len(slot))
        place = [-1] * (T * k)
        for r, i in enumerate(slot):
            place[i] = r
        n = len(slot)
        slot += [-1] * (T * k - n)
        slot = torch.tensor(slot, device="cuda")
        rows = torch.zeros((T * k, case["width"]), dtype=torch.float64, device="cuda")
        rows[:n] = s["x"].double()[torch.div(slot[:n], k, rounding_mode="floor")]
        token = torch.where(slot >= 0, torch.div(slot, k, rounding_mode="floor"), -1)
        made = [torch.tensor(offsets, device="cuda"), torch.tensor(place, device="cuda").view(T, k), slot, token]
        return (*[t.to(torch.int32) for t in made], rows)
    if kind in ("back", "grad"):
        T, k, D = case["tokens"], case["slots"], case["width"]
        place = s["plan"][1].long()
        x, rows, w = s["x"].double(), s["rows"].double(), s["weights"].double()
        if kind == "back":
            y = x.clone()
            for p in range(k):
                live = place[:, p] >= 0
                y[live] += w[live, p, None] * rows[place[live, p]]
            return y
        drows = torch.zeros((T * k, D), dtype=torch.float64, device="cuda")
        dw = torch.zeros((T, k), dtype=torch.float64, device="cuda")
        dx = torch.zeros((T, D), dtype=torch.float64, device="cuda")
        d_in = s["drows"].double()
        for p in range(k):
            live = (place[:, p] >= 0).nonzero()[:, 0]
            at = place[live, p]
            drows[at] = w[live, p, None] * x[live]
            dw[live, p] = torch.linalg.vecdot(x[live], rows[at])
            dx[live] += d_in[at]
        return drows, dw, dx
    if kind == "qk":
        rot, d = case["rot"], case["dim"]
        # The rotation as complex numbers.
        turn = torch.view_as_complex(s["table"].double())[s["pos"].long()][:, None]
        out = []
        for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
            y = x.double()
            y = y * (torch.linalg.vector_norm(y, dim=-1, keepdim=True).square() / d + 1e-6).rsqrt() * w.double()
            head = y[..., :rot]
            z = head.unflatten(-1, (-1, 2)) if case["pairs"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
            z = z.flatten(-2) if case["pairs"] else z.transpose(-1, -2).flatten(-2)
            out.append(torch.cat([z, y[..., rot:]], -1))
        return tuple(out)
    group, scale = case["heads"] // case["kv_heads"], case["dim"] ** -0.5
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    i = j = 0
    for m, n in zip(s["q_len"], s["k_len"]):
        for h in range(case["heads"]):
            if m == 0 or n == 0:
                continue
            q, k, v = s["q"][i:i + m, h].double(), s["k"][j:j + n, h // group].double(), s["v"][j:j + n, h // group].double()
            z = torch.mm(q, k.T) * scale
            if case["causal"]:
                z += torch.triu(torch.full((m, n), -math.inf, dtype=torch.float64, device="cuda"), n - m + 1)
            o = torch.softmax(z, -1) @ v
            out[i:i + m, h] = o.nan_to_num(0.0) if case["causal"] and m > n else o
        i, j = i + m, j + n
    return out
