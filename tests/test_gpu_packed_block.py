"""A DiT-MoE block on packed samples of different lengths, run through the public calls one after another: norm and
rotation of a fused projection's heads, attention, routing, the expert sort, grouped products, the way back; and the
expert half's gradients.  Against the same formulas in 64 bits.

Tolerances.  Every intermediate that is held in bf16 is read back and the next step checked against the formula of
what it was given, so that errors do not add up: each step's own bound, as derived in that call's tests.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, HALF = torch.bfloat16, 2.0 ** -8


@pytest.fixture(scope="module")
def M():
    from paper_2606_15615_gb300 import moeca
    return moeca


def f64(t):
    return t.detach().double().cpu().numpy()


def near(got, want, slack):
    err = np.abs(f64(got) - want)
    assert (err <= slack + HALF * (np.abs(want) + slack) + 2.0 ** -134).all(), float(err.max())


def test_block(M):
    lengths, D, H, Hk, d, E, k, F = [130, 7, 256, 0, 64], 144, 6, 3, 24, 8, 2, 96
    T = sum(lengths)
    g = torch.Generator().manual_seed(11)

    def weight(*shape):
        return (torch.randn(*shape, generator=g) / shape[-1] ** 0.5).to(BF).cuda()

    x = torch.randn(T, D, generator=g).to(BF).cuda()
    w_qkv, w_o, w_gate, w1, w2 = weight((H + 2 * Hk) * d, D), weight(D, H * d), weight(E, D), weight(E, F, D), weight(E, D, F)
    off = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(n) for n in lengths]).to(torch.int32).cuda()
    side = torch.stack([torch.arange(256) // 16, torch.arange(256) % 16], 1)
    table = M.rope_table(side, (12, 12)).cuda()
    qw, kw = (1 + 0.1 * torch.randn(2, d, generator=g)).cuda()

    # Attention sub-layer: heads normalised and turned in place, v as the projection left it.
    qkv = (x @ w_qkv.T).view(T, H + 2 * Hk, d)
    before = f64(qkv)
    q, kk, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    M.qk_norm_rope(q, kk, table, q_weight=qw, k_weight=kw, pos=pos, q_out=q, k_out=kk)
    for part, w, got in ((before[:, :H], f64(qw), q), (before[:, H:H + Hk], f64(kw), kk)):
        y = part / np.sqrt((part ** 2).mean(-1, keepdims=True) + 1e-6) * w
        cs = f64(table)[pos.cpu().numpy()][:, None]
        a, b = y[..., :d // 2], y[..., d // 2:]
        want = np.concatenate([a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]], -1)
        mag = np.abs(a) + np.abs(b)
        near(got, want, (d / 2 + 8) * 2.0 ** -23 * np.concatenate([mag, mag], -1))
    assert (f64(v) == before[:, H + Hk:]).all()
    o = M.attention(q, kk, v, q_offsets=off, k_offsets=off, max_q=max(lengths))
    i = 0
    for n in lengths:
        q6, k6, v6 = f64(q[i:i + n]), np.repeat(f64(kk[i:i + n]), H // Hk, 1), np.repeat(f64(v[i:i + n]), H // Hk, 1)
        if n:
            s = np.einsum("ihd,jhd->hij", q6, k6) * d ** -0.5
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            mag = np.einsum("ihd,jhd->hij", np.abs(q6), np.abs(k6)).max(-1) * d ** -0.5
            e = ((d + 2) * 2.0 ** -23 * mag + 2.0 ** -23 * np.abs(s).max(-1) + 2.0 ** -22).T[..., None]
            near(o[i:i + n], np.einsum("hij,jhd->ihd", p, v6),
                 (2 * e + n * 2.0 ** -22 + 2.0 ** -20 + 2.0 ** -8) * np.einsum("hij,jhd->ihd", p, np.abs(v6)))
        i += n
    h = x + o.reshape(T, H * d) @ w_o.T

    # Expert sub-layer: the router's call gives ids and weights; one branch in ten is left to the cache.
    ema = torch.zeros(T, E, device="cuda")
    ids, gates, tau = (torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda"),
                       torch.empty(E, device="cuda"))
    M.moeca_route_noalloc(M.moeca_route_args(M.MOECA_BF16, T, D, E, k, 0, 0, 0.65, 0.8, 0.6, h.data_ptr(), w_gate.data_ptr(), None,
                                             ema.data_ptr(), ids.data_ptr(), gates.data_ptr(), tau.data_ptr()))
    torch.cuda.synchronize()
    ids[::10, 1] = -1
    plan = M.expert_sort(ids, E)
    rows = M.expert_rows(h, plan)
    at = plan.offsets.tolist()
    hidden = torch.zeros(T * k, F, dtype=BF, device="cuda")
    out = torch.zeros(T * k, D, dtype=BF, device="cuda")
    for e in range(E):
        hidden[at[e]:at[e + 1]] = torch.nn.functional.gelu(rows[at[e]:at[e + 1]] @ w1[e].T)
        out[at[e]:at[e + 1]] = hidden[at[e]:at[e + 1]] @ w2[e].T
    y = M.expert_combine(out, plan, gates, x=h)
    live = (ids >= 0).cpu().numpy()
    place = plan.place.cpu().numpy()
    assert at[-1] == live.sum() and ((place >= 0) == live).all()
    token, slot = plan.token[:at[-1]].cpu().numpy(), plan.slot[:at[-1]].cpu().numpy()
    assert (f64(rows)[:at[-1]] == f64(h)[token]).all() and (slot // k == token).all()
    assert (ids.flatten().cpu().numpy()[slot] == np.repeat(np.arange(E), np.diff(at))).all()
    terms = np.where(live[..., None], f64(out)[np.maximum(place, 0)], 0.0) * f64(gates)[..., None]
    near(y, f64(h) + terms.sum(1), (k + 1) * 2.0 ** -23 * (np.abs(terms).sum(1) + np.abs(f64(h))))

    # The same lists carry the 8-bit rows: quantised gather, grouped products, cache rows combined by slot.
    def rows8(t):
        return M.q8_write(t.reshape(-1, t.shape[-1]), M.q8_empty(t.shape[0] * t.shape[1], t.shape[2]))

    x8 = M.q8_write(h, M.q8_empty(T * k, D), src=plan.token)
    hid8 = M.q8_matmul(x8, rows8(w1), plan.offsets, act="gelu", dtype=torch.float8_e4m3fn)
    cache = M.q8_empty(T * k, D)
    M.q8_matmul(hid8, rows8(w2), plan.offsets, dst=plan.slot, out=cache)
    slots = torch.where(ids >= 0, torch.arange(T * k, device="cuda").view(T, k), -1).to(torch.int32)
    y8 = M.q8_combine(cache, slots, gates, x=h)
    # e4m3 in five places (two operands twice, the result): relative 2^-4 each at most, half of that on average.
    assert np.linalg.norm(f64(y8) - f64(y)) <= 5 * 2.0 ** -4 * np.linalg.norm(terms.sum(1))

    # The expert half's gradients for a given dy, through the products by hand.
    dy = torch.randn(T, D, generator=g).to(BF).cuda()
    dout, dgates = M.expert_combine_grad(dy, out, plan, gates)
    drows = torch.zeros_like(rows)
    for e in range(E):
        s = slice(at[e], at[e + 1])
        z = (rows[s] @ w1[e].T).detach().requires_grad_()
        torch.nn.functional.gelu(z).backward(dout[s] @ w2[e])
        drows[s] = z.grad @ w1[e]
    dh = M.expert_rows_grad(drows, plan)
    got = np.where(live[..., None], f64(out)[np.maximum(place, 0)], 0.0) * f64(dy)[:, None]
    assert (np.abs(f64(dgates) - got.sum(-1)) <= (D + 1) * 2.0 ** -23 * np.abs(got).sum(-1)).all()
    flat = f64(gates).reshape(-1)[slot][:, None] * f64(dy)[token]
    near(dout[:at[-1]], flat, 2.0 ** -24 * np.abs(flat))
    back = np.where(live[..., None], f64(drows)[np.maximum(place, 0)], 0.0)
    near(dh, back.sum(1), k * 2.0 ** -23 * np.abs(back).sum(1))


def test_decoding_one_token_at_a_time_matches_the_whole_prompt(M):
    """The last row of a causal prompt, and the same token alone against the same keys."""
    lengths, H, Hk, d = [300, 1, 77], 8, 2, 64
    T = sum(lengths)
    g = torch.Generator().manual_seed(5)
    q = torch.randn(T, H, d, generator=g).to(BF).cuda()
    k, v = (torch.randn(T, Hk, d, generator=g).to(BF).cuda() for _ in range(2))
    off = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")
    whole = M.attention(q, k, v, q_offsets=off, k_offsets=off, causal=True)
    last = (off[1:] - 1).long()
    alone = M.attention(q[last], k, v, k_offsets=off, causal=True)
    # Two roundings of p and of the result apart, each against sum p |v| <= max |v|.
    tol = 4 * HALF * float(v.abs().max())
    assert float((alone.float() - whole[last].float()).abs().max()) <= tol
