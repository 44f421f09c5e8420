"""Operators of a whole transformer layer on packed tokens, as measurable cases.

Three operators, each as a user's program calls it, forward alone (inference) or forward and backward (training):

  qk_rotary        the norm of every head of q and k with the rotation by the token's place (time, row, column) in one pass, on the
                   packed rows that the projection wrote; backward: with the gradients of the norms' parameters
  cross_attention  the packed tokens of an image (or a few queries, or one) attend to another sequence of that image's, of another
                   length: packed or padded, key heads shared by several query heads, no key at all for some images
  feed_forward     the gated feed-forward block on packed rows: both projections, the activation and their product, then
                   the projection back onto the residual stream at token positions; backward: with the gradients of all weights,
                   in the weights' type

Shapes are those of the framework's workloads (ViT-S / ViT-B at 14 x 14 tokens, detection at 50 x 84, the two-image fp32 batch)
and odd ones beside them.  A program keeps its launches, buffers and tables (`prepare`); the inputs of a pass are read from the
buffers anew each time.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

EPS = 1e-6
BASE = 100.0          # of the rotation's frequencies: angles of a map's places


def _rotary(name, train, B, grid, pairs, H, Hk, Dh, lo, hi, dtype="bf16", norm="rms", layout="adjacent"):
    return dict(name=name, op="qk_rotary", train=train, B=B, t=grid[0], h=grid[1], w=grid[2], pairs_t=pairs[0], pairs_h=pairs[1], H=H, Hk=Hk,
                Dh=Dh, lo=lo, hi=hi, dtype=dtype, norm=norm, layout=layout)


def _cross(name, train, B, nq, qlo, qhi, L, klo, khi, H, Hk, Dh, padded, dtype="bf16"):
    return dict(name=name, op="cross_attention", train=train, B=B, nq=nq, qlo=qlo, qhi=qhi, L=L, klo=klo, khi=khi, H=H, Hk=Hk, Dh=Dh,
                padded=padded, dtype=dtype)


def _ffn(name, train, B, N, C, F, lo, hi, act="silu", bias=True, dtype="bf16"):
    return dict(name=name, op="feed_forward", train=train, B=B, N=N, C=C, F=F, lo=lo, hi=hi, act=act, bias=bias, dtype=dtype)


def listed():
    return [
        # one classification image at a time, as an online service does: bound by latency
        _rotary("rotary_one_image", False, 1, (1, 14, 14), (0, 16), 6, 6, 64, 0.10, 0.90),
        # a ragged batch in fp32, norms with mean and shift, pairs half a head apart
        _rotary("rotary_ragged_f32_train", True, 5, (1, 33, 47), (0, 8), 4, 4, 32, 0.10, 0.60, dtype="f32", norm="layer", layout="halves"),
        # a ViT-B-shaped training step
        _rotary("rotary_vit_b_train", True, 64, (1, 14, 14), (0, 16), 12, 12, 64, 0.05, 0.95),
        # video clips, three axes, four query heads to a key head: the largest of the rotations
        _rotary("rotary_video_train", True, 8, (8, 28, 28), (8, 12), 16, 4, 64, 0.30, 0.70),
        # the tokens of one image attend to the states of a caption
        _cross("cross_caption_one_image", False, 1, 196, 0.5, 0.5, 77, 0.5, 0.5, 6, 6, 64, True),
        # one new token reads a long sequence of another encoder, shared key heads: split over its length
        _cross("cross_one_token_long", False, 4, 1, 1.0, 1.0, 16000, 0.7, 1.0, 16, 4, 64, True),
        # small ragged fp32 training batch, some images without a key
        _cross("cross_ragged_f32_train", True, 7, 150, 0.0, 1.0, 90, 0.0, 1.0, 4, 2, 32, False, dtype="f32"),
        # ViT-B-shaped training step against padded captions
        _cross("cross_captions_vit_b_train", True, 64, 196, 0.05, 0.95, 77, 0.1, 1.0, 12, 12, 64, True),
        # tokens of larger images against the states of a second encoder of other length: the largest of the attentions
        _cross("cross_states_train", True, 8, 3136, 0.5, 1.0, 1024, 0.4, 1.0, 12, 4, 64, False),
        # one classification image
        _ffn("ffn_one_image", False, 1, 196, 384, 1024, 0.10, 0.90),
        # the two-image fp32 batch
        _ffn("ffn_tiny_f32_train", True, 2, 196, 64, 176, 0.20, 0.40, act="gelu", dtype="f32"),
        # ViT-B-shaped training step: the most multiplications of all
        _ffn("ffn_vit_b_train", True, 64, 196, 768, 2048, 0.05, 0.95),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    while True:
        op, train, dtype = rng.choice(["qk_rotary", "cross_attention", "feed_forward"]), rng.random() < 0.5, "f32" if rng.random() < 0.2 else "bf16"
        B, Dh = _log_int(rng, 1, 96), rng.choice([32, 64])
        lo = round(rng.uniform(0.0, 0.4), 2)
        hi = round(rng.uniform(lo + 0.05, 0.95), 2)
        Hk = _log_int(rng, 1, 12)
        H = Hk * rng.choice([1, 1, 1, 2, 3, 4, 8])
        if H > 24:
            continue
        if op == "qk_rotary":
            axes, n = rng.choice([1, 2, 2, 3]), Dh // 2
            grid = {1: (1, 1, _log_int(rng, 1, 6000)), 2: (1, _log_int(rng, 2, 64), _log_int(rng, 2, 96)),
                    3: (rng.randint(2, 16), rng.randint(2, 32), rng.randint(2, 32))}[axes]
            pairs = {1: (0, 0), 2: (0, n // 2), 3: (n // 4, n // 4 + n // 8)}[axes]
            c = _rotary("", train, B, grid, pairs, H, Hk, Dh, lo, hi, dtype, rng.choice(["rms", "rms", "layer", "none"]),
                        rng.choice(["adjacent", "halves"]))
            tokens = B * grid[0] * grid[1] * grid[2]
            fits = tokens <= 140_000 and tokens * lo >= 4 * B
        elif op == "cross_attention":
            few = rng.random() < 0.35
            nq = _log_int(rng, 1, 32) if few else _log_int(rng, 1, 4200)
            L = _log_int(rng, 1, 20000) if few else _log_int(rng, 1, 4200)
            klo = round(rng.uniform(0.0, 0.9), 2)
            khi = round(rng.uniform(klo + 0.05, 1.0), 2)
            qlo, qhi = (1.0, 1.0) if few else (lo, hi)
            if train and (nq < 8 or L * khi < 16):
                continue
            c = _cross("", train, B, nq, qlo, qhi, L, klo, khi, H, Hk, Dh, rng.random() < 0.5, dtype)
            fits = B * max(nq, L) <= 140_000 and B * H * nq * L <= 3.2e8 and nq * qlo >= 1 and L * klo >= 1
        else:
            C, F = 8 * _log_int(rng, 4, 128), 8 * _log_int(rng, 6, 360)
            c = _ffn("", train, B, _log_int(rng, 1, 4200), C, F, lo, hi, rng.choice(["silu", "gelu"]), rng.random() < 0.5, dtype)
            fits = B * c["N"] <= 140_000 and c["N"] * lo >= 4 and (dtype == "bf16" or B * c["N"] * C * F <= 3e9)
        del c["name"]
        if fits and _cost(c) <= most[op]:
            return c


# ---------------------------------------------------------------------------------- inputs
def _lens(g, B, n, lo, hi):
    frac = lo + (hi - lo) * torch.rand(B, generator=g, device="cuda")
    return (frac * n).round().long().clamp(0, n)


def _chosen(g, lens, N):
    """Which tokens of every image are selected: lens[b] of them, next to a random place on the image's line of tokens with
    some further off."""
    B = lens.numel()
    at = torch.rand(B, 1, generator=g, device="cuda") * N
    far = (torch.arange(N, device="cuda") - at).abs() * (0.5 + torch.rand(B, N, generator=g, device="cuda"))
    return far.argsort(1).argsort(1) < lens[:, None]


def _sums(lens):
    cu = torch.zeros(lens.numel() + 1, dtype=torch.int32, device="cuda")
    cu[1:] = lens.cumsum(0)
    return cu


def _selection(s, g, B, N, lo, hi):
    lens = _lens(g, B, N, lo, hi)
    mask = _chosen(g, lens, N)
    chosen = mask.view(-1).nonzero().view(-1)
    T = chosen.numel()
    gather_idx = torch.zeros(B * N, dtype=torch.int32, device="cuda")
    inv_pos = torch.full((B * N,), -1, dtype=torch.int32, device="cuda")
    gather_idx[:T] = chosen.int()
    inv_pos[chosen] = torch.arange(T, dtype=torch.int32, device="cuda")
    s.update(N=N, cap=B * N, T=T, gather_idx=gather_idx, inv_pos=inv_pos, total=torch.tensor([T], dtype=torch.int32, device="cuda"))


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    td = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    rnd = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    s = dict(c, td=td)
    if c["op"] == "qk_rotary":
        B, H, Hk, Dh = c["B"], c["H"], c["Hk"], c["Dh"]
        _selection(s, g, B, c["t"] * c["h"] * c["w"], c["lo"], c["hi"])
        param = lambda one, width: (one + 0.2 * rnd(width)).to(td)
        s.update(qkv=(rnd(s["cap"], (H + 2 * Hk) * Dh) * 1.5 + 0.2).to(td), gamma_q=None, gamma_k=None, beta_q=None, beta_k=None)
        if c["norm"] != "none":
            s.update(gamma_q=param(1.0, Dh), gamma_k=param(1.0, Dh))
        if c["norm"] == "layer":
            s.update(beta_q=param(0.0, Dh), beta_k=param(0.0, Dh))
        if c["train"]:
            s.update(dq_rot=rnd(s["cap"], H * Dh).to(td), dk_rot=rnd(s["cap"], Hk * Dh).to(td))
    elif c["op"] == "cross_attention":
        B, H, Hk, Dh, nq, L = c["B"], c["H"], c["Hk"], c["Dh"], c["nq"], c["L"]
        lens_q, lens_k = _lens(g, B, nq, c["qlo"], c["qhi"]), _lens(g, B, L, c["klo"], c["khi"])
        s.update(cap_q=B * nq, cap_k=B * L, lens_q=lens_q, lens_k=lens_k, cu_q=_sums(lens_q),
                 cu_k=_sums(torch.full_like(lens_k, L) if c["padded"] else lens_k), key_lens=lens_k.int() if c["padded"] else None,
                 q=rnd(B * nq, H * Dh).to(td), kv=rnd(B * L, 2 * Hk * Dh).to(td))
        if c["train"]:
            s.update(dout=rnd(B * nq, H * Dh).to(td))
    else:
        B, N, C, F = c["B"], c["N"], c["C"], c["F"]
        _selection(s, g, B, N, c["lo"], c["hi"])
        s.update(x=rnd(s["cap"], C).to(td), res=rnd(B, N, C).to(td), W=(rnd(2 * F, C) / C ** 0.5).to(td), W_down=(rnd(C, F) / F ** 0.5).to(td),
                 b=(0.3 * rnd(2 * F)).to(td) if c["bias"] else None, b_down=(0.3 * rnd(C)).to(td) if c["bias"] else None)
        if c["train"]:
            s.update(dy=rnd(B, N, C).to(td))
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """What a program keeps: result buffers, tables, workspaces, and the launches of the pass bound to them."""
    from paper_2410_23608_amd import spa
    td = s["td"]
    code = spa.SPA_BF16 if td == torch.bfloat16 else spa.SPA_F32
    zeros = lambda *shape, dtype=td: torch.zeros(*shape, dtype=dtype, device="cuda")
    f32 = dict(dtype=torch.float32)
    ws = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    if s["op"] == "qk_rotary":
        H, Hk, Dh, cap, C = s["H"], s["Hk"], s["Dh"], s["cap"], s["H"] * s["Dh"]
        grid, pairs = (s["t"], s["h"], s["w"]), (s["pairs_t"], s["pairs_h"])
        kind = {"rms": spa.SPA_NORM_RMS, "layer": spa.SPA_NORM_LAYER, "none": spa.SPA_NORM_NONE}[s["norm"]]
        layout = spa.SPA_ROTARY_HALVES if s["layout"] == "halves" else spa.SPA_ROTARY_ADJACENT
        table = spa.rotary_table(grid, Dh, pairs, BASE).cuda()
        q, k = s["qkv"][:, :C], s["qkv"][:, C:C + Hk * Dh]
        q_rot, k_rot = zeros(cap, C), zeros(cap, Hk * Dh)
        s["outputs"] = dict(q=q_rot, k=k_rot)
        s["launches"] = [spa.spa_qk_norm_rotary(q, k, s["gather_idx"], s["total"], s["gamma_q"], s["beta_q"], s["gamma_k"], s["beta_k"], kind,
                                                EPS, table, pairs, grid, H, Hk, Dh, q_rot, k_rot, layout, prepare=True)]
        if s["train"]:
            dqkv = zeros(cap, (H + 2 * Hk) * Dh)
            grads = {name: None if s[name] is None else zeros(Dh, **f32) for name in ("gamma_q", "beta_q", "gamma_k", "beta_k")}
            s["outputs"].update(dqkv=dqkv, **{"d" + name: t for name, t in grads.items()})
            s["launches"].append(spa.spa_qk_norm_rotary_bwd(
                s["dq_rot"], s["dk_rot"], q, k, s["gather_idx"], s["total"], s["gamma_q"], s["gamma_k"], kind, EPS, table, pairs, grid, H,
                Hk, Dh, dqkv[:, :C], dqkv[:, C:C + Hk * Dh], grads["gamma_q"], grads["beta_q"], grads["gamma_k"], grads["beta_k"],
                ws(spa.spa_qk_norm_rotary_bwd_workspace_bytes(cap, H, Hk, Dh, code)), layout, prepare=True))
    elif s["op"] == "cross_attention":
        B, H, Hk, Dh, nq, L, Ck = s["B"], s["H"], s["Hk"], s["Dh"], s["nq"], s["L"], s["Hk"] * s["Dh"]
        k, v = s["kv"][:, :Ck], s["kv"][:, Ck:]
        out = zeros(s["cap_q"], H * Dh)
        lse = zeros(H, s["cap_q"], **f32) if s["train"] else None
        s["outputs"] = dict(out=out)
        s["launches"] = [spa.spa_cross_attention(s["q"], k, v, s["cu_q"], s["cu_k"], s["key_lens"], B, nq, L, H, Hk, Dh, out, lse,
                                                 ws(spa.spa_cross_attention_workspace_bytes(B, nq, L, H, Hk, Dh, code)), prepare=True)]
        if s["train"]:
            dq, dkv = zeros(s["cap_q"], H * Dh), zeros(s["cap_k"], 2 * Ck)
            s["outputs"].update(dq=dq, dkv=dkv)
            s["launches"].append(spa.spa_cross_attention_bwd(
                s["q"], k, v, out, s["dout"], lse, s["cu_q"], s["cu_k"], s["key_lens"], B, nq, L, H, Hk, Dh, dq, dkv[:, :Ck], dkv[:, Ck:],
                ws(spa.spa_cross_attention_bwd_workspace_bytes(B, nq, L, H, Hk, Dh, code)), prepare=True))
    else:
        B, N, C, F, cap = s["B"], s["N"], s["C"], s["F"], s["cap"]
        act = spa.SPA_ACT_SILU if s["act"] == "silu" else spa.SPA_ACT_GELU
        h, y = zeros(cap, F), zeros(B, N, C)
        pre = zeros(cap, 2 * F) if s["train"] else None
        s["outputs"] = dict(y=y)
        s["launches"] = [spa.spa_gated_linear_packed(s["x"], None, s["total"], s["W"], s["b"], act, h, pre, prepare=True),
                         spa.spa_linear_packed_unpack(h, s["total"], s["W_down"], s["b_down"], s["gather_idx"], s["inv_pos"], s["res"], y,
                                                      prepare=True)]
        if s["train"]:
            d_pre, dx, dy = zeros(cap, 2 * F), zeros(cap, C), s["dy"].view(cap, C)
            dW, dW_down = zeros(2 * F, C, **f32), zeros(C, F, **f32)
            db, db_down = (zeros(2 * F, **f32), zeros(C, **f32)) if s["bias"] else (None, None)
            grads = _given(dict(dW=dW, dW_down=dW_down, db=db, db_down=db_down))
            # the optimizer takes the gradients in the weights' type
            handed = {name: t if td == t.dtype else zeros(*t.shape) for name, t in grads.items()}
            s["outputs"].update(dx=dx, **handed)
            s["launches"] += [
                spa.spa_gated_linear_packed_bwd(dy, s["gather_idx"], s["total"], s["W_down"], pre, act, d_pre, prepare=True),
                spa.spa_linear_packed_bwd_weight(dy, s["gather_idx"], h, None, None, s["total"], cap, dW_down, db_down,
                                                 ws(spa.spa_linear_bwd_weight_workspace_bytes(cap, F, C, td)), prepare=True),
                spa.spa_linear_packed_bwd_input(d_pre, None, s["total"], s["W"], cap, None, None, dx, prepare=True),
                spa.spa_linear_packed_bwd_weight(d_pre, None, s["x"], None, None, s["total"], cap, dW, db,
                                                 ws(spa.spa_linear_bwd_weight_workspace_bytes(cap, C, 2 * F, td)), prepare=True)]
            s["launches"] += [functools.partial(handed[name].copy_, t) for name, t in grads.items() if handed[name] is not t]
    s["outputs"] = _given(s["outputs"])


# ---------------------------------------------------------------------------------- the pass
def run(state):
    if own:
        for launch in state["launches"]:
            launch()
        return state["outputs"]
    return _given({"qk_rotary": _qk_rotary, "cross_attention": _cross_attention, "feed_forward": _feed_forward}[state["op"]](state))


def _given(outputs):
    """Without the results that the case at hand does not have (no shift, no gradient of one)."""
    return {name: t for name, t in outputs.items() if t is not None}


def _angles(s):
    """Cosine and sine of every pair's angle of the packed rows, [T, 1, Dh / 2], in 64 bits."""
    n = s["gather_idx"][:s["T"]].long() % s["N"]
    place = (n // (s["h"] * s["w"]), n // s["w"] % s["h"], n % s["w"])
    counts = (s["pairs_t"], s["pairs_h"], s["Dh"] // 2 - s["pairs_t"] - s["pairs_h"])
    parts = []
    for p, count in zip(place, counts):
        if count > 0:
            freq = BASE ** (-torch.arange(count, dtype=torch.float64, device="cuda") / count)
            parts.append(p[:, None].double() * freq)
    angle = torch.cat(parts, 1)[:, None]
    return torch.cos(angle), torch.sin(angle)


def _pairs_of(x, layout):
    half = x.shape[-1] // 2
    return (x[..., :half], x[..., half:]) if layout == "halves" else (x[..., 0::2], x[..., 1::2])


def _joined(a, b, layout):
    return torch.cat((a, b), -1) if layout == "halves" else torch.stack((a, b), -1).flatten(-2)


def _turned(x, cos, sin, layout):
    a, b = _pairs_of(x, layout)
    return _joined(a * cos - b * sin, a * sin + b * cos, layout)


def _qk_rotary(s):
    T, cap, H, Hk, Dh, td = s["T"], s["cap"], s["H"], s["Hk"], s["Dh"], s["td"]
    cos, sin = (t.float() for t in _angles(s))
    res, dqkv = {}, torch.zeros(cap, (H + 2 * Hk) * Dh, dtype=td, device="cuda") if s["train"] else None
    for name, first, heads in (("q", 0, H), ("k", H * Dh, Hk)):
        x = s["qkv"][:T, first:first + heads * Dh].float().view(T, heads, Dh)
        gamma, beta = s["gamma_" + name], s["beta_" + name]
        xh, r = x, None
        if s["norm"] != "none":
            if s["norm"] == "layer":
                xh = x - x.mean(-1, keepdim=True)
            r = torch.rsqrt((xh * xh).mean(-1, keepdim=True) + EPS)
            xh = xh * r
        u = xh if gamma is None else xh * gamma.float()
        if beta is not None:
            u = u + beta.float()
        out = torch.zeros(cap, heads * Dh, dtype=td, device="cuda")
        out[:T] = _turned(u, cos, sin, s["layout"]).reshape(T, -1).to(td)
        res[name] = out
        if s["train"]:
            du = _turned(s[f"d{name}_rot"][:T].float().view(T, heads, Dh), cos, -sin, s["layout"])
            dx = du
            if s["norm"] != "none":
                sums = lambda v: v.sum((0, 1), dtype=torch.float64).float()
                res["dgamma_" + name], res["dbeta_" + name] = sums(du * xh), sums(du) if beta is not None else None
                dx = du * gamma.float()
                if s["norm"] == "layer":
                    dx = dx - dx.mean(-1, keepdim=True)
                dx = (dx - xh * (dx * xh).mean(-1, keepdim=True)) * r
            dqkv[:T, first:first + heads * Dh] = dx.reshape(T, -1).to(td)
    res["dqkv"] = dqkv
    return res


def _cross_attention(s):
    B, H, Hk, Dh, td, Ck = s["B"], s["H"], s["Hk"], s["Dh"], s["td"], s["Hk"] * s["Dh"]
    n, m, scale = max(int(s["lens_q"].max()), 1), max(int(s["lens_k"].max()), 1), Dh ** -0.5
    place = lambda cu, lens, most: (torch.arange(most, device="cuda") < lens[:, None], cu.long()[:-1, None] + torch.arange(most, device="cuda"))
    okq, rows_q = place(s["cu_q"], s["lens_q"], n)
    okk, rows_k = place(s["cu_k"], s["lens_k"], m)
    rows_q, rows_k = torch.where(okq, rows_q, 0), torch.where(okk, rows_k, 0)
    # [B, Hk, n (H / Hk), Dh] and [B, Hk, m, Dh]: the query heads of a key head are rows of one product
    wide = lambda t: torch.where(okq[..., None], t[rows_q].float(), 0.0).view(B, n, Hk, H // Hk, Dh).permute(0, 2, 1, 3, 4).reshape(B, Hk, -1, Dh).contiguous()
    keys = lambda t: torch.where(okk[..., None], t[rows_k].float(), 0.0).view(B, m, Hk, Dh).transpose(1, 2).contiguous()
    back = lambda t: t.view(B, Hk, n, H // Hk, Dh).permute(0, 2, 1, 3, 4).reshape(B, n, H * Dh)[okq]
    q, k, v = wide(s["q"]), keys(s["kv"][:, :Ck]), keys(s["kv"][:, Ck:])
    S = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    S = torch.where(okk[:, None, None, :], S, float("-inf"))
    top = S.amax(3, keepdim=True)
    P = torch.exp(S - torch.where(top > float("-inf"), top, 0.0))
    total = P.sum(3, keepdim=True)
    P = P / torch.where(total > 0, total, 1.0)
    del S
    O = torch.matmul(P, v)
    out = torch.zeros(s["cap_q"], H * Dh, dtype=td, device="cuda")
    Tq = int(s["lens_q"].sum())
    out[:Tq] = back(O).to(td)
    res = dict(out=out)
    if s["train"]:
        dO = wide(s["dout"])
        dS = P * (torch.matmul(dO, v.transpose(2, 3).contiguous()) - (dO * O).sum(3, keepdim=True))
        dq, dkv = torch.zeros_like(out), torch.zeros(s["cap_k"], 2 * Ck, dtype=td, device="cuda")
        dq[:Tq] = back(torch.matmul(dS, k) * scale).to(td)
        dk = torch.matmul(dS.transpose(2, 3).contiguous(), q) * scale
        del dS
        dv = torch.matmul(P.transpose(2, 3).contiguous(), dO)
        at = rows_k[okk]
        for i, t in enumerate((dk, dv)):
            dkv[at, i * Ck:(i + 1) * Ck] = t.transpose(1, 2).reshape(B, m, Ck)[okk].to(td)
        res.update(dq=dq, dkv=dkv)
    return res


def _act(g, act):
    """The activation and its slope."""
    if act == "silu":
        sig = 1 / (1 + torch.exp(-g))
        return g * sig, sig * (1 + g * (1 - sig))
    cdf = 0.5 * (1 + torch.erf(g * 2 ** -0.5))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5


def _feed_forward(s):
    T, F, td, cap = s["T"], s["F"], s["td"], s["cap"]
    sel = s["gather_idx"][:T].long()
    x, W, W_down = s["x"][:T].float(), s["W"].float(), s["W_down"].float()
    pre = torch.matmul(x, W.T.contiguous())
    if s["bias"]:
        pre = pre + s["b"].float()
    a, slope = _act(pre[:, :F], s["act"])
    up = pre[:, F:]
    h = a * up
    z = torch.matmul(h, W_down.T.contiguous())
    if s["bias"]:
        z = z + s["b_down"].float()
    y = s["res"].float().view(cap, -1).clone()
    y[sel] += z
    res = dict(y=y.to(td).view_as(s["res"]))
    if s["train"]:
        dy = s["dy"].view(cap, -1)[sel].float()
        dh = torch.matmul(dy, W_down)
        d_pre = torch.cat((dh * up * slope, dh * a), 1)
        dx = torch.zeros_like(s["x"])
        dx[:T] = torch.matmul(d_pre, W).to(td)
        sums = lambda v: v.sum(0, dtype=torch.float64).to(td) if s["bias"] else None
        res.update(dx=dx, dW=torch.matmul(d_pre.T.contiguous(), x).to(td), dW_down=torch.matmul(dy.T.contiguous(), h).to(td), db=sums(d_pre),
                   db_down=sums(dy))
    return res


# ------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """The results in 64 bits, from the definitions."""
    s = prepare(case, seed)
    f = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    zeros = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")
    return _given({"qk_rotary": _exact_rotary, "cross_attention": _exact_cross, "feed_forward": _exact_ffn}[s["op"]](s, f, zeros))


def _exact_rotary(s, f, zeros):
    """Every pair of a head as a complex number that its angle turns."""
    T, cap, H, Hk, Dh, half = s["T"], s["cap"], s["H"], s["Hk"], s["Dh"], s["Dh"] // 2
    n = (s["gather_idx"][:T].long() % s["N"]).cpu().numpy()
    row, counts = n % (s["h"] * s["w"]), [s["pairs_t"], s["pairs_h"]]
    where, counts = [n // (s["h"] * s["w"]), row // s["w"], row % s["w"]], counts + [half - sum(counts)]
    angle = np.concatenate([np.outer(p, np.power(BASE, -np.arange(c) / max(c, 1))) for p, c in zip(where, counts)], 1)
    turn = torch.from_numpy(np.exp(1j * angle)).cuda()[:, None, :]
    split = (lambda x: torch.complex(x[..., :half], x[..., half:])) if s["layout"] == "halves" else (lambda x: torch.view_as_complex(x.unflatten(-1, (half, 2)).contiguous()))
    join = (lambda z: torch.cat((z.real, z.imag), -1)) if s["layout"] == "halves" else (lambda z: torch.view_as_real(z).flatten(-2))
    res = dict(dqkv=zeros(cap, (H + 2 * Hk) * Dh) if s["train"] else None)
    for name, first, heads in (("q", 0, H), ("k", H * Dh, Hk)):
        x = f["qkv"][:T, first:first + heads * Dh].reshape(T, heads, Dh)
        gamma, beta = f["gamma_" + name], f["beta_" + name]
        mu = x.mean(-1, keepdim=True) if s["norm"] == "layer" else torch.zeros_like(x[..., :1])
        sd = torch.sqrt(((x - mu) ** 2).mean(-1, keepdim=True) + EPS) if s["norm"] != "none" else torch.ones_like(x[..., :1])
        hat = (x - mu) / sd
        u = hat * (gamma if gamma is not None else 1.0) + (beta if beta is not None else 0.0)
        res[name] = zeros(cap, heads * Dh)
        res[name][:T] = join(split(u) * turn).reshape(T, -1)
        if s["train"]:
            du = join(split(f[f"d{name}_rot"][:T].reshape(T, heads, Dh)) * turn.conj())
            dx = du
            if s["norm"] != "none":
                res["dgamma_" + name] = (du * hat).sum((0, 1))
                res["dbeta_" + name] = du.sum((0, 1)) if beta is not None else None
                g = du * gamma
                dx = g - hat * (g * hat).mean(-1, keepdim=True)
                dx = (dx - g.mean(-1, keepdim=True) if s["norm"] == "layer" else dx) / sd
            res["dqkv"][:T, first:first + heads * Dh] = dx.reshape(T, -1)
    return res


def _exact_cross(s, f, zeros):
    """Image by image and head by head."""
    H, Hk, Dh, Ck = s["H"], s["Hk"], s["Dh"], s["Hk"] * s["Dh"]
    if s["B"] * H > 4096:
        return dict(out=None, dq=None, dkv=None) if s["train"] else dict(out=None)
    out = zeros(s["cap_q"], H * Dh)
    dq, dkv = (zeros(s["cap_q"], H * Dh), zeros(s["cap_k"], 2 * Ck)) if s["train"] else (None, None)
    cu_q, cu_k, lens = s["cu_q"].tolist(), s["cu_k"].tolist(), s["lens_k"].tolist()
    for b in range(s["B"]):
        i, j = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b] + lens[b])
        if cu_q[b] == cu_q[b + 1] or lens[b] == 0:
            continue
        for h in range(H):
            col, kc = slice(h * Dh, (h + 1) * Dh), h // (H // Hk) * Dh
            q, k, v = f["q"][i, col], f["kv"][j, kc:kc + Dh], f["kv"][j, Ck + kc:Ck + kc + Dh]
            P = torch.softmax(q @ k.T / math.sqrt(Dh), 1)
            out[i, col] = P @ v
            if s["train"]:
                dO = f["dout"][i, col]
                dP = dO @ v.T
                dS = P * (dP - (P * dP).sum(1, keepdim=True)) / math.sqrt(Dh)
                dq[i, col] = dS @ k
                dkv[j, kc:kc + Dh] += dS.T @ q
                dkv[j, Ck + kc:Ck + kc + Dh] += P.T @ dO
    return dict(out=out, dq=dq, dkv=dkv)


def _exact_ffn(s, f, zeros):
    T, F, cap, C = s["T"], s["F"], s["cap"], s["C"]
    sel, x = s["gather_idx"][:T].long(), f["x"][:T]
    g, u = x @ f["W"][:F].T, x @ f["W"][F:].T
    if s["bias"]:
        g, u = g + f["b"][:F], u + f["b"][F:]
    if s["act"] == "silu":
        p = torch.sigmoid(g)
        a, slope = g * p, p + g * p * (1 - p)
    else:
        p = torch.special.ndtr(g)
        a, slope = g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    y = f["res"].reshape(cap, C).clone()
    y[sel] = y[sel] + (a * u) @ f["W_down"].T + (f["b_down"] if s["bias"] else 0.0)
    res = dict(y=y.view_as(s["res"]))
    if s["train"]:
        dy = f["dy"].reshape(cap, C)[sel]
        dh = dy @ f["W_down"]
        dg, du = dh * u * slope, dh * a
        dx = zeros(cap, C)
        dx[:T] = dg @ f["W"][:F] + du @ f["W"][F:]
        res.update(dx=dx, dW=torch.cat((dg.T @ x, du.T @ x)), dW_down=dy.T @ (a * u), db=torch.cat((dg.sum(0), du.sum(0))) if s["bias"] else None,
                   db_down=dy.sum(0) if s["bias"] else None)
    return res


# ----------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    if c["op"] == "qk_rotary":
        T, width = c["B"] * c["t"] * c["h"] * c["w"] * (c["lo"] + c["hi"]) / 2, (c["H"] + c["Hk"]) * c["Dh"]
        rows, table = T * width * e, max(c["t"], c["h"], c["w"]) * c["Dh"] * 4
        nbytes, flops = 2 * rows + 4 * T + table, 12.0 * T * width
        if c["train"]:
            nbytes, flops = nbytes + 2 * rows, flops + 24.0 * T * width          # the gradient in and out
    elif c["op"] == "cross_attention":
        nq, nk = c["nq"] * (c["qlo"] + c["qhi"]) / 2, c["L"] * (c["klo"] + c["khi"]) / 2
        q, k = c["B"] * nq * c["H"] * c["Dh"] * e, c["B"] * nk * c["Hk"] * c["Dh"] * e
        nbytes, flops = 2 * q + 2 * k, 4.0 * c["B"] * nq * nk * c["H"] * c["Dh"]
        if c["train"]:
            nbytes, flops = nbytes + 2 * q + 2 * k, 3.5 * flops                  # dout in; dq, dk, dv out
    else:
        cap = c["B"] * c["N"]
        T, C, F = cap * (c["lo"] + c["hi"]) / 2, c["C"], c["F"]
        nbytes, flops = T * C * e + 2 * cap * C * e + 3 * F * C * e, 6.0 * T * C * F
        if c["train"]:
            nbytes, flops = nbytes + 2 * T * C * e + 3 * F * C * e, 3 * flops    # dy in; dx and the weights' gradients out
    return {"bytes": float(nbytes), "flops": float(flops)}


def _cost(c):
    """Rough seconds of a pass, to keep drawn cases within the largest listed one of their operator."""
    w = work(c)
    return w["bytes"] / 3e12 + w["flops"] / (20e12 if c["dtype"] == "f32" else 200e12)
