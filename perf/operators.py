"""The operators around the attention, as a program that uses this package
calls them, with their plain forms.

* ``rope``: the rows of a fused q, k, v projection become what the attention
  takes: RMS norm of every query and key row with learned weights, rotation by
  position (one axis, or time, height and width), key and value heads repeated
  for the query heads that share them, tokens inside heads.  Forward, and the
  backward with the gradients of the weights.
* ``append``: the same norm and rotation for new tokens while serving, then
  the attention's standardisation; keys and values go to their slots of a
  paged cache, standardised queries come back.
* ``paged``: Fastmax attention of new tokens over the paged cache: one token
  per sequence, or a chunk of a prompt, over all that went before or over a
  window and a few first tokens.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def _rope(call, B, N, Hq, Hkv, D, dtype, axes=1, rot=None, interleaved=False, norm=True):
    return {"call": call, "B": B, "N": N, "Hq": Hq, "Hkv": Hkv, "D": D, "dtype": dtype,
            "axes": axes, "rot": rot or D, "interleaved": interleaved, "norm": norm}


def _append(T, Hq, Hkv, D, page, pages, dtype, norm=True, interleaved=False, rot=None):
    return {"call": "append", "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page,
            "pages": pages, "dtype": dtype, "norm": norm, "interleaved": interleaved,
            "axes": 1, "rot": rot or D}


def _paged(S, longest, new, Hq, Hkv, D, page, dtype, p=2, unit=False, window=0, sinks=0,
           ragged=True, lens_seed=1):
    return {"call": "paged", "S": S, "longest": longest, "new": new, "Hq": Hq, "Hkv": Hkv,
            "D": D, "page": page, "dtype": dtype, "p": p, "unit": unit, "window": window,
            "sinks": sinks, "ragged": ragged, "lens_seed": lens_seed}


def listed():
    cases = {
        # Long Range Arena training (head size 32, about 2000 tokens, float32):
        # rotation without a norm, before a short layer, where latency counts
        "rope_fwd_lra_f32": _rope("rope_fwd", 2, 2048, 4, 4, 32, "f32", norm=False),
        # a GPT-style layer's rows, forward and backward
        "rope_fwd_gpt_bf16": _rope("rope_fwd", 4, 8192, 16, 16, 64, "bf16"),
        "rope_bwd_gpt_bf16": _rope("rope_bwd", 4, 8192, 16, 16, 64, "bf16"),
        # backward over image and video tokens (three axes of positions) at the
        # Llama-2 head size, four query heads to a key head, odd length
        "rope_bwd_axes_bf16": _rope("rope_bwd", 1, 4095, 32, 8, 128, "bf16", axes=3),
        # one user's next token in a 12-head layer
        "append_one_bf16": _append(1, 12, 12, 64, 64, 64, "bf16"),
        # the next tokens of a batch of odd size, shared heads
        "append_batch_bf16": _append(97, 32, 8, 128, 64, 512, "bf16"),
        # the tokens of several prompts at once
        "append_prompts_bf16": _append(16384, 32, 8, 128, 64, 320, "bf16"),
        # one user's next token after a prompt of odd length, first order with
        # unit-norm scores
        "paged_one_p1_bf16": _paged(1, 777, 1, 12, 12, 64, 64, "bf16", p=1, unit=True),
        # the next tokens of a batch, contexts of many lengths, shared heads
        "paged_batch_bf16": _paged(61, 8192, 1, 32, 8, 128, 64, "bf16"),
        # one very long context (the library's long sequence)
        "paged_long_bf16": _paged(1, 131072, 1, 32, 8, 128, 64, "bf16"),
        # a stream's window and first tokens, float32, small pages
        "paged_window_f32": _paged(32, 65536, 1, 8, 8, 64, 16, "f32", window=4096, sinks=4),
        # chunks of prompts over what is in the cache already
        "paged_chunk_bf16": _paged(4, 8192, 2048, 32, 8, 128, 64, "bf16"),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log_int(rng, lo, hi):
    hi = max(lo, int(hi))
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges; every bound keeps it below the
    largest listed case of its call."""
    family = rng.choice(["rope_fwd", "rope_bwd", "append", "append", "decode", "decode",
                         "window", "chunk"])
    D = rng.choice([16, 32, 64, 64, 128, 128])
    Hkv = rng.choice([1, 2, 3, 4, 8, 12, 16] if D < 128 else [1, 2, 4, 5, 8])
    Hq = Hkv * rng.choice([1, 1, 2, 4, 7, 8] if Hkv <= 4 else [1, 2, 4])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if family in ("rope_fwd", "rope_bwd"):
        most = (1 << 25) // (Hq * D) // (2 if dtype == "f32" else 1)
        B = rng.choice([1, 2, 4, 8])
        return _rope(family, B, _log_int(rng, 1, max(1, min(16384, most // B))), Hq, Hkv, D,
                     dtype, axes=rng.choice([1, 1, 2, 3]),
                     rot=rng.choice([D, D, max(16, D // 2)]),
                     interleaved=rng.random() < 0.3, norm=rng.random() < 0.7)
    page = rng.choice([16, 32, 64, 128, 256])
    if family == "append":
        most = min(16384, (1 << 26) // (Hq * D) // (2 if dtype == "f32" else 1))
        T = _log_int(rng, 1, most)
        return _append(T, Hq, Hkv, D, page, -(-T // page) + rng.choice([1, 7, 64]), dtype,
                       norm=rng.random() < 0.7, interleaved=rng.random() < 0.3,
                       rot=rng.choice([D, D, max(16, D // 2)]))
    p, unit = rng.choice([(2, False), (2, True), (1, True)])
    kw = {"p": p, "unit": unit, "ragged": rng.random() < 0.7, "lens_seed": rng.randrange(1000)}
    row = Hkv * D * (2 if dtype == "f32" else 1)
    if family == "decode":
        S = _log_int(rng, 1, 128)
        longest = _log_int(rng, 1, min(131072, (1 << 27) // row // S))
        return _paged(S, longest, 1, Hq, Hkv, D, page, dtype, **kw)
    if family == "window":
        S = _log_int(rng, 1, 64)
        longest = _log_int(rng, 64, min(65536, (1 << 28) // row // S))
        return _paged(S, longest, rng.choice([1, 1, 1, 4]), Hq, Hkv, D, page, dtype,
                      window=_log_int(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 64]), **kw)
    new = _log_int(rng, 2, 2048)
    S = rng.choice([1, 1, 2, 3, 4, 8])
    most = (1 << 38) // (Hq * D * new * S) // (4 if dtype == "f32" else 1)
    longest = max(new, _log_int(rng, new, max(new, min(32768, most, (1 << 27) // row // S))))
    if rng.random() < 0.3:
        kw.update(window=_log_int(rng, 16, 8192), sinks=rng.choice([0, 4, 64]))
    return _paged(S, longest, new, Hq, Hkv, D, page, dtype, **kw)


# --- what a user's program has in hand ---------------------------------------

def _table(rows, rot):
    """cos and sin of the rotation, float32 [rows, rot / 2], base 10000."""
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    a = torch.arange(rows, dtype=torch.float64)[:, None] * inv[None]
    return a.cos().float().cuda(), a.sin().float().cuda()


def _sections(case):
    """Pairs of channels per axis of positions."""
    half, axes = case["rot"] // 2, case["axes"]
    side = half // (axes + 1)
    return [half - side * (axes - 1)] + [side] * (axes - 1)


def _weights(case, gen):
    if not case["norm"]:
        return None, None
    return tuple(1.0 + 0.1 * torch.randn(case["D"], generator=gen, device="cuda")
                 for _ in range(2))


def _lens(case):
    """Lengths and new tokens of the sequences (the same for every seed)."""
    rng = random.Random(case["lens_seed"])
    top, new = case["longest"], case["new"]
    lens, news = [], []
    for s in range(case["S"]):
        n = top if s == 0 or not case["ragged"] else _log_int(rng, max(1, top // 16), top)
        t = new if s == 0 or not case["ragged"] else rng.randint(1, new)
        lens.append(n)
        news.append(min(t, n))
    return lens, news


def _standard(x):
    x = x - x.mean(-1, keepdim=True)
    return x / x.square().mean(-1, keepdim=True).sqrt()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, D, Hq, Hkv = DTYPES[case["dtype"]], case["D"], case["Hq"], case["Hkv"]

    def randn(*shape, dtype=dt):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    state = {"case": case}
    if case["call"] in ("rope_fwd", "rope_bwd"):
        B, N, axes = case["B"], case["N"], case["axes"]
        # the projection's output, q, k and v side by side in a token's row
        rows = randn(B, N, Hq + 2 * Hkv, D)
        state.update(zip(("q", "k", "v"), rows.split([Hq, Hkv, Hkv], dim=2)))
        state["wq"], state["wk"] = _weights(case, gen)
        state["cos"], state["sin"] = _table(N, case["rot"])
        n = torch.arange(N, dtype=torch.int32, device="cuda")
        # one axis: the token's index; more: frames of rows and columns
        cols = [n] if axes == 1 else [n // 256, n % 256 // 16, n % 16][:axes]
        state["pos"] = torch.stack(cols, -1).expand(B, N, axes).contiguous()
        state["sections"] = _sections(case)
        if case["call"] == "rope_bwd":
            for name in ("dq", "dk", "dv"):
                state[name] = randn(B, Hq, N, D)
        return state

    page = case["page"]
    if case["call"] == "append":
        T, pages = case["T"], case["pages"]
        rows = randn(T, Hq + 2 * Hkv, D)
        state.update(zip(("q", "k", "v"), rows.split([Hq, Hkv, Hkv], dim=1)))
        state["wq"], state["wk"] = _weights(case, gen)
        state["cos"], state["sin"] = _table(16384, case["rot"])
        state["pos"] = torch.randint(0, 16384, (T, 1), generator=gen, device="cuda",
                                     dtype=torch.int32)
        # a token in thirty is padding: it has no slot
        slots = torch.randperm(pages * page, generator=gen, device="cuda")[:T]
        pad = torch.rand(T, generator=gen, device="cuda") < 1.0 / 30
        state["slots"] = torch.where(pad, -torch.ones_like(slots), slots)
        state["k_cache"], state["v_cache"] = (randn(pages, Hkv, page, D) for _ in range(2))
        state["sections"] = _sections(case)
        return state

    lens, news = _lens(case)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32).cpu()
    table = torch.full((case["S"], max(need)), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    state["lens_host"], state["news_host"] = lens, news
    state["table"] = table.cuda()
    state["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    state["q_start"] = None
    if case["new"] > 1:
        start = [0]
        for t in news:
            start.append(start[-1] + t)
        state["q_start"] = torch.tensor(start, dtype=torch.int32).cuda()
    f32 = torch.float32
    state["q"] = _standard(randn(sum(news), Hq, D, dtype=f32)).to(dt)
    state["k_cache"] = torch.empty((pages, Hkv, page, D), dtype=dt, device="cuda")
    state["v_cache"] = torch.empty_like(state["k_cache"])
    for i in range(0, pages, 4096):
        shape = state["k_cache"][i:i + 4096].shape
        state["k_cache"][i:i + 4096] = _standard(randn(*shape, dtype=f32))
        state["v_cache"][i:i + 4096] = randn(*shape, dtype=f32)
    state["scale"] = 1.0 / D if case["unit"] else None
    return state


# --- plain forms: elementary operations in float32 ----------------------------

def _angles(state):
    """cos and sin of every token's rotation, [..., 1, rot / 2]."""
    pos, half = state["pos"].long(), state["case"]["rot"] // 2
    axis = torch.repeat_interleave(torch.arange(len(state["sections"]), device="cuda"),
                                   torch.tensor(state["sections"], device="cuda"))
    at = pos[..., axis]                                  # [..., rot / 2]
    j = torch.arange(half, device="cuda")
    return state["cos"][at, j].unsqueeze(-2), state["sin"][at, j].unsqueeze(-2)


def _halves(x, case):
    rot = case["rot"]
    if case["interleaved"]:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def _joined(a, b, rest, case):
    if case["interleaved"]:
        return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)
    return torch.cat([a, b, rest], -1)


def _norm(x, w):
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w


def _turn(x, cos, sin, case):
    a, b, rest = _halves(x, case)
    return _joined(a * cos - b * sin, b * cos + a * sin, rest, case)


def _plain_rope_fwd(state):
    case = state["case"]
    dt, group = DTYPES[case["dtype"]], case["Hq"] // case["Hkv"]
    cos, sin = _angles(state)
    q = _turn(_norm(state["q"].float(), state["wq"]), cos, sin, case).to(dt)
    k = _turn(_norm(state["k"].float(), state["wk"]), cos, sin, case).to(dt)
    return (q.transpose(1, 2).contiguous(),
            k.repeat_interleave(group, 2).transpose(1, 2).contiguous(),
            state["v"].repeat_interleave(group, 2).transpose(1, 2).contiguous())


def _plain_norm_bwd(x, w, dy):
    """Gradients of x * rsqrt(mean(x^2) + eps) * w."""
    if w is None:
        return dy, None
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    dw = (dy * x * r).sum((0, 1, 2))
    dy = dy * w
    return r * (dy - x * (r * r) * (dy * x).mean(-1, keepdim=True)), dw


def _plain_rope_bwd(state):
    case = state["case"]
    dt, B, N, Hkv = DTYPES[case["dtype"]], case["B"], case["N"], case["Hkv"]
    cos, sin = _angles(state)

    def rows(d):
        return d.float().transpose(1, 2)

    def shared(d):
        return rows(d).reshape(B, N, Hkv, -1, case["D"]).sum(3)

    dq, dwq = _plain_norm_bwd(state["q"], state["wq"], _turn(rows(state["dq"]), cos, -sin, case))
    dk, dwk = _plain_norm_bwd(state["k"], state["wk"], _turn(shared(state["dk"]), cos, -sin, case))
    out = {"dq": dq.to(dt).contiguous(), "dk": dk.to(dt).contiguous(),
           "dv": shared(state["dv"]).to(dt).contiguous()}
    return out if dwq is None else dict(out, dwq=dwq, dwk=dwk)


def _plain_append(state):
    case = state["case"]
    dt, page = DTYPES[case["dtype"]], case["page"]
    cos, sin = _angles(state)
    q = _standard(_turn(_norm(state["q"].float(), state["wq"]), cos, sin, case)).to(dt)
    k = _standard(_turn(_norm(state["k"].float(), state["wk"]), cos, sin, case)).to(dt)
    slots = state["slots"]
    # tokens without a slot write the row that a token with one writes too
    has = slots >= 0
    first = has.to(torch.int8).argmax()
    use = torch.where(has, torch.arange(len(slots), device="cuda"), first)
    to = slots[use].clamp(min=0)
    some = has.any()
    for cache, rows in ((state["k_cache"], k), (state["v_cache"], state["v"])):
        at = cache[to // page, :, to % page]
        cache[to // page, :, to % page] = torch.where(some, rows[use], at)
    return {"q": q, "k_cache": state["k_cache"], "v_cache": state["v_cache"]}


def _visible(pos, n, window, sinks):
    """Whether the query at position pos sees key n."""
    see = n <= pos
    return see & ((n > pos - window) | (n < sinks)) if window else see


def _plain_paged(state):
    case = state["case"]
    D, Hq, Hkv, page, new = case["D"], case["Hq"], case["Hkv"], case["page"], case["new"]
    dt, group = DTYPES[case["dtype"]], Hq // Hkv
    tau = 1.0 if state["scale"] is None else state["scale"]
    lens, news, out = state["lens_host"], state["news_host"], torch.empty_like(state["q"])
    window, sinks = case["window"], case["sinks"]
    by_len = sorted(range(case["S"]), key=lambda s: lens[s])
    start = [0]
    for t in news:
        start.append(start[-1] + t)
    at = 0
    while at < len(by_len):
        # sequences of like lengths together, within a few GB
        pick = [by_len[at]]
        while (at + len(pick) < len(by_len)
               and (len(pick) + 1) * lens[by_len[at + len(pick)]]
               * max(Hkv * D, Hq * new) <= 1 << 29):
            pick.append(by_len[at + len(pick)])
        at += len(pick)
        sel = torch.tensor(pick, device="cuda")
        top, most = max(lens[s] for s in pick), max(news[s] for s in pick)
        n = torch.arange(top, device="cuda")
        live = n[None] < state["lens"][sel].long()[:, None]              # [s, top]
        pages = state["table"][sel][:, :-(-top // page)].long().clamp(min=0)

        def rows(cache):
            x = cache[pages].float()                                     # [s, pages, Hkv, page, D]
            x = x.transpose(1, 2).reshape(len(pick), Hkv, -1, D)[:, :, :top]
            return x.masked_fill(~live[:, None, :, None], 0.0)

        k, v = rows(state["k_cache"]), rows(state["v_cache"])
        t = torch.arange(most, device="cuda")
        count = torch.tensor([news[s] for s in pick], device="cuda")
        row = torch.tensor([start[s] for s in pick], device="cuda")[:, None] + t
        row = torch.minimum(row, torch.tensor([start[s + 1] - 1 for s in pick],
                                              device="cuda")[:, None])
        pos = state["lens"][sel].long()[:, None] - count[:, None] + t    # [s, most]
        see = _visible(pos[:, :, None], n, window, sinks) & live[:, None]
        # heads in slices, within a few GB
        q = state["q"][row].float().reshape(len(pick), most, Hkv, group, D)
        step = max(1, (1 << 29) // (len(pick) * most * group * top))
        for h in range(0, Hkv, step):
            qh = q[:, :, h:h + step].permute(0, 2, 1, 3, 4).flatten(2, 3)
            s = torch.matmul(qh, k[:, h:h + step].transpose(-1, -2).contiguous()) * tau
            w = 1.0 + s
            if case["p"] == 2:
                w = w + 0.5 * s * s
            w = torch.where(see[:, None].repeat_interleave(group, 2), w, 0.0)
            o = torch.matmul(w, v[:, h:h + step]) / w.sum(-1, keepdim=True)
            o = o.unflatten(2, (most, group)).permute(0, 2, 1, 3, 4).to(dt)
            for i, s_ in enumerate(pick):
                heads = slice(h * group, (h + step) * group)
                out[start[s_]:start[s_ + 1], heads] = o[i, :news[s_]].flatten(1, 2)
    return out


def run(state):
    case, call = state["case"], state["case"]["call"]
    if not own:
        return {"rope_fwd": _plain_rope_fwd, "rope_bwd": _plain_rope_bwd,
                "append": _plain_append, "paged": _plain_paged}[call](state)
    from paper_2402_07901_amd import fastmax as fm
    if call == "paged":
        return fm.fastmax_paged_fwd(state["q"], state["k_cache"], state["v_cache"],
                                    state["table"], state["lens"], q_start=state["q_start"],
                                    max_q=case["new"], max_len=case["longest"], p=case["p"],
                                    scale=state["scale"], window=case["window"],
                                    sinks=case["sinks"])
    turn = {"wq": state["wq"], "wk": state["wk"], "eps": EPS, "sections": state["sections"],
            "interleaved": case["interleaved"]}
    table = (state["pos"], state["cos"], state["sin"])
    if call == "rope_fwd":
        return fm.fastmax_rope_fwd(state["q"], state["k"], state["v"], *table, **turn)
    if call == "rope_bwd":
        dq, dk, dv, dwq, dwk = fm.fastmax_rope_bwd(state["q"], state["k"], state["dq"],
                                                   state["dk"], state["dv"], *table, **turn)
        out = {"dq": dq, "dk": dk, "dv": dv}
        return out if dwq is None else dict(out, dwq=dwq, dwk=dwk)
    q = fm.fastmax_cache_append(state["q"], state["k"], state["v"], state["k_cache"],
                                state["v_cache"], state["slots"], *table, **turn)
    return {"q": q, "k_cache": state["k_cache"], "v_cache": state["v_cache"]}


# --- from the definitions, in 64 bits ------------------------------------------

def _exact_rotated(x, w, state):
    """Norm and rotation of rows x [..., H, D], channel by channel pair."""
    case = state["case"]
    if w is not None:
        x = w.double() * x / ((x * x).sum(-1, keepdim=True) / case["D"] + EPS).sqrt()
    half, cols = case["rot"] // 2, [None] * case["D"]
    axis = [a for a, n in enumerate(state["sections"]) for _ in range(n)]
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + half)
        where = state["pos"][..., axis[j]].long()
        c = state["cos"][:, j].double()[where][..., None]
        s = state["sin"][:, j].double()[where][..., None]
        cols[a] = c * x[..., a] - s * x[..., b]
        cols[b] = s * x[..., a] + c * x[..., b]
    for d in range(case["rot"], case["D"]):
        cols[d] = x[..., d]
    return torch.stack(cols, -1)


def _exact_heads(x, group):
    """[B, N, Hkv, D] as [B, Hkv * group, N, D]: query head h has key head h // group."""
    heads = torch.arange(x.shape[2] * group, device=x.device) // group
    return x[:, :, heads].permute(0, 2, 1, 3)


def _exact_rope(case, seed):
    state, group = prepare(case, seed), case["Hq"] // case["Hkv"]
    x = [state[n].double() for n in ("q", "k", "v")]
    w = [None if state[n] is None else state[n].double() for n in ("wq", "wk")]
    back = case["call"] == "rope_bwd"
    leaves = x + [t for t in w if t is not None]
    if back:
        for t in leaves:
            t.requires_grad_()
    out = (_exact_rotated(x[0], w[0], state).permute(0, 2, 1, 3),
           _exact_heads(_exact_rotated(x[1], w[1], state), group), _exact_heads(x[2], group))
    if not back:
        return out
    grads = torch.autograd.grad(out, leaves, [state[n].double() for n in ("dq", "dk", "dv")])
    return dict(zip(("dq", "dk", "dv", "dwq", "dwk"), grads))


def _exact_append(case, seed):
    state = prepare(case, seed)
    rows = {}
    for name, w in (("q", state["wq"]), ("k", state["wk"])):
        z = _exact_rotated(state[name].double(), w, state)
        z = z - z.sum(-1, keepdim=True) / case["D"]
        rows[name] = z / ((z * z).sum(-1, keepdim=True) / case["D"]).sqrt()
    keep = state["slots"] >= 0
    slots = state["slots"][keep]
    out = {"q": rows["q"]}
    for name, new in (("k_cache", rows["k"]), ("v_cache", state["v"].double())):
        flat = state[name].double().transpose(1, 2).flatten(0, 1)        # [slots, Hkv, D]
        flat[slots] = new[keep]
        out[name] = flat.unflatten(0, (-1, case["page"])).transpose(1, 2)
    return out


def _exact_paged(case, seed):
    state = prepare(case, seed)
    group, page = case["Hq"] // case["Hkv"], case["page"]
    tau = 1.0 if state["scale"] is None else state["scale"]
    out, row = [], 0
    for s, (n, t) in enumerate(zip(state["lens_host"], state["news_host"])):
        key = torch.arange(n, device="cuda")
        at = state["table"][s].long()[key // page]
        heads = []
        for h in range(case["Hkv"]):
            k = state["k_cache"][at, h, key % page].double()
            v = state["v_cache"][at, h, key % page].double()
            q = state["q"][row:row + t, h * group:(h + 1) * group].double()
            parts = []
            for i in range(0, t, 256):
                x = tau * torch.matmul(q[i:i + 256].flatten(0, 1), k.t().contiguous())
                w = 1 + x + (x * x / 2 if case["p"] == 2 else 0)
                pos = n - t + torch.arange(i, min(t, i + 256), device="cuda")
                gone = key[None] > pos[:, None]
                if case["window"]:
                    gone |= (key[None] <= pos[:, None] - case["window"]) & (key[None] >= case["sinks"])
                w = w.masked_fill(gone.repeat_interleave(group, 0), 0.0)
                parts.append(torch.matmul(w, v) / w.sum(-1, keepdim=True))
            heads.append(torch.cat(parts).unflatten(0, (t, group)))
        out.append(torch.cat(heads, 1))
        row += t
    return torch.cat(out)


def exact(case, seed):
    if case["call"] == "paged":
        return _exact_paged(case, seed)
    return (_exact_append if case["call"] == "append" else _exact_rope)(case, seed)


# --- what a pass cannot do without ----------------------------------------------

def work(case):
    D, Hq, Hkv = case["D"], case["Hq"], case["Hkv"]
    elt = 4 if case["dtype"] == "f32" else 2
    if case["call"] in ("rope_fwd", "rope_bwd", "append"):
        tokens = case["T"] if case["call"] == "append" else case["B"] * case["N"]
        half = case["rot"] // 2
        rows = 16384 if case["call"] == "append" else case["N"]
        table = 8 * half * min(rows, tokens) + 4 * tokens * case["axes"]
        narrow, wide = (Hq + 2 * Hkv) * D * elt, 3 * Hq * D * elt
        turned = (Hq + Hkv) * D * tokens
        if case["call"] == "append":
            return {"bytes": 2 * narrow * tokens + table + 8 * tokens, "flops": 14 * turned}
        if case["call"] == "rope_fwd":
            return {"bytes": (narrow + wide) * tokens + table, "flops": 7 * turned}
        reads = (Hq + Hkv) * D * elt if case["norm"] else 0     # the norm's own inputs
        shared = (2 * Hq - 2 * Hkv) * D * tokens
        return {"bytes": (narrow + wide + reads) * tokens + table,
                "flops": 15 * turned + shared}
    lens, news = _lens(case)
    window, sinks = case["window"], case["sinks"]
    keys = pairs = 0
    for n, t in zip(lens, news):
        first = n - t                             # the first new token's position
        if not window:
            keys += n
            pairs += t * first + t * (t + 1) // 2
        else:
            low = max(0, first - window + 1)      # the lowest key in a window
            keys += n - low + min(sinks, low)
            for pos in range(first, n):
                low = max(0, pos - window + 1)
                pairs += pos + 1 - low + min(sinks, low)
    moved = keys * Hkv * D * 2 + 2 * sum(news) * Hq * D
    return {"bytes": moved * elt + 4 * case["S"] + 4 * sum(-(-n // case["page"]) for n in lens),
            "flops": 4.0 * D * Hq * pairs}
