"""Streaming attention: rotary positions, a paged 8-bit cache of keys and values, and the attention that reads it.

A model that makes a clip frame by frame (or answers token by token) rotates its queries and keys by their positions, puts the
new keys and values into pages of a cache, and lets the new queries attend to everything cached.  A case's `op` says which
operator one pass is:

  rope    Y = R(positions) X over [B, H, N, d], or the gradient dX = R^T dY
  append  rotated keys, and values, of a ragged batch of new tokens into the pages of an e4m3 cache with a power of two as the
          scale of each page and head
  attend  softmax attention of the new tokens' queries over the cache, grouped heads, causal or not

Cache layout: K codes [pages, heads, P, d], V codes [pages, heads, d, P], scales float32 [pages, heads].
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

F8 = torch.float8_e4m3fn
LEAST_EXP = -100          # the least exponent of a page's scale


# ---- cases -------------------------------------------------------------------------------------------------

def _rope_case(way, B, H, N, d, dim, layout, axes, dtype, fused, scaled, far):
    """`axes`: 1 = index in a sequence, 3 = (frame, row, column) of a grid; `fused`: X is a slice of a [B, N, 3, H, d] projection;
    `far`: positions of the first axis begin below this."""
    return dict(op="rope", way=way, B=B, H=H, N=N, d=d, dim=dim, layout=layout, axes=axes, dtype=dtype, fused=fused, scaled=scaled, far=far)


def _append_case(seqs, new, spread, held, H, d, P, dim, layout, axes, dtype, fused):
    """`new` tokens a sequence, `spread`: "even" or "ragged" (some sequences none); `held`: tokens in the cache before, at most."""
    return dict(op="append", seqs=seqs, new=new, spread=spread, held=held, H=H, d=d, P=P, dim=dim, layout=layout, axes=axes, dtype=dtype, fused=fused)


def _attend_case(seqs, new, spread, held, Hq, Hkv, d, P, causal, dtype):
    return dict(op="attend", seqs=seqs, new=new, spread=spread, held=held, Hq=Hq, Hkv=Hkv, d=d, P=P, causal=causal, dtype=dtype)


def listed():
    out = []

    def add(name, case):
        out.append(dict(case, name=name))

    # Queries of 48 streams, one token each: a decoding step, where the launch is all it costs.
    add("rope_step", _rope_case("fwd", 1, 40, 48, 128, 128, "half", 1, "bf16", False, True, 75600))
    # Queries (or keys) of one layer at 720p, 21 latent frames, out of the fused projection: the ordinary call of a video model.
    add("rope_720p", _rope_case("fwd", 1, 40, 75600, 128, 128, "interleaved", 3, "bf16", True, False, 21))
    # Gradient of a guidance pair on an odd grid in fp32, three quarters of the head rotated.
    add("rope_grad_f32", _rope_case("bwd", 2, 12, 23715, 128, 96, "half", 3, "f32", False, True, 17))
    # One token of each of 48 streams into their last pages.
    add("append_step", _append_case(48, 1, "even", 16384, 8, 128, 128, 128, "half", 1, "bf16", False))
    # Three new 720p frames of one stream, 40 heads, out of the fused projection.
    add("append_frames_720p", _append_case(1, 10800, "even", 64800, 40, 128, 128, 128, "interleaved", 3, "bf16", True))
    # Prompts of mixed lengths in fp32 at head dimension 64, small pages, half the head rotated.
    add("append_ragged_f32", _append_case(9, 1500, "ragged", 2048, 12, 64, 32, 32, "half", 1, "f32", False))
    # The smallest attention: one token, two heads, a few hundred keys in fp32, as a unit test or a toy model makes it.
    add("attend_first_f32", _attend_case(1, 1, "even", 300, 2, 2, 64, 32, True, "f32"))
    # One token of each of 48 streams, five query heads to a cached one: the ordinary decoding step.
    add("attend_step_grouped", _attend_case(48, 1, "ragged", 16384, 40, 8, 128, 128, True, "bf16"))
    # One token over caches of a quarter of a million tokens, every head its own keys, the smallest pages.
    add("attend_step_264k", _attend_case(2, 1, "even", 264000, 24, 24, 128, 32, True, "bf16"))
    # One 720p frame against 21 cached ones (itself among them), both ways in time: a streaming video layer.
    add("attend_frame_720p", _attend_case(1, 3600, "even", 72000, 40, 40, 128, 128, False, "bf16"))
    # Prompts of mixed lengths, causal, three query heads to a cached one.
    add("attend_prompts_causal", _attend_case(8, 2500, "ragged", 4096, 24, 8, 128, 64, True, "bf16"))
    # Five proposed tokens of each of eight streams checked at once, in fp32.
    add("attend_draft_f32", _attend_case(8, 5, "even", 6144, 12, 4, 128, 64, True, "f32"))
    return out


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rope", "append", "append", "attend", "attend", "attend"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    layout = rng.choice(("half", "interleaved"))
    axes = rng.choice((1, 3))
    for _ in range(10000):
        d = rng.choice((64, 128, 128))
        dim = rng.choice((d, d, d // 2, 3 * d // 4, d // 2 + 6))
        if op == "rope":
            B, H, N = rng.choice((1, 1, 2, 3)), _log_int(rng, 2, 40), _log_int(rng, 1, 118800)
            if B * H * N * d > 4e8:
                continue
            return _rope_case(rng.choice(("fwd", "bwd")), B, H, N, d, dim, layout, axes, dtype, rng.choice((False, True)), rng.choice((False, True)),
                              rng.choice((64, 75600, 4000000)))
        seqs = _log_int(rng, 1, 64)
        new = 1 if rng.random() < 0.4 else _log_int(rng, 2, 11000)
        held = _log_int(rng, 1, 264000)
        spread = rng.choice(("even", "ragged"))
        P = rng.choice((32, 64, 128))
        Hkv = _log_int(rng, 1, 40)
        if op == "append":
            if seqs * new * Hkv * d > 6e7 or seqs * (new + held) * Hkv * d > 6e8:
                continue
            return _append_case(seqs, new, spread, held, Hkv, d, P, dim, layout, axes, dtype, rng.choice((False, True)))
        g = rng.choice((1, 1, 2, 3, 4, 5, 8))
        causal = rng.choice((True, True, False))
        pairs = float(seqs) * new * (held + new) * Hkv * g
        if 4.0 * d * pairs > (2e11 if dtype == "f32" else 4e12) or pairs > 8e9 or seqs * (new + held) * Hkv * d > 1.5e9 or Hkv * g > 40:
            continue
        return _attend_case(seqs, new, spread, held, Hkv * g, Hkv, d, P, causal, dtype)
    raise RuntimeError("no case found")


# ---- inputs ------------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case):
    """(new tokens, tokens held before) of every sequence: the same for every seed, so that a case is one amount of work."""
    S, n, held = case["seqs"], case["new"], case["held"]
    if case["spread"] == "even":
        return [n] * S, [held - (i * 37) % max(1, held // 8) for i in range(S)]
    r = np.random.RandomState(S * 7919 + n)
    new = [n] * S if n == 1 else [int(round(n * f)) for f in r.uniform(0.0, 1.0, S)]
    new[0] = n
    if n > 1 and S > 2:
        new[1], new[2] = 0, 1
    return new, [int(held ** f) for f in r.uniform(0.3, 1.0, S)]


def _axis_pairs(dim, axes):
    pairs = dim // 2
    return [pairs] if axes == 1 else [pairs - 2 * (pairs // 3), pairs // 3, pairs // 3]


def _rope_of(case, scaled):
    """The rotation's parameters as a plain dict: a long-context scaling of the first axis where `scaled`."""
    r = dict(dim=case["dim"], layout=case["layout"], axis_pairs=_axis_pairs(case["dim"], case["axes"]), theta=10000.0, factor=1.0, original_len=0.0,
             ramp_low=1.0, ramp_high=32.0, mscale=1.0)
    if scaled:
        r.update(factor=4.0, original_len=8192.0, mscale=0.1 * math.log(4.0) + 1.0)
    return r


def _positions(axes, n, start, device):
    """int32 [axes, n] from the index of the first token on: that index, or (frame, row, column) of a 45 x 80 grid."""
    p = torch.arange(n, device=device, dtype=torch.int64)
    if axes == 1:
        return (start + p)[None].to(torch.int32)
    return torch.stack([start + p // 3600, p % 3600 // 80, p % 80]).to(torch.int32)


def _own_rope(r):
    import paper_2604_20470_amd as dr
    return dr.RopeParams(r["dim"], layout=dr.ROPE_HALF if r["layout"] == "half" else dr.ROPE_INTERLEAVED, axis_pairs=r["axis_pairs"], theta=r["theta"],
                         factor=r["factor"], original_len=r["original_len"], ramp_low=r["ramp_low"], ramp_high=r["ramp_high"], mscale=r["mscale"])


def _pages(case, new, held):
    """(pages of each sequence, width of the page table, pages in the pool): some spare ones, as in a pool that is in use."""
    P = case["P"]
    need = [-(-(n + h) // P) for n, h in zip(new, held)]
    return need, max(need) + 1, sum(need) + 3


def _quantise(x, dims):
    """e4m3 codes of x with a power of two for each block (amax over `dims`), and its fp32 scale."""
    amax = x.abs().amax(dim=dims, keepdim=True).float()
    m, e = torch.frexp(amax / 448.0)
    e = torch.where(m == 0.5, e - 1, e).clamp(min=LEAST_EXP).float()
    s = torch.exp2(e)
    return (x.float() / s).to(F8), s.flatten(1)


def _cache(case, g, H, pool):
    """A pool of pages in use: normal values whose size varies by page and head, as activations do."""
    P, d, dev = case["P"], case["d"], "cuda"
    ks, vs, kc, vc = [], [], [], []
    step = max(1, int(2e8 // (H * P * d)))
    for a in range(0, pool, step):
        n = min(step, pool - a)
        size = torch.exp(0.4 * torch.randn(2, n, H, 1, 1, generator=g, device=dev))
        k, s = _quantise(torch.randn(n, H, P, d, generator=g, device=dev) * size[0], (2, 3))
        kc.append(k), ks.append(s)
        v, s = _quantise(torch.randn(n, H, d, P, generator=g, device=dev) * size[1], (2, 3))
        vc.append(v), vs.append(s)
    one = lambda v: v[0] if len(v) == 1 else torch.cat([x.view(torch.uint8) if x.dtype == F8 else x for x in v])  # noqa: E731
    return one(kc).view(F8), one(vc).view(F8), one(ks), one(vs)


def prepare(case, seed):
    dev, dt = "cuda", _dtype(case)
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 2 + 1)
    host = np.random.RandomState(int(seed) % (1 << 31))
    st = {"case": case}
    if case["op"] == "rope":
        B, H, N, d = case["B"], case["H"], case["N"], case["d"]
        if case["fused"]:
            x = torch.randn(B, N, 3, H, d, generator=g, device=dev, dtype=dt)[:, :, int(host.randint(3))].permute(0, 2, 1, 3)
        else:
            x = torch.randn(B, H, N, d, generator=g, device=dev, dtype=dt)
        st["x"], st["y"] = x, torch.empty(B, H, N, d, device=dev, dtype=dt)
        if case["axes"] == 1 and N <= 64:            # streams at places of their own
            st["positions"] = torch.from_numpy(host.randint(0, case["far"], (1, N)).astype(np.int32)).to(dev)
        else:
            st["positions"] = _positions(case["axes"], N, int(host.randint(case["far"])), dev)
        st["rope"] = _rope_of(case, case["scaled"])
    else:
        new, held = _lengths(case)
        S, T = len(new), sum(new)
        H = case["H"] if case["op"] == "append" else case["Hkv"]
        need, width, pool = _pages(case, new, held)
        st["k"], st["v"], st["k_scale"], st["v_scale"] = _cache(case, g, H, pool)
        ids, table, at = host.permutation(pool), np.zeros((S, width), np.int32), 0
        for i, n in enumerate(need):
            table[i, :n] = ids[at:at + n]
            at += n
        st["table"] = torch.from_numpy(table).to(dev)
        st["cu"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(dev)
        st["lens"] = torch.from_numpy((np.array(new) + np.array(held)).astype(np.int32)).to(dev)
        if case["op"] == "append":
            if case["fused"]:
                x = torch.randn(T, 3, H, case["d"], generator=g, device=dev, dtype=dt)
                st["new_k"], st["new_v"] = x[:, 1], x[:, 2]
            else:
                st["new_k"], st["new_v"] = (torch.randn(T, H, case["d"], generator=g, device=dev, dtype=dt) for _ in range(2))
            if case["axes"] == 1:
                st["positions"] = None               # the index in the sequence
            else:
                st["positions"] = torch.cat([_positions(3, n, h // 3600, dev) for n, h in zip(new, held)], 1).contiguous()
            st["rope"] = _rope_of(case, False)
        else:
            st["q"] = 1.5 * torch.randn(T, case["Hq"], case["d"], generator=g, device=dev, dtype=dt)
            st["o"] = torch.empty_like(st["q"])
            st["lse"] = torch.empty(case["Hq"], T, device=dev)
            st["longest"], st["most"] = max(n + h for n, h in zip(new, held)), max(new)
    if own:
        import paper_2604_20470_amd as dr
        st["ctx"] = dr.Context(torch.cuda.current_device())
        if "rope" in st:
            st["params"] = _own_rope(st["rope"])
        if "k" in st:
            st["cache"] = dr.PagedCache.of(st["k"], st["v"], st["k_scale"], st["v_scale"])
            st["batch"] = dr.CacheBatch(st["cu"], st["lens"], st["table"], T)
    return st


# ---- the plain forms ---------------------------------------------------------------------------------------

def _frequencies(r):
    """(angle per unit of position, axis) of every pair."""
    f, axis = [], []
    for a, n in enumerate(r["axis_pairs"]):
        base = r["theta"] ** (-np.arange(n, dtype=np.float64) / n)
        if a == 0 and r["factor"] != 1.0:
            keep = 0.0
            if r["original_len"] > 0:
                turns = r["original_len"] * base / (2.0 * math.pi)
                keep = np.clip((turns - r["ramp_low"]) / (r["ramp_high"] - r["ramp_low"]), 0.0, 1.0)
            base = base * ((1.0 - keep) / r["factor"] + keep)
        f.append(base)
        axis += [a] * n
    return np.concatenate(f), np.array(axis)


def _rotate(x, positions, r, back=False):
    """x [..., n, d] in fp32, positions [axes, n]: the angles in 64 bits, the rotation in 32."""
    f, axis = _frequencies(r)
    f, axis = torch.from_numpy(f).to(x.device), torch.from_numpy(axis).to(x.device)
    angle = positions.double()[axis].transpose(0, 1) * f
    c, s = (r["mscale"] * torch.cos(angle)).float(), (r["mscale"] * torch.sin(angle)).float()
    if back:
        s = -s
    dim = r["dim"]
    if r["layout"] == "half":
        a, b = x[..., :dim // 2], x[..., dim // 2:dim]
        return torch.cat([a * c - b * s, b * c + a * s, x[..., dim:]], -1)
    a, b = x[..., 0:dim:2], x[..., 1:dim:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., dim:]], -1)


def _places(st, T):
    """(sequence, index in the sequence) of every new token."""
    cu, lens = st["cu"].long(), st["lens"].long()
    n = cu[1:] - cu[:-1]
    seq = torch.repeat_interleave(torch.arange(n.numel(), device=cu.device), n, output_size=T)
    return seq, lens[seq] - cu[seq + 1] + torch.arange(T, device=cu.device)


def _fill(codes, scale, values, page, slot, kept, along):
    """values [T, H, d] into the pages' slots (on axis `along` of the codes); `kept`: for each page how many of its tokens stay."""
    T, H, d = values.shape
    pages = scale.shape[0]
    amax = torch.zeros(pages, H, device=values.device).index_reduce_(0, page, values.abs().amax(-1), "amax")
    m, e = torch.frexp(amax / 448.0)
    e = torch.where(m == 0.5, e - 1, e).clamp(min=LEAST_EXP)
    old = torch.frexp(scale)[1] - 1
    e = torch.where((kept > 0)[:, None], torch.maximum(e, old), e)
    touched = torch.zeros(pages, dtype=torch.bool, device=values.device).index_fill_(0, page, True)
    e = torch.where(touched[:, None], e, old)
    grown = torch.nonzero((e > old).any(1) & (kept > 0)).flatten()
    again = codes[grown].float() * torch.exp2((old - e)[grown].float())[:, :, None, None]
    at = torch.arange(codes.shape[along], device=values.device)
    stays = (at[None] < kept[grown][:, None]).view((-1, 1, codes.shape[2], 1) if along == 2 else (-1, 1, 1, codes.shape[3]))
    raw = codes.view(torch.uint8)
    raw[grown] = torch.where(stays, again.to(F8).view(torch.uint8), raw[grown])
    scale.copy_(torch.where(touched[:, None], torch.exp2(e.float()), scale))
    new = (values * torch.exp2(-e.float())[page][:, :, None]).to(F8).view(torch.uint8)
    if along == 2:
        raw[page, :, slot] = new
    else:
        raw[page, :, :, slot] = new


def _append(st):
    case = st["case"]
    T, P = st["new_k"].shape[0], case["P"]
    seq, index = _places(st, T)
    page, slot = st["table"].long()[seq, index // P], index % P
    positions = index[None] if st["positions"] is None else st["positions"]
    k = _rotate(st["new_k"].float().transpose(0, 1), positions, st["rope"]).transpose(0, 1)
    # tokens that a page holds already: the slots before the first new one, on the page of each sequence's first new token
    n = st["cu"][1:] - st["cu"][:-1]
    start = (st["lens"] - n).long()
    head = st["table"].long().gather(1, (start // P)[:, None])[:, 0]
    kept = torch.zeros(st["k"].shape[0], dtype=torch.long, device=seq.device)
    kept.scatter_reduce_(0, head, torch.where(n > 0, start % P, 0), "amax")
    _fill(st["k"], st["k_scale"], k, page, slot, kept, 2)
    _fill(st["v"], st["v_scale"], st["new_v"].float(), page, slot, kept, 3)
    return {"k": st["k"], "v": st["v"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _attend(st):
    """Sequences padded to the longest: queries [S, Hkv, most * group, d], keys [S, Hkv, longest, d]."""
    case = st["case"]
    Hq, Hkv, d, P = case["Hq"], case["Hkv"], case["d"], case["P"]
    q, G = st["q"], Hq // Hkv
    T, S, most, longest = q.shape[0], case["seqs"], st["most"], st["longest"]
    cu, lens = st["cu"].long(), st["lens"].long()
    table = st["table"].long()[:, :-(-longest // P)]
    sk, sv = st["k_scale"][table][..., None, None], st["v_scale"][table][..., None, None]
    k = (st["k"].view(torch.uint8)[table].view(F8).float() * sk).permute(0, 2, 1, 3, 4).reshape(S, Hkv, -1, d)
    v = (st["v"].view(torch.uint8)[table].view(F8).float() * sv).permute(0, 2, 1, 4, 3).reshape(S, Hkv, -1, d)
    seq, index = _places(st, T)
    row = torch.arange(T, device=q.device) - cu[seq]
    padded = torch.zeros(S, most, Hq, d, device=q.device)
    padded[seq, row] = q.float()
    rows = padded.view(S, most, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(S, Hkv, most * G, d)
    s = torch.matmul(rows, k.transpose(2, 3)).div_(math.sqrt(d))
    j = torch.arange(k.shape[2], device=q.device)
    hidden = (j >= lens[:, None])[:, None, None]
    if case["causal"]:
        n = cu[1:] - cu[:-1]
        i = (lens - n)[:, None] + torch.arange(most * G, device=q.device) // G
        hidden = hidden | (j > i[:, :, None])[:, None]
    s.masked_fill_(hidden, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(torch.isfinite(m), m, 0.0)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v).div_(total.clamp(min=1e-38)).view(S, Hkv, most, G, d).permute(0, 2, 1, 3, 4).reshape(S, most, Hq, d)
    lse = (m + total.log())[..., 0].view(S, Hkv, most, G).permute(0, 2, 1, 3).reshape(S, most, Hq)
    return {"o": o[seq, row].to(q.dtype), "lse": lse[seq, row].t().contiguous()}


def run(st):
    op = st["case"]["op"]
    if own:
        import paper_2604_20470_amd as dr
        if op == "rope":
            call = dr.dr_rope_fwd if st["case"]["way"] == "fwd" else dr.dr_rope_bwd
            call(st["ctx"], st["params"], st["x"], st["positions"], st["y"])
            return st["y"]
        if op == "append":
            dr.dr_cache_append(st["ctx"], st["cache"], st["batch"], st["new_k"], st["new_v"], rope=st["params"], positions=st["positions"])
            return {"k": st["k"], "v": st["v"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}
        dr.dr_cache_attn_fwd(st["ctx"], st["cache"], st["batch"], st["q"], st["o"], causal=st["case"]["causal"], lse=st["lse"])
        return {"o": st["o"], "lse": st["lse"]}
    if op == "rope":
        x = st["x"]
        return _rotate(x.float(), st["positions"], st["rope"], st["case"]["way"] == "bwd").to(x.dtype)
    return _append(st) if op == "append" else _attend(st)


# ---- what a pass cannot do without -------------------------------------------------------------------------

def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rope":
        n = case["B"] * case["H"] * case["N"]
        return {"bytes": 2.0 * n * case["d"] * es + 4.0 * case["axes"] * case["N"], "flops": 3.0 * n * case["dim"]}
    new, held = _lengths(case)
    T = sum(new)
    if case["op"] == "append":
        n = T * case["H"]
        touched = sum(-(-(a + b) // case["P"]) - b // case["P"] for a, b in zip(new, held) if a)
        index = 4.0 * (case["axes"] * T if case["axes"] > 1 else 0) + 4.0 * (touched + 2 * len(new))
        return {"bytes": 2.0 * n * case["d"] * (es + 1) + 8.0 * touched * case["H"] + index, "flops": 3.0 * n * case["dim"] + 4.0 * n * case["d"]}
    keys = sum(a + b for a, b in zip(new, held) if a)
    pages = sum(-(-(a + b) // case["P"]) for a, b in zip(new, held) if a)
    seen = sum(a * b + (a * (a + 1) // 2 if case["causal"] else a * a) for a, b in zip(new, held))
    return {"bytes": 2.0 * T * case["Hq"] * case["d"] * es + 4.0 * T * case["Hq"] + 2.0 * keys * case["Hkv"] * case["d"] + pages * (8.0 * case["Hkv"] + 4.0),
            "flops": 4.0 * case["d"] * case["Hq"] * seen}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------

def _exact_rotation(x, positions, r, back):
    """x [n, heads, d] in 64 bits, one pair of channels after another."""
    y = x.clone()
    pair = 0
    for a, n in enumerate(r["axis_pairs"]):
        for i in range(n):
            f = r["theta"] ** (-i / n)
            if a == 0 and r["factor"] != 1.0:
                if r["original_len"] > 0:
                    turns = r["original_len"] * f / (2.0 * math.pi)
                    keep = min(1.0, max(0.0, (turns - r["ramp_low"]) / (r["ramp_high"] - r["ramp_low"])))
                    f = (1.0 - keep) * f / r["factor"] + keep * f
                else:
                    f = f / r["factor"]
            phi = (positions[a].double() * f)[:, None]
            lo, hi = (pair, pair + r["dim"] // 2) if r["layout"] == "half" else (2 * pair, 2 * pair + 1)
            cos, sin = torch.cos(phi), torch.sin(-phi if back else phi)
            y[..., lo] = r["mscale"] * (x[..., lo] * cos - x[..., hi] * sin)
            y[..., hi] = r["mscale"] * (x[..., hi] * cos + x[..., lo] * sin)
            pair += 1
    return y


def _exact_e4m3(x):
    """The nearest e4m3 value, ties to the even code, of |x| <= 448 in 64 bits."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    e = torch.where(torch.exp2(e) > x.abs().clamp(min=2.0 ** -6), e - 1, e)
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _exact_pages(st, codes, scales, values, along):
    """One sequence, one page after another."""
    codes, scales = codes.float().double(), scales.double()
    cu, lens, table, P = st["cu"].tolist(), st["lens"].tolist(), st["table"].tolist(), st["case"]["P"]
    if along == 3:
        codes = codes.transpose(2, 3)
    for s in range(len(lens)):
        at, n = lens[s] - (cu[s + 1] - cu[s]), cu[s + 1] - cu[s]
        done = 0
        while done < n:
            page, slot = table[s][(at + done) // P], (at + done) % P
            m = min(P - slot, n - done)
            x = values[cu[s] + done:cu[s] + done + m].transpose(0, 1)                # [heads, m, d]
            top = x.abs().amax((1, 2))
            e = torch.ceil(torch.log2(top / 448.0)).clamp(min=LEAST_EXP)
            e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e)
            e = torch.where((top <= 448.0 * torch.exp2(e - 1)) & (e > LEAST_EXP), e - 1, e)
            if slot:
                old = torch.log2(scales[page])
                e = torch.maximum(e, old)
                shrunk = codes[page, :, :slot] * torch.exp2(old - e)[:, None, None]
                codes[page, :, :slot] = _exact_e4m3(shrunk)
            codes[page, :, slot:slot + m] = _exact_e4m3(x / torch.exp2(e)[:, None, None])
            scales[page] = torch.exp2(e)
            done += m
    return (codes.transpose(2, 3) if along == 3 else codes), scales


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        x = st["x"]
        y = torch.empty(x.shape, dtype=torch.float64, device=x.device)
        for b in range(x.shape[0]):
            y[b] = _exact_rotation(x[b].transpose(0, 1).double(), st["positions"], st["rope"], case["way"] == "bwd").transpose(0, 1)
        return y
    cu, lens = st["cu"].tolist(), st["lens"].tolist()
    if case["op"] == "append":
        if st["positions"] is None:
            index = [torch.arange(l - (b - a), l, device="cuda") for a, b, l in zip(cu[:-1], cu[1:], lens)]
            positions = torch.cat(index)[None]
        else:
            positions = st["positions"]
        # the rotated key is held in 32 bits before it is rounded to 8
        keys = _exact_rotation(st["new_k"].double(), positions, st["rope"], False).float().double()
        k, ks = _exact_pages(st, st["k"], st["k_scale"], keys, 2)
        v, vs = _exact_pages(st, st["v"], st["v_scale"], st["new_v"].double(), 3)
        return {"k": k, "v": v, "k_scale": ks, "v_scale": vs}
    if work(case)["flops"] > 6.5e12:
        return None
    Hq, Hkv, d, P = case["Hq"], case["Hkv"], case["d"], case["P"]
    o = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    raw_k, raw_v = st["k"].view(torch.uint8), st["v"].view(torch.uint8)
    for s in range(len(lens)):
        a, b, l = cu[s], cu[s + 1], lens[s]
        if b == a:
            continue
        ids = st["table"][s, :-(-l // P)].long()
        for h in range(Hkv):
            k = (raw_k[ids, h].view(F8).float().double() * st["k_scale"][ids, h].double()[:, None, None]).reshape(-1, d)[:l]
            v = (raw_v[ids, h].view(F8).float().double() * st["v_scale"][ids, h].double()[:, None, None]).transpose(1, 2).reshape(-1, d)[:l]
            for c in range(a, b, 4096):                                              # queries in pieces: the logits fit
                z = min(b, c + 4096)
                group = range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
                for i in group:
                    x = st["q"][c:z, i].double() @ k.t() / math.sqrt(d)
                    if case["causal"]:
                        place = l - b + torch.arange(c, z, device="cuda")
                        x = torch.where(torch.arange(l, device="cuda")[None] <= place[:, None], x, -math.inf)
                    total = torch.logsumexp(x, 1)
                    lse[i, c:z] = total
                    o[c:z, i] = torch.exp(x - total[:, None]) @ v
    return {"o": o, "lse": lse}
