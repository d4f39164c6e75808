"""Linear layers of 4-bit weights with a scale for every few inputs, dense and by expert, as measurable cases.

Kinds of passes:

  linear     y[n][m] = sum_k s[m][k // group] * (u[m][k] - z[m][k // group]) * x[n][k], u in 0..15; z is 8 ("sym")
             or a code of its own for every group ("zero")
  experts    the same for tokens sorted by expert: row p of expert e (offsets[e] <= p < offsets[e + 1]) is
             multiplied with that expert's matrix; its input is row rows[p] of x
  dispatch   (token, choice) pairs sorted by expert (stable), and the tokens' rows copied in that order
  combine    back: every token the weighted sum of its choices' rows
  backward   the gradient of combine: the rows' and the weights'

Ids outside the experts are padded tokens: they get no place, and rows behind the last sorted one stay as they were.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # BERT-large's attention output layer for one token: the smallest call, all latency
        dict(name="linear_1024x1024_n1_bf16", kind="linear", M=1024, K=1024, N=1, type="bf16", group=128, mode="sym"),
        # odd sizes and fp32 activations, three tokens: a classifier head
        dict(name="linear_1000x777_n3_f32", kind="linear", M=1000, K=777, N=3, type="f32", group=32, mode="zero"),
        # a wide layer of a large model for eight sequences at once: bound by reading the codes
        dict(name="linear_8192x8192_n8_f16", kind="linear", M=8192, K=8192, N=8, type="f16", group=128, mode="zero"),
        # BERT-large's feed-forward layer for a prompt
        dict(name="linear_4096x1024_n2048_bf16", kind="linear", M=4096, K=1024, N=2048, type="bf16", group=64, mode="sym"),
        # 32 sequences, one token each, through 64 small experts: a few rows an expert
        dict(name="experts_64_t32_k8_bf16", kind="experts", E=64, M=1408, K=2048, T=32, k=8, type="bf16", group=128, mode="sym", padded=0.0),
        # a prompt through sixteen experts of BERT-large's feed-forward width, some tokens padding
        dict(name="experts_16_t4096_k2_f16", kind="experts", E=16, M=4096, K=1024, T=4096, k=2, type="f16", group=128, mode="zero", padded=0.05),
        # one token to its two experts, and a batch of prompts
        dict(name="dispatch_8_t1_k2_bf16", kind="dispatch", E=8, T=1, k=2, H=1024, type="bf16", padded=0.0),
        dict(name="dispatch_64_t8192_k8_bf16", kind="dispatch", E=64, T=8192, k=8, H=2048, type="bf16", padded=0.1),
        # a few sequences' tokens back, an odd width; a batch of prompts
        dict(name="combine_16_t5_k4_f32", kind="combine", E=16, T=5, k=4, H=777, type="f32", padded=0.2),
        dict(name="combine_64_t8192_k8_bf16", kind="combine", E=64, T=8192, k=8, H=2048, type="bf16", padded=0.1),
        # a small training batch, and a large one
        dict(name="backward_8_t300_k2_f32", kind="backward", E=8, T=300, k=2, H=768, type="f32", padded=0.1),
        dict(name="backward_64_t4096_k8_bf16", kind="backward", E=64, T=4096, k=8, H=2048, type="bf16", padded=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "experts", "experts", "dispatch", "combine", "backward"])
    c = dict(kind=kind, type=rng.choice(["bf16", "bf16", "f16", "f32"]))
    if kind in ("linear", "experts"):
        M, K = _log(rng, 32, 8192), _log(rng, 32, 8192)
        if rng.random() < 0.7:                       # most layers are a multiple of 32 wide; some are not
            M, K = max(32, M // 32 * 32), max(32, K // 32 * 32)
        c.update(M=M, K=K, group=rng.choice([32, 64, 128, 128]), mode=rng.choice(["sym", "zero"]))
        if kind == "linear":
            c.update(N=min(_log(rng, 1, 2048), max(1, (1 << 33) // (M * K))))
        else:
            E = min(_log(rng, 2, 256), max(2, (1 << 27) // (M * K)))
            k = rng.randint(1, min(8, E))
            c.update(E=E, k=k, T=min(_log(rng, 1, 4096), max(1, (1 << 33) // (M * K * k))), padded=rng.choice([0.0, 0.05, 0.3]))
    else:
        E = _log(rng, 2, 512)
        k = rng.randint(1, min(8, E))
        H = _log(rng, 32, 8192)
        if rng.random() < 0.7:
            H = max(32, H // 32 * 32)
        c.update(E=E, k=k, H=H, T=min(_log(rng, 1, 32768), max(1, (1 << 26) // (H * k))), padded=rng.choice([0.0, 0.1, 0.5]))
    return c


# ------------------------------------------------------------------ inputs

def _weights(g, E, c):
    """Codes [E][M][K], scales [E][M][G] and zero points of normal weights, quantized group by group."""
    M, K, group = c["M"], c["K"], c["group"]
    G = -(-K // group)
    stype = torch.float16 if c["type"] == "f16" else torch.bfloat16
    codes = torch.empty((E, M, K), dtype=torch.uint8, device="cuda")
    scale = torch.empty((E, M, G), dtype=stype, device="cuda")
    zero = torch.empty((E, M, G), dtype=torch.uint8, device="cuda") if c["mode"] == "zero" else None
    step = max(1, (1 << 26) // (M * G * group))      # experts at once, so that the fp32 copies stay small
    for e in range(0, E, step):
        n = min(step, E - e)
        w = torch.zeros((n, M, G * group), device="cuda")
        w[:, :, :K] = torch.randn((n, M, K), generator=g, device="cuda") * 0.02
        w = w.view(n, M, G, group)
        if zero is None:
            s = (w.abs().amax(-1) / 7).to(stype)
            u = (w / s.float().unsqueeze(-1)).round().clamp(-7, 7) + 8
        else:
            lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
            s = ((hi - lo) / 15).to(stype)
            z = (-lo / s.float()).round().clamp(0, 15)
            u = ((w / s.float().unsqueeze(-1)).round() + z.unsqueeze(-1)).clamp(0, 15)
            zero[e:e + n] = z.to(torch.uint8)
        scale[e:e + n] = s
        codes[e:e + n] = u.reshape(n, M, G * group)[:, :, :K].to(torch.uint8)
    return codes, scale, zero


def _rows_of(g, n, width, c):
    """Activations: normal, a few channels much larger, as they are behind a transformer's norms."""
    x = torch.randn((n, width), generator=g, device="cuda")
    loud = torch.rand(width, generator=g, device="cuda") < 0.005
    return (x * torch.where(loud, 20.0, 1.0)).to(TYPES[c["type"]])


def _route(g, c):
    """Expert ids [T][k], the top choices of logits that favour some experts, and their weights; padded tokens have id -1."""
    T, E, k = c["T"], c["E"], c["k"]
    logits = torch.randn((T, E), generator=g, device="cuda") + 0.5 * torch.randn(E, generator=g, device="cuda")
    top, ids = logits.topk(k, dim=-1)
    gone = torch.rand(T, generator=g, device="cuda") < c["padded"]
    return torch.where(gone[:, None], -1, ids).int(), torch.softmax(top, dim=-1).contiguous()


def _sorted(ids, E, k):
    """offsets [E + 1], rows [T * k] (sorted position -> token, -1 behind the last), place [T][k] (pair -> position, -1: none)."""
    flat = ids.reshape(-1).long()
    kept = (flat >= 0) & (flat < E)
    key = torch.where(kept, flat, E)
    order = torch.sort(key, stable=True).indices
    counts = (key[:, None] == torch.arange(E, device=key.device)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    position = torch.empty_like(order)
    position[order] = torch.arange(order.numel(), device=order.device)
    place = torch.where(kept, position, -1).view(ids.shape)
    rows = torch.where(key[order] < E, order // k, -1)
    return offsets.int(), rows.int(), place.int()


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c, st = case, {"case": case}
    if c["kind"] == "linear":
        st["codes"], st["scale"], st["zero"] = _weights(g, 1, c)
        st["x"] = _rows_of(g, c["N"], c["K"], c)
        return st
    st["ids"], st["w"] = _route(g, c)
    if c["kind"] == "experts":
        st["codes"], st["scale"], st["zero"] = _weights(g, c["E"], c)
        st["x"] = _rows_of(g, c["T"], c["K"], c)
        st["offsets"], st["rows"], _ = _sorted(st["ids"], c["E"], c["k"])
    elif c["kind"] == "dispatch":
        st["x"] = _rows_of(g, c["T"], c["H"], c)
    else:
        st["place"] = _sorted(st["ids"], c["E"], c["k"])[2]
        st["ys"] = _rows_of(g, c["T"] * c["k"], c["H"], c)
        if c["kind"] == "backward":
            st["dy"] = torch.randn((c["T"], c["H"]), generator=g, device="cuda").to(TYPES[c["type"]])
    return st


def prepare(case, seed):
    st, c = _inputs(case, seed), case
    dt = TYPES[c["type"]]
    if own:
        from paper_2111_00153_b200 import binding as R
        st["type"] = {"f32": R.F32, "f16": R.F16, "bf16": R.BF16}[c["type"]]
        if c["kind"] in ("linear", "experts"):
            layer = R.rmsmp_gs4_layer_init(c.get("E", 1), c["M"], c["K"], c["group"], R.GS4_ZERO if c["mode"] == "zero" else R.GS4_SYM,
                                           R.F16 if c["type"] == "f16" else R.BF16)
            packed = torch.empty(layer.packed_bytes, dtype=torch.uint8, device="cuda")
            R.rmsmp_gs4_pack_codes(layer, st["codes"], st["scale"], st["zero"], packed)
            st["layer"], st["packed"] = layer, packed
            st["y"] = torch.zeros((c["N"] if c["kind"] == "linear" else c["T"] * c["k"], c["M"]), dtype=dt, device="cuda")
        elif c["kind"] == "dispatch":
            P = c["T"] * c["k"]
            st["offsets"] = torch.empty(c["E"] + 1, dtype=torch.int32, device="cuda")
            st["rows"] = torch.empty(P, dtype=torch.int32, device="cuda")
            st["place"] = torch.empty((c["T"], c["k"]), dtype=torch.int32, device="cuda")
            st["xs"] = torch.zeros((P, c["H"]), dtype=dt, device="cuda")
        elif c["kind"] == "combine":
            st["y"] = torch.empty((c["T"], c["H"]), dtype=dt, device="cuda")
        else:
            st["dys"] = torch.zeros((c["T"] * c["k"], c["H"]), dtype=dt, device="cuda")
            st["dw"] = torch.empty((c["T"], c["k"]), dtype=torch.float32, device="cuda")
    return st


# ------------------------------------------------------------------ one pass

def run(state):
    return _own(state) if own else _plain(state)


def _own(st):
    from paper_2111_00153_b200 import binding as R
    c, t = st["case"], st["type"]
    if c["kind"] == "linear":
        R.rmsmp_gs4_gemm(st["layer"], st["packed"], st["x"], t, c["N"], c["K"], st["y"], t, c["M"])
        return st["y"]
    T, k, E = c["T"], c["k"], c["E"]
    P = T * k
    if c["kind"] == "experts":
        R.rmsmp_gs4_gemm_experts(st["layer"], st["packed"], st["x"], t, T, c["K"], st["rows"], st["offsets"], P, st["y"], t, c["M"])
        return st["y"]
    H = c["H"]
    if c["kind"] == "dispatch":
        R.rmsmp_expert_sort(st["ids"], T, k, E, st["offsets"], st["rows"], st["place"])
        R.rmsmp_expert_gather(st["x"], t, T, H, H, st["rows"], P, st["xs"], H)
        return st["offsets"], st["rows"], st["place"], st["xs"]
    if c["kind"] == "combine":
        R.rmsmp_expert_combine(st["ys"], t, P, H, H, st["place"], st["w"], T, k, st["y"], H)
        return st["y"]
    R.rmsmp_expert_combine_backward(st["dy"], t, T, k, H, H, st["ys"], P, H, st["place"], st["w"], st["dys"], H, st["dw"])
    return st["dys"], st["dw"]


def _dequantized(st):
    c = st["case"]
    at = torch.arange(c["K"], device="cuda") // c["group"]
    s = st["scale"].float()[:, :, at]
    z = 8.0 if st["zero"] is None else st["zero"].float()[:, :, at]
    return (st["codes"].float() - z) * s


def _plain(st):
    c = st["case"]
    dt = TYPES[c["type"]]
    if c["kind"] == "linear":
        return (st["x"].float() @ _dequantized(st)[0].T).to(dt)
    T, k, E = c["T"], c["k"], c["E"]
    if c["kind"] == "experts":
        # the sorted rows laid out by (expert, rank), as many an expert as the fullest has: one batched product
        off, rows = st["offsets"].long(), st["rows"].long()
        p = torch.arange(T * k, device="cuda")
        e = (p[:, None] >= off[None, 1:]).sum(1)
        kept = e < E
        e = e.clamp(max=E - 1)
        most = max(1, int((off[1:] - off[:-1]).max()))
        rank = torch.where(kept, p - off[e], most)                     # rows behind the last: a slot that is cut off
        xs = torch.zeros((E, most + 1, c["K"]), device="cuda")
        xs[e, rank] = st["x"].float()[rows.clamp(min=0)]
        y = (xs[:, :most] @ _dequantized(st).transpose(1, 2))
        y = torch.where(kept[:, None], y[e, rank.clamp(max=most - 1)], 0.0)
        return y.to(dt)
    if c["kind"] == "dispatch":
        offsets, rows, place = _sorted(st["ids"], E, k)
        xs = torch.where(rows[:, None] >= 0, st["x"][rows.long().clamp(min=0)], 0)
        return offsets, rows, place, xs
    place = st["place"].long()
    kept = place >= 0
    chosen = st["ys"].float()[place.clamp(min=0)]                      # [T][k][H]
    if c["kind"] == "combine":
        return torch.where(kept[:, :, None], chosen * st["w"][:, :, None], 0.0).sum(1).to(dt)
    dy = st["dy"].float()
    dys = torch.zeros((T * k + 1, c["H"]), device="cuda")
    dys[torch.where(kept, place, T * k).reshape(-1)] = (dy[:, None] * st["w"][:, :, None]).reshape(T * k, -1)
    dw = torch.where(kept, (dy[:, None] * chosen).sum(-1), 0.0)
    return dys[:-1].to(dt), dw


# ------------------------------------------------------------------ the operators in 64 bits

def exact(case, seed):
    c = case
    st = _inputs(case, seed)
    if c["kind"] == "linear":
        return _product(st, 0, st["x"])
    T, k = c["T"], c["k"]
    if c["kind"] == "experts":
        y = torch.zeros((T * k, c["M"]), dtype=torch.float64, device="cuda")
        ends = st["offsets"].tolist()
        for e in range(c["E"]):
            a, b = ends[e], ends[e + 1]
            if b > a:
                y[a:b] = _product(st, e, st["x"].index_select(0, st["rows"][a:b]))
        return y
    if c["kind"] == "dispatch":
        # whole numbers are compared with the plain form's; the rows copied, by a count of the pairs in front of each
        flat = st["ids"].flatten().cpu().tolist()
        queues = [[] for _ in range(c["E"])]
        for i, e in enumerate(flat):
            if 0 <= e < c["E"]:
                queues[e].append(i // k)
        tokens = [t for q in queues for t in q]
        xs = torch.zeros((T * k, c["H"]), dtype=torch.float64, device="cuda")
        xs[:len(tokens)] = st["x"].double().index_select(0, torch.tensor(tokens, dtype=torch.long, device="cuda"))
        return None, None, None, xs
    H = c["H"]
    place, w = st["place"], st["w"].double()
    out = torch.zeros((T, H), dtype=torch.float64, device="cuda")
    dys = torch.zeros((T * k, H), dtype=torch.float64, device="cuda")
    dw = torch.zeros((T, k), dtype=torch.float64, device="cuda")
    for j in range(k):
        t = torch.nonzero(place[:, j] >= 0).flatten()
        p = place[t, j].long()
        if c["kind"] == "combine":
            out[t] += w[t, j, None] * st["ys"][p].double()
        else:
            dys[p] = w[t, j, None] * st["dy"][t].double()
            dw[t, j] = torch.einsum("th,th->t", st["dy"][t].double(), st["ys"][p].double())
    return out if c["kind"] == "combine" else (dys, dw)


def _product(st, e, x):
    """x times expert e's weights in 64 bits, group by group: the sum of codes times activations less the zero point's share, scaled."""
    c = st["case"]
    K, group = c["K"], c["group"]
    y = torch.zeros((x.shape[0], c["M"]), dtype=torch.float64, device="cuda")
    x = x.double()
    for g in range(-(-K // group)):
        a, b = g * group, min(K, (g + 1) * group)
        z = 8.0 if st["zero"] is None else st["zero"][e, :, g].double()
        part = x[:, a:b] @ st["codes"][e, :, a:b].double().T - x[:, a:b].sum(1, keepdim=True) * z
        y += part * st["scale"][e, :, g].double()
    return y


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    size = 4 if c["type"] == "f32" else 2
    if c["kind"] == "linear" or c["kind"] == "experts":
        G = -(-c["K"] // c["group"])
        weights = c["M"] * c["K"] / 2 + c["M"] * G * (2.5 if c["mode"] == "zero" else 2)
        if c["kind"] == "linear":
            n, x_rows, used = c["N"], c["N"], 1
        else:
            x_rows = c["T"] * (1 - c["padded"])
            n, used = x_rows * c["k"], c["E"] * (1 - (1 - c["k"] / c["E"]) ** x_rows)
        return {"bytes": used * weights + size * (x_rows * c["K"] + n * c["M"]), "flops": 2.0 * n * c["M"] * c["K"]}
    T, k, H = c["T"], c["k"], c["H"]
    kept = T * (1 - c["padded"])
    if c["kind"] == "dispatch":
        return {"bytes": 12.0 * T * k + 4 * (c["E"] + 1) + size * H * kept * (1 + k), "flops": 0.0}
    if c["kind"] == "combine":
        return {"bytes": 8.0 * T * k + size * H * (kept * k + T), "flops": 2.0 * kept * k * H}
    return {"bytes": 12.0 * T * k + size * H * (T + 2 * kept * k), "flops": 3.0 * kept * k * H}
