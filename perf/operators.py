"""The operators around the attention layer and the loss head, as measurable cases: attention over packed documents,
the token embedding and the normalisation, each forward and backward.

Four kinds of case, all through the public binding, outputs and workspaces allocated by the binding as it does by default:

  attn    the attention layer over sequences made of several documents, none of which sees another
          (`bdlm_attn_fwd_packed` / `bdlm_attn_bwd_packed` with a table of documents): forward alone, or a training step
  embed   rows of the embedding table looked up and scaled (`bdlm_embed_fwd`), or the table's gradient (`bdlm_embed_bwd`)
  norm    layer norm or root-mean-square norm with the residual's addition (`bdlm_norm_fwd`), or its gradients
          (`bdlm_norm_bwd`)

`own` chooses between the library's calls and the same operators in elementary torch operations in fp32; `exact` states
them once more in fp64.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


# ------------------------------------------------------------------------------------------------------------ cases
def _attn(name, H, H_kv, d, lens, M=0, window=0, step=True):
    """lens: the documents' lengths, in order, as text; M: block size of the noisy stream (0: clean tokens alone)."""
    return {"name": name, "kind": "attn", "H": H, "H_kv": H_kv, "d": d, "lens": ",".join(str(n) for n in lens), "M": M,
            "window": window, "step": step}


def _embed(name, T, D, V, masked, back, table="bf16", out="bf16"):
    """masked: the share of the tokens that are the mask token."""
    return {"name": name, "kind": "embed", "T": T, "D": D, "V": V, "masked": masked, "back": back, "table": table, "out": out}


def _norm(name, T, D, back, rms, x="bf16", w="bf16", bias=False, residual=True):
    return {"name": name, "kind": "norm", "T": T, "D": D, "back": back, "rms": rms, "x": x, "w": w, "bias": bias,
            "residual": residual}


def listed():
    return [
        # the smallest call: a unit-test sized layer on a few documents, one of them a single token
        _attn("attn_tiny", 2, 2, 64, [100, 1, 27, 128], step=False),
        # a prompt batch of a small model, nothing aligned: odd group size, head dimension 64, forward and backward
        _attn("attn_ragged", 12, 4, 64, [517, 3, 1200, 41, 1, 333, 905]),
        # the forward over a batch of packed texts of ordinary lengths
        _attn("attn_fwd_16k", 32, 8, 128, [611, 1403, 95, 2750, 388, 4096, 1024, 17, 833, 2967, 1200, 1000], step=False),
        # a training step of the block-diffusion layer, both streams, over packed documents of whole blocks
        _attn("attn_blocks_8k", 32, 8, 128, [640, 2048, 64, 3200, 1216, 1024], M=32),
        # the largest: a training step over long documents with short ones between them
        _attn("attn_step_32k", 32, 8, 128, [9000, 700, 12345, 200, 31, 6004, 4488]),
        # a decoding-sized lookup, where the launch is everything
        _embed("embed_fwd_tiny", 17, 1544, 32008, 0.0, False),
        # the lookup of a micro-batch of clean and noisy tokens, half of the noisy ones masked
        _embed("embed_fwd_16k", 16384, 4096, 128256, 0.25, False),
        # the gradient for a small model, sizes that are not round
        _embed("embed_bwd_ragged", 1531, 1544, 32008, 0.3, True),
        # the gradient for a Llama-3-8B-sized table, one token in four the mask token
        _embed("embed_bwd_16k", 16384, 4096, 128256, 0.25, True),
        # the norm before the loss head for a few tokens
        _norm("norm_fwd_tiny", 5, 1544, False, False, bias=True, residual=False),
        # the norm of a layer with its residual, as a training step's forward has it
        _norm("norm_fwd_16k", 16384, 4096, False, True),
        # and its gradients; the norm's largest
        _norm("norm_bwd_16k", 16384, 4096, True, False, bias=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    while True:
        kind = rng.choice(["attn", "embed", "norm"])
        if kind == "attn":
            H_kv = rng.choice([1, 2, 4, 8])
            M = rng.choice([0, 0, 0, 16, 32, 40])
            unit = max(M, 1)
            left = max(unit, _log_uniform(rng, 64, 32768) // unit * unit)
            top, lens = _log_uniform(rng, 64, 32768), []
            while left > 0 and len(lens) < 200:
                n = min(left, max(unit, _log_uniform(rng, 1, top) // unit * unit))
                lens.append(n)
                left -= n
            case = _attn("", H_kv * rng.choice([1, 2, 3, 4, 4, 8]), H_kv, rng.choice([64, 128, 128]), lens, M=M,
                         window=rng.choice([0, 0, 0, _log_uniform(rng, 16, 4096)]), step=rng.random() < 0.6)
        elif kind == "embed":
            D = _log_uniform(rng, 8, 8192)
            D = D if rng.random() < 0.3 else max(8, D // 8 * 8)
            table, out = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("fp16", "fp16"), ("fp32", "fp32"), ("fp32", "bf16"),
                                     ("fp32", "fp16")])
            case = _embed("", _log_uniform(rng, 1, 65536), D, _log_uniform(rng, 100, 128256), rng.choice([0.0, 0.1, 0.25, 0.5]),
                          rng.random() < 0.6, table, out)
        else:
            D = _log_uniform(rng, 8, 16384)
            D = D if rng.random() < 0.3 else max(8, D // 8 * 8)
            x, w = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32"),
                               ("fp32", "fp32")])
            case = _norm("", _log_uniform(rng, 1, 65536), D, rng.random() < 0.6, rng.random() < 0.5, x, w, rng.random() < 0.5,
                         rng.random() < 0.6)
        del case["name"]
        w = work(case)
        top = _TOP[kind]
        if w["flops"] <= top["flops"] and w["bytes"] <= top["bytes"]:
            return case


def _lens(case):
    return [int(n) for n in case["lens"].split(",")]


def _pairs(case):
    """Visible (query, key) pairs of one head, both streams."""
    total, M, W = 0, case["M"], case["window"]
    for n in _lens(case):
        if W == 0 or W >= n:
            total += n * (n + 1) // 2
        else:
            total += W * (W + 1) // 2 + (n - W) * W
        for b in range(n // M if M else 0):
            p = b * M
            total += M * M   # the block itself
            # row i of the block sees clean keys max(0, p + i - W + 1) .. p - 1
            total += M * p if W == 0 else sum(max(0, p - max(0, p + i - W + 1)) for i in range(M))
    return total


def work(case):
    if case["kind"] == "attn":
        T, H, H_kv, d = sum(_lens(case)), case["H"], case["H_kv"], case["d"]
        streams = 2 if case["M"] else 1
        q, kv, lse = 2 * T * H * d, 2 * T * H_kv * d, 4 * T * H
        # in: q, k, v (dO); out: O, lse (dq, dk, dv)
        b = q + 2 * kv + q + lse + (q + q + 2 * kv if case["step"] else 0)
        return {"bytes": streams * b, "flops": (14 if case["step"] else 4) * d * H * _pairs(case)}
    T, D = case["T"], case["D"]
    if case["kind"] == "embed":
        tb, ob = BYTES[case["table"]], BYTES[case["out"]]
        # forward: each row read and written; backward: each token's row read, the whole gradient written
        return {"bytes": 4 * T + (T * D * ob + case["V"] * D * tb if case["back"] else T * D * (tb + ob)), "flops": T * D}
    xb, wb = BYTES[case["x"]], BYTES[case["w"]]
    params = 2 if case["bias"] else 1
    stats = 4 * T * (1 if case["rms"] else 2)
    if case["back"]:   # dy, h (and the residual path's gradient) in, dx out; the weight in, its gradients out
        return {"bytes": T * D * xb * (4 if case["residual"] else 3) + (1 + params) * D * wb + stats, "flops": 12 * T * D}
    return {"bytes": T * D * xb * (4 if case["residual"] else 2) + params * D * wb + stats, "flops": 8 * T * D}


_TOP = {}
for _c in listed():
    _t = _TOP.setdefault(_c["kind"], {"bytes": 0, "flops": 0})
    for _k, _v in work(_c).items():
        _t[_k] = max(_t[_k], _v)


# ----------------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    state = {"case": case}
    if case["kind"] == "attn":
        T, H, H_kv, d = sum(_lens(case)), case["H"], case["H_kv"], case["d"]
        for s in ("clean", "noisy")[:2 if case["M"] else 1]:
            state["q_" + s] = rand(1, T, H, d).bfloat16()
            state["k_" + s] = rand(1, T, H_kv, d).bfloat16()
            state["v_" + s] = rand(1, T, H_kv, d).bfloat16()
            if case["step"]:
                state["do_" + s] = rand(1, T, H, d).bfloat16()
        ends = torch.tensor([0] + _lens(case), dtype=torch.int64).cumsum(0).int()
        state["cu_seqlens"] = ends.cuda()
        if own:   # the table that a program keeps for all layers of a packed batch
            from paper_2609_19242_b200 import binding
            state["docs"] = binding.bdlm_doc_table(ends)
        return state
    T, D = case["T"], case["D"]
    if case["kind"] == "embed":
        V = case["V"]
        # frequencies fall off as one over the rank, as those of a text's tokens do
        u = torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)
        ids = ((V + 1.0) ** u - 1.0).long().clamp(0, V - 1)
        perm_a = 2 * (V // 3) + 1
        while math.gcd(perm_a, V) != 1:
            perm_a += 1
        ids = ids * perm_a % V   # ranks scattered over the table
        masked = torch.rand(T, generator=gen, device="cuda") < case["masked"]
        ids = torch.where(masked, torch.full_like(ids, V - 1), ids)
        pad = torch.rand(T, generator=gen, device="cuda") < 0.01   # padding
        state["ids"] = torch.where(pad, torch.full_like(ids, -1), ids).int()
        state["scale"] = float(D) ** 0.5 if not case["back"] else 0.125
        if case["back"]:
            state["dout"] = rand(T, D).to(DT[case["out"]])
        else:
            state["table"] = (0.02 * rand(V, D)).to(DT[case["table"]])
        return state
    xt, wt = DT[case["x"]], DT[case["w"]]
    # a residual stream: a few channels much larger than the others, a mean that is not zero
    channel = 0.5 + rand(D).abs() + 10.0 * (torch.rand(D, generator=gen, device="cuda") < 0.01)
    x = rand(T, D) * channel + 0.3
    state["weight"] = (1.0 + 0.2 * rand(D)).to(wt)
    state["bias"] = (0.1 * rand(D)).to(wt) if case["bias"] else None
    state["eps"] = 1e-5
    if case["back"]:
        state["h"] = x.to(xt)
        mean, rstd = _stats(state["h"].double(), case["rms"], state["eps"])
        state["mean"], state["rstd"] = None if case["rms"] else mean.float(), rstd.float()
        state["dy"] = rand(T, D).to(xt)
        state["dh"] = rand(T, D).to(xt) if case["residual"] else None
    else:
        state["x"] = x.to(xt)
        state["residual"] = (rand(T, D) * channel).to(xt) if case["residual"] else None
    return state


def _stats(h, rms, eps):
    mean = torch.zeros_like(h[:, 0]) if rms else h.mean(1)
    return mean, ((h - mean[:, None]).square().mean(1) + eps).rsqrt()


# -------------------------------------------------------------------------------------------------------- plain forms
def _doc_mask(n, M, window, rows, device):
    """Which of the document's keys the rows see: [rows, n] clean keys, or, with the noisy stream, [rows, 2 n] with the
    noisy keys after the clean ones.  Rows: indices into the clean queries followed by the noisy ones."""
    i = rows % n if M else rows
    j = torch.arange(n, device=device)
    clean_row = (rows < n)[:, None]
    limit = torch.where(rows < n, i + 1, i // M * M if M else i)[:, None]
    clean = j[None] < limit
    if window > 0:
        clean = clean & (i[:, None] - j[None] < window)
    if not M:
        return clean
    return torch.cat([clean, ~clean_row & (i[:, None] // M == j[None] // M)], dim=1)


def _plain_attn(s):
    """Document by document, all heads at once, as many query rows at a time as memory holds scores for."""
    case = s["case"]
    H, H_kv, d, M = case["H"], case["H_kv"], case["d"], case["M"]
    G, scale, step = H // H_kv, 1.0 / math.sqrt(d), case["step"]
    streams = ("clean", "noisy") if M else ("clean",)
    join = lambda name, a, z: torch.cat([s[name + "_" + x][0, a:z].float() for x in streams]).transpose(0, 1)
    parts = {x: [] for x in ("o", "lse", "q", "k", "v")}
    a = 0
    for n in _lens(case):
        q = join("q", a, a + n).unflatten(0, (H_kv, G))                  # [H_kv, G, rows, d]
        k, v = join("k", a, a + n)[:, None], join("v", a, a + n)[:, None]   # [H_kv, 1, keys, d]
        do = join("do", a, a + n).unflatten(0, (H_kv, G)) if step else None
        a += n
        dk, dv = torch.zeros_like(k), torch.zeros_like(v)
        done = {"o": [], "lse": [], "q": []}
        for rows in torch.arange(q.shape[2], device="cuda").split(max(1, (1 << 29) // (H * k.shape[2]))):
            at = slice(int(rows[0]), int(rows[-1]) + 1)
            x = (q[:, :, at] @ k.transpose(2, 3)) * scale
            x = torch.where(_doc_mask(n, M, case["window"], rows, "cuda"), x, torch.full((), -math.inf, device="cuda"))
            top = x.max(dim=3, keepdim=True).values
            p = torch.exp(x - top)
            total = p.sum(dim=3, keepdim=True)
            p = p / total
            o = p @ v
            done["o"].append(o)
            done["lse"].append((top + torch.log(total))[..., 0])
            if step:
                g = do[:, :, at]
                ds = p * (g @ v.transpose(2, 3) - (g * o).sum(dim=3, keepdim=True)) * scale
                done["q"].append(ds @ k)
                dk += (ds.transpose(2, 3) @ q[:, :, at]).sum(dim=1, keepdim=True)
                dv += (p.transpose(2, 3) @ g).sum(dim=1, keepdim=True)
        for x, rows in done.items():
            if rows:
                parts[x].append(torch.cat(rows, dim=2).flatten(0, 1).unflatten(1, (len(streams), n)))   # [H, streams, n, ..]
        parts["k"].append(dk[:, 0].unflatten(1, (len(streams), n)))
        parts["v"].append(dv[:, 0].unflatten(1, (len(streams), n)))
    whole = lambda name, x: torch.cat([t[:, x] for t in parts[name]], dim=1)
    rows = lambda name, x: whole(name, x).transpose(0, 1).bfloat16()[None]
    out = []
    for x in range(len(streams)):
        out += [rows("o", x), whole("lse", x)[None]]
    if step:
        for x in range(len(streams)):
            out += [rows(name, x) for name in ("q", "k", "v")]
    return out


def _plain_embed(s):
    case, ids = s["case"], s["ids"].long()
    real = (ids >= 0) & (ids < case["V"])
    if case["back"]:
        rows = s["dout"].float() * real[:, None]
        grad = torch.zeros(case["V"], case["D"], device="cuda")
        grad.index_add_(0, ids.clamp(0, case["V"] - 1), rows)
        return grad.mul_(s["scale"]).to(DT[case["table"]])
    rows = s["table"][ids.clamp(0, case["V"] - 1)].float() * s["scale"]
    return (rows * real[:, None]).to(DT[case["out"]])


def _plain_norm(s):
    case = s["case"]
    xt, w = DT[case["x"]], s["weight"].float()
    if case["back"]:
        h, dy, rstd = s["h"].float(), s["dy"].float(), s["rstd"][:, None]
        n = (h if case["rms"] else h - s["mean"][:, None]) * rstd
        g = dy * w
        dx = g - n * (g * n).mean(1, keepdim=True)
        if not case["rms"]:
            dx = dx - g.mean(1, keepdim=True)
        dx = dx * rstd
        if case["residual"]:
            dx = dx + s["dh"].float()
        out = [dx.to(xt), (dy * n).sum(0).to(s["weight"].dtype)]
        return out + [dy.sum(0).to(s["weight"].dtype)] if case["bias"] else out
    h = s["x"]
    if case["residual"]:   # the sum is stored as the residual stream stores it, and normalised as stored
        h = (h.float() + s["residual"].float()).to(xt)
    hf = h.float()
    mean, rstd = _stats(hf, case["rms"], s["eps"])
    y = (hf - mean[:, None]) * rstd[:, None] * w
    if case["bias"]:
        y = y + s["bias"].float()
    return [y.to(xt), rstd] + ([h] if case["residual"] else []) + ([] if case["rms"] else [mean])


# --------------------------------------------------------------------------------------------------------- the calls
def _own_attn(s):
    from paper_2609_19242_b200 import binding
    case, M = s["case"], max(1, s["case"]["M"])
    noisy = [s["q_noisy"], s["k_noisy"], s["v_noisy"]] if case["M"] else [None, None, None]
    qkv = [s["q_clean"], s["k_clean"], s["v_clean"]] + noisy
    o_c, l_c, o_n, l_n = binding.bdlm_attn_fwd_packed(*qkv, M, docs=s["docs"], window=case["window"])
    out = [o_c, l_c] + ([o_n, l_n] if case["M"] else [])
    if case["step"]:
        grads = binding.bdlm_attn_bwd_packed(*qkv, o_c, l_c, o_n, l_n, s["do_clean"], s.get("do_noisy"), M, docs=s["docs"],
                                             window=case["window"])
        out += list(grads if case["M"] else grads[:3])
    return out


def run(state):
    case = state["case"]
    if not own:
        return {"attn": _plain_attn, "embed": _plain_embed, "norm": _plain_norm}[case["kind"]](state)
    from paper_2609_19242_b200 import binding
    if case["kind"] == "attn":
        return _own_attn(state)
    if case["kind"] == "embed":
        if case["back"]:
            return binding.bdlm_embed_bwd(state["dout"], state["ids"], case["V"], scale=state["scale"], dtype=DT[case["table"]])
        return binding.bdlm_embed_fwd(state["table"], state["ids"], scale=state["scale"], dtype=DT[case["out"]])
    if case["back"]:
        dx, dw, db = binding.bdlm_norm_bwd(state["dy"], state["h"], state["weight"], state["mean"], state["rstd"],
                                           dh=state["dh"], bias=case["bias"], rms=case["rms"])
        return [dx, dw, db] if case["bias"] else [dx, dw]
    y, h, mean, rstd = binding.bdlm_norm_fwd(state["x"], state["weight"], state["bias"], state["residual"], eps=state["eps"],
                                             rms=case["rms"])
    return [y, rstd] + ([h] if case["residual"] else []) + ([] if case["rms"] else [mean])


# ---------------------------------------------------------------------------------------------------- from the definition
def _exact_attn(case, s):
    """One head at a time: softmax over the visible keys, and the derivative of sum(O dO) by automatic differentiation."""
    M, W, d, G = case["M"], case["window"], case["d"], case["H"] // case["H_kv"]
    streams = ("clean", "noisy") if M else ("clean",)
    wide = {k: t[0].double() for k, t in s.items() if k[:2] in ("q_", "k_", "v_", "do")}
    names = [a + "_" + x for x in streams for a in ("q", "k", "v")]
    out = {("o", x): torch.zeros_like(wide["q_" + x]) for x in streams}
    out.update({("lse", x): torch.zeros(case["H"], wide["q_" + x].shape[0], device="cuda", dtype=torch.float64) for x in streams})
    out.update({("d", a): torch.zeros_like(wide[a]) for a in names})
    first = 0
    for n in _lens(case):
        at = slice(first, first + n)
        pos = torch.arange(n, device="cuda")
        ahead = pos[:, None] - pos[None, :]                         # how far the key lies behind the query
        reach = torch.ones_like(ahead, dtype=torch.bool) if W == 0 else ahead < W
        seen = {("clean", "clean"): (ahead >= 0) & reach}
        if M:
            block = pos // M
            seen["noisy", "clean"] = (block[:, None] > block[None, :]) & reach
            seen["noisy", "noisy"] = block[:, None] == block[None, :]
        for h in range(case["H"]):
            leaf = {}
            for a in names:
                leaf[a] = wide[a][at, h if a[0] == "q" else h // G].detach().clone().requires_grad_(case["step"])
            target = 0.0
            for x in streams:
                sources = [y for y in streams if (x, y) in seen]
                z = torch.cat([(leaf["q_" + x] @ leaf["k_" + y].T).div(d ** 0.5).masked_fill(~seen[x, y], -math.inf)
                               for y in sources], dim=1)
                got = torch.softmax(z, dim=1) @ torch.cat([leaf["v_" + y] for y in sources])
                out["o", x][at, h] = got.detach()
                out["lse", x][h, at] = torch.logsumexp(z.detach(), dim=1)
                if case["step"]:
                    target = target + (got * wide["do_" + x][at, h]).sum()
            if case["step"]:
                for a, g in zip(names, torch.autograd.grad(target, [leaf[a] for a in names])):
                    out["d", a][at, h if a[0] == "q" else h // G] += g
        first += n
    res = []
    for x in streams:
        res += [out["o", x][None], out["lse", x][None]]
    return res + ([out["d", a][None] for a in names] if case["step"] else [])


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attn":
        if 14e-12 * case["d"] * case["H"] * sum(n * n for n in _lens(case)) * (3 if case["M"] else 1) > 60.0:
            return None
        return _exact_attn(case, s)
    if case["kind"] == "embed":
        ids = s["ids"].long()
        at = torch.nonzero((ids >= 0) & (ids < case["V"]))[:, 0]
        if case["back"]:
            grad = torch.zeros(case["V"], case["D"], device="cuda", dtype=torch.float64)
            return grad.index_put_((ids[at],), s["dout"][at].double() * s["scale"], accumulate=True)
        out = torch.zeros(case["T"], case["D"], device="cuda", dtype=torch.float64)
        out[at] = s["table"].double()[ids[at]] * s["scale"]
        return out
    w = s["weight"].double()
    center = (lambda t: t) if case["rms"] else (lambda t: t - t.mean(1, keepdim=True))
    if case["back"]:
        # the statistics are inputs of the backward, given to 32 bits
        h, dy, inv = s["h"].double(), s["dy"].double(), s["rstd"].double()[:, None]
        unit = h * inv if case["rms"] else (h - s["mean"].double()[:, None]) * inv
        inner = dy * w[None]
        dx = (center(inner) - unit * torch.einsum("td,td->t", inner, unit)[:, None] / case["D"]) * inv
        if case["residual"]:
            dx = dx + s["dh"].double()
        res = [dx, torch.einsum("td,td->d", dy, unit)]
        return res + [dy.sum(0)] if case["bias"] else res
    h = s["x"].double()
    if case["residual"]:
        h = (h + s["residual"].double()).to(DT[case["x"]]).double()
    c = center(h)
    inv = 1.0 / torch.sqrt((c * c).sum(1) / case["D"] + s["eps"])
    y = c * inv[:, None] * w
    if case["bias"]:
        y = y + s["bias"].double()
    return [y, inv] + ([h] if case["residual"] else []) + ([] if case["rms"] else [h.sum(1) / case["D"]])
