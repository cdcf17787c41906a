"""The operators together, as a training step of a block-diffusion model uses them: embedding of clean and noisy tokens, norm,
attention over packed documents, norm with the residual, loss head over a tied table, and the way back, against the same
model in fp64 with automatic differentiation.

Tolerance.  Everything between the operators is stored in bf16, each time off by at most 2^-8 of the value (half a step).  A
gradient passes at most 16 such roundings (forward: embedding, norm, projection, attention's P and output, projection,
residual sum, norm; backward: dz, dH, norm, projection, attention's dS and gradients, projection, norm, table), and no
stage of this model enlarges relative errors in the 2-norm: 16 x 2^-8."""
import math

import numpy as np
import pytest
import torch

from paper_2609_19242_b200 import binding

pytestmark = pytest.mark.gpu

TOL = 16 * 2.0 ** -8
LENS, M, H, HKV, DH, D, V = [48, 16, 160, 32, 128], 16, 4, 2, 64, 264, 520
T, EPS, SCALE = sum(LENS), 1e-5, 0.75
MASK_TOKEN = V - 1


def _setup():
    g = torch.Generator().manual_seed(7)
    r = lambda *s: torch.randn(*s, generator=g)
    par = {"table": 0.7 * r(V, D), "w0": 1 + 0.1 * r(D), "qkv": r(D, (H + 2 * HKV) * DH) / D ** 0.5, "proj": r(H * DH, D) / (H * DH) ** 0.5,
           "w1": 1 + 0.1 * r(D), "b1": 0.1 * r(D)}
    par = {k: v.bfloat16().cuda() for k, v in par.items()}
    clean = torch.randint(0, V - 1, (T,), generator=g)
    masked = torch.rand(T, generator=g) < 0.5
    noisy = torch.where(masked, torch.full_like(clean, MASK_TOKEN), clean)
    labels = torch.where(masked, clean, torch.full_like(clean, -1))
    weight = torch.rand(T, generator=g) / T
    return par, torch.cat([clean, noisy]).int().cuda(), labels.int().cuda(), weight.cuda()


def _heads(qkv, rows):
    t = qkv[rows]
    q, k, v = t.split([H * DH, HKV * DH, HKV * DH], dim=1)
    return [x.reshape(1, T, -1, DH).contiguous() for x in (q, k, v)]


def _step(par, ids, labels, weight, docs):
    """Forward and backward with the library; returns the loss and the parameters' gradients."""
    c, n = slice(0, T), slice(T, 2 * T)
    x0 = binding.bdlm_embed_fwd(par["table"], ids, scale=SCALE)
    y0, _, _, rstd0 = binding.bdlm_norm_fwd(x0, par["w0"], eps=EPS, rms=True)
    qkv = y0 @ par["qkv"]
    streams = _heads(qkv, c) + _heads(qkv, n)
    o_c, l_c, o_n, l_n = binding.bdlm_attn_fwd_packed(*streams, M, docs=docs)
    o = torch.cat([o_c.view(T, -1), o_n.view(T, -1)])
    a = o @ par["proj"]
    y1, h1, mean1, rstd1 = binding.bdlm_norm_fwd(a, par["w1"], par["b1"], x0, eps=EPS)
    top = y1[n].contiguous()
    loss, _, lse = binding.bdlm_linear_ce_fwd(top, par["table"], labels, weight)
    dtop, dtable = binding.bdlm_linear_ce_bwd(top, par["table"], labels, lse, weight)
    dy1 = torch.cat([torch.zeros_like(dtop), dtop])
    dx1, dw1, db1 = binding.bdlm_norm_bwd(dy1, h1, par["w1"], mean1, rstd1, bias=True)
    do = dx1 @ par["proj"].T
    dproj = o.T @ dx1
    grads = binding.bdlm_attn_bwd_packed(*streams, o_c, l_c, o_n, l_n, do[c].reshape(1, T, H, DH).contiguous(),
                                         do[n].reshape(1, T, H, DH).contiguous(), M, docs=docs)
    flat = lambda t: torch.cat([x.view(T, -1) for x in t], dim=1)
    dqkv = torch.cat([flat(grads[:3]), flat(grads[3:])])
    dy0 = dqkv @ par["qkv"].T
    dx0, dw0, _ = binding.bdlm_norm_bwd(dy0.contiguous(), x0, par["w0"], None, rstd0, dh=dx1, rms=True)
    binding.bdlm_embed_bwd(dx0, ids, V, scale=SCALE, out=dtable, accumulate=True)   # the table is the head's too
    return loss, {"table": dtable, "w0": dw0, "qkv": y0.T @ dqkv, "proj": dproj, "w1": dw1, "b1": db1}


def _reference(par, ids, labels, weight):
    p = {k: v.double().cpu().requires_grad_(True) for k, v in par.items()}
    ids, labels, weight = ids.cpu().long(), labels.cpu().long(), weight.double().cpu()
    x0 = p["table"][ids] * SCALE
    y0 = x0 / (x0.square().mean(1, keepdim=True) + EPS).sqrt() * p["w0"]
    qkv = y0 @ p["qkv"]
    q, k, v = [t.reshape(2 * T, -1, DH) for t in qkv.split([H * DH, HKV * DH, HKV * DH], dim=1)]
    k, v = k.repeat_interleave(H // HKV, 1), v.repeat_interleave(H // HKV, 1)
    doc = torch.repeat_interleave(torch.arange(len(LENS)), torch.tensor(LENS))
    pos = torch.arange(T)
    same = doc[:, None] == doc[None]
    block = pos // M
    see = torch.zeros(2 * T, 2 * T, dtype=torch.bool)
    see[:T, :T] = same & (pos[:, None] >= pos[None])
    see[T:, :T] = same & (block[:, None] > block[None])
    see[T:, T:] = block[:, None] == block[None]
    z = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(DH)
    a = torch.einsum("hij,jhd->ihd", torch.softmax(z.masked_fill(~see, -math.inf), dim=2), v).reshape(2 * T, -1) @ p["proj"]
    y1 = torch.nn.functional.layer_norm(a + x0, (D,), p["w1"], p["b1"], EPS)
    logits = y1[T:] @ p["table"].T
    nll = torch.nn.functional.cross_entropy(logits, labels.clamp(min=0), reduction="none") * (labels >= 0)
    loss = (nll * weight).sum()
    loss.backward()
    return loss.detach(), {k: v.grad for k, v in p.items()}


def _compare(got, want):
    for name, w in want.items():
        err = float((got[name].double().cpu() - w).norm() / w.norm())
        assert err <= TOL, (name, err)


def test_training_step_matches_fp64():
    par, ids, labels, weight = _setup()
    docs = binding.bdlm_doc_table([0] + list(np.cumsum(LENS)))
    loss, grads = _step(par, ids, labels, weight, docs)
    torch.cuda.synchronize()
    assert binding.bdlm_get_device_status() == 0
    ref_loss, ref = _reference(par, ids, labels, weight)
    assert abs(float(loss) - float(ref_loss)) <= TOL * float(ref_loss)
    _compare(grads, ref)


def test_training_step_captured_and_replayed_on_other_tokens():
    """One graph holds the whole step; other tokens of the same documents go through it by copying them in."""
    par, ids, labels, weight = _setup()
    docs = binding.bdlm_doc_table([0] + list(np.cumsum(LENS)))
    _step(par, ids, labels, weight, docs)   # the products' library sets itself up outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, grads = _step(par, ids, labels, weight, docs)
    ids.copy_(torch.where(ids == MASK_TOKEN, ids, (ids * 7 + 3) % (V - 1)))
    labels.copy_(torch.where(labels < 0, labels, (labels * 7 + 3) % (V - 1)))
    graph.replay()
    torch.cuda.synchronize()
    assert binding.bdlm_get_device_status() == 0
    ref_loss, ref = _reference(par, ids, labels, weight)
    assert abs(float(loss) - float(ref_loss)) <= TOL * float(ref_loss)
    _compare(grads, ref)
