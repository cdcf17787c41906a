"""The normalisation against its fp64 oracle, through the binding.

Tolerances.  An output of type t is rounded once: eps(t)/2 of its value.  Before that everything is fp32: sums of D terms run
over at most 64 terms in a thread and then pairwise over at most 1024 threads (10 additions), so a sum is off by at most
80 x 2^-24 of the sum of its terms' magnitudes; SLACK = 128 x 2^-24 covers it with the few operations around it (the
reciprocal square root is within 2^-21)."""
import ctypes
import threading

import numpy as np
import pytest
import torch

from oracle import model_ops_oracle as orc
from paper_2609_19242_b200 import binding

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
SLACK = 128 * 2.0 ** -24


def _f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _half_ulp(t):
    return torch.finfo(t).eps / 2


def _inputs(T, D, x, w, seed=0, shift=0.3):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    channel = 0.5 + r(D).abs() + 10.0 * (torch.rand(D, generator=g) < 0.02)
    mk = lambda t, dt: t.to(dt).cuda()
    return {"x": mk(r(T, D) * channel + shift, x), "res": mk(r(T, D) * channel, x), "w": mk(1 + 0.2 * r(D), w), "b": mk(0.1 * r(D), w),
            "dy": mk(r(T, D), x), "dh": mk(r(T, D), x)}


def _check_forward(i, out, h, rms, eps, weight, bias, dt):
    y, _, mean, rstd = out
    h64, w64 = _f64(h), _f64(weight)
    ref, m64, r64 = orc.norm_forward(h64, w64, _f64(bias), rms, eps)
    size = np.abs(h64).mean(axis=1)
    n = (h64 - m64[:, None]) * r64[:, None]
    aw = 1.0 if weight is None else np.abs(w64)
    # the mean's error moves n by rstd x size, the statistics' relative errors scale it
    off = SLACK * aw * ((r64 * size)[:, None] + 2 * np.abs(n)) + (0 if bias is None else 2.0 ** -24 * np.abs(_f64(bias)))
    assert (np.abs(_f64(y) - ref) <= _half_ulp(dt) * (np.abs(ref) + off) + off).all()
    assert (np.abs(_f64(rstd) - r64) <= (SLACK + 2.0 ** -21) * r64 + SLACK * r64 ** 2 * size).all()
    if rms:
        assert mean is None
    else:
        assert (np.abs(_f64(mean) - m64) <= SLACK * size).all()


def _check_backward(grads, i, h, mean, rstd, weight, dh, bias, rms, dt, wt):
    dx, dw, db = grads
    args = [_f64(t) for t in (i["dy"], h, weight)]
    rx, rw, rb = orc.norm_backward(*args, _f64(mean), _f64(rstd), _f64(dh), rms)
    dy, h64, w64 = args
    r = _f64(rstd)[:, None]
    # h - mean cancels: its error is half an ulp of the larger of the two
    near = np.abs(h64) if rms else np.abs(h64) + np.abs(_f64(mean))[:, None]
    n = (h64 - (0 if rms else _f64(mean)[:, None])) * r
    dn = 2.0 ** -23 * near * r + 2.0 ** -23 * np.abs(n)
    g = dy if weight is None else dy * w64
    mg, mgn = np.abs(g).mean(axis=1, keepdims=True), np.abs(g * n).mean(axis=1, keepdims=True)
    mgd = (np.abs(g) * dn).mean(axis=1, keepdims=True)
    off = r * (SLACK * (np.abs(g) + mg + np.abs(n) * mgn) + dn * mgn + np.abs(n) * mgd) + (0 if dh is None else 2.0 ** -23 * np.abs(_f64(dh)))
    assert (np.abs(_f64(dx) - rx) <= _half_ulp(dt) * (np.abs(rx) + off) + off).all()
    T = h64.shape[0]
    # over the rows: one after the other in a CTA, the CTAs' sums in 16 shares one after the other
    chain = (T / 148 + 150) * 2.0 ** -24
    if weight is not None:
        ow = chain * np.abs(dy * n).sum(axis=0) + (np.abs(dy) * dn).sum(axis=0)
        assert (np.abs(_f64(dw) - rw) <= _half_ulp(wt) * (np.abs(rw) + ow) + ow).all()
    else:
        assert dw is None
    if bias and weight is not None:
        ob = chain * np.abs(dy).sum(axis=0)
        assert (np.abs(_f64(db) - rb) <= _half_ulp(wt) * (np.abs(rb) + ob) + ob).all()
    else:
        assert db is None


def _both(T, D, x=BF16, w=BF16, rms=False, affine=True, bias=True, residual=True, seed=0, eps=1e-5, shift=0.3):
    i = _inputs(T, D, x, w, seed, shift)
    weight, b = (i["w"], i["b"] if bias else None) if affine else (None, None)
    res, dh = (i["res"], i["dh"]) if residual else (None, None)
    out = binding.bdlm_norm_fwd(i["x"], weight, b, res, eps=eps, rms=rms)
    h = out[1]
    if residual:   # one fp32 addition, rounded once
        assert torch.equal(h, (i["x"].float() + res.float()).to(x))
    else:
        assert h is i["x"]
    grads = binding.bdlm_norm_bwd(i["dy"], h, weight, out[2], out[3], dh=dh, bias=bias, rms=rms)
    torch.cuda.synchronize()
    _check_forward(i, out, h, rms, eps, weight, b, x)
    _check_backward(grads, i, h, out[2], out[3], weight, dh, bias, rms, x, w)
    return out, grads


# rows of part of a warp, of a warp, of a CTA; vectors and single elements; every items-per-thread variant and its borders
@pytest.mark.parametrize("D", [1, 2, 7, 8, 24, 31, 64, 100, 127, 129, 256, 264, 512, 520, 1000, 1001, 1024, 1032, 1544, 2047, 2049, 4096,
                               4104, 8192, 8200, 8191, 16383, 16384, 16385, 20000, 32767, 32768])
def test_lengths_of_rows(D):
    _both(5, D)
    _both(3, D, FP32, FP32, rms=True)


@pytest.mark.parametrize("T", [1, 2, 3, 127, 300, 1531])
@pytest.mark.parametrize("D", [40, 333, 1544])
def test_numbers_of_rows(T, D):
    _both(T, D)


@pytest.mark.parametrize("D", [1, 9, 40, 100, 257, 300, 999, 1000, 2056, 4097, 8192])
def test_calls_of_one_cta_and_just_beyond(D):
    """The smallest backward calls form their sums in one CTA, in rows of whole periods; both sides of the rule, every period."""
    for T in sorted({1, 2, 3, 5, 7, 8, 13, max(1, 32768 // D), 32768 // D + 1}):
        if T <= 400:
            _both(T, D)


def test_more_rows_than_ctas_and_prefetched_rows():
    _both(3001, 4096, residual=True)
    _both(40001, 16, rms=True)
    _both(2999, 1001)


@pytest.mark.parametrize("x,w", [(BF16, BF16), (BF16, FP32), (FP16, FP16), (FP16, FP32), (FP32, FP32)])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("D", [37, 96, 1536, 5000, 16384])
def test_types(x, w, rms, D):
    _both(17, D, x, w, rms=rms)


@pytest.mark.parametrize("affine,bias,residual", [(False, False, False), (False, False, True), (True, False, False), (True, True, False),
                                                  (True, False, True)])
@pytest.mark.parametrize("D", [48, 2000, 12000])
def test_optional_operands(affine, bias, residual, D):
    for rms in (False, True):
        _both(9, D, affine=affine, bias=bias, residual=residual, rms=rms)


def test_mean_far_from_zero_and_constant_rows():
    """The variance is summed around the mean: a mean a thousand times the deviation costs nothing."""
    _both(33, 4096, FP32, FP32, shift=1000.0, residual=False)
    x = torch.full((3, 1544), 2.5, device="cuda", dtype=BF16)
    w, b = torch.ones(1544, device="cuda", dtype=BF16), torch.full((1544,), 0.25, device="cuda", dtype=BF16)
    y, _, mean, rstd = binding.bdlm_norm_fwd(x, w, b, eps=1e-4)
    assert (y == 0.25).all() and (mean == 2.5).all()
    assert (rstd - 100).abs().max() < 1e-3


def test_more_elements_than_32_bits_count():
    """2^31 elements lie before the last rows: those are the same as in a call of their own."""
    T, D, tail = 524288 + 300, 4096, 400
    x = torch.empty(T, D, device="cuda", dtype=BF16)
    i = _inputs(tail, D, BF16, BF16)
    x[:-tail] = 1.0
    x[-tail:] = i["x"]
    out = binding.bdlm_norm_fwd(x, i["w"], i["b"])
    want = binding.bdlm_norm_fwd(i["x"], i["w"], i["b"])
    for a, b in ((out[0], want[0]), (out[2], want[2]), (out[3], want[3])):
        assert torch.equal(a[-tail:], b)
    del out
    mean, rstd = torch.cat([torch.zeros(T - tail, device="cuda"), want[2]]), torch.cat([torch.ones(T - tail, device="cuda"), want[3]])
    dy = torch.zeros_like(x)
    dy[-tail:] = i["dy"]
    got = binding.bdlm_norm_bwd(dy, x, i["w"], mean, rstd, bias=True)
    ref = binding.bdlm_norm_bwd(i["dy"], i["x"], i["w"], want[2], want[3], bias=True)
    assert torch.equal(got[0][-tail:], ref[0]) and (got[0][:-tail] == 0).all()
    # the same sums in another order of rows
    for a, b, size in ((got[1], ref[1], (i["dy"].float() * (i["x"].float() - want[2][:, None]) * want[3][:, None]).abs().sum(0)),
                       (got[2], ref[2], i["dy"].float().abs().sum(0))):
        assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 2 * tail * 2.0 ** -24 * size).all()


def test_no_rows():
    x = torch.empty(0, 64, device="cuda", dtype=BF16)
    w = torch.ones(64, device="cuda", dtype=BF16)
    y, h, mean, rstd = binding.bdlm_norm_fwd(x, w)
    assert y.shape == (0, 64) and mean.shape == (0,)
    dw, db = torch.full((64,), 7.0, device="cuda", dtype=BF16), torch.full((64,), 7.0, device="cuda", dtype=BF16)
    binding.bdlm_norm_bwd(x, x, w, mean, rstd, bias=True, out=(torch.empty_like(x), dw, db))
    assert (dw == 0).all() and (db == 0).all()


def test_not_a_number_stays_in_its_row():
    i = _inputs(6, 1000, BF16, BF16)
    clean = binding.bdlm_norm_fwd(i["x"], i["w"], i["b"])
    bad = i["x"].clone()
    bad[2, 5], bad[4, 999] = float("nan"), float("inf")
    y, _, mean, rstd = binding.bdlm_norm_fwd(bad, i["w"], i["b"])
    keep = [0, 1, 3, 5]
    assert torch.equal(y[keep], clean[0][keep]) and y[2].isnan().all() and y[4].isnan().any()
    grads = binding.bdlm_norm_bwd(i["dy"], bad, i["w"], mean, rstd, bias=True)
    good = binding.bdlm_norm_bwd(i["dy"], i["x"], i["w"], clean[2], clean[3], bias=True)
    assert torch.equal(grads[0][keep], good[0][keep]) and grads[0][2].isnan().all() and grads[1].isnan().all()
    assert torch.equal(grads[2], good[2])


def test_rows_do_not_depend_on_each_other_and_calls_repeat_bit_for_bit():
    i = _inputs(700, 1544, BF16, BF16)
    a = binding.bdlm_norm_fwd(i["x"], i["w"], i["b"], i["res"])
    b = binding.bdlm_norm_fwd(i["x"][100:200].contiguous(), i["w"], i["b"], i["res"][100:200].contiguous())
    for x, y in zip(a, b):
        assert torch.equal(x[100:200], y)
    ga = binding.bdlm_norm_bwd(i["dy"], a[1], i["w"], a[2], a[3], dh=i["dh"], bias=True)
    gb = binding.bdlm_norm_bwd(i["dy"], a[1], i["w"], a[2], a[3], dh=i["dh"], bias=True)
    for x, y in zip(ga, gb):
        assert torch.equal(x, y)
    part = [t[100:200].contiguous() for t in (i["dy"], a[1], a[2], a[3], i["dh"])]
    gc = binding.bdlm_norm_bwd(part[0], part[1], i["w"], part[2], part[3], dh=part[4], bias=True)
    assert torch.equal(gc[0], ga[0][100:200])


@pytest.mark.parametrize("D", [96, 1544, 1001, 12000])
def test_outputs_over_inputs(D):
    i = _inputs(50, D, BF16, BF16)
    y, h, mean, rstd = binding.bdlm_norm_fwd(i["x"], i["w"], i["b"], i["res"])
    x, res = i["x"].clone(), i["res"].clone()
    binding.bdlm_norm_fwd(x, i["w"], i["b"], res, out=(x, res, torch.empty_like(mean), torch.empty_like(rstd)))
    assert torch.equal(x, y) and torch.equal(res, h)
    want = binding.bdlm_norm_bwd(i["dy"], h, i["w"], mean, rstd, dh=i["dh"])
    for target in ("dy", "dh", "h"):
        t = {"dy": i["dy"].clone(), "dh": i["dh"].clone(), "h": h.clone()}
        got = binding.bdlm_norm_bwd(t["dy"], t["h"], i["w"], mean, rstd, dh=t["dh"], out=(t[target], torch.empty_like(i["w"]), None))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_gradients_agree_with_differences():
    """dx, dweight and dbias of sum(y dy) against central differences of the library's own forward in fp32."""
    T, D, step = 4, 33, 1e-2
    i = _inputs(T, D, FP32, FP32, shift=0.0)
    x = i["x"] / i["x"].std()
    f = lambda x, w, b: float((binding.bdlm_norm_fwd(x, w, b)[0].double() * i["dy"].double()).sum())
    _, _, mean, rstd = binding.bdlm_norm_fwd(x, i["w"], i["b"])
    grads = binding.bdlm_norm_bwd(i["dy"], x, i["w"], mean, rstd, bias=True)
    for which, base in enumerate((x, i["w"], i["b"])):
        for at in ((0, 0), (3, 32), (1, 17)):
            at = at if which == 0 else at[1:]
            up, down = base.clone(), base.clone()
            up[at] += step
            down[at] -= step
            args = [x, i["w"], i["b"]]
            fu = f(*(up if k == which else t for k, t in enumerate(args)))
            fd = f(*(down if k == which else t for k, t in enumerate(args)))
            # the forward is off by about 2^-22 of sum |y dy| (~ 300), twice, over 2 steps; the third derivative times step^2 / 6
            assert abs((fu - fd) / (2 * step) - float(grads[which][at])) < 300 * 2.0 ** -22 / step + 5e-3


def test_under_capture_and_on_another_stream():
    i = _inputs(300, 1544, BF16, BF16)
    run = lambda: (binding.bdlm_norm_fwd(i["x"], i["w"], i["b"], i["res"]),)
    out, = run()
    step = lambda: binding.bdlm_norm_bwd(i["dy"], out[1], i["w"], out[2], out[3], dh=i["dh"], bias=True)
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fwd = binding.bdlm_norm_fwd(i["x"], i["w"], i["b"], i["res"])
        bwd = binding.bdlm_norm_bwd(i["dy"], fwd[1], i["w"], fwd[2], fwd[3], dh=i["dh"], bias=True)
    for t in (*fwd, *bwd):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip((*fwd, *bwd), (*out, *want)):
        assert torch.equal(a, b)


def test_untrained_weight_needs_no_workspace():
    i = _inputs(20, 200, BF16, BF16)
    out = binding.bdlm_norm_fwd(i["x"], i["w"], i["b"])
    want = binding.bdlm_norm_bwd(i["dy"], i["x"], i["w"], out[2], out[3], bias=True)
    dx, dw, db = binding.bdlm_norm_bwd(i["dy"], i["x"], i["w"], out[2], out[3], out=(torch.empty_like(i["x"]), None, None))
    assert dw is None and db is None and torch.equal(dx, want[0])
    got = binding.bdlm_norm_bwd(i["dy"], i["x"], i["w"], out[2], out[3], out=(torch.empty_like(i["x"]), None, torch.empty_like(i["b"])))
    assert torch.equal(got[2], want[2])


def test_refusals():
    i = _inputs(4, 64, BF16, BF16)
    with pytest.raises(ValueError):
        binding.bdlm_norm_fwd(i["x"], i["w"].float()[:32].contiguous())
    with pytest.raises(ValueError):
        binding.bdlm_norm_fwd(i["x"], i["w"], i["b"].float())
    with pytest.raises(ValueError):
        binding.bdlm_norm_fwd(i["x"], i["w"], residual=i["res"].float())
    with pytest.raises(binding.BdlmError):
        binding.bdlm_norm_fwd(i["x"], i["w"].half())
    with pytest.raises(binding.BdlmError):
        binding.bdlm_norm_fwd(i["x"], None, i["b"])
    with pytest.raises(AssertionError):
        binding.bdlm_norm_fwd(i["x"][:, ::2], i["w"][::2].contiguous())
    big = torch.zeros(1, 32776, device="cuda", dtype=BF16)
    with pytest.raises(binding.BdlmError) as e:
        binding.bdlm_norm_fwd(big)
    assert e.value.status == -2
    many = _inputs(1000, 64, BF16, BF16)
    out = binding.bdlm_norm_fwd(many["x"], many["w"])
    with pytest.raises(binding.BdlmError) as e:
        binding.bdlm_norm_bwd(many["dy"], many["x"], many["w"], out[2], out[3], workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -3
    out = binding.bdlm_norm_fwd(i["x"], i["w"])
    with pytest.raises(binding.BdlmError):
        binding.bdlm_norm_bwd(i["dy"], i["x"], i["w"], None, out[3])


@pytest.mark.parametrize("rms", [False, True])
def test_supplied_outputs_without_a_residual_return_x_as_h(rms):
    i = _inputs(5, 72, BF16, BF16)
    want = binding.bdlm_norm_fwd(i["x"], i["w"], rms=rms)
    buffer = torch.full_like(i["x"], 7.0)
    stats = lambda: torch.empty(5, dtype=FP32, device="cuda")
    got = binding.bdlm_norm_fwd(i["x"], i["w"], rms=rms, out=(torch.empty_like(i["x"]), buffer, None if rms else stats(), stats()))
    assert got[1] is i["x"] and (buffer == 7.0).all()
    for a, b in zip(got, want):
        assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("T, D, dt", [(1531, 16384, BF16), (700, 9000, FP16), (333, 32768, BF16), (300, 16383, BF16), (400, 16384, FP32)])
def test_clusters_give_the_same_bits_every_time(T, D, dt):
    """Rows that a cluster shares: the sums that its CTAs read from one another are complete and of the right row."""
    i = _inputs(T, D, dt, dt)
    first = None
    for _ in range(25):
        y, h, mean, rstd = binding.bdlm_norm_fwd(i["x"], i["w"], i["b"], i["res"])
        got = (y, h, mean, rstd) + binding.bdlm_norm_bwd(i["dy"], h, i["w"], mean, rstd, dh=i["dh"], bias=True)
        first = got if first is None else first
        assert all(torch.equal(a, b) for a, b in zip(got, first))
    _check_backward(first[4:], i, first[1], first[2], first[3], i["w"], i["dh"], True, False, dt, dt)


FAR = [(1, 100, FP32), (300, 100, FP32), (300, 333, FP32), (1, 4096, FP32), (300, 1544, FP32), (300, 4096, FP32), (300, 4095, FP32),
       (300, 16384, FP32), (300, 16383, FP32), (300, 100, BF16), (300, 4096, BF16), (300, 4095, FP16), (300, 12000, BF16), (300, 16383, FP16)]


def _far(T, D, dt):
    """Rows whose mean is a thousand times their deviation (16-bit rows, which hold no more: a hundred times)."""
    g = torch.Generator().manual_seed(T + D)
    x = (torch.randn(T, D, generator=g) + (1000.0 if dt == FP32 else 100.0)).to(dt).cuda()
    w = (1 + 0.2 * torch.randn(D, generator=g)).cuda()
    _, _, mean, rstd = binding.bdlm_norm_fwd(x, w)
    n = (_f64(x) - _f64(mean)[:, None]) * _f64(rstd)[:, None]
    return x, w, mean, rstd, n, g


@pytest.mark.parametrize("T, D, dt", FAR)
def test_normalised_values_of_the_backward_far_from_a_zero_mean(T, D, dt):
    """n = (h - mean) rstd is formed as it stands: a subtraction and a product, each off by half a step (2^-24 of the value), however
    far the mean lies from zero.  With a gradient of ones in one row alone dweight is that row's n: all else that is added to it is zero."""
    x, w, mean, rstd, n, _ = _far(T, D, dt)
    for row in sorted({0, T // 2, T - 1}):
        dy = torch.zeros_like(x)
        dy[row] = 1.0
        _, dw, db = binding.bdlm_norm_bwd(dy, x, w, mean, rstd, bias=True)
        assert (db == 1.0).all()
        assert (np.abs(_f64(dw) - n[row]) <= 2.0 ** -23 * np.abs(n[row]) + 1e-30).all()


@pytest.mark.parametrize("T, D, dt", FAR)
def test_gradient_of_rows_far_from_a_zero_mean(T, D, dt):
    """The sums' errors are those of the head of this file, n's those of the test above."""
    x, w, mean, rstd, n, gen = _far(T, D, dt)
    dy = (0.5 + torch.rand(T, D, generator=gen)).to(dt).cuda()
    dx, dw, _ = binding.bdlm_norm_bwd(dy, x, w, mean, rstd)
    rx, rw, _ = orc.norm_backward(_f64(dy), _f64(x), _f64(w), _f64(mean), _f64(rstd), None, False)
    r, g, dn = _f64(rstd)[:, None], _f64(dy) * _f64(w), 2.0 ** -23 * np.abs(n)
    mean_of = lambda t: t.mean(axis=1, keepdims=True)
    off = r * (SLACK * (np.abs(g) + mean_of(np.abs(g)) + np.abs(n) * mean_of(np.abs(g * n))) + dn * mean_of(np.abs(g * n)) +
               np.abs(n) * mean_of(np.abs(g) * dn))
    assert (np.abs(_f64(dx) - rx) <= _half_ulp(dt) * (np.abs(rx) + off) + off).all()
    ow = (T / 148 + 150) * 2.0 ** -24 * np.abs(_f64(dy) * n).sum(axis=0) + (np.abs(_f64(dy)) * dn).sum(axis=0)
    assert (np.abs(_f64(dw) - rw) <= ow).all()


def test_host_threads_with_calls_of_one_kernel_and_different_sizes():
    """The backward's shared memory follows from the call's rows.  Four threads, each with a stream of its own and its arguments ready, call
    the same kernel with little of it and with much."""
    jobs = []
    for T, D in ((148, 1032), (300, 4096)) * 2:
        i = _inputs(T, D, BF16, BF16)
        _, _, mean, rstd = binding.bdlm_norm_fwd(i["x"], i["w"], i["b"])
        want = binding.bdlm_norm_bwd(i["dy"], i["x"], i["w"], mean, rstd, bias=True)
        out = tuple(torch.empty_like(t) for t in want)
        p = binding.make_norm_params(T, D, BF16, BF16)
        ws = torch.empty(binding.bdlm_norm_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        stream = torch.cuda.Stream()
        args = [ctypes.byref(p)] + [ctypes.c_void_p(t.data_ptr()) for t in (i["dy"], i["x"], i["w"], mean, rstd)] + [None]
        args += [ctypes.c_void_p(t.data_ptr()) for t in (*out, ws)] + [ctypes.c_size_t(ws.numel()), ctypes.c_void_p(stream.cuda_stream)]
        jobs.append((args, out, want, (i, mean, rstd, p, ws, stream)))
    torch.cuda.synchronize()
    bwd, failed, start = binding.lib().bdlm_norm_bwd, [], threading.Barrier(len(jobs))

    def work(args):
        start.wait()
        for _ in range(20000):
            rc = bwd(*args)
            if rc != 0:
                failed.append(rc)
                return
    threads = [threading.Thread(target=work, args=(j[0],)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for _, out, want, _ in jobs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("D", [1, 9, 40])
def test_short_rows_of_the_largest_calls_of_one_cta(D):
    """As many rows as one CTA takes, and one more: up to 512 rows at once, each thread's summed over up to 64 rounds, so at most 576
    additions one after the other (beyond the limit fewer: a CTA has T / 148 rows and 148 CTAs' sums are added in 16 shares)."""
    for T in (32768 // D, 32768 // D + 1):
        i = _inputs(T, D, BF16, FP32)
        _, h, mean, rstd = binding.bdlm_norm_fwd(i["x"], i["w"], i["b"], i["res"])
        dx, dw, db = binding.bdlm_norm_bwd(i["dy"], h, i["w"], mean, rstd, dh=i["dh"], bias=True)
        rx, rw, rb = orc.norm_backward(_f64(i["dy"]), _f64(h), _f64(i["w"]), _f64(mean), _f64(rstd), _f64(i["dh"]), False)
        n = (_f64(h) - _f64(mean)[:, None]) * _f64(rstd)[:, None]
        dy, chain = np.abs(_f64(i["dy"])), 576 * 2.0 ** -24
        assert (np.abs(_f64(dw) - rw) <= (chain + 2.0 ** -23) * (dy * np.abs(n)).sum(axis=0)).all()
        assert (np.abs(_f64(db) - rb) <= chain * dy.sum(axis=0)).all()
        part = binding.bdlm_norm_bwd(i["dy"][:64], h[:64], i["w"], mean[:64], rstd[:64], dh=i["dh"][:64])
        assert torch.equal(part[0], dx[:64])
