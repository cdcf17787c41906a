"""What values that a row does not see may do to it: nothing, as long as they are finite in the forward, and as long as the products that the
backward forms with them are.  The kernels compute whole tiles, the hidden elements among them, and set P to zero there; in
the backward zero times a product that overflows fp32 would be NaN.

Each call is run twice, once with ordinary values and once with large ones in the places that the compared rows do not see; the
results have to be the same bits.  Forward: +-3e38 (bf16's largest are 3.39e38).  Backward: v and dO +-1e18, so that a dot product of
two such rows of 128 elements is at most 1.28e38, and the difference of two of them still finite; q and k +-1e3, so that the other
rows' own o and lse, which are inputs of the backward, are finite.  dQ of the fused kernel alone is
added up in an order of its own each time: fp32 sums of a few partial products, rounded once to bf16, so within one step (2^-7 of
the value) and 1e-4 of the largest one, which leaves room for a hundredfold cancellation in those sums."""
import pytest
import torch

from paper_2609_19242_b200 import binding

pytestmark = pytest.mark.gpu

AUTO, PORTABLE = binding.IMPL_AUTO, binding.IMPL_PORTABLE
PATHS = [(AUTO, True), (AUTO, False), (PORTABLE, False)]
CLEAN = ("q_clean", "k_clean", "v_clean", "do_clean")
NOISY = ("q_noisy", "k_noisy", "v_noisy", "do_noisy")


def _tensors(L, Ln, H, Hkv, d, batch=1, seed=0):
    g = torch.Generator().manual_seed(seed)
    mk = lambda rows, heads: torch.randn(batch, rows, heads, d, generator=g).to(torch.bfloat16).cuda() if rows else None
    return {n: mk(Ln if n.endswith("noisy") else L, Hkv if n[0] in "kv" else H) for n in CLEAN + NOISY}


def _large(t, names, rows, sizes):
    """sizes: of q and k, of v and dO."""
    out = dict(t)
    g = torch.Generator().manual_seed(99)
    for n in names:
        out[n] = t[n].clone()
        part, size = out[n][:, rows], sizes[n[0] not in "qk"]
        out[n][:, rows] = torch.where(torch.rand(part.shape, generator=g).cuda() < 0.5, size, -size).to(torch.bfloat16)
    return out


def _same(got, want, fused_dq):
    if not fused_dq:
        assert torch.equal(got, want)
        return
    a, b = got.float(), want.float()
    assert torch.isfinite(a).all() and ((a - b).abs() <= 2.0 ** -7 * b.abs() + 1e-4 * b.abs().max()).all()


def _packed(t, M, docs, impl, single):
    qkv = [t[n] for n in ("q_clean", "k_clean", "v_clean", "q_noisy", "k_noisy", "v_noisy")]
    out = binding.bdlm_attn_fwd_packed(*qkv, M, docs=docs, impl=impl)
    grads = binding.bdlm_attn_bwd_packed(*qkv, *out, t["do_clean"], t["do_noisy"], M, docs=docs, impl=impl, single_pass=single)
    torch.cuda.synchronize()
    assert binding.bdlm_get_device_status() == 0
    return out, grads


def _compare(got, want, mine, noisy, single):
    (o, lse, on, lsen), grads = got
    (wo, wlse, won, wlsen), wgrads = want
    _same(o[:, mine], wo[:, mine], False)
    _same(lse[:, :, mine], wlse[:, :, mine], False)
    for i in range(3):
        _same(grads[i][:, mine], wgrads[i][:, mine], single and i == 0)
    if noisy:
        _same(on[:, mine], won[:, mine], False)
        _same(lsen[:, :, mine], wlsen[:, :, mine], False)
        for i in range(3, 6):
            _same(grads[i][:, mine], wgrads[i][:, mine], single and i == 3)


def _forward(t, M, docs, impl):
    qkv = [t[n] for n in ("q_clean", "k_clean", "v_clean", "q_noisy", "k_noisy", "v_noisy")]
    out = binding.bdlm_attn_fwd_packed(*qkv, M, docs=docs, impl=impl)
    torch.cuda.synchronize()
    return out


def _outside(t, names, L, mine, sizes):
    for others in (slice(0, mine.start), slice(mine.stop, L)):
        t = _large(t, names, others, sizes)
    return t


@pytest.mark.parametrize("impl", [AUTO, PORTABLE])
@pytest.mark.parametrize("d", [64, 128])
def test_forward_beside_the_largest_values(d, impl):
    for M, names, mine in ((1, CLEAN, slice(150, 330)), (32, CLEAN + NOISY, slice(96, 384))):
        t = _tensors(576, 576 if M > 1 else 0, 4, 2, d)
        docs = binding.bdlm_doc_table([0, mine.start, mine.stop, 576])
        want, got = _forward(t, M, docs, impl), _forward(_outside(t, names, 576, mine, (3e38, 3e38)), M, docs, impl)
        for a, b in zip(got, want):
            if b is not None:
                at = (slice(None), mine) if b.dim() == 4 else (slice(None), slice(None), mine)
                assert torch.equal(a[at], b[at])


@pytest.mark.parametrize("impl,single", PATHS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("names", [("v_clean",), ("do_clean",), CLEAN], ids=["v", "do", "all"])
def test_large_values_of_other_documents(names, d, impl, single):
    t = _tensors(520, 0, 4, 2, d)
    docs = binding.bdlm_doc_table([0, 150, 330, 520])
    mine = slice(150, 330)
    _compare(_packed(_outside(t, names, 520, mine, (1e3, 1e18)), 1, docs, impl, single), _packed(t, 1, docs, impl, single), mine, False, single)


@pytest.mark.parametrize("impl,single", PATHS)
@pytest.mark.parametrize("d", [64, 128])
def test_large_values_of_other_documents_in_both_streams(d, impl, single):
    t = _tensors(576, 576, 4, 2, d)
    docs = binding.bdlm_doc_table([0, 96, 384, 576])
    mine = slice(96, 384)
    _compare(_packed(_outside(t, CLEAN + NOISY, 576, mine, (1e3, 1e18)), 32, docs, impl, single), _packed(t, 32, docs, impl, single), mine, True, single)


@pytest.mark.parametrize("single", [True, False])
def test_large_values_of_other_documents_on_pairs_of_ctas(single):
    t = _tensors(6144, 0, 32, 8, 128)
    docs = binding.bdlm_doc_table([0, 2900, 6144])
    mine = slice(0, 2900)
    _compare(_packed(_outside(t, CLEAN, 6144, mine, (1e3, 1e18)), 1, docs, AUTO, single), _packed(t, 1, docs, AUTO, single), mine, False, single)


@pytest.mark.parametrize("impl,single", PATHS)
@pytest.mark.parametrize("d", [64, 128])
def test_large_values_of_later_keys(d, impl, single):
    """Without documents: rows of both streams before a position, and values from it on."""
    M, cut = 40, 200
    t = _tensors(320, 320, 4, 2, d)

    def run(t):
        qkv = [t[n] for n in ("q_clean", "k_clean", "v_clean", "q_noisy", "k_noisy", "v_noisy")]
        out = binding.bdlm_attn_fwd(*qkv, M, impl=impl)
        return out, binding.bdlm_attn_bwd(*qkv, *out, t["do_clean"], t["do_noisy"], M, impl=impl, single_pass=single)
    out, grads = run(t)
    got, ggrads = run(_large(t, ("v_clean", "v_noisy"), slice(cut, 320), (1e3, 1e18)))
    for i in (0, 2):
        _same(got[i][:, :cut], out[i][:, :cut], False)
        _same(got[i + 1][:, :, :cut], out[i + 1][:, :, :cut], False)
        _same(ggrads[3 * (i // 2)][:, :cut], grads[3 * (i // 2)][:, :cut], single)
    _same(ggrads[5][:, :cut], grads[5][:, :cut], False)
