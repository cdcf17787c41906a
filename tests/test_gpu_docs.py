"""Attention over packed documents (a table of documents with the packed form) against the oracle run on each document by
itself, through the C ABI, both kernel families and both backward paths.

Tolerances: parity_util's for outputs; gradients are compared document by document, so that a wrong short one cannot hide
beside long ones.  Besides TOL_GRAD of the document's gradient they allow what D = dO . O, taken from the bf16 output, is off by:
|dD_i| <= 2^-8 |dO_i| |O_i| (twice the rounding) enters dQ_i as scale dD_i sum_j P_ij k_j, and dK as scale P^T (dD q), whose norm is at most
scale sqrt(n) |dD q|_F because no row of P sums to more than one and no column of n rows to more than n."""
import numpy as np
import pytest
import torch

from oracle import bdlm_oracle as orc
from paper_2609_19242_b200 import binding, synth

import parity_util as pu

pytestmark = pytest.mark.gpu

AUTO, PORTABLE = binding.IMPL_AUTO, binding.IMPL_PORTABLE
CLEAN_NAMES = ("q_clean", "k_clean", "v_clean", "do_clean")
NOISY_NAMES = ("q_noisy", "k_noisy", "v_noisy", "do_noisy")


def _inputs(L, Lq, Ln, H, Hkv, d, batch=1, seed=0):
    g = torch.Generator().manual_seed(seed)
    mk = lambda rows, heads, s: (torch.randn(batch, rows, heads, d, generator=g) * s).to(torch.bfloat16) if rows else None
    t = {"q_clean": mk(Lq, H, 1.0), "k_clean": mk(L, Hkv, 1.0), "v_clean": mk(L, Hkv, 1.0), "do_clean": mk(Lq, H, 1.0),
         "q_noisy": mk(Ln, H, 1.0), "k_noisy": mk(Ln, Hkv, 1.0), "v_noisy": mk(Ln, Hkv, 1.0), "do_noisy": mk(Ln, H, 1.0)}
    return t, {k: None if v is None else v.cuda() for k, v in t.items()}, {k: None if v is None else synth.to_f64(v) for k, v in t.items()}


def _run(g, M, docs, prefix=None, pos0=0, window=0, mode=0, impl=AUTO, single_pass=None):
    kw = dict(block_prefix=None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device="cuda"), clean_q_pos0=pos0,
              impl=impl, window=window, clean_mask_mode=mode, docs=docs)
    qkv = [g[n] for n in ("q_clean", "k_clean", "v_clean", "q_noisy", "k_noisy", "v_noisy")]
    out = binding.bdlm_attn_fwd_packed(*qkv, M, **kw)
    grads = binding.bdlm_attn_bwd_packed(*qkv, *out, g["do_clean"], g["do_noisy"], M, single_pass=single_pass, **kw)
    torch.cuda.synchronize()
    assert binding.bdlm_get_device_status() == 0
    return out, grads


def _norms(t):
    return np.sqrt((t ** 2).sum(axis=-1))


def _check(lens, M=1, H=2, Hkv=1, d=128, noisy=None, pos0=0, Lq=None, window=0, mode=0, impl=AUTO, single_pass=None, batch=1, before=0,
           after=0, seed=0):
    """noisy: None, "all" (every whole block of every document) or a sorted list of prefixes.  before, after: positions of no document."""
    cu = np.cumsum([before] + list(lens))
    L = int(cu[-1]) + after
    Lq = L - pos0 if Lq is None else Lq
    prefix = noisy
    if noisy == "all":
        prefix = [a + b * M for a, n in zip(cu, lens) for b in range(n // M)]
    nb = 0 if prefix is None else len(prefix)
    t, g, x = _inputs(L, Lq, nb * M, H, Hkv, d, batch, seed)
    docs = binding.bdlm_doc_table(torch.tensor(cu, dtype=torch.int32), L)
    out, grads = _run(g, M, docs, prefix, pos0, window, mode, impl, single_pass)
    got = {n: None if v is None else synth.to_f64(v) for n, v in
           zip(("o_clean", "lse_clean", "o_noisy", "lse_noisy", "dq_clean", "dk_clean", "dv_clean", "dq_noisy", "dk_noisy", "dv_noisy"), (*out, *grads))}
    scale, G = 1.0 / np.sqrt(d), H // Hkv
    seen_keys = np.zeros(L, dtype=bool)
    seen_blocks = np.zeros(nb, dtype=bool)
    for a, n in zip(cu, lens):
        z = a + n
        if n == 0:
            continue
        seen_keys[a:z] = True
        r0, r1 = max(a, pos0), min(z, pos0 + Lq)                 # this document's clean queries
        blocks = [b for b in range(nb) if a <= prefix[b] < z]
        seen_blocks[blocks] = True
        rows_n = np.concatenate([np.arange(b * M, (b + 1) * M) for b in blocks]) if blocks else np.zeros(0, dtype=int)
        rows_c = np.arange(r0 - pos0, r1 - pos0) if r1 > r0 else np.zeros(0, dtype=int)
        part = lambda name, rows: x[name][:, rows] if len(rows) else None
        kn, vn = part("k_noisy", rows_n), part("v_noisy", rows_n)
        if kn is None:
            kn = vn = np.zeros((batch, 0, Hkv, d))
        ref = orc.attn_packed(part("q_clean", rows_c), x["k_clean"][:, a:z], x["v_clean"][:, a:z], part("q_noisy", rows_n), kn, vn, M,
                              do_clean=part("do_clean", rows_c), do_noisy=part("do_noisy", rows_n),
                              block_prefix=[prefix[b] - a for b in blocks], clean_q_pos0=r0 - a, window=window, clean_mask_mode=mode)
        d_q = {}   # |dD_i| |q_i| bounds per stream, for dK
        for s, rows in (("clean", rows_c), ("noisy", rows_n)):
            if not len(rows):
                continue
            o, lse = got["o_" + s][:, rows], got["lse_" + s][:, :, rows]
            assert np.abs(o - ref["o_" + s]).max() <= pu.TOL_O * max(1.0, np.abs(ref["o_" + s]).max()), (s, a, n)
            assert np.abs(lse - ref["lse_" + s]).max() <= pu.TOL_LSE, (s, a, n)
            do = x["do_" + s][:, rows]
            dD = 2.0 ** -8 * _norms(do) * _norms(ref["o_" + s])   # [batch, rows, H]
            kmax = max(_norms(x["k_clean"][:, a:z]).max(), _norms(kn).max() if kn.shape[1] else 0.0)
            off = np.sqrt(((scale * dD * kmax) ** 2).sum())
            err = np.linalg.norm(got["dq_" + s][:, rows] - ref["dq_" + s])
            assert err <= pu.TOL_GRAD * np.linalg.norm(ref["dq_" + s]) + off, (s, a, n, err, off)
            d_q[s] = (dD * _norms(x["q_" + s][:, rows])) ** 2
        n_rows = (len(rows_c) + len(rows_n)) * G
        slack = scale * np.sqrt(max(n_rows, 1)) * np.sqrt(sum(v.sum() for v in d_q.values()))
        if not d_q:
            ref.update(dk_clean=np.zeros((batch, n, Hkv, d)), dv_clean=np.zeros((batch, n, Hkv, d)))
        for name, rows in (("clean", np.arange(a, z)), ("noisy", rows_n)):
            if not len(rows):
                continue
            for which, off in (("dk_", slack), ("dv_", 0.0)):
                have, want = got[which + name][:, rows], ref[which + name]
                err = np.linalg.norm(have - want)
                assert err <= pu.TOL_GRAD * np.linalg.norm(want) + off, (which + name, a, n, err, off)
    # positions of no document see nothing and are seen by nothing; a block at one of them sees itself only
    if Lq:
        rows = np.array([i for i in range(Lq) if not seen_keys[pos0 + i]], dtype=int)
        assert (got["o_clean"][:, rows] == 0).all() and np.isneginf(got["lse_clean"][:, :, rows]).all() and (got["dq_clean"][:, rows] == 0).all()
    assert (got["dk_clean"][:, ~seen_keys] == 0).all() and (got["dv_clean"][:, ~seen_keys] == 0).all()
    for b in np.nonzero(~seen_blocks)[0]:
        rows = np.arange(b * M, (b + 1) * M)
        ref = orc.attn_packed(None, np.zeros((batch, 0, Hkv, d)), np.zeros((batch, 0, Hkv, d)), x["q_noisy"][:, rows], x["k_noisy"][:, rows],
                              x["v_noisy"][:, rows], M, block_prefix=[0])
        assert np.abs(got["o_noisy"][:, rows] - ref["o_noisy"]).max() <= pu.TOL_O * max(1.0, np.abs(ref["o_noisy"]).max())
    for v in got.values():
        assert v is None or not np.isnan(v).any()
    return out, grads


PATHS = [(AUTO, True), (AUTO, False), (PORTABLE, False)]


@pytest.mark.parametrize("impl,single", PATHS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[1], [5], [128], [1, 1, 1], [127, 1, 129], [100, 1, 27, 128], [300, 2, 40, 0, 90], [64] * 9, [383, 257, 1], [1] * 200],
                         ids=lambda l: "-".join(map(str, l)))
def test_prompts_of_different_lengths(lens, d, impl, single):
    _check(lens, d=d, impl=impl, single_pass=single)


@pytest.mark.parametrize("impl,single", PATHS)
@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 1), (4, 2), (6, 2), (8, 1)])
def test_grouped_heads(H, Hkv, impl, single):
    _check([200, 33, 150], H=H, Hkv=Hkv, impl=impl, single_pass=single)
    _check([200, 33, 150], H=H, Hkv=Hkv, d=64, impl=impl, single_pass=single, batch=2)


@pytest.mark.parametrize("impl,single", PATHS)
@pytest.mark.parametrize("M,lens", [(16, [48, 16, 160, 96]), (32, [320, 32, 64, 128]), (40, [200, 40, 120]), (4, [100, 8, 60]), (128, [256, 128])])
def test_both_streams_over_documents_of_whole_blocks(M, lens, impl, single):
    _check(lens, M=M, H=4, Hkv=2, noisy="all", impl=impl, single_pass=single)
    _check(lens, M=M, H=3, Hkv=1, d=64, noisy="all", mode=1, impl=impl, single_pass=single)


@pytest.mark.parametrize("impl,single", PATHS)
def test_sampled_blocks(impl, single):
    """Anchors at a document's first and last positions, repeated ones, and past all documents."""
    _check([300, 77, 200], M=16, noisy=[0, 0, 1, 150, 299, 300, 301, 376, 377, 420, 576], pos0=0, impl=impl, single_pass=single)
    _check([300, 77, 200], M=16, noisy=[5, 290, 300, 377, 570, 577], Lq=0, impl=impl, single_pass=single)
    _check([64, 64], M=8, noisy=[3, 64, 127, 128, 128], Lq=0, impl=impl, single_pass=single)


@pytest.mark.parametrize("impl,single", PATHS)
def test_sliding_window(impl, single):
    for window in (1, 33, 150, 1000):
        _check([260, 40, 300], window=window, impl=impl, single_pass=single)
    _check([256, 64, 320], M=32, noisy="all", window=100, impl=impl, single_pass=single)


@pytest.mark.parametrize("impl,single", PATHS)
def test_a_run_of_queries_at_an_offset(impl, single):
    """A rank's piece of the packed sequence: it begins and ends inside documents, and misses others."""
    _check([150, 100, 260, 90], pos0=200, Lq=200, impl=impl, single_pass=single)
    _check([150, 100, 260, 90], pos0=330, Lq=1, impl=impl, single_pass=single)
    _check([150, 100, 260, 90], pos0=250, Lq=260, M=10, noisy=[0, 100, 160, 260, 500], impl=impl, single_pass=single)


@pytest.mark.parametrize("impl,single", PATHS)
def test_positions_of_no_document(impl, single):
    _check([100, 200], before=70, after=130, impl=impl, single_pass=single)
    _check([100, 1], after=300, impl=impl, single_pass=single)
    _check([96, 64], M=16, before=16, after=32, noisy=[0, 16, 64, 112, 160, 176, 180], impl=impl, single_pass=single)


def test_long_documents_on_pairs_of_ctas_and_clusters():
    """Sizes at which the backward shares key tiles among CTAs, or takes two at a time, whatever the documents are."""
    _check([700, 1300, 48], H=8, Hkv=1, single_pass=True)          # few tiles, many steps: clusters share them
    t, g, _ = _inputs(6144, 6144, 0, 32, 8, 128)
    lens = [6000, 144]
    docs = binding.bdlm_doc_table([0, 6000, 6144])
    out, grads = _run(g, 1, docs)
    # the documents by themselves, through the plain packed form
    for a, z in ((0, 6000), (6000, 6144)):
        part = {k: None if v is None else v[:, a:z].contiguous() for k, v in g.items()}
        qkv = [part[n] for n in ("q_clean", "k_clean", "v_clean")] + [None] * 3
        o, lse, _, _ = binding.bdlm_attn_fwd_packed(*qkv, 1)
        # the same products; a document that does not begin on a tile's first row is cut into tiles elsewhere
        assert float((out[0][:, a:z].float() - o.float()).abs().max()) <= pu.TOL_O
        assert float((out[1][:, :, a:z] - lse).abs().max()) <= pu.TOL_LSE
        ref = binding.bdlm_attn_bwd_packed(*qkv, o, lse, None, None, part["do_clean"], None, 1, single_pass=False)
        for have, want in zip(grads[:3], ref[:3]):
            assert pu.rel_l2(synth.to_f64(have[:, a:z]), synth.to_f64(want)) <= 1e-2


def test_one_document_is_the_plain_form_bit_for_bit():
    t, g, _ = _inputs(700, 700, 0, 4, 2, 128, batch=2)
    docs = binding.bdlm_doc_table([0, 700])
    out, grads = _run(g, 1, docs, single_pass=False)
    plain, pgrads = _run(g, 1, None, single_pass=False)
    for a, b in zip((*out[:2], *grads[:3]), (*plain[:2], *pgrads[:3])):
        assert torch.equal(a, b)


def test_neighbours_have_no_effect():
    """Other values in the other documents change nothing, large ones included."""
    t, g, _ = _inputs(900, 900, 0, 4, 2, 128)
    docs = binding.bdlm_doc_table([0, 250, 600, 900])
    out, grads = _run(g, 1, docs, single_pass=False)
    for k in CLEAN_NAMES:
        g[k][:, :250] *= 1000.0
        g[k][:, 600:] = 65000.0
    out2, grads2 = _run(g, 1, docs, single_pass=False)
    at = slice(250, 600)
    assert torch.equal(out[0][:, at], out2[0][:, at]) and torch.equal(out[1][:, :, at], out2[1][:, :, at])
    for a, b in zip(grads[:3], grads2[:3]):
        assert torch.equal(a[:, at], b[:, at])


def test_reproducible_two_pass_gradients_and_capture():
    t, g, _ = _inputs(640, 640, 0, 4, 2, 64)
    docs = binding.bdlm_doc_table([0, 100, 101, 400, 640])
    want, wgrads = _run(g, 1, docs, single_pass=False)
    graph = torch.cuda.CUDAGraph()
    qkv = [g[n] for n in ("q_clean", "k_clean", "v_clean")] + [None] * 3
    with torch.cuda.graph(graph):
        out = binding.bdlm_attn_fwd_packed(*qkv, 1, docs=docs)
        grads = binding.bdlm_attn_bwd_packed(*qkv, *out, g["do_clean"], None, 1, docs=docs, single_pass=False)
    for _ in range(2):
        for t in (*out[:2], *grads[:3]):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((*out[:2], *grads[:3]), (*want[:2], *wgrads[:3])):
            assert torch.equal(a, b)


def test_shards_of_the_keys_merge_to_the_whole():
    """Context shards cut across documents; a shard without a row's document leaves the row empty."""
    t, g, _ = _inputs(640, 640, 640, 4, 2, 128)
    docs = binding.bdlm_doc_table([0, 96, 128, 480, 640])
    qkv = [g[n] for n in ("q_clean", "k_clean", "v_clean", "q_noisy", "k_noisy", "v_noisy")]
    whole = binding.bdlm_attn_fwd_packed(*qkv, 32, docs=docs)
    parts = [binding.bdlm_attn_fwd_packed(*qkv, 32, docs=docs, kv_range=r, include_noisy_diag=diag)
             for r, diag in (((0, 100), True), ((100, 300), False), ((300, 300), False), ((300, 640), False))]
    assert torch.isneginf(parts[0][1][:, :, 480:]).all() and (parts[0][0][:, 480:] == 0).all()
    for s in (0, 2):
        o, lse = binding.bdlm_lse_merge([x[s] for x in parts], [x[s + 1] for x in parts])
        assert float((lse - whole[s + 1]).abs().max()) <= 1e-4
        # each partial output and the merged one are rounded: 2^-8 of the value each, the weights sum to one
        assert float((o.float() - whole[s].float()).abs().max()) <= 3 * 2.0 ** -8 * float(whole[s].float().abs().max())


def test_scale_and_passes_one_by_one():
    t, g, _ = _inputs(300, 300, 0, 4, 2, 64)
    docs = binding.bdlm_doc_table([0, 130, 300])
    qkv = [g[n] for n in ("q_clean", "k_clean", "v_clean")] + [None] * 3
    doubled = [(g["q_clean"].float() * 2).bfloat16()] + qkv[1:]
    out = binding.bdlm_attn_fwd_packed(*qkv, 1, docs=docs, scale=0.25)          # 64 ** -0.5 = 0.125
    twice = binding.bdlm_attn_fwd_packed(*doubled, 1, docs=docs)
    assert torch.equal(out[0], twice[0]) and torch.equal(out[1], twice[1])
    args = (*qkv, *out, g["do_clean"], None, 1)
    want = binding.bdlm_attn_bwd_packed(*args, docs=docs, scale=0.25, single_pass=False)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    got = tuple(torch.empty_like(x) for x in want[:3]) + (None,) * 3
    for one in (binding.PASS_DSUM, binding.PASS_DKDV, binding.PASS_DQ):
        binding.bdlm_attn_bwd_packed(*args, docs=docs, scale=0.25, single_pass=False, passes=one, workspace=ws, out=got)
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a, b)


def test_tables_on_two_streams():
    """A table made on one stream and used on others after an event, with calls of different documents at once."""
    t, g, _ = _inputs(512, 512, 0, 4, 2, 64)
    qkv = [g[n] for n in ("q_clean", "k_clean", "v_clean")] + [None] * 3
    tables = [binding.bdlm_doc_table(cu) for cu in ([0, 200, 512], [0, 1, 300, 301, 512])]
    want = [binding.bdlm_attn_fwd_packed(*qkv, 1, docs=d)[0].clone() for d in tables]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in tables], []
    for _ in range(4):
        for s, d in zip(streams, tables):
            with torch.cuda.stream(s):
                got.append(binding.bdlm_attn_fwd_packed(*qkv, 1, docs=d)[0])
    torch.cuda.synchronize()
    for i, o in enumerate(got):
        assert torch.equal(o, want[i % 2])


@pytest.mark.parametrize("impl,single", PATHS)
def test_blocks_that_documents_cut(impl, single):
    """Mask mode 1, blocks counted from position 0: a document's first and last blocks are cut by its ends."""
    lens, M = [70, 5, 1, 130, 94], 32
    cu = np.concatenate([[0], np.cumsum(lens)])
    L = int(cu[-1])
    t, g, x = _inputs(L, L, 0, 2, 1, 64)
    out, grads = _run(g, M, binding.bdlm_doc_table([int(c) for c in cu]), mode=1, impl=impl, single_pass=single)
    none = np.zeros((1, 0, 1, 64))
    dk, dv = np.zeros((1, L, 1, 64)), np.zeros((1, L, 1, 64))
    for a, z in zip(cu, cu[1:]):
        ref = orc.attn_packed(x["q_clean"][:, a:z], x["k_clean"], x["v_clean"], None, none, none, M, do_clean=x["do_clean"][:, a:z],
                              clean_q_pos0=a, clean_mask_mode=1, kv_begin=a, kv_end=z)
        assert np.abs(synth.to_f64(out[0][:, a:z]) - ref["o_clean"]).max() <= pu.TOL_O * max(1.0, np.abs(ref["o_clean"]).max())
        assert np.abs(synth.to_f64(out[1][:, :, a:z]) - ref["lse_clean"]).max() <= pu.TOL_LSE
        dk += ref["dk_clean"]
        dv += ref["dv_clean"]
        if z - a > 1:
            assert pu.rel_l2(synth.to_f64(grads[0][:, a:z]), ref["dq_clean"]) <= pu.TOL_GRAD
    assert pu.rel_l2(synth.to_f64(grads[1]), dk) <= pu.TOL_GRAD and pu.rel_l2(synth.to_f64(grads[2]), dv) <= pu.TOL_GRAD


def test_a_captured_call_takes_the_documents_of_a_rewritten_table():
    """The launches depend on a table's contents for their order alone: a table written again in place, for other documents of the
    same positions, is what a replay goes by."""
    t, g, _ = _inputs(900, 900, 0, 6, 2, 64)
    qkv = [g[n] for n in ("q_clean", "k_clean", "v_clean")] + [None] * 3
    docs = binding.bdlm_doc_table([0, 300, 900])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = binding.bdlm_attn_fwd_packed(*qkv, 1, docs=docs)
        grads = binding.bdlm_attn_bwd_packed(*qkv, *out, g["do_clean"], None, 1, docs=docs, single_pass=False)
    for cu in ([0, 900], [0, 1, 2, 700, 899, 900], [0, 300, 900]):
        new = torch.tensor(cu, dtype=torch.int32, device="cuda")
        assert binding.lib().bdlm_doc_table(new.data_ptr(), len(cu) - 1, 900, docs.buffer.data_ptr(), binding._stream()) == 0
        graph.replay()
        want, wgrads = _run(g, 1, binding.bdlm_doc_table(cu), single_pass=False)
        for a, b in zip((*out[:2], *grads[:3]), (*want[:2], *wgrads[:3])):
            assert torch.equal(a, b)


def test_table_of_documents():
    for cu, L in (([0, 4, 4, 9], 9), ([2, 5, 6], 8), ([0, 1], 1), ([3, 3, 3], 5)):
        table = binding.bdlm_doc_table(torch.tensor(cu, dtype=torch.int32, device="cuda"), L)
        want = [[p, p] for p in range(L + 1)]
        for a, z in zip(cu, cu[1:]):
            for p in range(a, z):
                want[p] = [a, z]
        assert table.table.cpu().tolist() == want
        assert table.max_len == max(z - a for a, z in zip(cu, cu[1:]))


def test_wrong_tables_stay_inside_the_tensors():
    """The library does not validate the entries on the device: wrong ones give wrong documents inside [0, L]."""
    cu = torch.tensor([50, 20, -7, 2 ** 31 - 1, 90], dtype=torch.int32, device="cuda")
    buffer = torch.full((binding.lib().bdlm_doc_table_bytes(64) // 4,), -1, dtype=torch.int32, device="cuda")
    assert binding.lib().bdlm_doc_table(cu.data_ptr(), 4, 64, buffer.data_ptr(), binding._stream()) == 0
    assert int(buffer.min()) >= 0 and int(buffer[:130].max()) <= 64 and (buffer[130:] == 0).all()   # one tile of each kind


def test_order_of_tiles():
    """The orders behind the table are the tiles by the work that they have, ties by place."""
    rng = np.random.default_rng(4)
    for lens in ([1000, 3, 700, 128, 128, 2000], list(rng.integers(1, 400, size=60)), [5]):
        cu = np.concatenate([[0], np.cumsum(lens)])
        L = int(cu[-1])
        docs = binding.bdlm_doc_table([int(c) for c in cu])
        begin, end = docs.table[:, 0].cpu().numpy(), docs.table[:, 1].cpu().numpy()
        at = 2 * (L + 1)
        for rows, queries in ((128, False), (128, True), (256, True)):
            n = -(-L // rows)
            work = [min(L, (t + 1) * rows) - begin[t * rows] if queries else end[min(L, (t + 1) * rows) - 1] - t * rows for t in range(n)]
            want = sorted(range(n), key=lambda t: (-work[t], t))
            assert docs.buffer[at:at + n].tolist() == [n - 1 - t if queries else t for t in want]
            at += n
        assert at == docs.buffer.numel()


def test_refusals():
    t, g, _ = _inputs(256, 256, 0, 2, 1, 64)
    qkv = [g[n] for n in ("q_clean", "k_clean", "v_clean")] + [None] * 3
    for bad in ([0], [0, 5, 3], [-1, 4], [[0, 4]], torch.tensor([0.0, 4.0])):
        with pytest.raises(ValueError):
            binding.bdlm_doc_table(bad)
    with pytest.raises(ValueError):
        binding.bdlm_doc_table([0, 100], 50)
    with pytest.raises(ValueError):
        binding.bdlm_attn_fwd_packed(*qkv, 1, docs=binding.bdlm_doc_table([0, 255]))
    with pytest.raises(ValueError):
        binding.bdlm_attn_fwd_packed(*qkv, 1, docs=binding.bdlm_doc_table([0, 256]), kv_chunks=(128, [128, 0]))


def test_documents_that_cut_blocks_are_refused():
    """A noisy block over a border would attend across two documents; given by its prefix, a block belongs to the document that it
    starts in."""
    t, g, _ = _inputs(256, 256, 256, 2, 1, 64)
    qkv = [g[n] for n in ("q_clean", "k_clean", "v_clean", "q_noisy", "k_noisy", "v_noisy")]
    whole, cut, padded = (binding.bdlm_doc_table(cu, 256) for cu in ([0, 96, 96, 256], [0, 100, 256], [0, 96, 250]))
    out = binding.bdlm_attn_fwd_packed(*qkv, 32, docs=whole)
    for docs in (cut, padded):
        with pytest.raises(ValueError):
            binding.bdlm_attn_fwd_packed(*qkv, 32, docs=docs)
        with pytest.raises(ValueError):
            binding.bdlm_attn_bwd_packed(*qkv, *out, g["do_clean"], g["do_noisy"], 32, docs=docs)
        prefix = torch.arange(0, 256, 32, dtype=torch.int32, device="cuda")
        binding.bdlm_attn_fwd_packed(*qkv, 32, docs=docs, block_prefix=prefix)
        binding.bdlm_attn_fwd_packed(*qkv[:3], None, None, None, 32, docs=docs)
    short = [x[:, :96].contiguous() for x in qkv[3:]]
    binding.bdlm_attn_fwd_packed(*qkv[:3], *short, 32, docs=padded)   # no block over its end
    torch.cuda.synchronize()


@pytest.mark.parametrize("single,window", [(True, 0), (False, 0), (True, 1700)])
def test_both_streams_of_long_documents_on_pairs_of_ctas(single, window):
    """Documents that begin anywhere in a pair's 256 keys, against the same documents by themselves; dK and dV have the same bits each time."""
    L, M, cu = 7680, 32, [0, 2912, 2976, 7680]
    t, g, _ = _inputs(L, L, L, 32, 8, 128)
    docs = binding.bdlm_doc_table(cu)
    out, grads = _run(g, M, docs, window=window, single_pass=single)
    for _ in range(6):
        _, again = _run(g, M, docs, window=window, single_pass=single)
        for i in (1, 2, 4, 5):
            assert torch.equal(again[i], grads[i]), i
    for a, z in zip(cu, cu[1:]):
        part = {k: v[:, a:z].contiguous() for k, v in g.items()}
        ref, rgrads = _run(part, M, None, window=window, single_pass=False)
        for s in (0, 2):   # the same products, cut into tiles elsewhere
            assert float((out[s][:, a:z].float() - ref[s].float()).abs().max()) <= pu.TOL_O
            assert float((out[s + 1][:, :, a:z] - ref[s + 1]).abs().max()) <= pu.TOL_LSE
        for have, want in zip(grads, rgrads):
            assert pu.rel_l2(synth.to_f64(have[:, a:z]), synth.to_f64(want)) <= 1e-2


def test_more_tiles_than_a_table_orders():
    """Past 4096 tiles of 128 positions a table holds no orders: the tiles start in their own."""
    L = 4096 * 128 + 999
    g = torch.Generator(device="cuda").manual_seed(0)
    q, k, v, do = (torch.randn(1, L, h, 64, generator=g, device="cuda").to(torch.bfloat16) for h in (2, 1, 1, 2))
    cu = sorted({0, L, *range(100, L, 311)})
    docs = binding.bdlm_doc_table(cu)
    assert docs.buffer.numel() == 2 * (L + 1)
    out = binding.bdlm_attn_fwd_packed(q, k, v, None, None, None, 1, docs=docs)
    for single in (True, False):
        grads = binding.bdlm_attn_bwd_packed(q, k, v, None, None, None, *out, do, None, 1, docs=docs, single_pass=single)
        for i in (0, 1, len(cu) // 2, len(cu) - 3, len(cu) - 2):
            a, z = cu[i], cu[i + 1]
            part = [x[:, a:z].contiguous() for x in (q, k, v, do)]
            ref = binding.bdlm_attn_fwd_packed(*part[:3], None, None, None, 1)
            rgrads = binding.bdlm_attn_bwd_packed(*part[:3], None, None, None, *ref, part[3], None, 1, single_pass=False)
            assert float((out[0][:, a:z].float() - ref[0].float()).abs().max()) <= pu.TOL_O
            assert float((out[1][:, :, a:z] - ref[1]).abs().max()) <= pu.TOL_LSE
            for have, want in zip(grads[:3], rgrads[:3]):
                assert pu.rel_l2(synth.to_f64(have[:, a:z]), synth.to_f64(want)) <= 1e-2
