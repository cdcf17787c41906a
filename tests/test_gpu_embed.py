"""The token embedding against its fp64 oracle, through the binding.

Tolerances.  The lookup is one fp32 product rounded once: (eps/2 + 2^-24) of the value.  A gradient row of n tokens is summed in
fp32: at most 2 `piece` additions one after the other (piece: 8, or T / 1024), or `piece` of them and then the parts of up to 11
pieces in order, or of more in sixteen shares, so for the sizes here it is off by at most (piece + T / (8 piece) + 16) x 2^-24 of the sum of the terms'
magnitudes (2 piece is less for T up to 147000), and rounded once."""
import numpy as np
import pytest
import torch

from oracle import model_ops_oracle as orc
from paper_2609_19242_b200 import binding

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [(BF16, BF16), (FP16, FP16), (FP32, FP32), (FP32, BF16), (FP32, FP16)]


def _f64(t):
    return t.detach().double().cpu().numpy()


def _half_ulp(t):
    return torch.finfo(t).eps / 2


def _tiny(t):
    """Half the distance of the type's smallest values."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def _ids(T, V, seed=0, masked=0.0, pad=0.05):
    rng = np.random.default_rng(seed)
    ids = np.minimum(((V + 1.0) ** rng.random(T)).astype(np.int64) - 1, V - 1)
    ids[rng.random(T) < masked] = V - 1
    ids[rng.random(T) < pad] = -1
    return ids


def _check_fwd(T, D, V, e=BF16, o=BF16, scale=1.0, ids=None):
    g = torch.Generator().manual_seed(T + D)
    table = torch.randn(V, D, generator=g).to(e).cuda()
    ids = _ids(T, V, D) if ids is None else ids
    out = binding.bdlm_embed_fwd(table, torch.tensor(ids, dtype=torch.int32, device="cuda"), scale=scale, dtype=o)
    assert out.shape == (T, D) and out.dtype == o
    ref = orc.embed_forward(_f64(table), ids, float(np.float32(scale)))
    assert (np.abs(_f64(out) - ref) <= (_half_ulp(o) + 2.0 ** -24 + 2.0 ** -33) * np.abs(ref) + _tiny(o)).all()


def _check_bwd(T, D, V, e=BF16, o=BF16, scale=1.0, ids=None, start=None, masked=0.0):
    g = torch.Generator().manual_seed(T + D)
    dout = torch.randn(T, D, generator=g).to(o).cuda()
    ids = _ids(T, V, D, masked) if ids is None else np.asarray(ids)
    dev = torch.tensor(ids, dtype=torch.int32, device="cuda")
    if start is None:
        out = torch.full((V, D), float("nan"), device="cuda", dtype=e)
        binding.bdlm_embed_bwd(dout, dev, V, scale=scale, out=out)
        again = binding.bdlm_embed_bwd(dout, dev, V, scale=scale, dtype=e)
        assert torch.equal(out, again)   # bitwise reproducible
        base = None
    else:
        first = torch.randn(V, D, generator=g).to(e).cuda()
        out = first.clone()
        binding.bdlm_embed_bwd(dout, dev, V, scale=scale, out=out, accumulate=True)
        base = _f64(first)
    s = float(np.float32(scale))
    ref = orc.embed_backward(_f64(dout), ids, V, s, base)
    size = orc.embed_backward(np.abs(_f64(dout)), ids, V, abs(s))
    piece = max(8, -(-T // 1024))
    off = (piece + T / (8 * piece) + 16) * 2.0 ** -24 * (size + (0 if base is None else np.abs(base)))
    assert (np.abs(_f64(out) - ref) <= _half_ulp(e) * (np.abs(ref) + off) + off + _tiny(e)).all()
    if base is not None:   # rows of tokens that do not occur stay as they were
        absent = np.setdiff1d(np.arange(V), ids)
        assert torch.equal(out[absent], first[absent])


@pytest.mark.parametrize("D", [1, 3, 8, 24, 100, 128, 1001, 1024, 1544, 4096, 9000])
@pytest.mark.parametrize("T", [1, 2, 7, 33, 500])
def test_lookup_sizes(T, D):
    _check_fwd(T, D, 300, scale=D ** 0.5)


@pytest.mark.parametrize("e,o", TYPES)
@pytest.mark.parametrize("D", [40, 77])
def test_types(e, o, D):
    _check_fwd(200, D, 50, e, o, scale=-0.7)
    _check_bwd(200, D, 50, e, o, scale=-0.7)
    _check_bwd(200, D, 50, e, o, scale=3.0, start=True)


@pytest.mark.parametrize("T", [1, 2, 8, 9, 31, 32, 33, 64, 100, 1531, 2048, 2049, 4097, 8193, 20000])
def test_gradient_numbers_of_tokens(T):
    """Every cluster size of the sort, pieces of eight tokens and of more."""
    _check_bwd(T, 40, 777, masked=0.3)


@pytest.mark.parametrize("D", [1, 3, 8, 24, 100, 1001, 1024, 1032, 1544, 4096])
def test_gradient_lengths_of_rows(D):
    _check_bwd(300, D, 211, masked=0.25)
    _check_bwd(300, D, 211, masked=0.25, start=True)


@pytest.mark.parametrize("V", [1, 2, 511, 512, 513, 5000, 128256, 262144, 1 << 20])
def test_gradient_sizes_of_the_table(V):
    """One to four digits of the sort; tables far larger than the number of tokens."""
    _check_bwd(600, 8, V, masked=0.2)


@pytest.mark.parametrize("case", ["one", "alternating", "none", "beyond", "descending", "runs", "last_only", "mixed_pads"])
@pytest.mark.parametrize("start", [None, True])
def test_gradient_patterns_of_ids(case, start):
    T, V = 3000, 97
    t = np.arange(T)
    ids = {"one": np.full(T, 41), "alternating": t % 2 * 96, "none": np.full(T, -1), "beyond": np.where(t % 3 == 0, V, np.where(t % 3 == 1, 2 ** 31 - 1, -2 ** 31)),
           "descending": (T - 1 - t) % V, "runs": t // 40 % V, "last_only": np.where(t == T - 1, 5, -1), "mixed_pads": np.where(t % 2 == 0, -7, t % V)}[case]
    _check_bwd(T, 72, V, FP32, FP32, ids=ids, start=start)


def test_a_run_over_every_piece_and_its_neighbours():
    """The mask token's run begins in one piece, covers many and ends in another, with short runs around it."""
    T, V = 5000, 64
    ids = np.concatenate([np.arange(13), np.full(4000, 30), np.arange(T - 4013) % 33 + 31])
    rng = np.random.default_rng(3)
    rng.shuffle(ids)
    _check_bwd(T, 264, V, FP32, BF16, ids=ids, scale=0.125)
    _check_bwd(T, 264, V, BF16, BF16, ids=ids, scale=0.125)


@pytest.mark.parametrize("start", [None, True])
@pytest.mark.parametrize("D", [5, 24, 4104])
def test_few_tokens_in_one_launch(D, start):
    for seed in range(4):
        rng = np.random.default_rng(seed)
        for T in (1, 3, 17, 32):
            _check_bwd(T, D, 9, ids=rng.integers(-2, 11, size=T), start=start)
    _check_bwd(32, D, 70000, FP32, FP32, ids=np.full(32, 69999), start=start)


@pytest.mark.parametrize("start", [None, True])
def test_runs_of_every_length_at_every_place_in_a_piece(start):
    """Pieces of eight tokens: runs inside one, over a border, over exactly one whole piece, over more, with padding behind."""
    for k in range(8):
        lens = [k + 1] + [n for n in range(1, 28) for _ in range(2)] + [8, 8, 16, 24, 7, 9, 17, 15, 23, 25]
        ids = np.repeat(np.arange(len(lens)), lens)
        _check_bwd(len(ids), 16, len(lens) + 3, FP32, FP32, ids=ids, start=start)
        ids = np.concatenate([ids, np.full(13 + k, -1)])
        _check_bwd(len(ids), 16, len(lens), BF16, BF16, ids=np.random.default_rng(k).permutation(ids), start=start)


def test_runs_in_longer_pieces():
    """Three tokens more than 1024 pieces of eight: pieces of nine."""
    T = 8195
    lens = []
    rng = np.random.default_rng(1)
    while sum(lens) < T:
        lens.append(int(rng.choice([1, 2, 8, 9, 10, 17, 18, 19, 27, 28, 100, 900])))
    ids = np.repeat(np.arange(len(lens)), lens)[:T]
    _check_bwd(T, 24, len(lens), FP32, FP32, ids=ids)
    _check_bwd(T, 24, len(lens), BF16, BF16, ids=rng.permutation(ids), start=True)


def test_many_tokens():
    _check_bwd(70001, 16, 3000, masked=0.5)


def test_more_elements_than_32_bits_count():
    """Tables and rows of tokens past 2^31 elements."""
    V, D = 524288 + 100, 4096
    table = torch.zeros(V, D, device="cuda", dtype=BF16)
    table[-5:] = torch.randn(5, D, device="cuda").to(BF16)
    ids = torch.tensor([V - 1, 0, V - 5, V, V - 3], dtype=torch.int32, device="cuda")
    out = binding.bdlm_embed_fwd(table, ids)
    for t, v in ((0, V - 1), (1, 0), (2, V - 5), (4, V - 3)):
        assert torch.equal(out[t], table[v])
    assert (out[3] == 0).all()
    grad = binding.bdlm_embed_bwd(out, ids, V, out=table)
    want = {V - 1: 0, V - 5: 2, V - 3: 4}
    for v in (V - 1, V - 2, V - 3, V - 4, V - 5):
        assert torch.equal(grad[v], out[want[v]]) if v in want else (grad[v] == 0).all()
    assert (grad[:-5] == 0).all()
    del table, grad
    T, D = 1 << 20, 2056
    dout = torch.ones(T, D, device="cuda", dtype=BF16)
    dout[:-8] = 0
    ids = torch.full((T,), 2, dtype=torch.int32, device="cuda")
    ids[-3:] = 1
    grad = binding.bdlm_embed_bwd(dout, ids, 3, dtype=BF16)
    assert (grad[0] == 0).all() and (grad[1] == 3).all() and (grad[2] == 5).all()


def test_no_tokens():
    table = torch.randn(10, 16, device="cuda").to(BF16)
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    assert binding.bdlm_embed_fwd(table, ids).shape == (0, 16)
    dout = torch.empty(0, 16, device="cuda", dtype=BF16)
    assert (binding.bdlm_embed_bwd(dout, ids, 10, out=table.clone()) == 0).all()
    kept = table.clone()
    binding.bdlm_embed_bwd(dout, ids, 10, out=kept, accumulate=True)
    assert torch.equal(kept, table)


def test_shapes_of_more_dimensions():
    table = torch.randn(50, 24, device="cuda").to(BF16)
    ids = torch.tensor(_ids(24, 50), dtype=torch.int32, device="cuda").view(2, 3, 4)
    out = binding.bdlm_embed_fwd(table, ids, scale=2.0)
    assert out.shape == (2, 3, 4, 24)
    assert torch.equal(out.view(24, 24), binding.bdlm_embed_fwd(table, ids.view(-1), scale=2.0))
    assert torch.equal(binding.bdlm_embed_bwd(out, ids, 50), binding.bdlm_embed_bwd(out.view(24, 24), ids.view(-1), 50))


def test_ids_and_rows_of_any_alignment_within_the_rules():
    """ids need four bytes only."""
    table = torch.randn(50, 24, device="cuda").to(BF16)
    ids = torch.tensor(_ids(41, 50), dtype=torch.int32, device="cuda")
    assert torch.equal(binding.bdlm_embed_fwd(table, ids[1:]), binding.bdlm_embed_fwd(table, ids)[1:])
    dout = torch.randn(40, 24, device="cuda").to(BF16)
    assert torch.equal(binding.bdlm_embed_bwd(dout, ids[1:], 50), binding.bdlm_embed_bwd(dout, ids[1:].clone(), 50))


def test_not_a_number_stays_with_its_token():
    V, T = 40, 500
    ids = _ids(T, V)
    dout = torch.randn(T, 24, device="cuda").to(BF16)
    dev = torch.tensor(ids, dtype=torch.int32, device="cuda")
    want = binding.bdlm_embed_bwd(dout, dev, V)
    bad = dout.clone()
    bad[ids == 3] = float("nan")
    bad[ids == -1] = float("inf")   # padding rows may hold anything
    got = binding.bdlm_embed_bwd(bad, dev, V)
    others = [v for v in range(V) if v != 3]
    assert got[3].isnan().all() and torch.equal(got[others], want[others])


def test_under_capture_on_another_stream_and_interleaved():
    T, D, V = 3000, 264, 500
    dout = torch.randn(T, D, device="cuda").to(BF16)
    a = torch.tensor(_ids(T, V, 1, 0.4), dtype=torch.int32, device="cuda")
    b = torch.tensor(_ids(T, V, 2, 0.1), dtype=torch.int32, device="cuda")
    want = [binding.bdlm_embed_bwd(dout, i, V) for i in (a, b)]
    # two streams at once, each with its own workspace
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for s, i in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                got.append(binding.bdlm_embed_bwd(dout, i, V))
    torch.cuda.synchronize()
    for k, t in enumerate(got):
        assert torch.equal(t, want[k % 2])
    graph = torch.cuda.CUDAGraph()
    ids = a.clone()
    with torch.cuda.graph(graph):
        rows = binding.bdlm_embed_fwd(want[0], ids)
        grad = binding.bdlm_embed_bwd(dout, ids, V)
    for i, w in zip((a, b, a), (want[0], want[1], want[0])):
        ids.copy_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(grad, w)
        assert torch.equal(rows, binding.bdlm_embed_fwd(want[0], i))


def test_gradient_of_a_tied_table_adds_to_the_loss_heads():
    """The head's dW and the embedding's gradient in one buffer, as for a table that is both."""
    T, D, V = 256, 128, 512
    h, w = torch.randn(T, D, device="cuda").to(BF16), (0.05 * torch.randn(V, D, device="cuda")).to(BF16)
    ids = torch.tensor(_ids(T, V, 5, 0.3), dtype=torch.int32, device="cuda")
    labels = torch.tensor(_ids(T, V, 6), dtype=torch.int32, device="cuda")
    _, _, lse = binding.bdlm_linear_ce_fwd(h, w, labels)
    dh, dw = binding.bdlm_linear_ce_bwd(h, w, labels, lse)
    got = dw.clone()
    binding.bdlm_embed_bwd(dh, ids, V, scale=0.5, out=got, accumulate=True)
    ref = orc.embed_backward(_f64(dh), ids.cpu().numpy(), V, 0.5, _f64(dw))
    size = orc.embed_backward(np.abs(_f64(dh)), ids.cpu().numpy(), V, 0.5, np.abs(_f64(dw)))
    off = 64 * 2.0 ** -24 * size
    assert (np.abs(_f64(got) - ref) <= _half_ulp(BF16) * (np.abs(ref) + off) + off).all()


def test_refusals():
    table = torch.randn(10, 16, device="cuda").to(BF16)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        binding.bdlm_embed_fwd(table, ids.long())
    with pytest.raises(ValueError):
        binding.bdlm_embed_fwd(table, ids.cpu())
    with pytest.raises(binding.BdlmError):
        binding.bdlm_embed_fwd(table, ids, dtype=FP32)
    with pytest.raises(binding.BdlmError):
        binding.bdlm_embed_fwd(table, ids, scale=float("inf"))
    dout = torch.randn(4, 16, device="cuda").to(BF16)
    with pytest.raises(ValueError):
        binding.bdlm_embed_bwd(dout, ids[:3], 10)
    with pytest.raises(ValueError):
        binding.bdlm_embed_bwd(dout, ids, 10, accumulate=True)
    with pytest.raises(ValueError):
        binding.bdlm_embed_bwd(dout, ids, 10, out=torch.empty(11, 16, device="cuda", dtype=BF16))
    with pytest.raises(binding.BdlmError) as e:
        binding.bdlm_embed_bwd(dout.repeat(20, 1), ids.repeat(20), 10, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -3
    with pytest.raises(AssertionError):
        binding.bdlm_embed_fwd(table[:, ::2], ids)


@pytest.mark.parametrize("e", [BF16, FP32])
@pytest.mark.parametrize("D", [1, 2, 5, 7, 31, 55, 56, 63, 64, 65, 120, 127, 128, 129])
def test_short_rows_and_what_lies_behind_the_table(D, e):
    """Rows that are zeroed by the vectors that cover them and the longer ones beside them, shares of CTAs that begin and end anywhere in
    a vector, one launch and three; memory behind the table stays as it was."""
    for T, V in ((3, 1), (32, 297), (33, 593), (300, 10007), (1000, 128256)):
        _check_bwd(T, D, V, e, e, masked=0.2)
        _check_bwd(T, D, V, e, e, masked=0.2, start=True)
        buffer = torch.full((V * D + 64,), 7.0, dtype=e, device="cuda")
        ids = _ids(T, V, D)
        dout = torch.randn(T, D, generator=torch.Generator().manual_seed(D)).to(e).cuda()
        binding.bdlm_embed_bwd(dout, torch.from_numpy(ids).int().cuda(), V, out=buffer[:V * D].view(V, D))
        assert (buffer[V * D:] == 7.0).all()
        absent = np.setdiff1d(np.arange(V), ids)
        assert (buffer[:V * D].view(V, D)[torch.from_numpy(absent).cuda()] == 0).all()


@pytest.mark.parametrize("D", [33, 40, 264])
@pytest.mark.parametrize("start", [None, True])
def test_runs_of_every_number_of_pieces(D, start):
    """Runs of 2 to 30 pieces of eight tokens, which begin and end anywhere in a piece: a warp adds the parts of the shorter ones, a
    whole CTA those of the longer ones."""
    rng = np.random.default_rng(D)
    lengths = rng.permutation(np.concatenate([np.arange(1, 250, 7), np.arange(8, 100, 8), [1] * 40]))
    ids = rng.permutation(np.repeat(np.arange(len(lengths)) * 3, lengths))
    assert len(ids) < 8192
    _check_bwd(len(ids), D, 3 * len(lengths), FP32, FP32, ids=ids, start=start)
    _check_bwd(len(ids), D, 3 * len(lengths), BF16, BF16, ids=ids, scale=0.25, start=start)


def test_rows_of_more_bytes_than_32_bits_count():
    """Rows of 2^31 bytes: those of tokens that do not occur are zeroed, by whole rows and not as short ones."""
    V, D = 4, 1 << 29
    dout = torch.zeros(1, D, device="cuda")
    dout[0, ::4099] = 3.0
    grad = torch.full((V, D), 7.0, device="cuda")
    binding.bdlm_embed_bwd(dout, torch.tensor([2], dtype=torch.int32, device="cuda"), V, out=grad)
    for v in range(V):
        assert torch.equal(grad[v], dout[0]) if v == 2 else not bool(grad[v].any())


# More than 8192 tokens are sorted by digits of nine bits or fewer, by one cluster; the calls above reach it with small tables alone.
@pytest.mark.parametrize("V", [1, 511, 512, 513, 262143, 262144, 1 << 20])
def test_sort_of_one_to_three_digits(V):
    _check_bwd(9000, 3, V, masked=0.2)


def test_sort_of_more_tokens_than_registers_hold():
    """More than 65536 tokens: a thread's pairs are read again in each of the three passes."""
    _check_bwd(70001, 3, 300000, masked=0.3)


def test_sort_of_four_digits():
    V, T = (1 << 27) + 5, 9000
    rng = np.random.default_rng(0)
    ids = np.concatenate([rng.integers(0, V, size=T - 1003), np.full(1000, V - 1), [0, V, -1]])
    rng.shuffle(ids)
    dout = torch.randn(T, 1, generator=torch.Generator().manual_seed(1)).cuda()
    got = binding.bdlm_embed_bwd(dout, torch.tensor(ids, dtype=torch.int32, device="cuda"), V)
    real = ids[(ids >= 0) & (ids < V)]
    uniq, place = np.unique(real, return_inverse=True)
    d64 = _f64(dout)[(ids >= 0) & (ids < V), 0]
    ref, size = np.zeros(len(uniq)), np.zeros(len(uniq))
    np.add.at(ref, place, d64)
    np.add.at(size, place, np.abs(d64))
    at = torch.from_numpy(uniq).cuda()
    # pieces of nine tokens; a run of 1000 in sixteen shares of its 112 pieces
    assert (np.abs(_f64(got[at, 0]) - ref) <= (9 + 112 / 16 + 16 + 1) * 2.0 ** -24 * size).all()
    got[at] = 0.0
    assert (got == 0).all()


@pytest.mark.parametrize("case", ["one", "alternating", "none", "beyond", "descending", "runs", "last_only", "mixed_pads"])
@pytest.mark.parametrize("start", [None, True])
def test_sort_patterns_of_ids(case, start):
    T, V = 9001, 1000
    t = np.arange(T)
    ids = {"one": np.full(T, 641), "alternating": t % 2 * 999, "none": np.full(T, -1), "beyond": np.where(t % 3 == 0, V, np.where(t % 3 == 1, 2 ** 31 - 1, -2 ** 31)),
           "descending": (T - 1 - t) % V, "runs": t // 40 % V, "last_only": np.where(t == T - 1, 5, -1), "mixed_pads": np.where(t % 2 == 0, -7, t % V)}[case]
    _check_bwd(T, 24, V, FP32, FP32, ids=ids, start=start)


@pytest.mark.parametrize("T", [9000, 70001])
def test_sort_under_capture_and_on_two_streams(T):
    D, V = 40, 5000
    dout = torch.randn(T, D, device="cuda").to(BF16)
    a = torch.tensor(_ids(T, V, 1, 0.4), dtype=torch.int32, device="cuda")
    b = torch.tensor(_ids(T, V, 2, 0.1), dtype=torch.int32, device="cuda")
    want = [binding.bdlm_embed_bwd(dout, i, V) for i in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, i in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                got.append(binding.bdlm_embed_bwd(dout, i, V))
    torch.cuda.synchronize()
    for k, t in enumerate(got):
        assert torch.equal(t, want[k % 2])
    ids = a.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grad = binding.bdlm_embed_bwd(dout, ids, V)
        added = binding.bdlm_embed_bwd(dout, ids, V, out=torch.zeros_like(grad), accumulate=True)
    for i, w in zip((a, b, a), (want[0], want[1], want[0])):
        ids.copy_(i)
        grad.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(grad, w) and torch.equal(added, w)
