"""CPU-only checks of the entry points for packed documents, the normalisation and the embedding: bad arguments are rejected
before a device is touched."""
import ctypes

import pytest
import torch

from paper_2609_19242_b200 import binding

OK, BAD16, BAD4 = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008), ctypes.c_void_p(0x1002)


def _norm(**kw):
    p = binding.make_norm_params(8000, 64, torch.bfloat16, torch.bfloat16, eps=1e-5)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw,code", [(dict(T=-1), -1), (dict(T=(1 << 30) + 1), -1), (dict(D=0), -1), (dict(dtype=3), -1), (dict(dtype=-1), -1),
                                     (dict(wdtype=1), -1), (dict(dtype=2, wdtype=0), -1), (dict(kind=2), -1), (dict(eps=-1.0), -1),
                                     (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(D=32769), -2)])
def test_norm_parameters(kw, code):
    L, p = binding.lib(), _norm(**kw)
    assert L.bdlm_norm_fwd(ctypes.byref(p), OK, None, OK, OK, OK, None, OK, OK, None) == code
    assert L.bdlm_norm_bwd(ctypes.byref(p), OK, OK, OK, OK, OK, None, OK, OK, OK, OK, 1 << 40, None) == code
    assert binding.bdlm_norm_workspace_bytes(p) == 0
    reserved = _norm()
    reserved.reserved[1] = 1
    assert L.bdlm_norm_fwd(ctypes.byref(reserved), OK, None, OK, OK, OK, None, OK, OK, None) == -1


def test_norm_pointers():
    L, p, rms = binding.lib(), _norm(), _norm(kind=1)
    fwd = lambda *a, p=p: L.bdlm_norm_fwd(ctypes.byref(p), *a, None)
    good = [OK, None, OK, OK, OK, None, OK, OK]
    for at, value in ((0, None), (4, None), (1, OK), (5, OK), (2, None), (0, BAD16), (2, BAD16), (3, BAD16), (4, BAD16), (6, BAD4), (7, BAD4)):
        a = list(good)
        a[at] = value    # (2, None): a bias without a weight; (1, OK): a residual without h; (5, OK): h without a residual
        assert fwd(*a) == -1, (at, value)
    assert fwd(*good, p=rms) == -1                    # the mean of a root-mean-square norm
    assert L.bdlm_norm_fwd(None, *good, None) == -1
    bwd = lambda *a, p=p, size=1 << 40: L.bdlm_norm_bwd(ctypes.byref(p), *a, size, None)
    good = [OK, OK, OK, OK, OK, OK, OK, OK, OK, OK]
    for at, value in ((0, None), (1, None), (2, None), (3, None), (4, None), (6, None), (9, None), (0, BAD16), (1, BAD16), (2, BAD16), (3, BAD4),
                      (4, BAD4), (5, BAD16), (6, BAD16), (7, BAD16), (8, BAD16), (9, BAD16)):
        a = list(good)
        a[at] = value
        assert bwd(*a) == -1, (at, value)
    assert bwd(*good, p=rms) == -1
    need = binding.bdlm_norm_workspace_bytes(p)
    assert need >= 2 * 64 * 4
    assert bwd(*good, size=need - 1) == -3


def test_norm_workspace_grows_to_a_bound():
    size = lambda T, D: binding.bdlm_norm_workspace_bytes(binding.make_norm_params(T, D, torch.bfloat16, torch.bfloat16))
    assert size(0, 64) == 0 and size(1, 4096) == 0 and size(5, 200) == 0   # a call of one CTA needs none
    assert size(1000, 4096) >= 2 * 4096 * 4
    assert size(1 << 30, 4096) == size(1 << 20, 4096) <= 2 * 148 * 4096 * 4
    assert all(size(T, 1001) <= 2 * 148 * 1001 * 4 for T in (5, 100, 10000))


def _embed(**kw):
    p = binding.make_embed_params(80, 64, 100, torch.bfloat16, torch.bfloat16)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw", [dict(T=-1), dict(T=(1 << 30) + 1), dict(D=0), dict(V=0), dict(V=(1 << 30) + 1), dict(table_dtype=3), dict(out_dtype=-1),
                                dict(out_dtype=2), dict(table_dtype=1), dict(scale=float("nan")), dict(scale=float("inf")), dict(accumulate=2),
                                dict(reserved=1)])
def test_embed_parameters(kw):
    L, p = binding.lib(), _embed(**kw)
    assert L.bdlm_embed_fwd(ctypes.byref(p), OK, OK, OK, None) == -1
    assert L.bdlm_embed_bwd(ctypes.byref(p), OK, OK, OK, OK, 1 << 40, None) == -1
    assert binding.bdlm_embed_workspace_bytes(p) == 0


def test_embed_pointers():
    L, p = binding.lib(), _embed()
    for a in ((None, OK, OK), (OK, None, OK), (OK, OK, None), (BAD16, OK, OK), (OK, BAD4, OK), (OK, OK, BAD16)):
        assert L.bdlm_embed_fwd(ctypes.byref(p), *a, None) == -1, a
    for a in ((None, OK, OK, OK), (OK, None, OK, OK), (OK, OK, None, OK), (OK, OK, OK, None), (BAD16, OK, OK, OK), (OK, BAD4, OK, OK),
              (OK, OK, BAD16, OK), (OK, OK, OK, BAD16)):
        assert L.bdlm_embed_bwd(ctypes.byref(p), *a, 1 << 40, None) == -1, a
    need = binding.bdlm_embed_workspace_bytes(p)
    assert need >= 2 * 80 * 8
    assert binding.bdlm_embed_workspace_bytes(_embed(T=32)) == 0   # a call of one launch needs none
    assert L.bdlm_embed_bwd(ctypes.byref(p), OK, OK, OK, OK, need - 1, None) == -3
    assert L.bdlm_embed_fwd(None, OK, OK, OK, None) == -1


def test_document_tables():
    L = binding.lib()
    for n, positions, cu, table in ((0, 8, OK, OK), (1, 0, OK, OK), (1, (1 << 30) + 1, OK, OK), (1, 8, None, OK), (1, 8, OK, None), (1, 8, BAD4, OK),
                                    (1, 8, OK, ctypes.c_void_p(0x1004))):
        assert L.bdlm_doc_table(cu, n, positions, table, None) == -1
    assert L.bdlm_doc_table_bytes(0) == 0 and L.bdlm_doc_table_bytes((1 << 30) + 1) == 0
    assert L.bdlm_doc_table_bytes(1000) == 4 * (2 * 1001 + 8 + 8 + 4)
    assert L.bdlm_doc_table_bytes(1 << 20) == 8 * ((1 << 20) + 1)
    p = binding.make_params(1, 256, 16, 4, 2, 64)
    g = binding.BdlmPackedGeometry()
    g.Lq_clean, g.n_blocks = 256, 8
    fwd = lambda d, g=g: L.bdlm_attn_fwd_docs(ctypes.byref(p), ctypes.byref(g), d and ctypes.byref(d), *([OK] * 10), None)
    bwd = lambda d, g=g: L.bdlm_attn_bwd_docs(ctypes.byref(p), ctypes.byref(g), d and ctypes.byref(d), *([OK] * 18), OK, 1 << 40, None)
    for call in (fwd, bwd):
        assert call(None) == -1
        for bad in (binding.BdlmDocs(None, 10, 0, 0), binding.BdlmDocs(0x1004, 10, 0, 0), binding.BdlmDocs(0x1000, -1, 0, 0),
                    binding.BdlmDocs(0x1000, 10, 1, 0), binding.BdlmDocs(0x1000, 10, 0, -1)):
            assert call(bad) == -1
        chunks = binding.BdlmPackedGeometry(256, 0, 8, 128, None, 0x1000, 0x1000)
        assert call(binding.BdlmDocs(0x1000, 10, 0, 0), chunks) == -2


def test_binding_refuses_tensors_that_are_not_on_the_device():
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    ids = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: binding.bdlm_norm_fwd(x), lambda: binding.bdlm_norm_bwd(x, x, None, None, torch.zeros(4)),
                 lambda: binding.bdlm_embed_fwd(x, ids), lambda: binding.bdlm_embed_bwd(x, ids, 9)):
        with pytest.raises(ValueError):
            call()


def test_document_starts_are_checked_on_the_host():
    for bad in ([0], [0, 5, 3], [-1, 4], [[0, 4]], torch.tensor([0.0, 4.0]), [0, 0]):
        with pytest.raises(ValueError):
            binding.bdlm_doc_table(bad)
    with pytest.raises(ValueError):
        binding.bdlm_doc_table([0, 100], 50)


def test_documents_that_cut_blocks_are_found():
    """Without block_prefix the blocks lie over the positions, and one that a document's border cuts would mix two documents."""
    buffer = torch.zeros(2 * 101, dtype=torch.int32)
    table = lambda *borders: binding.DocTable(buffer, 100, 100, 0, torch.tensor(borders))
    assert table(0, 32, 96).first_cut(32, 96) is None and table(0, 32, 96).first_cut(16, 96) is None
    assert table(0, 32, 50, 96).first_cut(32, 96) == 50
    assert table(10, 96).first_cut(32, 96) == 10       # positions of no document before the first
    assert table(0, 90).first_cut(32, 96) == 90        # and behind the last
    assert table(0, 90).first_cut(32, 64) is None      # no block lies there
    assert binding.DocTable(buffer, 100, 100, 0).first_cut(32, 96) is None   # borders not known


@pytest.mark.parametrize("D", [(1 << 30) + 1, 2 ** 31 - 1])
def test_embed_rows_too_long_to_count(D):
    L, p = binding.lib(), _embed(D=D, V=1)
    assert L.bdlm_embed_fwd(ctypes.byref(p), OK, OK, OK, None) == -1
    assert L.bdlm_embed_bwd(ctypes.byref(p), OK, OK, OK, OK, 1 << 60, None) == -1
    assert binding.bdlm_embed_workspace_bytes(p) == 0
    assert binding.bdlm_embed_workspace_bytes(_embed(D=1 << 30, V=1)) > 0


class _On:
    """A tensor as the binding sees it, on a device that need not be there."""

    def __init__(self, device, *shape, dtype=torch.bfloat16):
        self.index, self.shape, self.dtype, self.device, self.is_cuda = device, torch.Size(shape), dtype, f"cuda:{device}", True
        self.itemsize = dtype.itemsize

    def get_device(self):
        return self.index

    def numel(self):
        return self.shape.numel()

    @property
    def nbytes(self):
        return self.numel() * self.itemsize

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x1000


def test_workspaces_are_counted_in_bytes_and_stay_on_the_calls_device(monkeypatch):
    given = []

    class Library:
        def bdlm_norm_bwd(self, *a):
            given.append(a[10:12])
            return 0

        def bdlm_embed_bwd(self, *a):
            given.append(a[4:6])
            return 0
    monkeypatch.setattr(binding, "lib", Library)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    x, w, rstd, ids = _On(0, 100, 64), _On(0, 64), _On(0, 100, dtype=torch.float32), _On(0, 100, dtype=torch.int32)
    norm = lambda ws: binding.bdlm_norm_bwd(x, x, w, rstd, rstd, out=(x, w, None), workspace=ws)
    embed = lambda ws: binding.bdlm_embed_bwd(x, ids, 9, out=_On(0, 9, 64), workspace=ws)
    for call in (norm, embed):
        with pytest.raises(ValueError):
            call(_On(1, 1 << 20, dtype=torch.uint8))
        with pytest.raises(ValueError):
            call(_On(-1, 1 << 20, dtype=torch.uint8))
        call(_On(0, 1000, dtype=torch.float32))
        assert given.pop() == (0x1000, 4000) and not given
