"""The cache operators' sizes and refusals (no GPU), and the oracle against closed forms."""
import ctypes

import numpy as np
import pytest

from oracle import kv_oracle as ko
from paper_2603_05232_amd import binding

ONE, ODD, EIGHT = ctypes.c_void_p(16), ctypes.c_void_p(17), ctypes.c_void_p(8)      # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def test_sizes():
    size = binding.kv_page_bytes
    assert size(8, 64, 128, "bf16") == size(8, 64, 128, "fp16") == 2 * 64 * 8 * 128 * 2
    assert size(8, 64, 128, "fp8") == size(8, 64, 128, "i8") == 2 * 64 * 8 * 128 + 64 * 8 * 8          # codes and two scales a token and head
    assert size(1, 32, 1, "bf16") == 2 * 32 * 32 * 2 and size(1, 32, 80, "bf16") == 2 * 32 * 96 * 2    # a head completed to 32 values
    assert size(1, 32, 129, "bf16") == 2 * 32 * 192 * 2 and size(1, 32, 193, "bf16") == 2 * 32 * 256 * 2
    assert [size(*a) for a in ((0, 32, 64, "bf16"), (1025, 32, 64, "bf16"), (1, 48, 64, "bf16"), (1, 0, 64, "bf16"), (1, 4128, 64, "bf16"), (1, 32, 0, "bf16"), (1, 32, 257, "bf16"))] == [-1] * 7
    assert binding.load().kv_page_bytes(1, 32, 64, 9) == -1
    w = binding.kv_tables_workspace_bytes
    assert w(64, 2048) == 0 and w(64, 2049) > 0 and w(4097, 9000) == 0 and w(64, (1 << 20) + 1) == 0
    a = binding.kv_attention_workspace_bytes
    assert a(1, 32, 8, 128) > 0 and a(1, 33, 8, 128) == 0 and a(1, 4, 8, 128) == 0 and a(4097, 8, 8, 128) == 0 and a(1, 8, 8, 257) == 0 and a(0, 8, 8, 64) == 0
    assert a(64, 32, 8, 128) > a(1, 32, 8, 128)


def test_refusals_of_tables(lib):
    def t(lens=ONE, want=ONE, B=4, table=ONE, ldt=8, W=8, page=64, pool=ONE, P=100, left=ONE, N=16, nl=ONE, nf=ONE, slots=ONE, offsets=ONE, ws=None, wb=0):
        return lib.kv_tables(lens, want, B, table, ldt, W, page, pool, P, left, N, nl, nf, slots, offsets, ws, wb, None)
    assert t(B=-1) == t(B=4097) == t(N=-1) == t(N=(1 << 20) + 1) == t(page=16) == t(page=40) == t(page=0) == t(P=0) == t(P=1 << 25) == t(W=0) == t(W=1 << 25) == t(ldt=7) == 3
    assert t(lens=None) == t(want=None) == t(table=None) == t(pool=None) == t(left=None) == t(nl=None) == t(nf=None) == t(slots=None) == t(offsets=None) == 1
    assert t(lens=ODD) == t(table=ODD) == t(slots=ODD) == t(offsets=ODD) == 3
    assert t(N=9000) == 1 and t(N=9000, ws=ONE, wb=64) == 5 and t(N=9000, ws=EIGHT, wb=1 << 20) == 5 and t(ws=EIGHT, wb=1 << 20) == 5


def test_refusals_of_write_and_read(lib):
    def w(K=ONE, ldk=512, hk=64, V=ONE, ldv=512, hv=64, src=1, N=4, H=8, D=64, slots=ONE, pages=ONE, P=10, page=64, dtype=2):
        return lib.kv_write(K, ldk, hk, V, ldv, hv, src, N, H, D, slots, pages, P, page, dtype, None)
    assert w(src=2) == w(dtype=4) == w(dtype=-1) == 4
    assert w(N=-1) == w(N=(1 << 20) + 1) == w(H=0) == w(D=0) == w(D=257) == w(page=33) == w(P=0) == w(P=1 << 26) == w(ldk=-1) == w(hv=1 << 41) == 3
    assert w(K=None) == w(V=None) == w(slots=None) == w(pages=None) == 1 and w(N=0, K=None) == 0
    assert w(K=ODD) == w(V=ODD) == w(slots=ODD) == w(pages=EIGHT) == 3 and w(K=ctypes.c_void_p(18), src=0) == 3

    def r(pages=ONE, P=10, page=64, dtype=2, slots=ONE, N=4, H=8, D=64, out=1, K=ONE, ldk=512, hk=64, V=ONE, ldv=512, hv=64):
        return lib.kv_read(pages, P, page, dtype, slots, N, H, D, out, K, ldk, hk, V, ldv, hv, None)
    assert r(out=2) == r(dtype=4) == 4 and r(N=-1) == r(page=8) == r(P=0) == r(D=300) == r(hk=-1) == 3
    assert r(K=None) == r(V=None) == r(slots=None) == r(pages=None) == 1 and r(N=0) == 0 and r(pages=EIGHT) == r(V=ODD) == 3


def test_refusals_of_attention(lib):
    def a(Q=ONE, src=1, ldq=512, hq=64, pages=ONE, P=10, page=64, dtype=2, table=ONE, ldt=4, W=4, lens=ONE, B=2, Hq=8, H=4, D=64, scale=1.0, window=0, out=ONE, ldo=512, ho=64, ws=None, wb=0):
        return lib.kv_attention(Q, src, ldq, hq, pages, P, page, dtype, table, ldt, W, lens, B, Hq, H, D, scale, window, out, ldo, ho, ws, wb, None)
    assert a(src=2) == a(dtype=7) == 4
    assert a(B=-1) == a(B=4097) == a(Hq=9) == a(Hq=2) == a(Hq=2048, H=4) == a(H=0) == a(D=0) == a(D=257) == a(page=20) == a(P=0) == a(W=0) == a(ldt=3) == a(window=-1) == a(ldq=-1) == 3
    assert a(scale=float("nan")) == a(scale=float("inf")) == a(W=1 << 25, ldt=1 << 25) == 3
    assert a(Q=None) == a(pages=None) == a(table=None) == a(lens=None) == a(out=None) == a(wb=64) == 1 and a(B=0, Q=None) == 0
    assert a(Q=ODD) == a(out=ODD) == a(table=ODD) == a(lens=ODD) == a(pages=EIGHT) == 3 and a(ws=EIGHT, wb=1 << 20) == 5


def test_oracle_of_tables():
    table = np.array([[7, 9, -1, -1], [3, 4, 5, -1], [-1, -1, -1, -1]])
    #          grows within a page, shrinks by two pages, is new
    lens, left, slots, offsets, t, pool = ko.tables([40, 90, 0], [42, 5, 65], table, 32, [10, 11, 12, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0], 3, 70)
    assert lens == [42, 5, 65] and offsets == [0, 2, 2, 67]
    assert slots[:2] == [9 * 32 + 8, 9 * 32 + 9] and slots[67:] == [-1] * 3
    assert pool[3:5] == [4, 5] and t[2].tolist() == [5, 4, 12, -1] and left == 2                       # those given back lie on top
    assert slots[2:67] == list(range(160, 192)) + list(range(128, 160)) + [12 * 32]
    # too few pages: the first one that does not fit and those behind that need pages are left out
    lens, left, slots, offsets, t, pool = ko.tables([0, 0, 31], [33, 33, 32], np.full((3, 2), -1), 32, [1, 2, 3], 3, 100)
    assert lens == [33, 0, 32] and left == 1 and slots[33:66] == [-1] * 33 and offsets == [0, 33, 66, 67]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "i8", "fp8"])
def test_oracle_of_what_a_cache_holds(dtype):
    import torch
    x = torch.randn((50, 40), generator=torch.Generator().manual_seed(1)) * torch.logspace(-3, 3, 50)[:, None]
    got = ko.held(x.numpy(), dtype)
    if dtype in ("bf16", "fp16"):
        want = x.to(torch.bfloat16 if dtype == "bf16" else torch.float16).float().numpy()
    else:
        a = x.abs().amax(-1, keepdim=True)
        y = x * (torch.reciprocal(a) * ko.LARGEST[dtype])
        want = ((torch.round(y) if dtype == "i8" else y.to(torch.float8_e4m3fn).float()) * (a / torch.full_like(a, ko.LARGEST[dtype]))).numpy()
    assert np.array_equal(got, want)
    if dtype in ko.LARGEST:
        odd = ko.held(np.array([[0.0, 0.0], [np.inf, 1.0], [1.0, np.nan], [1e-38, 0.0]], np.float32), dtype)
        assert (odd[0] == 0).all() and np.isnan(odd[1:3]).all() and (odd[3] == 0).all()


def test_oracle_of_attention():
    rng = np.random.default_rng(3)
    q, v = rng.standard_normal((4, 8)), rng.standard_normal((6, 2, 8))
    seen = np.array([False, True, True, False, True, False])
    same = np.broadcast_to(rng.standard_normal((1, 2, 8)), (6, 2, 8))
    out = ko.attention(q, same, v, 0.3, seen)[0]
    assert np.allclose(out[:2], v[seen, 0].mean(0)) and np.allclose(out[2:], v[seen, 1].mean(0))        # equal scores: the mean; two heads to each of keys
    k = rng.standard_normal((6, 2, 8))
    assert np.allclose(ko.attention(q, 1e4 * k, v, 1.0, seen)[0][0], v[np.flatnonzero(seen)[(k[seen, 0] @ q[0]).argmax()], 0])
    assert (ko.attention(q, k, v, 1.0, np.zeros(6, bool))[0] == 0).all()
    d = 1e-6                                                                                            # its derivative along q
    f = lambda x: ko.attention(x, k, v, 0.5, seen)[0][0]  # noqa: E731
    s = 0.5 * k[seen, 0] @ q[0]
    p = np.exp(s - s.max()) / np.exp(s - s.max()).sum()
    e = np.zeros((4, 8))
    e[0, 2] = d
    want = 0.5 * ((p * k[seen, 0][:, 2]) @ v[seen, 0] - (p @ k[seen, 0][:, 2]) * (p @ v[seen, 0]))
    assert np.allclose((f(q + e) - f(q - e)) / (2 * d), want, atol=1e-7)


def test_every_call_of_a_cache_has_a_workspace_of_its_own(monkeypatch):
    """Calls that are under way at once, on streams or in captured graphs, share no memory."""
    import types

    import torch

    from paper_2603_05232_amd import kv_cache
    given = []
    monkeypatch.setattr(kv_cache, "binding", types.SimpleNamespace(kv_page_bytes=lambda *a: 64, kv_attention_workspace_bytes=lambda B, Hq, H, D: 1000,
                                                                   kv_attention=lambda *a, workspace=None, **kw: given.append(workspace)))
    cache = kv_cache.PagedCache("cpu", 3, 5, 2, 2, 16)
    assert cache.pool.tolist() == [4, 3, 2, 1, 0] and cache.left.tolist() == [5] and cache.lens.tolist() == [0, 0, 0]
    for _ in range(3):
        cache.attend(torch.zeros((3, 4, 16)))
    spans = [(w.data_ptr(), w.data_ptr() + w.numel()) for w in given]
    assert all(w.dtype == torch.uint8 and w.numel() >= 1000 for w in given) and all(a[1] <= b[0] or b[1] <= a[0] for i, a in enumerate(spans) for b in spans[:i])
    assert not any(w is v for w in given for v in vars(cache).values())


def test_scales_that_are_infinite_in_powers_of_two_are_refused(lib):
    """Scores are taken to the base 2: times 1.4427."""
    def a(scale):
        return lib.kv_attention(ONE, 1, 512, 64, ONE, 10, 64, 2, ONE, 4, 4, ONE, 2, 8, 4, 64, scale, 0, ONE, 512, 64, None, 0, None)
    assert a(3e38) == a(-3e38) == a(2.4e38) == 3
