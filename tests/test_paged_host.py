"""Windows and paged caches: what is refused on the host, before any device call; sizes; the plain form itself."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paged_plain
import paper_2510_24606_amd as dhsa

NULL, SHAPE, BUDGET, DTYPE, WORKSPACE, ALIGN = 1, 2, 4, 5, 6, 9
P = 4096        # an address that is aligned and never followed


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(dhsa.LIB_PATH):
        from paper_2510_24606_amd import build
        build.build()
    return dhsa.lib()


def prob(**kw):
    f = dict(T=10, n_seq=3, H_q=8, H_kv=2, D=128, dtype=dhsa.DHSA_BF16, page_size=16, n_pages=40, max_pages=8)
    f.update(kw)
    return dhsa.dhsa_paged(**f)


def dense(**kw):
    f = dict(L=100, H_q=8, H_kv=2, D=128, dtype=dhsa.DHSA_BF16)
    f.update(kw)
    return dhsa.dhsa_problem(**f)


def attend(p, Q=P, K=P, V=P, table=P, q_start=P, kv_len=P, O=P, lse=None, weights=None, decay=1.0, ws=P, n=1 << 40):
    return dhsa.lib().dhsa_paged_attend(C.byref(p) if p is not None else None, Q, K, V, table, q_start, kv_len, O, lse, weights, decay, ws,
                                        n, None)


def append(p, Kn=P, Vn=P, K=P, V=P, table=P, q_start=P, kv_len=P):
    return dhsa.lib().dhsa_paged_append(C.byref(p), Kn, Vn, K, V, table, q_start, kv_len, None, None)


def evict(p, K=P, V=P, W=P, table=P, kv_len=P, keep=32, first=4, recent=8, out=P, kv_out=P, ws=P, n=1 << 40):
    return dhsa.lib().dhsa_paged_evict(C.byref(p), K, V, W, table, kv_len, keep, first, recent, out, kv_out, None, ws, n, None)


def window(p, w=5, s=0, Q=P, K=P, V=P, O=P):
    return dhsa.lib().dhsa_window_prefill(C.byref(p) if p is not None else None, w, s, Q, K, V, O, None)


BAD = [
    (dict(dtype=7), DTYPE), (dict(D=96), SHAPE), (dict(H_q=7), SHAPE), (dict(H_kv=0), SHAPE), (dict(H_q=65535, H_kv=1), SHAPE),
    (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE),
]


@pytest.mark.parametrize("kw,code", BAD + [
    (dict(T=-1), SHAPE), (dict(T=1 << 30), SHAPE), (dict(n_seq=-1), SHAPE), (dict(n_seq=65536), SHAPE), (dict(page_size=0), SHAPE),
    (dict(n_pages=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(page_size=1 << 16, max_pages=1 << 15), SHAPE),
    (dict(window=-1), SHAPE), (dict(sinks=-1), SHAPE),
    (dict(k_stride_s=64), SHAPE), (dict(v_stride_s=129), ALIGN), (dict(k_stride_h=-8), SHAPE), (dict(v_stride_p=100), SHAPE),
    (dict(q_stride_t=132), ALIGN), (dict(o_stride_h=4), ALIGN), (dict(o_stride_t=-128), SHAPE), (dict(k_stride_p=1 << 62), SHAPE),
    (dict(kn_stride_t=130), ALIGN), (dict(vn_stride_h=-8), SHAPE),
    (dict(n_pages=1 << 24, page_size=16), SHAPE),          # 2^24 pages of 2^3 KiB: a head's K spans 128 GiB
    (dict(v_stride_p=1 << 31), SHAPE),
])
def test_problems_that_are_refused(kw, code):
    p = prob(**kw)
    assert attend(p) == code and append(p) == code and evict(p) == code
    assert dhsa.dhsa_paged_workspace_bytes(p) == 0 and dhsa.dhsa_paged_evict_workspace_bytes(p, 32) == 0
    with pytest.raises(dhsa.DhsaError):
        dhsa.alloc_paged(p)


@pytest.mark.parametrize("kw,code", BAD + [
    (dict(L=0), SHAPE), (dict(L=1 << 31), SHAPE), (dict(k_stride_l=64), SHAPE), (dict(v_stride_l=132), ALIGN), (dict(o_stride_h=-8), SHAPE),
    (dict(L=1 << 28), SHAPE),                               # 2^28 rows of 256 bytes span 64 GiB
    (dict(L=1 << 27, dtype=dhsa.DHSA_F32), SHAPE),
    (dict(L=(1 << 24) + 1), SHAPE), (dict(L=1 << 20, k_stride_l=2056), SHAPE),      # a bf16 head of more than 4 GiB
])
def test_windows_that_are_refused(kw, code):
    assert window(dense(**kw)) == code


def test_arguments_that_are_refused():
    p = prob()
    assert attend(None) == NULL and window(None) == NULL
    for name in ("Q", "K", "V", "table", "q_start", "kv_len", "O", "ws"):
        assert attend(p, **{name: None}) == NULL, name
    for name in ("Q", "K", "V", "O", "ws"):
        assert attend(p, **{name: P + 8}) == ALIGN, name
    for name in ("table", "q_start", "kv_len", "lse", "weights"):
        assert attend(p, **{name: P + 2}) == ALIGN, name
    for decay in (-0.5, 1.5, float("nan")):
        assert attend(p, decay=decay) == SHAPE
    assert attend(p, n=dhsa.dhsa_paged_workspace_bytes(p, False) - 1) == WORKSPACE
    assert attend(p, weights=P, n=dhsa.dhsa_paged_workspace_bytes(p) - 1) == WORKSPACE
    for name in ("Kn", "Vn", "K", "V", "table", "q_start", "kv_len"):
        assert append(p, **{name: None}) == NULL, name
    for name in ("Kn", "Vn", "K", "V"):
        assert append(p, **{name: P + 8}) == ALIGN, name
    for name in ("K", "V", "W", "table", "kv_len", "out", "kv_out", "ws"):
        assert evict(p, **{name: None}) == NULL, name
    for name in ("K", "V", "ws"):
        assert evict(p, **{name: P + 8}) == ALIGN, name
    for name in ("table", "kv_len", "out", "kv_out", "W"):
        assert evict(p, **{name: P + 1}) == ALIGN, name
    for keep, first, recent in (((1 << 30) + 1, 0, 0), (0, 0, 0), (-1, 0, 0), (4, -1, 0), (4, 0, -1), (4, 3, 2), (1 << 30, (1 << 31) - 1, (1 << 31) - 1)):
        assert evict(p, keep=keep, first=first, recent=recent) == BUDGET, (keep, first, recent)
    assert evict(p, n=dhsa.dhsa_paged_evict_workspace_bytes(p, 32) - 1) == WORKSPACE
    assert dhsa.dhsa_paged_evict_workspace_bytes(p, 0) == 0
    for name in ("Q", "K", "V", "O"):
        assert window(dense(), **{name: None}) == NULL and window(dense(), **{name: P + 8}) == ALIGN
    assert window(dense(), w=0) == SHAPE and window(dense(), w=-3) == SHAPE and window(dense(), s=-1) == SHAPE


def test_nothing_to_do_needs_nothing():
    empty = prob(n_seq=0, T=0)
    assert attend(empty, Q=None, K=None, V=None, table=None, q_start=None, kv_len=None, O=None, ws=None, n=0) == 0
    assert append(empty, None, None, None, None, None, None, None) == 0
    assert evict(empty, None, None, None, None, None, out=None, kv_out=None, ws=None, n=0) == 0
    assert attend(prob(T=0), Q=None, O=None, ws=None, n=0) == 0 and append(prob(T=0), Kn=None, Vn=None) == 0


def test_sizes():
    a, b = prob(), prob(max_pages=1 << 16, n_pages=1 << 20)
    assert dhsa.dhsa_paged_workspace_bytes(a, False) == dhsa.dhsa_paged_workspace_bytes(b, False) > 0      # not of the lengths
    c = prob(max_pages=64)
    # kept scores: 10 tokens of 3 sequences, groups of four: 14 rows of a kv-head for each of the pool's slots
    assert 4 * 14 * 2 * 16 * 40 <= dhsa.dhsa_paged_workspace_bytes(c) - dhsa.dhsa_paged_workspace_bytes(c, False) <= 4 * 14 * 2 * 16 * 40 + 40000
    assert dhsa.dhsa_paged_workspace_bytes(b) <= dhsa.dhsa_paged_workspace_bytes(b, False) + (1 << 32) + 4096
    many = prob(T=3000)
    assert dhsa.dhsa_paged_workspace_bytes(many) - dhsa.dhsa_paged_workspace_bytes(many, False) <= 8 * 3000 * 8 + 256     # many tokens: none
    assert dhsa.dhsa_paged_evict_workspace_bytes(a, 100) >= 4 * 3 * 2 * 101
    # no more lists than there are slots
    assert dhsa.dhsa_paged_evict_workspace_bytes(a, 1 << 30) == dhsa.dhsa_paged_evict_workspace_bytes(a, 16 * 8)


def test_the_wrapper_compares_tensors_with_the_problem():
    """A tensor of another shape, type or device than the problem says is refused before it becomes an address (all of these
    are on the CPU: the device alone refuses them here)."""
    K, table = torch.zeros((5, 2, 16, 64)), torch.zeros((2, 3), dtype=torch.int32)
    p = dhsa.paged_problem(K, K, table, 4, 7)
    assert (p.n_pages, p.H_kv, p.page_size, p.D, p.n_seq, p.max_pages, p.H_q, p.T) == (5, 2, 16, 64, 2, 3, 4, 7)
    assert (p.k_stride_p, p.k_stride_h, p.k_stride_s) == (2 * 16 * 64, 16 * 64, 64) and p.dtype == dhsa.DHSA_F32
    by_slot = torch.zeros((5, 16, 2, 64)).permute(0, 2, 1, 3)
    p = dhsa.paged_problem(by_slot, K, table, 4, 7)
    assert (p.k_stride_p, p.k_stride_h, p.k_stride_s) == (2 * 16 * 64, 64, 128)


def test_page_of_a_slot():
    """slot / page_size as the kernels compute it, for sizes and slots at the ends of their ranges."""
    rng = np.random.default_rng(0)
    sizes = np.unique(np.concatenate([np.arange(1, 200), 2 ** np.arange(31), 2 ** np.arange(1, 31) - 1, 2 ** np.arange(30) + 1,
                                      rng.integers(1, 1 << 30, 500)]))
    for d in (int(x) for x in sizes):
        sh = 31 + math.ceil(math.log2(d)) if d > 1 else 31
        while (1 << (sh - 31)) < d:
            sh += 1
        mul = (1 << sh) // d + 1
        assert mul < 1 << 32
        x = np.unique(np.clip(np.concatenate([rng.integers(0, 1 << 31, 50), np.arange(5), (1 << 31) - 1 - np.arange(5),
                                              d * rng.integers(0, max(1, (1 << 31) // d), 20),
                                              d * rng.integers(1, max(2, (1 << 31) // d), 20) - 1]), 0, (1 << 31) - 1))
        assert all((int(v) * mul) >> sh == int(v) // d for v in x), d


def test_plain_form():
    """The plain form against torch's own softmax over an explicit mask."""
    g = torch.Generator().manual_seed(1)
    q, k, v = torch.randn(2, 9, 64, generator=g), torch.randn(30, 64, generator=g), torch.randn(30, 64, generator=g)
    pos = torch.arange(21, 30)
    for w, s in ((0, 0), (1, 0), (4, 2), (100, 3), (7, 50)):
        o, lse, got, *_ = paged_plain.attend(q, k, v, pos, w, s)
        mask = torch.tensor([[j <= p and (w == 0 or p - j < w or j < s) for j in range(30)] for p in range(21, 30)])
        x = (q.double() @ k.double().T / 8).masked_fill(~mask, -math.inf)
        prob_ = torch.softmax(x, -1)
        torch.testing.assert_close(o, prob_ @ v.double())
        torch.testing.assert_close(lse, torch.logsumexp(x, -1))
        torch.testing.assert_close(got, prob_.sum((0, 1)))
