"""What the binding of the paged cache hands to the library, with a library that only writes down its arguments.  No GPU: the device
that tensors in host memory say they are on takes the place of the current one."""
import ctypes as C

import pytest
import torch

import paper_2510_24606_amd as dhsa


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(dhsa, "lib", lambda: r)
    monkeypatch.setattr(dhsa, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: torch.zeros(1).get_device())
    return r


class Elsewhere:
    """A tensor of another device."""

    def __init__(self, t):
        self.t = t

    def get_device(self):
        return 3

    def __getattr__(self, name):
        return getattr(self.t, name)


def tensors(n_seq=2, T=3, H_q=4, H_kv=2, D=64, page=16, n_pages=5, width=3):
    K = torch.zeros((n_pages, H_kv, page, D))
    table = torch.zeros((n_seq, width), dtype=torch.int32)
    t = dict(K=K, V=torch.zeros_like(K), table=table, Q=torch.zeros((H_q, T, D)), O=torch.zeros((H_q, T, D)),
             q_start=torch.zeros(n_seq + 1, dtype=torch.int32), kv_len=torch.zeros(n_seq, dtype=torch.int32), lse=torch.zeros((H_q, T)),
             weights=torch.zeros((n_pages, H_kv, page)), K_new=torch.zeros((H_kv, T, D)), V_new=torch.zeros((H_kv, T, D)),
             kv_out=torch.zeros(n_seq, dtype=torch.int32), idx=torch.zeros((n_seq, H_kv, 8), dtype=torch.int32),
             ws=torch.zeros(1000, dtype=torch.uint8))
    return t, dhsa.paged_problem(K, t["V"], table, H_q, T)


def attend(p, t):
    dhsa.dhsa_paged_attend(p, t["Q"], t["K"], t["V"], t["table"], t["q_start"], t["kv_len"], t["O"], t["ws"], lse=t["lse"], weights=t["weights"])


def append(p, t):
    dhsa.dhsa_paged_append(p, t["K_new"], t["V_new"], t["K"], t["V"], t["table"], t["q_start"], t["kv_len"], t["weights"])


def evict(p, t, keep=8, first=0, recent=0):
    dhsa.dhsa_paged_evict(p, t["K"], t["V"], t["weights"], t["table"], t["kv_len"], keep, first, recent, t["ws"], t["kv_out"], idx=t["idx"])


@pytest.mark.parametrize("call", [attend, evict])
def test_a_workspace_of_another_device_or_with_gaps_is_refused(call, recorder):
    t, p = tensors()
    call(p, t)
    assert recorder.calls[-1][1][-3:] == (t["ws"].data_ptr(), 1000, 0)
    for bad in (Elsewhere(t["ws"]), torch.zeros(1, dtype=torch.uint8).expand(1 << 20), t["ws"][::2]):
        with pytest.raises(ValueError, match="workspace"):
            call(p, dict(t, ws=bad))
    assert len(recorder.calls) == 1


def odd(t):
    """The same tensor with a stride of 3 wherever there is but one of something."""
    return t.as_strided(t.shape, [3 if n == 1 else x for n, x in zip(t.shape, t.stride())])


@pytest.mark.parametrize("kw", [dict(n_seq=1), dict(T=1), dict(n_pages=1, width=1), dict(page=1), dict(H_q=1, H_kv=1),
                                dict(n_seq=1, T=1, H_q=1, H_kv=1, page=1, n_pages=1, width=1)])
def test_strides_of_a_single_one_do_not_matter(kw, recorder):
    t, _ = tensors(**kw)
    t = {n: odd(x) for n, x in t.items()}
    p = dhsa.paged_problem(t["K"], t["V"], t["table"], t["Q"].shape[0], t["Q"].shape[1])
    for call in (attend, append, evict):
        call(p, t)
    assert len(recorder.calls) == 3
    L = t["K_new"].shape[1]
    dhsa.dhsa_window_prefill(dhsa.problem(t["Q"], t["K_new"], [0, L], L, V=t["V_new"]), t["Q"], t["K_new"], t["V_new"], t["O"], 5)
    for q in (t["Q"].expand(t["Q"].shape), t["Q"].transpose(0, 1).contiguous().transpose(0, 1)):
        attend(p, dict(t, Q=q))


def test_strides_that_matter_are_still_refused(recorder):
    t, p = tensors()
    for name, bad in (("table", torch.zeros((2, 9), dtype=torch.int32)[:, :3]), ("table", torch.zeros((3, 2), dtype=torch.int32).T),
                      ("lse", torch.zeros((3, 4)).T), ("weights", torch.zeros((5, 16, 2)).transpose(1, 2)), ("Q", t["Q"][:, :1].expand(4, 3, 64)),
                      ("K", t["K"][:, :1].expand(5, 2, 16, 64)), ("kv_len", torch.zeros(1, dtype=torch.int32).expand(2)),
                      ("O", torch.zeros((4, 64, 3)).transpose(1, 2))):
        with pytest.raises(ValueError, match=name):
            attend(p, dict(t, **{name: bad}))
    assert not recorder.calls


def test_the_library_does_not_look_at_strides_of_a_single_one():
    names = ["q_stride_t", "o_stride_t", "kn_stride_t", "vn_stride_t", "k_stride_p", "v_stride_p", "k_stride_s", "v_stride_s", "q_stride_h",
             "o_stride_h", "k_stride_h", "v_stride_h", "kn_stride_h", "vn_stride_h"]
    one = dict(T=1, n_seq=1, H_q=1, H_kv=1, D=64, dtype=dhsa.DHSA_BF16, page_size=1, n_pages=1, max_pages=1)
    two = dict(one, T=2, H_q=2, H_kv=2, page_size=2, n_pages=2)
    for name in names:
        for x in (3, -8, 1 << 62):
            assert dhsa.dhsa_paged_workspace_bytes(dhsa.dhsa_paged(**one, **{name: x})) > 0, name
            assert dhsa.dhsa_paged_workspace_bytes(dhsa.dhsa_paged(**two, **{name: x})) == 0, name
    for name in ("q_stride_h", "q_stride_l", "k_stride_h", "k_stride_l", "v_stride_h", "v_stride_l", "o_stride_h", "o_stride_l"):
        codes = [dhsa.lib().dhsa_window_prefill(C.byref(dhsa.dhsa_problem(L=n, H_q=n, H_kv=n, D=64, dtype=dhsa.DHSA_BF16, **{name: 3})), 5, 0,
                                                None, None, None, None, None) for n in (1, 2)]
        assert codes[0] == 1 and codes[1] in (2, 9), name           # DHSA_ERR_NULL: all else is right


def test_numbers_of_tokens_do_not_lose_their_high_bits(recorder):
    t, p = tensors()
    for keep, first, recent in (((1 << 32) + 8, 0, 0), (8, (1 << 32) + 1, 0), (8, 0, -(1 << 32)), (-(1 << 32) + 8, 0, 0)):
        dhsa.dhsa_paged_evict(p, t["K"], t["V"], t["weights"], t["table"], t["kv_len"], keep, first, recent, t["ws"], t["kv_out"])
        got = [C.c_int32(x).value for x in recorder.calls[-1][1][6:9]]
        code = C.CDLL(dhsa.LIB_PATH).dhsa_paged_evict(C.byref(p), None, None, None, None, None, *got, None, None, None, None, C.c_size_t(0), None)
        assert code == 4, got                            # DHSA_ERR_BUDGET


def test_a_budget_beyond_32_bits_has_no_workspace():
    t, p = tensors()
    assert dhsa.dhsa_paged_evict_workspace_bytes(p, 1 << 30) > 0
    for keep in ((1 << 32) + 8, 1 << 31, -(1 << 32) + 8):
        assert dhsa.dhsa_paged_evict_workspace_bytes(p, keep) == 0
