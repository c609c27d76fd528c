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
