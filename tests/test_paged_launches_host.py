"""Launch shapes and workspaces of paged attention with weights, with the launches recorded instead of made.  No GPU."""
import pytest

import paper_2510_24606_amd as dhsa
import test_launches_host

RECORDER = test_launches_host.RECORDER.replace("if (block.x == 256)", "if (0)")

ATTEND = """
import ctypes as C, sys
sys.modules["torch"] = None
C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
import paper_2510_24606_amd as dhsa
T, n_seq, dtype, pages, extra = map(int, sys.argv[2:])
p = dhsa.dhsa_paged(T=T, n_seq=n_seq, H_q=32, H_kv=8, D=128, dtype=dtype, page_size=64, n_pages=pages, max_pages=512)
at = 1 << 40                                          # an address that nothing reads
code = dhsa.lib().dhsa_paged_attend(C.byref(p), at, at, at, at, at, at, at, None, at, 1.0, at, dhsa.dhsa_paged_workspace_bytes(p) + extra, None)
assert code == 0, code
"""


@pytest.mark.parametrize("dtype,keys", [(0, 64), (1, 128)])
@pytest.mark.parametrize("T,n_seq", [(2048, 1), (255 + 512, 256), (64, 64), (100, 10)])
def test_weights_have_workgroups_for_scores_that_are_made_again(T, n_seq, dtype, keys, tmp_path, monkeypatch):
    """Whether scores are kept is settled by the lengths, on the device: a launch has a workgroup for every share that may have to
    be made again, or at least four for each of the 256 CUs."""
    monkeypatch.setattr(test_launches_host, "RECORDER", RECORDER)
    pages = 512
    x, y, z, threads = test_launches_host.launches(ATTEND, tmp_path, T, n_seq, dtype, pages, 0)[-1]
    assert (y, z, threads) == (1, 1, 256) and x >= min(1024, pages * 64 // keys * 8)


def sizes(T, n_seq, dtype):
    """Bytes with and without weights, and those of the references and sums that weights need in any case."""
    p = dhsa.dhsa_paged(T=T, n_seq=n_seq, H_q=32, H_kv=8, D=128, dtype=dtype, page_size=64, n_pages=9100, max_pages=512)
    return dhsa.dhsa_paged_workspace_bytes(p), dhsa.dhsa_paged_workspace_bytes(p, False), 8 * 32 * T + 255


@pytest.mark.parametrize("dtype", [0, 1])
def test_no_room_for_scores_that_nobody_keeps(dtype):
    """A single sequence of more than 32 rows a kv-head keeps none: neither type has room for them."""
    for T in (9, 100, 2048):
        full, bare, norm = sizes(T, 1, dtype)
        assert full <= bare + norm, T
    for T, n_seq in ((1, 1), (4, 1), (64, 64), (200, 64)):
        full, bare, norm = sizes(T, n_seq, dtype)
        assert full > bare + norm, (T, n_seq)


ATTEND_IN_ANOTHER = """
import ctypes as C, sys
sys.modules["torch"] = None
C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
import paper_2510_24606_amd as dhsa
n_seq, dtype = map(int, sys.argv[2:])
at = 1 << 40
sizes = [1, 2, 7, 8, 9, 16, 17, 33, 64, 65, 100, 255, 256, 257, 300, 511, 512, 513, 528, 529, 600, 2048, 4096, 70000]
probs = [dhsa.dhsa_paged(T=T, n_seq=n_seq, H_q=32, H_kv=8, D=128, dtype=dtype, page_size=64, n_pages=9100, max_pages=512) for T in sizes]
attend = lambda p, n: dhsa.lib().dhsa_paged_attend(C.byref(p), at, at, at, at, at, at, at, None, at, 1.0, at, n, None)
for i, p in enumerate(probs):
    for q in probs[i:]:
        assert attend(p, dhsa.dhsa_paged_workspace_bytes(q)) == 0, (p.T, q.T)
    assert attend(p, dhsa.dhsa_paged_workspace_bytes(p, False)) == (6 if p.T else 0), p.T      # (weights need their own part in any case)
"""


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n_seq", [1, 3, 64, 1000])
def test_a_workspace_of_more_tokens_serves_fewer(n_seq, dtype, tmp_path, monkeypatch):
    monkeypatch.setattr(test_launches_host, "RECORDER", RECORDER)
    assert test_launches_host.launches(ATTEND_IN_ANOTHER, tmp_path, n_seq, dtype)


LARGE = """
import ctypes as C, sys
sys.modules["torch"] = None
C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
import paper_2510_24606_amd as dhsa
T, heads = map(int, sys.argv[2:])
p = dhsa.dhsa_paged(T=T, n_seq=1, H_q=heads, H_kv=heads, D=64, dtype=1, page_size=64, n_pages=64, max_pages=64)
at = 1 << 40
assert dhsa.lib().dhsa_paged_attend(C.byref(p), at, at, at, at, at, at, at, None, None, 1.0, at, dhsa.dhsa_paged_workspace_bytes(p, False), None) == 0
"""


@pytest.mark.parametrize("T,heads", [(1 << 23, 64), (1 << 24, 64), ((1 << 24) + 77, 64), (1 << 25, 32)])
def test_grids_of_very_many_rows(T, heads, tmp_path, monkeypatch):
    """Rows beyond what 2^32 threads join (64 a workgroup of 256), tiles beyond what they attend."""
    recorder = test_launches_host.RECORDER.replace("if (block.x == 256)", "if (0)")
    recorder = recorder.replace('printf("\\n");', 'printf(" %d\\n", *(int *)args[1]);')          # 64 rows a workgroup marks a join
    monkeypatch.setattr(test_launches_host, "RECORDER", recorder)
    made = test_launches_host.launches(LARGE, tmp_path, T, heads)
    assert all(x * threads < 1 << 32 and (y, z) == (1, 1) for x, y, z, threads, _ in made)
    joined = sum(x for x, *_, per in made if per == 64)
    assert joined * 64 >= T * heads > joined * 64 - 64
